"""Appends, log probabilities and 4-bit numbers on the host side, without a GPU: refusals, and the plain forms that the GPU tests
compare with, against hand-worked values."""
import math

import pytest
import torch

import serve_more_reference as R
from paper_1603_06809_b200 import serve as S
from paper_1603_06809_b200.bcast import BCAST_ERR_INVAL, BCAST_OK, BcastError, _lib

BF = dict(dtype=torch.bfloat16)
INT = dict(dtype=torch.int32)


def append_args(**change):
    a = S.AppendArgs(dtype=0, batch=2, new_tokens=3, q_heads=4, kv_heads=2, dim=64, rot=64, eps=1e-6, own_cap=10)
    for f in ("q", "k", "v", "out", "own_k", "own_v"):
        getattr(a, f + "_stride")[:] = (3 * 4 * 64, 4 * 64, 64)
    for k, v in change.items():
        if isinstance(v, tuple):
            getattr(a, k)[:] = v
        else:
            setattr(a, k, v)
    return a


def logprobs_args(**change):
    a = S.LogprobsArgs(dtype=2, top=4, rows=3, vocab=100, logits_stride=100)
    for k, v in change.items():
        setattr(a, k, v)
    return a


def pack4_args(**change):
    a = S.Pack4Args(dtype=0, rows=3, k=64, values_stride=64, codes_stride=32)
    for k, v in change.items():
        setattr(a, k, v)
    return a


def linear4_args(**change):
    a = S.Linear4Args(dtype=0, tokens=3, k=64, n=5, x_stride=64, codes_stride=32, y_stride=5)
    for k, v in change.items():
        setattr(a, k, v)
    return a


MAKE = dict(append=append_args, logprobs=logprobs_args, pack4=pack4_args, unpack4=pack4_args, linear4=linear4_args)
BAD = [("append", c) for c in (dict(dtype=2), dict(batch=-1), dict(new_tokens=-1), dict(batch=65536), dict(batch=65535, new_tokens=65535), dict(q_heads=-1),
                               dict(q_heads=65536), dict(kv_heads=0), dict(kv_heads=1025), dict(batch=4096, new_tokens=4096, q_heads=200), dict(dim=0),
                               dict(dim=12), dict(dim=136), dict(rot=8), dict(rot=-16), dict(rot=80), dict(axes=-1), dict(axes=17), dict(eps=-1.0),
                               dict(eps=math.nan), dict(eps=math.inf), dict(own_cap=-1), dict(own_cap=1 << 31), dict(first=-1), dict(first=1 << 31),
                               dict(q_stride=(64, 64, 60)), dict(k_stride=(-8, 64, 64)), dict(v_stride=(1 << 39, 64, 64)), dict(out_stride=(64, 64, 0)),
                               dict(own_k_stride=(64, 56, 64)), dict(own_v_stride=(64, 64, 4)), dict(axes=1, positions_stride=(-1, 1)),
                               dict(page_table=16, page_size=0, num_pages=3), dict(page_table=16, page_size=4, num_pages=-1),
                               dict(page_table=16, page_size=4, num_pages=3, page_table_stride=2))] + \
      [("logprobs", c) for c in (dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 24), dict(vocab=0), dict(vocab=1 << 31), dict(top=-1),
                                 dict(top=33), dict(logits_stride=-1), dict(logits_stride=1 << 39))] + \
      [(op, c) for op in ("pack4", "unpack4") for c in (dict(dtype=3), dict(rows=-1), dict(rows=1 << 31), dict(k=0), dict(k=48), dict(k=1 << 25),
                                                        dict(values_stride=56), dict(values_stride=68), dict(codes_stride=16), dict(codes_stride=40))] + \
      [("linear4", c) for c in (dict(dtype=2), dict(tokens=-1), dict(tokens=(1 << 21) + 1), dict(k=0), dict(k=16), dict(k=80), dict(k=1 << 25), dict(n=0),
                                dict(n=1 << 25), dict(x_stride=32), dict(x_stride=66), dict(codes_stride=16), dict(codes_stride=33), dict(y_stride=4))]


@pytest.mark.parametrize("op,change", BAD)
def test_arguments_that_are_refused(op, change):
    assert getattr(_lib, f"bcast_serve_{op}")(MAKE[op](**change), None) == BCAST_ERR_INVAL


@pytest.mark.parametrize("change", [dict(dtype=2), dict(tokens=-1), dict(k=16), dict(n=0)])
def test_workspaces_that_are_refused(change):
    assert _lib.bcast_serve_linear4_workspace(linear4_args(**change)) == BCAST_ERR_INVAL


@pytest.mark.parametrize("op", sorted(MAKE))
def test_null_arguments(op):
    assert getattr(_lib, f"bcast_serve_{op}")(None, None) == BCAST_ERR_INVAL


@pytest.mark.parametrize("op,change", [("append", dict(batch=0)), ("append", dict(new_tokens=0)), ("logprobs", dict(rows=0)), ("pack4", dict(rows=0)),
                                       ("unpack4", dict(rows=0)), ("linear4", dict(tokens=0))])
def test_nothing_to_do_is_no_error(op, change):
    assert getattr(_lib, f"bcast_serve_{op}")(MAKE[op](**change), None) == BCAST_OK


def test_linear4_workspace():
    size = lambda **c: _lib.bcast_serve_linear4_workspace(linear4_args(**c))  # noqa: E731
    assert size(tokens=0) >= S.BCAST_SERVE_STATUS_BYTES
    for tokens in (1, 31, 64, 100, 129, 5000):
        for n in (1, 5000, 70000):
            # codes and scales of x, where it has more than 8 tokens; a tile has places for 32, 64, 128 or 256, of which the
            # last kind takes 224
            if tokens <= 8:
                assert size(tokens=tokens, n=n, k=1024) == S.BCAST_SERVE_STATUS_BYTES
                continue
            need = tokens * (1024 // 2 + 1024 // 32)
            assert need <= size(tokens=tokens, n=n, k=1024) - 256 <= need + 256 + (tokens // 7 + 256) * 32


def append_tensors():
    return dict(q=torch.zeros(2, 3, 4, 64, **BF), k=torch.zeros(2, 3, 2, 64, **BF), v=torch.zeros(2, 3, 2, 64, **BF), own_k=torch.zeros(2, 9, 2, 64, **BF),
                own_v=torch.zeros(2, 9, 2, 64, **BF), own_len=torch.zeros(2, **INT))


@pytest.mark.parametrize("change,word", [
    (dict(q=torch.zeros(2, 3, 4, 32, **BF)), "q: "), (dict(q=torch.zeros(2, 2, 4, 64, **BF)), "q: "), (dict(v=torch.zeros(2, 3, 1, 64, **BF)), "v: "),
    (dict(v=torch.zeros(2, 3, 2, 64, dtype=torch.float16)), "v: "), (dict(k=torch.zeros(3, 2, 64, **BF)), "dimensions"),
    (dict(own_k=torch.zeros(3, 9, 2, 64, **BF)), "own_k: "), (dict(own_v=torch.zeros(2, 8, 2, 64, **BF)), "own_v: "),
    (dict(own_len=torch.zeros(2, dtype=torch.int64)), "own_len: "), (dict(own_len=torch.zeros(4, **INT)[::2]), "own_len: "),
    (dict(new_len=torch.zeros(3, **INT)), "new_len: "), (dict(page_table=torch.zeros(2, dtype=torch.int64)), "page_table"),
    (dict(page_table=torch.zeros(3, 4, **INT)), "page_table: "), (dict(q_norm=torch.zeros(32, **BF)), "q_norm: "), (dict(k_norm=torch.zeros(64)), "k_norm: "),
    (dict(inv_freq=torch.zeros(32, dtype=torch.float64)), "inv_freq: "), (dict(inv_freq=torch.zeros(65)), "inv_freq"), (dict(inv_freq=torch.zeros(4, 8)), "inv_freq"),
    (dict(positions=torch.zeros(2, 3, **INT)), "go with inv_freq"), (dict(inv_freq=torch.zeros(32), axis=torch.zeros(32, **INT)), "goes with positions"),
    (dict(inv_freq=torch.zeros(32), positions=torch.zeros(2, 4, **INT)), "positions"), (dict(inv_freq=torch.zeros(32), positions=torch.zeros(2, 3, 17, **INT)), "positions"),
    (dict(inv_freq=torch.zeros(32), positions=torch.zeros(2, 3, 2)), "positions: "),
    (dict(inv_freq=torch.zeros(32), positions=torch.zeros(2, 3, 2, **INT), axis=torch.zeros(64, **INT)), "axis: "), ({}, "CUDA device")])
def test_append_refuses_by_name(change, word):
    t = {**append_tensors(), **change}
    with pytest.raises(BcastError) as e:
        S.bcast_serve_append(*[t.pop(x) for x in ("q", "k", "v", "own_k", "own_v", "own_len")], **t)
    assert e.value.code == BCAST_ERR_INVAL and word in str(e.value)


@pytest.mark.parametrize("args,more,word", [
    ((torch.zeros(2, 3, 4), torch.zeros(2, **INT)), {}, "dimensions"), ((torch.zeros(2, 4), torch.zeros(3, **INT)), {}, "tokens: "),
    ((torch.zeros(2, 4), torch.zeros(2, dtype=torch.int64)), {}, "tokens: "), ((torch.zeros(2, 4), torch.zeros(2, **INT)), dict(top=33), "top"),
    ((torch.zeros(2, 4), torch.zeros(2, **INT)), dict(top=-1), "top"), ((torch.zeros(2, 4).double(), torch.zeros(2, **INT)), {}, "Double"),
    ((torch.zeros(4, 2).t(), torch.zeros(2, **INT)), {}, "logits: "), ((torch.zeros(2, 4), torch.zeros(2, **INT)), {}, "CUDA device")])
def test_logprobs_refuses_by_name(args, more, word):
    with pytest.raises(BcastError) as e:
        S.bcast_serve_logprobs(*args, **more)
    assert e.value.code == BCAST_ERR_INVAL and word in str(e.value)


def test_4_bit_calls_refuse_by_name():
    codes, scales = torch.zeros(5, 32, dtype=torch.uint8), torch.zeros(1, 1, 32, 4, 4, dtype=torch.uint8)
    x = torch.zeros(2, 64, **BF)
    for call, word in ((lambda: S.bcast_serve_pack4(x[0]), "dimensions"), (lambda: S.bcast_serve_pack4(x.double()), "Double"),
                       (lambda: S.bcast_serve_pack4(x), "CUDA device"), (lambda: S.bcast_serve_unpack4(codes.int(), scales), "codes: "),
                       (lambda: S.bcast_serve_unpack4(codes, scales[:, :, :31]), "scales: "), (lambda: S.bcast_serve_unpack4(codes, scales), "CUDA device"),
                       (lambda: S.bcast_serve_linear4(x, codes[:, :16], scales), "codes: "), (lambda: S.bcast_serve_linear4(x, codes, scales[0]), "scales: "),
                       (lambda: S.bcast_serve_linear4(x, codes, scales, bias=torch.zeros(6, **BF)), "bias: "),
                       (lambda: S.bcast_serve_linear4(x.float(), codes, scales), "Float"), (lambda: S.bcast_serve_linear4(x, codes, scales), "CUDA device")):
        with pytest.raises(BcastError) as e:
            call()
        assert e.value.code == BCAST_ERR_INVAL and word in str(e.value)


# ---- the plain forms
def test_reference_append():
    k = torch.tensor([3.0, 4.0] * 8, dtype=torch.float16).reshape(1, 1, 1, 16)
    own = torch.full((1, 4, 1, 16), 9.0, dtype=torch.float16)
    inv = torch.zeros(8)
    inv[0] = math.pi / 2
    r = R.append(k, k, k, own, own, torch.tensor([2]), inv_freq=inv, interleaved=True, k_norm=torch.ones(16), eps=0.0)
    # mean of squares 12.5; place 1, so the first pair turns by a quarter
    root = math.sqrt(12.5)
    assert torch.allclose(r["own_k"][0][0, 1, 0, :4], torch.tensor([-4.0, 3.0, 3.0, 4.0]).double() / root, atol=1e-6)
    assert torch.allclose(r["q"][0][0, 0, 0, :4], torch.tensor([-4.0, 3.0, 3.0, 4.0]).double(), atol=1e-6)
    assert torch.equal(r["own_v"][0][0, 1, 0], k[0, 0, 0].double()) and bool((r["own_k"][0][0, [0, 2, 3]] == 9).all())
    r = R.append(None, k, k, own, own, torch.tensor([0]))
    assert r["q"] is None and bool((r["own_k"][0] == 9).all())


def test_reference_logprobs():
    l = torch.log(torch.tensor([[0.5, 0.25, 0.25, 0.0], [0.25, 0.25, 0.25, 0.25]]))
    (lp, _), (h, _), ids, (best, _) = R.logprobs(l, torch.tensor([1, 7]), 4)
    assert abs(float(lp[0]) - math.log(0.25)) < 1e-6 and lp[1] == -math.inf
    assert abs(float(h[0]) - 1.5 * math.log(2)) < 1e-6 and abs(float(h[1]) - math.log(4)) < 1e-6
    assert ids.tolist() == [[0, 1, 2, -1], [0, 1, 2, 3]] and best[0, 3] == -math.inf


def test_reference_pack():
    x = torch.zeros(1, 64)
    x[0, :10] = torch.tensor([6.0, 5.0, -5.0, 2.5, 3.5, 0.25, 0.75, 7.9, -0.3, 1.0])      # largest exponent 2: unit 1
    x[0, 32] = 2.0 ** -127                                                                 # unit 2^-127
    codes, scales = R.pack(x)
    assert scales.tolist() == [[127, 0]]
    assert codes[0, :10].tolist() == [7, 6, 14, 4, 6, 0, 2, 7, 9, 2] and int(codes[0, 32]) == 2
    v = R.values(codes, scales)
    assert v[0, :10].tolist() == [6, 4, -4, 2, 4, 0, 1, 6, -0.5, 1] and float(v[0, 32]) == 2.0 ** -127
    assert R.bytes_of(codes)[0, 0] == 7 + 16 * 6
    x[0, 40] = math.inf
    assert R.pack(x)[1].tolist() == [[127, 255]]
    t = R.tiled(torch.arange(130 * 5).reshape(130, 5).to(torch.uint8))
    assert t.shape == (2, 2, 32, 4, 4) and int(t[1, 1, 1, 0, 0]) == (129 * 5 + 4) % 256 and int(t[0, 0, 3, 2, 1]) == (67 * 5 + 1) % 256
