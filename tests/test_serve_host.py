"""The serving operators' host side without a GPU: symbols, argument checks, workspace sizes."""
import ctypes
import os
import re

import pytest
import torch

import serve_reference as R
from helpers import ROOT
from paper_1603_06809_b200 import serve as S
from paper_1603_06809_b200.bcast import BCAST_ERR_INVAL, BCAST_OK, BcastError, _lib


def test_symbols_match_the_header():
    with open(os.path.join(ROOT, "include", "bcast_serve.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    declared = set(re.findall(r"\b(bcast_serve_\w+)\s*\(", text))
    assert declared == set(S.SYMBOLS)
    for name in S.SYMBOLS:
        assert getattr(_lib, name)


def linear_args(**change):
    a = S.LinearArgs(dtype=0, num_adapters=2, rank=16, tokens=5, k=64, n=32, x_stride=64, weight_stride=64, y_stride=32)
    a.lora_a_stride[:] = (16 * 64, 64)
    a.lora_b_stride[:] = (32 * 16, 16)
    for k, v in change.items():
        setattr(a, k, v)
    return a


def attn_args(**change):
    a = S.AttnArgs(dtype=0, batch=2, new_tokens=1, q_heads=4, kv_heads=2, dim=64, page_size=0, scale=1.0, prefix_len=10, own_cap=0)
    for k, v in change.items():
        setattr(a, k, v)
    return a


def verify_args(**change):
    a = S.VerifyArgs(dtype=2, batch=2, drafts=3, vocab=100)
    for k, v in change.items():
        setattr(a, k, v)
    return a


MAKE = {"linear": linear_args, "attn": attn_args, "verify": verify_args}
BAD = [("linear", c) for c in (dict(dtype=2), dict(dtype=-1), dict(k=0), dict(k=60), dict(n=0), dict(tokens=-1), dict(rank=12), dict(rank=0), dict(rank=136),
                               dict(num_adapters=-1), dict(k=1 << 40), dict(tokens=1 << 40), dict(tokens=(1 << 21) + 1), dict(n=1 << 25), dict(num_adapters=65537))] + \
      [("attn", c) for c in (dict(dtype=2), dict(dim=0), dict(dim=12), dict(dim=136), dict(q_heads=3), dict(q_heads=0), dict(kv_heads=0), dict(batch=-1),
                             dict(new_tokens=-1), dict(prefix_len=-1), dict(own_cap=-1), dict(prefix_len=1 << 40), dict(batch=65535, new_tokens=65535))] + \
      [("verify", c) for c in (dict(dtype=3), dict(drafts=-1), dict(drafts=64), dict(vocab=0), dict(vocab=1 << 31), dict(batch=-1), dict(batch=1 << 20))]


@pytest.mark.parametrize("op,change", BAD)
def test_shapes_that_are_refused(op, change):
    a = MAKE[op](**change)
    assert getattr(_lib, f"bcast_serve_{op}")(a, None) == BCAST_ERR_INVAL
    assert getattr(_lib, f"bcast_serve_{op}_workspace")(a) == BCAST_ERR_INVAL


@pytest.mark.parametrize("op", ["linear", "attn", "verify"])
def test_null_arguments(op):
    assert getattr(_lib, f"bcast_serve_{op}")(None, None) == BCAST_ERR_INVAL
    assert getattr(_lib, f"bcast_serve_{op}_workspace")(None) == BCAST_ERR_INVAL


@pytest.mark.parametrize("op,change", [("linear", dict(tokens=0)), ("attn", dict(batch=0)), ("attn", dict(new_tokens=0)), ("verify", dict(batch=0))])
def test_nothing_to_do_is_no_error(op, change):
    assert getattr(_lib, f"bcast_serve_{op}")(MAKE[op](**change), None) == BCAST_OK


@pytest.mark.parametrize("op", ["linear", "attn", "verify"])
def test_workspace_holds_the_status_word_and_grows_with_the_work(op):
    size = getattr(_lib, f"bcast_serve_{op}_workspace")
    small = size(MAKE[op]())
    assert small >= S.BCAST_SERVE_STATUS_BYTES
    more = dict(linear=dict(tokens=4096), attn=dict(batch=512), verify=dict(batch=512))[op]
    assert size(MAKE[op](**more)) >= small


@pytest.mark.parametrize("change", [dict(x_stride=60), dict(x_stride=68), dict(y_stride=31), dict(weight_stride=8)])
def test_strides_that_are_refused(change):
    assert _lib.bcast_serve_linear(linear_args(**change), None) == BCAST_ERR_INVAL


def test_tensors_on_the_host_are_refused():
    x, w = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(8, 64, dtype=torch.bfloat16)
    with pytest.raises(BcastError) as e:
        S.bcast_serve_linear(x, w)
    assert e.value.code == BCAST_ERR_INVAL
    with pytest.raises(BcastError):
        S.bcast_serve_verify(torch.zeros(1, 1, 4), torch.zeros(1, 0, 4), torch.zeros(1, 0, dtype=torch.int32), torch.zeros(1, 0), torch.ones(1, 4), torch.ones(1))


def test_tensors_that_do_not_fit_together_are_refused_by_name():
    bf = dict(dtype=torch.bfloat16)
    x, w = torch.zeros(2, 64, **bf), torch.zeros(8, 64, **bf)
    a, b, ad, sc = torch.zeros(3, 8, 64, **bf), torch.zeros(3, 8, 8, **bf), torch.zeros(2, dtype=torch.int32), torch.ones(3)
    good = dict(lora_a=a, lora_b=b, adapter=ad, scale=sc)
    for change, word in ((dict(bias=torch.zeros(9, **bf)), "bias"), (dict(lora_b=None), "go together"), (dict(adapter=ad.long()), "adapter"),
                         (dict(scale=sc.double()), "scale"), (dict(lora_a=a[0]), "three dimensions"), (dict(lora_b=b[:, :7]), "lora_b")):
        with pytest.raises(BcastError) as e:
            S.bcast_serve_linear(x, w, **{**good, **change})
        assert e.value.code == BCAST_ERR_INVAL and word in str(e.value)
    with pytest.raises(BcastError) as e:
        S.bcast_serve_linear(x.t().contiguous().t(), w)
    assert "x: (2, 64) BFloat16 on cpu with strides (1, 2)" in str(e.value)
    q, p, o, n = torch.zeros(2, 1, 4, 64, **bf), torch.zeros(5, 2, 64, **bf), torch.zeros(2, 7, 2, 64, **bf), torch.zeros(2, dtype=torch.int32)
    for args, word in (((q, p, p[:4], o, o, n), "prefix_v"), ((q, p, p, o, o[:, :6], n), "own_v"), ((q, p, p, o, o, n.long()), "own_len"),
                       ((q[0], p, p, o, o, n), "dimensions"), ((q, p.half(), p, o, o, n), "prefix_k")):
        with pytest.raises(BcastError) as e:
            S.bcast_serve_attn(*args)
        assert word in str(e.value)


def test_strides_of_dimensions_with_one_entry():
    t = torch.zeros(1, 1, 4, 64).as_strided((1, 1, 4, 64), (3, 5, 64, 1))
    assert S._strides(t, 3) == (256, 256, 64)
    t = torch.zeros(6, 1, 64).as_strided((6, 1, 64), (64, 7, 1))
    assert S._strides(t, 2) == (64, 64)


# ---- the plain forms that the GPU tests compare with, against hand-worked values
def test_reference_linear():
    x = torch.tensor([[1.0, 2.0], [3.0, 4.0]], dtype=torch.float16)
    w = torch.tensor([[1.0, 0.0], [0.0, 1.0], [1.0, 1.0]], dtype=torch.float16)
    a = torch.tensor([[[1.0, 1.0]]], dtype=torch.float16)
    b = torch.tensor([[[1.0], [2.0], [3.0]]], dtype=torch.float16)
    y, _ = R.linear(x, w, None, a, b, torch.tensor([0, -1]), torch.tensor([2.0]))
    assert y.tolist() == [[1 + 6, 2 + 12, 3 + 18], [3, 4, 7]]


def test_reference_attn():
    q = torch.zeros(1, 2, 1, 8, dtype=torch.float16)
    v = torch.arange(1, 4, dtype=torch.float16).reshape(3, 1, 1).expand(3, 1, 8)
    own = torch.tensor([7.0, 9.0], dtype=torch.float16).reshape(1, 2, 1, 1).expand(1, 2, 1, 8)
    out, _, lse, _ = R.attn(q, v * 0, v, own * 0, own, torch.tensor([2]))
    assert out[0, 0, 0, 0] == (1 + 2 + 3 + 7) / 4 and abs(float(out[0, 1, 0, 0]) - 22 / 5) < 1e-12
    assert abs(float(lse[0, 1, 0]) - float(torch.log(torch.tensor(5.0, dtype=torch.float64)))) < 1e-12


def test_reference_verify():
    z = torch.log(torch.tensor([[[0.5, 0.25, 0.25], [0.1, 0.8, 0.1]]]))
    q = torch.tensor([[[0.9, 0.05, 0.05]]])
    one, e = torch.ones(1), torch.tensor([[1.0, 0.4, 0.5]])
    assert R.verify(z, q, torch.tensor([[0]]), torch.tensor([[0.5]]), e, one)[1].tolist() == [[0, 1]]
    assert R.verify(z, q, torch.tensor([[0]]), torch.tensor([[0.6]]), e, one)[1].tolist() == [[1, -1]]
