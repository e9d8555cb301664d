"""Cache appends, log probabilities and microscaled 4-bit numbers on the GPU against plain 64-bit forms, through the public
binding."""
import math
import os
import subprocess
import sys

import pytest
import torch

import serve_more_reference as R
from helpers import ROOT
from paper_1603_06809_b200 import serve as S
from paper_1603_06809_b200.bcast import BCAST_ERR_CAPACITY, BCAST_ERR_INVAL, BCAST_ERR_TIMEOUT, BcastError
from test_serve_gpu import DEV, TYPES, gen, inside, on_gpu, rand

pytestmark = pytest.mark.gpu


def close(got, want, bound, what):
    """As `inside`, with infinities and NaN at their places."""
    got = got.double().cpu()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN at other places"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), f"{what}: infinities at other places"
    over = (got - want).abs()[fine] - bound[fine]
    assert bool((over <= 0).all()), f"{what}: bound passed by {float(over.max())}"


# ------------------------------------------------------------------------------------------ append
def append_case(seed, B, n, HQ, H, D, dtype, *, rot=None, page=16, cap=40, norm=False, axes=0, interleaved=False, lengths=None, new=None, first=0,
                fused=True):
    g, dt = gen(seed), TYPES[dtype]
    rot = D // 16 * 16 if rot is None else rot
    if fused:
        q, k, v = rand(g, B, n, HQ + 2 * H, D, dtype=dt).split((HQ, H, H), dim=2)
    else:
        q, k, v = (rand(g, B, n, h, D, dtype=dt) for h in (HQ, H, H))
    c = dict(q=q if HQ else None, k=k, v=v)
    if page:
        each = -(-cap // page)
        c["page_table"] = torch.randperm(B * each, generator=g).to(torch.int32).reshape(B, each)
        shape = (B * each, page, H, D)
    else:
        shape = (B, cap, H, D)
    c.update(own_k=rand(g, *shape, dtype=dt), own_v=rand(g, *shape, dtype=dt))
    c["own_len"] = torch.tensor(lengths, dtype=torch.int32) if lengths else torch.randint(min(n, cap), cap + 1, (B,), generator=g, dtype=torch.int32)
    if new is not None:
        c["new_len"] = torch.tensor(new, dtype=torch.int32)
    if rot:
        c["inv_freq"] = (10000.0 ** -(torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)).float()
        if axes:
            c["positions"] = torch.randint(0, 5000, (B, n, axes), generator=g, dtype=torch.int32)
            c["axis"] = (torch.arange(rot // 2) % axes).to(torch.int32)
    if norm:
        c.update(q_norm=rand(g, D, dtype=dt) + 1, k_norm=rand(g, D, dtype=dt))
    c.update(first=first, interleaved=interleaved)
    return c


def check_append(c, **more):
    want = R.append(**c)
    d = {k: on_gpu(v) if torch.is_tensor(v) else v for k, v in c.items()}
    args = [d.pop(x) for x in ("q", "k", "v", "own_k", "own_v", "own_len")]
    out = S.bcast_serve_append(*args, **d, **more)
    torch.cuda.synchronize()
    if c["q"] is None:
        assert out is None
    else:
        close(out, *want["q"], "q")
    close(args[3], *want["own_k"], "own_k")
    close(args[4], *want["own_v"], "own_v")
    return out, args[3], args[4]


@pytest.mark.parametrize("D", [8, 16, 24, 32, 40, 48, 64, 72, 80, 96, 112, 120, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("norm,interleaved", [(False, False), (True, False), (True, True)])
def test_append_head_sizes(D, dtype, norm, interleaved):
    check_append(append_case(D, 3, 2, 5, 2, D, dtype, norm=norm, interleaved=interleaved))


@pytest.mark.parametrize("rot", [0, 16, 32, 48, 64, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_append_partial_rotation(rot, interleaved, norm):
    check_append(append_case(rot, 2, 3, 4, 4, 128, "bf16", rot=rot, interleaved=interleaved, norm=norm))


@pytest.mark.parametrize("HQ,H", [(0, 1), (0, 5), (1, 1), (3, 1), (8, 8), (17, 17), (64, 8), (70, 7)])
@pytest.mark.parametrize("B,n", [(1, 1), (7, 3), (120, 1)])
def test_append_heads(HQ, H, B, n):
    check_append(append_case(HQ + H, B, n, HQ, H, 64, "fp16", norm=True))


@pytest.mark.parametrize("page,cap", [(0, 40), (1, 7), (3, 11), (16, 40), (64, 64), (100, 300)])
@pytest.mark.parametrize("n", [1, 6])
def test_append_pages(page, cap, n):
    check_append(append_case(page, 5, n, 4, 2, 64, "bf16", page=page, cap=cap))


@pytest.mark.parametrize("axes", [1, 2, 3, 16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_axes(axes, interleaved):
    c = append_case(axes, 3, 4, 4, 2, 96, "bf16", axes=axes, interleaved=interleaved)
    check_append(c)
    c["axis"][3], c["axis"][5] = -1, axes                     # taken as axis 0
    check_append(c)
    del c["axis"]
    check_append(c)
    c["positions"] = c["positions"][:, :, 0]
    check_append(c)
    c["positions"] = torch.tensor([[2 ** 31 - 1], [-2 ** 31], [12345678]], dtype=torch.int32).expand(3, 4)
    check_append(c)


@pytest.mark.parametrize("first", [0, 1, 131072, 10 ** 6, 2 ** 31 - 1])
def test_append_far_positions(first):
    check_append(append_case(5, 2, 3, 3, 1, 128, "fp16", first=first, norm=True))


def test_append_lengths_at_their_ends():
    # empty, shorter than the new tokens, full, above the capacity, negative
    for page in (0, 8):
        c = append_case(6, 9, 4, 3, 2, 64, "bf16", page=page, cap=24, lengths=[0, 1, 4, 5, 24, 25, 28, 1000, -7])
        out, _, _ = check_append(c)
        assert not bool(out[0].any()) and not bool(out[1, :3].any()) and bool(out[7].any())


def test_append_padded_batches():
    for page in (0, 8):
        c = append_case(7, 8, 5, 3, 2, 64, "fp16", page=page, cap=24, lengths=[20] * 4 + [3, 0, 24, 5], new=[0, 1, 4, 5, 2, 0, 9, -3], norm=True)
        check_append(c)


def test_append_pages_that_are_not_there():
    c = append_case(8, 4, 3, 3, 2, 64, "bf16", page=4, cap=24, lengths=[3, 9, 14, 24])
    c["page_table"][1, 2] = -1
    c["page_table"][2, 2] = 10 ** 6
    c["page_table"][3] = -2 ** 31
    check_append(c)
    c = append_case(9, 4, 3, 3, 2, 64, "bf16", page=4, cap=24)
    c["own_k"], c["own_v"] = c["own_k"][:0], c["own_v"][:0]   # no pages at all
    check_append(c)
    c["page_table"] = c["page_table"][:, :0]
    check_append(c)


def test_append_nothing():
    for B, n in ((0, 3), (3, 0)):
        out, _, _ = check_append(append_case(10, B, n, 2, 1, 32, "bf16", lengths=[5] * B if B else None))
        assert out.shape == (B, n, 2, 32)


def test_append_strides():
    c = append_case(11, 3, 4, 4, 2, 64, "bf16", fused=False)
    c["q"] = c["q"].transpose(1, 2).contiguous().transpose(1, 2)                     # heads before tokens
    c["k"] = torch.cat([c["k"], c["k"]], dim=-1)[..., 64:]
    c["v"] = c["v"][:1].expand(3, 4, 2, 64)
    c["own_k"] = torch.cat([c["own_k"], c["own_k"]], dim=2)[:, :, 1:3]
    c["own_v"] = c["own_v"].transpose(1, 2).contiguous().transpose(1, 2)
    c["page_table"] = torch.cat([c["page_table"], c["page_table"]], dim=1)[:, :c["page_table"].shape[1]]
    out = torch.empty(3, 4, 4, 128, dtype=torch.bfloat16, device=DEV)[..., 32:96]
    got = check_append(c, out=out)[0]
    assert got.data_ptr() == out.data_ptr()


def test_append_copies_what_is_not_turned_bit_for_bit():
    c = append_case(12, 2, 2, 3, 2, 64, "bf16", rot=0)
    bits = torch.randint(-2 ** 15, 2 ** 15, (2, 2, 7, 64), generator=gen(13)).to(torch.int16).view(torch.bfloat16)      # NaN among them
    c["q"], c["k"], c["v"] = bits.split((3, 2, 2), dim=2)
    d = {k: on_gpu(v) if torch.is_tensor(v) else v for k, v in c.items()}
    out = S.bcast_serve_append(d["q"], d["k"], d["v"], d["own_k"], d["own_v"], d["own_len"], page_table=d["page_table"])
    assert torch.equal(out.cpu().view(torch.int16), c["q"].view(torch.int16))
    for b in range(2):
        for i in range(2):
            slot = int(c["own_len"][b]) - 2 + i
            at = int(c["page_table"][b, slot // 16]), slot % 16
            assert torch.equal(d["own_k"][at].cpu().view(torch.int16), c["k"][b, i].view(torch.int16))
            assert torch.equal(d["own_v"][at].cpu().view(torch.int16), c["v"][b, i].view(torch.int16))


def test_append_in_place():
    c = append_case(14, 40, 3, 8, 2, 128, "bf16", norm=True)
    want, _, _ = check_append(c)
    d = {k: on_gpu(v) if torch.is_tensor(v) else v for k, v in c.items()}
    args = [d.pop(x) for x in ("q", "k", "v", "own_k", "own_v", "own_len")]
    got = S.bcast_serve_append(*args, **d, out=args[0])
    assert got.data_ptr() == args[0].data_ptr() and torch.equal(got, want)


def test_append_zero_heads_and_large_values():
    c = append_case(15, 2, 2, 2, 1, 64, "bf16", norm=True)
    c["q"][0], c["k"][1] = 0.0, 0.0                           # the norm of nothing: eps alone
    c["q"][1] *= 1e15
    check_append(c)
    c = append_case(16, 2, 2, 2, 1, 64, "fp16")
    c["q"][:] = 60000.0
    d = {k: on_gpu(v) if torch.is_tensor(v) else v for k, v in c.items()}
    out = S.bcast_serve_append(d["q"], d["k"], d["v"], d["own_k"], d["own_v"], d["own_len"], page_table=d["page_table"])
    assert torch.equal(out, d["q"])                           # without inv_freq nothing turns


def test_append_cache_beyond_32_bits():
    # 2^31 numbers and more between the pages
    own = torch.empty(3, 16, 1, 64, dtype=torch.bfloat16, device=DEV)
    flat = torch.zeros(2 * (3 << 30) // 2 + 4096, dtype=torch.bfloat16, device=DEV)
    far = flat.as_strided((3, 16, 1, 64), (3 << 29, 64, 64, 1))
    assert 2 * (3 << 29) > 2 ** 31
    c = append_case(17, 1, 4, 2, 1, 64, "bf16", page=16, cap=48, lengths=[36], norm=True)
    c["page_table"] = torch.tensor([[0, 1, 2]], dtype=torch.int32)
    d = {k: on_gpu(v) if torch.is_tensor(v) else v for k, v in c.items()}
    args = [d.pop(x) for x in ("q", "k", "v", "own_k", "own_v", "own_len")]
    own.zero_()
    want = S.bcast_serve_append(*args[:3], own, own.clone(), args[5], **d)
    got = S.bcast_serve_append(*args[:3], far, own.clone(), args[5], **d)
    assert torch.equal(got, want) and torch.equal(far, own) and bool(own[2, :4].any()) and not bool(own[:2].any())


def test_append_many_tokens_at_once_and_one_by_one():
    c = append_case(18, 700, 100, 3, 1, 32, "bf16", page=8, cap=120, norm=True, axes=2)
    d = {k: on_gpu(v) if torch.is_tensor(v) else v for k, v in c.items()}
    args = [d.pop(x) for x in ("q", "k", "v", "own_k", "own_v", "own_len")]
    own = args[3].clone(), args[4].clone()
    whole = S.bcast_serve_append(*args, **d)
    for i in range(0, 100, 25):                               # the last 25 tokens are the last 25 of a call for fewer
        part = {k: v[:, i:i + 25] if k == "positions" else v for k, v in d.items()}
        got = S.bcast_serve_append(args[0][:, i:i + 25], args[1][:, i:i + 25], args[2][:, i:i + 25], *own, args[5] - (75 - i), **part)
        assert torch.equal(got, whole[:, i:i + 25])
    assert torch.equal(own[0], args[3]) and torch.equal(own[1], args[4])


# so many tokens of so few heads that two or four of them share a warp, against calls for one request at a time
@pytest.mark.parametrize("B,n", [(16, 300), (41, 301)])
@pytest.mark.parametrize("HQ,H,D,more", [(1, 1, 128, dict(norm=True)), (0, 1, 96, dict(interleaved=True, norm=True)), (3, 1, 64, dict(axes=3)), (2, 2, 40, dict(rot=32)),
                                         (5, 1, 16, dict(norm=True, rot=0)), (8, 1, 8, dict())])
@pytest.mark.parametrize("ragged", [False, True])
def test_append_several_tokens_to_a_warp(B, n, HQ, H, D, more, ragged):
    g = gen(B + D)
    c = append_case(B + D, B, n, HQ, H, D, "bf16", page=16, cap=n + 40, new=torch.randint(0, n + 1, (B,), generator=g).tolist() if ragged else None,
                    lengths=torch.randint(0, n + 60, (B,), generator=g).tolist(), **more)
    d = {k: on_gpu(v) if torch.is_tensor(v) else v for k, v in c.items()}
    args = [d.pop(x) for x in ("q", "k", "v", "own_k", "own_v", "own_len")]
    own = args[3].clone(), args[4].clone()
    whole = S.bcast_serve_append(*args, **d)
    for b in range(B):
        part = {k: v[b:b + 1] if k in ("positions", "page_table", "new_len") else v for k, v in d.items()}
        got = S.bcast_serve_append(None if args[0] is None else args[0][b:b + 1], args[1][b:b + 1], args[2][b:b + 1], *own, args[5][b:b + 1], **part)
        assert got is None if whole is None else torch.equal(got, whole[b:b + 1])
    assert torch.equal(own[0], args[3]) and torch.equal(own[1], args[4])


def test_append_page_that_stands_in_the_table_twice():
    c = append_case(19, 2, 1, 2, 1, 64, "bf16", page=4, cap=8, lengths=[3, 3])
    c["page_table"][:] = 0
    d = {k: on_gpu(v) if torch.is_tensor(v) else v for k, v in c.items()}
    before = d["own_v"].clone()
    S.bcast_serve_append(d["q"], d["k"], d["v"], d["own_k"], d["own_v"], d["own_len"], page_table=d["page_table"])
    got = d["own_v"][0, 2]
    assert torch.equal(got, d["v"][0, 0]) or torch.equal(got, d["v"][1, 0])
    before[0, 2] = got
    assert torch.equal(before, d["own_v"])


# ------------------------------------------------------------------------------------------ logprobs
def logprobs_case(seed, T, V, dtype, std=2.0):
    g = gen(seed)
    return rand(g, T, V, std=std, dtype=TYPES[dtype]), torch.randint(0, V, (T,), generator=g, dtype=torch.int32)


def check_logprobs(logits, tokens, top, **more):
    want = R.logprobs(logits, tokens, top)
    lp, h, ids, best = S.bcast_serve_logprobs(on_gpu(logits), on_gpu(tokens), top=top, **more)
    torch.cuda.synchronize()
    close(lp, *want[0], "logprobs")
    close(h, *want[1], "entropy")
    assert torch.equal(ids.cpu(), want[2]), f"top_tokens: rows {(ids.cpu() != want[2]).any(dim=1).nonzero()[:5].tolist()}"
    close(best, *want[3], "top_logprobs")
    return lp, h, ids, best


@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 31, 255, 256, 1000, 4096, 5003, 16391, 32000, 50001, 131072, 300007])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T", [1, 5])
def test_logprobs_sizes(V, dtype, T):
    check_logprobs(*logprobs_case(V + T, T, V, dtype), 20)


@pytest.mark.parametrize("T", [1, 2, 36, 37, 38, 73, 75, 147, 149, 295, 297, 600])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_logprobs_rows(T, dtype):
    check_logprobs(*logprobs_case(T, T, 17003, dtype), 5)


# on both sides of what makes a row another number of blocks'
@pytest.mark.parametrize("T,V", [(32, 33001), (33, 33001), (64, 17003), (65, 17003), (129, 65537), (130, 65537), (129, 16384), (130, 16385), (37, 262147), (74, 131075), (148, 65535),
                                 (148, 65536), (149, 65539), (296, 65536), (4, 4095), (4, 4096), (4, 8192), (64, 16385)])
@pytest.mark.parametrize("dtype,top", [("bf16", 5), ("fp32", 20)])
def test_logprobs_blocks_to_a_row(T, V, dtype, top):
    check_logprobs(*logprobs_case(V + T, T, V, dtype), top)


@pytest.mark.parametrize("top", [0, 1, 2, 8, 31, 32])
@pytest.mark.parametrize("V", [20, 40, 9001, 70000])
def test_logprobs_tops(top, V):
    check_logprobs(*logprobs_case(top + V, 3, V, "bf16"), top)


# every number of rows that changes how many blocks share one
@pytest.mark.parametrize("T,V", [(3, 70001), (400, 9000)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_logprobs_orders(T, V, dtype):
    l, x = logprobs_case(T, T, V, dtype)
    l[0] = torch.sort(l[0]).values
    l[1] = torch.sort(l[1], descending=True).values
    l[2] = 1.25                                               # all equal
    check_logprobs(l[:3], x[:3], 20)
    if T > 3:
        l[3] = 0.0
        l[3, ::256 * 8] = 7.0                                 # the largest all in one thread's share
        l[4] = -3.0
        l[4, 5000:5010] = 2.0
        l[5] = torch.randint(0, 3, (V,), generator=gen(1)).to(l.dtype)
        l[6, V // 2:] = 30000.0
        l[7] = torch.arange(V) % 2048                         # many equals of the largest
        l[8] = -0.0
        l[8, 1::2] = 0.0                                      # equal, whatever their sign
        check_logprobs(l, x, 20)
        check_logprobs(l, x, 32)


@pytest.mark.parametrize("V", [100, 4097, 70001])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_logprobs_masks(V, dtype):
    low, T = torch.finfo(TYPES[dtype]).min, 14
    l, x = logprobs_case(V, T, V, dtype)
    l[0], l[1], l[2] = -math.inf, low, math.nan               # nothing, everything alike, nothing
    l[3, 5:] = -math.inf                                      # few tokens left
    l[4, 5:] = low
    l[5, :V - 3] = -math.inf
    l[6, :V - 3] = low
    l[7, ::2] = math.nan
    l[8, 17] = math.inf
    l[9, 3::7] = math.inf
    l[10, :] = -math.inf
    l[10, V // 2] = -5.0
    l[11, :] = math.inf
    l[12, 1:] = low
    l[12, 0] = -math.inf
    l[13, 1:] = math.nan
    x[:] = torch.tensor([0, 1, 2, 3, 7, V - 1, 5, 2, 17, 4, V // 2, 6, 0, 1])
    for top in (1, 8, 32):
        check_logprobs(l, x, top)


# a warp to a row: many short rows, every kind of mask and of equals among them
@pytest.mark.parametrize("V", [1, 2, 7, 31, 33, 256, 257, 1025, 1999, 3291, 4093, 8191])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_logprobs_a_warp_to_a_row(V, dtype):
    low, T = torch.finfo(TYPES[dtype]).min, 1187
    l, x = logprobs_case(V, T, V, dtype)
    l[0], l[1], l[2], l[3], l[4] = -math.inf, low, math.nan, math.inf, 1.25
    l[5, 5:], l[6, 5:] = -math.inf, low
    l[7, ::2] = math.nan
    l[8, V // 2] = math.inf
    l[9, ::3] = math.inf
    l[10] = torch.sort(l[10]).values
    l[11] = torch.sort(l[11], descending=True).values
    l[12] = torch.randint(0, 3, (V,), generator=gen(1)).to(l.dtype)
    l[13] = torch.arange(V) % 512
    l[14] = -0.0
    l[14, 1::2] = 0.0
    l[15] = torch.linspace(-50, 50, V).to(l.dtype)
    l[16, 1:] = math.nan
    x[0], x[1], x[2], x[3] = 0, V - 1, -1, V
    for top in (0, 1, 8, 24, 25):
        check_logprobs(l, x, top)
    check_logprobs(l[1:, V // 2:], x[1:], 5)                  # rows that begin anywhere


def test_logprobs_tokens_that_are_none():
    l, x = logprobs_case(3, 6, 500, "fp32")
    x[:] = torch.tensor([-1, 500, 499, 0, -2 ** 31, 2 ** 31 - 1])
    lp = check_logprobs(l, x, 3)[0]
    assert torch.isinf(lp).tolist() == [True, True, False, False, True, True]


@pytest.mark.parametrize("scale", [1e-3, 1.0, 30.0, 1e4, 1e30])
def test_logprobs_peaks(scale):
    l, x = logprobs_case(4, 8, 8000, "fp32", std=scale)
    x[:4] = l[:4].argmax(dim=-1).to(torch.int32)
    check_logprobs(l, x, 8)
    # rows that rise all the way: what the sums are taken against moves again and again
    l[:, :] = torch.linspace(-50, 50, 8000)
    check_logprobs(l, x, 8)


@pytest.mark.parametrize("dtype,pad", [("bf16", 1), ("bf16", 8), ("fp16", 3), ("fp32", 1), ("fp32", 2)])
def test_logprobs_strides(dtype, pad):
    g = gen(5)
    l = rand(g, 7, 3001 + pad, dtype=TYPES[dtype])[:, pad:]
    check_logprobs(l, torch.arange(7, dtype=torch.int32), 6)
    l = l[:1].expand(7, 3001)                                 # one row for all
    check_logprobs(l, torch.arange(7, dtype=torch.int32), 6)


def test_logprobs_given_outputs():
    l, x = logprobs_case(6, 9, 1234, "bf16")
    want = check_logprobs(l, x, 4)
    out = dict(logprobs=torch.full((9,), 7.0, device=DEV), entropy=torch.full((9,), 7.0, device=DEV), top_tokens=torch.full((9, 4), 7, dtype=torch.int32, device=DEV),
               top_logprobs=torch.full((9, 4), 7.0, device=DEV))
    got = S.bcast_serve_logprobs(on_gpu(l), on_gpu(x), top=4, **out)
    assert all(a.data_ptr() == b.data_ptr() and torch.equal(a, c) for a, b, c in zip(got, out.values(), want))
    assert [t.shape[0] for t in S.bcast_serve_logprobs(on_gpu(l[:0]), on_gpu(x[:0]), top=4)] == [0] * 4
    for name, bad in (("logprobs", torch.zeros(8, device=DEV)), ("top_tokens", torch.zeros(9, 4, device=DEV)), ("top_logprobs", torch.zeros(9, 8, device=DEV)[:, ::2])):
        with pytest.raises(BcastError) as e:
            S.bcast_serve_logprobs(on_gpu(l), on_gpu(x), top=4, **{name: bad})
        assert e.value.code == BCAST_ERR_INVAL and name in str(e.value)


def test_logprobs_many_rows():
    l, x = logprobs_case(7, 70001, 40, "fp32")
    d, e = on_gpu(l), on_gpu(x)
    lp, h, ids, best = S.bcast_serve_logprobs(d, e, top=3)
    for a in (0, 65530, 69000):
        rows = slice(a, a + 12)
        want = R.logprobs(l[rows], x[rows], 3)
        close(lp[rows], *want[0], "logprobs")
        close(h[rows], *want[1], "entropy")
        assert torch.equal(ids[rows].cpu(), want[2])
    order = torch.sort(d, dim=-1, descending=True, stable=True).indices[:, :3]
    assert torch.equal(ids, order.int())


@pytest.mark.parametrize("T,V,dtype", [(2, 3000001, "fp16"), (600, 300007, "bf16"), (600, 150001, "fp32")])
def test_logprobs_long_rows(T, V, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(V)
    l = (torch.randn(T, V, generator=g, device=DEV) * 2).to(TYPES[dtype])
    x = torch.arange(T, device=DEV, dtype=torch.int32) * 7
    lp, h, ids, best = S.bcast_serve_logprobs(l, x, top=32)
    rows = sorted({0, 1, T // 2, T - 1})
    want = R.logprobs(l[rows].cpu(), x[rows].cpu(), 32)
    close(lp[rows], *want[0], "logprobs")
    close(h[rows], *want[1], "entropy")
    assert torch.equal(ids[rows].cpu(), want[2])
    close(best[rows], *want[3], "top_logprobs")
    # all rows, found another way
    bits = l.float().view(torch.int32)
    key = (torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() << 32) + torch.arange(V - 1, -1, -1, device=DEV)
    assert torch.equal(ids.long(), V - 1 - (key.topk(32, dim=-1).values & 0xffffffff))


def test_logprobs_beyond_32_bits():
    T, V = 17000, 131072                                      # 2.2e9 logits
    l = torch.zeros(T, V, dtype=torch.bfloat16, device=DEV)
    l[T - 1, V - 3] = 9.0
    x = torch.full((T,), V - 3, dtype=torch.int32, device=DEV)
    lp, h, ids, best = S.bcast_serve_logprobs(l, x, top=2)
    assert ids[T - 1].tolist() == [V - 3, 0] and ids[5].tolist() == [0, 1] and torch.equal(best[T - 1, 0], lp[T - 1])
    assert abs(float(lp[T - 1]) - (9 - math.log(V - 1 + math.exp(9)))) < 1e-5 and abs(float(h[7]) - math.log(V)) < 1e-5


# ------------------------------------------------------------------------------------------ 4-bit numbers
def special(x):
    """Zeros, ties, the type's ends and numbers that are none, a block each, over what is there."""
    f = torch.finfo(x.dtype)
    flat = x.reshape(-1, 32)
    for i, block in enumerate((torch.zeros(32), -torch.zeros(32), torch.arange(32) * 0.25, -torch.arange(32) * 0.125, torch.full((32,), f.max),
                               torch.full((32,), f.min), torch.full((32,), f.smallest_normal), torch.full((32,), f.smallest_normal * f.eps),
                               torch.arange(32) * f.smallest_normal, torch.linspace(-7.9, 7.9, 32), torch.tensor([math.inf] + [1.0] * 31),
                               torch.tensor([1.0] * 31 + [-math.inf]), torch.tensor([1.0] * 16 + [math.nan] * 16))):
        if i < len(flat):
            flat[i] = block.to(x.dtype)
    return x


def same(got, want):
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isnan(got)], want[~torch.isnan(want)])


@pytest.mark.parametrize("rows,k", [(1, 32), (1, 416), (3, 64), (31, 96), (128, 128), (129, 160), (200, 2048), (5, 2080), (257, 4128), (1000, 1056)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_pack_and_unpack(rows, k, dtype):
    g, dt = gen(rows + k), TYPES[dtype]
    power = torch.randint(-14, 12, (rows, k // 32, 1), generator=g) if dtype == "fp16" else torch.randint(-130, 120, (rows, k // 32, 1), generator=g)
    x = special((rand(g, rows, k // 32, 32).double() * torch.exp2(power.double())).to(dt).reshape(rows, k))
    want, scales = R.pack(x)
    codes, s = S.bcast_serve_pack4(on_gpu(x))
    assert torch.equal(s.cpu(), R.tiled(scales))
    assert torch.equal(codes.cpu(), R.bytes_of(want))
    exact = R.values(want, scales)
    for t in TYPES.values():
        assert same(S.bcast_serve_unpack4(codes, s, t).cpu(), exact.to(t)), t


def test_unpack_every_code_and_scale():
    codes = (torch.arange(256 * 32) // 2 % 16).reshape(256, 32).to(torch.uint8)
    codes[:, 1::2] = torch.arange(16, dtype=torch.uint8)
    scales = torch.arange(256, dtype=torch.uint8)[:, None]
    got = S.bcast_serve_unpack4(on_gpu(R.bytes_of(codes)), on_gpu(R.tiled(scales)), torch.float32)
    assert same(got.cpu(), R.values(codes, scales).float())


def test_pack_strides_and_given_outputs():
    g = gen(7)
    x = rand(g, 70, 200, dtype=torch.bfloat16)[:, 8:168]
    want, scales = R.pack(x)
    codes, s = torch.full((70, 112), 7, dtype=torch.uint8, device=DEV), torch.full((1, 2, 32, 4, 4), 7, dtype=torch.uint8, device=DEV)
    got = S.bcast_serve_pack4(on_gpu(x), codes=codes[:, 16:96], scales=s)
    assert got[0].data_ptr() == codes.data_ptr() + 16 and torch.equal(codes[:, 16:96].cpu(), R.bytes_of(want)) and torch.equal(s.cpu(), R.tiled(scales))
    assert bool((codes[:, :16] == 7).all()) and bool((codes[:, 96:] == 7).all())
    out = torch.full((70, 176), 7.0, device=DEV)
    S.bcast_serve_unpack4(codes[:, 16:96], s, torch.float32, out=out[:, 8:168])
    assert torch.equal(out[:, 8:168].cpu(), R.values(want, scales).float()) and bool((out[:, :8] == 7).all()) and bool((out[:, 168:] == 7).all())
    for call in (lambda: S.bcast_serve_pack4(on_gpu(x)[:, 4:132]), lambda: S.bcast_serve_unpack4(codes[:, 8:88], s),
                 lambda: S.bcast_serve_pack4(on_gpu(x)[:, :40]), lambda: S.bcast_serve_unpack4(codes[:, 16:96], s, torch.float32, out=out[:, 8:160])):
        with pytest.raises(BcastError) as e:
            call()
        assert e.value.code == BCAST_ERR_INVAL
    c, s = S.bcast_serve_pack4(on_gpu(x[:0]))
    assert c.shape == (0, 80) and s.shape == (0, 2, 32, 4, 4) and S.bcast_serve_unpack4(c, s).shape == (0, 160)


def linear4_case(seed, T, K, N, dtype, bias=True):
    g, dt = gen(seed), TYPES[dtype]
    codes, scales = R.pack(rand(g, N, K, std=K ** -0.5))
    return dict(x=rand(g, T, K, dtype=dt), w_codes=codes, w_scales=scales, bias=rand(g, N, dtype=dt) if bias else None)


def call_linear4(c, **more):
    return S.bcast_serve_linear4(on_gpu(c["x"]), on_gpu(R.bytes_of(c["w_codes"])), on_gpu(R.tiled(c["w_scales"])), bias=on_gpu(c["bias"]), **more)


def check_linear4(c, **more):
    want, bound = R.linear4(**c)
    y = call_linear4(c, **more)
    torch.cuda.synchronize()
    close(y, want, bound, "y")
    return y


@pytest.mark.parametrize("K,N", [(32, 1), (64, 8), (96, 128), (128, 129), (160, 127), (256, 200), (288, 33), (1024, 1000), (2080, 130), (8192, 64)])
@pytest.mark.parametrize("T", [1, 3, 40, 140])
def test_linear4_sizes(K, N, T):
    check_linear4(linear4_case(K + N, T, K, N, "bf16"))


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 256, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_linear4_tokens(T, dtype):
    check_linear4(linear4_case(T, T, 544, 264, dtype, bias=T % 2 == 0))


@pytest.mark.parametrize("T,K,N", [(450, 96, 19100), (1000, 320, 9000), (1345, 544, 5003), (225, 64, 38000)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_linear4_several_rounds_of_tiles(T, K, N, dtype):
    check_linear4(linear4_case(T + N, T, K, N, dtype))


def test_linear4_sums_of_its_own_numbers_are_exact():
    # whole numbers that 4 bits hold: no rounding but the result's
    g = gen(8)
    for T, K, N in ((5, 160, 70), (70, 512, 300), (300, 96, 260)):
        x = torch.tensor([0.0, 1, 2, 3, 4, -1, -2, -3, -4])[torch.randint(0, 9, (T, K), generator=g)]
        w = torch.tensor([0.0, 0.5, 1, 1.5, 2, 3, 4, -0.5, -6])[torch.randint(0, 9, (N, K), generator=g)]
        x[:, ::32], w[:, ::32] = 4.0, 4.0                     # so that every block's unit is 1
        codes, scales = R.pack(w)
        assert torch.equal(R.values(codes, scales), w.double()) and torch.equal(R.values(*R.pack(x)), x.double())
        y = call_linear4(dict(x=x.bfloat16(), w_codes=codes, w_scales=scales, bias=None))
        assert torch.equal(y.cpu(), (x.double() @ w.double().T).bfloat16())


@pytest.mark.parametrize("T,K,N", [(70001, 32, 130), (3, 32, 70000), (5000, 96, 4099), (9, 16384, 40), (8, 16384, 300)])
def test_linear4_long_sides(T, K, N):
    # whole numbers again: exact, whatever the order of the sums
    g = gen(T + N)
    x = torch.tensor([0.0, 1, 2, 3, 4, -1, -2, -3, -4])[torch.randint(0, 9, (T, K), generator=g)]
    w = torch.tensor([0.0, 0.5, 1, 1.5, 2, 3, 4, -0.5, -6])[torch.randint(0, 9, (N, K), generator=g)]
    x[:, ::32], w[:, ::32] = 4.0, 4.0
    codes, s = S.bcast_serve_pack4(on_gpu(w))
    y = S.bcast_serve_linear4(on_gpu(x.bfloat16()), codes, s)
    for a in range(0, T, 10000):
        assert torch.equal(y[a:a + 10000].cpu(), (x[a:a + 10000] @ w.T).bfloat16())


def test_linear4_scales_of_all_sizes():
    g = gen(9)
    c = linear4_case(9, 20, 256, 150, "bf16")
    c["x"] = (c["x"].reshape(20, 8, 32) * torch.exp2(torch.randint(-40, 40, (20, 8, 1), generator=g).float())).reshape(20, 256).bfloat16()
    c["w_scales"] = torch.randint(80, 170, c["w_scales"].shape, generator=g).to(torch.uint8)
    check_linear4(c)
    c["x"][:], c["bias"] = 0.0, None
    assert not bool(call_linear4(c).any())


def test_linear4_numbers_that_are_none():
    for T in (4, 200):
        c = linear4_case(10, T, 320, 150, "bf16")
        c["x"][1, 40], c["x"][2, 319] = math.nan, math.inf
        c["w_scales"][7, 3] = 255
        y = check_linear4(c)                                  # rows 1 and 2 and feature 7, and nothing else
        assert int(torch.isnan(y).sum()) == 2 * 150 + T - 2


def test_linear4_strides():
    c = linear4_case(11, 37, 192, 100, "fp16")
    want = check_linear4(c)
    wide = torch.full((100, 128), 255, dtype=torch.uint8, device=DEV)
    wide[:, 16:112] = on_gpu(R.bytes_of(c["w_codes"]))
    x = torch.full((37, 216), math.nan, dtype=torch.float16, device=DEV)
    x[:, 8:200] = on_gpu(c["x"])
    out = torch.full((37, 111), 7.0, dtype=torch.float16, device=DEV)
    y = S.bcast_serve_linear4(x[:, 8:200], wide[:, 16:112], on_gpu(R.tiled(c["w_scales"])), bias=on_gpu(c["bias"]), out=out[:, 3:103])
    assert torch.equal(y, want) and bool((out[:, :3] == 7).all()) and bool((out[:, 103:] == 7).all())
    with pytest.raises(BcastError):
        S.bcast_serve_linear4(x[:, 4:196], wide[:, 16:112], on_gpu(R.tiled(c["w_scales"])))
    assert S.bcast_serve_linear4(x[:0, 8:200], wide[:, 16:112], on_gpu(R.tiled(c["w_scales"]))).shape == (0, 100)


def test_linear4_repeats_bit_for_bit():
    for T, K, N in ((1, 4096, 512), (60, 4096, 1000), (600, 1056, 3000), (2000, 544, 6000)):
        c = linear4_case(T, T, K, N, "bf16")
        d = (on_gpu(c["x"]), on_gpu(R.bytes_of(c["w_codes"])), on_gpu(R.tiled(c["w_scales"])))
        ws = S.Workspace(DEV)
        first = S.bcast_serve_linear4(*d, workspace=ws)
        assert bool(torch.isfinite(first).all())
        for _ in range(20):
            assert torch.equal(S.bcast_serve_linear4(*d, workspace=ws), first)
        S.bcast_serve_status(ws)


def test_linear4_workspace_left_by_other_calls():
    # what a call leaves in its workspace means nothing to the next one
    ws = S.Workspace(DEV, 1 << 20)
    for T, K, N in ((100, 544, 200), (3, 96, 130), (130, 160, 70), (1, 4096, 128)):
        ws.reserve(0)[256:].fill_(255)
        check_linear4(linear4_case(T, T, K, N, "bf16"), workspace=ws)


# ------------------------------------------------------------------------------------------ streams, graphs, waits
def run_all(inputs, ws, outs=None, stream=None):
    """A run of the new operators as a step has it; returns all outputs."""
    a, lin, vocab = inputs
    o = outs or {}
    x = S.bcast_serve_linear4(lin["x"], lin["codes"], lin["scales"], workspace=ws, stream=stream, out=o.get("x"))
    q, k, v = x.view(4, 5, 8, 64).split((4, 2, 2), dim=2)
    q = S.bcast_serve_append(q, k, v, a["own_k"], a["own_v"], a["own_len"], page_table=a["page_table"], inv_freq=a["inv_freq"], stream=stream, out=o.get("q"))
    y = S.bcast_serve_attn(q, a["prefix"], a["prefix"], a["own_k"], a["own_v"], a["own_len"], page_table=a["page_table"], workspace=ws, stream=stream, out=o.get("y"))
    z = S.bcast_serve_linear4(y.view(20, 256), vocab["codes"], vocab["scales"], workspace=ws, stream=stream, out=o.get("z"))
    lp = S.bcast_serve_logprobs(z, a["tokens"], top=3, stream=stream, **{k: o[k] for k in ("logprobs", "entropy", "top_tokens", "top_logprobs") if k in o})
    return dict(x=x, q=q, y=y, z=z, logprobs=lp[0], entropy=lp[1], top_tokens=lp[2], top_logprobs=lp[3])


def all_inputs(seed):
    g = gen(seed)
    a = {k: on_gpu(v) if torch.is_tensor(v) else v for k, v in append_case(seed, 4, 5, 4, 2, 64, "bf16").items()}
    a["prefix"] = rand(g, 70, 2, 64, dtype=torch.bfloat16).to(DEV)
    a["tokens"] = torch.randint(0, 900, (20,), generator=g, dtype=torch.int32).to(DEV)
    packed = [dict(zip(("codes", "scales"), S.bcast_serve_pack4(rand(g, n, k, std=k ** -0.5).to(DEV)))) for n, k in ((512, 192), (900, 256))]
    packed[0]["x"] = rand(g, 20, 192, dtype=torch.bfloat16).to(DEV)
    return a, packed[0], packed[1]


def test_a_run_of_them_against_the_plain_forms():
    import serve_reference as R0
    inputs = all_inputs(20)
    a, lin, vocab = inputs
    before = {k: a[k].cpu() for k in ("own_k", "own_v")}
    got = {k: v.cpu() for k, v in run_all(inputs, S.Workspace(DEV)).items()}

    def plain_weight(d):
        codes, s = d["codes"].cpu(), d["scales"].cpu()
        n, b = codes.shape[0], codes.shape[1] // 16
        r, c = torch.arange(n)[:, None], torch.arange(b)[None, :]
        return torch.stack([codes & 15, codes >> 4], dim=-1).flatten(1), s[r // 128, c // 4, r % 32, r % 128 // 32, c % 4]
    close(got["x"], *R.linear4(lin["x"].cpu(), *plain_weight(lin)), "x")
    q, k, v = got["x"].view(4, 5, 8, 64).split((4, 2, 2), dim=2)
    host = {k: a[k].cpu() for k in ("own_len", "page_table", "inv_freq")}
    want = R.append(q, k, v, before["own_k"], before["own_v"], host["own_len"], page_table=host["page_table"], inv_freq=host["inv_freq"])
    close(got["q"], *want["q"], "q")
    close(a["own_k"], *want["own_k"], "own_k")
    close(a["own_v"], *want["own_v"], "own_v")
    y, bound, _, _ = R0.attn(got["q"], a["prefix"].cpu(), a["prefix"].cpu(), a["own_k"].cpu(), a["own_v"].cpu(), host["own_len"], host["page_table"])
    close(got["y"], y, bound, "y")
    close(got["z"], *R.linear4(got["y"].view(20, 256), *plain_weight(vocab)), "z")
    want = R.logprobs(got["z"], a["tokens"].cpu(), 3)
    close(got["logprobs"], *want[0], "logprobs")
    close(got["entropy"], *want[1], "entropy")
    assert torch.equal(got["top_tokens"], want[2])


@pytest.mark.parametrize("kept", [True, False])
def test_captured_and_replayed(kept):
    inputs, other = all_inputs(21), all_inputs(22)
    ws = S.Workspace(DEV) if kept else None
    want = [run_all(i, S.Workspace(DEV)) for i in (inputs, other)]
    outs = {k: torch.zeros_like(v) for k, v in want[0].items()}
    run_all(inputs, ws, outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_all(inputs, ws, outs)
    for turn in range(3):
        for t in outs.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(outs[k], want[0][k]) for k in outs), turn
    # other numbers in the same places
    for mine, new in zip(inputs, other):
        for k, v in mine.items():
            if torch.is_tensor(v):
                v.copy_(new[k])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(outs[k], want[1][k]) for k in outs)


@pytest.mark.parametrize("named", ["stream", "raw", "current"])
def test_streams(named):
    inputs = all_inputs(23)
    want = run_all(inputs, S.Workspace(DEV))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ws = S.Workspace(DEV)
    if named == "current":
        with torch.cuda.stream(side):
            got = run_all(inputs, ws)
    else:
        got = run_all(inputs, ws, stream=side if named == "stream" else side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)


def test_two_streams_at_once():
    cases = [all_inputs(24), all_inputs(25)]
    want = [run_all(c, S.Workspace(DEV)) for c in cases]
    torch.cuda.synchronize()
    streams, spaces = [torch.cuda.Stream() for _ in cases], [S.Workspace(DEV) for _ in cases]
    got = [[], []]
    for _ in range(10):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i].append(run_all(cases[i], spaces[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o[k], want[i][k]) for i in (0, 1) for o in got[i] for k in o)


def test_two_graphs_with_one_workspace():
    # replayed one after the other on one stream, in any order, each as it was captured
    cases = [all_inputs(27), all_inputs(28)]
    want = [run_all(c, S.Workspace(DEV)) for c in cases]
    ws = S.Workspace(DEV)
    outs = [{k: torch.zeros_like(v) for k, v in w.items()} for w in want]
    for c, o in zip(cases, outs):
        run_all(c, ws, o)
    torch.cuda.synchronize()
    graphs = []
    for c, o in zip(cases, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            run_all(c, ws, o)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1, 0)):
        for o in outs:
            for t in o.values():
                t.zero_()
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(outs[i][k], want[i][k]) for i in (0, 1) for k in want[i])
    S.bcast_serve_status(ws)


def test_weights_made_right_before_the_product():
    # the product's blocks begin early: not before the kernels ahead of them on the stream have written W and x
    g = gen(29)
    for T in (1, 8, 40, 500):
        w, x = on_gpu(rand(g, 3000, 512)), on_gpu(rand(g, T, 512, dtype=torch.bfloat16))
        codes, scales = S.bcast_serve_pack4(w)
        want = S.bcast_serve_linear4(x, codes, scales)
        torch.cuda.synchronize()
        ws, xx, cc, ss = S.Workspace(DEV, 1 << 22), torch.zeros_like(x), torch.zeros_like(codes), torch.zeros_like(scales)
        for _ in range(20):
            cc.zero_()
            xx.zero_()
            S.bcast_serve_pack4(w, codes=cc, scales=ss)
            y0 = S.bcast_serve_linear4(xx, cc, ss, workspace=ws)
            xx.copy_(x)
            y = S.bcast_serve_linear4(xx, cc, ss, workspace=ws)
            assert not bool(y0.any()) and torch.equal(y, want)


def test_workspace_that_is_too_small_in_a_capture():
    c = linear4_case(26, 100, 512, 200, "bf16")
    d = (on_gpu(c["x"]), on_gpu(R.bytes_of(c["w_codes"])), on_gpu(R.tiled(c["w_scales"])))
    ws = S.Workspace(DEV)
    one = torch.zeros(4, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.add_(1.0)
        with pytest.raises(BcastError) as e:
            S.bcast_serve_linear4(*d, out=torch.empty(100, 200, dtype=torch.bfloat16, device=DEV), workspace=ws)
        assert e.value.code == BCAST_ERR_CAPACITY


WAITS_CHILD = """
import sys
sys.path[:0] = [sys.argv[1], sys.argv[1] + "/tests"]
import torch
import test_serve_more_gpu as T
from paper_1603_06809_b200 import serve as S
from paper_1603_06809_b200.bcast import BcastError
ws = S.Workspace("cuda:0")
for i, (n, k, f) in enumerate([(1, 64, 100), (20, 4096, 256), (60, 2048, 500), (300, 544, 300), (2000, 544, 6000), (449, 64, 19200), (5, 8192, 300),
                               (8, 4096, 19000)]):
    c = T.linear4_case(i, n, k, f, "bf16")
    y = T.call_linear4(c, workspace=ws)
    try:
        S.bcast_serve_status(ws)
        print("CALL", i, 0)
    except BcastError as e:
        print("CALL", i, e.code)
print("END")
"""


@pytest.mark.parametrize("given_up", ["", "1"])
def test_waits_that_run_out_end_the_kernels(given_up):
    env = dict(os.environ)
    env.pop("BCAST_SERVE_GIVE_UP", None)
    if given_up:
        env["BCAST_SERVE_GIVE_UP"] = given_up
    out = subprocess.run([sys.executable, "-c", WAITS_CHILD, ROOT], env=env, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr[-2000:]
    want = BCAST_ERR_TIMEOUT if given_up else 0
    assert out.stdout.split("\n") == [f"CALL {i} {want}" for i in range(8)] + ["END", ""], out.stdout
