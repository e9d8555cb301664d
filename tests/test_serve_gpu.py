"""The serving operators on the GPU against plain 64-bit forms, through the public binding."""
import math

import pytest
import torch

import serve_reference as R
from paper_1603_06809_b200 import serve as S
from paper_1603_06809_b200.bcast import BCAST_ERR_CAPACITY, BCAST_ERR_INVAL, BcastError

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def rand(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g) * std).to(dtype)


def on_gpu(t):
    """A copy on the GPU with the same strides (broadcast and padded ones included)."""
    if t is None:
        return None
    if t.numel() == 0 or t.is_contiguous():
        return t.to(DEV)
    span = sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1
    flat = torch.as_strided(t, (span,), (1,)).to(DEV)
    return torch.as_strided(flat, t.shape, t.stride())


def inside(got, want, bound, what):
    got = got.double().cpu()
    assert not torch.isnan(got).any(), f"{what}: NaN"
    over = (got - want).abs() - bound
    assert bool((over <= 0).all()), f"{what}: {float((got - want).abs().max())} off, bound passed by {float(over.max())}"


# ------------------------------------------------------------------------------------------ linear
def linear_case(seed, T, K, N, L, rank, dtype, bias=True, how="mixed"):
    g, dt = gen(seed), TYPES[dtype]
    c = dict(x=rand(g, T, K, dtype=dt), weight=rand(g, N, K, std=K ** -0.5, dtype=dt))
    c["bias"] = rand(g, N, dtype=dt) if bias else None
    if L:
        c.update(lora_a=rand(g, L, rank, K, std=K ** -0.5, dtype=dt), lora_b=rand(g, L, N, rank, std=rank ** -0.5, dtype=dt),
                 scale=torch.rand(L, generator=g) * 2 + 0.1)
        if how == "mixed":
            a = torch.randint(-1, L, (T,), generator=g)
        elif how == "runs":
            a = torch.arange(T) * L // max(T, 1) % L
        elif how == "none":
            a = torch.full((T,), -1)
        else:
            a = torch.full((T,), L - 1)
        c["adapter"] = a.to(torch.int32)
    return c


def check_linear(c, **more):
    want, bound = R.linear(**c)
    d = {k: on_gpu(v) for k, v in c.items()}
    x, w = d.pop("x"), d.pop("weight")
    y = S.bcast_serve_linear(x, w, **d, **more)
    torch.cuda.synchronize()
    inside(y, want, bound, "y")
    return y


@pytest.mark.parametrize("T", [1, 2, 7, 16, 17, 33, 64, 65, 128, 130, 257, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_linear_tokens(T, dtype):
    check_linear(linear_case(T, T, 264, 200, 3, 16, dtype))


@pytest.mark.parametrize("K,N", [(8, 1), (8, 8), (64, 128), (72, 129), (512, 127), (1000, 1000), (2048, 33), (4096, 130), (8192, 64)])
@pytest.mark.parametrize("T", [3, 40, 140])
def test_linear_sizes(K, N, T):
    check_linear(linear_case(K + N, T, K, N, 2, 8, "bf16"))


@pytest.mark.parametrize("rank", [8, 16, 24, 40, 64, 72, 120, 128])
@pytest.mark.parametrize("T,dtype", [(5, "bf16"), (70, "fp16"), (200, "bf16")])
def test_linear_ranks(rank, T, dtype):
    check_linear(linear_case(rank, T, 136, 264, 4, rank, dtype))


@pytest.mark.parametrize("how", ["mixed", "runs", "none", "one"])
@pytest.mark.parametrize("T,L", [(1, 1), (9, 40), (64, 64), (150, 100), (513, 7)])
def test_linear_assignments(how, T, L):
    check_linear(linear_case(T + L, T, 128, 136, L, 16, "bf16", bias=False, how=how))


@pytest.mark.parametrize("T,K,N,L,rank,how", [(300, 72, 28500, 3, 16, "mixed"), (700, 136, 19100, 40, 64, "runs"), (513, 72, 19007, 5, 128, "mixed"),
                                              (1025, 200, 12000, 2, 24, "one"), (290, 64, 57000, 0, 0, "none")])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_linear_several_rounds_of_tiles(T, K, N, L, rank, how, dtype):
    # three rounds of tiles of 256 tokens and more: blocks that take one after the other
    assert -(-T // 256) * -(-N // 128) >= 3 * 148
    check_linear(linear_case(T + N, T, K, N, L, rank, dtype, how=how))


@pytest.mark.parametrize("T", [1, 30, 200])
def test_linear_without_adapters(T):
    check_linear(linear_case(T, T, 320, 136, 0, 0, "fp16"))


def test_linear_numbers_out_of_range_mean_no_adapter():
    c = linear_case(5, 20, 128, 64, 3, 16, "bf16")
    c["adapter"] = torch.tensor([3, -1, -7, 2 ** 31 - 1, -2 ** 31] * 4, dtype=torch.int32)
    a = check_linear(c)
    for k in ("lora_a", "lora_b", "adapter", "scale"):
        c[k] = None
    c = {k: v for k, v in c.items() if v is not None}
    assert torch.equal(a, check_linear(c))


def test_linear_strided_operands_and_output():
    g = gen(3)
    c = linear_case(3, 37, 128, 100, 3, 16, "bf16")
    pad = {"x": rand(g, 37, 200, dtype=torch.bfloat16)[:, 32:160], "weight": rand(g, 100, 256, std=0.1, dtype=torch.bfloat16)[:, :128],
           "lora_a": rand(g, 3, 20, 136, std=0.1, dtype=torch.bfloat16)[:, :16, 8:], "lora_b": rand(g, 3, 104, 32, dtype=torch.bfloat16)[:, :100, 16:]}
    c.update(pad)
    big = torch.full((37, 131), 7.0, dtype=torch.bfloat16, device=DEV)
    check_linear(c, out=big[:, 3:103])
    assert bool((big[:, :3] == 7).all()) and bool((big[:, 103:] == 7).all())


def test_linear_adapter_that_nobody_asked_for_may_hold_anything():
    c = linear_case(8, 50, 128, 96, 4, 16, "bf16")
    c["adapter"][c["adapter"] == 2] = 1
    c["lora_a"][2] = math.nan
    c["lora_b"][2] = math.inf
    c["scale"][2] = math.nan
    check_linear(c)


def test_linear_tokens_do_not_touch_each_other():
    c = linear_case(9, 80, 128, 96, 3, 16, "fp16")
    clean = check_linear(c).cpu()
    c["x"][13] = math.nan
    c["x"][61] = math.inf
    d = {k: on_gpu(v) for k, v in c.items()}
    y = S.bcast_serve_linear(d.pop("x"), d.pop("weight"), **d).cpu()
    keep = torch.ones(80, dtype=torch.bool)
    keep[[13, 61]] = False
    assert torch.equal(y[keep], clean[keep])
    assert bool(torch.isnan(y[13]).all()) and not bool(torch.isfinite(y[61]).all())


def test_linear_no_tokens():
    c = linear_case(1, 0, 64, 32, 2, 8, "bf16")
    d = {k: on_gpu(v) for k, v in c.items()}
    assert S.bcast_serve_linear(d.pop("x"), d.pop("weight"), **d).shape == (0, 32)


def test_linear_repeats_bit_for_bit():
    c = linear_case(11, 90, 1024, 300, 5, 32, "bf16")
    d = {k: on_gpu(v) for k, v in c.items()}
    x, w = d.pop("x"), d.pop("weight")
    ws = S.Workspace(DEV)
    first = S.bcast_serve_linear(x, w, workspace=ws, **d)
    for _ in range(20):
        assert torch.equal(first, S.bcast_serve_linear(x, w, workspace=ws, **d))
    S.bcast_serve_status(ws)


# ------------------------------------------------------------------------------------------ attn
def attn_case(seed, B, n, H, G, D, P, cap, page, dtype, lengths=None):
    g, dt = gen(seed), TYPES[dtype]
    c = dict(q=rand(g, B, n, H * G, D, dtype=dt), prefix_k=rand(g, P, H, D, dtype=dt), prefix_v=rand(g, P, H, D, dtype=dt))
    if page:
        each = -(-cap // page)
        pages = B * each + 2
        c.update(own_k=rand(g, pages, page, H, D, dtype=dt), own_v=rand(g, pages, page, H, D, dtype=dt),
                 page_table=torch.randperm(pages, generator=g)[:B * each].reshape(B, each).to(torch.int32))
    else:
        c.update(own_k=rand(g, B, cap, H, D, dtype=dt), own_v=rand(g, B, cap, H, D, dtype=dt))
    if lengths is None:
        lengths = torch.randint(min(n, cap), cap + 1, (B,), generator=g) if cap else torch.zeros(B)
    c["own_len"] = torch.as_tensor(lengths).to(torch.int32)
    return c


def check_attn(c, scale=None, **more):
    want, bound, lse, lse_bound = R.attn(scale=scale, **c)
    d = {k: on_gpu(v) for k, v in c.items()}
    table = d.pop("page_table", None)
    got_lse = torch.full(lse.shape, 5.0, device=DEV)
    out = S.bcast_serve_attn(*d.values(), page_table=table, scale=scale, lse=got_lse, **more) if list(d) == [
        "q", "prefix_k", "prefix_v", "own_k", "own_v", "own_len"] else S.bcast_serve_attn(
        d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"], page_table=table, scale=scale, lse=got_lse, **more)
    torch.cuda.synchronize()
    inside(out, want, bound, "out")
    got_lse = got_lse.double().cpu()
    empty = lse == -math.inf
    assert torch.equal(got_lse == -math.inf, empty)
    assert bool(((got_lse - lse).abs()[~empty] <= lse_bound[~empty]).all()), float((got_lse - lse).abs()[~empty].max())
    assert bool((out.cpu()[empty] == 0).all())
    return out


@pytest.mark.parametrize("P", [0, 1, 2, 31, 127, 128, 129, 255, 257, 500])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attn_prefix_lengths(P, dtype):
    check_attn(attn_case(P, 3, 1, 2, 4, 64, P, 70, 0, dtype))


@pytest.mark.parametrize("cap,page", [(0, 0), (1, 0), (2, 0), (15, 0), (16, 0), (33, 0), (64, 0), (65, 0), (130, 0), (300, 0),
                                      (1, 16), (16, 16), (17, 16), (40, 16), (100, 7), (130, 64), (200, 32), (129, 128), (30, 1)])
def test_attn_own_lengths(cap, page):
    check_attn(attn_case(cap + page, 4, 1, 2, 2, 64, 40, cap, page, "bf16"))


@pytest.mark.parametrize("D", [8, 16, 24, 40, 64, 72, 80, 96, 104, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attn_head_sizes(D, dtype):
    check_attn(attn_case(D, 2, 2, 2, 2, D, 150, 40, 16, dtype))


@pytest.mark.parametrize("n", [1, 2, 3, 5, 8, 17])
@pytest.mark.parametrize("H,G", [(1, 1), (2, 1), (1, 8), (3, 5), (2, 7), (1, 16)])
def test_attn_new_tokens_and_heads(n, H, G):
    check_attn(attn_case(n * 100 + H * 10 + G, 2, n, H, G, 64, 100, 40, 0, "bf16"))


@pytest.mark.parametrize("B", [1, 5, 16, 33, 70, 130])
def test_attn_batches(B):
    check_attn(attn_case(B, B, 1, 1, 4, 64, 140, 9, 4, "fp16"))


def test_attn_many_rows_on_one_head():
    check_attn(attn_case(77, 40, 3, 1, 4, 128, 200, 20, 16, "bf16"))


def test_attn_long_prefix_few_rows():
    check_attn(attn_case(78, 1, 1, 1, 2, 128, 9001, 5, 0, "bf16"))


def test_attn_long_own():
    check_attn(attn_case(79, 2, 1, 1, 4, 64, 10, 3001, 16, "bf16", lengths=[3001, 1777]))


@pytest.mark.parametrize("P", [0, 30])
def test_attn_rows_without_own_tokens(P):
    # lengths below the number of new tokens: the first new tokens see nothing of their own; negative and too
    # large lengths count as none and all
    c = attn_case(21, 6, 4, 2, 2, 64, P, 24, 8, "bf16", lengths=[0, 1, 3, 4, -5, 1000])
    check_attn(c)


def test_attn_nothing_at_all():
    c = attn_case(22, 3, 2, 2, 2, 64, 0, 0, 0, "fp16")
    check_attn(c)


@pytest.mark.parametrize("page", [0, 16])
def test_attn_rows_behind_the_length_may_hold_anything(page):
    c = attn_case(23, 4, 2, 2, 3, 64, 50, 80, page, "bf16", lengths=[2, 17, 33, 80])
    for name, bad in (("own_k", math.nan), ("own_v", math.inf)):
        for b, length in enumerate(c["own_len"].tolist()):
            for j in range(length, 80):
                if page:
                    c[name][c["page_table"][b, j // page], j % page] = bad
                else:
                    c[name][b, j] = bad
    check_attn(c)


def test_attn_pages_that_are_not_there():
    c = attn_case(24, 3, 1, 2, 2, 64, 20, 64, 16, "bf16", lengths=[64, 64, 40])
    c["page_table"][0, 1] = -1
    c["page_table"][1] = 10 ** 9
    c["page_table"][2, 0] = c["own_k"].shape[0]
    check_attn(c)
    c["prefix_k"], c["prefix_v"] = c["prefix_k"][:0], c["prefix_v"][:0]
    check_attn(c)


def test_attn_large_and_equal_scores():
    g = gen(25)
    c = attn_case(25, 2, 2, 1, 4, 64, 300, 40, 0, "bf16")
    c["q"] = c["q"] * 30
    check_attn(c)                                      # nearly one-hot weights
    c["q"] = torch.zeros_like(c["q"])
    check_attn(c)                                      # all weights equal
    c["q"] = rand(g, *c["q"].shape, std=40.0, dtype=torch.bfloat16)
    c["prefix_k"][200:] *= 8                           # the maximum grows late in the row
    check_attn(c)


def test_attn_scales():
    for scale in (0.0, 0.05, 1.0, -0.3):
        check_attn(attn_case(26, 2, 1, 2, 2, 64, 200, 30, 16, "fp16"), scale=scale)


@pytest.mark.parametrize("rows", [3, 60])
def test_attn_strides(rows):
    g = gen(27)
    B, n, H, G, D, P, cap = rows, 2, 2, 2, 72, 150, 20
    bf = torch.bfloat16
    c = attn_case(27, B, n, H, G, D, P, cap, 0, "bf16")
    c["q"] = rand(g, n, B, H * G, 80, dtype=bf).transpose(0, 1)[..., :D]
    c["prefix_k"] = rand(g, H, P, 96, dtype=bf).transpose(0, 1)[..., 8:80]
    c["prefix_v"] = rand(g, P, H, 2, D, dtype=bf)[:, :, 1]
    c["own_k"] = rand(g, H, B, cap, D, dtype=bf).permute(1, 2, 0, 3)
    c["own_v"] = rand(g, cap, B, H, 88, dtype=bf).transpose(0, 1)[..., 16:]
    out = torch.full((B, H * G, n, D), 3.0, dtype=bf, device=DEV).transpose(1, 2)
    check_attn(c, out=out)


def test_attn_requests_that_share_their_own_rows():
    c = attn_case(28, 1, 1, 2, 2, 64, 30, 40, 0, "bf16", lengths=[33])
    c["q"] = rand(gen(28), 5, 1, 4, 64, dtype=torch.bfloat16)
    c["own_k"], c["own_v"] = c["own_k"].expand(5, -1, -1, -1), c["own_v"].expand(5, -1, -1, -1)
    c["own_len"] = torch.tensor([33, 1, 40, 20, 0], dtype=torch.int32)
    check_attn(c)


def test_attn_requests_do_not_touch_each_other():
    c = attn_case(29, 6, 2, 2, 4, 64, 100, 30, 16, "bf16")
    clean = check_attn(c).cpu()
    c["q"][3] = math.nan
    for p in c["page_table"][1].tolist():
        c["own_v"][p] = math.inf
    d = {k: on_gpu(v) for k, v in c.items()}
    out = S.bcast_serve_attn(d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"], page_table=d["page_table"]).cpu()
    for b in (0, 2, 4, 5):
        assert torch.equal(out[b], clean[b])
    assert bool(torch.isnan(out[3]).all())


def test_attn_offsets_past_32_bits():
    # heads 2^32 elements apart: 8.6 GB per cache, of which a few rows are used
    B, cap, D, far = 2, 40, 64, 1 << 31
    c = attn_case(30, B, 1, 2, 2, D, 60, cap, 0, "bf16")
    want, bound, _, _ = R.attn(**c)
    d = {k: on_gpu(v) for k, v in c.items()}
    far_k = torch.empty(2 * far + (1 << 16), dtype=torch.bfloat16, device=DEV)

    def place(at, rows):
        for h in range(2):
            v = torch.as_strided(far_k, rows[..., 0, :].shape, tuple(rows[..., 0, :].contiguous().stride()), at + h * far)
            v.copy_(rows[..., h, :])
        st = list(rows[..., 0, :].contiguous().stride())
        return torch.as_strided(far_k, rows.shape, (*st[:-1], far, 1), at)
    pk, ok = place(0, d["prefix_k"]), place(1 << 15, d["own_k"])
    pv, ov = place(1 << 14, d["prefix_v"]), place((1 << 15) + (1 << 14), d["own_v"])
    out = S.bcast_serve_attn(d["q"], pk, pv, ok, ov, d["own_len"])
    inside(out, want, bound, "out")


def test_attn_repeats_bit_for_bit():
    c = attn_case(31, 9, 3, 2, 4, 128, 1000, 300, 16, "bf16")
    d = {k: on_gpu(v) for k, v in c.items()}
    ws = S.Workspace(DEV)
    go = lambda: S.bcast_serve_attn(d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"],  # noqa: E731
                                    page_table=d["page_table"], workspace=ws)
    first = go()
    for _ in range(20):
        assert torch.equal(first, go())
    S.bcast_serve_status(ws)


# ---- prefixes long enough for a kernel of their own: batch * kv_heads * ceil(n * G / 16) * P above 2^15
@pytest.mark.parametrize("P", [1025, 1151, 1152, 1153, 1279, 1281, 2100, 5000])
@pytest.mark.parametrize("B,H,G", [(17, 2, 4), (40, 1, 4)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attn_long_prefix_lengths(P, B, H, G, dtype):
    check_attn(attn_case(P + B, B, 1, H, G, 64, P, 30, 16, dtype))


@pytest.mark.parametrize("D", [8, 16, 24, 40, 64, 72, 80, 96, 104, 128])
@pytest.mark.parametrize("B,H", [(17, 2), (34, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attn_long_prefix_head_sizes(D, B, H, dtype):
    check_attn(attn_case(D + B, B, 1, H, 4, D, 1100, 20, 0, dtype))


@pytest.mark.parametrize("B,n,H,G", [(1, 1, 1, 1), (1, 3, 2, 5), (5, 4, 1, 7), (33, 2, 1, 2), (32, 1, 1, 4), (33, 1, 1, 4), (64, 1, 1, 4), (65, 1, 1, 4), (20, 5, 1, 8)])
def test_attn_long_prefix_rows(B, n, H, G):
    # rows of a key/value head from one to several tiles of 256, the last one with few
    P = -(-(1 << 15) // (B * H * -(-n * G // 16))) + 77
    check_attn(attn_case(B * 10 + n, B, n, H, G, 128, P, 9, 4, "bf16"))


@pytest.mark.parametrize("P,H,B,D,dtype", [(303105, 1, 1100, 64, "bf16"), (75791, 8, 300, 128, "fp16"), (134801, 3, 610, 96, "bf16")])
def test_attn_prefix_of_many_rows_and_tiles(P, H, B, D, dtype):
    # pairs of 128-row tiles and 64 tiles of tokens to an SM; a few rows of the result are compared
    G = 1
    tiles = -(-B * G // 128)
    B = B if tiles % 2 == 0 else B + 128
    tiles = -(-B * G // 128)
    assert tiles % 2 == 0 and tiles // 2 * H * -(-P // 128) >= 64 * 148
    g = gen(P)
    dt = TYPES[dtype]
    pool = rand(g, 4096 + 77, H, D, dtype=dt)                       # the prefix repeats a pool of tokens, shifted for its values
    at = torch.arange(P)
    pk, pv = pool[at % 4173], pool[(at * 7 + 5) % 4173]
    q, ok, ov = (rand(g, *shape, dtype=dt) for shape in ((B, 1, H * G, D), (B, 3, H, D), (B, 3, H, D)))
    ln = torch.randint(0, 4, (B,), generator=g).to(torch.int32)
    lse = torch.zeros(B, 1, H * G, device=DEV)
    out = S.bcast_serve_attn(*(t.to(DEV) for t in (q, pk, pv, ok, ov, ln)), lse=lse)
    torch.cuda.synchronize()
    rows = [0, 127, 128, B - 129, B - 1]
    want, bound, wl, wb = R.attn(q[rows], pk, pv, ok[rows], ov[rows], ln[rows])
    inside(out[rows], want, bound, "out")
    assert bool(((lse[rows].double().cpu() - wl).abs() <= wb).all())


@pytest.mark.parametrize("B", [17, 40])
def test_attn_long_prefix_without_own_tokens(B):
    c = attn_case(81, B, 3, 2, 2, 64, 1200, 16, 8, "bf16", lengths=[b % 6 for b in range(B)])
    check_attn(c)
    c["own_k"], c["own_v"] = torch.zeros(0, 8, 2, 64, dtype=torch.bfloat16), torch.zeros(0, 8, 2, 64, dtype=torch.bfloat16)
    check_attn(c)


@pytest.mark.parametrize("B", [17, 40])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attn_long_prefix_maximum_that_grows(B, dtype):
    g = gen(82)
    c = attn_case(82, B, 1, 2, 4, 64, 1300, 16, 0, dtype)
    for lo, factor in ((100, 3), (140, 8), (500, 20), (530, 30), (1000, 60), (1290, 90)):
        c["prefix_k"][lo:] = rand(g, 1300 - lo, 2, 64, std=factor, dtype=TYPES[dtype])      # it grows within tiles and between
    check_attn(c)
    c["q"] = torch.zeros_like(c["q"])
    check_attn(c)
    for scale in (0.0, 0.7, -0.2):
        check_attn(attn_case(83, B, 1, 2, 4, 64, 1300, 16, 0, dtype), scale=scale)


@pytest.mark.parametrize("B", [17, 40])
def test_attn_long_prefix_requests_do_not_touch_each_other(B):
    c = attn_case(84, B, 2, 1, 4, 64, 2000, 12, 16, "bf16")
    clean = check_attn(c).cpu()
    c["q"][3] = math.nan
    c["q"][7, :, 0, 0] = math.inf
    d = {k: on_gpu(v) for k, v in c.items()}
    out = S.bcast_serve_attn(d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"], page_table=d["page_table"]).cpu()
    keep = [b for b in range(B) if b not in (3, 7)]
    assert torch.equal(out[keep], clean[keep])
    assert bool(torch.isnan(out[3]).all()) and not bool(torch.isfinite(out[7, :, 0]).all())
    assert torch.equal(out[7, :, 1:], clean[7, :, 1:])


def test_attn_long_prefix_strides_and_far_heads():
    # heads 2^32 bytes apart, rows in wider ones
    B, D, P, far = 40, 72, 1000, 1 << 31
    bf = torch.bfloat16
    c = attn_case(85, B, 1, 2, 4, D, P, 20, 0, "bf16")
    want, bound, _, _ = R.attn(**c)
    d = {k: on_gpu(v) for k, v in c.items()}
    flat = torch.full((far + (1 << 20),), math.nan, dtype=bf, device=DEV)

    def place(at, rows):
        v = torch.as_strided(flat, rows.shape, (88, far, 1), at)
        v.copy_(rows)
        return v
    out = S.bcast_serve_attn(d["q"], place(0, d["prefix_k"]), place(1 << 18, d["prefix_v"]), d["own_k"], d["own_v"], d["own_len"])
    inside(out, want, bound, "out")


def test_attn_long_prefix_repeats_bit_for_bit():
    for B in (17, 40):
        c = attn_case(86, B, 3, 2, 4, 128, 3000, 300, 16, "bf16")
        d = {k: on_gpu(v) for k, v in c.items()}
        ws = S.Workspace(DEV)
        go = lambda: S.bcast_serve_attn(d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"],  # noqa: E731
                                        page_table=d["page_table"], workspace=ws)
        first = go()
        for _ in range(20):
            assert torch.equal(first, go())
        S.bcast_serve_status(ws)


# ------------------------------------------------------------------------------------------ verify
def verify_case(seed, B, n, V, dtype, greedy=False, near=0.4):
    g = gen(seed)
    logits = rand(g, B, n + 1, V, std=2.0)
    t = torch.rand(B, generator=g) * 0.8 + 0.5
    if greedy:
        t[::2] = 0.0
    tt = torch.where(t > 0, t, 1.0)[:, None, None]
    q = torch.softmax((logits[:, :n] + rand(g, B, n, V, std=near)) / tt, -1)
    e = torch.empty(B, n, V).exponential_(generator=g)
    x = (q / e).argmax(-1).to(torch.int32)
    logits = logits.to(TYPES[dtype])
    if greedy:
        x[::2] = torch.where(torch.rand(x[::2].shape, generator=g) < 0.7, logits[::2, :n].float().argmax(-1), x[::2]).to(torch.int32)
    return dict(logits=logits, draft_probs=q, draft_tokens=x, uniforms=torch.rand(B, n, generator=g),
                noise=torch.empty(B, V).exponential_(generator=g).clamp(min=1e-9), temperature=t)


def check_verify(c, **more):
    accepted, tokens, margin = R.verify(**c)
    assert margin > 1e-5, "inputs whose outcome 32 bits cannot tell"
    got = S.bcast_serve_verify(*(on_gpu(v) for v in c.values()), **more)
    assert torch.equal(got[0].cpu(), accepted)
    assert torch.equal(got[1].cpu(), tokens)
    return got


VERIFY_SIZES = [(1, 0, 5), (1, 1, 1), (1, 4, 2), (3, 4, 7), (4, 3, 31), (2, 5, 100), (9, 7, 257), (5, 1, 1000), (2, 4, 2047), (3, 3, 4099),
                (2, 63, 50), (33, 2, 300), (70, 33, 64), (2, 3, 33333)]


@pytest.mark.parametrize("B,n,V", VERIFY_SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("greedy", [False, True])
def test_verify_sizes(B, n, V, dtype, greedy):
    check_verify(verify_case(B * 1000 + n * 10 + V, B, n, V, dtype, greedy))


def test_verify_strides_and_odd_starts():
    g = gen(41)
    c = verify_case(41, 3, 4, 501, "bf16")
    wide = torch.empty(3, 7, 513, dtype=torch.bfloat16)
    wide[:, :5, 3:504] = c["logits"]
    c["logits"] = wide[:, :5, 3:504]
    q = torch.empty(4, 3, 503)
    q[:, :, 1:502] = c["draft_probs"].transpose(0, 1)
    c["draft_probs"] = q.transpose(0, 1)[:, :, 1:502]
    nz = torch.empty(3, 600)
    nz[:, 7:508] = c["noise"]
    c["noise"] = nz[:, 7:508]
    check_verify(c)
    c["noise"] = torch.empty(1, 501).exponential_(generator=g).expand(3, 501)      # one row for all requests
    check_verify(c)


def test_verify_ties_go_to_the_lowest_token():
    c = verify_case(42, 2, 2, 300, "bf16")
    c["logits"].fill_(1.0)
    c["temperature"][:] = torch.tensor([0.0, 1.0])
    c["draft_tokens"][0] = torch.tensor([0, 1], dtype=torch.int32)
    c["draft_probs"].fill_(1 / 512)
    c["draft_tokens"][1] = torch.tensor([299, 5], dtype=torch.int32)
    c["uniforms"][1] = torch.tensor([0.5, 0.5])
    c["noise"].fill_(1.0)
    got = S.bcast_serve_verify(*(on_gpu(v) for v in c.values()))
    assert got[0].tolist() == [1, 2]
    assert got[1].tolist() == [[0, 0, -1], [299, 5, 0]]


def test_verify_infinities_and_nan():
    c = verify_case(43, 6, 2, 400, "fp32")
    lg = c["logits"]
    c["temperature"] = torch.tensor([1.0, 1.0, 0.0, 0.7, 1.0, 0.0])
    lg[0, :, 100:] = -math.inf                              # most tokens forbidden
    c["draft_tokens"][0] = 250
    lg[1, 0, 17] = math.inf                                 # certain tokens
    lg[1, 0, 30] = math.inf
    c["draft_tokens"][1, 0], c["uniforms"][1, 0], c["draft_probs"][1, 0, 17] = 17, 0.9, 0.5
    lg[2, 0, :50] = math.nan                                # NaN counts as -infinity
    lg[2, 0, 60] = 99.0
    c["draft_tokens"][2, 0] = 60
    lg[3] = -math.inf                                       # no probabilities at all
    lg[4] = math.nan
    lg[5, 0] = -math.inf
    got = check_verify(c)
    assert got[1][3].tolist() == [-1, -1, -1] and got[1][4].tolist() == [-1, -1, -1] and got[1][5].tolist() == [-1, -1, -1]


def test_verify_drafts_out_of_range_and_equal_distributions():
    c = verify_case(44, 4, 3, 129, "fp32")
    c["draft_tokens"][0, 0], c["draft_tokens"][1, 1], c["draft_tokens"][2, 2] = -1, 129, 2 ** 31 - 1
    c["uniforms"][3, 0] = 2.0                               # refuses even a certain draft: p - q is zero everywhere
    c["draft_probs"][3, 0] = 1.0                            # and nothing is left of p either
    check_verify(c)


def test_verify_noise_that_cannot_win():
    c = verify_case(45, 2, 1, 64, "bf16")
    c["noise"][:, ::2] = 0.0
    c["noise"][:, 1::4] = math.nan
    check_verify(c)
    c["noise"][:] = -1.0
    check_verify(c)


def test_verify_first_place_rejected_and_all_accepted():
    c = verify_case(46, 2, 5, 200, "fp16", near=0.0)
    c["uniforms"][:] = torch.tensor([[1.9] * 5, [0.0] * 5])
    c["draft_probs"][0] = 0.6
    got = check_verify(c)
    assert got[0].tolist() == [0, 5]


def test_verify_no_requests():
    c = verify_case(47, 1, 2, 30, "fp32")
    got = S.bcast_serve_verify(*(on_gpu(v[:0]) for v in c.values()))
    assert got[0].shape == (0,) and got[1].shape == (0, 3)


def test_verify_draws_from_the_target_distribution():
    # 40000 requests with the same p and q: what comes first is distributed as p, whatever q is
    g, B, V = gen(48), 40000, 6
    logits = torch.tensor([[1.0, 0.0, -1.0, 0.5, 2.0, -2.0]] * 2).expand(B, 2, V)
    q = torch.softmax(torch.tensor([0.0, 1.5, 0.0, -1.0, 0.3, 0.2]), 0).expand(B, 1, V)
    x = torch.multinomial(q[0, 0], B, replacement=True, generator=g).to(torch.int32)[:, None]
    got = S.bcast_serve_verify(on_gpu(logits), on_gpu(q), x.to(DEV), torch.rand(B, 1, generator=g).to(DEV),
                               torch.empty(B, V).exponential_(generator=g).to(DEV), torch.ones(B, device=DEV))
    first = torch.bincount(got[1][:, 0].cpu().long(), minlength=V).double() / B
    p = torch.softmax(logits[0, 0].double(), 0)
    assert bool(((first - p).abs() <= 5 * torch.sqrt(p * (1 - p) / B)).all())


# ------------------------------------------------------------------------------------------ streams, graphs, refusals
def all_three(ws=None, stream=None):
    """One call of each operator; returns their inputs' closure and outputs."""
    l = {k: on_gpu(v) for k, v in linear_case(51, 24, 256, 200, 3, 16, "bf16").items()}
    a = {k: on_gpu(v) for k, v in attn_case(52, 5, 2, 2, 4, 64, 300, 50, 16, "bf16").items()}
    v = {k: on_gpu(t) for k, t in verify_case(53, 4, 3, 999, "bf16").items()}

    def go(ws, stream=None, outs=None):
        outs = outs or (None, None, None, None)
        y = S.bcast_serve_linear(l["x"], l["weight"], **{k: l[k] for k in ("bias", "lora_a", "lora_b", "adapter", "scale")},
                                 out=outs[0], workspace=ws, stream=stream)
        o = S.bcast_serve_attn(a["q"], a["prefix_k"], a["prefix_v"], a["own_k"], a["own_v"], a["own_len"], page_table=a["page_table"],
                               out=outs[1], workspace=ws, stream=stream)
        c, t = S.bcast_serve_verify(*v.values(), accepted=outs[2], tokens=outs[3], workspace=ws, stream=stream)
        return y, o, c, t
    return go


def test_other_streams_and_shared_workspace():
    go = all_three()
    want = go(S.Workspace(DEV))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ws = S.Workspace(DEV)
    for how in (side, side.cuda_stream):
        got = go(ws, how)
        side.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, got))
    with torch.cuda.stream(side):
        got = go(ws)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    assert all(torch.equal(x, y) for x, y in zip(want, go(None)))
    S.bcast_serve_status(ws)


def test_workspace_contents_do_not_matter():
    go = all_three()
    want = go(S.Workspace(DEV))
    ws = S.Workspace(DEV, 1 << 24)
    ws.reserve(1 << 24)[S.BCAST_SERVE_STATUS_BYTES:] = 0xff
    assert all(torch.equal(x, y) for x, y in zip(want, go(ws)))


def test_captured_into_a_graph():
    go = all_three()
    ws = S.Workspace(DEV, 1 << 24)
    want = go(ws)
    outs = tuple(torch.zeros_like(t) for t in want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(ws, outs=outs)
    for _ in range(2):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, outs))


def test_status_word():
    ws = S.Workspace(DEV)
    S.bcast_serve_status(ws)
    ws.reserve(256)[0] = 1
    with pytest.raises(BcastError) as e:
        S.bcast_serve_status(ws)
    assert e.value.code == -5
    S.bcast_serve_status(ws)


def refused(code, call):
    with pytest.raises(BcastError) as e:
        call()
    assert e.value.code == code


def test_linear_refusals():
    def go(change=None, **more):
        d = {k: on_gpu(v) for k, v in linear_case(61, 6, 64, 40, 2, 8, "bf16").items()}
        d.update(change or {})
        return S.bcast_serve_linear(d.pop("x"), d.pop("weight"), **d, **more)
    go()
    bf = dict(dtype=torch.bfloat16, device=DEV)
    for change in (dict(x=torch.zeros(6, 72, **bf)), dict(x=torch.zeros(6, 64, device=DEV)), dict(x=torch.zeros(6, 64, dtype=torch.bfloat16)),
                   dict(x=torch.zeros(64, 6, **bf).t()), dict(x=torch.zeros(6, 65, **bf)[:, 1:]), dict(x=torch.zeros(6 * 64 + 1, **bf)[1:].view(6, 64)),
                   dict(weight=torch.zeros(40, 68, **bf)[:, :64]), dict(bias=torch.zeros(41, **bf)), dict(adapter=torch.zeros(6, dtype=torch.int64, device=DEV)),
                   dict(scale=torch.zeros(2, dtype=torch.float64, device=DEV)), dict(lora_b=None), dict(lora_a=None),
                   dict(lora_a=torch.zeros(2, 12, 64, **bf), lora_b=torch.zeros(2, 40, 12, **bf)),
                   dict(lora_a=torch.zeros(2, 136, 64, **bf), lora_b=torch.zeros(2, 40, 136, **bf)),
                   dict(x=torch.zeros(6, 60, **bf), weight=torch.zeros(40, 60, **bf), lora_a=torch.zeros(2, 8, 60, **bf))):
        refused(BCAST_ERR_INVAL, lambda: go(change))
    refused(BCAST_ERR_INVAL, lambda: go(out=torch.zeros(6, 41, **bf)))
    refused(BCAST_ERR_INVAL, lambda: go(out=torch.zeros(1, 40, **bf).expand(6, 40)))
    small = S.Workspace(DEV)
    small._t = torch.zeros(256, dtype=torch.uint8, device=DEV)
    small.reserve = lambda *_: small._t
    refused(BCAST_ERR_CAPACITY, lambda: go(workspace=small))


def test_attn_refusals():
    def go(**change):
        d = {k: on_gpu(v) for k, v in attn_case(62, 2, 1, 2, 2, 64, 30, 20, 4, "fp16").items()}
        more = {k: change.pop(k) for k in ("out", "lse", "scale") if k in change}
        d.update(change)
        return S.bcast_serve_attn(d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"], page_table=d["page_table"], **more)
    go()
    h = dict(dtype=torch.float16, device=DEV)
    for change in (dict(q=torch.zeros(2, 1, 3, 64, **h)), dict(q=torch.zeros(2, 1, 4, 72, **h)), dict(q=torch.zeros(2, 1, 4, 64, device=DEV)),
                   dict(prefix_v=torch.zeros(31, 2, 64, **h)), dict(own_v=torch.zeros(12, 5, 2, 64, **h)), dict(own_len=torch.zeros(3, dtype=torch.int32, device=DEV)),
                   dict(own_len=torch.zeros(2, dtype=torch.int64, device=DEV)), dict(page_table=torch.zeros(3, 5, dtype=torch.int32, device=DEV)),
                   dict(prefix_k=torch.zeros(30, 2, 65, **h)[..., :64]), dict(prefix_k=torch.zeros(30 * 128 + 1, **h)[1:].view(30, 2, 64)),
                   dict(prefix_k=torch.zeros(30, 2, 64, dtype=torch.float16)), dict(scale=math.nan), dict(out=torch.zeros(2, 1, 4, 60, **h)),
                   dict(lse=torch.zeros(2, 1, 4, **h))):
        refused(BCAST_ERR_INVAL, lambda: go(**change))
    for D in (4, 12, 136, 256):
        def wide():
            d = {k: on_gpu(v) for k, v in attn_case(63, 2, 1, 2, 2, D, 30, 20, 4, "fp16").items()}
            return S.bcast_serve_attn(d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"], page_table=d["page_table"])
        refused(BCAST_ERR_INVAL, wide)


def test_verify_refusals():
    def go(**change):
        d = {k: on_gpu(v) for k, v in verify_case(64, 2, 3, 50, "fp32").items()}
        d.update(change)
        return S.bcast_serve_verify(*d.values())
    go()
    for change in (dict(logits=torch.zeros(2, 5, 50, device=DEV)), dict(logits=torch.zeros(2, 4, 50, dtype=torch.float64, device=DEV)),
                   dict(draft_probs=torch.zeros(2, 3, 50, dtype=torch.float16, device=DEV)), dict(draft_tokens=torch.zeros(2, 3, dtype=torch.int64, device=DEV)),
                   dict(uniforms=torch.zeros(3, 2, device=DEV).t()), dict(noise=torch.zeros(2, 50)), dict(temperature=torch.zeros(1, device=DEV)),
                   dict(noise=torch.zeros(50, 2, device=DEV).t())):
        refused(BCAST_ERR_INVAL, lambda: go(**change))
    refused(BCAST_ERR_INVAL, lambda: S.bcast_serve_verify(*(on_gpu(v) for v in verify_case(65, 1, 64, 9, "fp32").values())))
