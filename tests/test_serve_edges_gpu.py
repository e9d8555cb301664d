"""Arguments and arrays at the edge of what the serving operators take, against the plain 64-bit forms."""
import math
import os
import subprocess
import sys

import pytest
import torch

import serve_reference as R
from helpers import ROOT
from paper_1603_06809_b200 import replica as P
from paper_1603_06809_b200 import serve as S
from paper_1603_06809_b200.bcast import BCAST_ERR_CAPACITY, BCAST_ERR_TIMEOUT, BcastError
from test_serve_gpu import attn_case, check_linear, check_verify, inside, linear_case, on_gpu, verify_case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# ------------------------------------------------------------------------------------------ verify: temperatures
@pytest.mark.parametrize("B,n,V", [(1, 0, 40), (3, 4, 7), (4, 3, 2048), (9, 2, 5003), (2, 3, 33333)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t", [math.inf, 3e38, 1e30])
def test_verify_temperatures_without_end(B, n, V, dtype, t):
    # logits / temperature goes to zero: every token is as likely as any other
    c = verify_case(B + n + V, B, n, V, dtype)
    c["temperature"][:] = t
    if n:
        c["draft_probs"][:, 0] = 0.5 / V                      # first drafts that some uniforms accept, and some would not
        c["uniforms"][:, 0] *= 4
    check_verify(c)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_verify_infinite_temperature_over_the_tokens_that_are_allowed(dtype):
    V = 1000
    c = verify_case(71, 6, 2, V, dtype)
    c["temperature"][:] = torch.tensor([math.inf, math.inf, math.inf, 0.7, 0.0, math.inf])
    c["logits"][0, :, 100:] = -math.inf                       # most tokens forbidden
    c["logits"][1, :, ::3] = math.nan                         # NaN counts as -infinity
    c["logits"][2, :, 5:] = torch.finfo(c["logits"].dtype).min    # the lowest number is a number: divided by infinity it is 0
    c["logits"][5] = -math.inf                                # no probabilities
    c["draft_probs"][:, :] = 1.0 / V
    c["uniforms"][:, 0] = 0.5
    c["uniforms"][0, 1] = 12.0
    # the limit of softmax(l / T): the same for every token that has a probability at all
    flat = dict(c, logits=c["logits"].clone(), temperature=c["temperature"].clone())
    for b in (0, 1, 2, 5):
        z = c["logits"][b]
        flat["logits"][b] = torch.where(z > -math.inf, torch.zeros_like(z), torch.full_like(z, -math.inf))
        flat["temperature"][b] = 1.0
    accepted, tokens, margin = R.verify(**flat)
    assert margin > 1e-5
    got = S.bcast_serve_verify(*(on_gpu(v) for v in c.values()))
    assert torch.equal(got[0].cpu(), accepted) and torch.equal(got[1].cpu(), tokens)
    assert got[1][5].tolist() == [-1, -1, -1]


def test_verify_temperatures_that_are_none():
    # zero, negative and NaN: the largest logit
    c = verify_case(72, 4, 3, 700, "bf16", greedy=True)
    c["draft_tokens"][:] = c["logits"][:, :3].float().argmax(-1).to(torch.int32)
    c["draft_tokens"][1, 2] ^= 1
    c["temperature"][:] = 0.0
    want = check_verify(c)
    c["temperature"][:] = torch.tensor([-1.0, math.nan, -math.inf, -0.0])
    got = S.bcast_serve_verify(*(on_gpu(v) for v in c.values()))
    assert all(torch.equal(x, y) for x, y in zip(want, got))


# ------------------------------------------------------------------------------------------ attn: keys that are NaN
def attn_on_gpu(c):
    """(out, lse) on the host."""
    d = {k: on_gpu(v) for k, v in c.items()}
    lse = torch.zeros(d["q"].shape[:3], device=DEV)
    out = S.bcast_serve_attn(d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"], page_table=d.get("page_table"), lse=lse)
    return out.cpu(), lse.cpu()


# few rows and a short prefix; tiles of 128 rows; pairs of them
@pytest.mark.parametrize("B,P,first", [(2, 300, 0), (2, 300, 292), (40, 1300, 0), (40, 1300, 32), (40, 1300, 700), (40, 1300, 1288),
                                       (256, 151700, 0), (256, 151700, 151688)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attn_prefix_key_that_is_nan_reaches_its_head_only(B, P, first, dtype):
    # head h has its NaN in key first + h: all places of eight
    H, G = 8, 1 if B > 100 else 4
    c = attn_case(91, B, 1, H, G, 64, P, 6, 0, dtype)
    clean, clean_lse = attn_on_gpu(c)
    assert bool(clean.isfinite().all())
    for h in range(0, H, 2):
        c["prefix_k"][first + h, h] = math.nan
    out, lse = attn_on_gpu(c)
    head = torch.arange(H).repeat_interleave(G)
    assert bool(out[:, :, head % 2 == 0].isnan().all()) and bool(lse[:, :, head % 2 == 0].isnan().all())
    assert torch.equal(out[:, :, head % 2 == 1], clean[:, :, head % 2 == 1]) and torch.equal(lse[:, :, head % 2 == 1], clean_lse[:, :, head % 2 == 1])
    for h in range(H):
        c["prefix_k"][first + h, h, 3] = math.nan
    out, lse = attn_on_gpu(c)
    assert bool(out.isnan().all()) and bool(lse.isnan().all())


@pytest.mark.parametrize("P", [0, 40, 3000])
def test_attn_own_key_that_is_nan_reaches_the_rows_that_see_it(P):
    c = attn_case(92, 12, 4, 2, 2, 64, P, 40, 16, "bf16", lengths=[4 + 3 * b for b in range(12)])
    clean, clean_lse = attn_on_gpu(c)
    for b, length in enumerate(c["own_len"].tolist()):
        at = length - 2                                       # the last new token but one: rows 2 and 3 see it
        c["own_k"][c["page_table"][b, at // 16], at % 16, 1] = math.nan
    out, lse = attn_on_gpu(c)
    assert bool(out[:, 2:, 2:].isnan().all()) and bool(lse[:, 2:, 2:].isnan().all())
    assert torch.equal(out[:, :2], clean[:, :2]) and torch.equal(out[:, :, :2], clean[:, :, :2])
    assert torch.equal(lse[:, :2], clean_lse[:, :2]) and torch.equal(lse[:, :, :2], clean_lse[:, :, :2])


@pytest.mark.parametrize("tiles", range(1, 10))
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attn_every_number_of_tiles_to_a_block(tiles, dtype):
    # 192 blocks of 128 rows with the whole prefix each: the two halves of a block take every other tile of tokens
    B, H, D = 300, 64, 128
    c = attn_case(93 + tiles, B, 1, H, 1, D, 128 * tiles - 5, 3, 0, dtype)
    out, lse = attn_on_gpu(c)
    rows = [0, 127, 128, B - 1]
    want, bound, wl, wb = R.attn(**{k: v if k.startswith("prefix") else v[rows] for k, v in c.items()})
    inside(out[rows], want, bound, "out")
    assert bool(((lse[rows].double() - wl).abs() <= wb).all())
    for _ in range(5):
        assert torch.equal(attn_on_gpu(c)[0], out)


# ------------------------------------------------------------------------------------------ linear: tiles without adapters
@pytest.mark.parametrize("which", ["none", "even", "odd", "one"])
@pytest.mark.parametrize("rank", [16, 128])
def test_linear_blocks_that_go_from_tiles_with_adapters_to_tiles_without(which, rank):
    # blocks that take several tiles of 256 tokens, in some of which no token has an adapter
    T, K, N, L = 1300, 72, 19000, 6
    assert -(-T // 256) * -(-N // 128) >= 3 * 148
    c = linear_case(98, T, K, N, L, rank, "bf16", how="mixed")
    tile = torch.arange(T) // 256
    has = {"none": tile < 0, "even": tile % 2 == 0, "odd": tile % 2 == 1, "one": tile == 3}[which]
    c["adapter"][~has] = -1
    first = check_linear(c)
    for _ in range(10):
        assert torch.equal(check_linear_again(c), first)


def check_linear_again(c):
    d = {k: on_gpu(v) for k, v in c.items()}
    return S.bcast_serve_linear(d.pop("x"), d.pop("weight"), **d)


# ------------------------------------------------------------------------------------------ workspaces
def timed_out(ws, stream=None):
    with pytest.raises(BcastError) as e:
        S.bcast_serve_status(ws, stream)
    assert e.value.code == BCAST_ERR_TIMEOUT


def test_status_stays_when_the_workspace_grows():
    ws = S.Workspace(DEV)
    ws.reserve(1000)[0] = 1                                   # as a kernel that gave up leaves it
    assert ws.reserve(1 << 20).numel() >= 1 << 20
    timed_out(ws)
    S.bcast_serve_status(ws)                                  # told once
    ws.reserve(1 << 20)[0] = 1
    c = attn_case(95, 40, 4, 2, 4, 128, 3000, 20, 16, "bf16")
    d = {k: on_gpu(v) for k, v in c.items()}
    size = ws.reserve(0).numel()
    S.bcast_serve_attn(d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"], page_table=d["page_table"], workspace=ws)
    assert ws.reserve(0).numel() > size                       # a call that needed more
    timed_out(ws)
    side = torch.cuda.Stream()
    ws.reserve(0)[0] = 1
    side.wait_stream(torch.cuda.current_stream())
    ws.reserve(ws.reserve(0).numel() + 1, side)
    timed_out(ws, side)


def attn_calls():
    """A call that needs little workspace and one that needs much more; each takes workspace and out."""
    def call(c):
        d = {k: on_gpu(v) for k, v in c.items()}
        return lambda ws, **more: S.bcast_serve_attn(d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"],
                                                     page_table=d["page_table"], workspace=ws, **more)
    return call(attn_case(96, 5, 2, 2, 4, 64, 300, 50, 16, "bf16")), call(attn_case(97, 40, 4, 2, 4, 128, 3000, 20, 16, "bf16"))


@pytest.mark.parametrize("named", [False, True])
def test_graph_keeps_its_memory_when_the_workspace_grows(named):
    small, large = attn_calls()
    ws, side = S.Workspace(DEV), torch.cuda.Stream()
    want, more = small(ws), large(S.Workspace(DEV))
    out = torch.zeros_like(want)
    was = ws.reserve(0)
    at, size = was.data_ptr(), was.numel()
    del was
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        small(ws, out=out, **(dict(stream=side) if named else {}))
    assert torch.equal(large(ws), more)
    assert ws.reserve(0).data_ptr() != at
    # whoever asks for memory of that size now does not get what the graph writes to
    others = [torch.full((size,), 7, dtype=torch.uint8, device=DEV) for _ in range(3)]
    assert all(t.data_ptr() != at for t in others)
    for _ in range(2):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want) and torch.equal(large(ws), more)
    assert all(bool((t == 7).all()) for t in others)
    S.bcast_serve_status(ws)
    ws._kept[0][0] = 1                                        # a replay that gave up
    timed_out(ws)
    S.bcast_serve_status(ws)
    graph.reset()


def test_workspace_does_not_grow_in_a_capture():
    small, large = attn_calls()
    want = small(None)
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    for ws in (S.Workspace(DEV), S.Workspace(DEV, 1000)):
        held, call = ws._t, small if ws._t is None else large
        graph = torch.cuda.CUDAGraph()
        with pytest.raises(BcastError) as e:
            with torch.cuda.graph(graph):
                call(ws)
        assert e.value.code == BCAST_ERR_CAPACITY and "before the capture" in str(e.value)
        graph.reset()
        assert ws._t is held                                  # as it was, and of use
        torch.cuda.synchronize()
        assert torch.equal(small(ws), want)
        S.bcast_serve_status(ws)
    # without a workspace the call's memory is the graph's
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        small(None, out=out)
    for _ in range(2):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want)
    graph.reset()


def test_calls_outside_a_capture_keep_nothing():
    small, large = attn_calls()
    ws = S.Workspace(DEV)
    small(ws)
    large(ws)
    assert ws._kept == [] and not ws._captured


def test_status_of_a_workspace_that_no_call_used():
    side = torch.cuda.Stream()
    for stream in (None, side, side.cuda_stream):
        ws = S.Workspace(DEV)
        S.bcast_serve_status(ws, stream)
        assert ws._t is None                                  # nothing was made on another stream than the one that is read
        small, _ = attn_calls()
        small(ws, stream=stream)
        S.bcast_serve_status(ws, stream)


@pytest.mark.parametrize("op", ["linear", "attn", "verify"])
@pytest.mark.parametrize("raw", [False, True])
def test_inputs_let_go_of_before_a_named_stream_is_done(op, raw):
    if op == "linear":
        c = linear_case(99, 300, 256, 200, 3, 16, "bf16")
        call = lambda d, **k: S.bcast_serve_linear(d["x"], d["weight"], **{n: d[n] for n in ("bias", "lora_a", "lora_b", "adapter", "scale")}, **k)  # noqa: E731
    elif op == "attn":
        c = attn_case(99, 40, 2, 2, 4, 64, 1300, 50, 16, "bf16")
        call = lambda d, **k: S.bcast_serve_attn(d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"],  # noqa: E731
                                                 page_table=d["page_table"], **k)
    else:
        c = verify_case(99, 6, 3, 2000, "bf16")
        call = lambda d, **k: S.bcast_serve_verify(*d.values(), **k)  # noqa: E731
    d = {k: on_gpu(v) for k, v in c.items()}
    want = call(d)
    ws, side = S.Workspace(DEV, 1 << 24), torch.cuda.Stream()
    torch.cuda.synchronize()
    copies = {k: v.clone() for k, v in d.items()}
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                         # the stream is busy for some milliseconds
    got = call(copies, workspace=ws, stream=side.cuda_stream if raw else side)
    del copies
    # memory of the copies' sizes, if it were free already
    others = [torch.zeros_like(v) for v in d.values() for _ in range(2)]
    torch.cuda.synchronize()
    for x, y in zip(want if op == "verify" else (want,), got if op == "verify" else (got,)):
        assert torch.equal(x, y)
    del others


# ------------------------------------------------------------------------------------------ replicas
def test_replica_steps_until_its_cache_is_full():
    s = P.Shape(hidden=128, q_heads=4, kv_heads=2, dim=64, vocab=500, adapters=3, rank=8, prompt=150, page=8)
    layout = P.Layout(s)
    rep = P.Replica(s, layout, P.random_model(s, layout, 7, DEV), 5, 40)
    steps = 0
    with pytest.raises(ValueError):
        while steps < 100:
            rep.step(**P.drafted(s, 5, 3, 30 + steps, DEV))
            steps += 1
    before = rep.length.clone()
    assert 40 - 4 < int(before.max()) <= 40 and steps >= 10     # at most four tokens of a request to a step
    with pytest.raises(ValueError):
        rep.step(**P.drafted(s, 5, 3, 99, DEV))
    assert torch.equal(rep.length, before)
    while int(rep.length.max()) < 40:
        rep.step(**P.drafted(s, 5, 0, 60, DEV))                 # one token each still fits
    with pytest.raises(ValueError):
        rep.step(**P.drafted(s, 5, 0, 60, DEV))
    S.bcast_serve_status(rep.workspace)


# ------------------------------------------------------------------------------------------ waits that run out
WAITS_CHILD = r"""
import sys
import torch
sys.path[:0] = [sys.argv[1], sys.argv[1] + "/tests"]
from paper_1603_06809_b200 import bcast as B, serve as S
from test_serve_gpu import attn_case, linear_case, on_gpu


def told(ws):
    try:
        S.bcast_serve_status(ws)
        return "ok"
    except B.BcastError as e:
        return str(e.code)


def linear(ws, *size, **more):
    d = {k: on_gpu(v) for k, v in linear_case(1, *size, **more).items()}
    return S.bcast_serve_linear(d.pop("x"), d.pop("weight"), workspace=ws, **d)


def attn(ws, *size):
    d = {k: on_gpu(v) for k, v in attn_case(2, *size).items()}
    return S.bcast_serve_attn(d["q"], d["prefix_k"], d["prefix_v"], d["own_k"], d["own_v"], d["own_len"], workspace=ws)


calls = [lambda ws: linear(ws, 24, 1024, 200, 3, 16, "bf16"), lambda ws: linear(ws, 100, 512, 300, 0, 0, "fp16"),
         lambda ws: linear(ws, 1300, 72, 19000, 6, 128, "bf16"), lambda ws: attn(ws, 40, 1, 2, 4, 64, 1300, 6, 0, "bf16"),
         lambda ws: attn(ws, 40, 1, 2, 4, 128, 1300, 6, 0, "fp16"), lambda ws: attn(ws, 256, 1, 8, 1, 64, 151700, 6, 0, "bf16")]
for i, call in enumerate(calls):
    ws = S.Workspace("cuda:0")
    call(ws)
    first = told(ws)
    print("CALL", i, first, told(ws))                           # the word was cleared by the read
torch.cuda.synchronize()
print("END")
"""


@pytest.mark.parametrize("given_up,want", [("1", str(BCAST_ERR_TIMEOUT)), ("0", "ok"), ("", "ok")])
def test_waits_that_run_out_end_the_kernel_and_are_told(given_up, want):
    # The kernels have given up from the start: what they still issue touches the block's own memory alone and is waited
    # for, they come to their end and tell of it.
    env = dict(os.environ)
    env.pop("BCAST_SERVE_GIVE_UP", None)
    if given_up:
        env["BCAST_SERVE_GIVE_UP"] = given_up
    out = subprocess.run([sys.executable, "-c", WAITS_CHILD, ROOT], env=env, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr[-2000:]
    assert out.stdout.split("\n") == [f"CALL {i} {want} ok" for i in range(6)] + ["END", ""], out.stdout
