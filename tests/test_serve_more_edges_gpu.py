"""Edges of log probabilities and of replicas on the GPU: results that stand by themselves, log probabilities at their upper end, buffers
that a second broadcast fills."""
import io

import pytest
import torch

from paper_1603_06809_b200 import replica as P
from paper_1603_06809_b200 import serve as S
from test_serve_gpu import DEV, TYPES, gen, rand

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------ results that stand by themselves
@pytest.mark.parametrize("T", [1, 7])
@pytest.mark.parametrize("top", [0, 1, 20])
def test_logprobs_results_are_kept_and_saved_each_by_itself(T, top):
    g = gen(T + top)
    out = S.bcast_serve_logprobs(rand(g, T, 500).to(DEV), torch.arange(T, dtype=torch.int32, device=DEV), top=top)
    # a result holds no more memory than its own, and writing to one changes no other
    assert [t.untyped_storage().nbytes() for t in out] == [4 * t.numel() for t in out]
    want = [t.clone() for t in out]
    for i, t in enumerate(out):
        t.zero_()
        assert all(torch.equal(a, b) for a, b in zip(out[i + 1:], want[i + 1:]))
        t.copy_(want[i])
    file = io.BytesIO()
    torch.save(out, file)
    file.seek(0)
    assert all(torch.equal(a, b) and a.dtype == b.dtype for a, b in zip(torch.load(file), want))


# ------------------------------------------------------------------------------------------ log probabilities at their upper end
@pytest.mark.parametrize("T,V", [(600, 300), (3000, 2000), (500, 20000), (3, 70001)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_logprobs_are_never_above_zero(T, V, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(T + V)
    # one token that has all of the probability, wherever it is and whatever its logit
    l = torch.randn(T, V, generator=g, device=DEV)
    best = torch.randint(0, V, (T, 1), generator=g, device=DEV)
    l.scatter_(1, best, torch.rand(T, 1, generator=g, device=DEV) * 400 + 25)
    l[::3].clamp_(min=0.0).mul_(50.0)
    x = best[:, 0].to(torch.int32)
    lp, h, ids, top = S.bcast_serve_logprobs(l.to(TYPES[dtype]), x, top=3)
    assert bool((lp <= 0).all()) and bool((top <= 0).all()) and bool((h >= 0).all())
    assert bool((lp > -1e-3).any()) and torch.equal(torch.exp(lp) <= 1, torch.ones_like(lp, dtype=torch.bool))


# ------------------------------------------------------------------------------------------ buffers that are filled again
SMALL = dict(hidden=128, q_heads=4, kv_heads=2, dim=64, vocab=500, adapters=3, rank=8, prompt=150, page=8)


@pytest.mark.parametrize("more", [dict(), dict(bits=4), dict(bits=4, normed=True, rotation=10000.0)])
def test_a_replica_answers_from_what_its_buffer_holds_now(more):
    s = P.Shape(**SMALL, **more)
    layout = P.Layout(s)
    old, new = (P.random_model(s, layout, seed, DEV) for seed in (31, 32))
    inputs = P.drafted(s, 5, 2, 33, DEV)
    want = P._flat(P.Replica(s, layout, new, 5, 24).step(**inputs, top=3))
    buf = old.clone()
    rep = P.Replica(s, layout, buf, 5, 24)
    buf.copy_(new)                                            # as a second broadcast does
    got = P._flat(rep.step(**inputs, top=3))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("more", [dict(), dict(bits=4)])
def test_a_captured_step_answers_from_what_its_buffer_holds_now(more):
    s = P.Shape(**SMALL, **more)
    layout = P.Layout(s)
    old, new = (P.random_model(s, layout, seed, DEV) for seed in (34, 35))
    inputs = P.drafted(s, 4, 2, 36, DEV)
    want = [P._flat(P.Replica(s, layout, m, 4, 64).step(**inputs, top=3)) for m in (old, new)]
    assert not torch.equal(want[0][2], want[1][2])
    buf = old.clone()
    rep = P.Replica(s, layout, buf, 4, 64)
    rep.step(**inputs, top=3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = P._flat(rep.step(**inputs, top=3))
    for i, m in ((0, old), (1, new), (0, old)):
        buf.copy_(m)
        rep.length.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
