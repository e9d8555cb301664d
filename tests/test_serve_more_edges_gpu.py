"""Replicas whose buffers a second broadcast fills, on the GPU."""
import pytest
import torch

from paper_1603_06809_b200 import replica as P
from test_serve_gpu import DEV

pytestmark = pytest.mark.gpu


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
