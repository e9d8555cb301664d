"""Replicas that answer from their rank buffers: the message's layout, and whole steps after a broadcast."""
import math

import pytest
import torch

import serve_reference as R
from paper_1603_06809_b200 import replica as P
from paper_1603_06809_b200 import serve as S

SMALL = dict(hidden=128, q_heads=4, kv_heads=2, dim=64, vocab=500, adapters=3, rank=8, prompt=150, page=8)


def test_layout_covers_the_message_without_overlap():
    layout = P.Layout(P.Shape(**SMALL))
    buf = torch.zeros(layout.nbytes, dtype=torch.uint8)
    for i, v in enumerate(layout.views(buf).values()):
        v.view(torch.uint8).reshape(-1).fill_(i + 1)
        assert v.data_ptr() % 16 == buf.data_ptr() % 16 and v.is_contiguous()
    sizes = [math.prod(shape) * torch.empty(0, dtype=dtype).element_size() for _, shape, dtype in layout.at.values()]
    assert torch.bincount(buf.long())[1:].tolist() == sizes


@pytest.mark.gpu
@pytest.mark.parametrize("ranks,requests,drafts", [(1, 1, 0), (3, 5, 2), (8, 20, 4)])
def test_steps_after_a_broadcast(ranks, requests, drafts):
    s = P.Shape(**SMALL)
    layout = P.Layout(s)
    message = P.random_model(s, layout, 7, "cuda:0")
    bufs = P.broadcast_model(message, ranks, root=ranks - 1)
    assert all(torch.equal(b, message) for b in bufs)
    replicas = [P.Replica(s, layout, b, requests, 40) for b in bufs]
    for step in range(3):
        inputs = P.drafted(s, requests, drafts, 10 + step, "cuda:0")
        before = replicas[0].length.clone()
        outs = [r.step(**inputs) for r in replicas]
        assert all(torch.equal(x, y) for o in outs for x, y in zip(o, outs[0]))
        assert torch.equal(replicas[0].length, before + outs[0][0] + 1)
        assert bool((outs[0][1].gather(1, outs[0][0].long()[:, None]) >= 0).all())
    for r in replicas:
        S.bcast_serve_status(r.workspace)


@pytest.mark.gpu
def test_a_step_against_the_plain_forms():
    s = P.Shape(**SMALL)
    layout = P.Layout(s)
    buf = P.broadcast_model(P.random_model(s, layout, 8, "cuda:0"), 4)[2]
    rep = P.Replica(s, layout, buf, 6, 24)
    seen = []
    linear, attn = S.bcast_serve_linear, S.bcast_serve_attn
    S.bcast_serve_linear = lambda *a, **k: seen.append(linear(*a, **k)) or seen[-1]
    S.bcast_serve_attn = lambda *a, **k: seen.append(attn(*a, **k)) or seen[-1]
    try:
        inputs = P.drafted(s, 6, 2, 20, "cuda:0")
        rep.step(**inputs)
    finally:
        S.bcast_serve_linear, S.bcast_serve_attn = linear, attn
    qkv, o, logits = (t.cpu() for t in seen)
    w = {k: v.cpu() for k, v in layout.views(buf).items()}

    def near(got, want, bound):
        assert bool(((got.double() - want).abs() <= bound).all())
    near(qkv, *R.linear(inputs["x"].cpu().reshape(18, -1), w["w_qkv"], None, w["lora_a"], w["lora_b"],
                        inputs["adapter"].cpu().repeat_interleave(3), w["lora_scale"]))
    q, k, v = qkv.view(6, 3, 8, 64).split((4, 2, 2), dim=2)
    want, bound, _, _ = R.attn(q, w["prompt_k"], w["prompt_v"], k, v, torch.full((6,), 3))
    near(o, want, bound)
    near(logits, *R.linear(o.reshape(18, -1), w["w_out"]))


@pytest.mark.gpu
def test_command(capsys):
    out = P.main(["--ranks", "3", "--requests", "4", "--drafts", "2", "--prompt", "300", "--steps", "2"])
    assert out["replicas_agree"] and out["us_per_step"] > 0
    assert '"replicas_agree": true' in capsys.readouterr().out
