"""Replicas with 4-bit projections, normed and rotated heads, and log probabilities beside their answers."""
import math

import pytest
import torch

import serve_more_reference as R
import serve_reference as R0
from paper_1603_06809_b200 import replica as P
from paper_1603_06809_b200 import serve as S

SMALL = dict(hidden=128, q_heads=4, kv_heads=2, dim=64, vocab=500, adapters=3, rank=8, prompt=150, page=8)


@pytest.mark.parametrize("more", [dict(bits=4), dict(normed=True), dict(bits=4, normed=True, rotation=10000.0)])
def test_layouts_cover_the_message_without_overlap(more):
    layout = P.Layout(P.Shape(**SMALL, **more))
    buf = torch.zeros(layout.nbytes, dtype=torch.uint8)
    for i, v in enumerate(layout.views(buf).values()):
        v.view(torch.uint8).reshape(-1).fill_(i + 1)
        assert v.data_ptr() % 16 == buf.data_ptr() % 16 and v.is_contiguous()
    sizes = [math.prod(shape) * torch.empty(0, dtype=dtype).element_size() for _, shape, dtype in layout.at.values()]
    assert torch.bincount(buf.long())[1:].tolist() == sizes
    if more.get("bits") == 4:
        assert layout.at["w_out_codes"][1] == (500, 128) and layout.at["w_out_scales"][1] == (4, 2, 32, 4, 4) and "w_out" not in layout.at


@pytest.mark.parametrize("change", [dict(bits=8), dict(bits=4, hidden=120), dict(bits=4, q_heads=2, kv_heads=1, dim=8)])
def test_layouts_that_are_refused(change):
    with pytest.raises(ValueError):
        P.Layout(P.Shape(**{**SMALL, **change}))


def near(got, want, bound):
    assert bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.gpu
@pytest.mark.parametrize("more", [dict(bits=4), dict(normed=True), dict(rotation=10000.0), dict(bits=4, normed=True, rotation=10000.0, dtype=torch.float16)])
def test_a_step_against_the_plain_forms(more, monkeypatch):
    s = P.Shape(**SMALL, **more)
    layout = P.Layout(s)
    bufs = P.broadcast_model(P.random_model(s, layout, 8, "cuda:0"), 3)
    assert all(torch.equal(b, bufs[0]) for b in bufs)
    replicas = [P.Replica(s, layout, b, 6, 24) for b in bufs]
    rep, seen = replicas[1], {}
    for name in ("linear", "append", "attn", "linear4"):
        call = getattr(S, "bcast_serve_" + name)

        def kept(*a, _call=call, _name=name, **k):
            out = _call(*a, **k)
            seen.setdefault(_name, []).append(out)
            return out
        monkeypatch.setattr(S, "bcast_serve_" + name, kept)
    inputs = P.drafted(s, 6, 2, 20, "cuda:0")
    before = rep.own_k.cpu(), rep.own_v.cpu()
    accepted, tokens, (lp, entropy, ids, best) = rep.step(**inputs, top=4)
    monkeypatch.undo()
    w = {k: v.cpu() for k, v in rep.shared.items()}
    if s.bits == 4:
        codes, scales = w["w_qkv_codes"], w["w_qkv_scales"]
        r, c = torch.arange(s.qkv)[:, None], torch.arange(4)[None, :]
        plain = R.values(torch.stack([codes & 15, codes >> 4], dim=-1).flatten(1), scales[r // 128, c // 4, r % 32, r % 128 // 32, c % 4])
        assert torch.equal(plain.to(s.dtype), w["w_qkv"])
    qkv = seen["linear"][0].cpu()
    near(qkv, *R0.linear(inputs["x"].cpu().reshape(18, -1), w["w_qkv"], None, w["lora_a"], w["lora_b"], inputs["adapter"].cpu().repeat_interleave(3),
                         w["lora_scale"]))
    q, k, v = qkv.view(6, 3, 8, 64).split((4, 2, 2), dim=2)
    want = R.append(q, k, v, *before, torch.full((6,), 3), page_table=rep.table.cpu(), first=s.prompt, inv_freq=None if rep.inv_freq is None else rep.inv_freq.cpu(),
                    q_norm=w.get("q_norm"), k_norm=w.get("k_norm"))
    near(rep.own_k.cpu(), *want["own_k"])
    near(rep.own_v.cpu(), *want["own_v"])
    if s.normed or s.rotation:
        q = seen["append"][0].cpu()
        near(q, *want["q"])
    out, bound, _, _ = R0.attn(q, w["prompt_k"], w["prompt_v"], rep.own_k.cpu(), rep.own_v.cpu(), torch.full((6,), 3), rep.table.cpu())
    o = seen["attn"][0].cpu()
    near(o, out, bound)
    if s.bits == 4:
        codes, scales = w["w_out_codes"], w["w_out_scales"]
        r, c = torch.arange(500)[:, None], torch.arange(8)[None, :]
        logits = seen["linear4"][0].cpu()
        near(logits, *R.linear4(o.reshape(18, -1), torch.stack([codes & 15, codes >> 4], dim=-1).flatten(1), scales[r // 128, c // 4, r % 32, r % 128 // 32, c % 4]))
    else:
        logits = seen["linear"][1].cpu()
        near(logits, *R0.linear(o.reshape(18, -1), w["w_out"]))
    (want_lp, lp_bound), (h, h_bound), want_ids, (want_best, best_bound) = R.logprobs(logits, tokens.cpu().view(-1), 4)
    there = tokens.cpu().view(-1) >= 0
    near(lp.cpu().view(-1)[there], want_lp[there], lp_bound[there])
    assert bool(torch.isinf(lp.cpu().view(-1)[~there]).all())
    near(entropy.cpu().view(-1), h, h_bound)
    assert torch.equal(ids.cpu().view(18, 4), want_ids)
    near(best.cpu().view(18, 4), want_best, best_bound)
    # the other replicas answer alike, bit for bit
    for other in (replicas[0], replicas[2]):
        got = other.step(**inputs, top=4)
        assert torch.equal(got[0], accepted) and torch.equal(got[1], tokens) and all(torch.equal(x, y) for x, y in zip(got[2], (lp, entropy, ids, best)))
    for r in replicas:
        S.bcast_serve_status(r.workspace)


@pytest.mark.gpu
def test_a_step_that_neither_turns_nor_norms_stores_what_it_stored_before():
    s = P.Shape(**SMALL)
    layout = P.Layout(s)
    rep = P.Replica(s, layout, P.random_model(s, layout, 9, "cuda:0"), 5, 32)
    rep.length[:] = torch.tensor([0, 3, 7, 8, 20])
    before, length = rep.own_k.clone(), rep.length.clone()
    seen = []
    linear = S.bcast_serve_linear
    S.bcast_serve_linear = lambda *a, **k: seen.append(linear(*a, **k)) or seen[-1]
    try:
        rep.step(**P.drafted(s, 5, 3, 21, "cuda:0"))
    finally:
        S.bcast_serve_linear = linear
    k = seen[0].view(5, 4, 8, 64)[:, :, 4:6]
    at = length.long()[:, None] + torch.arange(4, device="cuda:0")
    before[rep.table.gather(1, at // 8).long(), at % 8] = k
    assert torch.equal(rep.own_k, before)


@pytest.mark.gpu
def test_steps_captured_into_a_graph():
    s = P.Shape(**SMALL, bits=4, normed=True, rotation=10000.0)
    layout = P.Layout(s)
    buf = P.random_model(s, layout, 11, "cuda:0")
    rep, twin = (P.Replica(s, layout, buf, 4, 64) for _ in range(2))
    inputs = P.drafted(s, 4, 2, 22, "cuda:0")
    for r in (rep, twin):
        r.step(**inputs, top=3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = rep.step(**inputs, top=3)
    for _ in range(3):
        graph.replay()
        want = twin.step(**inputs, top=3)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and all(torch.equal(x, y) for x, y in zip(got[2], want[2]))
    assert torch.equal(rep.own_k, twin.own_k) and torch.equal(rep.length, twin.length)


@pytest.mark.gpu
def test_command(capsys):
    out = P.main(["--ranks", "3", "--requests", "4", "--drafts", "2", "--prompt", "300", "--steps", "2", "--bits", "4", "--top", "5", "--normed", "--rotation", "10000"])
    assert out["replicas_agree"] and out["bits"] == 4 and out["us_per_step"] > 0
