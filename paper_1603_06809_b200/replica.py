"""A group of replicas that answer requests from what a broadcast put into their rank buffers.

The message of the broadcast is a model's weights, its low-rank adapters and the cache of a prompt that every
request starts with, one array after the other (:class:`Layout`).  After ``bcast_exec`` every rank's buffer
holds all of it, and a :class:`Replica` is a set of views into one of those buffers: nothing is copied out.
One :meth:`Replica.step` checks drafted tokens for a batch of requests with the three serving operators: the
shared projection with the requests' adapters, attention behind the shared prompt, the shared output projection,
and the acceptance of the drafts.  The model is one attention layer between the projections, with as many heads
and as wide as asked for; its weights are random.

    python -m paper_1603_06809_b200.replica [--ranks 4] [--requests 16] [--drafts 3] [--prompt 2048] [--steps 20]

runs the broadcast and one step on every replica, checks that the replicas agree, and prints the time of a step
as one JSON line.
"""
from __future__ import annotations

import argparse
import json
from dataclasses import dataclass

import torch

from . import bcast as B
from . import serve as S

ALIGN = 256           # bytes; rank buffers start on 16, the operators ask for 16


@dataclass(frozen=True)
class Shape:
    hidden: int = 512
    q_heads: int = 8
    kv_heads: int = 2
    dim: int = 64
    vocab: int = 4096
    adapters: int = 4
    rank: int = 16
    prompt: int = 2048
    page: int = 16
    dtype: torch.dtype = torch.bfloat16

    @property
    def qkv(self) -> int:
        return (self.q_heads + 2 * self.kv_heads) * self.dim


class Layout:
    """Where the arrays of a shape lie in the message: name -> (offset in bytes, shape, type)."""

    def __init__(self, s: Shape):
        self.at, self.nbytes = {}, 0
        for name, shape, dtype in (
                ("w_qkv", (s.qkv, s.hidden), s.dtype), ("lora_a", (s.adapters, s.rank, s.hidden), s.dtype),
                ("lora_b", (s.adapters, s.qkv, s.rank), s.dtype), ("lora_scale", (s.adapters,), torch.float32),
                ("w_out", (s.vocab, s.q_heads * s.dim), s.dtype), ("prompt_k", (s.prompt, s.kv_heads, s.dim), s.dtype),
                ("prompt_v", (s.prompt, s.kv_heads, s.dim), s.dtype)):
            self.at[name] = (self.nbytes, shape, dtype)
            n = torch.Size(shape).numel() * torch.empty(0, dtype=dtype).element_size()
            self.nbytes = -(-(self.nbytes + n) // ALIGN) * ALIGN

    def views(self, buf: torch.Tensor) -> dict:
        """The arrays inside one buffer of bytes."""
        out = {}
        for name, (at, shape, dtype) in self.at.items():
            n = torch.Size(shape).numel() * torch.empty(0, dtype=dtype).element_size()
            out[name] = buf[at:at + n].view(dtype).view(shape)
        return out


def random_model(s: Shape, layout: Layout, seed: int, device) -> torch.Tensor:
    """A message: random weights and a random prompt cache."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    buf = torch.zeros(layout.nbytes, dtype=torch.uint8, device=device)
    for name, v in layout.views(buf).items():
        if name == "lora_scale":
            v.fill_(1.0)
        else:
            std = 1.0 if name.startswith("prompt") else 0.5 * s.rank ** -0.5 if name == "lora_b" else v.shape[-1] ** -0.5
            v.copy_((torch.randn(v.shape, generator=g, device=device) * std).to(v.dtype))
    return buf


class Replica:
    """One rank: views into its buffer, the requests' own cache, and a workspace."""

    def __init__(self, s: Shape, layout: Layout, buf: torch.Tensor, requests: int, own_cap: int):
        self.s = s
        self.shared = layout.views(buf)
        each = -(-own_cap // s.page)
        pages = (requests * each, s.page, s.kv_heads, s.dim)
        self.own_k = torch.zeros(pages, dtype=s.dtype, device=buf.device)
        self.own_v = torch.zeros(pages, dtype=s.dtype, device=buf.device)
        self.table = torch.arange(requests * each, dtype=torch.int32, device=buf.device).reshape(requests, each)
        self.length = torch.zeros(requests, dtype=torch.int32, device=buf.device)
        self.cap, self.at_most = each * s.page, 0         # tokens of a request's cache; no length is above at_most
        self.workspace = S.Workspace(buf.device)

    def _make_room(self, n: int) -> None:
        # The lengths are on the GPU, which is waited for only when all drafts so far would have filled the cache.
        if self.at_most + n > self.cap:
            self.at_most = int(self.length.max()) if len(self.length) else 0
        if self.at_most + n > self.cap:
            raise ValueError(f"{n} new tokens: a request has {self.at_most} of its own already, and its cache holds {self.cap}")
        self.at_most += n

    def step(self, x, adapter, draft_probs, draft_tokens, uniforms, noise, temperature):
        """``x`` [requests, drafts + 1, hidden], the states of the last accepted token and of the drafts after it;
        ``adapter`` [requests] int32.  The tokens that are accepted stay in the cache, the others leave it.
        Returns (accepted, tokens) as ``bcast_serve_verify`` does; ``ValueError``, and nothing changed, where some
        request's cache has no room for all the new tokens."""
        s, w = self.s, self.shared
        R, n, _ = x.shape
        self._make_room(n)
        # the projection of all tokens at once, each with its request's adapter
        qkv = S.bcast_serve_linear(x.reshape(R * n, s.hidden), w["w_qkv"], lora_a=w["lora_a"], lora_b=w["lora_b"],
                                   adapter=adapter.repeat_interleave(n), scale=w["lora_scale"], workspace=self.workspace)
        qkv = qkv.view(R, n, s.q_heads + 2 * s.kv_heads, s.dim)
        q, k, v = qkv.split((s.q_heads, s.kv_heads, s.kv_heads), dim=2)
        # the new tokens' keys and values go behind the requests' own ones
        at = self.length.long()[:, None] + torch.arange(n, device=x.device)
        # (a graph that replays a step is not counted by _make_room: no index leaves the table there either)
        at.clamp_(max=self.cap - 1)
        page = self.table.gather(1, at // s.page).long()
        self.own_k[page, at % s.page] = k
        self.own_v[page, at % s.page] = v
        o = S.bcast_serve_attn(q, w["prompt_k"], w["prompt_v"], self.own_k, self.own_v, self.length + n, page_table=self.table,
                               workspace=self.workspace)
        logits = S.bcast_serve_linear(o.view(R * n, s.q_heads * s.dim), w["w_out"], workspace=self.workspace).view(R, n, s.vocab)
        accepted, tokens = S.bcast_serve_verify(logits, draft_probs, draft_tokens, uniforms, noise, temperature, workspace=self.workspace)
        self.length += accepted + 1
        return accepted, tokens


def broadcast_model(buf: torch.Tensor, ranks: int, root: int = 0, variant: int = B.BCAST_TUNED) -> torch.Tensor:
    """The message at every rank: [ranks, bytes], filled by the broadcast from ``root``."""
    bufs = torch.empty((ranks, buf.numel()), dtype=torch.uint8, device=buf.device)
    bufs[root].copy_(buf)
    plan = B.bcast_plan(ranks, root, buf.numel(), variant)
    B.bcast_exec([bufs[r] for r in range(ranks)], plan, torch.cuda.current_stream(buf.device))
    torch.cuda.current_stream(buf.device).synchronize()       # the plan's tables may go
    return bufs


def drafted(s: Shape, requests: int, drafts: int, seed: int, device):
    """Random inputs of one step: states, adapters, and drafts with their distributions and random numbers."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    rand = lambda *shape: torch.rand(shape, generator=g, device=device)  # noqa: E731
    probs = torch.softmax(torch.randn(requests, drafts, s.vocab, generator=g, device=device), -1)
    return dict(x=torch.randn(requests, drafts + 1, s.hidden, generator=g, device=device).to(s.dtype),
                adapter=torch.randint(-1, s.adapters, (requests,), generator=g, device=device, dtype=torch.int32),
                draft_probs=probs, draft_tokens=(probs / torch.empty_like(probs).exponential_(generator=g)).argmax(-1).to(torch.int32),
                uniforms=rand(requests, drafts), noise=torch.empty(requests, s.vocab, device=device).exponential_(generator=g),
                temperature=torch.where(rand(requests) < 0.25, 0.0, 0.8))


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--ranks", type=int, default=4)
    ap.add_argument("--requests", type=int, default=16, help="of each replica")
    ap.add_argument("--drafts", type=int, default=3)
    ap.add_argument("--prompt", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=20, help="timed steps")
    a = ap.parse_args(argv)
    dev = torch.device("cuda", torch.cuda.current_device())
    s = Shape(prompt=a.prompt)
    layout = Layout(s)
    bufs = broadcast_model(random_model(s, layout, 1, dev), a.ranks)
    cap = (a.steps + 4) * (a.drafts + 1)
    replicas = [Replica(s, layout, bufs[r], a.requests, cap) for r in range(a.ranks)]
    inputs = drafted(s, a.requests, a.drafts, 2, dev)
    first = [r.step(**inputs) for r in replicas]
    agree = all(torch.equal(x, y) for out in first for x, y in zip(out, first[0]))
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(3):
        replicas[0].step(**inputs)
    begin.record()
    for _ in range(a.steps):
        replicas[0].step(**inputs)
    end.record()
    torch.cuda.synchronize()
    for r in replicas:
        S.bcast_serve_status(r.workspace)
    out = dict(ranks=a.ranks, message_bytes=layout.nbytes, requests=a.requests, drafts=a.drafts, prompt=a.prompt, replicas_agree=agree,
               accepted=int(first[0][0].sum()), us_per_step=round(begin.elapsed_time(end) * 1e3 / a.steps, 1))
    print(json.dumps(out))
    return out


if __name__ == "__main__":
    main()
