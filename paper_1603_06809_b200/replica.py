"""A group of replicas that answer requests from what a broadcast put into their rank buffers.

The message of the broadcast is a model's weights, its low-rank adapters and the cache of a prompt that every
request starts with, one array after the other (:class:`Layout`).  After ``bcast_exec`` every rank's buffer
holds all of it, and a :class:`Replica` is a set of views into one of those buffers: a step answers from what the
buffer holds when it runs, also after another broadcast into it.
One :meth:`Replica.step` checks drafted tokens for a batch of requests with the serving operators: the
shared projection with the requests' adapters, the new tokens' norms, rotation and places in the cache, attention
behind the shared prompt, the shared output projection, the acceptance of the drafts, and, if asked for, the log
probabilities of what is answered.  The model is one attention layer between the projections, with as many heads
and as wide as asked for; its weights are random.  With ``Shape.bits`` 4 the projections travel in microscaled 4-bit
numbers: the output projection is used as it came, the first one, which takes adapters, is unpacked by every step into
memory that the replica keeps for it.

    python -m paper_1603_06809_b200.replica [--ranks 4] [--requests 16] [--drafts 3] [--prompt 2048] [--steps 20] [--bits 4] [--top 5]

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
    bits: int = 16                    # of the projections' weights in the message: 16, or 4
    rotation: float = 0.0             # base of the positions' rotation; 0: none
    normed: bool = False              # queries and keys of each head

    @property
    def qkv(self) -> int:
        return (self.q_heads + 2 * self.kv_heads) * self.dim


class Layout:
    """Where the arrays of a shape lie in the message: name -> (offset in bytes, shape, type)."""

    def __init__(self, s: Shape):
        self.at, self.nbytes = {}, 0

        def weight(name, n, k):
            if s.bits == 16:
                return [(name, (n, k), s.dtype)]
            return [(name + "_codes", (n, k // 2), torch.uint8), (name + "_scales", (-(-n // 128), -(-k // 128), 32, 4, 4), torch.uint8)]
        if s.bits not in (4, 16):
            raise ValueError(f"bits {s.bits}: 4 or 16")
        if s.bits == 4 and (s.hidden % 32 or s.q_heads * s.dim % 32):
            raise ValueError("4-bit weights: hidden and q_heads * dim are multiples of 32")
        for name, shape, dtype in (
                *weight("w_qkv", s.qkv, s.hidden), ("lora_a", (s.adapters, s.rank, s.hidden), s.dtype),
                ("lora_b", (s.adapters, s.qkv, s.rank), s.dtype), ("lora_scale", (s.adapters,), torch.float32),
                *weight("w_out", s.vocab, s.q_heads * s.dim), ("prompt_k", (s.prompt, s.kv_heads, s.dim), s.dtype),
                ("prompt_v", (s.prompt, s.kv_heads, s.dim), s.dtype),
                *((("q_norm", (s.dim,), s.dtype), ("k_norm", (s.dim,), s.dtype)) if s.normed else ())):
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
    views = layout.views(buf)
    for name, v in views.items():
        if name == "lora_scale":
            v.fill_(1.0)
        elif name.endswith("_norm"):
            v.copy_((torch.rand(v.shape, generator=g, device=device) + 0.5).to(v.dtype))
        elif name.endswith("_codes"):
            w = torch.randn((v.shape[0], 2 * v.shape[1]), generator=g, device=device) * (2 * v.shape[1]) ** -0.5
            S.bcast_serve_pack4(w, codes=v, scales=views[name[:-6] + "_scales"])
        elif not name.endswith("_scales"):
            std = 1.0 if name.startswith("prompt") else 0.5 * s.rank ** -0.5 if name == "lora_b" else v.shape[-1] ** -0.5
            v.copy_((torch.randn(v.shape, generator=g, device=device) * std).to(v.dtype))
    return buf


class Replica:
    """One rank: views into its buffer, the requests' own cache, and a workspace; with 4-bit weights also room for the first
    projection's in 16 bits."""

    def __init__(self, s: Shape, layout: Layout, buf: torch.Tensor, requests: int, own_cap: int):
        self.s = s
        self.shared = layout.views(buf)
        if s.bits == 4:                                   # its adapters are in 16 bits, and so is its product
            self.shared["w_qkv"] = torch.empty((s.qkv, s.hidden), dtype=s.dtype, device=buf.device)
            self._unpack()
        self.inv_freq = None
        if s.rotation:
            pairs = torch.arange(s.dim // 16 * 8, device=buf.device, dtype=torch.float64)
            self.inv_freq = (s.rotation ** -(pairs / max(len(pairs), 1))).float()
        each = -(-own_cap // s.page)
        pages = (requests * each, s.page, s.kv_heads, s.dim)
        self.own_k = torch.zeros(pages, dtype=s.dtype, device=buf.device)
        self.own_v = torch.zeros(pages, dtype=s.dtype, device=buf.device)
        self.table = torch.arange(requests * each, dtype=torch.int32, device=buf.device).reshape(requests, each)
        self.length = torch.zeros(requests, dtype=torch.int32, device=buf.device)
        self.cap, self.at_most = each * s.page, 0         # tokens of a request's cache; no length is above at_most
        self.workspace = S.Workspace(buf.device)

    def _unpack(self) -> None:
        # the first projection in 16 bits, as the buffer has it now: a broadcast may have filled it again
        w = self.shared
        S.bcast_serve_unpack4(w["w_qkv_codes"], w["w_qkv_scales"], self.s.dtype, out=w["w_qkv"])

    def _make_room(self, n: int) -> None:
        # The lengths are on the GPU, which is waited for only when all drafts so far would have filled the cache.
        if self.at_most + n > self.cap:
            self.at_most = int(self.length.max()) if len(self.length) else 0
        if self.at_most + n > self.cap:
            raise ValueError(f"{n} new tokens: a request has {self.at_most} of its own already, and its cache holds {self.cap}")
        self.at_most += n

    def step(self, x, adapter, draft_probs, draft_tokens, uniforms, noise, temperature, top=None):
        """``x`` [requests, drafts + 1, hidden], the states of the last accepted token and of the drafts after it;
        ``adapter`` [requests] int32.  The tokens that are accepted stay in the cache, the others leave it.
        Returns (accepted, tokens) as ``bcast_serve_verify`` does, and with ``top`` also (log probabilities of the tokens,
        entropy, the ``top`` most probable tokens, theirs), each [requests, drafts + 1, ...]: tokens that are not there (-1) have
        -infinity.  ``ValueError``, and nothing changed, where some request's cache has no room for all the new tokens."""
        s, w = self.s, self.shared
        R, n, _ = x.shape
        self._make_room(n)
        if s.bits == 4:
            self._unpack()
        # the projection of all tokens at once, each with its request's adapter
        qkv = S.bcast_serve_linear(x.reshape(R * n, s.hidden), w["w_qkv"], lora_a=w["lora_a"], lora_b=w["lora_b"],
                                   adapter=adapter.repeat_interleave(n), scale=w["lora_scale"], workspace=self.workspace)
        qkv = qkv.view(R, n, s.q_heads + 2 * s.kv_heads, s.dim)
        q, k, v = qkv.split((s.q_heads, s.kv_heads, s.kv_heads), dim=2)
        # the new tokens' keys and values go behind the requests' own ones.  (A graph that replays a step is not counted by
        # _make_room: a token that has no room then is not stored.)
        length = self.length + n
        turned = s.normed or s.rotation
        out = S.bcast_serve_append(q if turned else None, k, v, self.own_k, self.own_v, length, page_table=self.table, first=s.prompt,
                                   inv_freq=self.inv_freq, q_norm=w.get("q_norm"), k_norm=w.get("k_norm"))
        q = out if turned else q
        o = S.bcast_serve_attn(q, w["prompt_k"], w["prompt_v"], self.own_k, self.own_v, length, page_table=self.table, workspace=self.workspace)
        o = o.view(R * n, s.q_heads * s.dim)
        if s.bits == 4:
            logits = S.bcast_serve_linear4(o, w["w_out_codes"], w["w_out_scales"], workspace=self.workspace)
        else:
            logits = S.bcast_serve_linear(o, w["w_out"], workspace=self.workspace)
        accepted, tokens = S.bcast_serve_verify(logits.view(R, n, s.vocab), draft_probs, draft_tokens, uniforms, noise, temperature,
                                                workspace=self.workspace)
        self.length += accepted + 1
        if top is None:
            return accepted, tokens
        lp, entropy, ids, best = S.bcast_serve_logprobs(logits, tokens.view(-1), top=top)
        return accepted, tokens, (lp.view(R, n), entropy.view(R, n), ids.view(R, n, top), best.view(R, n, top))


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


def _flat(out):
    return [t for x in out for t in (x if isinstance(x, tuple) else (x,))]


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--ranks", type=int, default=4)
    ap.add_argument("--requests", type=int, default=16, help="of each replica")
    ap.add_argument("--drafts", type=int, default=3)
    ap.add_argument("--prompt", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=20, help="timed steps")
    ap.add_argument("--bits", type=int, default=16, choices=(4, 16), help="of the projections' weights")
    ap.add_argument("--top", type=int, default=None, help="answer with log probabilities and this many alternatives")
    ap.add_argument("--rotation", type=float, default=0.0, help="base of the positions' rotation, 0 for none")
    ap.add_argument("--normed", action="store_true", help="norm queries and keys")
    a = ap.parse_args(argv)
    dev = torch.device("cuda", torch.cuda.current_device())
    s = Shape(prompt=a.prompt, bits=a.bits, rotation=a.rotation, normed=a.normed)
    layout = Layout(s)
    bufs = broadcast_model(random_model(s, layout, 1, dev), a.ranks)
    cap = (a.steps + 4) * (a.drafts + 1)
    replicas = [Replica(s, layout, bufs[r], a.requests, cap) for r in range(a.ranks)]
    inputs = dict(drafted(s, a.requests, a.drafts, 2, dev), top=a.top)
    first = [r.step(**inputs) for r in replicas]
    agree = all(torch.equal(x, y) for out in first for x, y in zip(_flat(out), _flat(first[0])))
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
    out = dict(ranks=a.ranks, message_bytes=layout.nbytes, requests=a.requests, drafts=a.drafts, prompt=a.prompt, bits=a.bits, replicas_agree=agree,
               accepted=int(first[0][0].sum()), us_per_step=round(begin.elapsed_time(end) * 1e3 / a.steps, 1))
    print(json.dumps(out))
    return out


if __name__ == "__main__":
    main()
