"""The serving operators' measured cases, their plain forms and their definition in 64 bits.

A group of replicas that got the same bytes by a broadcast (a model's weights and the cache of a prompt
that every request starts with) answers requests.  Three operators are measured, each of which uses what is
shared once for all requests and adds what is a request's own:

  linear   y = x W^T + bias, the projection all tokens share, plus scale[a] * (x A[a]^T) B[a]^T with the low-rank
           adapter `a` of each token's request (-1: none)
  attn     attention of the newest tokens of every request over a prefix that all requests share, followed by the
           request's own tokens (in pages or in rows), the newest ones causal among themselves
  verify   acceptance of drafted tokens against the target's probabilities from given random numbers, and the token
           that follows the accepted ones: by the race argmax_i w_i / e_i with given exponential numbers e, where w
           is max(p - q, 0) after a rejection and p after the last drafted token; at temperature 0 by the largest logit

`own` selects between the plain form (elementary torch operations in 32 bits) and the library's kernels.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # one new token of one request with an adapter: the latency of a single call
        dict(name="linear_one", op="linear", tokens=1, requests=1, k=2048, n=2048, adapters=1, rank=16, bias=False, dtype="bf16"),
        # a decode step: one token of each of 64 requests, 32 adapters between them; bound by reading W and the adapters
        dict(name="linear_decode", op="linear", tokens=64, requests=64, k=4096, n=4096, adapters=32, rank=16, bias=False, dtype="bf16"),
        # a small mixed batch with ragged lengths and sizes that no tile divides
        dict(name="linear_ragged", op="linear", tokens=333, requests=9, k=2056, n=5003, adapters=5, rank=24, bias=True, dtype="fp16"),
        # prompts being read: 8192 tokens of 16 requests; bound by the matrix product
        dict(name="linear_prompts", op="linear", tokens=8192, requests=16, k=4096, n=4096, adapters=8, rank=64, bias=True, dtype="bf16"),
        # one request, one token, a short shared prefix: the latency of a single call
        dict(name="attn_one", op="attn", batch=1, new=1, kv_heads=4, group=2, dim=64, prefix=509, own_max=60, page=0, dtype="bf16"),
        # a decode step of 32 requests behind a prefix of 8 Ki tokens, own tokens in pages of 16
        dict(name="attn_decode", op="attn", batch=32, new=1, kv_heads=8, group=4, dim=128, prefix=8192, own_max=700, page=16, dtype="bf16"),
        # drafts of four tokens being checked (five new ones each): odd prefix, a head size that fills no tile
        dict(name="attn_drafts", op="attn", batch=13, new=5, kv_heads=2, group=8, dim=96, prefix=20011, own_max=1300, page=64, dtype="fp16"),
        # drafts of three tokens on 64 requests behind a prefix of 64 Ki tokens: bound by the matrix products
        dict(name="attn_long", op="attn", batch=64, new=4, kv_heads=8, group=4, dim=128, prefix=65536, own_max=1024, page=16, dtype="bf16"),
        # one request with a draft of four, a small vocabulary in 32 bits: the latency of a single call
        dict(name="verify_one", op="verify", batch=1, new=4, vocab=32000, greedy=False, dtype="fp32"),
        # 24 requests, some of them greedy, with a vocabulary that no vector divides
        dict(name="verify_odd", op="verify", batch=24, new=5, vocab=50001, greedy=True, dtype="fp16"),
        # the largest: 128 requests with drafts of seven over a vocabulary of 128 Ki, bound by reading the logits
        dict(name="verify_wide", op="verify", batch=128, new=7, vocab=131072, greedy=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    op = rng.choice(["linear", "attn", "verify"])
    if op == "linear":
        while True:
            tokens = _log(rng, 1, 8192)
            k, n = 8 * _log(rng, 64, 1024), _log(rng, 512, 8192)
            if tokens * k * n <= 8192 * 4096 * 4096:
                break
        requests = tokens if tokens <= 256 and rng.random() < 0.5 else rng.randint(1, min(tokens, 32))
        return dict(op=op, tokens=tokens, requests=requests, k=k, n=n, adapters=_log(rng, 1, 32),
                    rank=rng.choice([8, 16, 24, 32, 64, 128]), bias=rng.random() < 0.5, dtype=rng.choice(["bf16", "fp16"]))
    if op == "attn":
        while True:
            c = dict(op=op, batch=_log(rng, 1, 64), new=rng.choice([1, 1, 1, 2, 4, 5, 8]), kv_heads=rng.choice([1, 2, 4, 8]),
                     group=rng.choice([1, 2, 4, 5, 8]), dim=rng.choice([64, 96, 128, 128]), prefix=_log(rng, 100, 65536),
                     own_max=_log(rng, 16, 2048), page=rng.choice([0, 16, 32, 64]), dtype=rng.choice(["bf16", "fp16"]))
            rows = c["batch"] * c["new"] * c["kv_heads"] * c["group"]
            if rows * (c["prefix"] + c["own_max"]) <= 64 * 4 * 32 * 65536:
                return c
    return dict(op=op, batch=_log(rng, 1, 128), new=rng.randint(1, 7), vocab=_log(rng, 2000, 131072), greedy=rng.random() < 0.3,
                dtype=rng.choice(["bf16", "fp16", "fp32"]))


# ------------------------------------------------------------------------------------------------- inputs
def _cut(total, parts, g):
    """`parts` lengths of at least 1 that sum to `total`."""
    if parts == 1:
        return [total]
    at = torch.randperm(total - 1, generator=g)[:parts - 1].sort().values + 1
    at = torch.cat([torch.zeros(1, dtype=torch.int64), at, torch.full((1,), total)])
    return (at[1:] - at[:-1]).tolist()


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    h = torch.Generator()
    h.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        out = torch.empty(shape, dtype=dtype, device=dev)
        return out.normal_(0.0, std, generator=g)

    if case["op"] == "linear":
        T, K, N, L, R = case["tokens"], case["k"], case["n"], case["adapters"], case["rank"]
        # requests take the adapters in turn, in an order of their own, now and then none
        of_request = torch.arange(case["requests"]) % L
        of_request[torch.rand(case["requests"], generator=h) < (0.1 if case["requests"] > 4 else 0.0)] = -1
        of_request = of_request[torch.randperm(case["requests"], generator=h)]
        adapter = torch.repeat_interleave(of_request, torch.tensor(_cut(T, case["requests"], h))).to(torch.int32)
        st = dict(x=normal(T, K), weight=normal(N, K, std=K ** -0.5), lora_a=normal(L, R, K, std=K ** -0.5),
                  lora_b=normal(L, N, R, std=0.3 * R ** -0.5), adapter=adapter.to(dev),
                  scale=torch.empty(L, device=dev).uniform_(0.5, 2.0, generator=g), bias=normal(N, std=0.1) if case["bias"] else None)
    elif case["op"] == "attn":
        B, n, H, G, D, S, page = (case[x] for x in ("batch", "new", "kv_heads", "group", "dim", "own_max", "page"))
        S = max(S, n)
        own_len = torch.randint(n, S + 1, (B,), generator=h, dtype=torch.int32)
        own_len[0] = S
        st = dict(q=normal(B, n, H * G, D), prefix_k=normal(case["prefix"], H, D), prefix_v=normal(case["prefix"], H, D))
        if page:
            each = -(-S // page)
            table = torch.randperm(B * each, generator=h).to(torch.int32).reshape(B, each)
            st.update(own_k=normal(B * each, page, H, D), own_v=normal(B * each, page, H, D), page_table=table.to(dev))
        else:
            st.update(own_k=normal(B, S, H, D), own_v=normal(B, S, H, D), page_table=None)
        st.update(own_len=own_len.to(dev), scale=D ** -0.5)
    else:
        B, n, V = case["batch"], case["new"], case["vocab"]
        logits = normal(B, n + 1, V, std=2.0, dtype=torch.float32)
        temperature = torch.empty(B, device=dev).uniform_(0.6, 1.2, generator=g)
        if case["greedy"]:
            temperature[::3] = 0.0
        # the draft is a nearby model: its distribution q, and tokens drawn from it
        t = torch.where(temperature > 0, temperature, 1.0)[:, None, None]
        q = torch.softmax((logits[:, :n] + normal(B, n, V, std=0.35, dtype=torch.float32)) / t, dim=-1)
        tokens = (q / torch.empty_like(q).exponential_(generator=g)).argmax(dim=-1)
        greedy = (temperature == 0)[:, None] & (torch.rand(B, n, generator=h) < 0.8).to(dev)
        logits = logits.to(dt)
        tokens = torch.where(greedy, logits[:, :n].float().argmax(dim=-1), tokens).to(torch.int32)
        st = dict(logits=logits, draft_probs=q, draft_tokens=tokens, temperature=temperature,
                  uniforms=torch.rand(B, n, device=dev, generator=g), noise=torch.empty(B, V, device=dev).exponential_(generator=g))
        st["noise"].clamp_(min=1e-10)
    st["op"] = case["op"]
    if own:
        from paper_1603_06809_b200 import serve
        st["workspace"] = serve.Workspace(dev)
    return st


# ------------------------------------------------------------------------------------------------- plain forms
def _plain_linear(s):
    x = s["x"].float()
    y = x @ s["weight"].float().t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    L, R, K = s["lora_a"].shape
    T = x.shape[0]
    a = s["adapter"].long()
    # all adapters' low-rank parts of all tokens, then those of the tokens' own adapters kept
    low = (x @ s["lora_a"].float().reshape(L * R, K).t()).reshape(T, L, R)
    keep = a[:, None] == torch.arange(L, device=x.device)[None, :]
    low = torch.where(keep[:, :, None], low * s["scale"][None, :, None], 0.0)
    y = y + low.reshape(T, L * R) @ s["lora_b"].float().permute(0, 2, 1).reshape(L * R, -1)
    return y.to(s["x"].dtype)


def _plain_attn(s):
    q, pk, pv, ok, ov = (s[x].float() for x in ("q", "prefix_k", "prefix_v", "own_k", "own_v"))
    B, n, HQ, D = q.shape
    H = pk.shape[1]
    q = q.reshape(B, n, H, HQ // H, D).permute(2, 0, 1, 3, 4)                       # head, request, new, group, dim
    if s["page_table"] is not None:
        at = s["page_table"].long()
        ok, ov = ok[at].flatten(1, 2), ov[at].flatten(1, 2)
    S = ok.shape[1]
    sp = q.reshape(H, -1, D) @ pk.permute(1, 2, 0)                                   # head, rows, prefix
    so = q.permute(1, 0, 2, 3, 4).reshape(B, H, -1, D) @ ok.permute(0, 2, 3, 1)      # request, head, rows, own
    sp = sp.reshape(H, B, -1, pk.shape[0]).permute(1, 0, 2, 3) * s["scale"]
    last = s["own_len"].long()[:, None] - n + torch.arange(n, device=q.device)[None, :]
    seen = torch.arange(S, device=q.device)[None, None, :] <= last[:, :, None]       # request, new, own
    seen = seen[:, None, :, None, :].expand(B, H, n, HQ // H, S).reshape(B, H, -1, S)
    so = torch.where(seen, so * s["scale"], float("-inf"))
    top = torch.maximum(sp.amax(dim=-1), so.amax(dim=-1))[..., None]
    sp, so = torch.exp(sp - top), torch.exp(so - top)
    total = sp.sum(dim=-1, keepdim=True) + so.sum(dim=-1, keepdim=True)
    o = (sp.permute(1, 0, 2, 3).reshape(H, -1, pk.shape[0]) @ pv.permute(1, 0, 2)).reshape(H, B, -1, D).permute(1, 0, 2, 3)
    o = (o + so @ ov.permute(0, 2, 1, 3)) / total
    return o.reshape(B, H, n, HQ // H, D).permute(0, 2, 1, 3, 4).reshape(B, n, HQ, D).to(s["q"].dtype)


def _plain_verify(s):
    l, q, x, t = s["logits"].float(), s["draft_probs"], s["draft_tokens"].long(), s["temperature"]
    B, n = x.shape
    V = l.shape[-1]
    ids = torch.arange(V, device=l.device)
    best = l.argmax(dim=-1)
    z = l / torch.where(t > 0, t, 1.0)[:, None, None]
    e = torch.exp(z - z.amax(dim=-1, keepdim=True))
    p = e / e.sum(dim=-1, keepdim=True)
    px, qx = (v[:, :n].gather(2, x[:, :, None])[:, :, 0] for v in (p, q))
    good = torch.where((t > 0)[:, None], s["uniforms"] * qx < px, best[:, :n] == x)
    accepted = good.long().cumprod(dim=1).sum(dim=1)
    row = torch.arange(B, device=l.device)
    w = p[row, accepted]
    w = torch.where((accepted < n)[:, None], (w - q[row, accepted.clamp(max=n - 1)]).clamp(min=0.0), w)
    last = torch.where(t > 0, (w / s["noise"]).argmax(dim=-1), best[row, accepted])
    at = torch.arange(n + 1, device=l.device)[None, :]
    x = torch.cat([x, x[:, :1]], dim=1)
    tokens = torch.where(at < accepted[:, None], x, torch.where(at == accepted[:, None], last[:, None], -1))
    return dict(accepted=accepted.to(torch.int32), tokens=tokens.to(torch.int32))


def run(s):
    if not own:
        return {"linear": _plain_linear, "attn": _plain_attn, "verify": _plain_verify}[s["op"]](s)
    from paper_1603_06809_b200 import serve
    if s["op"] == "linear":
        return serve.bcast_serve_linear(s["x"], s["weight"], lora_a=s["lora_a"], lora_b=s["lora_b"], adapter=s["adapter"],
                                        scale=s["scale"], bias=s["bias"], workspace=s["workspace"])
    if s["op"] == "attn":
        return serve.bcast_serve_attn(s["q"], s["prefix_k"], s["prefix_v"], s["own_k"], s["own_v"], s["own_len"],
                                      page_table=s["page_table"], scale=s["scale"], workspace=s["workspace"])
    accepted, tokens = serve.bcast_serve_verify(s["logits"], s["draft_probs"], s["draft_tokens"], s["uniforms"], s["noise"],
                                                s["temperature"], workspace=s["workspace"])
    return dict(accepted=accepted, tokens=tokens)


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "linear":
        T, K, N, R = case["tokens"], case["k"], case["n"], case["rank"]
        used = min(case["adapters"], case["requests"])
        return dict(bytes=size * (T * K + N * K + T * N + used * R * (K + N)), flops=2.0 * T * (K * N + R * (K + N)))
    if case["op"] == "attn":
        B, n, H, G, D = (case[x] for x in ("batch", "new", "kv_heads", "group", "dim"))
        mean = (max(case["own_max"], n) + n) / 2.0                                   # own lengths are uniform
        keys = case["prefix"] * H + B * mean * H
        return dict(bytes=size * D * (2 * keys + 2 * B * n * H * G), flops=4.0 * D * B * n * H * G * (case["prefix"] + mean))
    B, n, V = case["batch"], case["new"], case["vocab"]
    return dict(bytes=B * V * (size * (n + 1) + 4 + 4), flops=4.0 * B * V * (n + 1))


# ------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    d = lambda v: v.to(torch.float64)  # noqa: E731
    if case["op"] == "linear":
        y = torch.mm(d(s["x"]), d(s["weight"]).T)
        if s["bias"] is not None:
            y += d(s["bias"])
        for a in range(case["adapters"]):
            rows = (s["adapter"] == a).nonzero()[:, 0]
            if len(rows):
                y[rows] += d(s["scale"][a]) * torch.mm(torch.mm(d(s["x"][rows]), d(s["lora_a"][a]).T), d(s["lora_b"][a]).T)
        return y
    if case["op"] == "attn":
        B, n, H, G, D = (case[x] for x in ("batch", "new", "kv_heads", "group", "dim"))
        out = torch.empty(B, n, H * G, D, dtype=torch.float64, device="cuda")
        lengths = s["own_len"].tolist()
        for h in range(H):
            pk, pv = d(s["prefix_k"][:, h]), d(s["prefix_v"][:, h])
            for b in range(B):
                if s["page_table"] is None:
                    k, v = s["own_k"][b, :lengths[b], h], s["own_v"][b, :lengths[b], h]
                else:
                    pages = s["page_table"][b].tolist()
                    k = torch.cat([s["own_k"][i, :, h] for i in pages])[:lengths[b]]
                    v = torch.cat([s["own_v"][i, :, h] for i in pages])[:lengths[b]]
                k, v = torch.cat([pk, d(k)]), torch.cat([pv, d(v)])
                for i in range(n):
                    end = len(k) - n + i + 1
                    w = torch.softmax(d(s["q"][b, i, h * G:(h + 1) * G]) @ k[:end].T * s["scale"], dim=-1)
                    out[b, i, h * G:(h + 1) * G] = w @ v[:end]
        return out
    B, n, V = case["batch"], case["new"], case["vocab"]
    accepted, tokens = [], []
    for b in range(B):
        t, drafted, said, count = float(s["temperature"][b]), s["draft_tokens"][b].tolist(), [], 0
        while True:
            z = d(s["logits"][b, count])
            if t > 0:
                p = torch.softmax(z / d(s["temperature"][b]), dim=0)
            else:
                p = torch.zeros_like(z)
                p[int((z == z.max()).nonzero()[0, 0])] = 1.0
            if count == n:
                break
            x, q = drafted[count], d(s["draft_probs"][b, count])
            if (float(d(s["uniforms"][b, count]) * q[x]) < float(p[x])) if t > 0 else float(p[x]) == 1.0:
                said.append(x)
                count += 1
                continue
            if t > 0:
                p = (p - q).clamp(min=0.0)
            break
        said.append(int((p / d(s["noise"][b])).argmax()) if t > 0 else int(p.argmax()))
        accepted.append(count)
        tokens.append(said + [-1] * (n + 1 - len(said)))
    return dict(accepted=torch.tensor(accepted, dtype=torch.int32, device="cuda"),
                tokens=torch.tensor(tokens, dtype=torch.int32, device="cuda"))
