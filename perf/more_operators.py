"""More of the serving operators' measured cases, their plain forms and their definition in 64 bits.

What a replica does between, before and behind the products and the attention of a step:

  append    new tokens' queries and keys, normed for each head if asked for, are rotated by their positions, and keys and
            values go to their places in the requests' caches (pages or rows)
  logprobs  log probability of a given token in every row of logits, the row's entropy and its most probable tokens
  pack      numbers to microscaled 4-bit ones (blocks of 32 along a row share a power of two) and back
  linear4   y = x W^T + bias, W held in 4 bits as after a broadcast, x taken to 4 bits on the way

`own` selects between the plain form (elementary torch operations in 32 bits) and the library's kernels.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # one new token of one request, small heads, no norms: the latency of a single call
        dict(name="append_one", op="append", batch=1, new=1, q_heads=8, kv_heads=2, dim=64, rot=64, axes=1, interleaved=False, norm=False,
             history=300, first=509, page=16, ragged=False, dtype="bf16"),
        # tokens of three images, positions in time, height and width, a head size that fills no power of two, ragged lengths
        dict(name="append_image", op="append", batch=3, new=1237, q_heads=16, kv_heads=2, dim=96, rot=96, axes=3, interleaved=True, norm=True,
             history=41, first=0, page=64, ragged=True, dtype="fp16"),
        # eight prompts being read behind a long shared prefix, normed heads: bound by moving queries, keys and values
        dict(name="append_prompts", op="append", batch=8, new=2048, q_heads=32, kv_heads=8, dim=128, rot=128, axes=1, interleaved=False, norm=True,
             history=500, first=131072, page=16, ragged=False, dtype="bf16"),
        # the token of one request that was just drawn, a small vocabulary in 32 bits: the latency of a single call
        dict(name="logprobs_one", op="logprobs", rows=1, vocab=32000, top=5, dtype="fp32"),
        # a decode step's rows, a vocabulary that no vector divides, the most alternatives a service usually answers with
        dict(name="logprobs_odd", op="logprobs", rows=37, vocab=50001, top=20, dtype="fp16"),
        # the tokens of a prompt, a vocabulary of 128 Ki: bound by reading the logits
        dict(name="logprobs_prompt", op="logprobs", rows=4096, vocab=131072, top=8, dtype="bf16"),
        # a projection with sizes that no tile divides
        dict(name="pack_odd", op="pack", rows=5003, k=2080, dtype="fp16"),
        # the output projection of a vocabulary of 64 Ki, before and after a broadcast: bound by moving it
        dict(name="pack_vocab", op="pack", rows=65536, k=4096, dtype="bf16"),
        # one new token: the latency of a single call
        dict(name="linear4_one", op="linear4", tokens=1, k=2048, n=2048, bias=False, dtype="bf16"),
        # a decode step of 64 requests: bound by reading W
        dict(name="linear4_decode", op="linear4", tokens=64, k=4096, n=4096, bias=False, dtype="bf16"),
        # a small batch with ragged lengths and sizes that no tile divides
        dict(name="linear4_ragged", op="linear4", tokens=333, k=2080, n=5003, bias=True, dtype="fp16"),
        # prompts being read: bound by the matrix product
        dict(name="linear4_prompts", op="linear4", tokens=8192, k=4096, n=4096, bias=True, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    op = rng.choice(["append", "logprobs", "pack", "linear4"])
    if op == "append":
        while True:
            dim = rng.choice([64, 96, 128, 128])
            h = rng.choice([1, 2, 4, 8])
            c = dict(op=op, batch=_log(rng, 1, 256), new=_log(rng, 1, 2048), q_heads=h * rng.choice([1, 2, 4, 5, 8]), kv_heads=h, dim=dim,
                     rot=rng.choice([dim, dim, dim // 2 // 16 * 16]), axes=rng.choice([1, 1, 3]), interleaved=rng.random() < 0.3,
                     norm=rng.random() < 0.5, history=_log(rng, 1, 4000) - 1, first=_log(rng, 1, 131072) - 1, page=rng.choice([0, 16, 32, 64]),
                     ragged=rng.random() < 0.3, dtype=rng.choice(["bf16", "fp16"]))
            moved = c["batch"] * c["new"] * (c["q_heads"] + 2 * h) * dim
            if moved <= 8 * 2048 * 48 * 128 and c["batch"] * (c["new"] + c["history"]) * h * dim <= 8 * 2548 * 8 * 128:
                return c
    if op == "logprobs":
        while True:
            c = dict(op=op, rows=_log(rng, 1, 4096), vocab=_log(rng, 2000, 262144), top=rng.choice([0, 1, 5, 8, 20]),
                     dtype=rng.choice(["bf16", "fp16", "fp32"]))
            if c["rows"] * c["vocab"] * (2 if c["dtype"] == "fp32" else 1) <= 4096 * 131072:
                return c
    if op == "pack":
        while True:
            c = dict(op=op, rows=_log(rng, 1, 65536), k=32 * _log(rng, 4, 512), dtype=rng.choice(["bf16", "fp16", "fp32"]))
            if c["rows"] * c["k"] * (2 if c["dtype"] == "fp32" else 1) <= 65536 * 4096:
                return c
    while True:
        c = dict(op=op, tokens=_log(rng, 1, 8192), k=32 * _log(rng, 16, 448), n=_log(rng, 512, 16384), bias=rng.random() < 0.5,
                 dtype=rng.choice(["bf16", "fp16"]))
        if c["tokens"] * c["k"] * c["n"] <= 8192 * 4096 * 4096 and c["n"] * c["k"] <= 16384 * 4096:
            return c


# ------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    h = torch.Generator()
    h.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0, dtype=dt):
        out = torch.empty(shape, dtype=dtype, device=dev)
        return out.normal_(mean, std, generator=g)

    if case["op"] == "append":
        B, n, HQ, H, D, page = (case[x] for x in ("batch", "new", "q_heads", "kv_heads", "dim", "page"))
        cap = n + case["history"]
        fresh = torch.randint(1, n + 1, (B,), generator=h) if case["ragged"] else torch.full((B,), n)
        before = torch.randint(0, case["history"] + 1, (B,), generator=h)
        # queries, keys and values as the projection leaves them: one row of a token after the other
        q, k, v = normal(B, n, HQ + 2 * H, D, std=1.5).split((HQ, H, H), dim=2)
        st = dict(q=q, k=k, v=v, own_len=(before + fresh).to(dev, torch.int32), new_len=fresh.to(dev, torch.int32) if case["ragged"] else None,
                  first=case["first"], interleaved=case["interleaved"], q_norm=None, k_norm=None, positions=None, axis=None)
        st["inv_freq"] = (10000.0 ** -(torch.arange(case["rot"] // 2, dtype=torch.float64) * 2 / case["rot"])).to(dev, torch.float32)
        if case["norm"]:
            st.update(q_norm=normal(D, std=0.2, mean=1.0), k_norm=normal(D, std=0.2, mean=1.0))
        if case["axes"] > 1:
            # frames of 24 x 31 patches: the pairs' axes in turn
            at = torch.arange(n)
            places = torch.stack([at // 744, at // 31 % 24, at % 31], dim=-1)[None] + torch.randint(0, 2000, (B, 1, 3), generator=h)
            st.update(positions=places.to(dev, torch.int32), axis=(torch.arange(case["rot"] // 2) % 3).to(dev, torch.int32))
        if page:
            each = -(-cap // page)
            table = torch.randperm(B * each, generator=h).to(torch.int32).reshape(B, each)
            st.update(own_k=normal(B * each, page, H, D), own_v=normal(B * each, page, H, D), page_table=table.to(dev))
        else:
            st.update(own_k=normal(B, cap, H, D), own_v=normal(B, cap, H, D), page_table=None)
    elif case["op"] == "logprobs":
        T, V = case["rows"], case["vocab"]
        logits = torch.empty(T, V, dtype=dt, device=dev)
        tokens = torch.empty(T, dtype=torch.int32, device=dev)
        for a in range(0, T, 512):
            l = normal(min(512, T - a), V, std=2.0, dtype=torch.float32)
            logits[a:a + 512] = l
            # tokens as a model draws them: by the race, so from the distribution itself
            tokens[a:a + 512] = (l - torch.empty_like(l).exponential_(generator=g).clamp_(min=1e-10).log_()).argmax(dim=-1).to(torch.int32)
        st = dict(logits=logits, tokens=tokens, top=case["top"])
    elif case["op"] == "pack":
        # rows of unlike size, as a projection's are
        x = normal(case["rows"], case["k"])
        x *= torch.empty(case["rows"], 1, device=dev).uniform_(0.01, 0.1, generator=g).to(dt)
        st = dict(x=x, dtype=dt)
    else:
        codes, scales = _pack(normal(case["n"], case["k"], std=case["k"] ** -0.5, dtype=torch.float32))
        st = dict(x=normal(case["tokens"], case["k"]), codes=codes, scales=_tiled(scales), bias=normal(case["n"], std=0.1) if case["bias"] else None)
        if own:
            from paper_1603_06809_b200 import serve
            st["workspace"] = serve.Workspace(dev)
    st["op"] = case["op"]
    return st


# ------------------------------------------------------------------------------------------------- plain forms
def _pack(x):
    """(codes [rows, k / 2], the even number's in the low half; scales [rows, k / 32]) of float32 numbers."""
    x = x.reshape(x.shape[0], -1, 32)
    exponent = x.abs().amax(dim=-1).view(torch.int32) >> 23
    scale = (exponent - 2).clamp(min=0)
    x = x * ((254 - scale) << 23).view(torch.float32)[:, :, None]
    size = x.abs()
    # 0, 1/2, 1, 3/2, 2, 3, 4, 6: a half-way number goes to the neighbour with the even code
    code = (size > 0.25).int() + (size >= 0.75) + (size > 1.25) + (size >= 1.75) + (size > 2.5) + (size >= 3.5) + (size > 5.0)
    code = (code | torch.signbit(x).int() << 3).reshape(x.shape[0], -1, 2)
    return (code[:, :, 0] | code[:, :, 1] << 4).to(torch.uint8), scale.to(torch.uint8)


def _tiled(scales):
    """Scales in the order the library holds them: tiles of 128 rows x 4 blocks, [rows / 128, blocks / 4, 32, 4, 4], row r of
    a tile at [r % 32, r / 32]."""
    n, b = scales.shape
    out = torch.zeros(-(-n // 128) * 128, -(-b // 4) * 4, dtype=torch.uint8, device=scales.device)
    out[:n, :b] = scales
    return out.reshape(out.shape[0] // 128, 4, 32, out.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous()


def _unpack(codes, scales):
    """Float32 numbers of codes and their scales [rows, k / 32]."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    x = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], dim=-1).reshape(codes.shape[0], -1, 32)
    s = scales.int()
    power = torch.where(s > 0, s << 23, 1 << 22).view(torch.float32)
    return (x * power[:, :, None]).reshape(codes.shape[0], -1)


def _untiled(scales, rows, blocks):
    return scales.permute(0, 3, 2, 1, 4).reshape(scales.shape[0] * 128, -1)[:rows, :blocks]


def _plain_append(s):
    q, k = s["q"].float(), s["k"].float()
    B, n, H, D = k.shape
    if s["q_norm"] is not None:
        q = q * torch.rsqrt((q * q).mean(dim=-1, keepdim=True) + 1e-6) * s["q_norm"].float()
        k = k * torch.rsqrt((k * k).mean(dim=-1, keepdim=True) + 1e-6) * s["k_norm"].float()
    new = s["new_len"] if s["new_len"] is not None else torch.full_like(s["own_len"], n)
    at = torch.arange(n, device=q.device)[None, :]
    slot = s["own_len"].long()[:, None] - n + at
    there = (at >= n - new[:, None]) & (slot >= 0)
    if s["positions"] is None:
        place = (s["first"] + slot)[:, :, None].double()
    else:
        place = s["positions"][:, :, s["axis"].long()].double()
    angle = place * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    R = 2 * s["inv_freq"].shape[0]

    def rotate(x):
        y = x.clone()
        a, b = (slice(0, R, 2), slice(1, R, 2)) if s["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., a] * sin + x[..., b] * cos
        return y
    q, k = torch.where(there[:, :, None, None], rotate(q), 0.0).to(s["q"].dtype), rotate(k).to(s["k"].dtype)
    b, i = there.nonzero(as_tuple=True)
    slot = slot[b, i]
    if s["page_table"] is None:
        page = b
    else:
        size = s["own_k"].shape[1]
        page, slot = s["page_table"][b, slot // size].long(), slot % size
    s["own_k"][page, slot] = k[b, i]
    s["own_v"][page, slot] = s["v"][b, i]
    return dict(q=q, own_k=s["own_k"], own_v=s["own_v"])


def _plain_logprobs(s):
    l = s["logits"].float()
    V = l.shape[1]
    top = l.amax(dim=-1, keepdim=True)
    z = l - top
    e = torch.exp(z)
    total = e.sum(dim=-1)
    log_total = torch.log(total)
    entropy = log_total - (e * z).sum(dim=-1) / total
    lp = z.gather(1, s["tokens"].long()[:, None])[:, 0] - log_total
    if s["top"] == 0:
        return dict(logprobs=lp, entropy=entropy)
    del e
    # distinct whole numbers in the order of the logits, the lower token first among equals
    bits = l.view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() << 32
    key += torch.arange(V - 1, -1, -1, device=l.device)
    ids = V - 1 - (key.topk(s["top"], dim=-1).values & 0xffffffff)
    return dict(logprobs=lp, entropy=entropy, top_tokens=ids.to(torch.int32), top_logprobs=z.gather(1, ids) - log_total[:, None])


def _plain_linear4(s):
    n, half = s["codes"].shape
    w = _unpack(s["codes"], _untiled(s["scales"], n, half // 16))
    y = _unpack(*_pack(s["x"].float())) @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(s["x"].dtype)


def run(s):
    if not own:
        if s["op"] == "pack":
            return _unpack(*_pack(s["x"].float())).to(s["dtype"])
        return {"append": _plain_append, "logprobs": _plain_logprobs, "linear4": _plain_linear4}[s["op"]](s)
    from paper_1603_06809_b200 import serve
    if s["op"] == "append":
        q = serve.bcast_serve_append(s["q"], s["k"], s["v"], s["own_k"], s["own_v"], s["own_len"], page_table=s["page_table"],
                                     new_len=s["new_len"], first=s["first"], positions=s["positions"], inv_freq=s["inv_freq"], axis=s["axis"],
                                     interleaved=s["interleaved"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=1e-6)
        return dict(q=q, own_k=s["own_k"], own_v=s["own_v"])
    if s["op"] == "logprobs":
        lp, entropy, ids, top = serve.bcast_serve_logprobs(s["logits"], s["tokens"], top=s["top"])
        return dict(logprobs=lp, entropy=entropy, **(dict(top_tokens=ids, top_logprobs=top) if s["top"] else {}))
    if s["op"] == "pack":
        return serve.bcast_serve_unpack4(*serve.bcast_serve_pack4(s["x"]), s["dtype"])
    return serve.bcast_serve_linear4(s["x"], s["codes"], s["scales"], bias=s["bias"], workspace=s["workspace"])


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "append":
        moved = case["batch"] * case["new"] * case["dim"]
        if case["ragged"]:                                                           # lengths are uniform
            moved = case["batch"] * (case["new"] + 1) / 2.0 * case["dim"]
        heads = case["q_heads"] + case["kv_heads"]
        return dict(bytes=2.0 * size * moved * (heads + case["kv_heads"]), flops=6.0 * moved * heads)
    if case["op"] == "logprobs":
        return dict(bytes=case["rows"] * (size * case["vocab"] + 12 + 8 * case["top"]), flops=6.0 * case["rows"] * case["vocab"])
    if case["op"] == "pack":                                                         # there and back
        return dict(bytes=case["rows"] * case["k"] * (2.0 * size + 2 * 17 / 32), flops=6.0 * case["rows"] * case["k"])
    T, K, N = case["tokens"], case["k"], case["n"]
    return dict(bytes=size * (T * K + T * N) + N * K * 17 / 32, flops=2.0 * T * K * N)


# ------------------------------------------------------------------------------------------------- 64 bits
def _exact_values(x):
    """The 4-bit values of numbers, by the definition: the nearest of the eight sizes, the even code among two as near."""
    d = x.to(torch.float64).reshape(x.shape[0], -1, 32)
    top = d.abs().amax(dim=-1, keepdim=True)
    power = torch.where(top > 0, torch.frexp(top).exponent.to(torch.float64) - 1, -200.0)      # floor(log2(top))
    unit = torch.exp2((power - 2).clamp(min=-127))
    best, off = torch.zeros_like(d), torch.full_like(d, math.inf)
    for v in (0, 1, 2, 4, 0.5, 1.5, 3, 6):                                                     # codes 0 2 4 6, then 1 3 5 7
        near = (d.abs() / unit - v).abs()
        best, off = torch.where(near < off, v, best), torch.minimum(near, off)
    return (torch.copysign(best, d) * unit).reshape(x.shape[0], -1)


def exact(case, seed):
    s = prepare(case, seed)
    d = lambda v: v.to(torch.float64)  # noqa: E731
    if case["op"] == "append":
        B, n, HQ, H, D, R = (case[x] for x in ("batch", "new", "q_heads", "kv_heads", "dim", "rot"))
        out = dict(q=torch.zeros(B, n, HQ, D, dtype=torch.float64, device="cuda"), own_k=d(s["own_k"]), own_v=d(s["own_v"]))
        first, second = (torch.arange(0, R, 2), torch.arange(1, R, 2)) if case["interleaved"] else (torch.arange(R // 2), torch.arange(R // 2, R))
        for b in range(B):
            length = int(s["own_len"][b])
            count = n if s["new_len"] is None else int(s["new_len"][b])
            rows = torch.arange(n - count, n, device="cuda")
            slots = torch.arange(length - count, length, device="cuda")
            parts = []
            for x, w in ((s["q"], s["q_norm"]), (s["k"], s["k_norm"])):
                x = d(x[b, rows])
                if w is not None:
                    x = x / torch.sqrt((x ** 2).sum(dim=-1, keepdim=True) / D + 1e-6) * d(w)
                if s["positions"] is None:
                    place = d(slots + case["first"])[:, None].expand(count, R // 2)
                else:
                    place = d(s["positions"][b, rows])[:, s["axis"].long()]
                turn = torch.polar(torch.ones_like(place), place * d(s["inv_freq"]))[:, None]
                turned = torch.complex(x[..., first], x[..., second]) * turn
                x[..., first], x[..., second] = turned.real, turned.imag
                parts.append(x)
            out["q"][b, rows] = parts[0]
            for name, x in (("own_k", parts[1]), ("own_v", d(s["v"][b, rows]))):
                if s["page_table"] is None:
                    out[name][b, slots] = x
                else:
                    pages = s["page_table"][b].long()
                    whole = out[name][pages].flatten(0, 1)
                    whole[slots] = x
                    out[name][pages] = whole.unflatten(0, (len(pages), case["page"]))
        return out
    if case["op"] == "logprobs":
        found = []
        for a in range(0, case["rows"], 256):
            p = torch.log_softmax(d(s["logits"][a:a + 256]), dim=-1)
            order = torch.sort(s["logits"][a:a + 256], dim=-1, descending=True, stable=True).indices[:, :max(case["top"], 1)]
            found.append((p.gather(1, s["tokens"][a:a + 256].long()[:, None])[:, 0], -(p.exp() * p).sum(dim=-1), order.to(torch.int32), p.gather(1, order)))
        lp, entropy, ids, top = (torch.cat(x) for x in zip(*found))
        return dict(logprobs=lp, entropy=entropy, **(dict(top_tokens=ids, top_logprobs=top) if case["top"] else {}))
    if case["op"] == "pack":
        step = max(1, (1 << 24) // case["k"])
        return torch.cat([_exact_values(s["x"][a:a + step]) for a in range(0, case["rows"], step)])
    # W's values from its codes, one bit field after the other
    low, high = s["codes"] & 15, s["codes"] >> 4
    code = torch.stack([low, high], dim=-1).flatten(1)
    size, mantissa = code >> 1 & 3, d(code & 1)
    w = torch.where(size == 0, mantissa / 2, (1 + mantissa / 2) * torch.exp2(d(size) - 1)) * (1 - 2 * d(code >> 3))
    n, k = w.shape
    r, c = torch.arange(n, device="cuda")[:, None], torch.arange(k // 32, device="cuda")[None, :]
    scale = s["scales"][r // 128, c // 4, r % 32, r % 128 // 32, c % 4]
    w = (w.reshape(n, -1, 32) * torch.exp2(d(scale) - 127)[:, :, None]).reshape(n, k)
    y = torch.mm(_exact_values(s["x"]), w.T)
    return y if s["bias"] is None else y + d(s["bias"])
