"""Plain 64-bit forms of the serving operators on the CPU, written from their definitions, with the bounds
that the tests hold the kernels to.  Shares no code with the library.

Bounds (u: unit roundoff of the data type, 2^-8 for bf16 and 2^-11 for fp16; one rounding of the result costs
u times its size).  Sums of n products in 32 bits: n * 2^-24 times the sum of the products' sizes.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def linear(x, weight, bias=None, lora_a=None, lora_b=None, adapter=None, scale=None):
    """(y, bound on the error of each entry)."""
    u = U[x.dtype]
    x, w = x.double(), weight.double()
    y = x @ w.T
    size = x.abs() @ w.abs().T
    if bias is not None:
        y = y + bias.double()
        size = size + bias.double().abs()
    err = (x.shape[1] + 256) * 2.0 ** -24 * size
    if lora_a is not None:
        for t in range(x.shape[0]):
            a = int(adapter[t])
            if 0 <= a < lora_a.shape[0]:
                A, Bm, s = lora_a[a].double(), lora_b[a].double(), float(scale[a])
                y[t] += s * (Bm @ (A @ x[t]))
                low = abs(s) * (A.abs() @ x[t].abs())
                # u = s A x in 32 bits, passed on as two numbers of the type (relative error u^2 at most, and
                # what is below the type's smallest numbers: 2^-24 per entry for fp16)
                err[t] += Bm.abs() @ ((x.shape[1] + 256) * 2.0 ** -24 * low + u * u * low + (2.0 ** -24 if u < 2.0 ** -10 else 0.0))
    return y, err + u * (y.abs() + err) + 1e-30


def own_rows(cache, page_table, b, length, head):
    """(rows [length, D], which of them are there) of request b."""
    if page_table is None:
        return cache[b, :length, head], torch.ones(length, dtype=torch.bool)
    page = cache.shape[1]
    rows = torch.zeros(length, cache.shape[3], dtype=cache.dtype)
    there = torch.zeros(length, dtype=torch.bool)
    for j in range(length):
        p = int(page_table[b, j // page])
        if 0 <= p < cache.shape[0]:
            rows[j] = cache[p, j % page, head]
            there[j] = True
    return rows, there


def attn(q, prefix_k, prefix_v, own_k, own_v, own_len, page_table=None, scale=None):
    """(out, bound, lse, bound of lse)."""
    u = U[q.dtype]
    B, n, HQ, D = q.shape
    P, H = prefix_k.shape[:2]
    scale = D ** -0.5 if scale is None else scale
    cap = own_k.shape[1] if page_table is None else page_table.shape[1] * own_k.shape[1]
    out = torch.zeros(B, n, HQ, D, dtype=torch.float64)
    bound = torch.zeros_like(out)
    lse = torch.full((B, n, HQ), -math.inf, dtype=torch.float64)
    lse_bound = torch.zeros_like(lse)
    for b in range(B):
        length = min(max(int(own_len[b]), 0), cap)
        for h in range(HQ):
            g = h // (HQ // H)
            k, there = own_rows(own_k, page_table, b, length, g)
            v, _ = own_rows(own_v, page_table, b, length, g)
            k = torch.cat([prefix_k[:, g], k]).double()
            v = torch.cat([prefix_v[:, g], v]).double()
            there = torch.cat([torch.ones(P, dtype=torch.bool), there])
            for i in range(n):
                end = P + max(length - n + i + 1, 0)
                keep = there[:end]
                if not bool(keep.any()):
                    continue
                kk, vv, qq = k[:end][keep], v[:end][keep], q[b, i, h].double()
                s = kk @ qq * scale
                top = s.max()
                w = torch.exp(s - top)
                p = w / w.sum()
                out[b, i, h] = p @ vv
                # a score off by ds changes its weight by exp(ds) - 1 < 2 ds; a weight is rounded to the type
                # before its product with v (u) and its exponential may be a polynomial good to 2^-12
                ds = float((kk.abs() @ qq.abs()).max()) * abs(scale) * (D + 8) * 2.0 ** -24 + float(s.abs().max()) * 2.0 ** -22
                rel = u + 2 * (2 * ds + 2.0 ** -12) + len(kk) * 2.0 ** -24
                bound[b, i, h] = rel * (p @ vv.abs())
                lse[b, i, h] = top + torch.log(w.sum())
                lse_bound[b, i, h] = ds + 2.0 ** -12 + len(kk) * 2.0 ** -24 + abs(float(lse[b, i, h])) * 2.0 ** -22
    tiny = 2.0 ** -24 if u < 2.0 ** -10 else 1e-30          # below fp16's smallest normal number the spacing is 2^-24
    return out, bound + u * (out.abs() + bound) + tiny, lse, lse_bound


def verify(logits, draft_probs, draft_tokens, uniforms, noise, temperature):
    """(accepted, tokens, margin): margin is the smallest relative distance of any decision from its tie, so that
    inputs whose outcome 32 bits cannot tell are recognised."""
    B, n1, V = logits.shape
    n = n1 - 1
    accepted, tokens, margin = [], [], math.inf
    for b in range(B):
        t, said, c = float(temperature[b]), [], 0

        def probs(i):
            z = logits[b, i].double()
            z = torch.where(torch.isnan(z), -math.inf, z)
            top = z.max()
            if top == -math.inf:
                return torch.zeros(V, dtype=torch.float64), -1
            best = int((z == top).nonzero()[0, 0])
            if t <= 0:
                p = torch.zeros(V, dtype=torch.float64)
                p[best] = 1.0
            elif top == math.inf:
                p = (z == top).double()
            else:
                p = torch.exp((z - top) / t)
            return p / p.sum(), best
        while c < n:
            p, best = probs(c)
            x = int(draft_tokens[b, c])
            if best < 0 or not 0 <= x < V:
                break
            if t <= 0:
                if x != best:
                    break
            else:
                left, right = float(uniforms[b, c].double() * draft_probs[b, c, x].double()), float(p[x])
                margin = min(margin, abs(left - right) / max(left, right, 1e-300))
                if not left < right:
                    break
            said.append(x)
            c += 1
        p, best = probs(c)
        if best < 0 or t <= 0:
            last = best
        else:
            e = noise[b].double()
            ok = e > 0
            w = (p - draft_probs[b, c].double()).clamp(min=0.0) if c < n else p
            if not bool(((w > 0) & ok).any()):
                w = p
            r = torch.where(ok & (w > 0), w / e, -math.inf)
            order = torch.sort(r, descending=True).values
            if V > 1 and float(order[1]) > 0 and math.isfinite(float(order[0])):
                # w = p - q is as inexact as p is: its relative error grows by p / w
                at = torch.argmax(r)
                margin = min(margin, float((order[0] - order[1]) / order[0] * (w[at] / p[at])))
            last = int((r == order[0]).nonzero()[0, 0]) if float(order[0]) > 0 else -1
        said.append(last)
        accepted.append(c)
        tokens.append(said + [-1] * (n1 - len(said)))
    return torch.tensor(accepted, dtype=torch.int32), torch.tensor(tokens, dtype=torch.int32).reshape(B, n1), margin
