"""Plain 64-bit forms of cache appends, log probabilities and microscaled 4-bit numbers on the CPU, written from their
definitions, with the bounds that the tests hold the kernels to.  Shares no code with the library.

A rounding costs at most u times the size of the value (bf16 2^-8, fp16 2^-11, 32 bits 2^-24); below fp16's smallest normal number
it costs 2^-25.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
E = 2.0 ** -24


def rounded(y, err, dtype):
    """The bound on y's error after its rounding, `err` before."""
    return err + U[dtype] * (y.abs() + err) + (2.0 ** -25 if dtype == torch.float16 else 1e-38)


# ---- append
def heads(x, weight, eps, angle, pairs):
    """(y, bound before its rounding) of one token's heads [heads, D]; `pairs`: the partners' places, angle their angles and the
    bound on these."""
    x = x.double()
    D = x.shape[-1]
    err = torch.zeros_like(x)
    if weight is not None:
        mean = (x * x).mean(dim=-1, keepdim=True)
        x = x / torch.sqrt(mean + eps) * weight.double()
        # a sum of D squares: D + 1 roundings; the division, eps, the inverse root to two units and two products
        err = x.abs() * ((D + 2) / 2 + 6) * E
    if angle is None:
        return x, err
    theta, off = angle
    first, second = pairs
    a, b, ea, eb = x[..., first], x[..., second], err[..., first], err[..., second]
    c, s = torch.cos(theta), torch.sin(theta)
    y, e = x.clone(), err.clone()
    # cosine and sine are off by the angle's error and two units; two products and their sum
    turn = (a.abs() + b.abs()) * (off + 3 * 2.0 ** -23 + 2 * E)
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    e[..., first] = ea * c.abs() + eb * s.abs() + turn
    e[..., second] = ea * s.abs() + eb * c.abs() + turn
    return y, e


def append(q, k, v, own_k, own_v, own_len, page_table=None, new_len=None, first=0, positions=None, inv_freq=None, axis=None, interleaved=False,
           q_norm=None, k_norm=None, eps=1e-6):
    """dict of (expected, bound): q, own_k, own_v.  A bound of zero asks for the very number."""
    B, n, H, D = k.shape
    cap = own_k.shape[1] if page_table is None else page_table.shape[1] * own_k.shape[1]
    out = None
    if q is not None:
        out = (torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64))
    ck, cv = own_k.double().clone(), own_v.double().clone()
    ek, ev = torch.zeros_like(ck), torch.zeros_like(cv)
    rot = 0 if inv_freq is None else 2 * len(inv_freq)
    j = torch.arange(rot // 2)
    pairs = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
    for b in range(B):
        for i in range(n):
            slot = int(own_len[b]) - n + i
            if slot < 0 or (new_len is not None and i < n - int(new_len[b])):
                continue
            angle = None
            if rot:
                if positions is None:
                    place = torch.full((rot // 2,), float(first + slot), dtype=torch.float64)
                else:
                    p = positions[b, i].reshape(-1)
                    which = torch.zeros(rot // 2, dtype=torch.int64) if axis is None else axis.long()
                    which = torch.where((which >= 0) & (which < len(p)), which, 0)
                    place = p[which].double()
                theta = place * inv_freq.double()
                # 1 / (2 pi) and the product with it in 64 bits, cut to 2^-64 of a turn and, multiplied, to 2^-25 of it
                angle = (theta, theta.abs() * 2.0 ** -51 + 2 * math.pi * 2.0 ** -25 + 2.0 ** -30)
            if q is not None:
                y, e = heads(q[b, i], q_norm, eps, angle, pairs)
                out[0][b, i], out[1][b, i] = y, rounded(y, e, q.dtype) if angle is not None or q_norm is not None else 0.0 * e
                if rot < D and q_norm is None and rot:
                    out[1][b, i, :, rot:] = 0.0
            if slot >= cap:
                continue
            page, at = b, slot
            if page_table is not None:
                page, at = int(page_table[b, slot // own_k.shape[1]]), slot % own_k.shape[1]
                if not 0 <= page < own_k.shape[0]:
                    continue
            y, e = heads(k[b, i], k_norm, eps, angle, pairs)
            ck[page, at], ek[page, at] = y, rounded(y, e, k.dtype) if angle is not None or k_norm is not None else 0.0 * e
            if rot < D and k_norm is None and rot:
                ek[page, at, :, rot:] = 0.0
            cv[page, at] = v[b, i].double()
    return dict(q=out, own_k=(ck, ek), own_v=(cv, ev))


# ---- log probabilities
def logprobs(logits, tokens, top):
    """(logprobs, bound), (entropy, bound), top_tokens, (top_logprobs, bound)."""
    T, V = logits.shape
    l = logits.double()
    l = torch.where(torch.isnan(l), -math.inf, l)
    lp, lp_bound, h, h_bound = (torch.zeros(T, dtype=torch.float64) for _ in range(4))
    ids = torch.full((T, top), -1, dtype=torch.int32)
    best, best_bound = torch.full((T, top), -math.inf, dtype=torch.float64), torch.zeros(T, top, dtype=torch.float64)
    for r in range(T):
        row = l[r]
        most = float(row.max())
        if most == -math.inf:
            logp = torch.full_like(row, -math.inf)
        elif most == math.inf:
            logp = torch.where(row == math.inf, -math.log(int((row == math.inf).sum())), -math.inf)
        else:
            z = row - most
            total = torch.exp(z).sum()
            logp = z - torch.log(total)
        p = torch.exp(logp)
        some = p > 0
        h[r] = -(p[some] * logp[some]).sum()
        # Sums of V terms in 32 bits, at most V / 256 + 64 of them one after the other; each term's exponent is off by three
        # roundings of its size and its exponential by 2^-22.  What a term is taken against may lie 8 below its row's
        # largest logit.
        far = float((p[some] * (row[some] - most).abs()).sum()) + 8.0 if math.isfinite(most) else 0.0
        rel = (V / 256 + 64) * E + 2.0 ** -22 + 4 * E * far
        log_total = float(torch.log(total)) if math.isfinite(most) else 0.0
        size = abs(log_total) + 8.0

        def bound(x):
            return rel + 4 * E * (size + x.abs()) if math.isfinite(most) else 4 * E * x.abs()
        h_bound[r] = rel * (1 + far) + 4 * E * (size + far) + (4 * E * float(h[r]))
        x = int(tokens[r])
        lp[r] = logp[x] if 0 <= x < V else -math.inf
        lp_bound[r] = bound(lp[r]) if math.isfinite(float(lp[r])) else 0.0
        order = torch.sort(row, descending=True, stable=True).indices
        order = order[torch.isfinite(logp[order])] if most == math.inf else order[row[order] > -math.inf]
        order = order[:top]
        ids[r, :len(order)] = order.to(torch.int32)
        best[r, :len(order)] = logp[order]
        best_bound[r, :len(order)] = torch.where(torch.isfinite(logp[order]), bound(logp[order]), 0.0)
    return (lp, lp_bound), (h, h_bound), ids, (best, best_bound)


# ---- microscaled 4-bit numbers
SIZES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def pack(x):
    """(codes [rows, k], scales' bytes [rows, k / 32]) of numbers, one code to an entry."""
    d = x.double().reshape(x.shape[0], -1, 32)
    most = d.abs().amax(dim=-1)
    bad = ~torch.isfinite(d).all(dim=-1)
    exponent = torch.frexp(torch.where(bad | (most == 0), 1.0, most)).exponent - 1            # floor(log2)
    byte = torch.where(most == 0, 0, (exponent - 2 + 127).clamp(min=0))
    size = torch.where(bad[..., None], 0.0, d).abs() / torch.exp2(byte.double() - 127)[..., None]
    sizes = torch.tensor(SIZES, dtype=torch.float64)
    near = (size[..., None] - sizes).abs()
    # the nearest; of two as near the one with the even code
    code = torch.where(near == near.amin(dim=-1, keepdim=True), torch.tensor([0, 11, 2, 13, 4, 15, 6, 17]), 99).amin(dim=-1)
    code = torch.where(code > 10, code - 10, code)
    code = torch.where(bad[..., None], 0, code + 8 * torch.signbit(d))
    return code.reshape(x.shape).to(torch.uint8), torch.where(bad, 255, byte).to(torch.uint8)


def values(codes, scales):
    """64-bit numbers of codes and scales as `pack` gives them."""
    v = torch.tensor(SIZES + tuple(-s for s in SIZES), dtype=torch.float64)[codes.long()].reshape(codes.shape[0], -1, 32)
    power = torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127))
    return (v * power[..., None]).reshape(codes.shape)


def bytes_of(codes):
    return codes[:, 0::2] | codes[:, 1::2] << 4


def tiled(scales):
    """In tiles of 128 rows x 4 blocks, entry by entry."""
    n, b = scales.shape
    out = torch.zeros(-(-n // 128), -(-b // 4), 32, 4, 4, dtype=torch.uint8)
    for c in range(b):
        r = torch.arange(n)
        out[r // 128, c // 4, r % 32, r % 128 // 32, c % 4] = scales[:, c]
    return out


def linear4(x, w_codes, w_scales, bias=None):
    """(y, bound)."""
    w, xx = values(w_codes, w_scales), values(*pack(x))
    y, size = xx @ w.T, xx.abs() @ w.abs().T
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    err = (x.shape[1] + 256) * E * size
    return y, rounded(y, err, x.dtype)
