"""Edges of cache appends and log probabilities, and of replicas that use them: angles of all sizes, results that stand by
themselves, log probabilities at their upper end, buffers that a second broadcast fills."""
import io
import math
from fractions import Fraction

import pytest
import torch

import serve_more_reference as R
from paper_1603_06809_b200 import replica as P
from paper_1603_06809_b200 import serve as S
from test_serve_gpu import DEV, TYPES, gen, rand

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------ angles
def two_pi(bits):
    """2 pi to that many bits behind the point, by Machin's formula in whole numbers."""
    def arctan(n):
        x = (1 << bits + 20) // n
        total, k, sign = x, 3, -1
        while x:
            x //= n * n
            total += sign * (x // k)
            k, sign = k + 2, -sign
        return total
    return Fraction(8 * (4 * arctan(5) - arctan(239)), 1 << bits + 20)


TWO_PI = two_pi(300)
# zero, of all exponents, of either sign, those of bases 1e4 to 1e7, neighbours of 2^26 and of powers of 2^32
FREQUENCIES = [0.0, 1e-45, 3e-39, 2e-38, 1e-30, 1e-20, 3e-13, 1e-9, 1e-7, 1.2409e-07, 2.5e-7, 1.1547e-4, 0.01, 0.5, 0.99999994, 1.0, 1.7, math.pi, 2 * math.pi, 37.5,
               4096.0, 2.0 ** 20 + 1, 2.0 ** 24, 1.5 * 2.0 ** 24, 2.0 ** 25 + 6, 7.3 * 2.0 ** 26, 1.9 * 2.0 ** 40, 1e15, 1e18, 3e20, 1e25, 6.5e26, 2.0 ** 89, 1e30, 1e38, 3.4e38,
               -1.0, -1e-7, -0.37, -37.5, -4097.0, -1e20, -2.0 ** 120, -3e-20, -0.0]
POSITIONS = [0, 1, 2, 3, -1, -5, 11, 1000, -77777, 131071, 2 ** 20 + 3, 12345678, 2 ** 31 - 1, -2 ** 31, 1 - 2 ** 31]


def turned(x, frequency, position):
    """x (cos t, sin t) with t = position * frequency, the angle reduced in whole numbers."""
    t = Fraction(frequency) * position
    quarters = round(t / (TWO_PI / 4))
    rest = float(t - quarters * TWO_PI / 4)
    c, s = math.cos(rest), math.sin(rest)
    c, s = ((c, s), (-s, c), (-c, -s), (s, -c))[quarters % 4]
    return x * c, x * s


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("by", ["positions", "slots"])
def test_append_angles_of_all_sizes(dtype, interleaved, by):
    # Pairs (x, 0): each result is one product, so that a small sine shows with all its digits.
    dt, pairs = TYPES[dtype], 48
    x = 1.0 if dtype == "bf16" else 32768.0
    f = torch.tensor((FREQUENCIES + [1.0] * pairs)[:pairs], dtype=torch.float32)
    places = POSITIONS if by == "positions" else [0, 1, 7, 1000, 131071, 2 ** 20 + 3, 2 ** 31 - 1]
    n = len(places)
    k = torch.zeros(n, 1, 1, 96, dtype=dt)
    k[..., (slice(0, 96, 2) if interleaved else slice(0, 48))] = x
    d = k.to(DEV)
    own_k, own_v = torch.zeros(n, 1, 1, 96, dtype=dt, device=DEV), torch.zeros(n, 1, 1, 96, dtype=dt, device=DEV)
    one = torch.ones(n, dtype=torch.int32, device=DEV)
    if by == "positions":
        q = S.bcast_serve_append(d, d, d, own_k, own_v, one, positions=torch.tensor(places, dtype=torch.int32, device=DEV)[:, None], inv_freq=f.to(DEV), interleaved=interleaved)
    else:
        q = torch.cat([S.bcast_serve_append(d[i:i + 1], d[i:i + 1], d[i:i + 1], own_k[i:i + 1], own_v[i:i + 1], one[i:i + 1], first=p, inv_freq=f.to(DEV), interleaved=interleaved)
                       for i, p in enumerate(places)])
    assert torch.equal(q, own_k)
    got = q.double().cpu().reshape(n, 2, 48) if not interleaved else q.double().cpu().reshape(n, 48, 2).transpose(1, 2)
    want = torch.tensor([[turned(x, float(v), p) for v in f] for p in places], dtype=torch.float64).transpose(1, 2)
    # The reduced angle: four roundings, of the position, the frequency's product with it, 1 / pi and the product with that,
    # and 2^-63 of a turn; cosine and sine to two units (2^-23 each); the product with x, and a sum with zero.
    err = want.abs() * (4 * R.E + 2 * 2.0 ** -23 + 2 * R.E) + x * 2 * math.pi * 2.0 ** -63
    over = (got - want).abs() - R.rounded(want, err, dt)
    worst = int(over.argmax())
    i, _, j = worst // (2 * pairs), worst // pairs % 2, worst % pairs
    assert bool((over <= 0).all()), f"frequency {float(f[j])}, position {places[i]}: {got[i, :, j].tolist()}, not {want[i, :, j].tolist()}"


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
