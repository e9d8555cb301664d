"""Arguments and arrays at the edge of what the serving operators take, against the plain 64-bit forms."""
import math

import pytest
import torch

import serve_reference as R
from paper_1603_06809_b200 import serve as S
from test_serve_gpu import check_verify, on_gpu, verify_case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# ------------------------------------------------------------------------------------------ verify: temperatures
@pytest.mark.parametrize("B,n,V", [(1, 0, 40), (3, 4, 7), (4, 3, 2048), (9, 2, 5003), (2, 3, 33333)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t", [math.inf, 3e38, 1e30])
def test_verify_temperatures_without_end(B, n, V, dtype, t):
    # logits / temperature goes to zero: every token is as likely as any other
    c = verify_case(B + n + V, B, n, V, dtype)
    c["temperature"][:] = t
    if n:
        c["draft_probs"][:, 0] = 0.5 / V                      # first drafts that some uniforms accept, and some would not
        c["uniforms"][:, 0] *= 4
    check_verify(c)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_verify_infinite_temperature_over_the_tokens_that_are_allowed(dtype):
    V = 1000
    c = verify_case(71, 6, 2, V, dtype)
    c["temperature"][:] = torch.tensor([math.inf, math.inf, math.inf, 0.7, 0.0, math.inf])
    c["logits"][0, :, 100:] = -math.inf                       # most tokens forbidden
    c["logits"][1, :, ::3] = math.nan                         # NaN counts as -infinity
    c["logits"][2, :, 5:] = torch.finfo(c["logits"].dtype).min    # the lowest number is a number: divided by infinity it is 0
    c["logits"][5] = -math.inf                                # no probabilities
    c["draft_probs"][:, :] = 1.0 / V
    c["uniforms"][:, 0] = 0.5
    c["uniforms"][0, 1] = 12.0
    # the limit of softmax(l / T): the same for every token that has a probability at all
    flat = dict(c, logits=c["logits"].clone(), temperature=c["temperature"].clone())
    for b in (0, 1, 2, 5):
        z = c["logits"][b]
        flat["logits"][b] = torch.where(z > -math.inf, torch.zeros_like(z), torch.full_like(z, -math.inf))
        flat["temperature"][b] = 1.0
    accepted, tokens, margin = R.verify(**flat)
    assert margin > 1e-5
    got = S.bcast_serve_verify(*(on_gpu(v) for v in c.values()))
    assert torch.equal(got[0].cpu(), accepted) and torch.equal(got[1].cpu(), tokens)
    assert got[1][5].tolist() == [-1, -1, -1]


def test_verify_temperatures_that_are_none():
    # zero, negative and NaN: the largest logit
    c = verify_case(72, 4, 3, 700, "bf16", greedy=True)
    c["draft_tokens"][:] = c["logits"][:, :3].float().argmax(-1).to(torch.int32)
    c["draft_tokens"][1, 2] ^= 1
    c["temperature"][:] = 0.0
    want = check_verify(c)
    c["temperature"][:] = torch.tensor([-1.0, math.nan, -math.inf, -0.0])
    got = S.bcast_serve_verify(*(on_gpu(v) for v in c.values()))
    assert all(torch.equal(x, y) for x, y in zip(want, got))
