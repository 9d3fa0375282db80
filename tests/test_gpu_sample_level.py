"""onela_sample_tokens depends on the logits' differences alone: rows at a level of 10^7 temperatures, drawn with uniforms next to a border of the running sum.

Every uniform here is the fp32 number nearest to a border and lies 5e-12 to 1.5e-10 from it.  A mass is good to 2e-13 (the exponential; its rounding to 2^-47 is
less), a border, a share of two sums of them, to twice that: the token is decided.  The oracle's sums are in 80 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2609_12399_b200 as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("unit", [8.0, 2.0 ** 77, 2.0 ** -20])
@pytest.mark.parametrize("level", [0, 15434033, -15432821, 1000003])
@pytest.mark.parametrize("vocab", [20000, 131072])
def test_draws_next_to_a_border(unit, level, vocab):
    rng = np.random.default_rng(vocab + abs(level))
    k = np.sort(rng.integers(0, 3, vocab))                      # the largest first: what all other masses have in common then shows
    x = (unit * (level - k)).astype(np.float32)               # (24 bits: exact)
    assert np.array_equal(x.astype(np.float64), unit * (level - k))
    run = np.cumsum(np.exp(-k.astype(np.longdouble)))
    border = run / run[-1]
    u = border.astype(np.float32)
    far = np.abs(u.astype(np.longdouble) - border)
    pick = np.flatnonzero((far > 5e-12) & (far < 1.5e-10) & (u < 1))[:2000]
    assert len(pick) > 40
    u = u[pick]
    want = np.searchsorted(run, u.astype(np.longdouble) * run[-1], side="right")
    logits = torch.tensor(x, device="cuda")[None].expand(len(u), vocab)
    tokens = torch.empty(len(u), dtype=torch.int32, device="cuda")
    P.onela_sample_tokens(logits, torch.tensor(u, device="cuda"), tokens, temperature=torch.full((len(u),), unit, device="cuda"))
    torch.cuda.synchronize()
    got = tokens.cpu().numpy()
    assert np.array_equal(got, want), (int((got != want).sum()), len(u))


@pytest.mark.parametrize("temperature", [1.0, math.inf])
def test_plus_infinity_at_any_temperature(temperature):
    x = torch.full((1, 5000), 3e38, device="cuda")
    x[0, 77] = x[0, 4000] = math.inf
    x[0, 5] = -math.inf
    u = torch.tensor([0.0, 0.4, 0.6, 0.999], device="cuda")
    tokens, logprobs = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(4, device="cuda")
    P.onela_sample_tokens(x.expand(4, 5000), u, tokens, temperature=torch.full((4,), temperature, device="cuda"), logprobs_out=logprobs)
    torch.cuda.synchronize()
    assert tokens.tolist() == [77, 77, 4000, 4000]
    assert torch.allclose(logprobs, torch.full((4,), -math.log(2.0), device="cuda"), rtol=2.0 ** -23, atol=0)
