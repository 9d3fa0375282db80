"""onela_delta_rule where the terms of a chunk differ by orders of magnitude: states that fade within 64 tokens, gates beyond 1 and below -1, keys and
values of very different size.  Every case token by token and in chunks, against Eq. 1 in 64 bits.

Tolerance, componentwise: a chunk of 64 tokens with X = beta (v - g S k), T = (I + A)^-1 (A_ij = beta_i (g_i / g_j) k_i . k_j below the diagonal), D = T X and
P_ij = (g_i / g_j) q_i . k_j may be off by 2^-17 of
        |g| |S| |q| + |P| |T| |X|   (an output) ,     |g_C| |S| + (|T| |X|)^T diag(|g_C / g|) |K|   (the state behind it) ,
all products of magnitudes (P's and A's dot products too: below, Pm and Am; an error dA of A costs D |T| dA |D|), and by the error of the state before it, passed on as the chunk passes the state on.  2^-17 = 128 x 2^-24: operands of two fp16 parts on either
side are off by 2^-22 each (8 steps of 2^-24), a sum of up to 24 matrix products, each of which truncates, by 2^-23 each time (48 steps), the running products of 64 gates
by half a step per factor (64), less than 8 for the rest.  Token by token every term has fewer roundings than that.  Outputs add half a step of their type.
What lies below 2^-110 may be lost: up to 2^-110 sqrt(dv) < 2^-106 of an output, 2^-110 sqrt(dv dk) <= 2^-103 of a state."""
import numpy as np
import pytest
import torch

import paper_2609_12399_b200 as P
from oracle import operators as plain

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
STEP = 2.0 ** -17
C = 64


def _bounds(q, k, v, alpha, beta, S):
    """Per chunk of one (sequence, value head): allowed error of its outputs [n, dv] and of the last state [dv, dk]."""
    n = len(q)
    out, err = np.zeros_like(v), np.zeros_like(S)
    for a in range(0, n, C):
        b = min(n, a + C)
        m = b - a
        al = alpha[a:b]
        ratio = np.tril(np.ones((m, m)))                      # ratio[i, j] = alpha_{j+1} .. alpha_i
        for i in range(1, m):
            ratio[i, :i] = ratio[i - 1, :i] * al[i]
        gi = np.cumprod(al)
        kk = k[a:b] @ k[a:b].T
        T = np.linalg.inv(np.eye(m) + np.tril(beta[a:b, None] * ratio * kk, -1))
        X = np.abs(beta[a:b, None]) * (np.abs(v[a:b]) + np.abs(gi)[:, None] * (np.abs(k[a:b]) @ np.abs(S).T))
        D = np.abs(T) @ X
        Am = np.abs(beta[a:b, None]) * np.tril(np.abs(ratio) * (np.abs(k[a:b]) @ np.abs(k[a:b]).T), -1)
        D = D + np.abs(T) @ (Am @ D)
        # what the error of the state before does: through S itself and through the deltas that it shifts
        dX = np.abs(beta[a:b] * gi)[:, None] * (np.abs(k[a:b]) @ err.T)
        dD = np.abs(T) @ dX
        Pm = np.tril(np.abs(ratio) * (np.abs(q[a:b]) @ np.abs(k[a:b]).T))
        out[a:b] = STEP * (np.abs(gi)[:, None] * (np.abs(q[a:b]) @ np.abs(S).T) + Pm @ D) + np.abs(gi)[:, None] * (np.abs(q[a:b]) @ err.T) + Pm @ dD
        w = np.abs(ratio[-1])[:, None]
        err = STEP * (np.abs(gi[-1]) * np.abs(S) + (w * D).T @ np.abs(k[a:b])) + np.abs(gi[-1]) * err + (w * dD).T @ np.abs(k[a:b])
        for t in range(a, b):
            S = alpha[t] * S
            S = S + beta[t] * np.outer(v[t] - S @ k[t], k[t])
    return out, err


def _check(q, k, v, alpha, beta, S, dtype, max_tokens):
    """One sequence, H heads: q, k [n, H, dk], v [n, H, dv], alpha, beta [n, H], S [H, dv, dk] (fp64 tensors that dtype holds, or are rounded to it)."""
    dev = lambda x, t: x.to(device="cuda", dtype=t).contiguous()  # noqa: E731
    q, k, v = (dev(x, DT[dtype]) for x in (q, k, v))
    alpha, beta, S = (dev(x, torch.float32) for x in (alpha, beta, S))
    n, H, dv = v.shape
    states, out = S[None].clone(), torch.zeros_like(v)
    starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    P.onela_delta_rule(q, k, v, alpha, beta, states, out, starts=starts, max_tokens=max_tokens, status=status)
    torch.cuda.synchronize()
    assert status.tolist() == [0, 0]
    c = lambda x: x.double().cpu().numpy()  # noqa: E731
    q, k, v, alpha, beta, S, out, states = (c(x) for x in (q, k, v, alpha, beta, S, out, states))
    ref, ref_states = plain.delta_rule(q, k, v, alpha, beta, S[None], [(0, n)], [0], [0])
    assert np.isfinite(out).all() and np.isfinite(states).all()
    half = torch.finfo(DT[dtype]).eps / 2
    for h in range(H):
        want = np.array([ref[t][h] for t in range(n)])
        allowed, allowed_state = _bounds(q[:, h], k[:, h], v[:, h], alpha[:, h], beta[:, h], S[h])
        err = np.abs(out[:, h] - want) - half * np.abs(want) * (1 + 2.0 ** -8)
        # (norms of a token's output: single elements may lie above the componentwise bound where all of it is one product's rounding)
        worst = np.maximum(err, 0)
        for t in range(n):
            assert np.linalg.norm(worst[t]) <= np.linalg.norm(allowed[t]) + 2.0 ** -106, (h, t, np.linalg.norm(worst[t]), np.linalg.norm(allowed[t]), np.linalg.norm(want[t]))
        e, a = np.linalg.norm(states[0, h] - ref_states[0, h]), np.linalg.norm(allowed_state)
        assert e <= a + 2.0 ** -103, (h, e, a, np.linalg.norm(ref_states[0, h]))


def _inputs(n, H=2, dk=128, dv=128, seed=0):
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)  # noqa: E731
    unit = lambda x: x / torch.linalg.vector_norm(x, dim=-1, keepdim=True)  # noqa: E731
    return dict(q=unit(rand(n, H, dk)), k=unit(rand(n, H, dk)), v=rand(n, H, dv), alpha=0.9 + 0.1 * torch.rand((n, H), generator=gen, dtype=torch.float64),
                beta=torch.rand((n, H), generator=gen, dtype=torch.float64), S=0.3 * rand(H, dv, dk))


SHAPES = [(128, 128), (64, 64), (32, 96)]


@pytest.mark.parametrize("dtype", ["fp32"])
@pytest.mark.parametrize("max_tokens", [1, 0])
@pytest.mark.parametrize("dk,dv", SHAPES)
@pytest.mark.parametrize("alpha", [0.8, 0.6, 0.45])
@pytest.mark.parametrize("beta", [0.0, 0.5])
def test_what_fades_within_a_chunk(dk, dv, alpha, beta, max_tokens, dtype):
    """No values behind the first token: outputs and the state fall by alpha per token, 10^-6 to 10^-22 in a chunk, and keep their places."""
    x = _inputs(100, dk=dk, dv=dv)
    x["alpha"][:] = alpha
    x["beta"][1:] = beta
    x["v"][1:] = 0
    _check(**x, dtype=dtype, max_tokens=max_tokens)


@pytest.mark.parametrize("dtype", ["fp32"])
@pytest.mark.parametrize("max_tokens", [1, 0])
@pytest.mark.parametrize("dk,dv", SHAPES)
def test_gates_below_minus_one(dk, dv, max_tokens, dtype):
    x = _inputs(64, dk=dk, dv=dv, seed=1)
    x["alpha"][:] = -1.2
    x["alpha"][5::7] = 0.3
    _check(**x, dtype=dtype, max_tokens=max_tokens)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("max_tokens", [1, 0])
@pytest.mark.parametrize("alpha", [1.2, 1.5, 4.0, -1.3])
def test_gates_beyond_one(alpha, max_tokens, dtype):
    """The state grows by up to 2^120 in 60 tokens; the first outputs are as exact as the last."""
    x = _inputs(60, seed=2)
    x["alpha"][:] = alpha
    _check(**x, dtype=dtype, max_tokens=max_tokens)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("max_tokens", [1, 0])
@pytest.mark.parametrize("gates", [(0.0, 1.0), (1e-6, 1e-6), (1e-20, 1.0), (-1.0, 1.0)])
def test_gates_of_any_size(gates, max_tokens, dtype):
    x = _inputs(150, seed=3)
    gen = torch.Generator().manual_seed(9)
    x["alpha"] = gates[0] + (gates[1] - gates[0]) * torch.rand(x["alpha"].shape, generator=gen, dtype=torch.float64)
    x["alpha"][70:75] = gates[0]
    _check(**x, dtype=dtype, max_tokens=max_tokens)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("max_tokens", [1, 0])
@pytest.mark.parametrize("small", [2.0 ** -10, 1e-6, 1e-12])
@pytest.mark.parametrize("first", [True, False])
def test_keys_of_different_size_in_a_chunk(first, small, max_tokens, dtype):
    x = _inputs(64, seed=4)
    part = slice(0, 32) if first else slice(32, 64)
    x["k"][part] *= small
    x["S"][:] = 0
    _check(**x, dtype=dtype, max_tokens=max_tokens)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("max_tokens", [1, 0])
@pytest.mark.parametrize("small", [1e-3, 1e-8])
def test_values_of_different_size_under_one_key(small, max_tokens, dtype):
    """The same key again and again, written over at once (beta 1): a value replaces the one before it."""
    x = _inputs(64, seed=5)
    x["k"][:] = x["k"][:1]
    x["q"][:] = x["k"]
    x["beta"][:] = 1
    x["v"][8:] *= small
    _check(**x, dtype=dtype, max_tokens=max_tokens)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_long_sequences_whose_maps_fade(dtype):
    """Cut into segments: the maps between them, which have no values, fade by 0.9^700 and 0.7^700."""
    for alpha in (0.9, 0.7):
        x = _inputs(2500, H=2, seed=6)
        x["alpha"][:] = alpha
        x["v"][:2300] = 0
        _check(**x, dtype=dtype, max_tokens=0)


@pytest.mark.parametrize("max_tokens", [1, 0])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("what", ["q", "k", "v", "alpha", "beta"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_token_that_is_not_finite_reaches_back_15_tokens_at_most(value, what, dtype, max_tokens):
    """Token 110 of 150: what lies before token 96 is what it is without it, bit for bit."""
    x = _inputs(150, seed=7)
    outs = []
    for bad in (False, True):
        y = {n: t.clone() for n, t in x.items()}
        if bad:
            y[what][110] = value
        dev = {n: t.to(device="cuda", dtype=DT[dtype] if n in "qkv" else torch.float32) for n, t in y.items()}
        states, out = dev["S"][None].clone(), torch.zeros_like(dev["v"])
        P.onela_delta_rule(dev["q"], dev["k"], dev["v"], dev["alpha"], dev["beta"], states, out, starts=torch.tensor([0, 150], dtype=torch.int32, device="cuda"), max_tokens=max_tokens)
        torch.cuda.synchronize()
        outs.append(out)
    assert torch.isfinite(outs[0]).all()
    assert torch.equal(outs[0][:96], outs[1][:96])
    if max_tokens == 1:
        assert torch.equal(outs[0][:110], outs[1][:110])
