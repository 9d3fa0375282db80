"""onela_norm_rotate against the plain form in 64 bits: norms, weights, rotations of both pairings, far and negative positions, strides,
in place, odd head widths and counts.

Tolerance, per element: half a step of the output type, and 32 steps of 2^-24 of the pair's magnitude.  (The sum of squares has at
most 8 + 5 roundings, half of which the root passes on; root, quotient, weight and scale round five times: 12 steps.  The fraction of a turn
is rounded to fp32 and, at 2^31 positions of frequency 1, off by 2^-53 x 2^29 turns in 64 bits; with the two functions' last places and the
rotation's three roundings: 17 steps.)"""
import numpy as np
import pytest
import torch

import paper_2609_12399_b200 as P
from oracle import operators as plain

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _check(got, ref, rotary, interleaved, dtype):
    half = torch.finfo(DT[dtype]).eps / 2
    mag = np.abs(ref).copy()
    if rotary:                                   # a pair's error is that of both its elements
        i = np.arange(rotary // 2)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
        both = mag[..., a] + mag[..., b]
        mag[..., a], mag[..., b] = both, both
    err = np.abs(got.double().cpu().numpy() - ref)
    assert np.all(err <= half * np.abs(ref) + 32 * 2.0 ** -24 * mag), float((err / (half * np.abs(ref) + 32 * 2.0 ** -24 * mag + 1e-300)).max())


def _run(n, hq, hk, d, dtype, norm, rotary=0, interleaved=False, positions=None, scale=1.0, weights=True, seed=0, magnitude=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q = (magnitude * torch.randn((n, hq, d), generator=gen, device="cuda")).to(DT[dtype])
    k = (magnitude * torch.randn((n, hk, d), generator=gen, device="cuda")).to(DT[dtype])
    w = [1 + 0.2 * torch.randn((d,), generator=gen, device="cuda") for _ in range(2)] if norm == "rms" and weights else [None, None]
    f = (10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / max(rotary, 1))).float() if rotary else None
    if rotary and positions is None:
        positions = torch.randint(0, 5000, (n,), generator=gen, device="cuda", dtype=torch.int32)
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    P.onela_norm_rotate(q, k, qo, ko, norm=norm, eps=1e-6, q_scale=scale, q_weight=w[0], k_weight=w[1], positions=positions, inv_freq=f, interleaved=interleaved)
    torch.cuda.synchronize()
    for x, y, wx, sc in ((q, qo, w[0], scale), (k, ko, w[1], 1.0)):
        ref = plain.norm_rotate(x.double().cpu().numpy(), norm, float(np.float32(1e-6)), float(np.float32(sc)), None if wx is None else wx.cpu().numpy(),
                                None if positions is None else positions.tolist(), None if f is None else f.cpu().numpy(), interleaved)
        _check(y, ref, rotary, interleaved, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [8, 32, 40, 64, 96, 128, 256])
@pytest.mark.parametrize("norm", ["l2", "rms", None])
def test_norms(dtype, d, norm):
    _run(37, 3, 2, d, dtype, norm, scale=d ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,rotary", [(32, 16), (32, 32), (64, 48), (96, 96), (128, 64), (128, 128), (256, 64), (256, 256)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation(dtype, d, rotary, interleaved):
    _run(29, 5, 1, d, dtype, "rms", rotary, interleaved)


@pytest.mark.parametrize("hq,hk", [(1, 0), (0, 1), (16, 2), (64, 8), (200, 3)])
@pytest.mark.parametrize("n", [1, 2, 67])
def test_head_counts(hq, hk, n):
    _run(n, hq, hk, 128, "bf16", "l2", 32)


@pytest.mark.parametrize("hq,hk,d", [(1, 0, 64), (2, 1, 256), (3, 4, 128), (5, 6, 32)])
def test_many_tokens_per_block(hq, hk, d):
    """Calls large enough for several tokens in a block; the last block is not full."""
    _run(12289 + hq, hq, hk, d, "bf16", "rms")


def test_far_and_negative_positions():
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 9, 131071, -7], dtype=torch.int32, device="cuda")
    _run(8, 2, 2, 128, "fp32", None, 128, False, pos)


@pytest.mark.parametrize("magnitude", [0.0, 1e-10, 1e15])
def test_zero_tiny_and_large_vectors(magnitude):
    """Zeros stay zeros (eps); 1e-10: eps outweighs the squares; 1e15: squares of 1e30 are still fp32 numbers."""
    _run(5, 2, 2, 64, "fp32", "l2", magnitude=magnitude)


def test_slices_of_one_projection_and_in_place():
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, hq, hk, d = 51, 4, 2, 64
    row = torch.randn((n, (hq + 2 * hk) * d), generator=gen, device="cuda").bfloat16()
    before = row.clone()
    q, k = row[:, :hq * d].view(n, hq, d), row[:, hq * d:(hq + hk) * d].view(n, hk, d)
    pos = torch.arange(n, device="cuda", dtype=torch.int32)
    f = (10000.0 ** (-torch.arange(0, d, 2, device="cuda") / d)).float()
    want = [torch.empty_like(x.contiguous()) for x in (q, k)]
    P.onela_norm_rotate(q, k, want[0], want[1], positions=pos, inv_freq=f)
    P.onela_norm_rotate(q, k, q, k, positions=pos, inv_freq=f)
    torch.cuda.synchronize()
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(row[:, (hq + hk) * d:], before[:, (hq + hk) * d:])


def test_other_stream_and_graph():
    gen = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randn((33, 4, 128), generator=gen, device="cuda").bfloat16()
    k = torch.randn((33, 4, 128), generator=gen, device="cuda").bfloat16()
    want, got = [torch.empty_like(q), torch.empty_like(k)], [torch.empty_like(q), torch.empty_like(k)]
    P.onela_norm_rotate(q, k, *want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    P.onela_norm_rotate(q, k, *got, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.onela_norm_rotate(q, k, *got)
    q.mul_(2.0)                                  # (exact in bf16: the same unit vectors but for eps)
    g.replay()
    P.onela_norm_rotate(q, k, *want)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_nothing_to_do():
    e = torch.empty((0, 4, 64), device="cuda")
    P.onela_norm_rotate(e, e, e.clone(), e.clone())
    z = torch.empty((3, 0, 64), device="cuda")
    P.onela_norm_rotate(z, z, z.clone(), z.clone())
