"""onela_sample_tokens against the plain form in 64 bits: every token equal (an input whose draw lies within 1e-9 of a border of the running sum
would be left out; the seeds here have none), log-probabilities to an fp32 rounding.

Tolerance of a logprob: 2^-24 of its value for the rounding, and 2^-40 for masses rounded to 2^-43 of the largest (at 360 000
tokens their sum is off by 2^-43 x 2^18.5 / 2 at most, while it is at least 1: 2^-25.5; near 0 a logprob is off by that)."""
import math

import numpy as np
import pytest
import torch

import paper_2609_12399_b200 as P
from oracle import operators as plain

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


def _sample(x, u, **kw):
    r = x.shape[0]
    f = lambda v, t: None if v is None else torch.tensor(v if isinstance(v, list) else [v] * r, dtype=t, device="cuda")  # noqa: E731
    tok, lp = torch.full((r,), -7, dtype=torch.int32, device="cuda"), torch.full((r,), 7.0, device="cuda")
    P.onela_sample_tokens(x, u, tok, temperature=f(kw.get("temperature"), torch.float32), top_k=f(kw.get("top_k"), torch.int32), top_p=f(kw.get("top_p"), torch.float32),
                          min_p=f(kw.get("min_p"), torch.float32), logprobs_out=lp)
    torch.cuda.synchronize()
    return tok.cpu().numpy(), lp.cpu().numpy()


def _compare(x, u, **kw):
    tok, lp = _sample(x, u, **kw)
    xs, us = x.float().cpu().numpy(), u.cpu().numpy()
    for i in range(len(us)):
        at = {k: (v[i] if isinstance(v, list) else v) for k, v in kw.items() if v is not None}
        for name in ("temperature", "top_p", "min_p"):
            if name in at:
                at[name] = float(np.float32(at[name]))
        want, logprob, border = plain.sample_row(xs[i], us[i], **at)
        if border < 1e-9 and want >= 0 and 0 < us[i] < 1:
            continue
        assert tok[i] == want, (i, tok[i], want, at, us[i])
        if math.isinf(logprob):
            assert lp[i] == logprob
        else:
            assert abs(lp[i] - logprob) <= 2.0 ** -24 * abs(logprob) + 2.0 ** -25, (i, lp[i], logprob)


def _logits(r, v, seed, dtype="fp32", spread=2.5, masked=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = spread * torch.randn((r, v), generator=gen, device="cuda")
    if masked:
        x.masked_fill_(torch.rand((r, v), generator=gen, device="cuda") < masked, -INF)
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32), torch.rand((r,), generator=gen, device="cuda")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("v", [1, 2, 7, 129, 1000, 4097, 32003])
@pytest.mark.parametrize("kw", [{}, {"temperature": 0.7}, {"top_k": 5}, {"top_p": 0.8}, {"min_p": 0.05}, {"temperature": 1.3, "top_k": 40, "top_p": 0.9, "min_p": 0.01},
                                {"top_k": 700, "top_p": 0.99}], ids=str)
def test_filters(dtype, v, kw):
    _compare(*_logits(9, v, 11 + v, dtype, masked=0.1 if v > 100 else 0.0), **kw)


@pytest.mark.parametrize("rows", [1, 3, 40, 150])
def test_rows_and_cluster_sizes(rows):
    _compare(*_logits(rows, 50021, rows, "bf16"), temperature=0.8, top_k=64, top_p=0.95)


@pytest.mark.parametrize("v", [131072, 200003, 360000])
def test_largest_vocabularies(v):
    _compare(*_logits(2, v, v), top_p=0.97, temperature=1.1)
    _compare(*_logits(2, v, v + 1), min_p=1e-4, top_k=20000)


def test_ties_are_kept_by_index():
    """Rows of few values: the end of the kept run lies inside a tie."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randint(-2, 3, (64, 6000), generator=gen, device="cuda").float()
    u = torch.rand((64,), generator=gen, device="cuda")
    for kw in ({"top_k": 1}, {"top_k": 777}, {"top_k": 1500, "top_p": 0.5}, {"top_p": 0.33}, {"top_p": 0.9, "min_p": 0.2}):
        _compare(x, u, **kw)
    flat = torch.full((8, 10007), -3.25, device="cuda")
    for kw in ({}, {"top_k": 10}, {"top_p": 0.5}, {"top_k": 1000, "top_p": 0.125}, {"min_p": 1.0}):
        _compare(flat, u[:8], **kw)


def test_values_far_apart_and_close():
    """Masks of the type's lowest value, values 1e30 apart, values that differ in the last place only, signed zeros, subnormals."""
    low = torch.finfo(torch.float32).min
    x, u = _logits(6, 5000, 8)
    x[0, 100:] = low
    x[1] = low
    x[2] = torch.linspace(-1e30, 1e30, 5000, device="cuda")
    x[3] = (torch.full((5000,), 1.0, device="cuda").view(torch.int32) + torch.arange(5000, device="cuda", dtype=torch.int32) % 37).view(torch.float32)
    x[4, ::2], x[4, 1::2] = 0.0, -0.0
    x[5] = torch.arange(5000, device="cuda").float() * 1e-42
    for kw in ({}, {"top_k": 50}, {"top_p": 0.5}, {"top_k": 2500, "top_p": 0.9, "temperature": 0.5}, {"temperature": 1e-3, "top_k": 3}, {"temperature": 50.0, "top_p": 0.1}):
        _compare(x, u, **kw)


def test_special_logits():
    x, u = _logits(8, 3000, 9)
    x[0, 5] = NAN
    x[1, ::2] = NAN
    x[2, 77] = x[2, 2999] = INF
    x[3] = -INF
    x[4] = NAN
    x[5] = -INF
    x[5, 1234] = -5.0
    x[6, 3] = INF
    x[6, 4] = NAN
    x[7, :] = INF
    for kw in ({}, {"top_k": 2}, {"top_p": 0.9}, {"top_k": 100, "top_p": 0.5, "min_p": 0.1}, {"temperature": 0.0}):
        _compare(x, u, **kw)
    tok, lp = _sample(x, u, top_p=0.5)
    assert tok[3] == -1 and tok[4] == -1 and lp[3] == -INF


def test_greedy_and_parameters_that_switch_off():
    x, u = _logits(12, 2049, 10, "bf16")
    _compare(x, u, temperature=[0.0, -1.0, NAN, 1.0, INF, 1e-30, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0], top_k=[0, -5, 2049, 3000, 1, 7, 0, 0, 0, 2048, 5, 5],
             top_p=[1.0, 1.5, NAN, 0.0, -1.0, 0.5, 1.0, 2.0, 0.999999, 0.9, 1.0, 0.0], min_p=[0.0, -1.0, NAN, 0.0, 0.5, 2.0, 1.0, 5.0, 0.0, 0.1, NAN, 1.0])


def test_uniforms_at_and_beyond_the_ends():
    x, _ = _logits(6, 1111, 12)
    u = torch.tensor([0.0, -3.0, NAN, 1.0, 7.0, 1.0 - 2.0 ** -24], device="cuda")
    _compare(x, u)
    _compare(x, u, top_k=3)


def test_strided_rows_streams_and_graphs():
    gen = torch.Generator(device="cuda").manual_seed(13)
    wide = torch.randn((5, 7001), generator=gen, device="cuda").bfloat16()
    u = torch.rand((5,), generator=gen, device="cuda")
    x = wide[:, 3:6001]                                    # rows start at odd places
    _compare(x, u, top_p=0.9)
    tok = torch.zeros((5,), dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    P.onela_sample_tokens(x, u, tok, stream=s)
    s.synchronize()
    want = _sample(x, u)[0]
    assert np.array_equal(tok.cpu().numpy(), want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.onela_sample_tokens(x, u, tok)
    u.copy_(torch.rand((5,), generator=gen, device="cuda"))
    g.replay()
    torch.cuda.synchronize()
    assert np.array_equal(tok.cpu().numpy(), _sample(x, u)[0])


def test_many_draws_from_one_row():
    """A row that is expanded over the draws (stride 0)."""
    x, _ = _logits(1, 3001, 21)
    u = torch.rand((7,), generator=torch.Generator(device="cuda").manual_seed(22), device="cuda")
    a, b = _sample(x.expand(7, 3001), u, top_k=50), _sample(x.expand(7, 3001).contiguous(), u, top_k=50)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_results_do_not_depend_on_the_rest_of_the_batch():
    x, u = _logits(150, 20011, 14)
    all_rows = _sample(x, u, top_p=0.9)
    for i in (0, 77, 149):
        one = _sample(x[i:i + 1], u[i:i + 1], top_p=0.9)
        assert one[0][0] == all_rows[0][i] and one[1][0] == all_rows[1][i]


def test_frequencies():
    """200 000 draws from one row: counts within five standard deviations of the masses."""
    n, r = 12, 200000
    gen = torch.Generator(device="cuda").manual_seed(15)
    row = torch.randn((1, n), generator=gen, device="cuda")
    u = torch.rand((r,), generator=gen, device="cuda")
    tok, _ = _sample(row.expand(r, n).contiguous(), u)
    p = torch.softmax(row[0].double(), 0).cpu().numpy()
    count = np.bincount(tok, minlength=n)
    assert np.all(np.abs(count - r * p) <= 5 * np.sqrt(r * p * (1 - p)))
