"""onela_delta_rule against Eq. 1 token by token in 64 bits: outputs and states of ragged batches, one token to some hundred, every head shape,
grouped heads, padding, fresh sequences, strides, bad slots and ranges.

Tolerance, relative to the 2-norm of the vector (an output) or matrix (a state): 2^-24 times 16 roundings per token - a row's dot product takes 16 / 2
in a lane and up to 4 across lanes, delta, decay and update four more - for the tokens that the state still remembers, at most 20 at gates in [0.9, 1]; outputs
add half a step of their type per element.  The chunked form (operands in two fp16 parts: 2^-22 per product, three products in a
chunk of 64 tokens) stays below that.

bf16 outputs of the chunked form come from S Q^T + D P^T with S (the state before the chunk), D (the chunk's update vectors) and P (weights
(g_i / g_j) q_i . k_j) rounded to fp16: every factor is off by up to 2^-11 of itself, evenly, so by 2^-11 / sqrt(3) in the mean square, independently.  The error's
mean square is then (2^-22 / 3) times the sum of the terms' squares, |S|^2 |q|^2 / dk + 2 sum_j (q . k_j)^2 |d_j|^2 over the chunk's tokens up to this
one (gates at most 1); three standard deviations are allowed."""
import numpy as np
import pytest
import torch

import paper_2609_12399_b200 as P
from oracle import operators as plain

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
UNTOUCHED = 123.0


class Batch:
    def __init__(self, lens, H=2, Hv=None, dk=64, dv=64, dtype="fp32", slots=None, fresh=None, seed=0, gates=(0.9, 1.0), extra_rows=3, extra_states=2, key_norm=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        Hv = Hv or H
        n, N = len(lens), sum(lens) + extra_rows
        rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
        unit = lambda x: x / torch.linalg.vector_norm(x, dim=-1, keepdim=True)  # noqa: E731
        self.q, self.k = unit(rand(N, H, dk)).to(DT[dtype]), (key_norm * unit(rand(N, H, dk))).to(DT[dtype])
        self.v = rand(N, Hv, dv).to(DT[dtype])
        self.alpha = gates[0] + (gates[1] - gates[0]) * torch.rand((N, Hv), generator=gen, device="cuda")
        self.beta = torch.sigmoid(rand(N, Hv))
        self.states = 0.3 * rand(n + extra_states, Hv, dv, dk)
        self.out = torch.full((N, Hv, dv), UNTOUCHED, dtype=DT[dtype], device="cuda")
        starts = np.concatenate(([0], np.cumsum(lens)))
        self.ranges = [(int(starts[i]), int(starts[i + 1])) for i in range(n)]
        self.slots = list(range(n)) if slots is None else slots
        self.fresh = [0] * n if fresh is None else fresh
        self.starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(2, dtype=torch.int32, device="cuda")
        self.dtype = dtype

    def i32(self, x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def run(self, max_tokens=0, stream=None, **over):
        self.chunked = (max_tokens or self.q.shape[0]) >= 32
        kw = over or dict(starts=self.starts, slots=self.i32(self.slots), fresh=self.i32(self.fresh), status=self.status)
        P.onela_delta_rule(self.q, self.k, self.v, self.alpha, self.beta, self.states, self.out, stream=stream, max_tokens=max_tokens, **kw)

    def reference(self, live=None):
        c = lambda x: x.double().cpu().numpy()  # noqa: E731
        slots = [s if live is None or live[i] else -1 for i, s in enumerate(self.slots)]
        self.trace = {}
        return plain.delta_rule(c(self.q), c(self.k), c(self.v), c(self.alpha), c(self.beta), c(self.states), self.ranges, slots, self.fresh, self.trace), slots

    def check(self, ref, slots, memory=20):
        (out, states), got, got_s = ref, self.out.double().cpu().numpy(), self.states.double().cpu().numpy()
        half = torch.finfo(DT[self.dtype]).eps / 2
        q, k = self.q.double().cpu().numpy(), self.k.double().cpu().numpy()
        g = got.shape[1] // q.shape[1]

        def rounding(a, t, h):           # of bf16 outputs in the chunked form
            if self.dtype != "bf16" or not self.chunked:
                return 0.0
            first = a + (t - a) // 64 * 64
            dots = (q[t, h // g] * k[first:t + 1, h // g]).sum(-1)
            deltas = np.array([self.trace[j][1][h] for j in range(first, t + 1)])
            terms = self.trace[first][0][h] ** 2 * (q[t, h // g] ** 2).sum() / q.shape[-1] + 2 * (dots ** 2 * deltas ** 2).sum()
            return 3 * 2.0 ** -11 / np.sqrt(3) * np.sqrt(terms)
        for i, (a, b) in enumerate(self.ranges):
            if slots[i] < 0:
                continue
            tol = 16 * min(max(b - a, 1), memory) * 2.0 ** -24
            for t in range(a, b):
                for h in range(got.shape[1]):
                    err = np.maximum(np.abs(got[t, h] - out[t][h]) - half * np.abs(out[t][h]), 0)
                    assert np.linalg.norm(err) <= tol * max(np.linalg.norm(out[t][h]), np.linalg.norm(states[slots[i], h]) / np.sqrt(got_s.shape[-1])) + rounding(a, t, h), (i, t, h)
            for h in range(got.shape[1]):
                assert np.linalg.norm(got_s[slots[i], h] - states[slots[i], h]) <= tol * np.linalg.norm(states[slots[i], h]) , (i, h)
        rows = {t for i, (a, b) in enumerate(self.ranges) if slots[i] >= 0 for t in range(a, b)}
        for t in range(got.shape[0]):
            if t not in rows:
                assert np.all(got[t] == UNTOUCHED), t
        used = {s for s in slots if s >= 0}
        for s in range(got_s.shape[0]):
            if s not in used:
                assert np.array_equal(got_s[s], states[s]), s


def _case(lens, max_tokens=0, memory=20, **kw):
    b = Batch(lens, **kw)
    ref, slots = b.reference()
    b.run(max_tokens)
    torch.cuda.synchronize()
    b.check(ref, slots, memory)
    assert b.status.tolist() == [0, 0]
    return b


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 64), (128, 128), (128, 256), (256, 256), (256, 512), (64, 96), (32, 160)])
@pytest.mark.parametrize("lens", [[1, 1, 1], [1, 3, 0, 7]])
def test_single_tokens_and_short_runs(dk, dv, dtype, lens):
    _case(lens, max_tokens=max(lens), dk=dk, dv=dv, dtype=dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,Hv", [(1, 1), (2, 4), (3, 9), (4, 4)])
def test_grouped_heads(H, Hv, dtype):
    _case([2, 5, 1], max_tokens=5, H=H, Hv=Hv, dk=128, dv=128, dtype=dtype)


def test_a_batch_that_fills_the_gpu():
    _case([1] * 40, max_tokens=1, H=8, Hv=16, dk=128, dv=128, dtype="bf16", slots=list(range(39, -1, -1)), fresh=[i % 3 == 0 for i in range(40)])


@pytest.mark.parametrize("max_tokens", [1, 0])
def test_padding_fresh_and_unused_states(max_tokens):
    _case([2, 0, 3, 1, 0, 90], max_tokens=max_tokens, slots=[5, 1, -1, 0, 7, 2], fresh=[0, 1, 0, 1, 0, 1], dk=128, dv=128, dtype="bf16")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 64), (64, 128), (128, 64), (128, 128), (128, 256), (256, 256), (128, 96)])
@pytest.mark.parametrize("lens", [[64], [65], [127, 1, 200], [300, 0, 17]])
def test_prompts(dk, dv, dtype, lens):
    _case(lens, dk=dk, dv=dv, dtype=dtype, fresh=[i % 2 for i in range(len(lens))])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_prompts_with_grouped_heads(dtype):
    _case([130, 70], H=2, Hv=6, dk=128, dv=128, dtype=dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("gates,memory", [((1.0, 1.0), 200), ((0.0, 1.0), 20), ((0.0, 0.0), 20), ((0.5, 0.6), 20)])
def test_gates(dtype, gates, memory):
    _case([200, 64], dk=128, dv=128, dtype=dtype, gates=gates, memory=memory)


@pytest.mark.parametrize("max_tokens", [1, 0])
def test_both_kernels_agree_with_the_recurrence_when_the_hint_is_wrong(max_tokens):
    """max_tokens chooses a kernel; results hold whatever it says."""
    _case([150, 1, 33], max_tokens=max_tokens, dk=128, dv=128, dtype="bf16")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dk,dv,H", [(128, 128, 2), (64, 64, 1), (64, 128, 2), (128, 64, 1), (32, 32, 3), (64, 96, 1)])
@pytest.mark.parametrize("lens,fresh", [([2500], [0]), ([1300, 40, 0, 2111], [1, 0, 1, 0])])
def test_long_prompts_of_few_heads(dk, dv, H, lens, fresh, dtype):
    """Sequences that are cut into segments, beside ones that are too short for it."""
    _case(lens, dk=dk, dv=dv, H=H, dtype=dtype, fresh=fresh, slots=[len(lens) - i for i in range(len(lens))])


@pytest.mark.parametrize("gates,memory", [((1.0, 1.0), 1500), ((0.98, 1.0), 200), ((0.0, 1.0), 20)])
def test_gates_of_long_prompts(gates, memory):
    for dtype in ("fp32", "bf16"):
        _case([1500], dk=128, dv=128, H=2, dtype=dtype, gates=gates, memory=memory)


@pytest.mark.parametrize("H,N", [(2, 1500), (40, 400)])
def test_states_that_fade_away_and_come_back(H, N):
    """Gates of about 0.4 and no values for most of the sequence: the state passes every exponent down to nothing (and so does the map of a segment),
    then values come again."""
    b = Batch([N], H=H, dk=128, dv=128, dtype="fp32", gates=(0.3, 0.5))
    b.v[:N - 90] = 0
    ref, slots = b.reference()
    b.run()
    torch.cuda.synchronize()
    assert torch.isfinite(b.out).all() and torch.isfinite(b.states).all()
    tail = {t: o for t, o in ref[0].items() if t >= N - 80}
    got = b.out.double().cpu().numpy()
    for t, o in tail.items():
        for h in range(0, H, 7):
            assert np.linalg.norm(got[t, h] - o[h]) <= 16 * 20 * 2.0 ** -24 * max(np.linalg.norm(o[h]), np.linalg.norm(ref[1][0, h]) / np.sqrt(128)), (t, h)
    assert np.linalg.norm(b.states[0].double().cpu().numpy() - ref[1][0]) <= 16 * 20 * 2.0 ** -24 * np.linalg.norm(ref[1][0])


def test_cut_prompts_in_strided_outputs_and_captured():
    """The segments' states lie in the rows of `out` meanwhile: what lies between the rows is not touched, and a replay does the same work."""
    b = Batch([1700, 90], H=2, dk=128, dv=128, dtype="bf16")
    ref, slots = b.reference()
    N = b.q.shape[0]
    outs = torch.full((N, 6, 128), UNTOUCHED, dtype=torch.bfloat16, device="cuda")
    b.out, first = outs[:, 2:4], b.states.clone()
    b.run()
    torch.cuda.synchronize()
    b.check(ref, slots)
    assert torch.all(outs[:, :2] == UNTOUCHED) and torch.all(outs[:, 4:] == UNTOUCHED)
    want = [b.out.clone(), b.states.clone()]
    args = dict(starts=b.starts, slots=b.i32(b.slots))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.run(**args)
    for _ in range(3):
        b.states.copy_(first)
        b.out.fill_(5.0)
        b.out[1790:] = UNTOUCHED
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.out, want[0]) and torch.equal(b.states, want[1])


def test_no_starts_no_slots():
    b = Batch([1] * 5, extra_rows=0, extra_states=0, dk=128, dv=128, dtype="bf16")
    ref, slots = b.reference()
    b.run(starts=None, slots=None, fresh=None, status=None)
    torch.cuda.synchronize()
    b.check(ref, slots)


@pytest.mark.parametrize("max_tokens", [1, 0])
def test_strided_inputs_and_states(max_tokens):
    b = Batch([70, 3], H=2, dk=64, dv=64, dtype="bf16")
    ref, slots = b.reference()
    N, S = b.q.shape[0], b.states.shape[0]
    packed = torch.zeros((N, 8, 64), dtype=torch.bfloat16, device="cuda")
    packed[:, 0:2], packed[:, 2:4], packed[:, 4:6] = b.q, b.k, b.v
    gates = torch.zeros((N, 5), device="cuda")
    gates[:, 0:2], gates[:, 3:5] = b.alpha, b.beta
    pool = torch.full((S, 3, 2, 64, 64), UNTOUCHED, device="cuda")      # [slot][layer][head]..: layer 1 of three
    pool[:, 1] = b.states
    outs = torch.full((N, 5, 64), UNTOUCHED, dtype=torch.bfloat16, device="cuda")
    b.q, b.k, b.v, b.alpha, b.beta, b.states, b.out = packed[:, 0:2], packed[:, 2:4], packed[:, 4:6], gates[:, 0:2], gates[:, 3:5], pool[:, 1], outs[:, 1:3]
    b.run(max_tokens)
    torch.cuda.synchronize()
    b.check(ref, slots)
    assert torch.all(pool[:, 0] == UNTOUCHED) and torch.all(pool[:, 2] == UNTOUCHED) and torch.all(outs[:, 0] == UNTOUCHED) and torch.all(outs[:, 3:] == UNTOUCHED)


@pytest.mark.parametrize("max_tokens", [1, 0])
@pytest.mark.parametrize("what", ["slot", "twice", "backwards", "behind", "overlap"])
def test_bad_slots_and_ranges_are_reported_and_left_alone(what, max_tokens):
    b = Batch([3, 66, 2, 5], dk=128, dv=128, dtype="bf16")
    live, starts, bad = [True] * 4, b.starts.tolist(), 2
    ranges = list(b.ranges)
    if what == "slot":
        b.slots[2] = b.states.shape[0]
    elif what == "twice":
        b.slots[2] = b.slots[0]
    elif what == "backwards":           # sequence 2 ends before it begins; sequence 3 then begins before an earlier one
        starts[3] = starts[2] - 1
        live[3] = False
    elif what == "behind":
        starts[4] = b.q.shape[0] + 1
        bad = 3
    else:
        starts[1] = starts[2] + 2       # sequence 1 runs backwards, sequence 2 begins before it
        ranges[0] = (starts[0], starts[1])
        live[2], bad = False, 1
    live[bad] = False
    b.starts = b.i32(starts)
    keep, b.ranges = b.ranges, [ranges[i] if live[i] else (0, 0) for i in range(4)]
    slots = [s if live[i] else -1 for i, s in enumerate(b.slots)]
    want_slots, b.slots = b.slots, slots
    ref, _ = b.reference()
    b.slots = want_slots
    b.run(max_tokens)
    torch.cuda.synchronize()
    code, at = b.status.tolist()
    assert code == P.binding.E_DEVICE_CHECK and not live[at], (code, at)
    b.slots = slots
    b.check(ref, slots)


@pytest.mark.parametrize("max_tokens", [1, 0])
def test_streams_and_graph_replays(max_tokens):
    """A captured call replayed twice continues from the state that the first replay left, as two calls do."""
    a, b = (Batch([70, 2, 1], dk=128, dv=128, dtype="bf16", seed=3) for _ in range(2))
    a.run(max_tokens); a.run(max_tokens)
    args = dict(starts=b.starts, slots=b.i32(b.slots), fresh=b.i32(b.fresh))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.run(max_tokens, **args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g.replay(); g.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.out, b.out) and torch.equal(a.states, b.states)


def test_long_keys_and_strong_gates():
    """Keys of norm 1.4 and beta in (0, 1): delta overshoots, the state stays bounded (|1 - beta k.k| <= 1)."""
    for dtype in ("fp32", "bf16"):
        _case([180], dk=128, dv=128, dtype=dtype, key_norm=1.4, memory=64)


def test_pieces_of_a_prompt_give_what_the_whole_gives():
    """Continuing from the stored state: 200 tokens at once and as 128 + 1 + 71."""
    whole = _case([200], dk=128, dv=128, dtype="bf16", seed=5)
    parts = Batch([200], dk=128, dv=128, dtype="bf16", seed=5)
    at = 0
    for n in (128, 1, 71):
        P.onela_delta_rule(*(x[at:at + n] for x in (parts.q, parts.k, parts.v, parts.alpha, parts.beta)), parts.states, parts.out[at:at + n],
                           starts=parts.i32([0, n]), slots=parts.i32([0]), max_tokens=n)
        at += n
    torch.cuda.synchronize()
    err = (whole.states[0] - parts.states[0]).norm() / whole.states[0].norm()
    assert err <= 2 * 16 * 20 * 2.0 ** -24                   # (both within the tolerance of the exact one)
