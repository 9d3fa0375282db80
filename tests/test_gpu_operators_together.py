"""The operators around the beam decode as a server uses them: prompts through a layer (head norms, the gated delta rule in chunks), the states handed
to the beam decode; and sampled generation token by token."""
import numpy as np
import pytest
import torch

import paper_2609_12399_b200 as P
from oracle import operators as plain

from _cases import REL_L2_BAR

pytestmark = pytest.mark.gpu


def test_prompts_through_a_layer_then_beams_on_their_states():
    R, H, d, W = 3, 2, 128, 40
    lens = [150, 64, 77]
    gen = torch.Generator(device="cuda").manual_seed(1)
    N = sum(lens)
    x = torch.randn((N, 3 * H * d), generator=gen, device="cuda").bfloat16()
    q, k, v = (x[:, i * H * d:(i + 1) * H * d].view(N, H, d) for i in range(3))
    alpha, beta = 0.9 + 0.1 * torch.rand((N, H), generator=gen, device="cuda"), torch.rand((N, H), generator=gen, device="cuda")
    starts = torch.tensor(np.concatenate(([0], np.cumsum(lens))), dtype=torch.int32, device="cuda")
    P.onela_norm_rotate(q, k, q, k, norm="l2", q_scale=d ** -0.5)                      # in the projection's own memory
    states, out = torch.zeros((R, H, d, d), device="cuda"), torch.empty((N, H, d), dtype=torch.bfloat16, device="cuda")
    P.onela_delta_rule(q, k, v, alpha, beta, states, out, starts=starts, max_tokens=max(lens))
    c = lambda t: t.double().cpu().numpy()  # noqa: E731
    s = starts.tolist()
    ref_out, ref_states = plain.delta_rule(c(q), c(k), c(v), c(alpha), c(beta), np.zeros((R, H, d, d)), list(zip(s[:-1], s[1:])), range(R), [0] * R)
    for t in range(N):
        assert np.linalg.norm(c(out[t]) - ref_out[t]) <= REL_L2_BAR * np.linalg.norm(ref_out[t])
    # beams on the states: the library's prefill of the same tokens leaves the same states, and a decode call of W beams reads them
    ctx = P.Onela(P.make_config(R, 1, H, d, d, W, 2, "bf16", "fp32", R * W * 2, 0))
    ctx.onela_init_shared_states(0, R, states.view(R, 1, H, d, d))
    other = P.Onela(P.make_config(R, 1, H, d, d, W, 2, "bf16", "fp32", R * W * 2, 0))
    for r in range(R):
        rows = slice(s[r], s[r + 1])
        other.onela_prefill_shared_state(r, 0, k[rows].contiguous(), v[rows].contiguous(), alpha[rows].contiguous(), beta[rows].contiguous())
        a, b = ctx.onela_export_shared_state(r, 0), other.onela_export_shared_state(r, 0)
        torch.cuda.synchronize()
        assert (a - b).norm() <= 1e-5 * b.norm()                                        # (both within 2e-5 / 4 of the exact one)
    kd, vd = torch.randn((R, W, H, d), generator=gen, device="cuda"), torch.randn((R, W, H, d), generator=gen, device="cuda").bfloat16()
    qd = torch.randn((R, W, H, d), generator=gen, device="cuda").bfloat16()
    kd = (kd / kd.norm(dim=-1, keepdim=True)).bfloat16()
    ad, bd = 0.9 + 0.1 * torch.rand((R, W, H), generator=gen, device="cuda"), torch.rand((R, W, H), generator=gen, device="cuda")
    od = torch.empty((R, W, H, d), device="cuda")
    ctx.onela_reorder_beams(0, R, None, W)
    ctx.onela_append_decode_step(0, R, 0, kd, vd, ad, bd, qd, od)
    torch.cuda.synchronize()
    for r in range(R):
        for w in range(W):
            S = ref_states[r] * c(ad[r, w])[:, None, None]
            delta = c(bd[r, w])[:, None] * (c(vd[r, w]) - np.einsum("hvk,hk->hv", S, c(kd[r, w])))
            o = np.einsum("hvk,hk->hv", S + delta[:, :, None] * c(kd[r, w])[:, None, :], c(qd[r, w]))
            for h in range(H):
                assert np.linalg.norm(c(od[r, w, h]) - o[h]) <= REL_L2_BAR * np.linalg.norm(o[h])


@pytest.mark.parametrize("captured", [False, True])
def test_sampled_generation(captured):
    """Six tokens for five sequences of a one-layer model with random weights.  Every step's outputs are those of Eq. 1 in 64 bits on the tokens
    that were drawn, and every token is the one that the plain form draws from the step's own logits."""
    n, H, d, V, steps = 5, 4, 64, 5003, 6
    gen = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    table = rand(V, 3 * H * d)                                                         # token -> q, k, v before their norms
    gates = torch.rand((V, 2 * H), generator=gen, device="cuda")
    head = rand(H * d, V) / 4
    uniforms = torch.rand((steps, n), generator=gen, device="cuda")
    temperature, top_p = torch.full((n,), 0.8, device="cuda"), torch.full((n,), 0.9, device="cuda")
    top_k = torch.tensor([0, 5, 50, 500, 5000], dtype=torch.int32, device="cuda")
    states = torch.zeros((n + 1, H, d, d), device="cuda")
    slots = torch.tensor([3, 0, 5, 1, 4], dtype=torch.int32, device="cuda")
    token, lp = torch.arange(n, dtype=torch.int32, device="cuda"), torch.empty((n,), device="cuda")
    u, out = torch.empty((n,), device="cuda"), torch.empty((n, H, d), device="cuda")
    qk, logits = torch.empty((2, n, H, d), device="cuda"), torch.empty((n, V), device="cuda")
    row = torch.empty((n, 3 * H * d), device="cuda")
    alpha, beta = torch.empty((n, H), device="cuda"), torch.empty((n, H), device="cuda")

    def step():
        at = token.long()
        row.copy_(table[at])
        alpha.copy_(0.8 + 0.2 * gates[at, :H])
        beta.copy_(gates[at, H:])
        q, k, v = (row[:, i * H * d:(i + 1) * H * d].view(n, H, d) for i in range(3))
        P.onela_norm_rotate(q, k, qk[0], qk[1])
        P.onela_delta_rule(qk[0], qk[1], v, alpha, beta, states, out, slots=slots)
        torch.matmul(out.view(n, H * d), head, out=logits)
        P.onela_sample_tokens(logits, u, token, temperature=temperature, top_k=top_k, top_p=top_p, logprobs_out=lp)

    graph = None
    if captured:
        keep = token.clone()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        token.copy_(keep)
        states.zero_()
    c = lambda t: t.double().cpu().numpy()  # noqa: E731
    S = np.zeros((n + 1, H, d, d))
    for t in range(steps):
        before = token.clone()
        u.copy_(uniforms[t])
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        x = c(table[before.long()]).reshape(n, 3, H, d)
        q, k = (y / np.sqrt((y * y).sum(-1, keepdims=True) + 1e-6) for y in (x[:, 0], x[:, 1]))
        ref, S = plain.delta_rule(q, k, x[:, 2], c(alpha), c(beta), S, [(i, i + 1) for i in range(n)], slots.tolist(), [0] * n)
        for i in range(n):
            # fp32 throughout: 16 roundings of 2^-24 per token so far, and the norms' 12
            assert np.linalg.norm(c(out[i]) - ref[i]) <= 28 * (t + 1) * 2.0 ** -24 * max(np.linalg.norm(ref[i]), np.linalg.norm(S[slots[i]]) / 8)
            want, logprob, border = plain.sample_row(logits[i].cpu().numpy(), float(u[i]), float(np.float32(0.8)), int(top_k[i]), float(np.float32(0.9)))
            assert border > 1e-9 and int(token[i]) == want
            assert abs(float(lp[i]) - logprob) <= 2.0 ** -24 * abs(logprob) + 2.0 ** -25


def test_no_tokens_and_no_states():
    """Sequences without a token: a fresh one gets the zero state, the others keep theirs; a batch of padding alone touches nothing."""
    e = torch.empty((0, 2, 64), device="cuda")
    g = torch.empty((0, 2), device="cuda")
    states = torch.ones((3, 2, 64, 64), device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for longest in (1, 100):
        states.fill_(1.0)
        P.onela_delta_rule(e, e.clone(), e.clone(), g, g.clone(), states, e.clone(), starts=i32([0, 0, 0]), slots=i32([2, 0]), fresh=i32([1, 0]), max_tokens=longest)
        torch.cuda.synchronize()
        assert torch.all(states[2] == 0) and torch.all(states[:2] == 1)
    x = torch.randn((2, 2, 64), device="cuda")
    out = torch.full_like(x, 7.0)
    status = i32([0, 0])
    P.onela_delta_rule(x, x.clone(), x.clone(), x[..., 0].contiguous(), x[..., 1].contiguous(), states[:0], out, slots=i32([-1, -1]), status=status)
    torch.cuda.synchronize()
    assert torch.all(out == 7) and status.tolist() == [0, 0]
    P.onela_delta_rule(x, x.clone(), x.clone(), x[..., 0].contiguous(), x[..., 1].contiguous(), states[:0], out, slots=i32([-1, 0]), status=status)
    torch.cuda.synchronize()
    assert torch.all(out == 7) and status.tolist() == [P.binding.E_DEVICE_CHECK, 1]


def test_calls_on_two_streams_at_once():
    """No call shares memory with another: the same work on two streams, interleaved, twenty times, gives the same bits."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    sets = []
    for _ in range(2):
        N, H, d = 200, 8, 128
        u = lambda t: t / t.norm(dim=-1, keepdim=True)  # noqa: E731
        q, k = (u(torch.randn((N, H, d), generator=gen, device="cuda")).bfloat16() for _ in range(2))
        v = torch.randn((N, H, d), generator=gen, device="cuda").bfloat16()
        a, b = 0.9 + 0.1 * torch.rand((N, H), generator=gen, device="cuda"), torch.rand((N, H), generator=gen, device="cuda")
        x, un = torch.randn((9, 40001), generator=gen, device="cuda"), torch.rand((9,), generator=gen, device="cuda")
        sets.append(dict(args=(q, k, v, a, b), states=torch.zeros((2, H, d, d), device="cuda"), out=torch.empty_like(v), x=x, u=un, tok=torch.zeros(9, dtype=torch.int32, device="cuda"),
                         starts=torch.tensor([0, 130, 200], dtype=torch.int32, device="cuda"), fresh=torch.ones(2, dtype=torch.int32, device="cuda"), p=torch.full((9,), 0.9, device="cuda")))

    def work(s, stream=None):
        P.onela_delta_rule(*s["args"], s["states"], s["out"], starts=s["starts"], fresh=s["fresh"], max_tokens=130, stream=stream)
        P.onela_sample_tokens(s["x"], s["u"], s["tok"], top_p=s["p"], stream=stream)

    for s in sets:
        work(s)
    torch.cuda.synchronize()
    want = [[s[n].clone() for n in ("out", "states", "tok")] for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(20):
        for s, st in zip(sets, streams):
            work(s, st)
    torch.cuda.synchronize()
    for s, w in zip(sets, want):
        assert all(torch.equal(s[n], x) for n, x in zip(("out", "states", "tok"), w))
