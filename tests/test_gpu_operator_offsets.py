"""Tensors in which offsets pass 32 bits: pools of states, logits and strided tokens of more than 2^31 elements."""
import numpy as np
import pytest
import torch

import paper_2609_12399_b200 as P
from oracle import operators as plain

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("tokens", [1, 70])
def test_state_pool(tokens):
    H, d, slots = 4, 128, 33500                                 # 2.2e9 floats
    gen = torch.Generator(device="cuda").manual_seed(1)
    u = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    q, k = (u(torch.randn((2 * tokens, H, d), generator=gen, device="cuda")) for _ in range(2))
    v = torch.randn((2 * tokens, H, d), generator=gen, device="cuda")
    a, b = 0.9 + 0.1 * torch.rand((2 * tokens, H), generator=gen, device="cuda"), torch.rand((2 * tokens, H), generator=gen, device="cuda")
    pool = torch.empty((slots, H, d, d), device="cuda")
    pool[0], pool[-1] = 0.1, torch.randn((H, d, d), generator=gen, device="cuda")
    c = lambda t: t.double().cpu().numpy()  # noqa: E731
    ref, states = plain.delta_rule(c(q), c(k), c(v), c(a), c(b), np.stack([c(pool[0]), c(pool[-1])]), [(0, tokens), (tokens, 2 * tokens)], [1, 0], [0, 0])
    out = torch.empty_like(v)
    P.onela_delta_rule(q, k, v, a, b, pool, out, starts=torch.tensor([0, tokens, 2 * tokens], dtype=torch.int32, device="cuda"),
                       slots=torch.tensor([slots - 1, 0], dtype=torch.int32, device="cuda"), max_tokens=tokens)
    torch.cuda.synchronize()
    tol = 16 * 20 * 2.0 ** -24                                  # (see test_gpu_delta.py)
    for i, s in ((0, pool[0]), (1, pool[-1])):
        assert np.linalg.norm(c(s) - states[i]) <= tol * np.linalg.norm(states[i])
    assert np.linalg.norm(c(out) - np.stack([ref[t] for t in range(2 * tokens)])) <= tol * np.linalg.norm(c(out))


def test_logits():
    R, V = 8700, 250000                                         # 2.2e9
    x = torch.zeros((R, V), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)
    x[-1] = torch.randn((V,), generator=gen, device="cuda")
    u = torch.rand((R,), generator=gen, device="cuda")
    tok = torch.empty((R,), dtype=torch.int32, device="cuda")
    P.onela_sample_tokens(x, u, tok, top_p=torch.full((R,), 0.9, device="cuda"))
    torch.cuda.synchronize()
    for i in (0, R // 2, R - 1):
        want, _, border = plain.sample_row(x[i].float().cpu().numpy(), float(u[i]), 1.0, 0, float(np.float32(0.9)))
        assert border < 1e-9 or int(tok[i]) == want


def test_tokens_far_apart():
    n, h, d, stride = 3, 2, 64, (1 << 30) + 64
    room = torch.empty((2 * stride + 4 * h * d,), dtype=torch.bfloat16, device="cuda")
    q, k, qo, ko = (room.as_strided((n, h, d), (stride, d, 1), i * h * d) for i in range(4))
    gen = torch.Generator(device="cuda").manual_seed(3)
    q.copy_(torch.randn((n, h, d), generator=gen, device="cuda"))
    k.copy_(torch.randn((n, h, d), generator=gen, device="cuda"))
    P.onela_norm_rotate(q, k, qo, ko)
    want = [torch.empty((n, h, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    P.onela_norm_rotate(q.contiguous(), k.contiguous(), *want)
    torch.cuda.synchronize()
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
