"""A map of a cut sequence that was given up (a second build of the library: one CTA of the maps' launch, its work done, says that a wait ran out): the launches
behind it, already queued, must not make a state of whatever lies in its place.  The call reports ONELA_E_TIMEOUT and leaves that head's state alone; other heads and
sequences, and the next call, are right.  In a child process, so that the product library and the test-hooks library never share one."""
import subprocess
import sys
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent


def _child():
    import ctypes

    import torch

    sys.path.insert(0, str(ROOT))
    import paper_2609_12399_b200 as P
    from paper_2609_12399_b200 import binding, build

    binding.LIB_PATH = build.build_testhooks()
    lib = binding.load_library()
    lib.onela_testhook_delta_map_fails.restype = ctypes.c_int
    lib.onela_testhook_delta_map_fails.argtypes = [ctypes.c_int]
    for d, dtype in ((128, torch.bfloat16), (64, torch.float32)):
        gen = torch.Generator(device="cuda").manual_seed(3)
        rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
        unit = lambda x: x / torch.linalg.vector_norm(x, dim=-1, keepdim=True)  # noqa: E731
        n, H = 2500, 2
        q, k, v = unit(rand(2 * n, H, d)).to(dtype), unit(rand(2 * n, H, d)).to(dtype), rand(2 * n, H, d).to(dtype)
        alpha, beta = 1 - 0.1 * torch.rand((2 * n, H), generator=gen, device="cuda"), torch.sigmoid(rand(2 * n, H))
        first = 0.3 * rand(2, H, d, d)
        starts = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")

        def run(part, fill):
            states, out, status = first.clone(), torch.full_like(v, fill), torch.zeros(2, dtype=torch.int32, device="cuda")
            assert lib.onela_testhook_delta_map_fails(part) == 0
            P.onela_delta_rule(q, k, v, alpha, beta, states, out, starts=starts, max_tokens=n, status=status)
            torch.cuda.synchronize()
            assert lib.onela_testhook_delta_map_fails(0) == 0
            return states, out, tuple(status.tolist())

        want, out, status = run(0, 0.0)
        assert status == (0, 0) and not torch.equal(want, first)
        for part in range(1, 64):                    # B of every segment, then M
            for fill in (0.0, 1.0):
                states, got, status = run(part, fill)
                if status == (0, 0):
                    break
                assert torch.equal(states[1], want[1]) and torch.equal(states[0, 1], want[0, 1]), (d, part)
                assert torch.equal(got[n:], out[n:]) and torch.equal(got[:n, 1], out[:n, 1]), (d, part)
                assert status == (binding.E_TIMEOUT, 0), (d, part, status)
                assert torch.equal(states[0, 0], first[0, 0]), (d, part)
            if status == (0, 0):
                break
        assert part > 3                              # (three segments or more: B of two or more, M of one or more)
        states, got, status = run(0, 2.0)
        assert status == (0, 0) and torch.equal(states, want) and torch.equal(got, out)
    print("reported, and the state left alone")


@pytest.mark.gpu
def test_a_map_that_was_given_up_makes_no_state():
    r = subprocess.run([sys.executable, __file__], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "reported, and the state left alone" in r.stdout


if __name__ == "__main__":
    _child()
