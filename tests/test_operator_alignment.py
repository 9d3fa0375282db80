"""Arrays of single numbers (gates, positions, slots, temperatures ..) that do not lie on 4-byte boundaries: a kernel would fault on them, the host refuses.  No GPU
needed: every call here is refused."""
import ctypes

import pytest

from paper_2609_12399_b200 import binding
from test_operator_refusals import A, _delta, _norm, _sample, lib  # noqa: F401

# (calls that pass every other check reach the launch: without a GPU they would return ONELA_E_CUDA)


@pytest.mark.parametrize("by", [1, 2, 3])
@pytest.mark.parametrize("field", ["positions", "inv_freq"])
def test_norm_rotate(lib, field, by):  # noqa: F811
    args = dict(rotary_dim=64, positions=9 * A, inv_freq=10 * A)
    args[field] += by
    assert lib.onela_norm_rotate(ctypes.byref(_norm(**args)), None) == binding.E_INVAL


@pytest.mark.parametrize("by", [1, 2, 3])
@pytest.mark.parametrize("field", ["alpha", "beta", "starts", "slots", "fresh", "status"])
def test_delta_rule(lib, field, by):  # noqa: F811
    """(Without sequences the call has nothing to do, and so passes where the field is on its boundary.)"""
    assert lib.onela_delta_rule(ctypes.byref(_delta(num_sequences=0, **{field: 8 * A})), None) == 0
    assert lib.onela_delta_rule(ctypes.byref(_delta(num_sequences=0, **{field: 8 * A + by})), None) == binding.E_INVAL


@pytest.mark.parametrize("by", [1, 2, 3])
@pytest.mark.parametrize("field", ["uniforms", "temperature", "top_p", "min_p", "top_k", "tokens_out", "logprobs_out"])
def test_sample_tokens(lib, field, by):  # noqa: F811
    assert lib.onela_sample_tokens(ctypes.byref(_sample(**{field: 8 * A + by})), None) == binding.E_INVAL


@pytest.mark.parametrize("kw", [
    dict(q=0), dict(k=A + 8), dict(v_stride=508), dict(q_stride=260), dict(out=0), dict(alpha=0), dict(gate_stride=3), dict(states=0), dict(state_stride=128 * 128),
    dict(starts=0), dict(slots=0, num_states=2), dict(out=A), dict(out=3 * A), dict(out=2 * A + 256, out_stride=768), dict(states=3 * A + 512), dict(states=7 * A),
])
def test_delta_rule_with_one_thing_wrong(lib, kw):  # noqa: F811
    """The calls of test_operator_refusals with states (1.3 MB) that overlap nothing otherwise."""
    assert lib.onela_delta_rule(ctypes.byref(_delta(**{"states": 64 * A, **kw})), None) == binding.E_INVAL
