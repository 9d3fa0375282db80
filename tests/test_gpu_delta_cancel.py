"""onela_delta_rule with bf16 outputs that are small differences: a query along a key that the token writes over, o = S k + (v - S k), and outputs of
states that have faded.  Rounding S, D or P to fewer bits than fp32 products have shows there, and nowhere with independent queries and keys.  Bounds as in
test_gpu_delta_range: componentwise 2^-17 of the terms, half a step of the type."""
import pytest
import torch

from test_gpu_delta_range import SHAPES, _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("max_tokens", [1, 0])
@pytest.mark.parametrize("dk,dv", SHAPES)
@pytest.mark.parametrize("size", [30.0, 1000.0])
def test_a_query_along_a_key_that_is_written_over(size, dk, dv, max_tokens, dtype):
    x = _inputs(100, dk=dk, dv=dv, seed=11)
    x["q"][:] = x["k"]
    x["beta"][:] = 1
    x["S"] *= size
    _check(**x, dtype=dtype, max_tokens=max_tokens)


@pytest.mark.parametrize("max_tokens", [1, 0])
@pytest.mark.parametrize("dk,dv", SHAPES)
@pytest.mark.parametrize("alpha", [0.8, 0.6, 0.45])
@pytest.mark.parametrize("beta", [0.0, 0.5])
def test_faded_outputs_in_bf16(dk, dv, alpha, beta, max_tokens):
    x = _inputs(100, dk=dk, dv=dv)
    x["alpha"][:] = alpha
    x["beta"][1:] = beta
    x["v"][1:] = 0
    _check(**x, dtype="bf16", max_tokens=max_tokens)


@pytest.mark.parametrize("max_tokens", [1, 0])
@pytest.mark.parametrize("dk,dv", SHAPES)
@pytest.mark.parametrize("alpha", [-1.2, -1.0, 0.95])
def test_usual_and_alternating_outputs_in_bf16(dk, dv, alpha, max_tokens):
    """Outputs of a state that is not small either: off by the rounding to bf16 and no more."""
    x = _inputs(64, dk=dk, dv=dv, seed=12)
    x["alpha"][:] = alpha
    x["alpha"][5::7] = 0.3
    _check(**x, dtype="bf16", max_tokens=max_tokens)
