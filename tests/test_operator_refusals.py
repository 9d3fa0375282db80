"""What the operators around the beam decode refuse, seen by the host before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2609_12399_b200 as P
from paper_2609_12399_b200 import binding, build

A = 1 << 20          # addresses that are never touched: every call here is refused, or has nothing to do


@pytest.fixture(scope="module")
def lib():
    build.build()
    return P.load_library()


def _norm(**kw):
    d = dict(q=A, k=2 * A, q_out=3 * A, k_out=4 * A, q_stride=512, k_stride=256, q_out_stride=512, k_out_stride=256, n_tokens=4, num_q_heads=4, num_k_heads=2,
             head_dim=128, norm=P.NORM_L2, dtype=P.DTYPE_BF16, eps=1e-6, q_scale=1.0)
    return binding.NormRotateArgs(**{**d, **kw})


def _delta(**kw):
    d = dict(q=A, k=2 * A, v=3 * A, alpha=4 * A, beta=5 * A, states=6 * A, out=7 * A, starts=8 * A, slots=9 * A, q_stride=256, k_stride=256, v_stride=512, out_stride=512,
             gate_stride=4, state_stride=4 * 128 * 128, n_tokens=10, num_sequences=3, num_states=5, num_heads=2, num_v_heads=4, dk=128, dv=128, dtype=P.DTYPE_BF16)
    return binding.DeltaRuleArgs(**{**d, **kw})


def _sample(**kw):
    d = dict(logits=A, uniforms=2 * A, tokens_out=3 * A, logits_stride=1000, rows=2, vocab=1000, dtype=P.DTYPE_F32)
    return binding.SampleArgs(**{**d, **kw})


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), binding.E_INVAL), (dict(k_out=0), binding.E_INVAL), (dict(q=A + 2), binding.E_INVAL), (dict(q_stride=511), binding.E_INVAL),
    (dict(q_stride=516), binding.E_INVAL), (dict(n_tokens=-1), binding.E_INVAL), (dict(num_q_heads=-1), binding.E_INVAL), (dict(dtype=2), binding.E_INVAL),
    (dict(norm=3), binding.E_INVAL), (dict(eps=-1.0), binding.E_INVAL), (dict(eps=float("nan")), binding.E_INVAL), (dict(head_dim=132), binding.E_UNSUPPORTED),
    (dict(head_dim=264), binding.E_UNSUPPORTED), (dict(head_dim=0), binding.E_INVAL), (dict(rotary_dim=24), binding.E_UNSUPPORTED), (dict(rotary_dim=144), binding.E_INVAL),
    (dict(rotary_dim=64), binding.E_INVAL), (dict(rotary_dim=64, positions=9 * A), binding.E_INVAL), (dict(q_weight=A + 4, norm=P.NORM_RMS), binding.E_INVAL),
    # outputs over inputs
    (dict(q_out=A + 16), binding.E_INVAL), (dict(k_out=A), binding.E_INVAL), (dict(q_out=2 * A - 1024), binding.E_INVAL), (dict(k_out=3 * A + 1024), binding.E_INVAL),
    (dict(q=A, q_stride=1024, q_out=A, q_out_stride=512), binding.E_INVAL),
    (dict(q_stride=1 << 50), binding.E_INVAL), (dict(n_tokens=1 << 45), binding.E_CAPACITY),
    (dict(num_q_heads=(1 << 20) + 1, q_stride=1 << 28), binding.E_CAPACITY), (dict(num_k_heads=(1 << 31) - 1), binding.E_CAPACITY),
    (dict(n_tokens=0), 0), (dict(num_q_heads=0, num_k_heads=0), 0),
])
def test_norm_rotate(lib, kw, status):
    assert lib.onela_norm_rotate(ctypes.byref(_norm(**kw)), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), binding.E_INVAL), (dict(k=A + 8), binding.E_INVAL), (dict(v_stride=508), binding.E_INVAL), (dict(q_stride=260), binding.E_INVAL), (dict(out=0), binding.E_INVAL),
    (dict(alpha=0), binding.E_INVAL), (dict(gate_stride=3), binding.E_INVAL), (dict(states=0), binding.E_INVAL), (dict(state_stride=128 * 128), binding.E_INVAL),
    (dict(num_heads=3), binding.E_INVAL), (dict(num_heads=0), binding.E_INVAL), (dict(num_v_heads=1), binding.E_INVAL), (dict(dk=96), binding.E_UNSUPPORTED),
    (dict(dk=512), binding.E_UNSUPPORTED), (dict(dv=48), binding.E_UNSUPPORTED), (dict(dv=544), binding.E_UNSUPPORTED), (dict(dv=0), binding.E_UNSUPPORTED),
    (dict(dtype=7), binding.E_INVAL), (dict(n_tokens=-1), binding.E_INVAL), (dict(num_sequences=-1), binding.E_INVAL), (dict(max_tokens=-1), binding.E_INVAL),
    (dict(starts=0), binding.E_INVAL), (dict(slots=0, num_states=2), binding.E_INVAL), (dict(num_sequences=70000), binding.E_CAPACITY),
    (dict(n_tokens=1 << 31), binding.E_CAPACITY), (dict(num_v_heads=65536), binding.E_CAPACITY), (dict(num_sequences=0), 0),
    # outputs and states over inputs and over one another
    (dict(out=A), binding.E_INVAL), (dict(out=3 * A), binding.E_INVAL), (dict(out=2 * A + 256, out_stride=768), binding.E_INVAL), (dict(states=3 * A + 512), binding.E_INVAL),
    (dict(states=7 * A), binding.E_INVAL),
])
def test_delta_rule(lib, kw, status):
    assert lib.onela_delta_rule(ctypes.byref(_delta(**kw)), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(logits=0), binding.E_INVAL), (dict(uniforms=0), binding.E_INVAL), (dict(tokens_out=0), binding.E_INVAL), (dict(logits=A + 2), binding.E_INVAL),
    (dict(logits_stride=999), binding.E_INVAL), (dict(vocab=0), binding.E_INVAL), (dict(rows=-1), binding.E_INVAL), (dict(dtype=2), binding.E_INVAL),
    (dict(vocab=360001, logits_stride=400000), binding.E_CAPACITY), (dict(rows=0), 0),
])
def test_sample_tokens(lib, kw, status):
    assert lib.onela_sample_tokens(ctypes.byref(_sample(**kw)), None) == status


@pytest.mark.parametrize("make,field", [(_norm, "num_q_heads"), (_norm, "rotary_dim"), (_delta, "num_sequences"), (_delta, "max_tokens"), (_sample, "vocab"), (_sample, "rows")])
def test_sizes_beyond_32_bits(make, field):
    """Cut off to 32 bits they would be small and pass."""
    make(**{field: 2 ** 31 - 1})
    for n in (2 ** 31, 2 ** 32 + 1, -2 ** 31 - 1):
        with pytest.raises(P.OnelaError, match=field):
            make(**{field: n})


def test_null_arguments(lib):
    for name in ("onela_norm_rotate", "onela_delta_rule", "onela_sample_tokens"):
        assert getattr(lib, name)(None, None) == binding.E_INVAL


def test_the_binding_names_what_is_wrong(lib):
    x = torch.zeros(3, 2, 64)
    with pytest.raises(ValueError, match="q: must live on the CUDA device"):
        P.onela_norm_rotate(x, x, x, x)
    with pytest.raises(TypeError, match="q: expected a torch tensor"):
        P.onela_norm_rotate([1], x, x, x)
    with pytest.raises(ValueError, match="float16"):
        P.onela_norm_rotate(x.half(), x.half(), x, x)
    with pytest.raises(ValueError, match="norm"):
        P.onela_norm_rotate(x, x, x, x, norm="layer")
    with pytest.raises(ValueError, match="go together"):
        P.onela_norm_rotate(x, x, x, x, positions=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="weights"):
        P.onela_norm_rotate(x, x, x, x, q_weight=torch.ones(64))
    with pytest.raises(ValueError, match="q: must live"):
        P.onela_delta_rule(x, x, x, x[..., 0], x[..., 0], torch.zeros(3, 2, 64, 64), x)
    with pytest.raises(ValueError, match="logits"):
        P.onela_sample_tokens(x, x[:, 0, 0], torch.zeros(3, dtype=torch.int32))


def test_structures_have_the_header_s_fields():
    """Field for field in the header's order (a binding that drifts would hand over garbage)."""
    import re
    from pathlib import Path
    text = re.sub(r"/\*.*?\*/", "", (Path(__file__).resolve().parent.parent / "include" / "onela.h").read_text(), flags=re.S)
    size = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "float": ctypes.c_float}
    for struct, cls in (("onela_norm_rotate_args", binding.NormRotateArgs), ("onela_delta_rule_args", binding.DeltaRuleArgs), ("onela_sample_args", binding.SampleArgs)):
        body = re.search(r"typedef struct %s \{(.*?)\}" % struct, text, flags=re.S).group(1)
        fields = []
        for decl in body.split(";"):
            m = re.match(r"\s*(?:const\s+)?(\w+)\s*(.*)", decl.strip(), flags=re.S)
            if m is None or not m.group(2):
                continue
            for name in m.group(2).split(","):
                name = name.strip()
                fields.append((name.lstrip("* ").removesuffix("_dev"), ctypes.c_void_p if name.startswith("*") else size[m.group(1)]))
        assert fields == [(n, t) for n, t in cls._fields_], struct
