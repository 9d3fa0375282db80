"""Cases of the operators around the beam decode: what a server of the library's models does before, beside and after it.

* ``norm``: queries and keys of a layer are normalised per head (and rotated by their positions, in attention layers).
* ``delta``: the gated delta rule over ragged sequences whose states live in a pool, prompts (chunked) and single tokens alike.
* ``sample``: one token per row of logits, with temperature, top-k, top-p and min-p, from random numbers that are inputs.

Keys of a ``norm`` case: tokens, heads (queries), k_heads, dim, dtype, norm ("l2" / "rms"), rotary (rotated elements, 0: none),
interleaved, far (largest position), packed (q and k are slices of one projection's output, written in place of nothing else).
Keys of a ``delta`` case: sequences, lo / hi (tokens per sequence, drawn evenly; lo = hi = 1: a decode step), pad (sequences of
the batch that are padding), fresh (share of the sequences that start from the zero state), heads (key heads), v_heads, dk, dv, dtype.
Keys of a ``sample`` case: rows, vocab, dtype, top_k, top_p, min_p (per-row values are drawn around these; 0: off), masked (share of
the tokens that a grammar forbids).
"""
from __future__ import annotations

import math
import random

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}
_ELEM = {"bf16": 2, "fp32": 4}


def _norm(name, **kw):
    case = dict(name=name, kind="norm", tokens=1, heads=32, k_heads=32, dim=128, dtype="bf16", norm="l2", rotary=0, interleaved=False, far=0, packed=False)
    case.update(kw)
    return case


def _delta(name, **kw):
    case = dict(name=name, kind="delta", sequences=1, lo=1, hi=1, pad=0, fresh=0.0, heads=16, v_heads=0, dk=128, dv=128, dtype="bf16")
    case.update(kw)
    case["v_heads"] = case["v_heads"] or case["heads"]
    return case


def _sample(name, **kw):
    case = dict(name=name, kind="sample", rows=1, vocab=1000, dtype="fp32", top_k=0, top_p=0.0, min_p=0.0, masked=0.0)
    case.update(kw)
    return case


def listed():
    return [
        # One token of one user's layer: latency of the smallest call.
        _norm("norm_one_token", heads=16, k_heads=16),
        # The prompt of a long user history, a Gated DeltaNet layer: unit queries and keys.
        _norm("norm_prompt_16384", tokens=16384),
        # An attention layer of a hybrid model: RMS norms with weights, a quarter of each head rotated, far positions, slices of one projection.
        _norm("norm_rotate_4099", tokens=4099, heads=16, k_heads=2, dim=256, norm="rms", rotary=64, far=1 << 20, packed=True),
        # One user generates: one token, latency.
        _delta("step_one_user"),
        # A full decode batch with padding, two value heads per key head.
        _delta("step_batch64", sequences=64, pad=3, v_heads=32),
        # Drafted tokens verified a few at a time, narrow fp32 heads.
        _delta("draft_37x5_fp32", sequences=37, lo=1, hi=5, dk=64, dv=64, dtype="fp32"),
        # One user's history through one layer.
        _delta("prompt_4096", lo=4096, hi=4096, fresh=1.0),
        # A batch of histories of very different lengths, some continued from a stored state.
        _delta("prompts_4_ragged", sequences=4, lo=1000, hi=8192, fresh=0.5, heads=32),
        # Two short histories of odd length, narrow heads, fp32.
        _delta("prompt_1021_fp32", sequences=2, lo=1021, hi=1021, fresh=1.0, dk=64, dv=64, dtype="fp32"),
        # One user, a text vocabulary, bf16 logits (many ties), the usual filters.
        _sample("sample_one_row", vocab=131072, dtype="bf16", top_k=50, top_p=0.9),
        # A decode batch over an odd vocabulary, a nucleus of the whole distribution.
        _sample("sample_batch64", rows=64, vocab=100003, top_p=0.95, min_p=0.001, masked=0.1),
        # Semantic-id codes: many short rows, temperature only.
        _sample("sample_codes_512", rows=512, vocab=1000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "delta", "delta", "sample"])
    if kind == "norm":
        case = _norm("", tokens=_log_int(rng, 1, 16384), heads=rng.choice([4, 8, 16, 24, 32]), k_heads=rng.choice([1, 2, 4, 8, 16]), dim=rng.choice([32, 64, 96, 128, 256]),
                     dtype=rng.choice(["bf16", "bf16", "fp32"]), norm=rng.choice(["l2", "rms"]), packed=rng.random() < 0.5)
        if rng.random() < 0.6:
            case.update(rotary=rng.choice([r for r in (16, 32, 64, 96, 128) if r <= case["dim"]]), interleaved=rng.random() < 0.3, far=_log_int(rng, 100, 1 << 24))
        while work(case)["bytes"] > work(_named("norm_prompt_16384"))["bytes"]:
            case["tokens"] //= 2
    elif kind == "delta":
        case = _delta("", heads=rng.choice([2, 4, 8, 16, 32]), dtype=rng.choice(["bf16", "bf16", "fp32"]), fresh=rng.choice([0.0, 0.3, 1.0]))
        case["dk"], case["dv"] = rng.choice([(128, 128)] * 4 + [(64, 64)] * 2 + [(32, 32), (128, 256), (256, 256)])
        case["v_heads"] = case["heads"] * (2 if case["heads"] <= 16 and rng.random() < 0.3 else 1)
        if rng.random() < 0.5:                                  # decode steps and drafts
            case["sequences"] = _log_int(rng, 1, 64)
            case["hi"] = rng.choice([1, 1, 1, 4, 9])
            case["pad"] = rng.randint(0, case["sequences"] // 4)
        else:                                                   # prompts, ragged
            case["sequences"] = _log_int(rng, 1, 8)
            case["hi"] = _log_int(rng, 17, 8192 if case["dk"] <= 128 else 512)
            case["lo"] = max(1, case["hi"] // rng.choice([1, 2, 8]))
        while work(case)["bytes"] > work(_named("prompts_4_ragged"))["bytes"]:
            case["sequences"] = max(1, case["sequences"] // 2)
            case["pad"] = min(case["pad"], case["sequences"] - 1)
            case["hi"] = max(case["lo"], case["hi"] * 3 // 4)
    else:
        case = _sample("", rows=_log_int(rng, 1, 512), vocab=_log_int(rng, 100, 200000), dtype=rng.choice(["fp32", "bf16"]), masked=rng.choice([0.0, 0.0, 0.3]))
        if rng.random() < 0.5:
            case["top_k"] = _log_int(rng, 1, 2000)
        if rng.random() < 0.6:
            case["top_p"] = round(rng.uniform(0.3, 0.99), 3)
        if rng.random() < 0.3:
            case["min_p"] = round(rng.uniform(0.001, 0.2), 4)
        while work(case)["bytes"] > work(_named("sample_batch64"))["bytes"]:
            case["rows"] = max(1, case["rows"] // 2)
    del case["name"]
    return case


def _named(name):
    return next(c for c in listed() if c["name"] == name)


def _lengths(case):
    """Tokens of each sequence (a property of the case, so that the work is one number)."""
    rng = random.Random(case["sequences"] * 7919 + case["hi"])
    n = [rng.randint(case["lo"], case["hi"]) for _ in range(case["sequences"])]
    n[rng.randrange(len(n))] = case["hi"]
    return n


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    return {"norm": _prepare_norm, "delta": _prepare_delta, "sample": _prepare_sample}[case["kind"]](case, gen, rng)


def _prepare_norm(case, gen, rng):
    n, hq, hk, d, dt = case["tokens"], case["heads"], case["k_heads"], case["dim"], _TORCH[case["dtype"]]
    if case["packed"]:                                          # q | k | something else, as a projection leaves them
        row = torch.empty((n, (hq + 2 * hk) * d), dtype=dt, device="cuda")
        row.copy_(_randn(gen, *row.shape))
        q, k = row[:, :hq * d].view(n, hq, d), row[:, hq * d:(hq + hk) * d].view(n, hk, d)
    else:
        q, k = _randn(gen, n, hq, d).to(dt), _randn(gen, n, hk, d).to(dt)
    s = dict(kind="norm", case=dict(case), q=q, k=k, q_out=torch.empty((n, hq, d), dtype=dt, device="cuda"), k_out=torch.empty((n, hk, d), dtype=dt, device="cuda"),
             norm=case["norm"], q_weight=None, k_weight=None, positions=None, inv_freq=None, interleaved=case["interleaved"],
             q_scale=d ** -0.5 if case["norm"] == "l2" else 1.0)
    if case["norm"] == "rms":
        s["q_weight"], s["k_weight"] = 1 + 0.1 * _randn(gen, d), 1 + 0.1 * _randn(gen, d)
    if case["rotary"]:
        r = case["rotary"]
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)).float()
        s["positions"] = torch.randint(0, case["far"], (n,), generator=gen, device="cuda", dtype=torch.int32)
    return s


def _prepare_delta(case, gen, rng):
    lens, hk, hv, dk, dv, dt = _lengths(case), case["heads"], case["v_heads"], case["dk"], case["dv"], _TORCH[case["dtype"]]
    n, total = len(lens), sum(lens)
    unit = lambda x: x / torch.linalg.vector_norm(x, dim=-1, keepdim=True)  # noqa: E731
    pool = n + 2                                                # a pool with states of others in it
    slots = rng.sample(range(pool), n)
    padded = set(rng.sample(range(n), case["pad"]))
    fresh = [rng.random() < case["fresh"] or case["fresh"] >= 1.0 for _ in range(n)]
    starts = [0]
    for x in lens:
        starts.append(starts[-1] + x)
    live = [i for i in range(n) if i not in padded]
    at = torch.tensor([[starts[i] + min(t, lens[i] - 1) for t in range(case["hi"])] for i in live], device="cuda")      # the plan of a padded batch
    within = torch.tensor([[t < lens[i] for t in range(case["hi"])] for i in live], device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(kind="delta", case=dict(case), q=unit(_randn(gen, total, hk, dk)).to(dt), k=unit(_randn(gen, total, hk, dk)).to(dt), v=_randn(gen, total, hv, dv).to(dt),
                alpha=1 - 0.1 * torch.rand((total, hv), generator=gen, device="cuda"), beta=torch.sigmoid(_randn(gen, total, hv)),
                states=0.3 * _randn(gen, pool, hv, dv, dk), out=torch.zeros((total, hv, dv), dtype=dt, device="cuda"),
                starts=None if case["hi"] == 1 else i32(starts), slots=i32([-1 if i in padded else slots[i] for i in range(n)]),
                fresh=i32([int(f) for f in fresh]), max_tokens=case["hi"],
                live_slots=torch.tensor([slots[i] for i in live], device="cuda"), live_fresh=torch.tensor([fresh[i] for i in live], device="cuda"),
                at=at, within=within, at_in=at[within])


def _prepare_sample(case, gen, rng):
    r, v = case["rows"], case["vocab"]
    x = 2.5 * _randn(gen, r, v)
    if case["masked"]:
        x.masked_fill_(torch.rand((r, v), generator=gen, device="cuda") < case["masked"], -math.inf)
    rand = lambda lo, hi: lo + (hi - lo) * torch.rand((r,), generator=gen, device="cuda")  # noqa: E731
    return dict(kind="sample", case=dict(case), logits=x.to(_TORCH[case["dtype"]]), uniforms=torch.rand((r,), generator=gen, device="cuda"),
                temperature=rand(0.6, 1.2),
                top_k=torch.randint(max(1, case["top_k"] // 2), case["top_k"] * 3 // 2 + 1, (r,), generator=gen, device="cuda", dtype=torch.int32) if case["top_k"] else None,
                top_p=(case["top_p"] * rand(0.9, 1.0)) if case["top_p"] else None, min_p=(case["min_p"] * rand(0.5, 1.5)) if case["min_p"] else None,
                tokens_out=torch.zeros((r,), dtype=torch.int32, device="cuda"), logprobs_out=torch.zeros((r,), device="cuda"))


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(state):
    if own:
        import paper_2609_12399_b200 as P
        s = state
        if s["kind"] == "norm":
            P.onela_norm_rotate(s["q"], s["k"], s["q_out"], s["k_out"], norm=s["norm"], eps=1e-6, q_scale=s["q_scale"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                                positions=s["positions"], inv_freq=s["inv_freq"], interleaved=s["interleaved"])
            return {"q": s["q_out"], "k": s["k_out"]}
        if s["kind"] == "delta":
            P.onela_delta_rule(s["q"], s["k"], s["v"], s["alpha"], s["beta"], s["states"], s["out"], starts=s["starts"], slots=s["slots"], fresh=s["fresh"],
                               max_tokens=s["max_tokens"])
            return {"out": s["out"], "states": s["states"]}
        P.onela_sample_tokens(s["logits"], s["uniforms"], s["tokens_out"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                              logprobs_out=s["logprobs_out"])
        return {"tokens": s["tokens_out"], "logprobs": s["logprobs_out"]}
    return {"norm": _plain_norm, "delta": _plain_delta, "sample": _plain_sample}[state["kind"]](state)


def _plain_norm(s):
    cos = sin = None
    if s["inv_freq"] is not None:                               # angles in 64 bits: far positions
        turn = s["positions"].double()[:, None] * s["inv_freq"].double()
        cos, sin = turn.cos().float()[:, None], turn.sin().float()[:, None]

    def one(x, weight, scale, out):
        x = x.float()
        sq = x * x
        x = x / (sq.sum(-1, keepdim=True) + 1e-6).sqrt() if s["norm"] == "l2" else x / (sq.mean(-1, keepdim=True) + 1e-6).sqrt() * weight
        if cos is not None:
            half = cos.shape[-1]
            a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if s["interleaved"] else (x[..., :half], x[..., half:2 * half])
            ra, rb = a * cos - b * sin, b * cos + a * sin
            turned = torch.stack((ra, rb), -1).flatten(-2) if s["interleaved"] else torch.cat((ra, rb), -1)
            x = torch.cat((turned, x[..., 2 * half:]), -1)
        return out.copy_(x * scale)

    return {"q": one(s["q"], s["q_weight"], s["q_scale"], s["q_out"]), "k": one(s["k"], s["k_weight"], 1.0, s["k_out"])}


def _plain_delta(s):
    at, within, g = s["at"], s["within"], s["v"].shape[1] // s["k"].shape[1]
    per_token = lambda x, rep: x[at].float().repeat_interleave(rep, 2).movedim(1, 0)  # noqa: E731   [time, sequence, head, ..]
    q, k, v = per_token(s["q"], g)[..., None], per_token(s["k"], g)[..., None], per_token(s["v"], 1)[..., None]
    inside = within[..., None]
    alpha = torch.where(inside, s["alpha"][at], 1.0).movedim(1, 0)[..., None, None]
    beta = torch.where(inside, s["beta"][at], 0.0).movedim(1, 0)[..., None, None]
    S = s["states"][s["live_slots"]] * (~s["live_fresh"])[:, None, None, None]
    outs = []
    for t in range(at.shape[1]):                                # the recurrence itself
        S = S * alpha[t]
        S = S + (beta[t] * (v[t] - S @ k[t])) * k[t].transpose(-1, -2)
        outs.append((S @ q[t])[..., 0])
    s["out"][s["at_in"]] = torch.stack(outs, 1)[within].to(s["out"].dtype)
    s["states"][s["live_slots"]] = S
    return {"out": s["out"], "states": s["states"]}


def _plain_sample(s):
    x = s["logits"].double()                                    # masses in 64 bits: long sums, values next to a border
    x = torch.where(x.isnan(), -math.inf, x)
    top = x.max(-1, keepdim=True).values
    w = torch.where(x == top, 1.0, ((x - top) / s["temperature"].double()[:, None]).exp())
    order = x.sort(dim=-1, descending=True, stable=True).indices
    ws = w.gather(-1, order)
    rank = torch.arange(x.shape[1], device=x.device)[None]
    kept = torch.ones_like(ws, dtype=torch.bool)
    if s["top_k"] is not None:
        kept &= rank < s["top_k"][:, None]
    if s["top_p"] is not None:
        mass = torch.where(kept, ws, 0.0).sum(-1, keepdim=True)
        kept &= ws.cumsum(-1) - ws < s["top_p"].double()[:, None] * mass
    if s["min_p"] is not None:
        kept &= ws >= s["min_p"].double()[:, None]
    kept[:, 0] = True
    w = torch.zeros_like(w).scatter_(-1, order, torch.where(kept, ws, 0.0))
    run_to = w.cumsum(-1)
    mass = run_to[:, -1:]
    token = (run_to <= s["uniforms"].double()[:, None] * mass).sum(-1, keepdim=True).clamp(max=x.shape[1] - 1)
    s["tokens_out"].copy_(token[:, 0])
    s["logprobs_out"].copy_((w.gather(-1, token) / mass).log()[:, 0])
    return {"tokens": s["tokens_out"], "logprobs": s["logprobs_out"]}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------
def work(case):
    e = _ELEM[case["dtype"]]
    if case["kind"] == "norm":
        n = case["tokens"] * (case["heads"] + case["k_heads"]) * case["dim"]
        return {"bytes": 2 * n * e + (case["tokens"] * 4 if case["rotary"] else 0), "flops": 4 * n}
    if case["kind"] == "delta":
        lens = _lengths(case)
        live = case["sequences"] - case["pad"]
        tokens = sum(lens) * live / len(lens)
        state = case["v_heads"] * case["dv"] * case["dk"]
        per_token = 2 * (case["heads"] * case["dk"] + case["v_heads"] * case["dv"]) * e + 8 * case["v_heads"]
        return {"bytes": tokens * per_token + (2 - min(1.0, case["fresh"])) * live * state * 4, "flops": 7 * tokens * state}
    n = case["rows"] * case["vocab"]
    return {"bytes": n * e + case["rows"] * 28, "flops": 4 * n}


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------
def exact(case, seed):
    return {"norm": _exact_norm, "delta": _exact_delta, "sample": _exact_sample}[case["kind"]](prepare(case, seed))


def _exact_norm(s):
    answers = {}
    for name, weight, scale in (("q", s["q_weight"], s["q_scale"]), ("k", s["k_weight"], 1.0)):
        x = s[name].double()
        if s["norm"] == "l2":
            y = x * torch.rsqrt(torch.einsum("nhd,nhd->nh", x, x) + 1e-6)[..., None]
        else:
            y = x * torch.rsqrt(torch.einsum("nhd,nhd->nh", x, x) / x.shape[-1] + 1e-6)[..., None] * weight.double()
        if s["inv_freq"] is not None:                           # pairs as complex numbers
            r = 2 * s["inv_freq"].numel()
            phase = torch.polar(torch.ones((), dtype=torch.float64, device=x.device).expand(x.shape[0], r // 2).contiguous(),
                                s["positions"].double()[:, None] * s["inv_freq"].double()[None])[:, None]
            i = torch.arange(r // 2, device=x.device)
            first, second = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + r // 2)
            z = torch.complex(y[..., first], y[..., second]) * phase
            y = y.clone()
            y[..., first], y[..., second] = z.real, z.imag
        answers[name] = y * scale
    return answers


def _exact_delta(s):
    out, states = s["out"].double(), s["states"].double()
    group = s["v"].shape[1] // s["k"].shape[1]
    head = torch.arange(s["v"].shape[1], device=out.device) // group
    slots, fresh = s["slots"].tolist(), s["fresh"].tolist()
    starts = s["starts"].tolist() if s["starts"] is not None else list(range(len(slots) + 1))
    if max(starts[i + 1] - starts[i] for i in range(len(slots))) * len(slots) > 40000:
        return None
    live = [i for i in range(len(slots)) if slots[i] >= 0]
    state = torch.stack([states[slots[i]] * (0 if fresh[i] else 1) for i in live])
    length = [starts[i + 1] - starts[i] for i in live]
    for t in range(max(length)):
        going = [j for j in range(len(live)) if t < length[j]]
        token = torch.tensor([starts[live[j]] + t for j in going], device=out.device)
        key, query, value = s["k"][token][:, head].double(), s["q"][token][:, head].double(), s["v"][token].double()
        a, b = s["alpha"][token].double()[..., None], s["beta"][token].double()[..., None]
        S = state if len(going) == len(live) else state[going]
        change = b * (value - a * torch.einsum("nhvk,nhk->nhv", S, key))
        S = a[..., None] * S + torch.einsum("nhv,nhk->nhvk", change, key)
        out[token] = torch.einsum("nhvk,nhk->nhv", S, query)
        if len(going) == len(live):
            state = S
        else:
            state[going] = S
    for j, i in enumerate(live):
        states[slots[i]] = state[j]
    return {"out": out, "states": states}


def _exact_sample(s):
    tokens, logprobs = [], []
    for r in range(s["logits"].shape[0]):
        x = s["logits"][r].double().nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
        best = x.max()
        ordered, index = torch.sort(x, descending=True, stable=True)
        p = torch.exp((ordered - best) / s["temperature"][r].double())
        count = x.numel() if s["top_k"] is None else min(x.numel(), int(s["top_k"][r]))
        if s["top_p"] is not None:                              # the shortest run that reaches the nucleus
            reach = p[:count].cumsum(0)
            count = min(count, 1 + int((reach < s["top_p"][r].double() * p[:count].sum()).sum()))
        if s["min_p"] is not None:
            count = min(count, max(1, int((p >= s["min_p"][r].double()).sum())))
        chosen, by_index = index[:count].sort()
        masses = p[:count][by_index]
        total = masses.sum()
        at = min(int(torch.searchsorted(masses.cumsum(0), (s["uniforms"][r].double() * total).view(1), right=True)), count - 1)
        tokens.append(int(chosen[at]))
        logprobs.append(float(torch.log(masses[at] / total)))
    return {"tokens": torch.tensor(tokens, dtype=torch.int32), "logprobs": torch.tensor(logprobs, dtype=torch.float64)}
