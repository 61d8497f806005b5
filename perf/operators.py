"""Operators around the attention of a sample group: the rows that go into a decode step (rotary
positions), the scores of the tokens that come out of the model, and the responses' pages.

Five kinds of pass:

* rotate  rotary positions on the Q and K rows of a token: `entry` "step" is one running step (every
          live slot of a context, all layers at once or one), "rows" a prompt's or a training batch's
          rows, `inverse` the gradient (rotation by the negative angle).
* score   log probability of one given token per row of logits, the entropy of the row's
          distribution, its `top` most probable entries, and the statistics its gradient goes by
          (the row's maximum and the log of its sum relative to it).
* grad    the gradient of these log probabilities (and entropies) with respect to the logits.
* branch  live samples fork into empty slots at several lengths (full pages shared, the last one
          copied); the branches' K/V then leave as dense rows, and the slots are given up again.
* carry   responses of an earlier iteration come back into empty slots as dense K/V rows, leave
          again the same way, and the slots are given up.

Shapes are those of this repository's presets (Qwen3-1.7B and 8B attention layouts, the tiny fp32
group), its tests (other head counts and sizes) and sizes between them; vocabularies are of ordinary
sizes, even and odd.  Q, K and V rows are N(0, 1).  Logits are normal with a spread of some units and
a padded, masked end; the given tokens are drawn from them.
"""

import math

import numpy as np
import torch

own = False

PAGE = 16  # tokens of a response page
SAMPLES = 1 << 20  # sample ids that a context's passes take from


def listed():
    qwen17 = {"q_heads": 16, "kv_heads": 8, "head_dim": 128}
    qwen8 = {"q_heads": 32, "kv_heads": 8, "head_dim": 128}
    plain = {"layout": "half", "rotary_dim": 128, "scaling": "none", "factor": 1.0, "inverse": False}
    return [
        # one layer's Q and K rows of a running step (throughput preset, 16 slots), out of the fused
        # projection: what each layer of a model calls before its attention; all latency
        {"name": "rotate_step_layer", "kind": "rotate", "entry": "step", "layers": 1, **qwen17, "tokens": 16,
         "first": 2048, **plain, "dtype": "bf16", "fused": True},
        # the same rows of all 28 layers, ahead of the launch that decodes every layer
        {"name": "rotate_step_28", "kind": "rotate", "entry": "step", "layers": 28, **qwen17, "tokens": 16,
         "first": 2048, **plain, "dtype": "bf16", "fused": False},
        # four prompts' rows of one layer before the prefill (8B-shaped preset), scaled for a long context
        {"name": "rotate_prompts_8b", "kind": "rotate", "entry": "rows", "layers": 1, **qwen8, "tokens": 7424,
         "first": 0, **plain, "scaling": "yarn", "factor": 4.0, "dtype": "bf16", "fused": True},
        # gradient rows in fp32: interleaved pairs, three quarters of a head, far positions, an odd count
        {"name": "rotate_gradient_f32", "kind": "rotate", "entry": "rows", "layers": 1, "q_heads": 32, "kv_heads": 4,
         "head_dim": 64, "tokens": 4097, "first": 1000003, "layout": "interleaved", "rotary_dim": 48,
         "scaling": "linear", "factor": 8.0, "inverse": True, "dtype": "f32", "fused": False},
        # the rows of one running step: 16 slots, the sampled tokens with 20 alternatives
        {"name": "score_step", "kind": "score", "rows": 16, "vocab": 151936, "top": 20, "temperature": 1.0,
         "masked": 267, "dtype": "bf16"},
        # a small batch of an odd vocabulary in fp32 at a temperature, five alternatives
        {"name": "score_f32_odd", "kind": "score", "rows": 301, "vocab": 50257, "top": 5, "temperature": 0.7,
         "masked": 0, "dtype": "f32"},
        # the old policy's log probabilities and entropies for a learner's batch
        {"name": "score_learner", "kind": "score", "rows": 2048, "vocab": 151936, "top": 0, "temperature": 1.0,
         "masked": 267, "dtype": "bf16"},
        # its gradient
        {"name": "grad_learner", "kind": "grad", "rows": 2048, "vocab": 151936, "temperature": 1.0, "masked": 267,
         "entropy": False, "dtype": "bf16"},
        # a small gradient in fp32 with an entropy bonus, odd vocabulary
        {"name": "grad_f32_entropy", "kind": "grad", "rows": 67, "vocab": 32003, "temperature": 0.9, "masked": 0,
         "entropy": True, "dtype": "f32"},
        # a tree of samples: three parents, a branch each, one layer of the tiny fp32 group
        {"name": "branch_tiny_f32", "kind": "branch", "layers": 1, "q_heads": 4, "kv_heads": 2, "head_dim": 64,
         "parents": "17,40,64", "fan": 1, "length": 64, "cache": "f32"},
        # the same over the throughput preset's layers, responses at ordinary lengths (the
        # most bytes but for the next)
        {"name": "branch_1p7b", "kind": "branch", "layers": 28, **qwen17, "parents": "1500,377,1024,801", "fan": 3,
         "length": 2048, "cache": "bf16"},
        # partial responses carried over into a new iteration, E4M3 cache
        {"name": "carry_1p7b_e4m3", "kind": "carry", "layers": 28, **qwen17,
         "lengths": "33,1024,512,7,2000,1333,640,255", "length": 2048, "cache": "e4m3"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_MOST = 2 * 2048 * 151936 * 2  # bytes of the largest listed pass


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "score", "score", "grad", "branch", "carry"])
    while True:
        if kind == "rotate":
            hkv, hpk, d = rng.choice([8, 8, 4, 2]), rng.choice([1, 2, 4, 8]), rng.choice([128, 128, 64])
            entry = rng.choice(["step", "rows"])
            dtype = rng.choice(["bf16", "bf16", "f32"])
            rd = rng.choice([d, d, d // 2, 2 * rng.randrange(1, d // 2 + 1)])
            scaling = rng.choice(["none", "none", "linear", "ntk", "yarn", "bands"])
            if scaling == "ntk" and rd <= 2:
                continue
            c = {"kind": kind, "entry": entry, "layers": _log_int(rng, 1, 36) if entry == "step" else 1,
                 "q_heads": hkv * hpk, "kv_heads": hkv, "head_dim": d,
                 "tokens": _log_int(rng, 1, (16 if dtype == "f32" else 64) // hpk) if entry == "step" else _log_int(rng, 1, 32768),
                 "first": rng.randrange(0, 4096) if entry == "step" else rng.choice([0, _log_int(rng, 1, 1 << 20)]),
                 "layout": rng.choice(["half", "interleaved"]), "rotary_dim": rd, "scaling": scaling,
                 "factor": 1.0 if scaling == "none" else float(rng.choice([2, 4, 8, 32])),
                 "inverse": entry == "rows" and rng.random() < 0.4, "dtype": dtype, "fused": rng.random() < 0.5}
        elif kind in ("score", "grad"):
            c = {"kind": kind, "rows": _log_int(rng, 1, 4096), "vocab": _log_int(rng, 1000, 262144),
                 "temperature": rng.choice([1.0, 1.0, 0.7, 1.3]), "dtype": rng.choice(["bf16", "bf16", "f32"])}
            c["masked"] = rng.choice([0, c["vocab"] // 500, c["vocab"] // 3])
            if kind == "score":
                c["top"] = rng.choice([0, 0, 1, 5, 20, 32]) if c["rows"] <= 512 else rng.choice([0, 0, 5])
            else:
                c["entropy"] = rng.random() < 0.5
        else:
            cache = rng.choice(["bf16", "bf16", "e4m3", "f32"])
            hkv, hpk = rng.choice([8, 8, 4, 2]), rng.choice([1, 2, 4, 8])
            d = 128 if cache == "e4m3" else rng.choice([128, 128, 64])
            cap = _log_int(rng, 32, 4096)
            c = {"kind": kind, "layers": _log_int(rng, 1, 36), "q_heads": hkv * hpk, "kv_heads": hkv, "head_dim": d,
                 "length": cap, "cache": cache}
            n, fan = rng.randrange(1, 9), rng.randrange(1, 5)
            lens = ",".join(str(_log_int(rng, 1, cap)) for _ in range(n))
            if kind == "branch":
                c.update(parents=lens, fan=fan)
            else:
                c.update(lengths=lens)
            rows = _slots(c) * hpk
            if rows > (16 if cache == "f32" else 128) or (cache == "e4m3" and rows < 16):
                continue
        if work(c)["bytes"] <= _MOST:
            return c


# ---------------------------------------------------------------------------------------------
# Sizes
# ---------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.float32 if case.get("dtype", case.get("cache")) == "f32" else torch.bfloat16


def _ints(text):
    return [int(x) for x in text.split(",")]


def _slots(case):
    if case["kind"] == "branch":
        return len(_ints(case["parents"])) * (1 + case["fan"])
    return len(_ints(case["lengths"]))


def _branches(case):
    """(parent index, tokens kept) of every branch: the parent's whole response, then earlier points."""
    fan = case["fan"]
    return [(i, max(1, n - n * b // (2 * fan))) for i, n in enumerate(_ints(case["parents"])) for b in range(fan)]


def _positions(case):
    """Position of every token: a running step's slots are at all response lengths below 1024."""
    n = case["tokens"]
    if case["entry"] == "step":
        return [case["first"] + (617 * s) % 1024 for s in range(n)]
    return list(range(case["first"], case["first"] + n))


BASE = 1000000.0       # rotary base
TRAINED = 8192         # positions the unscaled frequencies were trained on (yarn, bands)


def work(case):
    kind = case["kind"]
    if kind == "rotate":
        es = 4 if case["dtype"] == "f32" else 2
        rows = case["layers"] * case["tokens"] * (case["q_heads"] + case["kv_heads"])
        return {"bytes": 2 * rows * case["head_dim"] * es, "flops": 3 * rows * case["rotary_dim"]}
    if kind in ("score", "grad"):
        n = case["rows"] * case["vocab"]
        es = 4 if case["dtype"] == "f32" else 2
        if kind == "score":
            return {"bytes": n * es + case["rows"] * (20 + 8 * case["top"]), "flops": 5 * n}
        return {"bytes": 2 * n * es + case["rows"] * 24, "flops": 5 * n}
    es = 4 if case["cache"] == "f32" else 2                # rows handed over
    ks = {"f32": 4, "bf16": 2, "e4m3": 1}[case["cache"]]  # stored elements
    row = 2 * case["kv_heads"] * case["head_dim"] * case["layers"]  # K and V elements of a token
    if kind == "branch":
        # every parent read once, every branch's rows written, its part of a page stored
        parents = sum(_ints(case["parents"]))
        return {"bytes": row * (parents * ks + sum(t * es + t % PAGE * ks for _, t in _branches(case))), "flops": 0}
    return {"bytes": row * 2 * (ks + es) * sum(_ints(case["lengths"])), "flops": 0}


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rotate_inputs(case, seed):
    """Q and K rows [layers, tokens, heads, d]; fused: views of one projection output [.., Hq + 2 Hkv, d]."""
    gen = _generator(seed)
    L, T, hq, hkv, d = case["layers"], case["tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
    heads = hq + (2 if case["fused"] else 1) * hkv
    if case["fused"]:
        x = torch.randn(L, T, heads, d, generator=gen, device="cuda").to(_dtype(case))
        return x[:, :, :hq], x[:, :, hq:hq + hkv]
    q = torch.randn(L, T, hq, d, generator=gen, device="cuda").to(_dtype(case))
    k = torch.randn(L, T, hkv, d, generator=gen, device="cuda").to(_dtype(case))
    return q, k


def _logits(case, seed):
    """Logits [rows, vocab] (a masked end of -inf), the given token of each row (drawn from the row's
    distribution, every 16th row without one), upstream gradients of log probability and entropy."""
    gen = _generator(seed)
    n, v = case["rows"], case["vocab"]
    live = v - case["masked"]
    z = torch.empty(n, v, dtype=_dtype(case), device="cuda")
    tokens = torch.empty(n, dtype=torch.int32, device="cuda")
    step = max(1, (1 << 26) // v)
    for a in range(0, n, step):
        b = min(n, a + step)
        x = torch.randn(b - a, v, generator=gen, device="cuda")
        x *= 3.0
        z[a:b] = x.to(z.dtype)
        z[a:b, live:] = -math.inf
        u = torch.rand(b - a, v, generator=gen, device="cuda").clamp_(1e-9, 1 - 1e-7)
        u.log_().neg_().log_().neg_()  # Gumbel noise
        u.add_(z[a:b].float(), alpha=1.0 / case["temperature"])
        tokens[a:b] = u.argmax(1).int()
    if n > 1:
        tokens[15::16] = -1
    g_lp = torch.randn(n, generator=gen, device="cuda")
    g_h = 0.1 * torch.randn(n, generator=gen, device="cuda")
    return z, tokens, g_lp, g_h


def _kv(case, seed):
    """K and V rows [layers, tokens, kv_heads, d] of every response (branch: the parents'; carry: the parked ones')."""
    gen = _generator(seed)
    lens = _ints(case["parents"] if case["kind"] == "branch" else case["lengths"])
    return [tuple(torch.randn(case["layers"], n, case["kv_heads"], case["head_dim"], generator=gen, device="cuda").to(
        _dtype(case)) for _ in range(2)) for n in lens]


def _stored(case, x):
    if case["cache"] == "e4m3":
        return x.float().clamp(-448, 448).to(torch.float8_e4m3fn)
    return x


# ---------------------------------------------------------------------------------------------
# prepare
# ---------------------------------------------------------------------------------------------
def _frequencies(case):
    """Angle per position of every pair, float64, and the factor on cos and sin."""
    rd, s = case["rotary_dim"], case["factor"]
    pair = np.arange(rd // 2, dtype=np.float64)
    if case["scaling"] == "ntk":
        return (BASE * s ** (rd / (rd - 2.0))) ** (-2.0 * pair / rd), 1.0
    f = BASE ** (-2.0 * pair / rd)
    if case["scaling"] == "linear":
        return f / s, 1.0
    if case["scaling"] == "yarn":
        def at(turns):  # pair index whose wavelength makes `turns` turns over the trained positions
            return rd * math.log(TRAINED / (turns * 2 * math.pi)) / (2 * math.log(BASE))
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), rd - 1)
        ramp = np.clip((pair - lo) / max(hi - lo, 0.001), 0, 1)
        return f / s * ramp + f * (1 - ramp), 0.1 * math.log(s) + 1.0
    if case["scaling"] == "bands":
        turns = TRAINED * f / (2 * math.pi)  # turns over the trained positions
        smooth = np.clip((turns - 1.0) / (4.0 - 1.0), 0, 1)
        return (1 - smooth) * f / s + smooth * f, 1.0
    return f, 1.0


def _own_rotary(case):
    from paper_2506_22950_amd import infs

    return infs.Rotary(infs.make_rotary_config(
        head_dim=case["head_dim"], rotary_dim=case["rotary_dim"],
        layout=infs.ROTARY_INTERLEAVED if case["layout"] == "interleaved" else infs.ROTARY_HALF,
        scaling={"none": infs.ROTARY_NONE, "linear": infs.ROTARY_LINEAR, "ntk": infs.ROTARY_NTK,
                 "yarn": infs.ROTARY_YARN, "bands": infs.ROTARY_BANDS}[case["scaling"]],
        base=BASE, factor=case["factor"], trained_len=TRAINED, low=1.0,
        high=4.0 if case["scaling"] == "bands" else 32.0))


def _own_context(case, slots, prompt, cap, dtype, fp8=False):
    from paper_2506_22950_amd import infs

    return infs.Context(infs.make_config(
        num_layers=case["layers"], num_q_heads=case["q_heads"], num_kv_heads=case["kv_heads"],
        head_dim=case["head_dim"], num_prompts=1, slots_per_prompt=slots, samples_per_prompt=SAMPLES,
        max_prompt_len=prompt, max_suffix_len=cap, dtype=infs.F32 if dtype == "f32" else infs.BF16,
        flags=infs.FLAG_KV_FP8 if fp8 else 0), stream=torch.cuda.current_stream())


class _State:
    pass


def prepare(case, seed):
    st = _State()
    st.case = case
    return {"rotate": _prepare_rotate, "score": _prepare_score, "grad": _prepare_score, "branch": _prepare_pages,
            "carry": _prepare_pages}[case["kind"]](st, seed)


def _prepare_rotate(st, seed):
    case = st.case
    st.q, st.k = _rotate_inputs(case, seed)
    if own:
        st.rotary = _own_rotary(case)
        st.q_out, st.k_out = (torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in (st.q, st.k))
        if case["entry"] == "step":
            # a context whose slots hold responses of the positions' lengths
            n, cap = case["tokens"], 1024
            st.ctx = _own_context(case, n, case["first"], cap, case["dtype"])
            none = torch.zeros(case["layers"] * max(cap, case["first"]), case["kv_heads"], case["head_dim"],
                               dtype=st.q.dtype, device="cuda")
            for layer in range(case["layers"]):
                st.ctx.prefill_shared(0, layer, case["first"], none, none)
            lens = [p - case["first"] for p in _positions(case)]
            st.ctx.import_responses(list(range(n)), list(range(n)), lens, [none] * n, [none] * n)
            st.ctx.sync()
    else:
        f, st.amplitude = _frequencies(case)
        st.frequencies = torch.from_numpy(f).cuda()
        st.positions = torch.tensor(_positions(case), dtype=torch.int32, device="cuda")
    return st


def _prepare_score(st, seed):
    case = st.case
    st.z, st.tokens, st.g_lp, st.g_h = _logits(case, seed)
    n, top = case["rows"], case.get("top", 0)
    if case["kind"] == "grad":
        # what the forward pass left: the rows' maxima, the logs of their sums, their entropies
        st.stats = torch.empty(n, 2, device="cuda")
        st.entropy = torch.empty(n, device="cuda")
        step = max(1, (1 << 25) // case["vocab"])
        for a in range(0, n, step):
            x = st.z[a:a + step].double()
            m = x.amax(1)
            y = (x - m[:, None]) / case["temperature"]
            ls = torch.exp(y).sum(1).log()
            lp = (y - ls[:, None]).clamp_min_(-1e6)
            st.stats[a:a + step, 0], st.stats[a:a + step, 1] = m.float(), ls.float()
            st.entropy[a:a + step] = -(lp.exp() * lp).sum(1).float()
    if own:
        from paper_2506_22950_amd import infs

        st.scorer = infs.Scorer(infs.make_scorer_config(
            vocab=case["vocab"], dtype=infs.F32 if case["dtype"] == "f32" else infs.BF16, max_rows=n, top_k=top,
            temperature=case["temperature"]), stream=torch.cuda.current_stream())
        if case["kind"] == "score":
            st.logprob, st.out_entropy = (torch.empty(n, device="cuda") for _ in range(2))
            st.out_stats = torch.empty(n, 2, device="cuda")
            st.top_id = torch.empty(n, top, dtype=torch.int32, device="cuda")
            st.top_logprob = torch.empty(n, top, device="cuda")
        else:
            st.grad = torch.empty_like(st.z)
    return st


def _prepare_pages(st, seed):
    case = st.case
    kv = _kv(case, seed)
    lens = [k.shape[1] for k, _ in kv]
    slots, cap, fan = _slots(case), case["length"], case.get("fan", 0)
    if own:
        st.ctx = _own_context(case, slots, 16, cap, case["cache"], fp8=case["cache"] == "e4m3")
        none = torch.zeros(16, case["kv_heads"], case["head_dim"], dtype=_dtype(case), device="cuda")
        for layer in range(case["layers"]):
            st.ctx.prefill_shared(0, layer, 16, none, none)
        st.next_sample = 0
    else:
        st.per_slot = -(-cap // PAGE)
        st.dtype = torch.float8_e4m3fn if case["cache"] == "e4m3" else _dtype(case)
        # E4M3 codes are moved as bytes
        st.pool_k, st.pool_v = (torch.zeros(case["layers"], slots * st.per_slot * PAGE, case["kv_heads"], case["head_dim"],
                                            dtype=torch.uint8 if case["cache"] == "e4m3" else st.dtype, device="cuda")
                                for _ in range(2))
        st.free = list(range(slots * st.per_slot))[::-1]
    if case["kind"] == "carry":
        st.slots, st.kv, st.lens = list(range(slots)), kv, lens
    else:
        st.parents = list(range(0, slots, 1 + fan))
        st.kept = [t for _, t in _branches(case)]
        st.src = [st.parents[i] for i, _ in _branches(case)]
        st.slots = [s for s in range(slots) if s % (1 + fan)]
        st.lens = st.kept
        if own:
            _own_import(st, st.parents, lens, kv)
        else:
            st.pages = dict(zip(st.parents, _plain_import(st, kv)))
    if own:
        st.out = [tuple(torch.empty(case["layers"], n, case["kv_heads"], case["head_dim"], dtype=_dtype(case),
                                    device="cuda") for _ in range(2)) for n in st.lens]
        st.ctx.sync()
    return st


# ---------------------------------------------------------------------------------------------
# run
# ---------------------------------------------------------------------------------------------
def run(state):
    kind = state.case["kind"]
    if own:
        return {"rotate": _own_rotate, "score": _own_score, "grad": _own_grad, "branch": _own_branch,
                "carry": _own_carry}[kind](state)
    return {"rotate": _plain_rotate, "score": _plain_score, "grad": _plain_grad, "branch": _plain_branch,
            "carry": _plain_carry}[kind](state)


# ---- the framework's calls -------------------------------------------------------------------
def _rows(x, out):
    """A tensor [layers, tokens, heads, d] (any strides above a head's elements) as infs.rotary_rows takes it."""
    from paper_2506_22950_amd import infs

    return infs.rotary_rows(x, out, x.shape[2], in_strides=(x.stride(1), x.stride(2), x.stride(0)))


def _own_rotate(st):
    case = st.case
    q, k = _rows(st.q, st.q_out), _rows(st.k, st.k_out)
    if case["entry"] == "step":
        st.ctx.rotate_step(st.rotary, q, k, num_layers=case["layers"])
    else:
        from paper_2506_22950_amd import infs

        st.rotary.rotate_rows(infs.F32 if case["dtype"] == "f32" else infs.BF16, case["tokens"], q, k,
                              first_position=case["first"], inverse=case["inverse"], stream=torch.cuda.current_stream())
    return {"q": st.q_out, "k": st.k_out}


def _own_score(st):
    top = st.case["top"]
    st.scorer.score(st.z.shape[0], st.z, st.tokens, st.logprob, entropy=st.out_entropy, stats=st.out_stats,
                    top_id=st.top_id if top else None, top_logprob=st.top_logprob if top else None)
    out = {"logprob": st.logprob, "entropy": st.out_entropy, "stats": st.out_stats}
    if top:
        out.update(top_id=st.top_id, top_logprob=st.top_logprob)
    return out


def _own_grad(st):
    with_h = st.case["entropy"]
    st.scorer.grad(st.z.shape[0], st.z, st.tokens, st.stats, st.g_lp, st.grad,
                   entropy=st.entropy if with_h else None, d_entropy=st.g_h if with_h else None)
    return st.grad


def _own_import(st, slots, lens, kv):
    ids = list(range(st.next_sample, st.next_sample + len(slots)))
    st.next_sample += len(slots)
    st.ctx.import_responses(slots, ids, lens, [k for k, _ in kv], [v for _, v in kv])


def _own_leave(st):
    st.ctx.export_responses(st.slots, [k for k, _ in st.out], [v for _, v in st.out])
    for s in st.slots:
        st.ctx.retire_slot(s)
    return st.out


def _own_branch(st):
    ids = list(range(st.next_sample, st.next_sample + len(st.slots)))
    st.next_sample += len(st.slots)
    st.ctx.fork_slots(st.src, st.slots, ids, st.kept)
    return _own_leave(st)


def _own_carry(st):
    _own_import(st, st.slots, st.lens, st.kv)
    return _own_leave(st)


# ---- the plain forms -------------------------------------------------------------------------
def _plain_rotate(st):
    case = st.case
    angle = st.positions.double()[:, None] * st.frequencies
    if case["inverse"]:
        angle = -angle
    cos = (torch.cos(angle) * st.amplitude).float()[None, :, None]
    sin = (torch.sin(angle) * st.amplitude).float()[None, :, None]
    rd = case["rotary_dim"]

    def turn(x):
        out = x.float()
        r = out[..., :rd]
        if case["layout"] == "interleaved":
            a, b = r[..., 0::2], r[..., 1::2]
            y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = r[..., :rd // 2], r[..., rd // 2:]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([y, out[..., rd:]], -1).to(x.dtype)

    return {"q": turn(st.q), "k": turn(st.k)}


def _plain_score(st):
    case = st.case
    z = st.z.float()
    m = z.amax(1, keepdim=True)
    y = (z - m) / case["temperature"]
    e = torch.exp(y)
    s = e.sum(1, keepdim=True)
    ls = torch.log(s)
    given = st.tokens >= 0
    at = st.tokens.clamp_min(0).long()[:, None]
    logprob = torch.where(given, (y.gather(1, at) - ls)[:, 0], torch.zeros(()).cuda())
    entropy = (ls - (e * y.clamp_min(-1e30)).sum(1, keepdim=True) / s)[:, 0]
    out = {"logprob": logprob, "entropy": entropy, "stats": torch.cat([m, ls], 1)}
    if case["top"]:
        # by value, then by the lower index: both in one 64-bit key
        bits = z.view(torch.int32)
        key = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF).long() * (1 << 32) - torch.arange(z.shape[1], device="cuda")
        top = torch.topk(key, case["top"], dim=1, sorted=True).values
        idx = torch.remainder(-top, 1 << 32)
        out["top_id"] = idx.int()
        out["top_logprob"] = y.gather(1, idx) - ls
    return out


def _plain_grad(st):
    case = st.case
    m, ls = st.stats[:, :1], st.stats[:, 1:]
    lp = (st.z.float() - m) / case["temperature"] - ls
    p = torch.exp(lp)
    given = st.tokens >= 0
    g_lp = torch.where(given, st.g_lp, torch.zeros(()).cuda())[:, None]
    g = -g_lp * p
    g.scatter_add_(1, st.tokens.clamp_min(0).long()[:, None], g_lp)
    if case["entropy"]:
        g -= st.g_h[:, None] * p * (lp.clamp_min(-1e30) + st.entropy[:, None])
    return (g / case["temperature"]).to(st.z.dtype)


def _places(st, pages, n):
    """Where the n tokens of a response lie in the pool."""
    return [pages[t // PAGE] * PAGE + t % PAGE for t in range(n)]


def _plain_import(st, kv):
    """Dense rows into fresh pages; each response's list of pages."""
    pages = [[st.free.pop() for _ in range(-(-k.shape[1] // PAGE))] for k, _ in kv]
    at = torch.tensor([x for p, (k, _) in zip(pages, kv) for x in _places(st, p, k.shape[1])], device="cuda")
    st.pool_k[:, at] = _stored(st.case, torch.cat([k for k, _ in kv], 1)).view(st.pool_k.dtype)
    st.pool_v[:, at] = _stored(st.case, torch.cat([v for _, v in kv], 1)).view(st.pool_v.dtype)
    return pages


def _plain_export(st, pages):
    at = torch.tensor([x for p, n in zip(pages, st.lens) for x in _places(st, p, n)], device="cuda")
    k, v = (p[:, at].view(st.dtype).to(_dtype(st.case)).split(st.lens, 1) for p in (st.pool_k, st.pool_v))
    return list(zip(k, v))


def _plain_branch(st):
    # full pages are shared; a branch goes on in its last page: its own copy
    forks = [st.pages[src][:-(-t // PAGE)] for src, t in zip(st.src, st.kept)]
    part = [i for i, t in enumerate(st.kept) if t % PAGE]
    taken = [st.free.pop() for _ in part]
    if part:
        to = torch.tensor([x for p in taken for x in _places(st, [p], PAGE)], device="cuda")
        at = torch.tensor([x for i in part for x in _places(st, forks[i][-1:], PAGE)], device="cuda")
        st.pool_k[:, to] = st.pool_k[:, at]
        st.pool_v[:, to] = st.pool_v[:, at]
    for i, page in zip(part, taken):
        forks[i][-1] = page
    out = _plain_export(st, forks)
    st.free.extend(reversed(taken))
    return out


def _plain_carry(st):
    pages = _plain_import(st, st.kv)
    out = _plain_export(st, pages)
    st.free.extend(x for p in reversed(pages) for x in reversed(p))
    return out


# ---------------------------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    return {"rotate": _exact_rotate, "score": _exact_score, "grad": _exact_grad, "branch": _exact_pages,
            "carry": _exact_pages}[case["kind"]](case, seed)


def _exact_rotate(case, seed):
    """x_a + i x_b times amplitude * e^(i position frequency), pair by pair."""
    rd, s = case["rotary_dim"], case["factor"]
    freq, amplitude = [], 1.0
    for j in range(rd // 2):
        f = math.exp(-2.0 * j / rd * math.log(BASE))
        if case["scaling"] == "linear":
            f /= s
        elif case["scaling"] == "ntk":
            f = math.exp(-2.0 * j / rd * (math.log(BASE) + rd / (rd - 2.0) * math.log(s)))
        elif case["scaling"] == "bands":
            wave = 2 * math.pi / f
            if wave > TRAINED / 1.0:
                f /= s
            elif wave > TRAINED / 4.0:
                mix = (TRAINED / wave - 1.0) / 3.0
                f = (1 - mix) * f / s + mix * f
        elif case["scaling"] == "yarn":
            ends = [rd / 2 * math.log(TRAINED / turns / 2 / math.pi) / math.log(BASE) for turns in (32.0, 1.0)]
            lo, hi = max(math.floor(ends[0]), 0), min(math.ceil(ends[1]), rd - 1)
            mix = min(1.0, max(0.0, (j - lo) / max(hi - lo, 0.001)))
            f = mix * f / s + (1 - mix) * f
            amplitude = 1.0 + 0.1 * math.log(s)
        freq.append(f)
    sign = -1.0 if case["inverse"] else 1.0
    theta = sign * torch.tensor(_positions(case), dtype=torch.float64)[:, None] * torch.tensor(freq, dtype=torch.float64)
    turn = torch.polar(torch.full_like(theta, amplitude), theta).cuda()[None, :, None]

    def rotated(x):
        x = x.double()
        first = torch.arange(0, rd, 2) if case["layout"] == "interleaved" else torch.arange(rd // 2)
        second = first + (1 if case["layout"] == "interleaved" else rd // 2)
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    q, k = _rotate_inputs(case, seed)
    return {"q": rotated(q), "k": rotated(k)}


def _exact_score(case, seed):
    z, tokens, _, _ = _logits(case, seed)
    n, top = case["rows"], case["top"]
    logprob, entropy = (torch.empty(n, dtype=torch.float64, device="cuda") for _ in range(2))
    stats = torch.empty(n, 2, dtype=torch.float64, device="cuda")
    top_id = torch.empty(n, top, dtype=torch.int32, device="cuda")
    top_lp = torch.empty(n, top, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 25) // case["vocab"])
    for a in range(0, n, step):
        b = min(n, a + step)
        x = z[a:b].double() / case["temperature"]
        lse = torch.logsumexp(x, 1, keepdim=True)
        stats[a:b, 0] = z[a:b].double().amax(1)
        stats[a:b, 1] = lse[:, 0] - x.amax(1)
        lp = x - lse
        p = lp.exp()
        entropy[a:b] = -torch.where(p > 0, p * lp, torch.zeros_like(lp)).sum(1)
        rows = torch.arange(b - a, device="cuda")
        t = tokens[a:b].long()
        logprob[a:b] = torch.where(t >= 0, lp[rows, t.clamp_min(0)], torch.zeros_like(lp[:, 0]))
        place = torch.arange(case["vocab"], device="cuda")
        for j in range(top):  # the largest that is left, the first of them
            best = lp.amax(1, keepdim=True)
            at = torch.where(lp == best, place, case["vocab"]).amin(1)
            top_id[a:b, j], top_lp[a:b, j] = at.int(), best[:, 0]
            lp[rows, at] = -math.inf
    out = {"logprob": logprob, "entropy": entropy, "stats": stats}
    if top:
        out.update(top_id=top_id, top_logprob=top_lp)
    return out


def _exact_grad(case, seed):
    z, tokens, g_lp, g_h = _logits(case, seed)
    out = torch.empty(z.shape, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 25) // case["vocab"])
    for a in range(0, z.shape[0], step):
        x = z[a:a + step].double() / case["temperature"]
        p = torch.softmax(x, 1)
        t = tokens[a:a + step].long()
        rows = torch.arange(len(t), device="cuda")
        up = torch.where(t >= 0, g_lp[a:a + step].double(), torch.zeros_like(p[:, 0]))
        g = -up[:, None] * p
        g[rows, t.clamp_min(0)] += up
        if case["entropy"]:
            # H = -sum p log p; dH/dx_j = -p_j (log p_j + H)
            plogp = torch.where(p > 0, p * torch.log_softmax(x, 1), torch.zeros_like(p))
            h = -plogp.sum(1, keepdim=True)
            g -= g_h[a:a + step, None].double() * (plogp + p * h)
        out[a:a + step] = g / case["temperature"]
    return out


def _exact_pages(case, seed):
    def rounded(x):  # to the nearest of E4M3's values (ties to the even code), as float64
        if case["cache"] != "e4m3":
            return x.double()
        x = x.double().clamp(-448, 448)
        quantum = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
        return torch.round(x / quantum) * quantum

    kv = [(rounded(k), rounded(v)) for k, v in _kv(case, seed)]
    if case["kind"] == "carry":
        return kv
    return [(kv[i][0][:, :t].contiguous(), kv[i][1][:, :t].contiguous()) for i, t in _branches(case)]
