"""Operators of a sample group's model around the decode step: heads that are normed and rotated, the
attention of prompts and of a learner's batch, and the choice of the next tokens.

Five kinds of pass:

* norm         the norm of every Q and K head (root of the mean of squares, a weight per element) and its
               rotary position in one pass: `entry` "step" is one running step (every live slot of a
               context, all layers at once or one), "rows" a prompt's or a training batch's rows.
* norm_grad    its gradient with respect to the rows and to the weights.
* attend       causal attention of packed sequences with grouped heads, and the log of each row's sum.
               A sequence's queries are its last tokens: as many as its keys (a whole prompt, a learner's
               prompt and response) or fewer (a chunk of a prompt, further tokens of a conversation).
* attend_grad  its gradient with respect to Q, K and V.
* sample       one token per row of logits from given uniform numbers, at a temperature, from the entries
               that a count (top-k), a mass (top-p) and a share of the largest probability (min-p) leave.

Shapes are those of this repository's presets (Qwen3-1.7B and 8B attention layouts, the tiny fp32
group), its tests (other head counts and sizes) and sizes between them; vocabularies are of ordinary
sizes, even and odd.  Q, K and V rows are N(0, 1), norm weights lie around 1.  Logits are normal with a
spread of some units and a padded, masked end.
"""

import math

import numpy as np
import torch

own = False

SAMPLES = 1 << 20  # sample ids of a context
BASE = 1000000.0   # rotary base
EPS = 1e-6         # of the norm


def listed():
    qwen17 = {"q_heads": 16, "kv_heads": 8, "head_dim": 128}
    qwen8 = {"q_heads": 32, "kv_heads": 8, "head_dim": 128}
    return [
        # one layer's Q and K heads of a running step (throughput preset, 16 slots), out of the fused
        # projection: what each layer of a model calls before its attention; all latency
        {"name": "norm_step_layer", "kind": "norm", "entry": "step", "layers": 1, **qwen17, "tokens": 16, "first": 2048,
         "layout": "half", "rotary_dim": 128, "dtype": "bf16", "weights": "bf16", "fused": True},
        # four prompts' rows of one layer before their attention (8B-shaped preset)
        {"name": "norm_prompts_8b", "kind": "norm", "entry": "rows", "layers": 1, **qwen8, "tokens": 7424, "first": 0,
         "layout": "half", "rotary_dim": 128, "dtype": "bf16", "weights": "bf16", "fused": True},
        # a learner's gradient, fp32 weights
        {"name": "norm_grad_learner", "kind": "norm_grad", "layers": 1, **qwen17, "tokens": 8192, "first": 0,
         "layout": "half", "rotary_dim": 128, "dtype": "bf16", "weights": "f32", "fused": False},
        # a small gradient in fp32: interleaved pairs, three quarters of a head, far positions, an odd count
        {"name": "norm_grad_f32", "kind": "norm_grad", "layers": 1, "q_heads": 12, "kv_heads": 4, "head_dim": 64,
         "tokens": 1037, "first": 100003, "layout": "interleaved", "rotary_dim": 48, "dtype": "f32", "weights": "f32",
         "fused": False},
        # short prompts of the tiny fp32 group's heads, one of a single token: the smallest attention
        {"name": "attend_tiny_f32", "kind": "attend", "q_heads": 4, "kv_heads": 2, "head_dim": 64, "q_lens": "32,1,17,64",
         "k_lens": "", "dtype": "f32", "fused": False},
        # the prompts of the 8B-shaped preset in one pack (the most work but for a gradient)
        {"name": "attend_prompts_8b", "kind": "attend", **qwen8, "q_lens": "256,1024,2048,4096", "k_lens": "",
         "dtype": "bf16", "fused": True},
        # chunks of long prompts and single further tokens over what went before them, three heads a group
        {"name": "attend_chunks", "kind": "attend", "q_heads": 24, "kv_heads": 8, "head_dim": 64,
         "q_lens": "512,1,333,128,1", "k_lens": "4096,1777,2001,128,6001", "dtype": "bf16", "fused": False},
        # a learner's batch: prompts of 512 tokens, each with a response, ragged
        {"name": "attend_grad_learner", "kind": "attend_grad", **qwen17, "q_lens": "912,1536,640,2560,777,1345,2048,1001",
         "k_lens": "", "dtype": "bf16", "fused": False},
        # a small gradient in fp32 with odd lengths
        {"name": "attend_grad_f32", "kind": "attend_grad", "q_heads": 6, "kv_heads": 2, "head_dim": 64,
         "q_lens": "129,300,1,77", "k_lens": "", "dtype": "f32", "fused": False},
        # the next tokens of a running step: 16 slots
        {"name": "sample_step", "kind": "sample", "rows": 16, "vocab": 151936, "masked": 267, "temperature": 0.8,
         "top_k": 50, "top_p": 0.95, "min_p": 0.0, "dtype": "bf16"},
        # a batch of an odd vocabulary in fp32: a mass and a share of the largest probability
        {"name": "sample_f32_odd", "kind": "sample", "rows": 101, "vocab": 50257, "masked": 0, "temperature": 1.0,
         "top_k": 0, "top_p": 0.9, "min_p": 0.001, "dtype": "f32"},
        # many samplers' rows at once, from the whole distribution (a group's policy as it is)
        {"name": "sample_wide", "kind": "sample", "rows": 512, "vocab": 151936, "masked": 267, "temperature": 1.0,
         "top_k": 0, "top_p": 1.0, "min_p": 0.0, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_MOST_BYTES = 512 * 151936 * 2                      # of the largest listed pass of little arithmetic
_MOST_FLOPS = 180e9                                 # of the largest listed attention


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "attend", "attend", "attend_grad", "sample", "sample"])
    while True:
        if kind == "sample":
            c = {"kind": kind, "rows": _log_int(rng, 1, 2048), "vocab": _log_int(rng, 1000, 262144),
                 "temperature": rng.choice([1.0, 1.0, 0.6, 0.8, 1.3]), "dtype": rng.choice(["bf16", "bf16", "f32"])}
            c["masked"] = rng.choice([0, c["vocab"] // 500, c["vocab"] // 3])
            c["top_k"] = rng.choice([0, 0, 1, 20, 64, _log_int(rng, 1, c["vocab"])])
            c["top_p"] = rng.choice([1.0, 1.0, 0.95, 0.8, round(rng.uniform(0.05, 0.999), 3)])
            c["min_p"] = rng.choice([0.0, 0.0, 0.05, 0.001])
        else:
            hkv, hpk, d = rng.choice([8, 8, 4, 2, 1]), rng.choice([1, 2, 3, 4, 8]), rng.choice([128, 128, 64])
            c = {"kind": kind, "q_heads": hkv * hpk, "kv_heads": hkv, "head_dim": d,
                 "dtype": rng.choice(["bf16", "bf16", "f32"]), "fused": rng.random() < 0.5}
            if kind in ("norm", "norm_grad"):
                entry = "rows" if kind == "norm_grad" else rng.choice(["step", "rows"])
                if kind == "norm":
                    c["entry"] = entry
                c["layers"] = _log_int(rng, 1, 36) if entry == "step" else 1
                c["tokens"] = (_log_int(rng, 1, (16 if c["dtype"] == "f32" else 64) // hpk) if entry == "step"
                               else _log_int(rng, 1, 16384))
                c["first"] = rng.randrange(0, 4096) if entry == "step" else rng.choice([0, _log_int(rng, 1, 1 << 20)])
                c["layout"] = rng.choice(["half", "interleaved"])
                c["rotary_dim"] = rng.choice([d, d, d // 2, 2 * rng.randrange(1, d // 2 + 1)])
                c["weights"] = rng.choice([c["dtype"], "f32"])
            else:
                n = _log_int(rng, 1, 24)
                k_lens = [_log_int(rng, 1, 6144 if c["dtype"] == "bf16" else 1024) for _ in range(n)]
                chunks = rng.random() < 0.4
                q_lens = [rng.choice([1, k, _log_int(rng, 1, k)]) for k in k_lens] if chunks else k_lens
                c["q_lens"] = ",".join(map(str, q_lens))
                c["k_lens"] = ",".join(map(str, k_lens)) if chunks else ""
                # what the plain form pads to, in rows and columns of scores
                if n * max(q_lens) * max(k_lens) * hkv * hpk > 4 * 4096 * 4096 * 32:
                    continue
        w = work(c)
        if w["bytes"] <= _MOST_BYTES and w["flops"] <= _MOST_FLOPS:
            return c


# ---------------------------------------------------------------------------------------------
# Sizes
# ---------------------------------------------------------------------------------------------
def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _size(name):
    return 4 if name == "f32" else 2


def _lens(case):
    q = [int(x) for x in case["q_lens"].split(",")]
    return q, [int(x) for x in case["k_lens"].split(",")] if case["k_lens"] else q


def _starts(lens):
    return [sum(lens[:i]) for i in range(len(lens) + 1)]


def _positions(case):
    """Position of every token: a running step's slots are at all response lengths below 1024."""
    n = case["tokens"]
    if case.get("entry") == "step":
        return [case["first"] + (617 * s) % 1024 for s in range(n)]
    return list(range(case["first"], case["first"] + n))


def work(case):
    kind = case["kind"]
    if kind == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * _size(case["dtype"]) + case["rows"] * 16, "flops": 5 * n}
    heads, d, es = case["q_heads"] + case["kv_heads"], case["head_dim"], _size(case["dtype"])
    if kind in ("norm", "norm_grad"):
        n, w = case["layers"] * case["tokens"] * heads * d, 2 * case["layers"] * d
        if kind == "norm":
            return {"bytes": 2 * n * es + w * _size(case["weights"]), "flops": 7 * n}
        return {"bytes": 3 * n * es + w * (_size(case["weights"]) + 4), "flops": 16 * n}
    q_lens, k_lens = _lens(case)
    pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(q_lens, k_lens))  # (query, key) that meet
    q, kv = sum(q_lens) * case["q_heads"] * d * es, sum(k_lens) * case["kv_heads"] * d * es
    lse = sum(q_lens) * case["q_heads"] * 4
    if kind == "attend":
        return {"bytes": 2 * q + 2 * kv + lse, "flops": 4 * d * case["q_heads"] * pairs}
    return {"bytes": 4 * q + 4 * kv + lse, "flops": 10 * d * case["q_heads"] * pairs}


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _norm_inputs(case, seed):
    """Q and K rows [layers, tokens, heads, d] (fused: views of one projection output [.., Hq + 2 Hkv, d]), the
    weights [layers, d] of each, and gradients of the outputs."""
    gen = _generator(seed)
    L, T, hq, hkv, d = case["layers"], case["tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
    x = _randn(gen, L, T, hq + 2 * hkv, d).to(_type(case["dtype"]))
    q, k = x[:, :, :hq], x[:, :, hq:hq + hkv]
    if not case["fused"]:
        q, k = q.contiguous(), k.contiguous()
    wq, wk = ((1 + 0.1 * _randn(gen, L, d)).to(_type(case["weights"])) for _ in range(2))
    dq, dk = (_randn(gen, *t.shape).to(t.dtype) for t in (q, k))
    return q, k, wq, wk, dq, dk


def _attend_inputs(case, seed):
    """Packed rows q [Tq, Hq, d], k and v [Tk, Hkv, d] (fused, where queries and keys are the same tokens: views of
    one projection output) and a gradient of the output."""
    gen = _generator(seed)
    q_lens, k_lens = _lens(case)
    hq, hkv, d, t = case["q_heads"], case["kv_heads"], case["head_dim"], _type(case["dtype"])
    if case["fused"] and not case["k_lens"]:
        x = _randn(gen, sum(q_lens), hq + 2 * hkv, d).to(t)
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    else:
        q = _randn(gen, sum(q_lens), hq, d).to(t)
        k, v = (_randn(gen, sum(k_lens), hkv, d).to(t) for _ in range(2))
    return q, k, v, _randn(gen, sum(q_lens), hq, d).to(t)


def _logits(case, seed):
    """Logits [rows, vocab] with a masked end of -inf, and a uniform number per row."""
    gen = _generator(seed)
    n, v = case["rows"], case["vocab"]
    z = torch.empty(n, v, dtype=_type(case["dtype"]), device="cuda")
    step = max(1, (1 << 26) // v)
    for a in range(0, n, step):
        x = _randn(gen, min(n, a + step) - a, v)
        x *= 3.0
        z[a:a + step] = x.to(z.dtype)
    z[:, v - case["masked"]:] = -math.inf
    return z, torch.rand(n, generator=gen, device="cuda")


# ---------------------------------------------------------------------------------------------
# prepare
# ---------------------------------------------------------------------------------------------
class _State:
    pass


def prepare(case, seed):
    st = _State()
    st.case = case
    return {"norm": _prepare_norm, "norm_grad": _prepare_norm, "attend": _prepare_attend,
            "attend_grad": _prepare_attend, "sample": _prepare_sample}[case["kind"]](st, seed)


def _own_type(name):
    from paper_2506_22950_amd import infs

    return infs.F32 if name == "f32" else infs.BF16


def _prepare_norm(st, seed):
    case = st.case
    st.q, st.k, st.wq, st.wk, st.dq, st.dk = _norm_inputs(case, seed)
    if own:
        from paper_2506_22950_amd import infs

        st.rotary = infs.Rotary(infs.make_rotary_config(
            head_dim=case["head_dim"], rotary_dim=case["rotary_dim"], base=BASE,
            layout=infs.ROTARY_INTERLEAVED if case["layout"] == "interleaved" else infs.ROTARY_HALF))
        st.norms = infs.make_norms(weight_q=st.wq, weight_k=st.wk, dtype=_own_type(case["weights"]), eps=EPS,
                                   layer_stride=case["head_dim"])
        st.q_out, st.k_out = (torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in (st.q, st.k))
        if case["kind"] == "norm_grad":
            st.dw = torch.empty(2, case["head_dim"], device="cuda")
            st.workspace = torch.empty(infs.norm_rotate_grad_workspace(case["tokens"], case["head_dim"]),
                                       dtype=torch.uint8, device="cuda")
        elif case["entry"] == "step" and case["q_heads"] // case["kv_heads"] not in (1, 2, 4, 8):
            # heads that no context decodes: their rows, layer by layer
            st.ctx, st.positions = None, torch.tensor(_positions(case), dtype=torch.int32, device="cuda")
        elif case["entry"] == "step":
            # a context whose slots hold responses of the positions' lengths
            n, cap, first = case["tokens"], 1024, case["first"]
            st.ctx = infs.Context(infs.make_config(
                num_layers=case["layers"], num_q_heads=case["q_heads"], num_kv_heads=case["kv_heads"],
                head_dim=case["head_dim"], num_prompts=1, slots_per_prompt=n, samples_per_prompt=SAMPLES,
                max_prompt_len=first, max_suffix_len=cap, dtype=_own_type(case["dtype"])),
                stream=torch.cuda.current_stream())
            none = torch.zeros(case["layers"] * max(cap, first), case["kv_heads"], case["head_dim"],
                               dtype=st.q.dtype, device="cuda")
            for layer in range(case["layers"]):
                st.ctx.prefill_shared(0, layer, first, none, none)
            lens = [p - first for p in _positions(case)]
            st.ctx.import_responses(list(range(n)), list(range(n)), lens, [none] * n, [none] * n)
            st.ctx.sync()
    else:
        pairs = torch.arange(case["rotary_dim"] // 2, dtype=torch.float64, device="cuda")
        st.frequencies = BASE ** (-2.0 * pairs / case["rotary_dim"])
        st.positions = torch.tensor(_positions(case), dtype=torch.int32, device="cuda")
    return st


def _prepare_attend(st, seed):
    case = st.case
    st.q, st.k, st.v, st.d_o = _attend_inputs(case, seed)
    q_lens, k_lens = _lens(case)
    st.q_starts, st.k_starts = (torch.tensor(_starts(x), dtype=torch.int32, device="cuda") for x in (q_lens, k_lens))
    st.longest = max(q_lens), max(k_lens)  # what a batch is padded to
    if case["kind"] == "attend_grad":
        # what the forward pass left
        out = _plain_attend(st)
        st.o, st.lse = out["o"], out["lse"]
    if own:
        from paper_2506_22950_amd import infs

        st.attention = infs.Attention(infs.make_attention_config(
            num_q_heads=case["q_heads"], num_kv_heads=case["kv_heads"], head_dim=case["head_dim"],
            dtype=_own_type(case["dtype"]), max_tokens=sum(q_lens)), stream=torch.cuda.current_stream())
        if case["kind"] == "attend":
            st.o = torch.zeros(st.q.shape, dtype=st.q.dtype, device="cuda")
            st.lse = torch.zeros(st.q.shape[:2], device="cuda")
        else:
            st.out = [torch.zeros(x.shape, dtype=x.dtype, device="cuda") for x in (st.q, st.k, st.v)]
    return st


def _prepare_sample(st, seed):
    case = st.case
    st.z, st.u = _logits(case, seed)
    if own:
        from paper_2506_22950_amd import infs

        n = case["rows"]
        st.sampler = infs.Sampler(infs.make_sampler_config(vocab=case["vocab"], dtype=_own_type(case["dtype"]),
                                                           max_rows=n), stream=torch.cuda.current_stream())
        st.sampling = infs.make_sampling(**{k: case[k] for k in ("temperature", "top_k", "top_p", "min_p")})
        st.token, st.kept = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
        st.logprob = torch.empty(n, device="cuda")
    return st


# ---------------------------------------------------------------------------------------------
# run
# ---------------------------------------------------------------------------------------------
def run(state):
    kind = state.case["kind"]
    if own:
        return {"norm": _own_norm, "norm_grad": _own_norm_grad, "attend": _own_attend, "attend_grad": _own_attend_grad,
                "sample": _own_sample}[kind](state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "attend": _plain_attend,
            "attend_grad": _plain_attend_grad, "sample": _plain_sample}[kind](state)


# ---- the framework's calls -------------------------------------------------------------------
def _rows(x, out=None):
    """A tensor [.., tokens, heads, d] (any strides above a head's elements) as infs.rotary_rows takes it; out: dense."""
    from paper_2506_22950_amd import infs

    layer = x.stride(0) if x.dim() == 4 else 0
    return infs.rotary_rows(x, out, x.shape[-2], in_strides=(x.stride(-3), x.stride(-2), layer))


def _own_norm(st):
    from paper_2506_22950_amd import infs

    case = st.case
    q, k = _rows(st.q, st.q_out), _rows(st.k, st.k_out)
    if case["entry"] == "step" and st.ctx is None:
        for i in range(case["layers"]):
            st.rotary.norm_rotate_rows(_own_type(case["dtype"]), case["tokens"], infs.layer_norms(st.norms, i),
                                       _rows(st.q[i], st.q_out[i]), _rows(st.k[i], st.k_out[i]), positions=st.positions,
                                       stream=torch.cuda.current_stream())
    elif case["entry"] == "step":
        st.ctx.norm_rotate_step(st.rotary, st.norms, q, k, num_layers=case["layers"])
    else:
        st.rotary.norm_rotate_rows(_own_type(case["dtype"]), case["tokens"], st.norms, q, k, first_position=case["first"],
                                   stream=torch.cuda.current_stream())
    return {"q": st.q_out, "k": st.k_out}


def _own_norm_grad(st):
    case = st.case
    st.rotary.norm_rotate_grad(_own_type(case["dtype"]), case["tokens"], st.norms, q=_rows(st.q, st.q_out),
                               k=_rows(st.k, st.k_out), dq=_rows(st.dq), dk=_rows(st.dk), d_weight_q=st.dw[0],
                               d_weight_k=st.dw[1], workspace=st.workspace, first_position=case["first"],
                               stream=torch.cuda.current_stream())
    return {"q": st.q_out, "k": st.k_out, "weights": st.dw}


def _own_attend(st):
    st.attention.attend(len(st.q_starts) - 1, st.q.shape[0], st.q_starts, _rows(st.q, st.o), _rows(st.k), _rows(st.v),
                        lse=st.lse, k_tokens=st.k.shape[0], k_offsets=st.k_starts)
    return {"o": st.o, "lse": st.lse}


def _own_attend_grad(st):
    dq, dk, dv = st.out
    st.attention.grad(len(st.q_starts) - 1, st.q.shape[0], st.q_starts, _rows(st.q, dq), _rows(st.k, dk), _rows(st.v, dv),
                      o=_rows(st.o), d_o=_rows(st.d_o), lse=st.lse, k_tokens=st.k.shape[0], k_offsets=st.k_starts)
    return {"q": dq, "k": dk, "v": dv}


def _own_sample(st):
    st.sampler.sample(st.z.shape[0], st.z, st.u, st.token, logprob=st.logprob, kept=st.kept, sampling=st.sampling)
    return {"token": st.token, "logprob": st.logprob, "kept": st.kept}


# ---- the plain forms -------------------------------------------------------------------------
def _turned(case, x, cos, sin):
    rd = case["rotary_dim"]
    r = x[..., :rd]
    if case["layout"] == "interleaved":
        a, b = r[..., 0::2], r[..., 1::2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = r[..., :rd // 2], r[..., rd // 2:]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., rd:]], -1)


def _turns(st):
    angle = st.positions.double()[:, None] * st.frequencies
    return torch.cos(angle).float()[None, :, None], torch.sin(angle).float()[None, :, None]


def _plain_norm(st):
    cos, sin = _turns(st)

    def out(x, w):
        y = x.float()
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()[:, None, None]
        return _turned(st.case, y, cos, sin).to(x.dtype)

    return {"q": out(st.q, st.wq), "k": out(st.k, st.wk)}


def _plain_norm_grad(st):
    cos, sin = _turns(st)

    def out(x, w, dy):
        y = x.float()
        r = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
        y = y * r
        dz = _turned(st.case, dy.float(), cos, -sin)
        g = dz * w.float()[:, None, None]
        dx = r * (g - y * (g * y).mean(-1, keepdim=True))
        return dx.to(x.dtype), (dz * y).sum((0, 1, 2))

    (dq, dwq), (dk, dwk) = out(st.q, st.wq, st.dq), out(st.k, st.wk, st.dk)
    return {"q": dq, "k": dk, "weights": torch.stack([dwq, dwk])}


def _padded(starts, longest):
    """Where token t of every sequence lies among the packed rows, and whether it is there."""
    t = torch.arange(longest, device="cuda")
    there = t < (starts[1:] - starts[:-1])[:, None]
    return torch.where(there, starts[:-1, None] + t, 0).long(), there


def _scores(st, q, k):
    """Scores [sequences, Hkv, Hq/Hkv * queries, keys] in 32 bits, masked entries -inf, and which are not."""
    case = st.case
    n, (lq, lk), hpk = len(st.q_starts) - 1, st.longest, case["q_heads"] // case["kv_heads"]
    q_len, k_len = st.q_starts.diff(), st.k_starts.diff()
    last = torch.arange(lq, device="cuda") + (k_len - q_len)[:, None]  # the last key of each query
    seen = torch.arange(lk, device="cuda") <= last[:, :, None]
    seen &= (torch.arange(lk, device="cuda") < k_len[:, None])[:, None]
    seen = seen[:, None, None].expand(n, 1, hpk, lq, lk).reshape(n, 1, hpk * lq, lk)
    s = torch.matmul(q, k.transpose(-1, -2)) * case["head_dim"] ** -0.5
    return s.masked_fill_(~seen, -math.inf), seen


def _grouped(st, x, at):
    """Packed rows [T, H, d] as [sequences, Hkv, H/Hkv * tokens, d] in 32 bits."""
    hkv = st.case["kv_heads"]
    y = x[at].float().unflatten(2, (hkv, -1))  # [n, t, Hkv, g, d]
    return y.permute(0, 2, 3, 1, 4).flatten(2, 3)


def _packed(st, y, there, like):
    """_grouped's rows back in their places among those of `like`."""
    z = y.unflatten(2, (-1, there.shape[1])).permute(0, 3, 1, 2, 4).flatten(2, 3)
    return z[there].to(like.dtype).reshape(like.shape)


def _plain_attend(st):
    at_q, q_there = _padded(st.q_starts, st.longest[0])
    at_k, _ = _padded(st.k_starts, st.longest[1])
    s, _ = _scores(st, _grouped(st, st.q, at_q), _grouped(st, st.k, at_k))
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, _grouped(st, st.v, at_k)) / total
    lse = m + torch.log(total)
    return {"o": _packed(st, o, q_there, st.q), "lse": _packed(st, lse, q_there, st.q[..., :1].float())[..., 0]}


def _plain_attend_grad(st):
    at_q, q_there = _padded(st.q_starts, st.longest[0])
    at_k, k_there = _padded(st.k_starts, st.longest[1])
    q, o, d_o, k, v = (_grouped(st, x, at) for x, at in ((st.q, at_q), (st.o, at_q), (st.d_o, at_q), (st.k, at_k),
                                                         (st.v, at_k)))
    s, _ = _scores(st, q, k)
    p = s.sub_(_grouped(st, st.lse[..., None], at_q)).exp_()
    # padded queries give nothing to the keys
    p *= q_there[:, None, None].expand(-1, -1, q.shape[2] // q_there.shape[1], -1).flatten(2)[..., None]
    dv = torch.matmul(p.transpose(-1, -2), d_o)
    ds = torch.matmul(d_o, v.transpose(-1, -2))
    ds = ds.sub_((d_o * o).sum(-1, keepdim=True)).mul_(p).mul_(st.case["head_dim"] ** -0.5)
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(-1, -2), q)
    return {"q": _packed(st, dq, q_there, st.q), "k": _packed(st, dk, k_there, st.k), "v": _packed(st, dv, k_there, st.v)}


def _plain_sample(st):
    """64 bits: which entries a sum keeps, and where the drawn number falls, hang on the last digits."""
    case = st.case
    z = st.z.double()
    w = torch.exp((z - z.amax(1, keepdim=True)) / case["temperature"])
    z, order = torch.sort(z, dim=1, descending=True, stable=True)  # most probable first, equal ones by the lower index
    keep = z > -math.inf
    w = w.gather(1, order)
    if case["top_k"]:
        keep[:, case["top_k"]:] = False
    if case["top_p"] < 1:
        w = w * keep
        before = torch.cumsum(w, 1) - w
        keep &= before < case["top_p"] * w.sum(1, keepdim=True)
    if case["min_p"] > 0:
        keep &= w >= case["min_p"]
    w = torch.zeros_like(w).scatter_(1, order, w * keep)  # by index again
    sums = torch.cumsum(w, 1)
    total = sums[:, -1:]
    # the first whose sum is above the number's share of the total
    token = (sums > st.u.double()[:, None] * total).byte().argmax(1)
    logprob = torch.log(w.gather(1, token[:, None]) / total)[:, 0]
    return {"token": token.int(), "logprob": logprob.float(), "kept": keep.sum(1).int()}


# ---------------------------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    return {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "attend": _exact_attend,
            "attend_grad": _exact_attend, "sample": _exact_sample}[case["kind"]](case, seed)


def _turning(case):
    """The rotation of every token as a complex number per pair, and the elements of each pair."""
    rd = case["rotary_dim"]
    freq = [math.exp(-2.0 * j / rd * math.log(BASE)) for j in range(rd // 2)]
    theta = torch.tensor(_positions(case), dtype=torch.float64)[:, None] * torch.tensor(freq, dtype=torch.float64)
    first = torch.arange(0, rd, 2) if case["layout"] == "interleaved" else torch.arange(rd // 2)
    second = first + (1 if case["layout"] == "interleaved" else rd // 2)
    return torch.polar(torch.ones_like(theta), theta).cuda()[None, :, None], first, second


def _turn(x, turn, first, second):
    y = x.clone()
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_norm(case, seed):
    q, k, wq, wk, _, _ = _norm_inputs(case, seed)
    turn = _turning(case)

    def out(x, w):
        x = x.double()
        return _turn(x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["head_dim"] + EPS) * w.double()[:, None, None],
                     *turn)

    return {"q": out(q, wq), "k": out(k, wk)}


def _exact_norm_grad(case, seed):
    """y = w x / n with n = sqrt(|x|^2 / d + eps): the Jacobian's columns, element by element."""
    q, k, wq, wk, dq, dk = _norm_inputs(case, seed)
    turn, first, second = _turning(case)

    def out(x, w, dy):
        x, w = x.double(), w.double()[:, None, None]
        back = _turn(dy.double(), turn.conj(), first, second)
        n = torch.sqrt(x.square().sum(-1, keepdim=True) / case["head_dim"] + EPS)
        along = (back * w * x).sum(-1, keepdim=True)
        return back * w / n - x * along / (case["head_dim"] * n ** 3), (back * x / n).sum(dim=(0, 1, 2))

    (gq, gwq), (gk, gwk) = out(q, wq, dq), out(k, wk, dk)
    return {"q": gq, "k": gk, "weights": torch.stack([gwq, gwk])}


def _exact_attend(case, seed):
    """Sequence by sequence and head by head."""
    q, k, v, d_o = _attend_inputs(case, seed)
    hpk, scale = case["q_heads"] // case["kv_heads"], 1.0 / math.sqrt(case["head_dim"])
    grad = case["kind"] == "attend_grad"
    o, lse = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    dq, dk, dv = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (q, k, v))
    q_lens, k_lens = _lens(case)
    for a, n, b, m in zip(_starts(q_lens), q_lens, _starts(k_lens), k_lens):
        future = torch.ones(n, m, dtype=torch.bool, device="cuda").triu(m - n + 1)
        for h in range(case["q_heads"]):
            g = h // hpk
            x, y, z = q[a:a + n, h].double(), k[b:b + m, g].double(), v[b:b + m, g].double()
            s = (x @ y.T * scale).masked_fill(future, -math.inf)
            rows = torch.logsumexp(s, 1)
            p = torch.exp(s - rows[:, None])
            o[a:a + n, h], lse[a:a + n, h] = p @ z, rows
            if grad:
                up = d_o[a:a + n, h].double()
                dp = up @ z.T
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * scale
                dq[a:a + n, h] = ds @ y
                dk[b:b + m, g] += ds.T @ x
                dv[b:b + m, g] += p.T @ up
    return {"q": dq, "k": dk, "v": dv} if grad else {"o": o, "lse": lse}


def _exact_sample(case, seed):
    """Row by row on the host."""
    if case["rows"] * case["vocab"] > 100_000_000:
        return None  # some 30 ms a row
    z, u = _logits(case, seed)
    z, u = z.float().cpu().numpy(), u.cpu().numpy()
    tokens, kept, logprob = [], [], []
    for row, x in zip(z, u):
        p = np.exp((row.astype(np.float64) - float(row.max())) / case["temperature"])
        p /= p.sum()
        ranking = np.lexsort((np.arange(len(p)), -row))
        ranking = ranking[row[ranking] > -np.inf]
        if case["top_k"]:
            ranking = ranking[:case["top_k"]]
        if case["top_p"] < 1:
            mass = np.cumsum(p[ranking])
            ranking = ranking[:1 + int(np.sum(mass[:-1] < case["top_p"] * mass[-1]))]
        ranking = ranking[p[ranking] >= case["min_p"] * p.max()]
        chosen = np.sort(ranking)
        mass = np.cumsum(p[chosen])
        at = min(int(np.sum(mass <= float(x) * mass[-1])), len(chosen) - 1)
        tokens.append(int(chosen[at]))
        kept.append(len(chosen))
        logprob.append(math.log(p[chosen[at]] / mass[-1]))
    return {"token": np.array(tokens, dtype=np.int32), "logprob": np.array(logprob), "kept": np.array(kept, dtype=np.int32)}
