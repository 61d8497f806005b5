"""GPU: forked, taken-in and handed-out responses hold exactly the rows they were given (E4M3: rounded
as the oracle rounds them), and decode on them gives bit for bit what decode on responses grown token by
token gives."""

import numpy as np
import pytest

from oracle import round_e4m3
from paper_2506_22950_amd import infs

pytestmark = pytest.mark.gpu

# dtype/cache, head_dim, q heads, kv heads, slots per prompt: plain rows and MFMA prefixes
FORMATS = [("f32", 64, 4, 2, 6), ("f32", 128, 2, 1, 6), ("bf16", 64, 4, 2, 6), ("bf16", 128, 4, 2, 4), ("bf16", 128, 16, 8, 8),
           ("bf16", 64, 24, 3, 6), ("e4m3", 128, 8, 4, 8)]


def context(fmt, L=3, cap=100, prompts=1, pages=0, stream=None, plen=40, probe=0):
    import torch

    cache, d, hq, hkv, m = fmt
    ctx = infs.Context(infs.make_config(
        num_layers=L, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, num_prompts=prompts, slots_per_prompt=m,
        samples_per_prompt=500, max_prompt_len=64, max_suffix_len=cap, num_pages=pages, probe_tokens=probe,
        dtype=infs.F32 if cache == "f32" else infs.BF16, flags=infs.FLAG_KV_FP8 if cache == "e4m3" else 0),
        stream=stream or torch.cuda.current_stream())
    k = rows(fmt, plen, 1, seed=99)[0][0]
    for p in range(prompts):
        for layer in range(L):
            ctx.prefill_shared(p, layer, plen, k, k)
    ctx.keep = k
    return ctx


def rows(fmt, n, L, seed, scale=1.0):
    """K and V [L, n, Hkv, d] on the device."""
    import torch

    cache, d, _, hkv, _ = fmt
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if cache == "f32" else torch.bfloat16
    return [(torch.randn(L, n, hkv, d, generator=g) * scale).to(dt).cuda() for _ in range(2)]


def stored(fmt, x):
    """float64 values of rows as the cache holds them."""
    y = x.double().cpu().numpy()
    return round_e4m3(y) if fmt[0] == "e4m3" else y


def read(ctx, fmt, slot, L):
    """What the pages hold, float64 [L, n, Hkv, d] K and V, by the host read-back."""
    import torch

    out = []
    for layer in range(L):
        kv = ctx.read_response(slot, layer)
        if fmt[0] == "e4m3":
            kv = [torch.from_numpy(x).view(torch.float8_e4m3fn).double().numpy() for x in kv]
        elif fmt[0] == "bf16":
            kv = [torch.from_numpy(x.view(np.int16)).view(torch.bfloat16).double().numpy() for x in kv]
        out.append(kv)
    return [np.stack([x[i] for x in out]).astype(np.float64) for i in range(2)]


def export(ctx, fmt, slots, L, stride=0):
    """Hand out; buffers are one token longer than the response, filled with 5 first."""
    import torch

    cache, d, _, hkv, _ = fmt
    dt = torch.float32 if cache == "f32" else torch.bfloat16
    lens = [ctx.slot_state(s)[1] for s in slots]
    per = [max(n, stride) for n in lens]
    bufs = [[torch.full((L * p + 1, hkv, d), 5.0, dtype=dt, device="cuda") for p in per] for _ in range(2)]
    ctx.export_responses(slots, *bufs, layer_stride=stride * hkv * d * bufs[0][0].element_size() if slots else 0)
    out = []
    for b in bufs:
        for x, n, p in zip(b, lens, per):
            assert bool((x[L * p:] == 5).all()) and bool((x[:L * p].view(L, p, hkv, d)[:, n:] == 5).all())
    for i in range(len(slots)):
        out.append([b[i][:L * per[i]].view(L, per[i], hkv, d)[:, :lens[i]].double().cpu().numpy() for b in bufs])
    return out


@pytest.mark.parametrize("fmt", FORMATS, ids=str)
def test_import_and_export_round_trip(fmt):
    L, lens = 3, [0, 1, 15, 16, 17, 100][:fmt[4]]
    ctx = context(fmt)
    kv = [rows(fmt, n, L, 10 + i, scale=4.0) for i, n in enumerate(lens)]
    slots = list(range(len(lens)))
    ctx.import_responses(slots, [3 * i for i in slots], lens, [k for k, _ in kv], [v for _, v in kv])
    got = export(ctx, fmt, slots, L)
    for s in slots:
        assert ctx.slot_state(s) == (3 * s, lens[s])
        for x, y, z in zip(kv[s], got[s], read(ctx, fmt, s, L)):
            assert np.array_equal(stored(fmt, x), y) and np.array_equal(y, z)
    # some slots, in another order and one of them twice, with a layer stride
    order = slots[::-1] + slots[-1:]
    for s, pair in zip(order, export(ctx, fmt, order, L, stride=120)):
        for x, y in zip(kv[s], pair):
            assert np.array_equal(stored(fmt, x), y)
    export(ctx, fmt, [], L)
    ctx.destroy()


@pytest.mark.parametrize("fmt", [FORMATS[0], FORMATS[4], FORMATS[6]], ids=str)
def test_import_with_a_layer_stride_and_scattered_pages(fmt):
    # a pool whose free pages lie apart: responses of many runs of one page
    import torch

    L, m, cap = 2, fmt[4], 640
    ctx = context(fmt, L=L, cap=cap, pages=m * cap // 16)
    one = rows(fmt, 16, L, 5)
    for i in range(3):
        ctx.import_responses([i], [i], [16 * (i + 1)], [torch.cat([one[0]] * (i + 1), 1)], [torch.cat([one[1]] * (i + 1), 1)])
    ctx.retire_slot(1)
    ctx.import_responses([1], [50], [0], [one[0]], [one[1]])
    # slots 0 and 1 grow by turns, one page each: their pages interleave
    q = torch.zeros(L, m, fmt[2], fmt[1], dtype=one[0].dtype, device="cuda")
    nk, nv = rows(fmt, m, L, 6)
    o = torch.empty(L, m, fmt[2], fmt[1], device="cuda")
    for _ in range(100):
        for layer in range(L):
            ctx.decode_step(layer, q[layer], nk[layer], nv[layer], o[layer])
        ctx.end_step()
    ctx.retire_slot(0)
    ctx.retire_slot(2)
    n, stride = 500, 512
    k, v = rows(fmt, stride, L, 7)
    hkv, d = fmt[3], fmt[1]
    ctx.import_responses([0], [60], [n], [k], [v], layer_stride=stride * hkv * d * k.element_size())
    for x, y in zip((k, v), export(ctx, fmt, [0], L)[0]):
        assert np.array_equal(stored(fmt, x[:, :n]), y)
    assert ctx.slot_state(1)[1] == 100
    for x, y in zip((nk, nv), export(ctx, fmt, [1], L)[0]):
        assert np.array_equal(np.repeat(stored(fmt, x[:, 1:2]), 100, axis=1), y)
    ctx.destroy()


def decode(ctx, fmt, L, seed, entry, steps=1):
    """Decode steps with the same rows for the same seed; O of every step."""
    import torch

    S = ctx.config.num_prompts * fmt[4]
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if fmt[0] == "f32" else torch.bfloat16
    out = []
    for _ in range(steps):
        q = torch.randn(L, S, fmt[2], fmt[1], generator=g).to(dt).cuda()
        k, v = (torch.randn(L, S, fmt[3], fmt[1], generator=g).to(dt).cuda() for _ in range(2))
        o = torch.full((L, S, fmt[2], fmt[1]), 3.0, device="cuda")
        if entry == "layers":
            ctx.decode_step_layers(q, k, v, o)
        else:
            for layer in range(L):
                ctx.decode_step(layer, q[layer], k[layer], v[layer], o[layer])
        ctx.end_step()
        torch.cuda.synchronize()
        out.append(o)
    return out


@pytest.mark.parametrize("entry", ["layer", "layers"])
@pytest.mark.parametrize("fmt", FORMATS, ids=str)
def test_branches_go_on_like_responses_of_their_own(fmt, entry):
    # context A forks and decodes; context B holds the same tokens in pages of its own
    import torch

    L, m = 2, fmt[4]
    a, b = context(fmt, L=L), context(fmt, L=L)
    n0 = 37
    k, v = rows(fmt, n0, L, 21)
    a.import_responses([0], [0], [n0], [k], [v])
    lens = [37, 32, 16, 5, 0, 33, 17][:m - 1]
    dst = list(range(1, m))[:len(lens)]
    a.fork_slots([0] * len(dst), dst, [10 + i for i in dst], lens)
    parts = [(k[:, :n].contiguous(), v[:, :n].contiguous()) for n in [n0] + lens]
    b.import_responses([0] + dst, [0] + [10 + i for i in dst], [n0] + lens, [x for x, _ in parts], [x for _, x in parts])
    for x, y in zip(decode(a, fmt, L, 1, entry, 20), decode(b, fmt, L, 1, entry, 20)):
        assert torch.equal(x, y)
    # a branch of a branch; the parent gives up its slot, the branches keep the shared pages
    a.retire_slot(0)
    a.fork_slots([1], [0], [40], [50])
    b.retire_slot(0)
    kv = export(b, fmt, [1], L)[0]
    dt = torch.float32 if fmt[0] == "f32" else torch.bfloat16
    b.import_responses([0], [40], [50], *[[torch.from_numpy(x[:, :50].copy()).to(dt).cuda()] for x in kv])
    for x, y in zip(decode(a, fmt, L, 2, entry, 18), decode(b, fmt, L, 2, entry, 18)):
        assert torch.equal(x, y)
    for s in [0] + dst:
        assert a.slot_state(s) == b.slot_state(s)
        for x, y in zip(read(a, fmt, s, L), read(b, fmt, s, L)):
            assert np.array_equal(x, y)
    # retired branches' pages are recycled without touching what others share
    keep = [read(a, fmt, s, L) for s in dst[1:]]
    a.retire_slot(1)
    a.retire_slot(0)
    zk, zv = rows(fmt, 90, L, 30)
    a.import_responses([0, 1], [60, 61], [90, 90], [zk, zk], [zv, zv])
    for s, old in zip(dst[1:], keep):
        for x, y in zip(read(a, fmt, s, L), old):
            assert np.array_equal(x, y)
    a.sync()
    b.sync()
    a.destroy()
    b.destroy()


@pytest.mark.parametrize("fmt", [FORMATS[0], FORMATS[4], FORMATS[6]], ids=str)
def test_import_equals_growth_token_by_token(fmt):
    import torch

    L, m, n = 2, fmt[4], 35
    grown, taken = context(fmt, L=L), context(fmt, L=L)
    for s in range(m):
        grown.refill_slot(s, 0, s)
    decode(grown, fmt, L, 5, "layer", n)
    kv = export(grown, fmt, list(range(m)), L)
    dt = torch.float32 if fmt[0] == "f32" else torch.bfloat16
    dev = [[torch.from_numpy(x[i]).to(dt).cuda() for x in kv] for i in range(2)]
    taken.import_responses(list(range(m)), list(range(m)), [n] * m, *dev)
    for x, y in zip(decode(grown, fmt, L, 6, "layer", 15), decode(taken, fmt, L, 6, "layer", 15)):
        assert torch.equal(x, y)
    assert list(taken.sample_tokens(0)[:m]) == [15] * m and list(grown.sample_tokens(0)[:m]) == [50] * m
    grown.destroy()
    taken.destroy()


@pytest.mark.parametrize("fmt", [FORMATS[0], FORMATS[4], FORMATS[6]], ids=str)
def test_stale_pages_do_not_leak(fmt):
    # pages that held infinities and NaN are taken again: a part of a page's other tokens weigh nothing
    import torch

    L, m = 2, fmt[4]
    ctx, clean = context(fmt, L=L), context(fmt, L=L)
    k, v = rows(fmt, 100, L, 3)
    bad = [torch.full_like(k, float("nan")), torch.full_like(v, float("inf"))]
    if fmt[0] == "e4m3":  # a stored NaN is out of reach: the largest values
        bad = [torch.full_like(k, 448.0), torch.full_like(v, -448.0)]
    every = list(range(m))
    ctx.import_responses(every, every, [100] * m, [bad[0]] * m, [bad[1]] * m)
    for s in every:
        ctx.retire_slot(s)
    lens = [(7 * s) % 40 for s in every]
    parts = [(k[:, :n].contiguous(), v[:, :n].contiguous()) for n in lens]
    for c, base in ((ctx, 100), (clean, 0)):
        c.import_responses(every, [base + s for s in every], lens, [x for x, _ in parts], [x for _, x in parts])
    for entry in ("layer", "layers"):
        for x, y in zip(decode(ctx, fmt, L, 8, entry, 3), decode(clean, fmt, L, 8, entry, 3)):
            assert torch.equal(x, y) and bool(torch.isfinite(x).all())
    ctx.destroy()
    clean.destroy()


def test_e4m3_saturates_and_rounds_as_the_append():
    import torch

    fmt = FORMATS[6]
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    vals = bits.view(torch.bfloat16)
    vals = vals[torch.isfinite(vals.float())]
    per = fmt[3] * fmt[1]
    n = -(-vals.numel() // per)
    x = vals.repeat(2)[:n * per].view(1, n, fmt[3], fmt[1]).cuda()
    ctx = context(fmt, L=1, cap=n)
    ctx.import_responses([2], [2], [n], [x], [x.flip(1).contiguous()])
    k, v = export(ctx, fmt, [2], 1)[0]
    assert np.array_equal(k, stored(fmt, x)) and np.array_equal(v, stored(fmt, x.flip(1)))
    ctx.destroy()


def test_two_contexts_and_another_stream():
    # a response goes from a context on one stream to one on another, ordered by events
    import torch

    fmt, L, n = FORMATS[4], 2, 77
    side = torch.cuda.Stream()
    a, b = context(fmt, L=L), context(fmt, L=L, stream=side)
    k, v = rows(fmt, n, L, 4)
    bk, bv = torch.empty_like(k), torch.empty_like(v)
    torch.cuda.synchronize()
    a.import_responses([0], [0], [n], [k], [v])
    a.export_responses([0], [bk], [bv])
    side.wait_stream(torch.cuda.current_stream())
    b.import_responses([3], [9], [n], [bk], [bv])
    b.sync()
    for x, y in zip((k, v), read(b, fmt, 3, L)):
        assert np.array_equal(stored(fmt, x), y)
    a.destroy()
    b.destroy()


def test_import_into_hundreds_of_runs():
    # two responses grow by turns, one goes: every second page is free, each a run of its own, more than
    # one launch names
    import torch

    fmt, L, n = ("f32", 64, 1, 1, 4), 1, 16 * 330
    ctx = context(fmt, L=L, cap=n, pages=2 * 330 + 40)
    ctx.refill_slot(0, 0, 0)
    ctx.refill_slot(1, 0, 1)
    q = torch.zeros(4, 1, 64, device="cuda")
    k, v = rows(fmt, 4, L, 6)
    o = torch.empty(4, 1, 64, device="cuda")
    for _ in range(n):
        ctx.decode_step(0, q, k[0], v[0], o)
        ctx.end_step()
    ctx.retire_slot(0)
    nk, nv = rows(fmt, n, L, 7)
    part = 16 * 120 + 5  # more runs than a launch carries along
    ctx.import_responses([2, 3], [5, 6], [part, n - part], [nk[:, :part].contiguous(), nk[:, part:].contiguous()],
                         [nv[:, :part].contiguous(), nv[:, part:].contiguous()])
    got = export(ctx, fmt, [2, 3, 1], L)
    for x, i in ((nk, 0), (nv, 1)):
        assert np.array_equal(np.concatenate([got[0][i], got[1][i]], 1), x.double().cpu().numpy())
    assert np.array_equal(got[2][0], np.repeat(k[:, 1:2].double().cpu().numpy(), n, axis=1))
    ctx.sync()
    ctx.destroy()


def test_pages_beyond_32_bit_offsets():
    # 43 responses of 32000 tokens in a layer's pool of 5.6 GB: the last ones' pages lie beyond 4 GiB
    import torch

    fmt, n, m = ("bf16", 128, 16, 8, 48), 32000, 43
    ctx = context(fmt, L=1, cap=n, pages=m * 2000 + 8)
    g = torch.Generator(device="cuda").manual_seed(8)
    k, v = (torch.randint(-30000, 30000, (n, 8, 128), dtype=torch.int16, device="cuda", generator=g) for _ in range(2))
    slots = list(range(m))
    for i in slots:
        ctx.import_responses([i], [i], [n], [k if i % 2 else v], [v if i % 2 else k])
    last = m - 1
    ctx.retire_slot(0)
    ctx.fork_slots([last, last], [m, m + 1], [m, m + 1], [n, n - 11])
    bk, bv = torch.zeros_like(k), torch.zeros_like(v)
    for slot, t in ((1, n), (last - 1, n), (last, n), (m, n), (m + 1, n - 11)):
        bk.zero_(), bv.zero_()
        ctx.export_responses([slot], [bk], [bv])
        odd = slot % 2 if slot < m else last % 2
        for x, y in ((k if odd else v, bk), (v if odd else k, bv)):
            assert torch.equal(x[:t], y[:t]) and not bool(y[t:].any()), slot
    ctx.sync()
    ctx.destroy()
