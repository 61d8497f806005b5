"""GPU: pages and prefix rows that held NaN and infinities are used again: what lies behind the end of a
response or of a prompt weighs nothing, in every kind of kernel (helpers of test_gpu_responses.py)."""

import pytest

from tests.test_gpu_responses import context, decode, rows

pytestmark = pytest.mark.gpu

# dtype/cache, head_dim, q heads, kv heads, slots per prompt: 1 to 8 heads per KV head, prefixes over plain
# rows and over MFMA blocks
SHAPES = [("f32", 128, 1, 1, 6), ("f32", 64, 2, 1, 6), ("f32", 128, 4, 1, 4), ("f32", 64, 8, 1, 2),
          ("f32", 128, 8, 2, 1), ("bf16", 64, 2, 2, 6), ("bf16", 128, 4, 4, 6), ("bf16", 64, 8, 2, 2), ("bf16", 128, 8, 1, 1),
          ("bf16", 64, 4, 2, 20), ("bf16", 128, 8, 1, 8), ("bf16", 64, 8, 8, 32), ("bf16", 128, 16, 2, 16), ("e4m3", 128, 4, 4, 16),
          ("e4m3", 128, 8, 1, 8)]


@pytest.mark.parametrize("prompts", [1, 2])
@pytest.mark.parametrize("fmt", SHAPES, ids=str)
def test_values_behind_the_ends(fmt, prompts):
    import torch

    L, m, S = 2, fmt[4], fmt[4] * prompts
    cap, plen = 100, 64
    ctx = context(fmt, L=L, cap=cap, prompts=prompts, plen=plen)
    nan, inf = float("nan"), float("inf")
    k, v = rows(fmt, cap, L, 3)
    pk, pv = rows(fmt, plen, L, 4)
    slots = list(range(S))
    for kv in ((nan, inf), (inf, nan), (-inf, nan)):
        if fmt[0] == "e4m3":  # a stored NaN is out of reach: the largest values
            kv = (448.0, -448.0)
        ctx.reset()
        for p in range(prompts):
            for layer in range(L):
                ctx.prefill_shared(p, layer, plen, torch.full_like(pk[layer], kv[0]), torch.full_like(pv[layer], kv[1]))
        ctx.import_responses(slots, [s % m for s in slots], [cap] * S, [torch.full_like(k, kv[0])] * S,
                             [torch.full_like(v, kv[1])] * S)
        ctx.sync()
        ctx.reset()
        clean = context(fmt, L=L, cap=cap, prompts=prompts, plen=plen)
        clean.reset()
        plens = [37, 1][:prompts]
        lens = [(7 * s) % 40 for s in slots]
        parts = [(k[:, :n].contiguous(), v[:, :n].contiguous()) for n in lens]
        for c in (ctx, clean):
            for p, n in enumerate(plens):
                for layer in range(L):
                    c.prefill_shared(p, layer, n, pk[layer][:n].contiguous(), pv[layer][:n].contiguous())
            c.import_responses(slots, [s % m for s in slots], lens, [x for x, _ in parts], [x for _, x in parts])
        for entry in ("layer", "layers"):
            for x, y in zip(decode(ctx, fmt, L, 8, entry, 18), decode(clean, fmt, L, 8, entry, 18)):
                assert torch.equal(x, y) and bool(torch.isfinite(x).all()), (entry, kv)
        # grown from nothing on the same pages
        for c in (ctx, clean):
            for s in slots[::2]:
                c.retire_slot(s)
                c.refill_slot(s, s // m, m + s % m)
        for entry in ("layers", "layer"):
            for x, y in zip(decode(ctx, fmt, L, 9, entry, 3), decode(clean, fmt, L, 9, entry, 3)):
                assert torch.equal(x, y) and bool(torch.isfinite(x).all()), (entry, kv)
        clean.destroy()
    ctx.destroy()
