"""GPU: forked, taken-in and handed-out responses of several prompts, and where samples have probe tokens: a
response's row of the page table is then its sample's, not its slot's (helpers and formats of
test_gpu_responses.py)."""

import numpy as np
import pytest

from tests.test_gpu_responses import FORMATS, context, decode, export, read, rows, stored

pytestmark = pytest.mark.gpu

PICKED = [FORMATS[0], FORMATS[4], FORMATS[6]]


def probe_steps(ctx, fmt, L, prompt, n, steps, seed):
    """Probe steps of samples 0 .. n-1 of a prompt, with the same rows for the same seed."""
    import torch

    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if fmt[0] == "f32" else torch.bfloat16
    for _ in range(steps):
        q = torch.randn(L, n, fmt[2], fmt[1], generator=g).to(dt).cuda()
        k, v = (torch.randn(L, n, fmt[3], fmt[1], generator=g).to(dt).cuda() for _ in range(2))
        o = torch.empty(L, n, fmt[2], fmt[1], device="cuda")
        for layer in range(L):
            ctx.probe_step(layer, prompt, 0, n, None, q[layer], k[layer], v[layer], o[layer])
        ctx.end_probe_step()
        torch.cuda.synchronize()


@pytest.mark.parametrize("probe", [0, 4])
@pytest.mark.parametrize("fmt", PICKED, ids=str)
def test_round_trip_over_two_prompts(fmt, probe):
    L, m = 2, fmt[4]
    ctx = context(fmt, L=L, prompts=2, probe=probe)
    lens = [0, 1, 15, 16, 17, 100, 33, 64][:m]
    slots = [s for p in range(2) for s in range(p * m, p * m + len(lens))]
    ids = [7 * (s % m) + 3 for s in slots]  # the same samples of both prompts
    n = lens + lens[::-1]
    kv = [rows(fmt, x, L, 40 + i, scale=3.0) for i, x in enumerate(n)]
    ctx.import_responses(slots, ids, n, [k for k, _ in kv], [v for _, v in kv])
    order = slots[1::2] + slots[::2]
    for s, pair in zip(order, export(ctx, fmt, order, L)):
        i = slots.index(s)
        assert ctx.slot_state(s) == (ids[i], n[i])
        for x, y, z in zip(kv[i], pair, read(ctx, fmt, s, L)):
            assert np.array_equal(stored(fmt, x), y) and np.array_equal(y, z)
    ctx.sync()
    ctx.destroy()


@pytest.mark.parametrize("entry", ["layer", "layers"])
@pytest.mark.parametrize("probe", [0, 4])
@pytest.mark.parametrize("fmt", PICKED, ids=str)
def test_branches_over_two_prompts(fmt, probe, entry):
    # A forks, B grows the same sources and takes the branches' tokens into pages of their own
    import torch

    L, m = 2, fmt[4]
    a, b = context(fmt, L=L, prompts=2, probe=probe), context(fmt, L=L, prompts=2, probe=probe)
    for ctx in (a, b):
        if probe:
            probe_steps(ctx, fmt, L, 0, 3, probe, 1)
            probe_steps(ctx, fmt, L, 1, 3, probe - 1, 2)
        ctx.refill_slot(0, 0, 2)
        ctx.refill_slot(m + 1, 1, 1)
    grown = [decode(ctx, fmt, L, 3, entry, 34) for ctx in (a, b)]
    for x, y in zip(*grown):
        assert torch.equal(x, y)
    # of each source: inside the probe tokens, whole pages, a part of a page, all
    src = [0, 0, 0, m + 1, m + 1]
    dst = [1, 2, 3, m, m + 2]
    ids = [20, 21, 22, 20, 21]
    full = {s: a.slot_state(s)[1] for s in (0, m + 1)}
    assert full == {0: 34 + probe, m + 1: 34 + max(0, probe - 1)}
    lens = [3, 32, full[0], 17, 0]
    a.fork_slots(src, dst, ids, lens)
    kv = dict(zip((0, m + 1), export(b, fmt, [0, m + 1], L)))
    dt = torch.float32 if fmt[0] == "f32" else torch.bfloat16
    parts = [[torch.from_numpy(kv[s][i][:, :n].copy()).to(dt).cuda() for s, n in zip(src, lens)] for i in range(2)]
    b.import_responses(dst, ids, lens, *parts)
    for x, y in zip(decode(a, fmt, L, 4, entry, 19), decode(b, fmt, L, 4, entry, 19)):
        assert torch.equal(x, y)
    # a source goes, a branch branches, a new sample takes the freed slot
    for ctx in (a, b):
        ctx.retire_slot(0)
        ctx.refill_slot(0, 0, 1)
    assert a.slot_state(0) == (1, probe) == b.slot_state(0)
    a.retire_slot(m + 1)
    b.retire_slot(m + 1)
    a.fork_slots([m, m], [m + 1, m + 3], [30, 31], [36, 16])
    k, v = export(b, fmt, [m], L)[0]
    two = [[torch.from_numpy(x[:, :n].copy()).to(dt).cuda() for n in (36, 16)] for x in (k, v)]
    b.import_responses([m + 1, m + 3], [30, 31], [36, 16], *two)
    for x, y in zip(decode(a, fmt, L, 5, entry, 18), decode(b, fmt, L, 5, entry, 18)):
        assert torch.equal(x, y)
    for s in range(2 * m):
        assert a.slot_state(s) == b.slot_state(s)
        if a.slot_state(s)[0] >= 0:
            for x, y in zip(read(a, fmt, s, L), read(b, fmt, s, L)):
                assert np.array_equal(x, y)
    for ctx in (a, b):
        ctx.sync()
        ctx.destroy()


@pytest.mark.parametrize("probe", [0, 4])
def test_many_runs_in_the_second_prompt(probe):
    # more runs of pages than a launch carries along, in page-table rows behind the first prompt's
    import torch

    fmt, L, n = ("f32", 64, 1, 1, 4), 1, 16 * 120
    ctx = context(fmt, L=L, cap=n, pages=2 * 120 + 40, prompts=2, probe=probe)
    a, b = 4, 5
    ctx.refill_slot(a, 1, 0)
    ctx.refill_slot(b, 1, 1)
    q = torch.zeros(8, 1, 64, device="cuda")
    k, v = rows(fmt, 8, L, 6)
    o = torch.empty(8, 1, 64, device="cuda")
    for _ in range(n):
        ctx.decode_step(0, q, k[0], v[0], o)
        ctx.end_step()
    ctx.retire_slot(a)
    nk, nv = rows(fmt, n, L, 7)
    part = 16 * 99 + 5
    ctx.import_responses([6, 7], [77, 499], [part, n - part - 16], [nk[:, :part].contiguous(), nk[:, part:-16].contiguous()],
                         [nv[:, :part].contiguous(), nv[:, part:-16].contiguous()])
    got = export(ctx, fmt, [6, 7, b], L)
    for x, i in ((nk, 0), (nv, 1)):
        assert np.array_equal(np.concatenate([got[0][i], got[1][i]], 1), x[:, :-16].double().cpu().numpy())
    assert np.array_equal(got[2][0], np.repeat(k[:, b:b + 1].double().cpu().numpy(), n, axis=1))
    assert all(ctx.slot_state(s)[0] == -1 for s in range(4))
    ctx.sync()
    ctx.destroy()
