"""Forked, taken-in and handed-out responses, host side: refusals, and the slot and page state against a
reference model on long random call sequences (dry-run contexts, no GPU)."""

import numpy as np
import pytest

from paper_2506_22950_amd import infs

PAGE = 16


def context(m=4, prompts=2, G=64, L=2, cap=64, pages=0, probe=0, **over):
    c = dict(num_layers=L, num_q_heads=4, num_kv_heads=2, head_dim=64, num_prompts=prompts, slots_per_prompt=m,
             samples_per_prompt=G, max_prompt_len=32, max_suffix_len=cap, num_pages=pages, dtype=infs.F32,
             flags=infs.FLAG_DRY_RUN, probe_tokens=probe)
    c.update(over)
    ctx = infs.Context(infs.make_config(**c))
    for p in range(prompts):
        for layer in range(L):
            ctx.prefill_shared(p, layer, 8, None, None)
    return ctx


def status(call, *a, **kw):
    try:
        call(*a, **kw)
        return infs.OK
    except infs.InfsError as e:
        return e.status


def import_(ctx, slots, ids, lens, **kw):
    n = len(slots)
    return status(ctx.import_responses, slots, ids, lens, [None] * n, [None] * n, **kw)


def step(ctx, L=2):
    for layer in range(L):
        ctx.decode_step(layer, None, None, None, None)
    ctx.end_step()


def test_import_refusals():
    ctx = context()
    assert import_(ctx, [], [], []) == infs.OK
    assert import_(ctx, [8], [0], [3]) == infs.E_ARG
    assert import_(ctx, [-1], [0], [3]) == infs.E_ARG
    assert import_(ctx, [0], [64], [3]) == infs.E_ARG
    assert import_(ctx, [0], [-1], [3]) == infs.E_ARG
    assert import_(ctx, [0], [0], [-1]) == infs.E_ARG
    assert import_(ctx, [0, 0], [0, 1], [1, 1]) == infs.E_ARG
    assert import_(ctx, [0, 1], [0, 0], [1, 1]) == infs.E_ARG
    assert import_(ctx, [0], [0], [65]) == infs.E_CAPACITY
    assert import_(ctx, [0], [0], [3], layer_stride=8) == infs.E_ARG
    assert import_(ctx, [0], [0], [3], layer_stride=-16) == infs.E_ARG
    assert import_(ctx, [0], [0], [3], layer_stride=3 * 2 * 64 * 4 - 16) == infs.E_ARG
    assert all(ctx.slot_state(s) == (-1, 0) for s in range(8))
    # the same sample id of two prompts, an empty response, the longest one
    assert import_(ctx, [0, 4, 1], [0, 0, 1], [0, 64, 17], layer_stride=64 * 2 * 64 * 4) == infs.OK
    assert [ctx.slot_state(s) for s in (0, 4, 1)] == [(0, 0), (0, 64), (1, 17)]
    assert import_(ctx, [0], [2], [1]) == infs.E_STATE  # live
    assert import_(ctx, [2], [1], [1]) == infs.E_DUP
    ctx.retire_slot(4)
    ctx.decode_step(0, None, None, None, None)
    assert import_(ctx, [2], [3], [1]) == infs.E_STATE  # step open
    assert import_(ctx, list(range(8)) * 9, list(range(72)), [0] * 72) == infs.E_ARG  # more than 64


def test_fork_refusals():
    ctx = context()
    assert status(ctx.fork_slots, [], [], []) == infs.OK
    assert status(ctx.fork_slots, [0], [1], [1]) == infs.E_STATE  # source empty
    assert import_(ctx, [0, 4], [0, 0], [20, 5]) == infs.OK
    assert status(ctx.fork_slots, [0], [4], [1]) == infs.E_STATE  # destination live
    assert status(ctx.fork_slots, [0], [5], [1]) == infs.E_ARG    # another prompt
    assert status(ctx.fork_slots, [0], [0], [1]) == infs.E_STATE
    assert status(ctx.fork_slots, [0], [1], [0]) == infs.E_DUP
    assert status(ctx.fork_slots, [0], [1], [1], [21]) == infs.E_ARG
    assert status(ctx.fork_slots, [0], [1], [1], [-1]) == infs.E_ARG
    assert status(ctx.fork_slots, [9], [1], [1]) == infs.E_ARG
    assert status(ctx.fork_slots, [0], [9], [1]) == infs.E_ARG
    assert status(ctx.fork_slots, [0, 0], [1, 1], [1, 2]) == infs.E_ARG
    assert status(ctx.fork_slots, [0, 1], [1, 2], [1, 2]) == infs.E_STATE  # a branch is no source in its own call
    assert ctx.slot_state(1) == (-1, 0)
    assert status(ctx.fork_slots, [0, 0, 4], [1, 2, 5], [1, 2, 1], [20, 0, 5]) == infs.OK
    assert [ctx.slot_state(s) for s in (0, 1, 2, 5)] == [(0, 20), (1, 20), (2, 0), (1, 5)]
    ctx.decode_step(0, None, None, None, None)
    assert status(ctx.fork_slots, [0], [3], [3]) == infs.E_STATE  # step open


def test_export_refusals():
    ctx = context()
    assert status(ctx.export_responses, [0], [None], [None]) == infs.E_STATE
    assert status(ctx.export_responses, [8], [None], [None]) == infs.E_ARG
    assert import_(ctx, [0], [0], [20]) == infs.OK
    assert status(ctx.export_responses, [0], [None], [None], layer_stride=20) == infs.E_ARG
    assert status(ctx.export_responses, [0, 0], [None] * 2, [None] * 2) == infs.OK
    ctx.decode_step(0, None, None, None, None)
    assert status(ctx.export_responses, [0], [None], [None]) == infs.E_STATE


def test_probe_contexts():
    ctx = context(probe=3)
    ctx.probe_step(0, 0, 0, 2, [1, 0], None, None, None, None)
    assert import_(ctx, [0], [1], [4]) == infs.E_STATE  # probe step open
    ctx.probe_step(1, 0, 0, 2, [1, 0], None, None, None, None)
    ctx.end_probe_step()
    assert import_(ctx, [0], [0], [4]) == infs.E_STATE  # sample 0 has a probe token
    assert import_(ctx, [0], [1], [40]) == infs.OK
    ctx.refill_slot(1, 0, 0)
    assert ctx.slot_state(1) == (0, 1)
    assert status(ctx.fork_slots, [1, 0], [2, 3], [5, 6]) == infs.OK
    assert ctx.slot_state(2) == (5, 1) and ctx.slot_state(3) == (6, 40)
    ctx.release_sample(0, 7)
    ctx.retire_slot(2)
    assert status(ctx.fork_slots, [0], [2], [7]) == infs.E_DUP
    step(ctx)


def test_shared_pages_return_with_their_last_holder():
    # 6 pages: a response of 40 tokens takes 3 (two full, one part)
    ctx = context(m=4, prompts=1, pages=6)
    assert import_(ctx, [0], [0], [40]) == infs.OK            # 3 free
    assert status(ctx.fork_slots, [0] * 3, [1, 2, 3], [1, 2, 3], [40, 40, 32]) == infs.OK  # two part pages: 1 free
    ctx.retire_slot(0)                                        # its part page alone: 2 free
    assert import_(ctx, [0], [4], [33]) == infs.E_CAPACITY
    assert import_(ctx, [0], [4], [32]) == infs.OK            # 0 free
    assert status(ctx.fork_slots, [1], [2], [9], [40]) == infs.E_STATE
    ctx.retire_slot(0)                                        # 2 free
    ctx.retire_slot(1)                                        # 3 free
    ctx.retire_slot(2)                                        # 4 free; slot 3 still holds the two full pages
    assert import_(ctx, [0], [5], [64]) == infs.OK
    ctx.retire_slot(3)                                        # the last holder: 2 free
    assert import_(ctx, [1], [6], [32]) == infs.OK
    assert import_(ctx, [2], [7], [1]) == infs.E_CAPACITY
    ctx.reset()
    for layer in range(2):
        ctx.prefill_shared(0, layer, 8, None, None)
    assert import_(ctx, [0], [0], [64]) == infs.OK and import_(ctx, [1], [1], [32]) == infs.OK
    assert import_(ctx, [2], [2], [1]) == infs.E_CAPACITY


@pytest.mark.parametrize("seed", range(6))
def test_random_sequences_against_a_model(seed):
    rng = np.random.default_rng(seed)
    m, G, cap, pages = 5, 4000, 80, 10
    ctx = context(m=m, prompts=1, G=G, cap=cap, pages=pages, num_q_heads=2)
    free, refs = pages, {}
    held = [None] * m  # per slot: (sample, len, page objects)
    names = iter(range(1 << 30))
    nxt = 0
    seen = {infs.OK: 0, infs.E_CAPACITY: 0, infs.E_STATE: 0}

    def new():
        x = next(names)
        refs[x] = 1
        return x

    for _ in range(1500):
        op = rng.choice(["import", "fork", "retire", "step", "refill"])
        s = int(rng.integers(m))
        if op == "import":
            n = int(rng.choice([0, 1, 15, 16, 17, 32, 50, cap, int(rng.integers(cap + 1))]))
            need = -(-n // PAGE)
            want = infs.E_STATE if held[s] else infs.E_CAPACITY if need > free else infs.OK
            got = import_(ctx, [s], [nxt], [n])
            if want == infs.OK:
                held[s] = (nxt, n, [new() for _ in range(need)])
                free -= need
        elif op == "fork":
            dst = [int(x) for x in rng.permutation(m)[:rng.integers(1, 4)]]
            src = [int(rng.integers(m)) for _ in dst]
            ids = [nxt + i for i in range(len(dst))]
            lens = [int(rng.integers(0, held[x][1] + 1)) if held[x] else 0 for x in src]
            need = sum(x % PAGE != 0 for x in lens)
            bad = any(held[d] for d in dst) or any(held[x] is None for x in src)
            want = infs.E_STATE if bad else infs.E_CAPACITY if need > free else infs.OK
            got = status(ctx.fork_slots, src, dst, ids, lens)
            if want == infs.OK:
                for x, d, i, n in zip(src, dst, ids, lens):
                    shared = held[x][2][:n // PAGE]
                    for pg in shared:
                        refs[pg] += 1
                    held[d] = (i, n, shared + ([new()] if n % PAGE else []))
                free -= need
                nxt += len(dst)
        elif op == "retire":
            want = infs.OK if held[s] else infs.E_STATE
            got = status(ctx.retire_slot, s)
            if held[s]:
                for pg in held[s][2]:
                    refs[pg] -= 1
                    free += refs[pg] == 0
                held[s] = None
        elif op == "refill":
            want = infs.E_STATE if held[s] else infs.OK
            got = status(ctx.refill_slot, s, 0, nxt)
            if want == infs.OK:
                held[s] = (nxt, 0, [])
        else:
            need = sum(1 for h in held if h and h[1] % PAGE == 0)
            full = any(h and h[1] == cap for h in held)
            want = infs.E_CAPACITY if full or need > free else infs.OK
            got = status(ctx.decode_step, 0, None, None, None, None)
            if want == infs.OK:
                ctx.decode_step(1, None, None, None, None)
                ctx.end_step()
                for i, h in enumerate(held):
                    if h:
                        grown = h[2] + ([new()] if h[1] % PAGE == 0 else [])
                        held[i] = (h[0], h[1] + 1, grown)
                free -= need
        if op in ("import", "refill") and want == infs.OK:
            nxt += 1
        assert got == want, (op, got, want)
        seen[want] += 1
        assert [ctx.slot_state(i) for i in range(m)] == [(h[0], h[1]) if h else (-1, 0) for h in held]
    assert min(seen.values()) > 20, seen
