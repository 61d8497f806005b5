"""Responses carried over from an earlier iteration together with prefix reuse, on dry-run contexts: what the
group loop refuses before it changes anything, and the steps it then takes."""

import pytest

from paper_2506_22950_amd import infs
from paper_2506_22950_amd.group import decode_group, probe_group

L, M, K = 2, 3, 4
NONE = (None, None, None, None)


def context(probe=K, prompts=2, G=6):
    ctx = infs.Context(infs.make_config(
        num_layers=L, num_q_heads=4, num_kv_heads=2, head_dim=64, num_prompts=prompts, slots_per_prompt=M,
        samples_per_prompt=G, max_prompt_len=16, max_suffix_len=64, dtype=infs.F32, flags=infs.FLAG_DRY_RUN,
        probe_tokens=probe))
    for p in range(prompts):
        for layer in range(L):
            ctx.prefill_shared(p, layer, 8, None, None)
    return ctx


LENGTHS = [[9, 3, 20, 4, 7, 12], [5, 30, 2, 8, 6, 11]]
# of prompt 0 one below, one at, one above the probe tokens; of prompt 1 an empty one and one that is shorter
# than the probe phase
CARRIED = {(0, 0): (3, None, None), (0, 2): (4, None, None), (0, 5): (10, None, None), (1, 1): (0, None, None),
           (1, 2): (1, None, None)}


def state(ctx):
    return [ctx.slot_state(s) for s in range(2 * M)], [[ctx.probe_state(p, i) for i in range(6)] for p in range(2)]


def test_carried_samples_that_were_probed_are_refused_at_once():
    ctx = context()
    probe_group(ctx, LENGTHS, K, L, lambda *a: NONE)
    scheds = [infs.Sched(6, M, "fifo") for _ in range(2)]
    before = state(ctx)
    with pytest.raises(ValueError, match="probed"):
        decode_group(ctx, scheds, LENGTHS, L, lambda *a: NONE, reuse=K, carried=CARRIED)
    assert state(ctx) == before and all(s.pending == 6 for s in scheds)
    # without them the same objects go on
    decode_group(ctx, scheds, LENGTHS, L, lambda *a: NONE, reuse=K)
    ctx.destroy()


@pytest.mark.parametrize("tokens", [9, 10, -1])
def test_finished_carried_samples_are_refused_at_once(tokens):
    ctx = context(probe=0)
    scheds = [infs.Sched(6, M, "fifo") for _ in range(2)]
    before = state(ctx)
    with pytest.raises(ValueError, match="finished"):
        decode_group(ctx, scheds, LENGTHS, L, lambda *a: NONE, carried={(0, 0): (tokens, None, None)})
    assert state(ctx) == before and all(s.pending == 6 for s in scheds)
    ctx.destroy()


@pytest.mark.parametrize("entry", ["probe_step", "probe_step_layers"])
def test_carried_samples_are_left_out_of_the_probe_phase(entry):
    ctx = context()
    plog, log, done = [], [], []
    probe_group(ctx, LENGTHS, K, L, lambda *a: NONE, log=plog, entry=entry, carried=CARRIED)
    probed = {e[:2] for row in plog for e in row if e}
    assert probed == {(p, i) for p in range(2) for i in range(6)} - set(CARRIED)
    for p in range(2):
        for i in range(6):
            # those that finished within their probe tokens were released
            assert ctx.probe_state(p, i) == (0 if (p, i) in CARRIED else min(K, LENGTHS[p][i]))
    decode_group(ctx, [infs.Sched(6, M, "fifo") for _ in range(2)], LENGTHS, L, lambda *a: NONE, reuse=K,
                 carried=CARRIED, log=log, accepted=done)
    for p in range(2):
        for i, length in enumerate(LENGTHS[p]):
            start = CARRIED[p, i][0] if (p, i) in CARRIED else K
            assert [e[2] for row in log for e in row if e and e[:2] == (p, i)] == list(range(start + 1, length + 1)), (p, i)
        # samples that finished within their probe tokens take no slot
        assert sorted(done[p]) == [i for i in range(6) if (p, i) in CARRIED or LENGTHS[p][i] > K]
    ctx.destroy()
