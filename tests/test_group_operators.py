"""What the group loops ask of the operators that they are given, and that they run with them (dry run: checks and
state, nothing is launched)."""

import pytest

from paper_2506_22950_amd import infs
from paper_2506_22950_amd.group import decode_group, prefill_prompts, probe_group
from tests.test_rotary import config

L, M, G, V = 2, 3, 6, 50
LENGTHS = [[9, 3, 20, 4, 7, 12], [5, 30, 2, 8, 6, 11]]
NONE = (None, None, None, None)


def context(probe=0, prefill=True):
    ctx = infs.Context(infs.make_config(
        num_layers=L, num_q_heads=4, num_kv_heads=2, head_dim=64, num_prompts=2, slots_per_prompt=M,
        samples_per_prompt=G, max_prompt_len=16, max_suffix_len=64, dtype=infs.F32, flags=infs.FLAG_DRY_RUN,
        probe_tokens=probe))
    for p in range(2 if prefill else 0):
        for layer in range(L):
            ctx.prefill_shared(p, layer, 8, None, None)
    return ctx


def scheds():
    return [infs.Sched(G, M, "fifo") for _ in range(2)]


def test_operators_that_need_another():
    ctx, norms = context(probe=2), infs.make_norms()
    with pytest.raises(ValueError, match="norms go with rotary"):
        probe_group(ctx, LENGTHS, 2, L, lambda *a: NONE, norms=norms)
    with pytest.raises(ValueError, match="norms go with rotary"):
        decode_group(ctx, scheds(), LENGTHS, L, lambda *a: NONE, reuse=2, norms=norms)
    sampler = infs.Sampler(infs.make_sampler_config(vocab=V, dtype=infs.F32, max_rows=2 * M, flags=infs.FLAG_DRY_RUN))
    with pytest.raises(ValueError, match="draws"):
        decode_group(ctx, scheds(), LENGTHS, L, lambda *a: NONE, reuse=2, sampler=sampler)
    with pytest.raises(ValueError, match="draws"):
        decode_group(ctx, scheds(), LENGTHS, L, lambda *a: NONE, reuse=2, draws=lambda step: None)
    # nothing was done
    assert all(ctx.probe_state(p, i) == 0 for p in range(2) for i in range(G))
    ctx.destroy()


def test_prompts_that_do_not_fit_together():
    ctx, rotary, norms = context(prefill=False), infs.Rotary(config()), infs.make_norms()
    attention = infs.Attention(infs.make_attention_config(
        num_q_heads=4, num_kv_heads=2, head_dim=64, dtype=infs.F32, max_tokens=64, flags=infs.FLAG_DRY_RUN))
    asked = []

    def provide(layer):
        asked.append(layer)
        return NONE

    for more, match in ((dict(norms=norms), "norms go with rotary"), (dict(rotary=rotary), "positions"),
                        (dict(rotary=rotary, norms=norms), "positions")):
        with pytest.raises(ValueError, match=match):
            prefill_prompts(ctx, [8, 8], L, provide, attention, None, **more)
    other = infs.Attention(infs.make_attention_config(
        num_q_heads=4, num_kv_heads=2, head_dim=64, dtype=infs.F32, max_tokens=64, flags=infs.FLAG_DRY_RUN), stream=64)
    with pytest.raises(ValueError, match="stream"):
        prefill_prompts(ctx, [8, 8], L, provide, other, None)
    for over in (dict(num_q_heads=8), dict(num_kv_heads=1), dict(head_dim=128), dict(dtype=infs.BF16)):
        c = dict(num_q_heads=4, num_kv_heads=2, head_dim=64, dtype=infs.F32, max_tokens=64, flags=infs.FLAG_DRY_RUN)
        with pytest.raises(ValueError, match="attention"):
            prefill_prompts(ctx, [8, 8], L, provide, infs.Attention(infs.make_attention_config(**{**c, **over})), None)
    with pytest.raises(ValueError, match="prompts"):
        prefill_prompts(ctx, [8, 8, 8], L, provide, attention, None)
    assert not asked
    ctx.destroy()


def attention_for(ctx, max_tokens=64):
    c = ctx.config
    return infs.Attention(infs.make_attention_config(
        num_q_heads=c.num_q_heads, num_kv_heads=c.num_kv_heads, head_dim=c.head_dim, dtype=c.dtype, max_tokens=max_tokens,
        flags=infs.FLAG_DRY_RUN))


def test_prompts_with_a_rotary_of_other_heads():
    """Dense rows of the context's heads, taken for larger ones, would be read and written past their end."""
    ctx, asked = context(prefill=False), []
    for d in (32, 128):
        rotary = infs.Rotary(config(head_dim=d, rotary_dim=d))
        for norms in (None, infs.make_norms(dtype=infs.F32)):
            with pytest.raises(ValueError, match="rotary"):
                prefill_prompts(ctx, [8, 8], L, asked.append, attention_for(ctx), None, rotary, norms, positions=1 << 16)
    assert not asked
    ctx.destroy()


@pytest.mark.parametrize("lens,layers,max_tokens,match", [
    ([8, 17], L, 64, "prompt 1"), ([17], L, 64, "prompt 0"), ([8, -4], L, 64, "prompt 1"), ([16, 16], L, 31, "tokens"),
    ([8, 8], L + 1, 64, "layers")])
def test_prompts_that_no_pass_takes(lens, layers, max_tokens, match):
    """What the context or the attention would refuse later, behind rows that are rotated in place and prompts that are
    stored, is refused before anything is done."""
    ctx, asked = context(prefill=False), []
    with pytest.raises(ValueError, match=match):
        prefill_prompts(ctx, lens, layers, asked.append, attention_for(ctx, max_tokens), None)
    assert not asked
    prefill_prompts(ctx, [16, 0], L, lambda layer: [i << 20 for i in range(1, 5)], attention_for(ctx, 16), None)
    ctx.destroy()


def test_buffers_of_a_layer_live_through_its_calls():
    """provide()'s buffers may be its only references: they are held until the layer's calls are made."""
    import weakref

    class Buffer:
        def __init__(self, at):
            self.at = at

        def data_ptr(self):
            return self.at

    alive = []

    class Spy:
        def __init__(self, ctx):
            self.config, self.stream, self.ctx = ctx.config, ctx.stream, ctx

        def prefill_shared(self, *a):
            alive.append(sum(r() is not None for r in refs))
            self.ctx.prefill_shared(*a)

    refs = []

    def provide(layer):
        b = [Buffer(i << 20) for i in range(1, 5)]
        refs[:] = [weakref.ref(x) for x in b]
        return b

    ctx = context(prefill=False)
    prefill_prompts(Spy(ctx), [8, 3], L, provide, attention_for(ctx), 1 << 16)
    assert alive == [4] * (2 * L)
    ctx.destroy()
