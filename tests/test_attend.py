"""Attention of packed sequences, host side: every refusal (dry-run attentions: no GPU needed)."""

import math

import pytest

from paper_2506_22950_amd import infs
from tests.test_norm import AT, status


def config(**over):
    c = dict(num_q_heads=4, num_kv_heads=2, head_dim=64, dtype=infs.BF16, scale=0.0, max_tokens=100,
             flags=infs.FLAG_DRY_RUN)
    c.update(over)
    return infs.make_attention_config(**c)


@pytest.mark.parametrize("over", [
    {"num_q_heads": 0}, {"num_kv_heads": 0}, {"num_q_heads": 5}, {"num_q_heads": 4098}, {"num_q_heads": -4},
    {"head_dim": 32}, {"head_dim": 96}, {"head_dim": 256}, {"dtype": 2}, {"scale": -1.0}, {"scale": math.nan},
    {"scale": math.inf}, {"max_tokens": 0}, {"max_tokens": -1}, {"max_tokens": 1 << 30}, {"flags": 2}])
def test_config_refusals(over):
    assert status(infs.Attention, config(**over)) == infs.E_ARG


def test_config_limits_are_allowed():
    for over in ({"max_tokens": 1}, {"num_q_heads": 4096}, {"max_tokens": (1 << 30) - 1}, {"scale": 3.0}, {"head_dim": 128}):
        infs.Attention(config(**over)).destroy()


def rows(heads, **over):
    kw = dict(x=AT, out=None)
    kw.update(over)
    return infs.rotary_rows(kw.pop("x"), kw.pop("out"), heads, **kw)


CALLS = [
    ({}, True), ({"sequences": 0}, True), ({"q_tokens": 0}, True), ({"k_tokens": 0, "k_offsets": AT}, True),
    ({"k_tokens": 1 << 25, "k_offsets": AT}, True), ({"sequences": 1 << 20}, True),
    ({"sequences": -1}, False), ({"sequences": (1 << 20) + 1}, False), ({"q_tokens": -1}, False), ({"q_tokens": 101}, False),
    ({"k_tokens": 50}, False), ({"k_tokens": -1, "k_offsets": AT}, False), ({"k_tokens": 1 << 31, "k_offsets": AT}, False),
    ({"k_tokens": 1 << 27, "k_offsets": AT}, False),  # too many work-groups
    ({"q_offsets": AT + 2}, False), ({"k_offsets": AT + 1}, False),
    ({"q": None}, False), ({"k": None}, False), ({"v": None}, False),
    ({"q": rows(2, out=AT + 64)}, False), ({"k": rows(4)}, False), ({"v": rows(1)}, False),
    ({"q": rows(4, out=AT)}, False),  # outputs over the queries
    ({"q": rows(4, x=AT + 8, out=AT + 64)}, False), ({"q": rows(4, out=AT + 72)}, False), ({"k": rows(2, x=AT + 8)}, False),
    ({"v": rows(2, x=AT + 2)}, False), ({"k": rows(2, in_strides=(132, 0, 0))}, False),
    ({"v": rows(2, in_strides=(0, 68, 0))}, False), ({"k": rows(2, in_strides=(-128, 0, 0))}, False),
    ({"k": rows(2, in_strides=(0, 32, 0))}, False), ({"q": rows(4, out=AT + 64, out_strides=(260, 0, 0))}, False),
    ({"lse": AT + 2}, False)]


@pytest.mark.parametrize("kw,ok", CALLS)
def test_attend(kw, ok):
    a = infs.Attention(config())
    args = dict(sequences=3, q_tokens=100, q_offsets=AT, q=rows(4, out=AT + 64), k=rows(2), v=rows(2), lse=AT)
    args.update(kw)
    assert status(a.attend, **args) == (infs.OK if ok else infs.E_ARG)


@pytest.mark.parametrize("kw,ok", CALLS + [
    ({"o": None}, False), ({"d_o": None}, False), ({"o": rows(2)}, False), ({"d_o": rows(4, x=AT + 4)}, False),
    ({"k": rows(2, out=AT)}, False), ({"v": rows(2, out=AT)}, False), ({"k": rows(2, out=AT + 8)}, False)])
def test_grad(kw, ok):
    a = infs.Attention(config())
    args = dict(sequences=3, q_tokens=100, q_offsets=AT, q=rows(4, out=AT + 64), k=rows(2, out=AT + 64),
                v=rows(2, out=AT + 64), o=rows(4), d_o=rows(4), lse=AT)
    args.update(kw)
    assert status(a.grad, **args) == (infs.OK if ok else infs.E_ARG)


def test_null_attention():
    import ctypes

    lib = infs.load()
    assert lib.infs_attention_create(None, None, ctypes.byref(ctypes.c_void_p())) == infs.E_ARG
    assert lib.infs_attention_create(ctypes.byref(config()), None, None) == infs.E_ARG
    assert lib.infs_attend(None, 0, 0, None, 0, None, None, None, None, None) == infs.E_ARG
    assert lib.infs_attend_grad(None, 0, 0, None, 0, None, None, None, None, None, None, None) == infs.E_ARG
    lib.infs_attention_destroy(None)


@pytest.mark.parametrize("scale,ok", [(2.0 ** -64, True), (2.0 ** 64, True), (1e-38, False), (2.0 ** -65, False),
                                      (2.0 ** 65, False), (3e38, False)])
def test_range_of_the_scale(scale, ok):
    c = infs.make_attention_config(num_q_heads=4, num_kv_heads=2, head_dim=64, dtype=infs.BF16, scale=scale, max_tokens=9,
                                   flags=infs.FLAG_DRY_RUN)
    if ok:
        infs.Attention(c).destroy()
    else:
        with pytest.raises(infs.InfsError, match="scale"):
            infs.Attention(c)
