"""The choice of tokens, host side: every refusal (dry-run samplers: no GPU needed)."""

import math

import pytest

from paper_2506_22950_amd import infs
from tests.test_norm import AT, status


def config(**over):
    c = dict(vocab=1000, dtype=infs.BF16, max_rows=16, flags=infs.FLAG_DRY_RUN)
    c.update(over)
    return infs.make_sampler_config(**c)


@pytest.mark.parametrize("over", [{"vocab": 0}, {"vocab": (1 << 24) + 1}, {"dtype": 2}, {"dtype": -1}, {"max_rows": 0},
                                  {"max_rows": (1 << 22) + 1}, {"flags": 2}])
def test_config_refusals(over):
    assert status(infs.Sampler, config(**over)) == infs.E_ARG


def test_config_limits_are_allowed():
    for over in ({"vocab": 1}, {"vocab": 1 << 24}, {"max_rows": 1 << 22}):
        infs.Sampler(config(**over)).destroy()


@pytest.mark.parametrize("kw,ok", [
    ({}, True), ({"rows": 0, "logits": None, "uniform": None, "token": None}, True), ({"logprob": None}, True),
    ({"kept": None}, True), ({"row_stride": 1000}, True), ({"row_stride": 1001}, True), ({"each": AT}, True),
    ({"rows": -1}, False), ({"rows": 17}, False), ({"row_stride": 999}, False), ({"row_stride": -5}, False),
    ({"row_stride": (1 << 40) + 1}, False), ({"logits": AT + 1}, False), ({"uniform": AT + 2}, False),
    ({"token": AT + 1}, False), ({"logprob": AT + 2}, False), ({"kept": AT + 3}, False), ({"each": AT + 4}, False)])
def test_refusals(kw, ok):
    s = infs.Sampler(config())
    args = dict(rows=16, logits=AT, uniform=AT, token=AT, logprob=AT, kept=AT)
    args.update(kw)
    assert status(s.sample, **args) == (infs.OK if ok else infs.E_ARG)


@pytest.mark.parametrize("kw,ok", [
    ({}, True), ({"temperature": 2.0 ** -20}, True), ({"temperature": 2.0 ** 20}, True), ({"top_p": 1.0}, True),
    ({"top_p": 1e-300}, True), ({"min_p": 1.0}, True), ({"top_k": (1 << 31) - 1}, True),
    ({"temperature": -1.0}, False), ({"temperature": math.nan}, False), ({"temperature": 2.0 ** -21}, False),
    ({"temperature": 2.0 ** 21}, False), ({"top_p": -0.1}, False), ({"top_p": 1.1}, False), ({"top_p": math.nan}, False),
    ({"min_p": -0.1}, False), ({"min_p": 1.01}, False), ({"min_p": math.nan}, False), ({"top_k": -1}, False)])
def test_sampling(kw, ok):
    s = infs.Sampler(config())
    assert status(s.sample, 1, AT, AT, AT, sampling=infs.make_sampling(**kw)) == (infs.OK if ok else infs.E_ARG)
    # a device array of them is checked row by row where it is read
    assert status(s.sample, 1, AT, AT, AT, sampling=infs.make_sampling(**kw), each=AT) == infs.OK


def test_reserved_and_null():
    import ctypes

    s = infs.Sampler(config())
    p = infs.make_sampling()
    p.reserved = 1
    assert status(s.sample, 1, AT, AT, AT, sampling=p) == infs.E_ARG
    lib = infs.load()
    assert lib.infs_sampler_create(None, None, ctypes.byref(ctypes.c_void_p())) == infs.E_ARG
    assert lib.infs_sampler_create(ctypes.byref(config()), None, None) == infs.E_ARG
    assert lib.infs_choose_tokens(None, 0, None, 0, None, None, None, None, None, None) == infs.E_ARG
    lib.infs_sampler_destroy(None)
