"""Norms of heads with the rotation, host side: every refusal (no GPU needed: a refused call enqueues nothing,
dry-run contexts)."""

import math

import pytest

from paper_2506_22950_amd import infs
from paper_2506_22950_amd.group import context_for
from tests.test_rotary import config
from workload import get_config

AT = 0x10000  # an address that no refused call reads


def status(call, *a, **kw):
    try:
        call(*a, **kw)
        return infs.OK
    except infs.InfsError as e:
        assert not str(e).endswith("no error")
        return e.status


def rows(**over):
    kw = dict(x=AT, out=AT, heads=2)
    kw.update(over)
    return infs.rotary_rows(kw.pop("x"), kw.pop("out"), kw.pop("heads"), **kw)


BAD_NORMS = [{"dtype": 2}, {"dtype": -1}, {"eps": -1e-6}, {"eps": math.nan}, {"eps": math.inf}, {"layer_stride": -1},
             {"layer_stride": (1 << 40) + 1}, {"weight_q": AT + 1}, {"weight_k": AT + 1},
             {"weight_q": AT + 2, "dtype": infs.F32}]


@pytest.mark.parametrize("over", BAD_NORMS)
def test_norms(over):
    r = infs.Rotary(config())
    n = infs.make_norms(**{**dict(weight_q=AT, weight_k=AT), **over})
    assert status(r.norm_rotate_rows, infs.BF16, 5, n, rows(), rows()) == infs.E_ARG
    assert status(r.norm_rotate_rows, infs.BF16, 0, n, rows(), rows()) == infs.E_ARG
    assert status(r.norm_rotate_grad, infs.BF16, 5, n, rows(), None, rows(), None) == infs.E_ARG
    ctx = context_for(get_config("tiny_f32"), dry_run=True)
    assert status(ctx.norm_rotate_step, r, n, rows(heads=4), rows(heads=2)) == infs.E_ARG


def test_null_norms_and_rows():
    r = infs.Rotary(config())
    n = infs.make_norms(AT, AT)
    assert status(r.norm_rotate_rows, infs.BF16, 5, None, rows(), rows()) == infs.E_ARG
    assert status(r.norm_rotate_rows, infs.BF16, 5, n) == infs.E_ARG
    assert status(r.norm_rotate_rows, infs.BF16, 5, n, rows(x=None)) == infs.E_ARG
    assert status(r.norm_rotate_rows, infs.BF16, 5, n, rows(out=None)) == infs.E_ARG
    assert status(r.norm_rotate_rows, infs.BF16, 0, n, rows(x=None, out=None)) == infs.OK
    assert status(r.norm_rotate_rows, infs.BF16, 0, infs.make_norms(None, None), rows()) == infs.OK


@pytest.mark.parametrize("kw", [
    {"dtype": 2}, {"tokens": -1}, {"tokens": 1 << 31}, {"first_position": (1 << 31) - 4}, {"positions": AT + 2},
    {"q": {"heads": 0}}, {"q": {"heads": 4097}}, {"q": {"in_strides": (-1, 0, 0)}}, {"q": {"x": AT + 1, "out": AT + 1}},
    {"q": {"in_strides": (63, 0, 0), "out_strides": (63, 0, 0)}}, {"q": {"in_strides": (256, 0, 0)}}])
def test_rows(kw):
    r = infs.Rotary(config())
    n = infs.make_norms(AT, AT)
    kw = dict(kw)
    dtype, tokens, q = kw.pop("dtype", infs.BF16), kw.pop("tokens", 5), rows(**kw.pop("q", {}))
    assert status(r.norm_rotate_rows, dtype, tokens, n, q, None, **kw) == infs.E_ARG


def test_grad():
    r = infs.Rotary(config())
    n = infs.make_norms(AT, AT)
    ok = dict(q=rows(out=AT + 64), k=None, dq=rows(x=AT + 128, out=None), dk=None)

    def call(tokens=5, **over):
        return status(r.norm_rotate_grad, infs.BF16, tokens, n, **{**ok, **over})

    assert call(q=None) == infs.E_ARG
    assert call(dq=None) == infs.E_ARG
    assert call(k=rows()) == infs.E_ARG
    assert call(dk=rows()) == infs.E_ARG
    assert call(q=None, dq=None) == infs.E_ARG
    assert call(dq=rows(heads=3)) == infs.E_ARG
    assert call(dq=rows(x=None)) == infs.E_ARG
    assert call(dq=rows(x=AT + 129)) == infs.E_ARG
    assert call(dq=rows(in_strides=(-128, 0, 0))) == infs.E_ARG
    # written over the gradients of the outputs: their strides have to agree
    assert call(q=rows(out=AT + 128), dq=rows(x=AT + 128, in_strides=(256, 0, 0))) == infs.E_ARG
    assert call(d_weight_q=AT) == infs.E_ARG  # no workspace
    assert call(d_weight_k=AT, workspace=AT) == infs.E_ARG  # no rows
    assert call(d_weight_q=AT + 2, workspace=AT) == infs.E_ARG
    assert call(d_weight_q=AT, workspace=AT + 8) == infs.E_ARG
    assert infs.norm_rotate_grad_workspace(0, 128) == 0
    assert infs.norm_rotate_grad_workspace(3, 128) == 2 * 3 * 128 * 4
    assert infs.norm_rotate_grad_workspace(1 << 30, 128) == infs.norm_rotate_grad_workspace(4096, 128)


def test_steps_of_a_context():
    cfg = get_config("tiny_f32")
    ctx = context_for(cfg, dry_run=True, probe_tokens=4)
    r, n = infs.Rotary(config()), infs.make_norms(None, None, dtype=infs.F32)
    q, k = rows(heads=4), rows(heads=2)
    assert status(ctx.norm_rotate_step, r, n, q, k) == infs.OK  # no slot is live
    assert status(ctx.norm_rotate_step, r, None, q, k) == infs.E_ARG
    assert status(ctx.norm_rotate_step, r, n, k, q) == infs.E_ARG
    assert status(ctx.norm_rotate_step, r, n) == infs.E_ARG
    assert status(ctx.norm_rotate_step, r, n, q, k, num_layers=2) == infs.E_ARG
    assert status(ctx.norm_rotate_step, infs.Rotary(config(head_dim=128)), n, q, k) == infs.E_ARG
    assert status(ctx.norm_rotate_probe, r, n, 0, 0, 4, None, q, k) == infs.E_STATE  # no prefix
    for layer in range(cfg.layers):
        ctx.prefill_shared(0, layer, 32, None, None)
    assert status(ctx.norm_rotate_probe, r, n, 0, 0, 4, None, q, k) == infs.OK
    assert status(ctx.norm_rotate_probe, r, n, 0, 0, 99, None, q, k) == infs.E_ARG
    assert status(ctx.norm_rotate_probe, r, n, 1, 0, 4, None, q, k) == infs.E_ARG
    assert status(ctx.norm_rotate_probe, r, None, 0, 0, 4, None, q, k) == infs.E_ARG
    plain = context_for(cfg, dry_run=True)
    assert status(plain.norm_rotate_probe, r, n, 0, 0, 4, None, q, k) == infs.E_STATE
    assert "norms" in (lambda: [status(ctx.norm_rotate_step, r, None, q, k), ctx.last_error])()[1]


def test_layer_norms():
    n = infs.make_norms(1000, None, dtype=infs.BF16, layer_stride=64)
    m = infs.layer_norms(n, 3)
    assert m.weight_q == 1000 + 3 * 64 * 2 and m.weight_k is None
    assert infs.layer_norms(infs.make_norms(1000, 2000, dtype=infs.F32, layer_stride=64), 1).weight_k == 2000 + 256
