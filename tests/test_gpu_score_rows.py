"""GPU: scores and gradients of rows at the borders of what the calls take: tokens outside the vocabulary in
masked rows, gradients that lie otherwise than the logits, rows as long as a wavefront takes alone, the most
rows and the longest."""

import numpy as np
import pytest

from paper_2506_22950_amd import infs
from tests.test_gpu_score import HALF, U, Ref, close, grad_ref, logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,v", [(8, 1003), (1032, 1003)])  # a work-group a row, a wavefront a row
def test_tokens_outside_the_vocabulary_in_masked_rows(n, v, bf16):
    import torch

    z = torch.full((n, v), -np.inf, device="cuda").to(torch.bfloat16 if bf16 else torch.float32)
    z[1::2] = 1.5
    tok = torch.tensor([v, v, -2, -2, -1, -1, 5, 5] * (n // 8), dtype=torch.int32, device="cuda")
    s = infs.Scorer(infs.make_scorer_config(vocab=v, dtype=infs.BF16 if bf16 else infs.F32, max_rows=n),
                    stream=torch.cuda.current_stream())
    lp, h, st = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
    s.score(n, z, tok, lp, entropy=h, stats=st)
    d = torch.ones(n, device="cuda")
    outside = (tok >= v) | (tok < -1)
    none = torch.arange(n, device="cuda") % 2 == 0
    assert torch.equal(torch.isnan(lp), outside)
    assert bool((lp[tok == -1] == 0).all()) and bool((lp[none & (tok == 5)] == -np.inf).all())
    d[tok == -1] = float("nan")  # a row without a token takes no part of it
    for with_h in (False, True):
        g = torch.full_like(z, 7.0)
        s.grad(n, z, tok, st, d, g, entropy=h if with_h else None, d_entropy=torch.ones_like(h) if with_h else None)
        assert bool(torch.isnan(g[outside]).all()) and bool(torch.isfinite(g[~outside]).all())
        assert bool((g[none & ~outside] == 0).all())
    # without d_logprob the tokens play no part
    g = torch.full_like(z, 7.0)
    s.grad(n, z, tok, st, None, g, entropy=h, d_entropy=torch.ones_like(h))
    assert bool(torch.isfinite(g).all()) and bool((g[none] == 0).all())


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,v,stride,shift,grad_stride,grad_shift", [
    (5, 1001, 1008, 0, 1001, 0), (5, 1000, 1000, 0, 1003, 1), (4, 9001, 9005, 7, 9001, 2), (3, 50257, 50304, 0, 50257, 0),
    (3, 50257, 50257, 0, 50304, 0), (3, 16384, 16384, 0, 16384, 3), (1032, 1001, 1008, 0, 1001, 0), (1032, 999, 999, 0, 1000, 5),
    (2, 1, 1, 0, 3, 1), (3, 5, 8, 0, 5, 1)])
def test_gradient_rows_that_lie_otherwise_than_the_logits(n, v, stride, shift, grad_stride, grad_shift, bf16):
    import torch

    dt = torch.bfloat16 if bf16 else torch.float32
    flat = torch.full((shift + n * stride,), 50.0, dtype=dt, device="cuda")
    z = flat[shift:].view(n, stride)
    z[:, :v] = torch.from_numpy(logits(n, v, 61)).cuda().to(dt)
    tokens = np.random.default_rng(6).integers(-1, v, n)
    tok = torch.from_numpy(tokens.astype(np.int32)).cuda()
    s = infs.Scorer(infs.make_scorer_config(vocab=v, dtype=infs.BF16 if bf16 else infs.F32, max_rows=n),
                    stream=torch.cuda.current_stream())
    lp, h, st = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
    s.score(n, z, tok, lp, entropy=h, stats=st, row_stride=stride)
    ref = Ref(z[:, :v].double().cpu().numpy(), tokens, 1.0)
    g, gh = (torch.randn(n, generator=torch.Generator().manual_seed(i)) for i in (3, 4))
    for with_h in (False, True):
        out = torch.full((grad_shift + n * grad_stride + 8,), 9.0, dtype=dt, device="cuda")
        gt = out[grad_shift:grad_shift + n * grad_stride].view(n, grad_stride)
        s.grad(n, z, tok, st, g.cuda(), gt, entropy=h if with_h else None, d_entropy=gh.cuda() if with_h else None,
               row_stride=stride, grad_row_stride=grad_stride)
        want, err = grad_ref(ref, tokens, 1.0, g.double().numpy(), gh.double().numpy() * with_h)
        close(gt[:, :v], want, err + np.abs(want) * HALF[bf16])
        assert bool((gt[:, v:] == 9).all()) and bool((out[:grad_shift] == 9).all()) and bool((out[-8:] == 9).all())
        # the bits of a gradient that lies as the logits do
        same = torch.full_like(flat, 9.0)
        s.grad(n, z, tok, st, g.cuda(), same[shift:], entropy=h if with_h else None, d_entropy=gh.cuda() if with_h else None,
               row_stride=stride, grad_row_stride=stride)
        assert torch.equal(gt[:, :v], same[shift:].view(n, stride)[:, :v])
    assert torch.equal(z[:, v:], torch.full_like(z[:, v:], 50.0))


@pytest.mark.parametrize("bf16,n,v,top", [(True, 2047, 8192, 2), (True, 2048, 8191, 2), (True, 2048, 8192, 0), (True, 2048, 8192, 32),
                                          (True, 2051, 8193, 3), (False, 2048, 4096, 3), (False, 2050, 4095, 0),
                                          (False, 2048, 4097, 2)])
def test_the_longest_rows_of_a_wavefront(bf16, n, v, top):
    # On both sides of where a wavefront takes a row: from 2048 rows, up to 1024 vectors of 16 bytes.  There a
    # lane adds vocab / 64 terms, not vocab / 256: every bound that counts them widens by the difference.
    import torch

    dt = torch.bfloat16 if bf16 else torch.float32
    z = torch.from_numpy(logits(n, v, 71)).cuda().to(dt)
    tokens = np.random.default_rng(7).integers(-1, v, n)
    tok = torch.from_numpy(tokens.astype(np.int32)).cuda()
    s = infs.Scorer(infs.make_scorer_config(vocab=v, dtype=infs.BF16 if bf16 else infs.F32, max_rows=n, top_k=top),
                    stream=torch.cuda.current_stream())
    lp, h, st = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
    ids, tl = torch.empty(n, max(top, 1), dtype=torch.int32, device="cuda"), torch.empty(n, max(top, 1), device="cuda")
    s.score(n, z, tok, lp, entropy=h, stats=st, top_id=ids if top else None, top_logprob=tl if top else None)
    z64 = z.double().cpu().numpy()
    ref = Ref(z64, tokens, 1.0)
    more = (v / 64 - v / 256) * U
    weight = (ref.p * np.abs(ref.y)).sum(1)
    close(lp, ref.lp_t, ref.lp_err + more)
    close(h, ref.h, ref.h_err + more * (1 + weight))
    assert np.array_equal(st[:, 0].double().cpu().numpy(), ref.m)
    close(st[:, 1], ref.ls, ref.s_err + more + 2 * U * ref.ls)
    if top:
        order = np.argsort(-z64, axis=1, kind="stable")[:, :top]
        assert np.array_equal(ids.cpu().numpy(), order)
        want = np.take_along_axis(ref.lp, order, 1)
        close(tl, want, (ref.s_err + more)[:, None] + 8 * U * (np.abs(want) + 2 * ref.ls[:, None]))


@pytest.mark.parametrize("bf16,n,v,top", [(True, 1 << 23, 3, 2), (False, 1, 1 << 24, 32), (True, 2, 1 << 24, 5)])
def test_the_most_rows_and_the_longest(bf16, n, v, top):
    import torch

    dt = torch.bfloat16 if bf16 else torch.float32
    z = (torch.randn(n, v, generator=torch.Generator(device="cuda").manual_seed(81), device="cuda") * 3).to(dt)
    tokens = np.random.default_rng(8).integers(-1, v, n)
    tok = torch.from_numpy(tokens.astype(np.int32)).cuda()
    s = infs.Scorer(infs.make_scorer_config(vocab=v, dtype=infs.BF16 if bf16 else infs.F32, max_rows=n, top_k=top),
                    stream=torch.cuda.current_stream())
    lp, h, st = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
    ids, tl = torch.empty(n, top, dtype=torch.int32, device="cuda"), torch.empty(n, top, device="cuda")
    s.score(n, z, tok, lp, entropy=h, stats=st, top_id=ids, top_logprob=tl)
    g, out = torch.ones(n, device="cuda"), torch.full_like(z, 9.0)
    s.grad(n, z, tok, st, g, out)
    z64 = z.double().cpu().numpy()
    ref = Ref(z64, tokens, 1.0)
    close(lp, ref.lp_t, ref.lp_err)
    close(h, ref.h, ref.h_err)
    close(st[:, 1], ref.ls, ref.s_err + 2 * U * ref.ls)
    assert np.array_equal(st[:, 0].double().cpu().numpy(), ref.m)
    order = np.argsort(-z64, axis=1, kind="stable")[:, :top]
    assert np.array_equal(ids.cpu().numpy(), order)
    want, err = grad_ref(ref, tokens, 1.0, np.ones(n), np.zeros(n))
    close(out, want, err + np.abs(want) * HALF[bf16])
