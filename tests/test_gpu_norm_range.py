"""GPU: norms of heads, and their gradient, at the ends of the range: heads whose squares leave fp32 on either side, and
heads of zeros without an eps.  Formulas and tolerances of test_gpu_norm.py: a head that is scaled by a power of two has
the same roundings, and elements that become denormal by it stay within 2^-140 of their place (elements below 2^-119 of n)."""

import numpy as np
import pytest

from paper_2506_22950_amd import infs
from tests import test_gpu_norm as plain
from tests.test_gpu_norm import check
from tests.test_rotary import config

pytestmark = pytest.mark.gpu

SCALES = [1.0, 1e19, 3e-20, 1e20, 3e37, 1e-12, 2e-15, 1e-25, 3e-30]


def heads(T, h, d, bf16, seed, scales, zero=True):
    """Heads next to each other of every scale (and of zeros), so that lanes of a wavefront take both ways."""
    import torch

    x = torch.randn(T, h, d, generator=torch.Generator().manual_seed(seed))
    x = x * torch.tensor(scales)[torch.arange(T * h).view(T, h) % len(scales)][..., None]
    if zero:
        x.view(T * h, d)[5::7] = 0.0
    x = x.bfloat16() if bf16 else x
    return x.cuda(), x.double().numpy()


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6, 2.0])
@pytest.mark.parametrize("T,hq,hk,d,rd,layout,bf16", [
    (37, 6, 3, 128, 128, infs.ROTARY_HALF, True), (37, 6, 3, 128, 96, infs.ROTARY_INTERLEAVED, True),
    (33, 3, 1, 100, 50, infs.ROTARY_HALF, True), (40, 4, 2, 64, 64, infs.ROTARY_HALF, False),
    (700, 8, 2, 64, 6, infs.ROTARY_HALF, False), (5, 5, 5, 7, 2, infs.ROTARY_INTERLEAVED, False)])
def test_ends_of_the_range(T, hq, hk, d, rd, layout, bf16, eps, monkeypatch):
    import torch

    eps = float(np.float32(eps))
    monkeypatch.setattr(plain, "EPS", eps)
    r = infs.Rotary(config(head_dim=d, rotary_dim=rd, layout=layout))
    f, amp = r.frequencies()
    q, qn = heads(T, hq, d, bf16, 1, SCALES)
    k, kn = heads(T, hk, d, bf16, 2, SCALES)
    w, wn = plain.make((2, d), bf16, 3)
    # gradients of a size that leaves dx = .. / n within fp32 for the smallest n
    dq, dqn = plain.make((T, hq, d), bf16, 5, 1e-3)
    dk, dkn = plain.make((T, hk, d), bf16, 6, 1e-3)
    dt = infs.BF16 if bf16 else infs.F32
    norms = infs.make_norms(w[0], w[1], dt, eps)
    pos = np.arange(T) + 11
    args = dict(first_position=11, stream=torch.cuda.current_stream())
    qo, ko = torch.full_like(q, 7), torch.full_like(k, 7)
    r.norm_rotate_rows(dt, T, norms, infs.rotary_rows(q, qo, hq), infs.rotary_rows(k, ko, hk), **args)
    for got, x, ww in ((qo, qn, wn[0]), (ko, kn, wn[1])):
        some = (x != 0).any(-1)
        assert bool((got[torch.from_numpy(~some).cuda()] == 0).all()) and (~some).any()
        with np.errstate(invalid="ignore"):
            want, mag = plain.formula(x, ww, pos, f, amp, layout, rd)
        check(got[torch.from_numpy(some).cuda()], want[some], mag[some], bf16)
    ws = torch.empty(infs.norm_rotate_grad_workspace(T, d), dtype=torch.uint8, device="cuda")
    dw = torch.full((2, d), 9.0, device="cuda")
    r.norm_rotate_grad(dt, T, norms, infs.rotary_rows(q, qo, hq), infs.rotary_rows(k, ko, hk), infs.rotary_rows(dq, None, hq),
                       infs.rotary_rows(dk, None, hk), dw[0], dw[1], ws, **args)
    for i, (got, x, dy) in enumerate(((qo, qn, dqn), (ko, kn, dkn))):
        some = (x != 0).any(-1) | (eps > 0)
        if eps == 0:  # no direction to go by: nothing
            assert bool((got[torch.from_numpy(~some).cuda()] == 0).all()) and (~some).any()
        x = np.where(some[..., None], x, 1.0)  # (a head of zeros adds nothing to the weights' gradient)
        dx, mag, _, _ = plain.grads(x, wn[i], dy, pos, f, amp, layout, rd)
        check(got[torch.from_numpy(some).cuda()], dx[some], mag[some], bf16)
        heads_of = [plain.grads(x[:, [h]], wn[i], np.where(some[:, [h], None], dy[:, [h]], 0.0), pos, f, amp, layout, rd)
                    for h in range(x.shape[1])]
        terms = x.shape[0] * x.shape[1]
        check(dw[i], sum(g[2] for g in heads_of), sum(g[3] for g in heads_of) * (64 + terms) / (64 + x.shape[0]), False)


def test_denormal_heads():
    """Heads of fp32 denormals without an eps: what they hold is normed as it is."""
    import torch

    d = 64
    r = infs.Rotary(config(head_dim=d, rotary_dim=d))
    f, amp = r.frequencies()
    x = (torch.randn(9, 2, d, generator=torch.Generator().manual_seed(4)) * 1e-41).cuda()
    y = torch.empty_like(x)
    r.norm_rotate_rows(infs.F32, 9, infs.make_norms(eps=0.0, dtype=infs.F32), infs.rotary_rows(x, y, 2), first_position=3,
                       stream=torch.cuda.current_stream())
    x = x.double().cpu().numpy()
    z = x / np.sqrt((x * x).mean(-1, keepdims=True))
    want, mag = plain.rotated(z, np.arange(9) + 3, f, amp, infs.ROTARY_HALF, d)
    check(y, want, mag * 24 * 2.0 ** -24, False)


def test_infinities_and_nans_without_an_eps():
    """They are the head's own, as with an eps."""
    import torch

    d = 64
    r = infs.Rotary(config(head_dim=d, rotary_dim=d))
    x = torch.randn(4, 2, d, generator=torch.Generator().manual_seed(1)).cuda()
    x[0, 0] = 0.0
    x[1, 1, 3] = float("inf")
    x[2, 0, 5] = float("nan")
    y = torch.empty_like(x)
    r.norm_rotate_rows(infs.F32, 4, infs.make_norms(eps=0.0, dtype=infs.F32), infs.rotary_rows(x, y, 2),
                       stream=torch.cuda.current_stream())
    nan = torch.isnan(y)
    pair = [3, 3 + d // 2]
    assert bool((y[0, 0] == 0).all())
    assert bool(nan[1, 1, pair].all()) and bool(nan[2, 0].all()) and int(nan.sum()) == 2 + d
    assert bool((y[1, 1, [e for e in range(d) if e not in pair]] == 0).all())
