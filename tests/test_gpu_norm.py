"""GPU: norms of heads with the rotation, and their gradient, against the formulas in 64 bits.

Tolerances.  A head's sum of squares adds up to 16 products a lane and up to 6 exchanges, all positive: within
(16 + 6 + 2) 2^-24, half of that in 1/n; 1/n, x/n, times w: three roundings, so z is within 16 * 2^-24 of itself.
The rotation adds 8 * 2^-24 (|z_a| + |z_b|) (see test_gpu_rotary.py): within 24 * 2^-24 A (|z_a| + |z_b|), and half
a step of the output's type.  Gradient, with G the magnitude of g as |d_a| + |d_b|: g is within 8 * 2^-24 G,
sum(w g x) within 34 * 2^-24 sum(|w| G |x|), the rest by a few roundings, so d_x is within
64 * 2^-24 (|w| G + |x| sum(|w| G |x|) / (d n^2)) / n; a sum of R terms for d_w within (64 + R) 2^-24 of the sum of
their magnitudes."""

import numpy as np
import pytest

from paper_2506_22950_amd import infs
from paper_2506_22950_amd.group import context_for
from tests.test_gpu_rotary import rotated
from tests.test_rotary import config
from workload import get_config

pytestmark = pytest.mark.gpu

E32, EBF = 2.0 ** -24, 2.0 ** -8
EPS = float(np.float32(1e-5))


def make(shape, bf16, seed, scale=1.0):
    import torch

    x = torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale
    x = x.bfloat16() if bf16 else x
    return x.cuda(), x.double().numpy()


def normed(x, w):
    n = np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
    return x / n * w, n


def check(got, want, mag, bf16):
    got = got.double().cpu().numpy()
    bad = np.abs(got - want) > (mag + np.abs(want) * (EBF if bf16 else E32) + 1e-37) * 1.001
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.nanmax(np.abs(got - want))))


def formula(x, w, pos, freq, amp, layout, rd):
    z, _ = normed(x, w)
    y, mag = rotated(z, pos, freq, amp, layout, rd)
    return y, mag * 24 * E32


def grads(x, w, dy, pos, freq, amp, layout, rd):
    g, mag = rotated(dy, pos, freq, amp, layout, rd, inverse=True)
    n = np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
    d = x.shape[-1]
    dx = (w * g - x * (w * g * x).sum(-1, keepdims=True) / (d * n * n)) / n
    bound = 64 * E32 * (np.abs(w) * mag + np.abs(x) * (np.abs(w) * mag * np.abs(x)).sum(-1, keepdims=True) / (d * n * n)) / n
    terms = int(np.prod(x.shape[:-1]))
    return dx, bound, (g * x / n).reshape(-1, d).sum(0), (64 + terms) * E32 * (mag * np.abs(x) / n).reshape(-1, d).sum(0)


CASES = [
    # tokens, q heads, kv heads, head_dim, rotary_dim, layout, bf16, weights fp32
    (1, 1, 1, 64, 64, infs.ROTARY_HALF, True, False),
    (1, 16, 8, 128, 128, infs.ROTARY_HALF, True, True),
    (5, 4, 2, 64, 64, infs.ROTARY_INTERLEAVED, False, True),
    (37, 6, 3, 128, 64, infs.ROTARY_HALF, True, False),
    (37, 6, 3, 128, 116, infs.ROTARY_HALF, True, False),    # pairs that 16 bytes do not divide
    (37, 6, 3, 128, 96, infs.ROTARY_INTERLEAVED, True, True),
    (130, 32, 4, 64, 48, infs.ROTARY_INTERLEAVED, False, False),
    (130, 2, 2, 64, 6, infs.ROTARY_HALF, False, True),
    (33, 3, 1, 80, 80, infs.ROTARY_HALF, False, True),
    (33, 3, 1, 96, 32, infs.ROTARY_HALF, True, False),
    (33, 3, 1, 100, 50, infs.ROTARY_HALF, True, True),      # rows off 16 bytes
    (9, 5, 5, 7, 2, infs.ROTARY_INTERLEAVED, True, False),  # odd head size
    (9, 5, 5, 7, 6, infs.ROTARY_HALF, False, True),
    (9, 3, 2, 2, 2, infs.ROTARY_HALF, True, False),
    (300, 2, 1, 256, 256, infs.ROTARY_HALF, True, True),
    (300, 2, 1, 256, 256, infs.ROTARY_INTERLEAVED, False, False),
    (5, 300, 7, 64, 64, infs.ROTARY_HALF, True, False),     # more heads than a work-group holds
    (3000, 8, 2, 128, 128, infs.ROTARY_HALF, False, True),
    (3001, 8, 2, 64, 32, infs.ROTARY_INTERLEAVED, True, True),
    (5000, 1, 1, 16, 2, infs.ROTARY_HALF, False, False),
]


@pytest.mark.parametrize("T,hq,hk,d,rd,layout,bf16,w32", CASES)
def test_rows_and_gradient(T, hq, hk, d, rd, layout, bf16, w32):
    import torch

    r = infs.Rotary(config(head_dim=d, rotary_dim=rd, layout=layout, scaling=infs.ROTARY_YARN, factor=4.0))
    f, amp = r.frequencies()
    q, qn = make((T, hq, d), bf16, 1, 3.0)
    k, kn = make((T, hk, d), bf16, 2)
    wq, wqn = make((d,), bf16 and not w32, 3)
    wk, wkn = make((d,), bf16 and not w32, 4)
    dq, dqn = make((T, hq, d), bf16, 5)
    dk, dkn = make((T, hk, d), bf16, 6)
    pos = torch.randint(-1000, 100000, (T,), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    dt = infs.BF16 if bf16 else infs.F32
    norms = infs.make_norms(wq, wk, infs.BF16 if bf16 and not w32 else infs.F32, EPS)
    qo, ko = torch.full_like(q, 7), torch.full_like(k, 7)
    args = dict(positions=pos.cuda(), stream=torch.cuda.current_stream())
    r.norm_rotate_rows(dt, T, norms, infs.rotary_rows(q, qo, hq), infs.rotary_rows(k, ko, hk), **args)
    for got, x, w in ((qo, qn, wqn), (ko, kn, wkn)):
        want, mag = formula(x, w, pos.numpy(), f, amp, layout, rd)
        check(got, want, mag, bf16)
    ws = torch.empty(infs.norm_rotate_grad_workspace(T, d), dtype=torch.uint8, device="cuda")
    dwq, dwk = torch.full((d,), 9.0, device="cuda"), torch.full((d,), 9.0, device="cuda")
    for _ in range(2):  # the same bits again
        r.norm_rotate_grad(dt, T, norms, infs.rotary_rows(q, qo, hq), infs.rotary_rows(k, ko, hk), infs.rotary_rows(dq, None, hq),
                           infs.rotary_rows(dk, None, hk), dwq, dwk, ws, **args)
        first = dwq.clone() if _ == 0 else first
    assert torch.equal(first, dwq)
    for got, gw, x, w, dy in ((qo, dwq, qn, wqn, dqn), (ko, dwk, kn, wkn, dkn)):
        dx, mag, dw, wmag = grads(x, w, dy, pos.numpy(), f, amp, layout, rd)
        check(got, dx, mag, bf16)
        check(gw, dw, wmag, False)
    # over the gradients of the outputs, one tensor alone, no weights' gradient
    over = dk.clone()
    r.norm_rotate_grad(dt, T, norms, None, infs.rotary_rows(k, over, hk), None, infs.rotary_rows(over, None, hk), **args)
    assert torch.equal(over, ko)
    # in place
    over = q.clone()
    qo.zero_()
    r.norm_rotate_rows(dt, T, norms, infs.rotary_rows(q, qo, hq), **args)
    r.norm_rotate_rows(dt, T, norms, infs.rotary_rows(over, over, hq), **args)
    assert torch.equal(over, qo)
    over = q.clone()
    r.norm_rotate_grad(dt, T, norms, infs.rotary_rows(over, over, hq), None, infs.rotary_rows(dq, None, hq), None, dwq, None,
                       ws, **args)
    dx, mag, dw, wmag = grads(qn, wqn, dqn, pos.numpy(), f, amp, layout, rd)
    check(over, dx, mag, bf16)
    check(dwq, dw, wmag, False)


def test_strides_and_weights_left_out():
    """Rows out of one fused projection (heads of another buffer between them), outputs heads first, no weights,
    an element's alignment; what lies between stays."""
    import torch

    T, hq, hk, d = 29, 4, 2, 64
    r = infs.Rotary(config(head_dim=d, rotary_dim=d))
    f, amp = r.frequencies()
    for shift in (0, 1):
        x, _ = make((T * (hq + 2 * hk) * d + shift,), True, 1)
        fused = x[shift:].view(T, hq + 2 * hk, d)
        out = torch.full((hq, T + 3, d), 5.0, dtype=torch.bfloat16, device="cuda")
        r.norm_rotate_rows(infs.BF16, T, infs.make_norms(eps=EPS),
                           infs.rotary_rows(fused, out, hq, (fused.stride(0), d, 0), (d, (T + 3) * d, 0)),
                           first_position=11, stream=torch.cuda.current_stream())
        want, mag = formula(fused[:, :hq].double().cpu().numpy(), np.ones(d), np.arange(11, 11 + T), f, amp, infs.ROTARY_HALF, d)
        check(out[:, :T].transpose(0, 1), want, mag, True)
        assert bool((out[:, T:] == 5.0).all())


def test_special_values():
    """Zeros stay zeros, an infinity makes the head's other elements 0 and itself NaN, a NaN is the head's alone."""
    import torch

    d = 64
    r = infs.Rotary(config(head_dim=d, rotary_dim=d))
    x = torch.randn(4, 2, d, generator=torch.Generator().manual_seed(1)).cuda()
    x[0, 0] = 0.0
    x[1, 1, 3] = float("inf")
    x[2, 0, 5] = float("nan")
    y = torch.empty_like(x)
    s = torch.cuda.current_stream()
    r.norm_rotate_rows(infs.F32, 4, infs.make_norms(eps=EPS, dtype=infs.F32), infs.rotary_rows(x, y, 2), stream=s)
    assert bool((y[0, 0] == 0).all())
    nan = torch.isnan(y)
    pair = [3, 3 + d // 2]
    assert bool(nan[1, 1, pair].all()) and int(nan[1, 1].sum()) == 2
    rest = [e for e in range(d) if e not in pair]
    assert bool((y[1, 1, rest] == 0).all())
    assert bool(nan[2, 0].all())
    assert int(nan.sum()) == 2 + d


def test_no_tokens():
    import torch

    d = 64
    r = infs.Rotary(config(head_dim=d, rotary_dim=d))
    dw = torch.full((2, d), 3.0, device="cuda")
    x = torch.empty(1, 2, d, device="cuda")
    ws = torch.empty(64, dtype=torch.uint8, device="cuda")
    r.norm_rotate_grad(infs.F32, 0, infs.make_norms(dtype=infs.F32), infs.rotary_rows(x, x, 2), infs.rotary_rows(x, x, 2),
                       infs.rotary_rows(x, None, 2), infs.rotary_rows(x, None, 2), dw[0], dw[1], ws,
                       stream=torch.cuda.current_stream())
    assert bool((dw == 0).all())


@pytest.mark.parametrize("bf16", [False, True])
def test_running_and_probe_steps(bf16):
    """Rows of live slots at their positions, every layer with its weights; idle rows are left alone."""
    import torch

    d, L = 64, 3
    cfg = get_config("tiny_f32").with_(layers=L, dtype="bf16" if bf16 else "f32")
    ctx = context_for(cfg, stream=torch.cuda.current_stream(), probe_tokens=4)
    dt = torch.bfloat16 if bf16 else torch.float32
    kv = torch.randn(32, 2, d).to(dt).cuda()
    for layer in range(L):
        ctx.prefill_shared(0, layer, 32, kv, kv)
    r = infs.Rotary(config(head_dim=d, rotary_dim=d))
    f, amp = r.frequencies()
    w, wn = make((2, L, d), bf16, 4)
    norms = infs.make_norms(w[0], w[1], infs.BF16 if bf16 else infs.F32, EPS, layer_stride=d)
    o = torch.empty(4, 4, d, device="cuda")
    for step in range(2):  # two probe steps of samples 0, 1 and 3
        live = [True, True, False, True]
        q, qn = make((L, 4, 4, d), bf16, 10 + step)
        k, kn = make((L, 4, 2, d), bf16, 20 + step)
        qo, ko = torch.full_like(q, 5), torch.full_like(k, 5)
        ctx.norm_rotate_probe(r, norms, 0, 0, 4, live, infs.rotary_rows(q, qo, 4), infs.rotary_rows(k, ko, 2), num_layers=L)
        for layer in range(L):
            for got, x, ww in ((qo, qn, wn[0]), (ko, kn, wn[1])):
                want, mag = formula(x[layer], ww[layer], [32 + step] * 4, f, amp, infs.ROTARY_HALF, d)
                for j in range(4):
                    if live[j]:
                        check(got[layer, j], want[j], mag[j], bf16)
                    else:
                        assert bool((got[layer, j] == 5).all())
            ctx.probe_step(layer, 0, 0, 4, live, qo[layer], ko[layer], ko[layer], o)
        ctx.end_probe_step()
    none = torch.zeros(L, 64, 2, d, dtype=dt, device="cuda")
    ctx.import_responses([1, 3], [4, 5], [7, 50], [none] * 2, [none] * 2)
    ctx.refill_slot(0, 0, 0)
    pos = [34, 39, None, 82]
    q, qn = make((L, 4, 4, d), bf16, 30)
    k, kn = make((L, 4, 2, d), bf16, 31)
    qo, ko = torch.full_like(q, 5), torch.full_like(k, 5)
    ctx.norm_rotate_step(r, norms, infs.rotary_rows(q, qo, 4), infs.rotary_rows(k, ko, 2), num_layers=L)
    for layer in range(L):
        for got, x, ww in ((qo, qn, wn[0]), (ko, kn, wn[1])):
            want, mag = formula(x[layer], ww[layer], [p or 0 for p in pos], f, amp, infs.ROTARY_HALF, d)
            for j in range(4):
                if pos[j] is not None:
                    check(got[layer, j], want[j], mag[j], bf16)
                else:
                    assert bool((got[layer, j] == 5).all())
    one, other = torch.full_like(k, 5), infs.layer_norms(norms, 1)
    ctx.norm_rotate_step(r, other, None, infs.rotary_rows(k[1], one[1], 2))  # one layer, K alone
    assert torch.equal(one[1], ko[1])


def test_graph_and_streams():
    """Captured on a stream of its own and replayed with other inputs; eager calls between the replays."""
    import torch

    T, hq, hk, d = 70, 4, 2, 128
    r = infs.Rotary(config(head_dim=d, rotary_dim=d))
    norms_w, _ = make((2, d), True, 1)
    norms = infs.make_norms(norms_w[0], norms_w[1], infs.BF16, EPS)
    q, k, dq, dk = (torch.empty(T, h, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hk, hq, hk))
    out = [torch.empty_like(x) for x in (q, k, q, k)]
    dw = torch.empty(2, d, device="cuda")
    ws = torch.empty(infs.norm_rotate_grad_workspace(T, d), dtype=torch.uint8, device="cuda")

    def call(out, dw, ws, stream):
        r.norm_rotate_rows(infs.BF16, T, norms, infs.rotary_rows(q, out[0], hq), infs.rotary_rows(k, out[1], hk), stream=stream)
        r.norm_rotate_grad(infs.BF16, T, norms, infs.rotary_rows(q, out[2], hq), infs.rotary_rows(k, out[3], hk),
                           infs.rotary_rows(dq, None, hq), infs.rotary_rows(dk, None, hk), dw[0], dw[1], ws, stream=stream)

    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        call(out, dw, ws, side)
    eager, edw, ews = [torch.empty_like(x) for x in out], torch.empty_like(dw), torch.empty_like(ws)
    for i in range(4):
        for j, x in enumerate((q, k, dq, dk)):
            x.copy_(make(tuple(x.shape), True, 100 * i + j)[0])
        g.replay()
        call(eager, edw, ews, torch.cuda.current_stream())
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)
        assert torch.equal(dw, edw)
