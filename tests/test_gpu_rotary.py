"""GPU: rotary positions against the rotation of complex numbers in 64 bits.

Tolerance: an output is x_a c - x_b s with c and s off by at most E and three roundings of fp32, then
one rounding to the rows' type.  E: the angle is reduced in double (p f_j and its multiple of pi/2 are
off by 2^-53 of at most 2^31: 2.4e-7 at the far end, 1.2e-10 below 2^20), rounded to fp32 (2^-25 of
pi/4), the sums are short (2^-24 a step on values of at most 1, the last steps dominating: 2 of them).
So with a = |x_a|, b = |x_b|, A the amplitude: |error| <= A (a + b) (8 * 2^-24 + angle error) + half a
step of the output.  Gradients are the rotation by the negative angle: tested against that, and
against differences of the forward rotation."""

import numpy as np
import pytest

from paper_2506_22950_amd import infs
from tests.test_rotary import config

pytestmark = pytest.mark.gpu

F32_EPS, BF16_EPS = 2.0 ** -24, 2.0 ** -8  # half a step


def rotated(x, pos, freq, amp, layout, rd, inverse=False):
    """x [..., T, H, d] float64 -> (rotated, bound on |x_a| + |x_b| of each element's pair)."""
    y, mag = x.copy(), np.abs(x).copy()
    a = np.arange(0, rd, 2) if layout == infs.ROTARY_INTERLEAVED else np.arange(rd // 2)
    b = a + (1 if layout == infs.ROTARY_INTERLEAVED else rd // 2)
    theta = np.asarray(pos, dtype=np.float64)[:, None] * freq * (-1 if inverse else 1)
    turn = amp * np.exp(1j * theta)[:, None, :]
    z = (x[..., a] + 1j * x[..., b]) * turn
    y[..., a], y[..., b] = z.real, z.imag
    mag[..., a] = mag[..., b] = amp * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, mag


def check(got, want, mag, bf16, far=0.0):
    got = got.double().cpu().numpy()
    bound = mag * (8 * F32_EPS + far) + np.abs(want) * (BF16_EPS if bf16 else F32_EPS) + 1e-38
    bad = np.abs(got - want) > bound * 1.001
    assert not bad.any(), (int(bad.sum()), float((np.abs(got - want) / bound).max()))


def make(shape, bf16, seed):
    import torch

    x = torch.randn(*shape, generator=torch.Generator().manual_seed(seed))
    x = x.bfloat16() if bf16 else x
    return x.cuda(), x.double().numpy()


CASES = [
    # tokens, q heads, kv heads, head_dim, rotary_dim, layout, bf16
    (1, 1, 1, 64, 64, infs.ROTARY_HALF, True),
    (1, 16, 8, 128, 128, infs.ROTARY_HALF, True),
    (5, 4, 2, 64, 64, infs.ROTARY_INTERLEAVED, False),
    (37, 6, 3, 128, 64, infs.ROTARY_HALF, True),
    (37, 6, 3, 128, 96, infs.ROTARY_INTERLEAVED, True),
    (130, 32, 4, 64, 48, infs.ROTARY_INTERLEAVED, False),
    (130, 2, 2, 64, 6, infs.ROTARY_HALF, True),      # pairs that 16 bytes do not divide
    (33, 3, 1, 80, 80, infs.ROTARY_HALF, False),
    (33, 3, 1, 100, 50, infs.ROTARY_HALF, True),
    (9, 5, 5, 7, 2, infs.ROTARY_INTERLEAVED, True),  # odd head size
    (300, 2, 1, 256, 256, infs.ROTARY_HALF, True),
    (3000, 8, 2, 128, 128, infs.ROTARY_HALF, False),
    (3001, 8, 2, 64, 32, infs.ROTARY_INTERLEAVED, True),
    (5000, 1, 1, 16, 2, infs.ROTARY_HALF, False),
]


@pytest.mark.parametrize("T,hq,hk,d,rd,layout,bf16", CASES)
def test_rows(T, hq, hk, d, rd, layout, bf16):
    import torch

    r = infs.Rotary(config(head_dim=d, rotary_dim=rd, layout=layout))
    f, amp = r.frequencies()
    q, qn = make((T, hq, d), bf16, 1)
    k, kn = make((T, hk, d), bf16, 2)
    pos = torch.randint(-1000, 100000, (T,), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    dt = infs.BF16 if bf16 else infs.F32
    for inverse in (False, True):
        qo, ko = torch.full_like(q, 7), torch.full_like(k, 7)
        r.rotate_rows(dt, T, infs.rotary_rows(q, qo, hq), infs.rotary_rows(k, ko, hk), positions=pos.cuda(),
                      inverse=inverse, stream=torch.cuda.current_stream())
        for got, x in ((qo, qn), (ko, kn)):
            check(got, *rotated(x, pos.numpy(), f, amp, layout, rd, inverse), bf16)
    # positions that count up, in place, one tensor alone
    y = k.clone()
    r.rotate_rows(dt, T, k=infs.rotary_rows(y, y, hk), first_position=12345, stream=torch.cuda.current_stream())
    check(y, *rotated(kn, 12345 + np.arange(T), f, amp, layout, rd), bf16)
    assert torch.equal(q.double().cpu(), torch.from_numpy(qn)) and torch.equal(k.double().cpu(), torch.from_numpy(kn))


@pytest.mark.parametrize("scaling", [infs.ROTARY_LINEAR, infs.ROTARY_NTK, infs.ROTARY_YARN, infs.ROTARY_BANDS])
def test_scalings_and_far_positions(scaling):
    import torch

    high = 4.0 if scaling == infs.ROTARY_BANDS else 32.0
    r = infs.Rotary(config(head_dim=128, rotary_dim=128, scaling=scaling, factor=8.0, base=1e6, high=high))
    f, amp = r.frequencies()
    x, xn = make((6, 2, 128), False, 5)
    pos = torch.tensor([0, 1, 1 << 20, (1 << 31) - 1, -(1 << 31), 1234567891], dtype=torch.int32)
    out = torch.empty_like(x)
    r.rotate_rows(infs.F32, 6, infs.rotary_rows(x, out, 2), positions=pos.cuda(), stream=torch.cuda.current_stream())
    check(out, *rotated(xn, pos.numpy(), f, amp, infs.ROTARY_HALF, 128), False, far=2 * 2.0 ** -22)


@pytest.mark.parametrize("bf16", [True, False])
def test_strides_and_alignment(bf16):
    # rows out of a fused projection into head-major buffers, misaligned by an element; what lies between
    # the rows stays as it was
    import torch

    T, hq, hk, d, layers = 19, 4, 2, 64, 1
    r = infs.Rotary(config())
    f, amp = r.frequencies()
    dt = torch.bfloat16 if bf16 else torch.float32
    for shift in (0, 1):
        heads = hq + 2 * hk
        flat, flat_n = make((shift + T * heads * d,), bf16, 7)
        x, xn = flat[shift:].view(T, heads, d), flat_n[shift:].reshape(T, heads, d)
        pad = 16 if shift == 0 else 3
        qo = torch.full((hq, T + 1, d + pad), 9.0, dtype=dt, device="cuda")
        ko = torch.full((T, hk, d), 9.0, dtype=dt, device="cuda")
        q = infs.rotary_rows(x, qo, hq, in_strides=(heads * d, d, 0), out_strides=(d + pad, (T + 1) * (d + pad), 0))
        k = infs.rotary_rows(x[:, hq:], ko, hk, in_strides=(heads * d, d, 0))
        r.rotate_rows(infs.BF16 if bf16 else infs.F32, T, q, k, first_position=100, stream=torch.cuda.current_stream())
        pos = 100 + np.arange(T)
        want, mag = rotated(xn, pos, f, amp, infs.ROTARY_HALF, d)
        check(qo[:, :T, :d].transpose(0, 1), want[:, :hq], mag[:, :hq], bf16)
        check(ko, want[:, hq:hq + hk], mag[:, hq:hq + hk], bf16)
        assert bool((qo[:, T] == 9).all()) and bool((qo[:, :, d:] == 9).all())
        assert torch.equal(flat.double().cpu(), torch.from_numpy(flat_n))


def test_gradient_is_the_derivative():
    # g . R x is linear in x: its gradient R^T g (inverse) against central differences, which are exact up to
    # the roundings of two fp32 forward passes: |R x| <= 2 |x|, sums of 2 d terms over a step of 2h
    import torch

    T, H, d = 3, 2, 64
    r = infs.Rotary(config(rotary_dim=32, scaling=infs.ROTARY_YARN, factor=4.0))
    x, xn = make((T, H, d), False, 11)
    g, gn = make((T, H, d), False, 12)
    grad = torch.empty_like(g)
    s = torch.cuda.current_stream()
    r.rotate_rows(infs.F32, T, infs.rotary_rows(g, grad, H), first_position=50, inverse=True, stream=s)

    def forward(v):
        out = torch.empty_like(v)
        r.rotate_rows(infs.F32, T, infs.rotary_rows(v, out, H), first_position=50, stream=s)
        return float((out.double() * g.double()).sum())

    rng = np.random.default_rng(0)
    scale = float(np.abs(gn).sum()) * 4 * F32_EPS * 4 / (2 * 0.5)
    for _ in range(20):
        t, h, e = rng.integers(T), rng.integers(H), rng.integers(d)
        up, dn = x.clone(), x.clone()
        up[t, h, e] += 0.5
        dn[t, h, e] -= 0.5
        step = float(up[t, h, e]) - float(dn[t, h, e])
        assert abs((forward(up) - forward(dn)) / step - float(grad[t, h, e])) <= scale


def test_infinities_and_nan_stay_in_their_pairs():
    import torch

    r = infs.Rotary(config())
    x = torch.ones(2, 1, 64, device="cuda")
    x[0, 0, 3], x[1, 0, 40] = float("inf"), float("nan")
    r.rotate_rows(infs.F32, 2, infs.rotary_rows(x, x, 1), first_position=5, stream=torch.cuda.current_stream())
    finite = torch.isfinite(x).cpu()
    want = torch.ones(2, 1, 64, dtype=torch.bool)
    want[0, 0, [3, 35]] = False
    want[1, 0, [8, 40]] = False
    assert torch.equal(finite, want)


def test_captured_and_replayed():
    import torch

    T, H, d = 50, 4, 64
    r = infs.Rotary(config())
    f, amp = r.frequencies()
    x, _ = make((T, H, d), True, 21)
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.rotate_rows(infs.BF16, T, infs.rotary_rows(x, out, H), positions=pos, stream=torch.cuda.current_stream())
    del r  # the launch holds all it needs
    for i in range(3):
        y, yn = make((T, H, d), True, 30 + i)
        x.copy_(y)
        pos.copy_(torch.arange(T, device="cuda").int() * (i + 1))
        g.replay()
        torch.cuda.synchronize()
        check(out, *rotated(yn, np.arange(T) * (i + 1), f, amp, infs.ROTARY_HALF, d), True)


@pytest.mark.parametrize("bf16", [True, False])
def test_step_and_probe_positions(bf16):
    # rows of live slots turn at prompt length + tokens so far; idle slots' rows stay as they were
    import torch

    L, hq, hkv, d, m = 2, 4, 2, 64, 3
    ctx = infs.Context(infs.make_config(num_layers=L, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, num_prompts=2,
                                        slots_per_prompt=m, samples_per_prompt=8, max_prompt_len=64, max_suffix_len=64,
                                        dtype=infs.BF16 if bf16 else infs.F32, probe_tokens=4),
                       stream=torch.cuda.current_stream())
    S = 2 * m
    plen = [37, 0]
    for p in range(2):
        pk, _ = make((max(1, plen[p]), hkv, d), bf16, 40)
        for layer in range(L):
            ctx.prefill_shared(p, layer, plen[p], pk, pk)
    r = infs.Rotary(config())
    f, amp = r.frequencies()
    q, qn = make((L, S, hq, d), bf16, 41)
    k, kn = make((L, S, hkv, d), bf16, 42)
    o = torch.empty(L, S, hq, d, device="cuda")
    # one probe step of three samples of prompt 0, of which the middle one is idle
    n, live = 3, [1, 0, 1]
    pq, pk = q[:, :n].contiguous(), k[:, :n].contiguous()
    for step in range(2):
        qo, ko = torch.full_like(pq, 5), torch.full_like(pk, 5)
        ctx.rotate_probe(r, 0, 2, n, live, infs.rotary_rows(pq, qo, hq), infs.rotary_rows(pk, ko, hkv), num_layers=L)
        for j in range(n):
            for got, x in ((qo, qn), (ko, kn)):
                if not live[j]:
                    assert bool((got[:, j] == 5).all())
                    continue
                check(got[:, j:j + 1], *rotated(x[:, j:j + 1], [plen[0] + step], f, amp, infs.ROTARY_HALF, d), bf16)
        for layer in range(L):
            ctx.probe_step(layer, 0, 2, n, live, qo[layer], ko[layer], ko[layer], o[layer])
        ctx.end_probe_step()
    for s, i in ((0, 2), (2, 3), (4, 0)):  # sample 2 of prompt 0 has two probe tokens
        ctx.refill_slot(s, s // m, i)
    length = {0: 2, 2: 0, 4: 0}
    for step in range(3):
        qo, ko = torch.full_like(q, 5), torch.full_like(k, 5)
        if step == 1:  # layer by layer
            for layer in range(L):
                ctx.rotate_step(r, infs.rotary_rows(q[layer], qo[layer], hq), infs.rotary_rows(k[layer], ko[layer], hkv))
                ctx.decode_step(layer, qo[layer], ko[layer], ko[layer], o[layer])
        else:
            ctx.rotate_step(r, infs.rotary_rows(q, qo, hq), infs.rotary_rows(k, ko, hkv), num_layers=L)
            for layer in range(L):
                ctx.decode_step(layer, qo[layer], ko[layer], ko[layer], o[layer])
        for s in range(S):
            for got, x in ((qo, qn), (ko, kn)):
                if s not in length:
                    assert bool((got[:, s] == 5).all())
                    continue
                p = plen[s // m] + length[s]
                check(got[:, s:s + 1], *rotated(x[:, s:s + 1], [p], f, amp, infs.ROTARY_HALF, d), bf16)
        ctx.end_step()
        for s in length:
            length[s] += 1
    ctx.sync()
    ctx.destroy()


def test_more_tokens_than_a_launch():
    # two tokens a work-group (256 angles): over 2^23 tokens go in two launches, in place
    import torch

    T, d = (1 << 23) + 5, 256
    r = infs.Rotary(config(head_dim=d, rotary_dim=d))
    f, amp = r.frequencies()
    x = torch.ones(T, 1, d, dtype=torch.bfloat16, device="cuda")
    at = [0, 1, (1 << 22) + 3, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, T - 1]
    y, yn = make((len(at), 1, d), True, 51)
    x[at] = y
    for positions in (None, torch.arange(T, dtype=torch.int32, device="cuda") + 7):
        z = x.clone()
        r.rotate_rows(infs.BF16, T, k=infs.rotary_rows(z, z, 1), positions=positions, first_position=7,
                      stream=torch.cuda.current_stream())
        check(z[at], *rotated(yn, 7 + np.array(at), f, amp, infs.ROTARY_HALF, d), True, far=2.0 ** -24)
        same, _ = rotated(np.ones((2, 1, d)), [7 + 5, 7 + T - 3], f, amp, infs.ROTARY_HALF, d)
        assert np.abs(z[[5, T - 3]].double().cpu().numpy() - same).max() < 2 ** -7
