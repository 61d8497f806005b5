"""GPU: scores of tokens and their gradient against the definitions in 64 bits.

Tolerances, with u = 2^-24 (half a step of fp32), y = (z - m) / T: y log2 e is a difference and two
products with a rounded constant, off by at most 4u |y log2 e|; a power of two by the hardware 2u; a sum
of the row is a chain of at most K = vocab / 256 + 64 additions per thread and joins.  So S is off by
at most (K + 4 + 4 E|y|) u relative, E the mean over the distribution, which is what ln S is off by;
log p_t by that + 8u (|y_t| + ln S); the entropy by that + u E(|y| (K + 8 + 8 |y|)).  A gradient
p (A + B log p): p is off by r = S's + 8u (1 + |y| + ln S) relative, the bracket by 8u of its terms'
sizes and the entropy's error.  Half a step of the output's type on top."""

import math

import numpy as np
import pytest

from paper_2506_22950_amd import infs

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {True: 2.0 ** -8, False: 2.0 ** -24}


def scorer(**kw):
    import torch

    c = dict(dtype=infs.BF16, max_rows=4096, top_k=0, temperature=1.0)
    c.update(kw)
    return infs.Scorer(infs.make_scorer_config(**c), stream=torch.cuda.current_stream())


class Ref:
    """z [n, v] float64 (finite or -inf)."""

    def __init__(self, z, tokens, T):
        n, v = z.shape
        with np.errstate(all="ignore"):
            self.m = z.max(1)
            self.none = self.m == -np.inf
            y = np.where(z == -np.inf, -np.inf, (z - self.m[:, None]) / T)
            y[self.none] = -np.inf
            e = np.exp(y)
            S = e.sum(1)
            self.ls = np.log(S)
            self.lp = y - self.ls[:, None]
            self.p = np.where(self.none[:, None], 0.0, e / S[:, None])
            plp = np.where(self.p > 0, self.p * self.lp, 0.0)
            self.h = -plp.sum(1)
            ay = np.where(self.p > 0, np.abs(y), 0.0)
        self.y = y
        K = v / 256 + 64
        self.s_err = (K + 4 + 4 * (self.p * ay).sum(1)) * U
        self.h_err = self.s_err + U * (self.p * ay * (K + 8 + 8 * ay)).sum(1) + 2 * U * self.h
        rows = np.arange(n)
        t = np.clip(tokens, 0, v - 1)
        self.lp_t = np.where(tokens == -1, 0.0, np.where((tokens >= 0) & (tokens < v), self.lp[rows, t], np.nan))
        self.lp_t[self.none & (tokens >= 0) & (tokens < v)] = -np.inf
        ayt = np.where(np.isfinite(y[rows, t]), np.abs(y[rows, t]), 0.0)
        self.lp_err = self.s_err + 8 * U * (ayt + np.where(self.none, 0, self.ls))
        self.h[self.none] = 0.0


def close(got, want, err):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf])
    ok = np.isfinite(want)
    bad = np.abs(got[ok] - want[ok]) > np.broadcast_to(err, want.shape)[ok] + 1e-38
    assert not bad.any(), (int(bad.sum()), got[ok][bad][:4], want[ok][bad][:4])


def check(z, tokens, T, top, bf16, stride=None, shift=0, grads=True, entropy=True):
    """z: numpy float32 [n, v] of values that the type holds (finite or -inf); scored in a buffer with row
    stride `stride` that begins `shift` elements into an allocation."""
    import torch

    n, v = z.shape
    stride = stride or v
    dt = torch.bfloat16 if bf16 else torch.float32
    flat = torch.full((shift + n * stride + 8,), 50.0, dtype=dt, device="cuda")
    zt = flat[shift:shift + n * stride].view(n, stride)
    zt[:, :v] = torch.from_numpy(z).cuda().to(dt)
    z64 = zt[:, :v].double().cpu().numpy()
    tok = torch.from_numpy(np.asarray(tokens, dtype=np.int32)).cuda()
    ref = Ref(z64, np.asarray(tokens), T)
    s = scorer(vocab=v, dtype=infs.BF16 if bf16 else infs.F32, max_rows=n, top_k=top, temperature=T)
    lp, h = (torch.full((n,), 3.0, device="cuda") for _ in range(2))
    stats = torch.full((n, 2), 3.0, device="cuda")
    ids = torch.full((n, max(top, 1)), 77, dtype=torch.int32, device="cuda")
    tl = torch.full((n, max(top, 1)), 3.0, device="cuda")
    s.score(n, zt, tok, lp, entropy=h, stats=stats, top_id=ids if top else None, top_logprob=tl if top else None,
            row_stride=stride)
    close(lp, ref.lp_t, ref.lp_err)
    close(h, ref.h, ref.h_err)
    st = stats.double().cpu().numpy()
    assert np.array_equal(st[:, 0], ref.m)
    close(stats[:, 1], ref.ls, ref.s_err + 2 * U * np.where(ref.none, 0, ref.ls))
    if top:
        order = np.argsort(-z64, axis=1, kind="stable")[:, :top]
        vals = np.take_along_axis(z64, order, 1)
        want = np.full((n, top), -1)
        want[:, :order.shape[1]] = np.where(vals == -np.inf, -1, order)
        assert np.array_equal(ids.cpu().numpy(), want)
        wl = np.full((n, top), -np.inf)
        with np.errstate(all="ignore"):
            wl[:, :order.shape[1]] = np.where(vals == -np.inf, -np.inf, np.take_along_axis(ref.lp, order, 1))
        wl[want < 0] = -np.inf
        yt = np.where(np.isfinite(wl), np.abs(wl), 0)
        close(tl, wl, ref.s_err[:, None] + 8 * U * (yt + 2 * np.where(ref.none, 0, ref.ls)[:, None]))
    if grads:
        g = torch.randn(n, generator=torch.Generator().manual_seed(1))
        gh = torch.randn(n, generator=torch.Generator().manual_seed(2))
        for with_h in ((False, True) if entropy else (False,)):
            out = torch.full((shift + n * stride + 8,), 9.0, dtype=dt, device="cuda")
            gt = out[shift:shift + n * stride].view(n, stride)
            s.grad(n, zt, tok, stats, g.cuda(), gt, entropy=h if with_h else None,
                   d_entropy=gh.cuda() if with_h else None, row_stride=stride, grad_row_stride=stride)
            want, err = grad_ref(ref, np.asarray(tokens), T, g.double().numpy(), gh.double().numpy() * with_h)
            close(gt[:, :v], want, err + np.abs(want) * HALF[bf16])
            # what lies between and behind the rows stays
            assert bool((gt[:, v:] == 9).all()) and bool((out[:shift] == 9).all()) and bool((out[shift + n * stride:] == 9).all())
        assert torch.equal(zt[:, v:], torch.full_like(zt[:, v:], 50.0))
    return s, zt, tok, lp, h, stats


def grad_ref(ref, tokens, T, g, gh):
    n, v = ref.p.shape
    g = np.where(tokens == -1, 0.0, g)[:, None]
    gh = gh[:, None]
    lp = np.where(ref.p > 0, ref.lp, 0.0)
    want = -ref.p * g - gh * ref.p * (lp + ref.h[:, None])
    rows = np.arange(n)
    has = (tokens >= 0) & (tokens < v)
    want[rows[has], tokens[has]] += g[has, 0]
    want = want / T
    want[ref.none] = 0.0
    want[(tokens < -1) | (tokens >= v)] = np.nan
    r = ref.s_err[:, None] + 8 * U * (1 + np.abs(lp) + 2 * np.where(ref.none, 0, ref.ls)[:, None])
    size = np.abs(g) + np.abs(gh) * (np.abs(lp) + ref.h[:, None])
    err = (ref.p * (size * (r + 8 * U) + np.abs(gh) * (ref.h_err[:, None] + r)) + 4 * U * np.abs(g) * (np.abs(want) > 0)) / T
    return want, err + 1e-37


def logits(n, v, seed, spread=3.0):
    return (np.random.default_rng(seed).standard_normal((n, v)) * spread).astype(np.float32)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,v,top,T", [
    (1, 1, 1, 1.0), (1, 2, 2, 1.0), (3, 7, 4, 0.5), (1, 8, 8, 1.0), (5, 63, 32, 1.0), (2, 1000, 0, 1.0), (2, 1024, 5, 2.0),
    (1, 4097, 1, 1.0), (17, 8191, 3, 0.7), (3, 8192, 32, 1.0), (3, 8193, 32, 1.0), (1, 32003, 20, 1.0),
    (16, 50257, 20, 1.0), (2, 151936, 32, 1.0), (300, 5003, 7, 1.3), (2100, 1003, 2, 1.0), (1, 300001, 32, 1.0)])
def test_ordinary_rows(n, v, top, T, bf16):
    z = logits(n, v, 100 + n)
    tokens = np.random.default_rng(5).integers(-1, v, n)
    check(z, tokens, T, top, bf16)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("v,stride,shift", [(1001, 1001, 0), (1001, 1003, 1), (1000, 1024, 3), (9001, 9005, 7), (33, 40, 5),
                                            (5, 5, 1), (50257, 50257, 1)])
def test_strides_and_alignment(v, stride, shift, bf16):
    z = logits(6, v, 9)
    check(z, np.arange(6) % v, 1.0, 5, bf16, stride=stride, shift=shift)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("kind", ["ascending", "descending", "equal", "ties", "peaked", "wide", "one", "zeros"])
def test_orders_and_ties(kind, bf16):
    n, v = 3, 20011
    rng = np.random.default_rng(3)
    if kind in ("ascending", "descending"):
        z = np.sort(logits(n, v, 4), axis=1)
        z = z if kind == "ascending" else z[:, ::-1].copy()
    elif kind == "equal":
        z = np.full((n, v), 1.5, np.float32)
    elif kind == "ties":
        z = rng.integers(-3, 4, (n, v)).astype(np.float32)
    elif kind == "peaked":
        z = logits(n, v, 4, 0.1)
        z[:, 777] = 60.0
    elif kind == "wide":
        z = logits(n, v, 4, 1e4)
    elif kind == "one":  # everything but one entry masked
        z = np.full((n, v), -np.inf, np.float32)
        z[np.arange(n), [0, 10000, v - 1]] = [-5.0, 0.0, 7.0]
    else:  # both zeros are equal
        z = np.where(rng.random((n, v)) < 0.5, 0.0, -0.0).astype(np.float32)
    check(z, [5, 777, v - 1], 1.0, 32, bf16)


@pytest.mark.parametrize("bf16", [True, False])
def test_masks(bf16):
    import torch

    v = 12345
    z = logits(9, v, 8)
    low = float(torch.finfo(torch.bfloat16 if bf16 else torch.float32).min)
    z[0, 3000:] = -np.inf
    z[1, :9000] = -np.inf
    z[2, 5:] = -np.inf          # fewer left than alternatives
    z[3] = -np.inf              # nothing left
    z[4] = -np.inf              # nothing left, no token
    z[5, 100:] = low            # masked by the lowest value: its probability is 0, but it is an alternative
    z[6] = low                  # uniform
    z[7, ::2] = -np.inf
    z[8, 1:] = low
    tokens = [4000, 9001, 3, 6, -1, 200, 17, 1, 0]  # row 0's and row 7's second: a masked token
    check(z, tokens, 1.0, 32, bf16)


@pytest.mark.parametrize("n,v", [(300, 50000), (2100, 3000)])  # a work-group's batches, a wavefront's
def test_alternatives_among_lowest_values(n, v):
    # few entries at first, then the type's lowest values, alternatives too: by index, however late they come
    import torch

    low = float(torch.finfo(torch.float32).min)
    z = np.full((n, v), -np.inf, np.float32)
    z[:, 10], z[:, 200], z[:, 700] = 1.0, low, 2.0
    for i, at in enumerate((1100, 1500, 2047, 2048, v - 2, v - 1)):
        z[i % 3::3, at] = low
    z[1::5, 2500:] = low
    check(z, np.arange(n) % v, 1.0, 8, False, grads=False)


def test_tokens_out_of_range_give_nan():
    z = logits(4, 999, 1)
    check(z, [-2, 999, 2147483647, -2147483648], 1.0, 0, True)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("bf16", [True, False])
def test_nan_and_infinity_rows(bad, bf16):
    import torch

    v = 10007
    z = torch.from_numpy(logits(5, v, 2)).to(torch.bfloat16 if bf16 else torch.float32).cuda()
    for r, at in ((0, 0), (2, 5000), (4, v - 1)):
        z[r, at] = bad
    tok = torch.tensor([5, 6, 7, 8, -1], dtype=torch.int32, device="cuda")
    s = scorer(vocab=v, dtype=infs.BF16 if bf16 else infs.F32, top_k=3)
    lp, h = torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    st, ids, tl = torch.empty(5, 2, device="cuda"), torch.empty(5, 3, dtype=torch.int32, device="cuda"), torch.empty(5, 3, device="cuda")
    s.score(5, z, tok, lp, entropy=h, top_id=ids, top_logprob=tl, stats=st)
    g = torch.empty_like(z)
    s.grad(5, z, tok, st, torch.ones(5, device="cuda"), g, entropy=h, d_entropy=torch.ones(5, device="cuda"))
    nan = torch.tensor([True, False, True, False, True])
    assert torch.equal(torch.isnan(h).cpu(), nan) and torch.equal(torch.isnan(st[:, 1]).cpu(), nan)
    assert torch.equal(torch.isnan(lp).cpu(), torch.tensor([True, False, True, False, False])) and float(lp[4]) == 0
    assert bool((ids[nan.cuda()] == -1).all()) and bool((ids[~nan.cuda()] >= 0).all())
    assert bool(torch.isnan(tl[nan.cuda()]).all())
    assert bool(torch.isnan(g[nan.cuda()]).all()) and bool(torch.isfinite(g[~nan.cuda()]).all())


def test_parts_of_the_outputs():
    # any subset of the outputs gives what all of them together give
    import torch

    n, v = 7, 30011
    s, z, tok, lp, h, st = check(logits(n, v, 3), np.arange(n), 1.0, 6, True, grads=False)
    for names in (("lp",), ("h",), ("top",), ("st",), ("lp", "top"), ("h", "st")):
        o = {k: torch.empty_like(x) for k, x in (("lp", lp), ("h", h), ("st", st))}
        ids, tl = torch.empty(n, 6, dtype=torch.int32, device="cuda"), torch.empty(n, 6, device="cuda")
        s.score(n, z, tok if "lp" in names else None, o["lp"] if "lp" in names else None,
                entropy=o["h"] if "h" in names else None, stats=o["st"] if "st" in names else None,
                top_id=ids if "top" in names else None, top_logprob=tl if "top" in names else None)
        for k, x in (("lp", lp), ("h", h), ("st", st)):
            assert k not in names or torch.equal(o[k], x), (names, k)
        if "top" in names:
            assert bool((tl[:, :-1] >= tl[:, 1:]).all()) and bool((ids >= 0).all())


@pytest.mark.parametrize("n", [1, 16, 700])
def test_the_same_call_gives_the_same_bits(n):
    import torch

    v = 40009
    s, z, tok, lp, h, st = check(logits(n, v, 13), np.arange(n) % v, 1.0, 9, True, grads=False)
    for _ in range(5):
        lp2, h2, st2 = torch.empty_like(lp), torch.empty_like(h), torch.empty_like(st)
        s.score(n, z, tok, lp2, entropy=h2, stats=st2)
        assert torch.equal(lp, lp2) and torch.equal(h, h2) and torch.equal(st, st2)


def test_rows_beyond_32_bit_offsets():
    import torch

    v, stride = 4099, (1 << 31) + 24
    flat = torch.empty(stride + v, dtype=torch.bfloat16, device="cuda")
    z = logits(2, v, 6)
    for r in range(2):
        flat[r * stride:r * stride + v] = torch.from_numpy(z[r]).cuda()
    z64 = np.stack([flat[r * stride:r * stride + v].double().cpu().numpy() for r in range(2)])
    tok = torch.tensor([9, 4098], dtype=torch.int32, device="cuda")
    ref = Ref(z64, tok.cpu().numpy(), 1.0)
    s = scorer(vocab=v, max_rows=2, top_k=2)
    lp, h, st = torch.empty(2, device="cuda"), torch.empty(2, device="cuda"), torch.empty(2, 2, device="cuda")
    ids, tl = torch.empty(2, 2, dtype=torch.int32, device="cuda"), torch.empty(2, 2, device="cuda")
    s.score(2, flat, tok, lp, entropy=h, stats=st, top_id=ids, top_logprob=tl, row_stride=stride)
    close(lp, ref.lp_t, ref.lp_err)
    assert np.array_equal(ids.cpu().numpy(), np.argsort(-z64, axis=1, kind="stable")[:, :2])
    g = torch.ones(2, device="cuda")
    s.grad(2, flat, tok, st, g, flat, row_stride=stride, grad_row_stride=stride)  # over the logits
    got = torch.stack([flat[:v], flat[stride:]])
    want, err = grad_ref(ref, tok.cpu().numpy(), 1.0, np.ones(2), np.zeros(2))
    close(got, want, err + np.abs(want) * HALF[True])


def test_gradient_against_differences():
    # d/dz of  sum g log p_t + gh H  in fp32 against central differences of the 64-bit definition: their error
    # is h^2/6 of a third derivative of at most 2 (|g| + |gh| (ln v + 4)) / T^3, and 64-bit roundings over 2h
    import torch

    n, v, T, step = 3, 50, 0.8, 1e-4
    s, z, tok, lp, h, st = check(logits(n, v, 17, 1.0), [3, -1, 49], T, 0, False)
    g, gh = torch.tensor([1.0, -2.0, 0.5]), torch.tensor([0.3, 1.0, -0.7])
    out = torch.empty_like(z)
    s.grad(n, z, tok, st, g.cuda(), out, entropy=h, d_entropy=gh.cuda())
    z64, t = z.double().cpu().numpy(), np.array([3, -1, 49])

    def f(x):
        r = Ref(x, t, T)
        return r.lp_t * g.numpy() * (t >= 0) + r.h * gh.numpy()

    want = np.zeros((n, v))
    for j in range(v):
        d = np.zeros((n, v))
        d[:, j] = step
        want[:, j] = (f(z64 + d) - f(z64 - d)) / (2 * step)
    size = (np.abs(g.numpy()) + np.abs(gh.numpy()) * (math.log(v) + 4))[:, None]
    bound = step ** 2 * size / T ** 3 + 1e-15 * 20 / step + 100 * U * size / T
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= bound)


@pytest.mark.parametrize("n", [16, 700])
def test_captured_and_replayed(n):
    # a graph of a forward and a backward pass, replayed with other eager work of the scorer between
    import torch

    v = 33001
    s = scorer(vocab=v, max_rows=n, top_k=5)
    z = torch.zeros(n, v, dtype=torch.bfloat16, device="cuda")
    tok = torch.zeros(n, dtype=torch.int32, device="cuda")
    d = torch.ones(n, device="cuda")
    lp, h, st = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
    ids, tl = torch.empty(n, 5, dtype=torch.int32, device="cuda"), torch.empty(n, 5, device="cuda")
    out = torch.empty_like(z)
    side = torch.cuda.Stream()
    s2 = infs.Scorer(infs.make_scorer_config(vocab=v, dtype=infs.BF16, max_rows=n, top_k=5), stream=side)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        s2.score(n, z, tok, lp, entropy=h, top_id=ids, top_logprob=tl, stats=st)
        s2.grad(n, z, tok, st, d, out)
    for i in range(4):
        z.copy_(torch.from_numpy(logits(n, v, 50 + i)))
        tok.fill_(i * 7)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        torch.cuda.synchronize()
        e = [torch.empty_like(x) for x in (lp, h, ids, tl, st, out)]
        s.score(n, z, tok, e[0], entropy=e[1], top_id=e[2], top_logprob=e[3], stats=e[4])
        s.grad(n, z, tok, e[4], d, e[5])
        torch.cuda.synchronize()
        for a, b in zip(e, (lp, h, ids, tl, st, out)):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("bf16", [True, False])
def test_lowest_values_at_small_temperatures(bf16):
    # (z - m) / T passes the type's range: probability 0, no part in any sum
    import torch

    v = 5003
    z = logits(3, v, 21)
    z[0, 100:] = z[1, :4000] = z[2, 1::2] = float(torch.finfo(torch.bfloat16 if bf16 else torch.float32).min)
    check(z, [7, 4500, 0], 2.0 ** -10, 0, bf16)


@pytest.mark.parametrize("n,v", [(5, 9001), (3000, 501), (64, 4096)])
@pytest.mark.parametrize("bf16", [True, False])
def test_gradient_over_the_logits(n, v, bf16):
    import torch

    s, z, tok, lp, h, st = check(logits(n, v, 31), np.arange(n) % v, 1.0, 0, bf16, grads=False)
    z = z.contiguous()
    g, gh = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    out = torch.empty_like(z)
    s.grad(n, z, tok, st, g, out, entropy=h, d_entropy=gh)
    s.grad(n, z, tok, st, g, z, entropy=h, d_entropy=gh)
    assert torch.equal(z, out)


def test_two_scorers_at_once():
    # scorers on streams of their own, calls of both in flight; each gives what it gives alone
    import torch

    n, v, top = 16, 100003, 20
    z = [torch.from_numpy(logits(n, v, 41 + i)).cuda().to(torch.bfloat16) for i in range(2)]
    tok = torch.arange(n, dtype=torch.int32, device="cuda")

    def outputs():
        return (torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, top, dtype=torch.int32, device="cuda"),
                torch.empty(n, top, device="cuda"), torch.empty(n, 2, device="cuda"))

    def call(s, z, o):
        s.score(n, z, tok, o[0], entropy=o[1], top_id=o[2], top_logprob=o[3], stats=o[4])

    alone, s = [outputs() for _ in range(2)], scorer(vocab=v, max_rows=n, top_k=top)
    for i in range(2):
        call(s, z[i], alone[i])
    streams = [torch.cuda.Stream() for _ in range(2)]
    scorers = [infs.Scorer(infs.make_scorer_config(vocab=v, dtype=infs.BF16, max_rows=n, top_k=top), stream=x) for x in streams]
    got = [[outputs() for _ in range(20)] for _ in range(2)]
    torch.cuda.synchronize()
    for j in range(20):
        for i in range(2):
            call(scorers[i], z[(i + j) % 2], got[i][j])
    torch.cuda.synchronize()
    for i in range(2):
        for j in range(20):
            assert all(torch.equal(a, b) for a, b in zip(got[i][j], alone[(i + j) % 2])), (i, j)
