"""GPU: attention of packed sequences and its gradient against the formulas in 64 bits, and the gradient against
differences of the 64-bit forward pass.

Tolerances.  A score is a sum of d products, within S = scale sum|q k| (d + 2) 2^-24 + |s| 2^-22 (the exponent's
argument and exp2 itself); p = e^(s - lse) is then within 2 max S + |lse| 2^-23 + 2^-21 of itself, R for a row.  Over n
keys o is within sum(p |v|) (R + n 2^-24 + B) + half a step, B = 2^-8 where p is rounded to bf16 (0 in fp32), and lse
within max S + |lse| 2^-22 + (n + 8) 2^-24.  Gradient, from the o and lse that it is given: up.v and D are within
V = sum|up v| (d + 2) 2^-24 and U = sum|up o| (d + 2) 2^-24, so ds is within |ds| (R + B) + p (V + U) + p |up.v - D| 2^-22,
and dq, dk, dv are within the sums of that (of p (R + B)) times |k|, |q|, |up|, with n 2^-24 for the sum, and half a
step."""

import numpy as np
import pytest

from paper_2506_22950_amd import infs

pytestmark = pytest.mark.gpu

E32, EBF = 2.0 ** -24, 2.0 ** -8


def starts(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


class Case:
    """Inputs on the GPU; rows as views of buffers with strides, a tail of rows behind the last sequence."""

    def __init__(self, hq, hkv, d, bf16, q_lens, k_lens=None, scale=0.0, layout="dense", seed=1, tail=3, spread=1.0):
        import torch

        self.hq, self.hkv, self.d, self.bf16 = hq, hkv, d, bf16
        self.q_lens, self.k_lens = q_lens, k_lens if k_lens is not None else q_lens
        self.shared = k_lens is None
        self.scale = scale or 1.0 / np.sqrt(d)
        self.given_scale = scale
        self.dt = torch.bfloat16 if bf16 else torch.float32
        self.gen = torch.Generator().manual_seed(seed)
        self.tq, self.tk = sum(self.q_lens) + tail, sum(self.k_lens) + (tail if not self.shared else tail)
        if layout == "fused" and self.shared:
            x = torch.randn(self.tq, hq + 2 * hkv, d, generator=self.gen).to(self.dt).cuda()
            self.q, self.k, self.v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        elif layout == "heads":  # [H, T, d]
            self.q = torch.randn(hq, self.tq, d, generator=self.gen).to(self.dt).cuda().transpose(0, 1)
            self.k, self.v = (torch.randn(hkv, self.tk, d, generator=self.gen).to(self.dt).cuda().transpose(0, 1)
                              for _ in range(2))
        else:
            self.q = (spread * torch.randn(self.tq, hq, d, generator=self.gen)).to(self.dt).cuda()
            self.k, self.v = (torch.randn(self.tk, hkv, d, generator=self.gen).to(self.dt).cuda() for _ in range(2))
        self.d_o = torch.randn(self.tq, hq, d, generator=self.gen).to(self.dt).cuda()
        self.q_off = torch.tensor(starts(self.q_lens), dtype=torch.int32, device="cuda")
        self.k_off = torch.tensor(starts(self.k_lens), dtype=torch.int32, device="cuda")

    def attention(self, stream=None, max_tokens=None):
        import torch

        return infs.Attention(infs.make_attention_config(
            num_q_heads=self.hq, num_kv_heads=self.hkv, head_dim=self.d, dtype=infs.BF16 if self.bf16 else infs.F32,
            scale=self.given_scale, max_tokens=max_tokens or self.tq), stream=stream or torch.cuda.current_stream())

    def rows(self, x, out=None):
        st = (0, 0, 0) if out is None else (out.stride(0), out.stride(1), 0)
        return infs.rotary_rows(x, out, x.shape[1], (x.stride(0), x.stride(1), 0), st)

    def key_args(self):
        return {} if self.shared else dict(k_tokens=self.tk, k_offsets=self.k_off)

    def outputs(self):
        """o and lse, filled with what has to stay behind the sequences."""
        import torch

        return (torch.full((self.tq, self.hq, self.d), 7.0, dtype=self.dt, device="cuda"),
                torch.full((self.tq, self.hq), 7.0, device="cuda"))

    def attend(self, a, o, lse):
        a.attend(len(self.q_lens), self.tq, self.q_off, self.rows(self.q, o), self.rows(self.k), self.rows(self.v), lse,
                 **self.key_args())

    def grads(self):
        import torch

        return [torch.full((x.shape[0], x.shape[1], self.d), 7.0, dtype=self.dt, device="cuda") for x in (self.q, self.k, self.v)]

    def grad(self, a, out, o, lse):
        a.grad(len(self.q_lens), self.tq, self.q_off, self.rows(self.q, out[0]), self.rows(self.k, out[1]),
               self.rows(self.v, out[2]), self.rows(o), self.rows(self.d_o), lse, **self.key_args())

    def parts(self):
        """(query rows, key rows, head, mask of the keys seen) of every sequence and head."""
        qs, ks = starts(self.q_lens), starts(self.k_lens)
        for i, (n, m) in enumerate(zip(self.q_lens, self.k_lens)):
            seen = np.arange(m)[None, :] <= np.arange(n)[:, None] + m - n
            for h in range(self.hq):
                yield slice(qs[i], qs[i] + n), slice(ks[i], ks[i] + m), h, seen


def f64(x):
    return x.double().cpu().numpy()


def scores(c, q, k, seen):
    """Masked scores and S, the bound on their error."""
    s = c.scale * (q @ k.T)
    off = c.scale * (np.abs(q) @ np.abs(k).T) * (c.d + 2) * E32 + np.abs(s) * 2.0 ** -22
    return np.where(seen, s, -np.inf), np.where(seen, off, 0.0)


def check_forward(c, o, lse):
    q, k, v, got, got_lse = f64(c.q), f64(c.k), f64(c.v), f64(o), f64(lse)
    b = EBF if c.bf16 else 0.0
    for rq, rk, h, seen in c.parts():
        g = h // (c.hq // c.hkv)
        some = seen.any(1)
        s, off = scores(c, q[rq, h], k[rk, g], seen)
        want, want_lse = np.zeros_like(q[rq, h]), np.full(len(seen), -np.inf)
        if some.any():
            top = s[some].max(1)
            e = np.exp(s[some] - top[:, None])
            want_lse[some] = top + np.log(e.sum(1))
            p = e / e.sum(1, keepdims=True)
            want[some] = p @ v[rk, g]
            n = seen[some].sum(1)
            worst = off[some].max(1)
            rel = 2 * worst + np.abs(want_lse[some]) * 2.0 ** -23 + 2.0 ** -21
            bound = (p @ np.abs(v[rk, g])) * (rel + n * E32 + b)[:, None] + np.abs(want[some]) * (EBF if c.bf16 else E32) + 1e-37
            err = np.abs(got[rq, h][some] - want[some])
            assert np.all(err <= 1.001 * bound), (h, float((err / bound).max()))
            bl = worst + np.abs(want_lse[some]) * 2.0 ** -22 + (n + 8) * E32
            assert np.all(np.abs(got_lse[rq, h][some] - want_lse[some]) <= bl), h
        assert np.all(got[rq, h][~some] == 0) and np.all(got_lse[rq, h][~some] == -np.inf)
    end = sum(c.q_lens)
    assert np.all(got[end:] == 7) and np.all(got_lse[end:] == 7)


def check_grads(c, out, o, lse):
    q, k, v, up, o, lse = (f64(x) for x in (c.q, c.k, c.v, c.d_o, o, lse))
    b = EBF if c.bf16 else 0.0
    want, bound = [np.zeros(x.shape) for x in (q, k, v)], [np.zeros(x.shape) for x in (q, k, v)]
    for rq, rk, h, seen in c.parts():
        g = h // (c.hq // c.hkv)
        x, y, z, u = q[rq, h], k[rk, g], v[rk, g], up[rq, h]
        s, off = scores(c, x, y, seen)
        some = seen.any(1)
        row = np.where(some, lse[rq, h], 0.0)
        p = np.where(seen, np.exp(s - row[:, None]), 0.0)
        rel = (2 * off.max(1, initial=0.0) + np.abs(row) * 2.0 ** -23 + 2.0 ** -21)[:, None]
        dot = u @ z.T - (u * o[rq, h]).sum(1, keepdims=True)
        ds = p * dot
        far = (np.abs(u) @ np.abs(z).T + (np.abs(u) * np.abs(o[rq, h])).sum(1, keepdims=True)) * (c.d + 2) * E32
        ds_off = np.abs(ds) * (rel + b) + p * (far + np.abs(dot) * 2.0 ** -22)
        n, m = len(seen), seen.shape[1]
        terms = n * (c.hq // c.hkv)
        want[0][rq, h] = c.scale * ds @ y
        bound[0][rq, h] = c.scale * (ds_off + np.abs(ds) * m * E32) @ np.abs(y)
        want[1][rk, g] += c.scale * ds.T @ x
        bound[1][rk, g] += c.scale * (ds_off + np.abs(ds) * terms * E32).T @ np.abs(x)
        want[2][rk, g] += p.T @ u
        bound[2][rk, g] += (p * (rel + b + terms * E32)).T @ np.abs(u)
    for i, (name, w, e, ends) in enumerate(zip("qkv", want, bound, (sum(c.q_lens), sum(c.k_lens), sum(c.k_lens)))):
        got = f64(out[i])
        e = e + np.abs(w) * (EBF if c.bf16 else E32) + 1e-37
        err = np.abs(got - w)[:ends]
        assert np.all(err <= 1.001 * e[:ends]), (name, float((err / e[:ends]).max()))
        assert np.all(got[ends:] == 7), name


CASES = [
    # q heads, kv heads, d, bf16, q_lens, k_lens (None: the queries'), what else
    (1, 1, 64, True, [1], None, {}),
    (4, 2, 64, False, [32, 1, 17, 64], None, {}),
    (4, 2, 64, True, [32, 0, 1, 17, 64], None, {"layout": "fused"}),   # an empty sequence
    (2, 2, 128, True, [129, 63, 64, 65], None, {"layout": "heads"}),
    (2, 1, 128, False, [33, 31, 100], None, {"layout": "fused"}),
    (6, 2, 64, True, [300, 77], None, {}),                              # three heads a group
    (5, 1, 128, True, [57, 130], None, {}),
    (16, 1, 64, False, [21], None, {}),
    (24, 8, 64, True, [1, 40, 7], [513, 40, 200], {}),                  # chunks over what went before
    (4, 2, 128, False, [1, 20, 3], [97, 33, 3], {"layout": "heads"}),
    (4, 4, 64, True, [50, 20, 1], [20, 0, 1], {}),                      # rows that see no key
    (4, 2, 64, False, [70, 5], [10, 0], {}),
    (2, 2, 64, True, [0, 9], [33, 9], {}),                              # keys that no query sees
    (8, 8, 128, True, [1500], None, {"scale": 0.03125}),
    (4, 1, 128, True, [700, 3, 400], [900, 1300, 400], {}),
    (2, 1, 64, True, [60, 90], None, {"spread": 30.0}),                 # one key takes nearly all
    (2, 1, 128, False, [60, 90], None, {"spread": 30.0}),
    (3, 3, 64, False, [200], None, {"scale": 4.0}),
    (64, 64, 64, True, [700, 3, 400, 1], None, {}),                     # enough rows to fill the GPU with the largest tiles
    (48, 16, 128, True, [520, 130, 700], [600, 130, 901], {}),
    (64, 64, 64, False, [640, 411], None, {"layout": "fused"}),
    (32, 32, 128, False, [300, 1900], [333, 1900], {}),
    # enough rows for the tiles between
    (64, 64, 64, True, [129, 1, 170], None, {}),
    (64, 64, 128, True, [129, 1, 170], [200, 1, 333], {}),
    (64, 16, 128, True, [300, 37], [400, 37], {"layout": "fused"}),
    (128, 128, 64, False, [129, 1, 170], None, {}),
    (128, 128, 128, False, [129, 1, 170], [129, 7, 300], {}),
    (256, 256, 64, False, [130, 200], None, {}),
    (256, 256, 128, False, [130, 200], None, {}),
    (64, 64, 64, False, [150, 1, 111], None, {}),                       # fp32: with short walks
    (64, 64, 128, False, [150, 1, 111], [150, 30, 300], {}),
    # fp32: .. and for the largest
    (1024, 1024, 64, False, [256], None, {}),
    (1024, 512, 128, False, [250, 6], None, {}),
    (32, 4, 128, True, [2, 1, 3, 1, 1, 5, 8, 1, 2, 1, 1, 1, 4] * 6, None, {}),  # more sequences than lanes
]


@pytest.mark.parametrize("hq,hkv,d,bf16,q_lens,k_lens,more", CASES)
def test_against_formulas(hq, hkv, d, bf16, q_lens, k_lens, more):
    import torch

    c = Case(hq, hkv, d, bf16, q_lens, k_lens, **more)
    a = c.attention()
    o, lse = c.outputs()
    c.attend(a, o, lse)
    torch.cuda.synchronize()
    check_forward(c, o, lse)
    out = c.grads()
    c.grad(a, out, o, lse)
    torch.cuda.synchronize()
    check_grads(c, out, o, lse)
    again, (o2, _) = c.grads(), c.outputs()
    c.attend(a, o2, None)  # without lse; the same bits
    c.grad(a, again, o, lse)
    assert torch.equal(o, o2)
    for x, y in zip(out, again):
        assert torch.equal(x, y)


def reference(c, q, k, v):
    o = np.zeros_like(q)
    for rq, rk, h, seen in c.parts():
        g = h // (c.hq // c.hkv)
        s = np.where(seen, c.scale * (q[rq, h] @ k[rk, g].T), -np.inf)
        some = seen.any(1)
        e = np.exp(s[some] - s[some].max(1, keepdims=True))
        o[rq, h][some] = (e / e.sum(1, keepdims=True)) @ v[rk, g]
    return o


def test_gradient_against_differences():
    """Along random directions, central differences of the 64-bit forward pass (h = 2^-13: truncation of the order
    h^2, 1.5e-8, times third derivatives of order 10 of a sum of ~1e3 terms, rounding 1e-13 / h) against the fp32
    kernel's gradients, whose error along a direction is at most the sum of its elements' bounds; those are below
    2e-5 an element here, of random signs: 1e-3 of a sum of the order 100."""
    import torch

    c = Case(6, 2, 64, False, [23, 1, 9], [40, 1, 9], tail=0)
    a = c.attention()
    o, lse = c.outputs()
    c.attend(a, o, lse)
    out = c.grads()
    c.grad(a, out, o, lse)
    torch.cuda.synchronize()
    x, up, g = [f64(t) for t in (c.q, c.k, c.v)], f64(c.d_o), [f64(t) for t in out]
    rng = np.random.default_rng(0)
    h = 2.0 ** -13
    for i in range(3):
        for _ in range(4):
            way = rng.standard_normal(x[i].shape)
            at = [[y + s * h * way if j == i else y for j, y in enumerate(x)] for s in (1, -1)]
            want = ((reference(c, *at[0]) - reference(c, *at[1])) * up).sum() / (2 * h)
            assert abs((g[i] * way).sum() - want) <= 1e-3, (i, (g[i] * way).sum(), want)


@pytest.mark.parametrize("bf16,d", [(True, 64), (True, 128), (False, 64), (False, 128)])
@pytest.mark.parametrize("copies", [1, 40, 300])
def test_unseen_infinities_and_nans(bf16, d, copies):
    """A token's infinities and NaN change nothing that does not see it: later tokens' rows in V, K, Q and d_o, rows
    behind the sequence, another sequence's, another KV head's.  With many more sequences behind, so that the
    largest tiles are taken too."""
    import torch

    q_lens, bad = [70, 45], 37  # token 37 of sequence 0, in the middle of a tile
    c = Case(4, 2, d, bf16, q_lens + [115] * (2 * (copies - 1)), tail=5)
    end = sum(c.q_lens)
    clean_o, clean_lse = c.outputs()
    a = c.attention()
    c.attend(a, clean_o, clean_lse)
    clean = c.grads()
    c.grad(a, clean, clean_o, clean_lse)
    inf, nan = float("inf"), float("nan")
    for which in ("v", "k", "q", "d_o", "tail"):
        x = {"v": c.v, "k": c.k, "q": c.q, "d_o": c.d_o}.get(which)
        if which == "tail":
            kept = [t.clone() for t in (c.q, c.k, c.v, c.d_o)]
            for t in (c.q, c.k, c.v, c.d_o):
                t[end:] = nan  # rows behind the last sequence
        else:
            kept = x.clone()
            x[bad, 1, 3] = nan
            x[bad, 1, 9] = inf
            x[bad + 1, 1, 20] = -inf
        o, lse = c.outputs()
        c.attend(a, o, lse)
        out = c.grads()
        # the gradient is given the clean outputs, so that a row is reached by what it sees alone
        c.grad(a, out, clean_o, clean_lse)
        torch.cuda.synchronize()
        if which == "tail":
            assert torch.equal(o, clean_o) and torch.equal(lse, clean_lse)
            for x, y in zip(out, clean):
                assert torch.equal(x, y)
            for t, y in zip((c.q, c.k, c.v, c.d_o), kept):
                t.copy_(y)
            continue
        heads = {"v": [2, 3], "k": [2, 3], "q": [1], "d_o": []}[which]  # of the queries that it can reach
        def reached(h, t):
            return h in heads and (bad <= t < 70 if which in "vk" else t in (bad, bad + 1))
        for t in range(115):
            for h in range(4):
                if not reached(h, t):
                    assert torch.equal(o[t, h], clean_o[t, h]), (which, t, h)
                    assert lse[t, h] == clean_lse[t, h], (which, t, h)
        if which == "v":
            assert bool(torch.isnan(o[bad:70, 2:, 3]).all()) and not bool(torch.isnan(o[bad:70, 2:, 4:9]).any())
            assert bool((o[bad:70, 2:, 9] == inf).all()) and bool((o[bad + 1:70, 2:, 20] == -inf).all())
        dq, dk, dv = out
        g = 1 if which in "vk" else 0  # KV head that it belongs to
        qh = range(2 * g, 2 * g + 2)
        for t in range(115):
            for h in range(4):
                # dq of a row: through the keys and values that it sees, its own query and gradient
                own = h == 1 and t in (bad, bad + 1)
                if not ((which in "vk" and h in qh and bad <= t < 70) or (which in ("q", "d_o") and own)):
                    assert torch.equal(dq[t, h], clean[0][t, h]), (which, "dq", t, h)
            for h in range(2):
                # dk and dv of a key: through the rows that see it (a bad key's or value's own gradient apart)
                hit = h == g and ((which in "vk" and t < 70) or (which in ("q", "d_o") and t <= bad + 1))
                if which == "v" and not (h == g and t < 70):
                    assert torch.equal(dv[t, h], clean[2][t, h]), (which, "dv", t, h)
                if not hit:
                    assert torch.equal(dk[t, h], clean[1][t, h]), (which, "dk", t, h)
                    assert torch.equal(dv[t, h], clean[2][t, h]), (which, "dv", t, h)
        # what v and k reach ends with the rows that see them: rows before take dk and dv of their own
        if which == "d_o":
            assert not bool(torch.isnan(dv[bad + 2:70, 0]).any()) and bool(torch.isnan(dv[:bad + 1, 0, 3]).all())
        x.copy_(kept)


def test_scores_of_infinity():
    """Keys whose scores are -inf weigh nothing; a row of nothing else is NaN with lse -inf."""
    import torch

    c = Case(1, 1, 64, False, [40], tail=0)
    c.q[:, 0] = 0.0
    c.q[:, 0, 0] = 1.0
    c.k[:, 0] = 0.0
    c.k[:5, 0, 0] = -float("inf")
    a = c.attention()
    o, lse = c.outputs()
    c.attend(a, o, lse)
    assert bool(torch.isnan(o[:5]).all()) and bool((lse[:5] == -float("inf")).all())
    want = torch.cumsum(c.v[5:, 0].double(), 0) / torch.arange(1, 36, device="cuda")[:, None]
    assert float((o[5:, 0].double() - want).abs().max()) < 1e-5  # 35 terms of about 1, fp32
    assert float((lse[5:, 0].double() - torch.log(torch.arange(1, 36, device="cuda").double())).abs().max()) < 1e-6


def test_offsets_that_do_not_ascend_touch_nothing_else():
    """Offsets out of range or order: no fault, rows outside every clamped sequence stay."""
    import torch

    c = Case(2, 1, 64, True, [20, 20, 20], tail=40)
    a = c.attention()
    for off in ([0, 30, 10, 60], [-5, 20, 40, 60], [0, 20, 1000000, 60], [70, 60, 50, 40], [0, -100, -7, 2]):
        c.q_off = torch.tensor(off, dtype=torch.int32, device="cuda")
        for k_off in (None, torch.tensor([5, 4, 1 << 30, -1], dtype=torch.int32, device="cuda")):
            c.shared, c.k_off = k_off is None, k_off
            o, lse = c.outputs()
            c.attend(a, o, lse)
            out = c.grads()
            c.grad(a, out, o, lse)
            torch.cuda.synchronize()
            inside = [max(0, min(x, c.tq)) for x in off]
            last = max(inside)
            assert bool((o[last:] == 7).all()) and bool((out[0][last:] == 7).all())


def test_no_sequences_and_no_queries():
    import torch

    c = Case(2, 1, 64, True, [0, 0], [5, 9], tail=2)
    a = c.attention()
    o, lse = c.outputs()
    c.attend(a, o, lse)
    out = c.grads()
    c.grad(a, out, o, lse)
    a.attend(0, c.tq, None, c.rows(c.q, o), c.rows(c.k), c.rows(c.v), lse, k_tokens=c.tk, k_offsets=c.k_off)
    assert bool((o == 7).all()) and bool((lse == 7).all()) and bool((out[0] == 7).all())
    for x in out[1:]:
        assert bool((x[:14] == 0).all()) and bool((x[14:] == 7).all())


def test_graph_streams_and_two_attentions():
    """Captured on a stream of its own, replayed with other rows and other offsets of as many sequences; eager calls
    of another attention between the replays."""
    import torch

    c = Case(4, 2, 128, True, [90, 40, 70], tail=0)
    side = torch.cuda.Stream()
    a, b = c.attention(side), c.attention()
    o, lse = c.outputs()
    out = c.grads()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        c.attend(a, o, lse)
        c.grad(a, out, o, lse)
    for i, lens in enumerate(([90, 40, 70], [1, 198, 1], [0, 100, 100], [66, 67, 67])):
        gen = torch.Generator().manual_seed(50 + i)
        for x in (c.q, c.k, c.v, c.d_o):
            x.copy_(torch.randn(x.shape, generator=gen).to(x.dtype))
        c.q_lens = c.k_lens = lens
        c.q_off.copy_(torch.tensor(starts(lens), dtype=torch.int32))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        eo, el = c.outputs()
        c.attend(b, eo, el)
        eg = c.grads()
        c.grad(b, eg, eo, el)
        torch.cuda.synchronize()
        assert torch.equal(o, eo) and torch.equal(lse, el)
        for x, y in zip(out, eg):
            assert torch.equal(x, y)
        check_forward(c, eo, el)


@pytest.mark.parametrize("bf16,d", [(True, 64), (True, 128), (False, 64), (False, 128)])
@pytest.mark.parametrize("copies", [1, 5, 20])
def test_infinities_of_a_last_token(bf16, d, copies):
    """An infinite gradient of a sequence's last token reaches dv of every key as that infinity (p is above 0 for scores
    as near as these), also where the rows of the sequence end inside a tile; other elements of dv stay finite, other
    sequences' and KV heads' as they were.  With more sequences behind, so that every tile of keys is taken."""
    import torch

    lens = [300, 155]
    c = Case(16, 8, d, bf16, lens * copies, tail=2)
    a = c.attention()
    o, lse = c.outputs()
    c.attend(a, o, lse)
    clean = c.grads()
    c.grad(a, clean, o, lse)
    inf = float("inf")
    starts_of = starts(c.q_lens)
    bad = [0, len(c.q_lens) - 1]  # sequences
    for i in bad:
        c.d_o[int(starts_of[i + 1]) - 1, 5, 9] = inf     # KV head 2
        c.d_o[int(starts_of[i + 1]) - 1, 4, 21] = -inf
    out = c.grads()
    c.grad(a, out, o, lse)
    torch.cuda.synchronize()
    hit = torch.zeros(c.tk, dtype=torch.bool, device="cuda")
    for i in bad:
        hit[int(starts_of[i]):int(starts_of[i + 1])] = True
    dv = out[2]
    assert bool((dv[hit, 2, 9] == inf).all()), int(torch.isnan(dv[hit, 2, 9]).sum())
    assert bool((dv[hit, 2, 21] == -inf).all())
    rest = [e for e in range(d) if e not in (9, 21)]
    # what is finite is the same sum, of which the second pass may add some elements in another order
    want, got = clean[2][hit, 2][:, rest].double(), dv[hit, 2][:, rest].double()
    assert bool(torch.isfinite(got).all())
    assert float((got - want).abs().max()) <= (2.0 ** -8 if bf16 else 2.0 ** -18) * float(want.abs().max())
    others = [h for h in range(8) if h != 2]
    assert torch.equal(dv[:, others], clean[2][:, others]) and torch.equal(dv[~hit], clean[2][~hit])
    assert torch.equal(out[1][:, others], clean[1][:, others]) and torch.equal(out[1][~hit], clean[1][~hit])
