"""GPU: attention whose walks over keys (or, for their gradients, over rows) several work-groups share: few rows over
many keys, and their gradients.  The bounds are those of tests/test_gpu_attend.py (sums of n terms: the joins add no
terms, and a rescaling of a part is one rounding more, within them)."""

import numpy as np
import pytest

from tests.test_gpu_attend import Case, starts
from tests.test_gpu_attend import test_against_formulas as against_formulas

pytestmark = pytest.mark.gpu

CASES = [
    (2, 1, 128, True, [1], [20001]),                       # one token, as many parts as there are
    (2, 2, 64, True, [1], [70000]),
    (4, 2, 64, False, [1, 3], [9000, 513]),                # walks of different lengths, some of one part
    (8, 1, 128, False, [1], [5000]),
    (16, 8, 128, True, [1] * 8, [4000, 5000, 1, 3000, 512, 513, 7001, 300]),
    (4, 2, 64, True, [700], None),                         # causal: rows of a tile see parts, or nothing of them
    (2, 1, 128, True, [900, 0, 40], [900, 700, 1300]),
    (6, 2, 64, False, [129, 300, 1, 77], None),
    (4, 1, 128, False, [600], None),
    (32, 1, 128, True, [150], None),                       # many rows for few keys: the keys' gradients are shared
    (4, 2, 64, True, [1000], [300]),                       # rows that see no key, ahead of those that do
    (2, 1, 64, False, [3], [9000]),
]


@pytest.mark.parametrize("hq,hkv,d,bf16,q_lens,k_lens", CASES)
def test_shared_walks_against_formulas(hq, hkv, d, bf16, q_lens, k_lens):
    against_formulas(hq, hkv, d, bf16, q_lens, k_lens, {})


@pytest.mark.parametrize("bf16,d", [(True, 64), (True, 128), (False, 64), (False, 128)])
def test_unseen_infinities_and_nans_in_parts(bf16, d):
    """A late token's NaN and infinities change nothing that does not see it, in whichever part of a walk they are."""
    import torch

    n, bad = 1500, 1131
    c = Case(4, 2, d, bf16, [n], tail=5)
    a = c.attention()
    clean_o, clean_lse = c.outputs()
    c.attend(a, clean_o, clean_lse)
    clean = c.grads()
    c.grad(a, clean, clean_o, clean_lse)
    for which in ("v", "k", "q", "d_o"):
        x = getattr(c, which)
        kept = x.clone()
        x[bad, 0, 3], x[bad, 0, 9], x[bad + 1, 0, 20] = float("nan"), float("inf"), -float("inf")
        o, lse = c.outputs()
        c.attend(a, o, lse)
        out = c.grads()
        c.grad(a, out, clean_o, clean_lse)
        torch.cuda.synchronize()
        group = [2, 3]  # heads that it does not reach at all
        assert torch.equal(o[:, group], clean_o[:, group]) and torch.equal(lse[:, group], clean_lse[:, group])
        assert torch.equal(o[:bad], clean_o[:bad]) and torch.equal(lse[:bad], clean_lse[:bad])
        dq, dk, dv = out
        assert torch.equal(dq[:, group], clean[0][:, group])
        assert torch.equal(dk[:, 1], clean[1][:, 1]) and torch.equal(dv[:, 1], clean[2][:, 1])
        assert torch.equal(dq[:bad], clean[0][:bad])
        if which in ("q", "d_o"):  # the keys behind it do not see it
            assert torch.equal(dk[bad + 2:], clean[1][bad + 2:]) and torch.equal(dv[bad + 2:], clean[2][bad + 2:])
            assert torch.equal(o[bad + 2:], clean_o[bad + 2:]) and torch.equal(dq[bad + 2:], clean[0][bad + 2:])
        if which == "v":
            assert bool(torch.isnan(o[bad:n, :2, 3]).all()) and not bool(torch.isnan(o[bad:n, :2, 4:9]).any())
            assert bool((o[bad:n, :2, 9] == float("inf")).all()) and bool((o[bad + 1:n, :2, 20] == -float("inf")).all())
        x.copy_(kept)


def test_graph_of_shared_walks():
    """Captured and replayed with other offsets, walks of other lengths: the counters are left as they were."""
    import torch

    c = Case(4, 2, 128, True, [300, 2, 5], [1500, 4000, 900], tail=0)
    side = torch.cuda.Stream()
    a, b = c.attention(side), c.attention()
    o, lse = c.outputs()
    out = c.grads()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        c.attend(a, o, lse)
        c.grad(a, out, o, lse)
    for i, (q_lens, k_lens) in enumerate((([300, 2, 5], [1500, 4000, 900]), ([1, 305, 1], [6000, 399, 1]),
                                          ([0, 1, 306], [0, 6100, 300]), ([300, 2, 5], [1500, 4000, 900]))):
        gen = torch.Generator().manual_seed(80 + i)
        for x in (c.q, c.k, c.v, c.d_o):
            x.copy_(torch.randn(x.shape, generator=gen).to(x.dtype))
        c.q_off.copy_(torch.tensor(starts(q_lens), dtype=torch.int32))
        c.k_off.copy_(torch.tensor(starts(k_lens), dtype=torch.int32))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        eo, el = c.outputs()
        c.attend(b, eo, el)
        eg = c.grads()
        c.grad(b, eg, eo, el)
        torch.cuda.synchronize()
        assert torch.equal(o[:sum(q_lens)], eo[:sum(q_lens)]) and torch.equal(lse[:sum(q_lens)], el[:sum(q_lens)])
        for x, y, n in zip(out, eg, (sum(q_lens), sum(k_lens), sum(k_lens))):
            assert torch.equal(x[:n], y[:n])


def test_two_attentions_at_once():
    """Shared walks of two attentions on two streams: each has counters and parts of its own."""
    import torch

    streams = [torch.cuda.Stream() for _ in range(2)]
    cs = [Case(8, 2, 64, True, [1, 200], [8000, 3000], seed=3 + i) for i in range(2)]
    at = [c.attention(s) for c, s in zip(cs, streams)]
    outs = [[(*c.outputs(), c.grads()) for _ in range(12)] for c in cs]
    torch.cuda.synchronize()
    for i in range(12):
        for c, a, o in zip(cs, at, outs):
            c.attend(a, o[i][0], o[i][1])
            c.grad(a, o[i][2], o[i][0], o[i][1])
    torch.cuda.synchronize()
    for o in outs:
        for x in o[1:]:
            assert torch.equal(x[0], o[0][0]) and torch.equal(x[1], o[0][1])
            assert all(torch.equal(p, q) for p, q in zip(x[2], o[0][2]))
    assert np.isfinite(outs[0][0][0].double().cpu().numpy()).all()


@pytest.mark.parametrize("q_lens,k_lens", [([70, 9], [70, 9]), ([3], [2000]), ([700], [700])])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [20, 40, 60])
def test_scores_far_out(power, d, q_lens, k_lens):
    """Keys that are 0 but for one element, which counts down from 2^power to 2^power / 2: exact scores, of which each is so far
    below the one before that a row takes its first key's value alone, and lse is that score (to fp32's rounding of a
    product with the scale).  Equal scores share.  The gradients are finite."""
    import torch

    c = Case(2, 1, d, False, q_lens, k_lens, scale=1.0, tail=0)
    m = sum(k_lens)
    c.q.zero_(), c.k.zero_()
    c.q[:, :, 5] = 2.0 ** (power - 20)
    c.k[:, 0, 5] = 2.0 ** 20 - torch.arange(m, device="cuda").float() // 2 * 256  # two of each
    a = c.attention()
    o, lse = c.outputs()
    c.attend(a, o, lse)
    out = c.grads()
    c.grad(a, out, o, lse)
    torch.cuda.synchronize()
    ks, qs = starts(k_lens), starts(q_lens)
    for i, (n, mm) in enumerate(zip(q_lens, k_lens)):
        first = c.k[ks[i], 0, 5].double().item() * 2.0 ** (power - 20)
        pair = 2 if mm > 1 and c.k[ks[i], 0, 5] == c.k[ks[i] + 1, 0, 5] else 1
        for t in range(n):
            some = min(pair, t + mm - n + 1)
            want = c.v[ks[i]:ks[i] + some, 0].double().mean(0)
            assert (o[qs[i] + t].double() - want).abs().max() <= 2.0 ** -20 * 8, (i, t)
            assert abs(lse[qs[i] + t].double() - first).max() <= abs(first) * 2.0 ** -23 + 1, (i, t)
    assert all(bool(torch.isfinite(x).all()) for x in out)


@pytest.mark.parametrize("q_len", [1, 700])
def test_offsets_beyond_32_bits(q_len):
    """A sequence whose rows begin 4.3 GB into K, V and their gradients: what the same rows give in small buffers."""
    import torch

    from paper_2506_22950_amd import infs

    h, d, m, n = 16, 128, 700, (1 << 20) + 4000
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, d_o = (torch.randn(q_len, h, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    k, v, dk, dv = (torch.empty(n, h, d, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    for x in (k, v):
        x[n - m:] = torch.randn(m, h, d, generator=gen, device="cuda").bfloat16()
    a = infs.Attention(infs.make_attention_config(num_q_heads=h, num_kv_heads=h, head_dim=d, dtype=infs.BF16, max_tokens=q_len),
                       stream=torch.cuda.current_stream())

    def rows(x, out=None):
        return infs.rotary_rows(x, out, h)

    q_off, got = torch.tensor([0, q_len], dtype=torch.int32, device="cuda"), []
    for ks, vs, dks, dvs, total in ((k, v, dk, dv, n), (k[n - m:], v[n - m:], torch.empty_like(k[:m]), torch.empty_like(k[:m]), m)):
        k_off = torch.tensor([total - m, total], dtype=torch.int32, device="cuda")
        o, lse, dq = torch.empty_like(q), torch.empty(q_len, h, device="cuda"), torch.empty_like(q)
        a.attend(1, q_len, q_off, rows(q, o), rows(ks), rows(vs), lse, k_tokens=total, k_offsets=k_off)
        a.grad(1, q_len, q_off, rows(q, dq), rows(ks, dks), rows(vs, dvs), rows(o), rows(d_o), lse, k_tokens=total,
               k_offsets=k_off)
        got.append((o, lse, dq, dks[total - m:], dvs[total - m:]))
    torch.cuda.synchronize()
    for x, y in zip(got[0][:3], got[1][:3]):
        assert torch.equal(x, y)
    assert bool(torch.isfinite(got[0][0]).all())
    # The keys' gradients take work-groups by the number of keys, another one here: the same operands (p and ds in bf16) are
    # added in another order.  Two fp32 sums of q_len terms differ by at most 2 q_len 2^-24 of the sum of their sizes (formed
    # here with errors of 1e-3 at most), and each is rounded to bf16 by half a step: 2 * 2^-8 of the larger.
    kf, vf, qf, uf = (x.float().transpose(0, 1).contiguous() for x in (k[n - m:], v[n - m:], q, d_o))
    o, lse = got[0][0].float().transpose(0, 1).contiguous(), got[0][1].t().contiguous()
    seen = torch.ones(q_len, m, device="cuda").tril(m - q_len).bool()
    s = torch.bmm(qf, kf.transpose(1, 2).contiguous()) / d ** 0.5
    p = (s - lse[..., None]).exp() * seen
    ds = p * (torch.bmm(uf, vf.transpose(1, 2).contiguous()) - (uf * o).sum(-1, keepdim=True))
    sizes = (torch.bmm(ds.abs().transpose(1, 2).contiguous(), qf.abs()) / d ** 0.5,
             torch.bmm(p.transpose(1, 2).contiguous(), uf.abs()))
    for x, y, size in zip(got[0][3:], got[1][3:], sizes):
        bound = 2 * q_len * 2.0 ** -24 * 1.01 * size.transpose(0, 1) + 2.0 ** -7 * torch.maximum(x.float().abs(), y.float().abs())
        assert bool(((x.float() - y.float()).abs() <= bound).all())


@pytest.mark.parametrize("d", [64, 128])
def test_gradient_of_far_scores(d):
    """What the gradient's p is off by where scores lie far from 0: sequences of one token, whose only weight is 1, read off dv
    = p d_o.  Scores are one product (exact).  Roundings of 2^-24 of the exponent each: in lse the score times the scale, the
    base of its exponential (taken off again by the sum's logarithm) and the sum of both; here scale log2(e) and the base:
    5 2^-24 < 2^-21, so p is within a factor of e^(|lse| 2^-21), and 2^-21 for the exponential and the products.  Beyond
    2^26 powers of 2 (where lse's base is exact: 3 2^-24) it is lowered by 2^-21 of the exponent: below 2^-20.  o is p v / p:
    three roundings."""
    import torch

    n, scale = 2000, 0.3
    c = Case(1, 1, d, False, [1] * n, scale=scale, tail=0)
    c.q.zero_(), c.k.zero_()
    c.d_o.fill_(1.0)
    gen = torch.Generator().manual_seed(11)
    size = 2.0 ** (torch.rand(n, generator=gen).double() * 40 - 4)
    c.q[:, 0, 7] = (size / 1000).float().cuda()
    c.k[:, 0, 7] = (1000 * torch.randn(n, generator=gen).sign()).cuda()
    a = c.attention()
    o, lse = c.outputs()
    c.attend(a, o, lse)
    out = c.grads()
    c.grad(a, out, o, lse)
    torch.cuda.synchronize()
    far = lse[:, 0].double().abs()
    p = out[2][:, 0, 0].double()
    near = far <= 2.0 ** 26 * np.log(2.0)
    assert 1000 < int(near.sum()) < n - 100
    assert bool(((o - c.v).double().abs() <= 3.01 * 2.0 ** -24 * c.v.double().abs()).all())
    off = far[near] * 2.0 ** -21 + 2.0 ** -21
    assert bool(torch.isfinite(p).all()) and bool((p[near].log().abs() <= off).all())
    assert bool((p[~near] <= 2.0 ** -20).all())
