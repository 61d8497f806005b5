"""GPU: the choice of tokens where u falls exactly on the border between two weights.  Rows of `count` equal logits
(a power of two, so that weights, sums and u = k / count times them are exact) among masked entries, far apart: each
token is the first entry whose running sum is above u times the whole, and logprob -ln of how many are kept."""

import ctypes
import math

import numpy as np
import pytest

from paper_2506_22950_amd import infs
from tests.test_gpu_choose import Run

pytestmark = pytest.mark.gpu

WAYS = [{}, {"temperature": 0.5}, {"top_k": 3}, {"top_k": 600}, {"top_p": 0.75}, {"top_k": 4, "top_p": 0.5}, {"min_p": 0.5},
        {"top_k": 5000, "top_p": 0.5}]


def kept_of(count, way):
    n = min(count, way.get("top_k", count))
    return math.ceil(way.get("top_p", 1.0) * n)


def check(r, live, u, each):
    """live: the entries that are not masked, of every row."""
    t, k, lp = r.token.cpu().numpy(), r.kept.cpu().numpy(), r.logprob.cpu().numpy()
    for i, way in enumerate(each):
        n = kept_of(len(live[i]), way)
        want = live[i][int(u[i] * n)]
        assert (t[i], k[i]) == (want, n), (i, t[i], k[i], want, n, way)
        assert abs(lp[i] + math.log(n)) <= math.log(n) * 2.0 ** -24 + 1e-11, (i, lp[i], n)


def array_of(ways):
    import torch

    arr = (infs.Sampling * len(ways))(*[infs.make_sampling(**w) for w in ways])
    return torch.frombuffer(bytearray(ctypes.string_at(arr, ctypes.sizeof(arr))), dtype=torch.uint8).cuda()


def borders(v, seed):
    """(live entries, u) of rows of 2, 4 and 8 equal logits, one for each border."""
    rng = np.random.default_rng(seed)
    live, u = [], []
    for count in (2, 4, 8):
        at = np.sort(rng.choice(v, count, replace=False))
        if count == 2:
            at = np.array([0, min(5000, v - 1)])
        for k in range(count):
            live.append(at)
            u.append(k / count)
    return live, u


def rows_of(live, v, bf16, shift, value=3.25):
    """The rows with `shift` elements of +inf ahead of the first, and as many between them."""
    import torch

    n = len(live)
    buf = torch.full((n * (v + shift) + shift,), math.inf, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    z = buf[shift:].view(n, v + shift)
    z[:, :v] = -math.inf
    for i, at in enumerate(live):
        z[i, torch.from_numpy(at).cuda()] = value
    return z


@pytest.mark.parametrize("shift", [0, 3])
@pytest.mark.parametrize("v,bf16", [(9, False), (1003, True), (50257, False), (50257, True), (151936, True), (151936, False)])
def test_borders(v, bf16, shift):
    import torch

    live, u = borders(v, v + shift)
    z, ut = rows_of(live, v, bf16, shift), torch.tensor(u, device="cuda")
    for way in WAYS:
        r = Run(z, ut, vocab=v, row_stride=v + shift, sampling=infs.make_sampling(**way))
        check(r, live, u, [way] * len(u))
    each = [WAYS[i % len(WAYS)] for i in range(len(u))]
    check(Run(z, ut, vocab=v, row_stride=v + shift, each=array_of(each)), live, u, each)
    for i in (1, 5, 9):  # a row alone, in as many pieces as fill the GPU
        check(Run(z[i:i + 1], ut[i:i + 1], vocab=v, row_stride=v + shift), live[i:], u[i:], [{}])


@pytest.mark.parametrize("bf16", [True, False])
def test_borders_in_the_longest_rows(bf16):
    """More pieces than threads: a thread joins several, some of them masked throughout."""
    import torch

    v = 1 << 24
    live = [np.array([0, 4097, 9000, v // 2 + 5]), np.array([40000, v // 3, v - 4097, v - 1])]
    z = rows_of(live, v, bf16, 0)
    for k in range(4):
        u = [k / 4] * 2
        check(Run(z, torch.tensor(u, device="cuda")), live, u, [{}] * 2)


def test_masked_batches_weigh_nothing():
    """A token is written whatever u is, and never one of the masked entries: all u of 1/1024 steps over equal and
    unequal weights, of which the smallest are below 2^-200 of the largest."""
    import torch

    v, n = 70001, 1024
    u = torch.arange(n, device="cuda") / n
    for values in ([0.0, 0.0, 0.0, 0.0], [0.0, -200.0, 0.0, -400.0], [-0.5, 0.25, -1.0, 2.0]):
        z = torch.full((v,), -math.inf)
        at = [300, 20000, 45001, 70000]
        for i, x in zip(at, values):
            z[i] = x
        w = np.exp(np.array(values) - max(values))
        sums = np.cumsum(w)
        r = Run(z.cuda().expand(n, v).contiguous(), u)
        t = r.token.cpu().numpy()
        slack = 1e-12 if np.abs(w - np.round(w)).max() > 1e-80 else 0.0  # sums of ones are exact
        for i in range(n):
            allowed = {at[min(int((sums <= i / n * sums[-1] + d).sum()), 3)] for d in (-slack, 0.0, slack)}
            assert int(t[i]) in allowed, (values, i, t[i], allowed)
        assert (r.kept.cpu().numpy() == 4).all()


def test_rows_with_reserved_set():
    """What a call refuses for all rows is no token for one of them."""
    import torch

    v, n = 1003, 6
    live, u = [np.array([7, 900])] * n, [0.5] * n
    ways = [WAYS[i] for i in (0, 2, 4, 0, 2, 4)]
    each = array_of(ways)
    words = each.view(torch.int32).view(n, -1)
    words[3:, -1] = 1  # reserved, the last of a row's parameters
    r = Run(rows_of(live, v, True, 0), torch.tensor(u, device="cuda"), each=each)
    t, k, lp = r.token.cpu().numpy(), r.kept.cpu().numpy(), r.logprob.cpu().numpy()
    assert (t[3:] == -1).all() and (k[3:] == 0).all() and np.isnan(lp[3:]).all(), (t, k, lp)
    r.token, r.kept, r.logprob = r.token[:3], r.kept[:3], r.logprob[:3]
    check(r, live, u, ways[:3])


def test_first_entries_after_other_calls():
    """u = 0 without a filter, row by row, on a sampler whose rows were listed and summed by the call before: the first
    entry of any weight, whatever that call left in the workspace."""
    import torch

    from tests.test_gpu_choose import define, logits

    v, n = 50257, 6
    z, u, z64 = logits(n, v, True, 12, masked=70)
    z[:, :3] = -math.inf
    z64[:, :3] = -np.inf
    s = infs.Sampler(infs.make_sampler_config(vocab=v, dtype=infs.BF16, max_rows=n), stream=torch.cuda.current_stream())
    for before in ({"top_p": 0.9}, {"top_k": 900}, {"top_k": 900, "top_p": 0.9}):
        Run(z, u, sampler=s, each=array_of([before] * n)).check(z64, before)
        r = Run(z, torch.zeros(n, device="cuda"), sampler=s, each=array_of([{}] * n))
        assert (r.token == 3).all() and (r.kept == v - 73).all()
        assert all(define(row, 0.0)[0] == 3 for row in z64)
