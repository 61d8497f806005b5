"""GPU: scores and gradients of rows at the borders of what the calls take: tokens outside the vocabulary in
masked rows."""

import numpy as np
import pytest

from paper_2506_22950_amd import infs

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
