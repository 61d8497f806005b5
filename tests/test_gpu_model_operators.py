"""GPU: norms, rotary positions, attention over prompts, decoding, the choice of tokens, their scores and all gradients
together, as a group and its learner use them: a small model with normed heads reads its prompts, decodes two groups
of samples (with and without a probe phase), each token the one that was chosen from the step before, and learns from
them in one packed batch.  The same model in 64 bits takes the same tokens.

Tolerances (fp32, every weight matrix scaled so that its products keep the size of their inputs, h of size 1 and below
4).  A step's attention is within 1e-5 (as everywhere in these tests), every product of 64 or 256 terms within 256 *
2^-24 = 1.6e-5 of its terms' size, so an element of h errs by at most 3 such terms a layer and their effect through
the layer behind it: 2 * 3 * 1.6e-5 * 2 = 2e-4.  Logits are sums of 64 elements times weights of size 1/8, of random
signs: 2e-4 again.  A log probability is a logit less ln of their mean weight: 4e-4.
Gradients: each is a sum of at most 400 tokens' terms with relative errors of that size (2e-4 of the largest terms, of
random signs), against the largest element, which is such a sum too: 2e-3 of it."""

import numpy as np
import pytest

from paper_2506_22950_amd import infs
from paper_2506_22950_amd.group import decode_group, prefill_prompts, probe_group
from tests.test_gpu_choose import define
from tests.test_rotary import config

pytestmark = pytest.mark.gpu

L, D, HQ, HKV, HD, V, M, G, EPS = 2, 64, 4, 2, 64, 301, 3, 5, 1e-6
PROMPTS, LENGTHS = [11, 37], [[3, 20, 1, 7, 12], [5, 2, 9, 16, 4]]


class Model:
    """Weights in fp32 (device) and the same in 64 bits (host)."""

    def __init__(self, seed):
        import torch

        gen = torch.Generator().manual_seed(seed)

        def matrix(n, m):
            return torch.randn(n, m, generator=gen) / n ** 0.5

        host = {"emb": torch.randn(V, D, generator=gen), "out": matrix(D, V)}
        for layer in range(L):
            host.update({f"q{layer}": matrix(D, HQ * HD), f"k{layer}": matrix(D, HKV * HD), f"v{layer}": matrix(D, HKV * HD),
                         f"o{layer}": matrix(HQ * HD, D) / 2})
        host["wq"], host["wk"] = (1 + 0.3 * torch.randn(L, HD, generator=gen) for _ in range(2))
        self.w = {n: x.cuda() for n, x in host.items()}
        self.w64 = {n: x.double() for n, x in host.items()}
        self.norms = infs.make_norms(self.w["wq"], self.w["wk"], infs.F32, EPS, HD)

    def rows(self, h, layer):
        w, n = self.w, h.shape[0]
        return [(h @ w[f"{x}{layer}"]).view(n, heads, HD) for x, heads in (("q", HQ), ("k", HKV), ("v", HKV))]

    def logits64(self, tokens, lens, freq, leaves=None):
        """Logits of packed sequences, in 64 bits on the host."""
        import torch

        w = leaves or self.w64
        pos = torch.cat([torch.arange(n) for n in lens]).double()
        angle = pos[:, None] * torch.from_numpy(freq)[None]
        cos, sin = angle.cos()[:, None], angle.sin()[:, None]

        def turned(x, weight):
            x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * weight
            a, b = x[..., :HD // 2], x[..., HD // 2:]
            return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

        h = w["emb"][tokens]
        for layer in range(L):
            q, k, v = [(h @ w[f"{x}{layer}"]).view(-1, heads, HD) for x, heads in (("q", HQ), ("k", HKV), ("v", HKV))]
            q, k = turned(q, w["wq"][layer]), turned(k, w["wk"][layer])
            k, v = (x.repeat_interleave(HQ // HKV, 1) for x in (k, v))
            outs, at = [], 0
            for n in lens:
                a, b, c = (x[at:at + n].transpose(0, 1) for x in (q, k, v))
                s = (a @ b.transpose(1, 2)) / HD ** 0.5
                s = s.masked_fill(torch.ones(n, n).triu(1).bool(), -torch.inf)
                outs.append((s.softmax(-1) @ c).transpose(0, 1).reshape(n, HQ * HD))
                at += n
            h = h + torch.cat(outs) @ w[f"o{layer}"]
        return h @ w["out"]


@pytest.mark.parametrize("probe", [0, 2])
def test_group_and_learner(probe):
    import torch

    m = Model(seed=probe + 1)
    stream = torch.cuda.current_stream()
    ctx = infs.Context(infs.make_config(
        num_layers=L, num_q_heads=HQ, num_kv_heads=HKV, head_dim=HD, num_prompts=2, slots_per_prompt=M, samples_per_prompt=G,
        max_prompt_len=64, max_suffix_len=64, dtype=infs.F32, probe_tokens=probe), stream=stream)
    rotary = infs.Rotary(config())
    freq, _ = rotary.frequencies()
    sampler = infs.Sampler(infs.make_sampler_config(vocab=V, dtype=infs.F32, max_rows=2 * M), stream=stream)
    scorer = infs.Scorer(infs.make_scorer_config(vocab=V, dtype=infs.F32, max_rows=512), stream=stream)
    attention = infs.Attention(infs.make_attention_config(
        num_q_heads=HQ, num_kv_heads=HKV, head_dim=HD, dtype=infs.F32, max_tokens=512), stream=stream)
    gen = torch.Generator().manual_seed(9)
    prompts = [torch.randint(0, V, (n,), generator=gen) for n in PROMPTS]
    draw = torch.rand(2, G, 64, generator=gen, dtype=torch.float32)
    plain = infs.make_sampling()

    # the prompts
    state = {"h": m.w["emb"][torch.cat(prompts).cuda()]}
    T = sum(PROMPTS)

    def prompt_rows(layer):
        if layer:
            state["h"] = state["h"] + state["o"].view(T, -1) @ m.w[f"o{layer - 1}"]
        state["rows"], state["o"] = m.rows(state["h"], layer), torch.zeros(T, HQ, HD, device="cuda")
        return (*state["rows"], state["o"])

    offsets = torch.tensor([0, PROMPTS[0], T], dtype=torch.int32, device="cuda")
    positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in PROMPTS]).cuda()
    prefill_prompts(ctx, PROMPTS, L, prompt_rows, attention, offsets, rotary, m.norms, positions)
    h = state["h"] + state["o"].view(T, -1) @ m.w[f"o{L - 1}"]
    z = h[[PROMPTS[0] - 1, T - 1]] @ m.w["out"]  # each prompt's last token: what its samples begin with
    want = m.logits64(torch.cat(prompts), PROMPTS, freq)[[PROMPTS[0] - 1, T - 1]]
    assert (z.double().cpu() - want).abs().max() <= 4e-4

    tokens = [[[] for _ in range(G)] for _ in range(2)]    # chosen tokens, the first from the prompt
    logprobs = [[[] for _ in range(G)] for _ in range(2)]

    def choose(z, who):
        """One token for every row of z, row r for sample who[r] (None: nobody)."""
        n = z.shape[0]
        u = torch.tensor([draw[w[0], w[1], len(tokens[w[0]][w[1]])] if w else 0.5 for w in who]).cuda()
        token, logprob = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
        return z, u, dict(token=token, logprob=logprob, sampling=plain)

    def take(z, u, out, who):
        for r, w in enumerate(who):
            if w:
                t = define(z[r].double().cpu().numpy(), float(u[r]))
                assert int(out["token"][r]) == t[0]
                tokens[w[0]][w[1]].append(t[0])
                logprobs[w[0]][w[1]].append(float(out["logprob"][r]))

    for i in range(G):
        who = [(0, i), (1, i)]
        z, u, out = choose(z, who)
        sampler.sample(2, z, u, **out)
        take(z, u, out, who)

    # a step of `who`: the embeddings of their last tokens go in
    now = {}

    def step_rows(layer, who):
        if layer == 0:
            now["h"] = torch.stack([m.w["emb"][tokens[w[0]][w[1]][-1]] if w else torch.zeros(D, device="cuda") for w in who])
        else:
            now["h"] = now["h"] + now["o"].view(len(who), -1) @ m.w[f"o{layer - 1}"]
        now["rows"], now["o"] = m.rows(now["h"], layer), torch.zeros(len(who), HQ, HD, device="cuda")
        return (*now["rows"], now["o"])

    def step_logits(who):
        h = now["h"] + now["o"].view(len(who), -1) @ m.w[f"o{L - 1}"]
        return choose(h @ m.w["out"], who)

    if probe:
        now["who"] = None

        def probe_rows(step, p, first, n, layer):
            if layer == 0:
                now["who"] = [(p, first + j) if len(tokens[p][first + j]) <= min(probe, LENGTHS[p][first + j]) else None
                              for j in range(n)]
            return step_rows(layer, now["who"])

        def probe_chosen(step):
            z, u, out = step_logits(now["who"])
            sampler.sample(len(now["who"]), z, u, **out)
            take(z, u, out, now["who"])

        # (a probe step's samples are those that have drawn as many tokens as it has fed)
        probe_group(ctx, LENGTHS, probe, L, probe_rows, rotary=rotary, norms=m.norms, after_step=probe_chosen)
        assert all(len(tokens[p][i]) == min(probe, LENGTHS[p][i]) + 1 for p in range(2) for i in range(G))

    log, last = [], {}

    def rows(step, layer):
        last["who"] = [e[:2] if e else None for e in log[step]]
        return step_rows(layer, last["who"])

    def draws(step):
        last["drawn"] = step_logits(last["who"])
        return last["drawn"]

    scored = torch.empty(2 * M, device="cuda")

    def logits(step):  # what was just chosen, scored: the same log probability
        z, _, out = last["drawn"]
        return z, out["token"], dict(logprob=scored)

    def after(step):
        torch.cuda.synchronize()
        take(*last["drawn"], last["who"])
        got, want = scored.cpu().numpy(), last["drawn"][2]["logprob"].cpu().numpy()
        assert np.all(np.abs(got - want) <= 2e-5 * (1 + np.abs(want)))

    decode_group(ctx, [infs.Sched(G, M, "fifo") for _ in range(2)], LENGTHS, L, rows, log=log, after_step=after, reuse=probe,
                 rotary=rotary, norms=m.norms, sampler=sampler, draws=draws, scorer=scorer, logits=logits)
    ctx.sync()
    ctx.destroy()
    assert all(len(tokens[p][i]) == LENGTHS[p][i] + 1 for p in range(2) for i in range(G))

    # the learner's batch: every sample behind its prompt, packed; the loss is the mean log probability of its tokens
    who = [(p, i) for p in range(2) for i in range(G)]
    seqs = [torch.cat([prompts[p], torch.tensor(tokens[p][i])]) for p, i in who]
    fed, lens = torch.cat([s[:-1] for s in seqs]), [len(s) - 1 for s in seqs]
    # a row's target is the token behind it; the prompts' own are not scored
    target = torch.cat([torch.cat([torch.full((PROMPTS[p] - 1,), -1), torch.tensor(tokens[p][i])]) for p, i in who])
    n = len(fed)
    assert len(target) == n == sum(lens)
    w = m.w
    t_dev, target_dev = fed.cuda(), target.int().cuda()
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()
    positions = torch.cat([torch.arange(x, dtype=torch.int32) for x in lens]).cuda()
    kept, h = [], w["emb"][t_dev]

    def r(x, out=None):
        return infs.rotary_rows(x, out, x.shape[1])

    for layer in range(L):
        q, k, v = m.rows(h, layer)
        tq, tk, o = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
        lse = torch.empty(n, HQ, device="cuda")
        rotary.norm_rotate_rows(infs.F32, n, infs.layer_norms(m.norms, layer), r(q, tq), r(k, tk), positions=positions,
                                stream=stream)
        attention.attend(len(lens), n, offsets, r(tq, o), r(tk), r(v), lse)
        kept.append((h, q, k, v, tq, tk, o, lse))
        h = h + o.view(n, -1) @ w[f"o{layer}"]
    z = h @ w["out"]
    logprob, stats = torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
    scorer.score(n, z, target_dev, logprob, stats=stats)
    got = logprob.cpu().numpy()
    sampled = np.concatenate([np.concatenate([np.zeros(PROMPTS[p] - 1), logprobs[p][i]]) for p, i in who])
    leaves = {name: x.clone().requires_grad_() for name, x in m.w64.items()}
    z64 = m.logits64(fed, lens, freq, leaves)
    lp64 = z64.log_softmax(-1).gather(1, target.clamp(min=0)[:, None])[:, 0] * (target >= 0)
    assert np.abs(got - lp64.detach().numpy()).max() <= 4e-4
    assert np.abs(sampled - lp64.detach().numpy()).max() <= 4e-4
    count = int((target >= 0).sum())
    (lp64.sum() / count).backward()

    d_z = torch.empty_like(z)
    scorer.grad(n, z, target_dev, stats, torch.full((n,), 1.0 / count, device="cuda"), d_z)
    grads = {"out": h.T @ d_z, "wq": torch.empty(L, HD, device="cuda"), "wk": torch.empty(L, HD, device="cuda")}
    d_h = d_z @ w["out"].T
    workspace = torch.empty(infs.norm_rotate_grad_workspace(n, HD), dtype=torch.uint8, device="cuda")
    for layer in reversed(range(L)):
        h, q, k, v, tq, tk, o, lse = kept[layer]
        grads[f"o{layer}"] = o.view(n, -1).T @ d_h
        d_o = (d_h @ w[f"o{layer}"].T).view(n, HQ, HD)
        d_tq, d_tk, d_v, d_q, d_k = (torch.empty_like(x) for x in (q, k, v, q, k))
        attention.grad(len(lens), n, offsets, r(tq, d_tq), r(tk, d_tk), r(v, d_v), r(o), r(d_o), lse)
        rotary.norm_rotate_grad(infs.F32, n, infs.layer_norms(m.norms, layer), r(q, d_q), r(k, d_k), r(d_tq), r(d_tk),
                                grads["wq"][layer], grads["wk"][layer], workspace, positions=positions, stream=stream)
        for name, x in (("q", d_q), ("k", d_k), ("v", d_v)):
            grads[f"{name}{layer}"] = h.T @ x.view(n, -1)
            d_h = d_h + x.view(n, -1) @ w[f"{name}{layer}"].T
    grads["emb"] = torch.zeros_like(w["emb"]).index_add_(0, t_dev, d_h)
    for name, leaf in leaves.items():
        err, top = (grads[name].double().cpu() - leaf.grad).abs().max().item(), leaf.grad.abs().max().item()
        assert err <= 2e-3 * top, (name, err, top)
    for x in (attention, scorer, sampler):
        x.destroy()
