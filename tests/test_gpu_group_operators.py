"""GPU: rotary positions, scores, carried-over and forked responses together, as a group decode uses them.

Two iterations of a sample stream: the first stops after some completions and hands out the responses it
would discard, the second takes them in and finishes them.  Every step's rows are rotated to their
positions, every step's attention is checked against the 64-bit attention over the rotated rows, every
step's log probabilities against the 64-bit ones.  Tolerances of the attention are the decode's own
(1e-5 in fp32, 1e-2 in bf16, as everywhere in these tests)."""

import numpy as np
import pytest

from paper_2506_22950_amd import infs
from paper_2506_22950_amd.group import decode_group, probe_group
from tests.test_gpu_rotary import rotated
from tests.test_gpu_score import Ref, close
from tests.test_rotary import config

pytestmark = pytest.mark.gpu

L, HQ, HKV, M, G, V = 2, 4, 2, 4, 10, 5003


class Group:
    def __init__(self, bf16, d, plen, probe=0):
        import torch

        self.bf16, self.d, self.plen = bf16, d, plen
        self.dt = torch.bfloat16 if bf16 else torch.float32
        self.ctx = infs.Context(infs.make_config(
            num_layers=L, num_q_heads=HQ, num_kv_heads=HKV, head_dim=d, num_prompts=1, slots_per_prompt=M,
            samples_per_prompt=G, max_prompt_len=64, max_suffix_len=64, dtype=infs.BF16 if bf16 else infs.F32,
            probe_tokens=probe), stream=torch.cuda.current_stream())
        self.rotary = infs.Rotary(config(head_dim=d, rotary_dim=d, scaling=infs.ROTARY_YARN, factor=4.0))
        self.f, self.amp = self.rotary.frequencies()
        self.gen = torch.Generator().manual_seed(5)
        self.history = {}  # sample -> per layer lists of (k, v) float64 rows [HKV, d]

    def rows(self, *shape):
        import torch

        return torch.randn(*shape, generator=self.gen).to(self.dt).cuda()

    def turned(self, x, pos):
        """Rotated rows as the kernel stores them: checked elsewhere, taken from it here."""
        y = x.clone()
        n, h = x.shape[0], x.shape[1]
        import torch

        self.rotary.rotate_rows(infs.BF16 if self.bf16 else infs.F32, n, infs.rotary_rows(y, y, h),
                                positions=torch.tensor(pos, dtype=torch.int32, device="cuda"),
                                stream=torch.cuda.current_stream())
        want, mag = rotated(x.double().cpu().numpy(), pos, self.f, self.amp, infs.ROTARY_HALF, self.d)
        got = y.double().cpu().numpy()
        assert np.all(np.abs(got - want) <= mag * 2.0 ** -20 + np.abs(want) * (2.0 ** -8 if self.bf16 else 2.0 ** -24) + 1e-30)
        return got

    def prefill(self):
        self.prefix = []
        for layer in range(L):
            k, v = self.rows(self.plen, HKV, self.d), self.rows(self.plen, HKV, self.d)
            turned = self.turned(k, list(range(self.plen)))
            import torch

            self.ctx.prefill_shared(0, layer, self.plen, torch.from_numpy(turned).to(self.dt).cuda(), v)
            torch.cuda.synchronize()
            self.prefix.append((turned, v.double().cpu().numpy()))

    def attend(self, layer, sample, q):
        k = np.concatenate([self.prefix[layer][0], np.stack([x[0] for x in self.history[sample][layer]])])
        v = np.concatenate([self.prefix[layer][1], np.stack([x[1] for x in self.history[sample][layer]])])
        out = np.empty((HQ, self.d))
        for h in range(HQ):
            s = k[:, h // (HQ // HKV)] @ q[h] / np.sqrt(self.d)
            p = np.exp(s - s.max())
            out[h] = (p / p.sum()) @ v[:, h // (HQ // HKV)]
        return out

    def check_step(self, live, q, k, v, o):
        """live: (slot, sample, position of its token); raw rows q, k, v [L, n, H, d]; o: outputs."""
        for layer in range(L):
            for s, i, pos in live:
                tk = self.turned(k[layer, s:s + 1], [pos])[0]
                self.history.setdefault(i, [[] for _ in range(L)])[layer].append((tk, v[layer, s].double().cpu().numpy()))
                ref = self.attend(layer, i, self.turned(q[layer, s:s + 1], [pos])[0])
                err = np.abs(o[layer, s].double().cpu().numpy() - ref).max()
                assert err <= (1e-2 if self.bf16 else 1e-5), (layer, s, i, pos, err)


@pytest.mark.parametrize("entry", ["decode_step", "decode_step_layers"])
@pytest.mark.parametrize("bf16,d,plen", [(False, 64, 21), (True, 128, 40), (True, 64, 0)])
def test_two_iterations_of_a_stream(bf16, d, plen, entry):
    import torch

    g = Group(bf16, d, plen)
    lengths = [[3, 40, 7, 25, 12, 33, 5, 9, 20, 2]]
    scorer = infs.Scorer(infs.make_scorer_config(vocab=V, dtype=infs.BF16 if bf16 else infs.F32, max_rows=M, top_k=3),
                         stream=torch.cuda.current_stream())
    log, raw, scored = [], {}, {}

    def provide(step, layer):
        if step not in raw:
            q, k, v = g.rows(L, M, HQ, d), g.rows(L, M, HKV, d), g.rows(L, M, HKV, d)
            raw[step] = (q, k, v, q.clone(), k.clone(), torch.zeros(L, M, HQ, d, device="cuda"))
        q, k, v, q2, k2, o = raw[step]
        return q2[layer], k2[layer], v[layer], o[layer]  # rotated in place: the copies

    def logits(step):
        z = (torch.randn(M, V, generator=g.gen) * 3).to(g.dt).cuda()
        t = torch.randint(-1, V, (M,), generator=g.gen, dtype=torch.int32).cuda()
        out = dict(logprob=torch.empty(M, device="cuda"), entropy=torch.empty(M, device="cuda"),
                   top_id=torch.empty(M, 3, dtype=torch.int32, device="cuda"), top_logprob=torch.empty(M, 3, device="cuda"))
        scored[step] = (z, t, out)
        return scored[step]

    def after(step):
        torch.cuda.synchronize()
        q, k, v, _, _, o = raw.pop(step)
        g.check_step([(s, e[1], plen + e[2] - 1) for s, e in enumerate(log[step]) if e], q, k, v, o)
        z, t, out = scored.pop(step)
        z64, tok = z.double().cpu().numpy(), t.cpu().numpy()
        ref = Ref(z64, tok, 1.0)
        close(out["logprob"], ref.lp_t, ref.lp_err)
        close(out["entropy"], ref.h, ref.h_err)
        assert np.array_equal(out["top_id"].cpu().numpy(), np.argsort(-z64, axis=1, kind="stable")[:, :3])

    carried, kept = {}, {}

    def unfinished(left):
        bufs = [[torch.empty(L, n, HKV, d, dtype=g.dt, device="cuda") for _, _, _, n in left] for _ in range(2)]
        g.ctx.export_responses([x[0] for x in left], *bufs)
        for (_, p, i, n), k, v in zip(left, *bufs):
            carried[p, i] = (n, k, v)
            kept[i] = n

    g.prefill()
    accepted = []
    common = dict(after_step=after, entry=entry, rotary=g.rotary, scorer=scorer, logits=logits, log=log)
    decode_group(g.ctx, [infs.Sched(G, M, "fifo")], lengths, L, provide, stop_after=4, accepted=accepted,
                 unfinished=unfinished, **common)
    assert len(accepted[0]) == 4 and len(carried) >= 2
    # the second iteration: the finished samples are gone, the carried ones resume
    g.ctx.reset()
    for layer in range(L):
        g.ctx.prefill_shared(0, layer, plen, *[torch.from_numpy(x).to(g.dt).cuda() for x in g.prefix[layer]])
    torch.cuda.synchronize()
    order = [i for i in range(G) if i not in accepted[0]]
    renamed = {j: i for j, i in enumerate(order)}
    log.clear()
    history, g.history = g.history, {}
    for j, i in renamed.items():
        if i in kept:
            g.history[j] = [h[:kept[i]] for h in history[i]]
            assert len(g.history[j][0]) == kept[i]
    second = [[lengths[0][i] for i in order] + [1] * (G - len(order))]
    done = []
    decode_group(g.ctx, [infs.Sched(G, M, "fifo")], second, L, provide, accepted=done,
                 carried={(0, j): carried[0, i] for j, i in renamed.items() if (0, i) in carried}, **common)
    assert sorted(done[0]) == list(range(G))
    for j in range(len(order)):
        assert len(g.history[j][0]) == second[0][j]
    g.ctx.sync()
    g.ctx.destroy()


@pytest.mark.parametrize("entry", ["probe_step", "probe_step_layers"])
def test_probe_phase_with_rotary_positions(entry):
    import torch

    d, plen, k_probe = 64, 18, 3
    g = Group(False, d, plen, probe=k_probe)
    g.prefill()
    lengths = [[5, 2, 9, 4, 3, 7, 1, 6, 8, 2]]
    raw, plog = {}, []

    def provide(step, p, first, n, layer):
        if step not in raw:
            q, k, v = g.rows(L, n, HQ, d), g.rows(L, n, HKV, d), g.rows(L, n, HKV, d)
            raw[step] = (q, k, v, q.clone(), k.clone(), torch.zeros(L, n, HQ, d, device="cuda"))
        q, k, v, q2, k2, o = raw[step]
        return q2[layer].data_ptr(), k2[layer].data_ptr(), v[layer].data_ptr(), o[layer].data_ptr()

    steps = probe_group(g.ctx, lengths, k_probe, L, provide, log=plog, entry=entry, rotary=g.rotary)
    torch.cuda.synchronize()
    for step in range(steps):
        q, k, v, _, _, o = raw[step]
        g.check_step([(j, e[1], plen + e[2] - 1) for j, e in enumerate(plog[step]) if e], q, k, v, o)
    g.ctx.sync()
    g.ctx.destroy()


@pytest.mark.parametrize("bf16", [False, True])
def test_branches_score_and_go_on(bf16):
    # a sample forks at several lengths; the branches decode with positions of their own
    import torch

    d, plen = 128 if bf16 else 64, 11
    g = Group(bf16, d, plen)
    g.prefill()
    g.ctx.refill_slot(0, 0, 0)
    live = {0: 0}
    length = {0: 0}

    def step():
        q, k, v = g.rows(L, M, HQ, d), g.rows(L, M, HKV, d), g.rows(L, M, HKV, d)
        q2, k2, o = torch.empty_like(q), torch.empty_like(k), torch.zeros(L, M, HQ, d, device="cuda")
        g.ctx.rotate_step(g.rotary, infs.rotary_rows(q, q2, HQ), infs.rotary_rows(k, k2, HKV), num_layers=L)
        g.ctx.decode_step_layers(q2, k2, v, o)
        g.ctx.end_step()
        torch.cuda.synchronize()
        g.check_step([(s, i, plen + length[i]) for s, i in live.items()], q, k, v, o)
        for i in live.values():
            length[i] += 1

    for _ in range(35):
        step()
    at = {1: 35, 2: 32, 3: 7}
    g.ctx.fork_slots([0, 0, 0], [1, 2, 3], [1, 2, 3], [at[i] for i in (1, 2, 3)])
    for i, n in at.items():
        g.history[i] = [h[:n] for h in g.history[0]]
        live[i], length[i] = i, n
    for n in range(20):
        if n == 5:
            g.ctx.retire_slot(0)
            del live[0]
        step()
    g.ctx.sync()
    g.ctx.destroy()
