"""GPU: launches that start on another XCD than the context knows.  The start that the context knows is made
wrong again and again, so that every work-group of the next launches takes that path: outputs stay, bit for
bit, what the exchange through the coherence point gives, nothing is reported, and the launch tells the
context the start it had."""

import numpy as np
import pytest

from paper_2506_22950_amd import infs
from tests.gpu_harness import check_against_oracle, run_gpu_group
from workload import Workload, get_config

pytestmark = pytest.mark.gpu


def group():
    return get_config("qwen3_1p7b_g64").with_(layers=3, prompt_lens=(300,), samples_per_prompt=16,
                                              length_dist=("lognormal", 3.0, 0.5, 1, 40), max_suffix_len=40,
                                              pool_rows=None)


def misled(monkeypatch, every):
    """Every `every` steps: wait for the work, look at the start, put another one in its place."""
    seen = {"wrong": [], "after": [], "steps": 0}

    def patched(end):
        def f(ctx):
            end(ctx)
            if ctx.exchange_start() < 0:  # the harness plans its steps on a dry-run context
                return
            seen["steps"] += 1
            if seen["steps"] % every == 0:
                ctx.sync()
                start = ctx.exchange_start()
                seen["after"].append(start)
                wrong = (start + 1 + seen["steps"] % 7) % 8
                ctx.set_exchange_start(wrong)
                assert ctx.exchange_start() == wrong
                seen["wrong"].append(wrong)
        return f

    monkeypatch.setattr(infs.Context, "end_step", patched(infs.Context.end_step))
    monkeypatch.setattr(infs.Context, "end_probe_step", patched(infs.Context.end_probe_step))
    return seen


@pytest.mark.parametrize("every", [1, 6])  # 6: launches queue up behind the changed start
@pytest.mark.parametrize("entry,probe_entry,reuse", [
    ("decode_step_layers", "probe_step_layers", 0), ("decode_step", "probe_step", 0), ("decode_step_static", "probe_step", 0),
    ("decode_step_layers", "probe_step_layers", 4), ("decode_step", "probe_step", 4)])
def test_launches_find_another_start(monkeypatch, entry, probe_entry, reuse, every):
    cfg = group()
    wl = Workload(cfg)
    probes = [{}, {}]
    capture = lambda step: step % 6 == 5 or every == 1  # noqa: E731
    # mode 0 has the same split, so that both give the same bits
    plain = run_gpu_group(cfg, "sjf", wl=wl, entry=entry, probe_entry=probe_entry, reuse=reuse, exchange=0, capture=capture,
                          probe=probes[0])
    seen = misled(monkeypatch, every)
    _, log, _, cap, _, _ = run_gpu_group(cfg, "sjf", wl=wl, entry=entry, probe_entry=probe_entry, reuse=reuse, exchange=1,
                                         capture=capture, probe=probes[1])
    assert len(cap) > 5 and cap.keys() == plain[3].keys()
    for k in cap:
        assert np.array_equal(cap[k], plain[3][k]), k
    if reuse:
        for j, o in probes[0]["captured"].items():
            assert np.array_equal(o, probes[1]["captured"][j]), j
    # the wrong start was replaced by the launches' own, which hardly ever is the wrong one by chance
    replaced = [a != w for a, w in zip(seen["after"][1:], seen["wrong"])]
    assert len(replaced) >= 5 and sum(replaced) >= len(replaced) - 2, (seen["after"], seen["wrong"])
    check_against_oracle(cfg, wl, log, {k: cap[k] for k in list(cap)[::7]})


def test_start_is_an_xcd():
    import torch
    from paper_2506_22950_amd.group import context_for

    ctx = context_for(group(), stream=torch.cuda.current_stream())
    assert 0 <= ctx.exchange_start() < 8
    for bad in (-1, 8, 1 << 30):
        with pytest.raises(infs.InfsError) as e:
            ctx.set_exchange_start(bad)
        assert e.value.status == infs.E_ARG
    ctx.destroy()
