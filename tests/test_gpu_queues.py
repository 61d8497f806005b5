"""Streams beside the context's own: the hardware queue of a stream may change while the stream is
idle, and with it the XCD of a launch's first work-group.  Work-groups stay round robin over the XCDs,
so the XCD-local exchange of partials stays valid; results agree with the oracle, in either entry."""

import pytest

from tests.gpu_harness import check_against_oracle, run_gpu_group
from workload import Workload, get_config

pytestmark = pytest.mark.gpu


def busy_streams(n):
    # n other streams, each with a launch of its own while the current one is idle
    import torch

    x = torch.ones(4096, device="cuda")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(n)]
    for s in streams:
        with torch.cuda.stream(s):
            x.add(1)
        s.synchronize()
    return streams


@pytest.mark.parametrize("entry", ["decode_step_layers", "decode_step", "decode_step_static"])
def test_other_streams_while_a_group_decodes(entry):
    cfg = get_config("qwen3_1p7b_g64").with_(layers=2, prompt_lens=(300,), samples_per_prompt=16,
                                             length_dist=("lognormal", 3.0, 0.5, 1, 60), max_suffix_len=60,
                                             pool_rows=None)
    wl = Workload(cfg)
    keep = []

    def inspect(ctx, step, log):
        if step % 7 == 3:
            ctx.sync()
            keep.extend(busy_streams(5))

    ctx, log, _, cap, _, _ = run_gpu_group(cfg, "sjf", wl=wl, inspect=inspect, entry=entry)
    assert len(keep) >= 10
    check_against_oracle(cfg, wl, log, {k: cap[k] for k in list(cap)[::5]})


def test_contexts_made_on_any_queue_exchange_through_the_l2():
    import torch
    from paper_2506_22950_amd.group import context_for

    cfg = get_config("qwen3_1p7b_g64").with_(layers=1, prompt_lens=(64,))
    for s in busy_streams(8):
        with torch.cuda.stream(s):
            assert context_for(cfg, stream=s).exchange_mode() == 1
