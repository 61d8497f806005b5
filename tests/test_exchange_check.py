"""The agreement of a launch's work-groups on the XCD of the first one (csrc/plan.h), on the host:
tests/exchange_check.cpp is built with g++ against the header alone and plays launches whose work-groups
all start elsewhere, in part, or stray one by one; only those that agree may leave nothing behind.
And the host side of the start that a context knows."""

import os
import shutil
import subprocess

import pytest

from paper_2506_22950_amd import infs
from paper_2506_22950_amd.group import context_for
from workload import get_config

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2506_22950_amd", "csrc")


def test_agreement_on_the_start(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "exchange_check")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-Wall",
                        "-Wextra", "-Werror", "-I" + CSRC, os.path.join(HERE, "exchange_check.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe, "20000"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "failures 0" in r.stdout, r.stdout + r.stderr


def test_no_start_without_an_exchange():
    ctx = context_for(get_config("tiny_f32"), dry_run=True)
    assert ctx.exchange_start() == -1
    for start, want in ((0, infs.E_STATE), (7, infs.E_STATE), (-1, infs.E_ARG)):
        with pytest.raises(infs.InfsError) as e:
            ctx.set_exchange_start(start)
        assert e.value.status == want
    ctx.destroy()
