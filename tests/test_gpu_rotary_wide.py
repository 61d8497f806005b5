"""GPU: rotary positions of tokens with more units of work than a work-group has threads, so that its
wavefronts go round: every kind of unit, both layouts, both types, up to the most heads (the check and
its tolerance are those of test_gpu_rotary.py)."""

import pytest

from paper_2506_22950_amd import infs
from tests.test_gpu_rotary import test_rows as check_rows

pytestmark = pytest.mark.gpu

HALF, PAIRS = infs.ROTARY_HALF, infs.ROTARY_INTERLEAVED


@pytest.mark.parametrize("T,hq,hk,d,rd,layout,bf16", [
    # 16 bytes of first and 16 of second elements: 320, 576, 2048 units a token
    (1, 32, 8, 128, 128, HALF, True), (300, 32, 8, 128, 128, HALF, True), (5, 32, 4, 128, 128, HALF, False),
    (3, 96, 32, 256, 256, HALF, True),
    # the same with a rest behind the rotated part: 40 heads of 12 units
    (37, 32, 8, 128, 64, HALF, True),
    # 16 bytes of a head whose partners lie in other chunks: 640 and 1280 units
    (1, 32, 8, 128, 100, HALF, True), (300, 32, 8, 128, 100, HALF, True), (7, 32, 8, 128, 6, HALF, False),
    (3, 33, 9, 120, 100, HALF, True),  # heads of 15 chunks: lanes without work
    # neighbouring pairs: 1152 units, by 512 and by 256 threads
    (5, 64, 8, 128, 128, PAIRS, True), (300, 64, 8, 128, 128, PAIRS, True), (300, 64, 8, 128, 96, PAIRS, False),
    # elements: 3600 and 2400 units
    (3, 40, 8, 100, 50, HALF, True), (3, 40, 8, 75, 50, PAIRS, False),
    # the most heads
    (2, 4096, 4096, 16, 16, HALF, True), (2, 4096, 4096, 16, 6, HALF, True), (1, 4096, 4096, 16, 16, PAIRS, True),
    (1, 4096, 4096, 7, 2, HALF, False)])
def test_wide_tokens(T, hq, hk, d, rd, layout, bf16):
    check_rows(T, hq, hk, d, rd, layout, bf16)
