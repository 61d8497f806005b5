"""The host side of norms, packed attention and the choice of tokens under AddressSanitizer and
UndefinedBehaviorSanitizer: their refusal suites run again against the sanitized build (see
test_host_sanitizers.py)."""

import pytest

from tests import test_host_sanitizers_operators as operators

pytestmark = pytest.mark.sanitize

SUITES = ["tests/test_norm.py", "tests/test_attend.py", "tests/test_choose.py"]


def test_model_operators_under_asan_and_ubsan(monkeypatch):
    monkeypatch.setattr(operators, "SUITES", SUITES)
    operators.test_operators_under_asan_and_ubsan()
