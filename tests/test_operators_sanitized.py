"""The checks and refusals of epilogues, grouped products and activation gradients
under AddressSanitizer and UndefinedBehaviorSanitizer (host code only; no GPU)."""
from tests import test_sanitizers


def test_refusals_under_asan_and_ubsan(monkeypatch):
    monkeypatch.setattr(test_sanitizers, "SUITES", ["tests/test_operators_cpu.py"])
    test_sanitizers.test_cpu_suites_under_asan_and_ubsan()
