"""The checks and refusals of routing, scatter, combine, quantisation and products of 8-bit
integers under AddressSanitizer and UndefinedBehaviorSanitizer (host code only; no GPU)."""
from tests import test_sanitizers


def test_refusals_under_asan_and_ubsan(monkeypatch):
    monkeypatch.setattr(test_sanitizers, "SUITES", ["tests/test_experts_cpu.py"])
    test_sanitizers.test_cpu_suites_under_asan_and_ubsan()
