"""More refusals of the vocabulary operators: answered by the host checks, with no CUDA call made."""
import pytest


@pytest.fixture(scope="module")
def sats():
    from paper_2607_08991_gb300 import build, sats as s
    build.build_library()
    return s


def _selftest(s, z=0x100000, ld=8, T=2, V=8, labels=0x4000, loss=0x5000, d=0x200000, ld_d=8, row=0):
    return s.lib().sats_selftest_distill_timeout(z, ld, T, V, labels, loss, d, ld_d, row, None, None)


def test_selftest_of_the_distillation_waits(sats):
    s = sats
    assert _selftest(s, row=-1) == s.EINVAL and _selftest(s, row=2) == s.EINVAL and _selftest(s, T=0) == s.EINVAL
    assert _selftest(s, z=None) == s.EINVAL and _selftest(s, labels=None) == s.EINVAL
    assert _selftest(s, loss=None) == s.EINVAL and _selftest(s, d=None) == s.EINVAL and _selftest(s, ld_d=7) == s.EINVAL
    assert _selftest(s, V=2**31 - 64, ld=2**31 - 64) == s.ESHAPE
