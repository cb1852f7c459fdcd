"""More refusals of the vocabulary operators: answered by the host checks, with no CUDA call made."""
import pytest
import torch


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


@pytest.mark.parametrize("f32", [False, True])
def test_gradient_rows_over_logits_rows(sats, f32):
    # logits [5][8] in rows of 20 elements; a gradient `at` elements behind them in rows of 20 touches them unless it
    # begins 8 to 12 elements behind a row of theirs, or nothing of it lies where they are.  (Without a GPU what is not refused fails to
    # launch.)
    s, es, z = sats, 4 if f32 else 2, 0x100000
    tail = "_f32" if f32 else ""
    grad = getattr(s.lib(), "sats_distill_grad" + tail)
    both = getattr(s.lib(), "sats_distill_loss_grad" + tail)

    def refused(T, ld, at, ld_d):
        d = z + at * es
        a = grad(z, ld, T, 8, None, None, 0, 0x4000, 1.0, 0.0, 0x5000, None, d, ld_d, None, None)
        b = both(z, ld, T, 8, None, None, 0, 0x4000, 1.0, 0.0, None, 0x5000, d, ld_d, None, None)
        assert a == b and a in (s.EINVAL, s.ECUDA, s.OK)
        return a == s.EINVAL

    def touches(T, ld, at, ld_d):
        mine = {i * ld + k for i in range(T) for k in range(8)}
        return any(at + i * ld_d + k in mine for i in range(T) for k in range(8))

    if torch.cuda.is_available():
        pytest.skip("what is not refused would be launched")
    for T in (2, 5):
        for at in range(-120, 121):
            if at != 0:
                assert refused(T, 20, at, 20) == touches(T, 20, at, 20), (T, at)
    assert not refused(5, 20, 0, 20) and refused(5, 20, 0, 21) and refused(5, 20, 8, 21)
    assert refused(1, 20, 7, 20) and not refused(1, 20, 8, 20) and not refused(1, 20, 0, 31)
