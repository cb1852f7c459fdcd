"""Calls of the adjusted logits' gradient whose rows get in one another's way; no GPU."""
import pytest

from tests.test_decode_tail_refusals_cpu import _grad, sats  # noqa: F401


@pytest.mark.parametrize("f32", [False, True])
def test_gradient_over_logits_of_other_strides(sats, f32):  # noqa: F811
    """The logits begin where the gradient that comes in does, with rows further apart: rows that are written are logits of others."""
    s = sats
    es = 4 if f32 else 2
    at = 0x300000
    assert _grad(s, f32=f32, z=at, ld=128, dout=at, ld_dout=64, out=at, ld_out=64) == s.EINVAL
    assert _grad(s, f32=f32, z=at, ld=64, dout=at, ld_dout=128, out=at, ld_out=128) == s.EINVAL
    # elsewhere than dout, but over the logits' second row
    assert _grad(s, f32=f32, z=at, ld=256, dout=at, ld_dout=64, out=at + 250 * es, ld_out=256) == s.EINVAL
