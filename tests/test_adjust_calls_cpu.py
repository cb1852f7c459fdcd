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


def test_only_ids_that_count_are_read():
    """A row without settings need not have a history behind it, nor one with a short history more ids: every read of ids comes
    after the row's length is known, which is 0 where the settings are off, and is bounded by it."""
    import os
    import re
    from paper_2607_08991_gb300 import build
    with open(os.path.join(build.CSRC, "adjust.cu")) as f:
        text = f.read()
    kernel = text[text.index("adjust_kernel(const __grid_constant__"):text.index("// ------------------------------------------------------------------ host")]
    known = kernel.index("freq == 0.f) len = 0;")
    reads = [m.start() for m in re.finditer(r"load_ids\(|vectors4 \+", kernel)]
    assert len(reads) >= 3 and min(reads) > known
    assert "p.L" not in kernel[known:]
    assert re.findall(r"load_ids\(.*?, (\w+)\)", kernel[known:]) == ["len"] * 2
