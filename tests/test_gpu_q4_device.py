"""A handle of another GPU than the current one: refused, whatever the other arguments."""
import ctypes

import pytest
import torch

from oracle import q4
from tests.test_gpu_q4 import activations, sats, to_bf16, weights  # noqa: F401

pytestmark = pytest.mark.gpu


def test_handle_of_another_device(sats):  # noqa: F811
    q, s = weights(64, 40, 32, 1)
    w = sats.Q4(torch.from_numpy(q4.pack(q)).cuda(), to_bf16(s), 32)
    ws = sats.Q4Workspace(w, 2)
    x, y = activations(2, 64, torch.float32, 2), torch.full((2, 40), 7.0, device="cuda")
    device = ctypes.c_int.from_address(w.handle + 12)      # the handle's fourth int
    assert device.value == torch.cuda.current_device()
    device.value += 1
    try:
        with pytest.raises(sats.SatsError) as e:
            sats.q4_matmul(w, x, y, ws)
        assert e.value.status == sats.EINVAL
    finally:
        device.value -= 1
    torch.cuda.synchronize()
    assert (y == 7.0).all()
    sats.q4_matmul(w, x, y, ws)
    assert sats.get_error(ws) == sats.OK and not (y == 7.0).any()
