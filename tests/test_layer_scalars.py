"""Tensors without a dimension are no rows: refused in words like any other wrong shape."""
import pytest
import torch

import paper_2510_21956_amd as la
from test_binding import DeviceTensor


def test_scalars_are_refused():
    D = lambda t: DeviceTensor(torch.zeros((), dtype=t))
    x, byte = D(torch.float32), D(torch.uint8)
    for call in (lambda: la.la_pack_rows(x, byte, byte, la.LA_I8), lambda: la.la_unpack_rows(byte, byte, x, la.LA_I8),
                 lambda: la.la_pack_tensors([x], [byte], [byte], la.LA_I8),
                 lambda: la.la_rmsnorm_forward(x, None, None, x, None, None, None, None, None, 1e-6),
                 lambda: la.la_rmsnorm_forward(x, None, None, byte, byte, None, None, None, None, 1e-6, la.LA_I8),
                 lambda: la.la_rmsnorm_backward(x, None, None, x, x, None, x, None, None),
                 lambda: la.la_recurrence_step(x, x, x, x, la.LA_GATE_SIGMOID)):
        with pytest.raises(ValueError):
            call()
    s = torch.tensor(1.0)
    for call in (lambda: la.pack_rows(s, "int8"), lambda: la.unpack_rows(s, s, "int8", torch.float32), lambda: la.rms_norm(s),
                 lambda: la.rms_norm(s, checkpoint="int8"), lambda: la.rms_norm_quantised(s)):
        with pytest.raises(ValueError):
            call()
