"""Host-only checks of what the short convolution and the selective scan take and refuse at the edges of their range."""
import ctypes

import pytest
import torch

import paper_2510_21956_amd as la
from paper_2510_21956_amd import binding
from paper_2510_21956_amd.autograd import _rows_in_place
from test_selective_layer import _stand_in


def test_tensors_without_a_dimension_are_refused_in_words():
    x, w, A, B, none = torch.zeros(2, 8, 16), torch.zeros(16, 4), torch.zeros(16, 4), torch.zeros(2, 8, 4), torch.zeros(())
    assert binding.row_stride(none) is None and binding.row_stride(torch.zeros(3), 2) is None
    for call in (lambda: la.causal_conv(none, w), lambda: la.causal_conv(x, none), lambda: la.causal_conv(torch.zeros(16), w),
                 lambda: la.selective_scan(none, x, A, B, B), lambda: la.selective_scan(x, none, A, B, B),
                 lambda: la.selective_scan(x, x, none, B, B), lambda: la.selective_scan(x, x, A, none, B),
                 lambda: la.selective_scan(x, x, A, B, none), lambda: la.selective_scan(x, x, A, torch.zeros(4), torch.zeros(4)),
                 lambda: la.selective_scan(none, none, none, none, none)):
        with pytest.raises(ValueError):
            call()
    D = lambda *s, t=torch.bfloat16: _stand_in(torch.zeros(*s, dtype=t))  # noqa: E731
    F, none = torch.float32, _stand_in(torch.zeros((), dtype=torch.bfloat16))
    x, w, A, B = D(2, 8, 16), D(16, 4, t=F), D(16, 4, t=F), D(2, 8, 4)
    for call in (lambda: la.la_conv_forward(none, w, None, None, x, None, None, 1), lambda: la.la_conv_step(none, w, None, D(2, 3, 16), x, 1),
                 lambda: la.la_selective_forward(x, none, A, B, B, None, None, None, x, None, None, None, 1, None),
                 lambda: la.la_selective_step(none, x, A, B, B, None, None, D(2, 16, 4, t=F), x, 1),
                 lambda: la.la_selective_step(x, x, A, B, none, None, None, D(2, 16, 4, t=F), x, 1)):
        with pytest.raises(ValueError):
            call()


def test_rows_far_apart_are_copied_for_the_scan():
    """One row of every sequence of a long batch: the scan takes rows less than 2^24 elements apart, the others are copied, and
    those alone."""
    far, near = torch.empty_strided((2, 1, 16), (1 << 24, 16, 1), dtype=torch.bfloat16), torch.zeros(2, 9, 16)[:, 3:4]
    far.copy_(torch.arange(32.0).reshape(2, 1, 16))
    for t in (far, far.unflatten(2, (4, 4))):
        dims = t.dim() - 2
        assert binding.row_stride(t, dims) == binding.ROWS_APART == 1 << 24
        for copy in (binding._near(t, dims, None), _rows_in_place(t, dims, binding.ROWS_APART)):
            assert binding.row_stride(copy, dims) == 16 and torch.equal(copy, t)
        assert _rows_in_place(t, dims) is t  # the convolution reads them where they are
    assert binding._near(near, 1, None) is near and _rows_in_place(near, 1, binding.ROWS_APART) is near
    wide = torch.empty(1, 1, 1 << 24, dtype=torch.bfloat16)  # refused, not copied
    assert binding._near(wide, 1, None) is wide and binding._near(None, 1, None) is None


def test_channels_that_integers_would_pass_are_refused():
    """Numbers of channels next to 2^31, where rounding up to a workgroup's would overflow."""
    lib = la.load_library()
    p = [ctypes.c_void_p(0x10000000 + (k << 42)) for k in range(8)]
    for C in ((1 << 31) - 256, (1 << 31) - 64, (1 << 31) - 1):
        assert lib.la_conv_forward(p[0], C, p[1], None, None, p[2], None, None, 1, 1, C, 2, 1, 1, 1, None) == 2
        assert lib.la_conv_step(p[0], C, p[1], None, p[3], p[2], 1, 1, C, 2, 1, 1, 1, None) == 2
        assert lib.la_conv_backward(p[0], C, p[1], None, None, p[2], None, p[3], p[4], None, None, None, 1, 1, C, 2, 1, 1, 1, p[5], 1 << 41, None) == 2
        assert lib.la_conv_workspace_bytes(1, 1, C, 2) == 0
    assert lib.la_conv_workspace_bytes(1, 1, (1 << 31) - 257, 2) == 3 * 4 * ((1 << 31) - 257) // 256 * 256 + 256
