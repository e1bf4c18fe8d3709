"""Host-only checks of what the short convolution and the selective scan take and refuse at the edges of their range."""
import pytest
import torch

import paper_2510_21956_amd as la
from paper_2510_21956_amd import binding
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
