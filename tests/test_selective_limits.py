"""Host-only checks of what the short convolution and the selective scan take and refuse at the edges of their range."""
import ctypes
import os
import re
import struct
import subprocess

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


def _device_code(path):
    """The code objects for the GPU inside a library: bundles of a count, then offset, size and name of each."""
    data, at, magic = open(path, "rb").read(), 0, b"__CLANG_OFFLOAD_BUNDLE__"
    while (at := data.find(magic, at)) >= 0:
        here = at + 24
        count, = struct.unpack_from("<Q", data, here)
        here += 8
        for _ in range(count if count < 16 else 0):
            offset, size, n = struct.unpack_from("<3Q", data, here)
            if data[here + 24:here + 24 + n].startswith(b"hip") and size:
                yield data[at + offset:at + offset + size]
            here += 24 + n
        at += 24


def _registers(operand):
    m = re.match(r"-?\|?v(\d+)$|-?\|?v\[(\d+):(\d+)\]$", operand.strip().rstrip("|"))
    return range(0) if not m else range(int(m[1]), int(m[1]) + 1) if m[1] else range(int(m[2]), int(m[3]) + 1)


def test_other_lanes_registers_are_waited_for(tmp_path):
    """In the scan's kernels as they are built: two instructions, or a wait as long, between what writes a register and what reads
    another lane's place of it (DPP forms, swaps of halves and quarters); the compiler does not see into inline assembly."""
    tool = "/opt/rocm/llvm/bin/llvm-objdump"
    if not os.path.exists(tool):
        pytest.skip("no disassembler")
    la.load_library()
    code = [c for c in _device_code(binding.library_path()) if b"k_selective_back" in c]
    assert len(code) == 1
    (tmp_path / "code.o").write_bytes(code[0])
    text = subprocess.run([tool, "-d", "--no-show-raw-insn", str(tmp_path / "code.o")], check=True, capture_output=True, text=True).stdout
    written, now, seen = {}, 0, 0
    for line in text.splitlines():
        m = re.match(r"\s+(\w+)\s*([^/]*)", line)
        if not m:
            written = {}  # another function, or a label
            continue
        op, operands = m[1], m[2].split(",")
        now += 1
        swap = op.startswith("v_permlane") and "swap" in op
        if swap or op.endswith("_dpp") or " row_" in m[2] or "quad_perm" in m[2]:
            seen += 1
            for r in [*_registers(operands[0]), *_registers(operands[1])] if swap else _registers(operands[1].split(" ")[1]):
                assert now - written.get(r, -9) > 2, line
        if op == "s_nop":
            now += int(operands[0], 0)
        elif op.startswith("v_"):
            for r in [*_registers(operands[0]), *(_registers(operands[1]) if swap else ())]:
                written[r] = now
    assert seen > 10000


@pytest.mark.parametrize("value", [1 << 32, (1 << 32) + 1, -(1 << 40), 1 << 70])
def test_constants_beyond_32_bits_are_refused(value):
    """What a C int would cut off to a constant that there is."""
    D = lambda *s, t=torch.bfloat16: _stand_in(torch.zeros(*s, dtype=t))  # noqa: E731
    F = torch.float32
    x, y, w, A, B, h = D(2, 8, 16), D(2, 8, 16), D(16, 4, t=F), D(16, 4, t=F), D(2, 8, 4), D(2, 16, 4, t=F)
    for call in (lambda: la.la_conv_forward(x, w, None, None, y, None, None, value), lambda: la.la_conv_step(x, w, None, D(2, 3, 16), y, value),
                 lambda: la.la_conv_backward(x, w, None, None, y, None, D(2, 8, 16), None, None, None, None, value, None),
                 lambda: la.la_selective_forward(x, x, A, B, B, None, None, None, y, None, None, None, value, None),
                 lambda: la.la_selective_backward(x, x, A, B, B, None, None, D(1 << 16, t=torch.uint8), y, None, *(D(2, 8, 16) for _ in range(2)), None, D(2, 8, 4),
                                                  D(2, 8, 4), None, None, None, None, value, None),
                 lambda: la.la_selective_step(x, x, A, B, B, None, None, h, y, value)):
        with pytest.raises(ValueError, match="constants"):
            call()
