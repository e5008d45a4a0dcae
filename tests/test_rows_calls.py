"""More of what the calls on rows do on the host: what they refuse and what they ask of the runtime (nothing is launched: the device addresses are made up)."""
import ctypes
import os
import subprocess
import sys

import pytest

import paper_1801_02108_amd as sb

P = ctypes.c_void_p


def at(k, bytes_in=0):
    return P(0x7f0000000000 + (k << 28) + bytes_in)


X, RES, SUM, Y, GAIN, COUNT, W, WS, DG = (at(k) for k in range(9))
ROWS, C, COUT = 4 * 9, 64, 32


def norm(count, total=SUM, y=Y):
    return sb.lib().sbnet_rms_norm_on_tiles(X, RES, sb.BF16, count, 4, 9, C, GAIN, 1e-6, total, y, None)


def norm_i8(count):
    return sb.lib().sbnet_rms_norm_i8_on_tiles(X, RES, sb.BF16, count, 4, 9, C, GAIN, 1e-6, SUM, Y, WS, None)


def quantize(count):
    return sb.lib().sbnet_quantize_i8_on_tiles(X, sb.BF16, count, 4, 9, C, Y, WS, None)


def backward(count):
    return sb.lib().sbnet_rms_norm_backward_on_tiles(X, RES, SUM, sb.BF16, count, 4, 9, C, GAIN, 1e-6, Y, DG, W, 1 << 20, None)


def pointwise(count):
    return sb.lib().sbnet_pointwise_i8_on_tiles(X, WS, count, 4, 9, C, W, GAIN, None, COUT, 0, sb.BF16, Y, None)


STACK = ROWS * C * 2                              # bytes of a bf16 stack
HELD = [
    ("norm, the first word of y", norm, at(3)), ("norm, the last word of y", norm, at(3, STACK - 4)), ("norm, in sum", norm, at(2, 128)),
    ("norm codes, in sum", norm_i8, at(2, STACK - 4)), ("norm codes, in codes", norm_i8, at(3, 64)), ("norm codes, in scales", norm_i8, at(7, 4 * ROWS - 4)),
    ("quantiser, in codes", quantize, at(3, ROWS * C - 4)), ("quantiser, in scales", quantize, at(7)),
    ("gradients, in dx", backward, at(3, 4)), ("gradients, in dgain", backward, at(8, 4 * C - 4)), ("gradients, in the workspace", backward, at(6)),
    ("product, the first word of out", pointwise, at(3)), ("product, the last word of out", pointwise, at(3, ROWS * COUT * 2 - 4)),
]


@pytest.mark.parametrize("k", range(len(HELD)), ids=lambda k: HELD[k][0].replace(" ", "_"))
def test_a_count_inside_what_a_call_writes_is_refused(k):
    _, call, count = HELD[k]
    assert call(count) == sb.EINVAL
    text = sb.lib().sbnet_last_error().decode()
    assert "count" in text or "out overlaps an input" in text, text


RECORDER = """
#include <stdio.h>
int hipFuncSetAttribute(const void *f, int attribute, int value) { printf("%p %d %d\\n", f, attribute, value); fflush(stdout); return 0; }
int hipLaunchKernel(void) { return 0; }
int hipGetLastError(void) { return 0; }
"""
CHILD = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
P, I = ctypes.c_void_p, ctypes.c_int
call = lib.sbnet_pointwise_i8_on_tiles
call.argtypes = [P, P, P, I, I, I, P, P, P, I, I, I, P, P]
a = [0x7f0000000000 + (k << 32) for k in range(6)]
for cout in (64, 512, 128, 40):
    assert call(a[0], a[1], a[2], 200, 256, 256, a[3], a[4], None, cout, 0, 1, a[5], None) == 0
"""


def test_layers_of_one_kernel_ask_for_the_same_lds(tmp_path):
    """The amount is an attribute of the kernel, so that of a layer must not be what another thread's layer sets between.  The runtime's calls are
    taken by a recorder: no device is touched."""
    (tmp_path / "recorder.c").write_text(RECORDER)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-o", str(tmp_path / "recorder.so"), str(tmp_path / "recorder.c")])
    env = dict(os.environ, HIP_VISIBLE_DEVICES="", ROCR_VISIBLE_DEVICES="")
    r = subprocess.run([sys.executable, "-c", CHILD, str(tmp_path / "recorder.so"), sb.LIB_PATH], env=env, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr
    calls = [line.split() for line in r.stdout.splitlines()]
    assert len(calls) == 4 and len(set(map(tuple, calls))) == 1, r.stdout
    assert int(calls[0][2]) == 160 * 1024
