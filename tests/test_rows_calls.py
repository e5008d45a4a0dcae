"""More of what the calls on rows refuse on the host (nothing is launched: the device addresses are made up)."""
import ctypes

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
