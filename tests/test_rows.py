"""The calls on the rows of tile stacks without a GPU: what the C entry points and the binding refuse on the host, and the
oracle's functions pinned to torch's float64 autograd, to differences and to fixed values."""
import ctypes

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import oracle as orc
import paper_1801_02108_amd as sb

P = ctypes.c_void_p
A = 0x7f0000000000                 # fake, aligned device addresses, 256 MB apart: nothing is launched
B, C_, D, E, F_ = (P(A + k * (1 << 28)) for k in range(1, 6))
A = P(A)


def off(p, n):
    return P(p.value + n)


def last_error():
    return sb.lib().sbnet_last_error().decode()


def norm(x=A, res=None, dt=sb.BF16, count=B, cap=4, pixels=9, C=64, gain=None, eps=1e-6, total=None, y=D):
    return sb.lib().sbnet_rms_norm_on_tiles(x, res, dt, count, cap, pixels, C, gain, eps, total, y, None)


def norm_i8(x=A, res=None, dt=sb.BF16, count=B, cap=4, pixels=9, C=64, gain=None, eps=1e-6, total=None, codes=D, scales=E):
    return sb.lib().sbnet_rms_norm_i8_on_tiles(x, res, dt, count, cap, pixels, C, gain, eps, total, codes, scales, None)


def quantize(x=A, dt=sb.BF16, count=B, cap=4, pixels=9, C=64, codes=D, scales=E):
    return sb.lib().sbnet_quantize_i8_on_tiles(x, dt, count, cap, pixels, C, codes, scales, None)


def backward(s=A, dy=B, dsum=None, dt=sb.BF16, count=C_, cap=4, pixels=9, C=64, gain=None, eps=1e-6, dx=D, dgain=E, ws=F_,
             ws_bytes=1 << 20):
    return sb.lib().sbnet_rms_norm_backward_on_tiles(s, dy, dsum, dt, count, cap, pixels, C, gain, eps, dx, dgain, ws, ws_bytes, None)


def weights(w=A, dt=sb.BF16, cin=64, cout=32, codes=D, scales=E):
    return sb.lib().sbnet_quantize_weights_i8(w, dt, cin, cout, codes, scales, None)


def pointwise(codes=A, scales=B, count=C_, cap=4, pixels=9, pitch=64, w=D, ws=E, bias=None, cout=32, relu=0, dt=sb.BF16, out=F_):
    return sb.lib().sbnet_pointwise_i8_on_tiles(codes, scales, count, cap, pixels, pitch, w, ws, bias, cout, relu, dt, out, None)


NAN, INF = float("nan"), float("inf")
REFUSED = [
    (norm, dict(x=None), sb.EINVAL, "null"), (norm, dict(y=None), sb.EINVAL, "null"), (norm, dict(count=None), sb.EINVAL, "null"),
    (norm, dict(dt=sb.U8), sb.EUNSUPPORTED, "dtype"), (norm, dict(cap=-1), sb.EINVAL, "sizes"),
    (norm, dict(pixels=0), sb.EINVAL, "sizes"), (norm, dict(C=0), sb.EINVAL, "sizes"),
    (norm, dict(C=32769), sb.EUNSUPPORTED, "32768"), (norm, dict(cap=1 << 20, pixels=1 << 11), sb.EUNSUPPORTED, "rows"),
    (norm, dict(eps=0.0), sb.EINVAL, "eps"), (norm, dict(eps=-1e-6), sb.EINVAL, "eps"), (norm, dict(eps=NAN), sb.EINVAL, "eps"),
    (norm, dict(eps=INF), sb.EINVAL, "eps"),
    (norm, dict(res=C_), sb.EINVAL, "together"), (norm, dict(total=C_), sb.EINVAL, "together"),
    (norm, dict(x=off(A, 1)), sb.EINVAL, "aligned"), (norm, dict(gain=off(E, 2)), sb.EINVAL, "aligned"),
    (norm, dict(count=off(B, 2)), sb.EINVAL, "aligned"), (norm, dict(y=off(A, 16)), sb.EINVAL, "overlap"),
    (norm, dict(res=C_, total=D, y=D), sb.EINVAL, "overlap"), (norm, dict(res=C_, total=off(C_, 128)), sb.EINVAL, "overlap"),
    (norm, dict(res=C_, total=off(D, 2)), sb.EINVAL, "overlap"), (norm, dict(gain=D), sb.EINVAL, "gain"), (norm, dict(eps=1e-39), sb.EINVAL, "eps"),
    (norm_i8, dict(gain=off(E, 64)), sb.EINVAL, "gain"), (norm_i8, dict(gain=D), sb.EINVAL, "gain"), (norm_i8, dict(res=C_, total=F_, gain=F_), sb.EINVAL, "gain"),
    (backward, dict(gain=E), sb.EINVAL, "gain"), (backward, dict(gain=off(D, 8)), sb.EINVAL, "gain"), (backward, dict(gain=F_), sb.EINVAL, "gain"),
    (norm, dict(res=C_, total=E, y=off(C_, 4 * 9 * 64 * 2 - 2)), sb.EINVAL, "overlap"),
    (norm_i8, dict(codes=None), sb.EINVAL, "null"), (norm_i8, dict(scales=None), sb.EINVAL, "null"),
    (norm_i8, dict(eps=0.0), sb.EINVAL, "eps"), (norm_i8, dict(codes=A), sb.EINVAL, "overlap"), (norm_i8, dict(scales=D), sb.EINVAL, "overlap"),
    (norm_i8, dict(res=C_, total=D), sb.EINVAL, "overlap"), (norm_i8, dict(scales=off(E, 1)), sb.EINVAL, "aligned"),
    (norm_i8, dict(res=C_, total=E, scales=off(E, 4)), sb.EINVAL, "overlap"),
    (quantize, dict(x=None), sb.EINVAL, "null"), (quantize, dict(dt=sb.U8), sb.EUNSUPPORTED, "dtype"),
    (quantize, dict(C=40000), sb.EUNSUPPORTED, "32768"), (quantize, dict(scales=off(A, 32)), sb.EINVAL, "overlap"),
    (backward, dict(dy=None), sb.EINVAL, "null"), (backward, dict(ws=None), sb.EINVAL, "null"), (backward, dict(dgain=None), sb.EINVAL, "null"),
    (backward, dict(ws_bytes=64 * 4 - 1), sb.EINVAL, "workspace"), (backward, dict(ws=off(F_, 2)), sb.EINVAL, "aligned"),
    (backward, dict(dx=off(A, 2)), sb.EINVAL, "overlap"), (backward, dict(dx=off(B, 128)), sb.EINVAL, "overlap"),
    (backward, dict(dgain=off(A, 4)), sb.EINVAL, "overlap"), (backward, dict(ws=E), sb.EINVAL, "overlap"),
    (backward, dict(ws=off(D, 4)), sb.EINVAL, "overlap"), (backward, dict(eps=0.0), sb.EINVAL, "eps"),
    (backward, dict(dt=sb.U8), sb.EUNSUPPORTED, "dtype"), (backward, dict(C=32769), sb.EUNSUPPORTED, "32768"),
    (weights, dict(w=None), sb.EINVAL, "null"), (weights, dict(cin=0), sb.EINVAL, "sizes"), (weights, dict(cin=131057), sb.EUNSUPPORTED, "131056"),
    (weights, dict(codes=off(D, 8)), sb.EINVAL, "aligned"), (weights, dict(codes=off(A, 64)), sb.EINVAL, "overlap"),
    (weights, dict(dt=sb.U8), sb.EUNSUPPORTED, "dtype"),
    (pointwise, dict(scales=None), sb.EINVAL, "null"), (pointwise, dict(ws=None), sb.EINVAL, "null"), (pointwise, dict(out=None), sb.EINVAL, "null"),
    (pointwise, dict(pitch=72), sb.EUNSUPPORTED, "multiple of 16"), (pointwise, dict(pitch=131072), sb.EUNSUPPORTED, "131056"),
    (pointwise, dict(pitch=0), sb.EINVAL, "sizes"), (pointwise, dict(cout=0), sb.EINVAL, "sizes"), (pointwise, dict(pixels=-1), sb.EINVAL, "sizes"),
    (pointwise, dict(dt=sb.U8), sb.EUNSUPPORTED, "dtype"), (pointwise, dict(codes=off(A, 8)), sb.EINVAL, "aligned"),
    (pointwise, dict(out=off(F_, 8)), sb.EINVAL, "aligned"), (pointwise, dict(w=off(D, 4)), sb.EINVAL, "aligned"),
    (pointwise, dict(bias=off(F_, 1 << 20 | 2)), sb.EINVAL, "aligned"), (pointwise, dict(out=A), sb.EINVAL, "overlap"),
    (pointwise, dict(out=D), sb.EINVAL, "overlap"), (pointwise, dict(bias=F_), sb.EINVAL, "overlap"),
    (pointwise, dict(cap=1 << 16, pixels=1 << 15), sb.EUNSUPPORTED, "rows"),
    (pointwise, dict(cout=(1 << 26) + 1), sb.EUNSUPPORTED, "output channels"), (weights, dict(cout=(1 << 31) - 1), sb.EUNSUPPORTED, "output channels"),
]


@pytest.mark.parametrize("k", range(len(REFUSED)), ids=lambda k: "%s-%s" % (REFUSED[k][0].__name__, "-".join(REFUSED[k][1])))
def test_what_the_entry_points_refuse_on_the_host(k):
    call, args, code, text = REFUSED[k]
    assert call(**args) == code and text in last_error(), last_error()


def test_an_empty_stack_is_no_error_and_launches_nothing():
    for call in (norm, norm_i8, quantize, pointwise):
        assert call(cap=0) == sb.OK
    assert norm(cap=0, x=None, y=None) == quantize(cap=0, x=None, codes=None, scales=None) == sb.OK      # ... nor needs memory
    assert norm_i8(cap=0, x=None, codes=None, scales=None) == pointwise(cap=0, codes=None, scales=None, out=None) == sb.OK


def test_workspace_of_the_norm_gradient_is_one_row_of_sums_for_each_workgroup():
    f = sb.lib().sbnet_rms_norm_backward_workspace_bytes
    assert f(-1, 4, 8) == f(4, 0, 8) == f(4, 4, 0) == 0
    assert f(1, 1, 64) >= 64 * 4 and f(0, 4, 64) > 0
    assert f(1000, 256, 64) % (64 * 4) == 0 and f(1000, 256, 64) <= 4096 * 64 * 4 and f(1 << 20, 2000, 64) <= 4096 * 64 * 4


def fake(*shape, dtype=torch.bfloat16):
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device="cuda")


F32, I8, I32 = torch.float32, torch.int8, torch.int32
BINDING = [
    ("one dimension", lambda c: sb.rms_norm_on_tiles(fake(64), c), ValueError),
    ("residual of another shape", lambda c: sb.rms_norm_on_tiles(fake(4, 9, 64), c, residual=fake(4, 9, 32)), AssertionError),
    ("residual of another type", lambda c: sb.rms_norm_on_tiles(fake(4, 9, 64), c, residual=fake(4, 9, 64, dtype=F32)), TypeError),
    ("gain of another length", lambda c: sb.rms_norm_on_tiles(fake(4, 9, 64), c, gain=fake(63, dtype=F32)), AssertionError),
    ("gain of another type", lambda c: sb.rms_norm_on_tiles(fake(4, 9, 64), c, gain=fake(64)), TypeError),
    ("a sum without a residual", lambda c: sb.rms_norm_on_tiles(fake(4, 9, 64), c, sum_out=fake(4, 9, 64)), ValueError),
    ("strided rows", lambda c: sb.rms_norm_on_tiles(fake(4, 9, 128)[:, :, ::2], c), TypeError),
    ("host memory", lambda c: sb.rms_norm_on_tiles(torch.zeros(4, 9, 64), c), TypeError),
    ("count of two", lambda c: sb.rms_norm_on_tiles(fake(4, 9, 64), fake(2, dtype=I32)), AssertionError),
    ("count in 64 bits", lambda c: sb.rms_norm_on_tiles(fake(4, 9, 64), fake(1, dtype=torch.int64)), TypeError),
    ("eps that is no number", lambda c: sb.rms_norm_on_tiles(fake(4, 9, 64), c, eps="small"), TypeError),
    ("codes without the padding", lambda c: sb.rms_norm_i8_on_tiles(fake(4, 9, 60), c, codes=fake(4, 9, 60, dtype=I8)), AssertionError),
    ("scales of another shape", lambda c: sb.quantize_i8_on_tiles(fake(4, 9, 64), c, codes=fake(4, 9, 64, dtype=I8), scales=fake(36, dtype=F32)),
     AssertionError),
    ("dy of another shape", lambda c: sb.rms_norm_backward_on_tiles(fake(4, 9, 64), fake(4, 64), c), AssertionError),
    ("dsum of another type", lambda c: sb.rms_norm_backward_on_tiles(fake(4, 9, 64), fake(4, 9, 64), c, dsum=fake(4, 9, 64, dtype=F32)), TypeError),
    ("a 3x3 kernel", lambda c: sb.quantize_weights_i8(fake(3, 3, 64, 64)), AssertionError),
    ("bytes for codes", lambda c: sb.pointwise_i8_on_tiles(fake(4, 9, 64, dtype=torch.uint8), fake(4, 9, dtype=F32), c, fake(8, 64, dtype=I8),
                                                           fake(8, dtype=F32)), TypeError),
    ("weights of another width", lambda c: sb.pointwise_i8_on_tiles(fake(4, 9, 64, dtype=I8), fake(4, 9, dtype=F32), c, fake(8, 48, dtype=I8),
                                                                    fake(8, dtype=F32)), AssertionError),
    ("no scales of the weights", lambda c: sb.pointwise_i8_on_tiles(fake(4, 9, 64, dtype=I8), fake(4, 9, dtype=F32), c, fake(8, 64, dtype=I8), None),
     AssertionError),
    ("bias of another length", lambda c: sb.pointwise_i8_on_tiles(fake(4, 9, 64, dtype=I8), fake(4, 9, dtype=F32), c, fake(8, 64, dtype=I8),
                                                                  fake(8, dtype=F32), bias=fake(7, dtype=F32)), AssertionError),
    ("8-bit results", lambda c: sb.pointwise_i8_on_tiles(fake(4, 9, 64, dtype=I8), fake(4, 9, dtype=F32), c, fake(8, 64, dtype=I8),
                                                         fake(8, dtype=F32), dtype=I8), TypeError),
    ("a dtype that is none", lambda c: sb.pointwise_i8_on_tiles(fake(4, 9, 64, dtype=I8), fake(4, 9, dtype=F32), c, fake(8, 64, dtype=I8),
                                                                fake(8, dtype=F32), dtype="bf16"), TypeError),
]


@pytest.mark.parametrize("k", range(len(BINDING)), ids=lambda k: BINDING[k][0].replace(" ", "_"))
def test_what_the_binding_refuses(k):
    _, call, error = BINDING[k]
    with pytest.raises(error):
        call(fake(1, dtype=I32))


# ---- the oracle ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("gained", (False, True))
def test_oracle_norm_and_gradients_are_autograds(gained):
    r = np.random.default_rng(5)
    x, dy, ds = (r.standard_normal((3, 4, 7)) for _ in range(3))
    g = 1 + 0.2 * r.standard_normal(7) if gained else None
    tx = torch.from_numpy(x).requires_grad_()
    tg = torch.from_numpy(g).requires_grad_() if gained else None
    eps = float(np.float32(1e-3))
    y = tx * (tx.square().mean(-1, keepdim=True) + eps).pow(-0.5)
    y = y * tg if gained else y
    np.testing.assert_allclose(orc.rms_norm(x, g, 1e-3), y.detach().numpy(), rtol=1e-13)
    (y * torch.from_numpy(dy)).sum().add((tx * torch.from_numpy(ds)).sum()).backward()
    dx, dg = orc.rms_norm_backward(x, dy, g, ds, 1e-3)
    np.testing.assert_allclose(dx, tx.grad.numpy(), rtol=1e-11, atol=1e-13)
    if gained:
        np.testing.assert_allclose(dg, tg.grad.numpy(), rtol=1e-11, atol=1e-13)


def test_oracle_norm_gradient_is_the_limit_of_differences():
    r = np.random.default_rng(6)
    x, dy, g = r.standard_normal((2, 5)), r.standard_normal((2, 5)), 1 + 0.2 * r.standard_normal(5)
    dx, dg = orc.rms_norm_backward(x, dy, g)
    loss = lambda a, b: (orc.rms_norm(a, b) * dy).sum()
    h = 1e-6
    for i in range(2):
        for j in range(5):
            e = np.zeros_like(x)
            e[i, j] = h
            assert abs((loss(x + e, g) - loss(x - e, g)) / (2 * h) - dx[i, j]) < 1e-8
    for j in range(5):
        e = np.zeros_like(g)
        e[j] = h
        assert abs((loss(x, g + e) - loss(x, g - e)) / (2 * h) - dg[j]) < 1e-8


def test_oracle_quantiser_on_fixed_rows():
    v = np.array([[0, 0, 0], [127, -127, 63.5], [1, 0.5, -0.25], [np.inf, 1, 2], [np.nan, 1, 2], [2.0 ** -130, 0, 0], [3e38, -3e38, 1e38]], np.float32)
    codes, scales = orc.quantize_i8(v)
    assert codes.shape == (7, 16) and not codes[:, 3:].any()
    assert codes[:, :3].tolist() == [[0, 0, 0], [127, -127, 64], [127, 64, -32], [0, 0, 0], [0, 0, 0], [0, 0, 0], [127, -127, 42]]
    assert scales[0] == np.float32(2.0 ** -100) / np.float32(127) and scales[1] == 1 and np.isnan(scales[3:5]).all()
    assert scales[5] == scales[0] and np.isfinite(scales[6])


def test_oracle_product_is_the_product_of_what_the_codes_stand_for():
    r = np.random.default_rng(7)
    a, w = r.integers(-127, 128, (2, 3, 32)).astype(np.int8), r.integers(-127, 128, (5, 32)).astype(np.int8)
    sa, sw, b = r.random((2, 3)), r.random(5), r.standard_normal(5)
    want = torch.nn.functional.linear(torch.from_numpy(a * sa[..., None]), torch.from_numpy(w * sw[:, None]), torch.from_numpy(b))
    np.testing.assert_allclose(orc.pointwise_i8(a, sa, w, sw, b), want.numpy(), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(orc.pointwise_i8(a, sa, w, sw, b, relu=True), want.relu().numpy(), rtol=1e-12, atol=1e-12)
    sa[1, 2] = np.nan
    assert np.isnan(orc.pointwise_i8(a, sa, w, sw, b, relu=True)[1, 2]).all()
