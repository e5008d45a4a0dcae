"""GPU parity of the calls on the rows of tile stacks (root-mean-square norm with the residual's addition, its gradients, its
8-bit form, the row and weight quantisers, the pointwise product in 8-bit integers) against the float64 oracle.

Tolerances count roundings.  Half a step of the result's type relative to the value (bf16 2^-8, f16 2^-11, f32 2^-24; 2^-25 for
f16 values below its normal range), and steps of 2^-24 for the float32 arithmetic before it: a sum of n positive terms in chains of at most
32 terms per thread and trees of at most 12 levels is off by at most 44 of them, the square root halves that, and the mean, eps,
the reciprocal root (2) and two products add 6: 28; 32 are allowed.  A norm's gradient adds a product of three such factors: 96."""
import ctypes

import numpy as np
import pytest
import torch

import oracle as orc
import paper_1801_02108_amd as sb
from util import TORCH_DT

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}
MARK = 3.0                                        # what rows that must stay as they are hold


def step(msg):
    print("[case] " + msg, flush=True)


def rnd(seed):
    return np.random.default_rng(seed)


def dev(a, dtype="f32"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(TORCH_DT[dtype]).cuda()


def host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def cnt(n):
    return torch.tensor([n], dtype=torch.int32, device="cuda")


def within(got, ref, bound, what):
    assert got.shape == ref.shape, (got.shape, ref.shape)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), what
    fine = ~np.isnan(ref)
    err, bound = np.abs(got - ref)[fine], np.broadcast_to(bound, ref.shape)[fine]
    if err.size:
        k, wrong = np.argmax(err - bound), int((err > bound).sum())
        assert not wrong, "%s: %d of %d off, worst %g where %g is allowed (of %g)" % (what, wrong, err.size, err[k], bound[k], ref[fine][k])


def close_norm(got, s, gain, dtype, what, eps=1e-6):
    ref = orc.rms_norm(s, gain, eps)
    within(got, ref, np.abs(ref) * (HALF[dtype] * (1 + 32 * U) + 32 * U) + TINY[dtype], what)


def close_codes(codes, scales, v, what):
    """codes * scale against the unrounded rows v: half a code, and the float32 roundings of v (32) and of the two quotients."""
    c = v.shape[-1]
    assert not codes[..., c:].any(), what
    top = np.maximum(np.abs(v).max(-1), 2.0 ** -100)                          # as the quantiser is defined
    within(scales, top / 127.0, top / 127.0 * 36 * U, what + " scales")
    step_ = (top / 127.0)[..., None]
    within(codes[..., :c] * scales[..., None], v, step_ * (0.5 + 127 * 72 * U), what + " values")
    assert (np.abs(codes).max(-1) == 127)[top > 2.0 ** -100].all(), what


# sizes around the widths that a lane, a wave or a workgroup holds, multiples of 16 bytes and not
WIDTHS = [1, 2, 3, 7, 8, 15, 16, 17, 24, 31, 32, 33, 40, 63, 64, 65, 97, 120, 127, 128, 129, 200, 255, 256, 257, 384, 511, 512, 513, 520,
          1000, 1023, 1024, 1025, 1032, 2047, 2048, 2056, 4095, 4096, 4104, 8191, 8192, 8200, 16384, 16400, 20001, 32767, 32768]


def stack(r, cap, pixels, C, dtype):
    width = np.exp(0.5 * r.standard_normal(C))
    return dev(r.standard_normal((cap, pixels, C)) * width, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("C", WIDTHS)
def test_norm_and_its_codes(C, dtype):
    step("norm C %d %s" % (C, dtype))
    r = rnd(1000 + C)
    n, cap, pixels = 3, 5, 3 if C > 600 else 11
    x, res = stack(r, cap, pixels, C, dtype), stack(r, cap, pixels, C, dtype)
    gain = 1 + 0.2 * r.standard_normal(C)
    g = dev(gain)
    gain = host(g)
    out = torch.full_like(x, MARK)
    y, s = sb.rms_norm_on_tiles(x, cnt(n), g, out=out)
    assert y is out and s is x
    close_norm(host(y)[:n], host(x)[:n], gain, dtype, "norm")
    assert (y[n:] == MARK).all()
    total = torch.full_like(x, MARK)
    y, s = sb.rms_norm_on_tiles(x, cnt(n), None, residual=res, eps=0.5, sum_out=total)
    assert s is total and (s[n:] == MARK).all()
    want = (x.float() + res.float()).to(x.dtype)
    assert torch.equal(s[:n], want[:n])                                       # the sum is rounded once: the same bits
    close_norm(host(y)[:n], host(want)[:n], None, dtype, "norm with residual", 0.5)
    pitch = (C + 15) // 16 * 16
    codes = torch.full((cap, pixels, pitch), 77, dtype=torch.int8, device="cuda")
    scales = torch.full((cap, pixels), MARK, device="cuda")
    a, b, s8 = sb.rms_norm_i8_on_tiles(x, cnt(n), g, residual=res, codes=codes, scales=scales)
    assert a is codes and b is scales and torch.equal(s8[:n], want[:n])
    assert (codes[n:] == 77).all() and (scales[n:] == MARK).all()
    close_codes(host(codes)[:n], host(scales)[:n], orc.rms_norm(host(want)[:n], gain), "norm codes")
    a, b = sb.quantize_i8_on_tiles(x, cnt(n))
    oc, os_ = orc.quantize_i8(host(x)[:n])
    assert np.array_equal(a[:n].cpu().numpy(), oc) and np.array_equal(b[:n].cpu().numpy(), os_)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("C", WIDTHS)
def test_norm_gradients(C, dtype):
    step("norm backward C %d %s" % (C, dtype))
    r = rnd(2000 + C)
    n, cap, pixels = 4, 6, 3 if C > 600 else 37
    s, dy, ds = (stack(r, cap, pixels, C, dtype) for _ in range(3))
    g = dev(1 + 0.2 * r.standard_normal(C))
    for gain, extra in ((g, ds), (None, None)):
        out = torch.full_like(s, MARK)
        dx, dgain = sb.rms_norm_backward_on_tiles(s, dy, cnt(n), gain, dsum=extra, out=out)
        assert dx is out and (dx[n:] == MARK).all()
        check_gradients(s, dy, extra, gain, n, dx, dgain, dtype)
        again = sb.rms_norm_backward_on_tiles(s, dy, cnt(n), gain, dsum=extra)
        assert torch.equal(again[0][:n], dx[:n]) and torch.equal(again[1], dgain)           # the same bits every run


def check_gradients(s, dy, extra, gain, n, dx, dgain, dtype, eps=1e-6):
    hs, hd, he = host(s)[:n], host(dy)[:n], None if extra is None else host(extra)[:n]
    hg = None if gain is None else host(gain)
    rx, rg = orc.rms_norm_backward(hs, hd, hg, he, eps)
    root = np.sqrt((hs * hs).mean(-1, keepdims=True) + eps)
    gd, h = np.abs(hd if hg is None else hd * hg), np.abs(hs) / root
    parts = gd / root + h * (gd * h).mean(-1, keepdims=True) / root + (0 if he is None else np.abs(he))
    within(host(dx)[:n], rx, np.abs(rx) * HALF[dtype] + parts * 96 * U + TINY[dtype], "dx")
    # the rows' sums: a chain over a workgroup's rows and one over the workgroups, 700 terms at most between them here, and 32 for h
    within(host(dgain), rg, (np.abs(hd) * h).reshape(-1, s.shape[-1]).sum(0) * 732 * U, "dgain")


@pytest.mark.parametrize("count", [-2, 0, 1, 7, 9])
def test_counts_from_none_to_more_than_the_list_holds(count):
    step("count %d" % count)
    r = rnd(31)
    n, cap, pixels, C, N = min(max(count, 0), 7), 7, 9, 72, 40
    x, dy = stack(r, cap, pixels, C, "bf16"), stack(r, cap, pixels, C, "bf16")
    mark = torch.full_like(x, MARK)
    y, s = sb.rms_norm_on_tiles(x, cnt(count), None, residual=dy, out=mark.clone(), sum_out=mark.clone())
    assert (y[n:] == MARK).all() and (s[n:] == MARK).all()
    if n:
        close_norm(host(y)[:n], host(s)[:n], None, "bf16", "norm")
    dx, dgain = sb.rms_norm_backward_on_tiles(x, dy, cnt(count), out=mark.clone())
    assert (dx[n:] == MARK).all()
    if n:
        check_gradients(x, dy, None, None, n, dx, dgain, "bf16")
    else:
        assert not dgain.any()
    codes, scales = sb.quantize_i8_on_tiles(x, cnt(cap))
    w = torch.randint(-127, 128, (N, codes.shape[-1]), dtype=torch.int8, device="cuda")
    ws = torch.rand(N, device="cuda") + 0.5
    out = torch.full((cap, pixels, N), MARK, device="cuda", dtype=torch.bfloat16)
    sb.pointwise_i8_on_tiles(codes, scales, cnt(count), w, ws, out=out)
    assert (out[n:] == MARK).all()
    if n:
        close_product(out, codes, scales, w, ws, None, False, "bf16", n)


def test_an_empty_stack():
    step("empty stack")
    x = torch.empty((0, 9, 64), dtype=torch.bfloat16, device="cuda")
    y, s = sb.rms_norm_on_tiles(x, cnt(3), residual=x.clone())
    codes, scales = sb.quantize_i8_on_tiles(x, cnt(3))
    dx, dgain = sb.rms_norm_backward_on_tiles(x, x.clone(), cnt(3))
    out = sb.pointwise_i8_on_tiles(codes, scales, cnt(3), torch.zeros((8, 64), dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda"))
    assert y.shape == s.shape == dx.shape == x.shape and out.shape == (0, 9, 8) and codes.shape == (0, 9, 64) and not dgain.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [64, 33, 4096])
def test_results_may_take_the_place_of_inputs(C, dtype):
    step("in place C %d %s" % (C, dtype))
    r = rnd(41)
    n, cap, pixels = 3, 4, 5
    x, res, dy = (stack(r, cap, pixels, C, dtype) for _ in range(3))
    y0, s0 = sb.rms_norm_on_tiles(x, cnt(n), residual=res)
    for to_y, to_s in ((0, 1), (1, 0), (2, 0), (2, 1), (0, 2), (1, 2)):
        mine = [x.clone(), res.clone(), torch.full_like(x, MARK)]
        tail = [t[n:].clone() for t in mine]
        sb.rms_norm_on_tiles(mine[0], cnt(n), residual=mine[1], out=mine[to_y], sum_out=mine[to_s])
        assert torch.equal(mine[to_y][:n], y0[:n]) and torch.equal(mine[to_s][:n], s0[:n])
        assert all(torch.equal(t[n:], u) for t, u in zip(mine, tail))
    one = x.clone()
    sb.rms_norm_on_tiles(one, cnt(n), out=one)
    assert torch.equal(one[:n], sb.rms_norm_on_tiles(x, cnt(n))[0][:n])
    dx0, dg0 = sb.rms_norm_backward_on_tiles(x, dy, cnt(n), dsum=res)
    for k in range(3):
        mine = [x.clone(), dy.clone(), res.clone()]
        dx, dg = sb.rms_norm_backward_on_tiles(mine[0], mine[1], cnt(n), dsum=mine[2], out=mine[k])
        assert torch.equal(dx[:n], dx0[:n]) and torch.equal(dg, dg0) and torch.equal(dx[n:], (x, dy, res)[k][n:])
    codes0, scales0, _ = sb.rms_norm_i8_on_tiles(x, cnt(n), residual=res)
    mine = [x.clone(), res.clone()]
    codes, scales, s = sb.rms_norm_i8_on_tiles(mine[0], cnt(n), residual=mine[1], sum_out=mine[1])
    assert torch.equal(codes[:n], codes0[:n]) and torch.equal(scales[:n], scales0[:n]) and torch.equal(s[:n], s0[:n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [64, 35, 1032])
def test_stacks_that_start_at_any_element(C, dtype):
    step("unaligned C %d %s" % (C, dtype))
    r = rnd(43)
    n, pixels = 3, 7
    flat = dev(r.standard_normal(n * pixels * C + 8), dtype)
    for first in (1, 2, 4):
        x = flat[first:first + n * pixels * C].view(n, pixels, C)
        base = x.clone()
        out = flat.new_full((n * pixels * C + 8,), MARK)[first:first + n * pixels * C].view(n, pixels, C)
        y, _ = sb.rms_norm_on_tiles(x, cnt(n), out=out)
        close_norm(host(y), host(base), None, dtype, "norm")
        codes, scales = sb.quantize_i8_on_tiles(x, cnt(n))
        want = sb.quantize_i8_on_tiles(base, cnt(n))
        assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
        raw = torch.full((n * pixels * ((C + 15) // 16 * 16) + 1,), 5, dtype=torch.int8, device="cuda")[1:]
        codes, _ = sb.quantize_i8_on_tiles(x, cnt(n), codes=raw.view(n, pixels, -1))
        assert torch.equal(codes, want[0])
        dx, dgain = sb.rms_norm_backward_on_tiles(x, base, cnt(n), out=out)
        check_gradients(base, base, None, None, n, dx, dgain, dtype)


def test_other_ranks_of_stacks_are_the_same_rows():
    step("ranks")
    r = rnd(44)
    x = stack(r, 6, 12, 48, "f16")
    y0, _ = sb.rms_norm_on_tiles(x, cnt(5))
    q0 = sb.quantize_i8_on_tiles(x, cnt(5))
    w, ws = torch.randint(-127, 128, (24, 48), dtype=torch.int8, device="cuda"), torch.rand(24, device="cuda")
    p0 = sb.pointwise_i8_on_tiles(*q0, cnt(5), w, ws)
    for shape in ((6, 3, 4, 48), (6, 2, 3, 2, 48)):
        v = x.view(shape)
        assert torch.equal(sb.rms_norm_on_tiles(v, cnt(5))[0].view(6, 12, 48)[:5], y0[:5])
        q = sb.quantize_i8_on_tiles(v, cnt(5))
        assert q[0].shape == shape and q[1].shape == shape[:-1]
        p = sb.pointwise_i8_on_tiles(*q, cnt(5), w, ws)
        assert p.shape == shape[:-1] + (24,) and torch.equal(p.view(6, 12, 24)[:5], p0[:5])
    rows = x.view(72, 48)
    assert torch.equal(sb.rms_norm_on_tiles(rows, cnt(60))[0].view(6, 12, 48)[:5], y0[:5])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("C", [16, 33, 128, 1000, 5000])
def test_rows_of_zeros_infinities_nans_and_extremes(C, dtype):
    step("special rows C %d %s" % (C, dtype))
    r = rnd(51)
    big, small = {"bf16": (3e38, 1e-38), "f16": (65504.0, 6e-8), "f32": (3e38, 1e-40)}[dtype]
    v = r.standard_normal((8, 1, C)).astype(np.float32)
    v[0] = 0
    v[1, 0, C // 2] = np.inf
    v[2, 0, C - 1] = -np.inf
    v[3, 0, 0] = np.nan
    v[4] *= np.float32(small)
    v[5] = 0
    v[5, 0, 1] = -big
    v[6] = np.float32(2.0 ** -20)
    v[6, 0, 0] = 1.0
    x = dev(v, dtype)
    codes, scales = sb.quantize_i8_on_tiles(x, cnt(8))
    oc, os_ = orc.quantize_i8(host(x))
    assert np.array_equal(codes.cpu().numpy(), oc) and np.array_equal(scales.cpu().numpy(), os_, equal_nan=True)
    # the norm of the same rows without the largest (its squares pass float32's range, except in f16): NaN where the formula has it
    keep = [0, 1, 2, 3, 4, 6, 7] + ([5] if dtype == "f16" else [])
    y, _ = sb.rms_norm_on_tiles(x, cnt(8))
    hx, hy = host(x)[keep], host(y)[keep]
    with np.errstate(invalid="ignore"):
        close_norm(hy, hx, None, dtype, "norm of special rows")
    codes, scales, _ = sb.rms_norm_i8_on_tiles(x, cnt(8))
    assert np.array_equal(np.isnan(scales[:5, 0].cpu().numpy()), [False, True, True, True, False]) and not codes[:4].any()
    if dtype != "f16":
        assert not y[5].any()
    # a NaN scale reaches every result of its row, through the ReLU too, and no other row
    w, ws = torch.randint(-127, 128, (9, codes.shape[-1]), dtype=torch.int8, device="cuda"), torch.ones(9, device="cuda")
    out = sb.pointwise_i8_on_tiles(codes, scales, cnt(8), w, ws, relu=True, dtype=torch.float32)
    assert torch.equal(out.isnan().all(-1), scales.isnan()) and torch.equal(out.isnan().any(-1), scales.isnan())


@pytest.mark.parametrize("eps", [1.1754944e-38, 1e-30, 1e30])
def test_the_ends_of_eps(eps):
    step("eps %g" % eps)
    x = stack(rnd(52), 2, 3, 40, "f32")
    x[0] = 0
    y, _ = sb.rms_norm_on_tiles(x, cnt(2), eps=eps)
    close_norm(host(y), host(x), None, "f32", "norm", eps)
    dx, dgain = sb.rms_norm_backward_on_tiles(x, torch.ones_like(x), cnt(2), eps=eps)
    with np.errstate(over="ignore", invalid="ignore"):
        check_gradients(x, torch.ones_like(x), None, None, 2, dx, dgain, "f32", float(np.float32(eps)))


# ---- weights and product -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("cin,cout", [(1, 1), (3, 5), (16, 8), (64, 256), (100, 33), (256, 64), (777, 130), (4100, 70), (64, 1025)])
def test_weights_in_8_bits(cin, cout, dtype):
    step("weights %d %d %s" % (cin, cout, dtype))
    w = dev(rnd(60 + cin).standard_normal((1, 1, cin, cout)) * 0.1, dtype)
    w[0, 0, :, cout // 2] = 0
    codes, scales = sb.quantize_weights_i8(w)
    oc, os_ = orc.quantize_i8(host(w)[0, 0].T)
    assert np.array_equal(codes.cpu().numpy(), oc) and np.array_equal(scales.cpu().numpy(), os_)
    w[0, 0, 0, 0] = float("nan")
    codes, scales = sb.quantize_weights_i8(w)
    assert scales[0].isnan() and not codes[0].any() and (cout == 1 or not scales[1:].isnan().any())


def close_product(out, codes, scales, w, ws, bias, relu, dtype, n):
    """The sum is exact; its conversion, two products and the bias are rounded to 24 bits each, then the result to its type."""
    a, sa, hw, hs = host(codes)[:n], host(scales)[:n], host(w), host(ws)
    hb = 0.0 if bias is None else host(bias)
    ref = orc.pointwise_i8(a, sa, hw, hs, None if bias is None else hb, relu)
    prod = np.abs((a @ hw.T) * sa[..., None] * hs)
    within(host(out)[:n], ref, (prod * 3 + np.abs(prod + np.abs(hb))) * U * 1.01 + np.abs(ref) * HALF[dtype] * 1.01 + TINY[dtype], "product")


PRODUCTS = [
    # rows as (cap, pixels), pitch, outputs
    (1, 1, 16, 1), (1, 1, 16, 5), (1, 1, 4096, 4096), (1, 1, 64, 8), (2, 1, 2064, 96), (3, 1, 48, 33), (7, 1, 1040, 257), (9, 1, 8192, 64),
    (15, 1, 512, 512), (16, 1, 512, 520), (17, 1, 512, 128), (31, 1, 272, 100), (33, 1, 1024, 1000), (47, 1, 128, 4097), (64, 1, 2048, 256),
    (65, 1, 2048, 256), (100, 1, 144, 48), (1, 127, 128, 128), (129, 1, 1024, 384), (3, 100, 64, 256), (4, 324, 256, 64), (5, 256, 384, 96),
    (2, 289, 80, 17), (11, 81, 112, 200), (1, 513, 4096, 130), (600, 1, 320, 1031), (1025, 1, 640, 264), (2, 1000, 32, 12), (1500, 1, 1168, 1100),
    (1, 1, 131056, 3), (130, 1, 131056, 40),
    # long lists of narrow layers
    (30, 324, 256, 64), (33, 256, 64, 250), (33, 256, 128, 130), (40, 256, 384, 96), (129, 64, 512, 40), (9001, 1, 16, 1), (36, 289, 80, 333),
    (41, 256, 320, 512), (128, 81, 448, 200), (33, 255, 32, 513),
    # wide layers on long lists
    (4099, 1, 208, 4104), (2047, 1, 1040, 8201), (41, 100, 528, 4113),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("cap,pixels,pitch,N", PRODUCTS)
def test_pointwise_product(cap, pixels, pitch, N, dtype):
    step("pointwise %s" % ((cap, pixels, pitch, N, dtype),))
    g = torch.Generator(device="cuda").manual_seed(cap * 7 + pixels + pitch + N)
    total = cap + 1                                                    # one tile behind the active ones
    codes = torch.randint(-127, 128, (total, pixels, pitch), dtype=torch.int8, device="cuda", generator=g)
    w = torch.randint(-127, 128, (N, pitch), dtype=torch.int8, device="cuda", generator=g)
    scales = (torch.rand((total, pixels), device="cuda", generator=g) + 0.5) * 2.0 ** -12
    ws = (torch.rand(N, device="cuda", generator=g) + 0.5) * 2.0 ** -6
    bias = torch.randn(N, device="cuda", generator=g)
    for b, relu in ((bias, True), (None, False)):
        out = torch.full((total, pixels, N), MARK, dtype=TORCH_DT[dtype], device="cuda")
        got = sb.pointwise_i8_on_tiles(codes, scales, cnt(cap), w, ws, bias=b, relu=relu, out=out)
        assert got is out and (out[cap:] == MARK).all()
        close_product(out, codes, scales, w, ws, b, relu, dtype, cap)


@pytest.mark.parametrize("rows,pitch,N", [(1, 131056, 17), (40, 131056, 33), (300, 131056, 70), (600, 131056, 300)])
def test_sums_reach_the_ends_of_32_bits(rows, pitch, N):
    """Codes of -128 (no quantiser here writes them) on both sides: 131056 * 2^14 = 2^31 - 2^18."""
    step("largest sums %s" % ((rows, pitch, N),))
    codes = torch.full((rows, pitch), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, pitch), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    out = sb.pointwise_i8_on_tiles(codes, torch.ones(rows, device="cuda"), cnt(rows), w, torch.ones(N, device="cuda"), dtype=torch.float32)
    assert (out[:, ::2] == float(pitch * 2 ** 14)).all() and (out[:, 1::2] == float(np.float32(-128 * 127 * pitch))).all()


def test_long_stacks_pass_32_bit_offsets():
    """More than 2^31 elements and 2^32 bytes in each stack: the last rows against the same rows alone."""
    step("long stacks")
    C, pixels = 1024, 256
    cap = (1 << 32) // (2 * C * pixels) + 3
    x = torch.zeros((cap, pixels, C), dtype=torch.bfloat16, device="cuda")
    x[-2:] = stack(rnd(71), 2, pixels, C, "bf16")
    n = cnt(cap)
    y, s = sb.rms_norm_on_tiles(x, n, residual=x)
    y1, s1 = sb.rms_norm_on_tiles(x[-2:].clone(), cnt(2), residual=x[-2:].clone())
    assert torch.equal(y[-2:], y1) and torch.equal(s[-2:], s1) and not y[0].any() and not y[cap // 2].any()
    del y, s
    dx, _ = sb.rms_norm_backward_on_tiles(x, x, n)
    assert torch.equal(dx[-2:], sb.rms_norm_backward_on_tiles(x[-2:].clone(), x[-2:].clone(), cnt(2))[0])
    del dx
    codes, scales = sb.quantize_i8_on_tiles(torch.cat([x, x]), cnt(2 * cap))
    assert codes.numel() > 1 << 32
    c1, s1 = sb.quantize_i8_on_tiles(x[-2:].clone(), cnt(2))
    assert torch.equal(codes[-2:], c1) and torch.equal(scales[-2:], s1)
    w, ws = torch.randint(-127, 128, (2048, C), dtype=torch.int8, device="cuda"), torch.ones(2048, device="cuda")
    out = sb.pointwise_i8_on_tiles(codes, scales, cnt(2 * cap), w, ws)
    assert torch.equal(out[-2:], sb.pointwise_i8_on_tiles(c1, s1, cnt(2), w, ws)) and not out[:3].any()


# ---- together ------------------------------------------------------------------------------------------------------------
def chain(x, res, count, gain, w, ws, bias):
    codes, scales, s = sb.rms_norm_i8_on_tiles(x, count, gain, residual=res)
    return sb.pointwise_i8_on_tiles(codes, scales, count, w, ws, bias=bias, relu=True), s


def test_a_layer_between_gather_and_scatter():
    """Active blocks of a map: gathered, normed into 8 bits, multiplied, scattered onto a map; against the oracle's steps."""
    step("gather, norm, product, scatter")
    r = rnd(81)
    N, H, W, C, K, bo = 2, 21, 30, 40, 24, 6
    g, go, _, _ = sb.geometry(H, W, 1, 1, bo)
    mask = (r.random((N, H, W)) < 0.01).astype(np.uint8)
    idx, n = sb.reduce_mask(torch.from_numpy(mask).cuda(), g)
    active = int(n.item())
    assert 0 < active < idx.shape[0]
    x, w = dev(r.standard_normal((N, H, W, C)), "bf16"), dev(r.standard_normal((1, 1, C, K)) * 0.2, "bf16")
    gain, bias = dev(1 + 0.1 * r.standard_normal(C)), dev(r.standard_normal(K))
    tiles = sb.sparse_gather(x, idx, n, g)
    codes, scales, _ = sb.rms_norm_i8_on_tiles(tiles, n, gain)
    wc, ws = sb.quantize_weights_i8(w)
    t = sb.pointwise_i8_on_tiles(codes, scales, n, wc, ws, bias=bias, relu=True)
    y = sb.sparse_scatter(t, idx, n, go, torch.full((N, H, W, K), MARK, dtype=torch.bfloat16, device="cuda"))
    # the oracle on the device's codes (which the tests above hold against the oracle's norm)
    close_codes(host(codes)[:active], host(scales)[:active], orc.rms_norm(host(tiles)[:active], host(gain)), "codes")
    close_product(t, codes, scales, wc, ws, bias, True, "bf16", active)
    hi = idx[:active].cpu().numpy()
    want = orc.scatter(host(t)[:active], hi, orc.Geom(*go.astuple()), np.full((N, H, W, K), MARK))
    assert np.array_equal(host(y), want)
    # and near the layer without any 8-bit rounding: codes are off by at most half a step on each side
    ideal = np.maximum(orc.rms_norm(host(tiles)[:active], host(gain)) @ host(w)[0, 0] + host(bias), 0)
    got = host(t)[:active]
    assert np.sqrt(((got - ideal) ** 2).mean()) < 0.03 * np.sqrt((ideal ** 2).mean())


def test_a_training_step_of_the_norm_is_the_formulas():
    step("forward and backward")
    r = rnd(82)
    n, C = 5, 192
    x, res, dy, ds = (stack(r, 6, 49, C, "bf16") for _ in range(4))
    gain = dev(1 + 0.1 * r.standard_normal(C))
    y, s = sb.rms_norm_on_tiles(x, cnt(n), gain, residual=res)
    dx, dgain = sb.rms_norm_backward_on_tiles(s, dy, cnt(n), gain, dsum=ds)
    check_gradients(s, dy, ds, gain, n, dx, dgain, "bf16")
    # the slope of sum(y dy) + sum(s ds) along a direction, by differences of the forward formula on the stored sum
    d = r.standard_normal((n, 49, C))
    loss = lambda v: (orc.rms_norm(v, host(gain)) * host(dy)[:n]).sum() + (v * host(ds)[:n]).sum()
    h = 1e-5
    slope = (loss(host(s)[:n] + h * d) - loss(host(s)[:n] - h * d)) / (2 * h)
    ref, _ = orc.rms_norm_backward(host(s)[:n], host(dy)[:n], host(gain), host(ds)[:n])
    # dx is rounded to bf16: the slope by it is off by at most the sum of half steps
    assert abs((host(dx)[:n] * d).sum() - slope) < (np.abs(ref * d)).sum() * 2.0 ** -8


def graph_of(fn):
    fn()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = fn()
    return g, got


@pytest.mark.parametrize("rows", [1, 24, 700])
def test_captured_and_replayed_with_other_work_between(rows):
    step("graph of %d rows" % rows)
    C, N = 512, 264
    r = rnd(83)
    x, res, dy = (stack(r, rows, 1, C, "bf16") for _ in range(3))
    n, gain = cnt(rows), dev(1 + 0.1 * r.standard_normal(C))
    w, ws = sb.quantize_weights_i8(dev(r.standard_normal((1, 1, C, N)) * 0.05))

    def program():
        out, s = chain(x, res, n, gain, w, ws, None)
        dx, dgain = sb.rms_norm_backward_on_tiles(s, dy, n, gain, dsum=res)
        return out, s, dx, dgain

    ga, a = graph_of(program)
    gb, b = graph_of(program)                                         # a second graph of the same calls, its own workspaces
    for k in range(4):
        x.copy_(stack(rnd(90 + k), rows, 1, C, "bf16"))
        n.fill_(rows if k % 2 else max(1, rows // 2))
        active = int(n.item())
        want = [t.clone() for t in program()]
        for got in (a, b):
            for t in got:
                t.fill_(MARK)
        ga.replay()
        gb.replay()
        torch.cuda.synchronize()
        for got in (a, b):
            for t, u in zip(got[:3], want[:3]):
                assert torch.equal(t[:active], u[:active]) and (t[active:] == MARK).all()
            assert torch.equal(got[3], want[3])


def test_on_a_stream_of_its_own():
    step("side stream")
    r = rnd(84)
    x, res = stack(r, 300, 16, 256, "bf16"), stack(r, 300, 16, 256, "bf16")
    w, ws = sb.quantize_weights_i8(dev(r.standard_normal((1, 1, 256, 64)) * 0.05))
    n = cnt(300)
    want = chain(x, res, n, None, w, ws, None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [chain(x, res, n, None, w, ws, None) for _ in range(3)]
        back = sb.rms_norm_backward_on_tiles(x, res, n)
    here = sb.rms_norm_backward_on_tiles(x, res, n)                    # two at once, each with its own workspace
    torch.cuda.synchronize()
    for out, s in got:
        assert torch.equal(out, want[0]) and torch.equal(s, want[1])
    assert torch.equal(back[0], here[0]) and torch.equal(back[1], here[1])


def test_the_callers_workspace_is_used_and_only_that_much():
    step("workspace")
    r = rnd(85)
    s, dy = stack(r, 40, 5, 96, "f16"), stack(r, 40, 5, 96, "f16")
    need = sb.lib().sbnet_rms_norm_backward_workspace_bytes(40, 5, 96)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    got = sb.rms_norm_backward_on_tiles(s, dy, cnt(40), workspace=ws[:need])
    assert (ws[need:] == 0xA5).all() and not (ws[:need] == 0xA5).all()
    want = sb.rms_norm_backward_on_tiles(s, dy, cnt(40))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(sb.SbnetError) as e:
        sb.rms_norm_backward_on_tiles(s, dy, cnt(40), workspace=ws[:need - 4])
    assert e.value.code == sb.EINVAL and "workspace" in str(e.value)
