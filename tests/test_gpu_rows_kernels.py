"""The kernels behind the calls on rows, one by one: each product names the kernel that has to take it, so that a dispatch that moves shows;
counts from none to more than the list holds, far below the list's capacity too, on the kernels of long lists and wide layers.

Products are compared with the formula in 64 bits on the device.  The sum of codes is exact on both sides.  Its conversion, the product by
the row's scale and the fused step with channel scale and bias round to 24 bits each, the result once to its type: three steps of 2^-24
of the product without the bias, half a step of the result's type (bf16 2^-8, f16 2^-11, f32 2^-24) of the value with it, and 2^-25
for f16 values below its normal range; 1.01 is for the bounds being taken of rounded values."""
import re
import threading

import numpy as np
import pytest
import torch

import paper_1801_02108_amd as sb
from util import TORCH_DT, kernels, template_args

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}
MARK = 3.0                                        # what rows that must stay as they are hold


def step(msg):
    print("[case] " + msg, flush=True)


def cnt(n):
    return torch.tensor([n], dtype=torch.int32, device="cuda")


def product_inputs(cap, pixels, pitch, N):
    g = torch.Generator(device="cuda").manual_seed(cap * 7 + pixels + pitch + N)
    codes = torch.randint(-127, 128, (cap, pixels, pitch), dtype=torch.int8, device="cuda", generator=g)
    w = torch.randint(-127, 128, (N, pitch), dtype=torch.int8, device="cuda", generator=g)
    scales = (torch.rand((cap, pixels), device="cuda", generator=g) + 0.5) * 2.0 ** -12
    ws = (torch.rand(N, device="cuda", generator=g) + 0.5) * 2.0 ** -6
    return codes, scales, w, ws, torch.randn(N, device="cuda", generator=g)


def check_product(out, codes, scales, w, ws, bias, relu, dtype, n):
    """Rows of the first n tiles against the formula; the others as they were."""
    assert (out[n:] == MARK).all()
    wt = w.double().t().contiguous()
    for at in range(0, n, max(1, (1 << 24) // (codes.shape[1] * max(codes.shape[2], w.shape[0])))):
        to = min(n, at + max(1, (1 << 24) // (codes.shape[1] * max(codes.shape[2], w.shape[0]))))
        rows = codes[at:to].reshape(-1, codes.shape[2]).double()
        prod = (rows @ wt) * scales[at:to].reshape(-1, 1).double() * ws.double()
        ref = prod if bias is None else prod + bias.double()
        if relu:
            ref = ref.clamp(min=0.0)
        mag = prod.abs()
        allowed = (mag * 3 + (mag if bias is None else mag + bias.double().abs())) * U * 1.01 + ref.abs() * HALF[dtype] * 1.01 + TINY[dtype]
        err = (out[at:to].reshape(ref.shape).double() - ref).abs()
        assert not (err > allowed).any() and not err.isnan().any(), "%d off, worst by %g" % (int((err > allowed).sum()), float((err - allowed).max()))


def product_kernel(fn):
    name, = kernels(fn)
    return (re.search(r"i8_[a-z]+", name).group(0),) + template_args(name)[1:]


STREAMED = [
    # capacity, pixels, pitch, outputs, 64-channel pieces the kernel holds
    (36, 256, 64, 64, 1),                         # one group of 64 results, past the cache
    (20, 400, 64, 200, 1),                        # four, wider than the input; the last one of 8
    (20, 257, 48, 40, 1),                         # a piece and a group that are not full
    (40, 256, 128, 130, 2),                       # rows of results that do not start at 16 bytes
    (37, 257, 192, 128, 3),                       # two whole groups past the cache
    (49, 289, 192, 192, 3),                       # three
    (60, 289, 256, 200, 4),                       # three and one of 8
    (75, 256, 256, 256, 4),
    (29, 257, 320, 40, 6),                        # five pieces of six
    (49, 256, 384, 96, 6),
    (85, 81, 448, 16, 8),                         # seven of eight
    (77, 257, 512, 40, 8),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("cap,pixels,pitch,N,pieces", STREAMED)
def test_lists_that_are_streamed(cap, pixels, pitch, N, pieces, dtype):
    step("streamed %s" % ((cap, pixels, pitch, N, dtype),))
    codes, scales, w, ws, bias = product_inputs(cap, pixels, pitch, N)
    out, full = torch.full((cap, pixels, N), MARK, dtype=TORCH_DT[dtype], device="cuda"), cnt(cap)
    assert product_kernel(lambda: sb.pointwise_i8_on_tiles(codes, scales, full, w, ws, out=out)) == ("i8_stream", pieces)
    for n, b, relu in ((cap, bias, True), (cap - 1, None, False)):
        out.fill_(MARK)
        got = sb.pointwise_i8_on_tiles(codes, scales, cnt(n), w, ws, bias=b, relu=relu, out=out)
        assert got is out
        check_product(out, codes, scales, w, ws, b, relu, dtype, n)


OTHERS = [
    # rows, pitch, outputs, kernel and its tile in 16 (direct) or 32 (tiles) rows and channels a wave
    (5, 512, 500, "i8_direct", (1, 1, 8)),
    (16, 1040, 1000, "i8_direct", (1, 1, 8)),
    (5, 512, 5000, "i8_direct", (1, 2, 8)),
    (301, 2048, 250, "i8_direct", (1, 2, 8)),
    (5001, 512, 16, "i8_direct", (2, 1, 8)),
    (4999, 528, 9, "i8_direct", (2, 1, 8)),
    (601, 2000, 301, "i8_direct", (2, 2, 4)),
    (1101, 2000, 299, "i8_tiles", (2, 2, 1, 1)),
    (700, 528, 1000, "i8_tiles", (2, 2, 1, 1)),
    (1501, 528, 1001, "i8_tiles", (2, 2, 1, 2)),
    (1000, 1040, 2000, "i8_tiles", (2, 2, 1, 2)),
    (2112, 1040, 1024, "i8_tiles", (2, 2, 2, 2)),
    (9001, 1040, 1031, "i8_tiles", (2, 2, 2, 2)),
    (8191, 1040, 601, "i8_tiles", (2, 2, 4, 2)),
    (5003, 784, 3001, "i8_tiles", (2, 2, 4, 2)),
    (20001, 784, 1102, "i8_tiles", (2, 2, 4, 2)),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,pitch,N,kernel,shape", OTHERS)
def test_products_of_every_tile(rows, pitch, N, kernel, shape, dtype):
    step("%s %s %s" % (kernel, shape, (rows, pitch, N, dtype)))
    codes, scales, w, ws, bias = product_inputs(rows, 1, pitch, N)
    out, full = torch.full((rows, 1, N), MARK, dtype=TORCH_DT[dtype], device="cuda"), cnt(rows)
    assert product_kernel(lambda: sb.pointwise_i8_on_tiles(codes, scales, full, w, ws, out=out)) == (kernel,) + shape
    for n, b, relu in ((rows, bias, True), (rows - 1, None, False)):
        out.fill_(MARK)
        sb.pointwise_i8_on_tiles(codes, scales, cnt(n), w, ws, bias=b, relu=relu, out=out)
        check_product(out, codes, scales, w, ws, b, relu, dtype, n)


@pytest.mark.parametrize("rows,N,shape", [(1024, 300, (2, 2, 1, 1)), (2112, 1024, (2, 2, 2, 2)), (8192, 600, (2, 2, 4, 2))])
def test_the_largest_sums_through_lds(rows, N, shape):
    """Codes of -128 on both sides of 131056 channels: 131056 * 2^14 = 2^31 - 2^18, exact in float32, and 127 * -128 on the odd channels."""
    step("largest sums %s" % ((rows, N),))
    pitch = 131056
    codes = torch.full((rows, pitch), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, pitch), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    one, ones, out, full = torch.ones(rows, device="cuda"), torch.ones(N, device="cuda"), torch.empty((rows, N), device="cuda"), cnt(rows)
    assert product_kernel(lambda: sb.pointwise_i8_on_tiles(codes, one, full, w, ones, out=out)) == ("i8_tiles",) + shape
    assert (out[:, ::2] == float(pitch * 2 ** 14)).all() and (out[:, 1::2] == float(np.float32(-128 * 127 * pitch))).all()


COUNTED = [(300, 64, 64, 64, "i8_stream"), (200, 100, 256, 192, "i8_stream"), (300, 81, 512, 40, "i8_stream"),
           (50, 23, 2000, 299, "i8_tiles"), (300, 5, 528, 1001, "i8_tiles"), (133, 16, 1040, 1024, "i8_tiles"), (400, 21, 1040, 601, "i8_tiles"),
           (100, 7, 2000, 301, "i8_direct"), (5, 1, 512, 5000, "i8_direct")]


@pytest.mark.parametrize("cap,pixels,pitch,N,kernel", COUNTED)
def test_counts_far_below_and_above_the_capacity(cap, pixels, pitch, N, kernel):
    step("counts %s" % ((cap, pixels, pitch, N, kernel),))
    codes, scales, w, ws, bias = product_inputs(cap, pixels, pitch, N)
    n = cnt(0)
    out = torch.empty((cap, pixels, N), dtype=torch.bfloat16, device="cuda")
    assert product_kernel(lambda: sb.pointwise_i8_on_tiles(codes, scales, n, w, ws, bias=bias, out=out))[0] == kernel
    for count in (-2, 0, 1, 2, cap // 2, cap, cap + 2):
        n.fill_(count)
        out.fill_(MARK)
        sb.pointwise_i8_on_tiles(codes, scales, n, w, ws, bias=bias, out=out)
        check_product(out, codes, scales, w, ws, bias, False, "bf16", min(max(count, 0), cap))


@pytest.mark.parametrize("cap,pixels,C,dtype", [(1100, 324, 256, "bf16"), (3000, 7, 1032, "f16"), (900, 49, 97, "f32"), (600, 1, 8200, "bf16")])
def test_norms_on_a_few_tiles_of_a_long_list(cap, pixels, C, dtype):
    """The same bits as a list of just those tiles, and nothing else written.  (The first stacks pass the last-level cache by capacity.)"""
    step("norms of few tiles %s" % ((cap, pixels, C, dtype),))
    g = torch.Generator(device="cuda").manual_seed(cap + C)
    x, res, dy = (torch.randn((cap, pixels, C), generator=g, device="cuda").to(TORCH_DT[dtype]) for _ in range(3))
    gain = 1 + 0.1 * torch.randn(C, generator=g, device="cuda")
    pitch = (C + 15) // 16 * 16
    for count in (-2, 0, 1, 5, cap // 3, cap + 2):
        n = min(max(count, 0), cap)
        y, s, dx = (torch.full_like(x, MARK) for _ in range(3))
        codes, scales = torch.full((cap, pixels, pitch), 77, dtype=torch.int8, device="cuda"), torch.full((cap, pixels), MARK, device="cuda")
        sb.rms_norm_on_tiles(x, cnt(count), gain, residual=res, out=y, sum_out=s)
        assert (y[n:] == MARK).all() and (s[n:] == MARK).all()
        _, _, s8 = sb.rms_norm_i8_on_tiles(x, cnt(count), gain, residual=res, codes=codes, scales=scales)
        assert (codes[n:] == 77).all() and (scales[n:] == MARK).all()
        _, dgain = sb.rms_norm_backward_on_tiles(x, dy, cnt(count), gain, dsum=res, out=dx)
        assert (dx[n:] == MARK).all()
        if n == 0:
            assert not dgain.any()
            continue
        few = [t[:n].contiguous() for t in (x, res, dy)]
        y1, s1 = sb.rms_norm_on_tiles(few[0], cnt(n), gain, residual=few[1])
        assert torch.equal(y[:n], y1) and torch.equal(s[:n], s1) and torch.equal(s8[:n], s1)
        c1, k1, _ = sb.rms_norm_i8_on_tiles(few[0], cnt(n), gain, residual=few[1])
        assert torch.equal(codes[:n], c1) and torch.equal(scales[:n], k1)
        d1, _ = sb.rms_norm_backward_on_tiles(few[0], few[2], cnt(n), gain, dsum=few[1])
        assert torch.equal(dx[:n], d1)
        # dgain's order of summation goes by the capacity.  A chain of a thread's rows, one of the workgroup's places and one of a sixteenth of
        # the partial sums, each rounding at most the sum of magnitudes; h is 32 roundings off, as in the norm
        h = few[0].double() / (few[0].double().square().mean(-1, keepdim=True) + 1e-6).sqrt()
        terms = few[2].double() * h
        chain = n * pixels / 128 + 32 + 512 / 16 + 16 + 32
        assert ((dgain.double() - terms.sum((0, 1))).abs() <= terms.abs().sum((0, 1)) * chain * U).all()


@pytest.mark.parametrize("C", [64, 97, 2048])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_rows_whose_squares_pass_the_range_of_float32(dtype, C):
    """The norm gives zeros for such a row, whatever it holds: its gradients are zeros too (and the one past the norm), also where the sum of
    gain dy s passes the range."""
    step("rows past the range %d %s" % (C, dtype))
    g = torch.Generator(device="cuda").manual_seed(C)
    s, dy, ds = (torch.randn((6, 1, C), generator=g, device="cuda").to(TORCH_DT[dtype]) for _ in range(3))
    s[1], dy[1] = 2e38, 2.0                       # the sum is infinite
    s[3], dy[3] = 2e38, 2.0                       # ... of both signs, no number
    s[3, 0, C // 2:] = -2e38
    s[4, 0, 0] = 1e30                             # only the squares are
    assert not sb.rms_norm_on_tiles(s, cnt(6))[0][[1, 3, 4]].any()
    few = [0, 2, 5]
    for extra in (None, ds):
        dx, dgain = sb.rms_norm_backward_on_tiles(s, dy, cnt(6), dsum=extra)
        for k in (1, 3, 4):
            assert torch.equal(dx[k], torch.zeros_like(dx[k]) if extra is None else extra[k])
        dx1, dgain1 = sb.rms_norm_backward_on_tiles(s[few], dy[few], cnt(3), dsum=None if extra is None else extra[few])
        assert torch.equal(dx[few], dx1)
        terms = dy[few].double() * s[few].double() / (s[few].double().square().mean(-1, keepdim=True) + 1e-6).sqrt()
        assert ((dgain - dgain1).double().abs() <= terms.abs().sum((0, 1)) * 2 * (6 + 32) * U).all()      # (another order of the same sums)


@pytest.mark.parametrize("C", [64, 97, 2048, 20000])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gradients_of_rows_with_an_infinity_or_nan(dtype, C):
    """As the formula has it: no number in the whole row, and in dgain where the value stands (a NaN: everywhere); no other row."""
    step("infinities in gradients %d %s" % (C, dtype))
    g = torch.Generator(device="cuda").manual_seed(C)
    s, dy = (torch.randn((5, 1, C), generator=g, device="cuda").to(TORCH_DT[dtype]) for _ in range(2))
    clean = sb.rms_norm_backward_on_tiles(s, dy, cnt(5))[0]
    for at, v in ((0, float("inf")), (C - 1, float("-inf")), (C // 2, float("nan"))):
        bad = s.clone()
        bad[2, 0, at] = v
        dx, dgain = sb.rms_norm_backward_on_tiles(bad, dy, cnt(5))
        assert dx[2].isnan().all() and torch.equal(dx[[0, 1, 3, 4]], clean[[0, 1, 3, 4]])
        want = torch.full((C,), v != v, device="cuda")
        want[at] = True
        assert torch.equal(dgain.isnan(), want)


def test_two_threads_with_layers_of_different_widths():
    """Layers of one kernel that need different amounts of LDS, from two threads on streams of their own."""
    step("two threads")
    jobs = []
    for N in (64, 512):
        codes, scales, w, ws, bias = product_inputs(130, 256, 256, N)
        n = cnt(130)
        assert product_kernel(lambda: sb.pointwise_i8_on_tiles(codes, scales, n, w, ws, bias=bias)) == ("i8_stream", 4)
        want = sb.pointwise_i8_on_tiles(codes, scales, n, w, ws, bias=bias)
        jobs.append((codes, scales, n, w, ws, bias, want, torch.empty_like(want)))
    torch.cuda.synchronize()
    errors = []

    def work(job, stream):
        codes, scales, n, w, ws, bias, want, out = job
        try:
            with torch.cuda.stream(stream):
                for _ in range(500):
                    sb.pointwise_i8_on_tiles(codes, scales, n, w, ws, bias=bias, out=out)
            stream.synchronize()
            assert torch.equal(out, want)
        except Exception as e:                    # handed to the main thread
            errors.append(e)

    threads = [threading.Thread(target=work, args=(job, torch.cuda.Stream())) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
