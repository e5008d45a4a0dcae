"""Performance cases of the operators on the pixels of tile stacks: root-mean-square norm with the residual's addition, its
gradients, its 8-bit form, and the pointwise (1x1) product in 8-bit integers with a scale for each pixel and channel.

A case is a dict of plain values.  `kind` names the program that runs:

  norm            s = x + residual, y = s / sqrt(mean(s^2) + eps) * gain; returns y and s
  norm_backward   gradients of s and gain from the gradient of y and the one that reaches s past the norm
  pointwise       the activations' rows in 8 bits with a scale each, times 8-bit weights with a scale for each output channel
  norm_pointwise  norm with an 8-bit output, and the product that reads it; returns the product and s

A stack has `tiles` active tiles of `pixels` pixels with `c` channels: rows = tiles * pixels.  Widths and tile sizes are
those of the repository's benchmark and tests (16 x 16 tiles of 64 to 256 channels, 384 -> 96 units and the like) or generic
ones; single rows and small batches stand for a head or a sequence model that answers one item at a time.

Where `own` is false the operators are computed in elementary torch operations in 32 bits, each result rounded once.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_ES = {"f32": 4, "bf16": 2, "f16": 2}
_EPS = 1e-6


def listed():
    return [
        # one row: the norm in front of a head that answers a single item, all latency
        dict(name="norm_one_row", kind="norm", tiles=1, pixels=1, c=1024, dtype="bf16", residual=True),
        # a crowded full-resolution map's active tiles at the width of a residual unit
        dict(name="norm_tiles_256", kind="norm", tiles=440, pixels=256, c=256, dtype="bf16", residual=True),
        # odd everything: a width that no vector divides, tiles with their halo
        dict(name="norm_ragged", kind="norm", tiles=61, pixels=324, c=97, dtype="f16", residual=True),
        # long rows in float32, no residual
        dict(name="norm_wide_f32", kind="norm", tiles=4099, pixels=1, c=4096, dtype="f32", residual=False),
        # training step of the unit-width norm
        dict(name="norm_backward_tiles", kind="norm_backward", tiles=440, pixels=256, c=256, dtype="bf16", residual=True),
        # ... and on a short list of an odd width
        dict(name="norm_backward_ragged", kind="norm_backward", tiles=13, pixels=289, c=200, dtype="f16", residual=False),
        # the first 1x1 convolution of a residual unit on its input tiles
        dict(name="pointwise_reduce", kind="pointwise", tiles=440, pixels=324, c=256, out=64, dtype="bf16", relu=True, bias=True),
        # ... and the last one, four times as wide as its input
        dict(name="pointwise_expand", kind="pointwise", tiles=440, pixels=256, c=64, out=256, dtype="f16", relu=False, bias=True),
        # wide layers on a long batch: bound by the matrix cores
        dict(name="pointwise_large", kind="pointwise", tiles=8192, pixels=1, c=4096, out=8192, dtype="bf16", relu=False, bias=False),
        # one row through norm and product: the weights' bytes are all of it
        dict(name="norm_pointwise_one", kind="norm_pointwise", tiles=1, pixels=1, c=4096, out=4096, dtype="bf16", relu=False,
             bias=False, residual=True),
        # a small batch of rows, ragged
        dict(name="norm_pointwise_few", kind="norm_pointwise", tiles=23, pixels=1, c=2056, out=5125, dtype="f16", relu=True,
             bias=True, residual=True),
        # the widest residual unit's reduction behind a norm
        dict(name="norm_pointwise_tiles", kind="norm_pointwise", tiles=173, pixels=256, c=384, out=96, dtype="bf16", relu=True,
             bias=True, residual=True),
    ]


def _spread(rng, lo, hi):
    """A whole number whose logarithm is spread evenly over the range."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_backward", "pointwise", "norm_pointwise"])
    pixels = rng.choice([1, 1, 64, 81, 100, 256, 289, 324])
    case = dict(kind=kind, tiles=0, pixels=pixels, c=_spread(rng, 16, 8192), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
    if rng.random() < 0.6:                      # most widths are multiples of something; the others stay odd
        step = rng.choice([8, 16, 32, 64])
        case["c"] = max(step, case["c"] // step * step)
    if kind in ("norm", "norm_backward"):
        rows = _spread(rng, 1, max(1, 28_000_000 // case["c"]))
        case["residual"] = rng.random() < 0.6
    else:
        if kind == "norm_pointwise" and case["dtype"] == "f32":     # the 8-bit path answers in 16 bits behind a norm
            case["dtype"] = "bf16"
        case["out"] = _spread(rng, 16, 8192)
        if rng.random() < 0.6:
            step = rng.choice([8, 16, 32])
            case["out"] = max(step, case["out"] // step * step)
        most = min(36_000_000 // case["c"], 36_000_000 // case["out"], 250_000_000_000 // (case["c"] * case["out"]))
        rows = _spread(rng, 1, max(1, most))
        case["relu"] = rng.random() < 0.5
        case["bias"] = rng.random() < 0.5
        if kind == "norm_pointwise":
            case["residual"] = rng.random() < 0.6
    case["tiles"] = max(1, rows // pixels)
    return case


def _shape(case):
    return (case["tiles"], case["pixels"], case["c"])


def _rows(case):
    return case["tiles"] * case["pixels"]


def prepare(case, seed):
    """Inputs of one program: activations whose channels differ in size, as they do behind a few layers, gains near one,
    and weights that a program has quantised once, a scale for each output channel, rows padded with zeros to 16 codes."""
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 17)
    dt, c = _DT[case["dtype"]], case["c"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    width = torch.exp(0.5 * normal(c))
    st = dict(case=case, count=torch.full((1,), case["tiles"], dtype=torch.int32, device="cuda"),
              x=(normal(*_shape(case)) * width).to(dt))
    if case["kind"] != "pointwise":
        st["gain"] = 1.0 + 0.1 * normal(c)
        if case["residual"]:
            st["residual"] = (normal(*_shape(case)) * width).to(dt)
    if case["kind"] == "norm_backward":
        st["dy"] = normal(*_shape(case)).to(dt)
    if "out" in case:
        n, pitch = case["out"], (c + 15) // 16 * 16
        w = normal(n, c) * math.sqrt(2.0 / c)
        st["w_scales"] = w.abs().amax(1) / 127.0
        st["w_codes"] = torch.zeros((n, pitch), dtype=torch.int8, device="cuda")
        st["w_codes"][:, :c] = torch.round(w / st["w_scales"][:, None]).to(torch.int8)
        if case["bias"]:
            st["bias"] = 0.1 * normal(n)
    return st


def run(st):
    return _own(st) if own else _plain(st)


def _own(st):
    import paper_1801_02108_amd as sb
    case, count = st["case"], st["count"]
    kind = case["kind"]
    if kind == "norm":
        y, s = sb.rms_norm_on_tiles(st["x"], count, st["gain"], residual=st.get("residual"), eps=_EPS)
        return {"y": y, "s": s} if case["residual"] else {"y": y}
    if kind == "norm_backward":
        dx, dgain = sb.rms_norm_backward_on_tiles(st["x"], st["dy"], count, st["gain"], dsum=st.get("residual"), eps=_EPS)
        return {"dx": dx, "dgain": dgain}
    if kind == "pointwise":
        codes, scales = sb.quantize_i8_on_tiles(st["x"], count)
    else:
        codes, scales, s = sb.rms_norm_i8_on_tiles(st["x"], count, st["gain"], residual=st.get("residual"), eps=_EPS)
    y = sb.pointwise_i8_on_tiles(codes, scales, count, st["w_codes"], st["w_scales"], bias=st.get("bias"), relu=case["relu"],
                                 dtype=_DT[case["dtype"]])
    return {"y": y, "s": s} if kind == "norm_pointwise" and case["residual"] else {"y": y}


def _plain(st):
    case = st["case"]
    kind, dt = case["kind"], _DT[case["dtype"]]
    if kind == "norm_backward":
        s, dy, gain = st["x"].float(), st["dy"].float(), st["gain"]
        r = torch.rsqrt((s * s).mean(-1, keepdim=True) + _EPS)
        sh = s * r
        gd = gain * dy
        dx = r * (gd - sh * (gd * sh).mean(-1, keepdim=True))
        if case["residual"]:
            dx = dx + st["residual"].float()
        return {"dx": dx.to(dt), "dgain": (dy * sh).sum((0, 1))}
    if kind == "pointwise":
        v, s = st["x"].float(), None
    else:
        s = (st["x"].float() + st["residual"].float()).to(dt) if case["residual"] else None
        f = (st["x"] if s is None else s).float()
        v = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + _EPS) * st["gain"]
    if kind == "norm":
        out = {"y": v.to(dt)}
    else:
        top = v.abs().amax(-1, keepdim=True)
        codes = torch.round(v * (127.0 / top))
        w = st["w_codes"][:, :case["c"]].float()
        y = torch.matmul(codes.reshape(-1, case["c"]), w.t()).reshape(case["tiles"], case["pixels"], case["out"])
        y = y * (top / 127.0) * st["w_scales"]
        if case["bias"]:
            y = y + st["bias"]
        if case["relu"]:
            y = torch.relu(y)
        out = {"y": y.to(dt)}
    if s is not None:
        out["s"] = s
    return out


def work(case):
    """Bytes: activations, residual, gradients, weights and vectors read once, results written once (8-bit codes are passed
    from one call to the next and count as nothing).  Operations: the product's, or a few for each value of a norm."""
    rows, c, es = _rows(case), case["c"], _ES[case["dtype"]]
    kind = case["kind"]
    if kind == "norm":
        return {"bytes": rows * c * es * (4 if case["residual"] else 2) + 4 * c, "flops": 5 * rows * c}
    if kind == "norm_backward":
        return {"bytes": rows * c * es * (4 if case["residual"] else 3) + 8 * c, "flops": 12 * rows * c}
    n = case["out"]
    nbytes = rows * c * es + n * c + rows * n * es + n * (8 if case["bias"] else 4)
    if kind == "norm_pointwise":
        nbytes += 4 * c + (2 * rows * c * es if case["residual"] else 0)
    return {"bytes": nbytes, "flops": 2 * rows * c * n}


def exact(case, seed):
    """The same results from the definitions in 64 bits."""
    st = prepare(case, seed)
    rows, c = _rows(case), case["c"]
    x = st["x"].reshape(rows, c)
    if case["kind"] == "norm_backward":
        # with m = mean(x^2) + eps: y = x g / sqrt(m), so dx_j = g_j dy_j / sqrt(m) - x_j sum_i(g_i dy_i x_i) / (c m sqrt(m))
        x, dy, g = x.double(), st["dy"].reshape(rows, c).double(), st["gain"].double()
        m = torch.einsum("rc,rc->r", x, x) / c + _EPS
        t = torch.einsum("rc,rc,c->r", x, dy, g)
        dx = dy * g / torch.sqrt(m)[:, None] - x * (t / (c * m * torch.sqrt(m)))[:, None]
        if case["residual"]:
            dx += st["residual"].reshape(rows, c).double()
        return {"dx": dx.reshape(_shape(case)), "dgain": torch.einsum("rc,rc->c", dy, x / torch.sqrt(m)[:, None])}
    s = None
    if case["kind"] == "pointwise":
        v = x.double()
    else:
        if case["residual"]:                    # the stored sum is rounded to its type, and the norm is the stored sum's
            s = (x.double() + st["residual"].reshape(rows, c).double()).to(x.dtype)
            x = s
        x = x.double()
        v = x * st["gain"].double() / torch.sqrt(torch.einsum("rc,rc->r", x, x) / c + _EPS)[:, None]
    if case["kind"] == "norm":
        y, width = v, c
    else:
        step = v.abs().max(1).values / 127.0
        codes = torch.round(v / step[:, None])
        y, width = torch.empty((rows, case["out"]), dtype=torch.float64, device=v.device), case["out"]
        for at in range(0, rows, 16384):
            y[at:at + 16384] = codes[at:at + 16384] @ st["w_codes"][:, :c].double().t()
        y *= step[:, None]
        y *= st["w_scales"].double()
        if case["bias"]:
            y += st["bias"].double()
        if case["relu"]:
            y = y.clamp(min=0.0)
    out = {"y": y.reshape(case["tiles"], case["pixels"], width)}
    if s is not None:
        out["s"] = s.double().reshape(_shape(case))
    return out
