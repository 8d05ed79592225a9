"""The residual's addition and its norm on the GPU against fp64, at sizes,
places and values where they can go wrong."""
import numpy as np
import pytest
import torch

import coded_ref as ref
import paper_2608_23429_amd as cheb

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6
U = 2.0 ** -24                                   # fp32's half step, relative


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def half_step(y, out):
    """Half a step of the output's type at values y."""
    rel, tiny = {"bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25),
                 "f32": (U, 2.0 ** -150)}[out]
    return np.maximum(np.abs(y) * rel, tiny)


def reference(srcs, w, x_in, kind, gain, shift, eps=EPS):
    """(x, y, bound on y before its last rounding), [rows, dim] fp64.  The bound
    counts fp32 roundings: x's, h's, the factor's, the products' and the sum's."""
    x = np.zeros_like(srcs[0]) if x_in is None else x_in.copy()
    for a, s in zip(w, srcs):
        x = x + a * s
    rows, dim = x.shape
    size = np.abs(x)
    h = x
    if kind == "layer":
        h = x - x.mean(1, keepdims=True)
        size = size + np.abs(x).mean(1, keepdims=True)
    var = (h * h).mean(1, keepdims=True) + eps
    r = 1.0 / np.sqrt(var)
    g, b = np.ones((rows, dim)), np.zeros((rows, dim))
    if gain is not None:
        g = np.repeat(gain, rows // len(gain), 0)
    if shift is not None:
        b = np.repeat(shift, rows // len(shift), 0)
    y = h * r * g + b
    # the factor: its own rounding, and h's errors in the mean of the squares
    of_r = 2 + np.sqrt((size * size).mean(1, keepdims=True) / var)
    bound = U * ((2 * size + (of_r + 3) * np.abs(h)) * r * np.abs(g) + np.abs(y) + np.abs(b))
    return x, y, 1.01 * bound


def check(out, got, y, bound):
    """got: norm_output's buffers on the host."""
    rows, dim = y.shape
    if out in DTYPES:
        err = np.abs(f64(got).reshape(rows, dim) - y)
        assert (err <= bound + half_step(np.abs(y) + bound, out)).all(), err.max()
        return
    codes, scale = f64(got[0]).reshape(rows, dim), f64(got[1])
    if out == "fp8_row":
        top = np.abs(y).max(1)
        want = np.where(top > 0, np.maximum(top / 448, 2.0 ** -126), 1.0)
        assert (np.abs(scale - want) <= bound.max(1) / 448 + 2 * U * want).all()
        step = np.repeat(scale[:, None], dim, 1)
    else:
        width = -(-dim // 32)
        e = np.log2(scale.reshape(rows, width))
        assert (e == np.rint(e)).all()
        pad = np.zeros((rows, width * 32))
        pad[:, :dim] = np.abs(y)
        slack = np.zeros((rows, width * 32))
        slack[:, :dim] = bound
        top, slack = (v.reshape(rows, width, 32).max(2) for v in (pad, slack))
        assert (top <= 448 * 2.0 ** e + slack).all()
        assert ((top + slack > 448 * 2.0 ** (e - 1)) | (e == -120)).all()
        step = np.repeat(2.0 ** e, 32, 1)[:, :dim]
    err = np.abs(codes * step - y)
    # half a step: 2^-4 of the value, 2^-10 of the scale near zero; the row's
    # factor adds two fp32 roundings
    assert (err <= np.maximum((np.abs(y) + bound) * (2.0 ** -4 + 4 * U), step * 2.0 ** -10)
            + bound).all(), err.max()


def make(rows, dim, n, dtype, x_dtype, groups, seed):
    g = torch.Generator().manual_seed(seed)
    srcs = [(torch.randn(rows, dim, generator=g) * 2).to(DTYPES[dtype]) for _ in range(n)]
    x = (torch.randn(rows, dim, generator=g) * 3 + 0.5).to(DTYPES[x_dtype])
    gain = torch.randn(groups, dim, generator=g) * 0.3 + 1 if groups else None
    shift = torch.randn(groups, dim, generator=g) * 0.3 if groups else None
    return srcs, x, gain, shift


def cuda(*ts):
    return [None if t is None else t.cuda() for t in ts]


DIMS = [1, 3, 4, 31, 32, 33, 64, 100, 128, 129, 255, 256, 511, 768, 1000, 1152, 1155, 1537, 2049,
        4100, 6145, 9000, 16384]


@pytest.mark.parametrize("out", ["bf16", "f16", "f32", "mxfp8", "fp8_row"])
@pytest.mark.parametrize("dim", DIMS)
def test_add_norm_dims(dim, out):
    """Every row length, with rows that fill no block."""
    for rows, kind, dtype, x_dtype in ((1, "rms", "bf16", "f32"), (37, "layer", "f16", "bf16"),
                                       (6, "rms", "f32", "f16")):
        print(f"norm {rows}x{dim} {kind} {dtype} {x_dtype} {out}", flush=True)
        groups = 3 if rows == 6 else 1
        srcs, x, gain, shift = make(rows, dim, 2, dtype, x_dtype, groups, dim + rows)
        w = [0.75, -1.25]
        dev = cuda(*srcs)
        x_in, g, b = cuda(x, gain, shift)
        x_out, y = cheb.add_norm(dev, w, torch.empty_like(x_in), x_in, kind=kind, eps=EPS, gain=g,
                                 shift=b, out=DTYPES.get(out, out))
        want_x, want, bound = reference([f64(s) for s in srcs], w, f64(x), kind, f64(gain),
                                        f64(shift))
        # one rounding to fp32, one to the residual's type
        off = np.abs(f64(x_out) - want_x)
        assert (off <= half_step(want_x, "f32") + half_step(np.abs(want_x) * (1 + U),
                                                            x_dtype)).all(), off.max()
        check(out, y, want, bound)
        again = cheb.add_norm(dev, w, x_in, x_in, kind=kind, eps=EPS, gain=g, shift=b,
                              out=DTYPES.get(out, out))      # in place
        for p, q in zip((again[0],) + (again[1] if isinstance(y, tuple) else (again[1],)),
                        (x_out,) + (y if isinstance(y, tuple) else (y,))):
            assert torch.equal(p.view(torch.uint8), q.view(torch.uint8))


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("given", ["sources", "residual", "both"])
def test_add_norm_optional(given, kind):
    """No residual, no sources, no gain, no shift, no kept residual."""
    srcs, x, gain, shift = make(13, 160, 3, "bf16", "f32", 1, 4)
    w = [1.0, -2.0, 0.5]
    use = srcs if given != "residual" else []
    x_use = x if given != "sources" else None
    for g, b in ((None, None), (gain, None), (None, shift)):
        dev = cuda(*use)
        xd, gd, bd = cuda(x_use, g, b)
        x_out, y = cheb.add_norm(dev, w[:len(use)], None, xd, dim=160, kind=kind, gain=gd,
                                 shift=bd, out=torch.float32)
        assert x_out is None
        host = [f64(s) for s in use] or [np.zeros((13, 160))]
        _, want, bound = reference(host, w if use else [0.0], None if x_use is None else f64(x_use),
                                   kind, None if g is None else f64(g),
                                   None if b is None else f64(b))
        check("f32", y, want, bound)


@pytest.mark.parametrize("quant", [None, "mxint8", "mxfp8"])
@pytest.mark.parametrize("layout", ["slots", "interleaved"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim,first,n", [(1152, 0, 3), (1155, 5, 2), (7, 3, 8), (96, 64, 1),
                                         (2052, 8, 5)])
def test_residual_norm(dim, first, n, dtype, layout, quant):
    """Sources from a history: a middle tensor, rows that start anywhere in it
    and run across chunks, groups and blocks, in all layouts and formats."""
    print(f"residual_norm {dim} {first} {n} {dtype} {layout} {quant}", flush=True)
    rows = max(5, 60000 // dim)
    sizes = [777, first + rows * dim + 3, 64]
    g = torch.Generator().manual_seed(dim + n)
    steps = [[(torch.randn(m, generator=g) * 2).to(DTYPES[dtype]) for m in sizes]
             for _ in range(n)]
    cache = cheb.ChebCache(n, DTYPES[dtype], sizes, layout=layout, quant=quant)
    for k, segs in enumerate(steps):
        cache.push(float(k), cuda(*segs))
    w = np.random.default_rng(n).normal(size=n)
    x = torch.randn(rows, dim, generator=g) * 3
    gain = torch.rand(dim, generator=g) + 0.5
    held = [f64(s[1]) for s in steps]
    if quant is not None:
        held = [ref.entry([h], quant)[:len(h)] for h in held]
    srcs = [h[first:first + rows * dim].reshape(rows, dim) for h in held]
    want_x, want, bound = reference(srcs, w, f64(x), "rms", f64(gain)[None], None)
    for out in ("f32", "mxfp8"):
        x_in, gd = cuda(x, gain)
        x_out, y = cache.residual_norm(w, 1, torch.empty_like(x_in), x_in, dim=dim, first=first,
                                       rows=rows, eps=EPS, gain=gd, out=DTYPES.get(out, out))
        assert (np.abs(f64(x_out) - want_x) <= half_step(want_x, "f32") * 1.01).all()
        check(out, y, want, bound)
    cache.close()


@pytest.mark.parametrize("layout", ["slots", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_residual_is_residual_apply_16(dtype, layout):
    """x_out is cheb_residual_apply's bit for bit over 16-bit entries too."""
    numel = 7 * 768
    cache = cheb.ChebCache(3, DTYPES[dtype], [numel], layout=layout)
    g = torch.Generator().manual_seed(2)
    for k in range(3):
        cache.push(float(k), [torch.randn(numel, generator=g).to(DTYPES[dtype]).cuda()])
    x = torch.randn(numel, generator=g).cuda()
    w = [1.7, -3.3, 2.6]
    x_out, _ = cache.residual_norm(w, 0, torch.empty_like(x), x, dim=768)
    assert torch.equal(cache.residual_apply(w, [0], torch.empty_like(x), x), x_out)
    cache.close()


@pytest.mark.parametrize("layout", ["slots", "interleaved"])
def test_residual_is_residual_apply(layout):
    """x_out is cheb_residual_apply's bit for bit, and a history's."""
    n, numel, dim = 4, 5 * 1152, 1152
    g = torch.Generator().manual_seed(1)
    steps = [torch.randn(numel, generator=g).cuda() for _ in range(n)]
    x = torch.randn(numel, generator=g).cuda()
    cache = cheb.ChebCache(n, torch.float32, [numel], layout=layout)
    hist = cheb.ResidualHistory(n, [0], numel)
    for k, s in enumerate(steps):
        cache.push(float(k), [s])
        hist.push(float(k), [s])
    w = cheb.precompute_weights(cache.history(), [4.5])[0]
    plain = cache.residual_apply(w, [0], torch.empty_like(x), x)
    x_out, _ = cache.residual_norm(w, 0, torch.empty_like(x), x, dim=dim)
    assert torch.equal(plain, x_out)
    x_hist, y, w_hist = hist.predict_norm(4.5, torch.empty_like(x), x, dim=dim, kind="layer",
                                          out="mxfp8")
    assert torch.equal(plain, x_hist) and (w_hist == w).all()
    # rows from the middle on: the same rows
    x_part, y_part, _ = hist.predict_norm(4.5, None, x[2 * dim:4 * dim], dim=dim, first=2 * dim,
                                          rows=2, kind="layer", out="mxfp8")
    assert x_part is None
    assert torch.equal(y_part[0].view(torch.uint8), y[0][2:4].view(torch.uint8))
    assert torch.equal(y_part[1].view(torch.uint8), y[1][2:4].view(torch.uint8))
    cache.close()
    hist.close()


@pytest.mark.parametrize("dim", [40, 200, 1152, 2500, 7000])
def test_rows_that_are_not_finite(dim):
    """Zeros, values whose squares pass fp32's range, NaN and infinities: each
    stays in its row, and 8-bit outputs say NaN by their scale."""
    g = torch.Generator().manual_seed(dim)
    x = torch.randn(9, dim, generator=g)
    x[1] = 0.0
    x[2] *= 1e25
    x[3] *= 1e-30
    x[4, dim // 2] = float("nan")
    x[6, 1] = float("inf")
    x[7] *= 1e-3
    want_x, want, bound = reference([f64(x)], [1.0], None, "rms", None, None)
    fine = [0, 1, 2, 3, 5, 7, 8]
    for out in ("f32", "mxfp8", "fp8_row"):
        _, y = cheb.add_norm([x.cuda()], [1.0], out=DTYPES.get(out, out))
        if out == "f32":
            # eps is far above the squares of row 3
            check("f32", y[fine], want[fine], bound[fine])
            assert not np.isfinite(f64(y)[4]).any() and np.isnan(f64(y)[6, 1])
            assert (f64(y)[1] == 0).all()
            continue
        codes, scale = y
        check(out, (codes[fine], scale[fine]), want[fine], bound[fine])
        assert np.isnan(f64(scale)[4]).all() and (f64(codes)[4] == 0).all()
        if out == "fp8_row":
            assert np.isnan(f64(scale)[6]) and f64(scale)[1] == 1.0
        else:
            assert np.isnan(f64(scale)[6, 0]) and (f64(scale)[1] == 2.0 ** -120).all()


@pytest.mark.parametrize("dim", [40, 1155])
def test_no_rows_with_a_gain(dim):
    empty = torch.empty(0, dim, dtype=torch.bfloat16, device="cuda")
    gain = torch.ones(dim, device="cuda")
    for out in (torch.bfloat16, "fp8_row"):
        _, y = cheb.add_norm([empty], [1.0], None, empty, gain=gain, shift=gain, out=out)
        assert (y if isinstance(y, torch.Tensor) else y[0]).shape == (0, dim)


def test_refusals_of_outputs():
    x = torch.ones(4, 64, device="cuda")
    codes, scale = cheb.norm_output(4, 64, "mxfp8")
    for out in (None, (codes,), codes, (codes, codes), (codes[:3], scale), (codes, scale[:3]),
                (codes.t(), scale), (codes.cpu(), scale), torch.ones(4, 64), "bf16", torch.int8):
        with pytest.raises(cheb.ChebError):
            cheb.add_norm([x], [1.0], out=out)
    assert cheb.add_norm([x], [1.0], out=[codes, scale])[1][0] is codes


def test_no_rows_and_views():
    """No rows; and rows taken from the middle of larger tensors, whose
    neighbours stay as they were."""
    empty = torch.empty(0, 1155, dtype=torch.float16, device="cuda")
    x_out, y = cheb.add_norm([empty], [1.0], empty.clone(), empty.clone(), out="mxfp8")
    assert y[0].shape == (0, 1155) and y[1].shape == (0, 37)
    big = torch.randn(8, 1155, device="cuda").half()
    src, x = big[1:4], big[5:8].clone()
    dest = torch.full((5, 1155), 7.0, dtype=torch.float16, device="cuda")
    codes = torch.full((5, 1155), 7.0, device="cuda").to(torch.float8_e4m3fn)
    scale = torch.full((5,), 9.0, device="cuda")
    cheb.add_norm([src], [1.0], dest[1:4], x, out=(codes[1:4], scale[1:4]))
    for t in (dest, codes.float()):
        assert (t[0] == 7).all() and (t[4] == 7).all() and not (t[1:4] == 7).all()
    assert scale[0] == 9 and scale[4] == 9
    assert torch.equal(dest[1:4], (src.double() + x.double()).float().half())


@pytest.mark.parametrize("dim,out", [(1152, "mxfp8"), (1155, "fp8_row")])
def test_rows_past_32_bits(dim, out):
    """Element numbers past 2^32: the last rows are what a call on them alone
    gives, bit for bit, and rows before them what zeros give."""
    print(f"rows_past_32_bits {dim} {out}", flush=True)
    rows, last = (1 << 32) // dim + 50, 37
    src = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(last, dim, generator=torch.Generator().manual_seed(dim)).bfloat16().cuda()
    src[-last:] = tail
    codes, scale = cheb.norm_output(rows, dim, out)
    x = src.clone()
    cheb.add_norm([src], [1.5], x, x, out=(codes, scale))
    x_want, (want, want_scale) = cheb.add_norm([tail], [1.5], torch.empty_like(tail), tail, out=out)
    assert torch.equal(x[-last:], x_want) and not x[:-last].any()
    assert torch.equal(codes[-last:].view(torch.uint8), want.view(torch.uint8))
    assert torch.equal(scale[-last:].float(), want_scale.float())
    assert not codes[:-last].view(torch.uint8).any()


@pytest.mark.parametrize("quant", [None, "mxint8", "mxfp8"])
@pytest.mark.parametrize("layout", ["slots", "interleaved"])
def test_residual_norm_past_32_bits(layout, quant):
    """The end of a cached tensor of more than 2^32 elements."""
    print(f"residual_norm_past_32_bits {layout} {quant}", flush=True)
    dim, numel = 1152, (1 << 32) + 40 * 1152
    first = numel - 40 * dim
    g = torch.Generator().manual_seed(4)
    parts = [torch.randn(40 * dim, generator=g).bfloat16().cuda() for _ in range(2)]
    small = cheb.ChebCache(2, torch.bfloat16, [40 * dim], layout=layout, quant=quant)
    large = cheb.ChebCache(2, torch.bfloat16, [numel], layout=layout, quant=quant)
    whole = torch.zeros(numel, dtype=torch.bfloat16, device="cuda")
    for k, p in enumerate(parts):
        small.push(float(k), [p])
        whole[first:] = p
        large.push(float(k), [whole])
    del whole
    w = [-1.5, 2.5]
    want_x, want = small.residual_norm(w, 0, torch.empty(40 * dim, device="cuda"), dim=dim)
    x, y = large.residual_norm(w, 0, torch.empty(40 * dim, device="cuda"), dim=dim, first=first)
    assert torch.equal(x, want_x) and torch.equal(y, want)
    small.close()
    large.close()
