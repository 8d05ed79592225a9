"""How many bits the calls over 8-bit entries keep: residual updates against
exact sums, the two calls that update a residual against one another, and
values near fp32's largest with weights that take products past it."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import coded_ref as ref
import paper_2608_23429_amd as cheb

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
QUANTS = ("mxint8", "mxfp8")
LAYOUTS = ("slots", "interleaved")


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy().reshape(-1)


def ring(steps, dtype, quant, layout="slots"):
    """A full cache of these steps' tensors, and what its entries hold."""
    cache = cheb.ChebCache(len(steps), DTYPES[dtype], [s.numel() for s in steps[0]],
                           layout=layout, quant=quant)
    for k, segs in enumerate(steps):
        cache.push(float(k), [s.cuda() for s in segs])
    return cache, np.stack([ref.entry([f64(s) for s in segs], quant) for segs in steps])


def tensors(sizes, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * 3).to(DTYPES[dtype]) for n in sizes]


# Sampler times of a shifted schedule: Lagrange weights that are no short
# binary fractions, up to some hundreds.
def shifted_weights(n):
    t = np.linspace(1.0, 0.1, 3 * n + 2)
    t = 3.0 * t / (1.0 + 2.0 * t)
    return cheb.precompute_weights(t[:3 * n:3], [t[3 * n - 1]])[0]


@pytest.mark.parametrize("quant", QUANTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,tensors_,numel,layout", [
    (1, 1, 4608, "slots"), (3, 9, 4608, "interleaved"), (4, 2, 70000, "slots"),
    (6, 30, 1160, "interleaved"), (8, 56, 4096, "slots"), (8, 5, 33000, "interleaved")])
def test_residual_sums(n, tensors_, numel, layout, dtype, quant):
    """x_out = x_in + sum over tensors and entries, in fp64 with one rounding to
    fp32: half a step of the result, and an fp64 rounding for each term added
    (their products with a code are exact up to that) of the magnitudes' sum."""
    print(f"residual sums {n} {tensors_} {numel} {layout} {dtype} {quant}", flush=True)
    sizes = [numel] * tensors_
    cache, held = ring([tensors(sizes, dtype, 31 * n + k) for k in range(n)], dtype, quant, layout)
    w = shifted_weights(n)
    x = torch.randn(numel, generator=torch.Generator().manual_seed(n)) * 4
    at = np.array(cache.seg_offset)[:, None] + np.arange(numel)
    terms = np.concatenate([w[:, None, None] * held[:, at]], 0).reshape(n * tensors_, numel)
    size = np.abs(terms).sum(0) + np.abs(f64(x))
    want = f64(x) + terms.sum(0)                      # numpy's own roundings: as many again
    x_in = x.cuda()
    out = f64(cache.residual_apply(w, [0] * tensors_, torch.empty_like(x_in), x_in))
    slack = 2 * (n * tensors_ + 17) * 2.0 ** -53 * size
    assert (np.abs(out - want) <= np.maximum(np.abs(want), 2.0 ** -126) * 2.0 ** -24 + slack).all()
    cache.close()


def test_residual_sum_of_one_element():
    """The bound above to the last bit, by rational numbers: the exact sum of
    eight entries rounded once."""
    n = 8
    cache, held = ring([tensors([64], "f32", 5 + k) for k in range(n)], "f32", "mxint8")
    w = shifted_weights(n)
    x = torch.randn(64, generator=torch.Generator().manual_seed(1))
    x_in = x.cuda()
    out = f64(cache.residual_apply(w, [0], torch.empty_like(x_in), x_in))
    for i in range(64):
        exact = Fraction(float(x[i])) + sum(Fraction(float(a)) * Fraction(float(h))
                                            for a, h in zip(w, held[:, i]))
        size = abs(x[i]) + sum(abs(float(a) * float(h)) for a, h in zip(w, held[:, i]))
        assert abs(Fraction(float(out[i])) - exact) <= (
            abs(exact) * Fraction(2) ** -24 + Fraction(float(size)) * (n + 1) * Fraction(2) ** -53)
    cache.close()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("quant", QUANTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 3, 6, 8])
def test_residual_norm_is_residual_apply(n, dtype, quant, layout):
    """One cached tensor added to the residual: both calls give the same bits."""
    print(f"same bits {n} {dtype} {quant} {layout}", flush=True)
    numel = 45 * 768
    cache, _ = ring([tensors([numel], dtype, n + k) for k in range(n)], dtype, quant, layout)
    w = shifted_weights(n)
    x = torch.randn(numel, generator=torch.Generator().manual_seed(n)).cuda()
    x_out, _ = cache.residual_norm(w, 0, torch.empty_like(x), x, dim=768)
    assert torch.equal(cache.residual_apply(w, [0], torch.empty_like(x), x), x_out)
    cache.close()


def large(dtype):
    """Groups with values near the largest that fp32 (fp16) holds beside zeros
    and small ones, at two steps whose 2 a - b is in range."""
    top = 3.3e38 if dtype != "f16" else 6e4
    a, b = torch.zeros(96, dtype=torch.float64), torch.zeros(96, dtype=torch.float64)
    a[3], b[3] = 0.55 * top, 0.62 * top
    a[4], b[4] = -0.9 * top, -0.97 * top
    a[5], b[5] = 1.0, 1.0
    a[40], b[41] = 0.4 * top, 0.4 * top
    a[70], b[70] = 0.99 * top, 0.99 * top
    return [[a.to(DTYPES[dtype])], [b.to(DTYPES[dtype])]]


@pytest.mark.parametrize("quant", QUANTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_residual_of_large_values(dtype, quant):
    """Products past fp32's range that cancel, and zeros beside them, in both
    calls that update a residual."""
    cache, held = ring(large(dtype), dtype, quant)
    x = torch.linspace(-1, 1, 96)
    x_in = x.cuda()
    for w in ([2.0, -1.0], [1024.0, -1023.5], [3.0e5, -2.0e5], [1e-3, 0.0]):
        want = f64(x) + np.array(w) @ held[:, :96]
        with np.errstate(over="ignore"):
            rounded = want.astype(np.float32).astype(np.float64)
        for out in (cache.residual_apply(w, [0], torch.empty_like(x_in), x_in),
                    cache.residual_norm(w, 0, torch.empty_like(x_in), x_in, dim=96)[0]):
            out = f64(out)
            fine = np.isfinite(rounded)
            # both sums are of three fp64 terms
            off = 4 * 2.0 ** -53 * (np.abs(f64(x)) + np.abs(np.array(w)) @ np.abs(held[:, :96]))
            assert (np.abs(out - want) <= np.abs(want) * 2.0 ** -24 + off)[fine].all()
            np.testing.assert_array_equal(out[~fine], rounded[~fine])
    cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_residual_of_the_largest_value(dtype):
    """MXFP8 rounds fp32's largest value to 2^128, which every call but a read
    takes for what it is."""
    x = torch.zeros(64)
    x[5], x[9] = torch.finfo(DTYPES[dtype]).max, -1.5e38
    cache, held = ring([[x.to(DTYPES[dtype])]], dtype, "mxfp8")
    assert held[0, 5] == 2.0 ** 128
    r = torch.linspace(-1e37, 1e37, 64).cuda()
    want = (f64(r) + 0.25 * held[0, :64]).astype(np.float32)   # one rounding: exact in fp64
    for out in (cache.residual_apply([0.25], [0], torch.empty_like(r), r),
                cache.residual_norm([0.25], 0, torch.empty_like(r), r, dim=64)[0]):
        np.testing.assert_array_equal(f64(out), want.astype(np.float64))
    cache.close()


@pytest.mark.parametrize("quant", QUANTS)
def test_weights_past_fp32_refused(quant):
    cache, _ = ring([tensors([64], "f32", k) for k in range(2)], "f32", quant)
    x = torch.zeros(64, device="cuda")
    for call in (lambda w: cache.residual_apply(w, [0], x),
                 lambda w: cache.residual_norm(w, 0, dim=64)):
        call([3e38, -3e38])
        with pytest.raises(cheb.ChebError) as e:
            call([1.0, 4e38])
        assert e.value.name == "CHEB_E_NONFINITE"
    cache.close()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("quant", QUANTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_predict_of_large_values(dtype, quant, layout):
    """Zeros and small values beside ones near the largest, with weights whose
    product with the group's scale leaves fp32's range: an element whose own
    terms are in range is right.  The bound is that of any prediction: weights
    rounded, n products and sums, and half a step of the output's type."""
    print(f"predict large {dtype} {quant} {layout}", flush=True)
    cache, held = ring(large(dtype), dtype, quant, layout)
    held = held[:, :96]
    top = float(torch.finfo(DTYPES[dtype]).max)
    tiny, rel = {"bf16": (2.0 ** -134, 2.0 ** -8), "f16": (2.0 ** -25, 2.0 ** -11),
                 "f32": (2.0 ** -150, 2.0 ** -24)}[dtype]
    rows = np.array([[2.0, -1.0], [1024.0, -1023.5], [3.0e5, -2.0e5], [1e-3, 0.5], [0.0, 1.0]])
    outs = [f64(cache.extrapolate(w)) for w in rows]
    outs += [f64(o) for o in cache.extrapolate_multi(rows[:4])]
    for w, out in zip(np.concatenate([rows, rows[:4]]), outs):
        want, size = w @ held, np.abs(w) @ np.abs(held)
        fine = size < top * 0.99
        assert fine.sum() >= 80
        off = (len(w) + 2) * 2.0 ** (-53 if dtype == "f32" else -24) * size
        err = np.abs(out[:96] - want)
        assert (err <= off + np.maximum(np.abs(want) * rel, tiny) * 1.01)[fine].all()
        assert (out[96:] == 0).all()
    cache.close()


def test_predict_of_weights_past_fp32():
    """An fp32 cache's weights are fp64 of any size: terms that cancel, and
    zeros beside one that no fp64 number holds."""
    a, b = torch.zeros(64), torch.zeros(64)
    a[0], b[0], a[40] = 2.0 ** -100, 2.0 ** -100, 2.0 ** 100
    cache, _ = ring([[a], [b]], "f32", "mxfp8")
    out = f64(cache.extrapolate([2.0 ** 1000, -2.0 ** 1000]))[:64]
    assert out[40] == np.inf and not np.delete(out, 40).any()
    cache.close()


@pytest.mark.parametrize("quant,limit", [("mxint8", 2.0 ** 7), ("mxfp8", 2.0 ** 8)])
def test_predict_of_weights_at_the_limit(quant, limit):
    """Weights that fp32 rounds up to where they are divided."""
    x = torch.zeros(64)
    x[3], x[40] = torch.finfo(torch.bfloat16).max, 1.0
    cache, _ = ring([[x.bfloat16()]], "bf16", quant)
    for w in (limit * (1 - 2.0 ** -30), limit, limit * (1 - 2.0 ** -24)):
        out = f64(cache.extrapolate([w]))[:64]
        assert out[3] == np.inf and out[40] == limit and not np.delete(out, [3, 40]).any()
    cache.close()
