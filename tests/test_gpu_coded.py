"""Histories of 8-bit entries on the GPU: what a push stores and a read gives
back, predictions and residual updates from such entries, against the formats'
definition in fp64."""
import numpy as np
import pytest
import torch

import coded_ref as ref
import paper_2608_23429_amd as cheb

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -9, "f16": 2.0 ** -12, "f32": 2.0 ** -25}  # of the value, normal range
RAGGED = [5, 0, 4097, 1, 12295, 4096, 31, 8192 + 513]
QUANTS = ("mxint8", "mxfp8")
LAYOUTS = ("slots", "interleaved")


def values(sizes, dtype, seed, scale=1.0):
    """One step's tensors: normal values with a few channels many times the
    others."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for n in sizes:
        x = torch.randn(n, generator=g) * scale
        x[::37] *= 30.0
        out.append(x.to(DTYPES[dtype]))
    return out


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy().reshape(-1)


def fill(cache, steps):
    for k, segs in enumerate(steps):
        cache.push(float(k), [s.cuda() for s in segs])


def half_steps(y, dtype):
    """Half a step of the storage type at the values y."""
    tiny = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}[dtype]
    return np.maximum(np.abs(y) * 2 * HALF_STEP[dtype], tiny)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("quant", QUANTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_store_and_read(dtype, quant, layout):
    """Every element of every held entry is what the format says, exactly, at
    sizes that end anywhere in a block, and the padding is zero."""
    print(f"store {dtype} {quant} {layout}", flush=True)
    steps = [values(RAGGED, dtype, 11 + k) for k in range(4)]
    cache = cheb.ChebCache(3, DTYPES[dtype], RAGGED, layout=layout, quant=quant)
    assert cache.seg_offset == ref.offsets(RAGGED)[0]
    cache.arena.fill_(0xA5)
    fill(cache, steps)                                   # the first one is evicted
    for idx in range(3):
        got = f64(cache.read(idx))
        want = ref.entry([f64(s) for s in steps[1 + idx]], quant)
        np.testing.assert_array_equal(got, want)
        np.testing.assert_array_equal(f64(cache.entry(idx)), got)
    cache.close()


def special(dtype):
    """Groups of 32 at the formats' borders: zeros, one value, limits of the
    exponent's choice, ties, subnormals, the type's largest, infinities and
    NaN, and a finite group between two that are not."""
    t = torch.finfo(DTYPES[dtype])
    rows = [torch.zeros(32), -torch.zeros(32)]
    for top in (1.0, 127 / 64, 1.9921875, 448.0, 449.0, 452.0, 464.0, 480.0, 2.0 ** -14, t.tiny,
                t.smallest_normal / 8):
        r = torch.linspace(-1, 1, 32, dtype=torch.float64) * top
        r[5] = top
        rows.append(r)
    ties = torch.arange(32, dtype=torch.float64) + 0.5
    rows += [ties / 64, -ties / 64, ties * 2.0 ** -9, torch.full((32,), t.max / 4)]
    for bad in (float("nan"), float("inf"), -float("inf")):
        r = torch.linspace(-1, 1, 32)
        r[17] = bad
        rows += [r, torch.linspace(-2, 2, 32)]
    return torch.stack([r.double() for r in rows]).to(DTYPES[dtype]).reshape(-1)


@pytest.mark.parametrize("quant", QUANTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_store_borders(dtype, quant):
    print(f"borders {dtype} {quant}", flush=True)
    x = special(dtype)
    cache = cheb.ChebCache(1, DTYPES[dtype], [x.numel()], quant=quant)
    cache.push(0.0, [x.cuda()])
    got = f64(cache.read(0))[:x.numel()]
    want = ref.held(f64(x), quant)
    np.testing.assert_array_equal(got, want)
    cache.close()


def test_store_largest():
    """At fp32's largest magnitudes MXINT8 keeps the code at 127 and the sign."""
    x = torch.zeros(64)
    x[0], x[1], x[33] = torch.finfo(torch.float32).max, -torch.finfo(torch.float32).max, 2.0 ** 127
    cache = cheb.ChebCache(1, torch.float32, [64], quant="mxint8")
    cache.push(0.0, [x.cuda()])
    got = f64(cache.read(0))[:64]
    np.testing.assert_array_equal(got, ref.held(f64(x), "mxint8"))
    assert got[0] == 127 * 2.0 ** 121 and got[1] == -got[0]
    cache.close()


@pytest.mark.parametrize("quant", QUANTS)
def test_store_near_the_largest(quant):
    """Beside fp32's largest values small ones and zeros keep their own: a scale
    of 2^120 or more takes no other factor past the range."""
    x = torch.zeros(96)
    x[0], x[1], x[2] = 3.0e38, -2.9e38, 1.0
    x[40] = 1.5e38
    x[70] = torch.finfo(torch.float32).max
    cache = cheb.ChebCache(1, torch.float32, [96], quant=quant)
    cache.push(0.0, [x.cuda()])
    with np.errstate(over="ignore"):
        want = ref.held(f64(x), quant).astype(np.float32).astype(np.float64)
    np.testing.assert_array_equal(f64(cache.read(0))[:96], want)
    np.testing.assert_array_equal(f64(cache.extrapolate([1.0]))[:96], want)
    cache.close()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_read_plain_cache(dtype, layout):
    """cheb_cache_read gives a plain cache's entries bit for bit."""
    steps = [values(RAGGED, dtype, 3 + k) for k in range(3)]
    cache = cheb.ChebCache(2, DTYPES[dtype], RAGGED, layout=layout)
    fill(cache, steps)
    for idx in range(2):
        got = cache.read(idx)
        assert torch.equal(got.view(torch.uint8), cache.entry(idx).contiguous().view(torch.uint8))
        for v, s in zip(cache.segment_views(got), steps[1 + idx]):
            assert torch.equal(v.cpu(), s)
    cache.close()


@pytest.mark.parametrize("quant", QUANTS)
def test_one_group_not_finite(quant):
    """A NaN stays in its group of 32 through predictions and residual updates,
    whatever its entry's weight."""
    steps = [values([4096], "bf16", k) for k in range(2)]
    steps[0][0][100] = float("nan")
    cache = cheb.ChebCache(2, torch.bfloat16, [4096], quant=quant)
    fill(cache, steps)
    x = torch.randn(4096, device="cuda")
    for w in ([0.0, 1.0], [2.0, -1.0]):
        out = f64(cache.extrapolate(w))
        res = f64(cache.residual_apply(w, [0], torch.empty_like(x), x))
        for v in (out, res):
            assert np.isnan(v[96:128]).all() and np.isfinite(np.delete(v, slice(96, 128))).all()
    cache.close()


@pytest.mark.parametrize("waves", [-1, 3, 9])
def test_launch_config_reaches_coded(waves):
    """The tuning interface's cap changes no result."""
    steps = [values([300000], "bf16", k) for k in range(3)]
    cache = cheb.ChebCache(3, torch.bfloat16, [300000], quant="mxint8", layout="interleaved")
    fill(cache, steps)
    x = torch.randn(300000, device="cuda")
    want = [cache.extrapolate([1.0, -2.0, 3.0]),
            cache.residual_apply([1.0, -2.0, 3.0], [0], torch.empty_like(x), x)]
    try:
        cheb.cheb_set_launch_config(**dict(cheb.DEFAULT_LAUNCH_CONFIG, waves_per_cu=waves))
        assert torch.equal(cache.extrapolate([1.0, -2.0, 3.0]), want[0])
        assert torch.equal(cache.residual_apply([1.0, -2.0, 3.0], [0], torch.empty_like(x), x),
                           want[1])
    finally:
        cheb.cheb_set_launch_config(**cheb.DEFAULT_LAUNCH_CONFIG)
    cache.close()


def rows(n, m, seed):
    return np.random.default_rng(seed).normal(size=(m, n)) * 3


@pytest.mark.parametrize("quant", QUANTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,m,layout", [(1, 1, "slots"), (2, 1, "interleaved"), (3, 2, "slots"),
                                        (4, 8, "interleaved"), (5, 1, "slots"),
                                        (6, 1, "interleaved"), (6, 3, "interleaved"),
                                        (7, 4, "slots"), (8, 1, "interleaved"), (8, 8, "slots")])
def test_predict(n, m, layout, dtype, quant):
    """out = sum_k w_k value_k.  Weights rounded to fp32 and n products and
    sums in fp32: (n + 2) 2^-24 of the sum of magnitudes, and half a step of
    the output's type (fp32 caches: all in fp64)."""
    print(f"predict {n} {m} {layout} {dtype} {quant}", flush=True)
    sizes = [40961, 333, 70000]
    steps = [values(sizes, dtype, 100 * n + k) for k in range(n)]
    cache = cheb.ChebCache(n, DTYPES[dtype], sizes, layout=layout, quant=quant)
    fill(cache, steps)
    w = rows(n, m, n + m)
    outs = cache.extrapolate_multi(w) if m > 1 else [cache.extrapolate(w[0])]
    held = np.stack([ref.entry([f64(s) for s in segs], quant) for segs in steps])
    for row, out in zip(w, outs):
        want, size = row @ held, np.abs(row) @ np.abs(held)
        sums = (n + 2) * 2.0 ** (-24 if dtype != "f32" else -53) * size
        err = np.abs(f64(out) - want)
        assert (err <= sums + half_steps(np.abs(want) + sums, dtype)).all(), err.max()
        assert (f64(out)[ref.offsets(sizes)[0][1] + 333:ref.offsets(sizes)[0][2]] == 0).all()
    cache.close()


def residual_case(kind):
    """(tensor sizes, residual offsets, residual elements)."""
    if kind == "dit":
        return [4608] * 9, [0] * 9, 4608
    if kind == "token":
        return [8], [0], 8
    if kind == "joint":                          # text and image parts, and joint tensors
        img, txt = 5 * 1152, 333 * 8
        return [img, txt] * 3 + [img + txt] * 5, [txt, 0] * 3 + [0] * 5, img + txt
    # tensors that overlap in part, one that is not added, one that is empty,
    # more than one launch's table holds
    return [1024, 2048, 0, 512] * 40, [8, 1016, 0, -1] * 40, 4096


@pytest.mark.parametrize("quant", QUANTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind,n,layout", [("token", 1, "slots"), ("dit", 3, "interleaved"),
                                           ("dit", 2, "slots"), ("joint", 6, "interleaved"),
                                           ("joint", 8, "slots"), ("parts", 4, "interleaved"),
                                           ("joint", 1, "interleaved")])
def test_residual(kind, n, layout, dtype, quant):
    """x_out = x_in + the tensors' predictions: each one's sum in fp32, (n + 2)
    2^-24 of its magnitudes, and half a step of the fp32 residual."""
    print(f"residual {kind} {n} {layout} {dtype} {quant}", flush=True)
    sizes, off, numel = residual_case(kind)
    steps = [values(sizes, dtype, 7 * n + k) for k in range(n)]
    cache = cheb.ChebCache(n, DTYPES[dtype], sizes, layout=layout, quant=quant)
    fill(cache, steps)
    w = rows(n, 1, n)[0]
    x = torch.randn(numel, generator=torch.Generator().manual_seed(5)) * 4
    held = np.stack([ref.entry([f64(s) for s in segs], quant) for segs in steps])
    want, size = f64(x), np.abs(f64(x))
    for o, at, cnt in zip(off, cache.seg_offset, sizes):
        if o >= 0:
            want[o:o + cnt] += w @ held[:, at:at + cnt]
            size[o:o + cnt] += np.abs(w) @ np.abs(held[:, at:at + cnt])
    x_in = x.cuda()
    out = cache.residual_apply(w, off, torch.empty_like(x_in), x_in)
    bound = (n + 2) * 2.0 ** -24 * size
    err = np.abs(f64(out) - want)
    assert (err <= bound + half_steps(np.abs(want) + bound, "f32")).all(), err.max()
    np.testing.assert_array_equal(f64(cache.residual_apply(w, off, x_in, x_in)), f64(out))
    alone = cache.residual_apply(w, off, torch.empty_like(x_in))
    err = np.abs(f64(alone) + f64(x) - want)
    assert (err <= 2 * bound + half_steps(np.abs(want) + bound, "f32") + 2.0 ** -24 * size).all()
    cache.close()
