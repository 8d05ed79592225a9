"""The 8-bit entry formats from their definition, in fp64 (numpy): what an
entry of groups of 32 elements holds for given values."""
import numpy as np

BLOCK = 4096                     # elements a cached tensor is padded to


def padded(n):
    return -(-n // BLOCK) * BLOCK


def offsets(sizes):
    """Where tensors of those sizes start, and the entry's size."""
    ends = np.cumsum([0] + [padded(n) for n in sizes])
    return [int(o) for o in ends[:-1]], int(ends[-1])


def near_e4m3(v):
    """Nearest e4m3 value (largest 448, smallest 2^-9), ties to even."""
    k = np.frexp(v)[1] - 1                       # |v| in [2^k, 2^(k+1))
    step = np.ldexp(1.0, np.maximum(k, -6) - 3)
    return np.rint(v / step) * step


def exponents(top, limit):
    """Least e with top <= limit 2^e, kept within [-120, 127]."""
    e = np.full(top.shape, -120)
    for k in range(-120, 127):
        e += top > limit * 2.0 ** k
    return e


def groups(x, quant):
    """(code values, exponents, finite) of x in groups of 32."""
    g = np.asarray(x, dtype=np.float64).reshape(-1, 32)
    finite = np.isfinite(g).all(1)
    g = np.where(finite[:, None], g, 0.0)
    top = np.abs(g).max(1)
    if quant == "mxint8":
        e = exponents(top, 127 / 64)
        q = np.clip(np.rint(g / np.ldexp(1.0, e - 6)[:, None]), -127, 127)
    else:
        e = exponents(top, 448.0)
        q = near_e4m3(g / np.ldexp(1.0, e)[:, None])
    return q, e, finite


def held(x, quant):
    """The values an entry holds for x (whole groups of 32), fp64; a group
    with a NaN or an infinity is NaN."""
    q, e, finite = groups(x, quant)
    unit = np.ldexp(1.0, e - 6 if quant == "mxint8" else e)
    v = q * unit[:, None]
    v[~finite] = np.nan
    return v.reshape(-1)


def entry(segments, quant):
    """A whole entry: every tensor (fp64 values) padded with zeros."""
    off, size = offsets([len(s) for s in segments])
    x = np.zeros(size)
    for o, s in zip(off, segments):
        x[o:o + len(s)] = s
    return held(x, quant)
