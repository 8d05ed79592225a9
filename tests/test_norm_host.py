"""What the norm calls refuse, checked before any GPU work (no GPU needed:
addresses that are never followed)."""
import numpy as np
import pytest
import torch

import paper_2608_23429_amd as cheb
from paper_2608_23429_amd import _binding

ROWS, DIM = 4, 64
BASE = 1 << 20                    # distinct buffers, 1 MiB apart


def at(i, off=0):
    return (i + 1) * BASE + off


def norm(**kw):
    v = dict(rows=ROWS, dim=DIM, eps=1e-6, x_in=at(0), x_out=at(1), gain=at(2), shift=at(3),
             rows_per_group=ROWS, y=at(4), y_scale=None, kind=cheb.CHEB_NORM_RMS,
             x_dtype=cheb.CHEB_F32, out_format=cheb.CHEB_BF16)
    v.update(kw)
    return cheb.cheb_norm(*[v[n] for n, _ in cheb.cheb_norm._fields_])


def refused(name, call):
    with pytest.raises(cheb.ChebError) as e:
        call()
    assert e.value.name == name, str(e.value)


BAD = [
    ("CHEB_E_INVAL", dict(kind=2)), ("CHEB_E_INVAL", dict(kind=-1)),
    ("CHEB_E_DTYPE", dict(x_dtype=3)), ("CHEB_E_DTYPE", dict(out_format=5)),
    ("CHEB_E_DTYPE", dict(out_format=18)),
    ("CHEB_E_INVAL", dict(rows=-1)), ("CHEB_E_INVAL", dict(rows=1 << 26)),
    ("CHEB_E_INVAL", dict(dim=0)), ("CHEB_E_INVAL", dict(dim=16385)),
    ("CHEB_E_INVAL", dict(rows=(1 << 26) - 1, dim=16384)),
    ("CHEB_E_INVAL", dict(eps=-1.0)), ("CHEB_E_INVAL", dict(eps=float("nan"))),
    ("CHEB_E_INVAL", dict(eps=float("inf"))),
    ("CHEB_E_INVAL", dict(rows_per_group=0)),
    ("CHEB_E_INVAL", dict(y=None)),
    ("CHEB_E_INVAL", dict(out_format=cheb.CHEB_OUT_MXFP8)),          # no scales
    ("CHEB_E_INVAL", dict(y_scale=at(5))),                           # scales of a storage type
    ("CHEB_E_ALIGN", dict(x_in=at(0, 2))), ("CHEB_E_ALIGN", dict(x_out=at(1, 2))),
    ("CHEB_E_ALIGN", dict(y=at(4, 1))), ("CHEB_E_ALIGN", dict(gain=at(2, 1))),
    ("CHEB_E_ALIGN", dict(shift=at(3, 2))),
    ("CHEB_E_ALIGN", dict(out_format=cheb.CHEB_OUT_FP8_ROW, y_scale=at(5, 2))),
    ("CHEB_E_INVAL", dict(x_out=at(0, 64))),                         # partly over x_in
    ("CHEB_E_INVAL", dict(y=at(0))), ("CHEB_E_INVAL", dict(y=at(1, 8))),
    ("CHEB_E_INVAL", dict(y=at(2))), ("CHEB_E_INVAL", dict(y=at(3, 128))),
    ("CHEB_E_INVAL", dict(out_format=cheb.CHEB_OUT_MXFP8, y_scale=at(4, 8))),
    ("CHEB_E_INVAL", dict(x_out=at(6, 64))), ("CHEB_E_INVAL", dict(y=at(6, 16))),
]


@pytest.mark.parametrize("name,kw", BAD)
def test_add_norm_refuses(name, kw):
    refused(name, lambda: cheb.cheb_add_norm([at(6)], [1.0], cheb.CHEB_BF16, norm(**kw)))


def test_add_norm_refuses_sources():
    ok = norm()
    refused("CHEB_E_INVAL", lambda: cheb.cheb_add_norm([at(6)] * 9, [1.0] * 9, 0, ok))
    refused("CHEB_E_INVAL", lambda: cheb.cheb_add_norm([0], [1.0], 0, ok))
    refused("CHEB_E_INVAL", lambda: cheb.cheb_add_norm([at(6)], [1.0, 2.0], 0, ok))
    refused("CHEB_E_ALIGN", lambda: cheb.cheb_add_norm([at(6, 1)], [1.0], 0, ok))
    refused("CHEB_E_DTYPE", lambda: cheb.cheb_add_norm([at(6)], [1.0], 7, ok))
    refused("CHEB_E_NONFINITE", lambda: cheb.cheb_add_norm([at(6)], [float("nan")], 0, ok))
    refused("CHEB_E_INVAL", lambda: cheb.cheb_add_norm([], [], 0, norm(x_in=None)))
    rc = _binding.LIB.cheb_add_norm(None, 0, None, 0, None, None)
    assert rc == _binding.CHEB_E_INVAL
    # no rows: nothing to do, whatever the buffers
    cheb.cheb_add_norm([], [], 0, norm(rows=0, y=None))


class Ring:
    """A full plain cache whose arena is never touched: entries recorded by
    fused pushes, which launch nothing."""

    def __init__(self, sizes, n=2, dtype=cheb.CHEB_F32, fill=True):
        need, _ = cheb.cheb_cache_arena_bytes(n, dtype, sizes)
        self.arena = 1 << 40
        self.h = cheb.cheb_cache_create(n, dtype, sizes, self.arena, need)
        for k in range(n if fill else n - 1):
            cheb.cheb_cache_begin_push(self.h)
            cheb.cheb_cache_commit(self.h, float(k))


@pytest.mark.parametrize("name,kw", [c for c in BAD if 6 not in
                                     [(v or 0) // BASE - 1 for k, v in c[1].items()
                                      if k in ("x_out", "y")]])
def test_residual_norm_refuses(name, kw):
    r = Ring([ROWS * DIM])
    if "rows" in kw and kw["rows"] > 0 and "dim" not in kw:
        name = "CHEB_E_INVAL"
    refused(name, lambda: cheb.cheb_residual_norm(r.h, [1.0, 2.0], 0, 0, norm(**kw)))
    cheb.cheb_cache_destroy(r.h)


def test_residual_norm_refuses_places():
    r = Ring([100, ROWS * DIM + 8])
    w = [1.0, 2.0]

    def call(seg=1, first=0, w=w, **kw):
        return lambda: cheb.cheb_residual_norm(r.h, w, seg, first, norm(**kw))
    for bad in (call(seg=2), call(seg=-1), call(seg=0), call(first=9), call(first=-1),
                call(first=1 << 62), call(rows=5), call(y=r.arena), call(x_out=r.arena + 64)):
        refused("CHEB_E_INVAL", bad)
    refused("CHEB_E_NONFINITE", call(w=[1.0, float("inf")]))
    cheb.cheb_residual_norm(r.h, w, 1, 8, norm(rows=0, y=None))
    cheb.cheb_cache_begin_push(r.h)
    refused("CHEB_E_NOTREADY", call())
    cheb.cheb_cache_abort_push(r.h)
    refused("CHEB_E_NOTREADY", call())          # the oldest entry is gone
    cheb.cheb_cache_destroy(r.h)
    assert _binding.LIB.cheb_residual_norm(None, None, 0, 0, None, None) == _binding.CHEB_E_INVAL
    r = Ring([ROWS * DIM], fill=False)
    refused("CHEB_E_NOTREADY", lambda: cheb.cheb_residual_norm(r.h, w, 0, 0, norm()))
    cheb.cheb_cache_destroy(r.h)


def test_python_refuses():
    x = torch.zeros(4, 64)
    refused("CHEB_E_INVAL", lambda: cheb.add_norm([x], [1.0]))            # host memory
    refused("CHEB_E_INVAL", lambda: cheb.add_norm([], []))
    refused("CHEB_E_INVAL", lambda: cheb.add_norm([], [], None, x))
    refused("CHEB_E_DTYPE", lambda: cheb.norm_output(4, 64, "int8", "cpu"))
    refused("CHEB_E_DTYPE", lambda: cheb.norm_output(4, 64, torch.int32, "cpu"))
    y, s = cheb.norm_output(4, 33, "mxfp8", "cpu")
    assert y.shape == (4, 33) and s.shape == (4, 2) and s.dtype == torch.float8_e8m0fnu
    y, s = cheb.norm_output(4, 33, "fp8_row", "cpu")
    assert y.dtype == torch.float8_e4m3fn and s.shape == (4,) and s.dtype == torch.float32
    assert cheb.norm_output(2, 3, torch.float16, "cpu").shape == (2, 3)
    assert np.isclose(_binding.CHEB_MAX_NORM_DIM, 16384)
