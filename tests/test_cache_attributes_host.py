"""Measures of plain entries asked of an 8-bit cache are refused by the library's
own error, and are still attributes that it lacks (no GPU)."""
import pytest

import paper_2608_23429_amd as cheb
from test_stream_buffers_host import cache

NAMES = ["slot_stride_bytes", "chunk_elems", "entry_stride_elems"]


@pytest.mark.parametrize("name", NAMES)
def test_refused_for_8bit_entries(name):
    with pytest.raises(cheb.ChebError) as e:
        getattr(cache("mxint8"), name)
    assert e.value.name == "CHEB_E_INVAL" and "read()" in str(e.value)
    assert not hasattr(cache("mxint8"), name)


@pytest.mark.parametrize("name", NAMES + ["no_such_name"])
def test_others_lack_them_plainly(name):
    for c in (cache(), object.__new__(cheb.ChebCache)):
        with pytest.raises(AttributeError) as e:
            getattr(c, name)
        assert not isinstance(e.value, cheb.ChebError)
