"""Entries are read on the current device only, whatever their format (no GPU:
the stand-ins of the buffers' tests)."""
import pytest
import torch

import paper_2608_23429_amd as cheb
from test_stream_buffers_host import SIDE, Stream, cache, card, on_card  # noqa: F401


class Elsewhere(Stream):
    device = torch.device("cuda", 1)


@pytest.mark.parametrize("quant", [None, "mxint8"])
def test_read_on_another_device_refused(card, monkeypatch, quant):  # noqa: F811
    c, out = cache(quant), on_card(128, dtype=torch.bfloat16)
    assert c.read(0, out) is out and c.read(0, out, stream=SIDE) is out
    with pytest.raises(cheb.ChebError) as e:
        c.read(0, out, stream=Elsewhere())
    assert e.value.name == "CHEB_E_INVAL"
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(cheb.ChebError) as e:
        c.read(0, out)
    assert e.value.name == "CHEB_E_INVAL" and "current device" in str(e.value)
