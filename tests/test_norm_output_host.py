"""A norm's output that is not what norm_output gives is refused with the
library's error, whatever it is (no GPU)."""
import pytest
import torch

import paper_2608_23429_amd as cheb
from test_stream_buffers_host import card, on_card  # noqa: F401



@pytest.mark.parametrize("out", [
    lambda: (None, on_card(2, 2, dtype=torch.float8_e8m0fnu)),
    lambda: ("codes", on_card(2)), lambda: (3, 4), lambda: [None, None],
    lambda: (on_card(2, 64, dtype=torch.float8_e4m3fn), None), lambda: 5, lambda: (1, 2, 3)])
def test_output_of_other_kinds(card, out):  # noqa: F811
    with pytest.raises(cheb.ChebError):
        cheb.add_norm([on_card(2, 64)], [1.0], out=out())


@pytest.mark.parametrize("form", ["mxfp8", "fp8_row", torch.bfloat16])
def test_output_of_norm_output(card, form):  # noqa: F811
    out = cheb.norm_output(2, 64, form)
    assert cheb.add_norm([on_card(2, 64)], [1.0], out=out)[1] is out
