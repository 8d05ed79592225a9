"""e4m3 rows with one scale: the codes are the fp32 quotients of y and the
row's scale, rounded to nearest even, and the scale is max|y| / 448."""
import numpy as np
import pytest
import torch

import paper_2608_23429_amd as cheb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [4, 40, 255, 1155, 4100])
def test_codes_are_quotients(dim):
    """Over the y that the same call gives in fp32, bit for bit.  An fp32
    reciprocal moves about one code in a million."""
    print(f"row codes {dim}", flush=True)
    rows = (12 << 20) // dim
    g = torch.Generator(device="cuda").manual_seed(dim)
    x = torch.randn(rows, dim, generator=g, device="cuda")
    x[3], x[5] = 0.0, x[5] * 1e-22
    gain = torch.rand(dim, generator=g, device="cuda") + 0.5
    _, y = cheb.add_norm([x], [1.0], gain=gain, out=torch.float32)
    _, (codes, scale) = cheb.add_norm([x], [1.0], gain=gain, out="fp8_row")
    y, got, s = y.cpu().numpy(), codes.float().cpu().numpy(), scale.cpu().numpy()
    top = np.abs(y).max(1)
    want_s = np.where(top > 0, np.maximum(top / np.float32(448), np.float32(2.0 ** -126)),
                      np.float32(1))
    np.testing.assert_array_equal(s, want_s)
    q = (y / s[:, None]).astype(np.float64)            # numpy's fp32 division, then exact
    step = np.ldexp(1.0, np.maximum(np.frexp(q)[1] - 1, -6) - 3)
    np.testing.assert_array_equal(got.astype(np.float64), np.rint(q / step) * step)
