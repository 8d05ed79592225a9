"""Residual updates from 8-bit entries over many tiles: every launch shape, the
tiles that share lines of scales, ragged last tiles, and residuals past 2^32
elements."""
import pytest
import torch

import paper_2608_23429_amd as cheb

pytestmark = pytest.mark.gpu

# entries, tensors, residual elements: one, two, four and eight waves a tile, on
# both sides of every rule, with tiles past the last whole 128 and past 4096
SHAPES = [(4, 1, 700 * 512 + 8), (2, 3, 300 * 512 + 504), (1, 20, 129 * 512 + 16),
          (1, 30, 200 * 512 + 8), (3, 5, 700 * 512 + 24), (3, 24, 1152 * 512), (2, 24, 4096 * 512),
          (5, 24, 4096 * 512 + 8), (8, 25, 1000 * 512 + 248), (6, 30, 127 * 512 + 40)]


@pytest.mark.parametrize("quant", ["mxint8", "mxfp8"])
@pytest.mark.parametrize("layout", ["slots", "interleaved"])
@pytest.mark.parametrize("n,tensors,numel", SHAPES)
def test_residual_of_many_tiles(n, tensors, numel, layout, quant):
    """Against fp64 sums of what the entries hold: half a step of the result and
    an fp64 rounding for each term."""
    print(f"tiles {n} {tensors} {numel} {layout} {quant}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(n * tensors)
    cache = cheb.ChebCache(n, torch.float32, [numel] * tensors, layout=layout, quant=quant)
    w = [(-1.0) ** k * (1.37 + k) for k in range(n)]
    want = torch.randn(numel, generator=g, device="cuda").double()
    x, size = want.float(), want.abs()
    for k in range(n):
        cache.push(float(k), [torch.randn(numel, generator=g, device="cuda")
                              for _ in range(tensors)])
    want, size = x.double(), x.double().abs()
    for k in range(n):
        for v in cache.segment_views(cache.read(k)):     # exact: an fp32 cache
            want += w[k] * v.double()
            size += abs(w[k]) * v.double().abs()
    out = cache.residual_apply(w, [0] * tensors, torch.empty_like(x), x)
    bound = want.abs() * 2.0 ** -24 + 4 * (n * tensors + 8) * 2.0 ** -53 * size
    assert ((out.double() - want).abs() <= bound).all()
    assert torch.equal(cache.residual_apply(w, [0] * tensors, x, x), out)    # in place
    cache.close()


@pytest.mark.parametrize("layout", ["slots", "interleaved"])
def test_residual_past_32_bits(layout):
    """Two tensors of more than 2^32 elements, where tiles are one wave's: places
    on both sides are what a small residual gives, the rest is zero."""
    print(f"residual past 32 bits {layout}", flush=True)
    numel, piece = (1 << 32) + (5 << 12), 13 << 12
    places = [0, (1 << 31) - 4096, numel - piece]
    g = torch.Generator().manual_seed(6)
    parts = [torch.randn(piece, generator=g).bfloat16().cuda() for _ in places]
    src = torch.zeros(numel, dtype=torch.bfloat16, device="cuda")
    for at, p in zip(places, parts):
        src[at:at + piece] = p
    w = [1.37]
    small = cheb.ChebCache(1, torch.bfloat16, [piece] * 2, layout=layout, quant="mxint8")
    large = cheb.ChebCache(1, torch.bfloat16, [numel] * 2, layout=layout, quant="mxint8")
    large.push(0.0, [src, src])
    del src
    out = large.residual_apply(w, [0, 0], torch.empty(numel, device="cuda"))
    for at, p in zip(places, parts):
        small.push(float(at), [p, p])
        want = small.residual_apply(w, [0, 0], torch.empty(piece, device="cuda"))
        assert torch.equal(out[at:at + piece], want)
        out[at:at + piece] = 0
    assert not out.view(torch.int32).any()
    small.close()
    large.close()
