"""Outputs that calls make on a stream other than the current one, whose blocks
neither stream may take while the other still works on them."""
import pytest
import torch

import paper_2608_23429_amd as cheb

pytestmark = pytest.mark.gpu

N = 4 << 20


def filled(quant=None):
    cache = cheb.ChebCache(1, torch.bfloat16, [N], quant=quant)
    cache.push(0.0, [torch.full((N,), 3.0, dtype=torch.bfloat16, device="cuda")])
    torch.cuda.synchronize()
    return cache


def calls(cache, stream):
    x = torch.full((N // 1024, 1024), 3.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    return {
        "read": lambda: cache.read(0, stream=stream),
        "extrapolate": lambda: cache.extrapolate([1.0], stream=stream),
        "extrapolate_multi": lambda: cache.extrapolate_multi([[1.0]], stream=stream)[0],
        "add_norm": lambda: cheb.add_norm([x], [1.0], eps=0.0, stream=stream)[1],
        "residual_norm": lambda: cache.residual_norm([1.0], 0, dim=1024, eps=0.0,
                                                     stream=stream)[1],
    }


@pytest.mark.parametrize("quant", [None, "mxint8"])
@pytest.mark.parametrize("name", ["read", "extrapolate", "extrapolate_multi", "add_norm",
                                  "residual_norm"])
def test_block_freed_on_the_current_stream(name, quant):
    """A block that the current stream has just freed, and still reads, is not
    what a call on another stream writes to."""
    print(f"freed block {name} {quant}", flush=True)
    cache, stream = filled(quant), torch.cuda.Stream()
    call = calls(cache, stream)[name]
    total = torch.zeros(N, device="cuda")
    block = torch.full((N,), 1.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    for _ in range(64):
        total += block
    at = block.data_ptr()
    del block
    y = call()
    assert y.data_ptr() != at
    torch.cuda.synchronize()
    assert (total == 64).all()
    assert (y == (1.0 if "norm" in name else 3.0)).all()
    cache.close()


@pytest.mark.parametrize("name", ["read", "extrapolate", "add_norm"])
def test_output_dropped_while_the_current_stream_reads_it(name):
    """An output made on another stream, read on the current one and dropped:
    the next call's writes do not reach it before that."""
    print(f"dropped output {name}", flush=True)
    cache, stream = filled(), torch.cuda.Stream()
    call = calls(cache, stream)[name]
    want = 1.0 if "norm" in name else 3.0
    total = torch.zeros(N, device="cuda")
    torch.cuda.synchronize()
    y = call()
    torch.cuda.current_stream().wait_stream(stream)
    for _ in range(64):
        total += y.view(-1)
    del y
    with torch.cuda.stream(stream):
        torch.zeros(N, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    assert (total == 64 * want).all()
    cache.close()
