"""8-bit histories and the norm as a sampler uses them: full steps stored,
skipped steps predicted, applied to the residual and normed, on streams and in
captured graphs."""
import numpy as np
import pytest
import torch

import coded_ref as ref
import paper_2608_23429_amd as cheb
from test_gpu_norm import EPS, check, reference

pytestmark = pytest.mark.gpu

DIM, TXT, IMG, BLOCKS = 128, 33, 150, 2


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def layout():
    img, txt = IMG * DIM, TXT * DIM
    return ([img, txt] * BLOCKS + [img + txt] * BLOCKS, [txt, 0] * BLOCKS + [0] * BLOCKS,
            img + txt)


def step(sizes, t, seed):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) + t * torch.randn(n, generator=g)).bfloat16()
            for n in sizes]


@pytest.mark.parametrize("quant", ["mxint8", "mxfp8"])
def test_sampling_run(quant):
    """A schedule of full and skipped steps: every skipped step's prediction by
    the offline table, its residual and the norm of the image tokens agree with
    fp64 on what the entries hold, on a stream of its own."""
    sizes, off, numel = layout()
    T, n = 14, 3
    table = cheb.ChebTable(T, 1, 1, 3, n, [float(T - s) for s in range(T)])
    cache = cheb.ChebCache(n, torch.bfloat16, sizes, layout="interleaved", quant=quant)
    gain = (torch.rand(DIM, generator=torch.Generator().manual_seed(9)) + 0.5).cuda()
    x = torch.randn(numel, generator=torch.Generator().manual_seed(3)).cuda()
    held, skipped = [], 0
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for s in range(T):
            predicted, nodes, w = table.step(s)
            if not predicted:
                segs = step(sizes, 1.0 - s / T, 50 + s)
                cache.push(float(T - s), [v.cuda() for v in segs])
                held = (held + [ref.entry([f64(v) for v in segs], quant)])[-n:]
                continue
            skipped += 1
            out = cache.extrapolate_steps(table, s)[0]
            x_out = cache.residual_apply(w, off, torch.empty_like(x), x)
            img = x_out[TXT * DIM:].view(IMG, DIM)
            _, y = cheb.add_norm([], [], None, img, kind="rms", eps=EPS, gain=gain, out="mxfp8")
            stream.synchronize()
            entry = np.stack(held)
            want, size = w @ entry, np.abs(w) @ np.abs(entry)
            assert (np.abs(f64(out) - want) <= (n + 2) * 2.0 ** -24 * size
                    + np.maximum(np.abs(want) * 2.0 ** -8 * 1.01, 2.0 ** -134)).all()
            res, bound = f64(x), np.abs(f64(x))
            for o, at, cnt in zip(off, cache.seg_offset, sizes):
                res[o:o + cnt] += want[at:at + cnt]
                bound[o:o + cnt] += size[at:at + cnt]
            assert (np.abs(f64(x_out) - res) <= (n + 3) * 2.0 ** -24 * bound).all()
            _, y64, off_y = reference([f64(img)], [1.0], None, "rms", f64(gain)[None], None)
            check("mxfp8", y, y64, off_y)
    assert skipped >= 4
    cache.close()


def test_replayed_graph():
    """A full step and the skipped step after it, captured once: every replay
    gives what the same calls give eagerly, with new inputs in the same buffers
    and the program's own work between replays."""
    sizes, off, numel = layout()
    n = 2
    cache = cheb.ChebCache(n, torch.bfloat16, sizes, quant="mxint8")
    hist = cheb.ResidualHistory(n, [0], numel)
    segs = [torch.empty(m, dtype=torch.bfloat16, device="cuda") for m in sizes]
    x, x_out = torch.empty(numel, device="cuda"), torch.empty(numel, device="cuda")
    out = cache.new_output()
    y, scale = cheb.norm_output(numel // DIM, DIM, "mxfp8")
    w = [-0.5, 1.5]

    def fresh(seed):
        for t, v in zip(segs, step(sizes, 0.3, seed)):
            t.copy_(v)
        x.copy_(torch.randn(numel, generator=torch.Generator().manual_seed(seed)))

    def calls():
        cache.extrapolate(w, out)
        cache.residual_apply(w, off, x_out, x)
        hist.predict_norm(2.5, x_out, x_out, dim=DIM, kind="layer", out=(y, scale))

    def result():
        torch.cuda.synchronize()
        return [t.clone().view(torch.uint8) for t in (out, x_out, y, scale)]

    for k in range(n):                            # the ring's places in turn
        fresh(k)
        cache.push(float(k), segs)
        hist.push(float(k), [x])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()                                   # once before the capture
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in range(5):
        fresh(100 + seed)
        cache.reset()
        hist.cache.reset()
        for k in range(n):                        # same places, new entries
            fresh(100 + 10 * seed + k)
            cache.push(float(k), segs)
            hist.push(float(k), [x])
        calls()
        want = result()
        for t in (out, x_out, y, scale):
            t.view(torch.uint8).fill_(seed)
        torch.cuda.synchronize()
        graph.replay()
        for a, b in zip(want, result()):
            assert torch.equal(a, b)
    cache.close()
    hist.close()


def test_captured_push():
    """A push can be captured: each replay stores what the buffers then hold."""
    sizes = [5000, 77]
    cache = cheb.ChebCache(1, torch.float16, sizes, quant="mxfp8", layout="interleaved")
    segs = [torch.zeros(m, dtype=torch.float16, device="cuda") for m in sizes]
    out = cache.new_output()
    cache.push(0.0, segs)
    cache.read(0, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.push(1.0, segs)
        cache.read(0, out)
    for seed in range(4):
        host = [torch.randn(m, generator=torch.Generator().manual_seed(seed)).half()
                for m in sizes]
        for t, v in zip(segs, host):
            t.copy_(v)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(f64(out), ref.entry([f64(v) for v in host], "mxfp8"))
    cache.close()


def test_two_streams_two_caches():
    """Two caches worked on at once from two streams do not meet."""
    sizes = [300000]
    caches = [cheb.ChebCache(2, torch.bfloat16, sizes, quant=q) for q in ("mxint8", "mxfp8")]
    streams = [torch.cuda.Stream() for _ in caches]
    data = [[torch.randn(300000, generator=torch.Generator().manual_seed(7 * i + k)).bfloat16()
             for k in range(2)] for i in range(2)]
    dev = [[t.cuda() for t in d] for d in data]
    torch.cuda.synchronize()
    outs = [None, None]
    for k in range(2):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                caches[i].push(float(k), [dev[i][k]])
    for i in (0, 1):
        outs[i] = caches[i].extrapolate([0.0, 1.0], stream=streams[i])
    torch.cuda.synchronize()
    for i, q in enumerate(("mxint8", "mxfp8")):
        np.testing.assert_array_equal(f64(outs[i]), ref.entry([f64(data[i][1])], q))


def test_other_device_refused(monkeypatch):
    """A tensor that is not on the current device is refused, not launched on
    the wrong one."""
    x = torch.randn(4, 64, device="cuda")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: x.device.index + 1)
    with pytest.raises(cheb.ChebError) as e:
        cheb.add_norm([x], [1.0], out=torch.empty_like(x))
    assert e.value.name == "CHEB_E_INVAL"
    with pytest.raises(cheb.ChebError) as e:
        cheb.add_norm([], [], x, x, out=torch.empty_like(x))
    assert e.value.name == "CHEB_E_INVAL"
    cache = cheb.ChebCache(1, torch.float32, [256], device=x.device, quant="mxint8")
    for call in (lambda: cache.push(0.0, [x]), lambda: cache.read(0),
                 lambda: cache.extrapolate([1.0]), lambda: cache.extrapolate_multi([[1.0]]),
                 lambda: cache.extrapolate_at(0.5), lambda: cache.extrapolate_at_multi([0.5]),
                 lambda: cache.residual_apply([1.0], [0], x),
                 lambda: cache.residual_norm([1.0], 0, dim=64)):
        with pytest.raises(cheb.ChebError) as e:
            call()
        assert e.value.name == "CHEB_E_INVAL" and "current device" in str(e.value)


def test_python_refuses():
    x = torch.randn(6, 64, device="cuda")
    g = torch.ones(4, 64, device="cuda")
    y8 = cheb.norm_output(6, 64, "mxfp8")

    def refused(name, call):
        with pytest.raises(cheb.ChebError) as e:
            call()
        assert e.value.name == name, str(e.value)
    refused("CHEB_E_MISMATCH", lambda: cheb.add_norm([x], [1.0], None, x[:5]))
    refused("CHEB_E_MISMATCH", lambda: cheb.add_norm([x, x[:5]], [1.0, 1.0]))
    refused("CHEB_E_MISMATCH", lambda: cheb.add_norm([x], [1.0], x.half(), x))
    refused("CHEB_E_MISMATCH", lambda: cheb.add_norm([x], [1.0], dim=50))
    refused("CHEB_E_MISMATCH", lambda: cheb.add_norm([x], [1.0], gain=g))           # 6 rows in 4
    refused("CHEB_E_MISMATCH", lambda: cheb.add_norm([x], [1.0], gain=g[:2], shift=g[:3]))
    refused("CHEB_E_MISMATCH", lambda: cheb.add_norm([x], [1.0], gain=g[0].half()))
    refused("CHEB_E_MISMATCH", lambda: cheb.add_norm([x], [1.0], out=y8[0][:5].float()))
    refused("CHEB_E_MISMATCH", lambda: cheb.add_norm([x], [1.0], out=(y8[0], y8[1][:5])))
    refused("CHEB_E_INVAL", lambda: cheb.add_norm([x], [1.0], kind="batch"))
    refused("CHEB_E_INVAL", lambda: cheb.add_norm([x.t()], [1.0]))                 # strided
    refused("CHEB_E_INVAL", lambda: cheb.add_norm([x], [1.0, 2.0]))
    refused("CHEB_E_DTYPE", lambda: cheb.add_norm([x.double()], [1.0]))
    refused("CHEB_E_DTYPE", lambda: cheb.add_norm([x], [1.0], out="mxint8"))
    cache = cheb.ChebCache(2, torch.float32, [640], quant="mxfp8")
    for k in range(2):
        cache.push(float(k), [x.reshape(-1)[:640 - 256].repeat(2)[:640].contiguous()])
    refused("CHEB_E_INVAL", lambda: cache.residual_norm([1.0, 2.0], 1, dim=64))
    refused("CHEB_E_INVAL", lambda: cache.residual_norm([1.0], 0, dim=64))
    refused("CHEB_E_INVAL", lambda: cache.residual_norm([1.0, 2.0], 0, dim=64, first=641))
    refused("CHEB_E_INVAL", lambda: cache.residual_norm([1.0, 2.0], 0, dim=64, rows=11))
    refused("CHEB_E_INVAL", lambda: cache.residual_norm([1.0, 2.0], 0, dim=0))
    refused("CHEB_E_INVAL", lambda: cache.begin_push())
    refused("CHEB_E_MISMATCH", lambda: cache.read(0, torch.empty(10, device="cuda")))
    refused("CHEB_E_INVAL", lambda: cache.read(2))
    cache.close()
