"""Timed cases of the 8-bit history and of the norm that follows a predicted
residual.

Four operators: a full step quantised as it is written into the history and
read back ("store"), the skipped step's prediction from 8-bit entries
("predict"), the residual update from them ("residual"), and the residual's
addition with a norm and an 8-bit output ("norm").  Sizes are those of the
workloads the repository is exercised on (DiT-XL/2, PixArt-Sigma, FLUX.1-dev
and the single-tensor one), plus odd token counts and ragged tensors.

8-bit entries are groups of 32 consecutive elements of a cached tensor with
one power-of-two scale 2^e, where e is the least integer with max |x| <= L 2^e
(L = 127/64 for int8, 448 for e4m3), kept within [-120, 127].  An int8 code
stands for code 2^(e - 6), an e4m3 code for its value times 2^e.
"""
import math
from fractions import Fraction

import numpy as np
import torch
import torch.nn.functional as F

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
STEPS = 50                       # sampling steps; abscissa of step s is 1 - s / STEPS
PAD = 4096                       # elements a cached tensor is padded to in an 8-bit entry


# -- the cases -----------------------------------------------------------------

def _case(name, op, family, n, dtype, quant, m=1, batch=1, tokens=1, text=0, hidden=1152,
          blocks=1, layout="interleaved"):
    c = {"op": op, "family": family, "n": n, "m": m, "dtype": dtype, "quant": quant,
         "batch": batch, "tokens": tokens, "text": text, "hidden": hidden, "blocks": blocks,
         "layout": layout}
    if name is not None:
        c["name"] = name
    return c


def _norm(name, source, n, dtype, x_dtype, rows, dim, kind, out, groups=0, shift=False):
    c = {"op": "norm", "source": source, "n": n, "dtype": dtype, "x_dtype": x_dtype,
         "rows": rows, "dim": dim, "kind": kind, "out": out, "groups": groups, "shift": shift}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # One small tensor stored and read back: the launches and the host
        # path count.
        _case("store_tiny", "store", "flat", 2, "f32", "mxint8", batch=2, tokens=256),
        # DiT blocks of an odd token count and width: ragged tensors, each
        # padded in the entry.
        _case("store_ragged", "store", "dit", 3, "f16", "mxfp8", batch=2, tokens=1001, hidden=1155,
              blocks=12),
        # FLUX.1-dev 1024x1024: a full step's 76 module outputs.
        _case("store_flux", "store", "flux", 2, "bf16", "mxint8", tokens=4096, text=512,
              hidden=3072, blocks=19),
        # DiT-XL/2 256x256, one image with guidance, one skipped step.
        _case("predict_dit256", "predict", "dit", 3, "bf16", "mxfp8", batch=2, tokens=256,
              blocks=28, layout="slots"),
        # FLUX.1-dev 1024x1024, one skipped step from six entries.
        _case("predict_flux", "predict", "flux", 6, "bf16", "mxint8", tokens=4096, text=512,
              hidden=3072, blocks=19),
        # PixArt-Sigma 1024x1024 in half precision: the three skipped steps
        # between two full ones from one pass.
        _case("predict_pixart1024", "predict", "dit", 6, "f16", "mxint8", m=3, batch=2,
              tokens=4096, blocks=28),
        # DiT-XL/2 256x256 for one image with guidance, applied to the
        # residual stream.
        _case("residual_dit256", "residual", "dit", 3, "bf16", "mxint8", batch=2, tokens=256,
              blocks=28),
        # FLUX.1-dev, applied to the residual stream of text and image.
        _case("residual_flux", "residual", "flux", 6, "bf16", "mxint8", tokens=4096, text=512,
              hidden=3072, blocks=19),
        # One token: a pooled vector's residual and its norm.
        _norm("norm_token", "add", 1, "bf16", "bf16", 1, 1152, "rms", "bf16", groups=1),
        # PixArt-Sigma 1024x1024, the predicted output of one module added to
        # the residual, then a norm with gain into the block format of a
        # scaled matrix product.
        _norm("norm_pixart1024", "module", 6, "bf16", "f32", 8192, 1152, "rms", "mxfp8", groups=1),
        # DiT-XL/2 512x512, batch 8 with guidance: the collapsed history's
        # prediction and the final adaptive layer norm, a row of gains and
        # shifts an image.
        _norm("norm_dit512", "collapsed", 4, "f32", "f32", 16384, 1152, "layer", "mxfp8",
              groups=16, shift=True),
        # A module's output added to a half-precision residual of an odd
        # width, one scale a row.
        _norm("norm_odd", "add", 1, "f16", "f16", 5003, 1155, "rms", "fp8_row", groups=1),
    ]


MAX_BYTES = 3e9                  # of a drawn case, under half the largest listed one
MIN_ENTRY, MAX_ENTRY = 5e5, 4e8  # elements of one entry


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more case: any operator, history of 1 to 8, up to 4 targets, every
    storage type, code and layout, entries of 5e5 to 4e8 elements, odd token
    counts and widths, norms of one row to 3e4."""
    while True:
        op = rng.choice(("store", "predict", "predict", "residual", "norm", "norm"))
        n = rng.choice((1, 2, 2, 3, 3, 4, 5, 6, 6, 7, 8))
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        if op == "norm":
            source = rng.choice(("add", "module", "collapsed"))
            dim = rng.choice((384, 768, 1152, 1152, 1536, 2304, rng.randint(1, 4096)))
            rows = int(_log(rng, 1, 3e4))
            groups = rng.choice((0, 1, 1, 2, 4))
            if rows < groups or (groups and rows % groups):
                rows += groups - rows % groups
            kind = rng.choice(("rms", "rms", "layer"))
            x_dtype = "f32" if source != "add" else rng.choice(("f32", "bf16", "f16"))
            c = _norm(None, source, n if source != "add" else 1,
                      "f32" if source == "collapsed" else dtype, x_dtype, rows, dim, kind,
                      rng.choice(("bf16", "f16", "f32", "mxfp8", "mxfp8", "fp8_row")), groups,
                      bool(groups) and rng.random() < 0.5)
        else:
            quant = rng.choice(("mxint8", "mxint8", "mxfp8"))
            layout = rng.choice(("slots", "interleaved", "interleaved"))
            family = rng.choice(("dit", "dit", "flux", "flat"))
            hidden = rng.choice((384, 768, 1152, 1152))
            if op != "residual" and rng.random() < 0.3:
                hidden = rng.choice((385, 771, 1155))
            size = _log(rng, MIN_ENTRY, MAX_ENTRY)
            blocks = {"dit": rng.randint(1, 28), "flux": rng.randint(1, 15), "flat": 1}[family]
            batch = rng.choice((1, 2, 2, 4, 16)) if family != "flux" else 1
            tokens = max(1, int(size / (hidden * batch * blocks * {"dit": 2, "flux": 3, "flat": 1}[family])))
            text = min(tokens, rng.choice((0, rng.randint(1, 511), 512))) if family == "flux" else 0
            c = _case(None, op, family, n, dtype, quant, rng.randint(1, 4) if op == "predict" else 1,
                      batch, tokens, text, hidden, blocks, layout)
        if work(c)["bytes"] <= MAX_BYTES:
            return c


# -- shapes and schedule ---------------------------------------------------------

def _segments(c):
    """Element counts of the cached tensors of one full step."""
    if c["family"] == "flat":
        return [c["batch"] * c["tokens"] * c["hidden"]]
    if c["family"] == "dit":
        return [c["batch"] * c["tokens"] * c["hidden"]] * (2 * c["blocks"])
    img, txt = c["tokens"] * c["hidden"], c["text"] * c["hidden"]
    return [img, txt] * c["blocks"] + [img + txt] * (2 * c["blocks"])


def _padded(n):
    return -(-n // PAD) * PAD


def _residual_map(c):
    """(residual offset of each cached tensor, residual elements): text
    tokens first, image tokens after them, joint tensors over both."""
    segs = _segments(c)
    if c["family"] != "flux":
        return [0] * len(segs), segs[0]
    img, txt = segs[0], segs[1]
    return [txt, 0] * c["blocks"] + [0] * (2 * c["blocks"]), img + txt


def _x(step):
    return 1.0 - step / STEPS


def _schedule(c):
    """(steps of the held entries, skipped steps)."""
    m = c.get("m", 1)
    r = 4 if m == 1 else m + 1
    nodes = [1 + r * j for j in range(c["n"])]
    return nodes, [nodes[-1] + 1 + j for j in range(m)]


def _weights(c):
    """Lagrange coefficients of the held abscissae at each target, exact and
    then rounded to fp64."""
    nodes, targets = _schedule(c)
    x = [Fraction(_x(v)) for v in nodes]
    rows = []
    for target in targets:
        t, row = Fraction(_x(target)), []
        for j, xj in enumerate(x):
            w = Fraction(1)
            for k, xk in enumerate(x):
                if k != j:
                    w *= (t - xk) / (xj - xk)
            row.append(float(w))
        rows.append(row)
    return np.array(rows, dtype=np.float64)


# -- inputs ----------------------------------------------------------------------

def _rng(seed, salt=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) + 1_000_003 * salt)
    return g


def _features(rows, hidden, dtype, steps, seed, salt=0):
    """Values of rows x hidden features at the given steps, one tensor a
    step: a random quadratic of the step per element plus noise, times a
    log-normal factor per channel (some channels of a transformer's features
    are many times the others), rounded once to the storage type."""
    g = _rng(seed, salt)
    size = (rows, hidden)
    amp = torch.randn(hidden, generator=g, device="cuda").mul_(0.7).exp_()
    c0, c1, c2 = (torch.randn(size, generator=g, device="cuda") for _ in range(3))
    for s in steps:
        v = torch.randn(size, generator=g, device="cuda").mul_(0.02)
        t = _x(s)
        v.add_(c0).add_(c1, alpha=t).add_(c2, alpha=t * t).mul_(amp)
        yield v.to(DTYPES[dtype]).reshape(-1)


def _entries(c, seed, steps):
    return _features(sum(_segments(c)) // c["hidden"], c["hidden"], c["dtype"], steps, seed)


def _residual_values(c, seed):
    """A residual stream before the block stack, fp32."""
    return torch.randn(_residual_map(c)[1], generator=_rng(seed, 1), device="cuda").mul_(3.0)


def _norm_inputs(c, seed):
    """(sources, residual, gain, shift) of a norm case."""
    rows, dim, groups = c["rows"], c["dim"], c["groups"]
    srcs = list(_features(rows, dim, c["dtype"], _schedule(c)[0], seed, 2))
    g = _rng(seed, 3)
    x = torch.randn(rows * dim, generator=g, device="cuda").mul_(3.0).to(DTYPES[c["x_dtype"]])
    gain = torch.randn(groups, dim, generator=g, device="cuda").mul_(0.3).add_(1.0) if groups else None
    shift = torch.randn(groups, dim, generator=g, device="cuda").mul_(0.3) if c["shift"] else None
    return srcs, x, gain, shift


# -- plain forms -----------------------------------------------------------------

def _pad_segments(x, sizes):
    """One entry with each cached tensor padded with zeros; its last
    dimension holds the tensors of `sizes` back to back."""
    if all(n % PAD == 0 for n in sizes):
        return x
    return torch.cat([F.pad(s, (0, _padded(s.shape[-1]) - s.shape[-1]))
                      for s in x.split(sizes, dim=-1)], dim=-1)


def _two(e):
    """2^e in fp32, e in [-126, 127]."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x, quant):
    """(codes, exponents) of fp32 values in groups of 32."""
    g = x.view(-1, 32)
    top = g.abs().amax(1)
    bits = top.view(torch.int32)
    limit, emax = (0x7E0000, 0) if quant == "mxint8" else (0x600000, 8)
    e = ((bits + (0x7FFFFF - limit)) >> 23) - 127 - emax
    e = e.clamp(-120, 127)
    if quant == "mxint8":
        codes = torch.round(g * _two(6 - e)[:, None]).clamp(-127, 127).to(torch.int8)
    else:
        codes = (g * _two(-e)[:, None]).to(torch.float8_e4m3fn)
    return codes.view(x.shape), e.to(torch.int8)


def _read(codes, e, quant):
    """fp32 values of the codes."""
    unit = _two(e.to(torch.int32) - (6 if quant == "mxint8" else 0))
    return (codes.view(*e.shape, 32).float() * unit[..., None]).view(codes.shape)


def _weighted(s):
    """sum_k w_k value_k of every target, [m, entry]; in 64 bits where the
    storage type keeps more than fp32 sums give."""
    t = torch.float64 if s["dtype"] == "f32" else torch.float32
    w = torch.as_tensor(s["w"], dtype=t, device="cuda")
    v = _read(s["codes"], s["e"], s["quant"]).to(t)
    return torch.stack([(v * row[:, None]).sum(0) for row in w])


def _norm_plain(s):
    rows, dim = s["rows"], s["dim"]
    x = s["x"].double()
    x = x + (torch.stack(s["srcs"]).double() * s["w64"][:, None]).sum(0)
    x = x.float()
    h = x.view(rows, dim)
    if s["kind"] == "layer":
        h = h - h.mean(1, keepdim=True)
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + s["eps"])
    if s["gain"] is not None:
        groups = s["gain"].shape[0]
        y = y.view(groups, rows // groups, dim) * s["gain"][:, None]
        y = y + s["shift"][:, None] if s["shift"] is not None else y
    y = y.reshape(rows, dim)
    out = {"x": x.to(DTYPES[s["x_dtype"]])}
    if s["out"] in DTYPES:
        return out | {"y": y.to(DTYPES[s["out"]]).view(-1)}
    if s["out"] == "fp8_row":
        scale = y.abs().amax(1) / 448.0
        scale = torch.where(scale > 0, scale, torch.ones_like(scale))
        return out | {"y": (y / scale[:, None]).to(torch.float8_e4m3fn).view(-1), "scale": scale}
    y = F.pad(y, (0, -dim % 32))
    codes, e = _quantise(y.reshape(-1), "mxfp8")
    return out | {"y": codes.view(rows, -1)[:, :dim].reshape(-1),
                  "scale": (e.to(torch.int32) + 127).to(torch.uint8).view(torch.float8_e8m0fnu)}


# -- the calls ---------------------------------------------------------------------

def prepare(case, seed):
    c = case
    nodes, targets = _schedule(c)
    s = {"op": c["op"], "dtype": c["dtype"], "w": _weights(c)}
    if c["op"] == "norm":
        srcs, x, gain, shift = _norm_inputs(c, seed)
        s |= {k: c[k] for k in ("rows", "dim", "kind", "out", "source", "x_dtype")}
        s |= {"eps": 1e-6, "srcs": srcs, "x": x, "gain": gain, "shift": shift,
              "target": _x(targets[0])}
        s["w"] = s["w"][0] if c["source"] != "add" else np.ones(1)
        s["w64"] = torch.as_tensor(s["w"], device="cuda")
        s["x_out"] = torch.empty_like(x)
        if own:
            # The outputs' buffers and the history, as a sampler keeps them.
            import paper_2608_23429_amd as cheb
            s["y"] = cheb.norm_output(c["rows"], c["dim"], _out_format(c["out"]), x.device)
            if c["source"] == "module":
                cache = cheb.ChebCache(c["n"], DTYPES[c["dtype"]], [x.numel()], layout="slots")
                for step, v in zip(nodes, srcs):
                    cache.push(_x(step), [v])
                s["cache"] = cache
            elif c["source"] == "collapsed":
                hist = cheb.ResidualHistory(c["n"], [0], x.numel())
                for step, v in zip(nodes, srcs):  # entries of any size, as they are
                    hist.cache.push(_x(step), [v])
                s["hist"] = hist
        return s
    segs = _segments(c)
    s |= {"sizes": segs, "quant": c["quant"]}
    steps = nodes if c["op"] != "store" else nodes[:1]
    if own:
        import paper_2608_23429_amd as cheb
        s["cache"] = cheb.ChebCache(c["n"], DTYPES[c["dtype"]], segs, layout=c["layout"],
                                    quant=c["quant"])
    if c["op"] == "store":
        # A full step's tensors, each an allocation of its own.
        s["segs"] = [v.clone() for v in next(_entries(c, seed, steps)).split(segs)]
        s["t"] = 0.0
        if own:
            # A full ring, whose oldest entry makes room at every full step.
            s["out"], s["newest"] = s["cache"].new_output(), c["n"] - 1
            for k in range(c["n"]):
                s["cache"].push(1.0 + c["n"] - k, s["segs"])
        return s
    if own:
        for step, v in zip(nodes, _entries(c, seed, nodes)):
            s["cache"].push(_x(step), [t.clone() for t in v.split(segs)])
        s["outs"] = [s["cache"].new_output() for _ in targets] if c["op"] == "predict" else None
    else:
        held = [_quantise(_pad_segments(v, segs).float(), c["quant"])
                for v in _entries(c, seed, nodes)]
        s["codes"], s["e"] = (torch.stack(list(t)) for t in zip(*held))
    if c["op"] == "residual":
        s["off"], _ = _residual_map(c)
        s["family"], s["blocks"] = c["family"], c["blocks"]
        s["x"] = _residual_values(c, seed)
        s["x_out"] = torch.empty_like(s["x"])
    return s


def _out_format(name):
    return DTYPES.get(name, name)


def _run_own(s):
    if s["op"] == "store":
        s["t"] -= 1.0                          # the next full step
        s["cache"].push(s["t"], s["segs"])
        return {"entry": s["cache"].read(s["newest"], s["out"])}
    if s["op"] == "predict":
        if len(s["outs"]) == 1:
            return {"out": [s["cache"].extrapolate(s["w"][0], s["outs"][0])]}
        return {"out": s["cache"].extrapolate_multi(s["w"], s["outs"])}
    if s["op"] == "residual":
        return {"x": s["cache"].residual_apply(s["w"][0], s["off"], s["x_out"], s["x"])}
    how = {"dim": s["dim"], "kind": s["kind"], "eps": s["eps"], "gain": s["gain"],
           "shift": s["shift"], "out": s["y"]}
    if s["source"] == "module":
        x, y = s["cache"].residual_norm(s["w"], 0, s["x_out"], s["x"], **how)
    elif s["source"] == "collapsed":
        x, y, _ = s["hist"].predict_norm(s["target"], s["x_out"], s["x"], **how)
    else:
        import paper_2608_23429_amd as cheb
        x, y = cheb.add_norm(s["srcs"], s["w"], s["x_out"], s["x"], **how)
    return {"x": x, "y": y[0].view(-1), "scale": y[1].view(-1)} if isinstance(y, tuple) else \
        {"x": x, "y": y.view(-1)}


def run(state):
    s = state
    if own:
        return _run_own(s)
    if s["op"] == "norm":
        return _norm_plain(s)
    if s["op"] == "store":
        x = _pad_segments(torch.cat(s["segs"]).float(), s["sizes"])
        codes, e = _quantise(x, s["quant"])
        return {"entry": _read(codes, e, s["quant"]).to(DTYPES[s["dtype"]])}
    if s["op"] == "predict":
        out = _weighted(s).to(DTYPES[s["dtype"]])
        return {"out": list(out)}
    # Residual: the tensors of one size side by side, added up in 64 bits
    # (some hundred terms an element).
    v = _weighted(s)[0]
    x, sizes = s["x"].double(), s["sizes"]
    if s["family"] != "flux":
        v = v.view(len(sizes), -1)[:, :sizes[0]]
        return {"x": (x + v.sum(0, dtype=torch.float64)).float()}
    img, txt = sizes[0], sizes[1]
    pi, pt, pj = (_padded(n) for n in sizes[:2] + sizes[-1:])
    double = v[:s["blocks"] * (pi + pt)].view(s["blocks"], -1)
    joint = v[s["blocks"] * (pi + pt):].view(-1, pj)[:, :img + txt].sum(0, dtype=torch.float64)
    both = torch.cat([double[:, pi:pi + txt], double[:, :img]], 1).sum(0, dtype=torch.float64)
    return {"x": (x + both + joint).float()}


# -- what a pass cannot do without -------------------------------------------------

def work(case):
    c = case
    if c["op"] == "norm":
        el = c["rows"] * c["dim"]
        out = BYTES.get(c["out"], 1) * el
        scales = c["rows"] * -(-c["dim"] // 32) if c["out"] == "mxfp8" else \
            4 * c["rows"] if c["out"] == "fp8_row" else 0
        mod = 4 * c["dim"] * c["groups"] * (2 if c["shift"] else 1)
        return {"bytes": (c["n"] * BYTES[c["dtype"]] + 2 * BYTES[c["x_dtype"]]) * el + out + scales + mod,
                "flops": (2 * c["n"] + 6) * el}
    esz, el = BYTES[c["dtype"]], sum(_segments(c))
    if c["op"] == "store":
        return {"bytes": 2 * el * esz + 2 * el * 33 / 32, "flops": 3 * el}
    if c["op"] == "predict":
        return {"bytes": c["n"] * el * 33 / 32 + c["m"] * el * esz, "flops": 2 * c["n"] * c["m"] * el}
    return {"bytes": c["n"] * el * 33 / 32 + 8 * _residual_map(c)[1], "flops": 2 * c["n"] * el}


# -- the same in 64 bits -----------------------------------------------------------

def _two64(e):
    """2^e in 64 bits, for whole e far from the ends of their range."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _near_e4m3(v):
    """Nearest e4m3 value, ties to even: spacing 2^(k - 3) from 2^k on, 2^-9
    below 2^-6."""
    _, k = torch.frexp(v)                      # |v| in [2^(k-1), 2^k)
    step = _two64((k - 1).clamp(min=-6) - 3)
    return (torch.round(v / step) * step).clamp(-448, 448)


def _group_exponent(top, limit):
    """Least e with top <= limit 2^e, kept within [-120, 127]."""
    _, k = torch.frexp(top / limit)            # top / limit in [2^(k-1), 2^k), up to rounding
    e = torch.where(top == 0, torch.full_like(k, -120), k).clamp(-400, 400)
    e = e + (top > limit * _two64(e)).to(e.dtype)
    e = e - (top <= limit * _two64(e - 1)).to(e.dtype)
    return e.clamp(-120, 127)


def _held(x, quant):
    """What an 8-bit entry holds for 64-bit values x, from the definition."""
    parts = []
    for part in x.view(-1, 32).split(1 << 22):
        top = part.abs().amax(1)
        if quant == "mxint8":
            unit = _two64(_group_exponent(top, 127 / 64) - 6)[:, None]
            parts.append(torch.round(part / unit).clamp(-127, 127) * unit)
        else:
            unit = _two64(_group_exponent(top, 448.0))[:, None]
            parts.append(_near_e4m3(part / unit) * unit)
    return torch.cat(parts).view(-1)


def _held_entries(c, seed, steps):
    """Padded entries as held, fp64."""
    sizes = _segments(c)
    off = np.cumsum([0] + [_padded(n) for n in sizes])
    for v in _entries(c, seed, steps):
        x = torch.zeros(int(off[-1]), dtype=torch.float64, device="cuda")
        for o, t in zip(off, v.split(sizes)):
            x[int(o):int(o) + t.numel()] = t
        yield _held(x, c["quant"])


def exact(case, seed):
    c = case
    nodes, _ = _schedule(c)
    rows = _weights(c)
    if c["op"] == "norm":
        return _exact_norm(c, seed, rows[0])
    if c["op"] == "store":
        return {"entry": next(_held_entries(c, seed, nodes[:1]))}
    outs = [0.0 for _ in rows]
    for k, v in enumerate(_held_entries(c, seed, nodes)):
        outs = [o + float(row[k]) * v for o, row in zip(outs, rows)]
    if c["op"] == "predict":
        return {"out": outs}
    off, _ = _residual_map(c)
    x, at = _residual_values(c, seed).double(), 0
    for o, size in zip(off, _segments(c)):
        x[o:o + size] += outs[0][at:at + size]
        at += _padded(size)
    return {"x": x}


def _exact_norm(c, seed, w):
    srcs, x, gain, shift = _norm_inputs(c, seed)
    rows, dim = c["rows"], c["dim"]
    w = w if c["source"] != "add" else np.ones(1)
    x = x.double()
    for a, v in zip(w, srcs):
        x = x + float(a) * v.double()
    h = x.view(rows, dim)
    if c["kind"] == "layer":
        h = h - h.sum(1, keepdim=True) / dim
    y = h / torch.sqrt(h.square().sum(1, keepdim=True) / dim + 1e-6)
    if gain is not None:
        of_row = torch.arange(rows, device="cuda") // (rows // c["groups"])
        y = y * gain.double()[of_row]
        if shift is not None:
            y = y + shift.double()[of_row]
    if c["out"] in DTYPES:
        return {"x": x, "y": y.reshape(-1)}
    if c["out"] == "fp8_row":
        top = y.abs().amax(1)
        scale = torch.where(top > 0, top / 448.0, torch.ones_like(top))
        return {"x": x, "y": _near_e4m3(y / scale[:, None]).view(-1), "scale": scale}
    width = -(-dim // 32)
    padded = torch.zeros(rows, 32 * width, dtype=torch.float64, device="cuda")
    padded[:, :dim] = y
    e = _group_exponent(padded.view(rows, width, 32).abs().amax(2), 448.0)
    scale = _two64(e)
    codes = _near_e4m3(padded.view(rows, width, 32) / scale[..., None]).view(rows, -1)[:, :dim]
    return {"x": x, "y": codes.reshape(-1), "scale": scale.reshape(-1)}
