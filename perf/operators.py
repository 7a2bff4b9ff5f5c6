"""The 8-bit projection layer and the gradient clip of this library, as measurable cases.

A projection whose operands are held in 8 bits is, in a trainer's step: the residual's addition
and the RMS norm that write the product's first operand (e4m3 with a scale for each row and 128
columns), the product with the weight (a scale for each 128 x 128 block), the quantisation of the
gradient that comes back (groups along its rows for the input's gradient, along its columns for
the weight's), the two gradient products, the norm's backward, and at the end the clip of all
gradients by their global norm.  Sizes follow the repository's workloads: DiT-B is 768 wide with
333 tokens a sample (256 + 77) and groups of 8, the 1024^2 model has 4608 tokens a sample and
groups of 4; other widths are generic.

  norm       h = x + r, y = h / rms(h) * w, y in 8 bits:  h, values, scales, 1 / rms
  norm_grad  its backward pass:                           dx (also the residual's), dw
  quantize   a matrix in 8 bits: "row" (groups of 128 along a row), "col" (along a column),
             "row+col" (both from one read), "block" (128 x 128)
  product    C = A B^T of 8-bit operands with scales: "forward" (weight [N, K] in blocks),
             "dx" (the same weight read transposed), "dw" (both operands transposed, groups
             along the tokens)
  clip       out = g * min(1, max_norm / (norm + eps)) over all tensors of a model

An 8-bit output is returned as the float8 tensor that it is, beside its scales.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
TOP = 448.0  # the largest e4m3 value
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # serving: one token through the norm; latency
        dict(name="norm_token", op="norm", rows=1, d=4096, x="bf16", h="bf16"),
        # a group of four 1024^2 samples, residual stream in 32 bits as the library keeps it
        dict(name="norm_1024", op="norm", rows=18432, d=4096, x="bf16", h="f32"),
        # DiT-B, a group of 8: ordinary training size, bound by latency as much as by bytes
        dict(name="norm_grad_dit_b", op="norm_grad", rows=2664, d=768, x="bf16", h="f32"),
        # wide rows, an odd number of them, the stream in 16 bits
        dict(name="norm_grad_wide", op="norm_grad", rows=9217, d=5120, x="bf16", h="bf16"),
        # the gradient of a 1024^2 sample's projection, for both gradient products
        dict(name="quantize_grad", op="quantize", form="row+col", rows=4608, d=4096, x="bf16"),
        # a weight whose sides end inside a block, from its 32-bit master copy
        dict(name="quantize_weight_odd", op="quantize", form="block", rows=5000, d=2200, x="f32"),
        # serving: one token against a square weight; bound by reading the weight
        dict(name="product_token", op="product", form="forward", m=1, n=4096, k=4096, out="bf16"),
        # the widest product of a group of four 1024^2 samples; bound by the tensor pipe
        dict(name="product_1024", op="product", form="forward", m=18432, n=12288, k=4096, out="bf16"),
        # DiT-B, the input gradient of the qkv projection over the 16 endpoint rows of a window
        dict(name="product_dx_dit_b", op="product", form="dx", m=5328, n=768, k=2304, out="bf16"),
        # its weight gradient: few output tiles, a long sum over tokens
        dict(name="product_dw_dit_b", op="product", form="dw", m=2304, n=768, k=5328, out="f32"),
        # the smallest model's gradients: many short tensors, latency
        dict(name="clip_tiny", op="clip", width=64, depth=2, g="f32", clipped=True),
        # all gradients of DiT-B
        dict(name="clip_dit_b", op="clip", width=768, depth=12, g="f32", clipped=True),
    ]


_LARGEST = 1.8e12  # operations of the largest listed product
_LARGEST_ELEMENTS = 75_000_000  # of the largest listed norm


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "quantize", "product", "product", "product", "clip"])
    if op == "clip":
        return dict(op=op, width=64 * _log_int(rng, 1, 12), depth=_log_int(rng, 1, 12), g=rng.choice(["f32", "f32", "bf16"]),
                    clipped=rng.random() < 0.8)
    if op == "product":
        while True:
            c = dict(op=op, form=rng.choice(["forward", "forward", "dx", "dw"]), m=_log_int(rng, 1, 20000),
                     n=_log_int(rng, 64, 12288), k=_log_int(rng, 64, 12288), out="bf16")
            if c["form"] == "dw":  # a weight's sides, a sum over tokens
                c["m"], c["k"] = c["k"], c["m"]
                c["out"] = "f32"
            if work(c)["flops"] <= _LARGEST:
                return c
    while True:
        # widths: mostly multiples of 8, some that end anywhere
        d = _log_int(rng, 16, 1024) * 8 if rng.random() < 0.75 else _log_int(rng, 100, 8192)
        c = dict(op=op, rows=_log_int(rng, 1, 20000), d=d, x=rng.choice(["bf16", "bf16", "f32"]))
        if op == "quantize":
            c["form"] = rng.choice(["row", "col", "row+col", "block"])
        else:
            c["h"] = rng.choice(["bf16", "f32"])
        if c["rows"] * d <= _LARGEST_ELEMENTS:
            return c


def _groups(n):
    return -(-n // 128)


def work(case):
    c, size = case, {"bf16": 2, "f32": 4}
    if c["op"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        scales = _groups(k) * (m + (n if c["form"] == "dw" else _groups(n)))
        return {"bytes": m * k + n * k + 4 * scales + m * n * size[c["out"]], "flops": 2 * m * n * k}
    if c["op"] == "clip":
        total = _layout(c)[1]
        return {"bytes": 2 * total * size[c["g"]], "flops": 3 * total}
    e, x = c["rows"] * c["d"], size[c["x"]]
    if c["op"] == "norm":  # x and the stream read; the stream, 8 bits and scales written
        return {"bytes": e * (x + 2 * size[c["h"]] + 1) + 4 * c["d"] + 4 * c["rows"] * (_groups(c["d"]) + 1), "flops": 6 * e}
    if c["op"] == "norm_grad":  # dy, h and the stream's gradient read, dx written
        return {"bytes": e * (x + 3 * size[c["h"]]) + 8 * c["d"] + 4 * c["rows"], "flops": 10 * e}
    forms = c["form"].split("+")
    scales = sum({"row": c["rows"] * _groups(c["d"]), "col": c["d"] * _groups(c["rows"]),
                  "block": _groups(c["rows"]) * _groups(c["d"])}[f] for f in forms)
    return {"bytes": e * (x + len(forms)) + 4 * scales, "flops": 3 * e * len(forms)}


# ------------------------------------------------------------------ inputs
def _layout(c):
    """(offset, length) of every gradient tensor of a DiT of the case's width and depth in one
    flat buffer, each at a multiple of 64 elements, and the buffer's length."""
    d = c["width"]
    shapes = [d * 64, d, d * d, d, d * 256, d, d * d, d]
    for _ in range(c["depth"]):
        shapes += [6 * d * d, 6 * d, 3 * d * d, 3 * d, d * d, d, 4 * d * d, 4 * d, 4 * d * d, d]
    shapes += [2 * d * d, 2 * d, 64 * d, 64]
    at, off = [], 0
    for n in shapes:
        at.append((off, n))
        off += -(-n // 64) * 64
    return at, off


def _normal(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)


def _wide(seed, rows, d, dtype):
    """Activations as they are met: a few columns are much larger than the others."""
    x = _normal(seed, rows, d)
    col = _normal(seed + 1, d)
    return (x * torch.exp(0.5 * col) * torch.where(col > 2.5, 8.0, 1.0)).to(dtype)


def _buffers(rows, cols, form):
    """A matrix in 8 bits and its scales: row pitches of a multiple of 16 bytes."""
    q = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.float8_e4m3fn, device=DEV)[:, :cols]
    g = {"row": (_groups(cols), rows), "col": (_groups(rows), cols), "block": (_groups(rows), _groups(cols))}[form]
    s = torch.zeros(g[0], -(-g[1] // 4) * 4, device=DEV)[:, :g[1]]
    return q, s


def _as_held(x, form):
    """x as the user holds it: in 8 bits, in the buffers that the products read."""
    q, s = _buffers(*x.shape, form)
    for at, y in zip((q, s), _plain_quantize(x, form)):
        at.copy_(y)
    return q, s


def prepare(case, seed):
    c, seed = case, seed * 16
    s = dict(case=c)
    if c["op"] in ("norm", "norm_grad"):
        rows, d, xt, ht = c["rows"], c["d"], _DTYPES[c["x"]], _DTYPES[c["h"]]
        s["w"] = _normal(seed + 2, d, scale=0.2) + 1.0
        if c["op"] == "norm":
            s["x"], s["r"] = _wide(seed, rows, d, xt), _normal(seed + 3, rows, d, dtype=ht, scale=3.0)
            s["h"] = torch.empty_like(s["r"])
            s["q"], s["s"] = _buffers(rows, d, "row")
            s["rstd"] = torch.empty(rows, device=DEV)
        else:
            s["dy"] = _normal(seed, rows, d, dtype=xt, scale=1e-3)
            s["h"] = _wide(seed + 3, rows, d, ht)
            s["rstd"] = 1.0 / torch.sqrt(s["h"].float().square().mean(1) + EPS)
            s["dh"] = _normal(seed + 5, rows, d, dtype=ht, scale=1e-3)
            s["dx"], s["dw"] = torch.empty_like(s["h"]), torch.empty(d, device=DEV)
            # scratch of the weight's gradient: as much as the library asks for at most
            s["ws"] = torch.empty(1024 * (d + 64) * 4, dtype=torch.uint8, device=DEV)
    elif c["op"] == "quantize":
        s["x"] = _wide(seed, c["rows"], c["d"], _DTYPES[c["x"]])
        s["to"] = {f: _buffers(c["rows"], c["d"], f) for f in c["form"].split("+")}
    elif c["op"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        bf = torch.bfloat16
        if c["form"] == "dw":
            s["a"], s["b"] = _as_held(_normal(seed, k, m, dtype=bf), "col"), _as_held(_wide(seed + 3, k, n, bf), "col")
        else:
            s["a"] = _as_held(_wide(seed, m, k, bf), "row")
            w = _normal(seed + 3, *((n, k) if c["form"] == "forward" else (k, n)), dtype=bf, scale=k ** -0.5)
            s["b"] = _as_held(w, "block")
        s["c"] = torch.empty(m, n, dtype=_DTYPES[c["out"]], device=DEV)
    else:
        at, total = _layout(c)
        g = torch.zeros(total, dtype=_DTYPES[c["g"]], device=DEV)
        for i, (o, n) in enumerate(at):
            g[o:o + n] = _normal(seed * 64 + i, n, scale=1e-3 * (1 + i % 7))
        s["flat"], s["out_flat"] = g, torch.zeros_like(g)
        s["g"] = [g[o:o + n] for o, n in at]
        s["out"] = [s["out_flat"][o:o + n] for o, n in at]
        s["norm"] = torch.empty(2, device=DEV)
        s["ws"] = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
        s["max_norm"] = 1.0 if c["clipped"] else 1e4
    return s


# ------------------------------------------------------------------ the operators
def _padded(x):
    r, d = x.shape
    return torch.nn.functional.pad(x, (0, _groups(d) * 128 - d, 0, _groups(r) * 128 - r))


def _plain_quantize(x, form):
    """Values and scales of x in groups of 128 along its rows, its columns, or in blocks."""
    rows, d = x.shape
    x = x.float()
    if form == "row":
        p = torch.nn.functional.pad(x, (0, _groups(d) * 128 - d)).view(rows, -1, 128)
        a = p.abs().amax(2)
        s = (a / TOP).clamp(min=2.0 ** -126)
        q = (p / s[:, :, None]).clamp(-TOP, TOP).view(rows, -1)[:, :d]
        return q.to(torch.float8_e4m3fn), s.t()
    if form == "col":
        p = torch.nn.functional.pad(x, (0, 0, 0, _groups(rows) * 128 - rows)).view(-1, 128, d)
        s = (p.abs().amax(1) / TOP).clamp(min=2.0 ** -126)
        q = (p / s[:, None, :]).clamp(-TOP, TOP).view(-1, d)[:rows]
        return q.to(torch.float8_e4m3fn), s
    p = _padded(x).view(_groups(rows), 128, _groups(d), 128)
    s = (p.abs().amax((1, 3)) / TOP).clamp(min=2.0 ** -126)
    q = (p / s[:, None, :, None]).clamp(-TOP, TOP).view(_groups(rows) * 128, -1)[:rows, :d]
    return q.to(torch.float8_e4m3fn), s


def _spread(s, rows, d, form):
    """The scale of every element."""
    if form == "row":
        return s.t().repeat_interleave(128, 1)[:, :d]
    if form == "col":
        return s.repeat_interleave(128, 0)[:rows]
    return s.repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :d]


def _plain(s):
    c = s["case"]
    if c["op"] == "norm":
        h = (s["x"].float() + s["r"].float()).to(s["r"].dtype)
        rstd = torch.rsqrt(h.float().square().mean(1) + EPS)
        q, sc = _plain_quantize(h.float() * rstd[:, None] * s["w"], "row")
        return h, q, sc, rstd
    if c["op"] == "norm_grad":
        xhat = s["h"].float() * s["rstd"][:, None]
        dy = s["dy"].float()
        g = dy * s["w"]
        dx = s["dh"].float() + s["rstd"][:, None] * (g - xhat * (g * xhat).mean(1, keepdim=True))
        return dx.to(s["h"].dtype), (dy * xhat).sum(0)
    if c["op"] == "quantize":
        return [_plain_quantize(s["x"], f) for f in c["form"].split("+")]
    if c["op"] == "product":
        (a, sa), (b, sb) = s["a"], s["b"]
        fa, fb = ("col", "col") if c["form"] == "dw" else ("row", "block")
        a = a.float() * _spread(sa, *a.shape, fa)
        b = b.float() * _spread(sb, *b.shape, fb)
        return torch.matmul(a.t() if c["form"] == "dw" else a, b.t() if c["form"] == "forward" else b).to(s["c"].dtype)
    g = s["flat"].float()
    norm = g.square().sum(dtype=torch.float64).sqrt()
    coef = (s["max_norm"] / (norm + EPS)).clamp(max=1.0)
    return (g * coef.float()).to(s["flat"].dtype), torch.stack([norm, coef]).float()


def run(state):
    s = state
    if not own:
        return _plain(s)
    import paper_2607_17572_gb300 as jagg
    c = s["case"]
    if c["op"] == "norm":
        jagg.rms_norm_fp8(s["x"], s["q"], s["s"], residual=s["r"], weight=s["w"], eps=EPS, h_out=s["h"], rstd=s["rstd"])
        return s["h"], s["q"], s["s"], s["rstd"]
    if c["op"] == "norm_grad":
        jagg.rms_norm_bwd(s["dy"], s["h"], s["rstd"], s["dx"], weight=s["w"], dh=s["dh"], dweight=s["dw"], ws=s["ws"])
        return s["dx"], s["dw"]
    if c["op"] == "quantize":
        jagg.quantize_fp8(s["x"], **s["to"])
        return [s["to"][f] for f in c["form"].split("+")]
    if c["op"] == "product":
        (a, sa), (b, sb) = s["a"], s["b"]
        jagg.gemm_fp8(a, sa, b, sb, s["c"], a_trans=c["form"] == "dw", b_trans=c["form"] != "forward")
        return s["c"]
    jagg.grad_clip(s["g"], s["max_norm"], s["norm"], s["ws"], out=s["out"], eps=EPS)
    return s["out_flat"], s["norm"]


# ------------------------------------------------------------------ the same in 64 bits
def _e4m3(v):
    """Nearest e4m3 value, ties to even: 3 bits below the leading one, exponents from -6."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step).clamp(-TOP, TOP)


def _exact_quantize(y, form):
    rows, d = y.shape
    idx = {"row": (1, 128), "col": (128, 1), "block": (128, 128)}[form]
    gr, gc = -(-rows // idx[0]), -(-d // idx[1])
    group = (torch.arange(rows, device=DEV) // idx[0])[:, None] * gc + (torch.arange(d, device=DEV) // idx[1])
    a = torch.zeros(gr * gc, dtype=torch.float64, device=DEV)
    a.scatter_reduce_(0, group.reshape(-1), y.abs().reshape(-1), "amax")
    s = torch.maximum(a / TOP, torch.tensor(2.0 ** -126, dtype=torch.float64, device=DEV))
    q = _e4m3(y / s[group])
    s = s.view(gr, gc)
    return q, s.t().contiguous() if form == "row" else s


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "norm":
        h = s["x"].double() + s["r"].double()
        kept = h.to(torch.float32).to(s["r"].dtype).double()  # the stream is stored in its own type
        rstd = (kept.pow(2).sum(1) / c["d"] + EPS).pow(-0.5)
        q, sc = _exact_quantize(kept * rstd[:, None] * s["w"].double()[None, :], "row")
        return h, q, sc, rstd
    if c["op"] == "norm_grad":
        h, r, dy, w = s["h"].double(), s["rstd"].double()[:, None], s["dy"].double(), s["w"].double()
        inner = torch.einsum("rd,rd,d->r", dy, h, w)[:, None]
        return s["dh"].double() + r * dy * w - h * r.pow(3) * inner / c["d"], torch.einsum("rd,rd->d", dy, h * r)
    if c["op"] == "quantize":
        return [_exact_quantize(s["x"].double(), f) for f in c["form"].split("+")]
    if c["op"] == "product":
        (a, sa), (b, sb) = s["a"], s["b"]
        k, out = c["k"], torch.zeros(c["m"], c["n"], dtype=torch.float64, device=DEV)
        for g in range(_groups(k)):  # the definition: one partial product for each group of 128
            at = slice(g * 128, min(k, g * 128 + 128))
            ag = a[at].double().t() if c["form"] == "dw" else a[:, at].double()
            bg = b[:, at].double() if c["form"] == "forward" else b[at].double().t()
            if c["form"] == "dw":
                cols = sb[g].double()
            else:
                blocks = sb[:, g] if c["form"] == "forward" else sb[g]
                cols = blocks.double()[torch.arange(c["n"], device=DEV) // 128]
            out += sa[g].double()[:, None] * (ag @ bg.t()) * cols[None, :]
        return out
    g = s["flat"].double()
    norm = torch.linalg.vector_norm(g)
    coef = min(1.0, s["max_norm"] / (float(norm) + EPS))
    return g * coef, np.array([float(norm), coef])
