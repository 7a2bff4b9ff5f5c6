"""RMS norm with an 8-bit output, its backward, quantisation and the products of 8-bit operands,
against plain 64-bit forms (fp8_reference.py, where the tolerances are derived)."""
import os
import subprocess
import sys

import pytest
import torch

from fp8_reference import U, check_product, check_quantised, e4m3, groups, half_step, held

pytestmark = pytest.mark.gpu

jg = pytest.importorskip("paper_2607_17572_gb300")

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rand(*shape, dtype=torch.float32, scale=1.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + sum(shape) * 7)
    return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)


def _pitched(t, pad, offset=0):
    """The same matrix with a row pitch `pad` elements longer, `offset` elements into its buffer."""
    r, c = t.shape
    buf = torch.full((r * (c + pad) + offset,), 3.0, dtype=t.dtype, device=t.device)
    v = buf[offset:].view(r, c + pad)[:, :c]
    v.copy_(t)
    return v


def _codes(rows, cols, form, pad=0):
    """Buffers whose every byte is known, to see what a call leaves alone."""
    ld = -(-cols // 16) * 16 + pad
    raw = torch.full((rows + 2, ld), 0x55, dtype=torch.uint8, device="cuda")
    shape = {"row": (groups(cols), rows), "col": (groups(rows), cols), "block": (groups(rows), groups(cols))}[form]
    s_raw = torch.full((shape[0] + 1, -(-shape[1] // 4) * 4 + 4), -7.0, device="cuda")
    return raw, raw[:rows, :cols], s_raw, s_raw[:shape[0], :shape[1]]


def _untouched(raw, s_raw, rows, cols, shape):
    assert (raw[rows:] == 0x55).all() and (raw[:rows, cols:] == 0x55).all()
    assert (s_raw[shape[0]:] == -7.0).all() and (s_raw[:, shape[1]:] == -7.0).all()


def _sum_terms(d):
    """Additions on a path of a row's sum: a thread's run, the shuffles, the warps."""
    return max(32, d // 256 + 1) + 5 + 32


# ------------------------------------------------------------------ norm
@pytest.mark.parametrize("x,h", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,d,pad", [(1, 1, 0), (3, 127, 0), (5, 128, 8), (2, 129, 1), (7, 256, 0), (4, 264, 0), (9, 768, 0),
                                        (3, 1000, 24), (2, 1001, 0), (130, 1536, 0), (3, 4096, 0), (2, 8200, 0),
                                        (1, 32768, 0), (2, 32767, 0)])
def test_norm(rows, d, pad, x, h):
    xs = _pitched(_rand(rows, d, dtype=DT[x], seed=1), pad)
    r = _pitched(_rand(rows, d, dtype=DT[h], scale=3.0, seed=2), pad)
    w = _rand(d, scale=0.2, seed=3) + 1.0
    raw, q, s_raw, s = _codes(rows, d, "row", pad=16 if pad else 0)
    out, rstd = _pitched(torch.zeros_like(r), pad), torch.full((rows,), -1.0, device="cuda")
    jg.rms_norm_fp8(xs, q, s, residual=r, weight=w, eps=1e-6, h_out=out, rstd=rstd)
    kept = (xs.float() + r.float()).to(DT[h])  # one f32 addition, one rounding: the same bits
    assert torch.equal(out, kept)
    ref = (kept.double().pow(2).mean(1) + 1e-6).pow(-0.5)
    rel = (_sum_terms(d) / 2 + 6) * U
    assert ((rstd.double() - ref).abs() <= rel * ref).all()
    check_quantised(kept.double() * ref[:, None] * w.double(), q, s, "row", rel + 3 * U)
    _untouched(raw, s_raw, rows, d, s.shape)


@pytest.mark.parametrize("d", [256, 301])
def test_norm_options(d):
    """Without residual, weight, h or rstd; a bf16 weight; the stream updated in place; x off its
    16-byte alignment."""
    rows = 6
    x = _rand(rows, d, dtype=torch.bfloat16, seed=1)
    base = x.double()
    rel = (_sum_terms(d) / 2 + 9) * U
    q, s = jg.fp8_buffers(rows, d, "row")
    jg.rms_norm_fp8(x, q, s, eps=0.25)
    check_quantised(base * (base.pow(2).mean(1, keepdim=True) + 0.25).pow(-0.5), q, s, "row", rel)
    off = _pitched(x, 1, offset=1)
    q2, s2 = jg.fp8_buffers(rows, d, "row")
    jg.rms_norm_fp8(off, q2, s2, eps=0.25)
    check_quantised(base * (base.pow(2).mean(1, keepdim=True) + 0.25).pow(-0.5), q2, s2, "row", rel)
    w = _rand(d, dtype=torch.bfloat16, seed=2)
    r = _rand(rows, d, seed=3)
    both = (x.float() + r).double()
    jg.rms_norm_fp8(x, q, s, residual=r, weight=w, h_out=r)
    assert torch.equal(r.double(), both)
    check_quantised(both * (both.pow(2).mean(1, keepdim=True) + 1e-6).pow(-0.5) * w.double(), q, s, "row", rel)


@pytest.mark.parametrize("d", [512, 333])
def test_norm_extremes(d):
    """Rows of zeros, tiny and large rows, rows that hold a NaN or an infinity: each row on its own."""
    x = _rand(6, d, seed=5)
    x[1] = 0.0
    x[2] *= 1e-30
    x[3] *= 1e15
    x[4, 200] = float("nan")
    x[5, 7] = float("inf")
    q, s = jg.fp8_buffers(6, d, "row")
    rstd = torch.empty(6, device="cuda")
    jg.rms_norm_fp8(x, q, s, eps=1e-6, rstd=rstd)
    y = x.double() * (x.double().pow(2).mean(1, keepdim=True) + 1e-6).pow(-0.5)
    fine = [0, 1, 2, 3]
    check_quantised(y[fine], q[fine], s[:, fine], "row", (_sum_terms(d) / 2 + 9) * U)
    assert (held(q, s, "row")[1] == 0).all()
    assert held(q, s, "row")[4].isnan().all() and rstd[4].isnan()
    # 1 / rms is 0: the infinite element's group is NaN, the others are zeros
    v = held(q, s, "row")[5]
    assert v[:128].isnan().all() and (v[128:] == 0).all()


def test_norm_of_no_rows_launches_nothing():
    q, s = jg.fp8_buffers(0, 64, "row")
    n = jg.launch_count()
    jg.rms_norm_fp8(torch.empty(0, 64, device="cuda"), q, s)
    assert jg.launch_count() == n


# ------------------------------------------------------------------ norm backward
@pytest.mark.parametrize("y,h", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,d,pad", [(1, 1, 0), (3, 127, 0), (17, 128, 0), (2, 129, 1), (9, 256, 8), (700, 768, 0),
                                        (1300, 300, 0), (2500, 512, 0), (5, 1536, 0), (3, 1537, 0), (3, 4096, 0), (3, 4001, 0),
                                        (620, 5120, 0), (2, 5121, 0), (2, 8192, 0), (3, 8200, 0), (2, 32768, 0), (1, 32767, 0)])
def test_norm_backward(rows, d, pad, y, h):
    dy = _pitched(_rand(rows, d, dtype=DT[y], seed=1), pad)
    hs = _pitched(_rand(rows, d, dtype=DT[h], scale=2.0, seed=2), pad)
    dh = _pitched(_rand(rows, d, dtype=DT[h], seed=3), pad)
    w = _rand(d, scale=0.3, seed=4) + 1.0
    rstd = (hs.double().pow(2).mean(1) + 1e-6).pow(-0.5).float()
    dx = _pitched(torch.zeros_like(hs), pad)
    dw0 = _rand(d, seed=5)
    dw = dw0.clone()
    ws = jg.alloc_bytes(jg.rms_norm_bwd_workspace_bytes(rows, d))
    jg.rms_norm_bwd(dy, hs, rstd, dx, weight=w, dh=dh, dweight=dw, accumulate=True, ws=ws)
    # 64 bits, with the rstd that was given
    xh = hs.double() * rstd.double()[:, None]
    g = dy.double() * w.double()
    r = rstd.double()[:, None]
    ref = dh.double() + r * (g - xh * (g * xh).mean(1, keepdim=True))
    mag = dh.double().abs() + r * (g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
    err = (_sum_terms(d) + 10) * U * mag
    assert ((dx.double() - ref).abs() <= err + half_step(DT[h]) * (ref.abs() + err)).all()
    rw, mw = (dy.double() * xh).sum(0), (dy.double() * xh).abs().sum(0)
    assert ((dw.double() - dw0.double() - rw).abs() <= (rows + 4) * U * (mw + dw0.double().abs())).all()
    # overwritten, without the direct gradient, in the buffer that held dh, twice the same bits
    dw2, dw3, dx2 = torch.empty_like(dw), torch.full_like(dw, 9.0), dh.clone()
    jg.rms_norm_bwd(dy, hs, rstd, dx, weight=w, dh=dh, dweight=dw2, ws=ws)
    if pad == 0:
        jg.rms_norm_bwd(dy, hs, rstd, dx2, weight=w, dh=dx2, dweight=dw3, ws=ws)
        assert torch.equal(dx2, dx) and torch.equal(dw2, dw3)
    assert ((dw2.double() - rw).abs() <= (rows + 4) * U * mw).all()


def test_norm_backward_against_differences():
    """The gradient of sum(dy * y) + sum(dh * h) by central differences of the 64-bit norm."""
    rows, d, step = 4, 24, 1e-5
    h, dy, dh, w = (_rand(rows, d, seed=i).double() for i in (1, 2, 3, 4))
    w = w[0]

    def value(hh):
        y = hh * (hh.pow(2).mean(1, keepdim=True) + 1e-3).pow(-0.5) * w
        return (dy * y).sum() + (dh * hh).sum()

    diff = torch.empty_like(h)
    for i in range(rows):
        for j in range(d):
            e = torch.zeros_like(h)
            e[i, j] = step
            diff[i, j] = (value(h + e) - value(h - e)) / (2 * step)
    f = lambda t: t.float().contiguous()
    rstd = (h.pow(2).mean(1) + 1e-3).pow(-0.5).float()
    dx = torch.empty(rows, d, device="cuda")
    jg.rms_norm_bwd(f(dy), f(h), rstd, dx, weight=f(w), dh=f(dh))
    # differences: step^2 of the third derivative (a few units) and 1e-16 / step of rounding; f32: 1e-6
    assert (dx.double() - diff).abs().max().item() < 2e-5


def test_norm_backward_of_no_rows():
    e = torch.empty(0, 40, device="cuda")
    dw = torch.full((40,), 3.0, device="cuda")
    ws = jg.alloc_bytes(16)
    jg.rms_norm_bwd(e, e, torch.empty(0, device="cuda"), e, dweight=dw, accumulate=True, ws=ws)
    assert (dw == 3.0).all()
    jg.rms_norm_bwd(e, e, torch.empty(0, device="cuda"), e, dweight=dw, ws=ws)
    assert (dw == 0.0).all()


# ------------------------------------------------------------------ quantisation
@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 4096, 0), (127, 127, 0), (128, 128, 0), (129, 136, 8), (300, 129, 1),
                                           (260, 264, 0), (1, 333, 0), (1000, 16, 0)])
def test_quantise(rows, cols, pad, x):
    """Every form on its own and all from one read; the same codes either way."""
    xs = _pitched(_rand(rows, cols, dtype=DT[x], seed=1) * torch.exp(_rand(cols, seed=2)).to(DT[x]), pad)
    rm, cm = _rand(rows, seed=3).abs() + 0.1, _rand(cols, dtype=torch.bfloat16, seed=4)
    for mul in (dict(), dict(row_mul=rm, col_mul=cm)):
        y = xs.double()
        if mul:
            y = y * rm.double()[:, None] * cm.double()
        alone, together = {}, {}
        for f in ("row", "col", "block"):
            raw, q, s_raw, s = _codes(rows, cols, f, pad=16)
            jg.quantize_fp8(xs, **{f: (q, s)}, **mul)
            check_quantised(y, q, s, f, 2 * U if mul else 0.0)
            _untouched(raw, s_raw, rows, cols, s.shape)
            alone[f] = (q, s)
            together[f] = jg.fp8_buffers(rows, cols, f)
        jg.quantize_fp8(xs, **together, **mul)
        for f in alone:
            assert torch.equal(alone[f][0], together[f][0].view(torch.uint8)) and torch.equal(alone[f][1], together[f][1])


def test_quantise_extremes():
    """Zeros, values below f32's normal range, one non-finite value: the groups that hold it."""
    x = _rand(256, 256, seed=1)
    x[:, :128] = 0.0
    x[130, 140] = float("nan")
    x[3, 250] = float("-inf")
    x[128:, 200] = 1e-40
    b = {f: jg.fp8_buffers(256, 256, f) for f in ("row", "col", "block")}
    jg.quantize_fp8(x, **b)
    for f, (q, s) in b.items():
        v = held(q, s, f)
        assert (v[:, :128] == 0).all()
        if f != "block":  # x[128:, 200] on its own: a group whose largest magnitude is far below the rest
            fine = v.isfinite()
            ref = x.double()
            lim = held(torch.full_like(q.view(torch.uint8), 0x7E), s, f) * 2.0 ** -4
            assert ((v - ref).abs()[fine] <= lim[fine]).all()
        bad = v.isnan()
        want = torch.zeros_like(bad)
        for i, j in ((130, 140), (3, 250)):
            gi, gj = i // 128 * 128, j // 128 * 128
            want[slice(i, i + 1) if f == "row" else slice(gi, gi + 128), slice(j, j + 1) if f == "col" else slice(gj, gj + 128)] = True
        assert torch.equal(bad, want), f


def test_codes_round_to_nearest_even():
    """Values halfway between two codes, with a scale of exactly 1."""
    mant = torch.arange(16, device="cuda").double() / 16 + 1  # halves of the 3-bit steps
    v = torch.cat([mant * 2.0 ** e for e in range(-5, 8)] + [torch.arange(32, device="cuda").double() * 2.0 ** -10])
    for i in range(0, v.numel(), 127):
        part = torch.cat([torch.full((1,), 448.0, device="cuda", dtype=torch.float64), v[i:i + 127]])
        x = torch.stack([part, -part]).float()
        q, s = jg.fp8_buffers(2, part.numel(), "row")
        jg.quantize_fp8(x, row=(q, s))
        assert (s == 1.0).all()
        assert torch.equal(q.double(), e4m3(x.double()))


# ------------------------------------------------------------------ products
def _operand(rows, cols, form, seed, pad=0):
    x = _rand(rows, cols, seed=seed) * torch.exp(0.5 * _rand(cols, seed=seed + 50))
    raw, q, s_raw, s = _codes(rows, cols, form, pad=pad)
    jg.quantize_fp8(x, **{form: (q, s)})
    return q, s, held(q, s, form)


SIZES = [(1, 1, 1), (1, 128, 128), (1, 1000, 4096), (3, 77, 300), (16, 256, 640), (17, 130, 129), (33, 64, 1152),
         (64, 257, 96), (77, 768, 768), (128, 128, 2048), (129, 129, 129), (130, 500, 31), (200, 16, 512),
         (333, 384, 1100), (515, 1030, 260), (1000, 640, 2304)]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("a_trans,b_trans,b_form", [(0, 0, "block"), (0, 0, "row"), (0, 1, "block"), (0, 1, "col"),
                                                    (1, 0, "row"), (1, 0, "block"), (1, 1, "col"), (1, 1, "block")])
def test_product(M, N, K, a_trans, b_trans, b_form, out):
    a, sa, va = _operand(*((K, M) if a_trans else (M, K)), "col" if a_trans else "row", 1)
    b, sb, vb = _operand(*((K, N) if b_trans else (N, K)), b_form, 2, pad=16)
    buf = torch.full((M + 1, N + 5), 5.0, dtype=DT[out], device="cuda")
    c = buf[:M, :N]
    jg.gemm_fp8(a, sa, b, sb, c, a_trans=bool(a_trans), b_trans=bool(b_trans))
    check_product(c, va.t() if a_trans else va, vb.t() if b_trans else vb)
    assert (buf[M:] == 5.0).all() and (buf[:M, N:] == 5.0).all()


PLANS = [dict(pair=256), dict(pair=128), dict(nt=128, splits=1), dict(nt=128, splits=3), dict(nt=128, splits=8),
         dict(nt=16, splits=1, swap=True), dict(nt=32, splits=2, swap=True), dict(nt=64, splits=5, swap=True)]


@pytest.mark.parametrize("plan", range(len(PLANS)))
@pytest.mark.parametrize("a_trans,b_trans,b_form", [(0, 0, "block"), (0, 0, "row"), (0, 1, "block"), (0, 1, "col"),
                                                    (1, 0, "row"), (1, 0, "block"), (1, 1, "col"), (1, 1, "block")])
def test_product_by_every_kernel(plan, a_trans, b_trans, b_form):
    """Every kernel and tile on whole and ragged tiles, more tiles than CTA pairs, one k-block and more
    than 32 of them (the block scales' batch), outputs that TMA stores serve (rows of 16 bytes) and that
    they do not, with bias and accumulation."""
    plan = PLANS[plan]
    if plan.get("swap") and a_trans:
        pytest.skip("rows of A as accumulator columns need a K-major A")
    few = plan.get("swap") or plan.get("splits", 1) > 1
    sizes = [(1, 1, 1024), (70, 130, 1030), (256, 256, 1024)] + ([] if few else [(600, 777, 128), (300, 520, 4800), (2600, 4104, 256)])
    for M, N, K in sizes:
        a, sa, va = _operand(*((K, M) if a_trans else (M, K)), "col" if a_trans else "row", 1)
        b, sb, vb = _operand(*((K, N) if b_trans else (N, K)), b_form, 2, pad=16)
        va, vb = va.t() if a_trans else va, vb.t() if b_trans else vb
        bias = _rand(N, seed=7)
        kw = dict(a_trans=bool(a_trans), b_trans=bool(b_trans), **plan)
        for out, pad in (("bf16", 5), ("bf16", (8 - N) % 8 + 8), ("f32", 3), ("f32", (4 - N) % 4 + 4)):
            buf = torch.full((M + 1, N + pad), 5.0, dtype=DT[out], device="cuda")
            c = buf[:M, :N]
            jg.test_gemm_fp8(a, sa, b, sb, c, bias=bias, **kw)
            check_product(c, va, vb, bias=bias)
            if out == "f32":
                start = c.clone()
                jg.test_gemm_fp8(a, sa, b, sb, c, accumulate=True, **kw)
                check_product(c, va, vb, start=start)
            assert (buf[M:] == 5.0).all() and (buf[:M, N:] == 5.0).all()
    assert jg.device_status() == 0


@pytest.mark.parametrize("M,N,K,pad", [(1, 96, 512, 0), (5, 640, 1024, 0), (40, 130, 300, 3), (200, 136, 520, 0), (300, 261, 700, 1),
                                       (600, 512, 130, 4)])
def test_product_bias_and_accumulation(M, N, K, pad):
    a, sa, va = _operand(M, K, "row", 3)
    b, sb, vb = _operand(N, K, "block", 4)
    for bias in (_rand(N, seed=5), _rand(N, dtype=torch.bfloat16, seed=6)):
        for out in ("bf16", "f32"):
            c = torch.empty(M, N + pad, dtype=DT[out], device="cuda")[:, :N]
            jg.gemm_fp8(a, sa, b, sb, c, bias=bias)
            check_product(c, va, vb, bias=bias)
    start = _rand(M, N + pad, scale=10.0, seed=7)[:, :N]
    c = _pitched(start, pad)
    jg.gemm_fp8(a, sa, b, sb, c, accumulate=True)
    check_product(c, va, vb, start=start)
    again = _pitched(start, pad)
    jg.gemm_fp8(a, sa, b, sb, again, accumulate=True)
    assert torch.equal(c, again)


def test_product_of_empty_sides():
    q, s = jg.fp8_buffers(5, 0, "row")
    b, sb = jg.fp8_buffers(7, 0, "block")
    c = torch.full((5, 7), 4.0, device="cuda")
    bias = _rand(7)
    jg.gemm_fp8(q, s, b, sb, c, bias=bias)
    assert torch.equal(c, bias.expand(5, 7))
    jg.gemm_fp8(q, s, b, sb, c, accumulate=True)
    assert torch.equal(c, bias.expand(5, 7))
    n = jg.launch_count()
    q, s = jg.fp8_buffers(0, 64, "row")
    b, sb = jg.fp8_buffers(7, 64, "block")
    jg.gemm_fp8(q, s, b, sb, torch.empty(0, 7, device="cuda"))
    assert jg.launch_count() == n


@pytest.mark.parametrize("M", [4, 300])
def test_product_of_nan_groups_and_zero_scales(M):
    """A NaN group of a row of A reaches that row of C alone; one of B its 128 columns; codes that
    stand for NaN with a finite scale too."""
    N, K = 260, 512
    x = _rand(M, K, seed=1)
    x[2, 130] = float("nan")
    a, sa = jg.fp8_buffers(M, K, "row")
    jg.quantize_fp8(x, row=(a, sa))
    w = _rand(N, K, seed=2)
    w[200, 5] = float("inf")
    b, sb = jg.fp8_buffers(N, K, "block")
    jg.quantize_fp8(w, block=(b, sb))
    c = torch.empty(M, N, device="cuda")
    jg.gemm_fp8(a, sa, b, sb, c)
    want = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    want[2] = True
    want[:, 128:256] = True
    assert torch.equal(c.isnan(), want)
    sa2 = torch.zeros_like(sa)
    w[200, 5] = 0.0
    jg.quantize_fp8(w, block=(b, sb))
    x[2, 130] = 0.0
    jg.quantize_fp8(x, row=(a, sa))
    jg.gemm_fp8(a, sa2, b, sb, c)
    assert (c == 0).all()
    a.view(torch.uint8)[1, 300] = 0x7F
    jg.gemm_fp8(a, sa, b, sb, c)
    assert c[1].isnan().all() and c.isnan().sum().item() == N


@pytest.mark.parametrize("M", [2, 200])
def test_product_keeps_f32_across_groups(M):
    """Groups whose scales differ by 2^20 and that cancel: nothing is lost but f32's own rounding."""
    K, N = 384, 128
    a, sa, _ = _operand(M, K, "row", 1)
    b, sb, _ = _operand(N, K, "block", 2)
    with torch.no_grad():
        a.view(torch.uint8)[:, 256:] = a.view(torch.uint8)[:, :128] ^ 0x80  # group 2 = -group 0
        b.view(torch.uint8)[:, 256:] = b.view(torch.uint8)[:, :128]
        sa[0] = sa[2] = 2.0 ** 10
        sb[0, 0] = sb[0, 2] = 2.0 ** 10
    c = torch.empty(M, N, device="cuda")
    jg.gemm_fp8(a, sa, b, sb, c)
    check_product(c, held(a, sa, "row"), held(b, sb, "block"))


# ------------------------------------------------------------------ offsets beyond 32 bits
def test_matrices_of_more_than_2_31_elements():
    """The norm, its backward, quantisation and a product whose outputs have more than 2^31 elements: their
    last rows equal those of a small call on the same rows, bit for bit where the kernels do not sum
    over rows."""
    rows, d, tail = 2**31 // 4096 + 200, 4096, 200
    x = torch.randn(tail, d, device="cuda").bfloat16()
    big = torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda")
    big[-tail:] = x
    (q, s), (q1, s1) = jg.fp8_buffers(rows, d, "row"), jg.fp8_buffers(tail, d, "row")
    r, r1 = torch.empty(rows, device="cuda"), torch.empty(tail, device="cuda")
    h = torch.empty_like(big)
    jg.rms_norm_fp8(big, q, s, h_out=h, rstd=r)
    jg.rms_norm_fp8(x, q1, s1, rstd=r1)
    assert torch.equal(h[-tail:], x) and torch.equal(r[-tail:], r1) and torch.equal(s[:, -tail:], s1)
    assert torch.equal(q[-tail:].view(torch.uint8), q1.view(torch.uint8))
    dx1 = torch.empty_like(x)
    jg.rms_norm_bwd(x, x, r1, dx1)
    jg.rms_norm_bwd(big, big, r, h)
    # (few and many rows may be held by different numbers of threads: sums in another order)
    assert ((h[-tail:].double() - dx1.double()).abs() <= 2 * half_step(torch.bfloat16) * dx1.double().abs() + 1e-5).all()
    del h
    jg.quantize_fp8(big, row=(q, s))
    jg.quantize_fp8(x, row=(q1, s1))
    assert torch.equal(q[-tail:].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s[:, -tail:], s1)
    w, sw = jg.fp8_buffers(d, d, "block")
    jg.quantize_fp8(torch.randn(d, d, device="cuda"), block=(w, sw))
    for n in (d, d - 4):  # an output that TMA stores, and one that it does not
        wn, swn = w[:n], sw
        c, c1 = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda"), torch.empty(tail, n, dtype=torch.bfloat16, device="cuda")
        jg.test_gemm_fp8(q, s, wn, swn, c, pair=256)
        jg.test_gemm_fp8(q1, s1, wn, swn, c1, pair=256)
        assert torch.equal(c[-tail:], c1)
        jg.test_gemm_fp8(q, s, wn, swn, c, splits=1)
        jg.test_gemm_fp8(q1, s1, wn, swn, c1, splits=1)
        assert torch.equal(c[-tail:], c1)
    assert jg.device_status() == 0


# ------------------------------------------------------------------ together, and how calls are made
def _layer(M, d, n, seed):
    t = dict(x=_rand(M, d, dtype=torch.bfloat16, seed=seed), r=_rand(M, d, seed=seed + 1), w=_rand(d, scale=0.2, seed=seed + 2) + 1,
             W=_rand(n, d, seed=seed + 3) * d ** -0.5, dy=_rand(M, n, dtype=torch.bfloat16, seed=seed + 4))
    t["wq"] = jg.fp8_buffers(n, d, "block")
    jg.quantize_fp8(t["W"], block=t["wq"])
    t["q"], t["rstd"], t["h"] = jg.fp8_buffers(M, d, "row"), torch.empty(M, device="cuda"), torch.empty(M, d, device="cuda")
    t["qc"], t["gr"], t["gc"] = jg.fp8_buffers(M, d, "col"), jg.fp8_buffers(M, n, "row"), jg.fp8_buffers(M, n, "col")
    t["y"] = torch.empty(M, n, dtype=torch.bfloat16, device="cuda")
    t["dn"] = torch.empty(M, d, dtype=torch.bfloat16, device="cuda")
    t["dx"], t["dW"], t["dw"] = torch.empty(M, d, device="cuda"), torch.empty(n, d, device="cuda"), torch.empty(d, device="cuda")
    t["ws"] = jg.alloc_bytes(max(jg.rms_norm_bwd_workspace_bytes(M, d), jg.grad_clip_workspace_bytes(2)))
    t["norm"] = torch.empty(2, device="cuda")
    return t


def _step(t):
    """Forward and backward of a residual + norm + projection in 8 bits, and the clip of its gradients."""
    jg.rms_norm_fp8(t["x"], *t["q"], residual=t["r"], weight=t["w"], h_out=t["h"], rstd=t["rstd"])
    jg.gemm_fp8(*t["q"], *t["wq"], t["y"])
    jg.quantize_fp8(t["dy"], row=t["gr"], col=t["gc"])
    jg.quantize_fp8(t["h"], col=t["qc"], row_mul=t["rstd"], col_mul=t["w"])
    jg.gemm_fp8(*t["gr"], *t["wq"], t["dn"], b_trans=True)
    jg.gemm_fp8(*t["gc"], *t["qc"], t["dW"], a_trans=True, b_trans=True)
    jg.rms_norm_bwd(t["dn"], t["h"], t["rstd"], t["dx"], weight=t["w"], dweight=t["dw"], ws=t["ws"])
    jg.grad_clip([t["dW"], t["dw"]], 1.0, t["norm"], t["ws"])


OUT = ["h", "y", "dn", "dx", "dW", "dw", "norm"]


@pytest.mark.parametrize("M,d,n", [(1, 256, 384), (5, 768, 1000), (333, 768, 2304), (640, 1024, 512)])
def test_layer(M, d, n):
    """One training step of the layer, every stage against 64 bits on that stage's own inputs, and
    the whole against the unquantised layer: half a step of e4m3 is at most 2^-4 of the value, its
    rms over a step that over sqrt(3), two independent operands give sqrt(2) of it, 0.051 in all."""
    t = _layer(M, d, n, 11)
    _step(t)
    h = (t["x"].float() + t["r"]).double()
    rstd = (h.pow(2).mean(1, keepdim=True) + 1e-6).pow(-0.5)
    y = h * rstd * t["w"].double()
    rel = (_sum_terms(d) / 2 + 12) * U
    check_quantised(y, *t["q"], "row", rel)
    check_quantised(y, *t["qc"], "col", rel)
    X, W, G = held(*t["q"], "row"), held(*t["wq"], "block"), held(*t["gr"], "row")
    check_product(t["y"], X, W)
    check_product(t["dn"], G, W.t())
    coef = t["norm"][1].double()
    unclipped = torch.empty(n, d, device="cuda")
    jg.gemm_fp8(*t["gc"], *t["qc"], unclipped, a_trans=True, b_trans=True)
    check_product(unclipped, held(*t["gc"], "col").t(), held(*t["qc"], "col").t())
    assert ((t["dW"].double() - unclipped.double() * coef).abs() <= 2 * U * unclipped.double().abs()).all()
    norm = torch.sqrt(unclipped.double().pow(2).sum() + (t["dw"].double() / coef).pow(2).sum())
    assert abs(t["norm"][0].item() / norm.item() - 1) < 40 * U
    assert abs(coef.item() - min(1.0, 1.0 / (norm.item() + 1e-6))) < 40 * U
    for got, ref in ((t["y"], y @ t["W"].double().t()), (t["dn"], t["dy"].double() @ t["W"].double()),
                     (unclipped, t["dy"].double().t() @ y)):
        assert ((got.double() - ref).norm() / ref.norm()).item() < 0.0625


def test_layer_on_a_side_stream_and_in_graphs():
    """The step on another stream, and captured twice (two layers, one workspace) and replayed in turn:
    the same bits as the plain call."""
    a, b = _layer(40, 512, 640, 21), _layer(300, 384, 520, 31)
    b["ws"] = a["ws"] = jg.alloc_bytes(max(a["ws"].numel(), b["ws"].numel()))
    want = []
    for t in (a, b):
        _step(t)
        want.append({k: t[k].clone() for k in OUT})
    torch.cuda.synchronize()

    def check():
        torch.cuda.synchronize()
        for t, w in zip((a, b), want):
            for k in OUT:
                assert torch.equal(t[k], w[k]), k
                t[k].fill_(-3.0)

    check()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(a)
        _step(b)
    check()
    graphs = []
    for t in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _step(t)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        check()
    assert jg.device_status() == 0


def test_two_layers_at_once():
    """Two streams with a layer each, over and over without waiting for one another: the bits of the
    calls made alone."""
    layers = [_layer(333, 768, 1000, 41), _layer(24, 1024, 640, 51)]
    want = []
    for t in layers:
        _step(t)
        want.append({k: t[k].clone() for k in OUT})
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(20):
        for t, s in zip(layers, streams):
            with torch.cuda.stream(s):
                _step(t)
    torch.cuda.synchronize()
    for t, w in zip(layers, want):
        for k in OUT:
            assert torch.equal(t[k], w[k]), k
    assert jg.device_status() == 0


FIRST = """
import torch
import paper_2607_17572_gb300 as jg
x, w = torch.randn(40, 512, device="cuda"), torch.randn(640, 512, device="cuda")
(q, s), (wq, ws) = jg.fp8_buffers(40, 512, "row"), jg.fp8_buffers(640, 512, "block")
y, dx, rstd = torch.empty(40, 640, device="cuda"), torch.empty(40, 512, device="cuda"), torch.empty(40, device="cuda")
dw, n = torch.empty(512, device="cuda"), torch.empty(2, device="cuda")
work = jg.alloc_bytes(jg.rms_norm_bwd_workspace_bytes(40, 512) + jg.grad_clip_workspace_bytes(1))
def step():
    jg.rms_norm_fp8(x, q, s, rstd=rstd)
    jg.quantize_fp8(w, block=(wq, ws))
    jg.gemm_fp8(q, s, wq, ws, y)
    jg.rms_norm_bwd(x, x, rstd, dx, dweight=dw, ws=work)
    jg.grad_clip([dx], 1.0, n, work)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    step()
g.replay()
torch.cuda.synchronize()
outs = (y, dx, dw, n)
got = [t.clone() for t in outs]
step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, outs)) and jg.device_status() == 0
"""


def test_the_first_calls_of_a_process_may_be_captured():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_many_calls_of_one_product_give_the_same_bits():
    a, sa, _ = _operand(3, 4096, "row", 1)
    b, sb, _ = _operand(640, 4096, "block", 2)
    c = torch.empty(20, 3, 640, device="cuda")
    for i in range(20):
        jg.gemm_fp8(a, sa, b, sb, c[i])
    assert (c == c[0]).all()
    assert jg.device_status() == 0


# ------------------------------------------------------------------ refusals of the binding
def test_refusals():
    x = _rand(4, 64)
    q, s = jg.fp8_buffers(4, 64, "row")
    with pytest.raises(jg.JaggError, match="float32 or bfloat16"):
        jg.rms_norm_fp8(x.half(), q, s)
    with pytest.raises(jg.JaggError, match="expected"):
        jg.rms_norm_fp8(x, q, s[:, :3])
    with pytest.raises(jg.JaggError, match="float8"):
        jg.rms_norm_fp8(x, torch.empty(4, 64, device="cuda"), s)
    with pytest.raises(jg.JaggError, match="contiguous"):
        jg.rms_norm_fp8(_rand(64, 4).t(), q, s)
    with pytest.raises(jg.JaggError, match="CUDA"):
        jg.rms_norm_fp8(x.cpu(), q, s)
    with pytest.raises(jg.JaggError, match="pitch"):
        jg.rms_norm_fp8(x, torch.empty(4, 66, dtype=torch.float8_e4m3fn, device="cuda")[:, :64], s)
    with pytest.raises(jg.JaggError, match="multiple of 4"):
        jg.rms_norm_fp8(_rand(4, 200), jg.fp8_buffers(4, 200, "row")[0], torch.empty(2, 5, device="cuda")[:, :4])
    with pytest.raises(jg.JaggError, match="workspace"):
        jg.rms_norm_bwd(x, x, torch.empty(4, device="cuda"), torch.empty_like(x), dweight=torch.empty(64, device="cuda"))
    b, sb = jg.fp8_buffers(8, 64, "block")
    with pytest.raises(jg.JaggError, match="accumulation"):
        jg.gemm_fp8(q, s, b, sb, torch.empty(4, 8, dtype=torch.bfloat16, device="cuda"), accumulate=True)
    with pytest.raises(jg.JaggError, match="expected"):
        jg.gemm_fp8(q, s, b, sb, torch.empty(4, 9, device="cuda"))
    with pytest.raises(jg.JaggError, match="overlap"):
        jg.gemm_fp8(q, s, b, sb, torch.empty(8, device="cuda").expand(4, 8))
