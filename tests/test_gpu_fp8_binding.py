"""Views that the binding of the 8-bit operators takes, against the same calls on plain tensors.

A view may be off 16 bytes, which takes another kernel and another order of a row's sum: u = 2^-24 for each of
its d terms and for each of the few operations around it, relative to the sum of magnitudes."""
import pytest
import torch

from fp8_reference import U, check_product

pytestmark = pytest.mark.gpu

jg = pytest.importorskip("paper_2607_17572_gb300")


def _rand(*shape, dtype=torch.float32, seed=0):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def _cut(t, wide):
    """The one row of t as a row of a matrix of wider rows, whose other elements are known."""
    buf = torch.full((3, wide), 7.0, device="cuda").to(t.dtype)
    buf[1:2, :t.shape[1]] = t
    return buf, buf[1:2, :t.shape[1]]


def _alone(buf, cols):
    return (buf[0].float() == 7).all() and (buf[2].float() == 7).all() and (buf[1, cols:].float() == 7).all()


@pytest.mark.parametrize("d", [64, 65, 1024])
def test_a_single_row_cut_out_of_wider_ones(d):
    """Operands of one row with pitches of their own, among them such as are no multiple of anything."""
    x, r, w, dy = _rand(1, d, dtype=torch.bfloat16, seed=1), _rand(1, d, seed=2), _rand(d, seed=3), _rand(1, d, seed=4)
    (q, s), (q1, s1) = jg.fp8_buffers(1, d, "row"), jg.fp8_buffers(1, d, "row")
    h, rstd = torch.empty(1, d, device="cuda"), torch.empty(1, device="cuda")
    jg.rms_norm_fp8(x, q, s, residual=r, weight=w, h_out=h, rstd=rstd)
    buf, h1 = _cut(torch.zeros(1, d, device="cuda"), d + 37)
    rstd1 = torch.empty(1, device="cuda")
    jg.rms_norm_fp8(x, q1, s1, residual=_cut(r, d + 5)[1], weight=w, h_out=h1, rstd=rstd1)
    assert torch.equal(h1, h) and _alone(buf, d)
    rel = 2 * (d + 8) * U
    assert ((rstd1 - rstd).abs() <= rel * rstd).all() and ((s1 - s).abs() <= rel * s).all()
    dx = torch.empty(1, d, device="cuda")
    jg.rms_norm_bwd(dy, h, rstd, dx, weight=w, dh=r)
    buf, dx1 = _cut(torch.zeros(1, d, device="cuda"), d + 3)
    jg.rms_norm_bwd(dy, h1, rstd, dx1, weight=w, dh=_cut(r, d + 11)[1])
    g, xh = (dy * w).abs(), (h * rstd).abs()
    assert ((dx1 - dx).abs() <= rel * (r.abs() + rstd * (g + xh * (g * xh).mean()))).all() and _alone(buf, d)
    N = 96
    b = jg.fp8_buffers(N, d, "block")
    jg.quantize_fp8(_rand(N, d, seed=5), block=b)
    for dtype in (torch.float32, torch.bfloat16):
        c = torch.empty(1, N, dtype=dtype, device="cuda")
        jg.gemm_fp8(q, s, *b, c)
        buf, c1 = _cut(torch.zeros(1, N, device="cuda").to(dtype), N + 9)
        jg.gemm_fp8(q, s, *b, c1)
        assert torch.equal(c1, c) and _alone(buf, N)


@pytest.mark.parametrize("M", [1, 5, 300])
@pytest.mark.parametrize("K", [100, 700])
@pytest.mark.parametrize("b_trans", [False, True])
def test_block_scales_of_a_single_column(b_trans, K, M):
    """Scales off 16 bytes and without a pitch of their own: the product of the aligned ones."""
    shape = (K, 1) if b_trans else (1, K)
    a, b = jg.fp8_buffers(M, K, "row"), jg.fp8_buffers(*shape, "block")
    jg.quantize_fp8(_rand(M, K, seed=1), row=a)
    jg.quantize_fp8(_rand(*shape, seed=2), block=b)
    g = -(-K // 128)
    off = torch.empty(g + 1, device="cuda")[1:].view(b[1].shape)
    off.copy_(b[1])
    c, c1 = torch.empty(M, 1, device="cuda"), torch.empty(M, 1, device="cuda")
    jg.gemm_fp8(*a, *b, c, b_trans=b_trans)
    jg.gemm_fp8(*a, b[0], off, c1, b_trans=b_trans)
    assert torch.equal(c, c1)
    va = a[0].double() * a[1].double().t().repeat_interleave(128, 1)[:, :K]
    vb = (b[0].double().flatten() * b[1].double().flatten().repeat_interleave(128)[:K])[None]
    check_product(c, va, vb)
