"""Scales and codes to the bit: scale = max(amax / 448, 2^-126) and code = e4m3(x r), r = 1 / scale, with
one f32 rounding at the quotient, the reciprocal and the product each.

Nothing here has a tolerance.  The oracle divides in f64 and rounds to f32, which is the rounding of the exact
quotient of two f32 (53 bits are more than 2 * 24 + 1), and multiplies in f32."""
import pytest
import torch

from fp8_reference import TOP, peaks, spread

pytestmark = pytest.mark.gpu

jg = pytest.importorskip("paper_2607_17572_gb300")

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
FORMS = ("row", "col", "block")


def _check(y, q, s, form):
    """q, s hold the f32 matrix y; codes compared as bytes (the sign of a zero too), NaN as NaN."""
    want_s = (peaks(y, form).double() / TOP).float().clamp(min=2.0 ** -126)
    assert torch.equal(s.isnan(), want_s.isnan()) and torch.equal(s.nan_to_num(1.0), want_s.nan_to_num(1.0))
    r = (1.0 / spread(s, *y.shape, form)).float()
    want = (y * r).to(torch.float8_e4m3fn)
    got = q.view(torch.float8_e4m3fn)
    nan = want.float().isnan()
    assert torch.equal(got.float().isnan(), nan)
    diff = (got.view(torch.uint8) != want.view(torch.uint8)) & ~nan
    assert not diff.any(), f"{form}: {int(diff.sum())} of {diff.numel()} codes"


def _matrix(rows, cols, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, device="cuda", generator=g) * torch.exp(torch.randn(cols, device="cuda", generator=g))
    x = x.to(dtype)
    x[rows // 2, ::3] = -0.0
    return x


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 4096), (300, 1024), (1024, 776), (257, 1001), (130, 129), (1, 1)])
def test_quantised_codes(rows, cols, x):
    xs = _matrix(rows, cols, DT[x], 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    rm, cm = torch.rand(rows, device="cuda", generator=g) + 0.1, torch.randn(cols, device="cuda", generator=g)
    for mul in (dict(), dict(row_mul=rm, col_mul=cm)):
        y = xs.float()
        if mul:
            y = y * rm[:, None] * cm
        b = {f: jg.fp8_buffers(rows, cols, f) for f in FORMS}
        jg.quantize_fp8(xs, **b, **mul)
        for f in FORMS:
            _check(y, *b[f], f)


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [256, 250])
def test_codes_at_the_ends_of_the_range(cols, x):
    """Groups whose scales run from the floor 2^-126 to the largest, f32's subnormal values among them, and groups of
    which one element is infinite or NaN."""
    xs = _matrix(384, cols, torch.float32, 3)
    e = torch.linspace(-149, 124, 384, device="cuda").round()
    xs = xs.clamp(-4, 4).double() * torch.exp2(e.double())[:, None]
    for y in (xs, xs[torch.randperm(384, generator=torch.Generator().manual_seed(1)).cuda()]):
        y = y.float().to(DT[x])
        for at, bad in ((None, 0.0), ((5, 7), float("inf")), ((300, 140), float("-inf")), ((200, 3), float("nan"))):
            if at:
                y[at] = bad
            b = {f: jg.fp8_buffers(384, cols, f) for f in FORMS}
            jg.quantize_fp8(y, **b)
            for f in FORMS:
                _check(y.float(), *b[f], f)


def test_a_group_of_subnormal_values():
    """1e-40 among zeros: the scale's floor, and the code of 1e-40 times 2^126."""
    x = torch.zeros(256, 256, device="cuda")
    x[128:, 200] = 1e-40
    b = {f: jg.fp8_buffers(256, 256, f) for f in FORMS}
    jg.quantize_fp8(x, **b)
    code = (torch.tensor(1e-40, dtype=torch.float32).double() * 2.0 ** 126).to(torch.float8_e4m3fn)
    assert code.float() != 0
    for f in FORMS:
        q, s = b[f]
        assert (s == 2.0 ** -126).all()
        want = torch.zeros(256, 256, device="cuda")
        want[128:, 200] = code.float().item()
        assert torch.equal(q.float(), want)


@pytest.mark.parametrize("x,h", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,d", [(1, 128), (300, 768), (40, 4096), (9, 16384), (200, 1001), (30, 8195), (5, 9001)])
def test_norm_codes(rows, d, x, h):
    """y = h rstd w formed in f32 from what the call stored, and its scales and codes."""
    xs, r = _matrix(rows, d, DT[x], 4), _matrix(rows, d, DT[h], 5)
    w = torch.randn(d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(6))
    out, rstd = torch.empty_like(r), torch.empty(rows, device="cuda")
    q, s = jg.fp8_buffers(rows, d, "row")
    jg.rms_norm_fp8(xs, q, s, residual=r, weight=w, h_out=out, rstd=rstd)
    _check(out.float() * rstd[:, None] * w, q, s, "row")
    jg.rms_norm_fp8(xs, q, s, residual=r, weight=w * 1e-33, rstd=rstd)
    _check(out.float() * rstd[:, None] * (w * 1e-33), q, s, "row")


@pytest.mark.parametrize("d", [512, 333])
def test_rows_whose_squares_leave_f32(d):
    """Finite rows above the range of the sum: 1 / rms is 0, and so are the codes.  Small rows with eps = 0: as any
    other while their squares are normal numbers."""
    x = torch.randn(3, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(7))
    x[0] *= 1e25
    x[1] *= 1e-15
    q, s = jg.fp8_buffers(3, d, "row")
    rstd = torch.empty(3, device="cuda")
    jg.rms_norm_fp8(x, q, s, eps=0.0, rstd=rstd)
    assert rstd[0] == 0 and (q[0].float() == 0).all()
    ref = x[1:].double().pow(2).mean(1).pow(-0.5)
    # d terms and the shuffles, halved by the square root, the mean, the root and the reciprocal: u each
    assert ((rstd[1:].double() - ref).abs() <= (d / 2 + 40) * 2.0 ** -24 * ref).all()
    _check(x * rstd[:, None], q, s, "row")
