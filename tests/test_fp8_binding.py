"""What the binding of the 8-bit operators makes of its arguments, on the CPU: a call whose tensors are
all right ends at the check that they are on a GPU, and not before."""
import pytest
import torch

import paper_2607_17572_gb300 as jg


def _reaches_the_device_check(call, *args, **kw):
    with pytest.raises(jg.JaggError, match="must be CUDA tensors"):
        call(*args, **kw)


@pytest.fixture
def default_bfloat16():
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.bfloat16)
    yield
    torch.set_default_dtype(before)


@pytest.mark.parametrize("form", ["row", "col", "block"])
def test_scales_are_f32_whatever_the_default_dtype(default_bfloat16, form):
    q, s = jg.fp8_buffers(300, 200, form, "cpu")
    assert q.dtype == torch.float8_e4m3fn and s.dtype == torch.float32
    x = torch.empty(300, 200)
    _reaches_the_device_check(jg.quantize_fp8, x, **{form: (q, s)})


def _row(wide, cols, dtype=torch.float32):
    """A matrix of one row, cut out of wider ones."""
    return torch.zeros(3, wide, dtype=dtype)[1:2, :cols]


@pytest.mark.parametrize("d", [64, 65])
def test_the_pitch_of_a_single_row_says_nothing(d):
    q, s = jg.fp8_buffers(1, d, "row", "cpu")
    x = torch.zeros(1, d)
    _reaches_the_device_check(jg.rms_norm_fp8, x, q, s, residual=_row(200, d), h_out=_row(300, d))
    _reaches_the_device_check(jg.rms_norm_fp8, x, q, s, residual=torch.zeros(1, d), h_out=_row(300, d))
    _reaches_the_device_check(jg.rms_norm_bwd, x, _row(100, d), torch.zeros(1), torch.zeros(1, d), dh=_row(101, d))
    _reaches_the_device_check(jg.gemm_fp8, torch.zeros(2, 70, dtype=torch.uint8)[1:, :64], torch.zeros(1, 1),
                              *jg.fp8_buffers(d, 64, "block", "cpu"), _row(131, d))


def test_the_pitches_of_several_rows_have_to_agree():
    q, s = jg.fp8_buffers(2, 64, "row", "cpu")
    x, wide = torch.zeros(2, 64), torch.zeros(2, 80)[:, :64]
    with pytest.raises(jg.JaggError, match="pitch"):
        jg.rms_norm_fp8(x, q, s, residual=x, h_out=wide)
    with pytest.raises(jg.JaggError, match="pitch"):
        jg.rms_norm_bwd(x, x, torch.zeros(2), x, dh=wide)
    with pytest.raises(jg.JaggError, match="overlap"):
        jg.rms_norm_fp8(torch.zeros(64).expand(2, 64), q, s)


@pytest.mark.parametrize("K", [100, 700])
@pytest.mark.parametrize("b_trans", [False, True])
def test_block_scales_of_a_single_column_need_no_alignment(b_trans, K):
    """One column's block scales have the shape of its vector scales (of [K, 1]: always; of [1, K]: for one
    group) and mean the same; blocks may lie anywhere."""
    a, sa = jg.fp8_buffers(5, K, "row", "cpu")
    b = jg.fp8_buffers(*((K, 1) if b_trans else (1, K)), "block", "cpu")[0]
    g = -(-K // 128)
    sb = torch.ones(g + 1)[1:].view((g, 1) if b_trans else (1, g))
    d = jg._fp8_desc(a, sa, b, sb, torch.zeros(5, 1), False, b_trans, None, False, -1)
    assert d.b_block == 1 and d.b_scale == sb.data_ptr() and d.ldb_scale >= (1 if b_trans else g)
    _reaches_the_device_check(jg.gemm_fp8, a, sa, b, sb, torch.zeros(5, 1), b_trans=b_trans)


def test_the_form_of_b_is_seen_from_its_scales():
    a, sa = jg.fp8_buffers(5, 300, "row", "cpu")
    for N in (1, 2, 3, 128, 129, 384, 400):
        for b_trans in (False, True):
            shape = (300, N) if b_trans else (N, 300)
            for form in ("block", "col" if b_trans else "row"):
                b, sb = jg.fp8_buffers(*shape, form, "cpu")
                d = jg._fp8_desc(a, sa, b, sb, torch.zeros(5, N), False, b_trans, None, False, -1)
                # a [300, 1] matrix: both forms are the same addresses
                assert d.b_block == (form == "block" or (N == 1 and b_trans)), (N, b_trans, form)
                assert d.ldb_scale >= (sb.shape[1] if N > 1 or not b_trans else 1)
    b = jg.fp8_buffers(200, 300, "row", "cpu")[0]
    for wrong in ((1, 3), (3, 199), (2, 2), (200, 3)):
        with pytest.raises(jg.JaggError, match="expected"):
            jg._fp8_desc(a, sa, b, torch.zeros(*wrong), torch.zeros(5, 200), False, False, None, False, -1)
