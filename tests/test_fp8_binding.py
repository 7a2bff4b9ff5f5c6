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
