"""Argument errors of the 8-bit and clipping entry points are caught on the host, before any launch
(so these calls run without a device), and name the entry point."""
import ctypes

import pytest

FAKE = 1 << 20  # never dereferenced: every call fails first


@pytest.fixture(scope="module")
def jg():
    from paper_2607_17572_gb300 import _build
    _build.build()
    import paper_2607_17572_gb300 as jg
    jg.lib()
    return jg


def _refused(jg, status, code, *words):
    assert status == code, (status, jg.lib().jagg_last_error())
    text = jg.lib().jagg_last_error().decode()
    for w in words:
        assert w in text, text


NORM = dict(x=FAKE, x_dtype=1, ldx=64, residual=FAKE, h_dtype=0, ldh=64, weight=FAKE, w_dtype=0, rows=4, d=64, eps=1e-6,
            h_out=FAKE, q=FAKE, ldq=64, scale=FAKE, lds=4, rstd=FAKE, stream=None)


@pytest.mark.parametrize("change,code,word", [
    (dict(x=None), -1, "null"), (dict(q=None), -1, "null"), (dict(scale=None), -1, "null"), (dict(x_dtype=2), -1, "dtype"),
    (dict(rows=-1), -1, "rows"), (dict(d=0), -1, "d=0"), (dict(d=40000, ldx=40000, ldh=40000, ldq=40000), -2, "32768"),
    (dict(ldx=63), -1, "pitch"), (dict(ldh=63), -1, "pitch"), (dict(ldq=72), -1, "pitch"), (dict(ldq=48), -1, "pitch"),
    (dict(lds=3), -1, "scales"), (dict(lds=6), -1, "scales"), (dict(scale=FAKE + 4), -1, "scales"), (dict(q=FAKE + 8), -1, "aligned"), (dict(x=FAKE + 1), -1, "aligned"),
    (dict(residual=FAKE + 2), -1, "aligned"), (dict(eps=-1.0), -1, "eps"), (dict(eps=float("nan")), -1, "eps")])
def test_norm_refusals(jg, change, code, word):
    a = dict(NORM, **change)
    _refused(jg, jg.lib().jagg_rms_norm_fp8(*a.values()), code, "jagg_rms_norm_fp8", word)


BWD = dict(dy=FAKE, dy_dtype=1, lddy=64, h=FAKE, h_dtype=0, ldh=64, weight=FAKE, w_dtype=0, rstd=FAKE, dh=FAKE, dx=FAKE,
           ldg=64, rows=4, d=64, dweight=FAKE, accumulate=0, ws=FAKE, ws_bytes=4 * 64 * 4, stream=None)


@pytest.mark.parametrize("change,code,word", [
    (dict(dy=None), -1, "null"), (dict(h=None), -1, "null"), (dict(rstd=None), -1, "null"), (dict(dx=None), -1, "null"),
    (dict(h_dtype=7), -1, "dtype"), (dict(ldg=60), -1, "pitch"), (dict(lddy=60), -1, "pitch"), (dict(ws=None), -5, "workspace"),
    (dict(ws_bytes=1023), -5, "workspace"), (dict(ws=FAKE + 4), -1, "workspace"), (dict(dweight=FAKE + 2), -1, "dweight"),
    (dict(dx=FAKE + 2), -1, "aligned"), (dict(d=-3), -1, "d=-3"), (dict(d=1 << 20), -2, "32768")])
def test_norm_backward_refusals(jg, change, code, word):
    a = dict(BWD, **change)
    _refused(jg, jg.lib().jagg_rms_norm_bwd(*a.values()), code, "jagg_rms_norm_bwd", word)


def test_norm_backward_workspace(jg):
    f = jg.rms_norm_bwd_workspace_bytes
    assert f(0, 64) == 0 and f(1, 64) == 256 and f(10 ** 6, 64) == f(10 ** 7, 64)


@pytest.mark.parametrize("change,word", [
    (dict(), "no form"), (dict(row=(FAKE, 60, FAKE, 4)), "row"), (dict(col=(FAKE, 64, FAKE, 63)), "column"),
    (dict(block=(FAKE, 64, None, 1)), "without scales"), (dict(block=(FAKE + 4, 64, FAKE, 1)), "block"),
    (dict(block=(FAKE, 64, FAKE, 0)), "block"), (dict(row=(FAKE, 64, FAKE, 4), ldx=63), "pitch"),
    (dict(row=(FAKE, 64, FAKE, 4), x=None), "null"), (dict(row=(FAKE, 64, FAKE, 4), rows=1 << 24), "rows"),
    (dict(row=(FAKE, 64, FAKE, 4), x_dtype=5), "dtype"), (dict(col=(FAKE, 64, FAKE + 8, 64)), "column"),
    (dict(col=(FAKE, 64, FAKE, 66)), "column"), (dict(row=(FAKE, 64, FAKE, 4), row_mul=FAKE + 2), "aligned")])
def test_quantise_refusals(jg, change, word):
    o = {f: ctypes.byref(jg.Fp8Out(*change[f])) if f in change else None for f in ("row", "col", "block")}
    st = jg.lib().jagg_quantize_fp8(change.get("x", FAKE), change.get("x_dtype", 1), change.get("ldx", 64),
                                    change.get("rows", 4), 64, change.get("row_mul"), None, 0, o["row"], o["col"],
                                    o["block"], None)
    _refused(jg, st, -1, "jagg_quantize_fp8", word)


GEMM = dict(M=8, N=200, K=300, A=FAKE, lda=304, a_scale=FAKE, lda_scale=8, B=FAKE, ldb=304, b_scale=FAKE, ldb_scale=3,
            C=FAKE, ldc=200, bias=None, a_trans=0, b_trans=0, b_block=1, c_dtype=1, bias_dtype=0, accumulate=0)


@pytest.mark.parametrize("change,word", [
    (dict(M=-1), "outside"), (dict(N=1 << 31), "outside"), (dict(A=None), "A needs"), (dict(lda=300), "A needs"),
    (dict(lda=288), "A needs"), (dict(A=FAKE + 8), "A needs"), (dict(ldb=300), "B needs"), (dict(B=None), "B needs"),
    (dict(a_scale=None), "A's scales"), (dict(lda_scale=7), "A's scales"), (dict(ldb_scale=2), "B's scales"),
    (dict(b_block=0, ldb_scale=199), "B's scales"), (dict(b_block=0, ldb_scale=202), "B's scales"),
    (dict(b_block=0, ldb_scale=200, b_scale=FAKE + 4), "B's scales"), (dict(lda_scale=10), "A's scales"), (dict(b_trans=1, ldb=208, ldb_scale=1), "B's scales"),
    (dict(a_trans=1, lda=0), "A needs"), (dict(C=None), "output"), (dict(ldc=199), "output"), (dict(C=FAKE + 1), "output"),
    (dict(accumulate=1), "accumulation"), (dict(c_dtype=3), "dtype"), (dict(bias=FAKE + 2), "bias")])
def test_product_refusals(jg, change, word):
    d = jg.GemmFp8Desc(**dict(GEMM, **change))
    _refused(jg, jg.lib().jagg_gemm_fp8(ctypes.byref(d), None), -1, "jagg_gemm_fp8", word)


@pytest.mark.parametrize("plan,change,word", [
    ((64, 0, 1, 0), {}, "pair tiles"), ((0, 128, 0, 0), {}, "splits"), ((0, 128, 9, 0), {}, "splits"), ((0, 128, 4, 0), {}, "splits"),
    ((0, 64, 1, 0), {}, "tiles"), ((0, 128, 1, 1), {}, "tiles"), ((0, 16, 1, 1), dict(a_trans=1, lda=16), "tiles"),
    ((0, 128, 1, 0), dict(K=0), "empty"), ((256, 0, 1, 0), dict(M=0), "empty"), ((256, 0, 1, 0), dict(A=None), "A needs")])
def test_product_by_kernel_refusals(jg, plan, change, word):
    d = jg.GemmFp8Desc(**dict(GEMM, **change))
    _refused(jg, jg.lib().jagg_test_gemm_fp8(ctypes.byref(d), *plan, None), -1, "jagg_test_gemm_fp8", word)


def test_product_without_descriptor(jg):
    _refused(jg, jg.lib().jagg_gemm_fp8(None, None), -1, "null")


@pytest.mark.parametrize("change,code,word", [
    (dict(count=-1), -1, "tensors"), (dict(grads=None), -1, "list"), (dict(numel=None), -1, "list"), (dict(dtype=9), -1, "dtype"),
    (dict(norm_out=None), -1, "norm_out"), (dict(norm_out=FAKE + 2), -1, "norm_out"), (dict(ws=None), -5, "workspace"),
    (dict(ws_bytes=16), -5, "workspace"), (dict(ws=FAKE + 4), -1, "aligned"), (dict(lens=(4, -1)), -1, "tensor 1"),
    (dict(ptrs=(FAKE, 0)), -1, "null"), (dict(ptrs=(FAKE + 2, FAKE)), -1, "aligned"), (dict(max_norm=-0.5), -1, "negative"),
    (dict(max_norm=float("nan")), -1, "negative"), (dict(eps=-1e-9), -1, "negative")])
def test_clip_refusals(jg, change, code, word):
    ptrs = (ctypes.c_void_p * 2)(*change.get("ptrs", (FAKE, FAKE)))
    lens = (ctypes.c_int64 * 2)(*change.get("lens", (4, 4)))
    a = dict(grads=ptrs, numel=lens, count=2, dtype=0, norm_out=FAKE, ws=FAKE, ws_bytes=1 << 20)
    a.update({k: v for k, v in change.items() if k in a})
    grads = a.pop("grads")
    if not {"max_norm", "eps"} & set(change):
        _refused(jg, jg.lib().jagg_grad_norm(grads, *a.values(), None), code, "jagg_grad_norm", word)
    tail = (change.get("max_norm", 1.0), change.get("eps", 1e-6))
    st = jg.lib().jagg_grad_clip(grads, None, a["numel"], a["count"], a["dtype"], *tail, a["norm_out"], a["ws"],
                                 a["ws_bytes"], None)
    _refused(jg, st, code, "jagg_grad_clip", word)


def test_clip_workspace_grows_with_the_lists(jg):
    f = jg.grad_clip_workspace_bytes
    assert f(0) == f(1) == f(1000) > 0 and f(1001) == 2 * f(1)


@pytest.mark.parametrize("grads,out", [
    ((FAKE, FAKE), None),                                          # the same tensor twice, in place
    ((FAKE + 8, FAKE), None),                                      # the second ends inside the first
    ((FAKE, FAKE + 64), (FAKE + 64, FAKE + 128)),                  # an output over another gradient
    ((FAKE, FAKE + 64), (FAKE + 8, FAKE + 64)),                    # over its own gradient, shifted
    ((FAKE, FAKE + 64), (FAKE + 128, FAKE + 136))])                # over another output
def test_clip_of_overlapping_tensors(jg, grads, out):
    P = ctypes.c_void_p * 2
    st = jg.lib().jagg_grad_clip(P(*grads), P(*out) if out else None, (ctypes.c_int64 * 2)(4, 4), 2, 0, 1.0, 1e-6, FAKE, FAKE,
                                 1 << 20, None)
    _refused(jg, st, -1, "jagg_grad_clip", "overlap")
