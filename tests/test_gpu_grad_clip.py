"""The global gradient norm and the clip by it, against 64 bits.

Squares are summed in f32 over 32 terms of a thread (33 roundings, halved by the square root) and in
f64 beyond: norm and coefficient are within 20 u, u = 2^-24, and the output within one more product."""
import pytest
import torch

from fp8_reference import U, half_step

pytestmark = pytest.mark.gpu

jg = pytest.importorskip("paper_2607_17572_gb300")

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _tensors(sizes, dtype, scale=1.0, offset=0, seed=0):
    """Views of one buffer, each starting `offset` elements past a multiple of 64."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.zeros(sum(-(-n // 64) * 64 + 64 for n in sizes) + 64, dtype=dtype, device="cuda")
    out, at = [], offset
    for n in sizes:
        v = buf[at:at + n]
        v.copy_(torch.randn(n, device="cuda", generator=g) * scale)
        out.append(v)
        at += -(-n // 64) * 64 + 64
    return buf, out


def _norm(ts):
    return torch.sqrt(sum((t.double().pow(2).sum() for t in ts), torch.zeros((), dtype=torch.float64, device="cuda")))


def _ws(n):
    return jg.alloc_bytes(jg.grad_clip_workspace_bytes(n)).fill_(0xFF)


SETS = [[1], [5, 0, 3], [8192], [8191, 8193, 16384], [0, 0], [64] * 99, [300] * 101, [7] * 1000, [33] * 1001, [100, 70000, 1, 9000] * 520,
        [3_000_001, 12]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("case", range(len(SETS)))
def test_norm_and_clip(case, offset, dtype):
    sizes = SETS[case]
    buf, ts = _tensors(sizes, DT[dtype], offset=offset, seed=case)
    ws = _ws(len(ts))
    ref = _norm(ts).item()
    n1, n2 = torch.full((1,), -1.0, device="cuda"), torch.full((2,), -1.0, device="cuda")
    jg.grad_norm(ts, n1, ws)
    assert abs(n1.item() - ref) <= 20 * U * ref
    for max_norm in (0.5 * ref, 2.0 * ref + 1.0):
        coef = min(1.0, max_norm / (ref + 1e-6))
        # into other tensors, then in place
        obuf, outs = _tensors(sizes, DT[dtype], offset=offset, seed=99)
        before = buf.clone()
        jg.grad_clip(ts, max_norm, n2, ws, out=outs)
        assert torch.equal(buf, before)
        assert abs(n2[0].item() - ref) <= 20 * U * ref and abs(n2[1].item() - coef) <= 24 * U
        for t, o in zip(ts, outs):
            want = t.double() * coef
            assert ((o.double() - want).abs() <= (25 * U + half_step(DT[dtype])) * want.abs() + 2.0 ** -133).all()
        gaps = torch.ones_like(obuf, dtype=torch.bool)
        at = offset
        for n in sizes:
            gaps[at:at + n] = False
            at += -(-n // 64) * 64 + 64
        assert (obuf[gaps] == 0).all()
    half = 0.5 * ref
    jg.grad_clip(ts, half, n2, ws)
    for t, o in zip(ts, outs):
        want = o.double() * min(1.0, half / (ref + 1e-6))  # outs hold the gradients times 1
        assert ((t.double() - want).abs() <= (25 * U + half_step(DT[dtype])) * want.abs() + 2.0 ** -133).all()


@pytest.mark.parametrize("scale", [1e-25, 1e-18, 1e18, 1e30])
def test_squares_outside_f32(scale):
    _, ts = _tensors([5000, 100000], torch.float32, scale=scale)
    out = torch.empty(2, device="cuda")
    ref = _norm(ts).item()
    before = [t.clone() for t in ts]
    jg.grad_clip(ts, ref / 4, out, _ws(2), eps=0.0)
    assert abs(out[0].item() / ref - 1) <= 20 * U and abs(out[1].item() - 0.25) <= 24 * U
    for t, b in zip(ts, before):
        assert ((t.double() - 0.25 * b.double()).abs() <= 26 * U * b.double().abs()).all()


def test_zero_and_non_finite_gradients():
    out, ws = torch.empty(2, device="cuda"), _ws(2)
    z = [torch.zeros(1000, device="cuda"), torch.zeros(20000, device="cuda")]
    jg.grad_clip(z, 1.0, out, ws)
    assert out.tolist() == [0.0, 1.0] and all((t == 0).all() for t in z)
    jg.grad_clip(z, 1.0, out, ws, eps=0.0)
    assert out.tolist() == [0.0, 1.0] and all((t == 0).all() for t in z)
    z[0][3] = float("inf")
    z[1][5] = 2.0
    jg.grad_clip(z, 1.0, out, ws)
    assert out.tolist() == [float("inf"), 0.0]
    assert z[0][3].isnan() and z[0].isnan().sum() == 1 and (z[1] == 0).all()
    z[0][3] = float("nan")
    jg.grad_clip(z, 1.0, out, ws)
    assert out.isnan().all() and all(t.isnan().all() for t in z)


def test_no_limit():
    _, ts = _tensors([100, 9000], torch.float32)
    before = [t.clone() for t in ts]
    out, ws = torch.empty(2, device="cuda"), _ws(2)
    jg.grad_clip(ts, float("inf"), out, ws)
    assert out[1].item() == 1.0 and all(torch.equal(t, b) for t, b in zip(ts, before))
    ts[1][7] = float("inf")
    jg.grad_clip(ts, float("inf"), out, ws)
    assert out.tolist() == [float("inf"), 1.0] and torch.equal(ts[0], before[0])


def test_more_than_2_31_elements():
    """Offsets beyond 32 bits: the first, some middle and the last elements of one tensor."""
    n = 2**31 + 12345
    g = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(2, device="cuda")
    jg.grad_clip([g], 1.0, out, _ws(1))
    ref = float(n) ** 0.5
    assert abs(out[0].item() / ref - 1) <= 20 * U
    want = torch.tensor(1.0 / ref, dtype=torch.float64).to(torch.bfloat16)
    for part in (g[:3], g[2**31 - 3:2**31 + 3], g[-3:]):
        assert (part.cpu() == want).all()


def test_neighbouring_and_shared_inputs():
    """Tensors that touch are not an overlap, in any order, nor is an input that is only read listed twice;
    the norm counts such an input twice."""
    buf = torch.randn(3000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    parts = [buf[1000:2500], buf[:1000], buf[2500:]]
    before, norm = buf.clone(), buf.double().norm().item()
    out, ws = torch.empty(2, device="cuda"), _ws(3)
    jg.grad_clip(parts, 1.0, out, ws)
    assert abs(out[0].item() / norm - 1) <= 20 * U
    assert torch.equal(buf, before * out[1])
    outs = [torch.empty_like(before) for _ in range(2)]
    jg.grad_clip([before, before], 1.0, out, ws, out=outs)
    assert abs(out[0].item() / (2**0.5 * norm) - 1) <= 20 * U
    assert all(torch.equal(o, before * out[1]) for o in outs)


def test_clip_to_zero_and_no_tensors():
    _, ts = _tensors([100, 9000], torch.float32)
    out, ws = torch.empty(2, device="cuda"), _ws(2)
    jg.grad_clip(ts, 0.0, out, ws)
    assert out[1].item() == 0.0 and all((t == 0).all() for t in ts)
    jg.grad_clip([], 1.0, out, ws)
    assert out.tolist() == [0.0, 1.0]
    jg.grad_norm([], out[:1], ws)
    assert out[0].item() == 0.0


def test_the_same_bits_every_time_and_in_a_graph():
    sizes = [70001, 128, 3, 500000]
    _, ts = _tensors(sizes, torch.float32, seed=3)
    _, a = _tensors(sizes, torch.float32, seed=4)
    out, ws = torch.empty(2, device="cuda"), _ws(4)
    jg.grad_clip(ts, 0.1, out, ws, out=a)
    want, nrm = [t.clone() for t in a], out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        jg.grad_clip(ts, 0.1, out, ws, out=a)
    for _ in range(3):
        for t in a:
            t.fill_(9.0)
        out.fill_(-1.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, nrm) and all(torch.equal(x, y) for x, y in zip(a, want))


def test_the_gradient_of_a_window():
    """The flat gradient that dit_joint_vjp fills, clipped tensor by tensor as jagg_param_info lists it."""
    import synth
    cfg = jg.Config.from_workload(synth.WORKLOADS["tiny_dit_f32"])
    table = jg.param_table(cfg)
    flat = torch.zeros(jg.param_count(cfg), device="cuda")
    for i, p in enumerate(table):
        flat[p.offset:p.offset + p.numel] = torch.randn(p.numel, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i))
    views = [flat[p.offset:p.offset + p.numel] for p in table]
    out = torch.empty(2, device="cuda")
    before = flat.clone()
    jg.grad_clip(views, 1.0, out, _ws(len(views)))
    ref = before.double().norm().item()
    assert abs(out[0].item() / ref - 1) <= 20 * U
    want = before.double() / (ref + 1e-6)
    assert ((flat.double() - want).abs() <= 26 * U * want.abs()).all()


def test_refusals():
    x, out, ws = torch.zeros(10, device="cuda"), torch.empty(2, device="cuda"), _ws(1)
    with pytest.raises(jg.JaggError, match="one dtype"):
        jg.grad_clip([x, x.bfloat16()], 1.0, out, ws)
    with pytest.raises(jg.JaggError, match="float32 or bfloat16"):
        jg.grad_clip([x.double()], 1.0, out, ws)
    with pytest.raises(jg.JaggError, match="contiguous"):
        jg.grad_clip([torch.zeros(10, 2, device="cuda").t()], 1.0, out, ws)
    with pytest.raises(jg.JaggError, match="number or length"):
        jg.grad_clip([x], 1.0, out, ws, out=[x, x])
    with pytest.raises(jg.JaggError, match="negative"):
        jg.grad_clip([x], -1.0, out, ws)
    with pytest.raises(jg.JaggError, match="workspace"):
        jg.grad_clip([x], 1.0, out, ws[:8])
    with pytest.raises(jg.JaggError, match="CUDA"):
        jg.grad_norm([x.cpu()], out, ws)
