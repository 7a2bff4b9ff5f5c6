"""Plain 64-bit forms of the 8-bit operators, and the bounds that their rounding allows.

u = 2^-24 is half a step of f32 relative to the value.  A sum of n f32 terms, in whatever order,
is off by at most n u times the sum of magnitudes."""
import torch

U = 2.0 ** -24
TOP = 448.0


def groups(n):
    return -(-n // 128)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def e4m3(v):
    """Nearest e4m3 value of a float64 tensor (ties to even, saturating, NaN kept)."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step).clamp(-TOP, TOP)


def spread(scale, rows, cols, form):
    """The scale of every element, float64 [rows, cols]."""
    s = scale.double()
    if form == "row":
        return s.t().repeat_interleave(128, 1)[:, :cols]
    if form == "col":
        return s.repeat_interleave(128, 0)[:rows]
    return s.repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def peaks(y, form):
    """Largest magnitude of every group, in the scales' layout."""
    rows, cols = y.shape
    p = torch.nn.functional.pad(y.abs(), (0, groups(cols) * 128 - cols, 0, groups(rows) * 128 - rows))
    p = p.view(groups(rows), 128, groups(cols), 128)
    if form == "row":
        return p.amax(3).reshape(-1, groups(cols))[:rows].t()
    if form == "col":
        return p.amax(1).reshape(groups(rows), -1)[:, :cols]
    return p.amax((1, 3))


def check_quantised(y, q, scale, form, rel):
    """q, scale hold y (float64, finite), whose elements the kernel has to a relative `rel`: scales to
    that and their own two roundings; codes equal to the rounding of some value that near."""
    ref = (peaks(y, form) / TOP).clamp(min=2.0 ** -126)
    assert scale.shape == ref.shape
    assert ((scale.double() - ref).abs() <= (rel + 2 * U) * ref).all()
    v = y / spread(ref, *y.shape, form)
    # the element, the scale, the reciprocal and the product with it
    d = 2 * rel + 6 * U
    got = q.view(torch.float8_e4m3fn).double()
    lo, hi = e4m3(v - d * v.abs()), e4m3(v + d * v.abs())
    assert ((got >= lo) & (got <= hi)).all()


def held(q, scale, form):
    """The values that codes and scales stand for, float64."""
    return q.view(torch.float8_e4m3fn).double() * spread(scale, *q.shape, form)


def check_product(c, a, b, bias=None, start=None):
    """c against a b^T (+ bias) (+ start) of float64 operands [M, K], [N, K].  The tensor cores add a
    step's 32 aligned products and the accumulator with at least 23 bits kept of the largest:
    each of the K / 32 steps is off by at most 33 units of 2^-23 of its largest term, in all at most
    2^-18 of the sum of magnitudes of its group; the groups' sums, two scales and the additions
    after them are f32."""
    ref, mag = a @ b.t(), a.abs() @ b.abs().t()
    more = groups(a.shape[1]) + 8
    if bias is not None:
        ref, mag = ref + bias.double(), mag + bias.double().abs()
    if start is not None:
        ref, mag = ref + start.double(), mag + start.double().abs()
    err = (2.0 ** -18 + more * U) * mag
    err = err + half_step(c.dtype) * (ref.abs() + err)
    bad = ((c.double() - ref).abs() > err)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outside, worst {((c.double() - ref).abs() / mag).max():.3g}"
