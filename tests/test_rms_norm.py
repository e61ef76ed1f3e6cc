"""RMS norm with the residual's addition and 8-bit rows with scales, against the formula in 64 bits."""
import ctypes

import numpy as np
import pytest

from paper_2308_15030_b200 import binding

EPS = 1e-6
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}          # largest relative error of one rounding


# ------------------------------------------------------------------ refusals (host checks, no GPU needed)
def _args(**kw):
    base = dict(x=256, weight=256, out=256, x_stride=64, out_stride=64, n_rows=2, d=64, dtype=1, residual_dtype=1, group=0, eps=EPS)
    base.update(kw)
    return binding.RmsNormArgs(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(n_rows=-1), -1), (dict(d=0), -1), (dict(dtype=2), -1), (dict(residual_dtype=3), -1), (dict(dtype=0), -1),
    (dict(group=16), -1), (dict(group=96), -1), (dict(group=512), -1), (dict(group=-1), -1), (dict(eps=-1.0), -1),
    (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(x=None), -1), (dict(weight=None), -1),
    (dict(out=None), -1), (dict(residual_out=256, residual_out_stride=64), -1), (dict(out8=256, out8_stride=64), -1),
    (dict(scales=256, scales_stride=1), -1), (dict(x=257), -1), (dict(out=255), -1), (dict(x_stride=63), -1),
    (dict(out8=256, out8_stride=64, scales=256, scales_stride=1, group=32), -1),
    (dict(residual=256, residual_stride=63), -1), (dict(d=16385, x_stride=20000, out_stride=20000), -7)])
def test_refusals(kw, status):
    assert binding.lib().swapmoe_rms_norm(ctypes.byref(_args(**kw)), None) == status


def test_no_arguments_and_no_rows():
    assert binding.lib().swapmoe_rms_norm(None, None) == -1
    assert binding.lib().swapmoe_rms_norm(ctypes.byref(_args(n_rows=0, x=None)), None) == 0


def test_tensor_checks():
    import torch
    x = torch.zeros(2, 64)
    w = torch.ones(64)
    for kw in (dict(out=torch.zeros(2, 63)), dict(out=torch.zeros(1, 64)), dict(out=torch.zeros(2, 64, dtype=torch.bfloat16)),
               dict(out=torch.zeros(64, 2).t()), dict(out=torch.zeros(2, 64), residual_out=torch.zeros(2, 64)),
               dict(out8=torch.zeros(2, 64, dtype=torch.float8_e4m3fn)), dict(out=torch.zeros(2, 64))):   # the last: not on a GPU
        with pytest.raises(binding.SwapMoEError) as e:
            binding.rms_norm(x, w, EPS, **kw)
        assert e.value.status == -1
    with pytest.raises(binding.SwapMoEError):
        binding.rms_norm(x, torch.ones(63), EPS, out=torch.zeros(2, 64))
    with pytest.raises(binding.SwapMoEError):
        binding.rms_norm(x.half(), w, EPS, out=torch.zeros(2, 64))


# ------------------------------------------------------------------ on the GPU
def _reference(x, r, w, eps, group):
    """(h, y, scales) in 64 bits from float64 CPU tensors."""
    import torch
    h = x if r is None else x + r
    y = h * w / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    T, d = h.shape
    g = group or d
    n = -(-d // g)
    big = torch.nn.functional.pad(y.abs(), (0, n * g - d)).view(T, n, g).amax(2) / 448.0
    return h, y, big


def _rows(T, d, dt, gen, stride=None, offset=0, std=1.0):
    """[T, d] rows `stride` values apart that start `offset` values into their memory; the memory behind them is marked."""
    import torch
    stride = stride or d
    mem = torch.full((T * stride + offset + 8,), 7.0, device="cuda").to(dt)
    v = torch.as_strided(mem, (T, d), (stride, 1), offset)
    v.copy_(torch.empty(T, d, device="cuda").normal_(0.0, std, generator=gen))
    return v, mem


def _untouched(mem, T, d, stride, offset):
    import torch
    keep = torch.ones_like(mem, dtype=torch.bool)
    torch.as_strided(keep, (T, d), (stride, 1), offset).fill_(False)
    return bool((mem.float()[keep] == 7.0).all())


def _check(T, d, dtype="bf16", residual="same", out=True, group=None, stride=None, offset=0, x_values=None, eps=EPS):
    """One call against the reference, with everything that must not be written marked."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T * 10007 + d)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    stride = stride or d
    x, _ = _rows(T, d, dt, gen, stride, offset)
    if x_values is not None:
        x.copy_(x_values)
    w = torch.empty(d, device="cuda").normal_(1.0, 0.3, generator=gen).to(dt)
    rdt = torch.float32 if residual == "fp32" else dt
    r = ro = o = q = s = None
    if residual:
        r, _ = _rows(T, d, rdt, gen, stride, offset, std=2.0)
        ro, ro_mem = _rows(T, d, rdt, gen, stride, offset)
    if out:
        o, o_mem = _rows(T, d, dt, gen, stride, offset)
    n = -(-d // group) if group else 1
    if group is not None:
        q = torch.full((T + 1, d), 7.0, device="cuda").to(torch.float8_e4m3fn)
        s = torch.full((T + 1, n), 7.0, device="cuda")
    binding.rms_norm(x, w, eps, out=o, residual=r, residual_out=ro, out8=q, scales=s, group=group or 0)
    torch.cuda.synchronize()
    h, y, sc = _reference(x.double().cpu(), None if r is None else r.double().cpu(), w.double().cpu(), eps, group)
    # fp32 arithmetic: a sum of d squares in trees of at most 8 + 5 + 32 terms each, one square root, three products: well under
    # 40 roundings of 2^-24
    f32 = 40 * 2.0 ** -24
    if residual:
        # one addition in fp32, one rounding to the residual's type
        assert bool(((ro.double().cpu() - h).abs() <= h.abs() * (2.0 ** -24 + (HALF["bf16"] if rdt == torch.bfloat16 else 0)) * 1.01).all())
        assert _untouched(ro_mem, T, d, stride, offset)
    if out:
        # (h itself is the fp32 sum of x and the residual: an error of 2^-24 of |h|)
        tol = y.abs() * (f32 + HALF[dtype] * (dtype == "bf16")) * 1.01
        assert bool(((o.double().cpu() - y).abs() <= tol).all())
        assert _untouched(o_mem, T, d, stride, offset)
    if group is not None:
        assert bool(((s[:T].double().cpu() - sc).abs() <= sc * f32 * 2).all())
        assert bool((s[T:] == 7.0).all()) and bool((q[T:].float() == 7.0).all())
        # e4m3: half a step is 2^-4 of the value, 2^-10 below the smallest normal number
        got = q[:T].float().double().cpu()
        ideal = y / torch.where(sc > 0, sc, 1.0).repeat_interleave(group or d, 1)[:, :d]
        assert bool(((got - ideal).abs() <= torch.clamp(ideal.abs() * 2.0 ** -4, min=2.0 ** -10) * (1 + 1e-3)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d", [(1, 1), (1, 8), (3, 7), (2, 255), (5, 256), (4, 257), (1, 4096), (33, 1000), (300, 1003), (1200, 768),
                                 (2500, 512), (17, 8200), (3, 16384), (2, 16383)])
def test_widths_and_rows(T, d, dtype):
    _check(T, d, dtype)
    _check(T, d, dtype, group=0)


@pytest.mark.gpu
@pytest.mark.parametrize("group", [0, 32, 64, 128, 256])
@pytest.mark.parametrize("T,d", [(5, 512), (3, 1000), (700, 200), (2, 31), (1500, 1027)])
def test_eight_bit_groups(T, d, group):
    _check(T, d, group=group, out=False)
    _check(T, d, "fp32", group=group, residual=None)


@pytest.mark.gpu
@pytest.mark.parametrize("stride,offset", [(1024, 0), (1008, 8), (1008, 4), (1001, 0), (1021, 3)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides_and_offsets(stride, offset, dtype):
    _check(9, 1000, dtype, stride=stride, offset=offset, group=128)
    _check(600, 1000, dtype, stride=stride, offset=offset, group=0)


@pytest.mark.gpu
@pytest.mark.parametrize("residual", [None, "same", "fp32"])
@pytest.mark.parametrize("T", [7, 900])
def test_residual_types(T, residual):
    _check(T, 704, residual=residual, group=64)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [1e-30, 1e-20, 1e18, 1e25, 3e37])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_rows_of_any_magnitude(dtype, size, eps):
    import torch
    x = torch.linspace(-1.0, 1.0, 500, device="cuda").repeat(4, 1) * size
    _check(4, 500, dtype, residual=None, x_values=x, eps=eps, group=0 if eps == 0.0 or size > 1 else None)


@pytest.mark.gpu
def test_zero_rows_nan_and_infinity():
    import torch
    x = torch.ones(4, 512, dtype=torch.bfloat16, device="cuda")
    x[0] = 0
    x[1, 3] = float("nan")
    x[2, 5] = float("inf")
    w = torch.ones(512, dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(x)
    q = torch.empty(4, 512, dtype=torch.float8_e4m3fn, device="cuda")
    for group in (0, 128):
        s = torch.empty(4, 4 if group else 1, device="cuda")
        binding.rms_norm(x, w, EPS, out=o, out8=q, scales=s, group=group)
        assert bool((o[0] == 0).all()) and bool((q[0].float() == 0).all()) and bool((s[0] == 0).all())
        assert bool(o[1].isnan().all()) and bool(s[1].isnan().all()) and bool(q[1].float().isnan().all())
        assert bool(o[2, 5].isnan()) and bool((o[2, :5] == 0).all()) and bool((o[2, 6:] == 0).all())
        assert bool(s[2, 0].isnan())
        assert bool((o[3] == 1).all()) and bool((q[3].float() == 448).all())


@pytest.mark.gpu
@pytest.mark.parametrize("d", [512, 515])
def test_in_place(d):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.empty(40, d, device="cuda").normal_(generator=gen).bfloat16()
    r = torch.empty(40, d, device="cuda").normal_(generator=gen).bfloat16()
    w = torch.empty(d, device="cuda").normal_(1.0, 0.2, generator=gen).bfloat16()
    ro, o = torch.empty_like(x), torch.empty_like(x)
    binding.rms_norm(x, w, EPS, out=o, residual=r, residual_out=ro)
    x2, r2 = x.clone(), r.clone()
    binding.rms_norm(x2, w, EPS, out=x2, residual=r2, residual_out=r2)
    assert torch.equal(x2, o) and torch.equal(r2, ro)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 2500])
def test_the_addition_alone_and_the_norm_over_x(T):
    """Only residual_out; and the sum written over x while out goes elsewhere."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T)
    x = torch.empty(T, 512, device="cuda").normal_(generator=gen).bfloat16()
    r = torch.empty(T, 512, device="cuda").normal_(generator=gen).bfloat16()
    w = torch.ones(512, dtype=torch.bfloat16, device="cuda")
    ro, o, o2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    binding.rms_norm(x, w, EPS, residual=r, residual_out=ro)
    assert torch.equal(ro, (x.float() + r.float()).bfloat16())
    binding.rms_norm(x, w, EPS, out=o, residual=r)
    x2 = x.clone()
    binding.rms_norm(x2, w, EPS, out=o2, residual=r, residual_out=x2)
    assert torch.equal(x2, ro) and torch.equal(o2, o)


@pytest.mark.gpu
def test_weights_that_are_not_finite():
    import torch
    x = torch.ones(2, 256, device="cuda")
    w = torch.ones(256, device="cuda")
    w[3], w[70] = float("nan"), float("inf")
    o, q = torch.empty_like(x), torch.empty(2, 256, dtype=torch.float8_e4m3fn, device="cuda")
    for group in (0, 64):
        s = torch.empty(2, 4 if group else 1, device="cuda")
        binding.rms_norm(x, w, EPS, out=o, out8=q, scales=s, group=group)
        assert bool(o[:, 3].isnan().all()) and bool(o[:, 70].isinf().all())
        keep = torch.ones(256, dtype=torch.bool, device="cuda")
        keep[3] = keep[70] = False
        assert bool(((o[:, keep] - 1).abs() < 1e-5).all())
        assert bool(s[:, 0].isnan().all())
        if group:
            assert bool(s[:, 1].isinf().all()) and bool((s[:, 2:] > 0).all()) and bool((q.float()[:, 128:] == 448).all())


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(64, 1024, device="cuda").normal_(generator=gen).bfloat16()
    w = torch.empty(1024, device="cuda").normal_(1.0, 0.2, generator=gen).bfloat16()
    want, o = torch.empty_like(x), torch.empty_like(x)
    binding.rms_norm(x, w, EPS, out=want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.rms_norm(x, w, EPS, out=o, stream=side)
    side.synchronize()
    assert torch.equal(o, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.rms_norm(x, w, EPS, out=o)
        binding.rms_norm(o, w, EPS, out=o)
    o.zero_()
    g.replay()
    torch.cuda.synchronize()
    again = torch.empty_like(x)
    binding.rms_norm(want, w, EPS, out=again)
    torch.cuda.synchronize()
    assert torch.equal(o, again)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [5, 900])
@pytest.mark.parametrize("stride", [1000, 1003, 1005])
def test_the_weight_is_the_first_row(stride, T, dtype):
    """x and the weight begin at the same address; rows lie wherever the stride puts them."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(stride)
    mem = torch.empty(T, stride, device="cuda").normal_(generator=gen).to(torch.float32 if dtype == "fp32" else torch.bfloat16)
    x, w = mem[:, :1000], mem[0, :1000]
    o = torch.empty(T, 1000, dtype=mem.dtype, device="cuda")
    binding.rms_norm(x, w, EPS, out=o)
    _, y, _ = _reference(x.double().cpu(), None, w.double().cpu(), EPS, None)
    assert bool(((o.double().cpu() - y).abs() <= y.abs() * (40 * 2.0 ** -24 + HALF[dtype] * (dtype == "bf16")) * 1.01).all())


# ------------------------------------------------------------------ rows beside rows, and the ends of fp32's range
@pytest.mark.gpu
@pytest.mark.parametrize("group", [None, 0, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d", [(1500, 512), (700, 1000), (40, 2048)])
def test_a_row_hangs_on_itself(T, d, dtype, group):
    """NaN, infinities and huge values in some rows change no bit of the others, tiny ones among them."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(d)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    x = torch.empty(T, d, device="cuda").normal_(generator=gen)
    x[1::7] *= 1e-24
    x[2::7] *= 1e-35
    x = x.to(dt)
    w = torch.empty(d, device="cuda").normal_(1.0, 0.3, generator=gen).to(dt)

    def run(x):
        o = torch.empty_like(x)
        q = s = None
        if group is not None:
            q = torch.empty(T, d, dtype=torch.float8_e4m3fn, device="cuda")
            s = torch.empty(T, -(-d // group) if group else 1, device="cuda")
        binding.rms_norm(x, w, EPS, out=o, out8=q, scales=s, group=group or 0)
        return [o] + ([] if q is None else [q.view(torch.uint8), s])
    alone = run(x)
    odd = x.clone()
    at = torch.arange(0, T, 5, device="cuda")
    odd[at[0::3], 3] = float("nan")
    odd[at[1::3], 5] = float("inf")
    odd[at[2::3]] = 3e30
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[at] = False
    for a, b in zip(alone, run(odd)):
        assert torch.equal(a[keep], b[keep])
    _, y, _ = _reference(x.double().cpu(), None, w.double().cpu(), EPS, None)
    # (fp32 arithmetic as in _check, rounded once; the type's smallest steps where y is below its normal numbers)
    tol = y.abs() * (40 * 2.0 ** -24 + HALF[dtype] * (dtype == "bf16")) * 1.01 + (2.0 ** -134 if dtype == "bf16" else 2.0 ** -149)
    assert bool(((alone[0].double().cpu() - y).abs() <= tol).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [500, 512])
@pytest.mark.parametrize("eps", [2.0 ** -87, 2.0 ** -100, 2.0 ** -126])
@pytest.mark.parametrize("size", [1e-17, 1e-28, 1e-33, 1e-36])
def test_tiny_rows_beside_a_tiny_eps(size, eps, d, dtype):
    """eps far above and far below the squares of rows that are themselves out of the squares' range."""
    import torch
    x = torch.linspace(-1.0, 1.0, d, device="cuda").repeat(4, 1) * size
    for group in (None, 0, 128):
        _check(4, d, dtype, residual=None, x_values=x, eps=eps, group=group)


@pytest.mark.gpu
@pytest.mark.parametrize("size,weight", [(1e-14, 1e-26), (1e-12, 1e-27), (1e15, 1e20), (1e-10, 1e-28)])
def test_products_with_the_weight_outside_fp32(size, weight):
    """Rows with one 8-bit scale: h * weight leaves fp32's normal range, y does not."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty(50, 512, device="cuda").normal_(0.0, size, generator=gen)
    w = torch.empty(512, device="cuda").normal_(1.0, 0.1, generator=gen) * weight
    o, s = torch.empty_like(x), torch.empty(50, 1, device="cuda")
    q = torch.empty(50, 512, dtype=torch.float8_e4m3fn, device="cuda")
    binding.rms_norm(x, w, 0.0, out=o, out8=q, scales=s)
    _, y, sc = _reference(x.double().cpu(), None, w.double().cpu(), 0.0, 0)
    f32 = 40 * 2.0 ** -24
    assert bool(((o.double().cpu() - y).abs() <= y.abs() * f32).all())
    assert bool(((s.double().cpu() - sc).abs() <= sc * 2 * f32).all())
    ideal = y / sc
    assert bool(((q.float().double().cpu() - ideal).abs() <= torch.clamp(ideal.abs() * 2.0 ** -4, min=2.0 ** -10) * (1 + 1e-3)).all())
