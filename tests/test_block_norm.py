"""The norms behind and in front of a block with its gate and residual scale, against the formula in 64 bits."""
import ctypes

import pytest

from paper_2308_15030_b200 import binding

EPS = 1e-6
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}          # largest relative error of one rounding


# ------------------------------------------------------------------ refusals (host checks, no GPU needed)
def _args(**kw):
    base = dict(x=256, residual=256, weight=256, out=256, x_stride=64, residual_stride=64, out_stride=64, n_rows=2, d=64, dtype=1, residual_dtype=1,
                type8=0, group=0, eps=EPS, post_eps=EPS, scale=1.0)
    base.update(kw)
    return binding.BlockNormArgs(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(n_rows=-1), -1), (dict(d=0), -1), (dict(dtype=2), -1), (dict(residual_dtype=3), -1), (dict(dtype=0), -1), (dict(type8=2), -1),
    (dict(group=16), -1), (dict(group=96), -1), (dict(group=-1), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
    (dict(post_eps=float("inf")), -1), (dict(post_eps=-1e-6), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(x=None), -1),
    (dict(weight=None), -1), (dict(out=None), -1), (dict(out8=256, out8_stride=64), -1), (dict(scales=256, scales_stride=1), -1),
    (dict(x=257), -1), (dict(out=255), -1), (dict(gate=257), -1), (dict(post_weight=257), -1), (dict(x_stride=63), -1), (dict(gate=256, gate_stride=63), -1),
    (dict(residual_stride=63), -1), (dict(residual_out=256, residual_out_stride=63), -1),
    (dict(out8=256, out8_stride=64, scales=256, scales_stride=1, group=32), -1), (dict(d=16385, x_stride=20000, residual_stride=20000, out_stride=20000), -7)])
def test_refusals(kw, status):
    assert binding.lib().swapmoe_block_norm(ctypes.byref(_args(**kw)), None) == status


def test_no_arguments_and_no_rows():
    assert binding.lib().swapmoe_block_norm(None, None) == -1
    assert binding.lib().swapmoe_block_norm(ctypes.byref(_args(n_rows=0, x=None)), None) == 0


def test_tensor_checks():
    import torch
    x, w = torch.zeros(2, 64), torch.ones(64)
    good = dict(x=x, residual=torch.zeros(2, 64), weight=w, eps=EPS, out=torch.zeros(2, 64))
    for kw in (dict(x=torch.zeros(64)), dict(residual=torch.zeros(2, 63)), dict(residual=torch.zeros(1, 64)), dict(weight=torch.ones(63)),
               dict(weight=w.bfloat16()), dict(post_weight=torch.ones(65)), dict(gate=torch.ones(63)), dict(gate=torch.ones(1, 64)),
               dict(gate=torch.ones(2, 64).bfloat16()), dict(gate=torch.ones(2, 2, 64)), dict(out=torch.zeros(2, 64).half()),
               dict(residual_out=torch.zeros(2, 64).bfloat16()), dict(out8=torch.zeros(2, 64, dtype=torch.int8)), dict(scales=torch.zeros(2)),
               dict(out8=torch.zeros(2, 64, dtype=torch.uint8), scales=torch.zeros(2)), dict(x=x.half()), dict()):   # the last: not on a GPU
        with pytest.raises(binding.SwapMoEError) as e:
            binding.block_norm(**{**good, **kw})
        assert e.value.status == -1


# ------------------------------------------------------------------ on the GPU
def _norm(v, w, eps):
    import torch
    return v * w / torch.sqrt((v * v).mean(1, keepdim=True) + eps)


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


def _check(T, d, dtype="bf16", residual="same", post=True, gate="none", scale=1.0, out=True, type8=None, group=0, stride=None, offset=0, eps=EPS,
           change=None, in_place=False):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T * 10007 + d)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    rdt = torch.float32 if residual == "fp32" else dt
    stride = stride or d
    x, _ = _rows(T, d, dt, gen, stride, offset)
    r = _rows(T, d, rdt, gen, stride, offset, std=2.0)[0] if residual else None
    if change is not None:
        change(x, r)
    w = torch.empty(d, device="cuda").normal_(1.0, 0.3, generator=gen).to(dt)
    pw = torch.empty(d, device="cuda").normal_(1.0, 0.3, generator=gen).to(dt) if post else None
    g = None
    if gate == "channels":
        g = torch.empty(d, device="cuda").normal_(0.0, 1.0, generator=gen).to(dt)
    elif gate == "rows":
        g, _ = _rows(T, d, dt, gen, stride, offset)
    x64, r64 = x.double().cpu(), 0.0 if r is None else r.double().cpu()
    if in_place:
        ro, ro_mem = r, None
    else:
        ro, ro_mem = _rows(T, d, rdt, gen, stride, offset)
    o, o_mem = _rows(T, d, dt, gen, stride, offset) if out else (None, None)
    n = -(-d // group) if group else 1
    q = s = None
    if type8:
        q = torch.full((T + 1, d), 7, device="cuda").to(torch.int8 if type8 == "int8" else torch.float8_e4m3fn)
        s = torch.full((T + 1, n), 7.0, device="cuda")
    binding.block_norm(x, r, w, eps, out=o, residual_out=ro, post_weight=pw, gate=g, scale=scale, out8=q, scales=s, group=group)
    torch.cuda.synchronize()
    p = x64 if pw is None else _norm(x64, pw.double().cpu(), eps)
    if g is not None:
        p = p * g.double().cpu()
    p = p * scale
    h = r64 + p
    y = _norm(h, w.double().cpu(), eps)
    # a norm: a sum of d squares in trees of at most 8 + 5 + 32 terms each, one square root, and four products: well under 40
    # roundings of 2^-24.  The sum of residual and p adds p's error and one rounding; the second norm carries an error of h to y by y / h, and
    # by its root mean square to the whole row.
    f32 = 40 * 2.0 ** -24
    off_h = f32 * p.abs() + 2.0 ** -24 * h.abs()
    root = torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    off_y = off_h * w.double().cpu().abs() / root + y.abs() * (f32 + torch.sqrt((off_h * off_h).mean(1, keepdim=True)) / root)
    half_r = HALF["fp32" if rdt == torch.float32 else "bf16"]
    assert bool(((ro.double().cpu() - h).abs() <= half_r * h.abs() * 1.001 + off_h + 1e-40).all())
    if ro_mem is not None:
        assert _untouched(ro_mem, T, d, stride, offset)
    if out:
        assert bool(((o.double().cpu() - y).abs() <= HALF[dtype] * y.abs() * 1.001 + off_y + 1e-40).all())
        assert _untouched(o_mem, T, d, stride, offset)
    if type8:
        top = 127.0 if type8 == "int8" else 448.0
        width = group or d
        pad = torch.nn.functional.pad
        big = pad(y.abs(), (0, n * width - d)).view(T, n, width).amax(2)
        off_big = pad(off_y, (0, n * width - d)).view(T, n, width).amax(2)
        got_s = s[:T].double().cpu()
        assert bool(((got_s - big / top).abs() <= (off_big + 4 * 2.0 ** -24 * big) / top + 1e-40).all())
        cols = torch.arange(d) // width
        unit = got_s[:, cols]
        t = torch.where(unit > 0, y / torch.where(unit > 0, unit, 1.0), 0.0)
        off_t = torch.where(unit > 0, off_y / torch.where(unit > 0, unit, 1.0), 0.0) + 4 * 2.0 ** -24 * t.abs()
        # integers: half a step; e4m3: 2^-4 of the value, or half a step of 2^-9 below its normal range
        step = 0.5 if type8 == "int8" else torch.clamp(t.abs() * 2.0 ** -4, min=2.0 ** -10)
        assert bool(((q[:T].float().double().cpu() - t).abs() <= step + 1.07 * off_t + 1e-9).all())
        assert bool((q[T].float() == 7.0).all()) and bool((s[T] == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("d", [1, 3, 8, 31, 64, 200, 255, 256, 257, 1000, 1003, 2048, 4096, 4097, 8192, 8200, 16384])
@pytest.mark.parametrize("T,dtype", [(1, "bf16"), (3, "fp32"), (300, "bf16"), (2000, "fp32")])
def test_widths(T, d, dtype):
    if T * d > 1 << 23:
        T = 300
    _check(T, d, dtype, gate="channels", type8="int8")


@pytest.mark.gpu
@pytest.mark.parametrize("residual", ["same", "fp32", None])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate", ["none", "channels", "rows"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_forms(residual, post, gate, dtype):
    _check(70, 520, dtype, residual, post, gate, scale=0.37)
    _check(2, 1003, dtype, residual, post, gate, scale=-2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("type8", ["int8", "e4m3"])
@pytest.mark.parametrize("group", [0, 32, 64, 128, 256])
@pytest.mark.parametrize("T,d,dtype", [(5, 1024, "bf16"), (700, 768, "bf16"), (40, 1003, "fp32"), (3, 300, "bf16"), (600, 4096, "fp32")])
def test_8_bit_rows(type8, group, T, d, dtype):
    _check(T, d, dtype, gate="rows", type8=type8, group=group)
    _check(T, d, dtype, "fp32", out=False, type8=type8, group=group)


@pytest.mark.gpu
@pytest.mark.parametrize("stride,offset", [(72, 0), (64, 8), (65, 0), (64, 1), (71, 3)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides_and_starts(stride, offset, dtype):
    _check(37, 64, dtype, gate="rows", stride=stride, offset=offset, type8="int8")
    _check(37, 64, dtype, residual="fp32", stride=stride, offset=offset, type8="e4m3", group=32)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 900])
def test_the_residual_in_place(T):
    _check(T, 1024, "bf16", gate="channels", in_place=True)
    _check(T, 1024, "bf16", residual="fp32", in_place=True, type8="int8")


@pytest.mark.gpu
@pytest.mark.parametrize("type8", [None, "int8", "e4m3"])
def test_magnitudes_at_the_ends(type8):
    def loud(x, r):
        x[::3] *= 1e25
        r[1::3] *= 1e28
    def quiet(x, r):
        x *= 1e-25
        r.zero_()
    def zeros(x, r):
        x[::2] = 0.0
        r[::2] = 0.0
    for d, T in ((264, 7), (1024, 30), (1003, 5)):
        _check(T, d, "fp32", change=loud, type8=type8)
        _check(T, d, "bf16", change=loud, type8=type8, post=False)
        _check(T, d, "fp32", change=quiet, eps=0.0, type8=type8)
        _check(T, d, "fp32", change=quiet, eps=1e-30, type8=type8, post=False)
        _check(T, d, "fp32", change=zeros, type8=type8)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [256, 1003])
def test_rows_leave_their_neighbours_alone(d):
    """Infinities, NaN and values out of the squares' range change no bit of another row, and do to their own what the formula does."""
    import torch
    T = 12
    gen = torch.Generator(device="cuda").manual_seed(d)
    x, r = torch.randn(T, d, device="cuda", generator=gen), torch.randn(T, d, device="cuda", generator=gen)
    w = torch.rand(d, device="cuda", generator=gen) + 0.5

    def run(x, r):
        out, ro, q, s = torch.empty_like(x), torch.empty_like(r), torch.empty(T, d, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
        binding.block_norm(x, r, w, EPS, out=out, residual_out=ro, post_weight=w, gate=w, out8=q, scales=s)
        return out, ro, q, s
    first = run(x, r)
    x[2, 5], x[4, 7], r[6, 1], r[8, 3], x[10] = float("inf"), float("nan"), float("inf"), float("-inf"), 1e30
    again = run(x, r)
    calm = [0, 1, 3, 5, 7, 9, 11]
    assert all(torch.equal(a[calm], b[calm]) for a, b in zip(first, again))
    out, ro, q, s = again
    assert bool(torch.isnan(out[2, 5])) and bool((ro[2, 6:] == r[2, 6:]).all())      # an infinite block's finite columns are 0
    assert bool(torch.isnan(out[4]).all()) and bool(torch.isnan(s[4]))
    assert bool(torch.isnan(out[6, 1])) and bool((out[6, 2:] == 0).all()) and bool(torch.isnan(s[6]))
    assert bool(torch.isinf(ro[8, 3])) and bool(torch.isfinite(out[10]).all())


@pytest.mark.gpu
def test_behind_the_last_block():
    """Without a weight only the stream is written."""
    import torch
    x, r, w = torch.randn(50, 640, device="cuda"), torch.randn(50, 640, device="cuda"), torch.rand(640, device="cuda")
    ro, both, out = torch.empty_like(r), torch.empty_like(r), torch.empty_like(x)
    binding.block_norm(x, r, None, EPS, residual_out=ro, post_weight=w)
    binding.block_norm(x, r, w, EPS, residual_out=both, post_weight=w, out=out)
    assert torch.equal(ro, both)


@pytest.mark.gpu
def test_matches_rms_norm_where_it_is_that():
    import torch
    x, r, w = torch.randn(333, 1024, device="cuda").bfloat16(), torch.randn(333, 1024, device="cuda").bfloat16(), torch.rand(1024, device="cuda").bfloat16()
    a, b, ra, rb = (torch.empty_like(x) for _ in range(4))
    binding.rms_norm(x, w, EPS, out=a, residual=r, residual_out=ra)
    binding.block_norm(x, r, w, EPS, out=b, residual_out=rb)
    assert torch.equal(ra, rb)
    assert bool(((a.float() - b.float()).abs() <= 2 * 2.0 ** -8 * a.float().abs()).all())     # a step where the two lie next to a border


@pytest.mark.gpu
def test_streams_and_graphs():
    import torch
    x, r, w = torch.randn(100, 512, device="cuda"), torch.randn(100, 512, device="cuda"), torch.rand(512, device="cuda")
    want = torch.empty_like(x)
    binding.block_norm(x, r, w, EPS, out=want, post_weight=w)
    out, side = torch.zeros_like(x), torch.cuda.Stream()
    torch.cuda.synchronize()
    binding.block_norm(x, r, w, EPS, out=out, post_weight=w, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.block_norm(x, r, w, EPS, out=out, post_weight=w)
    x.mul_(3.0).add_(0.25)
    graph.replay()
    binding.block_norm(x, r, w, EPS, out=want, post_weight=w)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


# ------------------------------------------------------------------ a layer's own block
def test_post_norm_refusals():
    L = binding.lib()
    assert L.swapmoe_set_post_norm(None, 256, 1e-6, None, 1.0) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 7, 130])
def test_a_layers_block_with_sandwich_norms(T, dtype):
    """forward_block adds the normed, gated and scaled x: the same bits as block_norm and the layer's own forward, one after the other."""
    import numpy as np
    import torch
    from harness import Case
    from paper_2308_15030_b200 import inputs as I
    cfg = I.LayerConfig("post", I.BF16 if dtype == "bf16" else I.F32, T=T, d=128, f=256, E=8, k=2, K=4, seed=3)
    case = Case(cfg)
    L, dt = case.layer, torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(T)
    normal = lambda *s: torch.empty(*s, device="cuda").normal_(0.0, 1.0, generator=gen).to(dt)  # noqa: E731
    x, r, w, pw, g = normal(T, 128), normal(T, 128), normal(128), normal(128), normal(128)
    L.set_norm(w, EPS)
    plain, plain_r = torch.empty_like(x), r.clone()
    L.forward_block(x, plain_r, plain)
    for kw in (dict(weight=pw, eps=EPS, gate=g, scale=0.3), dict(weight=pw, eps=1e-3), dict(gate=g), dict(scale=-1.5)):
        L.set_post_norm(**kw)
        out, ro = torch.empty_like(x), r.clone()
        n0 = L.launch_count
        L.forward_block(x, ro, out)
        launches = L.launch_count - n0
        n, want_r, want = torch.empty_like(x), torch.empty_like(r), torch.empty_like(x)
        binding.block_norm(x, r, w, EPS, out=n, residual_out=want_r, post_weight=kw.get("weight"), post_eps=kw.get("eps", EPS), gate=kw.get("gate"),
                           scale=kw.get("scale", 1.0))
        n0 = L.launch_count
        L.forward(n, want)
        assert launches == L.launch_count - n0 + 1
        torch.cuda.synchronize()
        assert torch.equal(ro, want_r) and torch.equal(out, want)
    L.set_post_norm()
    out, ro = torch.empty_like(x), r.clone()
    L.forward_block(x, ro, out)
    assert torch.equal(out, plain) and torch.equal(ro, plain_r)
    for bad in (dict(weight=pw[:64]), dict(gate=g.float() if dtype == "bf16" else g.bfloat16()), dict(weight=pw.cpu()), dict(scale=float("nan")),
                dict(weight=pw, eps=-1.0)):
        with pytest.raises(binding.SwapMoEError) as e:
            L.set_post_norm(**bad)
        assert e.value.status == -1
