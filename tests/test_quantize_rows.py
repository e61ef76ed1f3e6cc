"""Rows to 8-bit integers with a scale each: the scale and the integers that IEEE division gives."""
import ctypes

import pytest

from paper_2308_15030_b200 import binding


# ------------------------------------------------------------------ refusals (host checks, no GPU needed)
def _args(**kw):
    base = dict(x=256, out8=256, scales=256, x_stride=64, out8_stride=64, n_rows=2, d=64, dtype=1, act=0)
    base.update(kw)
    return binding.QuantizeRowsArgs(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(n_rows=-1), -1), (dict(d=0), -1), (dict(dtype=2), -1), (dict(act=3), -1), (dict(act=-1), -1), (dict(x=None), -1), (dict(out8=None), -1),
    (dict(scales=None), -1), (dict(x=257), -1), (dict(x=258, dtype=0), -1), (dict(scales=258), -1), (dict(x_stride=63), -1),
    (dict(act=2, x_stride=127), -1), (dict(out8_stride=63), -1), (dict(d=32769, x_stride=40000, out8_stride=40000), -7)])
def test_refusals(kw, status):
    assert binding.lib().swapmoe_quantize_rows(ctypes.byref(_args(**kw)), None) == status


def test_no_arguments_and_no_rows():
    assert binding.lib().swapmoe_quantize_rows(None, None) == -1
    assert binding.lib().swapmoe_quantize_rows(ctypes.byref(_args(n_rows=0, x=None)), None) == 0


def test_tensor_checks():
    import torch
    good = dict(x=torch.zeros(2, 64), out8=torch.zeros(2, 64, dtype=torch.int8), scales=torch.zeros(2))
    for kw in (dict(x=torch.zeros(64)), dict(x=torch.zeros(2, 64).half()), dict(out8=torch.zeros(2, 64, dtype=torch.uint8)),
               dict(out8=torch.zeros(2, 63, dtype=torch.int8)), dict(scales=torch.zeros(3)), dict(scales=torch.zeros(2).bfloat16()),
               dict(act="gelu"), dict(act="swiglu"), dict(x=torch.zeros(2, 63), act="swiglu"), dict()):   # the last: not on a GPU
        with pytest.raises(binding.SwapMoEError) as e:
            binding.quantize_rows(**{**good, **kw})
        assert e.value.status == -1


# ------------------------------------------------------------------ on the GPU
def _division(y):
    """(integers, scales) of fp32 rows on the CPU: quotients rounded to fp32, then to integers."""
    import torch
    most = y.abs().amax(1)
    scales = torch.where(most == 0, 0.0, (most.double() / 127.0).float().clamp(min=2.0 ** -120))
    return torch.round(y / torch.where(scales > 0, scales, 1.0)[:, None]), scales


def _input(T, d, dt, gen, stride, offset):
    import torch
    mem = torch.empty(T * stride + offset, device="cuda").normal_(0.0, 1.0, generator=gen).to(dt)
    return torch.as_strided(mem, (T, d), (stride, 1), offset)


def _check(T, d, dtype="bf16", stride=None, offset=0, out_stride=None, out_offset=0, change=None):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T * 10007 + d)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    x = _input(T, d, dt, gen, stride or d, offset)
    if change is not None:
        change(x)
    out_stride = out_stride or d
    mem = torch.full((T * out_stride + out_offset + 64,), 77, dtype=torch.int8, device="cuda")
    q = torch.as_strided(mem, (T, d), (out_stride, 1), out_offset)
    scales = torch.full((T + 1,), 7.0, device="cuda")
    binding.quantize_rows(x, q, scales[:T])
    torch.cuda.synchronize()
    want_q, want_s = _division(x.float().cpu())
    assert torch.equal(scales[:T].cpu(), want_s)
    assert torch.equal(q.cpu().float(), want_q)
    keep = torch.ones_like(mem, dtype=torch.bool)
    torch.as_strided(keep, (T, d), (out_stride, 1), out_offset).fill_(False)
    assert bool((mem[keep] == 77).all()) and float(scales[T]) == 7.0


@pytest.mark.gpu
@pytest.mark.parametrize("d", [1, 3, 8, 31, 64, 255, 256, 257, 1000, 1003, 2048, 4096, 8191, 8192, 8200, 14336, 16384, 16392, 20000, 32768])
@pytest.mark.parametrize("T,dtype", [(1, "bf16"), (5, "fp32"), (700, "bf16")])
def test_widths(T, d, dtype):
    _check(T, d, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("stride,offset,out_stride,out_offset", [(72, 0, 64, 0), (64, 8, 80, 8), (65, 0, 65, 3), (64, 1, 64, 1), (71, 3, 67, 5)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides_and_starts(stride, offset, out_stride, out_offset, dtype):
    _check(37, 64, dtype, stride, offset, out_stride, out_offset)


@pytest.mark.gpu
def test_many_rows_and_ties():
    _check(5000, 768)
    _check(3000, 1024, "fp32")

    def halves(x):                       # the largest is 127: values half-way between integers go to the even one
        import torch
        x.copy_(torch.arange(x.numel(), device="cuda").view(x.shape) % 255 / 2.0)
        x[:, 0] = -127.0
    _check(9, 300, "fp32", change=halves)
    _check(9, 304, "bf16", change=halves)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_ends_of_the_range(dtype):
    def put(x):
        x[0] = 0.0
        x[1] *= 1e-38
        x[2] *= 2.0 ** -126
        x[3] = 1e-40
        x[4] *= 1e37
        x[5, 1:] = 0.0
        x[6, :] = -1.0
    _check(8, 264, dtype, change=put)


@pytest.mark.gpu
def test_infinities_and_nan():
    import torch
    x = torch.randn(4, 300, device="cuda")
    q, s = torch.empty(4, 300, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    binding.quantize_rows(x, q, s)
    q0, s0 = q.clone(), s.clone()
    x[1, 7], x[2, 9] = float("inf"), float("nan")
    binding.quantize_rows(x, q, s)
    assert bool(torch.isinf(s[1])) and bool(torch.isnan(s[2])) and bool((q[1:3] == 0).all())
    assert torch.equal(q[[0, 3]], q0[[0, 3]]) and torch.equal(s[[0, 3]], s0[[0, 3]])


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["relu", "swiglu"])
@pytest.mark.parametrize("T,d,dtype", [(1, 64, "bf16"), (40, 1003, "bf16"), (300, 1024, "fp32"), (33, 14336, "bf16"), (5, 17000, "fp32")])
def test_activations(act, T, d, dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.empty(T, d * (2 if act == "swiglu" else 1), device="cuda").normal_(0.0, 2.0, generator=gen)
    x = x if dtype == "fp32" else x.bfloat16()
    q, s = torch.empty(T, d, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    binding.quantize_rows(x, q, s, act=act)
    v = x.double().cpu()
    y = v.clamp(min=0.0) if act == "relu" else v[:, :d] / (1.0 + torch.exp(-v[:, :d])) * v[:, d:]
    # relu is exact; silu: |x| < 14, the exponential within 2 + 1.2 x 14 steps of 2^-23, the quotient and the product one rounding each
    off = 0.0 if act == "relu" else 20 * 2.0 ** -23
    want = y.abs().amax(1) / 127.0
    assert bool(((s.double().cpu() - want).abs() <= (off + 2.0 ** -24) * want).all())
    t = y / s.double().cpu()[:, None]
    assert bool(((q.double().cpu() - t).abs() <= 0.5 + (off + 2.0 ** -23) * t.abs() + 1e-9).all())


@pytest.mark.gpu
def test_streams_and_graphs():
    import torch
    x = torch.randn(200, 512, device="cuda").bfloat16()
    q, s = torch.zeros(200, 512, dtype=torch.int8, device="cuda"), torch.zeros(200, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    binding.quantize_rows(x, q, s, stream=side)
    torch.cuda.synchronize()
    want_q, want_s = _division(x.float().cpu())
    assert torch.equal(q.cpu().float(), want_q) and torch.equal(s.cpu(), want_s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.quantize_rows(x, q, s)
    x.normal_()
    graph.replay()
    torch.cuda.synchronize()
    want_q, want_s = _division(x.float().cpu())
    assert torch.equal(q.cpu().float(), want_q) and torch.equal(s.cpu(), want_s)
