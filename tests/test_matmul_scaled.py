"""Products of 8-bit integers with scales for tokens and channels, against exact sums."""
import ctypes

import pytest

from paper_2308_15030_b200 import binding

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}          # largest relative error of one rounding


# ------------------------------------------------------------------ refusals (host checks, no GPU needed)
def _args(**kw):
    base = dict(x=256, w=256, x_scales=256, w_scales=256, out=256, x_stride=64, w_stride=64, out_stride=32, n_tokens=2, k=64, n=32, dtype=1)
    base.update(kw)
    return binding.MatmulArgs(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(n_tokens=-1), -1), (dict(k=0), -1), (dict(n=0), -1), (dict(dtype=2), -1), (dict(x=None), -1), (dict(w=None), -1),
    (dict(x_scales=None), -1), (dict(w_scales=None), -1), (dict(out=None), -1), (dict(x=264), -1), (dict(w=257), -1), (dict(out=257), -1),
    (dict(out=258, dtype=0), -1), (dict(x_scales=258), -1), (dict(w_scales=258), -1), (dict(bias=258), -1), (dict(x_stride=63), -1),
    (dict(x_stride=72), -1), (dict(w_stride=72), -1), (dict(w_stride=48), -1), (dict(out_stride=31), -1),
    (dict(k=131072, x_stride=131072, w_stride=131072), -7)])
def test_refusals(kw, status):
    assert binding.lib().swapmoe_matmul_scaled(ctypes.byref(_args(**kw)), None) == status


def test_no_arguments_and_no_tokens():
    assert binding.lib().swapmoe_matmul_scaled(None, None) == -1
    assert binding.lib().swapmoe_matmul_scaled(ctypes.byref(_args(n_tokens=0, x=None)), None) == 0


@pytest.mark.parametrize("kw", [dict(n=2 ** 31 - 1, out_stride=2 ** 31), dict(n_tokens=2 ** 31 - 256), dict(n=2 ** 31 - 256, out_stride=2 ** 31)])
def test_sizes_beyond_int32_are_refused(kw):
    assert binding.lib().swapmoe_matmul_scaled(ctypes.byref(_args(**kw)), None) == -7


def test_tensor_checks():
    import torch
    i8 = dict(dtype=torch.int8)
    good = dict(x8=torch.zeros(2, 64, **i8), x_scales=torch.zeros(2), w8=torch.zeros(32, 64, **i8), w_scales=torch.zeros(32), out=torch.zeros(2, 32))
    for kw in (dict(x8=torch.zeros(2, 64)), dict(x8=torch.zeros(2, 64, dtype=torch.uint8)), dict(x8=torch.zeros(64, **i8)),
               dict(x8=torch.zeros(64, 2, **i8).t()), dict(x_scales=torch.zeros(3)), dict(x_scales=torch.zeros(2).half()),
               dict(w8=torch.zeros(32, 48, **i8)), dict(w8=torch.zeros(64, 32, **i8).t()), dict(w_scales=torch.zeros(64)[::2]),
               dict(bias=torch.zeros(31)), dict(out=torch.zeros(2, 31)), dict(out=torch.zeros(1, 32)), dict(out=torch.zeros(2, 32).half()),
               dict()):                                                                                    # the last: not on a GPU
        with pytest.raises(binding.SwapMoEError) as e:
            binding.matmul_scaled(**{**good, **kw})
        assert e.value.status == -1


# ------------------------------------------------------------------ on the GPU
def _operand(n, k, gen, stride=None, low=-128):
    import torch
    stride = stride or k + -k % 16
    mem = torch.randint(-128, 128, (n, stride), device="cuda", generator=gen, dtype=torch.int32).to(torch.int8)
    v = mem[:, :k]
    if low == "ends":
        v.copy_(torch.where(torch.rand(n, k, device="cuda", generator=gen) < 0.5, -128, 127).to(torch.int8))
    return v


def _check(T, K, N, dtype="bf16", bias=False, out_pad=0, x_pad=0, values=-128, stream=None, scales=None):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T * 1000003 + K * 1009 + N)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    x = _operand(T, K, gen, K + x_pad + -(K + x_pad) % 16, values)
    w = _operand(N, K, gen, None, values)
    xs = torch.empty(T, device="cuda").uniform_(0.001, 0.1, generator=gen)
    ws = torch.empty(N, device="cuda").uniform_(0.001, 0.1, generator=gen)
    if scales is not None:
        xs *= scales
    b = torch.empty(N, device="cuda").normal_(0.0, 3.0, generator=gen) if bias else None
    mem = torch.full((T + 2, N + out_pad), 7.0, device="cuda").to(dt)
    out = mem[1:T + 1, :N]
    binding.matmul_scaled(x, xs, w, ws, out, bias=b, stream=stream)
    torch.cuda.synchronize()
    acc = x.double().cpu() @ w.double().cpu().t()                       # whole numbers below 2^53
    y = acc * xs.double().cpu()[:, None] * ws.double().cpu()
    # the sum to fp32, two products, the bias: four roundings; then the result's own
    tol = 3 * 2.0 ** -24 * y.abs()
    if bias:
        y = y + b.double().cpu()
        tol = tol + 2.0 ** -24 * y.abs()
    tol = tol * 1.001 + HALF[dtype] * y.abs() + 1e-37
    assert bool(((out.double().cpu() - y).abs() <= tol).all())
    keep = torch.ones_like(mem, dtype=torch.bool)
    keep[1:T + 1, :N] = False
    assert bool((mem[keep] == 7.0).all())                               # nothing around the result is written
    assert binding.matmul_status() == (0, 0)
    return x, xs, w, ws, out


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 3, 8, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 96, 100, 127, 128, 129, 160, 200, 255, 256, 257, 300, 511, 777, 1024, 1500])
def test_token_counts(T):
    _check(T, 320, 384)


@pytest.mark.gpu
@pytest.mark.parametrize("T,K,N", [(T, K, N) for T in (1, 20, 100, 300) for K, N in (
    (1, 1), (1, 300), (16, 8), (17, 33), (100, 7), (127, 129), (128, 128), (129, 127), (130, 255), (256, 256), (257, 257), (1003, 600),
    (2048, 31), (4096, 64), (4111, 513), (64, 4096))])
def test_ragged_widths(T, K, N):
    _check(T, K, N, "fp32" if (K + N) % 2 else "bf16", bias=K % 3 == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 5, 40, 130, 600])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("out_pad", [0, 1, 3, 8])
def test_rows_inside_wider_ones(T, dtype, out_pad):
    _check(T, 200, 120, dtype, bias=True, out_pad=out_pad, x_pad=40)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 33, 300])
@pytest.mark.parametrize("K", [4096, 131071])
def test_largest_sums(T, K):
    _check(T, K, 130, "fp32", values="ends")


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 70, 400])
def test_all_lowest_values(T):
    """The largest sum there is: 2^14 (2^17 - 1)."""
    import torch
    K, N = 131071, 64
    x = torch.full((T, K + 1), -128, dtype=torch.int8, device="cuda")[:, :K]
    w = torch.full((N, K + 1), -128, dtype=torch.int8, device="cuda")[:, :K]
    out = torch.empty(T, N, device="cuda")
    one = torch.ones(max(T, N), device="cuda")
    binding.matmul_scaled(x, one[:T].contiguous(), w, one[:N].contiguous(), out)
    assert bool((out == float(16384 * K)).all())                        # 2^14 (2^17 - 1) has 17 bits: exact in fp32


@pytest.mark.gpu
def test_several_rounds_of_tiles():
    _check(3000, 384, 2300)
    _check(2100, 1100, 5200, "fp32")
    _check(7001, 4096, 900)                                             # groups of token tiles


@pytest.mark.gpu
@pytest.mark.parametrize("T,K,N", [(9, 4096, 1000), (37, 1024, 1000), (90, 8192, 100), (130, 2048, 500), (129, 64, 4), (257, 4111, 513), (333, 600, 33),
                                   (512, 1024, 257), (640, 14336, 257), (1000, 512, 100), (2000, 4096, 40), (4600, 256, 128)])
@pytest.mark.parametrize("dtype,out_pad", [("bf16", 0), ("fp32", 3)])
def test_narrow_matrices_in_several_groups_of_tokens(T, K, N, dtype, out_pad):
    _check(T, K, N, dtype, bias=True, out_pad=out_pad, x_pad=(16 - K) % 16 + 16)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [129, 200, 600, 1100])
@pytest.mark.parametrize("K,N", [(16, 5008), (129, 4999), (1003, 6033), (2048, 4800)])
@pytest.mark.parametrize("dtype,out_pad", [("bf16", 0), ("bf16", 1), ("bf16", 8), ("fp32", 0), ("fp32", 1)])
def test_wide_matrices(T, K, N, dtype, out_pad):
    _check(T, K, N, dtype, bias=K % 2 == 1, out_pad=out_pad)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 31, 33, 61, 64, 65, 96, 97, 128])
@pytest.mark.parametrize("K,N,dtype,out_pad", [(1000, 9600, "bf16", 0), (650, 9601, "fp32", 2), (2100, 19200, "fp32", 0)])
def test_few_tokens_of_wide_matrices(T, K, N, dtype, out_pad):
    _check(T, K, N, dtype, bias=N % 2 == 0, out_pad=out_pad)


@pytest.mark.gpu
@pytest.mark.parametrize("T,K,N", [(6500, 4096, 640), (13000, 2064, 300)])
def test_rows_beyond_a_scheduling_group(T, K, N):
    _check(T, K, N, "bf16", bias=True)


@pytest.mark.gpu
@pytest.mark.parametrize("T,K,N", [(130, 200, 5002), (333, 1024, 5028), (700, 640, 4838)])
@pytest.mark.parametrize("out_pad", [0, 1, 2, 4, 10])
def test_rows_of_an_even_width(T, K, N, out_pad):
    _check(T, K, N, "bf16", bias=True, out_pad=out_pad)


@pytest.mark.gpu
@pytest.mark.parametrize("T,N", [(300, 4864), (900, 2560)])
def test_all_lowest_values_of_wide_matrices(T, N):
    import torch
    K = 131071
    x = torch.full((T, K + 1), -128, dtype=torch.int8, device="cuda")[:, :K]
    w = torch.full((N, K + 1), -128, dtype=torch.int8, device="cuda")[:, :K]
    out = torch.empty(T, N, device="cuda")
    one = torch.ones(max(T, N), device="cuda")
    binding.matmul_scaled(x, one[:T].contiguous(), w, one[:N].contiguous(), out)
    assert bool((out == float(torch.tensor(2 ** 14 * K, dtype=torch.float32))).all())
    assert binding.matmul_status() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40, 300])
def test_scales_that_are_not_finite_or_zero(T):
    import torch
    x, xs, w, ws, _ = _check(T, 160, 96)
    out, first = torch.empty(T, 96, device="cuda"), torch.empty(T, 96, device="cuda")
    binding.matmul_scaled(x, xs, w, ws, first)
    for bad in (float("nan"), float("inf"), 0.0):
        xs2, ws2 = xs.clone(), ws.clone()
        xs2[T // 2], ws2[17] = bad, bad
        binding.matmul_scaled(x, xs2, w, ws2, out)
        want = (x.double() @ w.double().t()) * xs2.double()[:, None] * ws2.double()
        assert bool((torch.isnan(out) == torch.isnan(want)).all())
        fine = torch.ones_like(out, dtype=torch.bool)
        fine[T // 2], fine[:, 17] = False, False
        assert torch.equal(out[fine], first[fine])                      # the others keep their bits
        infinite = torch.isinf(want)
        assert torch.equal(out[infinite].double(), want[infinite])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 60, 300])
def test_streams_graphs_and_two_calls_at_once(T):
    import torch
    K, N = 1024, 640
    gen = torch.Generator(device="cuda").manual_seed(T)
    sets = []
    for _ in range(2):
        x, w = _operand(T, K, gen), _operand(N, K, gen)
        sets.append((x, torch.rand(T, device="cuda", generator=gen), w, torch.rand(N, device="cuda", generator=gen)))
    want = []
    for s in sets:
        out = torch.empty(T, N, device="cuda")
        binding.matmul_scaled(*s, out)
        want.append(out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [torch.zeros(T, N, device="cuda") for _ in sets]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, st, o in zip(sets, streams, outs):
            binding.matmul_scaled(*s, o, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph, out = torch.cuda.CUDAGraph(), torch.zeros(T, N, device="cuda")
    x, xs, w, ws = (t.clone() for t in sets[0])
    with torch.cuda.graph(graph):
        binding.matmul_scaled(x, xs, w, ws, out)
    for s, expected in zip(sets, want):
        for a, b in zip((x, xs, w, ws), s):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, expected)


@pytest.mark.gpu
def test_no_tokens():
    import torch
    out = torch.empty(0, 32, device="cuda")
    binding.matmul_scaled(torch.empty(0, 64, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"),
                          torch.zeros(32, 64, dtype=torch.int8, device="cuda"), torch.ones(32, device="cuda"), out)


@pytest.mark.gpu
@pytest.mark.parametrize("pad", [0, 1])
def test_offsets_beyond_32_bits(pad):
    """A result of more than 2^31 values, stored by boxes and one by one."""
    import torch
    T, K, N = 40000, 48, 60000
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w = _operand(T, K, gen), _operand(N, K, gen)
    one_t, one_n = torch.ones(T, device="cuda"), torch.ones(N, device="cuda")
    out = torch.empty(T, N + pad, dtype=torch.bfloat16, device="cuda")[:, :N]
    binding.matmul_scaled(x, one_t, w, one_n, out)
    for rows in (slice(0, 50), slice(35780, 35830), slice(T - 50, T)):
        want = (x[rows].float() @ w.float().t()).bfloat16()             # sums below 2^24: exact, one rounding each
        assert torch.equal(out[rows], want)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 20, 100, 400])
def test_right_behind_what_writes_its_operands(T):
    """Rows and weights come from the kernels directly in front, which a dependent launch may overlap."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T)
    K, N = 640, 384
    x8, xs, w8, ws = (torch.empty(T, K, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"), torch.empty(N, K, dtype=torch.int8, device="cuda"),
                      torch.empty(N, device="cuda"))
    out = torch.empty(T, N, device="cuda")
    for _ in range(20):
        x, w = torch.empty(T, K, device="cuda").normal_(generator=gen), torch.empty(N, K, device="cuda").normal_(generator=gen)
        torch.cuda.synchronize()
        binding.quantize_rows(x, x8, xs)
        binding.quantize_rows(w, w8, ws)
        binding.matmul_scaled(x8, xs, w8, ws, out)
        want = (x8.double() @ w8.double().t()) * xs.double()[:, None] * ws.double()
        assert bool(((out.double() - want).abs() <= 4 * 2.0 ** -24 * want.abs()).all())
