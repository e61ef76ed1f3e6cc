"""Low-rank adapters of many requests beside a shared projection, against the formula in 64 bits."""
import ctypes

import numpy as np
import pytest

from paper_2308_15030_b200 import binding


# ------------------------------------------------------------------ refusals (host checks, no GPU needed)
@pytest.mark.parametrize("kw,status", [
    (dict(n_adapters=0), -1), (dict(d_in=0), -1), (dict(d_out=0), -1), (dict(rank=0), -1), (dict(max_tokens=0), -1),
    (dict(dtype=2), -1), (dict(d_in=12), -7), (dict(d_out=12), -7), (dict(rank=12), -7), (dict(rank=136), -7),
    (dict(n_adapters=4097), -7), (dict(max_tokens=1 << 24), -7)])
def test_create_refusals(kw, status):
    base = dict(n_adapters=4, d_in=64, d_out=64, rank=8, dtype=1, max_tokens=4)
    base.update(kw)
    h, c = ctypes.c_void_p(), binding.AdaptersConfig(**base)
    assert binding.lib().swapmoe_adapters_create(ctypes.byref(h), ctypes.byref(c)) == status and not h


def test_null_handles():
    L = binding.lib()
    assert L.swapmoe_adapters_create(None, None) == -1
    assert L.swapmoe_adapters_destroy(None) == 0
    assert L.swapmoe_adapters_set_weights(None, 256, 256, None) == -1
    assert L.swapmoe_adapters_forward(None, 256, 64, None, 256, None, 0, 256, 64, 1, None) == -1


# ------------------------------------------------------------------ on the GPU
def _make(T, d, n, r, count, dtype="bf16", x8=False, seed=0, pad=0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16

    def rows(width):
        return torch.empty(T, width + pad, device="cuda").normal_(generator=gen).to(dt)[:, :width]
    x, y = rows(d), rows(n)
    xs = None
    if x8:
        xs = torch.empty(T, device="cuda").uniform_(0.001, 0.01, generator=gen)
        x = torch.empty(T, d + 2 * pad, device="cuda").normal_(0, 100, generator=gen).clamp(-448, 448).to(torch.float8_e4m3fn)[:, :d]
    A = torch.empty(count, r, d, device="cuda").normal_(0, d ** -0.5, generator=gen).to(dt)
    B = torch.empty(count, n, r, device="cuda").normal_(0, r ** -0.5, generator=gen).to(dt)
    scale = torch.empty(count, device="cuda").uniform_(-2, 2, generator=gen)
    bank = binding.AdapterBank(count, d, n, r, binding.F32 if dtype == "fp32" else binding.BF16, max_tokens=T)
    bank.set_weights(A, B, scale)
    return x, y, xs, A, B, scale, bank


def _reference(x, y, xs, A, B, scale, ids, dtype):
    """out in 64 bits, and how far each value may be off."""
    import torch
    x = x.double() * (1.0 if xs is None else xs.double()[:, None])
    T, d, r = x.shape[0], x.shape[1], A.shape[1]
    out = torch.zeros(T, B.shape[1], dtype=torch.float64, device="cuda") if y is None else y.double().clone()
    slack = torch.zeros_like(out)
    for a in range(A.shape[0]):
        t = torch.nonzero(ids == a)[:, 0]
        if t.numel() == 0:
            continue
        A64, B64, sc = A[a].double(), B[a].double(), float(scale[a])
        u, um = x[t] @ A64.T * sc, x[t].abs() @ A64.abs().T * abs(sc)
        out[t] += u @ B64.T
        if dtype == "bf16":
            # exact products, tensor-core sums that truncate (2^-23 of the terms' magnitude per step of 16 and per merge of
            # partial sums), u rounded to bf16 (2^-8)
            eu = (d / 16 + 64) * 2.0 ** -23 * um + 2.0 ** -8 * u.abs()
            slack[t] += (eu + (r / 16 + 8) * 2.0 ** -23 * u.abs()) @ B64.abs().T * 1.01
        else:
            # operands in two pieces of 11 bits: 2^-21 per product; sums as above in steps of 8, three products each
            eu = (2.0 ** -20 + (3 * d / 8 + 64) * 2.0 ** -23) * um
            slack[t] += (eu + (2.0 ** -20 + (3 * r / 8 + 8) * 2.0 ** -23) * (u.abs() + eu)) @ B64.abs().T
    slack += out.abs() * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -22) + 1e-30
    return out, slack


def _ids(T, count, seed, none=0.15, run=1):
    import torch
    rng = np.random.default_rng(seed)
    v = rng.integers(0, count, -(-T // run))
    v[rng.random(v.size) < none] = -1
    return torch.from_numpy(np.repeat(v, run)[:T].astype(np.int32)).cuda()


def _check(T, d, n, r, count, dtype="bf16", x8=False, ids=None, pad=0, with_y=True, seed=1):
    import torch
    x, y, xs, A, B, scale, bank = _make(T, d, n, r, count, dtype, x8, seed, pad)
    ids = _ids(T, count, seed) if ids is None else ids
    mem = torch.full((T + 2, n + pad), 3.0, device="cuda").to(y.dtype)
    out = mem[1:T + 1, :n]
    bank.forward(x, ids, y if with_y else None, out, x_scales=xs)
    torch.cuda.synchronize()
    want, slack = _reference(x, y if with_y else None, xs, A, B, scale, ids, dtype)
    err = (out.double() - want).abs()
    assert bool((err <= slack).all()), float((err / slack).max())
    idle = (ids < 0) | (ids >= count)
    assert torch.equal(out[idle], y[idle] if with_y else torch.zeros_like(y[idle]))
    assert bool((mem[0] == 3).all()) and bool((mem[T + 1] == 3).all()) and bool((mem[:, n:] == 3).all())
    again = torch.empty_like(out)
    bank.forward(x, ids, y if with_y else None, again, x_scales=xs)
    assert torch.equal(again, out)
    return x, y, xs, ids, out, bank


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,x8", [("bf16", False), ("bf16", True), ("fp32", False)])
@pytest.mark.parametrize("T,d,n,r,count", [(1, 64, 64, 8, 1), (1, 1024, 1024, 16, 8), (3, 4096, 512, 16, 5), (17, 704, 2240, 8, 40),
                                           (61, 1024, 4096, 16, 64), (64, 256, 256, 128, 3), (65, 1536, 1088, 40, 7),
                                           (200, 512, 768, 64, 9), (1000, 768, 960, 32, 4), (300, 72, 8, 24, 11), (130, 8, 200, 8, 300),
                                           (5, 48, 4104, 120, 2)])
def test_shapes(T, d, n, r, count, dtype, x8):
    _check(T, d, n, r, count, dtype, x8)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257])
def test_one_adapter_for_all(T):
    import torch
    _check(T, 512, 320, 16, 3, ids=torch.full((T,), 1, dtype=torch.int32, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [4, 70, 700])
def test_no_adapter_at_all_and_ids_outside_the_bank(T):
    import torch
    _check(T, 256, 256, 16, 4, ids=torch.full((T,), -1, dtype=torch.int32, device="cuda"))
    ids = torch.arange(T, dtype=torch.int32, device="cuda") % 7 - 1           # 4 and 5 are not in the bank
    ids[-1] = 2 ** 31 - 1
    ids[0] = -(2 ** 31)
    _check(T, 256, 256, 16, 4, ids=ids)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,x8", [("bf16", False), ("bf16", True), ("fp32", False)])
def test_strides_and_no_projection(dtype, x8):
    _check(50, 256, 320, 16, 6, dtype, x8, pad=8)
    _check(150, 256, 320, 16, 6, dtype, x8, pad=8, with_y=False)


@pytest.mark.gpu
@pytest.mark.parametrize("run", [3, 50, 512])
def test_runs_of_requests(run):
    _check(1531, 512, 768, 16, 12, ids=_ids(1531, 12, run, run=run))


@pytest.mark.gpu
def test_a_row_hangs_on_itself_and_its_adapter():
    """The same rows in another order give the same rows in that order; other rows' NaN stay theirs."""
    import torch
    x, y, xs, ids, out, bank = _check(333, 256, 320, 16, 5)
    p = torch.randperm(333, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    again = torch.empty_like(out)
    bank.forward(x[p].contiguous(), ids[p].contiguous(), y[p].contiguous(), again)
    assert torch.equal(again, out[p])
    x2 = x.clone()
    x2[7] = float("nan")
    ids[7] = 2
    bank.forward(x2, ids, y, again)
    keep = torch.arange(333, device="cuda") != 7
    assert torch.equal(again[keep], out[keep]) and bool(again[7].isnan().all())


@pytest.mark.gpu
def test_in_place_and_unit_scale():
    import torch
    x, y, xs, ids, out, bank = _check(90, 256, 320, 16, 5)
    y2 = y.clone()
    bank.forward(x, ids, y2, y2)
    assert torch.equal(y2, out)
    A, B, scale = bank._keep
    bank.set_weights(A, B)
    bank.forward(x, ids, y, y2)
    want, slack = _reference(x, y, None, A, B, torch.ones_like(scale), ids, "bf16")
    assert bool(((y2.double() - want).abs() <= slack).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T", [20, 500])
def test_two_captured_graphs_on_one_bank(T):
    import torch
    x, y, xs, ids, out, bank = _check(T, 256, 320, 16, 5)
    ids2 = (ids + 1) % 5
    o1, o2, w2 = torch.empty_like(out), torch.empty_like(out), torch.empty_like(out)
    bank.forward(x, ids2.contiguous(), y, w2)
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        bank.forward(x, ids, y, o1)
    with torch.cuda.graph(g2):
        bank.forward(x, ids2, y, o2)
    for _ in range(3):
        o1.zero_(), o2.zero_()
        g1.replay(), g2.replay(), g1.replay()
        torch.cuda.synchronize()
        assert torch.equal(o1, out) and torch.equal(o2, w2)


@pytest.mark.gpu
def test_refusals_with_a_bank():
    import torch
    bank = binding.AdapterBank(2, 64, 64, 8, binding.BF16, max_tokens=4)
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    L = binding.lib()

    def call(**kw):
        a = dict(x=x.data_ptr(), xs=64, sc=None, ids=ids.data_ptr(), y=None, ys=0, out=x.data_ptr(), os=64, T=4)
        a.update(kw)
        return L.swapmoe_adapters_forward(bank._h, a["x"], a["xs"], a["sc"], a["ids"], a["y"], a["ys"], a["out"], a["os"], a["T"], None)
    assert call() == -2                                        # no weights yet
    A = torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda")
    B = torch.zeros(2, 64, 8, dtype=torch.bfloat16, device="cuda")
    assert L.swapmoe_adapters_set_weights(bank._h, A.data_ptr() + 2, B.data_ptr(), None) == -1
    for a, b in ((A[:1], B), (A, B.float()), (A.cpu(), B)):
        with pytest.raises(binding.SwapMoEError) as e:
            bank.set_weights(a, b)
        assert e.value.status == -1
    bank.set_weights(A, B)
    for kw, st in ((dict(T=5), -3), (dict(T=-1), -1), (dict(T=0, x=None), 0), (dict(x=None), -1), (dict(ids=None), -1), (dict(out=None), -1),
                   (dict(xs=60), -1), (dict(xs=68), -1), (dict(os=63), -1), (dict(x=x.data_ptr() + 2), -1),
                   (dict(y=x.data_ptr(), ys=60), -1), (dict(ids=ids.data_ptr() + 1), -1)):
        assert call(**kw) == st, kw
    with pytest.raises(binding.SwapMoEError):
        bank.forward(x.float(), ids, None, x)
    with pytest.raises(binding.SwapMoEError):
        bank.forward(x, ids.long(), None, x)
    f = binding.AdapterBank(2, 64, 64, 8, binding.F32, max_tokens=4)
    assert L.swapmoe_adapters_set_weights(f._h, A.data_ptr(), B.data_ptr(), None) == 0
    assert L.swapmoe_adapters_forward(f._h, x.data_ptr(), 64, ids.data_ptr(), ids.data_ptr(), None, 0, x.data_ptr(), 64, 1, None) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d,r", [(1, 64, 8), (20, 256, 16), (100, 512, 64), (700, 256, 16), (3000, 512, 64), (300, 1024, 128)])
def test_infinities_and_the_largest_values(T, d, r, dtype):
    """Infinities in x, A, B and y, and finite values beyond bf16's largest, give what the formula gives."""
    import torch
    n, count = 136, 4
    x, y, _, A, B, scale, bank = _make(T, d, n, r, count, dtype, seed=T)
    A[:, :, 5], A[:, :, 6], scale[:] = A[:, :, 5].abs() + 0.01, A[:, :, 6].abs() * 2.0 ** -20, scale.abs() + 0.1
    B[:2] = B[:2].abs() + 0.01                         # adapters 0 and 1: infinities of one sign stay infinite
    A[1, :, 9], B[1, 40], B[1, 41, 0] = float("inf"), float("inf"), float("-inf")
    B[3, 50, 1], B[3, 51] = float("inf"), 0.0
    ids = torch.arange(T, dtype=torch.int32, device="cuda") % (count + 1) - 1
    ids[0] = 0
    x[::3, 5] = float("inf")
    x[1::7, 5] = float("-inf")
    if dtype == "fp32":
        x[2::3, 6] = 3.4e38                            # (bf16's largest is 3.39e38)
        B[0, 60] *= 2.0 ** -120
    y[::4, 7], y[1::4, 8] = float("inf"), float("nan")
    bank.set_weights(A, B, scale)
    for with_y in (True, False):
        out = torch.empty_like(y)
        bank.forward(x, ids, y if with_y else None, out)
        want, slack = _reference(x, y if with_y else None, None, A, B, scale, ids, dtype)
        if dtype == "fp32":
            # bf16's smallest step is 2^-133: what three pieces leave of an operand below 2^-110 (the weights of B[0, 60]) is up to half
            # of that, however small the operand; times the sum of |u|, which is at most that of |A| |x|
            for a in range(count):
                t = torch.nonzero(ids == a)[:, 0]
                slack[t] += 2.0 ** -134 * (x[t].double().abs() @ A[a].double().abs().T * scale[a].double()).sum(1)[:, None]
        want = torch.where(want.abs() > torch.finfo(y.dtype).max, want.sign() * float("inf"), want)
        assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.isinf(), want.isinf())
        infinite, finite = want.isinf(), want.isfinite()
        assert torch.equal(out.double()[infinite], want[infinite])
        assert bool(((out.double() - want).abs()[finite] <= slack[finite]).all())


# ------------------------------------------------------------------ what the pieces of the operands keep
def _pieces(v, n):
    """A float32 array as n bf16 pieces, each rounded to nearest from what the ones in front left."""
    import torch
    got, rest = [], torch.from_numpy(v)
    for _ in range(n):
        got.append(rest.bfloat16().double().numpy())
        rest = rest - rest.bfloat16().float()
    return got


def _product(x, w, n, most):
    """x w^T from n pieces each, of the products i, j those with i + j <= most; sums in 64 bits."""
    xs, ws = _pieces(x, n), _pieces(w, n)
    return sum(xs[i] @ ws[j].T for i in range(n) for j in range(n) if i + j <= most)


def _rms_limit(d, r):
    """Largest rms error of fp32 results relative to their rms, without y, for values of random signs.  A product of three pieces
    each and six of their products is off by 2^-24 per operand and twice 2^-24 for those left out: 2^-22; the six truncations of a
    step by 6 x 2^-23 of the step's sum, and steps of random signs add up as their results do: 16 x 2^-24 in all, for each of
    the two products.  The n = d / 16 (r / 16) steps are added in fp32: 2^-24 of the sum so far each, sqrt(n / 2) of the result; 8 for
    partial sums, scales and the last rounding."""
    return (32 + (d / 32) ** 0.5 + (r / 32) ** 0.5 + 8) * 2.0 ** -24


RMS_SHAPES = [(64, 8), (256, 16), (512, 64), (1024, 128), (4096, 16)]


@pytest.mark.parametrize("d,r", RMS_SHAPES)
def test_the_rms_limit_tells_three_pieces_from_two(d, r):
    """Two pieces (or three without the products of the small ones) are beyond the limit, three pieces and six products within."""
    rng = np.random.default_rng(d)
    x, A, B = (rng.normal(0, 1, s).astype(np.float32) for s in ((40, d), (r, d), (96, r)))
    u = x.astype(np.float64) @ A.T.astype(np.float64)
    want = u @ B.T.astype(np.float64)

    def error(n, most):
        got = _product(_product(x, A, n, most).astype(np.float32), B, n, most)
        return np.sqrt(np.mean((got - want) ** 2) / np.mean(want ** 2))
    assert error(3, 2) < 0.2 * _rms_limit(d, r)
    assert error(2, 1) > 1.2 * _rms_limit(d, r) and error(3, 1) > 1.2 * _rms_limit(d, r)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [7, 90, 400, 3000])
@pytest.mark.parametrize("d,r", RMS_SHAPES)
def test_fp32_banks_keep_24_bits(T, d, r):
    import torch
    n, count = 328, 3
    x, y, _, A, B, scale, bank = _make(T, d, n, r, count, "fp32", seed=d + T)
    ids = _ids(T, count, T, none=0.0)
    out = torch.empty_like(y)
    bank.forward(x, ids, None, out)
    want, _ = _reference(x, None, None, A, B, scale, ids, "fp32")
    assert float(((out.double() - want) ** 2).mean().sqrt() / (want ** 2).mean().sqrt()) <= _rms_limit(d, r)


@pytest.mark.gpu
@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T", [1, 20, 100, 700, 3000])
@pytest.mark.parametrize("d,r", [(64, 8), (64, 16), (128, 24), (256, 32), (256, 40), (256, 64), (512, 128)])
def test_bf16_banks_round_only_their_results(T, d, r, x8):
    """What lies between the two products is kept in two bf16 pieces: no error of the type's size but the results' own."""
    import torch
    n, count = 264, 3
    x, y, xs, A, B, scale, bank = _make(T, d, n, r, count, "bf16", x8, seed=r + T)
    ids = _ids(T, count, T, none=0.0)
    out = torch.empty_like(y)
    for with_y in (False, True):
        bank.forward(x, ids, y if with_y else None, out, x_scales=xs)
        want, _ = _reference(x, y if with_y else None, xs, A, B, scale, ids, "bf16")
        x64 = x.double() * (1.0 if xs is None else xs.double()[:, None])
        slack = want.abs() * 2.0 ** -8
        for a in range(count):
            t = torch.nonzero(ids == a)[:, 0]
            A64, B64, sc = A[a].double(), B[a].double(), abs(float(scale[a]))
            u, um = (x64[t] @ A64.T).abs() * sc, x64[t].abs() @ A64.abs().T * sc
            # products of bf16 are exact; truncating sums (2^-23 of the terms' magnitude per step of 16 and per merge of partial sums); the
            # factors 2^-22; two pieces 2^-8 x 2^-8; their two products, summed the same way
            eu = (d / 16 + 64) * 2.0 ** -23 * um + (2.0 ** -22 + 2.0 ** -16) * u
            slack[t] += (eu + (2 * r / 16 + 8) * 2.0 ** -23 * u) @ B64.abs().T * 1.01
        err = (out.double() - want).abs()
        assert bool((err <= slack + 1e-30).all()), float((err / slack).max())
