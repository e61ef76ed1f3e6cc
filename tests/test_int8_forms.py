"""The forms of the operators in 8-bit integers, which sizes choose, agree with one another bit by bit and serve every place a call can stand in."""
import pytest

from paper_2308_15030_b200 import binding


def _quantized(n, k, gen, std=1.0):
    import torch
    v = torch.empty(n, k, device="cuda").normal_(0.0, std, generator=gen)
    q, s = torch.empty(n, k + -k % 16, dtype=torch.int8, device="cuda")[:, :k], torch.empty(n, device="cuda")
    binding.quantize_rows(v, q, s)
    return q, s


# ------------------------------------------------------------------ the status word
@pytest.mark.parametrize("limit_ms", [0, -1, 1001])
def test_the_self_tests_limit_is_checked(limit_ms):
    assert binding.lib().swapmoe_selftest_matmul_wait(limit_ms, None) == -1


@pytest.mark.gpu
def test_a_timeout_is_reported_once_whatever_the_stream():
    """A wait that runs out ends its kernel, the next status call names it, and the word is clear when that call returns: a call on another stream,
    which nothing orders behind the first one's, finds none."""
    import torch
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    assert binding.matmul_status() == (0, 0)
    for _ in range(5):
        binding.selftest_matmul_wait(limit_ms=5, stream=a)
        assert binding.matmul_status(stream=a) == (-6, 99)              # SWAPMOE_ERR_DEVICE_TIMEOUT, wait code
        assert binding.matmul_status(stream=b) == (0, 0)
    binding.selftest_matmul_wait(limit_ms=5, stream=a)
    a.synchronize()
    assert binding.matmul_status(stream=b) == (-6, 99)                  # on another stream than the wait's
    assert binding.matmul_status(stream=a) == (0, 0)


@pytest.mark.gpu
def test_status_calls_of_many_threads_report_one_timeout_once():
    import threading
    import torch
    binding.selftest_matmul_wait(limit_ms=5)
    torch.cuda.synchronize()
    streams, got, gate = [torch.cuda.Stream() for _ in range(8)], [], threading.Barrier(8)

    def ask(stream):
        gate.wait()
        for _ in range(20):
            got.append(binding.matmul_status(stream=stream))
    threads = [threading.Thread(target=ask, args=(s,)) for s in streams]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert sorted(set(got)) == [(-6, 99), (0, 0)] and got.count((-6, 99)) == 1 and len(got) == 160


# ------------------------------------------------------------------ experts
@pytest.mark.gpu
@pytest.mark.parametrize("d,F,S,k", [(512, 704, 16, 2), (256, 320, 8, 1), (1024, 512, 64, 4), (128, 2112, 5, 3)])
@pytest.mark.parametrize("act", ["swiglu", "relu"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_tokens_experts_do_not_hang_on_the_batch(d, F, S, k, act, dtype):
    """The same tokens alone, in a call of few pairs (weights straight to registers) and in large calls (CTA pairs, pairs counted by
    every CTA or by a kernel of its own): integers are exact, hidden values the same, choices added in their order."""
    import torch
    T = 4200 // k
    gen = torch.Generator(device="cuda").manual_seed(d + F)
    nin = 2 if act == "swiglu" else 1
    w_in, in_scales = _quantized(S * nin * F, d, gen, d ** -0.5)
    w_out, out_scales = _quantized(S * d, F, gen, F ** -0.5)
    x, xs = _quantized(T, d, gen, 2.0)
    top, slots = torch.topk(torch.empty(T, S, device="cuda").normal_(generator=gen), k, 1)
    weights, slots = torch.softmax(top, 1), slots.to(torch.int32)
    slots[1, 0] = -1
    bank = binding.ExpertBank(S, d, F, k, binding.F32 if dtype == "fp32" else binding.BF16, act=binding.ACT_SWIGLU if act == "swiglu" else binding.ACT_RELU,
                              max_tokens=T)
    bank.set_weights(w_in.view(S, nin, F, d), in_scales.view(S, nin, F), w_out.view(S, d, F), out_scales.view(S, d))
    outs = []
    for n in (1, 3, 64 // k, 64 // k + 1, 300, T):                       # up to 64 pairs, and more; the last is beyond 4096
        out = torch.empty(n, d, device="cuda").to(torch.float32 if dtype == "fp32" else torch.bfloat16)
        bank.forward(x[:n], xs[:n], slots[:n], weights[:n], out)
        outs.append(out)
    for out in outs[:-1]:
        assert torch.equal(out, outs[-1][: len(out)]), len(out)
    assert binding.matmul_status() == (0, 0)


# ------------------------------------------------------------------ products
def _pair_width():
    """Columns of a matrix whose tiles of 128 are more than half of the SMs: calls of more than 32 tokens then run on CTA pairs."""
    import torch
    return 128 * (torch.cuda.get_device_properties(0).multi_processor_count // 2 + 2)


@pytest.mark.gpu
@pytest.mark.parametrize("K,extra,dtype", [(512, 0, "fp32"), (512, 0, "bf16"), (200, 5, "fp32"), (336, 2, "bf16"), (128, 7, "bf16")])
@pytest.mark.parametrize("bias", [True, False])
def test_a_tokens_product_does_not_hang_on_the_batch(K, extra, dtype, bias):
    """The same tokens in calls of up to eight (weights straight to registers), of 9 to 32 (clusters) and of more (CTA pairs)."""
    import torch
    N, T = _pair_width() + extra, 300
    gen = torch.Generator(device="cuda").manual_seed(K + extra)
    (x, xs), (w, ws) = _quantized(T, K, gen, 2.0), _quantized(N, K, gen, K ** -0.5)
    b = torch.empty(N, device="cuda").normal_(0.0, 2.0, generator=gen) if bias else None
    assert K * N <= 6 << 20
    outs = []
    for n in (1, 8, 20, 32, 70, T):
        out = torch.empty(n, N, device="cuda").to(torch.float32 if dtype == "fp32" else torch.bfloat16)
        binding.matmul_scaled(x[:n], xs[:n], w, ws, out, bias=b)
        outs.append(out)
    for out in outs[:-1]:
        assert torch.equal(out, outs[-1][: len(out)]), len(out)
    assert binding.matmul_status() == (0, 0)


# Products on CTA pairs, which serve every large matrix, in the places that a call can stand in.
PLACES = [("bf16", 0, 0), ("bf16", 0, 1), ("bf16", 2, 0), ("fp32", 0, 0), ("fp32", 1, 3)]          # dtype, columns beyond the tiles, columns behind a row


def _product(T, K, N, dtype, gen, pad):
    import torch
    (x, xs), (w, ws) = _quantized(T, K, gen, 2.0), _quantized(N, K, gen, K ** -0.5)
    out = torch.zeros(T, N + pad, device="cuda").to(torch.float32 if dtype == "fp32" else torch.bfloat16)[:, :N]
    return [x, xs, w, ws, out]


def _near(out, x, xs, w, ws):
    """Exact sums, two products in fp32, and the result's own rounding."""
    import torch
    want = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()
    half = 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24
    assert bool(((out.double() - want).abs() <= (3.01 * 2.0 ** -24 + 1.001 * half) * want.abs()).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,extra,pad", PLACES)
@pytest.mark.parametrize("T", [48, 400])
def test_pairs_right_behind_what_writes_their_operands(T, dtype, extra, pad):
    import torch
    K, N = 640, _pair_width() + extra
    gen = torch.Generator(device="cuda").manual_seed(T)
    x8, xs, w8, ws, out = _product(T, K, N, dtype, gen, pad)
    for i in range(10):
        x, w = torch.empty(T, K, device="cuda").normal_(0.0, 1.0 + i, generator=gen), torch.empty(N, K, device="cuda").normal_(generator=gen)
        torch.cuda.synchronize()
        binding.quantize_rows(x, x8, xs)
        binding.quantize_rows(w, w8, ws)
        binding.matmul_scaled(x8, xs, w8, ws, out)
        _near(out, x8, xs, w8, ws)
        # and one product right behind another, on its result
        binding.matmul_scaled(x8, xs, w8, ws, out)
        n8, ns = torch.empty(T, N + -N % 16, dtype=torch.int8, device="cuda")[:, :N], torch.empty(T, device="cuda")
        m8, ms = _quantized(N, N, gen, N ** -0.5) if i == 0 else (m8, ms)
        back = torch.empty(T, N, device="cuda", dtype=out.dtype)
        torch.cuda.synchronize()
        binding.matmul_scaled(x8, xs, w8, ws, out)
        binding.quantize_rows(out, n8, ns)
        binding.matmul_scaled(n8, ns, m8, ms, back)
        if i in (0, 9):
            _near(back, n8, ns, m8, ms)
    assert binding.matmul_status() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,extra,pad", PLACES)
def test_pairs_in_a_graph_and_on_two_streams(dtype, extra, pad):
    """Two products on CTA pairs side by side, one beside a product on clusters, and one captured and replayed with other operands."""
    import torch
    K, N, T = 1024, _pair_width() + extra, 300
    gen = torch.Generator(device="cuda").manual_seed(N + pad)
    sets = [_product(T, K, N, dtype, gen, pad), _product(T, K, N, dtype, gen, pad), _product(60, K, 640, dtype, gen, 0), _product(20, K, N, dtype, gen, pad)]
    want = []
    for s in sets:
        binding.matmul_scaled(*s)
        _near(s[4], *s[:4])
        want.append(s[4].clone())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for a, b in ((0, 1), (0, 2), (3, 1)):
        for i in (a, b):
            sets[i][4].zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            for i, st in zip((a, b), streams):
                binding.matmul_scaled(*sets[i], stream=st)
        torch.cuda.synchronize()
        assert torch.equal(sets[a][4], want[a]) and torch.equal(sets[b][4], want[b]), (a, b)
    graph, fixed = torch.cuda.CUDAGraph(), [t.clone() for t in sets[0][:4]]
    out = torch.zeros_like(want[0])
    fixed[0], fixed[2] = sets[0][0].contiguous().clone(), sets[0][2].contiguous().clone()
    with torch.cuda.graph(graph):
        binding.matmul_scaled(*fixed, out)
        binding.matmul_scaled(*fixed, out)
    for i in (1, 0, 1):
        for a, b in zip(fixed, sets[i]):
            a.copy_(b)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
    assert binding.matmul_status() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,extra,pad", PLACES)
def test_pairs_with_scales_that_are_not_finite_or_zero(dtype, extra, pad):
    import torch
    K, N, T = 160, _pair_width() + extra, 300
    gen = torch.Generator(device="cuda").manual_seed(pad)
    x, xs, w, ws, out = _product(T, K, N, dtype, gen, pad)
    binding.matmul_scaled(x, xs, w, ws, out)
    first = out.clone()
    for bad in (float("nan"), float("inf"), 0.0):
        xs2, ws2 = xs.clone(), ws.clone()
        xs2[T // 2], ws2[N - 1] = bad, bad
        binding.matmul_scaled(x, xs2, w, ws2, out)
        want = (x.double() @ w.double().t()) * xs2.double()[:, None] * ws2.double()
        assert bool((torch.isnan(out) == torch.isnan(want)).all())
        infinite, fine = torch.isinf(want), torch.ones_like(out, dtype=torch.bool)
        fine[T // 2], fine[:, N - 1] = False, False
        assert torch.equal(out[fine], first[fine])                      # the others keep their bits
        assert torch.equal(out[infinite].double(), want[infinite])


# ------------------------------------------------------------------ the first calls of a process
FIRST_CALLS = """
import threading, torch
from paper_2308_15030_b200 import binding
torch.cuda.set_device(0)
gate, bad = threading.Barrier(8), []
x, w = torch.randn(40, 256, device="cuda"), torch.randn(300, 256, device="cuda")
one = torch.ones(256, device="cuda")
torch.cuda.synchronize()

def work(i):
    try:
        stream = torch.cuda.Stream()
        x8, xs, w8, ws = torch.empty(40, 256, dtype=torch.int8, device="cuda"), torch.empty(40, device="cuda"), torch.empty(300, 256, dtype=torch.int8, device="cuda"), torch.empty(300, device="cuda")
        n, out = torch.empty_like(x), torch.empty(40, 300, device="cuda")
        torch.cuda.synchronize()
        gate.wait()
        if i % 2:
            binding.block_norm(x, None, one, 1e-6, out=n, stream=stream)
        binding.quantize_rows(x, x8, xs, stream=stream)
        binding.quantize_rows(w, w8, ws, stream=stream)
        binding.matmul_scaled(x8, xs, w8, ws, out, stream=stream)
        stream.synchronize()
        want = (x8.double() @ w8.double().t()) * xs.double()[:, None] * ws.double()
        assert bool(((out.double() - want).abs() <= 4 * 2.0 ** -24 * want.abs()).all())
    except Exception as e:
        bad.append(repr(e))
threads = [threading.Thread(target=work, args=(i,)) for i in range(8)]
[t.start() for t in threads]
[t.join() for t in threads]
assert not bad, bad
print("fine")
"""


@pytest.mark.gpu
def test_first_calls_of_a_process_from_many_threads():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, env={**os.environ, "PYTHONPATH": root}, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]


# ------------------------------------------------------------------ the 8-bit rows behind the norms
@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(3, 512), (700, 768), (40, 1003), (2000, 4096)])
@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("type8", ["int8", "e4m3"])
def test_8_bit_rows_of_the_norm_are_those_of_its_rows(T, d, group, type8):
    """Scales and 8-bit values against the norm's own fp32 rows, within the reciprocals' errors that the header gives: 2^-21 of the scale and of the quotient."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T + d)
    x, r = torch.empty(T, d, device="cuda").normal_(generator=gen), torch.empty(T, d, device="cuda").normal_(0.0, 3.0, generator=gen)
    w = torch.empty(d, device="cuda").normal_(1.0, 0.3, generator=gen)
    n, top = -(-d // group) if group else 1, 127.0 if type8 == "int8" else 448.0
    out, s = torch.empty_like(x), torch.empty(T, n, device="cuda")
    q = torch.empty(T, d, device="cuda").to(torch.int8 if type8 == "int8" else torch.float8_e4m3fn)
    binding.block_norm(x, r, w, 1e-6, out=out, post_weight=w, out8=q, scales=s, group=group)
    y, width, eps = out.double(), group or d, 2.0 ** -21
    most = torch.nn.functional.pad(y.abs(), (0, n * width - d)).view(T, n, width).amax(2)
    assert bool(((s.double() - most / top).abs() <= eps * most / top).all())
    t = y / s.double()[:, torch.arange(d, device="cuda") // width]
    # half a step: of integers 0.5; of e4m3 2^-4 of the value, or 2^-10 below its normal range
    step = torch.full_like(t, 0.5) if type8 == "int8" else torch.clamp(t.abs() * 2.0 ** -4, min=2.0 ** -10)
    assert bool(((q.float().double() - t).abs() <= step + 1.07 * eps * t.abs()).all())
    assert float(q.float().abs().max()) == top


def test_the_norm_of_wide_batches_does_not_spill(tmp_path):
    import os
    from test_kernel_resources_host import NVCC, ptxas_properties
    if not os.path.exists(NVCC):
        pytest.skip("needs nvcc")
    forms = ["%s, %s, 2, true, %s, 256, kBlockNormCtas" % (t, r, row8) for t, r in (("bf16", "float"), ("bf16", "bf16"), ("float", "float"))
             for row8 in ("true", "false")]
    source = '#include "block_norm.cuh"\nnamespace swapmoe {\n' + "".join(
        "template __global__ void block_norm_kernel<%s>(const __grid_constant__ BlockNormArgs);\n" % f for f in forms) + "}\n"
    props = {n: v for n, v in ptxas_properties(source, tmp_path).items() if "block_norm_kernel" in n}
    assert len(props) == len(forms)
    assert all(v == (0, 0, 0) for v in props.values()), props


# ------------------------------------------------------------------ a served block, step by step
@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 45, 1200])
def test_every_step_of_a_served_block(T):
    """Norms, the router's product, routing to resident experts, experts, shared projection, adapters beside it and the next block's norms:
    what each step writes against its definition in 64 bits on what the step before left."""
    import numpy as np
    import torch
    from test_adapters import _reference as adapters_reference
    from test_expert_bank import Case
    from test_route_groups import REL, TINY, reference as route_reference
    d, F, E, S, k, EPS = 512, 320, 32, 12, 2, 1e-6
    c = Case(T, d, F, S, k)
    gen = torch.Generator(device="cuda").manual_seed(T + 1)
    normal = lambda *s, std=1.0: torch.empty(*s, device="cuda").normal_(0.0, std, generator=gen)  # noqa: E731
    x, stream, w, pw = normal(T, d).bfloat16(), normal(T, d, std=2.0), normal(d).bfloat16(), normal(d).bfloat16()

    def norms(x, r, scale):
        """h and y of the norms around a block, and how far fp32 may be off: a norm under 40 roundings, as its own tests derive."""
        x64, f32 = x.double(), 40 * 2.0 ** -24
        p = scale * x64 * pw.double() / torch.sqrt((x64 * x64).mean(1, keepdim=True) + EPS)
        h = r.double() + p
        root = torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
        y = h * w.double() / root
        off_h = f32 * p.abs() + 2.0 ** -24 * h.abs()
        return h, y, off_h, off_h * w.double().abs() / root + y.abs() * (f32 + torch.sqrt((off_h * off_h).mean(1, keepdim=True)) / root)
    n8, ns, before = torch.empty(T, d, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"), stream.clone()
    binding.block_norm(x, stream, w, EPS, residual_out=stream, post_weight=pw, scale=0.5, out8=n8, scales=ns)
    h, y, off_h, off_y = norms(x, before, 0.5)
    assert bool(((stream.double() - h).abs() <= off_h + 2.0 ** -24 * h.abs()).all())
    most = y.abs().amax(1, keepdim=True) / 127.0
    assert bool(((ns.double()[:, None] - most).abs() <= 2.0 ** -21 * most + off_y.amax(1, keepdim=True) / 127.0).all())
    assert bool(((n8.double() * ns.double()[:, None] - y).abs() <= (0.5 + 127 * 2.0 ** -21) * ns.double()[:, None] + off_y).all())
    # the router
    (wr8, wrs), logits = _quantized(E, d, gen, d ** -0.5), torch.empty(T, E, device="cuda")
    binding.matmul_scaled(n8, ns, wr8, wrs, logits)
    _near(logits, n8, ns, wr8, wrs)
    table = torch.full((E,), -1, dtype=torch.int32, device="cuda")
    table[torch.randperm(E, device="cuda", generator=gen)[:S]] = torch.arange(S, dtype=torch.int32, device="cuda")
    experts, weights, slots = (torch.empty(T, k, dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.int32))
    binding.route(binding.Gate(renorm=True), logits, experts, weights, expert_to_slot=table, slots=slots)
    e, wt, s = route_reference(logits.cpu().numpy(), k, "softmax", 1, 1, 1, True, 1.0, table=table.cpu().numpy())
    assert np.array_equal(experts.cpu().numpy(), e) and np.array_equal(slots.cpu().numpy(), s)
    assert np.all(np.abs(weights.cpu().numpy().astype(np.float64) - wt) <= REL * wt + TINY)
    # the experts
    c.x, c.xs, c.slots, c.weights = n8, ns, slots, weights
    out = c.run()
    c.check(out)
    # the projection that all tokens share, and each token's adapter beside it
    (wp8, wps), shared = _quantized(d, d, gen, d ** -0.5), torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    binding.matmul_scaled(n8, ns, wp8, wps, shared)
    _near(shared, n8, ns, wp8, wps)
    n16, ids = (n8.float() * ns[:, None]).bfloat16(), torch.randint(-1, 3, (T,), device="cuda", generator=gen).to(torch.int32)
    A, B = normal(3, 8, d, std=d ** -0.5).bfloat16(), normal(3, d, 8, std=0.3).bfloat16()
    bank, both = binding.AdapterBank(3, d, d, 8, binding.BF16, max_tokens=T), torch.empty_like(shared)
    bank.set_weights(A, B)
    bank.forward(n16, ids, shared, both)
    want, slack = adapters_reference(n16, shared, None, A, B, torch.ones(3, device="cuda"), ids, "bf16")
    assert bool(((both.double() - want).abs() <= slack).all())
    # the next block's norms
    total, nxt, new = (out.float() + both.float()).bfloat16(), torch.empty_like(out), torch.empty_like(stream)
    binding.block_norm(total, stream, w, EPS, out=nxt, residual_out=new, post_weight=pw)
    h, y, off_h, off_y = norms(total, stream, 1.0)
    assert bool(((new.double() - h).abs() <= off_h + 2.0 ** -24 * h.abs()).all())
    assert bool(((nxt.double() - y).abs() <= 1.001 * 2.0 ** -8 * y.abs() + off_y + 1e-40).all())
    assert binding.matmul_status() == (0, 0)
