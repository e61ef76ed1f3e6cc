"""Experts in 8-bit integers behind a router, against the definition in 64 bits, alone and with the operators around them."""
import ctypes

import pytest

from paper_2308_15030_b200 import binding

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}          # largest relative error of one rounding


# ------------------------------------------------------------------ refusals (host checks, no GPU needed)
@pytest.mark.parametrize("kw,status", [
    (dict(n_slots=0), -1), (dict(d_model=0), -1), (dict(d_ff=-64), -1), (dict(top_k=0), -1), (dict(max_tokens=0), -1), (dict(dtype=2), -1),
    (dict(act=2), -1), (dict(n_slots=257), -7), (dict(top_k=17), -7), (dict(d_model=100), -7), (dict(d_ff=96), -7), (dict(d_model=32832), -7),
    (dict(d_ff=32832), -7), (dict(max_tokens=1 << 23), -7)])
def test_create_refuses_before_touching_the_device(kw, status):
    base = dict(n_slots=8, d_model=128, d_ff=256, top_k=2, dtype=1, act=1, max_tokens=16)
    h = ctypes.c_void_p()
    assert binding.lib().swapmoe_expert_bank_create(ctypes.byref(h), ctypes.byref(binding.ExpertBankConfig(**{**base, **kw}))) == status
    assert not h


def test_null_handles():
    L = binding.lib()
    assert L.swapmoe_expert_bank_create(None, None) == -1
    assert L.swapmoe_expert_bank_destroy(None) == 0
    assert L.swapmoe_expert_bank_set_weights(None, 256, 256, 256, 256) == -1
    assert L.swapmoe_expert_bank_forward(None, 256, 128, 256, 256, 256, 256, 128, 1, None) == -1


# ------------------------------------------------------------------ on the GPU
def _int8(n, k, gen, std):
    import torch
    v = torch.empty(n, k, device="cuda").normal_(0.0, std, generator=gen)
    s = v.abs().amax(1) / 127.0
    return (v / s[:, None]).round().to(torch.int8), s


class Case:
    def __init__(self, T, d, F, S, k, act="swiglu", dtype="bf16", none=0.0, max_tokens=None, seed=0, only=None):
        import torch
        gen = torch.Generator(device="cuda").manual_seed(T * 7919 + d + F + S * 31 + k + seed)
        self.T, self.d, self.F, self.S, self.k, self.act, self.dtype = T, d, F, S, k, act, dtype
        nin = 2 if act == "swiglu" else 1
        w, s = _int8(S * nin * F, d, gen, d ** -0.5)
        self.w_in, self.in_scales = w.view(S, nin, F, d), s.view(S, nin, F)
        w, s = _int8(S * d, F, gen, F ** -0.5)
        self.w_out, self.out_scales = w.view(S, d, F), s.view(S, d)
        self.bank = binding.ExpertBank(S, d, F, k, binding.F32 if dtype == "fp32" else binding.BF16,
                                       act=binding.ACT_SWIGLU if act == "swiglu" else binding.ACT_RELU, max_tokens=max_tokens or T)
        self.bank.set_weights(self.w_in, self.in_scales, self.w_out, self.out_scales)
        self.tokens(T, gen, none, only)

    def tokens(self, T, gen, none=0.0, only=None):
        import torch
        self.T = T
        self.x, self.xs = _int8(T, self.d, gen, 1.0)
        logits = torch.empty(T, self.S, device="cuda").normal_(0.0, 1.5, generator=gen) + torch.empty(self.S, device="cuda").normal_(0.0, 1.0, generator=gen)
        top, slots = torch.topk(logits, min(self.k, self.S), 1)
        if slots.shape[1] < self.k:                                      # more choices than slots: some twice
            slots, top = slots[:, torch.arange(self.k) % slots.shape[1]], top[:, torch.arange(self.k) % slots.shape[1]]
        self.slots, self.weights = slots.to(torch.int32).contiguous(), torch.softmax(top, 1).contiguous()
        if only is not None:
            self.slots.fill_(only)
        gone = torch.rand(T, self.k, device="cuda", generator=gen) < none
        self.slots[gone] = -1

    def run(self, out=None, stream=None):
        import torch
        if out is None:
            out = torch.full((self.T, self.d), 7.0, device="cuda").to(torch.float32 if self.dtype == "fp32" else torch.bfloat16)
        self.bank.forward(self.x, self.xs, self.slots, self.weights, out, stream=stream)
        return out

    def check(self, out):
        """Against 64 bits.  A hidden value that lies as near to the middle of two integers as fp32's errors reach may become either: a step
        there is allowed for, everywhere else only the roundings behind the exact sums."""
        import torch
        want = torch.zeros(self.T, self.d, dtype=torch.float64, device="cuda")
        tol = torch.zeros_like(want)
        for e in range(self.S):
            t, j = torch.nonzero(self.slots == e, as_tuple=True)
            if not t.numel():
                continue
            xs = self.xs[t].double()[:, None]
            u = [(self.x[t].double() @ w.double().t()) * xs * s.double() for w, s in zip(self.w_in[e], self.in_scales[e])]
            if self.act == "swiglu":
                h = u[0] / (1.0 + torch.exp(-u[0])) * u[1]
                # the two sums: three roundings each, the first one's by silu's slope times x over silu, at most 1 + |x|; the exponential is within
                # 2 + 1.2 |x| steps of 2^-23; quotient and product two more
                off = h.abs() * ((2.0 + u[0].abs()) * 3 * 2.0 ** -24 + (2.0 + 1.2 * u[0].abs()) * 2.0 ** -23 + 4 * 2.0 ** -24)
            else:
                h = u[0].clamp(min=0.0)
                off = h.abs() * 3 * 2.0 ** -24
            most = h.abs().amax(1, keepdim=True)
            scale = most / 127.0
            safe = torch.where(scale > 0, scale, 1.0)
            rel = (off / torch.where(h.abs() > 0, h.abs(), 1.0)).amax(1, keepdim=True)     # of the scale
            v = h / safe
            q = torch.round(v)
            near = ((v - torch.floor(v) - 0.5).abs() <= off / safe + v.abs() * (rel + 3 * 2.0 ** -24)).double()
            wt = self.weights[t, j].double()[:, None]
            os = self.out_scales[e].double()
            y = (q @ self.w_out[e].double().t()) * scale * os * wt
            step = (near @ self.w_out[e].double().t().abs()) * scale * os * wt.abs()
            want.index_add_(0, t, y)
            tol.index_add_(0, t, step + y.abs() * (rel + 10 * 2.0 ** -24) + self.k * 2.0 ** -24 * y.abs())
        tol = tol * (1 + 2.0 ** -8) + HALF[self.dtype] * want.abs() + 1e-30
        bad = (out.double() - want).abs() > tol
        assert not bool(bad.any()), (int(bad.sum()), torch.nonzero(bad)[:4].tolist())
        # the allowance is a small part of what there is to see
        if self.T * self.k > 8 and float(want.abs().max()) > 0:
            assert float(tol.norm()) < 0.1 * float(want.norm()) + 1e-12
        assert binding.matmul_status() == (0, 0)
        return want


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 3, 7, 16, 31, 33, 64, 65, 100, 128, 200, 300, 500, 1000, 2300])
@pytest.mark.parametrize("act", ["swiglu", "relu"])
def test_token_counts(T, act):
    c = Case(T, 256, 320, 8, 2, act)
    c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("d,F,S,k", [(64, 64, 1, 1), (64, 192, 4, 1), (192, 64, 16, 4), (320, 704, 48, 2), (512, 128, 256, 8), (1024, 512, 64, 4),
                                     (128, 2112, 5, 3), (768, 1088, 33, 16), (2048, 1024, 8, 2), (64, 64, 2, 5)])
@pytest.mark.parametrize("T,dtype", [(1, "bf16"), (19, "fp32"), (260, "bf16")])
def test_shapes(d, F, S, k, T, dtype):
    c = Case(T, d, F, S, k, dtype=dtype)
    c.check(c.run())
    c = Case(T, d, F, S, k, "relu", dtype)
    c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 70, 1500])
def test_choices_that_found_no_expert(T):
    import torch
    c = Case(T, 256, 192, 12, 3, none=0.4)
    c.slots[1] = -1                                                      # a token without any
    c.slots[2, 0], c.slots[3, 1] = 12, 2000000000                        # not in the bank
    out = c.run()
    c.check(out)
    assert bool((out[1] == 0).all())
    c.slots.fill_(-1)
    assert bool((c.run() == 0).all())
    c.slots.fill_(-2147483648)
    assert bool((c.run() == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40, 700, 2200])
def test_one_expert_takes_all(T):
    c = Case(T, 192, 256, 9, 2, only=4)                                  # both choices of a token too
    c.check(c.run())


@pytest.mark.gpu
def test_many_slots_of_few_rows_and_many_pairs():
    c = Case(3000, 128, 128, 200, 6)
    c.check(c.run())
    c = Case(9000, 64, 128, 3, 1)
    c.check(c.run())


@pytest.mark.gpu
def test_calls_of_different_sizes_on_one_bank():
    """What a large call leaves behind does not reach a small one, nor the other way round; the same call gives the same bits."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    c = Case(2500, 256, 192, 16, 2)
    first = c.run()
    c.check(first)
    keep = (c.x, c.xs, c.slots, c.weights, c.T)
    for T in (3, 2500, 1, 600, 2100):
        c.tokens(T, gen, none=0.2)
        a, b = c.run(), c.run()
        assert torch.equal(a, b)
        c.check(a)
    c.x, c.xs, c.slots, c.weights, c.T = keep
    assert torch.equal(c.run(), first)


@pytest.mark.gpu
@pytest.mark.parametrize("pad", [0, 1, 2, 8])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_inside_wider_ones(pad, dtype):
    import torch
    c = Case(33, 128, 128, 4, 2, dtype=dtype)
    want = c.run()
    wide = torch.zeros(33, 160, dtype=torch.int8, device="cuda")
    wide[:, :128] = c.x
    c.x = wide[:, :128]
    mem = torch.full((35, 128 + pad), 7.0, device="cuda").to(want.dtype)
    c.run(mem[1:34, :128])
    assert torch.equal(mem[1:34, :128], want)
    mem[1:34, :128] = 7.0
    assert bool((mem == 7.0).all())


@pytest.mark.gpu
def test_rows_that_are_not_finite_and_zero_rows():
    import torch
    for T in (20, 600):
        c = Case(T, 128, 192, 4, 2, dtype="fp32")
        first = c.run()
        c.xs[3], c.xs[5], c.xs[7] = float("nan"), float("inf"), 0.0
        c.x[9] = 0
        out = c.run()
        assert bool(torch.isnan(out[3]).all()) and not bool(torch.isfinite(out[5]).any()) and bool((out[7] == 0).all()) and bool((out[9] == 0).all())
        calm = torch.ones(T, dtype=torch.bool, device="cuda")
        calm[[3, 5, 7, 9]] = False
        assert torch.equal(out[calm], first[calm])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 900])
def test_streams_and_graphs(T):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T)
    c = Case(T, 256, 320, 8, 2)
    want = c.run()
    side, out = torch.cuda.Stream(), torch.zeros_like(want)
    torch.cuda.synchronize()
    c.run(out, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(out)
    fixed = (c.x, c.xs, c.slots, c.weights)
    for _ in range(3):
        c.tokens(T, gen, none=0.1)
        want = c.run()
        for a, b in zip(fixed, (c.x, c.xs, c.slots, c.weights)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.gpu
def test_refusals_of_a_bank():
    import torch
    c = Case(8, 128, 128, 4, 2)
    out = torch.full((9, 128), 7.0, device="cuda").bfloat16()
    nine = lambda t: torch.cat([t, t[:1]])  # noqa: E731
    with pytest.raises(binding.SwapMoEError) as e:
        c.bank.forward(nine(c.x), nine(c.xs), nine(c.slots), nine(c.weights), out)
    assert e.value.status == -3
    for kw in (dict(x8=c.x.float()), dict(x8=c.x[:, :64]), dict(x_scales=c.xs[:7]), dict(slots=c.slots.long()), dict(slots=c.slots[:, :1]),
               dict(weights=c.weights.bfloat16()), dict(out=out[:7]), dict(out=out.float()), dict(out=out.cpu()),
               dict(x8=torch.zeros(8, 136, dtype=torch.int8, device="cuda")[:, :128])):
        with pytest.raises(binding.SwapMoEError) as e:
            c.bank.forward(**{**dict(x8=c.x, x_scales=c.xs, slots=c.slots, weights=c.weights, out=out[:8]), **kw})
        assert e.value.status == -1, kw
    assert bool((out == 7.0).all())
    fresh = binding.ExpertBank(4, 128, 128, 2, binding.BF16, max_tokens=8)
    with pytest.raises(binding.SwapMoEError) as e:
        fresh.forward(c.x, c.xs, c.slots, c.weights, out[:8])
    assert e.value.status == -2
    with pytest.raises(binding.SwapMoEError):
        fresh.set_weights(c.w_in[:3], c.in_scales, c.w_out, c.out_scales)
    c.bank.forward(c.x[:0], c.xs[:0], c.slots[:0], c.weights[:0], out[:0])


@pytest.mark.gpu
@pytest.mark.parametrize("d,F,S,k,T", [(64, 32768, 2, 1, 1), (64, 32768, 2, 2, 19), (32768, 64, 2, 1, 3), (32768, 64, 1, 2, 40), (4096, 4096, 2, 2, 3),
                                       (1024, 1024, 16, 16, 1), (256, 256, 16, 4, 4), (256, 192, 5, 8, 2)])
def test_widest_experts_and_few_pairs(d, F, S, k, T):
    c = Case(T, d, F, S, k)
    c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("d,F,S,k,T", [(512, 256, 128, 8, 7), (512, 704, 16, 2, 24), (1024, 512, 64, 4, 10), (768, 2112, 32, 2, 7), (64, 64, 4, 3, 21),
                                       (128, 128, 5, 5, 11), (256, 128, 3, 16, 4), (64, 192, 9, 1, 64), (192, 4096, 6, 7, 3), (4096, 64, 40, 6, 10)])
@pytest.mark.parametrize("act,dtype", [("swiglu", "bf16"), ("relu", "fp32")])
def test_few_pairs_in_several_groups_of_tokens(d, F, S, k, T, act, dtype):
    c = Case(T, d, F, S, k, act, dtype)
    c.check(c.run())
    c = Case(T, d, F, S, k, act, dtype, none=0.3)
    c.slots[T - 1] = -1                                                  # the last token has no expert
    c.check(c.run())
    c = Case(T, d, F, S, k, act, dtype, only=S - 1)
    c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("d,F,S,k,T", [(4096, 64, 3, 1, 7000), (64, 4096, 5, 2, 3500), (2048, 2048, 2, 2, 6500)])
def test_rows_beyond_a_scheduling_group(d, F, S, k, T):
    """More rows than stay in L2 at once: both products walk them in groups."""
    c = Case(T, d, F, S, k)
    c.check(c.run())


@pytest.mark.gpu
def test_two_banks_at_once():
    """Banks of their own workspace on streams of their own, small and large calls side by side."""
    import torch
    banks = [Case(T, 512, 320, 8, 2, seed=T) for T in (1500, 2300, 3, 70)]
    want = [c.run() for c in banks]
    streams, outs = [torch.cuda.Stream() for _ in banks], [torch.zeros_like(w) for w in want]
    torch.cuda.synchronize()
    for _ in range(10):
        for c, st, o in zip(banks, streams, outs):
            c.run(o, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert binding.matmul_status() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 300])
def test_an_expert_is_swapped_in_place(T):
    """Weights are not copied: what is written into a slot between two calls, on the same stream, is what the next call multiplies."""
    import torch
    c = Case(T, 192, 256, 6, 2)
    c.check(c.run())
    for e in (1, 4):
        c.w_in[e].copy_(torch.randint(-127, 128, c.w_in[e].shape, device="cuda").to(torch.int8))
        c.in_scales[e].mul_(0.5)
        c.w_out[e].neg_()
        out = c.run()
        c.check(out)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 45, 1200])
def test_a_served_block(T):
    """Norms around the block, the router's product, routing to resident experts, experts, and the shared projection with its adapters,
    as a server strings them together; each step against the plain formula on what the step before left."""
    import torch
    d, F, E, S, k = 512, 320, 32, 12, 2
    c = Case(T, d, F, S, k)
    gen = torch.Generator(device="cuda").manual_seed(T)
    normal = lambda *s, std=1.0: torch.empty(*s, device="cuda").normal_(0.0, std, generator=gen)  # noqa: E731
    x, stream, w, pw = normal(T, d).bfloat16(), normal(T, d, std=2.0), normal(d).bfloat16(), normal(d).bfloat16()
    n8, ns = torch.empty(T, d, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    before = stream.clone()
    binding.block_norm(x, stream, w, 1e-6, residual_out=stream, post_weight=pw, scale=0.5, out8=n8, scales=ns)
    x64 = x.double()
    h = before.double() + 0.5 * x64 * pw.double() / torch.sqrt((x64 * x64).mean(1, keepdim=True) + 1e-6)
    y = h * w.double() / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6)
    assert bool(((n8.double() * ns.double()[:, None] - y).abs() <= (0.5 + 1e-3) * y.abs().amax(1, keepdim=True) / 127.0).all())
    # router: its weights quantised the same way
    wr, wr8, wrs = normal(E, d, std=d ** -0.5), torch.empty(E, d, dtype=torch.int8, device="cuda"), torch.empty(E, device="cuda")
    binding.quantize_rows(wr, wr8, wrs)
    logits = torch.empty(T, E, device="cuda")
    binding.matmul_scaled(n8, ns, wr8, wrs, logits)
    table = torch.full((E,), -1, dtype=torch.int32, device="cuda")
    table[torch.randperm(E, device="cuda", generator=gen)[:S]] = torch.arange(S, dtype=torch.int32, device="cuda")
    experts, weights, slots = (torch.empty(T, k, dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.int32))
    binding.route(binding.Gate(renorm=True), logits, experts, weights, expert_to_slot=table, slots=slots)
    c.x, c.xs, c.slots, c.weights = n8, ns, slots, weights
    out = c.run()
    c.check(out)
    # the projection that all tokens share, and each token's adapter beside it
    wp8, wps = _int8(d, d, gen, d ** -0.5)
    shared = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    binding.matmul_scaled(n8, ns, wp8, wps, shared)
    want = (n8.double() @ wp8.double().t()) * ns.double()[:, None] * wps.double()
    assert bool(((shared.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want.abs()).all())
    n16 = (n8.float() * ns[:, None]).bfloat16()
    A, B, ids = normal(3, 8, d, std=d ** -0.5).bfloat16(), normal(3, d, 8, std=0.3).bfloat16(), torch.randint(-1, 3, (T,), device="cuda", generator=gen).to(torch.int32)
    bank = binding.AdapterBank(3, d, d, 8, binding.BF16, max_tokens=T)
    bank.set_weights(A, B)
    both = torch.empty_like(shared)
    bank.forward(n16, ids, shared, both)
    # and the next block's norms take what came out
    nxt, new = torch.empty_like(out), torch.empty_like(stream)
    total = (out.float() + both.float()).bfloat16()
    binding.block_norm(total, stream, w, 1e-6, out=nxt, residual_out=new, post_weight=pw)
    t64 = total.double()
    h = stream.double() + t64 * pw.double() / torch.sqrt((t64 * t64).mean(1, keepdim=True) + 1e-6)
    assert bool(((new.double() - h).abs() <= 1e-5 * (h.abs() + stream.double().abs())).all())
