"""A layer with a gate of its own, and the pre-norm block: norm, router, experts and adapters run together."""
import numpy as np
import pytest

from paper_2308_15030_b200 import binding, inputs as I
from paper_2308_15030_b200.binding import Gate


# ------------------------------------------------------------------ refusals (host checks, no GPU needed)
def test_null_handles():
    import ctypes
    L = binding.lib()
    g = Gate()
    assert L.swapmoe_set_gate(None, ctypes.byref(g), None) == -1
    assert L.swapmoe_set_norm(None, 256, 1e-6) == -1
    assert L.swapmoe_forward_block(None, 256, 256, 256, 1, None, None, None) == -1
    assert L.swapmoe_adapters_check(None, 64, 64, 1, 1) == -1


class _Tensor:
    """What the checks ask of a tensor; its address is never used, a refused call does not reach the library."""
    def __init__(self, shape, dtype, device):
        import torch
        self.shape, self.dtype, self.device, self.is_cuda = shape, dtype, torch.device(device), device.startswith("cuda")

    def numel(self):
        return int(np.prod(self.shape))

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 256


def _stand_in(cls, device, **cfg):
    import ctypes
    import types
    import torch
    obj = object.__new__(cls)
    obj._h, obj._device, obj._keep, obj.last_T = ctypes.c_void_p(), torch.device(device), {}, 0
    obj.cfg = types.SimpleNamespace(**cfg)
    return obj


@pytest.mark.parametrize("current", [0, 1])
def test_tensors_of_other_devices_are_refused(monkeypatch, current):
    """A layer on cuda:1 and operands on cuda:0 or the CPU, or a call while another device is current: refused before the library."""
    import torch
    calls = []

    class Library:
        swapmoe_status_string = staticmethod(lambda status: b"refused")

        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0
    monkeypatch.setattr(binding, "lib", Library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
    L = _stand_in(binding.Layer, "cuda:1", E=8, d_model=64, dtype=binding.BF16, max_tokens=4)
    bank = _stand_in(binding.AdapterBank, "cuda:1")
    far_bank = _stand_in(binding.AdapterBank, "cuda:0")
    there = dict(x=_Tensor((4, 64), torch.bfloat16, "cuda:1"), residual=_Tensor((4, 64), torch.bfloat16, "cuda:1"),
                 out=_Tensor((4, 64), torch.bfloat16, "cuda:1"), adapters=bank, ids=_Tensor((4,), torch.int32, "cuda:1"), stream=0)

    def refused(f, *a, **kw):
        with pytest.raises(binding.SwapMoEError) as e:
            f(*a, **kw)
        assert e.value.status == -1 and not calls
    for device in ("cuda:0", "cpu"):
        refused(L.set_gate, Gate(), _Tensor((8,), torch.float32, device))
        refused(L.set_norm, _Tensor((64,), torch.bfloat16, device), 1e-6)
        rows = {n: _Tensor((4, 64), torch.bfloat16, device) for n in ("x", "residual", "out")}
        refused(L.forward_block, **dict(there, **rows))
        for n, t in rows.items():
            refused(L.forward_block, **dict(there, **{n: t}))
        refused(L.forward_block, **dict(there, ids=_Tensor((4,), torch.int32, device)))
    refused(L.forward_block, **dict(there, adapters=far_bank))
    if current == 0:
        refused(L.forward_block, **there)
        refused(L.set_norm, _Tensor((64,), torch.bfloat16, "cuda:1"), 1e-6)
    else:
        L.forward_block(**there)
        L.set_norm(_Tensor((64,), torch.bfloat16, "cuda:1"), 1e-6)
        L.set_gate(Gate(), _Tensor((8,), torch.float32, "cuda:1"))
        assert calls == ["swapmoe_forward_block", "swapmoe_set_norm", "swapmoe_set_gate"]
        calls.clear()


# ------------------------------------------------------------------ on the GPU
def _expected(case, midx, mgate, slot):
    """out in 64 bits from a routing: gate-weighted sum of the experts' FFN, hidden values rounded as the layer stores them."""
    cfg = case.cfg
    x = case.x.astype(np.float64)
    out = np.zeros((case.T, cfg.d))
    for s in range(cfg.K):
        a_in, a_out = (a[case.phys[s]].astype(np.float64) for a in (case.a_in, case.a_out))
        for j in range(cfg.k):
            t = np.nonzero(slot[:, j] == s)[0]
            if t.size == 0:
                continue
            if cfg.act == I.ACT_SWIGLU:
                u = x[t] @ a_in[0].T
                h = u / (1 + np.exp(-u)) * (x[t] @ a_in[1].T)
            else:
                h = np.maximum(x[t] @ a_in[0].T, 0)
            h = I.store_round(h.astype(np.float32), cfg.dtype).astype(np.float64)
            out[t] += mgate[t, j, None].astype(np.float64) * (h @ a_out.T)
    return out


def _case(T, E, k, K, dtype=I.BF16, act=I.ACT_RELU, d=128, f=256, max_tokens=None):
    from harness import Case
    cfg = I.LayerConfig("block", dtype, T=T, d=d, f=f, E=E, k=k, K=K, act=act, renorm=0, seed=7)
    rng = np.random.default_rng(E + K)
    return Case(cfg, s2e=rng.permutation(E)[:K], max_tokens=max_tokens)


GATES = [Gate("sigmoid", 8, 4, 2, True, 2.5), Gate("softmax", 4, 2, 1, False, 16.0), Gate("sigmoid")]


@pytest.mark.gpu
@pytest.mark.parametrize("gate", range(len(GATES)))
@pytest.mark.parametrize("T,E,k,K,dtype,act", [(1, 64, 2, 9, I.BF16, I.ACT_RELU), (5, 64, 1, 16, I.BF16, I.ACT_RELU),
                                               (64, 256, 4, 33, I.BF16, I.ACT_SWIGLU), (100, 160, 3, 20, I.F32, I.ACT_RELU),
                                               (4097, 64, 2, 12, I.BF16, I.ACT_RELU), (8300, 16, 1, 5, I.BF16, I.ACT_RELU),
                                               (9000, 16, 2, 5, I.F32, I.ACT_SWIGLU)])
def test_gate_of_its_own(T, E, k, K, dtype, act, gate):
    import torch
    import oracle
    from harness import TOL_IMP_REL, TOL_OUT
    from test_route_groups import REL, TINY, reference
    g = GATES[gate]
    case = _case(T, E, k, K, dtype, act)
    L = case.layer
    bias = np.random.default_rng(1).normal(0, 0.1, E).astype(np.float32) if g.score == 1 else None
    L.set_gate(g, None if bias is None else torch.from_numpy(bias).cuda())
    out = case.run()
    assert L.device_status() == (0, 0)
    lg = L.tap("logits")
    table = np.full(E, -1, np.int32)
    table[case.s2e] = np.arange(K)
    args = (k, "sigmoid" if g.score else "softmax", g.n_groups, g.topk_groups, g.group_top, g.renorm, g.scale, bias)
    ue, uw, _ = reference(lg, *args)
    me, mw, ms = reference(lg, *args, table)
    assert np.array_equal(L.tap("uidx"), ue) and np.array_equal(L.tap("midx"), me) and np.array_equal(L.tap("slot"), ms)
    for name, w in (("ugate", uw), ("mgate", mw)):
        assert np.all(np.abs(L.tap(name) - w) <= REL * np.abs(w) + TINY), name
    count, offset, perm, inv = oracle.permute(ms.astype(np.int32), K)
    for name, want in (("count", count), ("offset", offset), ("perm", perm), ("inv", inv)):
        assert np.array_equal(L.tap(name), want.reshape(L.tap(name).shape)), name
    xn = np.linalg.norm(case.x.astype(np.float64), axis=1)[:, None]
    imp, cnt, mimp = np.zeros(E), np.zeros(E), np.zeros(E)
    np.add.at(imp, ue, xn * np.abs(uw) * case.enorm[ue])
    np.add.at(cnt, ue, 1)
    np.add.at(mimp, me, xn * np.abs(mw) * case.enorm[me])
    assert np.max(np.abs(L.read_importance() - imp)) <= TOL_IMP_REL * imp.max()
    assert np.array_equal(L.read_score("count"), cnt)
    assert np.max(np.abs(L.read_score("eq1_masked") - mimp)) <= TOL_IMP_REL * mimp.max()
    ref = _expected(case, me, mw, ms)
    assert np.max(np.abs(out - ref)) <= TOL_OUT[dtype] * np.max(np.abs(ref))
    assert np.array_equal(case.run(), out)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 300])
def test_back_to_the_configurations_gate(T):
    case = _case(T, 32, 2, 8)
    L = case.layer
    first = case.run()
    names = ("uidx", "midx", "slot", "ugate", "mgate", "perm")
    taps = {n: L.tap(n) for n in names}
    L.set_gate(Gate("softmax"))                              # the configuration's gate, by the other kernel
    out = case.run()
    for n in names[:3]:
        assert np.array_equal(L.tap(n), taps[n]), n
    for n in names[3:5]:
        assert np.max(np.abs(L.tap(n) - taps[n])) <= 1e-6, n
    assert np.max(np.abs(out - first)) <= 2e-2 * np.max(np.abs(first))
    L.set_gate(Gate("sigmoid", 4, 2, 2, True))
    assert not np.array_equal(case.run(), first)
    L.set_gate(None)
    assert np.array_equal(case.run(), first)


def _block_inputs(case, dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(case.T)
    dt = torch.bfloat16 if dtype == I.BF16 else torch.float32
    T, d = case.T, case.cfg.d
    x = torch.empty(T, d, device="cuda").normal_(generator=gen).to(dt)
    r = torch.empty(T, d, device="cuda").normal_(0, 2, generator=gen).to(dt)
    w = torch.empty(d, device="cuda").normal_(1, 0.2, generator=gen).to(dt)
    A = torch.empty(5, 16, d, device="cuda").normal_(0, d ** -0.5, generator=gen).to(dt)
    B = torch.empty(5, d, 16, device="cuda").normal_(0, 0.25, generator=gen).to(dt)
    sc = torch.empty(5, device="cuda").uniform_(0.5, 1.5, generator=gen)
    ids = torch.randint(-1, 5, (T,), device="cuda", generator=gen).to(torch.int32)
    bank = binding.AdapterBank(5, d, d, 16, dtype, max_tokens=T)
    bank.set_weights(A, B, sc)
    return x, r, w, bank, ids


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [I.BF16, I.F32])
@pytest.mark.parametrize("own_gate", [False, True])
@pytest.mark.parametrize("T", [1, 3, 40, 500])
def test_block_is_its_parts(T, own_gate, dtype):
    import torch
    case = _case(T, 64, 2, 12, dtype)
    L = case.layer
    if own_gate:
        L.set_gate(Gate("sigmoid", 8, 4, 2, True, 2.5))
    x, r, w, bank, ids = _block_inputs(case, dtype)
    n, r1, want = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    binding.rms_norm(x, w, 1e-5, out=n, residual=r, residual_out=r1)
    L.forward(n, want)
    bank.forward(n, ids, want, want)
    L.set_norm(w, 1e-5)
    r2, out = r.clone(), torch.empty_like(x)
    L.forward_block(x, r2, out, bank, ids)
    torch.cuda.synchronize()
    assert torch.equal(r2, r1) and torch.equal(out, want)
    # without adapters, without a residual
    binding.rms_norm(x, w, 1e-5, out=n)
    L.forward(n, want)
    L.forward_block(x, None, out)
    assert torch.equal(out, want)
    assert L.device_status() == (0, 0)


@pytest.mark.gpu
def test_block_captured_and_on_another_stream():
    import torch
    case = _case(48, 64, 2, 12)
    L = case.layer
    L.set_gate(Gate("sigmoid", 8, 4, 2, True, 2.5))
    x, r, w, bank, ids = _block_inputs(case, I.BF16)
    L.set_norm(w, 1e-5)
    r1, want = r.clone(), torch.empty_like(x)
    L.forward_block(x, r1, want, bank, ids)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r2, out = r.clone(), torch.empty_like(x)
    side.wait_stream(torch.cuda.current_stream())
    L.forward_block(x, r2, out, bank, ids, stream=side)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(r2, r1)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.forward_block(x, r2, out, bank, ids)
        L.forward_block(out, r2, torch.empty_like(out), bank, ids)
    r2.copy_(r)
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.gpu
def test_block_refusals():
    import torch
    case = _case(8, 64, 2, 12)
    L, lib = case.layer, binding.lib()
    x, r, w, bank, ids = _block_inputs(case, I.BF16)
    out = torch.full_like(x, 3.0)

    def status(*a, **k):
        with pytest.raises(binding.SwapMoEError) as e:
            L.forward_block(*a, **k)
        return e.value.status
    assert status(x, r, out) == -2                             # no norm yet
    L.set_norm(w, 1e-5)
    for bad in (w[:64], w.float(), w.cpu()):
        with pytest.raises(binding.SwapMoEError):
            L.set_norm(bad, 1e-5)
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(binding.SwapMoEError):
            L.set_norm(w, eps)
    assert status(x, r, out, bank) == -1 and status(x, r, out, None, ids) == -1
    assert status(x, r, out, bank, ids.long()) == -1
    assert status(x, r, out, n_tokens=9) == -3
    small = binding.AdapterBank(5, 128, 128, 16, binding.BF16, max_tokens=4)
    assert status(x, r, out, small, ids) == -2                 # no weights
    other = binding.AdapterBank(5, 128, 64, 16, binding.BF16, max_tokens=8)
    assert status(x, r, out, other, ids) == -1
    keep = r.clone()
    torch.cuda.synchronize()
    assert bool((out == 3).all()) and torch.equal(r, keep)     # refused calls enqueue nothing
    L.forward_block(x, r, out, n_tokens=0)
    for g, b in ((Gate("softmax", 7), None), (Gate("softmax", 64, 1), None), (None, torch.zeros(64, device="cuda")),
                 (Gate(), torch.zeros(63, device="cuda")), (Gate(), torch.zeros(64))):
        with pytest.raises(binding.SwapMoEError) as e:
            L.set_gate(g, b)
        assert e.value.status == -1


@pytest.mark.gpu
def test_decode_stack_over_layers_with_gates_of_their_own():
    import torch
    from paper_2308_15030_b200.decode import DecodeStack, LayerState
    cases = [_case(6, 32, 2, 8) for _ in range(2)]
    states = []
    for c in cases:
        c.layer.set_gate(Gate("sigmoid", 4, 2, 2, True))
        host = [torch.empty((32,) + tuple(a.shape[1:]), dtype=torch.bfloat16).pin_memory() for a in (c.d_in, c.d_out_w)]
        states.append(LayerState(c.layer, np.asarray(c.s2e, np.int32), c.phys, [], c.d_in, c.d_out_w, host[0], host[1], enorm=c.enorm))
    x = torch.stack([c.d_x for c in cases])
    want = []
    for c in cases:
        o = torch.empty_like(c.d_x)
        c.layer.forward(c.d_x, o)
        want.append(o)
    out = torch.empty_like(x)
    stack = DecodeStack(states, frequency=100, graph_buffers=(torch.empty_like(x), out))
    stack.step_graph(x)
    torch.cuda.synchronize()
    assert torch.equal(out, torch.stack(want))


@pytest.mark.gpu
def test_block_refuses_rows_that_are_not_its_own():
    import torch
    case = _case(8, 64, 2, 12)
    L = case.layer
    x, r, w, bank, ids = _block_inputs(case, I.BF16)
    L.set_norm(w, 1e-5)
    out, keep = torch.full_like(x, 3.0), r.clone()
    wide = torch.zeros(x.shape[0], 2 * x.shape[1], dtype=x.dtype, device="cuda")[:, :x.shape[1]]
    for bad in (x.float(), x.cpu(), wide, x[:7]):
        for args in ((bad, r, out), (x, bad, out), (x, r, bad)):
            with pytest.raises(binding.SwapMoEError) as e:
                L.forward_block(*args, n_tokens=8)
            assert e.value.status == -1
    torch.cuda.synchronize()
    assert bool((out == 3).all()) and torch.equal(r, keep)


@pytest.mark.gpu
@pytest.mark.parametrize("E,G,tg,k", [(160, 8, 3, 4), (256, 8, 4, 4), (64, 4, 2, 3)])
def test_gate_over_groups_at_minus_infinity(E, G, tg, k):
    """Both selections of a layer with a gate of its own, logits and biases with groups switched off."""
    import torch
    from test_route_groups import REL, TINY, dead_biases, dead_logits, reference
    rng = np.random.default_rng(E)
    lg = dead_logits(rng, E, G)
    K = 24
    case = _case(len(lg), E, k, K)
    L = case.layer
    table = np.full(E, -1, np.int32)
    table[case.s2e] = np.arange(K)
    plain = rng.normal(0, 1.5, lg.shape).astype(np.float32)
    runs = [(Gate("softmax", G, tg, 1, True), None, lg), (Gate("sigmoid", G, tg, 2, False, 2.5), None, lg)]
    runs += [(Gate("sigmoid", G, tg, 2, True), bias, plain) for bias in dead_biases(rng, E, G)]
    for g, bias, logits in runs:
        L.set_gate(g, None if bias is None else torch.from_numpy(bias).cuda())
        L.forward_from_logits(case.d_x, torch.from_numpy(logits).cuda(), case.d_out)
        args = (k, "sigmoid" if g.score else "softmax", g.n_groups, g.topk_groups, g.group_top, g.renorm, g.scale, bias)
        ue, uw, _ = reference(logits, *args)
        me, mw, ms = reference(logits, *args, table)
        assert np.array_equal(L.tap("uidx"), ue)
        assert np.array_equal(L.tap("midx"), me) and np.array_equal(L.tap("slot"), ms)
        for name, w in (("ugate", uw), ("mgate", mw)):
            assert np.all(np.abs(L.tap(name) - w) <= REL * np.abs(w) + TINY), name


@pytest.mark.gpu
@pytest.mark.parametrize("T,own", [(3, 1), (300, 1), (2100, 2)])
def test_the_blocks_launches_are_counted(T, own):
    """The norm is one kernel, the adapters one, or two where a kernel groups many tokens by adapter first."""
    import torch
    case = _case(T, 64, 2, 12)
    L = case.layer
    x, r, w, bank, ids = _block_inputs(case, I.BF16)
    out = torch.empty_like(x)
    L.set_norm(w, 1e-5)

    def launches(f, *a):
        before = L.launch_count
        f(*a)
        return L.launch_count - before
    layer = launches(L.forward, x, out)
    assert launches(L.forward_block, x, r, out) == layer + 1
    assert launches(L.forward_block, x, r, out, bank, ids) == layer + 1 + own
    with pytest.raises(binding.SwapMoEError):
        L.forward_block(x, r, out, bank, ids.long())
    assert launches(L.forward_block, x, r, out, None, None, 0) == 0


DEPENDENT_EDGES = """
import ctypes
import sys
sys.path[:0] = ["tests", "."]
import torch
from paper_2308_15030_b200 import binding, inputs as I
from test_block import Gate, _block_inputs, _case


class Edge(ctypes.Structure):
    _fields_ = [(n, ctypes.c_ubyte) for n in ("from_port", "to_port", "type")] + [("reserved", ctypes.c_ubyte * 5)]


runtime = ctypes.CDLL(next(line.split()[-1] for line in open("/proc/self/maps") if "libcudart" in line))


def edges(f):
    f()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(g):
        f()
    h, n = ctypes.c_void_p(g.raw_cuda_graph()), ctypes.c_size_t(0)
    assert runtime.cudaGraphGetEdges_v2(h, None, None, None, ctypes.byref(n)) == 0 and n.value > 0
    ends, data = [(ctypes.c_void_p * n.value)() for _ in range(2)], (Edge * n.value)()
    assert runtime.cudaGraphGetEdges_v2(h, ends[0], ends[1], data, ctypes.byref(n)) == 0
    return sum(e.type == 1 for e in data)                    # cudaGraphDependencyTypeProgrammatic


T = 2100
case = _case(T, 64, 2, 12)
L = case.layer
x, r, w, bank, ids = _block_inputs(case, I.BF16)
out = torch.empty_like(x)
L.set_norm(w, 1e-5)
lg, e, wt = torch.zeros(T, 64, device="cuda"), torch.empty(T, 2, dtype=torch.int32, device="cuda"), torch.empty(T, 2, device="cuda")


def twice(f):
    return lambda: (f(), f())


got = [edges(twice(lambda: binding.rms_norm(x, w, 1e-5, out=out))), edges(twice(lambda: binding.route(Gate(), lg, e, wt))),
       edges(twice(lambda: bank.forward(x, ids, x, out))), edges(lambda: L.forward_block(x, r, out, bank, ids))]
print("EDGES", *got)
"""


@pytest.mark.gpu
@pytest.mark.parametrize("switch", ["0", "1"])
def test_dependent_launches_follow_the_switch(switch):
    """SWAPMOE_PDL=0: no kernel of these calls is launched before the one in front of it has ended."""
    import os
    import subprocess
    import sys
    import torch
    if not hasattr(torch.cuda.CUDAGraph, "raw_cuda_graph"):
        pytest.skip("no access to the captured graph")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", DEPENDENT_EDGES], cwd=root, env=dict(os.environ, SWAPMOE_PDL=switch),
                         capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
    got = [int(v) for v in run.stdout.split("EDGES")[1].split()]
    assert got == [0, 0, 0, 0] if switch == "0" else all(n > 0 for n in got), got


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,size", [(I.BF16, 2), (I.F32, 4)])
def test_the_rows_behind_the_norm_count_as_workspace(dtype, size):
    import torch
    case = _case(8, 16, 2, 6, dtype, max_tokens=40)
    L = case.layer
    x, r, w, bank, ids = _block_inputs(case, dtype)
    before = L.workspace_bytes
    for _ in range(2):                                       # allocated once
        L.set_norm(w, 1e-5)
        assert L.workspace_bytes == before + 40 * 128 * size
