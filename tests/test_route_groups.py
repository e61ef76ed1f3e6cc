"""Routing by groups of experts (softmax or sigmoid scores, balance bias, top-k, weights) against the definition in 64 bits."""
import ctypes

import numpy as np
import pytest

from paper_2308_15030_b200 import binding
from paper_2308_15030_b200.binding import Gate


# ------------------------------------------------------------------ refusals (host checks, no GPU needed)
def _call(gate=None, T=2, E=64, k=2, stride=64, logits=256, bias=None, table=None, experts=256, weights=256, slots=None):
    g = Gate() if gate is None else gate
    return binding.lib().swapmoe_route(ctypes.byref(g), logits, stride, bias, table, T, E, k, experts, weights, slots, None)


def _gate(**kw):
    g = Gate("sigmoid", 8, 4, 2, True, 2.5)
    for n, v in kw.items():
        setattr(g, n, v)
    return g


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), -1), (dict(E=0), -1), (dict(k=0), -1), (dict(k=65), -1), (dict(stride=63), -1), (dict(E=513, stride=513), -7),
    (dict(k=17), -7), (dict(logits=None), -1), (dict(experts=None), -1), (dict(weights=None), -1), (dict(slots=256), -1),
    (dict(table=256), -1), (dict(logits=258), -1), (dict(bias=2), -1), (dict(gate=_gate(score=2)), -1),
    (dict(gate=_gate(n_groups=0)), -1), (dict(gate=_gate(n_groups=7)), -1), (dict(gate=_gate(n_groups=64)), -1),
    (dict(gate=_gate(topk_groups=0)), -1), (dict(gate=_gate(topk_groups=9)), -1), (dict(gate=_gate(group_top=3)), -1),
    (dict(gate=_gate(group_top=0)), -1), (dict(gate=_gate(renorm=2)), -1), (dict(gate=_gate(scale=float("inf"))), -1),
    (dict(gate=_gate(topk_groups=1), k=9), -1)])
def test_refusals(kw, status):
    assert _call(**kw) == status


def test_no_gate_and_no_tokens():
    assert binding.lib().swapmoe_route(None, 256, 64, None, None, 2, 64, 2, 256, 256, None, None) == -1
    assert _call(T=0, logits=None) == 0
    with pytest.raises(binding.SwapMoEError):
        Gate("tanh")


def test_tensor_checks():
    import torch
    lg, e, w = torch.zeros(3, 8), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2)
    for a, kw in (((lg.bfloat16(), e, w), {}), ((lg, e.long(), w), {}), ((lg, e, w.double()), {}), ((lg, e, w[:2]), {}),
                  ((lg, e, w), dict(bias=torch.zeros(7))), ((lg, e, w), dict(expert_to_slot=torch.zeros(8, dtype=torch.int32))),
                  ((lg, e, w), dict(slots=e)), ((lg.t(), e, w), {}), ((lg, e, w), {})):                # the last: not on a GPU
        with pytest.raises(binding.SwapMoEError) as err:
            binding.route(Gate(), *a, **kw)
        assert err.value.status == -1


# ------------------------------------------------------------------ the definition, one token at a time
def reference(logits, k, score, n_groups, topk_groups, group_top, renorm, scale, bias=None, table=None):
    """(experts, weights, slots) of float32 logits [T, E], in 64 bits."""
    T, E = logits.shape
    size = E // n_groups
    l = logits.astype(np.float64)
    l[np.isnan(l)] = -np.inf
    allowed = [e for e in range(E) if table is None or table[e] >= 0]
    experts, weights = np.full((T, k), -1, np.int64), np.zeros((T, k))
    for t in range(T):
        if not allowed:
            continue
        top = max(l[t, e] for e in allowed)
        if score == "softmax":
            raw = {e: 1.0 if l[t, e] == top else float(np.exp(l[t, e] - top)) for e in allowed}
            total = sum(raw.values())
            s = {e: v / total for e, v in raw.items()}
        else:
            with np.errstate(over="ignore"):
                s = {e: float(1.0 / (1.0 + np.exp(-l[t, e]))) for e in allowed}
        if bias is None and (n_groups == 1 or group_top == 1):
            c = {e: l[t, e] for e in allowed}                # the same order, without the scores' rounding
        else:
            c = {e: s[e] + (0.0 if bias is None else float(bias[e])) for e in allowed}
        c = {e: -np.inf if np.isnan(v) else v for e, v in c.items()}
        groups = {}
        for e in allowed:
            groups.setdefault(e // size, []).append(e)
        value = {g: sum(sorted((c[e] for e in m), reverse=True)[:group_top]) for g, m in groups.items()}
        pool, taken = [], 0
        for g in sorted(groups, key=lambda g: (-value[g], g)):
            if taken >= topk_groups and len(pool) >= k:
                break
            pool += groups[g]
            taken += 1
        best = sorted(pool, key=lambda e: (-c[e], e))[:k]
        if renorm:
            m = max(l[t, e] for e in best)
            if score == "softmax":
                w = [1.0 if l[t, e] == m else float(np.exp(l[t, e] - m)) for e in best]
            else:
                sh = min(m, 0.0)
                w = [(1.0 if l[t, e] == sh else float(np.exp(l[t, e] - sh))) / (1.0 + float(np.exp(l[t, e]))) if m < 0 else s[e] for e in best]
            w = [v / sum(w) for v in w]
        else:
            w = [s[e] for e in best]
        experts[t, :len(best)] = best
        weights[t, :len(best)] = [v * scale for v in w]
    slots = np.where(experts >= 0, np.asarray(table)[np.maximum(experts, 0)], -1) if table is not None else None
    return experts, weights, slots


# fp32 weights: exponentials and reciprocals of a few units in the last place each, arguments rounded to 2^-24 of at most ~100,
# sums of up to 512 terms in trees of depth 16 + 5: well under 1e-5 of the value; below 1e-37 fp32 has no full precision left.
REL, TINY = 1e-5, 1e-36


def _check(logits, k, gate, bias=None, table=None, stride=None):
    import torch
    T, E = logits.shape
    stride = stride or E
    lg = torch.full((T, stride), 9.0, device="cuda")
    lg[:, :E] = torch.from_numpy(logits)
    experts = torch.full((T + 1, k), -7, dtype=torch.int32, device="cuda")
    weights = torch.full((T + 1, k), 7.0, device="cuda")
    slots = None if table is None else torch.full((T + 1, k), -7, dtype=torch.int32, device="cuda")
    cuda = lambda a, dt: None if a is None else torch.from_numpy(np.ascontiguousarray(a, dt)).cuda()    # noqa: E731
    binding.route(Gate(*gate), lg[:, :E], experts[:T], weights[:T], bias=cuda(bias, np.float32),
                  expert_to_slot=cuda(table, np.int32), slots=None if slots is None else slots[:T])
    torch.cuda.synchronize()
    score, G, tg, gt, renorm, scale = gate
    e, w, s = reference(logits, k, score, G, tg, gt, renorm, scale, bias, table)
    assert np.array_equal(experts[:T].cpu().numpy(), e)
    got = weights[:T].cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - w) <= REL * np.abs(w) + TINY), np.max(np.abs(got - w))
    assert bool((experts[T] == -7).all()) and bool((weights[T] == 7.0).all())
    if s is not None:
        assert np.array_equal(slots[:T].cpu().numpy(), s) and bool((slots[T] == -7).all())


def _table(rng, E, K):
    t = np.full(E, -1, np.int32)
    t[rng.permutation(E)[:K]] = rng.permutation(K)
    return t


SHAPES = [(1, 1, 1, 1), (4, 1, 1, 3), (8, 2, 1, 3), (64, 1, 1, 2), (64, 4, 2, 8), (160, 8, 3, 6), (256, 8, 4, 8), (256, 32, 32, 16),
          (40, 4, 4, 7), (256, 1, 1, 16), (384, 1, 1, 8), (512, 16, 5, 8), (500, 4, 2, 5), (32, 32, 9, 9), (96, 3, 1, 4), (33, 11, 5, 5)]


@pytest.mark.gpu
@pytest.mark.parametrize("score,renorm", [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)])
@pytest.mark.parametrize("E,G,tg,k", SHAPES)
def test_against_the_definition(E, G, tg, k, score, renorm):
    rng = np.random.default_rng(E + 31 * G + k)
    for T, with_bias, resident, top in ((1, False, 0, 1), (37, True, 0, 2), (19, True, max(k, E // 5), 1), (130, False, max(k, E // 3), 2)):
        logits = rng.normal(0, 2, (T, E)).astype(np.float32)
        bias = rng.normal(0, 0.1, E).astype(np.float32) if with_bias else None
        table = _table(rng, E, resident) if resident else None
        _check(logits, k, (score, G, tg, top, renorm, 1.5), bias, table, stride=E + (T % 3))


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,G,tg,k,top", [(256, 8, 4, 8, 2), (160, 8, 3, 6, 2), (64, 1, 1, 4, 1), (64, 4, 2, 4, 1)])
def test_choices_closer_than_fp32_tells_apart(score, E, G, tg, k, top):
    """A bias that makes all choices of a token equal up to its own rounding: the order hangs on what fp32 scores lose."""
    rng = np.random.default_rng(5)
    base = rng.normal(0, 1, E).astype(np.float32)
    l = base.astype(np.float64)
    s = 1 / (1 + np.exp(-l)) if score == "sigmoid" else np.exp(l - l.max()) / np.exp(l - l.max()).sum()
    bias = (0.75 - s).astype(np.float32)
    logits = np.stack([base, base, rng.normal(0, 1, E).astype(np.float32)])
    for renorm in (False, True):
        _check(logits, k, (score, G, tg, top, renorm, 1.0), bias)


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("E,G,tg,k", [(64, 1, 1, 4), (64, 8, 3, 4), (160, 8, 2, 6), (256, 8, 4, 8)])
def test_ties_go_to_the_lowest_index(E, G, tg, k, score, with_bias):
    rng = np.random.default_rng(3)
    logits = rng.integers(-2, 3, (40, E)).astype(np.float32)
    logits[0] = 0.0
    logits[1] = -0.0
    logits[2, ::2] = -0.0
    logits[2, 1::2] = 0.0
    bias = (rng.integers(0, 2, E) * 0.5).astype(np.float32) if with_bias else None
    _check(logits, k, (score, G, tg, 1, True, 1.0), bias)
    _check(logits, k, (score, G, tg, 1, False, 1.0), bias, _table(rng, E, E // 2))


@pytest.mark.gpu
@pytest.mark.parametrize("score,renorm", [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)])
@pytest.mark.parametrize("G,tg", [(1, 1), (4, 2)])
def test_infinities_nan_and_far_scores(G, tg, score, renorm):
    rng = np.random.default_rng(9)
    logits = rng.normal(0, 1, (8, 32)).astype(np.float32)
    logits[0, :] = -np.inf
    logits[1, :] = np.nan
    logits[2, 5:] = -np.inf
    logits[3, 7] = np.nan
    logits[4, 9] = np.inf
    logits[5] -= 60.0
    logits[6] *= 40.0
    logits[7] = -3.4028235e38
    _check(logits, 4, (score, G, tg, 1, renorm, 1.0))
    _check(logits, 4, (score, G, tg, 1, renorm, 1.0), table=_table(rng, 32, 6))
    bias = np.zeros(32, np.float32)
    bias[0], bias[1] = np.nan, -np.inf
    _check(logits[2:7], 4, (score, G, tg, 2, False, 1.0), bias)


@pytest.mark.gpu
@pytest.mark.parametrize("K", [0, 1, 3])
@pytest.mark.parametrize("G,tg", [(1, 1), (8, 2)])
def test_fewer_experts_than_wanted(G, tg, K):
    rng = np.random.default_rng(K)
    logits = rng.normal(0, 1, (21, 64)).astype(np.float32)
    for renorm in (False, True):
        _check(logits, 4, ("softmax", G, tg, 1, renorm, 1.0), table=_table(rng, 64, K))
        _check(logits, 4, ("sigmoid", G, tg, 2, renorm, 1.0), rng.normal(0, 0.1, 64), _table(rng, 64, K))


@pytest.mark.gpu
def test_agrees_with_the_layers_own_gate():
    """Softmax, no groups, no bias: what swapmoe_route_static makes of the same logits."""
    from harness import Case
    from paper_2308_15030_b200 import inputs as I
    import torch
    for renorm in (0, 1):
        case = Case(I.LayerConfig("r", I.BF16, T=120, d=128, f=128, E=48, k=3, K=9, renorm=renorm, seed=2))
        case.run()
        L = case.layer
        lg = torch.from_numpy(L.tap("logits")).cuda()
        e2s = np.full(48, -1, np.int32)
        e2s[case.s2e] = np.arange(9)
        e, w, s = (torch.empty(120, 3, dtype=dt, device="cuda") for dt in (torch.int32, torch.float32, torch.int32))
        binding.route(Gate("softmax", renorm=bool(renorm)), lg, e, w, expert_to_slot=torch.from_numpy(e2s).cuda(), slots=s)
        assert np.array_equal(e.cpu().numpy(), L.tap("midx")) and np.array_equal(s.cpu().numpy(), L.tap("slot"))
        assert np.max(np.abs(w.cpu().numpy() - L.tap("mgate"))) < 1e-6
        binding.route(Gate("softmax", renorm=bool(renorm)), lg, e, w)
        assert np.array_equal(e.cpu().numpy(), L.tap("uidx")) and np.max(np.abs(w.cpu().numpy() - L.tap("ugate"))) < 1e-6


@pytest.mark.gpu
def test_captured_and_many_tokens():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(4)
    lg = torch.empty(5000, 128, device="cuda").normal_(generator=gen)
    e, w = torch.empty(5000, 6, dtype=torch.int32, device="cuda"), torch.empty(5000, 6, device="cuda")
    gate = Gate("sigmoid", 4, 2, 2, True, 1.0)
    binding.route(gate, lg, e, w)
    want = e.clone(), w.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.route(gate, lg, e, w)
    e.zero_(), w.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(e, want[0]) and torch.equal(w, want[1])
    small = torch.empty(1, 6, dtype=torch.int32, device="cuda"), torch.empty(1, 6, device="cuda")
    for t in (0, 77, 4999):                                  # a token's choice does not hang on its batch
        binding.route(gate, lg[t:t + 1], *small)
        assert torch.equal(small[0][0], want[0][t]) and torch.equal(small[1][0], want[1][t])


# ------------------------------------------------------------------ groups that -infinity switches off, several experts per lane
DEAD_SHAPES = [(160, 8, 3, 6), (256, 8, 4, 8), (96, 4, 2, 4), (64, 4, 2, 8), (512, 16, 5, 8), (200, 5, 2, 4), (240, 15, 4, 5)]


def dead_logits(rng, E, G, repeats=8):
    """Rows with whole groups, all of a group but one, or experts at random at -infinity or NaN."""
    size, rows = E // G, []
    for _ in range(repeats):
        l = rng.normal(0, 1.5, (9, E)).astype(np.float32)
        l[0, :size] = -np.inf
        l[1, (G - 1) * size:] = -np.inf
        l[2, size:3 * size] = np.nan
        l[3, size:2 * size], l[3, 3 * size:4 * size] = -np.inf, np.nan
        l[4, :(G - 1) * size] = -np.inf
        l[5, 2 * size + 1:3 * size] = -np.inf
        l[6, 2 * size:3 * size - 1] = np.nan
        l[7, rng.random(E) < 0.7] = -np.inf
        l[8, :size] = -3.4028235e38
        rows.append(l)
    return np.concatenate(rows)


def dead_biases(rng, E, G):
    """Biases of -infinity over runs of experts: those of one lane, all but one of a group, a group, some at random."""
    size, lane = E // G, -(-E // 32)
    for off in (slice(lane, 2 * lane), slice(size + 1, 2 * size), slice(size, 2 * size), rng.random(E) < 0.4):
        bias = rng.normal(0, 0.1, E).astype(np.float32)
        bias[off] = -np.inf
        yield bias


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("top", [1, 2])
@pytest.mark.parametrize("E,G,tg,k", DEAD_SHAPES)
def test_groups_at_minus_infinity(E, G, tg, k, top, score):
    rng = np.random.default_rng(E + top)
    logits = dead_logits(rng, E, G)
    for renorm in (False, True):
        _check(logits, k, (score, G, tg, top, renorm, 1.0))
        _check(logits, k, (score, G, tg, top, renorm, 1.0), table=_table(rng, E, E // 2))


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("top", [1, 2])
@pytest.mark.parametrize("E,G,tg,k", DEAD_SHAPES)
def test_biases_of_minus_infinity(E, G, tg, k, top, score):
    rng = np.random.default_rng(E + 7 * top)
    logits = rng.normal(0, 1.5, (200, E)).astype(np.float32)
    for bias in dead_biases(rng, E, G):
        _check(logits, k, (score, G, tg, top, True, 1.0), bias)
        _check(logits, k, (score, G, tg, top, False, 2.5), bias, _table(rng, E, 2 * E // 3))
