"""Operators around the experts of a served MoE block, as measurable cases.

``norm``      the residual's addition and the root-mean-square norm in front of a layer, rows out in the layer's dtype, in 8 bits
              (e4m3) with scales, or both
``route``     routing from logits: softmax or sigmoid scores, a bias that balances the experts' load, groups of experts, top-k,
              renormalised weights; with a slot table only resident experts are chosen
``adapters``  low-rank adapters of many requests beside a projection that all of them share: out = y + scale * B (A x), every
              token with the adapter of its request

With ``own`` false a pass computes the operator in elementary torch operations, else it calls the library.
Widths and expert counts are those of ``inputs.CONFIGS`` and of the tests' ranges, with ragged ones between them.
"""
import torch

own = False


# ------------------------------------------------------------------ cases
def _norm(T, d, dtype="bf16", residual=True, wide=False, out=True, out8=False, group=0, pad=0):
    return {"op": "norm", "T": T, "d": d, "dtype": dtype, "residual": residual, "wide": wide, "out": out, "out8": out8,
            "group": group, "pad": pad}


def _route(T, E, k, score="softmax", bias=False, groups=1, topk_groups=1, group_top=1, renorm=True, scale=1.0, resident=0):
    return {"op": "route", "T": T, "E": E, "k": k, "score": score, "bias": bias, "groups": groups, "topk_groups": topk_groups,
            "group_top": group_top, "renorm": renorm, "scale": scale, "resident": resident}


def _adapters(T, d, n, r, count, dtype="bf16", x8=False, run=1, none=0.1):
    return {"op": "adapters", "T": T, "d": d, "n": n, "r": r, "count": count, "dtype": dtype, "x8": x8, "run": run, "none": none}


def listed():
    return [
        # One user's decode step: the smallest call, all latency.
        dict(_norm(1, 4096), name="norm_1"),
        # A decode batch whose rows go to an 8-bit projection (one scale per row) and, in bf16, to the experts.
        dict(_norm(61, 1024, out8=True), name="norm_8bit_61"),
        # Single precision, a width that is no multiple of anything, rows inside wider ones.
        dict(_norm(1531, 1003, dtype="fp32", pad=21), name="norm_fp32_1531"),
        # Prefill of a wide block, the residual stream kept in fp32, 8-bit rows with a scale per 128 columns.
        dict(_norm(16384, 4096, wide=True, out=False, out8=True, group=128), name="norm_16384"),
        # A few streams of a 64-expert layer, all experts in one group.
        dict(_route(3, 64, 2), name="route_3"),
        # A full decode batch: sigmoid scores with a balance bias, eight groups, only resident experts may serve.
        dict(_route(64, 256, 4, score="sigmoid", bias=True, groups=8, topk_groups=4, group_top=2, scale=2.5, resident=48),
             name="route_resident_64"),
        # Prefill: softmax scores, ragged group size, groups by their best expert, weights as they are.
        dict(_route(6011, 160, 6, groups=8, topk_groups=3, renorm=False, scale=16.0), name="route_6011"),
        # The largest prefill of a many-expert layer.
        dict(_route(16384, 256, 8, score="sigmoid", bias=True, groups=8, topk_groups=4, group_top=2, scale=2.5),
             name="route_16384"),
        # One user's decode step beside a small projection.
        dict(_adapters(1, 1024, 1024, 16, 8, none=0.0), name="adapters_1"),
        # A few dozen users with adapters of their own; the shared projection reads 8-bit rows, so the adapters do too.
        dict(_adapters(61, 4096, 4096, 16, 64, x8=True), name="adapters_8bit_61"),
        # Single precision, ragged widths, short runs of tokens per request.
        dict(_adapters(1531, 768, 2240, 8, 12, dtype="fp32", run=50), name="adapters_fp32_1531"),
        # Prefill of sixteen sequences of 512 tokens, an adapter of a larger rank each.
        dict(_adapters(8192, 4096, 4096, 64, 16, run=512, none=0.05), name="adapters_8192"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() + rng.random()))


WIDTHS = [512, 704, 768, 960, 1024, 1536, 2048, 4096]


def draw(rng):
    op = rng.choice(["norm", "route", "adapters"])
    if op == "norm":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        d = rng.choice(WIDTHS + [_log_int(rng, 64, 4096)])
        form = rng.choice(["out", "out8", "both"])
        return _norm(_log_int(rng, 1, 12000), d, dtype, residual=rng.random() < 0.8, wide=dtype == "bf16" and rng.random() < 0.3,
                     out=form != "out8", out8=form != "out", group=rng.choice([0, 128]), pad=rng.choice([0, 0, 8, 21]))
    if op == "route":
        groups, size = rng.choice([(1, 8), (1, 64), (1, 256), (4, 16), (8, 20), (8, 32), (4, 10), (16, 16), (2, 60)])
        E = groups * size
        k = rng.randint(1, min(8, size))
        sigmoid = rng.random() < 0.5
        topk_groups = rng.randint(1, groups)
        return _route(_log_int(rng, 1, 16384), E, k, "sigmoid" if sigmoid else "softmax", bias=sigmoid or rng.random() < 0.2,
                      groups=groups, topk_groups=topk_groups, group_top=rng.choice([1, 2]), renorm=rng.random() < 0.7,
                      scale=rng.choice([1.0, 2.5]), resident=0 if rng.random() < 0.6 else rng.randint(k, min(E, 64)))
    d, n = rng.choice(WIDTHS), rng.choice(WIDTHS + [1088, 2240])
    r = rng.choice([8, 16, 16, 32, 40, 64])
    if rng.random() < 0.5:
        return _adapters(_log_int(rng, 1, 256), d, n, r, rng.randint(1, 64), "bf16", x8=rng.random() < 0.3, run=1,
                         none=rng.choice([0.0, 0.1, 0.5]))
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    return _adapters(_log_int(rng, 64, 2500 if dtype == "fp32" else 6000), d, n, r, rng.randint(1, 24), dtype,
                     x8=dtype == "bf16" and rng.random() < 0.3, run=rng.choice([1, 37, 200, 512]), none=rng.choice([0.0, 0.1]))


# ------------------------------------------------------------------ inputs
EPS = 1e-6


class _State:
    pass


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _rows(T, d, dtype, gen, std=1.0, pad=0):
    """T rows of d normal values, with `pad` more columns behind each that belong to somebody else."""
    return torch.empty(T, d + pad, device="cuda").normal_(0.0, std, generator=gen).to(dtype)[:, :d]


def _norm_inputs(case, gen, s):
    T, d, dt = case["T"], case["d"], _dtype(case)
    s.x = _rows(T, d, dt, gen, pad=case["pad"])
    s.residual = None
    if case["residual"]:
        # a residual stream has grown over the layers, a few of its channels more than the others
        s.residual = torch.empty(T, d, device="cuda").normal_(0.0, 2.0, generator=gen)
        s.residual[:, :: max(1, d // 7)] *= 12.0
        s.residual = s.residual.to(torch.float32 if case["wide"] else dt)
    s.weight = torch.empty(d, device="cuda").normal_(1.0, 0.2, generator=gen).to(dt)


def _route_inputs(case, gen, s):
    T, E = case["T"], case["E"]
    s.logits = torch.empty(T, E, device="cuda").normal_(0.0, 1.5, generator=gen)
    s.logits += torch.empty(E, device="cuda").normal_(0.0, 0.7, generator=gen)          # some experts are asked for more
    s.bias = torch.empty(E, device="cuda").normal_(0.0, 0.05, generator=gen) if case["bias"] else None
    s.expert_to_slot = None
    if case["resident"]:
        resident = torch.randperm(E, device="cuda", generator=gen)[: case["resident"]]
        s.expert_to_slot = torch.full((E,), -1, dtype=torch.int32, device="cuda")
        s.expert_to_slot[resident] = torch.arange(case["resident"], dtype=torch.int32, device="cuda")


def _adapters_inputs(case, gen, s):
    T, d, n, r, count, dt = case["T"], case["d"], case["n"], case["r"], case["count"], _dtype(case)
    s.x = _rows(T, d, dt, gen)
    s.x_scales = None
    if case["x8"]:
        s.x_scales = s.x.float().abs().amax(1) / 448.0
        s.x = (s.x.float() / s.x_scales[:, None]).to(torch.float8_e4m3fn)
    s.y = _rows(T, n, dt, gen)
    s.A = torch.empty(count, r, d, device="cuda").normal_(0.0, d ** -0.5, generator=gen).to(dt)
    s.B = torch.empty(count, n, r, device="cuda").normal_(0.0, r ** -0.5, generator=gen).to(dt)
    s.scale = torch.empty(count, device="cuda").uniform_(0.25, 2.0, generator=gen)
    # requests are runs of tokens; a share of them has no adapter
    runs = -(-T // case["run"])
    ids = torch.randint(0, count, (runs,), device="cuda", generator=gen)
    ids[torch.rand(runs, device="cuda", generator=gen) < case["none"]] = -1
    s.ids = ids.repeat_interleave(case["run"])[:T].to(torch.int32).contiguous()


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = _State()
    s.case = case
    {"norm": _norm_inputs, "route": _route_inputs, "adapters": _adapters_inputs}[case["op"]](case, gen, s)
    return s


def _n_groups(case):
    return -(-case["d"] // case["group"]) if case["group"] else 1


def prepare(case, seed):
    """Inputs, and what a program keeps beside them: the buffers that the results go to, the gate, the bank of adapters."""
    s = _inputs(case, seed)
    dev = torch.device("cuda")
    if case["op"] == "norm":
        T, d = case["T"], case["d"]
        s.out = torch.empty(T, d, dtype=_dtype(case), device=dev) if case["out"] else None
        s.residual_out = torch.empty_like(s.residual) if case["residual"] else None
        s.out8 = torch.empty(T, d, dtype=torch.float8_e4m3fn, device=dev) if case["out8"] else None
        s.scales = torch.empty(T, _n_groups(case), device=dev) if case["out8"] else None
    elif case["op"] == "route":
        s.experts = torch.empty(case["T"], case["k"], dtype=torch.int32, device=dev)
        s.weights = torch.empty(case["T"], case["k"], device=dev)
        s.slots = torch.empty_like(s.experts) if case["resident"] else None
        s.gate = None
    else:
        s.out = torch.empty_like(s.y)
        s.bank = None
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    if own:
        return {"norm": _norm_own, "route": _route_own, "adapters": _adapters_own}[s.case["op"]](s)
    return {"norm": _norm_plain, "route": _route_plain, "adapters": _adapters_plain}[s.case["op"]](s)


def _library():
    from paper_2308_15030_b200 import binding
    return binding


def _norm_own(s):
    _library().rms_norm(s.x, s.weight, EPS, out=s.out, residual=s.residual, residual_out=s.residual_out, out8=s.out8,
                        scales=s.scales, group=s.case["group"])
    return [t for t in (s.out, s.residual_out, s.out8, s.scales) if t is not None]


def _norm_plain(s):
    c = s.case
    h = s.x.float()
    got = []
    if c["residual"]:
        h = h + s.residual.float()
        residual_out = h.to(s.residual.dtype)
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s.weight.float()
    if c["out"]:
        got.append(y.to(s.x.dtype))
    if c["residual"]:
        got.append(residual_out)
    if c["out8"]:
        g, n = c["group"] or c["d"], _n_groups(c)
        y = torch.nn.functional.pad(y, (0, n * g - c["d"])).view(c["T"], n, g)
        scales = y.abs().amax(2) / 448.0
        q = y / torch.where(scales > 0, scales, 1.0)[:, :, None]
        got += [q.view(c["T"], n * g)[:, : c["d"]].to(torch.float8_e4m3fn).contiguous(), scales]
    return got


def _route_own(s):
    binding, c = _library(), s.case
    if s.gate is None:
        s.gate = binding.Gate(c["score"], c["groups"], c["topk_groups"], c["group_top"], c["renorm"], c["scale"])
    binding.route(s.gate, s.logits, s.experts, s.weights, bias=s.bias, expert_to_slot=s.expert_to_slot, slots=s.slots)
    return [t for t in (s.experts, s.weights, s.slots) if t is not None]


def _route_plain(s):
    # Scores in 64 bits: of thousands of tokens some have two experts whose scores lie closer than 32 bits tell apart.
    c = s.case
    T, E, k, G = c["T"], c["E"], c["k"], c["groups"]
    low = float("-inf")
    allowed = torch.ones(E, dtype=torch.bool, device=s.logits.device) if s.expert_to_slot is None else s.expert_to_slot >= 0
    logits = s.logits.double()
    if c["score"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-logits))
    else:
        e = torch.where(allowed, logits, low)
        e = torch.exp(e - e.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    choice = score if s.bias is None else score + s.bias.double()
    choice = torch.where(allowed, choice, low)
    if G > 1:
        size = E // G
        best = torch.sort(choice.view(T, G, size), dim=2, descending=True)[0][:, :, : c["group_top"]]
        have = allowed.view(G, size).sum(1)
        value = torch.where(best > low, best, 0.0).sum(2)
        value = torch.where(have > 0, value, low)
        value, order = torch.sort(value, dim=1, descending=True, stable=True)
        # the best groups, and further ones as long as those in front hold fewer than k experts to choose from
        before = torch.cumsum(have[order], 1) - have[order]
        rank = torch.arange(G, device=order.device)
        taken = ((rank < c["topk_groups"]) | (before < k)) & (value > low)
        kept = torch.zeros_like(taken).scatter(1, order, taken)
        choice = torch.where(kept[:, :, None].expand(T, G, size).reshape(T, E), choice, low)
    experts = torch.sort(choice, dim=1, descending=True, stable=True)[1][:, :k]
    weights = torch.gather(score, 1, experts)
    if c["renorm"]:
        weights = weights / weights.sum(1, keepdim=True)
    got = [experts.to(torch.int32), (weights * c["scale"]).float()]
    if s.expert_to_slot is not None:
        got.append(s.expert_to_slot[experts])
    return got


def _adapters_own(s):
    binding, c = _library(), s.case
    if s.bank is None:
        s.bank = binding.AdapterBank(c["count"], c["d"], c["n"], c["r"], binding.F32 if c["dtype"] == "fp32" else binding.BF16,
                                     max_tokens=c["T"])
        s.bank.set_weights(s.A, s.B, s.scale)
    s.bank.forward(s.x, s.ids, s.y, s.out, x_scales=s.x_scales)
    return s.out


def _adapters_plain(s):
    # all adapters for all tokens, then a token keeps the part of its own
    c = s.case
    x = s.x.float()
    if s.x_scales is not None:
        x = x * s.x_scales[:, None]
    u = x @ s.A.float().view(-1, c["d"]).T
    mine = s.ids[:, None] == torch.arange(c["count"], device=s.ids.device, dtype=torch.int32)
    u = (u.view(c["T"], c["count"], c["r"]) * (mine * s.scale)[:, :, None]).view(c["T"], -1)
    return (s.y.float() + u @ s.B.float().permute(0, 2, 1).reshape(-1, c["n"])).to(s.y.dtype)


# ------------------------------------------------------------------ the same from the definitions, in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _norm_exact, "route": _route_exact, "adapters": _adapters_exact}[case["op"]](s)


def _norm_exact(s):
    c = s.case
    stream = s.x.double() if s.residual is None else torch.add(s.x.double(), s.residual.double())
    power = torch.linalg.vector_norm(stream, dim=1) ** 2 / c["d"]
    y = torch.einsum("td,t,d->td", stream, (power + EPS) ** -0.5, s.weight.double())
    got = [y] if c["out"] else []
    if s.residual is not None:
        got.append(stream)
    if c["out8"]:
        q, scales = torch.empty_like(y), []
        for lo in range(0, c["d"], c["group"] or c["d"]):
            part = y[:, lo : lo + (c["group"] or c["d"])]
            scales.append(part.abs().max(dim=1).values / 448.0)
            q[:, lo : lo + part.shape[1]] = part / scales[-1][:, None]
        got += [q, torch.stack(scales, 1)]
    return got


def _route_exact(s):
    c = s.case
    if c["T"] > 20000:
        return None
    E, G = c["E"], c["groups"]
    size = E // G
    logits = s.logits.double().cpu()
    bias = s.bias.double().cpu() if s.bias is not None else torch.zeros(E, dtype=torch.float64)
    allowed = torch.arange(E) if s.expert_to_slot is None else torch.nonzero(s.expert_to_slot.cpu() >= 0)[:, 0]
    score = torch.sigmoid(logits) if c["score"] == "sigmoid" else torch.zeros_like(logits)
    if c["score"] != "sigmoid":
        score[:, allowed] = torch.softmax(logits[:, allowed], 1)
    score, bias = score.numpy(), bias.numpy()
    allowed = allowed.numpy()
    group_of = {int(e): int(e) // size for e in allowed}
    members = {g: [e for e in group_of if group_of[e] == g] for g in sorted(set(group_of.values()))}
    weights = torch.zeros(c["T"], c["k"], dtype=torch.float64)
    for t in range(c["T"]):
        row = score[t]
        choice = row + bias
        value = {g: sum(sorted((choice[e] for e in m), reverse=True)[: c["group_top"]]) for g, m in members.items()}
        pool, taken = [], 0
        for g in sorted(value, key=lambda g: (-value[g], g)):
            if taken >= c["topk_groups"] and len(pool) >= c["k"]:
                break
            pool += members[g]
            taken += 1
        best = sorted(pool, key=lambda e: (-choice[e], e))[: c["k"]]
        total = sum(row[e] for e in best) if c["renorm"] else 1.0
        weights[t, : len(best)] = torch.tensor([c["scale"] * row[e] / total for e in best], dtype=torch.float64)
    return [None, weights] + ([None] if s.expert_to_slot is not None else [])


def _adapters_exact(s):
    x = s.x.double() if s.x_scales is None else s.x.double() * s.x_scales.double()[:, None]
    out = s.y.double()
    for a in range(s.case["count"]):
        rows = torch.nonzero(s.ids == a)[:, 0]
        if rows.numel():
            low = x[rows] @ s.A[a].double().T
            out[rows] += (low @ s.B[a].double().T) * s.scale[a].double()
    return out


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    nb = 4 if case.get("dtype") == "fp32" else 2
    T = case["T"]
    if case["op"] == "norm":
        d = case["d"]
        each = nb                                                        # x
        each += 2 * (4 if case["wide"] else nb) if case["residual"] else 0
        each += nb if case["out"] else 0
        each += 1 if case["out8"] else 0
        return {"bytes": T * d * each + d * nb + (T * _n_groups(case) * 4 if case["out8"] else 0), "flops": 6.0 * T * d}
    if case["op"] == "route":
        E, k = case["E"], case["k"]
        return {"bytes": T * (4 * E + 8 * k + (4 * k if case["resident"] else 0)) + 8 * E, "flops": 4.0 * T * E}
    d, n, r, count = case["d"], case["n"], case["r"], case["count"]
    runs = -(-T // case["run"]) * (1.0 - case["none"])
    touched = count * (1.0 - (1.0 - 1.0 / count) ** runs)                # expected, requests choose among them alike
    served = T * (1.0 - case["none"])
    x_bytes = served * (d + 4 if case["x8"] else d * nb)
    return {"bytes": x_bytes + 2 * T * n * nb + touched * (r * (d + n) * nb + 4) + 4 * T, "flops": 2.0 * served * r * (d + n)}
