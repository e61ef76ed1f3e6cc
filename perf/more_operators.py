"""Operators of a served block in 8-bit integers, as measurable cases.

``block_norm``  the norms behind and in front of a block in one pass: the block's output is normed, gated and scaled, added to the
                residual stream, and the sum is normed for the next block; rows out in the layer's dtype or in 8 bits with scales
``quantize``    rows to 8-bit integers with a scale each
``matmul``      a projection of 8-bit integers with a scale for each token and each channel
``experts``     the experts behind a router: feed-forward networks in 8-bit integers, tokens sent to the resident slots that
                routing chose, their results added by weight

With ``own`` false a pass computes the operator in elementary torch operations, else it calls the library.
Widths and expert counts are those of ``inputs.CONFIGS`` and of the tests' ranges, with ragged ones between them.
"""
import torch

own = False


# ------------------------------------------------------------------ cases
def _block_norm(T, d, dtype="bf16", post=True, gate="none", wide=False, out=True, out8=False, group=0, scale=1.0, pad=0):
    return {"op": "block_norm", "T": T, "d": d, "dtype": dtype, "post": post, "gate": gate, "wide": wide, "out": out, "out8": out8,
            "group": group, "scale": scale, "pad": pad}


def _quantize(T, d, dtype="bf16", pad=0):
    return {"op": "quantize", "T": T, "d": d, "dtype": dtype, "pad": pad}


def _matmul(T, K, N, dtype="bf16", bias=False, pad=0):
    return {"op": "matmul", "T": T, "K": K, "N": N, "dtype": dtype, "bias": bias, "pad": pad}


def _experts(T, d, F, slots, k, act="swiglu", none=0.0):
    # rows out in bf16: which of two integers a hidden value next to their border becomes is more than fp32's last bits
    return {"op": "experts", "T": T, "d": d, "F": F, "slots": slots, "k": k, "act": act, "dtype": "bf16", "none": none}


def listed():
    return [
        # One user's decode step between two blocks: the smallest call, all latency.
        dict(_block_norm(1, 4096), name="block_norm_1"),
        # Single precision, a gate for every token, a width that is no multiple of anything, rows inside wider ones.
        dict(_block_norm(1531, 1003, dtype="fp32", gate="rows", scale=0.5, pad=21), name="block_norm_fp32_1531"),
        # Prefill of a wide block: a gate per channel, the residual stream in fp32, 8-bit rows with a scale per 128 columns.
        dict(_block_norm(16384, 4096, gate="channels", wide=True, out=False, out8=True, group=128), name="block_norm_16384"),
        # A decode batch's rows on their way to a projection.
        dict(_quantize(61, 4096), name="quantize_61"),
        # Prefill rows of an expert's hidden width.
        dict(_quantize(8192, 14336), name="quantize_8192"),
        # One user's decode step: the weights are all that is read.
        dict(_matmul(1, 4096, 4096), name="matmul_1"),
        # A decode batch through a wide projection.
        dict(_matmul(61, 4096, 14336), name="matmul_61"),
        # Ragged widths, fp32 out, a bias, rows inside wider ones.
        dict(_matmul(1531, 1003, 2239, dtype="fp32", bias=True, pad=5), name="matmul_fp32_1531"),
        # Prefill of sixteen sequences of 512 tokens.
        dict(_matmul(8192, 4096, 14336), name="matmul_8192"),
        # A few streams of a layer with many small experts.
        dict(_experts(3, 1024, 512, 48, 2), name="experts_3"),
        # A decode batch that asks for most of the resident experts; some choices found none.
        dict(_experts(61, 2048, 1024, 64, 4, none=0.05), name="experts_61"),
        # Prefill of a layer with eight large experts.
        dict(_experts(4096, 4096, 14336, 8, 2), name="experts_4096"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() + rng.random()))


WIDTHS = [512, 704, 768, 960, 1024, 1536, 2048, 4096]


def draw(rng):
    op = rng.choice(["block_norm", "quantize", "matmul", "experts"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op == "block_norm":
        d = rng.choice(WIDTHS + [_log_int(rng, 64, 4096)])
        out8 = rng.random() < 0.5
        return _block_norm(_log_int(rng, 1, 12000), d, dtype, post=rng.random() < 0.8, gate=rng.choice(["none", "channels", "rows"]),
                           wide=dtype == "bf16" and rng.random() < 0.3, out=not out8 or rng.random() < 0.5, out8=out8,
                           group=rng.choice([0, 128]), scale=rng.choice([1.0, 0.22]), pad=rng.choice([0, 0, 8, 21]))
    if op == "quantize":
        return _quantize(_log_int(rng, 1, 12000), rng.choice(WIDTHS + [_log_int(rng, 64, 8000)]), dtype, pad=rng.choice([0, 0, 8, 21]))
    if op == "matmul":
        K = rng.choice(WIDTHS + [_log_int(rng, 64, 4096)])
        N = rng.choice(WIDTHS + [14336, _log_int(rng, 64, 8000)])
        return _matmul(_log_int(rng, 1, 8192), K, N, dtype, bias=rng.random() < 0.3, pad=rng.choice([0, 0, 5, 16]))
    d, F, slots = rng.choice([(512, 704, 16), (768, 2112, 32), (1024, 512, 64), (1024, 4096, 16), (2048, 1024, 48), (4096, 14336, 4)])
    slots = rng.randint(max(4, slots // 4), slots)
    return _experts(_log_int(rng, 1, 3500), d, F, slots, rng.randint(1, 4 if d < 4096 else 2), rng.choice(["swiglu", "swiglu", "relu"]),
                    none=rng.choice([0.0, 0.0, 0.05]))


# ------------------------------------------------------------------ inputs
EPS = 1e-6


class _State:
    pass


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _rows(T, d, dtype, gen, std=1.0, pad=0):
    """T rows of d normal values, with `pad` more columns behind each that belong to somebody else."""
    return torch.empty(T, d + pad, device="cuda").normal_(0.0, std, generator=gen).to(dtype)[:, :d]


def _int8(shape, gen, std, pad=0):
    """Rows of 8-bit integers and their scales, as normal values of that deviation give them; every row starts at a multiple of 16 bytes."""
    width = shape[-1] + pad
    width += -width % 16
    q, scales = torch.empty(*shape[:-1], width, dtype=torch.int8, device="cuda"), torch.empty(shape[:-1], device="cuda")
    for i in range(shape[0]) if len(shape) > 2 else [...]:
        v = torch.empty((*shape[1:-1], width) if len(shape) > 2 else (shape[0], width), device="cuda").normal_(0.0, std, generator=gen)
        scales[i] = v.abs().amax(-1) / 127.0
        q[i] = (v / scales[i][..., None]).round().to(torch.int8)
    return q[..., : shape[-1]], scales


def _block_norm_inputs(case, gen, s):
    T, d, dt = case["T"], case["d"], _dtype(case)
    # a block's output, a few of its tokens much louder than the others
    s.x = _rows(T, d, dt, gen, std=0.7, pad=case["pad"])
    s.x[:: 17] *= 20.0
    # a residual stream has grown over the layers, a few of its channels more than the others
    s.residual = torch.empty(T, d, device="cuda").normal_(0.0, 2.0, generator=gen)
    s.residual[:, :: max(1, d // 7)] *= 12.0
    s.residual = s.residual.to(torch.float32 if case["wide"] else dt)
    s.weight = torch.empty(d, device="cuda").normal_(1.0, 0.2, generator=gen).to(dt)
    s.post_weight = torch.empty(d, device="cuda").normal_(0.5, 0.2, generator=gen).to(dt) if case["post"] else None
    s.gate = None if case["gate"] == "none" else _rows(T if case["gate"] == "rows" else 1, d, dt, gen)
    if case["gate"] == "channels":
        s.gate = s.gate[0]


def _quantize_inputs(case, gen, s):
    s.x = _rows(case["T"], case["d"], _dtype(case), gen, pad=case["pad"])
    s.x[:, :: max(1, case["d"] // 5)] *= 6.0                           # a few channels are louder


def _matmul_inputs(case, gen, s):
    s.x8, s.x_scales = _int8((case["T"], case["K"]), gen, 1.0, pad=case["pad"])
    s.w8, s.w_scales = _int8((case["N"], case["K"]), gen, case["K"] ** -0.5, pad=case["pad"])
    s.bias = torch.empty(case["N"], device="cuda").normal_(0.0, 0.5, generator=gen) if case["bias"] else None


def _experts_inputs(case, gen, s):
    T, d, F, S, k = case["T"], case["d"], case["F"], case["slots"], case["k"]
    s.x8, s.x_scales = _int8((T, d), gen, 1.0)
    s.w_in, s.in_scales = _int8((S, (2 if case["act"] == "swiglu" else 1) * F, d), gen, d ** -0.5)
    s.w_out, s.out_scales = _int8((S, d, F), gen, F ** -0.5)
    logits = torch.empty(T, S, device="cuda").normal_(0.0, 1.5, generator=gen)
    logits += torch.empty(S, device="cuda").normal_(0.0, 0.7, generator=gen)           # some experts are asked for more
    top, slots = torch.topk(logits, k, 1)
    s.weights, s.slots = torch.softmax(top, 1), slots.to(torch.int32)
    missing = torch.rand(T, k, device="cuda", generator=gen) < case["none"]
    s.weights[missing], s.slots[missing] = 0.0, -1


_INPUTS = {"block_norm": _block_norm_inputs, "quantize": _quantize_inputs, "matmul": _matmul_inputs, "experts": _experts_inputs}


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = _State()
    s.case = case
    _INPUTS[case["op"]](case, gen, s)
    return s


def _n_groups(case):
    return -(-case["d"] // case["group"]) if case["group"] else 1


def prepare(case, seed):
    """Inputs, and what a program keeps beside them: the buffers that the results go to, the bank of experts."""
    s = _inputs(case, seed)
    T, dev = case["T"], torch.device("cuda")
    if case["op"] == "block_norm":
        s.out = torch.empty(T, case["d"], dtype=_dtype(case), device=dev) if case["out"] else None
        s.residual_out = torch.empty_like(s.residual)
        s.out8 = torch.empty(T, case["d"], dtype=torch.float8_e4m3fn, device=dev) if case["out8"] else None
        s.scales = torch.empty(T, _n_groups(case), device=dev) if case["out8"] else None
    elif case["op"] == "quantize":
        s.out8 = torch.empty(T, case["d"], dtype=torch.int8, device=dev)
        s.scales = torch.empty(T, device=dev)
    else:
        s.out = torch.empty(T, case["N"] if case["op"] == "matmul" else case["d"], dtype=_dtype(case), device=dev)
        s.bank = _bank(s) if own and case["op"] == "experts" else None
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    if own:
        return {"block_norm": _block_norm_own, "quantize": _quantize_own, "matmul": _matmul_own, "experts": _experts_own}[s.case["op"]](s)
    return {"block_norm": _block_norm_plain, "quantize": _quantize_plain, "matmul": _matmul_plain, "experts": _experts_plain}[s.case["op"]](s)


def _library():
    from paper_2308_15030_b200 import binding
    return binding


def _block_norm_own(s):
    _library().block_norm(s.x, s.residual, s.weight, EPS, out=s.out, residual_out=s.residual_out, post_weight=s.post_weight, gate=s.gate,
                          scale=s.case["scale"], out8=s.out8, scales=s.scales, group=s.case["group"])
    return [t for t in (s.out, s.residual_out, s.out8, s.scales) if t is not None]


def _block_norm_plain(s):
    c = s.case
    got = []
    p = s.x.float()
    if s.post_weight is not None:
        p = p * torch.rsqrt((p * p).mean(1, keepdim=True) + EPS) * s.post_weight.float()
    if s.gate is not None:
        p = p * s.gate.float()
    h = s.residual.float() + c["scale"] * p
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s.weight.float()
    if c["out"]:
        got.append(y.to(s.x.dtype))
    got.append(h.to(s.residual.dtype))
    if c["out8"]:
        g, n = c["group"] or c["d"], _n_groups(c)
        y = torch.nn.functional.pad(y, (0, n * g - c["d"])).view(c["T"], n, g)
        scales = y.abs().amax(2) / 448.0
        q = y / torch.where(scales > 0, scales, 1.0)[:, :, None]
        got += [q.view(c["T"], n * g)[:, : c["d"]].to(torch.float8_e4m3fn).contiguous(), scales]
    return got


def _quantize_own(s):
    _library().quantize_rows(s.x, s.out8, s.scales)
    return [s.out8, s.scales]


def _int8_rows(y):
    # the scale in 64 bits: which of two integers a value next to their border becomes hangs on its last bit
    scales = (y.abs().amax(-1).double() / 127.0).float()
    return torch.round(y / torch.where(scales > 0, scales, 1.0)[..., None]), scales


def _quantize_plain(s):
    q, scales = _int8_rows(s.x.float())
    return [q.to(torch.int8), scales]


def _matmul_own(s):
    _library().matmul_scaled(s.x8, s.x_scales, s.w8, s.w_scales, s.out, bias=s.bias)
    return s.out


def _matmul_plain(s):
    y = (s.x8.float() @ s.w8.float().T) * s.x_scales[:, None] * s.w_scales
    return (y if s.bias is None else y + s.bias).to(s.out.dtype)


def _bank(s):
    # made once, before the first token
    binding, c = _library(), s.case
    bank = binding.ExpertBank(c["slots"], c["d"], c["F"], c["k"], binding.F32 if c["dtype"] == "fp32" else binding.BF16,
                              act=binding.ACT_SWIGLU if c["act"] == "swiglu" else binding.ACT_RELU, max_tokens=c["T"])
    bank.set_weights(s.w_in, s.in_scales, s.w_out, s.out_scales)
    return bank


def _experts_own(s):
    if s.bank is None:                                                 # (inputs that were made for the plain form)
        s.bank = _bank(s)
    s.bank.forward(s.x8, s.x_scales, s.slots, s.weights, s.out)
    return s.out


def _experts_plain(s):
    # pairs (token, choice) in the order of their slots, every slot's rows filled up to the largest slot's number
    c = s.case
    T, d, F, S, k = c["T"], c["d"], c["F"], c["slots"], c["k"]
    flat = s.slots.reshape(-1).long()
    chosen = torch.nonzero(flat >= 0)[:, 0]
    order = chosen[torch.argsort(flat[chosen], stable=True)]
    slot = flat[order]
    counts = (slot[:, None] == torch.arange(S, device=slot.device)).sum(0)
    place = torch.arange(slot.numel(), device=slot.device) - (torch.cumsum(counts, 0) - counts)[slot]
    most = max(1, int(counts.max()))
    x = torch.zeros(S, most, d, device=slot.device)
    x[slot, place] = s.x8[order // k].float()
    x_scales = torch.zeros(S, most, 1, device=slot.device)
    x_scales[slot, place, 0] = s.x_scales[order // k]
    u = torch.bmm(x, s.w_in.float().transpose(1, 2)) * x_scales * s.in_scales[:, None]
    h = torch.relu(u) if c["act"] == "relu" else u[..., :F] / (1.0 + torch.exp(-u[..., :F])) * u[..., F:]
    q, h_scales = _int8_rows(h)
    y = torch.bmm(q, s.w_out.float().transpose(1, 2)) * h_scales[..., None] * s.out_scales[:, None]
    pairs = torch.zeros(T * k, d, device=slot.device)
    pairs[order] = y[slot, place] * s.weights.reshape(-1)[order][:, None]
    return pairs.view(T, k, d).sum(1).to(s.out.dtype)


# ------------------------------------------------------------------ the same from the definitions, in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    return {"block_norm": _block_norm_exact, "quantize": _quantize_exact, "matmul": _matmul_exact, "experts": _experts_exact}[case["op"]](s)


def _block_norm_exact(s):
    c = s.case
    block = s.x.double()
    if s.post_weight is not None:
        power = torch.linalg.vector_norm(block, dim=1) ** 2 / c["d"]
        block = torch.einsum("td,t,d->td", block, (power + EPS) ** -0.5, s.post_weight.double())
    if s.gate is not None:
        block = torch.mul(block, s.gate.double().expand(c["T"], c["d"]))
    stream = torch.add(s.residual.double(), block, alpha=c["scale"])
    power = torch.linalg.vector_norm(stream, dim=1) ** 2 / c["d"]
    y = torch.einsum("td,t,d->td", stream, (power + EPS) ** -0.5, s.weight.double())
    got = [y] if c["out"] else []
    got.append(stream)
    if c["out8"]:
        q, scales = torch.empty_like(y), []
        for lo in range(0, c["d"], c["group"] or c["d"]):
            part = y[:, lo : lo + (c["group"] or c["d"])]
            scales.append(part.abs().max(dim=1).values / 448.0)
            q[:, lo : lo + part.shape[1]] = part / scales[-1][:, None]
        got += [q, torch.stack(scales, 1)]
    return got


def _quantize_exact(s):
    return [None, s.x.double().abs().max(dim=1).values / 127.0]


def _matmul_exact(s):
    # sums of integers below 2^53: exact whatever their order
    y = torch.einsum("tk,nk->tn", s.x8.double(), s.w8.double())
    y = torch.einsum("tn,t,n->tn", y, s.x_scales.double(), s.w_scales.double())
    return y if s.bias is None else y + s.bias.double()


def _experts_exact(s):
    c = s.case
    out = torch.zeros(c["T"], c["d"], dtype=torch.float64, device=s.x8.device)
    for e in range(c["slots"]):
        tokens, choice = torch.nonzero(s.slots == e, as_tuple=True)
        if not tokens.numel():
            continue
        u = torch.einsum("td,fd->tf", s.x8[tokens].double(), s.w_in[e].double())
        u = torch.einsum("tf,t,f->tf", u, s.x_scales[tokens].double(), s.in_scales[e].double())
        h = u.clamp(min=0.0) if c["act"] == "relu" else torch.nn.functional.silu(u[:, : c["F"]]) * u[:, c["F"] :]
        scale = h.abs().max(dim=1).values / 127.0
        q = torch.round(h / torch.where(scale > 0, scale, torch.ones_like(scale))[:, None])
        y = torch.einsum("tf,df->td", q, s.w_out[e].double())
        out.index_add_(0, tokens, torch.einsum("td,t,d->td", y, scale * s.weights[tokens, choice].double(), s.out_scales[e].double()))
    return out


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    nb = 4 if case["dtype"] == "fp32" else 2
    T = case["T"]
    if case["op"] == "block_norm":
        d = case["d"]
        each = nb + 2 * (4 if case["wide"] else nb)                      # x, the residual in and out
        each += nb if case["gate"] == "rows" else 0
        each += nb if case["out"] else 0
        each += 1 if case["out8"] else 0
        return {"bytes": T * d * each + 3 * d * nb + (T * _n_groups(case) * 4 if case["out8"] else 0), "flops": 12.0 * T * d}
    if case["op"] == "quantize":
        return {"bytes": T * (case["d"] * (nb + 1) + 4), "flops": 3.0 * T * case["d"]}
    if case["op"] == "matmul":
        K, N = case["K"], case["N"]
        return {"bytes": T * K + N * K + T * N * nb + 4 * (T + N * (2 if case["bias"] else 1)), "flops": 2.0 * T * N * K}
    d, F, S, k = case["d"], case["F"], case["slots"], case["k"]
    n = 3 if case["act"] == "swiglu" else 2
    touched = S * (1.0 - (1.0 - k / S) ** T)                             # expected, tokens choose among them alike
    pairs = T * k * (1.0 - case["none"])
    return {"bytes": T * (d + 4) + touched * (n * d * F + 4 * ((n - 1) * F + d)) + 8 * T * k + T * d * nb, "flops": 2.0 * pairs * n * d * F}
