"""The forms of the operators in 8-bit integers, which sizes choose, agree with one another bit by bit and serve every place a call can stand in."""
import pytest

from paper_2308_15030_b200 import binding


def _quantized(n, k, gen, std=1.0):
    import torch
    v = torch.empty(n, k, device="cuda").normal_(0.0, std, generator=gen)
    q, s = torch.empty(n, k + -k % 16, dtype=torch.int8, device="cuda")[:, :k], torch.empty(n, device="cuda")
    binding.quantize_rows(v, q, s)
    return q, s


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
