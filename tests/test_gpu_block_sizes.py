"""GPU tests of the products over row groups where elements or bytes pass 32 bits: planes of more than 2^31 values,
groups whose weights start more than 4 GiB in, and 8-bit operands of more than 2 GiB.  The last rows or the last
group are checked, in 64 bits on the GPU."""
import pytest
import torch

from tests import blocks as K
from tests.test_gpu_ffn import B  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def silu(v):
    return v / (1.0 + torch.exp(-v))


def within(name, got, ref, terms, depth, factors=K.BF + 2.0 ** -16):
    """terms: the sum of the magnitudes that were added.  Their factors were rounded to bf16 once (2^-8; activations
    are good to 2^-16 here) unless they are inputs (factors = 0), they were summed in fp32 (2 depth 2^-24), and the
    result was rounded to bf16."""
    far = (got.double() - ref).abs() - (K.BF * ref.abs() + (factors + 2 * depth * K.F32) * terms * (1 + K.BF) + K.ATOL)
    assert bool((far <= 0).all()), f"{name}: beyond the bound by up to {far.max().item():.3g}"


def test_planes_of_more_than_31_bits(B):
    T, H, F, last = 66000, 64, 32768, 8
    assert T * F > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda std, *s: (torch.randn(*s, generator=g, device="cuda") * std).to(torch.bfloat16)
    x, w1, w3, w2 = rnd(1, T, H), rnd(0.125, 1, H, F), rnd(0.125, 1, H, F), rnd(0.01, 1, F, H)
    cfg = B.moe_ffn_config(T, H, F, 1, B.MOE_ACT_SILU)
    ws = torch.empty(B.moe_ffn_workspace_size(cfg, True), dtype=torch.uint8, device="cuda")
    gate, up, y = (torch.empty(T, n, dtype=torch.bfloat16, device="cuda") for n in (F, F, H))
    B.moe_ffn_forward(cfg, x, None, w1, w3, w2, gate, up, y, ws)
    X = x[-last:].double()
    G, U = X @ w1[0].double(), X @ w3[0].double()
    h = silu(G) * U
    eh = 2 * H * K.F32 * (X.abs() @ w1[0].double().abs() * 1.13 * U.abs() + X.abs() @ w3[0].double().abs() * silu(G).abs())
    # (a sum of 64 inputs' products that nearly cancels is off by up to 2 64 2^-24 of their magnitudes)
    within("gate", gate[-last:], G, X.abs() @ w1[0].double().abs(), H, 0)
    within("up", up[-last:], U, X.abs() @ w3[0].double().abs(), H, 0)
    within("y", y[-last:], h @ w2[0].double(), (h.abs() + eh / K.BF) @ w2[0].double().abs(), F)
    # gradients of the last rows alone reach the weights
    dy = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    dy[-last:] = rnd(1, last, H)
    dx, dw1, dw3, dw2 = (torch.empty_like(t) for t in (x, w1, w3, w2))
    B.moe_ffn_backward(cfg, dy, x, None, w1, w3, w2, gate, up, dx, dw1, dw3, dw2, ws)
    G, U, D = gate[-last:].double(), up[-last:].double(), dy[-last:].double()
    s = 1.0 / (1.0 + torch.exp(-G))
    dh = D @ w2[0].double().t()
    # dh's own fp32 sum: 2 H 2^-24 of its terms, which stay within 2^-10 of these
    dg, du = dh * U * s * (1 + G * (1 - s)), dh * silu(G)
    edh = 2 * H * K.F32 * (D.abs() @ w2[0].double().abs().t())
    eg, eu = edh * (U * s * (1 + G * (1 - s))).abs() / K.BF, edh * silu(G).abs() / K.BF
    w1t, w3t = w1[0].double().t(), w3[0].double().t()
    within("dx", dx[-last:], dg @ w1t + du @ w3t, (dg.abs() + eg) @ w1t.abs() + (du.abs() + eu) @ w3t.abs(), 2 * F)
    assert not dx[:-last].any()
    within("dw1", dw1[0], X.t() @ dg, X.abs().t() @ (dg.abs() + eg), T)
    within("dw3", dw3[0], X.t() @ du, X.abs().t() @ (du.abs() + eu), T)
    h = silu(G) * U
    within("dw2", dw2[0], h.t() @ D, h.abs().t() @ D.abs(), T)


def test_groups_beyond_4_gib_of_weights(B):
    T, H, F, G = 5, 16384, 32768, 6
    off = torch.tensor([0, 1, 1, 1, 1, 1, 5], dtype=torch.int32, device="cuda")
    assert 5 * H * F * 2 > 1 << 32
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda std, *s: (torch.randn(*s, generator=g, device="cuda") * std).to(torch.bfloat16)
    x = rnd(1, T, H)
    w = [torch.zeros(G, *s, dtype=torch.bfloat16, device="cuda") for s in ((H, F), (H, F), (F, H))]
    for t, std in zip(w, (0.008, 0.008, 0.006)):
        t[-1] = rnd(std, *t.shape[1:])
    cfg = B.moe_ffn_config(T, H, F, G, B.MOE_ACT_SILU)
    ws = torch.empty(B.moe_ffn_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    y = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    B.moe_ffn_forward(cfg, x, off, *w, None, None, y, ws)
    assert not y[0].any()
    X = x[1:].double()
    gate, up = X @ w[0][-1].double(), X @ w[1][-1].double()
    h = silu(gate) * up
    # the fp32 sums of gate and up: 2 H 2^-24 of their terms, about 2^-12 of a unit here
    e = 2 * H * K.F32 * (X.abs() @ w[0][-1].double().abs() * 1.13 * up.abs() + X.abs() @ w[1][-1].double().abs() * silu(gate).abs())
    W2 = w[2][-1].double()
    within("y", y[1:], h @ W2, (h.abs() + e / K.BF) @ W2.abs(), F)


def test_8_bit_rows_of_more_than_31_bits(B):
    T, D, N, last = 66000, 32768, 64, 8
    assert T * D > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda")
    x[-last:] = torch.randn(last, D, generator=g, device="cuda").to(torch.bfloat16)
    q, s = torch.empty(T, D, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    B.moe_quantize_rows_i8(T, D, x, q, s)
    eq, es = K.quantize_rows(x[-last:].float().cpu().numpy())
    assert torch.equal(q[-last:].cpu(), torch.from_numpy(eq)) and torch.equal(s[-last:].cpu(), torch.from_numpy(es))
    assert not q[:-last].any() and not s[:-last].any()
    wq = torch.randint(-128, 128, (1, N, D), generator=g, device="cuda", dtype=torch.int8)
    sw = torch.rand(1, N, generator=g, device="cuda")
    cfg = B.moe_gemm_i8_config(T, D, N, 1, B.MOE_ACT_NONE)
    ws = torch.empty(B.moe_gemm_i8_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    y = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    B.moe_gemm_i8(cfg, q, s, None, wq, sw, y, ws)
    ref = (q[-last:].double() @ wq[0].double().t()) * s[-last:, None].double() * sw[0].double()
    assert bool(((y[-last:].double() - ref).abs() <= (K.BF + 4 * K.F32) * ref.abs() + K.ATOL).all())
    assert not y[:-last].any()
