"""GPU tests that every part of every sum arrives: whole-numbered inputs whose sums are exact in fp32 in any order, so
that results equal the 64-bit ones after the documented roundings, bit for bit, at sizes that take every kind of tile
whole and in parts; 8-bit sums that cancel from beyond fp32's 24 bits; and norms of the errors on random inputs."""
import numpy as np
import pytest
import torch

from tests import block_plans as PL
from tests import blocks as K
from tests.test_gpu_ffn import B, Block, f64, untouched  # noqa: F401  (B is the fixture)
from tests.test_gpu_int8 import Gemm

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def sparse(g, *shape):
    """-1, 0 and 1; one value in four is not 0."""
    r = torch.randint(0, 8, shape, generator=g, device="cuda", dtype=torch.int8)
    return (r == 1).to(BF) - (r == 0).to(BF)


def rne(v):
    """float64 (whole numbers that fp32 holds) rounded to bf16."""
    return v.float().to(BF)


def same(name, got, ref, terms, unit=1.0):
    """got equals ref rounded to bf16.  terms: the sum of the magnitudes added, in units that divide each of them:
    below 2^24 of them no order of additions rounds anything."""
    assert (terms / unit).max().item() < 1 << 24, f"{name}: sums that fp32 may round"
    bad = got.float() != rne(ref).float()
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} differ, first at {bad.nonzero()[0].tolist()}"


class ExactBlock(Block):
    """A block of whole numbers.  Gates are 128 and a sum of some units: beyond 32, where both activations are their
    argument exactly (1 + e^-32 is 1) and their slopes 1.  The last channel of x is 1, w1's 128 and w3's 0 there."""

    def __init__(self, T, H, F, off, act, seed=0):
        g = torch.Generator(device="cuda").manual_seed(1000 * seed + T)
        G = PL.groups(off)
        self.T, self.H, self.F, self.G, self.act, self.off = T, H, F, G, act, off
        self.x, self.dy = sparse(g, T, H), sparse(g, T, H)
        self.w1, self.w3, self.w2 = sparse(g, G, H, F), sparse(g, G, H, F), sparse(g, G, F, H)
        self.x[:, -1], self.w1[:, -1], self.w3[:, -1] = 1, 128, 0

    def rows(self):
        o = K.running_offsets(self.off, self.T, self.G)
        return [(i, slice(int(a), int(b))) for i, (a, b) in enumerate(zip(o, o[1:]))]

    def verify_forward(self):
        (y, gate, up), whole = self.forward()
        for i, r in self.rows():
            if r.stop == r.start:
                continue
            x, w1, w3, w2 = (v.double() for v in (self.x[r], self.w1[i], self.w3[i], self.w2[i]))
            g, u = x @ w1, x @ w3
            assert g.min() >= 32 and g.max() <= 256 and u.abs().max() <= 256
            same("gate", gate[r], g, x.abs() @ w1.abs())
            same("up", up[r], u, x.abs() @ w3.abs())
            h = rne(g * u).double()
            same("y", y[r], h @ w2, h.abs() @ w2.abs())
        for t in whole.values():
            assert untouched(t[-64:])
        rest = ~self.covered().cuda()
        for t in (y, gate, up):
            assert untouched(t[rest])
        return gate, up

    def verify_backward(self, gate, up):
        r_, whole = self.backward(gate, up)
        for i, r in self.rows():
            if r.stop == r.start:
                for n in ("dw1", "dw3", "dw2"):
                    assert not r_[n][i].view(torch.int16).any()
                continue
            x, dy, g, u = (v[r].double() for v in (self.x, self.dy, gate, up))
            w1, w3, w2 = (v[i].double() for v in (self.w1, self.w3, self.w2))
            dh = dy @ w2.t()
            assert (dy.abs() @ w2.abs().t()).max() < 1 << 24
            dg, du, h = rne(dh * u).double(), rne(dh * g).double(), rne(g * u).double()
            dx, terms = dg @ w1.t() + du @ w3.t(), dg.abs() @ w1.abs().t() + du.abs() @ w3.abs().t()
            same("dx", r_["dx"][r][:, :-1], dx[:, :-1], terms[:, :-1])
            same("dx of the last channel", r_["dx"][r][:, -1], dx[:, -1], terms[:, -1], 128.0)
            same("dw1", r_["dw1"][i], x.t() @ dg, x.abs().t() @ dg.abs())
            same("dw3", r_["dw3"][i], x.t() @ du, x.abs().t() @ du.abs())
            same("dw2", r_["dw2"][i], h.t() @ dy, h.abs().t() @ dy.abs())
        for t in whole.values():
            assert untouched(t[-64:])
        assert untouched(r_["dx"][~self.covered().cuda()])


@pytest.mark.parametrize("T,H,F,off,act,plan", PL.FFN, ids=lambda v: str(v)[:24])
def test_every_part_of_every_sum(B, T, H, F, off, act, plan):
    b = ExactBlock(T, H, F, off, act, seed=31).cuda(B)
    p = B.moe_ffn_plan_host(b.cfg)
    assert {n: getattr(p, n).as_tuple() for n in plan} == plan
    b.verify_backward(*b.verify_forward())


# sizes of the other tests: rows that end inside tiles, ragged and empty groups
@pytest.mark.parametrize("T,H,F,off,act", [
    (8192, 64, 1024, None, "silu"), (8190, 192, 1024, None, "gelu"), (8190, 1024, 320, None, "silu"),
    (9000, 256, 960, [5, 4100, 4101, 8999], "silu"), (33, 128, 7168, [0, 1, 32], "silu"), (3000, 64, 64, None, "silu"),
    (2500, 64, 64, [0, 0, 2490, 2491], "gelu"), (1333, 640, 704, [0, 811, 1333], "silu"), (333, 1024, 2816, [0, 140, 233, 300, 333], "gelu"),
    (256, 128, 192, [3, 40, 40, 41, 200], "silu"), (700, 512, 1408, None, "silu")], ids=lambda v: str(v)[:24])
def test_every_part_of_every_sum_at_other_sizes(B, T, H, F, off, act):
    b = ExactBlock(T, H, F, off, act, seed=32).cuda(B)
    b.verify_backward(*b.verify_forward())


def cancelling(g, T, D, N, G, gated):
    """8-bit operands of depth D whose products' first half adds 9000 and more a term and whose second half takes it
    back but for a few of them off by 1; in the last 64 values of the depth units, and 64 x 64 for gates."""
    m = (D - 64) // 2
    i8 = dict(generator=g, device="cuda", dtype=torch.int8)
    x, w = torch.zeros(T, D, dtype=torch.int8, device="cuda"), torch.zeros(G, N, D, dtype=torch.int8, device="cuda")
    x[:, :m] = torch.randint(80, 127, (T, m), **i8)
    w[:, :, :m] = torch.randint(80, 127, (G, N, m), **i8)
    x[:, m:2 * m], w[:, :, m:2 * m] = x[:, :m].flip(1), -w[:, :, :m].flip(2)
    off = torch.rand(T, m, generator=g, device="cuda") < 4.0 / max(m, 1)
    x[:, m:2 * m] += off.to(torch.int8)
    x[:, 2 * m:], w[:, :, 2 * m:] = torch.randint(-1, 2, (T, D - 2 * m), **i8), torch.randint(-1, 2, (G, N, D - 2 * m), **i8)
    if gated:
        x[:, -1] = 64
        w[:, :N // 2, -1] = 64
    return x, w


@pytest.mark.parametrize("T,D,N,off,act,plan", PL.I8, ids=lambda v: str(v)[:24])
def test_8_bit_sums_are_exact(B, T, D, N, off, act, plan):
    gated, G = act != "none", PL.groups(off)
    g = torch.Generator(device="cuda").manual_seed(T + D)
    cfg = B.moe_gemm_i8_config(T, D, N, G, B.ACTS[act])
    assert B.moe_gemm_i8_plan_host(cfg).as_tuple() == plan
    x, w = cancelling(g, T, D, N, G, gated)
    # powers of two, so that a sum's one rounding is the last; gates stay beyond 32, where activations are exact
    sx = torch.exp2(torch.randint(-2, 3, (T,), generator=g, device="cuda").float())
    sw = torch.exp2(torch.randint(-2, 3, (G, N), generator=g, device="cuda").float())
    out = N // 2 if gated else N
    whole = torch.full((T * out + 64,), 0x4B4B, dtype=torch.int16, device="cuda").view(BF)
    y = whole[:T * out].view(T, out)
    ws = torch.empty(B.moe_gemm_i8_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    doff = None if off is None else torch.tensor(off, dtype=torch.int32, device="cuda")
    B.moe_gemm_i8(cfg, x, sx, doff, w, sw, y, ws)
    o = K.running_offsets(off, T, G)
    for i in range(G):
        r = slice(int(o[i]), int(o[i + 1]))
        if r.start == r.stop:
            continue
        v = x[r].double() @ w[i].double().t()
        scaled = v * sx[r, None].double() * sw[i].double()
        if gated:
            assert scaled[:, :out].min() >= 32 and (v[:, :out] * v[:, out:]).abs().max() < 1 << 24
            scaled = scaled[:, :out] * scaled[:, out:]
        else:
            assert v.abs().max() < 1 << 24
        bad = y[r].float() != rne(scaled).float()
        assert not bad.any(), f"group {i}: {int(bad.sum())} of {bad.numel()} differ, first at {bad.nonzero()[0].tolist()}"
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[int(o[0]):int(o[-1])] = False
    assert untouched(y[rest]) and untouched(whole[-64:])


@pytest.mark.parametrize("T,H,F,off,act", [
    (1, 128, 192, None, "silu"), (257, 128, 192, None, "gelu"), (290, 1024, 2112, None, "gelu"), (5, 64, 8192, None, "silu"),
    (33, 128, 7168, [0, 1, 32], "gelu"), (700, 256, 320, [0, 300, 301, 700], "silu"), (1333, 640, 704, [0, 811, 1333], "silu"),
    (3001, 64, 64, [0, 1, 2987], "gelu"), (4100, 256, 960, [5, 2100, 2101, 4099], "silu")], ids=lambda v: str(v)[:24])
def test_norms_of_the_errors(B, T, H, F, off, act):
    b = Block(T, H, F, PL.groups(off), off, act, seed=33).cuda(B)
    (y, gate, up), _ = b.forward()
    r, _ = b.backward(gate, up)
    refs, _ = b.oracle_forward()
    for n, got, ref in zip(("y", "gate", "up"), (y, gate, up), refs):
        K.norms(n, f64(got), ref)
    refs, _ = b.oracle_backward(gate, up)
    for n, ref in zip(("dx", "dw1", "dw3", "dw2"), refs):
        K.norms(n, f64(r[n]), ref)


def test_planes_of_more_than_31_bits_are_exact(B):
    """As many values as 32 bits cannot count: the last rows, and gradients that only the last rows have."""
    T, H, F, last = 66000, 64, 32768, 40
    g = torch.Generator(device="cuda").manual_seed(34)
    x, w1, w3, w2 = sparse(g, T, H), sparse(g, 1, H, F), sparse(g, 1, H, F), sparse(g, 1, F, H)
    x[:, -1], w1[:, -1], w3[:, -1] = 1, 128, 0
    dy = torch.zeros(T, H, dtype=BF, device="cuda")
    dy[-last:] = sparse(g, last, H)
    cfg = B.moe_ffn_config(T, H, F, 1, B.MOE_ACT_GELU)
    ws = torch.empty(B.moe_ffn_workspace_size(cfg, True), dtype=torch.uint8, device="cuda")
    gate, up, y = (torch.empty(T, n, dtype=BF, device="cuda") for n in (F, F, H))
    B.moe_ffn_forward(cfg, x, None, w1, w3, w2, gate, up, y, ws)
    dx, dw1, dw3, dw2 = (torch.empty_like(t) for t in (x, w1, w3, w2))
    B.moe_ffn_backward(cfg, dy, x, None, w1, w3, w2, gate, up, dx, dw1, dw3, dw2, ws)
    X, D, w1, w3, w2 = (v.double() for v in (x[-last:], dy[-last:], w1[0], w3[0], w2[0]))
    G, U = X @ w1, X @ w3
    h, dh = rne(G * U).double(), D @ w2.t()
    dg, du = rne(dh * U).double(), rne(dh * G).double()
    same("gate", gate[-last:], G, X.abs() @ w1.abs())
    same("up", up[-last:], U, X.abs() @ w3.abs())
    same("y", y[-last:], h @ w2, h.abs() @ w2.abs())
    ref, terms = dg @ w1.t() + du @ w3.t(), dg.abs() @ w1.abs().t() + du.abs() @ w3.abs().t()
    same("dx", dx[-last:][:, :-1], ref[:, :-1], terms[:, :-1])
    same("dx of the last channel", dx[-last:][:, -1], ref[:, -1], terms[:, -1], 128.0)
    assert not dx[:-last].any()
    same("dw1", dw1[0], X.t() @ dg, X.abs().t() @ dg.abs())
    same("dw3", dw3[0], X.t() @ du, X.abs().t() @ du.abs())
    same("dw2", dw2[0], h.t() @ D, h.abs().t() @ D.abs())


def bits(t):
    return t.contiguous().view(torch.int16)


# few rows whole and in parts, small tiles in parts, wide tiles
@pytest.mark.parametrize("T,H,F,G,off,off2", [
    (60, 128, 192, 3, [0, 20, 21, 60], [7, 30, 55, 58]), (5, 64, 8192, 2, [0, 2, 5], [0, 3, 5]),
    (300, 2048, 4096, 1, [0, 300], [0, 300]), (3001, 64, 64, 2, [0, 1, 2987], [14, 2000, 3001]),
    (12000, 1024, 1024, 3, [3, 40, 7041, 11990], [0, 6000, 6100, 12000])], ids=lambda v: str(v)[:24])
def test_bits_follow_from_the_config_and_the_row(B, T, H, F, G, off, off2):
    """The same rows elsewhere in their groups, among other rows and other offsets."""
    a, b = Block(T, H, F, G, off, "silu", seed=35), Block(T, H, F, G, off2, "silu", seed=36)
    for n in ("w1", "w3", "w2"):
        setattr(b, n, getattr(a, n))
    rng = np.random.default_rng(T)
    src, dst = [], []
    for g in range(G):
        r, s = np.arange(off[g], off[g + 1]), np.arange(off2[g], off2[g + 1])
        n = (min(len(r), len(s)) + 1) // 2
        src += rng.choice(r, n, replace=False).tolist()
        dst += rng.choice(s, n, replace=False).tolist()
    b.x[dst], b.dy[dst] = a.x[src], a.dy[src]
    a.cuda(B), b.cuda(B)
    src, dst = torch.tensor(src, device="cuda"), torch.tensor(dst, device="cuda")
    fa, fb = a.forward()[0], b.forward()[0]
    for p, q in zip(fa, fb):
        assert torch.equal(bits(p[src]), bits(q[dst]))
    ra, rb = a.backward(fa[1], fa[2])[0], b.backward(fb[1], fb[2])[0]
    assert torch.equal(bits(ra["dx"][src]), bits(rb["dx"][dst]))


@pytest.mark.parametrize("T,H,F,off,off2", [(300, 64, 64, [0, 90, 290], [10, 100, 300]), (3001, 64, 64, [0, 1200, 2987], [14, 1214, 3001]),
                                            (2100, 4096, 192, [0, 129, 300, 1000, 1000, 1000, 2100], [0, 1900, 2071, 2072, 2073, 2074, 2075])])
def test_bits_of_gradients_follow_from_the_config_and_the_group(B, T, H, F, off, off2):
    """The second group's rows elsewhere, behind another first group of other rows."""
    G, n = len(off) - 1, off[2] - off[1]
    a, b = Block(T, H, F, G, off, "gelu", seed=37), Block(T, H, F, G, off2, "gelu", seed=38)
    for w in ("w1", "w3", "w2"):
        getattr(b, w)[1] = getattr(a, w)[1]
    assert n == off2[2] - off2[1]
    for v in ("x", "dy"):
        getattr(b, v)[off2[1]:off2[2]] = getattr(a, v)[off[1]:off[2]]
    a.cuda(B), b.cuda(B)
    fa, fb = a.forward()[0], b.forward()[0]
    ra, rb = a.backward(fa[1], fa[2])[0], b.backward(fb[1], fb[2])[0]
    for w in ("dw1", "dw3", "dw2"):
        assert torch.equal(bits(ra[w][1]), bits(rb[w][1])), w


# against few rows by 8 waves, of one row: every other kind of tile, whole and in parts
@pytest.mark.parametrize("T,D,N,G,off,act", [
    (600, 4160, 272, 1, None, "silu"), (600, 192, 320, 2, [0, 300, 600], "gelu"), (9000, 448, 528, 1, None, "none"),
    (8190, 448, 48, 2, [0, 4000, 8190], "gelu"), (2100, 8256, 48, 1, None, "gelu"), (2100, 8256, 48, 1, None, "none"),
    (8190, 448, 1040, 2, [0, 4001, 8190], "gelu"), (12000, 448, 272, 1, None, "silu"), (5, 28736, 144, 1, None, "gelu")])
def test_8_bit_rows_have_the_same_bits_in_any_batch(B, T, D, N, G, off, act):
    g = Gemm(B, T, D, N, G, off, act, seed=39)
    y, _ = g.run()
    for r in sorted({0, min(7, T - 1), T // 2 - 1, T - 1}):
        group = 0 if off is None else int(r >= off[1])
        cfg = B.moe_gemm_i8_config(1, D, N, 1, B.ACTS[act])
        one = torch.empty(1, g.out, dtype=BF, device="cuda")
        ws = torch.empty(B.moe_gemm_i8_workspace_size(cfg), dtype=torch.uint8, device="cuda")
        B.moe_gemm_i8(cfg, g.d[0][r:r + 1], g.d[1][r:r + 1].clone(), None, g.d[2][group], g.d[3][group], one, ws)
        assert torch.equal(bits(one[0]), bits(y[r])), r


def test_gradients_of_groups_beyond_4_gib_of_weights_are_exact(B):
    """The last group's weights and gradients start more than 4 GiB in; groups without rows have gradients of 0."""
    T, H, F, G = 5, 16384, 32768, 6
    off = torch.tensor([0, 1, 1, 1, 1, 1, 5], dtype=torch.int32, device="cuda")
    assert 5 * H * F * 2 > 1 << 32
    g = torch.Generator(device="cuda").manual_seed(41)
    thin = lambda t, n: t * (torch.rand(t.shape, generator=g, device="cuda") < 1.0 / n).to(BF)
    x, dy = thin(sparse(g, T, H), 4), thin(sparse(g, T, H), 16)
    w1, w3, w2 = (torch.zeros(G, *s, dtype=BF, device="cuda") for s in ((H, F), (H, F), (F, H)))
    for w in (w1, w3, w2):
        w[-1] = sparse(g, *w.shape[1:])
    x[:, -1], w1[-1, -1], w3[-1, -1] = 1, 128, 0
    cfg = B.moe_ffn_config(T, H, F, G, B.MOE_ACT_SILU)
    assert B.moe_ffn_plan_host(cfg).dw.as_tuple() == ("wide", 1)
    ws = torch.empty(B.moe_ffn_workspace_size(cfg, True), dtype=torch.uint8, device="cuda")
    gate, up, y = (torch.empty(T, n, dtype=BF, device="cuda") for n in (F, F, H))
    B.moe_ffn_forward(cfg, x, off, w1, w3, w2, gate, up, y, ws)
    dx, dw1, dw3, dw2 = (torch.full_like(t, 3.0) for t in (x, w1, w3, w2))
    B.moe_ffn_backward(cfg, dy, x, off, w1, w3, w2, gate, up, dx, dw1, dw3, dw2, ws)
    # the first group's weights are zeros, so its gates are too and nothing comes of it
    assert not y[0].any() and not dx[0].any()
    for d in (dw1, dw3, dw2):
        assert not d[:-1].any()
    X, D, W1, W3, W2 = (v.double() for v in (x[1:], dy[1:], w1[-1], w3[-1], w2[-1]))
    A, U, dh = X @ W1, X @ W3, D @ W2.t()
    assert A.min() >= 32 and A.max() <= 256
    h, dg, du = rne(A * U).double(), rne(dh * U).double(), rne(dh * A).double()
    same("gate", gate[1:], A, X.abs() @ W1.abs())
    same("y", y[1:], h @ W2, h.abs() @ W2.abs())
    ref, terms = dg @ W1.t() + du @ W3.t(), dg.abs() @ W1.abs().t() + du.abs() @ W3.abs().t()
    same("dx", dx[1:, :-1], ref[:, :-1], terms[:, :-1])
    same("dx of the last channel", dx[1:, -1], ref[:, -1], terms[:, -1], 128.0)
    same("dw1", dw1[-1], X.t() @ dg, X.abs().t() @ dg.abs())
    same("dw3", dw3[-1], X.t() @ du, X.abs().t() @ du.abs())
    same("dw2", dw2[-1], h.t() @ D, h.abs().t() @ D.abs())
