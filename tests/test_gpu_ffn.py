"""GPU tests of the gated feed-forward block over row groups and of its backward pass against the 64-bit oracle:
odd and ragged groups, empty ones, rows of no group, offsets that are not offsets, infinities next to another
group's rows, other streams, captured graphs, and a run of training steps that ends in serving the block in 8 bits."""
import numpy as np
import pytest
import torch

from tests import blocks as K

pytestmark = pytest.mark.gpu
SENTINEL = 0x4B4B  # bf16 bits that no result here has


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21483_amd import binding
    return binding


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def filled(*shape):
    """A bf16 tensor of sentinels with 64 more behind it, which no call may touch."""
    n = int(np.prod(shape))
    whole = torch.full((n + 64,), SENTINEL, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    return whole[:n].view(*shape), whole


def untouched(t):
    return bool((t.contiguous().view(torch.int16) == SENTINEL).all())


class Block:
    """A block's inputs on the GPU and in 64 bits."""

    def __init__(self, T, H, F, G, off, act, seed=0, x_std=1.0):
        g = torch.Generator().manual_seed(1000 * seed + T)
        rnd = lambda std, *s: (torch.randn(*s, generator=g) * std).to(torch.bfloat16)
        self.T, self.H, self.F, self.G, self.act = T, H, F, G, act
        self.off = off
        self.x, self.dy = rnd(x_std, T, H), rnd(0.1, T, H)
        self.w1, self.w3, self.w2 = rnd(H ** -0.5, G, H, F), rnd(H ** -0.5, G, H, F), rnd(F ** -0.5, G, F, H)

    def cuda(self, B):
        self.B = B
        self.cfg = B.moe_ffn_config(self.T, self.H, self.F, self.G, B.ACTS[self.act])
        self.d = {n: getattr(self, n).cuda() for n in ("x", "dy", "w1", "w3", "w2")}
        self.d["off"] = None if self.off is None else torch.tensor(self.off, dtype=torch.int32, device="cuda")
        self.ws = torch.empty(max(B.moe_ffn_workspace_size(self.cfg, b) for b in (False, True)), dtype=torch.uint8,
                              device="cuda")
        return self

    def forward(self, keep=True, stream=None):
        d, o = self.d, {}
        y, o["y"] = filled(self.T, self.H)
        gate = up = None
        if keep:
            gate, o["gate"] = filled(self.T, self.F)
            up, o["up"] = filled(self.T, self.F)
        self.B.moe_ffn_forward(self.cfg, d["x"], d["off"], d["w1"], d["w3"], d["w2"], gate, up, y, self.ws, stream)
        return (y, gate, up), o

    def backward(self, gate, up, dx=True, dw=True, stream=None):
        d, o, r = self.d, {}, {}
        shapes = dict(dx=(self.T, self.H), dw1=(self.G, self.H, self.F), dw3=(self.G, self.H, self.F),
                      dw2=(self.G, self.F, self.H))
        for n, s in shapes.items():
            r[n], o[n] = filled(*s) if (dx if n == "dx" else dw) else (None, None)
        self.B.moe_ffn_backward(self.cfg, d["dy"], d["x"], d["off"], d["w1"], d["w3"], d["w2"], gate, up, r["dx"],
                                r["dw1"], r["dw3"], r["dw2"], self.ws, stream)
        return r, o

    def oracle_forward(self):
        return K.forward(f64(self.x), self.off, f64(self.w1), f64(self.w3), f64(self.w2), self.act, self.T)

    def oracle_backward(self, gate, up):
        return K.backward(f64(self.dy), f64(self.x), self.off, f64(self.w1), f64(self.w3), f64(self.w2), f64(gate),
                          f64(up), self.act)

    def covered(self):
        o = K.running_offsets(self.off, self.T, self.G)
        m = np.zeros(self.T, bool)
        m[o[0]:o[-1]] = True
        return torch.from_numpy(m)


def verify(b):
    """Forward and backward of one block against the oracle, and that nothing else was written."""
    (y, gate, up), whole = b.forward()
    torch.cuda.synchronize()
    refs, bounds = b.oracle_forward()
    rest = ~b.covered().cuda()
    for n, got, ref, bound in zip(("y", "gate", "up"), (y, gate, up), refs, bounds):
        K.check(n, f64(got), ref, bound)
        assert untouched(got[rest]) and untouched(whole[n][-64:]), n
    (y2, _, _), _ = b.forward(keep=False)
    assert torch.equal(y2.view(torch.int16), y.view(torch.int16)), "y depends on whether gate and up are kept"
    r, whole = b.backward(gate, up)
    torch.cuda.synchronize()
    refs, bounds = b.oracle_backward(gate, up)
    for n, ref, bound in zip(("dx", "dw1", "dw3", "dw2"), refs, bounds):
        K.check(n, f64(r[n]), ref, bound)
        assert untouched(whole[n][-64:]), n
    assert untouched(r["dx"][rest])
    return r, refs, bounds


ROWS = [1, 2, 31, 64, 65, 129, 256, 257, 333, 700]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T", ROWS)
def test_one_group_any_rows(B, T, act):
    verify(Block(T, 128, 192, 1, None, act).cuda(B))


@pytest.mark.parametrize("H,F", [(64, 64), (64, 320), (320, 64), (192, 448), (256, 256), (512, 1408), (1088, 576)])
@pytest.mark.parametrize("T", [7, 300])
def test_one_group_any_width(B, H, F, T):
    verify(Block(T, H, F, 1, [0, T], "silu", seed=1).cuda(B))


OFFSETS = {
    "even": [0, 64, 128, 192, 256],
    "odd": [0, 1, 70, 71, 255],
    "first_and_last_empty": [0, 0, 129, 255, 255],
    "rows_before_and_behind": [3, 40, 40, 41, 200],
    "all_empty": [17, 17, 17, 17, 17],
    "one_has_all": [0, 0, 0, 256, 256],
    # not offsets: read as their running maximum within [0, T]
    "outside": [-5, 30, 400, 500, 1 << 30],
    "descending": [200, 100, 256, 3, 0],
    "negative": [-(1 << 31), -1, -7, -2, -3],
}


@pytest.mark.parametrize("off", list(OFFSETS.values()), ids=list(OFFSETS))
def test_groups_of_any_rows(B, off):
    verify(Block(256, 128, 192, 4, off, "silu", seed=2).cuda(B))


@pytest.mark.parametrize("G,T", [(37, 500), (64, 90), (65, 1100), (512, 700)])
def test_many_groups(B, G, T):
    rng = np.random.default_rng(G)
    cut = np.sort(rng.integers(0, T + 1, G - 1))
    verify(Block(T, 64, 128, G, [0, *cut.tolist(), T], "gelu", seed=3).cuda(B))


def test_large_groups(B):
    """Several whole tiles of every kernel in each direction, and rows that end inside one."""
    verify(Block(1333, 640, 704, 2, [0, 811, 1333], "silu", seed=4).cuda(B))


def test_no_rows(B):
    b = Block(0, 64, 128, 3, [0, 0, 0, 0], "silu").cuda(B)
    b.forward()
    r, whole = b.backward(*(torch.empty(0, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    torch.cuda.synchronize()
    for n in ("dw1", "dw3", "dw2"):
        assert not r[n].view(torch.int16).any() and untouched(whole[n][-64:])


def test_infinities_and_nan_stay_in_their_rows_and_groups(B):
    """The last row of a group and the first of the next share a tile's depth in the weights' gradients."""
    b = Block(256, 128, 192, 4, [0, 101, 130, 200, 250], "silu", seed=5)
    clean = Block(256, 128, 192, 4, [0, 101, 130, 200, 250], "silu", seed=5)
    for r, v in ((100, float("inf")), (199, float("nan")), (255, float("nan"))):
        b.x[r, 7] = v
        b.dy[r, 3] = v
    b.cuda(B)
    clean.cuda(B)
    (y, gate, up), _ = b.forward()
    (yc, gc, uc), _ = clean.forward()
    ok = torch.ones(256, dtype=torch.bool)
    ok[[100, 199]] = False
    ok[250:] = False
    for a, c in ((y, yc), (gate, gc), (up, uc)):
        assert torch.equal(a.view(torch.int16)[ok.cuda()], c.view(torch.int16)[ok.cuda()])
    assert torch.isnan(y[199]).all() and not torch.isfinite(y[100]).any()
    r, _ = b.backward(gc, uc)
    c, _ = clean.backward(gc, uc)
    assert torch.equal(r["dx"].view(torch.int16)[ok.cuda()], c["dx"].view(torch.int16)[ok.cuda()])
    for n in ("dw1", "dw3", "dw2"):
        for g in (1, 3):  # groups without such a row
            assert torch.equal(r[n][g].view(torch.int16), c[n][g].view(torch.int16)), (n, g)
        for g in (0, 2):
            assert not torch.isfinite(r[n][g].float()).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_extreme_gates(B, act):
    """Gates of any size: the activation and its derivative end at 0 or 1, never in NaN."""
    b = Block(64, 64, 64, 1, None, act, seed=6).cuda(B)
    gate = torch.linspace(-1, 1, 64).repeat(64, 1) * torch.logspace(-3, 30, 64).unsqueeze(1)
    gate = gate.to(torch.bfloat16).cuda()
    up = torch.randn(64, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    r, _ = b.backward(gate, up)
    g64 = f64(gate)
    a, da, _, _ = K.act(np.clip(g64, -1e4, 1e4), act)  # beyond: 0 or v, 0 or 1
    a = np.where(g64 > 1e4, g64, a)
    D, W2 = f64(b.dy), f64(b.w2[0])
    dh = D @ W2.T
    dg, du = dh * f64(up) * da, dh * a
    ref = dg @ f64(b.w1[0]).T + du @ f64(b.w3[0]).T
    got = f64(r["dx"])
    assert np.isfinite(got).all()
    # bf16 dgate and dup (2^-8 each), fp32 sums and activations (under 2^-14 of the terms here), bf16 dx
    bound = (2.0 ** -8 + 2.0 ** -14) * (np.abs(dg) @ np.abs(f64(b.w1[0]).T) + np.abs(du) @ np.abs(f64(b.w3[0]).T)) \
        + 2.0 ** -8 * np.abs(ref) + 1e-30
    # near zero crossings of the exponential's range the terms carry dh's own fp32 error
    bound += 128 * K.F32 * (np.abs(D) @ np.abs(W2.T) * (np.abs(f64(up) * da) + np.abs(a))) @ \
        (np.abs(f64(b.w1[0]).T) + np.abs(f64(b.w3[0]).T))
    assert (np.abs(got - ref) <= bound).all()


def test_parts_of_the_backward_pass(B):
    b = Block(300, 128, 192, 2, [0, 120, 300], "silu", seed=7).cuda(B)
    (_, gate, up), _ = b.forward()
    full, _ = b.backward(gate, up)
    only_dx, _ = b.backward(gate, up, dw=False)
    only_dw, _ = b.backward(gate, up, dx=False)
    assert torch.equal(full["dx"].view(torch.int16), only_dx["dx"].view(torch.int16))
    for n in ("dw1", "dw3", "dw2"):
        assert torch.equal(full[n].view(torch.int16), only_dw[n].view(torch.int16)), n
    b.backward(gate, up, dx=False, dw=False)
    torch.cuda.synchronize()


def test_gradients_match_differences_of_the_loss(B):
    """d/de of sum(dy * y) along a direction, from central differences in 64 bits (exact to 1e-9 here), against the
    library's gradients: each is off by at most its bound times the direction's magnitude."""
    b = Block(97, 128, 192, 3, [0, 40, 41, 97], "gelu", seed=8).cuda(B)
    refs, _ = b.oracle_forward()
    gate, up = (torch.from_numpy(v).to(torch.bfloat16) for v in refs[1:])
    # the kept gate and up are rounded, so the oracle differentiates at theirs: the difference is in the bound
    r, _ = b.backward(gate.cuda(), up.cuda())
    p = {n: f64(getattr(b, n)) for n in ("x", "w1", "w3", "w2")}
    exact, _ = K.backward(f64(b.dy), *(p["x"], b.off, p["w1"], p["w3"], p["w2"]), refs[1], refs[2], b.act)
    rounded, bounds = b.oracle_backward(gate, up)
    rng = np.random.default_rng(0)
    for i, n in enumerate(("x", "w1", "w3", "w2")):
        v = rng.normal(size=p[n].shape)
        loss = []
        for e in (1e-5, -1e-5):
            q = dict(p, **{n: p[n] + e * v})
            (y, _, _), _ = K.forward(q["x"], b.off, q["w1"], q["w3"], q["w2"], b.act, b.T)
            loss.append(np.sum(y * f64(b.dy)))
        got = f64(r["d" + n])
        tol = np.sum((bounds[i] + np.abs(exact[i] - rounded[i])) * np.abs(v)) + 1e-6
        assert abs((loss[0] - loss[1]) / 2e-5 - np.sum(got * v)) <= tol, n


def test_same_bits_on_every_run_and_on_another_stream(B):
    b = Block(700, 256, 320, 3, [0, 300, 301, 700], "silu", seed=9).cuda(B)
    (y, gate, up), _ = b.forward()
    r, _ = b.backward(gate, up)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (None, s):
        (y2, g2, u2), _ = b.forward(stream=stream)
        if stream:
            stream.synchronize()
        r2, _ = b.backward(g2, u2, stream=stream)
        torch.cuda.synchronize()
        for a, c in ((y, y2), (gate, g2), (up, u2), *((r[n], r2[n]) for n in r)):
            assert torch.equal(a.view(torch.int16), c.view(torch.int16))


def test_tensors_that_start_inside_a_larger_one(B):
    b = Block(70, 64, 128, 1, None, "silu", seed=10).cuda(B)
    (y, _, _), _ = b.forward()
    for n in ("x", "w1", "w3", "w2"):
        t = torch.empty(b.d[n].numel() + 24, dtype=torch.bfloat16, device="cuda")[24:].view(b.d[n].shape)
        t.copy_(b.d[n])
        b.d[n] = t
    (y2, _, _), _ = b.forward()
    assert torch.equal(y.view(torch.int16), y2.view(torch.int16))
    b.d["x"] = torch.empty(70 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(70, 64)
    with pytest.raises(B.MoeError) as ei:
        b.forward()
    assert ei.value.status == B.MOE_ERR_INVALID_ARG


def test_binding_refuses_what_does_not_fit(B):
    b = Block(70, 64, 128, 2, [0, 30, 70], "silu").cuda(B)
    ok = dict(b.d)
    for n, t in [("x", ok["x"][:69]), ("w1", ok["w1"][:1]), ("w2", ok["w2"].float()), ("off", ok["off"][:2]),
                 ("off", ok["off"].long()), ("off", None), ("w3", ok["w3"].transpose(1, 2)), ("w3", ok["w3"].cpu()),
                 ("w1", None)]:
        b.d = dict(ok, **{n: t})
        with pytest.raises(ValueError):
            b.forward()
    b.d = ok
    b.ws = b.ws[:256]
    with pytest.raises(B.MoeError):
        b.forward()


def test_captured_passes_replay_on_new_inputs(B):
    """Two graphs that share a workspace, replayed in turn with eager work between them, against eager results."""
    blocks = [Block(333, 128, 192, 3, [0, 100, 101, 333], "silu", seed=s).cuda(B) for s in (11, 12)]
    blocks[1].ws = blocks[0].ws
    graphs = []
    for b in blocks:
        (y, gate, up), _ = b.forward()
        b.backward(gate, up)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            fwd, _ = b.forward()
            r, _ = b.backward(fwd[1], fwd[2])
        graphs.append((g, b, fwd, r))
    for turn in range(4):
        for g, b, fwd, r in graphs:
            b.d["x"].copy_(torch.randn(333, 128, generator=torch.Generator().manual_seed(turn)).to(torch.bfloat16))
            b.d["off"].copy_(torch.tensor([0, 50 * turn, 50 * turn + turn, 333 - turn], dtype=torch.int32))
            for t in (*fwd, *r.values()):
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (*fwd, *r.values())]
            (y, gate, up), _ = b.forward()
            e, _ = b.backward(gate, up)
            torch.cuda.synchronize()
            for a, c in zip(got, (y, gate, up, *e.values())):
                some = c.view(torch.int16) != SENTINEL
                assert torch.equal(a.view(torch.int16)[some], c.view(torch.int16)[some])


def test_layer_experts_in_training_then_served_in_8_bits(B):
    """The operators together, as a program uses them: the routing tables of a layer give the groups, two steps
    train its experts, and the trained block is quantised and served.  Each result is checked against the oracle on
    what the library was given."""
    from paper_2609_21483_amd import workloads as W
    T, H, F, E, k = 64, 128, 256, 8, 2
    shape = W.TINY
    idx = torch.from_numpy(W.random_routing(T, E, k, 3, skew=0.8)[0]).cuda()
    h = B.moe_init(B.make_config(shape))
    ws = torch.empty(B.moe_workspace_size(h), dtype=torch.uint8, device="cuda")
    B.moe_set_workspace(h, ws)
    B.moe_build_tables(h, idx)
    L = B.moe_workspace_layout(h)
    off = ws[L.off:L.off + 4 * (E + 1)].view(torch.int32)
    inv = ws[L.inv:L.inv + 4 * T * k].view(torch.int32)
    assert B.moe_sync_status(h) == B.MOE_OK
    b = Block(T * k, H, F, E, None, "silu", seed=13).cuda(B)
    b.off = off.cpu().tolist()
    tokens = torch.randn(T, H, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    b.d["x"] = tokens[(inv // k).long()].contiguous()
    b.d["off"] = off.clone()
    b.x = b.d["x"].cpu()
    for step in range(2):
        r, refs, bounds = verify(b)
        for n in ("w1", "w3", "w2"):
            b.d[n] -= 0.5 * r["d" + n]
            setattr(b, n, b.d[n].cpu())
    # served: gate and up in one operand, rows quantised before each product
    w13, s13 = torch.empty(E, 2 * F, H, dtype=torch.int8, device="cuda"), torch.empty(E, 2 * F, device="cuda")
    w2q, s2 = torch.empty(E, H, F, dtype=torch.int8, device="cuda"), torch.empty(E, H, device="cuda")
    B.moe_quantize_weights_i8(E, H, F, 2 * F, 0, b.d["w1"], w13, s13)
    B.moe_quantize_weights_i8(E, H, F, 2 * F, F, b.d["w3"], w13, s13)
    B.moe_quantize_weights_i8(E, F, H, H, 0, b.d["w2"], w2q, s2)
    X = T * k
    q, s = torch.empty(X, H, dtype=torch.int8, device="cuda"), torch.empty(X, device="cuda")
    hq, hs = torch.empty(X, F, dtype=torch.int8, device="cuda"), torch.empty(X, device="cuda")
    hid, y = (torch.empty(X, n, dtype=torch.bfloat16, device="cuda") for n in (F, H))
    c1, c2 = B.moe_gemm_i8_config(X, H, 2 * F, E, B.MOE_ACT_SILU), B.moe_gemm_i8_config(X, F, H, E, B.MOE_ACT_NONE)
    iws = torch.empty(max(B.moe_gemm_i8_workspace_size(c) for c in (c1, c2)), dtype=torch.uint8, device="cuda")
    B.moe_quantize_rows_i8(X, H, b.d["x"], q, s)
    B.moe_gemm_i8(c1, q, s, b.d["off"], w13, s13, hid, iws)
    B.moe_quantize_rows_i8(X, F, hid, hq, hs)
    B.moe_gemm_i8(c2, hq, hs, b.d["off"], w2q, s2, y, iws)
    torch.cuda.synchronize()
    for x, xq, xs in ((b.d["x"], q, s), (hid, hq, hs)):
        eq, es = K.quantize_rows(x.float().cpu().numpy())
        assert np.array_equal(xq.cpu().numpy(), eq) and np.array_equal(xs.cpu().numpy(), es)
    for a, sa, w, sw, out, act in ((q, s, w13, s13, hid, "silu"), (hq, hs, w2q, s2, y, "none")):
        ref, bound = K.gemm_i8(a.cpu().numpy(), sa.cpu().numpy(), b.off, w.cpu().numpy(), sw.cpu().numpy(), act)
        K.check("served", f64(out), ref, bound)
    # and against the block itself: every quantised value is off by at most half a step, scale / 2
    (ref, _, _), _ = b.oracle_forward()
    W13 = np.concatenate([f64(b.w1), f64(b.w3)], 2)
    for i in range(E):
        rows = slice(b.off[i], b.off[i + 1])
        x64, W2 = f64(b.x)[rows], f64(b.w2[i])
        dx, dw = 0.5 * s.cpu().numpy()[rows, None], 0.5 * s13[i].cpu().numpy()[None, :]
        ev = np.abs(x64).sum(1, keepdims=True) * dw + dx * np.abs(W13[i]).sum(0)[None] + H * dx * dw
        v = x64 @ W13[i]
        eh = 1.13 * ev[:, :F] * (np.abs(v[:, F:]) + ev[:, F:]) + np.abs(K.act(v[:, :F], "silu")[0]) * ev[:, F:]
        habs = np.abs(K.act(v[:, :F], "silu")[0] * v[:, F:]) + eh
        eh = eh + 2 * K.BF * habs + 0.5 * hs.cpu().numpy()[rows, None]
        bound = eh @ np.abs(W2) + (habs + eh).sum(1, keepdims=True) * 0.5 * s2[i].cpu().numpy()[None] + 2 * K.BF * np.abs(ref[rows])
        K.check("block in 8 bits", f64(y)[rows], ref[rows], 1.01 * bound)
    B.moe_destroy(h)


def test_weights_of_the_other_layout_are_refused(B):
    """[G][F][H], torch's Linear, holds as many values as [G][H][F]; x and y in any split of their rows are taken."""
    b = Block(70, 64, 128, 2, [0, 30, 70], "silu", seed=14).cuda(B)
    (y, gate, up), _ = b.forward()
    ok = dict(b.d)
    for n in ("w1", "w3", "w2"):
        b.d = dict(ok, **{n: ok[n].transpose(1, 2).contiguous()})
        with pytest.raises(ValueError, match="of shape"):
            b.forward()
        with pytest.raises(ValueError, match="of shape"):
            b.backward(gate, up)
    b.d = dict(ok, x=ok["x"].view(2, 35, 4, 16), w1=ok["w1"].flatten(), w3=ok["w3"].view(128, 128))
    (y2, _, _), _ = b.forward()
    assert torch.equal(y.view(torch.int16), y2.view(torch.int16))
