"""GPU tests of the gate's logits and gradients and of the routing's losses, element by element against 64 bits."""
import numpy as np
import pytest
import torch

from tests import gate_plans as GP
from tests import train_ref as R
from tests.blocks import BF, check

pytestmark = pytest.mark.gpu
MARK = 0x4B4B


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21483_amd import binding
    return binding


def marked(dtype, *shape):
    """A buffer whose values nothing has written, and 64 more behind it."""
    n = int(np.prod(shape))
    whole = torch.full(((n + 64) * torch.empty((), dtype=dtype).element_size() // 2,), MARK, dtype=torch.int16, device="cuda")
    return whole.view(dtype)[:n].view(*shape), whole


def clean(whole, n, dtype):
    assert (whole.view(dtype)[n:].view(torch.int16) == MARK).all()


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def dev_off(off):
    return None if off is None else torch.tensor(off, dtype=torch.int32, device="cuda")


def outside(off, S, T):
    """Rows of no sequence."""
    o = R.offsets(off, S, T)
    out = torch.ones(T, dtype=torch.bool)
    out[o[0]:o[-1]] = False
    return out.cuda(), o


class Gate:
    def __init__(self, B, T, H, E, off=None, S=1, seed=0):
        g = torch.Generator().manual_seed(seed + T + E)
        self.B, self.T, self.H, self.E, self.S, self.off = B, T, H, E, S, off
        self.cfg = B.moe_router_config(T, H, E, 1, S)
        self.x = torch.randn(T, H, generator=g).to(torch.bfloat16)
        self.wg = (0.05 * torch.randn(H, E, generator=g)).to(torch.bfloat16)
        self.bias, self.dl = torch.randn(E, generator=g), 1e-3 * torch.randn(T, E, generator=g)
        self.d = [t.cuda() for t in (self.x, self.wg, self.bias, self.dl)]
        self.doff = dev_off(off)

    def ws(self, backward):
        return torch.full((self.B.moe_gate_workspace_size(self.cfg, backward),), 0xA5, dtype=torch.uint8, device="cuda")

    def logits(self, bias=True, stream=None):
        out, whole = marked(torch.float32, self.T, self.E)
        self.B.moe_gate_logits(self.cfg, self.d[0], self.d[1], self.d[2] if bias else None, self.doff, out, self.ws(False), stream)
        torch.cuda.synchronize()
        clean(whole, out.numel(), torch.float32)
        return out

    def backward(self, want=("dx", "dwg", "dbias"), stream=None):
        dx, wx = marked(torch.bfloat16, self.T, self.H)
        dwg, ww = marked(torch.bfloat16, self.H, self.E)
        db, wb = marked(torch.float32, self.E)
        self.B.moe_gate_backward(self.cfg, self.d[3], self.d[0], self.d[1], self.doff, dx if "dx" in want else None,
                                 dwg if "dwg" in want else None, db if "dbias" in want else None, self.ws(True), stream)
        torch.cuda.synchronize()
        for whole, t, name in ((wx, dx, "dx"), (ww, dwg, "dwg"), (wb, db, "dbias")):
            clean(whole, t.numel() if name in want else 0, t.dtype)
        return dx, dwg, db

    def verify(self):
        out, o = outside(self.off, self.S, self.T)
        a, b = o[0], o[-1]
        x, wg = f64(self.x[a:b]), f64(self.wg)
        l = self.logits()
        check("logits", f64(l[a:b]), *R.gate_logits(x, wg, self.bias.numpy().astype(np.float64)))
        assert (l[out].view(torch.int16) == MARK).all()
        dx, dwg, db = self.backward()
        ref = R.gate_grad(self.dl[a:b].numpy(), x, wg)
        check("dx", f64(dx[a:b]), *ref[0])
        check("dwg", f64(dwg), *ref[1])
        check("dbias", f64(db), *ref[2])
        assert (dx[out].view(torch.int16) == MARK).all()


@pytest.mark.parametrize("E", [1, 2, 7, 8, 60, 64, 65, 128, 130, 256, 300, 512])
@pytest.mark.parametrize("T,H", [(1, 64), (33, 192), (130, 256), (300, 1088)])
def test_gate_of_any_size(B, T, H, E):
    Gate(B, T, H, E).verify()


@pytest.mark.parametrize("T", [2, 31, 32, 63, 64, 65, 127, 128, 129, 255, 257, 513, 1000, 2049])
def test_gate_of_any_rows(B, T):
    Gate(B, T, 128, 60, seed=1).verify()


@pytest.mark.parametrize("H", [64, 128, 320, 2048, 4096, 16384])
def test_gate_of_any_width(B, H):
    Gate(B, 70, H, 8, seed=2).verify()
    Gate(B, 70, H, 128, seed=2).verify()


SEQS = [[0, 64, 128, 256], [0, 1, 70, 255], [3, 40, 40, 200], [17, 17, 17, 17], [0, 0, 256, 256], [-5, 30, 400, 1 << 30],
        [200, 100, 256, 0], [255, 255, 255, 256]]


@pytest.mark.parametrize("off", SEQS, ids=str)
@pytest.mark.parametrize("E", [60, 128])
def test_gate_of_padded_batches(B, off, E):
    Gate(B, 256, 192, E, off, 3, seed=3).verify()


def test_rows_of_no_sequence_are_not_read(B):
    g = Gate(B, 300, 128, 60, [70, 100, 201], 2, seed=4)
    ref = [t.clone() for t in (g.logits()[70:201], g.backward()[0][70:201], *g.backward()[1:])]
    for t in (g.d[0], g.d[3]):
        t[:70] = float("nan")
        t[201:] = float("nan")
    for a, b in zip(ref, (g.logits()[70:201], g.backward()[0][70:201], *g.backward()[1:])):
        assert torch.equal(a, b)


def test_gate_gradients_that_are_not_wanted(B):
    g = Gate(B, 130, 192, 60, seed=5)
    dx, dwg, db = g.backward()
    for want, i in ((("dx",), 0), (("dwg",), 1), (("dbias",), 2)):
        assert torch.equal(g.backward(want)[i], (dx, dwg, db)[i])
    g.backward(())
    # the operands that the wanted ones do not need may be missing
    x, wg = g.d[0], g.d[1]
    g.d[0] = None
    assert torch.equal(g.backward(("dx", "dbias"))[0], dx)
    g.d[0], g.d[1] = x, None
    assert torch.equal(g.backward(("dwg",))[1], dwg)


def test_gate_without_rows(B):
    cfg = B.moe_router_config(0, 64, 12, 1, 1)
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    dl, wg = torch.empty(0, 12, device="cuda"), torch.ones(64, 12, dtype=torch.bfloat16, device="cuda")
    dwg, db = torch.ones_like(wg), torch.ones(12, device="cuda")
    ws = torch.empty(B.moe_gate_workspace_size(cfg, True), dtype=torch.uint8, device="cuda")
    B.moe_gate_backward(cfg, dl, e, wg, None, e, dwg, db, ws)
    assert not dwg.any() and not db.any()
    B.moe_gate_logits(cfg, e, wg, None, None, dl, ws)


def test_gate_of_a_nan_row_and_an_infinity(B):
    """A row's NaN reaches its own logits and dx, and every dwg; an expert's its column."""
    g = Gate(B, 140, 128, 60, seed=6)
    clean_l, (clean_dx, _, clean_db) = g.logits(), g.backward()
    g.d[0][77, 5] = float("nan")
    l = g.logits()
    assert torch.isnan(l[77]).all() and torch.equal(np_rest(l, 77), np_rest(clean_l, 77))
    dx, dwg, db = g.backward()
    assert torch.equal(dx, clean_dx) and torch.equal(db, clean_db)
    assert torch.isnan(dwg[5]).all() and not torch.isnan(np_rest(dwg, 5)).any()
    g.d[3][20, 3] = float("inf")
    dx, dwg, db = g.backward()
    assert torch.isinf(db[3]) and torch.equal(np_rest(dx, 20), np_rest(clean_dx, 20)) and not torch.isfinite(dx[20]).any()


def np_rest(t, row):
    keep = torch.ones(t.shape[0], dtype=torch.bool, device=t.device)
    keep[row] = False
    return t[keep]


def test_gate_of_a_long_batch(B):
    """A sum over 40000 rows, off by no lost part: whole numbers whose sums are exact."""
    T, H, E = 40000, 128, 60
    rng = np.random.default_rng(3)
    x, d = rng.integers(-4, 5, (T, H)).astype(np.float32), rng.integers(-4, 5, (T, E)).astype(np.float32)
    g = Gate(B, T, H, E, seed=7)
    g.d[0], g.d[3] = torch.from_numpy(x).to(torch.bfloat16).cuda(), torch.from_numpy(d).cuda()
    dx, dwg, db = g.backward()
    assert np.array_equal(f64(db), d.sum(0, dtype=np.float64))
    ref = x.T.astype(np.float64) @ d
    assert np.array_equal(f64(dwg), R.bf16(ref.astype(np.float32)).astype(np.float64))
    rdx, bdx = R.gate_grad(d[-300:], x[-300:].astype(np.float64), f64(g.wg))[0]
    check("dx", f64(dx[-300:]), rdx, bdx)


# (each kind of tile and number of parts that a product is computed by: logits by 1 to 16 parts of few rows or of a ring, by
# small and wide tiles; dx by strips of 1 to 4 times 64 columns, with dwg in one launch or behind it, and by both kinds of
# tiles; dwg by three, whole and in parts)
@pytest.mark.parametrize("T,H,E", [
    (33, 64, 8), (33, 64, 300), (1025, 64, 511), (33, 4096, 8), (33, 4096, 60), (33, 16384, 60), (133, 64, 190), (513, 64, 200),
    (517, 4096, 200), (513, 8192, 512), (6203, 4096, 190), (517, 16384, 200), (2049, 64, 200), (2051, 4096, 200), (4099, 4096, 200), (12301, 64, 200), (16403, 64, 200), (16403, 4096, 200),
    (16403, 8192, 130), (24001, 64, 300), (32801, 1088, 300), (40001, 128, 60), (8209, 192, 128)])
def test_gate_by_every_kind_of_tile(B, T, H, E):
    """Whole numbers whose sums are exact: no part is lost or added twice."""
    g = Gate(B, 8, 64, 1)
    g.T, g.H, g.E, g.S, g.cfg = T, H, E, 2, B.moe_router_config(T, H, E, 1, 2)
    r = torch.Generator(device="cuda").manual_seed(T)
    x, wg, d = (torch.randint(-4, 5, n, generator=r, device="cuda") for n in ((T, H), (H, E), (T, E)))
    g.d, g.doff = [x.to(torch.bfloat16), wg.to(torch.bfloat16), None, d.float()], dev_off([5, T // 2, T - 3])
    inside = slice(5, T - 3)
    l = g.logits(bias=False)
    assert torch.equal(l[inside].double(), x[inside].double() @ wg.double())
    assert (l[:5].view(torch.int16) == MARK).all() and (l[T - 3:].view(torch.int16) == MARK).all()
    dx, dwg, db = g.backward()
    assert torch.equal(dx[inside], (d[inside].double() @ wg.T.double().contiguous()).float().to(torch.bfloat16))
    assert (dx[:5].view(torch.int16) == MARK).all() and (dx[T - 3:].view(torch.int16) == MARK).all()
    assert torch.equal(dwg, (x[inside].T.double().contiguous() @ d[inside].double()).float().to(torch.bfloat16))
    assert torch.equal(db.double(), d[inside].double().sum(0))
    assert torch.equal(g.backward(("dx",))[0], dx) and torch.equal(g.backward(("dwg",))[1], dwg)


@pytest.mark.parametrize("T,H,E,plan", GP.GATE, ids=lambda v: str(v)[:24])
def test_gate_in_its_steady_state(B, T, H, E, plan):
    """The same at sizes whose rings and strips go round several times."""
    p = B.moe_gate_plan_host(B.moe_router_config(T, H, E, 1, 2))
    assert {n: getattr(p, n).as_tuple() for n in plan} == plan
    test_gate_by_every_kind_of_tile(B, T, H, E)


@pytest.mark.parametrize("T,H,E", [((1 << 21) + 37, 1088, 60), ((1 << 21) + 37, 1088, 300), (1 << 22, 64, 256)])
def test_gate_elements_past_32_bits(B, T, H, E):
    """More than 2^31 elements (2^32 bytes) of x and dx by every kind of product, and the largest batch of 256 experts,
    whose dlogits in bf16 are 2^31 bytes: whole numbers whose sums are exact, compared in all rows."""
    r = torch.Generator(device="cuda").manual_seed(E)
    whole = lambda *n: torch.randint(-4, 5, n, generator=r, device="cuda", dtype=torch.int8)  # noqa: E731
    x, wg, d = whole(T, H).to(torch.bfloat16), whole(H, E).to(torch.bfloat16), whole(T, E).float()
    cfg = B.moe_router_config(T, H, E, 1, 1)
    ws = torch.empty(max(B.moe_gate_workspace_size(cfg), B.moe_gate_workspace_size(cfg, True)), dtype=torch.uint8, device="cuda")
    l, dx = torch.empty(T, E, device="cuda"), torch.empty_like(x)
    dwg, db = torch.empty_like(wg), torch.empty(E, device="cuda")
    B.moe_gate_logits(cfg, x, wg, None, None, l, ws)
    B.moe_gate_backward(cfg, d, x, wg, None, dx, dwg, db, ws)
    w, sums = wg.double(), torch.zeros(H, E, dtype=torch.float64, device="cuda")
    wt = w.T.contiguous()
    for at in range(0, T, 1 << 18):
        rows = slice(at, min(at + (1 << 18), T))
        xd, dd = x[rows].double(), d[rows].double()
        assert torch.equal(l[rows].double(), xd @ w), at
        assert torch.equal(dx[rows], (dd @ wt).float().to(torch.bfloat16)), at
        sums += xd.T.contiguous() @ dd
    assert torch.equal(dwg, sums.float().to(torch.bfloat16)) and torch.equal(db.double(), d.double().sum(0))


@pytest.mark.parametrize("T,H,E", [(300, 192, 60), (1000, 1088, 128), (700, 256, 300)])
def test_products_of_unrounded_dlogits_by_two_calls(B, T, H, E):
    """dlogits of rows that add up to 0, as a softmax's do, and a gate with a part that all experts share, which cancels: the
    products of dlogits rounded to bf16 and of what that left, added, are those of dlogits to 2^-16 of the terms, where
    one call is off by up to 2^-8 of them."""
    g = Gate(B, T, H, E, seed=14)
    g.wg = (g.wg.float() + 4.0).to(torch.bfloat16)
    g.dl = g.dl - g.dl.mean(1, keepdim=True)
    g.d[1] = g.wg.cuda()
    high = g.dl.to(torch.bfloat16).float()
    parts = []
    for d in (high, g.dl - high):
        g.d[3] = d.cuda()
        parts.append([f64(t) for t in g.backward()])
    g.d[3] = g.dl.cuda()
    one = [f64(t) for t in g.backward()]
    d, x, wg = g.dl.numpy().astype(np.float64), f64(g.x), f64(g.wg)
    for name, exact, terms, n, a, b, c in zip(("dx", "dwg"), (d @ wg.T, x.T @ d), (np.abs(d) @ np.abs(wg).T, np.abs(x).T @ np.abs(d)),
                                              (E, T), *parts, one):
        # each product is rounded to bf16, what is left of the rest is 2^-16 of a term at most, sums are fp32
        check(name, a + b, exact, BF * (np.abs(a) + np.abs(b)) + (2.0 ** -16 + 4 * n * R.F32) * terms + 2 * R.TINY)
        check(name + " by one call", c, exact, BF * np.abs(c) + (BF + 2 * n * R.F32) * terms + R.TINY)
    off = lambda v: np.linalg.norm(v - d @ wg.T) / np.linalg.norm(d @ wg.T)  # noqa: E731
    # evenly spread roundings, 2^-8 / sqrt(3) of a norm at most, of the second product, whose norm is a sixth of dx's or less,
    # and of the first, which is dx but for it: sqrt(1 + 2 / 36) of that of dx
    assert off(parts[0][0] + parts[1][0]) < BF / 3 ** 0.5 * 1.2 < off(one[0])
    db = parts[0][2] + parts[1][2]
    check("dbias", db, d.sum(0), 4 * T * R.F32 * np.abs(d).sum(0))


# ---- losses ---------------------------------------------------------------------------------------------------------
class Loss:
    def __init__(self, B, T, E, k, off=None, S=1, seed=0, scale=1.0):
        rng = np.random.default_rng(seed + T + E)
        self.B, self.T, self.E, self.k, self.S, self.off = B, T, E, k, S, off
        self.cfg = B.moe_router_config(T, 64, E, k, S)
        self.l = (scale * rng.standard_normal((T, E)) - 0.3 * np.log1p(np.arange(E))).astype(np.float32)
        self.idx = np.argsort(-self.l, 1, kind="stable")[:, :k].astype(np.int32)
        self.dw, self.dloss = rng.standard_normal((T, k)).astype(np.float32) * 1e-2, np.array([0.7, 0.02], np.float32)
        self.update()

    def update(self):
        with np.errstate(invalid="ignore", over="ignore"):
            chosen = np.take_along_axis(self.l, np.clip(self.idx, 0, self.E - 1), 1)
            e = np.exp(chosen - chosen.max(1, keepdims=True, initial=np.finfo(np.float32).min))
            self.w = (e / e.sum(1, keepdims=True)).astype(np.float32)
        self.d = {n: torch.from_numpy(v).cuda() for n, v in dict(l=self.l, idx=self.idx, w=self.w, dw=self.dw, dloss=self.dloss).items()}
        self.doff = dev_off(self.off)

    def forward(self, stream=None):
        c, wc = marked(torch.int32, self.S, self.E)
        lse, wl = marked(torch.float32, self.T)
        out, wo = marked(torch.float32, 2)
        ws = torch.full((self.B.moe_route_loss_workspace_size(self.cfg),), 0xA5, dtype=torch.uint8, device="cuda")
        self.B.moe_route_loss(self.cfg, self.d["l"], self.d["idx"], self.doff, c, lse, out, ws, stream)
        torch.cuda.synchronize()
        for t, w in ((c, wc), (lse, wl), (out, wo)):
            clean(w, t.numel(), t.dtype)
        return c, lse, out

    def backward(self, c, lse, weights=True, losses=True, stream=None):
        out, whole = marked(torch.float32, self.T, self.E)
        d = self.d
        self.B.moe_route_loss_backward(self.cfg, d["l"], d["idx"], d["w"] if weights else None, self.doff, c, lse,
                                       d["dloss"] if losses else None, d["dw"] if weights else None, out, stream)
        torch.cuda.synchronize()
        clean(whole, out.numel(), torch.float32)
        return out

    def verify(self, **kw):
        out, o = outside(self.off, self.S, self.T)
        a, b = o[0], o[-1]
        c, lse, loss = self.forward()
        rc, rl, rloss, rel, zb = R.loss(self.l.astype(np.float64), self.idx, o, self.E, self.k)
        assert np.array_equal(c.cpu().numpy(), rc)
        dead = np.isneginf(rl[a:b])
        assert np.array_equal(np.isneginf(f64(lse[a:b])), dead)
        check("lse", f64(lse[a:b])[~dead], rl[a:b][~dead], R.lse_bound(rl[a:b][~dead]))
        assert (lse[out].view(torch.int16) == MARK).all()
        check("loss", f64(loss), np.array(rloss), np.array([rel * rloss[0] + 1e-37, zb]))
        lse[out] = float("nan")
        g = self.backward(c, lse, **kw)
        ref, bound = R.loss_grad(self.l.astype(np.float64), self.idx, self.w.astype(np.float64), o, rc, f64(lse),
                                 self.dloss.astype(np.float64) if kw.get("losses", True) else np.zeros(2),
                                 self.dw.astype(np.float64) if kw.get("weights", True) else None, self.E, self.k)
        check("dlogits", f64(g[a:b]), ref[a:b], bound[a:b])
        assert (g[out].view(torch.int16) == MARK).all()


@pytest.mark.parametrize("E,k", [(1, 1), (2, 1), (2, 2), (7, 3), (8, 2), (60, 6), (64, 8), (65, 1), (128, 8), (200, 5), (256, 8), (511, 7), (512, 8)])
@pytest.mark.parametrize("T", [1, 5, 64, 333])
def test_losses_of_any_size(B, T, E, k):
    Loss(B, T, E, k).verify()


@pytest.mark.parametrize("T", [2, 15, 16, 17, 100, 1023, 1025, 4000])
def test_losses_of_any_rows(B, T):
    Loss(B, T, 128, 8, seed=1).verify()
    Loss(B, T, 6, 2, [0, T // 3, T // 3, T - T // 5], 3, seed=1).verify()


@pytest.mark.parametrize("off", SEQS, ids=str)
def test_losses_of_padded_batches(B, off):
    Loss(B, 256, 60, 4, off, 3, seed=2).verify()


@pytest.mark.parametrize("S,T", [(37, 500), (64, 90), (65, 1100), (512, 700), (512, 5), (300, 1024), (85, 341)])
@pytest.mark.parametrize("E", [7, 8, 48])
def test_many_sequences(B, S, T, E):
    cut = np.sort(np.random.default_rng(S).integers(0, T + 1, S - 1))
    Loss(B, T, E, 3, [0, *cut.tolist(), T], S, seed=3).verify()
    Loss(B, T, E, 3, [T // 4, *np.clip(cut, T // 4, T // 2).tolist(), T // 2], S, seed=3).verify()


@pytest.mark.parametrize("T,E,S", [(1024, 16, 1), (1025, 16, 1), (1024, 17, 1), (128, 128, 32), (128, 128, 33), (32, 512, 8), (33, 512, 8)])
def test_losses_about_the_largest_batch_of_one_workgroup(B, T, E, S):
    Loss(B, T, E, 4, [T * i // S for i in range(S + 1)], S, seed=11).verify()


@pytest.mark.parametrize("kw", [dict(weights=False), dict(losses=False), dict(weights=False, losses=False)])
def test_gradients_of_some(B, kw):
    Loss(B, 130, 60, 6, [0, 50, 129], 2, seed=4).verify(**kw)


def test_large_logits(B):
    Loss(B, 200, 128, 8, seed=5, scale=30.0).verify()


@pytest.mark.parametrize("E", [8, 60, 128, 512])
def test_masked_experts_and_rows_without_any(B, E):
    g = Loss(B, 70, E, 2, [0, 30, 69], 2, seed=6)
    g.l[:, 3] = -np.inf                 # an expert that nobody may choose
    g.l[5, 1:] = -np.inf                # a row with one left
    g.l[7] = -np.inf                    # and with none
    g.l[40] = np.finfo(np.float32).min  # the lowest value everywhere is an even choice
    g.idx[7] = 1 << 30                  # what routing writes where nothing can be chosen
    g.idx[5, 1] = -1
    g.idx[11] = 4                       # the same expert twice
    g.update()
    g.w[7], g.w[5] = 0.0, [1.0, 0.0]
    g.d["w"] = torch.from_numpy(g.w).cuda()
    c, lse, _ = g.forward()
    d = g.backward(c, lse)
    assert not d[7].any() and torch.isfinite(d[:69]).all()
    masked = torch.isneginf(g.d["l"][:69]) & ~(g.d["idx"][:69, :, None] == torch.arange(E, device="cuda")).any(1)
    assert masked.any() and not d[:69][masked].any()
    # (lse^2 of the row of lowest values is infinite in fp32: the mean is taken without it)
    g.l[40] = 0.0
    g.update()
    g.w[7], g.w[5] = 0.0, [1.0, 0.0]
    g.d["w"] = torch.from_numpy(g.w).cuda()
    g.verify()


@pytest.mark.parametrize("E,k", [(1, 1), (8, 2), (60, 6), (128, 8), (200, 5), (300, 8), (511, 3)])
@pytest.mark.parametrize("losses", [True, False])
def test_rows_of_nothing_to_choose_have_no_gradient(B, E, k, losses):
    """Rows of -inf alone, with ids and weights as routing writes them (the smallest ids, NaN) and with finite weights:
    gradient 0 from the losses and from the weights, and the other rows as they are without them."""
    g = Loss(B, 70, E, k, [0, 30, 69], 2, seed=12)
    dead = [0, 7, 29, 68]
    g.l[dead] = -np.inf
    g.idx[dead] = np.arange(k)
    g.update()
    assert np.isnan(g.w[dead]).all()
    g.w[29] = np.linspace(0.1, 0.9, k)
    g.d["w"] = torch.from_numpy(g.w).cuda()
    c, lse, _ = g.forward()
    assert torch.isneginf(lse[dead]).all()
    d = g.backward(c, lse, losses=losses)
    assert not d[dead].any()
    w = g.w.copy()
    w[dead] = 0.0  # for the reference: no weights, no gradient
    ref, bound = R.loss_grad(g.l.astype(np.float64), g.idx, w.astype(np.float64), [0, 30, 69], c.cpu().numpy(), f64(lse),
                             g.dloss.astype(np.float64) if losses else np.zeros(2), g.dw.astype(np.float64), E, k)
    check("dlogits", f64(d[:69]), ref[:69], bound[:69])


@pytest.mark.parametrize("few", [True, False])
def test_gradients_of_experts_that_routing_may_not_choose(B, few):
    """A bias of -inf for all experts but one, or for all: routing fills its choices up with masked ones, of weight 0 (where
    none is left: of weight NaN), and the way back through logits, losses and weights has gradient 0 there."""
    T, H, E, k = 90, 128, 24, 3
    g = Gate(B, T, H, E, seed=13)
    g.d[2].fill_(float("-inf"))
    if few:
        g.d[2][5] = 0.5
    idx, w = torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")
    B.moe_route_topk_static(T, H, E, k, g.d[0], g.d[1], g.d[2], idx, w)
    torch.cuda.synchronize()
    want = torch.tensor([5, 0, 1] if few else [0, 1, 2], device="cuda")
    assert (idx == want).all()
    assert torch.equal(w, torch.tensor([1.0, 0, 0], device="cuda").expand(T, k)) if few else torch.isnan(w).all()
    l = g.logits()
    q = Loss(B, T, E, k)
    q.d.update(l=l, idx=idx, w=w)
    c, lse, loss = q.forward()
    assert (c[0, want.long()] == T).all() and int(c.sum()) == k * T
    # (one expert left has probability 1, exactly, and is chosen by every row; 16 roundings at most in each value)
    assert float(loss[0]) == pytest.approx(E / k if few else 0.0, rel=16 * R.F32)
    d = q.backward(c, lse)
    # by the one logit that is left: z 2 lse / T, the weights none, the balance loss the rounding of c - c
    rest = torch.zeros_like(d)
    if few:
        rest[:, 5] = 2 * 0.02 / T * lse
    torch.testing.assert_close(d, rest, rtol=16 * R.F32, atol=4 * R.F32 * 0.7 * E / (k * T))
    assert not d[:, torch.arange(E) != 5].any()


def test_a_nan_row_is_its_sequences(B):
    g = Loss(B, 90, 60, 4, [0, 40, 90], 2, seed=7)
    c0, lse0, _ = g.forward()
    d0 = g.backward(c0, lse0)
    g.d["l"][50, 7] = float("nan")
    g.d["l"][60, 8] = float("inf")
    c, lse, loss = g.forward()
    assert torch.equal(c, c0) and torch.isnan(lse[50]) and torch.isnan(lse[60]) and torch.isnan(loss).all()
    d = g.backward(c, lse)
    assert torch.isnan(d[50]).any() and torch.isnan(d[60]).any()
    rest = [r for r in range(90) if r not in (50, 60)]
    assert torch.equal(d[rest], d0[rest])


def test_losses_without_rows(B):
    cfg = B.moe_router_config(0, 64, 12, 2, 3)
    e = torch.empty(0, 12, device="cuda")
    c, loss = torch.ones(3, 12, dtype=torch.int32, device="cuda"), torch.ones(2, device="cuda")
    ws = torch.empty(B.moe_route_loss_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    off = dev_off([0, 0, 0, 0])
    i, f = torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    B.moe_route_loss(cfg, e, i, off, c, f, loss, ws)
    assert not c.any() and not loss.any()
    Loss(B, 20, 12, 2, [9, 9, 9, 9], 3).verify()


def test_losses_agree_with_the_routing_of_the_same_logits(B):
    """Counts of moe_route_topk_static's choices, over all sequences, are how often it chose each expert."""
    T, H, E, k = 600, 128, 24, 3
    g = Gate(B, T, H, E, seed=8)
    idx, w = torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")
    B.moe_route_topk_static(T, H, E, k, g.d[0], g.d[1], g.d[2], idx, w)
    l = g.logits()
    assert torch.equal(torch.topk(l, k, 1).indices.int(), idx)
    torch.testing.assert_close(torch.softmax(torch.topk(l, k, 1).values, 1), w, rtol=1e-5, atol=1e-6)
    q = Loss(B, T, E, k, [0, 100, 600], 2)
    q.l, q.idx = l.cpu().numpy(), idx.cpu().numpy()
    q.update()
    q.verify()
    assert torch.equal(q.forward()[0].sum(0).cpu(), torch.bincount(idx.cpu().flatten(), minlength=E).int())


def test_same_bits_on_every_run_stream_and_replay(B):
    g = Loss(B, 2000, 60, 6, [0, 700, 1999], 2, seed=9)
    h = Gate(B, 700, 192, 60, [0, 300, 650], 2, seed=9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def all_of(stream=None):
        c, lse, out = g.forward(stream)
        return [c, lse[:1999], out, g.backward(c, lse, stream=stream)[:1999], h.logits(stream=stream)[:650],
                *[t[:650] for t in h.backward(stream=stream)]]

    first = all_of()
    torch.cuda.synchronize()
    for a, b in zip(first, all_of(s)):
        assert torch.equal(a, b)
    f32 = torch.float32
    out = [torch.empty(2, 60, dtype=torch.int32, device="cuda"), torch.zeros(2000, device="cuda"), torch.empty(2, device="cuda"),
           torch.zeros(2000, 60, device="cuda"), torch.zeros(700, 60, device="cuda"), torch.zeros(700, 192, dtype=torch.bfloat16, device="cuda"),
           torch.empty(192, 60, dtype=torch.bfloat16, device="cuda"), torch.empty(60, dtype=f32, device="cuda")]
    ws = torch.empty(max(B.moe_route_loss_workspace_size(g.cfg), B.moe_gate_workspace_size(h.cfg, True), B.moe_gate_workspace_size(h.cfg)),
                     dtype=torch.uint8, device="cuda")

    def step():  # one workspace for all of them
        B.moe_route_loss(g.cfg, g.d["l"], g.d["idx"], g.doff, out[0], out[1], out[2], ws)
        B.moe_route_loss_backward(g.cfg, g.d["l"], g.d["idx"], g.d["w"], g.doff, out[0], out[1], g.d["dloss"], g.d["dw"], out[3])
        B.moe_gate_logits(h.cfg, h.d[0], h.d[1], h.d[2], h.doff, out[4], ws)
        B.moe_gate_backward(h.cfg, h.d[3], h.d[0], h.d[1], h.doff, out[5], out[6], out[7], ws)

    cg = torch.cuda.CUDAGraph()
    with torch.cuda.graph(cg):
        step()
    rng = np.random.default_rng(4)
    for turn in range(4):
        g.d["l"].copy_(torch.from_numpy(rng.standard_normal((2000, 60)).astype(np.float32)))
        h.d[3].copy_(torch.from_numpy(rng.standard_normal((700, 60)).astype(np.float32)))
        g.doff.copy_(torch.tensor([0, 400 * turn, 1999 - turn], dtype=torch.int32))
        h.doff.copy_(torch.tensor([turn, 300, 650 + turn], dtype=torch.int32))
        for t in out:
            t.zero_()
        cg.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        step()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, out)):
            assert torch.equal(a, b), (turn, i)


def test_binding_refuses_what_does_not_fit(B):
    g = Gate(B, 70, 128, 12, [0, 30, 70], 2)
    out, ws = torch.empty(70, 12, device="cuda"), g.ws(True)
    ok = [g.d[0], g.d[1], g.d[2], g.doff, out, ws]
    for i, bad in [(0, g.d[0][:69]), (0, g.d[0].float()), (1, g.d[1].t().contiguous()), (2, g.d[2][:11]), (3, g.doff[:2]), (3, None),
                   (4, out[:, :11]), (4, out.half()), (5, None), (0, None), (3, g.doff.long())]:
        args = list(ok)
        args[i] = bad
        with pytest.raises(ValueError):
            B.moe_gate_logits(g.cfg, *args)
    with pytest.raises(ValueError):
        B.moe_gate_backward(g.cfg, g.d[3][:60], g.d[0], g.d[1], g.doff, None, None, None, ws)
    q = Loss(B, 70, 12, 2, [0, 30, 70], 2)
    c, lse, loss = q.forward()
    ws = torch.empty(B.moe_route_loss_workspace_size(q.cfg), dtype=torch.uint8, device="cuda")
    ok = [q.d["l"], q.d["idx"], q.doff, c, lse, loss, ws]
    for i, bad in [(0, q.d["l"][:69]), (1, q.d["idx"].long()), (1, q.d["idx"][:, :1]), (3, c[:1]), (4, lse[:69]), (5, loss[:1]), (6, None)]:
        args = list(ok)
        args[i] = bad
        with pytest.raises(ValueError):
            B.moe_route_loss(q.cfg, *args)
    with pytest.raises(B.MoeError):
        B.moe_route_loss(q.cfg, *ok[:6], ws[:256])
    d = torch.empty(70, 12, device="cuda")
    with pytest.raises(B.MoeError):
        B.moe_route_loss_backward(q.cfg, q.d["l"], q.d["idx"], None, q.doff, c, lse, q.d["dloss"], q.d["dw"], d)


def test_elements_past_32_bits(B):
    """2^22 rows of 512 experts: 2^31 logits, 8.6 GB; the gradients take their place."""
    T, E, k = 1 << 22, 512, 2
    cfg = B.moe_router_config(T, 64, E, k, 2)
    l = torch.zeros(T, E, device="cuda")
    tail = Loss(B, 40, E, k, seed=10)
    l[-40:] = tail.d["l"]
    idx = torch.zeros(T, k, dtype=torch.int32, device="cuda")
    idx[-40:] = tail.d["idx"]
    c, lse, loss = torch.empty(2, E, dtype=torch.int32, device="cuda"), torch.empty(T, device="cuda"), torch.empty(2, device="cuda")
    ws = torch.empty(B.moe_route_loss_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    off = dev_off([0, T - 40, T])
    B.moe_route_loss(cfg, l, idx, off, c, lse, loss, ws)
    rc, rl, _, _, _ = R.loss(tail.l.astype(np.float64), tail.idx, [0, 40], E, k)
    assert np.array_equal(c[1].cpu().numpy(), rc[0]) and c[0, 0] == 2 * (T - 40) and not c[0, 1:].any()
    check("lse", f64(lse[-40:]), rl, R.lse_bound(rl))
    w, dw = torch.zeros(T, k, device="cuda"), torch.zeros(T, k, device="cuda")
    w[-40:], dw[-40:] = tail.d["w"], tail.d["dw"]
    B.moe_route_loss_backward(cfg, l, idx, w, off, c, lse, torch.tensor([0.7, 0.0], device="cuda"), dw, l)
    tail.dloss = np.array([0.7 / 2, 0.0], np.float32)  # one of two sequences
    ref, bound = R.loss_grad(tail.l.astype(np.float64), tail.idx, tail.w.astype(np.float64), [0, 40], rc, f64(lse[-40:]),
                             tail.dloss.astype(np.float64), tail.dw.astype(np.float64), E, k)
    check("dlogits", f64(l[-40:]), ref, bound)
