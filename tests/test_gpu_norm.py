"""GPU tests of the root-mean-square norm and its backward pass, element by element against 64 bits."""
import numpy as np
import pytest
import torch

from tests import train_ref as R
from tests.blocks import BF, F32, check

pytestmark = pytest.mark.gpu
EPS = 1e-5
MARK = 0x4B4B


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21483_amd import binding
    return binding


def normal(seed, *shape, std=1.0):
    return (std * torch.randn(*shape, generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16)


def marked(n, dtype):
    """A buffer of n values and 64 behind them that nothing may write."""
    size = torch.empty((), dtype=dtype).element_size()
    return torch.full(((n + 64) * size // 2,), MARK, dtype=torch.int16, device="cuda").view(dtype)


def untouched(*bufs_and_sizes):
    for buf, n in bufs_and_sizes:
        assert (buf[n:].view(torch.int16) == MARK).all()


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def forward(B, x, res, w, outs=("sum", "rstd", "y", "q"), stream=None):
    T, H = x.shape
    cfg = B.moe_rms_norm_config(T, H, EPS)
    buf = dict(sum=marked(T * H, torch.bfloat16), rstd=marked(T, torch.float32), y=marked(T * H, torch.bfloat16),
               q=marked(T * H, torch.int8), scale=marked(T, torch.float32))
    n = dict(sum=T * H, rstd=T, y=T * H, q=T * H, scale=T)
    want = set(outs) | ({"scale"} if "q" in outs else set())
    o = {k: buf[k][:n[k]] if k in want else None for k in buf}
    B.moe_rms_norm_forward(cfg, x, res, w, o["sum"], o["rstd"], o["y"], o["q"], o["scale"], stream)
    torch.cuda.synchronize()
    for k in buf:
        untouched((buf[k], n[k] if k in want else 0))
    return {k: v if v is None or v.numel() == T else v.view(T, H) for k, v in o.items()}


def verify(o, x, res, w):
    s, r, y, scale = R.norm(x.float().numpy(), None if res is None else res.float().numpy(), w.float().numpy(), EPS)
    if o["sum"] is not None:
        assert np.array_equal(o["sum"].float().cpu().numpy(), s)
    if o["rstd"] is not None:
        check("rstd", f64(o["rstd"]), r, R.RSTD * r)
    if o["y"] is not None:
        check("y", f64(o["y"]), y, (BF + 2 * R.Y) * np.abs(y) + R.TINY)
    if o["q"] is not None:
        check("scale", f64(o["scale"]), scale, R.SCALE * scale)
        q = f64(o["q"])
        # half a step, and what the quotient of two values that are off is off by
        assert np.abs(q).max() <= 127
        check("q", q * scale[:, None], y, np.broadcast_to(scale[:, None] * (0.5 + 127 * (R.Y + R.SCALE + 2 * F32)) + 1e-45, y.shape))
        assert (np.abs(q).max(1)[scale > 0] == 127).all()


@pytest.mark.parametrize("T,H", [(1, 8), (3, 64), (17, 120), (16, 128), (33, 136), (5, 512), (7, 520), (9, 1000), (4, 1024),
                                 (3, 1032), (5, 2048), (2, 2056), (3, 4096), (2, 4104), (3, 8192), (2, 8200), (2, 16384),
                                 (1, 4096), (259, 64)])
@pytest.mark.parametrize("residual", [True, False])
def test_forward(B, T, H, residual):
    x, w = normal(T, T, H), normal(H, H)
    x *= torch.exp(2 * torch.randn(T, 1, generator=torch.Generator().manual_seed(5))).to(torch.bfloat16)
    res = normal(7, T, H, std=2.0) if residual else None
    verify(forward(B, x.cuda(), None if res is None else res.cuda(), w.cuda()), x, res, w)


@pytest.mark.parametrize("outs", [("y",), ("q",), ("y", "q"), ("sum", "q"), ("rstd", "y"), ("sum", "rstd", "q")])
def test_outputs_that_are_not_wanted_are_not_written(B, outs):
    x, res, w = normal(1, 37, 1024), normal(2, 37, 1024), normal(3, 1024)
    o = forward(B, x.cuda(), res.cuda(), w.cuda(), outs)
    assert {k for k, v in o.items() if v is not None} == set(outs) | ({"scale"} if "q" in outs else set())
    verify(o, x, res, w)


@pytest.mark.parametrize("H", [64, 1000, 4096, 16384])
def test_in_place(B, H):
    T = 19
    x, res, w = normal(1, T, H), normal(2, T, H), normal(3, H)
    cfg = B.moe_rms_norm_config(T, H, EPS)
    ref = forward(B, x.cuda(), res.cuda(), w.cuda())
    for alias in ("residual", "x", "both"):
        a, b = x.cuda(), res.cuda()
        y = a if alias == "both" else torch.empty_like(a)
        B.moe_rms_norm_forward(cfg, a, b, w.cuda(), a if alias == "x" else b, None, y, None, None)
        torch.cuda.synchronize()
        assert torch.equal(a if alias == "x" else b, ref["sum"]) and torch.equal(y, ref["y"])


@pytest.mark.parametrize("H", [64, 768, 4096])
def test_rows_of_special_values(B, H):
    x, w = normal(1, 9, H), normal(2, H)
    x[0] = 0.0
    x[1, 3] = float("inf")
    x[2, 5] = float("nan")
    x[3] = 2.0 ** 100                     # the squares leave fp32
    x[4] = 1e-30                          # and vanish beside eps
    x[5] = -0.0
    x[6, 0] = float("-inf")
    w[1] = 0.0
    o = forward(B, x.cuda(), None, w.cuda())
    y, q, s, r = f64(o["y"]), f64(o["q"]), f64(o["scale"]), f64(o["rstd"])
    assert not y[0].any() and not q[0].any() and s[0] == 0 and not y[5].any() and s[5] == 0
    for row, col in ((1, 3), (6, 0)):
        assert r[row] == 0 and np.isnan(y[row, col]) and not np.delete(y[row], col).any()
        assert np.isnan(s[row]) and not q[row].any()
    assert np.isnan(y[2]).all() and np.isnan(s[2]) and not q[2].any()
    assert r[3] == 0 and not y[3].any() and s[3] == 0 and not q[3].any()
    some = [4, 7, 8]
    verify({k: v[some] for k, v in o.items()}, x[some], None, w)


@pytest.mark.parametrize("H", [128, 1000, 4096, 8200])
def test_a_row_has_the_same_bits_in_any_batch(B, H):
    x, res, w = normal(1, 300, H).cuda(), normal(2, 300, H).cuda(), normal(3, H).cuda()
    dy, dsum = normal(4, 300, H).cuda(), normal(5, 300, H).cuda()
    whole, part = forward(B, x, res, w), forward(B, x[123:130], res[123:130], w)
    for k in whole:
        assert torch.equal(whole[k][123:130], part[k]), k
    a, _ = backward(B, dy, dsum, whole["sum"], w, whole["rstd"])
    b, _ = backward(B, dy[123:130], dsum[123:130], part["sum"], w, part["rstd"].clone())
    assert torch.equal(a[123:130], b)


def backward(B, dy, dsum, s, w, r, want=("dx", "dweight"), stream=None):
    T, H = dy.shape
    cfg = B.moe_rms_norm_config(T, H, EPS)
    dx, dw = marked(T * H, torch.bfloat16), marked(H, torch.float32)
    ws = torch.full((B.moe_rms_norm_workspace_size(cfg),), 0xA5, dtype=torch.uint8, device="cuda")
    B.moe_rms_norm_backward(cfg, dy, dsum, s, w, r, dx[:T * H] if "dx" in want else None, dw[:H] if "dweight" in want else None,
                            ws, stream)
    torch.cuda.synchronize()
    untouched((dx, T * H if "dx" in want else 0), (dw, H if "dweight" in want else 0))
    return dx[:T * H].view(T, H), dw[:H]


@pytest.mark.parametrize("T,H", [(1, 8), (3, 64), (40, 120), (333, 128), (5, 512), (70, 520), (333, 1000), (4, 1024), (1030, 1032),
                                 (5, 2048), (7, 4096), (2, 4104), (3, 8192), (2, 16384), (5000, 64), (2100, 2048)])
@pytest.mark.parametrize("stream", [True, False])
def test_backward(B, T, H, stream):
    s, w, dy = normal(T, T, H, std=3.0), normal(H, H), normal(T + 1, T, H, std=0.01)
    dsum = normal(T + 2, T, H, std=0.01) if stream else None
    r = 1.0 / torch.sqrt(s.float().square().mean(1) + EPS)
    dx, dw = backward(B, dy.cuda(), None if dsum is None else dsum.cuda(), s.cuda(), w.cuda(), r.cuda())
    args = [t.float().numpy().astype(np.float64) if t is not None else None for t in (dy, dsum, s, w, r)]
    rdx, bdx, rdw, bdw = R.norm_grad(*args)
    check("dx", f64(dx), rdx, bdx)
    check("dweight", f64(dw), rdw, bdw)


# at least three passes of the workgroups over the rows, the last one ragged, at every number of threads and loads of a row
LONG = [(40001, 64), (16403, 128), (9001, 512), (3501, 1000), (1801, 2048), (801, 4096), (799, 8192), (601, 16384)]


@pytest.mark.parametrize("T,H", LONG)
def test_backward_over_several_passes(B, T, H):
    test_backward(B, T, H, True)


@pytest.mark.parametrize("T,H", LONG)
def test_rows_of_later_passes_have_the_same_bits_alone(B, T, H):
    dy, dsum, s, w = normal(1, T, H, std=0.01).cuda(), normal(2, T, H, std=0.01).cuda(), normal(3, T, H).cuda(), normal(4, H).cuda()
    r = torch.rand(T, device="cuda") + 0.5
    dx, _ = backward(B, dy, dsum, s, w, r)
    for a, b in ((T // 2 - 3, T // 2 + 4), (T - 7, T)):
        at = slice(a, b)
        assert torch.equal(dx[at], backward(B, dy[at], dsum[at], s[at], w, r[at].clone())[0])


def test_gradients_that_are_not_wanted(B):
    s, w, dy, r = normal(1, 70, 1000).cuda(), normal(2, 1000).cuda(), normal(3, 70, 1000).cuda(), torch.rand(70, device="cuda")
    dx, dw = backward(B, dy, None, s, w, r)
    assert torch.equal(backward(B, dy, None, s, w, r, ("dx",))[0], dx)
    assert torch.equal(backward(B, dy, None, s, w, r, ("dweight",))[1], dw)
    backward(B, dy, None, s, w, r, ())


def test_no_rows_have_no_weight_gradient(B):
    cfg = B.moe_rms_norm_config(0, 72, EPS)
    e = torch.empty(0, 72, dtype=torch.bfloat16, device="cuda")
    dw = torch.full((72,), 3.0, device="cuda")
    ws = torch.empty(B.moe_rms_norm_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    w = torch.ones(72, dtype=torch.bfloat16, device="cuda")
    B.moe_rms_norm_backward(cfg, e, None, e, w, torch.empty(0, device="cuda"), e, dw, ws)
    B.moe_rms_norm_forward(cfg, e, None, w, None, None, e, None, None)
    assert not dw.any()


@pytest.mark.parametrize("alias", ["dy", "dsum", "sum"])
@pytest.mark.parametrize("H", [120, 1000, 4096])
def test_backward_in_place(B, alias, H):
    T = 1500 if H < 4096 else 40
    t = dict(dy=normal(1, T, H).cuda(), dsum=normal(2, T, H).cuda(), sum=normal(3, T, H).cuda())
    w, r = normal(4, H).cuda(), torch.rand(T, device="cuda") + 0.5
    dx, dw = backward(B, t["dy"], t["dsum"], t["sum"], w, r)
    cfg = B.moe_rms_norm_config(T, H, EPS)
    ws = torch.empty(B.moe_rms_norm_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    dw2 = torch.empty_like(dw)
    B.moe_rms_norm_backward(cfg, t["dy"], t["dsum"], t["sum"], w, r, t[alias], dw2, ws)
    assert torch.equal(t[alias], dx) and torch.equal(dw2, dw)


def test_same_bits_on_every_run_stream_and_replay(B):
    T, H = 777, 1536
    x, res, w, dy = normal(1, T, H).cuda(), normal(2, T, H).cuda(), normal(3, H).cuda(), normal(4, T, H).cuda()
    cfg = B.moe_rms_norm_config(T, H, EPS)
    ws = torch.empty(B.moe_rms_norm_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    o = [torch.empty_like(x), torch.empty(T, device="cuda"), torch.empty_like(x), torch.empty(T, H, dtype=torch.int8, device="cuda"),
         torch.empty(T, device="cuda"), torch.empty_like(x), torch.empty(H, device="cuda")]

    def step(stream=None):
        B.moe_rms_norm_forward(cfg, x, res, w, *o[:5], stream)
        B.moe_rms_norm_backward(cfg, dy, o[2], o[0], w, o[1], o[5], o[6], ws, stream)

    step()
    torch.cuda.synchronize()
    first = [t.clone() for t in o]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    step(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, o))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for turn in range(4):
        x.copy_(normal(10 + turn, T, H))
        for t in o:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in o]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, o)), turn


def test_binding_refuses_what_does_not_fit(B):
    x, w, f = normal(1, 8, 64).cuda(), normal(2, 64).cuda(), torch.empty(8, device="cuda")
    q = torch.empty(8, 64, dtype=torch.int8, device="cuda")
    cfg = B.moe_rms_norm_config(8, 64, EPS)
    good = [x, None, w, None, None, x.clone(), None, None]
    for i, bad in [(0, x[:7]), (0, x.float()), (1, x[:, :32]), (2, w[:8]), (3, x.t()), (4, f[:7]), (4, f.double()), (5, x.view(torch.int16)),
                   (0, None), (2, None), (5, x.t().contiguous())]:
        args = list(good)
        args[i] = bad
        with pytest.raises(ValueError):
            B.moe_rms_norm_forward(cfg, *args)
    with pytest.raises(B.MoeError):
        B.moe_rms_norm_forward(cfg, *good[:5], None, None, None)
    with pytest.raises(B.MoeError):
        B.moe_rms_norm_forward(cfg, x, None, w, good[5], None, good[5], None, None)
    with pytest.raises(B.MoeError):
        B.moe_rms_norm_forward(cfg, *good[:5], x.clone(), q, None)
    ws = torch.empty(B.moe_rms_norm_workspace_size(cfg) - 1, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.MoeError):
        B.moe_rms_norm_backward(cfg, x, None, x, w, f, x.clone(), None, ws)
    with pytest.raises(ValueError):
        B.moe_rms_norm_backward(cfg, x, x[:4], x, w, f, x.clone(), None, ws)


def test_elements_past_32_bits(B):
    """2^22 rows of 1032 values: 8.7 GB a tensor, elements and bytes past 2^31 and 2^32."""
    T, H = 1 << 22, 1032
    x = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    tail = normal(1, 5, H)
    x[-5:] = tail.cuda()
    w = normal(2, H)
    y, r = torch.empty_like(x), torch.empty(T, device="cuda")
    B.moe_rms_norm_forward(B.moe_rms_norm_config(T, H, EPS), x, None, w.cuda(), None, r, y, None, None)
    verify(dict(sum=None, rstd=r[-5:], y=y[-5:], q=None, scale=None), tail, None, w)
    assert not y[:1000].any() and not y[T // 2 - 5:T // 2 + 5].any()
    cfg = B.moe_rms_norm_config(T, H, EPS)
    ws = torch.empty(B.moe_rms_norm_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    dw = torch.empty(H, device="cuda")
    B.moe_rms_norm_backward(cfg, y, None, x, w.cuda(), r, y, dw, ws)
    ty = forward(B, tail.cuda(), None, w.cuda())["y"]
    rdx, bdx, rdw, bdw = R.norm_grad(f64(ty), None, f64(tail), f64(w), f64(r[-5:]))
    check("dx", f64(y[-5:]), rdx, bdx)
    check("dweight", f64(dw), rdw, bdw + 20000 * F32 * np.abs(rdw))
