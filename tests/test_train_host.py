"""CPU tests of the norm, the gate, the routing's losses and AdamW: what the entry points and the binding refuse before
anything is launched, the reference's gradients against differences, and the random rounding's statistics.  No kernel
is launched here."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests import gate_plans as GP
from tests import train_ref as R

B = pytest.importorskip("paper_2609_21483_amd.binding", reason="libmoe.so not built")
P = C.c_void_p
AT = 1 << 20  # an aligned address that is never read: every call here is refused

CALLS = {
    "moe_rms_norm_forward": (B.moe_rms_norm_config, (8, 64, 1e-6), ["x", "residual", "weight", "sum", "rstd", "y", "q", "scale"], False),
    "moe_rms_norm_backward": (B.moe_rms_norm_config, (8, 64, 1e-6), ["dy", "dsum", "sum", "weight", "rstd", "dx", "dweight"], True),
    "moe_gate_logits": (B.moe_router_config, (8, 64, 4, 2, 1), ["x", "wg", "bias", "off", "logits"], True),
    "moe_gate_backward": (B.moe_router_config, (8, 64, 4, 2, 1), ["dlogits", "x", "wg", "off", "dx", "dwg", "dbias"], True),
    "moe_route_loss": (B.moe_router_config, (8, 64, 4, 2, 1), ["logits", "idx", "off", "counts", "lse", "loss"], True),
    "moe_route_loss_backward": (B.moe_router_config, (8, 64, 4, 2, 1),
                                ["logits", "idx", "w", "off", "counts", "lse", "dloss", "dw", "dlogits"], False),
}


def call(name, cfg=None, ws_bytes=1 << 30, **ptr):
    """Status of a call on made-up addresses."""
    kind, usual, names, has_ws = CALLS[name]
    c = None if cfg == "none" else C.byref(kind(*(cfg or usual)))
    at = {**{n: AT for n in names}, "ws": AT, **ptr}
    ws = [P(at["ws"]), ws_bytes] if has_ws else []
    for n, k in {"moe_rms_norm_forward": {"sum": 2}, "moe_gate_backward": {"dx": 2, "dwg": 3}}.get(name, {}).items():
        at[n] = k * AT if n not in ptr else at[n]  # (outputs of their own)
    return getattr(B.library(), name)(c, *[P(at[n]) for n in names], *ws, P(0))


@pytest.mark.parametrize("name,cfg", [
    (n, c) for n in ("moe_rms_norm_forward", "moe_rms_norm_backward")
    for c in ["none", (-1, 64, 1e-6), ((1 << 22) + 1, 64, 1e-6), (8, 0, 1e-6), (8, 12, 1e-6), (8, 16392, 1e-6), (8, 64, 0.0),
              (8, 64, -1e-6), (8, 64, float("nan")), (8, 64, float("inf"))]] + [
    (n, c) for n in ("moe_gate_logits", "moe_gate_backward")
    for c in ["none", (-1, 64, 4, 2, 1), ((1 << 22) + 1, 64, 4, 2, 1), (8, 32, 4, 2, 1), (8, 96, 4, 2, 1), (8, 16448, 4, 2, 1),
              (8, 64, 0, 2, 1), (8, 64, 513, 2, 1), (8, 64, 4, 2, 0), (8, 64, 4, 2, 513)]] + [
    (n, c) for n in ("moe_route_loss", "moe_route_loss_backward")
    for c in ["none", (-1, 64, 4, 2, 1), ((1 << 22) + 1, 64, 4, 2, 1), (8, 64, 0, 1, 1), (8, 64, 513, 2, 1), (8, 64, 4, 0, 1),
              (8, 64, 4, 5, 1), (8, 64, 16, 9, 1), (8, 64, 4, 2, 0), (8, 64, 4, 2, 513)]])
def test_bad_configs_are_refused(name, cfg):
    assert call(name, cfg) == B.MOE_ERR_INVALID_ARG
    assert B.moe_last_error()


@pytest.mark.parametrize("name", list(CALLS))
def test_missing_and_misaligned_tensors_are_refused(name):
    optional = {"moe_rms_norm_forward": {"residual", "sum", "rstd"}, "moe_rms_norm_backward": {"dsum", "dx", "dweight"},
                "moe_gate_logits": {"bias", "off"}, "moe_gate_backward": {"off", "dx", "dwg", "dbias"},
                "moe_route_loss": {"off"}, "moe_route_loss_backward": {"off", "dloss"}}[name]
    pair = {"q", "y"} if name == "moe_rms_norm_forward" else set()
    for arg in CALLS[name][2]:
        if arg not in optional | pair:
            assert call(name, **{arg: 0}) == B.MOE_ERR_INVALID_ARG, arg
        step = 2 if arg in ("off", "dloss") else 8
        assert call(name, **{arg: AT + step}) == B.MOE_ERR_INVALID_ARG, arg
        assert B.moe_last_error()
    if CALLS[name][3]:
        for bad in (dict(ws=0), dict(ws=AT + 128), dict(ws_bytes=128)):
            assert call(name, **bad) == B.MOE_ERR_INVALID_ARG, bad
    if "off" in CALLS[name][2]:
        assert call(name, (8, 64, 4, 2, 2), off=0) == B.MOE_ERR_INVALID_ARG


def test_other_refusals():
    assert call("moe_rms_norm_forward", (1 << 22, 8200, 1e-6)) == B.MOE_ERR_INVALID_ARG
    assert b"2^22" in B.library().moe_last_error()
    assert call("moe_rms_norm_forward", sum=AT, y=AT) == B.MOE_ERR_INVALID_ARG
    for same in (dict(dx=AT, x=AT), dict(dx=AT, wg=AT, x=4 * AT), dict(dwg=AT, wg=AT), dict(dwg=AT, x=AT, wg=4 * AT)):
        assert call("moe_gate_backward", **same) == B.MOE_ERR_INVALID_ARG
        assert next(iter(same)).encode() + b" is" in B.library().moe_last_error()
    assert call("moe_rms_norm_forward", y=0, q=0, scale=0) == B.MOE_ERR_INVALID_ARG
    assert call("moe_rms_norm_forward", q=0) == B.MOE_ERR_INVALID_ARG
    assert call("moe_rms_norm_forward", scale=0) == B.MOE_ERR_INVALID_ARG
    assert call("moe_rms_norm_forward", sum=3 * AT, y=3 * AT) == B.MOE_ERR_INVALID_ARG  # outputs on top of each other
    assert call("moe_route_loss_backward", w=0) == B.MOE_ERR_INVALID_ARG
    assert call("moe_route_loss_backward", dw=0) == B.MOE_ERR_INVALID_ARG


def test_calls_of_no_rows_that_write_nothing():
    assert call("moe_rms_norm_forward", (0, 64, 1e-6), x=0, y=0, q=0) == B.MOE_OK
    assert call("moe_gate_logits", (0, 64, 4, 2, 1), x=0, logits=0) == B.MOE_OK
    assert call("moe_route_loss_backward", (0, 64, 4, 2, 1), logits=0, dlogits=0) == B.MOE_OK


@pytest.mark.parametrize("T,E,S", [(0, 1, 1), (1, 512, 512), (1 << 22, 512, 512), (1 << 22, 1, 1), (17, 60, 5)])
def test_workspaces_are_small(T, E, S):
    """A loss's workspace holds the sums of about 1024 tiles and one for each sequence, whatever the batch."""
    c = B.moe_router_config(T, 64, E, 1, S)
    assert B.moe_route_loss_workspace_size(c) <= 8 * (E + 3) * (1024 + S + 8) + 4 * S * (E // 32 + 2) + 4 * (1024 + S) + 4096
    assert B.moe_rms_norm_workspace_size(B.moe_rms_norm_config(T, 64, 1e-6)) <= 256 + 4 * 64 * 16 * 1024


# ---- AdamW ---------------------------------------------------------------------------------------------------------
GOOD = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1, seed=0, state_bits=32)


def adamw(cfg=None, now=0, n=None, **t):
    one = B.moe_adamw_tensor(16, AT, AT, AT, AT, AT, None, None, 0.1, 0)
    for k, v in t.items():
        setattr(one, k, v or None if k not in ("n", "weight_decay", "grad_fp32") else v)
    arr = (B.moe_adamw_tensor * 1)(one)
    return B.library().moe_adamw(None if cfg == "none" else C.byref(B.moe_adamw_config(*{**GOOD, **(cfg or {})}.values())), arr,
                                 1 if n is None else n, P(now), P(0))


@pytest.mark.parametrize("cfg", ["none", dict(lr=-1e-3), dict(lr=float("nan")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
                                 dict(beta2=float("nan")), dict(eps=0.0), dict(eps=1e-16), dict(eps=float("inf")), dict(grad_scale=float("nan")),
                                 dict(grad_scale=float("inf")), dict(step=0), dict(step=-3), dict(state_bits=16),
                                 dict(state_bits=8)])
def test_adamw_refuses_bad_configs(cfg):
    assert adamw(cfg) == B.MOE_ERR_INVALID_ARG
    assert B.moe_last_error()


@pytest.mark.parametrize("bad", [dict(n=-1), dict(n=(1 << 40) + 1), dict(n=(1 << 36) - 4095), dict(param=0, master=0), dict(grad=0), dict(m=0), dict(v=0),
                                 dict(param=AT + 8), dict(master=AT + 8), dict(grad=AT + 8), dict(m=AT + 4), dict(v=AT + 8),
                                 dict(m_scale=AT), dict(v_scale=AT), dict(weight_decay=-0.1), dict(weight_decay=float("nan")),
                                 dict(grad_fp32=2)])
def test_adamw_refuses_bad_tensors(bad):
    if "n" in bad:
        one = (B.moe_adamw_tensor * 1)(B.moe_adamw_tensor(bad["n"], AT, AT, AT, AT, AT, None, None, 0.1, 0))
        st = B.library().moe_adamw(C.byref(B.moe_adamw_config(*GOOD.values())), one, 1, None, None)
    else:
        st = adamw(**bad)
    assert st == B.MOE_ERR_INVALID_ARG and b"tensor 0" in B.library().moe_last_error()


@pytest.mark.parametrize("bad", ["m_scale", "v_scale"])
def test_adamw_refuses_scales_off_their_values(bad):
    assert adamw(dict(state_bits=8), **{**dict(m_scale=AT, v_scale=AT), bad: AT + 2}) == B.MOE_ERR_INVALID_ARG
    assert b"scales" in B.library().moe_last_error()


def test_adamw_of_nothing():
    assert B.library().moe_adamw(C.byref(B.moe_adamw_config(*GOOD.values())), None, 0, None, None) == B.MOE_OK
    assert adamw(n=-1) == B.MOE_ERR_INVALID_ARG
    assert B.library().moe_adamw(C.byref(B.moe_adamw_config(*GOOD.values())), None, 1, None, None) == B.MOE_ERR_INVALID_ARG
    assert adamw(now=AT + 2) == B.MOE_ERR_INVALID_ARG
    empty = (B.moe_adamw_tensor * 2)()
    assert B.library().moe_adamw(C.byref(B.moe_adamw_config(*GOOD.values())), empty, 2, None, None) == B.MOE_OK


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(8, 64, dtype=torch.bfloat16)
    w, f = torch.zeros(64, dtype=torch.bfloat16), torch.zeros(8)
    with pytest.raises(ValueError, match="GPU memory"):
        B.moe_rms_norm_forward(B.moe_rms_norm_config(8, 64, 1e-6), x, None, w, None, None, x, None, None)
    with pytest.raises(ValueError, match="GPU memory"):
        B.moe_rms_norm_backward(B.moe_rms_norm_config(8, 64, 1e-6), x, None, x, w, f, x, None, None)
    c = B.moe_router_config(8, 64, 4, 2, 1)
    with pytest.raises(ValueError, match="GPU memory"):
        B.moe_gate_logits(c, x, x, None, None, f, None)
    with pytest.raises(ValueError, match="GPU memory"):
        B.moe_route_loss(c, f, f, None, f, f, f, None)
    with pytest.raises(ValueError, match="GPU memory"):
        B.moe_adamw_tensors([dict(param=w, grad=w, m=f, v=f)], 32)
    with pytest.raises(ValueError, match="8 or 32"):
        B.moe_adamw_tensors([], 16)


def test_calls_take_the_current_stream_without_torchs_own_shortcut(monkeypatch):
    """A torch that lacks the shortcut to the current stream's handle is asked for the stream itself."""
    import types
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev: types.SimpleNamespace(cuda_stream=0x1230 + dev))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    taken = []
    monkeypatch.setattr(B, "_lib", types.SimpleNamespace(some_call=lambda *a: taken.append(a) or B.MOE_OK))
    B._call("some_call", 3, None, 7)
    assert taken == [(7, 0x1233)]


# ---- the gate's tiles ----------------------------------------------------------------------------------------------
def gate_plan(T, H, E):
    p = B.moe_gate_plan_host(B.moe_router_config(T, H, E, 1, 1))
    return {n: getattr(p, n).as_tuple() for n in ("logits", "dx", "dwg")}


def test_the_gates_plan_query_refuses_bad_arguments():
    lib, out = B.library(), B.moe_gate_plan()
    assert lib.moe_gate_plan_host(None, C.byref(out)) == B.MOE_ERR_INVALID_ARG
    assert lib.moe_gate_plan_host(C.byref(B.moe_router_config(8, 64, 4, 1, 1)), None) == B.MOE_ERR_INVALID_ARG
    for cfg in [(-1, 64, 4, 2, 1), (8, 32, 4, 2, 1), (8, 64, 513, 2, 1), (8, 64, 4, 2, 0)]:
        assert lib.moe_gate_plan_host(C.byref(B.moe_router_config(*cfg)), C.byref(out)) == B.MOE_ERR_INVALID_ARG


@pytest.mark.parametrize("T,H,E,plan", GP.GATE, ids=lambda v: str(v)[:24])
def test_gate_sizes_take_their_plan(T, H, E, plan):
    assert gate_plan(T, H, E) == plan


def test_gate_sizes_cover_every_kind_of_tile_in_its_steady_state():
    """A ring's steady state is reached from its fifth stage on (it holds up to four), a strip's waits from the third
    strip of a part on, and every kind is covered whole and in parts where it has any."""
    from tests import test_gpu_router as G
    known = next(m.args[1] for m in G.test_gate_by_every_kind_of_tile.pytestmark if m.name == "parametrize")
    sizes = sorted({(T, H, E) for T, H, E, *_ in [*known, *GP.GATE]})
    logits, dx, dwg = set(), set(), set()
    for T, H, E in sizes:
        p = gate_plan(T, H, E)
        rows = T - 8  # (of the tests' sequences)
        stages = -(-rows // 64)
        tiles, parts = p["logits"]
        if tiles != "ring" or H // 64 // parts >= 5:
            logits.add((tiles, parts > 1))
        tiles, parts = p["dx"]
        if tiles != "strips":
            dx.add(tiles)
        elif -(-stages // parts) >= 4:
            dx.add((-(-E // 64), p["dwg"][0]))
        tiles, parts = p["dwg"]
        if stages // parts >= 5:
            dwg.add((tiles, parts > 1))
    assert logits >= {("few8", False), ("few8", True), ("few4", False), ("ring", False), ("ring", True), ("small", False), ("small", True),
                      ("wide", False)}
    assert dx >= {"small", "wide", (1, "ring"), (2, "ring"), (3, "ring"), (3, "broad"), (4, "ring"), (4, "broad"), (3, "wide"), (4, "wide")}
    assert dwg >= {("ring", False), ("ring", True), ("broad", True), ("wide", True)}


# ---- the reference -----------------------------------------------------------------------------------------------------
def difference(f, x, d, h=1e-5):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


def test_norm_gradients_are_those_of_differences():
    rng = np.random.default_rng(1)
    s, w, dy, dsum = (rng.standard_normal(n) for n in ((5, 24), 24, (5, 24), (5, 24)))
    eps = 1e-3
    y = lambda s, w: s / np.sqrt((s * s).mean(1, keepdims=True) + eps) * w  # noqa: E731
    r = 1 / np.sqrt((s * s).mean(1) + eps)
    dx, _, dw, _ = R.norm_grad(dy, dsum, s, w, r)
    d, e = rng.standard_normal(s.shape), rng.standard_normal(w.shape)
    assert np.isclose((dx * d).sum(), difference(lambda t: (y(t, w) * dy + t * dsum).sum(), s, d), rtol=1e-7)
    assert np.isclose((dw * e).sum(), difference(lambda t: (y(s, t) * dy).sum(), w, e), rtol=1e-7)


@pytest.mark.parametrize("off", [[0, 9], [0, 3, 3, 8], [2, 5, 7]])
def test_loss_gradients_are_those_of_differences(off):
    rng = np.random.default_rng(2)
    T, E, k = 9, 6, 3
    l = rng.standard_normal((T, E))
    idx = np.argsort(-l, 1)[:, :k]
    dw, dloss = rng.standard_normal((T, k)), np.array([0.7, 0.3])
    chosen = lambda l: np.take_along_axis(l, idx, 1)  # noqa: E731
    weights = lambda l: np.exp(chosen(l)) / np.exp(chosen(l)).sum(1, keepdims=True)  # noqa: E731

    def value(l):
        _, _, both, _, _ = R.loss(l, idx, off, E, k)
        return dloss[0] * both[0] + dloss[1] * both[1] + (weights(l) * dw)[off[0]:off[-1]].sum()

    counts, lse, _, _, _ = R.loss(l, idx, off, E, k)
    g, _ = R.loss_grad(l, idx, weights(l), off, counts, lse, dloss, dw, E, k)
    for _ in range(3):
        d = rng.standard_normal(l.shape)
        assert np.isclose((g * d).sum(), difference(value, l, d), rtol=1e-6, atol=1e-9)


def test_balance_is_one_where_all_is_even():
    l = np.zeros((8, 4))
    idx = np.arange(16).reshape(8, 2) % 4
    assert np.isclose(R.loss(l, idx, [0, 4, 8], 4, 2)[2][0], 1.0)


def test_random_bits_are_even_and_independent():
    """Over 2^18 values: each 16-bit field's mean and its correlation with the others, with the next value's, with
    another tensor's and another step's are within 5 standard errors."""
    n = 1 << 18
    a = R.random_bits(7, 3, 0, n).astype(np.float64) / 65535.0 - 0.5
    b = R.random_bits(7, 3, 1, n).astype(np.float64) / 65535.0 - 0.5
    c = R.random_bits(7, 4, 0, n).astype(np.float64) / 65535.0 - 0.5
    var = 1.0 / 12.0
    assert (np.abs(a.mean(1)) < 5 * (var / n) ** 0.5).all()
    near = 5 * var / n ** 0.5
    for u, v in [(a[0], a[1]), (a[0], a[2]), (a[1], a[2]), (a[0][1:], a[0][:-1]), (a[1][1:], a[1][:-1]), (a[2][256:], a[2][:-256]),
                 (a[0], b[0]), (a[1], b[1]), (a[2], b[2]), (a[0], c[0]), (a[1], c[1]), (a[2], c[2])]:
        assert abs((u * v).mean()) < near


def test_rounding_at_random_keeps_the_mean_and_an_average_alive():
    """v = 1 decays by 0.999 a step, a fortieth of half a step of e5m2 there: the mean of many follows, within 5
    standard errors of rounding noise, where rounding to the nearest would leave it at 1."""
    n, v = 256 * 64, np.ones(256 * 64)
    v[::256] = 1.75  # the block's largest, which stays exact
    for step in range(200):
        v *= 0.999
        v[::256] = 1.75
        scale = R.block_max(v) / 57344.0
        u = R.random_bits(11, step + 1, 0, n)[1]
        v = R.rounded_at_random(v, scale, u, 2, -14, 57344.0, True)[0] * np.repeat(scale, 256)
    rest = np.delete(v, np.arange(0, n, 256))
    assert abs(rest.mean() - 0.999 ** 200) < 5 * rest.std() / len(rest) ** 0.5
