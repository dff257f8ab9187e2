"""CPU tests of the operators over row groups: what the entry points refuse before anything is launched, what the
binding refuses, and the oracle's gradients against differences.  No kernel is launched here."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests import block_plans as PL
from tests import blocks as K

B = pytest.importorskip("paper_2609_21483_amd.binding", reason="libmoe.so not built")
P = C.c_void_p
AT = 1 << 20  # an aligned address that is never read: every call here is refused


def ffn(call="moe_ffn_forward", cfg=(8, 64, 64, 1, 1), off=None, ws_bytes=1 << 30, **ptr):
    """Status of a forward or backward call on made-up addresses."""
    c = B.moe_ffn_config(*cfg)
    names = ["x", "off", "w1", "w3", "w2", "gate", "up", "y"] if call == "moe_ffn_forward" else \
        ["dy", "x", "off", "w1", "w3", "w2", "gate", "up", "dx", "dw1", "dw3", "dw2"]
    at = dict({n: AT for n in names}, off=off, ws=AT)
    at.update(ptr)
    return getattr(B.library(), call)(C.byref(c), *[P(at[n]) for n in names], P(at["ws"]), ws_bytes, P(0))


def gemm(cfg=(8, 64, 64, 1, 0), off=None, ws_bytes=1 << 20, **ptr):
    c = B.moe_gemm_i8_config(*cfg)
    names = ["xq", "sx", "off", "wq", "sw", "y", "ws"]
    at = dict({n: AT for n in names}, off=off)
    at.update(ptr)
    return B.library().moe_gemm_i8(C.byref(c), *[P(at[n]) for n in names], ws_bytes, P(0))


BAD_FFN = [(-1, 64, 64, 1, 1), ((1 << 22) + 1, 64, 64, 1, 1), (8, 0, 64, 1, 1), (8, 96, 64, 1, 1), (8, 16448, 64, 1, 1),
           (8, 64, 32, 1, 1), (8, 64, 32832, 1, 1), (8, 64, 64, 0, 1), (8, 64, 64, 513, 1), (8, 64, 64, 1, 0),
           (8, 64, 64, 1, 3)]


@pytest.mark.parametrize("cfg", BAD_FFN)
def test_ffn_refuses_bad_config(cfg):
    n = C.c_size_t()
    c = B.moe_ffn_config(*cfg)
    assert B.library().moe_ffn_workspace_size(C.byref(c), 0, C.byref(n)) == B.MOE_ERR_INVALID_ARG
    for call in ("moe_ffn_forward", "moe_ffn_backward"):
        assert ffn(call, cfg, off=AT) == B.MOE_ERR_INVALID_ARG
        assert B.moe_last_error()


@pytest.mark.parametrize("call", ["moe_ffn_forward", "moe_ffn_backward"])
@pytest.mark.parametrize("bad", [dict(x=0), dict(w1=0), dict(w3=0), dict(w2=0), dict(up=0), dict(x=AT + 2), dict(w2=AT + 8),
                                 dict(gate=AT + 4), dict(ws=0), dict(ws=AT + 128), dict(ws_bytes=256),
                                 dict(cfg=(8, 64, 64, 2, 1))])
def test_ffn_refuses_bad_arguments(call, bad):
    assert ffn(call, **bad) == B.MOE_ERR_INVALID_ARG, bad
    assert B.moe_last_error()


@pytest.mark.parametrize("bad", [dict(dy=0), dict(gate=0), dict(dw1=0), dict(dw3=0), dict(dw2=0), dict(dw1=0, dw3=0),
                                 dict(dx=AT + 2), dict(dw2=AT + 2)])
def test_backward_refuses_bad_arguments(bad):
    assert ffn("moe_ffn_backward", **bad) == B.MOE_ERR_INVALID_ARG, bad


def test_forward_of_no_rows_is_nothing():
    assert ffn(cfg=(0, 64, 64, 1, 1), x=0, y=0, gate=0, up=0) == B.MOE_OK
    assert gemm((0, 64, 64, 1, 0), xq=0, y=0) == B.MOE_OK
    assert B.library().moe_quantize_rows_i8(0, 64, None, None, None, None) == B.MOE_OK


@pytest.mark.parametrize("cfg", [(-1, 64, 64, 1, 0), (8, 0, 64, 1, 0), (8, 80, 64, 1, 0), (8, 32832, 64, 1, 0),
                                 (8, 64, 0, 1, 0), (8, 64, 12, 1, 0), (8, 64, 24, 1, 1), (8, 64, 65544, 1, 0),
                                 (8, 64, 64, 0, 0), (8, 64, 64, 513, 0), (8, 64, 64, 1, 3), (8, 64, 64, 1, -1)])
def test_gemm_i8_refuses_bad_config(cfg):
    n = C.c_size_t()
    c = B.moe_gemm_i8_config(*cfg)
    assert B.library().moe_gemm_i8_workspace_size(C.byref(c), C.byref(n)) == B.MOE_ERR_INVALID_ARG
    assert gemm(cfg, off=AT) == B.MOE_ERR_INVALID_ARG
    assert B.moe_last_error()


@pytest.mark.parametrize("bad", [dict(xq=0), dict(sx=0), dict(wq=0), dict(sw=0), dict(y=0), dict(ws=0), dict(ws=AT + 64),
                                 dict(ws_bytes=0), dict(xq=AT + 4), dict(wq=AT + 8), dict(y=AT + 2), dict(sx=AT + 4),
                                 dict(cfg=(8, 64, 64, 2, 0))])
def test_gemm_i8_refuses_bad_arguments(bad):
    assert gemm(**bad) == B.MOE_ERR_INVALID_ARG, bad


def test_quantisers_refuse_bad_arguments():
    lib, bad = B.library(), B.MOE_ERR_INVALID_ARG
    for rows, cols in [(-1, 64), ((1 << 22) + 1, 64), (8, 0), (8, 72), (8, 32832)]:
        assert lib.moe_quantize_rows_i8(rows, cols, P(AT), P(AT), P(AT), None) == bad
    for a in [(0, AT, AT), (AT, 0, AT), (AT, AT, 0), (AT + 2, AT, AT), (AT, AT + 1, AT), (AT, AT, AT + 4)]:
        assert lib.moe_quantize_rows_i8(8, 64, *map(P, a), None) == bad
        assert lib.moe_quantize_weights_i8(1, 64, 64, 64, 0, *map(P, a), None) == bad
    for g, k, n, nq, first in [(0, 64, 64, 64, 0), (513, 64, 64, 64, 0), (1, 32, 64, 64, 0), (1, 64, 32, 64, 0),
                               (1, 64, 128, 64, 0), (1, 64, 64, 128, 65), (1, 64, 64, 128, -1), (1, 64, 64, 65600, 0),
                               (1, 32832, 64, 64, 0)]:
        assert lib.moe_quantize_weights_i8(g, k, n, nq, first, P(AT), P(AT), P(AT), None) == bad, (g, k, n, nq, first)


def test_workspace_sizes_grow_with_rows():
    a = B.moe_ffn_workspace_size(B.moe_ffn_config(100, 64, 128, 1, 1))
    b = B.moe_ffn_workspace_size(B.moe_ffn_config(100, 64, 128, 1, 1), True)
    assert a >= 100 * 128 * 2 and b >= 3 * 100 * 128 * 2
    assert B.moe_gemm_i8_workspace_size(B.moe_gemm_i8_config(100, 64, 128, 1, 0)) > 0


def test_binding_refuses_host_memory():
    c = B.moe_ffn_config(8, 64, 64, 1, 1)
    t = torch.zeros(8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU memory"):
        B.moe_ffn_forward(c, t, None, t, t, t, None, None, t, t)
    with pytest.raises(ValueError, match="GPU memory"):
        B.moe_ffn_backward(c, t, t, None, t, t, t, t, t, t, t, t, t, t)
    with pytest.raises(ValueError, match="GPU memory"):
        B.moe_gemm_i8(B.moe_gemm_i8_config(8, 64, 64, 1, 0), t, t, None, t, t, t, t)
    with pytest.raises(ValueError, match="GPU memory"):
        B.moe_quantize_rows_i8(8, 64, t, t, t)
    with pytest.raises(ValueError, match="GPU memory"):
        B.moe_quantize_weights_i8(1, 64, 64, 64, 0, t, t, t)


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_oracle_gradients_match_differences(name):
    """Central differences in 64 bits: with a step of 1e-5, off by about 1e-10 of the gradients' size."""
    rng = np.random.default_rng(5)
    T, H, F, G, off = 9, 6, 10, 3, [0, 4, 4, 8]
    p = dict(x=rng.normal(size=(T, H)), w1=rng.normal(size=(G, H, F)), w3=rng.normal(size=(G, H, F)),
             w2=rng.normal(size=(G, F, H)))
    dy = rng.normal(size=(T, H))

    def loss(q):
        (y, _, _), _ = K.forward(q["x"], off, q["w1"], q["w3"], q["w2"], name, T)
        return np.nansum(y * dy)

    (_, gate, up), _ = K.forward(p["x"], off, p["w1"], p["w3"], p["w2"], name, T)
    grads, _ = K.backward(dy, p["x"], off, p["w1"], p["w3"], p["w2"], gate, up, name)
    for key, g in zip(("x", "w1", "w3", "w2"), grads):
        g = np.nan_to_num(g)
        for i in np.ndindex(*p[key].shape):
            q = {k: v.copy() for k, v in p.items()}
            q[key][i] += 1e-5
            up_ = loss(q)
            q[key][i] -= 2e-5
            assert abs((up_ - loss(q)) / 2e-5 - g[i]) <= 1e-7 * max(1.0, np.abs(g).max()), (key, i)


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_oracle_derivative_of_the_activation(name):
    v = np.linspace(-12, 12, 481)
    a, da, _, _ = K.act(v, name)
    num = (K.act(v + 1e-5, name)[0] - K.act(v - 1e-5, name)[0]) / 2e-5
    assert np.max(np.abs(num - da)) <= 1e-8
    t = torch.from_numpy(v)
    ref = torch.nn.functional.silu(t) if name == "silu" else torch.nn.functional.gelu(t, approximate="tanh")
    assert np.max(np.abs(ref.numpy() - a)) <= 1e-12


@pytest.mark.parametrize("call", [lambda: ffn("moe_ffn_forward", (8, 64, 64, 2, 1), off=AT + 2),
                                  lambda: ffn("moe_ffn_backward", (8, 64, 64, 2, 1), off=AT + 1),
                                  lambda: gemm((8, 64, 64, 2, 0), off=AT + 2)])
def test_offsets_off_their_alignment_are_refused(call):
    assert call() == B.MOE_ERR_INVALID_ARG


BF = torch.bfloat16
G, H, F, T = 2, 64, 192, 6
# (a tensor's shape, the shape that a call wants; a CPU tensor's device is -1)
WHOLE_ROWS = [((G, H, F), (G, H, F)), ((G * H, F), (G, H, F)), ((1, G, H, F), (G, H, F)), ((H, F), (1, H, F)),
              ((G * H * F,), (G, H, F)), ((2, 3, H), (T, H)), ((T, 4, 16), (T, H)), ((1, H), (1, H)), ((H,), (1, H)),
              ((0, H), (0, H)), ((0,), (0, H)), ((0, 7), (0, H)), ((G, H, F, 1), (G, H, F)), ((T, 1), (T,)),
              ((2, 3), (T,)), ((), (1,))]
OTHER_ROWS = [((G, F, H), (G, H, F)), ((F, H), (1, H, F)), ((H, T), (T, H)), ((T * 16, 4), (T, H)),
              ((T // 2, 2 * H), (T, H)), ((T - 1, H), (T, H)), ((T - 1,), (T,)), ((T, H), (-1, H))]


@pytest.mark.parametrize("shape,want", WHOLE_ROWS, ids=str)
def test_binding_takes_tensors_whose_rows_are_whole(shape, want):
    t = torch.zeros(shape, dtype=BF)
    assert B._arg("w", t, BF, want, -1) == t.data_ptr()


@pytest.mark.parametrize("shape,want", OTHER_ROWS, ids=str)
def test_binding_refuses_tensors_of_other_rows(shape, want):
    """Another number of elements, or as many in rows of another length: the weights of torch's Linear, transposed
    rows."""
    with pytest.raises(ValueError, match="of shape"):
        B._arg("w", torch.zeros(shape, dtype=BF), BF, want, -1)


def ffn_plan(*cfg):
    return {n: getattr(B.moe_ffn_plan_host(B.moe_ffn_config(*cfg)), n).as_tuple() for n in ("up", "down", "dh", "dx", "dw")}


def test_plan_queries_refuse_bad_arguments():
    lib = B.library()
    for cfg in BAD_FFN:
        assert lib.moe_ffn_plan_host(C.byref(B.moe_ffn_config(*cfg)), C.byref(B.moe_ffn_plan())) == B.MOE_ERR_INVALID_ARG
    assert lib.moe_ffn_plan_host(C.byref(B.moe_ffn_config(8, 64, 64, 1, 1)), None) == B.MOE_ERR_INVALID_ARG
    assert lib.moe_ffn_plan_host(None, C.byref(B.moe_ffn_plan())) == B.MOE_ERR_INVALID_ARG
    assert lib.moe_gemm_i8_plan_host(C.byref(B.moe_gemm_i8_config(8, 64, 64, 1, 0)), None) == B.MOE_ERR_INVALID_ARG
    assert lib.moe_gemm_i8_plan_host(C.byref(B.moe_gemm_i8_config(8, 64, 12, 1, 0)), C.byref(B.moe_product_plan())) \
        == B.MOE_ERR_INVALID_ARG


@pytest.mark.parametrize("T,H,F,G", [(1, 64, 64, 1), (5, 64, 8192, 1), (5, 8256, 64, 1), (300, 2048, 4096, 1), (3001, 64, 64, 2),
                                     (333, 1024, 2816, 4), (8192, 4096, 14336, 1), (0, 64, 64, 3)])
def test_workspaces_hold_the_parts_of_the_plan(T, H, F, G):
    p = ffn_plan(T, H, F, G, 1)
    parts = lambda n, values: 4 * p[n][1] * values if p[n][1] > 1 else 0
    plane = (2 * T * F + 255) // 256 * 256
    cfg = B.moe_ffn_config(T, H, F, G, 1)
    assert B.moe_ffn_workspace_size(cfg) == 256 + plane + max(parts("up", 2 * T * F), parts("down", T * H))
    assert B.moe_ffn_workspace_size(cfg, True) == 256 + 3 * plane + max(
        parts("dh", T * F), parts("dx", T * H) + parts("dw", 3 * G * H * F))
    for act in (0, 1):
        c = B.moe_gemm_i8_config(T, H, F, G, act)
        s = B.moe_gemm_i8_plan_host(c).split
        assert B.moe_gemm_i8_workspace_size(c) == 256 + (4 * s * T * F if s > 1 else 0)


@pytest.mark.parametrize("H,F", [(4096, 14336), (2048, 8192), (8192, 4096), (1024, 1024)])
def test_a_whole_tile_of_few_rows_is_planned_as_one(H, F):
    """32 rows of one group are one row tile, as 31 are, and 64 are two."""
    a, b = ffn_plan(31, H, F, 1, 1), ffn_plan(32, H, F, 1, 1)
    assert a["up"] == b["up"] and a["down"] == b["down"]
    for act in (0, 1):
        a, b = (B.moe_gemm_i8_plan_host(B.moe_gemm_i8_config(T, H, F, 1, act)).as_tuple() for T in (31, 32))
        assert a == b


@pytest.mark.parametrize("T,H,F,off,act,plan", PL.FFN, ids=lambda v: str(v)[:24])
def test_block_sizes_take_their_plan(T, H, F, off, act, plan):
    assert ffn_plan(T, H, F, PL.groups(off), B.ACTS[act]) == plan


@pytest.mark.parametrize("T,D,N,off,act,plan", PL.I8, ids=lambda v: str(v)[:24])
def test_8_bit_sizes_take_their_plan(T, D, N, off, act, plan):
    assert B.moe_gemm_i8_plan_host(B.moe_gemm_i8_config(T, D, N, PL.groups(off), B.ACTS[act])).as_tuple() == plan


def test_sizes_cover_every_kind_of_tile_in_every_product():
    # (few rows by 4 waves and wide tiles never split the depth, and the products with dy are never of few rows)
    few, big = {("few4", False), ("few8", False), ("few8", True)}, {("small", False), ("small", True), ("wide", False)}
    for n in ("up", "down", "dh", "dx", "dw"):
        kinds = {(p[n][0], p[n][1] > 1) for *_, p in PL.FFN}
        assert kinds == (few | big if n in ("up", "down") else big), n
    for gated in (False, True):
        assert {(p[0], p[1] > 1) for *_, act, p in PL.I8 if (act != "none") == gated} == few | big, gated


def rounded(v):
    return torch.from_numpy(np.asarray(v, np.float32)).to(BF).double().numpy()


@pytest.mark.parametrize("T,H,F,lost", [(290, 512, 2112, 64), (5, 64, 8192, 32)])
def test_norms_show_a_lost_part_of_a_sum(T, H, F, lost):
    """With the library's roundings a result passes K.norms; without a step of one product's depth, or without one
    row of a group, it does not, though every element may be within K.check's bound."""
    rng = np.random.default_rng(T)
    x, dy = rounded(rng.normal(size=(T, H))), rounded(rng.normal(size=(T, H)))
    w1, w3 = (rounded(rng.normal(size=(1, H, F)) * H ** -0.5) for _ in range(2))
    w2 = rounded(rng.normal(size=(1, F, H)) * F ** -0.5)
    (y, gate, up), _ = K.forward(x, None, w1, w3, w2, "gelu", T)
    h = rounded(K.act(gate, "gelu")[0] * up)
    K.norms("y", rounded(h @ w2[0]), y)
    K.norms("gate", rounded(gate), gate)
    for cut in (slice(0, F - lost), slice(lost, F)):
        with pytest.raises(AssertionError):
            K.norms("y", rounded(h[:, cut] @ w2[0][cut]), y)
    # one tile's part alone
    some = rounded(h @ w2[0])
    some[:32, :64] = rounded(h[:32, lost:] @ w2[0][lost:, :64])
    with pytest.raises(AssertionError):
        K.norms("y", some, y)
    dw1 = x.T @ (dy @ w2[0].T)
    K.norms("dw1", rounded(x.T @ rounded(dy @ w2[0].T)), dw1)
    with pytest.raises(AssertionError):
        K.norms("dw1", rounded(x[:-1].T @ rounded(dy @ w2[0].T)[:-1]), dw1)
