"""GPU tests of the AdamW step: weights and states element by element against 64 bits, 8-bit states against the same
random bits, and their means over many steps."""
import numpy as np
import pytest
import torch

from tests import train_ref as R
from tests.blocks import BF, check

pytestmark = pytest.mark.gpu
MARK = 0x4B
CFG = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, grad_scale=0.5, step=7, seed=1234)


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21483_amd import binding
    return binding


def f64(t):
    return t.float().cpu().numpy().astype(np.float64).ravel()


class Guarded:
    """Tensors on the GPU with 64 bytes behind each that nothing may write."""

    def __init__(self):
        self.all = []

    def put(self, t):
        whole = torch.full((t.nbytes + 64,), MARK, dtype=torch.uint8, device="cuda")
        mine = whole[:t.nbytes].view(t.dtype).view(t.shape)
        mine.copy_(t)
        self.all.append((whole, t.nbytes))
        return mine

    def clean(self):
        assert all((w[n:] == MARK).all() for w, n in self.all)


def encoded(v, most, kind):
    """(8-bit values, scales) of an fp32 tensor, rounded to the nearest."""
    n = v.numel()
    full = torch.zeros(-(-n // 256) * 256)
    full[:n] = v
    scale = full.view(-1, 256).abs().amax(1) / most
    q = (full.view(-1, 256) / scale.clamp(min=1e-30)[:, None]).view(-1)[:n].to(kind)
    return q, scale


def tensor(n, mode, bits, grads, seed, decay=0.1, guard=None):
    """One entry of the list; mode: "both" (bf16 beside fp32), "bf16" or "fp32"."""
    g = torch.Generator().manual_seed(seed + n)
    guard = guard or Guarded()
    w = 0.05 * torch.randn(n, generator=g)
    t = dict(weight_decay=decay)
    if mode != "fp32":
        t["param"] = guard.put(w.to(torch.bfloat16))
    if mode != "bf16":
        t["master"] = guard.put(w)
    t["grad"] = guard.put((1e-3 * torch.randn(n, generator=g)).to(torch.bfloat16 if grads == "bf16" else torch.float32))
    m, v = 3e-4 * torch.randn(n, generator=g), (4e-4 * torch.randn(n, generator=g)).square()
    if bits == 8:
        for name, x, most, kind in (("m", m, 448.0, torch.float8_e4m3fn), ("v", v, 57344.0, torch.float8_e5m2)):
            q, s = encoded(x, most, kind)
            t[name], t[name + "_scale"] = guard.put(q), guard.put(s)
    else:
        t["m"], t["v"] = guard.put(m), guard.put(v)
    return t


def values(t, bits):
    """Weights, gradient and states in float64."""
    w = f64(t["master"] if t.get("master") is not None else t["param"])
    n = len(w)
    if bits == 32:
        return w, f64(t["grad"]), f64(t["m"]), f64(t["v"])
    rep = lambda s: np.repeat(f64(s), 256)[:n]  # noqa: E731
    # (a value times its scale is rounded to fp32)
    state = lambda k: (f64(t[k]) * rep(t[k + "_scale"])).astype(np.float32).astype(np.float64)  # noqa: E731
    return w, f64(t["grad"]), state("m"), state("v")


def config(B, bits, **kw):
    c = {**CFG, **kw}
    return B.moe_adamw_config(c["lr"], c["beta1"], c["beta2"], c["eps"], c["grad_scale"], c["step"], c["seed"], bits), \
        c


def verify(before, t, place, c, bits, decay):
    w, g, m, v = before
    (w1, ew), (m1, em), (v1, ev) = R.adamw(w, g, m, v, c, np.float64(np.float32(decay)))
    n = len(w)
    um, uv, up = R.random_bits(c["seed"], c["step"], place, n)
    if t.get("master") is not None:
        check("master", f64(t["master"]), w1, ew)
        if t.get("param") is not None:
            assert np.array_equal(f64(t["param"]), R.bf16(t["master"].cpu().numpy()).astype(np.float64).ravel())
    else:
        got = f64(t["param"])
        check("param", got, w1, 2 * BF * np.abs(w1) + ew + 2.0 ** -132)
        # the same random bits round the fp32 value: nearly everywhere the same neighbour
        bits32 = w1.astype(np.float32).view(np.uint32)
        same = ((bits32.astype(np.uint64) + up) >> np.uint64(16) << np.uint64(16)).astype(np.uint32).view(np.float32)
        # an fp32 value that is off by ew crosses one of 2^16 thresholds of a step of 2 BF |w| with probability
        # 2 ew / (2 BF |w|) or so
        odds = np.minimum(1.0, 2 * ew / (BF * np.maximum(np.abs(w1), 1e-30))).sum()
        assert (got != same).sum() <= odds + 6 * odds ** 0.5 + 3
    if bits == 32:
        check("m", f64(t["m"]), m1, em)
        check("v", f64(t["v"]), v1, ev)
        return
    for name, x, err, u, mant, least, most in (("m", m1, em, um, 3, -6, 448.0), ("v", v1, ev, uv, 2, -14, 57344.0)):
        scale = R.block_max(x) / most
        gone = R.block_max(x) < 2.0 ** -110
        assert (f64(t[name + "_scale"])[gone] == 0).all()
        scale = np.where(gone, 0.0, scale)
        check(name + "_scale", f64(t[name + "_scale"]), scale, 12 * R.F32 * scale)
        want, unit = R.rounded_at_random(x, scale, u, mant, least, most, name == "v")
        got = f64(t[name])
        rep = np.repeat(scale, 256)[:n]
        # within a step of the exact value, and the reference's neighbour but where an error crosses a threshold
        far = np.abs(got * rep - x) - 1.0001 * unit * rep - err
        assert (far <= 0)[(rep > 0) & ((name == "m") | (x > unit * rep))].all()
        odds = np.minimum(1.0, 2 * (err + 8 * R.F32 * np.abs(x)) / np.maximum(unit * rep, 1e-300) * (rep > 0)).sum()
        assert (got != want).sum() <= odds + 6 * odds ** 0.5 + 3, (name, int((got != want).sum()), odds)
        if name == "v":
            assert (got[(x > 0) & (rep > 0)] > 0).all()


SIZES = [1, 15, 16, 17, 255, 256, 257, 1000, 4095, 4096, 4097, 70001]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("mode", ["both", "bf16", "fp32"])
@pytest.mark.parametrize("grads", ["bf16", "fp32"])
def test_steps_of_any_size(B, bits, mode, grads):
    guard = Guarded()
    ts = [tensor(n, mode, bits, grads, 3, 0.01 * i, guard) for i, n in enumerate(SIZES)]
    before = [values(t, bits) for t in ts]
    grad = [t["grad"].clone() for t in ts]
    cfg, c = config(B, bits)
    B.moe_adamw(cfg, B.moe_adamw_tensors(ts, bits))
    torch.cuda.synchronize()
    guard.clean()
    for i, t in enumerate(ts):
        assert torch.equal(t["grad"], grad[i])
        verify(before[i], t, i, c, bits, 0.01 * i)


@pytest.mark.parametrize("bits", [32, 8])
def test_lists_of_any_length(B, bits):
    """More tensors than one launch takes, of all kinds, empty ones among them."""
    for count in (1, 63, 64, 65, 66, 67, 68, 83, 84, 85, 169, 200):
        guard = Guarded()
        kinds = [("both", "fp32"), ("bf16", "bf16"), ("fp32", "fp32")]
        ts = [tensor((37 * i) % 700 if i % 11 else 0, *[kinds[i % 3][0], bits, kinds[i % 3][1]], i, 0.1, guard) for i in range(count)]
        before = [values(t, bits) for t in ts]
        cfg, c = config(B, bits, step=2)
        B.moe_adamw(cfg, B.moe_adamw_tensors(ts, bits))
        torch.cuda.synchronize()
        guard.clean()
        for i, t in enumerate(ts):
            verify(before[i], t, i, c, bits, 0.1)


@pytest.mark.parametrize("kw", [dict(step=1), dict(step=1 << 24), dict(beta1=0.0), dict(beta2=0.0), dict(lr=0.0), dict(eps=1.0),
                                dict(beta1=0.99999, beta2=0.99999, step=1), dict(grad_scale=0.0), dict(grad_scale=-1e4),
                                dict(seed=0xFFFFFFFF)], ids=str)
@pytest.mark.parametrize("bits", [32, 8])
def test_any_config(B, bits, kw):
    t = tensor(3000, "both", bits, "fp32", 5)
    before = values(t, bits)
    cfg, c = config(B, bits, **kw)
    B.moe_adamw(cfg, B.moe_adamw_tensors([t], bits))
    verify(before, t, 0, c, bits, 0.1)


@pytest.mark.parametrize("grads", ["bf16", "fp32"])
@pytest.mark.parametrize("mode", ["both", "bf16", "fp32"])
@pytest.mark.parametrize("bits", [8, 32])
def test_tensors_that_are_slices_of_one_buffer(B, bits, mode, grads):
    """A model's tensors one behind the other, each from a block on: scales then start at any of four bytes' multiples."""
    sizes = [300, 1, 768, 255, 257, 5000, 4096]
    alone = [tensor(n, mode, bits, grads, seed=40) for n in sizes]
    at = np.cumsum([0] + [-(-n // 256) for n in sizes])
    whole, together = {}, [dict(weight_decay=t["weight_decay"]) for t in alone]
    for k in alone[0]:
        if k == "weight_decay":
            continue
        unit = 1 if k.endswith("_scale") else 256
        whole[k] = torch.full((int(at[-1]) * unit * alone[0][k].element_size(),), MARK, dtype=torch.uint8, device="cuda").view(alone[0][k].dtype)
        for t, u, b in zip(alone, together, at):
            u[k] = whole[k][b * unit:b * unit + t[k].numel()]
            u[k].copy_(t[k])
    before = {k: w.clone() for k, w in whole.items()}
    cfg, _ = config(B, bits)
    for ts in (alone, together):
        B.moe_adamw(cfg, B.moe_adamw_tensors(ts, bits))
    torch.cuda.synchronize()
    for k, w in whole.items():
        unit = 1 if k.endswith("_scale") else 256
        for t, u, b, n in zip(alone, together, at, sizes):
            assert torch.equal(t[k].view(torch.uint8), u[k].view(torch.uint8))
            end, e = b * unit + t[k].numel(), (b + -(-n // 256)) * unit
            assert torch.equal(w[end:e].view(torch.uint8), before[k][end:e].view(torch.uint8))


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_from_zeros(B, bits):
    t = tensor(1000, "both", bits, "fp32", 6)
    for k in ("m", "v", "m_scale", "v_scale"):
        if k in t:
            t[k].view(torch.uint8).zero_()
    t["grad"][256:600] = 0.0
    w0 = t["master"].clone()
    before = values(t, bits)
    cfg, c = config(B, bits, step=1)
    B.moe_adamw(cfg, B.moe_adamw_tensors([t], bits))
    verify(before, t, 0, c, bits, 0.1)
    # where there is no gradient only the decay acts
    torch.testing.assert_close(t["master"][256:600], w0[256:600] * (1 - 1e-2 * 0.1), rtol=1e-6, atol=0)


def test_blocks_of_any_magnitude_in_8_bits(B):
    """Blocks from the largest to the smallest gradients that fp32 holds, of zeros, and with one large value."""
    n = 256 * 12
    t = tensor(n, "fp32", 8, "fp32", 7)
    for k in ("m", "v", "m_scale", "v_scale"):
        t[k].view(torch.uint8).zero_()
    g = torch.randn(n, generator=torch.Generator().manual_seed(1))
    for b, size in enumerate([1e18, 1e10, 1.0, 1e-10, 1e-15, 1e-17, 1e-19, 1e-25, 1e-36, 1e-40, 0.0, 1e-9]):
        g[b * 256:(b + 1) * 256] *= size
    g[256 * 11] = 1e3
    t["grad"].copy_(g)
    before = values(t, 8)
    cfg, c = config(B, 8, step=1, grad_scale=1.0)
    B.moe_adamw(cfg, B.moe_adamw_tensors([t], 8))
    verify(before, t, 0, c, 8, 0.1)
    assert torch.isfinite(t["master"]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_that_are_not_finite(B, bits):
    t = tensor(1024, "both", bits, "fp32", 8)
    ref = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}
    t["grad"][300], t["grad"][700] = float("nan"), float("inf")
    cfg, c = config(B, bits)
    B.moe_adamw(cfg, B.moe_adamw_tensors([t], bits))
    B.moe_adamw(cfg, B.moe_adamw_tensors([ref], bits))
    bad = torch.zeros(1024, dtype=torch.bool)
    bad[[300, 700]] = True
    for k in ("param", "master"):
        got = t[k].cpu()
        assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], ref[k].cpu()[~bad])
    if bits == 32:
        assert not torch.isfinite(t["m"].cpu()[bad]).any() and torch.equal(t["m"].cpu()[~bad], ref["m"].cpu()[~bad])
        return
    # its block is NaN from now on, the others are as without it
    assert torch.isnan(t["m_scale"][[1, 2]]).all() and torch.isnan(t["v_scale"][[1, 2]]).all()
    for a in (slice(0, 256), slice(768, 1024)):
        assert torch.equal(t["m"][a].view(torch.uint8), ref["m"][a].view(torch.uint8))
    assert torch.equal(t["v_scale"][[0, 3]], ref["v_scale"][[0, 3]])
    t["grad"][300], t["grad"][700] = 0.0, 0.0
    B.moe_adamw(cfg, B.moe_adamw_tensors([t], bits))
    assert torch.isnan(t["master"][256:768]).all() and torch.isfinite(t["master"][:256]).all()


def clones(ts):
    return [{k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()} for t in ts]


def equal(a, b):
    return all(torch.equal(x[k].contiguous().view(torch.uint8), y[k].contiguous().view(torch.uint8))
               for x, y in zip(a, b) for k in x if isinstance(x[k], torch.Tensor))


@pytest.mark.parametrize("bits", [32, 8])
def test_scalars_on_the_device(B, bits):
    """now stands for the config's lr, grad_scale and step: the same bits; a NaN grad_scale skips the step."""
    ts = [tensor(n, mode, bits, "fp32", 9) for n, mode in ((700, "bf16"), (5000, "both"))]
    a, b = clones(ts), clones(ts)
    B.moe_adamw(config(B, bits)[0], B.moe_adamw_tensors(a, bits))
    now = torch.tensor([CFG["lr"], CFG["grad_scale"], CFG["step"]], device="cuda")
    other = config(B, bits, lr=0.5, grad_scale=3.0, step=99)[0]
    lst = B.moe_adamw_tensors(b, bits)
    B.moe_adamw(other, lst, now)
    assert equal(a, b)
    keep = clones(b)
    now[1] = float("nan")
    B.moe_adamw(other, lst, now)
    assert equal(keep, b)
    now.copy_(torch.tensor([CFG["lr"], CFG["grad_scale"], -4.0]))
    B.moe_adamw(other, lst, now)
    B.moe_adamw(config(B, bits, step=1)[0], B.moe_adamw_tensors(a, bits))
    assert equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
def test_replays_of_a_captured_step(B, bits):
    ts = [tensor(n, mode, bits, "bf16", 10) for n, mode in ((700, "bf16"), (5000, "both"), (33, "fp32"))]
    eager = clones(ts)
    now = torch.tensor([1e-2, 0.5, 1.0], device="cuda")
    lst, elst = B.moe_adamw_tensors(ts, bits), B.moe_adamw_tensors(eager, bits)
    cfg = config(B, bits)[0]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.moe_adamw(cfg, lst, now)
        now[2] += 1
    now.copy_(torch.tensor([1e-2, 0.5, 1.0]))
    for turn in range(5):
        for t, e in zip(ts, eager):
            t["grad"].copy_(1e-3 * torch.randn(t["grad"].shape, generator=torch.Generator().manual_seed(turn)))
            e["grad"].copy_(t["grad"])
        g.replay()
        torch.cuda.synchronize()
        B.moe_adamw(config(B, bits, step=1 + turn)[0], elst)
        torch.cuda.synchronize()
        assert equal(ts, eager), turn


@pytest.mark.parametrize("step", [(1 << 24) + 1, (1 << 24) + 3, (1 << 30) + 65, (1 << 31) - 1])
@pytest.mark.parametrize("bits", [32, 8])
def test_random_bits_of_steps_that_fp32_does_not_hold(B, bits, step):
    """Every step has random bits of its own, of 32-bit states' bf16 weights and of 8-bit states."""
    t = tensor(9000, "bf16", bits, "fp32", 21)
    before = values(t, bits)
    cfg, c = config(B, bits, step=step)
    B.moe_adamw(cfg, B.moe_adamw_tensors([t], bits))
    verify(before, t, 0, c, bits, 0.1)


def test_another_stream_and_a_second_run(B):
    ts = [tensor(n, "bf16", 8, "bf16", 11) for n in (700, 90000)]
    a, b = clones(ts), clones(ts)
    B.moe_adamw(config(B, 8)[0], B.moe_adamw_tensors(a, 8))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    B.moe_adamw(config(B, 8)[0], B.moe_adamw_tensors(b, 8), None, s)
    torch.cuda.synchronize()
    assert equal(a, b)


def test_8_bit_states_follow_an_average_over_many_steps(B):
    """Constant gradients with betas whose steps are far below half a step of the formats: the means over 64 Ki values
    follow the exact averages within 5 standard errors."""
    n = 1 << 16
    t = tensor(n, "fp32", 8, "fp32", 12)
    g = torch.full((n,), 0.3)
    g[::256] = 1.0  # the blocks' largest
    t["grad"].copy_(g)
    t["m"].copy_(torch.ones(n).to(torch.float8_e4m3fn))
    t["v"].copy_(torch.ones(n).to(torch.float8_e5m2))
    t["m_scale"].fill_(1.0)
    t["v_scale"].fill_(1.0)
    lst = B.moe_adamw_tensors([t], 8)
    steps = 300
    for i in range(steps):
        B.moe_adamw(B.moe_adamw_config(1e-6, 0.998, 0.998, 1e-8, 1.0, i + 1, 5, 8), lst)
    b = 0.998 ** steps
    rest = np.arange(n) % 256 != 0
    for name, at in (("m", 0.3), ("v", 0.09)):
        got = (f64(t[name]) * np.repeat(f64(t[name + "_scale"]), 256))[rest]
        want = b + (1 - b) * at
        assert abs(got.mean() - want) < 5 * got.std() / len(got) ** 0.5 + 1e-5, name


def test_weights_in_bf16_alone_keep_their_mean(B):
    """Steps of a sixteenth of half a step of bf16: a rounding to the nearest would leave every weight at 1."""
    n = 1 << 16
    t = tensor(n, "bf16", 32, "fp32", 13, decay=0.0)
    t["param"].fill_(1.0)
    t["grad"].fill_(1.0)
    t["m"].fill_(1.0)
    t["v"].fill_(1.0)
    lst = B.moe_adamw_tensors([t], 32)
    for i in range(64):
        B.moe_adamw(B.moe_adamw_config(2.0 ** -13, 0.9, 0.99, 1e-8, 1.0, 10000 + i, 5, 32), lst)
    got = f64(t["param"])
    assert abs(got.mean() - (1 - 64 * 2.0 ** -13)) < 5 * got.std() / n ** 0.5


def test_binding_refuses_what_does_not_fit(B):
    def bad(**kw):
        t = tensor(600, "both", 8, "fp32", 14)
        t.update(kw)
        with pytest.raises(ValueError):
            B.moe_adamw_tensors([t], 8)

    t = tensor(600, "both", 8, "fp32", 14)
    for kw in (dict(param=t["param"][:599]), dict(master=t["master"].half()), dict(grad=t["grad"].half()), dict(grad=None),
               dict(param=None, master=None), dict(m=t["m"].view(torch.uint8)), dict(v=t["v"].float()), dict(m_scale=t["m_scale"][:2]),
               dict(m_scale=None), dict(v=None), dict(speed=1.0), dict(param=t["param"].cpu()), dict(m=t["v"]),
               dict(grad=torch.zeros(1200, device="cuda")[::2])):
        bad(**kw)
    with pytest.raises(ValueError):
        B.moe_adamw_tensors([t], 32)
    with pytest.raises(ValueError, match="overlaps"):
        B.moe_adamw_tensors([t, t], 8)
    whole = torch.zeros(2000, device="cuda")
    a, b = tensor(600, "fp32", 32, "fp32", 1), tensor(600, "fp32", 32, "fp32", 2)
    a["master"], b["master"] = whole[:600], whole[512:1112]
    with pytest.raises(ValueError, match="overlaps"):
        B.moe_adamw_tensors([a, b], 32)
    b["master"], b["grad"] = whole[1200:1800], whole[512:1112]
    with pytest.raises(ValueError, match="overlaps"):
        B.moe_adamw_tensors([a, b], 32)
    b["grad"] = a["grad"]  # two may have the same gradient
    lst = B.moe_adamw_tensors([a, b], 32)
    with pytest.raises(ValueError):
        B.moe_adamw(config(B, 8)[0], lst)
    with pytest.raises(ValueError):
        B.moe_adamw(config(B, 32)[0], lst, torch.zeros(2, device="cuda"))
    B.moe_adamw(config(B, 32)[0], B.moe_adamw_tensors([], 32))


@pytest.mark.parametrize("bits", [8, 32])
def test_values_past_32_bits(B, bits):
    """A tensor of 2^32 + 1000 values in 8 bits, of 2^31 + 1000 with states in 32."""
    n = (1 << (32 if bits == 8 else 31)) + 1000
    kinds = dict(m=torch.float8_e4m3fn, v=torch.float8_e5m2) if bits == 8 else dict(m=torch.float32, v=torch.float32)
    big = dict(param=torch.zeros(n, dtype=torch.bfloat16, device="cuda"), grad=torch.zeros(n, dtype=torch.bfloat16, device="cuda"),
               m=torch.zeros(n, dtype=torch.uint8 if bits == 8 else torch.float32, device="cuda").view(kinds["m"]),
               v=torch.zeros(n, dtype=torch.uint8 if bits == 8 else torch.float32, device="cuda").view(kinds["v"]), weight_decay=0.1)
    blocks = -(-n // 256)
    first = (blocks - 5) * 256  # the last 5 blocks
    last = n - first
    src = tensor(last, "bf16", bits, "bf16", 17)
    for k in ("param", "grad", "m", "v"):
        big[k][first:].copy_(src[k]) if not (bits == 8 and k in "mv") else big[k].view(torch.uint8)[first:].copy_(src[k].view(torch.uint8))
    if bits == 8:
        for k in ("m_scale", "v_scale"):
            big[k] = torch.zeros(blocks, device="cuda")
            big[k][-5:] = src[k]
    before = values(src, bits)
    cfg, c = config(B, bits)
    B.moe_adamw(cfg, B.moe_adamw_tensors([big], bits))
    torch.cuda.synchronize()
    (w1, ew), (m1, em), (v1, ev) = R.adamw(*before, c, np.float64(np.float32(0.1)))
    up = R.random_bits(c["seed"], c["step"], 0, last, first)[2]
    got = f64(big["param"][first:])
    same = ((w1.astype(np.float32).view(np.uint32).astype(np.uint64) + up) >> np.uint64(16) << np.uint64(16)).astype(np.uint32).view(np.float32)
    assert (got != same).sum() <= 8 and np.abs(got - w1).max() <= (2 * BF * np.abs(w1) + ew).max()
    if bits == 8:
        assert (f64(big["m_scale"][-5:]) > 0).all() and not big["m_scale"][:1000].any()
    else:
        check("m", f64(big["m"][first:]), m1, em)
    assert not big["param"][:100000].any() and not big["param"][n // 2:n // 2 + 100000].any()


@pytest.mark.parametrize("bits", [8, 32])
def test_states_past_32_bits(B, bits):
    """The states and scales of the last blocks of a tensor of 2^32 + 1000 values in 8 bits, of 2^31 + 1000 in 32, value by
    value; the gradients of the others are 0, and so their states stay."""
    n = (1 << (32 if bits == 8 else 31)) + 1000
    blocks = -(-n // 256)
    first = (blocks - 5) * 256
    src = tensor(n - first, "bf16", bits, "fp32", 18)
    big = dict(weight_decay=0.1)
    for k in ("param", "grad", "m", "v") + (("m_scale", "v_scale") if bits == 8 else ()):
        size = blocks if k.endswith("_scale") else n
        whole = torch.zeros(size * src[k].element_size(), dtype=torch.uint8, device="cuda")
        whole[-src[k].nbytes:] = src[k].view(torch.uint8)
        big[k] = whole.view(src[k].dtype)
    before = values(src, bits)
    cfg, c = config(B, bits)
    B.moe_adamw(cfg, B.moe_adamw_tensors([big], bits))
    torch.cuda.synchronize()
    _, (m1, em), (v1, ev) = R.adamw(*before, c, np.float64(np.float32(0.1)))
    random = R.random_bits(c["seed"], c["step"], 0, n - first, first)
    for name, x, err, u, mant, least, most in (("m", m1, em, random[0], 3, -6, 448.0), ("v", v1, ev, random[1], 2, -14, 57344.0)):
        got = f64(big[name][first:])
        if bits == 32:
            check(name, got, x, err)
        else:
            scale = R.block_max(x) / most
            check(name + "_scale", f64(big[name + "_scale"][-5:]), scale, 12 * R.F32 * scale)
            want, unit = R.rounded_at_random(x, scale, u, mant, least, most, name == "v")
            # the reference's neighbour but where an error crosses one of 2^16 thresholds of a step, and never further than a step
            rep = np.repeat(scale, 256)[:n - first]
            odds = np.minimum(1.0, 2 * (err + 8 * R.F32 * np.abs(x)) / (unit * rep)).sum()
            assert (got != want).sum() <= odds + 6 * odds ** 0.5 + 3
            check(name, got, want, unit)
            assert not big[name + "_scale"][:-5].any()
        for at in range(0, first, 1 << 30):
            assert not big[name][at:min(at + (1 << 30), first)].view(torch.uint8).any()
