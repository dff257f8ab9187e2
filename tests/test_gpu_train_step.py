"""A training step of a mixture layer by the library: norm, routing, logits, losses, the experts' products, the way
back through all of them and AdamW, against autograd in 64 bits, and captured into a graph."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 1e-5
COEF = (0.05, 0.002)  # of the balance loss and of the z loss


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21483_amd import binding
    return binding


class Step:
    """x + residual -> norm -> gate and experts -> out = sum + experts' outputs, with <out, dout> and the routing's losses
    as the objective.  Rows are gathered and combined by the routing tables."""

    def __init__(self, B, bits, T=384, H=256, F=192, E=12, k=3, off=(0, 100, 300, 370), seed=0):
        g = torch.Generator().manual_seed(seed)
        n = lambda std, *s: (std * torch.randn(*s, generator=g)).to(torch.bfloat16).cuda()  # noqa: E731
        self.B, self.T, self.H, self.F, self.E, self.k, self.off, self.bits = B, T, H, F, E, k, off, bits
        self.x, self.res, self.dout = n(1.0, T, H), n(1.0, T, H), n(0.05, T, H)
        self.dout[off[-1]:] = 0
        self.p = dict(norm=(1 + 0.1 * torch.randn(H, generator=g)).to(torch.bfloat16).cuda(), wg=n(0.05, H, E),
                      w1=n(0.05, E, H, F), w3=n(0.05, E, H, F), w2=n(0.05, E, F, H))
        self.bias = (0.1 * torch.randn(E, generator=g)).cuda()
        e = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
        f32, i32, S = torch.float32, torch.int32, len(off) - 1
        self.ncfg, self.rcfg = B.moe_rms_norm_config(T, H, EPS), B.moe_router_config(T, H, E, k, S)
        self.fcfg = B.moe_ffn_config(T * k, H, F, E, B.MOE_ACT_SILU)
        self.seq_off = torch.tensor(off, dtype=i32, device="cuda")
        self.h = B.moe_init(B.moe_config(1, T, H, F, E, k, E, 0, 0, 0, 0))
        self.table = torch.empty(B.moe_workspace_size(self.h), dtype=torch.uint8, device="cuda")
        B.moe_set_workspace(self.h, self.table)
        lay = B.moe_workspace_layout(self.h)
        view = lambda at, count: self.table[at:at + 4 * count].view(i32)  # noqa: E731
        self.slot, self.inv, self.group_off = view(lay.slot, T * k), view(lay.inv, T * k), view(lay.off, E + 1)
        self.idx, self.w = e(T, k, dtype=i32), e(T, k, dtype=f32)
        self.sum, self.rstd, self.y = e(T, H), e(T, dtype=f32), e(T, H)
        self.logits, self.counts, self.lse, self.loss = e(T, E, dtype=f32), e(S, E, dtype=i32), e(T, dtype=f32), e(2, dtype=f32)
        self.gate, self.up, self.o = e(T * k, F), e(T * k, F), e(T * k, H)
        self.dlogits, self.dyg, self.dxr = e(T, E, dtype=f32), e(T, H), e(T * k, H)
        self.dloss = torch.tensor(COEF, device="cuda")
        self.d = {n_: torch.zeros_like(v) for n_, v in self.p.items()}
        self.d["norm"], self.d["bias"], self.dx = e(H, dtype=f32), e(E, dtype=f32), e(T, H)
        # one workspace for calls that run one after the other
        self.ws = e(max(B.moe_ffn_workspace_size(self.fcfg), B.moe_ffn_workspace_size(self.fcfg, True),
                        B.moe_gate_workspace_size(self.rcfg), B.moe_gate_workspace_size(self.rcfg, True),
                        B.moe_route_loss_workspace_size(self.rcfg), B.moe_rms_norm_workspace_size(self.ncfg)), dtype=torch.uint8)
        self.master = {n_: v.float() for n_, v in self.p.items() if n_ in ("norm", "wg")}
        tensors = []
        for name in ("norm", "wg", "bias", "w1", "w3", "w2"):
            t = dict(grad=self.d[name], weight_decay=0.0 if name in ("norm", "bias") else 0.1)
            w = self.bias if name == "bias" else self.p[name]
            if name == "bias":
                t["master"] = w
            else:
                t["param"] = w
                if name in self.master:
                    t["master"] = self.master[name]
            if bits == 8:
                for s, kind in (("m", torch.float8_e4m3fn), ("v", torch.float8_e5m2)):
                    t[s] = torch.zeros(w.shape, dtype=torch.uint8, device="cuda").view(kind)
                    t[s + "_scale"] = e(-(-w.numel() // 256), dtype=f32)
            else:
                t["m"], t["v"] = torch.zeros(w.shape, device="cuda"), torch.zeros(w.shape, device="cuda")
            tensors.append(t)
        self.states = tensors
        self.list = B.moe_adamw_tensors(tensors, bits)
        self.acfg = B.moe_adamw_config(1e-3, 0.9, 0.99, 1e-8, 1.0, 1, 5, bits)
        self.now = torch.tensor([1e-3, 1.0, 1.0], device="cuda")

    def close(self):
        self.B.moe_destroy(self.h)

    def norm(self):
        self.B.moe_rms_norm_forward(self.ncfg, self.x, self.res, self.p["norm"], self.sum, self.rstd, self.y, None, None)

    def route(self):
        self.B.moe_route(self.h, self.y, self.p["wg"], self.bias, self.k, self.idx, self.w)

    def forward(self):
        B, p = self.B, self.p
        B.moe_gate_logits(self.rcfg, self.y, p["wg"], self.bias, self.seq_off, self.logits, self.ws)
        B.moe_route_loss(self.rcfg, self.logits, self.idx, self.seq_off, self.counts, self.lse, self.loss, self.ws)
        self.token, self.slots = (self.inv // self.k).long(), self.slot.long()
        self.rows = self.y[self.token]
        B.moe_ffn_forward(self.fcfg, self.rows, self.group_off, p["w1"], p["w3"], p["w2"], self.gate, self.up, self.o, self.ws)
        mine = self.o[self.slots].float().view(self.T, self.k, self.H)
        self.out = self.sum.float() + (mine * self.w[:, :, None]).sum(1)
        return mine

    def backward(self, mine):
        B, p, d = self.B, self.p, self.d
        dw = (mine * self.dout.float()[:, None, :]).sum(2)
        do = (self.dout[self.token].float() * self.w.flatten()[self.inv.long()][:, None]).to(torch.bfloat16)
        B.moe_ffn_backward(self.fcfg, do, self.rows, self.group_off, p["w1"], p["w3"], p["w2"], self.gate, self.up, self.dxr,
                           d["w1"], d["w3"], d["w2"], self.ws)
        B.moe_route_loss_backward(self.rcfg, self.logits, self.idx, self.w, self.seq_off, self.counts, self.lse, self.dloss, dw,
                                  self.dlogits)
        B.moe_gate_backward(self.rcfg, self.dlogits, self.y, p["wg"], self.seq_off, self.dyg, d["wg"], d["bias"], self.ws)
        dy = (self.dxr[self.slots].float().view(self.T, self.k, self.H).sum(1) + self.dyg.float()).to(torch.bfloat16)
        B.moe_rms_norm_backward(self.ncfg, dy, self.dout, self.sum, p["norm"], self.rstd, self.dx, d["norm"], self.ws)

    def tensors(self):
        return [self.out, self.loss, self.counts, self.dx, *self.d.values(), *self.p.values(), self.bias,
                *[t[n] for t in self.states for n in ("m", "v")]]


def reference(s):
    """The objective's gradients by autograd in 64 bits, on the routing that the library chose."""
    f = lambda t: t.detach().double().cpu()  # noqa: E731
    p = {n: f(t).requires_grad_() for n, t in s.p.items()}
    bias, total = f(s.bias).requires_grad_(), f(s.sum).requires_grad_()
    y = total * torch.rsqrt((total * total).mean(1, keepdim=True) + EPS) * p["norm"]
    logits = y @ p["wg"] + bias
    idx = s.idx.cpu().long()
    w = torch.softmax(logits.gather(1, idx), 1)
    out = total
    for j in range(s.k):
        rows = []
        for t in range(s.T):
            e = int(idx[t, j])
            v = y[t]
            rows.append((torch.nn.functional.silu(v @ p["w1"][e]) * (v @ p["w3"][e])) @ p["w2"][e])
        out = out + w[:, j:j + 1] * torch.stack(rows)
    losses = torch.zeros(2, dtype=torch.float64)
    spans = [(a, b) for a, b in zip(s.off, s.off[1:]) if b > a]
    prob = torch.softmax(logits, 1)
    for a, b in spans:
        c = torch.bincount(idx[a:b].flatten(), minlength=s.E).double()
        losses[0] = losses[0] + s.E / (s.k * (b - a) ** 2) * (c * prob[a:b].sum(0)).sum() / len(spans)
    losses[1] = (torch.logsumexp(logits[s.off[0]:s.off[-1]], 1) ** 2).mean()
    ((out * f(s.dout)).sum() + COEF[0] * losses[0] + COEF[1] * losses[1]).backward()
    return out.detach(), losses.detach(), total.grad, {**{n: t.grad for n, t in p.items()}, "bias": bias.grad}


# Roundings to bf16 on the way, 2^-8 / sqrt(3) = 2.3e-3 of a 2-norm each: y, gate and up, h, o, do, their gradients, dh,
# dlogits, dxr, dyg, dy and the results; at most 20 of them meet in one result, independently: 1.1e-2
MOST = 20 ** 0.5 * 2.0 ** -8 / 3 ** 0.5


def test_a_steps_gradients_are_autograds(B):
    s = Step(B, 32, T=130, H=128, F=64, E=6, k=2, off=(0, 40, 40, 126))
    try:
        s.norm()
        s.route()
        s.backward(s.forward())
        assert B.moe_sync_status(s.h) == B.MOE_OK
        out, losses, dx, grads = reference(s)
        off = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())  # noqa: E731
        assert off(s.out, out) < MOST and off(s.loss, losses) < MOST
        assert off(s.dx, dx) < MOST
        for n, g in grads.items():
            assert off(s.d[n], g) < MOST, n
        assert torch.equal(s.counts.sum(0).cpu(), torch.bincount(s.idx[:126].cpu().flatten(), minlength=6).int())
    finally:
        s.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_is_the_eager_one(B, bits):
    """Everything behind the routing, the weights' update among it, replayed on new tokens, against eager steps: the same
    bits, whichever of the two has run how often."""
    a, b = Step(B, bits, seed=1), Step(B, bits, seed=1)
    try:
        def rest(s):
            s.backward(s.forward())
            s.B.moe_adamw(s.acfg, s.list, s.now)
            s.now[2:] += 1

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):  # torch's own first calls
            b.norm()
            b.route()
            b.forward()
        torch.cuda.current_stream().wait_stream(side)
        a.norm()
        a.route()
        b.norm()
        b.route()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            rest(b)
        for turn in range(4):
            g = torch.Generator().manual_seed(100 + turn)
            for t in ("x", "res"):
                v = torch.randn(a.T, a.H, generator=g).to(torch.bfloat16)
                getattr(a, t).copy_(v)
                getattr(b, t).copy_(v)
            for s in (a, b):
                s.norm()
                s.route()
            rest(a)
            graph.replay()
            torch.cuda.synchronize()
            for i, (u, v) in enumerate(zip(a.tensors(), b.tensors())):
                assert torch.equal(u.contiguous().view(torch.uint8), v.contiguous().view(torch.uint8)), (turn, i)
        assert float(a.now[2]) == 5.0 and torch.isfinite(a.loss).all()
    finally:
        a.close()
        b.close()


def test_the_balance_gradient_pushes_down_an_expert_that_is_chosen_too_often(B):
    """dlogits of the balance loss alone: above 0 in sum for that expert's column, and 0 over all."""
    s = Step(B, 32, T=256, H=128, F=64, E=8, k=2, off=(0, 256))
    try:
        s.bias[3] = 2.0
        s.dloss.copy_(torch.tensor([1.0, 0.0]))
        s.norm()
        s.route()
        s.forward()
        s.B.moe_route_loss_backward(s.rcfg, s.logits, s.idx, None, s.seq_off, s.counts, s.lse, s.dloss, None, s.dlogits)
        assert s.counts[0, 3] > 2 * s.counts[0].float().mean() and s.loss[0] > 1.05
        assert s.dlogits[:, 3].sum() > 0 and abs(float(s.dlogits.double().sum())) < 1e-4 * float(s.dlogits.double().abs().sum())
    finally:
        s.close()


def test_8_bit_rows_feed_the_8_bit_product(B):
    """moe_rms_norm_forward's q and scale are what moe_gemm_i8 takes: one token, and some."""
    for T in (1, 37):
        H, N = 512, 256
        g = torch.Generator().manual_seed(T)
        x, r, nw = (torch.randn(*v, generator=g).to(torch.bfloat16).cuda() for v in ((T, H), (T, H), (H,)))
        w = (0.05 * torch.randn(1, H, N, generator=g)).to(torch.bfloat16).cuda()
        wq, ws_ = torch.empty(1, N, H, dtype=torch.int8, device="cuda"), torch.empty(1, N, device="cuda")
        B.moe_quantize_weights_i8(1, H, N, N, 0, w, wq, ws_)
        q, scale, total = torch.empty(T, H, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(x)
        B.moe_rms_norm_forward(B.moe_rms_norm_config(T, H, EPS), x, r, nw, total, None, None, q, scale)
        cfg = B.moe_gemm_i8_config(T, H, N, 1, 0)
        y, ws = torch.empty(T, N, dtype=torch.bfloat16, device="cuda"), torch.empty(B.moe_gemm_i8_workspace_size(cfg), dtype=torch.uint8, device="cuda")
        B.moe_gemm_i8(cfg, q, scale, None, wq, ws_, y, ws)
        v = total.double()
        ref = (v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * nw.double()) @ w[0].double()
        # a value's rounding to 8 bits is evenly off by up to half a step, max / 127: with maxima of 4 to 5 standard
        # deviations 1.1e-2 of its norm, for the rows and for the weights
        assert float((y.double() - ref).norm() / ref.norm()) < 2 ** 0.5 * 1.2e-2
        # and the same rows by the quantiser from y in bf16 are a step off at most
        yb = torch.empty_like(x)
        B.moe_rms_norm_forward(B.moe_rms_norm_config(T, H, EPS), x, r, nw, None, None, yb, None, None)
        q2, s2 = torch.empty_like(q), torch.empty_like(scale)
        B.moe_quantize_rows_i8(T, H, yb, q2, s2)
        assert int((q.int() - q2.int()).abs().max()) <= 1


def test_current_stream_handles(B, monkeypatch):
    s = torch.cuda.Stream()
    dev = torch.cuda.current_device()
    for _ in range(2):  # by torch's shortcut, and without it
        assert B._current_stream(dev) == torch.cuda.current_stream(dev).cuda_stream
        with torch.cuda.stream(s):
            assert B._current_stream(dev) == s.cuda_stream
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)


def test_two_batches_at_once_on_two_streams(B):
    """Two batches at once on two streams, each with its own workspace, give what they give alone."""
    one, two = Step(B, 32, seed=3), Step(B, 32, seed=4)
    try:
        want = []
        for s in (one, two):
            s.norm()
            s.route()
            s.backward(s.forward())
            torch.cuda.synchronize()
            want.append([t.clone() for t in s.tensors()])
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for turn in range(3):
            for s, st in zip((one, two), streams):
                st.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(st):
                    s.norm()
                    s.backward(s.forward())
            torch.cuda.synchronize()
            for s, w in zip((one, two), want):
                for u, v in zip(s.tensors(), w):
                    assert np.array_equal(u.contiguous().view(torch.uint8).cpu().numpy(), v.contiguous().view(torch.uint8).cpu().numpy())
    finally:
        one.close()
        two.close()
