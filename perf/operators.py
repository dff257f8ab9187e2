"""The feed-forward operators as timed cases: the gated block over row groups, its backward pass, and the 8-bit
integer product that serves it.

Rows come ordered by group: group g (an expert, or the only one of a dense layer) has rows off[g] .. off[g+1].
``run`` computes a case in its plain form, elementary torch operations in fp32 rounded once, or with ``own`` by
the library's entry points.  A case is a dict of plain values:

what    "forward", "backward" or "int8"
rows    T, the rows of all groups together
hidden  H, the depth of the first product (int8: the depth K)
ffn     F, the block's inner width (int8: the outputs per row: F gated ones of 2F channels, or N plain ones)
groups  G; skew: group sizes are proportional to rank ** -skew (largest remainder), in an order drawn by the seed
act     the gate's activation: "silu" or "gelu" (tanh form); int8 also "none" (no gate)
keep    forward: gate and up are kept for the backward pass;  int8: x comes in bf16 and is quantised in the pass
"""
import math

import torch

own = False

KEYS = ("what", "rows", "hidden", "ffn", "groups", "skew", "act", "keep")


def _case(name, *values):
    return dict(name=name, **dict(zip(KEYS, values)))


def listed():
    return [
        # the smallest layer of the workloads, each expert with a few rows: launches and latency only
        _case("forward_tiny", "forward", 64, 128, 256, 8, 0.0, "silu", False),
        # one token through a wide dense block: its weights are the traffic
        _case("forward_token", "forward", 1, 4096, 14336, 1, 0.0, "silu", False),
        # a decode step over fine-grained experts: a row or two each, some without any
        _case("forward_decode_experts", "forward", 61, 2048, 768, 32, 1.2, "silu", False),
        # a training step's experts at an odd, uneven number of rows, gate and up kept
        _case("forward_experts", "forward", 4531, 2048, 1408, 16, 0.5, "silu", True),
        # a training step's dense block, gate and up kept
        _case("forward_dense", "forward", 8192, 4096, 14336, 1, 0.0, "silu", True),
        # a short batch of odd length over four experts, the other activation: gradients of the weights dominate
        _case("backward_short", "backward", 333, 1024, 2816, 4, 0.5, "gelu", False),
        # fine-grained experts over a full batch, some far longer than others
        _case("backward_experts", "backward", 16384, 2048, 768, 32, 1.2, "silu", False),
        # the dense block's backward pass
        _case("backward_dense", "backward", 8192, 4096, 14336, 1, 0.0, "silu", False),
        # one token served in 8 bits: quantised, then gate and up in one product
        _case("int8_token", "int8", 1, 4096, 14336, 1, 0.0, "silu", True),
        # a decode batch over experts: the down projections, on rows quantised before
        _case("int8_decode_experts", "int8", 133, 1408, 2048, 16, 0.5, "none", False),
        # a ragged prefill over experts: gate and up
        _case("int8_experts", "int8", 6007, 2048, 1408, 16, 0.5, "silu", True),
        # the down projection of a long prefill
        _case("int8_dense", "int8", 16384, 14336, 4096, 1, 0.0, "none", True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        what = rng.choice(["forward", "backward", "int8"])
        rows = log_int(1, 16384)
        hidden, ffn = 64 * log_int(1, 128), 64 * log_int(1, 256)
        groups = rng.choice([1, 1, log_int(2, 64), log_int(2, 64)])
        skew = rng.choice([0.0, 0.5, 1.2])
        act = rng.choice(["silu", "silu", "gelu"] + (["none", "none", "none"] if what == "int8" else []))
        keep = what != "backward" and rng.random() < 0.5
        case = dict(zip(KEYS, (what, rows, hidden, ffn, groups, skew, act, keep)))
        per_row = hidden * ffn * {"forward": 6, "backward": 12, "int8": 2 if act == "none" else 4}[what]
        most = {"forward": 2.8e12, "backward": 5.7e12, "int8": 1.9e12}[what]
        if rows * per_row <= most and hidden * ffn * groups <= 1 << 28:
            return case


def sizes(case):
    """Rows of each group, descending: proportional to rank ** -skew, the largest remainders rounded up."""
    share = [(i + 1.0) ** -case["skew"] for i in range(case["groups"])]
    exact_ = [case["rows"] * s / sum(share) for s in share]
    n = [int(v) for v in exact_]
    for i in sorted(range(len(n)), key=lambda i: (n[i] - exact_[i], i))[:case["rows"] - sum(n)]:
        n[i] += 1
    return n


def _inputs(case, seed):
    """Activations N(0, 1), weights N(0, 0.02^2), gradients N(0, 0.01^2), all bf16; for the 8-bit product rows of
    different magnitudes, and weights quantised for each output channel."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(std, *shape):
        out = torch.empty(*shape, dtype=torch.bfloat16, device="cuda")
        for i in range(shape[0]) if len(shape) == 3 else (slice(None),):
            out[i] = torch.randn(out[i].shape, device="cuda", generator=g).mul_(std)
        return out

    T, H, F, G = case["rows"], case["hidden"], case["ffn"], case["groups"]
    n = sizes(case)
    order = torch.randperm(G, generator=torch.Generator().manual_seed(seed)).tolist()
    off = [0]
    for i in order:
        off.append(off[-1] + n[i])
    st = dict(case=case, off=off, group_off=torch.tensor(off, dtype=torch.int32, device="cuda"), x=normal(1.0, T, H))
    if case["what"] == "int8":
        N = F if case["act"] == "none" else 2 * F
        st["x"] *= torch.exp(torch.randn(T, 1, device="cuda", generator=g)).to(torch.bfloat16)
        st["wq"] = torch.empty(G, N, H, dtype=torch.int8, device="cuda")
        st["w_scale"] = torch.empty(G, N, dtype=torch.float32, device="cuda")
        for i in range(G):
            w = torch.randn(N, H, device="cuda", generator=g).mul_(0.02)
            st["wq"][i], st["w_scale"][i] = quantized(w)
        if not case["keep"]:
            st["xq"], st["x_scale"] = quantized(st.pop("x").float())
        return st
    st["w1"], st["w3"], st["w2"] = normal(0.02, G, H, F), normal(0.02, G, H, F), normal(0.02, G, F, H)
    if case["what"] == "backward":
        # the rows that the forward pass kept
        st["gate"], st["up"] = (torch.empty(T, F, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for i, r in groups(off):
            st["gate"][r] = st["x"][r].float() @ st["w1"][i].float()
            st["up"][r] = st["x"][r].float() @ st["w3"][i].float()
        st["dy"] = normal(0.01, T, H)
    return st


def groups(off):
    """(index, rows) of each group that has rows."""
    return [(i, slice(a, b)) for i, (a, b) in enumerate(zip(off, off[1:])) if b > a]


def quantized(x):
    """Each row of an fp32 matrix in 8 bits: its scale is the largest magnitude / 127, all zeros where that is 0."""
    scale = x.abs().amax(dim=1) / 127.0
    q = torch.where(scale[:, None] > 0, torch.round(x / scale[:, None]), torch.zeros_like(x))
    return q.clamp(-127, 127).to(torch.int8), scale


def activation(g, act):
    """The gate's activation and its derivative."""
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * g * g)


def prepare(case, seed):
    st = _inputs(case, seed)
    if not own:
        return st
    from paper_2609_21483_amd import binding as B

    T, H, F, G = case["rows"], case["hidden"], case["ffn"], case["groups"]
    act = B.ACTS[case["act"]]

    def empty(*shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if case["what"] == "int8":
        N = F if case["act"] == "none" else 2 * F
        st["cfg"] = B.moe_gemm_i8_config(T, H, N, G, act)
        st["ws"] = empty(B.moe_gemm_i8_workspace_size(st["cfg"]), dtype=torch.uint8)
        if case["keep"]:
            st["xq"], st["x_scale"] = empty(T, H, dtype=torch.int8), empty(T, dtype=torch.float32)
        st["y"] = empty(T, F)
        return st
    st["cfg"] = B.moe_ffn_config(T, H, F, G, act)
    st["ws"] = empty(B.moe_ffn_workspace_size(st["cfg"], case["what"] == "backward"), dtype=torch.uint8)
    if case["what"] == "forward":
        st["y"] = empty(T, H)
        st["gate"], st["up"] = (empty(T, F), empty(T, F)) if case["keep"] else (None, None)
    else:
        st["dx"], st["dw1"], st["dw3"], st["dw2"] = empty(T, H), empty(G, H, F), empty(G, H, F), empty(G, F, H)
    return st


def _run_own(s):
    from paper_2609_21483_amd import binding as B

    case = s["case"]
    if case["what"] == "forward":
        B.moe_ffn_forward(s["cfg"], s["x"], s["group_off"], s["w1"], s["w3"], s["w2"], s["gate"], s["up"], s["y"], s["ws"])
        return dict(y=s["y"], gate=s["gate"], up=s["up"]) if case["keep"] else dict(y=s["y"])
    if case["what"] == "backward":
        B.moe_ffn_backward(s["cfg"], s["dy"], s["x"], s["group_off"], s["w1"], s["w3"], s["w2"], s["gate"], s["up"],
                           s["dx"], s["dw1"], s["dw3"], s["dw2"], s["ws"])
        return dict(dx=s["dx"], dw1=s["dw1"], dw3=s["dw3"], dw2=s["dw2"])
    if case["keep"]:
        B.moe_quantize_rows_i8(case["rows"], case["hidden"], s["x"], s["xq"], s["x_scale"])
    B.moe_gemm_i8(s["cfg"], s["xq"], s["x_scale"], s["group_off"], s["wq"], s["w_scale"], s["y"], s["ws"])
    return dict(y=s["y"])


def run(state):
    if own:
        return _run_own(state)
    s, case = state, state["case"]
    T, H, F, act = case["rows"], case["hidden"], case["ffn"], case["act"]
    if case["what"] == "int8":
        xq, x_scale = quantized(s["x"].float()) if case["keep"] else (s["xq"], s["x_scale"])
        y = torch.empty(T, F, dtype=torch.bfloat16, device="cuda")
        for i, r in groups(s["off"]):
            v = (xq[r].float() @ s["wq"][i].float().t()) * (x_scale[r, None] * s["w_scale"][i][None, :])
            y[r] = v if act == "none" else activation(v[:, :F], act)[0] * v[:, F:]
        return dict(y=y)
    if case["what"] == "forward":
        y = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
        kept = [torch.empty(T, F, dtype=torch.bfloat16, device="cuda") for _ in range(2 if case["keep"] else 0)]
        for i, r in groups(s["off"]):
            x = s["x"][r].float()
            gate, up = x @ s["w1"][i].float(), x @ s["w3"][i].float()
            y[r] = (activation(gate, act)[0] * up) @ s["w2"][i].float()
            for t, v in zip(kept, (gate, up)):
                t[r] = v
        return dict(y=y, gate=kept[0], up=kept[1]) if case["keep"] else dict(y=y)
    dx = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    dw1, dw3, dw2 = torch.zeros_like(s["w1"]), torch.zeros_like(s["w3"]), torch.zeros_like(s["w2"])
    for i, r in groups(s["off"]):
        x, dy, up = s["x"][r].float(), s["dy"][r].float(), s["up"][r].float()
        a, da = activation(s["gate"][r].float(), act)
        dh = dy @ s["w2"][i].float().t()
        dgate, dup = dh * up * da, dh * a
        dx[r] = dgate @ s["w1"][i].float().t() + dup @ s["w3"][i].float().t()
        dw1[i], dw3[i], dw2[i] = x.t() @ dgate, x.t() @ dup, (a * up).t() @ dy
    return dict(dx=dx, dw1=dw1, dw3=dw3, dw2=dw2)


def work(case):
    """Weights of the groups that have rows are read once, every gradient of a weight is written."""
    T, H, F, G = case["rows"], case["hidden"], case["ffn"], case["groups"]
    used = sum(1 for n in sizes(case) if n)
    if case["what"] == "forward":
        return {"bytes": 4.0 * T * H + 6.0 * H * F * used + (4.0 * T * F if case["keep"] else 0), "flops": 6.0 * T * H * F}
    if case["what"] == "backward":
        return {"bytes": 6.0 * T * H + 4.0 * T * F + 6.0 * H * F * (used + G), "flops": 12.0 * T * H * F}
    N = F if case["act"] == "none" else 2 * F
    x = 2.0 * T * H if case["keep"] else T * (H + 4.0)
    return {"bytes": x + (H + 4.0) * N * used + 2.0 * T * F, "flops": 2.0 * T * H * N}


def exact(case, seed):
    s = _inputs(case, seed)
    T, H, F, G = case["rows"], case["hidden"], case["ffn"], case["groups"]

    def zeros(*shape):
        return torch.zeros(*shape, dtype=torch.float64, device="cuda")

    def gated(v):
        """act(v) by its definition: v / (1 + e^-v), or v times the normal distribution's tanh form."""
        if case["act"] == "silu":
            return v / (1.0 + (-v).exp())
        return v / (1.0 + (-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)).exp())

    if case["what"] == "int8":
        if case["keep"]:
            # the scale is an fp32 value; quotients are rounded to whole numbers, halves to even
            scale = (s["x"].float().abs().max(dim=1).values / 127.0).double()
            q = s["x"].double().div(scale.where(scale > 0, torch.ones_like(scale))[:, None]).round().clamp(-127, 127)
        else:
            q, scale = s["xq"].double(), s["x_scale"].double()
        y = zeros(T, F)
        for i, (a, b) in enumerate(zip(s["off"], s["off"][1:])):
            v = q[a:b].mul(scale[a:b, None]).matmul(s["wq"][i].double().mul(s["w_scale"][i].double()[:, None]).t())
            y[a:b] = v if case["act"] == "none" else gated(v[:, :F]).mul(v[:, F:])
        return dict(y=y)
    if case["what"] == "forward":
        y, gate, up = zeros(T, H), zeros(T, F), zeros(T, F)
        for i, (a, b) in enumerate(zip(s["off"], s["off"][1:])):
            x = s["x"][a:b].double()
            gate[a:b], up[a:b] = x.matmul(s["w1"][i].double()), x.matmul(s["w3"][i].double())
            y[a:b] = gated(gate[a:b]).mul(up[a:b]).matmul(s["w2"][i].double())
        return dict(y=y, gate=gate, up=up) if case["keep"] else dict(y=y)
    dx, dw1, dw3, dw2 = zeros(T, H), zeros(G, H, F), zeros(G, H, F), zeros(G, F, H)
    for i, (a, b) in enumerate(zip(s["off"], s["off"][1:])):
        x, dy = s["x"][a:b].double(), s["dy"][a:b].double()
        g, u = s["gate"][a:b].double().requires_grad_(), s["up"][a:b].double().requires_grad_()
        with torch.enable_grad():
            h = gated(g).mul(u)
            dg, du = torch.autograd.grad(h, (g, u), dy.matmul(s["w2"][i].double().t()))
        dx[a:b] = dg.matmul(s["w1"][i].double().t()).add_(du.matmul(s["w3"][i].double().t()))
        dw1[i], dw3[i], dw2[i] = x.t().matmul(dg), x.t().matmul(du), h.detach().t().matmul(dy)
    return dict(dx=dx, dw1=dw1, dw3=dw3, dw2=dw2)
