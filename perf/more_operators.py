"""What a training step needs around the layer's products, as timed cases: the norm before the layer, the gate's
logits and their gradients, the router's losses, and the optimizer's step.

``run`` computes a case in its plain form, elementary torch operations in fp32 rounded once, or with ``own`` by the
library's entry points.  A case is a dict of plain values; ``what`` says which operator:

norm       root-mean-square norm of x + residual.  rows, hidden; residual: there is one (and the sum is kept);
           out: "bf16" or "i8" (8 bits, a scale for each row); keep: rows' factors are kept for the backward pass
norm_grad  its backward pass.  stream: the sum has a gradient of its own, which is added
logits     the gate's logits.  rows, hidden, experts, seqs, pad: rows behind the last sequence, which are left alone
gate_grad  the gradients of x, of the gate's matrix and of its bias
loss       balance loss and z loss of the routing, counts for each sequence and expert.  top_k
loss_grad  the logits' gradients from the losses' and from that of the routing weights
adamw      a step over many tensors.  tensors, elems: how many, and of how many values together; skew: sizes are
           proportional to rank ** -skew; bits: of the states (32 or 8); master: fp32 weights beside the bf16 ones;
           grads: "bf16" or "fp32"
"""
import math

import torch

own = False

EPS = 1e-6
BETA1, BETA2, ADAM_EPS, LR, DECAY, GRAD_SCALE, FIRST_STEP = 0.9, 0.999, 1e-8, 3e-4, 0.1, 0.5, 1000
BLOCK = 256  # values of an 8-bit state that share a scale


def listed():
    return [
        # one token of a decode step on its way into the 8-bit product: latency only
        dict(name="norm_token_i8", what="norm", rows=1, hidden=4096, residual=True, out="i8", keep=False),
        # a ragged prefill on its way there
        dict(name="norm_prefill_i8", what="norm", rows=6007, hidden=2048, residual=True, out="i8", keep=False),
        # a training step's batch before the layer
        dict(name="norm_train", what="norm", rows=32768, hidden=4096, residual=True, out="bf16", keep=True),
        # a short batch of odd length and width: few rows for the weight's gradient to be summed over
        dict(name="norm_grad_short", what="norm_grad", rows=333, hidden=1000, stream=False),
        # the backward pass of the training step's norm, inside a residual stream
        dict(name="norm_grad", what="norm_grad", rows=32768, hidden=4096, stream=True),
        # the logits of a training step's batch
        dict(name="logits", what="logits", rows=32768, hidden=4096, experts=128, seqs=4, pad=0),
        # an uneven, padded batch, a number of experts that no tile divides
        dict(name="gate_grad_short", what="gate_grad", rows=4531, hidden=2048, experts=60, seqs=5, pad=199),
        # the gradients of the training step's gate
        dict(name="gate_grad", what="gate_grad", rows=32768, hidden=4096, experts=128, seqs=4, pad=0),
        # the losses of a small layer's short batch: launches and latency
        dict(name="loss_short", what="loss", rows=333, experts=8, top_k=2, seqs=3, pad=20),
        # the gradient of a training step's routing, sixteen sequences
        dict(name="loss_grad", what="loss_grad", rows=32768, experts=128, top_k=8, seqs=16, pad=0),
        # the small tensors of a stack (norms, biases, gates of small layers) in one step
        dict(name="adamw_small", what="adamw", tensors=150, elems=3000000, skew=1.0, bits=32, master=True, grads="fp32"),
        # all experts of a layer, states in 8 bits
        dict(name="adamw_experts", what="adamw", tensors=96, elems=603979776, skew=0.0, bits=8, master=False, grads="bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        what = rng.choice(["norm", "norm_grad", "logits", "gate_grad", "loss", "loss_grad", "adamw"])
        rows = log_int(1, 32768)
        if what in ("norm", "norm_grad"):
            case = dict(what=what, rows=rows, hidden=8 * log_int(8, 1024))
            if what == "norm":
                case |= dict(residual=rng.random() < 0.7, out=rng.choice(["bf16", "i8"]), keep=rng.random() < 0.5)
            else:
                case |= dict(stream=rng.random() < 0.7)
        elif what == "adamw":
            tensors = log_int(1, 400)
            case = dict(what=what, tensors=tensors, elems=max(tensors, log_int(100, 300000000)), skew=rng.choice([0.0, 0.5, 1.0]),
                        bits=rng.choice([8, 32]), master=rng.random() < 0.5, grads=rng.choice(["bf16", "fp32"]))
        else:
            experts = rng.choice([log_int(2, 512), 8 * log_int(1, 64)])
            case = dict(what=what, rows=rows, experts=experts)
            if what in ("logits", "gate_grad"):
                case |= dict(hidden=64 * log_int(1, 128))
            else:
                case |= dict(top_k=rng.randint(1, min(experts, 8)))
            case |= dict(seqs=rng.choice([1, 1, log_int(1, 64)]), pad=rng.choice([0, rows // rng.randint(2, 20)]))
        w = work(case)
        if w["bytes"] <= 6.0e9 and w["flops"] <= 8.0e10 and rows * case.get("hidden", 0) <= 1 << 27:
            return case


def offsets(case):
    """Where the sequences start and end: lengths grow, the first may be empty, and rows behind the last are padding."""
    n, used = case["seqs"], case["rows"] - case["pad"]
    return [used * i * (i + 1) // (n * (n + 1)) for i in range(n)] + [used]


def tensor_sizes(case):
    share = [(i + 1.0) ** -case["skew"] for i in range(case["tensors"])]
    return [max(1, int(case["elems"] * s / sum(share))) for s in share]


def starts(case):
    """Where each tensor starts in the buffer that holds all of them, on a block's boundary, and the buffer's size."""
    at = [0]
    for n in tensor_sizes(case):
        at.append(at[-1] + -(-n // BLOCK) * BLOCK)
    return at


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, std, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, device="cuda", generator=g).mul_(std).to(dtype)


def _empty(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def _zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def _inputs(case, seed):
    """Activations N(0, 1) whose rows have different magnitudes, weights N(0, 0.02^2), norm weights about 1, gradients
    N(0, 0.01^2).  Outputs that leave rows alone are zero before."""
    g = _generator(seed)
    what, f32 = case["what"], torch.float32
    st = dict(case=case)
    if what in ("norm", "norm_grad"):
        T, H = case["rows"], case["hidden"]
        st["weight"] = (1.0 + 0.1 * torch.randn(H, device="cuda", generator=g)).to(torch.bfloat16)
        st["x"] = _normal(g, 1.0, T, H)
        st["x"] *= torch.exp(torch.randn(T, 1, device="cuda", generator=g)).to(torch.bfloat16)
        if what == "norm":
            st["residual"] = _normal(g, 2.0, T, H) if case["residual"] else None
            st["sum"] = _empty(T, H) if case["residual"] else None
            st["rstd"] = _empty(T, dtype=f32) if case["keep"] else None
            st["y"] = _empty(T, H)  # out = "i8": the values that q stands for
            st["q"], st["scale"] = (_empty(T, H, dtype=torch.int8), _empty(T, dtype=f32)) if case["out"] == "i8" else (None, None)
        else:
            st["rstd"] = 1.0 / torch.sqrt(st["x"].float().square().mean(1) + EPS)
            st["dy"] = _normal(g, 0.01, T, H)
            st["dsum"] = _normal(g, 0.01, T, H) if case["stream"] else None
            st["dx"], st["dweight"] = _empty(T, H), _empty(H, dtype=f32)
        return st
    if what == "adamw":
        at = starts(case)
        n = at[-1]
        st["step"], st["seed"], st["at"] = FIRST_STEP, seed & 0x7FFFFFFF, torch.tensor(at[:-1], device="cuda")
        weights = _normal(g, 0.02, n, dtype=f32)
        st["master"], st["param"] = weights if case["master"] else None, weights.to(torch.bfloat16)
        del weights
        st["grad"] = _normal(g, 1e-3, n, dtype=f32 if case["grads"] == "fp32" else torch.bfloat16)
        st["m"] = _normal(g, 2e-4, n, dtype=f32)
        st["v"] = _normal(g, 5e-4, n, dtype=f32).square_().add_(1e-8)
        for i, size in enumerate(tensor_sizes(case)):  # what lies between the tensors is 0 and stays so
            for name in ("param", "master", "grad", "m", "v") if at[i] + size < at[i + 1] else ():
                if st[name] is not None:
                    st[name][at[i] + size:at[i + 1]] = 0
        if case["bits"] == 8:
            for name, most, kind in (("m", 448.0, torch.float8_e4m3fn), ("v", 57344.0, torch.float8_e5m2)):
                t = st[name].view(-1, BLOCK)
                st[name + "_scale"] = t.abs().amax(1) / most
                st[name] = (t / st[name + "_scale"].clamp(min=1e-30)[:, None]).clamp_(-most, most).to(kind).view(-1)
        return st
    T, E, off = case["rows"], case["experts"], offsets(case)
    st["off"], st["seq_off"] = off, torch.tensor(off, dtype=torch.int32, device="cuda")
    if what in ("logits", "gate_grad"):
        H = case["hidden"]
        st["x"], st["wg"] = _normal(g, 1.0, T, H), _normal(g, 0.02, H, E)
        if what == "logits":
            st["bias"], st["logits"] = _normal(g, 0.5, E, dtype=f32), _zeros(T, E, dtype=f32)
        else:
            st["dlogits"] = _normal(g, 1e-4, T, E, dtype=f32)
            st["dx"], st["dwg"], st["dbias"] = _zeros(T, H), _empty(H, E), _empty(E, dtype=f32)
        return st
    k, S = case["top_k"], case["seqs"]
    prior = -0.5 * torch.log(1.0 + torch.randperm(E, device="cuda", generator=g))
    st["logits"] = torch.randn(T, E, device="cuda", generator=g) + prior
    top, idx = torch.sort(st["logits"], dim=1, descending=True, stable=True)
    st["topk_idx"] = idx[:, :k].to(torch.int32).contiguous()
    if what == "loss":
        st["counts"], st["lse"], st["loss"] = _empty(S, E, dtype=torch.int32), _zeros(T, dtype=f32), _empty(2, dtype=f32)
        return st
    st["topk_w"] = torch.softmax(top[:, :k], 1).contiguous()
    st["lse"] = torch.logsumexp(st["logits"], 1)
    chosen = torch.zeros(T, E, device="cuda").scatter_(1, st["topk_idx"].long(), 1.0)
    st["counts"] = torch.stack([chosen[a:b].sum(0) for a, b in zip(off, off[1:])]).to(torch.int32)
    st["dtopk_w"] = _normal(g, 1e-3, T, k, dtype=f32)
    st["dloss"] = torch.tensor([1e-2, 1e-3], device="cuda")
    st["dlogits"] = _zeros(T, E, dtype=f32)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if not own:
        return st
    # the config, the workspace and the list of tensors that a program keeps
    from paper_2609_21483_amd import binding as B

    what = case["what"]
    ws = 0
    if what in ("norm", "norm_grad"):
        st["cfg"] = B.moe_rms_norm_config(case["rows"], case["hidden"], EPS)
        ws = B.moe_rms_norm_workspace_size(st["cfg"]) if what == "norm_grad" else 0
    elif what == "adamw":
        st["cfg"] = B.moe_adamw_config(LR, BETA1, BETA2, ADAM_EPS, GRAD_SCALE, st["step"], st["seed"], case["bits"])
        at = starts(case)
        part = lambda name, i, n: None if st.get(name) is None else st[name][at[i]:at[i] + n]  # noqa: E731
        scale = lambda name, i: None if st.get(name) is None else st[name][at[i] // BLOCK:at[i + 1] // BLOCK]  # noqa: E731
        st["tensors"] = B.moe_adamw_tensors([
            dict(param=part("param", i, n), master=part("master", i, n), grad=part("grad", i, n), m=part("m", i, n),
                 v=part("v", i, n), m_scale=scale("m_scale", i), v_scale=scale("v_scale", i), weight_decay=DECAY)
            for i, n in enumerate(tensor_sizes(case))], case["bits"])
    else:
        st["cfg"] = B.moe_router_config(case["rows"], case.get("hidden", 64), case["experts"], case.get("top_k", 1), case["seqs"])
        if what in ("logits", "gate_grad"):
            ws = B.moe_gate_workspace_size(st["cfg"], what == "gate_grad")
        elif what == "loss":
            ws = B.moe_route_loss_workspace_size(st["cfg"])
    st["ws"] = _empty(ws, dtype=torch.uint8)
    return st


def _run_own(s):
    from paper_2609_21483_amd import binding as B

    case, what = s["case"], s["case"]["what"]
    if what == "norm":
        i8 = case["out"] == "i8"
        B.moe_rms_norm_forward(s["cfg"], s["x"], s["residual"], s["weight"], s["sum"], s["rstd"], None if i8 else s["y"],
                               s["q"], s["scale"])
    elif what == "norm_grad":
        B.moe_rms_norm_backward(s["cfg"], s["dy"], s["dsum"], s["x"], s["weight"], s["rstd"], s["dx"], s["dweight"], s["ws"])
    elif what == "logits":
        B.moe_gate_logits(s["cfg"], s["x"], s["wg"], s["bias"], s["seq_off"], s["logits"], s["ws"])
    elif what == "gate_grad":
        B.moe_gate_backward(s["cfg"], s["dlogits"], s["x"], s["wg"], s["seq_off"], s["dx"], s["dwg"], s["dbias"], s["ws"])
    elif what == "loss":
        B.moe_route_loss(s["cfg"], s["logits"], s["topk_idx"], s["seq_off"], s["counts"], s["lse"], s["loss"], s["ws"])
    elif what == "loss_grad":
        B.moe_route_loss_backward(s["cfg"], s["logits"], s["topk_idx"], s["topk_w"], s["seq_off"], s["counts"], s["lse"],
                                  s["dloss"], s["dtopk_w"], s["dlogits"])
    else:
        s["step"] += 1
        s["cfg"].step = s["step"]
        B.moe_adamw(s["cfg"], s["tensors"])


def _outputs(s):
    case, what = s["case"], s["case"]["what"]
    if what == "norm":
        if case["out"] == "i8":  # the values that the 8 bits stand for
            torch.mul(s["q"], s["scale"][:, None], out=s["y"])
        return {n: s[n] for n in ("sum", "rstd", "y", "scale") if s[n] is not None}
    if what == "adamw":
        names = ("param", "m", "v") + (("master",) if case["master"] else ()) + (("m_scale", "v_scale") if case["bits"] == 8 else ())
        return {n: s[n] for n in names}
    return {n: s[n] for n in {"norm_grad": ("dx", "dweight"), "logits": ("logits",), "gate_grad": ("dx", "dwg", "dbias"),
                              "loss": ("counts", "lse", "loss"), "loss_grad": ("dlogits",)}[what]}


def _members(s):
    """[S][n] ones where a row belongs to a sequence (of the rows that have one), and the sequences' lengths."""
    a, b = s["off"][0], s["off"][-1]
    row = torch.arange(a, b, device="cuda")[None, :]
    member = ((row >= s["seq_off"][:-1, None]) & (row < s["seq_off"][1:, None])).float()
    return member, member.sum(1)


def _mixed(h):
    """32 bits whose every bit depends on all of h's, modulo 2^32 (int64 tensors or numbers)."""
    mask = 0xFFFFFFFF
    h = ((h ^ (h >> 16)) * 0x761BCE4B) & mask
    h = ((h ^ (h >> 15)) * 0xA0D73955) & mask
    return h ^ (h >> 16)


def _random_bits(seed, step, tensor, i):
    """The random 32 bits of value i of a tensor in a step, of which the lower half rounds m and the upper v, and the 16
    that round its weight."""
    mask = 0xFFFFFFFF
    key = _mixed((_mixed((seed + step * 0xD22CD251) & mask) + tensor * 0xA5375919) & mask)
    h = _mixed((key + (i & mask) * 0x946BAFCD + (i >> 32) * 0x8952E2D3) & mask)
    return h, ((h * 0x761BCE4B) & mask) >> 16


def _steps(x, u, bits, least):
    """x >= 0 in whole steps of a floating format of `bits` bits of mantissa and normal exponents from `least` on, and
    its step there: rounded up with the probability that leaves the mean right (u: uniform in [0, 1))."""
    e = torch.frexp(x)[1] - 1
    unit = torch.ldexp(torch.ones_like(x), e.clamp(min=least) - bits)
    return torch.floor(x / unit + u), unit


def _adamw(s):
    case = s["case"]
    s["step"] += 1
    n = s["param"].numel()
    bits8 = case["bits"] == 8
    decode = lambda name: (s[name].float().view(-1, BLOCK) * s[name + "_scale"][:, None]).view(-1) if bits8 else s[name]  # noqa: E731
    g = s["grad"].float() * GRAD_SCALE
    m = BETA1 * decode("m") + (1.0 - BETA1) * g
    v = BETA2 * decode("v") + (1.0 - BETA2) * (g * g)
    c1, c2 = 1.0 - BETA1 ** s["step"], 1.0 - BETA2 ** s["step"]
    p = s["master"] if case["master"] else s["param"].float()
    p = p - LR * (DECAY * p + (m / c1) / (torch.sqrt(v / c2) + ADAM_EPS))
    if bits8 or not case["master"]:
        i = torch.arange(n, device="cuda")
        tensor = torch.bucketize(i, s["at"], right=True) - 1
        h, hp = _random_bits(s["seed"], s["step"], tensor, i - s["at"][tensor])
        del tensor, i
    if case["master"]:
        s["master"].copy_(p)
        s["param"].copy_(p)
    else:  # rounded up or down at random
        s["param"].copy_((((p.view(torch.int32) + hp.int()) >> 16) << 16).view(torch.float32))
        del hp
    if not bits8:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return
    for name, t, u, most, bits, least in (("m", m, h & 0xFFFF, 448.0, 3, -6), ("v", v, h >> 16, 57344.0, 2, -14)):
        scale = t.abs().view(-1, BLOCK).amax(1) / most
        x = (t.abs().view(-1, BLOCK) * torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))[:, None]).view(-1)
        steps, unit = _steps(x, u.float() / 65536.0, bits, least)
        if name == "v":  # what is not 0 does not become 0: it is divided by
            steps = torch.where(x > 0, steps.clamp(min=1.0), steps)
        s[name].copy_(torch.copysign((steps * unit).clamp(max=most), t).to(s[name].dtype))
        s[name + "_scale"].copy_(scale)


def run(state):
    s, case = state, state["case"]
    what = case["what"]
    if own:
        _run_own(s)
        return _outputs(s)
    if what == "norm":
        v = s["x"].float()
        if case["residual"]:
            s["sum"].copy_(v + s["residual"].float())
            v = s["sum"].float()
        r = 1.0 / torch.sqrt(v.square().mean(1) + EPS)
        if case["keep"]:
            s["rstd"].copy_(r)
        y = v * r[:, None] * s["weight"].float()
        if case["out"] == "bf16":
            s["y"].copy_(y)
        else:
            s["scale"].copy_(y.abs().amax(1) / 127.0)
            q = torch.where(s["scale"][:, None] > 0, torch.round(y / s["scale"][:, None]), torch.zeros_like(y))
            s["q"].copy_(q.clamp(-127, 127))
    elif what == "norm_grad":
        n, dy = s["x"].float() * s["rstd"][:, None], s["dy"].float()
        g = dy * s["weight"].float()
        dx = s["rstd"][:, None] * (g - n * (g * n).mean(1, keepdim=True))
        s["dx"].copy_(dx + s["dsum"].float() if case["stream"] else dx)
        s["dweight"].copy_((dy * n).sum(0))
    elif what == "logits":
        a, b = s["off"][0], s["off"][-1]
        s["logits"][a:b] = s["x"][a:b].float() @ s["wg"].float() + s["bias"]
    elif what == "gate_grad":
        a, b = s["off"][0], s["off"][-1]
        d = s["dlogits"][a:b]
        s["dx"][a:b] = d @ s["wg"].float().t()
        s["dwg"].copy_(s["x"][a:b].float().t() @ d)
        s["dbias"].copy_(d.sum(0))
    elif what in ("loss", "loss_grad"):
        a, b, E, k = s["off"][0], s["off"][-1], case["experts"], case["top_k"]
        member, n = _members(s)
        live, few = n > 0, n.clamp(min=1.0)
        logits, idx = s["logits"][a:b], s["topk_idx"][a:b]
        chosen = idx[:, :, None] == torch.arange(E, device="cuda")[None, None, :]
        if what == "loss":
            top = logits.amax(1)
            e = torch.exp(logits - top[:, None])
            total = e.sum(1)
            lse = torch.log(total) + top
            counts = member @ chosen.float().sum(1)
            balance = (counts * (member @ (e / total[:, None]))).sum(1) * E / (k * few * few)
            s["counts"].copy_(counts)
            s["lse"][a:b] = lse
            # no rows at all: no loss
            s["loss"].copy_(torch.stack([torch.where(live, balance, 0.0).sum() / live.sum().clamp(min=1),
                                         lse.square().sum() / n.sum().clamp(min=1.0)]))
        else:
            lse, w, dw = s["lse"][a:b], s["topk_w"][a:b], s["dtopk_w"][a:b]
            p = torch.exp(logits - lse[:, None])
            factor = s["dloss"][0] * E / (k * few * few * live.sum())
            c = member.t() @ (s["counts"].float() * factor[:, None])
            d = p * (c - (c * p).sum(1, keepdim=True)) + (s["dloss"][1] * 2.0 / n.sum()) * lse[:, None] * p
            dt = w * (dw - (w * dw).sum(1, keepdim=True))
            s["dlogits"][a:b] = d + (chosen.float() * dt[:, :, None]).sum(1)
    else:
        _adamw(s)
    return _outputs(s)


def work(case):
    what = case["what"]
    if what == "norm":
        n = float(case["rows"]) * case["hidden"]
        b = 2 * n + 2 * case["hidden"] + (4 * n if case["residual"] else 0) + (4 * case["rows"] if case["keep"] else 0)
        return {"bytes": b + (2 * n if case["out"] == "bf16" else n + 4 * case["rows"]), "flops": 5 * n}
    if what == "norm_grad":
        n = float(case["rows"]) * case["hidden"]
        return {"bytes": (8 if case["stream"] else 6) * n + 6.0 * case["hidden"] + 4.0 * case["rows"], "flops": 10 * n}
    if what == "adamw":
        n = float(sum(tensor_sizes(case)))
        states = 16 * n if case["bits"] == 32 else 4 * n + 16 * n / BLOCK
        return {"bytes": states + n * (4 if case["grads"] == "fp32" else 2) + n * (10 if case["master"] else 4), "flops": 15 * n}
    T, E = float(case["rows"] - case["pad"]), case["experts"]
    if what == "logits":
        return {"bytes": 2 * T * case["hidden"] + 2 * case["hidden"] * E + 4 * T * E, "flops": 2 * T * case["hidden"] * E}
    if what == "gate_grad":
        return {"bytes": 4 * T * case["hidden"] + 4 * case["hidden"] * E + 4 * T * E, "flops": 4 * T * case["hidden"] * E}
    k, S = case["top_k"], case["seqs"]
    if what == "loss":
        return {"bytes": 4 * T * (E + k + 1) + 4.0 * S * E, "flops": 5 * T * E}
    return {"bytes": 4 * T * (2 * E + 3 * k + 1) + 4.0 * S * E, "flops": 8 * T * E}


def exact(case, seed):
    s = _inputs(case, seed)
    what = case["what"]
    d = lambda name: s[name].double()  # noqa: E731
    if what == "norm":
        v = d("x")
        out = {}
        if case["residual"]:
            v = v + d("residual")
            out["sum"], v = v, v.to(torch.bfloat16).double()  # the norm is of the sum as it is kept
        length = v.pow(2).sum(1, keepdim=True).div(case["hidden"]).add(EPS).pow(0.5)
        if case["keep"]:
            out["rstd"] = length.reciprocal().squeeze(1)
        y = v.mul(d("weight")).div(length)
        if case["out"] == "i8":
            scale = y.abs().max(dim=1).values / 127
            y = y.div(scale.where(scale > 0, torch.ones_like(scale))[:, None]).round() * scale[:, None]
            out["scale"] = scale
        return dict(out, y=y)
    if what == "norm_grad":
        # the factors are an input here; dx by the projection that the norm's derivative is
        n = d("x").mul(d("rstd")[:, None])
        g = d("dy").mul(d("weight"))
        dx = g.sub(n.mul(torch.sum(g * n, 1, keepdim=True) / case["hidden"])).mul(d("rstd")[:, None])
        return dict(dx=dx.add(d("dsum")) if case["stream"] else dx, dweight=torch.sum(d("dy").mul(n), 0))
    if what == "adamw":
        def state(name):
            return d(name) if case["bits"] == 32 else d(name).view(-1, BLOCK).mul(d(name + "_scale")[:, None]).view(-1)

        step = s["step"] + 1
        g = d("grad").mul_(GRAD_SCALE)
        m = state("m").lerp_(g, 1 - BETA1)
        v = state("v").mul_(BETA2).addcmul_(g, g, value=1 - BETA2)
        p = d("master") if case["master"] else d("param")
        p = p.mul_(1 - LR * DECAY).addcdiv_(m, v.sqrt().div_(math.sqrt(1 - BETA2 ** step)).add_(ADAM_EPS),
                                            value=-LR / (1 - BETA1 ** step))
        out = dict(param=p, master=p if case["master"] else None)
        if case["bits"] == 32:
            return dict(out, m=m, v=v)
        # what the 8 bits are depends on random numbers
        return dict(out, m=None, v=None, m_scale=m.abs().view(-1, BLOCK).max(1).values / 448,
                    v_scale=v.view(-1, BLOCK).max(1).values / 57344)
    off = s["off"]
    a, b, T, E = off[0], off[-1], case["rows"], case["experts"]

    def placed(rows, *shape):
        full = torch.zeros(*shape, dtype=torch.float64, device="cuda")
        full[a:b] = rows
        return full

    if what == "logits":
        return dict(logits=placed(d("x")[a:b].matmul(d("wg")).add(d("bias")), T, E))
    if what == "gate_grad":
        dl = d("dlogits")[a:b]
        return dict(dx=placed(dl.matmul(d("wg").t()), T, case["hidden"]), dwg=d("x")[a:b].t().matmul(dl), dbias=dl.sum(0))
    k = case["top_k"]
    some = [(i, u, v) for i, (u, v) in enumerate(zip(off, off[1:])) if v > u]
    if what == "loss":
        balance, counts = 0.0, torch.zeros(case["seqs"], E, dtype=torch.int64, device="cuda")
        for i, u, v in some:
            counts[i] = torch.bincount(s["topk_idx"][u:v].flatten().long(), minlength=E)
            share = torch.softmax(d("logits")[u:v], 1).mean(0)
            balance = balance + (counts[i].double() / ((v - u) * k)).mul(share).sum() * E / len(some)
        lse = torch.logsumexp(d("logits")[a:b], 1)
        z = lse.pow(2).mean() if b > a else 0.0
        return dict(counts=None, lse=placed(lse, T), loss=torch.stack([torch.as_tensor(t, dtype=torch.float64, device="cuda") for t in (balance, z)]))
    # by differentiating the definition; the weights' part is that of a softmax over the chosen logits
    with torch.enable_grad():
        l = d("logits").requires_grad_()
        total = l.sum() * 0.0
        for i, u, v in some:
            c = d("counts")[i] / ((v - u) * k)
            total = total + s["dloss"][0].double() * E / len(some) * torch.softmax(l[u:v], 1).mean(0).mul(c).sum()
        if b > a:
            total = total + s["dloss"][1].double() * torch.logsumexp(l[a:b], 1).pow(2).mean()
        total.backward()
    dl, w, dw = l.grad, d("topk_w")[a:b], d("dtopk_w")[a:b]
    dl[a:b].scatter_add_(1, s["topk_idx"][a:b].long(), w * dw - w * (w * dw).sum(1, keepdim=True))
    return dict(dlogits=dl)
