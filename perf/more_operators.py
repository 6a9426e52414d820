"""The feed-forward operators whose speed is followed, with a plain form of each.

What lies around the FP8 linears of a feed-forward block, forward and backward: the layer norm before it, the matmul with a
bias, an activation and a residual sum in its epilogue (GPT), and the gated pair of projections (Llama 2).  FP8 operands are
codes with one power-of-two bias per tensor, value = code * 2^-bias; where an output is quantised too, its codes are those of
the bfloat16 output with the bias b = floor(log2(largest code / amax)) (Eq. 3 of the paper).

Case keys: kind, rows (tokens), n (columns of the output; of one of the two projections where gated), k (the contraction),
act, and truth values: bias, res (a residual tensor: added, or its gradient), keep (the values before the activation are
written for the backward pass), fq (codes of the output, and for matmuls the transposed codes).  Of the layer norm: n columns,
wide (float32 instead of bfloat16), pad (elements between the end of a row and the next).

  norm       y = (h - mean) rstd g + b, h = x or x + res; mean, rstd
  norm_bwd   dx (+ the residual's gradient), dg, db
  act        z = x w + bias; y = act(z) + res
  act_bwd    dz = (dy w^T) act'(z), its column sums; the column sums of dy
  glu        (g, u) = x (wg, wu) + bias; a = act(g) u
  glu_bwd    with t = dy w^T: dg = t u act'(g), du = t act(g)
"""
import math

import torch

own = False

FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}
EPS = 1e-5
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def listed():
    def case(name, kind, rows, n, k=0, act="none", bias=False, res=False, keep=False, fq=False, wide=False, pad=0):
        return dict(name=name, kind=kind, rows=rows, n=n, k=k, act=act, bias=bias, res=res, keep=keep, fq=fq, wide=wide, pad=pad)

    return [
        # One token of the 111M model: the latency of a norm.
        case("norm-1", "norm", 1, 768),
        # The norm between two blocks of a 13B-wide model in training: residual sum, codes for the next FP8 linear.
        case("norm-13b-res", "norm", 8192, 5120, res=True, keep=True, fq=True),
        # Odd sizes and padded rows in float32.
        case("norm-bwd-odd", "norm_bwd", 777, 1283, wide=True, pad=5),
        # The backward of a whole micro-batch, 70B width, with the residual branch's gradient added.
        case("norm-bwd-70b", "norm_bwd", 4096, 8192, res=True),
        # A single token through the second linear of a block: weight read, bias and residual in the epilogue.
        case("down-1", "act", 1, 4096, 11008, bias=True, res=True),
        # The first linear of a 13B-wide block in training: values kept for the backward pass, codes both ways.
        case("up-13b", "act", 4096, 13824, 5120, act="gelu", bias=True, keep=True, fq=True),
        # The backward of a small block (111M width, one short batch of odd length): launches count.
        case("act-bwd-111m", "act_bwd", 509, 2048, 768, act="gelu", bias=True, fq=True),
        # The backward of the 13B-wide block.
        case("act-bwd-13b", "act_bwd", 4096, 13824, 5120, act="gelu_tanh", bias=True, fq=True),
        # Decode of 16 sequences through the 70B gate and up projections: their weights at memory speed.
        case("glu-decode-16", "glu", 16, 28672, 8192, act="silu"),
        # The 70B gate and up projections in training: the largest case.
        case("glu-70b", "glu", 4096, 28672, 8192, act="silu", keep=True, fq=True),
        # The backward of the small layer the parity tests use, one ragged batch.
        case("glu-bwd-small", "glu_bwd", 300, 1408, 512, act="silu"),
        # The backward of a 7B block.
        case("glu-bwd-7b", "glu_bwd", 4096, 11008, 4096, act="silu", fq=True),
    ]


def draw(rng):
    while True:  # until one costs no more than the largest listed cases
        case = _draw(rng)
        w = work(case)
        if w["bytes"] < 3.5e8 and w["flops"] < 2e12:
            return case


def _draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "norm_bwd", "act", "act_bwd", "glu", "glu_bwd"])
    rows = rng.choice([log_int(1, 64), log_int(1, 8192), log_int(64, 8192)])
    flip = lambda: rng.random() < 0.5  # noqa: E731
    if kind in ("norm", "norm_bwd"):
        wide, res = rng.random() < 0.3, flip()
        vector = rng.random() < 0.7
        n = 8 * log_int(8, 2000) if vector else log_int(1, 16000)
        return dict(kind=kind, rows=rows, n=n, k=0, act="none", bias=False, res=res, keep=kind == "norm" and res,
                    fq=kind == "norm" and not wide and n % 8 == 0 and flip(), wide=wide,
                    pad=rng.choice([0, 0, 8 * log_int(1, 20)]) if vector else rng.choice([0, log_int(1, 50)]))
    width = lambda: rng.choice([768, 1024, 4096, 5120, 8192, 11008, 128 * log_int(1, 100), log_int(16, 9000)])  # noqa: E731
    gated = kind in ("glu", "glu_bwd")
    bias = flip() if kind != "act_bwd" else True
    return dict(kind=kind, rows=rows, n=width(), k=width(), act=rng.choice(ACTS[1:] if gated else ACTS), bias=bias,
                res=kind == "act" and flip(), keep=kind in ("act", "glu") and flip(), fq=flip(), wide=False, pad=0)


# ------------------------------------------------------------------ inputs
def power(b):
    """2^b as a float32 tensor, from its bits (torch's own powers of two can be off by an ulp)."""
    return ((b.to(torch.int32) + 127) << 23).view(torch.float32)


def coded(x, fmt):
    """Codes of a whole tensor and its bias (Eq. 3)."""
    m, e = torch.frexp(x.abs().amax())  # amax = m * 2^e, m in [1/2, 1); the largest codes are 0.875 * 2^9 and 2^16
    b = (9 if fmt == "e4m3" else 16) - e - (m > 0.875).to(e.dtype)
    b = torch.where(m == 0, torch.zeros_like(b), b).to(torch.int32)
    b = b.reshape(1)
    return (x * power(b)).to(FP8[fmt]), b


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rows, n, k, kind = case["rows"], case["n"], case["k"], case["kind"]
    state = dict(case=dict(case))

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device=dev) * std

    def padded(x):
        """The same values in rows that are `pad` elements apart."""
        wide = torch.zeros((x.shape[0], x.shape[1] + case["pad"]), dtype=x.dtype, device=dev)
        wide[:, :x.shape[1]] = x
        return wide[:, :x.shape[1]]

    if kind in ("norm", "norm_bwd"):
        dt = torch.float32 if case["wide"] else torch.bfloat16
        # hidden states: a mean that is not zero, a few large columns
        scale = 1 + 20 * (torch.rand(n, generator=g, device=dev) < 0.002)
        state["x"] = padded((normal(rows, n) * scale + normal(rows, 1, std=0.3)).to(dt))
        state["g"], state["b"] = (1 + normal(n, std=0.1)).to(dt), normal(n, std=0.1).to(dt)
        if kind == "norm" and case["res"]:
            state["res"] = padded(normal(rows, n).to(dt))
        if kind == "norm_bwd":
            state["dy"] = padded(normal(rows, n, std=1e-3).to(dt))
            if case["res"]:
                state["dres"] = padded(normal(rows, n, std=1e-3).to(dt))
            h = state["x"].double()  # the forward's statistics
            mean = h.mean(dim=1)
            state["mean"] = mean.float()
            state["rstd"] = (1 / torch.sqrt((h - mean[:, None]).square().mean(dim=1) + EPS)).float()
        return state
    outs = 2 * n if kind == "glu" else n
    fwd = kind in ("act", "glu")
    x = normal(rows, k, std=1.0 if fwd else 1e-4)
    if kind == "act_bwd":
        x = x.to(torch.bfloat16)
        state["dy"] = x
    state["x8"], state["bx"] = coded(x.float(), "e4m3" if fwd else "e5m2")
    state["w8"], state["bw"] = coded(normal(outs, k, std=1.2 / math.sqrt(k)), "e4m3")
    if fwd and case["bias"]:
        state["bias"] = normal(outs, std=0.2).to(torch.bfloat16)
    if case["res"]:
        state["res"] = normal(rows, n).to(torch.bfloat16)
    if kind == "act_bwd":
        state["z"] = normal(rows, n, std=1.2).to(torch.bfloat16)
    if kind == "glu_bwd":
        state["gu"] = normal(rows, 2 * n, std=1.2).to(torch.bfloat16)
    return state


# ------------------------------------------------------------------ the plain form
def plain_act(x, act):
    if act == "relu":
        return x.clamp(min=0)
    if act == "gelu":
        return 0.5 * x * torch.erfc(x * -math.sqrt(0.5))
    if act == "gelu_tanh":
        return x / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return x


def plain_slope(x, act):
    if act == "relu":
        return (x > 0).to(x.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(x * -math.sqrt(0.5)) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        s = 1 / (1 + torch.exp(-c * (x + 0.044715 * x ** 3)))
        return s + x * s * (1 - s) * c * (1 + 3 * 0.044715 * x * x)
    if act == "silu":
        s = 1 / (1 + torch.exp(-x))
        return s + x * s * (1 - s)
    return torch.ones_like(x)


def plain_codes(y, case):
    """Codes, transposed codes and bias of a bfloat16 output."""
    q, b = coded(y.float(), "e4m3" if case["kind"] in ("norm", "act", "glu") else "e5m2")
    return {"q": q, "bias": b} if case["kind"] == "norm" else {"q": q, "qT": q.t().contiguous(), "bias": b}


def plain_norm(s):
    c = s["case"]
    dt = s["x"].dtype
    h = s["x"]
    if c["res"]:
        h = (h.float() + s["res"].float()).to(dt)
    hf = h.float()
    mean = hf.mean(dim=1, keepdim=True)
    d = hf - mean
    rstd = 1 / torch.sqrt(d.square().mean(dim=1, keepdim=True) + EPS)
    y = (d * rstd * s["g"].float() + s["b"].float()).to(dt)
    out = {"y": y, "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if c["res"]:
        out["h"] = h
    return out | (plain_codes(y, c) if c["fq"] else {})


def plain_norm_bwd(s):
    dt = s["x"].dtype
    xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy"].float()
    w = dy * s["g"].float()
    dx = s["rstd"][:, None] * (w - w.mean(dim=1, keepdim=True) - xh * (w * xh).mean(dim=1, keepdim=True))
    if s["case"]["res"]:
        dx = dx + s["dres"].float()
    return {"dx": dx.to(dt), "dg": (dy * xh).sum(dim=0), "db": dy.sum(dim=0)}


def plain_matmul(s):
    """The matmul of the two operands' values, float32."""
    t = torch.matmul(s["x8"].float(), s["w8"].float().t())
    return t * power(-(s["bx"] + s["bw"]))


def plain_forward(s):
    c = s["case"]
    z = plain_matmul(s)
    if c["bias"]:
        z += s["bias"].float()
    if c["kind"] == "glu":
        g, u = z[:, :c["n"]], z[:, c["n"]:]
        y = plain_act(g, c["act"]) * u
    else:
        y = plain_act(z, c["act"])
        if c["res"]:
            y = y + s["res"].float()
    y = y.to(torch.bfloat16)
    out = {"y": y}
    if c["keep"]:
        out["z"] = z.to(torch.bfloat16)
    return out | (plain_codes(y, c) if c["fq"] else {})


def plain_backward(s):
    c = s["case"]
    t = plain_matmul(s)
    if c["kind"] == "glu_bwd":
        g, u = s["gu"][:, :c["n"]].float(), s["gu"][:, c["n"]:].float()
        dz = torch.cat([t * u * plain_slope(g, c["act"]), t * plain_act(g, c["act"])], dim=1)
    else:
        dz = t * plain_slope(s["z"].float(), c["act"])
    y = dz.to(torch.bfloat16)
    out = {"dz": y}
    if c["bias"]:
        out["db"] = dz.sum(dim=0).to(torch.bfloat16)
    if c["kind"] == "act_bwd":
        out["dby"] = s["dy"].float().sum(dim=0)
    return out | (plain_codes(y, c) if c["fq"] else {})


# ------------------------------------------------------------------ one pass
def handles(s):
    """The buffers that a user's program keeps between calls, made once."""
    if "F" not in s:
        from paper_2309_17224_amd import fp8lin as F
        c, dev = s["case"], torch.device("cuda")
        rows, n, kind = c["rows"], c["n"], c["kind"]
        e = lambda *shape, dt=torch.bfloat16: torch.empty(shape, dtype=dt, device=dev)  # noqa: E731
        s["fq"] = s["ws"] = s["db"] = s["keep"] = None
        cols = 2 * n if kind == "glu_bwd" else n
        if kind in ("norm", "norm_bwd"):
            dt = s["x"].dtype
            s["y"] = e(rows, n, dt=dt)
            if kind == "norm":
                s["mean"], s["rstd"] = e(rows, dt=torch.float32), e(rows, dt=torch.float32)
                s["h"] = e(rows, n, dt=dt) if c["res"] else None
            else:
                s["dg"], s["db"] = e(n, dt=torch.float32), e(n, dt=torch.float32)
                s["ws"] = F.layernorm_bwd_workspace(rows, n, dev)
        else:
            s["y"] = e(rows, cols)
            if c["keep"]:
                s["keep"] = e(rows, 2 * n if kind == "glu" else n)
            if kind in ("act_bwd", "glu_bwd") and c["bias"]:
                s["db"] = e(cols)
                s["ws"] = F.bias_grad_workspace(rows, cols, dev)
            if kind == "act_bwd":
                s["dby"] = e(c["k"], dt=torch.float32)
                s["wsy"] = F.bias_grad_workspace(rows, c["k"], dev)
        if c["fq"]:
            u8 = torch.uint8
            q, bias = e(rows, cols, dt=u8), torch.zeros(1, dtype=torch.int32, device=dev)
            qT = None if kind == "norm" else e(cols, rows, dt=u8)
            nb = F.gpt_layernorm_ws_bytes(rows) if kind == "norm" else F.fp8_linear_quantise_ws_bytes(rows, cols)
            # the bias that the call before found predicts this call's, as in the framework's own steps
            s["fq"] = F.FusedQuant(q, bias, e(max(nb, 4), dt=u8), F.E4M3 if kind in ("norm", "act", "glu") else F.E5M2,
                                   bias_pred=bias, qT=qT)
        s["act"] = {"none": F.ACT_NONE, "relu": F.ACT_RELU, "gelu": F.ACT_GELU, "gelu_tanh": F.ACT_GELU_TANH,
                    "silu": F.ACT_SILU}[c["act"]]
        s["codes"] = {name: s[name].view(torch.uint8) for name in ("x8", "w8") if name in s}
        s["F"] = F
    return s["F"]


def own_run(s):
    F, c = handles(s), s["case"]
    kind, fq = c["kind"], s["fq"]
    if kind == "norm":
        F.gpt_layernorm_quantise(s["x"], s["g"], s["b"], EPS, res=s.get("res"), h=s["h"], y=s["y"], mean=s["mean"],
                                 rstd=s["rstd"], fq=fq)
        out = {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        if c["res"]:
            out["h"] = s["h"]
    elif kind == "norm_bwd":
        F.gpt_layernorm_bwd(s["dy"], s["x"], s["g"], s["mean"], s["rstd"], dres=s.get("dres"), dx=s["y"], dg=s["dg"],
                            db=s["db"], ws=s["ws"])
        return {"dx": s["y"], "dg": s["dg"], "db": s["db"]}
    else:
        ops = (s["codes"]["x8"], s["bx"], s["codes"]["w8"], s["bw"])
        if kind == "act":
            F.fp8_linear_fwd_act(*ops, s["act"], bias=s.get("bias"), res=s.get("res"), z=s["keep"], y=s["y"], fq=fq)
        elif kind == "glu":
            F.fp8_linear_fwd_glu(*ops, s["act"], bias=s.get("bias"), gu=s["keep"], a=s["y"], fq=fq)
        elif kind == "act_bwd":
            F.fp8_linear_bwd_dx_act(*ops, s["z"], s["act"], dz=s["y"], db=s["db"], fq=fq, ws=s["ws"])
        else:
            F.fp8_linear_bwd_dx_glu(*ops, s["gu"], s["act"], dgu=s["y"], db=s["db"], fq=fq, ws=s["ws"])
        out = {"y" if kind in ("act", "glu") else "dz": s["y"]}
        if c["keep"]:
            out["z"] = s["keep"]
        if s["db"] is not None:
            out["db"] = s["db"]
        if kind == "act_bwd":
            out["dby"] = F.gpt_bias_grad(s["dy"], db=s["dby"], ws=s["wsy"])
    if c["fq"]:
        kind8 = FP8["e4m3" if kind in ("norm", "act", "glu") else "e5m2"]
        out |= {"q": fq.q.view(kind8), "bias": fq.bias}
        if kind != "norm":
            out["qT"] = fq.qT.view(kind8)
    return out


def run(s):
    if own:
        return own_run(s)
    kind = s["case"]["kind"]
    if kind == "norm":
        return plain_norm(s)
    if kind == "norm_bwd":
        return plain_norm_bwd(s)
    return plain_forward(s) if kind in ("act", "glu") else plain_backward(s)


def work(case):
    rows, n, k, kind = case["rows"], case["n"], case["k"], case["kind"]
    if kind in ("norm", "norm_bwd"):
        size = 4 if case["wide"] else 2
        if kind == "norm":
            tensors = 2 + 2 * case["res"]
            return {"bytes": rows * n * (size * tensors + case["fq"]) + 2 * n * size + 8 * rows, "flops": 8 * rows * n}
        return {"bytes": rows * n * size * (3 + case["res"]) + n * (size + 8) + 8 * rows, "flops": 14 * rows * n}
    outs = 2 * n if kind == "glu" else n
    nbytes = rows * k + outs * k
    if kind in ("act", "glu"):
        nbytes += rows * n * (2 + 2 * case["res"] + 2 * case["fq"]) + 2 * outs * case["bias"] + 2 * rows * outs * case["keep"]
    else:
        cols = 2 * n if kind == "glu_bwd" else n
        nbytes += rows * cols * (4 + 2 * case["fq"]) + 2 * cols * case["bias"]
        if kind == "act_bwd":
            nbytes += 2 * rows * k + 4 * k
    return {"bytes": nbytes, "flops": 2 * rows * outs * k}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    kind, n = case["kind"], case["n"]
    d = {name: v.double() for name, v in s.items() if isinstance(v, torch.Tensor)}
    if kind == "norm":
        h = d["x"] + d["res"] if case["res"] else d["x"]
        kept = h
        if case["res"]:
            h = h.to(s["x"].dtype).double()  # the norm is of the sum as it is kept
        var, mean = torch.var_mean(h, dim=1, correction=0, keepdim=True)
        rstd = torch.rsqrt(var + EPS)
        y = torch.addcmul(d["b"], (h - mean) * rstd, d["g"])
        out = {"y": y, "mean": mean.squeeze(1), "rstd": rstd.squeeze(1)}
        if case["res"]:
            out["h"] = kept
    elif kind == "norm_bwd":
        # the gradient through the mean and the spread, as a projection: the part of v = dy g / n along 1 and along the
        # normalised row is taken away
        unit = torch.stack([torch.ones_like(d["x"]), (d["x"] - d["mean"].unsqueeze(1)) * d["rstd"].unsqueeze(1)], dim=1)
        v = d["dy"] * d["g"]
        along = (unit * v.unsqueeze(1)).mean(dim=2)
        dx = (v - along[:, 0:1] - along[:, 1:2] * unit[:, 1]) * d["rstd"].unsqueeze(1)
        if case["res"]:
            dx = dx + d["dres"]
        return {"dx": dx, "dg": (d["dy"] * unit[:, 1]).sum(dim=0), "db": d["dy"].sum(dim=0)}
    else:
        scale = 0.5 ** float(s["bx"] + s["bw"])
        prod = (d["x8"] @ d["w8"].t().contiguous()) * scale
        if kind in ("act", "glu"):
            if case["bias"]:
                prod = prod + d["bias"]
            if kind == "glu":
                y = _act64(prod[:, :n], case["act"])[0] * prod[:, n:]
            else:
                y = _act64(prod, case["act"])[0]
                if case["res"]:
                    y = y + d["res"]
            out = {"y": y}
            if case["keep"]:
                out["z"] = prod
        else:
            if kind == "glu_bwd":
                value, slope = _act64(d["gu"][:, :n], case["act"])
                y = torch.cat([prod * d["gu"][:, n:] * slope, prod * value], dim=1)
            else:
                y = prod * _act64(d["z"], case["act"])[1]
            out = {"dz": y}
            if case["bias"]:
                out["db"] = y.sum(dim=0)
            if kind == "act_bwd":
                out["dby"] = d["dy"].sum(dim=0)
    if case["fq"]:
        codes = _grid(y.to(torch.bfloat16).double(), "e4m3" if kind in ("norm", "act", "glu") else "e5m2")
        out |= {"q": codes, "bias": None}  # a whole number: compared with the plain form's
        if kind != "norm":
            out["qT"] = codes.t()
    return out


def _act64(x, act):
    """act(x) and act'(x)."""
    if act == "none":
        return x, torch.ones_like(x)
    if act == "relu":
        return torch.where(x > 0, x, torch.zeros_like(x)), torch.where(x > 0, torch.ones_like(x), torch.zeros_like(x))
    if act == "silu":
        s = torch.sigmoid(x)
        return x * s, s * (1 + x * torch.sigmoid(-x))
    if act == "gelu":
        phi = torch.special.ndtr(x)
        return x * phi, phi + x * torch.exp(-x * x / 2) * (0.5 / math.pi) ** 0.5
    th = torch.tanh((2 / math.pi) ** 0.5 * (x + 0.044715 * x ** 3))
    return 0.5 * x * (1 + th), 0.5 * (1 + th) + 0.5 * x * (1 - th * th) * (2 / math.pi) ** 0.5 * (1 + 0.134145 * x * x)


def _grid(x, fmt):
    """A tensor on the format's grid after scaling: code values."""
    least, bits = (-6, 3) if fmt == "e4m3" else (-14, 2)
    amax = float(x.abs().max())
    b = math.floor(math.log2(TOP[fmt] / amax)) if amax > 0 else 0
    while amax * 2.0 ** b > TOP[fmt]:  # log2 rounded up
        b -= 1
    while 0 < amax * 2.0 ** (b + 1) <= TOP[fmt]:
        b += 1
    y = x * 2.0 ** b
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** least)))
    e = torch.where(torch.exp2(e) > y.abs(), e - 1, e).clamp(min=least)
    step = torch.exp2(e - bits)
    return torch.round(y / step) * step
