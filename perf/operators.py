"""The paged key/value cache operators whose speed is followed, with a plain form of each.

A serving step of a decoder layer appends the new tokens' keys and values to a paged cache, quantised to FP8 with one
power-of-two bias per token and key/value head (Eq. 3 of the paper), and attends over it; a cached range can be read back.

Layout of the cache (all page tensors are shared by the sequences; ``pages[s, i]`` is the page of positions
``i * page .. i * page + page - 1`` of sequence ``s``):

  k      [n_pages, kv_heads, page, d_head]            codes (uint8), or bfloat16
  v      [n_pages, kv_heads, page / 16, d_head, 16]   codes (uint8), or bfloat16: blocks of 16 tokens, tokens innermost
  k_exp  [n_pages, kv_heads, page]                    uint8: value = code * 2^(exp - 127)  (FP8 only); v_exp the same

Rows ``cu_rows[s] .. cu_rows[s+1]`` of a call belong to sequence ``s`` and are its last positions, up to ``kv_len[s]``.

Case keys: kind (append: write new tokens, then read them back; read: read whole sequences; attend: attention of the new
tokens; step: append, then attention), heads, kv_heads, d_head, fmt, page, seqs, new and past (tokens per sequence; the
largest where ragged), ragged (0: all alike, else the number that the lengths are drawn from), window (0: none).
"""
import math
import random

import torch

own = False

BLOCK = 16  # tokens in one block of v
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def listed():
    def case(name, kind, heads, kv_heads, d_head, fmt, page, seqs, new, past, ragged=0, window=0):
        return dict(name=name, kind=kind, heads=heads, kv_heads=kv_heads, d_head=d_head, fmt=fmt, page=page, seqs=seqs,
                    new=new, past=past, ragged=ragged, window=window)

    return [
        # One token of one sequence of the Llama 2 70B layer: the latency of a single decode step's write.
        case("append-1", "append", 64, 8, 128, "e4m3", 64, 1, 1, 1000),
        # A 2048-token prefill of the 70B layer (the layer workload's call), written whole.
        case("append-2048", "append", 64, 8, 128, "e4m3", 64, 1, 2048, 0),
        # Chunks of odd lengths at odd positions, 7B heads, E5M2 codes, small pages.
        case("append-7b-ragged", "append", 32, 32, 128, "e5m2", 16, 7, 601, 1500, 3),
        # Four 70B sequences taken out of the cache (moved to another format or another consumer).
        case("read-70b-4x4096", "read", 64, 8, 128, "e4m3", 64, 4, 4096, 0),
        # Short sequences of odd lengths, heads of 64 (GPT 111M: d_model 768), E5M2.
        case("read-111m-ragged", "read", 12, 12, 64, "e5m2", 16, 9, 700, 0, 5),
        # The smallest attention: one token over a few hundred (the small parity layer's heads).
        case("decode-tiny", "attend", 8, 2, 128, "e4m3", 16, 1, 1, 299),
        # Decode of 32 sequences of the 70B layer up to 16k tokens long: the cache read at memory speed.
        case("decode-70b-32", "attend", 64, 8, 128, "e4m3", 64, 32, 1, 16000, 7),
        # Decode without grouped heads (7B), E5M2 codes.
        case("decode-7b-16", "attend", 32, 32, 128, "e5m2", 32, 16, 1, 2500, 11),
        # A 512-token chunk over 8k cached tokens, 70B: chunked prefill, bound by the matrix cores.
        case("chunk-70b-512", "attend", 64, 8, 128, "e4m3", 64, 1, 512, 8192),
        # Two whole 7B prompts through an unquantised cache.
        case("prefill-7b-bf16", "attend", 32, 32, 128, "bf16", 64, 2, 2048, 0),
        # Chunks and single tokens in one call, heads of 64, a sliding window.
        case("mixed-111m", "attend", 12, 12, 64, "bf16", 16, 13, 333, 2000, 2, 1024),
        # A whole serving step of 64 70B sequences: the write and the attention together.
        case("step-70b-64", "step", 64, 8, 128, "e4m3", 64, 64, 1, 1500, 13),
    ]


def draw(rng):
    while True:  # until one costs no more than the largest listed cases
        case = _draw(rng)
        w = work(case)
        if w["bytes"] < 4.9e8 and w["flops"] < 1.4e11:
            return case


def _draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["append", "read", "attend", "attend", "attend", "step"])
    heads, kv_heads, d_head = rng.choice([(64, 8, 128), (32, 32, 128), (40, 40, 128), (8, 2, 128), (12, 12, 64),
                                          (28, 4, 128), (24, 8, 64), (16, 1, 128)])
    decode = kind == "step" or (kind == "attend" and rng.random() < 0.5)
    if kind == "read":
        seqs, new, past = log_int(1, 12), log_int(1, 3000), 0
    elif kind == "append":
        seqs, new, past = log_int(1, 12), log_int(1, 1000), rng.choice([0, log_int(1, 6000)])
    elif decode:
        seqs, new, past = log_int(1, 48), 1, log_int(1, 8000)
    else:
        seqs, new, past = log_int(1, 6), log_int(2, 700), rng.choice([0, log_int(1, 3000)])
    window = rng.choice([0, 0, 0, log_int(1, 2000)]) if kind in ("attend", "step") else 0
    return dict(kind=kind, heads=heads, kv_heads=kv_heads, d_head=d_head, fmt=rng.choice(["e4m3", "e4m3", "e5m2", "bf16"]),
                page=rng.choice([16, 32, 64, 128]), seqs=seqs, new=new, past=past,
                ragged=rng.choice([0, rng.randrange(1, 1000)]), window=window)


def lengths(case):
    """New tokens and tokens cached before them, for each sequence."""
    if not case["ragged"]:
        return [case["new"]] * case["seqs"], [case["past"]] * case["seqs"]
    r = random.Random(case["ragged"])
    new = [r.randint(1, case["new"]) for _ in range(case["seqs"])]
    past = [r.randint(0, case["past"]) for _ in range(case["seqs"])]
    if case["kind"] == "attend":  # the longest chunk, and single tokens beside it
        new = [case["new"] if i == 0 else 1 if i % 3 == 1 else n for i, n in enumerate(new)]
    return new, past


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    nh, nkv, dh, page = case["heads"], case["kv_heads"], case["d_head"], case["page"]
    new, past = lengths(case)
    total = [a + b for a, b in zip(new, past)]
    max_pages = -(-(case["new"] + case["past"]) // page)
    need = [-(-t // page) for t in total]
    n_pages = sum(need)
    order = torch.randperm(n_pages, generator=g, device=dev).tolist()
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [-1] * (max_pages - n))
        at += n
    i32 = dict(dtype=torch.int32, device=dev)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    rows = cu[-1]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device=dev) * std

    # the cache as earlier calls left it: every slot of every page holds a value
    state = dict(case=dict(case), rows=rows, max_rows=case["new"], max_pages=max_pages,
                 cu_rows=torch.tensor(cu, **i32), kv_len=torch.tensor(total, **i32), pages=torch.tensor(table, **i32))
    shape = (n_pages, nkv, page, dh)
    for name, std in (("k", 1.5), ("v", 1.0)):
        x = normal(*shape, std=std).to(torch.bfloat16)
        if case["fmt"] == "bf16":
            codes = x
        else:
            codes, exp = quantise(x.float(), case["fmt"])
            codes = codes.view(torch.uint8)
            state[name + "_exp"] = exp
        if name == "v":
            codes = codes.reshape(n_pages, nkv, page // BLOCK, BLOCK, dh).transpose(3, 4).contiguous()
        state[name] = codes
        del x
    if case["kind"] in ("append", "step"):
        state["qkv"] = normal(rows, (nh + 2 * nkv) * dh).to(torch.bfloat16)
        pos = torch.arange(max_pages * page, device=dev, dtype=torch.float64)
        freq = 10000.0 ** (-torch.arange(dh // 2, device=dev, dtype=torch.float64) / (dh // 2))
        ang = pos[:, None] * freq[None, :]
        state["table"] = torch.stack([ang.cos(), ang.sin()], dim=2).float().reshape(-1)
    if case["kind"] == "attend":
        state["q"] = normal(rows, nh * dh).to(torch.bfloat16)
    return state


# ------------------------------------------------------------------ the plain form
def quantise(x, fmt):
    """Codes and exponent bytes of the rows (last dimension) of x: bias b = floor(log2(max / amax)), codes of x * 2^b."""
    m, e = torch.frexp(x.abs().amax(dim=-1))  # amax = m * 2^e, m in [1/2, 1); the largest codes are 0.875 * 2^9 and 2^16
    b = (9 if fmt == "e4m3" else 16) - e - (m > 0.875).to(e.dtype)
    b = torch.where(m == 0, torch.zeros_like(b), b).clamp(max=126)
    return torch.ldexp(x, b[..., None]).to(FP8[fmt]), (127 - b).to(torch.uint8)


def tokens(s):
    """Sequence and position of every row of the call."""
    cu, kv = s["cu_rows"].long(), s["kv_len"].long()
    row = torch.arange(s["rows"], device=cu.device)
    seq = torch.searchsorted(cu, row, right=True) - 1
    return seq, kv[seq] - cu[seq + 1] + row


def places(s, seq, pos):
    """Page and slot of positions."""
    page = s["case"]["page"]
    return s["pages"][seq, pos // page].long().clamp(min=0), pos % page


def values(s, seq, pos):
    """Cached keys and values, float32 [..., kv_heads, d_head], at positions of sequences."""
    at, slot = places(s, seq, pos)
    k, v = s["k"][at, :, slot], s["v"][at, :, slot // BLOCK, :, slot % BLOCK]
    if s["case"]["fmt"] == "bf16":
        return k.float(), v.float()
    one = torch.ones((), device=k.device)
    kind = FP8[s["case"]["fmt"]]
    ke, ve = s["k_exp"][at, :, slot].int() - 127, s["v_exp"][at, :, slot].int() - 127
    return (k.view(kind).float() * torch.ldexp(one, ke)[..., None], v.view(kind).float() * torch.ldexp(one, ve)[..., None])


def plain_append(s):
    c = s["case"]
    nh, nkv, dh = c["heads"], c["kv_heads"], c["d_head"]
    seq, pos = tokens(s)
    x = s["qkv"].view(s["rows"], nh + 2 * nkv, dh)
    # in 64 bits: a sum that cancels can lie next to a border between two codes
    t = s["table"].view(-1, 1, dh // 2, 2)[pos].double()
    a, b = x[:, :nh + nkv, :dh // 2].double(), x[:, :nh + nkv, dh // 2:].double()
    rot = torch.cat([a * t[..., 0] - b * t[..., 1], b * t[..., 0] + a * t[..., 1]], dim=2).float()
    k, v = rot[:, nh:], x[:, nh + nkv:].float()
    at, slot = places(s, seq, pos)
    if c["fmt"] == "bf16":
        k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
    else:
        (k, ke), (v, ve) = quantise(k, c["fmt"]), quantise(v, c["fmt"])
        k, v = k.view(torch.uint8), v.view(torch.uint8)
        s["k_exp"][at, :, slot], s["v_exp"][at, :, slot] = ke, ve
    s["k"][at, :, slot] = k
    s["v"][at, :, slot // BLOCK, :, slot % BLOCK] = v
    return rot[:, :nh].reshape(s["rows"], nh * dh).to(torch.bfloat16)


def plain_read(s):
    k, v = values(s, *tokens(s))
    return k.reshape(s["rows"], -1).to(torch.bfloat16), v.reshape(s["rows"], -1).to(torch.bfloat16)


def plain_attend(s, q):
    """Rows padded to the longest chunk, keys to the longest sequence; what a row may not see gets weight 0."""
    c = s["case"]
    nh, nkv, dh, n = c["heads"], c["kv_heads"], c["d_head"], s["max_rows"]
    seq, pos = tokens(s)
    inside = torch.arange(s["rows"], device=q.device) - s["cu_rows"].long()[seq]
    ns, longest = s["kv_len"].numel(), s["max_pages"] * c["page"]
    qp = torch.zeros((ns, n, nh, dh), device=q.device)
    qp[seq, inside] = q.float().view(-1, nh, dh)
    pp = torch.full((ns, n), -1, device=q.device, dtype=torch.long)
    pp[seq, inside] = pos
    every = torch.arange(longest, device=q.device)
    k, v = values(s, torch.arange(ns, device=q.device)[:, None], every[None, :])
    grp = nh // nkv
    qp = qp.view(ns, n, nkv, grp, dh).permute(0, 2, 3, 1, 4).reshape(ns * nkv, grp * n, dh)
    k = k.permute(0, 2, 3, 1).reshape(ns * nkv, dh, longest).contiguous()
    v = v.permute(0, 2, 1, 3).reshape(ns * nkv, longest, dh).contiguous()
    score = torch.matmul(qp, k).mul_(dh ** -0.5).view(ns, nkv, grp, n, longest)
    seen = every <= pp[:, :, None]
    if c["window"]:
        seen &= every > pp[:, :, None] - c["window"]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(dim=-1, keepdim=True).clamp(min=-3e38)
    p = score.sub_(top).exp_()
    p /= p.sum(dim=-1, keepdim=True).clamp(min=1e-38)
    o = torch.matmul(p.view(ns * nkv, grp * n, longest), v).view(ns, nkv, grp, n, dh).permute(0, 3, 1, 2, 4)
    return o.reshape(ns, n, nh * dh)[seq, inside].to(torch.bfloat16)


# ------------------------------------------------------------------ one pass
def handles(s):
    """The framework's objects around the state's tensors, made once as a user's program makes them."""
    if "cache" not in s:
        from paper_2309_17224_amd import fp8lin as F
        c = s["case"]
        fmt = {"e4m3": F.E4M3, "e5m2": F.E5M2, "bf16": F.CACHE_BF16}[c["fmt"]]
        dev = s["k"].device
        s["cache"] = F.KVCache(s["k"].shape[0], c["kv_heads"], c["d_head"], c["page"], fmt, dev, k=s["k"], v=s["v"],
                               k_exp=s.get("k_exp"), v_exp=s.get("v_exp"))
        s["seqs"] = F.CacheSeqs(s["cu_rows"], s["kv_len"], s["pages"])
        bf = dict(dtype=torch.bfloat16, device=dev)
        if c["kind"] in ("append", "step"):
            s["q_out"] = torch.empty((s["rows"], c["heads"] * c["d_head"]), **bf)
        if c["kind"] in ("append", "read"):
            s["k_out"], s["v_out"] = (torch.empty((s["rows"], c["kv_heads"] * c["d_head"]), **bf) for _ in "kv")
        if c["kind"] in ("attend", "step"):
            s["o"] = torch.empty((s["rows"], c["heads"] * c["d_head"]), **bf)
            s["ws"] = F.cache_attention_workspace(s["rows"], c["heads"], s["cache"], s["seqs"], s["max_rows"])
        s["F"] = F
    return s["F"], s["cache"], s["seqs"]


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        F, cache, seqs = handles(s)
        if kind in ("append", "step"):
            q = F.llama_cache_append(s["qkv"], cache, seqs, c["heads"], table=s["table"], q=s["q_out"])
        if kind in ("append", "read"):
            k, v = F.llama_cache_read(cache, seqs, s["rows"], k=s["k_out"], v=s["v_out"])
        if kind in ("attend", "step"):
            o = F.llama_cache_attention(q if kind == "step" else s["q"], cache, seqs, c["heads"], s["max_rows"],
                                        window=c["window"], o=s["o"], ws=s["ws"])
    else:
        if kind in ("append", "step"):
            q = plain_append(s)
        if kind in ("append", "read"):
            k, v = plain_read(s)
        if kind in ("attend", "step"):
            o = plain_attend(s, q if kind == "step" else s["q"])
    if kind == "append":
        return {"q": q, "k": k, "v": v}
    if kind == "read":
        return {"k": k, "v": v}
    if kind == "attend":
        return {"o": o}
    out = {"o": o, "q": q, "k": s["k"], "v": s["v"]}  # the step's updated state: codes and exponents
    if c["fmt"] != "bf16":
        out |= {"k": s["k"].view(FP8[c["fmt"]]), "v": s["v"].view(FP8[c["fmt"]]), "k_exp": s["k_exp"], "v_exp": s["v_exp"]}
    return out


def work(case):
    nh, nkv, dh = case["heads"], case["kv_heads"], case["d_head"]
    new, past = lengths(case)
    rows, w = sum(new), case["window"]
    token = nkv * (4 * dh if case["fmt"] == "bf16" else 2 * dh + 2)  # keys and values of one cached token
    nbytes = flops = 0
    if case["kind"] in ("append", "step"):
        nbytes += rows * ((nh + 2 * nkv) * dh * 2 + 4 * dh + nh * dh * 2 + token)
        flops += rows * (nh + nkv) * dh * 3
    if case["kind"] in ("append", "read"):
        nbytes += rows * nkv * dh * 4
    if case["kind"] == "read":
        nbytes += rows * token
    if case["kind"] in ("attend", "step"):
        for n, p in zip(new, past):
            first = max(0, p + 1 - w) if w else 0  # the first key that any row sees
            nbytes += (p + n - first) * token
            pairs = sum(min(p + i + 1, w) for i in range(n)) if w else n * p + n * (n + 1) // 2
            flops += 4 * dh * nh * pairs
        nbytes += 2 * rows * nh * dh * 2
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    nh, nkv, dh, page, fmt = case["heads"], case["kv_heads"], case["d_head"], case["page"], case["fmt"]
    new, past = lengths(case)
    pages = s["pages"].tolist()
    kval = s["k"] if fmt == "bf16" else s["k"].view(FP8[fmt])
    vval = (s["v"] if fmt == "bf16" else s["v"].view(FP8[fmt])).transpose(3, 4).reshape(s["k"].shape)
    kval, vval = kval.double(), vval.double()  # codes
    kexp, vexp = (None, None) if fmt == "bf16" else (s["k_exp"].double() - 127, s["v_exp"].double() - 127)
    out = {name: [] for name in "qkvo"}
    row = 0
    for i, (n, p) in enumerate(zip(new, past)):
        used = torch.tensor(pages[i][:-(-(n + p) // page)], device=s["k"].device)
        K, V = (x[used].transpose(1, 2).reshape(-1, nkv, dh)[:n + p].clone() for x in (kval, vval))
        if fmt != "bf16":
            KE, VE = (x[used].transpose(1, 2).reshape(-1, nkv)[:n + p].clone() for x in (kexp, vexp))
        if case["kind"] in ("append", "step"):
            x = s["qkv"][row:row + n].double().view(n, nh + 2 * nkv, 2, dh // 2)
            z = torch.view_as_complex(s["table"].double().view(-1, dh // 2, 2)[p:p + n].contiguous())[:, None]
            turned = torch.complex(x[:, :nh + nkv, 0], x[:, :nh + nkv, 1]) * z
            turned = torch.cat([turned.real, turned.imag], dim=2)
            out["q"].append(turned[:, :nh].reshape(n, -1))
            fresh = [turned[:, nh:], x[:, nh + nkv:].reshape(n, nkv, dh)]
            if fmt == "bf16":
                K[p:], V[p:] = fresh
            else:
                (K[p:], KE[p:]), (V[p:], VE[p:]) = (_grid(f, fmt) for f in fresh)
            for val, exp, X, E in ((kval, kexp, K, None if fmt == "bf16" else KE), (vval, vexp, V, None if fmt == "bf16" else VE)):
                where = torch.arange(p, p + n, device=used.device)
                val[used[where // page], :, where % page] = X[p:]
                if E is not None:
                    exp[used[where // page], :, where % page] = E[p:]
        if fmt != "bf16":
            K, V = K * torch.exp2(KE)[..., None], V * torch.exp2(VE)[..., None]
        out["k"].append(K[p:].reshape(n, -1))
        out["v"].append(V[p:].reshape(n, -1))
        if case["kind"] in ("attend", "step"):
            # a step's queries are the rotated ones, a bfloat16 tensor
            q = out["q"][-1].to(torch.bfloat16) if case["kind"] == "step" else s["q"][row:row + n]
            q = q.double().view(n, nh, dh)
            pos = torch.arange(p, p + n, device=q.device)[:, None]
            key = torch.arange(n + p, device=q.device)[None, :]
            hide = key > pos
            if case["window"]:
                hide |= pos - key >= case["window"]
            heads = []
            for h in range(nh):
                a = (q[:, h] @ K[:, h * nkv // nh].t().contiguous()) / math.sqrt(dh)
                heads.append(torch.softmax(a.masked_fill(hide, -math.inf), dim=1) @ V[:, h * nkv // nh].contiguous())
            out["o"].append(torch.stack(heads, dim=1).reshape(n, -1))
        row += n
    got = {name: torch.cat(x) for name, x in out.items() if x}
    if case["kind"] == "append":
        return {name: got[name] for name in "qkv"}
    if case["kind"] == "read":
        return {name: got[name] for name in "kv"}
    if case["kind"] == "attend":
        return {"o": got["o"]}
    back = vval.reshape(-1, nkv, page // BLOCK, BLOCK, dh).transpose(3, 4).contiguous()
    res = {"o": got["o"], "q": got["q"], "k": kval, "v": back}
    if fmt != "bf16":
        res |= {"k_exp": None, "v_exp": None}  # whole numbers: compared with the plain form's
    return res


def _grid(x, fmt):
    """Rows of x on the format's grid after scaling: code values and the power of two that takes them back."""
    top, least, bits = (448.0, -6, 3) if fmt == "e4m3" else (57344.0, -14, 2)
    amax = x.abs().amax(dim=-1)
    b = torch.floor(torch.log2(top / amax.clamp(min=1e-300)))
    b = torch.where(amax * torch.exp2(b) > top, b - 1, b)  # log2 rounded up
    b = torch.where(amax * torch.exp2(b + 1) <= top, b + 1, b)
    b = torch.where(amax == 0, torch.zeros_like(b), b).clamp(max=126)
    y = x * torch.exp2(b)[..., None]
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** least)))
    e = torch.where(torch.exp2(e) > y.abs(), e - 1, e).clamp(min=least)
    step = torch.exp2(e - bits)
    return torch.round(y / step) * step, -b
