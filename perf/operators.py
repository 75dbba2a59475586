"""Operators around and beneath the MoE layer, as measurable cases.

  quant    a weight matrix into microscaled 4-bit rows (MXFP4: e2m1 codes, one
           power-of-two scale per 32 along the row) and back into values
  experts  the grouped SwiGLU forward of the 4-bit profiling model: activations
           and weights in MXFP4, fp32 sums, H re-quantised between the products
  balance  the router's balance loss per sequence with the per-expert counts,
           then the router's whole backward: the loss's and the gates' share of
           the logits' gradient, dX, the router's weight and bias gradients
  norm     the norms around a block: post-norm of the block's output with its
           gate and the residual scale, the residual stream, the next block's
           pre-norm; or its backward with every gradient, from what the forward
           of the same step left (the stream in its type, the rows' scales)

Ranges (what ``draw`` spreads over): 1 to 32768 tokens, d from 128 to 4096 and I
from 64 to 2816 in multiples of 8, 4 to 128 experts, top-1 to top-8, none to two
shared experts, even to Zipf popularity, 1 to 64 sequences of uneven lengths
(empty ones among them) with and without padding, bf16 mostly and fp32.

The plain forms compute in fp32 (fp64 for sums over tokens that decide a scale)
and round once at the end.
"""
import math

import torch

own = False
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6


# ------------------------------------------------------------------ cases ----

def listed():
    return [
        # one expert matrix of the test suite's unit workload, fp32
        dict(name="quant_tiny_f32", kind="quant", rows=2048, cols=128, dtype="f32"),
        # W_gate of a DeepSeek-MoE-shaped layer's 64 experts
        dict(name="quant_deepseek", kind="quant", rows=64 * 1408, cols=2048, dtype="bf16"),
        # generation through the LLaMA-MoE-shaped layer, one token (I = 688: a row ends inside a block)
        dict(name="experts_llama_1", kind="experts", T=1, d=4096, E=16, k=4, I=688, shared=0, skew="normal"),
        # one short prompt through the DeepSeek-MoE-shaped layer with its shared experts
        dict(name="experts_deepseek_333", kind="experts", T=333, d=2048, E=64, k=6, I=1408, shared=2, skew="normal"),
        # one layer of the DeepSeek-MoE-shaped stack's profiling pass
        dict(name="experts_deepseek_4096", kind="experts", T=4096, d=2048, E=64, k=6, I=1408, shared=0, skew="normal"),
        # the stress layer: 262144 rows, Zipf popularity
        dict(name="experts_stress_32768", kind="experts", T=32768, d=4096, E=64, k=8, I=1024, shared=0, skew="zipf"),
        # the unit workload's router: short uneven sequences, padded, fp32
        dict(name="balance_tiny_f32", kind="balance", T=256, d=128, E=8, k=2, dtype="f32", seqs=5, pad=0.2),
        # the benchmark's layer, four packed sequences
        dict(name="balance_deepseek_8192", kind="balance", T=8192, d=2048, E=64, k=6, dtype="bf16", seqs=4, pad=0.0),
        # generation: one token of each of 8 sequences around the LLaMA-MoE-shaped block
        dict(name="norm_llama_8", kind="norm", T=8, d=4096, dtype="bf16", back=False, post=True, gate=True),
        # the benchmark's layer: its forward, and its backward
        dict(name="norm_deepseek_8192", kind="norm", T=8192, d=2048, dtype="bf16", back=False, post=True, gate=True),
        dict(name="norm_bwd_deepseek_8192", kind="norm", T=8192, d=2048, dtype="bf16", back=True, post=True, gate=True),
        # fine-tuning in full precision, a width off every tile, pre-norm only with a layer scale
        dict(name="norm_bwd_f32_1023", kind="norm", T=1023, d=1000, dtype="f32", back=True, post=False, gate=False),
    ]


def _spread(rng, lo, hi, step):
    """A multiple of `step` in [lo, hi], spread over its logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choices(("quant", "experts", "balance", "norm"), (2, 4, 3, 3))[0]
    while True:
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        T, d, I = _spread(rng, 1, 32768, 1), _spread(rng, 128, 4096, 8), _spread(rng, 64, 2816, 8)
        E = rng.choice((4, 8, 16, 24, 32, 48, 64, 64, 96, 128))
        k = rng.randint(1, min(8, E))
        if kind == "quant":
            c = dict(kind=kind, rows=_spread(rng, 8, 262144, 1), cols=d, dtype=dtype)
            if c["rows"] * d > 64 * 1408 * 4096:
                continue
            return c
        if kind == "experts":
            c = dict(kind=kind, T=T, d=d, E=E, k=k, I=I, shared=rng.choice((0, 0, 1, 2)),
                     skew=rng.choice(("normal", "even", "zipf")))
            # the plain form pads every slot to the fullest one
            if T * min(E, 4 * k) * (2 * d + 6 * I) * 4 > 60e9 or work(c)["flops"] > 6e12 or E * d * I > 6e8:
                continue
            return c
        if kind == "balance":
            return dict(kind=kind, T=T, d=d, E=E, k=k, dtype=dtype, seqs=_spread(rng, 1, 64, 1),
                        pad=rng.choice((0.0, 0.0, 0.1, 0.5)))
        return dict(kind=kind, T=T, d=d, dtype=dtype, back=rng.random() < 0.6, post=rng.random() < 0.7, gate=rng.random() < 0.6)


def work(c):
    if c["kind"] == "quant":
        n, es = c["rows"] * c["cols"], 4 if c["dtype"] == "f32" else 2
        return {"bytes": n * (2 * es + 0.5 + 1 / 32), "flops": 0}
    if c["kind"] == "experts":
        T, d, E, k, I, sh = c["T"], c["d"], c["E"], c["k"], c["I"], c["shared"]
        slots = E * (1 - (1 - k / E) ** T) + sh
        rows = T * (k + sh)
        return {"bytes": slots * 3 * d * I * (0.5 + 1 / 32) + 2 * T * d + 2 * rows * d + 4 * T * k,
                "flops": 6.0 * rows * d * I}
    es = 4 if c["dtype"] == "f32" else 2
    T, d = c["T"], c["d"]
    if c["kind"] == "balance":
        E, k = c["E"], c["k"]
        return {"bytes": 2 * T * d * es + E * d * (es + 4) + 8 * T * E + 12 * T * k, "flops": 4.0 * T * d * E}
    return {"bytes": T * d * es * (6 if c["back"] else 4), "flops": 0}


# ---------------------------------------------------------------- prepare ----

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, std, dt=torch.float32):
    return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dt)


def _mx4(x):
    """x [..., cols] (fp32) in blocks of 32 along the row (the last one filled up with
    zeros): (the e2m1 values, signed, [..., blocks, 32]; the scales' exponents [..., blocks])."""
    pad = -x.shape[-1] % 32
    if pad:
        x = torch.nn.functional.pad(x, (0, pad))
    x = x.reshape(*x.shape[:-1], -1, 32)
    e = torch.frexp(x.abs().amax(-1))[1] - 3            # floor(log2 amax) - 2
    e = torch.where(x.abs().amax(-1) > 0, e, -127).clamp(-127, 127)
    a = torch.ldexp(x, -e[..., None]).abs().clamp(max=6.0)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign(torch.round(a / step) * step, x), e


def _values(x):
    """What x stands for after MXFP4, fp32, rows filled up to whole blocks."""
    q, e = _mx4(x)
    return torch.ldexp(q, e[..., None]).flatten(-2)


def _pack(x):
    """x [..., cols] as codes [..., ceil32(cols) / 2] (even columns in the low half of a
    byte) and scale bytes [..., ceil128(cols) / 32]."""
    q, e = _mx4(x.float())
    a = q.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code += (torch.signbit(q) * 8).to(torch.uint8)
    code = code.flatten(-2)
    s = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[-1] % 4))
    return (code[..., 0::2] | (code[..., 1::2] << 4)).contiguous(), s.contiguous()


def _unpack(codes, scale):
    """fp32 values [..., ceil32(cols)] of packed rows."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    v = table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    v = v.reshape(*v.shape[:-1], -1, 32)
    e = scale[..., :v.shape[-2]].int() - 127
    return torch.ldexp(v, e[..., None]).flatten(-2)


def _routing(g, T, E, k, skew):
    """Router logits with an uneven popularity, the top-k choices and their gates."""
    z = torch.randn((T, E), generator=g, device=DEV)
    if skew == "normal":
        z += torch.randn(E, generator=g, device=DEV)
    elif skew == "zipf":
        z -= 1.2 * torch.log(torch.randperm(E, generator=g, device=DEV).float() + 1)
    top, idx = torch.topk(z, k, dim=1)
    return z, idx.int(), torch.softmax(top, 1)


def prepare(c, seed):
    g = _gen(seed)
    s = dict(case=c)
    if c["kind"] == "quant":
        rows, cols, dt = c["rows"], c["cols"], DT[c["dtype"]]
        W = _normal(g, (rows, cols), 1 / math.sqrt(cols))
        W *= torch.exp(torch.randn((rows, 1), generator=g, device=DEV))   # rows of different norms
        W[::97] = 0                                                       # experts' dead rows
        s.update(W=W.to(dt), codes=torch.empty((rows, -(-cols // 32) * 16), dtype=torch.uint8, device=DEV),
                 scale=torch.empty((rows, -(-cols // 128) * 4), dtype=torch.uint8, device=DEV),
                 out=torch.empty((rows, cols), dtype=dt, device=DEV))
        return s
    T, d = c["T"], c["d"]
    if c["kind"] == "experts":
        E, k, I, sh = c["E"], c["k"], c["I"], c["shared"]
        S = E + sh
        _, idx, _ = _routing(g, T, E, k, c["skew"])
        # rows of a slot ordered by token, as the permutation leaves them
        flat = idx.long().flatten()
        order = torch.sort(flat * T + torch.arange(T * k, device=DEV) // k)[0]
        count = torch.bincount(flat, minlength=E)
        offsets = torch.cat((count.new_zeros(1), count.cumsum(0)))
        s.update(X=_normal(g, (T, d), 1.0, torch.bfloat16), perm_token=(order % T).int(), offsets=offsets.int(),
                 slot=order // T, most=int(count.max()), O=torch.empty((T * (k + sh), d), dtype=torch.bfloat16, device=DEV))
        for m, (r, n) in dict(g=(I, d), u=(I, d), d=(d, I)).items():
            qs = [_pack(_normal(g, (r, n), 1 / math.sqrt(n))) for _ in range(S)]
            s["q" + m], s["s" + m] = torch.stack([q for q, _ in qs]), torch.stack([x for _, x in qs])
        if own:
            from paper_2508_19078_amd import api
            s["tables"] = api.LayerTablesMX4(d, I, E, sh, *(list(s[n]) for n in ("qg", "qu", "qd", "sg", "su", "sd")))
            s["ws"] = torch.empty(api.moe_grouped_swiglu_fwd_mx4_workspace_size(s["tables"], T, k), dtype=torch.uint8,
                                  device=DEV)
        return s
    dt = DT[c["dtype"]]
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    if c["kind"] == "balance":
        E, k, B = c["E"], c["k"], c["seqs"]
        z, idx, gate = _routing(g, T, E, k, "normal")
        cut = torch.sort(torch.randint(0, T + 1, (B - 1,), generator=g, device=DEV))[0]
        ends = torch.full((1,), T, device=DEV)
        s.update(logits=z, idx=idx, gate=gate, dgate=_normal(g, (T, k), 0.1),
                 seg=torch.cat((torch.zeros_like(ends), cut, ends)).int(),
                 keep=(torch.rand(T, generator=g, device=DEV) >= c["pad"]).to(torch.uint8) if c["pad"] else None,
                 X=_normal(g, (T, d), 1.0, dt), Wr=_normal(g, (E, d), 1 / math.sqrt(d), dt), coef=0.01,
                 dloss=torch.ones(1, device=DEV), counts=new(B, E, dtype=torch.int32), dprob=new(B, E), loss=new(1),
                 dlogits=new(T, E), dX=new(T, d, dtype=dt), dWr=new(E, d), dbias=new(E))
        if own:
            from paper_2508_19078_amd import api
            s["ws"] = torch.empty(max(api.moe_balance_loss_workspace_size(T, E, B),
                                      api.moe_router_bwd_workspace_size(T, d, E)), dtype=torch.uint8, device=DEV)
        return s
    s.update(Y=_normal(g, (T, d), 0.3, dt), alpha=1.25, gate=torch.rand(T, generator=g, device=DEV) if c["gate"] else None,
             w_post=1 + _normal(g, (d,), 0.1), w_pre=1 + _normal(g, (d,), 0.1))
    if not c["back"]:
        s.update(X=_normal(g, (T, d), 1.0, dt), S=new(T, d, dtype=dt), N=new(T, d, dtype=dt),
                 rstd_y=new(T) if c["post"] else None, rstd_s=new(T))
        return s
    rstd = lambda v: (v.double().square().mean(1) + EPS).rsqrt().float()  # noqa: E731
    S = _normal(g, (T, d), 1.5, dt)
    s.update(S=S, rstd_s=rstd(S), rstd_y=rstd(s["Y"]) if c["post"] else None, dS=_normal(g, (T, d), 0.1, dt),
             dN=_normal(g, (T, d), 0.1, dt), dX=new(T, d, dtype=dt), dY=new(T, d, dtype=dt),
             dgate=new(T) if c["gate"] else None, dw_post=new(d), dw_pre=new(d))
    if own:
        from paper_2508_19078_amd import api
        s["ws"] = torch.empty(api.moe_sublayer_norm_bwd_workspace_size(T, d), dtype=torch.uint8, device=DEV)
    return s


# -------------------------------------------------------------------- run ----

def run(s):
    return {"quant": _quant, "experts": _experts, "balance": _balance, "norm": _norm}[s["case"]["kind"]](s)


def _quant(s):
    if own:
        from paper_2508_19078_amd import api
        api.moe_quantize_mxfp4(s["W"], s["codes"], s["scale"])
        api.moe_dequant_mxfp4(s["codes"], s["scale"], s["out"])
        return s["out"]
    W = s["W"]
    return _values(W.float())[:, :W.shape[1]].to(W.dtype)


def _experts(s):
    c = s["case"]
    T, d, E, k, I, sh = (c[n] for n in ("T", "d", "E", "k", "I", "shared"))
    if own:
        from paper_2508_19078_amd import api
        api.moe_grouped_swiglu_fwd_mx4(s["tables"], s["X"], s["perm_token"], s["offsets"], T, k, s["O"], s["ws"])
        return s["O"]
    Xq = _values(s["X"].float())
    # every routed slot's rows, filled up to the fullest slot's
    at = s["slot"] * s["most"] + torch.arange(T * k, device=DEV) - s["offsets"].long()[s["slot"]]
    rows = torch.zeros(E * s["most"], dtype=torch.long, device=DEV)
    rows[at] = s["perm_token"].long()
    out = _ffn(Xq[rows].view(E, s["most"], -1), s, slice(0, E), I, d).flatten(0, 1)[at]
    if sh:
        out = torch.cat((out, _ffn(Xq.expand(sh, T, -1), s, slice(E, E + sh), I, d).flatten(0, 1)))
    return out


def _ffn(x, s, slots, I, d):
    wg, wu = (_unpack(s["q" + m][slots], s["s" + m][slots]).transpose(1, 2).contiguous() for m in "gu")
    a, u = torch.bmm(x, wg), torch.bmm(x, wu)
    del wg, wu
    h = _values(a / (1 + torch.exp(-a)) * u)
    del a, u
    wd = _unpack(s["qd"][slots], s["sd"][slots]).transpose(1, 2).contiguous()
    return torch.bmm(h, wd).to(torch.bfloat16)


def _balance(s):
    c = s["case"]
    if own:
        from paper_2508_19078_amd import api
        api.moe_balance_loss(s["logits"], s["idx"], s["coef"], s["counts"], s["dprob"], s["loss"], s["ws"],
                             seg=s["seg"], keep=s["keep"])
        api.moe_balance_loss_bwd(s["logits"], s["dprob"], s["dloss"], s["dlogits"], seg=s["seg"], keep=s["keep"],
                                 gate=s["gate"], idx=s["idx"], dgate=s["dgate"])
        api.moe_router_bwd(s["dlogits"], s["X"], s["Wr"], s["ws"], dX=s["dX"], dWr=s["dWr"], dbias=s["dbias"])
        return {n: s[n] for n in ("counts", "dprob", "loss", "dlogits", "dX", "dWr", "dbias")}
    T, E, k, B = c["T"], c["E"], c["k"], c["seqs"]
    z, idx, t = s["logits"], s["idx"].long(), torch.arange(T, device=DEV)
    p = torch.exp(z - z.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    of = (t[:, None] >= s["seg"].long()[None, 1:]).sum(1).clamp(max=B - 1)        # the token's sequence
    live = torch.ones(T, dtype=torch.bool, device=DEV) if s["keep"] is None else s["keep"] != 0
    member = ((of[None, :] == torch.arange(B, device=DEV)[:, None]) & live[None, :]).double()
    chosen = torch.zeros((T, E), dtype=torch.float64, device=DEV).scatter_(1, idx, 1.0)
    counts, n = member @ chosen, member.sum(1)
    dprob = c["E"] * s["coef"] * counts / (k * n.sum() * n[:, None]).clamp(min=1)
    loss = (dprob * (member @ p.double())).sum().reshape(1)
    w = dprob.float()[of] * live[:, None]
    dz = s["dloss"] * p * (w - (p * w).sum(1, keepdim=True))
    gate, dg = s["gate"], s["dgate"]
    dz = dz.scatter_add(1, idx, gate * (dg - (gate * dg).sum(1, keepdim=True)))
    dt = s["X"].dtype
    return {"counts": counts.int(), "dprob": dprob.float(), "loss": loss.float(), "dlogits": dz,
            "dX": (dz @ s["Wr"].float()).to(dt), "dWr": dz.t().contiguous() @ s["X"].float(), "dbias": dz.double().sum(0).float()}


def _norm(s):
    c = s["case"]
    if own:
        from paper_2508_19078_amd import api
        how = dict(alpha=s["alpha"], gate=s["gate"], w_post=s["w_post"], w_pre=s["w_pre"], post_norm=c["post"])
        if not c["back"]:
            api.moe_sublayer_norm(s["X"], s["Y"], s["S"], s["N"], eps=EPS, rstd_y=s["rstd_y"], rstd_s=s["rstd_s"], **how)
            return {"S": s["S"], "N": s["N"]}
        api.moe_sublayer_norm_bwd(s["dS"], s["dN"], s["S"], s["Y"], s["rstd_s"], s["dX"], s["dY"], s["ws"],
                                  rstd_y=s["rstd_y"], dgate=s["dgate"], dw_post=s["dw_post"], dw_pre=s["dw_pre"], **how)
        return {n: s[n] for n in ("dX", "dY", "dw_post", "dw_pre") + (("dgate",) if c["gate"] else ())}
    dt, Y = s["Y"].dtype, s["Y"].float()
    g = s["gate"][:, None] if c["gate"] else 1.0
    if not c["back"]:
        u = Y * torch.rsqrt((Y * Y).mean(1, keepdim=True) + EPS) if c["post"] else Y
        S = (s["alpha"] * s["X"].float() + g * (u * s["w_post"])).to(dt)
        f = S.float()
        return {"S": S, "N": (f * torch.rsqrt((f * f).mean(1, keepdim=True) + EPS) * s["w_pre"]).to(dt)}
    u = Y * s["rstd_y"][:, None] if c["post"] else Y
    r, dN = s["rstd_s"][:, None], s["dN"].float()
    x = s["S"].float() * r
    q = dN * s["w_pre"]
    dS = s["dS"].float() + r * (q - x * (q * x).mean(1, keepdim=True))
    dY = g * dS * s["w_post"]
    if c["post"]:
        dY = s["rstd_y"][:, None] * (dY - u * (dY * u).mean(1, keepdim=True))
    out = {"dX": (s["alpha"] * dS).to(dt), "dY": dY.to(dt), "dw_pre": (dN * x).double().sum(0).float(),
           "dw_post": (g * dS * u).double().sum(0).float()}
    if c["gate"]:
        out["dgate"] = (dS * u * s["w_post"]).sum(1)
    return out


# ------------------------------------------------------------------ exact ----

def exact(c, seed):
    s = prepare(c, seed)
    return {"quant": _exact_quant, "experts": _exact_experts, "balance": _exact_balance, "norm": _exact_norm}[c["kind"]](s)


def _nearest(x):
    """MXFP4 of rows in fp64: the nearest of the 15 values, ties to the even code."""
    n = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, -n % 32)).unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top)))) - 2)
    # log2 may round up to a whole number just below a power of two
    scale = torch.where(scale * 4 > top, scale / 2, scale)
    scale = torch.where(top > 0, scale, torch.ones_like(scale))
    a = x.abs() / scale
    at = torch.zeros_like(a, dtype=torch.long)
    for code in range(7):
        mid = (E2M1[code] + E2M1[code + 1]) / 2
        at += (a > mid) | ((a == mid) & (code % 2 == 1))
    v = torch.tensor(E2M1, dtype=torch.float64, device=x.device)[at]
    return (torch.sign(x) * v * scale).flatten(-2)[..., :n]


def _exact_quant(s):
    W = s["W"]
    step = 8192
    return torch.cat([_nearest(W[i:i + step].double()) for i in range(0, W.shape[0], step)])


def _exact_experts(s):
    c = s["case"]
    T, d, E, k, I, sh = (c[n] for n in ("T", "d", "E", "k", "I", "shared"))
    X = _nearest(s["X"].double())
    out = torch.empty((T * (k + sh), d), dtype=torch.float64, device=DEV)
    at = s["offsets"].tolist()
    for e in range(E + sh):
        r0, r1 = (at[e], at[e + 1]) if e < E else (T * (k + e - E), T * (k + e - E + 1))
        if r0 == r1:
            continue
        wg, wu, wd = (_unpack(s["q" + m][e], s["s" + m][e]).double()[:, :n] for m, n in (("g", d), ("u", d), ("d", I)))
        for i in range(r0, r1, 4096):
            j = min(r1, i + 4096)
            x = X[s["perm_token"][i:j].long()] if e < E else X[i - r0:j - r0]
            a = x @ wg.T
            out[i:j] = _nearest(a * torch.sigmoid(a) * (x @ wu.T)) @ wd.T
    return out


def _exact_balance(s):
    c = s["case"]
    T, E, k, B = c["T"], c["E"], c["k"], c["seqs"]
    z, idx, at = s["logits"].double(), s["idx"].long(), s["seg"].tolist()
    p = torch.softmax(z, 1)
    live = torch.ones(T, dtype=torch.bool, device=DEV) if s["keep"] is None else s["keep"].bool()
    n = int(live.sum())
    counts = torch.zeros((B, E), dtype=torch.int32, device=DEV)
    dprob = torch.zeros((B, E), dtype=torch.float64, device=DEV)
    loss = torch.zeros(1, dtype=torch.float64, device=DEV)
    dz = torch.zeros_like(p)
    for b in range(B):
        m = live[at[b]:at[b + 1]]
        if not bool(m.any()):
            continue
        own_idx, pb = idx[at[b]:at[b + 1]][m], p[at[b]:at[b + 1]]
        counts[b] = torch.bincount(own_idx.flatten(), minlength=E).int()
        dprob[b] = s["coef"] * E * counts[b].double() / (float(k) * n * int(m.sum()))
        loss += (pb[m].sum(0) * dprob[b]).sum()
        dz[at[b]:at[b + 1]] = m[:, None] * pb * (dprob[b] - (pb @ dprob[b])[:, None])
    dz *= s["dloss"].double()
    gate, dg = s["gate"].double(), s["dgate"].double()
    for j in range(k):
        dz[torch.arange(T, device=DEV), idx[:, j]] += gate[:, j] * (dg[:, j] - (gate * dg).sum(1))
    return {"counts": counts, "dprob": dprob, "loss": loss, "dlogits": dz, "dX": dz @ s["Wr"].double(),
            "dWr": dz.T @ s["X"].double(), "dbias": dz.sum(0)}


def _exact_norm(s):
    c = s["case"]
    dt, d = s["Y"].dtype, c["d"]
    Y, a, b = s["Y"].double(), s["w_post"].double(), s["w_pre"].double()
    one = torch.ones((c["T"], 1), dtype=torch.float64, device=DEV)
    g = s["gate"].double()[:, None] if c["gate"] else one
    if not c["back"]:
        ry = (Y.square().mean(1, keepdim=True) + EPS).rsqrt() if c["post"] else one
        S = s["alpha"] * s["X"].double() + g * ry * Y * a
        kept = S.to(dt).double()                          # the stream is kept in its type
        return {"S": S, "N": kept * (kept.square().mean(1, keepdim=True) + EPS).rsqrt() * b}
    ry = s["rstd_y"].double()[:, None] if c["post"] else one
    S, rs, dN = s["S"].double(), s["rstd_s"].double()[:, None], s["dN"].double()
    dS = s["dS"].double() + rs * b * dN - S * rs ** 3 / d * (S * b * dN).sum(1, keepdim=True)
    dv = g * dS * a
    out = {"dX": s["alpha"] * dS, "dY": ry * dv - (Y * ry ** 3 / d * (Y * dv).sum(1, keepdim=True) if c["post"] else 0.0),
           "dw_pre": (dN * S * rs).sum(0), "dw_post": (g * dS * ry * Y).sum(0)}
    if c["gate"]:
        out["dgate"] = (dS * ry * Y * a).sum(1)
    return out
