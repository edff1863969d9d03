"""The operators that surround the quantized linears of a transformer block, as cases that can be prepared, run, checked and timed.

  norm     layer norm or its RMS form.  train: the forward call and the backward call with the reduction of the parameters'
           gradients, the input kept for the backward pass in 8 bits ("bits8") or as it is ("source"); else the forward alone
  act      the nonlinearity between the linears of an MLP: "swiglu" on [N, 2F] (gate, then up) or "gelu" (tanh form) on [N, F];
           train and keep as above
  ckpt     an activation of another operator kept in 8 bits and brought back
  product  weights packed as NVFP4 (two E2M1 codes per byte, an E4M3 scale per 16, FP32 outer scales) times the bf16
           activations of M tokens, for answers token by token

An 8-bit checkpoint holds E4M3 codes and one power of two per 128 elements of a row: the least 2^e (e from -126 to 120) with
max |x| <= 448 * 2^e.  Where `own` is false the operators are computed in their plain form, elementary torch operations in 32
bits; where it is true by the library's calls.
"""
import math

import torch
import torch.nn.functional as F

own = False

EPS = 1e-5
GROUP = 128                                   # elements of a row that share a power of two in an 8-bit checkpoint
GELU_C = 2.0 * math.sqrt(2.0 / math.pi)
GELU_A = 0.044715
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


# ------------------------------------------------------------------------------------------------------ the cases ----

def listed():
    return [
        # the norm of the 1024-hidden model while it answers: one token, launch and host time
        dict(name="norm_answer_1x1024", kind="norm", N=1, D=1024, norm="layer", type="bf16", keep="source", train=False),
        # a training step of the same norm: 16 sequences of 1024 tokens, its input kept in 8 bits
        dict(name="norm_16384x1024_bits8", kind="norm", N=16384, D=1024, norm="layer", type="bf16", keep="bits8", train=True),
        # the RMS norm of the 768-hidden model, 8 sequences of 1024 tokens, its input kept as it is
        dict(name="norm_8192x768_rms", kind="norm", N=8192, D=768, norm="rms", type="bf16", keep="source", train=True),
        # hidden size 16384, micro-batch 4 of 1024 tokens: long rows
        dict(name="norm_4096x16384_bits8", kind="norm", N=4096, D=16384, norm="layer", type="bf16", keep="bits8", train=True),
        # a residual stream in binary32 of an odd width (rows that start at no vector's alignment)
        dict(name="norm_1000x1023_f32", kind="norm", N=1000, D=1023, norm="layer", type="f32", keep="source", train=True),
        # between gate_up and down of the 1024-hidden model
        dict(name="swiglu_16384x4096_bits8", kind="act", N=16384, F=4096, act="swiglu", type="bf16", keep="bits8", train=True),
        # an MLP without a gate, packed sequences of odd total length
        dict(name="gelu_4099x2752_bits8", kind="act", N=4099, F=2752, act="gelu", type="bf16", keep="bits8", train=True),
        # an activation of the square layer, kept from the forward to the backward pass
        dict(name="ckpt_8192x8192", kind="ckpt", N=8192, D=8192, type="bf16"),
        # gate and up projection of the 1024-hidden model for one token
        dict(name="product_1x1024x8192", kind="product", M=1, D=1024, C=8192, outer="tensor", f32=False),
        # the square layer for one token
        dict(name="product_1x8192x8192", kind="product", M=1, D=8192, C=8192, outer="tensor", f32=False),
        # 16 answers at once, 1 x 128 outer blocks, hidden size 4096
        dict(name="product_16x4096x4096_block", kind="product", M=16, D=4096, C=4096, outer="block", f32=False),
        # an odd number of answers, outputs in binary32 (logits and sums that go on), ragged output width
        dict(name="product_5x2064x5003_f32", kind="product", M=5, D=2064, C=5003, outer="tensor", f32=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "act", "act", "ckpt", "product", "product", "product"])
    type_ = rng.choice(["bf16", "bf16", "f32"])
    most = 1 << (26 if type_ == "bf16" else 25)
    keep = rng.choice(["bits8", "source"])
    train = rng.random() < 0.8
    if kind == "norm":
        D = _log(rng, 64, 16384)
        N = min(_log(rng, 1, 16384), most // D)
        return dict(kind="norm", N=N, D=D, norm=rng.choice(["layer", "rms"]), type=type_, keep=keep, train=train)
    if kind == "act":
        Fw = _log(rng, 64, 16384)
        N = min(_log(rng, 1, 16384), most // Fw)
        return dict(kind="act", N=N, F=Fw, act=rng.choice(["swiglu", "gelu"]), type=type_, keep=keep, train=train)
    if kind == "ckpt":
        D = _log(rng, 64, 16384)
        return dict(kind="ckpt", N=min(_log(rng, 1, 16384), most // D), D=D, type=type_)
    outer = rng.choice(["tensor", "block"])
    unit = 16 if outer == "tensor" else 128
    D = unit * max(1, _log(rng, 128, 16384) // unit)
    C = min(_log(rng, 64, 16384), (1 << 26) // D)
    return dict(kind="product", M=_log(rng, 1, 64), D=D, C=C, outer=outer, f32=rng.random() < 0.3)


# ----------------------------------------------------------------------------------------------------- the inputs ----

def _type(case):
    return torch.bfloat16 if case["type"] == "bf16" else torch.float32


def _draws(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _activations(normal, rows, cols):
    """N(0, 1) with one entry in a thousand 50 times as large."""
    x = normal(rows, cols)
    return torch.where(normal(rows, cols) > 3.09, x * 50.0, x)


def _packed(w, outer):
    """Codes, scale bytes and outer scales of a float32 [C, D] matrix, rounded to nearest."""
    C, D = w.shape
    top = w.abs().amax().reshape(1, 1) if outer == "tensor" else w.abs().view(C, D // GROUP, GROUP).amax(2)
    gscale = top / 2688.0
    per16 = gscale.expand(C, D // 16) if outer == "tensor" else gscale.repeat_interleave(GROUP // 16, 1)
    g = w.view(C, D // 16, 16)
    scales = (g.abs().amax(2) / 6.0 / per16).to(torch.float8_e4m3fn)
    step = scales.float() * per16
    y = torch.where(step[..., None] > 0, g / step[..., None], torch.zeros_like(g))
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=w.device)
    code = (torch.bucketize(y.abs(), edges) + 8 * (y < 0)).to(torch.uint8).view(C, D // 2, 2)
    return (code[..., 0] | (code[..., 1] << 4)).contiguous(), scales.view(torch.uint8).contiguous(), gscale.view(-1).contiguous() if outer == "tensor" else gscale.contiguous()


def prepare(case, seed):
    normal = _draws(seed)
    s = {"case": case}
    if case["kind"] == "norm":
        N, D, t = case["N"], case["D"], _type(case)
        s["x"] = _activations(normal, N, D).to(t)
        s["gamma"] = 1.0 + 0.1 * normal(D)
        s["beta"] = 0.1 * normal(D) if case["norm"] == "layer" else None
        s["dy"] = (1e-3 * normal(N, D)).to(t)
    elif case["kind"] == "act":
        N, Fw, t = case["N"], case["F"], _type(case)
        s["h"] = _activations(normal, N, Fw * (2 if case["act"] == "swiglu" else 1)).to(t)
        s["da"] = (1e-3 * normal(N, Fw)).to(t)
    elif case["kind"] == "ckpt":
        s["x"] = _activations(normal, case["N"], case["D"]).to(_type(case))
    else:
        s["x"] = _activations(normal, case["M"], case["D"]).to(torch.bfloat16)
        s["codes"], s["scales"], s["gscale"] = _packed(0.02 * normal(case["C"], case["D"]), case["outer"])
    return s


# ------------------------------------------------------------------------------------------------------ one pass ----

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2510_27527_amd as tj
    B = tj.binding
    case = s["case"]
    if case["kind"] == "product":
        W = tj.NVFP4Tensor(s["codes"], s["scales"], s["gscale"], None, case["C"], case["D"], B.OUTER_TENSOR if case["outer"] == "tensor" else B.OUTER_BLOCK128)
        return {"y": tj.gemv(s["x"], W, B.OUT_F32 if case["f32"] else B.OUT_BF16)}
    out = B.OUT_BF16 if case["type"] == "bf16" else B.OUT_F32
    if case["kind"] == "ckpt":
        return {"x": tj.ckpt8_load(tj.ckpt8_save(s["x"]), out)}
    if case["kind"] == "norm":
        norm = B.NORM_LAYER if case["norm"] == "layer" else B.NORM_RMS
        if not case["train"]:
            return {"y": tj.norm_fwd(s["x"], s["gamma"], s["beta"], eps=EPS, norm=norm, out_dtype=out)}
        stats = tj.alloc_stats(case["N"])
        kept = tj.alloc_ckpt8(case["N"], case["D"]) if case["keep"] == "bits8" else None
        y = tj.norm_fwd(s["x"], s["gamma"], s["beta"], eps=EPS, norm=norm, out_dtype=out, stats=stats, ckpt=kept)
        dx, dgamma, dbeta = tj.norm_bwd(s["dy"], s["x"] if kept is None else kept, stats, s["gamma"], norm=norm, out_dtype=out)
        return {"y": y, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    act = B.ACT_SWIGLU if case["act"] == "swiglu" else B.ACT_GELU
    if not case["train"]:
        return {"a": tj.act_fwd(s["h"], act, out)}
    kept = tj.alloc_act_ckpt8(case["N"], case["F"], act) if case["keep"] == "bits8" else None
    a = tj.act_fwd(s["h"], act, out, ckpt=kept)
    return {"a": a, "dh": tj.act_bwd(s["da"], s["h"] if kept is None else kept, act, out)}


def _kept(x):
    """What an 8-bit checkpoint of x brings back, in 32 bits; rows in groups of 128, the last of a row may be shorter."""
    x = x.float()
    N, D = x.shape
    g = F.pad(x, (0, -D % GROUP)).view(N, -1, GROUP)
    m, p = torch.frexp(torch.where(torch.isfinite(g), g.abs(), torch.zeros_like(g)).amax(2, keepdim=True))
    e = (p - 9 + (m > 0.875).int()).clamp(-126, 120)
    e = torch.where(m == 0, torch.full_like(e, -126), e)
    code = torch.ldexp(g, -e).to(torch.float8_e4m3fn)
    return torch.ldexp(code.float(), e).view(N, -1)[:, :D]


def _sigmoid(z):
    return 1.0 / (1.0 + torch.exp(-z))


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "product":
        codes = s["codes"]
        table = torch.tensor(E2M1, device=codes.device)
        w = table[torch.stack((codes & 15, codes >> 4), 2).long()].view(case["C"], -1, 16) * s["scales"].view(torch.float8_e4m3fn).float()[..., None]
        w = w.view(case["C"], -1, GROUP) * s["gscale"][..., None] if case["outer"] == "block" else w * s["gscale"]
        y = s["x"].float() @ w.reshape(case["C"], case["D"]).t()
        return {"y": y if case["f32"] else y.to(torch.bfloat16)}
    t = _type(case)
    if case["kind"] == "ckpt":
        return {"x": _kept(s["x"]).to(t)}
    if case["kind"] == "norm":
        x, layer = s["x"].float(), case["norm"] == "layer"
        mean = x.mean(1, keepdim=True) if layer else torch.zeros_like(x[:, :1])
        rstd = 1.0 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
        y = (x - mean) * rstd * s["gamma"]
        out = {"y": (y + s["beta"] if layer else y).to(t)}
        if not case["train"]:
            return out
        xh = ((_kept(s["x"]) if case["keep"] == "bits8" else x) - mean) * rstd
        dy = s["dy"].float()
        g = dy * s["gamma"]
        dx = g - xh * (g * xh).mean(1, keepdim=True)
        out["dx"] = (rstd * (dx - g.mean(1, keepdim=True) if layer else dx)).to(t)
        out["dgamma"] = (dy * xh).sum(0)
        out["dbeta"] = dy.sum(0) if layer else None
        return out
    h = s["h"].float()
    Fw, swiglu = case["F"], case["act"] == "swiglu"
    if swiglu:
        g, u = h[:, :Fw], h[:, Fw:]
        out = {"a": (g * _sigmoid(g) * u).to(t)}
    else:
        out = {"a": (h * _sigmoid(GELU_C * (h + GELU_A * h * h * h))).to(t)}
    if not case["train"]:
        return out
    da = s["da"].float()
    if case["keep"] == "bits8":                   # gate and up are rows of their own in a checkpoint
        h = _kept(s["h"].reshape(-1, Fw)).reshape(h.shape)
    if swiglu:
        g, u = h[:, :Fw], h[:, Fw:]
        sg = _sigmoid(g)
        dh = torch.cat((da * u * sg * (1.0 + g * (1.0 - sg)), da * g * sg), 1)
    else:
        sg = _sigmoid(GELU_C * (h + GELU_A * h * h * h))
        dh = da * (sg + h * sg * (1.0 - sg) * GELU_C * (1.0 + 3.0 * GELU_A * h * h))
    out["dh"] = dh.to(t)
    return out


# ------------------------------------------------------------------------------------- the definition in 64 bits ----

def _exact_kept(x):
    """Rounding to E4M3 as a multiple of the unit of the value's own binade: units of 2^(floor(log2 |v|) - 3), not below 2^-9."""
    x = x.double()
    N, D = x.shape
    width = -(-D // GROUP) * GROUP
    v = torch.zeros(N, width, dtype=torch.float64, device=x.device)
    v[:, :D] = x
    v = v.view(N, width // GROUP, GROUP)
    a = torch.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0).abs().max(2, keepdim=True).values
    e = torch.ceil(torch.log2(a.clamp_min(2.0 ** -140) / 448.0))
    e = torch.where(a > 448.0 * torch.exp2(e), e + 1, e)
    e = torch.where(a <= 448.0 * torch.exp2(e - 1), e - 1, e).clamp(-126.0, 120.0)
    v = v * torch.exp2(-e)
    unit = torch.exp2((torch.frexp(v).exponent.double() - 4.0).clamp_min(-9.0))
    return (torch.round(v / unit) * unit * torch.exp2(e)).reshape(N, width)[:, :D]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "product":
        C, D = case["C"], case["D"]
        low, high = s["codes"].long() & 7, (s["codes"].long() >> 4) & 7
        sign = torch.stack((1.0 - (s["codes"] & 8).double() / 4.0, 1.0 - (s["codes"] >> 7).double() * 2.0), 2).view(C, D)
        idx = torch.stack((low, high), 2).view(C, D)
        mag = torch.where(idx < 2, idx * 0.5, (1.0 + 0.5 * (idx % 2)) * torch.exp2((idx // 2 - 1).double()))
        b = s["scales"].long()
        scale = torch.where(b < 8, b * 2.0 ** -9, (8.0 + b % 8) * torch.exp2((b // 8 - 10).double()))
        w = sign * mag * scale.repeat_interleave(16, 1)
        del sign, mag, idx
        w = w * (s["gscale"].double() if case["outer"] == "tensor" else s["gscale"].double().repeat_interleave(GROUP, 1))
        return {"y": torch.matmul(s["x"].double(), w.t().contiguous())}
    if case["kind"] == "ckpt":
        return {"x": _exact_kept(s["x"])}
    bits8 = case["keep"] == "bits8"
    if case["kind"] == "norm":
        x, gamma = s["x"].double(), s["gamma"].double()
        N, D = x.shape
        mu = x.sum(1, keepdim=True) / D if case["norm"] == "layer" else 0.0
        r = ((x - mu).pow(2).sum(1, keepdim=True) / D + EPS).rsqrt()
        out = {"y": (x - mu) * r * gamma + (s["beta"].double() if s["beta"] is not None else 0.0)}
        if case["train"]:
            z = ((_exact_kept(s["x"]) if bits8 else x) - mu) * r
            dy = s["dy"].double()
            along = (dy * gamma * z).sum(1, keepdim=True) / D
            shift = (dy * gamma).sum(1, keepdim=True) / D if case["norm"] == "layer" else 0.0
            out["dx"] = (dy * gamma - shift - z * along) * r
            out["dgamma"] = (dy * z).sum(0)
            out["dbeta"] = dy.sum(0) if case["norm"] == "layer" else None
        return out
    Fw = case["F"]
    h = s["h"].double()
    k = _exact_kept(s["h"].reshape(-1, Fw)).reshape(h.shape) if bits8 else h
    da = s["da"].double()
    if case["act"] == "swiglu":
        out = {"a": h[:, :Fw] * torch.sigmoid(h[:, :Fw]) * h[:, Fw:]}
        if case["train"]:
            sg = torch.sigmoid(k[:, :Fw])
            out["dh"] = torch.cat((da * k[:, Fw:] * (sg + k[:, :Fw] * sg * torch.sigmoid(-k[:, :Fw])), da * k[:, :Fw] * sg), 1)
        return out
    root = math.sqrt(2.0 / math.pi)
    out = {"a": 0.5 * h * (1.0 + torch.tanh(root * (h + GELU_A * h.pow(3))))}
    if case["train"]:
        th = torch.tanh(root * (k + GELU_A * k.pow(3)))
        out["dh"] = da * (0.5 * (1.0 + th) + 0.5 * k * (1.0 - th * th) * root * (1.0 + 3.0 * GELU_A * k.pow(2)))
    return out


# ----------------------------------------------------------------------------------------- what a pass must cost ----

def work(case):
    """Bytes: each input read once and each output written once, the checkpoint written by the forward and read by the backward call."""
    if case["kind"] == "product":
        M, D, C = case["M"], case["D"], case["C"]
        gs = 4.0 if case["outer"] == "tensor" else 4.0 * C * D / GROUP
        return {"bytes": C * D * 0.5625 + gs + 2.0 * M * D + M * C * (4.0 if case["f32"] else 2.0), "flops": 2.0 * M * D * C}
    e = 2.0 if case["type"] == "bf16" else 4.0
    bits8 = 1.0 + 1.0 / GROUP
    if case["kind"] == "ckpt":
        n = float(case["N"] * case["D"])
        return {"bytes": n * (e + bits8) + n * (bits8 + e), "flops": 2.0 * n}
    kept = bits8 if case["keep"] == "bits8" else 0.0
    if case["kind"] == "norm":
        n, D = float(case["N"] * case["D"]), case["D"]
        fwd = n * 2 * e + 8.0 * D
        if not case["train"]:
            return {"bytes": fwd, "flops": 8.0 * n}
        return {"bytes": fwd + n * kept + 8.0 * case["N"] + n * (2 * e + (kept or e)) + 8.0 * case["N"] + 12.0 * D, "flops": 22.0 * n}
    n, parts = float(case["N"] * case["F"]), 2.0 if case["act"] == "swiglu" else 1.0
    fwd = n * e * (parts + 1)
    if not case["train"]:
        return {"bytes": fwd, "flops": 6.0 * n}
    return {"bytes": fwd + n * parts * kept + n * e * (1 + parts) + n * parts * (kept or e), "flops": 18.0 * n}
