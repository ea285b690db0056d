"""The operators around the quantized layers of a transformer block, as cases that can be timed and compared.

A case is one call of one operator:

  kind "matvec"  segquant_w4_matvec: few rows times 4-bit weights with one scale (and zero-point) per channel and group of
                 inputs, the activation function in front, bias behind
  kind "pack"    segquant_quantize_w4_group and segquant_dequantize_w4_group: a weight matrix to those 4-bit weights and back
  kind "norm"    segquant_block_norm: end of one block and start of the next, H = R + alpha gate post(Y) and
                 O = norm(H) (1 + scale) + shift
  kind "codes"   segquant_block_norm_quantize: the same with O handed on as the e4m3 codes of the layer behind it

With `own` false `run` computes them in elementary torch operations, with `own` true through the package.
"""
import math

import torch

own = False

_E4M3 = torch.float8_e4m3fn


def _matvec(name, M, K, N, G, x="bf16", y="bf16", s="f32", zp=False, act="none"):
    return {"name": name, "kind": "matvec", "M": M, "K": K, "N": N, "G": G, "x": x, "y": y, "s": s, "zp": zp, "act": act}


def _pack(name, N, K, G, x="f32", s="f32", zp=False, out="bf16"):
    return {"name": name, "kind": "pack", "N": N, "K": K, "G": G, "x": x, "s": s, "zp": zp, "out": out}


def _norm(name, kind, M, C, T, x="bf16", p="bf16", pre="layer", post="none", res=True, mod=True, affine=False, alpha=1.0,
          P=1, dual=False):
    return {"name": name, "kind": kind, "M": M, "C": C, "T": T, "x": x, "p": p, "pre": pre, "post": post, "res": res,
            "mod": mod, "affine": affine, "alpha": alpha, "P": P, "dual": dual}


def listed():
    return [
        # adaLN projection of one conditioning vector, SiLU in front (DiT-XL/2): the smallest call, latency
        _matvec("matvec_adaln_1", 1, 1152, 6912, 128, act="silu"),
        # the same projection of an MMDiT block for a batch of 8, finer groups
        _matvec("matvec_adaln_8", 8, 1536, 9216, 64, act="silu"),
        # sizes that no tile divides, fp32 in and out, the finest groups with zero-points
        _matvec("matvec_ragged_f32", 5, 1111, 1003, 32, x="f32", y="f32", zp=True),
        # one token through a wide projection: the largest stream of weights
        _matvec("matvec_wide_1", 1, 8192, 28672, 128, s="bf16", zp=True),
        # a layer of an MMDiT block as it is loaded: fp32 weights, one scale per 128 inputs
        _pack("pack_fc1", 6144, 1536, 128),
        # a large layer kept in bf16, fine groups with zero-points
        _pack("pack_wide_zp", 18432, 4608, 32, x="bf16", s="bf16", zp=True),
        # a few tokens, fp32 activations, odd width: plain RMS norm with its weight
        _norm("norm_tokens_f32", "norm", 3, 1111, 3, x="f32", p="f32", pre="rms", res=False, mod=False, affine=True),
        # DiT-XL/2: gated residual and the modulated norm of the next block, 256 tokens per sample
        _norm("norm_dit", "norm", 2048, 1152, 256),
        # norms before and after the block, residual scale, one weight vector each
        _norm("norm_sandwich", "norm", 8858, 1536, 8858, pre="rms", post="rms", mod=False, affine=True, alpha=0.22),
        # one conditioning vector's batch of tokens straight to the codes of a DualScale layer, fp32, two K-segments
        _norm("codes_few_f32", "codes", 24, 1280, 8, x="f32", p="f32", P=2, dual=True),
        # MMDiT: gated residual and modulated norm straight to the codes of the QKV projection
        _norm("codes_mmdit", "codes", 8858, 1536, 4429),
        # SDXL-like block of 1280 channels at many tokens: residual, affine norm, codes
        _norm("codes_sdxl", "codes", 32768, 1280, 4096, mod=False, affine=True),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["matvec", "matvec", "matvec", "pack", "norm", "norm", "codes", "codes"])
    if kind in ("matvec", "pack"):
        while True:
            K, N = int(_log_uniform(rng, 64, 16384)), int(_log_uniform(rng, 64, 28672))
            if rng.random() < 0.7:
                K, N = K // 32 * 32, N // 16 * 16
            if K * N <= (8192 * 28672 if kind == "matvec" else 18432 * 4608):
                break
        G, s, zp = rng.choice([32, 64, 128, 128, 256]), rng.choice(["f32", "bf16"]), rng.random() < 0.5
        x = rng.choice(["bf16", "bf16", "f32"])
        if kind == "pack":
            c = _pack("", N, K, G, x, s, zp, rng.choice(["bf16", "f32"]))
        else:
            c = _matvec("", int(_log_uniform(rng, 1, 17)), K, N, G, x, rng.choice(["bf16", "bf16", "f32"]), s, zp,
                        rng.choice(["none", "none", "silu", "gelu"]))
    else:
        while True:
            M, C = int(_log_uniform(rng, 1, 32769)), int(_log_uniform(rng, 64, 12289))
            if rng.random() < 0.75:
                C = C // 8 * 8
            if M * C <= 8858 * 1536:
                break
        post = rng.choice(["none", "none", "rms", "layer"])
        c = _norm("", kind, M, C, rng.choice([1, 64, 256, 4429, M]), rng.choice(["bf16", "bf16", "f32"]),
                  rng.choice(["bf16", "f32"]), rng.choice(["layer", "rms"]), post, post != "none" or rng.random() < 0.7,
                  rng.random() < 0.6, rng.random() < 0.4, rng.choice([1.0, 1.0, 0.22]),
                  rng.choice([1, 1, 2, 3]) if kind == "codes" else 1, kind == "codes" and rng.random() < 0.4)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs

def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _pitched(t, dtype):
    """A copy of a matrix with rows on 16-byte boundaries, as the package wants them."""
    rows, cols = t.shape
    buf = torch.zeros((rows, (cols + 7) // 8 * 8), dtype=dtype, device="cuda")
    buf[:, :cols] = t
    return buf[:, :cols]


def _inputs(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "matvec":
        M, K, N = c["M"], c["K"], c["N"]
        groups = -(-K // c["G"])
        s["X"] = _randn(g, M, K).to(_dtype(c["x"]))
        Kb = (K + 1) // 2
        buf = torch.randint(0, 256, (N, -(-Kb // 16) * 16), generator=g, device="cuda", dtype=torch.uint8)
        if not c["zp"]:                                  # symmetric codes are in [-7, 7]: 0x8 becomes 0x9
            low, high = buf & 15, buf & 240
            buf = torch.where(low == 8, 9, low) | torch.where(high == 128, 144, high)
        s["W4"] = buf[:, :Kb]
        scale = (0.5 + torch.rand((groups, -(-N // 16) * 16), generator=g, device="cuda")) * 0.005
        s["s_w"] = scale.to(_dtype(c["s"]))[:, :N]
        s["z_w"] = None
        if c["zp"]:
            s["z_w"] = torch.randint(-3, 4, (groups, -(-N // 16) * 16), generator=g, device="cuda", dtype=torch.int8)[:, :N]
        s["bias"] = _randn(g, N) * 0.1
    elif c["kind"] == "pack":
        W = _randn(g, c["N"], c["K"]) * 0.02
        W *= torch.exp(0.5 * _randn(g, c["N"], 1))       # channels of different ranges
        s["W"] = _pitched(W, _dtype(c["x"]))
    else:
        M, C, T = c["M"], c["C"], c["T"]
        dt, pt = _dtype(c["x"]), _dtype(c["p"])
        s["R"] = _pitched(_randn(g, M, C) * (1.0 + 2.0 * torch.rand((M, 1), generator=g, device="cuda")) + 0.3, dt)
        s["Y"] = _pitched(_randn(g, M, C) * 1.5, dt) if c["res"] else None
        for k in ("gate", "scale", "shift", "w", "b", "post_w", "post_b"):
            s[k] = None
        if c["mod"]:                                     # the chunks of one projection of the conditioning vectors
            six = (_randn(g, -(-M // T), 6 * C) * 0.3).to(pt)
            s["shift"], s["scale"] = six[:, :C], six[:, C:2 * C]
            s["gate"] = six[:, 5 * C:] if c["res"] else None
        if c["affine"]:
            s["w"] = (1.0 + 0.2 * _randn(g, C)).to(pt)
            s["b"] = (0.2 * _randn(g, C)).to(pt) if c["pre"] == "layer" else None
        if c["post"] != "none":
            s["post_w"] = (1.0 + 0.2 * _randn(g, C)).to(pt)
            s["post_b"] = (0.2 * _randn(g, C)).to(pt) if c["post"] == "layer" else None
        if c["kind"] == "codes":
            P = min(c["P"], C)
            s["kb"] = [C * p // P for p in range(P)] + [C]
            s["s_pos"] = (4.0 + torch.rand((P,), generator=g, device="cuda")) / 448.0
            s["s_neg"] = s["s_pos"] * 0.75 if c["dual"] else None
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# ------------------------------------------------------------------------------------------------ plain forms

def _codes_of(W4, K):
    """Signed 4-bit codes of packed rows, code 2 j in the low nibble of byte j."""
    both = torch.stack((W4 & 15, W4 >> 4), 2).reshape(W4.shape[0], -1)[:, :K]
    return (both ^ 8).to(torch.int8) - 8


def _per_input(t, G, K):
    """[groups, N] -> [N, K]."""
    return t.t().repeat_interleave(G, 1)[:, :K]


def _weights(W4, s_w, z_w, G, K):
    c = _codes_of(W4, K).float()
    if z_w is not None:
        c -= _per_input(z_w, G, K)
    return c * _per_input(s_w.float(), G, K)


def _act32(x, act):
    if act == "silu":
        return x * torch.sigmoid(x)
    if act == "gelu":
        return x * 0.5 * torch.special.erfc(x * -math.sqrt(0.5))
    return x


def _plain_matvec(s):
    c = s["case"]
    x = _act32(s["X"].float(), c["act"])
    y = x @ _weights(s["W4"], s["s_w"], s["z_w"], c["G"], c["K"]).t() + s["bias"]
    return y.to(_dtype(c["y"]))


def _grouped(W, G):
    N, K = W.shape
    full = torch.zeros((N, -(-K // G) * G), dtype=W.dtype, device=W.device)
    full[:, :K] = W
    return full.view(N, -1, G)


def _plain_pack(s):
    c = s["case"]
    w = _grouped(s["W"].float(), c["G"])                  # the zeros behind a short last group change no extremum
    if c["zp"]:
        lo, hi = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
        top = hi - lo
        scale = (top / torch.full_like(top, 15.0)).to(_dtype(c["s"]))      # (by a number, torch multiplies with 1 / 15)
    else:
        top = w.abs().amax(2)
        scale = (top / torch.full_like(top, 7.0)).to(_dtype(c["s"]))
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    f = scale.float()
    if c["zp"]:
        z = -8.0 - torch.round(lo / f)
        codes = (torch.round(w / f[:, :, None]) + z[:, :, None]).clamp(-8, 7)
        back = (codes - z[:, :, None]) * f[:, :, None]
    else:
        back = torch.round(w / f[:, :, None]).clamp(-7, 7) * f[:, :, None]
    back = back.view(c["N"], -1)[:, :c["K"]].to(_dtype(c["out"]))
    out = [back, scale.t()]
    return out + [z.t().to(torch.int8)] if c["zp"] else out


def _norm32(x, kind, eps=1e-6):
    if kind == "rms":
        return x * torch.rsqrt((x * x).mean(1, keepdim=True) + eps)
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
        return x * torch.rsqrt((x * x).mean(1, keepdim=True) + eps)
    return x


def _plain_norm(s):
    c = s["case"]
    M, T = c["M"], c["T"]
    per_row = lambda v: v.float().repeat_interleave(T, 0)[:M]     # one vector per sample -> one per row
    h = s["R"].float()
    if s["Y"] is not None:
        u = _norm32(s["Y"].float(), c["post"])
        if s["post_w"] is not None:
            u = u * s["post_w"].float()
        if s["post_b"] is not None:
            u = u + s["post_b"].float()
        if s["gate"] is not None:
            u = u * per_row(s["gate"])
        h = h + c["alpha"] * u
    o = _norm32(h, c["pre"])
    if s["w"] is not None:
        o = o * s["w"].float()
    if s["b"] is not None:
        o = o + s["b"].float()
    if s["scale"] is not None:
        o = o * (1.0 + per_row(s["scale"])) + per_row(s["shift"])
    out = [h.to(s["R"].dtype)] if s["Y"] is not None else []
    if c["kind"] == "norm":
        return out + [o.to(s["R"].dtype)]
    widths = torch.tensor([b - a for a, b in zip(s["kb"], s["kb"][1:])], device="cuda")
    step = s["s_pos"].repeat_interleave(widths)
    if not c["dual"]:
        return out + [(o / step).clamp(-448, 448).to(_E4M3)]
    step_neg = s["s_neg"].repeat_interleave(widths)
    return out + [(o.clamp(min=0) / step).clamp(max=448).to(_E4M3), (o.clamp(max=0) / step_neg).clamp(min=-448).to(_E4M3)]


# ------------------------------------------------------------------------------------------------ the package's calls

def _own(s):
    from paper_2507_14811_b200 import binding as B

    c = s["case"]
    if c["kind"] == "matvec":
        return B.segquant_w4_matvec(s["X"], s["W4"], s["s_w"], c["G"], s["z_w"], s["bias"], act=c["act"], y_dtype=_dtype(c["y"]))
    if c["kind"] == "pack":
        W4, s_w, z_w = B.segquant_quantize_w4_group(s["W"], c["G"], s_dtype=_dtype(c["s"]), zero_points=c["zp"])
        back = B.segquant_dequantize_w4_group(W4, s_w, c["G"], c["K"], z_w, dtype=_dtype(c["out"]))
        return [back, s_w, z_w] if c["zp"] else [back, s_w]
    args = dict(Y=s["Y"], gate=s["gate"], alpha=c["alpha"], post=c["post"], post_w=s["post_w"], post_b=s["post_b"], norm=c["pre"],
                w=s["w"], b=s["b"], scale=s["scale"], shift=s["shift"], rows_per_sample=c["T"], eps=1e-6)
    if c["kind"] == "norm":
        H, O = B.segquant_block_norm(s["R"], **args)
        return [H, O] if s["Y"] is not None else [O]
    if "seg" not in s:                                    # the layer's segment table, kept with its scales
        s["seg"] = B.SegTable(s["kb"], [0, 8])
    H, c_pos, c_neg = B.segquant_block_norm_quantize(s["R"], s["seg"], s["s_pos"], s["s_neg"], "e4m3", **args)
    codes = [c_pos.view(_E4M3)] + ([c_neg.view(_E4M3)] if c["dual"] else [])
    return ([H] if s["Y"] is not None else []) + codes


def run(state):
    if own:
        return _own(state)
    return {"matvec": _plain_matvec, "pack": _plain_pack}.get(state["case"]["kind"], _plain_norm)(state)


# ------------------------------------------------------------------------------------------------ what is asked of a pass

def work(case):
    c = case
    size = {"f32": 4, "bf16": 2}
    if c["kind"] in ("matvec", "pack"):
        N, K = c["N"], c["K"]
        packed = N * ((K + 1) // 2) + N * -(-K // c["G"]) * (size[c["s"]] + (1 if c["zp"] else 0))
        if c["kind"] == "pack":                           # quantized, then read back
            return {"bytes": N * K * size[c["x"]] + 2 * packed + N * K * size[c["out"]], "flops": 4 * N * K}
        M = c["M"]
        return {"bytes": packed + M * K * size[c["x"]] + M * N * size[c["y"]] + 4 * N, "flops": 2 * M * N * K}
    M, C, ps = c["M"], c["C"], size[c["p"]]
    vectors = (2 + c["res"]) * C * -(-M // c["T"]) * ps if c["mod"] else 0
    vectors += C * ps * (c["affine"] * (2 if c["pre"] == "layer" else 1))
    vectors += C * ps * {"none": 0, "rms": 1, "layer": 2}[c["post"]]
    rows = size[c["x"]] * (3 if c["res"] else 1) + (size[c["x"]] if c["kind"] == "norm" else 2 if c["dual"] else 1)
    return {"bytes": M * C * rows + vectors, "flops": 12 * M * C}


# ------------------------------------------------------------------------------------------------ 64-bit results

def _exact_matvec(c, s):
    K, N, G = c["K"], c["N"], c["G"]
    x = s["X"].double()
    if c["act"] == "silu":
        x = x / (1.0 + torch.exp(-x))
    elif c["act"] == "gelu":
        x = 0.5 * x * (1.0 + torch.special.erf(x / math.sqrt(2.0)))
    y = s["bias"].double().expand(c["M"], N).clone()
    for g in range(-(-K // G)):
        k0, k1 = g * G, min(K, g * G + G)
        byte = s["W4"][:, k0 // 2:(k1 + 1) // 2].to(torch.int64)       # groups start at even inputs
        nib = torch.empty((N, 2 * byte.shape[1]), dtype=torch.float64, device="cuda")
        nib[:, 0::2], nib[:, 1::2] = byte % 16, byte // 16
        code = torch.where(nib >= 8, nib - 16, nib)[:, :k1 - k0]
        if c["zp"]:
            code = code - s["z_w"][g].double()[:, None]
        y += (x[:, k0:k1] @ code.t()) * s["s_w"][g].double()
    return y


def _exact_pack(c, s):
    W, G, K = s["W"].double(), c["G"], c["K"]
    f32 = lambda t: t.float().double()                    # a rounding that belongs to the definition
    stored = lambda t: f32(t).to(_dtype(c["s"])).double()
    back, scales, zeros = [], [], []
    for k0 in range(0, K, G):
        w = W[:, k0:k0 + G]
        if c["zp"]:
            lo, hi = w.min(1).values.clamp(max=0), w.max(1).values.clamp(min=0)
            sc = stored(f32(hi - lo) / 15.0)
        else:
            sc = stored(w.abs().max(1).values / 7.0)
        sc = torch.where(sc == 0, 1.0, sc)
        q = f32(w / sc[:, None]).round()
        if c["zp"]:
            z = -8.0 - f32(lo / sc).round()
            q = (q + z[:, None]).clamp(-8, 7) - z[:, None]
            zeros.append(z.to(torch.int8))
        else:
            q = q.clamp(-7, 7)
        back.append(q * sc[:, None])
        scales.append(sc)
    out = [torch.cat(back, 1), torch.stack(scales)]
    return out + [torch.stack(zeros)] if c["zp"] else out


def _exact_norm(c, s):
    d = {k: v.double() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
    sample = torch.arange(c["M"], device="cuda") // c["T"]

    def normed(x, kind, w, b):
        if kind != "none":
            mean = x.mean(1, keepdim=True) if kind == "layer" else 0.0
            x = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + 1e-6)
        x = x if w is None else x * w
        return x if b is None else x + b

    h = d["R"]
    out = []
    if d["Y"] is not None:
        u = normed(d["Y"], c["post"], d["post_w"], d["post_b"])
        h = h + c["alpha"] * (u if d["gate"] is None else u * d["gate"][sample])
        out.append(h)
    o = normed(h, c["pre"], d["w"], d["b"])
    if d["scale"] is not None:
        o = o * (1.0 + d["scale"][sample]) + d["shift"][sample]
    if c["kind"] == "norm":
        return out + [o]
    segment = torch.bucketize(torch.arange(c["C"], device="cuda"), torch.tensor(s["kb"][1:], device="cuda"), right=True)
    if not c["dual"]:                                     # quotients in front of the rounding to e4m3
        return out + [(o / d["s_pos"][segment]).clamp(-448, 448)]
    return out + [(o / d["s_pos"][segment]).clamp(0, 448), (o / d["s_neg"][segment]).clamp(-448, 0)]


def exact(case, seed):
    s = _inputs(case, seed)
    return {"matvec": _exact_matvec, "pack": _exact_pack}.get(case["kind"], _exact_norm)(case, s)
