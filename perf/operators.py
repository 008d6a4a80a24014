"""Performance cases of the operators around the linear layers, through ``paper_2509_25149_b200.binding``.

``norm``      h = x + residual, y = h / sqrt(mean(h^2) + eps) * gain, with the copies in 8 bits that the backward pass is to
              read; outputs y, h, 1 / sqrt(..) and the values of the copies;
``norm_bwd``  its gradient, from h as it was kept (bf16, binary32 or the copy in 8 bits);
``product``   act(A B^T + bias) + residual in one product, keeping z = A B^T + bias in bf16 or 8 bits where asked;
``act_bwd``   the gradient through the activation from the kept z, the bias gradient, and act(z) made again;
``copy``      an activation checkpoint: the copy in 8 bits (E4M3, a power-of-two scale per 32 elements) and its values in bf16;
``copy_bwd``  both gradients of a BF16 layer whose input was kept in 8 bits.

``run`` computes the plain form in elementary torch operations where ``own`` is false, else it calls the library.
"""
import math

import torch

own = False

EPS = 1e-5
ACTS = ("none", "relu2", "silu", "gelu")


def listed():
    return [
        # a token's norm in generation: launches and latency
        _norm("norm_one_token", 1, 5120, residual="bf16", copies=""),
        # the norm in front of a wide layer in training, whose input is kept in 8 bits for the weight gradient
        _norm("norm_training", 8192, 5120, residual="bf16", copies="y"),
        # its gradient, with the normalised sum kept in 8 bits; the residual path's gradient joins in
        _norm_bwd("norm_bwd_from_8_bits", 8192, 5120, kept="8", grad="bf16", accumulate=True),
        # odd sizes and a binary32 residual path
        _norm_bwd("norm_bwd_odd", 1003, 2056, kept="fp32", grad="fp32", accumulate=False),
        # one token through an output projection: the weight's bytes and latency
        _product("product_one_token", 1, 5120, 5120, act="none", residual=True, keep=""),
        # the up-projection of a training step: squared ReLU, what its gradient needs kept in 8 bits
        _product("product_ffn_up", 8192, 20480, 5120, act="relu2", residual=False, keep="8"),
        # a ragged batch through a ragged layer
        _product("product_ragged", 4088, 5128, 5112, act="gelu", residual=True, keep=""),
        # the gradient in front of the up-projection's two products, and the down-projection's input made again
        _act_bwd("act_bwd_ffn", 8192, 20480, act="relu2", kept="8", again=True, accumulate=False),
        # a small odd batch, bias gradient accumulated over microbatches
        _act_bwd("act_bwd_odd", 1003, 2056, act="gelu", kept="bf16", again=False, accumulate=True),
        # a checkpoint of a wide activation and its values for the backward pass
        _copy("copy_ffn", 8192, 20480, fp32=False),
        # few ragged rows of a binary32 stream
        _copy("copy_ragged", 333, 1048, fp32=True),
        # the gradients of a ragged BF16 layer from its checkpoint
        _copy_bwd("copy_bwd_ragged", 4088, 5128, 5112, accumulate=False),
    ]


def _named(name, case):
    return dict(case, name=name) if name else case


def _norm(name, rows, cols, residual, copies):
    return _named(name, {"kind": "norm", "rows": rows, "cols": cols, "residual": residual, "copies": copies})


def _norm_bwd(name, rows, cols, kept, grad, accumulate):
    return _named(name, {"kind": "norm_bwd", "rows": rows, "cols": cols, "kept": kept, "grad": grad, "accumulate": accumulate})


def _product(name, m, n, k, act, residual, keep):
    return _named(name, {"kind": "product", "m": m, "n": n, "k": k, "act": act, "residual": residual, "keep": keep})


def _act_bwd(name, rows, cols, act, kept, again, accumulate):
    return _named(name, {"kind": "act_bwd", "rows": rows, "cols": cols, "act": act, "kept": kept, "again": again,
                         "accumulate": accumulate})


def _copy(name, rows, cols, fp32):
    return _named(name, {"kind": "copy", "rows": rows, "cols": cols, "fp32": fp32})


def _copy_bwd(name, tokens, out, inp, accumulate):
    return _named(name, {"kind": "copy_bwd", "tokens": tokens, "out": out, "inp": inp, "accumulate": accumulate})


def _log(rng, lo, hi, unit=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / unit)) * unit))


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 1.3e15


def draw(rng):
    """One more case of the ranges above; no dearer than the dearest listed one."""
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw_one(rng)
        if _cost(case) <= most:
            return case


def _draw_one(rng):
    kind = rng.choices(["norm", "norm_bwd", "product", "act_bwd", "copy", "copy_bwd"], [3, 3, 4, 3, 2, 2])[0]
    rows, cols = _log(rng, 1, 16384), _log(rng, 64, 20480, 8)
    if kind == "norm":
        return _norm(None, rows, cols, rng.choice(["", "bf16", "bf16", "fp32"]), rng.choice(["", "y", "h", "yh"]))
    if kind == "norm_bwd":
        return _norm_bwd(None, rows, cols, rng.choice(["bf16", "fp32", "8"]), rng.choice(["bf16", "fp32", ""]), rng.random() < 0.5)
    if kind == "product":
        return _product(None, rows, _log(rng, 128, 20480, 8), _log(rng, 128, 20480, 8), rng.choice(ACTS), rng.random() < 0.5,
                        rng.choice(["", "", "bf16", "8"]))
    if kind == "act_bwd":
        return _act_bwd(None, rows, cols, rng.choice(ACTS), rng.choice(["bf16", "8"]), rng.random() < 0.5, rng.random() < 0.5)
    if kind == "copy":
        return _copy(None, rows, cols, rng.random() < 0.3)
    return _copy_bwd(None, _log(rng, 8, 16384, 8), _log(rng, 128, 20480, 8), _log(rng, 128, 20480, 8), rng.random() < 0.25)


# ------------------------------------------------------------------------------------------------- inputs ----
def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


def _activation(g, shape, dtype=torch.bfloat16):
    """Normal values of which one in a thousand is a hundred times as large."""
    x = torch.randn(shape, generator=g, device="cuda")
    far = torch.rand(shape, generator=g, device="cuda") < 0.001
    return torch.where(far, x * 100.0, x).to(dtype)


def _gain(g, cols):
    return 1.0 + 0.1 * torch.randn(cols, generator=g, device="cuda")


def _empty(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind in ("norm", "norm_bwd", "act_bwd", "copy"):
        shape = (case["rows"], case["cols"])
    if kind == "norm":
        s["x"] = _activation(g, shape)
        s["gain"] = _gain(g, shape[1])
        s["y"], s["rstd"] = _empty(*shape), _empty(shape[0], dtype=torch.float32)
        if case["residual"]:
            dtype = torch.float32 if case["residual"] == "fp32" else torch.bfloat16
            s["residual"] = _normal(g, shape, 2.0, dtype)
            s["h"] = _empty(*shape, dtype=dtype)
    elif kind == "norm_bwd":
        s["dy"] = _normal(g, shape, 1e-4)
        h = _activation(g, shape, torch.float32 if case["kept"] == "fp32" else torch.bfloat16)
        s["rstd"] = torch.rsqrt(h.double().square().mean(1) + EPS).float()
        if case["kept"] == "8":
            s["h_codes"], s["h_scales"] = _to_8(h.float())
        else:
            s["h"] = h
        s["gain"] = _gain(g, shape[1])
        dtype = torch.float32 if case["grad"] == "fp32" else torch.bfloat16
        if case["grad"]:
            s["residual_grad"] = _normal(g, shape, 1e-4, dtype)
        s["dh"] = _empty(*shape, dtype=dtype)
        s["dgain0"] = _normal(g, shape[1], 1e-2, torch.float32)
    elif kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"], s["b"] = _normal(g, (m, k)), _normal(g, (n, k), 0.02)
        s["bias"] = _normal(g, n, 0.5, torch.float32)
        if case["residual"]:
            s["residual"] = _normal(g, (m, n), 2.0)
        s["d"] = _empty(m, n)
        if case["keep"] == "bf16":
            s["z"] = _empty(m, n)
    elif kind == "act_bwd":
        s["da"] = _normal(g, shape, 1e-4)
        z = _normal(g, shape, 1.5)
        if case["kept"] == "8":
            s["z_codes"], s["z_scales"] = _to_8(z.float())
        else:
            s["z"] = z
        s["dz"] = _empty(*shape)
        if case["again"]:
            s["a"] = _empty(*shape)
        s["dbias0"] = _normal(g, shape[1], 1e-2, torch.float32)
    elif kind == "copy":
        s["x"] = _activation(g, shape, torch.float32 if case["fp32"] else torch.bfloat16)
        s["values"] = _empty(*shape)
    else:
        t, n, k = case["tokens"], case["out"], case["inp"]
        s["dy"], s["w"] = _normal(g, (t, n), 1e-4), _normal(g, (n, k), 0.02)
        s["x_codes"], s["x_scales"] = _to_8(_activation(g, (t, k)).float())
        s["dx"] = _empty(t, k)
        s["dw0"] = _normal(g, (n, k), 1e-3, torch.float32)
    return s


# ------------------------------------------------------------------------------------------- the plain form ----
def _to_8(x):
    """Codes and scale bytes of the copy in 8 bits of binary32 values [rows x cols]."""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    blocks = torch.nn.functional.pad(x, (0, 32 * nb - cols)).view(rows, nb, 32)
    m, e = torch.frexp(blocks.abs().amax(2))  # amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    byte = torch.where(m <= 0.875, e - 9, e - 8).add_(127).clamp_(0, 254)
    byte = torch.where(m == 0, torch.zeros_like(byte), byte)
    up = ((254 - byte) << 23).view(torch.float32)
    codes = (blocks * up[:, :, None]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8).view(rows, 32 * nb)[:, :cols].contiguous(), byte.to(torch.uint8)


def _from_8(codes, scales):
    """Their values in binary32."""
    s = scales.to(torch.int32)
    power = torch.where(s == 0, torch.full_like(s, 1 << 22), s << 23).view(torch.float32)
    return codes.view(torch.float8_e4m3fn).float() * power.repeat_interleave(32, 1)[:, :codes.shape[1]]


def _act(z, act):
    if act == "relu2":
        return z.clamp_min(0).square()
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_grad(z, act):
    if act == "relu2":
        return 2 * z.clamp_min(0)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        h = s["x"].float()
        if case["residual"]:
            h = h + s["residual"].float()
        rstd = torch.rsqrt(h.square().mean(1) + EPS)
        y = h * rstd[:, None] * s["gain"]
        out = {"y": y.bfloat16(), "rstd": rstd}
        if case["residual"]:
            out["h"] = h.to(s["h"].dtype)
        if "y" in case["copies"]:
            out["y8"] = _from_8(*_to_8(y)).bfloat16()
        if "h" in case["copies"]:
            out["h8"] = _from_8(*_to_8(h)).bfloat16()
        return out
    if kind == "norm_bwd":
        h = _from_8(s["h_codes"], s["h_scales"]) if case["kept"] == "8" else s["h"].float()
        xh = h * s["rstd"][:, None]
        dy = s["dy"].float()
        gy = dy * s["gain"]
        dh = s["rstd"][:, None] * (gy - xh * (gy * xh).mean(1, keepdim=True))
        if case["grad"]:
            dh = dh + s["residual_grad"].float()
        dgain = (dy * xh).sum(0)
        return {"dh": dh.to(s["dh"].dtype), "dgain": dgain + s["dgain0"] if case["accumulate"] else dgain}
    if kind == "product":
        z = s["a"].float() @ s["b"].float().t() + s["bias"]
        d = _act(z, case["act"])
        if case["residual"]:
            d = d + s["residual"].float()
        out = {"d": d.bfloat16()}
        if case["keep"]:
            out["z"] = (_from_8(*_to_8(z)) if case["keep"] == "8" else z).bfloat16()
        return out
    if kind == "act_bwd":
        z = _from_8(s["z_codes"], s["z_scales"]) if case["kept"] == "8" else s["z"].float()
        dz = s["da"].float() * _act_grad(z, case["act"])
        dbias = dz.sum(0)
        out = {"dz": dz.bfloat16(), "dbias": dbias + s["dbias0"] if case["accumulate"] else dbias}
        if case["again"]:
            out["a"] = _act(z, case["act"]).bfloat16()
        return out
    if kind == "copy":
        return {"values": _from_8(*_to_8(s["x"].float())).bfloat16()}
    dy, x = s["dy"].float(), _from_8(s["x_codes"], s["x_scales"])
    dw = dy.t() @ x
    return {"dx": (dy @ s["w"].float()).bfloat16(), "dw": dw + s["dw0"] if case["accumulate"] else dw}


# ------------------------------------------------------------------------------------------ the library's calls ----
def _kept_copy(B, s, name):
    """The copy in 8 bits that the program keeps, made of its codes and scale bytes."""
    if name not in s:
        codes, scales = s[name + "_codes"], s[name + "_scales"]
        s[name] = B.NVFP4Tensor(codes, scales, None, codes.shape[0], codes.shape[1], B.SF_LINEAR, B.FORMAT_MXFP8)
    return s[name]


def _new_copy(B, s, name, rows, cols):
    if name not in s:
        s[name] = B.alloc_tensor(rows, cols, B.SF_LINEAR, format=B.FORMAT_MXFP8)
        s[name + "_values"] = _empty(rows, cols)
    return s[name]


def _workspace(s, nbytes):
    """Scratch that the program keeps."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _started_with(s, name):
    """The buffer that a gradient is added into, as the microbatches before have left it."""
    if name not in s:
        s[name] = torch.empty_like(s[name + "0"])
    if s["case"]["accumulate"]:
        s[name].copy_(s[name + "0"])
    return s[name]


def _library(s):
    from paper_2509_25149_b200 import binding as B

    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        rows, cols = case["rows"], case["cols"]
        y8 = _new_copy(B, s, "y8", rows, cols) if "y" in case["copies"] else None
        h8 = _new_copy(B, s, "h8", rows, cols) if "h" in case["copies"] else None
        B.nvfp4_rmsnorm_fwd(s["x"], s["gain"], EPS, s["y"], s["rstd"], residual=s.get("residual"), h=s.get("h"), y8=y8, h8=h8)
        out = {"y": s["y"], "rstd": s["rstd"]}
        if case["residual"]:
            out["h"] = s["h"]
        for name, q in (("y8", y8), ("h8", h8)):
            if q is not None:
                out[name] = B.nvfp4_dequantize_bf16(q, s[name + "_values"])
        return out
    if kind == "norm_bwd":
        h = _kept_copy(B, s, "h") if case["kept"] == "8" else s["h"]
        dgain = _started_with(s, "dgain")
        ws = _workspace(s, B.nvfp4_rmsnorm_bwd_workspace_bytes(case["rows"], case["cols"]))
        B.nvfp4_rmsnorm_bwd(s["dy"], h, s["gain"], s["rstd"], s["dh"], dgain, ws, residual_grad=s.get("residual_grad"),
                            accumulate_dgain=case["accumulate"])
        return {"dh": s["dh"], "dgain": dgain}
    if kind == "product":
        z = _new_copy(B, s, "z8", case["m"], case["n"]) if case["keep"] == "8" else s.get("z")
        B.nvfp4_gemm_bf16_epilogue(s["a"], s["b"], s["d"], bias=s["bias"], act=getattr(B, "ACT_" + case["act"].upper()),
                                   residual=s.get("residual"), z=z)
        out = {"d": s["d"]}
        if case["keep"]:
            out["z"] = B.nvfp4_dequantize_bf16(z, s["z8_values"]) if case["keep"] == "8" else z
        return out
    if kind == "act_bwd":
        z = _kept_copy(B, s, "z") if case["kept"] == "8" else s["z"]
        dbias = _started_with(s, "dbias")
        ws = _workspace(s, B.nvfp4_act_bwd_workspace_bytes(case["rows"], case["cols"]))
        B.nvfp4_act_bwd(s["da"], z, getattr(B, "ACT_" + case["act"].upper()), s["dz"], a=s.get("a"), dbias=dbias,
                        accumulate_dbias=case["accumulate"], workspace=ws)
        out = {"dz": s["dz"], "dbias": dbias}
        if case["again"]:
            out["a"] = s["a"]
        return out
    if kind == "copy":
        q = _new_copy(B, s, "x8", case["rows"], case["cols"])
        if "opts" not in s:
            s["opts"] = B.quant_opts()
        B.nvfp4_quantize(s["x"], s["opts"], q)
        return {"values": B.nvfp4_dequantize_bf16(q, s["values"])}
    x8 = _kept_copy(B, s, "x")
    dw = _started_with(s, "dw")
    ws = _workspace(s, B.nvfp4_linear_bf16_bwd8_workspace_bytes(case["tokens"], case["inp"]))
    B.nvfp4_linear_bf16_bwd8(s["dy"], x8, s["w"], s["dx"], dw, ws, accumulate_dw=case["accumulate"])
    return {"dx": s["dx"], "dw": dw}


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    kind = case["kind"]
    if kind in ("product", "copy_bwd"):
        m, n, k = (case["m"], case["n"], case["k"]) if kind == "product" else (case["tokens"], case["out"], case["inp"])
        if kind == "product":
            kept = {"": 0, "bf16": 2, "8": 2}[case["keep"]]
            return {"bytes": 2.0 * (m * k + n * k) + m * n * (2.0 + 2.0 * case["residual"] + kept) + 4.0 * n, "flops": 2.0 * m * n * k}
        return {"bytes": 2.0 * (m * n + n * k + m * k) + m * k * 33 / 32 + n * k * (8.0 if case["accumulate"] else 4.0),
                "flops": 4.0 * m * n * k}
    size = float(case["rows"] * case["cols"])
    wide = {"": 0, "bf16": 2, "fp32": 4, "8": 33 / 32}
    if kind == "norm":
        return {"bytes": size * (4 + 2 * wide[case["residual"]] + 2 * len(case["copies"])) + 4.0 * (case["rows"] + case["cols"]),
                "flops": 8.0 * size}
    if kind == "norm_bwd":
        grad = 2 * wide[case["grad"]] or 2
        return {"bytes": size * (2 + wide[case["kept"]] + grad) + 4.0 * (case["rows"] + 2 * case["cols"]), "flops": 12.0 * size}
    if kind == "act_bwd":
        return {"bytes": size * (4 + wide[case["kept"]] + 2 * case["again"]) + 4.0 * case["cols"], "flops": 10.0 * size}
    return {"bytes": size * ((4 if case["fp32"] else 2) + 2), "flops": 4.0 * size}


# ------------------------------------------------------------------------------------------------ in 64 bits ----
def _values_of_copy(x):
    """What the copy in 8 bits of these values stands for, from the format's definition."""
    rows, cols = x.shape
    out = torch.empty_like(x)
    full = cols // 32 * 32
    for part, width in ((slice(0, full), 32), (slice(full, cols), cols - full)):
        if width == 0 or part.start == part.stop:
            continue
        b = x[:, part].reshape(rows, -1, width)
        top = b.abs().amax(2, keepdim=True)
        scale = torch.exp2(torch.ceil(torch.log2(top.clamp_min(1e-300) / 448.0)).clamp_min(-127.0))
        scale = torch.where(top > 448.0 * scale, 2 * scale, scale)  # (a logarithm next to a whole number)
        scale = torch.where((top <= 224.0 * scale) & (scale > 2.0 ** -127), scale / 2, scale)
        v = b / scale
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))).clamp_min(-6.0) - 3.0)
        out[:, part] = (torch.round(v / step) * step * scale).reshape(rows, -1)
    return out


def _decoded(codes, scales):
    c = codes.to(torch.int64)
    mantissa, exponent = (c & 7).double(), ((c >> 3) & 15).double()
    v = torch.where(exponent == 0, mantissa / 8 * 2.0 ** -6, (1 + mantissa / 8) * torch.exp2(exponent - 7))
    v = torch.where(c >= 128, -v, v)
    return v * torch.exp2(scales.double() - 127.0).repeat_interleave(32, 1)[:, :codes.shape[1]]


def _gate(z):
    """The logistic factor of the tanh form of GELU, and the derivative of its argument."""
    c = 2 * math.sqrt(2 / math.pi)
    return torch.sigmoid(c * z * (1 + 0.044715 * z.square())), c * (1 + 0.134145 * z.square())


def _act64(z, act):
    return {"none": lambda: z, "relu2": lambda: torch.where(z > 0, z * z, torch.zeros_like(z)),
            "silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * _gate(z)[0]}[act]()


def _slope64(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu2":
        return torch.where(z > 0, 2 * z, torch.zeros_like(z))
    s, slope = (torch.sigmoid(z), 1.0) if act == "silu" else _gate(z)
    return s + z * s * (1 - s) * slope


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        h = s["x"].double()
        if case["residual"]:
            h = (h + s["residual"].double()).float().double()  # (the sum is a binary32 number by definition)
        rstd = 1 / torch.sqrt((h * h).sum(1) / case["cols"] + EPS)
        y = h * rstd.unsqueeze(1) * s["gain"].double()
        out = {"y": y, "rstd": rstd}
        if case["residual"]:
            out["h"] = h
        if "y" in case["copies"]:
            out["y8"] = _values_of_copy(y)
        if "h" in case["copies"]:
            out["h8"] = _values_of_copy(h)
        return out
    if kind == "norm_bwd":
        h = _decoded(s["h_codes"], s["h_scales"]) if case["kept"] == "8" else s["h"].double()
        r = s["rstd"].double().unsqueeze(1)
        dy, n = s["dy"].double(), h * r
        gy = dy * s["gain"].double()
        dh = r * gy - r * n * ((gy * n).sum(1, keepdim=True) / case["cols"])
        if case["grad"]:
            dh += s["residual_grad"].double()
        dgain = (dy * n).sum(0)
        return {"dh": dh, "dgain": dgain + s["dgain0"].double() if case["accumulate"] else dgain}
    if kind == "product":
        z = torch.addmm(s["bias"].double(), s["a"].double(), s["b"].double().t())
        d = _act64(z, case["act"])
        if case["residual"]:
            d = d + s["residual"].double()
        out = {"d": d}
        if case["keep"]:
            out["z"] = _values_of_copy(z) if case["keep"] == "8" else z
        return out
    if kind == "act_bwd":
        z = _decoded(s["z_codes"], s["z_scales"]) if case["kept"] == "8" else s["z"].double()
        dz = s["da"].double() * _slope64(z, case["act"])
        dbias = dz.sum(0)
        out = {"dz": dz, "dbias": dbias + s["dbias0"].double() if case["accumulate"] else dbias}
        if case["again"]:
            out["a"] = _act64(z, case["act"])
        return out
    if kind == "copy":
        return {"values": _values_of_copy(s["x"].double())}
    dy = s["dy"].double()
    dw = dy.t() @ _decoded(s["x_codes"], s["x_scales"])
    return {"dx": dy @ s["w"].double(), "dw": dw + s["dw0"].double() if case["accumulate"] else dw}
