"""Performance cases of the operators at the ends of a training step, through ``paper_2509_25149_b200.binding``.

``heads``      the query and key heads of a QKV product: each head's root-mean-square norm, its gain, and the rotation by position;
``heads_bwd``  the gradient of that, with the gains' gradients;
``embed``      rows of the embedding table for given tokens, times a scale; a token outside of the table (padding) gives zeros;
``embed_bwd``  the table's gradient: the scaled sum of the gradient's rows for every token;
``logprob``    log probabilities of given tokens, the logarithm of the sum, the entropy and the likeliest alternatives (ties go to the
               lowest index); with ``train`` also the gradient of a weighted sum of log probabilities and entropies;
``clip``       the norm over the gradients of many tensors, and the gradients scaled to a largest norm.

``run`` computes the plain form in elementary torch operations where ``own`` is false, else it calls the library.
"""
import math

import torch

own = False

EPS = 1e-5


def listed():
    return [
        # queries and keys of a training step: 40 query and 8 key heads inside a QKV product, documents packed behind one another
        _heads("heads_training", 8192, 40, 8, 128, rotary=128, interleaved=False, far=False),
        # one token in generation, far into its text: launches and latency
        _heads("heads_one_token", 1, 40, 8, 128, rotary=128, interleaved=False, far=True),
        # their gradient in a training step
        _heads_bwd("heads_bwd_training", 8192, 40, 8, 128, rotary=128, interleaved=False, accumulate=False),
        # heads of an odd width of which only a part is rotated, neighbouring elements together; gains accumulated over microbatches
        _heads_bwd("heads_bwd_odd", 1003, 12, 4, 80, rotary=32, interleaved=True, accumulate=True),
        # the start of a forward pass over two sequences
        _embed("embed_training", 16384, 131072, 5120, fp32=False, scaled=False),
        # the end of its backward pass: the table's whole gradient, zeros included
        _embed_bwd("embed_bwd_training", 16384, 131072, 5120, fp32=False, accumulate=False, scaled=False),
        # a small odd batch with padding, added to what a tied output layer has put there
        _embed_bwd("embed_bwd_odd", 1003, 5003, 2056, fp32=True, accumulate=True, scaled=True),
        # the loss of a training step with its gradient, the entropy for the record
        _logprob("logprob_training", 8192, 131072, fp32=False, top=0, entropy=True, train=True, mask=False, scaled=False),
        # a sampled token with twenty alternatives, a part of the vocabulary ruled out
        _logprob("logprob_one_token", 1, 131072, fp32=False, top=20, entropy=True, train=False, mask=True, scaled=True),
        # a ragged batch with padding over an odd vocabulary in binary32, the entropy's gradient too
        _logprob("logprob_odd", 1003, 50257, fp32=True, top=0, entropy=True, train=True, mask=False, scaled=True),
        # binary32 gradients of several blocks, the clipped ones in bf16
        _clip("clip_blocks", 24, 104857600, kinds="fp32", out_fp32=False, odd=False, clipped=True),
        # many small tensors of odd sizes in both types, one behind the other
        _clip("clip_small", 60, 20011, kinds="mixed", out_fp32=True, odd=True, clipped=True),
    ]


def _named(name, case):
    return dict(case, name=name) if name else case


def _heads(name, rows, q, k, dim, rotary, interleaved, far):
    return _named(name, {"kind": "heads", "rows": rows, "q": q, "k": k, "dim": dim, "rotary": rotary, "interleaved": interleaved, "far": far})


def _heads_bwd(name, rows, q, k, dim, rotary, interleaved, accumulate):
    return _named(name, {"kind": "heads_bwd", "rows": rows, "q": q, "k": k, "dim": dim, "rotary": rotary, "interleaved": interleaved,
                         "far": False, "accumulate": accumulate})


def _embed(name, tokens, vocab, cols, fp32, scaled):
    return _named(name, {"kind": "embed", "tokens": tokens, "vocab": vocab, "cols": cols, "fp32": fp32, "scaled": scaled})


def _embed_bwd(name, tokens, vocab, cols, fp32, accumulate, scaled):
    return _named(name, {"kind": "embed_bwd", "tokens": tokens, "vocab": vocab, "cols": cols, "fp32": fp32, "accumulate": accumulate,
                         "scaled": scaled})


def _logprob(name, rows, vocab, fp32, top, entropy, train, mask, scaled):
    return _named(name, {"kind": "logprob", "rows": rows, "vocab": vocab, "fp32": fp32, "top": top, "entropy": entropy, "train": train,
                         "mask": mask, "scaled": scaled})


def _clip(name, tensors, largest, kinds, out_fp32, odd, clipped):
    return _named(name, {"kind": "clip", "tensors": tensors, "largest": largest, "kinds": kinds, "out_fp32": out_fp32, "odd": odd,
                         "clipped": clipped})


def _log(rng, lo, hi, unit=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / unit)) * unit))


def _cost(case):
    """Seconds at 5 TB/s, in which what the plain form passes over again counts."""
    again = {"embed_bwd": 1.5, "logprob": 4.0, "clip": 1.5}.get(case["kind"], 1.0)
    return work(case)["bytes"] * again / 5e12 + (case["rows"] * case["vocab"] * 1e-10 if case.get("top") else 0.0)


def draw(rng):
    """One more case of the ranges above; no dearer than the dearest listed one."""
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw_one(rng)
        if _cost(case) <= most:
            return case


def _draw_one(rng):
    kind = rng.choices(["heads", "heads_bwd", "embed", "embed_bwd", "logprob", "clip"], [3, 3, 2, 3, 4, 2])[0]
    rows = _log(rng, 1, 16384)
    if kind.startswith("heads"):
        dim, k = rng.choice([64, 80, 96, 128, 192, 256]), rng.randint(1, 8)
        q = k * rng.randint(1, 8)
        rotary = rng.choice([dim, dim, dim // 2 // 16 * 16, 0])
        if kind == "heads":
            return _heads(None, rows, q, k, dim, rotary, rng.random() < 0.4, rng.random() < 0.3)
        return _heads_bwd(None, rows, q, k, dim, rotary, rng.random() < 0.4, rng.random() < 0.4)
    if kind == "embed":
        return _embed(None, rows, _log(rng, 100, 131072), _log(rng, 64, 8192, 8), rng.random() < 0.4, rng.random() < 0.5)
    if kind == "embed_bwd":
        return _embed_bwd(None, rows, _log(rng, 100, 131072), _log(rng, 64, 8192, 8), rng.random() < 0.4, rng.random() < 0.5,
                          rng.random() < 0.5)
    if kind == "logprob":
        train = rng.random() < 0.5
        return _logprob(None, rows, _log(rng, 100, 160000), rng.random() < 0.4, 0 if train else rng.choice([0, 1, 5, 20, 32]),
                        rng.random() < 0.6, train, rng.random() < 0.3, rng.random() < 0.5)
    return _clip(None, _log(rng, 1, 400), _log(rng, 100, 50000000), rng.choice(["fp32", "bf16", "mixed"]), rng.random() < 0.6,
                 rng.random() < 0.4, rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------- inputs ----
def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


def _empty(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _tokens(g, n, vocab, padding):
    """Tokens of which the k-th comes about 1 / k as often as the first, every hundredth one padding where asked."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    t = (torch.exp(u * math.log(vocab + 1.0)).long() - 1).clamp_(0, vocab - 1)
    t = (t * 7919) % vocab if math.gcd(7919, vocab) == 1 else t  # (frequent tokens are not neighbours)
    return torch.where(torch.rand(n, generator=g, device="cuda") < 0.01, -1, t) if padding else t


def _grad_sizes(case):
    """Numbers of elements: matrices of the largest size and some way below it, and vectors between them."""
    sizes = [max(1, case["largest"] >> i % 3) if i % 4 < 2 else 1 + (i * 1237) % min(case["largest"], 20480) for i in range(case["tensors"])]
    return sizes if case["odd"] else [(n + 63) // 64 * 64 for n in sizes]


def _grad_kinds(case):
    return [case["kinds"] == "fp32" or (case["kinds"] == "mixed" and i % 3 != 1) for i in range(case["tensors"])]


def _views(flat, sizes):
    return list(torch.split(flat, sizes))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind in ("heads", "heads_bwd"):
        rows, q, k, dim = (case[n] for n in ("rows", "q", "k", "dim"))
        s["qkv"] = _normal(g, (rows, (q + 2 * k) * dim), 1.5)  # (the values' heads stand behind the keys')
        s["x"] = s["qkv"][:, :(q + k) * dim]
        s["gain_q"], s["gain_k"] = (1 + 0.1 * torch.randn(dim, generator=g, device="cuda") for _ in range(2))
        s["inv_freq"] = None
        if case["rotary"]:
            i = torch.arange(case["rotary"] // 2, device="cuda", dtype=torch.float64)
            s["inv_freq"] = torch.exp(-math.log(500000.0) * 2 * i / case["rotary"]).float()
        start = int(torch.randint(100000, 1000000, (1,), generator=g, device="cuda")) if case["far"] else 0
        s["positions"] = start + torch.arange(rows, device="cuda") % max(1, rows // 3)
        if kind == "heads":
            s["y"] = _empty(rows, (q + k) * dim)
        else:
            s["dy"] = _normal(g, (rows, (q + k) * dim), 1e-3)
            s["dqkv"] = _empty(rows, (q + 2 * k) * dim)
            s["dgain_q0"], s["dgain_k0"] = (_normal(g, dim, 1e-2, torch.float32) for _ in range(2))
    elif kind == "embed":
        s["table"] = _normal(g, (case["vocab"], case["cols"]), 0.02, torch.float32 if case["fp32"] else torch.bfloat16)
        s["tokens"] = _tokens(g, case["tokens"], case["vocab"], case["scaled"])
        s["out"] = _empty(case["tokens"], case["cols"])
    elif kind == "embed_bwd":
        s["tokens"] = _tokens(g, case["tokens"], case["vocab"], case["scaled"])
        s["dout"] = _normal(g, (case["tokens"], case["cols"]), 1e-3, torch.float32 if case["fp32"] else torch.bfloat16)
        if case["accumulate"]:
            s["dtable0"] = _normal(g, (case["vocab"], case["cols"]), 1e-3, torch.float32)
        s["dtable"] = _empty(case["vocab"], case["cols"], dtype=torch.float32)
    elif kind == "logprob":
        rows, vocab, dtype = case["rows"], case["vocab"], torch.float32 if case["fp32"] else torch.bfloat16
        wide = (vocab + 7) // 8 * 8  # (what the product in front of it has for columns)
        s["wide"] = _normal(g, (rows, wide), 3.0, dtype)
        if case["mask"]:
            s["wide"].masked_fill_(torch.rand(wide, generator=g, device="cuda") < 0.3, -math.inf)
            s["wide"][:, 0] = 1.0
        s["logits"] = s["wide"][:, :vocab]
        # tokens that a model likes: the largest of a few drawn ones
        some = torch.randint(0, vocab, (rows, 16), generator=g, device="cuda")
        s["targets"] = some.gather(1, s["logits"].gather(1, some).float().argmax(1, keepdim=True))[:, 0]
        if case["scaled"]:
            s["targets"] = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.05, -1, s["targets"])
            s["targets"][0] = 0
        if case["train"]:
            s["dlogprob"] = -torch.rand(rows, generator=g, device="cuda") / rows
            if case["entropy"]:
                s["dentropy"] = torch.full((rows,), -0.01 / rows, device="cuda")
            s["dlogits"] = _empty(rows, wide, dtype=dtype)
        for name in ("logprob", "lse", "entropy"):
            s[name] = _empty(rows, dtype=torch.float32)
        s["row_stats"] = _empty(rows, 2, dtype=torch.float32) if case["train"] else None
        if case["top"]:
            s["top_ids"] = _empty(rows, case["top"], dtype=torch.int32)
            s["top_logprobs"] = _empty(rows, case["top"], dtype=torch.float32)
    else:
        sizes, kinds = _grad_sizes(case), _grad_kinds(case)
        out_dtype = torch.float32 if case["out_fp32"] else torch.bfloat16
        by = {}
        for fp32 in (False, True):
            own_sizes = [n for n, f in zip(sizes, kinds) if f == fp32]
            dtype = torch.float32 if fp32 else torch.bfloat16
            by[fp32] = (iter(_views(_normal(g, sum(own_sizes), 1e-2, dtype), own_sizes)), None)
        s["grads"] = [next(by[f][0]) for f in kinds]
        s["out"] = _empty(sum(sizes), dtype=out_dtype)
        s["outs"] = _views(s["out"], sizes)
        s["sum"], s["stats"] = _empty(1, dtype=torch.float64), _empty(2, dtype=torch.float32)
    return s


SCALE = {"embed": 71.55418, "embed_bwd": 71.55418, "logprob": 1.25}  # of the cases that are scaled


def _scale(case):
    return SCALE[case["kind"]] if case["scaled"] else 1.0


def _max_norm(case):
    """Below or above the norm that the gradients have, 1e-2 times the root of their number."""
    return 1.0 if case["clipped"] and sum(_grad_sizes(case)) > 1e5 else 1e-2 if case["clipped"] else 1e4


# ------------------------------------------------------------------------------------------- the plain form ----
def _cos_sin(s):
    """Of position times inverse frequency, [rows x 1 x rotary / 2]: far positions need angles in 64 bits."""
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()
    return torch.cos(angle).float(), torch.sin(angle).float()


def _rotated(v, s, sign):
    case = s["case"]
    r = case["rotary"]
    if not r:
        return v
    c, n = _cos_sin(s)
    n = n * sign
    turned, rest = v[..., :r], v[..., r:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        return torch.cat([torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2), rest], -1)
    a, b = turned[..., :r // 2], turned[..., r // 2:]
    return torch.cat([a * c - b * n, b * c + a * n, rest], -1)


def _gains(s):
    case = s["case"]
    return torch.cat([s["gain_q"].expand(case["q"], -1), s["gain_k"].expand(case["k"], -1)])


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind in ("heads", "heads_bwd"):
        x = s["x"].float().unflatten(1, (case["q"] + case["k"], case["dim"]))
        rstd = torch.rsqrt(x.square().mean(2, keepdim=True) + EPS)
        n = x * rstd
        if kind == "heads":
            return {"y": _rotated(n * _gains(s), s, 1.0).flatten(1).bfloat16()}
        dy = _rotated(s["dy"].float().unflatten(1, x.shape[1:]), s, -1.0)
        gy = dy * _gains(s)
        dx = rstd * (gy - n * (gy * n).mean(2, keepdim=True))
        each = (dy * n).sum(0)
        out = {"dx": dx.flatten(1).bfloat16(), "dgain_q": each[:case["q"]].sum(0), "dgain_k": each[case["q"]:].sum(0)}
        if case["accumulate"]:
            out["dgain_q"] = out["dgain_q"] + s["dgain_q0"]
            out["dgain_k"] = out["dgain_k"] + s["dgain_k0"]
        return out
    if kind in ("embed", "embed_bwd"):
        there = (s["tokens"] >= 0) & (s["tokens"] < case["vocab"])
        at = torch.where(there, s["tokens"], 0)
        if kind == "embed":
            return {"out": torch.where(there[:, None], s["table"][at].float() * _scale(case), 0.0).bfloat16()}
        dtable = s["dtable0"].clone() if case["accumulate"] else torch.zeros_like(s["dtable"])
        rows = torch.where(there[:, None], s["dout"].float() * _scale(case), 0.0)
        return {"dtable": dtable.index_add_(0, at, rows)}
    if kind == "logprob":
        scale = _scale(case)
        x = s["logits"].float()
        m = x.amax(1, keepdim=True)
        d = (x - m) * scale
        e = torch.exp(d)
        total = e.sum(1, keepdim=True)
        log_total = torch.log(total)
        there = (s["targets"] >= 0) & (s["targets"] < case["vocab"])
        at = torch.where(there, s["targets"], 0)[:, None]
        out = {"lse": (m * scale + log_total)[:, 0]}
        out["logprob"] = torch.where(there, (d.gather(1, at) - log_total)[:, 0], 0.0)
        entropy = None
        if case["entropy"]:
            entropy = log_total - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total
            out["entropy"] = entropy[:, 0]
        if case["top"]:
            # whole numbers in the order of the logits, the lower index larger where they are equal
            bits = (x + 0.0).view(torch.int32).long()
            order = torch.where(bits >= 0, bits, -1 - (bits & 0x7FFFFFFF))
            keys = order * (1 << 31) + ((1 << 31) - 1 - torch.arange(case["vocab"], device="cuda"))
            ids = (1 << 31) - 1 - (torch.topk(keys, case["top"], 1).values & ((1 << 31) - 1))
            out["top_ids"] = ids.int()
            out["top_logprobs"] = d.gather(1, ids) - log_total
        if case["train"]:
            p = e.div_(total)
            weight = torch.where(there, s["dlogprob"], 0.0)[:, None]
            dz = p * -weight
            if case["entropy"]:
                dz -= s["dentropy"][:, None] * torch.where(p > 0, p * (d - log_total + entropy), 0.0)
            dz.scatter_add_(1, at, weight)
            out["dlogits"] = torch.nn.functional.pad(dz * scale, (0, s["dlogits"].shape[1] - case["vocab"])).to(s["dlogits"].dtype)
        return out
    norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
    most = _max_norm(case)
    factor = torch.where(norm > most, most / norm, 1.0).float()
    return {"stats": torch.stack([norm.float(), factor]), "out": torch.cat([(g.float() * factor).to(s["out"].dtype) for g in s["grads"]])}


# ------------------------------------------------------------------------------------------ the library's calls ----
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
    if kind == "heads":
        B.nvfp4_headnorm_fwd(s["x"], case["q"], case["k"], s["y"], gain_q=s["gain_q"], gain_k=s["gain_k"], eps=EPS, inv_freq=s["inv_freq"],
                             positions=s["positions"], interleaved=case["interleaved"])
        return {"y": s["y"]}
    if kind == "heads_bwd":
        dgain_q, dgain_k = _started_with(s, "dgain_q"), _started_with(s, "dgain_k")
        dx = s["dqkv"][:, :(case["q"] + case["k"]) * case["dim"]]
        ws = _workspace(s, B.nvfp4_headnorm_bwd_workspace_bytes(case["rows"], case["q"], case["k"], case["dim"]))
        B.nvfp4_headnorm_bwd(s["dy"], s["x"], case["q"], case["k"], dx, gain_q=s["gain_q"], gain_k=s["gain_k"], eps=EPS, dgain_q=dgain_q,
                             dgain_k=dgain_k, workspace=ws, inv_freq=s["inv_freq"], positions=s["positions"],
                             interleaved=case["interleaved"], accumulate_dgain=case["accumulate"])
        return {"dx": dx, "dgain_q": dgain_q, "dgain_k": dgain_k}
    if kind == "embed":
        B.nvfp4_embedding_fwd(s["tokens"], s["table"], s["out"], scale=_scale(case))
        return {"out": s["out"]}
    if kind == "embed_bwd":
        if case["accumulate"]:
            s["dtable"].copy_(s["dtable0"])
        ws = _workspace(s, B.nvfp4_embedding_bwd_workspace_bytes(case["tokens"], case["vocab"], case["cols"]))
        B.nvfp4_embedding_bwd(s["tokens"], s["dout"], s["dtable"], ws, scale=_scale(case), accumulate=case["accumulate"])
        return {"dtable": s["dtable"]}
    if kind == "logprob":
        entropy = s["entropy"] if case["entropy"] else None
        B.nvfp4_logprob_fwd(s["logits"], s["targets"], logprob=s["logprob"], lse=s["lse"], stats=s["row_stats"], entropy=entropy,
                            top_ids=s.get("top_ids"), top_logprobs=s.get("top_logprobs"), scale=_scale(case))
        out = {"lse": s["lse"], "logprob": s["logprob"]}
        if case["entropy"]:
            out["entropy"] = s["entropy"]
        if case["top"]:
            out["top_ids"], out["top_logprobs"] = s["top_ids"], s["top_logprobs"]
        if case["train"]:
            B.nvfp4_logprob_bwd(s["logits"], s["targets"], s["row_stats"], s["dlogits"], dlogprob=s["dlogprob"], entropy=entropy,
                                dentropy=s.get("dentropy"), scale=_scale(case))
            out["dlogits"] = s["dlogits"]
        return out
    if "list" not in s:
        s["list"] = B.grad_list(s["grads"], s["outs"])
    ws = _workspace(s, B.nvfp4_grad_sq_norm_workspace_bytes())
    B.nvfp4_grad_sq_norm(s["list"], s["sum"], ws)
    B.nvfp4_grad_clip(s["list"], s["sum"], _max_norm(case), s["stats"])
    return {"stats": s["stats"], "out": s["out"]}


def run(state):
    return _library(state) if own else _plain(state)


def _distinct(n, vocab):
    """How many different tokens n drawn ones are, about."""
    p = torch.log1p(1.0 / torch.arange(1, vocab + 1, dtype=torch.float64)) / math.log(vocab + 1.0)
    return float((1 - torch.exp(n * torch.log1p(-p.clamp_max(1 - 1e-12)))).sum())


def work(case):
    kind = case["kind"]
    if kind in ("heads", "heads_bwd"):
        size = float(case["rows"] * (case["q"] + case["k"]) * case["dim"])
        if kind == "heads":
            return {"bytes": 4 * size + 8.0 * case["rows"] + 8.0 * case["dim"], "flops": 10 * size}
        return {"bytes": 6 * size + 8.0 * case["rows"] + 16.0 * case["dim"], "flops": 20 * size}
    if kind in ("embed", "embed_bwd"):
        n, vocab, cols, wide = case["tokens"], case["vocab"], case["cols"], 4.0 if case["fp32"] else 2.0
        distinct = _distinct(n, vocab)
        if kind == "embed":
            return {"bytes": 8.0 * n + distinct * cols * wide + n * cols * 2.0, "flops": float(n * cols)}
        written = 8.0 * distinct * cols if case["accumulate"] else 4.0 * vocab * cols
        return {"bytes": 8.0 * n + n * cols * wide + written, "flops": 2.0 * n * cols}
    if kind == "logprob":
        size = float(case["rows"] * case["vocab"]) * (4.0 if case["fp32"] else 2.0)
        rows = case["rows"] * (20.0 + 8.0 * case["top"])
        return {"bytes": size * (2 if case["train"] else 1) + rows, "flops": (10.0 if case["train"] else 5.0) * case["rows"] * case["vocab"]}
    sizes, kinds = _grad_sizes(case), _grad_kinds(case)
    wide = 4.0 if case["out_fp32"] else 2.0
    return {"bytes": sum(n * ((4.0 if f else 2.0) + wide) for n, f in zip(sizes, kinds)), "flops": 3.0 * sum(sizes)}


# ------------------------------------------------------------------------------------------------ in 64 bits ----
def _pairs(v, case):
    """The rotated elements of the last axis as complex numbers, and the others."""
    r = case["rotary"]
    if case["interleaved"]:
        return torch.view_as_complex(v[..., :r].reshape(*v.shape[:-1], r // 2, 2).contiguous()), v[..., r:]
    return torch.complex(v[..., :r // 2].contiguous(), v[..., r // 2:r].contiguous()), v[..., r:]


def _turned(v, s, back):
    case = s["case"]
    if not case["rotary"]:
        return v
    z, rest = _pairs(v, case)
    angle = torch.outer(s["positions"].double(), s["inv_freq"].double())
    turn = torch.polar(torch.ones_like(angle), -angle if back else angle)
    z = z * turn.unsqueeze(1)
    if case["interleaved"]:
        return torch.cat([torch.view_as_real(z).reshape(*z.shape[:-1], case["rotary"]), rest], -1)
    return torch.cat([z.real, z.imag, rest], -1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("heads", "heads_bwd"):
        q, k, dim, rows = case["q"], case["k"], case["dim"], case["rows"]
        x = s["x"].double().reshape(rows, q + k, dim)
        length = torch.sqrt((x * x).sum(-1) / dim + EPS).unsqueeze(-1)
        gain = torch.cat([s["gain_q"].double().repeat(q), s["gain_k"].double().repeat(k)]).view(1, q + k, dim)
        if kind == "heads":
            return {"y": _turned(x / length * gain, s, False).reshape(rows, -1)}
        dy = _turned(s["dy"].double().reshape(rows, q + k, dim), s, True)
        by_gain = dy * x / length
        dx = dy * gain / length - x * (dy * gain * x).sum(-1, keepdim=True) / (dim * length ** 3)
        dq, dk = by_gain[:, :q].sum((0, 1)), by_gain[:, q:].sum((0, 1))
        if case["accumulate"]:
            dq, dk = dq + s["dgain_q0"].double(), dk + s["dgain_k0"].double()
        return {"dx": dx.reshape(rows, -1), "dgain_q": dq, "dgain_k": dk}
    if kind in ("embed", "embed_bwd"):
        ok = torch.nonzero((s["tokens"] >= 0) & (s["tokens"] < case["vocab"]))[:, 0]
        if kind == "embed":
            out = torch.zeros(case["tokens"], case["cols"], dtype=torch.float64, device="cuda")
            out[ok] = s["table"].index_select(0, s["tokens"][ok]).double() * _scale(case)
            return {"out": out}
        dtable = s["dtable0"].double() if case["accumulate"] else torch.zeros(case["vocab"], case["cols"], dtype=torch.float64, device="cuda")
        dtable.index_put_((s["tokens"][ok],), s["dout"][ok].double() * _scale(case), accumulate=True)
        return {"dtable": dtable}
    if kind == "logprob":
        rows, vocab, scale = case["rows"], case["vocab"], _scale(case)
        out = {n: torch.empty(rows, dtype=torch.float64, device="cuda") for n in ("lse", "logprob") + (("entropy",) if case["entropy"] else ())}
        if case["top"]:
            out["top_ids"] = torch.empty(rows, case["top"], dtype=torch.int32, device="cuda")
            out["top_logprobs"] = torch.empty(rows, case["top"], dtype=torch.float64, device="cuda")
        if case["train"]:
            out["dlogits"] = torch.zeros(s["dlogits"].shape, dtype=torch.float64, device="cuda")
        step = max(1, (1 << 28) // vocab)
        for r0 in range(0, rows, step):
            part = slice(r0, min(rows, r0 + step))
            z = s["logits"][part].double() * scale
            lse = torch.logsumexp(z, 1)
            lp = z - lse[:, None]
            t = s["targets"][part]
            there = (t >= 0) & (t < vocab)
            out["lse"][part] = lse
            out["logprob"][part] = torch.where(there, lp[torch.arange(len(t), device="cuda"), t.clamp(0, vocab - 1)], 0.0)
            surprise = torch.where(torch.isinf(lp), 0.0, -lp)
            p = torch.exp(lp)
            if case["entropy"]:
                out["entropy"][part] = (p * surprise).sum(1)
            if case["top"]:
                got = torch.sort(s["logits"][part].double(), dim=1, descending=True, stable=True)
                out["top_ids"][part] = got.indices[:, :case["top"]].int()
                out["top_logprobs"][part] = lp.gather(1, got.indices[:, :case["top"]])
            if case["train"]:
                hit = torch.zeros_like(p)
                hit[there, t[there]] = 1.0
                grad = (hit - p) * torch.where(there, s["dlogprob"][part].double(), 0.0)[:, None]
                if case["entropy"]:
                    grad += s["dentropy"][part].double()[:, None] * p * (surprise - (p * surprise).sum(1, keepdim=True))
                out["dlogits"][part, :vocab] = grad * scale
        return out
    norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in s["grads"]))
    most = _max_norm(case)
    factor = min(1.0, most / norm) if norm else 1.0
    return {"stats": torch.tensor([norm, factor], dtype=torch.float64, device="cuda"), "out": torch.cat([g.double() for g in s["grads"]]) * factor}
