"""Head norms with rotation, embedding, log probabilities and clipping against plain references in 64 bits."""
import math

import pytest
import torch

import ends_ref as R
from around_ref import guarded
from ends_ref import HALF, U, normal
from paper_2509_25149_b200 import binding as B

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def scratch(nbytes):
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device="cuda")


def new(*shape, dtype=FP32):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda") if dtype.is_floating_point else torch.full(shape, -7, dtype=dtype, device="cuda")


# ------------------------------------------------------------------------------------------------- heads ----
def heads_inputs(rows, hq, hk, dim, rotary, where, seed=1):
    x = normal((rows, (hq + hk) * dim), seed, 1.5)
    gq, gk = (1 + normal((dim,), seed + k, 0.2, FP32) for k in (1, 2))
    f = torch.exp(-torch.arange(rotary // 2, dtype=torch.float64) * 18.0 / max(rotary, 1)).float() if rotary else None
    p = {"rows": torch.arange(rows), "far": 999_983 + 7 * torch.arange(rows), "before": -torch.arange(rows) * 1000, "huge": (1 << 40) + torch.arange(rows)}[where]
    return x, gq, gk, f, p


def angle_off(f, p):
    """By how much an angle t can differ: position times frequency, both in 53 bits, is off by 2^-53 t in the reference and in the kernel, whose division
    by pi (a product with a rounded number, rounded) adds 2^-52 t."""
    return 0.0 if f is None else 4 * 2.0 ** -53 * float(p.abs().max()) * float(f.max())


HEADS = [  # rows, query heads, key heads, width, rotated, neighbours, positions, spare columns
    (1, 40, 8, 128, 128, False, "far", 1024),
    (1, 1, 0, 8, 0, False, "rows", 0),
    (3, 0, 1, 8, 0, True, "rows", 8),
    (5, 2, 1, 16, 16, False, "before", 0),
    (7, 3, 2, 24, 16, True, "rows", 16),
    (33, 4, 2, 64, 64, False, "rows", 0),
    (65, 6, 2, 80, 32, True, "rows", 8),
    (65, 6, 2, 80, 80, False, "far", 0),
    (129, 3, 3, 96, 48, False, "rows", 64),
    (200, 12, 4, 128, 128, True, "far", 0),
    (17, 5, 1, 192, 192, False, "huge", 0),
    (300, 7, 2, 256, 256, False, "rows", 0),
    (40, 3, 1, 256, 128, True, "before", 8),
    (2500, 8, 2, 128, 64, False, "rows", 256),
    # every place of a step filled, one and two heads to a lane, all widths of a group
    (64, 2, 2, 128, 128, True, "far", 0), (64, 2, 2, 128, 0, False, "rows", 8), (64, 4, 0, 64, 64, False, "rows", 0), (50, 1, 1, 256, 256, False, "rows", 0),
    (50, 2, 2, 256, 64, True, "rows", 0), (50, 8, 8, 64, 64, True, "before", 64), (50, 16, 16, 32, 32, False, "rows", 0), (50, 8, 8, 32, 16, True, "rows", 0),
    (50, 0, 16, 32, 16, False, "rows", 0), (3000, 8, 0, 128, 0, False, "rows", 0),
]


@pytest.mark.parametrize("case", HEADS, ids=str)
def test_heads(case):
    rows, hq, hk, dim, rotary, interleaved, where, spare = case
    x, gq, gk, f, p = heads_inputs(rows, hq, hk, dim, rotary, where)
    cols = (hq + hk) * dim
    want = R.heads_fwd(x.double(), hq, hk, gq, gk, 1e-5, f, p, interleaved)
    u = R.heads_fwd(x.double(), hq, hk, gq, gk, 1e-5, None, p, interleaved).unflatten(1, (hq + hk, dim))
    # roundings of the sum of squares, the root, the angle (half a turn at 2^-25), sine and cosine: below 2^-20 of both elements' magnitudes
    tol = HALF[BF16] * want.abs() + (2.0 ** -19 + angle_off(f, p)) * R.beside(u, rotary, interleaved).flatten(1)
    c = lambda t: None if t is None else t.cuda()
    xs, untouched = guarded(rows, cols, BF16, cols + spare, x)
    for pos in (p, p.int()) if p.abs().max() < 1 << 31 else (p,):
        y, clean = guarded(rows, cols, BF16, cols + 2 * spare)
        B.nvfp4_headnorm_fwd(xs, hq, hk, y, c(gq), c(gk), 1e-5, c(f), c(pos), interleaved)
        R.assert_within(y, want, tol, "y")
        assert clean() and untouched()
    again = xs.clone()
    B.nvfp4_headnorm_fwd(again, hq, hk, again, c(gq), c(gk), 1e-5, c(f), c(p), interleaved)  # in place
    assert torch.equal(again, y)
    if where == "rows":
        B.nvfp4_headnorm_fwd(xs, hq, hk, again, c(gq), c(gk), 1e-5, c(f), None, interleaved)
        assert torch.equal(again, y)
    B.nvfp4_headnorm_fwd(xs, hq, hk, again, None, c(gk), 1e-5, c(f), c(p), interleaved)
    ones = torch.ones(dim, device="cuda")
    B.nvfp4_headnorm_fwd(xs, hq, hk, y, ones, c(gk), 1e-5, c(f), c(p), interleaved)
    assert torch.equal(again, y)


def heads_gradient(x, dy, hq, hk, gq, gk, f, p, interleaved):
    leaves = [t.double().requires_grad_() for t in (x, gq, gk)]
    R.heads_fwd(leaves[0], hq, hk, leaves[1], leaves[2], 1e-5, f, p, interleaved).backward(dy.double())
    return [t.grad if t.grad is not None else torch.zeros_like(t) for t in leaves]


@pytest.mark.parametrize("case", HEADS, ids=str)
def test_heads_gradient(case):
    rows, hq, hk, dim, rotary, interleaved, where, spare = case
    x, gq, gk, f, p = heads_inputs(rows, hq, hk, dim, rotary, where)
    cols = (hq + hk) * dim
    dy = normal(x.shape, 9, 1e-2)
    dx64, dgq64, dgk64 = heads_gradient(x, dy, hq, hk, gq, gk, f, p, interleaved)
    h = x.double().unflatten(1, (hq + hk, dim))
    rstd = 1 / (h.square().mean(2, keepdim=True) + 1e-5).sqrt()
    n = h * rstd
    d = R.beside(dy.double().unflatten(1, (hq + hk, dim)), rotary, interleaved)
    gain = torch.cat([gq.double().expand(hq, -1), gk.double().expand(hk, -1)])
    reach = rstd * (d * gain.abs() + n.abs() * (d * gain.abs() * n.abs()).mean(2, keepdim=True))
    tol = HALF[BF16] * dx64.abs() + (2.0 ** -18 + 2 * angle_off(f, p)) * reach.flatten(1)
    # chains of less than 200 additions in all (a lane's, the lanes', the warps', the CTAs')
    of = (d * n.abs()).sum(0) * (1 + 2.0 ** 16 * angle_off(f, p))
    c = lambda t: None if t is None else t.cuda()
    xs, dys = guarded(rows, cols, BF16, cols + spare, x)[0], guarded(rows, cols, BF16, cols + 8, dy)[0]
    ws = scratch(B.nvfp4_headnorm_bwd_workspace_bytes(rows, hq, hk, dim))
    first = None
    for accumulate in (False, True):
        dx, clean = guarded(rows, cols, BF16, cols + spare)
        dgq, dgk = (normal((dim,), k, 1.0, FP32).cuda() for k in (11, 12))
        before = [t.double().cpu() if accumulate else torch.zeros(dim, dtype=torch.float64) for t in (dgq, dgk)]
        B.nvfp4_headnorm_bwd(dys, xs, hq, hk, dx, c(gq), c(gk), 1e-5, dgq, dgk, ws, c(f), c(p), interleaved, accumulate)
        R.assert_within(dx, dx64, tol, "dx")
        for got, want, b, t, name in ((dgq, dgq64, before[0], of[:hq].sum(0), "dgain_q"), (dgk, dgk64, before[1], of[hq:].sum(0), "dgain_k")):
            R.assert_within(got, want + b, 2.0 ** -16 * t + 2 * U * (want + b).abs(), name)
        assert clean()
        first = dx.clone() if first is None else first
        assert torch.equal(first, dx)
    for target in (dys, xs):  # in place of either
        a, b = dys.clone(), xs.clone()
        out = a if target is dys else b
        B.nvfp4_headnorm_bwd(a, b, hq, hk, out, c(gq), c(gk), 1e-5, None, None, None, c(f), c(p), interleaved)
        assert torch.equal(out, first)
    only = new(dim)
    again = new(dim)
    B.nvfp4_headnorm_bwd(dys, xs, hq, hk, dx, c(gq), c(gk), 1e-5, None, only, ws, c(f), c(p), interleaved)
    B.nvfp4_headnorm_bwd(dys, xs, hq, hk, dx, c(gq), c(gk), 1e-5, again, None, ws, c(f), c(p), interleaved)
    R.assert_within(only, dgk64, 2.0 ** -16 * of[hq:].sum(0), "dgain_k alone")
    R.assert_within(again, dgq64, 2.0 ** -16 * of[:hq].sum(0), "dgain_q alone")


def test_heads_gradient_against_differences():
    """The reference's own gradient, and through it the kernel's, along a random direction of the input."""
    rows, hq, hk, dim, rotary = 6, 2, 1, 32, 16
    x, gq, gk, f, p = heads_inputs(rows, hq, hk, dim, rotary, "far")
    dy = normal(x.shape, 9)
    v = normal(x.shape, 10, 1.0, torch.float64)
    dx = torch.empty_like(x, device="cuda")
    B.nvfp4_headnorm_bwd(dy.cuda(), x.cuda(), hq, hk, dx, gq.cuda(), gk.cuda(), 1e-5, inv_freq=f.cuda(), positions=p.cuda())
    g = lambda t: (R.heads_fwd(x.double() + t * v, hq, hk, gq, gk, 1e-5, f, p, False) * dy.double()).sum()
    along = float((g(1e-4) - g(-1e-4)) / 2e-4)
    got = float((dx.double().cpu() * v).sum())
    assert abs(got - along) <= float((HALF[BF16] * dx.double().cpu().abs() * v.abs()).sum()) + 1e-5 * abs(along)


@pytest.mark.parametrize("magnitude", [3e38, 1e20, 1e-20, 0.0])
def test_heads_of_any_finite_magnitude(magnitude):
    rows, hq, hk, dim = 9, 3, 2, 128
    x = (normal((rows, (hq + hk) * dim), 5).clamp(-1, 1).float() * magnitude).to(BF16)
    x[0, :dim] = 0
    f = torch.exp(-torch.arange(64) * 0.1).float()
    want = R.heads_fwd(x.double(), hq, hk, None, None, 1e-5, f, torch.arange(rows), False)
    u = R.heads_fwd(x.double(), hq, hk, None, None, 1e-5, None, None, False).unflatten(1, (hq + hk, dim))
    y = torch.empty_like(x, device="cuda")
    B.nvfp4_headnorm_fwd(x.cuda(), hq, hk, y, inv_freq=f.cuda())
    R.assert_within(y, want, HALF[BF16] * want.abs() + 2.0 ** -19 * R.beside(u, dim, False).flatten(1) + 2.0 ** -134, "y")


# --------------------------------------------------------------------------------------------- embedding ----
EMBED = [  # tokens, vocabulary, columns, spare columns
    (1, 1, 8, 0), (1, 100, 64, 8), (3, 7, 1000, 0), (33, 5, 136, 8), (257, 50, 2056, 0), (1003, 5003, 264, 16), (4096, 600, 72, 0), (5000, 3, 40, 8),
    (9001, 70001, 16, 0), (40000, 11, 24, 0), (20000, 300000, 8, 8), (70003, 1000, 16, 0), (100000, 600000, 8, 8),
    (4097, 9000, 8, 0), (32768, 900, 8, 0), (32769, 900, 8, 8),  # where the ways to sort change
]


def tokens_of(n, vocab, seed, padding=True):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, vocab, (n,), generator=g)
    often = torch.rand(n, generator=g) < 0.3
    t[often] = vocab // 2
    if padding and n > 2:
        t[torch.rand(n, generator=g) < 0.05] = -1
        t[n // 2], t[n - 1] = vocab, (1 << 40)
    return t


@pytest.mark.parametrize("case", EMBED, ids=str)
@pytest.mark.parametrize("types", [(BF16, BF16), (FP32, BF16), (BF16, FP32), (FP32, FP32)], ids=str)
def test_embedding(case, types):
    n, vocab, cols, spare = case
    t = tokens_of(n, vocab, 3)
    table = normal((vocab, cols), 4, 1.0, types[0])
    there = (t >= 0) & (t < vocab)
    for scale in (1.0, 3.1):
        want = torch.where(there[:, None], table[torch.where(there, t, 0)].float() * torch.tensor(scale), 0.0).to(types[1])
        tab, out = guarded(vocab, cols, types[0], cols + spare, table)[0], guarded(n, cols, types[1], cols + 2 * spare)
        B.nvfp4_embedding_fwd(t.cuda(), tab, out[0], scale)
        assert torch.equal(out[0].cpu(), want) and out[1]()
    narrow = torch.where(there, t, -5).int()
    B.nvfp4_embedding_fwd(narrow.cuda(), tab, out[0], scale)
    assert torch.equal(out[0].cpu(), want) and out[1]()


@pytest.mark.parametrize("case", EMBED, ids=str)
@pytest.mark.parametrize("dtype", [BF16, FP32], ids=str)
def test_embedding_gradient(case, dtype):
    n, vocab, cols, spare = case
    t = tokens_of(n, vocab, 3)
    dout = normal((n, cols), 5, 1e-2, dtype)
    before = normal((vocab, cols), 6, 1.0, FP32)
    there = (t >= 0) & (t < vocab)
    scale = 2.7
    sums, reach = (torch.zeros(vocab, cols, dtype=torch.float64).index_add_(0, t[there], v[there]) for v in (dout.double(), dout.double().abs()))
    count = torch.bincount(t[there], minlength=vocab).double()[:, None]
    g = guarded(n, cols, dtype, cols + spare, dout)[0]
    ws = scratch(B.nvfp4_embedding_bwd_workspace_bytes(n, vocab, cols))
    for accumulate in (False, True):
        # additions one by one at worst, the shares' sums and the product
        want = sums * float(torch.tensor(scale)) + (before.double() if accumulate else 0)
        tol = (count + 3) * U * reach * scale + 2 * U * want.abs()
        got = []
        for k in range(2):
            table, clean = guarded(vocab, cols, FP32, cols + spare, before)
            ws.fill_(255 * k)  # what a workspace held before says nothing
            B.nvfp4_embedding_bwd((t if k else torch.where(there, t, -1).int()).cuda(), g, table, ws, scale, accumulate)
            R.assert_within(table, want, tol, "dtable")
            assert clean()
            got.append(table.clone())
        assert torch.equal(got[0], got[1])
        none = count[:, 0] == 0
        assert torch.equal(got[0].cpu()[none], before[none] if accumulate else torch.zeros_like(before[none]))


@pytest.mark.parametrize("n", [1, 8, 9, 31, 32, 33, 255, 4097, 33000, 70001])
@pytest.mark.parametrize("token", [0, 2, -1, 3])
def test_embedding_gradient_of_one_token(n, token):
    """Every place has the same token, or is padding: a run over all chunks."""
    t, dout = torch.full((n,), token), normal((n, 16), 5)
    table = new(3, 16)
    B.nvfp4_embedding_bwd(t.cuda(), dout.cuda(), table, scratch(B.nvfp4_embedding_bwd_workspace_bytes(n, 3, 16)))
    want = torch.zeros(3, 16, dtype=torch.float64)
    if token in (0, 2):
        want[token] = dout.double().sum(0)
    # a chunk's additions one by one (n / 1024 + 8 at most, or 32), the chunks' in 64 bits
    R.assert_within(table, want, (max(n / 1024 + 8, 32) + 2) * U * dout.double().abs().sum(0) * (want != 0), "dtable")


def test_embedding_gradient_is_that_of_differences():
    """<dout, out(table + t v)> is linear in t: its slope is <dtable, v>."""
    n, vocab, cols = 50, 20, 24
    t, table, v, dout = tokens_of(n, vocab, 1), normal((vocab, cols), 2, 1.0, FP32), normal((vocab, cols), 3, 1.0, FP32), normal((n, cols), 4, 1.0, FP32)
    outs = []
    for k in (0.0, 1.0):
        out = new(n, cols)
        B.nvfp4_embedding_fwd(t.cuda(), (table + k * v).cuda(), out, 1.5)
        outs.append((out.double().cpu() * dout.double()).sum())
    dtable = new(vocab, cols)
    B.nvfp4_embedding_bwd(t.cuda(), dout.cuda(), dtable, scratch(B.nvfp4_embedding_bwd_workspace_bytes(n, vocab, cols)), 1.5)
    assert abs(float((dtable.double().cpu() * v.double()).sum() - (outs[1] - outs[0]))) < 1e-3


# ----------------------------------------------------------------------------------------------- logprob ----
def logits_of(rows, vocab, kind, dtype, seed=1):
    x = normal((rows, vocab), seed, 3.0, FP32)
    g = torch.Generator().manual_seed(seed + 1)
    if kind == "masked":
        x[torch.rand(rows, vocab, generator=g) < 0.4] = -math.inf
        x[0] = -math.inf
        x[-1] = -math.inf
        x[-1, vocab - 1] = 2.0
    elif kind == "few":  # all but some five are ruled out
        x[torch.rand(rows, vocab, generator=g) > 5 / vocab] = -math.inf
    elif kind == "lowest":
        x[torch.rand(rows, vocab, generator=g) < 0.4] = torch.finfo(dtype).min
        x[0] = torch.finfo(dtype).min
    elif kind == "equal":
        x[:] = 1.25
    elif kind == "steps":
        x = (x * 2).round() / 2
        x[x == 0] = torch.where(torch.rand(int((x == 0).sum()), generator=g) < 0.5, 0.0, -0.0)
    elif kind == "rising":
        x = torch.arange(vocab).float().expand(rows, -1) * 0.01
    elif kind == "large":
        x = x * 1000 + 20000
    elif kind == "sure":
        x[:, vocab // 2] = 200.0
    elif kind == "columns":  # the largest stand where one thread reads them
        x[:, ::4096] += 50
    return x.to(dtype)


LOGITS = [(rows, vocab, "plain") for rows, vocab in ((1, 1), (3, 2), (5, 7), (2, 8), (4, 33), (3, 1000), (2, 4097), (700, 257), (9, 32768), (2, 50257), (1, 131072), (160, 9000))]
LOGITS += [(5, vocab, kind) for kind in ("masked", "few", "lowest", "equal", "steps", "rising", "large", "sure", "columns") for vocab in (100, 5001, 70000)]
LOGITS += [(2049, 4104, "masked"), (2049, 4099, "steps"), (2048, 4200, "equal")]  # many rows of more than 4096: a warp takes each


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=str)
@pytest.mark.parametrize("case", LOGITS, ids=str)
def test_logprob(case, dtype):
    rows, vocab, kind = case
    x = logits_of(rows, vocab, kind, dtype)
    g = torch.Generator().manual_seed(7)
    targets = torch.randint(0, vocab, (rows,), generator=g)
    if rows > 2:
        targets[1], targets[2] = -1, vocab
    there = (targets >= 0) & (targets < vocab)
    wide = (vocab + 7) // 8 * 8 + 16
    xs, untouched = guarded(rows, vocab, dtype, wide, x)
    for scale in (1.0, 0.7):
        ref = R.Softmax(x, scale)
        lp, lse, stats, entropy = new(rows), new(rows), new(rows, 2), new(rows)
        B.nvfp4_logprob_fwd(xs, targets.cuda(), lp, lse, stats, entropy, scale=scale)
        at = torch.where(there, targets, 0)[:, None]
        want = torch.where(there, ref.log_p.gather(1, at)[:, 0], 0.0)
        R.assert_within(lp, want, torch.where(there, ref.log_p_off().gather(1, at)[:, 0], 0.0), "logprob")
        R.assert_within(lse, ref.lse, ref.lse_off, "lse")
        R.assert_within(entropy, ref.entropy, ref.entropy_off, "entropy")
        assert torch.equal(stats[:, 0].cpu(), x.float().max(1).values) and untouched()
        # each output alone is the same
        for name in ("logprob", "lse", "entropy"):
            alone = new(rows)
            B.nvfp4_logprob_fwd(xs, targets.int().cuda(), **{name: alone}, scale=scale)
            if name != "entropy":
                assert torch.equal(alone, {"logprob": lp, "lse": lse}[name])
            else:
                assert torch.equal(alone, entropy)
        for out_dtype in (dtype, FP32 if dtype == BF16 else BF16):
            dlp, de = normal((rows,), 8, 1.0, FP32), normal((rows,), 9, 0.3, FP32)
            for a, b in ((dlp, None), (None, de), (dlp, de)):
                out, clean = guarded(rows, wide - 8, out_dtype, wide + 8)
                c = lambda t: None if t is None else t.cuda()
                B.nvfp4_logprob_bwd(xs, None if a is None else targets.cuda(), stats, out, c(a), None if b is None else entropy, c(b), scale)
                grad, tol = ref.grad(targets, a, b, scale)
                R.assert_within(out[:, :vocab], grad, tol + HALF[out_dtype] * (grad.abs() + tol) + 1e-38, "dlogits")
                assert bool((out[:, vocab:] == 0).all()) and clean()
        out = xs.clone() if rows == 1 else guarded(rows, vocab, dtype, wide, x)[0]
        other = guarded(rows, vocab, dtype, wide)[0]
        for to, source in ((other, xs), (out, out)):  # in place too
            B.nvfp4_logprob_bwd(source, targets.cuda(), stats, to, dlp.cuda(), entropy, de.cuda(), scale)
        assert torch.equal(out, other)


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=str)
@pytest.mark.parametrize("case", LOGITS, ids=str)
def test_top_alternatives(case, dtype):
    rows, vocab, kind = case
    x = logits_of(rows, vocab, kind, dtype)
    xs = guarded(rows, vocab, dtype, (vocab + 7) // 8 * 8 + 8, x)[0]
    ref = R.Softmax(x, 1.3)
    for top in (1, 2, 5, 20, 32):
        if top > vocab:
            continue
        ids, lps, lse = new(rows, top, dtype=torch.int32), new(rows, top), new(rows)
        B.nvfp4_logprob_fwd(xs, top_ids=ids, top_logprobs=lps, lse=lse, scale=1.3)
        want = R.top_of(x, top)
        assert torch.equal(ids.cpu().long(), want), top
        R.assert_within(lps, ref.log_p.gather(1, want), ref.log_p_off().gather(1, want), "top_logprobs")
        R.assert_within(lse, ref.lse, ref.lse_off, "lse")
        again = new(rows, top, dtype=torch.int32)
        B.nvfp4_logprob_fwd(xs, top_ids=again, scale=1.3)
        assert torch.equal(again, ids)


def test_logprob_gradient_against_differences():
    rows, vocab, scale = 4, 37, 0.8
    x, targets = logits_of(rows, vocab, "plain", FP32), torch.tensor([3, -1, 36, 0])
    dlp, de, v = normal((rows,), 1, 1.0, FP32), normal((rows,), 2, 1.0, FP32), normal((rows, vocab), 3, 1.0, torch.float64)
    xs = guarded(rows, vocab, FP32, 40, x)[0]
    stats, entropy, out = new(rows, 2), new(rows), guarded(rows, vocab, FP32, 40)[0]
    B.nvfp4_logprob_fwd(xs, stats=stats, entropy=entropy, scale=scale)
    B.nvfp4_logprob_bwd(xs, targets.cuda(), stats, out, dlp.cuda(), entropy, de.cuda(), scale)

    def loss(t):
        s = R.Softmax(x.double() + t * v, scale)
        there = targets >= 0
        lp = torch.where(there, s.log_p.gather(1, targets.clamp(0)[:, None])[:, 0], 0.0)
        return float((lp * dlp.double() + s.entropy * de.double()).sum())

    along = (loss(1e-5) - loss(-1e-5)) / 2e-5
    assert abs(float((out.double().cpu() * v).sum()) - along) <= 1e-5 * (1 + abs(along))


# -------------------------------------------------------------------------------------------------- clip ----
def gradients(sizes, kinds, seed=1, std=1e-2, offset=0):
    out = []
    for i, (n, k) in enumerate(zip(sizes, kinds)):
        dtype = FP32 if k else BF16
        at = (offset + 3 * i) % 9
        flat = torch.zeros(n + 16, dtype=dtype, device="cuda")
        flat[at:at + n] = normal((n,), seed + i, std, dtype).cuda()
        out.append(flat[at:at + n])
    return out


GRADS = {
    "one": ([1], [True]), "some": ([5, 0, 8191, 8192, 8193, 3], [True, False, False, True, False, True]),
    "odd": ([1 + 37 * i % 9001 for i in range(80)], [i % 3 > 0 for i in range(80)]), "many": ([1 + i % 50 for i in range(1500)], [i % 2 > 0 for i in range(1500)]),
    "large": ([20_000_003, 7, 5_000_000], [True, False, False]), "empty": ([0, 0], [True, False]),
}


@pytest.mark.parametrize("out_dtype", [BF16, FP32, None], ids=str)
@pytest.mark.parametrize("name", GRADS)
def test_clipping(name, out_dtype):
    sizes, kinds = GRADS[name]
    grads = gradients(sizes, kinds)
    before = [g.clone() for g in grads]
    total = sum(float(g.double().square().sum()) for g in grads)
    norm = math.sqrt(total)
    outs = None if out_dtype is None else [torch.full((n + 4,), 7.0, dtype=out_dtype, device="cuda")[i % 4:i % 4 + n] for i, n in enumerate(sizes)]
    ws, got, stats = scratch(B.nvfp4_grad_sq_norm_workspace_bytes()), torch.full((1,), 5.0, dtype=torch.float64, device="cuda"), new(2)
    held = B.grad_list(grads, outs)
    B.nvfp4_grad_sq_norm(held, got, ws)
    assert abs(float(got) - total) <= 2.0 ** -20 * total  # eight squares added in binary32, 8 roundings at most
    B.nvfp4_grad_sq_norm(held, got, ws, accumulate=True)
    assert abs(float(got) - 2 * total) <= 2.0 ** -20 * total
    B.nvfp4_grad_sq_norm(held, got, ws)
    for most in (2 * norm + 1, 0.25 * norm + 1e-9):  # left alone, then scaled
        B.nvfp4_grad_clip(held, got, most, stats)
        factor = min(1.0, most / norm) if norm else 1.0
        R.assert_within(stats, torch.tensor([norm, factor]), torch.tensor([norm, factor]) * 2.0 ** -20, "stats")
        for g, b, o, n in zip(grads, before, outs or grads, sizes):
            want = b.double() * factor
            if factor == 1.0:
                assert torch.equal(o, b.to(o.dtype))
            else:
                R.assert_within(o, want, (HALF[o.dtype] + 2.0 ** -20) * want.abs() + 1e-40, "clipped")
            if outs is not None:
                assert torch.equal(g, b)
    for g, n in zip(grads, sizes):  # what stands around the tensors is left alone
        flat = torch.as_strided(g, (n + 16,), (1,), 0) if n else None
        if n:
            at = g.storage_offset()
            assert bool((flat[:at] == 0).all()) and bool((flat[at + n:] == 0).all())


@pytest.mark.parametrize("std", [1e30, 1e-25, 1e-38])
def test_norms_beyond_the_squares_of_binary32(std):
    grads = gradients([1003, 70001], [True, True], std=std)
    total = sum(float(g.double().square().sum()) for g in grads)
    got, stats = torch.zeros(1, dtype=torch.float64, device="cuda"), new(2)
    held = B.grad_list(grads)
    B.nvfp4_grad_sq_norm(held, got, scratch(B.nvfp4_grad_sq_norm_workspace_bytes()))
    assert abs(float(got) - total) <= 2.0 ** -20 * total
    before = [g.double() for g in grads]
    most = 0.5 * math.sqrt(total)
    B.nvfp4_grad_clip(held, got, most, stats)
    for g, b in zip(grads, before):
        R.assert_within(g, 0.5 * b, 2.0 ** -20 * b.abs() + 2.0 ** -149, "clipped")


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("kind", [True, False])
def test_a_norm_that_is_not_finite_gives_zeros(bad, kind):
    grads = gradients([77, 9001, 12], [kind, True, False])
    grads[0][5] = bad
    outs = [torch.ones_like(g) for g in grads]
    got, stats = torch.zeros(1, dtype=torch.float64, device="cuda"), new(2)
    for held, to in ((B.grad_list(grads, outs), outs), (B.grad_list(grads), grads)):
        B.nvfp4_grad_sq_norm(held, got, scratch(B.nvfp4_grad_sq_norm_workspace_bytes()))
        B.nvfp4_grad_clip(held, got, 1.0, stats)
        assert float(stats[1]) == 0.0 and not math.isfinite(float(stats[0]))
        assert all(bool((o == 0).all()) for o in to)
