"""The operators at the ends of a training step over the whole range of what they accept, logits and scales of any finite size among it, and behind the
library's own kernels."""
import math

import pytest
import torch

import ends_ref as R
from around_ref import guarded
from ends_ref import HALF, U, normal
from paper_2509_25149_b200 import binding as B

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def new(*shape, dtype=FP32):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda") if dtype.is_floating_point else torch.full(shape, -7, dtype=dtype, device="cuda")


# ----------------------------------------------------------------------------------------------- logprob ----
SIZES = [1e5, 5e6, 1.3e7, 1e8, 1e9, 3e9, 1e10, 1.2e10, 1e12, 1e20, 2.0 ** 90 * (1 - 2.0 ** -7), 2.0 ** 90, 2.0 ** 90 * (1 + 2.0 ** -7)]
KINDS = ["equal", "equal below", "one", "half below", "around", "around below", "up", "close"]


def far_logits(kind, vocab, dtype, seed=1):
    """A row to each size."""
    size = torch.tensor(SIZES, dtype=torch.float64)[:, None]
    x = normal((len(SIZES), vocab), seed, 3.0, torch.float64)
    if kind == "equal":
        x = size.expand(-1, vocab)
    elif kind == "equal below":  # every token is masked with a finite number
        x = -size.expand(-1, vocab)
    elif kind == "one":
        x = torch.zeros_like(x)
        x[:, vocab // 3] = size[:, 0]
    elif kind == "half below":
        x = torch.where(torch.arange(vocab) % 2 == 0, x, -size)
    elif kind in ("around", "around below"):
        x = (1 + 0.01 * x) * (size if kind == "around" else -size)
    elif kind == "up":  # from small to large: the row's maximum grows over the whole range
        x = torch.exp(torch.linspace(0, 1, vocab, dtype=torch.float64) * size.log())
    else:  # the largest ones differ by little in binary32, by a step or none in bf16
        x = size * (1 - torch.arange(vocab, dtype=torch.float64) % 37 * 2.0 ** -22)
    return x.to(dtype)


# rows of a warp, of a CTA (repeated so that there are many), of clusters
@pytest.mark.parametrize("dtype", [BF16, FP32], ids=str)
@pytest.mark.parametrize("scale", [1.0, 0.7, 1e6, 1e8, 2.0 ** 27, 2.0 ** -60], ids=str)
@pytest.mark.parametrize("vocab, times", [(100, 1), (4500, 12), (5001, 1), (40003, 1)])
def test_logits_of_any_finite_size(vocab, times, scale, dtype):
    wide = (vocab + 7) // 8 * 8 + 8
    for kind in KINDS:
        x = far_logits(kind, vocab, dtype)
        rows, many = len(x), len(x) * times
        ref = R.Softmax(x, scale)
        targets = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(7))
        targets[0], targets[-1], targets[1] = vocab // 3, vocab - 1, -1
        there = targets >= 0
        xs, tg = guarded(many, vocab, dtype, wide, x.repeat(times, 1))[0], targets.repeat(times).cuda()
        lp, lse, stats, entropy = new(many), new(many), new(many, 2), new(many)
        B.nvfp4_logprob_fwd(xs, tg, lp, lse, stats, entropy, scale=scale)
        alone_lp, alone_lse, alone_stats = new(many), new(many), new(many, 2)
        B.nvfp4_logprob_fwd(xs, tg, alone_lp, alone_lse, alone_stats, scale=scale)
        top = min(5, vocab)
        ids, tops = new(many, top, dtype=torch.int32), new(many, top)
        B.nvfp4_logprob_fwd(xs, top_ids=ids, top_logprobs=tops, scale=scale)
        # A log probability: roundings of the difference, of the scale in powers of two, of their product, of the sum's logarithm beside it,
        # of ln 2 and of the product with that, beside what the sum is off by.
        off = ref.sum_off[:, None] + 6 * U * (ref.surprise + ref.log_total.abs())
        at = torch.where(there, targets, 0)[:, None]
        want_lp, lp_off = torch.where(there, ref.log_p.gather(1, at)[:, 0], 0.0), torch.where(there, off.gather(1, at)[:, 0], 0.0)
        first = R.top_of(x, top)
        for k in sorted({0, times - 1}):
            part = slice(k * rows, (k + 1) * rows)
            for a, b in ((lp, lse), (alone_lp, alone_lse)):
                R.assert_within(a[part], want_lp, lp_off, f"{kind}: logprob")
                R.assert_within(b[part], ref.lse, ref.lse_off, f"{kind}: lse")
            R.assert_within(entropy[part], ref.entropy, ref.entropy_off, f"{kind}: entropy")
            assert torch.equal(stats[part, 0].cpu(), x.float().max(1).values)
            assert torch.equal(ids[part].cpu().long(), first), kind
            R.assert_within(tops[part], ref.log_p.gather(1, first), off.gather(1, first), f"{kind}: top_logprobs")
        dlp, de = normal((rows,), 8, 1.0, FP32), normal((rows,), 9, 0.3, FP32)
        for a, b, st in ((dlp, None, alone_stats), (None, de, stats), (dlp, de, stats)):
            c = lambda t: None if t is None else t.repeat(times).cuda()
            grad, tol = ref.grad(targets, a, b, scale)
            for out_dtype in (BF16, FP32):
                out = guarded(many, vocab, out_dtype, wide)[0]
                B.nvfp4_logprob_bwd(xs, None if a is None else tg, st, out, c(a), None if b is None else entropy, c(b), scale)
                for k in sorted({0, times - 1}):
                    R.assert_within(out[k * rows:(k + 1) * rows], grad, tol + HALF[out_dtype] * (grad.abs() + tol) + 1e-38, f"{kind}: dlogits")


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=str)
@pytest.mark.parametrize("rows, vocab", [(5, 1000), (160, 9000), (5, 9000), (5, 40000)])
def test_a_nan_among_logits_that_are_ruled_out(rows, vocab, dtype):
    """Rows 0 to 2 have a NaN: beside nothing but minus infinities; beside a target of minus infinity; beside a target far below.  Rows from 3 on have none."""
    x = normal((rows, vocab), 1, 2.0, dtype)
    x[0] = -math.inf
    x[0, 5] = math.nan
    x[1:3, vocab // 3] = math.nan
    x[1, 7], x[2, 7], x[3, 7] = -math.inf, torch.finfo(dtype).min, -math.inf
    x[4] = -math.inf
    z, tg, w = x.cuda(), torch.full((rows,), 7, device="cuda"), torch.ones(rows, device="cuda")
    bad = torch.arange(rows, device="cuda") < 3
    for with_entropy in (False, True):
        lp, lse, st, en, dz = new(rows), new(rows), new(rows, 2), new(rows) if with_entropy else None, torch.zeros_like(z)
        ids, tops = new(rows, 5, dtype=torch.int32), new(rows, 5)
        B.nvfp4_logprob_fwd(z, tg, lp, lse, st, en, ids, tops)
        for t in (lp, lse, en, tops[:, 0], tops[:, 4]):
            assert t is None or torch.equal(torch.isnan(t), bad)
        assert int(ids.min()) >= 0 and int(ids.max()) < vocab
        assert bool(torch.isinf(lp[3:5]).all()) and bool((lp[3:5] < 0).all())
        for dlogprob, dentropy in ((w, None), (None, w), (w, w)) if with_entropy else ((w, None),):
            B.nvfp4_logprob_bwd(z, None if dlogprob is None else tg, st, dz, dlogprob, None if dentropy is None else en, dentropy)
            assert bool(torch.isnan(dz[:3]).all()) and bool(torch.isfinite(dz[3:]).all()) and bool((dz[4] == 0).all())


# ------------------------------------------------------------------------------------------------- heads ----
LARGEST = torch.finfo(FP32).max


@pytest.mark.parametrize("dim", [16, 128, 256])
@pytest.mark.parametrize("eps", [1.0, 1e30, 1e38, 3e38, LARGEST], ids=str)
def test_heads_with_a_large_eps(eps, dim):
    """Sums of squares on both sides of the largest binary32 number, beside an eps of their size."""
    sizes = torch.tensor([1.0, 1e15, 1e17, 5e17, 1e18, 2e18, 5e18, 1e19, 3e19, 1e20, 1e22, 1e30, 3e38], dtype=torch.float64)
    hq, hk = 2, 1
    rows, cols = len(sizes), (hq + hk) * dim
    x = (normal((rows, cols), 5, 0.5, torch.float64).clamp(-1, 1) * sizes[:, None]).to(BF16)
    eps = float(torch.tensor(eps, dtype=FP32))
    f, dy = torch.exp(-torch.arange(8) * 0.5).float(), normal((rows, cols), 6)
    gain = 1 + normal((dim,), 7, 0.2, FP32)
    leaves = [t.double().requires_grad_() for t in (x, gain, gain)]
    want = R.heads_fwd(leaves[0], hq, hk, leaves[1], leaves[2], eps, f, torch.arange(rows), False)
    want.backward(dy.double())
    u = R.heads_fwd(x.double(), hq, hk, gain, gain, eps, None, None, False).unflatten(1, (hq + hk, dim))
    y, dx, dgq, dgk = torch.empty_like(x, device="cuda"), torch.empty_like(x, device="cuda"), new(dim), new(dim)
    ws = torch.empty(B.nvfp4_headnorm_bwd_workspace_bytes(rows, hq, hk, dim), dtype=torch.uint8, device="cuda")
    B.nvfp4_headnorm_fwd(x.cuda(), hq, hk, y, gain.cuda(), gain.cuda(), eps, f.cuda())
    B.nvfp4_headnorm_bwd(dy.cuda(), x.cuda(), hq, hk, dx, gain.cuda(), gain.cuda(), eps, dgq, dgk, ws, f.cuda())
    # the bounds of the ordinary heads: roundings of the sum of squares, the root, sine and cosine, and those of the sums in the gradient
    R.assert_within(y, want, HALF[BF16] * want.abs() + 2.0 ** -19 * R.beside(u, 16, False).flatten(1) + 2.0 ** -134, "y")
    h = x.double().unflatten(1, (hq + hk, dim))
    rstd = 1 / (h.square().mean(2, keepdim=True) + eps).sqrt()
    n, d = h * rstd, R.beside(dy.double().unflatten(1, (hq + hk, dim)), 16, False)
    reach = rstd * (d * gain.abs() + n.abs() * (d * gain.abs() * n.abs()).mean(2, keepdim=True))
    R.assert_within(dx, leaves[0].grad, HALF[BF16] * leaves[0].grad.abs() + 2.0 ** -18 * reach.flatten(1) + 2.0 ** -134, "dx")
    of = (d * n.abs()).sum(0)
    R.assert_within(dgq, leaves[1].grad, 2.0 ** -16 * of[:hq].sum(0), "dgain_q")
    R.assert_within(dgk, leaves[2].grad, 2.0 ** -16 * of[hq:].sum(0), "dgain_k")


@pytest.mark.parametrize("rotary", [0, 32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_small_heads_with_small_gains(interleaved, rotary):
    """x gain is below the smallest normal binary32 number, x gain / rms is not."""
    rows, hq, hk, dim, eps = 7, 2, 1, 32, 2.0 ** -126
    x = (normal((rows, (hq + hk) * dim), 5, 1.0, torch.float64) * 2.0 ** -119).to(BF16)
    gain = ((1 + normal((dim,), 7, 0.2, torch.float64)) * 2.0 ** -26).float()
    f = torch.exp(-torch.arange(rotary // 2) * 0.5).float() if rotary else None
    want = R.heads_fwd(x.double(), hq, hk, gain, gain, eps, f, torch.arange(rows), interleaved)
    u = R.heads_fwd(x.double(), hq, hk, gain, gain, eps, None, None, False).unflatten(1, (hq + hk, dim))
    y = torch.empty_like(x, device="cuda")
    B.nvfp4_headnorm_fwd(x.cuda(), hq, hk, y, gain.cuda(), gain.cuda(), eps, None if f is None else f.cuda(), interleaved=interleaved)
    R.assert_within(y, want, HALF[BF16] * want.abs() + 2.0 ** -19 * R.beside(u, rotary, interleaved).flatten(1), "y")


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=str)
@pytest.mark.parametrize("rows", [1, 2])
def test_gradient_over_the_logits_with_more_columns(rows, dtype):
    """The logits are the first columns of what the product wrote, and their gradient goes over all of them, one row too."""
    vocab, wide = 1003, 1024
    x = normal((rows, wide), 3, 2.0, dtype).cuda()
    tg, w, st = torch.arange(rows, device="cuda"), torch.ones(rows, device="cuda"), new(rows, 2)
    B.nvfp4_logprob_fwd(x[:, :vocab], tg, stats=st)
    want = new(rows, wide, dtype=dtype)
    B.nvfp4_logprob_bwd(x[:, :vocab], tg, st, want, w)
    assert bool((want[:, vocab:] == 0).all()) and bool(torch.isfinite(want).all())
    B.nvfp4_logprob_bwd(x[:, :vocab], tg, st, x, w)
    assert torch.equal(x, want)


# ------------------------------------------------------------------------------------------------- order ----
@pytest.mark.parametrize("n", [1, 5000, 40000])  # one launch for the order, a cluster, many launches
@pytest.mark.parametrize("reader", ["embedding", "norm"])
def test_a_table_is_read_to_its_end_before_it_is_zeroed(reader, n):
    """The reader is one of the library's own kernels, which lets the next launch begin early; the call behind it writes zeros beside its sort."""
    vocab, cols = 40000, 2048
    tokens, dout = torch.arange(n, device="cuda") % vocab, torch.ones((n, cols), dtype=BF16, device="cuda")
    ws = torch.empty(B.nvfp4_embedding_bwd_workspace_bytes(n, vocab, cols), dtype=torch.uint8, device="cuda")
    table, all_rows = torch.empty((vocab, cols), device="cuda"), torch.arange(vocab, device="cuda").flip(0)
    out, total = torch.empty((vocab, cols), device="cuda"), new(1, dtype=torch.float64)
    held, ws_n = B.grad_list([table]), torch.empty(B.nvfp4_grad_sq_norm_workspace_bytes(), dtype=torch.uint8, device="cuda")

    def both():
        if reader == "embedding":
            B.nvfp4_embedding_fwd(all_rows, table, out)
        else:
            B.nvfp4_grad_sq_norm(held, total, ws_n)
        B.nvfp4_embedding_bwd(tokens, dout, table, ws)

    def check():
        assert bool((out == 2.0).all()) if reader == "embedding" else float(total) == 4.0 * vocab * cols
        assert float(table.sum(dtype=torch.float64)) == float(n * cols)

    table.fill_(2.0)
    both()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(5):
        table.fill_(2.0)
        out.zero_()
        total.zero_()
        graph.replay()
        check()
        table.fill_(2.0)
        both()
        check()


def test_log_probabilities_on_two_streams():
    """Outputs of their own for each call, forward and backward in turn, beside another stream's."""
    def call(seed):
        z, tg, w = normal((9, 70000), seed, 3.0).cuda(), torch.arange(9, device="cuda") * 1000, normal((9,), seed + 1, 1.0, FP32).cuda()
        outs = [new(9), new(9), new(9, 2), new(9), new(9, 12, dtype=torch.int32), new(9, 12), torch.empty_like(z)]

        def run():
            B.nvfp4_logprob_fwd(z, tg, *outs[:6])
            B.nvfp4_logprob_bwd(z, tg, outs[2], outs[6], w, outs[3], w)

        return run, outs

    sets, want = [call(1), call(50)], []
    for run, outs in sets:
        run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(10):
        for _, outs in sets:
            for t in outs:
                t.zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for (run, _), stream in zip(sets, streams):
                with torch.cuda.stream(stream):
                    run()
        torch.cuda.synchronize()
        for (_, outs), right in zip(sets, want):
            assert all(torch.equal(a, b) for a, b in zip(outs, right))


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=str)
@pytest.mark.parametrize("scale", [0.25, 2.0 ** -30, 2.0 ** -60], ids=str)
@pytest.mark.parametrize("vocab", [9, 5001, 70000])
def test_logits_further_apart_than_the_largest_number(vocab, scale, dtype):
    """The difference of two logits is beyond binary32, its product with the scale is not."""
    x = torch.zeros((3, vocab), dtype=torch.float64)
    x[:, 0] = 3e38
    x[0, 1], x[1, vocab - 1], x[2, 1:] = -3e38, -2.5e38, -3.3e38
    x, targets = x.to(dtype), torch.tensor([1, vocab - 1, 4])
    xs = guarded(3, vocab, dtype, (vocab + 7) // 8 * 8, x)[0]
    lp, lse, entropy, ids, tops = new(3), new(3), new(3), new(3, 9, dtype=torch.int32), new(3, 9)
    B.nvfp4_logprob_fwd(xs, targets.cuda(), lp, lse, None, entropy, ids, tops, scale=scale)
    z = x.double() * scale
    want = z - z[:, :1]  # (the others' probabilities are 0 even at the smallest scale)
    assert torch.equal(ids.cpu().long(), R.top_of(x, 9))
    R.assert_within(lp, want.gather(1, targets[:, None])[:, 0], 4 * U * want.gather(1, targets[:, None])[:, 0].abs(), "logprob")
    R.assert_within(tops, want.gather(1, R.top_of(x, 9)), 4 * U * want.gather(1, R.top_of(x, 9)).abs(), "top_logprobs")
    R.assert_within(lse, z[:, 0], 4 * U * z[:, 0].abs(), "lse")
    assert bool((entropy == 0).all())
