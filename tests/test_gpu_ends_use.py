"""The operators at the ends of a training step as they are used: together with the layers, behind and beside other work, in graphs, and at sizes
beyond 2^31 elements."""
import math

import pytest
import torch

import ends_ref as R
from ends_ref import U, normal
from paper_2509_25149_b200 import binding as B
from paper_2509_25149_b200 import dp

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def scratch(nbytes):
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device="cuda")


def new(*shape, dtype=FP32):
    return torch.empty(shape, dtype=dtype, device="cuda")


# --------------------------------------------------------------------------------------------- a training step ----
V, VP, C, HQ, HK, D, N = 1003, 1008, 256, 3, 1, 64, 72  # vocabulary, the output layer's columns, width, heads, tokens


def attention(qk, v, causal):
    """One group of query heads over one key and value head."""
    q, k = qk[:, :HQ * D].unflatten(1, (HQ, D)), qk[:, HQ * D:]
    w = torch.einsum("thd,sd->hts", q, k) / math.sqrt(D)
    return torch.einsum("hts,sd->thd", torch.softmax(w.masked_fill(causal, -math.inf), 2), v).flatten(1)


def exact_step(p, tokens, targets, weight, bonus, positions, causal):
    """The model in 64 bits: embedding, norm, QKV product, head norms with rotation, attention, output product with residual, norm, output layer (tied to the
    embedding), weighted log probabilities and entropies."""
    there = (tokens >= 0) & (tokens < V)
    h0 = torch.where(there[:, None], p["table"][torch.where(there, tokens, 0)] * 16.0, 0.0)
    x = h0 * torch.rsqrt(h0.square().mean(1, keepdim=True) + 1e-5) * p["gain1"]
    qkv = x @ p["wqkv"].t()
    qk = R.heads_fwd(qkv[:, :(HQ + HK) * D], HQ, HK, p["gq"], p["gk"], 1e-5, p["freq"], positions, False)
    h1 = h0 + attention(qk, qkv[:, (HQ + HK) * D:], causal) @ p["wo"].t()
    y = h1 * torch.rsqrt(h1.square().mean(1, keepdim=True) + 1e-5) * p["gain2"]
    log_p = torch.log_softmax(y @ p["table"].t(), 1)
    ok = (targets >= 0) & (targets < V)
    lp = torch.where(ok, log_p.gather(1, torch.where(ok, targets, 0)[:, None])[:, 0], 0.0)
    entropy = -(log_p.exp() * log_p).sum(1)
    return lp, entropy, (lp * weight + entropy * bonus).sum()


def test_a_training_step_and_its_gradients():
    g = torch.Generator().manual_seed(1)
    tokens, targets = torch.randint(0, V, (N,), generator=g), torch.randint(0, V, (N,), generator=g)
    tokens[N - 5:], targets[N - 5:] = -1, -1  # a padded batch
    tokens[7] = tokens[11] = tokens[30] = 5
    positions = torch.cat([torch.arange(40), torch.arange(N - 40)])
    causal = torch.triu(torch.ones(N, N, dtype=torch.bool), 1)
    cpu = {"table": normal((V, C), 2, C ** -0.5), "wqkv": normal(((HQ + 2 * HK) * D, C), 3, C ** -0.5), "wo": normal((C, HQ * D), 4, (HQ * D) ** -0.5),
           "gain1": 1 + normal((C,), 5, 0.1, FP32), "gain2": 1 + normal((C,), 6, 0.1, FP32), "gq": 1 + normal((D,), 7, 0.1, FP32),
           "gk": 1 + normal((D,), 8, 0.1, FP32)}
    freq = torch.exp(-torch.arange(D // 2, dtype=torch.float64) * 0.2).float()
    weight, bonus = torch.where(targets >= 0, -1.0 / N, 0.0), torch.full((N,), -0.01 / N)

    # ---- the library's step
    d = {k: v.cuda() for k, v in cpu.items()}
    table = torch.zeros(VP, C, dtype=BF16, device="cuda")  # the output layer's rows come in multiples of 8
    table[:V] = d["table"]
    t, tg, pos, f = tokens.cuda(), targets.cuda(), positions.cuda(), freq.cuda()
    h0, x, rstd1 = new(N, C, dtype=BF16), new(N, C, dtype=BF16), new(N)
    B.nvfp4_embedding_fwd(t, table[:V], h0, 16.0)
    B.nvfp4_rmsnorm_fwd(h0, d["gain1"], 1e-5, x, rstd1)
    qkv = new(N, (HQ + 2 * HK) * D, dtype=BF16)
    B.nvfp4_linear_bf16_fwd(x, d["wqkv"], qkv)
    heads = qkv[:, :(HQ + HK) * D]
    qk = new(N, (HQ + HK) * D, dtype=BF16)
    B.nvfp4_headnorm_fwd(heads, HQ, HK, qk, d["gq"], d["gk"], 1e-5, f, pos)
    qk32, v32 = qk.float().requires_grad_(), qkv[:, (HQ + HK) * D:].float().requires_grad_()
    mixed32 = attention(qk32, v32, causal.cuda())
    mixed, h1, y, rstd2 = mixed32.detach().bfloat16(), new(N, C, dtype=BF16), new(N, C, dtype=BF16), new(N)
    B.nvfp4_gemm_bf16_epilogue(mixed, d["wo"], h1, residual=h0)
    B.nvfp4_rmsnorm_fwd(h1, d["gain2"], 1e-5, y, rstd2)
    logits = new(N, VP, dtype=BF16)
    B.nvfp4_linear_bf16_fwd(y, table, logits)
    lp, stats, entropy = new(N), new(N, 2), new(N)
    B.nvfp4_logprob_fwd(logits[:, :V], tg, lp, stats=stats, entropy=entropy)
    B.nvfp4_logprob_bwd(logits[:, :V], tg, stats, logits, weight.cuda(), entropy, bonus.cuda())  # in place, zeros in the spare columns
    dtable, dy = new(VP, C), new(N, C, dtype=BF16)
    B.nvfp4_linear_bf16_bwd(logits, y, table, C, dy, dtable)
    ws = scratch(max(B.nvfp4_rmsnorm_bwd_workspace_bytes(N, C), B.nvfp4_headnorm_bwd_workspace_bytes(N, HQ, HK, D),
                     B.nvfp4_embedding_bwd_workspace_bytes(N, V, C), B.nvfp4_grad_sq_norm_workspace_bytes()))
    grads = {"gain1": new(C), "gain2": new(C), "gq": new(D), "gk": new(D), "wqkv": new(*cpu["wqkv"].shape), "wo": new(*cpu["wo"].shape)}
    dh1 = new(N, C, dtype=BF16)
    B.nvfp4_rmsnorm_bwd(dy, h1, d["gain2"], rstd2, dh1, grads["gain2"], ws)
    dmixed = new(N, HQ * D, dtype=BF16)
    B.nvfp4_linear_bf16_bwd(dh1, mixed, d["wo"], HQ * D, dmixed, grads["wo"])
    mixed32.backward(dmixed.float())
    dqkv = new(N, (HQ + 2 * HK) * D, dtype=BF16)
    dqkv[:, (HQ + HK) * D:] = v32.grad
    B.nvfp4_headnorm_bwd(qk32.grad.bfloat16(), heads, HQ, HK, dqkv[:, :(HQ + HK) * D], d["gq"], d["gk"], 1e-5, grads["gq"], grads["gk"], ws, f, pos)
    dx = new(N, C, dtype=BF16)
    B.nvfp4_linear_bf16_bwd(dqkv, x, d["wqkv"], C, dx, grads["wqkv"])
    dh0 = new(N, C, dtype=BF16)
    B.nvfp4_rmsnorm_bwd(dx, h0, d["gain1"], rstd1, dh0, grads["gain1"], ws, residual_grad=dh1)
    B.nvfp4_embedding_bwd(t, dh0, dtable[:V], ws, 16.0, accumulate=True)  # beside the output layer's gradient
    assert bool((dtable[V:] == 0).all())
    grads["table"] = dtable[:V]
    B.nvfp4_device_status()

    # ---- the same in 64 bits
    p = {k: v.double().requires_grad_() for k, v in cpu.items()}
    p["freq"] = freq
    lp64, entropy64, loss = exact_step(p, tokens, targets, weight.double(), bonus.double(), positions, causal)
    loss.backward()
    rel = lambda got, want: float((got.detach().double().cpu() - want.detach()).norm() / want.detach().norm())
    # Ten or so roundings to bf16 in a row, each off by 2^-9 / sqrt(3) in the mean square, more where they meet in a difference
    assert rel(lp, lp64) < 0.02 and rel(entropy, entropy64) < 0.02
    for k, got in grads.items():
        assert rel(got, p[k].grad) < 0.04, k
    # and against differences of the exact loss along the table's gradient
    v = p["table"].grad / p["table"].grad.norm()
    with torch.no_grad():
        moved = lambda e: exact_step({**p, "table": p["table"] + e * v}, tokens, targets, weight.double(), bonus.double(), positions, causal)[2]
        along = float((moved(1e-5) - moved(-1e-5)) / 2e-5)
    assert abs(float((grads["table"].double().cpu() * v).sum()) - along) <= 0.04 * abs(along)

    # ---- clipped to half of their norm
    norm = math.sqrt(sum(float(gr.double().square().sum()) for gr in grads.values()))
    before = {k: gr.clone() for k, gr in grads.items()}
    clipper = dp.GradClipper(grads.values(), 0.5 * norm)
    for _ in range(2):
        s = clipper()
        assert abs(float(s[0]) / norm - 1) < 1e-5
        for k, gr in grads.items():
            R.assert_within(gr, 0.5 * before[k].double(), 2.0 ** -20 * before[k].double().abs() + 1e-40, k)
        for k, gr in grads.items():
            gr.copy_(before[k])


# -------------------------------------------------------------------------- behind, beside and inside other work ----
def calls(seed):
    """name -> (inputs that are overwritten, call, outputs) of every operator with workspaces of its own."""
    c = lambda t: t.cuda()
    x, dy = c(normal((130, 6 * 64), seed, 1.5)), c(normal((130, 6 * 64), seed + 1, 0.1))
    f, gain = c(torch.exp(-torch.arange(16).float())), c(1 + normal((64,), seed + 2, 0.1, FP32))
    y, dx, dgq, dgk = torch.empty_like(x), torch.empty_like(x), new(64), new(64)
    ws_h = scratch(B.nvfp4_headnorm_bwd_workspace_bytes(130, 4, 2, 64))
    t, rows = c(torch.randint(-1, 40, (700,), generator=torch.Generator().manual_seed(seed))), c(normal((700, 264), seed + 3))
    many, more = c(torch.randint(0, 40, (5000,), generator=torch.Generator().manual_seed(seed))), c(normal((5000, 264), seed + 3))
    table, emb, dtable, dmany = c(normal((40, 264), seed + 4)), new(700, 264, dtype=BF16), new(40, 264), new(40, 264)
    ws_e, ws_m = scratch(B.nvfp4_embedding_bwd_workspace_bytes(700, 40, 264)), scratch(B.nvfp4_embedding_bwd_workspace_bytes(5000, 40, 264))
    z = c(normal((9, 70000), seed + 5, 3.0))
    tg, lp, lse, st, en = c(torch.arange(9) * 1000), new(9), new(9), new(9, 2), new(9)
    ids, tops, dz, w = new(9, 12, dtype=torch.int32), new(9, 12), torch.empty_like(z), c(normal((9,), seed + 6, 1.0, FP32))
    grads = [c(normal((n,), seed + 7 + n % 5, 1.0, FP32 if n % 2 else BF16)) for n in (5, 40000, 123457)]
    outs = [torch.empty_like(g) for g in grads]
    total, stats, ws_g = new(1, dtype=torch.float64), new(2), scratch(B.nvfp4_grad_sq_norm_workspace_bytes())
    held = B.grad_list(grads, outs)

    def clip():
        B.nvfp4_grad_sq_norm(held, total, ws_g)
        B.nvfp4_grad_clip(held, total, 3.0, stats)

    return {
        "heads": ([x], lambda: B.nvfp4_headnorm_fwd(x, 4, 2, y, gain, gain, 1e-5, f), [y]),
        "heads_bwd": ([x, dy], lambda: B.nvfp4_headnorm_bwd(dy, x, 4, 2, dx, gain, gain, 1e-5, dgq, dgk, ws_h, f), [dx, dgq, dgk]),
        "embed": ([table], lambda: B.nvfp4_embedding_fwd(t, table, emb), [emb]),
        "embed_bwd": ([rows], lambda: B.nvfp4_embedding_bwd(t, rows, dtable, ws_e), [dtable]),
        "embed_bwd_many": ([more], lambda: B.nvfp4_embedding_bwd(many, more, dmany, ws_m), [dmany]),
        "logprob": ([z], lambda: B.nvfp4_logprob_fwd(z, tg, lp, lse, st, en, ids, tops), [lp, lse, st, en, ids, tops]),
        "logprob_bwd": ([z], lambda: (B.nvfp4_logprob_fwd(z, stats=st, entropy=en), B.nvfp4_logprob_bwd(z, tg, st, dz, w, en, w)), [dz]),
        "clip": (grads, clip, [total, stats, *outs]),
    }


NAMES = ["heads", "heads_bwd", "embed", "embed_bwd", "embed_bwd_many", "logprob", "logprob_bwd", "clip"]


def equal(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("name", NAMES)
def test_a_call_sees_what_precedes_it(name):
    """Inputs that a slow kernel, or a copy on another stream, has just written; directly and in a captured graph, twice in a row without a pause."""
    inputs, call, outputs = calls(1)[name]
    right = [t.clone() for t in inputs]
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]
    big, other = torch.randn((4096, 4096), device="cuda"), torch.cuda.Stream()

    def produce(beside):
        if beside:
            other.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(other):
                torch.mm(big, big)
                for t, r in zip(inputs, right):
                    t.copy_(r)
            torch.cuda.current_stream().wait_stream(other)
        else:
            torch.mm(big, big)
            for t, r in zip(inputs, right):
                torch.mul(r, 1, out=t)

    for _ in range(4):
        for beside in (False, True):
            for t in inputs:
                t.zero_()
            for t in outputs:
                t.zero_()
            produce(beside)
            call()
            call()
            for got, ref in zip(outputs, want):
                assert equal(got, ref), name
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        produce(False)
        call()
        call()
    for _ in range(4):
        for t in inputs:
            t.zero_()
        for t in outputs:
            t.zero_()
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip(outputs, want):
            assert equal(got, ref), name


def test_all_of_them_beside_each_other_on_two_streams():
    sets = [calls(1), calls(50)]
    want = []
    for s in sets:
        for name in NAMES:
            s[name][1]()
        torch.cuda.synchronize()
        want.append({name: [t.clone() for t in s[name][2]] for name in NAMES if name != "logprob"})
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for s in sets:
            for name in NAMES:
                for t in s[name][2]:
                    t.zero_()
        torch.cuda.synchronize()
        for k in range(len(NAMES)):
            for s, stream in zip(sets, streams):
                with torch.cuda.stream(stream):
                    s[NAMES[k]][1]()
        torch.cuda.synchronize()
        for s, w in zip(sets, want):
            for name, outs in w.items():
                assert all(equal(a, b) for a, b in zip(s[name][2], outs)), name


def test_the_table_is_not_written_before_its_readers_are_done():
    """A kernel that reads the table's gradient for long stands before the call that fills it with zeros."""
    V, C = 4000, 2048
    table, big = torch.ones(V, C, device="cuda"), torch.randn((4096, 4096), device="cuda")
    t, dout = torch.tensor([3], device="cuda"), torch.ones(1, C, dtype=BF16, device="cuda")
    ws = scratch(B.nvfp4_embedding_bwd_workspace_bytes(1, V, C))
    for _ in range(5):
        table.fill_(1.0)
        torch.mm(big, big)
        kept = [table.clone() for _ in range(3)]
        B.nvfp4_embedding_bwd(t, dout, table, ws)
        assert all(bool((k == 1).all()) for k in kept)
        assert bool((table[3] == 1).all()) and int(torch.count_nonzero(table)) == C


# ------------------------------------------------------------------------------------------- beyond 2^31 elements ----
def test_logits_beyond_2_31():
    rows, vocab = 17000, 131072
    z = torch.zeros(rows, vocab, dtype=BF16, device="cuda")
    g = torch.Generator("cuda").manual_seed(1)
    z[-3:] = torch.randn((3, vocab), generator=g, device="cuda").mul_(3).bfloat16()
    tg = torch.full((rows,), 131071, device="cuda")
    lp, st, en, ids = new(rows), new(rows, 2), new(rows), new(rows, 3, dtype=torch.int32)
    B.nvfp4_logprob_fwd(z, tg, lp, stats=st, entropy=en, top_ids=ids)
    ref = R.Softmax(z[-3:].cpu(), 1.0)
    R.assert_within(lp[-3:], ref.log_p[:, -1], ref.log_p_off()[:, -1], "logprob")
    assert torch.equal(ids[-3:].cpu().long(), R.top_of(z[-3:].cpu(), 3)) and ids[0].tolist() == [0, 1, 2]
    w = torch.full((rows,), 1.0, device="cuda")
    B.nvfp4_logprob_bwd(z, tg, st, z, w)
    grad, tol = ref.grad(tg[-3:].cpu(), w[-3:].cpu(), None, 1.0)
    R.assert_within(z[-3:], grad, tol + 2.0 ** -8 * (grad.abs() + tol) + 1e-38, "dlogits")
    assert abs(float(z[0, 0]) * vocab + 1) < 0.01 and float(z[0, -1]) > 0.99


def test_tables_beyond_2_31():
    vocab, cols, n = 1100000, 2048, 40
    t = torch.arange(n, device="cuda") % 3 + vocab - 3
    table = torch.zeros(vocab, cols, dtype=BF16, device="cuda")
    table[-3:] = normal((3, cols), 1).cuda()
    out = new(n, cols, dtype=BF16)
    B.nvfp4_embedding_fwd(t, table, out)
    assert torch.equal(out, table[t])
    del table
    dtable, dout = torch.ones(vocab, cols, device="cuda"), normal((n, cols), 2).cuda()
    B.nvfp4_embedding_bwd(t, dout, dtable, scratch(B.nvfp4_embedding_bwd_workspace_bytes(n, vocab, cols)))
    want = torch.zeros(3, cols, dtype=torch.float64).index_add_(0, (t - vocab + 3).cpu(), dout.double().cpu())
    R.assert_within(dtable[-3:], want, 20 * U * 14 * dout.double().abs().max().cpu(), "dtable")
    assert all(int(torch.count_nonzero(part)) == 0 for part in dtable[:-3].split(100000))


def test_heads_beyond_2_31():
    rows, ld = 350000, 6144 + 64
    x = torch.zeros(rows, ld, dtype=BF16, device="cuda")
    x[-2:] = normal((2, ld), 1).cuda()
    heads = x[:, :128 * 3]
    f = torch.exp(-torch.arange(64).float() * 0.1).cuda()
    want = R.heads_fwd(heads[-2:].double().cpu(), 2, 1, None, None, 1e-5, f.cpu(), torch.tensor([rows - 2, rows - 1]), False)
    B.nvfp4_headnorm_fwd(heads, 2, 1, heads, inv_freq=f)
    R.assert_within(heads[-2:], want, 2.0 ** -8 * want.abs() + 2.0 ** -17, "y")
    assert torch.equal(x[-2:, 384:].cpu(), normal((2, ld), 1)[:, 384:])


def test_gradients_beyond_2_31():
    n = (1 << 31) + 12345
    g = torch.full((n,), 0.5, dtype=BF16, device="cuda")
    g[-1] = 3.0
    total, stats = new(1, dtype=torch.float64), new(2)
    held = B.grad_list([g])
    B.nvfp4_grad_sq_norm(held, total, scratch(B.nvfp4_grad_sq_norm_workspace_bytes()))
    assert float(total) == 0.25 * (n - 1) + 9.0
    B.nvfp4_grad_clip(held, total, math.sqrt(float(total)) * 0.5, stats)
    assert abs(float(stats[1]) - 0.5) < 1e-6 and float(g[-1]) == 1.5 and bool((g[:-1] == 0.25).all())


# ------------------------------------------------------------------------------------------------- what is refused ----
@pytest.mark.parametrize("dtype", [BF16, FP32], ids=str)
@pytest.mark.parametrize("vocab", [1000, 9000, 40000])
def test_a_nan_logit_spoils_its_row_and_no_other(vocab, dtype):
    x = normal((6, vocab), 1, 2.0, dtype)
    x[2, vocab // 3] = math.nan
    x[4, vocab - 1] = -math.nan
    z, tg, w = x.cuda(), torch.arange(6, device="cuda"), torch.ones(6, device="cuda")
    lp, lse, st, en, dz = new(6), new(6), new(6, 2), new(6), torch.empty_like(z)
    ids, tops = new(6, 5, dtype=torch.int32), new(6, 5)
    B.nvfp4_logprob_fwd(z, tg, lp, lse, st, en, ids, tops)
    B.nvfp4_logprob_bwd(z, tg, st, dz, w, en, w)
    bad = torch.tensor([False, False, True, False, True, False], device="cuda")
    for t in (lp, lse, en):
        assert torch.equal(torch.isnan(t), bad)
    assert bool(torch.isnan(dz[bad]).all()) and bool(torch.isfinite(dz[~bad]).all()) and bool(torch.isfinite(tops[~bad]).all())
    assert int(ids.min()) >= 0 and int(ids.max()) < vocab
    good = x[[0, 1, 3, 5]]
    assert torch.equal(ids[~bad].cpu().long(), R.top_of(good, 5))


def test_the_bindings_refuse_what_they_cannot_take():
    x, f = torch.zeros(4, 384, dtype=BF16, device="cuda"), torch.ones(32, device="cuda")
    tok, tab = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(9, 384, device="cuda")
    z, lse, total = torch.zeros(4, 37, device="cuda"), new(4), new(1, dtype=torch.float64)
    ws = scratch(1 << 16)
    before = B.nvfp4_launch_count()
    for call in (lambda: B.nvfp4_headnorm_fwd(x, 4, 1, x),  # 384 columns are not five heads
                 lambda: B.nvfp4_headnorm_fwd(x.float(), 4, 2, x), lambda: B.nvfp4_headnorm_fwd(x, 4, 2, x.t()),
                 lambda: B.nvfp4_headnorm_fwd(x, 4, 2, x, inv_freq=f.cpu()), lambda: B.nvfp4_headnorm_fwd(x, 4, 2, x, positions=tok[:3]),
                 lambda: B.nvfp4_headnorm_fwd(x, 4, 2, x, gain_q=torch.ones(63, device="cuda")), lambda: B.nvfp4_headnorm_fwd(x.cpu(), 4, 2, x),
                 lambda: B.nvfp4_embedding_fwd(tok.float(), tab, x), lambda: B.nvfp4_embedding_fwd(tok, tab, x[:3]), lambda: B.nvfp4_embedding_fwd(tok[::2], tab, x[:2]),
                 lambda: B.nvfp4_embedding_bwd(tok, x, tab.bfloat16(), ws), lambda: B.nvfp4_embedding_bwd(tok, x, tab.cpu(), ws),
                 lambda: B.nvfp4_logprob_fwd(z.half(), lse=lse), lambda: B.nvfp4_logprob_fwd(z, lse=lse[:3]), lambda: B.nvfp4_logprob_fwd(z, tok[:2], lse),
                 lambda: B.nvfp4_logprob_fwd(z, top_ids=new(4, 3, dtype=torch.int64)), lambda: B.nvfp4_logprob_fwd(z, top_ids=new(4, 3, dtype=torch.int32), top_logprobs=new(4, 2)),
                 lambda: B.nvfp4_logprob_bwd(z, tok, new(4, 1), z, lse), lambda: B.nvfp4_logprob_bwd(z, tok, new(4, 2), z[:, :3].clone()[:2], lse),
                 lambda: B.grad_list([x.half()]), lambda: B.grad_list([x.t()]), lambda: B.grad_list([x, x.cpu()]), lambda: B.grad_list([x], [x[:2]]),
                 lambda: B.nvfp4_grad_sq_norm(B.grad_list([x]), new(1), ws)):
        with pytest.raises(AssertionError):
            call()
    for status, call in ((3, lambda: B.nvfp4_logprob_fwd(z, lse=lse)),  # rows 37 elements apart
                         (2, lambda: B.nvfp4_headnorm_fwd(x, 4, 2, x, inv_freq=torch.ones(36, device="cuda"))), (2, lambda: B.nvfp4_headnorm_fwd(x, 1, 0, x)),
                         (4, lambda: B.nvfp4_headnorm_fwd(x, 4, 2, x, eps=0.0)), (5, lambda: B.nvfp4_embedding_bwd(tok, x, tab, ws[:256])),
                         (2, lambda: B.nvfp4_logprob_fwd(new(4, 40), top_ids=new(4, 33, dtype=torch.int32))), (5, lambda: B.nvfp4_grad_sq_norm(B.grad_list([x]), total, ws[:256])),
                         (4, lambda: B.nvfp4_grad_clip(B.grad_list([x]), total, 0.0))):
        with pytest.raises(B.NVFP4Error) as e:
            call()
        assert e.value.status == status
    assert B.nvfp4_launch_count() == before
