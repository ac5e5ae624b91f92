"""GPU parity of the 8-bit matrices: quantisation, the norm that leaves in 8 bits, the product; and a vocabulary head as a whole.

A product of e4m3 numbers is exact in fp32; K of them are summed in fp32 by the tensor cores.  An addition there may truncate (one ulp,
2^-23, instead of half of one): |error| <= K 2^-23 sum |a w| at worst, and the rounding to the output's type."""
import numpy as np
import pytest
import torch

import _cat

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _ctx():
    from paper_2411_11925_b200 import api
    return api.Context(0)


def _empty(rows, K):
    from paper_2411_11925_b200 import api
    d, s = api.quant_empty(rows, K, "cuda")
    d.fill_(0x33); s.fill_(9)            # what was there before
    return d, s


def _quant(ctx, x):
    q = _empty(*x.shape)
    ctx.csd_quantize(x.shape[0], x.shape[1], x, *q)
    return q


def _check_bytes(q, y, slack, K):
    """y: float64 rows before quantisation, off by at most a factor 1 +- slack: the block's scale and each value's half step."""
    data, scale = (t.cpu().numpy() for t in q)
    rows, ld = data.shape
    full = np.zeros((rows, ld))
    full[:, :K] = y
    assert np.all(data[:, K:] & 0x7F == 0) and np.all(scale[:, ld // 128:] == 127)
    want = np.minimum(_cat.scale_bytes(full * (1 - slack)), _cat.scale_bytes(full * (1 + slack))), np.maximum(_cat.scale_bytes(full * (1 - slack)), _cat.scale_bytes(full * (1 + slack)))
    sc = scale[:, : ld // 128]
    assert np.all((sc >= want[0]) & (sc <= want[1]))
    got = _cat.dequantize(data, scale)
    unit = np.repeat(2.0 ** (sc.astype(np.float64) - 127), 128, axis=1)
    # half a step: 2^-4 of the value, 2^-10 of the scale below e4m3's normal range
    assert np.all(np.abs(got - full) <= np.maximum(2.0 ** -4 * np.abs(full), 2.0 ** -10 * unit) * (1 + 1e-9) + 2 * slack * np.abs(full))


@pytest.mark.parametrize("rows,K,dtype", [(1, 1, "f32"), (3, 127, "bf16"), (2, 128, "f16"), (5, 129, "f32"), (4, 1000, "bf16"), (7, 4096, "f16"), (3, 5000, "bf16"),
                                          (2, 8193, "f32"), (2, 40000, "bf16"), (300, 640, "f32")])
def test_quantize(rows, K, dtype):
    rng = np.random.default_rng(K)
    x = rng.standard_normal((rows, K)) * 10.0 ** rng.integers(-6, 6, (rows, 1))
    x[:, ::113] *= 40
    x[0, : min(K, 128)] = 0.0
    t = torch.from_numpy(x).cuda().to(TYPES[dtype]).clamp(-6e4, 6e4)
    ctx = _ctx()
    q = _quant(ctx, t)
    ctx.sync()
    _check_bytes(q, t.double().cpu().numpy(), 0.0, K)
    # what fits exactly comes back exactly: numbers of four significant bits in a narrow range, and powers of two of any size
    y = torch.from_numpy(rng.integers(-15, 16, (rows, K)).astype(np.float32) * 2.0 ** rng.integers(-10, 10, (rows, 1)).astype(np.float32)).cuda().to(TYPES[dtype])
    q = _quant(ctx, y)
    ctx.sync()
    np.testing.assert_array_equal(_cat.dequantize(q[0].cpu().numpy(), q[1].cpu().numpy())[:, :K], y.double().cpu().numpy())
    ctx.close()


def test_quantize_extremes():
    x = torch.zeros(8, 256, device="cuda")
    x[0, 3] = float("nan"); x[0, 200] = 5.0
    x[1, 130] = float("inf"); x[1, 5] = -448.0
    x[2] = 3.4e38; x[2, 128:] = -1e-44
    x[3, 0] = 448.0; x[3, 1] = 449.0 / 2 ** 9; x[3, 128] = 448.00003
    x[4, 0] = 2.0 ** -126; x[4, 128] = 1.5
    x[5, :128] = 2.0 ** -149
    ctx = _ctx()
    q = _quant(ctx, x)
    ctx.sync()
    s = q[1].cpu().numpy()
    got = _cat.dequantize(q[0].cpu().numpy(), s)
    assert s[0, 0] == 255 and np.all(np.isnan(got[0, :128])) and got[0, 200] == 5.0
    assert s[1, 1] == 255 and got[1, 5] == -448.0 and s[1, 0] == 127
    assert np.all(np.abs(got[2, :128] / 3.4e38 - 1) <= 2.0 ** -4) and np.all(np.isfinite(got[2]))
    assert s[3, 0] == 127 and s[3, 1] == 128 and got[3, 0] == 448.0
    assert np.all(got[6] == 0) and s[6, 0] == 127
    ctx.close()


@pytest.mark.parametrize("rows,K,dtype,res,weight", [(1, 1, "f32", True, True), (3, 130, "bf16", True, True), (1, 4096, "bf16", True, True), (5, 1000, "f16", False, True),
                                                     (9, 5000, "bf16", True, False), (3, 9000, "f32", True, True), (2, 33000, "f16", True, True), (600, 777, "f32", False, False)])
def test_norm_quantize(rows, K, dtype, res, weight):
    rng = np.random.default_rng(K + rows)
    t = lambda a: torch.from_numpy(a.astype(np.float32)).cuda().to(TYPES[dtype])  # noqa: E731
    x, r, w = t(rng.standard_normal((rows, K)) * 3), t(rng.standard_normal((rows, K))), t(1 + 0.2 * rng.standard_normal(K))
    h = x.double() + r.double() if res else x.double()
    y = h / torch.sqrt((h ** 2).mean(1, keepdim=True) + 1e-6) * (w.double() if weight else 1.0)
    ctx = _ctx()
    total = torch.full_like(x, 5.0)
    q = _empty(rows, K)
    ctx.csd_norm_quantize(rows, K, x, r if res else None, w if weight else None, 1e-6, total, *q)
    ctx.sync()
    # fp32: K terms in a thread and a tree of 10 levels for the mean (half of it under the root), its root, three products
    slack = 2.0 ** -24 * ((K / 256 + 20) / 2 + 2 + 2 + 3)
    _check_bytes(q, y.cpu().numpy(), slack, K)
    exact = h.float() if dtype == "f32" else (x.float() + (r.float() if res else 0.0)).to(TYPES[dtype])
    assert torch.equal(total, exact.to(TYPES[dtype]))
    # without the sum; in place; strided rows of a wider matrix: the same bytes
    q2 = _empty(rows, K)
    ctx.csd_norm_quantize(rows, K, x, r if res else None, w if weight else None, 1e-6, None, *q2)
    wide = torch.zeros(rows, K + 3, device="cuda", dtype=TYPES[dtype]); wide[:, 2:2 + K] = x
    q3 = _empty(rows, K)
    ctx.csd_norm_quantize(rows, K, wide[:, 2:2 + K], r if res else None, w if weight else None, 1e-6, wide[:, 2:2 + K], *q3)
    ctx.sync()
    for z in (q2, q3):
        assert torch.equal(z[0], q[0]) and torch.equal(z[1], q[1])
    assert torch.equal(wide[:, 2:2 + K], total) and torch.all(wide[:, :2] == 0) and torch.all(wide[:, 2 + K:] == 0)
    if res:
        q4, stream = _empty(rows, K), r.clone()
        ctx.csd_norm_quantize(rows, K, x, stream, w if weight else None, 1e-6, stream, *q4)
        ctx.sync()
        assert torch.equal(stream, total) and torch.equal(q4[0], q[0])
    ctx.close()


@pytest.mark.parametrize("M,N,K,dtype", [(1, 1, 1, "f32"), (1, 128, 128, "f32"), (3, 200, 130, "bf16"), (31, 129, 511, "f16"), (32, 1000, 512, "f32"), (33, 257, 513, "bf16"),
                                         (64, 384, 1024, "f32"), (65, 500, 700, "f16"), (129, 130, 256, "f32"), (224, 640, 2048, "bf16"), (225, 333, 1537, "f32"),
                                         (576, 2000, 640, "f16"), (1000, 1111, 3000, "f32"), (5, 40000, 256, "bf16"), (2, 777, 9000, "f32")])
def test_product(M, N, K, dtype):
    rng = np.random.default_rng(M + N + K)
    ctx = _ctx()
    # rows and blocks of very different sizes: a scale applied to the wrong row, block or operand shows
    a = torch.from_numpy((rng.standard_normal((M, K)) * 2.0 ** rng.integers(-3, 4, (M, 1)) * 2.0 ** np.repeat(rng.integers(-4, 5, (1, (K + 127) // 128)), 128, 1)[:, :K]).astype(np.float32)).cuda()
    w = torch.from_numpy((rng.standard_normal((N, K)) * K ** -0.5 * 2.0 ** rng.integers(-3, 4, (N, 1))).astype(np.float32)).cuda()
    qa, qw = _quant(ctx, a), _quant(ctx, w)
    out = torch.full((M + 1, N + 5), 3.0, device="cuda", dtype=TYPES[dtype])
    ctx.csd_quant_matmul(M, N, K, qa, qw, out[:M, 2:2 + N])
    ctx.sync()
    fa = torch.from_numpy(_cat.dequantize(*(t.cpu().numpy() for t in qa))).cuda()
    fw = torch.from_numpy(_cat.dequantize(*(t.cpu().numpy() for t in qw))).cuda()
    want, size = fa @ fw.T, fa.abs() @ fw.abs().T
    err = (out[:M, 2:2 + N].double() - want).abs()
    tol = K * 2.0 ** -23 * size + HALF_STEP[dtype] * want.abs() + (2.0 ** -25 if dtype == "f16" else 0.0)
    assert torch.all(err <= tol), float((err / tol.clamp(min=1e-300)).max())
    print("product", (M, N, K, dtype), "relative 2-norm error", float(err.norm() / want.norm()), "of the bound", float((err / tol.clamp(min=1e-300)).max()))
    # nothing beside the output's rows and columns is written
    out[:M, 2:2 + N] = 3.0
    assert torch.all(out == 3.0)
    # twice the same bits, into a dense output too
    dense = torch.zeros(M, N, device="cuda", dtype=TYPES[dtype]); again = torch.zeros_like(dense)
    ctx.csd_quant_matmul(M, N, K, qa, qw, dense)
    ctx.csd_quant_matmul(M, N, K, qa, qw, again)
    ctx.sync()
    assert torch.equal(dense, again) and torch.all((dense.double() - want).abs() <= tol)
    ctx.close()


def test_nan_blocks_stay_in_their_rows():
    ctx = _ctx()
    a = torch.randn(40, 300, device="cuda"); w = torch.randn(260, 300, device="cuda")
    a[7, 140] = float("nan"); w[129, 299] = float("inf")
    out = torch.zeros(40, 260, device="cuda")
    ctx.csd_quant_matmul(40, 260, 300, _quant(ctx, a), _quant(ctx, w), out)
    ctx.sync()
    bad = torch.isnan(out)
    assert torch.all(bad[7]) and torch.all(bad[:, 129])
    bad[7] = False; bad[:, 129] = False
    assert not bad.any()
    ctx.close()


def test_bad_arguments_are_refused():
    from paper_2411_11925_b200 import api
    ctx = _ctx()
    x = torch.zeros(2, 200, device="cuda")
    q, w = _empty(2, 200), _empty(5, 200)
    out = torch.zeros(2, 5, device="cuda")
    cases = [
        (ValueError, lambda: ctx.csd_quantize(2, 201, x, *q)), (ValueError, lambda: ctx.csd_quantize(3, 200, x, *q)),
        (ValueError, lambda: ctx.csd_quantize(2, 200, x.cpu(), *q)), (ValueError, lambda: ctx.csd_quantize(2, 200, x, q[0][:1], q[1])),
        (ValueError, lambda: ctx.csd_quantize(2, 200, x.double(), *q)), (ValueError, lambda: ctx.csd_quantize(2, 200, x, q[0], q[1].int())),
        (ValueError, lambda: ctx.csd_norm_quantize(2, 200, x, x.half(), None, 1e-6, None, *q)),
        (ValueError, lambda: ctx.csd_norm_quantize(2, 200, x, None, x[0, :100], 1e-6, None, *q)),
        (-1, lambda: ctx.csd_norm_quantize(2, 200, x, None, None, -1.0, None, *q)),
        (-1, lambda: ctx.csd_norm_quantize(2, 200, x, None, None, 1e-6, x[:1].expand(2, -1), *q)),     # rows of the sum overlap
        (ValueError, lambda: ctx.csd_quant_matmul(3, 5, 200, q, w, out)), (ValueError, lambda: ctx.csd_quant_matmul(2, 6, 200, q, w, out)),
        (TypeError, lambda: ctx.csd_quant_matmul(2, 5, 200, q[0], w, out)),
        (-1, lambda: ctx.csd_quant_matmul(2, 5, 200, q, w, out[:1].expand(2, -1))),
        (-1, lambda: ctx.csd_quant_matmul(0, 5, 200, q, w, out)),
        (-1, lambda: ctx.csd_quant_matmul(1, 5, 200, (q[0].view(-1)[3:259], q[1]), w, out)),           # not 16-byte aligned
        (-3, lambda: ctx.csd_quantize(1, (1 << 20) + 1, torch.zeros(1, (1 << 20) + 1, device="cuda"), *q)),
    ]
    for i, (want, call) in enumerate(cases):
        if isinstance(want, int):
            with pytest.raises(api.CsdError) as e:
                call()
            assert e.value.code == want, i
        else:
            with pytest.raises(want):
                call()
    ctx.sync()
    ctx.close()


def test_sums_in_place_keep_their_rows():
    """In place of an input only row on row: at another stride a row's sum would land where another block still reads."""
    from paper_2411_11925_b200 import api
    ctx = _ctx()
    buf = torch.zeros(4 * 256, device="cuda")
    x, tight = buf.view(4, 256)[:, :200], buf[:800].view(4, 200)
    one = buf[:200].expand(4, -1)
    q = _empty(4, 200)
    other = torch.zeros(4, 200, device="cuda")
    for a, r, s in ((x, None, tight), (one, None, tight), (other, x, tight), (other, one, tight)):
        with pytest.raises(api.CsdError) as e:
            ctx.csd_norm_quantize(4, 200, a, r, None, 1e-6, s, *q)
        assert e.value.code == -1
    ctx.csd_norm_quantize(4, 200, x, other, None, 1e-6, x, *q)
    ctx.csd_norm_quantize(1, 200, x[:1], other[:1], None, 1e-6, tight[:1], q[0][:1], q[1][:1])   # a single row has no stride
    ctx.sync()
    ctx.close()


def test_rows_beyond_32_bits():
    """Row strides of 2^31 elements of inputs, of the sum and of a product's output."""
    rows, K, N = 3, 200, 70
    rng = np.random.default_rng(5)
    ctx = _ctx()
    x = torch.from_numpy(rng.standard_normal((rows, K)).astype(np.float32)).cuda().bfloat16()
    far = torch.empty((rows - 1 << 31) + 256, dtype=torch.bfloat16, device="cuda")
    fx, fo = far.as_strided((rows, K), (1 << 31, 1)), far.as_strided((rows, N), (1 << 31, 1))
    fx.copy_(x)
    near, other, sums = _empty(rows, K), _empty(rows, K), torch.empty_like(x)
    ctx.csd_norm_quantize(rows, K, x, x, None, 1e-6, sums, *near)
    ctx.csd_norm_quantize(rows, K, fx, x, None, 1e-6, fx, *other)
    w = _quant(ctx, torch.from_numpy(rng.standard_normal((N, K)).astype(np.float32)).cuda())
    ctx.sync()
    assert torch.equal(near[0], other[0]) and torch.equal(near[1], other[1]) and torch.equal(fx, sums)
    out = torch.empty(rows, N, dtype=torch.bfloat16, device="cuda")
    ctx.csd_quant_matmul(rows, N, K, near, w, out)
    ctx.csd_quant_matmul(rows, N, K, near, w, fo)
    ctx.sync()
    assert torch.equal(out, fo)
    ctx.close()


def test_vocabulary_head_round_captured():
    """Norm, product, sampling, verification and resampling as one program, captured into a graph and replayed on new hidden states;
    each stage is checked against the plain form on the stage's own inputs."""
    B, gamma, V, K = 6, 4, 2500, 700
    rows = gamma + 1
    rng = np.random.default_rng(4)
    from paper_2411_11925_b200 import api
    s = torch.cuda.Stream()
    ctx = api.Context(0, s)
    f = lambda *sh: torch.from_numpy(rng.standard_normal(sh).astype(np.float32)).cuda()  # noqa: E731
    u = lambda *sh: torch.from_numpy(rng.random(sh).astype(np.float32)).cuda()  # noqa: E731
    wn, W, Wq = (1 + 0.1 * f(K)).bfloat16(), f(V, K) * 3 * K ** -0.5, None
    hp, hq, rp = f(B * rows, K).bfloat16(), f(B * gamma, K).bfloat16(), f(B * rows, K).bfloat16()
    ap, aq, w = _empty(B * rows, K), _empty(B * gamma, K), _empty(V, K)
    lp, lq = torch.zeros(B * rows, V, device="cuda"), torch.zeros(B * gamma, V, device="cuda", dtype=torch.bfloat16)
    tok = torch.zeros(B, gamma, dtype=torch.int32, device="cuda")
    dq, dp = torch.zeros(B * gamma, 5, dtype=torch.float64, device="cuda"), torch.zeros(B * rows, 5, dtype=torch.float64, device="cuda")
    lr, total = torch.zeros(B, gamma, device="cuda"), torch.zeros_like(hp)
    n, mask, new = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3))
    u0, ua, ub = u(B * gamma), u(B, gamma), u(B)
    params = (torch.full((B * rows,), 0.8, device="cuda"), torch.full((B * rows,), 60, dtype=torch.int32, device="cuda"), torch.full((B * rows,), 0.95, device="cuda"), None)
    ctx.csd_quantize(V, K, W, *w)

    def go():
        ctx.csd_norm_quantize(B * gamma, K, hq, None, wn, 1e-6, None, *aq)
        ctx.csd_quant_matmul(B * gamma, V, K, aq, w, lq)
        ctx.csd_cat_draft_sample(B * gamma, V, lq, None, u0, tok, None, dq)
        ctx.csd_norm_quantize(B * rows, K, hp, rp, wn, 1e-6, total, *ap)
        ctx.csd_quant_matmul(B * rows, V, K, ap, w, lp)
        ctx.csd_cat_verify(B, gamma, rows, V, lq, dq, lp, params, tok, ua, dp, lr, n, mask)
        ctx.csd_cat_resample(B, gamma, rows, V, lq, dq, lp, dp, n, ub, new)

    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        go()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            go()
    for k in range(2):
        with torch.cuda.stream(s):
            base = f(B, rows, K)
            hp.copy_(base.reshape(-1, K)); hq.copy_((base + rp.float().view(B, rows, K))[:, :gamma].reshape(-1, K) + 0.2 * f(B * gamma, K))
            g.replay()
        torch.cuda.synchronize()
        ctx.sync()
        fw = torch.from_numpy(_cat.dequantize(*(t.cpu().numpy() for t in w))).cuda()
        for a, l, half in ((aq, lq, 2.0 ** -8), (ap, lp, 2.0 ** -24)):
            fa = torch.from_numpy(_cat.dequantize(*(t.cpu().numpy() for t in a))).cuda()
            want = fa @ fw.T
            assert torch.all((l.double() - want).abs() <= K * 2.0 ** -23 * (fa.abs() @ fw.abs().T) + half * want.abs())
        assert torch.equal(total, (hp.float() + rp.float()).bfloat16())
        nl, hl, hlp = n.cpu().numpy(), lq.float().cpu().numpy(), lp.cpu().numpy().reshape(B, rows, V)
        fs = dict(temperature=float(np.float32(0.8)), top_k=60, top_p=float(np.float32(0.95)))
        for b in range(B):
            ok = []
            for i in range(gamma):
                pq, _ = _cat.probabilities(hl[b * gamma + i])
                pp, _ = _cat.probabilities(hlp[b, i], **fs)
                x, near = _cat.pick(pq, float(u0[b * gamma + i]))
                assert int(tok[b, i]) == x or near < 1e-10
                x = int(tok[b, i])
                ok.append(pp[x] > 0 and np.log(float(ua[b, i])) <= np.log(pp[x]) - np.log(pq[x]))
            assert nl[b] == (ok + [False]).index(False)
            j = int(nl[b])
            r, _ = _cat.probabilities(hlp[b, j], **fs)
            if j < gamma:
                r = np.maximum(r - _cat.probabilities(hl[b * gamma + j])[0], 0.0)
            x, near = _cat.pick(r, float(ub[b]))
            assert int(new[b]) == x or near < 1e-10 / r.sum()
    del g
    ctx.close()


@pytest.mark.parametrize("M,N,K,dtype", [(230, 30001, 700, "bf16"), (96, 60001, 300, "f32"), (70, 20000, 1200, "f16")])
def test_products_of_several_tiles_a_pair_of_blocks(M, N, K, dtype):
    """More tiles than pairs of blocks: accumulators, stages and groups of scales are used again, at odd numbers of column blocks too."""
    g = torch.Generator("cuda").manual_seed(K)
    ctx = _ctx()
    a = torch.randn(M, K, generator=g, device="cuda") * torch.exp2(torch.randint(-3, 4, (M, 1), generator=g, device="cuda").float())
    w = torch.randn(N, K, generator=g, device="cuda") * K ** -0.5 * torch.exp2(torch.randint(-3, 4, (N, 1), generator=g, device="cuda").float())
    a[:, 128:256] *= 64
    qa, qw = _quant(ctx, a), _quant(ctx, w)
    out = torch.full((M, N + 3), 3.0, device="cuda", dtype=TYPES[dtype])
    ctx.csd_quant_matmul(M, N, K, qa, qw, out[:, 1:1 + N])
    again = torch.zeros(M, N, device="cuda", dtype=TYPES[dtype])
    ctx.csd_quant_matmul(M, N, K, qa, qw, again)
    ctx.sync()
    fa, fw = (torch.from_numpy(_cat.dequantize(*(t.cpu().numpy() for t in q))).cuda() for q in (qa, qw))
    want, size = fa @ fw.T, fa.abs() @ fw.abs().T
    tol = K * 2.0 ** -23 * size + HALF_STEP[dtype] * want.abs() + (2.0 ** -25 if dtype == "f16" else 0.0)
    assert torch.all((out[:, 1:1 + N].double() - want).abs() <= tol) and torch.equal(out[:, 1:1 + N], again)
    assert torch.all(out[:, 0] == 3) and torch.all(out[:, 1 + N:] == 3)
    ctx.close()


def test_quantize_below_the_least_scale():
    """Blocks whose scale would lie below 2^-127 get that: the least normal number is 2 in it, the least subnormal one rounds to 0."""
    x = torch.zeros(2, 256, device="cuda")
    x[0, 0] = 2.0 ** -126; x[0, 128] = 1.5
    x[1, :128] = 2.0 ** -149
    ctx = _ctx()
    q = _quant(ctx, x)
    ctx.sync()
    s = q[1].cpu().numpy()
    got = _cat.dequantize(q[0].cpu().numpy(), s)
    assert s[0, 0] == 0 and s[0, 1] == 119 and s[1, 0] == 0
    assert got[0, 0] == 2.0 ** -126 and got[0, 128] == 1.5 and np.all(got[0, 1:128] == 0) and np.all(got[1] == 0)
    ctx.close()


@pytest.mark.parametrize("rows,K,dtype,off", [(3, 8200, "bf16", 0), (3, 9001, "bf16", 1), (5, 16384, "f16", 0), (2, 12003, "f16", 3), (300, 8193, "bf16", 0), (2, 16392, "bf16", 0), (3, 20001, "f32", 1)])
def test_norm_of_wide_rows_in_place(rows, K, dtype, off):
    """Rows of four pieces a thread, and rows that are read twice, on and off 16 bytes; the sum replaces the residual, or x, or both where they are one array."""
    rng = np.random.default_rng(K)
    t = lambda *sh: torch.from_numpy(rng.standard_normal(sh).astype(np.float32)).cuda().to(TYPES[dtype])  # noqa: E731
    w = t(K)
    ctx = _ctx()
    for which in ("residual", "x", "both"):
        bx, br = t(rows, K + 8), t(rows, K + 8)
        x = bx[:, off:off + K]
        r = x if which == "both" else br[:, off:off + K]
        keep = bx.clone(), br.clone()
        h = x.double() + r.double()
        rounded = (x.float() + r.float()).to(TYPES[dtype])
        y = h / torch.sqrt((h ** 2).mean(1, keepdim=True) + 1e-5) * w.double()
        q = _empty(rows, K)
        ctx.csd_norm_quantize(rows, K, x, r, w, 1e-5, x if which == "x" else r, *q)
        ctx.sync()
        # fp32: as in test_norm_quantize, rows read twice have K / 1024 more terms in a thread
        _check_bytes(q, y.cpu().numpy(), 2.0 ** -24 * ((K / 256 + 20) / 2 + 2 + 2 + 3), K)
        assert torch.equal(x if which != "residual" else r, rounded)
        for buf, was in zip((bx, br), keep):                   # nothing beside the rows, and not the other array
            same = buf == was
            same[:, off:off + K] |= torch.equal(buf[:, off:off + K], rounded)
            assert torch.all(same)
    ctx.close()
