"""GPU parity of the categorical-head calls against plain 64-bit forms (tests/_cat.py).

What may differ: a token whose border lies within the error of the weights' sums.  A weight is 2^-44 of the largest, rounded
(2^-45), from an exponential with a relative error below 2^-42; over V tokens a prefix, relative to a sum of at least 1, is off by less than
2^-41 + V 2^-45.  Log probabilities are differences of numbers of that error, returned in float32 (2^-24)."""
import numpy as np
import pytest
import torch

import _cat

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _ctx():
    from paper_2411_11925_b200 import api
    return api.Context(0)


def _border(V):
    return 2.0 ** -41 + V * 2.0 ** -45


def _dev(a, t=None):
    x = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return x if t is None else x.to(t)


def _f32(x):
    return x.float().cpu().numpy()


def _sample(ctx, logits, u, params, R, V, dist=True):
    tok = torch.full((R,), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((R,), 7.0, device="cuda")
    d = torch.zeros(R, 5, dtype=torch.float64, device="cuda") if dist else None
    ctx.csd_cat_draft_sample(R, V, logits, params, u, tok, lp, d)
    ctx.sync()
    return tok.cpu().numpy(), lp.cpu().numpy(), d.cpu().numpy() if dist else None


def _check_rows(l32, tok, lp, d, u, fs):
    V = l32.shape[1]
    for r in range(l32.shape[0]):
        order, logp, row = _cat.kept(l32[r], **fs[r])
        assert d[r, 3] == row[3], (r, d[r], row, fs[r])
        assert d[r, 1] == row[1] and d[r, 2] == row[2] and d[r, 4] == row[4], (r, d[r], row)
        if order.size == 0:
            assert tok[r] == -1 and lp[r] == -np.inf and d[r, 0] == -np.inf
            continue
        assert abs(d[r, 0] - row[0]) <= 2 * _border(V) + 4e-16 * (abs(row[0]) + abs(row[1])), (r, d[r], row)
        w = np.zeros(V)
        w[order] = np.exp(logp)
        want, near = _cat.pick(w, u[r])
        assert tok[r] == want or near < _border(V), (r, tok[r], want, near, fs[r])
        got = logp[np.flatnonzero(order == tok[r])[0]]
        assert abs(lp[r] - got) <= 2.0 ** -24 * abs(got) + 2 * _border(V) + 1e-15 * (abs(row[0]) + abs(row[1])), (r, lp[r], got)


def _filters(rng, R, mixed):
    one = lambda: dict(temperature=float(np.float32(rng.uniform(0.5, 1.5))), top_k=int(rng.choice([0, 1, 5, 50, 700])),  # noqa: E731
                       top_p=float(np.float32(rng.choice([1.0, 0.3, 0.9, 0.999]))), min_p=float(np.float32(rng.choice([0.0, 0.0, 0.02, 1.0]))))
    return [one() for _ in range(R)] if mixed else [dict() for _ in range(R)]


def _params(fs):
    if not fs[0]:
        return None
    col = lambda k, t: torch.tensor([f.get(k, {"temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0}[k]) for f in fs], dtype=t, device="cuda")  # noqa: E731
    return (col("temperature", torch.float32), col("top_k", torch.int32), col("top_p", torch.float32), col("min_p", torch.float32))


@pytest.mark.parametrize("R,V,dtype,mixed", [(1, 1, "f32", False), (3, 2, "f32", True), (6, 7, "bf16", True), (5, 127, "f16", True),
                                             (40, 1000, "f32", True), (7, 1000, "f32", False), (300, 4099, "bf16", True), (1, 16384, "f32", True),
                                             (37, 50003, "bf16", True), (2, 131072, "f16", False), (2, 131072, "f32", True), (1, 300001, "f32", True)])
def test_samples_match_the_plain_form(R, V, dtype, mixed):
    rng = np.random.default_rng(V + R)
    x = rng.standard_normal((R, V)) * 2.0
    x[:, rng.integers(0, V, 5)] += rng.uniform(0, 9, 5)
    x[rng.random((R, V)) < 0.1] = -np.inf
    x[rng.random((R, V)) < 0.01] = np.nan
    u = rng.random(R).astype(np.float32).clip(1e-7, 1 - 1e-7)
    fs = _filters(rng, R, mixed)
    ctx = _ctx()
    l = _dev(x.astype(np.float32), TYPES[dtype])
    tok, lp, d = _sample(ctx, l, _dev(u), _params(fs), R, V)
    _check_rows(_f32(l), tok, lp, d, u, fs)
    # the summaries alone are the same ones
    d2 = torch.zeros(R, 5, dtype=torch.float64, device="cuda")
    ctx.csd_cat_filter(R, V, l, _params(fs), d2)
    ctx.sync()
    np.testing.assert_array_equal(d2.cpu().numpy(), d)
    ctx.close()


@pytest.mark.parametrize("V,k,p", [(131072, 0, 0.95), (131072, 20000, 0.9), (60001, 5000, 1.0), (60001, 3000, 0.5), (9000, 0, 0.999), (131072, 0, 1.0)])
def test_wide_filters(V, k, p):
    """More tokens kept than a block sorts: flat rows, and rows of equals where only the index decides."""
    rng = np.random.default_rng(k + V)
    x = np.stack([rng.standard_normal(V), 1.5 * rng.standard_normal(V), np.zeros(V), np.round(2 * rng.standard_normal(V)), 1e-3 * rng.standard_normal(V),
                  1e6 + rng.standard_normal(V)]).astype(np.float32)
    u = rng.random(6).astype(np.float32)
    fs = [dict(temperature=1.0, top_k=k, top_p=float(np.float32(p)), min_p=mp) for mp in (0.0, float(np.float32(0.01)), 0.0, 0.0, 0.0, 0.0)]
    ctx = _ctx()
    tok, lp, d = _sample(ctx, _dev(x), _dev(u), _params(fs), 6, V)
    for r in range(6):
        order, logp, row = _cat.kept(x[r], **fs[r])
        if r != 2:   # (in a row of equals every border is a multiple of 1 / V: the count may be one off where p V is whole)
            assert d[r, 3] == row[3], (r, d[r], row)
    _check_rows(x[[0, 1, 3, 4, 5]], tok[[0, 1, 3, 4, 5]], lp[[0, 1, 3, 4, 5]], d[[0, 1, 3, 4, 5]], u[[0, 1, 3, 4, 5]], [fs[i] for i in (0, 1, 3, 4, 5)])
    n = _cat.kept(x[2], **fs[2])[2][3]
    assert abs(d[2, 3] - n) <= 1 and d[2, 2] == d[2, 3] - 1 and d[2, 1] == 0.0   # the first of the equals
    assert 0 <= tok[2] < d[2, 3]
    ctx.close()


def test_bins_that_end_near_zero_and_small_top_k_with_infinities():
    """Borders between bins, and the least logit of min-p, next to zero, where fp32 numbers lie dense; a threshold for a small top-k where a
    logit is infinite or the logits span the whole range."""
    rng = np.random.default_rng(77)
    V = 4000
    x = (1.5 * rng.standard_normal((40, V))).astype(np.float32)
    x[5, 7] = np.inf
    x[6, :10] = 3e38; x[6, 10:20] = -3e38
    x[7] = np.float32(3.912023); x[7, 5:] = 1e-20 * rng.standard_normal(V - 5)
    fs = [dict(temperature=1.0, top_k=int(rng.choice([3, 2000, 0, 255])), top_p=float(np.float32(rng.choice([0.95, 1.0]))), min_p=float(np.float32(rng.choice([0.0, 0.02])))) for _ in range(40)]
    for i in (5, 6):
        fs[i].update(top_k=17)
    fs[7].update(top_k=0, min_p=float(np.float32(0.02)))
    u = rng.random(40).astype(np.float32)
    ctx = _ctx()
    for R in (40, 400):     # few rows and many
        xs, us, ff = np.tile(x, (R // 40, 1)), np.tile(u, R // 40), fs * (R // 40)
        tok, lp, d = _sample(ctx, _dev(xs), _dev(us), _params(ff), R, V)
        _check_rows(xs[:40], tok[:40], lp[:40], d[:40], us[:40], ff[:40])
        assert np.array_equal(tok, np.tile(tok[:40], R // 40)) and np.array_equal(d, np.tile(d[:40], (R // 40, 1)))
    ctx.close()


def test_rows_that_decide_by_rules():
    """Masks and extremes: nothing left, one left, the type's lowest value, infinities, zero temperature, filters at their ends."""
    V = 600
    low = np.finfo(np.float32).min
    rng = np.random.default_rng(3)
    x = rng.standard_normal((16, V)).astype(np.float32)
    x[0] = -np.inf
    x[1] = np.nan
    x[2] = -np.inf; x[2, 417] = -50.0
    x[3] = low                                   # every token equally hopeless: uniform
    x[4] = low; x[4, 99] = 3.0
    x[5, 7] = np.inf                             # as the largest finite number
    x[6, 3] = x[6, 400] = 99.0                   # equals at the top, zero temperature: the first
    x[7, 5] = x[7, 450] = 50.0                   # top_k 1 among equals
    x[8] = -np.inf; x[8, [3, 90, 200]] = [0.0, -0.0, 0.0]   # zeros of both signs are equals
    x[9, ::2] = -np.inf                          # top_k beyond what is left
    x[13] = 1e38; x[13, 50] = 3e38               # scaled beyond the range
    fs = [dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0) for _ in range(16)]
    fs[3].update(temperature=0.5, top_p=0.5)
    fs[4].update(temperature=0.25)
    fs[6].update(temperature=0.0)
    fs[7].update(top_k=1)
    fs[8].update(top_k=2)
    fs[9].update(top_k=500)
    fs[10].update(top_p=0.0)
    fs[11].update(top_p=-1.0, top_k=3)
    fs[12].update(min_p=1.0)
    fs[13].update(temperature=0.1)
    fs[14].update(min_p=5.0)
    fs[15].update(top_k=-4, top_p=1.5, min_p=-1.0)
    u = np.full(16, 0.75, np.float32)
    ctx = _ctx()
    tok, lp, d = _sample(ctx, _dev(x), _dev(u), _params(fs), 16, V)
    _check_rows(x, tok, lp, d, u, fs)
    assert tok[0] == -1 and tok[1] == -1 and tok[2] == 417 and tok[4] == 99 and tok[5] == 7 and tok[6] == 3 and tok[7] == 5
    assert tok[8] == 90 and d[8, 3] == 2 and d[8, 2] == 90
    assert d[3, 3] == V // 2 and d[10, 3] == 1 and d[11, 3] == 1
    # the ends of the uniform
    for v in (1e-30, np.float32(1 - 2.0 ** -24), 0.0, 1.0):
        tok, lp, d = _sample(ctx, _dev(x), _dev(np.full(16, v, np.float32)), _params(fs), 16, V)
        assert np.all(tok[2:] >= 0) and np.all(np.isfinite(lp[2:]))
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_row_strides_and_alignments(dtype):
    """Rows in a wider matrix, at every offset from a 16-byte border, behind one another with a gap, and one row for all."""
    rng = np.random.default_rng(9)
    ctx = _ctx()
    wide = _dev(rng.standard_normal((5, 3011)).astype(np.float32) * 3, TYPES[dtype])
    u = rng.random(5).astype(np.float32)
    fs = _filters(rng, 5, True)
    for off in range(0, 9):
        for V in (1, 5, 1999):
            l = wide[:, off:off + V]
            tok, lp, d = _sample(ctx, l, _dev(u), _params(fs), 5, V)
            _check_rows(_f32(l), tok, lp, d, u, fs)
    same = wide[2:3, 11:2000].expand(5, -1)
    tok, lp, d = _sample(ctx, same, _dev(u), _params(fs), 5, 1989)
    _check_rows(_f32(same), tok, lp, d, u, fs)
    ctx.close()


def test_results_do_not_depend_on_how_a_row_is_spread():
    """One row alone (several blocks) and the same row in a large batch (one block) give the same bits."""
    rng = np.random.default_rng(21)
    V = 33001
    x = (rng.standard_normal((1, V)) * 1.5).astype(np.float32)
    u = np.array([0.613], np.float32)
    ctx = _ctx()
    for k, p in ((0, 1.0), (0, 0.9), (40, 1.0), (4000, 0.8)):
        f = dict(temperature=0.9, top_k=k, top_p=p, min_p=0.0)
        one = _sample(ctx, _dev(x), _dev(u), _params([f]), 1, V)
        for R in (60, 400):
            many = _sample(ctx, _dev(x).expand(R, -1), _dev(np.repeat(u, R)), _params([f] * R), R, V)
            for a, b in zip(one, many):
                assert np.all(b == a[0]), (k, p, R)
    ctx.close()


def _round(ctx, x_q, x_p, fq, fp, u0, u, w, B, gamma, rows, V):
    R = B * gamma
    tok = torch.zeros(B, gamma, dtype=torch.int32, device="cuda")
    dq = torch.zeros(R, 5, dtype=torch.float64, device="cuda"); dp = torch.zeros(B * rows, 5, dtype=torch.float64, device="cuda")
    lr = torch.zeros(B, gamma, device="cuda")
    n, mask, new = (torch.full((B,), 9, dtype=torch.int32, device="cuda") for _ in range(3))
    ctx.csd_cat_draft_sample(R, V, x_q, fq, u0, tok, None, dq)
    ctx.csd_cat_verify(B, gamma, rows, V, x_q, dq, x_p, fp, tok, u, dp, lr, n, mask)
    ctx.csd_cat_resample(B, gamma, rows, V, x_q, dq, x_p, dp, n, w, new)
    return tok, dq, dp, lr, n, mask, new


@pytest.mark.parametrize("B,gamma,bonus,V,tq,tp,close", [(1, 1, True, 3, "f32", "f32", 0.5), (9, 5, True, 1000, "bf16", "f32", 0.3),
                                                         (4, 32, False, 5003, "f16", "bf16", 0.2), (33, 4, True, 777, "f32", "f16", 1.0),
                                                         (170, 2, True, 20011, "bf16", "bf16", 0.4), (2, 3, False, 131072, "f32", "f32", 0.1)])
def test_round_matches_the_plain_form(B, gamma, bonus, V, tq, tp, close):
    rng = np.random.default_rng(V + B)
    rows = gamma + int(bonus)
    p = rng.standard_normal((B, rows, V)) * 2
    q = p[:, :gamma] + close * rng.standard_normal((B, gamma, V))
    p[rng.random(p.shape) < 0.05] = -np.inf
    x_q, x_p = _dev(q.reshape(-1, V).astype(np.float32), TYPES[tq]), _dev(p.reshape(-1, V).astype(np.float32), TYPES[tp])
    fq, fp = _filters(rng, B * gamma, True), _filters(rng, B * rows, True)
    u0, u, w = (rng.random(s).astype(np.float32).clip(1e-6, 1 - 1e-6) for s in (B * gamma, (B, gamma), B))
    ctx = _ctx()
    tok, dq, dp, lr, n, mask, new = [t.cpu().numpy() for t in _round(ctx, x_q, x_p, _params(fq), _params(fp), _dev(u0), _dev(u), _dev(w), B, gamma, rows, V)]
    ctx.sync()
    hq, hp = _f32(x_q), _f32(x_p).reshape(B, rows, V)
    for b in range(B):
        ok = []
        for i in range(gamma):
            pq, rq = _cat.probabilities(hq[b * gamma + i], **fq[b * gamma + i])
            pp, rp = _cat.probabilities(hp[b, i], **fp[b * rows + i])
            assert np.all(dq[b * gamma + i, 1:4] == rq[1:4]) and np.all(dp[b * rows + i, 1:4] == rp[1:4])
            x = tok[b, i]
            assert pq[x] > 0
            with np.errstate(divide="ignore"):
                want = np.log(pp[x]) - np.log(pq[x]) if pp[x] > 0 else -np.inf
            if np.isinf(want):
                assert lr[b, i] == want
            else:
                assert abs(lr[b, i] - want) <= 2.0 ** -24 * abs(want) + 4 * _border(V) + 1e-14 * 30
            ok.append(np.log(np.float64(u[b, i])) <= want)
        assert (int(mask[b]) & 0xFFFFFFFF) == sum(int(o) << i for i, o in enumerate(ok)), (b, ok)
        assert n[b] == (ok + [False]).index(False)
        j = int(n[b])
        if j == rows:
            assert new[b] == -1
            continue
        pp, _ = _cat.probabilities(hp[b, j], **fp[b * rows + j])
        r = pp
        if j < gamma:
            pq, _ = _cat.probabilities(hq[b * gamma + j], **fq[b * gamma + j])
            r = np.maximum(pp - pq, 0.0)
            r = r if r.sum() > 0 else pp
        want, near = _cat.pick(r, w[b])
        # probabilities to 2^-42, rounded to 2^-53: relative to what is left of p
        assert new[b] == want or near < (2.0 ** -41 + V * 2.0 ** -53) / r.sum(), (b, new[b], want, near)
    ctx.close()


def test_equal_models_accept_everything_and_rejections_without_residual_fall_back_to_p():
    B, gamma, V = 5, 4, 3001
    rng = np.random.default_rng(2)
    p = (rng.standard_normal((B * (gamma + 1), V)) * 2).astype(np.float32)
    x_p = _dev(p)
    x_q = _dev(p.reshape(B, gamma + 1, V)[:, :gamma].reshape(-1, V))
    u0, u, w = (rng.random(s).astype(np.float32) for s in (B * gamma, (B, gamma), B))
    ctx = _ctx()
    tok, dq, dp, lr, n, mask, new = _round(ctx, x_q, x_p, None, None, _dev(u0), _dev(u), _dev(w), B, gamma, gamma + 1, V)
    ctx.sync()
    assert torch.all(lr == 0) and torch.all(n == gamma) and torch.all(mask == 15)
    for b in range(B):
        pr, _ = _cat.probabilities(p.reshape(B, gamma + 1, V)[b, gamma])
        assert new[b] == _cat.pick(pr, w[b])[0]
    # a caller who rejects all the same: max(0, p - q) is nothing, the token is drawn from p
    zero = torch.zeros_like(n)
    ctx.csd_cat_resample(B, gamma, gamma + 1, V, x_q, dq, x_p, dp, zero, _dev(w), new)
    ctx.sync()
    for b in range(B):
        pr, _ = _cat.probabilities(p.reshape(B, gamma + 1, V)[b, 0])
        assert new[b] == _cat.pick(pr, w[b])[0]
    # counts out of range, and tokens that are none, are answered and touch nothing else
    n[:] = torch.tensor([-1, gamma + 1, 1 << 30, -(1 << 31), gamma], device="cuda", dtype=torch.int32)
    ctx.csd_cat_resample(B, gamma, gamma + 1, V, x_q, dq, x_p, dp, n, _dev(w), new)
    tok[0] = torch.tensor([-1, V, 1 << 30, -(1 << 31)], device="cuda", dtype=torch.int32)
    ctx.csd_cat_verify(B, gamma, gamma + 1, V, x_q, dq, x_p, None, tok, _dev(u), dp, lr, n, mask)
    ctx.sync()
    assert new[:4].tolist() == [-1] * 4 and int(new[4]) >= 0
    assert torch.all(lr[0] == -np.inf) and int(n[0]) == 0 and torch.all(n[1:] == gamma)
    ctx.close()


def test_masked_target_rows_reject_and_give_no_token():
    B, gamma, V = 3, 2, 500
    rng = np.random.default_rng(8)
    p = rng.standard_normal((B, gamma, V)).astype(np.float32)
    p[1] = -np.inf
    q = rng.standard_normal((B * gamma, V)).astype(np.float32)
    q[4] = np.nan                                    # a draft without a token
    u = np.full((B, gamma), 1e-6, np.float32)
    ctx = _ctx()
    tok, dq, dp, lr, n, mask, new = _round(ctx, _dev(q), _dev(p.reshape(-1, V)), None, None, _dev(np.full(6, 0.5, np.float32)), _dev(u),
                                           _dev(np.full(3, 0.5, np.float32)), B, gamma, gamma, V)
    ctx.sync()
    assert n.tolist() == [2, 0, 0] and new.tolist()[:2] == [-1, -1] and tok[2, 0] == -1 and lr[2, 0] == -np.inf
    pr, _ = _cat.probabilities(p[2, 0])
    assert int(new[2]) == _cat.pick(pr, 0.5)[0]      # nothing to take away from p
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_resampling_one_sequence_from_rows_off_16_bytes(dtype):
    """A single sequence still reads a later row: its last tokens, which a row that starts on 16 bytes would not push into one more piece."""
    gamma, V = 2, 4096
    wide = torch.zeros(gamma + 1, V + 1, dtype=TYPES[dtype], device="cuda")
    p = wide[:, :V]
    p[:, V - 1] = 20.0
    q = torch.zeros(gamma, V, dtype=TYPES[dtype], device="cuda")
    ctx = _ctx()
    dq, dp = (torch.zeros(r, 5, dtype=torch.float64, device="cuda") for r in (gamma, gamma + 1))
    ctx.csd_cat_filter(gamma, V, q, None, dq)
    ctx.csd_cat_filter(gamma + 1, V, p, None, dp)
    for n in range(gamma + 1):
        new = torch.full((1,), 9, dtype=torch.int32, device="cuda")
        ctx.csd_cat_resample(1, gamma, gamma + 1, V, q, dq, p, dp, torch.full_like(new, n), torch.full((1,), 0.5, device="cuda"), new)
        ctx.sync()
        assert int(new) == V - 1, n      # exp(20) against V - 1 ones: all but 1e-5 of the distribution
    ctx.close()


def test_summaries_that_give_no_weight_give_no_token():
    V = 700
    ctx = _ctx()
    q, p = torch.zeros(1, V, device="cuda"), torch.zeros(2, V, device="cuda")
    dq, dp = (torch.zeros(r, 5, dtype=torch.float64, device="cuda") for r in (1, 2))
    ctx.csd_cat_filter(1, V, q, None, dq)
    ctx.csd_cat_filter(2, V, p, None, dp)
    dp[:, 0] = 1000.0                                # a normaliser that is not these rows'
    for n in (0, 1):
        new = torch.full((1,), 9, dtype=torch.int32, device="cuda")
        ctx.csd_cat_resample(1, 1, 2, V, q, dq, p, dp, torch.full_like(new, n), torch.full((1,), 0.5, device="cuda"), new)
        ctx.sync()
        assert int(new) == -1, n
    ctx.close()


@pytest.mark.parametrize("R,V,k", [(3, 1000, 40), (3, 60001, 0)])
def test_rows_beyond_32_bits(R, V, k):
    """Row strides of 2^31 elements: the last row starts 2^32 elements and 2^33 bytes behind the first."""
    rng = np.random.default_rng(V)
    ctx = _ctx()
    x = _dev((rng.standard_normal((R, V)) * 3).astype(np.float32), torch.bfloat16)
    far = torch.empty((R - 1 << 31) + V, dtype=torch.bfloat16, device="cuda").as_strided((R, V), (1 << 31, 1))
    far.copy_(x)
    u = rng.random(R).astype(np.float32)
    fs = [dict(temperature=0.8, top_k=k, top_p=0.9, min_p=0.0)] * R
    a, b = _sample(ctx, far, _dev(u), _params(fs), R, V), _sample(ctx, x, _dev(u), _params(fs), R, V)
    for i, j in zip(a, b):
        assert np.array_equal(i, j)
    q, new = torch.zeros(2, V, device="cuda"), [torch.full((1,), 9, dtype=torch.int32, device="cuda") for _ in range(2)]
    dq, dp = torch.zeros(2, 5, dtype=torch.float64, device="cuda"), _dev(a[2])
    ctx.csd_cat_filter(2, V, q, None, dq)
    for l, o in ((far, new[0]), (x, new[1])):
        ctx.csd_cat_resample(1, 2, 3, V, q, dq, l, dp, torch.full_like(o, 2), torch.full((1,), 0.3, device="cuda"), o)
    ctx.sync()
    assert int(new[0]) == int(new[1]) >= 0
    ctx.close()


def test_bad_arguments_are_refused():
    from paper_2411_11925_b200 import api
    ctx = _ctx()
    l = torch.zeros(2, 8, device="cuda"); u = torch.zeros(2, device="cuda"); t = torch.zeros(2, dtype=torch.int32, device="cuda")
    d = torch.zeros(2, 5, dtype=torch.float64, device="cuda")
    cases = [
        (ValueError, lambda: ctx.csd_cat_filter(2, 9, l, None, d)),                     # rows of another length
        (ValueError, lambda: ctx.csd_cat_filter(3, 8, l, None, d)),                     # too few rows
        (ValueError, lambda: ctx.csd_cat_filter(2, 8, l.double(), None, d)),
        (ValueError, lambda: ctx.csd_cat_filter(2, 8, l.cpu(), None, d)),
        (ValueError, lambda: ctx.csd_cat_filter(2, 8, torch.zeros(8, 2, device="cuda").T, None, d)),
        (ValueError, lambda: ctx.csd_cat_filter(2, 8, l, None, d[:1])),
        (ValueError, lambda: ctx.csd_cat_filter(2, 8, l, None, d.float())),
        (TypeError, lambda: ctx.csd_cat_filter(2, 8, l, (u, t, u), d)),
        (ValueError, lambda: ctx.csd_cat_filter(2, 8, l, (u, u, u, u), d)),             # top_k is int32
        (TypeError, lambda: ctx.csd_cat_filter(2, 8, None, None, d)),
        (ValueError, lambda: ctx.csd_cat_draft_sample(2, 8, l, None, u[:1], t)),
        (TypeError, lambda: ctx.csd_cat_draft_sample(2, 8, l, None, u, None)),
        (-1, lambda: ctx.csd_cat_filter(0, 8, l, None, d)),
        (-3, lambda: ctx.csd_cat_filter(1, (1 << 19) + 1, torch.zeros(1, (1 << 19) + 1, device="cuda"), None, d)),
        (-2, lambda: ctx.csd_cat_verify(1, 1, 3, 8, l, d, torch.zeros(3, 8, device="cuda"), None, t, u, torch.zeros(3, 5, dtype=torch.float64, device="cuda"), u, t)),
        (-3, lambda: ctx.csd_cat_verify(1, 33, 33, 8, torch.zeros(33, 8, device="cuda"), torch.zeros(33, 5, dtype=torch.float64, device="cuda"),
                                        torch.zeros(33, 8, device="cuda"), None, torch.zeros(33, dtype=torch.int32, device="cuda"), torch.zeros(33, device="cuda"),
                                        torch.zeros(33, 5, dtype=torch.float64, device="cuda"), torch.zeros(33, device="cuda"), t)),
    ]
    for want, call in cases:
        if isinstance(want, int):
            with pytest.raises(api.CsdError) as e:
                call()
            assert e.value.code == want
        else:
            with pytest.raises(want):
                call()
    ctx.sync()
    ctx.close()


def test_captured_calls_replay_on_new_inputs_and_other_streams():
    B, gamma, V = 6, 3, 9001
    rng = np.random.default_rng(31)
    s = torch.cuda.Stream()
    from paper_2411_11925_b200 import api
    ctx, plain = api.Context(0, s), _ctx()
    x_q, x_p = torch.zeros(B * gamma, V, device="cuda"), torch.zeros(B * (gamma + 1), V, device="cuda")
    u0, u, w = (_dev(rng.random(n).astype(np.float32)) for n in (B * gamma, (B, gamma), B))
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        _round(ctx, x_q, x_p, None, None, u0, u, w, B, gamma, gamma + 1, V)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            out = _round(ctx, x_q, x_p, None, None, u0, u, w, B, gamma, gamma + 1, V)
    for k in range(3):
        p = rng.standard_normal((B, gamma + 1, V)).astype(np.float32)
        with torch.cuda.stream(s):
            x_p.copy_(_dev(p.reshape(-1, V)))
            x_q.copy_(_dev((p[:, :gamma] + 0.3 * rng.standard_normal((B, gamma, V))).reshape(-1, V).astype(np.float32)))
            g.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        want = _round(plain, x_q, x_p, None, None, u0, u, w, B, gamma, gamma + 1, V)
        plain.sync()
        for a, b in zip(got, want):
            assert torch.equal(a, b), k
    ctx.sync()
    del g
    ctx.close(); plain.close()


@pytest.mark.parametrize("R,V,dtype", [(5, 1000, "f32"), (40, 30001, "bf16"), (300, 700, "f16"), (3, 100003, "f32"), (400, 33001, "f32")])
def test_a_certain_token_has_log_probability_zero(R, V, dtype):
    """One token kept, whatever leaves it alone and however large its logit: the normaliser is its scaled logit.  By one block a row (the first
    three) and by the three kernels, with several parts a row and with one."""
    rng = np.random.default_rng(V)
    m = rng.uniform(-40, 60, R)
    m[::3] = rng.uniform(60, 3000, m[::3].size)
    x = (m[:, None] - rng.uniform(0.5, 20, (R, V))).astype(np.float32)
    at = rng.integers(0, V, R)
    x[np.arange(R), at] = m
    l = _dev(x, TYPES[dtype])
    x = _f32(l)
    u = _dev(rng.random(R).astype(np.float32))
    T = float(np.float32(0.7))
    one = np.full_like(x, -np.inf)
    one[np.arange(R), at] = x[np.arange(R), at]
    ctx = _ctx()
    for rows, f in ((x, dict(temperature=T, top_k=1)), (x, dict(temperature=0.0)), (x, dict(temperature=T, top_p=1e-6)), (x, dict(temperature=T, top_k=1, top_p=0.5)),
                    (x, dict(temperature=T, min_p=1.0)), (one, dict(temperature=T)), (one, dict(temperature=T, top_p=0.9)), (one, dict(temperature=T, top_k=5))):
        l = _dev(rows, TYPES[dtype])
        tok, lp, d = _sample(ctx, l, u, _params([f] * R), R, V)
        alone = d[:, 3] == 1          # (16-bit logits may have equals at the top)
        assert alone.sum() > R / 2
        assert np.all(lp[alone] == 0) and np.all(d[alone, 0] == d[alone, 1]), f
        assert np.all(lp <= 0) and np.all(tok[alone] == d[alone, 2])
    ctx.close()


def test_certain_drafts_of_certain_targets_are_accepted():
    """Greedy rows of p and q that keep the same token: the ratio is 0, and a uniform of 1 accepts."""
    B, gamma, V = 50, 4, 2000
    rng = np.random.default_rng(6)
    p = (rng.standard_normal((B * gamma, V)) + rng.uniform(-40, 60, (B * gamma, 1))).astype(np.float32)
    q = (p + rng.uniform(-3, 3, (B * gamma, 1))).astype(np.float32)
    at = rng.integers(0, V, B * gamma)
    for x in (p, q):
        x[np.arange(B * gamma), at] += 10
    greedy = _params([dict(temperature=0.0)] * (B * gamma))
    u1 = torch.ones(B, gamma, device="cuda")
    ctx = _ctx()
    tok, dq, dp, lr, n, mask, new = _round(ctx, _dev(q), _dev(p), greedy, greedy, u1.view(-1), u1, u1[:, 0].contiguous(), B, gamma, gamma, V)
    ctx.sync()
    assert np.array_equal(tok.cpu().numpy().ravel(), at) and torch.all(lr == 0) and torch.all(n == gamma) and torch.all(mask == 15)
    ctx.close()


def _check_kept(x, d, fs):
    for r in range(x.shape[0]):
        row = _cat.kept(x[r], **fs[r])[2]
        assert np.array_equal(d[r, 1:], row[1:]), (r, d[r], row, fs[r])


@pytest.mark.parametrize("R,V", [(1, 1000), (60, 2000), (400, 33001), (3, 100003)])
def test_equals_by_scaling_go_by_index(R, V):
    """Different logits that scale to the same number are equals, of which the index decides: neighbours in the last bit, products beyond the range, and
    products that are zero or next to it.  By one block a row (the first two), by the three kernels with one part a row and with several."""
    ctx = _ctx()
    u = _dev(np.full(R, 0.5, np.float32))
    a, b = np.float32(1.75 + 2.0 ** -23), np.float32(1.75 + 2.0 ** -22)
    assert a < b and a * np.float32(1.25) == b * np.float32(1.25)
    near, big, flat = np.zeros((R, V), np.float32), np.zeros((R, V), np.float32), np.zeros((R, V), np.float32)
    near[:, 0] = a; near[:, 4] = b
    near[:, V - 1] = b; near[:, V // 2] = a
    big[:, 3] = 4.0; big[:, 7] = 5.0; big[:, 9] = -np.inf; big[:, V - 5] = 6.0
    flat[:, 1] = -np.inf; flat[:, 5:90] = 3.0; flat[:, V - 2] = 2.0
    small = np.tile(np.float32(1.0) + np.arange(V, dtype=np.float32) * np.float32(2.0 ** -23), (R, 1))
    for x, T in ((near, 0.8), (big, 2e-38), (flat, np.inf), (small, 1e38)):
        for k in (1, 2, 3, 20, 200):
            for p in (1.0, 0.7):
                fs = [dict(temperature=float(np.float32(T)), top_k=k, top_p=p)] * R
                _, _, d = _sample(ctx, _dev(x), u, _params(fs), R, V)
                _check_kept(x[:1], d[:1], fs)
                assert np.array_equal(d, np.repeat(d[:1], R, 0))
    ctx.close()


@pytest.mark.parametrize("R,V", [(400, 33001), (2, 100003), (30, 20000)])
def test_small_top_k_of_large_logits(R, V):
    """Logits of a million and a few units: many neighbours in the last bit, at temperatures that make equals of some of them."""
    rng = np.random.default_rng(R)
    ctx = _ctx()
    for k in (1, 20, 50):
        x = (1e6 + rng.standard_normal((R, V))).astype(np.float32)
        fs = [dict(temperature=float(np.float32(rng.uniform(0.5, 1.3))), top_k=k) for _ in range(R)]
        _, _, d = _sample(ctx, _dev(x), _dev(np.full(R, 0.5, np.float32)), _params(fs), R, V)
        _check_kept(x, d, fs)
    ctx.close()


def test_a_uniform_of_zero_accepts_no_token_that_is_not_kept():
    """log 0 is no larger than a ratio of -inf: tokens that p masks or filters out, and numbers that are no tokens, are rejected all the same."""
    B, gamma, V = 6, 3, 300
    rng = np.random.default_rng(13)
    p = rng.standard_normal((B, gamma, V)).astype(np.float32)
    tok = np.tile(np.array([5, 6, 7], np.int32), (B, 1))
    p[:, :, 5:8] = 4.0
    p[0, 1, 6] = -np.inf                      # masked by p
    p[1, 0, 5] = -9.0                         # not among p's top-k
    tok[2, 0], tok[3, 2], tok[4, 1] = -1, V, np.iinfo(np.int32).min
    q = _dev(rng.standard_normal((B * gamma, V)).astype(np.float32))
    f = lambda rows: _params([dict(top_k=9)] * rows)  # noqa: E731
    dq, dp = (torch.zeros(B * gamma, 5, dtype=torch.float64, device="cuda") for _ in range(2))
    lr, n, mask = torch.zeros(B, gamma, device="cuda"), torch.full((B,), 9, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    ctx = _ctx()
    ctx.csd_cat_filter(B * gamma, V, q, None, dq)
    for u in (0.0, 2.0 ** -149):
        ctx.csd_cat_verify(B, gamma, gamma, V, q, dq, _dev(p.reshape(-1, V)), f(B * gamma), _dev(tok), torch.full((B, gamma), u, device="cuda"), dp, lr, n, mask)
        ctx.sync()
        assert n.tolist() == [1, 0, 0, 2, 1, 3] and mask.tolist() == [5, 6, 6, 3, 5, 7], u
    ctx.close()


@pytest.mark.parametrize("V,tq,tp", [(701, "f32", "f32"), (5003, "bf16", "bf16"), (5003, "bf16", "f32")])
def test_summaries_of_other_rows_give_some_token_or_none(V, tq, tp):
    """Whatever the summaries say, the answer is -1 or a token, nothing outside the rows is read (they end where their memory does), and the next call is
    right: normalisers far off either way, cuts of -inf, numbers that are none."""
    B, gamma, nan, inf = 4, 2, np.nan, np.inf
    rng = np.random.default_rng(V)
    p, q = (_dev((rng.standard_normal((r, V)) * 2).astype(np.float32), TYPES[t]) for r, t in ((B * (gamma + 1), tp), (B * gamma, tq)))
    dp, dq = torch.zeros(B * (gamma + 1), 5, dtype=torch.float64, device="cuda"), torch.zeros(B * gamma, 5, dtype=torch.float64, device="cuda")
    n = torch.tensor([0, 1, 2, 0], dtype=torch.int32, device="cuda")
    w = _dev(np.array([0.1, 0.5, 0.999, 1.0], np.float32))
    ctx = _ctx()
    ctx.csd_cat_filter(B * gamma, V, q, None, dq)
    ctx.csd_cat_filter(B * (gamma + 1), V, p, None, dp)
    right, new = torch.full((B,), 9, dtype=torch.int32, device="cuda"), torch.full((B,), 9, dtype=torch.int32, device="cuda")
    ctx.csd_cat_resample(B, gamma, gamma + 1, V, q, dq, p, dp, n, w, right)
    ctx.sync()
    for col, values in ((0, (-30.0, -3000.0, -4000.0, -5000.0, -1e30, -1e300, 1e30, nan, inf, -inf)), (1, (-inf, nan, inf, -1e300)),
                        (2, (nan, 1e300, -1e300, inf)), (3, (nan, 1e300, inf)), (4, (nan, inf, -1.0, 0.0, 1e30, -1e300))):
        for v in values:
            for both in (False, True):
                fp, fq = dp.clone(), dq.clone()
                fp[:, col] = v
                if both:
                    fq[:, col] = v
                if col == 2:
                    fp[:, 1] = -inf; fq[:, 1] = -inf
                new.fill_(V)
                ctx.csd_cat_resample(B, gamma, gamma + 1, V, q, fq, p, fp, n, w, new)
                ctx.sync()
                assert torch.all((new >= -1) & (new < V)), (col, v, both, new)
    # a cut of -inf with every index is no cut
    fp = dp.clone(); fp[:, 1] = -inf; fp[:, 2] = 1e9
    ctx.csd_cat_resample(B, gamma, gamma + 1, V, q, dq, p, fp, n, w, new)
    ctx.sync()
    assert torch.equal(new, right)
    ctx.csd_cat_resample(B, gamma, gamma + 1, V, q, dq, p, dp, n, w, new)
    ctx.sync()
    assert torch.equal(new, right)
    ctx.close()


@pytest.mark.parametrize("R,V,dtype", [(2, 1000, "f32"), (30, 30001, "bf16"), (200, 20011, "f16"), (400, 33001, "f32"), (3, 100003, "f32")])
def test_infinite_and_overflowing_logits_at_the_top(R, V, dtype):
    """Logits that are infinite, or are once scaled, are the largest ones, equals by index: they are what every filter keeps first, and a greedy row's token."""
    rng = np.random.default_rng(V)
    base = (2 * rng.standard_normal((R, V))).astype(np.float32)
    big = {"f32": 3e38, "bf16": 3e38, "f16": 6e4}[dtype]
    few, many = base.copy(), base.copy()
    few[:, V // 3] = np.inf
    many[:, [V - 1, 17, V // 2]] = np.inf
    many[:, 5] = big; many[:, 9] = -np.inf
    ctx = _ctx()
    u = _dev(rng.random(R).astype(np.float32))
    for x in (few, many):
        l = _dev(x, TYPES[dtype])
        for f in (dict(temperature=0.0), dict(top_k=1), dict(top_k=2), dict(top_k=17), dict(top_k=300), dict(top_k=700, top_p=0.5), dict(top_k=1, top_p=0.9), dict(top_p=0.4),
                  dict(top_p=0.9), dict(min_p=0.5), dict(top_k=2, min_p=0.5), dict(top_p=0.9, min_p=0.1), dict()):
            for T in (1.0, 0.25):
                g = {"temperature": T, **f}
                tok, lp, d = _sample(ctx, l, u, _params([g] * R), R, V)
                h = _f32(l[:1])
                _check_rows(h, tok[:1], lp[:1], d[:1], u[:1].cpu().numpy(), [g])
                assert np.all(np.isin(tok, [V // 3] if x is few else ([V - 1, 17, V // 2] + [5] * (T < 1 and dtype != "f16"))))
                for r in rng.integers(0, R, 2):
                    assert np.array_equal(d[r, 1:], _cat.kept(_f32(l[r:r + 1])[0], **g)[2][1:]), (r, g, d[r])
    ctx.close()


@pytest.mark.parametrize("R,V", [(2, 1000), (400, 33001), (3, 100003)])
def test_temperatures_at_the_ends_of_their_range(R, V):
    """A subnormal temperature, whose reciprocal is beyond fp32, and an infinite one beside an infinite logit: what is 0 stays 0, what is infinite infinite."""
    ctx = _ctx()
    u = _dev(np.full(R, 0.5, np.float32))
    fmax, T = np.finfo(np.float32).max, float(np.float32(1e-40))
    x = np.full((R, V), -1.0, np.float32)
    x[:, 4] = 0.0; x[:, 9] = -np.inf; x[:, V - 3] = -1e-40
    for f in (dict(), dict(top_k=1), dict(top_k=3), dict(top_k=500), dict(top_p=0.6), dict(top_k=500, top_p=0.6), dict(min_p=0.9)):
        tok, lp, d = _sample(ctx, _dev(x), u, _params([dict(temperature=T, **f)] * R), R, V)
        low = np.float32(np.float32(-1e-40) * fmax)         # (about -0.03)
        z = 1 + np.exp(np.float64(low))
        kept = {0: V - 1, 1: 1, 3: 3, 500: 500}[f.get("top_k", 0)]
        n = min(kept, 2) if "top_p" in f or "min_p" in f else kept
        assert np.all(d[:, 4] == fmax) and np.all(d[:, 3] == n), (f, d[0])
        if n == 1:
            assert np.all(tok == 4) and np.all(lp == 0) and np.all(d[:, 0] == 0)
        else:
            assert np.all(tok == 4) and np.all(np.abs(d[:, 0] - np.log(z)) < _border(V)) and np.all(d[:, 1] == (low if n == 2 else -fmax))
    x = np.zeros((R, V), np.float32)
    x[:, 7] = np.inf; x[:, 3] = -np.inf; x[:, 5] = np.nan; x[:, 11] = fmax
    for f, n in ((dict(), V - 2), (dict(top_k=1), 1), (dict(top_k=3), 3), (dict(top_k=500), 500), (dict(top_p=0.9), 1), (dict(top_k=500, top_p=0.9), 1), (dict(min_p=0.5), 1)):
        tok, lp, d = _sample(ctx, _dev(x), u, _params([dict(temperature=np.inf, **f)] * R), R, V)
        assert np.all(tok == 7) and np.all(lp == 0) and np.all(d[:, 3] == n) and np.all(d[:, 0] == fmax), (f, d[0], tok[0], lp[0])
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_of_a_row_and_one_block_give_the_same_bits(dtype):
    """A row of 45001 alone (many parts), in a batch of 30 (one block that holds it) and of 400 (three kernels, one part), rows on and off 16 bytes."""
    rng = np.random.default_rng(22)
    V = 45001
    wide = _dev((rng.standard_normal((1, V + 3)) * 1.5).astype(np.float32), TYPES[dtype])
    u = np.array([0.613], np.float32)
    ctx = _ctx()
    for off in (0, 1, 3):
        x = wide[:, off:off + V]
        for f in (dict(), dict(top_p=0.9), dict(top_k=40), dict(top_k=4000, top_p=0.8), dict(top_k=200, top_p=0.95, min_p=0.01), dict(top_k=300), dict(min_p=0.05), dict(temperature=0.0)):
            f = {"temperature": 0.9, **f}
            one = _sample(ctx, x, _dev(u), _params([f]), 1, V)
            _check_rows(_f32(x), *one, u, [f])
            for R in (5, 30, 400):
                many = _sample(ctx, x.expand(R, -1), _dev(np.repeat(u, R)), _params([f] * R), R, V)
                for a, b in zip(one, many):
                    assert np.all(b == a[0]), (f, off, R)
    ctx.close()


def test_more_rows_than_a_group():
    """1500 rows go in two groups that share the workspace, each row with filters of its own: the bits of calls of 100 rows (one block a row)."""
    R, V = 1500, 20011
    rng = np.random.default_rng(23)
    x = torch.randn(R, V, generator=torch.Generator("cuda").manual_seed(1), device="cuda") * 2
    x[::7, 100:9000] = -np.inf
    fs = [[dict(), dict(top_p=0.9), dict(top_k=20), dict(top_k=1500, top_p=0.7), dict(min_p=0.02), dict(temperature=0.0), dict(top_k=100, top_p=0.9, min_p=0.01)][r % 7 if r % 5 else 1]
          for r in range(R)]
    fs = [{"temperature": float(np.float32(rng.uniform(0.6, 1.4))), **f} for f in fs]
    u = rng.random(R).astype(np.float32)
    ctx = _ctx()
    tok, lp, d = _sample(ctx, x, _dev(u), _params(fs), R, V)
    for r in range(0, R, 100):
        for a, b in zip(_sample(ctx, x[r:r + 100], _dev(u[r:r + 100]), _params(fs[r:r + 100]), 100, V), (tok, lp, d)):
            assert np.array_equal(a, b[r:r + 100]), r
    at = [0, 1, 2, 3, 4, 5, 6, 749, 750, 751, 752, 753, 754, 1498, 1499]
    _check_rows(_f32(x[at]), tok[at], lp[at], d[at], u[at], [fs[i] for i in at])
    ctx.close()


def test_more_sequences_than_a_group():
    """5000 sequences are resampled in two groups: the tokens of calls of 1000."""
    B, V = 5000, 515
    g = torch.Generator("cuda").manual_seed(2)
    p, q = torch.randn(2 * B, V, generator=g, device="cuda") * 2, torch.randn(B, V, generator=g, device="cuda") * 2
    dp, dq = torch.zeros(2 * B, 5, dtype=torch.float64, device="cuda"), torch.zeros(B, 5, dtype=torch.float64, device="cuda")
    n = torch.randint(3, (B,), generator=g, device="cuda").to(torch.int32)     # (2: out of range)
    w = torch.rand(B, generator=g, device="cuda")
    ctx = _ctx()
    ctx.csd_cat_filter(2 * B, V, p, None, dp)
    ctx.csd_cat_filter(B, V, q, None, dq)
    new, part = (torch.full((B,), 9999, dtype=torch.int32, device="cuda") for _ in range(2))
    for _ in range(2):                                                          # tickets are zero again after a call
        ctx.csd_cat_resample(B, 1, 2, V, q, dq, p, dp, n, w, new)
    for b in range(0, B, 1000):
        e = b + 1000
        ctx.csd_cat_resample(1000, 1, 2, V, q[b:e], dq[b:e], p[2 * b:2 * e], dp[2 * b:2 * e], n[b:e], w[b:e], part[b:e])
    ctx.sync()
    assert torch.equal(new, part) and torch.equal(new == -1, n == 2)
    hp, hq = p.view(B, 2, V).cpu().numpy(), q.cpu().numpy()
    for b in (0, 1, 2, 3, 4095, 4096, 4097, 4998, 4999):
        j = int(n[b])
        if j < 2:
            r = _cat.probabilities(hp[b, j])[0]
            if j == 0:
                r = np.maximum(r - _cat.probabilities(hq[b])[0], 0.0)
            want, near = _cat.pick(r, float(w[b]))
            assert int(new[b]) == want or near < (2.0 ** -41 + V * 2.0 ** -53) / r.sum()
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_long_16_bit_rows_with_top_k_and_top_p(dtype):
    """Many parts a row, many equals: top-k ends in a bin of its own behind top-p's, before it, and in the same one."""
    R, V = 4, 100003
    rng = np.random.default_rng(24)
    x = 2 * rng.standard_normal((R, V))
    x[:, rng.integers(0, V, 40)] += 5
    l = _dev(x.astype(np.float32), TYPES[dtype])
    u = rng.random(R).astype(np.float32)
    ctx = _ctx()
    for k, p, mp in ((3000, 0.5, 0.0), (1000, 0.9, 0.0), (300, 0.999, 0.0), (20000, 0.6, 0.0), (5000, 0.3, 0.004), (700, 0.7, 0.05)):
        fs = [dict(temperature=float(np.float32(t)), top_k=k + i, top_p=float(np.float32(p)), min_p=float(np.float32(mp))) for i, t in enumerate((1.0, 0.7, 1.2, 0.9))]
        _check_rows(_f32(l), *_sample(ctx, l, _dev(u), _params(fs), R, V), u, fs)
    ctx.close()


def test_workspaces_that_grow_leave_captured_calls_their_own():
    """A graph of small calls, then larger calls of the same context (its buffers are replaced), then the graph again, and small calls."""
    from paper_2411_11925_b200 import api
    rng = np.random.default_rng(25)
    s = torch.cuda.Stream()
    ctx, plain = api.Context(0, s), _ctx()

    def inputs(B, gamma, V):
        f = lambda *sh: _dev((rng.standard_normal(sh) * 2).astype(np.float32))  # noqa: E731
        u = lambda *sh: _dev(rng.random(sh).astype(np.float32))  # noqa: E731
        return (f(B * gamma, V), f(B * (gamma + 1), V), None, None, u(B * gamma), u(B, gamma), u(B), B, gamma, gamma + 1, V)

    small, large = inputs(2, 2, 70001), inputs(30, 4, 80001)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        _round(ctx, *small)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            out = _round(ctx, *small)
        big = _round(ctx, *large)                 # larger in rows, parts and sums
        g.replay()
        again = _round(ctx, *small)
        big2 = _round(ctx, *large)
        for o in out:
            o.fill_(-3)
        g.replay()
    torch.cuda.synchronize()
    want, want_big = _round(plain, *small), _round(plain, *large)
    plain.sync()
    for a, b, c in zip(out, again, want):
        assert torch.equal(a, c) and torch.equal(b, c)
    for a, b, c in zip(big, big2, want_big):
        assert torch.equal(a, c) and torch.equal(b, c)
    ctx.sync()
    del g
    ctx.close(); plain.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_largest_vocabulary(dtype):
    """2^19 tokens, rows on and off 16 bytes (one piece more): equals throughout (sums next to 2^63), flat rows, peaks; sampling and resampling."""
    V = 1 << 19
    rng = np.random.default_rng(26)
    wide = torch.zeros(3, V + 9, dtype=TYPES[dtype], device="cuda")
    u = np.array([0.25, 0.9999999, 0.5], np.float32)
    ctx = _ctx()
    for off in (0, 1, 7):
        x = wide[:, off:off + V]
        x.zero_()
        x[1] = _dev(1.5 * rng.standard_normal(V).astype(np.float32), TYPES[dtype])
        x[2] = _dev(2 * rng.standard_normal(V).astype(np.float32), TYPES[dtype])
        x[2, [5, V // 2, V - 1]] = 25.0
        h = _f32(x)
        for f in (dict(), dict(top_p=0.9), dict(top_k=100), dict(top_k=300000)):
            fs = [{"temperature": 1.0, **f}] * 3
            tok, lp, d = _sample(ctx, x, _dev(u), _params(fs), 3, V)
            _check_rows(h[1:], tok[1:], lp[1:], d[1:], u[1:], fs[1:])
            n = f.get("top_k", V) if "top_p" not in f else int(np.ceil(np.float64(np.float32(0.9)) * V))
            # (equals: weights of 2^44 and a few units, all the same)
            assert d[0, 3] == n and d[0, 2] == n - 1 and d[0, 1] == 0 and abs(d[0, 0] - np.log(n)) < 1e-15 * 20 and tok[0] == int(np.ceil(0.25 * n)) - 1
        q = torch.zeros(3, V, device="cuda")
        dq, dp = (torch.zeros(3, 5, dtype=torch.float64, device="cuda") for _ in range(2))
        new = torch.full((3,), -5, dtype=torch.int32, device="cuda")
        ctx.csd_cat_filter(3, V, q, None, dq)
        ctx.csd_cat_filter(3, V, x, None, dp)
        ctx.csd_cat_resample(3, 1, 1, V, q, dq, x, dp, torch.zeros_like(new), _dev(u), new)
        ctx.sync()
        for b in range(3):
            p, _ = _cat.probabilities(h[b])
            r = np.maximum(p - 1.0 / V, 0.0)
            r = p if b == 0 else r
            want, near = _cat.pick(r, u[b])
            assert int(new[b]) == want or near < (2.0 ** -41 + V * 2.0 ** -53) / r.sum(), (off, b, int(new[b]), want)
    ctx.close()


def test_many_short_rows():
    R, V = 200000, 5
    g = torch.Generator("cuda").manual_seed(3)
    x, u = torch.randn(R, V, generator=g, device="cuda"), torch.rand(R, generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)
    ctx = _ctx()
    tok, lp, d = _sample(ctx, x, u, None, R, V)
    p = torch.softmax(x.double(), 1)
    c = torch.cumsum(p, 1)
    want = (c < u.double()[:, None] * c[:, -1:]).sum(1)
    near = (c - u.double()[:, None]).abs().amin(1) < 1e-12
    tok = torch.from_numpy(tok).cuda().long()
    assert torch.all((tok == want) | near)
    assert torch.all((torch.from_numpy(lp).cuda().double() - torch.log(p.gather(1, tok[:, None])[:, 0])).abs() < 1e-6)
    assert np.all(d[:, 3] == V)
    ctx.close()


@pytest.mark.parametrize("at_p,at_q", [(5000.0, 5000.0), (1e6, 0.0), (0.0, -1e6), (-3e38, 1e30)])
def test_resampling_of_large_logits(at_p, at_q):
    """Normalisers so large that a difference from them has to be formed with care, of p, of q, of both: the residual of the rows as they round."""
    B, gamma, V = 6, 2, 3001
    rng = np.random.default_rng(27)
    p = (2 * rng.standard_normal((B, gamma + 1, V)) + at_p).astype(np.float32)
    q = (2 * rng.standard_normal((B * gamma, V)) + at_q).astype(np.float32)
    u0, u, w = rng.random(B * gamma).astype(np.float32), rng.random((B, gamma)).astype(np.float32), rng.random(B).astype(np.float32).clip(1e-6)
    ctx = _ctx()
    tok, dq, dp, lr, n, mask, new = _round(ctx, _dev(q), _dev(p.reshape(-1, V)), None, None, _dev(u0), _dev(u), _dev(w), B, gamma, gamma + 1, V)
    for j in range(gamma + 1):
        n.fill_(j)
        ctx.csd_cat_resample(B, gamma, gamma + 1, V, _dev(q), dq, _dev(p.reshape(-1, V)), dp, n, _dev(w), new)
        ctx.sync()
        for b in range(B):
            r, _ = _cat.probabilities(p[b, j])
            if j < gamma:
                rest = np.maximum(r - _cat.probabilities(q[b * gamma + j])[0], 0.0)
                r = rest if rest.sum() > 0 else r
            want, near = _cat.pick(r, w[b])
            # (a summary is rounded to fp64: 2^-53 of the normaliser, in the exponent)
            assert int(new[b]) == want or near < (2.0 ** -40 + 2.0 ** -52 * (abs(at_p) if abs(at_p) < 1e7 else 0) + V * 2.0 ** -53) / r.sum(), (b, j)
    ctx.close()


def test_two_contexts_on_two_streams_at_once():
    from paper_2411_11925_b200 import api
    rng = np.random.default_rng(28)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ctxs, plain = [api.Context(0, s) for s in streams], _ctx()
    args = []
    for k in range(2):
        B, gamma, V = 20 + 30 * k, 3, 60001
        f = lambda *sh: _dev((rng.standard_normal(sh) * 2).astype(np.float32))  # noqa: E731
        u = lambda *sh: _dev(rng.random(sh).astype(np.float32))  # noqa: E731
        fp = _params([dict(temperature=0.9, top_k=[0, 50, 4000][r % 3], top_p=0.9) for r in range(B * (gamma + 1))])
        args.append((f(B * gamma, V), f(B * (gamma + 1), V), None, fp, u(B * gamma), u(B, gamma), u(B), B, gamma, gamma + 1, V))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k].append(_round(ctxs[k], *args[k]))
    torch.cuda.synchronize()
    for k in range(2):
        want = _round(plain, *args[k])
        plain.sync()
        for out in got[k]:
            for a, b in zip(out, want):
                assert torch.equal(a, b)
    for c in ctxs + [plain]:
        c.sync()
        c.close()
