"""Performance cases of the categorical (vocabulary) head: final norm, 8-bit vocabulary product, sampling, verification, resampling.

A model whose tokens come from a vocabulary has, where a diffusion head has its T-step chain, a root-mean-square norm of the
backbone's output, one product with the vocabulary matrix, and explicit distributions p and q.  A speculative round is then:
draft tokens sampled from the filtered q, the accept test of their ratios, and a token drawn from max(0, p - q) (or from p, where
all drafts were accepted).  Each case is one call of that path.  `run` computes it from elementary torch operations, or, where
`own` is set, through the calls of `paper_2411_11925_b200.api`.

A distribution is kept as one row of five float64 numbers: log of its normaliser, the smallest scaled logit that is kept, the
highest index kept among equals of it, how many tokens are kept, and the reciprocal temperature.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_FMAX = torch.finfo(torch.float32).max
_EPS = 1e-6


# ------------------------------------------------------------------------------------------------------------ the cases
def _sample(name, R, V, dtype, kind, T, k, p, mp=0.0, masked=0.0):
    c = {"call": "sample", "R": R, "V": V, "dtype": dtype, "kind": kind, "T": T, "top_k": k, "top_p": p, "min_p": mp, "masked": masked}
    return {"name": name, **c} if name else c


def _pair(name, call, B, gamma, V, dtype, kind, T, k, p, mp=0.0, bonus=True):
    c = {"call": call, "B": B, "gamma": gamma, "V": V, "dtype": dtype, "kind": kind, "T": T, "top_k": k, "top_p": p, "min_p": mp,
         "bonus": bonus}
    return {"name": name, **c} if name else c


def _norm(name, M, K, dtype, residual=True):
    c = {"call": "norm", "M": M, "K": K, "dtype": dtype, "residual": residual}
    return {"name": name, **c} if name else c


def _matmul(name, M, N, K, dtype):
    c = {"call": "matmul", "M": M, "N": N, "K": K, "dtype": dtype}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one draft position of one sequence, a codebook of image tokens with its wide flat distributions: latency
        _sample("sample_one", 1, 16384, "f32", "flat", 1.0, 2000, 0.95),
        # a text vocabulary of odd size, a batch of requests with their own settings, a third of the tokens masked
        _sample("sample_mixed_odd", 37, 50003, "bf16", "peaked", 0.8, 50, 0.95, 0.02, 0.3),
        # a large batch over a large vocabulary, nucleus sampling without top-k
        _sample("sample_large", 512, 131072, "f32", "peaked", 0.9, 0, 0.92),
        # verification of a few drafts of a few sequences
        _pair("verify_few", "verify", 4, 5, 32768, "bf16", "peaked", 1.0, 0, 0.95),
        # verification of the batch of the workload table (64 sequences, 8 drafts) with the bonus position
        _pair("verify_batch", "verify", 64, 8, 65536, "bf16", "peaked", 0.9, 200, 0.9),
        # the token behind the accepted prefix: odd vocabulary and batch, no bonus row
        _pair("resample_odd", "resample", 37, 7, 50003, "f32", "peaked", 1.0, 0, 0.95, bonus=False),
        # the same for a large batch without any filter, flat distributions
        _pair("resample_batch", "resample", 256, 4, 131072, "bf16", "flat", 1.0, 0, 1.0),
        # the final norm of one position
        _norm("norm_one", 1, 4096, "bf16"),
        # the final norm of a prefill, rows that are no multiple of the block of 128
        _norm("norm_prefill", 8192, 5000, "bf16"),
        # the vocabulary product of one position: reads every weight for one row
        _matmul("matmul_one", 1, 32768, 4096, "f32"),
        # of a verified batch (64 sequences, 8 drafts and the bonus position)
        _matmul("matmul_verify", 576, 65536, 2048, "bf16"),
        # of a scored prompt, sizes off every tile
        _matmul("matmul_ragged", 2333, 50003, 4000, "f16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    call = rng.choice(["sample", "sample", "verify", "resample", "norm", "matmul", "matmul"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if call == "norm":
        K = _log_int(rng, 128, 8192)
        return _norm("", _log_int(rng, 1, min(16384, (1 << 25) // K)), K, dtype, rng.random() < 0.7)
    if call == "matmul":
        K, N = _log_int(rng, 256, 8192), _log_int(rng, 1000, 131072)
        return _matmul("", _log_int(rng, 1, max(1, min(4096, (1 << 38) // (N * K)))), N, K, dtype)
    V = _log_int(rng, 1000, 131072)
    kind = rng.choice(["flat", "peaked"])
    T, k = rng.uniform(0.5, 1.3), rng.choice([0, _log_int(rng, 1, 4096)])
    p, mp = rng.choice([1.0, rng.uniform(0.6, 0.99)]), rng.choice([0.0, 0.0, rng.uniform(0.005, 0.2)])
    if call == "sample":
        return _sample("", _log_int(rng, 1, min(1024, (1 << 25) // V)), V, dtype, kind, T, k, p, mp, rng.choice([0.0, rng.uniform(0.1, 0.9)]))
    gamma = _log_int(rng, 1, 16)
    B = _log_int(rng, 1, max(1, min(256, (1 << 25) // (V * (gamma + 1)))))
    return _pair("", call, B, gamma, V, dtype, kind, T, k, p, mp, rng.random() < 0.7)


def _pitch(K):
    blocks = (K + 127) // 128
    return 128 * blocks, (blocks + 3) // 4 * 4


def work(case):
    es = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]]
    if case["call"] == "norm":
        M, K = case["M"], case["K"]
        ld, ls = _pitch(K)
        return {"bytes": float(M * K * es * (3 if case["residual"] else 1) + K * es + M * (ld + ls)), "flops": 7.0 * M * K}
    if case["call"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        ld, ls = _pitch(K)
        return {"bytes": float((M + N) * (ld + ls) + M * N * es), "flops": 2.0 * M * N * K}
    V = case["V"]
    if case["call"] == "sample":
        return {"bytes": float(case["R"] * (V * es + 5 * 4 + 4 + 4 + 40)), "flops": 4.0 * case["R"] * V}
    B, g = case["B"], case["gamma"]
    rows = g + 1 if case["bonus"] else g
    if case["call"] == "verify":
        return {"bytes": float(B * (rows * (V * es + 16 + 40) + g * (40 + es + 12) + 8)), "flops": 4.0 * B * rows * V}
    # one row of p for each sequence (none where all drafts were accepted and there is no bonus row), one of q unless all were
    part = g / (g + 1)
    reads = 2 * part + (1 - part if case["bonus"] else 0)
    return {"bytes": float(B * (reads * V * es + 2 * 40 + 12)), "flops": 6.0 * B * part * V}


# ----------------------------------------------------------------------------------------------------------- the inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed & 0x7FFFFFFF)


def _logits(g, rows, V, kind):
    """Scaled like those of a head: flat ones (image tokens), or a bulk with a few likely tokens above it (text)."""
    x = torch.randn(rows, V, generator=g, device="cuda")
    if kind == "flat":
        return x.mul_(1.5)
    x.mul_(2.2)
    at = torch.randint(V, (rows, 12), generator=g, device="cuda")
    up = torch.rand(rows, 12, generator=g, device="cuda") * 6 + 8
    return x.scatter_(1, at, up)


def _settings(g, case, rows):
    """Each request has its own temperature; top-k, top-p and min-p are the case's."""
    T = case["T"] * (0.9 + 0.2 * torch.rand(rows, generator=g, device="cuda"))
    full = lambda v, t: torch.full((rows,), v, dtype=t, device="cuda")  # noqa: E731
    return {"temperature": T, "top_k": full(case["top_k"], torch.int32), "top_p": full(case["top_p"], torch.float32),
            "min_p": full(case["min_p"], torch.float32)}


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda").clamp_(1e-6, 1 - 1e-6)


def _empty(dtype, *shape):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def prepare(case, seed):
    g, dt = _gen(seed), _TYPES[case["dtype"]]
    s = {"case": case}
    call = case["call"]
    if call == "norm":
        M, K = case["M"], case["K"]
        x = torch.randn(M, K, generator=g, device="cuda")
        x[:, :: 97] *= 12.0          # the few large channels of a backbone's output
        s["x"] = x.to(dt)
        s["residual"] = torch.randn(M, K, generator=g, device="cuda").to(dt) if case["residual"] else None
        s["weight"] = (1 + 0.1 * torch.randn(K, generator=g, device="cuda")).to(dt)
        ld, ls = _pitch(K)
        s["out"] = (_empty(torch.uint8, M, ld), _empty(torch.uint8, M, ls), _empty(dt, M, K) if case["residual"] else None)
        return s
    if call == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        s["a"] = _quantize(torch.randn(M, K, generator=g, device="cuda"))
        s["w"] = _quantize(torch.randn(N, K, generator=g, device="cuda").mul_(K ** -0.5))
        s["out"] = _empty(dt, M, N)
        return s
    V = case["V"]
    if call == "sample":
        R = case["R"]
        x = _logits(g, R, V, case["kind"])
        if case["masked"]:
            x.masked_fill_(torch.rand(R, V, generator=g, device="cuda") < case["masked"], -math.inf)
        s["logits"], s["set"], s["u"] = x.to(dt), _settings(g, case, R), _uniform(g, R)
        s["out"] = (_empty(torch.int32, R), _empty(torch.float32, R), _empty(torch.float64, R, 5))
        return s
    B, gamma = case["B"], case["gamma"]
    rows = gamma + 1 if case["bonus"] else gamma
    p = _logits(g, B * rows, V, case["kind"])
    q = p.view(B, rows, V)[:, :gamma] + 0.5 * torch.randn(B, gamma, V, generator=g, device="cuda")
    s["p"], s["q"] = p.to(dt), q.reshape(B * gamma, V).to(dt)
    s["set_p"], set_q = _settings(g, case, B * rows), _settings(g, case, B * gamma)
    s["dist_q"], t, w = _filter(s["q"], **set_q)
    if call == "verify":
        s["token"] = _pick(w, _uniform(g, B * gamma), s["dist_q"])
        s["u"] = _uniform(g, B, gamma)
        s["out"] = (_empty(torch.float64, B * rows, 5), _empty(torch.float32, B, gamma), _empty(torch.int32, B), _empty(torch.int32, B))
        return s
    s["dist_p"] = _filter(s["p"], **s["set_p"])[0]
    s["n_accept"] = torch.randint(gamma + 1, (B,), generator=g, device="cuda").to(torch.int32)
    s["w"] = _uniform(g, B)
    s["x_new"] = _empty(torch.int32, B)
    return s


# ------------------------------------------------------------------------------------------------------ the plain forms
def _quantize(y):
    """[rows, K] in 8 bits (e4m3), a power-of-two scale (e8m0) for each block of 128: the smallest under which the block fits.
    Bytes, rows padded with zeros to whole blocks and the scales to a multiple of four."""
    M, K = y.shape
    ld, ls = _pitch(K)
    y = torch.nn.functional.pad(y, (0, ld - K)).view(M, ld // 128, 128)
    m, e = torch.frexp(y.abs().amax(2))                     # amax = m 2^e, m in [1/2, 1): 448 = 0.875 * 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(m == 0, torch.zeros_like(e), e)
    data = torch.ldexp(y, -e[:, :, None]).to(torch.float8_e4m3fn).view(M, ld)
    scale = torch.nn.functional.pad(e + 127, (0, ls - e.shape[1]), value=127).to(torch.uint8)
    return data.view(torch.uint8), scale


def _values(q):
    data, scale = q
    M, ld = data.shape
    e = scale[:, : ld // 128].to(torch.int32) - 127
    return torch.ldexp(data.view(torch.float8_e4m3fn).float().view(M, ld // 128, 128), e[:, :, None]).view(M, ld)


def _scaled(l, inv_t):
    """Scaled logits in 32 bits; what is masked (-inf, NaN) is -inf, everything else finite."""
    live = ~(torch.isnan(l) | (l == -math.inf))
    t = (l.float() * inv_t[:, None]).clamp_(-_FMAX, _FMAX)
    return t.masked_fill_(~live, -math.inf)


def _filter(l, temperature, top_k, top_p, min_p):
    """The kept tokens: top-k, of these the shortest prefix (largest first, equals by index) that reaches top_p of their sum, of these
    all at least min_p times as likely as the likeliest.  Returns the row's summary, the scaled logits and the kept weights."""
    R, V = l.shape
    greedy = temperature <= 0
    inv_t = torch.where(greedy, torch.ones_like(temperature), 1.0 / temperature)
    t = _scaled(l, inv_t)
    s, order = torch.sort(t, dim=1, descending=True, stable=True)
    top = s[:, :1].double()
    live = (t > -math.inf).sum(1)
    k = torch.where(greedy, torch.ones_like(live), torch.where(top_k <= 0, V, top_k.long())).minimum(live)
    rank = torch.arange(V, device=l.device)[None, :]
    w = torch.where(rank < k[:, None], torch.exp(s.double() - top), 0.0)
    c = torch.cumsum(w, 1)
    limit = torch.where(top_p < 1, top_p.double(), math.inf) * c[:, -1]
    keep = (rank < k[:, None]) & (c - w < limit[:, None]) & (w >= torch.where(min_p > 0, min_p, 0.0).double()[:, None])
    keep |= (rank == 0) & (live > 0)[:, None]
    n = keep.sum(1)
    at = (n - 1).clamp_(min=0)[:, None]
    some = n > 0
    last = torch.where(some, order.gather(1, at)[:, 0], -1)
    cut = torch.where(some, s.gather(1, at)[:, 0].double(), math.inf)
    z = torch.where(keep, w, 0.0).sum(1)
    norm = torch.where(some, top[:, 0] + torch.log(z), -math.inf)
    dist = torch.stack([norm, cut, last.double(), n.double(), inv_t.double()], 1)
    return dist, t, _kept(t, dist) * torch.exp(t.double() - torch.where(some, top[:, 0], 0.0)[:, None])


def _kept(t, dist):
    index = torch.arange(t.shape[1], device=t.device)[None, :]
    cut = dist[:, 1:2]
    return (t > cut) | ((t == cut) & (index <= dist[:, 2:3]))


def _pick(w, u, dist):
    """The first token whose cumulative weight, in index order, reaches u times their sum; -1 where there is none."""
    c = torch.cumsum(w, 1)
    token = (c < (u.double() * c[:, -1])[:, None]).sum(1).clamp_(max=w.shape[1] - 1)
    return torch.where(dist[:, 3] > 0, token, -1).to(torch.int32)


def _log_prob(l, dist, token):
    """log of a token's probability, from its logit alone."""
    at = token.long().clamp(min=0)[:, None]
    t = _scaled(l.gather(1, at), dist[:, 4].float())[:, 0].double()
    kept = (token >= 0) & ((t > dist[:, 1]) | ((t == dist[:, 1]) & (token <= dist[:, 2])))
    return torch.where(kept, t - dist[:, 0], -math.inf)


def _probs(l, dist):
    t = _scaled(l, dist[:, 4].float())
    norm = torch.where(dist[:, 3] > 0, dist[:, 0], 0.0)[:, None]
    return _kept(t, dist) * torch.exp(t.double() - norm)


def _plain(s):
    case = s["case"]
    call = case["call"]
    if call == "norm":
        h = s["x"].float() + s["residual"].float() if case["residual"] else s["x"].float()
        y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + _EPS) * s["weight"].float()
        return *_quantize(y), h.to(s["x"].dtype) if case["residual"] else None
    if call == "matmul":
        return (_values(s["a"]) @ _values(s["w"]).T).to(_TYPES[case["dtype"]])
    if call == "sample":
        dist, t, w = _filter(s["logits"], **s["set"])
        token = _pick(w, s["u"], dist)
        return token, _log_prob(s["logits"], dist, token).float(), dist
    B, g, V = case["B"], case["gamma"], case["V"]
    rows = g + 1 if case["bonus"] else g
    if call == "verify":
        dist = _filter(s["p"], **s["set_p"])[0]
        lp = _log_prob(s["p"].view(B, rows, V)[:, :g].reshape(B * g, V), dist.view(B, rows, 5)[:, :g].reshape(B * g, 5), s["token"])
        lq = _log_prob(s["q"], s["dist_q"], s["token"])
        ratio = torch.where(lp == -math.inf, -math.inf, torch.where(lq == -math.inf, math.inf, lp - lq)).view(B, g)
        ok = (torch.log(s["u"].double()) <= ratio).to(torch.int32)
        mask = (ok << torch.arange(g, device=ok.device, dtype=torch.int32)).sum(1).to(torch.int32)
        return dist, ratio.float(), torch.cumprod(ok, 1).sum(1).to(torch.int32), mask
    n = s["n_accept"].long()
    b = torch.arange(B, device="cuda")
    row = b * rows + n.clamp(max=rows - 1)
    rejected = n < g
    qrow = b * g + n.clamp(max=g - 1)
    dist = s["dist_p"][row]
    p = _probs(s["p"][row], dist)
    r = torch.where(rejected[:, None], (p - _probs(s["q"][qrow], s["dist_q"][qrow])).clamp_(min=0.0), p)
    r = torch.where(r.sum(1, keepdim=True) > 0, r, p)
    token = _pick(r, s["w"], dist)
    return torch.where(rejected | (rows > g), token, -1).to(torch.int32)


# ------------------------------------------------------------------------------------------------------------- one pass
_context = None


def _ctx():
    global _context
    if _context is None:
        from paper_2411_11925_b200 import api
        _context = api.Context(torch.cuda.current_device())
    return _context


def run(s):
    case = s["case"]
    call = case["call"]
    if not own:
        out = _plain(s)
        if call == "norm":
            return {"data": out[0].view(torch.float8_e4m3fn), "scale": out[1].view(torch.float8_e8m0fnu), "sum": out[2]}
        if call == "sample":
            return {"token": out[0], "log_prob": out[1], "dist": out[2]}
        if call == "verify":
            return {"dist_p": out[0], "logratio": out[1], "n_accept": out[2], "mask": out[3]}
        return out
    ctx = _ctx()
    if call == "norm":
        data, scale, total = s["out"]
        ctx.csd_norm_quantize(case["M"], case["K"], s["x"], s["residual"], s["weight"], _EPS, total, data, scale)
        return {"data": data.view(torch.float8_e4m3fn), "scale": scale.view(torch.float8_e8m0fnu), "sum": total}
    if call == "matmul":
        ctx.csd_quant_matmul(case["M"], case["N"], case["K"], s["a"], s["w"], s["out"])
        return s["out"]
    V = case["V"]
    if call == "sample":
        f, (token, logp, dist) = s["set"], s["out"]
        ctx.csd_cat_draft_sample(case["R"], V, s["logits"], (f["temperature"], f["top_k"], f["top_p"], f["min_p"]), s["u"], token, logp, dist)
        return {"token": token, "log_prob": logp, "dist": dist}
    B, g = case["B"], case["gamma"]
    rows = g + 1 if case["bonus"] else g
    if call == "verify":
        f, (dist, ratio, n, mask) = s["set_p"], s["out"]
        ctx.csd_cat_verify(B, g, rows, V, s["q"], s["dist_q"], s["p"], (f["temperature"], f["top_k"], f["top_p"], f["min_p"]), s["token"],
                           s["u"], dist, ratio, n, mask)
        return {"dist_p": dist, "logratio": ratio, "n_accept": n, "mask": mask}
    ctx.csd_cat_resample(B, g, rows, V, s["q"], s["dist_q"], s["p"], s["dist_p"], s["n_accept"], s["w"], s["x_new"])
    return s["x_new"]


# ------------------------------------------------------------------------------------- the definitions, in 64 bits
def _exact_dist(l, f):
    """Row summaries in 64 bits: the tokens are ranked by (value, index) and the three filters are three counts."""
    R, V = l.shape
    T = f["temperature"]
    inv = torch.where(T > 0, 1.0 / T, torch.ones_like(T))
    t = (l.to(torch.float32) * inv.unsqueeze(1)).to(torch.float64)
    ranked, index = torch.sort(-t, dim=1, stable=True)
    ranked = -ranked
    alive = torch.isfinite(ranked).sum(1)
    count = torch.where(f["top_k"] > 0, f["top_k"].to(torch.int64), V).minimum(alive)
    count = torch.where(T > 0, count, 1)
    place = torch.arange(V, device=l.device).expand(R, V)
    e = torch.softmax(ranked.masked_fill(place >= count.unsqueeze(1), -math.inf), 1)
    before = torch.cumsum(e, 1).roll(1, 1)
    before[:, 0] = 0.0
    p = torch.where(f["top_p"] < 1, f["top_p"].to(torch.float64), 2.0)
    by_mass = (before < p.unsqueeze(1)).sum(1).clamp(min=1)
    floor = torch.where(f["min_p"] > 0, torch.log(f["min_p"].to(torch.float64)), -math.inf)
    by_min = (ranked >= (ranked[:, 0] + floor).unsqueeze(1)).sum(1).clamp(min=1)
    n = torch.minimum(torch.minimum(count, by_mass), by_min)
    end = (n - 1).unsqueeze(1)
    norm = torch.logsumexp(ranked.masked_fill(place >= n.unsqueeze(1), -math.inf), 1)
    return torch.stack([norm, ranked.gather(1, end).squeeze(1), index.gather(1, end).squeeze(1).to(torch.float64), n.to(torch.float64),
                        inv.to(torch.float64)], 1), t


def _exact_in(t, index, d):
    return (t > d[:, 1]) | ((t == d[:, 1]) & (index <= d[:, 2]))


def exact(case, seed):
    """What run() returns, in 64 bits; None for the whole numbers."""
    s = prepare(case, seed)
    call = case["call"]
    if call == "norm":
        x = s["x"].to(torch.float64)
        total = x + s["residual"].to(torch.float64) if case["residual"] else x
        y = total / torch.sqrt(torch.mean(total ** 2, 1, keepdim=True) + _EPS) * s["weight"].to(torch.float64)
        M, K = y.shape
        ld, ls = _pitch(K)
        block = torch.zeros(M, ld, dtype=torch.float64, device=y.device)
        block[:, :K] = y
        block = block.view(M, -1, 128)
        scale = torch.ones(M, ls, dtype=torch.float64, device=y.device)
        scale[:, : ld // 128] = torch.exp2(torch.ceil(torch.log2(block.abs().amax(2) / 448.0)))
        data = block / scale[:, : ld // 128].unsqueeze(2)     # before its rounding to 8 bits
        return {"data": data.view(M, ld), "scale": scale, "sum": total if case["residual"] else None}
    if call == "matmul":
        def full(q):
            data, scale = q
            f = torch.pow(2.0, scale.to(torch.float64) - 127.0)[:, : data.shape[1] // 128]
            return data.view(torch.float8_e4m3fn).to(torch.float64) * f.repeat_interleave(128, dim=1)
        return full(s["a"]) @ full(s["w"]).t()
    if call == "sample":
        d, t = _exact_dist(s["logits"], s["set"])
        place = torch.arange(case["V"], device=t.device).unsqueeze(0)
        kept = (t > d[:, 1:2]) | ((t == d[:, 1:2]) & (place <= d[:, 2:3]))
        c = torch.cumsum(torch.softmax(t.masked_fill(~kept, -math.inf), 1), 1)
        token = torch.searchsorted(c, (s["u"].to(torch.float64) * c[:, -1]).unsqueeze(1)).clamp(max=case["V"] - 1)
        return {"token": None, "log_prob": t.gather(1, token).squeeze(1) - d[:, 0], "dist": d}
    if call == "verify":
        B, g, V = case["B"], case["gamma"], case["V"]
        rows = g + 1 if case["bonus"] else g
        d, t = _exact_dist(s["p"], s["set_p"])
        x = s["token"].to(torch.int64)
        row = torch.arange(B * g, device=x.device) // g * rows + torch.arange(B * g, device=x.device) % g
        tp = t[row, x]
        tq = (s["q"].to(torch.float32)[torch.arange(B * g, device=x.device), x] * s["dist_q"][:, 4].to(torch.float32)).to(torch.float64)
        ratio = (tp - d[row, 0]) - (tq - s["dist_q"][:, 0])
        ratio = torch.where(_exact_in(tq, x, s["dist_q"]), ratio, math.inf)
        ratio = torch.where(_exact_in(tp, x, d[row]), ratio, -math.inf)
        return {"dist_p": d, "logratio": ratio.view(B, g), "n_accept": None, "mask": None}
    return None
