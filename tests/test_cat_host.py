"""CPU-side checks of the categorical heads and 8-bit matrices: the plain forms the GPU tests compare with, the host call, and what
the binding refuses before it reaches a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import _cat
from paper_2411_11925_b200 import build


def test_plain_filter_against_its_definition():
    rng = np.random.default_rng(0)
    for V in (1, 5, 40):
        x = np.round(2 * rng.standard_normal(V), 1).astype(np.float32)     # with equals
        for k, p, mp, T in ((0, 1.0, 0.0, 1.0), (3, 1.0, 0.0, 0.5), (0, 0.6, 0.0, 1.0), (7, 0.8, 0.05, 1.3), (0, 1.0, 0.3, 1.0), (0, 1.0, 0.0, 0.0)):
            order, logp, row = _cat.kept(x, temperature=T, top_k=k, top_p=p, min_p=mp)
            t, _ = _cat.scaled(x, T)
            full = sorted(range(V), key=lambda i: (-t[i], i))
            want = full[:k] if k else full
            if T == 0.0:
                want = full[:1]
            w = np.exp(t.astype(np.float64) - t.max())
            if p < 1:
                total, run, keep = sum(w[i] for i in want), 0.0, []
                for i in want:
                    keep.append(i)
                    run += w[i]
                    if run >= np.float32(p) * total:
                        break
                want = keep
            want = [i for i in want if w[i] >= mp or i == full[0]]
            assert list(order) == want
            assert abs(np.exp(logp).sum() - 1) < 1e-12 and row[3] == len(want) and row[2] == want[-1]
    assert _cat.kept(np.full(4, -np.inf, np.float32))[0].size == 0


def test_plain_pick_and_residual_frequencies():
    rng = np.random.default_rng(1)
    p, q = rng.dirichlet(np.ones(6)), rng.dirichlet(np.ones(6))
    # draft, accept or resample: the token is distributed as p
    n, count = 40000, np.zeros(6)
    r = np.maximum(p - q, 0)
    for u0, u, w in rng.random((n, 3)):
        x = _cat.pick(q, u0)[0]
        count[x if u <= p[x] / q[x] else _cat.pick(r, w)[0]] += 1
    assert np.all(np.abs(count / n - p) < 5 * np.sqrt(p * (1 - p) / n))


def test_e4m3_bytes_match_torch():
    b = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(b).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    np.testing.assert_array_equal(_cat.e4m3(b), want)
    y = np.zeros((5, 128)); y[0, 3] = 448; y[1, 3] = -449; y[2, 0] = 1.75; y[3, 0] = 1.7500001
    s = _cat.scale_bytes(y).ravel()
    assert list(s) == [127, 128, 119, 120, 127]
    assert np.all(np.abs(y).max(1) <= 448 * 2.0 ** (s.astype(float) - 127))


def test_quant_pitch():
    from paper_2411_11925_b200 import api
    assert [api.quant_pitch(k) for k in (1, 128, 129, 512, 513, 4000)] == [(128, 4), (128, 4), (256, 4), (512, 4), (640, 8), (4096, 32)]
    for k in (0, -5, (1 << 20) + 1):
        with pytest.raises(api.CsdError):
            api.quant_pitch(k)
    d, s = api.quant_empty(3, 200, "cpu")
    assert d.shape == (3, 256) and s.shape == (3, 4) and d.dtype == torch.uint8


def test_null_context_is_refused():
    lib = ctypes.CDLL(build.build_library())
    z = ctypes.c_void_p(0)
    assert lib.csd_cat_filter(z, 1, 4, z, z, z) == -1
    assert lib.csd_cat_draft_sample(z, 1, 4, z, z, z, z, z, z) == -1
    assert lib.csd_cat_verify(z, 1, 1, 1, 4, z, z, z, z, z, z, z, z, z, z) == -1
    assert lib.csd_cat_resample(z, 1, 1, 1, 4, z, z, z, z, z, z, z) == -1
    i64, f = ctypes.c_int64(0), ctypes.c_float(1e-6)
    assert lib.csd_quantize(z, 1, 4, 0, z, i64, z, z) == -1
    assert lib.csd_norm_quantize(z, 1, 4, 0, z, i64, z, i64, z, f, z, i64, z, z) == -1
    assert lib.csd_quant_matmul(z, 1, 4, 4, z, z, 0, z, i64) == -1
    assert lib.csd_quant_pitch(4, None, None) == -1


def test_the_binding_refuses_host_tensors_and_wrong_types_before_the_library():
    from paper_2411_11925_b200 import _marshal as m
    l, u, t, d = torch.zeros(2, 8), torch.zeros(2), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 5, dtype=torch.float64)
    q = (torch.zeros(2, 128, dtype=torch.uint8), torch.zeros(2, 4, dtype=torch.uint8))
    for call in (lambda: m.cat_filter(0, 0, 2, 8, l, None, d), lambda: m.cat_draft_sample(0, 0, 2, 8, l, None, u, t, None, d),
                 lambda: m.cat_verify(0, 0, 1, 2, 2, 8, l, d, l, None, t, u, d, u, t, None),
                 lambda: m.cat_resample(0, 0, 1, 2, 2, 8, l, d, l, d, t, u, t), lambda: m.quantize(0, 0, 2, 8, l, *q),
                 lambda: m.norm_quantize(0, 0, 2, 8, l, None, None, 1e-6, None, *q), lambda: m.quant_matmul(0, 0, 2, 2, 8, q, q, l)):
        with pytest.raises(ValueError, match="cuda:0"):
            call()
    for call in (lambda: m.cat_filter(0, 0, 2, 8, l.numpy(), None, d), lambda: m.quant_matmul(0, 0, 2, 2, 8, q[0], q, l), lambda: m.cat_filter(0, 0, 2, 8),
                 lambda: m.cat_filter(0, 0, "2", 8, l, None, d)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(OverflowError):
        m.cat_filter(0, 0, 1 << 40, 8, l, None, d)
