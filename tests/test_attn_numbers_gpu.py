"""Numbers at the ends of decoding's arithmetic, against the fp64 reference:
large values under rising scores, and caps of any size.

Tolerances are those of test_attn_gpu.py.
"""
import numpy as np
import pytest

from oracle import attn as R
from paper_2608_30963_amd import kvx
from tests import gpu_util as U
from tests import test_attn_gpu as A

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


@pytest.mark.parametrize("dtype,m,d", [("bf16", 1, 128), ("bf16", 70, 64), ("bf16", 70, 128),
                                       ("bf16", 70, 256), ("f32", 70, 64), ("f32", 70, 128)])
def test_large_values_under_rising_scores(dtype, m, d):
    """Scores that rise by 70 bits over six tiles of 64 slots, of values about
    2^60: their average is far from fp32's largest number."""
    T = U.torch()
    print(f"[attn] large values {dtype} {m} x {d}", flush=True)
    n, hq = 6144, 4
    cache = A.Cache([n], 2, d, dtype, 64)
    g = T.Generator().manual_seed(8)
    rows = T.randn(n, 2, d, generator=g) * 0.1
    rows[..., 0] += T.linspace(-480.0, 480.0, n)[:, None]
    rows = rows.to(A._dt(dtype))
    values = (T.randn(n, 2, d, generator=g) * 2.0 ** 60).to(A._dt(dtype))
    blk, slot = cache.place(0, np.arange(n))
    cache.dev[0][1, blk, :, slot] = rows.cuda()
    cache.dev[1][1, blk, :, slot] = values.cuda()
    q = A._rows(m, hq, d, dtype, 3, 0.1)
    q[..., 0] = d ** 0.5
    att = kvx.Attention(kvx.ModelShape(2, 2, d, 1e4), hq,
                        kvx.KVX_BF16 if dtype == "bf16" else kvx.KVX_F32)
    out, lse = T.zeros_like(q), T.zeros(m, hq, device="cuda")
    att.forward(kvx.make_attn_io(cache.struct, A._int([n]), q, out=out, lse=lse, layer=1, max_new=m,
                                 q_start=A._int([0, m])), att.workspace())
    T.cuda.synchronize()
    ro, rl, mag, size = R.attend(A._f64(q), A._f64(rows), A._f64(values), d ** -0.5)
    delta = A._delta(size, d, 0.0)
    rel = 2 * delta + (n + 64) * EPS + (2.0 ** -8 if dtype == "bf16" else 0.0)
    tol = mag * rel[..., None] + (2.0 ** -8 * np.abs(ro) if dtype == "bf16" else 0.0)
    oh = A._f64(out)
    assert np.isfinite(oh).all(), "non-finite output"
    assert (np.abs(oh - ro) <= tol).all()
    assert (np.abs(A._f64(lse) - rl) <= delta + (n + 64) * EPS + 2.0 ** -22 * (1 + np.abs(rl))).all()
    att.close()


@pytest.mark.parametrize("cap", [20.0, 100.0, 130.0, 1e4, 1e6, 1e9])
@pytest.mark.parametrize("m,d", [(1, 128), (3, 256), (75, 64), (75, 128), (70, 256)])
def test_bf16_scores_under_any_cap(m, d, cap):
    """bf16 attention under caps from a score's size to far beyond: up to 128 a
    score errs by 2^-22 of the cap, above by 2^-21 of its terms."""
    T = U.torch()
    print(f"[attn] bf16 cap {cap} {m} x {d}", flush=True)
    n, hq = 400, 4
    cache = A.Cache([n], 2, d, "bf16", 16)
    q = A._rows(m, hq, d, "bf16", 3)
    att = kvx.Attention(kvx.ModelShape(2, 2, d, 1e4), hq, kvx.KVX_BF16, softcap=cap)
    out, lse = T.zeros_like(q), T.zeros(m, hq, device="cuda")
    att.forward(kvx.make_attn_io(cache.struct, A._int([n]), q, out=out, lse=lse, layer=1, max_new=m,
                                 q_start=A._int([0, m])), att.workspace())
    T.cuda.synchronize()
    ro, rl, mag, size = R.attend(A._f64(q), cache.f64(0, 1, 0), cache.f64(1, 1, 0), d ** -0.5, cap)
    delta = (d + 8) * EPS * size + (2.0 ** -22 * cap if cap <= 128 else 2.0 ** -21 * size)
    tol = mag * (2 * delta + (n + 64) * EPS + 2.0 ** -8)[..., None] + 2.0 ** -8 * np.abs(ro)
    assert (np.abs(A._f64(out) - ro) <= tol).all(), (np.abs(A._f64(out) - ro) / tol).max()
    ltol = delta + (n + 64) * EPS + 2.0 ** -22 * (1 + np.abs(rl))
    assert (np.abs(A._f64(lse) - rl) <= ltol).all(), (np.abs(A._f64(lse) - rl) / ltol).max()
    att.close()


@pytest.mark.parametrize("cap", [1e-6, 0.5, 2.0, 20.0, 1000.0, 1e6])
@pytest.mark.parametrize("m,d", [(1, 128), (75, 64), (75, 128), (70, 256)])
def test_bf16_weights_under_any_cap(m, d, cap):
    """Cached tokens' weights, which are fp32 whatever the keys are: a score errs
    by 2^-21 of its terms, by single tokens and by chunks alike."""
    T = U.torch()
    print(f"[mass] bf16 cap {cap} {m} x {d}", flush=True)
    n, hq = 400, 4
    cache = A.Cache([n], 2, d, "bf16", 16)
    q = A._rows(m, hq, d, "bf16", 3)
    att = kvx.Attention(kvx.ModelShape(2, 2, d, 1e4), hq, kvx.KVX_BF16, softcap=cap)
    k = cache.f64(0, 1, 0)
    lse = T.from_numpy(R.attend(A._f64(q), k, k, d ** -0.5, cap)[1].astype(np.float32)).cuda()
    mass = T.zeros(1, 2, n, device="cuda")
    att.mass(kvx.make_attn_io(cache.struct, A._int([n]), q, lse=lse, layer=1, max_new=m, mass=mass,
                              q_start=A._int([0, m])))
    T.cuda.synchronize()
    given = A._f64(lse)
    ref, size = R.mass(A._f64(q), k, given, d ** -0.5, cap)
    delta = ((d + 8) * EPS + 2.0 ** -21) * size
    tol = ref * (2 * delta + (m * hq + 64) * EPS + 4 * EPS * (np.abs(given).max() + 1)) + 2.0 ** -126
    assert (np.abs(A._f64(mass)[0] - ref) <= tol).all(), (np.abs(A._f64(mass)[0] - ref) / tol).max()
    att.close()
