"""Decoding on a translated cache at the ends of its lengths: contexts that have
outgrown their cache, and lengths whose products pass 32 bits.

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


def _bits(t):
    T = U.torch()
    return t.view(T.int16 if t.dtype == T.bfloat16 else T.int32)


OUTGROWN = [
    # name, dtype, hq, hkv, d, page, slots of each context, new, tokens past the capacity
    ("one", "bf16", 12, 2, 128, 16, [64, 64], 1, 1),
    ("one_contiguous", "f32", 4, 2, 64, 0, [40, 40], 1, 1),
    ("one_far", "bf16", 4, 2, 256, 16, [48, 48], 1, 1000),
    ("chunk_by_one", "bf16", 8, 2, 128, 16, [640, 640], 40, 1),
    ("chunk_by_half", "bf16", 4, 4, 64, 0, [300, 300], 130, 65),
    ("chunk_by_all", "f32", 4, 2, 128, 16, [160, 160], 33, 33),
    ("few_by_some", "bf16", 4, 2, 128, 16, [1024, 1024], 6, 2),
]


@pytest.mark.parametrize("case", OUTGROWN, ids=[c[0] for c in OUTGROWN])
@pytest.mark.parametrize("by_slot", [False, True], ids=["pos", "by_slot"])
def test_append_past_the_capacity(case, by_slot):
    """Slots past the capacity are not stored, and no other slot changes but
    those of the new tokens that fit; queries turn all the same."""
    name, dtype, hq, hkv, d, page, lens, m, over = case
    T = U.torch()
    print(f"[outgrown append] {name}", flush=True)
    cache = A.Cache(lens, hkv, d, dtype, page)
    assert all(n == (cache.table.shape[1] * page if page else lens[0]) for n in lens)
    before = [t.clone() for t in cache.dev]
    rows = m * len(lens)
    x = [A._rows(rows, h, d, dtype, 10 + i) for i, h in enumerate((hq, hkv, hkv))]
    slots = np.concatenate([np.arange(n + over - m, n + over) for n in lens])
    pos = None if by_slot else np.arange(rows, dtype=np.int32)[None] * 7
    att = kvx.Attention(kvx.ModelShape(2, hkv, d, 1e4), hq,
                        kvx.KVX_BF16 if dtype == "bf16" else kvx.KVX_F32)
    q = T.zeros_like(x[0])
    io = kvx.make_attn_io(cache.struct, A._int(n + over for n in lens), q, layer=1, max_new=m,
                          q_start=A._int(A._starts([m] * len(lens))), new_q=x[0], new_k=x[1],
                          new_v=x[2], pos=None if by_slot else T.from_numpy(pos).cuda())
    att.append(io)
    T.cuda.synchronize()
    freq = 1e4 ** (-2.0 * np.arange(d // 2) / d)
    rq, rk = (R.rotate(A._f64(t), slots[None] if by_slot else pos, freq, [0] * (d // 2))
              for t in x[:2])

    def close(got, ref, src):
        pair = np.abs(src[..., :d // 2]) + np.abs(src[..., d // 2:])
        tol = np.concatenate([pair, pair], -1) * (2 * 1.2e-7 + 4 * EPS)
        return (np.abs(got - ref) <= tol + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0)).all()

    assert close(A._f64(q), rq, A._f64(x[0]))
    for r, j in enumerate(slots):
        b = r // m
        if j >= lens[b]:
            continue
        blk, slot = (int(t[0]) for t in cache.place(b, [j]))
        assert close(A._f64(cache.dev[0][1, blk, :, slot]), rk[r], A._f64(x[1][r])), (name, r)
        assert T.equal(cache.dev[1][1, blk, :, slot], x[2][r]), (name, r)
        for t in cache.dev + before:
            t[1, blk, :, slot] = 0
    for t, o in zip(cache.dev, before):
        assert T.equal(_bits(t), _bits(o)), f"{name}: another slot changed"
    att.close()


def _attend(q, k, v, scale, p0, window, prefix):
    """attend() for slots p0 + i of which the cache holds the first len(k)."""
    n, grp = len(k), q.shape[1] // k.shape[1]
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, size = np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
    got = np.zeros((k.shape[1], n))
    for i in range(len(q)):
        see = R.visible(p0 + i, n, window, prefix)
        if not see.any():
            continue
        for h in range(q.shape[1]):
            kh, vh = k[see, h // grp], v[see, h // grp]
            s = scale * (kh @ q[i, h])
            top = s.max()
            e = np.exp(s - top)
            out[i, h], mag[i, h] = e @ vh / e.sum(), e @ np.abs(vh) / e.sum()
            lse[i, h] = top + np.log(e.sum())
            size[i, h] = scale * (np.abs(kh) @ np.abs(q[i, h])).max()
            got[h // grp, see] += np.exp(s - np.float32(lse[i, h]))
    return out, lse, mag, size, got


@pytest.mark.parametrize("case", OUTGROWN, ids=[c[0] for c in OUTGROWN])
@pytest.mark.parametrize("window", [0, 20])
def test_attention_past_the_capacity(case, window):
    """New tokens see what is cached by their own slots' numbers; a window that
    starts past the last slot leaves nothing."""
    name, dtype, hq, hkv, d, page, lens, m, over = case
    T = U.torch()
    print(f"[outgrown attention] {name} window {window}", flush=True)
    cache = A.Cache(lens, hkv, d, dtype, page)
    q = A._rows(m * len(lens), hq, d, dtype, 3)
    att = kvx.Attention(kvx.ModelShape(2, hkv, d, 1e4), hq,
                        kvx.KVX_BF16 if dtype == "bf16" else kvx.KVX_F32)
    out = T.full_like(q, 7.0)
    lse = T.full((m * len(lens), hq), 7.0, device="cuda")
    kw = dict(layer=1, max_new=m, window=window, q_start=A._int(A._starts([m] * len(lens))))
    tokens = A._int(n + over for n in lens)
    ws = att.workspace()
    ws.fill_(0xFF)
    att.forward(kvx.make_attn_io(cache.struct, tokens, q, out=out, lse=lse, **kw), ws)
    room = max(lens)
    mass = T.full((len(lens), hkv, room), 7.0, device="cuda")
    refs = [_attend(A._f64(q)[b * m:b * m + m], cache.f64(0, 1, b), cache.f64(1, 1, b), d ** -0.5,
                    n + over - m, window, 0) for b, n in enumerate(lens)]
    given = T.from_numpy(np.concatenate([r[1] for r in refs]).astype(np.float32)).cuda()
    att.mass(kvx.make_attn_io(cache.struct, tokens, q, lse=given, mass=mass, **kw))
    T.cuda.synchronize()
    oh, lh, mh = A._f64(out), A._f64(lse), A._f64(mass)
    for b, n in enumerate(lens):
        sl = slice(b * m, b * m + m)
        ro, rl, mag, size, weight = refs[b]
        delta = A._delta(size, d, 0.0)
        rel = 2 * delta + (n + 64) * EPS + (2.0 ** -8 if dtype == "bf16" else 0.0)
        tol = mag * rel[..., None] + (2.0 ** -8 * np.abs(ro) if dtype == "bf16" else 0.0)
        assert (np.abs(oh[sl] - ro) <= tol).all(), (name, b)
        seen = np.isfinite(rl)
        assert (lh[sl][~seen] == -np.inf).all(), (name, b)
        err = np.abs(lh[sl][seen] - rl[seen])
        assert (err <= delta[seen] + (n + 64) * EPS + 2.0 ** -22 * (1 + np.abs(rl[seen]))).all()
        rel = 2 * _top(delta) + (m * hq + 64) * EPS + 4 * EPS * (np.abs(rl[seen]).max(initial=0) + 1)
        assert (np.abs(mh[b] - weight) <= weight * rel + 2 * EPS * weight + 2.0 ** -126).all()
    att.close()


def _top(x):
    return x.max(initial=0.0)


def _repeated(n, page, blocks, d, dtype, seed=0):
    """One context of n slots of one KV head, whose table names `blocks` blocks
    over and over: (cache, rows(kv, slots))."""
    T = U.torch()
    g = T.Generator().manual_seed(seed)
    dev = [T.randn(1, blocks, 1, page, d, generator=g).to(A._dt(dtype)) for _ in range(2)]
    table = (T.arange(-(-n // page), dtype=T.int32) * 5 % blocks).view(1, -1).cuda()
    host = [A._f64(t) for t in dev]
    gpu = [t.cuda() for t in dev]

    def rows(kv, j):
        return host[kv][0, j // page * 5 % blocks, :, j % page]

    return kvx.make_cache(gpu[0], gpu[1], table), rows


@pytest.mark.parametrize("hq,n,m", [(128, 17_000_011, 1), (32, 67_200_003, 1), (128, 17_000_011, 2)])
def test_attention_of_slots_times_heads_past_32_bits(hq, n, m):
    """A cache so long that its slots times the heads of a group pass 2^31;
    blocks repeat, so that it takes little memory, and a window bounds the work."""
    T = U.torch()
    print(f"[long attention] {hq} heads, {n} slots", flush=True)
    assert n * hq > 2 ** 31
    d, window = 64, 3000
    cache, rows = _repeated(n, 64, 7, d, "bf16")
    q = A._rows(m, hq, d, "bf16", 3)
    att = kvx.Attention(kvx.ModelShape(1, 1, d, 1e4), hq, kvx.KVX_BF16)
    out, lse = T.zeros_like(q), T.zeros(m, hq, device="cuda")
    att.forward(kvx.make_attn_io(cache, A._int([n]), q, out=out, lse=lse, window=window, max_new=m,
                                 q_start=A._int([0, m])), att.workspace())
    T.cuda.synchronize()
    j = np.arange(n - window - m, n)
    ro, rl, mag, size = R.attend(A._f64(q), rows(0, j), rows(1, j), d ** -0.5, 0.0, window)
    delta = A._delta(size, d, 0.0)
    tol = mag * (2 * delta + (window + 64) * EPS + 2.0 ** -8)[..., None] + 2.0 ** -8 * np.abs(ro)
    assert (np.abs(A._f64(out) - ro) <= tol).all()
    assert (np.abs(A._f64(lse) - rl) <= delta + (window + 64) * EPS + 2.0 ** -22 * (1 + np.abs(rl))).all()
    att.close()


@pytest.mark.parametrize("hq,n,m", [(128, 17_000_011, 1), (256, 9_000_011, 2)])
def test_weights_of_slots_times_heads_past_32_bits(hq, n, m):
    """The same of the cached tokens' weights: those that a window leaves out,
    which are nearly all, stay as they were."""
    T = U.torch()
    print(f"[long weights] {hq} heads, {n} slots", flush=True)
    assert n * hq > 2 ** 31
    d, window = 64, 3000
    cache, rows = _repeated(n, 64, 7, d, "bf16")
    q = A._rows(m, hq, d, "bf16", 3)
    att = kvx.Attention(kvx.ModelShape(1, 1, d, 1e4), hq, kvx.KVX_BF16)
    j = np.arange(n - window - m, n)
    _, rl, _, _ = R.attend(A._f64(q), rows(0, j), rows(1, j), d ** -0.5, 0.0, window)
    lse = T.from_numpy(rl.astype(np.float32)).cuda()
    mass = T.full((1, 1, n), 0.5, device="cuda")
    att.mass(kvx.make_attn_io(cache, A._int([n]), q, lse=lse, window=window, max_new=m,
                              q_start=A._int([0, m]), mass_in=mass, mass=mass))
    T.cuda.synchronize()
    assert (mass[0, 0, :int(j[0]) + 1] == 0.5).all()
    ref, size = R.mass(A._f64(q), rows(0, j), A._f64(lse), d ** -0.5, 0.0, window)
    rel = 2 * A._delta(size, d, 0.0) + (m * hq + 64) * EPS + 4 * EPS * (np.abs(rl).max() + 1)
    got = A._f64(mass[0, 0, int(j[0]):])
    assert (np.abs(got - 0.5 - ref[0]) <= ref[0] * rel + 2 * EPS * (0.5 + ref[0]) + 2.0 ** -126).all()
    att.close()


def test_weights_in_a_cache_of_far_more_slots_than_tokens():
    """Room for 131072 slots in each of 1100 contexts of 70 tokens: more workgroups
    by the room than a launch has."""
    T = U.torch()
    print("[mass] room for 144 million slots", flush=True)
    batch, hkv, hq, d, page, n, m = 1100, 8, 128, 16, 16, 70, 3
    room = 131072
    assert room // 128 * batch * hkv * 512 > 2 ** 32
    per = -(-n // page)
    table = T.full((batch, room // page), 2 ** 30, dtype=T.int32, device="cuda")
    table[:, :per] = T.arange(batch * per, dtype=T.int32, device="cuda").view(batch, per)
    g = T.Generator("cuda").manual_seed(0)
    k = T.randn(1, batch * per, hkv, page, d, device="cuda", generator=g).bfloat16()
    q = T.randn(batch * m, hq, d, device="cuda", generator=g).bfloat16()
    lse = T.full((batch * m, hq), 4.5, device="cuda")
    mass = T.full((batch, hkv, room), 7.0, device="cuda")
    att = kvx.Attention(kvx.ModelShape(1, hkv, d, 1e4), hq, kvx.KVX_BF16)
    att.mass(kvx.make_attn_io(kvx.make_cache(k, k, table), A._int([n] * batch), q, lse=lse, mass=mass,
                              max_new=m, q_start=A._int(range(0, batch * m + 1, m))))
    T.cuda.synchronize()
    assert (mass[:, :, n:] == 0).all()
    kh, qh, got = A._f64(k), A._f64(q), A._f64(mass[:, :, :n])
    for b in range(0, batch, 61):
        rows = kh[0, b * per:b * per + per].transpose(0, 2, 1, 3).reshape(per * page, hkv, d)[:n]
        ref, size = R.mass(qh[b * m:b * m + m], rows, np.full((m, hq), 4.5), d ** -0.5)
        rel = 2 * A._delta(size, d, 0.0) + (m * hq + 64) * EPS + 4 * EPS * 5.5
        assert (np.abs(got[b] - ref) <= ref * rel + 2.0 ** -126).all(), b
    att.close()
