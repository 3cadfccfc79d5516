"""Serving on caches of 8 bits, with sinks and drafted trees, on the GPU, against
the fp64 reference.

Tolerances are those of decoding (test_attn_gpu.py): a score is an fp32 sum of D
exact products and a few more roundings, so off by (D + 8) 2^-24 of its terms'
magnitudes, with a tanh cap by another 2^-22 cap; bf16 rounds a weight and an
output by 2^-8 of them.  Numbers of 8 bits enter exactly, scales are powers of two.
"""
import numpy as np
import pytest

from oracle import attn as R
from oracle import serve as V
from paper_2608_30963_amd import kvx
from tests import gpu_util as U
from tests.serve_util import DT, Cache8, masks, random_tree
from tests.test_attn_gpu import EPS, Cache, _delta, _dt, _f64, _int, _rows, _starts

pytestmark = pytest.mark.gpu


def _attention(dtype, hkv, d, hq, cap=0.0, layers=2, **kw):
    return kvx.Attention(kvx.ModelShape(layers, hkv, d, 1e4), hq,
                         kvx.KVX_BF16 if dtype == "bf16" else kvx.KVX_F32, softcap=cap, **kw)


VIEWS = [
    # name, dtype, code ("": dtype's), hq, hkv, d, page, (new, cached), options
    # options: window, sink, prefix, cap, tree (roots), strided, scale, depth (False: none given)
    ("i8_one", "bf16", "i8", 12, 2, 128, 16, [(1, 300)], {}),
    ("i8_one_slot", "bf16", "i8", 4, 4, 64, 16, [(1, 1)], {}),
    ("i8_ragged", "bf16", "i8", 28, 4, 128, 16, [(1, 700), (1, 1), (1, 64), (1, 65), (1, 1023)], {}),
    ("i8_long", "bf16", "i8", 7, 1, 128, 64, [(1, 9001)], {}),
    ("i8_group_33", "bf16", "i8", 33, 1, 64, 16, [(1, 500), (1, 40)], {}),
    ("i8_256", "bf16", "i8", 8, 4, 256, 32, [(1, 900), (1, 30)], dict(cap=50.0)),
    ("e4m3_one", "bf16", "e4m3", 12, 2, 128, 16, [(1, 300)], {}),
    ("e4m3_ragged", "bf16", "e4m3", 28, 4, 128, 0, [(1, 700), (1, 1), (1, 64), (1, 65)], {}),
    ("e4m3_256", "bf16", "e4m3", 8, 4, 256, 16, [(1, 900), (1, 33)], dict(cap=30.0)),
    ("e4m3_80", "bf16", "e4m3", 6, 2, 80, 48, [(1, 300), (1, 3)], {}),
    ("i8_16", "bf16", "i8", 3, 1, 16, 5, [(33, 100), (1, 9)], {}),
    ("e4m3_192", "bf16", "e4m3", 4, 2, 192, 16, [(40, 130)], {}),
    ("i8_few", "bf16", "i8", 12, 2, 128, 16, [(3, 200), (5, 5), (2, 77)], {}),
    ("i8_chunk", "bf16", "i8", 12, 2, 128, 16, [(150, 400)], {}),
    ("e4m3_chunk", "bf16", "e4m3", 14, 2, 128, 48, [(100, 333), (1, 50), (0, 20), (37, 37)], {}),
    ("e4m3_chunk_64", "bf16", "e4m3", 4, 2, 64, 16, [(260, 260)], {}),
    ("i8_chunk_256", "bf16", "i8", 8, 4, 256, 32, [(140, 500), (64, 64)], dict(cap=50.0)),
    ("i8_chunk_80", "bf16", "i8", 2, 2, 80, 7, [(131, 200)], {}),
    ("i8_chunk_prefix", "bf16", "i8", 6, 2, 96, 16, [(90, 120), (60, 61)], dict(prefix=[70, 61])),
    ("i8_window", "bf16", "i8", 6, 2, 128, 16, [(90, 220), (1, 300)], dict(window=64)),
    ("i8_sink", "bf16", "i8", 8, 2, 128, 16, [(1, 500), (1, 30)], dict(window=100, sink=4)),
    ("e4m3_sink_chunk", "bf16", "e4m3", 8, 2, 128, 16, [(90, 500), (10, 30)], dict(window=100, sink=40)),
    ("i8_strided", "bf16", "i8", 4, 2, 64, 16, [(30, 90), (1, 40)], dict(strided=True)),
    ("e4m3_strided", "bf16", "e4m3", 4, 2, 128, 0, [(1, 90), (1, 40)], dict(strided=True)),
    ("i8_large_scores", "bf16", "i8", 4, 2, 128, 16, [(40, 200), (1, 150)], dict(scale=30.0)),
    ("i8_tiny", "bf16", "i8", 4, 2, 128, 16, [(40, 200), (1, 150)], dict(size=2.0 ** -60)),
    ("before_first", "bf16", "e4m3", 4, 2, 64, 16, [(20, 12), (5, 0), (6, 6)], {}),
    ("i8_many", "bf16", "i8", 4, 1, 64, 16, [(1, 1 + 13 * i % 97) for i in range(300)], {}),
    ("sink_one", "bf16", "", 8, 4, 256, 32, [(1, 900), (1, 30), (1, 129)], dict(window=128, sink=4, cap=50.0)),
    ("sink_into_window", "bf16", "", 4, 2, 128, 16, [(1, 300), (1, 131)], dict(window=128, sink=64)),
    ("sink_past_window", "bf16", "", 4, 2, 128, 16, [(1, 300)], dict(window=40, sink=280)),
    ("sink_past_all", "bf16", "", 4, 2, 128, 16, [(30, 300)], dict(window=40, sink=1000)),
    ("sink_f32", "f32", "", 6, 2, 128, 0, [(1, 600), (1, 31)], dict(window=33, sink=5)),
    ("sink_chunk", "bf16", "", 8, 4, 256, 32, [(140, 500), (64, 64)], dict(window=50, sink=4, cap=50.0)),
    ("sink_chunk_1", "bf16", "", 2, 1, 64, 16, [(70, 300)], dict(window=1, sink=1)),
    ("sink_chunk_f32", "f32", "", 6, 2, 128, 0, [(75, 410), (20, 33)], dict(window=100, sink=70)),
    ("sink_chunk_f32_256", "f32", "", 4, 2, 256, 16, [(70, 240)], dict(cap=50.0, window=64, sink=3)),
    ("sink_prefix", "bf16", "", 6, 2, 128, 16, [(90, 220)], dict(prefix=[200], window=64, sink=20)),
    ("sink_long", "bf16", "", 7, 1, 128, 64, [(1, 9001), (40, 5000)], dict(window=4096, sink=128)),
    ("sink_strided", "bf16", "", 4, 2, 64, 16, [(30, 90), (1, 70)], dict(window=20, sink=3, strided=True)),
    ("sink_before_first", "bf16", "", 4, 2, 64, 16, [(20, 12), (5, 0), (6, 6)], dict(window=4, sink=2)),
    ("sink_none_seen", "f32", "", 2, 1, 64, 16, [(1, 0), (1, 3)], dict(window=4, sink=2)),
    ("tree_4", "bf16", "", 28, 4, 128, 16, [(4, 300), (4, 4), (3, 64)], dict(tree=1)),
    ("tree_16", "bf16", "", 12, 2, 128, 16, [(16, 1000)], dict(tree=1)),
    ("tree_16_f32", "f32", "", 12, 2, 128, 16, [(16, 400), (7, 7)], dict(tree=1)),
    ("tree_64", "bf16", "", 28, 4, 128, 16, [(64, 700), (33, 90), (1, 20), (0, 9)], dict(tree=1)),
    ("tree_100", "bf16", "", 4, 4, 64, 0, [(100, 333), (65, 65)], dict(tree=2)),
    ("tree_cap_256", "bf16", "", 8, 4, 256, 32, [(20, 500), (31, 64)], dict(tree=1, cap=50.0)),
    ("tree_window", "bf16", "", 8, 2, 128, 16, [(40, 500), (12, 20)], dict(tree=1, window=64, sink=4)),
    ("tree_window_3", "bf16", "", 8, 2, 128, 16, [(40, 500), (12, 20)], dict(tree=1, window=3, sink=2)),
    ("tree_i8", "bf16", "i8", 28, 4, 128, 16, [(64, 700), (33, 90), (1, 20)], dict(tree=1)),
    ("tree_e4m3", "bf16", "e4m3", 12, 2, 128, 16, [(4, 700), (2, 9)], dict(tree=1)),
    ("tree_i8_256", "bf16", "i8", 8, 4, 256, 16, [(20, 300)], dict(tree=1, cap=30.0, window=100, sink=4)),
    ("tree_no_depth", "bf16", "", 8, 2, 128, 16, [(40, 500)], dict(tree=1, depth=False)),
    ("tree_before_first", "bf16", "", 4, 2, 64, 16, [(20, 12), (5, 0)], dict(tree=3)),
    # more contexts than a wave has lanes, pieces of chunks by their lengths
    ("tree_many", "bf16", "i8", 4, 1, 64, 16, [(9 + i % 30, 50 + 37 * i % 400) for i in range(90)],
     dict(tree=1)),
    ("chunk_many", "bf16", "", 4, 1, 64, 16, [(9 + i % 30, 50 + 37 * i % 400) for i in range(90)],
     dict(window=40, sink=5)),
    ("chunk_uneven", "bf16", "e4m3", 8, 2, 128, 16, [(20, 3000), (20, 40), (0, 5), (20, 700)], {}),
    ("one_of_many", "bf16", "i8", 8, 2, 128, 64, [(1, 20000)] + [(1, 3)] * 5, {}),
    # contiguous caches whose last 16 slots are not all there, at an edge of the window
    ("contiguous_37", "bf16", "i8", 8, 2, 128, 0, [(1, 37), (1, 20)], dict(window=9, sink=2)),
    ("contiguous_101", "bf16", "", 8, 2, 128, 0, [(1, 101), (1, 5), (1, 97)], dict(window=30, sink=3)),
    ("contiguous_chunk_77", "bf16", "e4m3", 8, 2, 128, 0, [(20, 77), (12, 61)], dict(window=30, sink=3)),
    ("group_16", "bf16", "i8", 16, 1, 128, 16, [(1, 700)], {}),
    ("group_17", "bf16", "i8", 17, 1, 128, 16, [(1, 700)], dict(window=300, sink=9)),
    ("group_17_e4m3", "bf16", "e4m3", 17, 1, 256, 16, [(1, 333)], dict(cap=20.0)),
    ("group_32", "bf16", "", 32, 1, 128, 16, [(1, 700)], dict(window=300, sink=9)),
    ("cap_large", "bf16", "i8", 4, 2, 128, 16, [(1, 200), (1, 40)], dict(cap=1000.0)),
    ("cap_large_chunk", "bf16", "e4m3", 4, 2, 128, 16, [(40, 200)], dict(cap=1000.0)),
    ("few_nodes_window", "bf16", "e4m3", 4, 2, 128, 16, [(8, 300), (3, 9)], dict(tree=2, window=20, sink=4)),
]


def _problem(dtype, code, hq, hkv, d, page, spec, opt, seed=0, extra=0):
    new, lens = [m for m, _ in spec], [n for _, n in spec]
    if code:
        cache = Cache8(lens, hkv, d, code, page, strided=opt.get("strided", False), seed=seed,
                       extra=extra, size=opt.get("size", 1.0))
    else:
        cache = Cache(lens, hkv, d, dtype, page, flash=opt.get("strided", False), seed=seed, extra=extra)
    starts = _starts(new)
    q = _rows(starts[-1], hq, d, dtype, seed + 1, opt.get("scale", 1.0) / opt.get("size", 1.0),
              3 if opt.get("strided") else 0)
    kw = dict(layer=1, max_new=max(new), window=opt.get("window", 0), sink=opt.get("sink", 0),
              q_start=None if all(m == 1 for m in new) else _int(starts),
              prefix=_int(opt["prefix"]) if "prefix" in opt else None)
    sights, depths = [], []
    rng = np.random.default_rng(seed + 5)
    words = -(-max(new) // 32)
    tree = np.zeros((starts[-1], words), np.int32)
    for b, (m, n) in enumerate(spec):
        if "tree" in opt:
            up = random_tree(m, rng, opt["tree"])
            see, depth = V.tree_sight(up, n, opt.get("window", 0), opt.get("sink", 0))
            nodes = V.tree_sight(up, 10 ** 4 + m, opt.get("window", 0), 0)[0][:, 10 ** 4:]
            if opt.get("sink"):
                nodes = nodes | np.array([[see[i, n - m + k] if n - m + k >= 0 else False for k in range(m)]
                                          for i in range(m)]).reshape(m, m)
            tree[starts[b]:starts[b + 1]] = masks(up, nodes, words)
            if opt.get("depth", True) is False:  # rows in order: no window to count in
                depth = list(range(m))
            depths += depth
        else:
            see = V.sight(m, n, opt.get("window", 0), opt.get("sink", 0),
                          opt["prefix"][b] if "prefix" in opt else 0)
        sights.append(see)
    if "tree" in opt:
        kw.update(tree=U.torch().from_numpy(tree).cuda(), q_start=_int(starts),
                  depth=_int(depths) if opt.get("depth", True) else None)
    return cache, q, starts, _int(lens), kw, sights


def check_rows(name, dtype, d, cap, qh, oh, lh, k, v, see):
    """One context's outputs and log-sum-exp against the reference's."""
    n = see.shape[1]
    ro, rl, mag, size = V.attend(qh, k, v, see, d ** -0.5, cap)
    delta = _delta(size, d, cap)
    rel = 2 * delta + (n + 64) * EPS
    if dtype == "bf16":
        rel = rel + 2.0 ** -8
    tol = mag * rel[..., None] + (2.0 ** -8 * np.abs(ro) if dtype == "bf16" else 0.0)
    # numbers below 2^-126 may count as zero: each of n weights, times a value, and
    # the output (codes are often zero, so that nothing larger stands beside them)
    tol = tol + 2.0 ** -126 * (1 + n * np.abs(v).max(initial=0.0))
    assert np.isfinite(oh).all(), f"{name}: non-finite output"
    worst = np.abs(oh - ro) - tol
    assert worst.max(initial=-1) <= 0, f"{name}: {worst.max()} over"
    seen = np.isfinite(rl)
    assert (lh[~seen] == -np.inf).all(), f"{name}: lse of an empty row"
    ltol = delta + (n + 64) * EPS + 2.0 ** -22 * (1 + np.abs(np.where(seen, rl, 0.0)))
    err = np.abs(np.where(seen, lh, 0.0) - np.where(seen, rl, 0.0))
    assert (err <= ltol).all(), f"{name}: lse off by {err.max()}"


@pytest.mark.parametrize("case", VIEWS, ids=[c[0] for c in VIEWS])
def test_forward_view(case):
    name, dtype, code, hq, hkv, d, page, spec, opt = case
    T = U.torch()
    print(f"[view] {name}", flush=True)
    cache, q, starts, tokens, kw, sights = _problem(dtype, code, hq, hkv, d, page, spec, opt)
    cap = opt.get("cap", 0.0)
    att = _attention(dtype, hkv, d, hq, cap)
    pad = 3 if opt.get("strided") else 0
    wide = T.full((starts[-1], hq + pad, d), 7.0, dtype=_dt(dtype), device="cuda")
    out = wide[:, :hq]
    lse = T.full((starts[-1], hq), float("nan"), device="cuda")
    io = kvx.make_attn_io(cache.struct, tokens, q, out=out, lse=lse, **kw)
    ws = att.workspace(io)
    ws.fill_(0xFF)  # NaN wherever read before written
    att.forward(io, ws)
    T.cuda.synchronize()
    if pad:
        assert (wide[:, hq:] == 7.0).all(), "wrote outside its rows"
    first, first_lse = out.clone(), lse.clone()
    ws.fill_(0)
    att.forward(io, ws)
    T.cuda.synchronize()
    assert T.equal(first.view(-1, d), out.reshape(-1, d)) and T.equal(first_lse, lse), "bits differ"
    qh, oh, lh = _f64(q), _f64(out), _f64(lse)
    for b in range(len(spec)):
        sl = slice(starts[b], starts[b + 1])
        check_rows(f"{name} context {b}", dtype, d, cap, qh[sl], oh[sl], lh[sl], cache.f64(0, 1, b),
                   cache.f64(1, 1, b), sights[b])
    att.close()


def test_empty_view_is_forward():
    """No sinks, no tree and the model's own cache: the plain call's bits."""
    T = U.torch()
    for m, window in ((1, 0), (50, 30)):
        cache = Cache([200], 2, 64, "bf16", 16)
        q = _rows(m, 4, 64, "bf16", 1)
        att = _attention("bf16", 2, 64, 4)
        ws, outs = att.workspace(), []
        for view in (None, kvx.AttnView(), False):
            out = T.zeros_like(q)
            io = kvx.make_attn_io(cache.struct, _int([200]), q, out=out, layer=1, max_new=m,
                                  q_start=_int([0, m]), window=window)
            if view is False:
                att.forward(io, ws)
            else:
                kvx.kvx_attn_forward_view(att.handle, io, view, ws)
            T.cuda.synchronize()
            outs.append(out)
        assert T.equal(outs[0], outs[2]) and T.equal(outs[1], outs[2])
        att.close()


def test_hidden_numbers_may_be_anything():
    """NaN, infinities, NaN scales and codes that are no numbers in slots that a row does
    not see change no bit of it; rows that see a NaN are NaN."""
    T = U.torch()
    for dtype, code, m, n, window, sink, tree in (
            ("bf16", "", 40, 200, 30, 4, 0), ("f32", "", 40, 200, 30, 4, 0), ("bf16", "", 1, 200, 30, 4, 0),
            ("bf16", "", 24, 100, 0, 0, 1), ("bf16", "", 3, 100, 0, 0, 1), ("f32", "", 24, 100, 0, 0, 1),
            ("bf16", "i8", 40, 200, 30, 4, 0), ("bf16", "e4m3", 1, 200, 30, 4, 0),
            ("bf16", "e4m3", 24, 100, 0, 0, 1), ("bf16", "i8", 3, 100, 0, 0, 1),
            ("bf16", "e4m3", 130, 300, 0, 0, 0), ("bf16", "i8", 2, 70, 0, 0, 0)):
        print(f"[hidden] {dtype} {code} {m} of {n}, window {window}", flush=True)
        opt = dict(window=window, sink=sink)
        if tree:
            opt["tree"] = tree
        cache, q, starts, tokens, kw, sights = _problem(dtype, code, 8, 2, 64, 16, [(m, n)], opt)
        att = _attention(dtype, 2, 64, 8)
        ws, outs = att.workspace(), []
        bad = sorted({n - 1} | ({n - m // 2 - 1} if m > 2 else set()) | ({6, 33} if window else set()))
        for spoiled in (False, True):
            for i, j in enumerate(bad if spoiled else []):
                blk, slot = (int(x[0]) for x in cache.place(0, [j]))
                if not code:
                    for e in range(2):
                        cache.dev[e][1, blk, :, slot] = float("nan") if i % 2 == e else float("inf")
                elif i % 2 or code == "i8":
                    cache.dscale[1, blk, :, slot] = float("nan")
                else:
                    cache.dev[0][1, blk, :, slot] = 127  # no number
                    cache.dev[1][1, blk, :, slot] = 255
            out = T.zeros_like(q)
            att.forward(kvx.make_attn_io(cache.struct, tokens, q, out=out, **kw), ws)
            T.cuda.synchronize()
            outs.append(_f64(out))
        hidden = 0
        for i in range(m):
            if sights[0][i, bad].any():
                assert np.isnan(outs[1][i]).all(), (dtype, code, i)
            else:
                hidden += 1
                assert (outs[0][i] == outs[1][i]).all(), (dtype, code, i)
        assert hidden or m == 1 or window
        att.close()


@pytest.mark.parametrize("dtype,code,m,d", [("bf16", "", 1, 128), ("bf16", "i8", 1, 128),
                                            ("bf16", "e4m3", 140, 128), ("f32", "", 70, 64),
                                            ("bf16", "i8", 70, 256)])
def test_view_of_scores_that_rise(dtype, code, m, d):
    """Scores from -200 to 200 along the slots, and the other way round, through a
    window with sinks at the far end."""
    T = U.torch()
    n, hq = 900, 4
    for rising in (1.0, -1.0):
        opt = dict(window=700, sink=50)
        cache, q, starts, tokens, kw, sights = _problem(dtype, code, hq, 2, d, 64, [(m, n)], opt)
        g = T.Generator().manual_seed(8)
        rows = T.randn(n, 2, d, generator=g) * 0.1
        rows[..., 0] += T.linspace(-200.0, 200.0, n)[:, None] * rising
        blk, slot = cache.place(0, np.arange(n))
        if code:
            c, s = V.encode(rows.numpy(), code)
            cache.dev[0][1, blk, :, slot] = T.from_numpy(c).cuda()
            cache.dscale[1, blk, :, slot, 0] = T.from_numpy(s).bfloat16().cuda()
            k = V.decode(c, s, code)
        else:
            cache.dev[0][1, blk, :, slot] = rows.to(_dt(dtype)).cuda()
            k = _f64(rows.to(_dt(dtype)))
        q = q * 0.1
        q[..., 0] = d ** 0.5
        att = _attention(dtype, 2, d, hq)
        out, lse = T.zeros_like(q), T.zeros(m, hq, device="cuda")
        att.forward(kvx.make_attn_io(cache.struct, tokens, q, out=out, lse=lse, **kw), att.workspace())
        T.cuda.synchronize()
        check_rows(f"{dtype} {code} {rising}", dtype, d, 0.0, _f64(q), _f64(out), _f64(lse), k,
                   cache.f64(1, 1, 0), sights[0])
        att.close()


# ---------------------------------------------------------------------------
# Caches of 8 bits: written and read back
# ---------------------------------------------------------------------------

PACK = [
    # name, dtype, code, layers, hkv, d, page (plain), page (coded), lens, options
    ("one", "bf16", "i8", 1, 1, 64, 16, 16, [1], {}),
    ("i8", "bf16", "i8", 3, 2, 128, 16, 16, [200, 61, 0], {}),
    ("e4m3", "bf16", "e4m3", 3, 2, 128, 16, 32, [200, 61, 1], {}),
    ("f32_i8", "f32", "i8", 2, 3, 80, 7, 0, [90, 33], {}),
    ("f32_e4m3", "f32", "e4m3", 2, 1, 256, 0, 5, [90, 133], {}),
    ("e4m3_256", "bf16", "e4m3", 2, 4, 256, 32, 32, [300, 299], {}),
    ("i8_192", "bf16", "i8", 2, 2, 192, 16, 48, [130], {}),
    ("i8_16", "bf16", "i8", 2, 2, 16, 3, 16, [45], {}),
    ("strided", "bf16", "e4m3", 2, 2, 64, 16, 16, [70, 20], dict(strided=True)),
    ("long", "bf16", "i8", 1, 1, 128, 64, 64, [20001], {}),
]


def _values(x, kind, rng):
    """Rows that are hard to code."""
    if kind == "sizes":
        x = x * 2.0 ** rng.integers(-60, 60, x.shape[:-1] + (1,))
    elif kind == "edges":
        # ties, largest codes and the borders of scales
        x = rng.choice([0.0, 0.5, 1.5, 2.5, 126.5, 127.0, 127.5, 128.0, 432.0, 448.0, 464.0, -448.0,
                        -127.0, 17.0, 18.0, 19.0], x.shape)
        x = x * 2.0 ** rng.integers(-20, 20, x.shape[:-1] + (1,))
    elif kind == "special":
        x = rng.choice([0.0, -0.0, 1.0, 2.0 ** -126, 3.0e38, -3.3e38, 2.0 ** 127, 1e-40], x.shape)
        x[::3] = 0.0
        x.reshape(-1, x.shape[-1])[::5, 3] = np.nan
        x.reshape(-1, x.shape[-1])[1::7, -1] = np.inf
    return x


@pytest.mark.parametrize("kind", ["plain", "sizes", "edges", "special"])
@pytest.mark.parametrize("case", PACK, ids=[c[0] for c in PACK])
def test_pack_and_unpack(case, kind):
    name, dtype, code, layers, hkv, d, page, page8, lens, opt = case
    T = U.torch()
    print(f"[pack] {name} {kind}", flush=True)
    flash = opt.get("strided", False)
    cache = Cache(lens, hkv, d, dtype, page, layers=layers, flash=flash)
    coded = Cache8(lens, hkv, d, code, page8, layers=layers, strided=flash)
    rng = np.random.default_rng(3)
    src = [[[None] * len(lens) for _ in range(layers)] for _ in range(2)]
    for kv in range(2):
        view = cache.dev[kv].transpose(2, 3) if flash else cache.dev[kv]
        for l in range(layers):
            for b, n in enumerate(lens):
                x = T.from_numpy(_values(rng.standard_normal((n, hkv, d)), kind, rng)).to(_dt(dtype))
                blk, slot = cache.place(b, np.arange(n))
                view[l, blk, :, slot] = x.cuda()
                src[kv][l][b] = _f64(x)
    for t in coded.base[:2]:
        t.fill_(55)
    coded.base[2].fill_(3.0)
    att = _attention(dtype, hkv, d, hkv, layers=layers)
    io = kvx.make_pack_io(cache.struct, coded.struct, _int(lens))
    att.pack(io)
    T.cuda.synchronize()
    written = 0
    for kv in range(2):
        for l in range(layers):
            for b, n in enumerate(lens):
                c, s = coded.read(kv, l, b, np.arange(n))
                rc, rs = V.encode(src[kv][l][b], code)
                assert (c == rc).all(), (name, kv, l, b, np.argwhere(c != rc)[:4])
                assert ((s == rs) | (np.isnan(s) & np.isnan(rs))).all(), (name, kv, l, b)
                written += n * hkv
    left = sum(int((t == 55).all(-1).sum()) for t in coded.dev)
    rows = 2 * int(np.prod(coded.dev[0].shape[:-1]))
    assert left >= rows - written, "wrote elsewhere"
    assert int((coded.base[2] == 3.0).sum()) == coded.base[2].numel() - written
    # and back
    for t in cache.dev:
        t.fill_(9.0)
    att.unpack(io)
    T.cuda.synchronize()
    for kv in range(2):
        for l in range(layers):
            for b, n in enumerate(lens):
                got = _f64(cache.read(kv, l, b, n))
                ref = V.decode(*V.encode(src[kv][l][b], code), code)
                assert ((got == ref) | (np.isnan(got) & np.isnan(ref))).all(), (name, kv, l, b)
    left = sum(int((t == 9.0).all(-1).sum()) for t in cache.dev)
    assert left >= 2 * int(np.prod(cache.dev[0].shape[:-1])) - written, "wrote elsewhere"
    att.close()


APPEND = [
    # name, code, hq, hkv, d, page, (new, cached), axes, options
    ("one", "i8", 12, 2, 128, 16, [(1, 300)], 1, {}),
    ("decode", "e4m3", 28, 4, 128, 16, [(1, 17 * i + 1) for i in range(9)], 1, {}),
    ("chunk_axes", "i8", 4, 2, 128, 16, [(33, 100), (0, 8), (70, 70)], 3, {}),
    ("d80", "e4m3", 3, 1, 80, 7, [(21, 60), (2, 2)], 2, {}),
    ("d256", "i8", 8, 4, 256, 0, [(5, 5), (1, 9)], 1, {}),
    ("by_slot", "e4m3", 4, 4, 64, 16, [(10, 45), (3, 3)], 1, dict(pos=None)),
    ("far", "i8", 2, 1, 128, 16, [(6, 50)], 1, dict(pos=2 ** 30)),
    ("before_first_slot", "e4m3", 4, 2, 64, 16, [(9, 4), (3, 0)], 1, {}),
    ("strided", "i8", 4, 2, 64, 16, [(8, 40), (4, 4)], 1, dict(strided=True)),
    ("d16", "e4m3", 2, 1, 16, 3, [(5, 9)], 4, {}),
    ("prompts", "e4m3", 7, 1, 128, 16, [(500, 900), (333, 333)], 1, {}),
]


@pytest.mark.parametrize("case", APPEND, ids=[c[0] for c in APPEND])
def test_append_coded(case):
    name, code, hq, hkv, d, page, spec, axes, opt = case
    T = U.torch()
    print(f"[append8] {name}", flush=True)
    new, lens = [m for m, _ in spec], [n for _, n in spec]
    starts = _starts(new)
    rows = int(starts[-1])
    cache = Cache8(lens, hkv, d, code, page, strided=opt.get("strided", False))
    before = [t.clone() for t in cache.base]
    x = [_rows(rows, h, d, "bf16", 10 + i, pad=3 if opt.get("strided") else 0)
         for i, h in enumerate((hq, hkv, hkv))]
    if rows > 2:
        x[1][1, 0, 3] = float("inf")
        x[2][2, hkv - 1, d - 1] = float("nan")
    rng = np.random.default_rng(1)
    axis = [e % axes for e in range(d // 2)]
    slots = np.concatenate([np.arange(n - m, n) for m, n in spec])
    pos = None
    if opt.get("pos", 0) is not None:
        pos = rng.integers(0, 5000, (axes, rows)).astype(np.int32) + np.int32(opt.get("pos", 0))
    att = _attention("bf16", hkv, d, hq, pair_axis=axis)
    q = T.zeros((rows, hq, d), dtype=T.bfloat16, device="cuda")
    kw = dict(layer=1, q_start=_int(starts), max_new=max(new),
              pos=None if pos is None else T.from_numpy(pos).cuda())
    att.append(kvx.make_attn_io(cache.struct, _int(lens), q, new_q=x[0], new_k=x[1], new_v=x[2], **kw))
    T.cuda.synchronize()
    # queries as the plain call's, but for the sine's and cosine's last bits
    at = np.broadcast_to(slots, (axes, rows)) if pos is None else pos
    freq = 1e4 ** (-2.0 * np.arange(d // 2) / d)
    rq, rk = (R.rotate(_f64(t), at, freq, axis) for t in x[:2])
    src = _f64(x[0])
    pair = np.abs(src[..., :d // 2]) + np.abs(src[..., d // 2:])
    tol = np.concatenate([pair, pair], -1) * 6 * EPS + 2.0 ** -8 * np.abs(rq)
    assert (np.abs(_f64(q) - rq) <= tol).all(), f"{name} q"
    rv = _f64(x[2])
    for b, (m, n) in enumerate(spec):
        for i in range(m):
            j, r = n - m + i, starts[b] + i
            if j < 0:
                continue
            for kv, ref in ((0, rk[r]), (1, rv[r])):
                c, s = cache.read(kv, 1, b, [j])
                rc, rs = V.encode(ref, code)
                odd = np.isnan(rs)
                assert (np.isnan(s[0]) == odd).all() and (c[0][odd] == 0).all(), (name, kv, r)
                if kv == 1:
                    assert (c[0] == rc).all() and (s[0] == rs)[~odd].all(), (name, r)
                    continue
                # rotated in 64 bits and taken to fp32 once: off by 2^-24 before
                # its code's rounding, half a step of at most 2^-4 or of the row's
                # largest number over 127
                y = V.decode(c, s, code)[0]
                near = 2.0 ** -4 * np.abs(ref) + 2.0 ** -10 * s[0][:, None] if code == "e4m3" else \
                    0.5 * s[0][:, None]
                with np.errstate(invalid="ignore"):
                    good = np.abs(y - ref) <= near + 2 * EPS * np.abs(ref)
                assert good[~odd].all(), (name, kv, r)
                top = np.abs(ref).max(-1) * (1 + 2 * EPS)
                assert (top[~odd] <= (V.MOST[code] * s[0] * (1 + 4 * EPS))[~odd]).all()
                assert (top[~odd] * (1 + 4 * EPS) >= (V.MOST[code] * s[0] / 2)[~odd]).all()
            blk, slot = (int(t[0]) for t in cache.place(b, [j]))
            for t in (cache.dev[0], cache.dev[1], cache.dscale):
                t[1, blk, :, slot] = 0
            for t, o in zip((cache.dev[0], cache.dev[1], cache.dscale), before):
                o = o[..., :d].transpose(2, 3) if cache.strided and o.dtype == T.uint8 else \
                    o[..., 1, :].transpose(2, 3) if cache.strided else o
                o[1, blk, :, slot] = 0
    for t, o in zip(cache.base, before):
        bits = T.int16 if t.dtype == T.bfloat16 else T.uint8
        assert T.equal(t.view(bits), o.view(bits)), "wrote elsewhere"
    att.close()


def test_append_coded_parts():
    """Only queries, only keys and values: the same bits as the whole call's, and for
    values those of the plain call packed."""
    T = U.torch()
    spec = [(12, 40), (3, 20)]
    starts, lens = _starts([m for m, _ in spec]), [n for _, n in spec]
    x = [_rows(15, h, 64, "bf16", 30 + h) for h in (4, 2, 2)]
    att = _attention("bf16", 2, 64, 4)

    def run(q, **new):
        cache = Cache8(lens, 2, 64, "i8", 16)
        att.append(kvx.make_attn_io(cache.struct, _int(lens), q, q_start=_int(starts), max_new=12, **new))
        T.cuda.synchronize()
        return cache.dev + [cache.dscale.view(T.int16)]

    q = T.zeros_like(x[0])
    whole = run(q, new_q=x[0], new_k=x[1], new_v=x[2])
    q2 = x[0].clone()
    none = run(q2, new_q=q2)
    assert T.equal(q, q2) and not T.equal(whole[0], none[0])
    for a, b in zip(whole, run(None, new_k=x[1], new_v=x[2])):
        assert T.equal(a, b)
    plain = Cache(lens, 2, 64, "bf16", 16)
    att.append(kvx.make_attn_io(plain.struct, _int(lens), q, q_start=_int(starts), max_new=12,
                                new_k=x[1], new_v=x[2]))
    packed = Cache8(lens, 2, 64, "i8", 16)
    att.pack(kvx.make_pack_io(plain.struct, packed.struct, _int(lens)))
    coded = Cache8(lens, 2, 64, "i8", 16)
    att.append(kvx.make_attn_io(coded.struct, _int(lens), q, q_start=_int(starts), max_new=12,
                                new_k=x[1], new_v=x[2]))
    T.cuda.synchronize()
    for b, (m, n) in enumerate(spec):
        j = np.arange(n - m, n)
        for a, o in zip(packed.read(1, 0, b, j), coded.read(1, 0, b, j)):
            assert (a == o).all()
    att.close()


def test_attention_over_codes_is_attention_over_what_they_stand_for():
    """A bf16 cache, coded and read back exactly: within a rounding of the weights."""
    T = U.torch()
    for m in (1, 60):
        coded = Cache8([333], 2, 128, "e4m3", 16)
        plain = Cache([333], 2, 128, "bf16", 16)
        att = _attention("bf16", 2, 128, 8)
        att.unpack(kvx.make_pack_io(plain.struct, coded.struct, _int([333])))
        q = _rows(m, 8, 128, "bf16", 4)
        outs = []
        for c in (coded, plain):
            out, lse = T.zeros_like(q), T.zeros(m, 8, device="cuda")
            att.forward(kvx.make_attn_io(c.struct, _int([333]), q, out=out, lse=lse, layer=1, max_new=m,
                                         q_start=_int([0, m])), att.workspace())
            T.cuda.synchronize()
            outs.append((_f64(out), _f64(lse)))
        see = V.sight(m, 333)
        for o, l in outs:
            check_rows(f"{m}", "bf16", 128, 0.0, _f64(q), o, l, coded.f64(0, 1, 0), coded.f64(1, 1, 0), see)
        att.close()


# ---------------------------------------------------------------------------
# Trees
# ---------------------------------------------------------------------------

TREES = [
    # name, (nodes, cached) of each context, roots, back, words, window, sink, axes, shift
    ("one", [(1, 5)], 1, 1, 1, 0, 0, 1, False),
    ("chain", [(40, 100)], 1, 1, 2, 0, 0, 1, False),
    ("bushy", [(64, 64), (7, 100), (0, 3), (33, 40)], 1, 60, 2, 0, 0, 3, True),
    ("forest", [(31, 200), (32, 32)], 5, 9, 1, 0, 0, 1, True),
    ("window", [(50, 90), (12, 12)], 1, 3, 4, 6, 0, 2, False),
    ("window_sink", [(50, 52), (12, 300)], 1, 2, 2, 3, 4, 1, False),
    ("large", [(1000, 1500), (300, 300)], 2, 40, 32, 0, 0, 1, False),
    ("before_first_slot", [(20, 12), (5, 0)], 3, 5, 1, 4, 2, 1, False),
    ("many", [(1 + i % 9, 20 + i) for i in range(300)], 1, 4, 1, 0, 0, 1, False),
]


@pytest.mark.parametrize("case", TREES, ids=[c[0] for c in TREES])
def test_tree(case):
    name, spec, roots, back, words, window, sink, axes, shifted = case
    T = U.torch()
    print(f"[tree] {name}", flush=True)
    rng = np.random.default_rng(2)
    up = [random_tree(m, rng, roots, back) for m, _ in spec]
    starts = _starts([m for m, _ in spec])
    rows = int(starts[-1])
    shift = rng.integers(-5, 50, len(spec)) if shifted else np.zeros(len(spec), int)
    att = _attention("bf16", 1, 64, 1, pair_axis=[e % axes for e in range(32)])
    mask = T.full((rows + 1, words), -7, dtype=T.int32, device="cuda")
    depth = T.full((rows + 1,), -7, dtype=T.int32, device="cuda")
    pos = T.full((axes, rows), -7, dtype=T.int32, device="cuda")
    io = kvx.make_tree_io(_int([n for _, n in spec]), _int([p for t in up for p in t]), mask, depth=depth,
                          pos=pos, q_start=_int(starts), window=window, sink=sink,
                          shift=_int(shift) if shifted else None)
    att.tree(io)
    T.cuda.synchronize()
    assert (mask[rows:] == -7).all() and (depth[rows:] == -7).all()
    for b, (m, n) in enumerate(spec):
        sl = slice(starts[b], starts[b + 1])
        see = np.zeros((m, m), bool)
        for i, path in enumerate(V.paths(up[b])):
            for before, k in enumerate(path):
                see[i, k] = window == 0 or before < window or n - m + len(path) - 1 - before < sink
        d = np.array([len(p) - 1 for p in V.paths(up[b])], int)
        assert (mask[sl].cpu().numpy() == masks(up[b], see, words)).all(), (name, b)
        assert (depth[sl].cpu().numpy() == d).all(), (name, b)
        assert (pos[:, sl].cpu().numpy() == n - m + d + shift[b]).all(), (name, b)
    att.close()


def test_tree_of_wrong_parents_ends():
    """Parents that are not before their node count as none; nodes past the words see
    nothing drafted."""
    T = U.torch()
    up = [-1, 5, 2, 1000, -3, 4, 2 ** 31 - 1] + list(range(6, 60))
    mask = T.full((len(up), 1), -7, dtype=T.int32, device="cuda")
    depth = T.full((len(up),), -7, dtype=T.int32, device="cuda")
    att = _attention("bf16", 1, 64, 1)
    att.tree(kvx.make_tree_io(_int([100]), _int(up), mask, depth=depth, q_start=_int([0, len(up)])))
    T.cuda.synchronize()
    see = np.zeros((len(up), len(up)), bool)
    for i, path in enumerate(V.paths(up)):
        if i < 32:
            see[i, path] = True
    assert (mask.cpu().numpy() == masks(up, see[:, :32], 1)[:, :1]).all()
    assert (depth[32:] == 0).all()
    att.close()


ACCEPT = [
    # name, dtype, code, layers, hkv, d, page, (new, cached), paths, options
    ("one", "bf16", "", 2, 2, 128, 16, [(8, 40)], [[0, 2, 5]], {}),
    ("none", "bf16", "", 2, 2, 64, 16, [(8, 40)], [[]], {}),
    ("all", "bf16", "", 2, 2, 64, 16, [(8, 40)], [list(range(8))], {}),
    ("chained", "bf16", "", 3, 1, 128, 7, [(40, 60)], [[1, 2, 3, 4, 5, 6, 7, 8, 9, 20, 21, 39]], {}),
    ("long", "f32", "", 2, 2, 256, 16, [(64, 64)], [list(range(4, 64, 2))], {}),
    ("ragged", "bf16", "", 2, 4, 80, 16, [(5, 30), (0, 9), (1, 1), (33, 50)], [[0, 4], [], [0], [3, 30, 32]], {}),
    ("i8", "bf16", "i8", 2, 2, 128, 16, [(16, 40), (9, 100)], [[0, 3, 9, 15], [8]], {}),
    ("e4m3_f32", "f32", "e4m3", 2, 2, 256, 0, [(16, 40), (9, 100)], [[2, 3, 4], [0, 1, 7]], {}),
    ("strided", "bf16", "i8", 2, 2, 64, 16, [(16, 40)], [[1, 3, 9, 15]], dict(strided=True)),
    ("strided_plain", "bf16", "", 2, 2, 64, 16, [(16, 40)], [[1, 3, 9, 15]], dict(strided=True)),
    ("many", "bf16", "e4m3", 2, 2, 64, 16, [(12, 20 + i) for i in range(100)],
     [[i % 3, 3 + i % 4, 11] for i in range(100)], {}),
]


@pytest.mark.parametrize("case", ACCEPT, ids=[c[0] for c in ACCEPT])
def test_accept(case):
    name, dtype, code, layers, hkv, d, page, spec, path, opt = case
    T = U.torch()
    print(f"[accept] {name}", flush=True)
    lens = [n for _, n in spec]
    if code:
        cache = Cache8(lens, hkv, d, code, page, layers=layers, strided=opt.get("strided", False))
        held = cache.dev + [cache.dscale.view(T.int16)]
    else:
        cache = Cache(lens, hkv, d, dtype, page, layers=layers, flash=opt.get("strided", False))
        bits = T.int16 if dtype == "bf16" else T.int32
        held = [(t.transpose(2, 3) if cache.flash else t).view(bits) for t in cache.dev]
    want = [t.clone() for t in held]
    for b, (m, n) in enumerate(spec):
        for i, k in enumerate(path[b]):
            of, to = (tuple(int(x[0]) for x in cache.place(b, [n - m + y])) for y in (k, i))
            for w, t in zip(want, held):
                w[:, to[0], :, to[1]] = t[:, of[0], :, of[1]]
    longest = max(1, max(len(p) for p in path)) + 2
    table = _int([x for p in path for x in p + [99] * (longest - len(p))]).view(len(spec), longest)
    tokens, left = _int(lens), _int([-7] * len(spec))
    att = _attention(dtype, hkv, d, hkv, layers=layers)
    att.accept(kvx.make_accept_io(cache.struct, tokens, table, _int([len(p) for p in path]),
                                  q_start=_int(_starts([m for m, _ in spec])), tokens_out=left))
    T.cuda.synchronize()
    assert left.tolist() == [n - m + len(p) for (m, n), p in zip(spec, path)]
    assert tokens.tolist() == lens
    for w, t in zip(want, held):
        assert T.equal(w, t), name
    att.close()


def test_accept_of_paths_that_lead_nowhere():
    """Entries outside of the nodes, counts past them and slots past the capacity move
    nothing."""
    T = U.torch()
    cache = Cache([40, 30], 1, 64, "bf16", 0)
    held = [t.view(T.int16) for t in cache.dev]
    want = [t.clone() for t in held]
    for w, t in zip(want, held):
        w[:, 0, :, 32] = t[:, 0, :, 33]  # the one that is there
    left = _int([0, 0])
    att = _attention("bf16", 1, 64, 1)
    path = _int([-1, 8, 1 << 30, 5, 0, 1, 2, 3]).view(2, 4)
    path[0, 0] = 1  # slot 33 to 32; 8 and 2^30 lead out; 5 (slot 37) to 35
    for w, t in zip(want, held):
        w[:, 0, :, 35] = t[:, 0, :, 37]
    att.accept(kvx.make_accept_io(cache.struct, _int([40, 50]), path, _int([9, 9]),
                                  q_start=_int([0, 8, 12]), tokens_out=left))
    T.cuda.synchronize()
    assert left.tolist() == [36, 50]
    for w, t in zip(want, held):
        assert T.equal(w, t)
    att.close()


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("code", ["", "i8", "e4m3"])
def test_drafted_steps_equal_tokens_one_by_one(code):
    """A tree's accepted path, read in one call and moved behind the context, against
    the same tokens stored and read one by one."""
    T = U.torch()
    hq, hkv, d, n = 8, 2, 128, 90
    rng = np.random.default_rng(5)
    make = (lambda: Cache8([n], hkv, d, code, 16, extra=40)) if code else \
        (lambda: Cache([n], hkv, d, "bf16", 16, extra=40))
    drafted, single = make(), make()
    att = _attention("bf16", hkv, d, hq)
    ws = att.workspace()
    m = 20
    up = random_tree(m, rng, 1, 4)
    path = V.paths(up)[m - 1][::-1]
    x = [_rows(m, h, d, "bf16", 60 + i) for i, h in enumerate((hq, hkv, hkv))]
    mask = T.zeros((m, 1), dtype=T.int32, device="cuda")
    depth, pos = T.zeros(m, dtype=T.int32, device="cuda"), T.zeros((1, m), dtype=T.int32, device="cuda")
    start, tokens = _int([0, m]), _int([n + m])
    att.tree(kvx.make_tree_io(tokens, _int(up), mask, depth=depth, pos=pos, q_start=start))
    q, out = T.zeros_like(x[0]), T.zeros_like(x[0])
    io = kvx.make_attn_io(drafted.struct, tokens, q, layer=1, q_start=start, max_new=m, new_q=x[0],
                          new_k=x[1], new_v=x[2], pos=pos, out=out, tree=mask, depth=depth)
    att.append(io)
    att.forward(io, ws)
    left = T.zeros_like(tokens)
    table = _int(path).view(1, -1)
    att.accept(kvx.make_accept_io(drafted.struct, tokens, table, _int([len(path)]), q_start=start,
                                  tokens_out=left))
    T.cuda.synchronize()
    assert left.tolist() == [n + len(path)]
    for i, k in enumerate(path):
        one = [t[k:k + 1] for t in x]
        q1, o1 = T.zeros_like(one[0]), T.zeros_like(one[0])
        io1 = kvx.make_attn_io(single.struct, _int([n + i + 1]), q1, layer=1, new_q=one[0], new_k=one[1],
                               new_v=one[2], out=o1)
        att.append(io1)
        att.forward(io1, ws)
        T.cuda.synchronize()
        assert T.equal(q1[0], q[k]), i
        # two orders of the same sums, each within the tolerance of the other
        o, r = _f64(o1[0]), _f64(out[k])
        assert (np.abs(o - r) <= 2 * (2.0 ** -8 * np.abs(r) + 2.0 ** -7)).all(), i
    j = np.arange(n + len(path))
    for kv in range(2):
        if code:
            for a, b in zip(drafted.read(kv, 1, 0, j), single.read(kv, 1, 0, j)):
                assert (a == b).all()
        else:
            assert T.equal(drafted.read(kv, 1, 0, len(j)), single.read(kv, 1, 0, len(j)))
    att.close()


@pytest.mark.parametrize("code", ["", "i8", "e4m3"])
def test_captured_steps(code):
    """A captured step of drafting (tree, append, forward, accept) replayed at other
    lengths, trees and inputs gives the eager calls' bits, on another stream."""
    T = U.torch()
    hq, hkv, d, lens, new = 12, 2, 128, [100, 333, 64], [16, 3, 9]
    rng = np.random.default_rng(6)
    starts = _starts(new)
    rows = int(starts[-1])
    att = _attention("bf16", hkv, d, hq)

    def side():
        cache = Cache8(lens, hkv, d, code, 16, extra=80) if code else \
            Cache(lens, hkv, d, "bf16", 16, extra=80)
        x = [T.zeros(rows, h, d, dtype=T.bfloat16, device="cuda") for h in (hq, hkv, hkv)]
        t = dict(x=x, tokens=_int(lens), left=_int([0] * 3), parent=_int([-1] * rows),
                 mask=T.zeros((rows, 1), dtype=T.int32, device="cuda"), depth=_int([0] * rows),
                 pos=_int([0] * rows).view(1, rows), q=T.zeros_like(x[0]), out=T.zeros_like(x[0]),
                 lse=T.zeros(rows, hq, device="cuda"), path=_int([0] * 12).view(3, 4), count=_int([0] * 3),
                 ws=att.workspace(), cache=cache)
        qs = _int(starts)
        tree = kvx.make_tree_io(t["tokens"], t["parent"], t["mask"], depth=t["depth"], pos=t["pos"],
                                q_start=qs, window=50, sink=4)
        io = kvx.make_attn_io(cache.struct, t["tokens"], t["q"], layer=1, q_start=qs, max_new=16,
                              new_q=x[0], new_k=x[1], new_v=x[2], pos=t["pos"], out=t["out"], lse=t["lse"],
                              window=50, sink=4, tree=t["mask"], depth=t["depth"])
        acc = kvx.make_accept_io(cache.struct, t["tokens"], t["path"], t["count"], q_start=qs,
                                 tokens_out=t["left"])

        def step():
            att.tree(tree)
            att.append(io)
            att.forward(io, t["ws"])
            att.accept(acc)
            t["tokens"].copy_(t["left"])

        return t, step

    a, step_a = side()
    b, step_b = side()
    stream = T.cuda.Stream()
    stream.wait_stream(T.cuda.current_stream())
    graph = T.cuda.CUDAGraph()
    with T.cuda.graph(graph, stream=stream):
        step_a()
    for turn in range(4):
        up = [p for m in new for p in random_tree(m, rng, 1, 3)]
        paths = [sorted(rng.choice(m, min(m, 3), replace=False).tolist()) for m in new]
        x = [T.randn_like(t) for t in a["x"]]
        for t in (a, b):
            for u, v in zip(t["x"], x):
                u.copy_(v)
            t["parent"].copy_(_int(up))
            t["tokens"] += _int(new)
            t["path"].copy_(_int([k for p in paths for k in p + [-1] * (4 - len(p))]).view(3, 4))
            t["count"].copy_(_int([len(p) for p in paths]))
        T.cuda.synchronize()
        graph.replay()
        T.cuda.synchronize()
        step_b()
        T.cuda.synchronize()
        for k in ("mask", "depth", "pos", "q", "out", "lse", "tokens"):
            assert T.equal(a[k], b[k]), (turn, k)
        assert a["tokens"].tolist() == [n + 3 * (turn + 1) for n in lens]
        for u, v in zip(a["cache"].dev, b["cache"].dev):
            assert T.equal(u.view(T.uint8), v.view(T.uint8)), turn
    T.cuda.synchronize()
    del graph
    att.close()


def test_validation_and_faults(monkeypatch):
    T = U.torch()
    spec = [(8, 40), (3, 20)]
    att = _attention("bf16", 2, 64, 4)
    ws = att.workspace()
    cache, q, starts, tokens, kw, _ = _problem("bf16", "i8", 4, 2, 64, 16, spec, dict(tree=1))
    plain = Cache([n for _, n in spec], 2, 64, "bf16", 16)
    x = [_rows(11, h, 64, "bf16", 9 + h) for h in (4, 2, 2)]
    io = kvx.make_attn_io(cache.struct, tokens, q, out=T.zeros_like(q), new_q=x[0], new_k=x[1],
                          new_v=x[2], **kw)
    parent = _int([p for m, _ in spec for p in range(-1, m - 1)])
    tree = kvx.make_tree_io(tokens, parent, kw["tree"].clone(), q_start=kw["q_start"])
    path, count = _int([0, 2, 1, 2]).view(2, 2), _int([2, 1])
    acc = kvx.make_accept_io(cache.struct, tokens, path, count, q_start=kw["q_start"],
                             tokens_out=T.zeros_like(tokens))
    pack = kvx.make_pack_io(plain.struct, cache.struct, tokens)
    calls = dict(append=lambda: att.append(io), forward=lambda: att.forward(io, ws),
                 tree=lambda: att.tree(tree), accept=lambda: att.accept(acc), pack=lambda: att.pack(pack),
                 unpack=lambda: att.unpack(pack))
    monkeypatch.setenv("KVX_VALIDATE", "1")
    for call in calls.values():
        call()

    def refused(names, status=kvx.KVX_EDATA):
        for name in names.split():
            with pytest.raises(kvx.KvxError) as e:
                calls[name]()
            assert e.value.status == status, name

    for bad in (-1, 10 ** 6):
        tokens[0] = bad
        refused("append forward accept pack unpack")
    tokens[0] = 7  # fewer than its nodes
    refused("tree accept")
    tokens[0] = 40
    keep = cache.table.clone()
    cache.table[0, 2] = 10 ** 6  # the block of slots 32..39
    refused("append forward accept pack unpack")
    cache.table.copy_(keep)
    plain.table[0, 0] = -1
    refused("pack unpack")
    parent[3] = 3
    refused("tree")
    path[0, 1] = 8
    refused("accept")
    path[0] = _int([2, 2])
    refused("accept")
    path[0] = _int([0, 2])
    count[1] = 3
    refused("accept")
    monkeypatch.delenv("KVX_VALIDATE")
    monkeypatch.setenv("KVX_FAULT", "launch")
    refused(" ".join(calls), kvx.KVX_EHIP)
    T.cuda.synchronize()
    att.close()


def test_sinks_validate_the_blocks_that_they_reach(monkeypatch):
    T = U.torch()
    cache = Cache([200], 2, 64, "bf16", 16)
    q = _rows(1, 4, 64, "bf16", 1)
    att = _attention("bf16", 2, 64, 4)
    ws = att.workspace()
    monkeypatch.setenv("KVX_VALIDATE", "1")
    cache.table[0, 1:5] = 10 ** 6  # between the sinks and the window: not read through
    outs = []
    for sink in (4, 16):
        out = T.zeros_like(q)
        att.forward(kvx.make_attn_io(cache.struct, _int([200]), q, out=out, layer=1, window=100, sink=sink),
                    ws)
        T.cuda.synchronize()
        check_rows("", "bf16", 64, 0.0, _f64(q), _f64(out), V.attend(
            _f64(q), cache.f64(0, 1, 0), cache.f64(1, 1, 0), V.sight(1, 200, 100, sink), 0.125)[1],
            cache.f64(0, 1, 0), cache.f64(1, 1, 0), V.sight(1, 200, 100, sink))
        outs.append(out)
    with pytest.raises(kvx.KvxError):
        att.forward(kvx.make_attn_io(cache.struct, _int([200]), q, out=out, layer=1, window=100, sink=17), ws)
    att.close()


def test_outgrown_caches():
    """A context of more tokens than its cache has slots: those past it are neither
    stored nor seen."""
    T = U.torch()
    for code, m, grown, sink in (("i8", 1, 7, 4), ("", 1, 60, 4), ("", 40, 60, 4), ("e4m3", 40, 20, 4),
                                 ("i8", 1, 300, 3)):
        print(f"[outgrown] {code} {m} by {grown}", flush=True)
        n, window = 96, 50
        cache = Cache8([n], 2, 64, code, 16) if code else Cache([n], 2, 64, "bf16", 16)
        q = _rows(m, 4, 64, "bf16", 3)
        att = _attention("bf16", 2, 64, 4)
        out, lse = T.zeros_like(q), T.zeros(m, 4, device="cuda")
        io = kvx.make_attn_io(cache.struct, _int([n + grown]), q, out=out, lse=lse, layer=1, max_new=m,
                              q_start=_int([0, m]), window=window, sink=sink)
        att.forward(io, att.workspace())
        T.cuda.synchronize()
        see = V.sight(m, n + grown, window, sink)[:, :n]
        check_rows(code, "bf16", 64, 0.0, _f64(q), _f64(out), _f64(lse), cache.f64(0, 1, 0),
                   cache.f64(1, 1, 0), see)
        if code:
            held = [t.clone() for t in cache.base[:2]]
            x = [_rows(m, 2, 64, "bf16", 5 + i) for i in range(2)]
            att.append(kvx.make_attn_io(cache.struct, _int([n + grown + m]), None, layer=1, max_new=m,
                                        q_start=_int([0, m]), new_k=x[0], new_v=x[1]))
            T.cuda.synchronize()
            if grown >= 0:
                for t, o in zip(cache.base[:2], held):
                    assert T.equal(t, o)
        att.close()


def test_offsets_past_32_bits():
    """A layer of codes past 2^32 bytes."""
    T = U.torch()
    hkv, d, bs, nb = 2, 128, 16, 1_100_000  # 4.5e9 codes a layer
    k = T.zeros((1, nb, hkv, bs, d), dtype=T.int8, device="cuda")
    v = T.zeros_like(k)
    scale = T.zeros((1, nb, hkv, bs, 2), dtype=T.bfloat16, device="cuda")
    table = _int([3, nb - 1, nb // 2 + 5, nb - 9]).view(1, 4)
    n = 60
    att = kvx.Attention(kvx.ModelShape(1, hkv, d, 1e4), 4, kvx.KVX_BF16)
    cache = kvx.make_cache8(k, v, scale, table)
    x = [_rows(n, hkv, d, "bf16", 8 + i) for i in range(2)]
    att.append(kvx.make_attn_io(cache, _int([n]), None, new_k=x[0], new_v=x[1], q_start=_int([0, n]),
                                max_new=n, pos=_int([0] * n).view(1, n)))
    rows = [V.decode(*V.encode(_f64(t), "i8"), "i8") for t in x]
    for m in (1, 20):
        q = _rows(m, 4, d, "bf16", 3)
        out, lse = T.zeros_like(q), T.zeros(m, 4, device="cuda")
        att.forward(kvx.make_attn_io(cache, _int([n]), q, out=out, lse=lse, max_new=m, q_start=_int([0, m])),
                    att.workspace())
        T.cuda.synchronize()
        check_rows("", "bf16", d, 0.0, _f64(q), _f64(out), _f64(lse), rows[0], rows[1], V.sight(m, n))
    att.close()


def test_rows_of_no_context_stay():
    """Rows behind the last context's, and outputs of other contexts, are left as they were."""
    T = U.torch()
    for m in (1, 40):
        cache = Cache8([50, 70], 2, 64, "i8", 16)
        att = _attention("bf16", 2, 64, 4)
        rows = 2 * m + 5
        q = _rows(rows, 4, 64, "bf16", 1)
        out, lse = T.full_like(q, 7.0), T.full((rows, 4), 7.0, device="cuda")
        att.forward(kvx.make_attn_io(cache.struct, _int([50, 70]), q, out=out, lse=lse, layer=1, max_new=m,
                                     q_start=_int([0, m, 2 * m])), att.workspace())
        T.cuda.synchronize()
        assert (out[2 * m:] == 7.0).all() and (lse[2 * m:] == 7.0).all()
        assert not (out[:2 * m] == 7.0).all(-1).any()
        att.close()


def test_more_new_tokens_than_said():
    """max_new chooses the kernel: too small a one changes no more than roundings."""
    T = U.torch()
    for m, said in ((40, 1), (9, 1), (40, 5)):
        cache, q, starts, tokens, kw, sights = _problem("bf16", "i8", 8, 2, 128, 16, [(m, 300), (3, 90)],
                                                        dict(window=100, sink=4))
        kw["max_new"] = said
        att = _attention("bf16", 2, 128, 8)
        out, lse = T.zeros_like(q), T.zeros(starts[-1], 8, device="cuda")
        att.forward(kvx.make_attn_io(cache.struct, tokens, q, out=out, lse=lse, **kw), att.workspace())
        T.cuda.synchronize()
        for b in range(2):
            sl = slice(starts[b], starts[b + 1])
            check_rows(f"{m} {said}", "bf16", 128, 0.0, _f64(q)[sl], _f64(out)[sl], _f64(lse)[sl],
                       cache.f64(0, 1, b), cache.f64(1, 1, b), sights[b])
        att.close()


def test_masks_and_depths_may_be_anything():
    """Bits of nodes that are not there, and depths outside of the tree, are no reads out
    of range: bits past the last node see nothing, depths count as the nearest that may be."""
    T = U.torch()
    n, m = 90, 20
    cache, q, starts, tokens, kw, sights = _problem("bf16", "", 8, 2, 64, 16, [(m, n)], dict(tree=1))
    att = _attention("bf16", 2, 64, 8)
    ws, outs = att.workspace(), []
    for spoil in (0, -(1 << 20), 1 << 30):
        if spoil:
            kw["tree"] |= -(1 << m)  # bits 20..31
            kw["depth"][:] = spoil
        out, lse = T.zeros_like(q), T.zeros(m, 8, device="cuda")
        att.forward(kvx.make_attn_io(cache.struct, tokens, q, out=out, lse=lse, **kw), ws)
        T.cuda.synchronize()
        outs.append((out, lse))
    for o, l in outs[1:]:  # without a window, depths change nothing
        assert T.equal(o, outs[0][0]) and T.equal(l, outs[0][1])
    att.close()


def test_garbage_behind_the_tokens():
    """Slots past a context's tokens in the blocks that its last ones share: NaN, as a
    fresh allocation may hold, at every length around a block's end."""
    T = U.torch()
    for code, d in (("", 128), ("", 256), ("i8", 128), ("e4m3", 128)):
        for page in (16, 48, 0):
            lens = [1, 15, 16, 17, 31, 32, 33, 47, 48, 49, 100]
            cache = Cache8(lens, 2, d, code, page, extra=20) if code else \
                Cache(lens, 2, d, "bf16", page, extra=20)
            q = _rows(len(lens), 8, d, "bf16", 1)
            att = _attention("bf16", 2, d, 8)
            out, lse = T.zeros_like(q), T.zeros(len(lens), 8, device="cuda")
            att.forward(kvx.make_attn_io(cache.struct, _int(lens), q, out=out, lse=lse, layer=1, window=20,
                                         sink=3), att.workspace())
            T.cuda.synchronize()
            for b, n in enumerate(lens):
                sl = slice(b, b + 1)
                check_rows(f"{code} {page} {n}", "bf16", d, 0.0, _f64(q)[sl], _f64(out)[sl], _f64(lse)[sl],
                           cache.f64(0, 1, b), cache.f64(1, 1, b), V.sight(1, n, 20, 3))
            att.close()


def test_two_streams_at_once():
    """Two handles' calls on two streams, each with its workspace, give the bits that they
    give one after the other."""
    T = U.torch()
    sides = []
    for i in range(2):
        cache, q, starts, tokens, kw, _ = _problem("bf16", "i8", 28, 4, 128, 16,
                                                   [(1, 700 + 50 * i), (1, 90), (1, 3000)], dict(window=600, sink=4),
                                                   seed=i)
        att = _attention("bf16", 4, 128, 28)
        out = T.zeros_like(q)
        io = kvx.make_attn_io(cache.struct, tokens, q, out=out, **kw)
        sides.append((cache, att, att.workspace(), out, io, T.cuda.Stream()))
    T.cuda.synchronize()
    alone = []
    for _, att, ws, out, io, _ in sides:
        att.forward(io, ws)
        T.cuda.synchronize()
        alone.append(out.clone())
    for _ in range(20):
        for _, att, ws, out, io, stream in sides:
            att.forward(io, ws, stream)
    T.cuda.synchronize()
    for a, side in zip(alone, sides):
        assert T.equal(a, side[3])
        side[1].close()
