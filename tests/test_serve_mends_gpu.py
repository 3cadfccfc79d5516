"""Calls of serving (kvx_serve.h) that were once answered wrongly, refused or slow."""
import numpy as np
import pytest

from paper_2608_30963_amd import kvx
from tests import gpu_util as U
from tests.serve_util import Cache8
from tests.test_attn_gpu import _int, _rows
from tests.test_serve_gpu import _problem

pytestmark = pytest.mark.gpu


def _least_ms(call, turns=5):
    """The least time of a call, by the device's own clock."""
    T = U.torch()
    times = []
    for _ in range(turns):
        a, b = T.cuda.Event(enable_timing=True), T.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        T.cuda.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


@pytest.mark.parametrize("d,page", [(128, 16), (128, 0), (256, 16), (64, 48)])
@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_what_lies_behind_the_tokens_costs_nothing(code, d, page):
    """Slots past a context's tokens that hold NaN scales and codes that are no numbers,
    or zeros: the same bits, and no row is computed a second time (which took two hundred
    times as long)."""
    T = U.torch()
    lens, m = [2003, 1029], 140
    att = kvx.Attention(kvx.ModelShape(2, 2, d, 1e4), 8, kvx.KVX_BF16)
    ws, outs, took = att.workspace(), [], []
    q = _rows(2 * m, 8, d, "bf16", 1)
    for garbage in (False, True):
        cache = Cache8(lens, 2, d, code, page, extra=20)  # code 127 and NaN behind
        if not garbage:
            for t in cache.base[:2]:
                t[t == 127] = 0
            cache.base[2].nan_to_num_(nan=1.0)
            for kv in range(2):  # the tokens' own codes
                for b, n in enumerate(lens):
                    blk, slot = cache.place(b, np.arange(n))
                    full = Cache8(lens, 2, d, code, page, extra=20) if kv == b == 0 else full
                    cache.dev[kv][:, blk, :, slot] = full.dev[kv][:, blk, :, slot]
        out, lse = T.zeros_like(q), T.zeros(2 * m, 8, device="cuda")
        io = kvx.make_attn_io(cache.struct, _int(lens), q, out=out, lse=lse, layer=1, max_new=m,
                              q_start=_int([0, m, 2 * m]))
        att.forward(io, ws)
        T.cuda.synchronize()
        outs.append((out, lse))
        took.append(_least_ms(lambda: att.forward(io, ws)))
    assert T.equal(outs[0][0], outs[1][0]) and T.equal(outs[0][1], outs[1][1])
    assert took[1] < 3 * took[0], took
    att.close()


@pytest.mark.parametrize("d", [64, 128, 192, 256])
@pytest.mark.parametrize("code", ["", "i8", "e4m3"])
def test_hidden_values_of_single_tokens(code, d):
    """Values that are no numbers, in tiles at an edge that single tokens' kernel clears:
    rows that do not see them keep their bits, rows that see one are NaN or infinite."""
    T = U.torch()
    m, n = 3, 200
    for window, sink, bad in ((30, 4, [6, 33, n - 32, n - 31, n - 1]), (0, 0, [n - 2]), (30, 4, [100])):
        cache, q, starts, tokens, kw, sights = _problem("bf16", code, 4, 2, d, 16, [(m, n), (1, 50)],
                                                        dict(window=window, sink=sink))
        att = kvx.Attention(kvx.ModelShape(2, 2, d, 1e4), 4, kvx.KVX_BF16)
        ws, outs = att.workspace(), []
        for spoiled in (False, True):
            for i, j in enumerate(bad if spoiled else []):
                blk, slot = (int(x[0]) for x in cache.place(0, [j]))
                if code == "i8":
                    cache.dscale[1, blk, :, slot, 1] = float("nan")
                elif code:
                    cache.dev[1][1, blk, :, slot] = 127 if i % 2 else 255
                else:
                    cache.dev[1][1, blk, :, slot] = float("nan") if i % 2 else -float("inf")
            out = T.zeros_like(q)
            att.forward(kvx.make_attn_io(cache.struct, tokens, q, out=out, **kw), ws)
            T.cuda.synchronize()
            outs.append(out.double().cpu().numpy())
        assert np.isfinite(outs[0]).all() and (outs[0][m:] == outs[1][m:]).all()
        for i in range(m):
            if sights[0][i, bad].any():
                assert not np.isfinite(outs[1][i]).any(), (window, i)
            else:
                assert (outs[0][i] == outs[1][i]).all(), (window, i)
        att.close()
