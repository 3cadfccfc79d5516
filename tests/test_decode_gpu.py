"""The decoding example on the GPU: translated cache, question, answer, budget."""
import gc

import numpy as np
import pytest

from oracle import attn as R
from tests import gpu_util as U

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _memory_as_before():
    """The stand-in layers' products leave torch's matrix library a workspace,
    cut out of whatever block was cached; other tests rely on blocks that are
    wholly free going back to the driver."""
    yield
    T = U.torch()
    T.cuda.synchronize()
    gc.collect()
    T._C._cuda_clearCublasWorkspaces()
    T.cuda.empty_cache()


def _decoder(config, batch, budget, slack):
    from examples import decode as E
    T = U.torch()
    shape, k, v, table, lengths = E.handoff(config, 120, batch, 64)
    heads, cap = E.HEADS[config]
    dec = E.Decoder(shape, heads, cap, k, v, table, lengths, budget, slack)
    g = T.Generator("cuda").manual_seed(1)
    dec.read(T.randn(batch, 9, dec.model.width, device="cuda", generator=g).to(T.bfloat16))
    return dec, lengths


def _rows(dec, which, layer, b, n):
    j = np.arange(n)
    blk = dec.table.cpu().numpy()[b][j // 16].astype(np.int64)
    return (dec.k, dec.v)[which].cpu()[layer][blk, :, j % 16].double().numpy()


@pytest.mark.parametrize("config,batch", [(2, 1), (3, 2)])
def test_replayed_steps_are_the_eager_ones(config, batch):
    """Captured steps, with an eviction between them, give the eager steps' bits."""
    T = U.torch()
    print(f"[decode] config {config}, {batch} contexts", flush=True)
    a, lengths = _decoder(config, batch, 40, 20)
    b, _ = _decoder(config, batch, 40, 20)
    evictions = 0
    for i in range(30):
        before = a.longest
        x = a.step().clone()
        T.cuda.synchronize()
        y = b.step(eager=True)
        T.cuda.synchronize()
        evictions += a.longest <= before
        for s, t in ((x, y), (a.tokens, b.tokens), (a.pos, b.pos), (a.mass, b.mass), (a.k, b.k),
                     (a.v, b.v)):
            assert T.equal(s, t), (config, i)
        assert T.isfinite(x).all()
    # 40 + 9 tokens after the question; the 12th step would be the 61st, the next eviction
    # comes 20 steps later
    assert evictions == 1
    assert a.pos.tolist() == [n + 9 + 30 for n in lengths]
    assert max(a.tokens.tolist()) == a.longest
    a.close()
    b.close()


def test_a_step_attends_to_what_is_cached():
    """The last step's attention after an eviction, of the last layer, is the
    64-bit one of the rows that its cache holds: scores err by (D + 8) 2^-24 of
    their terms, bf16 weights and outputs round by 2^-8."""
    T = U.torch()
    print("[decode] against 64 bits", flush=True)
    dec, lengths = _decoder(3, 2, 40, 20)
    for _ in range(5):
        dec.step(eager=True)
    T.cuda.synchronize()
    last = dec.model.shape.n_layers - 1
    d = dec.model.shape.head_dim
    q = dec.one["qkv"][:, :dec.model.n_heads].double().cpu().numpy()
    out = dec.one["out"][:, last].double().cpu().numpy()
    for b, n in enumerate(dec.tokens.tolist()):
        assert n < lengths[b]
        ro, _, mag, size = R.attend(q[b:b + 1], _rows(dec, 0, last, b, n),
                                    _rows(dec, 1, last, b, n), d ** -0.5, 50.0)
        rel = 2 * ((d + 8) * 2.0 ** -24 * size + 2.0 ** -22 * 50.0) + (n + 64) * 2.0 ** -24
        tol = mag * (rel + 2.0 ** -8)[..., None] + 2.0 ** -8 * np.abs(ro)
        assert (np.abs(out[b:b + 1] - ro) <= tol).all(), b
    dec.close()


def test_eviction_keeps_the_rows_of_most_weight():
    """An eviction leaves, in their order, the rows of the first, the last and
    the heaviest tokens of each head of each layer."""
    T = U.torch()
    print("[decode] eviction", flush=True)
    dec, _ = _decoder(2, 1, 48, 200)
    dec.step(eager=True)
    T.cuda.synchronize()
    n = dec.tokens.tolist()[0]
    weight = dec.mass.double().cpu().numpy()
    layers = (0, dec.model.shape.n_layers - 1)
    before = {(w, l): _rows(dec, w, l, 0, n) for w in (0, 1) for l in layers}
    dec.evict()
    T.cuda.synchronize()
    assert dec.tokens.tolist() == [48]
    kept = dec.kept.cpu().numpy()
    for l in layers:
        for h in range(dec.model.shape.n_kv_heads):
            want = R.keep(weight[l, 0, h, :n], 48, 4, 6)
            assert (kept[l, 0, h] == want).all()
            for w in (0, 1):
                assert (_rows(dec, w, l, 0, 48)[:, h] == before[w, l][want, h]).all()
    dec.close()
