"""Eviction (kvx_attn_evict) at sizes where its launches and buffers end: many
kept tokens, and weights for fewer slots than are cached."""
import numpy as np
import pytest

from oracle import attn as R
from paper_2608_30963_amd import kvx
from tests import gpu_util as U
from tests import test_attn_gpu as A

pytestmark = pytest.mark.gpu


def test_keep_far_beyond_the_cache():
    """A budget of more tokens than one launch has workgroups for, on a small
    cache: everything is kept, whole."""
    T = U.torch()
    print("[evict] keep beyond the cache", flush=True)
    lens, d, keep = [100, 7], 256, 2_200_000
    cache, dst = (A.Cache(lens, 1, d, "f32", 16, layers=1, seed=s) for s in (0, 9))
    w = T.rand(1, 2, 1, 128, device="cuda")
    mass = w.clone()
    kept = T.full((1, 2, 1, keep), -7, dtype=T.int32, device="cuda")
    left = A._int([0, 0])
    att = kvx.Attention(kvx.ModelShape(1, 1, d, 1e4), 1, kvx.KVX_F32)
    att.evict(kvx.make_evict_io(cache.struct, A._int(lens), mass, kept, keep, sink=4, recent=8,
                                mass_out=mass, tokens_out=left, dst=dst.struct))
    T.cuda.synchronize()
    assert left.tolist() == lens
    for b, n in enumerate(lens):
        assert (kept[0, b, 0, :n].cpu().numpy() == np.arange(n)).all()
        assert (kept[0, b, 0, n:] == -1).all()
        assert T.equal(mass[0, b, 0, :n], w[0, b, 0, :n])
        for kv in range(2):
            assert T.equal(dst.read(kv, 0, b, n), cache.rows[kv][0][b])
    att.close()


def test_millions_of_rows_to_other_memory():
    """More rows than a launch has workgroups for at one step each.  The source
    names 5 blocks over and over, so that it takes little memory."""
    T = U.torch()
    print("[evict] 2.2 million rows", flush=True)
    d, page, keep, n = 256, 32, 2_200_000, 2_300_005
    g = T.Generator().manual_seed(0)
    src = [T.randn(1, 5, 1, page, d, generator=g).cuda() for _ in range(2)]
    table = (T.arange(-(-n // page), dtype=T.int32) * 3 % 5).view(1, -1).cuda()
    dst = [T.zeros(1, 1, 1, keep, d, device="cuda") for _ in range(2)]
    w = T.rand(1, 1, 1, n, device="cuda", generator=T.Generator("cuda").manual_seed(1))
    kept = T.full((1, 1, 1, keep), -7, dtype=T.int32, device="cuda")
    left = A._int([0])
    att = kvx.Attention(kvx.ModelShape(1, 1, d, 1e4), 1, kvx.KVX_F32)
    att.evict(kvx.make_evict_io(kvx.make_cache(src[0], src[1], table), A._int([n]), w, kept, keep,
                                sink=4, recent=100, tokens_out=left,
                                dst=kvx.make_cache(dst[0], dst[1])))
    T.cuda.synchronize()
    assert left.tolist() == [keep]
    weight = w[0, 0, 0].cpu().numpy().astype(np.float64)
    always = np.zeros(n, bool)
    always[:4] = always[-100:] = True
    rest = np.flatnonzero(~always)
    rest = rest[np.argsort(-weight[rest], kind="stable")[:keep - 104]]
    want = T.from_numpy(np.sort(np.concatenate([np.flatnonzero(always), rest]))).cuda()
    assert T.equal(kept[0, 0, 0].long(), want)
    for s, t in zip(src, dst):
        for i in range(0, keep, 200_000):
            j = want[i:i + 200_000]
            assert T.equal(t[0, 0, 0, i:i + 200_000], s[0, j // page * 3 % 5, 0, j % page])
    att.close()


@pytest.mark.parametrize("lens,room,keep,sink,recent", [
    ([200, 61], 150, 100, 4, 16), ([200, 149], 150, 180, 4, 60), ([9000, 30], 8200, 900, 4, 850),
    ([50], 1, 20, 2, 3)])
@pytest.mark.parametrize("in_place", [False, True], ids=["out", "in_place"])
def test_weights_of_fewer_slots_than_are_cached(lens, room, keep, sink, recent, in_place):
    """Cached tokens past the weights' slots count as weight 0: the protected
    ones stay, and lengths are those of the cache."""
    T = U.torch()
    print(f"[evict] {lens} tokens, weights of {room} slots", flush=True)
    hkv, d = 2, 64
    cache = A.Cache(lens, hkv, d, "bf16", 16)
    rng = np.random.default_rng(4)
    w = rng.exponential(size=(2, len(lens), hkv, room)).astype(np.float32)
    w[..., ::7] = -1.0
    mass = T.from_numpy(w.copy()).cuda()
    guard = T.full((mass.numel() + 64,), 5.0, device="cuda")
    out = mass if in_place else guard[:mass.numel()].view(mass.shape)
    kept = T.full((2, len(lens), hkv, keep), -7, dtype=T.int32, device="cuda")
    left = T.zeros(len(lens), dtype=T.int32, device="cuda")
    att = kvx.Attention(kvx.ModelShape(2, hkv, d, 1e4), hkv, kvx.KVX_BF16)
    att.evict(kvx.make_evict_io(cache.struct, A._int(lens), mass, kept, keep, sink=sink,
                                recent=recent, mass_out=out, tokens_out=left))
    T.cuda.synchronize()
    assert left.tolist() == [min(n, keep) for n in lens]
    assert (guard[mass.numel():] == 5.0).all()
    got, wo = kept.cpu().numpy(), out.cpu().numpy()
    for b, n in enumerate(lens):
        for l in range(2):
            for h in range(hkv):
                full = np.zeros(max(n, room), np.float32)
                full[:room] = w[l, b, h]
                ref = R.keep(full[:n], keep, sink, recent)
                assert (got[l, b, h, :len(ref)] == ref).all(), (l, b, h)
                assert (got[l, b, h, len(ref):] == -1).all()
                r = min(len(ref), room)
                assert (wo[l, b, h, :r] == full[ref][:r]).all()
                assert (wo[l, b, h, r:min(room, max(n, keep))] == 0).all()
                for kv in range(2):
                    rows = cache.read(kv, l, b, len(ref))[:, h]
                    assert T.equal(rows, cache.rows[kv][l][b][ref, h]), (l, b, h, kv)
    att.close()


def test_more_weights_than_an_index_holds_are_refused():
    T = U.torch()
    cache = A.Cache([20], 1, 64, "bf16", 16, layers=1)
    att = kvx.Attention(kvx.ModelShape(1, 1, 64, 1e4), 1, kvx.KVX_BF16)
    mass = T.zeros(1, 1, 1, 32, device="cuda")
    kept = T.full((1, 1, 1, 8), -7, dtype=T.int32, device="cuda")
    io = kvx.make_evict_io(cache.struct, A._int([20]), mass, kept, 8, mass_out=mass)
    io.mass_capacity = 2 ** 31 - 1
    with pytest.raises(kvx.KvxError) as e:
        att.evict(io)
    T.cuda.synchronize()
    assert e.value.status == kvx.KVX_ESHAPE and (kept == -7).all()
    att.close()


def test_more_selections_than_a_launch_has():
    """4.3 million (layer, context, KV head) selections of one of two tokens."""
    T = U.torch()
    print("[evict] 4.3 million selections", flush=True)
    layers, batch, hkv, d = 1050, 2, 2048, 16
    assert layers * batch * hkv > 2 ** 22
    g = T.Generator("cuda").manual_seed(0)
    k, v = (T.randn(layers, batch, hkv, 2, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    w = T.rand(layers, batch, hkv, 2, device="cuda", generator=g)
    dst = [T.zeros(layers, batch, hkv, 1, d, dtype=T.bfloat16, device="cuda") for _ in range(2)]
    kept = T.full((layers, batch, hkv, 1), -7, dtype=T.int32, device="cuda")
    left = A._int([0, 0])
    att = kvx.Attention(kvx.ModelShape(layers, hkv, d, 1e4), hkv, kvx.KVX_BF16)
    att.evict(kvx.make_evict_io(kvx.make_cache(k, v), A._int([2, 2]), w, kept, 1, tokens_out=left,
                                dst=kvx.make_cache(dst[0], dst[1])))
    T.cuda.synchronize()
    want = (w[..., 1] > w[..., 0]).long()  # a tie keeps the first
    assert left.tolist() == [1, 1]
    assert T.equal(kept[..., 0].long(), want)
    for s, t in zip((k, v), dst):
        assert T.equal(t[..., 0, :], T.where(want[..., None] == 1, s[..., 1, :], s[..., 0, :]))
    att.close()


@pytest.mark.parametrize("over", [1, 500])
def test_a_context_that_has_outgrown_its_cache(over):
    """The cached slots are what is kept of, the last of them the recent ones."""
    T = U.torch()
    print(f"[evict] {over} tokens past the capacity", flush=True)
    n, hkv, d, keep = 64, 2, 64, 20
    cache = A.Cache([n], hkv, d, "bf16", 16)
    w = np.random.default_rng(2).exponential(size=(2, 1, hkv, n)).astype(np.float32)
    mass = T.from_numpy(w.copy()).cuda()
    kept = T.full((2, 1, hkv, keep), -7, dtype=T.int32, device="cuda")
    left = A._int([0])
    att = kvx.Attention(kvx.ModelShape(2, hkv, d, 1e4), hkv, kvx.KVX_BF16)
    att.evict(kvx.make_evict_io(cache.struct, A._int([n + over]), mass, kept, keep, sink=2, recent=5,
                                mass_out=mass, tokens_out=left))
    T.cuda.synchronize()
    assert left.tolist() == [keep]
    for l in range(2):
        for h in range(hkv):
            ref = R.keep(w[l, 0, h], keep, 2, 5)
            assert (kept[l, 0, h].cpu().numpy() == ref).all()
            for kv in range(2):
                assert T.equal(cache.read(kv, l, 0, keep)[:, h], cache.rows[kv][l][0][ref, h])
    att.close()
