"""Arguments of decoding that would be read as something else, refused on the
host (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2608_30963_amd import kvx

INT, F32, BF16 = torch.int32, torch.float32, torch.bfloat16


def _cache(dt=BF16):
    k, v = (torch.zeros(2, 4, 2, 16, 64, dtype=dt) for _ in range(2))
    return kvx.make_cache(k, v, torch.zeros(2, 2, dtype=INT))


def _io(**kw):
    q, k, v, out = (torch.zeros(3, h, 64, dtype=BF16) for h in (4, 2, 2, 4))
    base = dict(q=q, new_q=q, new_k=k, new_v=v, out=out, q_start=torch.zeros(3, dtype=INT),
                pos=torch.zeros(2, 3, dtype=INT), prefix=torch.zeros(2, dtype=INT),
                lse=torch.zeros(3, 4), mass_in=torch.zeros(2, 2, 32), mass=torch.zeros(2, 2, 32))
    tokens = kw.pop("tokens", torch.zeros(2, dtype=INT))
    cache = kw.pop("cache", None) or _cache()
    base.update(kw)
    return kvx.make_attn_io(cache, tokens, **base)


def test_calls_are_built():
    io = _io()
    assert (io.batch, io.rows, io.mass_capacity) == (2, 3, 32)
    _io(q=None, new_q=None, out=None, lse=None)
    _io(pos=None, q_start=None, prefix=None, mass_in=None, mass=None, new_q=None)
    wide = torch.zeros(3, 8, 64, dtype=BF16)  # strided rows
    _io(q=wide[:, :4], new_q=wide[:, 2:6], new_k=wide[:, :2], new_v=wide[:, 6:], out=wide[:, 4:])
    _io(tokens=torch.zeros(2, dtype=INT), mass=torch.zeros(3, 2, 2, 32)[1])


@pytest.mark.parametrize("kw", [
    dict(tokens=torch.zeros(2, dtype=torch.int64)), dict(tokens=torch.zeros(4, dtype=INT)[::2]),
    dict(q_start=torch.zeros(3, dtype=torch.int64)), dict(q_start=torch.zeros(2, dtype=INT)),
    dict(pos=torch.zeros(1, 3, dtype=INT).expand(2, 3)), dict(pos=torch.zeros(2, 3)),
    dict(pos=torch.zeros(3, 2, dtype=INT)), dict(pos=torch.zeros(3, 2, dtype=INT).t()),
    dict(prefix=torch.zeros(1, dtype=INT)), dict(prefix=torch.zeros(2, dtype=torch.int16)),
    dict(lse=torch.zeros(3, 4, dtype=torch.float64)), dict(lse=torch.zeros(3, 3)),
    dict(lse=torch.zeros(4, 3).t()), dict(mass=torch.zeros(2, 2, 32, dtype=BF16)),
    dict(mass=torch.zeros(2, 32, 2).transpose(1, 2)), dict(mass_in=torch.zeros(2, 2, 31)),
    dict(q=torch.zeros(3, 4, 64)), dict(out=torch.zeros(3, 2, 64, dtype=BF16)),
    dict(new_v=torch.zeros(2, 2, 64, dtype=BF16)), dict(new_k=torch.zeros(3, 2, 32, dtype=BF16)),
    dict(new_q=torch.zeros(3, 256, dtype=BF16)), dict(cache=_cache(F32)),
    dict(tokens=torch.zeros(2, dtype=INT, device="meta"))],
    ids=lambda kw: next(iter(kw)))
def test_tensors_of_another_kind_are_refused(kw):
    with pytest.raises(ValueError):
        _io(**kw)


def test_caches_of_another_layout_are_refused():
    k = torch.zeros(2, 4, 2, 16, 64, dtype=BF16)
    with pytest.raises(ValueError):
        kvx.make_cache(k, k.float())
    with pytest.raises(ValueError):
        kvx.make_cache(k.transpose(2, 3), k.transpose(2, 3))
    with pytest.raises(ValueError):
        kvx.make_cache(k, k[:, :2].contiguous())
    for table in (torch.zeros(2, 2, dtype=torch.int64), torch.zeros(2, 4, dtype=INT)[:, ::2]):
        with pytest.raises(ValueError):
            kvx.make_cache(k, k, table)
    s = k.stride()
    kvx.make_cache(k.transpose(2, 3), k.transpose(2, 3), None, (s[0], s[1], s[2], s[3]),
                   capacity=16)


def test_evictions_of_another_kind_are_refused():
    tokens, mass = torch.zeros(2, dtype=INT), torch.zeros(2, 2, 2, 32)
    kept = torch.zeros(2, 2, 2, 8, dtype=INT)
    kvx.make_evict_io(_cache(), tokens, mass, kept, 8, mass_out=mass,
                      tokens_out=torch.zeros_like(tokens), dst=_cache())
    for kw in (dict(tokens=tokens.long()), dict(mass=mass.double()), dict(kept=kept.long()),
               dict(kept=kept[..., :7].contiguous()), dict(mass_out=mass[..., ::2]),
               dict(tokens_out=tokens.long()), dict(tokens_out=tokens[:1]), dict(dst=_cache(F32))):
        args = dict(tokens=tokens, mass=mass, kept=kept)
        args.update(kw)
        with pytest.raises(ValueError):
            kvx.make_evict_io(_cache(), args.pop("tokens"), args.pop("mass"), args.pop("kept"), 8,
                              **args)


def _attention(n_heads=4, dtype=kvx.KVX_BF16, n_axes=2, **model):
    """The checks of an Attention, without its handle."""
    shape = dict(n_layers=2, n_kv_heads=2, head_dim=64, rope_base=1e4)
    shape.update(model)
    att = object.__new__(kvx.Attention)
    att.handle, att.model, att.n_heads, att.dtype = None, kvx.ModelShape(**shape), n_heads, dtype
    att.n_axes = n_axes
    return att


@pytest.mark.parametrize("kw,word", [
    (dict(), "GPU"), (dict(n_heads=8), "GPU"), (dict(dtype=kvx.KVX_F32), "bytes"),
    (dict(n_kv_heads=4), "KV"), (dict(head_dim=128), "KV")])
def test_structs_of_another_model_are_refused(kw, word):
    """On the CPU every struct is refused, before any call of the library."""
    for call, io in (("append", _io()), ("mass", _io()),
                     ("evict", kvx.make_evict_io(_cache(), torch.zeros(2, dtype=INT),
                                                 torch.zeros(2, 2, 2, 32),
                                                 torch.zeros(2, 2, 2, 8, dtype=INT), 8))):
        with pytest.raises(ValueError, match=word):
            getattr(_attention(**kw), call)(io)
    with pytest.raises(ValueError, match=word):
        _attention(**kw).forward(_io(), torch.zeros(8))


@pytest.mark.parametrize("kw", [
    dict(softcap=1e-39), dict(softcap=1e-320), dict(softcap=3e38), dict(softcap=1e300),
    dict(scale=1e39), dict(scale=1e-39), dict(softcap=1e38, scale=1e-3), dict(softcap=1e-30, scale=1e9)])
def test_scales_and_caps_past_fp32_are_refused(kw):
    """The kernels would have an infinite scale, or no cap where one was asked for."""
    base = dict(model=kvx.Model(2, 2, 64, 1e4, None), n_heads=4, dtype=kvx.KVX_BF16, scale=0.0,
                softcap=0.0, n_axes=1, pair_axis=None)
    base.update(kw)
    h = C.c_void_p(123)
    assert kvx.load().kvx_attn_create(C.byref(kvx.AttnDesc(**base)), C.byref(h)) == kvx.KVX_EINVAL
    assert h.value is None
