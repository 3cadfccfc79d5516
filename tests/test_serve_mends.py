"""Calls of serving and decoding whose caches or block tables are smaller than the call
says, which would be read out of range (no GPU needed)."""
import pytest
import torch

from paper_2608_30963_amd import kvx
from tests.test_attn_refusals import BF16, INT, _attention, _cache
from tests.test_serve_refusals import _cache8


def _calls(cache, batch, layer=0):
    """(name, struct) of every call that reads or writes one cache."""
    tokens = torch.zeros(batch, dtype=INT)
    q, k = torch.zeros(batch, 4, 64, dtype=BF16), torch.zeros(batch, 2, 64, dtype=BF16)
    io = kvx.make_attn_io(cache, tokens, q, layer=layer, new_q=q, new_k=k, new_v=k, out=q)
    yield "append", io
    yield "forward", kvx.make_attn_io(cache, tokens, q, layer=layer, out=q, window=4, sink=1)
    path = torch.zeros(batch, 2, dtype=INT)
    yield "accept", kvx.make_accept_io(cache, tokens, path, tokens)
    if isinstance(cache, kvx.Cache8):
        yield "pack", kvx.make_pack_io(_wide(batch), cache, tokens)
        yield "unpack", kvx.make_pack_io(_wide(batch), cache, tokens)
    else:
        mass, kept = torch.zeros(2, batch, 2, 32), torch.zeros(2, batch, 2, 8, dtype=INT)
        yield "evict", kvx.make_evict_io(cache, tokens, mass, kept, 8)
        yield "evict", kvx.make_evict_io(_wide(batch), tokens, mass, kept, 8, dst=cache)


def _wide(batch):
    """A cache that has room for all of them."""
    k = torch.zeros(2, batch, 2, 32, 64, dtype=BF16)
    return kvx.make_cache(k, k.clone())


def _call(att, name, io):
    getattr(att, name)(*((io, torch.zeros(8)) if name == "forward" else (io,)))


@pytest.mark.parametrize("make", [_cache, _cache8], ids=["plain", "coded"])
def test_block_tables_of_too_few_contexts_are_refused(make):
    att = _attention()
    cache = make()  # a table of two contexts
    for batch, word in ((2, "GPU"), (3, "table")):
        for name, io in _calls(cache, batch):
            with pytest.raises(ValueError, match=word):
                _call(att, name, io)


@pytest.mark.parametrize("coded", [False, True])
def test_caches_of_too_few_contexts_or_layers_are_refused(coded):
    att = _attention()
    k = torch.zeros(2, 3, 2, 16, 64, dtype=torch.int8 if coded else BF16)
    cache = kvx.make_cache8(k, k.clone(), torch.zeros(2, 3, 2, 16, 2, dtype=BF16)) if coded else \
        kvx.make_cache(k, k.clone())
    for batch, layer, word in ((3, 1, "GPU"), (4, 1, "contexts")):
        for name, io in _calls(cache, batch, layer):
            with pytest.raises(ValueError, match=word):
                _call(att, name, io)
    deep = _attention(n_layers=3)
    for name, io in _calls(cache, 3, 2):
        with pytest.raises(ValueError, match="layers"):
            _call(deep, name, io)
    for name, io in list(_calls(cache, 3, 1))[:2]:  # a layer that it has
        with pytest.raises(ValueError, match="GPU"):
            _call(deep, name, io)
