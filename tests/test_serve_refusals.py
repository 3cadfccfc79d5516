"""Arguments of serving (kvx_serve.h) that are refused on the host, the layouts of
its structs, and its reference's own rules (no GPU needed)."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import serve as V
from paper_2608_30963_amd import kvx
from tests.test_attn_refusals import BF16, F32, INT, _attention, _cache

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")


def _cache8(dt=torch.int8, **kw):
    k, v = (torch.zeros(2, 4, 2, 16, 64, dtype=torch.uint8).view(dt) for _ in range(2))
    return kvx.make_cache8(k, v, torch.zeros(2, 4, 2, 16, 2, dtype=BF16), torch.zeros(2, 2, dtype=INT), **kw)


def test_calls_refuse_null():
    lib = kvx.load()
    one = C.c_void_p(1)
    io, view, c8 = kvx.AttnIO(), kvx.AttnView(), kvx.Cache8()
    pack, tree, acc = kvx.PackIO(), kvx.TreeIO(), kvx.AcceptIO()
    E = kvx.KVX_EINVAL
    assert lib.kvx_attn_append_coded(None, C.byref(io), C.byref(c8), None) == E
    assert lib.kvx_attn_append_coded(one, None, C.byref(c8), None) == E
    assert lib.kvx_attn_append_coded(one, C.byref(io), None, None) == E
    for call, s in ((lib.kvx_attn_pack, pack), (lib.kvx_attn_unpack, pack), (lib.kvx_attn_tree, tree),
                    (lib.kvx_attn_accept, acc)):
        assert call(None, C.byref(s), None) == E
        assert call(one, None, None) == E
    assert lib.kvx_attn_forward_view(None, C.byref(io), None, None, 0, None) == E
    assert lib.kvx_attn_forward_view(None, C.byref(io), C.byref(view), None, 0, None) == E
    view.sink = 1
    io.window = 1
    assert lib.kvx_attn_forward_view(None, C.byref(io), C.byref(view), None, 0, None) == E
    assert lib.kvx_attn_forward_view(one, None, C.byref(view), None, 0, None) == E


def test_struct_layouts_match_header(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not available")
    pairs = [(kvx.Cache8, "kvx_cache8"), (kvx.PackIO, "kvx_pack_io"), (kvx.TreeIO, "kvx_tree_io"),
             (kvx.AttnView, "kvx_attn_view"), (kvx.AcceptIO, "kvx_accept_io")]
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "kvx_serve.h"', "int main(void) {"]
    expect = []
    for cls, cname in pairs:
        lines.append(f'  printf("%zu\\n", sizeof({cname}));')
        expect.append(C.sizeof(cls))
        for f in cls._fields_:
            lines.append(f'  printf("%zu\\n", offsetof({cname}, {f[0]}));')
            expect.append(getattr(cls, f[0]).offset)
    lines += ["  return 0;", "}"]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines) + "\n")
    subprocess.run([gcc, "-std=c99", "-I", INCLUDE, str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True,
                                          text=True).stdout.split()]
    assert got == expect


def test_caches_of_8_bits():
    assert _cache8().code == kvx.KVX_CODE_I8 and _cache8(torch.float8_e4m3fn).code == kvx.KVX_CODE_E4M3
    assert _cache8(torch.uint8, code=kvx.KVX_CODE_E4M3).code == kvx.KVX_CODE_E4M3
    k, s = torch.zeros(2, 4, 2, 16, 64, dtype=torch.int8), torch.zeros(2, 4, 2, 16, 2, dtype=BF16)
    kvx.make_cache8(k, k.clone(), s)
    for args in ((k.to(BF16), k.to(BF16), s), (k.view(torch.uint8), k.view(torch.uint8), s),
                 (k, k.view(torch.float8_e4m3fn), s), (k, k, s.float()), (k, k, s[..., :1].contiguous()),
                 (k, k, s[:, :2].contiguous()), (k, k, s.transpose(2, 3)), (k.transpose(2, 3),) * 2 + (s,),
                 (k, k, s, torch.zeros(2, 2, dtype=torch.int64))):
        with pytest.raises(ValueError):
            kvx.make_cache8(*args)


def _io(**kw):
    q, k, v, out = (torch.zeros(3, h, 64, dtype=BF16) for h in (4, 2, 2, 4))
    base = dict(q=q, new_q=q, new_k=k, new_v=v, out=out, q_start=torch.zeros(3, dtype=INT))
    cache = kw.pop("cache", None) or _cache8()
    base.update(kw)
    return kvx.make_attn_io(cache, torch.zeros(2, dtype=INT), **base)


def test_views_are_built():
    io = _io(sink=4, tree=torch.zeros(3, 2, dtype=INT), depth=torch.zeros(3, dtype=INT))
    assert (io.view.sink, io.view.tree_words) == (4, 2) and io.view.cache8 and not io.cache.k
    assert _io(cache=_cache()).view is None
    assert _io(cache=_cache(), sink=1).view.cache8 is None
    for kw in (dict(tree=torch.zeros(3, 2)), dict(tree=torch.zeros(6, dtype=INT)),
               dict(tree=torch.zeros(2, 4, dtype=INT)), dict(tree=torch.zeros(2, 3, dtype=INT).t()),
               dict(depth=torch.zeros(2, dtype=INT)), dict(depth=torch.zeros(3, dtype=torch.int64)),
               dict(q=torch.zeros(3, 4, 64)), dict(new_k=torch.zeros(3, 2, 64, dtype=torch.int8))):
        with pytest.raises(ValueError):
            _io(**kw)


def test_structs_of_another_kind_are_refused():
    tokens = torch.zeros(2, dtype=INT)
    parent, mask = torch.zeros(5, dtype=INT), torch.zeros(5, 2, dtype=INT)
    kvx.make_tree_io(tokens, parent, mask, depth=parent.clone(), pos=torch.zeros(1, 5, dtype=INT),
                     q_start=torch.zeros(3, dtype=INT), shift=tokens)
    for kw in (dict(tokens=tokens.long()), dict(parent=parent.long()), dict(mask=mask.float()),
               dict(mask=mask[:4]), dict(mask=mask.flatten()), dict(depth=parent[:4]),
               dict(pos=torch.zeros(1, 4, dtype=INT)), dict(q_start=tokens), dict(shift=tokens[:1]),
               dict(mask=torch.zeros(5, 4, dtype=INT)[:, ::2])):
        args = dict(tokens=tokens, parent=parent, mask=mask)
        args.update(kw)
        with pytest.raises(ValueError):
            kvx.make_tree_io(args.pop("tokens"), args.pop("parent"), args.pop("mask"), **args)
    path = torch.zeros(2, 4, dtype=INT)
    for cache in (_cache(), _cache8()):
        kvx.make_accept_io(cache, tokens, path, tokens, q_start=torch.zeros(3, dtype=INT), tokens_out=path[:, 0].clone())
        for kw in (dict(path=path.long()), dict(path=path[:1]), dict(path=path[:, ::2]), dict(count=tokens[:1]),
                   dict(tokens_out=tokens.long()), dict(q_start=tokens), dict(path=path.flatten())):
            args = dict(path=path, count=tokens)
            args.update(kw)
            with pytest.raises(ValueError):
                kvx.make_accept_io(cache, tokens, args.pop("path"), args.pop("count"), **args)
    kvx.make_pack_io(_cache(), _cache8(), tokens)
    with pytest.raises(ValueError):
        kvx.make_pack_io(_cache(), _cache8(), tokens.long())


@pytest.mark.parametrize("kw,word", [
    (dict(), "GPU"), (dict(n_kv_heads=4), "KV"), (dict(head_dim=128), "KV"), (dict(n_layers=3), "layers|GPU"),
    (dict(dtype=kvx.KVX_F32), "bytes|GPU")])
def test_structs_of_another_model_are_refused(kw, word):
    """On the CPU every struct is refused, before any call of the library."""
    tokens = torch.zeros(2, dtype=INT)
    att = _attention(**kw)
    pack = kvx.make_pack_io(_cache(), _cache8(), tokens)
    acc = kvx.make_accept_io(_cache8(), tokens, torch.zeros(2, 4, dtype=INT), tokens)
    for call, io in (("append", _io()), ("pack", pack), ("unpack", pack), ("accept", acc)):
        with pytest.raises(ValueError, match=word):
            getattr(att, call)(io)
    with pytest.raises(ValueError, match=word):
        att.forward(_io(), torch.zeros(8))
    tree = kvx.make_tree_io(tokens, tokens, torch.zeros(2, 1, dtype=INT), pos=torch.zeros(1, 2, dtype=INT))
    with pytest.raises(ValueError, match="GPU"):
        att.tree(tree)


def test_codes_of_the_reference():
    """The reference's codes are the nearest ones, and its scales the least."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((300, 16)) * 2.0 ** rng.integers(-120, 120, (300, 1))
    x[0], x[1, 2], x[2, 3] = 0.0, np.nan, np.inf
    for code, table in (("i8", np.arange(-127.0, 128.0)), ("e4m3", np.concatenate([-V.E4M3[:0:-1], V.E4M3]))):
        c, s = V.encode(x, code)
        assert np.isnan(s[1:3]).all() and (c[1:3] == 0).all() and s[0] == 2.0 ** -100
        y = V.decode(c, s, code)
        for i in range(300):
            if i in (1, 2):
                continue
            assert s[i] == 2.0 ** -100 or np.abs(x[i]).max() > V.MOST[code] * s[i] / 2
            assert np.abs(x[i]).max() <= V.MOST[code] * s[i]
            best = np.abs(table[:, None] * s[i] - x[i]).min(0)
            assert (np.abs(y[i] - x[i]) == best).all()
    if hasattr(torch, "float8_e4m3fn"):
        y = torch.from_numpy(x[3:] / V.encode(x, "e4m3")[1][3:, None])
        assert (y.to(torch.float8_e4m3fn).view(torch.uint8).numpy() == V.encode(x, "e4m3")[0][3:]).all()


def test_sights_of_the_reference():
    """A chain sees what tokens in order see; sinks add to a window."""
    for m, n, window, sink in ((5, 12, 0, 0), (7, 30, 6, 2), (9, 9, 3, 4), (4, 3, 2, 1)):
        see, depth = V.tree_sight([i - 1 for i in range(m)], n, window, sink)
        want = V.sight(m, n, window, sink)
        assert (see == want).all() and depth == list(range(m))
        assert (V.sight(m, n, window, 0) <= want).all()
