"""Refusals of kvx_attn.h's entry points, made on the host before any device
work, and the layouts of its structs (no GPU needed)."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2608_30963_amd import kvx

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")


def _desc(**kw):
    base = dict(model=kvx.Model(2, 2, 64, 1e4, None), n_heads=4, dtype=kvx.KVX_BF16, scale=0.0,
                softcap=0.0, n_axes=1, pair_axis=None)
    base.update(kw)
    return kvx.AttnDesc(**base)


def test_create_refuses():
    lib = kvx.load()
    assert lib.kvx_attn_create(None, None) == kvx.KVX_EINVAL
    d = _desc()
    assert lib.kvx_attn_create(C.byref(d), None) == kvx.KVX_EINVAL
    axis = (C.c_uint8 * 32)(*([0] * 31 + [2]))
    inv = (C.c_double * 32)(*([float("nan")] * 32))
    for kw, status in (({"n_heads": 5}, kvx.KVX_EINVAL), ({"n_heads": 0}, kvx.KVX_EINVAL),
                       ({"dtype": 2}, kvx.KVX_EINVAL), ({"scale": -1.0}, kvx.KVX_EINVAL),
                       ({"scale": float("inf")}, kvx.KVX_EINVAL),
                       ({"softcap": -1.0}, kvx.KVX_EINVAL),
                       ({"softcap": float("nan")}, kvx.KVX_EINVAL),
                       ({"n_axes": 0}, kvx.KVX_EINVAL), ({"n_axes": 5}, kvx.KVX_EINVAL),
                       ({"n_axes": 2, "pair_axis": C.cast(axis, C.c_void_p).value}, kvx.KVX_EINVAL),
                       ({"model": kvx.Model(0, 2, 64, 1e4, None)}, kvx.KVX_EINVAL),
                       ({"model": kvx.Model(2, 2, 64, float("nan"), None)}, kvx.KVX_EINVAL),
                       ({"model": kvx.Model(2, 2, 64, 1e4, C.cast(inv, C.c_void_p).value)},
                        kvx.KVX_EINVAL),
                       ({"model": kvx.Model(2, 2, 72, 1e4, None)}, kvx.KVX_EUNSUPPORTED),
                       ({"model": kvx.Model(2, 2, 512, 1e4, None)}, kvx.KVX_EUNSUPPORTED)):
        h = C.c_void_p(123)
        assert lib.kvx_attn_create(C.byref(_desc(**kw)), C.byref(h)) == status, kw
        assert h.value is None
    kvx.kvx_attn_destroy(None)


def test_calls_refuse_null():
    lib = kvx.load()
    io, ev = kvx.AttnIO(), kvx.EvictIO()
    n = C.c_size_t(9)
    assert lib.kvx_attn_append(None, C.byref(io), None) == kvx.KVX_EINVAL
    assert lib.kvx_attn_append(C.c_void_p(1), None, None) == kvx.KVX_EINVAL
    assert lib.kvx_attn_forward(None, C.byref(io), None, 0, None) == kvx.KVX_EINVAL
    assert lib.kvx_attn_mass(None, C.byref(io), None) == kvx.KVX_EINVAL
    assert lib.kvx_attn_evict(None, C.byref(ev), None) == kvx.KVX_EINVAL
    assert lib.kvx_attn_evict(C.c_void_p(1), None, None) == kvx.KVX_EINVAL
    assert lib.kvx_attn_workspace_bytes(None, C.byref(n)) == kvx.KVX_EINVAL and n.value == 0
    assert lib.kvx_attn_workspace_bytes(C.c_void_p(1), None) == kvx.KVX_EINVAL


def test_binding_checks_shapes():
    import torch
    with pytest.raises(ValueError):
        kvx.kvx_attn_create(kvx.ModelShape(1, 1, 64, 1e4), 1, kvx.KVX_BF16, pair_axis=[0] * 31)
    k = torch.zeros(1, 1, 1, 4, 64)
    c = kvx.make_cache(k, k)
    assert c.capacity == 4 and c.block_table is None
    q = torch.zeros(64, 2, 2).transpose(0, 2)
    with pytest.raises(ValueError):
        kvx.make_attn_io(c, torch.zeros(1, dtype=torch.int32), q)


def test_struct_layouts_match_header(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not available")
    pairs = [(kvx.AttnDesc, "kvx_attn_desc"), (kvx.Cache, "kvx_cache"),
             (kvx.AttnIO, "kvx_attn_io"), (kvx.EvictIO, "kvx_evict_io")]
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "kvx_attn.h"',
             "int main(void) {"]
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


def test_recorded_traffic_goes_by_the_fused_kernel_alone(tmp_path, monkeypatch):
    """Sources of decoding are no part of the fused launch: the benchmark's
    recorded traffic holds whatever they are."""
    import bench
    src = tmp_path / "csrc"
    shutil.copytree(bench.KERNEL_SOURCES, src)
    monkeypatch.setattr(bench, "KERNEL_SOURCES", str(src))
    h0 = bench.kernel_source_hash()
    for f in sorted(src.glob("attn*")):
        with open(f, "a") as fh:
            fh.write("\n// edit\n")
    assert bench.kernel_source_hash() == h0
    assert bench.recorded("qwen2.5-7b->qwen2.5-1.5b", "bf16x2", 4096, 1, "contiguous",
                          "traffic_bytes_per_launch") is not None
