"""Caches and trees of the tests of serving (kvx_serve.h)."""
import numpy as np

from oracle import serve as V
from paper_2608_30963_amd import kvx
from tests import gpu_util as U
from tests.test_attn_gpu import Cache, _f64, _int, _starts  # noqa: F401

DT = {"i8": "int8", "e4m3": "float8_e4m3fn"}


class Cache8:
    """A cache of 8 bits of `layers` layers whose contexts hold lens tokens: their
    numbers (k, v [layer][context][n, H, D] in 64 bits) and their places on the
    device.  Slots past a context's tokens, and the spare block that unused table
    entries name, hold code 127, of e4m3 no number, and NaN scales."""

    def __init__(self, lens, hkv, d, code, page, layers=2, strided=False, seed=0, extra=0, size=1.0):
        T = U.torch()
        rng = np.random.default_rng(seed + 77)
        self.lens, self.page, self.code, self.layers, self.strided = lens, page, code, layers, strided
        batch, cap = len(lens), max(max(lens) + extra, 1)
        if page:
            per = -(-cap // page)
            nb = batch * per + 1
            perm = rng.permutation(nb)
            table = np.full((batch, per), int(perm[-1]), np.int32)
            k = 0
            for b, n in enumerate(lens):
                used = -(-(n + extra) // page)
                table[b, :used] = perm[k:k + used]
                k += used
            self.host_table, self.table = table, T.from_numpy(table).cuda()
            outer, slots = nb, page
        else:
            self.host_table = self.table = None
            outer, slots = batch, cap
        self.shape = (layers, outer, hkv, slots, d)
        # strided: [layer][block][slot][head], rows of D + 16 bytes, scales with gaps
        if strided:
            codes = [np.full((layers, outer, slots, hkv, d + 16), 127, np.uint8) for _ in range(2)]
            self.codes = [c[..., :d].transpose(0, 1, 3, 2, 4) for c in codes]
            scale = np.full((layers, outer, slots, hkv, 3, 2), np.nan, np.float32)
            self.scale = scale[..., 1, :].transpose(0, 1, 3, 2, 4)
        else:
            codes = [np.full(self.shape, 127, np.uint8) for _ in range(2)]
            self.codes = codes
            scale = np.full(self.shape[:-1] + (2,), np.nan, np.float32)
            self.scale = scale
        self.rows = [[[None] * batch for _ in range(layers)] for _ in range(2)]
        for kv in range(2):
            for l in range(layers):
                for b, n in enumerate(lens):
                    x = rng.standard_normal((n, hkv, d)) * size * np.exp(rng.standard_normal((1, hkv, 1)))
                    c, s = V.encode(x, code)
                    blk, slot = self.place(b, np.arange(n))
                    self.codes[kv][l, blk, :, slot] = c
                    self.scale[l, blk, :, slot, kv] = s
                    self.rows[kv][l][b] = V.decode(c, s, code)
        dt = getattr(T, DT[code])
        self.base = [T.from_numpy(c).cuda() for c in codes] + [T.from_numpy(scale).bfloat16().cuda()]
        if strided:
            self.dev = [t[..., :d].transpose(2, 3) for t in self.base[:2]]
            self.dscale = self.base[2][..., 1, :].transpose(2, 3)
            s = self.dev[0].stride()[:4]
            ss = [x // 2 for x in self.dscale.stride()[:4]]
            kw = dict(stride=s, scale_stride=ss,
                      code=kvx.KVX_CODE_I8 if code == "i8" else kvx.KVX_CODE_E4M3)
            kw.update(dict(block_size=page, num_blocks=outer) if page else dict(capacity=cap))
            self.struct = kvx.make_cache8(self.dev[0], self.dev[1], self.dscale, self.table, **kw)
        else:
            self.dev, self.dscale = self.base[:2], self.base[2]
            self.struct = kvx.make_cache8(*(t.view(dt) for t in self.dev), self.dscale, self.table)

    def place(self, b, j):
        j = np.asarray(j)
        if self.page:
            return self.host_table[b][j // self.page].astype(np.int64), j % self.page
        return np.full_like(j, b), j

    def read(self, kv, l, b, j):
        """(codes [n, H, D], scales [n, H]) of slots j of a context on the device."""
        blk, slot = self.place(b, j)
        codes = self.dev[kv].cpu().numpy()[l][blk, :, slot]
        return codes, self.dscale.float().cpu().numpy()[l][blk, :, slot, kv]

    def f64(self, kv, l, b):
        return self.rows[kv][l][b]


def random_tree(m, rng, roots=1, back=6):
    """Parents of a tree (or several) of m nodes."""
    return [-1 if i < roots else int(max(0, i - rng.integers(1, back + 1))) for i in range(m)]


def masks(parents, see, words):
    """[m, words] as int32 of the seen nodes."""
    m = len(parents)
    out = np.zeros((m, words), np.uint32)
    for i in range(m):
        for k in range(see.shape[1]):
            if see[i, k]:
                out[i, k // 32] |= np.uint32(1 << (k % 32))
    return out.view(np.int32)
