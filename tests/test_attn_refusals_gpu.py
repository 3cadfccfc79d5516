"""Structs that are not of an Attention's model, refused before they are run."""
import pytest

from paper_2608_30963_amd import kvx
from tests import gpu_util as U
from tests import test_attn_gpu as A

pytestmark = pytest.mark.gpu


def test_structs_of_another_model_are_refused():
    T = U.torch()
    cache = A.Cache([20], 2, 64, "bf16", 16)
    q, k, v = (A._rows(1, h, 64, "bf16", h) for h in (4, 2, 2))

    def io(**kw):
        base = dict(q=q, new_q=q, new_k=k, new_v=v, out=T.zeros_like(q),
                    lse=T.zeros(1, 4, device="cuda"), mass=T.zeros(1, 2, 32, device="cuda"))
        base.update(kw)
        return kvx.make_attn_io(cache.struct, A._int([20]), **base)

    att = kvx.Attention(kvx.ModelShape(2, 2, 64, 1e4), 4, kvx.KVX_BF16, pair_axis=[0, 1] * 16)
    att.append(io(pos=A._int([3, 4]).view(2, 1)))
    wide = A._rows(1, 8, 64, "bf16", 1)
    bad = [dict(pos=A._int([3]).view(1, 1)), dict(q=wide, new_q=wide, out=wide, lse=None),
           dict(new_k=q, new_v=q), dict(mass=T.zeros(1, 1, 32, device="cuda"))]
    for kw in bad:
        for call in (lambda s: att.append(s), lambda s: att.mass(s),
                     lambda s: att.forward(s, att.workspace())):
            with pytest.raises(ValueError):
                call(io(**kw))
    mass, kept = T.zeros(1, 1, 2, 32, device="cuda"), T.zeros(1, 1, 2, 8, dtype=T.int32, device="cuda")
    with pytest.raises(ValueError):
        att.evict(kvx.make_evict_io(cache.struct, A._int([20]), mass, kept, 8))
    T.cuda.synchronize()
    att.close()
