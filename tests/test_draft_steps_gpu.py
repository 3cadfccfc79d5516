"""Steps of the example of drafting that follow each other."""
import pytest

from tests import gpu_util as U
from tests.test_draft_gpu import _drafter

pytestmark = pytest.mark.gpu


def test_replayed_steps_do_not_wait_for_the_device():
    """A step that surely fits asks the device nothing; one that may not fit looks at the
    lengths, and is refused if it does not."""
    T = U.torch()
    d, lengths = _drafter(2, 1)
    drafted = T.zeros(1, d.nodes, dtype=T.int64, device="cuda")
    d.step(drafted)
    T.cuda.synchronize()
    T.cuda.set_sync_debug_mode("error")
    try:
        for _ in range(8):
            d.step(drafted)
    finally:
        T.cuda.set_sync_debug_mode("default")
    T.cuda.synchronize()
    with pytest.raises(ValueError, match="fit"):
        for _ in range(200):
            d.step(drafted)
    assert d.room - d.nodes < int(d.tokens.max()) <= d.room
    d.close()
