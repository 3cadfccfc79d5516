"""The example of drafting on a compressed translated cache."""
import pytest

from tests import gpu_util as U

pytestmark = pytest.mark.gpu


def _drafter(config, batch, **kw):
    from examples import draft as D
    from examples.decode import HEADS, handoff
    shape, k, v, table, lengths = handoff(config, 60, batch, 100)
    heads, cap = HEADS[config]
    return D.Drafter(shape, heads, cap, k, v, table, lengths, **kw), lengths


@pytest.mark.parametrize("config,batch,kw", [(2, 1, {}), (3, 2, dict(nodes=9, window=40, sink=4))])
def test_replayed_trees_are_the_eager_ones(config, batch, kw):
    """Captured and replayed steps accept what eager ones do and leave the same cache, and
    guesses that are the target's own choices are accepted."""
    T = U.torch()
    print(f"[draft] config {config}, {batch} contexts", flush=True)
    a, lengths = _drafter(config, batch, **kw)
    b, _ = _drafter(config, batch, **kw)
    g = T.Generator("cuda").manual_seed(3)
    root = T.zeros(batch, dtype=T.int64, device="cuda")
    grown = T.tensor(lengths, device="cuda")
    for turn in range(4):
        drafted = T.randint(0, 32, (batch, a.nodes), device="cuda", generator=g)
        drafted[:, 0] = root
        if turn:  # the first child is what the target chose there a turn ago
            drafted[:, 1] = a.chosen[:, 0]
        ca, la = a.step(drafted)
        cb, lb = b.step(drafted, eager=True)
        T.cuda.synchronize()
        assert T.equal(ca, cb) and T.equal(la, lb) and T.equal(a.tokens, b.tokens), turn
        assert T.equal(a.path, b.path) and (ca >= 1).all() and (ca <= a.deepest).all()
        for x in range(batch):  # every accepted node is what was chosen after its parent
            path = a.path[x, :int(ca[x])].tolist()
            for parent, node in zip(path, path[1:]):
                assert a.up[node] == parent and drafted[x, node] == a.chosen[x, parent]
        grown += ca
        assert a.tokens.tolist() == grown.tolist()
        root = la.clone()
    for x, y in ((a.k, b.k), (a.v, b.v), (a.scale.view(T.int16), b.scale.view(T.int16))):
        assert T.equal(x, y)
    a.close()
    b.close()


def test_main_runs(capsys):
    from examples import draft as D
    D.main(["--tokens", "64", "--steps", "3", "--nodes", "8"])
    assert "tokens accepted" in capsys.readouterr().out
