"""What the example of drafting asks for before it uses the GPU."""
import pytest


def test_no_steps_are_refused():
    from examples import draft as D
    for bad in (["--steps", "0"], ["--steps", "-1"], ["--nodes", "0"]):
        with pytest.raises(SystemExit):
            D.main(bad)


@pytest.mark.parametrize("nodes,deepest", [(1, 1), (2, 2), (16, 5), (255, 8), (256, 9), (512, 10)])
def test_the_cache_has_room_for_every_path(nodes, deepest, monkeypatch):
    """Should every tree's longest path be accepted, the last tree still fits."""
    from examples import draft as D

    class Asked(Exception):
        pass

    def handoff(config, tokens, batch, room):
        raise Asked(room)

    monkeypatch.setattr(D, "handoff", handoff)
    with pytest.raises(Asked) as e:
        D.main(["--steps", "50", "--nodes", str(nodes)])
    assert e.value.args[0] >= 50 * deepest + nodes
