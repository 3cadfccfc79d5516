"""What the example of drafting asks for before it uses the GPU."""
import pytest


def test_no_steps_are_refused():
    from examples import draft as D
    for bad in (["--steps", "0"], ["--steps", "-1"], ["--nodes", "0"]):
        with pytest.raises(SystemExit):
            D.main(bad)
