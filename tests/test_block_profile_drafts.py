"""block_profile's trees of drafted tokens, without a GPU."""
import pytest

from paper_2606_03770_gb300 import block_profile as P


def test_branching():
    assert P.branching("1") == [-1, 0]
    assert P.branching("1.1.1") == [-1, 0, 1, 2]
    assert P.branching("3.2") == [-1, 0, 0, 0, 1, 1, 2, 2, 3, 3]
    assert len(P.branching("63")) == 64
    for bad in ("", "0", "2.", "a", "-1", "64", "3.3.3.3", "1.5x", "999999999"):
        with pytest.raises(ValueError):
            P.branching(bad)
    with pytest.raises(SystemExit):
        P.main(["--draft", "0"])
