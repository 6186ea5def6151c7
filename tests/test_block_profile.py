"""block_profile without a GPU: what it refuses, and what it gives the planner."""
import pytest

from paper_2606_03770_gb300 import block_profile as P
from paper_2606_03770_gb300 import workloads as W


def test_models_with_other_weights_are_refused(capsys):
    """The block's weights have 4 bits: no rates of it for a model whose weights have 16."""
    with pytest.raises(ValueError, match="4-bit"):
        P.measure(W.CONFIGS["c1_tiny"]["model"], 64, 64, 2)
    with pytest.raises(SystemExit):
        P.main(["--config", "c1_tiny"])
    assert "c1_tiny" in capsys.readouterr().err
