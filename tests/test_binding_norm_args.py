"""Arguments of the norm calls that are no tensors are named."""

import pytest

import paper_2505_22918_amd as rt


@pytest.mark.parametrize("bad", [1.0, [1.0, 2.0], "weight"])
def test_weights_that_are_no_tensors(bad):
    with pytest.raises(ValueError, match="weight must be a CUDA tensor"):
        rt._norm_weight(bad, "weight", None)
