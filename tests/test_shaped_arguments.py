"""What sam_argmax_shaped of the binding checks before it hands addresses on."""
from __future__ import annotations

import pytest
import torch

import paper_2512_18337_b200 as S


@pytest.mark.parametrize("streams", [torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), torch.zeros(3, dtype=torch.int64),
                                     torch.zeros(3), torch.zeros(0, dtype=torch.int32)], ids=str)
def test_streams_of_another_length_or_type(streams):
    """They are read on the device for every row."""
    with pytest.raises(ValueError, match="one entry per row"):
        S.sam_argmax_shaped(16, 100, 3, 2, 100, 16, S.SamShape(100), 16, streams=streams)
