"""What AttentionBlocks refuses before it touches a device (no GPU)."""
import pytest
import torch

from paper_2609_34054_b200 import inputs as I
from paper_2609_34054_b200.block import AttentionBlocks


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("n_layers,max_rows", [(0, 8), (-1, 8), (2, 0)])
def test_no_layers_or_rows(n_layers, max_rows, shared):
    """Without a layer the stream would be x and whatever the output buffer holds."""
    with pytest.raises(ValueError, match="at least one layer"):
        AttentionBlocks(None, I.C1, n_layers, max_rows, shared_weights=shared)


@pytest.mark.parametrize("shape", [(9, 64), (4, 32), (4, 1), (4,), (2, 4, 64)])
def test_streams_that_do_not_fit(shape):
    """Among them shapes that a copy into the stream would spread over it."""
    blocks = AttentionBlocks.__new__(AttentionBlocks)
    blocks.px, blocks.geo, blocks.n_layers, blocks.e4m3, blocks.r = None, None, 1, False, torch.zeros(8, 64)
    with pytest.raises(ValueError, match="the blocks take up to 8 rows of 64"):
        blocks.forward(torch.zeros(shape), None, None)
