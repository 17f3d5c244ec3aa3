"""Calls of the operators on a cache in 4 bits, and of the norms, that their documentation allows: host side.  No GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2502_12665_amd import binding as b
    b.lib()
    return b


@pytest.mark.parametrize("batch", [1, 2, 4])
def test_layouts_of_no_tokens(B, batch):
    """Projections of no tokens, of a batch as of one sequence: nothing is refused (their strides say nothing)."""
    d = B.make_dims(batch, 8, 2, 128, 16, 100, 128)
    qkv = torch.zeros(batch, 5, 1536)
    for x in (torch.zeros(batch, 0, 1024), qkv[:, :0, :1024], torch.zeros(batch, 0, 8, 128), qkv[:, 2:2, :1024].unflatten(-1, (8, 128))):
        B._projected(d, x, "q", 8, 0)
    with pytest.raises(ValueError):
        B._projected(d, torch.zeros(batch, 0, 512), "q", 8, 0)
