"""Calls of the operators on a cache in 4 bits, and of the norms, that their documentation allows and that lie beside the ordinary ones,
against plain float64 forms, through the C ABI."""
import pytest
import torch

from paper_2502_12665_amd import binding as B

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("batch", [1, 4])
def test_norms_of_no_tokens(batch):
    """n_new 0 is a no-op, of a batch too."""
    dims = B.make_dims(batch, 8, 2, D, 16, 100, 128)
    qkv = torch.zeros(batch, 0, 12 * D, device="cuda")
    out = torch.empty(batch, 8, 0, D, device="cuda")
    B.qk_norm_rope(dims, qkv[..., : 8 * D], qkv[..., 8 * D: 10 * D], 0, None, None, 1e-6, None, None, q_norm=out,
                   k_norm=torch.empty(batch, 2, 0, D, device="cuda"))
    torch.cuda.synchronize()
