"""Calls of the operators on a cache in 4 bits, and of the norms, that their documentation allows and that lie beside the ordinary ones,
against plain float64 forms, through the C ABI."""
import pytest
import torch

from paper_2502_12665_amd import binding as B
from tests.test_gpu_kv4 import Case, run_attend

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


@pytest.mark.parametrize("G, shared", [(1, False), (4, False), (3, True), (7, True)])
@pytest.mark.parametrize("q_at, k_at", [(5, 70), (5, 69), (69, 5), (100, 3)])
def test_window_of_large_elements_that_do_not_meet(G, shared, q_at, k_at):
    """A query and keys of 2^100 each, in different elements, also in two of a pair that is not turned (the last token's never is): no
    product that counts is beyond float32, the logits are 0 and the output is the mean of the values, exactly (sums of few bits)."""
    c = Case([8], G, 1, 16, "f32", seed=101, bounds=False)
    c.inv = torch.zeros(64, dtype=torch.float64)            # (no rotation)
    c.k[0] = torch.zeros(1, 8, D)
    c.k[0][:, :, k_at] = 2.0 ** 100
    c.append(c.lens)
    c.q = torch.zeros(1, G, D)
    c.q[..., q_at] = 2.0 ** 100
    got = run_attend(c, [[[] for _ in range(1 if shared else G)]], 1, shared, 8, 0, q_rot=c.q)[0]
    want = c.seq(0, 0)[3].mean(0)
    assert torch.equal(got[0].double(), want.expand(G, D))
