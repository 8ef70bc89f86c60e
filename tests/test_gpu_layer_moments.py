"""The optimizer's moments where their numbers come to an end: gradients of any NaN."""
import pytest
import torch

from paper_2311_16883_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,word", [(torch.float32, -1), (torch.float32, 0x7FFFFFFF), (torch.float32, 0x7F800001), (torch.bfloat16, -1), (torch.bfloat16, 0x7FFF)])
def test_a_nan_of_any_bits_makes_both_moments_of_its_block_nan(dtype, word):
    g = torch.full((300,), 1e-3, dtype=dtype)
    g.view(torch.int32 if dtype == torch.float32 else torch.int16)[130] = word
    assert bool(g[130].isnan())
    batch = B.AdamWBatch([torch.zeros(300, device="cuda")], [g.cuda()], bits=8)
    B.bsr_adamw_batched(batch, lr=1e-3, step=1)
    m, r, scales = batch.states[0]
    assert (scales[:, 1] == 255).all() and not (scales[:, (0, 2)] == 255).any()
    for codes, row, which in ((m, 0, "m"), (r, 1, "r")):
        values = B.bsr_adamw_state_values(codes, scales[row].contiguous(), which)
        assert bool(values[128:256].isnan().all()) and not bool(values[:128].isnan().any()) and not bool(values[256:].isnan().any())
    assert bool(batch.params[0][130].isnan()) and int(batch.params[0].isnan().sum()) == 1
