"""What the token operators' Python calls refuse before anything is launched: workspaces that kernels could not write to."""
import pytest
import torch

from paper_2311_16883_amd import binding as B

pytestmark = pytest.mark.gpu


def calls_with_a_workspace():
    """(bytes that the call asks for, the call with a given workspace)."""
    x, ids = torch.zeros(3000, 8, device="cuda"), torch.zeros(3000, dtype=torch.int64, device="cuda")
    e2, w = torch.zeros(3000, 2, dtype=torch.int64, device="cuda"), torch.zeros(3000, 2, device="cuda")
    g = torch.zeros(3000, device="cuda")
    return [
        (B.bsr_embedding_grad_workspace_bytes(3000, 9, 8), lambda ws: B.bsr_embedding_grad(ids, x, 9, ws=ws)),
        (B.bsr_expert_sort_workspace_bytes(6000, 4), lambda ws: B.bsr_expert_sort(e2, 4, ws=ws)),
        (B.bsr_distill_workspace_bytes(3000, 8, 2), lambda ws: B.bsr_distill_loss(x, e2, w, ws=ws)),
        (B.bsr_distill_workspace_bytes(3000, 8, 2), lambda ws: B.bsr_distill_loss_grad(x, e2, w, g, ws=ws)),
    ]


@pytest.mark.parametrize("which", range(4))
def test_a_workspace_is_packed_bytes_on_the_device(which):
    need, call = calls_with_a_workspace()[which]
    assert need > 16
    whole = torch.empty(2 * need, dtype=torch.uint8, device="cuda")
    call(whole)
    call(whole[:need])
    call(whole[:need].view(1, need))
    for ws in (torch.empty(need, dtype=torch.uint8), whole[:16].expand(need, 16), torch.empty(1, dtype=torch.uint8, device="cuda").expand(need),
               whole[::2], torch.empty(need, dtype=torch.int8, device="cuda"), torch.empty(need, device="cuda")):
        assert ws.numel() >= need
        with pytest.raises(ValueError, match="ws must be"):
            call(ws)
    with pytest.raises(TypeError, match="ws must be a tensor"):
        call(need)
    with pytest.raises(B.BsrError) as e:
        call(whole[:need - 1])
    assert e.value.code == B.BSR_ERR_WORKSPACE


def test_sizes_beyond_the_limits_are_refused_before_anything_of_their_size_is_allocated():
    ids, empty = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda")
    x = torch.zeros(4, 8, device="cuda")
    for experts in (1025, 1 << 34, 1 << 40, (1 << 63) - 1):
        with pytest.raises(B.BsrError) as e:
            B.bsr_expert_sort(ids, experts)
        assert e.value.code == B.BSR_ERR_LIMIT
    for vocab in (1 << 30, 1 << 34, 1 << 40, 1 << 61, (1 << 63) - 1):
        for tokens, rows in ((ids, x), (empty, x[:0])):
            with pytest.raises(B.BsrError) as e:
                B.bsr_embedding_grad(tokens, rows, vocab)
            assert e.value.code == B.BSR_ERR_SHAPE
