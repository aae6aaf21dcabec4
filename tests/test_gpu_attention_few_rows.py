"""Packed prompts of as many rows as the split begins with: the handle's own workspace is used where a caller's is."""
import pytest
import torch

from paper_2311_09549_amd.attention import Attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,head_dim,rows", [(1, 256, 128), (1, 256, 160), (1, 136, 416), (8, 256, 417), (1, 200, 512), (1, 128, 512), (1, 128, 1024), (1, 64, 1700)])
def test_own_workspace_as_a_callers(dtype, heads, head_dim, rows):
    gen = torch.Generator().manual_seed(rows)
    q, k, v = (torch.randn(rows, h, head_dim, generator=gen).to(dtype).cuda() for h in (heads, 1, 1))
    attention = Attention(heads, 1, head_dim, dtype)
    starts = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    workspace = torch.full((attention.prompt_ws_bytes // 4,), float("nan"), device="cuda")
    assert torch.equal(attention.prompt(q, k, v, starts), attention.prompt(q, k, v, starts, workspace=workspace))
