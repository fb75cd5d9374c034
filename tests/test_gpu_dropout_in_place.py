"""Dropout in place, on maps whose rows take several turns of a work-group and
whose work-groups take several turns of the rows."""
import pytest
import torch

from parity import say
from paper_2509_05512_amd import quan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("n,c,h,w", [(3, 37, 60, 61), (1, 515, 70, 70), (40, 16, 50, 50), (2, 2049, 3, 5)])
def test_in_place(n, c, h, w, dtype):
    say(f"dropout in place {n} {c} {h} {w} {dtype}")
    g = torch.Generator().manual_seed(1)
    x = torch.randn((n, h, w, 4, c), generator=g).to(dtype).cuda().permute(0, 3, 4, 1, 2)
    rng = torch.tensor([5, 6], dtype=torch.int64, device="cuda")
    for p in (0.0, 0.3):
        want = quan.quan_dropout(x, p, rng)
        held = x.clone(memory_format=torch.preserve_format)
        assert torch.equal(quan.quan_dropout(held, p, rng, out=held), want)
