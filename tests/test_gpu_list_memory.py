"""What an optimizer over a list keeps alive."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu


def test_data_that_a_parameter_had_is_freed():
    n = 64 << 20
    p = torch.nn.Parameter(torch.zeros(n, device="cuda"))
    opt = B.AdamW([p, torch.zeros(2, 3, device="cuda")], bits=8)
    held = torch.cuda.memory_allocated()
    p.data = torch.ones(n, dtype=torch.bfloat16, device="cuda")            # half the size
    assert torch.cuda.memory_allocated() == held - 2 * n
    opt.step([torch.ones(n, device="cuda"), None], lr=0.5, t=0)
    assert bool((p == 0.5).all())
    for other in (torch.zeros(n + 1, device="cuda"), torch.zeros(n // 2, 2, device="cuda")):
        p.data = other
        with pytest.raises(ValueError, match="shapes"):
            opt.step([torch.ones_like(other), None], lr=0.5, t=1)
