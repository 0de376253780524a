"""The gradient of a shared bias summed over more than 2^31 elements: every column its own value."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_shared_bias_past_31_bits(dtype):
    n, vocab = 36000, 60001
    keep = vocab // 32 * 32
    row = (torch.arange(vocab, device="cuda") % 8 + 1).to(dtype)           # sums of up to 288000: exact in fp32
    sign = torch.ones(n, 1, dtype=dtype, device="cuda")
    sign[::3] = -1                                                         # 24000 rows count up, 12000 down
    d = row * sign
    d[-1, 7:11] = 16                                                       # and the last row otherwise
    want = row.double() * (24000 - 12000)
    want[7:11] += 16 - row[7:11].double() * float(sign[-1])
    mask = torch.full((1, (vocab + 31) // 32), -1, dtype=torch.int32, device="cuda")
    mask[0, -1] = 0
    got = B.adjust_logits_grad(d, d, mask=mask, bias="shared", out=d).bias
    assert torch.equal(got[:keep], want[:keep].to(dtype)) and not got[keep:].any()
