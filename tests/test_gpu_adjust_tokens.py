"""Tokens and named words at the ends of their types count nowhere, in no chunk of the vocabulary."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("itype", [torch.int32, torch.int64])
@pytest.mark.parametrize("length", [40, 5000])
def test_tokens_outside_the_vocabulary(itype, length):
    n, vocab = 3, 40_001
    g = torch.Generator().manual_seed(31)
    ends = torch.iinfo(itype)
    bad = torch.tensor([ends.min, ends.min + 1, ends.min + 8192, ends.max, ends.max - 1, -1, -8192, vocab, vocab + 8192, 2 ** 31 - 1, -2 ** 31], dtype=itype)
    if itype == torch.int64:                     # the low half of these is a word
        bad = torch.cat([bad, torch.tensor([2 ** 32, 2 ** 32 + 5, -2 ** 32 + 7, 2 ** 62 + 9])])
    z = torch.randn(n, vocab, generator=g).cuda()
    history = torch.randint(0, vocab, (n, length), generator=g).to(itype)
    where = torch.rand(n, length, generator=g) < 0.5
    mixed = torch.where(where, bad[torch.randint(0, bad.numel(), (n, length), generator=g)], history).cuda()
    plain = torch.where(where, torch.full_like(history, -1), history).cuda()
    words = torch.randint(0, vocab, (n, 2 * bad.numel()), generator=g).to(itype)
    words[:, ::2] = bad
    value = torch.randn(words.shape, generator=g).cuda()
    clean = words.clone()
    clean[:, ::2] = -1
    for out in (None, z):
        y = [B.adjust_logits(z.clone(), history=h, repetition=1.7, frequency=0.3, presence=0.1, bias_index=w.cuda(), bias_value=value,
                             out=None if out is None else z.clone()) for h, w in ((mixed, words), (plain, clean))]
        assert torch.equal(*y) and not torch.equal(y[0], z)
    d = [B.adjust_logits_grad(z, z, history=h, repetition=1.7, bias_index=w.cuda()) for h, w in ((mixed, words), (plain, clean))]
    assert torch.equal(d[0].logits, d[1].logits) and torch.equal(d[0].value, d[1].value) and not d[0].value[:, ::2].any()
    seen = torch.zeros(n, vocab, dtype=torch.bool)
    for i in range(n):
        seen[i, history[i][~where[i]].long()] = True
    assert torch.equal((d[0].logits != z).cpu(), seen & (z != 0).cpu())
