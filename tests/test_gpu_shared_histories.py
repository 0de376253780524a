"""Adjusted logits of many rows that share histories, where a block goes on from row to row with one table: the bits of calls in which every row
has a history of its own, and some rows against the definition in 64 bits."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B
from test_gpu_adjust import check, plain, plain_grad
from rounding import between

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# A block takes several rows in turn once there are about 19000 rows times chunks of the vocabulary, here four (ragged: two at the end), two, and two
# of three chunks of a larger vocabulary.  Histories of up to 4096 tokens are counted in 16 bits, longer ones in 32.
SHAPES = {"ends inside a block": (40002, 100, 3, 40), "two histories": (40002, 100, 20001, 4000), "long": (40002, 67, 13334, 5000),
          "long, ends inside a block": (20001, 33, 59, 4500), "several chunks": (7002, 20001, 1167, 3000)}


def walk(n, share, length, g):
    """Lengths (or starts) from row to row: the same, a token more, about as many more as a block has threads (128 or 256), more than that, fewer, and
    from the beginning again."""
    step = torch.tensor([0, 1, 1, 1, 2, 127, 128, 129, 255, 256, 257, 700, -1, -3, -200, -10 ** 6])[torch.randint(0, 16, (n,), generator=g)].tolist()
    out, at = [], 0
    for i in range(n):
        at = 0 if i % share == 0 and step[i] % 2 else min(max(at + step[i], -1), length + 1)
        out.append(at)
    return torch.tensor(out, dtype=torch.int32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_rows_in_turn_are_rows_alone(shape, dtype):
    n, vocab, share, length = SHAPES[shape]
    g = torch.Generator().manual_seed(21)
    z = (torch.randn(n, vocab, generator=g) * 3).to(dtype)
    dy = torch.randn(n, vocab, generator=g).to(dtype)
    history = torch.randint(-2, vocab + 2, (n // share, length), generator=g).to(torch.int32)
    r = {"lengths": walk(n, share, length, g), "start": walk(n, share, length, g), "repetition": torch.rand(n, generator=g) + 0.5,
         "frequency": torch.randn(n, generator=g), "presence": torch.randn(n, generator=g)}
    mask = torch.randint(-2 ** 31, 2 ** 31, (n, (vocab + 31) // 32), generator=g).to(torch.int32)
    bias = torch.randn(vocab, generator=g).to(dtype)
    zc, dc, rc, mc = z.cuda(), dy.cuda(), {k: v.cuda() for k, v in r.items()}, mask.cuda()
    shared, alone = history.cuda(), history.cuda().repeat_interleave(share, 0)
    some = torch.cat([torch.arange(12), torch.randint(0, n, (12,), generator=g), torch.arange(n - 6, n)])
    for rules in (dict(), dict(mask=mc), dict(mask=mc[:1], bias=bias.cuda())):
        want = B.adjust_logits(zc, history=alone, **rc, **rules)
        got = B.adjust_logits(zc, history=shared, **rc, **rules)
        assert torch.equal(got, want)
        place = zc.clone()
        assert torch.equal(B.adjust_logits(place, history=shared, **rc, out=place, **rules), want)
        picked = {k: v[some] for k, v in r.items()} | {"history": history[some // share]}
        picked |= {k: v.cpu() if v.shape[0] != n else v.cpu()[some] for k, v in rules.items()}
        check(got[some.cuda()], *plain(z[some], picked))

        rules.pop("bias", None)
        given = dict(lengths=rc["lengths"], repetition=rc["repetition"], **rules)
        d_want = B.adjust_logits_grad(zc, dc, history=alone, **given)
        for out in (None, dc.clone()):
            d = dc if out is None else out
            assert torch.equal(B.adjust_logits_grad(zc, d, history=shared, out=out, **given).logits, d_want.logits)
        both = B.adjust_logits_grad(zc, dc, history=shared, bias="shared", **given)
        assert torch.equal(both.logits, d_want.logits)
        assert torch.equal(both.bias, B.adjust_logits_grad(zc, dc, bias="shared", **rules).bias)      # (penalties do not touch it)
        dz, *_ = plain_grad(z[some], dy[some], picked)
        assert between(d_want.logits[some.cuda()].cpu(), dz, U * dz.abs())
