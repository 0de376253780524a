"""Log probabilities: a common offset of the logits, rows that every part of the chip shares, words at every boundary."""
import math

import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
# vocabulary sizes: less than a vector, one and several rounds of a block; with few rows they are shared by 1, 2, 4 and 8 CTAs
SIZES = [5, 130, 1023, 1024, 1031, 2050, 4099, 8200, 33001]


def rows_of(dtype, rows, vocab, shift):
    """A buffer whose rows start `shift` elements after a 16-byte boundary, each at another one where the stride is odd."""
    wide = torch.empty(rows * (vocab + 3) + shift + 8, dtype=dtype, device="cuda")
    return wide[shift:shift + rows * (vocab + 3)].view(rows, vocab + 3)[:, :vocab]


@pytest.mark.parametrize("offset", [1e4, -1e4, 65536.0])
@pytest.mark.parametrize("scale", [1.0, 0.5])
@pytest.mark.parametrize("rows,vocab", [(1, 300), (3, 5000), (2, 40000), (400, 1000)])
def test_a_common_offset_changes_nothing(rows, vocab, scale, offset):
    g = torch.Generator(device="cuda").manual_seed(2)
    z = torch.randint(-12, 13, (rows, vocab), generator=g, device="cuda").float()          # whole numbers: the sum is exact
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    a = B.token_logprobs(z, t, scale=scale, top=min(20, vocab))
    b = B.token_logprobs(z + offset, t, scale=scale, top=min(20, vocab))
    logp = torch.log_softmax(z.double() * scale, 1)
    want = logp.gather(1, t[:, None])[:, 0]
    # log s is rounded at up to 2^4, the difference to it at up to 2^5, 2^x is good to 2^-21 and the sums of a thread's
    # vocab / 256 terms and of 16 joins add 2^-24 each at most
    tol = (2 ** 4 + 2 ** 5) * 2.0 ** -24 + 2.0 ** -21 + 2.0 ** -24 * (vocab / 256 + 16)
    for r in (a, b):
        assert ((r.logprob.double() - want).abs().max().item()) <= tol
        best = logp.gather(1, r.top_index.long())
        assert ((r.top_logprob.double() - best).abs().max().item()) <= tol
        assert bool((r.logprob <= 0).all()) and bool((r.top_logprob <= 0).all())
    assert torch.equal(a.top_index, b.top_index)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_certain_word_has_no_positive_log_probability(dtype):
    # the words before it leave the reference below it by every amount that does not move it
    vocab = 6000
    for lead in [0.25 * k for k in range(48)]:
        z = torch.full((2, vocab), -30.0, device="cuda")
        z[:, :2000] = -1.0 - 20 * torch.rand(2000, device="cuda")
        z[:, 5] = 1.0
        z[:, 5990] = 1.0 + lead
        t = torch.tensor([5990, 5], device="cuda")
        r = B.token_logprobs(z.to(dtype), t, top=3)
        logp = torch.log_softmax(z.to(dtype).double(), 1)
        assert bool((r.logprob <= 0).all()) and bool((r.top_logprob <= 0).all())
        assert ((r.logprob.double() - logp.gather(1, t[:, None])[:, 0]).abs().max().item()) <= 3e-6


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 20, 40, 100])
@pytest.mark.parametrize("vocab", SIZES)
def test_equal_words_count_once_each(vocab, rows, dtype):
    # n words of the same value: lse and entropy are log n; one lost or doubled word changes them by 1 / n
    for shift in (0, 1, 3):
        z = rows_of(dtype, rows, vocab, shift)
        z.fill_(0.5)
        t = torch.zeros(rows, dtype=torch.int64, device="cuda")
        # the sum is a whole number below 2^24: exact; its logarithm and the sum with 0.5 are rounded at up to 16
        for top in (0, min(7, vocab)):
            r = B.token_logprobs(z, t, top=top)
            tol = 3 * 16 * 2.0 ** -24
            assert tol < 0.5 / vocab
            for got, want in ((r.lse, 0.5 + math.log(vocab)), (r.entropy, math.log(vocab)), (r.logprob, -math.log(vocab))):
                assert ((got.double() - want).abs().max().item()) <= tol


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", SIZES)
def test_one_word_at_every_boundary(vocab, dtype):
    # the dominant word visits the ends of the row and both sides of every place where a part, a head or a tail may end
    places = {p for k in range(9) for p in range((vocab * k) // 8 - 9, (vocab * k) // 8 + 10)} | set(range(20))
    places = sorted(p for p in places if 0 <= p < vocab)
    for shift in (0, 1, 5):
        for rows in ([len(places)] if vocab > 4000 else [1, len(places)]):          # one by one, and all at once
            for first in range(0, len(places), rows):
                if rows == 1 and first % 5:
                    continue
                some = places[first:first + rows]
                z = rows_of(dtype, len(some), vocab, shift)
                z.fill_(-2.0)
                t = torch.tensor(some, device="cuda")
                z[torch.arange(len(some), device="cuda"), t] = 6.0
                r = B.token_logprobs(z, t, top=2 if vocab > 1 else 1)
                want = -math.log1p((vocab - 1) * math.exp(-8.0))
                # exact to the roundings of 2^x, the sums and one logarithm (values up to 16); twice the word or none of it
                # changes the result by log 2 or to -8 and less
                assert ((r.logprob.double() - want).abs().max().item()) <= 2.0 ** -20 + 2.0 ** -24 * (vocab / 256 + 64)
                assert torch.equal(r.top_index[:, 0].long(), t)
                assert torch.equal(r.top_index[:, 1].long(), (t == 0).long())


@pytest.mark.parametrize("rows", [1, 3, 18, 37, 74, 75])
def test_few_rows_of_a_long_vocabulary(rows):
    # rows shared by 8, 8, 4, 2 and 1 CTAs: one word each of n is lost or doubled if a part ends in the wrong place
    vocab = 40007
    z = rows_of(torch.float32, rows, vocab, 1)
    z.fill_(-math.inf)
    places = torch.arange(0, vocab, 5001, device="cuda")
    z[:, places] = 1.0
    z[:, -1] = 1.0
    n = len(places) + 1
    t = torch.full((rows,), vocab - 1, dtype=torch.int64, device="cuda")
    r = B.token_logprobs(z, t, top=n)
    assert ((r.entropy.double() - math.log(n)).abs().max().item()) <= 1e-6
    assert ((r.logprob.double() + math.log(n)).abs().max().item()) <= 1e-6
    assert torch.equal(r.top_index, torch.cat([places, t[:1]]).int().repeat(rows, 1))
