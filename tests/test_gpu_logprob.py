"""Token log probabilities, entropy, alternatives and gradient, through the C ABI, against 64-bit formulas."""
import math

import pytest
import torch

from paper_2412_05270_b200 import binding as B
from rounding import between

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
SIZES = [(1, 1), (3, 2), (5, 7), (2, 33), (4, 255), (7, 1000), (300, 1029), (1, 32000), (2, 70001), (16, 5000), (170, 4096)]


def make(rows, vocab, dtype, seed, mask=0.0, pad=0, itype=torch.int64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(rows, vocab + pad, generator=g, device="cuda") * 3
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    if mask:
        z[torch.rand(z.shape, generator=g, device="cuda") < mask] = -math.inf
        z[rows // 2] = -math.inf                       # nothing left
        t[rows // 3] = -100                            # ignored
        t[rows - 1] = vocab
    return z.to(dtype)[:, :vocab], t.to(itype)


def exact(z, t, scale):
    z = (z.float() * scale).double()                   # the product is rounded to fp32 by definition of the inputs here
    rows, vocab = z.shape
    lse = torch.logsumexp(z, 1)
    dead = torch.isneginf(lse)
    logp = torch.where(dead[:, None], -math.inf, z - torch.where(dead, 0.0, lse)[:, None])
    p = logp.exp()
    ent = torch.special.entr(p).sum(1)
    live = (t >= 0) & (t < vocab)
    chosen = logp.gather(1, t.long().clamp(0, vocab - 1)[:, None])[:, 0]
    return z, lse, logp, p, ent, live, torch.where(live, chosen, 0.0), dead


def rel_p(z):
    """How far p may be off, relatively: the argument of the exponential is a difference of fp32 numbers of size up to
    zmax log2 e (each rounded), 2^x is good to 2^-22, and a thread adds vocab / 256 terms before a tree of 8 + 8."""
    size = torch.where(torch.isfinite(z), z.abs(), 0.0).amax().item()
    return 2.0 ** -21 + 2.0 ** -24 * (8 * size + z.shape[1] / 256 + 32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("mask,pad", [(0.0, 0), (0.4, 5)])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_forward_matches_64_bits(rows, vocab, mask, pad, dtype):
    for scale, itype in ((1.0, torch.int64), (0.7, torch.int32)):
        z, t = make(rows, vocab, dtype, 1, mask, pad, itype)
        top = min(vocab, 20)
        got = B.token_logprobs(z, t, scale=scale, top=top)
        zz, lse, logp, p, ent, live, chosen, dead = exact(z, t, scale)
        tol = rel_p(zz)
        size = 1 + torch.where(dead, 0.0, lse).abs()

        def near(a, b, bound):
            assert torch.equal(torch.isinf(a.double()), torch.isinf(b))
            d = (a.double() - b).abs()
            assert bool((torch.where(torch.isinf(b), 0.0, d) <= bound).all()), float(torch.where(torch.isinf(b), 0.0, d).max())
        near(got.lse, lse, tol * size)
        near(got.logprob, chosen, tol * (size + torch.where(torch.isinf(chosen), 0.0, chosen).abs()))
        near(got.entropy, ent, 2 * tol * (2 + math.log(vocab)))
        assert bool((got.logprob[~live] == 0).all())
        # the order of the alternatives is that of the fp32 values, equal ones by rising index
        val, idx = torch.sort((z.float() * scale), dim=1, descending=True, stable=True)
        assert torch.equal(got.top_index.long(), idx[:, :top])
        near(got.top_logprob, logp.gather(1, idx[:, :top]), tol * (size[:, None] + logp.gather(1, idx[:, :top]).abs().nan_to_num(posinf=0.0)))
        plain = B.token_logprobs(z, t, scale=scale)
        assert plain.top_index is None and torch.equal(plain.lse, got.lse) and torch.equal(plain.entropy, got.entropy)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["equal", "falling", "rising", "masked", "two values", "lowest"])
def test_alternatives_when_many_words_tie_or_lie_in_order(kind, dtype):
    # more candidates than the collecting buffer holds, ties everywhere, order against the threads' stride
    for vocab in (40, 5000, 70000):
        i = torch.arange(vocab, device="cuda", dtype=torch.float32)
        row = {"equal": torch.full_like(i, 1.5), "falling": -i / vocab * 8, "rising": i / vocab * 8, "masked": torch.full_like(i, -math.inf),
               "two values": (i % 3 == 1).float(), "lowest": torch.full_like(i, torch.finfo(dtype).min)}[kind]
        z = row.to(dtype).repeat(3, 1)
        z[1] = z[1].flip(0)
        t = torch.zeros(3, dtype=torch.int64, device="cuda")
        got = B.token_logprobs(z, t, top=32)
        val, idx = torch.sort(z.float(), dim=1, descending=True, stable=True)
        assert torch.equal(got.top_index.long(), idx[:, :32])


@pytest.mark.parametrize("dtype", DTYPES)
def test_alternatives_that_one_thread_holds(dtype):
    # the best words all lie where one thread looks: every thread's bound is low, most words pass it
    vocab = 64000
    z = -torch.rand(2, vocab, device="cuda") - 1
    step = 256 * (16 // z.to(dtype).element_size())
    z[:, ::step] = torch.arange(vocab // step + (vocab % step > 0), device="cuda", dtype=torch.float32)
    z = z.to(dtype)
    t = torch.ones(2, dtype=torch.int64, device="cuda")
    got = B.token_logprobs(z, t, top=32)
    assert torch.equal(got.top_index.long(), torch.sort(z.float(), dim=1, descending=True, stable=True)[1][:, :32])


def test_nan_inf_and_large_values():
    z = torch.randn(5, 3000, device="cuda")
    z[0, 17] = float("nan")
    z[1, 2999] = float("inf")
    z[2, :] = 3e38
    z[3, :] = -3e38
    z[4, 0] = 1e4
    t = torch.zeros(5, dtype=torch.int64, device="cuda")
    got = B.token_logprobs(z, t, top=3)
    assert bool(got.lse[:2].isnan().all()) and bool(got.entropy[:2].isnan().all()) and bool(got.logprob[:2].isnan().all())
    assert got.top_index[1, 0] == 2999
    # all equal: entropy log V whatever the size of the values
    assert torch.allclose(got.entropy[3].double(), torch.tensor(math.log(3000.0), dtype=torch.float64, device="cuda"), rtol=1e-5)
    assert got.logprob[4] == 0 and got.entropy[4] == 0
    assert got.top_index[0, 0] == z[0].nan_to_num(nan=-math.inf).argmax()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("mask,pad", [(0.0, 0), (0.4, 5)])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_gradient_matches_64_bits(rows, vocab, mask, pad, dtype):
    for scale, with_entropy in ((1.0, True), (1.3, False)):
        z, t = make(rows, vocab, dtype, 2, mask, pad)
        g = torch.randn(rows, device="cuda")
        h = torch.randn(rows, device="cuda") if with_entropy else None
        f = B.token_logprobs(z, t, scale=scale)
        got = B.token_logprobs_grad(z, t, f.lse, f.entropy, g, h, scale=scale)
        zz, lse, logp, p, ent, live, chosen, dead = exact(z, t, scale)
        gl = torch.where(live, g.double(), 0.0)[:, None]
        hh = h.double()[:, None] if with_entropy else torch.zeros(rows, 1, dtype=torch.float64, device="cuda")
        logp0 = torch.where(p > 0, logp, 0.0)
        hot = torch.zeros_like(zz).scatter_(1, t.clamp(0, vocab - 1)[:, None], (live & ~dead).double()[:, None])
        want = scale * (gl * (hot - p) - hh * p * (logp0 + ent[:, None]))
        tol = 2 * rel_p(zz)
        size = scale * (gl.abs() * (hot + p) + hh.abs() * p * (logp0.abs() + ent[:, None] + 1) * 2)
        # an fp32 exponent's worth of absolute room: p below the normal range is 0
        bound = tol * (size + scale * p * (gl.abs() + hh.abs()) * (lse.nan_to_num(neginf=0.0).abs() + 1)[:, None]) + 1e-37
        assert between(got, want, bound)
        assert bool((got[dead] == 0).all())
        assert bool((got[torch.isinf(z) & ~dead[:, None] & (hot == 0)] == 0).all())
        # in place, in a strided buffer
        same = z.clone() if pad == 0 else z
        B.token_logprobs_grad(same, t, f.lse, f.entropy, g, h, scale=scale, out=same)
        assert torch.equal(same, got)


def test_gradient_against_differences():
    # L = sum g logp + h H in 64 bits, central differences of 1e-4: error of order 1e-8 |L'''| and 1e-16 / 1e-4
    rows, vocab, scale = 3, 50, 0.8
    z, t = make(rows, vocab, torch.float32, 3)
    g, h = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    f = B.token_logprobs(z, t, scale=scale)
    got = B.token_logprobs_grad(z, t, f.lse, f.entropy, g, h, scale=scale).double()

    def loss(x):
        logp = torch.log_softmax(x * scale, 1)
        return (g.double() * logp.gather(1, t[:, None])[:, 0] - h.double() * (logp.exp() * logp).sum(1))
    eps = 1e-4
    for j in range(vocab):
        d = torch.zeros(rows, vocab, dtype=torch.float64, device="cuda")
        d[:, j] = eps
        diff = (loss(z.double() + d) - loss(z.double() - d)) / (2 * eps)
        assert bool(((diff - got[:, j]).abs() <= 1e-5 * (1 + g.abs() + 10 * h.abs())).all())


def test_on_another_stream_and_long_offsets():
    side = torch.cuda.Stream()
    # rows 2^28 elements apart: the last row's offset passes 2^31
    base = torch.zeros(9 * 2 ** 28 + 64, dtype=torch.bfloat16, device="cuda")
    z = base[: 9 * 2 ** 28].view(9, 2 ** 28)[:, :64]
    z.copy_(torch.randn(9, 64, device="cuda"))
    t = torch.arange(9, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    a = B.token_logprobs(z, t, top=4, stream=side)
    d = B.token_logprobs_grad(z, t, a.lse, a.entropy, a.lse, None, stream=side)
    side.synchronize()
    b = B.token_logprobs(z.contiguous(), t, top=4)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert torch.equal(d, B.token_logprobs_grad(z.contiguous(), t, a.lse, a.entropy, a.lse, None))


def test_refusals():
    z = torch.zeros(4, 30, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    f = B.token_logprobs(z, t)
    for kw in (dict(scale=0.0), dict(scale=float("inf")), dict(top=33), dict(top=31), dict(top=-1)):
        with pytest.raises(B.ApolloError) as e:
            B.token_logprobs(z, t, **kw)
        assert e.value.code == B.ERR_INVALID_ARG, kw
    for bad in ((z.half(), t), (z.t(), t), (z, t[:3]), (z, t.float()), (z.cpu(), t), (z[0], t)):
        with pytest.raises(ValueError):
            B.token_logprobs(*bad)
    with pytest.raises(ValueError):
        B.token_logprobs_grad(z, t, f.lse[:2], f.entropy, f.lse)
    with pytest.raises(ValueError):
        B.token_logprobs_grad(z, t, f.lse, f.entropy, f.lse, out=torch.zeros(4, 29, device="cuda"))
    with pytest.raises(B.ApolloError) as e:
        B.token_logprobs_grad(z, t, f.lse, None, f.lse, f.lse)           # an entropy term without the entropy
    assert e.value.code == B.ERR_INVALID_ARG
    assert B.token_logprobs(z[:0], t[:0]).lse.shape == (0,)
