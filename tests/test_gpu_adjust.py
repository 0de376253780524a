"""Adjusted logits and their gradient against the definition in 64 bits, on the CPU."""
import math

import pytest
import torch

from paper_2412_05270_b200 import binding as B
from rounding import between

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = [torch.float32, torch.bfloat16]
NAMES = ("history", "lengths", "start", "repetition", "frequency", "presence", "bias", "bias_index", "bias_value", "mask")


def make(n, vocab, dtype, g, length=0, share=1, itype=torch.int32, bias=None, words=0, allowed=None, one_mask=False, scalars=False):
    """Logits and rules on the CPU."""
    r = {}
    z = (torch.randn(n, vocab, generator=g) * 3).to(dtype)
    if length:
        r["history"] = torch.randint(-2, vocab + 2, (n // share, length), generator=g).to(itype)
        r["lengths"] = torch.randint(-1, length + 3, (n,), generator=g, dtype=torch.int32)
        r["start"] = torch.randint(-1, length + 1, (n,), generator=g, dtype=torch.int32)
        if scalars:
            r |= {"repetition": 1.25, "frequency": 0.5, "presence": -0.25}
        else:
            r |= {"repetition": torch.rand(n, generator=g) + 0.5, "frequency": torch.randn(n, generator=g), "presence": torch.randn(n, generator=g)}
    if bias:
        r["bias"] = torch.randn(*((vocab,) if bias == "shared" else (n, vocab)), generator=g).to(dtype)
    if words:
        r["bias_index"] = torch.randint(-1, vocab + 1, (n, words), generator=g).to(itype)
        r["bias_index"][:, words // 2] = r["bias_index"][:, 0]
        r["bias_index"][:, -1] = r["bias_index"][:, 0]
        r["bias_value"] = torch.randn(n, words, generator=g) * 2
    if allowed is not None:
        rows = 1 if one_mask else n
        bits = torch.rand(rows, (vocab + 31) // 32, 32, generator=g) < allowed
        if not one_mask and n > 2:
            bits[n // 2] = False
        r["mask"] = (bits.long() << torch.arange(32)).sum(-1).to(torch.int32)
    return z, r


def rules_in_64(n, vocab, r):
    """(seen, count from start, repetition, frequency, presence, allowed) with a row each."""
    column = lambda x: x.double()[:, None] if isinstance(x, torch.Tensor) else torch.full((n, 1), float(torch.tensor(x)), dtype=torch.float64)
    seen, count = torch.zeros(n, vocab, dtype=torch.bool), torch.zeros(n, vocab, dtype=torch.float64)
    h = r.get("history")
    if h is not None:
        for i in range(n):
            row = h[i // (n // h.shape[0])].long()
            length = row.numel() if r.get("lengths") is None else max(0, min(int(r["lengths"][i]), row.numel()))
            start = 0 if r.get("start") is None else max(0, int(r["start"][i]))
            seen[i, [w for w in row[:length].tolist() if 0 <= w < vocab]] = True
            for w in row[start:length].tolist():
                if 0 <= w < vocab:
                    count[i, w] += 1
    allowed = torch.ones(n, vocab, dtype=torch.bool)
    if r.get("mask") is not None:
        j = torch.arange(vocab)
        allowed = ((r["mask"].view(-1, (vocab + 31) // 32)[:, j // 32] >> (j % 32)) & 1).bool().expand(n, vocab)
    return seen, count, column(r.get("repetition", 1.0)), column(r.get("frequency", 0.0)), column(r.get("presence", 0.0)), allowed


def plain(z, r):
    """(adjusted logits, how far fp32 may be from them)."""
    n, vocab = z.shape
    seen, count, rho, phi, pi, allowed = rules_in_64(n, vocab, r)
    x = z.double()
    x = torch.where(seen, torch.where(x > 0, x / rho, x * rho), x)
    penalty = torch.where(count > 0, phi * count + pi, 0.0)
    size = x.abs() + torch.where(count > 0, (phi * count).abs() + pi.abs(), 0.0)
    x = x - penalty
    if r.get("bias") is not None:
        x = x + r["bias"].double()
        size = size + r["bias"].double().abs()
    k = 0
    if r.get("bias_index") is not None:
        k = r["bias_index"].shape[1]
        for i in range(n):
            for w, v in zip(r["bias_index"][i].tolist(), r["bias_value"][i].double().tolist()):
                if 0 <= w < vocab:
                    x[i, w] += v
                    size[i, w] += abs(v)
    # division, penalty, difference, bias, sum of the named values: half a step of the largest of them each
    return torch.where(allowed, x, -math.inf), (5 + k) * U * size


def cuda(r):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in r.items()}


def check(got, want, bound):
    got = got.cpu()
    masked = want == -math.inf
    assert torch.equal(got == -math.inf, masked)
    assert between(got[~masked], want[~masked], bound[~masked])


SHAPES = [(1, 1), (3, 7), (5, 33), (2, 2047), (4, 2049), (2, 8200), (1, 20001), (64, 1000), (300, 160)]
RULES = {
    "nothing": dict(),
    "history": dict(length=40),
    "history of 64 bits": dict(length=300, itype=torch.int64, scalars=True),
    "one token": dict(length=1),
    "mask": dict(allowed=0.5),
    "one mask": dict(allowed=0.97, one_mask=True),
    "bias": dict(bias="shared"),
    "bias for each row": dict(bias="row", allowed=0.9),
    "words": dict(words=5),
    "words of 64 bits": dict(words=300, itype=torch.int64),
    "everything": dict(length=129, bias="shared", words=9, allowed=0.6),
    "everything by row": dict(length=50, bias="row", words=40, allowed=0.02),
}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rules", list(RULES))
@pytest.mark.parametrize("shape", SHAPES)
def test_adjusted_logits(shape, rules, dtype):
    g = torch.Generator().manual_seed(1)
    z, r = make(*shape, dtype, g, **RULES[rules])
    want, bound = plain(z, r)
    zc, rc = z.cuda(), cuda(r)
    got = B.adjust_logits(zc, **rc)
    check(got, want, bound)
    assert torch.equal(zc.cpu(), z)
    assert B.adjust_logits(zc, **rc, out=zc) is zc and torch.equal(zc, got)              # in place
    wide = torch.full((shape[0], shape[1] + 9), 5.0, dtype=dtype, device="cuda")         # rows cut out of a wider buffer
    view = wide[:, 3: 3 + shape[1]]
    view.copy_(z)
    assert torch.equal(B.adjust_logits(view, **rc), got)
    B.adjust_logits(view, **rc, out=view)
    assert torch.equal(view, got) and bool((wide[:, :3] == 5).all()) and bool((wide[:, 3 + shape[1]:] == 5).all())


@pytest.mark.parametrize("share", [2, 3, 12])
def test_rows_that_share_a_history(share):
    g = torch.Generator().manual_seed(2)
    z, r = make(12, 100, torch.float32, g, length=30, share=share)
    check(B.adjust_logits(z.cuda(), **cuda(r)), *plain(z, r))
    one = r["history"][:1].expand(12, 30)                      # stride 0
    got = B.adjust_logits(z.cuda(), **(cuda(r) | {"history": one.cuda().expand(12, 30)}))
    check(got, *plain(z, r | {"history": one}))
    column = torch.randint(0, 100, (30, 12), generator=g).t()  # stride 12 between tokens
    check(B.adjust_logits(z.cuda(), **(cuda(r) | {"history": column.cuda()})), *plain(z, r | {"history": column}))


def test_long_histories_and_all_of_one_word():
    g = torch.Generator().manual_seed(3)
    z, r = make(2, 5000, torch.float32, g, length=70001)
    r["lengths"] = torch.tensor([70001, 65537], dtype=torch.int32)
    r["start"] = torch.tensor([0, 30000], dtype=torch.int32)
    r["history"][1] = 4999
    check(B.adjust_logits(z.cuda(), **cuda(r)), *plain(z, r))


def test_the_ends_of_the_type():
    """Masks of the type's lowest value, infinities and NaN: where words are masked, and where they are not."""
    for dtype in DTYPES:
        low = torch.finfo(dtype).min
        z = torch.tensor([[low, 1.0, math.nan, math.inf, -math.inf, 0.0, -0.0, 2.0]], dtype=dtype, device="cuda")
        history = torch.arange(8, dtype=torch.int32, device="cuda")[None]
        y = B.adjust_logits(z, history=history, repetition=2.0)
        assert y[0, 0] == -math.inf and y[0, 1] == 0.5 and bool(y[0, 2].isnan()) and y[0, 3] == math.inf and y[0, 4] == -math.inf and y[0, 5] == 0 and y[0, 7] == 1
        mask = torch.tensor([[0b11100010]], dtype=torch.int32, device="cuda")
        y = B.adjust_logits(z, history=history, repetition=2.0, mask=mask)
        assert y[0].tolist() == [-math.inf, 0.5, -math.inf, -math.inf, -math.inf, 0.0, 0.0, 1.0]
        y = B.adjust_logits(z, mask=torch.zeros(1, 1, dtype=torch.int32, device="cuda"), out=z)
        assert bool((y == -math.inf).all())
        r = B.token_logprobs(z, torch.zeros(1, dtype=torch.int64, device="cuda"), top=3)
        assert r.lse.item() == -math.inf and r.logprob.item() == -math.inf and r.top_index.tolist() == [[0, 1, 2]]


def test_no_rows_and_no_tokens():
    z = torch.zeros(0, 50, device="cuda")
    assert B.adjust_logits(z, history=torch.zeros(0, 9, dtype=torch.int32, device="cuda"), mask=torch.zeros(0, 2, dtype=torch.int32, device="cuda")).shape == (0, 50)
    d = B.adjust_logits_grad(z, z, bias="shared")
    assert d.logits.shape == (0, 50) and d.bias.tolist() == [0.0] * 50
    z = torch.randn(3, 50, device="cuda")
    assert torch.equal(B.adjust_logits(z, history=torch.zeros(3, 0, dtype=torch.int64, device="cuda"), repetition=2.0), z)
    none = torch.zeros(3, 0, dtype=torch.int32, device="cuda")
    assert torch.equal(B.adjust_logits(z, bias_index=none, bias_value=none.float()), z)
    assert B.adjust_logits_grad(z, z, bias_index=none).value.shape == (3, 0)


# ---------------------------------------------------------------- gradient
def plain_grad(z, dy, r):
    """The gradients in 64 bits: logits', of a bias for each row, of the named values."""
    n, vocab = z.shape
    seen, _, rho, _, _, allowed = rules_in_64(n, vocab, r)
    a = torch.where(allowed, dy.double(), 0.0)
    dz = torch.where(seen, torch.where(z > 0, a / rho, a * rho), a)
    value = None
    if r.get("bias_index") is not None:
        i = r["bias_index"].long()
        value = torch.where((i >= 0) & (i < vocab), a.gather(1, i.clamp(0, vocab - 1)), 0.0)
    return dz, a, value


def check_grad(got, z, dy, r, bias):
    n = z.shape[0]
    dz, a, value = plain_grad(z, dy, r)
    assert between(got.logits.cpu(), dz, U * dz.abs())
    if bias == "row":
        assert torch.equal(got.bias.cpu().double(), a)
    elif bias == "shared":
        assert between(got.bias.cpu(), a.sum(0), n * U * a.abs().sum(0))     # n sums of fp32
    else:
        assert got.bias is None
    assert (got.value is None) == (value is None) and (value is None or torch.equal(got.value.cpu().double(), value))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bias", ["none", "shared", "row"])
@pytest.mark.parametrize("rules", ["nothing", "history", "history of 64 bits", "mask", "one mask", "words", "everything"])
@pytest.mark.parametrize("shape", SHAPES + [(700, 45)])
def test_gradients(shape, rules, bias, dtype):
    g = torch.Generator().manual_seed(4)
    z, r = make(*shape, dtype, g, **RULES[rules])
    dy = torch.randn(*shape, generator=g).to(dtype)
    given = {k: v for k, v in cuda(r).items() if k in ("history", "lengths", "repetition", "mask", "bias_index")}
    zc, dc = z.cuda(), dy.cuda()
    got = B.adjust_logits_grad(zc, dc, bias=bias, **given)
    check_grad(got, z, dy, r, bias)
    assert torch.equal(dc.cpu(), dy)
    again = B.adjust_logits_grad(zc, dc, bias=bias, out=dc, **given)                     # in place
    assert again.logits is dc
    for a, b in zip(got, again):
        assert (a is None and b is None) or torch.equal(a, b)
    wide = torch.full((shape[0], shape[1] + 5), 3.0, dtype=dtype, device="cuda")
    view = wide[:, 1: 1 + shape[1]]
    view.copy_(dy)
    again = B.adjust_logits_grad(zc, view, bias=bias, out=view, **given)
    for a, b in zip(got, again):
        assert (a is None and b is None) or torch.equal(a, b)
    assert bool((wide[:, 0] == 3).all()) and bool((wide[:, 1 + shape[1]:] == 3).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_the_gradient_is_that_of_differences(dtype):
    """With powers of two everywhere a difference quotient of the operator itself is exact, unless its two ends are on either side of zero."""
    g = torch.Generator().manual_seed(5)
    n, vocab = 4, 70
    z = torch.randint(1, 8, (n, vocab), generator=g).to(dtype) * torch.where(torch.rand(n, vocab, generator=g) < 0.5, -1, 1).to(dtype)
    _, r = make(n, vocab, dtype, g, length=40, allowed=0.7, scalars=True)
    r |= {"repetition": 2.0, "frequency": 0.0, "presence": 0.0}
    rc = cuda(r)
    up, down = (B.adjust_logits(z.cuda() + s, **rc).double() for s in (0.5, -0.5))
    quotient = torch.where(up == -math.inf, 0.0, up - down)
    dy = torch.ones(n, vocab, dtype=dtype, device="cuda")
    given = {k: rc[k] for k in ("history", "lengths", "repetition", "mask")}
    assert torch.equal(B.adjust_logits_grad(z.cuda(), dy, **given).logits.double(), quotient)


def test_equal_bits_in_every_run():
    g = torch.Generator().manual_seed(6)
    z, r = make(1000, 3001, torch.float32, g, length=64, words=64, bias="shared", allowed=0.8)
    r["bias_index"][:, ::2] = 7
    rc = cuda(r)
    dy = torch.randn(1000, 3001, generator=g).cuda()
    first = B.adjust_logits(z.cuda(), **rc)
    given = {k: rc[k] for k in ("history", "lengths", "repetition", "mask", "bias_index")}
    grads = B.adjust_logits_grad(z.cuda(), dy, bias="shared", **given)
    for _ in range(5):
        assert torch.equal(first, B.adjust_logits(z.cuda(), **rc))
        assert all(torch.equal(a, b) for a, b in zip(grads, B.adjust_logits_grad(z.cuda(), dy, bias="shared", **given)))


def test_captured_and_on_another_stream():
    g = torch.Generator().manual_seed(7)
    z, r = make(16, 4000, torch.bfloat16, g, length=100, words=8, bias="shared", allowed=0.8)
    zc, rc, dy = z.cuda(), cuda(r), torch.randn(16, 4000, generator=g).bfloat16().cuda()
    given = {k: rc[k] for k in ("history", "lengths", "repetition", "mask", "bias_index")}
    want, d_want = B.adjust_logits(zc, **rc), B.adjust_logits_grad(zc, dy, bias="shared", **given)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got, d_got = B.adjust_logits(zc, **rc, stream=s), B.adjust_logits_grad(zc, dy, bias="shared", **given, stream=s)
    s.synchronize()
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(d_got, d_want))
    held = torch.zeros_like(zc)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.adjust_logits(held, **rc)
        d_got = B.adjust_logits_grad(held, dy, bias="shared", **given)
    held.copy_(zc)
    graph.replay()
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(d_got, d_want))


# ---------------------------------------------------------------- refusals
def test_calls_that_are_refused():
    z = torch.zeros(4, 100, device="cuda")
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")
    for kw in (dict(history=i32(3, 5)), dict(history=i32(5)), dict(history=i32(4, 5).float()), dict(history=i32(4, 5), lengths=i32(3)),
               dict(history=i32(4, 5), lengths=i32(4).long()), dict(history=i32(4, 5), repetition=torch.ones(3, device="cuda")),
               dict(history=i32(4, 5).cpu()), dict(bias=torch.zeros(99, device="cuda")), dict(bias=torch.zeros(100, device="cuda").bfloat16()),
               dict(bias_index=i32(4, 2)), dict(bias_value=torch.zeros(4, 2, device="cuda")), dict(bias_index=i32(3, 2), bias_value=torch.zeros(3, 2, device="cuda")),
               dict(bias_index=i32(4, 2), bias_value=torch.zeros(4, 3, device="cuda")), dict(mask=i32(4, 3)), dict(mask=i32(2, 4)), dict(mask=i32(4, 4).long()),
               dict(out=torch.zeros(4, 99, device="cuda")), dict(out=torch.zeros(4, 100))):
        with pytest.raises(ValueError):
            B.adjust_logits(z, **kw)
    for kw, code in ((dict(history=i32(4, 5), repetition=0.0), B.ERR_INVALID_ARG), (dict(history=i32(4, 5), repetition=math.inf), B.ERR_INVALID_ARG),
                     (dict(history=i32(4, 5), frequency=math.nan), B.ERR_INVALID_ARG), (dict(history=i32(1, 1 << 20)), B.ERR_SHAPE),
                     (dict(bias_index=i32(4, 1025), bias_value=torch.zeros(4, 1025, device="cuda")), B.ERR_SHAPE)):
        with pytest.raises(B.ApolloError) as e:
            B.adjust_logits(z, **kw)
        assert e.value.code == code
    with pytest.raises(ValueError):
        B.adjust_logits(z.t())
    with pytest.raises(ValueError):
        B.adjust_logits(z.half())
    with pytest.raises(ValueError):
        B.adjust_logits_grad(z, z, bias="all")
    with pytest.raises(ValueError):
        B.adjust_logits_grad(z, z[:3])
    with pytest.raises(B.ApolloError) as e:
        B.adjust_logits_grad(z, z.clone(), bias="shared", workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == B.ERR_WORKSPACE
    assert not z.any()


def test_values_of_a_gradient_that_the_call_before_has_left():
    """In place, words alone: nothing of the call may start before the masks of the call before it are written."""
    g = torch.Generator(device="cuda").manual_seed(11)
    start = torch.randn(4096, 32000, generator=g, device="cuda").bfloat16()
    mask = torch.randint(-2 ** 31, 2 ** 31, (4096, 1000), generator=g, device="cuda").to(torch.int32)
    index = torch.randint(0, 32000, (4096, 8), generator=g, device="cuda")
    allowed = mask.gather(1, index // 32) >> (index % 32) & 1
    want = torch.where(allowed == 1, start.gather(1, index).float(), -math.inf)
    for _ in range(3):
        d = start.clone()
        B.adjust_logits(d, mask=mask, out=d)
        r = B.adjust_logits_grad(d, d, bias_index=index, out=d)
        assert torch.equal(r.value, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(129, 20011), (300, 16391), (1111, 515)])
def test_a_shared_bias_of_odd_rows_in_several_chunks(shape, dtype):
    g = torch.Generator().manual_seed(13)
    z, r = make(*shape, dtype, g, allowed=0.7)
    dy = torch.randn(*shape, generator=g).to(dtype)
    a = torch.where(rules_in_64(*shape, r)[-1], dy.double(), 0.0)
    got = B.adjust_logits_grad(z.cuda(), dy.cuda(), bias="shared", mask=r["mask"].cuda())
    assert torch.equal(got.logits.cpu().double(), a)
    # a sum of n values in fp32, rounded once more to the type: n - 1 half steps of the partial sums' sizes, half a step of the result
    want, half = a.sum(0), torch.finfo(dtype).eps / 2
    assert bool(((got.bias.cpu().double() - want).abs() <= shape[0] * U * a.abs().sum(0) + half * want.abs() * (1 + half)).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_in_place_with_a_bias_in_several_chunks(dtype):
    g = torch.Generator().manual_seed(14)
    z, r = make(3, 40_005, dtype, g, length=6000, bias="shared", words=63, allowed=0.8)
    want, bound = plain(z, r)
    zc, rc = z.cuda(), cuda(r)
    got = B.adjust_logits(zc, **rc)
    check(got, want, bound)
    B.adjust_logits(zc, **rc, out=zc)
    assert torch.equal(zc, got)
