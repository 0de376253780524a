"""Embedding lookup and its gradient by sorted tokens, through the C ABI, against 64-bit sums."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B
from rounding import between

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
# (tokens, rows, dim): one token, odd sizes, rows of fewer elements than a vector, windows that end inside a token's
# segment, more keys than one digit (256), than two (65536), dims above what one thread group covers
SIZES = [(1, 1, 1), (1, 5, 8), (31, 7, 3), (32, 3, 16), (33, 3, 17), (64, 300, 24), (257, 2, 129), (1000, 40, 64),
         (4097, 300, 40), (5000, 70001, 8), (3000, 1, 33), (300, 1000, 2056), (130, 9, 4100)]


def make(tokens, rows, dim, dtype, seed, itype=torch.int64, hot=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    index = torch.randint(0, rows, (tokens,), generator=g, device="cuda")
    if hot:                                   # most positions name one token: a segment over many windows
        index[torch.rand(tokens, generator=g, device="cuda") < 0.8] = rows // 2
    pad = torch.rand(tokens, generator=g, device="cuda")
    index[pad < 0.05] = -1
    index[pad > 0.97] = rows + 3
    x = torch.randn(tokens, dim, generator=g, device="cuda").to(dtype)
    table = torch.randn(rows, dim, generator=g, device="cuda").to(dtype)
    return index.to(itype), x, table


def lookup(table, index, scale):
    live = (index >= 0) & (index < table.shape[0])
    out = table.float()[index.long().clamp(0, table.shape[0] - 1)] * scale
    out[~live] = 0
    return out.to(table.dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("itype", [torch.int32, torch.int64])
@pytest.mark.parametrize("tokens,rows,dim", SIZES)
def test_lookup_is_exact(tokens, rows, dim, dtype, itype):
    index, _, table = make(tokens, rows, dim, dtype, 1, itype)
    for scale in (1.0, dim ** 0.5):
        # one product in fp32, one rounding: nothing else can come out
        assert torch.equal(B.embedding(table, index, scale), lookup(table, index, torch.tensor(scale, device="cuda")))


def test_lookup_into_a_wider_buffer_and_of_any_index_shape():
    index, _, table = make(60, 50, 24, torch.bfloat16, 2)
    wide = torch.full((60, 40), 7.0, dtype=torch.bfloat16, device="cuda")
    B.embedding(table, index, 2.0, out=wide[:, 3:27])
    assert torch.equal(wide[:, 3:27], lookup(table, index, 2.0))
    assert bool((wide[:, :3] == 7).all()) and bool((wide[:, 27:] == 7).all())
    assert torch.equal(B.embedding(table, index.view(4, 15)), lookup(table, index, 1.0).view(4, 15, 24))
    assert B.embedding(table, index[:0]).shape == (0, 24)


def grad_bound(index, x, rows, scale, before=None):
    """The 64-bit sums and what fp32 sums in any order and one product may differ by, before the result is rounded."""
    live = (index >= 0) & (index < rows)
    i, v = index[live].long(), x[live].double()
    total = torch.zeros(rows, x.shape[1], dtype=torch.float64, device="cuda").index_add_(0, i, v) * scale
    size = torch.zeros_like(total).index_add_(0, i, v.abs()) * abs(scale)
    count = torch.zeros(rows, dtype=torch.float64, device="cuda").index_add_(0, i, torch.ones_like(i, dtype=torch.float64))
    if before is not None:
        total = total + before.double()
        size = size + before.double().abs()
    return total, size * (count[:, None] + 2) * 2.0 ** -24


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hot", [False, True])
@pytest.mark.parametrize("tokens,rows,dim", SIZES)
def test_gradient_matches_64_bit_sums(tokens, rows, dim, hot, dtype):
    index, x, _ = make(tokens, rows, dim, dtype, 3, torch.int64 if hot else torch.int32, hot)
    out = torch.full((rows, dim), float("nan"), dtype=dtype, device="cuda")
    got = B.embedding_grad(x, index, rows, scale=1.5, out=out)
    assert got is out
    want, bound = grad_bound(index, x, rows, 1.5)
    assert between(got, want, bound)
    assert torch.equal(got, B.embedding_grad(x, index, rows, scale=1.5))          # the same bits again


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,rows,dim", [(1, 3, 8), (70, 4, 24), (1000, 50, 17), (4097, 300, 40)])
def test_gradient_accumulates(tokens, rows, dim, dtype):
    index, x, before = make(tokens, rows, dim, dtype, 4, hot=True)
    got = B.embedding_grad(x, index, rows, scale=0.5, out=before.clone(), accumulate=True)
    want, bound = grad_bound(index, x, rows, 0.5, before)
    assert between(got, want, bound)
    untouched = torch.ones(rows, dtype=torch.bool, device="cuda")
    untouched[index[(index >= 0) & (index < rows)]] = False
    assert torch.equal(got[untouched], before[untouched])


def test_gradient_of_a_slice_of_rows_and_of_unaligned_buffers():
    index, x, _ = make(200, 30, 48, torch.bfloat16, 5)
    wide = torch.randn(200, 60, device="cuda").to(torch.bfloat16)
    part = wide[:, 5:53]                                                    # stride 60, first element 10 bytes in
    want, bound = grad_bound(index, part, 30, 1.0)
    odd = torch.full((30 * 48 + 1,), 9.0, dtype=torch.bfloat16, device="cuda")[1:].view(30, 48)
    got = B.embedding_grad(part, index, 30, out=odd)
    assert between(got, want, bound)


def test_gradient_without_tokens_or_without_live_ones():
    x = torch.randn(40, 16, device="cuda")
    none = torch.full((40,), -1, device="cuda")
    assert not B.embedding_grad(x, none, 10).any()
    assert not B.embedding_grad(x[:0], none[:0], 10).any()
    keep = torch.randn(10, 16, device="cuda")
    assert torch.equal(B.embedding_grad(x, none, 10, out=keep.clone(), accumulate=True), keep)


def test_gradient_is_the_derivative_of_the_lookup():
    # the lookup is linear in the table: <c, lookup(table + d) - lookup(table)> = <gradient(c), d> up to rounding
    index, c, table = make(300, 20, 32, torch.float32, 6)
    d = torch.randn(20, 32, device="cuda") * 0.5
    lhs = (c.double() * (B.embedding(table + d, index, 3.0).double() - B.embedding(table, index, 3.0).double())).sum()
    grad = B.embedding_grad(c, index, 20, scale=3.0)
    rhs = (grad.double() * ((table + d).double() - table.double())).sum()
    size = (c.double().abs().sum(1).max() * 300 * 8 * 3).item()
    assert abs((lhs - rhs).item()) <= size * 2.0 ** -22


def test_on_another_stream():
    side = torch.cuda.Stream()
    index, x, table = make(3000, 500, 256, torch.bfloat16, 7)
    side.wait_stream(torch.cuda.current_stream())
    a = B.embedding(table, index, 2.0, stream=side)
    b = B.embedding_grad(x, index, 500, stream=side)
    side.synchronize()
    assert torch.equal(a, B.embedding(table, index, 2.0)) and torch.equal(b, B.embedding_grad(x, index, 500))


def test_refusals():
    table = torch.zeros(10, 8, device="cuda")
    index = torch.zeros(4, dtype=torch.int64, device="cuda")
    for bad in (dict(table=table.half()), dict(index=index.float()), dict(table=table.t()), dict(index=index.cpu()),
                dict(out=torch.zeros(4, 9, device="cuda")), dict(out=torch.zeros(4, 8, device="cuda").bfloat16())):
        with pytest.raises(ValueError):
            B.embedding(**{"table": table, "index": index, **bad})
    with pytest.raises(B.ApolloError) as e:
        B.embedding(table, index, scale=float("nan"))
    assert e.value.code == B.ERR_INVALID_ARG
    x = torch.zeros(4, 8, device="cuda")
    with pytest.raises(ValueError):
        B.embedding_grad(x, index[:3], 10)
    with pytest.raises(ValueError):
        B.embedding_grad(x, index, 10, accumulate=True)
    with pytest.raises(B.ApolloError) as e:
        B.embedding_grad(x, index, 10, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == B.ERR_WORKSPACE
    with pytest.raises(B.ApolloError) as e:
        B.embedding_grad_workspace_bytes(-1, 10, 8)
    assert e.value.code == B.ERR_SHAPE
