"""AdamW over a list of tensors with moments of 8 or 32 bits, and the global norm, against their definitions in 64 bits."""
import math

import pytest
import torch

import adamw8 as Q
from paper_2412_05270_b200 import binding as B
from rounding import between

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
B1, B2, EPS = 0.9, 0.999, 1e-8
SEED = 0x0123456789ABCDEF
SIZES = [1, 7, 8, 255, 0, 256, 257, 1000, 8191, 8192, 8193, 70001]
DTYPES = [torch.float32, torch.bfloat16]


def tensors(sizes, dtypes, std, g):
    return [(torch.randn(n, generator=g) * std).to(dtypes[i % len(dtypes)]).cuda() for i, n in enumerate(sizes)]


def gradients(sizes, dtypes, g):
    """Entries that differ by powers of two from block to block and within one, zeros and a whole block of them among them."""
    out = []
    for i, n in enumerate(sizes):
        x = torch.randn(n, generator=g) * 1e-3 * torch.exp2(torch.randint(-9, 9, (n,), generator=g).float())
        x[::11] = 0
        x[256:512] = 0
        out.append(x.to(dtypes[i % len(dtypes)]).cuda())
    return out


class Reference:
    """One step from the state as it is, in 64 bits, and how far fp32 may be from it."""

    def __init__(self, opt, params, grads, lr, t, wd, factor=1.0, bits=8):
        self.numels = [p.numel() for p in params]
        first = Q.blocks_of(self.numels)
        n = first[-1]
        if bits == 8:
            m, v, *_ = Q.read(opt.state, n)
        else:
            m, v = opt.state.cpu().view(torch.float32).double().view(2, n, Q.BLOCK)
        g, p = Q.padded(grads, self.numels) * factor, Q.padded(params, self.numels)
        self.m, self.v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
        # m: constants, the factor's product, a product and a fused sum, a half step each; v: two products more, nothing cancels
        # (and what fp32 cannot hold below its normal range)
        self.dm = 5 * U * (B1 * m.abs() + (1 - B1) * g.abs()) + 2.0 ** -148
        self.dv = 7 * U * self.v + 2.0 ** -148
        c1, c2 = 1 - B1 ** (t + 1), 1 - B2 ** (t + 1)
        den = (self.v / c2).sqrt() + EPS
        update = self.m / c1 / den
        # the root halves v's error and is right to 2 steps; quotient, sum, corrections: 8 steps in all; v near nothing: an absolute error
        # of the root, which EPS covers
        d_den = 0.5 * self.dv / c2 / den.clamp(min=EPS) + 4 * U * den
        self.dp = lr * (self.dm / c1 / den + update.abs() * (d_den / den + 8 * U) + 4 * U * (wd * p).abs()) + 2 * U * p.abs()
        self.p = p - lr * (update + wd * p)
        self.first = first

    def check(self, opt, params, bits, t):
        n = self.first[-1]
        for x, k, size in zip(params, self.first, self.numels):
            at = slice(k * Q.BLOCK, k * Q.BLOCK + size)
            assert between(x.cpu().view(-1), self.p.view(-1)[at], self.dp.view(-1)[at])
        if bits == 32:
            m, v = opt.state.cpu().view(torch.float32).double().view(2, n, Q.BLOCK)
            assert bool(((m - self.m).abs() <= self.dm).all()) and bool(((v - self.v).abs() <= self.dv).all())
            return
        m, v, cm, cv, k = Q.read(opt.state, n)
        chance = Q.chances(n, SEED, t)
        for x, dx, c, e, binades in ((self.m.abs(), self.dm, cm, k[:, 0], 16), (self.v, self.dv, cv, k[:, 1], 32)):
            # rounding is monotone in the value and in the block's largest one
            tops = [(x + s * dx).clamp(min=0).amax(1) for s in (-1, 1)]
            assert bool((e >= Q.exponent(tops[0], binades)).all()) and bool((e <= Q.exponent(tops[1], binades)).all())
            lo, hi = (Q.code((x + s * dx).clamp(min=0), e, chance, binades) for s in (-1, 1))
            assert bool(((c >= lo) & (c <= hi)).all())
        assert bool((m * self.m >= -self.dm).all())                        # signs


@pytest.mark.parametrize("pdt", [DTYPES[:1], DTYPES[1:], DTYPES])
@pytest.mark.parametrize("gdt", [DTYPES[:1], DTYPES[1:], DTYPES[::-1]])
@pytest.mark.parametrize("bits", [8, 32])
def test_steps_match_the_definition(bits, gdt, pdt):
    g = torch.Generator().manual_seed(5)
    sizes = SIZES + [33 + 17 * i for i in range(60)] if len(pdt) == 1 else SIZES
    params = tensors(sizes, pdt, 0.02, g)
    opt = B.AdamW(params, bits=bits, beta1=B1, beta2=B2, eps=EPS, seed=SEED)
    for t in (0, 1, 2, 5_000_000_000):
        grads = gradients(sizes, gdt, g)
        ref = Reference(opt, params, grads, 3e-3, t, 0.1, bits=bits)
        opt.step(grads, lr=3e-3, t=t, wd=0.1)
        ref.check(opt, params, bits, t)
        if bits == 8:
            n = ref.first[-1]
            m, v, *_ = Q.read(opt.state, n)
            mm, vv = opt.moments()
            assert torch.equal(mm.cpu().double().view(n, -1), m) and torch.equal(vv.cpu().double().view(n, -1), v)


def test_thousands_of_tensors_take_several_launches():
    g = torch.Generator().manual_seed(6)
    sizes = [1 + i % 300 for i in range(2500)]
    params = tensors(sizes, DTYPES, 0.02, g)
    opt = B.AdamW(params, bits=8, beta1=B1, beta2=B2, eps=EPS, seed=SEED)
    grads = gradients(sizes, DTYPES, g)
    ref = Reference(opt, params, grads, 1e-2, 0, 0.0)
    opt.step(grads, lr=1e-2, t=0)
    ref.check(opt, params, 8, 0)
    want = math.sqrt(sum(float(x.double().square().sum()) for x in grads))
    assert abs(B.grad_norm(grads)[0].item() - want) <= 18 * U * want


@pytest.mark.parametrize("bits", [8, 32])
def test_a_parameter_without_a_gradient_stays(bits):
    g = torch.Generator().manual_seed(7)
    params = tensors([300, 500, 700], DTYPES, 0.02, g)
    opt = B.AdamW(params, bits=bits, seed=SEED)
    grads = gradients([300, 500, 700], DTYPES, g)
    opt.step(grads, lr=1e-2, t=0)
    before, was = [p.clone() for p in params], [x.clone().view(-1, 256) for x in opt.moments()]
    opt.step([grads[0], None, grads[2]], lr=1e-2, t=1, wd=0.1)
    assert torch.equal(params[1], before[1]) and not torch.equal(params[0], before[0]) and not torch.equal(params[2], before[2])
    for x, w in zip(opt.moments(), was):
        x = x.view(-1, 256)
        assert torch.equal(x[2:4], w[2:4]) and not torch.equal(x[:2], w[:2]) and not torch.equal(x[4:], w[4:])
    opt.step([None, None, None], lr=1e-2, t=2)


def test_equal_bits_on_any_stream_and_after_a_checkpoint():
    g = torch.Generator().manual_seed(8)
    start = tensors(SIZES, DTYPES, 0.02, g)
    grads = [gradients(SIZES, DTYPES, g) for _ in range(4)]
    ends = []
    for how in ("plain", "again", "stream", "resumed"):
        params = [p.clone() for p in start]
        opt = B.AdamW(params, seed=SEED)
        stream = torch.cuda.Stream() if how == "stream" else None
        torch.cuda.synchronize()
        for t in range(4):
            if how == "resumed" and t == 2:
                opt = B.AdamW(params, seed=SEED, state=opt.state.clone())
            opt.step(grads[t], lr=1e-2, t=t, wd=0.1, stream=stream)
        torch.cuda.synchronize()
        ends.append(params + [opt.state])
    for other in ends[1:]:
        assert all(torch.equal(a, b) for a, b in zip(ends[0], other))
    # another seed rounds otherwise
    params = [p.clone() for p in start]
    opt = B.AdamW(params, seed=SEED + 1)
    opt.step(grads[0], lr=1e-2, t=0)
    first = B.AdamW([p.clone() for p in start], seed=SEED)
    first.step(grads[0], lr=1e-2, t=0)
    assert not torch.equal(opt.state, first.state) and all(torch.equal(a, b) for a, b in zip(params, first.params))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_captured_step_is_replayed_with_other_values(bits):
    g = torch.Generator().manual_seed(9)
    start = tensors(SIZES, DTYPES, 0.02, g)
    grads = [gradients(SIZES, DTYPES, g) for _ in range(4)]
    held = [x.clone() for x in grads[0]]
    params = [p.clone() for p in start]
    opt = B.AdamW(params, bits=bits, seed=SEED)
    lr, t = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        factor = B.grad_norm(held, 0.5)
        opt.step(held, lr=lr, t=t, wd=0.1, factor=factor[1:])
    eager = B.AdamW([p.clone() for p in start], bits=bits, seed=SEED)
    for i in range(4):
        for h, x in zip(held, grads[i]):
            h.copy_(x)
        lr.fill_(0.01 * (i + 1))
        t.fill_(10 * i)
        graph.replay()
        eager.step(grads[i], lr=torch.full((1,), 0.01 * (i + 1), device="cuda"), t=torch.tensor([10 * i], device="cuda"), wd=0.1,
                   factor=B.grad_norm(grads[i], 0.5)[1:])
        assert all(torch.equal(a, b) for a, b in zip(params + [opt.state], eager.params + [eager.state]))
    # numbers instead of tensors: the bias corrections are rounded from the same doubles
    plain = B.AdamW([p.clone() for p in start], bits=bits, seed=SEED)
    for i in range(4):
        plain.step(grads[i], lr=float(torch.tensor(0.01 * (i + 1))), t=10 * i, wd=0.1, factor=B.grad_norm(grads[i], 0.5)[1:])
    for a, b in zip(plain.params, eager.params):
        # (the two logarithms and exponentials may differ in their last bit, so a correction by half a step of fp32, and what a step
        # of the code makes of that: 4 updates of at most lr (1 + 1/8), a rounding of the type)
        assert bool(((a.double() - b.double()).abs() <= 0.1 * 1.2 + torch.finfo(a.dtype).eps * a.double().abs()).all())


@pytest.mark.parametrize("bits", [8, 32])
def test_a_factor_that_is_not_finite_changes_nothing(bits):
    g = torch.Generator().manual_seed(10)
    params = tensors(SIZES, DTYPES, 0.02, g)
    opt = B.AdamW(params, bits=bits, seed=SEED)
    grads = gradients(SIZES, DTYPES, g)
    opt.step(grads, lr=1e-2, t=0)
    before = [x.clone() for x in params + [opt.state]]
    for bad in (math.inf, -math.inf, math.nan):
        opt.step(grads, lr=1e-2, t=1, factor=torch.full((1,), bad, device="cuda"))
        grads[7][3] = bad
        r = B.grad_norm(grads, 1.0)
        assert not math.isfinite(r[0].item()) and math.isnan(r[1].item())
        opt.step(grads, lr=1e-2, t=1, factor=r[1:])
    assert all(torch.equal(a, b) for a, b in zip(before, params + [opt.state]))


def test_a_gradient_that_is_not_finite_stays_in_its_block():
    g = torch.Generator().manual_seed(11)
    params = [torch.randn(2048, generator=g).cuda()]
    grads = [torch.randn(2048, generator=g).cuda()]
    clean = B.AdamW([params[0].clone()], seed=SEED)
    clean.step(grads, lr=1e-2, t=0)
    grads[0][300], grads[0][900], grads[0][901] = math.inf, math.nan, -math.inf
    opt = B.AdamW(params, seed=SEED)
    opt.step(grads, lr=1e-2, t=0)
    m, v = opt.moments()
    wm, wv = clean.moments()
    assert m[300] == math.inf and v[300] == math.inf and m[901] == -math.inf and bool(m[900].isnan()) and bool(v[900].isnan())
    spoilt = torch.zeros(8, 256, dtype=torch.bool, device="cuda")
    spoilt[[1, 3]] = True
    spoilt = spoilt.view(-1)
    assert torch.equal(m[~spoilt], wm[~spoilt]) and torch.equal(v[~spoilt], wv[~spoilt])
    others = torch.ones(2048, dtype=torch.bool, device="cuda")
    others[[300, 900, 901]] = False
    assert torch.equal(params[0][others], clean.params[0][others])         # the update is formed before rounding
    assert bool(m[others].isfinite().all()) and bool(v[others].isfinite().all())


@pytest.mark.parametrize("size", [1e-30, 1e-18, 1e-12, 1.0, 1e9, 1e18])
def test_moments_of_any_size(size):
    """Codes cover every exponent: entries of 1e-18 to 1e18 (1e-30: v is below what fp32 holds, m is not)."""
    g = torch.Generator().manual_seed(12)
    x = torch.randn(4096, generator=g) * size
    params = [torch.zeros(4096, device="cuda")]
    opt = B.AdamW(params, seed=SEED)
    opt.step([x.cuda()], lr=1e-2, t=0)
    m, v = (y.cpu().double() for y in opt.moments())
    want_m, want_v = 0.1 * x.double(), 0.001 * x.double().square()
    # a step of the code above or below: 1/8 of the value; or below the smallest code of the block
    low = want_m.abs().view(-1, 256).amax(1, keepdim=True).expand(-1, 256).reshape(-1) * 2.0 ** -14
    assert bool(((m - want_m).abs() <= want_m.abs() / 8 + low).all())
    if size >= 1e-18:
        # (1e-18: v is 1e-39, below fp32's normal range, where the codes are (c % 8) / 8 2^-126: 2^-129 apart whatever the value)
        assert bool(((v - want_v).abs() <= want_v / 8 + 2.0 ** -129 + want_v.view(-1, 256).amax(1, keepdim=True).expand(-1, 256).reshape(-1) * 2.0 ** -30).all())


def test_a_moment_moves_although_its_codes_are_far_apart():
    """A constant gradient: the mean of v follows 1 - b2^t.  A step adds at most (an eighth of v) (a thousandth) of variance, which decays by
    b2^2 a step: a standard deviation below 0.25 of v for one element, 0.001 for the mean of 65536; eight of those."""
    params = [torch.zeros(65536, device="cuda")]
    grads = [torch.full((65536,), 0.5, device="cuda")]
    opt = B.AdamW(params, seed=SEED)
    for t in range(1500):
        opt.step(grads, lr=0.0, t=t)
    m, v = opt.moments()
    want = 0.25 * (1 - B2 ** 1500)
    assert abs(v.double().mean().item() - want) <= 0.008 * 0.25
    # m: variance at most 1/4 (an eighth)^2 a step, decaying by b1^2: 0.15 of m for one element
    assert abs(m.double().mean().item() - 0.5) <= 8 * 0.15 * 0.5 / 256
    for t in range(1500, 3000):                                # and back down
        opt.step([torch.zeros_like(grads[0])], lr=0.0, t=t)
    m, v = opt.moments()
    assert abs(v.double().mean().item() - want * B2 ** 1500) <= 0.008 * 0.25


def test_c_i_is_one_without_bias_correction():
    p = torch.zeros(8, device="cuda")
    opt = B.AdamW([p], bits=32, bias_correction=False)
    opt.step([torch.full((8,), 2.0, device="cuda")], lr=1.0, t=0)
    want = -(0.1 * 2.0) / (math.sqrt(0.001 * 4.0) + 1e-8)
    assert bool(((p.double() - want).abs() <= 16 * U * abs(want)).all())


# ---------------------------------------------------------------- norm
@pytest.mark.parametrize("sizes", [[1], [0, 1], [8191, 8192, 8193], [3, 100_003, 5], [1 << 20] * 3, [17] * 49, [5] * 2000])
@pytest.mark.parametrize("std", [1e-38, 1e-25, 1e-3, 1.0, 1e19, 1e30])
def test_norm_matches_the_definition(sizes, std):
    g = torch.Generator().manual_seed(13)
    grads = tensors(sizes, DTYPES, std, g)
    want = math.sqrt(sum(float(x.double().square().sum()) for x in grads))
    r = B.grad_norm(grads, want / 3 if want else 1.0)
    # a thread's 32 squares in fp32, half of their errors; joined in 64 bits; a rounding (below the normal range an absolute one)
    assert abs(r[0].item() - want) <= 18 * U * want + 2.0 ** -149
    assert abs(r[1].item() - 1 / 3) <= 20 * U / 3
    assert B.grad_norm(grads, want * 2)[1].item() == 1.0 and B.grad_norm(grads)[1].item() == 1.0
    assert torch.equal(B.grad_norm(grads, 7.0), B.grad_norm([x.clone() for x in grads], 7.0))


def test_norm_of_rows_that_differ_by_all_of_fp32():
    x = torch.zeros(3 * 8192, device="cuda")
    x[0], x[5], x[8192 + 9], x[2 * 8192:] = 1e-30, 3e-30, 2e25, 0.0
    assert abs(B.grad_norm([x])[0].item() - 2e25) <= 2 * U * 2e25
    x[8192 + 9] = 0
    want = math.hypot(x[0].item(), x[5].item())
    assert abs(B.grad_norm([x])[0].item() - want) <= 2 * U * want
    assert B.grad_norm([torch.zeros(5000, device="cuda")], 1.0).tolist() == [0.0, 1.0]
    assert B.grad_norm([torch.zeros(0, device="cuda")], 1.0).tolist() == [0.0, 1.0]


def test_norm_leaves_out_what_is_missing():
    g = torch.Generator().manual_seed(14)
    a, b = tensors([300, 400], DTYPES, 1.0, g)
    assert torch.equal(B.grad_norm([a, None, b], 1.0), B.grad_norm([a, b], 1.0))
    out, ws = torch.zeros(2, device="cuda"), torch.empty(B.grad_norm_workspace_bytes(2), dtype=torch.uint8, device="cuda")
    assert B.grad_norm([a, b], 1.0, out=out, workspace=ws) is out and torch.equal(out, B.grad_norm([a, b], 1.0))


# ---------------------------------------------------------------- refusals
def test_lists_that_are_refused():
    p = torch.zeros(64, device="cuda")
    q = torch.zeros(128, device="cuda")
    for bad in ([], [None], [p, p], [p, p.view(8, 8)], [torch.zeros(8, 8, device="cuda").t()], [torch.zeros(8)], [torch.zeros(8, dtype=torch.float16, device="cuda")]):
        with pytest.raises(ValueError):
            B.AdamW(bad)
    with pytest.raises(B.ApolloError):
        B.AdamW([p], bits=16)
    for state in (torch.zeros(3, dtype=torch.uint8, device="cuda"), torch.zeros(514, device="cuda"), torch.zeros(514, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            B.AdamW([p], state=state)
    opt = B.AdamW([p, q])
    g = [torch.ones_like(p), torch.ones_like(q)]
    for grads in ([g[0]], g[::-1], [g[0], g[1].view(2, 64)], [g[0], g[1].cpu()], [g[0], g[1].half()], [g[0], torch.ones(256, device="cuda")[::2]]):
        with pytest.raises(ValueError):
            opt.step(grads, lr=0.1, t=0)
    for kw in (dict(lr=math.nan, t=0), dict(lr=0.1, t=-1), dict(lr=0.1, t=0, wd=math.inf)):
        with pytest.raises(B.ApolloError):
            opt.step(g, **kw)
    for kw in (dict(lr=torch.zeros(2, device="cuda"), t=0), dict(lr=0.1, t=torch.zeros(1, device="cuda")), dict(lr=0.1, t=0, factor=torch.ones(1))):
        with pytest.raises(ValueError):
            opt.step(g, **kw)
    with pytest.raises(B.ApolloError) as e:
        opt.step([g[0], torch.ones(129, device="cuda")[1:]], lr=0.1, t=0)              # 4-byte offset
    assert e.value.code == B.ERR_ALIGN
    assert not p.any() and not q.any() and not opt.state.any()
    for kw in (dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(eps=math.nan)):
        with pytest.raises(B.ApolloError):
            B.AdamW([p], **kw).step([g[0]], lr=0.1, t=0)


def test_norms_that_are_refused():
    p = torch.zeros(64, device="cuda")
    for bad in ([], [None], [p.half()], [p.cpu()], [torch.zeros(8, 8, device="cuda").t()]):
        with pytest.raises(ValueError):
            B.grad_norm(bad)
    for m in (0.0, -1.0, math.nan):
        with pytest.raises(B.ApolloError):
            B.grad_norm([p], m)
    with pytest.raises(ValueError):
        B.grad_norm([p], out=torch.zeros(3, device="cuda"))
    with pytest.raises(B.ApolloError) as e:
        B.grad_norm([p], workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == B.ERR_WORKSPACE
