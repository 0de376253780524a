"""Operators around the optimizer step and the logits, as cases that can be timed and compared.

Four operators: the global norm of a list of gradients with the factor that clips it, the AdamW step over a list of tensors with
states in 8 or 32 bits, the adjustment of logits (penalties for repeated tokens, biases, grammar masks) and its gradient.  `run`
computes them in plain torch operations in 32 bits, or, where `own` is true, through the package's public calls; `exact` computes
the same from the definitions in 64 bits.

States in 8 bits: blocks of 256 elements share an exponent byte k per moment.  A code c stands for (1 + (c % 8) / 8) 2^(k + c // 8 - 127);
m has a sign and 7 bits, code 0 is zero; v has 8 bits.  Rounding is stochastic, with 16 bits per element from Philox4x32-10 (key: the
seed; counter: block, lane of 8 elements, step).
"""
import math

import torch

own = False

LR, WD, B1, B2, ADAM_EPS = 1e-3, 0.1, 0.9, 0.999, 1e-8
MAX_NORM = 1.0
SEED = 0x1234ABCD5678EF01
BLOCK = 256
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases
def _list(name, op, vocab, dim, inter, layers, p, g, **kw):
    return {"name": name, "op": op, "vocab": vocab, "dim": dim, "inter": inter, "layers": layers, "p": p, "g": g, **kw}


def _rows(name, op, rows, vocab, dtype, **kw):
    base = {"history": 0, "share": 1, "rho": 1.0, "freq": 0.0, "pres": 0.0, "bias": "none", "sparse": 0, "mask": 1.0, "one_mask": False, "place": False}
    return {"name": name, "op": op, "rows": rows, "vocab": vocab, "dtype": dtype, **{**base, **kw}}


def listed():
    return [
        # every gradient of a 60M model, 8 layers of seven matrices, table, head and gains: what clipping reads each step
        _list("norm 60M model", "norm", 32000, 512, 1376, 8, "bf16", "bf16"),
        # fp32 gradients of a 1B model's ends, rows of odd length
        _list("norm ends ragged f32", "norm", 32001, 2047, 0, 24, "f32", "f32"),
        # the gains of a 7B model alone: 65 vectors, the smallest call, latency counts
        _list("adamw32 gains 7B", "adamw", 0, 4096, 0, 32, "f32", "f32", bits=32, clip=False, t=10),
        # table, head and gains of a 60M model, clipped, states in 8 bits
        _list("adamw8 ends 60M", "adamw", 32000, 512, 0, 8, "bf16", "bf16", bits=8, clip=True, t=0),
        # table and head of a 7B model: the largest list
        _list("adamw8 ends 7B", "adamw", 32000, 4096, 0, 32, "bf16", "bf16", bits=8, clip=True, t=5000),
        # fp32 weights with bf16 gradients, odd sizes, states in 32 bits
        _list("adamw32 ragged f32", "adamw", 32001, 1029, 2731, 2, "f32", "bf16", bits=32, clip=False, t=100),
        # serving: 16 sequences of up to 512 tokens, their next token, a grammar for each, in place
        _rows("adjust decode 16", "adjust", 16, 32000, "bf16", history=512, rho=1.15, freq=0.2, pres=0.4, mask=0.1, place=True),
        # a large serving batch with long histories and a few biased words each, fp32
        _rows("adjust long f32", "adjust", 129, 50001, "f32", history=8191, rho=1.2, freq=0.1, pres=0.0, sparse=63, place=True),
        # a training batch of 8 sequences: every position with the tokens before it, a shared bias, one mask for all
        _rows("adjust train 8192", "adjust", 8192, 32000, "bf16", history=1024, share=1024, rho=1.1, freq=0.1, pres=0.1, bias="shared", mask=0.97, one_mask=True),
        # the gradient of a small batch, rows with nothing left to choose
        _rows("adjust grad 64", "grad", 64, 32000, "bf16", history=256, rho=1.15, mask=0.1, sparse=16),
        # fp32, odd sizes, a bias for each row
        _rows("adjust grad ragged f32", "grad", 777, 50001, "f32", history=333, rho=0.9, bias="row", mask=0.6),
        # the gradient of the training batch, summed over the rows for the shared bias
        _rows("adjust grad train 8192", "grad", 8192, 32000, "bf16", history=1024, share=1024, rho=1.1, bias="shared", mask=0.97, one_mask=True),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm; half the time a multiple of 8."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, v // 8 * 8) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["norm", "adamw", "adamw", "adamw", "adjust", "adjust", "grad", "grad"])
    if op in ("norm", "adamw"):
        dim = _log(rng, 64, 4096)
        vocab = rng.choice([0, 1, 1, 1]) * min(_log(rng, 1000, 64000), (1 << 26) // dim)
        layers = rng.randint(1, 32)
        inter = _log(rng, dim, 4 * dim) if rng.random() < 0.4 else 0
        if inter:
            layers = max(1, min(layers, (1 << 26) // (4 * dim * dim + 3 * dim * inter)))
        case = {"op": op, "vocab": vocab, "dim": dim, "inter": inter, "layers": layers, "p": rng.choice(["bf16", "f32"]), "g": rng.choice(["bf16", "f32"])}
        if op == "adamw":
            case |= {"bits": rng.choice([8, 8, 32]), "clip": rng.random() < 0.5, "t": rng.choice([0, 1, 10, 1000, 100000])}
        return case
    vocab = _log(rng, 1000, 130000)
    rows = min(_log(rng, 1, 8192), (1 << 27) // vocab)
    case = {"op": op, "rows": rows, "vocab": vocab, "dtype": rng.choice(["bf16", "bf16", "f32"]),
            "history": rng.choice([0, 1, 1]) * min(_log(rng, 1, 16384), (1 << 23) // rows), "share": 1, "rho": rng.choice([0.9, 1.1, 1.3]),
            "freq": rng.choice([0.0, 0.3]), "pres": rng.choice([0.0, 0.5]), "bias": rng.choice(["none", "none", "shared", "row"]),
            "sparse": rng.choice([0, 0, 1, 30, 300]), "mask": rng.choice([1.0, 0.02, 0.5, 0.99]), "one_mask": rng.random() < 0.3,
            "place": op == "adjust" and rng.random() < 0.5}
    if case["history"] and rows % 4 == 0 and rng.random() < 0.4:
        case["share"] = rows // 4
    return case


def _shapes(case):
    """Table and head, the matrices where there are any, two gains a layer and the last one."""
    v, d, i = case["vocab"], case["dim"], case["inter"]
    ends = [(v, d)] * 2 if v else []
    layer = [(d, d)] * 4 + [(d, i)] * 2 + [(i, d)] if i else []
    return ends + (layer + [(d,)] * 2) * case["layers"] + [(d,)]


def _sizes(case):
    """Elements of each tensor, and the blocks of BLOCK before it."""
    sizes = [math.prod(s) for s in _shapes(case)]
    first = [0]
    for n in sizes:
        first.append(first[-1] + (n + BLOCK - 1) // BLOCK)
    return sizes, first


# ---------------------------------------------------------------- inputs
def _tokens(n, vocab, g):
    """Tokens as frequent as words: the k-th of the vocabulary about 1/k of the time."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1.0)) - 1).to(torch.int32).clamp_(0, vocab - 1)


def _prepare_list(case, g, s):
    sizes, first = _sizes(case)
    total = first[-1] * BLOCK
    live = torch.zeros(total, dtype=torch.bool, device="cuda")
    for n, b in zip(sizes, first):
        live[b * BLOCK: b * BLOCK + n] = True

    def flat(std, dtype):
        return (torch.randn(total, generator=g, device="cuda") * std * live).to(dtype)
    # (gradients of a block differ in size by a few powers of two, as rows of a table do)
    spread = torch.exp2(torch.randint(-6, 3, (first[-1], 1), generator=g, device="cuda").float())
    grads = (flat(1e-3, torch.float32).view(-1, BLOCK) * spread).view(-1)
    s["G"] = grads.to(DT[case["g"]])
    s["grads"] = [s["G"][b * BLOCK: b * BLOCK + n].view(x) for n, b, x in zip(sizes, first, _shapes(case))]
    if case["op"] == "norm":
        return
    s["P"] = flat(0.02, DT[case["p"]])
    s["params"] = [s["P"][b * BLOCK: b * BLOCK + n].view(x) for n, b, x in zip(sizes, first, _shapes(case))]
    m = (flat(3e-4, torch.float32).view(-1, BLOCK) * spread).view(-1)
    v = (flat(1e-3, torch.float32).view(-1, BLOCK) * spread).view(-1).square_()
    if case["t"] == 0:
        m, v = torch.zeros_like(m), torch.zeros_like(v)
    # the states as a program keeps them between steps: one buffer, m of all tensors, v of all tensors (8 bits: then the exponent
    # bytes, m's and v's of each block)
    if case["bits"] == 32:
        s["state"] = torch.cat([m, v]).view(torch.uint8)
    else:
        half = torch.full((total // BLOCK, BLOCK), 1 << 15, device="cuda", dtype=torch.int32)
        (cm, km), (cv, kv) = _encode(m.abs().view(-1, BLOCK), half, 15), _encode(v.view(-1, BLOCK), half, 31)
        cm |= (m < 0).view(-1, BLOCK).int() << 7
        s["state"] = torch.cat([cm.view(-1), cv.view(-1), torch.stack([km, kv], 1).view(-1)]).to(torch.uint8)
    if own:
        from paper_2412_05270_b200 import binding as B
        s["opt"] = B.AdamW(s["params"], bits=case["bits"], beta1=B1, beta2=B2, eps=ADAM_EPS, seed=SEED, state=s["state"])


def _prepare_rows(case, g, s):
    n, v, dt = case["rows"], case["vocab"], DT[case["dtype"]]
    z = torch.randn(n, v, generator=g, device="cuda") * 2.0
    z[torch.arange(n, device="cuda"), torch.randint(0, v, (n,), generator=g, device="cuda")] += 6.0
    s["z"] = z.to(dt)
    length = case["history"]
    s["history"] = s["lengths"] = s["start"] = None
    if length:
        share = case["share"]
        s["history"] = _tokens(n // share * length, v, g).view(n // share, length)
        s["history"][torch.rand(s["history"].shape, generator=g, device="cuda") < 0.01] = -1
        if share == 1:
            s["lengths"] = torch.randint(length // 2, length + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
        else:                                     # position t of its sequence: the tokens before it
            s["lengths"] = (torch.arange(n, device="cuda", dtype=torch.int32) % share * length // share).to(torch.int32)
        s["start"] = s["lengths"] // 4            # the prompt
    per_row = torch.rand(n, generator=g, device="cuda") * 0.2 + 0.9
    s["rho"], s["freq"], s["pres"] = case["rho"] * per_row, case["freq"] * per_row, case["pres"] * per_row
    s["bias"] = None
    if case["bias"] != "none":
        s["bias"] = (torch.randn(*([v] if case["bias"] == "shared" else [n, v]), generator=g, device="cuda") * 0.3).to(dt)
    s["b_index"] = s["b_value"] = None
    if case["sparse"]:
        k = case["sparse"]
        s["b_index"] = torch.randint(-1, v, (n, k), generator=g, device="cuda", dtype=torch.int32)
        s["b_index"][:, -1] = s["b_index"][:, 0]          # a word that is named twice gets both
        s["b_value"] = torch.randn(n, k, generator=g, device="cuda") * 2.0
    s["mask"] = None
    if case["mask"] < 1.0:
        words = (v + 31) // 32
        bits = torch.rand(1 if case["one_mask"] else n, words, 32, generator=g, device="cuda") < case["mask"]
        if n > 3 and not case["one_mask"]:
            bits[n // 3] = False                          # a row with nothing left
        powers = torch.ones((), dtype=torch.int64, device="cuda") << torch.arange(32, device="cuda")
        s["mask"] = (bits * powers).sum(-1).to(torch.int32)
    if case["op"] == "grad":
        s["dy"] = (torch.randn(n, v, generator=g, device="cuda") / n).to(dt)
        s["out"] = torch.empty_like(s["dy"])
    else:
        s["out"] = s["z"] if case["place"] else torch.empty_like(s["z"])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    (_prepare_list if case["op"] in ("norm", "adamw") else _prepare_rows)(case, g, s)
    return s


# ---------------------------------------------------------------- one pass
def _norm(s):
    norm = s["G"].double().square().sum().sqrt()          # 64 bits: the sum is long
    factor = torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)
    return torch.stack([norm, factor]).float()


def _mulhilo(a, c):
    p = a * c                                             # wraps as 64 unsigned bits would
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _dither(blocks, t):
    """16 random bits for each element: (blocks, BLOCK) int32."""
    c0 = torch.arange(blocks, device="cuda", dtype=torch.int64)[:, None].expand(blocks, 32)
    c1 = torch.arange(32, device="cuda", dtype=torch.int64).expand(blocks, 32)
    c2, c3 = torch.full_like(c1, t & 0xFFFFFFFF), torch.full_like(c1, t >> 32)
    k0, k1 = SEED & 0xFFFFFFFF, SEED >> 32
    for _ in range(10):
        h0, l0 = _mulhilo(c0, 0xD2511F53)
        h1, l1 = _mulhilo(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], -1)             # (blocks, 32, 4)
    return torch.stack([words & 0xFFFF, words >> 16], -1).view(blocks, BLOCK).int()


def _encode(x, dither, top):
    """Codes and exponents of the blocks x >= 0; top: the largest exponent of a code."""
    bits = x.contiguous().view(torch.int32)
    k = (((bits.amax(1) + 0xFFFFF) >> 23) - top).clamp_(0, 255 - top)
    return (((bits + dither * 16) >> 20) - k[:, None] * 8).clamp_(0, top * 8 + 7), k


def _decode(code, k):
    return ((code.int() << 20) + (k.int()[:, None] << 23)).view(torch.float32)


def _split(state, bits):
    """m, v (and, of 8 bits, the exponents) of a flat state."""
    if bits == 32:
        return state.view(torch.float32).chunk(2)
    n = state.numel() // (2 * BLOCK + 2) * BLOCK
    return state[:n].view(-1, BLOCK), state[n: 2 * n].view(-1, BLOCK), state[2 * n:].view(-1, 2)


def _moments(state, bits):
    if bits == 32:
        m, v = _split(state, bits)
        return {"m": m, "v": v}
    cm, cv, k = _split(state, bits)
    mag = torch.where((cm & 127) == 0, 0.0, _decode(cm & 127, k[:, 0]))
    m = torch.where(cm > 127, -mag, mag)
    return {"m": m.to(torch.bfloat16).view(-1), "v": _decode(cv, k[:, 1]).to(torch.bfloat16).view(-1)}


def _adamw(s):
    c = s["case"]
    g = s["G"].float()
    if c["clip"]:
        g = g * _norm(s)[1]
    if c["bits"] == 32:
        m, v = _split(s["state"], 32)
        m.mul_(B1).add_(g * (1 - B1))
        v.mul_(B2).add_(g.square() * (1 - B2))
    else:
        cm, cv, k = _split(s["state"], 8)
        g = g.view(-1, BLOCK)
        mag = torch.where((cm & 127) == 0, 0.0, _decode(cm & 127, k[:, 0]))
        m = torch.where(cm > 127, -mag, mag) * B1 + g * (1 - B1)
        v = _decode(cv, k[:, 1]) * B2 + g.square() * (1 - B2)
        dither = _dither(cm.shape[0], c["t"])
        new_m, km = _encode(m.abs(), dither, 15)
        new_v, kv = _encode(v, dither, 31)
        cm.copy_(new_m | ((m < 0).int() << 7))
        cv.copy_(new_v)
        k.copy_(torch.stack([km, kv], 1))
    p = s["P"].float().view(g.shape)
    step = (m / (1 - B1 ** (c["t"] + 1))) / ((v / (1 - B2 ** (c["t"] + 1))).sqrt() + ADAM_EPS) + WD * p
    s["P"].copy_((p - LR * step).view(-1))
    return {"P": s["P"], **_moments(s["state"], c["bits"])}


def _counts(s, from_start):
    """How often each word occurs in each row's history."""
    n, v = s["case"]["rows"], s["case"]["vocab"]
    h = s["history"].repeat_interleave(s["case"]["share"], 0)
    at = torch.arange(h.shape[1], device="cuda")
    live = (h >= 0) & (h < v) & (at < s["lengths"][:, None])
    if from_start:
        live &= at >= s["start"][:, None]
    counts = torch.zeros(n, v, dtype=torch.int32, device="cuda")
    return counts.scatter_add_(1, h.clamp(0, v - 1).long(), live.int())


def _allowed(s):
    j = torch.arange(s["case"]["vocab"], device="cuda")
    return ((s["mask"][:, j >> 5] >> (j & 31)) & 1) > 0


def _adjust(s):
    c = s["case"]
    x = s["z"].float()
    if s["history"] is not None:
        rho = s["rho"][:, None]
        x = torch.where(_counts(s, False) > 0, torch.where(x > 0, x / rho, x * rho), x)
        d = _counts(s, True)
        x = x - torch.where(d > 0, s["freq"][:, None] * d + s["pres"][:, None], 0.0)
    if s["bias"] is not None:
        x = x + s["bias"].float()
    if s["b_index"] is not None:
        i = s["b_index"]
        live = (i >= 0) & (i < c["vocab"])
        x = x.scatter_add(1, i.clamp(0, c["vocab"] - 1).long(), torch.where(live, s["b_value"], 0.0))
    if s["mask"] is not None:
        x = torch.where(_allowed(s), x, -math.inf)
    return s["out"].copy_(x)


def _adjust_grad(s):
    c = s["case"]
    a = s["dy"].float()
    if s["mask"] is not None:
        a = torch.where(_allowed(s), a, 0.0)
    out = {}
    if c["bias"] == "shared":
        out["bias"] = a.sum(0).to(s["bias"].dtype)
    elif c["bias"] == "row":
        out["bias"] = a.to(s["bias"].dtype)
    if s["b_index"] is not None:
        i = s["b_index"]
        out["value"] = torch.where((i >= 0) & (i < c["vocab"]), a.gather(1, i.clamp(0, c["vocab"] - 1).long()), 0.0)
    if s["history"] is not None:
        rho = s["rho"][:, None]
        a = torch.where(_counts(s, False) > 0, torch.where(s["z"] > 0, a / rho, a * rho), a)
    out["logits"] = s["out"].copy_(a)
    return out


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        return {"norm": _norm, "adamw": _adamw, "adjust": _adjust, "grad": _adjust_grad}[op](s)
    from paper_2412_05270_b200 import binding as B
    if op == "norm":
        return B.grad_norm(s["grads"], MAX_NORM)
    if op == "adamw":
        factor = B.grad_norm(s["grads"], MAX_NORM)[1:] if c["clip"] else None
        s["opt"].step(s["grads"], lr=LR, wd=WD, t=c["t"], factor=factor)
        m, v = s["opt"].moments()
        return {"P": s["P"], "m": m, "v": v}
    rules = {"history": s["history"], "lengths": s["lengths"], "repetition": s["rho"], "mask": s["mask"], "bias_index": s["b_index"]}
    if op == "adjust":
        return B.adjust_logits(s["z"], start=s["start"], frequency=s["freq"], presence=s["pres"], bias=s["bias"], bias_value=s["b_value"],
                               out=s["out"], **rules)
    r = B.adjust_logits_grad(s["z"], s["dy"], bias=c["bias"], out=s["out"], **rules)
    return {k: x for k, x in r._asdict().items() if x is not None}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] in ("norm", "adamw"):
        n = sum(math.prod(s) for s in _shapes(case))
        g = 2 if case["g"] == "bf16" else 4
        if case["op"] == "norm":
            return {"bytes": n * g + 8, "flops": 2 * n}
        p = 2 if case["p"] == "bf16" else 4
        # states in 8 bits: codes read and written, the values they stand for given back
        state = 16 if case["bits"] == 32 else 4 + 4 + 4 / BLOCK
        return {"bytes": n * (g + 2 * p + state), "flops": 16 * n}
    n, v, length = case["rows"], case["vocab"], case["history"]
    e = 2 if case["dtype"] == "bf16" else 4
    rules = (n // case["share"] * length + n * (length > 0) * 2) * 4 + n * case["sparse"] * 8
    if case["mask"] < 1.0:
        rules += (1 if case["one_mask"] else n) * (v + 31) // 32 * 4
    dense = {"none": 0, "shared": v * e, "row": n * v * e}[case["bias"]]
    if case["op"] == "grad":
        return {"bytes": 2 * n * v * e + dense + rules, "flops": 2 * n * v}
    if case["place"] and case["bias"] == "none":          # only the words that change
        touched = n * (min(v, length) / 4 + case["sparse"]) * 2 * e + n * v * (1 - case["mask"]) * e
        return {"bytes": touched + rules, "flops": 2 * n * (length + case["sparse"])}
    return {"bytes": 2 * n * v * e + dense + rules, "flops": 4 * n * v}


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_norm(grads):
    # (in pieces: the squares of the largest list in 64 bits would take 2 GB more)
    total = sum(float(torch.linalg.vector_norm(x.double())) ** 2 for x in grads)
    return math.sqrt(total), min(1.0, MAX_NORM / math.sqrt(total)) if total else 1.0


def _exact_words(blocks, t):
    """The four words of each (block, lane) of Philox4x32-10, products in halves of 16 bits."""
    low = 0xFFFF

    def product(c, a):
        a0, a1, c0, c1 = a & low, a >> 16, c & low, c >> 16
        mid = a1 * c0 + ((a0 * c0) >> 16)
        cross = a0 * c1 + (mid & low)
        return a1 * c1 + (mid >> 16) + (cross >> 16), ((cross & low) << 16) | ((a0 * c0) & low)

    n = torch.arange(blocks * 32, device="cuda", dtype=torch.int64)
    x = [n // 32, n % 32, torch.full_like(n, t % 2 ** 32), torch.full_like(n, t // 2 ** 32)]
    key = [SEED % 2 ** 32, SEED // 2 ** 32]
    for r in range(10):
        (ha, la), (hb, lb) = product(0xD2511F53, x[0]), product(0xCD9E8D57, x[2])
        x = [hb ^ x[1] ^ key[0], lb, ha ^ x[3] ^ key[1], la]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    return x


def _exact_round(x, chance, top):
    """The values that blocks x >= 0 of 64 bits are held as."""
    biggest = x.amax(1, keepdim=True)
    _, e = torch.frexp(torch.where(biggest > 0, biggest, 1.0))           # biggest = f 2^e, 1/2 <= f < 1
    e = torch.where(biggest > (1 - 2.0 ** -4) * torch.exp2(e.double()), e + 1, e)      # it may be rounded up to the next power
    least = torch.where(biggest > 0, (e - 1 - top).double(), -127.0).clamp(min=-127.0)      # exponent of code 0
    _, at = torch.frexp(torch.where(x > 0, x, 1.0))
    unit = torch.exp2((at - 4).double())
    y = torch.floor(x / unit + chance) * unit
    floor = torch.exp2(least)
    return torch.where((x > 0) & (y > floor), y, floor), floor


def _exact_adamw(case, s):
    t, sizes = case["t"], _sizes(case)
    g = s["G"].double()
    if case["clip"]:
        g *= _exact_norm(s["grads"])[1]
    old = _moments(s["state"], case["bits"])
    m, v = old["m"].double().view(-1), old["v"].double().view(-1)
    m = m + (g - m) * (1 - B1)
    v = v + (g * g - v) * (1 - B2)
    del g
    p = s["P"].double()
    p = p * (1 - LR * WD) - LR * (m / (1 - math.pow(B1, t + 1))) / (torch.sqrt(v / (1 - math.pow(B2, t + 1))) + ADAM_EPS)
    if case["bits"] == 32:
        return {"P": p, "m": m, "v": v}
    blocks = sizes[1][-1]
    chance = torch.empty(blocks * 32, 8, dtype=torch.float64, device="cuda")
    for i, w in enumerate(_exact_words(blocks, t)):
        chance[:, 2 * i], chance[:, 2 * i + 1] = (w % 65536) / 65536, (w // 65536) / 65536
    chance = chance.view(blocks, BLOCK)
    m, v = m.view(blocks, BLOCK), v.view(blocks, BLOCK)
    size, least = _exact_round(m.abs(), chance, 15)
    m = torch.where(size > least, torch.sign(m) * size, 0.0)
    v, least = _exact_round(v, chance, 31)
    v = torch.where((least <= 2.0 ** -127) & (v <= least), 0.0, v)       # a block of zeros
    return {"P": p, "m": m, "v": v}


def _exact_rows(case, s):
    n, v = case["rows"], case["vocab"]
    open_ = torch.ones(1, v, dtype=torch.bool, device="cuda")
    if s["mask"] is not None:
        bit = torch.arange(32, device="cuda", dtype=torch.int32)
        open_ = torch.bitwise_right_shift(s["mask"][:, :, None], bit).bitwise_and(1).bool().flatten(1)[:, :v]
    seen = count = None
    if s["history"] is not None:
        length = s["history"].shape[1]
        rows = torch.arange(n, device="cuda")[:, None].expand(n, length)
        tokens, at = s["history"][rows // case["share"], torch.arange(length, device="cuda")], torch.arange(length, device="cuda")
        valid = (tokens >= 0) & (tokens < v) & (at < s["lengths"][:, None])
        late = valid & (at >= s["start"][:, None])
        seen = torch.bincount((rows * v + tokens)[valid], minlength=n * v).view(n, v) > 0
        count = torch.bincount((rows * v + tokens)[late], minlength=n * v).view(n, v)
    i = s["b_index"]
    named = None if i is None else (i >= 0) & (i < v)
    rho = s["rho"].double()[:, None]
    if case["op"] == "adjust":
        y = s["z"].double()
        if seen is not None:
            y *= torch.where(seen, torch.where(y > 0, 1 / rho, rho), 1.0)
            y -= s["freq"].double()[:, None] * count + s["pres"].double()[:, None] * (count > 0)
        if s["bias"] is not None:
            y += s["bias"].double()
        if i is not None:
            y.index_put_((torch.arange(n, device="cuda")[:, None].expand_as(i)[named], i[named].long()), s["b_value"].double()[named], accumulate=True)
        return y.masked_fill_(~open_, -math.inf)
    a = s["dy"].double() * open_
    out = {}
    if case["bias"] != "none":
        out["bias"] = a.sum(0) if case["bias"] == "shared" else a.clone()
    if i is not None:
        out["value"] = a[torch.arange(n, device="cuda")[:, None], i.clamp(0, v - 1).long()] * named
    if seen is not None:
        a *= torch.where(seen, torch.where(s["z"] > 0, 1 / rho, rho), 1.0)
    out["logits"] = a
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return torch.tensor(_exact_norm(s["grads"]), dtype=torch.float64)
    return _exact_adamw(case, s) if case["op"] == "adamw" else _exact_rows(case, s)
