"""The operators this package adds around the optimizer step, as cases that can be timed and compared.

Three families: the orthogonalised update of 2-D weights (Newton-Schulz products, with momentum and decay),
the embedding lookup with its gradient, and the log probabilities of given tokens with entropy, top
alternatives and gradient.  `run` computes them in plain torch operations in 32 bits, or, where `own` is
true, through the package's public calls; `exact` computes the same from the definitions in 64 bits.
"""
import math

import torch

own = False

NS = (3.4445, -4.7750, 2.0315)      # coefficients of the quintic step
EPS = 1e-7
LR, WD, MU = 0.02, 0.01, 0.95
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one attention matrix of a small model, orthogonalised by itself: the smallest call, latency counts
        {"name": "ortho 512x512", "op": "ortho", "hidden": 512, "inter": 0, "layers": 1, "dtype": "bf16", "grad": "row_scaled"},
        # one layer of a small model: seven matrices of two shapes, one of them tall
        {"name": "ortho layer 1024", "op": "ortho", "hidden": 1024, "inter": 2736, "layers": 1, "dtype": "bf16", "grad": "student_t3"},
        # half the list of a 60M model, 28 small matrices: one optimizer step
        {"name": "muon 60M 4 layers", "op": "muon", "hidden": 512, "inter": 1376, "layers": 4, "dtype": "bf16", "grad": "row_scaled"},
        # a 1B layer in fp32: 5461 columns, rows that start on no 16-byte boundary
        {"name": "muon 1B layer f32", "op": "muon", "hidden": 2048, "inter": 5461, "layers": 1, "dtype": "f32", "grad": "outlier_cols"},
        # a 7B layer in bf16: the largest matrices
        {"name": "muon 7B layer", "op": "muon", "hidden": 4096, "inter": 11008, "layers": 1, "dtype": "bf16", "grad": "normal"},
        # the next token of 64 sequences
        {"name": "embed decode 64", "op": "embed", "tokens": 64, "vocab": 32000, "dim": 4096, "dtype": "bf16", "scale": 64.0, "pad": False},
        # a training batch, tokens as frequent as words are
        {"name": "embed batch 32768", "op": "embed", "tokens": 32768, "vocab": 32000, "dim": 2048, "dtype": "bf16", "scale": 1.0, "pad": False},
        # the gradient of that table, every row of it written
        {"name": "embed grad 16384", "op": "embed_grad", "tokens": 16384, "vocab": 32000, "dim": 2048, "dtype": "bf16", "scale": 1.0, "pad": False, "add": False},
        # fp32, odd sizes, padded positions, added to what an earlier microbatch left
        {"name": "embed grad ragged f32", "op": "embed_grad", "tokens": 4099, "vocab": 32001, "dim": 1029, "dtype": "f32", "scale": 32.0, "pad": True, "add": True},
        # serving: the chosen tokens of 16 sequences with their 20 best alternatives
        {"name": "logprob decode 16", "op": "logprob", "rows": 16, "vocab": 32000, "dtype": "bf16", "top": 20, "scale": 1.25, "mask": 0.0, "pad": 0, "grad": False},
        # fp32 logits cut out of a wider buffer, masked words, rows with nothing left, ignored targets
        {"name": "logprob masked f32", "op": "logprob", "rows": 777, "vocab": 50001, "dtype": "f32", "top": 5, "scale": 1.0, "mask": 0.3, "pad": 14, "grad": True},
        # a training batch: forward and gradient, with an entropy term
        {"name": "logprob train 8192", "op": "logprob", "rows": 8192, "vocab": 32000, "dtype": "bf16", "top": 0, "scale": 1.0, "mask": 0.0, "pad": 0, "grad": True},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm; half the time a multiple of 8."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, v // 8 * 8) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["ortho", "muon", "muon", "embed", "embed_grad", "embed_grad", "logprob", "logprob", "logprob"])
    dtype = "bf16" if op == "ortho" else rng.choice(["bf16", "bf16", "f32"])
    if op in ("ortho", "muon"):
        hidden = _log(rng, 256, 2400 if dtype == "f32" else 4096)
        inter = 0 if rng.random() < 0.3 else min(4 * hidden, 11008, _log(rng, hidden, 4 * hidden))
        most = 4 if hidden < 700 else 2 if hidden < 1500 else 1
        return {"op": op, "hidden": hidden, "inter": inter, "layers": rng.randint(1, most), "dtype": dtype,
                "grad": rng.choice(["normal", "row_scaled", "student_t3", "outlier_cols"])}
    if op == "embed":
        dim = _log(rng, 64, 4096)
        return {"op": op, "tokens": min(_log(rng, 1, 65536), (1 << 26) // dim), "vocab": _log(rng, 1000, 64000), "dim": dim, "dtype": dtype,
                "scale": rng.choice([1.0, math.sqrt(dim)]), "pad": rng.random() < 0.3}
    if op == "embed_grad":
        dim = _log(rng, 64, 4096)
        return {"op": op, "tokens": min(_log(rng, 1, 65536), (1 << 26) // dim), "vocab": _log(rng, 1000, 64000), "dim": dim, "dtype": dtype,
                "scale": rng.choice([1.0, math.sqrt(dim)]), "pad": rng.random() < 0.3, "add": rng.random() < 0.3}
    vocab = _log(rng, 1000, 130000)
    grad = rng.random() < 0.6
    rows = min(_log(rng, 1, 8192), (1 << 27) // vocab)
    top = rng.choice([0, 0, 1, 5, 20])
    return {"op": op, "rows": min(rows, 1024) if top else rows, "vocab": vocab, "dtype": dtype, "top": top, "scale": rng.choice([1.0, 0.7, 1.25]),
            "mask": rng.choice([0.0, 0.0, 0.3]), "pad": rng.choice([0, 0, 3, 16]), "grad": grad}


def _shapes(case):
    h, i = case["hidden"], case["inter"]
    layer = [(h, h)] if i == 0 else [(h, h)] * 4 + [(h, i)] * 2 + [(i, h)]
    return layer * case["layers"]


# ---------------------------------------------------------------- inputs
def _gradient(shape, kind, g):
    x = torch.randn(*shape, generator=g, device="cuda")
    if kind == "row_scaled":
        x *= torch.pow(10.0, torch.rand(shape[0], 1, generator=g, device="cuda") * 2 - 1)
    elif kind == "student_t3":
        x /= torch.sqrt(torch.randn(3, *shape, generator=g, device="cuda").square_().sum(0) / 3)
    elif kind == "outlier_cols":
        x *= torch.where(torch.rand(1, shape[1], generator=g, device="cuda") < 0.01, 50.0, 1.0)
    return x * 1e-3


def _tokens(n, vocab, g):
    """Tokens as frequent as words: the k-th of the vocabulary about 1/k of the time."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1.0)) - 1).long().clamp_(0, vocab - 1)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, dt = case["op"], DT[case["dtype"]]
    s = {"case": case}
    if op in ("ortho", "muon"):
        shapes = _shapes(case)
        s["G"] = [_gradient(x, case["grad"], g).to(dt) for x in shapes]
        if op == "ortho":
            s["O"] = [torch.empty(x, dtype=dt, device="cuda") for x in shapes]
        else:
            s["W"] = [(torch.randn(*x, generator=g, device="cuda") * 0.02).to(dt) for x in shapes]
            s["M"] = [_gradient(x, case["grad"], g) * 0.3 for x in shapes]
        if own:
            from paper_2412_05270_b200 import binding as B
            cfg = B.make_muon_config(dtype=B.DT_BF16 if dt == torch.bfloat16 else B.DT_F32, steps=5, coef=NS, momentum=MU, nesterov=True,
                                     scale=B.MUON_SCALE_SHAPE, eps=EPS)
            s["opt"] = B.Muon(shapes, cfg)
    elif op in ("embed", "embed_grad"):
        n, v, d = case["tokens"], case["vocab"], case["dim"]
        s["index"] = _tokens(n, v, g)
        if case["pad"]:
            s["index"][1:][torch.rand(n - 1, generator=g, device="cuda") < 0.1] = -1
        if op == "embed":
            s["E"] = (torch.randn(v, d, generator=g, device="cuda") * 0.02).to(dt)
            s["out"] = torch.empty(n, d, dtype=dt, device="cuda")
        else:
            s["dY"] = (torch.randn(n, d, generator=g, device="cuda") * 1e-3).to(dt)
            s["dE"] = (torch.randn(v, d, generator=g, device="cuda") * 1e-2).to(dt) if case["add"] else torch.empty(v, d, dtype=dt, device="cuda")
            if own:
                from paper_2412_05270_b200 import binding as B
                s["ws"] = torch.empty(B.embedding_grad_workspace_bytes(n, v, d), dtype=torch.uint8, device="cuda")
    else:
        n, v = case["rows"], case["vocab"]
        z = torch.randn(n, v + case["pad"], generator=g, device="cuda") * 2.0
        t = torch.randint(0, v, (n,), generator=g, device="cuda")
        z[torch.arange(n, device="cuda"), t] += 4.0
        if case["mask"]:
            z[torch.rand(z.shape, generator=g, device="cuda") < case["mask"]] = -math.inf
            if n > 3:
                z[n // 3] = -math.inf
            t[16::17] = -100
        s["z"], s["t"] = z.to(dt)[:, :v], t
        if case["grad"]:
            s["g"] = torch.randn(n, generator=g, device="cuda") / n
            s["h"] = torch.randn(n, generator=g, device="cuda") * 0.01 / n
            s["dz"] = torch.empty(n, v, dtype=dt, device="cuda")
    return s


# ---------------------------------------------------------------- one pass
def _ns_step(x):
    a, b, c = NS
    gram = x @ x.T
    return a * x + (b * gram + c * (gram @ gram)) @ x


def _ns(u):
    x = u.T if u.shape[0] > u.shape[1] else u
    x = x / (x.square().sum().sqrt() + EPS)
    for _ in range(5):
        x = _ns_step(x)
    return x.T if u.shape[0] > u.shape[1] else x


def _muon(w, g, m):
    m.mul_(MU).add_(g.float() * (1 - MU))
    o = _ns((1 - MU) * g.float() + MU * m)
    w.copy_(w.float() - LR * (math.sqrt(max(1.0, w.shape[0] / w.shape[1])) * o + WD * w.float()))
    return w


def _embed(s):
    e, i = s["E"], s["index"]
    live = (i >= 0) & (i < e.shape[0])
    s["out"].copy_(torch.where(live[:, None], e[i.clamp(0, e.shape[0] - 1)].float() * s["case"]["scale"], 0.0))
    return s["out"]


def _embed_grad(s):
    i, d = s["index"], s["dE"]
    live = (i >= 0) & (i < d.shape[0])
    acc = torch.zeros(d.shape, dtype=torch.float32, device="cuda")
    acc.index_add_(0, i[live], s["dY"][live].float())
    acc *= s["case"]["scale"]
    d.copy_(acc + d.float() if s["case"]["add"] else acc)
    return d


def _logprob(s):
    c = s["case"]
    z = s["z"].float() * c["scale"]
    n, v = z.shape
    t = s["t"]
    live = (t >= 0) & (t < v)
    at = torch.arange(n, device="cuda"), t.clamp(0, v - 1)
    top = z.amax(1)
    base = torch.where(torch.isinf(top), 0.0, top)
    e = torch.exp(z - base[:, None])
    total = e.sum(1)
    lse = torch.log(total) + base
    some = total > 0
    p = torch.where(some[:, None], e / total[:, None], 0.0)
    entropy = torch.where(some, lse - (p * torch.where(p > 0, z, 0.0)).sum(1), 0.0)
    lp = torch.where(live, torch.where(some, z[at] - lse, -math.inf), 0.0)
    out = {"logprob": lp, "entropy": entropy, "lse": lse}
    if c["top"]:
        val, idx = torch.sort(z, dim=1, descending=True, stable=True)
        val, idx = val[:, : c["top"]], idx[:, : c["top"]]
        out["top_logprob"] = torch.where(some[:, None], val - lse[:, None], -math.inf)
        out["top_index"] = idx.to(torch.int32)
    if c["grad"]:
        gl = torch.where(live, s["g"], 0.0)
        d = -p * (gl[:, None] + s["h"][:, None] * torch.where(p > 0, z - lse[:, None] + entropy[:, None], 0.0))
        d[at] += torch.where(some, gl, 0.0)
        s["dz"].copy_(d * c["scale"])
        out["dz"] = s["dz"]
    return out


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == "ortho":
            return [o.copy_(_ns(g.float())) for o, g in zip(s["O"], s["G"])]
        if op == "muon":
            return {"W": [_muon(w, g, m) for w, g, m in zip(s["W"], s["G"], s["M"])], "M": s["M"]}
        return {"embed": _embed, "embed_grad": _embed_grad, "logprob": _logprob}[op](s)
    from paper_2412_05270_b200 import binding as B
    c = s["case"]
    if op == "ortho":
        s["opt"].orthogonalize(s["G"], s["O"])
        return s["O"]
    if op == "muon":
        s["opt"].step(s["W"], s["G"], s["M"], LR, WD)
        return {"W": s["W"], "M": s["M"]}
    if op == "embed":
        return B.embedding(s["E"], s["index"], scale=c["scale"], out=s["out"])
    if op == "embed_grad":
        return B.embedding_grad(s["dY"], s["index"], c["vocab"], scale=c["scale"], out=s["dE"], accumulate=c["add"], workspace=s["ws"])
    r = B.token_logprobs(s["z"], s["t"], scale=c["scale"], top=c["top"])
    out = {"logprob": r.logprob, "entropy": r.entropy, "lse": r.lse}
    if c["top"]:
        out["top_logprob"], out["top_index"] = r.top_logprob, r.top_index
    if c["grad"]:
        out["dz"] = B.token_logprobs_grad(s["z"], s["t"], r.lse, r.entropy, s["g"], s["h"], scale=c["scale"], out=s["dz"])
    return out


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op in ("ortho", "muon"):
        shapes = _shapes(case)
        params = sum(r * c for r, c in shapes)
        flops = 0.0
        for r, c in shapes:
            m, n = min(r, c), max(r, c)
            # A = X X^T and A^2 are symmetric (half the products); two steps can share X's two long products:
            # X <- P(A2) P(A1) X with A2 = P(A1)^2 A1
            one, two = 3.0 * m * m * n + m ** 3, 3.0 * m * m * n + 5.0 * m ** 3
            flops += 2 * min(2 * one, two) + one
        return {"bytes": params * (2 * e if op == "ortho" else 3 * e + 8), "flops": flops}
    if op in ("embed", "embed_grad"):
        n, v, d = case["tokens"], case["vocab"], case["dim"]
        distinct = sum(1 - (1 - math.log((k + 2) / (k + 1)) / math.log(v + 1)) ** n for k in range(v))
        if op == "embed":
            return {"bytes": (distinct + n) * d * e + 8 * n, "flops": n * d}
        return {"bytes": n * d * e + (2 * distinct if case["add"] else v) * d * e + 8 * n, "flops": n * d}
    n, v = case["rows"], case["vocab"]
    passes = 3 if case["grad"] else 1
    return {"bytes": passes * n * v * e + 8 * n + (20 if case["grad"] else 12) * n + 8 * n * case["top"], "flops": (10 if case["grad"] else 4) * n * v}


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_ortho(u):
    flip = u.shape[0] > u.shape[1]
    y = (u.t() if flip else u).contiguous()
    y = y / (torch.linalg.norm(y) + EPS)
    a, b, c = NS
    for _ in range(5):
        q = torch.matmul(y, y.t())
        q = torch.addmm(q, q, q, beta=b, alpha=c)
        y = torch.addmm(y, q, y, beta=a)
    return y.t().contiguous() if flip else y


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "ortho":
        return [_exact_ortho(x.double()) for x in s["G"]]
    if op == "muon":
        new_w, new_m = [], []
        for w, g, m in zip(s["W"], s["G"], s["M"]):
            g, mom = g.double(), m.double()
            mom = mom * MU + g * (1 - MU)
            o = _exact_ortho(g * (1 - MU) + mom * MU)
            gain = max(1.0, w.shape[0] / w.shape[1]) ** 0.5
            new_w.append(w.double() * (1 - LR * WD) - o * (LR * gain))
            new_m.append(mom)
        return {"W": new_w, "M": new_m}
    if op == "embed":
        keep = (s["index"] >= 0).double()
        return s["E"].double().index_select(0, s["index"].clamp(min=0)) * (keep * case["scale"])[:, None]
    if op == "embed_grad":
        v, d = s["dE"].shape
        sums = torch.zeros(v + 1, d, dtype=torch.float64, device="cuda")        # padded positions go to a row of their own
        where = torch.where(s["index"] < 0, v, s["index"])
        sums.scatter_add_(0, where[:, None].expand(-1, d), s["dY"].double())
        sums = sums[:v] * case["scale"]
        return sums + s["dE"].double() if case["add"] else sums
    z = s["z"].double() * case["scale"]
    rows, v = z.shape
    lse = torch.logsumexp(z, 1)
    alive = ~torch.isinf(lse)
    logp = torch.where(alive[:, None], z - torch.where(alive, lse, 0.0)[:, None], -math.inf)
    p = logp.exp()
    entropy = torch.special.entr(p).sum(1)
    counted = (s["t"] >= 0) & (s["t"] < v)
    chosen = logp.gather(1, s["t"].clamp(0, v - 1)[:, None])[:, 0]
    out = {"logprob": torch.where(counted, chosen, 0.0), "entropy": entropy, "lse": lse}
    if case["top"]:
        order = torch.argsort(z, dim=1, descending=True, stable=True)[:, : case["top"]]
        out["top_logprob"], out["top_index"] = logp.gather(1, order), order.to(torch.int32)
    if case["grad"]:
        one_hot = torch.zeros_like(z)
        one_hot.scatter_(1, s["t"].clamp(0, v - 1)[:, None], (counted & alive).double()[:, None])
        g = torch.where(counted, s["g"].double(), 0.0)
        dz = g[:, None] * (one_hot - p) - s["h"].double()[:, None] * (p * entropy[:, None] - torch.special.entr(p))
        out["dz"] = dz * case["scale"]
    return out
