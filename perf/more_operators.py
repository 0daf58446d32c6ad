"""Timing cases of the operators that train a layer's experts: products of rows grouped by expert with the experts'
matrices and the gradients of those products, the gated activation with row weights forward and backward, the orthogonalised
update of matrices, and the optimiser step around it.

Sizes come from the workloads of this repository: hidden sizes 256, 2048 and 2880 with experts of 768 and 2880, 32 or 128
experts, 4 or 8 of them per token, the estimator's matrices; rows run from one token's choices to a long batch of tokens.
The plain forms below are elementary torch operations in 32 bits; `exact` is the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)       # of the orthogonalising iteration, which is run five times
ITERATIONS = 5
MOMENTUM, LR, DECAY, RMS = 0.95, 1e-4, 0.01, 0.2


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token's eight choices among 128 experts, gate and up rows together: eight experts' weights are streamed, latency
        dict(name="product_one_token", op="product", rows=8, tail=0, experts=128, n=1536, k=2048, dtype="bf16", transpose=False),
        # a prompt of 512 tokens, top-8, down projection: most experts get some 30 rows, their weights are what is read
        dict(name="product_prompt", op="product", rows=4096, tail=0, experts=128, n=2048, k=768, dtype="bf16", transpose=False),
        # a training batch of 8192 tokens, some of them padding: matrix products
        dict(name="product_training", op="product", rows=65536, tail=1200, experts=128, n=1536, k=2048, dtype="bf16", transpose=False),
        # gradient of the inputs of 32 experts 2880 wide, a training batch of 8192 tokens, top-4
        dict(name="input_grad_training", op="product", rows=32768, tail=0, experts=32, n=5760, k=2880, dtype="bf16", transpose=True),
        # weight gradients of a small float32 layer, a ragged batch
        dict(name="weight_grad_small", op="weight_grad", rows=1205, tail=5, experts=8, n=256, k=180, dtype="f32", out="f32"),
        # weight gradients of a training batch; experts' sizes differ by a factor of ten
        dict(name="weight_grad_training", op="weight_grad", rows=65536, tail=1200, experts=128, n=1536, k=2048, dtype="bf16", out="bf16"),
        # the activation of one token's eight choices, with their gates: latency
        dict(name="swiglu_one_token", op="swiglu_forward", rows=8, cols=768, dtype="bf16", weighted=True),
        # its backward pass over a training batch: bandwidth
        dict(name="swiglu_backward_training", op="swiglu_backward", rows=65536, cols=768, dtype="bf16", weighted=True),
        # one small matrix by itself: a chain of small products
        dict(name="orthogonalise_small", op="orthogonalise", count=1, m=256, n=256, dtype="f32"),
        # a stack of wide matrices
        dict(name="orthogonalise_stack", op="orthogonalise", count=8, m=1024, n=4096, dtype="bf16"),
        # the three matrices of the 2048-wide layers' estimator, one of them tall
        dict(name="muon_estimator", op="muon", tensors="estimator", grad="f32", copy=True),
        # gate, up and down of 16 experts
        dict(name="muon_experts", op="muon", tensors="experts", grad="bf16", copy=True),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["product", "product", "product", "weight_grad", "weight_grad", "swiglu_forward", "swiglu_backward",
                     "orthogonalise", "muon"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op in ("product", "weight_grad"):
        step = rng.choice([1, 8, 32, 64])      # odd sizes, and those that models have
        n, k = (max(step, _log_int(rng, 8, 4096) // step * step) for _ in range(2))
        experts = _log_int(rng, 1, max(1, min(256, 300_000_000 // (n * k))))
        most = min((1 << 27) // max(n, k), 400_000_000_000 // (2 * n * k), 65536)
        rows = _log_int(rng, 1, max(1, most if dtype == "bf16" else most // 8))
        c = dict(op=op, rows=rows, tail=rng.choice([0, 0, min(rows // 2, rng.randint(0, 300))]), experts=experts, n=n, k=k, dtype=dtype)
        if op == "product":
            return dict(c, transpose=rng.random() < 0.5)
        return dict(c, out="f32" if dtype == "f32" else rng.choice(["f32", "bf16"]))
    if op in ("swiglu_forward", "swiglu_backward"):
        cols = _log_int(rng, 4, 8192)
        return dict(op=op, rows=_log_int(rng, 1, (1 << 25) // cols), cols=cols, dtype=dtype, weighted=rng.random() < 0.7)
    if op == "orthogonalise":
        m, n = (_log_int(rng, 4, 3000) for _ in range(2))
        most = int(4e10 / (min(m, n) ** 2 * max(m, n)))
        return dict(op=op, count=_log_int(rng, 1, max(1, min(64, most))), m=m, n=n, dtype=dtype)
    return dict(op=op, tensors="drawn", pick=rng.randrange(1 << 30), grad=rng.choice(["f32", "bf16"]), copy=rng.random() < 0.5)


def _stacks(case):
    """[how many, rows, columns] of each stack of matrices that an optimiser step updates."""
    if case["tensors"] == "estimator":         # proj, ffn_in and ffn_out at H = 2048, m = 4, n = 2
        return [[1, 512, 2048], [1, 1024, 512], [1, 512, 1024]]
    if case["tensors"] == "experts":
        return [[16, 768, 2048], [16, 768, 2048], [16, 2048, 768]]
    import random
    r = random.Random(case["pick"])
    pick = lambda: [_log_int(r, 1, 8), _log_int(r, 8, 1500), _log_int(r, 8, 1500)]  # noqa: E731
    return [pick() for _ in range(r.randint(1, 6))]


# ------------------------------------------------------------------------------------------------ inputs
def _group_sizes(case, seed):
    """Rows of each expert: some are liked much more than others, in a small batch many get none."""
    r = np.random.default_rng(int(seed))
    liked = np.exp(0.6 * r.standard_normal(case["experts"]))
    rows = case["rows"] - case["tail"]
    if rows <= 16 and case["experts"] >= rows:                     # one token: a row for each of its experts
        sizes = np.zeros(case["experts"], dtype=np.int64)
        sizes[r.choice(case["experts"], rows, replace=False)] = 1
        return sizes
    return r.multinomial(rows, liked / liked.sum())


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    s = dict(case)
    op = case["op"]
    if op in ("product", "weight_grad"):
        rows, experts, n, k, dt = case["rows"], case["experts"], case["n"], case["k"], DTYPES[case["dtype"]]
        sizes = _group_sizes(case, seed)
        s["sizes"], s["longest"] = sizes.tolist(), int(max(1, sizes.max()))
        s["ends"] = torch.from_numpy(np.cumsum(sizes).astype(np.int32)).to("cuda")
        if op == "product":
            s["x"] = rand(rows, n if case["transpose"] else k).to(dt)
            s["w"] = torch.empty(experts, n, k, dtype=dt, device="cuda")
            s["w"].normal_(std=k ** -0.5, generator=g)
        else:
            s["dy"], s["x"] = (0.1 * rand(rows, n)).to(dt), rand(rows, k).to(dt)
    elif op in ("swiglu_forward", "swiglu_backward"):
        rows, cols, dt = case["rows"], case["cols"], DTYPES[case["dtype"]]
        s["a"] = (1.5 * rand(rows, 2 * cols)).to(dt)
        s["weight"] = torch.rand(rows, generator=g, device="cuda") if case["weighted"] else None
        if op == "swiglu_backward":
            s["dh"] = (0.1 * rand(rows, cols)).to(dt)
    elif op == "orthogonalise":
        s["g"] = _gradient(rand, case["count"], case["m"], case["n"]).to(DTYPES[case["dtype"]])
    else:
        s["p"] = [0.03 * rand(*shape) for shape in _stacks(case)]
        s["g"] = [_gradient(rand, *shape).to(DTYPES[case["grad"]]) for shape in _stacks(case)]
        s["m"] = [10.0 * _gradient(rand, *shape) for shape in _stacks(case)]
        s["copy"] = [p.to(torch.bfloat16) for p in s["p"]] if case["copy"] else None
        if own:
            from paper_2603_19289_amd import training
            s["optimizer"] = training.Muon(s["p"], lr=LR, momentum=MOMENTUM, weight_decay=DECAY, update_rms=RMS, iterations=ITERATIONS,
                                           coefficients=COEFFICIENTS, copies=s["copy"], states={"m": s["m"]})
    return s


def _gradient(rand, count, m, n):
    """Matrices as gradients are: a few directions that stand out of noise; the rows' and columns' sizes differ."""
    few = min(4, m, n)
    strong = torch.bmm(rand(count, m, few), rand(count, few, n)) * few ** -0.5
    return 1e-3 * (rand(count, m, n) + 0.5 * strong) * torch.exp(0.3 * rand(count, m, 1)) * torch.exp(0.3 * rand(count, 1, n))


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["op"]
    if own:
        from paper_2603_19289_amd import training
        if op == "product":
            return training.grouped_product(s["x"], s["w"], s["ends"], transpose=s["transpose"])
        if op == "weight_grad":
            return training.grouped_weight_grad(s["dy"], s["x"], s["ends"], dtype=DTYPES[s["out"]])
        if op == "swiglu_forward":
            return training.swiglu_forward(s["a"], s["weight"])
        if op == "swiglu_backward":
            return training.swiglu_backward(s["dh"], s["a"], s["weight"])
        if op == "orthogonalise":
            return training.orthogonalise(s["g"], iterations=ITERATIONS, coefficients=COEFFICIENTS)
        s["optimizer"].step(s["g"])
        return {"p": s["p"], "m": s["m"], "copy": s["copy"]}
    if op == "product":
        return _product(s)
    if op == "weight_grad":
        return _weight_grad(s)
    if op == "swiglu_forward":
        return _swiglu(s)
    if op == "swiglu_backward":
        return _swiglu_backward(s)
    if op == "orthogonalise":
        return _orthogonal(s["g"].float()).to(torch.bfloat16)
    return _muon(s)


# ------------------------------------------------------------------------------------------------ plain forms
def _places(s):
    """Which row lies at each place [experts, longest group], and which of the places are rows."""
    ends = s["ends"].long()
    begins = torch.cat([ends.new_zeros(1), ends[:-1]])
    at = begins[:, None] + torch.arange(s["longest"], device="cuda")
    there = at < ends[:, None]
    return torch.where(there, at, 0), there


def _product(s):
    x, w = s["x"], s["w"]
    cols = s["k"] if s["transpose"] else s["n"]
    if s["longest"] == 1:                      # a few rows: only the experts that have one
        expert = torch.searchsorted(s["ends"], torch.arange(s["rows"], dtype=torch.int32, device="cuda"), right=True)
        live = (expert < s["experts"])[:, None]
        v = w[expert.clamp(max=s["experts"] - 1)].float()
        y = (v * x.float()[:, :, None]).sum(1) if s["transpose"] else (v * x.float()[:, None]).sum(2)
        return torch.where(live, y, 0.0).to(x.dtype)
    at, there = _places(s)
    v = w.float()
    part = torch.bmm(x.float()[at], v if s["transpose"] else v.transpose(1, 2))
    y = torch.zeros(s["rows"] + 1, cols, device="cuda")
    y[torch.where(there, at, s["rows"])] = part
    return y[:-1].to(x.dtype)


def _weight_grad(s):
    at, there = _places(s)
    dy = torch.where(there[:, :, None], s["dy"].float()[at], 0.0)
    return torch.bmm(dy.transpose(1, 2), s["x"].float()[at]).to(DTYPES[s["out"]])


def _halves(s):
    return s["a"].float().split(s["cols"], dim=1)


def _swiglu(s):
    gate, up = _halves(s)
    h = gate / (1.0 + torch.exp(-gate)) * up
    return (h if s["weight"] is None else h * s["weight"][:, None]).to(s["a"].dtype)


def _swiglu_backward(s):
    gate, up = _halves(s)
    dh = s["dh"].float()
    share = 1.0 / (1.0 + torch.exp(-gate))
    act = gate * share
    dweight = None
    if s["weight"] is not None:
        dweight = (dh * act * up).sum(1)
        dh = dh * s["weight"][:, None]
    da = torch.cat([dh * up * share * (1.0 + gate * (1.0 - share)), dh * act], dim=1)
    return da.to(s["a"].dtype), dweight


def _orthogonal(g):
    a, b, c = COEFFICIENTS
    tall = g.shape[1] > g.shape[2]
    x = g.transpose(1, 2).contiguous() if tall else g
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt().float()
    x = torch.where(norm > 0, x / norm, 0.0)
    for _ in range(ITERATIONS):
        square = torch.bmm(x, x.transpose(1, 2))
        x = a * x + torch.bmm(b * square + c * torch.bmm(square, square), x)
    return x.transpose(1, 2) if tall else x


def _muon(s):
    for i, (p, g, m) in enumerate(zip(s["p"], s["g"], s["m"])):
        g = g.float()
        m.copy_(m * MOMENTUM + g)
        o = _orthogonal(g + m * MOMENTUM)
        p.copy_(p * (1.0 - LR * DECAY) - o * (LR * RMS * math.sqrt(max(p.shape[1:]))))
        if s["copy"] is not None:
            s["copy"][i].copy_(p)
    return {"p": s["p"], "m": s["m"], "copy": s["copy"]}


# ------------------------------------------------------------------------------------------------ work
def _products(count, m, n):
    m, n = min(m, n), max(m, n)
    return ITERATIONS * count * 2 * (2 * m * m * n + m ** 3)


def work(case):
    op, size = case["op"], 2 if case.get("dtype") == "bf16" else 4
    if op in ("product", "weight_grad"):
        rows, n, k = case["rows"], case["n"], case["k"]
        live = rows - case["tail"]
        if op == "product":                    # experts that get no row need not be read: few rows touch few experts
            touched = min(case["experts"], live)
            return dict(bytes=size * (rows * (n + k) + touched * n * k) + 4 * case["experts"], flops=2 * live * n * k)
        out = 2 if case["out"] == "bf16" else 4
        return dict(bytes=size * live * (n + k) + out * case["experts"] * n * k + 4 * case["experts"], flops=2 * live * n * k)
    if op in ("swiglu_forward", "swiglu_backward"):
        n, gates = case["rows"] * case["cols"], 4 * case["rows"] if case["weighted"] else 0
        if op == "swiglu_forward":
            return dict(bytes=3 * n * size + gates, flops=6 * n)
        return dict(bytes=5 * n * size + 2 * gates, flops=16 * n)
    if op == "orthogonalise":
        n = case["count"] * case["m"] * case["n"]
        return dict(bytes=n * (size + 2), flops=_products(case["count"], case["m"], case["n"]))
    n = sum(math.prod(shape) for shape in _stacks(case))
    each = 16 + (4 if case["grad"] == "f32" else 2) + (2 if case["copy"] else 0)
    return dict(bytes=n * each, flops=sum(_products(*shape) for shape in _stacks(case)))


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_orthogonal(g):
    """By the definition: the iteration acts on the singular values alone."""
    a, b, c = COEFFICIENTS
    norm = torch.linalg.vector_norm(g, dim=(1, 2), keepdim=True)
    x = g / torch.where(norm > 0, norm, torch.ones_like(norm))
    small = x.shape[1] <= x.shape[2]
    for _ in range(ITERATIONS):
        if small:
            q = x @ x.mT
            x = torch.baddbmm(x, q, torch.baddbmm(x, q, x, beta=b, alpha=c), beta=a)
        else:
            q = x.mT.contiguous() @ x
            x = torch.baddbmm(x, torch.baddbmm(x, x, q, beta=b, alpha=c), q, beta=a)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("product", "weight_grad"):
        n, k, begin = case["n"], case["k"], 0
        if op == "product":
            y = torch.zeros(case["rows"], k if case["transpose"] else n, dtype=torch.float64, device="cuda")
        else:
            y = torch.zeros(case["experts"], n, k, dtype=torch.float64, device="cuda")
        for e, size in enumerate(s["sizes"]):
            if size:
                some = slice(begin, begin + size)
                if op == "weight_grad":
                    y[e] = s["dy"][some].double().t().contiguous() @ s["x"][some].double()
                elif case["transpose"]:
                    y[some] = s["x"][some].double() @ s["w"][e].double()
                else:
                    y[some] = (s["w"][e].double() @ s["x"][some].double().t().contiguous()).t()
                begin += size
        return y
    if op in ("swiglu_forward", "swiglu_backward"):
        a = s["a"].double()
        gate, up = a[:, :case["cols"]], a[:, case["cols"]:]
        share = torch.sigmoid(gate)
        weight = torch.ones(case["rows"], 1, dtype=torch.float64, device="cuda") if s["weight"] is None else s["weight"].double()[:, None]
        if op == "swiglu_forward":
            return weight * torch.nn.functional.silu(gate) * up
        dh = s["dh"].double()
        slope = share + gate * share * torch.sigmoid(-gate)
        return torch.hstack([weight * dh * up * slope, weight * dh * gate * share]), \
            None if s["weight"] is None else torch.linalg.vecdot(dh, gate * share * up)
    if op == "orthogonalise":
        return _exact_orthogonal(s["g"].double())
    out = {"p": [], "m": [], "copy": [] if case["copy"] else None}
    for p, g, m in zip(s["p"], s["g"], s["m"]):
        g, p = g.double(), p.double()
        m = torch.add(g, m.double(), alpha=MOMENTUM)
        o = _exact_orthogonal(torch.add(g, m, alpha=MOMENTUM))
        p = p - LR * DECAY * p - LR * RMS * max(p.shape[1], p.shape[2]) ** 0.5 * o
        out["p"].append(p)
        out["m"].append(m)
        if case["copy"]:
            out["copy"].append(p)
    return out
