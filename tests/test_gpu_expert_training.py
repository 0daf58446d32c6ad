"""The operators that train a layer's experts, against their definitions in 64 bits.

Products are tested with small whole numbers: every partial sum is then a whole number below 2^24 that float holds, whatever the order,
so that a float32 result has to be equal and a bfloat16 one the nearest.  Products of other values have a bound that counts one rounding
(or, inside a matrix instruction, one cut: twice as much) for each of the K terms of a sum.  The other bounds are counted where they stand.
u = 2^-24 is half a step of float, `half(t)` that of an output's type."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def half(t):
    return torch.finfo(t).eps / 2


def rng(seed):
    return torch.Generator().manual_seed(seed)


def whole(shape, g, most=4):
    return torch.randint(-most, most + 1, shape, generator=g).float()


def close(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, what
    off = (got - want).abs() - bound
    worst = off.max().item() if off.numel() else -1.0
    assert not math.isnan(worst) and worst <= 0.0, f"{what}: over its bound by {worst:.3e}, largest error {(got - want).abs().max().item():.3e}"


def bounds(ends, rows):
    """The groups that ends stands for, whatever it holds."""
    begins, last = [], 0
    for e in ends:
        begins.append(last)
        last = max(last, min(max(e, 0), rows))
    return list(zip(begins, begins[1:] + [last]))


def product(x, w, ends, transpose):
    y = torch.zeros(x.shape[0], w.shape[2 if transpose else 1], dtype=torch.float64)
    for e, (b, t) in enumerate(bounds(ends, x.shape[0])):
        y[b:t] = x[b:t].double() @ (w[e].double() if transpose else w[e].double().t())
    return y


def weight_grad(dy, x, ends):
    return torch.stack([dy[b:t].double().t() @ x[b:t].double() for b, t in bounds(ends, x.shape[0])])


def i32(ends):
    return torch.tensor(ends, dtype=torch.int32, device="cuda")


# sizes of the groups (rows behind the last: a final negative number), n, k
GROUPS = [([1], 1, 1), ([0], 8, 8), ([5, 0, 3], 7, 9), ([64], 64, 64), ([130, 1, 0, 127, -9], 136, 200), ([17] * 5, 65, 63), ([0, 0, 300, 0], 256, 72),
          ([1] * 8 + [0] * 20, 96, 128), ([3, 200, 40, -1], 33, 257), ([129, 127], 128, 320), ([1] * 256, 24, 40), ([0] * 255 + [20], 16, 24),
          ([2, 0] * 30, 40, 1030), ([600, 500], 260, 264), ([-4], 8, 16), ([9, 70, 5], 1, 70), ([9, 70, 5], 70, 1),
          ([3, 0, 17, 1, -2], 300, 130), ([16, 1], 1031, 67), ([2, 5], 128, 3)]


def groups(case):
    sizes, n, k = case
    tail = -sizes[-1] if sizes[-1] < 0 else 0
    sizes = [s for s in sizes if s >= 0] or [0]
    ends, rows = [], 0
    for s in sizes:
        rows += s
        ends.append(rows)
    return ends, rows + tail, n, k


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", GROUPS, ids=str)
def test_grouped_product(case, dtype, transpose):
    from paper_2603_19289_amd import training as T
    ends, rows, n, k = groups(case)
    g = rng(rows * 31 + n * 7 + k)
    x, w = whole((rows, n if transpose else k), g), whole((len(ends), n, k), g)
    want = product(x, w, ends, transpose)
    t = TYPES[dtype]
    for kind in (torch.float32, torch.bfloat16):
        got = T.grouped_product(x.to("cuda", t), w.to("cuda", t), i32(ends), transpose=transpose, dtype=kind)
        assert got.dtype == kind and torch.equal(got.cpu(), want.to(kind)), (kind, (got.cpu().double() - want).abs().max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", GROUPS, ids=str)
def test_grouped_weight_grad(case, dtype):
    from paper_2603_19289_amd import training as T
    ends, rows, n, k = groups(case)
    g = rng(rows * 37 + n * 5 + k)
    dy, x = whole((rows, n), g), whole((rows, k), g)
    dy[rows - 1:], x[rows - 1:] = (dy[rows - 1:], x[rows - 1:]) if ends[-1] == rows else (float("nan"), float("inf"))   # belongs to nobody
    want = weight_grad(dy, x, ends)
    t = TYPES[dtype]
    for kind in (torch.float32, torch.bfloat16):
        got = T.grouped_weight_grad(dy.to("cuda", t), x.to("cuda", t), i32(ends), dtype=kind)
        assert got.dtype == kind and torch.equal(got.cpu(), want.to(kind)), kind


LARGE = [([700, 0, 1, 2000, 333, -50], 512, 768), ([100] * 40, 256, 520), ([4096], 1024, 1024), ([31, 2, 5000], 328, 2048), ([2500, 9], 40, 4096),
         ([40] * 100, 384, 256)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", LARGE, ids=str)
def test_larger_groups(case, dtype):
    """Whole numbers again, more rows than one tile has, in all three directions."""
    from paper_2603_19289_amd import training as T
    ends, rows, n, k = groups(case)
    g = torch.Generator("cuda").manual_seed(rows + n)
    t = TYPES[dtype]
    x, dy, w = (torch.randint(-3, 4, s, generator=g, device="cuda").to(t) for s in ((rows, k), (rows, n), (len(ends), n, k)))
    e = i32(ends)
    y, dx, dw = T.grouped_product(x, w, e), T.grouped_product(dy, w, e, transpose=True), T.grouped_weight_grad(dy, x, e)
    for i, (b, f) in enumerate(bounds(ends, rows)):
        assert torch.equal(y[b:f], (x[b:f].double() @ w[i].double().t()).to(t)), i
        assert torch.equal(dx[b:f], (dy[b:f].double() @ w[i].double()).to(t)), i
        assert torch.equal(dw[i], (dy[b:f].double().t() @ x[b:f].double()).to(t)), i
    assert not y[ends[-1]:].any() and not dx[ends[-1]:].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,n,k", [([9000, 0, 5, 700], 40, 72), ([20000], 56, 24), ([3000, 6000], 200, 136), ([4000, 4100], 75, 33), ([12345, 1, 0], 9, 1)], ids=str)
def test_weight_gradients_of_long_groups(sizes, n, k, dtype):
    """Rows that are split among workgroups and whose sums are joined: whole numbers that float holds, equal whatever the order."""
    from paper_2603_19289_amd import training as T
    ends, rows, n, k = groups((sizes, n, k))
    g = torch.Generator("cuda").manual_seed(rows)
    t = TYPES[dtype]
    dy, x = (torch.randint(-3, 4, s, generator=g, device="cuda").to(t) for s in ((rows + 3, n), (rows + 3, k)))
    want = torch.stack([dy[b:f].double().t() @ x[b:f].double() for b, f in bounds(ends, rows)])
    for kind in (torch.float32, torch.bfloat16):
        out = torch.full((len(sizes), n, k + 5), 2.0, dtype=kind, device="cuda")
        T.grouped_weight_grad(dy, x, i32(ends), dtype=kind, out=out[:, :, :k])
        assert torch.equal(out[:, :, :k], want.to(kind)) and torch.all(out[:, :, k:] == 2.0)


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,n,k", [([2, 0, -1], 7000, 3701), ([7], 7104, 7104), ([1, 16, 0, 6], 4000, 3328)], ids=str)
def test_few_rows_of_large_matrices(sizes, n, k, dtype, transpose):
    from paper_2603_19289_amd import training as T
    ends, rows, n, k = groups((sizes, n, k))
    g = torch.Generator("cuda").manual_seed(rows + n)
    x, w = (torch.randint(-3, 4, s, generator=g, device="cuda").to(TYPES[dtype]) for s in ((rows, n if transpose else k), (len(ends), n, k)))
    got = T.grouped_product(x, w, i32(ends), transpose=transpose, dtype=torch.float32)
    for i, (b, f) in enumerate(bounds(ends, rows)):
        assert torch.equal(got[b:f], (x[b:f].double() @ (w[i].double() if transpose else w[i].double().t())).float()), i
    assert not got[ends[-1]:].any()


@pytest.mark.parametrize("dtype,rows,experts,n,k", [("f32", 333, 3, 130, 700), ("bf16", 333, 3, 136, 704), ("bf16", 50, 7, 96, 2048), ("bf16", 301, 2, 75, 333)])
def test_products_of_any_values(dtype, rows, experts, n, k):
    """2 u for each term of a sum, and for float32 the products' own rounding; half a step of what goes out."""
    from paper_2603_19289_amd import training as T
    g, t = rng(rows), TYPES[dtype]
    x, dy, w = (torch.randn(s, generator=g).to(t) for s in ((rows, k), (rows, n), (experts, n, k)))
    ends = sorted(torch.randint(0, rows + 1, (experts,), generator=g).tolist())
    e = i32(ends)
    on = lambda v: v.to("cuda")  # noqa: E731
    for kind in (torch.float32, t):
        out = half(kind) if kind != torch.float32 else 0.0
        for got, f, a, b, terms in ((T.grouped_product(on(x), on(w), e, dtype=kind), lambda p, q: product(p, q, ends, False), x, w, k),
                                    (T.grouped_product(on(dy), on(w), e, transpose=True, dtype=kind), lambda p, q: product(p, q, ends, True), dy, w, n),
                                    (T.grouped_weight_grad(on(dy), on(x), e, dtype=kind), lambda p, q: weight_grad(p, q, ends), dy, x, rows)):
            want, size = f(a, b), f(a.abs(), b.abs())
            close(got, want, (2 * terms + 8) * U * size * (1 + out) + out * want.abs(), f"{kind} {terms}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_group_ends_of_any_value(dtype):
    """Ends that fall, lie outside of the rows, or repeat: groups are what the running maximum says."""
    from paper_2603_19289_amd import training as T
    g, t, rows = rng(5), TYPES[dtype], 90
    for ends in ([40, 20, 60, 60], [-5, 1000, 3, 2000], [2 ** 31 - 1, 0, 0, 5], [-2 ** 31, -1, 0, 17], [90, 90, 90, 90]):
        x, dy, w = (whole(s, g) for s in ((rows, 24), (rows, 40), (4, 40, 24)))
        e = i32(ends)
        on = lambda v: v.to("cuda", t)  # noqa: E731
        assert torch.equal(T.grouped_product(on(x), on(w), e, dtype=torch.float32).cpu().double(), product(x, w, ends, False))
        assert torch.equal(T.grouped_product(on(dy), on(w), e, transpose=True, dtype=torch.float32).cpu().double(), product(dy, w, ends, True))
        assert torch.equal(T.grouped_weight_grad(on(dy), on(x), e, dtype=torch.float32).cpu().double(), weight_grad(dy, x, ends))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("inter,hidden,pad", [(24, 40, 0), (24, 40, 8), (21, 37, 3), (64, 128, 1)])
def test_parts_of_expert_blocks(inter, hidden, pad, dtype):
    """Gate and up rows, and the down matrix, as parts of experts' blocks: read there, and their gradients written there; padded rows."""
    from paper_2603_19289_amd import training as T
    g, t, experts, ends, rows = rng(inter), TYPES[dtype], 5, [7, 7, 30, 33, 60], 66
    blocks = torch.full((experts, 3 * inter * hidden + pad), 7.0)
    blocks[:, :3 * inter * hidden] = whole((experts, 3 * inter * hidden), g)
    at = blocks.to("cuda", t)
    gate_up = at[:, :2 * inter * hidden].unflatten(1, (2 * inter, hidden))
    down = at[:, 2 * inter * hidden:3 * inter * hidden].unflatten(1, (hidden, inter))
    wide = torch.full((rows, hidden + 2 * pad), 9.0)
    wide[:, pad:pad + hidden] = whole((rows, hidden), g)
    x = wide.to("cuda", t)[:, pad:pad + hidden]
    h = whole((rows, inter), g).to("cuda", t)
    e = i32(ends)
    ref = lambda v: v.float().cpu()  # noqa: E731
    assert torch.equal(ref(T.grouped_product(x, gate_up, e)), product(ref(x), ref(gate_up), ends, False).to(t).float())
    assert torch.equal(ref(T.grouped_product(h, down, e)), product(ref(h), ref(down), ends, False).to(t).float())
    assert torch.equal(ref(T.grouped_product(x, down, e, transpose=True)), product(ref(x), ref(down), ends, True).to(t).float())
    grads = torch.full_like(at, 5.0)
    into = grads[:, 2 * inter * hidden:3 * inter * hidden].unflatten(1, (hidden, inter))
    before = into._version
    got = T.grouped_weight_grad(x, h, e, out=into)
    assert got is into and into._version > before
    assert torch.equal(ref(into), weight_grad(ref(x), ref(h), ends).to(t).float())
    grads[:, 2 * inter * hidden:3 * inter * hidden] = 5.0
    assert torch.all(grads == 5.0)                       # nothing beside it was written
    out = torch.full((rows, 2 * inter + 2 * pad + 1), 3.0, device="cuda", dtype=t)
    T.grouped_product(x, gate_up, e, out=out[:, pad:pad + 2 * inter])
    assert torch.equal(ref(out[:, pad:pad + 2 * inter]), product(ref(x), ref(gate_up), ends, False).to(t).float())
    out[:, pad:pad + 2 * inter] = 3.0
    assert torch.all(out == 3.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_row_for_all_and_one_matrix_for_all(dtype):
    from paper_2603_19289_amd import training as T
    g, t = rng(3), TYPES[dtype]
    x, w = whole((1, 48), g), whole((1, 32, 48), g)
    many, every = x.expand(8, 48), w.expand(8, 32, 48)
    got = T.grouped_product(x.to("cuda", t).expand(8, 48), w.to("cuda", t).expand(8, 32, 48), i32(range(1, 9)))
    assert torch.equal(got.cpu(), product(many, every, list(range(1, 9)), False).to(t))
    dw = T.grouped_weight_grad(whole((8, 32), g).to("cuda", t), x.to("cuda", t).expand(8, 48), i32([8]))
    assert dw.shape == (1, 32, 48)
    none = T.grouped_product(torch.empty(0, 48, device="cuda", dtype=t), w.to("cuda", t), i32([0]))
    assert none.shape == (0, 32)
    empty = T.grouped_weight_grad(torch.empty(0, 32, device="cuda", dtype=t), torch.empty(0, 48, device="cuda", dtype=t), i32([0, 0]))
    assert empty.shape == (2, 32, 48) and not empty.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite_stays_in_its_row_and_its_expert(dtype):
    """A row with NaN or infinity spoils its own results and its expert's gradient; a matrix with one spoils its expert's rows; what lies
    behind the last group spoils nothing."""
    from paper_2603_19289_amd import training as T
    g, t, ends, rows = rng(8), TYPES[dtype], [40, 70, 140], 150
    x, dy, w = (whole(s, g) for s in ((rows, 72), (rows, 88), (3, 88, 72)))
    x[50, 71], x[145:], dy[145:] = float("nan"), float("inf"), float("nan")
    w[2, 5, 5] = float("inf")
    on = lambda v: v.to("cuda", t)  # noqa: E731
    y = T.grouped_product(on(x), on(w), i32(ends)).cpu()
    clean = x.clone()
    clean[50, 71] = clean[145:] = 0.0
    want = product(clean, torch.nan_to_num(w, posinf=0.0), ends, False).to(t)
    assert y[50].isnan().all() and not y[140:].any()
    keep = torch.ones(rows, 88, dtype=torch.bool)
    keep[50], keep[70:140, 5] = False, False
    assert torch.equal(y[keep], want[keep]) and not y[70:140, 5].isfinite().any()
    dw = T.grouped_weight_grad(on(dy), on(x), i32(ends)).cpu()
    want = weight_grad(dy, clean, ends).to(t)
    assert dw[1][:, 71].isnan().all()
    dw[1, :, 71] = want[1, :, 71] = 0.0
    assert torch.equal(dw, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_beyond_32_bits(dtype):
    from paper_2603_19289_amd import training as T
    g, t = rng(2), TYPES[dtype]
    far = (1 << 32) + 64
    store = torch.empty(far + 64 * 64, dtype=t, device="cuda")
    w = torch.as_strided(store, (2, 32, 64), (far, 64, 1))
    x, dy, values = whole((40, 64), g), whole((40, 32), g), whole((2, 32, 64), g)
    w.copy_(values)
    ends = [17, 40]
    assert torch.equal(T.grouped_product(x.to("cuda", t), w, i32(ends)).cpu(), product(x, values, ends, False).to(t))
    assert torch.equal(T.grouped_product(dy.to("cuda", t), w, i32(ends), transpose=True).cpu(), product(dy, values, ends, True).to(t))
    assert torch.equal(T.grouped_weight_grad(dy.to("cuda", t), x.to("cuda", t), i32(ends), out=w).cpu(), weight_grad(dy, x, ends).to(t))
    rows = torch.as_strided(store, (3, 64), ((1 << 31), 1))
    rows.copy_(x[:3])
    assert torch.equal(T.grouped_product(rows, values.to("cuda", t), i32([1, 3])).cpu(), product(x[:3], values, [1, 3], False).to(t))


# ------------------------------------------------------------------------------------------------ gated activation
def gated_reference(a, weight):
    gate, up = a.double().chunk(2, dim=1)
    s = torch.sigmoid(gate)
    w = torch.ones(a.shape[0], 1, dtype=torch.float64) if weight is None else weight.double()[:, None]
    return gate, up, s, w


SHAPES = [(1, 1), (3, 5), (8, 768), (33, 64), (7, 129), (5, 128), (40, 2048), (9, 2049), (2, 5000), (300, 24), (17, 721)]


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_swiglu(rows, cols, dtype, weighted):
    """The sigmoid: its argument's rounding counts |g| u (twice, with the constant's), an exponential within 2 u, a sum, a reciprocal or
    division within 2 u: (2 |g| + 6) u of it.  Three more products: (2 |g| + 10) u."""
    from paper_2603_19289_amd import training as T
    g, t = rng(rows * 1009 + cols), TYPES[dtype]
    a = (2.0 * torch.randn(rows, 2 * cols, generator=g)).to(t)
    dh = torch.randn(rows, cols, generator=g).to(t)
    weight = torch.rand(rows, generator=g) if weighted else None
    on = lambda v: None if v is None else v.to("cuda")  # noqa: E731
    gate, up, s, w = gated_reference(a, weight)
    off = (2 * gate.abs() + 10) * U
    h = w * gate * s * up
    out = half(t)
    close(T.swiglu_forward(on(a), on(weight)), h, (off + out) * h.abs() * 1.001, "h")
    da, dw = T.swiglu_backward(on(dh), on(a), on(weight))
    d = dh.double()
    want_up, act = d * w * gate * s, gate * s
    slope = 1.0 + gate * (1.0 - s)
    want_gate = d * w * up * s * slope
    off_slope = gate.abs() * (s * off + 2 * U) + 2 * U * (1 + slope.abs())
    off_gate = (d * w * up * s).abs() * off_slope + off * want_gate.abs()
    close(da, torch.cat([want_gate, want_up], 1), torch.cat([off_gate * (1 + out) + out * want_gate.abs(), (off + out) * want_up.abs() * 1.001], 1), "da")
    if not weighted:
        assert dw is None
        return
    terms = d * act * up
    close(dw, terms.sum(1), ((off + (cols / 8 + 16) * U) * terms.abs()).sum(1), "dweight")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_swiglu_far_values_and_strides(dtype):
    """Gates far from zero give what the limits are; rows may lie apart, begin at odd addresses or be one for all."""
    from paper_2603_19289_amd import training as T
    t = TYPES[dtype]
    a = torch.tensor([[-1000.0, 1000.0, -88.0, 88.0, 0.0, -0.0, 30.0, -30.0, 1.5, 2.0, 1.0, 1.0, 3.0, 5.0, 1.0, 1.0]], dtype=t)
    gate, up, s, _ = gated_reference(a, None)
    h = T.swiglu_forward(a.to("cuda"))
    close(h, gate * s * up, (half(t) + 300 * U) * (gate * s * up).abs() + 1e-36, "h")
    da, _ = T.swiglu_backward(torch.ones(1, 8, dtype=t, device="cuda"), a.to("cuda"))
    want = torch.cat([up * s * (1 + gate * (1 - s)), gate * s], 1)
    close(da, want, (half(t) + 3000 * U) * want.abs() + 1e-33, "da")
    g = rng(4)
    wide = torch.randn(30, 47, generator=g).to("cuda", t)
    part = wide[:, 3:3 + 26]
    assert torch.equal(T.swiglu_forward(part), T.swiglu_forward(part.contiguous()))
    assert torch.equal(T.swiglu_backward(wide[:, 1:14], part)[0], T.swiglu_backward(wide[:, 1:14].contiguous(), part.contiguous())[0])
    one = part[:1].expand(30, 26)
    assert torch.equal(T.swiglu_forward(one), T.swiglu_forward(one.contiguous()))
    assert T.swiglu_forward(part[:0]).shape == (0, 13)


def test_swiglu_gradients_against_differences():
    """Central differences in 64 bits of the formula, step 1e-4: their own error is of the order of 1e-8 of third derivatives below 10."""
    from paper_2603_19289_amd import training as T
    g = rng(6)
    a, dh, w = torch.randn(3, 20, generator=g), torch.randn(3, 10, generator=g), torch.rand(3, generator=g)
    da, dw = (v.cpu().double() for v in T.swiglu_backward(dh.cuda(), a.cuda(), w.cuda()))

    def f(a, w):
        gate, up, s, v = gated_reference(a, w)
        return (v * gate * s * up * dh.double()).sum()
    for r in range(3):
        for c in range(20):
            step = torch.zeros(3, 20, dtype=torch.float64)
            step[r, c] = 1e-4
            assert abs((f(a.double() + step, w) - f(a.double() - step, w)) / 2e-4 - da[r, c]) < 1e-5
        step = torch.zeros(3, dtype=torch.float64)
        step[r] = 1e-4
        assert abs((f(a.double(), w.double() + step) - f(a.double(), w.double() - step)) / 2e-4 - dw[r]) < 1e-5


def test_rows_beyond_32_bits_of_offset():
    from paper_2603_19289_amd import training as T
    store = torch.empty((1 << 32) + 64, dtype=torch.bfloat16, device="cuda")
    a = torch.as_strided(store, (3, 32), (1 << 31, 1))
    a.copy_(torch.randn(3, 32, generator=rng(1)))
    assert torch.equal(T.swiglu_forward(a), T.swiglu_forward(a.contiguous()))


# ------------------------------------------------------------------------------------------------ orthogonalised updates
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
H = 2.0 ** -11                                           # half a step of float16, which holds X, A and B


def orthogonal(g, iterations=5, coefficients=COEFFICIENTS):
    """The iteration in 64 bits, and how far (Frobenius norm) roundings of X, A and B to float16 can take its result.  An error of X grows
    with the function of the singular values that a step is: by at most its steepest slope, or its largest ratio to its argument.  Sums in
    float add 2 u a term, taken as a fifth of a half step each; a thousandth of X for what is of second order."""
    a, b, c = coefficients
    x = g.double()
    x = x.t() if x.shape[0] > x.shape[1] else x
    norm = x.norm()
    if norm == 0:
        return g.double(), 0.0
    x = x / norm
    err = H
    for _ in range(iterations):
        sigma = torch.linalg.svdvals(x)
        grid = torch.linspace(max(0.0, sigma.min().item() - err), sigma.max().item() + err, 4000, dtype=torch.float64)
        steep = torch.maximum((a + 3 * b * grid ** 2 + 5 * c * grid ** 4).abs(), (a + b * grid ** 2 + c * grid ** 4).abs()).max().item()
        q = x @ x.t()
        poly = a * torch.eye(len(q), dtype=torch.float64) + b * q + c * q @ q
        top = sigma.max().item()
        new = poly @ x
        rounding = (abs(b) + 2 * abs(c) * top ** 2) * q.norm().item() * top + poly.norm().item() * top + new.norm().item()
        err = steep * err + 1.2 * H * rounding
        x = new
    x = x.t() if g.shape[0] > g.shape[1] else x
    return x, err * 1.1 + 1e-3 * x.norm().item()


def well(m, n, seed, low=0.3):
    """A matrix with singular values between `low` and one."""
    g = rng(seed)
    k = min(m, n)
    u, v = (torch.linalg.qr(torch.randn(d, k, generator=g, dtype=torch.float64))[0] for d in (m, n))
    return ((u * torch.linspace(low, 1.0, k, dtype=torch.float64)) @ v.t()).float()


# about where matrices become too large for one workgroup, and others
MATRICES = [(64, 256), (257, 64), (48, 455), (48, 456), (33, 455), (32, 764), (32, 765), (20, 768), (16, 1533), (64, 380), (64, 381), (380, 64), (65, 65), (16, 1532), (1540, 16), (17, 700), (40, 508), (48, 509), (3, 1530), (1, 1533), (1, 1), (1, 9), (9, 1), (2, 3), (8, 8), (5, 64), (64, 5), (33, 70), (70, 33), (128, 128), (130, 257), (300, 129), (256, 520), (100, 2000), (1030, 72)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", MATRICES)
def test_orthogonalise(m, n, dtype):
    from paper_2603_19289_amd import training as T
    g = (well(m, n, m * 3001 + n) * 0.02).to(TYPES[dtype])
    got = T.orthogonalise(g.to("cuda"))
    assert got.dtype == torch.bfloat16 and got.shape == g.shape
    want, err = orthogonal(g)
    off = (got.cpu().double() - want).norm().item()
    assert off <= err + half(torch.bfloat16) * want.norm().item(), (off, err, want.norm().item())
    s = torch.linalg.svdvals(got.cpu().double())
    assert s.min() > 0.6 and s.max() < 1.3
    one, err = orthogonal(g, 1)
    assert (T.orthogonalise(g.to("cuda"), iterations=1).cpu().double() - one).norm().item() <= err + half(torch.bfloat16) * one.norm().item()


def test_orthogonalise_stacks_strides_and_scales():
    """Each matrix of a stack by itself, whatever its scale; zeros stay zeros; what is not finite makes its own matrix NaN; strided input
    and output; iterations and coefficients of the caller's."""
    from paper_2603_19289_amd import training as T
    base = torch.stack([well(40, 72, s) for s in range(6)])
    alone = torch.stack([T.orthogonalise(m.to("cuda")) for m in base])
    scaled = base.clone()
    scaled[0] *= 2.0 ** -60
    scaled[1] *= 2.0 ** -115
    scaled[2] *= 2.0 ** 100
    first = got = T.orthogonalise(scaled.to("cuda"))
    # powers of two change nothing, where the values have them: times 2^-115 those below 2^-11 are denormal and have lost bits before
    # the call, so that matrix is another one and goes by its own bound
    for i in (0, 2, 3, 4, 5):
        assert torch.equal(got[i], alone[i]), i
    want, err = orthogonal(scaled[1])
    assert (got[1].cpu().double() - want).norm().item() <= err + half(torch.bfloat16) * want.norm().item()
    scaled[3] = 0.0
    scaled[4, 3, 7] = float("inf")
    scaled[5, 39, 71] = float("nan")
    got = T.orthogonalise(scaled.to("cuda"))
    assert torch.equal(got[:3], first[:3]) and not got[3].any() and got[4:].isnan().all()
    store = torch.full((6, 50, 90), 8.0, device="cuda")
    store[:, 5:45, 7:79] = base.to("cuda")
    out = torch.full((6, 45, 100), 4.0, device="cuda", dtype=torch.bfloat16)
    T.orthogonalise(store[:, 5:45, 7:79], out=out[:, 2:42, 9:81])
    assert torch.equal(out[:, 2:42, 9:81], alone)
    out[:, 2:42, 9:81] = 4.0
    assert torch.all(out == 4.0)
    tall = T.orthogonalise(base.transpose(1, 2).contiguous().to("cuda"))
    assert torch.equal(tall.transpose(1, 2), alone)
    want, err = orthogonal(base[0], 3, (1.5, -0.5, 0.0))
    got = T.orthogonalise(base[0].to("cuda"), iterations=3, coefficients=(1.5, -0.5, 0.0))
    assert (got.cpu().double() - want).norm().item() <= err + half(torch.bfloat16) * want.norm().item()
    for shape in ((0, 5, 5), (3, 0, 4), (2, 4, 0), (0, 0)):
        assert T.orthogonalise(torch.empty(shape, device="cuda")).shape == shape


def test_denormal_matrices_are_orthogonalised_too():
    from paper_2603_19289_amd import training as T
    g = torch.zeros(8, 8)
    g[range(8), range(8)] = 2.0 ** -140
    got = T.orthogonalise(g.to("cuda"))
    want, err = orthogonal(g)
    assert (got.cpu().double() - want).norm().item() <= err + half(torch.bfloat16) * want.norm().item()


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_muon_steps(grad, nesterov):
    """Three steps of matrices and stacks, wide and upright.  Momenta are the float formula's bit for bit; parameters are off by the
    update's own bound and three roundings; copies are the parameters rounded."""
    from paper_2603_19289_amd import training as T
    shapes = [(40, 24), (3, 16, 33), (2, 50, 20), (7, 7)]
    lr, mu, decay, rms = 0.01, 0.9, 0.1, 0.2
    flat = lambda s: well(s[-2], s[-1], sum(s)) if len(s) == 2 else torch.stack([well(s[1], s[2], i + sum(s)) for i in range(s[0])])  # noqa: E731
    p = [(torch.randn(s, generator=rng(i)) * 0.1).cuda() for i, s in enumerate(shapes)]
    copies = [torch.zeros_like(t, dtype=torch.bfloat16) if i != 1 else None for i, t in enumerate(p)]
    opt = T.Muon(p, lr=lr, momentum=mu, nesterov=nesterov, weight_decay=decay, update_rms=rms, copies=copies)
    m = [torch.zeros(s) for s in shapes]
    for step in range(3):
        before = [t.cpu().clone() for t in p]
        versions = [t._version for t in p]
        g = [flat(s).mul(0.5 + step).to(TYPES[grad]) for s in shapes]
        opt.step([t.cuda() for t in g], grad_scale=0.5)
        for i, s in enumerate(shapes):
            scaled = g[i].float() * 0.5
            m[i] = m[i] * mu + scaled
            assert torch.equal(opt.states()["m"][i].cpu(), m[i]), (step, s)
            u = scaled + m[i] * mu if nesterov else m[i]
            assert p[i]._version > versions[i]
            rate = lr * rms * math.sqrt(max(s[-2:]))
            for q, v, w in zip(p[i].cpu().view(-1, *s[-2:]), u.view(-1, *s[-2:]), before[i].view(-1, *s[-2:])):
                o, err = orthogonal(v)
                want = w.double() * (1 - lr * decay) - rate * o
                assert (q.double() - want).norm().item() <= rate * err + 4 * U * (w.double().norm().item() + rate * o.norm().item()), (step, s)
            if copies[i] is not None:
                assert torch.equal(copies[i], p[i].to(torch.bfloat16))


@pytest.mark.parametrize("rows,cols", [(24, 40), (72, 130), (130, 72)])
def test_muon_copies_into_expert_blocks(rows, cols):
    from paper_2603_19289_amd import training as T
    blocks = torch.full((4, 3 * rows * cols + 5), 6.0, dtype=torch.bfloat16, device="cuda")
    part = blocks[:, rows * cols:2 * rows * cols].unflatten(1, (rows, cols))
    p = torch.randn(4, rows, cols, device="cuda")
    T.Muon([p], lr=0.1, copies=[part]).step([torch.randn(4, rows, cols, device="cuda")])
    assert torch.equal(part, p.to(torch.bfloat16))
    part.fill_(6.0)
    assert torch.all(blocks == 6.0)
    with pytest.raises(ValueError):
        T.Muon([p], lr=0.1, copies=[torch.zeros(4, cols, rows, dtype=torch.bfloat16, device="cuda").transpose(1, 2)])


@pytest.mark.parametrize("shape", [(300, 200), (20, 70, 130), (9, 130, 66), (5, 777, 1111), (5, 1111, 777), (3, 1500, 1030)], ids=str)
def test_muon_of_larger_matrices(shape):
    """Every size of tile, wide and upright: parameters go by what orthogonalise returns, which is off from the update by one rounding to bfloat16;
    a matrix of a stack gets what it gets by itself; copies are the parameters rounded."""
    from paper_2603_19289_amd import training as T
    g = torch.randn(shape, generator=rng(1)).cuda()
    p = torch.randn(shape, generator=rng(2)).cuda() * 0.1
    before, copy = p.double(), torch.zeros(shape, device="cuda", dtype=torch.bfloat16)
    lr, decay, rms = 0.1, 0.3, 0.2
    T.Muon([p], lr=lr, momentum=0.0, nesterov=False, weight_decay=decay, update_rms=rms, copies=[copy]).step([g])
    o = T.orthogonalise(g)
    for i in range(shape[0] if len(shape) == 3 else 0):
        assert torch.equal(T.orthogonalise(g[i]), o[i]), i
    rate, o = lr * rms * math.sqrt(max(shape[-2:])), o.double()
    bound = rate * o.abs() * half(torch.bfloat16) / (1 - half(torch.bfloat16)) + 4 * U * (before.abs() + rate * o.abs())
    close(p, (before * (1 - lr * decay) - rate * o).cpu(), bound.cpu(), shape)
    assert torch.equal(copy, p.to(torch.bfloat16))


def test_muon_leaves_out_parameters_without_gradient():
    from paper_2603_19289_amd import training as T
    p = [torch.randn(8, 16, device="cuda") for _ in range(3)]
    before = [t.clone() for t in p]
    opt = T.Muon(p, lr=0.1)
    versions = [t._version for t in p]
    opt.step([None, torch.randn(8, 16, device="cuda"), None])
    assert torch.equal(p[0], before[0]) and torch.equal(p[2], before[2]) and not torch.equal(p[1], before[1])
    assert [t._version > v for t, v in zip(p, versions)] == [False, True, False]
    opt.step([None] * 3)
    scale = torch.tensor(0.0, device="cuda")
    opt.step([None, torch.full((8, 16), float("nan"), device="cuda"), None], grad_scale=1.0)
    assert p[1].isnan().all() and torch.equal(p[0], before[0])
    opt.step([torch.randn(8, 16, device="cuda"), None, None], grad_scale=scale)       # nothing to go by: only the decay
    assert torch.equal(p[0], before[0] * torch.tensor(1.0 - 0.1 * 0.01, device="cuda"))


def test_muon_of_small_and_large_matrices_together():
    """In one call, with and without a gradient here and there: the same bits as each by itself."""
    from paper_2603_19289_amd import training as T
    shapes = [(70, 90), (3, 20, 30), (64, 381), (8, 8), (2, 64, 380), (5, 100, 66)]
    make = lambda s, seed: torch.stack([well(s[-2], s[-1], seed + i) for i in range(s[0])]) if len(s) == 3 else well(*s, seed)  # noqa: E731
    g = [make(s, 10 * i).cuda() for i, s in enumerate(shapes)]
    p = [torch.randn(s, generator=rng(i)).cuda() for i, s in enumerate(shapes)]
    alone = [t.clone() for t in p]
    T.Muon(p, lr=0.1).step([t if i != 3 else None for i, t in enumerate(g)])
    for i, t in enumerate(alone):
        if i != 3:
            T.Muon([t], lr=0.1).step([g[i]])
        assert torch.equal(p[i], t), i


def test_muon_of_more_stacks_than_one_launch_takes():
    from paper_2603_19289_amd import training as T
    shapes = [(3 + i % 7, 5 + i % 11) for i in range(61)]
    g = [well(*s, seed=i) for i, s in enumerate(shapes)]
    p = [torch.zeros(s, device="cuda") for s in shapes]
    T.Muon(p, lr=1.0, weight_decay=0.0, momentum=0.0, nesterov=False, update_rms=1.0).step([t.cuda() for t in g])
    for t, s, v in zip(p, shapes, g):
        want, err = orthogonal(v)
        assert (t.cpu().double() + want * math.sqrt(max(s))).norm().item() <= math.sqrt(max(s)) * (err + 4 * U * want.norm().item())


# ------------------------------------------------------------------------------------------------ together
def experts_pass(x, ids, gates, w_in, w_out, dout):
    """A layer's experts forward and backward, as a training step runs them."""
    from paper_2603_19289_amd import training as T
    tokens, k = ids.shape
    order = torch.sort(ids.flatten(), stable=True).indices
    ends = torch.cumsum(torch.bincount(ids.flatten(), minlength=w_in.shape[0]), 0).to(torch.int32)
    token = order // k
    rows, gate = x[token], gates.flatten()[order]
    a = T.grouped_product(rows, w_in, ends)
    h = T.swiglu_forward(a, gate)
    y = T.grouped_product(h, w_out, ends)
    out = torch.zeros(tokens, x.shape[1], device=x.device).index_add_(0, token, y.float())
    dy = dout.to(x.dtype)[token]
    dw_out = T.grouped_weight_grad(dy, h, ends, dtype=torch.float32)
    da, dgate = T.swiglu_backward(T.grouped_product(dy, w_out, ends, transpose=True), a, gate)
    dw_in = T.grouped_weight_grad(da, rows, ends, dtype=torch.float32)
    dx = torch.zeros(tokens, x.shape[1], device=x.device).index_add_(0, token, T.grouped_product(da, w_in, ends, transpose=True).float())
    dgates = torch.zeros(tokens * k, device=x.device).index_copy_(0, order, dgate).view(tokens, k)
    return out, dx, dgates, dw_in, dw_out


def experts_reference(x, ids, gates, w_in, w_out, dout):
    x, gates, w_in, w_out = (t.detach().cpu().double().requires_grad_() for t in (x, gates, w_in, w_out))
    ids = ids.cpu()
    parts = []
    for t in range(x.shape[0]):
        y = 0.0
        for j, e in enumerate(ids[t].tolist()):
            gate, up = (w_in[e] @ x[t]).chunk(2)
            y = y + gates[t, j] * (w_out[e] @ (torch.nn.functional.silu(gate) * up))
        parts.append(y)
    out = torch.stack(parts)
    return (out.detach(), *torch.autograd.grad(out, (x, gates, w_in, w_out), dout.cpu().double()))


def layer_inputs(tokens, experts, k, hidden, inter, dtype, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    t = TYPES[dtype]
    ids = torch.rand(tokens, experts, generator=g, device="cuda").topk(k, dim=1).indices.to(torch.int32)
    gates = torch.softmax(rand(tokens, k), 1)
    return ((rand(tokens, hidden)).to(t), ids, gates, (rand(experts, 2 * inter, hidden) * hidden ** -0.5).to(t),
            (rand(experts, hidden, inter) * inter ** -0.5).to(t), rand(tokens, hidden).to(t).float())


@pytest.mark.parametrize("dtype,tokens,experts,k,hidden,inter", [("f32", 21, 6, 2, 40, 24), ("bf16", 21, 6, 2, 40, 24), ("f32", 64, 8, 4, 64, 33), ("bf16", 50, 12, 3, 128, 64)])
def test_a_layers_experts_forward_and_backward(dtype, tokens, experts, k, hidden, inter):
    """All of them together, against the layer's own formula and its gradients in 64 bits.  In bfloat16 each of up to seven values between
    inputs and a result is rounded, each by half a step at most: with values that add up at random the whole is off by that much of its norm."""
    args = layer_inputs(tokens, experts, k, hidden, inter, dtype)
    got, want = experts_pass(*args), experts_reference(*args)
    limit = 7 * half(torch.bfloat16) if dtype == "bf16" else 200 * U
    for name, a, b in zip(("out", "dx", "dgates", "dw_in", "dw_out"), got, want):
        assert (a.cpu().double() - b).norm() <= limit * b.norm(), (name, ((a.cpu().double() - b).norm() / b.norm()).item())


def test_training_steps_captured_and_replayed():
    """Forward, backward and Muon in a graph, replayed with other inputs and other groups in place, eager work between: the same bits."""
    from paper_2603_19289_amd import training as T
    tokens, experts, k, hidden, inter = 48, 10, 3, 72, 40
    x, ids, gates, w_in, w_out, dout = layer_inputs(tokens, experts, k, hidden, inter, "bf16")
    rows = tokens * k

    def new():
        masters = [w_in.float().clone(), w_out.float().clone()]
        copies = [w_in.clone(), w_out.clone()]
        return masters, copies, T.Muon(masters, lr=0.02, copies=copies)

    def step(rows_in, gate, ends, dy, copies, opt):
        a = T.grouped_product(rows_in, copies[0], ends)
        h = T.swiglu_forward(a, gate)
        y = T.grouped_product(h, copies[1], ends)
        da, dgate = T.swiglu_backward(T.grouped_product(dy, copies[1], ends, transpose=True), a, gate)
        opt.step([T.grouped_weight_grad(da, rows_in, ends), T.grouped_weight_grad(dy, h, ends)])
        return y, dgate

    def inputs(seed):
        x, ids, gates, _, _, dout = layer_inputs(tokens, experts, k, hidden, inter, "bf16", seed)
        ids = (ids % (1 + seed % experts)).to(torch.int32)                # other groups, many of them empty
        order = torch.sort(ids.flatten(), stable=True).indices
        ends = torch.cumsum(torch.bincount(ids.flatten(), minlength=experts), 0).to(torch.int32)
        return x[order // k], gates.flatten()[order], ends, dout.to(torch.bfloat16)[order // k]

    held = [t.clone() for t in inputs(0)]
    masters, copies, opt = new()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*held, copies, opt)                                          # memory is asked for once before the capture
    torch.cuda.current_stream().wait_stream(side)
    masters, copies, opt = new()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        result = step(*held, copies, opt)
    eager_masters, eager_copies, eager = new()
    for seed in (1, 2, 3, 7, 9):
        fresh = inputs(seed)
        for a, b in zip(held, fresh):
            a.copy_(b)
        graph.replay()
        want = step(*fresh, eager_copies, eager)
        torch.cuda.synchronize()
        assert rows == held[0].shape[0]
        for a, b in zip((*result, *masters, *copies, *opt.states()["m"]), (*want, *eager_masters, *eager_copies, *eager.states()["m"])):
            assert torch.equal(a, b), seed


def test_streams_and_equal_bits():
    """Two calls at once on two streams, each with its own memory, and the same again: equal bits."""
    from paper_2603_19289_amd import training as T
    x, ids, gates, w_in, w_out, dout = layer_inputs(200, 8, 2, 256, 96, "bf16")
    g = [well(120, 200, s).cuda() for s in range(2)]
    want = [t.clone() for t in experts_pass(x, ids, gates, w_in, w_out, dout)], [T.orthogonalise(m) for m in g]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for s, m in zip(streams, g):
            with torch.cuda.stream(s):
                got.append((experts_pass(x, ids, gates, w_in, w_out, dout), T.orthogonalise(m)))
        torch.cuda.synchronize()
        for (layer, o), q in zip(got, want[1]):
            assert torch.equal(o, q)
            for a, b, name in zip(layer, want[0], ("out", "dx", "dgates", "dw_in", "dw_out")):
                if name not in ("out", "dx"):            # torch's index_add_ adds in any order
                    assert torch.equal(a, b), name
