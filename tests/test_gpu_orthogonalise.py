"""The orthogonalised update against the same iteration in 64 bits.

One step, element by element.  A plane pair keeps v to RHO = 2^-22 |v| (two roundings to 11 bits) or to half a step of the smallest
half-precision number, 2^-25, over the planes' scale, which is at least 2^13 over the bound of what it holds: 2^-38 of the bound.  A product of two
plane pairs over an inner dimension K leaves lo lo out, 2^-22 |A||B|, and makes at most 3 K + 4 additions that lose 2^-23 of a partial sum of at
most |A||B| each: kappa(K) = 2^-22 + (3 K + 4) 2^-23.  FP32 operations of the epilogue: 2^-24 each.  Errors propagate linearly
through S = X X^T, P = b S + c S S, a X + P X (step_bound); second-order terms are within the 2 percent added.

Several steps.  Every step is taken to perturb X by at most 2^-20 of the largest singular value times max(1, |a| + |b| + |c|) in the 2-norm (roundings
are of independent sign), and a perturbation grows by at most the largest |p'| in each step that follows, p being odd."""
import pytest
import torch

import paper_2609_09095_b200 as oz

pytestmark = pytest.mark.gpu

TYPE = {torch.bfloat16: oz.OZ_BF16, torch.float16: oz.OZ_F16, torch.float32: oz.OZ_F32}
USUAL = (3.4445, -4.7750, 2.0315)
RHO, U24 = 2.0 ** -22, 2.0 ** -24


def update(g, out_dtype=torch.float32, steps=5, coefficients=USUAL, eps=1e-7, out=None, stream=None, workspace=None):
    """g (count, rows, cols), any strides with unit last one"""
    count, rows, cols = g.shape
    out = torch.full((count, rows, cols), 7.0, dtype=out_dtype, device="cuda") if out is None else out
    need = oz.oz_orthogonalise_workspace_bytes(cols, rows, count)
    workspace = torch.full((need,), 0xAA, dtype=torch.uint8, device="cuda") if workspace is None else workspace
    oz.check(oz.oz_orthogonalise(cols, rows, count, TYPE[g.dtype], g, g.stride(1), g.stride(0), steps, coefficients, eps, TYPE[out.dtype], out,
                                 out.stride(1), out.stride(0), workspace, need, stream), "oz_orthogonalise")
    return out


def normalised(g, eps):
    x = g.double()
    return x / (x.square().sum().sqrt() + eps)


def iterate(x, steps, abc):
    a, b, c = abc
    if x.shape[0] > x.shape[1]:
        return iterate(x.T, steps, abc).T
    for _ in range(steps):
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return x


def kappa(K):
    return RHO + (3 * K + 4) * 2.0 ** -23


def step_bound(x, abc):
    """x: the exact X, r <= c"""
    a, b, c = (abs(v) for v in abc)
    r, n = x.shape
    ax = x.abs()
    ex = (RHO + U24) * ax + 2.0 ** -38
    s = x @ x.T
    asz = ax @ ax.T
    es = ex @ ax.T + ax @ ex.T + kappa(n) * asz
    es = es + RHO * s.abs() + 2.0 ** -38
    ps = b * s.abs() + c * (s.abs() @ s.abs())
    ep = b * es + c * (es @ s.abs() + s.abs() @ es + kappa(r) * (s.abs() @ s.abs())) + 4 * U24 * ps
    top = max(b + c, 2.0 ** -40)
    ep = ep + RHO * ps + 2.0 ** -38 * top
    return 1.02 * (a * ex + ep @ ax + ps @ ex + kappa(r) * (ps @ ax) + 4 * U24 * (a * ax + ps @ ax))


def check_one_step(g, abc, eps=1e-7, out_dtype=torch.float32):
    got = update(g[None], out_dtype, 1, abc, eps)[0]
    x = normalised(g, eps)
    exact = iterate(x, 1, abc)
    e = step_bound(x, abc) if x.shape[0] <= x.shape[1] else step_bound(x.T, abc).T
    tol = e + (exact.abs() + e) * torch.finfo(out_dtype).eps / 2 + (2.0 ** -25 if out_dtype == torch.float16 else 0.0)
    off = (got.double() - exact).abs()
    assert (off <= tol).all(), f"{float((off / tol).max())} tolerances"


def tensor(*shape, seed, dtype=torch.float32, scale=1.0):
    return (scale * torch.randn(*shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))).to(dtype)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 9), (7, 1), (8, 16), (16, 8), (33, 40), (64, 64), (129, 127), (127, 300), (257, 130), (130, 1000)])
@pytest.mark.parametrize("abc", [(1.0, 0.0, 0.0), (0.0, 1.0, 0.0), (0.0, 0.0, 1.0), USUAL, (1.5, -0.5, 0.0)])
def test_one_step(rows, cols, abc):
    check_one_step(tensor(rows, cols, seed=1), abc)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_types(dtype, out_dtype):
    check_one_step(tensor(70, 90, seed=2, dtype=dtype), USUAL, out_dtype=out_dtype)
    check_one_step(tensor(90, 70, seed=3, dtype=dtype), USUAL, out_dtype=out_dtype)


def test_planes_keep_22_bits():
    """|G| + eps a power of two: X is G shifted.  Integers of 21 bits pass the step (1, 0, 0) and no step at all unchanged."""
    gen = torch.Generator("cuda").manual_seed(4)
    for rows, cols in ((24, 40), (40, 24), (130, 70)):
        g = torch.randint(-(1 << 21) + 1, 1 << 21, (rows, cols), device="cuda", generator=gen).float()
        norm = g.double().square().sum().sqrt().item()
        power = 2.0 ** 40
        for steps in (0, 1):
            got = update(g[None], steps=steps, coefficients=(1.0, 0.0, 0.0), eps=power - norm)[0]
            # 2^-40 of the bound is 2^-40 of the range: integers over 2^40 with 15 bits to spare below
            exact = g.double() / power
            assert ((got.double() - exact).abs() <= 2.0 ** -39 * (1 if steps else 0) + 0.0).all()
        power = 2.0 ** torch.tensor(norm).log2().ceil().item()
        got = update(g[None], steps=1, coefficients=(1.0, 0.0, 0.0), eps=power - norm)[0]
        assert torch.equal(got.double(), g.double() / power)


def spread_bound(steps, abc, largest):
    a, b, c = abc
    s = torch.linspace(0, largest, 2001, dtype=torch.float64)
    slope = (a + 3 * b * s ** 2 + 5 * c * s ** 4).abs().max().item()
    each = 2.0 ** -20 * largest * max(1.0, abs(a) + abs(b) + abs(c))
    return each * sum(slope ** t for t in range(steps))


@pytest.mark.parametrize("count,rows,cols", [(1, 128, 512), (3, 200, 77), (2, 1009, 517), (5, 64, 64), (1, 520, 1544), (1, 2100, 2056), (40, 96, 200), (12, 520, 520)])
@pytest.mark.parametrize("dtype,out_dtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16)])
def test_five_steps(count, rows, cols, dtype, out_dtype):
    g = tensor(count, rows, cols, seed=5, dtype=dtype, scale=1e-3)
    got = update(g, out_dtype)
    assert oz.oz_query_status() in (oz.OZ_OK, oz.OZ_ERR_RANGE)
    for i in range(count):
        exact = iterate(normalised(g[i], 1e-7), 5, USUAL)
        off = (got[i].double() - exact).norm()
        # a perturbation of 2-norm d has a Frobenius norm of at most sqrt(r) d
        tol = min(rows, cols) ** 0.5 * spread_bound(5, USUAL, 1.3) + (exact.norm() * torch.finfo(out_dtype).eps / 2)
        assert off <= tol, (i, float(off / tol))
        # held against the usual FP32 iteration too: no further off than 4 of its errors and the rounding
        plain = iterate_f32(g[i])
        assert off <= 4 * (plain.double() - exact).norm() + 2 * exact.norm() * (torch.finfo(out_dtype).eps / 2), i


def iterate_f32(g):
    a, b, c = USUAL
    x = g.float()
    x = x.T if g.shape[0] > g.shape[1] else x
    x = x / (x.square().sum().sqrt() + 1e-7)
    for _ in range(5):
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.T if g.shape[0] > g.shape[1] else x


def test_extremes():
    # zeros, with and without eps; one element; a matrix of rank one; huge and tiny numbers
    z = torch.zeros(2, 5, 9, device="cuda")
    for eps in (0.0, 1e-7):
        assert not update(z, eps=eps).any()
    x = 1.0
    for _ in range(5):
        x = USUAL[0] * x + USUAL[1] * x ** 3 + USUAL[2] * x ** 5
    one = update(torch.full((1, 1, 1), -3.0, device="cuda"), eps=0.0)
    assert abs(one.item() + x) <= spread_bound(5, USUAL, 1.3)
    for scale in (1e37, 1e-37, 1e-44):
        g = tensor(1, 40, 30, seed=6) * scale
        exact = iterate(normalised(g[0], 0.0), 5, USUAL)
        off = (update(g, eps=0.0)[0].double() - exact).norm()
        assert off <= 30 ** 0.5 * spread_bound(5, USUAL, 1.3)
    assert oz.oz_query_status() in (oz.OZ_OK, oz.OZ_ERR_RANGE)


def test_non_finite_stays_in_its_matrix():
    for poison in (float("nan"), float("inf"), float("-inf")):
        g = tensor(3, 50, 60, seed=7)
        g[1, 49, 59] = poison
        for steps in (0, 5):
            got = update(g, steps=steps)
            assert oz.oz_query_status() == oz.OZ_ERR_NONFINITE_INPUT
            assert got[1].isnan().all() and got[0].isfinite().all() and got[2].isfinite().all()
        clean = g.clone()
        clean[1] = 1.0
        assert torch.equal(update(clean)[0], got[0]) and torch.equal(update(clean)[2], got[2])


def test_strides_in_place_and_neighbours():
    count, rows, cols = 2, 45, 70
    flat = tensor(count * 5000 + 3, seed=8)
    g = flat[3:].as_strided((count, rows, cols), (5000, 101, 1))
    held = torch.full((count * 5001 + 1,), 9.0, device="cuda")
    out = held[1:].as_strided((count, rows, cols), (5001, 77, 1))
    before = flat.clone()
    got = update(g, out=out)
    assert torch.equal(flat, before)
    want = update(g.contiguous())
    assert torch.equal(got, want)
    mask = torch.ones_like(held, dtype=torch.bool)
    mask[1:].as_strided((count, rows, cols), (5001, 77, 1))[:] = False
    assert (held[mask] == 9.0).all()
    for steps in (0, 5):
        same = g.contiguous().clone()
        assert torch.equal(update(same, out=same, steps=steps), update(g.contiguous(), steps=steps))


def test_deterministic_graph_and_streams():
    g = [tensor(2, 300, 500, seed=9, dtype=torch.bfloat16), tensor(2, 500, 300, seed=10, dtype=torch.bfloat16)]
    need = oz.oz_orthogonalise_workspace_bytes(500, 300, 2)
    want = [update(x, torch.bfloat16) for x in g]
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in g]
    outs = [torch.zeros_like(x) for x in g]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for x, o, w, s in zip(g, outs, spaces, streams):
            update(x, out=o, workspace=w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    static, out = g[0].clone(), torch.zeros_like(g[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        update(static, out=out, workspace=spaces[0])
    for x in (g[0], g[0].flip(1).contiguous(), g[0]):
        static.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, update(x, torch.bfloat16))


def test_experts_step():
    """The operators as a training step uses them: forward, gradients of inputs and weights, update of all experts' weights."""
    sizes, m, k = [300, 0, 41, 171], 136, 264
    offsets = torch.tensor([0] + sizes).cumsum(0).cuda()
    n, groups = sum(sizes), len(sizes)
    x, w = tensor(n, k, seed=11, dtype=torch.bfloat16), tensor(groups, m, k, seed=12, dtype=torch.bfloat16, scale=k ** -0.5)
    y = torch.zeros(n, m, dtype=torch.bfloat16, device="cuda")
    oz.check(oz.oz_gemm_grouped(1, m, n, k, groups, offsets, oz.OZ_BF16, w, k, m * k, x, k, oz.OZ_BF16, 0.0, y, m))
    dy = (y.float() - 1.0).bfloat16()                       # gradient of sum (y - 1)^2 / 2
    dx, dw = torch.zeros(n, k, dtype=torch.bfloat16, device="cuda"), torch.zeros(groups, m, k, device="cuda")
    oz.check(oz.oz_gemm_grouped(0, k, n, m, groups, offsets, oz.OZ_BF16, w, k, m * k, dy, m, oz.OZ_BF16, 0.0, dx, k))
    oz.check(oz.oz_gemm_grouped_wgrad(k, m, n, groups, offsets, oz.OZ_BF16, x, k, dy, m, oz.OZ_F32, 0.0, dw, k, m * k))
    o = update(dw)
    cuts = offsets.tolist()
    for g, (lo, hi) in enumerate(zip(cuts, cuts[1:])):
        exact_dw = dy[lo:hi].double().T @ x[lo:hi].double()
        exact_dx = dy[lo:hi].double() @ w[g].double()
        size = dy[lo:hi].double().abs().T @ x[lo:hi].double().abs()
        assert ((dw[g].double() - exact_dw).abs() <= (hi - lo + 2) * 2.0 ** -23 * size).all()
        size = dy[lo:hi].double().abs() @ w[g].double().abs()
        assert ((dx[lo:hi].double() - exact_dx).abs() <= (m + 2) * 2.0 ** -23 * size * 1.01 + exact_dx.abs() * 2.0 ** -8).all()
        if hi == lo:
            assert not dw[g].any() and not o[g].any()
        else:
            exact = iterate(normalised(dw[g], 1e-7), 5, USUAL)
            assert (o[g].double() - exact).norm() <= m ** 0.5 * spread_bound(5, USUAL, 1.3) + exact.norm() * U24


@pytest.mark.parametrize("count,rows,cols", [(1, 128, 2048), (1, 2049, 128), (2, 20, 513), (3, 129, 256), (200, 100, 300), (150, 128, 129), (1, 3, 2048), (5, 17, 1100)])
def test_narrow_and_its_borders(count, rows, cols):
    """One launch in shared memory up to 128 x 2048 (513 columns leave the last block of a cluster without any), the general form next to it."""
    g = tensor(count, rows, cols, seed=13)
    got = update(g)
    assert oz.oz_query_status() in (oz.OZ_OK, oz.OZ_ERR_RANGE)
    for i in range(0, count, 37):
        exact = iterate(normalised(g[i], 1e-7), 5, USUAL)
        off = (got[i].double() - exact).norm()
        assert off <= min(rows, cols) ** 0.5 * spread_bound(5, USUAL, 1.3) + exact.norm() * U24
        assert off <= 4 * (iterate_f32(g[i]).double() - exact).norm() + 2 * exact.norm() * U24


@pytest.mark.parametrize("rows,cols", [(300, 260), (260, 300), (700, 150)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_general_in_place_and_strided(rows, cols, dtype):
    g = tensor(2, rows, cols, seed=14, dtype=dtype)
    want = update(g, dtype)
    same = g.clone()
    assert torch.equal(update(same, out=same), want)
    held = torch.full((2 * rows * (cols + 3) + 1,), 5.0, dtype=dtype, device="cuda")
    out = held[1:].as_strided((2, rows, cols), (rows * (cols + 3), cols + 3, 1))
    source = torch.zeros(2, rows + 2, cols + 5, dtype=dtype, device="cuda")
    source[:, 1:1 + rows, 3:3 + cols] = g
    got = update(source[:, 1:1 + rows, 3:3 + cols], out=out)
    # the sum of squares is taken in another order there: the last bit of the norm may differ
    exact = iterate(normalised(g[0], 1e-7), 5, USUAL)
    assert (got[0].double() - want[0].double()).norm() <= 2 * min(rows, cols) ** 0.5 * spread_bound(5, USUAL, 1.3) + exact.norm() * torch.finfo(dtype).eps
    mask = torch.ones_like(held, dtype=torch.bool)
    mask[1:].as_strided((2, rows, cols), (rows * (cols + 3), cols + 3, 1))[:] = False
    assert (held[mask] == 5.0).all()


def test_one_matrix_for_all():
    g = tensor(1, 200, 140, seed=15)
    want = update(g)
    shared = g[0].as_strided((3, 200, 140), (0, 140, 1))
    got = update(shared)
    for i in range(3):
        assert (got[i].double() - want[0].double()).norm() <= 2 * 140 ** 0.5 * spread_bound(5, USUAL, 1.3)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("rows,cols", [(60, 90), (310, 300), (1, 5000), (2047, 128), (130, 5001)])
def test_many_steps_reach_orthogonal_rows(rows, cols):
    """The cubic iteration p(s) = (3 s - s^3) / 2 has p(1) = 1 and p'(1) = 0: what is left is one step's perturbation, 2^-20 max(1, |a| + |b|) = 2^-19 of the
    2-norm, twice in O O^T and sqrt(r) of it in the Frobenius norm."""
    o = update(tensor(1, rows, cols, seed=16), steps=40, coefficients=(1.5, -0.5, 0.0))[0].double()
    o = o if rows <= cols else o.T
    r = o.shape[0]
    assert (o @ o.T - torch.eye(r, device="cuda", dtype=torch.float64)).norm() <= 2 * r ** 0.5 * 2.0 ** -19


def test_beside_other_calls_of_the_library():
    """Between emulated products on one stream, and three kinds of calls on three streams at once: the results of the same calls alone, bit for bit."""
    a, b = tensor(1, 600, 700, seed=17), tensor(1, 100, 400, seed=18, dtype=torch.bfloat16)
    want_a, want_b = update(a), update(b, torch.bfloat16)
    x, w = tensor(900, 512, seed=19, dtype=torch.bfloat16), tensor(4, 640, 512, seed=20, dtype=torch.bfloat16, scale=0.05)
    offsets = torch.tensor([0, 100, 600, 600, 900]).cuda()

    def experts(y, stream=None):
        oz.check(oz.oz_gemm_grouped(1, 640, 900, 512, 4, offsets, oz.OZ_BF16, w, 512, 640 * 512, x, 512, oz.OZ_BF16, 0.0, y, 640, stream))
        return y

    want_y = experts(torch.zeros(900, 640, dtype=torch.bfloat16, device="cuda"))
    n = 512
    A, B = (torch.randn(n, n, dtype=torch.float64, device="cuda") for _ in range(2))
    C = torch.zeros(n, n, dtype=torch.float64, device="cuda")
    product_space = torch.empty(oz.oz_workspace_bytes(n, n, n, oz.OZ_SET_S, 0), dtype=torch.uint8, device="cuda")
    oz.check(oz.oz_set_workspace(product_space))
    oz.check(oz.oz_dgemm(n, n, n, A, n, B, n, C, n))
    want_c = C.clone()
    spaces = [torch.empty(oz.oz_orthogonalise_workspace_bytes(g.shape[2], g.shape[1], 1), dtype=torch.uint8, device="cuda") for g in (a, b)]
    out_a, out_b, out_y = torch.zeros_like(want_a), torch.zeros_like(want_b), torch.zeros_like(want_y)
    for _ in range(5):
        for call in (lambda: experts(out_y), lambda: update(a, out=out_a, workspace=spaces[0]), lambda: update(b, out=out_b, workspace=spaces[1])):
            C.zero_()
            oz.check(oz.oz_dgemm(n, n, n, A, n, B, n, C, n))
            call()
            assert torch.equal(C, want_c)
    assert torch.equal(out_a, want_a) and torch.equal(out_b, want_b) and torch.equal(out_y, want_y)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(10):
        update(a, out=out_a, workspace=spaces[0], stream=streams[0])
        update(b, out=out_b, workspace=spaces[1], stream=streams[1])
        experts(out_y, streams[2])
    torch.cuda.synchronize()
    assert torch.equal(out_a, want_a) and torch.equal(out_b, want_b) and torch.equal(out_y, want_y)
    oz.oz_set_workspace(None)


def test_phases_of_seconds():
    """X X^T of one row is one tile: the other blocks wait for it through 350 million elements, more than 2 s.  4096 of them are +-1 and all others zero,
    so that X = G / 64, X X^T = 1 and 2 X - 1.5 X + 0.5 X = X are exact."""
    n = 350_000_000
    torch.cuda.empty_cache()
    need = oz.oz_orthogonalise_workspace_bytes(n, 1, 1)
    if torch.cuda.mem_get_info()[0] < need + 6 * n + (3 << 30):
        pytest.skip("the planes of this row fill a whole device")
    try:
        g = torch.zeros(1, 1, n, dtype=torch.bfloat16, device="cuda")
        at = torch.arange(4096, device="cuda") * 85_000 + 17
        g[0, 0, at] = (1.0 - 2.0 * (at % 2)).bfloat16()
        got = update(g, steps=1, coefficients=(2.0, -1.5, 0.5), eps=0.0, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
        assert oz.oz_query_status() in (oz.OZ_OK, oz.OZ_ERR_RANGE)
        assert torch.equal(got[0, 0, at], g[0, 0, at].float() / 64) and torch.count_nonzero(got).item() == 4096
    finally:
        g = got = None
        torch.cuda.empty_cache()


def poisoned_workspace(cols, rows, count):
    """All bits set: every half-precision number in it is NaN, and what is read before it is written shows."""
    return torch.full((oz.oz_orthogonalise_workspace_bytes(cols, rows, count),), 0xFF, dtype=torch.uint8, device="cuda")


# tiles of 64, 128 and 256 columns, one to six blocks of 256 rows, X as it is and transposed, borders inside a tile
@pytest.mark.parametrize("count,rows,cols", [(1, 310, 300), (2, 300, 310), (1, 257, 1030), (1, 1400, 1450), (12, 520, 520), (2, 1501, 1300), (16, 512, 2048), (16, 2047, 510)])
@pytest.mark.parametrize("dtype,out_dtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float16), (torch.float16, torch.bfloat16)])
def test_general_form_element_by_element(count, rows, cols, dtype, out_dtype):
    """One step, all matrices.  16-bit results take a X in through P's diagonal: P + a I is held in planes, whose bound has a beside b and c, and its product
    with X loses kappa of a |X| more."""
    a = USUAL[0]
    g = tensor(count, rows, cols, seed=21, dtype=dtype)
    got = update(g, out_dtype, 1, workspace=poisoned_workspace(cols, rows, count))
    assert oz.oz_query_status() in (oz.OZ_OK, oz.OZ_ERR_RANGE)
    for i in range(count):
        x, y = normalised(g[i], 1e-7), got[i].double()
        x, y = (x, y) if rows <= cols else (x.T, y.T)
        exact, e = iterate(x, 1, USUAL), step_bound(x, USUAL)
        if out_dtype != torch.float32:
            ax = x.abs()
            e = e + 1.02 * a * ((RHO + kappa(x.shape[0]) + 4 * U24) * ax + 2.0 ** -38 * ax.sum(0))
        tol = e + (exact.abs() + e) * torch.finfo(out_dtype).eps / 2 + (2.0 ** -25 if out_dtype == torch.float16 else 0.0)
        off = (y - exact).abs()
        assert (off <= tol).all(), (i, float((off / tol).nan_to_num(float("inf")).max()))


def fp32_error(x, steps=5):
    """The exact update of X and how far the usual iteration in FP32 is off, in the Frobenius norm."""
    exact = iterate(x, steps, USUAL)
    return exact, (iterate(x.float(), steps, USUAL).double() - exact).norm()


def hold_near(got, g, eps=1e-7):
    """Every matrix no further off than 4 errors of the FP32 iteration and the rounding of the result."""
    for i in range(g.shape[0]):
        exact, fp32 = fp32_error(normalised(g[i], eps))
        off = (got[i].double() - exact).norm()
        assert off <= 4 * fp32 + 2 * exact.norm() * torch.finfo(got.dtype).eps / 2, (i, float(off / exact.norm()))


@pytest.mark.parametrize("count,rows,cols", [(3, 300, 260), (2, 260, 300), (4, 700, 150), (3, 90, 120), (2, 520, 530)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strided_batch_close(count, rows, cols, dtype):
    """All matrices of a strided batch against 64 bits, and element by element against the contiguous call: both are within 4 errors of the FP32
    iteration of the exact update before they are rounded, each by half a step."""
    g = tensor(count, rows, cols, seed=22, dtype=dtype)
    want = update(g, dtype, workspace=poisoned_workspace(cols, rows, count))
    hold_near(want, g)
    source = torch.zeros(count, rows + 2, cols + 5, dtype=dtype, device="cuda")
    source[:, 1:1 + rows, 3:3 + cols] = g
    held = torch.full((count * (rows * (cols + 3) + 7) + 1,), 5.0, dtype=dtype, device="cuda")
    out = held[1:].as_strided((count, rows, cols), (rows * (cols + 3) + 7, cols + 3, 1))
    got = update(source[:, 1:1 + rows, 3:3 + cols], out=out, workspace=poisoned_workspace(cols, rows, count))
    hold_near(got, g)
    for i in range(count):
        _, fp32 = fp32_error(normalised(g[i], 1e-7))
        w = want[i].double().abs()
        assert ((got[i].double() - want[i].double()).abs() <= 8 * fp32 + torch.finfo(dtype).eps * (w + 8 * fp32)).all(), i


@pytest.mark.parametrize("rows,cols", [(40, 30), (300, 200)])
def test_scales_close(rows, cols):
    """From the largest numbers to subnormal ones: the update does not depend on the scale."""
    for scale in (1e37, 1e-3, 1e-37, 1e-43):
        g = tensor(2, rows, cols, seed=23) * scale
        hold_near(update(g, eps=0.0, workspace=poisoned_workspace(cols, rows, 2)), g, eps=0.0)
    assert oz.oz_query_status() in (oz.OZ_OK, oz.OZ_ERR_RANGE)


@pytest.mark.parametrize("rows,cols", [(200, 140), (100, 90)])
def test_one_matrix_for_all_close(rows, cols):
    g = tensor(1, rows, cols, seed=24)
    got = update(g[0].as_strided((3, rows, cols), (0, cols, 1)), workspace=poisoned_workspace(cols, rows, 3))
    hold_near(got, g.expand(3, rows, cols))


def test_update_of_experts_gradients_close():
    """Gradients of uneven groups, an empty one among them, straight into the update."""
    sizes, m, k = [300, 0, 41, 171], 136, 264
    offsets = torch.tensor([0] + sizes).cumsum(0).cuda()
    n, groups = sum(sizes), len(sizes)
    x, dy = tensor(n, k, seed=25, dtype=torch.bfloat16), tensor(n, m, seed=26, dtype=torch.bfloat16)
    for dw_dtype in (torch.float32, torch.bfloat16):
        dw = torch.zeros(groups, m, k, dtype=dw_dtype, device="cuda")
        oz.check(oz.oz_gemm_grouped_wgrad(k, m, n, groups, offsets, oz.OZ_BF16, x, k, dy, m, TYPE[dw_dtype], 0.0, dw, k, m * k))
        o = update(dw, workspace=poisoned_workspace(k, m, groups))
        assert not o[1].any()
        used = [0, 2, 3]
        hold_near(o[used], dw[used])


@pytest.mark.parametrize("count,rows,cols", [(1, 1024, 1024), (3, 1009, 517), (16, 512, 2048), (1, 2048, 2048), (2, 300, 260), (2, 100, 700)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_16_bit_results_are_rounded_from_fp32_accuracy(count, rows, cols, dtype):
    """Held to 4 errors of the FP32 iteration before the rounding as well: at most 4 times as many results as that has are not the exact update correctly rounded
    (how many there are goes with the error before the rounding), and 6 standard deviations of such a count."""
    g = tensor(count, rows, cols, seed=27, dtype=dtype)
    got = update(g, dtype)
    mine = usual = 0
    for i in range(count):
        x = normalised(g[i], 1e-7)
        rounded = iterate(x, 5, USUAL).to(dtype)
        mine += (got[i] != rounded).sum().item()
        usual += (iterate(x.float(), 5, USUAL).to(dtype) != rounded).sum().item()
    assert mine <= 4 * usual + 6 * (4 * usual + 1) ** 0.5, (mine, usual)
