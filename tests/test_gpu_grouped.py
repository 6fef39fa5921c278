"""Grouped products against plain products in 64 bits.

Tolerance of an element, before any run: a product of two 16-bit numbers is exact in FP32, and each of the at most K + 1 additions (K products, the
old value) loses at most a unit in the last place, 2^-23 of a magnitude that is at most S = (|A| |B|)_ij + |C_ij|, whatever the order
and whether the adder rounds or cuts off: e = (K + 1) 2^-23 S.  The result is then rounded once: half a step of its type relative to the value,
and for f16 half of its smallest step, 2^-25, near zero.  Together  e + (|exact| + e) eps / 2 + tiny."""
import pytest
import torch

import paper_2609_09095_b200 as oz

pytestmark = pytest.mark.gpu

OZ_TYPE = {torch.bfloat16: oz.OZ_BF16, torch.float16: oz.OZ_F16, torch.float32: oz.OZ_F32}


def within(got, exact, size, K, what=""):
    e = (K + 1) * 2.0 ** -23 * size
    tol = e + (exact.abs() + e) * torch.finfo(got.dtype).eps / 2 + (2.0 ** -25 if got.dtype == torch.float16 else 2.0 ** -134)
    off = (got.double() - exact).abs()
    bad = ~(off <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} elements, worst {float((off / tol)[bad].max()) if off.isfinite().all() else off.max()} tolerances"


def offsets_of(sizes, first=0):
    return torch.tensor([first] + list(sizes), dtype=torch.int64).cumsum(0).cuda()


def run_grouped(x, w, offsets, out, transA, beta=0.0, lda=None, strideA=None, ldb=None, ldc=None, stream=None):
    """x (n, k) rows are tokens, w (groups, m, k) for transA = 1 or (groups, k, m) for transA = 0, out (n, m), by their own strides."""
    groups = offsets.numel() - 1
    m, k = (w.shape[1], w.shape[2]) if transA else (w.shape[2], w.shape[1])
    oz.check(oz.oz_gemm_grouped(transA, m, x.shape[0], k, groups, offsets, OZ_TYPE[x.dtype], w, w.stride(1) if lda is None else lda,
                                w.stride(0) if strideA is None else strideA, x, x.stride(0) if ldb is None else ldb, OZ_TYPE[out.dtype], beta,
                                out, out.stride(0) if ldc is None else ldc, stream), "oz_gemm_grouped")
    return out


def run_wgrad(x, dy, offsets, out, beta=0.0, stream=None):
    """out (groups, rows of dy, columns of x) += dy^T x over the tokens of each group"""
    oz.check(oz.oz_gemm_grouped_wgrad(x.shape[1], dy.shape[1], x.shape[0], offsets.numel() - 1, offsets, OZ_TYPE[x.dtype], x, x.stride(0), dy,
                                      dy.stride(0), OZ_TYPE[out.dtype], beta, out, out.stride(1), out.stride(0), stream), "oz_gemm_grouped_wgrad")
    return out


def check_grouped(x, w, offsets, out, old, transA, beta):
    cuts = offsets.tolist()
    K = x.shape[1]
    touched = torch.zeros(x.shape[0], dtype=torch.bool)
    for g, (lo, hi) in enumerate(zip(cuts, cuts[1:])):
        if hi == lo:
            continue
        touched[lo:hi] = True
        a = (w[g].T if transA else w[g]).double()
        exact, size = x[lo:hi].double() @ a, x[lo:hi].double().abs() @ a.abs()
        if beta:
            exact, size = exact + old[lo:hi].double(), size + old[lo:hi].double().abs()
        within(out[lo:hi], exact, size, K, f"group {g} of {len(cuts) - 1}")
    assert torch.equal(out[~touched.cuda()], old[~touched.cuda()]), "columns of no group"


def tensor(*shape, dtype, seed, scale=1.0):
    return (torch.randn(*shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)) * scale).to(dtype)


# (sizes, first, behind, m, k)
SHAPES = [([1], 0, 0, 8, 8),
          ([1], 0, 0, 128, 64),
          ([0, 1, 0, 1, 0, 0], 0, 0, 256, 512),
          ([3, 0, 17, 1], 2, 5, 136, 200),
          ([16, 32, 31, 33], 0, 0, 64, 1032),
          ([255, 256, 257], 0, 1, 320, 72),
          ([700, 0, 5], 0, 9, 1000, 520),
          ([130], 1, 1, 1, 8),
          ([64, 63], 0, 0, 129, 1),
          ([5] * 70, 0, 3, 257, 96),
          ([0, 0, 0], 3, 4, 40, 48),
          ([513, 1027], 0, 0, 776, 2056)]


@pytest.mark.parametrize("sizes,first,behind,m,k", SHAPES)
@pytest.mark.parametrize("transA", [0, 1])
@pytest.mark.parametrize("dtype,out_dtype", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, torch.float32)])
def test_grouped(sizes, first, behind, m, k, transA, dtype, out_dtype):
    offsets = offsets_of(sizes, first)
    n = first + sum(sizes) + behind
    x = tensor(n, k, dtype=dtype, seed=1)
    w = tensor(len(sizes), *((m, k) if transA else (k, m)), dtype=dtype, seed=2, scale=k ** -0.5)
    old = tensor(n, m, dtype=out_dtype, seed=3)
    for beta in (0.0, 1.0):
        out = run_grouped(x, w, offsets, old.clone(), transA, beta)
        assert oz.oz_query_status() in (oz.OZ_OK, oz.OZ_ERR_RANGE)
        check_grouped(x, w, offsets, out, old, transA, beta)


@pytest.mark.parametrize("sizes,first,behind,m,k", SHAPES)
@pytest.mark.parametrize("dtype,out_dtype", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, torch.float32),
                                             (torch.float16, torch.float32)])
def test_wgrad(sizes, first, behind, m, k, dtype, out_dtype):
    offsets = offsets_of(sizes, first)
    n = first + sum(sizes) + behind
    x, dy = tensor(n, k, dtype=dtype, seed=4), tensor(n, m, dtype=dtype, seed=5, scale=0.1)
    old = tensor(len(sizes), m, k, dtype=out_dtype, seed=6)
    cuts = offsets.tolist()
    for beta in (0.0, 1.0):
        out = run_wgrad(x, dy, offsets, old.clone(), beta)
        assert oz.oz_query_status() in (oz.OZ_OK, oz.OZ_ERR_RANGE)
        for g, (lo, hi) in enumerate(zip(cuts, cuts[1:])):
            a, b = dy[lo:hi].double(), x[lo:hi].double()
            exact, size = a.T @ b, a.abs().T @ b.abs()
            if beta:
                exact, size = exact + old[g].double(), size + old[g].double().abs()
            within(out[g], exact, size, hi - lo, f"group {g}")
            if hi == lo:
                assert torch.equal(out[g], old[g] if beta else torch.zeros_like(old[g]))


@pytest.mark.parametrize("m,k", [(96, 80), (33, 41), (264, 520)])
@pytest.mark.parametrize("transA", [0, 1])
def test_strides_and_addresses(m, k, transA):
    """Leading dimensions larger than the matrices, odd ones, addresses that are aligned to the element only, one matrix for all groups."""
    sizes = [40, 0, 7, 290]
    offsets = offsets_of(sizes)
    n = sum(sizes)
    for pad, shift, shared in ((8, 8, False), (1, 0, False), (8, 1, False), (8, 0, True), (3, 5, True)):
        ld = (k if transA else m) + pad
        lines = m if transA else k
        stride = ld * (lines + (8 if pad == 8 else 1))
        flat = tensor(shift + len(sizes) * stride, dtype=torch.bfloat16, seed=7, scale=k ** -0.5)[shift:]
        w = flat.as_strided((len(sizes), lines, ld - pad), (0 if shared else stride, ld, 1))
        x = tensor(shift + n * (k + pad), dtype=torch.bfloat16, seed=8)[shift:].as_strided((n, k), (k + pad, 1))
        held = tensor(shift + n * (m + pad), dtype=torch.bfloat16, seed=9)
        before = held.clone()
        out = held[shift:].as_strided((n, m), (m + pad, 1))
        old = out.clone()
        run_grouped(x, w, offsets, out, transA)
        check_grouped(x, w, offsets, out, old, transA, 0.0)
        mask = torch.ones_like(held, dtype=torch.bool)
        mask[shift:].as_strided((n, m), (m + pad, 1))[:] = False
        assert torch.equal(held[mask], before[mask]), "between the columns of C"
        # gradient of the weights from the same operands, into a strided result
        dy = tensor(shift + n * (m + pad), dtype=torch.bfloat16, seed=10, scale=0.1)[shift:].as_strided((n, m), (m + pad, 1))
        grad = torch.zeros(len(sizes) * m * (k + pad) + 5, device="cuda").as_strided((len(sizes), m, k), (m * (k + pad) + 1, k + pad, 1))
        run_wgrad(x, dy, offsets, grad)
        for g, (lo, hi) in enumerate(zip(offsets.tolist(), offsets.tolist()[1:])):
            a, b = dy[lo:hi].double(), x[lo:hi].double()
            within(grad[g], a.T @ b, a.abs().T @ b.abs(), hi - lo)


def test_unused_values_do_not_spread():
    """NaN and Inf in columns of no group, in the weights of an empty group, and in the columns of another group."""
    sizes, first, behind, m, k = [37, 0, 70, 300], 3, 30, 200, 136
    offsets = offsets_of(sizes, first)
    n = first + sum(sizes) + behind
    for poison in (float("nan"), float("inf"), float("-inf")):
        x, dy = tensor(n, k, dtype=torch.bfloat16, seed=11), tensor(n, m, dtype=torch.bfloat16, seed=12)
        w = tensor(4, m, k, dtype=torch.bfloat16, seed=13)
        x[:first] = x[n - behind:] = dy[:first] = dy[n - behind:] = poison
        w[1] = poison
        old = tensor(n, m, dtype=torch.bfloat16, seed=14)
        check_grouped(x, w, offsets, run_grouped(x, w, offsets, old.clone(), 1), old, 1, 0.0)
        grad = run_wgrad(x, dy, offsets, torch.full((4, m, k), 7.0, device="cuda"))
        assert grad.isfinite().all() and not grad[1].any()
        # one token of group 2 and its gradient
        x[first + 40, 5], dy[first + 41, 9] = poison, poison
        y = run_grouped(x, w, offsets, old.clone(), 1)
        inside = y[first:n - behind]
        assert not inside[40].isfinite().any() and inside[:40].isfinite().all() and inside[41:].isfinite().all()
        grad = run_wgrad(x, dy, offsets, torch.zeros(4, m, k, device="cuda"))
        assert grad[0].isfinite().all() and not grad[1].any() and grad[3].isfinite().all()
        bad = ~grad[2].isfinite()
        want = torch.zeros_like(bad)
        want[:, 5], want[9, :] = True, True
        assert torch.equal(bad, want)


def test_bad_offsets_are_reported():
    n, m, k = 300, 64, 96
    x, w, dy = tensor(n, k, dtype=torch.bfloat16, seed=15), tensor(3, m, k, dtype=torch.bfloat16, seed=16), tensor(n, m, dtype=torch.bfloat16, seed=17)
    for offsets in ([0, 200, 100, 300], [-5, 10, 20, 300], [0, 10, 20, 301], [0, 2 ** 40, 7, -2 ** 40]):
        off = torch.tensor(offsets, dtype=torch.int64, device="cuda")
        held = torch.zeros(n + 8, m, dtype=torch.bfloat16, device="cuda")
        run_grouped(x, w, off, held[:n], 1)
        assert oz.oz_query_status() == oz.OZ_ERR_INVALID_ARG
        assert not held[n:].any()
        run_wgrad(x, dy, off, torch.zeros(3, m, k, device="cuda"))
        assert oz.oz_query_status() == oz.OZ_ERR_INVALID_ARG
    run_grouped(x, w, offsets_of([100, 100, 100]), held[:n], 1)
    assert oz.oz_query_status() == oz.OZ_OK


def test_gradients_against_differences():
    """Integers small enough that every product and sum is exact: with L = sum(r * y), L(w + h e) - L(w - h e) = 2 h dL/dw, and the same for x, exactly."""
    sizes, m, k = [19, 0, 45, 1], 24, 40
    offsets = offsets_of(sizes)
    n = sum(sizes)
    gen = torch.Generator("cuda").manual_seed(18)

    def small(*shape):
        return torch.randint(-3, 4, shape, device="cuda", generator=gen).to(torch.bfloat16)

    x, w, r = small(n, k), small(4, m, k), small(n, m)
    dw = run_wgrad(x, r, offsets, torch.empty(4, m, k, device="cuda"))
    dx = run_grouped(r, w, offsets, torch.empty(n, k, device="cuda"), 0)

    def loss(x, w):
        y = run_grouped(x, w, offsets, torch.zeros(n, m, device="cuda"), 1)
        return (y.double() * r.double()).sum().item()

    for g, i, j in ((0, 0, 0), (0, 23, 39), (1, 5, 5), (2, 11, 7), (3, 23, 1)):
        up, down = w.clone(), w.clone()
        up[g, i, j] += 2
        down[g, i, j] -= 2
        assert loss(x, up) - loss(x, down) == 4 * dw[g, i, j].item()
    for t, j in ((0, 0), (18, 39), (19, 3), (63, 20), (64, 39)):
        up, down = x.clone(), x.clone()
        up[t, j] += 2
        down[t, j] -= 2
        assert loss(up, w) - loss(down, w) == 4 * dx[t, j].item()


def test_graph_replays_with_new_offsets_and_streams():
    sizes, m, k = [200, 60, 0, 40], 264, 328
    n = 300
    x, w, dy = tensor(n, k, dtype=torch.float16, seed=19), tensor(4, m, k, dtype=torch.float16, seed=20, scale=0.05), tensor(n, m, dtype=torch.float16, seed=21)
    offsets = offsets_of(sizes)
    y, dw = torch.zeros(n, m, dtype=torch.float16, device="cuda"), torch.zeros(4, m, k, device="cuda")
    oz.oz_query_status()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run_grouped(x, w, offsets, y, 1)
        run_wgrad(x, dy, offsets, dw)
    for new in (sizes, [0, 0, 300, 0], [1, 2, 3, 294], [75, 75, 75, 75]):
        offsets.copy_(offsets_of(new))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check_grouped(x, w, offsets, y, torch.zeros_like(y), 1, 0.0)
        cuts = offsets.tolist()
        for g, (lo, hi) in enumerate(zip(cuts, cuts[1:])):
            a, b = dy[lo:hi].double(), x[lo:hi].double()
            within(dw[g], a.T @ b, a.abs().T @ b.abs(), hi - lo)
    # two calls at once on two streams, against the same calls one after the other: bit for bit
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [torch.zeros_like(y), torch.zeros(4, m, k, device="cuda")]
    torch.cuda.synchronize()
    for _ in range(5):
        run_grouped(x, w, offsets, outs[0], 1, stream=streams[0])
        run_wgrad(x, dy, offsets, outs[1], stream=streams[1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], y) and torch.equal(outs[1], dw)


def test_most_groups_and_beyond_32_bits():
    groups = oz.OZ_GROUPS_MAX
    sizes = [(7 * g) % 3 for g in range(groups)]
    offsets = offsets_of(sizes)
    n, m, k = sum(sizes) + 2, 16, 32
    x, w = tensor(n, k, dtype=torch.bfloat16, seed=22), tensor(groups, m, k, dtype=torch.bfloat16, seed=23)
    old = tensor(n, m, dtype=torch.float32, seed=24)
    check_grouped(x, w, offsets, run_grouped(x, w, offsets, old.clone(), 1), old, 1, 0.0)
    dy = tensor(n, m, dtype=torch.bfloat16, seed=25)
    grad = run_wgrad(x, dy, offsets, torch.zeros(groups, m, k, device="cuda"))
    pos = torch.repeat_interleave(torch.arange(groups), torch.tensor(sizes)).cuda()
    for c in range(0, n - 2, 400):
        assert torch.isfinite(grad[pos[c]]).all()
    lo, hi = offsets[groups - 2].item(), offsets[groups - 1].item()
    within(grad[groups - 2], dy[lo:hi].double().T @ x[lo:hi].double(), dy[lo:hi].double().abs().T @ x[lo:hi].double().abs(), hi - lo)
    # rows whose elements lie beyond 2^31: the last 100 of 70000 tokens of 32768 features
    n, m, k = 70000, 8, 32768
    x = torch.zeros(n, k, dtype=torch.bfloat16, device="cuda")
    x[-100:] = tensor(100, k, dtype=torch.bfloat16, seed=26)
    w = tensor(2, m, k, dtype=torch.bfloat16, seed=27, scale=k ** -0.5)
    offsets = torch.tensor([n - 100, n - 60, n], dtype=torch.int64, device="cuda")
    old = tensor(n, m, dtype=torch.float32, seed=28)
    check_grouped(x, w, offsets, run_grouped(x, w, offsets, old.clone(), 1), old, 1, 0.0)
    dy = tensor(n, m, dtype=torch.bfloat16, seed=29)
    grad = run_wgrad(x, dy, offsets, torch.zeros(2, m, k, device="cuda"))
    a, b = dy[-60:].double(), x[-60:].double()
    within(grad[1], a.T @ b, a.abs().T @ b.abs(), 60)


# sizes that the rule sends to each tile shape: 32 columns undivided and shared by 2 and 4, 64, 128, 256
@pytest.mark.parametrize("sizes,m,k", [([1], 2048, 1024), ([1, 0, 1], 4096, 1032), ([2] * 40, 640, 520), ([0, 40, 24, 50], 1024, 256), ([60] * 16, 2048, 200),
                                       ([1000, 900, 2000], 1304, 328)])
@pytest.mark.parametrize("transA", [0, 1])
@pytest.mark.parametrize("dtype,out_dtype", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32)])
def test_tile_shapes(sizes, m, k, transA, dtype, out_dtype):
    offsets = offsets_of(sizes, 1)
    n = 1 + sum(sizes) + 2
    x = tensor(n, k, dtype=dtype, seed=30)
    w = tensor(len(sizes), *((m, k) if transA else (k, m)), dtype=dtype, seed=31, scale=k ** -0.5)
    old = tensor(n, m, dtype=out_dtype, seed=32)
    for beta in (0.0, 1.0):
        check_grouped(x, w, offsets, run_grouped(x, w, offsets, old.clone(), transA, beta), old, transA, beta)
    assert oz.oz_query_status() in (oz.OZ_OK, oz.OZ_ERR_RANGE)


def test_long_sums_in_fp32():
    """Sums of positive numbers, whose running value only grows: each of the K / 16 additions of the tensor core to it cuts off less than a unit in the
    last place, 2^-23, of an accumulator that is started again every 512 indices and so holds at most 512 / K of the whole (and a unit more for a
    sixteen's own sum); what is started again is added with rounding, 2^-24 of the whole each time."""
    K = 8192
    x, w = tensor(3, K, dtype=torch.bfloat16, seed=33).abs(), tensor(1, 256, K, dtype=torch.bfloat16, seed=34).abs()
    y = run_grouped(x, w, offsets_of([3]), torch.zeros(3, 256, device="cuda"), 1)
    exact = x.double() @ w[0].double().T
    # numbers are alike enough that a piece's share of the sum is at most twice its share of the indices
    steps = 512 // 16 + 17
    tol = exact * (steps * 2.0 ** -23 + K // 512 * 2.0 ** -24)
    assert ((y.double() - exact).abs() <= tol).all()
    grad = run_wgrad(w[0].T.contiguous(), w[0].T.contiguous(), offsets_of([K]), torch.zeros(1, 256, 256, device="cuda"))[0]
    exact = w[0].double() @ w[0].double().T
    assert ((grad.double() - exact).abs() <= exact * (steps * 2.0 ** -23 + K // 512 * 2.0 ** -24)).all()


def test_broadcast_inputs():
    """One row of tokens for a whole group (stride 0 is expanded by the caller), the same expert twice, the same gradient for all tokens."""
    m, k = 264, 136
    offsets = offsets_of([100, 30])
    x = tensor(1, k, dtype=torch.bfloat16, seed=35).expand(130, k).contiguous()
    w = tensor(1, m, k, dtype=torch.bfloat16, seed=36, scale=0.1).expand(2, m, k)
    y = run_grouped(x, w, offsets, torch.zeros(130, m, dtype=torch.float32, device="cuda"), 1)
    assert torch.equal(y, y[:1].expand_as(y))
    dy = torch.ones(130, m, dtype=torch.bfloat16, device="cuda")
    grad = run_wgrad(x, dy, offsets, torch.zeros(2, m, k, device="cuda"))
    for g, count in ((0, 100), (1, 30)):
        exact = count * x[0].double()
        assert ((grad[g].double() - exact).abs() <= (count + 1) * 2.0 ** -23 * exact.abs()).all()


def test_fp32_results_lose_as_little_as_fp32_sums():
    """Sums of positive numbers, of which the tensor core only ever cuts off.  An accumulator takes 320 inner indices in 20 additions and grows evenly;
    each addition loses half a unit in the mean, at most 2^-24 of what the accumulator then holds, together (20 + 1) / 2 2^-24 of a segment.  What is
    rounded to nearest afterwards has no mean."""
    K = 4096
    x, w = tensor(64, K, dtype=torch.bfloat16, seed=37).abs(), tensor(1, 320, K, dtype=torch.bfloat16, seed=38).abs()
    y = run_grouped(x, w, offsets_of([64]), torch.zeros(64, 320, device="cuda"), 1)
    dx = run_grouped(x, w.transpose(1, 2).contiguous(), offsets_of([64]), torch.zeros(64, 320, device="cuda"), 0)
    grad = run_wgrad(w[0].T.contiguous(), x.T.contiguous(), offsets_of([K]), torch.zeros(1, 64, 320, device="cuda"))[0]
    exact = x.double() @ w[0].double().T
    for got in (y, dx, grad):
        loss = ((exact - got.double()) / exact).mean().item()
        assert abs(loss) <= 10.5 * 2.0 ** -24, loss * 2 ** 24


# 16-bit results of at most 256 tokens a group leave by rows, through shared memory, where C's columns begin on 16 bytes: widths that end inside eight
# numbers, inside the 64 of a warp and inside a tile, with numbers behind them that stay
@pytest.mark.parametrize("m,k", [(1, 1), (5, 7), (40, 33), (129, 100), (257, 259), (300, 516), (64, 1027)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_wgrad_by_rows_ends_anywhere(m, k, dtype):
    sizes = [100, 0, 37, 1, 250]
    offsets = offsets_of(sizes, 3)
    n, groups = 3 + sum(sizes) + 2, len(sizes)

    def padded(cols, seed, scale):
        ld = (cols + 7) // 8 * 8
        return tensor(n, ld, dtype=dtype, seed=seed, scale=scale)[:, :cols]

    x, dy = padded(k, 39, 1.0), padded(m, 40, 0.1)
    ldc = (k + 7) // 8 * 8 + 8
    stride = m * ldc + 16
    held = torch.full((groups * stride,), 9.0, dtype=dtype, device="cuda")
    grad = held.as_strided((groups, m, k), (stride, ldc, 1))
    run_wgrad(x, dy, offsets, grad)
    cuts = offsets.tolist()
    for g, (lo, hi) in enumerate(zip(cuts, cuts[1:])):
        a, b = dy[lo:hi].double(), x[lo:hi].double()
        within(grad[g], a.T @ b, a.abs().T @ b.abs(), hi - lo, f"group {g}")
    mask = torch.ones_like(held, dtype=torch.bool)
    mask.as_strided((groups, m, k), (stride, ldc, 1))[:] = False
    assert (held[mask] == 9.0).all(), "behind the rows"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_16_bit_results_of_long_sums(dtype):
    """Sums of positive numbers over more than two accumulators of 4096 inner indices.  Each of the 256 additions to an accumulator, and the sixteen's own
    sum, cuts off less than 2^-23 of what the accumulator holds at its end, the additions of the accumulators round by 2^-24; then one rounding
    to the type."""
    K = 9000
    x, w = tensor(5, K, dtype=dtype, seed=41).abs(), tensor(1, 136, K, dtype=dtype, seed=42, scale=1 / 64).abs()
    y = run_grouped(x, w, offsets_of([5]), torch.zeros(5, 136, dtype=dtype, device="cuda"), 1)
    xs, ws = torch.zeros(K, 8, dtype=dtype, device="cuda"), w[0].T.contiguous()
    xs[:, :5] = x.T
    grad = run_wgrad(ws, xs, offsets_of([K]), torch.zeros(1, 8, 136, dtype=dtype, device="cuda"))[0, :5]
    exact = x.double() @ w[0].double().T
    lost = 257 * 2.0 ** -23 + 3 * 2.0 ** -24
    for got in (y, grad):
        assert ((got.double() - exact).abs() <= exact * (lost + (1 + lost) * torch.finfo(dtype).eps / 2)).all()


def test_same_call_same_bits():
    """All forms that a launch can take, three times each."""
    for groups, each, m, k in ((1, 1, 2048, 1024), (8, 2, 512, 512), (16, 40, 1000, 520), (4, 700, 1304, 328), (2, 33, 41, 37)):
        sizes = [each + (g % 3) * (each // 4) for g in range(groups)]
        offsets = offsets_of(sizes)
        n = sum(sizes)
        x, w, dy = tensor(n, k, dtype=torch.bfloat16, seed=43), tensor(groups, m, k, dtype=torch.bfloat16, seed=44, scale=k ** -0.5), tensor(n, m, dtype=torch.bfloat16, seed=45)
        for out in (torch.bfloat16, torch.float32):
            y = [run_grouped(x, w, offsets, torch.zeros(n, m, dtype=out, device="cuda"), 1) for _ in range(3)]
            dx = [run_grouped(dy, w, offsets, torch.zeros(n, k, dtype=out, device="cuda"), 0) for _ in range(3)]
            dw = [run_wgrad(x, dy, offsets, torch.zeros(groups, m, k, dtype=out, device="cuda")) for _ in range(3)]
            for r in (y, dx, dw):
                assert torch.equal(r[0], r[1]) and torch.equal(r[0], r[2])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_16_bit_results_are_rounded_from_fp32_sums(dtype):
    """Of results that are not the exact value correctly rounded there are at most 4 times as many as a product in FP32 has: how many there are goes with the
    error before the rounding, of which 4 times that of FP32 is what the update of a parameter is held to as well."""
    K = 4096
    x, w = tensor(512, K, dtype=dtype, seed=46), tensor(1, 1024, K, dtype=dtype, seed=47, scale=1 / 64)
    zero = torch.zeros(512, 1024, dtype=dtype, device="cuda")
    y = run_grouped(x, w, offsets_of([512]), zero.clone(), 1)
    dx = run_grouped(x, w.transpose(1, 2).contiguous(), offsets_of([512]), zero.clone(), 0)
    grad = run_wgrad(w[0].T.contiguous(), x.T.contiguous(), offsets_of([K]), zero[None].clone())[0]
    rounded, plain = (x.double() @ w[0].double().T).to(dtype), (x.float() @ w[0].float().T).to(dtype)
    for got in (y, dx, grad):
        assert (got != rounded).sum() <= 4 * (plain != rounded).sum()
