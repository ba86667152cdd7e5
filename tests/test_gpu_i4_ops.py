"""Products with 4-bit weights on the GPU against their definitions (oracle/rows4.py), at the sizes and values where they can go wrong."""
import numpy as np
import pytest
import torch

import paper_2603_03383_amd as P
from oracle import rows4

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TD = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}  # half a step, relative to the value
LEAST = {"bf16": 0.0, "fp16": 2.0 ** -25, "fp32": 0.0}              # half of binary16's smallest step
GUARD = 3  # rows behind the last, which no call may write


def _np(t):
    return t.detach().double().cpu().numpy()


def _rng(*seed):
    return np.random.default_rng(list(seed))


def _dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(TD[dtype])


class Matrix:
    """A packed matrix, and what it stands for."""

    def __init__(self, rng, n, k, group, zeros, dtype, powers=False):
        groups = -(-k // group)
        self.codes = rng.integers(0, 16, (n, k), dtype=np.uint8)
        scales = 2.0 ** -rng.integers(0, 4, (n, groups)) if powers else rng.uniform(0.5, 1.5, (n, groups)) / np.sqrt(k)
        scales = _dev(scales, dtype)
        self.zeros = rng.integers(0, 16, (n, groups), dtype=np.uint8) if zeros else None
        self.scales = _np(scales)
        self.values = rows4.values(self.codes, self.scales, self.zeros, group)
        self.packed = torch.empty(P.medusa_packed_i4_bytes(n, k, group, zeros), dtype=torch.uint8, device=DEV)
        P.medusa_pack_codes_i4(_dev(self.codes), scales, None if self.zeros is None else _dev(self.zeros), group, self.packed, n)

    def weight_of_sums(self, x, group):
        """Sum over k of |x| times the codes' and zero points' magnitudes as the products meet them, scaled: what rounding errors go by."""
        k = self.codes.shape[1]
        spread = lambda t: np.repeat(np.asarray(t, np.float64), group, axis=1)[:, :k]  # noqa: E731
        z = 8.0 if self.zeros is None else spread(self.zeros)
        return np.abs(x) @ ((32 + self.codes + z) * spread(self.scales)).T


def _ws(need, rows, n, k):
    return torch.empty(need(rows, n, k), dtype=torch.uint8, device=DEV)


def linear(x, m, group, n, out, stream=None):
    rows, k = x.shape
    y = torch.full((rows + GUARD, n), 7.5, dtype=TD[out], device=DEV)
    P.medusa_linear_i4(x, m.packed, group, m.zeros is not None, y[:rows], _ws(P.medusa_linear_i4_workspace_bytes, rows, n, k), stream)
    assert bool((y[rows:] == 7.5).all())
    return y[:rows]


def swiglu(x, gate, up, group, n):
    rows, k = x.shape
    y = torch.full((rows + GUARD, n), 7.5, dtype=x.dtype, device=DEV)
    P.medusa_swiglu_i4(x, gate.packed, up.packed, group, gate.zeros is not None, y[:rows], _ws(P.medusa_swiglu_i4_workspace_bytes, rows, n, k))
    assert bool((y[rows:] == 7.5).all())
    return y[:rows]


# rows, columns, features
SHAPES = [(1, 1, 1), (1, 16, 128), (2, 5, 31), (3, 17, 33), (4, 64, 129), (5, 48, 256), (8, 100, 500), (15, 688, 256), (16, 33, 1387), (17, 160, 640),
          (31, 7, 2050), (32, 512, 96), (33, 1025, 130), (63, 96, 4096), (64, 272, 1024), (65, 40, 385), (90, 1387, 400), (129, 200, 256), (200, 70, 1000)]
KINDS = [("bf16", 128, False), ("fp16", 128, True), ("bf16", 64, True), ("fp16", 64, False), ("bf16", 32, False), ("fp16", 32, True), ("bf16", 32, True)]


@pytest.mark.parametrize("rows,n,k", SHAPES)
@pytest.mark.parametrize("dtype,group,zeros", KINDS)
def test_linear_of_integers_is_exact(dtype, group, zeros, rows, n, k):
    """Rows of small integers and scales that are powers of two: every sum is a multiple of 1 / 8 below 2^21, so fp32 holds it and no order changes it."""
    rng = _rng(rows, n, k, group)
    m = Matrix(rng, n, k, group, zeros, dtype, powers=True)
    x = _dev(rng.integers(-4, 5, (rows, k)).astype(np.float32), dtype)
    assert np.array_equal(_np(linear(x, m, group, n, "fp32")), rows4.linear(_np(x), m.values))


def _tolerance(x, m, group, k):
    # a step of the matrix cores adds 32 products to a sum: up to 16 roundings' worth (five levels and the sum itself, truncating); 128 features are
    # four steps; taking off the zero point and scaling are two more roundings; then one addition per group and eight between waves
    return (4 * 16 + 2 + 8) * 2.0 ** -24 * m.weight_of_sums(x, group) + -(-k // group) * 2.0 ** -24 * (np.abs(x) @ np.abs(m.values).T)


@pytest.mark.parametrize("rows,n,k", SHAPES)
@pytest.mark.parametrize("dtype,group,zeros", KINDS)
def test_linear(dtype, group, zeros, rows, n, k):
    rng = _rng(rows, n, k, group, 1)
    m = Matrix(rng, n, k, group, zeros, dtype)
    x = _dev(rng.standard_normal((rows, k)).astype(np.float32), dtype)
    want, tol = rows4.linear(_np(x), m.values), _tolerance(_np(x), m, group, k)
    for out in ("fp32", "bf16", "fp16"):
        off = np.abs(_np(linear(x, m, group, n, out)) - want)
        assert (off <= tol * (1 + HALF[out]) + HALF[out] * np.abs(want) + LEAST[out]).all(), (out, off.max())


@pytest.mark.parametrize("rows,n,k", SHAPES)
@pytest.mark.parametrize("dtype,group,zeros", KINDS)
def test_swiglu(dtype, group, zeros, rows, n, k):
    rng = _rng(rows, n, k, group, 2)
    gate, up = Matrix(rng, n, k, group, zeros, dtype), Matrix(rng, n, k, group, zeros, dtype)
    x = _dev(rng.standard_normal((rows, k)).astype(np.float32), dtype)
    xs = _np(x)
    want = rows4.swiglu(xs, gate.values, up.values)
    g, u = rows4.linear(xs, gate.values), rows4.linear(xs, up.values)
    tg, tu = _tolerance(xs, gate, group, k), _tolerance(xs, up, group, k)
    # SiLU's slope is at most 1.1 and it is at most |g|; exponential, sum, quotient and product: 8 roundings of fp32 at most
    tol = 1.1 * tg * (np.abs(u) + tu) + np.abs(g) * tu + 8 * 2.0 ** -24 * np.abs(want)
    off = np.abs(_np(swiglu(x, gate, up, group, n)) - want)
    assert (off <= tol * (1 + HALF[dtype]) + HALF[dtype] * np.abs(want) + LEAST[dtype]).all(), off.max()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_pack_weight_is_the_definition(dtype, group, zeros):
    """A product with the unit rows reads the matrix back."""
    rng = _rng(group, zeros)
    n, k = 37, 300
    w = rng.standard_normal((n, k)) * 10.0 ** rng.uniform(-3, 1, (n, 1))
    w[3] = 0
    w[4] = np.abs(w[4])
    w[5] = -np.abs(w[5])
    w[6, :] = 0.25
    if dtype == "fp16":
        w[7] *= 1e-6  # scales in binary16's subnormals, or zero
    src = _dev(w.astype(np.float32), dtype)
    codes, scales, points = rows4.quantize(src.float().cpu().numpy(), group, zeros, dtype)
    packed = torch.empty(P.medusa_packed_i4_bytes(n, k, group, zeros), dtype=torch.uint8, device=DEV)
    P.medusa_pack_weight_i4(src, group, packed, n, zeros=zeros)
    same = torch.empty_like(packed)
    P.medusa_pack_codes_i4(_dev(codes), _dev(scales, dtype), _dev(points) if zeros else None, group, same, n)
    assert torch.equal(packed, same)
    y = torch.empty(k, n, dtype=torch.float32, device=DEV)
    P.medusa_linear_i4(torch.eye(k, dtype=TD[dtype], device=DEV), packed, group, zeros, y, _ws(P.medusa_linear_i4_workspace_bytes, k, n, k))
    assert np.array_equal(_np(y).T, rows4.values(codes, scales, points if zeros else None, group))


@pytest.mark.parametrize("dtype,group,zeros", KINDS)
def test_stacked_matrices(dtype, group, zeros):
    """Matrices packed one behind the other are one matrix."""
    rng = _rng(7, group)
    k, heights = 260, (48, 16, 21)
    w = _dev(rng.standard_normal((sum(heights), k)).astype(np.float32), dtype)
    size = P.medusa_packed_i4_bytes(sum(heights), k, group, zeros)
    whole, parts = (torch.zeros(size, dtype=torch.uint8, device=DEV) for _ in range(2))
    P.medusa_pack_weight_i4(w, group, whole, sum(heights), zeros=zeros)
    at = 0
    for h in heights:
        P.medusa_pack_weight_i4(w[at:at + h], group, parts, sum(heights), at // P.MDZ_I4_TILE_ROWS, zeros=zeros)
        at += h
    assert torch.equal(whole, parts)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("k", [256, 261])
def test_rows_that_are_not_finite_stay_alone(dtype, zeros, k):
    rng = _rng(9, k)
    m = Matrix(rng, 40, k, 64, zeros, dtype)
    x = _dev(rng.standard_normal((20, k)).astype(np.float32), dtype)
    clean = linear(x, m, 64, 40, "fp32").clone()
    x[3, 17], x[5, k - 1], x[18, 0] = float("nan"), float("inf"), float("-inf")
    got = linear(x, m, 64, 40, "fp32")
    for r in range(20):
        if r in (3, 5, 18):
            w = m.values[:, {3: 17, 5: k - 1, 18: 0}[r]]
            assert not torch.isfinite(got[r]).cpu().numpy()[w != 0].any()
        else:
            assert torch.equal(got[r], clean[r])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_group_that_is_not_finite(dtype):
    w = torch.randn(20, 256, device=DEV, dtype=TD[dtype])
    w[2, 70], w[11, 200] = float("nan"), float("inf")
    for zeros in (False, True):
        packed = torch.empty(P.medusa_packed_i4_bytes(20, 256, 64, zeros), dtype=torch.uint8, device=DEV)
        P.medusa_pack_weight_i4(w, 64, packed, 20, zeros=zeros)
        y = torch.empty(5, 20, device=DEV)
        P.medusa_linear_i4(torch.randn(5, 256, device=DEV, dtype=TD[dtype]), packed, 64, zeros, y, _ws(P.medusa_linear_i4_workspace_bytes, 5, 20, 256))
        bad = torch.isnan(y)
        assert bad[:, [2, 11]].all() and int(bad.sum()) == 10


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,n,k", [(3, 50, 256), (40, 81, 390)])
def test_rows_and_outputs_that_start_on_any_element(dtype, rows, n, k):
    rng = _rng(rows, 3)
    m = Matrix(rng, n, k, 32, True, dtype)
    x = _dev(rng.standard_normal((rows, k)).astype(np.float32), dtype)
    want = linear(x, m, 32, n, dtype)
    for shift in (1, 3):
        room = torch.empty(rows * k + shift, dtype=TD[dtype], device=DEV)[shift:].view(rows, k).copy_(x)
        out = torch.empty(rows * n + shift, dtype=TD[dtype], device=DEV)[shift:].view(rows, n)
        P.medusa_linear_i4(room, m.packed, 32, True, out, _ws(P.medusa_linear_i4_workspace_bytes, rows, n, k))
        assert torch.equal(out, want)


def test_a_row_does_not_depend_on_its_neighbours_and_calls_repeat():
    """The same kernel, the same bits: a row alone among 16, and each call again."""
    rng = _rng(21)
    m = Matrix(rng, 300, 1000, 128, False, "bf16")
    x = _dev(rng.standard_normal((64, 1000)).astype(np.float32), "bf16")
    y = linear(x, m, 128, 300, "fp32").clone()
    assert torch.equal(linear(x, m, 128, 300, "fp32"), y)
    other = x.clone()
    other[:30] = 0
    assert torch.equal(linear(other, m, 128, 300, "fp32")[30:], y[30:])


def test_no_rows():
    rng = _rng(5)
    m = Matrix(rng, 32, 64, 64, False, "bf16")
    P.medusa_linear_i4(torch.empty(0, 64, dtype=torch.bfloat16, device=DEV), m.packed, 64, False, torch.empty(0, 32, device=DEV))
    P.medusa_swiglu_i4(torch.empty(0, 64, dtype=torch.bfloat16, device=DEV), m.packed, m.packed, 64, False, torch.empty(0, 32, dtype=torch.bfloat16, device=DEV))


def test_on_another_stream_and_in_a_graph():
    rng = _rng(31)
    n, k, group = 500, 1408, 128
    gate, up = Matrix(rng, n, k, group, False, "bf16"), Matrix(rng, n, k, group, False, "bf16")
    down = Matrix(rng, 200, n, group, False, "bf16")
    for rows in (1, 64, 150):
        x = _dev(rng.standard_normal((rows, k)).astype(np.float32), "bf16")
        u, y = torch.empty(rows, n, dtype=torch.bfloat16, device=DEV), torch.empty(rows, 200, device=DEV)
        ws = torch.empty(max(P.medusa_swiglu_i4_workspace_bytes(rows, n, k), P.medusa_linear_i4_workspace_bytes(rows, 200, n)), dtype=torch.uint8, device=DEV)

        def block():
            P.medusa_swiglu_i4(x, gate.packed, up.packed, group, False, u, ws)
            P.medusa_linear_i4(u, down.packed, group, False, y, ws)
        block()
        want = y.clone()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            block()
        for _ in range(3):
            y.zero_(), u.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)
        y.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            block()
        side.synchronize()
        assert torch.equal(y, want)
