"""The 8-bit integer operators on the GPU against their definitions (oracle/rows8.py), at the sizes and values where they can go wrong."""
import numpy as np
import pytest
import torch

import paper_2603_03383_amd as P
from oracle import rows8

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TD = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# half a step of a type, relative to the value, and (binary16 alone reaches it here) half its smallest step
HALF = {"bf16": (2.0 ** -8, 0.0), "fp16": (2.0 ** -11, 2.0 ** -25), "fp32": (2.0 ** -24, 0.0)}
GUARD = 3  # rows behind the last, which no call may write


def _np(t):
    return t.detach().float().cpu().numpy()


def _gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def _normal(gen, *shape, std=1.0, dtype=torch.float32):
    return torch.empty(*shape, device=DEV).normal_(0.0, std, generator=gen).to(dtype)


class Out:
    """Outputs of a row operator, with guard rows behind them."""

    def __init__(self, rows, d, dtype, values=True):
        self.rows = rows
        self.all = [torch.full((rows + GUARD, d), 77, dtype=torch.int8, device=DEV), torch.full((rows + GUARD,), 7.5, device=DEV),
                    torch.full((rows + GUARD, d), 7.5, dtype=TD[dtype], device=DEV) if values else None]
        self.codes, self.scales, self.values = (None if t is None else t[:rows] for t in self.all)

    def check_guard(self):
        for t, v in zip(self.all, (77, 7.5, 7.5)):
            assert t is None or bool((t[self.rows:] == v).all())


def _odd_rows(t):
    """Some rows that have no scale or an unusual one."""
    n, d = t.shape
    if n >= 8:
        t[1] = 0
        t[2, d // 2] = float("nan")
        t[3, d - 1] = float("inf")
        t[4, 0] = float("-inf")
        t[5] *= 1e-30
        t[6] = -0.0
    return t


def check_rows(o, codes, scales, dtype, scale_steps):
    """Codes are the definition's, scales within scale_steps half steps of fp32 of it, values the product rounded."""
    got_codes, got_scales = o.codes.cpu().numpy(), o.scales.cpu().numpy().astype(np.float64)
    assert np.array_equal(got_codes, codes)
    assert np.array_equal(np.isnan(got_scales), np.isnan(scales))
    fine = np.isfinite(scales)
    assert (np.abs(got_scales - scales)[fine] <= scale_steps * 2.0 ** -24 * np.abs(scales)[fine] + 2.0 ** -149).all()
    if o.values is not None:
        v = got_codes.astype(np.float64) * got_scales[:, None]
        rel, least = HALF[dtype]
        got = _np(o.values).astype(np.float64)
        assert np.array_equal(np.isnan(got), np.isnan(v))
        with np.errstate(invalid="ignore"):
            # the product is rounded to fp32 first (its smallest step: 2^-149), then to the type
            assert not (np.abs(got - v) > np.abs(v) * (rel * (1 + 2.0 ** -23) + 2.0 ** -24) + least + 2.0 ** -148).any()
    o.check_guard()


ROW_SHAPES = [(1, 1), (3, 2), (9, 5), (8, 64), (64, 256), (15, 688), (90, 1387), (1, 4096), (64, 4096), (33, 5120), (8, 8192), (9, 8193),
              (8, 11008), (8, 16388), (3, 40001)]


@pytest.mark.parametrize("rows,d", ROW_SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_quantize_rows(dtype, rows, d):
    src = _odd_rows(_normal(_gen(rows * d), rows, d)).to(TD[dtype])
    o = Out(rows, d, dtype)
    P.medusa_quantize_rows_i8(src, o.codes, o.scales, o.values)
    codes, scales = rows8.quantize_rows(_np(src))
    check_rows(o, codes, scales.astype(np.float64), dtype, 0)


@pytest.mark.parametrize("rows,d", ROW_SHAPES)
@pytest.mark.parametrize("dtype,delta", [("bf16", "fp32"), ("bf16", "bf16"), ("fp16", "fp16"), ("fp16", None), ("fp32", "fp32")])
def test_residual_rmsnorm(dtype, delta, rows, d):
    g = _gen(rows * d + 1)
    x = _odd_rows(_normal(g, rows, d, std=3.0))
    dl = None if delta is None else _normal(g, rows, d, std=0.3, dtype=TD[delta])
    gain = (1 + _normal(g, d, std=0.3)).to(TD[dtype])
    o = Out(rows, d, dtype)
    x_all = torch.full((rows + GUARD, d), 7.5, device=DEV)
    x_out = x_all[:rows]
    P.medusa_residual_rmsnorm_i8(x, dl, gain, 1e-5, x_out, o.codes, o.scales, o.values)
    x_ref, codes, scales = rows8.rmsnorm_rows(_np(x), None if dl is None else _np(dl), _np(gain), 1e-5)
    assert np.array_equal(_np(x_out), x_ref, equal_nan=True) and bool((x_all[rows:] == 7.5).all())
    # d squares, each rounded and summed in chains of at most d / 64 + 16 additions, halved by the root; the mean, eps, root, reciprocal, the
    # scale's two factors: six more roundings
    check_rows(o, codes, scales, dtype, d / 128 + 16)
    # in place, without the values, and without the sum: the same codes and scales
    again, bare = Out(rows, d, dtype, values=False), Out(rows, d, dtype, values=False)
    P.medusa_residual_rmsnorm_i8(x, dl, gain, 1e-5, None, bare.codes, bare.scales)
    P.medusa_residual_rmsnorm_i8(x, dl, gain, 1e-5, x, again.codes, again.scales)
    assert np.array_equal(_np(x), x_ref, equal_nan=True)
    for other in (again, bare):
        assert torch.equal(other.codes, o.codes) and np.array_equal(_np(other.scales), _np(o.scales), equal_nan=True)
        other.check_guard()


def test_norm_of_large_and_small_rows():
    """eps decides rows far below it; a zero row with eps = 0 stays zero."""
    x = torch.tensor([[1e-12, -2e-12, 3e-12, 0], [0, 0, 0, 0], [1e15, -1e15, 5e14, 0]], device=DEV)
    gain = torch.tensor([1, 0.5, -2, 1], dtype=torch.bfloat16, device=DEV)
    for eps in (1e-5, 0.0):
        o = Out(3, 4, "bf16")
        P.medusa_residual_rmsnorm_i8(x, None, gain, eps, None, o.codes, o.scales, o.values)
        with np.errstate(divide="ignore"):
            _, codes, scales = rows8.rmsnorm_rows(_np(x), None, _np(gain), eps)
        assert np.array_equal(o.codes.cpu().numpy(), codes)
        fine = [0, 2] if eps == 0 else [0, 1, 2]  # (the zero row's codes are zero; its scale is then of no account)
        assert np.allclose(_np(o.scales)[fine], scales[fine], rtol=16 * 2.0 ** -24, atol=0)


@pytest.mark.parametrize("rows,ffn", [(1, 1), (3, 2), (9, 5), (8, 64), (64, 688), (7, 1387), (1, 11008), (65, 11008), (8, 12800), (8, 13824),
                                      (9, 16385), (3, 40001)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_swiglu(dtype, rows, ffn):
    g = _gen(rows * ffn + 2)
    gu = _odd_rows(_normal(g, rows, 2 * ffn, std=2.0)).to(TD[dtype])
    if rows >= 8:
        gu[7, 0], gu[7, ffn] = -200.0, 1.0  # the sigmoid of a gate far below zero underflows
    o = Out(rows, ffn, dtype)
    P.medusa_swiglu_i8(gu, o.codes, o.scales, o.values)
    with np.errstate(all="ignore"):
        t = rows8.swiglu_rows(_np(gu))
    bad = ~np.isfinite(t).all(axis=1)
    amax = np.where(bad, 0, np.abs(np.where(np.isfinite(t), t, 0)).max(axis=1))
    scales = np.where(amax / 127 > 2.0 ** -149, amax / 127, 1.0)
    got_scales, got = o.scales.cpu().numpy().astype(np.float64), o.codes.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isnan(got_scales), bad) and not got[bad].any()
    ok = ~bad
    # Relative error of a value in half steps of fp32: the exponential 4 (two of its last bits), which the sum can pass on whole, the sum, the
    # quotient and the product 1 each: 7; the scale has its own rounding too.  Values below fp32's normal range have its smallest steps.
    small = np.abs(_np(gu)).max(axis=1) < 1e-20
    assert (np.abs(got_scales - scales)[ok] <= 8 * 2.0 ** -24 * scales[ok] + 2.0 ** -147).all()
    # a code is within half a step of the value over the scale, both as the kernel has them: up to 127 steps with 7 + 8 + 1 half steps of error
    quot = t[ok & ~small] / scales[ok & ~small, None]
    assert (np.abs(got[ok & ~small] - quot) <= 0.5 + 127 * 16 * 2.0 ** -24).all()
    check_rows(o, o.codes.cpu().numpy(), np.where(bad, np.nan, scales), dtype, 8 + (2.0 ** 24 if small.any() else 0))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_swiglu_of_extreme_gates(dtype):
    """Gates where the exponential overflows, vanishes or its argument is infinite: the sigmoid is 0 or 1."""
    big = float(torch.finfo(TD[dtype]).max)
    gate = torch.tensor([[big, -big, 1e5, -1e5, 90.0, -90.0, 0.0, -0.0], [-big, -1e30, -500.0, -200.0, -1e5, -1e10, -300.0, 0.0]], device=DEV)
    up = torch.tensor([[1.0, 1.0, -1.0, 1.0, 2.0, 1.0, 5.0, 5.0], [1.0, -1.0, 1.0, 3.0, 1.0, 1.0, 1.0, 7.0]], device=DEV)
    gu = torch.cat([gate, up], dim=1).to(TD[dtype])
    o = Out(2, 8, dtype)
    P.medusa_swiglu_i8(gu, o.codes, o.scales, o.values)
    assert o.codes.cpu().numpy().tolist() == [[127, 0, 0, 0, 0, 0, 0, 0], [0] * 8]
    # row 1 holds nothing above 200 e^-200, which fp32 does not have
    assert abs(float(o.scales[0]) / (float(gu[0, 0]) / 127) - 1) < 2.0 ** -22 and float(o.scales[1]) == 1.0
    o.check_guard()


def make_linear(m, n, k, seed=0, offset=0, full=False):
    """Codes of bell-shaped rows (or extreme ones), the rows starting `offset` bytes behind an aligned address; the packed matrix."""
    g = _gen(seed + m + 3 * n + 7 * k)
    if full:
        codes = lambda r: torch.full((r, k), -128, dtype=torch.int8, device=DEV)  # noqa: E731
    else:
        codes = lambda r: _normal(g, r, k, std=40).round().clamp(-128, 127).to(torch.int8)  # noqa: E731
    flat = torch.full((m * k + offset + 64,), 55, dtype=torch.int8, device=DEV)
    x = flat[offset:offset + m * k].view(m, k)
    x.copy_(codes(m))
    w = codes(n)
    sx, sw = (0.5 + torch.rand(r, device=DEV, generator=g) for r in (m, n))
    packed = torch.full((P.medusa_packed_i8_bytes(n, k),), 33, dtype=torch.uint8, device=DEV)
    P.medusa_pack_codes_i8(w, sw / 64, packed, n)
    return x, sx, w, sw / 64, packed


def workspace(m, n, k):
    """Exactly the bytes asked for, full of ones: nothing in it has to be set."""
    return torch.full((P.medusa_linear_i8_workspace_bytes(m, n, k),), 255, dtype=torch.uint8, device=DEV)


def check_linear(x, sx, w, sw, packed, out):
    m, n = x.shape[0], w.shape[0]
    y_all = torch.full((m * n + 64,), 7.5, dtype=TD[out], device=DEV)
    y = y_all[:m * n].view(m, n)
    P.medusa_linear_i8(x, sx, packed, y, workspace(m, n, x.shape[1]))
    sums = (x.double() @ w.double().t().contiguous()) if m * n * x.shape[1] > 1 << 28 else \
        torch.from_numpy(rows8.linear(x.cpu().numpy(), np.ones(m), w.cpu().numpy(), np.ones(n))[0]).to(DEV)
    ref = sums * sx.double()[:, None] * sw.double()
    rel, least = HALF[out]
    # the sum, the scales' product and the two multiplied: three roundings in fp32, then the output's
    err = (y.double() - ref).abs() - ref.abs() * (3.001 * 2.0 ** -24 + (0 if out == "fp32" else rel)) - least
    assert float(err.max()) <= 0
    assert bool((y_all[m * n:] == 7.5).all())
    return y


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 16, 16), (2, 17, 5), (15, 100, 63), (16, 64, 64), (17, 40, 65), (33, 129, 127), (64, 256, 128),
                                   (64, 1000, 1387), (1, 6144, 4096), (48, 300, 688), (64, 4096, 4096), (65, 272, 256), (90, 1024, 512),
                                   (97, 33, 100), (128, 129, 192), (129, 512, 1024), (200, 1000, 1000), (257, 513, 384), (300, 64, 8192),
                                   (500, 2048, 640), (1030, 700, 256)])
@pytest.mark.parametrize("out", ["fp32", "bf16", "fp16"])
def test_linear(out, m, n, k):
    check_linear(*make_linear(m, n, k), out)


# (tile rows, tile columns, parts of K) that a product of (rows, columns) over about so many features is cut into: every tile, whole and in parts
PLANS = [((16, 16, 1), (1, 50, 1150)), ((16, 32, 1), (9, 4305, 1150)), ((16, 48, 1), (16, 8355, 1150)), ((32, 16, 1), (17, 30, 1150)),
         ((32, 32, 1), (33, 47, 1146)), ((32, 32, 4), (33, 17, 2645)), ((32, 48, 1), (17, 8327, 1109)), ((64, 48, 1), (33, 8575, 1117)),
         ((64, 48, 6), (36, 1453, 2968)), ((64, 64, 1), (65, 6478, 1113)), ((64, 64, 8), (35, 1553, 4743)), ((64, 96, 1), (67, 8235, 1131)),
         ((64, 96, 8), (33, 2082, 4082)), ((96, 64, 1), (65, 11657, 1136)), ((96, 64, 8), (69, 1697, 4932)), ((128, 64, 1), (97, 12831, 1127)),
         ((128, 64, 6), (2053, 99, 5274)), ((128, 128, 1), (65, 17990, 1112)), ((128, 128, 8), (66, 2739, 7967)),
         ((256, 128, 1), (131, 18221, 1136)), ((256, 128, 3), (138, 8408, 6439)), ((256, 192, 1), (268, 21467, 1122)),
         ((256, 192, 2), (130, 18164, 5058))]


@pytest.mark.parametrize("plan,shape", PLANS)
def test_linear_every_tile(plan, shape):
    """More stages than any ring has, row and column blocks that end inside a tile; features that end inside a cache line, and rows that
    start anywhere and go through the workspace."""
    m, n, k = shape
    for k in (k // 16 * 16 + 16, k | 1):
        got = P.medusa_linear_i8_plan(m, n, k)
        assert (got["tile_rows"], got["tile_cols"], got["k_splits"]) == plan
        check_linear(*make_linear(m, n, k), "bf16")


@pytest.mark.parametrize("m,n,k,offset", [(3, 33, 100, 1), (64, 256, 256, 4), (64, 512, 4096, 8), (70, 256, 256, 1), (200, 512, 1024, 3),
                                          (300, 256, 1001, 15)])
def test_linear_rows_off_alignment(m, n, k, offset):
    check_linear(*make_linear(m, n, k, offset=offset), "fp32")


@pytest.mark.parametrize("out", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("m,n,k", [(1, 61, 128), (5, 64, 100), (24, 47, 256), (33, 17, 2645), (70, 258, 1024), (130, 1003, 256), (300, 769, 512)])
def test_linear_into_outputs_that_start_anywhere(out, m, n, k):
    """Four columns leave as one store from any element's address: the same results bit for bit, and nothing around them is written."""
    x, sx, w, sw, packed = make_linear(m, n, k)
    want = torch.empty(m, n, dtype=TD[out], device=DEV)
    P.medusa_linear_i8(x, sx, packed, want, workspace(m, n, k))
    for first in (1, 2, 3):
        buf = torch.full((first + m * n + 8,), 7.5, dtype=TD[out], device=DEV)
        P.medusa_linear_i8(x, sx, packed, buf[first:first + m * n].view(m, n), workspace(m, n, k))
        assert torch.equal(buf[first:first + m * n].view(m, n), want)
        assert bool((buf[:first] == 7.5).all()) and bool((buf[first + m * n:] == 7.5).all())


@pytest.mark.parametrize("m", [1, 64, 130])
def test_linear_largest_sum(m):
    """-128 times -128 over the longest row: 2^31 - 16384, the largest sum there can be."""
    x, sx, w, sw, packed = make_linear(m, 16, 131071, full=True)
    y = check_linear(x, sx, w, sw, packed, "fp32")
    assert float((y / (sx[:, None] * sw)).min()) > 2.147e9


@pytest.mark.parametrize("n,k", [(700, 1024), (4096, 4096), (130, 1000)])
def test_linear_rows_do_not_depend_on_the_batch(n, k):
    x, sx, w, sw, packed = make_linear(513, n, k)
    whole = torch.empty(513, n, device=DEV)
    P.medusa_linear_i8(x, sx, packed, whole, workspace(513, n, k))
    for m in (1, 9, 16, 40, 64, 65, 96, 128, 160, 300):
        y = torch.empty(m, n, device=DEV)
        P.medusa_linear_i8(x[:m], sx[:m], packed, y, workspace(m, n, k))
        assert torch.equal(y, whole[:m]), m


def test_offsets_beyond_32_bits():
    """More than 2^32 codes in a batch's rows, and in a matrix: the last rows are right, from the row kernels through the product."""
    rows, k, n = 270_000, 16_384, 48
    src = torch.empty(rows, k, dtype=torch.bfloat16, device=DEV).fill_(1.0)
    tail = _normal(_gen(1), 5, k, dtype=torch.bfloat16)
    src[-5:] = tail
    codes, scales = torch.empty(rows, k, dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    P.medusa_quantize_rows_i8(src, codes, scales)
    del src
    want, want_scales = rows8.quantize_rows(_np(tail))
    assert np.array_equal(codes[-5:].cpu().numpy(), want) and np.array_equal(_np(scales[-5:]), want_scales)
    assert bool((codes[:-5] == 127).all())
    _, _, w, sw, packed = make_linear(1, n, k)
    y = torch.empty(rows, n, device=DEV)
    P.medusa_linear_i8(codes, scales, packed, y, workspace(rows, n, k))
    ref = rows8.linear(want, want_scales, w.cpu().numpy(), sw.cpu().numpy())[1]
    assert np.abs(_np(y[-5:]) - ref).max() <= 3.001 * 2.0 ** -24 * np.abs(ref).max()
    assert bool((y[:-5] == y[0]).all())
    # the same codes as weights: rows of the matrix beyond 2^32
    packed = torch.empty(P.medusa_packed_i8_bytes(rows, k), dtype=torch.uint8, device=DEV)
    P.medusa_pack_codes_i8(codes, scales, packed, rows)
    x, sx = w[:40].contiguous(), sw[:40].contiguous()
    for m in (3, 40):
        y = torch.empty(m, rows, device=DEV)
        P.medusa_linear_i8(x[:m], sx[:m], packed, y, workspace(m, rows, k))
        assert np.abs(_np(y[:, -5:]) - ref[:, :m].T).max() <= 3.001 * 2.0 ** -24 * np.abs(ref).max()
        assert bool((y[:, :-5] == y[:, :1]).all())


def test_linear_of_rows_without_a_scale():
    """A row that had a NaN comes out NaN, a weight row too; their neighbours are untouched."""
    src = _normal(_gen(4), 20, 256)
    src[3, 7] = float("nan")
    w = _normal(_gen(5), 40, 256, std=0.02, dtype=torch.bfloat16)
    w[11, 0] = float("inf")
    codes, scales = torch.empty(20, 256, dtype=torch.int8, device=DEV), torch.empty(20, device=DEV)
    P.medusa_quantize_rows_i8(src, codes, scales)
    packed = torch.empty(P.medusa_packed_i8_bytes(40, 256), dtype=torch.uint8, device=DEV)
    P.medusa_pack_weight_i8(w, packed, 40)
    y = torch.empty(20, 40, device=DEV)
    P.medusa_linear_i8(codes, scales, packed, y, workspace(20, 40, 256))
    nan = torch.isnan(y)
    assert bool(nan[3].all()) and bool(nan[:, 11].all()) and int(nan.sum()) == 20 + 40 - 1


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,k", [(1, 1), (33, 100), (256, 1387), (48, 4096)])
def test_pack_weight_is_the_quantiser_and_matrices_stack(dtype, n, k):
    """A stack of matrices multiplied with unit rows gives the weights' rows in 8 bits back."""
    g = _gen(n + k)
    first, last = _normal(g, 32, k, std=0.02, dtype=TD[dtype]), _odd_rows(_normal(g, n, k, std=0.02)).to(TD[dtype])
    total = 32 + n
    packed = torch.full((P.medusa_packed_i8_bytes(total, k),), 99, dtype=torch.uint8, device=DEV)
    P.medusa_pack_weight_i8(first, packed, total)
    P.medusa_pack_weight_i8(last, packed, total, 32 // P.MDZ_I8_TILE_ROWS)
    codes, scales = rows8.quantize_rows(np.concatenate([_np(first), _np(last)]))
    by_codes = torch.full_like(packed, 44)
    P.medusa_pack_codes_i8(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), by_codes, total)
    assert torch.equal(packed, by_codes)
    some = sorted({0, k // 2, k - 1})
    x = torch.zeros(len(some), k, dtype=torch.int8, device=DEV)
    for r, c in enumerate(some):
        x[r, c] = 1
    y = torch.empty(len(some), total, device=DEV)
    P.medusa_linear_i8(x, torch.ones(len(some), device=DEV), packed, y, workspace(len(some), total, k))
    assert np.array_equal(y.cpu().numpy(), (codes[:, some].astype(np.float32) * scales[:, None]).T, equal_nan=True)


def test_no_rows():
    g = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    o = Out(0, 64, "bf16")
    P.medusa_quantize_rows_i8(torch.empty(0, 64, device=DEV, dtype=torch.bfloat16), o.codes, o.scales, o.values)
    P.medusa_residual_rmsnorm_i8(torch.empty(0, 64, device=DEV), None, g, 1e-5, None, o.codes, o.scales, o.values)
    P.medusa_swiglu_i8(torch.empty(0, 128, device=DEV, dtype=torch.bfloat16), o.codes, o.scales, o.values)
    _, _, _, _, packed = make_linear(1, 32, 64)
    P.medusa_linear_i8(torch.empty(0, 64, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV), packed, torch.empty(0, 32, device=DEV))
    torch.cuda.synchronize()
    o.check_guard()


def block(x, gain, w_gate_up, w_down, buf):
    """A feed-forward block out of the operators, as a layer has it: norm, product, SwiGLU, product, residual."""
    rows, ffn = x.shape[0], buf["ffn"]
    P.medusa_residual_rmsnorm_i8(x, None, gain, 1e-5, None, buf["c1"], buf["s1"])
    P.medusa_linear_i8(buf["c1"], buf["s1"], w_gate_up, buf["gu"], buf["ws"])
    P.medusa_swiglu_i8(buf["gu"], buf["c2"], buf["s2"])
    P.medusa_linear_i8(buf["c2"], buf["s2"], w_down, buf["y"], buf["ws"])
    P.medusa_residual_rmsnorm_i8(x, buf["y"], gain, 1e-5, x, buf["c1"], buf["s1"], buf["v"])
    return x, buf["v"]


def make_block(rows, d, ffn, seed=1):
    g = _gen(seed)
    wgu, wd = _normal(g, 2 * ffn, d, std=0.02, dtype=torch.bfloat16), _normal(g, d, ffn, std=0.02, dtype=torch.bfloat16)
    packed = []
    for w in (wgu, wd):
        packed.append(torch.empty(P.medusa_packed_i8_bytes(*w.shape), dtype=torch.uint8, device=DEV))
        P.medusa_pack_weight_i8(w, packed[-1], w.shape[0])
    ws = max(P.medusa_linear_i8_workspace_bytes(rows, 2 * ffn, d), P.medusa_linear_i8_workspace_bytes(rows, d, ffn))
    e = lambda *s, dtype=torch.float32: torch.empty(*s, device=DEV, dtype=dtype)  # noqa: E731
    buf = dict(ffn=ffn, c1=e(rows, d, dtype=torch.int8), s1=e(rows), gu=e(rows, 2 * ffn, dtype=torch.bfloat16), c2=e(rows, ffn, dtype=torch.int8),
               s2=e(rows), y=e(rows, d), v=e(rows, d, dtype=torch.bfloat16), ws=torch.empty(ws, dtype=torch.uint8, device=DEV))
    gain = (1 + _normal(g, d, std=0.3)).to(torch.bfloat16)
    return gain, wgu, wd, packed[0], packed[1], buf


def block_reference(x, gain, wgu, wd):
    """The same block in 64 bits on the 8-bit weights, activations unquantised."""
    f = lambda t: torch.from_numpy(rows8.roundtrip_rows(_np(t))).to(DEV)  # noqa: E731
    x = x.double()
    norm = lambda v: v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-5) * gain.double()  # noqa: E731
    gate, up = (norm(x) @ f(wgu).t().contiguous()).chunk(2, dim=1)
    x = x + (gate * torch.sigmoid(gate) * up) @ f(wd).t().contiguous()
    return x, norm(x)


@pytest.mark.parametrize("rows,d,ffn", [(1, 512, 1376), (64, 1024, 2816), (90, 512, 1387), (300, 1024, 2816)])
def test_a_feed_forward_block(rows, d, ffn):
    gain, wgu, wd, p1, p2, buf = make_block(rows, d, ffn)
    x0 = _normal(_gen(9), rows, d)
    want_x, want_v = block_reference(x0, gain, wgu, wd)
    got_x, got_v = block(x0.clone(), gain, p1, p2, buf)
    # A code is off by up to half a step of max / 127: uniform, so 1 / sqrt(12) of a step; rows of bell-shaped numbers have their largest at
    # under 4.5 standard deviations, products of them under 12: 4.5 / 127 / sqrt(12) = 1.0 % and 12 / 127 / sqrt(12) = 2.7 % of the activations' norm
    # reach the two products.  The first product's 1.0 % (of gate and of up alike) and the second's 2.7 % add in squares: under 3.1 % of the update.
    assert float((got_x.double() - want_x).norm() / (want_x - x0).norm()) < 0.031
    # the values that follow add 1.0 % of their own; the update is a part of x
    assert float((got_v.double() - want_v).norm() / want_v.norm()) < 0.031 + 0.011


def test_captured_and_replayed_on_another_stream():
    """The block in a graph, replayed with other inputs and the program's own work between, against eager calls; scratch shared by two graphs."""
    rows, d, ffn = 64, 1024, 2816
    gain, wgu, wd, p1, p2, buf = make_block(rows, d, ffn)
    few = dict(buf, **{k: torch.empty_like(buf[k][:5]) for k in ("c1", "s1", "gu", "c2", "s2", "y", "v")})
    x, x5 = torch.empty(rows, d, device=DEV), torch.empty(5, d, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(x.normal_(), gain, p1, p2, buf)
        block(x5.normal_(), gain, p1, p2, few)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for xs, b in ((x, buf), (x5, few)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            block(xs, gain, p1, p2, b)
    for trip in range(4):
        x0, x50 = _normal(_gen(20 + trip), rows, d), _normal(_gen(30 + trip), 5, d)
        x.copy_(x0), x5.copy_(x50)
        graphs[0].replay()
        got = x.clone(), buf["v"].clone()
        graphs[1].replay()
        got5 = x5.clone(), few["v"].clone()
        buf["ws"].fill_(trip)  # nothing is kept in the scratch
        torch.cuda.synchronize()
        for start, g, b in ((x0, got, buf), (x50, got5, few)):
            want = block(start.clone(), gain, p1, p2, b)
            assert torch.equal(g[0], want[0]) and torch.equal(g[1], want[1]), trip
