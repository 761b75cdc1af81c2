"""Grouped products, their gradients and their 8-bit form against the formulas in 64 bits.

Tolerances, per element, with S = the sum of absolute products behind it and D their number: fp32 sums of D products are
off by at most D 2^-24 S to first order, whatever the order of the additions (D + 8 here, for the terms behind it), and the rounding
to bf16 adds 2^-8 of the value (2^-8 is the type's half step).  The 8-bit matrix instruction adds the 128 products of a block with fewer
bits: 2^-12 of S, see the header; where all numbers are integers of at most four bits it has nothing to lose, and
only the additions of the blocks count."""
import math

import pytest
import torch

from paper_2501_10375_amd import moe, products

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
HALF_STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
UNTOUCHED = 7.25


def normal(*shape, dtype=F32, seed=0, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000 * seed + sum(shape))
    return (torch.randn(shape, device=DEV, generator=g) * std).to(dtype)


def table(counts, before=0):
    o = [before]
    for c in counts:
        o.append(o[-1] + c)
    return o, torch.tensor(o, dtype=torch.int32, device=DEV)


def workspace(E, N, K, dtype, rows):
    w = products.alloc_workspace(products.make_product(E, N, K, dtype), rows)
    return w.fill_(0x5A)


def check(got, want, size, depth, out_dtype, label):
    """got against want (64 bits) with size = S."""
    assert got.dtype == out_dtype
    tol = (depth + 8) * 2.0 ** -24 * size + HALF_STEP[out_dtype] * want.abs()
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all(), label
    worst = float((off / tol.clamp_min(1e-300)).max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{label}: {worst:.3g} times the tolerance"


def reference(form, o, a, b):
    """Blocks of the result and of S: forward/dgrad [(slice, value, size)] per expert, wgrad value and size [E, N, K]."""
    a, out = a.double(), []
    for e in range(len(o) - 1):
        r = slice(o[e], o[e + 1])
        if form == "wgrad":
            x = b[r].double()
            out.append((e, a[r].T @ x, a[r].abs().T @ x.abs()))
        else:
            m = b[e].double().T if form == "forward" else b[e].double()
            out.append((r, a[r] @ m, a[r].abs() @ m.abs()))
    return out


SHAPES = [   # rows of each expert, N, K, rows of nobody before and behind
    ([1], 64, 64, 0, 0),
    ([0, 1, 0], 128, 64, 0, 0),
    ([5, 0, 16, 17], 192, 320, 3, 6),
    ([33, 1, 0, 0, 64, 31, 2, 0], 512, 256, 0, 1),
    ([129, 257, 40], 320, 448, 2, 0),
    ([0, 0], 64, 128, 5, 4),
    ([700], 704, 576, 0, 0),
    ([2] * 64, 128, 192, 0, 0),
    ([3, 600, 0, 90], 256, 1088, 1, 1),
    ([1, 1], 4096, 1024, 0, 0),
    ([20, 3], 1024, 4096, 0, 0),
    ([300, 20, 1000], 1024, 512, 0, 7),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts,N,K,before,behind", SHAPES)
def test_products_and_gradients(counts, N, K, before, behind, dtype):
    E = len(counts)
    o, offsets = table(counts, before)
    R = o[-1] + behind
    x, dy = normal(R, K, dtype=dtype, seed=1), normal(R, N, dtype=dtype, seed=2)
    w = normal(E, N, K, dtype=dtype, seed=3)
    ws = workspace(E, N, K, dtype, R)
    nobody = [i for i in range(R) if i < o[0] or i >= o[-1]]
    y, dx = (torch.full((R, n), UNTOUCHED, dtype=dtype, device=DEV) for n in (N, K))
    products.moe_grouped_product(x, offsets, w, y, ws)
    products.moe_grouped_product_dgrad(dy, offsets, w, dx, ws)
    for form, got, a, depth in (("forward", y, x, K), ("dgrad", dx, dy, N)):
        assert (got[nobody] == UNTOUCHED).all(), form
        for r, want, size in reference(form, o, a, w):
            check(got[r], want, size, depth, dtype, f"{form} rows {r.start}-{r.stop}")
    want = reference("wgrad", o, dy, x)
    for out_dtype in {dtype, F32}:
        dw = torch.full((E, N, K), UNTOUCHED, dtype=out_dtype, device=DEV)
        products.moe_grouped_product_wgrad(dy, x, offsets, dw, False, ws)
        for e, value, size in want:
            check(dw[e], value, size, counts[e], out_dtype, f"wgrad {out_dtype} expert {e}")
    dw = normal(E, N, K, seed=4)
    old = dw.double()
    products.moe_grouped_product_wgrad(dy, x, offsets, dw, True, ws)
    for e, value, size in want:
        check(dw[e], old[e] + value, old[e].abs() + size, counts[e] + 1, F32, f"wgrad accumulated, expert {e}")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_one_expert_needs_no_table(dtype):
    R, N, K = 77, 192, 256
    x, dy, w = normal(R, K, dtype=dtype, seed=1), normal(R, N, dtype=dtype, seed=2), normal(1, N, K, dtype=dtype, seed=3)
    ws, (_, offsets) = workspace(1, N, K, dtype, R), table([R])
    out = []
    for o in (None, offsets):
        y, dx, dw = torch.empty(R, N, dtype=dtype, device=DEV), torch.empty(R, K, dtype=dtype, device=DEV), torch.empty(1, N, K, device=DEV)
        products.moe_grouped_product(x, o, w, y, ws)
        products.moe_grouped_product_dgrad(dy, o, w, dx, ws)
        products.moe_grouped_product_wgrad(dy, x, o, dw, False, ws)
        out.append((y, dx, dw))
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_no_rows():
    E, N, K = 3, 64, 128
    o = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    w, ws = normal(E, N, K, dtype=BF16), workspace(E, N, K, BF16, 0)
    x, y = torch.empty(0, K, dtype=BF16, device=DEV), torch.empty(0, N, dtype=BF16, device=DEV)
    products.moe_grouped_product(x, o, w, y, ws)
    products.moe_grouped_product_dgrad(y, o, w, x, ws)
    dw = torch.full((E, N, K), UNTOUCHED, device=DEV)
    products.moe_grouped_product_wgrad(y, x, o, dw, True, ws)
    assert (dw == UNTOUCHED).all()
    products.moe_grouped_product_wgrad(y, x, o, dw, False, ws)
    assert (dw == 0).all()


@pytest.mark.parametrize("values", [[-5, 3, 9], [0, 12, 4], [2, 40, 50], [20, 30, 40]])
def test_tables_out_of_range_stay_inside_the_buffers(values):
    """Values outside [0, rows] count as the nearer end, a range that ends before it begins as none: nothing is read or written outside."""
    R, E, N, K = 12, 2, 64, 64
    x, w, ws = normal(R, K, dtype=BF16, seed=1), normal(E, N, K, dtype=BF16, seed=3), workspace(E, N, K, BF16, R)
    y = torch.full((R + 64, N), UNTOUCHED, dtype=BF16, device=DEV)
    offsets = torch.tensor(values, dtype=torch.int32, device=DEV)
    products.moe_grouped_product(x, offsets, w, y[:R], ws)
    assert (y[R:] == UNTOUCHED).all()
    a, b, c = (min(max(v, 0), R) for v in values)
    if a <= b <= c:
        for e, r in enumerate((slice(a, b), slice(b, c))):
            m = w[e].double().T
            check(y[r], x[r].double() @ m, x[r].double().abs() @ m.abs(), K, BF16, f"expert {e}")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_not_a_number_stays_with_its_rows_and_expert(dtype):
    """NaN in a row, in an expert's matrix and behind the last row reach what the formulas say and nothing else."""
    counts, N, K = [20, 31, 45], 128, 192
    o, offsets = table(counts)
    R = o[-1] + 3
    x, dy, w = normal(R, K, dtype=dtype, seed=1), normal(R, N, dtype=dtype, seed=2), normal(3, N, K, dtype=dtype, seed=3)
    x[o[-1]:] = math.nan
    dy[o[-1]:] = math.inf
    x[25, 7] = math.nan           # a row of expert 1
    w[2, 70, 100] = math.inf      # feature 70 of expert 2
    ws = workspace(3, N, K, dtype, R)
    y, dx, dw = torch.zeros(R, N, dtype=dtype, device=DEV), torch.zeros(R, K, dtype=dtype, device=DEV), torch.zeros(3, N, K, device=DEV)
    products.moe_grouped_product(x, offsets, w, y, ws)
    products.moe_grouped_product_dgrad(dy, offsets, w, dx, ws)
    products.moe_grouped_product_wgrad(dy, x, offsets, dw, False, ws)
    bad = torch.zeros(R, N, dtype=torch.bool, device=DEV)
    bad[25], bad[o[2]:o[3], 70] = True, True
    assert torch.equal(~torch.isfinite(y), bad)
    bad = torch.zeros(R, K, dtype=torch.bool, device=DEV)
    bad[o[2]:o[3], 100] = True
    assert torch.equal(~torch.isfinite(dx), bad)
    bad = torch.zeros(3, N, K, dtype=torch.bool, device=DEV)
    bad[1, :, 7] = True
    assert torch.equal(~torch.isfinite(dw), bad)


def test_gradients_are_those_of_the_product():
    """d/dt of <dy, product(x + t u, w + t v)> by central differences in 64 bits on the formula, against the gradients."""
    counts, N, K = [9, 0, 30], 64, 128
    o, offsets = table(counts)
    R = o[-1]
    x, dy, w, u, v = (normal(*s, seed=i) for i, s in enumerate(((R, K), (R, N), (3, N, K), (R, K), (3, N, K))))
    ws = workspace(3, N, K, F32, R)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    products.moe_grouped_product_dgrad(dy, offsets, w, dx, ws)
    products.moe_grouped_product_wgrad(dy, x, offsets, dw, False, ws)

    def value(t):
        s = 0.0
        for e in range(3):
            r = slice(o[e], o[e + 1])
            s += float((dy[r].double() * ((x[r].double() + t * u[r].double()) @ (w[e].double() + t * v[e].double()).T)).sum())
        return s

    t = 2.0 ** -10   # (the function is of second degree in t: central differences are exact but for rounding)
    numeric = (value(t) - value(-t)) / (2 * t)
    analytic = float((dx.double() * u.double()).sum() + (dw.double() * v.double()).sum())
    size = float((dx.double() * u.double()).abs().sum() + (dw.double() * v.double()).abs().sum())
    assert abs(numeric - analytic) <= (N + K) * 2.0 ** -24 * size + 1e-9 * size


# ---- 8 bits

def e4m3_of(v):
    """float64 -> nearest e4m3 value, ties to even, by its definition."""
    _, ex = torch.frexp(v)
    step = ((ex.long() - 1).clamp_min(-6) - 3 + 1023).bitwise_left_shift(52).view(torch.float64)   # 2^n from its bits
    return torch.round(v / step) * step


def quantised(v, rows):
    """Values and scales of a matrix [R, K] in blocks of rows x 128, by the definition in 64 bits; both as float64."""
    R, K = v.shape
    pad = torch.nn.functional.pad(v.double(), (0, -K % 128, 0, -R % rows))
    b = pad.view(pad.shape[0] // rows, rows, pad.shape[1] // 128, 128)
    amax = b.abs().amax((1, 3))
    scale = (amax.clamp_min(2.0 ** -60) / 448).float().double()
    q = e4m3_of((b / scale[:, None, :, None]).float().double())
    return q.reshape(pad.shape)[:R, :K], scale


def same_bits(q, want):
    """e4m3 numbers (uint8) against their values: equal, zeros of either sign alike."""
    return torch.equal(q.view(torch.float8_e4m3fn).double(), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R,K", [(1, 64), (3, 128), (17, 192), (64, 4096), (1000, 704), (5, 14336)])
def test_rows_are_quantised_to_the_nearest(R, K, dtype):
    x = normal(R, K, seed=5) * torch.exp(3 * normal(R, 1, seed=6))
    x[0, : K // 2] = 0
    if R > 2:
        x[1] = 0                                     # blocks of zeros
        x[2] *= 2.0 ** -70                           # all below the least scale
    x = x.to(dtype)
    q = torch.full((R + 1, K), 0x55, dtype=torch.uint8, device=DEV)
    scales = torch.full((R + 1, -(-K // 128)), UNTOUCHED, device=DEV)
    products.moe_quantize_rows_fp8(x, q[:R], scales[:R])
    want, scale = quantised(x, 1)
    assert torch.equal(scales[:R].double(), scale)
    assert same_bits(q[:R], want)
    assert (q[R] == 0x55).all() and (scales[R] == UNTOUCHED).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("E,N,K", [(1, 64, 64), (2, 128, 192), (3, 320, 448), (1, 64, 1024), (2, 704, 128)])
def test_weights_are_quantised_to_the_nearest(E, N, K, dtype):
    w = normal(E, N, K, seed=7) * torch.exp(normal(E, N, 1, seed=8))
    w[0, :64, :64] = 0
    w = w.to(dtype)
    nb, kb = -(-N // 128), -(-K // 128)
    q, q_t = (torch.full(s, 0x55, dtype=torch.uint8, device=DEV) for s in ((E, N, K), (E, K, N)))
    scales, scales_t = torch.empty(E, nb, kb, device=DEV), torch.empty(E, kb, nb, device=DEV)
    products.moe_quantize_weights_fp8(w, q, scales, q_t, scales_t)
    for e in range(E):
        want, scale = quantised(w[e], 128)
        assert torch.equal(scales[e].double(), scale)
        assert same_bits(q[e], want)
    assert torch.equal(q_t, q.transpose(1, 2)) and torch.equal(scales_t, scales.transpose(1, 2))
    alone, s = torch.empty_like(q), torch.empty_like(scales)
    products.moe_quantize_weights_fp8(w, alone, s)
    assert torch.equal(alone, q) and torch.equal(s, scales)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_extreme_values_are_quantised(dtype):
    """Every e4m3 tie and its neighbours, the type's largest values, and blocks with infinities and NaN."""
    top = torch.finfo(dtype).max
    steps = torch.arange(0, 128 * 16, device=DEV, dtype=torch.float64).view(16, 128) * 2.0 ** -2   # up to 511.75, ties among them
    steps = steps.clamp_max(448)
    steps[:, 127] = 448                        # scale 1
    x = torch.cat([steps, -steps, steps * 2.0 ** -40, torch.full((1, 128), top, device=DEV, dtype=torch.float64)]).to(dtype)
    bad = torch.ones(3, 256, device=DEV, dtype=dtype)
    bad[0, 5], bad[1, 200], bad[2, 127] = math.inf, math.nan, -math.inf
    for v in (x, bad):
        q = torch.empty(v.shape, dtype=torch.uint8, device=DEV)
        scales = torch.empty(v.shape[0], v.shape[1] // 128, device=DEV)
        products.moe_quantize_rows_fp8(v, q, scales)
        values = q.view(torch.float8_e4m3fn).float()
        if v is x:
            want, scale = quantised(x, 1)
            assert torch.equal(scales.double(), scale) and torch.equal(values.double(), want)
        else:
            broken = torch.zeros(3, 2, dtype=torch.bool, device=DEV)
            broken[0, 0] = broken[1, 1] = broken[2, 0] = True
            assert torch.equal(torch.isnan(scales), broken)
            assert torch.equal(torch.isnan(values), broken.repeat_interleave(128, 1))


FP8_SHAPES = SHAPES + [([40, 0, 300], 384, 640, 2, 3), ([1000, 1000], 512, 896, 0, 0)]


@pytest.mark.parametrize("integers", [True, False])
@pytest.mark.parametrize("counts,N,K,before,behind", FP8_SHAPES)
def test_fp8_products(counts, N, K, before, behind, integers):
    E = len(counts)
    o, offsets = table(counts, before)
    R, kb, nb = o[-1] + behind, -(-K // 128), -(-N // 128)
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    if integers:
        xq, wq = (torch.randint(-15, 16, s, device=DEV, generator=g).float().to(torch.float8_e4m3fn) for s in ((R, K), (E, N, K)))
    else:
        xq, wq = ((torch.randn(s, device=DEV, generator=g) * 150).clamp(-448, 448).to(torch.float8_e4m3fn) for s in ((R, K), (E, N, K)))
    xs, ws_ = (torch.exp(torch.randn(s, device=DEV, generator=g)) for s in ((R, kb), (E, nb, kb)))
    y = torch.full((R, N), UNTOUCHED, dtype=BF16, device=DEV)
    products.moe_grouped_product_fp8(xq, xs, offsets, wq, ws_, y, workspace(E, N, K, BF16, R))
    assert all((y[i] == UNTOUCHED).all() for i in range(R) if i < o[0] or i >= o[-1])
    x = xq.double() * xs.double().repeat_interleave(128, 1)[:, :K]
    for e in range(E):
        r = slice(o[e], o[e + 1])
        m = wq[e].double() * ws_[e].double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
        want, size = x[r] @ m.T, x[r].abs() @ m.abs().T
        tol = (kb + 8) * 2.0 ** -24 * size + 2.0 ** -8 * want.abs() + (0 if integers else 2.0 ** -12) * size
        off = (y[r].double() - want).abs()
        assert torch.isfinite(y[r]).all()
        assert (off <= tol).all(), f"expert {e}: {float((off / tol).max()):.3g} times the tolerance"


def test_fp8_gradient_of_the_rows_through_the_transposed_weights():
    """dx of a product in 8 bits: the product of quantised dy with q_t and swapped features."""
    counts, N, K = [30, 0, 65], 320, 192
    o, offsets = table(counts)
    R = o[-1]
    w, dy = normal(3, N, K, dtype=BF16, seed=3), normal(R, N, dtype=BF16, seed=2)
    nb, kb = -(-N // 128), -(-K // 128)
    q, q_t = torch.empty(3, N, K, dtype=torch.uint8, device=DEV), torch.empty(3, K, N, dtype=torch.uint8, device=DEV)
    s, s_t = torch.empty(3, nb, kb, device=DEV), torch.empty(3, kb, nb, device=DEV)
    products.moe_quantize_weights_fp8(w, q, s, q_t, s_t)
    dq, ds = torch.empty(R, N, dtype=torch.uint8, device=DEV), torch.empty(R, nb, device=DEV)
    products.moe_quantize_rows_fp8(dy, dq, ds)
    dx = torch.empty(R, K, dtype=BF16, device=DEV)
    products.moe_grouped_product_fp8(dq, ds, offsets, q_t, s_t, dx, workspace(3, K, N, BF16, R))
    values = dq.view(torch.float8_e4m3fn).double() * ds.double().repeat_interleave(128, 1)[:, :N]
    for e in range(3):
        r = slice(o[e], o[e + 1])
        m = q[e].view(torch.float8_e4m3fn).double() * s[e].double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
        want, size = values[r] @ m, values[r].abs() @ m.abs()
        assert ((dx[r].double() - want).abs() <= (2.0 ** -12 + (nb + 8) * 2.0 ** -24) * size + 2.0 ** -8 * want.abs()).all()


def test_not_a_number_in_8_bits_stays_with_its_block():
    counts, N, K = [20, 31], 192, 320
    o, offsets = table(counts)
    R = o[-1]
    x, w = normal(R, K, dtype=BF16, seed=1), normal(2, N, K, dtype=BF16, seed=3)
    x[25, 200], w[0, 130, 3] = math.nan, math.inf
    xq, xs = torch.empty(R, K, dtype=torch.uint8, device=DEV), torch.empty(R, 3, device=DEV)
    wq, ws_ = torch.empty(2, N, K, dtype=torch.uint8, device=DEV), torch.empty(2, 2, 3, device=DEV)
    products.moe_quantize_rows_fp8(x, xq, xs)
    products.moe_quantize_weights_fp8(w, wq, ws_)
    y = torch.zeros(R, N, dtype=BF16, device=DEV)
    products.moe_grouped_product_fp8(xq, xs, offsets, wq, ws_, y, workspace(2, N, K, BF16, R))
    bad = torch.zeros(R, N, dtype=torch.bool, device=DEV)
    bad[25], bad[:20, 128:] = True, True     # a row; the features of a tile of expert 0's matrix
    assert torch.equal(torch.isnan(y), bad)
