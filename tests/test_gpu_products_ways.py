"""Grouped products at shapes that are known to reach each variant of the few-row kernel, with more rows of an expert than a pass serves, the longest
contractions of the small 8-bit tiles, and gradients of rows in 8 bits through every kernel (see test_products_rules.py for which shape takes
which).  Tolerances as in test_gpu_products.py."""
import math

import pytest
import torch

from paper_2501_10375_amd import products
from products_shapes import BEHIND_SMALL_FP8, FEW_ROWS_BF16, FEW_ROWS_FP8, GRADIENT_FP8, SMALL_FP8
from test_gpu_products import BF16, DEV, UNTOUCHED, check, normal, reference, table, workspace

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8
E4M3 = torch.float8_e4m3fn
FP8 = [shape for shape, _ in FEW_ROWS_FP8] + SMALL_FP8 + BEHIND_SMALL_FP8


def label(v):
    return "+".join(map(str, v)) if isinstance(v, list) and len(v) < 9 else f"{len(v)} experts" if isinstance(v, list) else None


def spread(m, rows, R, K):
    """Scales of blocks of rows x 128, one for each value, in 64 bits."""
    return m.double().repeat_interleave(rows, -2)[..., :R, :].repeat_interleave(128, -1)[..., :K]


@pytest.mark.parametrize("counts,N,K", [shape for shape, _ in FEW_ROWS_BF16], ids=label)
def test_few_rows(counts, N, K):
    E, (o, offsets) = len(counts), table(counts)
    R = o[-1]
    x, w = normal(R, K, dtype=BF16, seed=1), normal(E, N, K, dtype=BF16, seed=3)
    y = torch.full((R + 1, N), UNTOUCHED, dtype=BF16, device=DEV)
    products.moe_grouped_product(x, offsets, w, y[:R], workspace(E, N, K, BF16, R))
    assert (y[R] == UNTOUCHED).all()
    for r, want, size in reference("forward", o, x, w):
        check(y[r], want, size, K, BF16, f"rows {r.start}-{r.stop}")


@pytest.mark.parametrize("counts,N,K", [shape for shape, _ in FEW_ROWS_BF16], ids=label)
def test_not_a_number_stays_in_its_row_from_pass_to_pass(counts, N, K):
    """NaN in every expert's first row reaches no other, whichever pass that is in."""
    E, (o, offsets) = len(counts), table(counts)
    R = o[-1]
    x, w, ws = normal(R, K, dtype=BF16, seed=1), normal(E, N, K, dtype=BF16, seed=3), workspace(E, N, K, BF16, R)
    bad = torch.zeros(R, dtype=torch.bool, device=DEV)
    bad[[a for a, b in zip(o, o[1:]) if b > a]] = True
    want = torch.empty(R, N, dtype=BF16, device=DEV)
    products.moe_grouped_product(x, offsets, w, want, ws)
    x[bad, K // 2] = math.nan
    y = torch.empty_like(want)
    products.moe_grouped_product(x, offsets, w, y, ws)
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], want[~bad])


@pytest.mark.parametrize("counts,N,K", FP8, ids=label)
def test_8_bits(counts, N, K):
    """Integers of four bits, whose sums inside a block lose nothing: of 128 products below 2^8, multiples of one, an eight keeps 13 bits behind its largest."""
    E, (o, offsets) = len(counts), table(counts)
    R, kb, nb = o[-1], -(-K // 128), -(-N // 128)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    xq, wq = (torch.randint(-15, 16, s, device=DEV, generator=g).to(torch.float16).to(E4M3) for s in ((R, K), (E, N, K)))
    xs, wsc = (torch.exp(torch.randn(s, device=DEV, generator=g)) for s in ((R + 1, kb), (E, nb, kb)))
    xs[R] = math.nan
    y = torch.full((R + 1, N), UNTOUCHED, dtype=BF16, device=DEV)
    products.moe_grouped_product_fp8(xq, xs[:R], offsets, wq, wsc, y[:R], workspace(E, N, K, BF16, R))
    assert (y[R] == UNTOUCHED).all()
    x = xq.double() * spread(xs[:R], 1, R, K)
    for e in range(E):
        r = slice(o[e], o[e + 1])
        if counts[e]:
            m = wq[e].double() * spread(wsc[e], 128, N, K)
            check(y[r], x[r] @ m.T, x[r].abs() @ m.abs().T, kb, BF16, f"expert {e}")


@pytest.mark.parametrize("counts,N,K", FP8, ids=label)
def test_not_a_number_in_8_bits_stays_in_its_row_from_pass_to_pass(counts, N, K):
    E, (o, offsets) = len(counts), table(counts)
    R, kb, nb = o[-1], -(-K // 128), -(-N // 128)
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    xq, wq = (torch.randint(-15, 16, s, device=DEV, generator=g).to(torch.float16).to(E4M3) for s in ((R, K), (E, N, K)))
    xs, wsc, ws = torch.ones(R, kb, device=DEV), torch.ones(E, nb, kb, device=DEV), workspace(E, N, K, BF16, R)
    bad = torch.zeros(R, dtype=torch.bool, device=DEV)
    bad[[a for a, b in zip(o, o[1:]) if b > a]] = True
    want, y = torch.empty(R, N, dtype=BF16, device=DEV), torch.empty(R, N, dtype=BF16, device=DEV)
    products.moe_grouped_product_fp8(xq, xs, offsets, wq, wsc, want, ws)
    numbers = xq.view(torch.uint8)
    numbers[bad, K - 1] = 0x7F
    products.moe_grouped_product_fp8(xq, xs, offsets, wq, wsc, y, ws)
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], want[~bad])
    numbers[bad, K - 1] = 0
    xs[bad, kb - 1] = math.inf      # and an infinite scale
    products.moe_grouped_product_fp8(xq, xs, offsets, wq, wsc, y, ws)
    assert not torch.isfinite(y[bad]).any() and torch.equal(y[~bad], want[~bad])


@pytest.mark.parametrize("counts,N,K,kernel", GRADIENT_FP8, ids=label)
def test_gradients_of_rows_in_8_bits(counts, N, K, kernel):
    """dx of a product in 8 bits: the product of quantised dy with the transposed weights and exchanged features."""
    E, (o, offsets) = len(counts), table(counts)
    R, nb, kb = o[-1], -(-N // 128), -(-K // 128)
    w, dy = normal(E, N, K, dtype=BF16, seed=3), normal(R, N, dtype=BF16, seed=2)
    q, q_t = (torch.empty(s, dtype=torch.uint8, device=DEV) for s in ((E, N, K), (E, K, N)))
    s, s_t = torch.empty(E, nb, kb, device=DEV), torch.empty(E, kb, nb, device=DEV)
    products.moe_quantize_weights_fp8(w, q, s, q_t, s_t)
    dq, ds = torch.empty(R, N, dtype=torch.uint8, device=DEV), torch.empty(R, nb, device=DEV)
    products.moe_quantize_rows_fp8(dy, dq, ds)
    dx = torch.full((R + 1, K), UNTOUCHED, dtype=BF16, device=DEV)
    products.moe_grouped_product_fp8(dq, ds, offsets, q_t, s_t, dx[:R], workspace(E, K, N, BF16, R))
    assert (dx[R] == UNTOUCHED).all()
    values = dq.view(E4M3).double() * spread(ds, 1, R, N)
    for e in range(E):
        r = slice(o[e], o[e + 1])
        m = q[e].view(E4M3).double() * spread(s[e], 128, N, K)
        want, size = values[r] @ m, values[r].abs() @ m.abs()
        tol = (7 * 2.0 ** -13 + 2.0 ** -18 + (nb + 8) * U) * size + H * want.abs()
        assert ((dx[r].double() - want).abs() <= tol).all(), f"expert {e}"
