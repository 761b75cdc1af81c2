"""Grouped products of as many rows as a call may have, 2^23, most of them one expert's."""
import pytest
import torch

from paper_2501_10375_amd import moe, products
from test_gpu_products import BF16, DEV, F32, UNTOUCHED, check, normal, quantised, reference, table, workspace

pytestmark = pytest.mark.gpu
R, E, N, K = 1 << 23, 3, 64, 128
COUNTS, BEFORE = [70001, R - 70001 - 3 - 5, 3], 2   # two rows of nobody before, three behind


def pieces(o, step=1 << 19):
    """Spans of rows of one expert each."""
    for e, (a, b) in enumerate(zip(o, o[1:])):
        for r in range(a, b, step):
            yield e, slice(r, min(r + step, b))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows(dtype):
    o, offsets = table(COUNTS, BEFORE)
    ws, nobody = workspace(E, N, K, dtype, R), [0, 1, R - 3, R - 2, R - 1]
    for form, n_in, n_out in (("forward", K, N), ("dgrad", N, K)):
        a, w, out = normal(R, n_in, dtype=dtype, seed=1), normal(E, N, K, dtype=dtype, seed=3), torch.full((R, n_out), UNTOUCHED, dtype=dtype, device=DEV)
        (products.moe_grouped_product if form == "forward" else products.moe_grouped_product_dgrad)(a, offsets, w, out, ws)
        assert (out[nobody] == UNTOUCHED).all()
        for e, r in pieces(o):
            (_, want, size), = reference(form, [0, r.stop - r.start], a[r], w[e:e + 1])
            check(out[r], want, size, n_in, dtype, f"{form} rows {r.start}-{r.stop}")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradients_of_matrices(dtype):
    """Numbers -1, 0 and 1: sums of up to 2^23 products are exact in fp32 in any order."""
    o, offsets = table(COUNTS, BEFORE)
    g = torch.Generator(device=DEV)
    g.manual_seed(9)
    x, dy = (torch.randint(-1, 2, (R, n), device=DEV, generator=g, dtype=torch.int8).to(dtype) for n in (K, N))
    want = torch.zeros(E, N, K, dtype=torch.float64, device=DEV)
    for e, r in pieces(o):
        want[e] += dy[r].double().T @ x[r].double()
    ws, dw = workspace(E, N, K, dtype, R), torch.full((E, N, K), UNTOUCHED, device=DEV)
    products.moe_grouped_product_wgrad(dy, x, offsets, dw, False, ws)
    assert torch.equal(dw.double(), want)
    products.moe_grouped_product_wgrad(dy, x, offsets, dw, True, ws)   # (still below 2^24)
    assert torch.equal(dw.double(), 2 * want)


def test_8_bits():
    o, offsets = table(COUNTS, BEFORE)
    x, w = normal(R, K, dtype=BF16, seed=1), normal(E, N, K, dtype=BF16, seed=3)
    q, s = torch.full((R, K), 0x55, dtype=torch.uint8, device=DEV), torch.empty(R, 1, device=DEV)
    products.moe_quantize_rows_fp8(x, q, s)
    wq, wsc = torch.empty(E, N, K, dtype=torch.uint8, device=DEV), torch.empty(E, 1, 1, device=DEV)
    products.moe_quantize_weights_fp8(w, wq, wsc)
    y = torch.full((R, N), UNTOUCHED, dtype=BF16, device=DEV)
    products.moe_grouped_product_fp8(q, s, offsets, wq, wsc, y, workspace(E, N, K, BF16, R))
    assert (y[:2] == UNTOUCHED).all() and (y[-3:] == UNTOUCHED).all()
    for e, r in pieces(o):
        numbers, scale = quantised(x[r], 1)
        assert torch.equal(q[r].view(torch.float8_e4m3fn).double(), numbers) and torch.equal(s[r].double(), scale)
        a, m = numbers * scale, wq[e].view(torch.float8_e4m3fn).double() * wsc[e].double()
        want, size = a @ m.T, a.abs() @ m.abs().T
        tol = (7 * 2.0 ** -13 + 2.0 ** -18 + 9 * 2.0 ** -24) * size + 2.0 ** -8 * want.abs()
        assert ((y[r].double() - want).abs() <= tol).all(), f"rows {r.start}-{r.stop}"


def test_one_row_more_is_refused():
    x, y, w = (torch.empty(s, dtype=BF16, device=DEV) for s in ((R + 1, 64), (R + 1, 64), (1, 64, 64)))
    ws = workspace(1, 64, 64, BF16, R)
    for call in (lambda: products.moe_grouped_product(x, None, w, y, ws), lambda: products.moe_grouped_product_dgrad(y, None, w, x, ws),
                 lambda: products.moe_grouped_product_wgrad(y, x, None, w, False, ws)):
        with pytest.raises(moe.MoeError):
            call()
