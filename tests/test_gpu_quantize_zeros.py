"""Zeros keep their sign in quantisation: value / scale has the sign of the value, whether the value is a zero or its quotient is
rounded to one.  Every bit is compared."""
import pytest
import torch

from paper_2501_10375_amd import products
from test_gpu_products import BF16, DEV, F32, normal, quantised

pytestmark = pytest.mark.gpu


def with_zeros(*shape, dtype):
    """Numbers of both signs, a quarter of them zeros, a quarter with quotients below half of the least e4m3 number (2^-10)."""
    x = normal(*shape, seed=21)
    x[..., 0::4] *= 0.0            # +0 and -0
    x[..., 1::4] *= 2.0 ** -30
    return x.to(dtype)


def bits(v, rows):
    """Bytes of the e4m3 numbers of a matrix in blocks of rows x 128, by the definition in 64 bits, and the sign of the value."""
    numbers, _ = quantised(v, rows)
    magnitude = numbers.abs().float().to(torch.float8_e4m3fn).view(torch.uint8)
    return magnitude | (torch.signbit(v).to(torch.uint8) << 7)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R,K", [(1, 64), (5, 192), (70, 1024)])
def test_rows(R, K, dtype):
    x = with_zeros(R, K, dtype=dtype)
    x[-1] = -0.0                   # a row of nothing else
    q, scales = torch.full((R, K), 0x55, dtype=torch.uint8, device=DEV), torch.empty(R, -(-K // 128), device=DEV)
    products.moe_quantize_rows_fp8(x, q, scales)
    assert torch.equal(q, bits(x, 1))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("E,N,K", [(1, 64, 64), (2, 192, 320)])
def test_weights_and_transposed_weights(E, N, K, dtype):
    w = with_zeros(E, N, K, dtype=dtype)
    w[0, :64, :64] = -0.0
    q, q_t = (torch.full(s, 0x55, dtype=torch.uint8, device=DEV) for s in ((E, N, K), (E, K, N)))
    nb, kb = -(-N // 128), -(-K // 128)
    scales, scales_t = torch.empty(E, nb, kb, device=DEV), torch.empty(E, kb, nb, device=DEV)
    products.moe_quantize_weights_fp8(w, q, scales, q_t, scales_t)
    want = torch.stack([bits(m, 128) for m in w])
    assert torch.equal(q, want)
    assert torch.equal(q_t, want.transpose(1, 2))
