"""Host-side checks of the grouped products that need no GPU: exported symbols, refusals, sizes."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "moe_products.h")
OK, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008)   # never dereferenced: validation fails first
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    from paper_2501_10375_amd import build, moe, products

    if not os.path.exists(moe.LIB_PATH):
        build.build()
    return products.lib()


def _product(**kw):
    from paper_2501_10375_amd import moe, products

    base = dict(n_experts=8, out_features=512, in_features=256, dtype=moe.MOE_BF16)
    base.update(kw)
    return products.MoeProduct(**base)


def test_library_exports_every_declared_symbol(L):
    from paper_2501_10375_amd import products

    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    declared = set(re.findall(r"\b(moe_[a-z0-9_]+)\s*\(", text))
    assert declared == set(products.EXPORTS)
    for name in declared:
        assert hasattr(L, name), name


@pytest.mark.parametrize("kw,code", [
    (dict(out_features=0), -2), (dict(out_features=96), -2), (dict(in_features=100), -2), (dict(in_features=-64), -2),
    (dict(out_features=(1 << 20) + 64), -2), (dict(out_features=1 << 16, in_features=(1 << 15) + 64), -2),
    (dict(n_experts=0), -2), (dict(n_experts=65), -2), (dict(dtype=2), -3), (dict(dtype=-1), -3),
])
def test_bad_products_are_refused(L, kw, code):
    n, p = ctypes.c_size_t(0), _product(**kw)
    pp = ctypes.byref(p)
    assert L.moe_product_workspace_bytes(pp, 16, ctypes.byref(n)) == code
    assert L.moe_grouped_product(pp, 4, OK, OK, OK, OK, OK, BIG, None) == code
    assert L.moe_grouped_product_dgrad(pp, 4, OK, OK, OK, OK, OK, BIG, None) == code
    assert L.moe_grouped_product_wgrad(pp, 4, OK, OK, OK, OK, 0, 0, OK, BIG, None) == code
    assert L.moe_grouped_product_fp8(pp, 4, OK, OK, OK, OK, OK, OK, OK, BIG, None) == code
    assert L.moe_quantize_weights_fp8(pp, OK, OK, OK, None, None, None) == code


def test_products_validate_before_any_device_work(L):
    from paper_2501_10375_amd import moe

    p = _product()
    pp = ctypes.byref(p)
    size = ctypes.c_size_t(0)
    assert L.moe_product_workspace_bytes(pp, 4, ctypes.byref(size)) == 0 and size.value > 0
    assert L.moe_product_workspace_bytes(pp, 4, None) == moe.MOE_ERR_NULL
    assert L.moe_product_workspace_bytes(None, 4, ctypes.byref(size)) == moe.MOE_ERR_NULL
    assert L.moe_product_workspace_bytes(pp, -1, ctypes.byref(size)) == moe.MOE_ERR_SHAPE
    assert L.moe_product_workspace_bytes(pp, (1 << 23) + 1, ctypes.byref(size)) == moe.MOE_ERR_SHAPE
    calls = {   # positions of the pointers (after product and rows): all required
        "moe_grouped_product": (L.moe_grouped_product, [OK] * 5, ()),
        "moe_grouped_product_dgrad": (L.moe_grouped_product_dgrad, [OK] * 5, ()),
        "moe_grouped_product_fp8": (L.moe_grouped_product_fp8, [OK] * 7, ()),
    }
    for name, (fn, ptrs, _) in calls.items():
        for i in range(len(ptrs)):
            for bad, code in ((None, moe.MOE_ERR_NULL), (ODD, moe.MOE_ERR_ALIGN)):
                args = list(ptrs)
                args[i] = bad
                assert fn(pp, 4, *args, BIG, None) == code, (name, i, bad)
        assert fn(pp, -1, *ptrs, BIG, None) == moe.MOE_ERR_SHAPE, name
        assert fn(pp, (1 << 23) + 1, *ptrs, BIG, None) == moe.MOE_ERR_SHAPE, name
        assert fn(pp, 4, *ptrs, size.value - 1, None) == moe.MOE_ERR_WORKSPACE, name
        assert fn(None, 4, *ptrs, BIG, None) == moe.MOE_ERR_NULL, name
    for i in range(5):
        for bad, code in ((None, moe.MOE_ERR_NULL), (ODD, moe.MOE_ERR_ALIGN)):
            args = [OK] * 5
            args[i] = bad
            assert L.moe_grouped_product_wgrad(pp, 4, *args[:4], 0, 0, args[4], BIG, None) == code, (i, bad)
    wgrad = lambda dtype, acc, size=BIG: L.moe_grouped_product_wgrad(pp, 4, OK, OK, OK, OK, dtype, acc, OK, size, None)  # noqa: E731
    assert wgrad(moe.MOE_BF16, 1) == moe.MOE_ERR_DTYPE     # sums over calls are held in fp32
    assert wgrad(2, 0) == moe.MOE_ERR_DTYPE
    assert wgrad(moe.MOE_F32, 0, 0) == moe.MOE_ERR_WORKSPACE
    f32 = _product(dtype=moe.MOE_F32)
    assert L.moe_grouped_product_wgrad(ctypes.byref(f32), 4, OK, OK, OK, OK, moe.MOE_BF16, 0, OK, BIG, None) == moe.MOE_ERR_DTYPE
    assert L.moe_grouped_product_fp8(ctypes.byref(f32), 4, OK, OK, OK, OK, OK, OK, OK, BIG, None) == moe.MOE_ERR_DTYPE
    # no rows: accepted without touching the device, per-row buffers may be missing
    assert L.moe_grouped_product(pp, 0, None, OK, OK, None, OK, BIG, None) == 0
    assert L.moe_grouped_product_dgrad(pp, 0, None, OK, OK, None, OK, BIG, None) == 0
    assert L.moe_grouped_product_fp8(pp, 0, None, None, OK, OK, OK, None, OK, BIG, None) == 0
    assert L.moe_grouped_product_wgrad(pp, 0, None, None, OK, OK, moe.MOE_F32, 1, OK, BIG, None) == 0
    # one expert needs no table
    one = _product(n_experts=1)
    assert L.moe_grouped_product(ctypes.byref(one), 0, None, None, OK, None, OK, BIG, None) == 0


def test_quantisers_validate_before_any_device_work(L):
    from paper_2501_10375_amd import moe

    rows = L.moe_quantize_rows_fp8
    assert rows(4, 256, 2, OK, OK, OK, None) == moe.MOE_ERR_DTYPE
    assert rows(-1, 256, 1, OK, OK, OK, None) == moe.MOE_ERR_SHAPE
    assert rows(4, 100, 1, OK, OK, OK, None) == moe.MOE_ERR_SHAPE
    assert rows(4, 0, 1, OK, OK, OK, None) == moe.MOE_ERR_SHAPE
    for i in range(3):
        for bad, code in ((None, moe.MOE_ERR_NULL), (ODD, moe.MOE_ERR_ALIGN)):
            args = [OK] * 3
            args[i] = bad
            assert rows(4, 256, 1, *args, None) == code
    assert rows(0, 256, 1, None, None, None, None) == 0
    p = _product()
    weights = lambda *a: L.moe_quantize_weights_fp8(ctypes.byref(p), *a, None)  # noqa: E731
    for i in range(3):
        for bad, code in ((None, moe.MOE_ERR_NULL), (ODD, moe.MOE_ERR_ALIGN)):
            args = [OK] * 5
            args[i] = bad
            assert weights(*args) == code
    assert weights(OK, OK, OK, OK, None) == moe.MOE_ERR_NULL      # transposed numbers without their scales
    assert weights(OK, OK, OK, None, OK) == moe.MOE_ERR_NULL
    assert weights(OK, OK, OK, ODD, OK) == moe.MOE_ERR_ALIGN


def test_binding_refuses_cpu_tensors_and_other_types():
    from paper_2501_10375_amd import products

    x, w, y = torch.zeros(4, 64), torch.zeros(1, 64, 64), torch.zeros(4, 64)
    ws = torch.zeros(256, dtype=torch.uint8)
    with pytest.raises(ValueError):
        products.moe_grouped_product(x, None, w, y, ws)
    with pytest.raises(TypeError):
        products.moe_grouped_product(x.half(), None, w, y, ws)
    with pytest.raises(ValueError):
        products.moe_quantize_rows_fp8(x, y.to(torch.uint8), torch.zeros(4, 1))
    with pytest.raises(TypeError):   # the numbers have to be e4m3
        products._e4m3(y, (4, 64), "q", 0)
