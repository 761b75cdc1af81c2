"""Which kernel a grouped product runs on follows from its sizes: the rules compiled for the host, so that shapes of the GPU tests that are meant
for a kernel are known to reach it, and every variant that a call can take is known to have one."""
import ctypes
import os
import random
import subprocess

import pytest

import test_gpu_products as basic
import test_gpu_products_used as used
from products_shapes import BEHIND_SMALL_FP8, FEW_ROWS_BF16, FEW_ROWS_FP8, GRADIENT_FP8, SMALL_FP8

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2501_10375_amd", "csrc")
FORWARD, DGRAD, WGRAD = 0, 1, 2
FEW, SMALL, LARGE = 0, 1, 2
UNITS = 256   # CUs of an MI355X


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("rules") / "rules.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", path, os.path.join(HERE, "products_rules_model.cpp")], check=True)
    return ctypes.CDLL(path)


def way(rules, form, fp8, E, R, N, K):
    return rules.products_way(form, int(fp8), E, R, N, K)


def few(rules, fp8, E, R, N, K):
    out = (ctypes.c_int * 3)()
    rules.products_few_rows(int(fp8), E, R, N, K, UNITS, out)
    return tuple(out)


def rows_of(counts, nobody):
    return sum(counts) + nobody


@pytest.mark.parametrize("fp8,cases", [(False, FEW_ROWS_BF16), (True, FEW_ROWS_FP8)])
def test_shapes_for_few_rows_take_the_variant_they_are_for(rules, fp8, cases):
    for (counts, N, K), variant in cases:
        assert way(rules, FORWARD, fp8, len(counts), sum(counts), N, K) == FEW, (counts, N, K)
        assert few(rules, fp8, len(counts), sum(counts), N, K) == variant, (counts, N, K)


def test_every_variant_of_few_rows_has_shapes_of_several_passes(rules):
    """Over the whole range of sizes: which variants a call can take, and which of them can have more rows than a pass serves."""
    rng = random.Random(0)
    seen = {False: {}, True: {}}
    for _ in range(200000):
        E = rng.choice((1, 2, 3, 4, 7, 8, 16, 33, 64))
        R = max(1, int(2 ** rng.uniform(0, 10)))
        N, K = (64 * max(1, int(2 ** rng.uniform(0, 10))) for _ in range(2))
        for fp8 in (False, True):
            if way(rules, FORWARD, fp8, E, R, N, K) == FEW:
                v = few(rules, fp8, E, R, N, K)
                seen[fp8][v] = seen[fp8].get(v, False) or R > 16 * v[0]
    for fp8, cases in ((False, FEW_ROWS_BF16), (True, FEW_ROWS_FP8)):
        tested = {}
        for (counts, _, _), v in cases:
            tested[v] = tested.get(v, False) or max(counts) > 16 * v[0]
        assert tested == seen[fp8], "bf16 8 bits".split()[fp8]


def test_shapes_at_the_end_of_the_small_tiles(rules):
    for counts, N, K in SMALL_FP8:
        assert way(rules, FORWARD, True, len(counts), sum(counts), N, K) == SMALL
    for counts, N, K in BEHIND_SMALL_FP8:
        assert way(rules, FORWARD, True, len(counts), sum(counts), N, K) == LARGE
    assert max(-(-K // 128) for _, _, K in SMALL_FP8) == 55


def test_no_call_brings_the_small_tiles_more_blocks_than_they_have_room_for(rules):
    room = rules.products_most_small_blocks()
    for K in range(64, 16384, 64):
        for R in (9, 33, 100):
            for E, N in ((1, 64), (3, 64), (1, 4096)):
                if way(rules, FORWARD, True, E, R, N, K) == SMALL:
                    assert -(-K // 128) < room


def test_gradient_shapes_take_their_way(rules):
    for counts, N, K, name in GRADIENT_FP8:
        assert way(rules, FORWARD, True, len(counts), sum(counts), K, N) == {"few": FEW, "small": SMALL, "large": LARGE}[name]


def test_every_form_has_tested_shapes_of_every_way(rules):
    """The shapes of the tests of results, with their rows of nobody."""
    ways = {(form, fp8): set() for form, fp8 in ((FORWARD, False), (DGRAD, False), (WGRAD, False), (FORWARD, True))}
    for counts, N, K, before, behind in basic.SHAPES:
        for form in (FORWARD, DGRAD, WGRAD):
            ways[form, False].add(way(rules, form, False, len(counts), rows_of(counts, before + behind), N, K))
    for counts, N, K in used.FORWARD:
        ways[FORWARD, False].add(way(rules, FORWARD, False, len(counts), rows_of(counts, 5), N, K))
        ways[DGRAD, False].add(way(rules, DGRAD, False, len(counts), rows_of(counts, 5), K, N))
        ways[FORWARD, True].add(way(rules, FORWARD, True, len(counts), rows_of(counts, 2), N, K))
    matrices = next(m for m in used.test_matrices_gradients_are_cut_in_every_way.pytestmark if m.name == "parametrize" and m.args[0] == "counts,N,K")
    for counts, N, K in matrices.args[1]:
        ways[WGRAD, False].add(way(rules, WGRAD, False, len(counts), rows_of(counts, 3), N, K))
    assert ways == {(FORWARD, False): {FEW, SMALL, LARGE}, (DGRAD, False): {SMALL, LARGE}, (WGRAD, False): {SMALL, LARGE}, (FORWARD, True): {FEW, SMALL, LARGE}}
    # one call after another, replays and streams: small tiles, few rows, large tiles
    mixed = [[way(rules, FORWARD, fp8, len(c), sum(c), N, K) for c, N, K in used.MIXED] for fp8 in (False, True)]
    assert mixed == [[SMALL, FEW, LARGE]] * 2


def test_one_workspace_serves_every_shape_of_a_type():
    import torch

    from paper_2501_10375_amd import build, moe, products

    if not os.path.exists(moe.LIB_PATH):
        build.build()
    for dtype, size in ((torch.bfloat16, 66.9e6), (torch.float32, 33.6e6)):
        sizes = {products.moe_product_workspace_bytes(products.make_product(E, N, K, dtype), rows)
                 for E, N, K in ((1, 64, 64), (8, 14336, 4096), (8, 4096, 14336), (64, 1408, 2048), (1, 64, 1 << 20)) for rows in (0, 1, 300, 8192, 1 << 23)}
        assert len(sizes) == 1 and abs(sizes.pop() - size) < 0.1e6
