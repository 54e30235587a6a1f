"""Which kernels the block-scaled products, their expert forms and the experts' gradients run (csrc/dispatch.h), over their whole
range on the host."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NCU = 256
DIRECT_NONE, DIRECT_64H, TILES_256X128, TILES_256 = 0, 3, 1, 2

SOURCE = """
#include "%s"
extern "C" void product(long long M, long long N, long long K, int out_bytes, int ncu, long long *o) {
    const sb::ProductPlan p = sb::plan_product(M, N, K, sb::PRODUCT_F8, out_bytes, ncu, sb::TILES_256X128);
    o[0] = p.first_rows, o[1] = p.tile_rows, o[2] = p.rest, o[3] = p.split;
}
extern "C" void expert_product(long long M, long long N, long long K, long long experts, int out_bytes, int ncu, long long *o) {
    const sb::ExpertProductPlan p = sb::plan_expert_product(M, N, K, experts, out_bytes, ncu);
    o[0] = p.rest, o[1] = p.split, o[2] = p.runs, o[3] = p.cut;
}
extern "C" void expert_gradient(long long b, long long n, long long m, long long experts, int ncu, long long *o) {
    const sb::ExpertGradPlan p = sb::plan_expert_gradient(b, n, m, experts, ncu);
    o[0] = p.small, o[1] = p.splits;
}
extern "C" int few_rows(long long M, long long N, long long K, long long experts) { return sb::plan_few_rows(M, N, K, experts); }
extern "C" int few_runs(long long M, long long experts) { return sb::plan_few_runs(M, experts); }
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    folder = tmp_path_factory.mktemp("plans")
    src, lib = folder / "plans.cpp", folder / "plans.so"
    src.write_text(SOURCE % os.path.join(ROOT, "paper_2304_13013_amd", "csrc", "dispatch.h"))
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-Wall", "-Werror", str(src), "-o", str(lib)], check=True)
    lib = ctypes.CDLL(str(lib))
    ll, out = ctypes.c_longlong, ctypes.POINTER(ctypes.c_longlong)
    lib.product.argtypes = [ll, ll, ll, ctypes.c_int, ctypes.c_int, out]
    lib.expert_product.argtypes = [ll, ll, ll, ll, ctypes.c_int, ctypes.c_int, out]
    lib.expert_gradient.argtypes = [ll, ll, ll, ll, ctypes.c_int, out]
    lib.few_rows.argtypes = [ll, ll, ll, ll]
    lib.few_runs.argtypes = [ll, ll]
    return lib


def call(f, count, *args):
    out = (ctypes.c_longlong * count)()
    f(*args, out)
    return list(out)


def sizes(seed, count):
    rng = random.Random(seed)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))
    for _ in range(count):
        yield log(1, 2000000), 64 * log(1, 2048), 128 * log(1, 1024), log(1, 1024)
    for M in (1, 16, 17, 64, 65, 255, 256, 257):
        for N, K in ((64, 128), (131072, 128), (64, 131072), (1280, 5120)):
            for E in (1, 2, 1024):
                yield M, N, K, E


def test_plain_products_are_covered_once(plans):
    for M, N, K, _ in sizes(1, 4000):
        for out_bytes in (2, 4):
            first, tiles, rest, split = call(plans.product, 4, M, N, K, out_bytes, NCU)
            assert 0 <= first <= tiles <= M and first % 256 == 0, (M, N, K)
            assert (split == DIRECT_NONE) == (tiles == M) and split <= DIRECT_64H
            assert rest in (TILES_256X128, TILES_256)


def test_expert_products_have_workgroups(plans):
    for M, N, K, E in sizes(2, 4000):
        for out_bytes in (2, 4):
            rest, split, runs, _ = call(plans.expert_product, 4, M, N, K, E, out_bytes, NCU)
            assert rest in (TILES_256X128, TILES_256)
            if split != DIRECT_NONE:
                assert 1 <= runs <= 64 and N // 32 * E * runs < 2 ** 31, (M, N, K, E)
        assert 1 <= plans.few_runs(M, E)


def test_few_rows_read_little_again(plans):
    """At most 16 rows of a weight in the mean, or a small product; a grid that fits."""
    for M, N, K, E in sizes(3, 6000):
        if plans.few_rows(M, N, K, E):
            runs = plans.few_runs(M, E)
            assert M <= 16 or M <= 4 * E or -(-M // 16) * (N // 32) * K <= 2 ** 20, (M, N, K, E)
            assert N // 32 * E * runs < 2 ** 31


def test_expert_gradients_have_items(plans):
    for M, n, m, E in sizes(4, 3000):
        n, m = min(n, 8192), min(64 * (m // 128), 8192) or 64
        for b in (0, M):
            small, splits = call(plans.expert_gradient, 2, b, n, m, E, NCU)
            assert small in (0, 1) and 1 <= splits <= 16, (b, n, m, E)
    # A size of each kind: whole ranges on small tiles, split ones, large tiles.
    assert call(plans.expert_gradient, 2, 5003, 768, 1088, 24, NCU) == [1, 1]
    assert call(plans.expert_gradient, 2, 30000, 640, 704, 2, NCU)[1] > 1
    assert call(plans.expert_gradient, 2, 16448, 1024, 4096, 8, NCU) == [0, 1]


def test_cut_of_expert_products(plans):
    """Only 256x256 tiles of more than a round give their last tile rows away, and only where the experts' cut tile rows are few."""
    cuts = 0
    for M, N, K, E in list(sizes(11, 4000)) + [(16448, 1024, 4096, 8), (33500, 1024, 4096, 8), (17000, 1024, 8192, 8)]:
        for out_bytes in (2, 4):
            rest, split, _, cut = call(plans.expert_product, 4, M, N, K, E, out_bytes, NCU)
            assert cut in (0, NCU)
            if cut:
                cuts += 1
                assert rest == TILES_256 and split == DIRECT_NONE and E * -(-N // 256) <= NCU // 4 and (M / 256 + E) * -(-N // 256) > NCU
    assert cuts >= 6
    assert call(plans.expert_product, 4, 16448, 1024, 4096, 8, 2, NCU)[3] == NCU
    assert call(plans.expert_product, 4, 16448, 4096, 1024, 8, 2, NCU)[3] == 0
