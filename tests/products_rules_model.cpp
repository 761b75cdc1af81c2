// The rules of csrc/products_rules.h for tests on the host.
#include "products_rules.h"

using namespace moe::products;

extern "C" int products_way(int form, int fp8, int experts, int rows, int n, int k) {
    return choose_way(static_cast<Form>(form), {experts, rows, n, k}, fp8 != 0);
}

extern "C" int products_few_rows(int fp8, int experts, int rows, int n, int k, int compute_units, int* out) {
    const FewRows v = choose_few_rows({experts, rows, n, k}, fp8 != 0, compute_units);
    out[0] = v.row_fragments;
    out[1] = v.feature_fragments;
    out[2] = v.waves;
    return 0;
}

extern "C" int products_most_small_blocks() { return kMostSmallBlocks; }
