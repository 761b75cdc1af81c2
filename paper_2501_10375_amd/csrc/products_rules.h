// Which kernels a grouped product runs on, from its sizes alone: without anything of the device, for the launches and for tests on the host.
#pragma once

namespace moe {
namespace products {

// What a product computes, as out[row, feature] = sum over c of q(row, c) * p(feature, c):
//   kForward  q = x,  p = W_e,    c = in_features
//   kDgrad    q = dy, p = W_e^T,  c = out_features
//   kWgrad    q = dy^T, p = x^T,  c = the rows of expert e; an output matrix for every expert
enum Form { kForward, kDgrad, kWgrad };

struct Size {
    int experts, rows, n, k;   // n = out_features, k = in_features
};

// Which kernels a bf16 or 8-bit product runs on.
enum Way { kFewRows, kSmallTiles, kLargeTiles };

// Blocks of 128 of an 8-bit contraction that the small tiles' kernel has room for.  (A guard: the rule below, which allows 60 K steps less five, asks for 55 at most.)
constexpr int kMostSmallBlocks = 56;

// The host knows the rows of a call, not of its experts: their tiles of 64 rows are taken to be rows / 64 and half a tile for each expert.  A workgroup of the small
// tiles takes its K steps and what five of them would take, and every CU as many workgroups as there are for each of them; the large tiles are planned and
// joined first, and read less for an MFMA.  Of few rows the experts' weights are a stream.  Times in us (experts, out, in features, rows), few rows / small / large:
//   forward  4, 2048, 2048, 16: 7.8, 8.9, 14; 1, 4096, 4096, 24: 17, 14.8, 15; 8, 4096, 4096, 64: 48, 41, 48; 64, 1408, 2048, 64: 34, 33, 35; 1, 1024, 1024, 1000: -, 7.1,
//            17; 1, 2048, 2048, 512: -, 9.5, 24; 1, 4096, 4096, 300: -, 23, 26; 8, 4096, 1024, 1000: -, 20, 21; 1, 8192, 1024, 700: -, 23, 18; 1, 2048, 2048, 2048: -, 29, 27
//   dgrad    1, 2048, 2048, 512: -, 9.7, 24; 16, 1408, 2048, 1030: -, 21, 23; 8, 4096, 1024, 1000: -, 32, 26; 1, 1024, 8192, 700: -, 22, 20
//   wgrad    1, 1024, 1024, 1000: -, 7.4, 25; 1, 512, 512, 4096: -, 18, 24; 1, 2048, 2048, 2048: -, 33, 47; 8, 1024, 1024, 600: -, 12, 15; of more tiles, which store more than
//            they compute, 4, 2048, 2048, 300: -, 20, 18; 16, 1408, 2048, 30: -, 42, 24; where a third of the rows, an expert's under a skewed gate, are more than 100 K
//            steps, 64, 256, 256, 32000: -, 38, 32 (evenly 18, 27); 1, 512, 512, 8000: -, 32, 27
//   8 bits   1, 4096, 4096, 24: 10.5, 13.1, 14; 16, 512, 4096, 100: 8.5, 13.4, 14; 1, 4096, 4096, 60: 19, 13, 17; 16, 1408, 2048, 150: 15, 11, 17; 1, 4096, 4096, 300: 88, 16, 24; 4, 2048,
//            2048, 600: 35, 11, 16; 8, 4096, 1024, 1000: -, 17, 15; 1, 2048, 8192, 20: 16, 23, 15; 8, 14336, 4096, 64: 83, -, 107, 154 90 to 105, -, 97 to 104
// (as long as the weights are read fast, from a memory-side cache of 256 MiB, up to 16 rows an expert are few in 8 bits).
inline Way choose_way(Form form, const Size& a, bool fp8) {
    const bool forward = form == kForward;
    if (forward && (a.rows <= (fp8 ? 32 : 16) || (fp8 && a.rows <= 8 * a.experts))) return kFewRows;
    const double active = a.experts < a.rows ? a.experts : a.rows;
    const double across = forward ? a.n / 64 : a.k / 64;
    const double down = form == kWgrad ? (double)a.experts * (a.n / 64) : a.rows / 64.0 + 0.5 * active;
    const double steps = form == kWgrad ? a.rows / (64.0 * a.experts) + 0.5 : forward ? a.k / (fp8 ? 128.0 : 64.0) : a.n / 64.0;
    const double tiles = across * down, load = (tiles < 256 ? 1.0 : tiles / 256) * (steps + 5);
    const bool deep = form == kWgrad && a.rows > 6400L * (a.experts < 3 ? a.experts : 3);
    if (fp8 ? load <= 60 && (a.k + 127) / 128 <= kMostSmallBlocks : forward ? load <= 110 : form == kDgrad ? load <= 83 : load <= 150 && tiles <= 2048 && !deep)
        return kSmallTiles;
    if (!forward) return kLargeTiles;
    const bool cached = (double)active * a.n * a.k <= 256.0 * (1 << 20);
    return (fp8 ? cached && a.rows <= 320 && a.rows <= 16 * a.experts : a.rows <= 4 * a.experts) ? kFewRows : kLargeTiles;
}

// The few-row kernel's fragments of 16 rows that a pass serves, fragments of 16 features of a workgroup, and wavefronts that share the contraction.
struct FewRows {
    int row_fragments, feature_fragments, waves;
};

// 8 bits: one fragment of rows a pass up to eight rows an expert, two beyond; feature fragments that share the rows' loads where there are workgroups enough
// (8, 14336, 4096, 64 in ones, twos, fours: 101, 84, 83 us; 154 with two of rows: -, 106, 90; 1, 4096, 4096, 24: -, 11, 14).  bf16: one of each (8, 14336, 4096,
// 64: 188, 203, 204), and eight wavefronts where four would leave the CUs with few and each still has 16 K steps (8, 4096, 14336, 2: 42 -> 37 us; with less,
// 8 bits 16, 6400, 4096, 2: 12.2 -> 15.4).
inline FewRows choose_few_rows(const Size& a, bool fp8, int compute_units) {
    const int active = a.experts < a.rows ? a.experts : a.rows;   // experts with rows at most
    if (!fp8) return {1, 1, (long)active * (a.n / 16) <= 4L * compute_units && a.k / 64 >= 8 * 16 ? 8 : 4};
    if (a.rows <= 16) return {1, 1, 4};
    if (a.rows <= 8 * a.experts) return {1, 2, 4};
    return {2, (long)active * (a.n / 64) <= 2L * compute_units ? 2 : 4, 4};
}

}  // namespace products
}  // namespace moe
