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

// The host knows the rows of a call, not of its experts: their tiles of 64 rows are taken to be rows / 64 and half a tile for each expert.  A workgroup of
// the small tiles takes its K steps and what five of them would take, and every CU as many workgroups as there are for each of them; the large tiles are
// planned and joined first, and read less for an MFMA.  Of few rows the experts' weights are a stream; as long as they are read fast, from a memory-side cache of
// 256 MiB, up to 16 rows an expert are few in 8 bits.  Times in us, * what the rule takes, routed evenly or
// mildly skewed (Zipf 0.5 to 0.8) unless noted:
//
//   experts, out, in, rows            few rows  small  large        experts, out, in, rows            small  large
//   forward  4, 2048, 2048, 16           7.8*     8.9    14         dgrad  1, 2048, 2048, 512           9.7*    24
//            1, 4096, 4096, 24          17       14.8*   15                16, 1408, 2048, 1030        21*      23
//            8, 4096, 4096, 64          48       41*     48                8, 4096, 1024, 1000         32       26*
//            64, 1408, 2048, 128        62       71*     84                1, 1024, 8192, 700          22       20*
//            64, 1408, 2048, 256        64*      71      85         wgrad  1, 1024, 1024, 1000          7.4*    25
//            1, 1024, 1024, 1000         -        7.1*   17                1, 512, 512, 4096           18*      24
//            1, 4096, 4096, 300          -       23*     26                1, 2048, 2048, 2048         33*      47
//            1, 8192, 1024, 700          -       23      18*               8, 1024, 1024, 600          12*      15
//            1, 2048, 2048, 2048         -       29      27*               4, 2048, 2048, 300 (*)      20       18*
//   8 bits   1, 4096, 4096, 24          10.5*    13.1    14                16, 1408, 2048, 30 (*)      42       24*
//            1, 2048, 8192, 20          16*      23      15                64, 256, 256, 19200         13.8*    17
//            1, 4096, 4096, 60          19       13*     17                  the same, Zipf 1.2        26*      30
//            16, 1408, 2048, 128        10.8*    11.2    16                64, 256, 256, 32000         18.7     27*
//            16, 1408, 2048, 150 (Z)    15       11*     17                  the same, Zipf 1.2        38       32*
//            64, 1408, 2048, 512        32*      33      35                1, 512, 512, 8000           32       28*
//            16, 512, 4096, 128          8.5*    13.4    14         (*) many tiles, which store more than they compute; (Z) Zipf 1.2
//            4, 2048, 2048, 600         35       11*     16
//            8, 4096, 1024, 1000         -       17      15*
//            8, 14336, 4096, 64         83*       -     107
//            8, 14336, 4096, 154        90 to 105 -      97 to 104*
//
// What the host does not see is the skew, and the rule pays for it where it is strong.  Few rows read an expert's weights again for every 16 of its rows: 64 experts of
// 1408 x 2048 with Zipf 1.2, 8 bits, 512 rows 67 where small tiles take 31, bf16, 256 rows 72 (43); all rows on one expert 102 (8.5) and 63 (9.0).  wgrad of more than
// 6400 rows for each of up to three experts is taken to have an expert with a third of them, more K steps than a workgroup of the small tiles should have: evenly routed
// it is half as slow again.
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
