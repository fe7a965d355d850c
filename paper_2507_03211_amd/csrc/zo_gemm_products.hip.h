// Products of the gradients on the matrix cores: tiles by estimated time, and the launches (the LM head's gradient, zo_gemm_grad.hip, whose
// sizes the constants were fitted to, and the linear layers', zo_linear_grad.hip).
#pragma once
#include "zo_gemm_tiles.hip.h"

namespace zo {
namespace {

template <int DT, int EPI, class OP> hipError_t launch_product(Tile t, const Args &a, const typename OP::Arg &op)
{
    switch (t) {
    case T256x256: return launch_pipe<DT, EPI, Shape<4, 4, 2>, OP>(a, op);
    case T256x192: return launch_pipe<DT, EPI, Shape<4, 3, 2>, OP>(a, op);
    case T256x128: return launch_pipe<DT, EPI, Shape<4, 2, 2>, OP>(a, op);
    case T192x128: return launch_pipe<DT, EPI, Shape<3, 2, 3>, OP>(a, op);
    case T128x128: return launch_pipe<DT, EPI, Shape<2, 2, 4>, OP>(a, op);
    default: return launch_small_t<DT, EPI, 1, false, OP>(a, op);
    }
}
using ByRows = Product<true, true>;         // G^T x: contraction over the rows, outside in both
using ByWords = Product<false, true>;       // G e: contraction over G's columns (the head's words), outside in e

// dx's shares and de in one launch, where few rows have both in 64 x 64 tiles: dx reads e while de is written.  dx first, and rings of two stages,
// five workgroups to a CU, for both.  us of the whole call, over and over on the same buffers (20 rows take 69.5 where every call has an
// e and a de of its own, 61.7 beside that on one pair), two launches / one: 20 rows of 768 x 50272 64.1 / 61.0 (rings of three 64.3, of four
// 72.4, de first 64.4, the two interleaved 73.7), 20 of 2048 156.5 / 144.1, 64 of 512 x 10000 27.7 / 25.1, 100 of 512 x 20000 39.8 / 35.9,
// 20 of 5120 x 8192 70.6 / 67.5.  Long contractions want the deeper ring and stay by themselves: by slabs a
// share, 1 row of 4096 x 32000 (62) 195.0 / 181.3, 33 of 4096 x 20000 (78) 106.0 / 109.6, 64 of 2048 x 50272 (98) 155.7 / 153.2, 1 of 5120 x 128000
// (125) 821.9 / 873.4, 20 of 8192 x 50272 (196) 572.7 / 585.7; 4000 rows of 8 x 64, 63 slabs in de, 50.8 / 62.9.
// EPI: 7 where dx has shares; a linear layer's dx may have one (6, 10): rows x n x k 20 x 768 x 768 14.2 / 11.1, 200 x 768 x 768 13.8 / 11.1, 3 x 576 x 4096 13.4 /
// 10.6, 100 x 1024 x 1024 13.8 / 12.5.
constexpr int kBothSlabs = 64, kBothRows = 512;
struct SmallTiles { const uint16_t *x, *w; void *y; int m, n, k, tiles_m, tiles_n, total; };
constexpr int kBothStages = 2;
template <int DT, int EPI = 7>
__global__ __launch_bounds__(256, 2) void head_both_kernel(SmallTiles a, SmallTiles b, ByWords::Arg op_a, ByRows::Arg op_b, int blocks_a)
{
    if ((int)blockIdx.x < blocks_a)
        small_tile<DT, EPI, 1, false, ByWords, kBothStages>(a.x, a.w, nullptr, nullptr, nullptr, a.y, a.m, a.n, a.k, a.tiles_m, a.tiles_n, a.total, op_a, (int)blockIdx.x);
    else
        small_tile<DT, 6, 1, false, ByRows, kBothStages>(b.x, b.w, nullptr, nullptr, nullptr, b.y, b.m, b.n, b.k, b.tiles_m, b.tiles_n, b.total, op_b, (int)blockIdx.x - blocks_a);
}
template <int DT, int EPI = 7> hipError_t launch_both(const Args &dx, const ByWords::Arg &op_dx, const Args &de, const ByRows::Arg &op_de)
{
    auto tiles = [](const Args &a) {
        const int tm = (a.m_half + 63) / 64, tn = (a.n + 63) / 64;
        return SmallTiles{(const uint16_t *)a.x, (const uint16_t *)a.wt_p, a.y, a.m_half, a.n, a.k, tm, tn, a.n_sign * tm * tn};
    };
    const SmallTiles a = tiles(dx), b = tiles(de);
    const int blocks_a = (a.total + 7) / 8 * 8, blocks_b = (b.total + 7) / 8 * 8;
    head_both_kernel<DT, EPI><<<dim3(blocks_a + blocks_b), dim3(256), kBothStages * kSmallStageBytes<1>, dx.s>>>(a, b, op_dx, op_de, blocks_a);
    return hipGetLastError();
}

// The tile of least estimated time in us: start + slabs (rounds slab + full busy) + rounds round + operand MB operand + output MB output,
// where a round of tiles that fills more than half of the CUs also pays slabs busy b, b = 0 .. 1 from half full to full (64 x 64 tiles, two
// on a CU: slab for one alone, busy for two).  Constants: least relative squares over 2674 shapes (8 - 8192 rows, d 128 - 5120, vocabularies
// 2 k - 50 k, operands far), every tile of each product timed, for dx with 1 - 40 shares and its sum's launch; shapes' best and up to 1.6 times
// it.  The pick against the best: logits 1.2 % slower on average (one shape in 25 more than 10 %), de 0.3 %, dx 1.8 %; by the linear
// layers' constants 1.7, 0.9 and 3.5 %.
enum ProductKind { kLogits, kByRows, kByWords };
constexpr Tile kProductTiles[] = {T256x256, T256x192, T256x128, T192x128, T128x128, T64x64};
constexpr int kLeastSlabs[] = {3, 3, 3, 4, 5, 1};
static const struct { float start, slab, busy, round, operand, output; } kProductCost[3][6] = {
    {{7.99f, 1.06f, 0.45f, 2.54f, 0.021f, 0.210f},
     {4.52f, 0.82f, 0.35f, 5.09f, 0.032f, 0.105f},
     {3.06f, 0.65f, 0.19f, 3.58f, 0.045f, 0.170f},
     {3.28f, 0.47f, 0.22f, 2.87f, 0.054f, 0.161f},
     {2.82f, 0.41f, 0.12f, 1.44f, 0.076f, 0.271f},
     {2.28f, 0.25f, 0.43f, 1.76f, 0.091f, 0.000f}},
    {{2.47f, 1.12f, 0.33f, 3.66f, 0.015f, 0.069f},
     {3.59f, 0.85f, 0.35f, 2.47f, 0.020f, 0.041f},
     {3.19f, 0.60f, 0.28f, 1.98f, 0.045f, 0.000f},
     {3.35f, 0.51f, 0.20f, 1.48f, 0.020f, 0.000f},
     {3.23f, 0.40f, 0.14f, 0.92f, 0.019f, 0.000f},
     {3.46f, 0.23f, 0.41f, 0.23f, 0.000f, 0.069f}},
    {{3.61f, 1.00f, 0.47f, 4.50f, 0.030f, 0.078f},
     {3.81f, 0.80f, 0.37f, 2.88f, 0.024f, 0.086f},
     {2.81f, 0.65f, 0.22f, 1.80f, 0.023f, 0.112f},
     {3.13f, 0.47f, 0.24f, 1.62f, 0.032f, 0.101f},
     {2.87f, 0.38f, 0.16f, 1.26f, 0.056f, 0.063f},
     {2.58f, 0.20f, 0.38f, 0.20f, 0.095f, 0.141f}},
};
float product_us(ProductKind kind, int t, int shares, int m, int n, int n_slabs)
{
    const auto &c = kProductCost[kind][t];
    const float n_cu = cu_count() ? (float)cu_count() : 256.0f, slabs = (float)n_slabs, slots = t == T64x64 ? 2 * n_cu : n_cu;
    const float tiles = (float)shares * (float)((m + kTileRows[t] - 1) / kTileRows[t]) * (float)((n + kTileColumns[t] - 1) / kTileColumns[t]);
    const float full = __builtin_floorf(tiles / slots), part = tiles / slots - full, rounds = full + (part > 0 ? 1.0f : 0.0f);
    const float operand_mb = ((float)m + (float)n) * slabs * (float)shares * (BK * 2e-6f), output_mb = (float)m * (float)n * (float)shares * (kind == kByWords ? 4e-6f : 2e-6f);
    float us = c.start + rounds * c.round + operand_mb * c.operand + output_mb * c.output;
    if (t == T64x64) {
        const float lone = part > 0 && part <= 0.5f ? 1.0f : 0.0f;
        us += slabs * ((rounds - lone) * c.busy + lone * c.slab);
    } else {
        us += slabs * (rounds * c.slab + (full + (part > 0.5f ? 2 * part - 1 : 0.0f)) * c.busy);
    }
    return us;
}
Tile pick_product(ProductKind kind, int shares, int m, int n, int slabs, float *us = nullptr)
{
    Tile best = T64x64;
    float best_us = 0.0f;
    for (Tile t : kProductTiles) {
        if (slabs < kLeastSlabs[t]) continue;
        const float v = product_us(kind, t, shares, m, n, slabs);
        if (best_us == 0.0f || v < best_us) { best = t; best_us = v; }
    }
    if (us) *us = best_us;
    return best;
}
// de's words: those of whole rounds of one tile, and what is left in a launch of its own, in tiles of its own, where that is estimated to be
// faster.  8192 x 768 x 50272: 591 tiles of 256 x 256 are 2.3 rounds on 256 CUs; two rounds and 216 tiles of 192 x 128 take the whole
// call from 2094 us to 2032.  17 shapes that the rule cuts: 1.018 times as fast on average (0.998 - 1.040), to the same bits.
constexpr float kCutGain = 0.99f;
struct Words { Tile tile; int words; Tile rest; };
Words pick_words(int words, int d, int slabs)
{
    float best;
    const Tile all = pick_product(kByRows, 1, words, d, slabs, &best);
    Words w{all, words, all};
    const int n_cu = cu_count() ? cu_count() : 256;
    for (Tile t : kProductTiles) {
        if (t == T64x64 || slabs < kLeastSlabs[t]) continue;
        const int columns = (d + kTileColumns[t] - 1) / kTileColumns[t];
        const int first = (int)((int64_t)words * columns / kTileRows[t] / n_cu) * n_cu / columns * kTileRows[t];
        if (first <= 0 || first >= words) continue;
        float rest_us;
        const Tile rest = pick_product(kByRows, 1, words - first, d, slabs, &rest_us);
        const float us = product_us(kByRows, t, 1, first, d, slabs) + rest_us;
        if (us < kCutGain * best) { best = us; w = Words{t, first, rest}; }
    }
    return w;
}
// of the launch that adds up dx's shares
float shares_us(int shares, int rows, int d) { return 3.1f + (float)shares * (float)rows * (float)d * (4e-6f * 0.117f) + (shares < 8 ? 0.014f * (float)shares : 0.0f); }

size_t up(size_t v, size_t a = 256) { return (v + a - 1) / a * a; }

// A launch's size is counted in threads, by 32 bits: workgroups of 256, one a tile where tiles are 64 x 64 (the larger ones' kernel has one a CU).
constexpr int64_t kMostBlocks = (1ll << 24) - 8;
int64_t small_blocks(Tile t, int shares, int m, int n)
{
    return t == T64x64 ? ((int64_t)shares * ((m + 63) / 64) * ((n + 63) / 64) + 7) / 8 * 8 : 0;
}

}  // namespace
}  // namespace zo
