// Gradient of the tied LM head and its cross entropy on the matrix cores (bf16 / fp16 parameters).
//
//   l = x e^T,  lse_r = log sum_v exp(l_rv),  G = exp(l - lse) - onehot(target),  dx = scale G e,  de = scale G^T x
//
// G exists one piece of the vocabulary at a time, rounded to the parameters' 16-bit type because that is what the matrix instructions
// take: each element is off by half a step, a product's sum by about as much as its own final rounding (the largest element, that of the
// target, is p - 1 formed in fp32).  Where one piece holds the whole vocabulary there are three products of 2 rows vocab d flop: the logits
// leave 16-bit distances from their strip's maximum where G will lie, with the strips' (maximum, sum) pairs, and a pass over these makes G.
// Where it takes more, four: the logits for lse alone (the fused cross entropy of the forward pass, which leaves pairs and no logits), then
// again, piece by piece, for G.  Operands stay as they lie: G, e and x are read with the contraction as the outer index where a
// product wants it so (zo_gemm_tiles.hip.h).
#include "zo_gemm_tiles.hip.h"

namespace zo {

namespace {

// ------------------------------------------------------------------ around the products
// Row r as the products over rows take it: x [rows, d] -> [rows_p, dp], zeros in rows that do not count (so that whatever these hold meets
// no sum), in rows beyond the last and in columns beyond d.  Eight elements a thread and turn.
__device__ __forceinline__ void head_row(const uint16_t *__restrict__ x, uint4 *__restrict__ out, int r, bool counts, int d, int dp, int first, int step)
{
    for (int c = first; c < dp / 8; c += step)
        out[(size_t)r * (dp / 8) + c] = counts && 8 * c < d ? *(const uint4 *)(x + (size_t)r * d + 8 * c) : uint4{0, 0, 0, 0};
}
__global__ __launch_bounds__(256) void head_rows_kernel(const uint16_t *__restrict__ x, const int32_t *__restrict__ target, uint4 *__restrict__ out, int rows, int d, int dp)
{
    const int r = blockIdx.x;
    head_row(x, out, r, r < rows && target[r] >= 0, d, dp, threadIdx.x, 256);
}

// A row's (maximum, sum) pairs -> its loss and what G takes of it: logsumexp rounded to fp32 and the exponent's share on top, which is
// the rest of it in units of log 2 and, in fp16, the factor 2^15.  Rows that do not count: loss 0, infinity (G = 0).  One wavefront a row.
__global__ __launch_bounds__(256) void head_lse_kernel(const float2 *__restrict__ partials, int n_partial, const float *__restrict__ target_logit,
                                                       const int32_t *__restrict__ target, float *__restrict__ row_loss, float2 *__restrict__ stats, int rows,
                                                       int vocab, float shift)
{
    const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (r >= rows) return;
    const int tg = target[r];
    if (tg < 0) {
        if (lane == 0) { row_loss[r] = 0.0f; stats[r] = float2{INFINITY, 0.0f}; }
        return;
    }
    const float2 *p = partials + (size_t)r * n_partial;
    constexpr int KEEP = 8;                                     // in registers, all under way together; the rest is read twice
    float2 v[KEEP];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) v[i] = lane + 64 * i < n_partial ? p[lane + 64 * i] : float2{-INFINITY, 0.0f};
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) mx = v[i].x > mx ? v[i].x : mx;
    for (int i = lane + 64 * KEEP; i < n_partial; i += 64) mx = p[i].x > mx ? p[i].x : mx;
    mx = wave_max(mx);
    double s = 0.0;
    auto add = [&](float2 q) {
        if (q.y != 0.0f) s += (double)q.y * (double)__expf(q.x - mx);           // (NaN is not left out, whatever its maximum)
    };
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (64 * i < n_partial) add(v[i]);
    for (int i = lane + 64 * KEEP; i < n_partial; i += 64) add(p[i]);
    s = wave_sum(s);
    if (lane != 0) return;
    const double lse = tg < vocab ? log(s) + (double)mx : (double)__builtin_nan("");
    const float hi = (float)lse;
    row_loss[r] = (float)(lse - (double)target_logit[r]);
    stats[r] = float2{hi, (float)(((double)hi - lse) * 1.4426950408889634) + shift};
}

// Distances and pairs of a row -> its loss and, in place, its G (as in epilogue 5); zeros in rows that do not count, past the last row and past
// the last word.  Workgroup (r, y) takes the y-th part of a row, which works its logsumexp again; four of them are on a CU.  us of the
// whole call with 1 / 2 / 4 parts, 768 x 50272: 20 rows 70.4 / 66.2 / 64.1, 100 rows 81.4 / 77.3 / 76.1, 300 rows 138.4 / 135.8 / 136.5,
// 600 rows 218.4 / 218.0 / 221.2, 1048 rows 317 / 312 / 318, 2048 rows 541 / 544 / 557; 512 x 10000: 64 rows 28.8 / 28.1 / 27.8, 300 rows
// 44.4 / 44.4 / 46.4, 500 rows 47.4 / 48.5 / 52.5, 1000 rows 69.4 / 72.1 / 80.8.  Bound by memory,
// 4 bytes a word.  NT: what passes the memory-side cache anyway goes past the L2, 8192 rows 339 -> 306 us (5.4 TB/s); 300 rows 18 -> 20.
// `xs`, if not null: takes the row of x on the way (see head_row), where the logits come from x itself.
template <int DT, bool NT>
__global__ __launch_bounds__(512) void head_gradient_kernel(uint4 *__restrict__ grad, const float2 *__restrict__ pairs, int n_pairs, int strip,
                                                            const float *__restrict__ hit, const int32_t *__restrict__ target, float *__restrict__ row_loss,
                                                            int rows, int vocab, int width, const uint16_t *__restrict__ x, uint4 *__restrict__ xs, int d)
{
    __shared__ float red_f[16];
    __shared__ double red_d[16];
    constexpr float kOne = DT == kFP16 ? 32768.0f : 1.0f, kShift = DT == kFP16 ? 15.0f : 0.0f;
    const int r = blockIdx.x, tg = r < rows ? target[r] : -1;
    uint4 *out = grad + (size_t)r * (width / 8);
    auto load = [](const uint4 *at) { return NT ? __builtin_bit_cast(uint4, __builtin_nontemporal_load((const u32x4 *)at)) : *at; };
    const int each = (width / 8 + gridDim.y - 1) / gridDim.y, first = each * blockIdx.y, last = first + each < width / 8 ? first + each : width / 8;
    if (xs && blockIdx.y == gridDim.y - 1) head_row(x, xs, r, tg >= 0, d, d, threadIdx.x, 512);
    if (tg < 0) {
        if (r < rows && threadIdx.x == 0 && blockIdx.y == 0) row_loss[r] = 0.0f;
        for (int c = first + threadIdx.x; c < last; c += 512) out[c] = uint4{0, 0, 0, 0};
        return;
    }
    const float2 *p = pairs + (size_t)r * n_pairs;
    uint4 q = first + (int)threadIdx.x < last ? load(out + first + threadIdx.x) : uint4{0, 0, 0, 0};      // on its way while logsumexp is worked
    float mx = -INFINITY;
    for (int i = threadIdx.x; i < n_pairs; i += 512) mx = p[i].x > mx ? p[i].x : mx;
    mx = block_max(mx, red_f);
    double s = 0.0;                                             // (a strip with a NaN is not left out, whatever its maximum)
    for (int i = threadIdx.x; i < n_pairs; i += 512)
        if (p[i].y != 0.0f) s += (double)p[i].y * (double)__expf(p[i].x - mx);
    s = block_sum(s, red_d);
    const double lse = tg < vocab ? log(s) + (double)mx : (double)__builtin_nan("");
    if (threadIdx.x == 0 && blockIdx.y == 0) row_loss[r] = (float)(lse - (double)hit[r]);
    const float hi = (float)lse, rest = (float)(((double)hi - lse) * 1.4426950408889634) + kShift;
    const float at_target = tg < vocab ? __builtin_amdgcn_exp2f(__builtin_fmaf(hit[r] - hi, 1.44269504f, rest)) - kOne : 0.0f;
    for (int c = first + threadIdx.x; c < last; c += 512) {
        const uint4 next = c + 512 < last ? load(out + c + 512) : uint4{0, 0, 0, 0};
        if (8 * c < vocab) {                                   // (words are a multiple of eight)
            const float base = __builtin_fmaf(p[8 * c / strip].x - hi, 1.44269504f, rest);
            const float none = base - INFINITY;                // of the last step; a row that is not a number stays one
            uint32_t *words = &q.x;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t lo = words[e] & 0xffff, up = words[e] >> 16;
                auto value = [&](uint32_t steps) {
                    return __builtin_amdgcn_exp2f(__builtin_fmaf((float)steps, -1.44269504f * 32.0f / 65535.0f, steps == 65535 ? none : base));
                };
                words[e] = pack2<DT>(value(lo), value(up));
            }
            if (c == tg >> 3) {
                const uint32_t t = Prec<DT>::acc2a(at_target);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if ((tg & 7) >> 1 == e) words[e] = tg & 1 ? (words[e] & 0xffff) | t << 16 : (words[e] & ~0xffffu) | t;
            }
        } else {
            q = uint4{0, 0, 0, 0};
        }
        if constexpr (NT) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, q), (u32x4 *)(out + c));
        else out[c] = q;
        q = next;
    }
}

// dx = rn(alpha sum_z part[z]): the shares of the contraction over the vocabulary.  Eight elements a thread; with L > 1 the workgroup's L
// groups of threads take every L-th share each, and their sums meet in LDS (20 rows of 768, 40 shares: 6.6 us with L = 1).
template <int DT, int L>
__global__ __launch_bounds__(256) void head_dx_kernel(const float4 *__restrict__ part, int shares, size_t n8, float alpha, uint4 *__restrict__ dx)
{
    constexpr int N = 256 / L;
    __shared__ float4 sums[L > 1 ? L : 1][N][2];
    const int group = threadIdx.x / N, t = threadIdx.x % N;
    const size_t step = (size_t)gridDim.x * N;
    for (size_t i0 = (size_t)blockIdx.x * N; i0 < n8; i0 += step) {
        const size_t i = i0 + t < n8 ? i0 + t : n8 - 1;
        float4 a{0, 0, 0, 0}, b{0, 0, 0, 0};
#pragma unroll 4
        for (int z = group; z < shares; z += L) {
            const float4 p = part[2 * (z * n8 + i)], q = part[2 * (z * n8 + i) + 1];
            a = float4{a.x + p.x, a.y + p.y, a.z + p.z, a.w + p.w};
            b = float4{b.x + q.x, b.y + q.y, b.z + q.z, b.w + q.w};
        }
        if constexpr (L > 1) {
            __syncthreads();
            sums[group][t][0] = a;
            sums[group][t][1] = b;
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int g = 1; g < L; ++g) {
                    const float4 p = sums[g][t][0], q = sums[g][t][1];
                    a = float4{a.x + p.x, a.y + p.y, a.z + p.z, a.w + p.w};
                    b = float4{b.x + q.x, b.y + q.y, b.z + q.z, b.w + q.w};
                }
            }
        }
        auto two = [&](float lo, float hi) { return pack2<DT>(alpha * lo, alpha * hi); };
        if (group == 0 && i0 + t < n8) dx[i] = uint4{two(a.x, a.y), two(a.z, a.w), two(b.x, b.y), two(b.z, b.w)};
    }
}

// ------------------------------------------------------------------ the products
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
using Logits = Product<false, false>;       // x rows, words: both with k inside
using ByRows = Product<true, true>;         // G^T x: contraction over the rows, outside in both
using ByWords = Product<false, true>;       // G e: contraction over the words, outside in e

// dx's shares and de in one launch, where few rows have both in 64 x 64 tiles: dx reads e while de is written.  dx first, and rings of two stages,
// five workgroups to a CU, for both.  us of the whole call, over and over on the same buffers (20 rows take 69.5 where every call has an
// e and a de of its own, 61.7 beside that on one pair), two launches / one: 20 rows of 768 x 50272 64.1 / 61.0 (rings of three 64.3, of four
// 72.4, de first 64.4, the two interleaved 73.7), 20 of 2048 156.5 / 144.1, 64 of 512 x 10000 27.7 / 25.1, 100 of 512 x 20000 39.8 / 35.9,
// 20 of 5120 x 8192 70.6 / 67.5.  Long contractions want the deeper ring and stay by themselves: by slabs a
// share, 1 row of 4096 x 32000 (62) 195.0 / 181.3, 33 of 4096 x 20000 (78) 106.0 / 109.6, 64 of 2048 x 50272 (98) 155.7 / 153.2, 1 of 5120 x 128000
// (125) 821.9 / 873.4, 20 of 8192 x 50272 (196) 572.7 / 585.7; 4000 rows of 8 x 64, 63 slabs in de, 50.8 / 62.9.
constexpr int kBothSlabs = 64, kBothRows = 512;
struct SmallTiles { const uint16_t *x, *w; void *y; int m, n, k, tiles_m, tiles_n, total; };
constexpr int kBothStages = 2;
template <int DT>
__global__ __launch_bounds__(256, 2) void head_both_kernel(SmallTiles a, SmallTiles b, ByWords::Arg op_a, ByRows::Arg op_b, int blocks_a)
{
    if ((int)blockIdx.x < blocks_a)
        small_tile<DT, 7, 1, false, ByWords, kBothStages>(a.x, a.w, nullptr, nullptr, nullptr, a.y, a.m, a.n, a.k, a.tiles_m, a.tiles_n, a.total, op_a, (int)blockIdx.x);
    else
        small_tile<DT, 6, 1, false, ByRows, kBothStages>(b.x, b.w, nullptr, nullptr, nullptr, b.y, b.m, b.n, b.k, b.tiles_m, b.tiles_n, b.total, op_b, (int)blockIdx.x - blocks_a);
}
template <int DT> hipError_t launch_both(const Args &dx, const ByWords::Arg &op_dx, const Args &de, const ByRows::Arg &op_de)
{
    auto tiles = [](const Args &a) {
        const int tm = (a.m_half + 63) / 64, tn = (a.n + 63) / 64;
        return SmallTiles{(const uint16_t *)a.x, (const uint16_t *)a.wt_p, a.y, a.m_half, a.n, a.k, tm, tn, a.n_sign * tm * tn};
    };
    const SmallTiles a = tiles(dx), b = tiles(de);
    const int blocks_a = (a.total + 7) / 8 * 8, blocks_b = (b.total + 7) / 8 * 8;
    head_both_kernel<DT><<<dim3(blocks_a + blocks_b), dim3(256), kBothStages * kSmallStageBytes<1>, dx.s>>>(a, b, op_dx, op_de, blocks_a);
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

// G is held for `width` words at a time: as many as kPieceBytes hold (8192 rows: the whole of 50272 words), in `shares` shares of
// share_words for the product with e, whose outputs [rows, d] are few tiles where rows are few.
constexpr size_t kPieceBytes = 1u << 30;
struct HeadPlan {
    int rows_p, dp, width, pieces, shares, share_words, pairs, strip;
    Tile logits, by_words;
    Words by_rows;                              // of a whole piece
    bool both;                                  // de and dx in one launch
    bool fits;                                  // every launch's tiles
    size_t xs, g, stats, pair, hit, part, total;
};
// A launch's size is counted in threads, by 32 bits: workgroups of 256, one a tile where tiles are 64 x 64 (the larger ones' kernel has one a CU).
constexpr int64_t kMostBlocks = (1ll << 24) - 8;
int64_t small_blocks(Tile t, int shares, int m, int n)
{
    return t == T64x64 ? ((int64_t)shares * ((m + 63) / 64) * ((n + 63) / 64) + 7) / 8 * 8 : 0;
}
HeadPlan head_plan(int rows, int d, int vocab)
{
    HeadPlan p{};
    p.rows_p = (rows + BK - 1) / BK * BK;
    p.dp = (d + BK - 1) / BK * BK;
    const size_t fit = kPieceBytes / (2 * (size_t)p.rows_p) / BK * BK;
    const int most = (int)(fit < (size_t)BK ? BK : fit > (size_t)vocab ? (size_t)vocab : fit);
    const int whole = (vocab + BK - 1) / BK;                     // slabs of words
    p.pieces = (vocab + most - 1) / most;
    const int slabs = (whole + p.pieces - 1) / p.pieces;
    float best = 0.0f;
    for (int z = 1; z <= 64 && z <= slabs; z += z < 8 ? 1 : z < 16 ? 2 : 4) {
        float us;
        const Tile t = pick_product(kByWords, z, rows, d, (slabs + z - 1) / z, &us);
        us += shares_us(z, rows, d);
        if (best == 0.0f || us < best) { best = us; p.shares = z; p.by_words = t; }
    }
    p.share_words = (slabs + p.shares - 1) / p.shares * BK;
    p.width = p.share_words * p.shares;
    p.pieces = (vocab + p.width - 1) / p.width;
    const int columns = p.pieces == 1 ? p.width : vocab;          // of the first product
    p.logits = pick_product(kLogits, 1, p.rows_p, columns, p.dp / BK);
    p.strip = kTileColumns[p.logits] / 2;                        // a wavefront's columns of the tile
    p.pairs = 2 * ((columns + kTileColumns[p.logits] - 1) / kTileColumns[p.logits]);
    const int words = vocab < p.width ? vocab : p.width;
    p.by_rows = pick_words(words, d, p.rows_p / BK);
    p.both = p.pieces == 1 && p.by_rows.tile == T64x64 && p.by_rows.words == words && p.by_words == T64x64 && p.share_words <= kBothSlabs * BK && p.rows_p <= kBothRows;
    // (a piece's logits are 2^30 bytes; its words behind whole rounds of tiles are fewer than a round)
    const int64_t de = small_blocks(p.by_rows.tile, 1, p.by_rows.words, d), dx = small_blocks(p.by_words, p.shares, rows, d);
    p.fits = small_blocks(p.logits, 1, p.rows_p, columns) <= kMostBlocks && de <= kMostBlocks && dx <= kMostBlocks && (!p.both || de + dx <= kMostBlocks);
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o = up(o + bytes); return at; };
    p.xs = take(2 * (size_t)p.rows_p * p.dp);
    p.stats = p.pieces == 1 ? 0 : take((size_t)rows * sizeof(float2));
    p.pair = take((size_t)rows * p.pairs * 8);
    p.hit = take(4 * (size_t)rows);
    p.g = take(2 * (size_t)p.rows_p * p.width);
    p.part = take(4 * (size_t)p.shares * rows * d);
    p.total = o;
    return p;
}

template <int DT>
hipError_t head_grad(const uint16_t *x, const uint16_t *e, const int32_t *target, float *row_loss, uint16_t *dx, uint16_t *de, char *ws, int rows, int d,
                     int vocab, float scale, hipStream_t s)
{
    const HeadPlan p = head_plan(rows, d, vocab);
    if (!p.fits) return hipErrorNotSupported;
    uint16_t *xs = (uint16_t *)(ws + p.xs), *g = (uint16_t *)(ws + p.g);
    float2 *stats = (float2 *)(ws + p.stats);
    float *part = (float *)(ws + p.part);
    const float alpha = DT == kFP16 ? scale * 0x1p-15f : scale;
    hipError_t err = hipSuccess;
    // the logits of a whole vocabulary come from x itself where its rows are whole slabs: the copy is made on the way, with G
    const bool direct = p.pieces == 1 && p.dp == d;
    if (!direct) {
        head_rows_kernel<<<dim3(p.rows_p), dim3(256), 0, s>>>(x, target, (uint4 *)xs, rows, d, p.dp);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    auto logits_of = [&](int v0, int words) {
        Logits::Arg op{};
        op.ldx = p.dp;
        op.ldw = op.w_row = d;
        op.w_end = (uint64_t)(uintptr_t)(e + (size_t)vocab * d);
        op.stats = stats; op.target = target; op.rows = rows; op.words = words; op.first_word = v0;
        return op;
    };
    float2 *pair = (float2 *)(ws + p.pair);
    float *hit = (float *)(ws + p.hit);
    if (p.pieces == 1) {
        Logits::Arg op = logits_of(0, vocab);
        op.pairs = pair; op.hit = hit;
        const Args a{direct ? x : xs, e, nullptr, nullptr, nullptr, g, 1, direct ? rows : p.rows_p, p.width, p.dp, s};
        if ((err = launch_product<DT, 9, Logits>(p.logits, a, op)) != hipSuccess) return err;
        const int enough = 640 / p.rows_p, parts = enough < 1 ? 1 : enough < 4 ? enough : 4;
        auto gradient = p.rows_p * (size_t)p.width * 2 > (size_t)256 << 20 ? head_gradient_kernel<DT, true> : head_gradient_kernel<DT, false>;
        gradient<<<dim3(p.rows_p, parts), dim3(512), 0, s>>>((uint4 *)g, pair, p.pairs, p.strip, hit, target, row_loss, rows, vocab, p.width, x,
                                                             direct ? (uint4 *)xs : nullptr, d);
    } else {
        const Args a{xs, e, nullptr, target, hit, pair, 1, rows, vocab, p.dp, s};
        if ((err = launch_product<DT, 4, Logits>(p.logits, a, logits_of(0, vocab))) != hipSuccess) return err;
        head_lse_kernel<<<dim3((rows + 3) / 4), dim3(256), 0, s>>>(pair, p.pairs, hit, target, row_loss, stats, rows, vocab, DT == kFP16 ? 15.0f : 0.0f);
    }
    if ((err = hipGetLastError()) != hipSuccess) return err;
    ByWords::Arg op_by_words{};
    op_by_words.ldx = p.width; op_by_words.ldw = d;
    op_by_words.xz = p.share_words; op_by_words.wz = (uint64_t)p.share_words * d;
    op_by_words.w_end = (uint64_t)(uintptr_t)(e + (size_t)vocab * d);
    auto by_words = [&](int v0) { return Args{g, e + (size_t)v0 * d, nullptr, nullptr, nullptr, part, p.shares, rows, d, p.share_words, s}; };
    for (int v0 = 0; v0 < vocab; v0 += p.width) {
        const int words = vocab - v0 < p.width ? vocab - v0 : p.width;
        if (p.pieces > 1) {
            const Logits::Arg op = logits_of(v0, words);
            const Args a{xs, e + (size_t)v0 * d, nullptr, nullptr, nullptr, g, 1, p.rows_p, p.width, p.dp, s};
            if ((err = launch_product<DT, 5, Logits>(pick_product(kLogits, 1, p.rows_p, p.width, p.dp / BK), a, op)) != hipSuccess) return err;
        }
        {
            ByRows::Arg op{};
            op.ldx = p.width; op.ldw = p.dp;
            op.x_end = (uint64_t)(uintptr_t)(g + (size_t)p.rows_p * p.width);
            op.w_end = (uint64_t)(uintptr_t)(xs + (size_t)p.rows_p * p.dp);
            op.alpha = alpha;
            const Words w = words == p.width || p.pieces == 1 ? p.by_rows : pick_words(words, d, p.rows_p / BK);
            const Args a{g, xs, nullptr, nullptr, nullptr, de + (size_t)v0 * d, 1, w.words, d, p.rows_p, s};
            if (p.both) {
                if ((err = launch_both<DT>(by_words(v0), op_by_words, a, op)) != hipSuccess) return err;
                continue;
            }
            if ((err = launch_product<DT, 6, ByRows>(w.tile, a, op)) != hipSuccess) return err;
            if (w.words < words) {
                const Args b{g + w.words, xs, nullptr, nullptr, nullptr, de + (size_t)(v0 + w.words) * d, 1, words - w.words, d, p.rows_p, s};
                if ((err = launch_product<DT, 6, ByRows>(w.rest, b, op)) != hipSuccess) return err;
            }
        }
        err = v0 == 0 ? launch_product<DT, 7, ByWords>(p.by_words, by_words(v0), op_by_words) : launch_product<DT, 8, ByWords>(p.by_words, by_words(v0), op_by_words);
        if (err != hipSuccess) return err;
    }
    const size_t n8 = (size_t)rows * d / 8;
    auto sum = [&](auto kern, size_t each) {
        const size_t blocks = (n8 + each - 1) / each;
        kern<<<dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s>>>((const float4 *)part, p.shares, n8, alpha, (uint4 *)dx);
    };
    if (p.shares >= 8) sum(head_dx_kernel<DT, 8>, 32);
    else sum(head_dx_kernel<DT, 1>, 256);
    return hipGetLastError();
}

}  // namespace

size_t head_grad_mfma_scratch(int rows, int d, int vocab)
{
    const HeadPlan p = head_plan(rows, d, vocab);
    return p.fits ? p.total : 0;
}

bool head_grad_mfma_plan(int rows, int d, int vocab, int32_t *plan)
{
    const HeadPlan p = head_plan(rows, d, vocab);
    if (!p.fits) return false;
    auto tile = [](Tile t) { return kTileRows[t] << 16 | kTileColumns[t]; };
    plan[0] = tile(pick_product(kLogits, 1, p.rows_p, p.width, p.dp / BK));
    plan[1] = tile(p.by_rows.tile);
    plan[2] = tile(p.by_words);
    plan[3] = p.shares;
    plan[4] = p.pieces;
    plan[5] = p.by_rows.words;
    plan[6] = tile(p.by_rows.rest);
    return true;
}

hipError_t launch_head_grad_mfma(const void *x, const void *e, const int32_t *target, void *row_loss, void *dx, void *de, void *scratch, int dtype, int rows,
                                 int d, int vocab, float scale, hipStream_t s)
{
    auto f = dtype == kBF16 ? head_grad<kBF16> : head_grad<kFP16>;
    return f((const uint16_t *)x, (const uint16_t *)e, target, (float *)row_loss, (uint16_t *)dx, (uint16_t *)de, (char *)scratch, rows, d, vocab, scale, s);
}

}  // namespace zo
