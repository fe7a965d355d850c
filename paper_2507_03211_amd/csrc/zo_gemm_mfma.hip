// Sign-batched linear layer on the matrix cores (bf16 / fp16 inputs, fp32 accumulate).
//
// This is where a ZO step spends its time: the paired forward passes of Eq. 1 (DistZO2,
// Preliminaries; PertP workflow Step 2 runs the two signs on two devices, here both signs are
// one launch on one device, rows [0, m_half) against W+ and rows [m_half, 2 m_half) against W-).
//
//   y[row, n] = sum_k x[row, k] wt[n, k]  (+ bias, ReLU, residual add)
//
// Both operands are K-contiguous ("TN"), which is what v_mfma_f32_32x32x16_{bf16,f16} wants:
// every lane feeds 8 consecutive k of one row.  The weight tile is the MFMA A operand and the
// activation tile the B operand, so a lane's 16 accumulators are 4 runs of 4 consecutive n of
// one output row, which makes the epilogue 8/16-byte stores.
//
// Three kernels (K a multiple of 64; others take the plain kernel):
//  * linear_mfma_pipe_kernel, for K of some slabs and more: one persistent workgroup of 2 x 2 waves per CU that walks its
//    XCD's share of the tile list, tiles of 256 x 256 down to 128 x 128 with slabs of 64 k.  Operand tiles go from global
//    memory straight into LDS (global_load_lds_dwordx4, no register staging), whole 128-byte lines per tile row, several
//    slabs ahead, and the pipeline runs on from one tile into the next.  16-byte chunks are XOR-swizzled on the global
//    side so that fragment reads are free of bank conflicts.  Tiles are numbered so that each XCD (its own L2) owns a
//    contiguous band of 8 tile-rows and walks it column by column.  Outputs leave through LDS as whole rows.
//  * linear_mfma_small_kernel, 64 x 64 tiles, one workgroup per tile and two or more of them per CU: any number of slabs,
//    and shapes so small that what counts is how many CUs take part.
//  * linear_mfma_split_kernel, 32 x 32 tiles whose waves share the contraction: shapes so small that each tile has a CU of its own.
// pick_tile() at the end chooses between the tile shapes.  The first two kernels and their epilogues are in zo_gemm_tiles.hip.h.
#include "zo_gemm_tiles.hip.h"

namespace zo {

namespace {

// ------------------------------------------------------------------ few tiles, deep contractions
// One output tile of 32 x 32 per workgroup; its four waves take every fourth slab of the contraction each, through rings of
// their own (kSplitStages slabs of 32 rows of x and of the weights), so that nothing waits for another wave until the four
// partial sums meet in LDS, in a fixed order.  For shapes whose tiles leave most CUs idle at 64 x 64: four times as many take part, a
// CU loads half as much a slab, and the chain of slabs is a fourth as long.  What bounds it is a CU's loads: 32 KB of lines under way at
// most, 55 B/ns from far memory and 110 from the L2.  Two stages are as fast as three (a second workgroup fits besides).
// The other tilings add up a contraction slab by slab; here every fourth slab, then the four sums.  The error is no larger, but a row's last
// bits depend on which tiling its launch takes, and so on how many rows and signs share the launch.
// Both signs of m_half x n x k, us, operands far / near, 64 x 64 tiles -> here: 96 x 1024 x 4096 20.7 / 15.5 -> 12.2 / 7.1, 213 x 576 x
// 2304 11.3 / 10.0 -> 7.0 / 5.4, 68 x 384 x 1536 8.6 / 7.6 -> 5.4 / 4.5, 213 x 576 x 576 5.6 / 4.9 -> 4.3 / 3.7.
constexpr int kSplitStages = 2, kSplitBytes = 4 * kSplitStages * 64 * BK * 2;
template <int DT, int EPI>
__global__ __launch_bounds__(256, 2) void linear_mfma_split_kernel(
    const uint16_t *__restrict__ x, const uint16_t *__restrict__ wt_p, const uint16_t *__restrict__ wt_m, const uint16_t *__restrict__ b_p,
    const uint16_t *__restrict__ b_m, void *__restrict__ y, int m_half, int n, int k, int tiles_m, int tiles_n, int total)
{
    constexpr int ST = kSplitStages, BM = 32, BN = 32, L = 8, CPR = BK / 8;      // L: loads of a slab, four of x and four of w
    extern __shared__ __attribute__((aligned(16))) uint4 smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int fr = lane & 31, fh = lane >> 5;
    const int per_xcd = (total + 7) / 8;
    const int lin = ((int)blockIdx.x & 7) * per_xcd + ((int)blockIdx.x >> 3);
    if (((int)blockIdx.x >> 3) >= per_xcd || lin >= total) return;
    int sign, trow, tcol;
    tile_at(lin, tiles_m, tiles_n, sign, trow, tcol);
    const int m0 = trow * BM, n0 = tcol * BN;
    const uint64_t xbase = uniform64((uint64_t)(uintptr_t)(x + ((size_t)sign * m_half + m0) * k));
    const uint64_t wbase = uniform64((uint64_t)(uintptr_t)((sign ? wt_m : wt_p) + (size_t)n0 * k));
    auto swz = [](int r) { return (r >> 1) & 7; };              // chunk c of row r sits at slot c ^ swz(r)
    uint32_t off[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int row = (i & 3) * 8 + (lane >> 3), first = i < 4 ? m0 : n0, end = i < 4 ? m_half : n;
        int r = first + row; r = r < end ? r : end - 1;                      // clamped: never stored
        off[i] = ((uint32_t)(r - first) * (uint32_t)k + ((lane & 7) ^ swz(row)) * 8) * 2u;
    }
    // the epilogue's operands of this thread: row tid / 8, columns 4 (tid % 8) ..
    const int er = m0 + (tid >> 3), ec = n0 + 4 * (tid & 7);
    const bool live = er < m_half && ec < n;
    const size_t eo = ((size_t)sign * m_half + (er < m_half ? er : m_half - 1)) * n + (ec < n ? ec : n - 4);
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4 *)smem + (uint32_t)wave * (ST * 8192u);
    auto load_slab = [&](int slab, uint32_t stage) {
        const uint32_t adv = (uint32_t)slab * (BK * 2);
#pragma unroll
        for (int i = 0; i < L; ++i) gload_lds16((i < 4 ? xbase : wbase) + adv, off[i], ring + stage * 8192u + (uint32_t)i * 1024u);
    };
    f32x16 acc = {};
    const int nk = k / BK, mine = (nk - wave + 3) / 4;                        // slabs wave, wave + 4, ..
#pragma unroll
    for (int s = 0; s < ST; ++s)
        if (s < mine) load_slab(wave + 4 * s, s);
    uint32_t rd = 0;
    for (int i = 0; i < mine; ++i) {
        if (i + ST - 1 < mine) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((ST - 1) * L) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const uint4 *st = smem + (wave * ST + rd) * 512;
        uint4 xf[4], wf[4];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const int slot = (2 * ks + fh) ^ swz(fr);
            xf[ks] = st[fr * CPR + slot];
            wf[ks] = st[256 + fr * CPR + slot];
        }
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) acc = mfma32<DT>(wf[ks], xf[ks], acc);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                       // the stage's reads are in registers
        if (i + ST < mine) load_slab(wave + 4 * (i + ST), rd);
        rd = rd + 1 == ST ? 0 : rd + 1;
    }
    // the four partial sums meet in LDS: row fr, runs of four columns 8 g + 4 fh
    __syncthreads();
    float *part = (float *)smem;
    constexpr int PITCH = 36;
#pragma unroll
    for (int g = 0; g < 4; ++g)
        *(float4 *)(part + (wave * 32 + fr) * PITCH + 8 * g + 4 * fh) = float4{acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
    __syncthreads();
    float v[4];
    {
        const float *q = part + (tid >> 3) * PITCH + 4 * (tid & 7);
        const f32x4 a = *(const f32x4 *)q, b = *(const f32x4 *)(q + 32 * PITCH), c = *(const f32x4 *)(q + 64 * PITCH), d = *(const f32x4 *)(q + 96 * PITCH);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (a[e] + b[e]) + (c[e] + d[e]);
    }
    if (!live) return;
    if constexpr (EPI != 3) {
        const uint2 raw = *(const uint2 *)((sign ? b_m : b_p) + ec);
        const float bias[4] = {Prec<DT>::w2f((uint16_t)(raw.x & 0xffff)), Prec<DT>::w2f((uint16_t)(raw.x >> 16)), Prec<DT>::w2f((uint16_t)(raw.y & 0xffff)), Prec<DT>::w2f((uint16_t)(raw.y >> 16))};
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += bias[e];
    }
    if constexpr (EPI < 2) {
        if constexpr (EPI == 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = v[e] > 0.0f ? v[e] : 0.0f;
        }
        uint2 o;
        o.x = (uint32_t)Prec<DT>::acc2a(v[0]) | ((uint32_t)Prec<DT>::acc2a(v[1]) << 16);
        o.y = (uint32_t)Prec<DT>::acc2a(v[2]) | ((uint32_t)Prec<DT>::acc2a(v[3]) << 16);
        *(uint2 *)((uint16_t *)y + eo) = o;
    } else {
        f32x4 *p = (f32x4 *)((float *)y + eo);
        f32x4 o = {v[0], v[1], v[2], v[3]};
        if constexpr (EPI == 2) { const f32x4 h = *p; o = f32x4{h.x + o.x, h.y + o.y, h.z + o.z, h.w + o.w}; }
        *p = o;
    }
}

// A wave's rows of a 64 x 64 tile are 64 (16-bit) or 128 bytes long: parts of cache lines, all of them when n is not a
// multiple of 64.  Written past the L2 each part is a memory transaction of its own, left there it meets the rest of its
// line.  fp32 read-modify-write: always left in the L2 (median 1.02 - 1.2 times as fast, 0.87 - 1.6, the more the shorter the
// contraction).  16-bit: left there where one or two slabs make the outputs most of the traffic and rows share lines (5740 x
// 4592 x 64 57 -> 26 us, 6217 x 6320 x 128 76 -> 57); past it otherwise, where operands want the room (2 % from 512 on; whole
// lines 4096 x 16384 x 64 70 -> 58).
template <int DT, int EPI, int TN> hipError_t launch_small(const Args &a)
{
    if constexpr (EPI < 2) {
        if (a.k >= 3 * BK || a.n % 64 == 0) return launch_small_t<DT, EPI, TN, true>(a);
    }
    return launch_small_t<DT, EPI, TN, false>(a);
}

template <int DT, int EPI> hipError_t launch_split(const Args &a)
{
    const int tiles_m = (a.m_half + 31) / 32, tiles_n = (a.n + 31) / 32, total = a.n_sign * tiles_m * tiles_n;
    auto kern = linear_mfma_split_kernel<DT, EPI>;
    static std::atomic<uint64_t> lds_allowed{0};
    const hipError_t e = once_per_device(lds_allowed, [&] {
        return hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kSplitBytes);
    });
    if (e != hipSuccess) return e;
    kern<<<dim3((total + 7) / 8 * 8), dim3(256), kSplitBytes, a.s>>>((const uint16_t *)a.x, (const uint16_t *)a.wt_p, (const uint16_t *)a.wt_m,
                                                                         (const uint16_t *)a.b_p, (const uint16_t *)a.b_m, a.y, a.m_half, a.n, a.k,
                                                                         tiles_m, tiles_n, total);
    return hipGetLastError();
}

template <int DT, int EPI> hipError_t launch_tile(Tile t, const Args &a)
{
    switch (t) {
    case T256x256: return launch_pipe<DT, EPI, Shape<4, 4, 2>>(a);
    case T256x192: return launch_pipe<DT, EPI, Shape<4, 3, 2>>(a);
    case T256x128: return launch_pipe<DT, EPI, Shape<4, 2, 2>>(a);
    case T192x128: return launch_pipe<DT, EPI, Shape<3, 2, 3>>(a);
    case T128x128: return launch_pipe<DT, EPI, Shape<2, 2, 4>>(a);
    case T64x64: return launch_small<DT, EPI, 1>(a);
    default: return launch_split<DT, EPI>(a);
    }
}

// Do the 32 x 32 tiles get a CU each, and five slabs at least?  They are then faster than any other shape: over 159 shapes (24 - 870 rows
// a sign, n 80 - 5120, k 320 - 14592, all epilogues) 1.52 times in the geometric mean, 1.19 at least, operands far; over 30 others
// far 1.57 (1.18 - 2.05), near 1.74 (1.20 - 2.49).
// The line is short of where they stop gaining.  From one to two tiles a CU they gain 1.12 far, 1.18 near in the mean (39 shapes), up to
// 1.26 and 1.33, but lose up to 8 and 12 % where a sign has few rows and many columns (28 x 4944 x 5248 28.1 -> 30.5 us, 25 x 4544 x 384
// 4.7 -> 4.9); past two they lose (536 x 512 x 2048 12.7 -> 13.1, 642 x 400 x 9280 39.9 -> 47.3).  With two to four slabs they gain 1.15
// (1.07 - 1.27, 0.3 - 0.6 us of a launch's 3.5; 30 shapes of up to a tile a CU).  Both are left to 64 x 64 tiles, with the bits they have there.
bool one_small_tile_a_cu(int n_sign, int m_half, int n, int k)
{
    const long tiles = (long)n_sign * ((m_half + 31) / 32) * ((n + 31) / 32);
    return k >= 5 * BK && tiles <= (cu_count() ? cu_count() : 256);
}

// The tile shape with the least estimated time in us: start + rounds (slabs slab + epilogue), where a round of tiles that
// fills more than half of the CUs also pays slabs busy b, b = 0 .. 1 from half full to full (a full chip clocks lower and
// shares the fabric).  fp32 outputs are paid for by the rounds' share of the chip (their bursts share the memory), with and
// without the running sum read, the first round at a price of its own: the caches take part of it, and of what a 64 x 64
// tile writes nearly all, while from the second round on it pays most per byte (half lines).
// Constants: least squares over 90 shapes (m_half 96 .. 8192, n and k 512 .. 19200) timed with every tile shape; those of
// fp32 outputs over 973 shapes (m_half 64 .. 8192, n 240 .. 20000, k from 64): one price for both fp32 epilogues and all
// rounds, from shapes of k >= 512 alone, had sent short contractions with large outputs to 64 x 64 tiles, up to twice the
// time of the code before the rule (us, that / one price / here: 1374 x 14048 x 384 fp32 57 / 92 / 55, 2185 x 15512 x 512
// residual 168 / 230 / 170).  Over 1688 shapes of more than 11 us, all epilogues: on average 1.2 % slower than the best tile
// of each; 12 more than 5 % slower than the code before, the worst 12 %.
// The 256 x 256 tile gets 3 % credit: near a tie it is the one that long contractions lose least with.  In us, picked
// here / the former choice between 256 x 256 and a register-staged 128 x 128 kernel, m_half x n x k: 536 x 2304 x 768
// 9.0 / 17.1, 692 x 5120 x 5120 84 / 115, 1028 x 1024 x 4096 30 / 53, 391 x 704 x 2816 13 / 39, 8192 x 2304 x 768 61 / 70.
Tile pick_tile(int n_sign, int m_half, int n, int k, int epi)
{
    struct Out { float first, more; };
    static const struct { int min_slabs; float start, slab, busy, out16; Out rmw, out32; } kCost[T32x32] = {
        {3, 4.9f, 1.00f, 0.52f, 3.5f, {26.1f, 21.3f}, {9.0f, 11.4f}}, {3, 3.6f, 0.79f, 0.38f, 3.1f, {20.9f, 16.7f}, {7.0f, 9.0f}},
        {3, 3.6f, 0.59f, 0.28f, 1.6f, {12.0f, 11.4f}, {2.7f, 7.0f}},  {4, 4.1f, 0.49f, 0.21f, 0.9f, {7.9f, 7.6f}, {1.2f, 5.0f}},
        {5, 4.1f, 0.38f, 0.16f, 0.3f, {4.3f, 4.5f}, {0.0f, 3.1f}},    {1, 2.6f, 0.21f, 0.41f, 0.4f, {0.5f, 2.5f}, {0.0f, 1.3f}}};
    if (one_small_tile_a_cu(n_sign, m_half, n, k)) return T32x32;
    const float n_cu = cu_count() ? (float)cu_count() : 256.0f, slabs = (float)(k / BK);
    Tile best = kTiles;
    float best_us = 0.0f;
    for (int t = 0; t < T32x32; ++t) {
        const auto &c = kCost[t];
        if (k / BK < c.min_slabs) continue;
        const float tiles = (float)n_sign * (float)((m_half + kTileRows[t] - 1) / kTileRows[t]) * (float)((n + kTileColumns[t] - 1) / kTileColumns[t]);
        const float slots = t == T64x64 ? 2 * n_cu : n_cu;        // workgroups at a time
        const float full = __builtin_floorf(tiles / slots), part = tiles / slots - full, rounds = full + (part > 0 ? 1.0f : 0.0f);
        float us = c.start;
        if (t == T64x64) {
            // two workgroups per CU: `slab` for one alone, `busy` for the two together
            const float lone = part > 0 && part <= 0.5f ? 1.0f : 0.0f;
            us += slabs * ((rounds - lone) * c.busy + lone * c.slab);
        } else {
            us += slabs * (rounds * c.slab + (full + (part > 0.5f ? 2 * part - 1 : 0.0f)) * c.busy);
        }
        const Out &o = epi == 2 ? c.rmw : c.out32;
        us += epi < 2 ? c.out16 * rounds : full + part < 1 ? o.first * part : o.first + o.more * (full + part - 1);
        if (t == T256x256) us *= 0.97f;
        if (best == kTiles || us < best_us) { best = (Tile)t; best_us = us; }
    }
    return best;
}

// LM head (epilogue 4): strips of 128 columns per (max, sum-exp) pair when tiles 256 columns wide fill half the CUs, else
// strips of 64.  The callers' scratch is sized for either.
bool wide_strips(int n_sign, int m_half, int n, int k)
{
    if (k < 3 * BK) return false;
    const long tiles = (long)n_sign * ((m_half + 255) / 256) * ((n + 255) / 256);
    return tiles >= 128;
}

// Its tile.  256 columns wide: the height of least estimated time in us, start + slabs (rounds slab + r share) + rounds out +
// r out_share, with r the rounds and the last one's fraction.  Constants: least squares over 1100 shapes (40 - 4500 rows a
// sign, vocabularies 2 k - 64 k and OPT's 50272, d 192 - 2700) timed with each height; the picked one is on average 0.15 %
// slower than the best.  (By padded rows alone, from one vocabulary, shorter tiles were taken where they need a round more:
// 616 rows, d 1280, 6824 columns 31.8 us at 256, 37.4 at 128.)  In us, heights 256 / 192 / 128, vocabulary 50272: 1048
// rows, d 2048, 419 / 399 / 428; 700 rows, d 1024, 148 / 159 / 161; 536 rows, d 768, 118 / 98 / 109; 300 rows 92 / 83 /
// 76; 100 rows 54 / 51 / 46.  (These last while the epilogue spent one instruction more per logit, 1 - 2 % of each.)
enum HeadTile { H256x256, H192x256, H128x256, H128x128, H64x128 };
HeadTile pick_head(int n_sign, int m_half, int n, int k)
{
    if (!wide_strips(n_sign, m_half, n, k)) return k / BK > 4 ? H128x128 : H64x128;
    static const struct { int rows, min_slabs; float start, slab, share, out, out_share; } kCost[3] = {
        {256, 3, 9.2f, 0.99f, 0.44f, 3.6f, 0.0f}, {192, 3, 9.0f, 1.13f, 0.0f, 2.4f, 0.4f}, {128, 4, 9.2f, 0.86f, 0.0f, 1.3f, 0.3f}};
    const float n_cu = cu_count() ? (float)cu_count() : 256.0f, slabs = (float)(k / BK);
    HeadTile best = H256x256;
    float best_us = 0.0f;
    for (int t = 0; t < 3; ++t) {
        const auto &c = kCost[t];
        if (k / BK < c.min_slabs) continue;
        const float r = (float)n_sign * (float)((m_half + c.rows - 1) / c.rows) * (float)((n + 255) / 256) / n_cu;
        const float us = c.start + slabs * (__builtin_ceilf(r) * c.slab + r * c.share) + __builtin_ceilf(r) * c.out + r * c.out_share;
        if (t == 0 || us < best_us) { best = (HeadTile)t; best_us = us; }
    }
    return best;
}

template <int DT> hipError_t launch_ce(const Args &a)
{
    switch (pick_head(a.n_sign, a.m_half, a.n, a.k)) {
    case H256x256: return launch_pipe<DT, 4, Shape<4, 4, 2>>(a);
    case H192x256: return launch_pipe<DT, 4, Shape<3, 4, 2>>(a);
    case H128x256: return launch_pipe<DT, 4, Shape<2, 4, 3>>(a);
    case H128x128: return launch_pipe<DT, 4, Shape<2, 2, 4>>(a);
    default: return launch_small<DT, 4, 2>(a);
    }
}

template <int DT> hipError_t launch_t(const Args &a, int epi)
{
    const Tile t = epi == 4 ? kTiles : pick_tile(a.n_sign, a.m_half, a.n, a.k, epi);
    switch (epi) {
    case 0: return launch_tile<DT, 0>(t, a);
    case 1: return launch_tile<DT, 1>(t, a);
    case 2: return launch_tile<DT, 2>(t, a);
    case 3: return launch_tile<DT, 3>(t, a);
    default: return launch_ce<DT>(a);
    }
}

}  // namespace

int mfma_linear_tile(int n_sign, int m_half, int n, int k, int epilogue)
{
    if (!mfma_linear_supported(m_half, n, k)) return 0;
    if (epilogue == 4) {
        static const int kHead[] = {256 << 16 | 256, 192 << 16 | 256, 128 << 16 | 256, 128 << 16 | 128, 64 << 16 | 128};
        return kHead[pick_head(n_sign, m_half, n, k)];
    }
    const Tile t = pick_tile(n_sign, m_half, n, k, epilogue);
    return kTileRows[t] << 16 | kTileColumns[t];
}

int mfma_ce_partials(int n_sign, int m_half, int n, int k) { return wide_strips(n_sign, m_half, n, k) ? 2 * ((n + 255) / 256) : 2 * ((n + 127) / 128); }

bool mfma_linear_supported(int m_half, int n, int k) { return m_half >= 1 && n >= 8 && n < kMaxColumns && n % 8 == 0 && k >= BK && k % BK == 0; }

hipError_t launch_linear_mfma(const void *x, const void *wt_p, const void *wt_m, const void *b_p, const void *b_m, void *y,
                              int dtype, int n_sign, int m_half, int n, int k, int epilogue, hipStream_t s)
{
    if (!mfma_linear_supported(m_half, n, k) || (dtype != kBF16 && dtype != kFP16)) return hipErrorInvalidValue;
    // 16-byte pieces everywhere (operand loads, row-wise stores, bias through the scalar cache)
    if ((uintptr_t)x % 16 || (uintptr_t)wt_p % 16 || (uintptr_t)wt_m % 16 || (uintptr_t)y % 16) return hipErrorInvalidValue;
    if (epilogue != 3 && epilogue != 4 && ((uintptr_t)b_p % 16 || (uintptr_t)b_m % 16)) return hipErrorInvalidValue;
    const Args a{x, wt_p, wt_m, b_p, b_m, y, n_sign, m_half, n, k, s};
    return dtype == kBF16 ? launch_t<kBF16>(a, epilogue) : launch_t<kFP16>(a, epilogue);
}

}  // namespace zo
