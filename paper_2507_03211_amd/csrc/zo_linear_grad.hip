// Backward pass of the linear layer y = x W^T + b with the forward call's epilogues: G = dy, or dy [y > 0] behind a ReLU,
//
//   dx = G W   (times [x > 0] where x is a ReLU's output),   dW = G^T x,   db = sum_r G
//
// 16-bit types: two products of 2 rows n k flop on the tiles of zo_gemm_tiles.hip.h, every operand as it lies (the contraction over G's
// columns has W with k outside, the one over the rows both).  Where there are few tiles a product's contraction is cut into shares whose
// fp32 sums a last launch adds up.  G is dy itself where that is 16-bit and its rows are whole slabs, else a copy made on the way of the pass
// that sums its columns: an fp32 dy is rounded to 16 bits there, because that is what the matrix instructions take (half a step an
// element; db sums the fp32 numbers).  fp32 parameters: everything in fp64, one launch.
#include "zo_gemm_products.hip.h"

namespace zo {

namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ the pass over dy
// G's rows and the sums of its columns, eight columns a thread, LANES threads to a row; the workgroup's 256 / LANES groups of them take every so
// many-th row of the workgroup's share.  WIDE: dy is fp32.  g [rows, width] may be null (dy is G already); so may db and part.  One share: db at
// once; more: part[share][n], for the launch that adds up shares.  LANES 64: whole lines of a row.  4: 64 rows at a time, for up to
// kNarrowRows rows in one share, where no product has shares to add up either and that launch, 4 us, is saved.  us of the whole call, wide / narrow: 300 x
// 2048 x 2048 23.8 / 21.1, 1048 x 2048 x 8192 81.0 / 79.4, 2000 x 768 x 2304 34.0 / 38.4, 2000 x 5120 x 5120 199.7 / 202.0.
template <int DT, bool WIDE, bool RELU, int LANES>
__global__ __launch_bounds__(256) void grad_rows_kernel(const void *__restrict__ dy, const uint16_t *__restrict__ y, uint4 *__restrict__ g,
                                                        float *__restrict__ part, uint16_t *__restrict__ db, int rows, int n, int width, int each)
{
    constexpr int AHEAD = 4;
    constexpr int GROUPS = 256 / LANES;
    __shared__ float sums[GROUPS][LANES][8];
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const int c = ((int)blockIdx.x * LANES + lane) * 8;
    const int first = (int)blockIdx.y * each, last = first + each < rows ? first + each : rows;
    const bool live = c < n;
    float sum[8] = {};
    for (int r0 = first + group; r0 < last; r0 += GROUPS * AHEAD) {
        float4 wide[AHEAD][2];
        uint4 in[AHEAD], kept[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int r = r0 + GROUPS * i;
            const bool on = live && r < last;
            const size_t at = (size_t)(on ? r : first) * n + (live ? c : 0);
            if constexpr (WIDE) {
                const float4 *p = (const float4 *)((const float *)dy + at);
                wide[i][0] = on ? p[0] : float4{0, 0, 0, 0};
                wide[i][1] = on ? p[1] : float4{0, 0, 0, 0};
            } else {
                in[i] = on ? *(const uint4 *)((const uint16_t *)dy + at) : uint4{0, 0, 0, 0};
            }
            if constexpr (RELU) kept[i] = on ? *(const uint4 *)(y + at) : uint4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int r = r0 + GROUPS * i;
            if (r >= last) break;
            uint32_t out[4];
            float v[8];
            if constexpr (WIDE) {
                const float w[8] = {wide[i][0].x, wide[i][0].y, wide[i][0].z, wide[i][0].w, wide[i][1].x, wide[i][1].y, wide[i][1].z, wide[i][1].w};
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = w[e];
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = pack2<DT>(w[2 * e], w[2 * e + 1]);
            } else {
                const uint32_t w[4] = {in[i].x, in[i].y, in[i].z, in[i].w}, k[4] = {kept[i].x, kept[i].y, kept[i].z, kept[i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    out[e] = RELU ? above_zero<DT>(k[e], w[e]) : w[e];
                    v[2 * e] = Prec<DT>::a2acc((uint16_t)(out[e] & 0xffff));
                    v[2 * e + 1] = Prec<DT>::a2acc((uint16_t)(out[e] >> 16));
                }
            }
            if (g && c < width) g[((size_t)r * width + c) / 8] = uint4{out[0], out[1], out[2], out[3]};
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[e];
        }
    }
    if (!db && !part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[group][lane][e] = sum[e];
    __syncthreads();
    for (int i = threadIdx.x; i < 8 * LANES; i += 256) {
        const int col = (int)blockIdx.x * LANES * 8 + i;
        if (col >= n) continue;
        float s = 0.0f;
#pragma unroll 8
        for (int w = 0; w < GROUPS; ++w) s += sums[w][i / 8][i % 8];
        if (part) part[(size_t)blockIdx.y * n + col] = s;
        else db[col] = Prec<DT>::acc2a(s);
    }
}
constexpr int kNarrowRows = 1024;

// ------------------------------------------------------------------ sums of shares
// out = rn(sum_z part[z]), eight elements a thread, zeros where `keep` is not above zero (if there is one); the workgroup's `groups` groups of
// threads take every groups-th share each and their sums meet in LDS.  Up to three results a launch.
struct SharesJob { const float4 *part; uint4 *out; const uint4 *keep; size_t n8; int shares, groups, blocks; };
struct SharesJobs { SharesJob job[3]; };
template <int DT>
__global__ __launch_bounds__(256) void shares_sum_kernel(SharesJobs jobs)
{
    __shared__ float4 sums[256][2];
    int block = (int)blockIdx.x, j = 0;
    while (j < 2 && block >= jobs.job[j].blocks) block -= jobs.job[j++].blocks;
    const SharesJob job = jobs.job[j];
    const int per = 256 / job.groups, group = threadIdx.x / per, t = threadIdx.x % per;
    for (size_t i0 = (size_t)block * per; i0 < job.n8; i0 += (size_t)job.blocks * per) {
        const size_t i = i0 + t < job.n8 ? i0 + t : job.n8 - 1;
        float4 a{0, 0, 0, 0}, b{0, 0, 0, 0};
        auto add = [&](const float4 &p, const float4 &q) {
            a = float4{a.x + p.x, a.y + p.y, a.z + p.z, a.w + p.w};
            b = float4{b.x + q.x, b.y + q.y, b.z + q.z, b.w + q.w};
        };
#pragma unroll 4
        for (int z = group; z < job.shares; z += job.groups) add(job.part[2 * (z * job.n8 + i)], job.part[2 * (z * job.n8 + i) + 1]);
        if (job.groups > 1) {
            __syncthreads();
            sums[threadIdx.x][0] = a;
            sums[threadIdx.x][1] = b;
            __syncthreads();
            if (group == 0)
                for (int g = 1; g < job.groups; ++g) add(sums[g * per + t][0], sums[g * per + t][1]);
        }
        if (group != 0 || i0 + t >= job.n8) continue;
        uint4 o{pack2<DT>(a.x, a.y), pack2<DT>(a.z, a.w), pack2<DT>(b.x, b.y), pack2<DT>(b.z, b.w)};
        if (job.keep) {
            const uint4 k = job.keep[i];
            o = uint4{above_zero<DT>(k.x, o.x), above_zero<DT>(k.y, o.y), above_zero<DT>(k.z, o.z), above_zero<DT>(k.w, o.w)};
        }
        job.out[i] = o;
    }
}

// ------------------------------------------------------------------ both products in one launch
// Where neither product fills the chip for long: dW's tiles on some CUs (workgroups 0 .. blocks_w - 1, persistent, one a CU), dx's on the others, tiles of
// one shape.  What bounds such a call is not the multiplies but rounds of tiles that leave CUs empty, each launch's first loads and last stores, and the
// sums of shares that a product needs to fill the chip by itself.  us of the whole call, bf16, two launches / one: 8192 x 768 x 768 45.7 / 39.5, 8192 x
// 2304 x 768 75.0 / 68.7, 2000 x 2304 x 768 37.1 / 26.6, 2000 x 768 x 768 25.3 / 18.6, 1500 x 1536 x 1536 35.5 / 28.9, 4096 x 4096 x 1024 80.4 / 69.3,
// 8192 x 4096 x 1024 173 / 158, 32768 x 512 x 512 75.8 / 70.6, 400 x 1024 x 4096 19.9 / 15.8, 300 x 512 x 512 14.6 / 11.3; of 34 sizes the worst pick is 4096 x 2048 x 2048, 78.9 / 80.1.
struct PairTiles { const uint16_t *x, *w; void *y; int m, n, k, tiles_m, tiles_n, total; };
template <int DT, int EPIW, int EPIX, class SH>
__global__ __launch_bounds__(256) void linear_pair_kernel(PairTiles dw, PairTiles dx, ByRows::Arg op_w, ByWords::Arg op_x, int blocks_w)
{
    const int block = (int)blockIdx.x;
    if (block < blocks_w)
        pipe_tiles<DT, EPIW, SH, ByRows>(dw.x, dw.w, nullptr, nullptr, nullptr, dw.y, dw.m, dw.n, dw.k, dw.tiles_m, dw.tiles_n, dw.total, op_w, block, blocks_w);
    else
        pipe_tiles<DT, EPIX, SH, ByWords>(dx.x, dx.w, nullptr, nullptr, nullptr, dx.y, dx.m, dx.n, dx.k, dx.tiles_m, dx.tiles_n, dx.total, op_x, block - blocks_w,
                                          (int)gridDim.x - blocks_w);
}
template <int DT, int EPIW, int EPIX, class SH> hipError_t launch_pair_of(const Args &dw, const ByRows::Arg &op_w, const Args &dx, const ByWords::Arg &op_x, int blocks_w, int blocks_x)
{
    auto tiles = [](const Args &a) {
        const int tm = (a.m_half + SH::BM - 1) / SH::BM, tn = (a.n + SH::BN - 1) / SH::BN;
        return PairTiles{(const uint16_t *)a.x, (const uint16_t *)a.wt_p, a.y, a.m_half, a.n, a.k, tm, tn, a.n_sign * tm * tn};
    };
    if (cu_count() == 0 || dw.k / BK <= SH::A || dx.k / BK <= SH::A) return hipErrorInvalidValue;
    auto kern = linear_pair_kernel<DT, EPIW, EPIX, SH>;
    static std::atomic<uint64_t> lds_allowed{0};
    const hipError_t e = once_per_device(lds_allowed, [&] { return hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, SH::kLdsBytes); });
    if (e != hipSuccess) return e;
    kern<<<dim3(blocks_w + blocks_x), dim3(256), SH::kLdsBytes, dw.s>>>(tiles(dw), tiles(dx), op_w, op_x, blocks_w);
    return hipGetLastError();
}
template <int DT, int EPIW, int EPIX> hipError_t launch_pair(Tile t, const Args &dw, const ByRows::Arg &op_w, const Args &dx, const ByWords::Arg &op_x, int blocks_w, int blocks_x)
{
    return t == T256x256   ? launch_pair_of<DT, EPIW, EPIX, Shape<4, 4, 2>>(dw, op_w, dx, op_x, blocks_w, blocks_x)
           : t == T256x128 ? launch_pair_of<DT, EPIW, EPIX, Shape<4, 2, 2>>(dw, op_w, dx, op_x, blocks_w, blocks_x)
                           : launch_pair_of<DT, EPIW, EPIX, Shape<2, 2, 4>>(dw, op_w, dx, op_x, blocks_w, blocks_x);
}

// ------------------------------------------------------------------ the plan of a call
struct LinearPlan {
    int width;                              // of G's copy; 0: dy is G
    int x_shares, x_share;                  // shares of dx's contraction over n, and the columns of one
    int w_shares, w_share;                  // of dW's over the rows
    int sum_shares, sum_each;               // of the column sums, and the rows of one
    bool narrow;                            // one share, by narrow workgroups
    int pair_w, pair_x;                     // workgroups of dW and of dx where one launch has both; 0: launches of their own
    Tile pair_tile;
    Tile x_tile, w_tile;
    Words w_rows;                           // dW's rows, where its sum has one share: what whole rounds of a tile hold and the rest
    bool both, fits;                        // one launch for both products; every launch's tiles fit one
    size_t g, x_part, w_part, sums, total;
};
constexpr float kPairMost = 250.0f, kPairGain = 0.95f;         // (longer calls have many rounds: nothing to gain; estimates nearer than that are a toss-up)
constexpr int kSumBlocks = 1024;            // workgroups of the pass over dy, about: four to a CU
// One launch of both products, dx in one share: the tile, dW's shares and the CUs of each of least estimated time, if that is below `limit`.  By the
// costs of launches of their own, with what the faster clock of a chip that is not full saves counted for both together.
void pick_pair(LinearPlan &p, int rows, int n, int k, int n_slabs, int r_slabs, float limit)
{
    const int n_cu = cu_count() ? cu_count() : 256;
    for (Tile t : {T256x256, T256x128, T128x128}) {
        if (n_slabs < kLeastSlabs[t]) continue;
        auto tiles = [&](int m) { return (m + kTileRows[t] - 1) / kTileRows[t] * ((k + kTileColumns[t] - 1) / kTileColumns[t]); };
        const auto &cx = kProductCost[kByWords][t], &cw = kProductCost[kByRows][t];
        const int tx = tiles(rows), sx = n_slabs;
        const float x_mb = (float)(rows + k) * (float)sx * (BK * 2e-6f) * cx.operand + (float)rows * (float)k * 4e-6f * cx.output;
        for (int z = 1; z <= 64 && z <= r_slabs; z += z < 8 ? 1 : z < 16 ? 2 : 4) {
            const int sw = (r_slabs + z - 1) / z, tw = z * tiles(n);
            if (sw < kLeastSlabs[t]) break;
            const float w_mb = (float)(n + k) * (float)(sw * z) * (BK * 2e-6f) * cw.operand + (float)n * (float)k * (float)z * 2e-6f * cw.output;
            const float fixed = (cx.start > cw.start ? cx.start : cw.start) + x_mb + w_mb + (z > 1 ? shares_us(z, n, k) : 0.0f);
            const float work_w = (float)tw * (float)sw, work_x = (float)tx * (float)sx, part = work_w / (work_w + work_x);
            for (int i = -1; i < 3; ++i) {
                const int bw = ((int)(part * (float)n_cu) / 8 + i) * 8, bx = n_cu - bw;
                if (bw < 8 || bx < 8) continue;
                const float rw = (float)(((tw + 7) / 8 + bw / 8 - 1) / (bw / 8)), rx = (float)(((tx + 7) / 8 + bx / 8 - 1) / (bx / 8));
                // (how busy the chip is while the longer one lasts)
                const float longest = rw * (float)sw > rx * (float)sx ? rw * (float)sw : rx * (float)sx, full = (work_w + work_x) / ((float)n_cu * longest);
                const float busy = full > 0.5f ? 2 * full - 1 : 0.0f;
                const float uw = rw * ((float)sw * (cw.slab + busy * cw.busy) + cw.round), ux = rx * ((float)sx * (cx.slab + busy * cx.busy) + cx.round);
                const float us = fixed + (uw > ux ? uw : ux);
                if (us >= limit) continue;
                limit = us;
                p.pair_w = bw; p.pair_x = bx;
                p.pair_tile = t;
                p.x_shares = 1; p.w_shares = z;
            }
        }
    }
    if (!p.pair_w) return;
    p.x_tile = pick_product(kByWords, 1, rows, k, n_slabs);         // (for calls that want one of the two)
    p.w_tile = pick_product(kByRows, p.w_shares, n, k, (r_slabs + p.w_shares - 1) / p.w_shares);
}
LinearPlan work_out(int rows, int n, int k, int epilogue)
{
    LinearPlan p{};
    const bool copy = epilogue != 0 || n % BK != 0;
    const int n_slabs = (n + BK - 1) / BK, r_slabs = (rows + BK - 1) / BK;
    float best = 0.0f;
    for (int z = 1; z <= 64 && z <= n_slabs; z += z < 8 ? 1 : z < 16 ? 2 : 4) {
        if (!copy && n_slabs % z) continue;                      // (a share's slabs past dy's rows would be the next rows')
        float us;
        const Tile t = pick_product(kByWords, z, rows, k, (n_slabs + z - 1) / z, &us);
        if (z > 1) us += shares_us(z, rows, k);
        if (best == 0.0f || us < best) { best = us; p.x_shares = z; p.x_tile = t; }
    }
    const float x_us = best;
    best = 0.0f;
    for (int z = 1; z <= 64 && z <= r_slabs; z += z < 8 ? 1 : z < 16 ? 2 : 4) {
        float us;
        const Tile t = pick_product(kByRows, z, n, k, (r_slabs + z - 1) / z, &us);
        if (z > 1) us += shares_us(z, n, k);
        if (best == 0.0f || us < best) { best = us; p.w_shares = z; p.w_tile = t; }
    }
    if (best + x_us < kPairMost) pick_pair(p, rows, n, k, n_slabs, r_slabs, kPairGain * (best + x_us));
    p.x_share = (n_slabs + p.x_shares - 1) / p.x_shares * BK;
    p.width = copy ? p.x_share * p.x_shares : 0;
    p.w_share = (r_slabs + p.w_shares - 1) / p.w_shares * BK;
    p.w_rows = p.w_shares == 1 && !p.pair_w ? pick_words(n, k, r_slabs) : Words{p.w_tile, n, p.w_tile};
    p.w_tile = p.w_rows.tile;
    p.both = !p.pair_w && p.x_tile == T64x64 && p.w_tile == T64x64 && p.w_rows.words == n && p.w_shares == 1 && p.x_share <= kBothSlabs * BK && r_slabs * BK <= kBothRows;
    const int64_t dx = small_blocks(p.x_tile, p.x_shares, rows, k), dw = small_blocks(p.w_tile, p.w_shares, p.w_rows.words, k);
    p.fits = dx <= kMostBlocks && dw <= kMostBlocks && (!p.both || dx + dw <= kMostBlocks);
    const int columns = ((copy ? p.width : n) + 511) / 512, most = kSumBlocks / columns > 1 ? kSumBlocks / columns : 1;
    p.sum_shares = rows <= 64 ? 1 : (rows + 15) / 16 < most ? (rows + 15) / 16 : most;
    p.sum_each = ((rows + p.sum_shares - 1) / p.sum_shares + 3) / 4 * 4;
    p.sum_shares = (rows + p.sum_each - 1) / p.sum_each;
    p.narrow = p.sum_shares > 1 && rows <= kNarrowRows && p.x_shares == 1 && p.w_shares == 1;
    if (p.narrow) { p.sum_shares = 1; p.sum_each = rows; }
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o = up(o + bytes); return at; };
    p.g = take(2 * (size_t)rows * p.width);
    p.x_part = take(p.x_shares > 1 ? 4 * (size_t)p.x_shares * rows * k : 0);
    p.w_part = take(p.w_shares > 1 ? 4 * (size_t)p.w_shares * n * k : 0);
    p.sums = take(p.sum_shares > 1 ? 4 * (size_t)p.sum_shares * n : 0);
    p.total = o > 256 ? o : 256;
    return p;
}
// A thread's plans of late, by their sizes: a program goes through the same few over and over, and to work one out takes the host up to 25 us, as long
// as the device needs for a small call.
const LinearPlan &linear_plan(int rows, int n, int k, int epilogue)
{
    struct Kept { int rows, n, k, epilogue, n_cu; LinearPlan plan; };
    static thread_local Kept kept[32];                         // (rows 0: none)
    Kept &at = kept[(((((uint32_t)rows * 31u + (uint32_t)n) * 31u + (uint32_t)k) * 31u + (uint32_t)epilogue) * 0x9e3779b1u) >> 27];
    if (at.rows != rows || at.n != n || at.k != k || at.epilogue != epilogue || at.n_cu != cu_count()) at = Kept{rows, n, k, epilogue, cu_count(), work_out(rows, n, k, epilogue)};
    return at.plan;
}

template <int DT>
hipError_t linear_grad(const uint16_t *x, const uint16_t *w, const uint16_t *y, const void *dy, uint16_t *dx, uint16_t *dw, uint16_t *db, char *ws, int rows,
                       int n, int k, int epilogue, bool relu_x, hipStream_t s)
{
    const LinearPlan &p = linear_plan(rows, n, k, epilogue);
    if (!p.fits) return hipErrorNotSupported;
    hipError_t err = hipSuccess;
    const bool copy = p.width != 0 && (dx || dw);
    float *sums = db && p.sum_shares > 1 ? (float *)(ws + p.sums) : nullptr;
    if (copy || db) {
        auto kern = [&](auto lanes) {
            constexpr int L = decltype(lanes)::value;
            return epilogue >= 2 ? grad_rows_kernel<DT, true, false, L> : epilogue == 1 ? grad_rows_kernel<DT, false, true, L> : grad_rows_kernel<DT, false, false, L>;
        };
        const int width = copy ? p.width : n, columns = p.narrow ? 32 : 512;
        (p.narrow ? kern(std::integral_constant<int, 4>{}) : kern(std::integral_constant<int, 64>{}))<<<dim3((width + columns - 1) / columns, p.sum_shares), dim3(256), 0, s>>>(dy, y, copy ? (uint4 *)(ws + p.g) : nullptr, sums, sums ? nullptr : db, rows, n,
                                                                           width, p.sum_each);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    const uint16_t *g = copy ? (const uint16_t *)(ws + p.g) : (const uint16_t *)dy;
    const int ldg = copy ? p.width : n;
    ByWords::Arg op_x{};
    op_x.ldx = ldg; op_x.ldw = k;
    op_x.xz = p.x_share; op_x.wz = (uint64_t)p.x_share * k;
    op_x.w_end = (uint64_t)(uintptr_t)(w + (size_t)n * k);
    op_x.alpha = 1.0f;
    op_x.keep = x;
    const Args a{g, w, nullptr, nullptr, nullptr, p.x_shares > 1 ? (void *)(ws + p.x_part) : dx, p.x_shares, rows, k, p.x_share, s};
    ByRows::Arg op_w{};
    op_w.ldx = ldg; op_w.ldw = k;
    op_w.xz = (uint64_t)p.w_share * ldg; op_w.wz = (uint64_t)p.w_share * k;
    op_w.x_end = (uint64_t)(uintptr_t)(g + (size_t)rows * ldg);
    op_w.w_end = (uint64_t)(uintptr_t)(x + (size_t)rows * k);
    op_w.alpha = 1.0f;
    const Args b{g, x, nullptr, nullptr, nullptr, p.w_shares > 1 ? (void *)(ws + p.w_part) : dw, p.w_shares, p.w_rows.words, k, p.w_share, s};
    if (dx && dw && p.pair_w) {
        auto pair = [&](auto epi_w, auto epi_x) { return launch_pair<DT, decltype(epi_w)::value, decltype(epi_x)::value>(p.pair_tile, b, op_w, a, op_x, p.pair_w, p.pair_x); };
        auto with = [&](auto epi_w) { return relu_x ? pair(epi_w, std::integral_constant<int, 10>{}) : pair(epi_w, std::integral_constant<int, 6>{}); };
        err = p.w_shares > 1 ? with(std::integral_constant<int, 7>{}) : with(std::integral_constant<int, 6>{});
        if (err != hipSuccess) return err;
    } else if (dx && dw && p.both) {
        err = p.x_shares > 1 ? launch_both<DT>(a, op_x, b, op_w) : relu_x ? launch_both<DT, 10>(a, op_x, b, op_w) : launch_both<DT, 6>(a, op_x, b, op_w);
        if (err != hipSuccess) return err;
    } else {
        // (dW first: what it reads of x is near when dx's results are held against it)
        if (dw) {
            err = p.w_shares > 1 ? launch_product<DT, 7, ByRows>(p.w_tile, b, op_w) : launch_product<DT, 6, ByRows>(p.w_tile, b, op_w);
            if (err != hipSuccess) return err;
            if (p.w_rows.words < n) {
                const Args rest{g + p.w_rows.words, x, nullptr, nullptr, nullptr, dw + (size_t)p.w_rows.words * k, 1, n - p.w_rows.words, k, p.w_share, s};
                if ((err = launch_product<DT, 6, ByRows>(p.w_rows.rest, rest, op_w)) != hipSuccess) return err;
            }
        }
        if (dx) {
            err = p.x_shares > 1 ? launch_product<DT, 7, ByWords>(p.x_tile, a, op_x) : relu_x ? launch_product<DT, 10, ByWords>(p.x_tile, a, op_x)
                                                                                             : launch_product<DT, 6, ByWords>(p.x_tile, a, op_x);
            if (err != hipSuccess) return err;
        }
    }
    SharesJobs jobs{};
    int count = 0, blocks = 0;
    auto add = [&](const void *part, int shares, size_t elements, uint16_t *out, const uint16_t *keep) {
        SharesJob &j = jobs.job[count++];
        j.part = (const float4 *)part; j.out = (uint4 *)out; j.keep = (const uint4 *)keep;
        j.n8 = elements / 8;
        j.shares = shares;
        // groups of threads: enough for every CU to have a workgroup, as long as each has two shares
        j.groups = 1;
        while (j.groups < 32 && 4 * j.groups <= shares && j.n8 * j.groups < 256 * 512) j.groups *= 2;
        const size_t need = (j.n8 * j.groups + 255) / 256;
        j.blocks = (int)(need < 4096 ? need : 4096);
        blocks += j.blocks;
    };
    if (dx && p.x_shares > 1) add(ws + p.x_part, p.x_shares, (size_t)rows * k, dx, relu_x ? x : nullptr);
    if (dw && p.w_shares > 1) add(ws + p.w_part, p.w_shares, (size_t)n * k, dw, nullptr);
    if (sums) add(sums, p.sum_shares, n, db, nullptr);
    if (!blocks) return hipSuccess;
    shares_sum_kernel<DT><<<dim3(blocks), dim3(256), 0, s>>>(jobs);
    return hipGetLastError();
}

// ------------------------------------------------------------------ fp64
// All three results in one launch: the first x_tiles workgroups have tiles of dx, the next w_tiles of dW, the others 64 columns of db each.  A
// workgroup owns 16 TB x 16 TB outputs, its W wavefronts take every W-th 16-deep piece of the contraction straight from memory into
// v_mfma_f64_16x16x4 operands, and the partial sums meet in LDS, in a fixed order.
template <int TB, int W>
__global__ __launch_bounds__(64 * W) void linear_grad_f64_kernel(const double *__restrict__ x, const float *__restrict__ w, const double *__restrict__ y,
                                                                 const double *__restrict__ dy, double *__restrict__ dx, float *__restrict__ dw, float *__restrict__ db,
                                                                 int rows, int n, int k, bool relu_x, int x_tiles, int w_tiles)
{
    constexpr int BT = 16 * TB;
    __shared__ double part[W][BT][BT + 1];
    const int block = (int)blockIdx.x;
    auto grad = [&](int r, int c) {
        const size_t at = (size_t)r * n + c;
        return y && !(y[at] > 0.0) ? 0.0 : dy[at];
    };
    if (block >= x_tiles + w_tiles) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (block - x_tiles - w_tiles) * 64 + lane;
        double s = 0.0;
        if (c < n)
            for (int r = wave; r < rows; r += W) s += grad(r, c);
        double *sums = &part[0][0][0];
        sums[threadIdx.x] = s;
        __syncthreads();
        if (wave == 0 && c < n) {
#pragma unroll
            for (int v = 1; v < W; ++v) s += sums[64 * v + lane];
            db[c] = (float)s;
        }
        return;
    }
    const bool of_x = block < x_tiles;
    const int tile = of_x ? block : block - x_tiles;
    const int tiles_k = (k + BT - 1) / BT, i0 = tile / tiles_k * BT, j0 = tile % tiles_k * BT;
    const int m = of_x ? rows : n, depth = of_x ? n : rows;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
    f64x4 acc[TB][TB] = {};
#pragma unroll 2
    for (int k0 = 16 * wave; k0 < depth; k0 += 16 * W) {
        f64x4 av[TB], bv[TB];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int kk = k0 + 4 * g + q, kc = kk < depth ? kk : depth - 1;
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const int i = i0 + 16 * t + r16 < m ? i0 + 16 * t + r16 : m - 1, j = j0 + 16 * t + r16 < k ? j0 + 16 * t + r16 : k - 1;   // clamped: never stored
                const double a = of_x ? grad(i, kc) : grad(kc, i);
                const double b = of_x ? (double)w[(size_t)kc * k + j] : x[(size_t)kc * k + j];
                av[t][q] = kk < depth ? a : 0.0;
                bv[t][q] = kk < depth ? b : 0.0;
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < TB; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f64_16x16x4f64(av[i][q], bv[j][q], acc[i][j], 0, 0, 0);
    }
    // element e of a lane's result: row 4 e + lane / 16, column lane % 16 of the 16 x 16 block
#pragma unroll
    for (int i = 0; i < TB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) part[wave][16 * i + 4 * q + g][16 * j + r16] = acc[i][j][q];
    __syncthreads();
    for (int o = threadIdx.x; o < BT * BT; o += 64 * W) {
        const int i = i0 + o / BT, j = j0 + o % BT;
        if (i >= m || j >= k) continue;
        double v = 0.0;
#pragma unroll
        for (int z = 0; z < W; ++z) v += part[z][o / BT][o % BT];
        const size_t at = (size_t)i * k + j;
        if (of_x) dx[at] = relu_x && !(x[at] > 0.0) ? 0.0 : v;
        else dw[at] = (float)v;
    }
}

long f64_blocks(int rows, int n, int k, int bt)
{
    const long tiles_k = (k + bt - 1) / bt;
    return ((rows + bt - 1) / bt + (n + bt - 1) / bt) * tiles_k + (n + 63) / 64;
}
// 32 x 32 outputs a workgroup where these are enough for every CU
bool f64_many(int rows, int n, int k) { return f64_blocks(rows, n, k, 32) >= 512; }

hipError_t linear_grad_f64(const double *x, const float *w, const double *y, const double *dy, double *dx, float *dw, float *db, int rows, int n, int k,
                           bool relu_x, hipStream_t s)
{
    auto go = [&](auto kern, int bt, int waves) {
        const int tiles_k = (k + bt - 1) / bt, x_tiles = dx ? (rows + bt - 1) / bt * tiles_k : 0, w_tiles = dw ? (n + bt - 1) / bt * tiles_k : 0;
        kern<<<dim3(x_tiles + w_tiles + (db ? (n + 63) / 64 : 0)), dim3(64 * waves), 0, s>>>(x, w, y, dy, dx, dw, db, rows, n, k, relu_x, x_tiles, w_tiles);
        return hipGetLastError();
    };
    return f64_many(rows, n, k) ? go(linear_grad_f64_kernel<2, 4>, 32, 4) : go(linear_grad_f64_kernel<1, 8>, 16, 8);
}

}  // namespace

size_t linear_grad_scratch(int dtype, int rows, int n, int k, int epilogue)
{
    if (dtype == kFP32) return f64_blocks(rows, n, k, 32) < 1l << 24 ? 256 : 0;
    const LinearPlan &p = linear_plan(rows, n, k, epilogue);
    return p.fits ? p.total : 0;
}

bool linear_grad_plan(int rows, int n, int k, int epilogue, int32_t *plan)
{
    const LinearPlan &p = linear_plan(rows, n, k, epilogue);
    if (!p.fits) return false;
    auto tile = [](Tile t) { return kTileRows[t] << 16 | kTileColumns[t]; };
    plan[0] = tile(p.x_tile);
    plan[1] = tile(p.w_tile);
    plan[2] = p.x_shares;
    plan[3] = p.w_shares;
    plan[4] = p.width;
    plan[5] = p.sum_shares;
    plan[6] = p.w_rows.words;
    plan[7] = tile(p.w_rows.rest);
    plan[8] = p.pair_w ? tile(p.pair_tile) : p.both ? tile(T64x64) : 0;
    plan[9] = p.pair_w ? p.pair_w : p.both ? (int32_t)small_blocks(T64x64, 1, n, k) : 0;
    return true;
}

hipError_t launch_linear_grad(const void *x, const void *w, const void *y, const void *dy, void *dx, void *dw, void *db, void *scratch, int dtype, int rows,
                              int n, int k, int epilogue, bool relu_x, hipStream_t s)
{
    if (epilogue != 1) y = nullptr;
    if (dtype == kFP32) {
        if (f64_blocks(rows, n, k, 32) >= 1l << 24) return hipErrorNotSupported;
        return linear_grad_f64((const double *)x, (const float *)w, (const double *)y, (const double *)dy, (double *)dx, (float *)dw, (float *)db, rows, n, k,
                               relu_x, s);
    }
    auto f = dtype == kBF16 ? linear_grad<kBF16> : linear_grad<kFP16>;
    return f((const uint16_t *)x, (const uint16_t *)w, (const uint16_t *)y, dy, (uint16_t *)dx, (uint16_t *)dw, (uint16_t *)db, (char *)scratch, rows, n, k,
             epilogue, relu_x, s);
}

}  // namespace zo
