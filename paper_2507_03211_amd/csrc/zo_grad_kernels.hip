// Gradient of the model's last module: LayerNorm forward with its statistics and its backward pass, the elementwise parts of
// the LM head's cross-entropy gradient with the fp64 products of fp32 parameters, and the global norm and clipping of a
// model's gradients.  (DistZO2 trains by the two losses of Eq. 1 alone; the last module is the one whose exact gradient
// needs no other module's, and z . grad L is what Eq. 2's g estimates.)
#include "zo_kernels.h"
#include "zo_types.hip.h"

namespace zo {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

#define ZO_DISPATCH_DT(dtype, CALL)                  \
    switch (dtype) {                                 \
    case kFP32: { constexpr int DT = kFP32; CALL; } break; \
    case kBF16: { constexpr int DT = kBF16; CALL; } break; \
    case kFP16: { constexpr int DT = kFP16; CALL; } break; \
    default: return hipErrorInvalidValue;            \
    }

// ------------------------------------------------------------------ LayerNorm backward
// With xh = (h - mean) rstd and a = dy g:   dh = rstd (a - mean_c(a) - xh mean_c(a xh)),
//                                           dg = sum_r dy xh,  db = sum_r dy.
// One pass over dy and h: a workgroup takes every gridDim-th row (or group of four), works dh row by row and adds up its rows' share
// of dg and db, which it leaves in part[workgroup][2][d]; layernorm_dweight_kernel adds the workgroups' shares in order.  Bound by memory:
// 10 bytes an element of 16-bit types.

// Rows of any length and type: one workgroup a row, its share of the weights' gradient added up in `part` itself (each thread its own columns).
template <int DT>
__global__ __launch_bounds__(256) void layernorm_grad_kernel(const void *dy_, const void *resid, const void *gain, const void *mean_, const void *rstd_,
                                                             void *dresid, void *part_, int rows, int d, bool accumulate, bool weights)
{
    using P = Prec<DT>;
    using Acc = typename P::Acc;
    __shared__ Acc red[16];
    const typename P::W *g = (const typename P::W *)gain;
    Acc *part = (Acc *)part_ + (size_t)blockIdx.x * 2 * d;
    for (int row = blockIdx.x; row < rows; row += gridDim.x) {
        const typename P::A *dy = (const typename P::A *)dy_ + (size_t)row * d;
        const typename P::R *h = (const typename P::R *)resid + (size_t)row * d;
        const Acc mean = ((const Acc *)mean_)[row], rstd = ((const Acc *)rstd_)[row];
        Acc sa = 0, sx = 0;
        for (int c = threadIdx.x; c < d; c += blockDim.x) {
            const Acc v = P::a2acc(dy[c]), xh = ((Acc)h[c] - mean) * rstd;
            if (dresid) {
                const Acc a = v * (Acc)P::w2f(g[c]);
                sa += a;
                sx += a * xh;
            }
            if (weights) {
                const bool first = row == (int)blockIdx.x;
                part[c] = first ? v * xh : part[c] + v * xh;
                part[d + c] = first ? v : part[d + c] + v;
            }
        }
        if (!dresid) continue;
        sa = block_sum(sa, red) / (Acc)d;
        sx = block_sum(sx, red) / (Acc)d;
        typename P::R *out = (typename P::R *)dresid + (size_t)row * d;
        for (int c = threadIdx.x; c < d; c += blockDim.x) {
            const Acc a = P::a2acc(dy[c]) * (Acc)P::w2f(g[c]), xh = ((Acc)h[c] - mean) * rstd;
            const Acc v = rstd * (a - sa - xh * sx);
            out[c] = (typename P::R)(accumulate ? out[c] + v : v);
        }
    }
}

__device__ __forceinline__ float fused(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
__device__ __forceinline__ double fused(double a, double b, double c) { return __builtin_fma(a, b, c); }

// Rows in registers: NV pieces of VW elements a lane, WPR wavefronts a row (one: four rows at a time).  VW = 4 where rows of 16-bit types
// are a multiple of four elements long and buffers aligned, else 1.  The next row is on its way while one is worked; gain and the weights'
// sums stay in registers throughout.  One workgroup a CU is enough: us with 256 / 512 of them, bf16, launch of the sums below included,
// 8192 rows of 768 19.3 / 19.3, of 1536 30.0 / 31.9, 4096 60.8 / 69, 5120 79.2 / 86 (floor 81.9 at the copy rate, which leaves the
// memory-side cache out), 12288 195 / 204; 2048 is the exception, 39.5 / 37.6.  Wavefronts a row, the best number of pieces of each: 1536
// columns 30.0 (1) / 32.6 (2) / 32.4 (4), 2048 37.6 / 37.1 / 37.6, where 8 pieces and one wavefront take 314 registers, and 1003 rows
// 12.0 / 11.8 / 11.4; 5120 79.2 (4) / 84.8 (8).  Element by element, 4096 rows of 1101 25 us, of 2603 39.8, of 4802 52.6 (46 - 102 - 178 with
// the kernel for any length).
template <int DT, int NV, int WPR, int VW>
__global__ __launch_bounds__(WPR == 1 ? 256 : 64 * WPR) void layernorm_grad_rows_kernel(
    const typename Prec<DT>::A *__restrict__ dy, const typename Prec<DT>::R *__restrict__ resid, const typename Prec<DT>::W *__restrict__ gain,
    const typename Prec<DT>::Acc *__restrict__ mean_, const typename Prec<DT>::Acc *__restrict__ rstd_, typename Prec<DT>::R *__restrict__ dresid,
    typename Prec<DT>::Acc *__restrict__ part, int rows, int d, bool accumulate, bool weights)
{
    using P = Prec<DT>;
    using Acc = typename P::Acc;                                // the residual stream's type too
    static_assert(std::is_same_v<Acc, typename P::R>, "");
    typedef typename P::A act_t __attribute__((ext_vector_type(VW)));
    typedef typename P::W gain_t __attribute__((ext_vector_type(VW)));
    typedef Acc acc_t __attribute__((ext_vector_type(VW)));
    struct Pair { Acc a, x; };
    constexpr int LANES = 64 * WPR, RPB = WPR == 1 ? 4 : 1;     // lanes a row, rows at a time
    __shared__ Pair sums[2][WPR];
    extern __shared__ __attribute__((aligned(16))) char shared_raw[];   // WPR == 1: [2][d], the four wavefronts' sums
    const int tid = threadIdx.x, lane = tid % LANES, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nvec = d / VW, step = (int)gridDim.x * RPB;
    const Acc inv_d = (Acc)1 / (Acc)d;
    auto inside = [&](int i) { return lane + LANES * i < nvec; };
    auto col = [&](int i) { return inside(i) ? lane + LANES * i : nvec - 1; };
    gain_t gv[NV];
    acc_t dg[NV] = {}, db[NV] = {};
    if (dresid) {
#pragma unroll
        for (int i = 0; i < NV; ++i) gv[i] = ((const gain_t *)gain)[col(i)];
    }
    struct Row { acc_t h[NV]; act_t dy[NV]; Acc mean, rstd; };
    auto load = [&](int row, Row &r) {
#pragma unroll
        for (int i = 0; i < NV; ++i) r.dy[i] = ((const act_t *)(dy + (size_t)row * d))[col(i)];
#pragma unroll
        for (int i = 0; i < NV; ++i) r.h[i] = ((const acc_t *)(resid + (size_t)row * d))[col(i)];
        r.mean = mean_[row];
        r.rstd = rstd_[row];
    };
    int row = (int)blockIdx.x * RPB + (WPR == 1 ? wave : 0);
    Row cur, nxt;
    if (row < rows) load(row, cur);
    for (int turn = 0; row < rows; row += step, turn ^= 1) {
        const int next = row + step;
        if (next < rows) load(next, nxt);
        Acc sa = 0, sx = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int e = 0; e < VW; ++e) {
                const Acc v = inside(i) ? P::a2acc(cur.dy[i][e]) : (Acc)0;
                const Acc xh = (cur.h[i][e] - cur.mean) * cur.rstd, a = v * (Acc)P::w2f(gv[i][e]);
                sa += a;
                sx = fused(a, xh, sx);
                dg[i][e] = fused(v, xh, dg[i][e]);
                db[i][e] += v;
            }
        }
        if (dresid) {
            sa = wave_sum(sa);
            sx = wave_sum(sx);
            if constexpr (WPR > 1) {                            // two sets of slots: a wavefront may be a row ahead of its neighbours
                if ((tid & 63) == 0) sums[turn][wave] = Pair{sa, sx};
                __syncthreads();
                sa = sx = 0;
#pragma unroll
                for (int w = 0; w < WPR; ++w) { sa += sums[turn][w].a; sx += sums[turn][w].x; }
            }
            sa *= inv_d;
            sx *= inv_d;
            acc_t *out = (acc_t *)(dresid + (size_t)row * d);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                acc_t o;
#pragma unroll
                for (int e = 0; e < VW; ++e)
                    o[e] = cur.rstd * (fused(P::a2acc(cur.dy[i][e]), (Acc)P::w2f(gv[i][e]), -sa) - (cur.h[i][e] - cur.mean) * cur.rstd * sx);
                if (inside(i)) {
                    acc_t *at = out + lane + LANES * i;
                    if (accumulate) {
                        const acc_t before = *at;
#pragma unroll
                        for (int e = 0; e < VW; ++e) o[e] += before[e];
                    }
                    *at = o;
                }
            }
        }
        cur = nxt;
    }
    if (!weights) return;
    part += (size_t)blockIdx.x * 2 * d;
    acc_t *pg = (acc_t *)part, *pb = (acc_t *)(part + d);
    if constexpr (WPR > 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (inside(i)) { pg[lane + LANES * i] = dg[i]; pb[lane + LANES * i] = db[i]; }
    } else {
        // the wavefronts add theirs one after the other, the last one writes
        acc_t *sg = (acc_t *)shared_raw, *sb = (acc_t *)((Acc *)shared_raw + d);
        for (int w = 0; w < 4; ++w) {
            if (wave == w) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if (!inside(i)) continue;
                    const int c = lane + LANES * i;
                    acc_t a = dg[i], b = db[i];
                    if (w > 0) {
#pragma unroll
                        for (int e = 0; e < VW; ++e) { a[e] += sg[c][e]; b[e] += sb[c][e]; }
                    }
                    (w < 3 ? sg : pg)[c] = a;
                    (w < 3 ? sb : pb)[c] = b;
                }
            }
            __syncthreads();
        }
    }
}

// Few rows, of any length and type, in one launch: the first `rows` workgroups work a row's dh each, the others 32 columns of dg and db
// each, eight rows at a time.  dy and h are read twice, which is nothing next to a second launch.
template <int DT>
__global__ __launch_bounds__(256) void layernorm_grad_few_kernel(const void *dy_, const void *resid, const void *gain, const void *mean_, const void *rstd_,
                                                                 void *dresid, void *dgain, void *dbias, int rows, int d, bool accumulate, int row_blocks)
{
    using P = Prec<DT>;
    using Acc = typename P::Acc;
    __shared__ Acc red[16];
    __shared__ Acc cols[2][8][32];
    if ((int)blockIdx.x < row_blocks) {
        const size_t row = blockIdx.x;
        const typename P::A *dy = (const typename P::A *)dy_ + row * d;
        const typename P::R *h = (const typename P::R *)resid + row * d;
        const typename P::W *g = (const typename P::W *)gain;
        const Acc mean = ((const Acc *)mean_)[row], rstd = ((const Acc *)rstd_)[row];
        Acc sa = 0, sx = 0;
#pragma unroll 4
        for (int c = threadIdx.x; c < d; c += 256) {
            const Acc a = P::a2acc(dy[c]) * (Acc)P::w2f(g[c]);
            sa += a;
            sx += a * (((Acc)h[c] - mean) * rstd);
        }
        sa = block_sum(sa, red) / (Acc)d;
        sx = block_sum(sx, red) / (Acc)d;
        typename P::R *out = (typename P::R *)dresid + row * d;
#pragma unroll 4
        for (int c = threadIdx.x; c < d; c += 256) {
            const Acc a = P::a2acc(dy[c]) * (Acc)P::w2f(g[c]), xh = ((Acc)h[c] - mean) * rstd;
            const Acc v = rstd * (a - sa - xh * sx);
            out[c] = (typename P::R)(accumulate ? out[c] + v : v);
        }
        return;
    }
    const int lane = threadIdx.x & 31, sub = threadIdx.x >> 5, c = ((int)blockIdx.x - row_blocks) * 32 + lane;
    Acc dg = 0, db = 0;
    if (c < d) {
#pragma unroll 4
        for (int r = sub; r < rows; r += 8) {
            const Acc v = P::a2acc(((const typename P::A *)dy_)[(size_t)r * d + c]);
            const Acc xh = ((Acc)((const typename P::R *)resid)[(size_t)r * d + c] - ((const Acc *)mean_)[r]) * ((const Acc *)rstd_)[r];
            dg += v * xh;
            db += v;
        }
    }
    cols[0][sub][lane] = dg;
    cols[1][sub][lane] = db;
    __syncthreads();
    if (sub < 2 && c < d) {
        Acc v = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) v += cols[sub][k][lane];
        ((typename P::W *)(sub ? dbias : dgain))[c] = P::f2w((float)v);
    }
}

// The workgroups' shares -> dg and db.  64 columns a workgroup, its sixteen wavefronts every sixteenth share each.
template <int DT>
__global__ __launch_bounds__(1024) void layernorm_dweight_kernel(const void *part_, void *dgain, void *dbias, int d, int shares)
{
    using P = Prec<DT>;
    using Acc = typename P::Acc;
    __shared__ Acc red[16][64];
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    Acc s = 0;
    if (c < 2 * d) {
#pragma unroll 4
        for (int r = sub; r < shares; r += 16) s += ((const Acc *)part_)[(size_t)r * 2 * d + c];
    }
    red[sub][lane] = s;
    __syncthreads();
    if (sub == 0 && c < 2 * d) {
        Acc v = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) v += red[k][lane];
        ((typename P::W *)(c < d ? dgain : dbias))[c < d ? c : c - d] = P::f2w((float)v);
    }
}

// Which rows go through registers: up to 12288 elements by fours, 8192 (24 elements a lane spill) 16-bit ones and 4096 fp64 ones one by one.
bool norm_grad_in_registers(int dtype, int d, bool fours) { return d <= (dtype == kFP32 ? 4096 : fours ? 12288 : 8192); }

// Few rows take one launch.  us, one launch / two: 256 rows of 768 5.2 / 7.7, of 5120 8.8 / 10.2, 400 rows of 2048 8.6 / 8.4; rows of 12288
// are slow one by one, 64 of them 14.6 / 10.1, 256 23.8 / 16.2, of 8101 18.3 / 14.7.
bool norm_grad_few(int dtype, int rows, int d) { return rows <= 256 && (d <= 5120 || !norm_grad_in_registers(dtype, d, d % 4 == 0)); }

// How many workgroups a backward pass over many rows has, each with a share of the weights' gradient: one a CU, and two rows (eight, where
// wavefronts have rows of their own) for each at least.  The kernel for any length, where a row is a workgroup's whole latency: one row, 1024
// at most.  us with 256 / 512 / 1024 / 2048 of them, bf16: 1000 rows of 13001 251 / 141 / 83 / 83, 4096 rows of 8193 723 / 438 / 297 / 242, of
// 13001 1180 / 705 / 523 / 389; fp32 parameters, 4096 rows of 5120 655 / 478 / 344 / 290.  2048 would take twice the scratch, 16 KiB a
// column, for rows longer than any in use.
int norm_grad_shares(int dtype, int rows, int d)
{
    const bool registers = norm_grad_in_registers(dtype, d, d % 4 == 0);
    const int each = !registers ? 1 : d <= 1536 ? 8 : 2, most = registers ? 256 : 1024, n = (rows + each - 1) / each;
    return n < most ? n : most;
}

// ------------------------------------------------------------------ LM head: cross entropy's gradient
// Of fp32 parameters, with fp64 activations and sums (16-bit types: zo_gemm_grad.hip).  The vocabulary is worked in pieces of
// `width` words whose logits [rows, width] are the only ones in memory.  RowState: per row
// the running maximum and sum of exponentials over the pieces so far, and the target's logit.
struct RowState { double max, sum, hit; };

// Takes a piece's logits into the rows' states.  `words`: how many words the piece has.
__global__ __launch_bounds__(256) void head_stats_kernel(const double *__restrict__ logits, const int32_t *__restrict__ target, RowState *__restrict__ state,
                                                         int words, int first_word)
{
    __shared__ double red[16];
    const size_t r = blockIdx.x;
    const double *lg = logits + r * words;
    double mx = -INFINITY;
    for (int c = threadIdx.x; c < words; c += blockDim.x) mx = lg[c] > mx ? lg[c] : mx;
    mx = block_max(mx, red);
    const double ref = mx > -INFINITY ? mx : 0.0;              // of minus infinities and NaN alone: their sum is 0 or NaN
    double s = 0.0;
    for (int c = threadIdx.x; c < words; c += blockDim.x) s += exp(lg[c] - ref);
    s = block_sum(s, red);
    if (threadIdx.x != 0) return;
    RowState st = first_word ? state[r] : RowState{-INFINITY, 0.0, 0.0};
    const int at = target[r] - first_word;
    if (at >= 0 && at < words) st.hit = lg[at];
    const double top = st.max > mx ? st.max : mx;
    // what has no maximum above minus infinity adds its sum as it is: 0, or NaN if one of its logits is
    auto share = [&](double m, double v) { return m > -INFINITY ? v * exp(m - top) : v; };
    st.sum = share(st.max, st.sum) + share(mx, s);
    st.max = top;
    state[r] = st;
}

// Logits of a piece -> G = exp(l - lse) - [word is the target], 0 in rows that do not count, NaN in those whose target lies
// beyond the vocabulary.  `row_loss`: with one of the pieces, else null.
__global__ __launch_bounds__(256) void head_probs_kernel(double *__restrict__ logits, const int32_t *__restrict__ target, const RowState *__restrict__ state,
                                                         double *__restrict__ row_loss, int words, int first_word, int vocab)
{
    const size_t r = blockIdx.x;
    const int tg = target[r];
    const RowState st = state[r];
    const double nan = __builtin_nan(""), lse = tg >= vocab ? nan : st.max + log(st.sum);
    if (row_loss && threadIdx.x == 0 && blockIdx.y == 0) row_loss[r] = tg < 0 ? 0.0 : lse - st.hit;
    const int at = tg - first_word, c = blockIdx.y * blockDim.x + threadIdx.x;
    if (c >= words) return;
    double *lg = logits + r * words + c;
    *lg = tg < 0 ? 0.0 : c == at ? expm1(*lg - lse) : exp(*lg - lse);
}

// Both of the above in one launch, for a vocabulary in one piece of up to kSoftmaxWords: a row's logits stay in registers between.
constexpr int kSoftmaxWords = 4096;
__global__ __launch_bounds__(256) void head_softmax_kernel(double *__restrict__ logits, const int32_t *__restrict__ target, double *__restrict__ row_loss, int vocab)
{
    __shared__ double red[16];
    constexpr int NE = kSoftmaxWords / 256;
    const size_t r = blockIdx.x;
    const int tg = target[r];
    double *lg = logits + r * vocab;
    double v[NE], mx = -INFINITY, s = 0.0;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        const int c = threadIdx.x + 256 * i;
        v[i] = c < vocab ? lg[c] : -INFINITY;
    }
    const double hit = tg >= 0 && tg < vocab ? lg[tg] : 0.0;
#pragma unroll
    for (int i = 0; i < NE; ++i) mx = v[i] > mx ? v[i] : mx;
    mx = block_max(mx, red);
#pragma unroll
    for (int i = 0; i < NE; ++i)
        if (256 * i < vocab) s += exp(v[i] - mx);
    s = block_sum(s, red);
    const double lse = tg >= vocab ? __builtin_nan("") : mx + log(s);
    if (threadIdx.x == 0) row_loss[r] = tg < 0 ? 0.0 : lse - hit;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        const int c = threadIdx.x + 256 * i;
        if (c < vocab) lg[c] = tg < 0 ? 0.0 : c == tg ? expm1(v[i] - lse) : exp(v[i] - lse);
    }
}

// dx = scale G e (rows of G and dx: `rows`; added to what is there with `accumulate`) and de = scale G^T x, one launch: the first dx_tiles
// workgroups have tiles of dx, the others of de.  A workgroup owns 16 TB x 16 TB outputs, its W wavefronts take every W-th 16-deep piece
// of the contraction straight from memory into v_mfma_f64_16x16x4 operands, and the partial sums meet in LDS, in a fixed order (as in the
// layers of this precision).  x's rows whose target does not count are taken as zeros, whatever they hold, and dx's are zeros.
template <int TB, int W>
__global__ __launch_bounds__(64 * W) void head_products_kernel(const double *__restrict__ grad, const float *__restrict__ e, const double *__restrict__ x,
                                                               const int32_t *__restrict__ target, double *__restrict__ dx, float *__restrict__ de,
                                                               int rows, int words, int d, double scale, bool accumulate, int dx_tiles)
{
    typedef double f64x4 __attribute__((ext_vector_type(4)));
    constexpr int BT = 16 * TB;
    __shared__ double part[W][BT][BT + 1];
    const bool by_words = (int)blockIdx.x < dx_tiles;           // of dx, the contraction over the words
    const int tile = by_words ? (int)blockIdx.x : (int)blockIdx.x - dx_tiles;
    const int tiles_d = (d + BT - 1) / BT, i0 = tile / tiles_d * BT, j0 = tile % tiles_d * BT;
    const int m = by_words ? rows : words, k = by_words ? words : rows;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
    f64x4 acc[TB][TB] = {};
#pragma unroll 2
    for (int k0 = 16 * wave; k0 < k; k0 += 16 * W) {
        f64x4 av[TB], bv[TB];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int kk = k0 + 4 * g + q, kc = kk < k ? kk : k - 1;
            const bool live = kk < k && (by_words || target[kc] >= 0);
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const int i = i0 + 16 * t + r16 < m ? i0 + 16 * t + r16 : m - 1, j = j0 + 16 * t + r16 < d ? j0 + 16 * t + r16 : d - 1;   // clamped: never stored
                const double a = by_words ? grad[(size_t)i * words + kc] : grad[(size_t)kc * words + i];
                const double b = by_words ? (double)e[(size_t)kc * d + j] : x[(size_t)kc * d + j];
                av[t][q] = live ? a : 0.0;
                bv[t][q] = live ? b : 0.0;
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
        if (i >= m || j >= d) continue;
        double v = 0.0;
#pragma unroll
        for (int w = 0; w < W; ++w) v += part[w][o / BT][o % BT];
        v *= scale;
        if (by_words) {
            double *at = dx + (size_t)i * d + j;
            *at = target[i] < 0 ? 0.0 : accumulate ? *at + v : v;
        } else {
            de[(size_t)i * d + j] = (float)v;
        }
    }
}

// ------------------------------------------------------------------ global norm and clipping
// Chunk c of a batch: its tensor (found by the lanes side by side), where it starts and its elements.
struct ClipPlace { uint64_t src, dst; size_t at; uint32_t n; };
template <int N> __device__ __forceinline__ ClipPlace clip_place(const ClipBatchOf<N> &b, uint32_t c)
{
    const int lane = threadIdx.x & 63;
    int t = -1;
    for (int i = 0; i < b.n; i += 64) t += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < b.n && b.first[i + lane] <= c));
    t = __builtin_amdgcn_readfirstlane(t);
    const uint64_t src = b.src[t];
    const uint32_t end = t + 1 < b.n ? b.first[t + 1] : b.chunks;
    return {src & 0xffffffffffffull, b.dst[t], (size_t)(c - b.first[t]) * kClipChunk, c + 1 == end ? (uint32_t)(src >> 48) + 1 : kClipChunk};
}

// f(element, the 16 bytes that start there) over a chunk of n elements, what lies past its end as zeros; in a whole chunk kClipAhead pieces a
// thread are under way together.
constexpr int kClipAhead = 8;
template <typename W, class F> __device__ __forceinline__ void clip_chunk(const W *src, uint32_t n, F &&f)
{
    constexpr uint32_t E = 16 / sizeof(W), STEP = 256 * E;
    static_assert(kClipChunk % (kClipAhead * STEP) == 0, "a chunk is whole bursts");
    if (n == kClipChunk) {
        for (uint32_t i0 = 0; i0 < kClipChunk; i0 += kClipAhead * STEP) {
            uint4 v[kClipAhead];
#pragma unroll
            for (int k = 0; k < kClipAhead; ++k) v[k] = *(const uint4 *)(src + i0 + k * STEP + threadIdx.x * E);
#pragma unroll
            for (int k = 0; k < kClipAhead; ++k) f(i0 + k * STEP + threadIdx.x * E, v[k]);
        }
        return;
    }
    for (uint32_t i = threadIdx.x * E; i < n; i += STEP) {
        union { uint4 v; W w[E]; } u;
        if (i + E <= n) u.v = *(const uint4 *)(src + i);
        else
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) u.w[e] = i + e < n ? src[i + e] : (W)0;
        f(i, u.v);
    }
}
template <typename W> __device__ __forceinline__ W clip_element(const uint4 &v, int e)
{
    const uint32_t words[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(W) == 4) return __uint_as_float(words[e]);
    else return (W)(e & 1 ? words[e / 2] >> 16 : words[e / 2] & 0xffff);
}

// sum g^2 of a batch of tensors, one partial sum per workgroup, in fp64: no square of an fp32 number leaves its range, and the
// sum of 10^9 squares is good to 1e-11 whatever their order.  `seen`: slots that an earlier batch has written (these add to it).
template <int DT, int N>
__global__ __launch_bounds__(256) void grad_norm_kernel(ClipBatchOf<N> b, double *__restrict__ part, int seen)
{
    using W = typename Prec<DT>::W;
    __shared__ double red[16];
    constexpr int E = 16 / sizeof(W);
    double s[4] = {0.0, 0.0, 0.0, 0.0};                         // side by side: a chain of one would wait for each fma
    for (uint32_t c = blockIdx.x; c < b.chunks; c += gridDim.x) {
        const ClipPlace t = clip_place(b, c);
        clip_chunk((const W *)t.src + t.at, t.n, [&](uint32_t, const uint4 &v) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const double g = (double)Prec<DT>::w2f(clip_element<W>(v, e));
                s[e & 3] = __builtin_fma(g, g, s[e & 3]);
            }
        });
    }
    const double sum = block_sum((s[0] + s[1]) + (s[2] + s[3]), red);
    if (threadIdx.x == 0) part[blockIdx.x] = (int)blockIdx.x < seen ? part[blockIdx.x] + sum : sum;
}

// dst = rn(c src), c = max / norm where norm exceeds max, else 1; where the norm is not a finite number, zeros.  Every workgroup adds up the
// partial sums itself, in the same order.  Gradients of up to the memory-side cache's 256 MiB are found there the second time: stores past it
// leave them there (125 M bf16 gradients into another buffer 122 us, 150 with plain stores; from the last chunk down 122).  117 us with
// one launch a pass (501 MB that must move, 98 us at the copy rate), where tables of 124 tensors took two.
template <int DT, int N>
__global__ __launch_bounds__(256) void grad_scale_kernel(ClipBatchOf<N> b, const double *__restrict__ part, int n_part, float max_norm, double *__restrict__ out, bool write_norm)
{
    using P = Prec<DT>;
    using W = typename P::W;
    __shared__ double red[16];
    constexpr int E = 16 / sizeof(W);
    double s = 0.0;
    for (int i = threadIdx.x; i < n_part; i += blockDim.x) s += part[i];
    const double norm = __builtin_sqrt(block_sum(s, red));
    const bool finite = norm - norm == 0.0;
    const double coef = !finite ? 0.0 : norm > (double)max_norm ? (double)max_norm / norm : 1.0;
    if (write_norm && blockIdx.x == 0 && threadIdx.x == 0) { out[0] = norm; out[1] = coef; }
    // c as a fraction from a half to one and a power of two: c itself may lie beyond fp32's range where c src does not
    int power;
    const float fraction = (float)frexp(coef, &power);
    for (uint32_t c = blockIdx.x; c < b.chunks; c += gridDim.x) {
        const ClipPlace t = clip_place(b, c);
        if (coef == 1.0 && t.dst == t.src) continue;
        const uint32_t n = t.n;
        W *dst = (W *)t.dst + t.at;
        clip_chunk((const W *)t.src + t.at, n, [&](uint32_t i, const uint4 &v) {
            union { u32x4 v; W w[E]; } o;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float g = P::w2f(clip_element<W>(v, e));
                // fp32: the product in fp64, rounded once.  16-bit types: c's rounding to fp32 and the product's are 2^-12 of their half step and less
                if constexpr (DT == kFP32) o.w[e] = finite ? (float)(coef * (double)g) : 0.0f;
                else o.w[e] = P::f2w(finite ? ldexpf(fraction * g, power) : 0.0f);
            }
            if (i + E <= n) __builtin_nontemporal_store(o.v, (u32x4 *)(dst + i));
            else
                for (int e = 0; e < E; ++e)
                    if (i + e < n) dst[i + e] = o.w[e];
        });
    }
}

}  // namespace

// ------------------------------------------------------------------ launchers

namespace {
struct NormGrad {
    const void *dy, *resid, *gain, *mean, *rstd;
    void *dresid, *part;
    int rows, d;
    bool accumulate, weights;
};
template <int DT, int NV, int WPR, int VW = 4> void norm_grad_rows(const NormGrad &a, int shares, hipStream_t s)
{
    using P = Prec<DT>;
    using Acc = typename P::Acc;
    layernorm_grad_rows_kernel<DT, NV, WPR, VW><<<dim3(shares), dim3(WPR == 1 ? 256 : 64 * WPR), WPR == 1 ? 2 * a.d * sizeof(Acc) : 0, s>>>(
        (const typename P::A *)a.dy, (const typename P::R *)a.resid, (const typename P::W *)a.gain, (const Acc *)a.mean, (const Acc *)a.rstd,
        (typename P::R *)a.dresid, (Acc *)a.part, a.rows, a.d, a.accumulate, a.weights);
}
template <int DT> void norm_grad(const NormGrad &a, int shares, hipStream_t s)
{
    const bool fours = DT != kFP32 && a.d % 4 == 0 && ((uintptr_t)a.resid | (uintptr_t)a.dresid) % 16 == 0 && ((uintptr_t)a.dy | (uintptr_t)a.gain) % 8 == 0;
    if (!norm_grad_in_registers(DT, a.d, fours)) {
        layernorm_grad_kernel<DT><<<dim3(shares), dim3(256), 0, s>>>(a.dy, a.resid, a.gain, a.mean, a.rstd, a.dresid, a.part, a.rows, a.d, a.accumulate,
                                                                    a.weights);
        return;
    }
    if constexpr (DT != kFP32) {
        if (fours && a.d <= 1536) {
            switch ((a.d + 255) / 256) {
            case 1: return norm_grad_rows<DT, 1, 1>(a, shares, s);
            case 2: return norm_grad_rows<DT, 2, 1>(a, shares, s);
            case 3: return norm_grad_rows<DT, 3, 1>(a, shares, s);
            case 4: return norm_grad_rows<DT, 4, 1>(a, shares, s);
            case 5: return norm_grad_rows<DT, 5, 1>(a, shares, s);
            default: return norm_grad_rows<DT, 6, 1>(a, shares, s);
            }
        }
        if (fours && a.d <= 5120) {
            switch ((a.d + 1023) / 1024) {
            case 2: return norm_grad_rows<DT, 2, 4>(a, shares, s);
            case 3: return norm_grad_rows<DT, 3, 4>(a, shares, s);
            case 4: return norm_grad_rows<DT, 4, 4>(a, shares, s);
            default: return norm_grad_rows<DT, 5, 4>(a, shares, s);
            }
        }
        if (fours && a.d <= 8192) return norm_grad_rows<DT, 4, 8>(a, shares, s);
        if (fours) return norm_grad_rows<DT, 6, 8>(a, shares, s);
        if (a.d > 4096) return norm_grad_rows<DT, 16, 8, 1>(a, shares, s);
        if (a.d > 2048) return norm_grad_rows<DT, 16, 4, 1>(a, shares, s);
    } else if (a.d > 2048) {
        return norm_grad_rows<DT, 8, 8, 1>(a, shares, s);
    }
    if (a.d > 512) return norm_grad_rows<DT, 8, 4, 1>(a, shares, s);
    norm_grad_rows<DT, 8, 1, 1>(a, shares, s);
}
}  // namespace

size_t layernorm_grad_scratch(int dtype, int rows, int d)
{
    return norm_grad_few(dtype, rows, d) ? 256 : (size_t)norm_grad_shares(dtype, rows, d) * 2 * d * acc_bytes(dtype);
}

hipError_t launch_layernorm_grad(const void *dy, const void *resid, const void *gain, const void *mean, const void *rstd, void *dresid, void *dgain,
                                 void *dbias, void *scratch, int dtype, int rows, int d, bool accumulate, hipStream_t s)
{
    if (norm_grad_few(dtype, rows, d)) {
        const int row_blocks = dresid ? rows : 0, blocks = row_blocks + (dgain ? (d + 31) / 32 : 0);
        ZO_DISPATCH_DT(dtype, (layernorm_grad_few_kernel<DT><<<dim3(blocks), dim3(256), 0, s>>>(dy, resid, gain, mean, rstd, dresid, dgain, dbias, rows, d,
                                                                                               accumulate, row_blocks)));
        return hipGetLastError();
    }
    const NormGrad a{dy, resid, gain, mean, rstd, dresid, scratch, rows, d, accumulate, dgain != nullptr};
    const int shares = norm_grad_shares(dtype, rows, d);
    ZO_DISPATCH_DT(dtype, norm_grad<DT>(a, shares, s));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !dgain) return e;
    ZO_DISPATCH_DT(dtype, (layernorm_dweight_kernel<DT><<<dim3((2 * d + 63) / 64), dim3(1024), 0, s>>>(scratch, dgain, dbias, d, shares)));
    return hipGetLastError();
}

namespace {
// Words of a piece: logits of 2^25 words and rows (256 MiB) at most, 64 words at least.
int head_f64_width(int rows, int vocab)
{
    const long w = (1l << 25) / rows / 64 * 64;
    return w >= vocab ? vocab : (int)(w < 64 ? 64 : w);
}
// 32 x 32 outputs a workgroup where dx has enough of them (or de too many of 16 x 16 for a grid of 2^32 threads)
bool head_f64_many(int rows, int d, int words)
{
    return (long)((rows + 31) / 32) * ((d + 31) / 32) >= 256 || (long)((words + 15) / 16) * ((d + 15) / 16) > 1l << 22;
}
// Does a grid, counted in threads by 32 bits, hold both products' workgroups of 256?
bool head_f64_fits(int rows, int d, int vocab)
{
    return ((long)((rows + 31) / 32) + (head_f64_width(rows, vocab) + 31) / 32) * ((d + 31) / 32) < 1l << 24;
}
size_t head_f64_state(int rows) { return ((size_t)rows * sizeof(RowState) + 255) / 256 * 256; }

hipError_t head_grad_f64(const double *x, const float *e, const int32_t *target, double *row_loss, double *dx, float *de, void *scratch, int rows, int d,
                         int vocab, double scale, hipStream_t s)
{
    RowState *state = (RowState *)scratch;
    double *logits = (double *)((char *)scratch + head_f64_state(rows));
    const int width = head_f64_width(rows, vocab);
    auto piece = [&](int v0) { return vocab - v0 < width ? vocab - v0 : width; };
    auto make_logits = [&](int v0) {
        const float *w = e + (size_t)v0 * d;
        return launch_linear(x, w, w, nullptr, nullptr, logits, kFP32, 1, rows, piece(v0), d, 3, true, s);
    };
    hipError_t err = hipSuccess;
    const bool together = width == vocab && vocab <= kSoftmaxWords;
    if (together) {
        if ((err = make_logits(0)) != hipSuccess) return err;
        head_softmax_kernel<<<dim3(rows), dim3(256), 0, s>>>(logits, target, row_loss, vocab);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    for (int v0 = 0; v0 < vocab && !together; v0 += width) {
        if ((err = make_logits(v0)) != hipSuccess) return err;
        head_stats_kernel<<<dim3(rows), dim3(256), 0, s>>>(logits, target, state, piece(v0), v0);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    for (int v0 = 0; v0 < vocab; v0 += width) {
        // (a single piece's logits are still there)
        if (width < vocab && (err = make_logits(v0)) != hipSuccess) return err;
        const int n = piece(v0);
        if (!together) {
            head_probs_kernel<<<dim3(rows, (n + 255) / 256), dim3(256), 0, s>>>(logits, target, state, v0 == 0 ? row_loss : nullptr, n, v0, vocab);
            if ((err = hipGetLastError()) != hipSuccess) return err;
        }
        auto products = [&](auto kern, int bt, int waves) {
            const long tiles_d = (d + bt - 1) / bt, dx_tiles = (rows + bt - 1) / bt * tiles_d, de_tiles = (n + bt - 1) / bt * tiles_d;
            kern<<<dim3((unsigned)(dx_tiles + de_tiles)), dim3(64 * waves), 0, s>>>(logits, e + (size_t)v0 * d, x, target, dx, de + (size_t)v0 * d, rows, n, d,
                                                                                   scale, v0 > 0, (int)dx_tiles);
            return hipGetLastError();
        };
        if ((err = head_f64_many(rows, d, n) ? products(head_products_kernel<2, 4>, 32, 4) : products(head_products_kernel<1, 8>, 16, 8)) != hipSuccess) return err;
    }
    return hipSuccess;
}
}  // namespace

size_t head_grad_scratch(int dtype, int rows, int d, int vocab)
{
    if (dtype != kFP32) return head_grad_mfma_scratch(rows, d, vocab);
    if (!head_f64_fits(rows, d, vocab)) return 0;
    return head_f64_state(rows) + (size_t)rows * head_f64_width(rows, vocab) * sizeof(double);
}

hipError_t launch_head_grad(const void *x, const void *e, const int32_t *target, void *row_loss, void *dx, void *de, void *scratch, int dtype, int rows,
                            int d, int vocab, float scale, hipStream_t s)
{
    if (dtype != kFP32) return launch_head_grad_mfma(x, e, target, row_loss, dx, de, scratch, dtype, rows, d, vocab, scale, s);
    if (!head_f64_fits(rows, d, vocab)) return hipErrorNotSupported;
    return head_grad_f64((const double *)x, (const float *)e, target, (double *)row_loss, (double *)dx, (float *)de, scratch, rows, d, vocab, (double)scale, s);
}

namespace {
// f(batch, whether it is the first) over batches of N tensors
template <int N, class F> hipError_t clip_batches(const void *const *src, void *const *dst, const uint64_t *numel, int n_tensors, F &&f)
{
    // tensors of a batch: as many as its table holds, and chunk numbers of 31 bits
    ClipBatchOf<N> b{};
    bool first = true;
    auto flush = [&] {
        if (b.n == 0) return hipSuccess;
        const hipError_t e = f(b, first);
        first = false;
        b.n = 0;
        b.chunks = 0;
        return e;
    };
    for (int i = 0; i < n_tensors; ++i) {
        if (numel[i] == 0) continue;
        const uint64_t chunks = (numel[i] + kClipChunk - 1) / kClipChunk;
        if (b.n == N || b.chunks + chunks >= (1ull << 31)) {
            const hipError_t e = flush();
            if (e != hipSuccess) return e;
        }
        b.src[b.n] = (uint64_t)(uintptr_t)src[i] | (numel[i] - (chunks - 1) * kClipChunk - 1) << 48;
        b.dst[b.n] = (uint64_t)(uintptr_t)dst[i];
        b.first[b.n++] = b.chunks;
        b.chunks += (uint32_t)chunks;
    }
    return flush();
}

template <int DT, int N>
hipError_t grad_clip(const void *const *src, void *const *dst, const uint64_t *numel, int n_tensors, float max_norm, double *norm, double *part, hipStream_t s)
{
    int slots = 0;
    auto grid = [](const ClipBatchOf<N> &b) { return dim3(b.chunks < kClipSlots ? b.chunks : kClipSlots); };
    hipError_t err = clip_batches<N>(src, dst, numel, n_tensors, [&](const ClipBatchOf<N> &b, bool) {
        grad_norm_kernel<DT, N><<<grid(b), dim3(256), 0, s>>>(b, part, slots);
        slots = (int)grid(b).x > slots ? (int)grid(b).x : slots;
        return hipGetLastError();
    });
    if (err != hipSuccess) return err;
    bool done = false;
    err = clip_batches<N>(src, dst, numel, n_tensors, [&](const ClipBatchOf<N> &b, bool first) {
        grad_scale_kernel<DT, N><<<grid(b), dim3(256), 0, s>>>(b, part, slots, max_norm, norm, first);
        done = true;
        return hipGetLastError();
    });
    if (err != hipSuccess || done) return err;
    grad_scale_kernel<DT, N><<<dim3(1), dim3(256), 0, s>>>(ClipBatchOf<N>{}, part, 0, max_norm, norm, true);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_grad_clip(const void *const *src, void *const *dst, const uint64_t *numel, int n_tensors, int dtype, float max_norm, double *norm,
                            void *scratch, hipStream_t s)
{
    auto go = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        // a kernel's arguments are copied at each launch, 4 KiB of the long table: a few small tensors take 11.4 us with the short one, 12.4 with
        // the long; more tensors than the short table holds would take launches of 4 us each
        auto f = n_tensors <= kClipFew ? grad_clip<DT, kClipFew> : grad_clip<DT, kClipMax>;
        return f(src, dst, numel, n_tensors, max_norm, norm, (double *)scratch, s);
    };
    return dtype == kFP32 ? go(std::integral_constant<int, kFP32>{}) : dtype == kBF16 ? go(std::integral_constant<int, kBF16>{}) : go(std::integral_constant<int, kFP16>{});
}

}  // namespace zo
