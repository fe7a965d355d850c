// Gradient of the model's last module: LayerNorm forward with its statistics and its backward pass, the elementwise parts of
// the LM head's cross-entropy gradient with the fp64 products of fp32 parameters, and the global norm and clipping of a
// model's gradients.  (DistZO2 trains by the two losses of Eq. 1 alone; the last module is the one whose exact gradient
// needs no other module's, and z . grad L is what Eq. 2's g estimates.)
#include "zo_kernels.h"
#include "zo_types.hip.h"

namespace zo {

namespace {

#define ZO_DISPATCH_DT(dtype, CALL)                  \
    switch (dtype) {                                 \
    case kFP32: { constexpr int DT = kFP32; CALL; } break; \
    case kBF16: { constexpr int DT = kBF16; CALL; } break; \
    case kFP16: { constexpr int DT = kFP16; CALL; } break; \
    default: return hipErrorInvalidValue;            \
    }

// ------------------------------------------------------------------ LayerNorm forward, statistics kept
// mean = sum h / d, rstd = 1 / sqrt(sum (h - mean)^2 / d + eps), y = g (h - mean) rstd + b.  One workgroup per row.
template <int DT>
__global__ __launch_bounds__(256) void layernorm_stats_kernel(const void *resid, const void *gain, const void *bias, void *y, void *mean_out,
                                                              void *rstd_out, int d, float eps)
{
    using P = Prec<DT>;
    using Acc = typename P::Acc;
    __shared__ Acc red[16];
    const size_t row = blockIdx.x;
    const typename P::R *h = (const typename P::R *)resid + row * d;
    const typename P::W *g = (const typename P::W *)gain, *b = (const typename P::W *)bias;
    typename P::A *out = (typename P::A *)y + row * d;
    Acc s = 0;
    for (int c = threadIdx.x; c < d; c += blockDim.x) s += (Acc)h[c];
    const Acc mean = block_sum(s, red) / (Acc)d;
    Acc v = 0;
    for (int c = threadIdx.x; c < d; c += blockDim.x) { const Acc t = (Acc)h[c] - mean; v += t * t; }
    const Acc var = block_sum(v, red) / (Acc)d;
    Acc rstd;
    if constexpr (sizeof(Acc) == 8) rstd = 1.0 / __builtin_sqrt(var + (double)eps);
    else rstd = 1.0f / __builtin_sqrtf(var + eps);
    if (threadIdx.x == 0) {
        ((Acc *)mean_out)[row] = mean;
        ((Acc *)rstd_out)[row] = rstd;
    }
    for (int c = threadIdx.x; c < d; c += blockDim.x) out[c] = P::acc2a(((Acc)h[c] - mean) * rstd * (Acc)P::w2f(g[c]) + (Acc)P::w2f(b[c]));
}

// ------------------------------------------------------------------ LayerNorm backward
// With xh = (h - mean) rstd and a = dy g:   dh = rstd (a - mean_c(a) - xh mean_c(a xh)),
//                                           dg = sum_r dy xh,  db = sum_r dy.
// One workgroup per row for dh.
template <int DT>
__global__ __launch_bounds__(256) void layernorm_dresid_kernel(const void *dy_, const void *resid, const void *gain, const void *mean_, const void *rstd_,
                                                               void *dresid, int d, int accumulate)
{
    using P = Prec<DT>;
    using Acc = typename P::Acc;
    __shared__ Acc red[16];
    const size_t row = blockIdx.x;
    const typename P::A *dy = (const typename P::A *)dy_ + row * d;
    const typename P::R *h = (const typename P::R *)resid + row * d;
    const typename P::W *g = (const typename P::W *)gain;
    typename P::R *out = (typename P::R *)dresid + row * d;
    const Acc mean = ((const Acc *)mean_)[row], rstd = ((const Acc *)rstd_)[row];
    Acc sa = 0, sx = 0;
    for (int c = threadIdx.x; c < d; c += blockDim.x) {
        const Acc a = P::a2acc(dy[c]) * (Acc)P::w2f(g[c]);
        sa += a;
        sx += a * (((Acc)h[c] - mean) * rstd);
    }
    sa = block_sum(sa, red) / (Acc)d;
    sx = block_sum(sx, red) / (Acc)d;
    for (int c = threadIdx.x; c < d; c += blockDim.x) {
        const Acc a = P::a2acc(dy[c]) * (Acc)P::w2f(g[c]), xh = ((Acc)h[c] - mean) * rstd;
        const Acc v = rstd * (a - sa - xh * sx);
        out[c] = accumulate ? out[c] + (typename P::R)v : (typename P::R)v;
    }
}

// Gain's and bias's gradient: workgroup (x, y) adds up 64 columns over the y-th run of `run` rows, four rows at a time, and
// leaves its two sums in part[y]; layernorm_dweight_finish_kernel adds the runs in order.
template <int DT>
__global__ __launch_bounds__(256) void layernorm_dweight_kernel(const void *dy_, const void *resid, const void *mean_, const void *rstd_, void *part_,
                                                                int rows, int d, int run)
{
    using P = Prec<DT>;
    using Acc = typename P::Acc;
    __shared__ Acc red[2][4][64];
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    const int first = blockIdx.y * run, last = first + run < rows ? first + run : rows;
    Acc dg = 0, db = 0;
    if (c < d) {
        for (int r = first + sub; r < last; r += 4) {
            const Acc v = P::a2acc(((const typename P::A *)dy_)[(size_t)r * d + c]);
            const Acc xh = ((Acc)((const typename P::R *)resid)[(size_t)r * d + c] - ((const Acc *)mean_)[r]) * ((const Acc *)rstd_)[r];
            dg += v * xh;
            db += v;
        }
    }
    red[0][sub][lane] = dg;
    red[1][sub][lane] = db;
    __syncthreads();
    if (sub == 0 && c < d) {
        Acc *part = (Acc *)part_ + (size_t)blockIdx.y * 2 * d;
        part[c] = (red[0][0][lane] + red[0][1][lane]) + (red[0][2][lane] + red[0][3][lane]);
        part[d + c] = (red[1][0][lane] + red[1][1][lane]) + (red[1][2][lane] + red[1][3][lane]);
    }
}

template <int DT>
__global__ __launch_bounds__(256) void layernorm_dweight_finish_kernel(const void *part_, void *dgain, void *dbias, int d, int runs)
{
    using P = Prec<DT>;
    using Acc = typename P::Acc;
    __shared__ Acc red[4][64];
    const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    Acc s = 0;
    if (c < 2 * d)
        for (int r = sub; r < runs; r += 4) s += ((const Acc *)part_)[(size_t)r * 2 * d + c];
    red[sub][lane] = s;
    __syncthreads();
    if (sub == 0 && c < 2 * d) {
        const Acc v = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
        ((typename P::W *)(c < d ? dgain : dbias))[c < d ? c : c - d] = P::f2w((float)v);
    }
}

// Rows per run of the weights' sums: so many runs that their workgroups fill the chip, 64 rows at least.
int dweight_run(int rows, int d)
{
    const int columns = (d + 63) / 64;
    int runs = (2048 + columns - 1) / columns;
    runs = runs < 1 ? 1 : runs;
    const int run = (rows + runs - 1) / runs;
    return run < 64 ? 64 : run;
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
    double s = 0.0;
    for (int c = threadIdx.x; c < words; c += blockDim.x) s += exp(lg[c] - mx);
    s = block_sum(s, red);
    if (threadIdx.x != 0) return;
    RowState st = first_word ? state[r] : RowState{-INFINITY, 0.0, 0.0};
    const int at = target[r] - first_word;
    if (at >= 0 && at < words) st.hit = lg[at];
    const double top = st.max > mx ? st.max : mx;
    st.sum = (st.max > -INFINITY ? st.sum * exp(st.max - top) : 0.0) + s * exp(mx - top);
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

// c[i, j] (+)= scale sum_k a(i, k) b(k, j): a's element at a[i ai + k ak], b's row k at b[k n].  64 x 64 outputs a workgroup, 16
// terms a slab.  Rows of b (`live_k`) or of c (`live_i`) whose target does not count are taken as zeros, whatever they hold.
template <typename TB, typename TC>
__global__ __launch_bounds__(256) void head_product_kernel(const double *__restrict__ a, size_t ai, size_t ak, const TB *__restrict__ b, TC *__restrict__ c, int m,
                                                           int n, int k, double scale, int accumulate, const int32_t *__restrict__ live_k,
                                                           const int32_t *__restrict__ live_i)
{
    constexpr int B = 64, S = 16;
    __shared__ double as[S][B + 1], bs[S][B + 1];
    const int i0 = blockIdx.y * B, j0 = blockIdx.x * B, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    double acc[4][4] = {};
    for (int k0 = 0; k0 < k; k0 += S) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int idx = threadIdx.x + 256 * e;
            // neighbouring threads along whichever index is contiguous
            const int ar = ak == 1 ? idx / S : idx % B, akk = ak == 1 ? idx % S : idx / B;
            as[akk][ar] = k0 + akk < k && i0 + ar < m ? a[(size_t)(i0 + ar) * ai + (size_t)(k0 + akk) * ak] : 0.0;
            const int bc = idx % B, bkk = idx / B;
            const bool in = k0 + bkk < k && j0 + bc < n && (!live_k || live_k[k0 + bkk] >= 0);
            bs[bkk][bc] = in ? (double)b[(size_t)(k0 + bkk) * n + (j0 + bc)] : 0.0;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < S; ++kk) {
            double x[4], y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = as[kk][ty + 16 * e]; y[e] = bs[kk][tx + 16 * e]; }
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[p][q] += x[p] * y[q];
        }
        __syncthreads();
    }
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = i0 + ty + 16 * p, j = j0 + tx + 16 * q;
            if (i >= m || j >= n) continue;
            TC *at = c + (size_t)i * n + j;
            const double v = live_i && live_i[i] < 0 ? 0.0 : scale * acc[p][q];
            *at = (TC)(accumulate ? (double)*at + v : v);
        }
}

// ------------------------------------------------------------------ global norm and clipping
// The tensor of chunk `c`: lanes compare the table's first chunks side by side.  All lanes return the same.
__device__ __forceinline__ int clip_tensor(const ClipBatch &b, uint32_t c)
{
    const int lane = threadIdx.x & 63;
    int t = 0;
    for (int i = 0; i < b.n; i += 64) t += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < b.n && b.d[i + lane].first <= c));
    return __builtin_amdgcn_readfirstlane(t - 1);
}

template <int DT> __device__ __forceinline__ void clip_load(const void *src, uint32_t n, uint32_t i, float (&v)[16 / sizeof(typename Prec<DT>::W)])
{
    using W = typename Prec<DT>::W;
    constexpr int E = 16 / sizeof(W);
    const W *p = (const W *)src + i;
    if (i + E <= n) {
        W w[E];
        *(uint4 *)w = *(const uint4 *)p;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = Prec<DT>::w2f(w[e]);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = i + e < n ? Prec<DT>::w2f(p[e]) : 0.0f;
    }
}

// sum g^2 of a batch of tensors, one partial sum per workgroup, in fp64: no square of an fp32 number leaves its range, and the
// sum of 10^9 squares is good to 1e-11 whatever their order.  `seen`: slots that an earlier batch has written (these add to it).
template <int DT>
__global__ __launch_bounds__(256) void grad_norm_kernel(ClipBatch b, double *__restrict__ part, int seen)
{
    __shared__ double red[16];
    constexpr int E = 16 / sizeof(typename Prec<DT>::W);
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < b.chunks; c += gridDim.x) {
        const ClipDesc &t = b.d[clip_tensor(b, c)];
        const uint32_t local = c - t.first, n = local + 1 == t.chunks ? t.last : kClipChunk;
        const void *src = (const typename Prec<DT>::W *)t.src + (size_t)local * kClipChunk;
        for (uint32_t i = threadIdx.x * E; i < n; i += blockDim.x * E) {
            float v[E];
            clip_load<DT>(src, n, i, v);
#pragma unroll
            for (int e = 0; e < E; ++e) s = __builtin_fma((double)v[e], (double)v[e], s);
        }
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) part[blockIdx.x] = (int)blockIdx.x < seen ? part[blockIdx.x] + s : s;
}

// dst = rn(c src), c = max / norm where norm exceeds max, else 1; where the norm is not a finite number, zeros.  Every workgroup adds up the
// partial sums itself, in the same order.  The chunks are taken from the last one down: those read last are the ones still in the
// memory-side cache.
template <int DT>
__global__ __launch_bounds__(256) void grad_scale_kernel(ClipBatch b, const double *__restrict__ part, int n_part, float max_norm, double *__restrict__ out, bool write_norm)
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
    for (uint32_t c0 = blockIdx.x; c0 < b.chunks; c0 += gridDim.x) {
        const uint32_t c = b.chunks - 1 - c0;
        const ClipDesc &t = b.d[clip_tensor(b, c)];
        if (coef == 1.0 && t.dst == t.src) continue;
        const uint32_t local = c - t.first, n = local + 1 == t.chunks ? t.last : kClipChunk;
        const void *src = (const W *)t.src + (size_t)local * kClipChunk;
        W *dst = (W *)t.dst + (size_t)local * kClipChunk;
        for (uint32_t i = threadIdx.x * E; i < n; i += blockDim.x * E) {
            float v[E];
            clip_load<DT>(src, n, i, v);
            W w[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                // fp32: the product in fp64, rounded once.  16-bit types: the fp32 product's rounding is 2^-13 of theirs and less
                if constexpr (DT == kFP32) w[e] = finite ? (float)(coef * (double)v[e]) : 0.0f;
                else w[e] = P::f2w(finite ? (float)coef * v[e] : 0.0f);
            }
            if (i + E <= n) *(uint4 *)(dst + i) = *(uint4 *)w;
            else
                for (int e = 0; e < E; ++e)
                    if (i + e < n) dst[i + e] = w[e];
        }
    }
}

}  // namespace

// ------------------------------------------------------------------ launchers
hipError_t launch_layernorm_stats(const void *resid, const void *gain, const void *bias, void *y, void *mean, void *rstd, int dtype, int rows, int d,
                                  float eps, hipStream_t s)
{
    ZO_DISPATCH_DT(dtype, (layernorm_stats_kernel<DT><<<dim3(rows), dim3(256), 0, s>>>(resid, gain, bias, y, mean, rstd, d, eps)));
    return hipGetLastError();
}

size_t layernorm_grad_scratch(int dtype, int rows, int d)
{
    const int run = dweight_run(rows, d);
    return (size_t)((rows + run - 1) / run) * 2 * d * acc_bytes(dtype);
}

hipError_t launch_layernorm_grad(const void *dy, const void *resid, const void *gain, const void *mean, const void *rstd, void *dresid, void *dgain,
                                 void *dbias, void *scratch, int dtype, int rows, int d, bool accumulate, hipStream_t s)
{
    if (dresid) {
        ZO_DISPATCH_DT(dtype, (layernorm_dresid_kernel<DT><<<dim3(rows), dim3(256), 0, s>>>(dy, resid, gain, mean, rstd, dresid, d, accumulate)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!dgain) return hipSuccess;
    const int run = dweight_run(rows, d), runs = (rows + run - 1) / run;
    ZO_DISPATCH_DT(dtype, (layernorm_dweight_kernel<DT><<<dim3((d + 63) / 64, runs), dim3(256), 0, s>>>(dy, resid, mean, rstd, scratch, rows, d, run)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    ZO_DISPATCH_DT(dtype, (layernorm_dweight_finish_kernel<DT><<<dim3((2 * d + 63) / 64), dim3(256), 0, s>>>(scratch, dgain, dbias, d, runs)));
    return hipGetLastError();
}

namespace {
// Words of a piece: logits of 2^25 words and rows (256 MiB) at most, 64 words at least.
int head_f64_width(int rows, int vocab)
{
    const long w = (1l << 25) / rows / 64 * 64;
    return w >= vocab ? vocab : (int)(w < 64 ? 64 : w);
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
    for (int v0 = 0; v0 < vocab; v0 += width) {
        if ((err = make_logits(v0)) != hipSuccess) return err;
        head_stats_kernel<<<dim3(rows), dim3(256), 0, s>>>(logits, target, state, piece(v0), v0);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    for (int v0 = 0; v0 < vocab; v0 += width) {
        // (a single piece's logits are still there)
        if (width < vocab && (err = make_logits(v0)) != hipSuccess) return err;
        const int n = piece(v0);
        head_probs_kernel<<<dim3(rows, (n + 255) / 256), dim3(256), 0, s>>>(logits, target, state, v0 == 0 ? row_loss : nullptr, n, v0, vocab);
        if ((err = hipGetLastError()) != hipSuccess) return err;
        head_product_kernel<float, double><<<dim3((d + 63) / 64, (rows + 63) / 64), dim3(256), 0, s>>>(
            logits, (size_t)n, 1, e + (size_t)v0 * d, dx, rows, d, n, scale, v0 > 0, nullptr, target);
        if ((err = hipGetLastError()) != hipSuccess) return err;
        head_product_kernel<double, float><<<dim3((d + 63) / 64, (n + 63) / 64), dim3(256), 0, s>>>(
            logits, 1, (size_t)n, x, de + (size_t)v0 * d, n, d, rows, scale, 0, target, nullptr);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    return hipSuccess;
}
}  // namespace

size_t head_grad_scratch(int dtype, int rows, int d, int vocab)
{
    if (dtype != kFP32) return head_grad_mfma_scratch(rows, d, vocab);
    return head_f64_state(rows) + (size_t)rows * head_f64_width(rows, vocab) * sizeof(double);
}

hipError_t launch_head_grad(const void *x, const void *e, const int32_t *target, void *row_loss, void *dx, void *de, void *scratch, int dtype, int rows,
                            int d, int vocab, float scale, hipStream_t s)
{
    if (dtype != kFP32) return launch_head_grad_mfma(x, e, target, row_loss, dx, de, scratch, dtype, rows, d, vocab, scale, s);
    return head_grad_f64((const double *)x, (const float *)e, target, (double *)row_loss, (double *)dx, (float *)de, scratch, rows, d, vocab, (double)scale, s);
}

namespace {
template <class F> hipError_t clip_batches(const void *const *src, void *const *dst, const uint64_t *numel, int n_tensors, bool backwards, F &&f)
{
    // tensors of a batch: as many as its table holds, and chunk numbers of 31 bits
    ClipBatch b{};
    hipError_t err = hipSuccess;
    bool any = false;
    auto flush = [&] {
        if (b.n == 0) return hipSuccess;
        const hipError_t e = f(b, any);
        any = true;
        b.n = 0;
        b.chunks = 0;
        return e;
    };
    for (int j = 0; j < n_tensors; ++j) {
        const int i = backwards ? n_tensors - 1 - j : j;
        if (numel[i] == 0) continue;
        const uint64_t chunks = (numel[i] + kClipChunk - 1) / kClipChunk;
        if (b.n == kClipMax || b.chunks + chunks >= (1ull << 31))
            if ((err = flush()) != hipSuccess) return err;
        b.d[b.n++] = ClipDesc{src[i], dst ? dst[i] : nullptr, b.chunks, (uint32_t)chunks, (uint32_t)(numel[i] - (chunks - 1) * kClipChunk), 0};
        b.chunks += (uint32_t)chunks;
    }
    return flush();
}
}  // namespace

hipError_t launch_grad_clip(const void *const *src, void *const *dst, const uint64_t *numel, int n_tensors, int dtype, float max_norm, double *norm,
                            void *scratch, hipStream_t s)
{
    double *part = (double *)scratch;
    int slots = 0;
    hipError_t err = clip_batches(src, nullptr, numel, n_tensors, false, [&](const ClipBatch &b, bool) {
        const int grid = (int)(b.chunks < kClipSlots ? b.chunks : kClipSlots);
        ZO_DISPATCH_DT(dtype, (grad_norm_kernel<DT><<<dim3(grid), dim3(256), 0, s>>>(b, part, slots)));
        slots = grid > slots ? grid : slots;
        return hipGetLastError();
    });
    if (err != hipSuccess) return err;
    bool done = false;
    err = clip_batches(src, dst, numel, n_tensors, true, [&](const ClipBatch &b, bool later) {
        const int grid = (int)(b.chunks < kClipSlots ? b.chunks : kClipSlots);
        ZO_DISPATCH_DT(dtype, (grad_scale_kernel<DT><<<dim3(grid), dim3(256), 0, s>>>(b, part, slots, max_norm, norm, !later)));
        done = true;
        return hipGetLastError();
    });
    if (err != hipSuccess || done) return err;
    ZO_DISPATCH_DT(dtype, (grad_scale_kernel<DT><<<dim3(1), dim3(256), 0, s>>>(ClipBatch{}, part, 0, max_norm, norm, true)));
    return hipGetLastError();
}

}  // namespace zo
