// AdamW step over many tensors in one pass (clipped gradients of the last modules -> weights).
//
//   g = c grad,  m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,
//   p <- p - (lr wd p + lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps))
//
// Elements go in blocks of 256, a block per wavefront and four elements per lane, because that is what shares a scale where moments are
// held in 8 bits: new moments, their largest magnitude and the 8-bit numbers all come out of one read.  Every operation below is one fp32
// rounding (division and square root too), so results are the same bits on any IEEE-754 machine.
#include "zo_kernels.h"
#include "zo_rng.hip.h"
#include "zo_types.hip.h"

namespace zo {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = kAdamBlock;
constexpr int kBlocksAhead = 4;                                 // of a wavefront: their loads are under way together
constexpr int kChunkBlocks = kAdamChunk / kBlock;
static_assert(kAdamChunk % (4 * kBlocksAhead * kBlock) == 0, "a chunk is whole rounds of four wavefronts");

// the largest of 64 unsigned numbers, in every lane (as wave_sum<float> goes: no trip through LDS)
__device__ __forceinline__ uint32_t wave_umax(uint32_t v)
{
    auto both = [](auto r) { return r[0] > r[1] ? r[0] : r[1]; };
    v = both(__builtin_amdgcn_permlane32_swap(v, v, false, false));
    v = both(__builtin_amdgcn_permlane16_swap(v, v, false, false));
    auto turned = [](uint32_t x, auto ctrl) {
        const uint32_t t = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, decltype(ctrl)::value, 0xf, 0xf, true);
        return t > x ? t : x;
    };
    v = turned(v, std::integral_constant<int, 0x128>{});       // row_ror:8
    v = turned(v, std::integral_constant<int, 0x124>{});
    v = turned(v, std::integral_constant<int, 0x122>{});
    return turned(v, std::integral_constant<int, 0x121>{});
}

// Four e4m3 numbers and back (nearest even, as the hardware converts; |y| is at most 448 and a rounding, never past the largest number).
__device__ __forceinline__ uint32_t to_e4m3(const float (&y)[4])
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
}
__device__ __forceinline__ void from_e4m3(uint32_t w, float scale, float (&x)[4])
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0] * scale; x[1] = lo[1] * scale; x[2] = hi[0] * scale; x[3] = hi[1] * scale;
}

// A block's new numbers as e4m3 and a scale, the largest magnitude / 448.  LOW (no number is negative): what is above zero stays above it,
// so that a root that is small beside its block's largest never makes a division by eps alone.  A block that holds anything not finite
// gets a scale that is not a number; one below 448 x 2^-126 in all its magnitudes is zeros.
template <bool LOW> __device__ __forceinline__ uint32_t hold8(const float (&x)[4], float &scale)
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t b = __float_as_uint(x[e]) & 0x7fffffffu;
        top = b > top ? b : top;
    }
    top = (uint32_t)__builtin_amdgcn_readfirstlane((int)wave_umax(top));       // (one for the wavefront: its tests are scalar)
    scale = __uint_as_float(top) * (1.0f / 448.0f);
    float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (top >= 0x7f800000u) {
        scale = __uint_as_float(0x7fc00000u);
    } else if (!(scale >= 0x1p-126f)) {
        scale = 0.0f;
    } else {
        const float inverse = 1.0f / scale;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[e] = x[e] * inverse;
            // (2^-9 for what is above zero, as no root of an fp32 number is below 2^-75; zero for zero)
            if (LOW) y[e] = __builtin_fmaxf(y[e], __builtin_fminf(x[e] * 0x1p100f, 0x1p-9f));
        }
    }
    return to_e4m3(y);
}

// The correctly rounded square root of four numbers.  Where all of a wavefront's lie between 2^-90 and 2^120: from the hardware's reciprocal root and
// one correction with the exact remainder, 6 instructions a number (the compiler's, for the whole range, takes 16).  The two differ for none of the 2^24
// numbers of two neighbouring powers of two, and a power of four goes through every step unchanged.
__device__ __forceinline__ float near_root(float v)
{
    const float y = __builtin_amdgcn_rsqf(v), s = v * y;
    return __builtin_fmaf(__builtin_fmaf(-s, s, v), 0.5f * y, s);
}
__device__ __forceinline__ void roots(const float (&v)[4], float (&root)[4])
{
    const float low = __builtin_fminf(__builtin_fminf(v[0], v[1]), __builtin_fminf(v[2], v[3])), high = __builtin_fmaxf(__builtin_fmaxf(v[0], v[1]), __builtin_fmaxf(v[2], v[3]));
    const bool plain = low > 0x1p-90f && high < 0x1p120f && v[0] == v[0] && v[1] == v[1] && v[2] == v[2] && v[3] == v[3];
    if (__builtin_amdgcn_ballot_w64(!plain) == 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) root[e] = near_root(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) root[e] = __builtin_sqrtf(v[e]);       // (rounded to nearest; the intrinsic of that name is a step off at times)
    }
}

// Chunk c of a batch: its tensor (found by the lanes side by side), its first element and how many it has.
#define ZO_GLOBAL __attribute__((address_space(1)))            // (addresses out of a table would take flat accesses, which go by the LDS too)
struct AdamPlace { ZO_GLOBAL char *param, *state; const ZO_GLOBAL char *grad; uint64_t at; uint32_t n, tensor; };
template <int N> __device__ __forceinline__ AdamPlace adam_place(const AdamBatchOf<N> &b, uint32_t c)
{
    const int lane = threadIdx.x & 63;
    int t = -1;
    for (int i = 0; i < b.n; i += 64) t += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < b.n && b.first[i + lane] <= c));
    t = __builtin_amdgcn_readfirstlane(t);
    const uint64_t param = b.param[t];
    const uint32_t end = t + 1 < b.n ? b.first[t + 1] : b.chunks;
    return {(ZO_GLOBAL char *)(uintptr_t)(param & 0xffffffffffffull), (ZO_GLOBAL char *)(uintptr_t)b.state[t], (const ZO_GLOBAL char *)(uintptr_t)b.grad[t],
            (uint64_t)(c - b.first[t]) * kAdamChunk,
            c + 1 == end ? (uint32_t)(param >> 48) + 1 : kAdamChunk, (uint32_t)t};
}

// four stored numbers of a tensor, `left` of which exist (WHOLE: all)
template <typename W> struct Four { typedef W type __attribute__((ext_vector_type(4))); };
template <bool WHOLE, typename W> __device__ __forceinline__ typename Four<W>::type load4(const ZO_GLOBAL W *p, int left)
{
    typename Four<W>::type f = {};
    if (WHOLE || left >= 4) return *(const ZO_GLOBAL typename Four<W>::type *)p;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) f[e] = p[e];
    return f;
}
template <bool WHOLE, typename W> __device__ __forceinline__ void store4(ZO_GLOBAL W *p, const typename Four<W>::type &f, int left)
{
    if (WHOLE || left >= 4) {
        *(ZO_GLOBAL typename Four<W>::type *)p = f;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) p[e] = f[e];
}

// kBlocksAhead blocks from block r of a chunk on, as many as the chunk has (WHOLE: all of them and every element).
template <int DT, int BITS, bool SR, bool WHOLE> __device__ __forceinline__ void adamw_blocks(const AdamPlace &t, int r, const AdamScalars &k, float coef, int power)
{
    using P = Prec<DT>;
    using W = typename P::W;
    using F = typename Four<W>::type;
    const int lane = threadIdx.x & 63;
    F pw[kBlocksAhead], gw[kBlocksAhead];
    f32x4 m32[BITS == 32 ? kBlocksAhead : 1], v32[BITS == 32 ? kBlocksAhead : 1];
    uint32_t m8[kBlocksAhead], v8[kBlocksAhead];
    f32x2 scale[kBlocksAhead];
    ZO_GLOBAL W *param = (ZO_GLOBAL W *)t.param + t.at + r * kBlock + 4 * lane;
    const ZO_GLOBAL W *grad = (const ZO_GLOBAL W *)t.grad + t.at + r * kBlock + 4 * lane;
    ZO_GLOBAL char *state = t.state + (t.at / kBlock + r) * kAdamBlockBytes<BITS>;
    auto any = [&](int i) { return WHOLE || (r + i) * kBlock < (int)t.n; };          // all of a wavefront's lanes: a state's blocks are whole
    auto left = [&](int i) { return (int)t.n - (r + i) * kBlock - 4 * lane; };
#pragma unroll
    for (int i = 0; i < kBlocksAhead; ++i) {
        if (!any(i)) continue;
        pw[i] = load4<WHOLE, W>(param + i * kBlock, left(i));
        gw[i] = load4<WHOLE, W>(grad + i * kBlock, left(i));
        const ZO_GLOBAL char *s = state + i * kAdamBlockBytes<BITS>;
        if constexpr (BITS == 32) {
            m32[i] = *(const ZO_GLOBAL f32x4 *)(s + 16 * lane);
            v32[i] = *(const ZO_GLOBAL f32x4 *)(s + 1024 + 16 * lane);
        } else {
            m8[i] = *(const ZO_GLOBAL uint32_t *)(s + 4 * lane);
            v8[i] = *(const ZO_GLOBAL uint32_t *)(s + 256 + 4 * lane);
            scale[i] = *(const ZO_GLOBAL f32x2 *)(s + 512);
        }
    }
#pragma unroll
    for (int i = 0; i < kBlocksAhead; ++i) {
        if (!any(i)) continue;
        float m[4], v[4], root[4], g[4];
        if constexpr (BITS == 32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) { m[e] = m32[i][e]; v[e] = v32[i][e]; }
        } else {
            from_e4m3(m8[i], scale[i].x, m);
            from_e4m3(v8[i], scale[i].y, root);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = root[e] * root[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) g[e] = coef * P::w2f(gw[i][e]);
        if (power) {
#pragma unroll
            for (int e = 0; e < 4; ++e) g[e] = ldexpf(g[e], power);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool in = WHOLE || e < left(i);               // (what lies behind a tensor's end, in its state's last block, is zeros)
            m[e] = in ? k.b1 * m[e] + k.c1 * g[e] : 0.0f;
            v[e] = in ? k.b2 * v[e] + (k.c2 * g[e]) * g[e] : 0.0f;
        }
        roots(v, root);
        u32x4 word{};
        if constexpr (SR) word = philox_block(k.seed, k.first_tensor + t.tensor, (t.at + (uint32_t)((r + i) * kBlock + 4 * lane)) / 4, 3u);
        const uint32_t words[4] = {word.x, word.y, word.z, word.w};
        F now;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float p = P::w2f(pw[i][e]), moved = p - (k.decay * p + k.rate * m[e] / (k.root * root[e] + k.eps));
            if constexpr (SR) now[e] = DT == kBF16 ? sr_to_bf16(moved, words[e]) : sr_to_f16(moved, words[e]);
            else now[e] = P::f2w(moved);
        }
        store4<WHOLE, W>(param + i * kBlock, now, left(i));
        ZO_GLOBAL char *s = state + i * kAdamBlockBytes<BITS>;
        if constexpr (BITS == 32) {
            *(ZO_GLOBAL f32x4 *)(s + 16 * lane) = f32x4{m[0], m[1], m[2], m[3]};
            *(ZO_GLOBAL f32x4 *)(s + 1024 + 16 * lane) = f32x4{v[0], v[1], v[2], v[3]};
        } else {
            float m_scale, v_scale;
            const uint32_t m_now = hold8<false>(m, m_scale), v_now = hold8<true>(root, v_scale);
            *(ZO_GLOBAL uint32_t *)(s + 4 * lane) = m_now;
            *(ZO_GLOBAL uint32_t *)(s + 256 + 4 * lane) = v_now;
            if (lane == 0) *(ZO_GLOBAL f32x2 *)(s + 512) = f32x2{m_scale, v_scale};
        }
    }
}

// One launch for up to N tensors; a chunk of 4096 elements is a workgroup's at a time, four blocks of 256 a wavefront's, whose loads are all under way
// before the first is worked (8-bit moments, below: 332 us, two blocks 336, one 345; no difference with 32 bits).  Bound by memory with 32-bit moments: 43 M bf16 weights, 22 bytes each, 187 us (5.1 TB/s; a copy runs
// at 5.0).  With 8-bit moments and words for rounding by its instructions: 10.06 bytes an element, 137 M bf16 weights 324 - 335 us (4.1 - 4.2 TB/s, 276 at the copy
// rate): some 350 a block, of which Philox's 19 multiplies take four times as long as others and division, two scales and their maxima the most of the rest.
template <int DT, int BITS, bool SR, int N>
__global__ __launch_bounds__(256) void adamw_kernel(AdamBatchOf<N> b, AdamScalars k)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // the clipping's coefficient, as an fp32 number and, where it lies beyond these, a power of two
    float coef = 1.0f;
    int power = 0;
    if (k.norm) {
        const double norm = *k.norm;
        if (!(norm - norm == 0.0)) return;                      // nothing is written
        if (norm > (double)k.max_norm) {
            coef = (float)frexp((double)k.max_norm / norm, &power);
            power = __builtin_amdgcn_readfirstlane(power);
            if (power > -120) {
                coef = ldexpf(coef, power);
                power = 0;
            }
        }
    }
    for (uint32_t c = blockIdx.x; c < b.chunks; c += gridDim.x) {
        const AdamPlace t = adam_place(b, c);
        for (int r = wave * kBlocksAhead; r < kChunkBlocks && r * kBlock < (int)t.n; r += 4 * kBlocksAhead) {
            if ((r + kBlocksAhead) * kBlock <= (int)t.n) adamw_blocks<DT, BITS, SR, true>(t, r, k, coef, power);
            else adamw_blocks<DT, BITS, SR, false>(t, r, k, coef, power);
        }
    }
}

template <int DT, int BITS, bool SR, int N>
hipError_t adamw(void *const *param, const void *const *grad, void *const *state, const uint64_t *numel, int n_tensors, AdamScalars k, hipStream_t s)
{
    // tensors of a launch: as many as its table holds, and chunk numbers of 31 bits
    AdamBatchOf<N> b{};
    int first_tensor = 0;
    auto flush = [&](int next) {
        hipError_t e = hipSuccess;
        if (b.chunks) {
            k.first_tensor = first_tensor;
            adamw_kernel<DT, BITS, SR, N><<<dim3(b.chunks < kAdamGrid ? b.chunks : kAdamGrid), dim3(256), 0, s>>>(b, k);
            e = hipGetLastError();
        }
        b.n = 0;
        b.chunks = 0;
        first_tensor = next;
        return e;
    };
    for (int i = 0; i < n_tensors; ++i) {
        const uint64_t chunks = (numel[i] + kAdamChunk - 1) / kAdamChunk;
        // (an empty tensor takes part in the numbering: the table's places are the tensors' own)
        if (b.n == N || b.chunks + chunks >= (1ull << 31)) {
            const hipError_t e = flush(i);
            if (e != hipSuccess) return e;
        }
        b.param[b.n] = (uint64_t)(uintptr_t)param[i] | (chunks ? (numel[i] - (chunks - 1) * kAdamChunk - 1) << 48 : 0);
        b.grad[b.n] = (uint64_t)(uintptr_t)grad[i];
        b.state[b.n] = (uint64_t)(uintptr_t)state[i];
        b.first[b.n++] = b.chunks;
        b.chunks += (uint32_t)chunks;
    }
    return b.chunks ? flush(n_tensors) : hipSuccess;
}

}  // namespace

hipError_t launch_adamw(void *const *param, const void *const *grad, void *const *state, const uint64_t *numel, int n_tensors, int dtype, int bits,
                        const AdamScalars &k, bool stochastic, hipStream_t s)
{
    auto go = [&](auto dt, auto b, auto sr) {
        constexpr int DT = decltype(dt)::value, BITS = decltype(b)::value;
        constexpr bool SR = decltype(sr)::value && DT != kFP32;
        auto f = n_tensors <= kAdamFew ? adamw<DT, BITS, SR, kAdamFew> : adamw<DT, BITS, SR, kAdamMax>;
        return f(param, grad, state, numel, n_tensors, k, s);
    };
    auto rounded = [&](auto dt, auto b) { return stochastic ? go(dt, b, std::true_type{}) : go(dt, b, std::false_type{}); };
    auto held = [&](auto dt) { return bits == 8 ? rounded(dt, std::integral_constant<int, 8>{}) : rounded(dt, std::integral_constant<int, 32>{}); };
    return dtype == kFP32 ? held(std::integral_constant<int, kFP32>{}) : dtype == kBF16 ? held(std::integral_constant<int, kBF16>{}) : held(std::integral_constant<int, kFP16>{});
}

}  // namespace zo
