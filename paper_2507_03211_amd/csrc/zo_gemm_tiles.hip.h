// Matrix tiles of the 16-bit products, device side: what the linear layers (zo_gemm_mfma.hip) and the products of the LM head's
// gradient (zo_gemm_grad.hip) are made of.  Every kernel computes y[i, j] = sum_k x(i, k) w(j, k) in fp32 and hands the sums to an epilogue.
#pragma once
#include "zo_device_once.h"
#include "zo_kernels.h"
#include "zo_types.hip.h"

namespace zo {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));   // native vector: arrays of it stay in registers
typedef float f32x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr int BK = 64;                      // contraction slab; k is a multiple of it

// two outputs per conversion instruction (round to nearest even, as the single one does)
template <int DT> __device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    const f32x2 pr = {lo, hi};
    if constexpr (DT == kBF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, bf16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, f16x2));
}

// How a kernel's operands lie in memory.  Plain: rows of k elements (a linear layer's activations and weights, per sign).
// Product<XK, WK>: rows at a stride of their own, or (XK, WK) with the contraction as the outer index, element (i, k) at
// [k * stride + i]; `sign` then counts shares of the contraction, each with a partial result of its own.  Shares begin
// xz / wz elements apart.  An operand with k outside is read through a buffer that ends where its memory does (x_end, w_end: addresses):
// k beyond it are zeros.  So is a w with k inside, whose rows may end inside the last slab (kRagged): the lanes whose 16 bytes lie past the
// row's w_row elements ask for what lies past the buffer.
struct Plain {
    static constexpr bool kPlain = true, kXK = false, kWK = false, kRagged = false;
    struct Arg {};
};
template <bool XK, bool WK> struct Product {
    static constexpr bool kPlain = false, kXK = XK, kWK = WK, kRagged = !WK;
    struct Arg {
        uint64_t ldx, ldw, xz, wz, x_end, w_end;
        int w_row;
        float alpha;                        // epilogue 6: factor of the result
        // epilogues 5 and 9
        const float2 *stats;                // 5: per row, logsumexp (rounded; infinity in rows that do not count) and what goes on top of the exponent
        float2 *pairs;                      // 9: per row and strip
        float *hit;                         // 9: the target's logit
        const int32_t *target;
        int rows, words, first_word;        // rows and words that exist; the first word's number
    };
};
constexpr int kMaxColumns = 1 << 24;        // 16 fp32 rows within 2^30 bytes: what an epilogue pass addresses with 32 bits

template <int DT> __device__ __forceinline__ f32x16 mfma32(const uint4 &a, const uint4 &b, const f32x16 &c)
{
    if constexpr (DT == kBF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}


// Epilogue 4 (tied LM head fused with the cross-entropy reduction): nothing of the logits is stored.  A lane
// holds TN * 16 logits of one row (4 runs of 4 consecutive columns per MFMA tile); it reduces them to a
// (maximum, sum of exp) pair, merges with the other lane half (the remaining columns of the wave's range)
// and the wave writes one pair per row and per wave-column-range (the row's maximum there is also returned); the lane that holds the target column
// stores that logit.  A last small kernel merges the pairs of a row into logsumexp - target logit.
// Argument reuse for this epilogue: bias_p -> int32 target[rows], bias_m -> float target_logit[rows],
// y -> float2 partial[rows][n_partial].
template <int TN>
__device__ __forceinline__ float ce_partial_row(f32x16 (&a)[TN], int col0, int fh, int n, bool live, int tg,
                                                float *tgt_logit_row, float2 *partial_slot)
{
    // `live` false: a row past the ragged end of the tile.  It takes part (the two halves of the wave exchange their
    // results below) and stores nothing; its pointers are those of the last valid row.
    //
    // A lane's 16 TN logits in register order k = 16 tn + i sit at columns col0 + 32 tn + 8 (i / 4) + 4 fh + i % 4,
    // which grow with k.  Nothing here keeps one compare result per element alive (64 of them, the same for every
    // row block, is what the compiler would hoist and then spill): the ragged strip of the vocabulary is masked by
    // arithmetic, the target logit is picked by a tree of selects on the bits of its register number.
    constexpr int NE = 16 * TN;
    float v[NE];
#pragma unroll
    for (int k = 0; k < NE; ++k) v[k] = a[k / 16][k % 16];
    if (col0 + 32 * TN > n) {                      // wave-uniform: only the last strip of the vocabulary
        // number of this lane's registers that lie inside the vocabulary
        int kmax = 0;
#pragma unroll
        for (int g = 0; g < 4 * TN; ++g) {         // runs of 4 columns: col0 + 32 (g / 4) + 8 (g % 4) + 4 fh + 0..3
            const int c0 = col0 + 32 * (g / 4) + 8 * (g % 4) + 4 * fh, left = n - c0;
            kmax += left < 0 ? 0 : left > 4 ? 4 : left;
        }
        const float kf = (float)kmax - 0.5f;
#pragma unroll
        for (int k = 0; k < NE; ++k) {
            // (kf - k) * inf is +inf for registers inside, -inf outside (never 0 * inf); min(., 0) makes it 0 or -inf
            const float pen = __builtin_fminf((kf - (float)k) * INFINITY, 0.0f);
            v[k] += pen;
        }
    }
#pragma unroll
    for (int k = 0; k < NE; ++k) a[k / 16][k % 16] = v[k];     // (for a caller that goes on with them: one copy in registers, not two)
    // (two maxima and four sums side by side: with one wave per SIMD an instruction that waits for the one before it issues
    // after 8 cycles instead of 5, and 64 additions in a row are half of such waits.  With the row targets loaded together, see
    // the caller: LM head of 50272 columns, us before / here: 8176 rows a sign, d 768, 1048 / 1022; 1048 rows, d 2048, 389 / 384)
    float mx2[2] = {v[0], v[1]};
#pragma unroll
    for (int k = 2; k < NE; k += 4) {
        mx2[0] = __builtin_fmaxf(__builtin_fmaxf(v[k], v[k + 1]), mx2[0]);
        if (k + 2 < NE) mx2[1] = __builtin_fmaxf(__builtin_fmaxf(v[k + 2], v[k + 3]), mx2[1]);
    }
    const float mx = __builtin_fmaxf(mx2[0], mx2[1]);
    // exp(v - mx) as 2^(v L - c), c = rn(mx L): one fma and one exponential per logit, where subtracting first and scaling
    // then takes one instruction more of some six.  c's rounding is taken out of the sum again (the fma that finds it is
    // exact), so that the pair belongs to mx itself.  That holds while 2^(c's rounding) is an fp32 number: up to |mx| = 2^30
    // half a unit of c is at most 64.  Beyond, two logits are equal or at least 64 apart, where an exponential to any base
    // from 2 up is lost in the sum, and base 2 needs no scale: c = mx, differences exact.
    // LM head of 50272 columns, before -> after in us: 8176 rows a sign, d 768, 1071 -> 1056; 2048 rows 286 -> 279; 1048
    // rows, d 2048, 391 -> 387.  Error against fp64 unchanged (rms 2.6e-7 at logits of about 1, 3.4e-6 at 8).
    // (no logit above minus infinity, as past the vocabulary, or none that is a number: the lowest number, and the sum is 0 or NaN)
    const float ms = __builtin_fmaxf(mx, -0x1.fffffep127f);
    const float L = __builtin_fabsf(ms) > 0x1p30f ? 1.0f : 1.44269504f, c = ms * L;
    float sum4[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < NE; ++k) sum4[k & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(v[k], L, -c));
    float sum = (sum4[0] + sum4[1]) + (sum4[2] + sum4[3]);
    sum *= __builtin_amdgcn_exp2f(-__builtin_fmaf(ms, L, -c));
    // the target column, if it is one of this lane's: register 16 (rel / 32) + 4 (rel / 8 % 4) + rel % 4 of the lane
    // half rel / 4 % 2
    const int rel = tg - col0;
    const bool mine = rel >= 0 && rel < 32 * TN && ((rel >> 2) & 1) == fh;
    const int which = (rel >> 5) * 16 + ((rel >> 3) & 3) * 4 + (rel & 3);
    if (__builtin_amdgcn_ballot_w64(mine) != 0) {        // of 50272 columns a wave holds 128: one wave in twelve
        float t[NE];
#pragma unroll
        for (int k = 0; k < NE; ++k) t[k] = v[k];
#pragma unroll
        for (int bit = 0, cnt = NE; cnt > 1; ++bit, cnt = (cnt + 1) / 2) {
            const bool odd = (which >> bit) & 1;
#pragma unroll
            for (int k = 0; k < (cnt + 1) / 2; ++k) t[k] = odd && 2 * k + 1 < cnt ? t[2 * k + 1] : t[2 * k];
        }
        if (live && mine) *tgt_logit_row = t[0];
    }
    const float mo = __shfl_xor(ms, 32, 64), so = __shfl_xor(sum, 32, 64);
    const float m2 = __builtin_fmaxf(ms, mo);
    const float s2 = sum * __expf(ms - m2) + so * __expf(mo - m2);
    if (live && fh == 0) *partial_slot = float2{m2, s2};
    return m2;
}

constexpr int kGroupM = 8;                      // tile-rows per band

// 16 bytes per lane from global memory straight into LDS: lane L lands at lds_off + 16 L.
// Issued from asm so that the waits are ours: the compiler would otherwise drain every
// outstanding load before the next LDS read, which defeats the overlap.
// The address is a wave-uniform 64-bit base (scalar registers: the k advance of the pipeline costs no vector
// instruction) plus a 32-bit per-lane byte offset that stays the same for the whole tile.
__device__ __forceinline__ void gload_lds16(uint64_t base, uint32_t lane_off, uint32_t lds_off)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(lane_off), "s"(base), "s"(lds_off) : "memory", "m0");
}
// The same with a buffer (four scalar registers) as the base: bytes past its end are zeros.
__device__ __forceinline__ void gload_lds16(u32x4 buffer, uint32_t lane_off, uint32_t lds_off)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(lane_off), "s"(buffer), "s"(lds_off) : "memory", "m0");
}
// What a slab that starts at `base` is read from.
template <bool BOUNDED> __device__ __forceinline__ auto slab_source(uint64_t base, uint64_t end)
{
    if constexpr (BOUNDED) {
        const uint64_t left = end > base ? end - base : 0;
        return u32x4{(uint32_t)base, (uint32_t)(base >> 32), left < 0x7fffffffu ? (uint32_t)left : 0x7fffffffu, 0x00020000u};
    } else {
        return base;
    }
}

// Tiles of an operand with k outside lie in LDS as they do in memory, [k][CH chunks of 16 bytes], and their fragments come from the
// transposing read ds_read_b64_tr_b16: in every group of 16 lanes lane j hands in the address of four elements of k row
// j / 4 and gets back four k of column j.  Chunks are XOR-swizzled by k so that the four rows of a read lie on different quarters of the 64 banks.
typedef short v4i16 __attribute__((ext_vector_type(4)));
template <int CH> __device__ __forceinline__ int k_swizzle(int k) { return CH % 16 == 0 ? (k & 3) << 2 : ((k >> 1) & 1) << 2; }
// element offset of this lane's first read of the fragment at column c0 (a multiple of 32)
template <int CH> __device__ __forceinline__ int k_offset(int c0, int lane)
{
    const int j = lane & 15, k = 8 * (lane >> 5) + (j >> 2), chunk = c0 / 8 + 2 * ((lane >> 4) & 1) + ((j & 3) >> 1);
    return (k * CH + (chunk ^ k_swizzle<CH>(k))) * 8 + 4 * (j & 1);
}
// eight k of a column: the k-step ks of the slab
template <int CH> __device__ __forceinline__ uint4 k_fragment(const uint4 *tile, int offset, int ks)
{
    typedef __attribute__((address_space(3))) v4i16 *lds;
    const uint16_t *p = (const uint16_t *)tile + offset + ks * 16 * CH * 8;
    const v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(p + 4 * CH * 8));
    const uint2 lo = __builtin_bit_cast(uint2, a), hi = __builtin_bit_cast(uint2, b);
    return uint4{lo.x, lo.y, hi.x, hi.y};
}

__device__ __forceinline__ uint64_t uniform64(uint64_t v)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return ((uint64_t)hi << 32) | lo;
}

// Tile `lin` of the list -> sign, first row, tile column.  The list runs through the signs, in each through bands of 8
// tile-rows, in a band column by column: what an XCD works on at one time shares operand slabs in its L2, and a band
// never mixes the two signs, which share no weights.
__device__ __forceinline__ void tile_at(int lin, int tiles_m, int tiles_n, int &sign, int &trow, int &tcol)
{
    const int per_sign = tiles_m * tiles_n;
    sign = lin / per_sign;
    const int in_sign = lin % per_sign, band = in_sign / (kGroupM * tiles_n), rem = in_sign % (kGroupM * tiles_n);
    const int band_rows = tiles_m - band * kGroupM < kGroupM ? tiles_m - band * kGroupM : kGroupM;
    trow = band * kGroupM + rem % band_rows;
    tcol = rem / band_rows;
}

// Epilogue 5 (the LM head's gradient): a row's logits become G = exp(l - lse) - [word is the target], times 2^15 in fp16 (probabilities
// down to 2^-29 are normal numbers there, down to 2^-39 numbers at all), to be stored as 16-bit numbers.  The exponent is (l - lse) log2(e)
// with lse in two parts, so that large logits lose nothing.  Words beyond the last one are zeros.  Registers as in ce_partial_row; one row
// block at a time (of four at once, 64 values each, a quarter spilled).
template <int DT, int TN>
__device__ __forceinline__ void gradient_row(f32x16 (&a)[TN], float2 st, int rel, int words_left, int fh)
{
    constexpr float kOne = DT == kFP16 ? 32768.0f : 1.0f;
    if (words_left < 32 * TN) {                                // wave-uniform: only the last strip of the vocabulary
        int kmax = 0;
#pragma unroll
        for (int g = 0; g < 4 * TN; ++g) {
            const int left = words_left - (32 * (g / 4) + 8 * (g % 4) + 4 * fh);
            kmax += left < 0 ? 0 : left > 4 ? 4 : left;
        }
        const float kf = (float)kmax - 0.5f;
#pragma unroll
        for (int k = 0; k < 16 * TN; ++k) a[k / 16][k % 16] += __builtin_fminf((kf - (float)k) * INFINITY, 0.0f);
    }
#pragma unroll
    for (int k = 0; k < 16 * TN; ++k) a[k / 16][k % 16] = __builtin_amdgcn_exp2f(__builtin_fmaf(a[k / 16][k % 16] - st.x, 1.44269504f, st.y));
    // rows that do not count: zeros whatever the words hold (a word that is not a number gives no number less infinity)
    const bool none = st.x == INFINITY;
    if (__builtin_amdgcn_ballot_w64(none) != 0) {
#pragma unroll
        for (int k = 0; k < 16 * TN; ++k) a[k / 16][k % 16] = none ? 0.0f : a[k / 16][k % 16];
    }
    const bool mine = rel >= 0 && rel < 32 * TN && ((rel >> 2) & 1) == fh;
    const int which = mine ? (rel >> 5) * 16 + ((rel >> 3) & 3) * 4 + (rel & 3) : -1;
    if (__builtin_amdgcn_ballot_w64(mine) != 0) {
#pragma unroll
        for (int k = 0; k < 16 * TN; ++k) a[k / 16][k % 16] -= which == k ? kOne : 0.0f;
    }
}

// Epilogues 0 - 3 and 5 - 9 of a wave's 32 TM x 32 TN outputs (rows m0 + wm 32 TM .., columns n0 + wn 32 TN .. of sign `sign`).
// 9: epilogue 4's pairs, and every logit as its distance from the pair's maximum in steps of 32 / 65535 (a distance of 32
// and more counts as none: e^-32 of the strip's largest; half a step is 2^-12 of a probability, half of fp16's own half step).
// 5: 16-bit, the values as they are; 6: 16-bit, times alpha; 7: fp32; 8: added to fp32 sums; all without bias.
// `stage`: kTileStageBytes<TN> bytes of LDS that are this wave's alone.  NT: non-temporal accesses (see launch_small).
template <int TN> constexpr int kTileStageBytes = (TN & (TN - 1)) ? 2048 * TN + 512 : 2048 * TN;
template <int DT, int EPI, int TM, int TN, bool NT, class ARG = Plain::Arg>
__device__ __forceinline__ void store_tile(const f32x16 (&acc)[TN][TM], char *stage, const uint16_t *__restrict__ bias, void *__restrict__ y,
                                           int sign, int m_half, int n, int m0, int n0, int wm, int wn, int lane, const ARG &op = {})
{
    const int fr = lane & 31, fh = lane >> 5;
    // Output through LDS so that global stores are whole rows: in the MFMA layout a lane holds runs of 4
    // consecutive columns of ONE row and a wave instruction would touch 32 rows with 16 or 32 bytes each.
    // A wave stages 2 KiB x TN at a time (32 rows of two-byte columns, or 16 rows of fp32).  No workgroup barrier.  Rows whose
    // length is a power of two are XOR-swizzled by the row: the run-wise writes and the row-wise 16-byte reads are free of
    // bank conflicts (16-bit rows of one tile apart, see chunk16 below).  Others have 16 bytes of padding, which leaves two
    // lanes per bank in the writes (15 % of the LDS cycles of a 12-slab launch of 256 x 192 tiles).
    constexpr bool kOut16 = (EPI == 0 || EPI == 1 || EPI == 5 || EPI == 6 || EPI == 9);              // 2-byte outputs; else fp32
    constexpr bool kAdd = EPI == 2 || EPI == 8, kBias = EPI < 3;
    constexpr int RP = kOut16 ? 32 : 16;                         // rows per pass
    constexpr int NPASS = 32 * TM / RP;
    constexpr int RB = (kOut16 ? 64 : 128) * TN;                 // bytes per row
    constexpr bool kXor = (TN & (TN - 1)) == 0;
    constexpr int PITCH = kXor ? RB : RB + 16;
    constexpr int NRUN = 8 * TN, LPR = RB / 16;                  // runs of 4 columns, 16-byte pieces per row
    constexpr int NIO = RP * LPR / 64;                           // pieces per lane and pass
    static_assert(RP * PITCH <= kTileStageBytes<TN>, "a pass fits the wave's staging area");
    const int ncol0 = n0 + wn * 32 * TN;
    // Bias: 2-byte outputs take it before the rounding, so per run of the MFMA layout (the same 16 runs
    // for every row block); fp32 outputs take it after the LDS pass, where a lane always holds the same
    // 4 columns.
    // They come through the scalar cache (a wave-uniform address in the constant address space: 16 bytes
    // = the 8 columns of a run pair, of which the lane half keeps its 4): a vector load here would make
    // the compiler wait for every outstanding vector memory operation, the next tile's loads included.
    float bvals[kOut16 && kBias ? TN : 1][4][4];
    if constexpr (kOut16 && kBias) {
        typedef const __attribute__((address_space(4))) u32x4 *cptr;
        const uint64_t bbase = uniform64((uint64_t)(uintptr_t)bias);
#pragma unroll
        for (int tn = 0; tn < TN; ++tn)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                int c8 = ncol0 + tn * 32 + 8 * g;               // wave-uniform; clamped: columns >= n are never stored
                c8 = c8 + 8 <= n ? c8 : n - 8;
                const u32x4 raw = *(cptr)(uintptr_t)(bbase + 2u * (uint32_t)c8);
                const uint32_t lo = fh ? raw.z : raw.x, hi = fh ? raw.w : raw.y;
                bvals[tn][g][0] = Prec<DT>::w2f((uint16_t)(lo & 0xffff));
                bvals[tn][g][1] = Prec<DT>::w2f((uint16_t)(lo >> 16));
                bvals[tn][g][2] = Prec<DT>::w2f((uint16_t)(hi & 0xffff));
                bvals[tn][g][3] = Prec<DT>::w2f((uint16_t)(hi >> 16));
            }
    }
    // Addresses: a wave-uniform base for the pass (scalar registers) plus a per-lane offset that is worked out once.  With a
    // 64-bit address and both bounds worked out per row the epilogue was 1650 (16-bit outputs) / 2980 (residual)
    // instructions per wave and 256 x 256 tile instead of 1390 / 2150.
    // 16-bit outputs: a row mask of one compare with a constant.  fp32: buffer accesses, which drop (or read as zero) what
    // lies past the pass's last row, and lanes whose columns lie past the end point behind any buffer.  With a branch
    // around each piece the compiler cannot count what is under way and lets every piece of the residual epilogue wait for
    // all memory operations before it, the stores of the piece before included: us, m_half x n x k, code with both bounds
    // per row / branches / here, residual: 8192 x 4096 x 1024 184 / 188 / 175, 2794 x 16304 x 512 193 / 205 / 185, 8192 x
    // 5120 x 5120 670 / 680 / 656.  (16-bit outputs wait for nothing here; as buffer stores they were up to 6 % slower.)
    constexpr int ES = kOut16 ? 2 : 4;
    constexpr int NBV = 64 % LPR == 0 ? 1 : 3;                   // a lane's column and row step repeat after this many pieces
    constexpr int RSTEP = 64 * NBV / LPR;                        // rows between those
    static_assert(64 * NBV % LPR == 0 && NIO % NBV == 0, "pieces repeat");
    const int row0 = m0 + wm * 32 * TM;
    const uint64_t ybase = uniform64((uint64_t)(uintptr_t)y + (((uint64_t)sign * m_half + row0) * n + ncol0) * ES);
    constexpr uint32_t kOutside = 0xc0000000u;                   // with a pass's offsets on top still below 2^32 (kMaxColumns)
    uint32_t voff[NBV];
    int rows_left[NBV];          // rows from the lane's first one to the end of the output; none where its columns lie past the end
#pragma unroll
    for (int v = 0; v < NBV; ++v) {
        const int r = (64 * v + lane) / LPR, c = (64 * v + lane) % LPR;
        const bool in = ncol0 + c * (16 / ES) < n;
        rows_left[v] = in ? m_half - row0 - r : 0;
        voff[v] = kOut16 || in ? (uint32_t)r * (uint32_t)n * ES + (uint32_t)c * 16u : kOutside;
    }
    const uint32_t step = (uint32_t)RSTEP * (uint32_t)n * ES;
    // 16-bit: piece i of the pass that starts at the wave-uniform address `at`, which moves on with every NBV pieces
    typedef __attribute__((address_space(1))) f32x4 *out4;
    auto piece = [&](uint64_t at, int i) { return (out4)((__attribute__((address_space(1))) char *)(uintptr_t)at + voff[i % NBV]); };
    auto valid = [&](int pass, int i) { return pass * RP + i / NBV * RSTEP < rows_left[i % NBV]; };
    uint64_t at_store = ybase;
    // fp32: the rows of a pass that exist, up to the last one's last column, and piece i's offset in them
    auto pass_rows = [&](int pass) {
        const int left = m_half - row0 - pass * RP, rows = left < RP ? left : RP;
        const uint32_t bytes = left > 0 && ncol0 < n ? ((uint32_t)(rows - 1) * (uint32_t)n + (uint32_t)(n - ncol0)) * ES : 0u;
        const uint64_t first = ybase + (uint64_t)pass * RP * (uint32_t)n * ES;
        return __builtin_amdgcn_make_buffer_rsrc((void *)(uintptr_t)first, 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
    };
    auto offset = [&](int i) { return voff[i % NBV] + (uint32_t)(i / NBV) * step; };
    constexpr int kPolicy = NT && kAdd ? 2 : 0;                 // of a buffer access: non-temporal or not
    // Residual epilogue: the reads of the running sum that a pass needs are all issued one pass ahead
    // (a load may not overtake an earlier store that the compiler cannot tell apart from it).  Reading
    // further ahead (two passes, which is what the registers allow) changes nothing: what the tile waits
    // for is the bandwidth of all workgroups' read-modify-write bursts arriving together, not one latency.
    f32x4 hres[2][kAdd ? NIO : 1];
    auto load_res = [&](int pass, f32x4 (&h)[kAdd ? NIO : 1]) {
        // read once, written once: neither the running sum nor any output is worth an L2 line that
        // an operand slab could keep (non-temporal loads and stores)
        const auto rows = pass_rows(pass);
#pragma unroll
        for (int i = 0; i < NIO; ++i) h[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, offset(i), 0, kPolicy));
    };
    float bias4[EPI == 2 ? NBV : 1][4] = {};
    if constexpr (kAdd) load_res(0, hres[0]);
    if constexpr (EPI == 2) {
#pragma unroll
        for (int v = 0; v < NBV; ++v) {
            const int nc = ncol0 + (64 * v + lane) % LPR * 4;
            if (nc < n) {
                const uint2 braw = *(const uint2 *)(bias + nc);
                bias4[v][0] = Prec<DT>::w2f((uint16_t)(braw.x & 0xffff));
                bias4[v][1] = Prec<DT>::w2f((uint16_t)(braw.x >> 16));
                bias4[v][2] = Prec<DT>::w2f((uint16_t)(braw.y & 0xffff));
                bias4[v][3] = Prec<DT>::w2f((uint16_t)(braw.y >> 16));
            }
        }
    }
    // 16-bit rows that are a power of two long: the chunk (two runs) is XORed by row bits, and the half within it flips with
    // row bit kFlip, a whole piece's rows at a time on the way out.  Written runs are 8 bytes of 32 rows (lanes): they spread
    // over all 64 banks, and those of 16 rows over the 32 that an access of 8 bytes a lane reaches in one go.  (TN == 1 has
    // no row bit to flip by that is one value per piece and within 16 rows: two lanes per bank there.)
    constexpr int kFlip = TN == 1 ? 4 : 3;
    auto chunk16 = [](int r) {
        return TN == 4 ? (r & 7) | ((r >> 4) & 1) << 3 : TN == 2 ? ((r >> 1) & 3) | ((r ^ (r >> 4)) & 1) << 2 : ((r >> 2) & 3);
    };
    // epilogue 5: what the lane's rows need, all at once
    float2 st[EPI == 5 ? TM : 1];
    int rel[EPI == 5 || EPI == 9 ? TM : 1];
    if constexpr (EPI == 9) {                                  // (here: the targets)
#pragma unroll
        for (int tm = 0; tm < TM; ++tm) {
            const int r = row0 + tm * 32 + fr;
            rel[tm] = op.target[r < op.rows ? r : op.rows - 1];
        }
    }
    if constexpr (EPI == 5) {
#pragma unroll
        for (int tm = 0; tm < TM; ++tm) {
            const int r = row0 + tm * 32 + fr, at = r < op.rows ? r : op.rows - 1;
            const int tg = op.target[at];
            st[tm] = op.stats[at];
            if (r >= op.rows) st[tm].x = INFINITY;
            rel[tm] = r < op.rows && tg >= 0 ? tg - op.first_word - ncol0 : -1;
        }
    }
#pragma unroll
    for (int pass = 0; pass < NPASS; ++pass) {
        const int tm = pass * RP / 32;                          // MFMA row block of this pass
        f32x16 grad[EPI == 5 || EPI == 9 ? TN : 1];
        if constexpr (EPI == 9) {
#pragma unroll
            for (int tn = 0; tn < TN; ++tn) grad[tn] = acc[tn][tm];
            const int r = row0 + tm * 32 + fr, at = r < op.rows ? r : op.rows - 1, strips = 2 * ((n + 64 * TN - 1) / (64 * TN));
            const float top = ce_partial_row<TN>(grad, ncol0, fh, op.words, r < op.rows, rel[tm], op.hit + at,
                                                 op.pairs + (size_t)at * strips + ncol0 / (32 * TN));
#pragma unroll
            for (int k = 0; k < 16 * TN; ++k) grad[k / 16][k % 16] = __builtin_fmaf(grad[k / 16][k % 16], -0x1p-5f, top * 0x1p-5f);
        }
        if constexpr (EPI == 5) {
#pragma unroll
            for (int tn = 0; tn < TN; ++tn) grad[tn] = acc[tn][tm];
            gradient_row<DT, TN>(grad, st[tm], rel[tm], op.words - ncol0, fh);
        }
        if constexpr (kAdd) {
            if (pass + 1 < NPASS) load_res(pass + 1, hres[(pass + 1) & 1]);
        }
        // fp32: the pass covers rows 16 (pass % 2) .. + 15 of the block, held by the lanes with that fr / 16
        if (kOut16 || (fr >> 4) == (pass & 1)) {
#pragma unroll
            for (int tn = 0; tn < TN; ++tn)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (EPI == 5 || EPI == 9) v[e] = grad[tn][4 * g + e];
                        else v[e] = acc[tn][tm][4 * g + e];
                        if constexpr (kOut16 && kBias) v[e] += bvals[tn][g][e];
                        if constexpr (EPI == 6) v[e] *= op.alpha;
                        if constexpr (EPI == 1) v[e] = v[e] > 0.0f ? v[e] : 0.0f;
                    }
                    const int run = tn * 8 + 2 * g + fh;         // which run of 4 columns of the row
                    if constexpr (kOut16) {
                        uint2 o;
                        if constexpr (EPI == 9) {              // 0 .. 1 to 0 .. 65535, nearest, what lies outside to the ends: one instruction for two
                            auto steps2 = [](float lo, float hi) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pknorm_u16(lo, hi)); };
                            o = uint2{steps2(v[0], v[1]), steps2(v[2], v[3])};
                        } else {
                            o = uint2{pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3])};
                        }
                        const int slot = kXor ? (((tn * 4 + g) ^ chunk16(fr)) << 1) + (fh ^ ((fr >> kFlip) & 1)) : run;
                        *(uint2 *)(stage + fr * PITCH + (slot << 3)) = o;
                    } else {
                        *(float4 *)(stage + (fr & 15) * PITCH + ((kXor ? run ^ (fr & 15 & (NRUN - 1)) : run) << 4)) = float4{v[0], v[1], v[2], v[3]};
                    }
                }
        }
        asm volatile("" ::: "memory");      // the wave's LDS operations execute in order; keep the compiler to it too
        if constexpr (kOut16) {
#pragma unroll
            for (int i = 0; i < NIO; ++i) {
                const int r = (64 * i + lane) / LPR, c = (64 * i + lane) % LPR;
                u32x4 q = *(const u32x4 *)(stage + r * PITCH + ((kXor ? c ^ chunk16(r) : c) << 4));
                if (kXor && ((i * 64 / LPR) >> kFlip & 1)) q = u32x4{q.z, q.w, q.x, q.y};
                if (valid(pass, i)) {
                    if constexpr (NT) __builtin_nontemporal_store(__builtin_bit_cast(f32x4, q), piece(at_store, i));
                    else *piece(at_store, i) = __builtin_bit_cast(f32x4, q);
                }
                if (i % NBV == NBV - 1) at_store = uniform64(at_store + step);
            }
        } else {
            const auto rows = pass_rows(pass);
#pragma unroll
            for (int i = 0; i < NIO; ++i) {
                const int r = (64 * i + lane) / LPR, c = (64 * i + lane) % LPR;
                f32x4 q = *(const f32x4 *)(stage + r * PITCH + ((kXor ? c ^ (r & (NRUN - 1)) : c) << 4));
                if constexpr (EPI == 8) {
                    const f32x4 h = hres[pass & 1][i];
                    q = f32x4{h.x + q.x, h.y + q.y, h.z + q.z, h.w + q.w};
                }
                if constexpr (EPI == 2) {
                    const f32x4 h = hres[pass & 1][i];
                    const float *b4 = bias4[i % NBV];
                    q = f32x4{h.x + (q.x + b4[0]), h.y + (q.y + b4[1]), h.z + (q.z + b4[2]), h.w + (q.w + b4[3])};
                }
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, q), rows, offset(i), 0, kPolicy);
            }
        }
        asm volatile("" ::: "memory");
    }
}

// ------------------------------------------------------------------ pipelined tiles
// What a tile shape is made of: 2 x 2 waves, each with TM x TN matrix tiles of 32 x 32; loads run A slabs ahead.
template <int TM_, int TN_, int A_> struct Shape {
    static constexpr int TM = TM_, TN = TN_, A = A_;
    static constexpr int BM = 64 * TM, BN = 64 * TN;
    static constexpr int STX = A + 1, STW = A;                   // LDS stages of the activation tile / of the weight tile
    static constexpr int XU4 = BM * (BK / 8), WU4 = BN * (BK / 8);   // uint4 per stage
    static constexpr int kLdsBytes = (STX * XU4 + STW * WU4) * 16;
    static constexpr int LX = 2 * TM, LW = 2 * TN, NM = TM * TN, R = TM + TN;   // loads per wave and slab; multiplies and fragments per quarter
    static_assert(NM % 2 == 0 && R <= NM, "the schedules below");
    // Fragment reads that have gone out before multiply j of quarter q, for the quarter after it.
    static constexpr int reads(int q, int j)
    {
        const int c = q == 3 ? j : q == 2 ? (NM >= 8 ? 2 : 4) * j : NM == 2 * R ? j / 2 : (R * j + NM - 2) / (NM - 1);
        return c > R ? R : c;
    }
    // Activation loads that have gone out before slot s of the 2 NM + NM / 2 multiplies ahead of the barrier; weight loads
    // before slot s of the NM / 2 + NM behind it.
    static constexpr int xloads(int s)
    {
        if (TM == 4 && TN == 4) return s <= 0 ? 0 : s <= 6 ? 1 : s <= 12 ? 2 : s <= 16 ? 3 : s <= 22 ? 4 : s <= 28 ? 5 : s <= 36 ? 6 : s <= 38 ? 7 : 8;
        const int P = 2 * NM + NM / 2, c = (LX * s + P - 1) / P;
        return c > LX ? LX : c;
    }
    static constexpr int wloads(int s)
    {
        const int P = NM / 2 + NM, c = (LW * s + P - 1) / P;
        return c > LW ? LW : c;
    }
    // everything goes out exactly once, and the last fragments of a slab ahead of its barrier
    static_assert(reads(0, 0) == 0 && reads(0, NM) == R && reads(2, 0) == 0 && reads(2, NM / 2) == R && reads(3, 0) == 0 && reads(3, NM) == R, "");
    static_assert(xloads(0) == 0 && xloads(2 * NM + NM / 2) == LX && wloads(0) == 0 && wloads(NM / 2 + NM) == LW, "");
};

template <int DT, int EPI, class SH, class OP = Plain>
__global__ __launch_bounds__(256) void linear_mfma_pipe_kernel(const uint16_t *__restrict__ x, const uint16_t *__restrict__ wt_p,
                                                             const uint16_t *__restrict__ wt_m, const uint16_t *__restrict__ b_p,
                                                             const uint16_t *__restrict__ b_m, void *__restrict__ y, int m_half,
                                                             int n, int k, int tiles_m, int tiles_n, int total, typename OP::Arg op)
{
    constexpr bool XK = OP::kXK, WK = OP::kWK;
    constexpr int CHX = SH::BM / 8, CHW = SH::BN / 8;           // chunks of a k row, where k lies outside
    constexpr int TM = SH::TM, TN = SH::TN, A = SH::A, BM = SH::BM, BN = SH::BN, LX = SH::LX, LW = SH::LW, NM = SH::NM;
    extern __shared__ __attribute__((aligned(16))) uint4 smem[];
    // Persistent workgroups, one per CU: the hardware deals consecutive workgroup ids round-robin to the 8 XCDs,
    // so workgroup b sits on XCD b % 8 and is that XCD's slot b / 8; it walks the XCD's contiguous share of the
    // tile list, slot, slot + slots, ...  The software pipeline does not stop between tiles: while the last two
    // slabs of a tile are multiplied the first two slabs of the next tile are already being loaded, and they land
    // during the epilogue.
    const int per_xcd = (total + 7) / 8, slots = (int)gridDim.x / 8;
    const int xcd = (int)blockIdx.x % 8, slot0 = (int)blockIdx.x / 8;
    auto tile_lin = [&](int it) {                                   // -1: no such tile
        const int sl = slot0 + slots * it, lin = xcd * per_xcd + sl;
        return (sl < per_xcd && lin < total) ? lin : -1;
    };
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;

    // Load assignment: one wave instruction moves 8 tile rows x 128 bytes (whole cache lines); wave w,
    // instruction i of n covers rows (n w + i) * 8 .. + 7; lane -> (row, 16-byte slot).  The slot holds logical
    // chunk slot ^ (row / 2 mod 8): 16 consecutive rows of one logical chunk then sit on 16 distinct
    // 16-byte positions of the 64-bank (256-byte wide) LDS, so fragment reads are conflict-free.
    const int lrow = lane >> 3, lslot = lane & 7;
    struct Tile {
        int sign, m0, n0, tcol;
        uint64_t xbase, wbase;          // first row of the tile in x / in the sign's weights (wave-uniform)
        uint32_t xg[LX], wg[LW];        // byte offsets of this lane's loads from those (clamped at ragged edges)
    };
    // rows of w that exist, and the first one of a tile at column n0 (epilogues 5 and 9: G is wider than there are words, by whole tiles too)
    const int w_rows = [&] { if constexpr (EPI == 5 || EPI == 9) return op.words; else return n; }();
    auto w_first = [&](int n0) { if constexpr (EPI == 5 || EPI == 9) return n0 < w_rows ? n0 : w_rows - 1; else return n0; };
    auto setup = [&](int lin, Tile &t) {
        int trow;
        tile_at(lin, tiles_m, tiles_n, t.sign, trow, t.tcol);
        t.m0 = trow * BM;
        t.n0 = t.tcol * BN;
        if constexpr (OP::kPlain) {
            const uint16_t *xa = x + (size_t)t.sign * m_half * k;
            const uint16_t *wt = t.sign ? wt_m : wt_p;
            t.xbase = uniform64((uint64_t)(uintptr_t)(xa + (size_t)t.m0 * k));
            t.wbase = uniform64((uint64_t)(uintptr_t)(wt + (size_t)t.n0 * k));
        } else {
            t.xbase = uniform64((uint64_t)(uintptr_t)(x + (size_t)t.sign * op.xz + (size_t)t.m0 * (XK ? 1 : op.ldx)));
            t.wbase = uniform64((uint64_t)(uintptr_t)(wt_p + (size_t)t.sign * op.wz + (size_t)w_first(t.n0) * (WK ? 1 : op.ldw)));
        }
        const uint32_t ldx = [&] { if constexpr (OP::kPlain) return (uint32_t)k; else return (uint32_t)op.ldx; }();
        const uint32_t ldw = [&] { if constexpr (OP::kPlain) return (uint32_t)k; else return (uint32_t)op.ldw; }();
#pragma unroll
        for (int i = 0; i < LX; ++i) {
            if constexpr (XK) {
                const int p = (wave * LX + i) * 64 + lane, kr = p / CHX, slot = p % CHX;
                t.xg[i] = ((uint32_t)kr * ldx + (uint32_t)(slot ^ k_swizzle<CHX>(kr)) * 8) * 2u;
            } else {
                const int row = (wave * LX + i) * 8 + lrow;
                int xr = t.m0 + row; xr = xr < m_half ? xr : m_half - 1;       // clamp: masked at the store
                t.xg[i] = ((uint32_t)(xr - t.m0) * ldx + (lslot ^ ((row >> 1) & 7)) * 8) * 2u;
            }
        }
#pragma unroll
        for (int i = 0; i < LW; ++i) {
            if constexpr (WK) {
                const int p = (wave * LW + i) * 64 + lane, kr = p / CHW, slot = p % CHW;
                t.wg[i] = ((uint32_t)kr * ldw + (uint32_t)(slot ^ k_swizzle<CHW>(kr)) * 8) * 2u;
            } else {
                const int row = (wave * LW + i) * 8 + lrow;
                int wr = t.n0 + row; wr = wr < w_rows ? wr : w_rows - 1;
                t.wg[i] = ((uint32_t)(wr - w_first(t.n0)) * ldw + (lslot ^ ((row >> 1) & 7)) * 8) * 2u;
            }
        }
    };
    // from one slab's first byte to the next one's
    auto at_x = [&](uint64_t base, int slab) {
        if constexpr (XK) return base + (uint64_t)slab * (2u * BK) * op.ldx;
        else return base + 2u * (uint32_t)(slab * BK);
    };
    auto at_w = [&](uint64_t base, int slab) {
        if constexpr (WK) return base + (uint64_t)slab * (2u * BK) * op.ldw;
        else return base + 2u * (uint32_t)(slab * BK);
    };
    auto source_x = [&](uint64_t base) { if constexpr (XK) return slab_source<true>(base, op.x_end); else return base; };
    auto source_w = [&](uint64_t base) { if constexpr (WK || OP::kRagged) return slab_source<true>(base, op.w_end); else return base; };
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4 *)smem;
    const int nk = k / BK;                              // > A (the launcher sees to it)
    // Slabs are numbered through all the tiles of this workgroup.  x slab g lives in x stage g % (A + 1), w slab g in w
    // stage g % A (after the x stages).  Kept as rotating scalars (uint4 index into smem): the stages of slabs g and
    // g + 1, and the x stage of slab g - 1, which x slab g + A will go into.
    constexpr uint32_t kXEnd = SH::STX * SH::XU4, kWEnd = kXEnd + SH::STW * SH::WU4;
    auto next_x = [](uint32_t st) { st += SH::XU4; return st == kXEnd ? 0u : st; };
    auto next_w = [](uint32_t st) { st += SH::WU4; return st == kWEnd ? kXEnd : st; };
    uint32_t xs0 = 0, xs1 = next_x(0), xfree = kXEnd - SH::XU4;
    uint32_t ws0 = kXEnd, ws1 = next_w(kXEnd);
    auto lds_x = [&](uint32_t stage) { return lds_base + stage * 16u + (uint32_t)(wave * LX) * 1024u; };   // this wave's slice
    auto lds_w = [&](uint32_t stage) { return lds_base + stage * 16u + (uint32_t)(wave * LW) * 1024u; };

    f32x16 acc[TN][TM];
    const int fr = lane & 31, fh = lane >> 5, sw = (fr >> 1) & 7;
    const int xrow = (wm * 32 * TM + fr) * 8, wrow = (wn * 32 * TN + fr) * 8;     // uint4 index of the lane's first rows
    uint4 wfa[TN], xfa[TM], wfb[TN], xfb[TM];                             // two fragment sets: one multiplies while one loads
    int xko[XK ? TM : 1], wko[WK ? TN : 1];
    if constexpr (XK) {
#pragma unroll
        for (int t = 0; t < TM; ++t) xko[t] = k_offset<CHX>(wm * 32 * TM + 32 * t, lane);
    }
    if constexpr (WK) {
#pragma unroll
        for (int t = 0; t < TN; ++t) wko[t] = k_offset<CHW>(wn * 32 * TN + 32 * t, lane);
    }
    // One fragment of set (wf, xf) for k-step ks of the slab in stages (xst, wst), in the order the multiplies need them:
    // wf0, xf0 .. , wf1 ..
    auto frag1 = [&](uint32_t xst, uint32_t wst, int ks, int idx, uint4 (&wf)[TN], uint4 (&xf)[TM]) {
        const uint4 *xs = smem + xst;
        const uint4 *ws = smem + wst;
        const int slot = (2 * ks + fh) ^ sw;
        const bool is_x = idx >= 1 && idx <= TM;
        const int t = idx == 0 ? 0 : is_x ? idx - 1 : idx - TM;
        if (is_x) {
            if constexpr (XK) xf[t] = k_fragment<CHX>(xs, xko[t], ks);
            else xf[t] = xs[xrow + t * 256 + slot];
        } else {
            if constexpr (WK) wf[t] = k_fragment<CHW>(ws, wko[t], ks);
            else wf[t] = ws[wrow + t * 256 + slot];
        }
    };
    // ragged rows of w: what a lane's offsets get in the slab being loaded (a row's chunks are swizzled by two patterns, by the load's parity)
    uint32_t w_past[2] = {0, 0};
    auto ragged_slab = [&](bool last) {
        if constexpr (OP::kRagged) {
#pragma unroll
            for (int q = 0; q < 2; ++q) w_past[q] = last && (nk - 1) * BK + (lslot ^ (4 * q + (lrow >> 1))) * 8 >= op.w_row ? 0x80000000u : 0u;
        }
    };
    // Multiplies j0 .. j1-1 of the TM x TN fragment product of set (wf, xf), quarter q of the slab.  Before multiply j go
    // out: the fragment reads that SH::reads has due there, of set (nwf, nxf) for k-step nks of the slab in stages (nxst,
    // nwst); the global->LDS load that SH::xloads / SH::wloads has due at slot s0 + j, into LDS at `st`.
    //  `first`: the product starts the accumulators (first quarter of a tile's first slab) instead of adding to them.
    auto mma_rl = [&](const uint4 (&wf)[TN], const uint4 (&xf)[TM], int q, int j0, int j1, uint4 (&nwf)[TN], uint4 (&nxf)[TM],
                      uint32_t nxst, uint32_t nwst, int nks, const auto &offs, const auto &gbase, uint32_t st, bool is_x, int s0,
                      bool first = false) {
#pragma unroll
        for (int j = j0; j < j1; ++j) {
            const int r0 = SH::reads(q, j), r1 = SH::reads(q, j + 1);
            if (r1 > r0) {
#pragma unroll
                for (int r = r0; r < r1; ++r) frag1(nxst, nwst, nks, r, nwf, nxf);
                __builtin_amdgcn_sched_barrier(0);
            }
            const int l0 = is_x ? SH::xloads(s0 + j) : SH::wloads(s0 + j), l1 = is_x ? SH::xloads(s0 + j + 1) : SH::wloads(s0 + j + 1);
            if (l1 > l0) {
#pragma unroll
                for (int l = l0; l < l1; ++l) {
                    if (OP::kRagged && !is_x) gload_lds16(gbase, offs[l] | w_past[l & 1], st + l * 1024u);
                    else gload_lds16(gbase, offs[l], st + l * 1024u);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // back and forth over the activation fragments, so that one operand changes from one multiply to
            // the next, not both (a little less switching on a chip whose clock is set by its power)
            const int wi = j / TM, xi = (wi & 1) ? TM - 1 - j % TM : j % TM;
            if (first) {
                f32x16 zero;
#pragma unroll
                for (int i = 0; i < 16; ++i) zero[i] = 0.0f;
                acc[wi][xi] = mfma32<DT>(wf[wi], xf[xi], zero);
            } else {
                acc[wi][xi] = mfma32<DT>(wf[wi], xf[xi], acc[wi][xi]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Software pipeline (in brackets: the 256 x 256 tile).  The LDS holds A + 1 [3] stages of the activation tile and A [2]
    // of the weight tile, so the activation half of every slab's loads is issued A slab-times ahead and the weight half
    // nearly so: with a single slab of lookahead for everything the multiplies wait on memory latency.  One wave per SIMD
    // means nothing else hides an instruction that is slow to issue, so neither the global->LDS loads nor the
    // LDS fragment reads come in bursts: each sits alone between two multiplies and issues while the matrix
    // pipe works on the one before.  The fragments of a quarter slab (TM TN [16] multiplies) are read during the quarter
    // before it, into the set of registers the quarter before that used.  The barrier sits in the middle of
    // the third quarter, once this wave's last LDS reads of slab g are in registers.
    // sched_barrier(0) pins the order (the compiler would sink each LDS read down to its first use).
    //
    // One slab: multiplies slab g (fragment set A holds its first quarter), loads slab g + A from (xb, wb) with
    // the lane offsets (xo, wo).  x(g+A) goes into the activation stage that slab g-1 left at the previous barrier:
    // its loads sit under the multiplies before this slab's barrier; w(g+A) can only follow the barrier: its
    // loads sit under the multiplies after it.
    auto slab = [&](uint64_t xat, uint64_t wat, const uint32_t (&xo)[LX], const uint32_t (&wo)[LW], bool first, bool last = false) {
        ragged_slab(last);
        const auto xb = source_x(xat);
        const auto wb = source_w(wat);
        const uint32_t stx = lds_x(xfree), stw = lds_w(ws0);
        constexpr int NB = NM / 2;
        mma_rl(wfa, xfa, 0, 0, NM, wfb, xfb, xs0, ws0, 1, xo, xb, stx, true, 0, first);
        mma_rl(wfb, xfb, 1, 0, NM, wfa, xfa, xs0, ws0, 2, xo, xb, stx, true, NM);
        // the last fragments of slab g, several reads at a time, so that they have landed when the barrier's wait comes
        mma_rl(wfa, xfa, 2, 0, NB, wfb, xfb, xs0, ws0, 3, xo, xb, stx, true, 2 * NM);
        // slab g+1 landed (what was loaded after it may still be out); slab g fully in registers
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((A - 1) * LX + (A - 2) * LW) : "memory");
        __builtin_amdgcn_s_barrier();
        mma_rl(wfa, xfa, 2, NB, NM, wfb, xfb, xs0, ws0, 3, wo, wb, stw, false, -NB);
        // the first fragments of slab g+1 early in the quarter: the loop's back edge waits for all LDS reads
        mma_rl(wfb, xfb, 3, 0, NM, wfa, xfa, xs1, ws1, 0, wo, wb, stw, false, NM - NB);
        if constexpr (A == 2) {                 // three and two stages: moves alone
            const uint32_t tx = xfree, tw = ws0;
            xfree = xs0; xs0 = xs1; xs1 = tx;
            ws0 = ws1; ws1 = tw;
        } else {
            xfree = xs0;
            xs0 = xs1; xs1 = next_x(xs1);
            ws0 = ws1; ws1 = next_w(ws1);
        }
    };

    Tile cur, nxt;
    int lin = tile_lin(0);
    if (lin < 0) return;
    setup(lin, cur);
    int it = 0;                                         // tile number of this workgroup
    // prologue of the first tile only: slabs 0 .. A - 1, fragments of the first quarter
    {
        uint32_t px = xs0, pw = ws0;
#pragma unroll
        for (int g = 0; g < A; ++g) {
#pragma unroll
            for (int i = 0; i < LX; ++i) gload_lds16(source_x(at_x(cur.xbase, g)), cur.xg[i], lds_x(px) + i * 1024u);
#pragma unroll
            for (int i = 0; i < LW; ++i) gload_lds16(source_w(at_w(cur.wbase, g)), cur.wg[i], lds_w(pw) + i * 1024u);
            px = next_x(px); pw = next_w(pw);
        }
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((A - 1) * (LX + LW)) : "memory");               // slab 0 landed
    __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int idx = 0; idx < SH::R; ++idx) frag1(xs0, ws0, 0, idx, wfa, xfa);

    for (;;) {
        const int lin_next = tile_lin(it + 1);
        const bool has_next = lin_next >= 0;
        if (has_next) {
            setup(lin_next, nxt);
        } else {
            // no successor: the A slabs loaded ahead are this tile's last over again, which nothing reads
            nxt = cur;
            nxt.xbase = at_x(nxt.xbase, nk - A);
            nxt.wbase = at_w(nxt.wbase, nk - A);
        }
        // all slabs but the last A load A slabs ahead in this tile; the first one starts the accumulators
        slab(at_x(cur.xbase, A), at_w(cur.wbase, A), cur.xg, cur.wg, true, A == nk - 1);
        for (int kt = 1; kt < nk - A; ++kt)
            slab(at_x(cur.xbase, kt + A), at_w(cur.wbase, kt + A), cur.xg, cur.wg, false, kt + A == nk - 1);
        // the last A load the first A slabs of the next tile
#pragma unroll
        for (int g = 0; g < A; ++g)
            slab(at_x(nxt.xbase, g), at_w(nxt.wbase, g), nxt.xg, nxt.wg, false);

        // ---- epilogue of tile `cur`
        const int sign = cur.sign, m0 = cur.m0, n0 = cur.n0;
        const uint16_t *bias = sign ? b_m : b_p;
        if constexpr (EPI == 4) {
            const int n_partial = 2 * tiles_n;
            // the rows' targets all at once: one by one, each would wait for its load and for the stores of the row block before
            int target[TM];
#pragma unroll
            for (int tm = 0; tm < TM; ++tm) {
                const int mr = m0 + wm * 32 * TM + tm * 32 + fr;
                target[tm] = ((const int32_t *)b_p)[(size_t)sign * m_half + (mr < m_half ? mr : m_half - 1)];
            }
#pragma unroll
            for (int tm = 0; tm < TM; ++tm) asm volatile("" : "+v"(target[tm]));
#pragma unroll
            for (int tm = 0; tm < TM; ++tm) {
                const int mr = m0 + wm * 32 * TM + tm * 32 + fr;
                const size_t row = (size_t)sign * m_half + (mr < m_half ? mr : m_half - 1);
                f32x16 a[TN];
#pragma unroll
                for (int t = 0; t < TN; ++t) a[t] = acc[t][tm];
                ce_partial_row<TN>(a, n0 + wn * 32 * TN, fh, n, mr < m_half, target[tm], (float *)b_m + row, (float2 *)y + row * n_partial + (cur.tcol * 2 + wn));
            }
        } else {
            // staged in the wave's own slice of the activation stage that the tile's last slab has just left (every wave
            // finished reading that stage before the slab's barrier, and the next loads into the slice are this wave's
            // own, issued after the epilogue)
            static_assert(kTileStageBytes<TN> <= 1024 * LX, "a pass fits the slice");
            char *stage = (char *)(smem + xfree) + wave * (1024 * LX);
            // (G is read again at once)
            store_tile<DT, EPI, TM, TN, EPI != 5 && EPI != 9>(acc, stage, bias, y, sign, m_half, n, m0, n0, wm, wn, lane, op);
        }
        if (!has_next) break;
        cur = nxt;
        ++it;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                 // the tail loads land before LDS is released
}


// ------------------------------------------------------------------ small tiles
// One output tile of 64 x (64 TN) per workgroup of 2 x 2 waves, each with 1 x TN matrix tiles; slabs of 64 k through a ring
// of up to ST LDS stages, one barrier per slab, and a second workgroup on the CU to work while this one waits.  For shapes
// with few tiles: a slab of a larger tile is loaded at about 58 bytes a nanosecond and CU whatever the shape (what the
// in-order return of loads that partly miss the L2 allows), so the more CUs take part, the sooner the operands are in.
// m_half 160, n 2560, k 10240: 155 us on 128 x 128 register-staged tiles, 95 on pipelined 128 x 128, 50 here (240 CUs).
constexpr int kSmallStages = 4;
template <int TN> constexpr int kSmallStageBytes = (64 + 64 * TN) * BK * 2;
template <int DT, int EPI, int TN, bool NT, class OP, int ST>
__device__ __forceinline__ void small_tile(
    const uint16_t *__restrict__ x, const uint16_t *__restrict__ wt_p, const uint16_t *__restrict__ wt_m, const uint16_t *__restrict__ b_p,
    const uint16_t *__restrict__ b_m, void *__restrict__ y, int m_half, int n, int k, int tiles_m, int tiles_n, int total, const typename OP::Arg &op,
    int block)
{
    constexpr bool XK = OP::kXK, WK = OP::kWK;
    constexpr int CHX = 8, CHW = 8 * TN;                        // chunks of a k row, where k lies outside
    constexpr int BM = 64, BN = 64 * TN, LX = 2, LW = 2 * TN, L = LX + LW, CPR = BK / 8;
    constexpr uint32_t kStageBytes = kSmallStageBytes<TN>;
    extern __shared__ __attribute__((aligned(16))) uint4 smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const int fr = lane & 31, fh = lane >> 5;

    // consecutive workgroup ids go round-robin to the 8 XCDs; each takes a contiguous share of the tile list
    const int per_xcd = (total + 7) / 8;
    const int lin = (block & 7) * per_xcd + (block >> 3);
    if ((block >> 3) >= per_xcd || lin >= total) return;
    int sign, trow, tcol;
    tile_at(lin, tiles_m, tiles_n, sign, trow, tcol);
    const int m0 = trow * BM, n0 = tcol * BN;
    uint64_t xbase, wbase;
    const int w_rows = [&] { if constexpr (EPI == 5 || EPI == 9) return op.words; else return n; }();      // as in the kernel above
    const int w_first = (EPI == 5 || EPI == 9) && n0 >= w_rows ? w_rows - 1 : n0;
    if constexpr (OP::kPlain) {
        xbase = uniform64((uint64_t)(uintptr_t)(x + ((size_t)sign * m_half + m0) * k));
        wbase = uniform64((uint64_t)(uintptr_t)((sign ? wt_m : wt_p) + (size_t)n0 * k));
    } else {
        xbase = uniform64((uint64_t)(uintptr_t)(x + (size_t)sign * op.xz + (size_t)m0 * (XK ? 1 : op.ldx)));
        wbase = uniform64((uint64_t)(uintptr_t)(wt_p + (size_t)sign * op.wz + (size_t)w_first * (WK ? 1 : op.ldw)));
    }
    const uint32_t ldx = [&] { if constexpr (OP::kPlain) return (uint32_t)k; else return (uint32_t)op.ldx; }();
    const uint32_t ldw = [&] { if constexpr (OP::kPlain) return (uint32_t)k; else return (uint32_t)op.ldw; }();

    // one wave instruction loads 8 tile rows of 128 bytes; chunk c of row r sits at slot c ^ (r / 2 mod 8)
    auto swz = [](int r) { return (r >> 1) & 7; };
    uint32_t off[L];                            // LX loads of x, LW of w
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int row = (i < LX ? wave * LX + i : wave * LW + i - LX) * 8 + (lane >> 3);
        const int first = i < LX ? m0 : w_first, end = i < LX ? m_half : w_rows;
        int r = first + row; r = r < end ? r : end - 1;                      // clamped: never stored
        off[i] = ((uint32_t)(r - first) * (i < LX ? ldx : ldw) + ((lane & 7) ^ swz(row)) * 8) * 2u;
        if (i < LX ? XK : WK) {
            const int CH = i < LX ? CHX : CHW, p = (i < LX ? wave * LX + i : wave * LW + i - LX) * 64 + lane, kr = p / CH;
            off[i] = ((uint32_t)kr * (i < LX ? ldx : ldw) + (uint32_t)((p % CH) ^ (i < LX ? k_swizzle<CHX>(kr) : k_swizzle<CHW>(kr))) * 8) * 2u;
        }
    }
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4 *)smem;
    // a load of w's whose 16 bytes lie past the end of a ragged row
    auto past = [&](int slab, int i) {
        if constexpr (OP::kRagged) return slab * BK + (int)((lane & 7) ^ swz((wave * LW + i - LX) * 8 + (lane >> 3))) * 8 >= op.w_row;
        else return false;
    };
    auto load_slab = [&](int slab, uint32_t stage) {
        const uint32_t st = lds_base + stage * kStageBytes, adv = (uint32_t)slab * (BK * 2);
        const auto xs = [&] { if constexpr (XK) return slab_source<true>(xbase + (uint64_t)adv * op.ldx, op.x_end); else return xbase + adv; }();
        const auto ws = [&] {
            if constexpr (WK) return slab_source<true>(wbase + (uint64_t)adv * op.ldw, op.w_end);
            else if constexpr (OP::kRagged) return slab_source<true>(wbase + adv, op.w_end);
            else return wbase + adv;
        }();
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (i < LX) gload_lds16(xs, off[i], st + (uint32_t)(wave * LX + i) * 1024u);
            else gload_lds16(ws, past(slab, i) ? off[i] | 0x80000000u : off[i], st + (uint32_t)(BM / 8 + wave * LW + i - LX) * 1024u);
        }
    };

    f32x16 acc[TN][1] = {};
    const int xrow = (wm * 32 + fr) * CPR, wrow = (BM + wn * 32 * TN + fr) * CPR;
    int wko[WK ? TN : 1];
    if constexpr (WK) {
#pragma unroll
        for (int t = 0; t < TN; ++t) wko[t] = k_offset<CHW>(wn * 32 * TN + 32 * t, lane);
    }
    const int xko = XK ? k_offset<CHX>(wm * 32, lane) : 0;
    auto mult_slab = [&](uint32_t stage) {
        const uint4 *st = smem + stage * (kStageBytes / 16);
#pragma unroll
        for (int ks = 0; ks < BK / 16; ++ks) {
            const int slot = (2 * ks + fh) ^ swz(fr);
            uint4 wf[TN];
            uint4 xf;
            if constexpr (XK) xf = k_fragment<CHX>(st, xko, ks);
            else xf = st[xrow + slot];
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                if constexpr (WK) wf[t] = k_fragment<CHW>(st + BM * CPR, wko[t], ks);
                else wf[t] = st[wrow + t * 32 * CPR + slot];
            }
#pragma unroll
            for (int t = 0; t < TN; ++t) acc[t][0] = mfma32<DT>(wf[t], xf, acc[t][0]);
        }
    };
    const int nk = k / BK;
#pragma unroll
    for (int s = 0; s < ST - 1; ++s)
        if (s < nk) load_slab(s, s);
    uint32_t rd = 0, wr = ST - 1;
    int kt = 0;
    for (; kt < nk - (ST - 2); ++kt) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((ST - 2) * L) : "memory");   // slab kt landed (this wave's part)
        __builtin_amdgcn_s_barrier();
        if (kt + ST - 1 < nk) load_slab(kt + ST - 1, wr);
        mult_slab(rd);
        rd = rd + 1 == ST ? 0 : rd + 1;
        wr = wr + 1 == ST ? 0 : wr + 1;
    }
    for (; kt < nk; ++kt) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        mult_slab(rd);
        rd = rd + 1 == ST ? 0 : rd + 1;
    }

    // ---- epilogue
    if constexpr (EPI == 4) {
        const int n_partial = 2 * tiles_n, mr = m0 + wm * 32 + fr;
        const size_t row = (size_t)sign * m_half + (mr < m_half ? mr : m_half - 1);
        f32x16 a[TN];
#pragma unroll
        for (int t = 0; t < TN; ++t) a[t] = acc[t][0];
        ce_partial_row<TN>(a, n0 + wn * 32 * TN, fh, n, mr < m_half, ((const int32_t *)b_p)[row], (float *)b_m + row,
                           (float2 *)y + row * n_partial + (tcol * 2 + wn));
    } else {
        static_assert(4 * kTileStageBytes<TN> <= (int)kStageBytes, "the staging areas fit the ring, of one stage at least");
        __syncthreads();                                          // every wave is done with the ring
        store_tile<DT, EPI, 1, TN, NT>(acc, (char *)smem + wave * kTileStageBytes<TN>, sign ? b_m : b_p, y, sign, m_half, n, m0, n0, wm, wn, lane, op);
    }
}
template <int DT, int EPI, int TN, bool NT, class OP = Plain>
__global__ __launch_bounds__(256, 2) void linear_mfma_small_kernel(
    const uint16_t *__restrict__ x, const uint16_t *__restrict__ wt_p, const uint16_t *__restrict__ wt_m, const uint16_t *__restrict__ b_p,
    const uint16_t *__restrict__ b_m, void *__restrict__ y, int m_half, int n, int k, int tiles_m, int tiles_n, int total, typename OP::Arg op)
{
    small_tile<DT, EPI, TN, NT, OP, kSmallStages>(x, wt_p, wt_m, b_p, b_m, y, m_half, n, k, tiles_m, tiles_n, total, op, (int)blockIdx.x);
}

// ------------------------------------------------------------------ launchers
// CUs of the current device, rounded down to whole XCDs' worth; 0 when the runtime does not say
inline int cu_count()
{
    static int n_cu = 0;
    if (n_cu == 0) {
        int dev = 0, v = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
        n_cu = v >= 8 ? v / 8 * 8 : 8;
    }
    return n_cu;
}

struct Args {
    const void *x, *wt_p, *wt_m, *b_p, *b_m;
    void *y;
    int n_sign, m_half, n, k;
    hipStream_t s;
};

template <int DT, int EPI, class SH, class OP = Plain> hipError_t launch_pipe(const Args &a, const typename OP::Arg &op = {})
{
    const int tiles_m = (a.m_half + SH::BM - 1) / SH::BM, tiles_n = (a.n + SH::BN - 1) / SH::BN;
    const int total = a.n_sign * tiles_m * tiles_n, n_cu = cu_count();
    if (n_cu == 0 || a.k / BK <= SH::A) return hipErrorInvalidValue;
    // persistent workgroups: one per CU (their LDS allows no second one), a multiple of the 8 XCDs
    const int want = (total + 7) / 8 * 8;
    const dim3 grid(want < n_cu ? want : n_cu), block(256);
    auto kern = linear_mfma_pipe_kernel<DT, EPI, SH, OP>;
    static std::atomic<uint64_t> lds_allowed{0};
    const hipError_t e = once_per_device(lds_allowed, [&] {
        return hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, SH::kLdsBytes);
    });
    if (e != hipSuccess) return e;
    kern<<<grid, block, SH::kLdsBytes, a.s>>>((const uint16_t *)a.x, (const uint16_t *)a.wt_p, (const uint16_t *)a.wt_m, (const uint16_t *)a.b_p,
                                                   (const uint16_t *)a.b_m, a.y, a.m_half, a.n, a.k, tiles_m, tiles_n, total, op);
    return hipGetLastError();
}
template <int DT, int EPI, int TN, bool NT, class OP = Plain> hipError_t launch_small_t(const Args &a, const typename OP::Arg &op = {})
{
    const int tiles_m = (a.m_half + 63) / 64, tiles_n = (a.n + 64 * TN - 1) / (64 * TN), total = a.n_sign * tiles_m * tiles_n;
    auto kern = linear_mfma_small_kernel<DT, EPI, TN, NT, OP>;
    static std::atomic<uint64_t> lds_allowed{0};
    const hipError_t e = once_per_device(lds_allowed, [&] {
        return hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kSmallStages * kSmallStageBytes<TN>);
    });
    if (e != hipSuccess) return e;
    // no more stages than there are slabs: with one or two, 8 or 5 workgroups fit a CU instead of 2, and what such a shape
    // takes is the workgroups' latency (both signs 6217 x 6320 x 64, 16-bit outputs: 70 -> 41 us)
    const int stages = a.k / BK < kSmallStages ? a.k / BK : kSmallStages;
    kern<<<dim3((total + 7) / 8 * 8), dim3(256), stages * kSmallStageBytes<TN>, a.s>>>((const uint16_t *)a.x, (const uint16_t *)a.wt_p,
                                                                                       (const uint16_t *)a.wt_m, (const uint16_t *)a.b_p,
                                                                                       (const uint16_t *)a.b_m, a.y, a.m_half, a.n, a.k,
                                                                                       tiles_m, tiles_n, total, op);
    return hipGetLastError();
}

enum Tile { T256x256, T256x192, T256x128, T192x128, T128x128, T64x64, T32x32, kTiles };
constexpr int kTileRows[kTiles] = {256, 256, 256, 192, 128, 64, 32}, kTileColumns[kTiles] = {256, 192, 128, 128, 128, 64, 32};

}  // namespace
}  // namespace zo
