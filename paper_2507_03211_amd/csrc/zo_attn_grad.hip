// Backward pass of the causal multi-head attention.  With P = softmax(q k^T / sqrt(d_head)) over the keys a query sees, and per query
// D = sum_c dO O (which is sum_k P dP):
//
//   dV = P^T dO,   dP = dO V^T,   dS = P (dP - D),   dQ = dS K / sqrt(d_head),   dK = dS^T Q / sqrt(d_head)
//
// Matrix path (16-bit types, heads of 64, 80, 96, 112, 128), three launches:
//   rows     D, and in fp16 what bounds dS (below)
//   queries  a wavefront's 32 queries against the keys they see: S, dP, dQ.  The softmax runs along (one pass, a reference that is raised
//            as scores pass it), so that logsumexp comes out at the end, for the third launch
//   keys     a wavefront's 32 keys against the queries that see them: S, dP, dV, dK
// Seven products instead of five: with dQ from the launch over the keys it would take sums of other workgroups', in memory and in an order
// that changes.  Both are computed so that a lane owns a column of the scores (a query there, a key here), and the contraction of the second
// products follows the accumulators' layout of the first, so P and dS never leave registers: rows 16 s + 4 h + {0..3}, 16 s + 8 + 4 h + {0..3}
// for lane half h, with which the transposing LDS read fetches the other operand too.
// Anything else: a workgroup per query, then per key, in the activations' own precision.
#include "zo_kernels.h"
#include "zo_types.hip.h"

namespace zo {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace {

template <int DT> __device__ __forceinline__ f32x16 mfma32(const uint4 &a, const uint4 &b, const f32x16 &c)
{
    if constexpr (DT == kBF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <int DT> __device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const f32x2 v = {a, b};
    if constexpr (DT == kBF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}
// a value of this lane's and of the one 32 places away, in an order that sum and maximum do not care for
__device__ __forceinline__ void swap_halves(float x, float &a, float &b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}

constexpr int kOwn = 128, kTile = 64;      // rows of a workgroup's own (32 a wavefront), rows of a tile that streams through LDS

// fp16: dS = P (dP - D) may lie anywhere: |dP| and |D| are at most A B, with A the largest norm of a row of dO and B of a row of V in the
// sequence and head, so 2^e dS with 2^e = 2^14 / (2 A B) rounded down is within the type whatever P is, and numbers 2^28 below that bound are still
// normal ones.  2^-e is taken out of the fp32 sums.  bf16 has fp32's range: e = 0.
struct RowTops { float out2, value2; };                         // of 64 rows: the largest |dO|^2 and |V|^2
__device__ __forceinline__ int scale_exponent(const RowTops *tops, int tiles)
{
    float a = 0.0f, b = 0.0f;
    for (int t = threadIdx.x & 63; t < tiles; t += 64) {
        a = tops[t].out2 > a ? tops[t].out2 : a;
        b = tops[t].value2 > b ? tops[t].value2 : b;
    }
    const float ab = __builtin_sqrtf(wave_max(a)) * __builtin_sqrtf(wave_max(b));
    // (nothing to scale, or nothing that scaling saves)
    return ab > 0.0f && ab < 0x1p100f ? 12 - (int)((__float_as_uint(ab) >> 23) & 0xff) + 127 : 0;
}

// D of 64 rows of one head of one sequence; 16 lanes a row and head (8 where it has 8 pieces of 16 bytes).
template <int DT, int DH>
__global__ __launch_bounds__(256) void attn_grad_rows_kernel(const uint16_t *__restrict__ qkv, const uint16_t *__restrict__ out, const uint16_t *__restrict__ dout,
                                                             float *__restrict__ delta, RowTops *__restrict__ tops, int seq, int n_heads, int tiles)
{
    constexpr int PIECES = DH / 8, LANES = PIECES <= 8 ? 8 : 16, ROWS = 256 / LANES;
    __shared__ float top[2][4];
    const int tile = (int)blockIdx.x % tiles, pair = (int)blockIdx.x / tiles, s = pair / n_heads, head = pair % n_heads, d = n_heads * DH;
    const int piece = threadIdx.x % LANES;
    float most_out = 0.0f, most_value = 0.0f;
    for (int r0 = 0; r0 < kTile; r0 += ROWS) {
        const int r = tile * kTile + r0 + (int)threadIdx.x / LANES;
        const bool live = r < seq && piece < PIECES;
        const size_t row = (size_t)s * seq + (r < seq ? r : 0), at = row * d + head * DH + (piece < PIECES ? 8 * piece : 0);
        const uint4 zero{0, 0, 0, 0};
        const uint4 o = live ? *(const uint4 *)(out + at) : zero, g = live ? *(const uint4 *)(dout + at) : zero;
        const uint4 v = live && DT == kFP16 ? *(const uint4 *)(qkv + at + row * 2 * d + 2 * d) : zero;
        float sum = 0.0f, out2 = 0.0f, value2 = 0.0f;
        auto two = [&](uint32_t a, uint32_t b, uint32_t c) {
#pragma unroll
            for (int e = 0; e < 32; e += 16) {
                const float fa = Prec<DT>::a2acc((uint16_t)(a >> e)), fb = Prec<DT>::a2acc((uint16_t)(b >> e));
                sum = __builtin_fmaf(fa, fb, sum);
                if constexpr (DT == kFP16) {
                    const float fc = Prec<DT>::a2acc((uint16_t)(c >> e));
                    out2 = __builtin_fmaf(fb, fb, out2);
                    value2 = __builtin_fmaf(fc, fc, value2);
                }
            }
        };
        two(o.x, g.x, v.x); two(o.y, g.y, v.y); two(o.z, g.z, v.z); two(o.w, g.w, v.w);
#pragma unroll
        for (int m = LANES / 2; m > 0; m >>= 1) {
            sum += __shfl_xor(sum, m, 64);
            if constexpr (DT == kFP16) {
                out2 += __shfl_xor(out2, m, 64);
                value2 += __shfl_xor(value2, m, 64);
            }
        }
        if (piece == 0 && r < seq) delta[(size_t)pair * seq + r] = sum;
        if constexpr (DT == kFP16) {
            most_out = out2 > most_out ? out2 : most_out;
            most_value = value2 > most_value ? value2 : most_value;
        }
    }
    if constexpr (DT == kFP16) {
        most_out = wave_max(most_out);
        most_value = wave_max(most_value);
        if ((threadIdx.x & 63) == 0) { top[0][threadIdx.x >> 6] = most_out; top[1][threadIdx.x >> 6] = most_value; }
        __syncthreads();
        if (threadIdx.x == 0) {
            RowTops t{};
            for (int w = 0; w < 4; ++w) {
                t.out2 = top[0][w] > t.out2 ? top[0][w] : t.out2;
                t.value2 = top[1][w] > t.value2 ? top[1][w] : t.value2;
            }
            tops[blockIdx.x] = t;
        }
    }
}

// Tiles of 64 rows in LDS, [row][piece of 16 bytes]: read by rows (32 rows, one piece: an operand with its contraction over the channels) and, by the
// transposing read, by columns (4 rows x 32 bytes per 16 lanes: one with its contraction over the rows).  Pieces are XOR-swizzled by the row so that
// both are free of bank conflicts: 16 rows of one piece lie on 16 distinct 16-byte places of the 256-byte bank line, four rows on its
// four quarters.  Rows are padded to 192 or 256 bytes (80 and 112 channels); what lies there is a piece over again, for channels that are not stored.
template <int DH> struct TileShape {
    static constexpr int CHD = DH / 8, CH = DH == 64 ? 8 : DH <= 96 ? 12 : 16, KS = DH / 16, CT = (DH + 31) / 32, PIECES = kTile * CH;
    static __device__ __forceinline__ int swizzle(int r) { return CH == 16 ? (r & 3) << 2 | ((r >> 2) & 3) : CH == 12 ? (r >> 2) & 3 : ((r >> 1) & 1) << 2 | ((r >> 2) & 3); }
    static constexpr int in_row(int piece) { return piece < CHD ? piece : piece - 2; }
};
template <int DH> struct TileReader : TileShape<DH> {
    using T = TileShape<DH>;
    int row[T::KS], column[T::CT][2];       // u32x4 index of (row lane % 32, k-step s); element offset of a column fragment, row base 0 or 8 mod 16
    __device__ __forceinline__ TileReader(int lane)
    {
        const int fr = lane & 31, fh = lane >> 5, j = lane & 15;
#pragma unroll
        for (int s = 0; s < T::KS; ++s) row[s] = fr * T::CH + ((2 * s + fh) ^ T::swizzle(fr));
#pragma unroll
        for (int c = 0; c < T::CT; ++c)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int r = 8 * b + 4 * fh + (j >> 2), chan = c * 32 + 16 * ((lane >> 4) & 1) + 4 * (j & 3);
                column[c][b] = (r * T::CH + ((chan >> 3) ^ T::swizzle(r))) * 8 + (chan & 7);
            }
    }
    // rows half * 32 + lane % 32, channels of k-step s
    __device__ __forceinline__ uint4 by_row(const u32x4 *tile, int half, int s) const { return __builtin_bit_cast(uint4, tile[half * 32 * T::CH + row[s]]); }
    // channels of tile c, rows first + {4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3}, first a multiple of 16
    __device__ __forceinline__ uint4 by_column(const u32x4 *tile, int first, int c) const
    {
        typedef __attribute__((address_space(3))) v4i16 *lds;
        const uint16_t *p = (const uint16_t *)tile + first * T::CH * 8;
        const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(p + column[c][0])));
        const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(p + column[c][1])));
        return uint4{lo.x, lo.y, hi.x, hi.y};
    }
};
// 64 rows of a matrix, straight into LDS; rows past the end of the sequence come as zeros (the buffer ends there).
__device__ __forceinline__ void dma16(u32x4 rows, uint32_t lane_off, uint32_t lds_off)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(lane_off), "s"(rows), "s"(lds_off) : "memory", "m0");
}
__device__ __forceinline__ void dma4(u32x4 rows, uint32_t lane_off, uint32_t lds_off)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(lane_off), "s"(rows), "s"(lds_off) : "memory", "m0");
}
__device__ __forceinline__ u32x4 buffer_of(uint64_t first, uint32_t bytes)
{
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)first), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(first >> 32)),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}
template <int DH> struct TileLoader : TileShape<DH> {
    using T = TileShape<DH>;
    static constexpr int LOADS = T::PIECES / 256;               // of a wavefront
    uint32_t off[LOADS];
    uint64_t base;
    uint32_t ld;
    int wave;
    // `first`: the sequence's first row, this head's first channel
    __device__ __forceinline__ TileLoader(const uint16_t *first, int ld_, int lane, int wave_) : base((uint64_t)(uintptr_t)first), ld((uint32_t)ld_ * 2u), wave(wave_)
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int p = 64 * (LOADS * wave + i) + lane, r = p / T::CH;
            off[i] = (uint32_t)r * ld + (uint32_t)T::in_row((p % T::CH) ^ T::swizzle(r)) * 16u;
        }
    }
    __device__ __forceinline__ void load(u32x4 *tile, int row0, int seq) const
    {
        const int left = seq - row0 < kTile ? seq - row0 : kTile;
        const u32x4 rows = buffer_of(base + (uint64_t)row0 * ld, (uint32_t)(left - 1) * ld + DH * 2);
        const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4 *)tile;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) dma16(rows, off[i], lds + (uint32_t)(LOADS * wave + i) * 1024u);
    }
};

// Which workgroup has which rows of which (sequence, head): consecutive workgroups go round-robin to the 8 XCDs, all tiles of a pair to one of
// them, whose L2 then holds what they share.
struct Item { int pair, tile; };
__device__ __forceinline__ Item item_of(int block, int tiles) { return {block / 8 / tiles * 8 + block % 8, block / 8 % tiles}; }

// ------------------------------------------------------------------ queries
template <int DT, int DH>
__global__ __launch_bounds__(256, 2) void attn_grad_queries_kernel(const uint16_t *__restrict__ qkv, const uint16_t *__restrict__ dout, uint16_t *__restrict__ dqkv,
                                                                   const float *__restrict__ delta, float *__restrict__ lse, const RowTops *__restrict__ tops,
                                                                   int seq, int n_heads, int pairs, int tiles)
{
    using T = TileShape<DH>;
    constexpr int KS = T::KS, CT = T::CT;
    // the reference is raised when a scaled score passes it by this much: unnormalised probabilities are 2^kRaise at most
    constexpr int kRaise = 4;
    __shared__ u32x4 ks[2][T::PIECES], vs[2][T::PIECES];
    const Item item = item_of((int)blockIdx.x, tiles);
    if (item.pair >= pairs) return;
    const int s = item.pair / n_heads, head = item.pair % n_heads, d = n_heads * DH, ld = 3 * d;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 31, fh = lane >> 5;
    const int q0 = (tiles - 1 - item.tile) * kOwn, w0 = q0 + 32 * wave, q = w0 + fr;          // the longest first
    const uint16_t *base = qkv + (size_t)s * seq * ld + head * DH;
    const float sc = 1.4426950408889634f / __builtin_sqrtf((float)DH);
    const int e = DT == kFP16 ? scale_exponent(tops + (size_t)item.pair * ((seq + kTile - 1) / kTile), (seq + kTile - 1) / kTile) - kRaise : 0;
    const float factor = DT == kFP16 ? ldexpf(1.0f, e) : 1.0f;

    uint4 qf[KS], of[KS];
    {
        const uint16_t *qp = base + (size_t)(q < seq ? q : 0) * ld + 8 * fh, *op = dout + ((size_t)s * seq + (q < seq ? q : 0)) * d + head * DH + 8 * fh;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            qf[i] = q < seq ? *(const uint4 *)(qp + 16 * i) : uint4{0, 0, 0, 0};
            of[i] = q < seq ? *(const uint4 *)(op + 16 * i) : uint4{0, 0, 0, 0};
        }
    }
    const float dl = (q < seq ? delta[(size_t)item.pair * seq + q] : 0.0f) * factor;
    const TileReader<DH> read(lane);
    const TileLoader<DH> load_k(base + d, ld, lane, wave), load_v(base + 2 * d, ld, lane, wave);
    f32x16 acc[CT] = {};
    float m_run = -INFINITY, moff = 0.0f, thr = -INFINITY, l_lane = 0.0f;
    const int last = q0 + kOwn <= seq ? q0 + kOwn : seq, n_tiles = (last + kTile - 1) / kTile;
    load_k.load(ks[0], 0, seq);
    load_v.load(vs[0], 0, seq);
    for (int t = 0; t < n_tiles; ++t) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (t + 1 < n_tiles) {
            load_k.load(ks[(t + 1) & 1], (t + 1) * kTile, seq);
            load_v.load(vs[(t + 1) & 1], (t + 1) * kTile, seq);
        }
        const u32x4 *kt = ks[t & 1], *vt = vs[t & 1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int first = t * kTile + 32 * h;
            if (first > w0) continue;                           // keys that none of the wavefront's queries sees
            f32x16 S = {}, dP = {};
#pragma unroll
            for (int i = 0; i < KS; ++i) S = mfma32<DT>(read.by_row(kt, h, i), qf[i], S);
#pragma unroll
            for (int i = 0; i < KS; ++i) dP = mfma32<DT>(read.by_row(vt, h, i), of[i], dP);
            if (first == w0) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (8 * (i >> 2) + 4 * fh + (i & 3) > fr) S[i] = -INFINITY;
            }
            float top = S[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top = __builtin_fmaxf(top, S[i]);
            if (__builtin_amdgcn_ballot_w64(top > thr) != 0) {
                float a, b;
                swap_halves(top, a, b);
                const float m_new = __builtin_fmaxf(__builtin_fmaxf(a, b), m_run), alpha = __builtin_amdgcn_exp2f((m_run - m_new) * sc);
                l_lane *= alpha;
#pragma unroll
                for (int c = 0; c < CT; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[c][i] *= alpha;
                m_run = m_new;
                moff = -m_new * sc;
                thr = m_new + (float)kRaise / sc;
            }
            uint4 ds[2];
            uint32_t *w = &ds[0].x;
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                float v[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(S[i + j], sc, moff));
                    l_lane += p;
                    v[j] = p * (DT == kFP16 ? __builtin_fmaf(dP[i + j], factor, -dl) : dP[i + j] - dl);
                }
                w[i / 2] = pack2<DT>(v[0], v[1]);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int c = 0; c < CT; ++c) acc[c] = mfma32<DT>(read.by_column(kt, 32 * h + 16 * k, c), ds[k], acc[c]);
        }
    }
    if (q >= seq) return;
    float a, b;
    swap_halves(l_lane, a, b);
    const float l = a + b;
    if (fh == 0) lse[(size_t)item.pair * seq + q] = m_run * sc + __builtin_amdgcn_logf(l);
    const float scale = 1.0f / (l * __builtin_sqrtf((float)DH)) * (DT == kFP16 ? ldexpf(1.0f, -e) : 1.0f);
    uint16_t *dq = dqkv + ((size_t)s * seq + q) * ld + head * DH + 4 * fh;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            if (32 * c + 2 * i < DH)
                *(uint2 *)(dq + 32 * c + 2 * i) = uint2{pack2<DT>(acc[c][i] * scale, acc[c][i + 1] * scale), pack2<DT>(acc[c][i + 2] * scale, acc[c][i + 3] * scale)};
}

// ------------------------------------------------------------------ keys
template <int DT, int DH>
__global__ __launch_bounds__(256, DH <= 96 ? 2 : 1) void attn_grad_keys_kernel(const uint16_t *__restrict__ qkv, const uint16_t *__restrict__ dout, uint16_t *__restrict__ dqkv,
                                                                const float *__restrict__ delta, const float *__restrict__ lse, const RowTops *__restrict__ tops,
                                                                int seq, int n_heads, int pairs, int tiles)
{
    using T = TileShape<DH>;
    constexpr int KS = T::KS, CT = T::CT;
    constexpr int kShift = DT == kFP16 ? 14 : 0;               // probabilities carry 2^kShift: down to 2^-28 they are normal numbers
    __shared__ u32x4 qs[2][T::PIECES], os[2][T::PIECES];
    __shared__ float rows[2][2][kTile];                         // logsumexp and D of a tile's queries
    const Item item = item_of((int)blockIdx.x, tiles);
    if (item.pair >= pairs) return;
    const int s = item.pair / n_heads, head = item.pair % n_heads, d = n_heads * DH, ld = 3 * d;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 31, fh = lane >> 5;
    const int k0 = item.tile * kOwn, w0 = k0 + 32 * wave, key = w0 + fr;                      // the longest first
    const uint16_t *base = qkv + (size_t)s * seq * ld + head * DH;
    const float sc = 1.4426950408889634f / __builtin_sqrtf((float)DH);
    const int e = DT == kFP16 ? scale_exponent(tops + (size_t)item.pair * ((seq + kTile - 1) / kTile), (seq + kTile - 1) / kTile) : 0;
    const float factor = DT == kFP16 ? ldexpf(1.0f, e - kShift) : 1.0f;
    uint4 kf[KS], vf[KS];
    {
        const uint16_t *kp = base + d + (size_t)(key < seq ? key : 0) * ld + 8 * fh;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            kf[i] = key < seq ? *(const uint4 *)(kp + 16 * i) : uint4{0, 0, 0, 0};
            vf[i] = key < seq ? *(const uint4 *)(kp + d + 16 * i) : uint4{0, 0, 0, 0};
        }
    }
    const TileReader<DH> read(lane);
    const TileLoader<DH> load_q(base, ld, lane, wave), load_o(dout + (size_t)s * seq * d + head * DH, d, lane, wave);
    auto load = [&](int t) {
        load_q.load(qs[t & 1], t * kTile, seq);
        load_o.load(os[t & 1], t * kTile, seq);
        if (wave < 2) {                                          // (queries past the end get zeros: their dO is, too)
            const int left = seq - t * kTile < kTile ? seq - t * kTile : kTile;
            const float *from = (wave ? delta : lse) + (size_t)item.pair * seq + t * kTile;
            dma4(buffer_of((uint64_t)(uintptr_t)from, (uint32_t)left * 4), 4 * lane, (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float *)&rows[t & 1][wave][0]);
        }
    };
    f32x16 dk[CT] = {}, dv[CT] = {};
    const int t0 = k0 / kTile, n_tiles = (seq + kTile - 1) / kTile;
    load(t0);
    for (int t = t0; t < n_tiles; ++t) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (t + 1 < n_tiles) load(t + 1);
        const u32x4 *qt = qs[t & 1], *ot = os[t & 1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int first = t * kTile + 32 * h;
            if (first < w0) continue;                           // queries that see none of the wavefront's keys
            f32x16 S = {}, dP = {};
#pragma unroll
            for (int i = 0; i < KS; ++i) S = mfma32<DT>(read.by_row(qt, h, i), kf[i], S);
#pragma unroll
            for (int i = 0; i < KS; ++i) dP = mfma32<DT>(read.by_row(ot, h, i), vf[i], dP);
            uint4 ps[2], ds[2];
            uint32_t *pw = &ps[0].x, *dw = &ds[0].x;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 ls = *(const float4 *)&rows[t & 1][0][32 * h + 8 * g + 4 * fh], dl = *(const float4 *)&rows[t & 1][1][32 * h + 8 * g + 4 * fh];
                const float lr[4] = {ls.x, ls.y, ls.z, ls.w}, dr[4] = {dl.x, dl.y, dl.z, dl.w};
                float p[4], v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[4 * g + j], sc, (float)kShift - lr[j]));
                    if (first == w0 && 8 * g + 4 * fh + j < fr) p[j] = 0.0f;
                    v[j] = p[j] * (DT == kFP16 ? (dP[4 * g + j] - dr[j]) * factor : dP[4 * g + j] - dr[j]);
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    pw[2 * g + j] = pack2<DT>(p[2 * j], p[2 * j + 1]);
                    dw[2 * g + j] = pack2<DT>(v[2 * j], v[2 * j + 1]);
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    dv[c] = mfma32<DT>(read.by_column(ot, 32 * h + 16 * k, c), ps[k], dv[c]);
                    dk[c] = mfma32<DT>(read.by_column(qt, 32 * h + 16 * k, c), ds[k], dk[c]);
                }
        }
    }
    if (key >= seq) return;
    const float k_scale = (DT == kFP16 ? ldexpf(1.0f, -e) : 1.0f) / __builtin_sqrtf((float)DH), v_scale = DT == kFP16 ? 0x1p-14f : 1.0f;
    uint16_t *to = dqkv + ((size_t)s * seq + key) * ld + d + head * DH + 4 * fh;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            if (32 * c + 2 * i < DH) {
                auto four = [&](const f32x16 &a, float f) { return uint2{pack2<DT>(a[i] * f, a[i + 1] * f), pack2<DT>(a[i + 2] * f, a[i + 3] * f)}; };
                *(uint2 *)(to + 32 * c + 2 * i) = four(dk[c], k_scale);
                *(uint2 *)(to + d + 32 * c + 2 * i) = four(dv[c], v_scale);
            }
}

template <int DT, int DH>
hipError_t attn_grad(const uint16_t *qkv, const uint16_t *out, const uint16_t *dout, uint16_t *dqkv, char *ws, int n_seq, int seq, int n_heads, hipStream_t s)
{
    const int pairs = n_seq * n_heads, row_tiles = (seq + kTile - 1) / kTile, tiles = (seq + kOwn - 1) / kOwn;
    float *delta = (float *)ws, *lse = delta + (size_t)pairs * seq;
    RowTops *tops = (RowTops *)(lse + (size_t)pairs * seq);
    attn_grad_rows_kernel<DT, DH><<<dim3(pairs * row_tiles), dim3(256), 0, s>>>(qkv, out, dout, delta, tops, seq, n_heads, row_tiles);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    const dim3 grid((pairs + 7) / 8 * 8 * tiles);
    attn_grad_queries_kernel<DT, DH><<<grid, dim3(256), 0, s>>>(qkv, dout, dqkv, delta, lse, tops, seq, n_heads, pairs, tiles);
    if ((err = hipGetLastError()) != hipSuccess) return err;
    attn_grad_keys_kernel<DT, DH><<<grid, dim3(256), 0, s>>>(qkv, dout, dqkv, delta, lse, tops, seq, n_heads, pairs, tiles);
    return hipGetLastError();
}

// ------------------------------------------------------------------ other heads and precisions
// A workgroup per query of a head: logsumexp over the keys it sees, D, dQ.  128 threads have a key each, then a channel each.
template <int DT>
__global__ __launch_bounds__(128) void attn_grad_query_kernel(const void *__restrict__ qkv_, const void *__restrict__ out_, const void *__restrict__ dout_, void *__restrict__ dqkv_,
                                                              void *__restrict__ rows_, int seq, int n_heads, int d_head, size_t n_rows)
{
    using P = Prec<DT>;
    using A = typename P::A;
    using Acc = typename P::Acc;
    __shared__ Acc own[2][128], ds[128], red[16];
    const int head = (int)blockIdx.y, d = n_heads * d_head, tid = threadIdx.x;
    const size_t row = blockIdx.x, first = row / seq * seq, ld = 3 * (size_t)d;
    const int q = (int)(row - first);
    const A *qkv = (const A *)qkv_ + head * d_head, *out = (const A *)out_ + row * d + head * d_head, *dout = (const A *)dout_ + row * d + head * d_head;
    const Acc scale = (Acc)1 / (Acc)__builtin_sqrt((double)d_head);
    const bool mine = tid < d_head;
    own[0][tid] = mine ? P::a2acc(qkv[row * ld + tid]) : (Acc)0;
    own[1][tid] = mine ? P::a2acc(dout[tid]) : (Acc)0;
    const Acc delta = block_sum(mine ? own[1][tid] * P::a2acc(out[tid]) : (Acc)0, red);          // (has a barrier)
    auto dot = [&](int which, int key, int part) {
        const A *p = qkv + (first + key) * ld + part * d;
        Acc v = 0;
        for (int c = 0; c < d_head; ++c) v += own[which][c] * P::a2acc(p[c]);
        return v;
    };
    Acc top = -INFINITY, sum = 0;
    for (int k = tid; k <= q; k += 128) {
        const Acc sco = dot(0, k, 1) * scale, m = sco > top ? sco : top;
        sum = sum * (Acc)exp(top - m) + (Acc)exp(sco - m);
        top = m;
    }
    const Acc most = block_max(top, red);
    const Acc l = block_sum(sum != (Acc)0 ? sum * (Acc)exp(top - most) : (Acc)0, red), lse = most + (Acc)log(l);
    Acc dq = 0;
    for (int k0 = 0; k0 <= q; k0 += 128) {
        const int k = k0 + tid;
        __syncthreads();
        ds[tid] = k <= q ? (Acc)exp(dot(0, k, 1) * scale - lse) * (dot(1, k, 2) - delta) : (Acc)0;
        __syncthreads();
        const int n = q - k0 + 1 < 128 ? q - k0 + 1 : 128;
        if (mine)
            for (int j = 0; j < n; ++j) dq += ds[j] * P::a2acc(qkv[(first + k0 + j) * ld + d + tid]);
    }
    if (mine) ((A *)dqkv_)[row * ld + head * d_head + tid] = P::acc2a(dq * scale);
    if (tid == 0) {
        Acc *rows = (Acc *)rows_ + (size_t)head * n_rows + row;
        rows[0] = delta;
        rows[(size_t)n_heads * n_rows] = lse;
    }
}
// A workgroup per key of a head: dK and dV over the queries that see it.
template <int DT>
__global__ __launch_bounds__(128) void attn_grad_key_kernel(const void *__restrict__ qkv_, const void *__restrict__ dout_, void *__restrict__ dqkv_, const void *__restrict__ rows_,
                                                            int seq, int n_heads, int d_head, size_t n_rows)
{
    using P = Prec<DT>;
    using A = typename P::A;
    using Acc = typename P::Acc;
    __shared__ Acc own[2][128], ps[128], ds[128];
    const int head = (int)blockIdx.y, d = n_heads * d_head, tid = threadIdx.x;
    const size_t row = blockIdx.x, first = row / seq * seq, ld = 3 * (size_t)d;
    const int key = (int)(row - first);
    const A *qkv = (const A *)qkv_ + head * d_head, *dout = (const A *)dout_ + head * d_head;
    const Acc *delta = (const Acc *)rows_ + (size_t)head * n_rows + first, *lse = delta + (size_t)n_heads * n_rows;
    const Acc scale = (Acc)1 / (Acc)__builtin_sqrt((double)d_head);
    const bool mine = tid < d_head;
    own[0][tid] = mine ? P::a2acc(qkv[row * ld + d + tid]) : (Acc)0;
    own[1][tid] = mine ? P::a2acc(qkv[row * ld + 2 * d + tid]) : (Acc)0;
    auto dot = [&](int which, const A *p) {
        Acc v = 0;
        for (int c = 0; c < d_head; ++c) v += own[which][c] * P::a2acc(p[c]);
        return v;
    };
    Acc dk = 0, dv = 0;
    for (int q0 = key; q0 < seq; q0 += 128) {
        const int q = q0 + tid;
        __syncthreads();
        ps[tid] = q < seq ? (Acc)exp(dot(0, qkv + (first + q) * ld) * scale - lse[q]) : (Acc)0;
        ds[tid] = q < seq ? ps[tid] * (dot(1, dout + (first + q) * d) - delta[q]) : (Acc)0;
        __syncthreads();
        const int n = seq - q0 < 128 ? seq - q0 : 128;
        if (mine)
            for (int j = 0; j < n; ++j) {
                dk += ds[j] * P::a2acc(qkv[(first + q0 + j) * ld + tid]);
                dv += ps[j] * P::a2acc(dout[(first + q0 + j) * d + tid]);
            }
    }
    if (!mine) return;
    A *to = (A *)dqkv_ + row * ld + d + head * d_head + tid;
    to[0] = P::acc2a(dk * scale);
    to[d] = P::acc2a(dv);
}
template <int DT>
hipError_t attn_grad_plain(const void *qkv, const void *out, const void *dout, void *dqkv, void *ws, int n_seq, int seq, int n_heads, int d_head, hipStream_t s)
{
    const size_t rows = (size_t)n_seq * seq;
    const dim3 grid((unsigned)rows, (unsigned)n_heads);
    attn_grad_query_kernel<DT><<<grid, dim3(128), 0, s>>>(qkv, out, dout, dqkv, ws, seq, n_heads, d_head, rows);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    attn_grad_key_kernel<DT><<<grid, dim3(128), 0, s>>>(qkv, dout, dqkv, ws, seq, n_heads, d_head, rows);
    return hipGetLastError();
}

bool on_matrix_cores(int dtype, int d_head) { return dtype != kFP32 && (d_head == 64 || d_head == 80 || d_head == 96 || d_head == 112 || d_head == 128); }

}  // namespace

size_t attention_grad_scratch(int dtype, int n_seq, int seq, int n_heads, int d_head)
{
    const size_t pairs = (size_t)n_seq * n_heads, row_tiles = ((size_t)seq + kTile - 1) / kTile;
    // a launch's size is counted in threads, by 32 bits, and in workgroups of the second dimension by 16
    if (on_matrix_cores(dtype, d_head)) {
        if ((pairs + 7) / 8 * 8 * row_tiles >= (size_t)1 << 24) return 0;
        return 2 * 4 * pairs * seq + pairs * row_tiles * sizeof(RowTops);
    }
    if ((size_t)n_seq * seq >= (size_t)1 << 25 || n_heads > 65535) return 0;
    return 2 * acc_bytes(dtype) * pairs * seq;
}

hipError_t launch_attention_grad(const void *qkv, const void *out, const void *dout, void *dqkv, void *scratch, int dtype, int n_seq, int seq, int n_heads,
                                 int d_head, hipStream_t s)
{
    if (attention_grad_scratch(dtype, n_seq, seq, n_heads, d_head) == 0) return hipErrorNotSupported;
    if (!on_matrix_cores(dtype, d_head)) {
        auto f = dtype == kFP32 ? attn_grad_plain<kFP32> : dtype == kBF16 ? attn_grad_plain<kBF16> : attn_grad_plain<kFP16>;
        return f(qkv, out, dout, dqkv, scratch, n_seq, seq, n_heads, d_head, s);
    }
    auto go = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        auto f = d_head == 64 ? attn_grad<DT, 64> : d_head == 80 ? attn_grad<DT, 80> : d_head == 96 ? attn_grad<DT, 96> : d_head == 112 ? attn_grad<DT, 112> : attn_grad<DT, 128>;
        return f((const uint16_t *)qkv, (const uint16_t *)out, (const uint16_t *)dout, (uint16_t *)dqkv, (char *)scratch, n_seq, seq, n_heads, s);
    };
    return dtype == kBF16 ? go(std::integral_constant<int, kBF16>{}) : go(std::integral_constant<int, kFP16>{});
}

}  // namespace zo
