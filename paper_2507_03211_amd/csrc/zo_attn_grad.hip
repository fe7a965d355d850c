// Backward pass of the causal multi-head attention.  With P = softmax(q k^T / sqrt(d_head)) over the keys a query sees, and per query
// D = sum_c dO O (which is sum_k P dP):
//
//   dV = P^T dO,   dP = dO V^T,   dS = P (dP - D),   dQ = dS K / sqrt(d_head),   dK = dS^T Q / sqrt(d_head)
//
// Matrix path (16-bit types, heads of 64, 80, 96, 112, 128), two launches, and in fp16 one before them that finds what bounds dS (below):
//   queries  a wavefront's 32 queries against the keys they see: D, S, dP, dQ.  The softmax runs along (one pass, a reference that is raised
//            as scores pass it), so that the reference and the sum come out at the end, for the other launch
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
typedef float f32x4 __attribute__((ext_vector_type(4)));

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

constexpr int kShort = 128;                 // positions of a sequence up to which D is summed from P dP (attn_grad_queries_kernel)
constexpr int kOwn = 128, kTile = 64;      // rows of a workgroup's own (32 a wavefront), rows of a tile that streams through LDS

// fp16: dS = P (dP - D) may lie anywhere: |dP| and |D| are at most A B, with A the largest norm of a row of dO and B of a row of V in the
// sequence and head, so 2^e dS with 2^e = 2^14 / (2 A B) rounded down is within the type whatever P is, and numbers 2^28 below that bound are still
// normal ones.  2^-e is taken out of the fp32 sums.  bf16 has fp32's range: e = 0.
// What the keys' launch's probabilities carry: 2^kShift, with which they are normal numbers of fp16 down to 2^-28.
template <int DT> constexpr int kShift = DT == kFP16 ? 14 : 0;
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

// The largest |dO|^2 and |V|^2 of 64 rows of one head of one sequence; 16 lanes a row (8 where it has 8 pieces of 16 bytes).
template <int DH>
__global__ __launch_bounds__(256) void attn_grad_tops_kernel(const uint16_t *__restrict__ qkv, const uint16_t *__restrict__ dout, RowTops *__restrict__ tops, int seq,
                                                             int n_heads, int tiles)
{
    constexpr int PIECES = DH / 8, LANES = PIECES <= 8 ? 8 : 16, ROWS = 256 / LANES, TURNS = kTile / ROWS;
    __shared__ float top[2][4];
    const int tile = (int)blockIdx.x % tiles, pair = (int)blockIdx.x / tiles, s = pair / n_heads, head = pair % n_heads, d = n_heads * DH;
    const int piece = threadIdx.x % LANES;
    uint4 x[TURNS][2];                                          // all under way together
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        const int r = tile * kTile + i * ROWS + (int)threadIdx.x / LANES;
        const bool live = r < seq && piece < PIECES;
        const size_t row = (size_t)s * seq + (r < seq ? r : 0), at = row * d + head * DH + (piece < PIECES ? 8 * piece : 0);
        x[i][0] = live ? *(const uint4 *)(dout + at) : uint4{0, 0, 0, 0};
        x[i][1] = live ? *(const uint4 *)(qkv + at + row * 2 * d + 2 * d) : uint4{0, 0, 0, 0};
    }
    float most[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < TURNS; ++i)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const uint32_t w[4] = {x[i][which].x, x[i][which].y, x[i][which].z, x[i][which].w};
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = Prec<kFP16>::a2acc((uint16_t)(w[e / 2] >> (16 * (e & 1))));
                sum = __builtin_fmaf(v, v, sum);
            }
#pragma unroll
            for (int m = LANES / 2; m > 0; m >>= 1) sum += __shfl_xor(sum, m, 64);
            most[which] = sum > most[which] ? sum : most[which];
        }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const float m = wave_max(most[which]);
        if ((threadIdx.x & 63) == 0) top[which][threadIdx.x >> 6] = m;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        const float *t = top[threadIdx.x];
        const float a = t[0] > t[1] ? t[0] : t[1], b = t[2] > t[3] ? t[2] : t[3];
        (&tops[blockIdx.x].out2)[threadIdx.x] = a > b ? a : b;
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
// A stage's tiles begin at multiples of 4 KiB, and the pieces of a row and of four rows differ in address bits that nothing else sets, so that an exclusive
// or with a constant leads from one piece's address to another's: a register for the rows, two for the columns, instead of one for each piece.
template <int DH> struct TileReader : TileShape<DH> {
    using T = TileShape<DH>;
    static constexpr bool kXor = T::CH != 12;                   // (192-byte rows: pieces within aligned groups of four only)
    uint32_t row[kXor ? 1 : 2], column[2];  // byte offset of (row lane % 32, k-step 0 (1)); of a column fragment, row base 0 or 8 mod 16
    __device__ __forceinline__ TileReader(int lane)
    {
        const int fr = lane & 31, fh = lane >> 5, j = lane & 15;
#pragma unroll
        for (int s = 0; s < (kXor ? 1 : 2); ++s) row[s] = (fr * T::CH + ((2 * s + fh) ^ T::swizzle(fr))) * 16;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int r = 8 * b + 4 * fh + (j >> 2), chan = 16 * ((lane >> 4) & 1) + 4 * (j & 3);
            column[b] = (r * T::CH + ((chan >> 3) ^ T::swizzle(r))) * 16 + 2 * (chan & 7);
        }
    }
    static __device__ __forceinline__ uint32_t address(const u32x4 *tile) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const u32x4 *)tile; }
    // rows lane % 32, channels of k-step s; `tile`: the first row
    __device__ __forceinline__ uint4 by_row(const u32x4 *tile, int s) const
    {
        const uint32_t at = kXor ? (address(tile) + row[0]) ^ (uint32_t)(32 * s) : address(tile) + row[s % (kXor ? 1 : 2)] + (s / 2) * 64;
        return __builtin_bit_cast(uint4, *(__attribute__((address_space(3))) const u32x4 *)(uintptr_t)at);
    }
    // channels of tile c, rows first + {4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3}, first a multiple of 16
    __device__ __forceinline__ uint4 by_column(const u32x4 *tile, int first, int c) const
    {
        typedef __attribute__((address_space(3))) v4i16 *lds;
        auto at = [&](int b) {
            const uint32_t base = address(tile) + column[b];
            return (kXor ? base ^ (uint32_t)(64 * c) : base + 64 * c) + (uint32_t)(first * T::CH * 16);
        };
        const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(uintptr_t)at(0)));
        const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(uintptr_t)at(1)));
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
// LEAN (rows of 16 pieces): a register instead of one a load.  A load's rows lie four behind the last one's, and its swizzle differs in the two lowest bits.
template <int DH, bool LEAN = false> struct TileLoader : TileShape<DH> {
    using T = TileShape<DH>;
    static constexpr int LOADS = T::PIECES / 256;               // of a wavefront
    static_assert(!LEAN || (T::CHD == 16 && LOADS == 4), "rows of 256 bytes, at multiples of these from one another");
    uint32_t off[LEAN ? 1 : LOADS];
    uint32_t ld;
    int wave;
    __device__ __forceinline__ TileLoader(int ld_, int lane, int wave_) : ld((uint32_t)ld_ * 2u), wave(wave_)
    {
#pragma unroll
        for (int i = 0; i < (LEAN ? 1 : LOADS); ++i) {
            const int p = 64 * (LOADS * wave + i) + lane, r = p / T::CH;
            off[i] = (uint32_t)r * ld + (uint32_t)T::in_row((p % T::CH) ^ T::swizzle(r)) * 16u;
        }
    }
    // `first`: the sequence's first row, this head's first channel
    __device__ __forceinline__ void load(u32x4 *tile, const uint16_t *first, int row0, int seq) const
    {
        const int left = seq - row0 < kTile ? seq - row0 : kTile;
        const u32x4 rows = buffer_of((uint64_t)(uintptr_t)first + (uint64_t)row0 * ld, (uint32_t)(left - 1) * ld + DH * 2);
        const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4 *)tile;
        uint32_t at = off[0];
        if constexpr (LEAN) asm volatile("" : "+v"(at));         // (or the others are worked out ahead of the loop, and kept)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) dma16(rows, LEAN ? (at ^ (uint32_t)(16 * i)) + (uint32_t)(4 * i) * ld : off[i], lds + (uint32_t)(LOADS * wave + i) * 1024u);
    }
};

// Which workgroup has which rows of which (sequence, head): the longest tiles of all pairs first, so that what is left at a launch's end is
// short; consecutive workgroups go round-robin to the 8 XCDs, all tiles of a pair to one of them.  All tiles of a pair, then the next one's:
// 4 x 2048, 40 heads of 128 744 us of the whole call, here 693; of 64 410 / 367; 16 x 512, 12 of 64 58.8 / 53.5; 8 x 131, 32 of 80 fp16 40.7 / 35.7.
struct Item { int pair, tile; };
__device__ __forceinline__ Item item_of(int block, int pairs)
{
    const int row = (pairs + 7) / 8 * 8;
    return {block % row, block / row};
}

__device__ __forceinline__ void put(uint4 (&w)[2], int i, uint32_t v)      // word i of two fragments
{
    uint4 &f = w[i >> 2];
    if ((i & 3) == 0) f.x = v;
    else if ((i & 3) == 1) f.y = v;
    else if ((i & 3) == 2) f.z = v;
    else f.w = v;
}

// ------------------------------------------------------------------ queries
// 32 keys at a time: S, dP beside the exponentials, dQ; two wavefronts per SIMD (210 registers at 128 channels).  Pipelined over two
// units, with keys in three stages, it was no faster (4 x 2048, 40 heads of 128 656 us of the whole call in bf16 both ways, of 80 500 / 491, 16 x 512, 12 of 64 52.6 / 51.4).
// Three workgroups to a CU at 96 channels 610 us, four at 64 454 (registers), where this has 554 and 367.
// D: of sequences up to kShort positions (SHORT) the sum of P dP, by a pass ahead; of longer ones that of dO times `out`, whose rounding to 16 bits then makes the
// gradients little worse.  Error of all three against 64 bits over that of fp32 arithmetic, both rounded: by `out` 1.67 at 2 positions, 1.57 at 8, 1.51 at 16,
// 1.48 at 128, 1.46 at 300; by the pass 1.23 - 1.44.  us of the whole call by `out` / by the pass: 8 x 64, 32 heads of 80 fp16 18.3 / 18.5, 8 x 128 bf16 23.8 / 25.0,
// 16 x 128, 40 of 128 73.7 / 72.3, 256 x 64, 12 of 64 76.3 / 72.2.
template <int DT, int DH, bool SHORT>
__global__ __launch_bounds__(256, 2) void attn_grad_queries_kernel(const uint16_t *__restrict__ qkv, const uint16_t *__restrict__ out, const uint16_t *__restrict__ dout,
                                                                   uint16_t *__restrict__ dqkv, float *__restrict__ rows, const RowTops *__restrict__ tops,
                                                                   int seq, int n_heads, int pairs, int tiles)
{
    using T = TileShape<DH>;
    constexpr int KS = T::KS, CT = T::CT, R = 4;
    // the reference is raised when a scaled score passes it by this much: unnormalised probabilities are 2^kRaise at most
    constexpr int kRaise = 4;
    const float lazy = (float)kRaise * __builtin_sqrtf((float)DH) / 1.4426950408889634f;
    __shared__ __attribute__((aligned(256))) u32x4 ks[2][T::PIECES], vs[2][T::PIECES];
    const Item item = item_of((int)blockIdx.x, pairs);
    if (item.pair >= pairs) return;
    const int s = item.pair / n_heads, head = item.pair % n_heads, d = n_heads * DH, ld = 3 * d;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 31, fh = lane >> 5;
    const int q0 = (tiles - 1 - item.tile) * kOwn, w0 = q0 + 32 * wave, q = w0 + fr;          // the longest first
    const uint16_t *base = qkv + (size_t)s * seq * ld + head * DH;
    const float sc = 1.4426950408889634f / __builtin_sqrtf((float)DH);
    const int row_tiles = (seq + kTile - 1) / kTile;
    // (fp16: probabilities carry 2^e, and with them dS; so does their sum)
    const int e = DT == kFP16 ? scale_exponent(tops + (size_t)item.pair * row_tiles, row_tiles) - kRaise : 0;
    // A score against the reference, as an exponent of two.  The difference first: it is exact where it counts.  A product of the reference and sc would be
    // off by its last place, which for large scores is all of P
    auto exponent = [&](float s, float m) { return DT == kFP16 ? __builtin_fmaf(s - m, sc, (float)e) : (s - m) * sc; };

    uint4 qf[KS], of[KS];
    const size_t at = ((size_t)s * seq + (q < seq ? q : 0)) * d + head * DH + 8 * fh;
    {
        const uint16_t *qp = base + (size_t)(q < seq ? q : 0) * ld + 8 * fh, *gp = dout + at;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            of[i] = q < seq ? *(const uint4 *)(gp + 16 * i) : uint4{0, 0, 0, 0};
            qf[i] = q < seq ? *(const uint4 *)(qp + 16 * i) : uint4{0, 0, 0, 0};
        }
    }
    const TileReader<DH> read(lane);
    const TileLoader<DH> loader(ld, lane, wave);
    const int last = q0 + kOwn <= seq ? q0 + kOwn : seq, n_tiles = (last + kTile - 1) / kTile;
    auto load = [&](int t) {
        if (t >= n_tiles) return;
        loader.load(ks[t & 1], base + d, t * kTile, seq);
        loader.load(vs[t & 1], base + 2 * d, t * kTile, seq);
    };
    auto mask = [&](f32x16 &x) {                                // keys behind the query, of the unit on the diagonal
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (8 * (i >> 2) + 4 * fh + (i & 3) > fr) x[i] = -INFINITY;
    };
    auto maximum = [&](const f32x16 &x) {
        float top = __builtin_fmaxf(__builtin_fmaxf(x[0], x[1]), x[2]);
#pragma unroll
        for (int i = 3; i < 15; i += 2) top = __builtin_fmaxf(__builtin_fmaxf(x[i], x[i + 1]), top);
        return __builtin_fmaxf(top, x[15]);
    };
    float minus_d = 0.0f, a, b;
    if constexpr (SHORT) {
        float m = -INFINITY, l = 0.0f, sum = 0.0f;
        load(0);
        for (int t = 0; t < n_tiles; ++t) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            load(t + 1);
            for (int h = 0; h < 2; ++h) {
                const int first = t * kTile + 32 * h;
                if (first > w0) break;
                const u32x4 *kt = ks[t & 1] + h * 32 * T::CH, *vt = vs[t & 1] + h * 32 * T::CH;
                f32x16 S = {}, dP = {};
#pragma unroll
                for (int i = 0; i < KS; ++i) S = mfma32<DT>(read.by_row(kt, i), qf[i], S);
#pragma unroll
                for (int i = 0; i < KS; ++i) dP = mfma32<DT>(read.by_row(vt, i), of[i], dP);
                if (first == w0) mask(S);
                swap_halves(maximum(S), a, b);
                const float m_new = __builtin_fmaxf(__builtin_fmaxf(a, b), m), alpha = __builtin_amdgcn_exp2f((m - m_new) * sc);
                l *= alpha;
                sum *= alpha;
                m = m_new;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float p = __builtin_amdgcn_exp2f((S[j] - m) * sc);
                    l += p;
                    sum = __builtin_fmaf(p, dP[j], sum);
                }
            }
        }
        __syncthreads();                                        // (the tiles are loaded again)
        swap_halves(l, a, b);
        l = a + b;
        swap_halves(sum, a, b);
        minus_d = -(a + b) / l;
    } else {
        const uint16_t *op = out + at;
        uint4 o[KS];
#pragma unroll
        for (int i = 0; i < KS; ++i) o[i] = q < seq ? *(const uint4 *)(op + 16 * i) : uint4{0, 0, 0, 0};
        auto two = [&](uint32_t a, uint32_t b) {
#pragma unroll
            for (int e = 0; e < 32; e += 16) minus_d = __builtin_fmaf(-Prec<DT>::a2acc((uint16_t)(a >> e)), Prec<DT>::a2acc((uint16_t)(b >> e)), minus_d);
        };
#pragma unroll
        for (int i = 0; i < KS; ++i) { two(o[i].x, of[i].x); two(o[i].y, of[i].y); two(o[i].z, of[i].z); two(o[i].w, of[i].w); }
        swap_halves(minus_d, a, b);
        minus_d = a + b;
    }
    f32x16 acc[CT] = {};
    float m_run = -INFINITY, l_lane = 0.0f;
    load(0);
    for (int t = 0; t < n_tiles; ++t) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        load(t + 1);
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            const int first = t * kTile + 32 * h;
            if (first > w0) break;                              // keys that none of the wavefront's queries sees
            const u32x4 *kt = ks[t & 1] + h * 32 * T::CH, *vt = vs[t & 1] + h * 32 * T::CH;
            f32x16 S = {}, dP;
            uint4 ring[R];
#pragma unroll
            for (int i = 0; i < R; ++i) ring[i] = read.by_row(kt, i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                S = mfma32<DT>(ring[i % R], qf[i], S);
                __builtin_amdgcn_sched_barrier(0);
                ring[i % R] = i + R < KS ? read.by_row(kt, i + R) : read.by_row(vt, i + R - KS);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) dP[j] = minus_d;
            if (first == w0) mask(S);
            const float most = maximum(S);
            if (__builtin_amdgcn_ballot_w64(most - m_run > lazy) != 0) {
                swap_halves(most, a, b);
                const float m_new = __builtin_fmaxf(__builtin_fmaxf(a, b), m_run), alpha = __builtin_amdgcn_exp2f((m_run - m_new) * sc);
                l_lane *= alpha;
#pragma unroll
                for (int c = 0; c < CT; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[c][i] *= alpha;
                m_run = m_new;
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                dP = mfma32<DT>(ring[(KS + i) % R], of[i], dP);
                __builtin_amdgcn_sched_barrier(0);
                if (i + R < KS) ring[(KS + i) % R] = read.by_row(vt, i + R);
#pragma unroll
                for (int j = 16 * i / KS; j < 16 * (i + 1) / KS; ++j) {
                    S[j] = __builtin_amdgcn_exp2f(exponent(S[j], m_run));
                    l_lane += S[j];
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            uint4 ds[2], kc = read.by_column(kt, 0, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                put(ds, j, pack2<DT>(S[2 * j] * dP[2 * j], S[2 * j + 1] * dP[2 * j + 1]));
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 2 * CT; ++i) {
                const int n = i + 1;
                uint4 kn{};
                if (n < 2 * CT) kn = read.by_column(kt, 16 * (n / CT), n % CT);
                __builtin_amdgcn_sched_barrier(0);
                acc[i % CT] = mfma32<DT>(kc, ds[i / CT], acc[i % CT]);
                __builtin_amdgcn_sched_barrier(0);
                kc = kn;
            }
        }
    }
    if (q >= seq) return;
    swap_halves(l_lane, a, b);
    const float l = a + b;
    // for the other launch, in two numbers: in one, as a logsumexp, the sum would be rounded to the scores' last place
    if (fh == 0) {
        const size_t row = (size_t)item.pair * seq + q;
        *(f32x2 *)(rows + 2 * row) = f32x2{m_run, (float)kShift<DT> - __builtin_amdgcn_logf(ldexpf(l, -e))};
        rows[2 * (size_t)pairs * seq + row] = minus_d;
    }
    const float scale = 1.0f / (l * __builtin_sqrtf((float)DH));
    uint16_t *dq = dqkv + ((size_t)s * seq + q) * ld + head * DH + 4 * fh;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            if (32 * c + 2 * i < DH)
                *(uint2 *)(dq + 32 * c + 2 * i) = uint2{pack2<DT>(acc[c][i] * scale, acc[c][i + 1] * scale), pack2<DT>(acc[c][i + 2] * scale, acc[c][i + 3] * scale)};
}

// ------------------------------------------------------------------ keys
// 32 queries at a time: S, dP beside P's exponentials, then dV and dK.  Two wavefronts per SIMD, whose waits each other's multiplies fill, are worth more than
// one whose own are pipelined (386 registers; 4 x 2048, 40 heads of 128 742 us of the whole call / 657, of 112 720 / 635, of 96 582 / 535, of 64 350 / 345, 16 x 512, 12 of 64 54.1 /
// 51.7, when a row had one number, its logsumexp, which is wrong for large scores).  A row's reference and sum apart cost a subtraction and a read more a score: 663 / 681, 638 / 654,
// 541 / 554, 348 / 367, 50.5 / 53.5.  At 128 channels dK, dV, K and V leave 64 of 256 registers for the rest, so that nothing is held ahead but two fragments and two rows' numbers,
// and a load's addresses are worked out as it goes out (four rows' numbers and addresses kept: spills, 793).  4 x 2048, 40 heads of 128: 372 - 383 us, matrix cores busy 46 % of the
// cycles, vector units 32, LDS 31 without conflicts; the queries' launch 294 - 302, 43, 42 and 22 %.
template <int DT, int DH>
__global__ __launch_bounds__(256, 2) void attn_grad_keys_kernel(const uint16_t *__restrict__ qkv, const uint16_t *__restrict__ dout, uint16_t *__restrict__ dqkv,
                                                                const float *__restrict__ rows, const RowTops *__restrict__ tops,
                                                                int seq, int n_heads, int pairs, int tiles)
{
    using T = TileShape<DH>;
    constexpr int KS = T::KS, CT = T::CT, R = 2, AHEAD = KS < 7 ? 2 : 1;
    __shared__ __attribute__((aligned(256))) u32x4 qs[2][T::PIECES], os[2][T::PIECES];
    __shared__ __attribute__((aligned(16))) float refs[2][kTile][2], minus_d[2][kTile];   // of a tile's queries: reference and kShift - logarithm of the sum, minus D
    const Item item = item_of((int)blockIdx.x, pairs);
    if (item.pair >= pairs) return;
    const int s = item.pair / n_heads, head = item.pair % n_heads, d = n_heads * DH, ld = 3 * d;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 31, fh = lane >> 5;
    const int k0 = item.tile * kOwn, w0 = k0 + 32 * wave, key = w0 + fr;                      // the longest first
    const uint16_t *base = qkv + (size_t)s * seq * ld + head * DH, *obase = dout + (size_t)s * seq * d + head * DH;
    const float sc = 1.4426950408889634f / __builtin_sqrtf((float)DH);
    const int e = DT == kFP16 ? scale_exponent(tops + (size_t)item.pair * ((seq + kTile - 1) / kTile), (seq + kTile - 1) / kTile) : 0;
    const float factor = DT == kFP16 ? ldexpf(1.0f, e - kShift<DT>) : 1.0f;
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
    const TileLoader<DH, DH == 128> load_q(ld, lane, wave), load_o(d, lane, wave);
    const int t0 = k0 / kTile, n_tiles = (seq + kTile - 1) / kTile;
    auto load = [&](int t) {
        if (t >= n_tiles) return;
        load_q.load(qs[t & 1], base, t * kTile, seq);
        load_o.load(os[t & 1], obase, t * kTile, seq);
        if (wave < 3) {                                          // (queries past the end get zeros: their dO is, too)
            const int left = seq - t * kTile < kTile ? seq - t * kTile : kTile;
            const size_t row = (size_t)item.pair * seq + t * kTile;
            auto lds = [](float *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float *)p; };
            // (the lane's number anew: kept, it is spilled at 128 channels, and its reload waits for the tiles: 693 us for 681)
            int all = -1;
            asm volatile("" : "+s"(all));
            const int lane = __builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0));
            if (wave < 2) dma4(buffer_of((uint64_t)(uintptr_t)(rows + 2 * row), (uint32_t)left * 8), 4 * lane + 256 * wave, lds(&refs[t & 1][32 * wave][0]));
            else dma4(buffer_of((uint64_t)(uintptr_t)(rows + 2 * (size_t)pairs * seq + row), (uint32_t)left * 4), 4 * lane, lds(&minus_d[t & 1][0]));
        }
    };
    f32x16 dk[CT] = {}, dv[CT] = {};
    load(t0);
    for (int t = t0; t < n_tiles; ++t) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        load(t + 1);
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            const int first = t * kTile + 32 * h;
            if (first < w0) continue;                           // queries that see none of the wavefront's keys
            const u32x4 *qt = qs[t & 1] + h * 32 * T::CH, *ot = os[t & 1] + h * 32 * T::CH;
            // S from zero on, by the same products in the same order as in the queries' launch: the same bits, of which the reference is one
            f32x16 S = {}, dP;                                  // (from minus D on)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 v = *(const f32x4 *)&minus_d[t & 1][32 * h + 8 * g + 4 * fh];
#pragma unroll
                for (int j = 0; j < 4; ++j) dP[4 * g + j] = v[j];
            }
            auto two_refs = [&](int j) { return *(const f32x4 *)&refs[t & 1][32 * h + 8 * (j >> 2) + 4 * fh + (j & 3)][0]; };
            f32x4 ref[AHEAD];                                   // of rows 2 i, 2 i + 1
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) ref[i] = two_refs(2 * i);
            uint4 ring[R];
#pragma unroll
            for (int i = 0; i < R; ++i) ring[i] = read.by_row(qt, i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                S = mfma32<DT>(ring[i % R], kf[i], S);
                __builtin_amdgcn_sched_barrier(0);
                ring[i % R] = i + R < KS ? read.by_row(qt, i + R) : read.by_row(ot, i + R - KS);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (first == w0) {                                  // queries that do not see the key
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (8 * (i >> 2) + 4 * fh + (i & 3) < fr) S[i] = -INFINITY;
            }
            uint4 ps[2], ds[2];
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                dP = mfma32<DT>(ring[(KS + i) % R], vf[i], dP);
                __builtin_amdgcn_sched_barrier(0);
                if (i + R < KS) ring[(KS + i) % R] = read.by_row(ot, i + R);
#pragma unroll
                for (int j = 16 * i / KS; j < 16 * (i + 1) / KS; ++j) {
                    const f32x4 &r = ref[j / 2 % AHEAD];
                    S[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[j] - r[2 * (j & 1)], sc, r[2 * (j & 1) + 1]));
                    if ((j & 1) && j + 2 * AHEAD - 1 < 16) ref[j / 2 % AHEAD] = two_refs(j + 2 * AHEAD - 1);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            uint4 oc = read.by_column(ot, 0, 0), qc = read.by_column(qt, 0, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                auto scaled = [&](float v) { return DT == kFP16 ? v * factor : v; };
                put(ps, j, pack2<DT>(S[2 * j], S[2 * j + 1]));
                put(ds, j, pack2<DT>(S[2 * j] * scaled(dP[2 * j]), S[2 * j + 1] * scaled(dP[2 * j + 1])));
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 2 * CT; ++i) {
                const int k = i / CT, c = i % CT, n = i + 1;
                uint4 on{}, qn{};
                if (n < 2 * CT) { on = read.by_column(ot, 16 * (n / CT), n % CT); qn = read.by_column(qt, 16 * (n / CT), n % CT); }
                __builtin_amdgcn_sched_barrier(0);
                dv[c] = mfma32<DT>(oc, ps[k], dv[c]);
                dk[c] = mfma32<DT>(qc, ds[k], dk[c]);
                __builtin_amdgcn_sched_barrier(0);
                oc = on; qc = qn;
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
    float *rows = (float *)ws;                                  // of each query two numbers, then, of each, minus D
    RowTops *tops = (RowTops *)(rows + 3 * (size_t)pairs * seq);
    hipError_t err = hipSuccess;
    if constexpr (DT == kFP16) {
        attn_grad_tops_kernel<DH><<<dim3(pairs * row_tiles), dim3(256), 0, s>>>(qkv, dout, tops, seq, n_heads, row_tiles);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    const dim3 grid((pairs + 7) / 8 * 8 * tiles);
    auto queries = seq <= kShort ? attn_grad_queries_kernel<DT, DH, true> : attn_grad_queries_kernel<DT, DH, false>;
    queries<<<grid, dim3(256), 0, s>>>(qkv, out, dout, dqkv, rows, tops, seq, n_heads, pairs, tiles);
    if ((err = hipGetLastError()) != hipSuccess) return err;
    attn_grad_keys_kernel<DT, DH><<<grid, dim3(256), 0, s>>>(qkv, dout, dqkv, rows, tops, seq, n_heads, pairs, tiles);
    return hipGetLastError();
}

// ------------------------------------------------------------------ other heads and precisions
// A workgroup per query of a head: maximum and sum of the softmax over the keys it sees, D, dQ.  128 threads have a key each, then a channel each.
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
    const Acc one_over = (Acc)1 / block_sum(sum != (Acc)0 ? sum * (Acc)exp(top - most) : (Acc)0, red);
    Acc dq = 0;
    for (int k0 = 0; k0 <= q; k0 += 128) {
        const int k = k0 + tid;
        __syncthreads();
        ds[tid] = k <= q ? (Acc)exp(dot(0, k, 1) * scale - most) * one_over * (dot(1, k, 2) - delta) : (Acc)0;
        __syncthreads();
        const int n = q - k0 + 1 < 128 ? q - k0 + 1 : 128;
        if (mine)
            for (int j = 0; j < n; ++j) dq += ds[j] * P::a2acc(qkv[(first + k0 + j) * ld + d + tid]);
    }
    if (mine) ((A *)dqkv_)[row * ld + head * d_head + tid] = P::acc2a(dq * scale);
    if (tid == 0) {
        Acc *rows = (Acc *)rows_ + (size_t)head * n_rows + row;
        rows[0] = delta;
        rows[(size_t)n_heads * n_rows] = most;                 // (and the sum by itself: logsumexp would round it to the scores' last place)
        rows[2 * (size_t)n_heads * n_rows] = one_over;
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
    const Acc *delta = (const Acc *)rows_ + (size_t)head * n_rows + first, *most = delta + (size_t)n_heads * n_rows, *one_over = most + (size_t)n_heads * n_rows;
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
        ps[tid] = q < seq ? (Acc)exp(dot(0, qkv + (first + q) * ld) * scale - most[q]) * one_over[q] : (Acc)0;
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
        return 3 * 4 * pairs * seq + pairs * row_tiles * sizeof(RowTops);
    }
    if ((size_t)n_seq * seq >= (size_t)1 << 25 || n_heads > 65535) return 0;
    return 3 * acc_bytes(dtype) * pairs * seq;
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
