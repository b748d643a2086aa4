// The key-value cache in 4 bits: rows written and read, sparse attention over the selected rows, and the weight each got.
//
// A cache row holds one 576-element latent KV row in 400 bytes:
//   bytes   0..255  512 latent features as 4-bit floats c (sign, 2 exponent bits, 1 fraction bit: 0 .5 1 1.5 2 3 4 6),
//                   feature f in the low (f even) or high (f odd) half of byte f / 2
//   bytes 256..383  64 rotary features, bf16, as they came
//   bytes 384..387  biased exponents 127 + e_j of the features 128 j .. 128 j + 127, 255: the block is not a number
//   bytes 388..399  zero
// and stands for c * 2^e_j: e_j is the least e with max |x| <= 6 * 2^e, held to [-100, 100].  Scales are powers of two so
// that every value is a bf16 (2 significant bits) and nothing but the choice of c rounds: a reader multiplies exact values.
// One scale for 128 features is what the product with V can afford: there it goes into P (below), once per block and row;
// for N(0,1) features the relative error is 0.125, 0.117 with blocks of 32.
//
//   kv4_write_kernel  one wave per row: 16 lanes a block, its maximum by data-parallel moves, codes by the converting
//                     instruction (ties to the even code).  Bound by memory: 1152 bytes in, 400 out.
//   kv4_read_kernel   the way back to bf16, exact.
//   kv4_attn_kernel   O = softmax(sm_scale Q K^T) V over the rows that idx names.  See there.
//   kv4_probs_kernel  the heads' mean of that softmax per selected row, from the log-sum-exps.
#include <algorithm>
#include <cstddef>

#include "ic_common.hpp"

namespace ic {

namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
typedef __attribute__((ext_vector_type(2))) int i32x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;

constexpr int kRowB = IC_KV4_ROW_BYTES;
constexpr int kLat = 512, kRow = 576;
constexpr int kRopeOff = 256, kScaleOff = 384;
constexpr int kMinE = -100, kMaxE = 100;

// Row of the cache that holds logical position s of sequence b, or -1.
__device__ __forceinline__ int64_t kv4_row(const PagedView &pv, int b, int s, int len, int Lk, int64_t pool_rows)
{
    if (s < 0 || s >= len) return -1;
    const int64_t r = pv.page_table ? paged_row(pv, b, s) : (int64_t)b * Lk + s;
    return r >= 0 && r < pool_rows ? r : -1;
}

__device__ __forceinline__ int seq_len(const PagedView &pv, int b, int Lk)
{
    return pv.seq_lens ? min(pv.seq_lens[b], Lk) : Lk;
}

// (by value: a bit cast of a vector's element takes the vector's first)
__device__ __forceinline__ bf16x2 as_pair(unsigned int x) { return __builtin_bit_cast(bf16x2, x); }
__device__ __forceinline__ u16x2 as_u16x2(unsigned int x) { return __builtin_bit_cast(u16x2, x); }

// Maximum over the 16 lanes of a row, in every lane of it.
__device__ __forceinline__ float row16_max(float x)
{
    auto turn = [](float v, auto c) __attribute__((always_inline)) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(c)::value, 0xf, 0xf, true));
    };
    x = fmaxf(x, turn(x, std::integral_constant<int, 0x121>{}));            // row_ror:1, 2, 4, 8
    x = fmaxf(x, turn(x, std::integral_constant<int, 0x122>{}));
    x = fmaxf(x, turn(x, std::integral_constant<int, 0x124>{}));
    x = fmaxf(x, turn(x, std::integral_constant<int, 0x128>{}));
    return x;
}

__global__ __launch_bounds__(256) void kv4_write_kernel(Kv4RowsArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t n = (int64_t)a.B * a.Tn, stride = (int64_t)gridDim.x * 4;
    for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < n; r += stride) {
        const int b = (int)(r / a.Tn), i = (int)(r - (int64_t)b * a.Tn);
        const int len = seq_len(a.pv, b, a.Lk);
        const int64_t pos = a.pv.seq_lens ? (int64_t)len - a.Tn + i : a.pos0 + i;
        const int64_t row = pos < 0 || pos >= len ? -1 : kv4_row(a.pv, b, (int)pos, len, a.Lk, a.pool_rows);
        if (row < 0) continue;                                              // (wave-uniform)
        const unsigned short *src = (const unsigned short *)a.rows + r * kRow;
        const u32x4 x = *(const u32x4 *)(src + 8 * lane);                   // features 8 lane ..: 16 lanes a block
        const unsigned int rope = lane < 32 ? ((const unsigned int *)(src + kLat))[lane] : 0u;
        unsigned int top = 0;                                               // max |x| as bits: ordered as the values, NaN above inf
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned int lo = x[j] & 0x7FFFu, hi = (x[j] >> 16) & 0x7FFFu;
            top = max(top, max(lo, hi));
        }
        top = (unsigned int)row16_max((float)top);                          // (15-bit integers are exact in fp32)
        const bool finite = top < 0x7F80u;
        // least e with max <= 6 2^e = 1.5 2^(e+2); the bits of 1.5 are exponent 127, fraction 0x40
        const int e = max(kMinE, min(kMaxE, (int)((top + 0x3Fu) >> 7) - 127 - 2));
        const float scale = __uint_as_float((unsigned)(e + 127) << 23);
        unsigned int code = 0;
        if (finite) {
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(x[0]), scale, 0);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(x[1]), scale, 1);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(x[2]), scale, 2);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(x[3]), scale, 3);
        }
        const int byte = finite ? e + 127 : 255;
        unsigned char *dst = (unsigned char *)a.kv4 + row * kRowB;
        ((unsigned int *)dst)[lane] = code;
        const unsigned int scales = (unsigned)__builtin_amdgcn_readlane(byte, 0) | (unsigned)__builtin_amdgcn_readlane(byte, 16) << 8 |
                                    (unsigned)__builtin_amdgcn_readlane(byte, 32) << 16 | (unsigned)__builtin_amdgcn_readlane(byte, 48) << 24;
        if (lane < 36) ((unsigned int *)(dst + kRopeOff))[lane] = lane < 32 ? rope : (lane == 32 ? scales : 0u);
    }
}

__device__ __forceinline__ float scale_of(unsigned int byte)                // 2^(byte - 127), 255: NaN
{
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte << 23);
}

// eight codes -> eight bf16
__device__ __forceinline__ bf16x8 widen(unsigned int c, float scale)
{
    bf16x8 r;
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
    r[0] = p0[0]; r[1] = p0[1]; r[2] = p1[0]; r[3] = p1[1]; r[4] = p2[0]; r[5] = p2[1]; r[6] = p3[0]; r[7] = p3[1];
    return r;
}

__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4RowsArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t n = (int64_t)a.B * a.Tn, stride = (int64_t)gridDim.x * 4;
    for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < n; r += stride) {
        const int b = (int)(r / a.Tn), i = (int)(r - (int64_t)b * a.Tn);
        const int len = seq_len(a.pv, b, a.Lk);
        const int64_t pos = a.pv.seq_lens ? (int64_t)len - a.Tn + i : a.pos0 + i;
        const int64_t row = pos < 0 || pos >= len ? -1 : kv4_row(a.pv, b, (int)pos, len, a.Lk, a.pool_rows);
        unsigned short *dst = (unsigned short *)a.out + r * kRow;
        u32x4 v = u32x4{0u, 0u, 0u, 0u};
        unsigned int rope = 0;
        if (row >= 0) {
            const unsigned char *src = (const unsigned char *)a.kv4 + row * kRowB;
            const unsigned int code = ((const unsigned int *)src)[lane], byte = src[kScaleOff + (lane >> 4)];
            if (lane < 32) rope = ((const unsigned int *)(src + kRopeOff))[lane];
            v = byte == 255u ? u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u} : __builtin_bit_cast(u32x4, widen(code, scale_of(byte)));
        }
        *(u32x4 *)(dst + 8 * lane) = v;
        if (lane < 32) ((unsigned int *)(dst + kLat))[lane] = rope;
    }
}

// ---- attention ------------------------------------------------------------------------------------------------------
//
// A wave works alone on tiles of 32 selected rows, all 32 heads at once, with v_mfma_f32_32x32x16_bf16:
//   S [rows x heads] = K Q^T.   Q stays in registers (B operand, 144 registers).  The A operand wants eight features of a
//       row per lane: a lane reads 16 bytes, the codes of 32 features that share a scale, for four instructions; which
//       features an instruction contracts is free as long as K and Q agree.
//   O^T [features x heads] += V^T P^T.  P comes out of S in the layout that the B operand takes (lane = head; the rows of an
//       accumulator's 16 registers are the contraction index), so it never leaves the registers.  The A operand wants 8 rows
//       of one feature per lane: the 4-bit transposing LDS read hands a lane one feature of 16 rows.  Their scales differ by
//       row, and a conversion has one: V is converted without its scales, and P 2^(e_j), the rows' scales of block j, is what
//       V's block j is multiplied with.  P is bf16 there (as V is exact, the one rounding of the product: relative 2^-9); a
//       power of two is then a subtraction from its exponent, two rows an instruction.  It saturates at zero, and P is held
//       times 2^100 (kMaxE) so that the difference is never negative.
// The rows' bytes go from memory into LDS without passing through registers, three tiles of 12800 bytes per wave: 4-bit tiles
// are what lets all of this fit (a bf16 tile would be three times as large), and no wave waits for another.
// Registers: 256 of O^T, 144 of Q and about 100 more: one wave per SIMD.

constexpr int kT = 32;                        // rows of a tile
constexpr int kTileB = kT * kRowB;            // 12800
constexpr int kRing = 3;
constexpr float kPBias = 100.f;               // P is held times 2^100
constexpr float kLag = 12.f;                  // log2 units a row may exceed its reference before the sums are scaled anew: 2^(100 + 12 + 11)
                                              // (2048 rows) is still a float
constexpr int kAmount = (127 + 100) << 7;     // what the exponent byte b is subtracted from, as a bf16 exponent: (227 - b) << 7

// Rows m and m + 16 of a tile are 6400 bytes apart, the same LDS bank; the transposing read takes rows 0-3, 8-11, 16-19, 24-27
// (or the others) together, so the matrix row m >= 16 is the tile's row 16 + ((m - 16) ^ 4): then those are 16 different banks.
__device__ __forceinline__ int tile_row(int m) { return m ^ ((m & 16) >> 2); }

__device__ __forceinline__ unsigned int lds_offset(const void *p)
{
    return (unsigned int)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}

// All 32 rows of a tile, two per instruction: lanes 0-24 the first, 25-49 the second, 16 bytes each; LDS receives them one
// behind the other.  row: the cache row of tile row (lane & 31), -1: none (row 0 is fetched and not used).
__device__ __forceinline__ void fetch_tile(const unsigned char *kv4, int row, unsigned int lds, int lane)
{
    const int second = lane >= 25 ? 1 : 0, piece = lane - 25 * second;
    const int safe = row < 0 ? 0 : row;
    const unsigned char *base = kv4 + 16 * (piece < 25 ? piece : 0);
    if (lane < 50) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = __builtin_amdgcn_ds_bpermute(4 * (2 * i + second), safe);
            const unsigned char *p = base + (int64_t)r * kRowB;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds + i * 2 * kRowB), "v"(p) : "memory");
        }
    }
}

// The lane's number, worked out where it is needed: kept, it and what depends on it would take registers from O^T and Q.
__device__ __forceinline__ int lane_now()
{
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
    return l;
}

// 32 words (lanes 0-31) to LDS, one behind the other.
__device__ __forceinline__ void fetch_words(const int32_t *p, unsigned int lds, int lane)
{
    if (lane < 32) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(p) : "memory");
}

// What a wave fetches, tile after tile of all of its queries, ahead of what it computes: a step asks for the rows of the tile two
// steps on, the page numbers of the one four on and the entries of idx of the one six on, 18 instructions that leave nothing
// in registers.  Loads return in order, so 18 outstanding at the beginning of a step mean that everything from the step
// before the last has arrived.  (Nothing else loads within the loop over a query's tiles.)
constexpr int kAhead = 18;
struct Words {
    int32_t idx[8][kT], page[4][kT];          // of tile n in [n % 8], [n % 4]
};
struct Cursor {
    int q;                                    // query row; n_queries and more: none
    int tile, b, len;                         // len: 0 where there is no such tile
};

template <int W>
struct Fetch {
    const Kv4AttnArgs &a;
    Words *words;
    unsigned int words0, ring0;               // LDS
    int nq, stride;                           // (B Tq is below 2^30, a stride 1024 at most)
    int s0, s1, n_tiles, first;
    Cursor rows, pages, ids;
    unsigned int n;                           // tile number of `rows`

    __device__ __forceinline__ Fetch(const Kv4AttnArgs &a_, Words *w, unsigned int ring, int q, int stride_, int split, int first_)
        : a(a_), words(w), ring0(ring), nq(a_.B * a_.Tq), stride(stride_), first(first_)
    {
        words0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_offset(w));
        s0 = split * a.split_len;
        s1 = min(s0 + a.split_len, a.k_sel);
        n_tiles = (s1 - s0 + kT - 1) / kT;
        rows.q = q;
        rows.tile = first;
        place(rows);
        pages = ids = rows;
        n = 0;
    }
    __device__ __forceinline__ void place(Cursor &c) const
    {
        const bool there = c.q < nq && c.tile < n_tiles;
        c.b = there ? (int)((unsigned)c.q / (unsigned)a.Tq) : 0;
        c.len = there ? (a.pv.seq_lens ? min(load_uniform(a.pv.seq_lens + c.b), a.Lk) : a.Lk) : 0;
    }
    __device__ __forceinline__ void next(Cursor &c) const
    {
        c.tile += W;
        if (c.tile >= n_tiles) {
            c.tile = first;
            c.q += W == 1 ? stride : nq;      // (waves that share a query have one)
            place(c);
        }
    }
    __device__ __forceinline__ void ask_ids(unsigned int m, int lane)
    {
        const int64_t q = min(ids.q, nq - 1);
        const int s = min(s0 + ids.tile * kT + (lane & 31), a.k_sel - 1);
        fetch_words(a.idx + q * a.k_sel + s, words0 + (m & 7) * (kT * 4), lane);
        next(ids);
    }
    __device__ __forceinline__ void ask_pages(unsigned int m, int lane)
    {
        const int s = words->idx[m & 7][lane & 31];
        const int32_t *p = a.idx;             // (not paged: any word)
        if (a.pv.page_table) p = a.pv.page_table + (int64_t)pages.b * a.pv.max_pages + (s >= 0 && s < pages.len ? s >> a.pv.page_shift : 0);
        fetch_words(p, words0 + (unsigned)offsetof(Words, page) + (m & 3) * (kT * 4), lane);
        next(pages);
    }
    // the rows of tile m into LDS at `at`; returns which of them there are
    __device__ __forceinline__ unsigned int ask_rows(unsigned int m, unsigned int at, int lane)
    {
        const int s = words->idx[m & 7][lane & 31], page = words->page[m & 3][lane & 31];
        const int slot = s0 + rows.tile * kT + (lane & 31);
        int64_t r = a.pv.page_table ? ((int64_t)page << a.pv.page_shift) + (s & ((1 << a.pv.page_shift) - 1)) : (int64_t)rows.b * a.Lk + s;
        const bool there = slot < s1 && s >= 0 && s < rows.len && r >= 0 && r < a.pool_rows;
        fetch_tile((const unsigned char *)a.KV4, there ? (int)r : -1, ring0 + at, lane);
        next(rows);
        return (unsigned int)__ballot(there);
    }
};

__device__ __forceinline__ float half_max(float x) { return fmaxf(x, __shfl_xor(x, 32)); }
__device__ __forceinline__ float half_sum(float x) { return x + __shfl_xor(x, 32); }

// O^T times a factor per head.  The accumulators live in registers that only matrix instructions and moves reach, and the asm
// that reads them brings its own wait for the matrix instruction before it.
__device__ __forceinline__ void scale_tiles(f32x16 (&o)[16], float f)
{
    asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");
#pragma unroll
    for (int t = 0; t < 16; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float x;
            asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(o[t][i]));
            x *= f;
            asm volatile("v_accvgpr_write_b32 %0, %1" : "=a"(o[t][i]) : "v"(x));
        }
    asm volatile("s_nop 7\n\ts_nop 7" ::: "memory");
}

// Four registers of a tile of O^T, times f: read where they are used (all 256 at once would displace everything else).
__device__ __forceinline__ f32x4 read4(const f32x16 &o, int i4, float f)
{
    f32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float x;
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(o[4 * i4 + e]));
        y[e] = x * f;
    }
    return y;
}

// Four products into an accumulator that lives in ordinary registers: O^T takes all of the accumulation registers, and left to
// itself the compiler puts every accumulator there.  It knows nothing of these instructions' timing, so each brings the two
// wait states behind the conversions that wrote its operands, and the last the wait for its result.
__device__ __forceinline__ void mfma4_first(f32x16 &s, bf16x8 a0, bf16x8 a1, bf16x8 a2, bf16x8 a3, const bf16x8 (&b)[4])
{
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %5, 0\n\tv_mfma_f32_32x32x16_bf16 %0, %2, %6, %0\n\t"
        "v_mfma_f32_32x32x16_bf16 %0, %3, %7, %0\n\tv_mfma_f32_32x32x16_bf16 %0, %4, %8, %0"
        : "=&v"(s) : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]));
}
__device__ __forceinline__ void mfma4(f32x16 &s, bf16x8 a0, bf16x8 a1, bf16x8 a2, bf16x8 a3, const bf16x8 (&b)[4])
{
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %5, %0\n\tv_mfma_f32_32x32x16_bf16 %0, %2, %6, %0\n\t"
        "v_mfma_f32_32x32x16_bf16 %0, %3, %7, %0\n\tv_mfma_f32_32x32x16_bf16 %0, %4, %8, %0"
        : "+v"(s) : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]));
}
__device__ __forceinline__ void mfma4_last(f32x16 &s, bf16x8 a0, bf16x8 a1, bf16x8 a2, bf16x8 a3, const bf16x8 (&b)[4])
{
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %5, %0\n\tv_mfma_f32_32x32x16_bf16 %0, %2, %6, %0\n\t"
        "v_mfma_f32_32x32x16_bf16 %0, %3, %7, %0\n\tv_mfma_f32_32x32x16_bf16 %0, %4, %8, %0\n\ts_nop 15\n\ts_nop 7"
        : "+v"(s) : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]));
}

// W waves of the workgroup share a (query, split): each takes every W-th tile and they meet at the end.
template <int W>
__global__ __launch_bounds__(256, 1) void kv4_attn_kernel(Kv4AttnArgs a)
{
    __shared__ __attribute__((aligned(16))) unsigned char ring[4][kRing][kTileB];
    __shared__ __attribute__((aligned(16))) unsigned short amounts[4][2][4][2][16];   // [wave][turn][block][half][register]
    __shared__ Words words[4];
    __shared__ float wave_ml[4][2][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5;
    const int nq = a.B * a.Tq;
    // W = 1: the waves of an XCD (every eighth workgroup) walk through neighbouring queries, whose selections overlap
    const int wg = (int)blockIdx.x, wgs = (int)gridDim.x;
    const int q0 = W > 1 ? wg / a.n_splits : (wgs & 7) == 0 ? ((wg & 7) * (wgs >> 3) + (wg >> 3)) * 4 + wave : wg * 4 + wave;
    const int split = W > 1 ? wg - q0 * a.n_splits : 0;
    if (W == 1 && q0 >= nq) return;
    Fetch<W> f(a, &words[wave], (unsigned)__builtin_amdgcn_readfirstlane((int)lds_offset(&ring[wave][0][0])), q0, wgs * 4, split, W == 1 ? 0 : wave);
#pragma unroll
    for (unsigned int i = 0; i < 6; ++i) f.ask_ids(i, lane);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (unsigned int i = 0; i < 4; ++i) f.ask_pages(i, lane);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    unsigned int ok0 = f.ask_rows(0, 0, lane), ok1 = f.ask_rows(1, kTileB, lane);       // rows that the tiles in the ring have
    unsigned int n = 0, at = 0, at2 = 2 * kTileB;                           // tile number; in the ring: the tile, the one two behind it
#pragma unroll 1
  for (int q = q0; q < nq; q += f.stride) {
    // Q as the B operand: head l32; chunk j, step s: features 64 j + 32 g + 8 s ..; then the rotary ones, 16 r + 8 g ..  (Lanes
    // without a head take the first one, and write nothing.)
    bf16x8 ql[8][4], qr[4];
    {
        const unsigned short *qp = (const unsigned short *)a.Q + ((int64_t)q * a.H_q + (l32 < a.H_q ? l32 : 0)) * kRow;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int s = 0; s < 4; ++s)
                ql[j][s] = *(const bf16x8 *)(qp + 64 * j + 32 * g + 8 * s);
#pragma unroll
        for (int r = 0; r < 4; ++r) qr[r] = *(const bf16x8 *)(qp + kLat + 16 * r + 8 * g);
    }

    f32x16 o[16];
#pragma unroll
    for (int t = 0; t < 16; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    // (Q has arrived before the loop, which must not wait for it, and is in these registers throughout)
    auto pin = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(ql[j][0]), "+v"(ql[j][1]), "+v"(ql[j][2]), "+v"(ql[j][3]));
        asm volatile("" : "+v"(qr[0]), "+v"(qr[1]), "+v"(qr[2]), "+v"(qr[3]));
    };
    pin();
#pragma unroll 1
    for (int t = f.first; t < f.n_tiles; t += W) {
#pragma unroll
        for (int t2 = 0; t2 < 16; ++t2) asm volatile("" : "+a"(o[t2]));
        pin();
        const unsigned char *buf = &ring[wave][0][0] + at;
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kAhead) : "memory");   // (and the reads of the ring's free tile are through)
        const int ln = lane_now(), l32 = ln & 31, g = ln >> 5;
        const unsigned int ok2 = f.ask_rows(n + 2, at2, ln);
        f.ask_pages(n + 4, ln);
        f.ask_ids(n + 6, ln);
        ++n;
        const unsigned int ok = ok0;                                        // bit: tile row
        ok0 = ok1;
        ok1 = ok2;
        at = at == 2 * kTileB ? 0 : at + kTileB;
        at2 = at2 == 2 * kTileB ? 0 : at2 + kTileB;
        if (ok == 0u) continue;
        // S = K Q^T
        const unsigned char *kp = buf + tile_row(l32) * kRowB;
        const unsigned int sc = *(const unsigned int *)(kp + kScaleOff);
        {                                       // the subtractions of P's exponents, in the order of the accumulator's registers
            const int reg = 4 * (l32 >> 3) + (l32 & 3), half = (l32 >> 2) & 1;
            if (g == 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    amounts[wave][0][j][half][reg] = (unsigned short)(kAmount - (int)(((sc >> (8 * j)) & 255u) << 7));
            }
        }
        f32x16 s;
        u32x4 kc[2];                            // (what is read ahead is bounded by hand: the compiler counts on registers that O^T has)
        kc[0] = *(const u32x4 *)(kp + g * 16);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j < 7) kc[(j + 1) & 1] = *(const u32x4 *)(kp + (2 * (j + 1) + g) * 16);
            const u32x4 c = kc[j & 1];
            const float f = scale_of((sc >> (8 * (j >> 1))) & 255u);
            if (j == 0)
                mfma4_first(s, widen(c[0], f), widen(c[1], f), widen(c[2], f), widen(c[3], f), ql[j]);
            else
                mfma4(s, widen(c[0], f), widen(c[1], f), widen(c[2], f), widen(c[3], f), ql[j]);
            __builtin_amdgcn_sched_barrier(0);
        }
        mfma4_last(s, *(const bf16x8 *)(kp + kRopeOff + 16 * g), *(const bf16x8 *)(kp + kRopeOff + 32 + 16 * g), *(const bf16x8 *)(kp + kRopeOff + 64 + 16 * g),
                   *(const bf16x8 *)(kp + kRopeOff + 96 + 16 * g), qr);
        __builtin_amdgcn_sched_barrier(0);
        // register i is matrix row 8 (i / 4) + 4 g + i % 4
        if (ok != 0xFFFFFFFFu) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int tr = 8 * (i >> 2) + 4 * (i < 8 ? g : 1 - g) + (i & 3);
                s[i] = (ok >> tr) & 1u ? s[i] * a.scale_log2e : -INFINITY;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] *= a.scale_log2e;
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        top = half_max(top);
        if (__ballot(top > m + kLag) != 0ull) {                             // (m = -inf: the first rows)
            const float mn = fmaxf(m, top), keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= keep;
            scale_tiles(o, keep);
        }
        const float ref = m == -INFINITY ? 0.f : m - kPBias;
        u16x2 p[8];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float p0 = __builtin_amdgcn_exp2f(s[i] - ref), p1 = __builtin_amdgcn_exp2f(s[i + 1] - ref);
            l += p0 + p1;
            p[i >> 1] = __builtin_bit_cast(u16x2, __builtin_convertvector((f32x2{p0, p1}), bf16x2));
        }
        // O^T += V^T P^T
        const int vm = 8 * ((ln & 15) >> 2) + 4 * g + (ln & 3);
        const unsigned char *vp = buf + tile_row(vm) * kRowB + ((ln >> 4) & 1) * 8;
        typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
        i32x2 vc[2];
        vc[0] = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2 *)vp);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4 d[2];
            d[0] = *(const u32x4 *)&amounts[wave][0][j][g][0];
            d[1] = *(const u32x4 *)&amounts[wave][0][j][g][8];
            u32x4 pj[2];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                pj[i >> 2][i & 3] = __builtin_bit_cast(unsigned int, __builtin_elementwise_sub_sat(p[i], as_u16x2(d[i >> 2][i & 3])));
#pragma unroll
            for (int t4 = 0; t4 < 4; ++t4) {
                const int ft = 4 * j + t4;
                if (ft < 15) vc[(ft + 1) & 1] = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2 *)(vp + (ft + 1) * 16));
                const i32x2 c = vc[ft & 1];
                o[ft] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen((unsigned)c[0], 1.f), __builtin_bit_cast(bf16x8, pj[0]), o[ft], 0, 0, 0);
                o[ft] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen((unsigned)c[1], 1.f), __builtin_bit_cast(bf16x8, pj[1]), o[ft], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");              // (the last products, before their sums are read)
    l = half_sum(l);

    float mine = 1.f;                          // weight of this wave's part
    if constexpr (W > 1) {
        // the waves' parts: weights by their maxima, then each wave sums a quarter of the features, in two rounds through the rings
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                    // nothing more arrives in the rings
        __syncthreads();
        if (g == 0) {
            wave_ml[wave][0][l32] = m;
            wave_ml[wave][1][l32] = l;
        }
        __syncthreads();
        float mt = -INFINITY, lt = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) mt = fmaxf(mt, wave_ml[w][0][l32]);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float mw = wave_ml[w][0][l32];
            lt += mw == -INFINITY ? 0.f * wave_ml[w][1][l32] : wave_ml[w][1][l32] * __builtin_amdgcn_exp2f(mw - mt);
        }
        mine = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mt);
        m = mt;
        l = lt;
    }
    const float inv = l == 0.f ? 0.f : 0x1p100f / l;                        // (the sums of P V are without the bias)
    const bool mine_h = l32 < a.H_q;
    const int64_t head = (int64_t)q * a.H_q + l32, part = ((int64_t)q * a.n_splits + split) * a.H_q + l32;
    // features 32 ft + 8 i4 + 4 g + 0 .. 3 of the head
    auto store = [&](int ft, int i4, f32x4 y) __attribute__((always_inline)) {
        const int f = 32 * ft + 8 * i4 + 4 * g;
        if (!mine_h) return;
        if (W > 1 && a.n_splits > 1) {
            *(f32x4 *)((float *)a.part_o + part * kLat + f) = y * inv;
        } else {
            typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
            *(bf16x4 *)((__bf16 *)a.O + head * kLat + f) = __builtin_convertvector(y * inv, bf16x4);
        }
    };
    if constexpr (W == 1) {
#pragma unroll
        for (int ft = 0; ft < 16; ++ft)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) store(ft, i4, read4(o[ft], i4, 1.f));
    } else {
        f32x4 *sh = (f32x4 *)&ring[0][0][0];   // [from][owner][tile of the round][register / 4][lane]
#pragma unroll
        for (int round = 0; round < 2; ++round) {
#pragma unroll
            for (int w = 0; w < W; ++w)
                if (w != wave)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i4 = 0; i4 < 4; ++i4) sh[(((wave * 4 + w) * 2 + k) * 4 + i4) * 64 + lane] = read4(o[4 * w + 2 * round + k], i4, mine);
            __syncthreads();
#pragma unroll
            for (int w = 0; w < W; ++w)
                if (w == wave)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i4 = 0; i4 < 4; ++i4) {
                            f32x4 x = read4(o[4 * w + 2 * round + k], i4, mine);
#pragma unroll
                            for (int from = 0; from < W; ++from)
                                if (from != w) x += sh[(((from * 4 + w) * 2 + k) * 4 + i4) * 64 + lane];
                            store(4 * w + 2 * round + k, i4, x);
                        }
            if (round == 0) __syncthreads();
        }
    }
    if (g == 0 && mine_h && (W == 1 || wave == 0)) {
        if (W > 1 && a.n_splits > 1) {
            a.part_ml[2 * part] = l == 0.f ? -INFINITY : (l != l ? l : m);   // (the merge leaves out what has no maximum)
            a.part_ml[2 * part + 1] = l * 0x1p-100f;
        } else if (a.lse) {
            a.lse[head] = l == 0.f ? -INFINITY : (m + __builtin_log2f(l) - kPBias) * 0.6931471805599453f;
        }
    }
    if (W > 1) break;                          // (one query)
  }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// ---- the weight each selected row received --------------------------------------------------------------------------
//
// probs[q, slot] = 1/H sum_h exp(sm_scale <Q[h], K[row]> - lse[h]).  The same tiles as above with the operands exchanged:
// heads are the matrix rows, cache rows the columns, so a lane holds 16 heads of one cache row and adds them up by itself.
__global__ __launch_bounds__(256, 1) void kv4_probs_kernel(Kv4AttnArgs a)
{
    __shared__ __attribute__((aligned(16))) unsigned char ring[4][kRing][kTileB];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int l32 = lane & 31, g = lane >> 5;
    const int64_t q = blockIdx.x / a.n_splits;
    const int split = (int)(blockIdx.x - q * a.n_splits);
    const int b = (int)(q / a.Tq);
    const int len = seq_len(a.pv, b, a.Lk);
    const int s0 = split * a.split_len, s1 = min(s0 + a.split_len, a.k_sel);
    const int32_t *idx = a.idx + q * a.k_sel;
    const unsigned char *kv4 = (const unsigned char *)a.KV4;
    bf16x8 ql[8][4], qr[4];
    float off[16];                              // of head 8 (i / 4) + 4 g + i % 4, log2 units
    {
        const unsigned short *qp = (const unsigned short *)a.Q + (q * a.H_q + (l32 < a.H_q ? l32 : 0)) * kRow;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int s = 0; s < 4; ++s)
                ql[j][s] = *(const bf16x8 *)(qp + 64 * j + 32 * g + 8 * s);
#pragma unroll
        for (int r = 0; r < 4; ++r) qr[r] = *(const bf16x8 *)(qp + kLat + 16 * r + 8 * g);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int h = 8 * (i >> 2) + 4 * g + (i & 3);
            off[i] = h < a.H_q ? a.lse[q * a.H_q + h] * 1.4426950408889634f : INFINITY;
        }
    }
    const float inv_h = 1.f / (float)a.H_q;
    auto row_of = [&](int tile) -> int {
        const int s = s0 + tile * kT + l32;
        if (s >= s1) return -1;
        return (int)kv4_row(a.pv, b, idx[s], len, a.Lk, a.pool_rows);
    };
    const int n_tiles = (s1 - s0 + kT - 1) / kT;
    const unsigned int ring0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_offset(&ring[wave][0][0]));
    int row0 = wave < n_tiles ? row_of(wave) : -1, row1 = wave + 4 < n_tiles ? row_of(wave + 4) : -1;
    fetch_tile(kv4, row0, ring0, lane);
    fetch_tile(kv4, row1, ring0 + kTileB, lane);
    unsigned int rat = 0, rat2 = 2 * kTileB;
#pragma unroll 1
    for (int t = wave; t < n_tiles; t += 4) {
        const int row2 = t + 8 < n_tiles ? row_of(t + 8) : -1;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        fetch_tile(kv4, row2, ring0 + rat2, lane);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * 16) : "memory");
        const unsigned char *kp = &ring[wave][0][0] + rat + l32 * kRowB;
        const unsigned int sc = *(const unsigned int *)(kp + kScaleOff);
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const u32x4 c = *(const u32x4 *)(kp + (2 * j + g) * 16);
            const float f = scale_of((sc >> (8 * (j >> 1))) & 255u);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ql[j][e], widen(c[e], f), s, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const bf16x8 k = *(const bf16x8 *)(kp + kRopeOff + 32 * r + 16 * g);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qr[r], k, s, 0, 0, 0);
        }
        float p = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (off[i] != INFINITY) p += __builtin_amdgcn_exp2f(s[i] * a.scale_log2e - off[i]);
        p = half_sum(p);
        const int at = s0 + t * kT + l32;
        if (g == 0 && at < s1) a.probs[q * a.k_sel + at] = row0 >= 0 ? p * inv_h : 0.f;
        row0 = row1;
        row1 = row2;
        rat = rat == 2 * kTileB ? 0 : rat + kTileB;
        rat2 = rat2 == 2 * kTileB ? 0 : rat2 + kTileB;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

unsigned rows_grid(const Kv4RowsArgs &a)
{
    const int64_t wgs = ((int64_t)a.B * a.Tn + 3) / 4;
    return (unsigned)(wgs < (1 << 20) ? wgs : 1 << 20);
}

} // namespace

hipError_t launch_kv4_write(const Kv4RowsArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(kv4_write_kernel, dim3(rows_grid(a)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4RowsArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(kv4_read_kernel, dim3(rows_grid(a)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_kv4_attn(const Kv4AttnArgs &a, bool together, hipStream_t st)
{
    const int64_t units = (int64_t)a.B * a.Tq * a.n_splits;
    if (together)
        hipLaunchKernelGGL((kv4_attn_kernel<4>), dim3((unsigned)units), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((kv4_attn_kernel<1>), dim3((unsigned)std::min<int64_t>(256, (units + 3) / 4)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_kv4_probs(const Kv4AttnArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(kv4_probs_kernel, dim3((unsigned)((int64_t)a.B * a.Tq * a.n_splits)), dim3(256), 0, st, a);
    return hipGetLastError();
}

} // namespace ic
