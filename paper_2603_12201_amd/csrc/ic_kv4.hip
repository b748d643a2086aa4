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
// for N(0,1) features the relative error is 0.125, and 0.115 with blocks of 32.
//
//   kv4_write_kernel  one wave per row: 16 lanes a block, its maximum by data-parallel moves, codes by the converting
//                     instruction (ties to the even code).  Bound by memory: 1152 bytes in, 400 out; 131072 rows 41 to
//                     45 us, 4.5 to 4.9 TB/s, what a large copy reaches.
//   kv4_read_kernel   the way back to bf16, exact: the same rows in 31 us behind the former.
//   kv4_attn_kernel, kv4_attn_few_kernel
//                     O = softmax(sm_scale Q K^T) V over the rows that idx names.  See there.
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
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
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

// Row of the cache that row i of sequence b goes to, or -1.
__device__ __forceinline__ int64_t row_of(const Kv4RowsArgs &a, int b, int i)
{
    const int n = a.pv.seq_lens ? a.pv.seq_lens[b] : a.Lk, len = min(n, a.Lk);
    const int64_t pos = a.pv.seq_lens ? (int64_t)n - a.Tn + i : a.pos0 + i;   // (n may be beyond Lk: the rows there are left out)
    return pos < 0 || pos >= len ? -1 : kv4_row(a.pv, b, (int)pos, len, a.Lk, a.pool_rows);
}

// (by value: a bit cast of a vector's element takes the vector's first)
__device__ __forceinline__ bf16x2 as_pair(unsigned int x) { return __builtin_bit_cast(bf16x2, x); }
__device__ __forceinline__ float as_float(unsigned int x) { return __uint_as_float(x); }
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
        const int64_t row = row_of(a, b, i);
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

// 2^(byte - 127); 255 makes an infinity of it, with which the conversion gives a NaN for every code
__device__ __forceinline__ float scale_of(unsigned int byte) { return __uint_as_float(byte << 23); }

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
        const int64_t row = row_of(a, b, i);
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
//       V's block j is multiplied with.  P is bf16 there (as V is exact, the one rounding of the product: relative 2^-8); a
//       power of two is then a subtraction from its exponent, two rows an instruction.  It saturates at zero, and P is held
//       times 2^100 (kMaxE) so that the difference is never negative.
// The rows' bytes go from memory into LDS without passing through registers; the codes of four tiles, 8 KB each, and the
// rotary part of one are what a wave has there: bf16 tiles would be three times as large.  No wave waits for another.
// 32768 queries of 2048 rows: 4.7 to 4.8 ms, 940 to 965 TFLOP/s where a plain product of 8192^3 reaches 1141.  Bound by issue: an instruction
// takes a wave 4.3 to 4.7 clocks, a product 13, and a tile has some 850, 68 of them products (without the fetches 4.2 ms; the fetches alone 2.4).
// Registers: 256 of O^T, 144 of Q and about 100 more: one wave per SIMD, which issues in order, so the 68 matrix instructions
// of a tile (32 clocks each) have the rest, about 6 vector instructions each, dealt out between them by hand: a step multiplies
// K of one tile and V of the tile before it, and works out the softmax of the former during the latter.
// The reference of the softmax is the running maximum, but followed only when a row exceeds it by more than a.lag (log2
// units): 12 while k_sel rows times 6 2^(100 + 12) is a float (k_sel <= 8192), 0 above.

constexpr int kT = 32;                        // rows of a tile
constexpr int kCodeB = kT * 256, kRopeB = kT * 128;
constexpr int kRing = 4;                      // tiles whose codes are in LDS
constexpr float kPBias = 100.f;               // P is held times 2^100
constexpr int kAmount = (127 + 100) << 7;     // what the exponent byte b is subtracted from, as a bf16 exponent: (227 - b) << 7

// What a wave has in LDS.  Rows lie 256 (128) bytes apart, so a row's 16-byte pieces are stored in an order of its own, piece c
// of row r at c ^ (r % 16) (of the rotary part at c ^ (r / 2 % 8)): 16 rows' pieces c then are in 16 different bank groups.
// The transposing read takes matrix rows 0-3, 8-11, 16-19, 24-27 (or the others) together, so the matrix row m >= 16 is the
// tile's row 16 + ((m - 16) ^ 4): those too are 16 different r % 16.
struct Tiles {
    static constexpr int kSlotB = kCodeB;     // from a tile of the ring to the next
    unsigned char code[4][kRing][kCodeB];     // [wave]
    __device__ __forceinline__ unsigned char *codes(int wave) { return &code[wave][0][0]; }
    unsigned char rope[4][kRopeB];
    int32_t idx[4][8][kT], page[4][4][kT];    // of tile n in [n % 8], [n % 4]
    unsigned int scale[4][4][kT];             // the rows' four exponent bytes, tile n in [n % 4]
    unsigned short amount[4][2][4][2][16];    // what is subtracted from P: tile n in [n % 2][block][half][register of the accumulator]
    unsigned int code_at[4][4][8];            // where the rows of the tile that is asked for next are: row 4 i + k at [k][i],
    unsigned int rope_at[4][2][8][4];         // row 8 i + k at [n % 2][k][i]
};
__device__ __forceinline__ int tile_row(int m) { return m ^ ((m & 16) >> 2); }

__device__ __forceinline__ unsigned int lds_offset(const void *p)
{
    return (unsigned int)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}

// The lane's number, worked out where it is needed: kept, it and what depends on it would take registers from O^T and Q.
__device__ __forceinline__ int lane_now()
{
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
    return l;
}

// 16 bytes per lane, or 4 for lanes 0-31, to LDS at lds + at, one behind the other; from an address of its own, or a base and an
// offset r + piece.  (All 64 lanes are active where these are called.  m0 is written two instructions ahead of its use.)
__device__ __forceinline__ void to_lds16(const void *p, unsigned int lds, int at)
{
    asm volatile("s_add_u32 m0, %0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p), "s"(at) : "memory", "scc");
}
__device__ __forceinline__ void to_lds16(const void *base, unsigned int r, unsigned int piece, unsigned int lds, int at)
{
    unsigned int off;
    asm volatile("s_add_u32 m0, %1, %4\n\tv_add_u32 %0, %2, %3\n\tglobal_load_lds_dwordx4 %0, %5" : "=&v"(off) : "s"(lds), "v"(r), "v"(piece), "i"(at), "s"(base) : "memory", "scc");
}
__device__ __forceinline__ void to_lds4(const void *p, unsigned int lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b32 exec_hi, 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b32 exec_hi, -1" ::"s"(lds), "v"(p) : "memory");
}
__device__ __forceinline__ void to_lds4(const void *base, unsigned int off, unsigned int lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b32 exec_hi, 0\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b32 exec_hi, -1" ::"s"(lds), "v"(off), "s"(base) : "memory");
}

// What a wave fetches, tile after tile of all of its queries, ahead of what it computes.  In the step of tile n, in this order:
// the codes of tile n + 2 (8 instructions), the page numbers of n + 4, the entries of idx of n + 6, a wait for all but these
// and the one before them (kAhead), and when tile n's rotary part has been read that of n + 1 (4) and the exponents of n + 3.  Nothing of
// it passes through registers, loads return in order, and nothing else loads within the loop over a query's tiles: behind the
// wait, everything that earlier steps have asked for but their last has arrived.  (Without a page table nothing asks for page numbers.
// kv4_attn_few_kernel has an order of its own, given there.)
struct Cursor {
    int q;                                    // query row; n_queries and more: none
    int tile, b, len;                         // len: 0 where there is no such query
};

// W waves share a query: each takes every W-th tile.  WIDE: rows behind 4 GB, in the 32-bit offsets of the others they are not.
template <int W, bool PAGED, bool WIDE, typename LDS>
struct Fetch {
    static constexpr int kAhead = 10 + PAGED; // what may be on its way behind the wait
    const Kv4AttnArgs &a;
    LDS &lds;
    unsigned int code0, rope0, idx0, page0, scale0;   // LDS addresses of this wave's
    int wave;
    int nq, stride;                           // (B Tq is below 2^30, a stride 1024 at most)
    int s0, n_slots, n_tiles, first;
    Cursor rows, pages, ids;
    const int32_t *ids_at;                    // idx of the query at `ids`

    __device__ __forceinline__ Fetch(const Kv4AttnArgs &a_, LDS &lds_, int wave_, int q, int stride_, int split, int first_)
        : a(a_), lds(lds_), wave(wave_), nq(a_.B * a_.Tq), stride(stride_), first(first_)
    {
        auto at = [](const void *p) { return (unsigned)__builtin_amdgcn_readfirstlane((int)lds_offset(p)); };
        code0 = at(lds.codes(wave));
        rope0 = at(&lds.rope[wave][0]);
        idx0 = at(&lds.idx[wave][0][0]);
        page0 = at(&lds.page[wave][0][0]);
        scale0 = at(&lds.scale[wave][0][0]);
        s0 = split * a.split_len;
        n_slots = min(a.split_len, a.k_sel - s0);
        n_tiles = (n_slots + kT - 1) / kT;
        rows.q = q;
        rows.tile = first;
        place(rows);
        pages = ids = rows;
        ids_at = a.idx + ((int64_t)min(q, nq - 1) * a.k_sel + s0);
    }
    __device__ __forceinline__ void place(Cursor &c) const
    {
        const bool there = c.q < nq && c.tile < n_tiles;
        c.b = there ? (int)((unsigned)c.q / (unsigned)a.Tq) : 0;
        c.len = there ? (a.pv.seq_lens ? max(0, min(load_uniform(a.pv.seq_lens + c.b), a.Lk)) : a.Lk) : 0;
    }
    __device__ __forceinline__ bool next(Cursor &c) const
    {
        c.tile += W;
        if (c.tile < n_tiles) return false;
        c.tile = first;
        c.q += W == 1 ? stride : nq;          // (waves that share a query have one)
        place(c);
        return true;
    }
    __device__ __forceinline__ void next_ids()
    {
        if (next(ids)) ids_at = a.idx + ((int64_t)min(ids.q, nq - 1) * a.k_sel + s0);
    }
    __device__ __forceinline__ void advance()
    {
        next(rows);
        if (PAGED) next(pages);
        next_ids();
    }
    __device__ __forceinline__ void ask_ids(unsigned int m, int lane) const
    {
        const int t = min(ids.tile, n_tiles - 1) * kT;                      // (a wave without a tile asks for the last one)
        to_lds4(ids_at + t, 4u * min(lane & 31, n_slots - 1 - t), idx0 + (m & 7) * (kT * 4));
    }
    __device__ __forceinline__ int entry(unsigned int m, int lane) const { return lds.idx[wave][m & 7][lane & 31]; }
    __device__ __forceinline__ int page(unsigned int m, int lane) const { return PAGED ? lds.page[wave][m & 3][lane & 31] : 0; }
    __device__ __forceinline__ void ask_pages(unsigned int m, int s) const        // s: entry() of tile m
    {
        if (PAGED)
            to_lds4(a.pv.page_table + (int64_t)pages.b * a.pv.max_pages, (unsigned)s < (unsigned)pages.len ? 4u * (unsigned)(s >> a.pv.page_shift) : 0u,
                    page0 + (m & 3) * (kT * 4));
    }
    // Finds the rows of the tile m at `rows` (s and pg: its entry() and page()), asks for their exponents and leaves where they are
    // for ask_code() and ask_rope(): row numbers (WIDE) or byte offsets, of row 0 where there is none.  Returns which there are.
    __device__ __forceinline__ unsigned int find_rows(unsigned int m, int s, int pg, int lane)
    {
        bool there = ((unsigned)s < (unsigned)rows.len) & ((lane & 31) < n_slots - rows.tile * kT);
        unsigned int r;
        if (PAGED) {
            const unsigned int last = (unsigned)(a.pool_rows - 1);
            r = ((unsigned)pg << a.pv.page_shift) + ((unsigned)s & ((1u << a.pv.page_shift) - 1u));
            there = there & ((unsigned)pg <= last >> a.pv.page_shift) & (r <= last);
        } else {
            r = (unsigned)(rows.b * a.Lk) + (unsigned)s;                    // (B Lk <= pool_rows < 2^31)
        }
        r = there ? (WIDE ? r : r * (unsigned)kRowB) : 0u;
        const int k = lane & 31;
        lds.code_at[wave][k & 3][k >> 2] = r;                               // (both halves of the lanes write the same)
        lds.rope_at[wave][m & 1][k & 7][k >> 3] = r;
        if (WIDE)
            to_lds4((const unsigned char *)a.KV4 + ((uint64_t)r * kRowB + kScaleOff), scale0 + (m & 3) * (kT * 4));
        else
            to_lds4(a.KV4, r + kScaleOff, scale0 + (m & 3) * (kT * 4));
        return (unsigned int)__ballot(there);
    }
    template <int AT> __device__ __forceinline__ void ask16(unsigned int r, unsigned int piece, unsigned int to) const
    {
        if (WIDE)
            to_lds16((const unsigned char *)a.KV4 + ((uint64_t)r * kRowB + piece), to, AT);
        else
            to_lds16(a.KV4, r, piece, to, AT);
    }
    // four rows' codes, 16 lanes each: row 4 i + lane / 16, at code_at[lane / 16][i]
    __device__ __forceinline__ u32x4 code_rows(int i4, int lane) const { return *(const u32x4 *)&lds.code_at[wave][lane >> 4][4 * i4]; }
    static __device__ __forceinline__ unsigned int code_piece(int lane) { return 16u * ((lane & 15) ^ (lane >> 4)); }
    template <int I> __device__ __forceinline__ void ask_code(unsigned int to, unsigned int r, unsigned int piece) const { ask16<I * 1024>(r, piece ^ (64u * (I & 3)), to); }
    __device__ __forceinline__ unsigned int code_slot(unsigned int m) const { return code0 + (m & (kRing - 1)) * LDS::kSlotB; }
    // eight rows' rotary parts, 8 lanes each: row 8 i + lane / 8
    __device__ __forceinline__ u32x4 rope_rows(unsigned int m, int lane) const { return *(const u32x4 *)&lds.rope_at[wave][m & 1][lane >> 3][0]; }
    static __device__ __forceinline__ unsigned int rope_piece(int lane) { return kRopeOff + 16u * ((lane & 7) ^ (lane >> 4)); }
    template <int I> __device__ __forceinline__ void ask_rope(unsigned int r, unsigned int piece) const { ask16<I * 1024>(r, piece ^ (64u * (I & 1)), rope0); }
    __device__ __forceinline__ void ask_codes(unsigned int to, int lane) const
    {
        const u32x4 r0 = code_rows(0, lane), r1 = code_rows(1, lane);
        const unsigned int piece = code_piece(lane);
        ask_code<0>(to, r0[0], piece);
        ask_code<1>(to, r0[1], piece);
        ask_code<2>(to, r0[2], piece);
        ask_code<3>(to, r0[3], piece);
        ask_code<4>(to, r1[0], piece);
        ask_code<5>(to, r1[1], piece);
        ask_code<6>(to, r1[2], piece);
        ask_code<7>(to, r1[3], piece);
    }
    __device__ __forceinline__ void ask_ropes(unsigned int m, int lane) const
    {
        const u32x4 r = rope_rows(m, lane);
        const unsigned int piece = rope_piece(lane);
        ask_rope<0>(r[0], piece);
        ask_rope<1>(r[1], piece);
        ask_rope<2>(r[2], piece);
        ask_rope<3>(r[3], piece);
    }
    // the start: everything that the steps before tile 0's would have asked for
    __device__ __forceinline__ void begin(int lane, unsigned int (&ok)[3])
    {
#pragma unroll 1
        for (unsigned int i = 0; i < 6; ++i) {
            ask_ids(i, lane);
            next_ids();
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (PAGED) {
#pragma unroll 1
            for (unsigned int i = 0; i < 4; ++i) {
                ask_pages(i, entry(i, lane));
                next(pages);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
#pragma unroll
        for (unsigned int i = 0; i < 3; ++i) {
            ok[i] = find_rows(i, entry(i, lane), page(i, lane), lane);
            next(rows);
            if (i < 2) ask_codes(code_slot(i), lane);
            if (i == 0) ask_ropes(0, lane);
        }
        asm volatile("s_waitcnt vmcnt(10)" ::: "memory");                   // (tile 0 has arrived)
    }
    // the same where there is one step, which then asks for nothing
    __device__ __forceinline__ void begin_one(int lane, unsigned int (&ok)[3])
    {
        ask_ids(0, lane);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (PAGED) {
            ask_pages(0, entry(0, lane));
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        ok[0] = find_rows(0, entry(0, lane), page(0, lane), lane);
        ok[1] = ok[2] = 0;
        ask_codes(code_slot(0), lane);
        ask_ropes(0, lane);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
};

// Over the lanes l and l + 32.
__device__ __forceinline__ float half_max(float x)
{
    const u32x2 y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(as_float(y[0]), as_float(y[1]));
}
__device__ __forceinline__ float half_sum(float x)
{
    const u32x2 y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return as_float(y[0]) + as_float(y[1]);
}

// The exponents of P are s scale - ref, in one rounding, with the reference's own bias in ref = m - kPBias.  By references of
// kFar and more those roundings are powers of two of their own (at 2^30, 64 of them) and P would leave the range of a float: there
// the scores are by the reference before they are scaled, s' = (s scale - m) / scale, rounded as m is, and ref is the bias alone.
constexpr float kFar = 0x1p20f;
__device__ __forceinline__ float far_scores(f32x16 &s, float m, float ref, float scale)
{
#pragma clang fp contract(off)
    if (__ballot(__builtin_fabsf(m) >= kFar && m != -INFINITY) == 0ull) return ref;
    const float by = m == -INFINITY ? 0.f : m, back = __builtin_amdgcn_rcpf(scale);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float z = s[i] * scale;
        s[i] = (z - by) * back;
    }
    return m == -INFINITY ? 0.f : -kPBias;
}

// O^T times a factor per head, a tile at a time: the accumulators live in registers that only matrix instructions and moves
// reach, and all of them out at once would displace everything else.
template <int N> __device__ __forceinline__ void scale_tiles(f32x16 (&o)[N], float f)
{
#pragma unroll
    for (int t = 0; t < N; ++t) {
        f32x16 y = o[t];
        asm volatile("" : "+v"(y));
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] *= f;
        asm volatile("" : "+a"(y));
        o[t] = y;
        __builtin_amdgcn_sched_barrier(0);
    }
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

// A product into an accumulator that lives in ordinary registers: O^T takes all of the accumulation registers, and left to
// itself the compiler puts every accumulator there.  It knows nothing of these instructions' timing: between the conversions that
// write an operand and the product that reads it there is another product or an s_nop (two wait states are needed), and behind the last
// product comes mfma_settle() (11 wait states before the sum may be read).
__device__ __forceinline__ void mfma_new(f32x16 &s, bf16x8 x, bf16x8 y) { asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(x), "v"(y)); }
__device__ __forceinline__ void mfma_add(f32x16 &s, bf16x8 x, bf16x8 y) { asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(x), "v"(y)); }
__device__ __forceinline__ void mfma_settle(f32x16 &s) { asm volatile("s_nop 13" : "+v"(s)); }

// Many queries: each of the 1024 waves has queries of its own, one after the other.
template <bool PAGED, bool WIDE>
__global__ __launch_bounds__(256, 1) void kv4_attn_kernel(Kv4AttnArgs a)
{
    __shared__ __attribute__((aligned(1024))) Tiles lds;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int nq = a.B * a.Tq;
    // the waves of an XCD (every eighth workgroup) walk through neighbouring queries, whose selections overlap
    const int wg = (int)blockIdx.x, wgs = (int)gridDim.x;
    const int q0 = (wgs & 7) == 0 ? ((wg & 7) * (wgs >> 3) + (wg >> 3)) * 4 + wave : wg * 4 + wave;
    if (q0 >= nq) return;
    Fetch<1, PAGED, WIDE, Tiles> f(a, lds, wave, q0, wgs * 4, 0, 0);
    unsigned int n = 0, ok[3];                 // tile number; which rows it and the next two have
    f.begin(lane_now(), ok);
#pragma unroll 1
  for (int q = q0; q < nq; q += f.stride) {
    // Q as the B operand: head l32; chunk j, step s: features 64 j + 32 g + 8 s ..; then the rotary ones, 16 r + 8 g ..  (Lanes
    // without a head take the first one, and write nothing.)
    bf16x8 ql[8][4], qr[4];
    {
        const int ln = lane_now(), l32 = ln & 31, g = ln >> 5;
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
    u16x2 p[8];                                // of the tile before: bf16, two rows of the accumulator's registers each
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = u16x2{0, 0};

    // (Q has arrived before the loop, which must not wait for it, and is in these registers throughout)
    auto pin = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(ql[j][0]), "+v"(ql[j][1]), "+v"(ql[j][2]), "+v"(ql[j][3]));
        asm volatile("" : "+v"(qr[0]), "+v"(qr[1]), "+v"(qr[2]), "+v"(qr[3]));
    };
    pin();
    typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
    // V's codes, feature tile ft, as the A operand: lane (feature ln & 31, half g), rows of the accumulator's registers
    auto v_row = [&](int ln) __attribute__((always_inline)) { return tile_row(8 * ((ln & 15) >> 2) + 4 * (ln >> 5) + (ln & 3)); };
    auto v_codes = [&](const unsigned char *row, int ft, int r16) __attribute__((always_inline)) -> i32x2 {
        return __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2 *)(row + ((16 * ft) ^ r16)));
    };
    auto v_at = [&](unsigned int m2, int r, int ln) __attribute__((always_inline)) {
        return &lds.code[wave][0][0] + (m2 & (kRing - 1)) * kCodeB + r * 256 + ((ln >> 4) & 1) * 8;
    };
    struct Amount { u32x4 d[2]; };
    auto amounts = [&](unsigned int m2, int j, int g2) __attribute__((always_inline)) {
        Amount x;
        x.d[0] = *(const u32x4 *)&lds.amount[wave][m2 & 1][j][g2][0];
        x.d[1] = *(const u32x4 *)&lds.amount[wave][m2 & 1][j][g2][8];
        return x;
    };
    auto scaled = [&](u16x2 x, const Amount &am, int i) __attribute__((always_inline)) {
        return __builtin_bit_cast(unsigned int, __builtin_elementwise_sub_sat(x, as_u16x2(am.d[i >> 2][i & 3])));
    };
    // O^T += V^T P^T of the tile before, by itself
    auto pv_alone = [&](unsigned int m2) __attribute__((always_inline)) {
        const int ln = lane_now(), r = v_row(ln);
        const unsigned char *row = v_at(m2, r, ln);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const Amount am = amounts(m2, j, ln >> 5);
            u32x4 pj[2];
#pragma unroll
            for (int i = 0; i < 8; ++i) pj[i >> 2][i & 3] = scaled(p[i], am, i);
#pragma unroll
            for (int t4 = 0; t4 < 4; ++t4) {
                const int ft = 4 * j + t4;
                const i32x2 c = v_codes(row, ft, 16 * (r & 15));
                o[ft] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen((unsigned)c[0], 1.f), __builtin_bit_cast(bf16x8, pj[0]), o[ft], 0, 0, 0);
                o[ft] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen((unsigned)c[1], 1.f), __builtin_bit_cast(bf16x8, pj[1]), o[ft], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    bool anew = false;                         // the sums are still by the reference before the last
    float keep = 1.f;
    // K's codes, chunk j, as the A operand: lane (row ln & 31, half g)
    auto k_at = [&](unsigned int m2, int kr) __attribute__((always_inline)) { return &lds.code[wave][0][0] + (m2 & (kRing - 1)) * kCodeB + kr * 256; };
    auto k_codes = [&](const unsigned char *row, int j, int gr) __attribute__((always_inline)) { return *(const u32x4 *)(row + ((32 * j) ^ gr)); };
    u32x4 kc[3];                               // chunks j in [j % 3]; of the tile that comes 0 and 1, and its exponents
    unsigned int sc;
    {
        const int ln = lane_now(), kr = tile_row(ln & 31), gr = 16 * ((ln >> 5) ^ (kr & 15));
        kc[0] = k_codes(k_at(n, kr), 0, gr);
        kc[1] = k_codes(k_at(n, kr), 1, gr);
        sc = lds.scale[wave][n & 3][kr];
    }
#pragma unroll 1
    for (int t = 0; t < f.n_tiles; ++t, ++n) {
        if (anew) scale_tiles(o, keep);
#pragma unroll
        for (int t2 = 0; t2 < 16; ++t2) asm volatile("" : "+a"(o[t2]));
        pin();
        const int ln = lane_now(), l32 = ln & 31, g = ln >> 5, kr = tile_row(l32), gr = 16 * (g ^ (kr & 15));
        f32x16 s;
        u32x4 pj[2][2];
        i32x2 vc[4];                            // feature tiles ft in [ft % 4]
        Amount am;
        const int vr = v_row(ln), r16 = 16 * (vr & 15);
        const unsigned int m1 = n - 1;
        const unsigned char *const vrow = v_at(m1, vr, ln);
        if (ok[0] == 0u) {
            // no rows: nothing to score; the tile before may wait for its product
            f.ask_codes(f.code_slot(n + 2), ln);
            f.ask_pages(n + 4, f.entry(n + 4, ln));
            f.ask_ids(n + 6, ln);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(f.kAhead) : "memory");
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = -INFINITY;
            am = amounts(m1, 0, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) pj[0][i >> 2][i & 3] = scaled(p[i], am, i);
#pragma unroll
            for (int ft = 0; ft < 3; ++ft) vc[ft] = v_codes(vrow, ft, r16);
            am = amounts(m1, 1, g);
        } else {
            // S = K Q^T of this tile
            const unsigned char *const krow = k_at(n, kr), *const rrow = &lds.rope[wave][0] + kr * 128;
            const int rr = 16 * (g ^ (kr >> 1 & 7));
            auto rope_piece = [&](int r) __attribute__((always_inline)) { return *(const bf16x8 *)(rrow + ((32 * r) ^ rr)); };
            bf16x8 kb[3], rk[3];
            u32x4 cr;
            const unsigned int to = f.code_slot(n + 2), piece = f.code_piece(ln);
            float sf[4];
            int pe = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) sf[j] = scale_of((sc >> (8 * j)) & 255u);
            kb[0] = widen(kc[0][0], sf[0]);
            kb[1] = widen(kc[0][1], sf[0]);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int j = i >> 2, e = i & 3;
                if (i == 0)
                    mfma_new(s, kb[0], ql[0][0]);
                else
                    mfma_add(s, kb[i % 3], ql[j][e]);
                __builtin_amdgcn_sched_barrier(0);
                if (i < 30) kb[(i + 2) % 3] = widen(kc[((i + 2) >> 2) % 3][(i + 2) & 3], sf[(i + 2) >> 3]);
                if (e == 0 && j < 6) kc[(j + 2) % 3] = k_codes(krow, j + 2, gr);
                if (i == 1 || i == 11) cr = f.code_rows(i > 1, ln);
                if (i == 6) f.template ask_code<0>(to, cr[0], piece);
                if (i == 7) f.template ask_code<1>(to, cr[1], piece);
                if (i == 8) f.template ask_code<2>(to, cr[2], piece);
                if (i == 9) f.template ask_code<3>(to, cr[3], piece);
                if (i == 16) f.template ask_code<4>(to, cr[0], piece);
                if (i == 17) f.template ask_code<5>(to, cr[1], piece);
                if (i == 18) f.template ask_code<6>(to, cr[2], piece);
                if (i == 19) f.template ask_code<7>(to, cr[3], piece);
                if (i == 2 || i == 3 || i == 4 || i == 5) {
                    // the subtractions from P's exponents, in the order of the accumulator's registers (both halves write the same)
                    const int jj = i - 2;
                    lds.amount[wave][n & 1][jj][(l32 >> 2) & 1][4 * (l32 >> 3) + (l32 & 3)] = (unsigned short)(kAmount - (int)(((sc >> (8 * jj)) & 255u) << 7));
                }
                if (PAGED && i == 13) pe = f.entry(n + 4, ln);
                if (i == 20) f.ask_pages(n + 4, pe);
                if (i == 21) f.ask_ids(n + 6, ln);
                if (i == 22) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(f.kAhead) : "memory");
                if (i == 12) am = amounts(m1, 0, g);
                if (i >= 23 && i < 26) rk[i - 23] = rope_piece(i - 23);
                if (i >= 26 && i < 30) {
                    pj[0][(2 * (i - 26)) >> 2][(2 * (i - 26)) & 3] = scaled(p[2 * (i - 26)], am, 2 * (i - 26));
                    pj[0][(2 * (i - 26) + 1) >> 2][(2 * (i - 26) + 1) & 3] = scaled(p[2 * (i - 26) + 1], am, 2 * (i - 26) + 1);
                }
                if (i >= 27 && i < 30) vc[i - 27] = v_codes(vrow, i - 27, r16);
                if (i == 30) am = amounts(m1, 1, g);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                mfma_add(s, rk[r % 3], qr[r]);
                __builtin_amdgcn_sched_barrier(0);
                if (r == 0) rk[0] = rope_piece(3);
            }
            mfma_settle(s);
            // register i is matrix row 8 (i / 4) + 4 g + i % 4
            if (ok[0] != 0xFFFFFFFFu) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int tr = 8 * (i >> 2) + 4 * (i < 8 ? g : 1 - g) + (i & 3);
                    s[i] = (ok[0] >> tr) & 1u ? s[i] : -INFINITY;
                }
            }
        }
        // O^T += V^T P^T of the tile before, and this tile's P
        bf16x8 vb[3];
        unsigned int ok3 = 0;
        int e3 = 0, p3 = 0;
        vb[0] = widen((unsigned)vc[0][0], 1.f);
        vb[1] = widen((unsigned)vc[0][1], 1.f);
        const u32x4 ro = f.rope_rows(n + 1, ln);
        const unsigned int rpiece = f.rope_piece(ln);
        float top = 0.f, ref = 0.f;
        u16x2 pn[8];
        float p0 = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const int ft = i >> 1, j = i >> 3, k = i & 7;
            o[ft] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[i % 3], __builtin_bit_cast(bf16x8, pj[j & 1][i & 1]), o[ft], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (i < 30) vb[(i + 2) % 3] = widen((unsigned)vc[((i + 2) >> 1) & 3][i & 1], 1.f);
            if ((i & 1) == 0 && ft + 3 < 16) vc[(ft + 3) & 3] = v_codes(vrow, ft + 3, r16);
            if (j < 3 && k >= 3 && k < 7) {
                pj[(j + 1) & 1][(2 * (k - 3)) >> 2][(2 * (k - 3)) & 3] = scaled(p[2 * (k - 3)], am, 2 * (k - 3));
                pj[(j + 1) & 1][(2 * (k - 3) + 1) >> 2][(2 * (k - 3) + 1) & 3] = scaled(p[2 * (k - 3) + 1], am, 2 * (k - 3) + 1);
            }
            if (k == 7 && j < 2) am = amounts(m1, j + 2, g);
            if (i == 2) top = fmaxf(s[0], s[1]);
            if (i >= 2 && i < 9) top = fmaxf(fmaxf(top, s[2 * i - 2]), s[2 * i - 1]);
            if (i == 4) f.template ask_rope<0>(ro[0], rpiece);
            if (i == 5) f.template ask_rope<1>(ro[1], rpiece);
            if (i == 6) f.template ask_rope<2>(ro[2], rpiece);
            if (i == 7) f.template ask_rope<3>(ro[3], rpiece);
            if (i == 9) {
                top = half_max(top) * a.scale_log2e;
                anew = __ballot(top > m + a.lag) != 0ull;                    // (m = -inf: the first rows)
            }
            if (i == 10) {
                const float mn = anew ? fmaxf(m, top) : m;
                keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
                m = mn;
                l *= keep;
                ref = far_scores(s, m, m == -INFINITY ? 0.f : m - kPBias, a.scale_log2e);
            }
            if (i >= 12 && i < 28) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i - 12], a.scale_log2e, -ref));
                l += x;
                if (i & 1)
                    pn[(i - 12) >> 1] = __builtin_bit_cast(u16x2, __builtin_convertvector((f32x2{p0, x}), bf16x2));
                else
                    p0 = x;
            }
            if (i == 8) {
                e3 = f.entry(n + 3, ln);
                p3 = f.page(n + 3, ln);
            }
            if (i == 16) ok3 = f.find_rows(n + 3, e3, p3, ln);
            if (i == 22) sc = lds.scale[wave][(n + 1) & 3][kr];
            if (i == 24) kc[0] = k_codes(k_at(n + 1, kr), 0, gr);
            if (i == 25) kc[1] = k_codes(k_at(n + 1, kr), 1, gr);
            __builtin_amdgcn_sched_barrier(0);
        }
        f.advance();
        ok[0] = ok[1];
        ok[1] = ok[2];
        ok[2] = ok3;
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = pn[i];
    }
    if (anew) scale_tiles(o, keep);
    pv_alone(n - 1);
    asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");              // (the last products, before their sums are read)
    const int lane = lane_now(), l32 = lane & 31, g = lane >> 5;
    l = half_sum(l);

    const float inv = l == 0.f ? 0.f : 0x1p100f / l;                        // (the sums of P V are without the bias)
    const int64_t head = (int64_t)q * a.H_q + l32;
    if (l32 < a.H_q) {
        // features 32 ft + 8 i4 + 4 g + 0 .. 3 of the head
#pragma unroll
        for (int ft = 0; ft < 16; ++ft)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4)
                *(bf16x4 *)((__bf16 *)a.O + head * kLat + 32 * ft + 8 * i4 + 4 * g) = __builtin_convertvector(read4(o[ft], i4, inv), bf16x4);
        if (g == 0 && a.lse) a.lse[head] = l == 0.f ? -INFINITY : (m + __builtin_log2f(l) - kPBias) * 0.6931471805599453f;
    }
  }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// Few queries: the four waves of a workgroup share one, or a split of one.  In a step each scores a tile; they agree on the
// reference by the four tiles' maxima, and each multiplies all four tiles' P with its own 128 features of V, which are one
// block: its sums of O are 64 registers, and there is nothing to add up between the waves at the end (with a tile's product
// to itself each wave had all 512 features, and their sum through LDS took 10 000 clocks).  What bounds a launch is latency:
// entries, page numbers and rows from memory one after the other, Q meanwhile (36 KB, once in LDS for all four waves: read
// by each from memory it took 9 000 clocks), then 2.8 us a step of 128 rows.  Measured back to back in a graph: 32 rows of one
// query 7.3 us (15.3 before these two), 2048 rows in 16 splits 12.4 with their merge, 40 queries of 2048 rows 24.3.  The last
// step asks for nothing (a microsecond of it).
// In a step: S, barrier, asks for the rotary part of n + 1, codes of n + 2, page numbers of n + 4 and entries of n + 6, softmax, a wait for
// all but these, row numbers of n + 3, exponents asked for, barrier, the product with V.  The next step's rotary part then has
// kAhead instructions behind it.
struct FewTiles {
    static constexpr int kSlotB = 4 * kCodeB;
    unsigned char code[3][4][kCodeB];         // [ring][wave]
    u32x4 p[2][4][2][64];                     // P: step n in [n % 2][wave][registers 0-3, 4-7 (rows in pairs)][lane]; at first Q, from code[2] on
    unsigned char rope[4][kRopeB];
    int32_t idx[4][8][kT], page[4][4][kT];
    unsigned int scale[4][4][kT];
    unsigned short amount[2][4][4][2][16];    // [n % 2][wave][block][half][register]
    unsigned int code_at[4][4][8], rope_at[4][2][8][4];
    float top[2][4][32], sum[4][32];
    __device__ __forceinline__ unsigned char *codes(int wave) { return &code[0][wave][0]; }
};

// LDS writes are there for the workgroup's other waves, reads are done.  (No wait for what is on its way from memory.)
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Q into LDS, a quarter of the heads per wave: head h 1152 h bytes on, its 16-byte piece c at c ^ (h / 2 % 8) (16 heads' pieces are
// then in 16 different bank groups).  Nine instructions.
__device__ __forceinline__ void ask_q(const Kv4AttnArgs &a, int q, unsigned int lds, int wave, int lane)
{
#pragma unroll
    for (int i = 0; i < 9; ++i) {
        const int at = 576 * wave + 64 * i + lane, h = at / 72, c = at - 72 * h;
        to_lds16((const unsigned char *)a.Q + (((int64_t)q * a.H_q + (h < a.H_q ? h : 0)) * (2 * kRow) + 16 * (c ^ (h >> 1 & 7))), lds + 16 * (576 * wave + 64 * i), 0);
    }
}
// A lane's pieces of it: head lane & 31; chunk j, step s: features 64 j + 32 g + 8 s ..; then the rotary ones, 16 r + 8 g ..
__device__ __forceinline__ void read_q(const unsigned char *lds, int lane, bf16x8 (&ql)[8][4], bf16x8 (&qr)[4])
{
    const int h = lane & 31, g = lane >> 5, x = h >> 1 & 7;
    const unsigned char *row = lds + h * (2 * kRow);
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int s = 0; s < 4; ++s) ql[j][s] = *(const bf16x8 *)(row + 16 * ((8 * j + 4 * g + s) ^ x));
#pragma unroll
    for (int r = 0; r < 4; ++r) qr[r] = *(const bf16x8 *)(row + 16 * ((64 + 2 * r + g) ^ x));
}

template <bool PAGED, bool WIDE>
__global__ __launch_bounds__(256, 1) void kv4_attn_few_kernel(Kv4AttnArgs a)
{
    __shared__ __attribute__((aligned(1024))) FewTiles lds;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int l32 = lane & 31, g = lane >> 5;
    const int q = (int)blockIdx.x / a.n_splits, split = (int)blockIdx.x - q * a.n_splits;
    Fetch<4, PAGED, WIDE, FewTiles> f(a, lds, wave, q, 0, split, wave);
    static_assert(sizeof(lds.code[2]) + sizeof(lds.p) >= 32 * 2 * kRow, "Q");
    unsigned char *const q_lds = &lds.code[2][0][0];
    ask_q(a, q, (unsigned)__builtin_amdgcn_readfirstlane((int)lds_offset(q_lds)), wave, lane);
    unsigned int n = 0, slot = 0, ok[3];
    const int n_steps = (f.n_tiles + 3) / 4;
    if (n_steps > 1)
        f.begin(lane, ok);
    else
        f.begin_one(lane, ok);
    meet();                                    // (Q was asked for before what begin() has waited for)
    bf16x8 ql[8][4], qr[4];
    read_q(q_lds, lane, ql, qr);
    f32x16 o[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    const int kr = tile_row(l32), gr = 16 * (g ^ (kr & 15)), rr = 16 * (g ^ (kr >> 1 & 7));
    const int vr = tile_row(8 * ((lane & 15) >> 2) + 4 * g + (lane & 3)), r16 = 16 * (vr & 15);
    auto k_at = [&](unsigned int at) __attribute__((always_inline)) { return &lds.code[at][wave][kr * 256]; };
    u32x4 kc[3];                               // K's codes, chunks j in [j % 3]; of the tile that comes 0 and 1, and its exponents
    kc[0] = *(const u32x4 *)(k_at(0) + gr);
    kc[1] = *(const u32x4 *)(k_at(0) + (32 ^ gr));
    unsigned int sc = lds.scale[wave][0][kr];
    auto pin = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(ql[j][0]), "+v"(ql[j][1]), "+v"(ql[j][2]), "+v"(ql[j][3]));
        asm volatile("" : "+v"(qr[0]), "+v"(qr[1]), "+v"(qr[2]), "+v"(qr[3]));
    };
    pin();
#pragma unroll 1
    for (int t = 0; t < n_steps; ++t, ++n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+a"(o[i]));
        pin();
        // S = K Q^T of this wave's tile
        f32x16 s;
        if (ok[0] == 0u) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = -INFINITY;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(f.kAhead) : "memory");
        } else {
            const unsigned char *const krow = k_at(slot), *const rrow = &lds.rope[wave][kr * 128];
            bf16x8 kb[3], rk[3];
            float sf[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) sf[j] = scale_of((sc >> (8 * j)) & 255u);
            kb[0] = widen(kc[0][0], sf[0]);
            kb[1] = widen(kc[0][1], sf[0]);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int j = i >> 2, e = i & 3;
                if (i == 0)
                    mfma_new(s, kb[0], ql[0][0]);
                else
                    mfma_add(s, kb[i % 3], ql[j][e]);
                __builtin_amdgcn_sched_barrier(0);
                if (i < 30) kb[(i + 2) % 3] = widen(kc[((i + 2) >> 2) % 3][(i + 2) & 3], sf[(i + 2) >> 3]);
                if (e == 0 && j < 6) kc[(j + 2) % 3] = *(const u32x4 *)(krow + ((32 * (j + 2)) ^ gr));
                if (i >= 2 && i < 6)
                    lds.amount[n & 1][wave][i - 2][(l32 >> 2) & 1][4 * (l32 >> 3) + (l32 & 3)] = (unsigned short)(kAmount - (int)(((sc >> (8 * (i - 2))) & 255u) << 7));
                if (i == 25) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(f.kAhead) : "memory");  // (what was asked for behind the rotary part)
                if (i >= 26 && i < 29) rk[i - 26] = *(const bf16x8 *)(rrow + ((32 * (i - 26)) ^ rr));
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                mfma_add(s, rk[r % 3], qr[r]);
                __builtin_amdgcn_sched_barrier(0);
                if (r == 0) rk[0] = *(const bf16x8 *)(rrow + (96 ^ rr));
            }
            mfma_settle(s);
            if (ok[0] != 0xFFFFFFFFu) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int tr = 8 * (i >> 2) + 4 * (i < 8 ? g : 1 - g) + (i & 3);
                    s[i] = (ok[0] >> tr) & 1u ? s[i] : -INFINITY;
                }
            }
        }
        float top = fmaxf(s[0], s[1]);
#pragma unroll
        for (int i = 2; i < 16; i += 2) top = fmaxf(fmaxf(top, s[i]), s[i + 1]);
        top = half_max(top) * a.scale_log2e;
        lds.top[n & 1][wave][l32] = top;
        meet();
        // (everybody is through the step before: the ring's third tile is free)
        float tops[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) tops[w] = lds.top[n & 1][w][l32];
        const unsigned int two = slot == 0 ? 2 : slot - 1;
        const bool more = t + 1 < n_steps;
        if (more) {
            f.ask_ropes(n + 1, lane);
            f.ask_codes((unsigned)__builtin_amdgcn_readfirstlane((int)(f.code0 + two * FewTiles::kSlotB)), lane);
            f.ask_pages(n + 4, f.entry(n + 4, lane));
            f.ask_ids(n + 6, lane);
        }
        top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        if (__ballot(top > m + a.lag) != 0ull) {                             // (the same in every wave)
            const float mn = fmaxf(m, top), keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= keep;
            scale_tiles(o, keep);
        }
        const float ref = far_scores(s, m, m == -INFINITY ? 0.f : m - kPBias, a.scale_log2e);
        u32x4 p[2];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale_log2e, -ref)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i + 1], a.scale_log2e, -ref));
            l += p0 + p1;
            p[i >> 3][(i >> 1) & 3] = __builtin_bit_cast(unsigned int, __builtin_convertvector((f32x2{p0, p1}), bf16x2));
        }
        lds.p[n & 1][wave][0][lane] = p[0];
        lds.p[n & 1][wave][1][lane] = p[1];
        if (more) {
            ok[0] = ok[1];
            ok[1] = ok[2];
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(f.kAhead + 3) : "memory");  // (this step's: the page numbers of n + 3 were asked for a step ago)
            ok[2] = f.find_rows(n + 3, f.entry(n + 3, lane), f.page(n + 3, lane), lane);
            f.advance();
        }
        meet();
        // O^T += V^T P^T of the four tiles, this wave's features.  (A tile without rows: its P is 0, and any code is a number.)
        typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
        u32x4 pv[2][2], am[2][2];
        i32x2 vc[2][4];
        const unsigned char *const vrow = &lds.code[slot][0][vr * 256 + ((lane >> 4) & 1) * 8];
        auto v_get = [&](int w) __attribute__((always_inline)) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pv[w & 1][h] = lds.p[n & 1][w][h][lane];
                am[w & 1][h] = *(const u32x4 *)&lds.amount[n & 1][w][wave][g][8 * h];
            }
#pragma unroll
            for (int t4 = 0; t4 < 4; ++t4) vc[w & 1][t4] = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2 *)(vrow + w * kCodeB + ((64 * wave + 16 * t4) ^ r16)));
        };
        v_get(0);
        slot = slot == 2 ? 0 : slot + 1;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (4 * t + w >= f.n_tiles) break;
            if (w < 3) v_get(w + 1);
            if (w == 3) {
                kc[0] = *(const u32x4 *)(k_at(slot) + gr);
                kc[1] = *(const u32x4 *)(k_at(slot) + (32 ^ gr));
                sc = lds.scale[wave][(n + 1) & 3][kr];
            }
            u32x4 pj[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    pj[h][i] = __builtin_bit_cast(unsigned int, __builtin_elementwise_sub_sat(as_u16x2(pv[w & 1][h][i]), as_u16x2(am[w & 1][h][i])));
#pragma unroll
            for (int t4 = 0; t4 < 4; ++t4) {
                const i32x2 c = vc[w & 1][t4];
                o[t4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen((unsigned)c[0], 1.f), __builtin_bit_cast(bf16x8, pj[0]), o[t4], 0, 0, 0);
                o[t4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen((unsigned)c[1], 1.f), __builtin_bit_cast(bf16x8, pj[1]), o[t4], 0, 0, 0);
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds.sum[wave][l32] = half_sum(l);
    meet();
    l = (lds.sum[0][l32] + lds.sum[1][l32]) + (lds.sum[2][l32] + lds.sum[3][l32]);
    if (l32 >= a.H_q) return;
    const float inv = l == 0.f ? 0.f : 0x1p100f / l;
    const int64_t head = (int64_t)q * a.H_q + l32, part = ((int64_t)q * a.n_splits + split) * a.H_q + l32;
#pragma unroll
    for (int t4 = 0; t4 < 4; ++t4)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
            const f32x4 y = f32x4{o[t4][4 * i4], o[t4][4 * i4 + 1], o[t4][4 * i4 + 2], o[t4][4 * i4 + 3]} * inv;
            const int at = 128 * wave + 32 * t4 + 8 * i4 + 4 * g;
            if (a.n_splits > 1)
                *(f32x4 *)((float *)a.part_o + part * kLat + at) = y;
            else
                *(bf16x4 *)((__bf16 *)a.O + head * kLat + at) = __builtin_convertvector(y, bf16x4);
        }
    if (g != 0 || wave != 0) return;
    if (a.n_splits > 1) {
        a.part_ml[2 * part] = l == 0.f ? -INFINITY : (l != l ? l : m);       // (the merge leaves out what has no maximum)
        a.part_ml[2 * part + 1] = l * 0x1p-100f;
    } else if (a.lse) {
        a.lse[head] = l == 0.f ? -INFINITY : (m + __builtin_log2f(l) - kPBias) * 0.6931471805599453f;
    }
}

// ---- the weight each selected row received --------------------------------------------------------------------------
//
// probs[q, slot] = 1/H sum_h exp(sm_scale <Q[h], K[row]> - lse[h]).  The same tiles as above with the operands exchanged:
// heads are the matrix rows, cache rows the columns, so a lane holds 16 heads of one cache row and adds them up by itself.
// A step multiplies one tile and, between its products, takes the exponentials of the tile before.  What bounds it are the
// rows' lines from L2: 8191 queries of 2048 rows in 600 us, 11.2 TB/s of rows, what the fetches of kv4_attn_kernel without its
// arithmetic ran at (a row of 400 bytes lies in 5 lines of 128, asked for as 6).
struct ProbTiles {
    static constexpr int kSlotB = kCodeB;
    unsigned char code[4][3][kCodeB];         // [wave][ring]
    unsigned char q[32 * 2 * kRow];           // (four waves to a query)
    unsigned char rope[4][kRopeB];
    int32_t idx[4][8][kT], page[4][4][kT];
    unsigned int scale[4][4][kT];
    unsigned int code_at[4][4][8], rope_at[4][2][8][4];
    float off[4][32];                         // the heads' log-sum-exps in log2 units
    __device__ __forceinline__ unsigned char *codes(int wave) { return &code[wave][0][0]; }
};

template <int W, bool PAGED, bool WIDE>
__global__ __launch_bounds__(256, 1) void kv4_probs_kernel(Kv4AttnArgs a)
{
    __shared__ __attribute__((aligned(1024))) ProbTiles lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5;
    const int nq = a.B * a.Tq;
    const int wg = (int)blockIdx.x, wgs = (int)gridDim.x;
    const int q0 = W > 1 ? wg / a.n_splits : (wgs & 7) == 0 ? ((wg & 7) * (wgs >> 3) + (wg >> 3)) * 4 + wave : wg * 4 + wave;
    const int split = W > 1 ? wg - q0 * a.n_splits : 0;
    if (W == 1 && q0 >= nq) return;
    Fetch<W, PAGED, WIDE, ProbTiles> f(a, lds, wave, q0, wgs * 4, split, W == 1 ? 0 : wave);
    if (W > 1) ask_q(a, q0, (unsigned)__builtin_amdgcn_readfirstlane((int)lds_offset(lds.q)), wave, lane);
    unsigned int n = 0, slot = 0, ok[3];
    f.begin(lane, ok);
    if (W > 1) meet();
    const float inv_h = 1.f / (float)a.H_q;
    const int gr = 16 * (g ^ (l32 & 15)), rr = 16 * (g ^ (l32 >> 1 & 7));
    auto k_at = [&](unsigned int at) __attribute__((always_inline)) { return &lds.code[wave][at][l32 * 256]; };
#pragma unroll 1
  for (int q = q0; q < nq; q += f.stride) {
    bf16x8 ql[8][4], qr[4];
    if (W > 1) {
        read_q(lds.q, lane, ql, qr);
    } else {
        const unsigned short *qp = (const unsigned short *)a.Q + ((int64_t)q * a.H_q + (l32 < a.H_q ? l32 : 0)) * kRow;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int s = 0; s < 4; ++s)
                ql[j][s] = *(const bf16x8 *)(qp + 64 * j + 32 * g + 8 * s);
#pragma unroll
        for (int r = 0; r < 4; ++r) qr[r] = *(const bf16x8 *)(qp + kLat + 16 * r + 8 * g);
    }
    // (heads that are not there: nothing is left of exp2(s - inf))
    lds.off[wave][l32] = l32 < a.H_q ? a.lse[(int64_t)q * a.H_q + l32] * 1.4426950408889634f : INFINITY;
    float z[16];                                // of the tile before: log2 of the probabilities of heads 8 (i / 4) + 4 g + i % 4
    unsigned int have = 0;
    int at = -1;                                // its slot of this lane
    auto pin = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(ql[j][0]), "+v"(ql[j][1]), "+v"(ql[j][2]), "+v"(ql[j][3]));
        asm volatile("" : "+v"(qr[0]), "+v"(qr[1]), "+v"(qr[2]), "+v"(qr[3]));
#pragma unroll
        for (int i = 0; i < 16; ++i) asm volatile("" : "+v"(z[i]));
    };
    auto write = [&](float p) __attribute__((always_inline)) {
        p = half_sum(p);
        if (g == 0 && (unsigned)at < (unsigned)f.n_slots) a.probs[(int64_t)q * a.k_sel + f.s0 + at] = (have >> l32) & 1u ? p * inv_h : 0.f;
    };
    auto finish = [&]() __attribute__((always_inline)) {
        float p = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) p += __builtin_amdgcn_exp2f(z[i]);
        write(p);
    };
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    pin();
    u32x4 kc[3];                               // K's codes, chunks j in [j % 3]; of the tile that comes 0 and 1, and its exponents
    kc[0] = *(const u32x4 *)(k_at(slot) + gr);
    kc[1] = *(const u32x4 *)(k_at(slot) + (32 ^ gr));
    unsigned int sc = lds.scale[wave][n & 3][l32];
#pragma unroll 1
    for (int t = f.first; t < f.n_tiles; t += W, ++n) {
        pin();
        const unsigned int two = slot == 0 ? 2 : slot - 1;
        const unsigned int to = f.code0 + two * kCodeB, rpiece = f.rope_piece(lane);
        u32x4 ro;
        int e3 = 0, p3 = 0;
        f32x16 s;
        f32x4 off[4];
        auto ask_ropes = [&]() __attribute__((always_inline)) {
            f.template ask_rope<0>(ro[0], rpiece);
            f.template ask_rope<1>(ro[1], rpiece);
            f.template ask_rope<2>(ro[2], rpiece);
            f.template ask_rope<3>(ro[3], rpiece);
        };
        if (ok[0] == 0u) {
            f.ask_codes(to, lane);
            f.ask_pages(n + 4, f.entry(n + 4, lane));
            f.ask_ids(n + 6, lane);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(f.kAhead) : "memory");
            finish();
            // (what is written for this tile is zero, whatever its z)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = off[i >> 2][i & 3] = 0.f;
            e3 = f.entry(n + 3, lane);
            p3 = f.page(n + 3, lane);
            ro = f.rope_rows(n + 1, lane);
            ask_ropes();
        } else {
            const unsigned char *const krow = k_at(slot), *const rrow = &lds.rope[wave][l32 * 128];
            bf16x8 kb[3], rk[3];
            float sf[4], p = 0.f;
            u32x4 cr;
            int pe = 0;
            const unsigned int piece = f.code_piece(lane);
#pragma unroll
            for (int j = 0; j < 4; ++j) sf[j] = scale_of((sc >> (8 * j)) & 255u);
            kb[0] = widen(kc[0][0], sf[0]);
            kb[1] = widen(kc[0][1], sf[0]);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int j = i >> 2, e = i & 3;
                if (i == 0)
                    mfma_new(s, ql[0][0], kb[0]);
                else
                    mfma_add(s, ql[j][e], kb[i % 3]);
                __builtin_amdgcn_sched_barrier(0);
                if (i < 30) kb[(i + 2) % 3] = widen(kc[((i + 2) >> 2) % 3][(i + 2) & 3], sf[(i + 2) >> 3]);
                if (e == 0 && j < 6) kc[(j + 2) % 3] = *(const u32x4 *)(krow + ((32 * (j + 2)) ^ gr));
                if (i == 1 || i == 11) cr = f.code_rows(i > 1, lane);
                if (i == 6) f.template ask_code<0>(to, cr[0], piece);
                if (i == 7) f.template ask_code<1>(to, cr[1], piece);
                if (i == 8) f.template ask_code<2>(to, cr[2], piece);
                if (i == 9) f.template ask_code<3>(to, cr[3], piece);
                if (i == 16) f.template ask_code<4>(to, cr[0], piece);
                if (i == 17) f.template ask_code<5>(to, cr[1], piece);
                if (i == 18) f.template ask_code<6>(to, cr[2], piece);
                if (i == 19) f.template ask_code<7>(to, cr[3], piece);
                if (PAGED && i == 13) pe = f.entry(n + 4, lane);
                if (i == 20) f.ask_pages(n + 4, pe);
                if (i == 21) f.ask_ids(n + 6, lane);
                if (i == 22) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(f.kAhead) : "memory");
                if (i >= 23 && i < 26) rk[i - 23] = *(const bf16x8 *)(rrow + ((32 * (i - 23)) ^ rr));
                if (i >= 2 && i < 18) p += __builtin_amdgcn_exp2f(z[i - 2]);
                if (i == 14) e3 = f.entry(n + 3, lane);
                if (i == 24) p3 = f.page(n + 3, lane);
                if (i == 30) ro = f.rope_rows(n + 1, lane);
                if (i >= 26 && i < 30) off[i - 26] = *(const f32x4 *)&lds.off[wave][8 * (i - 26) + 4 * g];
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                mfma_add(s, qr[r], rk[r % 3]);
                __builtin_amdgcn_sched_barrier(0);
                if (r == 0) rk[0] = *(const bf16x8 *)(rrow + (96 ^ rr));
                if (r == 1) write(p);
                __builtin_amdgcn_sched_barrier(0);
            }
            ask_ropes();
            mfma_settle(s);
        }
        // (in place: a loop around new values copies them)
#pragma unroll
        for (int i = 0; i < 16; ++i) asm volatile("v_fma_f32 %0, %1, %2, -%3" : "+v"(z[i]) : "v"(s[i]), "s"(a.scale_log2e), "v"(off[i >> 2][i & 3]));
        have = ok[0];
        at = t * kT + l32;
        ok[0] = ok[1];
        ok[1] = ok[2];
        ok[2] = f.find_rows(n + 3, e3, p3, lane);
        f.advance();
        slot = slot == 2 ? 0 : slot + 1;
        kc[0] = *(const u32x4 *)(k_at(slot) + gr);
        kc[1] = *(const u32x4 *)(k_at(slot) + (32 ^ gr));
        sc = lds.scale[wave][(n + 1) & 3][l32];
    }
    finish();
    if (W > 1) break;
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

// Whether a row of the cache begins behind 4 GB, where an offset of 32 bits does not reach (the bytes within a row that are added to it included).
bool kv4_wide(const Kv4AttnArgs &a) { return (uint64_t)a.pool_rows * kRowB > 0xFFFFFFFFull; }

// Kernel forms by what a cache is.
#define IC_KV4_FORMS(KERNEL, GRID)                                                                                              \
    do {                                                                                                                        \
        const dim3 block(256), grid((unsigned)(GRID));                                                                          \
        const bool paged = a.pv.page_table != nullptr, wide = kv4_wide(a);                                                      \
        if (paged && wide) hipLaunchKernelGGL((KERNEL(true, true)), grid, block, 0, st, a);                                     \
        else if (paged) hipLaunchKernelGGL((KERNEL(true, false)), grid, block, 0, st, a);                                       \
        else if (wide) hipLaunchKernelGGL((KERNEL(false, true)), grid, block, 0, st, a);                                        \
        else hipLaunchKernelGGL((KERNEL(false, false)), grid, block, 0, st, a);                                                 \
    } while (0)
#define IC_KV4_MANY(P, L) kv4_attn_kernel<P, L>
#define IC_KV4_FEW(P, L) kv4_attn_few_kernel<P, L>
#define IC_KV4_PROBS1(P, L) kv4_probs_kernel<1, P, L>
#define IC_KV4_PROBS4(P, L) kv4_probs_kernel<4, P, L>

hipError_t launch_kv4_attn(const Kv4AttnArgs &a, bool together, hipStream_t st)
{
    const int64_t units = (int64_t)a.B * a.Tq * a.n_splits;
    if (together)
        IC_KV4_FORMS(IC_KV4_FEW, units);
    else
        IC_KV4_FORMS(IC_KV4_MANY, std::min<int64_t>(256, (units + 3) / 4));
    return hipGetLastError();
}

hipError_t launch_kv4_probs(const Kv4AttnArgs &a, bool together, hipStream_t st)
{
    const int64_t units = (int64_t)a.B * a.Tq * a.n_splits;
    if (together)
        IC_KV4_FORMS(IC_KV4_PROBS4, units);
    else
        IC_KV4_FORMS(IC_KV4_PROBS1, std::min<int64_t>(256, (units + 3) / 4));
    return hipGetLastError();
}

} // namespace ic
