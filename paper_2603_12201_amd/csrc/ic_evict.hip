// Eviction from a cache by accumulated attention weight: what each position received, which positions stay, and their rows
// moved together.
//
//   weight_kernel   weight[s] = in[s] + sum over the query rows of probs at the slots that name s.  A workgroup owns a range of
//                   positions in LDS and adds there in 64-bit fixed point (units of 2^-48), so the order of the additions
//                   does not show in the sum.  Bound by memory (probs and idx once), or for a few rows by the launch.
//   evict_kernel    the n_keep positions of a sequence that stay: the first n_first, the last n_recent, and the largest weights
//                   among the others (equal weights: the lower position).  See there.
//   compact_kernel  rows of several caches to their new places.  Bound by memory.
#include "ic_common.hpp"

namespace ic {

namespace {

typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;

// p in [0, 1] in units of 2^-48, rounded down; what is not a number counts as 0
__device__ __forceinline__ unsigned long long fixed48(float p)
{
    p = fminf(fmaxf(p, 0.f), 1.f);                                          // (fmaxf of NaN and 0 is 0)
    const float a = p * 0x1p24f;
    const unsigned int hi = (unsigned int)a;
    const unsigned int lo = (unsigned int)((a - (float)hi) * 0x1p24f);
    return ((unsigned long long)hi << 24) + lo;
}

constexpr int kWeightThreads = 1024;
constexpr int kMaxRange = 16384;              // positions of a range: 128 KB of LDS
constexpr int kFewRange = 4096;               // of a range when there are few entries (weight_plan())
constexpr int kMaxChunkRows = 1 << 15;        // rows whose sum fits 64 bits: 2^15 2^48

template <int RANGE>
__global__ __launch_bounds__(kWeightThreads) void weight_kernel(WeightArgs a)
{
    __shared__ unsigned long long sum[RANGE];
    const int tid = threadIdx.x;
    const int range = blockIdx.x % a.n_ranges, rest = blockIdx.x / a.n_ranges;
    const int chunk = rest % a.n_chunks, b = rest / a.n_chunks;
    const int lo = range * a.range, n = min(a.range, a.Lk - lo);
    const int64_t t0 = (int64_t)chunk * a.chunk_rows, t1 = min(t0 + a.chunk_rows, (int64_t)a.Tq);
    const int64_t at = ((int64_t)b * a.Tq + t0) * a.k_sel, entries = (t1 - t0) * a.k_sel;
    const int32_t *idx = a.idx + at;
    const float *p = a.probs + at;
    const int64_t w0 = (int64_t)b * a.Lk + lo;
    // what was there, asked for ahead of everything (4096 positions: 4 a thread)
    float in[kFewRange / kWeightThreads];
    if (RANGE == kFewRange && a.n_chunks == 1 && a.in)
#pragma unroll
        for (int j = 0; j < kFewRange / kWeightThreads; ++j) in[j] = a.in[w0 + min(j * kWeightThreads + tid, n - 1)];
    for (int i = tid; i < n; i += kWeightThreads) sum[i] = 0ull;
    __syncthreads();
    // eight entries a thread at a time: one after the other, their loads take as long as everything else (67 us against 26 for 8191 rows of 2048)
    constexpr int kAtOnce = 8;
    for (int64_t e0 = 0; e0 < entries; e0 += kAtOnce * kWeightThreads) {
        const int32_t *const ie = idx + e0;
        const float *const pe = p + e0;
        const int left = (int)min((int64_t)kAtOnce * kWeightThreads, entries - e0);
        int s[kAtOnce];
        float v[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int e = u * kWeightThreads + tid;
            s[u] = (int)((unsigned)ie[min(e, left - 1)] - (unsigned)lo);    // (without overflow for any entry)
            s[u] = e < left && s[u] >= 0 && s[u] < n ? s[u] : -1;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) v[u] = pe[s[u] >= 0 ? u * kWeightThreads + tid : 0];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            if (s[u] >= 0) atomicAdd(&sum[s[u]], fixed48(v[u]));
    }
    __syncthreads();
    if (a.n_chunks > 1) {
        unsigned long long *const part = a.part + (((int64_t)b * a.n_chunks + chunk) * a.Lk + lo);
        for (int i = tid; i < n; i += kWeightThreads) part[i] = sum[i];
    } else if (RANGE == kFewRange) {
#pragma unroll
        for (int j = 0; j < kFewRange / kWeightThreads; ++j) {
            const int i = j * kWeightThreads + tid;
            if (i < n) a.out[w0 + i] = (float)((a.in ? (double)in[j] : 0.0) + (double)sum[i] * 0x1p-48);
        }
    } else {
        for (int i = tid; i < n; i += kWeightThreads) a.out[w0 + i] = (float)((a.in ? (double)a.in[w0 + i] : 0.0) + (double)sum[i] * 0x1p-48);
    }
}

// The chunks' sums: 2^per_log2 threads to a position, whose sums are added in their order.
__global__ __launch_bounds__(1024) void weight_sum_kernel(WeightArgs a, int per_log2)
{
    __shared__ double sums[1024];
    const int tid = threadIdx.x, n_log2 = 10 - per_log2, x = tid & ((1 << n_log2) - 1), y = tid >> n_log2;
    const int64_t all = (int64_t)a.B * a.Lk, w = ((int64_t)blockIdx.x << n_log2) + x;
    if (w < all) {
        const int64_t b = w / a.Lk;
        const unsigned long long *const part = a.part + (b * a.n_chunks * a.Lk + (w - b * a.Lk));
        double t = 0.0;
#pragma unroll 4
        for (int c = y; c < a.n_chunks; c += 1 << per_log2) t += (double)part[(int64_t)c * a.Lk] * 0x1p-48;
        sums[tid] = t;
    }
    __syncthreads();
    if (y == 0 && w < all) {
        double t = a.in ? (double)a.in[w] : 0.0;
        for (int c = 0; c < 1 << per_log2; ++c) t += sums[(c << n_log2) + x];
        a.out[w] = (float)t;
    }
}

// Order of the weights as unsigned integers (-0 and +0 are one value, a NaN is above infinity).
__device__ __forceinline__ unsigned int weight_key(float w)
{
    if (w != w) return 0xFFFFFFFFu;
    const unsigned int u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// ---- which positions stay -------------------------------------------------------------------------------------------
//
// Three digits of the keys, 11, 11 and 10 bits, from the top: a digit's histogram over the keys whose higher digits are the
// border's says which value of it the border has and how many keys are still to be taken below; after the third the border is
// one key, and of its positions the lowest are taken.  Keys stay in registers, 1024 apart, so a (register, wave) pair is a run
// of 64 positions and the places of the kept ones follow from those runs' counts.
// What positions hold most often is zero (nothing ever selected them): additions to one LDS word go one after the other, so the
// keys of zero are counted by ballots.

constexpr int kEvictThreads = 1024;
constexpr unsigned int kZeroKey = 0x80000000u;

// From `bins` (descending: bin t of this thread's digit order), the digit at which the running number reaches `left`.
struct Digit {
    unsigned int value, left;                 // the border's digit; how many of the keys that have it are taken
};
__device__ __forceinline__ Digit find_digit(const unsigned int (&n)[2], int n_bins, unsigned int left, unsigned int *sh, int tid)
{
    // n[0]: the higher bin (n_bins - 1 - 2 t), n[1]: the one below it
    const int lane = tid & 63, wave = tid >> 6;
    const unsigned int own = n[0] + n[1], incl = wave_incl_scan(own);
    if (lane == 63) sh[wave] = incl;
    __syncthreads();
    unsigned int before = incl - own;
#pragma unroll
    for (int v = 0; v < kEvictThreads / 64; ++v) before += v < wave ? sh[v] : 0u;
    if (before < left && left <= before + own) {
        const bool low = before + n[0] < left;
        sh[16] = (unsigned)(n_bins - 1 - 2 * tid - (low ? 1 : 0));
        sh[17] = left - before - (low ? n[0] : 0u);
    }
    __syncthreads();
    const Digit d = {sh[16], sh[17]};
    __syncthreads();
    return d;
}

__device__ __forceinline__ unsigned int digit_of(unsigned int k, int level) { return level == 0 ? k >> 21 : level == 1 ? k >> 10 & 2047u : k & 1023u; }
__device__ __forceinline__ bool same_above(unsigned int k, unsigned int border, int level)   // the digits above `level` are the border's
{
    return level == 0 || (level == 1 ? k >> 21 == border >> 21 : k >> 10 == border >> 10);
}

// A level's histogram of this workgroup's keys that lie in [lo, hi), from position p0.
template <int R>
__device__ __forceinline__ void count_digits(unsigned int *hist, const unsigned int (&key)[R], int p0, int lo, int hi, unsigned int border, int level, int tid)
{
    const int n_bins = level == 2 ? 1024 : 2048;
    for (int i = tid; i < n_bins; i += kEvictThreads) hist[i] = 0;
    __syncthreads();
    unsigned int zeros = 0;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int i = p0 + j * kEvictThreads + tid;
        const bool mine = i >= lo && i < hi && same_above(key[j], border, level), zero = key[j] == kZeroKey;
        zeros += (unsigned)__popcll(__ballot(mine && zero));
        if (mine && !zero) atomicAdd(&hist[digit_of(key[j], level)], 1u);
    }
    if ((tid & 63) == 0 && zeros != 0u) atomicAdd(&hist[digit_of(kZeroKey, level)], zeros);
    __syncthreads();
}

// Writes what stays of a run of R * 1024 positions from p0: those with take_all or above the border, and of the ties the first
// `left`, `ties0` of which lie before p0.  at0: how many positions in front of p0 stay.
template <int R>
__device__ __forceinline__ void emit_kept(const EvictArgs &a, int b, int p0, int lo, int hi, int len, bool any, unsigned int border, unsigned int left,
                                          unsigned int ties0, unsigned int at0, const unsigned int (&key)[R], const float (&w)[R],
                                          unsigned int (*runs)[2], int tid)
{
    const int lane = tid & 63, wave = tid >> 6;
    constexpr int kWaves = kEvictThreads / 64, kRuns = R * kWaves;
    const unsigned long long below = (1ull << lane) - 1;
    // counts of the runs: {kept for certain, ties}
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int i = p0 + j * kEvictThreads + tid;
        const bool in = i < len, inner = i >= lo && i < hi;
        const unsigned long long ma = __ballot(in && (!inner || (any && key[j] > border))), mt = __ballot(in && inner && any && key[j] == border);
        if (lane == 0) {
            runs[j * kWaves + wave][0] = (unsigned)__popcll(ma);
            runs[j * kWaves + wave][1] = (unsigned)__popcll(mt);
        }
    }
    __syncthreads();
    if (wave == 0) {                           // exclusive sums over the runs, 64 at a time
        unsigned int sa = 0, st = ties0;
        for (int r0 = 0; r0 < kRuns; r0 += 64) {
            const int r = r0 + lane;
            const unsigned int na = r < kRuns ? runs[r][0] : 0u, nt = r < kRuns ? runs[r][1] : 0u;
            const unsigned int ia = wave_incl_scan(na), it = wave_incl_scan(nt);
            if (r < kRuns) {
                runs[r][0] = sa + ia - na;
                runs[r][1] = st + it - nt;
            }
            sa += (unsigned)__builtin_amdgcn_readlane((int)ia, 63);
            st += (unsigned)__builtin_amdgcn_readlane((int)it, 63);
        }
    }
    __syncthreads();
    int32_t *keep = a.keep + (int64_t)b * a.n_keep;
    float *kept = a.kept ? a.kept + (int64_t)b * a.n_keep : nullptr;
    const unsigned int ties_taken0 = min(ties0, left);
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int i = p0 + j * kEvictThreads + tid;
        const bool in = i < len, inner = i >= lo && i < hi;
        const bool sure = in && (!inner || (any && key[j] > border)), tie = in && inner && any && key[j] == border;
        const unsigned long long ma = __ballot(sure), mt = __ballot(tie);
        const unsigned int ties = runs[j * kWaves + wave][1] + (unsigned)__popcll(mt & below);       // of the sequence, before this position
        if (sure || (tie && ties < left)) {
            const unsigned int at = at0 + runs[j * kWaves + wave][0] + (unsigned)__popcll(ma & below) + min(ties, left) - ties_taken0;
            if (at < (unsigned)a.n_keep) {
                keep[at] = i;
                if (kept) kept[at] = w[j];
            }
        }
    }
}

// What every form does first: the sequence's length and number, and all of the outputs where nothing has to go.
// Returns false when nothing else is to be done.
__device__ __forceinline__ bool evict_begin(const EvictArgs &a, int b, int part, int n_parts, bool write, int *len_out, int tid)
{
    const int len = a.seq_lens ? max(0, min(a.seq_lens[b], a.Lk)) : a.Lk;
    const int n = min(len, a.n_keep);
    *len_out = len;
    if (write) {
        if (tid == 0 && part == 0) a.lens[b] = n;
        const bool all = len <= a.n_keep;
        for (int i = (all ? 0 : n) + part * kEvictThreads + tid; i < a.n_keep; i += n_parts * kEvictThreads) {
            const int64_t at = (int64_t)b * a.n_keep + i;
            a.keep[at] = i < n ? i : -1;
            if (a.kept) a.kept[at] = i < n ? a.weight[(int64_t)b * a.Lk + i] : 0.f;
        }
    }
    return len > a.n_keep;
}

// One workgroup per sequence of up to R * 1024 positions.
template <int R>
__global__ __launch_bounds__(kEvictThreads) void evict_kernel(EvictArgs a)
{
    __shared__ unsigned int hist[2048], sh[32];
    __shared__ unsigned int runs[R * kEvictThreads / 64][2];
    const int tid = threadIdx.x, b = blockIdx.x;
    int len;
    if (!evict_begin(a, b, 0, 1, true, &len, tid)) return;
    const int lo = a.n_first, hi = len - a.n_recent, want = a.n_keep - a.n_first - a.n_recent;
    float w[R];
    unsigned int key[R];
#pragma unroll
    for (int j = 0; j < R; ++j) w[j] = a.weight[(int64_t)b * a.Lk + min(j * kEvictThreads + tid, len - 1)];
#pragma unroll
    for (int j = 0; j < R; ++j) key[j] = weight_key(w[j]);
    unsigned int border = 0, left = (unsigned)want;
    if (want > 0) {
#pragma unroll
        for (int level = 0; level < 3; ++level) {
            count_digits<R>(hist, key, 0, lo, hi, border, level, tid);
            const int n_bins = level == 2 ? 1024 : 2048, bin = n_bins - 1 - 2 * tid;
            const unsigned int n[2] = {bin > 0 ? hist[bin] : 0u, bin > 0 ? hist[bin - 1] : 0u};
            const Digit d = find_digit(n, n_bins, left, sh, tid);
            border |= d.value << (level == 0 ? 21 : level == 1 ? 10 : 0);
            left = d.left;
        }
    }
    emit_kept<R>(a, b, 0, lo, hi, len, want > 0, border, left, 0u, 0u, key, w, runs, tid);
}

// Longer sequences: a workgroup per 8192 positions and a launch per digit, and one that writes.  Each launch adds up the
// workgroups' histograms of the digit before it (4 KB each) by itself.  Bound by latency: weights, histograms, LDS additions one
// after the other.  200 000 positions: 28 us in four launches (430 in one workgroup; 35 with 16384 positions and 8 KB each, 29
// with 4096), 32 sequences of 65536 in 30.
constexpr int kPart = kEvictPart, kPartR = kPart / kEvictThreads;
struct PartCounts {
    unsigned int hist[2][1024], last[512];    // two bins a word: a part has no more than 8192 keys
    unsigned int above[2];                    // inner keys above the border by the first digit; by the second
    unsigned int border[2], left[2];          // (of part 0: as the second and the third launch have found them)
};

template <int LEVEL>
__global__ __launch_bounds__(kEvictThreads) void evict_part_kernel(EvictArgs a)
{
    __shared__ unsigned int hist[2048], sh[32];
    __shared__ unsigned int runs[kPartR * kEvictThreads / 64][2];
    __shared__ unsigned int before[2];
    const int tid = threadIdx.x;
    const int b = blockIdx.x / a.n_parts, part = blockIdx.x - b * a.n_parts;
    int len;
    if (!evict_begin(a, b, part, a.n_parts, LEVEL == 3, &len, tid)) return;
    const int lo = a.n_first, hi = len - a.n_recent, want = a.n_keep - a.n_first - a.n_recent;
    const int p0 = part * kPart;
    if (p0 >= len || (LEVEL < 3 && want == 0)) return;
    const int live = (len - 1) / kPart + 1;                                 // parts that hold positions
    PartCounts *const seq = (PartCounts *)a.ws + (int64_t)b * a.n_parts, *const own = seq + part;
    float w[kPartR];
    unsigned int key[kPartR];
#pragma unroll
    for (int j = 0; j < kPartR; ++j) w[j] = a.weight[(int64_t)b * a.Lk + min(p0 + j * kEvictThreads + tid, len - 1)];
    unsigned int border = 0, left = (unsigned)want;
    if (LEVEL >= 2 && want > 0) {
        border = seq[0].border[LEVEL - 2];
        left = seq[0].left[LEVEL - 2];
    }
    if (LEVEL == 3 && tid < 2) before[tid] = 0;
    if (LEVEL >= 1 && want > 0) {
        // the digit of the level before: the parts' histograms together
        constexpr int n_bins = LEVEL == 3 ? 1024 : 2048;
        const int bin = n_bins - 1 - 2 * tid;
        unsigned int n[2] = {0u, 0u}, front[2] = {0u, 0u};                  // of all parts; of those before this one
        if (bin > 0) {
#pragma unroll 8
            for (int c = 0; c < live; ++c) {
                const unsigned int *h = LEVEL == 3 ? seq[c].last : seq[c].hist[(LEVEL - 1) & 1];
                const unsigned int x = h[bin >> 1];
                n[0] += x >> 16;
                n[1] += x & 0xFFFFu;
                if (LEVEL == 3 && c < part) {
                    front[0] += x >> 16;
                    front[1] += x & 0xFFFFu;
                }
            }
        }
        const Digit d = find_digit(n, n_bins, left, sh, tid);
        border |= d.value << (LEVEL == 1 ? 21 : LEVEL == 2 ? 10 : 0);
        left = d.left;
        if (LEVEL == 3 && bin > 0) {
            const unsigned int over = ((unsigned)bin > d.value ? front[0] : 0u) + ((unsigned)(bin - 1) > d.value ? front[1] : 0u);
            const unsigned int tie = ((unsigned)bin == d.value ? front[0] : 0u) + ((unsigned)(bin - 1) == d.value ? front[1] : 0u);
            if (over) atomicAdd(&before[0], over);
            if (tie) atomicAdd(&before[1], tie);
        }
    }
#pragma unroll
    for (int j = 0; j < kPartR; ++j) key[j] = weight_key(w[j]);
    if (LEVEL < 3) {
        count_digits<kPartR>(hist, key, p0, lo, hi, border, LEVEL, tid);
        unsigned int *out = LEVEL == 2 ? own->last : own->hist[LEVEL & 1];
        if (tid < (LEVEL == 2 ? 512 : 1024)) out[tid] = hist[2 * tid] | hist[2 * tid + 1] << 16;
        if (LEVEL >= 1) {
            // keys above the border by the digit that this launch has found (equal in the digits before it)
            unsigned int n = 0;
#pragma unroll
            for (int j = 0; j < kPartR; ++j) {
                const bool over = LEVEL == 1 ? key[j] >> 21 > border >> 21 : (key[j] >> 21 == border >> 21 && key[j] >> 10 > border >> 10);
                const int i = p0 + j * kEvictThreads + tid;
                n += (unsigned)__popcll(__ballot(i >= lo && i < hi && over));
            }
            if ((tid & 63) == 0) sh[tid >> 6] = n;
            __syncthreads();
            if (tid == 0) {
                unsigned int t = 0;
                for (int v = 0; v < kEvictThreads / 64; ++v) t += sh[v];
                own->above[LEVEL - 1] = t;
            }
        }
        if (LEVEL >= 1 && part == 0 && tid == 0) {
            // (a place of each launch's own: this one's workgroups read what the one before it left)
            own->border[LEVEL - 1] = border;
            own->left[LEVEL - 1] = left;
        }
        return;
    }
    __syncthreads();
    // positions that stay in front of this part
    const int outer = min(p0, lo) + max(0, p0 - max(hi, lo));
    unsigned int at = (unsigned)outer, ties = 0;
    if (want > 0) {
#pragma unroll 8
        for (int c = 0; c < part; ++c) at += seq[c].above[0] + seq[c].above[1];
        ties = before[1];
        at += before[0] + min(ties, left);
    }
    emit_kept<kPartR>(a, b, p0, lo, hi, len, want > 0, border, left, ties, at, key, w, runs, tid);
}

constexpr int kMoveRows = 32;                 // rows of a workgroup

// PAST: past the caches (launch_compact())
template <typename T, bool PAST>
__device__ __forceinline__ void move_rows(const CompactArgs &a, int c, const int64_t *src, const int64_t *dst, int tid)
{
    const int per = a.row_bytes[c] / (int)sizeof(T), total = kMoveRows * per;
    for (int i = tid; i < total; i += 256) {
        const int r = i / per, k = i - r * per;
        const int64_t s = src[r], d = dst[r];
        if (s >= 0 && s < a.src_rows[c] && d >= 0 && d < a.dst_rows[c]) {
            const T x = *((const T *)(a.src[c] + s * a.row_bytes[c]) + k);
            T *const to = (T *)(a.dst[c] + d * a.row_bytes[c]) + k;
            if (PAST)
                __builtin_nontemporal_store(x, to);
            else
                *to = x;
        }
    }
}

template <bool PAST>
__global__ __launch_bounds__(256) void compact_kernel(CompactArgs a)
{
    __shared__ int64_t src[kMoveRows], dst[kMoveRows];
    const int tid = threadIdx.x, c = blockIdx.y;
    const unsigned int per_seq = (unsigned)(a.n_keep - 1) / kMoveRows + 1, at = blockIdx.z * gridDim.x + blockIdx.x;   // (see launch_compact())
    if (at / per_seq >= (unsigned)a.B) return;
    const int b = (int)(at / per_seq), j0 = (int)(at - b * per_seq) * kMoveRows;
    if (tid < kMoveRows) {
        const int j = j0 + tid;
        const int s = j < a.n_keep ? a.keep[(int64_t)b * a.n_keep + j] : -1;
        const bool there = s >= 0 && s < a.Lk;
        src[tid] = !there ? -1 : a.sv.page_table ? paged_row(a.sv, b, s) : (int64_t)b * a.Lk + s;
        dst[tid] = !there ? -1 : a.dv.page_table ? paged_row(a.dv, b, j) : (int64_t)b * a.n_keep + j;
    }
    __syncthreads();
    const uintptr_t any = (uintptr_t)a.src[c] | (uintptr_t)a.dst[c] | (uintptr_t)a.row_bytes[c];
    if (any % 16 == 0)
        move_rows<u32x4, PAST>(a, c, src, dst, tid);
    else
        move_rows<unsigned int, PAST>(a, c, src, dst, tid);
}

} // namespace

// n things by `per` (both may be near 2^31).
static int groups(int n, int per) { return (n - 1) / per + 1; }

// Ranges and chunks of a call.  One chunk: the launch writes the weights itself.
// A range is what LDS holds, as every range's workgroup goes through all of the entries; with no more than 16 of them per
// position of a short range that costs less than the positions, and four times the workgroups take them (32 sequences of 65536
// positions, 2048 entries each: 7.8 us against 11.5; one of 200 000, 32768 entries: 8.7 against 12.6).
void weight_plan(WeightArgs &a)
{
    const int most = (int64_t)a.Tq * a.k_sel <= 16 * kFewRange ? kFewRange : kMaxRange;
    a.range = a.Lk < most ? a.Lk : most;
    a.n_ranges = groups(a.Lk, a.range);
    int chunks = 1;
    if (a.Tq > 16) {
        chunks = 256 / (a.B * a.n_ranges > 256 ? 256 : a.B * a.n_ranges);
        if (chunks > a.Tq / 16) chunks = a.Tq / 16;
    }
    const int least = groups(a.Tq, kMaxChunkRows);
    if (chunks < least) chunks = least;
    a.chunk_rows = groups(a.Tq, chunks);
    a.n_chunks = groups(a.Tq, a.chunk_rows);
}

hipError_t launch_weight_add(const WeightArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)(a.B * a.n_ranges * a.n_chunks)), block(kWeightThreads);
    if (a.range <= kFewRange)
        hipLaunchKernelGGL((weight_kernel<kFewRange>), grid, block, 0, st, a);
    else
        hipLaunchKernelGGL((weight_kernel<kMaxRange>), grid, block, 0, st, a);
    if (a.n_chunks > 1) {
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        int per_log2 = 1;
        while (per_log2 < 5 && (1 << per_log2) < a.n_chunks) ++per_log2;
        const int64_t n = 1024 >> per_log2;
        hipLaunchKernelGGL(weight_sum_kernel, dim3((unsigned)(((int64_t)a.B * a.Lk + n - 1) / n)), dim3(1024), 0, st, a, per_log2);
    }
    return hipGetLastError();
}

// A workgroup holds up to 32768 keys, 16384 in half of the registers; longer sequences are taken in parts, from 16384 positions on
// where the parts have a compute unit each (24000 positions: 1 sequence 20 us in parts and 29 in a workgroup, 32 22 and 29, 256
// 49 and 33; 16384: 19 and 16, 20 and 17, 33 and 20).
int evict_parts(int B, int Lk)
{
    const int parts = groups(Lk, kPart);
    return Lk > 32 * kEvictThreads || (Lk > 16 * kEvictThreads && (int64_t)B * parts <= 256) ? parts : 0;
}
size_t evict_ws_bytes(int B, int Lk) { return (size_t)B * evict_parts(B, Lk) * sizeof(PartCounts); }

hipError_t launch_evict_keep(EvictArgs a, hipStream_t st)
{
    a.n_parts = evict_parts(a.B, a.Lk);
    if (a.n_parts == 0) {
        const int per = (a.Lk + kEvictThreads - 1) / kEvictThreads;
        const dim3 grid((unsigned)a.B), block(kEvictThreads);
        if (per <= 1)
            hipLaunchKernelGGL((evict_kernel<1>), grid, block, 0, st, a);
        else if (per <= 8)
            hipLaunchKernelGGL((evict_kernel<8>), grid, block, 0, st, a);
        else if (per <= 16)
            hipLaunchKernelGGL((evict_kernel<16>), grid, block, 0, st, a);
        else
            hipLaunchKernelGGL((evict_kernel<32>), grid, block, 0, st, a);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)(a.B * a.n_parts)), block(kEvictThreads);
    hipLaunchKernelGGL((evict_part_kernel<0>), grid, block, 0, st, a);
    hipLaunchKernelGGL((evict_part_kernel<1>), grid, block, 0, st, a);
    hipLaunchKernelGGL((evict_part_kernel<2>), grid, block, 0, st, a);
    hipLaunchKernelGGL((evict_part_kernel<3>), grid, block, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_compact(const CompactArgs &a, hipStream_t st)
{
    // a dimension of a launch has less than 2^32 threads: 2^23 workgroups a step of z, up to 2^31 of them
    const int64_t wgs = (int64_t)a.B * groups(a.n_keep, kMoveRows), x = wgs < (1 << 23) ? wgs : 1 << 23;
    const dim3 grid((unsigned)x, (unsigned)a.n_caches, (unsigned)((wgs + x - 1) / x)), block(256);
    int64_t bytes = 0;
    for (int c = 0; c < a.n_caches; ++c) bytes += (int64_t)a.B * a.n_keep * a.row_bytes[c];
    // What is more than the last cache holds (256 MB) goes past the caches: the step behind would not find it there, and it is faster
    // (344 MB 144 us against 150).
    if (bytes > (int64_t)256 << 20)
        hipLaunchKernelGGL((compact_kernel<true>), grid, block, 0, st, a);
    else
        hipLaunchKernelGGL((compact_kernel<false>), grid, block, 0, st, a);
    return hipGetLastError();
}

} // namespace ic
