// Eviction from a cache by accumulated attention weight: what each position received, which positions stay, and their rows
// moved together.
//
//   weight_kernel   weight[s] = in[s] + sum over the query rows of probs at the slots that name s.  A workgroup owns a range of
//                   positions in LDS and adds there in 64-bit fixed point (units of 2^-48), so the order of the additions
//                   does not show in the sum.  Bound by memory (probs and idx once), or for a few rows by the launch.
//   evict_kernel    the n_keep positions of a sequence that stay: the first n_first, the last n_recent, and the largest weights
//                   among the others (equal weights: the lower position).  Radix selection on the bits, then the positions in
//                   order.
//   compact_kernel  rows of several caches to their new places.  Bound by memory.
#include "ic_common.hpp"

namespace ic {

namespace {

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
constexpr int kMaxChunkRows = 1 << 15;        // rows whose sum fits 64 bits: 2^15 2^48

__global__ __launch_bounds__(kWeightThreads) void weight_kernel(WeightArgs a)
{
    __shared__ unsigned long long sum[kMaxRange];
    const int tid = threadIdx.x;
    const int range = blockIdx.x % a.n_ranges, rest = blockIdx.x / a.n_ranges;
    const int chunk = rest % a.n_chunks, b = rest / a.n_chunks;
    const int lo = range * a.range, n = min(a.range, a.Lk - lo);
    for (int i = tid; i < n; i += kWeightThreads) sum[i] = 0ull;
    __syncthreads();
    const int64_t t0 = (int64_t)chunk * a.chunk_rows, t1 = min(t0 + a.chunk_rows, (int64_t)a.Tq);
    const int64_t at = ((int64_t)b * a.Tq + t0) * a.k_sel, entries = (t1 - t0) * a.k_sel;
    const int32_t *idx = a.idx + at;
    const float *p = a.probs + at;
    for (int64_t e = tid; e < entries; e += kWeightThreads) {
        const int s = idx[e] - lo;
        if (s >= 0 && s < n) atomicAdd(&sum[s], fixed48(p[e]));
    }
    __syncthreads();
    for (int i = tid; i < n; i += kWeightThreads) {
        if (a.n_chunks == 1) {
            const int64_t w = (int64_t)b * a.Lk + lo + i;
            a.out[w] = (float)((a.in ? (double)a.in[w] : 0.0) + (double)sum[i] * 0x1p-48);
        } else {
            a.part[((int64_t)b * a.n_chunks + chunk) * a.Lk + lo + i] = sum[i];
        }
    }
}

__global__ __launch_bounds__(256) void weight_sum_kernel(WeightArgs a)
{
    const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (w >= (int64_t)a.B * a.Lk) return;
    const int64_t b = w / a.Lk, s = w - b * a.Lk;
    double t = a.in ? (double)a.in[w] : 0.0;
    for (int c = 0; c < a.n_chunks; ++c) t += (double)a.part[(b * a.n_chunks + c) * a.Lk + s] * 0x1p-48;
    a.out[w] = (float)t;
}

// Order of the weights as unsigned integers (-0 and +0 are one value, a NaN is above infinity).
__device__ __forceinline__ unsigned int weight_key(float w)
{
    if (w != w) return 0xFFFFFFFFu;
    const unsigned int u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One workgroup per sequence.
__global__ __launch_bounds__(1024) void evict_kernel(EvictArgs a)
{
    __shared__ unsigned int hist[256], wave_n[2][16];
    __shared__ unsigned int s_prefix, s_left;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = blockIdx.x;
    const int len = a.seq_lens ? max(0, min(a.seq_lens[b], a.Lk)) : a.Lk;
    const float *w = a.weight + (int64_t)b * a.Lk;
    int32_t *keep = a.keep + (int64_t)b * a.n_keep;
    float *kept = a.kept ? a.kept + (int64_t)b * a.n_keep : nullptr;
    const int n = min(len, a.n_keep);
    if (tid == 0) a.lens[b] = n;
    for (int i = n + tid; i < a.n_keep; i += 1024) {
        keep[i] = -1;
        if (kept) kept[i] = 0.f;
    }
    if (len <= a.n_keep) {
        for (int i = tid; i < n; i += 1024) {
            keep[i] = i;
            if (kept) kept[i] = w[i];
        }
        return;
    }
    // of the positions [lo, hi) the `want` largest
    const int lo = a.n_first, hi = len - a.n_recent, want = a.n_keep - a.n_first - a.n_recent;
    unsigned int prefix = 0, left = (unsigned)want;
    for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i = lo + tid; i < hi; i += 1024) {
            const unsigned int k = weight_key(w[i]);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            unsigned int above = 0;
            int d = 255;
            while (d > 0 && above + hist[d] < left) above += hist[d--];
            s_prefix = prefix | (unsigned)d << shift;
            s_left = left - above;
        }
        __syncthreads();
        prefix = s_prefix;
        left = s_left;
    }
    // prefix is the key of the last one taken, `left` of the positions that have it are taken, the lowest
    int done = 0;
    unsigned int ties = 0;
    for (int i0 = 0; i0 < len; i0 += 1024) {
        const int i = i0 + tid;
        bool above = false, tie = false;
        float x = 0.f;
        if (i < len) {
            x = w[i];
            const unsigned int k = weight_key(x);
            const bool inner = i >= lo && i < hi;
            above = !inner || (want > 0 && k > prefix);
            tie = inner && want > 0 && k == prefix;
        }
        const unsigned long long mt = __ballot(tie), below = (1ull << lane) - 1;
        if (lane == 0) wave_n[0][wave] = __popcll(mt);
        __syncthreads();
        unsigned int before = ties, all = ties;
        for (int v = 0; v < 16; ++v) {
            if (v < wave) before += wave_n[0][v];
            all += wave_n[0][v];
        }
        const bool take = above || (tie && before + __popcll(mt & below) < left);
        ties = all;
        const unsigned long long mk = __ballot(take);
        if (lane == 0) wave_n[1][wave] = __popcll(mk);
        __syncthreads();
        int at = done;
        for (int v = 0; v < 16; ++v) {
            if (v < wave) at += wave_n[1][v];
            done += wave_n[1][v];
        }
        at += __popcll(mk & below);
        if (take && at < a.n_keep) {
            keep[at] = i;
            if (kept) kept[at] = x;
        }
        __syncthreads();
    }
}

constexpr int kMoveRows = 32;                 // rows of a workgroup

template <typename T>
__device__ __forceinline__ void move_rows(const CompactArgs &a, int c, const int64_t *src, const int64_t *dst, int tid)
{
    const int per = a.row_bytes[c] / (int)sizeof(T), total = kMoveRows * per;
    for (int i = tid; i < total; i += 256) {
        const int r = i / per, k = i - r * per;
        const int64_t s = src[r], d = dst[r];
        if (s >= 0 && s < a.src_rows[c] && d >= 0 && d < a.dst_rows[c])
            *(T *)(a.dst[c] + d * a.row_bytes[c] + (int64_t)k * sizeof(T)) = *(const T *)(a.src[c] + s * a.row_bytes[c] + (int64_t)k * sizeof(T));
    }
}

__global__ __launch_bounds__(256) void compact_kernel(CompactArgs a)
{
    __shared__ int64_t src[kMoveRows], dst[kMoveRows];
    const int tid = threadIdx.x, c = blockIdx.y;
    const int per_seq = (a.n_keep + kMoveRows - 1) / kMoveRows;
    const int b = blockIdx.x / per_seq, j0 = (blockIdx.x - b * per_seq) * kMoveRows;
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
        move_rows<u32x4>(a, c, src, dst, tid);
    else
        move_rows<unsigned int>(a, c, src, dst, tid);
}

} // namespace

// Ranges and chunks of a call.  One chunk: the launch writes the weights itself.
void weight_plan(WeightArgs &a)
{
    a.range = a.Lk < kMaxRange ? a.Lk : kMaxRange;
    a.n_ranges = (a.Lk + a.range - 1) / a.range;
    int chunks = 1;
    if (a.Tq > 16) {
        chunks = 256 / (a.B * a.n_ranges > 256 ? 256 : a.B * a.n_ranges);
        if (chunks > a.Tq / 16) chunks = a.Tq / 16;
    }
    const int least = (a.Tq + kMaxChunkRows - 1) / kMaxChunkRows;
    if (chunks < least) chunks = least;
    a.chunk_rows = (a.Tq + chunks - 1) / chunks;
    a.n_chunks = (a.Tq + a.chunk_rows - 1) / a.chunk_rows;
}

hipError_t launch_weight_add(const WeightArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(weight_kernel, dim3((unsigned)(a.B * a.n_ranges * a.n_chunks)), dim3(kWeightThreads), 0, st, a);
    if (a.n_chunks > 1) {
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(weight_sum_kernel, dim3((unsigned)(((int64_t)a.B * a.Lk + 255) / 256)), dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

hipError_t launch_evict_keep(const EvictArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(evict_kernel, dim3((unsigned)a.B), dim3(1024), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_compact(const CompactArgs &a, hipStream_t st)
{
    const int per_seq = (a.n_keep + kMoveRows - 1) / kMoveRows;
    hipLaunchKernelGGL(compact_kernel, dim3((unsigned)(a.B * per_seq), (unsigned)a.n_caches), dim3(256), 0, st, a);
    return hipGetLastError();
}

} // namespace ic
