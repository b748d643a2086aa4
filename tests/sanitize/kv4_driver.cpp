// Walks the host side of the 4-bit cache's and of eviction's entry points, sizes at the ends of their ranges among them, in a build
// whose host code is instrumented.  No GPU is needed: every call is rejected before any launch.  Test infrastructure
// (tests/test_kv4_sanitizers.py builds and runs it); prints "kv4 sanitizer run ok".
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <initializer_list>

#include "indexcache.h"

#define CHECK(x) do { if (!(x)) { std::fprintf(stderr, "check failed line %d: %s (%s)\n", __LINE__, #x, ic_last_error()); return 1; } } while (0)

int main()
{
    void *one = (void *)4096;
    int32_t *ints = (int32_t *)one;
    float *floats = (float *)one;
    const int32_t big = INT32_MAX;

    ic_kv4_desc kd;
    std::memset(&kd, 0, sizeof kd);
    kd.B = 1; kd.Tn = big; kd.Lk = big; kd.pool_rows = big;
    CHECK(ic_kv4_write(&kd, nullptr, nullptr, one, nullptr) == IC_ERR_NULL);
    CHECK(ic_kv4_read(&kd, nullptr, one, (void *)4104, nullptr) == IC_ERR_SHAPE);
    kd.B = big;
    CHECK(ic_kv4_write(&kd, nullptr, one, one, nullptr) == IC_ERR_SHAPE);
    kd.Tn = 1;
    CHECK(ic_kv4_write(&kd, nullptr, one, one, nullptr) == IC_ERR_SHAPE);        // B Lk rows are not there
    kd.B = 1; kd.pos0 = INT64_MIN;
    CHECK(ic_kv4_read(&kd, nullptr, one, one, nullptr) == IC_ERR_SHAPE);

    ic_attn_desc at;
    std::memset(&at, 0, sizeof at);
    at.B = 1; at.Tq = 1; at.Lk = big; at.H_q = 32; at.d_qk = 576; at.d_v = 512; at.row_elems = 576; at.sm_scale = 0.04f;
    const int32_t ks[] = {1, 2048, 1 << 24, (1 << 24) + 1, big};
    for (int32_t k : ks)
        for (int32_t nq : {1, 127, 255, 256, 513, big / 2, big}) {
            at.k_sel = k;
            at.Tq = nq;
            const bool fits = k <= 1 << 24 && nq <= big / 2;
            const size_t need = ic_sparse_attn_kv4_workspace(&at);
            CHECK(fits || need == 0);
            const ic_status s = ic_sparse_attn_kv4(&at, nullptr, big, nullptr, one, ints, one, nullptr, one, need, nullptr);
            CHECK(s == (fits ? IC_ERR_NULL : k > 1 << 24 && nq <= big / 2 ? IC_ERR_UNSUPPORTED : IC_ERR_SHAPE));
            CHECK(ic_attn_probs_kv4(&at, nullptr, big, one, one, ints, nullptr, floats, nullptr) == s);
        }

    for (int32_t B : {1, 40, 65535, 65536, big})
        for (int32_t Tq : {1, 17, 32768, 32769, big})
            for (int32_t Lk : {1, 4096, 4097, 16384, 200000, big}) {
                const bool fits = B <= 65535 && (int64_t)B * Tq <= big && (int64_t)B * Lk <= big;
                const size_t need = ic_attn_weight_add_workspace(B, Tq, big, Lk);
                CHECK(fits || need == 0);
                CHECK(ic_attn_weight_add(B, Tq, big, Lk, nullptr, ints, nullptr, floats, one, need, nullptr) ==
                      (fits ? IC_ERR_NULL : B > 65535 ? IC_ERR_UNSUPPORTED : IC_ERR_SHAPE));
                CHECK(!fits || need == 0 || ic_attn_weight_add(B, Tq, big, Lk, floats, ints, nullptr, floats, one, need - 1, nullptr) == IC_ERR_WORKSPACE);
                CHECK(!fits || ic_attn_weight_add(B, Tq, 1, Lk, floats, ints, nullptr, floats, one, need, nullptr) == IC_ERR_SHAPE);   // on itself
            }

    for (int32_t B : {1, 7, 1 << 20, big})
        for (int32_t Lk : {1, 1024, 16384, 16385, 32769, 200000, big - 8191, big}) {
            const bool holds = (int64_t)B * Lk <= big, fits = holds && Lk <= big - 8191;
            const size_t need = ic_evict_keep_workspace(B, Lk);
            CHECK(fits || need == 0);
            CHECK(ic_evict_keep(B, Lk, nullptr, nullptr, Lk, 0, 0, ints, ints, nullptr, one, need, nullptr) ==
                  (fits ? IC_ERR_NULL : holds ? IC_ERR_UNSUPPORTED : IC_ERR_SHAPE));
            CHECK(ic_evict_keep(B, Lk, floats, nullptr, Lk, big, big, ints, ints, nullptr, one, need, nullptr) == IC_ERR_SHAPE);
            CHECK(!fits || ic_evict_keep(B, Lk, floats, nullptr, Lk, 0, 0, ints, ints, floats, one, need, nullptr) == IC_ERR_SHAPE);   // on itself
        }

    ic_cache_move m[IC_MAX_MOVE_CACHES];
    std::memset(m, 0, sizeof m);
    for (auto &c : m) { c.src = one; c.dst = (void *)(4096 + ((uintptr_t)1 << 50)); c.src_rows = c.dst_rows = (int64_t)1 << 40; c.row_bytes = 1 << 20; }
    CHECK(ic_cache_compact(m, IC_MAX_MOVE_CACHES, 1, big, big, ints, nullptr, nullptr, nullptr) == IC_ERR_SHAPE);   // one destination twice
    CHECK(ic_cache_compact(m, IC_MAX_MOVE_CACHES + 1, 1, big, big, ints, nullptr, nullptr, nullptr) == IC_ERR_SHAPE);
    CHECK(ic_cache_compact(m, 1, big, big, big, ints, nullptr, nullptr, nullptr) == IC_ERR_SHAPE);
    m[0].src_rows = INT64_MAX;
    CHECK(ic_cache_compact(m, 1, 1, big, 1, ints, nullptr, nullptr, nullptr) == IC_ERR_SHAPE);
    std::puts("kv4 sanitizer run ok");
    return 0;
}
