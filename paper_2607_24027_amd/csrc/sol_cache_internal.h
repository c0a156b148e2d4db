// Internal interface between the C ABI of the serving operators (sol_cache_api.cpp) and their gfx950
// kernels (sol_cache.hip, sol_cache_attn.hip).  Not installed; not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace sol {

// Sets the text of sol_attn_last_error() on this thread; returns `code`.
int set_error(int code, const char* text);

constexpr int kPage = 64;   // tokens of a page

// Byte offsets inside one page of one head.
template <int D>
struct PageLayout {
    static constexpr int k = 0, ks = 32 * D, v = 34 * D, vs = 66 * D, bytes = 68 * D;
};

struct Strides {
    long long b, h, n;   // elements
};

struct RopeArgs {
    const void *q, *k;
    void *qo, *ko;
    Strides sq, sk, sqo, sko;
    const void *wq, *wk;
    const float *cos, *sin;
    const int32_t* positions;
    int B, Hq, Hk, N, d, P, rot, pairs, dtype, wdtype;
    float eps;
};
hipError_t launch_qk_norm_rope(const RopeArgs& a, hipStream_t st);

struct TablesArgs {
    const int32_t *lens, *add;
    int32_t *table, *ring;
    const int32_t* state;
    int32_t *lens_out, *state_out, *row_start, *slots, *positions;
    int S, max_pages, P, rows;
};
constexpr int kMaxRequests = 4096;
hipError_t launch_cache_tables(const TablesArgs& a, hipStream_t st);

struct AppendArgs {
    const void *k, *v;
    Strides sk, sv;
    uint8_t* store;
    const int32_t* slots;
    int T, H, d, P, dtype;
};
hipError_t launch_cache_append(const AppendArgs& a, hipStream_t st);

struct ReadArgs {
    const uint8_t* store;
    const int32_t* slots;
    void *k, *v;
    Strides sk, sv;
    int T, H, d, P, dtype;
};
hipError_t launch_cache_read(const ReadArgs& a, hipStream_t st);

struct CacheAttnArgs {
    const void* q;
    void* out;
    Strides sq, so;
    const uint8_t* store;
    const int32_t *table, *lens, *row_start, *positions;
    int S, T, max_rows, Hq, Hk, d, P, max_pages, granule, dtype;
    void* ws;
};
size_t cache_attn_workspace_bytes(int S, int T, int max_rows, int Hq, int Hk, int d, int max_pages);
hipError_t launch_cache_attn(const CacheAttnArgs& a, hipStream_t st);

}  // namespace sol
