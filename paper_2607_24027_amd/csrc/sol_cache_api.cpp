// C ABI of the serving operators: argument checks and launches.  Checks run entirely on the host and return before any
// HIP call.  Nothing is allocated and nothing is kept between calls.
#include "../../include/sol_cache.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/sol_attn.h"
#include "sol_cache_internal.h"

namespace {

int fail(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return sol::set_error(code, buf);
}

int done(hipError_t e, const char* what) {
    if (e != hipSuccess) return fail(SOL_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    return sol::set_error(SOL_OK, "");
}

int check_head(int d, int dtype) {
    if (dtype != SOL_BF16 && dtype != SOL_F32) return fail(SOL_ERR_INVALID_ARG, "dtype must be SOL_BF16 or SOL_F32 (got %d)", dtype);
    if (d != 64 && d != 128) return fail(SOL_ERR_UNSUPPORTED, "d must be 64 or 128 (got %d)", d);
    return SOL_OK;
}

int check_store(const void* store, int heads, int P) {
    if (!store) return fail(SOL_ERR_INVALID_ARG, "store must be non-null");
    if (reinterpret_cast<uintptr_t>(store) & 15) return fail(SOL_ERR_INVALID_ARG, "store must start on 16 bytes");
    if (heads <= 0 || P <= 0) return fail(SOL_ERR_INVALID_ARG, "heads and pages must be positive (got %d, %d)", heads, P);
    if (P > (1 << 24) || heads > 65535) return fail(SOL_ERR_UNSUPPORTED, "at most 16,777,216 pages of 65,535 heads (got %d, %d)", P, heads);
    return SOL_OK;
}

// Rows of d channels: any stride, but no negative ones, and offsets that a 64-bit sum holds.
int check_strides(const char* name, const long long* s, int n) {
    if (!s) return fail(SOL_ERR_INVALID_ARG, "the strides of %s must be given", name);
    for (int i = 0; i < n; ++i)
        if (s[i] < 0 || s[i] > (1LL << 40)) return fail(SOL_ERR_INVALID_ARG, "stride %lld of %s is out of range", s[i], name);
    return SOL_OK;
}

sol::Strides three(const long long* s) { return {s[0], s[1], s[2]}; }
sol::Strides two(const long long* s) { return {0, s[0], s[1]}; }

#define SOL_CHECK(x) \
    if (int rc = (x)) return rc

}  // namespace

extern "C" {

int sol_qk_norm_rope(const void* q, const void* k, void* q_out, void* k_out, const long long* q_strides,
                     const long long* k_strides, const long long* q_out_strides, const long long* k_out_strides,
                     const void* q_weight, const void* k_weight, const float* cos, const float* sin,
                     const int32_t* positions, int B, int Hq, int Hk, int N, int d, int P, int rot, int pairs, float eps,
                     int dtype, int weight_dtype, void* stream) {
    SOL_CHECK(check_head(d, dtype));
    if (weight_dtype != SOL_BF16 && weight_dtype != SOL_F32)
        return fail(SOL_ERR_INVALID_ARG, "weight_dtype must be SOL_BF16 or SOL_F32 (got %d)", weight_dtype);
    if (B <= 0 || N <= 0 || Hq < 0 || Hk < 0 || Hq + (long long)Hk == 0)
        return fail(SOL_ERR_INVALID_ARG, "B, N and the heads must be positive (got %d, %d, %d, %d)", B, N, Hq, Hk);
    if (Hq + (long long)Hk > 65535 || (long long)B * N > (1LL << 27))
        return fail(SOL_ERR_UNSUPPORTED, "too many heads or tokens (got %lld, %lld)", Hq + (long long)Hk, (long long)B * N);
    if (!q != (Hq == 0) || !k != (Hk == 0) || !q != !q_out || !k != !k_out)
        return fail(SOL_ERR_INVALID_ARG, "q and k need heads and an output each, or neither");
    if (q && (q == q_out || q_out == k || q_out == k_out)) return fail(SOL_ERR_INVALID_ARG, "q_out must not alias q, k or k_out");
    if (k && (k == k_out || k_out == q)) return fail(SOL_ERR_INVALID_ARG, "k_out must not alias q or k");
    if (q) {
        SOL_CHECK(check_strides("q", q_strides, 3));
        SOL_CHECK(check_strides("q_out", q_out_strides, 3));
    }
    if (k) {
        SOL_CHECK(check_strides("k", k_strides, 3));
        SOL_CHECK(check_strides("k_out", k_out_strides, 3));
    }
    if (pairs != SOL_ROPE_HALVES && pairs != SOL_ROPE_PAIRS) return fail(SOL_ERR_INVALID_ARG, "pairs must be SOL_ROPE_HALVES or SOL_ROPE_PAIRS (got %d)", pairs);
    if (rot < 0 || rot > d || rot % 8) return fail(SOL_ERR_INVALID_ARG, "rot must be a multiple of 8 from 0 to d (got %d)", rot);
    if (rot > 0 && (!cos || !sin || P <= 0)) return fail(SOL_ERR_INVALID_ARG, "cos and sin of at least one position must be given");
    if (rot > 0 && !positions && N > P) return fail(SOL_ERR_INVALID_ARG, "without positions the tables need a row for each token (%d rows, %d tokens)", P, N);
    if (!(eps > 0.f) || std::isinf(eps)) return fail(SOL_ERR_INVALID_ARG, "eps must be positive and finite");
    sol::RopeArgs a{};
    a.q = q, a.k = k, a.qo = q_out, a.ko = k_out;
    if (q) a.sq = three(q_strides), a.sqo = three(q_out_strides);
    if (k) a.sk = three(k_strides), a.sko = three(k_out_strides);
    a.wq = q_weight, a.wk = k_weight, a.cos = cos, a.sin = sin, a.positions = positions;
    a.B = B, a.Hq = Hq, a.Hk = Hk, a.N = N, a.d = d, a.P = P, a.rot = rot, a.pairs = pairs;
    a.dtype = dtype, a.wdtype = weight_dtype, a.eps = eps;
    return done(sol::launch_qk_norm_rope(a, static_cast<hipStream_t>(stream)), "norm and rotation");
}

int sol_cache_tables(const int32_t* lens, const int32_t* add, int32_t* table, int32_t* ring, const int32_t* state,
                     int32_t* lens_out, int32_t* state_out, int32_t* row_start, int32_t* slots, int32_t* positions, int S,
                     int max_pages, int P, int rows, void* stream) {
    if (!lens || !add || !table || !ring || !state || !lens_out || !state_out || !row_start)
        return fail(SOL_ERR_INVALID_ARG, "lens, add, table, ring, state, lens_out, state_out and row_start must be non-null");
    if (S <= 0 || max_pages <= 0 || P <= 0 || rows < 0)
        return fail(SOL_ERR_INVALID_ARG, "S, max_pages and P must be positive, rows not negative (got %d, %d, %d, %d)", S, max_pages, P, rows);
    if (rows > 0 && (!slots || !positions)) return fail(SOL_ERR_INVALID_ARG, "slots and positions must be non-null");
    if (lens_out == lens || state_out == state) return fail(SOL_ERR_INVALID_ARG, "lens_out and state_out must not alias lens and state");
    if (S > sol::kMaxRequests) return fail(SOL_ERR_UNSUPPORTED, "at most %d requests (got %d)", sol::kMaxRequests, S);
    if (P > (1 << 24) || max_pages > (1 << 24) || (long long)S * max_pages > (1LL << 30) || rows > (1 << 30))
        return fail(SOL_ERR_UNSUPPORTED, "too many pages, table entries or rows (got %d, %lld, %d)", P, (long long)S * max_pages, rows);
    sol::TablesArgs a{lens, add, table, ring, state, lens_out, state_out, row_start, slots, positions, S, max_pages, P, rows};
    return done(sol::launch_cache_tables(a, static_cast<hipStream_t>(stream)), "page tables");
}

int sol_cache_append(const void* k, const void* v, const long long* k_strides, const long long* v_strides, void* store,
                     const int32_t* slots, int T, int heads, int d, int P, int dtype, void* stream) {
    if (!k || !v || !slots) return fail(SOL_ERR_INVALID_ARG, "k, v and slots must be non-null");
    SOL_CHECK(check_head(d, dtype));
    SOL_CHECK(check_store(store, heads, P));
    if (T <= 0) return fail(SOL_ERR_INVALID_ARG, "T must be positive (got %d)", T);
    if ((long long)T * heads > (1LL << 28)) return fail(SOL_ERR_UNSUPPORTED, "too many tokens and heads (got %d, %d)", T, heads);
    SOL_CHECK(check_strides("k", k_strides, 2));
    SOL_CHECK(check_strides("v", v_strides, 2));
    sol::AppendArgs a{k, v, two(k_strides), two(v_strides), static_cast<uint8_t*>(store), slots, T, heads, d, P, dtype};
    return done(sol::launch_cache_append(a, static_cast<hipStream_t>(stream)), "append");
}

int sol_cache_read(const void* store, const int32_t* slots, void* k_out, void* v_out, const long long* k_strides,
                   const long long* v_strides, int T, int heads, int d, int P, int dtype, void* stream) {
    if (!slots || (!k_out && !v_out)) return fail(SOL_ERR_INVALID_ARG, "slots and one of k_out and v_out must be non-null");
    SOL_CHECK(check_head(d, dtype));
    SOL_CHECK(check_store(store, heads, P));
    if (T <= 0) return fail(SOL_ERR_INVALID_ARG, "T must be positive (got %d)", T);
    if ((long long)T * heads > (1LL << 28)) return fail(SOL_ERR_UNSUPPORTED, "too many tokens and heads (got %d, %d)", T, heads);
    if (k_out == v_out) return fail(SOL_ERR_INVALID_ARG, "k_out and v_out must differ");
    if (k_out) SOL_CHECK(check_strides("k_out", k_strides, 2));
    if (v_out) SOL_CHECK(check_strides("v_out", v_strides, 2));
    sol::ReadArgs a{static_cast<const uint8_t*>(store), slots, k_out, v_out, {}, {}, T, heads, d, P, dtype};
    if (k_out) a.sk = two(k_strides);
    if (v_out) a.sv = two(v_strides);
    return done(sol::launch_cache_read(a, static_cast<hipStream_t>(stream)), "read");
}

size_t sol_cache_bytes(int P, int heads, int d) {
    if (P <= 0 || heads <= 0 || P > (1 << 24) || heads > 65535 || (d != 64 && d != 128)) return SIZE_MAX;
    return (size_t)P * heads * 68 * d;
}

static int check_attn(int S, int T, int max_rows, int Hq, int Hk, int d, int max_pages) {
    if (S <= 0 || T <= 0 || max_rows <= 0 || max_pages <= 0)
        return fail(SOL_ERR_INVALID_ARG, "S, T, max_rows and max_pages must be positive (got %d, %d, %d, %d)", S, T, max_rows, max_pages);
    if (Hq <= 0 || Hk <= 0 || Hq % Hk) return fail(SOL_ERR_INVALID_ARG, "Hq must be a positive multiple of Hk (got %d, %d)", Hq, Hk);
    if (d != 64 && d != 128) return fail(SOL_ERR_UNSUPPORTED, "d must be 64 or 128 (got %d)", d);
    if (S > sol::kMaxRequests) return fail(SOL_ERR_UNSUPPORTED, "at most %d requests (got %d)", sol::kMaxRequests, S);
    if (max_pages > (1 << 24) || (long long)S * max_pages > (1LL << 30)) return fail(SOL_ERR_UNSUPPORTED, "too many table entries");
    // launches of fewer than 2^32 threads
    if (Hq > 65535 || (long long)T * Hq > (1LL << 24) || (long long)S * Hk > (1LL << 18))
        return fail(SOL_ERR_UNSUPPORTED, "too many query rows or requests (got %d tokens of %d heads, %d requests of %d)", T, Hq, S, Hk);
    return SOL_OK;
}

size_t sol_cache_workspace_bytes(int S, int T, int max_rows, int Hq, int Hk, int d, int max_pages) {
    if (check_attn(S, T, max_rows, Hq, Hk, d, max_pages)) return SIZE_MAX;
    return sol::cache_attn_workspace_bytes(S, T, max_rows, Hq, Hk, d, max_pages);
}

int sol_cache_forward(const void* q, const long long* q_strides, void* out, const long long* out_strides,
                      const void* store, const int32_t* table, const int32_t* lens, const int32_t* row_start,
                      const int32_t* positions, int S, int T, int max_rows, int Hq, int Hk, int d, int P, int max_pages,
                      int causal_granule, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!q || !out || !table || !lens || !row_start || !positions)
        return fail(SOL_ERR_INVALID_ARG, "q, out, table, lens, row_start and positions must be non-null");
    if (q == out) return fail(SOL_ERR_INVALID_ARG, "out must not alias q");
    SOL_CHECK(check_head(d, dtype));
    SOL_CHECK(check_attn(S, T, max_rows, Hq, Hk, d, max_pages));
    SOL_CHECK(check_store(store, Hk, P));
    SOL_CHECK(check_strides("q", q_strides, 2));
    SOL_CHECK(check_strides("out", out_strides, 2));
    if (causal_granule < 1) return fail(SOL_ERR_INVALID_ARG, "causal_granule must be >= 1 (got %d)", causal_granule);
    const size_t need = sol::cache_attn_workspace_bytes(S, T, max_rows, Hq, Hk, d, max_pages);
    if (workspace_bytes < need || (need && !workspace))
        return fail(SOL_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", workspace ? workspace_bytes : (size_t)0, need);
    if (reinterpret_cast<uintptr_t>(workspace) & 15) return fail(SOL_ERR_INVALID_ARG, "workspace must start on 16 bytes");
    sol::CacheAttnArgs a{q, out, two(q_strides), two(out_strides), static_cast<const uint8_t*>(store), table, lens, row_start,
                         positions, S, T, max_rows, Hq, Hk, d, P, max_pages, causal_granule, dtype, workspace};
    return done(sol::launch_cache_attn(a, static_cast<hipStream_t>(stream)), "attention over the cache");
}

}  // extern "C"
