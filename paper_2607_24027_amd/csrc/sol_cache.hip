// Serving operators around the 4-bit cache: norm and rotation of queries and keys, page tables, append and
// read-back.  The attention over the cache is in sol_cache_attn.hip.
#include "sol_cache_internal.h"

#include <algorithm>
#include <climits>

namespace sol {
namespace {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// Round to nearest even; NaN stays NaN.
__device__ __forceinline__ uint32_t f32_to_bf16(float x) {
    const uint32_t b = __float_as_uint(x);
    if ((b & 0x7fffffffu) > 0x7f800000u) return (b >> 16) | 0x40u;
    return (b + 0x7fffu + ((b >> 16) & 1u)) >> 16;
}

struct BF16 {
    static constexpr int size = 2;
};
struct F32 {
    static constexpr int size = 4;
};

// Four consecutive elements at element offset `at` of p.  VEC: p and `at` are multiples of 8 bytes (bf16) or 16 bytes (f32).
template <class E, bool VEC>
__device__ __forceinline__ f32x4 load4(const void* p, long long at) {
    f32x4 r;
    if constexpr (E::size == 2) {
        const uint16_t* x = static_cast<const uint16_t*>(p) + at;
        if constexpr (VEC) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(x);
            r[0] = __uint_as_float(w[0] << 16);
            r[1] = __uint_as_float(w[0] & 0xffff0000u);
            r[2] = __uint_as_float(w[1] << 16);
            r[3] = __uint_as_float(w[1] & 0xffff0000u);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = bf16_to_f32(x[i]);
        }
    } else {
        const float* x = static_cast<const float*>(p) + at;
        if constexpr (VEC) {
            r = *reinterpret_cast<const f32x4*>(x);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = x[i];
        }
    }
    return r;
}

template <class E, bool VEC>
__device__ __forceinline__ void store4(void* p, long long at, f32x4 r) {
    if constexpr (E::size == 2) {
        uint16_t* x = static_cast<uint16_t*>(p) + at;
        const uint32_t a = f32_to_bf16(r[0]), b = f32_to_bf16(r[1]), c = f32_to_bf16(r[2]), d = f32_to_bf16(r[3]);
        if constexpr (VEC) {
            *reinterpret_cast<u32x2*>(x) = u32x2{a | (b << 16), c | (d << 16)};
        } else {
            x[0] = (uint16_t)a, x[1] = (uint16_t)b, x[2] = (uint16_t)c, x[3] = (uint16_t)d;
        }
    } else {
        float* x = static_cast<float*>(p) + at;
        if constexpr (VEC) {
            *reinterpret_cast<f32x4*>(x) = r;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = r[i];
        }
    }
}

// ---------------------------------------------------------------------------
// Norm and rotation.  D / 8 lanes hold a head of a token, each two runs of four channels, so that both members of every
// rotated pair are in one lane: with halves lane i < rot/8 holds the runs i and i + rot/8 (of four channels), the other
// lanes consecutive runs of what is not rotated; with pairs lane i holds the runs 2i and 2i + 1.  A thread keeps its
// token's cosines and sines for the heads [h0, h0 + heads) it goes through: read for each head they would be twice the heads'
// bytes in bf16.  blockIdx.x: tokens, blockIdx.y: heads of q and k.  Bound by memory: 75,600 tokens of 80 heads 0.67 ms, 4.7 TB/s
// (a large copy: 4.9); 48 tokens of 40 heads 3.7 us, a launch.
// ---------------------------------------------------------------------------
template <class E, int D, bool VEC>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const RopeArgs a, const int heads) {
    constexpr int LPR = D / 8, ROWS = 256 / LPR;
    const int lane = threadIdx.x % LPR;
    const long long t = (long long)blockIdx.x * ROWS + threadIdx.x / LPR;
    if (t >= (long long)a.B * a.N) return;
    const int b = (int)(t / a.N), n = (int)(t % a.N);
    const int quads = a.rot / 8;   // rotated runs of four in each half
    const bool turned = lane < quads;
    int c0, c1;
    if (a.pairs) {
        c0 = 8 * lane, c1 = c0 + 4;
    } else if (turned) {
        c0 = 4 * lane, c1 = c0 + a.rot / 2;
    } else {
        c0 = 8 * lane, c1 = c0 + 4;   // quads lanes hold 8 quads channels: the others go on at 8 quads
    }
    int pos = n;
    if (a.positions) pos = a.positions[t];
    if (pos < 0 || (a.rot > 0 && pos >= a.P)) return;   // uniform over the lanes of a row
    f32x4 cs = {1.f, 1.f, 1.f, 1.f}, sn = {0.f, 0.f, 0.f, 0.f};
    if (turned) {
        const long long at = (long long)pos * (a.rot / 2) + 4 * lane;
        cs = load4<F32, VEC>(a.cos, at);
        sn = load4<F32, VEC>(a.sin, at);
    }
    auto weights = [&](const void* w, f32x4& w0, f32x4& w1) {
        w0 = w1 = f32x4{1.f, 1.f, 1.f, 1.f};
        if (!w) return;
        if (a.wdtype == 0) {
            w0 = load4<BF16, VEC>(w, c0);
            w1 = load4<BF16, VEC>(w, c1);
        } else {
            w0 = load4<F32, VEC>(w, c0);
            w1 = load4<F32, VEC>(w, c1);
        }
    };
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, a.Hq + a.Hk);
    auto part = [&](const void* x, void* y, const Strides& sx, const Strides& sy, const void* w, int lo, int hi) {
        if (lo >= hi) return;
        f32x4 w0, w1;
        weights(w, w0, w1);
        const long long xi = b * sx.b + n * sx.n, yi = b * sy.b + n * sy.n;
        f32x4 next0 = load4<E, VEC>(x, xi + lo * sx.h + c0), next1 = load4<E, VEC>(x, xi + lo * sx.h + c1);
        for (int h = lo; h < hi; ++h) {
            f32x4 x0 = next0, x1 = next1;
            if (h + 1 < hi) {
                next0 = load4<E, VEC>(x, xi + (h + 1) * sx.h + c0);
                next1 = load4<E, VEC>(x, xi + (h + 1) * sx.h + c1);
            }
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) ss += x0[i] * x0[i] + x1[i] * x1[i];
#pragma unroll
            for (int m = 1; m < LPR; m *= 2) ss += __shfl_xor(ss, m);
            const float r = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
            x0 = x0 * r * w0, x1 = x1 * r * w1;
            f32x4 y0, y1;
            if (a.pairs) {
                y0[0] = x0[0] * cs[0] - x0[1] * sn[0], y0[1] = x0[1] * cs[0] + x0[0] * sn[0];
                y0[2] = x0[2] * cs[1] - x0[3] * sn[1], y0[3] = x0[3] * cs[1] + x0[2] * sn[1];
                y1[0] = x1[0] * cs[2] - x1[1] * sn[2], y1[1] = x1[1] * cs[2] + x1[0] * sn[2];
                y1[2] = x1[2] * cs[3] - x1[3] * sn[3], y1[3] = x1[3] * cs[3] + x1[2] * sn[3];
            } else {
                y0 = x0 * cs - x1 * sn;
                y1 = x1 * cs + x0 * sn;
            }
            store4<E, VEC>(y, yi + h * sy.h + c0, y0);
            store4<E, VEC>(y, yi + h * sy.h + c1, y1);
        }
    };
    part(a.q, a.qo, a.sq, a.sqo, a.wq, min(h0, a.Hq), min(h1, a.Hq));
    part(a.k, a.ko, a.sk, a.sko, a.wk, max(h0, a.Hq) - a.Hq, h1 - a.Hq);
}

// ---------------------------------------------------------------------------
// Page tables.  Every workgroup scans the lengths (at most four requests a thread) into shared memory; then the new table
// entries and the rows are dealt to all workgroups by binary searches in the sums, and the first one writes what there is once.
// New entries lie behind the used part of a table row and in front of the ring, pages that come back behind the ring's
// last: no workgroup reads what another writes.  Bound by latency: 48 requests that get a token each 4.1 us, 1,024 requests with
// 127,000 new rows and 6,900 pages given back 13.5 us, of which the pages given back, by one workgroup, take 6.
// ---------------------------------------------------------------------------
constexpr int kTablesThreads = 1024, kTablesRows = 2048;

// First index with sum[i] > x, of n ascending sums.
__device__ __forceinline__ int upper_bound(const int* sum, int n, int x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sum[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

__global__ __launch_bounds__(kTablesThreads) void cache_tables_kernel(const TablesArgs a) {
    __shared__ int s_rows_need[2 * kMaxRequests], s_gone[kMaxRequests];               // inclusive sums
    int *const s_rows = s_rows_need, *const s_need = s_rows_need + kMaxRequests;
    __shared__ int s_len[kMaxRequests];                                                // held length; ~length: refused
    __shared__ long long w_rows[16];
    __shared__ int w_need[16], w_gone[16], s_taken;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int S = a.S, MP = a.max_pages, P = a.P;
    const long long room = (long long)MP * kPage;
    const int head = ((a.state[0] % P) + P) % P, count = min(max(a.state[1], 0), P);
    if (tid == 0) s_taken = 0;
    // thread tid owns requests [e0, e1)
    const int per = (S + kTablesThreads - 1) / kTablesThreads;
    const int e0 = min(tid * per, S), e1 = min(e0 + per, S);
    long long rows = 0;
    int need = 0, gone = 0;
    auto step = [&](int s, long long& r, int& nd, int& gn, int& len, long long& want, bool& full) {
        len = (int)min((long long)max(a.lens[s], 0), room);
        const long long add = a.add[s];
        r = max(add, 0ll);
        full = add > 0 && len + add > room;
        want = full ? len : max(len + add, 0ll);
        const int before = (len + kPage - 1) / kPage, after = (int)((want + kPage - 1) / kPage);
        nd = max(after - before, 0);
        gn = max(before - after, 0);
    };
    for (int s = e0; s < e1; ++s) {
        long long r, want;
        int nd, gn, len;
        bool full;
        step(s, r, nd, gn, len, want, full);
        rows += r, need += nd, gone += gn;
    }
    long long rows_in = rows;
    int need_in = need, gone_in = gone;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const long long x = __shfl_up(rows_in, m);
        const int y = __shfl_up(need_in, m), z = __shfl_up(gone_in, m);
        if (lane >= m) rows_in += x, need_in += y, gone_in += z;
    }
    if (lane == 63) w_rows[wave] = rows_in, w_need[wave] = need_in, w_gone[wave] = gone_in;
    __syncthreads();
    rows_in -= rows, need_in -= need, gone_in -= gone;
    for (int w = 0; w < wave; ++w) rows_in += w_rows[w], need_in += w_need[w], gone_in += w_gone[w];
    for (int s = e0; s < e1; ++s) {
        long long r, want;
        int nd, gn, len;
        bool full;
        step(s, r, nd, gn, len, want, full);
        rows_in += r, need_in += nd, gone_in += gn;
        const bool granted = !full && (nd == 0 || need_in <= count);
        const int row_end = (int)min(rows_in, (long long)INT_MAX);
        s_rows[s] = row_end;
        s_need[s] = need_in;
        s_gone[s] = gone_in;
        s_len[s] = granted ? len : ~len;
        if (granted && nd > 0) atomicMax(&s_taken, need_in);   // the largest of the granted sums, whatever the order
        if (blockIdx.x == 0) {
            a.lens_out[s] = granted ? (int)want : len;
            a.row_start[s + 1] = row_end;
        }
    }
    if (blockIdx.x == 0 && tid == 0) a.row_start[0] = 0;
    __syncthreads();
    const int taken = s_taken;
    auto held = [&](int s) { return s_len[s] < 0 ? ~s_len[s] : s_len[s]; };
    // places of the ring: head < P, and ranks up to P
    auto place = [&](int at) { return at >= P ? at - P : at; };
    auto fresh = [&](int rank) { return a.ring[place(head + rank)]; };
    for (int r = blockIdx.x * kTablesThreads + tid; r < taken; r += gridDim.x * kTablesThreads) {
        const int s = upper_bound(s_need, S, r);
        const int page = (held(s) + kPage - 1) / kPage + r - (s ? s_need[s - 1] : 0);
        a.table[(long long)s * MP + page] = fresh(r);
    }
    const int total_rows = s_rows[S - 1];
    // the first of several workgroups has no rows: it has the pages that come back
    const int part = gridDim.x > 1 ? (int)blockIdx.x - 1 : 0;
    for (int t = part * kTablesRows + tid; part >= 0 && t < min(a.rows, (part + 1) * kTablesRows); t += kTablesThreads) {
        int slot = -1, pos = -1;
        if (t < total_rows) {
            const int s = upper_bound(s_rows, S, t);
            if (s_len[s] >= 0) {
                const int len = s_len[s], used = (len + kPage - 1) / kPage;
                pos = len + t - (s ? s_rows[s - 1] : 0);
                const int p = pos / kPage;
                const int page = p < used ? a.table[(long long)s * MP + p] : fresh((s ? s_need[s - 1] : 0) + p - used);
                slot = page >= 0 && page < P ? page * kPage + pos % kPage : -1;
            }
        }
        a.slots[t] = slot;
        a.positions[t] = pos;
    }
    if (blockIdx.x) return;
    // Pages that come back, in order: the valid ones of 8,192 entries at a time, eight to a thread.  Every request marks the first of
    // its entries with its number; the largest mark up to an entry is the number of its request.
    constexpr int kGone = 2 * kMaxRequests;
    static_assert(kGone == 8 * kTablesThreads, "eight entries to a thread");
    const int total_gone = s_gone[S - 1];
    int* const mark = s_rows_need;
    int base = 0;
    for (int r0 = 0; r0 < total_gone; r0 += kGone) {
        __syncthreads();   // the sums, and the marks and counts of the round before, have been read
        for (int i = tid; i < kGone; i += kTablesThreads) mark[i] = 0;
        __syncthreads();
        for (int s = e0; s < e1; ++s) {
            const int first = s ? s_gone[s - 1] : 0, end = s_gone[s];
            if (first < end && end > r0 && first < r0 + kGone) mark[max(first - r0, 0)] = s + 1;
        }
        __syncthreads();
        const int first = r0 + 8 * tid;
        int owner[8], page[8], valid = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) owner[i] = i ? max(owner[i - 1], mark[8 * tid + i]) : mark[8 * tid];
        int before = owner[7];
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int x = __shfl_up(before, m);
            if (lane >= m) before = max(before, x);
        }
        if (lane == 63) w_gone[wave] = before;
        before = __shfl_up(before, 1);
        if (lane == 0) before = 0;
        __syncthreads();
        for (int w = 0; w < wave; ++w) before = max(before, w_gone[w]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int s = max(owner[i], before) - 1;
            page[i] = -1;
            if (first + i < total_gone) page[i] = a.table[(long long)s * MP + (held(s) + kPage - 1) / kPage - (s_gone[s] - first - i)];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) valid += page[i] >= 0 && page[i] < P;
        int upto = valid;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int x = __shfl_up(upto, m);
            if (lane >= m) upto += x;
        }
        if (lane == 63) w_need[wave] = upto;
        __syncthreads();
        int rank = base + upto - valid;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) rank += w_need[w];
            base += w_need[w];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (page[i] < 0 || page[i] >= P) continue;
            if (rank < P - count) a.ring[place(place(head + count) + rank)] = page[i];
            ++rank;
        }
    }
    if (tid == 0) {
        a.state_out[0] = place(head + taken);
        a.state_out[1] = count - taken + min(base, P - count);
    }
}

// ---------------------------------------------------------------------------
// Append and read-back: a wave takes eight tokens of a head.  Keys: lane 8j + p holds channels D/8 p ... of token j, whose codes
// lie side by side in the page.  Values: lane 8r + j holds the channel runs r, r + 8, r + 16, r + 24 of token j, so that tokens
// in a row, whose codes of a run are neighbouring bytes in the page, leave in one piece.  Bound by memory: 3,600 tokens of 40 heads
// 23 us and 25 us, 4.0 and 3.7 TB/s (31 and 32 us with a token's values on neighbouring lanes); 48 tokens of 8 heads 4.3 us each.
// ---------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ int k_scale_at(int tok, int group) {   // byte of a group's scale inside the key scales
    const int t = tok & 31, swapped = (t & 19) | ((t & 4) << 1) | ((t & 8) >> 1);
    return (((group & 1) * 32 + swapped) * (D / 64) + (group >> 1)) * 2 + (tok >> 5);
}

// N consecutive elements, N = 2 or a multiple of 4.
template <class E, bool VEC, int N>
__device__ __forceinline__ void load_run(const void* p, long long at, float (&x)[N]) {
    if constexpr (N == 2) {
        if constexpr (E::size == 2) {
            const uint16_t* q = static_cast<const uint16_t*>(p) + at;
            if constexpr (VEC) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(q);
                x[0] = __uint_as_float(w << 16), x[1] = __uint_as_float(w & 0xffff0000u);
            } else {
                x[0] = bf16_to_f32(q[0]), x[1] = bf16_to_f32(q[1]);
            }
        } else {
            const float* q = static_cast<const float*>(p) + at;
            if constexpr (VEC) {
                const f32x2 w = *reinterpret_cast<const f32x2*>(q);
                x[0] = w[0], x[1] = w[1];
            } else {
                x[0] = q[0], x[1] = q[1];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const f32x4 v = load4<E, VEC>(p, at + i);
            x[i] = v[0], x[i + 1] = v[1], x[i + 2] = v[2], x[i + 3] = v[3];
        }
    }
}

template <class E, bool VEC, int N>
__device__ __forceinline__ void store_run(void* p, long long at, const float (&x)[N]) {
    if constexpr (N == 2) {
        if constexpr (E::size == 2) {
            uint16_t* q = static_cast<uint16_t*>(p) + at;
            const uint32_t a = f32_to_bf16(x[0]), b = f32_to_bf16(x[1]);
            if constexpr (VEC) *reinterpret_cast<uint32_t*>(q) = a | (b << 16);
            else q[0] = (uint16_t)a, q[1] = (uint16_t)b;
        } else {
            float* q = static_cast<float*>(p) + at;
            if constexpr (VEC) *reinterpret_cast<f32x2*>(q) = f32x2{x[0], x[1]};
            else q[0] = x[0], q[1] = x[1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) store4<E, VEC>(p, at + i, f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]});
    }
}

// Magnitudes order as integers, NaN above infinity.
template <int N>
__device__ __forceinline__ uint32_t magnitude(const float (&x)[N]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    return top;
}

// floor(log2 m) - 2, one more past 7/4 of the power of two: adding 2^21 - 1 to the bits carries from 1.75 + 1 ulp on.
__device__ __forceinline__ int exponent_of(uint32_t top, int lo, int hi) {
    return min(max((int)((top + 0x1fffffu) >> 23) - 127 - 2, lo), hi);
}

__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Eight channels' codes in a dword (fewer: in its low bytes).
template <int N>
__device__ __forceinline__ uint32_t encode(const float* x, float scale) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
    if constexpr (N >= 4) c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
    if constexpr (N >= 8) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
    }
    return c;
}

template <int N>
__device__ __forceinline__ void decode(uint32_t c, float scale, float* x) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0);
    x[0] = a[0], x[1] = a[1];
    if constexpr (N >= 4) {
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
        x[2] = b[0], x[3] = b[1];
    }
    if constexpr (N >= 8) {
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3);
        x[4] = b[0], x[5] = b[1], x[6] = d[0], x[7] = d[1];
    }
}

// A lane's place in the tokens and in the pages: of its key part (k) and of its value part (v).
struct Places {
    int t0, h, jk, p, jv, r, slot_k, slot_v;
    bool there_k, there_v;   // the token is one of the call, and its slot one of the store
};

__device__ __forceinline__ bool places(int T, int H, int P, const int32_t* slots, Places& x) {
    const int lane = threadIdx.x & 63;
    const long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    x.t0 = (int)(item / H) * 8;
    if (x.t0 >= T) return false;
    x.h = (int)(item % H);
    x.jk = lane >> 3, x.p = lane & 7, x.jv = lane & 7, x.r = lane >> 3;
    x.slot_k = x.t0 + x.jk < T ? slots[x.t0 + x.jk] : -1;
    x.slot_v = x.t0 + x.jv < T ? slots[x.t0 + x.jv] : -1;
    x.there_k = x.slot_k >= 0 && x.slot_k / kPage < P;
    x.there_v = x.slot_v >= 0 && x.slot_v / kPage < P;
    return true;
}

template <class E, int D, bool VEC>
__global__ __launch_bounds__(256) void cache_append_kernel(const AppendArgs a) {
    using L = PageLayout<D>;
    constexpr int CK = D / 8, CV = D / 32, GROUPS = D / 32;
    Places x;
    if (!places(a.T, a.H, a.P, a.slots, x)) return;   // whole waves
    float k[CK] = {}, v[4][CV] = {};
    if (x.there_k) load_run<E, VEC>(a.k, x.h * a.sk.h + (x.t0 + x.jk) * a.sk.n + CK * x.p, k);
    if (x.there_v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) load_run<E, VEC>(a.v, x.h * a.sv.h + (x.t0 + x.jv) * a.sv.n + CV * (x.r + 8 * i), v[i]);
    }
    uint32_t top_k = magnitude(k), top_v[GROUPS];
    top_k = max(top_k, (uint32_t)__shfl_xor((int)top_k, 1));
    if constexpr (D == 64) top_k = max(top_k, (uint32_t)__shfl_xor((int)top_k, 2));
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        top_v[g] = D == 128 ? magnitude(v[g]) : max(magnitude(v[2 * g]), magnitude(v[2 * g + 1]));
#pragma unroll
        for (int m = 8; m < 64; m *= 2) top_v[g] = max(top_v[g], (uint32_t)__shfl_xor((int)top_v[g], m));
    }
    // tokens with an infinity or NaN in either part: bit j
    uint32_t all_v = 0;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) all_v = max(all_v, top_v[g]);
    uint64_t mk = __ballot(top_k >= 0x7f800000u), bad = __ballot(all_v >= 0x7f800000u) & 0xff;
    if (mk) {
#pragma unroll
        for (int j = 0; j < 8; ++j) bad |= (mk >> (8 * j) & 0xff) ? 1u << j : 0;
    }
    if (x.there_k) {
        uint8_t* page = a.store + ((long long)(x.slot_k / kPage) * a.H + x.h) * L::bytes;
        const int tok = x.slot_k % kPage, e = exponent_of(top_k, -100, 125);
        const bool nan = bad >> x.jk & 1;
        const float scale = power(e);
        if constexpr (D == 128) *reinterpret_cast<u32x2*>(page + L::k + tok * (D / 2) + 8 * x.p) = u32x2{encode<8>(k, scale), encode<8>(k + 8, scale)};
        else *reinterpret_cast<uint32_t*>(page + L::k + tok * (D / 2) + 4 * x.p) = encode<8>(k, scale);
        if (x.p % (32 / CK) == 0) page[L::ks + k_scale_at<D>(tok, x.p / (32 / CK))] = nan ? 255 : (uint8_t)(e + 127);
    }
    if (x.there_v) {
        uint8_t* page = a.store + ((long long)(x.slot_v / kPage) * a.H + x.h) * L::bytes;
        const int tok = x.slot_v % kPage;
        const bool nan = bad >> x.jv & 1;
        uint8_t* to = page + L::v + ((tok >> 3) * 32 * 8 + (tok & 7)) * (D / 64) + x.r * (D / 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t code = nan ? 0 : encode<CV>(v[i], power(exponent_of(top_v[D == 128 ? i : i >> 1], -23, 13)));
            if constexpr (D == 128) *reinterpret_cast<uint16_t*>(to + 8 * i * (D / 8)) = (uint16_t)code;
            else to[8 * i * (D / 8)] = (uint8_t)code;
        }
        // lane (r, j) writes the scale of group r
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
            if (x.r == g) page[L::vs + ((tok >> 3) * GROUPS + g) * 8 + (tok & 7)] = nan ? (uint8_t)(127 - 23) : (uint8_t)(exponent_of(top_v[g], -23, 13) + 127);
    }
}

template <class E, int D, bool VEC>
__global__ __launch_bounds__(256) void cache_read_kernel(const ReadArgs a) {
    using L = PageLayout<D>;
    constexpr int CK = D / 8, CV = D / 32, GROUPS = D / 32;
    const float not_a_number = __uint_as_float(0x7fc00000u);
    Places x;
    if (!places(a.T, a.H, a.P, a.slots, x)) return;
    if (a.k && x.t0 + x.jk < a.T) {
        float k[CK] = {};
        if (x.there_k) {
            const uint8_t* page = a.store + ((long long)(x.slot_k / kPage) * a.H + x.h) * L::bytes;
            const int tok = x.slot_k % kPage;
            const uint32_t byte = page[L::ks + k_scale_at<D>(tok, x.p / (32 / CK))];
            const float scale = __uint_as_float(byte << 23);
            if constexpr (D == 128) {
                const u32x2 c = *reinterpret_cast<const u32x2*>(page + L::k + tok * (D / 2) + 8 * x.p);
                decode<8>(c[0], scale, k);
                decode<8>(c[1], scale, k + 8);
            } else {
                decode<8>(*reinterpret_cast<const uint32_t*>(page + L::k + tok * (D / 2) + 4 * x.p), scale, k);
            }
            if (byte == 255) {
#pragma unroll
                for (int i = 0; i < CK; ++i) k[i] = not_a_number;
            }
        }
        store_run<E, VEC>(a.k, x.h * a.sk.h + (x.t0 + x.jk) * a.sk.n + CK * x.p, k);
    }
    if (a.v && x.t0 + x.jv < a.T) {
        float v[4][CV] = {};
        if (x.there_v) {
            const uint8_t* page = a.store + ((long long)(x.slot_v / kPage) * a.H + x.h) * L::bytes;
            const int tok = x.slot_v % kPage;
            const bool nan = page[L::ks + k_scale_at<D>(tok, 0)] == 255;
            const uint8_t* from = page + L::v + ((tok >> 3) * 32 * 8 + (tok & 7)) * (D / 64) + x.r * (D / 8);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t byte = page[L::vs + ((tok >> 3) * GROUPS + (D == 128 ? i : i >> 1)) * 8 + (tok & 7)];
                uint32_t c;
                if constexpr (D == 128) c = *reinterpret_cast<const uint16_t*>(from + 8 * i * (D / 8));
                else c = from[8 * i * (D / 8)];
                decode<CV>(c, __uint_as_float(byte << 23), v[i]);
                if (nan) {
#pragma unroll
                    for (int y = 0; y < CV; ++y) v[i][y] = not_a_number;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) store_run<E, VEC>(a.v, x.h * a.sv.h + (x.t0 + x.jv) * a.sv.n + CV * (x.r + 8 * i), v[i]);
    }
}

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool aligned(const Strides& s, int size) { return ((s.b | s.h | s.n) * size & 15) == 0; }

}  // namespace

hipError_t launch_qk_norm_rope(const RopeArgs& a, hipStream_t st) {
    const int size = a.dtype == 0 ? 2 : 4;
    bool vec = aligned(a.wq) && aligned(a.wk) && aligned(a.cos) && aligned(a.sin);
    if (a.Hq) vec = vec && aligned(a.q) && aligned(a.qo) && aligned(a.sq, size) && aligned(a.sqo, size);
    if (a.Hk) vec = vec && aligned(a.k) && aligned(a.ko) && aligned(a.sk, size) && aligned(a.sko, size);
    const long long tokens = (long long)a.B * a.N;
    const int rows = 2048 / a.d;   // of a workgroup
    const long long blocks = (tokens + rows - 1) / rows;
    const int all = a.Hq + a.Hk;
    const int heads = (int)std::min<long long>(std::max<long long>(blocks * all / 2048, 1), std::min(all, 16));
    const dim3 grid((unsigned)blocks, (unsigned)((all + heads - 1) / heads));
#define SOL_ROPE(E, D)                                                     \
    do {                                                                   \
        if (vec) qk_norm_rope_kernel<E, D, true><<<grid, 256, 0, st>>>(a, heads);   \
        else qk_norm_rope_kernel<E, D, false><<<grid, 256, 0, st>>>(a, heads);      \
    } while (0)
    if (a.dtype == 0) {
        if (a.d == 128) SOL_ROPE(BF16, 128);
        else SOL_ROPE(BF16, 64);
    } else {
        if (a.d == 128) SOL_ROPE(F32, 128);
        else SOL_ROPE(F32, 64);
    }
#undef SOL_ROPE
    return hipGetLastError();
}

hipError_t launch_cache_tables(const TablesArgs& a, hipStream_t st) {
    const int parts = (int)(((long long)a.rows + kTablesRows - 1) / kTablesRows), grid = parts > 1 ? parts + 1 : 1;
    cache_tables_kernel<<<grid, kTablesThreads, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t st) {
    const int size = a.dtype == 0 ? 2 : 4;
    const bool vec = aligned(a.k) && aligned(a.v) && aligned(a.sk, size) && aligned(a.sv, size);
    const unsigned grid = (unsigned)(((long long)((a.T + 7) / 8) * a.H + 3) / 4);   // a wave for eight tokens of a head
#define SOL_APPEND(E, D)                                               \
    do {                                                               \
        if (vec) cache_append_kernel<E, D, true><<<grid, 256, 0, st>>>(a);      \
        else cache_append_kernel<E, D, false><<<grid, 256, 0, st>>>(a);         \
    } while (0)
    if (a.dtype == 0) {
        if (a.d == 128) SOL_APPEND(BF16, 128);
        else SOL_APPEND(BF16, 64);
    } else {
        if (a.d == 128) SOL_APPEND(F32, 128);
        else SOL_APPEND(F32, 64);
    }
#undef SOL_APPEND
    return hipGetLastError();
}

hipError_t launch_cache_read(const ReadArgs& a, hipStream_t st) {
    const int size = a.dtype == 0 ? 2 : 4;
    const bool vec = aligned(a.k) && aligned(a.v) && (!a.k || aligned(a.sk, size)) && (!a.v || aligned(a.sv, size));
    const unsigned grid = (unsigned)(((long long)((a.T + 7) / 8) * a.H + 3) / 4);   // a wave for eight tokens of a head
#define SOL_READ(E, D)                                                 \
    do {                                                               \
        if (vec) cache_read_kernel<E, D, true><<<grid, 256, 0, st>>>(a);        \
        else cache_read_kernel<E, D, false><<<grid, 256, 0, st>>>(a);           \
    } while (0)
    if (a.dtype == 0) {
        if (a.d == 128) SOL_READ(BF16, 128);
        else SOL_READ(BF16, 64);
    } else {
        if (a.d == 128) SOL_READ(F32, 128);
        else SOL_READ(F32, 64);
    }
#undef SOL_READ
    return hipGetLastError();
}

}  // namespace sol
