// Attention over the 4-bit cache.
//
// S^T = K Q^T and O^T = V^T P^T on 32 x 32 tiles, keys respectively channels on the rows and query rows on the lanes
// (lane l: column l & 31, half h = l >> 5).  A query row is a (token, query head of the group) pair of one key/value head.
//
//   q . k   v_mfma_scale_f32_32x32x64_f8f6f4 takes the codes of the cache as they lie in memory, with their scales.  Its
//           other operand holds q as a sum of 6-bit floats (e2m3, four significant bits each, every term at a sixteenth of the
//           scale of the one before): three terms for bf16, which has eight significant bits, six for f32.  6-bit operands run at
//           twice the rate of 8-bit ones (32 against 64 cycles), and the products of two terms with narrow exponents are summed
//           without loss, which those of 8-bit floats are not.
//   p . v   values are converted to f16 (exact), probabilities to f16 too: v_mfma_f32_32x32x16_f16.
//
// Row i of a key tile is key i with bits 2 and 3 exchanged: the accumulator registers of a lane then are the eight consecutive
// keys that its half of the second product's operand wants, and P never leaves its lane.
#include "sol_cache_internal.h"

#include <algorithm>
#include <cmath>

namespace sol {
namespace {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x6 __attribute__((ext_vector_type(6)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x32 __attribute__((ext_vector_type(32)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kTile = 32;             // query rows of a wave
constexpr int kUnits = 2048;          // pieces of work that a launch aims at: 8 waves a compute unit
constexpr int kLeastPages = 2;        // least pages of a piece
constexpr float kShift = 7.0f;        // probabilities are held as 2^7 p: f16 keeps all bits down to 2^-21 of the maximum's
constexpr float kSlack = 8.0f;        // log2 by which a logit may pass the running maximum before it is raised (2^15 < 65504)
constexpr float kLowest = -3.402823466e38f;

// The piece of work of one workgroup.
struct Piece {
    int s, hk, tile, chunk, chunks;   // request, key/value head, tile of query rows, share of the keys
    int p0, p1;                       // pages
    int row0, rows, len;              // rows of the request: the first one, and how many (token, head) pairs
    long long slot0;                  // piece number of share 0 of this tile
};

struct Request {
    int row0, rows, len, pages, tiles;   // rows: (token, head) pairs of a key/value head
};

__device__ __forceinline__ Request request(const CacheAttnArgs& a, int s, int G) {
    Request r;
    const int first = min(max(a.row_start[s], 0), a.T), last = min(max(a.row_start[s + 1], first), a.T);
    r.row0 = first;
    r.rows = min(last - first, a.max_rows) * G;
    r.len = min(max(a.lens[s], 0), a.max_pages * kPage);
    r.pages = max((r.len + kPage - 1) / kPage, 1);
    r.tiles = (r.rows + kTile - 1) / kTile;
    return r;
}

// Pages of a piece: every tile of every request is cut into pieces of about the same number of pages, kUnits pieces in all
// (and one more a tile at most).  By the lanes of one wave.
__device__ __forceinline__ int pages_of_piece(const CacheAttnArgs& a, int G) {
    const int lane = threadIdx.x & 63;
    long long sum = 0;
    for (int s = lane; s < a.S; s += 64) {
        const Request r = request(a, s, G);
        sum += (long long)r.tiles * r.pages;
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m);
    return (int)max((sum * a.Hk + kUnits - 1) / kUnits, (long long)kLeastPages);
}

// Piece `id` (BY_TILE: tile `id`, its share 0) of the launch; false past the last.  Pieces go by request, head, share, tile.
template <bool BY_TILE>
__device__ __forceinline__ bool find_piece(const CacheAttnArgs& a, int G, long long id, Piece& out) {
    const int lane = threadIdx.x & 63;
    const int per = pages_of_piece(a, G);
    long long base = 0, slots = 0;   // pieces (tiles) and pieces before this round's requests
    for (int s0 = 0; s0 < a.S; s0 += 64) {
        const int s = s0 + lane;
        Request r = {};
        int chunks = 0;
        if (s < a.S) {
            r = request(a, s, G);
            chunks = (r.pages + per - 1) / per;
        }
        const long long pieces = (long long)r.tiles * chunks * a.Hk;
        const long long mine = BY_TILE ? (long long)r.tiles * a.Hk : pieces;
        long long upto = mine, slot_upto = pieces;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const long long x = __shfl_up(upto, m), y = __shfl_up(slot_upto, m);
            if (lane >= m) upto += x, slot_upto += y;
        }
        const uint64_t hit = __ballot(base + upto > id);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            const long long within = id - (base + __shfl(upto - mine, l));
            out.s = s0 + l;
            out.row0 = __shfl(r.row0, l);
            out.rows = __shfl(r.rows, l);
            out.len = __shfl(r.len, l);
            const int tiles = __shfl(r.tiles, l), pages = __shfl(r.pages, l);
            out.chunks = __shfl(chunks, l);
            const long long first = slots + __shfl(slot_upto - pieces, l);
            if (BY_TILE) {
                out.hk = (int)(within / tiles);
                out.tile = (int)(within % tiles);
                out.chunk = 0;
            } else {
                out.hk = (int)(within / ((long long)tiles * out.chunks));
                const int rest = (int)(within % ((long long)tiles * out.chunks));
                out.chunk = rest / tiles;
                out.tile = rest % tiles;
            }
            out.slot0 = first + (long long)out.hk * tiles * out.chunks + out.tile;
            // equal shares of the pages
            out.p0 = (int)((long long)pages * out.chunk / out.chunks);
            out.p1 = (int)((long long)pages * (out.chunk + 1) / out.chunks);
            return true;
        }
        base += __shfl(upto, 63);
        slots += __shfl(slot_upto, 63);
    }
    return false;
}

// Shares of one tile lie `tiles` pieces apart.
__device__ __forceinline__ int tiles_of(const Piece& p) { return (p.rows + kTile - 1) / kTile; }

// ---------------------------------------------------------------------------
// Query rows: 32 channels of a lane's row, as terms of 6-bit floats.
// ---------------------------------------------------------------------------
template <int NT>
struct Split {
    u32x6 w[NT];
    int scale[NT];
};

template <int NT>
__device__ __forceinline__ Split<NT> split_row(const float (&x)[32]) {
    Split<NT> r;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    // the largest magnitude lies in (3.75, 7.5] 2^e
    int e = (int)((top + 0xfffffu) >> 23) - 127 - 2;
    e = min(max(e, -100), 125);
    f32x16 even, odd;   // the conversion interleaves its two operands
#pragma unroll
    for (int i = 0; i < 16; ++i) even[i] = x[2 * i], odd[i] = x[2 * i + 1];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float scale = __uint_as_float((uint32_t)(e + 127 - 4 * t) << 23);
        r.w[t] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, scale);
        r.scale[t] = top >= 0x7f800000u ? 255 : e + 127 - 4 * t;   // infinities and NaN make the row NaN
        if (t + 1 < NT) {
            const f32x32 y = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(r.w[t], scale);
#pragma unroll
            for (int i = 0; i < 16; ++i) even[i] -= y[2 * i], odd[i] -= y[2 * i + 1];
        }
    }
    return r;
}

template <bool F32IN, bool VEC>
__device__ __forceinline__ void load_row(const void* q, long long at, float (&x)[32]) {
    if constexpr (F32IN) {
        const float* p = static_cast<const float*>(q) + at;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (VEC) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(p + 4 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[4 * i + j] = v[j];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) x[4 * i + j] = p[4 * i + j];
            }
        }
    } else {
        const uint16_t* p = static_cast<const uint16_t*>(q) + at;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (VEC) {
                const u32x4 v = *reinterpret_cast<const u32x4*>(p + 8 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[8 * i + 2 * j] = __uint_as_float(v[j] << 16);
                    x[8 * i + 2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[8 * i + j] = __uint_as_float((uint32_t)p[8 * i + j] << 16);
            }
        }
    }
}

template <bool F32OUT, bool VEC>
__device__ __forceinline__ void store_run(void* out, long long at, f32x4 v, int n) {   // n = 2 or 4 channels
    if constexpr (F32OUT) {
        float* p = static_cast<float*>(out) + at;
        if (VEC && n == 4) {
            *reinterpret_cast<f32x4*>(p) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) p[i] = v[i];
        }
    } else {
        uint16_t* p = static_cast<uint16_t*>(out) + at;
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = __float_as_uint(v[i]);
            b[i] = (x & 0x7fffffffu) > 0x7f800000u ? (x >> 16) | 0x40u : (x + 0x7fffu + ((x >> 16) & 1u)) >> 16;
        }
        if constexpr (VEC) {
            if (n == 4) *reinterpret_cast<u32x2*>(p) = u32x2{b[0] | (b[1] << 16), b[2] | (b[3] << 16)};
            else *reinterpret_cast<uint32_t*>(p) = b[0] | (b[1] << 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) p[i] = (uint16_t)b[i];
        }
    }
}

__device__ __forceinline__ int swap23(int i) { return (i & 19) | ((i & 4) << 1) | ((i & 8) >> 1); }

// One page's bytes, as a lane holds them.
template <int D>
struct PageRegs {
    u32x4 k[2][D / 64];      // [32-key window][64-channel chunk]: 32 channels of one key
    u32x4 v[4];              // [16-key step]: eight keys of D / 32 channels (d = 64: eight bytes)
    u32x2 vs[4];             // their eight scales
    uint32_t ks;             // scale bytes [chunk][window]
};

template <int D>
__device__ __forceinline__ void load_page(const uint8_t* page, PageRegs<D>& r) {
    using L = PageLayout<D>;
    const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5;
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
            r.k[w][c] = *reinterpret_cast<const u32x4*>(page + L::k + (32 * w + swap23(i)) * (D / 2) + (2 * c + h) * 16);
    if constexpr (D == 128) r.ks = *reinterpret_cast<const uint32_t*>(page + L::ks + lane * 4);
    else r.ks = *reinterpret_cast<const uint16_t*>(page + L::ks + lane * 2);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int oct = 2 * u + h;
        if constexpr (D == 128) {
            r.v[u] = *reinterpret_cast<const u32x4*>(page + L::v + (oct * 32 + i) * 16);
        } else {
            const u32x2 x = *reinterpret_cast<const u32x2*>(page + L::v + (oct * 32 + i) * 8);
            r.v[u] = u32x4{x[0], x[1], 0, 0};
        }
        r.vs[u] = *reinterpret_cast<const u32x2*>(page + L::vs + (oct * (D / 32) + i / (1024 / D)) * 8);
    }
}

// The eight keys' f16 values of channel tile t (channels D/32 i + t), from a lane's bytes of a 16-key step.
template <int D>
__device__ __forceinline__ void values_f16(const u32x4 v, const float (&scale)[8], f16x8 (&out)[D / 32]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {   // keys 2j, 2j + 1
#pragma unroll
        for (int b = 0; b < D / 64; ++b) {
            f16x2 x, y;
            if constexpr (D == 128) {
                x = b ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[j], scale[2 * j], 1) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[j], scale[2 * j], 0);
                y = b ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[j], scale[2 * j + 1], 3) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[j], scale[2 * j + 1], 2);
            } else {
                x = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[j >> 1], scale[2 * j], 2) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[j >> 1], scale[2 * j], 0);
                y = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[j >> 1], scale[2 * j + 1], 3) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v[j >> 1], scale[2 * j + 1], 1);
            }
            out[2 * b][2 * j] = x[0], out[2 * b][2 * j + 1] = y[0];
            out[2 * b + 1][2 * j] = x[1], out[2 * b + 1][2 * j + 1] = y[1];
        }
    }
}

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// ---------------------------------------------------------------------------
// A wave a piece: 32 query rows against pages [p0, p1).  Both sums of a row run over the page's keys in registers; the next page's
// bytes are loaded while this one's are used.
// ---------------------------------------------------------------------------
template <int D, bool F32T, bool VEC>
__global__ __launch_bounds__(64) void cache_attn_kernel(const CacheAttnArgs a, const float scale_log2) {
    using L = PageLayout<D>;
    constexpr int NT = F32T ? 6 : 3, NC = D / 64, CT = D / 32;
    const int lane = threadIdx.x & 63, j = lane & 31, h = lane >> 5;
    const int G = a.Hq / a.Hk;
    Piece pc;
    if (!find_piece<false>(a, G, blockIdx.x, pc)) return;

    // this lane's query row
    const int r = pc.tile * kTile + j;
    const bool valid = r < pc.rows;
    const int token = pc.row0 + (valid ? r / G : 0), head = pc.hk * G + (valid ? r % G : 0);
    const int pos = a.positions[token];
    int sees = 0;
    if (pos >= 0) sees = (int)min(((long long)pos / a.granule + 1) * a.granule, (long long)pc.len);
    Split<NT> q[NC];
    const long long qi = head * a.sq.h + token * a.sq.n;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        float x[32];
        load_row<F32T, VEC>(a.q, qi + 64 * c + 32 * h, x);
        q[c] = split_row<NT>(x);
    }
    int most = sees, least = sees;
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
        most = max(most, __shfl_xor(most, m));
        least = min(least, __shfl_xor(least, m));
    }
    most = __builtin_amdgcn_readfirstlane(most);
    least = __builtin_amdgcn_readfirstlane(least);
    const int p0 = __builtin_amdgcn_readfirstlane(pc.p0);
    const int p1 = min(__builtin_amdgcn_readfirstlane(pc.p1), (most + kPage - 1) / kPage);
    const int* table = a.table + (long long)__builtin_amdgcn_readfirstlane(pc.s) * a.max_pages;
    const long long page_stride = (long long)a.Hk * L::bytes;
    const uint8_t* store = a.store + (long long)__builtin_amdgcn_readfirstlane(pc.hk) * L::bytes;

    f32x16 o[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = kLowest, l = 0.f;

    // the next page that is there, from p on
    auto next = [&](int& p, int& id) {
        while (p < p1) {
            id = table[p];
            if (id >= 0 && id < a.P) return true;
            ++p;
        }
        return false;
    };
    int p = p0, id = 0;
    PageRegs<D> cur;
    bool more = next(p, id);
    if (more) load_page<D>(store + id * page_stride, cur);
    while (more) {
        const int key0 = p * kPage;
        ++p;
        more = next(p, id);
        PageRegs<D> nxt = cur;
        if (more) load_page<D>(store + id * page_stride, nxt);

        f32x16 s[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[w][i] = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                i32x8 ka = {};
#pragma unroll
                for (int i = 0; i < 4; ++i) ka[i] = (int)cur.k[w][c][i];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    i32x8 qb = {};
#pragma unroll
                    for (int i = 0; i < 6; ++i) qb[i] = (int)q[c].w[t][i];
                    switch (2 * c + w) {   // the byte of the key scales is an immediate
                    case 0: s[w] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qb, s[w], 4, 2, 0, (int)cur.ks, 0, q[c].scale[t]); break;
                    case 1: s[w] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qb, s[w], 4, 2, 1, (int)cur.ks, 0, q[c].scale[t]); break;
                    case 2: s[w] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qb, s[w], 4, 2, 2, (int)cur.ks, 0, q[c].scale[t]); break;
                    default: s[w] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qb, s[w], 4, 2, 3, (int)cur.ks, 0, q[c].scale[t]); break;
                    }
                }
            }
        }
        // register 8u + 4b + e of window w is key 32w + 16u + 8h + 4b + e
        const bool edge = key0 + kPage > least;
        if (edge) {
            const int left = sees - key0 - 8 * h;
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * w + 16 * (i >> 3) + (i & 7) >= left) s[w][i] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[w][i]);
        top = fmaxf(top, other_half(top)) * scale_log2;
        if (__any(top > m + kSlack)) {
            const float up = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - up);
            m = up;
            l *= alpha;
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] *= alpha;
        }
        const float off = kShift - m;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            f16x8 ph, pl;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float e[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) e[x] = __builtin_amdgcn_exp2f(fmaf(s[u >> 1][8 * (u & 1) + 2 * i + x], scale_log2, off));
                const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(e[0], e[1]));
                ph[2 * i] = hi[0], ph[2 * i + 1] = hi[1];
                l = __builtin_amdgcn_fdot2(hi, f16x2{1, 1}, l, false);
                if constexpr (F32T) {
                    const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(e[0] - (float)hi[0], e[1] - (float)hi[1]));
                    pl[2 * i] = lo[0], pl[2 * i + 1] = lo[1];
                    l = __builtin_amdgcn_fdot2(lo, f16x2{1, 1}, l, false);
                }
            }
            float vs[8];
#pragma unroll
            for (int i = 0; i < 2; ++i) {   // the conversion reads the exponent only
                vs[4 * i + 0] = __uint_as_float(cur.vs[u][i] << 23);
                vs[4 * i + 1] = __uint_as_float(cur.vs[u][i] << 15);
                vs[4 * i + 2] = __uint_as_float(cur.vs[u][i] << 7);
                vs[4 * i + 3] = __uint_as_float(cur.vs[u][i] >> 1);
            }
            if (key0 + kPage > most) {   // what lies behind the last token may be anything: a finite scale keeps 0 v = 0
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (key0 + 16 * u + 8 * h + i >= most) vs[i] = 1.0f;
            }
            f16x8 va[CT];
            values_f16<D>(cur.v[u], vs, va);
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(va[t], ph, o[t], 0, 0, 0);
                if constexpr (F32T) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(va[t], pl, o[t], 0, 0, 0);
            }
        }
        cur = nxt;
    }
    l += other_half(l);
    if (!valid) return;
    // register i of channel tile t is channel CT (8 (i >> 2) + 4h + (i & 3)) + t
    if (pc.chunks == 1) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        const long long oi = head * a.so.h + token * a.so.n;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < CT; ++t) v[t] = o[t][i] * inv;
            store_run<F32T, VEC>(a.out, oi + CT * (8 * (i >> 2) + 4 * h + (i & 3)), v, CT);
        }
        return;
    }
    const long long slot = pc.slot0 + (long long)pc.chunk * tiles_of(pc);   // blockIdx.x
    float* part = static_cast<float*>(a.ws) + slot * (kTile * (D + 2));
    if (h == 0) part[2 * j] = m, part[2 * j + 1] = l;
    float* po = part + 2 * kTile + j * D;
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int t = 0; t < CT; ++t) po[CT * (8 * (i >> 2) + 4 * h + (i & 3)) + t] = o[t][i];
}

// ---------------------------------------------------------------------------
// Joins the shares of a tile, in their order: a workgroup a tile, a wave a row at a time, D / 64 channels a lane.
// ---------------------------------------------------------------------------
template <int D, bool F32T>
__global__ __launch_bounds__(256) void cache_join_kernel(const CacheAttnArgs a, const long long pieces) {
    constexpr int CL = D / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int G = a.Hq / a.Hk;
    Piece pc;
    if (!find_piece<true>(a, G, blockIdx.x, pc) || pc.chunks == 1) return;
    const int tiles = tiles_of(pc);
    if (pc.slot0 + (long long)(pc.chunks - 1) * tiles >= pieces) return;   // rows that overlap: no room was asked for
    const float* part = static_cast<const float*>(a.ws) + pc.slot0 * (kTile * (D + 2));
    const long long stride = (long long)tiles * (kTile * (D + 2));
    for (int j = wave; j < kTile; j += 4) {
        const int r = pc.tile * kTile + j;
        if (r >= pc.rows) break;
        float top = kLowest;
        for (int c = lane; c < pc.chunks; c += 64) top = fmaxf(top, part[c * stride + 2 * j]);
#pragma unroll
        for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
        float l = 0.f, o[CL] = {};
        for (int c = 0; c < pc.chunks; ++c) {
            const float* at = part + c * stride;
            const float w = __builtin_amdgcn_exp2f(at[2 * j] - top);
            l += w * at[2 * j + 1];
#pragma unroll
            for (int i = 0; i < CL; ++i) o[i] += w * at[2 * kTile + j * D + CL * lane + i];
        }
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        const long long oi = (pc.hk * G + r % G) * a.so.h + (pc.row0 + r / G) * a.so.n + CL * lane;
#pragma unroll
        for (int i = 0; i < CL; ++i) store_run<F32T, false>(a.out, oi + i, f32x4{o[i] * inv, 0.f, 0.f, 0.f}, 1);
    }
}

// Tiles of a launch at most, whatever the lengths: a request's last tile may be part full.
long long most_tiles(int S, int T, int max_rows, int Hq, int Hk) {
    const long long rows = std::min((long long)T, (long long)S * max_rows) * (Hq / Hk);
    return (rows / kTile + std::min(S, T)) * Hk;
}

// Pieces at most: pages_of_piece() rounds a piece's pages up, so a tile adds one to kUnits; and no tile has more than its pages give.
long long most_pieces(int S, int T, int max_rows, int Hq, int Hk, int max_pages) {
    const long long tiles = most_tiles(S, T, max_rows, Hq, Hk);
    return std::min(tiles + kUnits, tiles * ((max_pages + kLeastPages - 1) / kLeastPages));
}

}  // namespace

size_t cache_attn_workspace_bytes(int S, int T, int max_rows, int Hq, int Hk, int d, int max_pages) {
    if (max_pages <= kLeastPages) return 0;   // a piece a tile
    return (size_t)most_pieces(S, T, max_rows, Hq, Hk, max_pages) * kTile * (d + 2) * sizeof(float);
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, hipStream_t st) {
    const int size = a.dtype == 0 ? 2 : 4;
    const bool vec = ((reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.out)) & 15) == 0 &&
                     ((a.sq.h | a.sq.n | a.so.h | a.so.n) * size & 15) == 0;
    const float scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)a.d));
    const unsigned grid = (unsigned)most_pieces(a.S, a.T, a.max_rows, a.Hq, a.Hk, a.max_pages);
    const unsigned tiles = (unsigned)most_tiles(a.S, a.T, a.max_rows, a.Hq, a.Hk);
    const bool join = a.max_pages > kLeastPages;
#define SOL_ATTN(D, F)                                                                         \
    do {                                                                                       \
        if (vec) cache_attn_kernel<D, F, true><<<grid, 64, 0, st>>>(a, scale_log2);            \
        else cache_attn_kernel<D, F, false><<<grid, 64, 0, st>>>(a, scale_log2);               \
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;                       \
        if (join) cache_join_kernel<D, F><<<tiles, 256, 0, st>>>(a, grid);                           \
    } while (0)
    if (a.dtype == 0) {
        if (a.d == 128) SOL_ATTN(128, false);
        else SOL_ATTN(64, false);
    } else {
        if (a.d == 128) SOL_ATTN(128, true);
        else SOL_ATTN(64, true);
    }
#undef SOL_ATTN
    return hipGetLastError();
}

}  // namespace sol
