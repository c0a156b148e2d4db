// Attention over the 4-bit cache.
//
// S^T = K Q^T and O^T = V^T P^T, keys respectively channels on the rows of the matrix tiles and query rows on the lanes.  A query
// row is a (token, query head of the group) pair of one key/value head.
//
//   q . k   v_mfma_scale_f32_*_f8f6f4 takes the codes of the cache as they lie in memory, with their scales.  Its other operand
//           holds q log2(e) / sqrt(d) as a sum of 6-bit floats (e2m3, four significant bits each, every term at a sixteenth of
//           the scale of the one before): three terms for bf16, six for f32.  6-bit operands run at twice the rate of 8-bit
//           ones (32 against 64 cycles for 32 x 32 x 64), and sums of their products lose nothing, where those of 8-bit
//           floats, whose exponents reach further, were off by 2^-15 of the largest product.  The accumulators start at
//           7 - m, m the running maximum: what comes out is the exponent of 2^7 p, and nothing is left to do but exp2.
//   p . v   bf16 rows: values are converted to f16 (exact), probabilities to f16 too: v_mfma_f32_*_f16.  f32 rows: values and three
//           terms of each probability in bf16, all exact: v_mfma_f32_*_bf16.
//
// Two kernels.  Requests of few rows: a wave takes 16 rows and a share of the keys, bytes of the cache go from memory to
// registers (cache_few_kernel); short requests are not cut, or by the waves of a workgroup only.  Others: four waves of 32 rows share tiles in LDS, whose values are converted
// once for the 128 rows (cache_many_kernel).  cache_mixed_kernel is both, for calls with requests of both.  Both cut the work of all requests into pieces of about the same number of pages,
// whose partial results cache_join_kernel joins in the order of the keys.
#include "sol_cache_internal.h"

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstddef>
#include <type_traits>

namespace sol {
namespace {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x6 __attribute__((ext_vector_type(6)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x32 __attribute__((ext_vector_type(32)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kFewTile = 16, kManyTile = 128;   // query rows of a piece
// (token, head) rows of a request past which it goes to cache_many_kernel.  The two cross between 48 and 64 against 4,096 tokens
// (8 requests: 24, 32, 48 and 64 rows 30, 30, 35 and 41 us on the few, 33, 33, 38 and 39 on the many), f32 past 64 (48 and 64 rows 44 and
// 48 us on the few, 52 and 53 on the many).
constexpr int kFewRows = 48;
// With a table of no more pages and no more rows than that in all, every request is one of few rows: a workgroup for 16 rows fills the
// GPU sooner (one and 8 requests of 64 tokens over 1,000, 32 heads: 22 and 38 us on the many, 10 and 25 on the few; 48 of them 73 and 88).
constexpr int kShortPages = 32, kShortRows = 16 * 1024;
constexpr int kManyWhole = 8;                   // pages of a table up to which many rows are not cut
constexpr int kFewWaves = 4;                    // waves of a workgroup of cache_few_kernel
constexpr int kFewSlots = 12 * 256;             // waves of it that the GPU holds, 12 a compute unit
constexpr int kManySlots = 512;                 // workgroups of cache_many_kernel that it holds, two a compute unit (bf16 at d = 64 takes 158 registers and three run)
constexpr int kRounds = 7;                      // fillings of those slots at most (below 8: a lane for each of eight requests)
constexpr int kManyRounds = 2;                  // past 64 requests, whose lanes hold several of them
constexpr int kFewCost = 2, kManyCost = 20;     // what starting a piece and joining its result costs, in pages
constexpr int kLeastPages = 2;                  // least pages of a piece
constexpr int kRun = 16;                        // neighbouring pieces that a die gets in a row (an eighth of all: 17% slower on ragged requests)
// Tiles of few rows from which each is a wave's, if the longest request has no more pages than that: a workgroup of four waves for each of
// them is quicker for fewer (128 and 400 requests of 500 tokens, 8 heads: 20 and 66 us by workgroups, 19 and 49 by waves) and longer ones
// (400 of 2,000: 178 and 210 us).
constexpr int kManyTiles = 1024, kWavePages = 16;
constexpr float kFewJoin = 1.f / 512, kManyJoin = 1.f / 32;   // what writing and reading a piece's result takes, in pages of a piece
constexpr int kSlackPieces = 64;                // the pages of a piece are formed in f32
// "Pages of a piece" where no tile is cut: a tile is a wave's, or (few rows) a workgroup's.
constexpr int kWave = 1 << 30, kWhole = INT_MAX;
// Probabilities are held as 2^7 p: f16 keeps all bits down to 2^-21 of the maximum's, and ends at 2^-31.  Further down with a higher start
// (2^14, and 2^15.5 for kMost) the maximum is raised more often: causal prefills 6 to 8% slower (d = 64, 2,048 rows over 6,144 tokens 150 and 160 us).
constexpr float kShift = 7.0f;
constexpr float kMost = 15.0f;   // exponent past which the running maximum is raised: 2^15 < 65504
constexpr float kLowest = -3.402823466e38f;

// The piece of work of one workgroup.
struct Piece {
    int s, hk, tile, chunk, chunks;   // request, key/value head, tile of query rows, share of the keys
    int p0, p1;                       // pages
    int row0, rows, len;              // the request's first row, its (token, head) pairs of a key/value head, its length
    int tiles;
    unsigned slot0;                   // piece number of share 0 of this tile; shares lie `tiles` apart
};

struct Request {
    int row0, rows, len, pages, tiles;
};

// Requests with rows in (LO, HI] take part.
struct Part {
    int tile, slots, cost, lo, hi;
    int whole;   // few rows: pages of the longest request up to which no tile is cut
    int uncut;   // kWave or kWhole where the table has no more, otherwise 0: a plan is formed
    bool few;    // the part of cache_few_kernel
    unsigned room;   // results of pieces that the workspace holds
};

__device__ __forceinline__ Request request(const CacheAttnArgs& a, const Part& part, int s, int G) {
    Request r;
    const int first = min(max(a.row_start[s], 0), a.T), last = min(max(a.row_start[s + 1], first), a.T);
    r.row0 = first;
    r.rows = min(last - first, a.max_rows) * G;
    if (r.rows <= part.lo || r.rows > part.hi) r.rows = 0;
    r.len = min(max(a.lens[s], 0), a.max_pages * kPage);
    r.pages = max((r.len + kPage - 1) / kPage, 1);
    r.tiles = (r.rows + part.tile - 1) / part.tile;
    return r;
}

// Inclusive sum over the lanes of a wave.
template <class T>
__device__ __forceinline__ T scan_add(T x) {
    static_assert(sizeof(T) == 4, "");
#define SOL_STEP(ctrl, rows)                                                                                           \
    x += __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, rows, 0xf, false))
    SOL_STEP(0x111, 0xf);   // one to eight lanes to the right inside rows of 16
    SOL_STEP(0x112, 0xf);
    SOL_STEP(0x114, 0xf);
    SOL_STEP(0x118, 0xf);
    SOL_STEP(0x142, 0xa);   // the last lane of rows 0 and 2 to rows 1 and 3
    SOL_STEP(0x143, 0xc);   // lane 31 to rows 2 and 3
#undef SOL_STEP
    return x;
}

template <class T>
__device__ __forceinline__ T at_lane(T x, int lane) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

// Largest value of a wave's lanes, none below 0.
__device__ __forceinline__ float wave_max(float x) {
#define SOL_STEP(ctrl, rows)                                                                                              \
    x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, rows, 0xf, false)))
    SOL_STEP(0x111, 0xf);
    SOL_STEP(0x112, 0xf);
    SOL_STEP(0x114, 0xf);
    SOL_STEP(0x118, 0xf);
    SOL_STEP(0x142, 0xa);
    SOL_STEP(0x143, 0xc);
#undef SOL_STEP
    return at_lane(x, 63);
}

// Fillings of the slots at most that a plan is made for, of tiles that take up less than half of them or more.  The workspace has room
// for no more.
__host__ __device__ constexpr int most_rounds(int S, bool half) { return S > 64 ? kManyRounds : half ? kRounds : 1; }

// Pages of a piece, at most, by which `tiles` tiles of `pages` pages in all become no more pieces than fill the slots k times.
__device__ __forceinline__ int pages_for(float pages, float tiles, int slots, int k) {
    const float room = (float)slots * (float)k - tiles;   // each tile rounds up by one piece at most
    return room < 1.f ? kWave : (int)fmaxf(ceilf(pages / room), (float)kLeastPages);
}

// Pages of a piece, at most: every tile of every request is cut into equal pieces of no more.  With few tiles, the pieces fill the slots
// once; with many, it is chosen among fillings of one to kRounds times by the time that pieces dealt to free slots take, their
// mean share and a quarter of a piece (half a piece and 12 pages a start: 2,048 rows over 6,144 tokens 300 us, 266 with these; 32
// ragged requests 245, 260).  Past 64 requests (more loads for each lane) it is kManyRounds fillings, or no cut at all.  By the
// lanes of one wave, on values that all waves of a launch see alike.  `planned`: the choice as another launch made it (not read
// where it is quicker formed again than fetched from memory that another die wrote).  r: the lane's request, of up to 64.
__device__ __forceinline__ int plan_pages(const CacheAttnArgs& a, const Part& part, const int* planned, Request& r) {
#pragma clang fp contract(off)   // two kernels form the plan: the same roundings in both
    const int lane = threadIdx.x & 63, G = a.Hq / a.Hk;
    float sum = 0.f, tiles = 0.f, longest = 0.f;
    r = Request{};
    if (part.uncut) {
        if (lane < a.S) r = request(a, part, lane, G);   // past 64 they are read later
        return part.uncut;
    }
    if (planned && a.S > 64) return *planned;
    auto count = [&](int s) {
        r = request(a, part, s, G);
        if (r.tiles) longest = fmaxf(longest, (float)r.pages);
        sum += (float)r.tiles * (float)r.pages;
        tiles += (float)r.tiles;
    };
    if (lane < a.S) count(lane);
#pragma unroll 4
    for (int s = lane + 64; s < a.S; s += 64) count(s);
    sum = at_lane(scan_add(sum), 63) * (float)a.Hk;
    tiles = at_lane(scan_add(tiles), 63) * (float)a.Hk;
    longest = wave_max(longest);
    // Few rows are not cut either where the longest request is at most twice what a workgroup has to read on average (300 requests of
    // one token over 2,000, 8 heads: 168 us in pieces, 148 without; 31 over 8,000, at three times: 101 and 111).
    // Many rows: not cut for requests of up to a page for four tiles (8 and 48 requests of 16 tokens over 1,000, 8 heads: 27 and 56 us
    // in pieces, 25 and 39 without; 48 over 3,000: 96 and 89).
    if (!part.few && longest <= fminf(0.25f * tiles, 64.f)) return kWave;
    if (part.few && tiles >= kManyTiles && longest <= kWavePages) return kWave;
    if (part.few && longest <= fmaxf((float)part.whole, sum * (2.0f * kFewWaves / kFewSlots))) return kWhole;
    int per = pages_for(sum, tiles, part.slots, most_rounds(a.S, false));
    // Pieces of n pages make a join of pages / n shares, which it goes through in rounds of 16 of a row: the sum of n and the rounds
    // is least at the root (24 rows against 32,768 tokens of 8 heads: the call 34 us without this, 31 with it).  So is the sum of n and
    // the results of all pages / n pieces, 66 kB each of 128 rows (64 and 128 rows of 32 heads over 2,500 tokens: 31 and 35 us
    // without, 25 and 30 with it; f32, 48 requests of one row of 16 heads over 3,000: 35 and 28).
    per = max(per, (int)ceilf(sqrtf(fmaxf(longest * (1.0f / 16), sum * (part.few ? kFewJoin : kManyJoin)))));
    if (a.S <= 64 && tiles > 0.5f * (float)part.slots) {
        if (planned) return *planned;
        const float heads = (float)a.Hk;
        auto cost_of = [&](float pieces, float longest) {
            return (sum + pieces * (float)part.cost) / (float)part.slots + 0.25f * (longest + (float)part.cost);
        };
        float least = INFINITY;
        if (a.S <= 8) {   // lane 8 (k - 1) + s: all k at once (1.5 us less than one after the other)
            const float t = (float)__shfl(r.tiles, lane & 7), pages = (float)__shfl(r.pages, lane & 7);
            const int p = pages_for(sum, tiles, part.slots, (lane >> 3) + 1);
            const float chunks = fmaxf(ceilf(pages / (float)p), 1.f);
            float pieces = t * chunks * heads, longest = t > 0.f ? pages / chunks : 0.f;
#pragma unroll
            for (int m = 1; m < 8; m *= 2) {
                pieces += __shfl_xor(pieces, m);
                longest = fmaxf(longest, __shfl_xor(longest, m));
            }
            const float cost = cost_of(pieces, longest);
#pragma unroll
            for (int k = 0; k < kRounds; ++k) {
                const float c = at_lane(cost, 8 * k);
                if (c < least) least = c, per = at_lane(p, 8 * k);
            }
        } else {
            for (int k = 1; k <= kRounds; ++k) {
                const int p = pages_for(sum, tiles, part.slots, k);
                const float pages = (float)r.pages, chunks = fmaxf(ceilf(pages / (float)p), 1.f);
                const float pieces = at_lane(scan_add((float)r.tiles * chunks * heads), 63), longest = wave_max(r.tiles ? pages / chunks : 0.f);
                const float cost = cost_of(pieces, longest);
                if (cost < least) least = cost, per = p;
            }
        }
    }
    return per;
}

// Piece `id` (BY_TILE: share 0 of tile `id`) of a launch whose pieces have up to `per` pages; false past the last.  Pieces go by
// request, head, share, tile.  By the lanes of one wave; r as plan_pages() leaves it.
template <bool BY_TILE>
__device__ __forceinline__ bool find_piece(const CacheAttnArgs& a, const Part& part, int per, Request r, unsigned id, bool spread, Piece& out) {
    const int lane = threadIdx.x & 63, G = a.Hq / a.Hk;
    if (spread) {
        // Neighbouring workgroups run on different dies.  Each die gets runs of neighbouring pieces, which share keys in its
        // cache; short ones in turn, so that the requests' lengths even out.
        unsigned total = 0;
        for (int s = lane; s < a.S; s += 64) {
            if (a.S > 64) r = request(a, part, s, G);
            total += (unsigned)(r.tiles * (r.pages / per + (r.pages % per != 0))) * a.Hk;
        }
        total = at_lane(scan_add(total), 63);
        const unsigned run = min((total + 7) / 8, (unsigned)kRun), turn = id / 8;
        if (total == 0) return false;
        id = (turn / run * 8 + id % 8) * run + turn % run;
        if (id >= total) return false;
    }
    unsigned base = 0, slots = 0;   // pieces (tiles) and pieces before this round's requests
    for (int s0 = 0; s0 < a.S; s0 += 64) {
        const int s = s0 + lane;
        if (a.S > 64) r = s < a.S ? request(a, part, s, G) : Request{};
        const int chunks = r.pages / per + (r.pages % per != 0);
        const unsigned pieces = (unsigned)(r.tiles * chunks) * a.Hk;
        const unsigned mine = BY_TILE ? (unsigned)r.tiles * a.Hk : pieces;
        const unsigned slot_upto = scan_add(pieces), upto = BY_TILE ? scan_add(mine) : slot_upto;
        const uint64_t hit = __ballot(base + upto > id);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            const unsigned within = id - (base + at_lane(upto - mine, l));
            out.s = s0 + l;
            out.row0 = at_lane(r.row0, l);
            out.rows = at_lane(r.rows, l);
            out.len = at_lane(r.len, l);
            out.tiles = at_lane(r.tiles, l);
            const int pages = at_lane(r.pages, l);
            out.chunks = at_lane(chunks, l);
            const unsigned each = BY_TILE ? out.tiles : out.tiles * out.chunks;
            if (each == 0) return false;
            out.hk = (int)(within / each);
            const unsigned rest = within % each;
            out.chunk = (int)(rest / (unsigned)out.tiles);
            out.tile = (int)(rest % (unsigned)out.tiles);
            out.slot0 = slots + at_lane(slot_upto - pieces, l) + (unsigned)(out.hk * out.tiles * out.chunks + out.tile);
            // equal shares of the pages
            out.p0 = (int)((long long)pages * out.chunk / out.chunks);
            out.p1 = (int)((long long)pages * (out.chunk + 1) / out.chunks);
            return out.hk < a.Hk && out.chunk < out.chunks;   // rows that overlap may wrap the sums
        }
        base += at_lane(upto, 63);
        slots += at_lane(slot_upto, 63);
    }
    return false;
}

// A part's workspace: the pages of a piece, then the pieces' results.
struct PartSpace {
    int per;
    int unused[63];
    float results[1];
};
constexpr size_t kPartHeader = offsetof(PartSpace, results);

// The piece of a workgroup, found by its first wave.  The attention kernel plans, and leaves the plan to the join.
template <bool JOIN>
__device__ __forceinline__ bool find_piece_shared(const CacheAttnArgs& a, const Part& part, PartSpace* ws, unsigned id, bool spread, Piece& out) {
    __shared__ Piece s_piece;
    __shared__ int s_found;
    if (threadIdx.x < 64) {
        Request r;
        const int per = plan_pages(a, part, JOIN ? &ws->per : nullptr, r);
        if (!JOIN && id == 0 && ws && threadIdx.x == 0) ws->per = per;
        const bool found = !(JOIN && per >= kWave) && find_piece<JOIN>(a, part, per, r, id, spread, out);
        if (threadIdx.x == 0) s_piece = out, s_found = found;
    }
    __syncthreads();
    int w[sizeof(Piece) / 4];
    __builtin_memcpy(w, &s_piece, sizeof w);
#pragma unroll
    for (int& x : w) x = __builtin_amdgcn_readfirstlane(x);
    __builtin_memcpy(&out, w, sizeof w);
    return __builtin_amdgcn_readfirstlane(s_found);
}

// ---------------------------------------------------------------------------
// Query rows: 32 channels of a lane's row, as terms of 6-bit floats.  Byte t of the scales is that of term t.
// ---------------------------------------------------------------------------
// The conversions write their results before they have read all of their operands, which the compiler does not know: it gives both the
// same registers where it can, and the last term comes out wrong (errors of 3e-3 where 1.7e-3 is the rounding).  Hence results
// marked as written early.  The compiler does not look for waits inside: what wrote the operands, and what reads the results, may
// be neighbours, and two wait states on each side are as many as any vector instruction but the matrix ones asks for.
__device__ __forceinline__ u32x6 to_6_bits(const f32x16& even, const f32x16& odd, float scale) {   // interleaves the two
    u32x6 r;
    asm("s_nop 1\n\tv_cvt_scalef32_2xpk16_fp6_f32 %0, %1, %2, %3\n\ts_nop 1" : "=&v"(r) : "v"(even), "v"(odd), "v"(scale));
    return r;
}
__device__ __forceinline__ f32x32 from_6_bits(const u32x6& x, float scale) {
    f32x32 r;
    asm("s_nop 1\n\tv_cvt_scalef32_pk32_f32_fp6 %0, %1, %2\n\ts_nop 1" : "=&v"(r) : "v"(x), "v"(scale));
    return r;
}

template <int NT>
struct Split {
    u32x6 w[NT];
    uint32_t scale[(NT + 3) / 4];
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
    f32x16 even, odd;
#pragma unroll
    for (int i = 0; i < 16; ++i) even[i] = x[2 * i], odd[i] = x[2 * i + 1];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const uint32_t byte = e + 127 - 4 * t;
        const float scale = __uint_as_float(byte << 23);
        r.w[t] = to_6_bits(even, odd, scale);
        if (t % 4 == 0) r.scale[t / 4] = 0;
        r.scale[t / 4] |= byte << (8 * (t % 4));
        if (t + 1 < NT) {
            const f32x32 y = from_6_bits(r.w[t], scale);
#pragma unroll
            for (int i = 0; i < 16; ++i) even[i] -= y[2 * i], odd[i] -= y[2 * i + 1];
        }
    }
    if (top >= 0x7f800000u) {   // infinities and NaN make the row NaN
#pragma unroll
        for (int i = 0; i < (NT + 3) / 4; ++i) r.scale[i] = ~0u;
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

// Eight values (keys) of each channel of a lane's bytes, BYTES bytes (two channels each) a key, in f16 or bf16 (F32T), both exact.
// scale[k]: exponent of key k, as a float of which the conversion reads the exponent only.
template <int BYTES, bool F32T>
__device__ __forceinline__ void values_of(const uint32_t* v, const float (&scale)[8], u32x4* out) {
#define SOL_CVT(w, s, sel)                                                                         \
    (F32T ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, sel))     \
          : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, sel)))
#pragma unroll
    for (int j = 0; j < 4; ++j) {   // keys 2j, 2j + 1
#pragma unroll
        for (int b = 0; b < BYTES; ++b) {
            uint32_t x, y;
            if constexpr (BYTES == 2) {
                x = b ? SOL_CVT(v[j], scale[2 * j], 1) : SOL_CVT(v[j], scale[2 * j], 0);
                y = b ? SOL_CVT(v[j], scale[2 * j + 1], 3) : SOL_CVT(v[j], scale[2 * j + 1], 2);
            } else {
                x = j & 1 ? SOL_CVT(v[j >> 1], scale[2 * j], 2) : SOL_CVT(v[j >> 1], scale[2 * j], 0);
                y = j & 1 ? SOL_CVT(v[j >> 1], scale[2 * j + 1], 3) : SOL_CVT(v[j >> 1], scale[2 * j + 1], 1);
            }
            out[2 * b][j] = __builtin_amdgcn_perm(y, x, 0x05040100u);
            out[2 * b + 1][j] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        }
    }
#undef SOL_CVT
}

__device__ __forceinline__ void scales_of(uint32_t b, float* scale) {
    scale[0] = __uint_as_float(b << 23);
    scale[1] = __uint_as_float(b << 15);
    scale[2] = __uint_as_float(b << 7);
    scale[3] = __uint_as_float(b >> 1);
}

// Probabilities of eight keys as operands of the second product: f16, rounded to nearest, or for f32 rows three bf16 terms that hold
// all bits of an f32 at any size.  (Two f16 terms lose those of small ones: beside a token that stands 22 nats above all others
// and whose value is 0, outputs were off by 1e-2 to 1e-1.  2,048 f32 rows over 6,144 tokens, 32 heads: 400 us with them, 470 with three.)
template <bool F32T>
struct Probs {
    u32x4 w[F32T ? 3 : 1];
};

// Keys 2i and 2i + 1 of them; their sum, in f32, is added to l.  (A sum of the rounded ones by v_dot2_f32_f16 takes half the
// instructions, but they do not run beside those of the matrix cores.)
template <bool F32T>
__device__ __forceinline__ void cut_pair(float e0, float e1, Probs<F32T>& p, int i, float& l) {
    l += e0;
    l += e1;
    if constexpr (F32T) {
#pragma unroll
        for (int t = 0; t < 3; ++t) {   // each takes the upper eight significant bits of what is left
            const uint32_t b0 = __float_as_uint(e0), b1 = __float_as_uint(e1);
            p.w[t][i] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
            e0 -= __uint_as_float(b0 & 0xffff0000u);
            e1 -= __uint_as_float(b1 & 0xffff0000u);
        }
    } else {
        p.w[0][i] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)e0, (_Float16)e1});
    }
}

// o + v p, on 16 x 16 x 32 or 32 x 32 x 16 tiles.
template <bool F32T, class O>
__device__ __forceinline__ void add_values(const u32x4& v, const Probs<F32T>& p, O& o) {
    constexpr bool SMALL = sizeof(O) == sizeof(f32x4);
    if constexpr (F32T) {
#pragma unroll
        for (int t = 2; t >= 0; --t) {
            const bf16x8 a = __builtin_bit_cast(bf16x8, v), b = __builtin_bit_cast(bf16x8, p.w[t]);
            if constexpr (SMALL) o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, o, 0, 0, 0);
            else o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, o, 0, 0, 0);
        }
    } else {
        const f16x8 a = __builtin_bit_cast(f16x8, v), b = __builtin_bit_cast(f16x8, p.w[0]);
        if constexpr (SMALL) o = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, o, 0, 0, 0);
        else o = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, o, 0, 0, 0);
    }
}

__device__ __forceinline__ int row_limit(const CacheAttnArgs& a, int token, int len) {
    const int pos = a.positions[token];
    return pos < 0 ? 0 : (int)min(((long long)pos / a.granule + 1) * a.granule, (long long)len);
}

// The pages of a piece in order, those that are not there left out.  A lane holds the table entry of one of 64 pages.
struct Pages {
    const int* table;
    int P, end, base;    // pages base ... base + 63 are in `entry`
    uint64_t there;      // those of them that are there and not yet given out
    int entry, p;        // p: the page that next() found

    __device__ __forceinline__ void fill() {
        const int at = base + (int)(threadIdx.x & 63);
        entry = at < end ? table[at] : -1;
        there = __ballot(entry >= 0 && entry < P);
    }
    __device__ __forceinline__ Pages(const int* t, int P_, int p0, int p1) : table(t), P(P_), end(p1), base(p0), there(0), entry(-1), p(p0) { fill(); }
    // Leaves out pages from `to` on; whether the one that next() found stays.
    __device__ __forceinline__ bool limit(int to) {
        end = min(end, to);
        const int n = end - base;
        if (n < 64) there &= n > 0 ? (1ull << n) - 1 : 0;
        return p < end;
    }
    // The next page's place in the store, or -1.
    __device__ __forceinline__ int next() {
        while (!there) {
            base += 64;
            if (base >= end) return -1;
            fill();
        }
        const int l = __builtin_ctzll(there);
        there &= there - 1;
        p = base + l;
        return __builtin_amdgcn_readlane(entry, l);
    }
};

// Raises the running maximum of a lane's row (exponents s, sums l and o) to `top`, the row's largest exponent, where that is past
// `most`: -infinity before the row has seen a key, kMost afterwards.  For a wave in which one row's is; returns the change.
__device__ __forceinline__ float raise(float top, float& m, float& most, float& alpha) {
    const bool fresh = most < 0.f;
    float by = fresh ? top - kShift : fmaxf(top - kShift, 0.f);
    if (top == -INFINITY) by = 0.f;
    else most = kMost;
    alpha = fresh ? 0.f : __builtin_amdgcn_exp2f(-by);
    m += by;
    return by;
}

// ---------------------------------------------------------------------------
// Few rows: a wave a piece, 16 query rows (lane l: row l & 15) against pages [p0, p1).  Bound by the bytes of the cache.  Lane
// group g = l >> 4 holds channels 32g ... of the keys (16 x 16 x 128: one scale a lane; at d = 64 the upper groups hold
// zeros).  Row 4g + e of key tile b of a 32-key window is key 8g + 4b + e: registers e of the tiles 0 and 1 are then the
// eight consecutive keys that group g holds of the second product's operand.  Registers are filled again as soon as they
// are used: the keys of the next page are on their way during the second product, its values during the next first one.  32-row
// tiles need 256 registers and more (one wave a SIMD: 102 us against 66 at 48 requests of 200 to 32,000 tokens, 8 heads of 128
// channels, 340 MB: 5.1 TB/s, a large copy reaches 4.9); this takes 165, three waves a SIMD.
// ---------------------------------------------------------------------------
template <int D>
struct FewPage {
    u32x4 k[4];            // [2 w + b]
    u32x4 v[2][D / 64];    // [w]: eight keys of D / 16 channels
    u32x2 vs[2];
    uint32_t ks;           // byte 2 b + w
};

// A lane's byte offsets inside a page: the page itself is a scalar address.
struct FewOffsets {
    uint32_t k, ks, v, vs;
};

template <int D>
__device__ __forceinline__ FewOffsets few_offsets() {
    using L = PageLayout<D>;
    const unsigned lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    FewOffsets o;
    o.k = L::k + (8 * (i >> 2) + (i & 3)) * (D / 2) + 16 * g;
    // scale of (key, group g) at [g & 1][key with bits 2 and 3 exchanged][g >> 1][w]
    o.ks = L::ks + ((g & 1) * 32 + 16 * (i >> 3) + 4 * ((i >> 2) & 1) + (i & 3)) * (D / 32) + (g >> 1) * 2;
    o.v = L::v + (g * 32 + 2 * i) * (D / 8);
    o.vs = L::vs + (g * (D / 32) + i / (512 / D)) * 8;
    return o;
}

template <int D>
__device__ __forceinline__ void few_load_k(const uint8_t* page, const FewOffsets& at, FewPage<D>& r) {
    if (D == 64 && (threadIdx.x & 32)) {
#pragma unroll
        for (int t = 0; t < 4; ++t) r.k[t] = u32x4{0, 0, 0, 0};
        r.ks = 0x7f7f7f7fu;
        return;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
        r.k[t] = *reinterpret_cast<const u32x4*>(page + (32 * (t >> 1) + 4 * (t & 1)) * (D / 2) + at.k);
    r.ks = *reinterpret_cast<const uint16_t*>(page + at.ks) | ((uint32_t)*reinterpret_cast<const uint16_t*>(page + 8 * (D / 32) + at.ks) << 16);
}

template <int D>
__device__ __forceinline__ void few_load_v(const uint8_t* page, const FewOffsets& at, FewPage<D>& r) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
#pragma unroll
        for (int c = 0; c < D / 64; ++c)   // 32 bytes (d = 64: 16) of two channel runs
            r.v[w][c] = *reinterpret_cast<const u32x4*>(page + w * 128 * (D / 8) + 16 * c + at.v);
        r.vs[w] = *reinterpret_cast<const u32x2*>(page + w * (D / 8) * 8 + at.vs);
    }
}

template <int D, bool F32T, bool EDGE>
__device__ __forceinline__ void few_first(const FewPage<D>& pg, const Split<F32T ? 6 : 3>& q, int key0, int sees, float off, f32x4 (&s)[4]) {
    constexpr int NT = F32T ? 6 : 3;
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = f32x4{off, off, off, off};
#define SOL_MFMA(t, ks_byte, n, q_byte)                                                                                   \
    s[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(i32x8{(int)pg.k[t][0], (int)pg.k[t][1], (int)pg.k[t][2], (int)pg.k[t][3], 0, 0, 0, 0},   \
                                                            i32x8{(int)q.w[n][0], (int)q.w[n][1], (int)q.w[n][2], (int)q.w[n][3], (int)q.w[n][4], (int)q.w[n][5], 0, 0}, \
                                                            s[t], 4, 2, ks_byte, (int)pg.ks, q_byte, (int)q.scale[(n) / 4])
#define SOL_TERM(n, q_byte) SOL_MFMA(0, 0, n, q_byte), SOL_MFMA(1, 2, n, q_byte), SOL_MFMA(2, 1, n, q_byte), SOL_MFMA(3, 3, n, q_byte)
    SOL_TERM(0, 0);
    SOL_TERM(1, 1);
    SOL_TERM(2, 2);
    if constexpr (NT == 6) {
        SOL_TERM(3, 3);
        SOL_TERM(4, 0);
        SOL_TERM(5, 1);
    }
#undef SOL_TERM
#undef SOL_MFMA
    if constexpr (EDGE) {
        const int left = sees - key0 - 8 * g;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (32 * (t >> 1) + 4 * (t & 1) + e >= left) s[t][e] = -INFINITY;
    }
}

template <int D, bool F32T, bool EDGE>
__device__ __forceinline__ void few_second(const FewPage<D>& pg, f32x4 (&s)[4], int key0, int last, float& m, float& most, float& l,
                                           f32x4 (&o)[D / 16]) {
    const int g = (threadIdx.x & 63) >> 4;
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = __builtin_elementwise_maximum(top, s[t][e]);
    if (__any(top > most)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        float alpha;
        const float by = raise(top, m, most, alpha);
        l *= alpha;
#pragma unroll
        for (int t = 0; t < 4; ++t) s[t] -= by;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) o[t] *= alpha;
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        Probs<F32T> p = {};
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                cut_pair<F32T>(__builtin_amdgcn_exp2f(s[2 * w + b][2 * e]), __builtin_amdgcn_exp2f(s[2 * w + b][2 * e + 1]), p, 2 * b + e, l);
        float vs[8];
        scales_of(pg.vs[w][0], vs);
        scales_of(pg.vs[w][1], vs + 4);
        if constexpr (EDGE) {   // what lies behind the last token may be anything: a finite scale keeps 0 v = 0
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (key0 + 32 * w + 8 * g + i >= last) vs[i] = 1.0f;
        }
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            // 16 bytes: eight keys of two bytes (d = 128), or two runs of eight bytes (d = 64)
            const uint32_t bytes[4] = {pg.v[w][c][0], pg.v[w][c][1], pg.v[w][c][2], pg.v[w][c][3]};
            u32x4 va[4];
            if constexpr (D == 128) {
                values_of<2, F32T>(bytes, vs, va);
            } else {
                values_of<1, F32T>(bytes, vs, va);
                values_of<1, F32T>(bytes + 2, vs, va + 2);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) add_values(va[t], p, o[4 * c + t]);
        }
    }
}

// Row j of a wave's 16 against the piece's pages: running maximum (kLowest: it has seen no key), sum and sums of values of lane group 0 ... 3.
template <int D, bool F32T, bool VEC>
__device__ __forceinline__ void few_rows(const CacheAttnArgs& a, const Piece& pc, float scale_log2, float& m, float& l, f32x4 (&o)[D / 16]) {
    using L = PageLayout<D>;
    constexpr int NT = F32T ? 6 : 3, CT = D / 16;
    const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const int G = a.Hq / a.Hk;

    // memory is asked for the first page, the rows' positions and the rows at once
    const long long page_stride = (long long)a.Hk * L::bytes;
    const uint8_t* store = a.store + (long long)pc.hk * L::bytes;
    Pages pages(a.table + (long long)pc.s * a.max_pages, a.P, pc.p0, pc.p1);
    FewPage<D> pg;
    const FewOffsets at = few_offsets<D>();
    int id = pages.next();
    const uint8_t* page = store + id * page_stride;
    if (id >= 0) {
        few_load_k<D>(page, at, pg);
        few_load_v<D>(page, at, pg);
    }
    const int r = pc.tile * kFewTile + j;
    const bool valid = r < pc.rows;
    const int token = pc.row0 + (valid ? r / G : 0), head = pc.hk * G + (valid ? r % G : 0);
    float x[32];
    if (D == 128 || g < 2) {
        load_row<F32T, VEC>(a.q, head * a.sq.h + token * a.sq.n + 32 * g, x);
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = 0.f;
    }
    const int sees = row_limit(a, token, pc.len);
    int last = sees, least = sees;
#pragma unroll
    for (int m = 1; m < 16; m *= 2) {
        last = max(last, __shfl_xor(last, m));
        least = min(least, __shfl_xor(least, m));
    }
    last = __builtin_amdgcn_readfirstlane(last);
    least = __builtin_amdgcn_readfirstlane(least);
    if (!pages.limit((last + kPage - 1) / kPage)) id = -1;

    f32x4 s[4];
#pragma unroll
    for (int t = 0; t < CT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float most = -INFINITY;
    m = l = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] *= scale_log2;
    const Split<NT> q = split_row<NT>(x);
    auto step = [&](auto edge) __attribute__((always_inline)) {
        constexpr bool EDGE = decltype(edge)::value;
        const int key0 = pages.p * kPage;
        id = pages.next();
        few_first<D, F32T, EDGE>(pg, q, key0, sees, kShift - m, s);
        if (id >= 0) {
            page = store + id * page_stride;
            few_load_k<D>(page, at, pg);
        }
        few_second<D, F32T, EDGE>(pg, s, key0, last, m, most, l, o);
        if (id >= 0) few_load_v<D>(page, at, pg);
    };
    while (id >= 0 && pages.p * kPage + kPage <= least) step(std::false_type{});
    while (id >= 0) step(std::true_type{});
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (most < 0.f) m = kLowest;
}

// What the waves of a workgroup have found for one tile.
template <int D>
struct alignas(16) FewResults {
    float o[kFewWaves][kFewTile][D + 4], ml[kFewWaves][kFewTile][2];
};

// A workgroup's part of the work: its waves share the pages of a tile where no tile is cut, and join their results in LDS; otherwise
// each has a piece of its own.
template <int D, bool F32T, bool VEC>
__device__ __forceinline__ void few_block(const CacheAttnArgs& a, const Part& part, float scale_log2, PartSpace* ws, unsigned block, unsigned pieces,
                                          FewResults<D>& all) {
    constexpr int CT = D / 16, LANES = D / 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 15, g = lane >> 4;
    const int G = a.Hq / a.Hk;
    Piece pc;
    Request request_of_lane;
    const int per = plan_pages(a, part, nullptr, request_of_lane);
    if (block == 0 && ws && threadIdx.x == 0) ws->per = per;
    const bool whole = per == kWhole;
    const unsigned piece = whole ? block : kFewWaves * block + wave;
    if (piece >= pieces || !find_piece<false>(a, part, per, request_of_lane, piece, false, pc)) return;
    if (whole) {
        const unsigned pages = pc.p1;
        pc.p0 = (int)(pages * wave / kFewWaves), pc.p1 = (int)(pages * (wave + 1) / kFewWaves);
    }
    f32x4 o[CT];
    float m, l;
    few_rows<D, F32T, VEC>(a, pc, scale_log2, m, l, o);
    // register e of channel tile t is channel CT (4g + e) + t
    const int r0 = pc.tile * kFewTile, rows = min(kFewTile, pc.rows - r0);
    auto place = [&](int row) { return (pc.hk * G + (r0 + row) % G) * a.so.h + (pc.row0 + (r0 + row) / G) * a.so.n; };
    if (whole) {
        if (g == 0) all.ml[wave][j][0] = m, all.ml[wave][j][1] = l;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int t = 0; t < CT; t += 4)
                *reinterpret_cast<f32x4*>(&all.o[wave][j][CT * (4 * g + e) + t]) = f32x4{o[t][e], o[t + 1][e], o[t + 2][e], o[t + 3][e]};
        __syncthreads();
        const int at = 4 * (threadIdx.x % LANES);
        for (int row = threadIdx.x / LANES; row < rows; row += 64 * kFewWaves / LANES) {
            float top = kLowest;
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, all.ml[w][row][0]);
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            l = 0.f;
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                const float x = __builtin_amdgcn_exp2f(all.ml[w][row][0] - top);
                l += x * all.ml[w][row][1];
                sum += x * *reinterpret_cast<const f32x4*>(&all.o[w][row][at]);
            }
            const float inv = l == 0.f ? 0.f : 1.0f / l;
            store_run<F32T, VEC>(a.out, place(row) + at, sum * inv, 4);
        }
    } else if (j < rows && pc.chunks == 1) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        const long long oi = place(j);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int t = 0; t < CT; t += 4)
                store_run<F32T, VEC>(a.out, oi + CT * (4 * g + e) + t, f32x4{o[t][e], o[t + 1][e], o[t + 2][e], o[t + 3][e]} * inv, 4);
    } else if (j < rows && piece < part.room) {   // rows that overlap: no room was asked for
        float* to = ws->results + (long long)piece * (kFewTile * (D + 2));
        if (g == 0) to[2 * j] = m, to[2 * j + 1] = l;
        float* po = to + 2 * kFewTile + j * D;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int t = 0; t < CT; t += 4)
                *reinterpret_cast<f32x4*>(po + CT * (4 * g + e) + t) = f32x4{o[t][e], o[t + 1][e], o[t + 2][e], o[t + 3][e]};
    }
}

template <int D, bool F32T, bool VEC>
__global__ __launch_bounds__(64 * kFewWaves, F32T && D == 128 ? 2 : 3) void cache_few_kernel(const CacheAttnArgs a, const Part part, const float scale_log2,
                                                                                             PartSpace* ws, const unsigned pieces) {
    __shared__ FewResults<D> results;
    few_block<D, F32T, VEC>(a, part, scale_log2, ws, blockIdx.x, pieces, results);
}

// ---------------------------------------------------------------------------
// Many rows: four waves of 32 query rows (lane l: row l & 31, half h = l >> 5) on one piece.  A page lies in LDS as operands: the
// codes of the keys as they are (32 x 32 x 64: a lane's 32 channels of a key), the values as f16, converted by thread t for eight
// keys of D / 32 channels.  Two stages: while a page is used, the next one is converted from registers, and the one after is on its
// way.  Row i of a 32-key window is key i with bits 2 and 3 exchanged, so that the registers 8u ... 8u + 7 of the first
// product are the eight consecutive keys that a lane holds of the second one's operand.
//
// Bound by what the matrix cores may draw: 3,600 rows of 40 heads over 75,600 tokens take 4.75 to 5.1 ms by the card, 1,090 to
// 1,170 TFLOP/s at 1.9 GHz, where a large bf16 matrix product reaches 1,160.  The bare instructions of a page, on random data from
// registers, take 0.77 us a wave and page whether one, two or three waves share a SIMD, on constant data 0.55; here it is 0.85.
// That leaves nothing for an order of the loop: products of the next page before the sums of this one, a window at a time
// with three waves a SIMD, eight waves to a workgroup, values a step ahead of their use: all within 2% or slower.
// ---------------------------------------------------------------------------
__device__ __forceinline__ int swap23(int i) { return (i & 19) | ((i & 4) << 1) | ((i & 8) >> 1); }

template <int D>
struct Stage {
    u32x4 k[2 * (D / 64) * 64];     // [window][64-channel chunk][lane]
    u32x4 v[4 * (D / 32) * 64];     // [16-key step][channel tile][lane]
    uint32_t ks[64];                // scale bytes [chunk][window] of a lane
};

// A thread's part of a page: 16 bytes of keys (d = 64: of the first 128 threads), and of the values eight keys of a channel run.
template <int D>
struct ManyPage {
    u32x4 k, v;
    u32x2 vs;
    uint32_t ks;
};

template <int D>
__device__ __forceinline__ void many_load(const uint8_t* page, ManyPage<D>& r) {
    using L = PageLayout<D>;
    const unsigned t = threadIdx.x, lane = t & 63, i = lane & 31, h = lane >> 5;
    if (t < 2 * D) {
        const unsigned w = D == 128 ? t >> 7 : t >> 6, c = D == 128 ? (t >> 6) & 1 : 0;
        r.k = *reinterpret_cast<const u32x4*>(page + (L::k + (32 * w + swap23(i)) * (D / 2) + (2 * c + h) * 16));
    }
    if constexpr (D == 128) {
        r.v = *reinterpret_cast<const u32x4*>(page + (L::v + t * 16));
    } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(page + (L::v + t * 8));
        r.v = u32x4{x[0], x[1], 0, 0};
    }
    r.vs = *reinterpret_cast<const u32x2*>(page + (L::vs + ((t >> 5) * (D / 32) + (t & 31) / (1024 / D)) * 8));
    if (t < 64) {
        if constexpr (D == 128) r.ks = *reinterpret_cast<const uint32_t*>(page + (L::ks + t * 4));
        else r.ks = *reinterpret_cast<const uint16_t*>(page + (L::ks + t * 2));
    }
}

// left: tokens of the page that there are; what lies behind them may be anything, and a finite scale keeps 0 v = 0.
template <int D, bool F32T>
__device__ __forceinline__ void many_store(const ManyPage<D>& r, Stage<D>& st, int left) {
    constexpr int CT = D / 32;
    const int t = threadIdx.x;
    if (t < 2 * D) st.k[t] = r.k;
    if (t < 64) st.ks[t] = r.ks;
    float vs[8];
    scales_of(r.vs[0], vs);
    scales_of(r.vs[1], vs + 4);
    if (left < kPage) {
        asm volatile("" : "+s"(left));   // a branch, not instructions more for every page
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (8 * (t >> 5) + i >= left) vs[i] = 1.0f;
    }
    const uint32_t bytes[4] = {r.v[0], r.v[1], r.v[2], r.v[3]};
    u32x4 va[CT];
    values_of<D / 64, F32T>(bytes, vs, va);
#pragma unroll
    for (int c = 0; c < CT; ++c) st.v[((t >> 6) * CT + c) * 64 + (t & 63)] = va[c];   // keys 16 (t >> 6) + 8 (t >> 5 & 1) ...
}

template <int D, bool F32T>
__device__ __forceinline__ void many_page(const Stage<D>& st, const Split<F32T ? 6 : 3> (&q)[D / 64], int key0, bool edge, int sees,
                                          float& m, float& most, f32x16& off, float& l, f32x16 (&o)[D / 32]) {
    constexpr int NT = F32T ? 6 : 3, NC = D / 64, CT = D / 32;
    const int lane = threadIdx.x & 63, h = lane >> 5;
    f32x16 s[2] = {off, off};
    const int ks = (int)st.ks[lane];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const u32x4 k0 = st.k[c * 64 + lane], k1 = st.k[(NC + c) * 64 + lane];
#define SOL_MFMA(win, kk, ks_byte, n, q_byte)                                                                               \
    s[win] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(i32x8{(int)kk[0], (int)kk[1], (int)kk[2], (int)kk[3], 0, 0, 0, 0}, \
                                                           i32x8{(int)q[c].w[n][0], (int)q[c].w[n][1], (int)q[c].w[n][2], (int)q[c].w[n][3], (int)q[c].w[n][4], (int)q[c].w[n][5], 0, 0}, \
                                                           s[win], 4, 2, ks_byte, ks, q_byte, (int)q[c].scale[(n) / 4])
#define SOL_TERM(n, q_byte)                                                            \
    do {                                                                               \
        if (c == 0) SOL_MFMA(0, k0, 0, n, q_byte), SOL_MFMA(1, k1, 1, n, q_byte);      \
        else SOL_MFMA(0, k0, 2, n, q_byte), SOL_MFMA(1, k1, 3, n, q_byte);             \
    } while (0)
        SOL_TERM(0, 0);
        SOL_TERM(1, 1);
        SOL_TERM(2, 2);
        if constexpr (NT == 6) {
            SOL_TERM(3, 3);
            SOL_TERM(4, 0);
            SOL_TERM(5, 1);
        }
#undef SOL_TERM
#undef SOL_MFMA
    }
    // register 8u + 4b + e of window w is key 32w + 16u + 8h + 4b + e
    if (edge) {
        int left = sees - key0 - 8 * h;
        asm volatile("" : "+v"(left));   // a branch, not an instruction more for every logit of every page
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (32 * w + 16 * (i >> 3) + (i & 7) >= left) s[w][i] = -INFINITY;
    }
    // A row that sees a NaN is NaN whatever its maximum; fmaxf() takes another instruction for each logit, to quiet it (1% slower).
    float top = s[0][0];
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = __builtin_elementwise_maximum(top, s[w][i]);
    if (__any(top > most)) {
        top = fmaxf(top, __shfl_xor(top, 32));
        float alpha;
        const float by = raise(top, m, most, alpha);
        l *= alpha;
#pragma unroll
        for (int i = 0; i < 16; ++i) off[i] = kShift - m;
#pragma unroll
        for (int w = 0; w < 2; ++w) s[w] -= by;
#pragma unroll
        for (int t = 0; t < CT; ++t) o[t] *= alpha;
    }
    // a wave in this part goes first: its vector instructions fill the gaps of the other one's products
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        Probs<F32T> p = {};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            cut_pair<F32T>(__builtin_amdgcn_exp2f(s[u >> 1][8 * (u & 1) + 2 * i]), __builtin_amdgcn_exp2f(s[u >> 1][8 * (u & 1) + 2 * i + 1]),
                           p, i, l);
#pragma unroll
        for (int t = 0; t < CT; ++t) add_values(st.v[(u * CT + t) * 64 + lane], p, o[t]);
    }
    __builtin_amdgcn_s_setprio(0);
}

template <int D>
struct ManySpace {
    Stage<D> stage[2];
    int last[4];
};

template <int D, bool F32T, bool VEC>
__device__ __forceinline__ void many_piece(const CacheAttnArgs& a, const Part& part, float scale_log2, PartSpace* ws, unsigned piece,
                                           ManySpace<D>& lds) {
    using L = PageLayout<D>;
    constexpr int NT = F32T ? 6 : 3, NC = D / 64, CT = D / 32;
    Stage<D>* const stage = lds.stage;
    int* const s_last = lds.last;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 31, h = lane >> 5;
    const int G = a.Hq / a.Hk;
    Piece pc;
    if (!find_piece_shared<false>(a, part, ws, piece, true, pc)) return;
    const unsigned slot = pc.slot0 + (unsigned)pc.chunk * pc.tiles;

    // memory is asked for the first page, the rows' positions and the rows at once
    const long long page_stride = (long long)a.Hk * L::bytes;
    const uint8_t* store = a.store + (long long)pc.hk * L::bytes;
    Pages pages(a.table + (long long)pc.s * a.max_pages, a.P, pc.p0, pc.p1);
    ManyPage<D> pg;
    int id = pages.next();
    if (id >= 0) many_load<D>(store + id * page_stride, pg);
    const int r = pc.tile * kManyTile + 32 * wave + j;
    const bool valid = r < pc.rows;
    const int token = pc.row0 + (valid ? r / G : 0), head = pc.hk * G + (valid ? r % G : 0);
    int sees = row_limit(a, token, pc.len);
    if (!valid) sees = 0;
    Split<NT> q[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        float x[32];
        load_row<F32T, VEC>(a.q, head * a.sq.h + token * a.sq.n + 64 * c + 32 * h, x);
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] *= scale_log2;
        q[c] = split_row<NT>(x);
    }
    int last = sees, least = valid ? sees : INT_MAX;
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
        last = max(last, __shfl_xor(last, m));
        least = min(least, __shfl_xor(least, m));
    }
    last = __builtin_amdgcn_readfirstlane(last);   // 0 where the wave has no rows
    least = __builtin_amdgcn_readfirstlane(least);
    if (lane == 0) s_last[wave] = last;
    __syncthreads();
    const int all = max(max(s_last[0], s_last[1]), max(s_last[2], s_last[3]));
    bool more = pages.limit(__builtin_amdgcn_readfirstlane((all + kPage - 1) / kPage)) && id >= 0;

    f32x16 o[CT], off;
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = 0.f, most = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) off[i] = kShift;

    // the page of tokens key0 ... is in stage[turn], the one after it in registers
    int turn = 0, key0 = pages.p * kPage;
    if (more) {
        many_store<D, F32T>(pg, stage[0], pc.len - key0);
        id = pages.next();
        if (id >= 0) many_load<D>(store + id * page_stride, pg);
    }
    __syncthreads();
    while (more) {
        const int now = key0;
        more = id >= 0;
        if (more) {
            key0 = pages.p * kPage;
            many_store<D, F32T>(pg, stage[turn ^ 1], pc.len - key0);
            id = pages.next();
            if (id >= 0) many_load<D>(store + id * page_stride, pg);
        }
        if (now < last) many_page<D, F32T>(stage[turn], q, now, now + kPage > least, sees, m, most, off, l, o);
        turn ^= 1;
        __syncthreads();
    }
    l += __shfl_xor(l, 32);
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
    if (slot >= part.room) return;   // rows that overlap: no room was asked for
    float* to = ws->results + (long long)slot * (kManyTile * (D + 2));
    const int row = 32 * wave + j;
    if (h == 0) to[2 * row] = most < 0.f ? kLowest : m, to[2 * row + 1] = l;
    float* po = to + 2 * kManyTile + row * D;
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int t = 0; t < CT; ++t) po[CT * (8 * (i >> 2) + 4 * h + (i & 3)) + t] = o[t][i];
}

template <int D, bool F32T, bool VEC>
__global__ __launch_bounds__(256, 2) void cache_many_kernel(const CacheAttnArgs a, const Part part, const float scale_log2,
                                                                                                       PartSpace* ws) {
    __shared__ ManySpace<D> lds;
    many_piece<D, F32T, VEC>(a, part, scale_log2, ws, blockIdx.x, lds);
}

// Both in one launch: the many first (their pieces are the longest), then the few, which fill what the last ones leave.
template <int D, bool F32T, bool VEC>
__global__ __launch_bounds__(256, 2) void cache_mixed_kernel(const CacheAttnArgs a, const Part few, const Part many, const float scale_log2,
                                                             PartSpace* few_ws, PartSpace* many_ws, const unsigned few_pieces,
                                                             const unsigned many_pieces) {
    static_assert(64 * kFewWaves == 256, "one shape of workgroups");
    __shared__ union Space {
        __device__ Space() {}
        ManySpace<D> many;
        FewResults<D> few;
    } lds;
    if (blockIdx.x < many_pieces) many_piece<D, F32T, VEC>(a, many, scale_log2, many_ws, blockIdx.x, lds.many);
    else few_block<D, F32T, VEC>(a, few, scale_log2, few_ws, blockIdx.x - many_pieces, few_pieces, lds.few);
}

// ---------------------------------------------------------------------------
// Joins the shares of a tile's rows, of both kernels' pieces in one launch, in an order that the plan fixes.  D / 4 threads hold a row, four
// channels each; where there are fewer rows than groups, the shares are dealt to several groups, whose sums are added in LDS.  Bound
// by latency: the plan, the maxima, the sums: 5 to 7 us for single tokens; 60 us for 230 MB of a frame's shares.
// ---------------------------------------------------------------------------
constexpr int kJoinThreads = 512;

struct JoinPart {
    Part part;
    PartSpace* ws;
    unsigned tiles, per_tile;   // per_tile workgroups a tile, for `rows` rows each
    int rows;
};

template <int D, bool F32T, bool VEC>
__global__ __launch_bounds__(kJoinThreads) void cache_join_kernel(const CacheAttnArgs a, const JoinPart first_part, const JoinPart second_part) {
    constexpr int LANES = D / 4, GROUPS = kJoinThreads / LANES;
    __shared__ f32x4 s_o[GROUPS][LANES];
    __shared__ float s_l[GROUPS];
    const int G = a.Hq / a.Hk;
    const unsigned head = first_part.tiles * first_part.per_tile;
    const bool second = blockIdx.x >= head;
    const JoinPart jp = second ? second_part : first_part;
    const Part part = jp.part;
    const unsigned block = blockIdx.x - (second ? head : 0);
    Piece pc;
    if (!find_piece_shared<true>(a, part, jp.ws, block / jp.per_tile, false, pc) || pc.chunks == 1) return;
    if (pc.slot0 + (uint64_t)(pc.chunks - 1) * pc.tiles >= part.room) return;   // rows that overlap: no room was asked for
    const long long stride = (long long)pc.tiles * (part.tile * (D + 2));
    const float* const tile = jp.ws->results + (long long)pc.slot0 * (part.tile * (D + 2));
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int row0 = jp.rows * (block % jp.per_tile), first = pc.tile * part.tile + row0;
    const int rows = min(pc.rows - first, jp.rows);   // of this workgroup
    int width = 1;   // rows at a time, a power of two
    while (width < GROUPS && width < rows) width *= 2;
    const int shares = GROUPS / width, share = group / width;
    for (int j0 = 0; j0 < rows; j0 += width) {
        const int j = j0 + group % width;
        const float* at = tile + 2 * (row0 + j);   // (max, sum) pairs of the rows
        const float* ot = tile + 2 * part.tile + (row0 + j) * D + 4 * lane;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
        if (j < rows) {
            float top = kLowest;
            for (int c = lane; c < pc.chunks; c += LANES) top = fmaxf(top, at[c * stride]);
#pragma unroll
            for (int x = 1; x < LANES; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
            for (int c0 = share; c0 < pc.chunks; c0 += 4 * shares) {   // the loads of four shares at a time
                f32x2 ml[4];
                f32x4 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const long long c = min(c0 + i * shares, pc.chunks - 1) * stride;
                    ml[i] = *reinterpret_cast<const f32x2*>(at + c);
                    v[i] = *reinterpret_cast<const f32x4*>(ot + c);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = c0 + i * shares < pc.chunks ? __builtin_amdgcn_exp2f(ml[i][0] - top) : 0.f;
                    l += c0 + i * shares < pc.chunks ? w * ml[i][1] : 0.f;   // what is read twice may be infinite
                    o += c0 + i * shares < pc.chunks ? w * v[i] : f32x4{0.f, 0.f, 0.f, 0.f};
                }
            }
        }
        if (shares > 1) {
            __syncthreads();   // the sums of the rows before have been read
            s_o[group][lane] = o;
            if (lane == 0) s_l[group] = l;
            __syncthreads();
            if (share == 0)
                for (int x = 1; x < min(shares, pc.chunks); ++x) o += s_o[group + x * width][lane], l += s_l[group + x * width];
        }
        if (share == 0 && j < rows) {
            const float inv = l == 0.f ? 0.f : 1.0f / l;
            const int r = first + j;
            store_run<F32T, VEC>(a.out, (pc.hk * G + r % G) * a.so.h + (pc.row0 + r / G) * a.so.n + 4 * lane, o * inv, 4);
        }
    }
}

// Tiles of a launch at most, whatever the lengths: a request's last tile may be part full.
long long most_tiles(const Part& part, int S, int T, int max_rows, int Hq, int Hk) {
    const int G = Hq / Hk;
    const long long rows = std::min((long long)T, (long long)S * max_rows) * G;
    // a request of this part has more than lo rows
    const long long requests = std::min<long long>(std::min(S, T), rows / (part.lo + 1));
    return (rows / part.tile + requests) * Hk;
}

// Pieces at most where tiles are cut: what fills the slots as often as a plan may; and no tile has more than its pages give.  More tiles
// than that are not cut, and none leaves a result behind.
long long most_cut(const Part& part, int S, long long tiles, int max_pages) {
    const long long rounds = most_rounds(S, tiles > part.slots / 2);   // of no fewer tiles than there are
    return std::min(rounds * part.slots + kSlackPieces, tiles * ((max_pages + kLeastPages - 1) / kLeastPages));
}

struct Plan {
    Part few, many;
    bool use_few, use_many;
    long long few_pieces, many_pieces, few_tiles, many_tiles, few_blocks;
    size_t few_bytes, many_bytes;
    int few_quads;   // fours of rows of a tile of the few, at most
};

// Which kernels a call needs: requests of up to kFewRows rows go to the one for few rows, unless there is one request only, whose
// rows the caller bounds; where no request can have more, nothing goes to the other.
Plan make_plan(int S, int T, int max_rows, int Hq, int Hk, int d, int max_pages) {
    Plan p{};
    const long long most = (long long)std::min(max_rows, T) * (Hq / Hk);
    p.use_many = most > kFewRows && (max_pages > kShortPages || (long long)T * Hq > kShortRows);
    p.use_few = !p.use_many || S > 1;
    p.few = {kFewTile, kFewSlots, kFewCost, 0, p.use_many ? kFewRows : INT_MAX, 0, 0, true, 0};
    p.many = {kManyTile, kManySlots, kManyCost, p.use_few ? kFewRows : 0, INT_MAX, 0, max_pages > kManyWhole ? 0 : kWave, false, 0};
    if (p.use_few) {
        const int rows = p.use_many ? std::min(max_rows, std::max(1, kFewRows / (Hq / Hk))) : max_rows;
        p.few_quads = (int)(std::min<long long>((long long)rows * (Hq / Hk), kFewTile) + 3) / 4;
        p.few_tiles = most_tiles(p.few, S, T, rows, Hq, Hk);
        // Up to so many pages a tile is a workgroup's: no join, and no launch for it where the table has no more (8 requests of one token,
        // 8 heads of 128: 1,000 tokens 12 us in pieces, 9 without, 2,000 tokens 13 and 14; 48 of them over 2,000: 29 and 23).  The
        // tiles that there may be are up to half as many again as there are.
        p.few.whole = p.few_tiles >= 128 ? 32 : 16;
        if (max_pages <= p.few.whole) p.few.uncut = p.few_tiles >= kManyTiles / 2 * 3 && max_pages <= kWavePages ? kWave : kWhole;
        p.few.room = p.few.uncut ? 0 : (unsigned)most_cut(p.few, S, p.few_tiles, max_pages);
        p.few_pieces = std::max<long long>(p.few_tiles, p.few.room);
        p.few_blocks = std::max(p.few_tiles, (p.few_pieces + kFewWaves - 1) / kFewWaves);
        p.few_bytes = !p.few.uncut ? kPartHeader + (size_t)p.few.room * kFewTile * (d + 2) * sizeof(float) : 0;
    }
    if (p.use_many) {
        auto turns = [](long long pieces) { return (pieces / (8 * kRun) + 1) * 8 * kRun; };   // whole turns of runs
        p.many_tiles = most_tiles(p.many, S, T, max_rows, Hq, Hk);
        p.many.room = p.many.uncut ? 0 : (unsigned)turns(most_cut(p.many, S, p.many_tiles, max_pages));
        p.many_pieces = std::max<long long>(turns(p.many_tiles), p.many.room);
        p.many_bytes = !p.many.uncut ? kPartHeader + (size_t)p.many.room * kManyTile * (d + 2) * sizeof(float) : 0;
    }
    return p;
}

}  // namespace

size_t cache_attn_workspace_bytes(int S, int T, int max_rows, int Hq, int Hk, int d, int max_pages) {
    const Plan p = make_plan(S, T, max_rows, Hq, Hk, d, max_pages);
    return p.few_bytes + p.many_bytes;
}

template <int D, bool F32T, bool VEC>
static hipError_t launch(const CacheAttnArgs& a, const Plan& p, hipStream_t st) {
    const float scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)a.d));
    PartSpace* few_ws = p.few_bytes ? static_cast<PartSpace*>(a.ws) : nullptr;
    PartSpace* many_ws = p.many_bytes ? reinterpret_cast<PartSpace*>(static_cast<char*>(a.ws) + p.few_bytes) : nullptr;
    // One launch for both kernels saves the second one's 4 to 8 us (8 requests of one token over 2,000, one of 256 rows: 52 and 45 us).
    // Where that leaves the few two waves a SIMD instead of three (d = 128 in bf16, 64 in f32), it is slower once their keys take
    // longer than a launch: 31 requests of one token and one of 512 rows, 8 heads of 128, 2,000, 4,000 and 16,000 tokens: 70, 78 and
    // 162 us in two launches, 68, 77 and 171 in one.  The table bounds what there may be to read.
    const bool one = p.use_many && p.use_few &&
                     (F32T == (D == 128) || (long long)a.S * a.max_pages * a.Hk * PageLayout<D>::bytes <= 1 << 27);
    if (one) {
        const unsigned grid = (unsigned)(p.many_pieces + p.few_blocks);
        cache_mixed_kernel<D, F32T, VEC><<<grid, 256, 0, st>>>(a, p.few, p.many, scale_log2, few_ws, many_ws, (unsigned)p.few_pieces,
                                                               (unsigned)p.many_pieces);
    } else {
        if (p.use_many) cache_many_kernel<D, F32T, VEC><<<(unsigned)p.many_pieces, 256, 0, st>>>(a, p.many, scale_log2, many_ws);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        if (p.use_few) cache_few_kernel<D, F32T, VEC><<<(unsigned)p.few_blocks, 64 * kFewWaves, 0, st>>>(a, p.few, scale_log2, few_ws, (unsigned)p.few_pieces);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    JoinPart few{p.few, few_ws, few_ws ? (unsigned)p.few_tiles : 0u, (unsigned)p.few_quads, 4};
    // Few tiles have many shares each: a workgroup then takes fewer of a tile's rows, down to four (64 rows against 32,768
    // tokens of 8 heads: the call 47 us with 32 rows to a workgroup, 34 with four).
    int rows = 32;
    while (rows > 4 && p.many_tiles * (kManyTile / rows) < 512) rows /= 2;
    JoinPart many{p.many, many_ws, many_ws ? (unsigned)p.many_tiles : 0u, (unsigned)(kManyTile / rows), rows};
    if (const unsigned grid = few.tiles * few.per_tile + many.tiles * many.per_tile) {
        cache_join_kernel<D, F32T, VEC><<<grid, kJoinThreads, 0, st>>>(a, few, many);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, hipStream_t st) {
    const int size = a.dtype == 0 ? 2 : 4;
    const bool vec = ((reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.out)) & 15) == 0 &&
                     ((a.sq.h | a.sq.n | a.so.h | a.so.n) * size & 15) == 0;
    const Plan p = make_plan(a.S, a.T, a.max_rows, a.Hq, a.Hk, a.d, a.max_pages);
    if (a.dtype == 0) {
        if (a.d == 128) return vec ? launch<128, false, true>(a, p, st) : launch<128, false, false>(a, p, st);
        return vec ? launch<64, false, true>(a, p, st) : launch<64, false, false>(a, p, st);
    }
    if (a.d == 128) return vec ? launch<128, true, true>(a, p, st) : launch<128, true, false>(a, p, st);
    return vec ? launch<64, true, true>(a, p, st) : launch<64, true, false>(a, p, st);
}

}  // namespace sol
