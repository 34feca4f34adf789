// Attention of a tree of new tokens over a paged pool, for gfx950.
//
// The mathematics.  For one request and key/value head, the rows are its new
// tokens times the query heads that share the head (row r: token r / G, head
// h G + r % G), and all rows meet the same keys.  A tile of keys is taken in
// with the running maximum m and sum l of the softmax (in powers of two, the
// scale times log2 e applied to the 32-bit product):
//   S = K Q^T,  m' = max(m, max S),  P = 2^(S - m'),
//   l' = l 2^(m - m') + sum P,  O' = O 2^(m - m') + V^T P,
// and the parts (m, l, O) of separate key ranges join by the same rule.
//
// What bounds it.  A key's row and a value's row (4 dim bytes) meet up to
// G T rows, 4 dim products each: below about 250 rows the pool's bytes
// bound the call, above that the matrix instructions.  Measured, 32 query
// heads over 8 of 128 dims, 16-bit:
//   64 single tokens over 500 to 16000 cached ones   239 us, 5.0 TB/s
//   8 tokens over 260 thousand (64 heads over 8)     210 us, 5.1 TB/s
//   16 trees of 64 over 1000 to 8000                 113 us, 2.2 TB/s, 513 TFLOP/s
//   4 pieces of prompts, 1000 to 2048 tokens over
//   none to 12000                                    403 us, 734 TFLOP/s (393 to
//   429 from one machine to another)
// where a copy of 2 GiB reaches 4.9 TB/s, reading alone 6.3 and a large product
// of matrices 1250 TFLOP/s.
//
// The work.  A workgroup takes an item: row tile rt of one request and head,
// and a range of its keys.  Up to 64 rows, four wavefronts take it
// (tree_attention_kernel): kRowWaves of them share a tile of keys in LDS, 32
// rows each; 4 / kRowWaves groups take tiles in turn and are joined at the
// end, so that few rows still keep four wavefronts' loads under way.  For more
// rows, four or eight wavefronts share every tile (tree_attention_wide_kernel).
// Keys are cut into ranges where the requests alone would leave compute units
// idle; the parts of cut ranges go to the workspace and a second kernel joins
// them.  Only the device knows the lengths: with up to 64 requests every
// wavefront makes the plan for itself, a request a lane; with more a small
// kernel ahead lists the items, which costs 7 to 8 us (one request of 1000
// tokens 20 us for 27, 64 of them 238 us for 246).
//
// Operands.  Products are 32x32x16 matrix instructions with the keys as the
// rows of the first one: its result then holds, in each lane, one query row
// and keys 8 i + 4 (lane / 32) + 0..3, which is the layout that the second
// product's operand needs when the values are read in the same order of keys.
// The weights never leave the registers.  Values are read from LDS by the
// transposing load, four keys of one column a lane.  Chunks of 16 bytes are
// permuted within a row of LDS so that the keys' 16-byte reads and the
// values' transposing reads touch every bank once.
//
// Tree.  A lane's row knows its token; the tokens that it sees in a tile of
// 32 or 64 new tokens are a word of bits, collected by walking up from the
// token.  Tiles of new tokens are taken from the last to the first, so each
// walk goes on where the one before it stopped.

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "coop.h"
#include "coop_pages.h"

namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kRows = 32;            // rows of a wavefront
constexpr uint32_t kParentsInLds = 512;   // trees up to this size are walked in LDS
constexpr uint32_t kPlanThreads = 1024;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -__builtin_inff();
constexpr float kSlack = 8.f;  // how far, in powers of two, the largest weight may grow

struct Item {  // rows [32 kRowWaves rt, ...) of a request and head, tiles [first, last)
    uint32_t request, row_tile, head, first, last;
    uint32_t part;  // where its result goes in the workspace; kWhole: to the output
    uint32_t pad[2];  // (32 bytes)
};
constexpr uint32_t kWhole = ~0u;

struct Join {  // rows whose keys were cut into `parts` ranges
    uint32_t request, row_tile, head, parts, first;
    uint32_t pad[3];
};

struct Head {
    uint32_t items, joins;
    uint32_t pad[6];
};

struct Args {
    coop_rows_t q, k, v;
    coop_cache_t cache;
    const uint64_t* offsets;
    const int32_t* parents;
    const int32_t* table;
    const uint64_t* lengths;
    uint16_t* out;
    uint64_t tokens;
    uint32_t requests, max_pages, q_heads, group;
    uint32_t page_shift;  // page_size is 2^page_shift; 32: not a power of two
    // keys' and values' rows lie alike, and a row's offset is 32-bit products
    // of these
    bool narrow;
    uint32_t page_bytes, place_bytes;
    float scale;
    // the plan and the workspace
    uint32_t tile_keys, row_tile_rows, slots, least, least_more, chunk_multiple, max_items, part_rows;
    Head* head;
    Item* items;
    Join* joins;
    float* part_out;   // [part][part_rows][kDim]
    float2* part_sum;  // [part][part_rows] (m, l)
};

// ---------------------------------------------------------------------------
// The plan
// ---------------------------------------------------------------------------

struct Extent {
    uint64_t first;    // first new token
    uint32_t tokens;   // new tokens
    uint32_t cached;   // cached tokens that the table can name
};

__device__ __forceinline__ Extent extent(const Args& a, uint32_t b) {
    Extent e;
    const uint64_t o0 = a.offsets[b], o1 = min(a.offsets[b + 1], a.tokens);
    e.first = o0;
    e.tokens = o0 < o1 ? static_cast<uint32_t>(o1 - o0) : 0u;
    const uint64_t most = static_cast<uint64_t>(a.max_pages) * a.cache.page_size;
    e.cached = a.cache.num_pages ? static_cast<uint32_t>(min(a.lengths[b], most)) : 0u;
    return e;
}

__device__ __forceinline__ uint32_t ceil_div(uint32_t x, uint32_t y) { return (x + y - 1) / y; }

// v of the lane that a step of a scan adds: one, two, four, eight lanes below in
// rows of 16, then the last lane of the row before, then lane 31; 0 where there
// is none.
template <int kStep>
__device__ __forceinline__ uint32_t from_below(uint32_t v) {
    constexpr int kControl = kStep < 4 ? 0x110 + (1 << kStep) : kStep == 4 ? 0x142 : 0x143;
    constexpr int kRowMask = kStep < 4 ? 0xf : kStep == 4 ? 0xa : 0xc;
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), kControl, kRowMask, 0xf, false));
}

template <int kStep>
__device__ __forceinline__ uint64_t from_below(uint64_t v) {
    return from_below<kStep>(static_cast<uint32_t>(v)) |
           static_cast<uint64_t>(from_below<kStep>(static_cast<uint32_t>(v >> 32))) << 32;
}

// Running sums over a wavefront's lanes.
template <class U>
__device__ __forceinline__ U scan_lanes(U v) {
    v += from_below<0>(v);
    v += from_below<1>(v);
    v += from_below<2>(v);
    v += from_below<3>(v);
    v += from_below<4>(v);
    return v + from_below<5>(v);
}

__device__ __forceinline__ uint32_t from_lane(uint32_t v, uint32_t lane) {
    return __builtin_amdgcn_readlane(v, lane);
}
__device__ __forceinline__ uint64_t from_lane(uint64_t v, uint32_t lane) {
    return from_lane(static_cast<uint32_t>(v), lane) |
           static_cast<uint64_t>(from_lane(static_cast<uint32_t>(v >> 32), lane)) << 32;
}

template <class U>
__device__ __forceinline__ U wave_sum(U v) { return from_lane(scan_lanes(v), 63); }

// Pairs (a request's row tile and head) of many tiles are cut into ranges of
// `chunk` tiles, all of one length.  Workgroups take ranges as they come free,
// a.slots of them at once.
//  - If ranges that cut the whole work W evenly among the slots all fit at
//    once, they end together; 128 keys at least, where all fit anyhow: a start,
//    an end and a part to join cost as much as some 200 keys.  With 512 keys at
//    least, four sequences of 100 to 700 tokens took 14.2 us for 11.0, one tree
//    of 64 tokens after 1000 (32 heads over 8 of 128 dims) 31 us for 23, after
//    8000 34 us for 33.
//  - Where pairs leave too many remainders for that, ranges of half the length
//    keep the wait for the last ones short, 1024 keys at least: 48 trees over
//    e4m3 keys took 119 us for 109 with 512 and 124 us with 2048, 64 trees of
//    12 tokens 132 and 148 for 126, 64 single tokens the same 234 with each.
//    Even ranges throughout took 260 us for the last.
// Other lengths, tried until their ranges fit, gained less than this plan grew,
// which every wavefront makes: 64 single tokens took 241 us for 234.
// Ranges no shorter than W / n tiles leave at most 2 n parts.
__device__ __forceinline__ uint32_t chunk_of(const Args& a, uint64_t work, uint32_t slots, uint32_t least) {
    const float even = ceilf(static_cast<float>(work) / static_cast<float>(slots)) + 1.f;
    const uint32_t n = even < 0x1p30f ? max(static_cast<uint32_t>(even), least) : 1u << 30;
    return (n + a.chunk_multiple - 1) / a.chunk_multiple * a.chunk_multiple;
}

// (`ranges(n)`: how many ranges of n tiles there are)
template <class Ranges>
__device__ __forceinline__ uint32_t chunk_of(const Args& a, uint64_t work, Ranges ranges) {
    const uint32_t even = chunk_of(a, work, a.slots, a.least);
    return ranges(even) <= a.slots ? even : chunk_of(a, work, 2 * a.slots, a.least_more);
}

__device__ __forceinline__ uint32_t row_tiles_of(const Args& a, uint32_t tokens) {
    return static_cast<uint32_t>((static_cast<uint64_t>(tokens) * a.group + a.row_tile_rows - 1) / a.row_tile_rows);
}

__device__ __forceinline__ uint32_t tiles_of(const Args& a, const Extent& e) {
    return e.tokens ? ceil_div(e.cached, a.tile_keys) + ceil_div(e.tokens, a.tile_keys) : 0;
}

// The plan of at most 64 requests, which every wavefront makes for itself: a
// lane holds a request's numbers.
struct LanePlan {
    Extent e;
    uint32_t chunk, tiles, pairs, ranges;
    uint32_t items, cuts, joins;  // running sums, this request's included
};

__device__ __forceinline__ LanePlan lane_plan(const Args& a, uint32_t lane) {
    LanePlan p;
    p.e = Extent{0, 0, 0};
    if (lane < a.requests) p.e = extent(a, lane);
    const uint32_t heads = static_cast<uint32_t>(a.cache.heads);
    p.tiles = tiles_of(a, p.e);
    p.pairs = row_tiles_of(a, p.e.tokens) * heads;
    const uint64_t work = wave_sum(static_cast<uint64_t>(p.pairs) * p.tiles);
    p.chunk = chunk_of(a, work, [&](uint32_t n) { return wave_sum(p.pairs * ceil_div(p.tiles, n)); });
    p.ranges = ceil_div(p.tiles, p.chunk);
    const bool cut = p.ranges > 1;
    p.items = scan_lanes(p.pairs * p.ranges);
    p.cuts = scan_lanes(cut ? p.pairs * p.ranges : 0u);
    p.joins = scan_lanes(cut ? p.pairs : 0u);
    return p;
}

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// The item and its request as scalars.
__device__ __forceinline__ Item uniform(const Item& i) {
    return {uniform(i.request), uniform(i.row_tile), uniform(i.head), uniform(i.first),
            uniform(i.last), uniform(i.part), {0, 0}};
}
__device__ __forceinline__ Extent uniform(const Extent& e) {
    Extent r;
    r.first = uniform(static_cast<uint32_t>(e.first)) |
              static_cast<uint64_t>(uniform(static_cast<uint32_t>(e.first >> 32))) << 32;
    r.tokens = uniform(e.tokens);
    r.cached = uniform(e.cached);
    return r;
}

__device__ __forceinline__ Extent extent_of(const LanePlan& p, uint32_t r) {
    Extent e;
    e.first = from_lane(static_cast<uint32_t>(p.e.first), r) |
              static_cast<uint64_t>(from_lane(static_cast<uint32_t>(p.e.first >> 32), r)) << 32;
    e.tokens = from_lane(p.e.tokens, r);
    e.cached = from_lane(p.e.cached, r);
    return e;
}

// Consecutive workgroups go to the eight dies in turn, and consecutive items to
// consecutive heads.  Heads that lie side by side in a pool's rows are in few
// of a die's cache channels each, so a die that met one head only would work
// with these; the heads are turned from one row tile, range and request to the
// next.
__device__ __forceinline__ uint32_t turned(uint32_t head, uint32_t by, uint32_t heads) {
    return (head + by % heads) % heads;
}

// Item i of the plan; false if it has no such item.
__device__ __forceinline__ bool item_of(const Args& a, const LanePlan& p, uint32_t i, Item* it,
                                        Extent* e) {
    const uint64_t past = __ballot(p.items > i);
    if (!past) return false;
    const uint32_t r = static_cast<uint32_t>(__builtin_ctzll(past));
    const uint32_t pairs = from_lane(p.pairs, r), ranges = from_lane(p.ranges, r);
    const uint32_t j = i - (from_lane(p.items, r) - pairs * ranges);
    const uint32_t c = j / pairs, k = j - c * pairs, heads = static_cast<uint32_t>(a.cache.heads);
    *e = extent_of(p, r);
    it->request = r;
    it->row_tile = k / heads;
    it->head = turned(k - it->row_tile * heads, r + c + it->row_tile, heads);
    it->first = c * p.chunk;
    it->last = min(from_lane(p.tiles, r), it->first + p.chunk);
    const uint32_t pair = it->row_tile * heads + it->head;
    it->part = ranges > 1 ? from_lane(p.cuts, r) - pairs * ranges + pair * ranges + c : kWhole;
    return true;
}

__device__ __forceinline__ void join_of(const Args& a, const LanePlan& p, uint32_t i, Join* jn,
                                        Extent* e) {
    const uint32_t r = static_cast<uint32_t>(__builtin_ctzll(__ballot(p.joins > i)));
    const uint32_t pairs = from_lane(p.pairs, r), heads = static_cast<uint32_t>(a.cache.heads);
    const uint32_t pair = i - (from_lane(p.joins, r) - pairs);
    *e = extent_of(p, r);
    jn->request = r;
    jn->row_tile = pair / heads;
    jn->head = pair - jn->row_tile * heads;
    jn->parts = from_lane(p.ranges, r);
    jn->first = from_lane(p.cuts, r) - pairs * jn->parts + pair * jn->parts;
}

// More requests: one workgroup lists the items and the joins.
__global__ __launch_bounds__(kPlanThreads) void attention_plan_kernel(Args a) {
    __shared__ uint64_t part[kPlanThreads / 64][3];
    __shared__ uint32_t item_base[kPlanThreads + 1], cut_base[kPlanThreads], join_base[kPlanThreads + 1];
    __shared__ uint32_t request_rows[kPlanThreads], request_tiles[kPlanThreads];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, w = tid >> 6;
    const uint32_t heads = static_cast<uint32_t>(a.cache.heads);
    uint64_t work = 0;
    for (uint32_t b = tid; b < a.requests; b += kPlanThreads) {
        const Extent e = extent(a, b);
        work += static_cast<uint64_t>(row_tiles_of(a, e.tokens)) * heads * tiles_of(a, e);
    }
    auto block_sum = [&](uint64_t v) {
        v = wave_sum(v);
        __syncthreads();
        if (lane == 0) part[w][0] = v;
        __syncthreads();
        v = 0;
        for (uint32_t i = 0; i < kPlanThreads / 64; ++i) v += part[i][0];
        return v;
    };
    work = block_sum(work);
    const uint32_t chunk = chunk_of(a, work, [&](uint32_t n) {
        uint64_t ranges = 0;
        for (uint32_t b = tid; b < a.requests; b += kPlanThreads) {
            const Extent e = extent(a, b);
            ranges += static_cast<uint64_t>(row_tiles_of(a, e.tokens)) * heads * ceil_div(tiles_of(a, e), n);
        }
        return block_sum(ranges);
    });
    __syncthreads();
    uint32_t items0 = 0, cuts0 = 0, joins0 = 0;  // of the requests before this batch
    for (uint32_t b0 = 0; b0 < a.requests; b0 += kPlanThreads) {
        const uint32_t b = b0 + tid;
        uint32_t tiles = 0, rt = 0;
        if (b < a.requests) {
            const Extent e = extent(a, b);
            rt = row_tiles_of(a, e.tokens);
            tiles = tiles_of(a, e);
        }
        const uint32_t pairs = rt * heads, ranges = ceil_div(tiles, chunk);
        const uint64_t mine[3] = {static_cast<uint64_t>(pairs) * ranges,
                                  ranges > 1 ? static_cast<uint64_t>(pairs) * ranges : 0,
                                  ranges > 1 ? pairs : 0};
        uint64_t sum[3], all[3];
        for (int k = 0; k < 3; ++k) {
            sum[k] = scan_lanes(mine[k]);
        }
        __syncthreads();
        if (lane == 63)
            for (int k = 0; k < 3; ++k) part[w][k] = sum[k];
        __syncthreads();
        for (int k = 0; k < 3; ++k) {
            all[k] = 0;
            for (uint32_t i = 0; i < kPlanThreads / 64; ++i) {
                if (i < w) sum[k] += part[i][k];
                all[k] += part[i][k];
            }
        }
        item_base[tid] = static_cast<uint32_t>(min(sum[0] - mine[0], static_cast<uint64_t>(kWhole)));
        cut_base[tid] = static_cast<uint32_t>(sum[1] - mine[1]);
        join_base[tid] = static_cast<uint32_t>(sum[2] - mine[2]);
        request_rows[tid] = rt;
        request_tiles[tid] = tiles;
        if (tid == kPlanThreads - 1) {
            item_base[kPlanThreads] = static_cast<uint32_t>(min(sum[0], static_cast<uint64_t>(kWhole)));
            join_base[kPlanThreads] = static_cast<uint32_t>(sum[2]);
        }
        __syncthreads();
        const uint32_t n = min(item_base[kPlanThreads], a.max_items - items0);
        for (uint32_t i = tid; i < n; i += kPlanThreads) {
            uint32_t lo = 0, hi = kPlanThreads;  // the last request whose items start at or before i
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) >> 1;
                if (item_base[mid] <= i) lo = mid;
                else hi = mid;
            }
            const uint32_t j = i - item_base[lo], p = request_rows[lo] * heads;
            const uint32_t c = j / p, k = j - c * p;
            const uint32_t t = request_tiles[lo], r = ceil_div(t, chunk);
            Item it;
            it.request = b0 + lo;
            it.row_tile = k / heads;
            it.head = turned(k - it.row_tile * heads, it.request + c + it.row_tile, heads);
            it.first = c * chunk;
            it.last = min(t, it.first + chunk);
            const uint32_t pair = it.row_tile * heads + it.head;
            it.part = r > 1 ? cuts0 + cut_base[lo] + pair * r + c : kWhole;
            it.pad[0] = it.pad[1] = 0;
            a.items[items0 + i] = it;
        }
        for (uint32_t i = tid; i < join_base[kPlanThreads]; i += kPlanThreads) {
            uint32_t lo = 0, hi = kPlanThreads;
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) >> 1;
                if (join_base[mid] <= i) lo = mid;
                else hi = mid;
            }
            const uint32_t pair = i - join_base[lo], r = ceil_div(request_tiles[lo], chunk);
            Join jn;
            jn.request = b0 + lo;
            jn.row_tile = pair / heads;
            jn.head = pair - jn.row_tile * heads;
            jn.parts = r;
            jn.first = cuts0 + cut_base[lo] + pair * r;
            jn.pad[0] = jn.pad[1] = jn.pad[2] = 0;
            a.joins[joins0 + i] = jn;
        }
        items0 += n;
        cuts0 += static_cast<uint32_t>(all[1]);
        joins0 += join_base[kPlanThreads];
        __syncthreads();
    }
    if (tid == 0) {
        a.head->items = items0;
        a.head->joins = joins0;
    }
}

// ---------------------------------------------------------------------------
// Number types
// ---------------------------------------------------------------------------

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
    typedef __bf16 Vec8 __attribute__((ext_vector_type(8)));
    typedef __bf16 Vec2 __attribute__((ext_vector_type(2)));
    static constexpr uint32_t kExponent = 0x7f80u;
    static constexpr float kLift = 0.f;  // the largest weight is taken as 2^kLift
    static __device__ __forceinline__ f32x16 mfma(u32x4 x, u32x4 y, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Vec8, x),
                                                       __builtin_bit_cast(Vec8, y), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) {
        const Vec2 v = {static_cast<__bf16>(x), static_cast<__bf16>(y)};
        return __builtin_bit_cast(uint32_t, v);
    }
    static __device__ __forceinline__ float value(uint16_t bits) {
        return __uint_as_float(static_cast<uint32_t>(bits) << 16);
    }
    template <bool kUpper>
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t word) {
        return __builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, 1.f, kUpper));
    }
};

struct Fp16 {
    typedef _Float16 Vec8 __attribute__((ext_vector_type(8)));
    typedef _Float16 Vec2 __attribute__((ext_vector_type(2)));
    static constexpr uint32_t kExponent = 0x7c00u;
    // Numbers below 2^-14 have a fixed step of 2^-24, which a sum of many small
    // weights would feel (a first token with a score far above all others).
    // Lifted, weights are at most 2^(kLift + kSlack) = 2^15, which fp16 holds,
    // and lose bits only from 2^-21 of the largest down.
    static constexpr float kLift = 7.f;
    static __device__ __forceinline__ f32x16 mfma(u32x4 x, u32x4 y, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Vec8, x),
                                                      __builtin_bit_cast(Vec8, y), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) {
        const Vec2 v = {static_cast<_Float16>(x), static_cast<_Float16>(y)};
        return __builtin_bit_cast(uint32_t, v);
    }
    static __device__ __forceinline__ float value(uint16_t bits) {
        return static_cast<float>(__builtin_bit_cast(_Float16, bits));
    }
    template <bool kUpper>
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t word) {
        return __builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, 1.f, kUpper));
    }
};

// ---------------------------------------------------------------------------
// The attention kernel
// ---------------------------------------------------------------------------

// Up to 64 rows: memory bounds it, so a tile's rows are on their way through
// registers while the tile before is in use, and what an 8-bit tile holds is
// converted (exactly) once, as it goes to LDS.  The queries stay in LDS: a
// wavefront's sums, scores and the rows under way leave no registers for them.
// 64 single tokens over 500 to 16000 cached ones: 225 us for 1.19 GB, with one
// wavefront along the rows; 64 trees of 12 tokens, 48 rows, over 200 to 4000:
// 95 us for 355 MB, with two.
template <class T, bool kE4M3, uint32_t kDim, uint32_t kRowWaves>
struct Shape {
    static_assert(kRowWaves == 1 || kRowWaves == 2, "more rows are the wide kernel's");
    static constexpr uint32_t kGroups = 4 / kRowWaves;
    static constexpr uint32_t kKeys = 32;  // of a tile
    static constexpr uint32_t kGroupThreads = 64 * kRowWaves;
    static constexpr uint32_t kChunks = kDim / 8;  // 16-byte chunks of a row in LDS
    static constexpr uint32_t kLoads = kKeys * kChunks / kGroupThreads;      // a thread's, a tile
    static constexpr uint32_t kLoads8 = kLoads / 2;                          // with 8-bit rows
    static constexpr uint32_t kTileBytes = kKeys * kDim * 2;
    static constexpr uint32_t kDTiles = kDim / 32;
    static constexpr uint32_t kBytes = kGroups * 2 * kTileBytes;
    static_assert(kLoads8 >= 1, "a thread has a load of every kind");
};

// Where chunk c of row r lies in its row.
template <uint32_t kDim>
__device__ __forceinline__ uint32_t key_chunk(uint32_t r, uint32_t c) {
    return kDim == 64 ? c ^ ((r >> 1) & 7u) : c ^ (r & 15u);
}
template <uint32_t kDim>
__device__ __forceinline__ uint32_t value_chunk(uint32_t r, uint32_t c) {
    return kDim == 64 ? c ^ (((r >> 1) & 1u) << 2) : c ^ ((r & 3u) << 2);
}

// Device memory by name: a load through a pointer that itself comes from LDS
// would otherwise be one that may mean LDS, and every wait for LDS would wait
// for it too.
typedef const __attribute__((address_space(1))) uint8_t* Global;

__device__ __forceinline__ u32x4 load16(Global p) {
    return *reinterpret_cast<const __attribute__((address_space(1))) u32x4*>(p);
}

struct RowAt {  // where a tile's key and value rows are in memory
    Global k;
    Global v;
};

// What a lane's row sees of the new tokens: its own token and that one's
// ancestors, found by walking up.
struct Sight {
    const int32_t* parents;  // the request's; null: each token's parent is the one before it
    const int32_t* tree;     // the same in LDS, if in_lds
    bool in_lds;
    int32_t token;           // the row's, -1: sees none
    int32_t at, up;          // the walk's place (-1: it has ended), and that one's parent

    __device__ __forceinline__ int32_t parent_of(int32_t i) const {
        if (in_lds) return *((const __attribute__((address_space(3))) int32_t*)tree + i);
        return *((const __attribute__((address_space(1))) int32_t*)parents + i);
    }

    __device__ __forceinline__ void start() {
        at = token;
        up = at - 1;
        if (at >= 0 && parents) {
            up = parent_of(at);
            if (up < -1 || up >= at) at = -1;  // void
        }
    }

    __device__ __forceinline__ void climb() {
        const int32_t next = up;
        if (next < 0) {
            at = -1;
            return;
        }
        const int32_t above = parents ? parent_of(next) : next - 1;
        at = above < -1 || above >= next ? -1 : next;
        up = above;
    }

    // The tokens [k0, k0 + kKeys) that it sees, as bits; calls come with
    // falling k0.
    template <uint32_t kKeys>
    __device__ __forceinline__ uint64_t of_tile(int32_t k0) {
        uint64_t sees = 0;
        if (!parents) {
            const int32_t past = token - k0;
            if (token >= 0 && past >= 0) sees = past >= 63 ? ~0ull : (2ull << past) - 1;
            return kKeys == 64 ? sees : sees & 0xffffffffu;
        }
        while (at >= k0 + static_cast<int32_t>(kKeys)) climb();
        while (at >= k0) {
            sees |= 1ull << (at - k0);
            climb();
        }
        return sees;
    }
};

// A lane's place in its pair, and the tiles that the item takes.
struct Place {
    uint32_t token, q_head;
    bool lives;              // the row exists
    uint32_t part_row;       // the row's number in its row tile
    uint32_t cached_tiles, new_tiles, first, last;
};

// Cached keys' tiles come first, then those of new tokens, from the last that
// any of the item's rows can see to the first.
template <uint32_t kKeys>
__device__ __forceinline__ Place place_of(const Args& a, const Item& item, const Extent& e, uint32_t part_row) {
    Place p;
    const uint32_t rows = e.tokens * a.group, row0 = item.row_tile * a.row_tile_rows, row = row0 + part_row;
    p.part_row = part_row;
    p.lives = row < rows;
    p.token = row / a.group;
    p.q_head = item.head * a.group + row % a.group;
    p.cached_tiles = ceil_div(e.cached, kKeys);
    p.new_tiles = (min(rows, row0 + a.row_tile_rows) - 1) / a.group / kKeys + 1;
    p.first = item.first;
    p.last = min(item.last, p.cached_tiles + p.new_tiles);
    return p;
}

// The item of this workgroup; false if there is none.
__device__ __forceinline__ bool take_item(const Args& a, Item* item, Extent* e) {
    if (a.requests <= 64) {
        if (!item_of(a, lane_plan(a, threadIdx.x & 63u), blockIdx.x, item, e)) return false;
    } else {
        if (blockIdx.x >= a.head->items) return false;
        *item = a.items[blockIdx.x];
        *e = extent(a, item->request);
    }
    *item = uniform(*item);
    *e = uniform(*e);
    return true;
}

// Masks the scores of a tile and moves the sums' base.  Scores are s * factor;
// where keys are masked, or the factor is negative and does not keep the
// maximum, they are formed here, and the factor becomes one.  The base is
// T::kLift below the largest score, and stays until a weight passes 2^kLift by
// 2^kSlack: weights are then at most 2^(kLift + kSlack), which the type holds,
// and the accumulators are seldom scaled (l and o have a common factor that the
// division takes out).  Returns what o is to be multiplied by.
template <class T, uint32_t kTiles>
__device__ __forceinline__ float new_base(f32x16* s, uint64_t sees, uint64_t full, uint32_t hi,
                                          float* factor, float* m, float* l) {
    if (*factor < 0.f || !__all(sees == full)) {
#pragma unroll
        for (uint32_t t = 0; t < kTiles; ++t) {
            const uint32_t bits = static_cast<uint32_t>(sees >> (32 * t)) >> (4 * hi);
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i)
                s[t][i] = (bits >> (8 * (i >> 2) + (i & 3))) & 1u ? s[t][i] * *factor : kLowest;
        }
        *factor = 1.f;
    }
    float top = s[0][0];
#pragma unroll
    for (uint32_t t = 0; t < kTiles; ++t)
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
    top = fmaxf(top, __shfl_xor(top, 32, 64)) * *factor - T::kLift;
    float grow = 1.f;
    if (__any(top > *m + kSlack)) {
        const float m2 = fmaxf(*m, top);
        grow = m2 == kLowest ? 1.f : __builtin_amdgcn_exp2f(*m - m2);
        *m = m2;
        *l *= grow;
    }
    return grow;
}

// The weights of a tile's scores, as pairs of the products' type; returns
// their sum before that rounding.  (The matrix instructions take operands of 16
// bits, so weights lose half a step of bf16 or fp16, 2^-9 or 2^-12 of the power
// of two below them; what multiplies them, the values, has 16 bits already.)
template <class T, uint32_t kTiles>
__device__ __forceinline__ float weights_of(const f32x16* s, float factor, float m, uint32_t (*p)[8]) {
    const float base = m == kLowest ? 0.f : m;  // no score above the lowest yet
    float sum = 0.f;
#pragma unroll
    for (uint32_t t = 0; t < kTiles; ++t)
#pragma unroll
        for (uint32_t i = 0; i < 16; i += 2) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[t][i], factor, -base));
            const float y = __builtin_amdgcn_exp2f(fmaf(s[t][i + 1], factor, -base));
            sum += x + y;
            p[t][i / 2] = T::pack(x, y);
        }
    return sum;
}

// Writes a row, or its part.
template <class T, uint32_t kDim, uint32_t kKeys>
__device__ __forceinline__ void write_row(const Args& a, const Item& item, const Extent& e, const Place& p,
                                          Sight& sight, bool odd, uint32_t hi, f32x16* o, float m, float l) {
    if (!p.lives) return;
    const uint32_t dim = static_cast<uint32_t>(a.cache.dim);
    if (p.last > p.cached_tiles && odd) {
        // Values that are not finite were left out of the products, where a
        // weight of zero would not keep them from rows that do not see them.
        // The rows that see them take them here (weights are above zero).
        const uint32_t tiles = p.cached_tiles + p.new_tiles;
        const int32_t below = static_cast<int32_t>((tiles - max(p.first, p.cached_tiles)) * kKeys);
        const int32_t from = static_cast<int32_t>((tiles - p.last) * kKeys);
        for (sight.start(); sight.at >= from; sight.climb()) {
            if (sight.at >= below) continue;
            const uint16_t* const v = static_cast<const uint16_t*>(a.v.data) +
                                      (e.first + sight.at) * a.v.stride[0] + item.head * a.v.stride[1];
#pragma unroll
            for (uint32_t t = 0; t < kDim / 32; ++t)
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i) {
                    const uint32_t d = 32 * t + 8 * (i >> 2) + 4 * hi + (i & 3);
                    const uint16_t bits = d < dim ? v[d] : 0;
                    if ((bits & T::kExponent) == T::kExponent) o[t][i] += T::value(bits);
                }
        }
    }
    if (item.part == kWhole) {
        bool is_void = false;
        if (sight.parents) {
            const int32_t up = sight.parents[p.token];
            is_void = up < -1 || up >= static_cast<int32_t>(p.token);
        }
        uint16_t* const to = a.out + ((e.first + p.token) * a.q_heads + p.q_head) * dim;
        const float inverse = 1.f / l;  // (its rounding is far below that of the result)
#pragma unroll
        for (uint32_t t = 0; t < kDim / 32; ++t)
#pragma unroll
            for (uint32_t i = 0; i < 16; i += 4) {
                const uint32_t d = 32 * t + 2 * i + 4 * hi;
                if (d >= dim) continue;
                uint2 x = make_uint2(T::pack(o[t][i] * inverse, o[t][i + 1] * inverse),
                                     T::pack(o[t][i + 2] * inverse, o[t][i + 3] * inverse));
                if (is_void) x = make_uint2(0, 0);
                *reinterpret_cast<uint2*>(to + d) = x;
            }
    } else {
        const uint64_t at = static_cast<uint64_t>(item.part) * a.part_rows + p.part_row;
        float* const to = a.part_out + at * kDim;
#pragma unroll
        for (uint32_t t = 0; t < kDim / 32; ++t)
#pragma unroll
            for (uint32_t i = 0; i < 16; i += 4)
                *reinterpret_cast<float4*>(to + 32 * t + 2 * i + 4 * hi) =
                    make_float4(o[t][i], o[t][i + 1], o[t][i + 2], o[t][i + 3]);
        if (hi == 0) a.part_sum[at] = make_float2(m, l);
    }
}

// Zeroes the halves of four words that are not finite; whether there were any.
// (An exponent of ones carries into the place of the sign, and no further.)
template <class T>
__device__ __forceinline__ bool only_finite(u32x4* x) {
    constexpr uint32_t kBoth = T::kExponent * 0x10001u, kOne = (T::kExponent & -T::kExponent) * 0x10001u;
    uint32_t any = 0;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) any |= ((*x)[i] & kBoth) + kOne;
    if (!(any & 0x80008000u)) return false;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t odd = (((*x)[i] & kBoth) + kOne) & 0x80008000u;
        if (odd & 0x8000u) (*x)[i] &= 0xffff0000u;
        if (odd & 0x80000000u) (*x)[i] &= 0x0000ffffu;
    }
    return true;
}

template <class T, bool kE4M3, uint32_t kDim, uint32_t kRowWaves>
__global__ __launch_bounds__(kThreads, kDim == 256 ? 1 : 2) void tree_attention_kernel(Args a) {
    using S = Shape<T, kE4M3, kDim, kRowWaves>;
    constexpr uint32_t kKeys = S::kKeys, kLoads = S::kLoads, kLoads8 = S::kLoads8;
    constexpr uint64_t kFull = 0xffffffffull;
    __shared__ __align__(16) uint8_t tiles[S::kBytes];
    __shared__ __align__(16) uint8_t queries[kRowWaves * kRows * kDim * 2];
    __shared__ RowAt rows_at[4][kKeys];           // one copy a wavefront
    __shared__ int32_t tree[kParentsInLds];
    __shared__ uint32_t odd;                      // whether new values are not all finite
    __shared__ float joined[4][kRows][2];

    const uint32_t tid = threadIdx.x, lane = tid & 63u;
    Item item;
    Extent e;
    if (!take_item(a, &item, &e)) return;
    const uint32_t w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t group = w / kRowWaves, row_wave = w % kRowWaves;
    const uint32_t gtid = tid - group * S::kGroupThreads;
    const uint32_t n = lane & 31u, hi = lane >> 5;
    const uint32_t dim = static_cast<uint32_t>(a.cache.dim);
    const uint32_t page_size = static_cast<uint32_t>(a.cache.page_size);
    auto page_at = [&](uint32_t pos) { return a.page_shift < 32 ? pos >> a.page_shift : pos / page_size; };
    const Place place = place_of<kKeys>(a, item, e, row_wave * kRows + n);
    const uint32_t cached_tiles = place.cached_tiles, new_tiles = place.new_tiles;
    const uint32_t first = place.first, last = place.last;

    uint8_t* const key_tile = tiles + group * 2 * S::kTileBytes;
    uint8_t* const value_tile = key_tile + S::kTileBytes;

    Sight sight;
    sight.parents = a.parents ? a.parents + e.first : nullptr;
    sight.tree = tree;
    sight.in_lds = a.parents && e.tokens <= kParentsInLds && last > cached_tiles;
    sight.token = place.lives && last > cached_tiles ? static_cast<int32_t>(place.token) : -1;
    if (sight.in_lds)
        for (uint32_t i = tid; i < e.tokens; i += kThreads) tree[i] = sight.parents[i];
    if (tid == 0) odd = 0;
    // the rows' queries, permuted as the keys are
    uint8_t* const query_tile = queries + row_wave * kRows * kDim * 2;
    if (group == 0) {
        const uint16_t* const base = static_cast<const uint16_t*>(a.q.data) +
                                     (e.first + place.token) * a.q.stride[0] + place.q_head * a.q.stride[1];
#pragma unroll
        for (uint32_t c = 0; c < kDim / 16; ++c) {
            const uint32_t d = 16 * c + 8 * hi;
            u32x4 x = {0, 0, 0, 0};
            if (place.lives && d < dim) x = *reinterpret_cast<const u32x4*>(base + d);
            *reinterpret_cast<u32x4*>(query_tile + (n * S::kChunks + key_chunk<kDim>(n, 2 * c + hi)) * 16) = x;
        }
    }
    __syncthreads();  // (all groups read the queries, which the first one writes)
    sight.start();

    f32x16 o[S::kDTiles];
#pragma unroll
    for (uint32_t t = 0; t < S::kDTiles; ++t)
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = kLowest, l = 0.f;

    const float new_scale = a.scale * kLog2e;
    const float cached_scale = kE4M3 ? new_scale * a.cache.k_scale[item.head] : new_scale;
    const float value_scale = kE4M3 ? a.cache.v_scale[item.head] : 1.f;
    bool scaled = false;  // whether o has met the cached values' scale

    // rows that do not count are read from a place that is there and left out
    const Global spare = (Global)(a.q.data);
    const uint64_t size = kE4M3 ? 1 : 2;
    const Global ck = (Global)(a.cache.k) + item.head * a.cache.k_stride[2] * size;
    const Global cv = (Global)(a.cache.v) + item.head * a.cache.v_stride[2] * size;

    // A tile's page number for lane's key (lanes past the tile repeat it).
    const uint32_t my_key = lane % kKeys;
    auto page_of = [&](uint32_t tile) -> int32_t {
        const uint32_t pos = tile * kKeys + my_key;
        if (tile >= cached_tiles || pos >= e.cached) return -1;
        return a.table[static_cast<uint64_t>(item.request) * a.max_pages + page_at(pos)];
    };
    // Writes where the tile's rows are; returns which of its keys count.
    auto locate = [&](uint32_t tile, int32_t page) -> uint64_t {
        RowAt r = {spare, spare};
        bool counts = false;
        if (tile < cached_tiles) {
            const uint32_t pos = tile * kKeys + my_key;
            counts = pos < e.cached && static_cast<uint32_t>(page) < a.cache.num_pages;
            if (counts) {
                const uint32_t in_page = pos - page_at(pos) * page_size, p = static_cast<uint32_t>(page);
                if (a.narrow) {
                    const uint64_t at = static_cast<uint64_t>(p) * a.page_bytes + in_page * a.place_bytes;
                    r.k = ck + at;
                    r.v = cv + at;
                } else {
                    r.k = ck + (p * a.cache.k_stride[0] + in_page * a.cache.k_stride[1]) * size;
                    r.v = cv + (p * a.cache.v_stride[0] + in_page * a.cache.v_stride[1]) * size;
                }
            }
        } else {
            const uint32_t j = (cached_tiles + new_tiles - 1 - tile) * kKeys + my_key;
            counts = j < e.tokens;
            if (counts) {
                r.k = (Global)(a.k.data) + ((e.first + j) * a.k.stride[0] + item.head * a.k.stride[1]) * 2;
                r.v = (Global)(a.v.data) + ((e.first + j) * a.v.stride[0] + item.head * a.v.stride[1]) * 2;
            }
        }
        if (lane < kKeys) rows_at[w][my_key] = r;
        return __ballot(counts) & kFull;
    };

    u32x4 kreg[kLoads], vreg[kLoads];
    const uint32_t chunk = gtid % S::kChunks, row_of_load = gtid / S::kChunks;
    constexpr uint32_t kRowStep = S::kGroupThreads / S::kChunks;
    constexpr uint32_t kChunks8 = S::kChunks / 2, kRowStep8 = S::kGroupThreads / kChunks8;
    const uint32_t chunk8 = gtid % kChunks8, row_of_load8 = gtid / kChunks8;
    auto load = [&](uint32_t tile) {
        if (kE4M3 && tile < cached_tiles) {
            const uint32_t byte = chunk8 * 16 < dim ? chunk8 * 16 : 0;
#pragma unroll
            for (uint32_t j = 0; j < kLoads8; ++j) {
                const RowAt r = rows_at[w][row_of_load8 + j * kRowStep8];
                kreg[j] = load16(r.k + byte);
                vreg[j] = load16(r.v + byte);
            }
        } else {
            const uint32_t byte = chunk * 8 < dim ? chunk * 16 : 0;
#pragma unroll
            for (uint32_t j = 0; j < kLoads; ++j) {
                const RowAt r = rows_at[w][row_of_load + j * kRowStep];
                kreg[j] = load16(r.k + byte);
                vreg[j] = load16(r.v + byte);
            }
        }
    };
    auto put = [&](uint32_t r, uint32_t c, u32x4 kx, u32x4 vx) {
        *reinterpret_cast<u32x4*>(key_tile + (r * S::kChunks + key_chunk<kDim>(r, c)) * 16) = kx;
        *reinterpret_cast<u32x4*>(value_tile + (r * S::kChunks + value_chunk<kDim>(r, c)) * 16) = vx;
    };
    auto store = [&](uint32_t tile, uint64_t counts) {
        const bool whole = counts == kFull && dim == kDim;
        const u32x4 zero = {0, 0, 0, 0};
        if (kE4M3 && tile < cached_tiles) {
#pragma unroll
            for (uint32_t j = 0; j < kLoads8; ++j) {
                const uint32_t r = row_of_load8 + j * kRowStep8;
                u32x4 kx = kreg[j], vx = vreg[j];
                if (!whole && !(((counts >> r) & 1u) && chunk8 * 16 < dim)) kx = vx = zero;
                u32x4 k2[2], v2[2];
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    k2[i >> 1][2 * (i & 1)] = T::template from_e4m3<false>(kx[i]);
                    k2[i >> 1][2 * (i & 1) + 1] = T::template from_e4m3<true>(kx[i]);
                    v2[i >> 1][2 * (i & 1)] = T::template from_e4m3<false>(vx[i]);
                    v2[i >> 1][2 * (i & 1) + 1] = T::template from_e4m3<true>(vx[i]);
                }
                put(r, 2 * chunk8, k2[0], v2[0]);
                put(r, 2 * chunk8 + 1, k2[1], v2[1]);
            }
        } else {
            bool found = false;
#pragma unroll
            for (uint32_t j = 0; j < kLoads; ++j) {
                const uint32_t r = row_of_load + j * kRowStep;
                u32x4 kx = kreg[j], vx = vreg[j];
                if (!whole && !(((counts >> r) & 1u) && chunk * 8 < dim)) kx = vx = zero;
                if (tile >= cached_tiles)
                    found |= only_finite<T>(&vx);
                put(r, chunk, kx, vx);
            }
            if (found) odd = 1;
        }
    };
    auto wave_sync = [&]() {  // a wavefront's LDS operations keep their order
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    auto sync = [&]() {
        if (kRowWaves == 1) wave_sync();
        else __syncthreads();
    };

    const uint32_t rounds = last > first ? ceil_div(last - first, S::kGroups) : 0;
    uint32_t tile = first + group;
    uint64_t counts = 0, next_counts = 0;
    int32_t next_page = -1;
    if (rounds) {
        const int32_t page = tile < last ? page_of(tile) : -1;
        next_page = tile + S::kGroups < last ? page_of(tile + S::kGroups) : -1;
        if (tile < last) counts = locate(tile, page);
        sync();
        if (tile < last) load(tile);
        sync();
    }
    for (uint32_t round = 0; round < rounds; ++round, tile += S::kGroups) {
        const bool here = tile < last, more = tile + S::kGroups < last;
        if (here) store(tile, counts);
        if (more) next_counts = locate(tile + S::kGroups, next_page);
        sync();
        if (tile + 2 * S::kGroups < last) next_page = page_of(tile + 2 * S::kGroups);
        if (more) load(tile + S::kGroups);
        if (here) {
            const bool is_new = tile >= cached_tiles;
            f32x16 s;
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
            for (uint32_t c = 0; c < kDim / 16; ++c) {
                const uint32_t place = (n * S::kChunks + key_chunk<kDim>(n, 2 * c + hi)) * 16;
                const u32x4 qx = *reinterpret_cast<const u32x4*>(query_tile + place);
                const u32x4 kx = *reinterpret_cast<const u32x4*>(key_tile + place);
                s = T::mfma(kx, qx, s);
            }
            // which keys this lane's row sees
            uint64_t sees = counts;
            if (is_new)
                sees = sight.of_tile<kKeys>(static_cast<int32_t>((cached_tiles + new_tiles - 1 - tile) * kKeys));
            float factor = is_new ? new_scale : cached_scale;
            float grow = new_base<T, 1>(&s, sees, kFull, hi, &factor, &m, &l);
            uint32_t p[8];
            l += weights_of<T, 1>(&s, factor, m, &p);
            if (kE4M3 && is_new && !scaled) {
                grow *= value_scale;
                scaled = true;
            }
            if (!__all(grow == 1.f))
#pragma unroll
                for (uint32_t t = 0; t < S::kDTiles; ++t)
#pragma unroll
                    for (uint32_t i = 0; i < 16; ++i) o[t][i] *= grow;
            const uint32_t g = lane & 15u;
#pragma unroll
            for (uint32_t half = 0; half < 2; ++half) {
                const u32x4 px = {p[4 * half], p[4 * half + 1], p[4 * half + 2], p[4 * half + 3]};
                const uint32_t r = 16 * half + 4 * hi + (g >> 2);
#pragma unroll
                for (uint32_t dt = 0; dt < S::kDTiles; ++dt) {
                    const uint32_t d = 32 * dt + (lane & 16u) + 4 * (g & 3u);
                    typedef __attribute__((address_space(3))) s16x4 Lds;
                    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(
                        value_tile + (r * S::kChunks + value_chunk<kDim>(r, d / 8)) * 16 + (d & 4) * 2));
                    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(
                        value_tile + ((r + 8) * S::kChunks + value_chunk<kDim>(r + 8, d / 8)) * 16 +
                        (d & 4) * 2));
                    const uint2 a0 = __builtin_bit_cast(uint2, v0), a1 = __builtin_bit_cast(uint2, v1);
                    const u32x4 vx = {a0.x, a0.y, a1.x, a1.y};
                    o[dt] = T::mfma(vx, px, o[dt]);
                }
            }
        }
        counts = next_counts;
        sync();
    }
    l += __shfl_xor(l, 32, 64);
    if (kE4M3 && !scaled)
#pragma unroll
        for (uint32_t t = 0; t < S::kDTiles; ++t)
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) o[t][i] *= value_scale;

    // join the groups: each scales its part to the common maximum and adds
    // it to the first one's, a group after the other
    __syncthreads();
    if (hi == 0) {
        joined[w][n][0] = m;
        joined[w][n][1] = l;
    }
    __syncthreads();
    float m_all = kLowest, l_all = 0.f;
    for (uint32_t g = 0; g < S::kGroups; ++g) m_all = fmaxf(m_all, joined[g * kRowWaves + row_wave][n][0]);
    const float base = m_all == kLowest ? 0.f : m_all;
    for (uint32_t g = 0; g < S::kGroups; ++g)
        l_all += joined[g * kRowWaves + row_wave][n][1] *
                 __builtin_amdgcn_exp2f(joined[g * kRowWaves + row_wave][n][0] - base);
    const float part = __builtin_amdgcn_exp2f(m - base);
    // [row wave][element][lane]: every lane has the same elements in each group
    float* const sums = reinterpret_cast<float*>(tiles) + row_wave * (kDim / 2) * 64 + lane;
    static_assert(kRowWaves * kDim * 32 * 4 <= S::kBytes, "the sums fit where the tiles were");
    for (uint32_t g = 1; g < S::kGroups; ++g) {
        if (group == g)
#pragma unroll
            for (uint32_t t = 0; t < S::kDTiles; ++t)
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i) {
                    float* const x = sums + (16 * t + i) * 64;
                    *x = (g == 1 ? 0.f : *x) + o[t][i] * part;
                }
        __syncthreads();
    }
    if (group != 0) return;
#pragma unroll
    for (uint32_t t = 0; t < S::kDTiles; ++t)
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) o[t][i] = o[t][i] * part + sums[(16 * t + i) * 64];
    m = m_all;
    l = l_all;
    write_row<T, kDim, kKeys>(a, item, e, place, sight, odd, hi, o, m, l);
}

// ---------------------------------------------------------------------------
// The attention kernel for many rows
// ---------------------------------------------------------------------------

// kWaves wavefronts, four or eight, share every tile, 32 rows each, and the
// matrix instructions bound the work.  Tiles are brought to LDS without passing
// through registers, in two buffers each for keys and values; every wavefront
// brings its part of each tile, and one barrier a tile remains.  Eight
// wavefronts bring each tile once for 256 rows where two workgroups of four on
// the compute unit bring it twice, and turn to it at other times.  Operands are
// read from LDS a few products ahead (the compiler alone reads each where it is
// needed, and every product then waits for LDS).  8-bit tiles stay 8-bit in LDS
// and become operands as they are read.
//
// Four pieces of prompts (above) take 403 us, 734 TFLOP/s; a SIMD's matrix unit
// is busy 38 % of the time and its vector unit 44 %, seldom at once.  Taking the
// scores of the next tile ahead of the softmax needs more registers than there
// are (twice the time, spilled); two sets of wavefronts that take turns, one at
// the products while the other weighs, took 391 us where this took 388 and cost
// the other calls here 3 to 10 %.  The lambdas are inlined by force, which
// decides what stays in registers (64 trees of 32 tokens, heads of 256: 291 us
// for 310).  48 trees of 1 to 40 tokens over e4m3 take 111 us: 1.6 TB/s, 330
// TFLOP/s.
template <bool kE4M3, uint32_t kDim, uint32_t kWaves>
struct Wide {
    static constexpr uint32_t kKeys = kDim == 256 ? 32 : 64;
    static constexpr uint32_t kChunks = kDim / 8;     // 16-byte chunks of a 16-bit row
    static constexpr uint32_t kChunks8 = kDim / 16;   // and of an 8-bit row
    static constexpr uint32_t kOwnRows = kKeys / kWaves;   // rows that a wavefront brings
    static constexpr uint32_t kLoads = kOwnRows * kChunks / 64, kLoads8 = kOwnRows * kChunks8 / 64;
    static constexpr uint32_t kTileBytes = kKeys * kDim * 2;
    static constexpr uint32_t kSTiles = kKeys / 32, kDTiles = kDim / 32;
    static_assert(kLoads >= 1 && (!kE4M3 || kLoads8 >= 1), "every wavefront brings something");
};

// Where chunk c of an 8-bit row r lies in its row.
template <uint32_t kDim>
__device__ __forceinline__ uint32_t chunk_of_8(uint32_t r, uint32_t c) {
    return kDim == 64 ? c ^ ((r >> 2) & 3u) : kDim == 128 ? c ^ ((r >> 1) & 7u) : c ^ (r & 15u);
}

// What is read in place of rows that do not count.
__device__ uint4 zero_row[kRows];
static_assert(sizeof(zero_row) >= 2 * coop_pages::kMaxDim, "a row of zeros");

// Products in order, each one's operand read from LDS kAhead products before
// it; no read or product moves across another step.
constexpr uint32_t kAhead = 4;

template <uint32_t kProducts, class Read, class Multiply>
__device__ __forceinline__ void products(Read read, Multiply multiply) {
    u32x4 x[kAhead];
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) x[i] = read(i);
#pragma unroll
    for (uint32_t i = 0; i < kProducts; ++i) {
        __builtin_amdgcn_sched_barrier(0x6);  // (scalar and vector arithmetic may move)
        multiply(i, x[i % kAhead]);
        if (i + kAhead < kProducts) x[i % kAhead] = read(i + kAhead);
    }
    __builtin_amdgcn_sched_barrier(0x6);
}

struct Eight { static constexpr bool value = true; };   // bits of a tile's numbers
struct Sixteen { static constexpr bool value = false; };
struct Keys { static constexpr bool value = true; };     // what is brought
struct Values { static constexpr bool value = false; };

template <class T, bool kE4M3, uint32_t kDim, uint32_t kWaves>
__global__ __launch_bounds__(64 * kWaves, kDim == 256 ? 1 : 2) void tree_attention_wide_kernel(Args a) {
    using W = Wide<kE4M3, kDim, kWaves>;
    constexpr uint32_t kKeys = W::kKeys;
    constexpr uint64_t kFull = kKeys == 64 ? ~0ull : 0xffffffffull;
    __shared__ __align__(16) uint8_t keys0[W::kTileBytes], keys1[W::kTileBytes];
    __shared__ __align__(16) uint8_t values0[W::kTileBytes], values1[W::kTileBytes];
    __shared__ int32_t tree[kParentsInLds];
    __shared__ uint32_t odd;

    const uint32_t tid = threadIdx.x, lane = tid & 63u;
    Item item;
    Extent e;
    if (!take_item(a, &item, &e)) return;
    const uint32_t w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t n = lane & 31u, hi = lane >> 5;
    const uint32_t dim = static_cast<uint32_t>(a.cache.dim);
    const uint32_t page_size = static_cast<uint32_t>(a.cache.page_size);
    auto page_at = [&](uint32_t pos) { return a.page_shift < 32 ? pos >> a.page_shift : pos / page_size; };
    const Place place = place_of<kKeys>(a, item, e, w * kRows + n);
    const uint32_t cached_tiles = place.cached_tiles, all_tiles = place.cached_tiles + place.new_tiles;
    const uint32_t first = place.first, last = place.last;

    const uint64_t size = kE4M3 ? 1 : 2;
    const Global ck = (Global)(a.cache.k) + item.head * a.cache.k_stride[2] * size;
    const Global cv = (Global)(a.cache.v) + item.head * a.cache.v_stride[2] * size;
    const Global nk = (Global)(a.k.data) + (e.first * a.k.stride[0] + item.head * a.k.stride[1]) * 2;
    const Global nv = (Global)(a.v.data) + (e.first * a.v.stride[0] + item.head * a.v.stride[1]) * 2;
    const Global zeros = (Global)(&zero_row[0]);

    // A lane knows where the rows of the tile's key lane % kKeys are, as offsets
    // from the tile's base; kNowhere: a row that does not count.
    constexpr uint64_t kNowhere = ~0ull;
    const uint32_t my_key = lane % kKeys;
    const uint32_t table_end = min(cached_tiles, last) * kKeys < e.cached ? min(cached_tiles, last) * kKeys : e.cached;
    const int32_t* const table = a.table + static_cast<uint64_t>(item.request) * a.max_pages;
    auto page_of = [&](uint32_t tile) __attribute__((always_inline)) -> int32_t {
        const uint32_t pos = tile * kKeys + my_key;
        return pos < table_end ? table[page_at(pos)] : -1;
    };
    struct Where {
        uint64_t k, v;
        uint64_t counts;  // which of the tile's keys count
    };
    auto locate = [&](uint32_t tile, int32_t page) __attribute__((always_inline)) {
        Where r = {kNowhere, kNowhere, 0};
        if (tile < cached_tiles) {
            const uint32_t pos = tile * kKeys + my_key;
            if (static_cast<uint32_t>(page) < static_cast<uint32_t>(a.cache.num_pages)) {
                const uint32_t in_page = pos - page_at(pos) * page_size, p = static_cast<uint32_t>(page);
                if (a.narrow) {
                    r.k = static_cast<uint64_t>(p) * a.page_bytes + in_page * a.place_bytes;
                    r.v = r.k;
                } else {
                    r.k = (p * a.cache.k_stride[0] + in_page * a.cache.k_stride[1]) * size;
                    r.v = (p * a.cache.v_stride[0] + in_page * a.cache.v_stride[1]) * size;
                }
            }
        } else {
            const uint32_t j = (all_tiles - 1 - tile) * kKeys + my_key;
            if (tile < last && j < e.tokens) {
                r.k = j * a.k.stride[0] * 2;
                r.v = j * a.v.stride[0] * 2;
            }
        }
        const uint64_t all = __ballot(r.k != kNowhere);
        r.counts = kKeys == 64 ? all : all & 0xffffffffu;
        return r;
    };
    auto from = [&](uint64_t v, uint32_t r) __attribute__((always_inline)) -> uint64_t {
        return static_cast<uint64_t>(__shfl(static_cast<uint32_t>(v), r, 64)) |
               static_cast<uint64_t>(__shfl(static_cast<uint32_t>(v >> 32), r, 64)) << 32;
    };
    auto fetch = [](Global p, uint8_t* to) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                         (__attribute__((address_space(3))) void*)to, 16, 0, 0);
    };
    // Brings this wavefront's rows of a tile's keys or values: lane by lane to
    // consecutive chunks of LDS, so each lane fetches the chunk whose place that
    // is.
    auto bring = [&](uint32_t tile, uint64_t offset, uint64_t counts, Global cache_base, Global new_base,
                     uint8_t* to, auto of_keys) __attribute__((always_inline)) {
        if (tile >= last) return;
        const bool cached = tile < cached_tiles;
        const bool plain = dim == kDim && counts == kFull;  // nothing is zeroed
        const Global base = cached ? cache_base : new_base;
        auto row_of = [&](uint32_t r) {
            const uint64_t at = from(offset, r);
            return !plain && at == kNowhere ? zeros : base + at;
        };
        if (kE4M3 && cached) {
#pragma unroll
            for (uint32_t j = 0; j < W::kLoads8; ++j) {
                const uint32_t slot = j * 64 + lane, r = w * W::kOwnRows + slot / W::kChunks8;
                const uint32_t c = chunk_of_8<kDim>(r, slot % W::kChunks8) * 16;
                const Global row = row_of(r);
                fetch(plain || c < dim ? row + c : zeros, to + (w * W::kOwnRows * W::kChunks8 + j * 64) * 16);
            }
        } else {
#pragma unroll
            for (uint32_t j = 0; j < W::kLoads; ++j) {
                const uint32_t slot = j * 64 + lane, r = w * W::kOwnRows + slot / W::kChunks;
                const uint32_t c = (decltype(of_keys)::value ? key_chunk<kDim>(r, slot % W::kChunks)
                                                             : value_chunk<kDim>(r, slot % W::kChunks)) * 16;
                const Global row = row_of(r);
                fetch(plain || c < 2 * dim ? row + c : zeros, to + (w * W::kOwnRows * W::kChunks + j * 64) * 16);
            }
        }
    };
    auto bring_keys = [&](uint32_t tile, const Where& at, uint8_t* to) __attribute__((always_inline)) {
        bring(tile, at.k, at.counts, ck, nk, to, Keys());
    };
    auto bring_values = [&](uint32_t tile, const Where& at, uint8_t* to) __attribute__((always_inline)) {
        bring(tile, at.v, at.counts, cv, nv, to, Values());
    };
    // Takes out of this wavefront's rows of new values what is not finite.
    auto clean = [&](uint8_t* values) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t j = 0; j < W::kLoads; ++j) {
            u32x4* const p = reinterpret_cast<u32x4*>(values) + w * W::kOwnRows * W::kChunks + j * 64 + lane;
            u32x4 x = *p;
            if (only_finite<T>(&x)) {
                *p = x;
                odd = 1;
            }
        }
    };
    auto arrived = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): what this wavefront brings is there
        asm volatile("" ::: "memory");
    };

    // the first tile's rows are on their way before anything else is
    const int32_t first_page = page_of(first), second_page = page_of(first + 1);
    int32_t page = page_of(first + 2);
    Where now = locate(first, first_page);  // of the tile that is next
    bring_keys(first, now, keys0);
    bring_values(first, now, values0);

    Sight sight;
    sight.parents = a.parents ? a.parents + e.first : nullptr;
    sight.tree = tree;
    sight.in_lds = a.parents && e.tokens <= kParentsInLds && last > cached_tiles;
    sight.token = place.lives && last > cached_tiles ? static_cast<int32_t>(place.token) : -1;
    if (sight.in_lds)
        for (uint32_t i = tid; i < e.tokens; i += 64 * kWaves) tree[i] = sight.parents[i];
    if (tid == 0) odd = 0;
    u32x4 q[kDim / 16];
    {
        const uint16_t* const base = static_cast<const uint16_t*>(a.q.data) +
                                     (e.first + place.token) * a.q.stride[0] + place.q_head * a.q.stride[1];
#pragma unroll
        for (uint32_t c = 0; c < kDim / 16; ++c) {
            const uint32_t d = 16 * c + 8 * hi;
            q[c] = u32x4{0, 0, 0, 0};
            if (place.lives && d < dim) q[c] = *reinterpret_cast<const u32x4*>(base + d);
        }
    }
    Where next = locate(first + 1, second_page);
    f32x16 o[W::kDTiles];
#pragma unroll
    for (uint32_t t = 0; t < W::kDTiles; ++t)
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = kLowest, l = 0.f;
    const float new_scale = a.scale * kLog2e;
    const float cached_scale = kE4M3 ? new_scale * a.cache.k_scale[item.head] : new_scale;
    const float value_scale = kE4M3 ? a.cache.v_scale[item.head] : 1.f;
    bool scaled = false;  // whether o has met the cached values' scale
    // a wavefront without rows brings its part of the tiles and does nothing else
    const bool works = __ballot(place.lives) != 0;

    // an operand as it is read, and as products take it
    auto operand = [](u32x4 x, auto width) -> u32x4 {
        if constexpr (decltype(width)::value)
            return {T::template from_e4m3<false>(x[0]), T::template from_e4m3<true>(x[0]),
                    T::template from_e4m3<false>(x[1]), T::template from_e4m3<true>(x[1])};
        else
            return x;
    };
    // the products of a tile's keys with the rows' queries
    auto scores = [&](const uint8_t* __restrict__ keys, f32x16* to, auto width) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t t = 0; t < W::kSTiles; ++t)
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) to[t][i] = 0.f;
        products<kDim / 16 * W::kSTiles>(
            [&](uint32_t i) -> u32x4 {
                const uint32_t c = i / W::kSTiles, r = 32 * (i % W::kSTiles) + n;
                if constexpr (decltype(width)::value) {
                    const uint2 x = *reinterpret_cast<const uint2*>(
                        keys + (r * W::kChunks8 + chunk_of_8<kDim>(r, c)) * 16 + hi * 8);
                    return {x.x, x.y, 0, 0};
                } else {
                    return *reinterpret_cast<const u32x4*>(
                        keys + (r * W::kChunks + key_chunk<kDim>(r, 2 * c + hi)) * 16);
                }
            },
            [&](uint32_t i, u32x4 x) {
                const uint32_t t = i % W::kSTiles;
                to[t] = T::mfma(operand(x, width), q[i / W::kSTiles], to[t]);
            });
    };
    // Where a lane's four values of each 32 columns are, in a tile's first 16 keys
    // (rows 16 apart are permuted alike).  Sums that the compiler takes apart
    // grow into chains whose array it no longer knows, and a read of that waits
    // for everything on its way to LDS.
    uint32_t value_at[W::kDTiles];
#pragma unroll
    for (uint32_t dt = 0; dt < W::kDTiles; ++dt) {
        const uint32_t g = lane & 15u, r = 4 * hi + (g >> 2), d = 32 * dt + (lane & 16u) + 4 * (g & 3u);
        value_at[dt] = (r * W::kChunks + value_chunk<kDim>(r, d / 8)) * 16 + (d & 4) * 2;
        asm volatile("" : "+v"(value_at[dt]));
    }
    // adds a tile's values by their weights
    auto add = [&](const uint8_t* __restrict__ values, uint32_t (*p)[8], auto width) __attribute__((always_inline)) {
        const uint32_t g = lane & 15u;
        products<2 * W::kSTiles * W::kDTiles>(
            [&](uint32_t i) -> u32x4 {
                const uint32_t dt = i % W::kDTiles;
                if constexpr (decltype(width)::value) {
                    const uint32_t r0 = 16 * (i / W::kDTiles) + 4 * hi;
                    // eight rows of 16 columns: keys 0..3 and 8..11 of the lane's half
                    typedef int i32x2 __attribute__((ext_vector_type(2)));
                    typedef __attribute__((address_space(3))) i32x2 Two;
                    const uint32_t r = r0 + ((g >> 1) & 3u) + (g & 8u), c = 2 * dt + ((lane >> 4) & 1u);
                    const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                        (Two*)(values + (r * W::kChunks8 + chunk_of_8<kDim>(r, c)) * 16 + (g & 1u) * 8));
                    return {static_cast<uint32_t>(x[0]), static_cast<uint32_t>(x[1]), 0, 0};
                } else {
                    typedef __attribute__((address_space(3))) s16x4 Four;
                    const uint8_t* const at = values + (value_at[dt] + 16 * (i / W::kDTiles) * kDim * 2);
                    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four*)at);
                    // (rows eight apart are permuted alike)
                    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four*)(at + 8 * kDim * 2));
                    const uint2 a0 = __builtin_bit_cast(uint2, v0), a1 = __builtin_bit_cast(uint2, v1);
                    return {a0.x, a0.y, a1.x, a1.y};
                }
            },
            [&](uint32_t i, u32x4 x) {
                const uint32_t dt = i % W::kDTiles, t = i / W::kDTiles / 2, half = i / W::kDTiles % 2;
                const u32x4 px = {p[t][4 * half], p[t][4 * half + 1], p[t][4 * half + 2], p[t][4 * half + 3]};
                o[dt] = T::mfma(operand(x, width), px, o[dt]);
            });
    };
    // The weights of a tile's scores; moves the sums' base.
    auto weigh = [&](uint32_t tile, uint64_t counts, f32x16* s, uint32_t (*p)[8], auto width) __attribute__((always_inline)) {
        constexpr bool kNew = kE4M3 && !decltype(width)::value;  // (a 16-bit tile of an 8-bit cache's call)
        const bool is_new = kNew || tile >= cached_tiles;
        uint64_t sees = counts;
        if (is_new) sees = sight.of_tile<kKeys>(static_cast<int32_t>((all_tiles - 1 - tile) * kKeys));
        float factor = is_new ? new_scale : cached_scale;
        float grow = new_base<T, W::kSTiles>(s, sees, kFull, hi, &factor, &m, &l);
        if (kNew && !scaled) {
            grow *= value_scale;
            scaled = true;
        }
        if (!__all(grow == 1.f))
#pragma unroll
            for (uint32_t t = 0; t < W::kDTiles; ++t)
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i) o[t][i] *= grow;
        l += weights_of<T, W::kSTiles>(s, factor, m, p);
    };
    // The page's number is there as all that was brought is.  Said ahead of what
    // is brought next: a wait for it later would be one for that too.
    auto located = [&](uint32_t tile) __attribute__((always_inline)) {
        asm volatile("" : "+v"(page));
        return locate(tile, page);
    };
    // A tile, on its way to `keys` and `values`.
    auto step = [&](uint32_t tile, auto width, uint8_t* __restrict__ keys, uint8_t* __restrict__ values,
                    uint8_t* __restrict__ keys_to, uint8_t* __restrict__ values_to) __attribute__((always_inline)) {
        arrived();
        if ((kE4M3 && !decltype(width)::value) || tile >= cached_tiles) clean(values);
        __syncthreads();
        const uint64_t counts = now.counts;
        const Where after = located(tile + 2);
        bring_keys(tile + 1, next, keys_to);
        bring_values(tile + 1, next, values_to);
        now = next;
        next = after;
        page = page_of(tile + 3);
        if (!works) return;
        f32x16 s[W::kSTiles];
        uint32_t p[W::kSTiles][8];
        scores(keys, s, width);
        weigh(tile, counts, s, p, width);
        add(values, p, width);
    };
    __syncthreads();  // (the tree, and that no value is odd yet)
    sight.start();
    uint32_t tile = first;
    if constexpr (kE4M3) {
        const uint32_t end = min(last, cached_tiles);
        for (; tile + 1 < end; tile += 2) {
            step(tile, Eight(), keys0, values0, keys1, values1);
            step(tile + 1, Eight(), keys1, values1, keys0, values0);
        }
        if (tile < end) {  // (an odd number: the buffers' parts are exchanged)
            step(tile++, Eight(), keys0, values0, keys1, values1);
            if (tile < last) step(tile++, Sixteen(), keys1, values1, keys0, values0);
        }
    }
    for (; tile < last; tile += 2) {
        step(tile, Sixteen(), keys0, values0, keys1, values1);
        if (tile + 1 < last) step(tile + 1, Sixteen(), keys1, values1, keys0, values0);
    }
    l += __shfl_xor(l, 32, 64);
    if (kE4M3 && !scaled)
#pragma unroll
        for (uint32_t t = 0; t < W::kDTiles; ++t)
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) o[t][i] *= value_scale;
    write_row<T, kDim, kKeys>(a, item, e, place, sight, odd, hi, o, m, l);
}

// Joins the parts of rows whose keys were cut.  A row's parts are dealt to
// kWaves wavefronts: four (a workgroup a row) where there are few rows and so
// many parts, one where there are many rows.  Reading the parts bounds it (19
// us of the 113 for 16 trees of 64 tokens, 66 MB; 4 us for four short
// sequences).  With four or one wavefront a row, the whole call: one token over
// 16000 cached ones 24.4 : 26.3 us, 16 trees of 64 137 : 114.
template <class T, uint32_t kDim, uint32_t kWaves>
__global__ __launch_bounds__(kThreads) void attention_join_kernel(Args a) {
    constexpr uint32_t kEach = kDim / 64, kRowsAtOnce = 4 / kWaves;
    __shared__ float sums[4][kDim + 64];
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool few = a.requests <= 64;
    LanePlan plan;
    if (few) plan = lane_plan(a, lane);
    const uint64_t joins = few ? from_lane(plan.joins, 63) : a.head->joins;
    const uint32_t dim = static_cast<uint32_t>(a.cache.dim);
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * kRowsAtOnce + (kWaves == 1 ? w : 0);
         i < joins * a.part_rows; i += static_cast<uint64_t>(gridDim.x) * kRowsAtOnce) {
        const uint32_t pair = static_cast<uint32_t>(i / a.part_rows);
        const uint32_t r = static_cast<uint32_t>(i - static_cast<uint64_t>(pair) * a.part_rows);
        Join j;
        Extent e;
        if (few) {
            join_of(a, plan, pair, &j, &e);
        } else {
            j = a.joins[pair];
            e = extent(a, j.request);
        }
        const uint32_t row = j.row_tile * a.row_tile_rows + r;
        if (row >= e.tokens * a.group) continue;
        const uint32_t token = row / a.group, qh = j.head * a.group + row % a.group;
        const float2* const part_sum = a.part_sum + static_cast<uint64_t>(j.first) * a.part_rows + r;
        const float* const part_out =
            a.part_out + (static_cast<uint64_t>(j.first) * a.part_rows + r) * kDim + lane * kEach;
        float m = kLowest;
        for (uint32_t p = lane; p < j.parts; p += 64) m = fmaxf(m, part_sum[static_cast<uint64_t>(p) * a.part_rows].x);
        for (uint32_t d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
        const float base = m == kLowest ? 0.f : m;
        float l = 0.f, o[kEach];
#pragma unroll
        for (uint32_t c = 0; c < kEach; ++c) o[c] = 0.f;
#pragma unroll 4
        for (uint32_t p = kWaves == 1 ? 0 : w; p < j.parts; p += kWaves) {
            const float2 ml = part_sum[static_cast<uint64_t>(p) * a.part_rows];
            const float x = __builtin_amdgcn_exp2f(ml.x - base);
            l += ml.y * x;
#pragma unroll
            for (uint32_t c = 0; c < kEach; ++c)
                o[c] += part_out[static_cast<uint64_t>(p) * a.part_rows * kDim + c] * x;
        }
        if (kWaves > 1) {
#pragma unroll
            for (uint32_t c = 0; c < kEach; ++c) sums[w][lane * kEach + c] = o[c];
            if (lane == 0) sums[w][kDim] = l;
            __syncthreads();
#pragma unroll
            for (uint32_t c = 0; c < kEach; ++c) {
                const uint32_t d = lane * kEach + c;
                o[c] = (sums[0][d] + sums[1][d]) + (sums[2][d] + sums[3][d]);
            }
            l = (sums[0][kDim] + sums[1][kDim]) + (sums[2][kDim] + sums[3][kDim]);
            __syncthreads();
            if (w) continue;
        }
        bool is_void = false;
        if (a.parents) {
            const int32_t p = a.parents[e.first + token];
            is_void = p < -1 || p >= static_cast<int32_t>(token);
        }
        uint16_t* const to = a.out + ((e.first + token) * a.q_heads + qh) * dim;
#pragma unroll
        for (uint32_t c = 0; c < kEach; ++c)
            if (lane * kEach + c < dim)
                to[lane * kEach + c] =
                    static_cast<uint16_t>(is_void ? 0u : T::pack(o[c] / l, 0.f) & 0xffffu);
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

constexpr uint64_t kMost = (1ull << 31) - 1;

// (a launch has fewer than 2^32 threads, 256 an item)
constexpr uint64_t kMostRows = 1ull << 28, kMostPairs = 1ull << 22;

bool counts_valid(uint64_t requests, uint64_t tokens, uint64_t q_heads, uint64_t heads,
                  uint64_t dim) {
    return heads && heads <= coop_pages::kMaxHeads && q_heads && q_heads <= coop_pages::kMaxHeads &&
           q_heads % heads == 0 && requests < kMost && tokens <= kMost &&
           tokens * q_heads <= kMostRows && requests * heads <= kMostPairs && dim &&
           dim <= coop_pages::kMaxDim && dim % 8 == 0;
}

struct Plan {
    uint32_t dim;        // padded
    uint32_t row_waves;
    uint32_t tile_keys;
    uint32_t slots;
    uint32_t most_parts;
    uint32_t part_rows;
    uint64_t max_items, pairs;
    size_t items_offset, joins_offset, sum_offset, out_offset, bytes;
};

// The wavefronts that share every tile of keys, 32 rows each: as many as the
// rows of an average request fill.  The lengths are on the device, the average
// is all that the host knows of them.  A batch of unlike requests has the
// average's tiles for all: 255 single tokens over 500 to 4000 with a piece of
// 2048 over 2000 (36 rows on average, two wavefronts) take 605 us, the two as
// calls of their own 362 and 153; 63 over 500 to 16000 with a piece of 1024 (68
// rows, four) 315 us, apart 233 and 81.
//
// Measured with 64 requests of 200 to 4000 cached tokens, 32 query heads over 8
// of 128 dims in bf16 (us, the fewer wavefronts first):
//   1 or 2:   48 rows 128 : 105,    64 rows 129 : 106,    24 rows   - : 92
//   2 or 4:   48 rows 105 : 110,    64 rows 106 : 112,    96 rows 166 : 117
//   4 or 8:  128 rows 123 : 180,   160 rows 190 : 178,   256 rows 200 : 193,
//            320 rows 273 : 316,   384 rows 287 : 325
// and with 32, 16 or 8 requests
//   4 or 8:  512 rows 197 : 183,   640 rows 242 : 251,   896 rows 318 : 309,
//           2048 rows of one prompt 348 : 315,  4096 rows of one prompt 411 : 365.
// So eight wavefronts pay where the rows are no more than four would be given
// (an even number of fours), or are so many that the last tile weighs little.
// They do not for e4m3, whose values the matrix instructions take only after
// a conversion that every wavefront makes for itself (256 rows 190 : 196, one
// prompt of 2048 rows 329 : 328), nor for 64 dims, where a tile is half the
// work between two barriers (256 rows 113 : 132, one prompt of 2048 rows
// 203 : 221); with 256 dims the sums of two wavefronts a SIMD do not fit the
// registers.
uint32_t row_waves_of(uint64_t mean, uint32_t dim, bool e4m3) {
    if (mean <= 32) return 1;
    if (mean <= 64) return 2;
    const uint64_t fours = (mean + 4 * kRows - 1) / (4 * kRows);
    return dim == 128 && !e4m3 && (fours % 2 == 0 || fours > 6) ? 8 : 4;
}

Plan plan_of(uint64_t requests, uint64_t tokens, uint64_t q_heads, uint64_t heads, uint64_t dim,
             bool e4m3) {
    Plan p;
    p.dim = dim <= 64 ? 64 : dim <= 128 ? 128 : 256;
    const uint64_t group = q_heads / heads, rows = tokens * group;
    p.row_waves = row_waves_of(requests ? (rows + requests - 1) / requests : 0, p.dim, e4m3);
    p.tile_keys = p.row_waves >= 4 && p.dim != 256 ? 64 : 32;
    // workgroups that 256 compute units hold at once (by registers and LDS)
    p.slots = (p.dim == 256 ? 256 : 512) / (p.row_waves == 8 ? 2 : 1);
    const uint64_t tile_rows = kRows * p.row_waves;
    p.part_rows = static_cast<uint32_t>(rows < tile_rows ? rows : tile_rows);
    p.pairs = heads * ((rows + tile_rows - 1) / tile_rows + requests);
    p.most_parts = 4 * p.slots + 8;  // (a few more than the plan's lengths allow, which are rounded)
    p.max_items = p.most_parts + p.pairs;
    auto next = [](size_t x) { return (x + 255) & ~static_cast<size_t>(255); };
    p.items_offset = 256;
    p.joins_offset = next(p.items_offset + p.max_items * sizeof(Item));
    p.sum_offset = next(p.joins_offset + p.most_parts / 2 * sizeof(Join));
    p.out_offset = next(p.sum_offset + 1ull * p.most_parts * p.part_rows * sizeof(float2));
    p.bytes = p.out_offset + 1ull * p.most_parts * p.part_rows * p.dim * sizeof(float);
    return p;
}

template <class T, bool kE4M3, uint32_t kDim>
void launch(const Plan& p, const Args& a, uint32_t joins, hipStream_t s) {
    constexpr uint32_t kMost8 = kDim == 128 && !kE4M3 ? 8 : 4;  // (others are not built)
    auto kernel = p.row_waves == 1   ? tree_attention_kernel<T, kE4M3, kDim, 1>
                  : p.row_waves == 2 ? tree_attention_kernel<T, kE4M3, kDim, 2>
                  : p.row_waves == 4 ? tree_attention_wide_kernel<T, kE4M3, kDim, 4>
                                     : tree_attention_wide_kernel<T, kE4M3, kDim, kMost8>;
    hipLaunchKernelGGL(kernel, dim3(a.max_items), dim3(p.row_waves == 8 ? 512 : kThreads), 0, s, a);
    if (joins) {
        // the rows of all pairs: no more than a workgroup each keeps busy, or more
        auto join = p.pairs * p.part_rows <= 1024 ? attention_join_kernel<T, kDim, 4>
                                                  : attention_join_kernel<T, kDim, 1>;
        hipLaunchKernelGGL(join, dim3(joins), dim3(kThreads), 0, s, a);
    }
}

template <class T, bool kE4M3>
void launch_dim(const Plan& p, const Args& a, uint32_t joins, hipStream_t s) {
    if (p.dim == 64) launch<T, kE4M3, 64>(p, a, joins, s);
    else if (p.dim == 128) launch<T, kE4M3, 128>(p, a, joins, s);
    else launch<T, kE4M3, 256>(p, a, joins, s);
}

}  // namespace

extern "C" {

coop_status_t coop_tree_attention_workspace_size(uint64_t num_requests, uint64_t num_tokens,
                                                 uint64_t q_heads, uint64_t heads, uint64_t dim,
                                                 size_t* bytes_out) {
    if (!bytes_out || !counts_valid(num_requests, num_tokens, q_heads, heads, dim))
        return COOP_ERR_INVALID;
    // (the pool's type, which the plan depends on, is not asked for here)
    size_t bytes = 0;
    if (num_requests && num_tokens)
        for (const bool e4m3 : {false, true}) {
            const Plan p = plan_of(num_requests, num_tokens, q_heads, heads, dim, e4m3);
            bytes = p.bytes > bytes ? p.bytes : bytes;
        }
    *bytes_out = bytes;
    return COOP_OK;
}

coop_status_t coop_tree_attention(const coop_rows_t* q, const coop_rows_t* k_new,
                                  const coop_rows_t* v_new, int32_t type, uint64_t q_heads,
                                  uint64_t num_tokens, const uint64_t* token_offsets,
                                  const int32_t* parents, const coop_cache_t* cache,
                                  const int32_t* table, uint64_t max_pages,
                                  const uint64_t* lengths, uint64_t num_requests, float scale,
                                  void* out, void* workspace, size_t workspace_bytes,
                                  void* stream) {
    if (!q || !k_new || !v_new || !cache) return COOP_ERR_INVALID;
    if (const coop_status_t rc = coop_pages::check_cache(*cache, type)) return rc;
    if (!counts_valid(num_requests, num_tokens, q_heads, cache->heads, cache->dim) ||
        max_pages > kMost || max_pages * cache->page_size > kMost)
        return COOP_ERR_INVALID;
    if (num_tokens == 0) return COOP_OK;
    if (!coop_pages::rows_valid(*q, num_tokens, q_heads, cache->dim) ||
        !coop_pages::rows_valid(*k_new, num_tokens, cache->heads, cache->dim) ||
        !coop_pages::rows_valid(*v_new, num_tokens, cache->heads, cache->dim))
        return COOP_ERR_INVALID;
    if (!out || !coop_pages::aligned16(out) || !token_offsets) return COOP_ERR_INVALID;
    if (num_requests == 0) return COOP_OK;
    if (!lengths || (max_pages && !table)) return COOP_ERR_INVALID;
    const Plan p = plan_of(num_requests, num_tokens, q_heads, cache->heads, cache->dim,
                           cache->type == COOP_E4M3);
    if (!workspace || workspace_bytes < p.bytes) return COOP_ERR_WORKSPACE;
    if (!coop_pages::aligned16(workspace)) return COOP_ERR_INVALID;
    Args a;
    a.q = *q;
    a.k = *k_new;
    a.v = *v_new;
    a.cache = *cache;
    a.offsets = token_offsets;
    a.parents = parents;
    a.table = table;
    a.lengths = lengths;
    a.out = static_cast<uint16_t*>(out);
    a.tokens = num_tokens;
    a.requests = static_cast<uint32_t>(num_requests);
    a.max_pages = static_cast<uint32_t>(max_pages);
    a.q_heads = static_cast<uint32_t>(q_heads);
    a.group = static_cast<uint32_t>(q_heads / cache->heads);
    a.page_shift = (cache->page_size & (cache->page_size - 1)) == 0
                       ? static_cast<uint32_t>(__builtin_ctzll(cache->page_size)) : 32u;
    const uint64_t size = cache->type == COOP_E4M3 ? 1 : 2;
    a.narrow = cache->k_stride[0] == cache->v_stride[0] && cache->k_stride[1] == cache->v_stride[1] &&
               cache->k_stride[0] * size < 1ull << 32 && cache->k_stride[1] * size < 1ull << 32 &&
               cache->k_stride[1] * size * cache->page_size < 1ull << 32;
    a.page_bytes = static_cast<uint32_t>(cache->k_stride[0] * size);
    a.place_bytes = static_cast<uint32_t>(cache->k_stride[1] * size);
    a.scale = scale;
    a.tile_keys = p.tile_keys;
    a.row_tile_rows = kRows * p.row_waves;
    a.slots = p.slots;
    a.least = 128 / p.tile_keys;
    a.least_more = 1024 / p.tile_keys;
    a.chunk_multiple = p.row_waves < 4 ? 4 / p.row_waves : 1;
    a.part_rows = p.part_rows;
    // the tiles that a pair can have at most, and the ranges that this allows
    const uint64_t tiles = (max_pages * cache->page_size + p.tile_keys - 1) / p.tile_keys +
                           (num_tokens + p.tile_keys - 1) / p.tile_keys;
    const unsigned __int128 most = static_cast<unsigned __int128>(p.pairs) * tiles / a.least + 1;
    const uint64_t cuts = 2 * most < p.most_parts ? static_cast<uint64_t>(2 * most) : p.most_parts;
    a.max_items = static_cast<uint32_t>(cuts + p.pairs);
    char* const ws = static_cast<char*>(workspace);
    a.head = reinterpret_cast<Head*>(ws);
    a.items = reinterpret_cast<Item*>(ws + p.items_offset);
    a.joins = reinterpret_cast<Join*>(ws + p.joins_offset);
    a.part_sum = reinterpret_cast<float2*>(ws + p.sum_offset);
    a.part_out = reinterpret_cast<float*>(ws + p.out_offset);
    // rows can be cut only if one can have more tiles than the shortest range
    const uint64_t join_rows = cuts / 2 * a.part_rows;
    const uint32_t joins = tiles > a.least ? static_cast<uint32_t>(join_rows < 2048 ? join_rows : 2048) : 0;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (num_requests > 64) {
        hipLaunchKernelGGL(attention_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
        if (hipGetLastError() != hipSuccess) return COOP_ERR_HIP;
    }
    const bool e4m3 = cache->type == COOP_E4M3;
    if (type == COOP_BF16) {
        if (e4m3) launch_dim<Bf16, true>(p, a, joins, s);
        else launch_dim<Bf16, false>(p, a, joins, s);
    } else {
        if (e4m3) launch_dim<Fp16, true>(p, a, joins, s);
        else launch_dim<Fp16, false>(p, a, joins, s);
    }
    return hipGetLastError() == hipSuccess ? COOP_OK : COOP_ERR_HIP;
}

}  // extern "C"
