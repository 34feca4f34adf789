// Paged pools: block tables, slot maps and cache writes for gfx950.
//
// coop_page_tables on a small pool is one launch.  Its first workgroup does
// what needs one view of the pool: free pages are bits in LDS, set where rows
// give pages back, counted, and handed out by rank.  The other workgroups move
// the table's entries that stay.  On a large pool, launches on the caller's
// stream:
//  1. copy: kind_out = kind (left out when the two are one array).
//  2. rows: every table entry is read once and written once: those a row keeps
//     as they are, the others as -1; the pages of entries that a row no longer
//     needs become free in kind_out.
//  3. count: the free pages of each tile of 4096 pages, and (one workgroup
//     more) the running sum of the pages that rows ask for.
//  4. take: the free page of rank r (over the tiles' counts) belongs to the
//     first row whose running sum exceeds r, if that sum is at most the number
//     of free pages: nothing is listed or sorted, each page finds its own row.
//
// What bounds it.  A small pool is a chain of some ten dependent steps of one
// workgroup: 6.5 us for 8 sequences on 406 pages, 18 us for 512 on 107 thousand
// (2.6 MB in all).  A large one is four launches, each with its start and its
// searches: 3.4, 8.0, 5.9 and 11.9 us for 4096 sequences on 772 thousand pages,
// where 21 MB are read and written, 4.2 us at the rate of a large copy.
//
// coop_slot_map and coop_cache_write are one launch each.

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "coop.h"
#include "coop_pages.h"

namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kTilePages = 4096;   // pages a workgroup counts or hands out
constexpr uint32_t kScanThreads = 1024;
constexpr uint32_t kMaxGrid = 1u << 16;
constexpr uint32_t kLaneTokens = 4, kWaveTokens = 64 * kLaneTokens;  // of the slot map

struct RowAsk {
    uint32_t first;  // entries that the row keeps
    uint32_t count;  // pages that it asks for
};

__device__ __forceinline__ uint32_t in_use(int32_t held, uint32_t cols) {
    return held <= 0 ? 0u : min(static_cast<uint32_t>(held), cols);
}

// Entries that a sequence of `length` tokens needs; `held` of them if they are
// more than a row has.
__device__ __forceinline__ uint32_t needed(uint64_t length, uint64_t page, uint32_t held,
                                           uint32_t cols, bool* wide) {
    const uint64_t n = length / page + (length % page != 0);
    *wide = n > cols;
    return *wide ? held : static_cast<uint32_t>(n);
}

__global__ __launch_bounds__(kThreads) void pages_copy_kernel(const uint8_t* __restrict__ in,
                                                              uint8_t* __restrict__ out,
                                                              uint32_t n) {
    const bool aligned = ((reinterpret_cast<uintptr_t>(in) | reinterpret_cast<uintptr_t>(out)) & 15u) == 0;
    for (uint64_t p = (blockIdx.x * kThreads + threadIdx.x) * 16ull; p < n; p += gridDim.x * kThreads * 16ull) {
        if (aligned && p + 16 <= n)
            *reinterpret_cast<uint4*>(out + p) = *reinterpret_cast<const uint4*>(in + p);
        else
            for (uint64_t i = p; i < min(p + 16, static_cast<uint64_t>(n)); ++i) out[i] = in[i];
    }
}

__global__ __launch_bounds__(kThreads) void pages_rows_kernel(
    const int32_t* table, const int32_t* held, const uint64_t* lengths, uint64_t page,
    uint32_t rows, uint32_t cols, uint32_t pages, int32_t* table_out, uint8_t* kind_out) {
    for (uint32_t b = blockIdx.x; b < rows; b += gridDim.x) {
        const uint32_t h = in_use(held[b], cols);
        bool wide;
        const uint32_t keep = min(h, needed(lengths[b], page, h, cols, &wide));
        const uint64_t base = static_cast<uint64_t>(b) * cols;
        for (uint32_t c = threadIdx.x; c < cols; c += kThreads) {
            int32_t e = -1;
            if (c < h) {
                e = table[base + c];
                if (c >= keep) {
                    if (static_cast<uint32_t>(e) < pages) kind_out[e] = COOP_FREE;
                    e = -1;
                }
            }
            table_out[base + c] = e;
        }
    }
}

__device__ __forceinline__ uint64_t scan64(uint64_t v, uint32_t lane) {
    for (uint32_t d = 1; d < 64; d <<= 1) {
        const uint64_t up = __shfl_up(v, d, 64);
        if (lane >= d) v += up;
    }
    return v;
}

constexpr uint32_t kRowsEach = 4;  // consecutive rows of a thread

__global__ __launch_bounds__(kScanThreads) void pages_count_kernel(
    const uint8_t* kind, uint32_t pages, uint32_t tiles, const int32_t* held,
    const uint64_t* lengths, uint64_t page, uint32_t rows, uint32_t cols,
    uint32_t* __restrict__ tile_free, uint64_t* __restrict__ upto, RowAsk* __restrict__ ask,
    uint32_t* status) {
    __shared__ uint64_t part[kScanThreads / 64];
    __shared__ uint32_t any_wide;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, w = tid >> 6;
    if (blockIdx.x > 0) {
        const uint32_t tile = blockIdx.x - 1, p0 = tile * kTilePages;
        uint32_t n = 0;
        for (uint32_t i = tid; i < kTilePages; i += kScanThreads)
            n += p0 + i < pages && kind[p0 + i] == COOP_FREE;
        for (uint32_t m = 32; m; m >>= 1) n += __shfl_xor(n, m, 64);
        if (lane == 0) part[w] = n;
        __syncthreads();
        if (tid == 0) {
            uint64_t s = 0;
            for (uint32_t i = 0; i < kScanThreads / 64; ++i) s += part[i];
            tile_free[tile] = static_cast<uint32_t>(s);
        }
        return;
    }
    // the first workgroup: the rows' running sum
    if (tid == 0) any_wide = 0;
    uint64_t carry = 0;
    for (uint64_t b0 = 0; b0 < rows; b0 += kScanThreads * kRowsEach) {
        const uint64_t b = b0 + tid * kRowsEach;
        uint32_t first[kRowsEach], count[kRowsEach];
        uint64_t mine = 0;
        bool any = false;
#pragma unroll
        for (uint32_t i = 0; i < kRowsEach; ++i) {
            first[i] = count[i] = 0;
            if (b + i < rows) {
                const uint32_t h = in_use(held[b + i], cols);
                bool wide;
                const uint32_t need = needed(lengths[b + i], page, h, cols, &wide);
                any |= wide;
                first[i] = min(h, need);
                count[i] = need > h ? need - h : 0;
                mine += count[i];
            }
        }
        const uint64_t sum = scan64(mine, lane);
        __syncthreads();
        if (any) any_wide = 1;
        if (lane == 63) part[w] = sum;
        __syncthreads();
        uint64_t at = carry + sum - mine;
        for (uint32_t i = 0; i < kScanThreads / 64; ++i) {
            if (i < w) at += part[i];
            carry += part[i];
        }
#pragma unroll
        for (uint32_t i = 0; i < kRowsEach; ++i) {
            at += count[i];
            if (b + i < rows) {
                upto[b + i] = at;
                ask[b + i] = {first[i], count[i]};
            }
        }
    }
    __syncthreads();
    if (tid == 0) *status = any_wide ? 2u : 0u;
}

// For each of kCount values t, the first i in [0, n) with v[i] > t (v never
// decreases), n if there is none: a wavefront tries 64 places at a time, for
// all the values at once, so that their loads do not wait for one another.
template <uint32_t kCount>
__device__ __forceinline__ void first_past(const uint64_t* __restrict__ v, uint32_t n, const uint64_t* t,
                                           uint32_t lane, uint32_t* found) {
    uint32_t lo[kCount], hi[kCount];  // v[i] > t for i >= hi, not for i < lo
#pragma unroll
    for (uint32_t k = 0; k < kCount; ++k) {
        lo[k] = 0;
        hi[k] = n;
    }
    // (all intervals shrink alike: 64-fold, to a step of the one before)
    for (uint64_t size = n; size > 64;) {
        const uint32_t step = static_cast<uint32_t>((size + 63) >> 6);
        uint64_t m[kCount];
#pragma unroll
        for (uint32_t k = 0; k < kCount; ++k) {
            const uint64_t i = lo[k] + static_cast<uint64_t>(lane) * step;
            m[k] = __ballot(i >= hi[k] || v[i] > t[k]);
        }
#pragma unroll
        for (uint32_t k = 0; k < kCount; ++k) {
            const uint32_t f = m[k] ? static_cast<uint32_t>(__builtin_ctzll(m[k])) : 64u;
            const uint64_t end = lo[k] + static_cast<uint64_t>(f) * step;
            lo[k] = f ? lo[k] + (f - 1) * step + 1 : lo[k];
            hi[k] = end < hi[k] ? static_cast<uint32_t>(end) : hi[k];
        }
        size = step;
    }
    uint64_t m[kCount];
#pragma unroll
    for (uint32_t k = 0; k < kCount; ++k) {
        const uint64_t i = static_cast<uint64_t>(lo[k]) + lane;
        m[k] = __ballot(i >= hi[k] || v[i] > t[k]);
    }
#pragma unroll
    for (uint32_t k = 0; k < kCount; ++k)
        found[k] = m[k] ? min(lo[k] + static_cast<uint32_t>(__builtin_ctzll(m[k])), hi[k]) : hi[k];
}

// The same for one lane, known to lie in [lo, hi].
__device__ __forceinline__ uint32_t first_past_between(const uint64_t* __restrict__ v, uint32_t lo,
                                                       uint32_t hi, uint64_t t) {
    while (lo < hi) {
        const uint32_t mid = lo + ((hi - lo) >> 1);
        if (v[mid] > t) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

__global__ __launch_bounds__(kScanThreads) void pages_take_kernel(
    uint8_t* kind, uint32_t pages, uint32_t tiles, const uint32_t* __restrict__ tile_free,
    const uint64_t* __restrict__ upto, const RowAsk* __restrict__ ask, uint32_t rows, uint32_t cols,
    uint8_t taken, int32_t* table_out, int32_t* held_out, uint32_t* status, uint64_t* free_pages) {
    __shared__ uint64_t part[2][kScanThreads / 64];
    __shared__ uint32_t wave_free[kScanThreads / 64];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, w = tid >> 6;
    // free pages in all, and before this tile
    uint64_t all = 0, before = 0;
    for (uint32_t i = tid; i < tiles; i += kScanThreads) {
        const uint32_t n = tile_free[i];
        all += n;
        before += i < blockIdx.x ? n : 0u;
    }
    constexpr uint32_t kEach = kTilePages / kScanThreads;  // consecutive pages of a thread
    const uint32_t p0 = blockIdx.x * kTilePages + tid * kEach;
    uint32_t is_free = 0;
    if (blockIdx.x < tiles)
        for (uint32_t i = 0; i < kEach; ++i)
            if (p0 + i < pages && kind[p0 + i] == COOP_FREE) is_free |= 1u << i;
    const uint32_t own = __popc(is_free);
    const uint32_t sum = static_cast<uint32_t>(scan64(own, lane));
    for (uint32_t m = 32; m; m >>= 1) {
        all += __shfl_xor(all, m, 64);
        before += __shfl_xor(before, m, 64);
    }
    if (lane == 63) {
        part[0][w] = all;
        part[1][w] = before;
        wave_free[w] = sum;
    }
    __syncthreads();
    all = before = 0;
    for (uint32_t i = 0; i < kScanThreads / 64; ++i) {
        all += part[0][i];
        before += part[1][i];
    }
    // rows before the first whose sum passes the free pages are granted; the
    // wavefront's ranks lie between two rows
    uint64_t r0 = before;
    for (uint32_t i = 0; i < w; ++i) r0 += wave_free[i];
    const uint64_t r1 = r0 + wave_free[w], wanted[3] = {all, r0, r1 ? r1 - 1 : 0};
    uint32_t found[3];
    first_past<3>(upto, rows, wanted, lane, found);
    const uint32_t granted = found[0];
    const uint64_t handed = granted ? upto[granted - 1] : 0;
    if (blockIdx.x == tiles) {  // one workgroup more: the rows' own results
        bool refused = false;
        for (uint64_t b = tid; b < rows; b += kScanThreads) {
            const RowAsk s = ask[b];
            held_out[b] = static_cast<int32_t>(b < granted ? s.first + s.count : s.first);
            refused |= b >= granted && s.count;
        }
        if (refused) atomicOr(status, 1u);
        if (tid == 0) *free_pages = all - handed;
        return;
    }
    if (r0 >= min(r1, handed)) return;
    const uint32_t lo = found[1], hi = min(found[2], granted - 1);
    uint64_t r = r0 + sum - own;
    if (!own || r >= handed) return;
    uint32_t b = first_past_between(upto, lo, hi, r);
    for (uint32_t i = 0; i < kEach; ++i) {
        if (!((is_free >> i) & 1u)) continue;
        if (r >= handed) return;
        while (upto[b] <= r) ++b;
        const RowAsk s = ask[b];
        const uint32_t c = s.first + static_cast<uint32_t>(r - (upto[b] - s.count));
        table_out[static_cast<uint64_t>(b) * cols + c] = static_cast<int32_t>(p0 + i);
        kind[p0 + i] = taken;
        ++r;
    }
}

// ---------------------------------------------------------------------------
// Small pools: one launch
// ---------------------------------------------------------------------------

constexpr uint32_t kSmallPages = 1u << 17;  // pages whose bits the first workgroup keeps
constexpr uint32_t kSmallRows = 512;
constexpr uint32_t kPageChunks = kSmallPages / 16 / kScanThreads;  // of 16 pages, a thread's

// Which of 16 kinds are free, as bits: a byte is zero if adding 127 to its low
// seven bits does not reach its top bit and that bit is zero.
__device__ __forceinline__ uint32_t free_of(uint4 kinds) {
    static_assert(COOP_FREE == 0, "free pages are zero bytes");
    const uint32_t words[4] = {kinds.x, kinds.y, kinds.z, kinds.w};
    uint32_t bits = 0;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t zero = (~(((words[i] & 0x7f7f7f7fu) + 0x7f7f7f7fu) | words[i]) >> 7) & 0x01010101u;
        bits |= ((zero | zero >> 7 | zero >> 14 | zero >> 21) & 15u) << (4 * i);
    }
    return bits;
}

// The low four bits as bytes of ones.
__device__ __forceinline__ uint32_t bytes_of(uint32_t bits) {
    const uint32_t b = bits & 15u;
    return ((b | b << 7 | b << 14 | b << 21) & 0x01010101u) * 0xffu;
}

// The entries of a row that neither are given back nor taken.
__device__ __forceinline__ void copy_row(const int32_t* table, int32_t* table_out, uint64_t base,
                                         uint32_t keep, uint32_t top, uint32_t cols, uint32_t tid,
                                         uint32_t threads) {
    if (table_out != table)
        for (uint32_t c = tid; c < keep; c += threads) table_out[base + c] = table[base + c];
    for (uint32_t c = top + tid; c < cols; c += threads) table_out[base + c] = -1;
}

// Workgroup 0 hands out pages; the others each move rows (none where they were
// moved by a launch before).  They touch different entries: a row's first
// min(held, need) and those past max(held, need) are moved, those between are
// workgroup 0's.  With held_out == held a row may already show its new count
// to the workgroup that moves it, which then has the same entries to write,
// or -1 where workgroup 0 has written it before it wrote the count.
__global__ __launch_bounds__(kScanThreads) void pages_small_kernel(
    const uint8_t* kind, uint32_t pages, const int32_t* table, uint32_t rows, uint32_t cols,
    const int32_t* held, const uint64_t* lengths, uint64_t page, uint32_t page_shift, uint8_t taken,
    int32_t* table_out, int32_t* held_out, uint8_t* kind_out, uint32_t* status,
    uint64_t* free_pages) {
    __shared__ uint32_t free_bits[kSmallPages / 32], taken_bits[kSmallPages / 32];
    __shared__ uint32_t group_rank[kSmallPages / 64];  // free pages before each 64
    __shared__ uint64_t row_upto[kSmallRows];
    __shared__ uint32_t row_first[kSmallRows], row_need[kSmallRows], row_held[kSmallRows], back_rows[kSmallRows];
    __shared__ uint64_t part[kScanThreads / 64];
    __shared__ uint32_t backs, flags, granted_rows;
    const uint32_t tid = threadIdx.x, lane = tid & 63u;
    const uint32_t w = __builtin_amdgcn_readfirstlane(tid >> 6);
    auto need_of = [&](uint64_t length, uint32_t h, bool* wide) {
        const uint64_t n = page_shift < 64 ? (length >> page_shift) + ((length & (page - 1)) != 0)
                                           : length / page + (length % page != 0);
        *wide = n > cols;
        return *wide ? h : static_cast<uint32_t>(n);
    };
    if (blockIdx.x > 0) {
        // four wavefronts a row
        const uint32_t quarter = w >> 2, qtid = tid & 255u;
        for (uint32_t b = (blockIdx.x - 1) * 4 + quarter; b < rows; b += (gridDim.x - 1) * 4) {
            const uint32_t h = in_use(held[b], cols);
            bool wide;
            const uint32_t need = need_of(lengths[b], h, &wide);
            copy_row(table, table_out, static_cast<uint64_t>(b) * cols, min(h, need), max(h, need),
                     cols, qtid, 256);
        }
        return;
    }
    // the pool's kinds, 16 pages a load, and its rows
    const bool aligned = ((reinterpret_cast<uintptr_t>(kind) | reinterpret_cast<uintptr_t>(kind_out)) & 15u) == 0;
    const uint32_t chunks = (pages + 15) >> 4;
    uint4 kinds[kPageChunks];
#pragma unroll
    for (uint32_t j = 0; j < kPageChunks; ++j) {
        const uint32_t c = j * kScanThreads + tid;
        kinds[j] = make_uint4(0x02020202u, 0x02020202u, 0x02020202u, 0x02020202u);
        if (c >= chunks) continue;
        if (aligned && c * 16 + 16 <= pages) {
            kinds[j] = reinterpret_cast<const uint4*>(kind)[c];
        } else {
            uint32_t words[4] = {0, 0, 0, 0};
            for (uint32_t i = 0; i < 16; ++i)
                words[i >> 2] |= (c * 16 + i < pages ? kind[c * 16 + i] : 2u) << (8 * (i & 3));
            kinds[j] = make_uint4(words[0], words[1], words[2], words[3]);
        }
    }
    if (tid == 0) backs = flags = 0;
    uint32_t h = 0, need = 0;
    bool wide = false;
    if (tid < rows) {
        h = in_use(held[tid], cols);
        need = need_of(lengths[tid], h, &wide);
        row_first[tid] = min(h, need);
        row_need[tid] = need;
        row_held[tid] = h;
    }
    const uint32_t count = need > h ? need - h : 0;
    __syncthreads();
    if (tid < rows && need < h) back_rows[atomicAdd(&backs, 1u)] = tid;
    if (wide) atomicOr(&flags, 2u);
#pragma unroll
    for (uint32_t j = 0; j < kPageChunks; ++j) {
        const uint32_t c = j * kScanThreads + tid;
        if (j * kScanThreads >= chunks) {  // (no such pages)
            reinterpret_cast<uint16_t*>(free_bits)[c] = 0;
            continue;
        }
        reinterpret_cast<uint16_t*>(free_bits)[c] = static_cast<uint16_t>(free_of(kinds[j]));
        reinterpret_cast<uint16_t*>(taken_bits)[c] = 0;
    }
    {   // the rows' running sum
        const uint64_t sum = scan64(count, lane);
        if (lane == 63) part[w] = sum;
        __syncthreads();
        uint64_t before = 0;
        for (uint32_t i = 0; i < w; ++i) before += part[i];
        if (tid < kSmallRows) row_upto[tid] = before + sum;
    }
    // pages given back: a wavefront a row, four entries a lane at a time
    const uint32_t n_back = backs;
    for (uint32_t i = w; i < n_back; i += kScanThreads / 64) {
        const uint32_t b = back_rows[i], first = row_need[b], last = row_held[b];
        const uint64_t base = static_cast<uint64_t>(b) * cols;
        for (uint32_t c0 = first; c0 < last; c0 += 256) {
            uint32_t p[4];
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                const uint32_t c = c0 + 64 * j + lane;
                p[j] = c < last ? static_cast<uint32_t>(table[base + c]) : ~0u;
            }
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                const uint32_t c = c0 + 64 * j + lane;
                if (c < last) table_out[base + c] = -1;
                if (p[j] < pages) atomicOr(&free_bits[p[j] >> 5], 1u << (p[j] & 31u));
            }
        }
    }
    __syncthreads();
    {   // free pages before each group of 64: two groups a thread
        static_assert(kSmallPages / 64 == 2 * kScanThreads, "a thread counts two groups");
        const uint32_t n0 = __popc(free_bits[4 * tid]) + __popc(free_bits[4 * tid + 1]);
        const uint32_t n1 = __popc(free_bits[4 * tid + 2]) + __popc(free_bits[4 * tid + 3]);
        const uint64_t sum = scan64(n0 + n1, lane);
        if (lane == 63) part[w] = sum;
        __syncthreads();
        uint32_t before = 0;
        for (uint32_t i = 0; i < w; ++i) before += static_cast<uint32_t>(part[i]);
        group_rank[2 * tid] = before + static_cast<uint32_t>(sum) - n0 - n1;
        group_rank[2 * tid + 1] = before + static_cast<uint32_t>(sum) - n1;
    }
    uint64_t all = 0;
    for (uint32_t i = 0; i < kScanThreads / 64; ++i) all += part[i];
    // the first row whose running sum passes the free pages
    const bool fits = tid < rows && row_upto[tid] <= all;
    if (tid == 0) granted_rows = 0;
    __syncthreads();
    const uint64_t fit_mask = __ballot(fits);
    if (lane == 0 && fit_mask) atomicAdd(&granted_rows, static_cast<uint32_t>(__popcll(fit_mask)));
    __syncthreads();
    const uint32_t granted = granted_rows;
    const uint64_t handed = granted ? row_upto[granted - 1] : 0;
    // pages taken: a thread takes 32 pages at a time; its first free one finds
    // its row by search, the others go on from there
    for (uint32_t i = tid; i < (pages + 31) / 32; i += kScanThreads) {
        uint32_t r = group_rank[i >> 1] + (i & 1u ? __popc(free_bits[i - 1]) : 0u);
        uint32_t bits = free_bits[i], took = 0;
        if (!bits || r >= handed) continue;
        uint32_t b = 0;
        for (uint32_t hi = granted; b < hi;) {
            const uint32_t mid = (b + hi) >> 1;
            if (row_upto[mid] > r) hi = mid;
            else b = mid + 1;
        }
        uint32_t upto = static_cast<uint32_t>(row_upto[b]);
        uint32_t before = b ? static_cast<uint32_t>(row_upto[b - 1]) : 0;
        int32_t* to = table_out + static_cast<uint64_t>(b) * cols + row_first[b];
        for (; bits && r < handed; ++r) {
            const uint32_t bit = __builtin_ctz(bits);
            bits &= bits - 1;
            took |= 1u << bit;
            while (upto <= r) {  // (rows that ask for nothing are passed over)
                before = upto;
                upto = static_cast<uint32_t>(row_upto[++b]);
                to = table_out + static_cast<uint64_t>(b) * cols + row_first[b];
            }
            to[r - before] = static_cast<int32_t>(32 * i + bit);
        }
        taken_bits[i] = took;
    }
    if (tid >= granted && tid < rows && count) atomicOr(&flags, 1u);
    // refused: nothing there (a wavefront a row; one thread a row took 420 us for
    // 16000 entries that take 17 us when they are granted)
    for (uint32_t b = granted + w; b < rows; b += kScanThreads / 64)
        for (uint32_t c = row_held[b] + lane; c < row_need[b]; c += 64)
            table_out[static_cast<uint64_t>(b) * cols + c] = -1;
    __syncthreads();
    if (tid < rows) held_out[tid] = static_cast<int32_t>(tid < granted ? need : min(h, need));
    if (tid == 0) {
        *status = flags;
        *free_pages = all - handed;
    }
#pragma unroll
    for (uint32_t j = 0; j < kPageChunks; ++j) {
        const uint32_t c = j * kScanThreads + tid;
        if (c >= chunks) continue;
        const uint32_t is_free = reinterpret_cast<const uint16_t*>(free_bits)[c];
        const uint32_t is_taken = reinterpret_cast<const uint16_t*>(taken_bits)[c];
        uint32_t words[4] = {kinds[j].x, kinds[j].y, kinds[j].z, kinds[j].w};
        if (is_taken | (is_free ^ free_of(kinds[j]))) {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                words[i] = (words[i] & ~bytes_of(is_free >> (4 * i))) |
                           (bytes_of(is_taken >> (4 * i)) & (taken * 0x01010101u));
        }
        if (aligned && c * 16 + 16 <= pages) {
            reinterpret_cast<uint4*>(kind_out)[c] = make_uint4(words[0], words[1], words[2], words[3]);
        } else {
            for (uint32_t i = 0; i < 16; ++i)
                if (c * 16 + i < pages)
                    kind_out[c * 16 + i] = static_cast<uint8_t>(words[i >> 2] >> (8 * (i & 3)));
        }
    }
}

// The rows' part of the kernel above as a launch of its own.
__global__ __launch_bounds__(kThreads) void pages_small_rows_kernel(
    const int32_t* table, uint32_t rows, uint32_t cols, const int32_t* held,
    const uint64_t* lengths, uint64_t page, int32_t* table_out) {
    for (uint32_t b = blockIdx.x; b < rows; b += gridDim.x) {
        const uint32_t h = in_use(held[b], cols);
        bool wide;
        const uint32_t need = needed(lengths[b], page, h, cols, &wide);
        copy_row(table, table_out, static_cast<uint64_t>(b) * cols, min(h, need), max(h, need), cols,
                 threadIdx.x, kThreads);
    }
}

// One wavefront takes 256 consecutive tokens at a time.  The requests of its
// first and last token are found together, 64 probes at a time, and its lanes
// search between the two: tokens of a prompt share their request, and single
// tokens of 64 requests are six steps apart.  Loads that depend on one another
// bound it: 4.3 us for 8 tokens, 10.8 us for 1.2 million of 4096
// sequences.
__global__ __launch_bounds__(kThreads) void slot_map_kernel(
    const int32_t* __restrict__ table, uint32_t rows, uint32_t cols,
    const int32_t* __restrict__ held, const uint64_t* __restrict__ lengths,
    const uint64_t* __restrict__ offsets, uint64_t tokens, uint64_t page, uint32_t page_shift,
    uint32_t pages, int64_t* __restrict__ slots) {
    const uint32_t lane = threadIdx.x & 63u;
    const uint64_t wave = static_cast<uint64_t>(blockIdx.x) * (kThreads / 64) +
                          __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (uint64_t t0 = wave * kWaveTokens; t0 < tokens;
         t0 += static_cast<uint64_t>(gridDim.x) * (kThreads / 64) * kWaveTokens) {
        const uint64_t t1 = min(t0 + kWaveTokens, tokens) - 1;
        const uint64_t ends[2] = {t0, t1};
        uint32_t between[2];
        first_past<2>(offsets, rows + 1, ends, lane, between);
        // a lane's consecutive tokens: the first is searched for, the others
        // mostly are of the same request
        uint64_t t = t0 + lane * kLaneTokens;
        if (t > t1) continue;
        uint32_t at = first_past_between(offsets, between[0], between[1], t);
        uint64_t end = 0, length = 0;
        uint32_t used = 0;
        const int32_t* row = table;
        bool fresh = true;
#pragma unroll
        for (uint32_t i = 0; i < kLaneTokens; ++i, ++t) {
            if (t > t1) break;
            if (!fresh && end <= t) {
                do ++at;
                while (at <= rows && offsets[at] <= t);
                fresh = true;
            }
            int64_t slot = -1;
            if (at > 0 && at <= rows) {
                if (fresh) {
                    const uint32_t b = at - 1;
                    end = offsets[at];
                    length = lengths[b];
                    used = in_use(held[b], cols);
                    row = table + static_cast<uint64_t>(b) * cols;
                    fresh = false;
                }
                const uint64_t behind = end - t;  // at least 1
                if (behind <= length) {
                    const uint64_t pos = length - behind;
                    const uint64_t c = page_shift < 64 ? pos >> page_shift : pos / page;
                    if (c < used) {
                        const int32_t p = row[c];
                        if (static_cast<uint32_t>(p) < pages)
                            slot = static_cast<int64_t>(static_cast<uint64_t>(p) * page + (pos - c * page));
                    }
                }
            }
            slots[t] = slot;
        }
    }
}

// n / d for n < 2^31 by a product: m = ceil(2^(31 + s) / d) with 2^s >= d, so
// that the product's error n (m d - 2^(31 + s)) stays below 2^(31 + s).
struct Divide {
    uint32_t m, s, d;
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const {
        return static_cast<uint32_t>((static_cast<uint64_t>(n) * m) >> (31 + s));
    }
};

Divide divide_by(uint32_t d) {
    Divide r;
    r.d = d;
    r.s = 0;
    while ((1ull << r.s) < d) ++r.s;
    r.m = static_cast<uint32_t>(((1ull << (31 + r.s)) + d - 1) / d);
    return r;
}

// x / scale.  For scales of ordinary size, `inverse` is 1 / scale and the
// product with it is corrected by its remainder, which gives the rounded
// quotient; a quotient of 512 or more ends at the largest number anyway.  The
// remainder is taken with the sign that keeps a zero's: y scale - x is plus zero
// for either zero x, and what is added to y then is minus zero.  (Ordinary
// scales are above zero, and none takes a number other than zero to zero: the
// least is 2^-133 over 2^15, twice the 32-bit step, and the product is off by
// one step at most.)
__device__ __forceinline__ float quotient(float x, float scale, float inverse, bool ordinary) {
    if (!ordinary) return x / scale;
    const float y = x * inverse;
    return fabsf(y) >= 512.f ? y : fmaf(-fmaf(y, scale, -x), inverse, y);
}

// Pairs of numbers in e4m3, limited to its largest value; NaN stays NaN.
__device__ __forceinline__ uint32_t four_e4m3(const float* x) {
    float y[4];
    for (int i = 0; i < 4; ++i) y[i] = x[i] == x[i] ? __builtin_amdgcn_fmed3f(x[i], -448.f, 448.f) : x[i];
    int word = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], word, true));
}

struct WriteArgs {
    coop_rows_t k, v;
    coop_cache_t cache;
    const int64_t* slots;
    uint64_t tokens;
    uint32_t per;         // chunks of a token's key row (and of its value row)
    uint32_t at_once;     // per * at_once is about 2^30
    uint32_t page_shift;  // 64: page_size is not a power of two
    Divide by_per, by_chunks;
    int32_t type;
};

// A thread takes a chunk (eight elements) of a token's key row and the same of
// its value row; consecutive threads take consecutive chunks.  Memory bounds it:
// 65536 tokens of 8 heads of 128 into an e4m3 pool, 383 MB, take 84.6 us (4.5
// TB/s), 64 tokens 2.9 us.  Divisions of 64 bits and by the scales took 109 us.
template <bool kE4M3>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(WriteArgs a) {
    const coop_cache_t& cache = a.cache;
    const uint64_t places = cache.num_pages * cache.page_size;
    const uint64_t each = static_cast<uint64_t>(a.per) * a.at_once;
    // items are counted from a multiple of at_once tokens, in 31 bits
    for (uint64_t block = blockIdx.x * static_cast<uint64_t>(kThreads);
         block < a.tokens * a.per; block += static_cast<uint64_t>(gridDim.x) * kThreads) {
        const uint64_t far = block < each ? 0 : block / each;  // (the same for the whole workgroup)
        const uint32_t i = static_cast<uint32_t>(block - far * each) + threadIdx.x;
        const uint32_t near = a.by_per(i), j = i - near * a.per;
        const uint64_t t = far * a.at_once + near;
        if (t >= a.tokens) continue;
        const uint32_t h = a.by_chunks(j), c = j - h * a.by_chunks.d;
        const uint64_t slot = static_cast<uint64_t>(a.slots[t]);
        if (slot >= places) continue;
        const uint4 kx = *reinterpret_cast<const uint4*>(
            static_cast<const uint16_t*>(a.k.data) + t * a.k.stride[0] + h * a.k.stride[1] + c * 8);
        const uint4 vx = *reinterpret_cast<const uint4*>(
            static_cast<const uint16_t*>(a.v.data) + t * a.v.stride[0] + h * a.v.stride[1] + c * 8);
        const uint64_t p = a.page_shift < 64 ? slot >> a.page_shift : slot / cache.page_size;
        const uint64_t o = slot - p * cache.page_size;
        const uint64_t at_k = p * cache.k_stride[0] + o * cache.k_stride[1] + h * cache.k_stride[2] + c * 8;
        const uint64_t at_v = p * cache.v_stride[0] + o * cache.v_stride[1] + h * cache.v_stride[2] + c * 8;
        if (!kE4M3) {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(cache.k) + at_k) = kx;
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(cache.v) + at_v) = vx;
        } else {
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const float scale = (side ? cache.v_scale : cache.k_scale)[h], inverse = 1.f / scale;
                const bool ordinary = scale >= 0x1p-60f && scale <= 0x1p15f &&
                                      (~__float_as_uint(scale) & 0x7fffffu) != 0;
                const uint4 x = side ? vx : kx;
                const uint32_t word[4] = {x.x, x.y, x.z, x.w};
                float y[8];
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e)
                    y[e] = quotient(coop_pages::to_float(static_cast<uint16_t>(word[e >> 1] >> (16 * (e & 1))), a.type),
                                    scale, inverse, ordinary);
                *reinterpret_cast<uint2*>((side ? static_cast<uint8_t*>(cache.v) + at_v
                                                : static_cast<uint8_t*>(cache.k) + at_k)) =
                    make_uint2(four_e4m3(y), four_e4m3(y + 4));
            }
        }
    }
}

uint32_t grid_for(uint64_t items, uint32_t each) {
    const uint64_t g = (items + each - 1) / each;
    return static_cast<uint32_t>(g < kMaxGrid ? g : kMaxGrid);
}

constexpr uint64_t kMost = (1ull << 31) - 1;

// s if n is 2^s, 64 if it is no power of two
uint32_t shift_of(uint64_t n) {
    return (n & (n - 1)) == 0 ? static_cast<uint32_t>(__builtin_ctzll(n)) : 64u;
}

struct TablesLayout {
    uint32_t tiles;
    size_t upto_offset, ask_offset, bytes;
};

// One workgroup reads and hands out the pages of such a pool.  One launch or
// four, with the slot map behind it (us, calls from a host one after another):
// 512 rows on 107 thousand pages 25 : 35.  Launched ahead, so that only the
// device counts: 8 rows 11 : 17, 256 rows on 54 thousand pages 21 : 24, 512
// rows 25 : 25, and 36 : 26 where a third of them give back all that they hold,
// which one workgroup has to read; 1000 such rows 50 : 33.  So 512 rows are where
// the device is even; calls from a host gain there, replays of a batch in which
// many sequences end lose.
bool is_small(uint64_t pages, uint64_t rows) { return pages <= kSmallPages && rows <= kSmallRows; }

TablesLayout tables_layout(uint64_t pages, uint64_t rows) {
    TablesLayout l;
    if (is_small(pages, rows)) return {0, 0, 0, 0};
    l.tiles = static_cast<uint32_t>((pages + kTilePages - 1) / kTilePages);
    l.upto_offset = (l.tiles * sizeof(uint32_t) + 255) & ~static_cast<size_t>(255);
    l.ask_offset = l.upto_offset + rows * sizeof(uint64_t);
    l.bytes = l.ask_offset + rows * sizeof(RowAsk);
    return l;
}

struct Span {
    const void* at;
    uint64_t bytes;
};

// Whether two arrays share a byte.
bool overlap(const Span& a, const Span& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    return a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}

}  // namespace

extern "C" {

coop_status_t coop_page_tables_workspace_size(uint64_t num_pages, uint64_t num_requests,
                                              size_t* bytes_out) {
    if (!bytes_out || num_pages > kMost || num_requests > kMost) return COOP_ERR_INVALID;
    *bytes_out = tables_layout(num_pages, num_requests).bytes;
    return COOP_OK;
}

coop_status_t coop_page_tables(const uint8_t* kind, uint64_t num_pages, const int32_t* table,
                               uint64_t num_requests, uint64_t max_pages, const int32_t* held,
                               const uint64_t* lengths, uint64_t page_size, uint8_t taken,
                               int32_t* table_out, int32_t* held_out, uint8_t* kind_out,
                               uint32_t* status, uint64_t* free_pages, void* workspace,
                               size_t workspace_bytes, void* stream) {
    if (num_pages > kMost || num_requests > kMost || max_pages > kMost || page_size == 0)
        return COOP_ERR_INVALID;
    if (taken != COOP_EVICTABLE && taken != COOP_PINNED) return COOP_ERR_INVALID;
    if (num_pages && (!kind || !kind_out)) return COOP_ERR_INVALID;
    if (num_requests && (!held || !lengths || !held_out)) return COOP_ERR_INVALID;
    if (num_requests && max_pages && (!table || !table_out)) return COOP_ERR_INVALID;
    if (!status || !free_pages) return COOP_ERR_INVALID;
    const TablesLayout l = tables_layout(num_pages, num_requests);
    {   // an output is its input or apart from every input, and from the others
        const uint64_t tb = num_requests * max_pages * 4, hb = num_requests * 4, nb = num_requests * 8;
        const Span in[4] = {{table, tb}, {held, hb}, {kind, num_pages}, {lengths, nb}};
        const Span out[6] = {{table_out, tb}, {held_out, hb}, {kind_out, num_pages},
                             {status, sizeof(*status)}, {free_pages, sizeof(*free_pages)},
                             {workspace, workspace ? l.bytes : 0}};
        for (int o = 0; o < 6; ++o) {
            for (int i = 0; i < 4; ++i)
                if (!(o == i && i < 3 && out[o].at == in[i].at) && overlap(out[o], in[i])) return COOP_ERR_INVALID;
            for (int i = 0; i < o; ++i)
                if (overlap(out[o], out[i])) return COOP_ERR_INVALID;
        }
    }
    if (l.bytes && (!workspace || workspace_bytes < l.bytes)) return COOP_ERR_WORKSPACE;
    if (l.bytes && !coop_pages::aligned16(workspace)) return COOP_ERR_INVALID;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint32_t pages = static_cast<uint32_t>(num_pages), rows = static_cast<uint32_t>(num_requests);
    const uint32_t cols = static_cast<uint32_t>(max_pages);
    uint32_t* const tile_free = static_cast<uint32_t*>(workspace);
    uint64_t* const upto =
        reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + l.upto_offset);
    RowAsk* const ask = reinterpret_cast<RowAsk*>(static_cast<char*>(workspace) + l.ask_offset);
    if (is_small(num_pages, num_requests)) {
        // (rows are moved ahead of it where the counts are updated in place but
        // the table is not: a new count would show entries that are not there)
        const bool ahead = held_out == held && table_out != table;
        const uint32_t movers = rows && cols ? (rows + 3) / 4 : 0;
        if (ahead && movers) {
            hipLaunchKernelGGL(pages_small_rows_kernel, dim3(rows), dim3(kThreads), 0, s, table, rows,
                               cols, held, lengths, page_size, table_out);
            if (hipGetLastError() != hipSuccess) return COOP_ERR_HIP;
        }
        hipLaunchKernelGGL(pages_small_kernel, dim3(1 + (ahead ? 0 : movers)), dim3(kScanThreads), 0, s,
                           kind, pages, table, rows, cols, held, lengths, page_size,
                           shift_of(page_size), taken, table_out, held_out, kind_out, status,
                           free_pages);
        return hipGetLastError() == hipSuccess ? COOP_OK : COOP_ERR_HIP;
    }
    if (pages && kind_out != kind) {
        hipLaunchKernelGGL(pages_copy_kernel, dim3(grid_for(pages, kThreads * 16)), dim3(kThreads), 0, s,
                           kind, kind_out, pages);
        if (hipGetLastError() != hipSuccess) return COOP_ERR_HIP;
    }
    if (rows && cols) {
        hipLaunchKernelGGL(pages_rows_kernel, dim3(grid_for(rows, 1)), dim3(kThreads), 0, s, table,
                           held, lengths, page_size, rows, cols, pages, table_out, kind_out);
        if (hipGetLastError() != hipSuccess) return COOP_ERR_HIP;
    }
    hipLaunchKernelGGL(pages_count_kernel, dim3(l.tiles + 1), dim3(kScanThreads), 0, s, kind_out,
                       pages, l.tiles, held, lengths, page_size, rows, cols, tile_free, upto,
                       ask, status);
    if (hipGetLastError() != hipSuccess) return COOP_ERR_HIP;
    hipLaunchKernelGGL(pages_take_kernel, dim3(l.tiles + 1), dim3(kScanThreads), 0, s, kind_out,
                       pages, l.tiles, tile_free, upto, ask, rows, cols, taken, table_out, held_out,
                       status, free_pages);
    return hipGetLastError() == hipSuccess ? COOP_OK : COOP_ERR_HIP;
}

coop_status_t coop_slot_map(const int32_t* table, uint64_t num_requests, uint64_t max_pages,
                            const int32_t* held, const uint64_t* lengths,
                            const uint64_t* token_offsets, uint64_t num_tokens,
                            uint64_t page_size, uint64_t num_pages, int64_t* slots,
                            void* stream) {
    if (num_tokens == 0) return COOP_OK;
    if (num_pages > kMost || num_requests > kMost - 1 || max_pages > kMost || page_size == 0 ||
        page_size > kMost || num_tokens > (1ull << 60))
        return COOP_ERR_INVALID;
    if (!slots || !token_offsets) return COOP_ERR_INVALID;
    if (num_requests && (!held || !lengths)) return COOP_ERR_INVALID;
    if (num_requests && max_pages && !table) return COOP_ERR_INVALID;
    const Span out = {slots, num_tokens * sizeof(*slots)};
    for (const Span& in : {Span{table, num_requests * max_pages * sizeof(*table)},
                           Span{held, num_requests * sizeof(*held)},
                           Span{lengths, num_requests * sizeof(*lengths)},
                           Span{token_offsets, (num_requests + 1) * sizeof(*token_offsets)}})
        if (overlap(out, in)) return COOP_ERR_INVALID;
    hipLaunchKernelGGL(slot_map_kernel, dim3(grid_for(num_tokens, kThreads / 64 * kWaveTokens)), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), table, static_cast<uint32_t>(num_requests),
                       static_cast<uint32_t>(max_pages), held, lengths, token_offsets, num_tokens,
                       page_size, shift_of(page_size), static_cast<uint32_t>(num_pages), slots);
    return hipGetLastError() == hipSuccess ? COOP_OK : COOP_ERR_HIP;
}

coop_status_t coop_cache_write(const coop_rows_t* k, const coop_rows_t* v, int32_t type,
                               const int64_t* slots, uint64_t num_tokens,
                               const coop_cache_t* cache, void* stream) {
    if (!cache || !k || !v) return COOP_ERR_INVALID;
    if (const coop_status_t rc = coop_pages::check_cache(*cache, type)) return rc;
    if (num_tokens == 0 || cache->num_pages == 0) return COOP_OK;
    if (!slots || num_tokens > (1ull << 40)) return COOP_ERR_INVALID;
    if (!coop_pages::rows_valid(*k, num_tokens, cache->heads, cache->dim) ||
        !coop_pages::rows_valid(*v, num_tokens, cache->heads, cache->dim))
        return COOP_ERR_INVALID;
    WriteArgs a;
    a.k = *k;
    a.v = *v;
    a.cache = *cache;
    a.slots = slots;
    a.tokens = num_tokens;
    a.per = static_cast<uint32_t>(cache->heads * (cache->dim / 8));
    a.at_once = (1u << 30) / a.per;
    a.page_shift = shift_of(cache->page_size);
    a.by_per = divide_by(a.per);
    a.by_chunks = divide_by(static_cast<uint32_t>(cache->dim / 8));
    a.type = type;
    auto kernel = cache->type == COOP_E4M3 ? cache_write_kernel<true> : cache_write_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3(grid_for(num_tokens * a.per, kThreads)), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), a);
    return hipGetLastError() == hipSuccess ? COOP_OK : COOP_ERR_HIP;
}

}  // extern "C"
