// Paged pools: block tables, slot maps and cache writes for gfx950.
//
// coop_page_tables, out of place, four launches on the caller's stream:
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

struct RowState {  // what step 4 needs of a row
    uint64_t upto;   // pages asked for by this row and those before it
    uint32_t first;  // entries that it keeps
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
    for (uint64_t p = blockIdx.x * kThreads + threadIdx.x; p < n; p += gridDim.x * kThreads)
        out[p] = in[p];
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

__global__ __launch_bounds__(kScanThreads) void pages_count_kernel(
    const uint8_t* kind, uint32_t pages, uint32_t tiles, const int32_t* held,
    const uint64_t* lengths, uint64_t page, uint32_t rows, uint32_t cols,
    uint32_t* __restrict__ tile_free, RowState* __restrict__ state, uint32_t* status) {
    __shared__ uint64_t part[kScanThreads / 64];
    __shared__ uint32_t any_wide;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, w = tid >> 6;
    if (blockIdx.x < tiles) {
        const uint32_t p0 = blockIdx.x * kTilePages;
        uint32_t n = 0;
        for (uint32_t i = tid; i < kTilePages; i += kScanThreads)
            n += p0 + i < pages && kind[p0 + i] == COOP_FREE;
        for (uint32_t m = 32; m; m >>= 1) n += __shfl_xor(n, m, 64);
        if (lane == 0) part[w] = n;
        __syncthreads();
        if (tid == 0) {
            uint64_t s = 0;
            for (uint32_t i = 0; i < kScanThreads / 64; ++i) s += part[i];
            tile_free[blockIdx.x] = static_cast<uint32_t>(s);
        }
        return;
    }
    // the last workgroup: the rows' running sum
    if (tid == 0) any_wide = 0;
    uint64_t carry = 0;
    for (uint32_t b0 = 0; b0 < rows; b0 += kScanThreads) {
        const uint32_t b = b0 + tid;
        uint32_t h = 0, need = 0;
        bool wide = false;
        if (b < rows) {
            h = in_use(held[b], cols);
            need = needed(lengths[b], page, h, cols, &wide);
        }
        const uint32_t count = need > h ? need - h : 0;
        uint64_t sum = count;
        for (uint32_t d = 1; d < 64; d <<= 1) {
            const uint64_t up = __shfl_up(sum, d, 64);
            if (lane >= d) sum += up;
        }
        __syncthreads();
        if (wide) any_wide = 1;
        if (lane == 63) part[w] = sum;
        __syncthreads();
        uint64_t before = carry, all = 0;
        for (uint32_t i = 0; i < kScanThreads / 64; ++i) {
            if (i < w) before += part[i];
            all += part[i];
        }
        if (b < rows) state[b] = {before + sum, min(h, need), count};
        carry += all;
    }
    __syncthreads();
    if (tid == 0) *status = any_wide ? 2u : 0u;
}

// The first row in [0, rows) whose running sum exceeds r; rows if none.
__device__ __forceinline__ uint32_t row_of(const RowState* state, uint32_t rows, uint64_t r) {
    uint32_t lo = 0, hi = rows;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) >> 1;
        if (state[mid].upto > r) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

__global__ __launch_bounds__(kScanThreads) void pages_take_kernel(
    uint8_t* kind, uint32_t pages, uint32_t tiles, const uint32_t* __restrict__ tile_free,
    const RowState* __restrict__ state, uint32_t rows, uint32_t cols, uint8_t taken,
    int32_t* table_out, int32_t* held_out, uint32_t* status, uint64_t* free_pages) {
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
    for (uint32_t m = 32; m; m >>= 1) {
        all += __shfl_xor(all, m, 64);
        before += __shfl_xor(before, m, 64);
    }
    if (lane == 0) {
        part[0][w] = all;
        part[1][w] = before;
    }
    __syncthreads();
    all = before = 0;
    for (uint32_t i = 0; i < kScanThreads / 64; ++i) {
        all += part[0][i];
        before += part[1][i];
    }
    // rows before the first whose sum passes the free pages are granted
    const uint32_t granted = row_of(state, rows, all);
    const uint64_t handed = granted ? state[granted - 1].upto : 0;
    if (blockIdx.x == tiles) {  // one workgroup more: the rows' own results
        bool refused = false;
        for (uint32_t b = tid; b < rows; b += kScanThreads) {
            const RowState s = state[b];
            held_out[b] = static_cast<int32_t>(b < granted ? s.first + s.count : s.first);
            refused |= b >= granted && s.count;
        }
        if (refused) atomicOr(status, 1u);
        if (tid == 0) *free_pages = all - handed;
        return;
    }
    if (before >= handed) return;
    constexpr uint32_t kEach = kTilePages / kScanThreads;  // consecutive pages of a thread
    const uint32_t p0 = blockIdx.x * kTilePages + tid * kEach;
    uint32_t is_free = 0;
    for (uint32_t i = 0; i < kEach; ++i)
        if (p0 + i < pages && kind[p0 + i] == COOP_FREE) is_free |= 1u << i;
    const uint32_t own = __popc(is_free);
    uint32_t sum = own;
    for (uint32_t d = 1; d < 64; d <<= 1) {
        const uint32_t up = __shfl_up(sum, d, 64);
        if (lane >= d) sum += up;
    }
    if (lane == 63) wave_free[w] = sum;
    __syncthreads();
    uint64_t r = before + sum - own;
    for (uint32_t i = 0; i < w; ++i) r += wave_free[i];
    uint32_t b = rows;
    for (uint32_t i = 0; i < kEach; ++i) {
        if (!((is_free >> i) & 1u)) continue;
        if (r >= handed) return;
        if (b >= rows || state[b].upto <= r) b = row_of(state, rows, r);
        const RowState s = state[b];
        const uint32_t c = s.first + static_cast<uint32_t>(r - (s.upto - s.count));
        table_out[static_cast<uint64_t>(b) * cols + c] = static_cast<int32_t>(p0 + i);
        kind[p0 + i] = taken;
        ++r;
    }
}

__global__ __launch_bounds__(kThreads) void slot_map_kernel(
    const int32_t* __restrict__ table, uint32_t rows, uint32_t cols,
    const int32_t* __restrict__ held, const uint64_t* __restrict__ lengths,
    const uint64_t* __restrict__ offsets, uint64_t tokens, uint64_t page, uint32_t pages,
    int64_t* __restrict__ slots) {
    for (uint64_t t = static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x; t < tokens;
         t += static_cast<uint64_t>(gridDim.x) * kThreads) {
        int64_t slot = -1;
        // the last request that starts at or before t
        uint32_t lo = 0, hi = rows + 1;
        while (lo < hi) {
            const uint32_t mid = (lo + hi) >> 1;
            if (offsets[mid] > t) hi = mid;
            else lo = mid + 1;
        }
        if (lo > 0 && lo <= rows) {
            const uint32_t b = lo - 1;
            const uint64_t length = lengths[b], behind = offsets[lo] - t;  // behind >= 1
            if (behind <= length) {
                const uint64_t pos = length - behind, c = pos / page;
                if (c < in_use(held[b], cols)) {
                    const int32_t p = table[static_cast<uint64_t>(b) * cols + c];
                    if (static_cast<uint32_t>(p) < pages)
                        slot = static_cast<int64_t>(static_cast<uint64_t>(p) * page + pos % page);
                }
            }
        }
        slots[t] = slot;
    }
}

// x / scale in e4m3, limited to its largest value.
__device__ __forceinline__ uint32_t to_e4m3(float x, float scale) {
    float y = x / scale;
    if (y == y) y = fminf(fmaxf(y, -448.f), 448.f);
    return __builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 0xffu;
}

template <bool kE4M3>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(
    coop_rows_t k, coop_rows_t v, int32_t type, const int64_t* __restrict__ slots, uint64_t tokens,
    coop_cache_t cache) {
    const uint32_t chunks = static_cast<uint32_t>(cache.dim) / 8;  // of eight elements
    const uint32_t heads = static_cast<uint32_t>(cache.heads);
    const uint64_t per = static_cast<uint64_t>(chunks) * heads;
    const uint64_t places = cache.num_pages * cache.page_size;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x; i < tokens * per;
         i += static_cast<uint64_t>(gridDim.x) * kThreads) {
        const uint64_t t = i / per;
        const uint32_t j = static_cast<uint32_t>(i - t * per), h = j / chunks, c = j - h * chunks;
        const uint64_t slot = static_cast<uint64_t>(slots[t]);
        if (slot >= places) continue;
        const uint64_t p = slot / cache.page_size, o = slot - p * cache.page_size;
        for (int side = 0; side < 2; ++side) {
            const coop_rows_t& in = side ? v : k;
            const uint64_t* st = side ? cache.v_stride : cache.k_stride;
            const uint4 x = *reinterpret_cast<const uint4*>(
                static_cast<const uint16_t*>(in.data) + t * in.stride[0] + h * in.stride[1] + c * 8);
            const uint64_t at = p * st[0] + o * st[1] + h * st[2] + c * 8;
            void* const to = side ? cache.v : cache.k;
            if (!kE4M3) {
                *reinterpret_cast<uint4*>(static_cast<uint16_t*>(to) + at) = x;
            } else {
                const float scale = (side ? cache.v_scale : cache.k_scale)[h];
                const uint32_t word[4] = {x.x, x.y, x.z, x.w};
                uint32_t q[2] = {0, 0};
                for (uint32_t e = 0; e < 8; ++e) {
                    const uint16_t bits = static_cast<uint16_t>(word[e >> 1] >> (16 * (e & 1)));
                    q[e >> 2] |= to_e4m3(coop_pages::to_float(bits, type), scale) << (8 * (e & 3));
                }
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(to) + at) = make_uint2(q[0], q[1]);
            }
        }
    }
}

uint32_t grid_for(uint64_t items, uint32_t each) {
    const uint64_t g = (items + each - 1) / each;
    return static_cast<uint32_t>(g < kMaxGrid ? g : kMaxGrid);
}

constexpr uint64_t kMost = (1ull << 31) - 1;

struct TablesLayout {
    uint32_t tiles;
    size_t state_offset, bytes;
};

TablesLayout tables_layout(uint64_t pages, uint64_t rows) {
    TablesLayout l;
    l.tiles = static_cast<uint32_t>((pages + kTilePages - 1) / kTilePages);
    l.state_offset = (l.tiles * sizeof(uint32_t) + 255) & ~static_cast<size_t>(255);
    l.bytes = l.state_offset + rows * sizeof(RowState);
    return l;
}

// Whether [a, a + na) and [b, b + nb) share a byte.
bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na && nb && x < y + nb && y < x + na;
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
    {   // an output is its input or apart from every input
        const uint64_t tb = num_requests * max_pages * 4, hb = num_requests * 4, nb = num_requests * 8;
        const struct { const void* out; uint64_t bytes; const void* in; } outs[3] = {
            {table_out, tb, table}, {held_out, hb, held}, {kind_out, num_pages, kind}};
        const struct { const void* in; uint64_t bytes; } ins[4] = {
            {table, tb}, {held, hb}, {kind, num_pages}, {lengths, nb}};
        for (const auto& o : outs)
            for (const auto& i : ins)
                if (!(o.in == i.in && o.out == o.in) && overlap(o.out, o.bytes, i.in, i.bytes))
                    return COOP_ERR_INVALID;
    }
    const TablesLayout l = tables_layout(num_pages, num_requests);
    if (l.bytes && (!workspace || workspace_bytes < l.bytes)) return COOP_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint32_t pages = static_cast<uint32_t>(num_pages), rows = static_cast<uint32_t>(num_requests);
    const uint32_t cols = static_cast<uint32_t>(max_pages);
    uint32_t* const tile_free = static_cast<uint32_t*>(workspace);
    RowState* const state =
        reinterpret_cast<RowState*>(static_cast<char*>(workspace) + l.state_offset);
    if (pages && kind_out != kind) {
        hipLaunchKernelGGL(pages_copy_kernel, dim3(grid_for(pages, kThreads)), dim3(kThreads), 0, s,
                           kind, kind_out, pages);
        if (hipGetLastError() != hipSuccess) return COOP_ERR_HIP;
    }
    if (rows && cols) {
        hipLaunchKernelGGL(pages_rows_kernel, dim3(grid_for(rows, 1)), dim3(kThreads), 0, s, table,
                           held, lengths, page_size, rows, cols, pages, table_out, kind_out);
        if (hipGetLastError() != hipSuccess) return COOP_ERR_HIP;
    }
    hipLaunchKernelGGL(pages_count_kernel, dim3(l.tiles + 1), dim3(kScanThreads), 0, s, kind_out,
                       pages, l.tiles, held, lengths, page_size, rows, cols, tile_free, state,
                       status);
    if (hipGetLastError() != hipSuccess) return COOP_ERR_HIP;
    hipLaunchKernelGGL(pages_take_kernel, dim3(l.tiles + 1), dim3(kScanThreads), 0, s, kind_out,
                       pages, l.tiles, tile_free, state, rows, cols, taken, table_out, held_out,
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
    hipLaunchKernelGGL(slot_map_kernel, dim3(grid_for(num_tokens, kThreads)), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), table, static_cast<uint32_t>(num_requests),
                       static_cast<uint32_t>(max_pages), held, lengths, token_offsets, num_tokens,
                       page_size, static_cast<uint32_t>(num_pages), slots);
    return hipGetLastError() == hipSuccess ? COOP_OK : COOP_ERR_HIP;
}

coop_status_t coop_cache_write(const coop_rows_t* k, const coop_rows_t* v, int32_t type,
                               const int64_t* slots, uint64_t num_tokens,
                               const coop_cache_t* cache, void* stream) {
    if (!cache || !k || !v) return COOP_ERR_INVALID;
    if (const coop_status_t rc = coop_pages::check_cache(*cache, type)) return rc;
    if (num_tokens == 0 || cache->num_pages == 0) return COOP_OK;
    if (!slots || num_tokens > (1ull << 40)) return COOP_ERR_INVALID;
    if (!coop_pages::rows_valid(*k, num_tokens) || !coop_pages::rows_valid(*v, num_tokens))
        return COOP_ERR_INVALID;
    const uint64_t items = num_tokens * cache->heads * (cache->dim / 8);
    auto kernel = cache->type == COOP_E4M3 ? cache_write_kernel<true> : cache_write_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3(grid_for(items, kThreads)), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), *k, *v, type, slots, num_tokens, *cache);
    return hipGetLastError() == hipSuccess ? COOP_OK : COOP_ERR_HIP;
}

}  // extern "C"
