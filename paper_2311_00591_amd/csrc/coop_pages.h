// What the paged-pool sources share: checks of their descriptors on the host,
// and number conversions.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "coop.h"

#pragma GCC visibility push(hidden)

namespace coop_pages {

constexpr uint64_t kMaxDim = 256;
constexpr uint64_t kMaxHeads = 1u << 16;
constexpr uint64_t kMaxStride = 1ull << 40;
constexpr uint64_t kMaxReach = 1ull << 60;   // elements: offsets in bytes stay below 2^62

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Whether the last element of rows of `dim`, `count[i]` of them `stride[i]`
// apart along dimension i, is so near that the kernels' 64-bit offsets hold.
template <int kDims>
inline bool reach_valid(const uint64_t (&count)[kDims], const uint64_t (&stride)[kDims], uint64_t dim) {
    unsigned __int128 reach = dim;
    for (int i = 0; i < kDims; ++i)
        if (count[i]) reach += static_cast<unsigned __int128>(count[i] - 1) * stride[i];
    return reach <= kMaxReach;
}

// COOP_OK if the cache's description is sound and rows of `type` can be stored
// in it or meet it in products.
inline coop_status_t check_cache(const coop_cache_t& c, int32_t type) {
    if (type != COOP_BF16 && type != COOP_FP16) return COOP_ERR_INVALID;
    const bool e4m3 = c.type == COOP_E4M3;
    if (!e4m3 && c.type != type) return COOP_ERR_INVALID;
    const uint64_t chunk = e4m3 ? 16 : 8;  // elements in 16 bytes
    if (c.dim == 0 || c.dim > kMaxDim || c.dim % chunk) return COOP_ERR_INVALID;
    if (c.heads == 0 || c.heads > kMaxHeads || c.page_size == 0) return COOP_ERR_INVALID;
    if (c.num_pages > (1ull << 31) - 1 || c.page_size > (1ull << 31) - 1) return COOP_ERR_INVALID;
    if (e4m3 ? !c.k_scale || !c.v_scale : c.k_scale || c.v_scale) return COOP_ERR_INVALID;
    for (int i = 0; i < 3; ++i)
        if (c.k_stride[i] % chunk || c.v_stride[i] % chunk || c.k_stride[i] > kMaxStride ||
            c.v_stride[i] > kMaxStride)
            return COOP_ERR_INVALID;
    const uint64_t count[3] = {c.num_pages, c.page_size, c.heads};
    if (!reach_valid(count, c.k_stride, c.dim) || !reach_valid(count, c.v_stride, c.dim))
        return COOP_ERR_INVALID;
    if (c.num_pages && (!c.k || !c.v || !aligned16(c.k) || !aligned16(c.v))) return COOP_ERR_INVALID;
    return COOP_OK;
}

// Whether rows of 16-bit numbers can be read 16 bytes at a time.
inline bool rows_valid(const coop_rows_t& r, uint64_t tokens, uint64_t heads, uint64_t dim) {
    if (r.stride[0] % 8 || r.stride[1] % 8) return false;
    if (r.stride[0] > kMaxStride || r.stride[1] > kMaxStride) return false;
    if (!reach_valid({tokens, heads}, r.stride, dim)) return false;
    return tokens == 0 || (r.data && aligned16(r.data));
}

__device__ __forceinline__ float to_float(uint16_t bits, int32_t type) {
    if (type == COOP_BF16) return __uint_as_float(static_cast<uint32_t>(bits) << 16);
    return static_cast<float>(__builtin_bit_cast(_Float16, bits));
}

}  // namespace coop_pages

#pragma GCC visibility pop
