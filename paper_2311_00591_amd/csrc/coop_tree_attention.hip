// Attention of a tree of new tokens over a paged pool, for gfx950.
//
// One wavefront a new token and query head: it walks the request's cached keys
// and then the token's ancestors, with the running maximum m and sum l of the
// softmax:  m' = max(m, s),  l' = l e^(m - m') + e^(s - m'),
// o' = o e^(m - m') + e^(s - m') v,  out = o / l.

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "coop.h"
#include "coop_pages.h"

namespace {

struct Args {
    coop_rows_t q, k, v;
    coop_cache_t cache;
    const uint64_t* offsets;
    const int32_t* parents;
    const int32_t* table;
    const uint64_t* lengths;
    uint16_t* out;
    uint64_t tokens;
    uint32_t requests, max_pages, q_heads, type;
    float scale;
};

__device__ __forceinline__ uint16_t from_float(float x, uint32_t type) {
    if (type == COOP_FP16) return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}

// One element of the cache as a 32-bit number, without its head's scale.
__device__ __forceinline__ float cached(const void* base, uint64_t at, int32_t cache_type) {
    if (cache_type == COOP_E4M3)
        return __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(base)[at], 0);
    return coop_pages::to_float(static_cast<const uint16_t*>(base)[at], cache_type);
}

__global__ __launch_bounds__(64) void tree_attention_kernel(Args a) {
    const uint32_t lane = threadIdx.x, dim = static_cast<uint32_t>(a.cache.dim);
    const uint64_t t = blockIdx.x / a.q_heads;
    const uint32_t hq = static_cast<uint32_t>(blockIdx.x - t * a.q_heads);
    const uint32_t h = hq / (a.q_heads / static_cast<uint32_t>(a.cache.heads));
    uint32_t lo = 0, hi = a.requests + 1;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) >> 1;
        if (a.offsets[mid] > t) hi = mid;
        else lo = mid + 1;
    }
    if (lo == 0 || lo > a.requests) return;
    const uint32_t b = lo - 1;
    const uint64_t first = a.offsets[b];
    const int64_t self = static_cast<int64_t>(t - first);
    float q[4], o[4] = {0, 0, 0, 0}, m = -__builtin_inff(), l = 0;
    const uint16_t* const qr =
        static_cast<const uint16_t*>(a.q.data) + t * a.q.stride[0] + hq * a.q.stride[1];
    for (uint32_t i = 0; i < 4; ++i)
        q[i] = lane + 64 * i < dim ? coop_pages::to_float(qr[lane + 64 * i], a.type) : 0.f;
    const bool is_void = a.parents && (a.parents[t] < -1 || a.parents[t] >= self);

    auto visit = [&](const float* kx, const float* vx, float ks, float vs) {
        float s = 0;
        for (uint32_t i = 0; i < 4; ++i) s += q[i] * kx[i];
        for (uint32_t d = 32; d; d >>= 1) s += __shfl_xor(s, d, 64);
        s *= a.scale * ks;
        const float top = fmaxf(m, s);
        const float was = m == top ? 1.f : __expf(m - top);
        const float p = __expf(s - top);
        l = l * was + p;
        for (uint32_t i = 0; i < 4; ++i) o[i] = o[i] * was + p * vs * vx[i];
        m = top;
    };

    if (!is_void) {
        const uint64_t most = static_cast<uint64_t>(a.max_pages) * a.cache.page_size;
        const uint64_t n = a.lengths[b] < most ? a.lengths[b] : most;
        const float ks = a.cache.k_scale ? a.cache.k_scale[h] : 1.f;
        const float vs = a.cache.v_scale ? a.cache.v_scale[h] : 1.f;
        float kx[4], vx[4];
        for (uint64_t j = 0; j < n; ++j) {
            const int32_t page = a.table[static_cast<uint64_t>(b) * a.max_pages + j / a.cache.page_size];
            if (static_cast<uint32_t>(page) >= a.cache.num_pages) continue;
            const uint64_t place = j % a.cache.page_size;
            const uint64_t ka = page * a.cache.k_stride[0] + place * a.cache.k_stride[1] + h * a.cache.k_stride[2];
            const uint64_t va = page * a.cache.v_stride[0] + place * a.cache.v_stride[1] + h * a.cache.v_stride[2];
            for (uint32_t i = 0; i < 4; ++i) {
                const uint32_t d = lane + 64 * i;
                kx[i] = d < dim ? cached(a.cache.k, ka + d, a.cache.type) : 0.f;
                vx[i] = d < dim ? cached(a.cache.v, va + d, a.cache.type) : 0.f;
            }
            visit(kx, vx, ks, vs);
        }
        int64_t j = self;
        while (j >= 0) {
            const uint64_t row = first + j;
            int64_t up = j - 1;
            if (a.parents) {
                up = a.parents[row];
                if (up < -1 || up >= j) break;
            }
            const uint16_t* const kr = static_cast<const uint16_t*>(a.k.data) + row * a.k.stride[0] + h * a.k.stride[1];
            const uint16_t* const vr = static_cast<const uint16_t*>(a.v.data) + row * a.v.stride[0] + h * a.v.stride[1];
            for (uint32_t i = 0; i < 4; ++i) {
                const uint32_t d = lane + 64 * i;
                kx[i] = d < dim ? coop_pages::to_float(kr[d], a.type) : 0.f;
                vx[i] = d < dim ? coop_pages::to_float(vr[d], a.type) : 0.f;
            }
            visit(kx, vx, 1.f, 1.f);
            j = up;
        }
    }
    uint16_t* const to = a.out + (t * a.q_heads + hq) * dim;
    for (uint32_t i = 0; i < 4; ++i)
        if (lane + 64 * i < dim) to[lane + 64 * i] = from_float(is_void ? 0.f : o[i] / l, a.type);
}

constexpr uint64_t kMost = (1ull << 31) - 1;

bool counts_valid(uint64_t requests, uint64_t tokens, uint64_t q_heads, uint64_t heads,
                  uint64_t dim) {
    return heads && heads <= coop_pages::kMaxHeads && q_heads && q_heads <= coop_pages::kMaxHeads &&
           q_heads % heads == 0 && requests < kMost && tokens <= kMost &&
           tokens * q_heads <= kMost && dim && dim <= coop_pages::kMaxDim && dim % 8 == 0;
}

}  // namespace

extern "C" {

coop_status_t coop_tree_attention_workspace_size(uint64_t num_requests, uint64_t num_tokens,
                                                 uint64_t q_heads, uint64_t heads, uint64_t dim,
                                                 size_t* bytes_out) {
    if (!bytes_out || !counts_valid(num_requests, num_tokens, q_heads, heads, dim))
        return COOP_ERR_INVALID;
    *bytes_out = 0;
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
        max_pages > kMost)
        return COOP_ERR_INVALID;
    if (num_tokens == 0) return COOP_OK;
    if (!coop_pages::rows_valid(*q, num_tokens) || !coop_pages::rows_valid(*k_new, num_tokens) ||
        !coop_pages::rows_valid(*v_new, num_tokens))
        return COOP_ERR_INVALID;
    if (!out || !coop_pages::aligned16(out) || !token_offsets) return COOP_ERR_INVALID;
    if (num_requests == 0) return COOP_OK;
    if (!lengths || (max_pages && !table)) return COOP_ERR_INVALID;
    size_t need = 0;
    coop_tree_attention_workspace_size(num_requests, num_tokens, q_heads, cache->heads, cache->dim,
                                       &need);
    if (need && (!workspace || workspace_bytes < need)) return COOP_ERR_WORKSPACE;
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
    a.type = static_cast<uint32_t>(type);
    a.scale = scale;
    hipLaunchKernelGGL(tree_attention_kernel, dim3(static_cast<uint32_t>(num_tokens * q_heads)),
                       dim3(64), 0, static_cast<hipStream_t>(stream), a);
    return hipGetLastError() == hipSuccess ? COOP_OK : COOP_ERR_HIP;
}

}  // extern "C"
