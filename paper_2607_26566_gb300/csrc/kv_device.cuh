// Device helpers of the key/value cache kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "kv.hpp"

namespace t2i {

// The address of a slot's row; null where the table or the pool has none.
__device__ __forceinline__ uint8_t* kv_row(const KvPages& p, uint32_t seq, int64_t slot, uint32_t layer, uint32_t which,
                                           uint32_t head) {
    if (slot < 0 || slot >> p.token_shift >= int64_t(p.table_pages)) return nullptr;
    const uint32_t page = uint32_t(p.table[seq * p.table_stride + uint64_t(slot >> p.token_shift)]);
    if (page >= p.total_pages) return nullptr;
    const uint64_t row = ((uint64_t((layer * 2 + which) * p.kv_heads + head)) << p.token_shift) +
                         (uint64_t(slot) & ((uint64_t(1) << p.token_shift) - 1));
    return reinterpret_cast<uint8_t*>(p.pool + page * p.page_bytes + row * (p.head_dim * 2));
}

// Sequence s's new tokens: the first one's row and their number, within the
// token arrays whatever starts holds, and its length, within the table row.
struct KvSeq {
    int32_t first, n, len;
};
__device__ __forceinline__ KvSeq kv_seq(const KvPages& p, const KvTokens& t, uint32_t s) {
    KvSeq q;
    const int64_t cap = int64_t(p.table_pages) << p.token_shift;
    int64_t b, e;
    if (t.starts) {
        b = t.starts[s];
        e = t.starts[s + 1];
    } else {
        b = int64_t(s) * t.each;
        e = b + t.each;
    }
    b = b < 0 ? 0 : b;
    e = e > int64_t(t.n_tokens) ? int64_t(t.n_tokens) : e;
    const int64_t len = t.lens[s];
    const int64_t n = e - b;
    const bool ok = n > 0 && len >= n && len <= cap;
    q.first = int32_t(b);
    q.n = ok ? int32_t(n) : 0;
    q.len = ok ? int32_t(len) : 0;
    return q;
}

// The sequence of token t, by a 32-way search of a warp (all lanes call it).
__device__ __forceinline__ uint32_t kv_owner(const KvTokens& k, uint32_t t) {
    if (!k.starts) return t / k.each;
    const uint32_t lane = threadIdx.x & 31u;
    uint32_t lo = 0, n = k.n_seqs;
    while (n > 1) {
        const uint32_t step = (n + 31) / 32;
        const uint32_t i = lane * step;
        const bool before = i < n && k.starts[lo + i] <= int32_t(t);
        const uint32_t c = __popc(__ballot_sync(0xFFFFFFFFu, before));
        const uint32_t at = c ? (c - 1) * step : 0;
        lo += at;
        n = min(step, n - at);
    }
    return lo;
}

template <class T>
struct Kv16;
template <>
struct Kv16<__nv_bfloat16> {
    static __device__ __forceinline__ float2 to2(uint32_t v) {
        return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&v));
    }
    static __device__ __forceinline__ uint32_t from2(float a, float b) {
        const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&r);
    }
    static __device__ __forceinline__ __nv_bfloat16 from1(float a) { return __float2bfloat16_rn(a); }
};
template <>
struct Kv16<__half> {
    static __device__ __forceinline__ float2 to2(uint32_t v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }
    static __device__ __forceinline__ uint32_t from2(float a, float b) {
        const __half2 r = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&r);
    }
    static __device__ __forceinline__ __half from1(float a) { return __float2half_rn(a); }
};

// Eight consecutive elements as fp32, and back to 16 bits.
template <class T>
__device__ __forceinline__ void kv_load8(const T* p, float (&x)[8]) {
    if constexpr (sizeof(T) == 4) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = Kv16<T>::to2(w[i]);
            x[2 * i] = f.x, x[2 * i + 1] = f.y;
        }
    }
}
template <class T>
__device__ __forceinline__ void kv_store8(T* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(Kv16<T>::from2(x[0], x[1]), Kv16<T>::from2(x[2], x[3]),
                                              Kv16<T>::from2(x[4], x[5]), Kv16<T>::from2(x[6], x[7]));
}

}  // namespace t2i
