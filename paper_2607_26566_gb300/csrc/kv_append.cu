// Appending keys and values to the cache (per-head RMS norm and rotation of
// queries and keys on the way), and keeping the accepted rows of a draft.
#include "kv_device.cuh"
#include "t2istore.h"

namespace t2i {
namespace {

// Sixteen lanes hold a head's row, eight elements a lane.
constexpr uint32_t kLanes = 16;
constexpr uint32_t kThreads = 256;
constexpr uint32_t kGroups = kThreads / kLanes;

// The rotation of a row that lies over sixteen lanes. c, s: the pair's cosine
// and sine for each of the lane's eight elements.
struct Turn {
    float c[8], s[8];
};

// The lane's cosines and sines; NaN for a position that the tables lack.
__device__ __forceinline__ void load_turn(const KvAppend& a, int32_t pos, uint32_t e0, Turn& t) {
    const uint32_t half = a.rotary_dim / 2;
    const bool known = pos >= 0 && pos < int64_t(a.n_positions);
    const float* cs = a.cos_table + uint64_t(known ? pos : 0) * half;
    const float* sn = a.sin_table + uint64_t(known ? pos : 0) * half;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t e = e0 + i;
        t.c[i] = 1.0f;
        t.s[i] = 0.0f;
        if (e < a.rotary_dim) {
            const uint32_t p = a.interleaved ? e / 2 : e < half ? e : e - half;
            t.c[i] = known ? cs[p] : __int_as_float(0x7FC00000);
            t.s[i] = known ? sn[p] : __int_as_float(0x7FC00000);
        }
    }
}

// Norm (w not null) and rotation of one row, in fp32. `row`: 128 floats of
// shared memory of these sixteen lanes.
__device__ __forceinline__ void norm_turn(const KvAppend& a, float (&x)[8], const float* w, const Turn& t, uint32_t e0,
                                          float* row, uint32_t mask) {
    if (w) {
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
#pragma unroll
        for (int d = 8; d; d >>= 1) ss += __shfl_xor_sync(mask, ss, d, kLanes);
        const float r = 1.0f / sqrtf(ss / float(a.pages.head_dim) + a.eps);
        if (e0 < a.pages.head_dim) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] *= r * w[e0 + i];
        }
    }
    if (!a.rotary_dim) return;
    const uint32_t half = a.rotary_dim / 2;
    __syncwarp(mask);
#pragma unroll
    for (int i = 0; i < 8; ++i) row[e0 + i] = x[i];
    __syncwarp(mask);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t e = e0 + i;
        if (e < a.rotary_dim) {
            const bool second = a.interleaved ? e & 1 : e >= half;
            const uint32_t other = a.interleaved ? e ^ 1 : second ? e - half : e + half;
            const float o = row[other];
            x[i] = second ? x[i] * t.c[i] + o * t.s[i] : x[i] * t.c[i] - o * t.s[i];
        }
    }
}

template <class T, class TI>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ KvAppend a) {
    __shared__ float rows[kGroups][128];
    const uint32_t g = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    const uint32_t mask = 0xFFFFu << (threadIdx.x & 16u);
    const uint32_t t = blockIdx.x, e0 = lane * 8;
    const bool mine = e0 < a.pages.head_dim;
    const uint32_t seq = kv_owner(a.tok, t);
    const KvSeq s = kv_seq(a.pages, a.tok, seq);
    const int32_t i = int32_t(t) - s.first;
    const bool real = i >= 0 && i < s.n;
    const int64_t slot = real ? int64_t(s.len) - s.n + i : -1;
    Turn turn;
    load_turn(a, a.positions ? a.positions[t] : int32_t(slot), e0, turn);
    const uint32_t K = a.pages.kv_heads, D = a.pages.head_dim;
    for (uint32_t h = blockIdx.y * kGroups + g; h < a.q_heads + 2 * K; h += gridDim.y * kGroups) {
        float x[8] = {};
        const bool is_q = h < a.q_heads;
        const uint32_t j = is_q ? h : h - a.q_heads;  // keys, then values
        const bool is_v = !is_q && j >= K;
        const TI* src = is_q   ? static_cast<const TI*>(a.q) + t * a.q_stride + uint64_t(h) * D
                        : is_v ? static_cast<const TI*>(a.v) + t * a.v_stride + uint64_t(j - K) * D
                               : static_cast<const TI*>(a.k) + t * a.k_stride + uint64_t(j) * D;
        if (mine) kv_load8(src + e0, x);
        if (!is_v) norm_turn(a, x, is_q ? a.q_norm : a.k_norm, turn, e0, rows[g], mask);
        T* dst = is_q ? static_cast<T*>(a.q_out) + t * a.q_out_stride + uint64_t(h) * D
                      : reinterpret_cast<T*>(kv_row(a.pages, seq, slot, a.pages.layer, is_v, is_v ? j - K : j));
        if (mine && dst) kv_store8(dst + e0, x);
    }
}

// One thread moves one 16-byte column of every accepted row, eight rows at a
// time: a path ascends, so a row's new slot is at or before its old one, and no
// row is overwritten before it was read.
constexpr uint32_t kCommitThreads = 256;
__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const __grid_constant__ KvCommit c) {
    const uint32_t s = blockIdx.x, per = c.pages.head_dim / 8;
    const uint32_t at = blockIdx.y * kCommitThreads + threadIdx.x;
    if (at >= c.pages.layers * 2 * c.pages.kv_heads * per) return;
    const uint32_t row = at / per, col = at % per;
    const uint32_t head = row % c.pages.kv_heads, which = row / c.pages.kv_heads % 2, layer = row / c.pages.kv_heads / 2;
    const uint32_t n = uint32_t(min(max(c.counts[s], 0), int32_t(c.max_path)));
    const int64_t ctx = c.ctx[s];
    const int32_t* path = c.path + uint64_t(s) * c.max_path;
    for (uint32_t i0 = 0; i0 < n; i0 += 8) {
        uint4 v[8];
        uint4* to[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            to[i] = nullptr;
            const int32_t from = i0 + i < n ? path[i0 + i] : -1;
            if (from < 0 || uint32_t(from) == i0 + i) continue;
            const uint8_t* src = kv_row(c.pages, s, ctx + from, layer, which, head);
            uint8_t* dst = kv_row(c.pages, s, ctx + i0 + i, layer, which, head);
            if (!src || !dst) continue;
            v[i] = *reinterpret_cast<const uint4*>(src + col * 16);
            to[i] = reinterpret_cast<uint4*>(dst + col * 16);
        }
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (to[i]) *to[i] = v[i];
    }
}

template <class T, class TI>
cudaError_t append_as(const KvAppend& a, cudaStream_t stream) {
    const uint32_t heads = a.q_heads + 2 * a.pages.kv_heads;
    // a few tokens: a head to a group, over as many blocks as that takes
    const uint32_t y = a.tok.n_tokens >= 1024 ? 1 : (heads + kGroups - 1) / kGroups;
    append_kernel<T, TI><<<dim3(a.tok.n_tokens, y), kThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv_append(const KvAppend& a, uint32_t dtype, uint32_t in_dtype, cudaStream_t stream) {
    if (dtype == T2I_BF16) {
        if (in_dtype == T2I_F32) return append_as<__nv_bfloat16, float>(a, stream);
        if (in_dtype == T2I_F16) return append_as<__nv_bfloat16, __half>(a, stream);
        return append_as<__nv_bfloat16, __nv_bfloat16>(a, stream);
    }
    if (in_dtype == T2I_F32) return append_as<__half, float>(a, stream);
    if (in_dtype == T2I_F16) return append_as<__half, __half>(a, stream);
    return append_as<__half, __nv_bfloat16>(a, stream);
}

cudaError_t launch_kv_commit(const KvCommit& c, cudaStream_t stream) {
    const uint32_t cols = c.pages.layers * 2 * c.pages.kv_heads * (c.pages.head_dim / 8);
    commit_kernel<<<dim3(c.n_seqs, (cols + kCommitThreads - 1) / kCommitThreads), kCommitThreads, 0, stream>>>(c);
    return cudaGetLastError();
}

}  // namespace t2i
