// Attention over the cache: one warp a token and head.
#include "kv_device.cuh"
#include "t2istore.h"

namespace t2i {
namespace {

template <class T>
__global__ void __launch_bounds__(128) attend_kernel(const __grid_constant__ KvAttend a) {
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t t = blockIdx.x, h = blockIdx.y * 4 + warp;
    const uint32_t seq = kv_owner(a.tok, t);
    if (h >= a.q_heads) return;
    const KvSeq s = kv_seq(a.pages, a.tok, seq);
    const int32_t i = int32_t(t) - s.first;
    if (i < 0 || i >= s.n || i >= int32_t(a.tok.max_new)) return;
    const uint32_t D = a.pages.head_dim, e0 = lane * 4, kh = h / a.group;
    const int32_t ctx = s.len - s.n;
    const uint64_t word = a.tree ? a.tree[t] : 0;
    const int32_t pos = a.tree ? ctx + __popcll(word) - 1 : ctx + i;
    int32_t lo = 0, hi = pos + 1;
    if (a.tree) hi = s.len;
    if (a.spans) lo = max(a.spans[2 * t], 0), hi = min(a.spans[2 * t + 1], s.len);
    const float slope = a.slopes ? a.slopes[h] : 0.0f;
    float q[4] = {}, o[4] = {}, m = -INFINITY, l = 0.0f;
    const bool mine = e0 < D;
    auto load4 = [&](const void* p, float (&x)[4]) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        const float2 u = Kv16<T>::to2(v.x), w = Kv16<T>::to2(v.y);
        x[0] = u.x, x[1] = u.y, x[2] = w.x, x[3] = w.y;
    };
    if (mine) load4(static_cast<const T*>(a.q) + t * a.q_stride + uint64_t(h) * D + e0, q);
    for (int32_t j = lo; j < hi; ++j) {
        int32_t kpos = j;
        if (a.tree && j >= ctx) {
            if (!(word >> (j - ctx) & 1)) continue;
            kpos = ctx + __popcll(a.tree[s.first + j - ctx]) - 1;
        }
        if (a.window && kpos <= pos - int64_t(a.window)) continue;
        const uint8_t* kr = kv_row(a.pages, seq, j, a.pages.layer, 0, kh);
        float k[4] = {}, v[4] = {};
        if (mine && kr) {
            load4(kr + e0 * 2, k);
            load4(kv_row(a.pages, seq, j, a.pages.layer, 1, kh) + e0 * 2, v);
        }
        float x = q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3];
#pragma unroll
        for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
        x *= a.scale;
        if (a.softcap != 0.0f) x = a.softcap * tanhf(x / a.softcap);
        x -= slope * fabsf(float(pos - kpos));
        const float top = fmaxf(m, x), c = expf(m - top), p = expf(x - top);
        m = top;
        l = l * c + p;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] * c + p * v[e];
    }
    const float r = l > 0.0f ? 1.0f / l : 0.0f;
    if (mine)
        *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + t * a.out_stride + uint64_t(h) * D + e0) =
            make_uint2(Kv16<T>::from2(o[0] * r, o[1] * r), Kv16<T>::from2(o[2] * r, o[3] * r));
    if (a.lse && lane == 0) a.lse[uint64_t(t) * a.q_heads + h] = l > 0.0f ? m + logf(l) : -INFINITY;
}

}  // namespace

cudaError_t launch_kv_attend(const KvAttend& a, uint32_t dtype, cudaStream_t stream) {
    const dim3 grid(a.tok.n_tokens, (a.q_heads + 3) / 4);
    if (dtype == T2I_BF16)
        attend_kernel<__nv_bfloat16><<<grid, 128, 0, stream>>>(a);
    else
        attend_kernel<__half><<<grid, 128, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace t2i
