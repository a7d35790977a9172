// Accumulated attention: what each slot gets from new tokens.
#pragma once

#include "kv_attend.cuh"
#include "t2istore.h"

namespace t2i {
namespace {

// A thread a slot.
template <class T>
__global__ void __launch_bounds__(128) weigh_kernel(const __grid_constant__ KvWeigh w) {
    const KvAttend& a = w.a;
    __shared__ float qs[128];
    tc::pdl_launch();
    tc::pdl_wait();
    const uint32_t s = blockIdx.y / a.pages.kv_heads, h = blockIdx.y % a.pages.kv_heads, D = a.pages.head_dim;
    const KvSeq q = kv_seq(a.pages, a.tok, s);
    const int32_t ctx = q.len - q.n, m = min(q.n, int32_t(a.tok.max_new));
    for (int64_t j0 = int64_t(blockIdx.x) * 128; j0 < q.len; j0 += int64_t(gridDim.x) * 128) {
        const int32_t j = int32_t(j0) + int32_t(threadIdx.x);
        const T* key = j < q.len ? reinterpret_cast<const T*>(kv_row(a.pages, s, j, a.pages.layer, 0, h)) : nullptr;
        KvSum sum;
        for (int32_t i = 0; i < m; ++i) {
            const KvQuery y = kv_query(a, q, i);
            const bool see = j < q.len && (j >= y.first || j < int32_t(a.sinks)) && j < y.last;
            for (uint32_t g = 0; g < a.group; ++g) {
                const uint32_t head = h * a.group + g;
                __syncthreads();
                if (threadIdx.x < D)
                    qs[threadIdx.x] = float(static_cast<const T*>(a.q)[uint64_t(q.first + i) * a.q_stride + head * D + threadIdx.x]);
                __syncthreads();
                if (!see) continue;
                float x = 0.0f;
                if (key)
                    for (uint32_t d = 0; d < D; d += 8) {
                        float k[8];
                        kv_load8(key + d, k);
                        for (int e = 0; e < 8; ++e) x += k[e] * qs[d + e];
                    }
                x *= a.scale;
                if (a.softcap != 0.0f) x = a.softcap * tanhf(x / a.softcap);
                if (a.slopes) x -= a.slopes[head] * fabsf(float(y.pos - j));
                const float lse = w.lse[uint64_t(q.first + i) * a.q_heads + head];
                if (lse != -INFINITY) sum.add(expf(x - lse));
            }
        }
        if (j < q.len && uint32_t(j) < w.n_slots) {
            float* at = w.weights + s * w.seq_stride + h * w.head_stride + j;
            *at = sum.value() + (j < ctx && w.decay != 0.0f ? w.decay * *at : 0.0f);
        }
    }
}

template <class T>
cudaError_t launch_weigh(const KvWeigh& w, const KvLaunch& l, cudaStream_t stream) {
    return launch_pdl(weigh_kernel<T>, dim3((w.a.max_len + 127) / 128, w.a.tok.n_seqs * w.a.pages.kv_heads), 128, 0, stream, w);
}

}  // namespace
}  // namespace t2i
