// Appending keys and values to the cache (per-head RMS norm and rotation of
// queries and keys on the way), and keeping the accepted rows of a draft.
#include "kv_attend.cuh"
#include "t2istore.h"

namespace t2i {
namespace {

// Sixteen lanes hold a head's row, eight elements a lane, so that a row is one
// 16-byte vector a lane and a norm's sum four shuffles. A block takes one token (or a
// share of its heads): its cosines, sines, norm weights and place in the cache are
// looked up once for all heads, and each group of sixteen lanes loads its next head
// before it works on the one it has. Bound by memory at many tokens (each byte is
// read and written once), by the chain of look-ups at few. Measured: seven prompts of 8.7k
// tokens in all, 32 + 2 x 8 heads of 128, norms and interleaved pairs, 45 us (4.8 TB/s); 192 tokens
// from fp32 5.2 us, one token 2.3 us (in a graph of 50 calls).
constexpr uint32_t kLanes = 16;
constexpr uint32_t kThreads = 64;  // (of 256, 128, 64, 32: prompts of 8.7k tokens 58.8, 47.4, 46.2, 54.0 us)
constexpr uint32_t kGroups = kThreads / kLanes;

// How a pair's other element is reached: interleaved pairs lie in one lane; halves
// that are multiples of eight elements lie at the same place in another lane; others
// go through shared memory.
enum Turn : int { kNone, kInLane, kAcross, kAnywhere };

// Eight elements as they are loaded.
template <class T>
struct Raw {
    uint4 v[sizeof(T) / 2];
};
template <class T>
__device__ __forceinline__ void unpack(const Raw<T>& r, float (&x)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x[4 * i] = __uint_as_float(r.v[i].x), x[4 * i + 1] = __uint_as_float(r.v[i].y);
            x[4 * i + 2] = __uint_as_float(r.v[i].z), x[4 * i + 3] = __uint_as_float(r.v[i].w);
        }
    } else {
        const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = Kv16<T>::to2(w[i]);
            x[2 * i] = f.x, x[2 * i + 1] = f.y;
        }
    }
}

// Eight floats, in two vectors where their address allows it.
__device__ __forceinline__ void eight(const float* p, float (&x)[8], uint32_t vectors) {
    if (vectors) {
        const float4 u = reinterpret_cast<const float4*>(p)[0], v = reinterpret_cast<const float4*>(p)[1];
        x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = p[i];
    }
}

template <class T, class TI, int TURN>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ KvAppend a) {
    __shared__ float rows[TURN == kAnywhere ? kGroups : 1][128];
    const uint32_t g = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    const uint32_t mask = 0xFFFFu << (threadIdx.x & 16u);
    const uint32_t t = blockIdx.x, e0 = lane * 8;
    const uint32_t K = a.pages.kv_heads, D = a.pages.head_dim, heads = a.q_heads + 2 * K, step = gridDim.y * kGroups;
    const bool mine = e0 < D;
    tc::pdl_launch();
    tc::pdl_wait();
    // the token's rows: head h of queries, then keys, then values lies h rows behind these
    const uint32_t in_row = D * uint32_t(sizeof(TI)), QK = a.q_heads + K;
    const uint8_t* const q0 = reinterpret_cast<const uint8_t*>(static_cast<const TI*>(a.q) + t * a.q_stride + e0);
    const uint8_t* const k0 = reinterpret_cast<const uint8_t*>(static_cast<const TI*>(a.k) + t * a.k_stride + e0) - uint64_t(a.q_heads) * in_row;
    const uint8_t* const v0 = reinterpret_cast<const uint8_t*>(static_cast<const TI*>(a.v) + t * a.v_stride + e0) - uint64_t(QK) * in_row;
    auto load = [&](uint32_t h) {
        Raw<TI> r{};
        if (!mine) return r;
        const uint8_t* src = (h < a.q_heads ? q0 : h < QK ? k0 : v0) + uint64_t(h) * in_row;
#pragma unroll
        for (uint32_t i = 0; i < sizeof(TI) / 2; ++i) r.v[i] = reinterpret_cast<const uint4*>(src)[i];
        return r;
    };
    uint32_t h = blockIdx.y * kGroups + g;
    Raw<TI> next{};
    if (h < heads) next = load(h);
    float wq[8] = {}, wk[8] = {};
    if (mine && a.q_norm) eight(a.q_norm + e0, wq, a.vectors);
    if (mine && a.k_norm) eight(a.k_norm + e0, wk, a.vectors);

    const uint32_t seq = kv_owner(a.tok, t);
    const KvSeq s = kv_seq(a.pages, a.tok, seq);
    const int32_t i = int32_t(t) - s.first;
    const int64_t slot = i >= 0 && i < s.n ? int64_t(s.len) - s.n + i : -1;
    // the token's first row in the cache (key head 0 of the layer), and from head to head
    uint8_t* const place = kv_row(a.pages, seq, slot, a.pages.layer, 0, 0);
    const uint64_t apart = uint64_t(D * 2) << a.pages.token_shift;
    uint8_t* const cache0 = place + e0 * 2 - a.q_heads * apart;
    uint8_t* const out0 = reinterpret_cast<uint8_t*>(static_cast<T*>(a.q_out) + t * a.q_out_stride + e0);

    // the pair's cosine and sine for each of the lane's elements; NaN for a position that the tables lack
    float co[8], si[8];
    const uint32_t half = a.rotary_dim / 2;
    if (TURN != kNone) {
        const int32_t pos = a.positions ? a.positions[t] : int32_t(slot);
        const bool known = pos >= 0 && pos < int64_t(a.n_positions);
        const float* cs = a.cos_table + uint64_t(known ? pos : 0) * half;
        const float* sn = a.sin_table + uint64_t(known ? pos : 0) * half;
        if (TURN == kAcross && e0 < a.rotary_dim) {
            const uint32_t p = e0 < half ? e0 : e0 - half;
            eight(cs + p, co, a.vectors);
            eight(sn + p, si, a.vectors);
        } else {
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) {
                const uint32_t e = e0 + k;
                co[k] = 1.0f, si[k] = 0.0f;
                if (e < a.rotary_dim) {
                    const uint32_t p = TURN == kInLane || a.interleaved ? e / 2 : e < half ? e : e - half;
                    co[k] = cs[p], si[k] = sn[p];
                }
            }
        }
        if (!known && e0 < a.rotary_dim) {
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k)
                if (e0 + k < a.rotary_dim) co[k] = si[k] = __int_as_float(0x7FC00000);
        }
    }

    const float per_dim = 1.0f / float(D);
    for (; h < heads; h += step) {
        const Raw<TI> raw = next;
        if (h + step < heads) next = load(h + step);
        float x[8];
        unpack<TI>(raw, x);
        const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + K;
        if (!is_v && (is_q ? a.q_norm : a.k_norm)) {
            float ss = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) ss += x[k] * x[k];
#pragma unroll
            for (int d = 8; d; d >>= 1) ss += __shfl_xor_sync(mask, ss, d, kLanes);
            const float r = rsqrtf(ss * per_dim + a.eps);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] *= r * (is_q ? wq[k] : wk[k]);
        }
        if (TURN != kNone && !is_v) {
            if (TURN == kInLane) {
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    const float u = x[k], v = x[k + 1];
                    x[k] = u * co[k] - v * si[k];
                    x[k + 1] = v * co[k] + u * si[k];
                }
            } else if (TURN == kAcross) {
                const bool turned = e0 < a.rotary_dim, second = e0 >= half;
                const int from = int(lane) + (!turned ? 0 : second ? -int(half / 8) : int(half / 8));
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float o = __shfl_sync(mask, x[k], from, kLanes);
                    if (turned) x[k] = second ? x[k] * co[k] + o * si[k] : x[k] * co[k] - o * si[k];
                }
            } else {
                float* row = rows[g % (TURN == kAnywhere ? kGroups : 1)];
                __syncwarp(mask);
#pragma unroll
                for (int k = 0; k < 8; ++k) row[e0 + k] = x[k];
                __syncwarp(mask);
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) {
                    const uint32_t e = e0 + k;
                    if (e < a.rotary_dim) {
                        const bool second = a.interleaved ? e & 1 : e >= half;
                        const float o = row[a.interleaved ? e ^ 1 : second ? e - half : e + half];
                        x[k] = second ? x[k] * co[k] + o * si[k] : x[k] * co[k] - o * si[k];
                    }
                }
            }
        }
        uint8_t* const dst = is_q ? out0 + uint64_t(h) * (D * 2) : cache0 + uint64_t(h) * apart;
        if (mine && (is_q || place)) kv_store8(reinterpret_cast<T*>(dst), x);
    }
}

// One thread moves one 16-byte column of every accepted row, eight rows at a
// time: a path ascends, so a row's new slot is at or before its old one, and no
// row is overwritten before it was read. Bound by memory at many sequences: paths of six
// rows of 96 sequences in 28 layers, 8 heads of 128, 25 us (3.9 TB/s); by the launch's
// latency at few: one path in a layer 2.3 us (in a graph of 50 calls).
constexpr uint32_t kCommitThreads = 256;
__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const __grid_constant__ KvCommit c) {
    tc::pdl_launch();
    tc::pdl_wait();
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
cudaError_t append_as(const KvAppend& args, cudaStream_t stream) {
    KvAppend a = args;
    const uint64_t at = reinterpret_cast<uint64_t>(a.cos_table) | reinterpret_cast<uint64_t>(a.sin_table) |
                        reinterpret_cast<uint64_t>(a.q_norm) | reinterpret_cast<uint64_t>(a.k_norm);
    a.vectors = at % 16 == 0 && a.rotary_dim % 8 == 0;  // (half a row of the tables: a multiple of four floats)
    const uint32_t heads = a.q_heads + 2 * a.pages.kv_heads;
    // a few tokens: a head to a group, over as many blocks as that takes. So / a block a token, 32 + 2 x 8 heads, us: 1
    // token 2.9 / 10.4, 256 6.1 / 10.7, 768 13.1 / 14.2, 1,024 16.3 / 14.3, 4,096 57 / 29.
    const dim3 grid(a.tok.n_tokens, a.tok.n_tokens >= 1024 ? 1 : (heads + kGroups - 1) / kGroups);
    if (!a.rotary_dim) return launch_pdl(append_kernel<T, TI, kNone>, grid, kThreads, 0, stream, a);
    if (a.interleaved && a.rotary_dim % 8 == 0) return launch_pdl(append_kernel<T, TI, kInLane>, grid, kThreads, 0, stream, a);
    if (!a.interleaved && a.rotary_dim % 16 == 0) return launch_pdl(append_kernel<T, TI, kAcross>, grid, kThreads, 0, stream, a);
    return launch_pdl(append_kernel<T, TI, kAnywhere>, grid, kThreads, 0, stream, a);
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
    return launch_pdl(commit_kernel, dim3(c.n_seqs, (cols + kCommitThreads - 1) / kCommitThreads), kCommitThreads, 0, stream, c);
}

}  // namespace t2i
