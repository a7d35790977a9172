// Keeping a cache bounded: which slots of a sequence stay (by their accumulated
// attention), and their rows moved together.
#include <cooperative_groups.h>

#include <algorithm>
#include <atomic>

#include "kv_attend.cuh"
#include "t2istore.h"

namespace t2i {
namespace {

namespace cg = cooperative_groups;

// ------------------------------------------------------------------ select
// The r largest of a row's weights, of equals the first: the r-th largest is found by its bits (weights as numbers whose
// order is that of the integers, NaN as the lowest), eleven, eleven and ten at a time, from counts of each value of
// these bits; then one pass in the order of slots writes those above it and the first ones equal to it. Counts are
// integers, so their order does not matter. A cluster of blocks shares a row; each has its part of the row in shared
// memory, so that weights are read once, and adds up the counts of all. A part that does not fit is read from memory
// in each pass.
constexpr uint32_t kSelThreads = 512;
constexpr uint32_t kSelWarps = kSelThreads / 32;
constexpr uint32_t kBins = 2048;
constexpr uint32_t kMostBlocks = 8;  // of a cluster
constexpr uint32_t kPartMost = 40960;  // weights of a part in shared memory: 160 KiB

// A weight's place in the order: 0 for NaN, 0 and -0 alike.
__device__ __forceinline__ uint32_t order_of(float w) {
    if (w != w) return 0;
    const uint32_t b = __float_as_uint(w + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct SelShared {
    uint32_t hist[3][kBins];
    uint32_t warp_sums[2][kSelWarps];
    uint32_t base[2][kSelWarps];  // such slots of the warps before, in the block
    uint32_t mine[2];     // this block's slots above the threshold (or staying whatever they weigh), and equal to it
    uint32_t bin, above, in;
};

__global__ void __launch_bounds__(kSelThreads) select_kernel(const __grid_constant__ KvSelect c, const uint32_t part_room) {
    extern __shared__ float part[];
    __shared__ SelShared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t blocks = cluster.num_blocks(), rank = cluster.block_rank();
    const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const uint32_t row = blockIdx.x / blocks, s = row / c.n_heads, head = row % c.n_heads;
    for (uint32_t i = tid; i < 3 * kBins; i += kSelThreads) (&sh.hist[0][0])[i] = 0;
    tc::pdl_launch();
    tc::pdl_wait();
    const int32_t given = c.lens[s];
    const uint32_t len = given > 0 && uint32_t(given) <= c.n_slots ? uint32_t(given) : 0;
    uint32_t n = min(len, c.keep);
    if (c.keeps) n = min(n, uint32_t(max(c.keeps[s], 0)));
    const uint32_t a = min(c.sinks, n), b = min(c.recent, n - a);
    if (tid == 0 && rank == 0 && head == 0) c.counts[s] = int32_t(n);
    const float* const w = c.weights + s * c.seq_stride + head * c.head_stride;
    float* const out = c.weights_out ? c.weights_out + s * c.out_seq_stride + head * c.out_head_stride : nullptr;
    int32_t* const kept = c.kept + s * c.kept_seq_stride + head * c.kept_head_stride;
    if (n == 0) return;  // (of all of the cluster's blocks)

    // this block's slots, and in it those that are chosen by weight
    const uint32_t per = (len + blocks - 1) / blocks;
    const uint32_t j0 = min(len, rank * per), j1 = min(len, j0 + per);
    const uint32_t f0 = max(j0, a), f1 = min(j1, len - b);
    const bool here = per <= part_room;
    if (here)
        for (uint32_t j = j0 + tid; j < j1; j += kSelThreads) part[j - j0] = w[j];
    __syncthreads();
    auto at = [&](uint32_t j) { return here ? part[j - j0] : w[j]; };

    // the threshold: weights above `edge` stay, and the first `ties` of those equal to it
    uint32_t need = n - a - b, edge = 0xFFFFFFFFu, ties = 0;
    if (need == len - a - b) {
        edge = 0, ties = need;
    } else if (need) {
        uint32_t prefix = 0, known = 0;  // the leading bits so far, and how many
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const uint32_t bits = pass < 2 ? 11 : 10, shift = 32 - known - bits;
            uint32_t* const h = sh.hist[pass];
            for (uint32_t j = f0 + tid; j < f1; j += kSelThreads) {
                const uint32_t k = order_of(at(j));
                if (known == 0 || k >> (32 - known) == prefix) atomicAdd(&h[k >> shift & ((1u << bits) - 1)], 1u);
            }
            cluster.sync();
            // each thread: four bins, highest first, of all blocks
            uint32_t v[4] = {0, 0, 0, 0};
            const uint32_t b0 = kBins - 4 - tid * 4;
            for (uint32_t r = 0; r < blocks; ++r) {
                const uint4 x = *reinterpret_cast<const uint4*>(cluster.map_shared_rank(h, r) + b0);
                v[0] += x.w, v[1] += x.z, v[2] += x.y, v[3] += x.x;
            }
            const uint32_t sum = v[0] + v[1] + v[2] + v[3];
            uint32_t inc = sum;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, inc, d);
                if (lane >= uint32_t(d)) inc += o;
            }
            if (lane == 31) sh.warp_sums[0][warp] = inc;
            __syncthreads();
            uint32_t before = inc - sum;
            for (uint32_t i = 0; i < warp; ++i) before += sh.warp_sums[0][i];
            if (before < need && before + sum >= need) {
                int i = 0;
                while (before + v[i] < need) before += v[i++];
                sh.bin = b0 + 3 - i, sh.above = before, sh.in = v[i];
            }
            __syncthreads();
            prefix = prefix << bits | sh.bin;
            known += bits;
            need -= sh.above;
            const bool all = sh.in == need;  // the whole bin stays
            edge = known == 32 ? prefix : prefix << (32 - known);
            ties = need;
            __syncthreads();
            if (all) {
                if (known < 32) --edge, ties = 0;  // (edge > 0: a bin 0 with all of the rest would be every slot)
                break;
            }
        }
    }
    // in the order of slots: a warp has a stretch of the block's, counts it, and writes
    const uint32_t stretch = ((j1 - j0 + kSelWarps - 1) / kSelWarps + 31) / 32 * 32;
    const uint32_t w0 = min(j1, j0 + warp * stretch), w1 = min(j1, w0 + stretch);
    auto look = [&](uint32_t j, bool& over, bool& equal) {
        over = equal = false;
        if (j >= w1) return 0.0f;
        const float x = at(j);
        const bool held = j < a || j >= len - b;
        const uint32_t k = order_of(x);
        over = held || k > edge;
        equal = !held && k == edge;
        return x;
    };
    uint32_t overs = 0, equals = 0;
    for (uint32_t j = w0; j < w1; j += 32) {
        bool over, equal;
        look(j + lane, over, equal);
        overs += __popc(__ballot_sync(0xFFFFFFFFu, over));
        equals += __popc(__ballot_sync(0xFFFFFFFFu, equal));
    }
    if (lane == 0) sh.warp_sums[0][warp] = overs, sh.warp_sums[1][warp] = equals;
    __syncthreads();
    overs = equals = 0;
    for (uint32_t i = 0; i < kSelWarps; ++i) {
        if (i == warp && lane == 0) sh.base[0][warp] = overs, sh.base[1][warp] = equals;
        overs += sh.warp_sums[0][i], equals += sh.warp_sums[1][i];
    }
    if (tid == 0) sh.mine[0] = overs, sh.mine[1] = equals;
    cluster.sync();
    overs = sh.base[0][warp], equals = sh.base[1][warp];
    for (uint32_t r = 0; r < rank; ++r) {
        const uint32_t* m = cluster.map_shared_rank(sh.mine, r);
        overs += m[0], equals += m[1];
    }
    const bool copy = out && (here || out != w);
    for (uint32_t j = w0; j < w1; j += 32) {
        bool over, equal;
        const float x = look(j + lane, over, equal);
        const uint32_t mo = __ballot_sync(0xFFFFFFFFu, over), me = __ballot_sync(0xFFFFFFFFu, equal), lower = (1u << lane) - 1;
        const uint32_t e = equals + __popc(me & lower);
        const uint32_t to = overs + __popc(mo & lower) + min(e, ties);
        if (over || (equal && e < ties)) {
            kept[to] = int32_t(j + lane);
            if (copy) out[to] = x;
        }
        overs += __popc(mo), equals += __popc(me);
    }
    cluster.sync();  // (shared memory lives until the others have read it; and kept is complete)
    if (out && !copy && rank == 0) {
        // in place, from memory: a slot's weight moves down, so a stretch is read before it is written over
        for (uint32_t i0 = 0; i0 < n; i0 += kSelThreads) {
            const uint32_t i = i0 + tid;
            float x = 0.0f;
            if (i < n) x = __ldcg(w + __ldcg(kept + i));
            __syncthreads();
            if (i < n) out[i] = x;
            __syncthreads();
        }
    }
}

// ------------------------------------------------------------------ evict
// A block moves the rows of one key head's keys or values (or a share of their columns), a chunk of rows at a time: all
// of a chunk's loads come before its stores, and a row's new slot is at or before its old one, so no row is overwritten
// before it was read.
constexpr uint32_t kEvictThreads = 256;
constexpr uint32_t kEvictDeep = 8;  // rows of a thread in a chunk
__global__ void __launch_bounds__(kEvictThreads) evict_kernel(const __grid_constant__ KvEvict c, const uint32_t cols) {
    tc::pdl_launch();
    tc::pdl_wait();
    const KvPages& p = c.pages;
    const uint32_t s = blockIdx.x / p.kv_heads, head = blockIdx.x % p.kv_heads;
    const uint32_t which = blockIdx.y % 2, layer = p.layer + blockIdx.y / 2;
    const uint32_t rows = kEvictThreads / cols, r = threadIdx.x / cols, col = blockIdx.z * cols + threadIdx.x % cols;
    const bool mine = r < rows && col * 8 < p.head_dim;
    const uint32_t n = uint32_t(min(max(c.counts[s], 0), int32_t(c.max_kept)));
    const int32_t* const kept = c.kept + s * c.kept_seq_stride + head * c.kept_head_stride;
    for (uint32_t i0 = 0; i0 < n; i0 += rows * kEvictDeep) {
        uint4 v[kEvictDeep];
        uint4* to[kEvictDeep];
#pragma unroll
        for (uint32_t k = 0; k < kEvictDeep; ++k) {
            const uint32_t i = i0 + k * rows + r;
            to[k] = nullptr;
            if (!mine || i >= n) continue;
            const int32_t from = kept[i];
            if (from <= int32_t(i)) continue;
            const uint8_t* src = kv_row(p, s, from, layer, which, head);
            uint8_t* dst = kv_row(p, s, i, layer, which, head);
            if (!src || !dst) continue;
            v[k] = *reinterpret_cast<const uint4*>(src + col * 16);
            to[k] = reinterpret_cast<uint4*>(dst + col * 16);
        }
        __syncthreads();
#pragma unroll
        for (uint32_t k = 0; k < kEvictDeep; ++k)
            if (to[k]) *to[k] = v[k];
    }
}

}  // namespace

cudaError_t launch_kv_select(const KvSelect& c, uint32_t sms, cudaStream_t stream) {
    const uint32_t rows = c.n_seqs * c.n_heads;
    const uint32_t most = c.max_len;
    uint32_t blocks = 1;
    while (blocks < kMostBlocks && (most / blocks > kPartMost || (most / blocks > 2048 && rows * blocks * 2 <= sms * 2))) blocks *= 2;
    const uint32_t room = std::min((most + blocks - 1) / blocks, kPartMost);
    static std::atomic<uint64_t> ready{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !(ready.load() >> dev & 1)) {
        e = cudaFuncSetAttribute(select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kPartMost * 4));
        if (e != cudaSuccess) return e;
        if (dev < 64) ready |= uint64_t(1) << dev;
    }
    cudaLaunchConfig_t l{};
    l.gridDim = dim3(rows * blocks);
    l.blockDim = dim3(kSelThreads);
    l.dynamicSmemBytes = room * 4;
    l.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = blocks, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    l.attrs = at;
    l.numAttrs = 2;
    return cudaLaunchKernelEx(&l, select_kernel, c, room);
}

cudaError_t launch_kv_evict(const KvEvict& c, uint32_t sms, cudaStream_t stream) {
    const uint32_t vectors = c.pages.head_dim / 8;
    const uint64_t units = uint64_t(c.n_seqs) * c.pages.kv_heads * 2 * c.layers;
    // few units: a block has a share of the columns, of 32 bytes at least
    uint32_t parts = 1;
    while (parts < 8 && units * parts < 2 * sms && vectors / parts >= 4) parts *= 2;
    const uint32_t cols = (vectors + parts - 1) / parts;
    return launch_pdl(evict_kernel, dim3(c.n_seqs * c.pages.kv_heads, 2 * c.layers, parts), kEvictThreads, 0, stream, c, cols);
}

}  // namespace t2i
