// Keeping a cache bounded: which slots of a sequence stay (by their accumulated
// attention), and their rows moved together.
#include <cooperative_groups.h>

#include <algorithm>

#include "kv_attend.cuh"
#include "t2istore.h"

namespace t2i {
namespace {

namespace cg = cooperative_groups;

// ------------------------------------------------------------------ select
// The r largest of a row's weights, of equals the first: the r-th largest is found by its bits (weights as numbers whose
// order is that of the integers, NaN as the lowest), eleven, eleven and ten at a time, from counts of each value of
// these bits; then one pass in the order of slots writes those above it and the first ones equal to it. Counts are
// integers, so their order does not matter. A cluster of blocks shares a row and adds up the counts of all of them. A
// warp has a stretch of its block's slots, I to a lane, in registers, so that weights are read once; a row that is longer
// than its caller said, or than a cluster holds (131,072), is read from memory in each pass.
// Bound by instructions: some 75 for each 32 weights (order, counts, votes, places) and 500 a warp beside them. Measured: 64
// x 8 rows of up to 16k slots to 4k 32-33 us, 8 rows of 131k to 8k 21 us, 8 of 1,100 6.4 us. In shared memory in place of
// registers the first took 57 us, in blocks of 512 threads 35.
constexpr uint32_t kSelThreads = 1024;
constexpr uint32_t kSelWarps = kSelThreads / 32;
constexpr uint32_t kBins = 2048;
constexpr uint32_t kMostBlocks = 8;  // of a cluster

// A weight's place in the order: 0 for NaN, 0 and -0 alike.
__device__ __forceinline__ uint32_t order_of(float w) {
    const uint32_t b = __float_as_uint(w + 0.0f);
    const uint32_t k = b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
    return w != w ? 0 : k;
}
constexpr uint32_t kLowest = 0x007FFFFFu, kHighest = 0xFF800000u;  // of -infinity and infinity
__device__ __forceinline__ float weight_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

struct SelShared {
    uint32_t hist[3][kBins];
    uint32_t warp_sums[2][kSelWarps];
    uint32_t mine[2];     // this block's slots above the threshold (or staying whatever they weigh), and equal to it
    uint32_t bin, above, in;
};

// One row, by a cluster. HELD: a lane's I weights are in registers.
template <int I, bool HELD>
__device__ __forceinline__ void select_row(const KvSelect& c, SelShared& sh, uint32_t s, uint32_t head, uint32_t len, uint32_t n) {
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t blocks = cluster.num_blocks(), rank = cluster.block_rank();
    const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const uint32_t a = min(c.sinks, n), b = min(c.recent, n - a);
    const float* const w = c.weights + s * c.seq_stride + head * c.head_stride;
    float* const out = c.weights_out ? c.weights_out + s * c.out_seq_stride + head * c.out_head_stride : nullptr;
    int32_t* const kept = c.kept + s * c.kept_seq_stride + head * c.kept_head_stride;
    auto sync = [&]() {
        if (blocks > 1)
            cluster.sync();
        else
            __syncthreads();
    };
    // the warp's slots, and in it those that are chosen by weight
    const uint32_t stretch = (len + blocks * kSelThreads - 1) / (blocks * kSelThreads) * 32;
    const uint32_t w0 = min(uint64_t(len), uint64_t(rank * kSelWarps + warp) * stretch), w1 = min(len, w0 + stretch);
    const int mine = int((w1 - w0 + 31) / 32);  // of each lane, the last one maybe not
    float held[HELD ? I : 1];
    if (HELD) {
#pragma unroll
        for (int i = 0; i < I; ++i) held[i] = w0 + i * 32 + lane < w1 ? w[w0 + i * 32 + lane] : 0.0f;
    }
    // f(slot, weight) for the lane's slots in turn, also (with any weight) for those from w1 on
    auto each = [&](auto&& f) {
        if constexpr (HELD) {
#pragma unroll
            for (int i = 0; i < I; ++i) {
                if (i >= mine) break;
                f(w0 + i * 32 + lane, held[i]);
            }
        } else {
            for (uint32_t j = w0; j < w1; j += 32) f(j + lane, j + lane < w1 ? w[j + lane] : 0.0f);
        }
    };

    // the lane's slots that are there, and those that are chosen by weight, a bit each (HELD)
    uint32_t live = 0, choice = 0;
    if (HELD) {
        auto below = [](uint32_t n) { return n >= 32 ? ~0u : (1u << n) - 1; };  // of slots at 32 i + lane
        auto bits = [&](uint32_t j) { return below(j > w0 + lane ? (j - w0 - lane + 31) / 32 : 0); };
        live = bits(w1), choice = bits(min(w1, len - b)) & ~bits(a);
    }

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
            if (pass)
                for (uint32_t i = tid; i < kBins / 4; i += kSelThreads) reinterpret_cast<uint4*>(h)[i] = make_uint4(0, 0, 0, 0);
            if (pass) __syncthreads();  // (the first one's are zeros from the start)
            // numbers between these have the leading bits (NaN, and what no number has, are not looked for by them)
            const uint32_t lo = known ? prefix << (32 - known) : 0, hi = known ? lo + (0xFFFFFFFFu >> known) : 0xFFFFFFFFu;
            if (HELD && pass == 0) {
#pragma unroll
                for (int i = 0; i < I; ++i) {
                    if (i >= mine) break;
                    if (choice >> i & 1) atomicAdd(&h[order_of(held[HELD ? i : 0]) >> 21], 1u);
                }
            } else if (HELD && lo >= kLowest) {
                const float from = weight_of(lo), upto = weight_of(hi == 0x7FFFFFFFu ? hi - 1 : min(hi, kHighest));
#pragma unroll
                for (int i = 0; i < I; ++i) {
                    if (i >= mine) break;
                    if (held[HELD ? i : 0] >= from && held[HELD ? i : 0] <= upto && (choice >> i & 1))
                        atomicAdd(&h[order_of(held[HELD ? i : 0]) >> shift & ((1u << bits) - 1)], 1u);
                }
            } else {
                uint32_t i = 0;
                each([&](uint32_t j, float x) {
                    const uint32_t k = order_of(x);
                    const bool counts = HELD ? choice >> i++ & 1 : j >= a && j < min(w1, len - b);
                    if (counts && k >= lo && k <= hi) atomicAdd(&h[k >> shift & ((1u << bits) - 1)], 1u);
                });
            }
            sync();
            // each thread: two bins, the higher first, of all blocks
            static_assert(kBins == 2 * kSelThreads, "");
            uint2 v = make_uint2(0, 0);
            const uint32_t b0 = kBins - 2 - tid * 2;
            auto add = [&](const uint2& x) { v.x += x.y, v.y += x.x; };
            if (blocks == 1) {
                add(*reinterpret_cast<const uint2*>(h + b0));
            } else {
                uint2 x[kMostBlocks];
#pragma unroll
                for (uint32_t r = 0; r < kMostBlocks; ++r)
                    x[r] = r < blocks ? *reinterpret_cast<const uint2*>(cluster.map_shared_rank(h, r) + b0) : make_uint2(0, 0);
#pragma unroll
                for (uint32_t r = 0; r < kMostBlocks; ++r) add(x[r]);
            }
            const uint32_t sum = v.x + v.y;
            uint32_t inc = sum;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, inc, d);
                if (lane >= uint32_t(d)) inc += o;
            }
            if (lane == 31) sh.warp_sums[0][warp] = inc;
            __syncthreads();
            uint32_t before = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? sh.warp_sums[0][lane] : 0) + inc - sum;
            if (before < need && before + sum >= need) {
                const bool second = before + v.x < need;
                sh.bin = second ? b0 : b0 + 1, sh.above = second ? before + v.x : before, sh.in = second ? v.y : v.x;
            }
            __syncthreads();
            prefix = prefix << bits | sh.bin;
            known += bits;
            need -= sh.above;
            const bool all = sh.in == need;  // the whole bin stays
            edge = known == 32 ? prefix : prefix << (32 - known);
            ties = need;
            if (all) {
                if (known < 32) --edge, ties = 0;  // (edge > 0: a bin 0 with all of the rest would be every slot)
                break;
            }
        }
    }
    // in the order of slots: a warp counts its stretch, then writes it
    const float at = weight_of(edge == 0x7FFFFFFFu ? edge - 1 : edge);  // (-0 has 0's place: what is above an edge just below that is above -0x1p-149)
    const bool low = edge < kLowest;  // (no number is below: all of them are above)
    auto look = [&](uint32_t j, float x, bool& over, bool& equal) {
        const bool stays = j < a || j >= len - b;
        over = j < w1 && (stays || (low ? x == x : x > at));
        equal = j < w1 && !stays && (edge == 0 ? x != x : x == at);
    };
    uint32_t overs = 0, equals = 0, over_bits = 0, equal_bits = 0;  // (HELD: a bit a slot of the lane)
    if (HELD) {
        if (edge == 0) {
#pragma unroll
            for (int i = 0; i < I; ++i) over_bits |= uint32_t(held[HELD ? i : 0] == held[HELD ? i : 0]) << i;
            equal_bits = choice & ~over_bits;
        } else {
#pragma unroll
            for (int i = 0; i < I; ++i) {
                if (i >= mine) break;
                over_bits |= uint32_t(low ? held[HELD ? i : 0] == held[HELD ? i : 0] : held[HELD ? i : 0] > at) << i;
                equal_bits |= uint32_t(held[HELD ? i : 0] == at) << i;
            }
            equal_bits &= choice;
        }
        over_bits = (over_bits & choice) | (live & ~choice);
        overs = __reduce_add_sync(0xFFFFFFFFu, __popc(over_bits)), equals = __reduce_add_sync(0xFFFFFFFFu, __popc(equal_bits));
    } else {
        each([&](uint32_t j, float x) {
            bool over, equal;
            look(j, x, over, equal);
            overs += __popc(__ballot_sync(0xFFFFFFFFu, over));
            equals += __popc(__ballot_sync(0xFFFFFFFFu, equal));
        });
    }
    const bool none_equal = equals == 0;
    __syncthreads();  // (warp_sums are read)
    if (lane == 0) sh.warp_sums[0][warp] = overs, sh.warp_sums[1][warp] = equals;
    __syncthreads();
    {  // of the warps before; and the block's
        const uint32_t o = lane < kSelWarps ? sh.warp_sums[0][lane] : 0, e = lane < kSelWarps ? sh.warp_sums[1][lane] : 0;
        overs = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? o : 0), equals = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? e : 0);
        const uint32_t all_o = __reduce_add_sync(0xFFFFFFFFu, o), all_e = __reduce_add_sync(0xFFFFFFFFu, e);
        if (tid == 0) sh.mine[0] = all_o, sh.mine[1] = all_e;
    }
    if (blocks > 1) {
        cluster.sync();
        for (uint32_t r = 0; r < rank; ++r) {
            const uint32_t* m = cluster.map_shared_rank(sh.mine, r);
            overs += m[0], equals += m[1];
        }
    }
    const bool copy = out && (HELD || out != w);
    const uint32_t lower = (1u << lane) - 1;
    if (HELD && none_equal) {
        uint32_t base = overs + min(equals, ties);
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if (i >= mine) break;
            const bool over = over_bits >> i & 1;
            const uint32_t mo = __ballot_sync(0xFFFFFFFFu, over);
            if (over) {
                const uint32_t to = base + __popc(mo & lower);
                kept[to] = int32_t(w0 + i * 32 + lane);
                if (copy) out[to] = held[HELD ? i : 0];
            }
            base += __popc(mo);
        }
    } else {
        uint32_t i = 0;
        each([&](uint32_t j, float x) {
            bool over, equal;
            if (HELD)
                over = over_bits >> i & 1, equal = equal_bits >> i & 1, ++i;
            else
                look(j, x, over, equal);
            const uint32_t mo = __ballot_sync(0xFFFFFFFFu, over), me = __ballot_sync(0xFFFFFFFFu, equal);
            const uint32_t e = equals + __popc(me & lower);
            const uint32_t to = overs + __popc(mo & lower) + min(e, ties);
            if (over || (equal && e < ties)) {
                kept[to] = int32_t(j);
                if (copy) out[to] = x;
            }
            overs += __popc(mo), equals += __popc(me);
        });
    }
    if (blocks > 1 || !HELD) sync();  // (shared memory lives until the others have read it; and kept is complete)
    if (!HELD && out && !copy && rank == 0) {
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

template <int I>
__global__ void __launch_bounds__(kSelThreads, 1) select_kernel(const __grid_constant__ KvSelect c) {
    __shared__ SelShared sh;
    const uint32_t blocks = cg::this_cluster().num_blocks(), rank = cg::this_cluster().block_rank();
    const uint32_t row = blockIdx.x / blocks, s = row / c.n_heads, head = row % c.n_heads;
    for (uint32_t i = threadIdx.x; i < kBins / 4; i += kSelThreads) reinterpret_cast<uint4*>(sh.hist[0])[i] = make_uint4(0, 0, 0, 0);
    tc::pdl_launch();
    tc::pdl_wait();
    const int32_t given = c.lens[s];
    const uint32_t len = given > 0 && uint32_t(given) <= c.n_slots ? uint32_t(given) : 0;
    uint32_t n = min(len, c.keep);
    if (c.keeps) n = min(n, uint32_t(max(c.keeps[s], 0)));
    if (threadIdx.x == 0 && rank == 0 && head == 0) c.counts[s] = int32_t(n);
    if (n == 0) return;  // (of all of the cluster's blocks)
    __syncthreads();
    if (len <= blocks * (I * kSelThreads))
        select_row<I, true>(c, sh, s, head, len, n);
    else
        select_row<I, false>(c, sh, s, head, len, n);
}

// ------------------------------------------------------------------ evict
// A block moves the rows of one key head's keys and values (or a share of their columns), a chunk of rows at a time: all
// of a chunk's loads come before its stores, and a row's new slot is at or before its old one, so no row is overwritten
// before it was read. Where a chunk's rows lie is looked up once, by a thread a row, while the chunk before is moved.
// Bound by memory: rows are read once and written once, past the caches. Measured: 64 sequences of up to 16k slots to 4k
// each, 8 heads of 128 (2.15 GB): 339 us, 6.3 TB/s.
constexpr uint32_t kEvictThreads = 256;
constexpr uint32_t kEvictDeep = 4;  // rows of a thread in a chunk
// Rows of a chunk, at most: what two columns of threads or more come to. Where a row is one vector (heads of 8) half of the
// threads only look up; places for all of them would take 32 KiB of shared memory of every other form too.
constexpr uint32_t kEvictRows = kEvictThreads / 2 * kEvictDeep;
__global__ void __launch_bounds__(kEvictThreads, 4) evict_kernel(const __grid_constant__ KvEvict c, const uint32_t cols) {
    __shared__ ulonglong2 place[2][kEvictRows];  // a row's key: where it is and where it goes; 0: it stays
    tc::pdl_launch();
    tc::pdl_wait();
    const KvPages& p = c.pages;
    const uint32_t s = blockIdx.x / p.kv_heads, head = blockIdx.x % p.kv_heads, layer = p.layer + blockIdx.y;
    const uint32_t rows = min(kEvictThreads / cols, kEvictRows / kEvictDeep), chunk = rows * kEvictDeep;
    const uint32_t r = threadIdx.x / cols, col = blockIdx.z * cols + threadIdx.x % cols;
    const bool mine = r < rows && col * 8 < p.head_dim;
    const uint32_t n = uint32_t(min(max(c.counts[s], 0), int32_t(c.max_kept)));
    const int32_t* const kept = c.kept + s * c.kept_seq_stride + head * c.kept_head_stride;
    const uint64_t apart = (uint64_t(p.kv_heads) << p.token_shift) * (p.head_dim * 2);  // from a slot's key to its value
    auto look_up = [&](uint32_t i0, ulonglong2* to) {
        for (uint32_t k = threadIdx.x; k < chunk; k += kEvictThreads) {
            const uint32_t i = i0 + k;
            ulonglong2 at = make_ulonglong2(0, 0);
            const int32_t from = i < n ? kept[i] : 0;
            if (i < n && from > int32_t(i)) {
                const uint8_t* src = kv_row(p, s, from, layer, 0, head);
                const uint8_t* dst = kv_row(p, s, i, layer, 0, head);
                if (src && dst) at = make_ulonglong2(reinterpret_cast<uint64_t>(src), reinterpret_cast<uint64_t>(dst));
            }
            to[k] = at;
        }
    };
    look_up(0, place[0]);
    __syncthreads();
    for (uint32_t i0 = 0, b = 0; i0 < n; i0 += chunk, b ^= 1) {
        uint4 key[kEvictDeep], val[kEvictDeep];
        uint64_t to[kEvictDeep];
#pragma unroll
        for (uint32_t k = 0; k < kEvictDeep; ++k) {
            to[k] = 0;
            if (!mine) continue;
            const ulonglong2 at = place[b][k * rows + r];
            to[k] = at.y;
            if (!at.y) continue;
            const uint8_t* src = reinterpret_cast<const uint8_t*>(at.x) + col * 16;
            key[k] = __ldcs(reinterpret_cast<const uint4*>(src));
            val[k] = __ldcs(reinterpret_cast<const uint4*>(src + apart));
        }
        if (i0 + chunk < n) look_up(i0 + chunk, place[b ^ 1]);
        __syncthreads();
#pragma unroll
        for (uint32_t k = 0; k < kEvictDeep; ++k) {
            if (!to[k]) continue;
            uint8_t* dst = reinterpret_cast<uint8_t*>(to[k]) + col * 16;
            __stcs(reinterpret_cast<uint4*>(dst), key[k]);
            __stcs(reinterpret_cast<uint4*>(dst + apart), val[k]);
        }
    }
}

}  // namespace

template <int I>
cudaError_t launch_select(const KvSelect& c, uint32_t blocks, cudaStream_t stream) {
    cudaLaunchConfig_t l{};
    l.gridDim = dim3(c.n_seqs * c.n_heads * blocks);
    l.blockDim = dim3(kSelThreads);
    l.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = blocks, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    l.attrs = at;
    l.numAttrs = 2;
    return cudaLaunchKernelEx(&l, select_kernel<I>, c);
}

cudaError_t launch_kv_select(const KvSelect& c, uint32_t sms, cudaStream_t stream) {
    const uint64_t rows = uint64_t(c.n_seqs) * c.n_heads;
    // blocks to a row: what holds it, and more while SMs are idle and a thread has more than two weights
    uint32_t blocks = 1;
    while (blocks < kMostBlocks && (c.max_len / blocks > 16 * kSelThreads || (c.max_len / blocks > 2 * kSelThreads && rows * blocks * 2 <= sms))) blocks *= 2;
    const uint32_t each = (c.max_len + blocks * kSelThreads - 1) / (blocks * kSelThreads);
    return each <= 2 ? launch_select<2>(c, blocks, stream) : each <= 8 ? launch_select<8>(c, blocks, stream) : launch_select<16>(c, blocks, stream);
}

cudaError_t launch_kv_evict(const KvEvict& c, uint32_t sms, cudaStream_t stream) {
    const uint32_t vectors = c.pages.head_dim / 8;
    const uint64_t units = uint64_t(c.n_seqs) * c.pages.kv_heads * c.layers;
    // Fewer units than blocks that an SM's four places take: a block has a share of the columns, of 32 bytes at least (or
    // all of a narrower row). 512 units of 4,096 rows of 256 bytes with 1, 2 and 4 shares: 360, 338, 565 us.
    uint32_t parts = 1;
    while (parts < 8 && units * parts < 4 * sms && vectors / parts >= 4) parts *= 2;
    const uint32_t cols = (vectors + parts - 1) / parts;
    return launch_pdl(evict_kernel, dim3(c.n_seqs * c.pages.kv_heads, c.layers, parts), kEvictThreads, 0, stream, c, cols);
}

}  // namespace t2i
