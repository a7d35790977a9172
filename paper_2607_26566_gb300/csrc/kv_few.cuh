// Attention of few new tokens a sequence (a decoding step, a short draft): up to 32
// queries to a key head.
//
// Such a call reads every key and value once and does little with it, so it is
// bound by memory: the kernel's business is to keep loads in flight on every SM.
// The products are turned round: S^T = K Q^T and O^T = V^T P^T, so that the 128
// rows that a tensor core product has are keys (and dimensions of V), not padded
// queries, and K and V go from memory (TMA) through shared memory to the tensor
// cores without passing a register. A thread of the softmax warps is one key of a
// 128-key tile, and, for the accumulators, one dimension.
//
// Work split: all tiles of all units (a sequence, a key head), in order, are cut
// into equal runs, two an SM, whatever the lengths. A unit that lies in several
// runs is joined by a second kernel from partial sums in the workspace, in the
// order of the runs: results do not depend on timing.
//
// Softmax: a query's scores are weighed against a reference, its first tile's
// maximum, that is raised only when a score exceeds it by 2^8 (the accumulators, in
// fp32, have the room), so most tiles need no exchange between threads but one
// vote. Weights go to the product as two 16-bit numbers (the rounded weight and
// what the rounding left): products are not what bounds this kernel, and the
// weights keep 16 bits or more. In fp16, which ends at 2^-25, the reference lies
// below the maximum (kLift).
//
// Measured: a token each of 64 sequences of up to 16k slots (2.2 GB of keys and values,
// 32 heads over 8 of 128) 331 us, 6.8 TB/s; of 48 of up to 9k in a window of 4,096, heads
// of 64, scores capped, 28-29 us; of 192 of 600 slots 85 us (70 at the copy rate); of 256 of
// 100 slots 41 us, 5 us a segment in each of an SM's two blocks: half of it scores and
// weights, a quarter the products, a quarter the output; of one sequence of 700 slots 12.4
// us, of which the two launches and the chain of one tile are all.
#pragma once

#include <atomic>
#include <type_traits>

#include "kv_attend.cuh"
#include "t2istore.h"

namespace t2i {
namespace {

using namespace tc;

constexpr int kSoftThreads = 128;
constexpr int kThreads = kSoftThreads + 64;  // + the loading warp and the product warp
constexpr uint32_t kSlot = 16384;            // 128 rows of 64 elements
constexpr uint32_t kAhead = 4;
constexpr float kRaise = 8.0f;  // in units of log2; weights are below 2^(kRaise + kLift)
// A thread adds its keys' weights up over so many tiles, then they join the warp's sum: a thread's own sum over a long
// run lost what is below half a unit of it (a key far above 131,072 others: 4e-5 of the sum).
constexpr int32_t kSumTiles = 16;

template <int N, int NS>
struct Shape {
    // shared memory: ring of K and V tiles, queries, weights (and what stands in
    // static shared memory: kFixed at most). A product over heads of 64 reads the
    // 16 KiB behind its V tile too, for rows that nobody looks at.
    static constexpr uint32_t kFixed = 2048 + 48 * N;
    static constexpr uint32_t kPad = NS == 1 ? kSlot : 0;
    static constexpr uint32_t kQ = N * 128 * NS;
    static constexpr uint32_t kP = N * 512;  // two parts
    static constexpr uint32_t kEntry = kSlot * NS;
    static constexpr uint32_t kBlocks = 2;  // an SM: one's loads and products run beside the other's softmax
    static constexpr uint32_t kRoom = 228 * 1024 / kBlocks - 1024 - 1024 - kFixed - kQ - kP - kPad;
    static constexpr uint32_t kEntries = kRoom / kEntry < 12 ? kRoom / kEntry : 12;
    static constexpr uint32_t kBytes = 1024 + kEntry * kEntries + kQ + kP + kPad;
    static constexpr uint32_t kTmem = 3 * N <= 64 ? 64 : 128;  // two tiles' scores and the accumulators
    static_assert(kEntries >= 2, "a tile of K and one of V");
    static_assert(N <= 32, "the workspace is laid out for two blocks of 32 rows an SM");
    static constexpr uint32_t kPart = N * (64 * NS) + 2 * N;  // floats of a part: O^T, maxima, sums
};

// The run of tiles of one block, segment by segment (a segment: the tiles of the
// run that lie in one unit). The loading warp walks it and leaves each segment, with
// its queries, to the others.
struct Walk {
    uint32_t s, h;
    int64_t at, end;    // the next tile of all, and the end of the run
    int64_t unit;       // the unit's first tile of all
    int32_t tile, n, nt;  // the segment's first tile in the unit, its tiles, the unit's
    KvSeq q;
    KvSpan span;
    int32_t rows;
    bool more;  // segments behind this one
};

struct Shared {
    uint64_t full[12], empty[12];
    uint64_t s_full[2], p_full, pv_done, q_free;
    // Segments that are handed out. Four, so that no barrier runs ahead of who waits for it: the one that follows a
    // segment by three is written behind that segment's last scores' weights.
    uint64_t q_full[kAhead];
    Walk walk[kAhead];
    uint32_t tmem, dead;
    int32_t start_seq, start_rest;
    int64_t sums[kThreads / 32];
};

// A unit in several runs, noted at the run that holds its second part: the runs
// b0 to b1 hold it, the first as that block's part 0 or 1, the others as part 0.
struct Join {
    int32_t first, rows, h;  // the sequence's first token, its rows (queries of a key head), the key head
    int32_t b0, b1, second, valid;
};

struct Few {
    KvAttend a;
    Join* join;        // [blocks]
    float* part;       // [2 * blocks][kPart]
    uint32_t* fault;   // host-mapped: set where a wait ran out
    uint32_t no_loads; // testing: nothing is loaded or handed out, so that waits run out
};

__device__ __forceinline__ int32_t unit_tiles(const KvAttend& a, const KvSeq& q, KvSpan& sp) {
    if (q.n == 0) return 0;
    sp = kv_span(a, q, 0, min(q.n, int32_t(a.tok.max_new)));
    return max(1, (sp.hi + kTileKeys - 1) / kTileKeys - sp.lo / kTileKeys);
}

__device__ __forceinline__ void walk_seq(const KvAttend& a, Walk& w) {
    w.nt = 0;
    for (; w.s < a.tok.n_seqs; ++w.s) {
        w.q = kv_seq(a.pages, a.tok, w.s);
        w.nt = unit_tiles(a, w.q, w.span);
        if (w.nt) break;
    }
}
__device__ __forceinline__ void walk_unit(const KvAttend& a, Walk& w) {
    w.rows = min(w.q.n, int32_t(a.tok.max_new)) * int32_t(a.group);
    w.n = int32_t(min(int64_t(w.nt - w.tile), w.end - w.at));
    w.more = w.at + w.n < w.end;
}
__device__ __forceinline__ void walk_start(const KvAttend& a, Walk& w, uint32_t s, int32_t rest, int64_t at, int64_t end) {
    w.s = s, w.at = at, w.end = end;
    walk_seq(a, w);
    const int32_t nt = max(w.nt, 1);
    w.h = rest / nt;
    w.tile = rest % nt;
    w.unit = at - w.tile;
    walk_unit(a, w);
}
__device__ __forceinline__ bool walk_next(const KvAttend& a, Walk& w) {
    w.at += w.n;
    if (w.at >= w.end) return false;
    w.tile = 0;
    w.unit = w.at;
    if (++w.h == a.pages.kv_heads) {
        w.h = 0;
        ++w.s;
        walk_seq(a, w);
        if (w.nt == 0) return false;
    }
    walk_unit(a, w);
    return true;
}
// first slot of the unit's tile i
__device__ __forceinline__ int32_t tile_slot(const Walk& w, int32_t i) { return (w.span.lo / kTileKeys + i) * kTileKeys; }

// Sum or maximum over a warp's lanes of each of n = 16 or 32 columns: lane i gets
// column i % n.
template <int n, bool kMax>
__device__ __forceinline__ float columns(float (&v)[n], uint32_t lane) {
    auto join = [](float x, float y) { return kMax ? fmaxf(x, y) : x + y; };
    if constexpr (n == 16) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = join(v[i], __shfl_xor_sync(0xFFFFFFFFu, v[i], 16));
    }
#pragma unroll
    for (int d = n / 2; d; d >>= 1) {
        const bool up = lane & d;
#pragma unroll
        for (int i = 0; i < d; ++i) {
            const float keep = up ? v[i + d] : v[i], send = up ? v[i] : v[i + d];
            v[i] = join(keep, __shfl_xor_sync(0xFFFFFFFFu, send, d));
        }
    }
    return v[0];
}

template <class T, int N, int NS, Mod MOD>
__global__ void __launch_bounds__(kThreads, Shape<N, NS>::kBlocks) few_kernel(const __grid_constant__ Few f, const __grid_constant__ CUtensorMap map) {
    using Sh = Shape<N, NS>;
    constexpr bool kMod = MOD != Mod::kNone;
    constexpr bool kBf16 = sizeof(T) == 2 && !std::is_same<T, __half>::value;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    uint8_t* const mem = raw + (base - smem_u32(raw));
    const uint32_t ring = base, qs = ring + Sh::kEntry * Sh::kEntries, ps = qs + Sh::kQ;
    __shared__ __align__(16) Shared sh;
    __shared__ __align__(16) float top[N], scale_by[N], red[4][N];
    __shared__ __align__(16) int32_t first[N], last[N], pos[N];
    __shared__ __align__(16) uint64_t word[N];
    static_assert(N == 16 || N == 32, "a lane, or two, a query");
    __shared__ float slope[N];
    const KvAttend& a = f.a;
    const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    volatile uint32_t* dead = &sh.dead;

    auto bar = [&](const uint64_t& b) { return smem_u32(&b); };
    if (tid == 0) {
        for (uint32_t i = 0; i < Sh::kEntries; ++i) mbar_init(bar(sh.full[i]), 1), mbar_init(bar(sh.empty[i]), 1);
        mbar_init(bar(sh.s_full[0]), 1), mbar_init(bar(sh.s_full[1]), 1);
        mbar_init(bar(sh.p_full), kSoftThreads), mbar_init(bar(sh.pv_done), 1), mbar_init(bar(sh.q_free), 1);
        for (uint32_t i = 0; i < kAhead; ++i) mbar_init(bar(sh.q_full[i]), 32);
        sh.dead = 0;
        fence_mbar_init();
        tma_prefetch_map(&map);
    }
    if (warp == 5) tmem_alloc(smem_u32(&sh.tmem), Sh::kTmem);
    pdl_launch();
    pdl_wait();
    if (tid == 0) f.join[blockIdx.x].valid = 0;  // (also where a wait runs out before the note is written)

    // the block's run of tiles
    const int64_t K = a.pages.kv_heads;
    const uint32_t per = (a.tok.n_seqs + kThreads - 1) / kThreads;
    int64_t mine = 0;
    for (uint32_t s = tid * per; s < min(a.tok.n_seqs, (tid + 1) * per); ++s) {
        KvSpan sp;
        const KvSeq q = kv_seq(a.pages, a.tok, s);
        mine += unit_tiles(a, q, sp);
    }
    // inclusive scan over the block's threads, in tiles of one key head
    int64_t inc = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t o = __shfl_up_sync(0xFFFFFFFFu, inc, d);
        if (lane >= uint32_t(d)) inc += o;
    }
    if (lane == 31) sh.sums[warp] = inc;
    fence_before();
    __syncthreads();
    fence_after();
    int64_t before = 0, total = 0;
#pragma unroll
    for (uint32_t i = 0; i < kThreads / 32; ++i) {
        if (i < warp) before += sh.sums[i];
        total += sh.sums[i];
    }
    inc += before;
    total *= K;
    const int64_t blocks = min(int64_t(gridDim.x), total);
    const int64_t run0 = blocks ? blockIdx.x * total / blocks : 0, run1 = blocks ? (blockIdx.x + 1) * total / blocks : 0;
    const bool busy = blockIdx.x < blocks;
    if (busy) {
        const int64_t lo = (inc - mine) * K, hi = inc * K;
        if (run0 >= lo && run0 < hi) {  // this thread's sequences hold the run's first tile
            int64_t p = lo;
            for (uint32_t s = tid * per;; ++s) {
                KvSpan sp;
                const KvSeq q = kv_seq(a.pages, a.tok, s);
                const int64_t n = int64_t(unit_tiles(a, q, sp)) * K;
                if (run0 < p + n) {
                    sh.start_seq = int32_t(s);
                    sh.start_rest = int32_t(run0 - p);
                    break;
                }
                p += n;
            }
        }
    }
    __syncthreads();
    const uint32_t tmem = sh.tmem;

    if (busy && warp == 4) {
        // ---------------------------------------------------------- loads
        Walk w;
        walk_start(a, w, sh.start_seq, sh.start_rest, run0, run1);
        const uint32_t shift = a.pages.token_shift;
        const uint32_t box = shift < 7 ? 1u << shift : 128u, boxes = 128u / box;
        const uint32_t T_mask = (1u << shift) - 1;
        uint32_t n = 0, u = 0;
        // A segment's queries, a 16-byte vector a lane in turn: on their way while the segment before is worked on, and
        // to shared memory (64 dimensions at a time, 128-byte swizzle) when its last scores are there.
        constexpr uint32_t kRowVecs = NS * 8, kVecs = N * kRowVecs / 32, kStep = 32 / kRowVecs;
        uint4 qv[kVecs];
        auto ask = [&]() {
            const uint32_t D = a.pages.head_dim, G = a.group, x = lane % kRowVecs;
            uint32_t c = lane / kRowVecs, t = c / G, g = c % G;
            const T* const q0 = static_cast<const T*>(a.q) + uint64_t(w.q.first) * a.q_stride + uint64_t(w.h) * G * D + x * 8;
#pragma unroll
            for (uint32_t k = 0; k < kVecs; ++k, c += kStep) {
                const bool real = int32_t(c) < w.rows && x * 8 < D;
                qv[k] = real ? *reinterpret_cast<const uint4*>(q0 + t * a.q_stride + g * D) : make_uint4(0, 0, 0, 0);
                g += kStep % G, t += kStep / G;
                if (g >= G) g -= G, ++t;
            }
        };
        auto publish = [&]() -> bool {
            if (u && !mbar_wait(bar(sh.q_free), (u - 1) & 1, dead)) return false;
            const uint32_t x = lane % kRowVecs;
            uint32_t c = lane / kRowVecs;
#pragma unroll
            for (uint32_t k = 0; k < kVecs; ++k, c += kStep)
                *reinterpret_cast<uint4*>(mem + (qs - base) + x / 8 * (N * 128) + c * 128 + ((x % 8) ^ (c % 8)) * 16) = qv[k];
            if (lane == 0) sh.walk[u % kAhead] = w;
            fence_async_smem();
            mbar_arrive(bar(sh.q_full[u % kAhead]));
            ++u;
            return true;
        };
        for (bool more = !f.no_loads; more; more = walk_next(a, w)) {
            ask();
            const int32_t row_k = int32_t(((a.pages.layer * 2) * a.pages.kv_heads + w.h) << shift);
            const int32_t row_v = row_k + int32_t(a.pages.kv_heads << shift);
            const int32_t* table = a.pages.table + w.s * a.pages.table_stride;
            for (int32_t i = 0; i < w.n; ++i) {
                const uint32_t slot = uint32_t(tile_slot(w, w.tile + i)) + lane * box;
                int32_t page = -1;
                if (lane < boxes && slot < uint32_t(w.q.len)) page = table[slot >> shift];
                // what the pool lacks, and what lies behind the sequence, is filled with zeros
                const bool none = uint32_t(page) >= a.pages.total_pages;
                const int32_t z = none ? int32_t(a.pages.total_pages) : page;
                const int32_t y = int32_t(slot & T_mask);
#pragma unroll
                for (int kv = 0; kv < 2; ++kv, ++n) {
                    const uint32_t e = n % Sh::kEntries;
                    if (!mbar_wait(bar(sh.empty[e]), (n / Sh::kEntries & 1) ^ 1, dead)) goto loads_done;
                    if (lane == 0) mbar_expect(bar(sh.full[e]), Sh::kEntry);
                    __syncwarp();
                    if (lane < boxes)
                        for (int x = 0; x < NS; ++x)
                            tma_load(ring + e * Sh::kEntry + x * kSlot + lane * box * 128, &map, x * 64,
                                     (kv ? row_v : row_k) + y, z, bar(sh.full[e]));
                    if (i == 0 && kv == 0 && !__all_sync(0xFFFFFFFFu, publish())) {
                        ++n;
                        goto loads_done;
                    }
                }
            }
        }
    loads_done:
        __syncwarp();
        if (*dead) {  // the copies in flight land before the block ends
            uint32_t late = 0;
            for (uint32_t k = n > Sh::kEntries ? n - Sh::kEntries : 0; k < n; ++k)
                mbar_wait(bar(sh.full[k % Sh::kEntries]), k / Sh::kEntries & 1, &late);
        }
    } else if (busy && warp == 5) {
        // ---------------------------------------------------------- products
        constexpr uint32_t kQk = instr_desc(kBf16, false, false, 128, N);
        constexpr uint32_t kPv = instr_desc(kBf16, true, true, 128, N);
        const uint32_t ksteps = (a.pages.head_dim + 15) / 16;
        // keys and queries: rows of 64 elements, swizzled; values: the same rows, read along the keys; weights:
        // eight columns to 16 bytes, a key after the other
        const uint64_t kd = smem_desc(ring, 16, 1024, 2), qd = smem_desc(qs, 16, 1024, 2), vd = smem_desc(ring, kSlot, 1024, 2);
        const uint64_t pd = smem_desc(ps, 128, 2048, 0);
        uint32_t n = 0, u = 0;  // tiles and segments of the run
        bool fresh_before = false, more;
        auto pv = [&](uint32_t i, bool fresh) {
            const uint32_t e = (2 * i + 1) % Sh::kEntries;
            mbar_wait(bar(sh.p_full), i & 1, dead);
            mbar_wait(bar(sh.full[e]), (2 * i + 1) / Sh::kEntries & 1, dead);
            fence_after();
            if (elect() && !*dead) {
                const uint64_t v0 = desc_at(vd, e * Sh::kEntry);
#pragma unroll
                for (int part = 0; part < 2; ++part)
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        mma_ss(tmem + 2 * N, desc_at(v0, k * 2048), desc_at(pd, part * (N * 256) + k * 256), kPv,
                               !(fresh && part == 0 && k == 0));
                mma_commit(bar(sh.empty[e]));
                mma_commit(bar(sh.pv_done));
            }
            __syncwarp();
        };
        do {
            const bool got = mbar_wait(bar(sh.q_full[u % kAhead]), u / kAhead & 1, dead);
            if (!__all_sync(0xFFFFFFFFu, got)) break;
            const int32_t tiles = sh.walk[u % kAhead].n;
            more = sh.walk[u % kAhead].more;
            ++u;
            for (int32_t i = 0; i < tiles; ++i, ++n) {
                const uint32_t e = (2 * n) % Sh::kEntries;
                mbar_wait(bar(sh.full[e]), (2 * n) / Sh::kEntries & 1, dead);
                fence_after();
                if (elect() && !*dead) {
                    const uint64_t k0 = desc_at(kd, e * Sh::kEntry);
#pragma unroll
                    for (uint32_t k = 0; k < 4 * NS; ++k) {
                        if (k >= ksteps) break;
                        mma_ss(tmem + (n & 1) * N, desc_at(k0, (k / 4) * kSlot + (k % 4) * 32),
                               desc_at(qd, (k / 4) * (N * 128) + (k % 4) * 32), kQk, k != 0);
                    }
                    mma_commit(bar(sh.empty[e]));
                    mma_commit(bar(sh.s_full[n & 1]));
                    if (i + 1 == tiles) mma_commit(bar(sh.q_free));
                }
                __syncwarp();
                if (n) pv(n - 1, fresh_before);
                fresh_before = i == 0;
            }
        } while (more);
        if (n) pv(n - 1, fresh_before);
        if (*dead) {  // the products in flight end before the tensor memory is freed
            const uint64_t t0 = now_ns();
            while (now_ns() - t0 < 50000) {
            }
        }
    } else if (busy) {
        // ---------------------------------------------------------- softmax
        const uint32_t D = a.pages.head_dim;
        const uint32_t lanes = tmem + (warp << 21);  // this warp's 32 lanes
        const float k2 = a.scale * kLog2e;
        const float cap_in = kMod && a.softcap != 0.0f ? a.scale / a.softcap : 0.0f, cap2 = a.softcap * kLog2e;
        uint32_t n = 0;
        bool more;
        for (uint32_t u = 0;; ++u) {
            const bool got = mbar_wait(bar(sh.q_full[u % kAhead]), u / kAhead & 1, dead);
            if (bar_any<1, kSoftThreads>(!got)) break;  // (also: top and red were read before they are written again)
            const Walk w = sh.walk[u % kAhead];
            more = w.more;
            const int32_t ctx = w.q.len - w.q.n;
            if (tid < N) {
                KvQuery q{0, INT32_MAX, 0, 0};
                float sl = 0.0f;
                if (int32_t(tid) < w.rows) {
                    q = kv_query(a, w.q, int32_t(tid / a.group));
                    if (kMod && a.slopes) sl = a.slopes[w.h * a.group + tid % a.group] * kLog2e;
                }
                top[tid] = -INFINITY;
                first[tid] = q.first, last[tid] = q.last, pos[tid] = q.pos, word[tid] = q.word;
                slope[tid] = sl;
            }
            if (tid == 0 && w.at == run0) {
                // this run's note of a unit that began in the run before it
                const int64_t b0 = ((w.unit + 1) * blocks - 1) / total, b1 = ((w.unit + w.nt) * blocks - 1) / total;
                const bool here = w.tile > 0 && b0 + 1 == int64_t(blockIdx.x);
                f.join[blockIdx.x] = {w.q.first, w.rows, int32_t(w.h), int32_t(b0), int32_t(b1), b0 * total / blocks != w.unit, here};
            }
            bar_sync<1, kSoftThreads>();

            float sum[N] = {};  // of the thread's keys' weights
            KvSum all;          // ... and of the warp's so far, column lane % N
            auto add_up = [&]() {
                all.add(columns<N, false>(sum, lane));
#pragma unroll
                for (int c = 0; c < N; ++c) sum[c] = 0.0f;
            };
            for (int32_t i = 0; i < w.n; ++i, ++n) {
                const int32_t slot0 = tile_slot(w, w.tile + i), key = slot0 + int32_t(tid);
                const bool masked = slot0 < w.span.all_lo || slot0 + kTileKeys > w.span.all_hi;
                // a drafted key's bit and position
                uint64_t bit = 0;
                int32_t kpos = key;
                if (a.tree && key >= ctx && key < w.q.len && key - ctx < 64) {
                    bit = uint64_t(1) << (key - ctx);
                    kpos = ctx + __popcll(kv_word(a, w.q, key - ctx)) - 1;
                }
                const uint32_t s_at = lanes + (n & 1) * N;
                mbar_wait(bar(sh.s_full[n & 1]), n >> 1 & 1, dead);
                fence_after();
                float x[N];  // scores, then weights
                if constexpr (N == 32)
                    tmem_ld32(s_at, x);
                else
                    tmem_ld16(s_at, x);
                wait_ld(x);
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    if (kMod) {
                        x[c] = cap_in != 0.0f ? capped<MOD == Mod::kFine>(x[c], cap_in, cap2) : x[c] * k2;
                        x[c] -= slope[c] * fabsf(float(pos[c] - kpos));
                    } else {
                        x[c] *= k2;
                    }
                }
                if (masked) {
                    uint32_t see = 0;
#pragma unroll
                    for (int c = 0; c < N; ++c)
                        see |= uint32_t(kpos >= first[c] && (key < last[c] || (word[c] & bit))) << c;
#pragma unroll
                    for (int c = 0; c < N; ++c) x[c] = see & (1u << c) ? x[c] : -INFINITY;
                }
                // the product before this one is complete: its weights may be overwritten, its accumulators scaled
                bool over_with = n == 0;
                auto last_product = [&]() {
                    if (!over_with) mbar_wait(bar(sh.pv_done), (n - 1) & 1, dead);
                    over_with = true;
                };
                // references become the tile's maxima (red: of each warp's keys), less kLift
                auto raise = [&]() {
                    bar_sync<1, kSoftThreads>();
                    if (tid < N) {
                        const float was = top[tid];
                        const float most = fmaxf(fmaxf(red[0][tid], red[1][tid]), fmaxf(red[2][tid], red[3][tid]));
                        const float now = fmaxf(most - kLift<T>, was);
                        top[tid] = now;
                        scale_by[tid] = was == now ? 1.0f : exp2_approx(was - now);
                    }
                    bar_sync<1, kSoftThreads>();
                    if (i) {
                        last_product();
                        fence_after();
#pragma unroll 1
                        for (int c0 = 0; c0 < N; c0 += 16) {
                            float o[16];
                            tmem_ld16(lanes + 2 * N + c0, o);
                            wait_ld(o);
#pragma unroll
                            for (int c = 0; c < 16; ++c) o[c] *= scale_by[c0 + c];
                            tmem_st16(lanes + 2 * N + c0, reinterpret_cast<uint32_t*>(o));
                        }
                        wait_st();
#pragma unroll
                        for (int c = 0; c < N; ++c) sum[c] *= scale_by[c];
                        all.scale(scale_by[lane % N]);
                    }
                };
                // their scores are looked at while the product before this one runs
                bool over = false;
#pragma unroll
                for (int c = 0; c < N; ++c) over |= x[c] > top[c] + (kRaise + kLift<T>);
                if (bar_any<1, kSoftThreads>(over)) {
                    float y[N];
#pragma unroll
                    for (int c = 0; c < N; ++c) y[c] = x[c];
                    const float m = columns<N, true>(y, lane);
                    if (lane < N) red[warp][lane] = m;
                    raise();
                }
                // weights: rounded, and the rest, eight columns to a 16-byte row of the operand
                last_product();
#pragma unroll
                for (int c = 0; c < N; c += 8) {
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float m = top[c + j + k];
                            x[c + j + k] = exp2_approx(x[c + j + k] - (m == -INFINITY ? 0.0f : m));
                        }
                        hi[j / 2] = Kv16<T>::from2(x[c + j], x[c + j + 1]);
                        const float2 r = Kv16<T>::to2(hi[j / 2]);
                        lo[j / 2] = Kv16<T>::from2(x[c + j] - r.x, x[c + j + 1] - r.y);
                    }
                    uint8_t* at = mem + (ps - base) + c / 8 * 2048 + tid * 16;
                    *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    *reinterpret_cast<uint4*>(at + N * 256) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
#pragma unroll
                for (int c = 0; c < N; ++c) sum[c] += x[c];
                if (i % kSumTiles == kSumTiles - 1) add_up();
                // values that none of the unit's queries sees may be anything: zeros, as their weights are
                if (slot0 < w.span.lo || slot0 + kTileKeys > w.span.hi) {
                    const uint32_t e = (2 * n + 1) % Sh::kEntries;
                    mbar_wait(bar(sh.full[e]), (2 * n + 1) / Sh::kEntries & 1, dead);
                    if (key < w.span.lo || key >= w.span.hi) {
#pragma unroll 1
                        for (int k = 0; k < NS * 8; ++k)
                            *reinterpret_cast<uint4*>(mem + e * Sh::kEntry + k / 8 * kSlot + tid * 128 + k % 8 * 16) =
                                make_uint4(0, 0, 0, 0);
                    }
                }
                fence_async_smem();
                fence_before();
                mbar_arrive(bar(sh.p_full));
            }
            // the segment's sums over the warps
            add_up();
            if (lane < N) red[warp][lane] = all.value();
            mbar_wait(bar(sh.pv_done), (n - 1) & 1, dead);
            fence_after();
            bar_sync<1, kSoftThreads>();
            const bool whole = w.n == w.nt;
            const uint32_t d = tid;
            float* part = f.part + (uint64_t(blockIdx.x) * 2 + (w.at == run0 ? 0 : 1)) * Sh::kPart;
            if (whole) {
                // lane c: the sum of column c's weights, and what divides by it
                const uint32_t mc = lane % N;
                const float l = red[0][mc] + red[1][mc] + red[2][mc] + red[3][mc], r = l == 0.0f ? 0.0f : 1.0f / l;
                if (a.lse && warp == 0 && lane < N && int32_t(lane) < w.rows)
                    a.lse[uint64_t(w.q.first + lane / a.group) * a.q_heads + w.h * a.group + lane % a.group] =
                        l == 0.0f ? -INFINITY : (top[lane] + log2f(l)) * kLn2;
                T* at = static_cast<T*>(a.out) + uint64_t(w.q.first) * a.out_stride + uint64_t(w.h) * a.group * D + d;
                const uint64_t on = a.out_stride - uint64_t(a.group - 1) * D;  // from a token's last head to the next token
                uint32_t g = 0;
#pragma unroll 1
                for (int c0 = 0; c0 < w.rows; c0 += 16) {
                    float o[16];
                    tmem_ld16(lanes + 2 * N + c0, o);
                    wait_ld(o);
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        const float by = __shfl_sync(0xFFFFFFFFu, r, c0 + c);
                        if (c0 + c < w.rows) {
                            if (d < D) *at = Kv16<T>::from1(o[c] * by);
                            const bool next = ++g == a.group;
                            at += next ? on : D;
                            if (next) g = 0;
                        }
                    }
                }
            } else {  // a part of the unit: to the workspace
#pragma unroll 1
                for (int c0 = 0; c0 < w.rows; c0 += 16) {
                    float o[16];
                    tmem_ld16(lanes + 2 * N + c0, o);
                    wait_ld(o);
                    if (d < 64 * NS) {
                        float* at = part + c0 * (64 * NS) + d;
#pragma unroll
                        for (int c = 0; c < 16; ++c) __stcg(at + c * (64 * NS), o[c]);
                    }
                }
            }
            if (!whole && tid < N) {
                __stcg(part + N * 64 * NS + tid, top[tid]);
                __stcg(part + N * 64 * NS + N + tid, red[0][tid] + red[1][tid] + red[2][tid] + red[3][tid]);
            }
            fence_before();
            if (!more) break;
        }
    }
    __syncthreads();
    if (tid == 0 && *dead) *f.fault = 1;
    if (warp == 5) {
        fence_after();
        tmem_free(tmem, Sh::kTmem);
    }
}

// Joins the units that lie in several runs: a block for each run's note, a warp
// for each query.
template <class T, int N, int NS>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ Few f) {
    using Sh = Shape<N, NS>;
    using V = typename std::conditional<NS == 2, float4, float2>::type;
    constexpr int kVec = 2 * NS;
    const KvAttend& a = f.a;
    pdl_launch();
    pdl_wait();
    const Join j = f.join[blockIdx.x];
    if (!j.valid) return;
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, D = a.pages.head_dim;
    const int32_t col = int32_t(blockIdx.y * 8 + warp);
    if (col >= j.rows) return;
    auto part = [&](int32_t b) { return f.part + (uint64_t(b) * 2 + (b == j.b0 && j.second ? 1 : 0)) * Sh::kPart; };
    float top = -INFINITY;
    for (int32_t b = j.b0 + int32_t(lane); b <= j.b1; b += 32) top = fmaxf(top, __ldcg(part(b) + N * 64 * NS + col));
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    float o[kVec] = {}, l = 0.0f;
    for (int32_t b0 = j.b0; b0 <= j.b1; b0 += 32) {
        const int32_t b = b0 + int32_t(lane);
        float w = 0.0f;
        if (b <= j.b1) {
            const float m = __ldcg(part(b) + N * 64 * NS + col);
            w = m == top ? 1.0f : exp2_approx(m - top);
            l += w * __ldcg(part(b) + N * 64 * NS + N + col);
        }
        const int32_t n = min(32, j.b1 - b0 + 1);
#pragma unroll 8
        for (int32_t k = 0; k < n; ++k) {
            const float wk = __shfl_sync(0xFFFFFFFFu, w, k);
            const V v = __ldcg(reinterpret_cast<const V*>(part(b0 + k) + col * (64 * NS)) + lane);
            const float* x = reinterpret_cast<const float*>(&v);
#pragma unroll
            for (int e = 0; e < kVec; ++e) o[e] += wk * x[e];
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, d);
    const uint64_t row = uint64_t(j.first + col / int32_t(a.group));
    const uint32_t head = uint32_t(j.h) * a.group + uint32_t(col) % a.group;
    const float r = l == 0.0f ? 0.0f : 1.0f / l;
    T* out = static_cast<T*>(a.out) + row * a.out_stride + uint64_t(head) * D + lane * kVec;
    if (lane * kVec < D) {
#pragma unroll
        for (int e = 0; e < kVec; e += 2) reinterpret_cast<uint32_t*>(out)[e / 2] = Kv16<T>::from2(o[e] * r, o[e + 1] * r);
    }
    if (a.lse && lane == 0) a.lse[row * a.q_heads + head] = l == 0.0f ? -INFINITY : (top + log2f(l)) * kLn2;
}

template <class T, int N, int NS, Mod MOD>
cudaError_t launch_as(const Few& f, const CUtensorMap& map, uint32_t sms, cudaStream_t stream) {
    constexpr uint32_t bytes = Shape<N, NS>::kBytes;
    static std::atomic<uint64_t> ready{0};  // devices whose kernel may take this much shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !(ready.load() >> dev & 1)) {
        e = cudaFuncSetAttribute(few_kernel<T, N, NS, MOD>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(bytes));
        if (e != cudaSuccess) return e;
        if (dev < 64) ready |= uint64_t(1) << dev;
    }
    const uint64_t units = f.a.tok.n_seqs;
    const uint32_t blocks = attend_blocks(f.a, sms * Shape<N, NS>::kBlocks, units);
    e = launch_pdl(few_kernel<T, N, NS, MOD>, dim3(blocks), kThreads, bytes, stream, f, map);
    if (e != cudaSuccess) return e;
    return launch_pdl(join_kernel<T, N, NS>, dim3(blocks, (N + 7) / 8), 256, 0, stream, f);
}

template <class T, int N, int NS>
cudaError_t launch_mod(const Few& f, const CUtensorMap& map, uint32_t sms, cudaStream_t stream) {
    switch (mod_of(f.a)) {
        case Mod::kNone: return launch_as<T, N, NS, Mod::kNone>(f, map, sms, stream);
        case Mod::kSome: return launch_as<T, N, NS, Mod::kSome>(f, map, sms, stream);
        default: return launch_as<T, N, NS, Mod::kFine>(f, map, sms, stream);
    }
}

template <class T, int N>
cudaError_t launch_n(const Few& f, const CUtensorMap& map, uint32_t sms, cudaStream_t stream) {
    return f.a.pages.head_dim <= 64 ? launch_mod<T, N, 1>(f, map, sms, stream) : launch_mod<T, N, 2>(f, map, sms, stream);
}

template <class T>
cudaError_t launch_t(const Few& f, const CUtensorMap& map, uint32_t sms, cudaStream_t stream) {
    const uint32_t rows = f.a.group * f.a.tok.max_new;
    return rows <= 16 ? launch_n<T, 16>(f, map, sms, stream) : launch_n<T, 32>(f, map, sms, stream);
}

constexpr uint64_t join_bytes(uint32_t sms) { return (uint64_t(sms) * 2 * sizeof(Join) + 255) / 256 * 256; }  // two blocks an SM

template <class T>
cudaError_t launch_few(const KvAttend& a, const KvLaunch& l, cudaStream_t stream) {
    Few f;
    f.a = a;
    f.join = static_cast<Join*>(l.workspace);
    f.part = reinterpret_cast<float*>(static_cast<uint8_t*>(l.workspace) + join_bytes(l.sms));
    f.fault = l.fault;
    f.no_loads = l.no_loads;
    return launch_t<T>(f, *l.map, l.sms, stream);
}

}  // namespace
}  // namespace t2i
