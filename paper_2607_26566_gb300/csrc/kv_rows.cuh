// Attention of more new tokens a sequence (prompts, chunks of them, trees): over 32
// queries to a key head.
//
// Bound by the tensor cores: 4 * 128 * head_dim operations for each query and 128-
// key tile. A block takes 256 rows (a row: one query of one new token; the heads of
// a group lie side by side, so shared keys are loaded once for all of them) as two
// stages of 128. While one stage's four warps do the softmax of a tile, the other's
// products run: S = Q K^T to tensor memory, a thread takes one row of S, writes
// its weights over it (16 bits each), and O += P V reads them there. K and V come by
// TMA. Scores are weighed against a reference that need not be the maximum so far: it
// is raised only behind a tile whose weights add up to over 2^8, so most tiles look
// for no maximum and rescale nothing.
//
// Weights are rounded to the cache's type before the product (as accurate as the
// values that they weigh: the output's own rounding is as large), the sums are not.
//
// Work split: a plan (by a kernel of its own, or, of up to 64 row tiles, by every block
// for itself) lists the row tiles and the slots that each one sees; all key tiles of all
// (sequence, key head, row tile) units, in order, and what each unit costs beside them,
// are cut into as many equal runs as there are SMs. A unit in several runs is joined by a
// last kernel, in the order of the runs.
//
// Measured: a prompt of 8190 tokens, 32 heads over 8 of 128, 400-420 us, 1.31-1.37
// PFLOP/s of what is visible; 24 drafts of 60 tokens over contexts up to 8k, the same heads, 118 us;
// one draft of 21 tokens over 1.5k slots 18 us; three chunks of 600 tokens of packed documents, 16 heads of
// 80, with spans and a bias, 48 us.
#pragma once

#include <atomic>
#include <type_traits>

#include "kv_attend.cuh"
#include "t2istore.h"

namespace t2i {
namespace {

using namespace tc;

constexpr int kRows = 256;            // of a unit
// Two stages of 128 threads, and 128 more: the loading warp, the product warp and two
// that idle, so that registers can be shared out by groups of four warps (a softmax
// thread holds its row's 128 scores).
constexpr int kRowThreads = 384;
constexpr int kRowRegs = 168, kSoftRegs = 192, kOtherRegs = 120;
static_assert(kSoftRegs * 256 + kOtherRegs * 128 <= kRowRegs * kRowThreads, "what a block was launched with");
constexpr uint32_t kEntryBytes = 32768;  // a tile of K or V, 128 rows of 128 elements
constexpr uint32_t kRowEntries = 4;
constexpr uint32_t kRowSmem = 1024 + 2 * kEntryBytes + kRowEntries * kEntryBytes;
constexpr uint32_t kRowPart = kRows * 128 + 2 * kRows;  // floats of a part: O, maxima, sums
// A row's scores are weighed against a reference: its first tile's maximum (less
// kLift), raised behind a tile whose weights add up to more than kRaise (the
// accumulators follow in the next tile), and at once where they add up to more than
// kFar, so that no weight exceeds it.
template <class T>
constexpr float kUnitOf = 1.0f;  // 2^kLift: the weight of the maximum
template <>
constexpr float kUnitOf<__half> = 0x1p7f;
template <class T>
constexpr float kRaiseOf = 256.0f * kUnitOf<T>;
template <class T>
constexpr float kFarOf = 0x1p64f;
template <>
constexpr float kFarOf<__half> = 65504.0f;  // fp16's largest

struct PlanTile {
    int32_t s, m;       // the sequence, and which 256 rows of it
    KvSpan span;
    KvSeq q;
    int32_t rows;       // of the tile
    int32_t nt;         // key tiles
    int32_t last;       // the sequence's last row tile
    int64_t before;     // cost of the tiles before it: key tiles, and Rows::cost for each
    int64_t seq_before, seq_total;  // ... of the sequences before its own; of its own
};
struct PlanHead {
    int64_t total;
    int32_t tiles;
};

// What a unit costs beside its key tiles (its queries' way to shared memory, the first scores without a product
// beside them, its output), in key tiles: it lies before its tiles when runs are cut. Measured with 0, 1, 2, 3, 4
// and 5: a prompt of 8190 tokens with 32 heads of 128 527, 490, 454, 424, 399, 403 us; 24 drafts of 60 tokens over
// contexts up to 8k 132, 127, 124, 120, 118, 118. Scores with a bias or a cap make tiles dearer, so that a unit
// costs fewer of them. With 1, 2, 3 and 4: the prompt with a cap 957, 933, 946, 957, with a bias 770, 772, 782, 791;
// the drafts with a cap 214, 209, 213, 219, with a bias 207, 204, 205, 201; chunks of 600 tokens with a bias 95, 95,
// 97, 100, with spans and a bias 48, 47, 52, 54, with spans and a cap 55, 55, 60, 61. (With spans alone, which go
// with the plain scores, 42, 42, 45, 47.)
constexpr int32_t kUnitCost = 4, kUnitCostMod = 2;

// A unit in several runs, noted at the run that holds its second part: the runs
// b0 to b1 hold it, the first as that block's part 0 or 1, the others as part 0.
struct Join {
    int32_t first, m, rows, h;  // the sequence's first token, the unit's row tile, its rows, its key head
    int32_t b0, b1, second, valid;
};

struct Rows {
    KvAttend a;
    PlanHead* head;
    int32_t* firsts;   // [n_seqs + 1]: each sequence's first tile
    PlanTile* plan;
    uint32_t most;     // entries of plan
    int32_t cost;      // of a unit beside its key tiles, in key tiles: kUnitCost or kUnitCostMod
    Join* join;        // [blocks]
    float* part;       // [2 * blocks][kRowPart]
    uint32_t* fault;
    uint32_t no_loads; // testing: nothing is loaded or handed out, so that waits run out
};

__device__ __forceinline__ int32_t row_tiles(const KvAttend& a, const KvSeq& q) {
    return int32_t((uint64_t(min(q.n, int32_t(a.tok.max_new))) * a.group + kRows - 1) / kRows);
}

// The span of a row tile, by a warp.
__device__ __forceinline__ KvSpan tile_span(const KvAttend& a, const KvSeq& q, int32_t t0, int32_t t1, int32_t lane) {
    if (!a.spans) return kv_span(a, q, t0, t1);
    KvSpan r{INT32_MAX, 0, 0, INT32_MAX};
    for (int32_t i = t0 + lane; i < t1; i += 32) {
        const KvSpan x = kv_span(a, q, i, i + 1);
        if (x.hi > x.lo) r.lo = min(r.lo, x.lo), r.hi = max(r.hi, x.hi);
        r.all_lo = max(r.all_lo, x.all_lo), r.all_hi = min(r.all_hi, x.all_hi);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        r.lo = min(r.lo, __shfl_xor_sync(0xFFFFFFFFu, r.lo, d));
        r.hi = max(r.hi, __shfl_xor_sync(0xFFFFFFFFu, r.hi, d));
        r.all_lo = max(r.all_lo, __shfl_xor_sync(0xFFFFFFFFu, r.all_lo, d));
        r.all_hi = min(r.all_hi, __shfl_xor_sync(0xFFFFFFFFu, r.all_hi, d));
    }
    if (r.lo >= r.hi) r.lo = r.hi = 0;
    return r;
}

// Exclusive scan of one number a thread over the block; *total: their sum.
template <int THREADS>
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* sums, int64_t* total) {
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int64_t inc = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t o = __shfl_up_sync(0xFFFFFFFFu, inc, d);
        if (lane >= uint32_t(d)) inc += o;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = inc;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (uint32_t i = 0; i < THREADS / 32; ++i) {
        if (i < warp) before += sums[i];
        all += sums[i];
    }
    *total = all;
    return before + inc - v;
}

// The plan, by a block: `firsts` [n_seqs + 1] and `plan` in global memory, or in
// shared memory where they fit. Returns the row tiles; *total: the cost of one head's.
template <int THREADS>
__device__ __forceinline__ int32_t make_plan(const Rows& f, PlanTile* plan, int32_t* firsts, int64_t* sums, int64_t* total) {
    const KvAttend& a = f.a;
    const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    // 1. each sequence's first tile
    const uint32_t per = (a.tok.n_seqs + THREADS - 1) / THREADS;
    const uint32_t s0 = tid * per, s1 = min(a.tok.n_seqs, s0 + per);
    int64_t mine = 0, all;
    for (uint32_t s = s0; s < s1; ++s) mine += row_tiles(a, kv_seq(a.pages, a.tok, s));
    int64_t at = block_scan<THREADS>(mine, sums, &all);
    // more than the call's tokens make: starts that make no sense
    const int32_t tiles = all > int64_t(f.most) ? 0 : int32_t(all);
    for (uint32_t s = s0; s < s1; ++s) {
        firsts[s] = int32_t(at);
        if (s + 1 < s1) at += row_tiles(a, kv_seq(a.pages, a.tok, s));
    }
    if (tid == 0) firsts[a.tok.n_seqs] = tiles;
    __syncthreads();
    // 2. a warp a tile
    KvTokens owner = a.tok;
    owner.starts = firsts;
    for (int32_t j = int32_t(warp); j < tiles; j += THREADS / 32) {
        const uint32_t s = kv_owner(owner, uint32_t(j));
        const KvSeq q = kv_seq(a.pages, a.tok, s);
        const int32_t m = j - firsts[s], G = int32_t(a.group);
        const int32_t end = int32_t(min(int64_t(min(q.n, int32_t(a.tok.max_new))) * G, (int64_t(m) + 1) * kRows));
        const KvSpan sp = tile_span(a, q, m * kRows / G, (end + G - 1) / G, int32_t(lane));
        if (lane == 0) {
            PlanTile& t = plan[j];
            t.s = int32_t(s), t.m = m, t.span = sp, t.q = q, t.rows = end - m * kRows;
            t.nt = max(1, (sp.hi + kTileKeys - 1) / kTileKeys - sp.lo / kTileKeys);
            t.last = j + 1 == firsts[s + 1];
        }
    }
    __syncthreads();
    // 3. the cost before each tile, and of its sequence
    const int32_t tper = (tiles + THREADS - 1) / THREADS;
    const int32_t j0 = int32_t(tid) * tper, j1 = min(tiles, j0 + tper);
    mine = 0;
    for (int32_t j = j0; j < j1; ++j) mine += plan[j].nt + f.cost;
    at = block_scan<THREADS>(mine, sums, &all);
    for (int32_t j = j0; j < j1; ++j) {
        plan[j].before = at;
        at += plan[j].nt + f.cost;
    }
    __syncthreads();
    for (int32_t j = j0; j < j1; ++j) {
        PlanTile& t = plan[j];
        const int32_t a0 = firsts[t.s], a1 = firsts[t.s + 1];
        t.seq_before = plan[a0].before;
        t.seq_total = (a1 < tiles ? plan[a1].before : all) - t.seq_before;
    }
    *total = all;
    return tiles;
}

constexpr int kPlanThreads = 1024;
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const __grid_constant__ Rows f) {
    __shared__ int64_t sums[kPlanThreads / 32];
    pdl_launch();
    pdl_wait();
    int64_t total;
    const int32_t tiles = make_plan<kPlanThreads>(f, f.plan, f.firsts, sums, &total);
    if (threadIdx.x == 0) f.head->total = total, f.head->tiles = tiles;
}

// Up to so many row tiles (by their bound) every block makes the plan for itself, in
// shared memory: it saves a kernel and its way through memory.
constexpr uint32_t kOwnPlan = 64;

// The run of one block, unit by unit: in a sequence, key head by key head, its row
// tiles. The loading warp walks it, one unit ahead of its loads, and leaves each
// unit in shared memory for the others.
struct Unit {
    KvSpan span;
    KvSeq q;
    int32_t s, m, h, rows;
    int32_t tile, n, nt;  // the segment's first key tile in the unit, its key tiles, the unit's
    int32_t more;         // another unit follows
    int64_t at;           // the segment's first tile of all
    int32_t draft[64];    // positions of the drafted tokens, if there is a tree
};
struct RowWalk {
    int64_t at, end;  // the segment's place among all tiles and units' costs, and the run's end
    int64_t unit;     // the place of the unit's first tile
    int32_t j, h, tile, n;
    PlanTile t;
};
// The run's part of the unit that begins (with its cost) at place `start`.
__device__ __forceinline__ void walk_segment(const Rows& f, RowWalk& w, int64_t start) {
    w.unit = start + f.cost;
    if (w.at < w.unit) w.at = w.unit;
    w.tile = int32_t(w.at - w.unit);
    w.n = int32_t(min(w.unit + w.t.nt, w.end) - w.at);
}
__device__ __forceinline__ bool walk_next(const Rows& f, const PlanTile* plan, RowWalk& w) {
    const int64_t start = w.unit + w.t.nt;
    w.at = start;
    if (start + f.cost >= w.end) return false;  // (nothing of the next unit but its cost)
    if (!w.t.last) {
        ++w.j;
    } else if (w.h + 1 < int32_t(f.a.pages.kv_heads)) {
        ++w.h;
        w.j -= w.t.m;
    } else {
        ++w.j;
        w.h = 0;
    }
    w.t = plan[w.j];
    walk_segment(f, w, start);
    return true;
}
__device__ __forceinline__ int32_t tile_slot(const KvSpan& s, int32_t i) { return (s.lo / kTileKeys + i) * kTileKeys; }

constexpr uint32_t kUnits = 8;      // in shared memory at a time
constexpr uint32_t kUnitReaders = 9;  // eight softmax warps and the product warp

struct RowShared {
    uint64_t full[kRowEntries], empty[kRowEntries];
    uint64_t s_full[2], q_full[2];
    uint64_t p_full[2], pv_done[2];
    uint64_t unit_full[kUnits], unit_empty[kUnits];
    Unit unit[kUnits];
    uint32_t tmem, dead;
    int32_t start_j, start_h, start_at;
    int32_t firsts[kOwnPlan + 1];
    int64_t sums[kRowThreads / 32];
    PlanTile plan[kOwnPlan];
};

__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// a condition that seldom holds
__device__ __forceinline__ bool rare(bool c) { return __builtin_expect(c, 0); }

template <class T, Mod MOD>
__global__ void __launch_bounds__(kRowThreads, 1) rows_kernel(const __grid_constant__ Rows f, const __grid_constant__ CUtensorMap map) {
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value, kMod = MOD != Mod::kNone;
    constexpr float kFar = kFarOf<T>, kRaise = kRaiseOf<T>, kUnit = kUnitOf<T>;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    uint8_t* const mem = raw + (base - smem_u32(raw));
    const uint32_t ring = base + 2 * kEntryBytes;  // behind the two stages' queries
    __shared__ __align__(16) RowShared sh;
    const KvAttend& a = f.a;
    const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const uint32_t D = a.pages.head_dim;
    volatile uint32_t* dead = &sh.dead;

    auto bar = [&](const uint64_t& b) { return smem_u32(&b); };
    if (tid == 0) {
        for (uint32_t i = 0; i < kRowEntries; ++i) mbar_init(bar(sh.full[i]), 1), mbar_init(bar(sh.empty[i]), 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(sh.s_full[i]), 1), mbar_init(bar(sh.p_full[i]), 128);
            mbar_init(bar(sh.pv_done[i]), 1), mbar_init(bar(sh.q_full[i]), 128);
        }
        for (uint32_t i = 0; i < kUnits; ++i) mbar_init(bar(sh.unit_full[i]), 1), mbar_init(bar(sh.unit_empty[i]), kUnitReaders);
        sh.dead = 0;
        fence_mbar_init();
        tma_prefetch_map(&map);
    }
    // (a unit that was never handed out has no rows: what a warp meets whose wait ran out)
    for (uint32_t i = tid; i < sizeof(sh.unit) / 4; i += kRowThreads) reinterpret_cast<uint32_t*>(sh.unit)[i] = 0;
    if (warp == 9) tmem_alloc(smem_u32(&sh.tmem), 512);
    pdl_launch();
    pdl_wait();
    if (tid == 0) f.join[blockIdx.x].valid = 0;

    const bool own = f.most <= kOwnPlan;
    const PlanTile* const plan = own ? sh.plan : f.plan;
    int64_t total;
    int32_t tiles;
    if (own) {
        tiles = make_plan<kRowThreads>(f, sh.plan, sh.firsts, sh.sums, &total);
        __syncthreads();
    } else {
        total = f.head->total, tiles = f.head->tiles;
    }
    const int64_t K = a.pages.kv_heads;
    total *= K;
    const int64_t blocks = min(int64_t(gridDim.x), total);
    const bool busy = blockIdx.x < blocks;
    const int64_t run0 = busy ? blockIdx.x * total / blocks : 0, run1 = busy ? (blockIdx.x + 1) * total / blocks : 0;
    if (busy) {
        for (int32_t j = int32_t(tid); j < tiles; j += kRowThreads) {
            const PlanTile& t = plan[j];
            const int64_t in = run0 - t.seq_before * K;
            if (in < 0 || in >= t.seq_total * K) continue;
            const int64_t r = in % t.seq_total - (t.before - t.seq_before);
            if (r < 0 || r >= t.nt + f.cost) continue;
            sh.start_j = j, sh.start_h = int32_t(in / t.seq_total), sh.start_at = int32_t(r);
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = 0;  // (all 512 columns are allocated)

    if (busy && warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == 8) {
            // ---------------------------------------------------------- loads
            RowWalk w;
            w.at = run0, w.end = run1, w.j = sh.start_j, w.h = sh.start_h;
            w.t = plan[w.j];
            walk_segment(f, w, run0 - sh.start_at);
            if (w.n < 0) w.n = 0;  // nothing but a unit's cost: a unit without tiles, and without another
            const bool none = w.n == 0;
            uint32_t u = 0;  // units left in shared memory
            auto publish = [&]() -> bool {
                if (!mbar_wait(bar(sh.unit_empty[u % kUnits]), (u / kUnits & 1) ^ 1, dead)) return false;
                Unit& o = sh.unit[u % kUnits];
                if (lane == 0) {
                    o.span = w.t.span, o.q = w.t.q, o.s = w.t.s, o.m = w.t.m, o.h = w.h, o.rows = w.t.rows;
                    o.tile = w.tile, o.n = w.n, o.nt = w.t.nt, o.at = w.at, o.more = !none && w.unit + w.t.nt + f.cost < w.end;
                }
                if (a.tree) {
                    const int32_t ctx = w.t.q.len - w.t.q.n;
                    for (int32_t b = int32_t(lane); b < 64; b += 32)
                        o.draft[b] = b < w.t.q.n ? ctx + __popcll(kv_word(a, w.t.q, b)) - 1 : INT32_MIN;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(sh.unit_full[u % kUnits]));
                ++u;
                return true;
            };
            if (!f.no_loads) publish();
            const uint32_t shift = a.pages.token_shift;
            const uint32_t box = shift < 7 ? 1u << shift : 128u, boxes = 128u / box;
            const uint32_t mask = (1u << shift) - 1;
            const int halves = D > 64 ? 2 : 1;
            uint32_t n = 0;
            bool more = !none && !f.no_loads;
            while (more) {
                const int32_t row_k = int32_t((a.pages.layer * 2 * a.pages.kv_heads + w.h) << shift);
                const int32_t row_v = row_k + int32_t(a.pages.kv_heads << shift);
                const int32_t* table = a.pages.table + uint32_t(w.t.s) * a.pages.table_stride;
                const int32_t slot0 = tile_slot(w.t.span, w.tile), tiles = w.n, len = w.t.q.len;
                for (int32_t i = 0; i < tiles; ++i) {
                    const uint32_t slot = uint32_t(slot0 + i * kTileKeys) + lane * box;
                    int32_t page = -1;
                    if (lane < boxes && slot < uint32_t(len)) page = table[slot >> shift];
                    // what the pool lacks, and what lies behind the sequence, is filled with zeros
                    const int32_t z = uint32_t(page) >= a.pages.total_pages ? int32_t(a.pages.total_pages) : page;
                    const int32_t y = int32_t(slot & mask);
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv, ++n) {
                        const uint32_t e = n % kRowEntries;
                        if (!mbar_wait(bar(sh.empty[e]), (n / kRowEntries & 1) ^ 1, dead)) goto loads_done;
                        if (lane == 0) mbar_expect(bar(sh.full[e]), uint32_t(halves) * 16384u);
                        __syncwarp();
                        if (lane < boxes)
                            for (int x = 0; x < halves; ++x)
                                tma_load(ring + e * kEntryBytes + x * 16384 + lane * box * 128, &map, x * 64,
                                         (kv ? row_v : row_k) + y, z, bar(sh.full[e]));
                    }
                    if (i == 0) {  // the next unit, while this one's loads are under way
                        more = walk_next(f, plan, w);
                        if (more && !publish()) goto loads_done;
                    }
                }
            }
        loads_done:
            __syncwarp();
            if (*dead) {  // the copies in flight land before the block ends
                uint32_t late = 0;
                for (uint32_t k = n > kRowEntries ? n - kRowEntries : 0; k < n; ++k)
                    mbar_wait(bar(sh.full[k % kRowEntries]), k / kRowEntries & 1, &late);
            }
        } else if (warp == 9) {
            // ---------------------------------------------------------- products
            const uint32_t dn = (D + 15) / 16;
            constexpr uint32_t kQk = instr_desc(kBf16, false, false, 128, 128);
            const uint32_t kPv = instr_desc(kBf16, false, true, 128, 0) | (dn * 2) << 17;
            // queries and keys: rows of 64 elements, swizzled; values: the same rows, read along the keys
            const uint64_t qd = smem_desc(base, 16, 1024, 2), kd = smem_desc(ring, 16, 1024, 2), vd = smem_desc(ring, 16384, 1024, 2);
            // Products run in the order of issue, and the queue in front of the tensor cores is short, so what
            // stands between two products must be as well: all of tensor memory is the block's and begins at
            // column 0, and what the first stage has waited for the second one need not. (odd: the tile's
            // parity, whose entries of the ring are 2 odd and 2 odd + 1.)
            uint32_t units = 0, second = 0;   // units begun, and those with a second stage
            uint32_t pp[2] = {0, 0}, kv = 0;  // parities of the next weights of each stage, and of the ring
            int32_t left = 0;                 // tiles of the unit after this one
            bool two = false, follows = false, fresh = true;
            auto qk = [&](uint32_t odd, int st) {
                const uint32_t e = odd * 2;
                const uint64_t k0 = desc_at(kd, e * kEntryBytes), q0 = desc_at(qd, st * kEntryBytes);
                if (elect()) {
#pragma unroll
                    for (uint32_t k = 0; k < 8; ++k) {
                        if (k >= dn) break;
                        const uint32_t off = (k / 4) * 16384 + (k % 4) * 32;
                        mma_ss(st * 128, desc_at(q0, off), desc_at(k0, off), kQk, k != 0);
                    }
                    mma_commit(bar(sh.s_full[st]));
                }
                __syncwarp();
            };
            // (One commit a batch, as far as that goes: each takes a place in the queue. So the tile's keys are
            // handed back behind the first product with its values, and pv_done is for a unit's last tile.)
            auto pv = [&](uint32_t odd, int st, bool end) {
                const uint32_t e = odd * 2 + 1;
                const uint64_t v0 = desc_at(vd, e * kEntryBytes);
                mbar_wait(bar(sh.p_full[st]), pp[st], dead);
                pp[st] ^= 1;
                fence_after();
                if (elect()) {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        mma_ts(256 + st * 128, st * 128 + k * 8, desc_at(v0, k * 2048), kPv, !(fresh && k == 0));
                    if (end) mma_commit(bar(sh.pv_done[st]));
                    if (st == 0) mma_commit(bar(sh.empty[e - 1]));
                    if (st || !two) mma_commit(bar(sh.empty[e]));
                }
                __syncwarp();
            };
            // the next unit: both stages' queries are there
            auto unit = [&]() {
                mbar_wait(bar(sh.unit_full[units % kUnits]), units / kUnits & 1, dead);
                const Unit& o = sh.unit[units % kUnits];
                left = o.n, follows = o.more, two = o.rows > 128;
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(sh.unit_empty[units % kUnits]));
                mbar_wait(bar(sh.q_full[0]), units & 1, dead);
                if (two) mbar_wait(bar(sh.q_full[1]), second++ & 1, dead);
                ++units;
            };
            // A tile (its values are there): its products with them, and between these the next tile's scores;
            // false behind the last. Waits that seldom wait stand where products are queued.
            auto tile = [&](uint32_t odd) {
                const bool same = --left > 0;
                kv ^= odd;
                pv(odd, 0, !same);
                if (!rare(!same)) {
                    mbar_wait(bar(sh.full[2 - 2 * odd]), kv, dead);
                    qk(odd ^ 1, 0);
                }
                if (two) pv(odd, 1, !same);
                if (rare(!same)) {
                    if (!follows || *dead) return false;
                    unit();
                    mbar_wait(bar(sh.full[2 - 2 * odd]), kv, dead);
                    qk(odd ^ 1, 0);
                }
                const bool ok = mbar_wait(bar(sh.full[3 - 2 * odd]), kv, dead);
                if (two) qk(odd ^ 1, 1);
                fresh = !same;
                return ok;
            };
            unit();
            if (left) {
                mbar_wait(bar(sh.full[0]), 0, dead);
                fence_after();
                qk(0, 0);
                if (two) qk(0, 1);
                mbar_wait(bar(sh.full[1]), 0, dead);
                for (uint32_t odd = 0; tile(odd); odd ^= 1) {
                }
            }
            if (*dead) {  // the products in flight end before the tensor memory is freed
                const uint64_t t0 = now_ns();
                while (now_ns() - t0 < 50000) {
                }
            }
        }
    } else if (busy) {
        // ---------------------------------------------------------- softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
        const int st = warp / 4;
        const uint32_t r = tid % 128;  // the row of the stage
        const uint32_t lanes = tmem + ((warp % 4) << 21), s_at = lanes + st * 128, o_at = lanes + 256 + st * 128;
        // a negative scale turns the queries' signs, so that the largest product is the largest score
        const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
        const float k2 = fabsf(a.scale) * kLog2e;
        const bool cap = kMod && a.softcap != 0.0f;
        const float cap_in = cap ? fabsf(a.scale) / a.softcap : 0.0f, cap2 = a.softcap * kLog2e;
        const float kk = cap ? 1.0f : k2;  // what is left to scale after the cap
        bool gone = false;  // a wait ran out: what lies in shared memory is not to be gone by
        auto unit = [&](uint32_t u) -> const Unit& {
            const bool got = mbar_wait(bar(sh.unit_full[u % kUnits]), u / kUnits & 1, dead);
            if (!__all_sync(0xFFFFFFFFu, got)) gone = true;
            return sh.unit[u % kUnits];
        };
        auto done_with = [&](uint32_t u) {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sh.unit_empty[u % kUnits]));
        };
        // a row of a unit's queries to shared memory, 64 dimensions at a time, 128-byte swizzle
        auto load_q = [&](const Unit& o) {
            if (st && o.rows <= 128) return;  // no second stage
            const uint32_t row = uint32_t(o.m) * kRows + st * 128 + r;
            const bool real = int32_t(st * 128 + r) < o.rows && !gone;
            const uint32_t t = row / a.group, g = row % a.group;
            const uint4* src = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + uint64_t(o.q.first + t) * a.q_stride +
                                                              uint64_t(o.h * a.group + g) * D);
            uint8_t* dst = mem + st * kEntryBytes + r * 128;
#pragma unroll
            for (uint32_t x0 = 0; x0 < 16; x0 += 8) {
                uint4 v[8];
#pragma unroll
                for (uint32_t x = 0; x < 8; ++x) v[x] = real && (x0 + x) * 8 < D ? src[x0 + x] : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (uint32_t x = 0; x < 8; ++x)
                    *reinterpret_cast<uint4*>(dst + x0 / 8 * 16384 + (x ^ (r % 8)) * 16) =
                        make_uint4(v[x].x ^ flip, v[x].y ^ flip, v[x].z ^ flip, v[x].w ^ flip);
            }
            fence_async_smem();
            mbar_arrive(bar(sh.q_full[st]));
        };
        {
            const Unit& o = unit(0);
            if (tid == 0) {
                // this run's note of a unit that began in the run before it
                const int64_t u0 = o.at - o.tile;
                const int64_t b0 = ((u0 + 1) * blocks - 1) / total, b1 = ((u0 + o.nt) * blocks - 1) / total;
                const bool here = !gone && o.n > 0 && o.tile > 0 && b0 + 1 == int64_t(blockIdx.x);
                f.join[blockIdx.x] = {o.q.first, o.m, o.rows, o.h, int32_t(b0), int32_t(b1), b0 * total / blocks != u0, here};
            }
            load_q(o);
        }
        uint32_t n = 0, on = 0;  // tiles and units of this stage
        bool more = unit(0).n > 0;
        if (!more) done_with(0);
        for (uint32_t u = 0; more; ++u) {
            const Unit& o = unit(u);
            more = o.more && !gone;
            if (st && o.rows <= 128) {
                if (more) load_q(unit(u + 1));
                done_with(u);
                continue;
            }
            const KvSpan span = o.span;
            const int32_t ctx = o.q.len - o.q.n, tiles = o.n;
            const bool real = int32_t(st * 128 + r) < o.rows && !gone;
            KvQuery qy{0, INT32_MAX, 0, 0};
            float slope = 0.0f;
            if (real) {
                const uint32_t row = uint32_t(o.m) * kRows + st * 128 + r;
                qy = kv_query(a, o.q, int32_t(row / a.group));
                if (kMod && a.slopes) slope = a.slopes[o.h * a.group + row % a.group] * kLog2e;
            }
            if (a.tree && real)  // of the drafted tokens, those that are there and inside the window
                for (int b = 0; b < 64; ++b)
                    if (o.draft[b] < qy.first) qy.word &= ~(uint64_t(1) << b);
            float ref = -INFINITY, pend = 1.0f;  // pend: what O, once it is there, has to be scaled by
            bool late = false;                   // ... of some row of the warp
            KvSum sum;
            for (int32_t i = 0; i < tiles; ++i, ++n) {
                const int32_t slot0 = tile_slot(span, o.tile + i);
                const bool masked = slot0 < span.all_lo || slot0 + kTileKeys > span.all_hi;
                const bool drafts = a.tree && slot0 + kTileKeys > ctx;
                // the row's visible keys of the tile, a bit each
                uint64_t see0 = 0, see1 = 0;
                if (rare(masked)) {
                    const int32_t d = ctx - slot0;
                    if (drafts) {
                        see0 = d >= 64 ? 0 : d >= 0 ? qy.word << d : d > -64 ? qy.word >> -d : 0;
                        see1 = d >= 128 ? 0 : d >= 64 ? qy.word << (d - 64) : d > 0 ? qy.word >> (64 - d) : 0;
                    }
                    auto below = [](int64_t n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; };
                    const int64_t f0 = int64_t(qy.first) - slot0, l0 = int64_t(qy.last) - slot0;
                    see0 |= below(l0) & ~below(f0);
                    see1 |= below(l0 - 64) & ~below(f0 - 64);
                }
                mbar_wait(bar(sh.s_full[st]), n & 1, dead);
                fence_after();
                if (rare(cap)) {
                    // the cap takes two special functions a score: once, back to tensor memory
#pragma unroll 1
                    for (int c0 = 0; c0 < 128; c0 += 32) {
                        float y[32];
                        tmem_ld32(s_at + c0, y);
                        wait_ld(y);
#pragma unroll
                        for (int c = 0; c < 32; ++c) y[c] = capped<MOD == Mod::kFine>(y[c], cap_in, cap2);
                        tmem_st16(s_at + c0, reinterpret_cast<uint32_t*>(y));
                        tmem_st16(s_at + c0 + 16, reinterpret_cast<uint32_t*>(y) + 16);
                    }
                    wait_st();
                }
                float x[128];
                tmem_ld32(s_at, x), tmem_ld32(s_at + 32, x + 32), tmem_ld32(s_at + 64, x + 64), tmem_ld32(s_at + 96, x + 96);
                wait_ld(x);
                // bias (scores in units of log2 from here on, if kMod) and mask
                if (kMod) {
                    // (differences first: fp32 does not count beyond 2^24)
                    const float ahead = float(qy.pos - slot0);
                    if (rare(drafts && a.slopes)) {
#pragma unroll
                        for (int c = 0; c < 128; ++c) {
                            const int32_t key = slot0 + c;
                            const int32_t at = key >= ctx ? o.draft[min(key - ctx, 63)] : key;
                            const float far = float(int32_t(uint32_t(qy.pos) - uint32_t(at)));
                            x[c] = x[c] * kk - slope * fabsf(far);
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < 128; ++c) x[c] = x[c] * kk - slope * fabsf(ahead - float(c));
                    }
                }
                if (rare(masked)) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) x[c] = (c < 64 ? see0 >> c : see1 >> (c - 64)) & 1 ? x[c] : -INFINITY;
                }
                // weights against the reference so far; the first keys that a row sees set it
                float part;
                bool set = i == 0;
#pragma unroll 1
                for (int pass = 0; pass < 2; ++pass) {
                    if (rare(set)) {
                        float t0 = max3(x[0], x[1], x[2]), t1 = x[3];
#pragma unroll
                        for (int c = 4; c < 128; c += 4) t0 = max3(t0, x[c], x[c + 1]), t1 = max3(t1, x[c + 2], x[c + 3]);
                        const float m = fmaxf(t0, t1) * (kMod ? 1.0f : k2) - kLift<T>;
                        if (m > ref) {
                            const float by = i ? exp2_approx(ref - m) : 1.0f;  // at first there is nothing to scale
                            ref = m, sum.scale(by), pend *= by;
                        }
                        late = i != 0;
                    }
                    const float off = ref == -INFINITY ? 0.0f : -ref;
                    const uint64_t off2 = pack2(off, off), by2 = pack2(kMod ? 1.0f : k2, kMod ? 1.0f : k2);
                    uint64_t sum2 = 0, sum3 = 0;
#pragma unroll
                    for (int c0 = 0; c0 < 128; c0 += 32) {
                        uint32_t p[16];
#pragma unroll
                        for (int c = 0; c < 32; c += 4) {
                            float u0, u1, u2, u3;
                            unpack2(fma2(pack2(x[c0 + c], x[c0 + c + 1]), by2, off2), u0, u1);
                            unpack2(fma2(pack2(x[c0 + c + 2], x[c0 + c + 3]), by2, off2), u2, u3);
                            u0 = exp2_approx(u0), u1 = exp2_approx(u1), u2 = exp2_approx(u2), u3 = exp2_approx(u3);
                            sum2 = add2(sum2, pack2(u0, u1));
                            sum3 = add2(sum3, pack2(u2, u3));
                            p[c / 2] = Kv16<T>::from2(u0, u1);
                            p[c / 2 + 1] = Kv16<T>::from2(u2, u3);
                        }
                        tmem_st16(s_at + c0 / 2, p);  // weights 2c and 2c + 1 to column c, over scores that are read
                    }
                    float u0, u1;
                    unpack2(add2(sum2, sum3), u0, u1);
                    part = u0 + u1;
                    // too far above the reference for the weights' type, or the first that the row sees:
                    // raised at once, and once more
                    set = __any_sync(0xFFFFFFFFu, part > kFar || (ref == -INFINITY && (!masked || (see0 | see1))));
                    if (!rare(set)) break;
                    wait_st();
                }
                if (rare(late)) {
                    // (the products of the tile before were complete before this one's scores)
#pragma unroll 1
                    for (uint32_t d0 = 0; d0 < D; d0 += 16) {
                        float y[16];
                        tmem_ld16(o_at + d0, y);
                        wait_ld(y);
#pragma unroll
                        for (int c = 0; c < 16; ++c) y[c] *= pend;
                        tmem_st16(o_at + d0, reinterpret_cast<uint32_t*>(y));
                    }
                    pend = 1.0f, late = false;
                }
                if (rare(st == 0 && (slot0 < span.lo || slot0 + kTileKeys > span.hi))) {
                    // values that none of the unit's queries sees may be anything: zeros, as their weights are
                    const uint32_t e = (2 * n + 1) % kRowEntries;
                    mbar_wait(bar(sh.full[e]), (2 * n + 1) / kRowEntries & 1, dead);
                    const int32_t key = slot0 + int32_t(r);
                    if (key < span.lo || key >= span.hi) {
#pragma unroll 1
                        for (int k = 0; k < 16; ++k)
                            if (k < 8 || D > 64)
                                *reinterpret_cast<uint4*>(mem + 2 * kEntryBytes + e * kEntryBytes + k / 8 * 16384 + r * 128 +
                                                          k % 8 * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_smem();
                }
                wait_st();
                fence_before();
                mbar_arrive(bar(sh.p_full[st]));
                sum.add(part);
                // for the next tile: the reference, and what the accumulators follow it by
                late = __any_sync(0xFFFFFFFFu, part > kRaise);
                if (rare(late) && part > kRaise) {
                    ref += log2f(part) - kLift<T>;
                    pend = kUnit / part;
                    sum.scale(pend);
                }
            }
            if (more) load_q(unit(u + 1));  // the next unit's scores start while this one is written
            mbar_wait(bar(sh.pv_done[st]), on++ & 1, dead);
            fence_after();
            const float all = sum.value();
            if (tiles == o.nt) {
                const bool real = int32_t(st * 128 + r) < o.rows && !gone;
                const uint32_t row = uint32_t(o.m) * kRows + st * 128 + r;
                const float by = all == 0.0f ? 0.0f : pend / all;
                const uint64_t orow = uint64_t(o.q.first) + row / a.group;
                const uint32_t head = o.h * a.group + row % a.group;
                T* out = static_cast<T*>(a.out) + orow * a.out_stride + uint64_t(head) * D;
                for (uint32_t c0 = 0; c0 < D; c0 += 16) {
                    float y[16];
                    tmem_ld16(o_at + c0, y);
                    wait_ld(y);
#pragma unroll
                    for (int c = 0; c < 16; c += 8) {
                        if (!real || c0 + c >= D) continue;
                        float z[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) z[k] = y[c + k] * by;
                        kv_store8(out + c0 + c, z);
                    }
                }
                if (real && a.lse) a.lse[orow * a.q_heads + head] = all == 0.0f ? -INFINITY : (ref + log2f(all)) * kLn2;
            } else {
                // a part of the unit: [head_dim / 4][256 rows] of four, maxima, sums
                float* part = f.part + (uint64_t(blockIdx.x) * 2 + (o.at == run0 ? 0 : 1)) * kRowPart;
                const uint32_t pr = st * 128 + r;
                for (uint32_t c0 = 0; c0 < D; c0 += 16) {
                    float y[16];
                    tmem_ld16(o_at + c0, y);
                    wait_ld(y);
#pragma unroll
                    for (int c = 0; c < 16; c += 4)
                        __stcg(reinterpret_cast<float4*>(part) + (c0 + c) / 4 * kRows + pr,
                               make_float4(y[c] * pend, y[c + 1] * pend, y[c + 2] * pend, y[c + 3] * pend));
                }
                __stcg(part + kRows * 128 + pr, ref);
                __stcg(part + kRows * 128 + kRows + pr, all);
            }
            fence_before();
            done_with(u);
        }
    }
    __syncthreads();
    if (tid == 0 && *dead) *f.fault = 1;
    if (warp == 9) {
        fence_after();
        tmem_free(sh.tmem, 512);
    }
}

// Joins the units that lie in several runs: a block for 32 rows of a run's note, a
// lane a row.
template <class T>
__global__ void __launch_bounds__(512) rows_join_kernel(const __grid_constant__ Rows f) {
    const KvAttend& a = f.a;
    pdl_launch();
    pdl_wait();
    const Join j = f.join[blockIdx.x];
    if (!j.valid) return;
    const uint32_t warp = threadIdx.x / 32, D = a.pages.head_dim;  // warp: which four dimensions, and four more 64 on
    const int32_t r = int32_t(blockIdx.y * 32 + threadIdx.x % 32);
    if (r >= j.rows || warp * 4 >= D) return;
    const bool more = warp * 4 + 64 < D;
    float top = -INFINITY, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f), o1 = o;
    auto add = [](float4& s, float x, const float4& v) { s.x += x * v.x, s.y += x * v.y, s.z += x * v.z, s.w += x * v.w; };
    auto by = [](float4& s, float x) { s.x *= x, s.y *= x, s.z *= x, s.w *= x; };
    for (int32_t b0 = j.b0; b0 <= j.b1; b0 += 4) {  // four parts' loads at a time
        float m[4], s[4], now = top;
        float4 v[4], v1[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int32_t b = b0 + k;
            m[k] = -INFINITY, s[k] = 0.0f;
            v[k] = v1[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (b > j.b1) continue;
            const float* p = f.part + (uint64_t(b) * 2 + (b == j.b0 && j.second ? 1 : 0)) * kRowPart;
            m[k] = __ldcg(p + kRows * 128 + r), s[k] = __ldcg(p + kRows * 128 + kRows + r);
            v[k] = __ldcg(reinterpret_cast<const float4*>(p) + warp * kRows + r);
            if (more) v1[k] = __ldcg(reinterpret_cast<const float4*>(p) + (warp + 16) * kRows + r);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) now = fmaxf(now, m[k]);
        const float was = top == now ? 1.0f : exp2_approx(top - now);
        l *= was, by(o, was), by(o1, was);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (b0 + k > j.b1) continue;
            const float x = m[k] == now ? 1.0f : exp2_approx(m[k] - now);
            l += x * s[k], add(o, x, v[k]), add(o1, x, v1[k]);
        }
        top = now;
    }
    const uint32_t row = uint32_t(j.m) * kRows + uint32_t(r), head = uint32_t(j.h) * a.group + row % a.group;
    const uint64_t orow = uint64_t(j.first) + row / a.group;
    const float rl = l == 0.0f ? 0.0f : 1.0f / l;
    T* out = static_cast<T*>(a.out) + orow * a.out_stride + uint64_t(head) * D + warp * 4;
    by(o, rl), by(o1, rl);
    *reinterpret_cast<uint2*>(out) = make_uint2(Kv16<T>::from2(o.x, o.y), Kv16<T>::from2(o.z, o.w));
    if (more) *reinterpret_cast<uint2*>(out + 64) = make_uint2(Kv16<T>::from2(o1.x, o1.y), Kv16<T>::from2(o1.z, o1.w));
    if (a.lse && warp == 0) a.lse[orow * a.q_heads + head] = l == 0.0f ? -INFINITY : (top + log2f(l)) * kLn2;
}

constexpr uint64_t up256(uint64_t n) { return (n + 255) / 256 * 256; }
// the parts of the workspace, in order: head, notes, firsts, plan, parts
uint64_t plan_tiles(uint64_t n_seqs, uint64_t n_tokens, uint64_t group) { return n_tokens * group / kRows + n_seqs + 1; }

template <class T, Mod MOD>
cudaError_t launch_rows_as(const Rows& f, const CUtensorMap& map, uint32_t sms, cudaStream_t stream) {
    static std::atomic<uint64_t> ready{0};  // devices whose kernel may take this much shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !(ready.load() >> dev & 1)) {
        e = cudaFuncSetAttribute(rows_kernel<T, MOD>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kRowSmem));
        if (e != cudaSuccess) return e;
        if (dev < 64) ready |= uint64_t(1) << dev;
    }
    if (f.most > kOwnPlan && (e = launch_pdl(plan_kernel, dim3(1), kPlanThreads, 0, stream, f)) != cudaSuccess) return e;
    const uint32_t blocks = attend_blocks(f.a, sms, f.most);
    if ((e = launch_pdl(rows_kernel<T, MOD>, dim3(blocks), kRowThreads, kRowSmem, stream, f, map)) != cudaSuccess) return e;
    return launch_pdl(rows_join_kernel<T>, dim3(blocks, kRows / 32), 512, 0, stream, f);
}

template <class T>
cudaError_t launch_rows(const KvAttend& a, const KvLaunch& l, cudaStream_t stream) {
    Rows f;
    f.a = a;
    uint8_t* p = static_cast<uint8_t*>(l.workspace);
    f.head = reinterpret_cast<PlanHead*>(p);
    p += 256;
    f.join = reinterpret_cast<Join*>(p);
    p += up256(l.sms * sizeof(Join));
    f.firsts = reinterpret_cast<int32_t*>(p);
    p += up256((uint64_t(a.tok.n_seqs) + 1) * 4);
    f.plan = reinterpret_cast<PlanTile*>(p);
    f.most = uint32_t(plan_tiles(a.tok.n_seqs, a.tok.n_tokens, a.group));
    p += up256(uint64_t(f.most) * sizeof(PlanTile));
    f.part = reinterpret_cast<float*>(p);
    f.fault = l.fault;
    f.no_loads = l.no_loads;
    const Mod mod = mod_of(a);
    // (Without Mod::kNone scores are scaled before they are masked: a scale of 0 would turn a masked -infinity into NaN.)
    const bool none = mod == Mod::kNone && a.scale != 0.0f;
    f.cost = none ? kUnitCost : kUnitCostMod;
    if (none) return launch_rows_as<T, Mod::kNone>(f, *l.map, l.sms, stream);
    return mod == Mod::kFine ? launch_rows_as<T, Mod::kFine>(f, *l.map, l.sms, stream)
                             : launch_rows_as<T, Mod::kSome>(f, *l.map, l.sms, stream);
}

}  // namespace
}  // namespace t2i
