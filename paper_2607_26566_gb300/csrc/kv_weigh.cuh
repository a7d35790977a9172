// Accumulated attention: what each slot of the cache gets from new tokens, the sum of exp(score - lse) over the tokens
// that see it and the heads that share its key.
//
// With an attention's log-sum-exp at hand no maximum and no second product is needed: S^T = K Q^T on the tensor cores,
// 128 keys to the rows of a product and N queries to its columns, so that a thread has one key, adds its row up, and
// nothing goes from thread to thread. A unit is 256 keys of one key head in two halves, one to each half of the warps
// that add up: its keys are loaded once (TMA), its queries, 128 columns at a time, once for both halves.
//
// Two regimes. Where all queries of a key head are one column tile or two (a decoding step, an observation window) the
// keys stream through a ring: one tile over long contexts is bound by reading them, two by what a unit takes (3.15 us, of
// which the sums of two steps are 2.1). Of more (a prompt) keys stay while column tiles pass, and the call is bound by
// shared memory, whose data stage is 90% busy: 51% with threads' reads, in the loop the log-sum-exps, 38% with the products'
// operands; beside it an exponential a score.
//
// Work split: the column tiles (steps) of all units, in order, are cut into equal runs, one to an SM. A unit that lies in
// several runs is joined by a second kernel, in the order of the runs; with one or two tiles units are not cut. Results do
// not depend on timing.
//
// Accuracy: products are exact, sums fp32 (what a thread adds up over tiles keeps what its additions lose). The argument of
// the exponential, score - lse in units of log2, is rounded once in fp32 from a scale that is rounded too: 2e-6 of a
// weight whose score and lse are 30, 3e-7 of a prompt's sums.
//
// Measured, 32 heads over 8 of 128: one token over 700 slots 5.6 us; a token each of 64 sequences of up to 16k slots (1.16
// GB) 178 us, 6.5 TB/s; a prompt of 8190 tokens 244-263 us, 1.05-1.13 PFLOP/s of what is visible, where products and loads
// alone (nothing added up) took 193; 32 tokens of nine prompts of up to 7k, 28 heads over 4, 23-24 us. (With half of a
// tile's columns to each group of warps, in place of tiles in turn, the last two took 257 and 23.5.)
#pragma once

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "kv_attend.cuh"
#include "t2istore.h"

namespace t2i {
namespace {

using namespace tc;

constexpr int kUnitKeys = 256;
constexpr uint32_t kHalfSlot = 16384;  // 128 keys of 64 elements
constexpr uint32_t kWeighUnits = 8;    // handed out at a time
constexpr int kPartFloats = kUnitKeys;

// Column tiles of a sequence: one; two, one to a group of warps, whose log-sum-exps stay, like the one's, while a run is in
// one key head; or so many that keys stay while they pass, and units are cut where runs end.
enum class Tiles { kOne, kFew, kMany };

template <int N, int NS, Tiles HOW>
struct WeighShape {
    static constexpr uint32_t kHalf = kHalfSlot * NS;                        // a half's keys
    // ... in both halves' rings. A half has its own: with one ring the product warp of one half could wait for a phase of an
    // entry that the other half was still two behind on.
    static constexpr uint32_t kKeys = (HOW == Tiles::kMany ? 3 : N > 32 ? 4 : 6) * (NS == 1 ? 2 : 1);
    static constexpr uint32_t kKeys0 = (kKeys + 1) / 2, kKeys1 = kKeys / 2;
    // the entry of a half's n-th keys, and its phase
    static __device__ __forceinline__ uint32_t entry(uint32_t half, uint32_t n) { return half ? kKeys0 + n % kKeys1 : n % kKeys0; }
    static __device__ __forceinline__ uint32_t phase(uint32_t half, uint32_t n) { return (half ? n / kKeys1 : n / kKeys0) & 1; }
    static constexpr uint32_t kQ = N * 128 * NS;                             // a column tile
    static constexpr uint32_t kQs = HOW == Tiles::kMany ? (NS == 1 ? 5 : 3) : N == 16 || NS == 1 ? 4 : 2;
    static constexpr uint32_t kBufs = N > 32 ? 2 : 4;                      // tiles of scores of each half
    static_assert(N != 128 || kBufs == 2, "a place for each group's scores");
    static constexpr uint32_t kTmem = 2 * kBufs * N;
    static constexpr uint32_t kBytes = 1024 + kHalf * kKeys + kQ * kQs;
    // The warps that add up come in groups of four: one a half, or two, which take tiles (of one tile: units) in turn. Then a
    // loading warp and a product warp for each half (one's products run while the other waits; of many tiles there is one
    // loading warp, and one that idles).
    static constexpr int kGroups = N == 128 ? 4 : 2;
    static constexpr int kCols = N;
    static constexpr int kSpanCols = N < 64 ? N : 64;  // whose spans are held at a time
    static constexpr int kSumWarps = 4 * kGroups, kThreads = kSumWarps * 32 + 128;
    static constexpr int kRegs = 96, kSumRegs = 104, kOtherRegs = 64;
    static_assert(kGroups != 4 || kSumRegs * kSumWarps * 32 + kOtherRegs * 128 <= kRegs * kThreads, "what a block was launched with");
    static constexpr uint32_t kFixed = 8192 + kSumWarps * (kCols * 8 + kSpanCols * 8);  // static shared memory, at most
    static_assert(kBytes + kFixed + 1024 <= 228 * 1024, "an SM's shared memory");
    static constexpr int kChunk = kCols < 32 ? kCols : 32;  // columns that a thread works on at a time
};

struct WeighUnit {
    KvSeq q;
    int32_t s, h, slot0;  // the unit's first slot
    int32_t tile, n;      // the segment's first column tile, and how many
    int32_t dry;          // no token sees its slots
    int32_t whole, part;  // the segment is all of the unit; else its place in the workspace
    int32_t more;
};
struct WeighJoin {
    int32_t s, h, slot0, ctx, len;
    int32_t b0, b1, second, valid;
};

struct Weigh {
    KvWeigh w;
    int32_t per_tile;   // tokens of a column tile
    int32_t per_token;  // columns of a token in a tile
    int32_t slices;     // column tiles of a token (1 unless it has more heads than a tile columns)
    int32_t skips;      // units that no token sees are left alone
    WeighJoin* join;    // [blocks]
    float* part;        // [2 * blocks][kPartFloats]
    int2* hulls;        // with spans: slots outside which a column tile's tokens see nothing
    uint32_t* fault;
    uint32_t no_loads;
};

__device__ __forceinline__ int32_t weigh_tokens(const KvAttend& a, const KvSeq& q) { return min(q.n, int32_t(a.tok.max_new)); }

// Units of a sequence: those of its sinks, then those from its windows on; all where the weights so far decay.
struct UnitList {
    int32_t head, lo, n;
};
__device__ __forceinline__ UnitList unit_list(const Weigh& f, const KvSeq& q) {
    UnitList u{0, 0, 0};
    if (q.n == 0) return u;
    const KvAttend& a = f.w.a;
    if (f.skips && a.window) {
        const int64_t lo = int64_t(q.len) - q.n + 1 - int64_t(a.window);
        if (lo > 0) {
            u.lo = int32_t(lo / kUnitKeys);
            u.head = min((int32_t(a.sinks) + kUnitKeys - 1) / kUnitKeys, u.lo);
        }
    }
    u.n = u.head + (q.len + kUnitKeys - 1) / kUnitKeys - u.lo;
    return u;
}
__device__ __forceinline__ int32_t unit_slot(const UnitList& u, int32_t i) { return (i < u.head ? i : u.lo + i - u.head) * kUnitKeys; }

// The column tiles [lo, hi) that see something of a unit; none: hi <= lo.
__device__ __forceinline__ int2 unit_tiles(const Weigh& f, const KvSeq& q, uint32_t s, int32_t slot0) {
    const KvAttend& a = f.w.a;
    const int32_t ctx = q.len - q.n, m = weigh_tokens(a, q), slot1 = min(slot0 + kUnitKeys, q.len);
    if (a.spans) {
        const int2* const hull = f.hulls + q.first / f.per_tile + s;
        const int32_t tiles = (m + f.per_tile - 1) / f.per_tile;
        int2 r = make_int2(tiles, 0);
        for (int32_t t = 0; t < tiles; ++t) {
            const int2 x = hull[t];
            if (x.x < slot1 && x.y > slot0) r.x = min(r.x, t), r.y = t + 1;
        }
        return make_int2(r.x * f.slices, r.y * f.slices);
    }
    const int32_t i0 = max(0, slot0 - ctx);
    int64_t i1 = m;
    if (a.window && slot0 >= int32_t(a.sinks)) i1 = min(i1, int64_t(slot1) - 1 + int64_t(a.window) - ctx);
    if (i0 >= i1) return make_int2(0, 0);
    return make_int2(i0 / f.per_tile * f.slices, int32_t((i1 + f.per_tile - 1) / f.per_tile) * f.slices);
}
// What a unit costs where runs are cut: its steps, and so many before them (its keys' way, tiles with a mask, its sums'
// way out). Measured with 4, 6 and 9: prompts of 4,096 tokens 76, 74, 77 us, of 8,190 252, 246, 246 (before tiles were taken
// in turn with 0, 2, 4, 8 and 14 284, 273, 265, 262 and 266).
constexpr int32_t kUnitCost = 6;
__device__ __forceinline__ int32_t unit_cost(int2 tiles) { return tiles.y > tiles.x ? kUnitCost + tiles.y - tiles.x : 1; }

// The cost of one head of a sequence: its units, where none is cut; else by a warp.
template <bool FLAT>
__device__ __forceinline__ int64_t seq_cost(const Weigh& f, const KvSeq& q, uint32_t s, uint32_t lane) {
    const UnitList u = unit_list(f, q);
    if (FLAT) return u.n;
    int64_t n = 0;
    for (int32_t i = int32_t(lane); i < u.n; i += 32) n += unit_cost(unit_tiles(f, q, s, unit_slot(u, i)));
#pragma unroll
    for (int d = 16; d; d >>= 1) n += __shfl_xor_sync(0xFFFFFFFFu, n, d);
    return n;
}

struct WeighShared {
    uint64_t k_full[12], k_empty[12], q_full[5], q_empty[5];
    uint64_t s_full[2][4], s_empty[2][4];
    uint64_t sum_full[2][2], sum_empty[2][2];  // [half][parity of the unit]
    float sum[2][2][128];  // of the groups with the odd tiles
    uint64_t unit_full[kWeighUnits], unit_empty[kWeighUnits];
    WeighUnit unit[kWeighUnits];
    uint32_t tmem, dead;
    int32_t start_seq;
    int64_t start_rest, start_steps;
    int64_t sums[20];
};

// Spans of column tiles, a thread a tile.
__global__ void __launch_bounds__(128) hull_kernel(const __grid_constant__ Weigh f) {
    const KvAttend& a = f.w.a;
    pdl_launch();
    pdl_wait();
    const uint32_t s = blockIdx.x;
    const KvSeq q = kv_seq(a.pages, a.tok, s);
    const int32_t m = weigh_tokens(a, q), tiles = (m + f.per_tile - 1) / f.per_tile;
    for (int32_t t = int32_t(threadIdx.x); t < tiles; t += 128) {
        int2 r = make_int2(INT32_MAX, 0);
        for (int32_t i = t * f.per_tile; i < min(m, (t + 1) * f.per_tile); ++i) {
            const int2 x = reinterpret_cast<const int2*>(a.spans)[q.first + i];
            const int32_t lo = max(x.x, 0), hi = min(x.y, q.len);
            if (hi > lo) r.x = min(r.x, lo), r.y = max(r.y, hi);
        }
        f.hulls[q.first / f.per_tile + s + t] = r;
    }
}

template <class T, int N, int NS, bool MOD, Tiles HOW>
__global__ void __launch_bounds__(WeighShape<N, NS, HOW>::kThreads, 1)
    weigh_kernel(const __grid_constant__ Weigh f, const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap q_map) {
    using Sh = WeighShape<N, NS, HOW>;
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    constexpr bool kFlat = HOW != Tiles::kMany;  // units are not cut
    constexpr int kChunk = Sh::kChunk;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t ring = base, qs = ring + Sh::kHalf * Sh::kKeys;
    __shared__ __align__(16) WeighShared sh;
    constexpr int kThreads = Sh::kThreads, kSumWarps = Sh::kSumWarps, kCols = Sh::kCols;
    // each adding warp's own: of its columns the log-sum-exps in units of log2, negative; spans, slopes
    __shared__ __align__(16) float lse_of[kSumWarps][kCols];
    __shared__ __align__(16) int2 span_of[kSumWarps][Sh::kSpanCols];
    __shared__ __align__(16) float slope_of[MOD ? kSumWarps : 1][kCols];
    __shared__ __align__(16) float token_of[MOD ? N : 4];  // a column's token, counted in the tile
    static_assert(sizeof(WeighShared) + N * 4 <= 8192, "kFixed");
    const KvAttend& a = f.w.a;
    const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    volatile uint32_t* dead = &sh.dead;
    auto bar = [&](const uint64_t& b) { return smem_u32(&b); };
    if (tid == 0) {
        for (uint32_t i = 0; i < Sh::kKeys; ++i) mbar_init(bar(sh.k_full[i]), 1), mbar_init(bar(sh.k_empty[i]), 1);
        for (uint32_t i = 0; i < Sh::kQs; ++i) mbar_init(bar(sh.q_full[i]), 1), mbar_init(bar(sh.q_empty[i]), 2);
        for (uint32_t i = 0; i < Sh::kBufs; ++i)
            for (int h = 0; h < 2; ++h) mbar_init(bar(sh.s_full[h][i]), 1), mbar_init(bar(sh.s_empty[h][i]), 4);
        for (uint32_t i = 0; i < kWeighUnits; ++i) mbar_init(bar(sh.unit_full[i]), 1), mbar_init(bar(sh.unit_empty[i]), kSumWarps + 2);
        for (int h = 0; h < 2; ++h)
            for (int i = 0; i < 2; ++i) mbar_init(bar(sh.sum_full[h][i]), 4), mbar_init(bar(sh.sum_empty[h][i]), 4);
        sh.dead = 0;
        sh.start_seq = -1;
        fence_mbar_init();
        tma_prefetch_map(&map), tma_prefetch_map(&q_map);
    }
    {  // rows of the queries' ring that no box fills: their columns, whose log-sum-exp is infinite, add 0 (see `odd`)
        const uint32_t real = uint32_t(f.per_tile * f.per_token), idle = N - real;
        for (uint32_t i = tid; i < idle * Sh::kQs * NS * 8; i += kThreads) {
            const uint32_t row = i / 8 % idle, piece = i / 8 / idle;
            *reinterpret_cast<uint4*>(raw + (qs - smem_u32(raw)) + piece * (N * 128) + (real + row) * 128 + i % 8 * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_async_smem();
    }
    if (MOD && tid < N) token_of[tid] = float(int32_t(tid) / f.per_token);
    if (warp == kSumWarps + 1) tmem_alloc(smem_u32(&sh.tmem), Sh::kTmem);
    pdl_launch();
    pdl_wait();
    if (!kFlat && tid == 0) f.join[blockIdx.x].valid = 0;

    // the block's run of steps: sequences by threads (by warps, where a unit may have several steps)
    const int64_t K = a.pages.kv_heads;
    const uint32_t who = kFlat ? tid : warp, all = kFlat ? kThreads : kThreads / 32;
    const uint32_t per = (a.tok.n_seqs + all - 1) / all;
    int64_t mine = 0;
    for (uint32_t s = who * per; s < min(a.tok.n_seqs, (who + 1) * per); ++s)
        mine += seq_cost<kFlat>(f, kv_seq(a.pages, a.tok, s), s, lane);
    int64_t lo = 0, total = 0;  // the cost of a head of the sequences before, and of all
    if (kFlat) {
        int64_t inc = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t o = __shfl_up_sync(0xFFFFFFFFu, inc, d);
            if (lane >= uint32_t(d)) inc += o;
        }
        if (lane == 31) sh.sums[warp] = inc;
        lo = inc - mine;
    } else if (lane == 0) {
        sh.sums[warp] = mine;
    }
    fence_before();
    __syncthreads();
    fence_after();
    for (uint32_t i = 0; i < kThreads / 32; ++i) {
        if (i < warp) lo += sh.sums[i];
        total += sh.sums[i];
    }
    total *= K;
    const int64_t blocks = min(int64_t(gridDim.x), total);
    bool busy = blockIdx.x < blocks;
    const int64_t run0 = busy ? blockIdx.x * total / blocks : 0, run1 = busy ? (blockIdx.x + 1) * total / blocks : 0;
    if (busy && run0 >= lo * K && run0 < (lo + mine) * K) {
        int64_t p = lo * K;
        // (bounded, like the loads' way from sequence to sequence: lengths that change during the call find no end otherwise)
        for (uint32_t s = who * per; s < min(a.tok.n_seqs, (who + 1) * per); ++s) {
            const int64_t steps = seq_cost<kFlat>(f, kv_seq(a.pages, a.tok, s), s, lane);
            if (run0 < p + steps * K) {
                if (kFlat || lane == 0) sh.start_seq = int32_t(s), sh.start_rest = run0 - p, sh.start_steps = steps;
                break;
            }
            p += steps * K;
        }
    }
    __syncthreads();
    const uint32_t tmem = sh.tmem;
    if (busy && sh.start_seq < 0) {
        busy = false;
        if (tid == 0) sh.dead = 1;
    }

    if (busy && warp >= kSumWarps) {
        if (Sh::kGroups == 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Sh::kOtherRegs));
        if (warp == kSumWarps || (kFlat && warp == kSumWarps + 3)) {
        // ---------------------------------------------------------- loads
        // A warp a half: both walk the run, the first hands units out and loads queries. (One warp for both halves issued a
        // load of 2 KiB, as pages of 16 tokens have them, every 66 ns: a token each of 64 sequences of up to 16k slots 243
        // us, with two 179.) Where keys stay for many column tiles one warp loads both.
        const uint32_t half0 = warp == kSumWarps ? 0 : 1;
        constexpr uint32_t kLoads = kFlat ? 1 : 2;
        int32_t s = sh.start_seq, h = int32_t(sh.start_rest / sh.start_steps), i = 0;  // sequence, key head, unit
        int64_t at = run0, unit;  // the segment's first place, the unit's
        KvSeq q = kv_seq(a.pages, a.tok, s);
        UnitList list = unit_list(f, q);
        {
            int64_t rest = sh.start_rest % sh.start_steps;
            if (kFlat) {
                i = int32_t(rest), rest = 0;
            } else {
                for (;; i += 32) {  // the warp looks at 32 units at a time
                    const int32_t mine = i + int32_t(lane) < list.n ? unit_cost(unit_tiles(f, q, s, unit_slot(list, i + int32_t(lane)))) : 0;
                    int64_t inc = mine;
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) {
                        const int64_t o = __shfl_up_sync(0xFFFFFFFFu, inc, d);
                        if (lane >= uint32_t(d)) inc += o;
                    }
                    const uint32_t found = __ballot_sync(0xFFFFFFFFu, rest < inc);
                    if (found) {
                        const int l = __ffs(found) - 1;
                        rest -= __shfl_sync(0xFFFFFFFFu, inc - mine, l);
                        i += l;
                        break;
                    }
                    rest -= __shfl_sync(0xFFFFFFFFu, inc, 31);
                    if (i + 32 >= list.n) break;  // (never: the costs add up)
                }
            }
            unit = at - rest;
        }
        const uint32_t shift = a.pages.token_shift;
        const uint32_t box = shift < 7 ? 1u << shift : 128u, boxes = 128u / box;
        const uint32_t T_mask = (1u << shift) - 1;
        const uint32_t q_bytes = uint32_t(f.per_tile * f.per_token) * 128 * NS;
        uint32_t u = 0, kn = 0, qn = 0;
        // A segment's pages, a lane a box: looked up while the segment before is loaded.
        int32_t page[kLoads], ahead[kLoads];
        auto pages_at = [&]() {
            const int32_t* table = a.pages.table + uint32_t(s) * a.pages.table_stride;
#pragma unroll
            for (uint32_t k = 0; k < kLoads; ++k) {
                const uint32_t slot = uint32_t(unit_slot(list, i)) + (half0 + k) * 128 + lane * box;
                ahead[k] = lane < boxes && slot < uint32_t(q.len) ? table[slot >> shift] : -1;
            }
        };
        pages_at();
        for (bool more = !f.no_loads; more; ++u) {
            // the segment
            const int32_t slot0 = unit_slot(list, i);
            const int2 tiles = unit_tiles(f, q, s, slot0);
            const bool dry = tiles.y <= tiles.x;
            const int32_t steps = max(1, tiles.y - tiles.x);
            const int64_t unit0 = unit + (kFlat || dry ? 0 : kUnitCost);  // its first step
            if (at < unit0) at = unit0;
            const int32_t skip = kFlat ? 0 : int32_t(at - unit0);
            // (0: a run of nothing but a unit's cost)
            const int32_t n = kFlat ? steps : int32_t(max(int64_t(0), min(int64_t(steps - skip), run1 - at)));
            const int32_t first = q.first, head0 = h * int32_t(a.group);
            const int32_t row = int32_t((a.pages.layer * 2 * a.pages.kv_heads + h) << shift);
            at = kFlat ? unit + 1 : unit0 + steps;  // the next unit's place
            more = at < run1;
#pragma unroll
            for (uint32_t k = 0; k < kLoads; ++k) page[k] = ahead[k];
            if (half0 == 0 && !mbar_wait(bar(sh.unit_empty[u % kWeighUnits]), (u / kWeighUnits & 1) ^ 1, dead)) break;
            if (half0 == 0 && lane == 0) {
                WeighUnit& o = sh.unit[u % kWeighUnits];
                o.q = q, o.s = s, o.h = h, o.slot0 = slot0;
                o.tile = tiles.x + skip, o.n = n, o.dry = dry, o.whole = n == steps, o.part = u ? 1 : 0, o.more = more;
                mbar_arrive(bar(sh.unit_full[u % kWeighUnits]));
                if (!kFlat && u == 0) {
                    // this run's note of a unit that began in the run before it
                    const int64_t b0 = ((unit0 + 1) * blocks - 1) / total, b1 = ((unit0 + steps) * blocks - 1) / total;
                    const bool here = skip > 0 && b0 + 1 == int64_t(blockIdx.x);
                    f.join[blockIdx.x] = {s, h, slot0, q.len - q.n, q.len, int32_t(b0), int32_t(b1), b0 * total / blocks < unit, here};
                }
            }
            __syncwarp();
            if (more) {  // the next unit (the segment ended with this one)
                unit = at;
                if (++i >= list.n) {
                    i = 0;
                    if (++h == int32_t(K)) {
                        h = 0;
                        do {
                            if (++s >= int32_t(a.tok.n_seqs)) {
                                *dead = 1;
                                goto loads_done;
                            }
                            q = kv_seq(a.pages, a.tok, s);
                            list = unit_list(f, q);
                        } while (list.n == 0);
                    }
                }
                pages_at();
            }
            if (!dry && n) {
#pragma unroll
                for (uint32_t k = 0; k < kLoads; ++k) {
                    const uint32_t slot = uint32_t(slot0) + (half0 + k) * 128 + lane * box, e = Sh::entry(half0 + k, kn);
                    // what the pool lacks, and what lies behind the sequence, is filled with zeros
                    const int32_t z = uint32_t(page[k]) >= a.pages.total_pages ? int32_t(a.pages.total_pages) : page[k];
                    if (!mbar_wait(bar(sh.k_empty[e]), Sh::phase(half0 + k, kn) ^ 1, dead)) goto loads_done;
                    if (lane == 0) mbar_expect(bar(sh.k_full[e]), Sh::kHalf);
                    __syncwarp();
                    if (lane < boxes)
                        for (int x = 0; x < NS; ++x)
                            tma_load(ring + e * Sh::kHalf + x * kHalfSlot + lane * box * 128, &map, x * 64, row + int32_t(slot & T_mask), z,
                                     bar(sh.k_full[e]));
                }
                ++kn;
                if (half0) continue;
                for (int32_t t = tiles.x + skip; t < tiles.x + skip + n; ++t, ++qn) {
                    const uint32_t e = qn % Sh::kQs;
                    if (!mbar_wait(bar(sh.q_empty[e]), (qn / Sh::kQs & 1) ^ 1, dead)) goto loads_done;
                    if (lane == 0) {
                        mbar_expect(bar(sh.q_full[e]), q_bytes);
                        const int32_t token = first + t / f.slices * f.per_tile, head = head0 + t % f.slices * f.per_token;
                        for (int x = 0; x < NS; ++x)
                            tma_load(qs + e * Sh::kQ + x * (N * 128), &q_map, x * 64, head, token, bar(sh.q_full[e]));
                    }
                    __syncwarp();
                }
            }
        }
    loads_done:
        __syncwarp();
        if (*dead) {  // the copies in flight land before the block ends
            uint32_t late = 0;
            for (uint32_t h = half0; h < half0 + kLoads; ++h) {
                const uint32_t ring_of = h ? Sh::kKeys1 : Sh::kKeys0;
                for (uint32_t k = kn > ring_of ? kn - ring_of : 0; k <= kn; ++k)  // (the last may not have been issued: a second's wait)
                    mbar_wait(bar(sh.k_full[Sh::entry(h, k)]), Sh::phase(h, k), &late);
            }
            for (uint32_t k = qn > Sh::kQs ? qn - Sh::kQs : 0; k < qn; ++k) mbar_wait(bar(sh.q_full[k % Sh::kQs]), k / Sh::kQs & 1, &late);
        }
    } else if (warp <= kSumWarps + 2) {
        // ---------------------------------------------------------- products
        const uint32_t half = warp - (kSumWarps + 1);
        constexpr uint32_t kQk = instr_desc(kBf16, false, false, 128, N);
        const uint32_t ksteps = (a.pages.head_dim + 15) / 16;
        // keys and queries: rows of 64 elements, 128-byte swizzle
        const uint64_t kd = smem_desc(ring, 16, 1024, 2), qd = smem_desc(qs, 16, 1024, 2);
        // (One lane issues them all: what stands between two products is short.)
        bool more = lane == 0, ok = true;
        // (Where two groups of warps take turns, each has one of the two places for scores, whatever tiles a unit begins and
        // ends with: a wait names one of two phases, so nobody may wait at a place whose other phase is another's.)
        uint32_t kn = 0, qn = 0, n = 0, taken[2] = {0, 0};
        auto products = [&](uint64_t k0, uint64_t q0, uint32_t to, auto all) {
#pragma unroll
            for (uint32_t x = 0; x < 4 * NS; ++x) {
                if (!decltype(all)::value && x >= ksteps) break;
                mma_ss(to, desc_at(k0, (x / 4) * kHalfSlot + (x % 4) * 32), desc_at(q0, (x / 4) * (N * 128) + (x % 4) * 32), kQk, x != 0);
            }
        };
        for (uint32_t u = 0; more && ok; ++u) {
            if (!mbar_wait(bar(sh.unit_full[u % kWeighUnits]), u / kWeighUnits & 1, dead)) break;
            const WeighUnit& o = sh.unit[u % kWeighUnits];
            const int32_t steps = o.dry ? 0 : o.n, tile0 = o.tile;
            more = o.more;
            mbar_arrive(bar(sh.unit_empty[u % kWeighUnits]));
            if (!steps) continue;
            const uint32_t ek = Sh::entry(half, kn);
            ok = mbar_wait(bar(sh.k_full[ek]), Sh::phase(half, kn), dead);
            const uint64_t k0 = desc_at(kd, ek * Sh::kHalf);
            for (int32_t i = 0; i < steps && ok; ++i, ++n, ++qn) {
                const uint32_t turn = HOW == Tiles::kOne ? u & 1 : uint32_t(tile0 + i) & 1;
                const uint32_t eq = qn % Sh::kQs, buf = Sh::kGroups == 4 ? turn : n % Sh::kBufs;
                const uint32_t phase = Sh::kGroups == 4 ? (turn ? taken[1] : taken[0]) & 1 : n / Sh::kBufs & 1;
                if (turn) ++taken[1];
                else ++taken[0];
                ok = mbar_wait(bar(sh.s_empty[half][buf]), phase ^ 1, dead) &&
                     mbar_wait(bar(sh.q_full[eq]), qn / Sh::kQs & 1, dead);
                if (!ok) break;
                fence_after();
                const uint64_t q0 = desc_at(qd, eq * Sh::kQ);
                const uint32_t to = tmem + (half * Sh::kBufs + buf) * N;
                if (ksteps == 4 * NS)
                    products(k0, q0, to, std::true_type());
                else
                    products(k0, q0, to, std::false_type());
                mma_commit(bar(sh.s_full[half][buf]));
                mma_commit(bar(sh.q_empty[eq]));
            }
            if (ok) mma_commit(bar(sh.k_empty[ek]));
            ++kn;
        }
        __syncwarp();
        if (*dead) {  // the products in flight end before the tensor memory is freed
            const uint64_t t0 = now_ns();
            while (now_ns() - t0 < 50000) {
            }
        }
    }
    } else if (busy) {
        // ---------------------------------------------------------- weights
        if (Sh::kGroups == 4) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Sh::kSumRegs));
        const int half = warp / 4 % 2, side = warp / 8;  // which 128 keys, and which tiles: the even or the odd ones
        constexpr bool kTurns = Sh::kGroups == 4, kTileTurns = kTurns && HOW != Tiles::kOne, kUnitTurns = kTurns && HOW == Tiles::kOne;
        constexpr int kStep = kTileTurns ? 2 : 1;
        const uint32_t key = tid % 128;
        const uint32_t lanes = tmem + ((warp % 4) << 21) + half * Sh::kBufs * N;
        const float k2 = a.scale * kLog2e;
        const bool cap = MOD && a.softcap != 0.0f;
        const float cap_in = cap ? a.scale / a.softcap : 0.0f, cap2 = a.softcap * kLog2e;
        const uint64_t k22 = pack2(k2, k2);
        // the lane's columns of a tile: token and head, counted in the tile
        constexpr int kMine = kCols < 32 ? 1 : kCols / 32;
        uint32_t place_of[kMine];  // token, and the head above it
        float next[kMine];         // their log-sum-exps of the next tile
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const uint32_t c = k * 32 + lane, t = c / uint32_t(f.per_token);
            place_of[k] = k * 32 + int32_t(lane) >= kCols ? 0xFFFFu : t | (c - t * uint32_t(f.per_token)) << 16;  // (0xFFFF: none)
        }
        auto token_at = [&](int k) { return int32_t(place_of[k] & 0xFFFFu); };
        auto head_at = [&](int k) { return int32_t(place_of[k] >> 16); };
        // the first token and query of a column tile
        auto tile_at = [&](int32_t tile) {
            if (f.slices == 1) return make_int2(tile * f.per_tile, 0);
            const int32_t t = tile / f.slices;
            return make_int2(t * f.per_tile, (tile - t * f.slices) * f.per_token);
        };
        constexpr bool kLean = !kFlat && !MOD;
        const bool lean = f.slices == 1 && !a.spans;
        // Columns of no query have queries of zeros: 0 for a finite key, and no number for one that is not, whose scores then
        // are not finite in any column (of a query that is). So the first score of some columns says whether those of no
        // query have to be left out, and what a finite key costs is one comparison: prompts of 8,190 tokens 244 us (242
        // without), of seven heads to a key head 211 (209). With a mask wherever there are such columns 250 and 232.
        auto odd = [](float score) { return __builtin_expect(!(fabsf(score) < INFINITY), 0); };
        auto below = [](int32_t n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; };  // the first n of 32 columns
        // of the tile that begins with token t0 and the head's query g0 (first: the sequence's first token)
        auto look_up = [&](int32_t first, int32_t h, int32_t m, int32_t t0, int32_t g0) {
            const float* const at = f.w.lse + uint64_t(uint32_t(first + t0)) * a.q_heads + h * a.group + g0;
#pragma unroll
            for (int k = 0; k < kMine; ++k) {
                const bool real = token_at(k) < min(f.per_tile, m - t0) && head_at(k) < int32_t(a.group) - g0;
                next[k] = at[real ? uint32_t(token_at(k)) * a.q_heads + uint32_t(head_at(k)) : 0];  // (a tile has a first column)
                if (!real) next[k] = -INFINITY;
            }
        };
        // the weight so far of the thread's slot of a unit
        auto weight_so_far = [&](const WeighUnit& o) {
            const int32_t slot = o.slot0 + half * 128 + int32_t(key);
            const bool old = slot < o.q.len - o.q.n && uint32_t(slot) < f.w.n_slots && f.w.decay != 0.0f;
            return old ? f.w.weights[uint32_t(o.s) * f.w.seq_stride + uint32_t(o.h) * f.w.head_stride + slot] : 0.0f;
        };
        float then = 0.0f;  // ... of the next unit
        bool then_known = false;
        // ... and what was looked up to its place, with slopes
        auto put = [&](int32_t h, int32_t m, int32_t t0, int32_t g0) {
#pragma unroll
            for (int k = 0; k < kMine; ++k) {
                const int32_t c = k * 32 + int32_t(lane);
                if (kCols < 32 && c >= kCols) break;
                lse_of[warp][c] = next[k] == -INFINITY ? -INFINITY : -next[k] * kLog2e;
                if (MOD) {
                    const bool real = token_at(k) < min(f.per_tile, m - t0) && head_at(k) < int32_t(a.group) - g0;
                    slope_of[MOD ? warp : 0][c] = a.slopes && real ? a.slopes[h * a.group + g0 + head_at(k)] * kLog2e : 0.0f;
                }
            }
        };
        // spans of kSpanCols columns from c0 on
        auto put_spans = [&](int c0, int32_t first, int32_t m, int32_t t0, int32_t g0) {
            __syncwarp();
            for (int c = int(lane); c < Sh::kSpanCols; c += 32) {
                const int32_t t = (c0 + c) / f.per_token, g = (c0 + c) % f.per_token;
                int2 span = make_int2(0, 0);
                if (t < min(f.per_tile, m - t0) && g < int32_t(a.group) - g0) span = reinterpret_cast<const int2*>(a.spans)[first + t0 + t];
                span_of[warp][c] = span;
            }
            __syncwarp();
        };
        int32_t had_s = -1, had_h = -1;  // whose log-sum-exps are there (kFlat)
        bool known = false;              // `next` is the next tile's
        uint32_t n = 0;  // the group's tiles
        bool more = true;
        for (uint32_t u = 0; more; ++u) {
            const bool got = mbar_wait(bar(sh.unit_full[u % kWeighUnits]), u / kWeighUnits & 1, dead);
            if (!__all_sync(0xFFFFFFFFu, got)) break;
            const WeighUnit& rec = sh.unit[u % kWeighUnits];
            const int32_t s = rec.s, h = rec.h, len = rec.q.len, ctx = len - rec.q.n, first = rec.q.first, m = weigh_tokens(a, rec.q);
            const int32_t slot = rec.slot0 + half * 128 + int32_t(key), steps = rec.dry ? 0 : rec.n;
            const bool dry = rec.dry, whole = rec.whole, none = rec.n == 0;
            const int32_t in_part = rec.part, tile0 = rec.tile;
            more = rec.more;
            if (none) break;
            const bool turn = !kUnitTurns || int(u & 1) == side;  // this group's unit
            const bool mine = (kUnitTurns ? turn : side == 0) && slot < len && uint32_t(slot) < f.w.n_slots;
            float* const place = f.w.weights + uint32_t(s) * f.w.seq_stride + uint32_t(h) * f.w.head_stride + slot;
            float held = then;
            if (!kFlat && whole && mine && slot < ctx && f.w.decay != 0.0f) held = *place;
            if (kFlat) {  // the next unit's, on their way while this one is worked on
                if (!then_known) held = weight_so_far(rec);
                then_known = false;
                if (more) {
                    const uint32_t v = u + 1;
                    const bool out = mbar_test(bar(sh.unit_full[v % kWeighUnits]), v / kWeighUnits & 1);
                    if (__all_sync(0xFFFFFFFFu, out)) then = weight_so_far(sh.unit[v % kWeighUnits]), then_known = true;
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sh.unit_empty[u % kWeighUnits]));
            // the tokens [i0, i1) that see the slot, and those that see all of the warp's slots
            int32_t i0 = max(0, slot - ctx), i1 = m;
            if (a.window && slot >= int32_t(a.sinks)) i1 = int32_t(min(int64_t(m), int64_t(slot) + int64_t(a.window) - ctx));
            const int32_t all0 = __reduce_max_sync(0xFFFFFFFFu, i0), all1 = a.spans ? 0 : __reduce_min_sync(0xFFFFFFFFu, i1);
            if (slot >= len) i1 = 0;  // (what lies behind the sequence is not written, so it may be added up)
            KvSum sum;
            for (int32_t i = kTileTurns ? (tile0 ^ side) & 1 : 0; i < steps && turn; i += kStep) {
                int2 at0 = tile_at(tile0 + i);
                // (which way a tile goes does not depend on whether its log-sum-exps came early: sums are added up in one order)
                if (!kFlat && !known) look_up(first, h, m, at0.x, at0.y), known = true;
                if (kLean && lean && at0.x >= all0) {
                    // Tiles that all of the warp's slots see, and the group's next of which is complete: nothing to decide.
                    const uint64_t stride = uint64_t(uint32_t(f.per_tile)) * (a.q_heads * kStep);
                    const float* at = f.w.lse + uint64_t(uint32_t(first + at0.x)) * a.q_heads + h * a.group;
                    uint32_t offset[kMine];
#pragma unroll
                    for (int k = 0; k < kMine; ++k)
                        offset[k] = token_at(k) >= f.per_tile ? 0xFFFFFFFFu : uint32_t(token_at(k)) * a.q_heads + uint32_t(head_at(k));
#pragma unroll 1
                    for (; i + kStep < steps && at0.x + (kStep + 1) * f.per_tile <= all1; i += kStep, at0.x += kStep * f.per_tile) {
                        __syncwarp();
#pragma unroll
                        for (int k = 0; k < kMine; ++k) lse_of[warp][k * 32 + lane] = next[k] == -INFINITY ? -INFINITY : -next[k] * kLog2e;
                        __syncwarp();
                        at += stride;
#pragma unroll
                        for (int k = 0; k < kMine; ++k) next[k] = offset[k] == 0xFFFFFFFFu ? -INFINITY : at[offset[k]];
                        const uint32_t buf = uint32_t(side);  // (kTileTurns)
                        const bool there = mbar_wait(bar(sh.s_full[half][buf]), n++ & 1, dead);
                        if (!__all_sync(0xFFFFFFFFu, there)) goto weights_done;
                        fence_after();
                        uint64_t add0 = 0, add1 = 0;
#pragma unroll 1
                        for (int c0 = 0; c0 < kCols; c0 += 64) {
                            float x[64];
#pragma unroll
                            for (int c = 0; c < 64; c += 32) tmem_ld32(lanes + buf * N + c0 + c, x + c);
                            wait_ld(x);
                            if (c0 + 64 >= kCols) {
                                fence_before();
                                __syncwarp();
                                if (lane == 0) mbar_arrive(bar(sh.s_empty[half][buf]));
                            }
                            if (odd(x[0])) {
                                const int32_t n = f.per_tile * f.per_token - c0;
#pragma unroll
                                for (int c = 0; c < 64; ++c) x[c] = below(n - c / 32 * 32) & (1u << c % 32) ? x[c] : 0.0f;
                            }
#pragma unroll
                            for (int c = 0; c < 64; c += 4) {
                                const ulonglong2 l = *reinterpret_cast<const ulonglong2*>(lse_of[warp] + c0 + c);
                                float y0, y1, y2, y3;
                                unpack2(fma2(pack2(x[c], x[c + 1]), k22, l.x), y0, y1);
                                unpack2(fma2(pack2(x[c + 2], x[c + 3]), k22, l.y), y2, y3);
                                add0 = add2(add0, pack2(exp2_approx(y0), exp2_approx(y1)));
                                add1 = add2(add1, pack2(exp2_approx(y2), exp2_approx(y3)));
                            }
                        }
                        float y0, y1;
                        unpack2(add2(add0, add1), y0, y1);
                        sum.add(y0 + y1);
                    }
                }
                const int32_t t0 = at0.x, g0 = at0.y;
                if (!kFlat || kTileTurns || s != had_s || h != had_h) {
                    if (kFlat) {
                        // (a group's tile of a key head is the same for all its units)
                        if (s != had_s || h != had_h) look_up(first, h, m, t0, g0), had_s = s, had_h = h, known = true;
                    }
                    if (known) {
                        known = false;
                        __syncwarp();
                        put(h, m, t0, g0);
                        __syncwarp();
                    }
                }
                const float ahead = float(ctx + t0 - slot);
                const bool plain = t0 >= all0 && t0 + f.per_tile <= all1 && g0 + f.per_token <= int32_t(a.group);
                // the thread's visible columns [v0, v1), where not all are
                int32_t v0 = 0, v1 = f.per_tile * f.per_token;
                if (!plain) {
                    const int32_t cols = min(f.per_tile, m - t0) * min(f.per_token, int32_t(a.group) - g0);
                    v0 = a.spans ? 0 : min(max(i0 - t0, 0), f.per_tile) * f.per_token;
                    v1 = slot >= len ? 0 : a.spans ? cols : min(min(max(i1 - t0, 0), f.per_tile) * f.per_token, cols);
                }
                if (!kFlat) {  // the group's next tile's, on their way while this one is worked on
                    if (i + kStep < steps) {
                        const int2 b = tile_at(tile0 + i + kStep);
                        look_up(first, h, m, b.x, b.y), known = true;
                    } else if (more) {
                        const uint32_t v = u + 1;
                        const WeighUnit& o = sh.unit[v % kWeighUnits];
                        const bool out = mbar_test(bar(sh.unit_full[v % kWeighUnits]), v / kWeighUnits & 1);
                        if (__all_sync(0xFFFFFFFFu, out)) {
                            const int32_t j = (o.tile ^ side) & 1;
                            const int2 b = tile_at(o.tile + j);
                            if (!o.dry && j < o.n) look_up(o.q.first, o.h, weigh_tokens(a, o.q), b.x, b.y), known = true;
                        }
                    }
                }
                float part[4] = {};
                const uint32_t buf = kTurns ? uint32_t(side) : n % Sh::kBufs;
                const bool there = mbar_wait(bar(sh.s_full[half][buf]), kTurns ? n & 1 : n / Sh::kBufs & 1, dead);
                ++n;
                if (!__all_sync(0xFFFFFFFFu, there)) goto weights_done;
                fence_after();
#pragma unroll 1
                for (int c0 = 0; c0 < kCols; c0 += kChunk) {
                    float x[kChunk];
                    if constexpr (kChunk == 16)
                        tmem_get16(lanes + buf * N + c0, x);
                    else
                        tmem_get32(lanes + buf * N + c0, x);
                    if (c0 + kChunk == kCols) {  // the scores are read: their columns may be written again
                        fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(sh.s_empty[half][buf]));
                    }
                    const bool some = !plain || odd(x[0]);
                    // scores, less the log-sum-exp, in units of log2
#pragma unroll
                    for (int c = 0; c < kChunk; c += 4) {
                        const float4 l = *reinterpret_cast<const float4*>(lse_of[warp] + c0 + c);
                        if (MOD) {
                            const float4 sl = *reinterpret_cast<const float4*>(slope_of[MOD ? warp : 0] + c0 + c);
                            const float4 tk = *reinterpret_cast<const float4*>(token_of + (MOD ? c0 + c : 0));
                            const float sls[4] = {sl.x, sl.y, sl.z, sl.w}, ls[4] = {l.x, l.y, l.z, l.w}, tks[4] = {tk.x, tk.y, tk.z, tk.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                float z = cap ? capped<true>(x[c + k], cap_in, cap2) : x[c + k] * k2;
                                z -= sls[k] * fabsf(ahead + tks[k]);
                                x[c + k] = z + ls[k];
                            }
                        } else {
                            x[c] = fmaf(x[c], k2, l.x), x[c + 1] = fmaf(x[c + 1], k2, l.y);
                            x[c + 2] = fmaf(x[c + 2], k2, l.z), x[c + 3] = fmaf(x[c + 3], k2, l.w);
                        }
                    }
                    if (some) {
                        uint32_t see = 0;
                        if (a.spans) {
                            if (c0 % Sh::kSpanCols == 0) put_spans(c0, first, m, t0, g0);
#pragma unroll 4
                            for (int c = 0; c < kChunk; ++c) {
                                const int2 sp = span_of[warp][c0 % Sh::kSpanCols + c];
                                see |= uint32_t(slot >= sp.x && slot < sp.y && c0 + c < v1) << c;
                            }
                        } else {
                            see = below(v1 - c0) & ~below(v0 - c0);
                        }
#pragma unroll
                        for (int c = 0; c < kChunk; ++c) x[c] = see & (1u << c) ? x[c] : -INFINITY;
                    }
#pragma unroll
                    for (int c = 0; c < kChunk; c += 4) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) part[k] += exp2_approx(x[c + k]);
                    }
                }
                sum.add((part[0] + part[1]) + (part[2] + part[3]));
            }
            float got_all = sum.value();
            if (kUnitTurns && !turn) continue;
            if (kTileTurns) {  // the sums of the even and the odd tiles meet
                const uint32_t b = u & 1;
                float* const other = sh.sum[half][b];
                if (side) {
                    const bool there = mbar_wait(bar(sh.sum_empty[half][b]), (u >> 1 & 1) ^ 1, dead);
                    if (!__all_sync(0xFFFFFFFFu, there)) goto weights_done;
                    other[key] = got_all;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(sh.sum_full[half][b]));
                    continue;
                }
                const bool there = mbar_wait(bar(sh.sum_full[half][b]), u >> 1 & 1, dead);
                if (!__all_sync(0xFFFFFFFFu, there)) goto weights_done;
                got_all += other[key];
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(sh.sum_empty[half][b]));
            }
            if (!whole)
                __stcg(f.part + (uint64_t(blockIdx.x) * 2 + in_part) * kPartFloats + half * 128 + key, got_all);
            else if (mine && !(dry && f.w.decay == 1.0f && slot < ctx))
                *place = got_all + (slot < ctx && f.w.decay != 0.0f ? f.w.decay * held : 0.0f);
        }
    weights_done:;
    }
    __syncthreads();
    if (tid == 0 && *dead) *f.fault = 1;
    if (warp == kSumWarps + 1) {
        fence_after();
        tmem_free(tmem, Sh::kTmem);
    }
}

// Joins the units that lie in several runs: a block for each run's note, a thread a slot.
__global__ void __launch_bounds__(kUnitKeys) weigh_join_kernel(const __grid_constant__ Weigh f) {
    pdl_launch();
    pdl_wait();
    const WeighJoin j = f.join[blockIdx.x];
    if (!j.valid) return;
    const int32_t slot = j.slot0 + int32_t(threadIdx.x);
    if (slot >= j.len || uint32_t(slot) >= f.w.n_slots) return;
    KvSum sum;
    for (int32_t b = j.b0; b <= j.b1; ++b)
        sum.add(__ldcg(f.part + (uint64_t(b) * 2 + (b == j.b0 && j.second ? 1 : 0)) * kPartFloats + threadIdx.x));
    float* const place = f.w.weights + uint32_t(j.s) * f.w.seq_stride + uint32_t(j.h) * f.w.head_stride + slot;
    *place = sum.value() + (slot < j.ctx && f.w.decay != 0.0f ? f.w.decay * *place : 0.0f);
}

constexpr uint64_t weigh_up(uint64_t n) { return (n + 255) / 256 * 256; }
// the workspace's parts, in order: notes, parts, hulls
uint64_t weigh_hulls(uint64_t n_seqs, uint64_t n_tokens, uint64_t per_tile) { return n_tokens / per_tile + n_seqs + 1; }

template <class T, int N, int NS, bool MOD, Tiles HOW>
cudaError_t launch_weigh_as(const Weigh& f, const CUtensorMap& map, const CUtensorMap& q_map, uint32_t sms, cudaStream_t stream) {
    constexpr uint32_t bytes = WeighShape<N, NS, HOW>::kBytes;
    static std::atomic<uint64_t> ready{0};  // devices whose kernel may take this much shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !(ready.load() >> dev & 1)) {
        e = cudaFuncSetAttribute(weigh_kernel<T, N, NS, MOD, HOW>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(bytes));
        if (e != cudaSuccess) return e;
        if (dev < 64) ready |= uint64_t(1) << dev;
    }
    const KvAttend& a = f.w.a;
    if (a.spans && (e = launch_pdl(hull_kernel, dim3(a.tok.n_seqs), 128, 0, stream, f)) != cudaSuccess) return e;
    // no more blocks than there may be steps, going by max_len
    const uint64_t tiles = HOW == Tiles::kMany ? (uint64_t(a.tok.max_new) / f.per_tile + 1) * f.slices : 1;
    const uint64_t steps = uint64_t(a.tok.n_seqs) * a.pages.kv_heads * (uint64_t(a.max_len) / kUnitKeys + 1);
    const uint32_t blocks = uint32_t(steps > sms / tiles ? sms : steps * tiles);
    if ((e = launch_pdl(weigh_kernel<T, N, NS, MOD, HOW>, dim3(blocks), WeighShape<N, NS, HOW>::kThreads, bytes, stream, f, map, q_map)) != cudaSuccess) return e;
    return HOW == Tiles::kMany ? launch_pdl(weigh_join_kernel, dim3(blocks), kUnitKeys, 0, stream, f) : cudaSuccess;
}

template <class T, int N, int NS, Tiles HOW>
cudaError_t launch_weigh_mod(const Weigh& f, const CUtensorMap& map, const CUtensorMap& q_map, uint32_t sms, cudaStream_t stream) {
    return f.w.a.softcap != 0.0f || f.w.a.slopes ? launch_weigh_as<T, N, NS, true, HOW>(f, map, q_map, sms, stream)
                                                 : launch_weigh_as<T, N, NS, false, HOW>(f, map, q_map, sms, stream);
}

template <class T, int N, Tiles HOW>
cudaError_t launch_weigh_n(const Weigh& f, const KvLaunch& l, cudaStream_t stream) {
    const KvAttend& a = f.w.a;
    CUtensorMap q_map;
    // the queries as [tokens][heads][head_dim]: a column tile's in one box (64 elements at a time)
    const cudaError_t e = l.encode_queries(a, f.per_token, f.per_tile, &q_map);
    if (e != cudaSuccess) return e;
    return a.pages.head_dim <= 64 ? launch_weigh_mod<T, N, 1, HOW>(f, *l.map, q_map, l.sms, stream)
                                  : launch_weigh_mod<T, N, 2, HOW>(f, *l.map, q_map, l.sms, stream);
}

template <class T>
cudaError_t launch_weigh(const KvWeigh& w, const KvLaunch& l, cudaStream_t stream) {
    Weigh f{};
    f.w = w;
    f.skips = w.decay == 1.0f && !w.a.spans;
    uint8_t* p = static_cast<uint8_t*>(l.workspace);
    f.join = reinterpret_cast<WeighJoin*>(p);
    p += weigh_up(l.sms * sizeof(WeighJoin));
    f.part = reinterpret_cast<float*>(p);
    p += weigh_up(uint64_t(l.sms) * 2 * kPartFloats * sizeof(float));
    f.hulls = reinterpret_cast<int2*>(p);
    f.fault = l.fault;
    f.no_loads = l.no_loads;
    // tiles of at most 128 columns, of whole tokens (or of a share of a token's heads), equally many
    const uint32_t most = w.a.tok.max_new, columns = std::min<uint32_t>(w.a.group, 128), tokens = 128 / columns;
    f.per_token = int32_t(columns);
    f.slices = int32_t((w.a.group + columns - 1) / columns);
    const uint32_t tiles = (most + tokens - 1) / tokens;
    f.per_tile = int32_t((most + tiles - 1) / tiles);
    if (uint64_t(tiles) * f.slices == 1) {
        const uint32_t rows = columns * most;
        if (rows <= 16) return launch_weigh_n<T, 16, Tiles::kOne>(f, l, stream);
        if (rows <= 32) return launch_weigh_n<T, 32, Tiles::kOne>(f, l, stream);
        if (rows <= 64) return launch_weigh_n<T, 64, Tiles::kOne>(f, l, stream);
        return launch_weigh_n<T, 128, Tiles::kOne>(f, l, stream);
    }
    // Two: 32 tokens of nine prompts of up to 7k slots 22 us, as if there were many 33; of one of 3k 10 against 15. (Three
    // are slower so, 81 against 74 us, but over short contexts.) Spans go with many.
    if (uint64_t(tiles) * f.slices == 2 && !w.a.spans) return launch_weigh_n<T, 128, Tiles::kFew>(f, l, stream);
    return launch_weigh_n<T, 128, Tiles::kMany>(f, l, stream);
}

}  // namespace
}  // namespace t2i
