// What the attention kernels over the cache share: which slots a sequence's new
// tokens see, and the scores.
#pragma once

#include <type_traits>

#include "kv_device.cuh"
#include "tc.cuh"

namespace t2i {

constexpr int kTileKeys = 128;       // keys of a tile
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// A softmax's reference is so many powers of two below the maximum that it goes by. Weights go to the product in
// 16 bits, and fp16 keeps nothing below 2^-25: without a lift, 131,072 keys at 2^-26 of the largest, 0.2% of the sum,
// were no part of the output. With 2^7 a weight is off by 2^-32 of the largest at most (and by its own rounding),
// and the largest stay below fp16's end (2^15 in kv_few.cuh, kFarOf in kv_rows.cuh). bf16 has fp32's exponents.
template <class T>
constexpr float kLift = 0.0f;
template <>
constexpr float kLift<__half> = 7.0f;

// Slots [lo, hi) outside which none of tokens [t0, t1) of sequence q sees anything,
// and slots [all_lo, all_hi) that all of them see.
struct KvSpan {
    int32_t lo, hi, all_lo, all_hi;
};
__device__ __forceinline__ KvSpan kv_span(const KvAttend& a, const KvSeq& q, int32_t t0, int32_t t1) {
    const int32_t ctx = q.len - q.n;
    KvSpan r;
    if (a.spans) {
        r = {INT32_MAX, 0, 0, INT32_MAX};
        for (int32_t i = t0; i < t1; ++i) {
            const int2 s = reinterpret_cast<const int2*>(a.spans)[q.first + i];
            const int32_t f = max(s.x, 0), l = min(s.y, q.len);
            if (l > f) r.lo = min(r.lo, f), r.hi = max(r.hi, l);
            r.all_lo = max(r.all_lo, f), r.all_hi = min(r.all_hi, l);
        }
        if (r.lo >= r.hi) r.lo = r.hi = 0;
        return r;
    }
    const int64_t w = a.window ? int64_t(a.window) : int64_t(INT32_MAX);
    if (a.tree) {
        // positions lie between ctx - 1 (a word without bits) and ctx + n - 1
        r.lo = int32_t(max(int64_t(0), ctx - w));
        r.hi = q.len;
        r.all_lo = a.window ? int32_t(max(int64_t(0), ctx + q.n - w)) : 0;
        r.all_hi = ctx;
        return r;
    }
    r.lo = int32_t(max(int64_t(0), ctx + t0 + 1 - w));
    r.hi = ctx + t1;
    r.all_lo = int32_t(max(int64_t(0), ctx + t1 - w));
    r.all_hi = ctx + t0 + 1;
    return r;
}

// The word of drafted token i of a sequence: bits behind its tokens (a caller's word
// of ones) count nothing.
__device__ __forceinline__ uint64_t kv_word(const KvAttend& a, const KvSeq& q, int32_t i) {
    const uint64_t w = a.tree[q.first + i];
    return q.n < 64 ? w & ((uint64_t(1) << q.n) - 1) : w;
}

// One query: it sees the keys of slots below `last`, and of the drafted tokens in
// `word`, whose position is `first` or above. pos: its own position.
struct KvQuery {
    int32_t first, last, pos;
    uint64_t word;
};
__device__ __forceinline__ KvQuery kv_query(const KvAttend& a, const KvSeq& q, int32_t i) {
    const int32_t ctx = q.len - q.n, t = q.first + i;
    KvQuery r;
    r.word = 0;
    r.pos = ctx + i;
    r.last = r.pos + 1;
    if (a.tree) {
        r.word = kv_word(a, q, i);
        r.pos = ctx + __popcll(r.word) - 1;
        r.last = ctx;
    }
    r.first = a.window ? int32_t(max(int64_t(0), int64_t(r.pos) + 1 - int64_t(a.window))) : 0;
    if (a.spans) {
        const int2 s = reinterpret_cast<const int2*>(a.spans)[t];
        r.first = max(s.x, 0), r.last = min(s.y, q.len);
    }
    return r;
}

// What becomes of a product before the mask: it is scaled only, or capped and less
// the distance's bias, or that with a softcap above kFineCap.
enum class Mod { kNone, kSome, kFine };
constexpr float kFineCap = 64.0f;
inline Mod mod_of(const KvAttend& a) {
    return a.softcap > kFineCap ? Mod::kFine : a.softcap != 0.0f || a.slopes ? Mod::kSome : Mod::kNone;
}

// A capped score in units of log2, from a raw product (cap in log2 units; cap_in =
// scale / softcap).
template <bool FINE>
__device__ __forceinline__ float capped(float s, float cap_in, float cap) {
    // tanh(y) = 1 - 2 / (exp(2y) + 1), within 2e-7: 1.3e-5 of a score at kFineCap, and too far for a cap high above
    // the score (0.2 at 10^6). There it is, near 0, the beginning of its Taylor series, y - y^3 / 3 + 2 y^5 / 15 -
    // 17 y^7 / 315 + 62 y^9 / 2835. At the line between them (0.35) the one is within 3e-7 of tanh(y), the other
    // within 6e-7; below and above it is less. (Taken for every cap: 48 sequences in a window of 4,096, 29.2 -> 33.3
    // us, a prompt of 8190 tokens 920 -> 1107; chosen within one kernel, 29.9 and 943.)
    if (!FINE) return cap - 2.0f * cap * tc::rcp_approx(tc::exp2_approx(s * cap_in * (2.0f * kLog2e)) + 1.0f);
    const float y = s * cap_in, z = y * y;
    const float far = 1.0f - 2.0f * tc::rcp_approx(tc::exp2_approx(y * (2.0f * kLog2e)) + 1.0f);
    const float near = y + y * z * (-1.0f / 3.0f + z * (2.0f / 15.0f + z * (-17.0f / 315.0f + z * (62.0f / 2835.0f))));
    return cap * (z < 0.35f * 0.35f ? near : far);
}

// A sum of many positive numbers, with what its roundings lost (within a unit of the sum's last place or two,
// whatever their number; the compiler keeps the order of fp32 operations).
struct KvSum {
    float sum = 0.0f, lost = 0.0f;
    __device__ __forceinline__ void add(float x) {
        const float s = sum + x, big = fmaxf(sum, x), small = fminf(sum, x);
        lost += small - (s - big);
        sum = s;
    }
    __device__ __forceinline__ void scale(float by) { sum *= by, lost *= by; }
    __device__ __forceinline__ float value() const { return sum + lost; }
};

// Blocks of an attention launch: no more than there are key tiles, going by max_len
// (a block without any still takes its place on an SM and has to be waited for).
inline uint32_t attend_blocks(const KvAttend& a, uint32_t most, uint64_t units) {
    const uint64_t tiles = units * a.pages.kv_heads * (uint64_t(a.max_len) / kTileKeys + 1);
    return uint32_t(tiles < most ? tiles : most);
}

// A launch whose set-up overlaps the kernel before it on the stream.
template <class... Args>
inline cudaError_t launch_pdl(void (*kernel)(Args...), dim3 grid, uint32_t threads, uint32_t smem, cudaStream_t stream,
                       const typename std::common_type<Args>::type&... args) {
    cudaLaunchConfig_t c{};
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    c.attrs = at;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, kernel, args...);
}

}  // namespace t2i
