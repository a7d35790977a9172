// The key/value cache in the store's pages: what its host side (kv.cu) and its
// kernels (kv_append.cu, kv_few.cuh, kv_rows.cuh) share. The calls are described in
// include/t2istore.h.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace t2i {

// Where the rows of one layer lie.
struct KvPages {
    uint64_t pool;         // device address of page 0
    uint64_t page_bytes;
    uint32_t total_pages;
    uint32_t token_shift;  // log2 of the tokens of a page
    uint32_t kv_heads;
    uint32_t head_dim;
    uint32_t layers;
    uint32_t layer;
    const int32_t* table;
    uint64_t table_stride;
    uint32_t table_pages;
};

// A call's sequences and their new tokens.
struct KvTokens {
    const int32_t* lens;
    const int32_t* starts;  // null: `each` tokens of every sequence
    uint32_t each;
    uint32_t n_seqs;
    uint32_t n_tokens;
    uint32_t max_new;
};

struct KvAppend {
    KvPages pages;
    KvTokens tok;
    const void* q;
    const void* k;
    const void* v;
    void* q_out;
    uint64_t q_stride, k_stride, v_stride, q_out_stride;
    const float* q_norm;
    const float* k_norm;
    const float* cos_table;
    const float* sin_table;
    const int32_t* positions;
    uint32_t q_heads;  // 0: keys and values only
    uint32_t rotary_dim;
    uint32_t n_positions;
    uint32_t interleaved;
    float eps;
    uint32_t vectors;  // the launch's own: norm weights and tables may be read in 16 bytes
};

struct KvAttend {
    KvPages pages;
    KvTokens tok;
    const void* q;
    void* out;
    float* lse;
    uint64_t q_stride, out_stride;
    const float* slopes;
    const int32_t* spans;
    const uint64_t* tree;
    uint32_t q_heads;
    uint32_t group;  // q_heads / kv_heads
    uint32_t window;
    uint32_t max_len;
    float scale;
    float softcap;
};

struct KvCommit {
    KvPages pages;
    const int32_t* ctx;
    const int32_t* path;
    const int32_t* counts;
    uint32_t n_seqs;
    uint32_t max_path;
};

// dtype and in_dtype: T2I_BF16, T2I_F16, T2I_F32
cudaError_t launch_kv_append(const KvAppend& a, uint32_t dtype, uint32_t in_dtype, cudaStream_t stream);
cudaError_t launch_kv_commit(const KvCommit& c, cudaStream_t stream);

// What an attention launch needs beside its arguments.
struct KvLaunch {
    // the pool as [pages][rows of a page][head_dim], in boxes of 64 elements by
    // min(page tokens, 128) rows, 128-byte swizzle; elements outside read as zeros
    const CUtensorMap* map;
    void* workspace;
    uint32_t* fault;  // host memory that the device writes: not 0 after a wait that ran out
    uint32_t sms;
    uint32_t no_loads;  // testing: the loading warps do nothing
};
// Up to this many queries to a key head (new tokens of a sequence x heads of a group) kv_few.cuh, above it
// kv_rows.cuh. Queries, and us of the one / the other, for a sequence of 1.5k slots, 24 of 8k (heads of 128) and 3 of
// 3k (heads of 64): 32: 15.3 / 16.9, 137 / 141, 19.2 / 18.5; 36 (with 64 columns) 22.5 / 17.1, 201 / 148, 26 / 19;
// 128: 24 / 19, 389 / 148, 35 / 20.
constexpr uint32_t kFewRows = 32;
cudaError_t launch_kv_few_bf16(const KvAttend& a, const KvLaunch& l, cudaStream_t stream);
cudaError_t launch_kv_few_f16(const KvAttend& a, const KvLaunch& l, cudaStream_t stream);
uint64_t kv_few_workspace(uint32_t sms);
// more of them
cudaError_t launch_kv_rows_bf16(const KvAttend& a, const KvLaunch& l, cudaStream_t stream);
cudaError_t launch_kv_rows_f16(const KvAttend& a, const KvLaunch& l, cudaStream_t stream);
uint64_t kv_rows_workspace(uint32_t sms, uint32_t n_seqs, uint32_t n_tokens, uint32_t group);

}  // namespace t2i
