// kv_rows.cuh for a cache of bf16.
#include "kv_rows.cuh"

namespace t2i {

uint64_t kv_rows_workspace(uint32_t sms, uint32_t n_seqs, uint32_t n_tokens, uint32_t group) {
    return 256 + up256(sms * sizeof(Join)) + up256((uint64_t(n_seqs) + 1) * 4) +
           up256(plan_tiles(n_seqs, n_tokens, group) * sizeof(PlanTile)) + uint64_t(sms) * 2 * kRowPart * sizeof(float);
}

cudaError_t launch_kv_rows_bf16(const KvAttend& a, const KvLaunch& l, cudaStream_t stream) {
    return launch_rows<__nv_bfloat16>(a, l, stream);
}

}  // namespace t2i
