#include "kv_weigh.cuh"

namespace t2i {

cudaError_t launch_kv_weigh_bf16(const KvWeigh& w, const KvLaunch& l, cudaStream_t stream) {
    return launch_weigh<__nv_bfloat16>(w, l, stream);
}

uint64_t kv_weigh_workspace(uint32_t sms, uint32_t n_seqs, uint32_t n_tokens, uint32_t group) { return 0; }

}  // namespace t2i
