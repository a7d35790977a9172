// kv_weigh.cuh for a cache of bf16 (the two types compile side by side).
#include "kv_weigh.cuh"

namespace t2i {

cudaError_t launch_kv_weigh_bf16(const KvWeigh& w, const KvLaunch& l, cudaStream_t stream) {
    return launch_weigh<__nv_bfloat16>(w, l, stream);
}

uint64_t kv_weigh_workspace(uint32_t sms, uint32_t n_seqs, uint32_t n_tokens) {
    // (hulls of a token each at most: a tile's tokens follow from max_new, which this does not know)
    return weigh_up(sms * sizeof(WeighJoin)) + weigh_up(uint64_t(sms) * 2 * kPartFloats * sizeof(float)) +
           weigh_up(weigh_hulls(n_seqs, n_tokens, 1) * sizeof(int2));
}

}  // namespace t2i
