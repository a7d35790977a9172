// kv_few.cuh for a cache of bf16 (the two types compile side by side).
#include "kv_few.cuh"

namespace t2i {

uint64_t kv_few_workspace(uint32_t sms) {
    return join_bytes(sms) + uint64_t(sms) * 4 * Shape<32, 2>::kPart * sizeof(float);
}

cudaError_t launch_kv_few_bf16(const KvAttend& a, const KvLaunch& l, cudaStream_t stream) {
    return launch_few<__nv_bfloat16>(a, l, stream);
}

}  // namespace t2i
