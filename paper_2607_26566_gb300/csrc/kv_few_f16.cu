// kv_few.cuh for a cache of fp16.
#include "kv_few.cuh"

namespace t2i {

cudaError_t launch_kv_few_f16(const KvAttend& a, const KvLaunch& l, cudaStream_t stream) {
    return launch_few<__half>(a, l, stream);
}

}  // namespace t2i
