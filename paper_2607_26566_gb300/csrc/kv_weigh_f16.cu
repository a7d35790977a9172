// kv_weigh.cuh for a cache of fp16.
#include "kv_weigh.cuh"

namespace t2i {

cudaError_t launch_kv_weigh_f16(const KvWeigh& w, const KvLaunch& l, cudaStream_t stream) {
    return launch_weigh<__half>(w, l, stream);
}

}  // namespace t2i
