// kv_rows.cuh for a cache of fp16.
#include "kv_rows.cuh"

namespace t2i {

cudaError_t launch_kv_rows_f16(const KvAttend& a, const KvLaunch& l, cudaStream_t stream) {
    return launch_rows<__half>(a, l, stream);
}

}  // namespace t2i
