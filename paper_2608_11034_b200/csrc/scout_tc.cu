// Host side of scout_tc.cuh: tensor maps, and the counter of waits that gave up, which is never reset.
#include <cuda.h>

#include <mutex>

#include "scout_replay.h"
#include "scout_tc.cuh"

namespace scout {
namespace tc {
namespace {

__device__ uint32_t g_gave_up;

using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                            const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// the driver's encoder, looked up through the runtime so that the library does not link against the driver
Encode encoder() {
    static Encode f = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult how;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &how) != cudaSuccess ||
            how != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<Encode>(p);
    }();
    return f;
}

}  // namespace

int tensor_map(CUtensorMap *map, bool bf16, const void *base, int rank, const uint64_t *dims, const uint64_t *strides, uint32_t box_rows) {
    const Encode f = encoder();
    if (!f) {
        set_cuda_error(cudaErrorNotSupported, "cuTensorMapEncodeTiled");
        return SCOUT_ERR_CUDA;
    }
    cuuint64_t d[5], s[5];
    cuuint32_t box[5] = {64, box_rows, 1, 1, 1}, one[5] = {1, 1, 1, 1, 1};
    for (int i = 0; i < rank; ++i) d[i] = dims[i];
    for (int i = 0; i + 1 < rank; ++i) s[i] = strides[i];
    const auto encode = [&] {
        return f(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank, const_cast<void *>(base), d, s, box,
                 one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    CUresult r = encode();
    if (r != CUDA_SUCCESS) {
        // The driver's calls want a context on the calling thread, which the runtime puts there with the thread's first call of its own
        // that needs one: in a new thread (autograd's, say) that may still be to come.
        int dev = 0;
        SCOUT_CUDA(cudaGetDevice(&dev));
        SCOUT_CUDA(cudaSetDevice(dev));
        r = encode();
    }
    if (r != CUDA_SUCCESS) {
        set_cuda_error(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
        return SCOUT_ERR_CUDA;
    }
    return SCOUT_OK;
}

int gave_up_counter(uint32_t **counter) {
    static std::mutex lock;
    static uint32_t *known[64] = {};
    int dev = 0;
    SCOUT_CUDA(cudaGetDevice(&dev));
    std::lock_guard<std::mutex> hold(lock);
    if (dev < 64 && known[dev]) {
        *counter = known[dev];
        return SCOUT_OK;
    }
    void *p = nullptr;
    SCOUT_CUDA(cudaGetSymbolAddress(&p, g_gave_up));
    *counter = (uint32_t *)p;
    if (dev < 64) known[dev] = *counter;
    return SCOUT_OK;
}

}  // namespace tc
}  // namespace scout

extern "C" int scout_replay_waits(uint32_t *total) {
    using namespace scout;
    if (!total) return SCOUT_ERR_INVALID;
    uint32_t *p = nullptr;
    if (int rc = tc::gave_up_counter(&p)) return rc;
    SCOUT_CUDA(cudaDeviceSynchronize());
    SCOUT_CUDA(cudaMemcpy(total, p, sizeof *total, cudaMemcpyDeviceToHost));
    return SCOUT_OK;
}

extern "C" int scout_replay_error(uint32_t *count) {
    using namespace scout;
    static std::mutex lock;
    static uint32_t reported[64] = {};  // by device
    if (!count) return SCOUT_ERR_INVALID;
    int dev = 0;
    uint32_t total = 0;
    SCOUT_CUDA(cudaGetDevice(&dev));
    if (dev >= 64) return SCOUT_ERR_UNSUPPORTED;
    if (int rc = scout_replay_waits(&total)) return rc;
    std::lock_guard<std::mutex> hold(lock);
    *count = total - reported[dev];
    reported[dev] = total;
    return SCOUT_OK;
}
