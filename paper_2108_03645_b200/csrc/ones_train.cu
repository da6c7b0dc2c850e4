// What the training-step operators share: tensor maps, the device's size, the status of their waits.
#include <atomic>

#include "ones_matmul.cuh"
#include "ones_train.h"
#include "ones_train_internal.h"

namespace ones {

int device_sms() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return kSms;
    n = known[dev & 63].load(std::memory_order_relaxed);
    if (n) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 2) return kSms;
    known[dev & 63].store(n, std::memory_order_relaxed);
    return n;
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

cudaError_t make_map(CUtensorMap* out, const Operand& o, int rows, int k, int batch, bool f16, int box_rows) {
    static std::atomic<EncodeFn> encode{nullptr};
    EncodeFn fn = encode.load(std::memory_order_relaxed);
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        cudaError_t err = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found);
        if (err != cudaSuccess) return err;
        if (found != cudaDriverEntryPointSuccess || !p) return cudaErrorNotSupported;
        fn = reinterpret_cast<EncodeFn>(p);
        encode.store(fn, std::memory_order_relaxed);
    }
    const cuuint64_t inner = o.mn ? rows : k, outer = o.mn ? k : rows;
    const cuuint64_t dims[3] = {inner, outer, (cuuint64_t)batch};
    const cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)(batch > 1 ? o.batch_ld : o.ld * (int64_t)outer) * 2};
    const cuuint32_t box[3] = {64, o.mn ? (cuuint32_t)kTileK : (cuuint32_t)box_rows, 1};
    const cuuint32_t unit[3] = {1, 1, 1};
    const CUresult res = fn(out, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
                            const_cast<void*>(o.p), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return res == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace ones

namespace {
const ones::WaitControl* const kWaits[] = {&ones::norm_waits, &ones::loss_waits, &ones::update_waits};
}

extern "C" {

int ones_train_status(void* cuda_stream) {
    if (cudaStreamSynchronize(reinterpret_cast<cudaStream_t>(cuda_stream)) != cudaSuccess) return ONES_ERR_CUDA;
    unsigned any = 0;
    for (const ones::WaitControl* w : kWaits) {
        unsigned expired = 0;
        if (w->expired(&expired) != cudaSuccess) return ONES_ERR_CUDA;
        any |= expired;
    }
    return any ? ONES_ERR_TIMEOUT : ONES_OK;
}

int ones_train_wait_limit(unsigned long long ns) {
    for (const ones::WaitControl* w : kWaits)
        if (w->limit(ns) != cudaSuccess) return ONES_ERR_CUDA;
    return ONES_OK;
}

int ones_train_wait_for_nothing(int which, int times, void* cuda_stream) {
    if (which < 0 || which > 2) return ONES_ERR_BAD_PARAM;
    return kWaits[which]->nothing(times, reinterpret_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // extern "C"
