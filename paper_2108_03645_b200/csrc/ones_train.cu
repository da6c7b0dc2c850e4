// What the training-step operators share: tensor maps, the device's size, the status of their waits.
#include <atomic>

#include "ones_attention.cuh"
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

cudaError_t encode_box(CUtensorMap* out, const void* p, const uint64_t (&dims)[3], const uint64_t (&strides)[2], const uint32_t (&box)[3], bool f16) {
    static std::atomic<EncodeFn> encode{nullptr};
    EncodeFn fn = encode.load(std::memory_order_relaxed);
    if (!fn) {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        cudaError_t err = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
        if (err != cudaSuccess) return err;
        if (found != cudaDriverEntryPointSuccess || !f) return cudaErrorNotSupported;
        fn = reinterpret_cast<EncodeFn>(f);
        encode.store(fn, std::memory_order_relaxed);
    }
    const cuuint64_t d[3] = {dims[0], dims[1], dims[2]}, s[2] = {strides[0], strides[1]};
    const cuuint32_t b[3] = {box[0], box[1], box[2]}, unit[3] = {1, 1, 1};
    const CUresult res = fn(out, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
                            const_cast<void*>(p), d, s, b, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return res == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t make_map(CUtensorMap* out, const Operand& o, int rows, int k, int batch, bool f16, int box_rows) {
    const uint64_t inner = o.mn ? rows : k, outer = o.mn ? k : rows;
    const uint64_t dims[3] = {inner, outer, (uint64_t)batch};
    const uint64_t strides[2] = {(uint64_t)o.ld * 2, (uint64_t)(batch > 1 ? o.batch_ld : o.ld * (int64_t)outer) * 2};
    const uint32_t box[3] = {64, o.mn ? (uint32_t)kTileK : (uint32_t)box_rows, 1};
    return encode_box(out, o.p, dims, strides, box, f16);
}

}  // namespace ones

namespace {
const ones::WaitControl* const kWaits[] = {&ones::norm_waits, &ones::loss_waits, &ones::update_waits, &ones::attention_waits,
                                            &ones::attention_back_waits};
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
    if (which < 0 || which > 4) return ONES_ERR_BAD_PARAM;
    return kWaits[which]->nothing(times, reinterpret_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? ONES_OK : ONES_ERR_CUDA;
}

}  // extern "C"
