// Host side that the training-step entry points share.
#include "train_common.cuh"

namespace fp {
namespace train {

void* driver_function(const char* name, std::atomic<void*>* known) {
    void* f = known->load(std::memory_order_acquire);
    if (!f) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint(name, &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        known->store(f, std::memory_order_release);
    }
    return f;
}

bool Buffers::ask(uint64_t a, uint64_t* start, uint64_t* size) const {
    typedef CUresult (*GetAttributes)(unsigned, CUpointer_attribute*, void**, CUdeviceptr);
    static std::atomic<void*> known;
    const GetAttributes get = (GetAttributes)driver_function("cuPointerGetAttributes", &known);
    if (!get || !a) return false;
    unsigned type = 0, managed = 0;
    int dev = -1;
    CUdeviceptr from = 0;
    size_t bytes = 0;
    CUpointer_attribute what[5] = {CU_POINTER_ATTRIBUTE_MEMORY_TYPE, CU_POINTER_ATTRIBUTE_IS_MANAGED, CU_POINTER_ATTRIBUTE_DEVICE_ORDINAL,
                                   CU_POINTER_ATTRIBUTE_RANGE_START_ADDR, CU_POINTER_ATTRIBUTE_RANGE_SIZE};
    void* to[5] = {&type, &managed, &dev, &from, &bytes};
    if (get(5, what, to, (CUdeviceptr)a) != CUDA_SUCCESS) return false;      // an address that the driver does not know: type 0
    if (!(managed || (type == CU_MEMORYTYPE_DEVICE && dev == dev_))) return false;
    *start = bytes ? (uint64_t)from : a;
    *size = bytes ? (uint64_t)bytes : 1;
    return true;
}

}  // namespace train
}  // namespace fp
