// DLPack's C interface to tensors: the structures of its public header that the native calls use.
#pragma once

#include <stdint.h>

namespace {

struct DLDevice {
    int32_t type, id;
};
struct DLDataType {
    uint8_t code, bits;
    uint16_t lanes;
};
struct DLTensor {
    void* data;
    DLDevice device;
    int32_t ndim;
    DLDataType dtype;
    int64_t *shape, *strides;
    uint64_t byte_offset;
};
struct DLPackExchangeAPI {
    uint32_t major, minor;
    void *previous, *allocator, *from_object, *to_object;
    int (*tensor_from_object)(void* object, DLTensor* out);
    void* current_work_stream;
};

// The capsule's name where torch_tensors.cpp made it, whose function refuses negated views.
constexpr char kBuiltExchange[] = "draco_torch_tensors";

}  // namespace
