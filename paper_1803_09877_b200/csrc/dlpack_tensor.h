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

// What torch_tensors.cpp offers, in a capsule whose name has the number of its functions (a module that was built earlier may be left): both that
// read a tensor refuse negated views, the second gives the address of memory that may be written; the third tells autograd that it has been.
struct BuiltExchange {
    DLPackExchangeAPI read;
    int (*written_from_object)(void* object, DLTensor* out);
    int (*increment_version)(void* object);
};
constexpr char kBuiltExchange[] = "draco_torch_tensors_3";

}  // namespace
