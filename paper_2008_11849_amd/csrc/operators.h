// The operators around the products: what the boundary (operators.cpp) hands to the device side (norm.hip,
// dequantize.hip, adapters.hip).  Descriptors arrive here checked and filled in: batch >= 1, every pitch >= N.
#pragma once
#include <cstddef>
#include <cstdint>
#include <string>

#include "../../include/sparsert.h"

namespace sparsert {

int set_error(int code, const std::string &msg);   // (api.cpp)

// Is `stream` one of the current device?
bool stream_of_current_device(void *stream);

struct NormCall {
    sparsert_norm d;
    const void *X, *R;
    const float *gamma;
    void *H, *Y;
    float *scale, *workspace;   // workspace: NULL or norm_workspace bytes
    void *stream;
};
size_t norm_workspace(const sparsert_norm &d);
int launch_norm(const NormCall &c, std::string &err);

struct DequantCall {
    sparsert_dequant d;
    const int32_t *C;
    const float *row, *col;
    void *Y, *stream;
};
int launch_dequantize(const DequantCall &c, std::string &err);

struct AdaptersCall {
    sparsert_adapter_set d;
    const void *X, *down, *up;
    const int32_t *index;
    const float *alpha;
    const void *C;
    const float *row, *col;
    void *Y, *workspace, *stream;
};
size_t adapters_workspace(const sparsert_adapter_set &d);
int launch_adapters(const AdaptersCall &c, std::string &err);

}  // namespace sparsert
