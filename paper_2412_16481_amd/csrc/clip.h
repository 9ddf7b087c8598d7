// Internal interface between the C ABI (flash3d_api.hip) and the gradient clipping kernels (clip.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace f3d {

constexpr int CLIP_MAX_TENSORS = 65536;
constexpr int CLIP_TENSORS = 128;       // tensors that travel in the arguments of one launch
constexpr int CLIP_MAX_PARTS = 4096;    // partial sums of squares

struct ClipTensor {
    const char* in;
    char* out;
    long long size;                     // elements
    int type;
    int first;                          // chunks of the tensors before it
};

// what one launch of the first kernel carries: an array of structures would repeat their padding
struct ClipBatch {
    const char* in[CLIP_TENSORS];
    char* out[CLIP_TENSORS];
    long long size_type[CLIP_TENSORS];  // size * 4 + type
    int first[CLIP_TENSORS + 1];        // chunks of this launch's tensors before the i-th
    int tensors;
    int at;                             // tensors before this launch's
    int chunks_at;                      // their chunks
    int parts_at;                       // first of its partial sums
};
static_assert(sizeof(ClipBatch) <= 4096 - 64, "kernel arguments hold 4 KB");

struct ClipArgs {
    const void* const* in;              // host arrays
    void* const* out;
    const int64_t* sizes;
    const int32_t* types;
    int tensors;
    float max_norm;
    float* norm;
    double* parts;                      // [CLIP_MAX_PARTS]
    ClipTensor* table;                  // [tensors]
};

hipError_t clip_launch(const ClipArgs& a, hipStream_t stream);
long long clip_chunks(const void* in, int64_t size, int type);

}  // namespace f3d
