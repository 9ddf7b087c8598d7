// The global norm of the gradients of a training step (attention, maps, layer norm: any number of tensors of different types) and
// their scaling to a largest norm.
//
//   norm = sqrt(sum over tensors, elements of g^2),  c = min(1, max_norm / (norm + 1e-6)),  out = c g
//
// Two passes over the data, one launch each: a workgroup cannot scale before the last square has been added. Tensors are cut into
// chunks of 32 KB that start at a multiple of 16 bytes, and workgroups walk over the chunks of all tensors, so a hundred vectors
// of a few elements cost a hundred chunks and no launches. The first launch gets its tensors in the kernel's arguments (128 of them;
// more take further launches) and leaves them in the workspace for the second. Squares and their sums are held in binary64: no
// finite gradient overflows them, and the instructions (a conversion and a multiply-add per element) hide behind the loads. Every
// workgroup of the second pass adds up the first pass's sums for itself, in a fixed order: the same call gives the same bits.
//
// Bound: HBM, every gradient read twice and written once. 400 million bfloat16 elements in 672 tensors, 2.4 GB: 183 us for the squares and
// 296 for the scaling = 4.4 and 5.4 TB/s. 336 small tensors: 15 us, beside which the host's work on 336 tensors counts for more.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "clip.h"
#include "elem.h"

namespace f3d {

namespace {

constexpr int CTH = 256;
constexpr int PIECES = 2048;            // 16-byte pieces of a chunk

// Elements [0, size) of a tensor lie in the pieces of 16 bytes from the one on that its first byte is in. `skip`: elements of that
// piece before the tensor.
__device__ __forceinline__ int skipped(const char* p, int bytes) { return (int)((uintptr_t)p & 15) / bytes; }

// which of `n` tensors the chunk belongs to, from the chunks before each (first[0] = 0): 64 at a time, the last that begins at or before it
__device__ __forceinline__ int tensor_of(const int* first, int stride, int n, int chunk)
{
    const int lane = threadIdx.x & 63;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) / 64, i = lane * step;
        const bool before = i < n && first[(size_t)(lo + i) * stride] <= chunk;
        const int k = __popcll(__builtin_amdgcn_ballot_w64(before)) - 1;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double v, double* box)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = v;
    __syncthreads();
    return (box[0] + box[1]) + (box[2] + box[3]);
}

template <int TYPE>
__device__ __forceinline__ double squares(const char* in, long long size, long long chunk)
{
    using E = Elems<TYPE>;
    using one = typename E::one;
    constexpr int W = E::W;
    const int skip = skipped(in, sizeof(one));
    const uint4* const base = reinterpret_cast<const uint4*>(in - (size_t)skip * sizeof(one));
    const long long end = size + skip;                // in elements from `base` on
    const long long p0 = chunk * PIECES;
    double s = 0.0;
    if (p0 * W >= skip && (p0 + PIECES) * W <= end) { // all of the chunk's pieces are the tensor's
#pragma unroll
        for (int k = 0; k < PIECES / CTH; k += 4) {
            uint4 u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = base[p0 + (k + i) * CTH + threadIdx.x];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x[W];
                E::unpack(u[i], x);
#pragma unroll
                for (int e = 0; e < W; ++e) s = __builtin_fma((double)x[e], (double)x[e], s);
            }
        }
        return s;
    }
    for (long long p = p0 + threadIdx.x; p < p0 + PIECES && p * W < end; p += CTH) {
        if (p * W >= skip && (p + 1) * W <= end) {
            float x[W];
            E::unpack(base[p], x);
#pragma unroll
            for (int e = 0; e < W; ++e) s = __builtin_fma((double)x[e], (double)x[e], s);
        } else {                                      // the tensor's first or last piece: its elements alone
            for (int e = 0; e < W; ++e) {
                const long long i = p * W + e - skip;
                if (i < 0 || i >= size) continue;
                const double x = (double)E::to_f32(reinterpret_cast<const one*>(in)[i]);
                s = __builtin_fma(x, x, s);
            }
        }
    }
    return s;
}

__global__ __launch_bounds__(CTH) void k_clip_norm(ClipBatch b, double* parts, ClipTensor* table)
{
    __shared__ double box[4];
    if (blockIdx.x == 0 && threadIdx.x < (unsigned)b.tensors) {
        const int i = threadIdx.x;
        ClipTensor t;
        t.in = b.in[i];
        t.out = b.out[i];
        t.size = b.size_type[i] >> 2;
        t.type = (int)(b.size_type[i] & 3);
        t.first = b.chunks_at + b.first[i];
        table[b.at + i] = t;
    }
    double s = 0.0;
    const int chunks = b.first[b.tensors];
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int i = __builtin_amdgcn_readfirstlane(tensor_of(b.first, 1, b.tensors, c));
        const long long size = b.size_type[i] >> 2, chunk = c - b.first[i];
        const int type = (int)(b.size_type[i] & 3);
        if (type == F3D_BF16) s += squares<F3D_BF16>(b.in[i], size, chunk);
        else if (type == F3D_F16) s += squares<F3D_F16>(b.in[i], size, chunk);
        else s += squares<F3D_F32>(b.in[i], size, chunk);
    }
    s = block_sum(s, box);
    if (threadIdx.x == 0) parts[b.parts_at + blockIdx.x] = s;
}

// The factor, in two where binary32 would hold it with fewer bits (norms past 10^38 times the largest one): the second is a power of two.
struct Factor {
    float by, then;
};
__device__ __forceinline__ float operator*(float x, Factor c) { return x * c.by * c.then; }

template <int TYPE>
__device__ __forceinline__ void scale(const char* in, char* out, long long size, long long chunk, Factor c)
{
    using E = Elems<TYPE>;
    using one = typename E::one;
    constexpr int W = E::W;
    const int skip = skipped(in, sizeof(one));
    const long long end = size + skip, p0 = chunk * PIECES;
    const uint4* const base = reinterpret_cast<const uint4*>(in - (size_t)skip * sizeof(one));
    if (skipped(out, sizeof(one)) != skip) {          // no common pieces: element by element
        const one* const x = reinterpret_cast<const one*>(in);
        one* const y = reinterpret_cast<one*>(out);
        const long long i0 = p0 * W - skip, i1 = min(i0 + PIECES * W, size);
        for (long long i = max(i0, 0ll) + threadIdx.x; i < i1; i += CTH) y[i] = E::from_f32(E::to_f32(x[i]) * c);
        return;
    }
    uint4* const to = reinterpret_cast<uint4*>(out - (size_t)skip * sizeof(one));
    if (p0 * W >= skip && (p0 + PIECES) * W <= end) {
#pragma unroll
        for (int k = 0; k < PIECES / CTH; k += 4) {
            uint4 u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = base[p0 + (k + i) * CTH + threadIdx.x];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x[W];
                E::unpack(u[i], x);
#pragma unroll
                for (int e = 0; e < W; ++e) x[e] = x[e] * c;
                to[p0 + (k + i) * CTH + threadIdx.x] = E::pack(x);
            }
        }
        return;
    }
    for (long long p = p0 + threadIdx.x; p < p0 + PIECES && p * W < end; p += CTH) {
        if (p * W >= skip && (p + 1) * W <= end) {
            float x[W];
            E::unpack(base[p], x);
#pragma unroll
            for (int e = 0; e < W; ++e) x[e] = x[e] * c;
            to[p] = E::pack(x);
        } else {
            for (int e = 0; e < W; ++e) {
                const long long i = p * W + e - skip;
                if (i >= 0 && i < size) reinterpret_cast<one*>(out)[i] = E::from_f32(E::to_f32(reinterpret_cast<const one*>(in)[i]) * c);
            }
        }
    }
}

__global__ __launch_bounds__(CTH) void k_clip_scale(const ClipTensor* table, int tensors, int chunks, const double* parts, int n_parts,
                                                    float max_norm, float* norm_out)
{
    __shared__ double box[4];
    double s = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < n_parts; i += CTH) s += parts[i];
    const double norm = sqrt(block_sum(s, box));
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    double ratio = (double)max_norm / (norm + 1e-6);
    // a norm that is no number stays one in every gradient; no norm is longer than an infinite largest one
    if (ratio > 1.0 || isinf(max_norm)) ratio = 1.0;
    Factor c = {(float)ratio, 1.0f};
    if (ratio < 0x1p-120) c = {(float)(ratio * 0x1p64), 0x1p-64f};
    for (int k = blockIdx.x; k < chunks; k += gridDim.x) {
        const int at = chunks - 1 - k;                // what the first pass read last may still be in a cache
        const int i = __builtin_amdgcn_readfirstlane(tensor_of(&table->first, sizeof(ClipTensor) / sizeof(int), tensors, at));
        const ClipTensor t = table[i];
        if (c.by == 1.0f && t.in == t.out) continue;     // in place and short enough: every element is what it has to be
        if (t.type == F3D_BF16) scale<F3D_BF16>(t.in, t.out, t.size, at - t.first, c);
        else if (t.type == F3D_F16) scale<F3D_F16>(t.in, t.out, t.size, at - t.first, c);
        else scale<F3D_F32>(t.in, t.out, t.size, at - t.first, c);
    }
}

}  // namespace

long long clip_chunks(const void* in, int64_t size, int type)
{
    const int bytes = elem_bytes(type);
    const long long end = size + (long long)((uintptr_t)in & 15) / bytes;
    const long long per = (long long)PIECES * (16 / bytes);
    return size ? (end + per - 1) / per : 0;
}

hipError_t clip_launch(const ClipArgs& a, hipStream_t stream)
{
    const int launches = (a.tensors + CLIP_TENSORS - 1) / CLIP_TENSORS;
    const int most = CLIP_MAX_PARTS / (launches > 2 ? launches : 2);   // eight workgroups per compute unit are all that run at a time
    int parts = 0, chunks = 0, at = 0;
    while (at < a.tensors) {
        ClipBatch b;
        b.at = at;
        b.chunks_at = chunks;
        b.parts_at = parts;
        b.tensors = 0;
        b.first[0] = 0;
        for (; b.tensors < CLIP_TENSORS && at < a.tensors; ++at) {
            const int i = b.tensors++;
            b.in[i] = static_cast<const char*>(a.in[at]);
            b.out[i] = static_cast<char*>(a.out ? a.out[at] : const_cast<void*>(a.in[at]));
            b.size_type[i] = a.sizes[at] * 4 + a.types[at];
            b.first[i + 1] = b.first[i] + (int)clip_chunks(a.in[at], a.sizes[at], a.types[at]);
        }
        const int mine = b.first[b.tensors], blocks = mine < 1 ? 1 : mine < most ? mine : most;
        k_clip_norm<<<(unsigned)blocks, CTH, 0, stream>>>(b, a.parts, a.table);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        parts += blocks;
        chunks += mine;
    }
    const int blocks = chunks < 1 ? 1 : chunks < 2048 ? chunks : 2048;
    k_clip_scale<<<(unsigned)blocks, CTH, 0, stream>>>(a.table, a.tensors, chunks, a.parts, parts, a.max_norm, a.norm);
    return hipGetLastError();
}

}  // namespace f3d
