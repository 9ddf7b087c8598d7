// Device helpers shared by the cross attention's forward (cross.hip) and backward (cross_bwd.hip): segments and their rows, the
// layout of staged rows in LDS, 16-bit element types.
#pragma once
#include "attn_common.h"
#include "cross.h"

namespace f3d {

namespace {

template <bool F16>
struct Half {
    // Bounds of a sum of exponentials taken against the reference 0. bfloat16: binary32 has room for the products with values of 2^80 on
    // either side. binary16: a probability above 65504 rounds to infinity, and what is lost of those below 2^-14 stays below 2^-25 a
    // key of the sum.
    static constexpr float SUM_LO = F16 ? 1.0f : 0x1p-40f, SUM_HI = F16 ? 65504.f : 0x1p40f;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        if constexpr (F16) {
            const f32x2 x = {lo, hi};
            const f16x2 y = __builtin_convertvector(x, f16x2);   // round to nearest even
            return *reinterpret_cast<const uint32_t*>(&y);
        } else {
            return pack_bf16(lo, hi);
        }
    }
    static __device__ __forceinline__ float sum2(uint32_t pair, float c)   // c + both halves of the pair
    {
        const uint32_t ones = F16 ? 0x3C003C00u : 0x3F803F80u;
        if constexpr (F16) return __builtin_amdgcn_fdot2(*reinterpret_cast<const f16x2*>(&pair), *reinterpret_cast<const f16x2*>(&ones), c, false);
        else return __builtin_amdgcn_fdot2_f32_bf16(*reinterpret_cast<const bf16x2*>(&pair), *reinterpret_cast<const bf16x2*>(&ones), c, false);
    }
    static __device__ __forceinline__ f32x16 mfma(const U4& x, const U4& y, f32x16 c)
    {
        if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(x.f, y.f, c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.b, y.b, c, 0, 0, 0);
    }
};

// A segment's rows in a tensor of n: [from, from + span), of which the first `len` take part. Whatever the arrays hold, the rows
// are the tensor's.
struct Rows {
    int from, span, len;
};

// first row of segment b; no offsets: one segment of all rows
__device__ __forceinline__ int offset_of(const int32_t* offsets, int n, int b) { return offsets ? min(max(offsets[b], 0), n) : b ? n : 0; }

__device__ __forceinline__ Rows rows_of(const int32_t* offsets, const int32_t* lens, int n, int b)
{
    Rows r;
    r.from = offset_of(offsets, n, b);
    r.span = max(offset_of(offsets, n, b + 1) - r.from, 0);
    r.len = lens ? min(max(lens[b], 0), r.span) : r.span;
    return r;
}

// Row blocks: segment b owns the block slots from first_slot(b) on; a block is 2^shift rows, a row of the tensor counts `per` times
// (once per head that shares keys). floor((o + len) / B) - floor(o / B) + 1 is room for ceil(len / B) blocks wherever o is, so
// neither the host nor another segment has to know how many there are.
__device__ __forceinline__ long long first_slot(const int32_t* offsets, int n, int b, int per, int shift)
{
    return ((long long)offset_of(offsets, n, b) * per >> shift) + b;
}

// The segment that owns the slot, 64 candidates at a time: the last whose slots begin at or before it
__device__ __forceinline__ int segment_of(const int32_t* offsets, int n, int segments, int per, int shift, int slot)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, left = segments;
    while (left > 1) {
        const int step = (left + 63) / 64, i = lane * step;
        const bool before = i < left && first_slot(offsets, n, lo + min(i, left - 1), per, shift) <= slot;
        // as a signed number: none begins before a slot in front of the first segment
        const int owned = (int)__popcll(__builtin_amdgcn_ballot_w64(before)), k = owned > 0 ? owned - 1 : 0;
        lo += k * step;
        left = min(step, left - k * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Which piece of work is this workgroup's. Workgroups go to the eight XCDs in turn; each XCD takes `turn` consecutive pieces, then the
// next eight turns follow: neighbours, which read the same keys (or rows), share an L2, and segments of different lengths are still
// spread over all of them. (16 ragged segments of up to 2047 rows and 1500 keys, 12 heads of 64 channels: 120 us, and 149 with one eighth
// of all pieces to each XCD, which leaves the XCDs of the short segments idle.)
__device__ __forceinline__ uint32_t piece_of(uint32_t turn)
{
    const uint32_t i = blockIdx.x >> 3, round = i / turn;
    return (round * 8 + (blockIdx.x & 7)) * turn + (i - round * turn);
}

// Rows of one head in LDS: row-major, the 16-byte pieces of a row xor-swizzled by the row, so that neither 16 rows read at one
// piece nor the four rows x 64 bytes of a transposing read meet in a bank (256 bytes of them).
template <int D>
struct Tile {
    static constexpr int NC = D / 8;              // 16-byte pieces of a row
    static constexpr int ROWB = D * 2;            // bytes of a row
    static constexpr int BYTES = 32 * ROWB;       // of a tile of 32 rows
    static constexpr int KS = D / 16;             // steps of a product over the channels
    static constexpr int MT = D <= 32 ? 1 : D / 32;   // blocks of 32 channels
    static __device__ __forceinline__ int swizzle(int row)
    {
        if (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
        if (D == 64) return ((row & 2) << 1) | ((row >> 2) & 3);
        if (D == 32) return (row >> 2) & 3;
        return (row >> 3) & 1;
    }
    // byte offset of channels 16 ks + 8 hf .. of row l32: an operand whose rows are the tile's
    static __device__ __forceinline__ uint32_t row_piece(int lane, int ks)
    {
        const int l32 = lane & 31, hf = lane >> 5;
        return l32 * ROWB + (((2 * ks + hf) ^ swizzle(l32)) << 4);
    }
    // The transposing read that delivers X^T (rows: channels, k: the tile's rows in the order of the score registers). In a group
    // of 16 lanes lane 4 j + c hands in the address of channels 4 c .. 4 c + 3 of row 4 hf + j, and of rows 8, 16, 24 further on: the
    // swizzle of a row 8 further on differs in one bit, 16 further on it is the same. At 16 channels the second group of 16
    // lanes repeats the first: the result rows it feeds are never read.
    static __device__ __forceinline__ uint32_t transposed(int lane)
    {
        const int i16 = lane & 15, j = i16 >> 2, c = i16 & 3, g16 = (lane >> 4) & 1, hf = lane >> 5;
        const int row = 4 * hf + j, piece = (D == 16 ? 0 : 2 * g16) + (c >> 1);
        return row * ROWB + ((piece ^ swizzle(row)) << 4) + (c & 1) * 8;
    }
    static constexpr uint32_t FLIP = D == 16 ? 16 : 32;   // of the address, for rows 8 and 24 further on
};

// X^T of channels 32 mt .. of the tile whose transposed() address is `at` (with `flip` = at ^ FLIP)
template <int D>
__device__ __forceinline__ void read_transposed(U4& x0, U4& x1, uint32_t at, uint32_t flip, int mt)
{
    constexpr int STEP = 8 * Tile<D>::ROWB;
    const uint32_t a = at ^ (mt * 64), f = flip ^ (mt * 64);
    const uint2 y0 = lds_read_tr(a), y1 = lds_read_tr(f + STEP), y2 = lds_read_tr(a + 2 * STEP), y3 = lds_read_tr(f + 3 * STEP);
    x0.u = make_uint4(y0.x, y0.y, y1.x, y1.y);
    x1.u = make_uint4(y2.x, y2.y, y3.x, y3.y);
}

// Rows [0, from) and [to, n) of a tensor, which no segment owns, get zeros from all workgroups of the grid's first dimension together; there
// are none as a rule
__device__ __forceinline__ void zero_rows(uint16_t* x, int n, int from, int to, uint32_t row_bytes)
{
    if (from == 0 && to == n) return;
    const long long head = (long long)min(from, to) * row_bytes / 16, tail = (long long)to * row_bytes / 16, all = (long long)n * row_bytes / 16;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < head + all - tail; i += (long long)gridDim.x * blockDim.x)
        reinterpret_cast<uint4*>(x)[i < head ? i : tail + (i - head)] = make_uint4(0, 0, 0, 0);
}

constexpr int vm_wait(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }   // s_waitcnt operand: the memory counter alone

// Keys and values in LDS for the kernels whose waves own query rows: stages of ROWS keys, NBUF of them resident. At 128 channels a stage
// is one tile, so that two workgroups fit on a compute unit; loops go over two of them then (LOOP: stages, together an even number of tiles).
template <int D>
struct RowStage {
    using T = Tile<D>;
    static constexpr int ROWS = D == 16 ? 128 : D == 128 ? 32 : 64;
    static constexpr int TILES = ROWS / 32;
    static constexpr int LOOP = TILES == 1 ? 2 : 1;
    static constexpr int BYTES = ROWS * T::ROWB;      // of K, and of V
    static constexpr int NBUF = D == 32 || D == 128 ? 4 : 3;
    static constexpr int LPW = ROWS * T::NC / 256;    // loads per lane, stage and tensor
    static constexpr int TOTAL = NBUF * 2 * BYTES;
};

// The keys of a workgroup of four waves on their way through LDS: K of buffer b at b BYTES from `lds` on, V NBUF BYTES further on. Where
// they fit they are staged once and stay; else stage after stage, over and over for the row blocks of a run, each NBUF - 1 stages
// before it is read.
template <int D>
struct KeyRing {
    using T = Tile<D>;
    using S = RowStage<D>;
    const char* k;
    const char* v;
    uint32_t lds, row_bytes;
    int nkeys, nst, total, asked, next, wave;         // total, asked: stages over all row blocks; next: the keys of the one to ask for
    bool stays;
    int srow[S::LPW];
    uint32_t scol[S::LPW];

    __device__ __forceinline__ void start(const uint16_t* keys, const uint16_t* values, uint64_t first, uint32_t pitch, int n, int blocks, uint32_t at, int w)
    {
        k = reinterpret_cast<const char*>(keys) + first;
        v = reinterpret_cast<const char*>(values) + first;
        lds = at;
        row_bytes = pitch;
        nkeys = n;
        wave = w;
        nst = (n + S::ROWS - 1) / S::ROWS;
        stays = nst <= S::NBUF;
        total = stays ? nst : nst * blocks;
        asked = next = 0;
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < S::LPW; ++i) {
            const int p = (wave * S::LPW + i) * 64 + lane;
            srow[i] = p / T::NC;
            scol[i] = ((p % T::NC) ^ T::swizzle(srow[i])) << 4;
        }
        fill(0, stays ? S::NBUF : S::NBUF - 1);
    }
    __device__ __forceinline__ void request(int buf)
    {
#pragma unroll
        for (int i = 0; i < S::LPW; ++i) {
            const int key = min(next * S::ROWS + srow[i], nkeys - 1);   // past the end: the last key again
            const uint64_t at = (uint64_t)(uint32_t)key * row_bytes + scol[i];
            const uint32_t to = lds + buf * S::BYTES + (wave * S::LPW + i) * 1024;
            lds_dma16(k + at, to);
            lds_dma16(v + at, to + S::NBUF * S::BYTES);
        }
        ++asked;
        next = next + 1 == nst ? 0 : next + 1;
    }
    // the next `n` stages, as far as there are any, to the buffers from `buf` on
    __device__ __forceinline__ void fill(int buf, int n)
    {
        for (int i = 0; i < n && asked < total; ++i) {
            request(buf);
            buf = buf + 1 == S::NBUF ? 0 : buf + 1;
        }
    }
    // In the last tile of the stage in buffer `buf`, `read` stages before it: the next one is handed over to the readers, and the buffer
    // of the one before this is asked for again. Whoever arrives has its own loads of the next stage and has read the one before this.
    __device__ __forceinline__ void hand_over(int buf, int read)
    {
        if (S::NBUF > 3 && asked - read > 1) __builtin_amdgcn_s_waitcnt(vm_wait((S::NBUF - 3) * 2 * S::LPW));   // but the stages behind it
        else __builtin_amdgcn_s_waitcnt(vm_wait(0));
        __syncthreads();
        if (asked < total) request(buf == 0 ? S::NBUF - 1 : buf - 1);
    }
};

}  // namespace

}  // namespace f3d
