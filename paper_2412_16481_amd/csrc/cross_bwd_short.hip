// Cross attention backward for few keys beside many rows (the points of a scan and a prompt): up to 128 keys a segment, head_dim 16 and 32.
// There every wave can hold the gradients of ALL keys of a (segment, key/value head) in registers, so a row is looked at once: scores,
// exponentials and dP serve dq, dk and dv together, where the two kernels of cross_bwd.hip work them out twice.
//
// K and V stay in LDS. A wave takes tiles of 32 rows; Q and dO of the next tile are on their way into its own part of LDS meanwhile
// (no barrier but the one behind the keys). Per tile of 32 keys, scores transposed (keys x rows, a lane owns 16 keys of ONE row):
//   S^T = K Q^T,  dP^T = V dO^T - D  (the accumulator starts from -D),  P = 2^(S mul - lse),  dS = P o dP,
//   dQ^T += K^T dS^T                 dS^T, packed to bf16, is the B operand as it lies,
//   dV^T += dO^T P, dK^T += Q^T dS   P and dS go through LDS (32 x 32 each) and come back transposed: a lane then owns one KEY, and the rows
//                                    are in the order in which the transposing read delivers Q^T and dO^T.
// The waves of a workgroup add up their sums at the end, in order; a segment's rows are split over workgroups whose sums the join of
// cross_bwd.hip adds up. Bound: the vector ALU's issue port (exponentials, packing) and LDS. 200000 rows, 77 keys, 4 x 16 channels: 44 us
// with the join, where the two kernels of cross_bwd.hip take 93. 128 keys of 32 channels would need more registers and LDS than two workgroups have.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cross_common.h"

namespace f3d {

namespace {

constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ f32x16 mfma(const U4& x, const U4& y, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.b, y.b, c, 0, 0, 0);
}

// A 32 x 32 tile of bf16 in LDS, 64 bytes a row, its 8-byte pieces xor-swizzled by the row: 32 rows written at one piece fall on
// different banks, and so do the four rows of a transposing read.
struct Square {
    static __device__ __forceinline__ uint32_t at(int row, int piece) { return row * 64 + ((piece ^ ((row >> 2) & 7)) << 3); }
};

__device__ __forceinline__ void lds_write8(uint32_t addr, uint32_t x, uint32_t y)
{
    const u32x2 v = {x, y};
    *(__attribute__((address_space(3))) u32x2*)(uintptr_t)addr = v;
}

// one 4-byte global -> LDS load per lane, as lds_dma16
__device__ __forceinline__ void lds_dma4(const void* g, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(g) : "memory", "m0");
}

template <int D, int NT>   // NT: tiles of 32 keys
__global__ __launch_bounds__(256, 2) void k_cross_bwd_short(CrossBwdArgs b)
{
    using T = Tile<D>;
    constexpr int KS = T::KS;
    static_assert(T::MT == 1, "one block of channels");
    constexpr int KEYS = 32 * NT, KBYTES = KEYS * T::ROWB, LPT = T::BYTES / 1024;   // loads per lane, row tile and tensor
    constexpr int NB = 2;                             // row tiles in LDS: the one at work and the next ones on their way
    constexpr int STORES = D == 16 ? 2 : 4;           // of a row tile's dq
    constexpr int MEET = 4 * KEYS * D * 4;            // one gradient's sums of the four waves
    constexpr int LSE = NB * 3 * T::BYTES, SQUARES = LSE + NB * 128;   // a wave's LDS: Q, dO, O of its row tiles, their lse, a key tile's P and dS
    constexpr int OWN = SQUARES + 4096;
    constexpr int TOTAL = 2 * KBYTES + T::BYTES + 4 * OWN;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[TOTAL > MEET ? TOTAL : MEET];
    const CrossArgs& a = b.f;
    const uint32_t sK = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (blockIdx.y == 0) {
        // rows of no segment, of both tensors
        const int q0 = offset_of(a.q_offsets, a.n_q, 0), q1 = offset_of(a.q_offsets, a.n_q, a.segments);
        zero_rows(b.dq, a.n_q, q0, q1, (uint32_t)a.H * T::ROWB);
        if (b.row_parts == 1) {
            const int k0 = offset_of(a.kv_offsets, a.n_kv, 0), k1 = offset_of(a.kv_offsets, a.n_kv, a.segments);
            zero_rows(b.dk, a.n_kv, k0, k1, (uint32_t)a.K * T::ROWB);
            zero_rows(b.dv, a.n_kv, k0, k1, (uint32_t)a.K * T::ROWB);
        }
    }
    // (part, key/value head) and the segment: the heads of the same rows, which share their lines, on one XCD (a row of the grid is whole turns)
    const uint32_t u = piece_of((uint32_t)a.K);
    const int part = (int)(u / (uint32_t)a.K), kh = (int)(u - (uint32_t)part * a.K), seg = blockIdx.y;
    if (part >= b.row_parts) return;
    const Rows qs = rows_of(a.q_offsets, a.q_lens, a.n_q, seg), kv = rows_of(a.kv_offsets, a.kv_lens, a.n_kv, seg);
    const int rows = qs.span * a.G, live = qs.len * a.G;
    const int row0 = part * b.row_chunk, row1 = min(rows, row0 + b.row_chunk);   // this workgroup's, some of them behind the segment's length
    const int nkeys = min(kv.len, KEYS), span = min(kv.span, KEYS);
    const uint32_t sV = sK + KBYTES, own = sV + KBYTES + T::BYTES + wave * OWN, square = own + SQUARES;

    // ---- keys and values
    if (nkeys > 0 && row0 < live) {
        const uint32_t row_bytes = (uint32_t)a.K * T::ROWB;
        const uint64_t first = (uint64_t)kv.from * row_bytes + (uint64_t)kh * T::ROWB;
#pragma unroll
        for (int i = 0; i < (KEYS * T::NC + 255) / 256; ++i) {
            const int blk = wave + 4 * i, p = blk * 64 + lane, key = p / T::NC;
            if (blk * 64 >= KEYS * T::NC) break;      // wave-uniform
            const uint64_t at = first + (uint64_t)(uint32_t)min(key, nkeys - 1) * row_bytes + (((p % T::NC) ^ T::swizzle(key & 31)) << 4);
            lds_dma16(reinterpret_cast<const char*>(a.k) + at, sK + blk * 1024);
            lds_dma16(reinterpret_cast<const char*>(a.v) + at, sV + blk * 1024);
        }
    }
    // ---- a tile of rows to this wave's LDS. Tiles past the end are asked for all the same (of the last row that counts): the number
    //      of loads behind a tile is then always the same
    const auto place_of = [&](int row) __attribute__((always_inline)) {
        const int i = divide(row, a.G, a.by_g), g = row - i * a.G;
        return (uint32_t)(qs.from + i) * (uint32_t)a.H + (uint32_t)(kh * a.G + g);
    };
    constexpr int LOADS = 3 * LPT + 1;
    auto request = [&](int r0, int buf) __attribute__((always_inline)) {
        const uint32_t to = own + buf * 3 * T::BYTES;
#pragma unroll
        for (int i = 0; i < LPT; ++i) {
            const int p = i * 64 + lane, r = p / T::NC;
            const uint64_t at = (uint64_t)place_of(min(r0 + r, live - 1)) * T::ROWB + (((p % T::NC) ^ T::swizzle(r)) << 4);
            lds_dma16(reinterpret_cast<const char*>(a.q) + at, to + i * 1024);
            lds_dma16(reinterpret_cast<const char*>(b.dout) + at, to + T::BYTES + i * 1024);
            lds_dma16(reinterpret_cast<const char*>(a.out) + at, to + 2 * T::BYTES + i * 1024);
        }
        if (lane < 32) lds_dma4(a.lse + place_of(min(r0 + lane, live - 1)), own + LSE + buf * 128);
    };
    const int r_first = row0 + wave * 32, live1 = nkeys > 0 ? min(row1, live) : 0;
    if (r_first < live1) {
#pragma unroll
        for (int i = 0; i < NB - 1; ++i) request(r_first + 128 * i, i);
    }
    __builtin_amdgcn_s_waitcnt(vm_wait(0));
    __syncthreads();

    // Keys past the end repeat the last one: their scores are as good as any, and of what they add to dk and dv nothing is stored. For dq the
    // tile that is not full has a copy in which they are zeros.
    if (nkeys & 31) {
        const int first = nkeys & ~31;
        for (int p = tid; p < 32 * T::NC; p += 256) {
            const uint4 x = lds_read16(sK + first * T::ROWB + p * 16);
            const bool in = first + p / T::NC < nkeys;
            lds_write8(sK + 2 * KBYTES + p * 16, in ? x.x : 0u, in ? x.y : 0u);
            lds_write8(sK + 2 * KBYTES + p * 16 + 8, in ? x.z : 0u, in ? x.w : 0u);
        }
        __syncthreads();
    }

    f32x16 dk[NT], dv[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) dk[j] = dv[j] = f32x16{0};
    uint32_t off[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) off[ks] = T::row_piece(lane, ks);
    const uint32_t tr = T::transposed(lane);
    uint32_t put[4], get[4];                          // of the squares
    {
        const int i16 = lane & 15, jj = i16 >> 2, c = i16 & 3, g16 = (lane >> 4) & 1;
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            put[r4] = square + Square::at(l32, 2 * r4 + hf);                       // keys 8 r4 + 4 hf .. of row l32
            get[r4] = square + Square::at(4 * hf + jj + 8 * r4, 4 * g16 + c);      // keys 16 g16 + 4 c .. of that row
        }
    }
    const float mul = a.s_mul;
    int buf = 0;
    for (int r0 = r_first; r0 < live1; r0 += 128, buf = buf + 1 == NB ? 0 : buf + 1) {
        const int row = r0 + l32;
        // this tile has landed once only what was asked for and stored since is outstanding
        __builtin_amdgcn_s_waitcnt(vm_wait((NB - 2) * LOADS + (NB - 1) * STORES));
        asm volatile("" ::: "memory");
        request(r0 + 128 * (NB - 1), buf == 0 ? NB - 1 : buf - 1);   // over the tile before this one
        const uint32_t sQ = own + buf * 3 * T::BYTES, sG = sQ + T::BYTES, sO = sG + T::BYTES;
        U4 qf[KS], gf[KS], xq[2], xg[2];
        float dot = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[ks].u = lds_read16(sQ + off[ks]);
            gf[ks].u = lds_read16(sG + off[ks]);
        }
        read_transposed<D>(xq[0], xq[1], sQ + tr, (sQ + tr) ^ T::FLIP, 0);
        read_transposed<D>(xg[0], xg[1], sG + tr, (sG + tr) ^ T::FLIP, 0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            U4 of;
            of.u = lds_read16(sO + off[ks]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t y = (&of.u.x)[e], z = (&gf[ks].u.x)[e];
                dot += __uint_as_float(y << 16) * __uint_as_float(z << 16);
                dot += __uint_as_float(y & 0xFFFF0000u) * __uint_as_float(z & 0xFFFF0000u);
            }
        }
        dot += __shfl_xor(dot, 32, 64);
        // made opaque, so that what the keys' addresses and the mask of the last tile are worked out from is not kept for all tiles at once
        uint32_t keys = sK;
        int nk = nkeys;
        asm volatile("" : "+s"(keys), "+s"(nk));
        const float lse = *(const __attribute__((address_space(3))) float*)(uintptr_t)(own + LSE + buf * 128 + l32 * 4);
        const float nl = row < live ? -LOG2E * lse : -INFINITY;   // rows that take no part: probabilities exactly zero
        f32x16 minus_d, dq = f32x16{0}, s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) minus_d[r] = -dot;

        // The key tiles follow each other one step apart: between the exponentials of tile j stand the products of tile j + 1 and the
        // gradients from P and dS of tile j - 1, which are back from LDS by then.
        f32x16 sn, dpn;
        U4 y[4];
        auto gradients = [&](int j, int half) __attribute__((always_inline)) {
            dv[j] = mfma(xg[half], y[half], dv[j]);
            dk[j] = mfma(xq[half], y[2 + half], dk[j]);
        };
        auto turned = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {             // P, then dS 2 KB further on
                const uint32_t at = (h >> 1) * 2048;
                const uint2 lo = lds_read_tr(get[2 * (h & 1)] + at), hi = lds_read_tr(get[2 * (h & 1) + 1] + at);
                y[h].u = make_uint4(lo.x, lo.y, hi.x, hi.y);
            }
        };
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            U4 kf, vf;
            kf.u = lds_read16(keys + off[ks]);
            vf.u = lds_read16(keys + off[ks] + KBYTES);
            s = mfma(kf, qf[ks], ks == 0 ? f32x16{0} : s);
            dp = mfma(vf, gf[ks], ks == 0 ? minus_d : dp);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            U4 p0, p1, d0, d1, k0, k1, kf[KS], vf[KS];
            const auto prob = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
                for (int r = r0; r < r0 + 4; ++r) {
                    s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], mul, nl));
                    dp[r] *= s[r];
                }
            };
            if (j + 1 < NT) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    kf[ks].u = lds_read16(keys + off[ks] + (j + 1) * T::BYTES);
                    vf[ks].u = lds_read16(keys + off[ks] + (KBYTES + (j + 1) * T::BYTES));
                }
            }
            if (j > 0) turned();
            F3D_SB();
            prob(0);
            F3D_SB();
            if (j + 1 < NT) {
                sn = mfma(kf[0], qf[0], f32x16{0});
                dpn = mfma(vf[0], gf[0], minus_d);
            }
            F3D_SB();
            prob(4);
            F3D_SB();
            if (j + 1 < NT && KS == 2) {
                sn = mfma(kf[KS - 1], qf[KS - 1], sn);
                dpn = mfma(vf[KS - 1], gf[KS - 1], dpn);
            }
            if (j > 0) gradients(j - 1, 0);
            F3D_SB();
            prob(8);
            F3D_SB();
            if (j > 0) gradients(j - 1, 1);
            F3D_SB();
            const uint32_t kt = 32 * j + 32 > nk ? keys + 2 * KBYTES : keys + j * T::BYTES;
            read_transposed<D>(k0, k1, kt + tr, (kt + tr) ^ T::FLIP, 0);
            prob(12);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                (&p0.u.x)[e] = pack_bf16(s[2 * e], s[2 * e + 1]);
                (&p1.u.x)[e] = pack_bf16(s[8 + 2 * e], s[8 + 2 * e + 1]);
                (&d0.u.x)[e] = pack_bf16(dp[2 * e], dp[2 * e + 1]);
                (&d1.u.x)[e] = pack_bf16(dp[8 + 2 * e], dp[8 + 2 * e + 1]);
            }
            asm volatile("" ::: "memory");            // a wave's LDS operations take place in their order
            lds_write8(put[0], p0.u.x, p0.u.y);
            lds_write8(put[1], p0.u.z, p0.u.w);
            lds_write8(put[2], p1.u.x, p1.u.y);
            lds_write8(put[3], p1.u.z, p1.u.w);
            lds_write8(put[0] + 2048, d0.u.x, d0.u.y);
            lds_write8(put[1] + 2048, d0.u.z, d0.u.w);
            lds_write8(put[2] + 2048, d1.u.x, d1.u.y);
            lds_write8(put[3] + 2048, d1.u.z, d1.u.w);
            asm volatile("" ::: "memory");
            F3D_SB();
            if (32 * j < nk) {
                dq = mfma(k0, d0, dq);
                dq = mfma(k1, d1, dq);
            }
            F3D_SB();
            s = sn;
            dp = dpn;
        }
        turned();
        gradients(NT - 1, 0);
        gradients(NT - 1, 1);
        asm volatile("" ::: "memory");
        if (row < live1) {
            uint16_t* const to = b.dq + (size_t)place_of(row) * D;
#pragma unroll
            for (int r4 = 0; r4 < STORES; ++r4)
                *reinterpret_cast<uint2*>(to + 8 * r4 + 4 * hf) = make_uint2(pack_bf16(dq[4 * r4] * b.scale, dq[4 * r4 + 1] * b.scale),
                                                                            pack_bf16(dq[4 * r4 + 2] * b.scale, dq[4 * r4 + 3] * b.scale));
        }
    }
    // rows behind the segment's length, or without keys
    for (int row = max(row0, live1) + wave * 32 + l32; row < row1; row += 128) {
        uint16_t* const to = b.dq + (size_t)place_of(row) * D;
#pragma unroll
        for (int r4 = 0; r4 < STORES; ++r4) *reinterpret_cast<uint2*>(to + 8 * r4 + 4 * hf) = make_uint2(0, 0);
    }

    // ---- the four waves' sums, added in order, dk and then dv, through the LDS that all have left
    float* const meet = reinterpret_cast<float*>(smem);   // [4][KEYS][D]
    __builtin_amdgcn_s_waitcnt(vm_wait(0));           // nothing is on its way there any more
    const size_t all = (size_t)a.n_kv * a.K * D;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const f32x16& x = which ? dv[j] : dk[j];
#pragma unroll
            for (int r4 = 0; r4 < STORES; ++r4)
                *reinterpret_cast<float4*>(meet + ((wave * KEYS + 32 * j + l32) * D + 8 * r4 + 4 * hf)) =
                    make_float4(x[4 * r4], x[4 * r4 + 1], x[4 * r4 + 2], x[4 * r4 + 3]);
        }
        __syncthreads();
        for (int i = tid; i < span * (D / 4); i += 256) {
            const int key = i / (D / 4), c = (i % (D / 4)) * 4;
            const size_t at = ((size_t)(kv.from + key) * a.K + kh) * D + c;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            if (key < nkeys) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float4 x = *reinterpret_cast<const float4*>(meet + ((w * KEYS + key) * D + c));
                    y = make_float4(y.x + x.x, y.y + x.y, y.z + x.z, y.w + x.w);
                }
            }
            const float m = which ? 1.0f : b.scale;
            y = make_float4(y.x * m, y.y * m, y.z * m, y.w * m);
            if (b.row_parts > 1) *reinterpret_cast<float4*>(b.part_dkv + ((size_t)which * b.row_parts + part) * all + at) = y;
            else *reinterpret_cast<uint2*>((which ? b.dv : b.dk) + at) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
        }
    }
}

template <int D>
hipError_t launch(const CrossBwdArgs& b, int tiles, hipStream_t stream)
{
    const dim3 grid(cross_grid(b.row_parts, b.f.K, b.f.K), (unsigned)b.f.segments);
    switch (tiles) {
        case 1: k_cross_bwd_short<D, 1><<<grid, 256, 0, stream>>>(b); break;
        case 2: k_cross_bwd_short<D, 2><<<grid, 256, 0, stream>>>(b); break;
        case 3: k_cross_bwd_short<D, 3><<<grid, 256, 0, stream>>>(b); break;
        default:
            if constexpr (D == 16) k_cross_bwd_short<D, 4><<<grid, 256, 0, stream>>>(b);
            else return hipErrorInvalidValue;         // registers and LDS
    }
    return hipGetLastError();
}

}  // namespace

hipError_t cross_bwd_short_launch(const CrossBwdArgs& b, int head_dim, int tiles, hipStream_t stream)
{
    if (tiles < 1 || tiles > 4) return hipErrorInvalidValue;
    switch (head_dim) {
        case 16: return launch<16>(b, tiles, stream);
        case 32: return launch<32>(b, tiles, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace f3d
