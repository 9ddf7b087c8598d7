// Layer norm over the channels of every row, forward and backward (Section 4.2, block equations: LN in front of the attention and
// of the MLP), with the row gather that puts rows into bucket-major order.
//
//   forward   y[p] = (x[r] - mu_p) rs_p gamma + beta,  r = row_in[p],  rs_p = 1 / sqrt(var_p + eps)
//   backward  xh = (x[r] - mu_p) rs_p,  g = dy[p] gamma,
//             dx[r] = rs_p (g - mean(g) - xh mean(g xh)) + residual[r],
//             dgamma = sum_p dy[p] xh,  dbeta = sum_p dy[p]
//
// A team of 8 to 256 threads holds one row in registers, up to 32 elements each, so a row is read once: the forward takes the mean
// and then the squares about it, both from the registers (sums of x and x^2 side by side would cancel where a row's mean is large).
// The backward's teams keep their columns from row to row, so the sums of the weights' gradients stay in registers
// too; a workgroup adds up its teams at its end and leaves 2 c sums in the workspace, which a second launch adds up in a fixed
// order: the same call gives the same bits.
//
// Bound: HBM. Measured: 914601 rows of 256 bfloat16 channels forward 176 us = 5.3 TB/s, backward with a residual and the weights' gradients
// 381 us = 4.9 TB/s; 9001 rows of 1537 binary32 channels, which begin at no multiple of 16 bytes, backward 41 us = 4.0 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "elem.h"
#include "norm.h"

namespace f3d {

namespace {

constexpr int NTH = 256;      // threads of a workgroup
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// Sum over the TPR threads of a team, in every one of them. A team of a whole workgroup joins its waves through LDS: `box` is
// written again only behind the next barrier of the next sum, so two boxes taken in turn need one barrier a sum.
template <int TPR>
__device__ __forceinline__ float team_sum(float v, float* box)
{
#pragma unroll
    for (int d = 1; d < (TPR < 64 ? TPR : 64); d *= 2) v += __shfl_xor(v, d, 64);
    if (TPR <= 64) return v;
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = v;
    __syncthreads();
    return (box[0] + box[1]) + (box[2] + box[3]);
}

template <int TPR>
__device__ __forceinline__ float2 team_sum2(float v, float w, float* box)
{
#pragma unroll
    for (int d = 1; d < (TPR < 64 ? TPR : 64); d *= 2) {
        v += __shfl_xor(v, d, 64);
        w += __shfl_xor(w, d, 64);
    }
    if (TPR <= 64) return make_float2(v, w);
    if ((threadIdx.x & 63) == 0) {
        box[threadIdx.x >> 6] = v;
        box[4 + (threadIdx.x >> 6)] = w;
    }
    __syncthreads();
    return make_float2((box[0] + box[1]) + (box[2] + box[3]), (box[4] + box[5]) + (box[6] + box[7]));
}

// A row cut into 16-byte pieces: so many whole ones, and the elements behind them.
struct Cut {
    int pieces, rest;
};

// 16, 8 and 4 bytes at the alignment of 16-bit elements
typedef u32x4 loose16 __attribute__((aligned(2)));
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef u32x2 loose8 __attribute__((aligned(2)));
typedef uint32_t loose4 __attribute__((aligned(2)));
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef f32x4 loose_f32x4 __attribute__((aligned(4)));

// A thread's part of a row: pieces t, t + TPR, .. of W elements. What is past the row's end counts as zeros. WIDE: every row begins at a
// multiple of 16 bytes and is whole pieces. Other rows are moved 16 bytes at a time as well, at whatever address they have; of what
// is left at the end 16 bytes are read and 8, 4 and 2 written. 100000 rows of 1537 bfloat16 channels forward 170 us, backward 234; element
// by element 370 and 671 (20000 of 4001 binary32 channels 124 and 189; 150 and 273).
template <int TYPE, bool WIDE, int TPR, int V>
struct Part {
    using E = Elems<TYPE>;
    using one = typename E::one;
    static constexpr int W = E::W;
    static constexpr int N = V * W;                   // elements of a thread
    static constexpr int PER = 4 / (int)sizeof(one);  // elements of four bytes
    using piece = typename std::conditional<WIDE, u32x4, loose16>::type;

    static __device__ __forceinline__ Cut cut(int c) { return {c / W, WIDE ? 0 : c % W}; }
    // elements [0, W) of piece v of this thread that the row has
    static __device__ __forceinline__ int has(Cut cut, int t, int v)
    {
        const int i = t + v * TPR;
        return i < cut.pieces ? W : !WIDE && i == cut.pieces ? cut.rest : 0;
    }
    static __device__ __forceinline__ uint4 load_rest(const one* at, int rest)
    {
        const uint32_t* const p = reinterpret_cast<const uint32_t*>(at);
        const int words = rest / PER;
        uint4 u = make_uint4(0, 0, 0, 0);
        if (words & 2) {
            const u32x2 y = *reinterpret_cast<const loose8*>(p);
            u.x = y.x;
            u.y = y.y;
        }
        if (words & 1) (words & 2 ? u.z : u.x) = *reinterpret_cast<const loose4*>(p + (words & 2));
        if (PER == 2 && (rest & 1)) (words == 0 ? u.x : words == 1 ? u.y : words == 2 ? u.z : u.w) = *reinterpret_cast<const uint16_t*>(p + words);
        return u;
    }
    static __device__ __forceinline__ void store_rest(one* at, int rest, const uint4& u)
    {
        uint32_t* const p = reinterpret_cast<uint32_t*>(at);
        const int words = rest / PER;
        if (words & 2) {
            const u32x2 y = {u.x, u.y};
            *reinterpret_cast<loose8*>(p) = y;
        }
        if (words & 1) *reinterpret_cast<loose4*>(p + (words & 2)) = words & 2 ? u.z : u.x;
        if (PER == 2 && (rest & 1)) *reinterpret_cast<uint16_t*>(p + words) = (uint16_t)(words == 0 ? u.x : words == 1 ? u.y : words == 2 ? u.z : u.w);
    }
    // the piece without its first `drop` elements, zeros behind
    static __device__ __forceinline__ uint4 dropped(uint4 u, int drop)
    {
        const int words = drop / PER;
        if (words & 2) u = make_uint4(u.z, u.w, 0, 0);
        if (words & 1) u = make_uint4(u.y, u.z, u.w, 0);
        if (PER == 2 && (drop & 1)) u = make_uint4(u.x >> 16 | u.y << 16, u.y >> 16 | u.z << 16, u.z >> 16 | u.w << 16, u.w >> 16);
        return u;
    }
    // The last piece of a row that is no whole pieces is read as the row's last 16 bytes, so that every thread has one load a piece
    static __device__ __forceinline__ void load(const one* row, int t, Cut cut, float (&x)[N])
    {
        const bool shorter = !WIDE && cut.pieces == 0;   // than one piece
        uint4 u[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = t + v * TPR;
            u[v] = make_uint4(0, 0, 0, 0);
            if (i < cut.pieces + (cut.rest != 0) && !shorter) {
                const int at = WIDE || i < cut.pieces ? i * W : i * W - (W - cut.rest);
                const u32x4 y = *reinterpret_cast<const piece*>(row + at);
                u[v] = make_uint4(y.x, y.y, y.z, y.w);
            }
        }
        if (shorter && t == 0 && cut.rest != 0) u[0] = load_rest(row, cut.rest);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!WIDE && cut.rest != 0 && !shorter && t + v * TPR == cut.pieces) u[v] = dropped(u[v], W - cut.rest);
            E::unpack(u[v], *reinterpret_cast<float(*)[W]>(x + v * W));
        }
    }
    template <bool STREAMED = false>
    static __device__ __forceinline__ void store(one* row, int t, Cut cut, const float (&x)[N])
    {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint4 u = E::pack(*reinterpret_cast<const float(*)[W]>(x + v * W));
            if (t + v * TPR < cut.pieces) {
                const u32x4 y = {u.x, u.y, u.z, u.w};
                piece* const to = reinterpret_cast<piece*>(row) + t + v * TPR;
                if (STREAMED) __builtin_nontemporal_store(y, to);
                else *to = y;
            } else if (!WIDE && t + v * TPR == cut.pieces) {
                store_rest(row + cut.pieces * W, cut.rest, u);
            }
        }
    }
    // the row's weights, `none` where there are none
    static __device__ __forceinline__ void weights(const float* w, float none, int t, Cut cut, float (&x)[N])
    {
        using four = typename std::conditional<WIDE, f32x4, loose_f32x4>::type;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float* const at = w + (t + v * TPR) * W;
            const int n = has(cut, t, v);
#pragma unroll
            for (int e = 0; e < W; ++e) x[v * W + e] = none;
            if (!w) continue;
            if (n == W) {
#pragma unroll
                for (int e = 0; e < W; e += 4) {
                    const f32x4 f = *reinterpret_cast<const four*>(at + e);
                    x[v * W + e] = f.x;
                    x[v * W + e + 1] = f.y;
                    x[v * W + e + 2] = f.z;
                    x[v * W + e + 3] = f.w;
                }
            } else if (!WIDE) {
#pragma unroll
                for (int e = 0; e < W - 1; ++e)
                    if (e < n) x[v * W + e] = at[e];
            }
        }
    }
};

// R rows a team, all requested before the first is looked at. STREAMED: results past the caches, from 4 MB on. 914601
// rows of 256 bfloat16 channels: 178 us with both, 259 with one row a team and cached results
template <int TYPE, bool WIDE, int TPR, int V, int R, bool STREAMED>
__global__ __launch_bounds__(NTH) void k_norm(NormArgs a)
{
    using P = Part<TYPE, WIDE, TPR, V>;
    using one = typename P::one;
    constexpr int TEAMS = NTH / TPR;
    __shared__ float box[2 * R][8];
    const int t = threadIdx.x % TPR;
    const long long first = (long long)blockIdx.x * (TEAMS * R) + threadIdx.x / TPR;
    const Cut cut = P::cut(a.c);
    size_t r[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const long long p = min(first + k * TEAMS, (long long)a.n - 1);   // past the end: the last row again, which is not stored
        r[k] = (size_t)(a.row_in ? a.row_in[p] : p);
    }
    float x[R][P::N];
#pragma unroll
    for (int k = 0; k < R; ++k) P::load(static_cast<const one*>(a.x) + r[k] * a.c, t, cut, x[k]);
    float g[P::N], b[P::N];
    P::weights(a.gamma, 1.f, t, cut, g);
    P::weights(a.beta, 0.f, t, cut, b);
    const float inv = 1.0f / a.c;
    float mu[R], rs[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < P::N; ++i) s += x[k][i];
        mu[k] = team_sum<TPR>(s, box[k]) * inv;
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
        float q = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int n = P::has(cut, t, v);          // the zeros past the end are no elements
            if (n == 0) continue;
#pragma unroll
            for (int e = 0; e < P::W; ++e) {
                const float off = WIDE || e < n ? x[k][v * P::W + e] - mu[k] : 0.f;
                q += off * off;
            }
        }
        rs[k] = 1.0f / sqrtf(team_sum<TPR>(q, box[R + k]) * inv + a.eps);
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const long long p = first + k * TEAMS;
        if (p >= a.n) break;
#pragma unroll
        for (int i = 0; i < P::N; ++i) x[k][i] = (x[k][i] - mu[k]) * rs[k] * g[i] + b[i];
        P::template store<STREAMED>(static_cast<one*>(a.y) + (size_t)p * a.c, t, cut, x[k]);
        if (t == 0) {
            if (a.mean) a.mean[p] = mu[k];
            if (a.rstd) a.rstd[p] = rs[k];
        }
    }
}

// WEIGHTS: the sums of the weights' gradients are wanted
template <int TYPE, bool WIDE, int TPR, int V, int R, bool WEIGHTS, bool STREAMED>
__global__ __launch_bounds__(NTH) void k_norm_bwd(NormBwdArgs a)
{
    using P = Part<TYPE, WIDE, TPR, V>;
    using one = typename P::one;
    constexpr int TEAMS = NTH / TPR;
    __shared__ float box[2 * R][8];
    const int t = threadIdx.x % TPR;
    const Cut cut = P::cut(a.c);
    const float inv = 1.0f / a.c;
    float g[P::N], dg[P::N], db[P::N];
    P::weights(a.gamma, 1.f, t, cut, g);
#pragma unroll
    for (int i = 0; i < P::N; ++i) dg[i] = db[i] = 0.f;
    int turn = 0;
    for (long long first = (long long)blockIdx.x * (TEAMS * R) + threadIdx.x / TPR; first < a.n; first += (long long)gridDim.x * (TEAMS * R), turn ^= R) {
        size_t r[R];
        float x[R][P::N], dy[R][P::N], mu[R], rs[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const bool has = first + k * TEAMS < a.n;  // past the end: zeros
            const long long p = has ? first + k * TEAMS : 0;
            r[k] = (size_t)(has && a.row_in ? a.row_in[p] : p);
            mu[k] = has ? a.mean[p] : 0.f;
            rs[k] = has ? a.rstd[p] : 0.f;
            P::load(static_cast<const one*>(a.dy) + (size_t)p * a.c, t, has ? cut : Cut{0, 0}, dy[k]);
        }
#pragma unroll
        for (int k = 0; k < R; ++k) P::load(static_cast<const one*>(a.x) + r[k] * a.c, t, first + k * TEAMS < a.n ? cut : Cut{0, 0}, x[k]);
        float m1[R], m2[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int i = 0; i < P::N; ++i) {
                x[k][i] = (x[k][i] - mu[k]) * rs[k];  // past the row's end dy and with it every term is zero
                if (WEIGHTS) {
                    dg[i] += dy[k][i] * x[k][i];
                    db[i] += dy[k][i];
                }
                dy[k][i] *= g[i];
                s1 += dy[k][i];
                s2 += dy[k][i] * x[k][i];
            }
            const float2 s = team_sum2<TPR>(s1, s2, box[turn + k]);
            m1[k] = s.x * inv;
            m2[k] = s.y * inv;
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (first + k * TEAMS >= a.n) break;
#pragma unroll
            for (int i = 0; i < P::N; ++i) dy[k][i] = rs[k] * (dy[k][i] - m1[k] - x[k][i] * m2[k]);
            if (a.residual) {
                P::load(static_cast<const one*>(a.residual) + r[k] * a.c, t, cut, x[k]);
#pragma unroll
                for (int i = 0; i < P::N; ++i) dy[k][i] += x[k][i];
            }
            P::template store<STREAMED>(static_cast<one*>(a.dx) + r[k] * a.c, t, cut, dy[k]);
        }
    }
    if (!WEIGHTS) return;
    // one element of every thread at a time: the teams of a workgroup meet in LDS
    __shared__ float meet[2][NTH];
    // a workgroup that is alone has the whole sums
    float* const gamma_to = gridDim.x == 1 ? a.dgamma : a.part + (size_t)blockIdx.x * 2 * a.c;
    float* const beta_to = gridDim.x == 1 ? a.dbeta : a.part + ((size_t)blockIdx.x * 2 + 1) * a.c;
#pragma unroll
    for (int i = 0; i < P::N; ++i) {
        if (TEAMS > 1) {
            __syncthreads();
            meet[0][threadIdx.x] = dg[i];
            meet[1][threadIdx.x] = db[i];
            __syncthreads();
        }
        if (threadIdx.x < TPR) {
            float u = dg[i], w = db[i];
#pragma unroll
            for (int k = 1; k < TEAMS; ++k) {
                u += meet[0][k * TPR + t];
                w += meet[1][k * TPR + t];
            }
            const int col = (t + i / P::W * TPR) * P::W + i % P::W;
            if (col < a.c) {
                if (gamma_to) gamma_to[col] = u;
                if (beta_to) beta_to[col] = w;
            }
        }
    }
}

// The sums of `blocks` workgroups: 16 columns by 64 groups of workgroups at a time
__global__ __launch_bounds__(1024) void k_norm_bwd_join(const float* part, int blocks, int c, float* dgamma, float* dbeta)
{
    __shared__ float meet[64][17];
    const int col = blockIdx.x * 16 + (threadIdx.x & 15), k = threadIdx.x >> 4;
    float s = 0.f;
    if (col < 2 * c) {
#pragma unroll 16
        for (int b = k; b < blocks; b += 64) s += part[(size_t)b * 2 * c + col];
    }
    meet[k][threadIdx.x & 15] = s;
    __syncthreads();
    s = meet[threadIdx.x & 63][threadIdx.x >> 6];     // a wave has the 64 sums of one column
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d, 64);
    const int of = blockIdx.x * 16 + (threadIdx.x >> 6);
    if ((threadIdx.x & 63) == 0 && of < 2 * c) {
        float* const to = of < c ? dgamma : dbeta;
        if (to) to[of < c ? of : of - c] = s;
    }
}

constexpr size_t STREAMED_BYTES = (size_t)4 << 20;
// Passes over the rows that one workgroup takes by itself instead of leaving its sums to a second launch: 8 rows of 256 bfloat16 channels
// (one pass) 3.6 us against 6.1, 32 rows (four) 5.5 against 6.7, four rows of 1537 binary32 channels (four) 6.3 against 6.6.
constexpr int ALONE = 4;

struct Forward {
    const NormArgs& a;
    hipStream_t stream;
    template <int TYPE, bool WIDE, int TPR, int V>
    hipError_t go() const
    {
        constexpr int TEAMS = NTH / TPR;
        // four rows on their way a wave; two of a workgroup's where a thread has up to 16 of their 16-bit elements (40000 rows of 4096 127 -> 113 us)
        constexpr int R = TPR == 256 ? (TYPE != F3D_F32 && V <= 2 ? 2 : 1) : 4 / V;
        const long long steps = ((long long)a.n + TEAMS - 1) / TEAMS;
        if ((size_t)a.n * a.c * sizeof(typename Elems<TYPE>::one) >= STREAMED_BYTES)
            k_norm<TYPE, WIDE, TPR, V, R, true><<<(unsigned)((steps + R - 1) / R), NTH, 0, stream>>>(a);
        else
            k_norm<TYPE, WIDE, TPR, V, 1, false><<<(unsigned)steps, NTH, 0, stream>>>(a);
        return hipGetLastError();
    }
};

struct Backward {
    const NormBwdArgs& a;
    hipStream_t stream;
    template <int TYPE, bool WIDE, int TPR, int V, int R, bool STREAMED>
    hipError_t with() const
    {
        constexpr int TEAMS = NTH / TPR * R;
        const long long steps = ((long long)a.n + TEAMS - 1) / TEAMS;
        if (!a.dgamma && !a.dbeta) {
            k_norm_bwd<TYPE, WIDE, TPR, V, R, false, STREAMED><<<(unsigned)steps, NTH, 0, stream>>>(a);
            return hipGetLastError();
        }
        // two rows a team at least: a workgroup's sums cost it the write of two rows in binary32
        const long long most = norm_bwd_max_blocks(a.n, a.c), want = steps <= ALONE ? 1 : (steps * R + 1) / 2;
        const int blocks = (int)(want < most ? want : most);
        k_norm_bwd<TYPE, WIDE, TPR, V, R, true, STREAMED><<<(unsigned)blocks, NTH, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || blocks == 1) return e;
        k_norm_bwd_join<<<(unsigned)((2 * a.c + 15) / 16), 1024, 0, stream>>>(a.part, blocks, a.c, a.dgamma, a.dbeta);
        return hipGetLastError();
    }
    template <int TYPE, bool WIDE, int TPR, int V>
    hipError_t go() const
    {
        constexpr int R = (TPR == 256 && V > 1) || V > 2 ? 1 : 2;
        const bool large = (size_t)a.n * a.c * sizeof(typename Elems<TYPE>::one) >= STREAMED_BYTES;
        return large ? with<TYPE, WIDE, TPR, V, R, true>() : with<TYPE, WIDE, TPR, V, 1, false>();
    }
};

// A team is as small as keeps a thread's part of a row in one 16-byte piece, up to a wave, then the parts grow to four pieces, then
// a workgroup takes the row. Parts of 32 elements leave no registers for rows of any alignment: 100000 rows of 1537 bfloat16 channels,
// backward, 314 us by a wave, 234 by a workgroup.
template <int TYPE, bool WIDE, class F>
hipError_t by_width(const F& f, int c)
{
    const int pieces = (c + Elems<TYPE>::W - 1) / Elems<TYPE>::W;
    if (pieces <= 8) return f.template go<TYPE, WIDE, 8, 1>();
    if (pieces <= 16) return f.template go<TYPE, WIDE, 16, 1>();
    if (pieces <= 32) return f.template go<TYPE, WIDE, 32, 1>();
    if (pieces <= 64) return f.template go<TYPE, WIDE, 64, 1>();
    if (pieces <= 128) return f.template go<TYPE, WIDE, 64, 2>();
    if (pieces <= 256) {
        if constexpr (WIDE || TYPE == F3D_F32) return f.template go<TYPE, WIDE, 64, 4>();
        else return f.template go<TYPE, WIDE, 256, 1>();
    }
    if (pieces <= 512) return f.template go<TYPE, WIDE, 256, 2>();
    if (pieces <= 1024) return f.template go<TYPE, WIDE, 256, 4>();
    if constexpr (TYPE == F3D_F32) return f.template go<TYPE, WIDE, 256, 8>();
    return hipErrorInvalidValue;
}

template <class F>
hipError_t by_type(const F& f, int type, int c, int wide)
{
    switch (type) {
        case F3D_BF16: return wide ? by_width<F3D_BF16, true>(f, c) : by_width<F3D_BF16, false>(f, c);
        case F3D_F16: return wide ? by_width<F3D_F16, true>(f, c) : by_width<F3D_F16, false>(f, c);
        default: return wide ? by_width<F3D_F32, true>(f, c) : by_width<F3D_F32, false>(f, c);
    }
}

}  // namespace

int64_t norm_bwd_max_blocks(int64_t n, int c)
{
    const int64_t most = c <= 2048 ? 1024 : 512, want = (n + 1) / 2;
    return want < 1 ? 1 : want < most ? want : most;
}

hipError_t norm_launch(const NormArgs& a, hipStream_t stream) { return by_type(Forward{a, stream}, a.type, a.c, a.wide); }

hipError_t norm_bwd_launch(const NormBwdArgs& a, hipStream_t stream)
{
    if (a.n == 0) {   // no rows: the weights' gradients are zero all the same
        k_norm_bwd_join<<<(unsigned)((2 * a.c + 15) / 16), 1024, 0, stream>>>(a.part, 0, a.c, a.dgamma, a.dbeta);
        return hipGetLastError();
    }
    return by_type(Backward{a, stream}, a.type, a.c, a.wide);
}

}  // namespace f3d
