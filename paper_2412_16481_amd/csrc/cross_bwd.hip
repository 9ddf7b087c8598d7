// Cross attention backward for gfx950.
//
//   P = exp(S - lse),  dP = dO v^T,  D_i = sum_c dO_ic O_ic,  dS = P o (dP - D),
//   dq = scale dS k,  dk = scale dS^T q,  dv = P^T dO,  the last two summed over the heads that share the key/value head
//
// P and dS are rounded to bf16, as the matrix instructions take them; every sum is held in binary32.
// Two kernels, as for the attention inside scopes, and neither needs atomics:
//   k_cross_bwd_dq    owns query rows, streams K and V, works out D on the way. Scores are computed transposed (keys x rows), so a lane
//                     owns 16 keys of ONE row: lse and D are per-lane scalars, and dS^T, packed to bf16, is the B operand of
//                     dQ^T += K^T dS^T.
//   k_cross_bwd_dkdv  owns 128 keys of a key/value head, streams the rows of all heads that share it (after the first kernel: it reads
//                     D). Scores are rows x keys, a lane owns 16 rows of ONE key; P and dS are the B operands of dV^T += dO^T P and
//                     dK^T += Q^T dS. The sum over shared heads is the sum over rows. 128 channels: k_cross_bwd_dkdv_wide.
// Up to 128 keys of 16 channels, or 96 of 32, go to the one kernel of cross_bwd_short.hip.
// Few keys beside many rows (or the reverse) leave one of the two with a handful of workgroups: then its sum over rows (over keys) is split
// into parts, kept in binary32 and added up in a fixed order by a last kernel.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "cross_common.h"

namespace f3d {

namespace {

constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ f32x16 mfma(const U4& x, const U4& y, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.b, y.b, c, 0, 0, 0);
}

// 32 channels of a result's row from the lane that owns it, in binary32 (`part`) or rounded
template <int D, int MT>
__device__ __forceinline__ void store_row(float* part, uint16_t* to, const f32x16 (&acc)[MT], int hf, float mul, bool has)
{
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int r4 = 0; r4 < (D == 16 ? 2 : 4); ++r4) {
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            if (has) y = make_float4(acc[mt][4 * r4] * mul, acc[mt][4 * r4 + 1] * mul, acc[mt][4 * r4 + 2] * mul, acc[mt][4 * r4 + 3] * mul);
            const int c = mt * 32 + 8 * r4 + 4 * hf;
            if (part) *reinterpret_cast<float4*>(part + c) = y;
            else *reinterpret_cast<uint2*>(to + c) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
        }
    }
}

// Runs of row blocks, stages and their hand-over as in the forward kernel. Per tile of 32 keys a wave has 2 KS MFMAs for the scores and dP
// (of the NEXT tile, issued between the exponentials of the current one; -D is the accumulator dP starts from) and 2 MT for dQ. Bound: the
// matrix cores and, at 16 and 32 channels, the vector ALU's issue port. 8 ragged segments of up to 2047 rows and 1500 keys, 16 heads of 128
// channels on 4: 212 us; 250 with the products of a tile and its exponentials one after the other.
template <int D, bool SPLIT>
__global__ __launch_bounds__(256, 2) void k_cross_bwd_dq(CrossBwdArgs b)
{
    using T = Tile<D>;
    using S = RowStage<D>;
    constexpr int KS = T::KS, MT = T::MT, NBUF = S::NBUF;
    constexpr int BM = 128;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[S::TOTAL];
    const CrossArgs& a = b.f;
    const uint32_t sK = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
    constexpr uint32_t KV = NBUF * S::BYTES;          // from a row of K to the same of V
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (!SPLIT) zero_rows(b.dq, a.n_q, offset_of(a.q_offsets, a.n_q, 0), offset_of(a.q_offsets, a.n_q, a.segments), (uint32_t)a.H * T::ROWB);
    const uint32_t u = piece_of(a.turn);
    const uint32_t x = u / (uint32_t)a.K;
    const int kh = (int)(u - x * a.K), slot = (int)(SPLIT ? x / (uint32_t)a.parts : x), part = SPLIT ? (int)(x - (uint32_t)slot * a.parts) : 0;
    if (slot >= a.slots) return;
    const int seg = segment_of(a.q_offsets, a.n_q, a.segments, a.G, a.run_shift, slot);
    const Rows qs = rows_of(a.q_offsets, a.q_lens, a.n_q, seg), kv = rows_of(a.kv_offsets, a.kv_lens, a.n_kv, seg);
    const long long run = slot - first_slot(a.q_offsets, a.n_q, seg, a.G, a.run_shift);
    const int rows = qs.span * a.G, live = qs.len * a.G;
    if (run < 0 || (run << a.run_shift) >= rows) return;
    const int first_row = (int)(run << a.run_shift);
    const int blocks = (min(rows - first_row, 1 << a.run_shift) + BM - 1) / BM;
    const int key0 = SPLIT ? part * a.chunk : 0;
    const int nkeys = first_row >= live ? 0 : SPLIT ? min(max(kv.len - key0, 0), a.chunk) : kv.len;

    const uint32_t row_bytes = (uint32_t)a.K * T::ROWB;
    KeyRing<D> ring;
    ring.start(a.k, a.v, (uint64_t)(kv.from + key0) * row_bytes + (uint64_t)kh * T::ROWB, row_bytes, nkeys, blocks, sK, wave);

    uint32_t off[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) off[ks] = sK + T::row_piece(lane, ks);
    const uint32_t toff = sK + T::transposed(lane);
    const float mul = a.s_mul;
    if (nkeys > 0) {
        __builtin_amdgcn_s_waitcnt(vm_wait(0));
        __syncthreads();
    }

    U4 qf[KS], gf[KS];
    f32x16 acc[MT], minus_d;
    float nl;
    // One unit: dS = P o (dP - D) of the current tile (keys from kbase on, at `at`) and its dQ, with the products of the next (at `an`)
    auto unit = [&](f32x16& s, f32x16& dp, uint32_t at, int kbase, f32x16& sn, f32x16& dpn, uint32_t an) __attribute__((always_inline)) {
        constexpr int EP = 16 / (2 * KS);
        U4 kf[2], vf[2], p0, p1, x[2][2];
        if (kbase + 32 > nkeys) {                     // keys past the end repeat one: their dS is dropped
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (kbase + 8 * (r >> 2) + 4 * hf + (r & 3) >= nkeys) dp[r] = 0.f;
        }
        const auto prob = [&](int r) __attribute__((always_inline)) { dp[r] *= __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], mul, nl)); };
        kf[0].u = lds_read16(off[0] + an);
        vf[0].u = lds_read16(off[0] + an + KV);
        F3D_SB();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (ks + 1 < KS) {
                kf[(ks + 1) & 1].u = lds_read16(off[ks + 1] + an);
                vf[(ks + 1) & 1].u = lds_read16(off[ks + 1] + an + KV);
            }
            if (ks == KS - 1) read_transposed<D>(x[0][0], x[0][1], toff + at, (toff + at) ^ T::FLIP, 0);
            F3D_SB();
#pragma unroll
            for (int e = 0; e < EP; ++e) prob(2 * ks * EP + e);
            F3D_SB();
            sn = mfma(kf[ks & 1], qf[ks], ks == 0 ? f32x16{0} : sn);
            F3D_SB();
#pragma unroll
            for (int e = 0; e < EP; ++e) prob((2 * ks + 1) * EP + e);
            F3D_SB();
            dpn = mfma(vf[ks & 1], gf[ks], ks == 0 ? minus_d : dpn);
            F3D_SB();
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) (&p0.u.x)[e] = pack_bf16(dp[2 * e], dp[2 * e + 1]);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt + 1 < MT) read_transposed<D>(x[(mt + 1) & 1][0], x[(mt + 1) & 1][1], toff + at, (toff + at) ^ T::FLIP, mt + 1);
            F3D_SB();
            acc[mt] = mfma(x[mt & 1][0], p0, acc[mt]);
            F3D_SB();
            if (mt == 0) {
#pragma unroll
                for (int e = 0; e < 4; ++e) (&p1.u.x)[e] = pack_bf16(dp[8 + 2 * e], dp[8 + 2 * e + 1]);
                F3D_SB();
            }
            acc[mt] = mfma(x[mt & 1][1], p1, acc[mt]);
            F3D_SB();
        }
    };

    f32x16 sa, sb, da, db;
    int buf = 0, read = 0;                            // read: stages over all row blocks
    // A block's rows are asked for a block ahead, where the registers allow it
    constexpr bool AHEAD = D <= 64;
    U4 nq[KS], ng[KS], no[KS];
    float nlse = 0.f;
    uint32_t place = 0;
    auto fetch_row = [&](int blk) __attribute__((always_inline)) {
        const int r = min(first_row + blk * BM + wave * 32 + l32, max(live, 1) - 1);   // past the end, or behind the segment's length: a row that counts, dropped
        const int i = divide(r, a.G, a.by_g), g = r - i * a.G;
        place = (uint32_t)(qs.from + i) * (uint32_t)a.H + (uint32_t)(kh * a.G + g);
        const uint64_t from = (uint64_t)place * T::ROWB + hf * 16;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            nq[ks].u = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(a.q) + from + ks * 32);
            ng[ks].u = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(b.dout) + from + ks * 32);
            no[ks].u = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(a.out) + from + ks * 32);
        }
        nlse = a.lse[place];
    };
    if (AHEAD) fetch_row(0);
    for (int blk = 0; blk < blocks; ++blk) {
        const int row = first_row + blk * BM + wave * 32 + l32;
        const bool takes = row < live, busy = first_row + blk * BM + wave * 32 < live;
        if (!AHEAD) fetch_row(blk);
        {
            float dot = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                qf[ks] = nq[ks];
                gf[ks] = ng[ks];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t y = (&no[ks].u.x)[e], z = (&ng[ks].u.x)[e];
                    dot += __uint_as_float(y << 16) * __uint_as_float(z << 16);
                    dot += __uint_as_float(y & 0xFFFF0000u) * __uint_as_float(z & 0xFFFF0000u);
                }
            }
            dot += __shfl_xor(dot, 32, 64);
            if (takes && part == 0 && hf == 0) b.dsum[place] = dot;
            nl = takes && nkeys > 0 ? -LOG2E * nlse : -INFINITY;   // rows that take no part: probabilities exactly zero
            if (AHEAD && blk + 1 < blocks) fetch_row(blk + 1);
#pragma unroll
            for (int r2 = 0; r2 < 16; ++r2) minus_d[r2] = -dot;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[mt] = f32x16{0};
        }
        if (ring.stays) buf = 0;
        if (nkeys > 0 && busy) {
            sa = f32x16{0};
            da = minus_d;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                U4 kf, vf;
                kf.u = lds_read16(off[ks] + buf * S::BYTES);
                vf.u = lds_read16(off[ks] + buf * S::BYTES + KV);
                sa = mfma(kf, qf[ks], sa);
                da = mfma(vf, gf[ks], da);
            }
        }
        auto stage = [&](int st, auto first_tile) __attribute__((always_inline)) {
            const int bufn = buf + 1 == NBUF ? 0 : buf + 1;
            const uint32_t at0 = buf * S::BYTES, an0 = bufn * S::BYTES;
#pragma unroll
            for (int t4 = 0; t4 < S::TILES; ++t4) {
                if (t4 + 1 == S::TILES && !ring.stays) ring.hand_over(buf, ++read);
                const int kbase = st * S::ROWS + t4 * 32;
                if (!busy || kbase >= nkeys) continue;
                const uint32_t at = at0 + t4 * T::BYTES, an = t4 + 1 < S::TILES ? at + T::BYTES : an0;
                if (((t4 + decltype(first_tile)::value) & 1) == 0) unit(sa, da, at, kbase, sb, db, an);
                else unit(sb, db, at, kbase, sa, da, an);
            }
            buf = bufn;
        };
        for (int st = 0; st < ring.nst; st += S::LOOP) {
            stage(st, std::integral_constant<int, 0>{});
            if (S::LOOP == 1) continue;
            if (st + 1 >= ring.nst) break;
            stage(st + 1, std::integral_constant<int, 1>{});
        }
        if (row >= rows) continue;
        const int i = divide(row, a.G, a.by_g), g = row - i * a.G;
        const size_t at = (size_t)(qs.from + i) * a.H + kh * a.G + g;
        float* const p = SPLIT ? b.part_dq + ((size_t)part * a.n_q * a.H + at) * D : nullptr;
        store_row<D, MT>(p, b.dq + at * D, acc, hf, b.scale, takes && nkeys > 0);
    }
}

// The query rows stream through LDS in stages of KStage::ROWS, three of them resident. Per tile of 32 rows a wave has 4 KS MFMAs for the
// scores and dP (of the NEXT tile: they are issued between the exponentials of the current one) and 4 MT for the two gradients. The
// starting accumulators of a tile are read from LDS: -lse (in the score's units) and -D of its rows, so neither costs a
// subtraction, and rows past the end have -infinity there: their probabilities are exactly zero. 16 ragged segments of up to 2047 rows and
// 1500 keys, 12 heads of 64 channels on 4: 225 us, and dQ 149.
template <int D>
struct KStage {
    using T = Tile<D>;
    static constexpr int ROWS = D == 16 ? 128 : 64;
    static constexpr int TILES = ROWS / 32;
    static constexpr int BYTES = ROWS * T::ROWB;      // of one operand
    static constexpr int NBUF = 3;
    static constexpr int LPW = ROWS * T::NC / 256;
    static constexpr int TOTAL = NBUF * 2 * BYTES;
};

template <int D, bool SPLIT>
__global__ __launch_bounds__(256, 2) void k_cross_bwd_dkdv(CrossBwdArgs b)
{
    using T = Tile<D>;
    using S = KStage<D>;
    constexpr int KS = T::KS, MT = T::MT, LPW = S::LPW, NBUF = S::NBUF, BM = 128, SHIFT = 7;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[S::TOTAL];
    __shared__ __attribute__((aligned(16))) float sl[NBUF][S::ROWS], sd[NBUF][S::ROWS];
    const CrossArgs& a = b.f;
    const uint32_t sQ = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem, sG = sQ + NBUF * S::BYTES;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (!SPLIT) {
        const int from = offset_of(a.kv_offsets, a.n_kv, 0), to = offset_of(a.kv_offsets, a.n_kv, a.segments);
        zero_rows(b.dk, a.n_kv, from, to, (uint32_t)a.K * T::ROWB);
        zero_rows(b.dv, a.n_kv, from, to, (uint32_t)a.K * T::ROWB);
    }
    const uint32_t u = piece_of(b.kv_turn);
    const uint32_t x = u / (uint32_t)a.K;
    const int kh = (int)(u - x * a.K), part = SPLIT ? (int)(x / (uint32_t)b.kv_slots) : 0, slot = (int)(x - (uint32_t)part * b.kv_slots);
    if (SPLIT ? part >= b.row_parts : slot >= b.kv_slots) return;
    const int seg = segment_of(a.kv_offsets, a.n_kv, a.segments, 1, SHIFT, slot);
    const Rows qs = rows_of(a.q_offsets, a.q_lens, a.n_q, seg), kv = rows_of(a.kv_offsets, a.kv_lens, a.n_kv, seg);
    const long long blk = slot - first_slot(a.kv_offsets, a.n_kv, seg, 1, SHIFT);
    if (blk < 0 || blk * BM >= kv.span) return;
    const int row0 = SPLIT ? part * b.row_chunk : 0, live = qs.len * a.G;
    const int nrows = blk * BM >= kv.len ? 0 : SPLIT ? min(max(live - row0, 0), b.row_chunk) : live;

    const uint32_t row_bytes = (uint32_t)a.H * T::ROWB;
    const float mul = a.s_mul, lmul = -LOG2E / a.s_mul;
    int srow[LPW];
    uint32_t scol[LPW];
#pragma unroll
    for (int i = 0; i < LPW; ++i) {
        const int p = (wave * LPW + i) * 64 + lane;
        srow[i] = p / T::NC;
        scol[i] = ((p % T::NC) ^ T::swizzle(srow[i])) << 4;
    }
    float nl = 0.f, nd = 0.f;                         // of row `tid` of the stage requested last
    auto request = [&](int st) __attribute__((always_inline)) {
        const uint32_t to = (st % NBUF) * S::BYTES;
        if (tid < S::ROWS) {
            const int r = st * S::ROWS + tid, rc = row0 + min(r, nrows - 1);
            const int q = divide(rc, a.G, a.by_g), g = rc - q * a.G;
            const size_t at = (size_t)(qs.from + q) * a.H + kh * a.G + g;
            const float l = a.lse[at], d = b.dsum[at];
            nl = r < nrows ? l * lmul : -INFINITY;
            nd = -d;
        }
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
            const int r = row0 + min(st * S::ROWS + srow[i], nrows - 1);
            const int q = divide(r, a.G, a.by_g), g = r - q * a.G;
            const uint64_t at = (uint64_t)(qs.from + q) * row_bytes + (uint32_t)(kh * a.G + g) * T::ROWB + scol[i];
            lds_dma16(reinterpret_cast<const char*>(a.q) + at, sQ + to + (wave * LPW + i) * 1024);
            lds_dma16(reinterpret_cast<const char*>(b.dout) + at, sG + to + (wave * LPW + i) * 1024);
        }
    };
    auto keep_sums = [&](int st) __attribute__((always_inline)) {
        if (tid < S::ROWS) {
            sl[st % NBUF][tid] = nl;
            sd[st % NBUF][tid] = nd;
        }
    };
    const int nst = (nrows + S::ROWS - 1) / S::ROWS;
    if (nst > 0) {
        request(0);
        keep_sums(0);
    }
    if (nst > 1) request(1);

    const long long key = blk * BM + wave * 32 + l32;
    const bool has = key < kv.len && nrows > 0;
    const bool busy = blk * BM + wave * 32 < kv.len;
    U4 kf[KS], vf[KS];
    f32x16 dk[MT], dv[MT];
    {
        const size_t at = ((size_t)(kv.from + min(key, (long long)max(kv.len, 1) - 1)) * a.K + kh) * D + hf * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            kf[ks].u = *reinterpret_cast<const uint4*>(a.k + at + ks * 16);
            vf[ks].u = *reinterpret_cast<const uint4*>(a.v + at + ks * 16);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) dk[mt] = dv[mt] = f32x16{0};
    }
    uint32_t off[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) off[ks] = sQ + T::row_piece(lane, ks);
    constexpr uint32_t GQ = NBUF * S::BYTES;          // from a row of Q to the same of dO
    const uint32_t tr = sQ + T::transposed(lane);

    auto start = [&](f32x16& s, f32x16& dp, int buf, int t4) __attribute__((always_inline)) {
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            const float4 l = *reinterpret_cast<const float4*>(&sl[buf][t4 * 32 + 8 * r4 + 4 * hf]);
            const float4 d = *reinterpret_cast<const float4*>(&sd[buf][t4 * 32 + 8 * r4 + 4 * hf]);
            s[4 * r4] = l.x, s[4 * r4 + 1] = l.y, s[4 * r4 + 2] = l.z, s[4 * r4 + 3] = l.w;
            dp[4 * r4] = d.x, dp[4 * r4 + 1] = d.y, dp[4 * r4 + 2] = d.z, dp[4 * r4 + 3] = d.w;
        }
    };
    // One unit: P = 2^s, dS = P o dp of the current tile (at `at`) and its gradients, with the products of the next one (at `an` of
    // buffer `nbuf`, its tile `nt`) in between
    auto unit = [&](f32x16& s, f32x16& dp, uint32_t at, f32x16& sn, f32x16& dpn, uint32_t an, int nbuf, int nt) __attribute__((always_inline)) {
        constexpr int EP = 16 / (2 * KS);             // elements behind each of the products
        U4 qf[2], gf[2], p0, p1, d0, d1, x[2][4];
        const auto prob = [&](int r) __attribute__((always_inline)) {
            s[r] = __builtin_amdgcn_exp2f(s[r] * mul);
            dp[r] *= s[r];
        };
        const auto turned = [&](int mt) __attribute__((always_inline)) {
            const uint32_t t = tr + at;
            read_transposed<D>(x[mt & 1][0], x[mt & 1][1], t + GQ, (t + GQ) ^ T::FLIP, mt);
            read_transposed<D>(x[mt & 1][2], x[mt & 1][3], t, t ^ T::FLIP, mt);
        };
        start(sn, dpn, nbuf, nt);
        qf[0].u = lds_read16(off[0] + an);
        gf[0].u = lds_read16(off[0] + an + GQ);
        F3D_SB();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (ks + 1 < KS) {
                qf[(ks + 1) & 1].u = lds_read16(off[ks + 1] + an);
                gf[(ks + 1) & 1].u = lds_read16(off[ks + 1] + an + GQ);
            }
            if (ks == KS - 1) turned(0);
            F3D_SB();
#pragma unroll
            for (int e = 0; e < EP; ++e) prob(2 * ks * EP + e);
            F3D_SB();
            sn = mfma(qf[ks & 1], kf[ks], sn);
            F3D_SB();
#pragma unroll
            for (int e = 0; e < EP; ++e) prob((2 * ks + 1) * EP + e);
            F3D_SB();
            dpn = mfma(gf[ks & 1], vf[ks], dpn);
            F3D_SB();
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            (&p0.u.x)[e] = pack_bf16(s[2 * e], s[2 * e + 1]);
            (&d0.u.x)[e] = pack_bf16(dp[2 * e], dp[2 * e + 1]);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt + 1 < MT) turned(mt + 1);
            F3D_SB();
            dv[mt] = mfma(x[mt & 1][0], p0, dv[mt]);
            dk[mt] = mfma(x[mt & 1][2], d0, dk[mt]);
            F3D_SB();
            if (mt == 0) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    (&p1.u.x)[e] = pack_bf16(s[8 + 2 * e], s[8 + 2 * e + 1]);
                    (&d1.u.x)[e] = pack_bf16(dp[8 + 2 * e], dp[8 + 2 * e + 1]);
                }
                F3D_SB();
            }
            dv[mt] = mfma(x[mt & 1][1], p1, dv[mt]);
            dk[mt] = mfma(x[mt & 1][3], d1, dk[mt]);
            F3D_SB();
        }
    };
    // Stage st + 1 is handed over to the readers and the buffer of stage st - 1 requested again for st + 2: whoever arrives has its own
    // loads of st + 1 and has read the last of st - 1.
    auto handover = [&](int st) __attribute__((always_inline)) {
        if (st + 1 < nst) keep_sums(st + 1);
        __builtin_amdgcn_s_waitcnt(vm_wait(0));
        __syncthreads();
        if (st + 2 < nst) request(st + 2);
    };

    if (nst > 0) {
        __builtin_amdgcn_s_waitcnt(vm_wait(0));       // stage 0 is here, and with it stage 1
        __syncthreads();
        f32x16 sa, da, sb, db;
        start(sa, da, 0, 0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            U4 qf, gf;
            qf.u = lds_read16(off[ks]);
            gf.u = lds_read16(off[ks] + GQ);
            sa = mfma(qf, kf[ks], sa);
            da = mfma(gf, vf[ks], da);
        }
        for (int st = 0, buf = 0; st < nst; ++st) {
            const int bufn = buf + 1 == NBUF ? 0 : buf + 1;
            const uint32_t at = buf * S::BYTES, an = bufn * S::BYTES;
#pragma unroll
            for (int t4 = 0; t4 < S::TILES; t4 += 2) {
                if (busy) unit(sa, da, at + t4 * T::BYTES, sb, db, at + (t4 + 1) * T::BYTES, buf, t4 + 1);
                if (t4 + 2 < S::TILES) {
                    if (busy) unit(sb, db, at + (t4 + 1) * T::BYTES, sa, da, at + (t4 + 2) * T::BYTES, buf, t4 + 2);
                } else {
                    handover(st);                     // what is computed ahead of the last tile of all reads some buffer and is never used
                    if (busy) unit(sb, db, at + (t4 + 1) * T::BYTES, sa, da, an, bufn, 0);
                }
            }
            buf = bufn;
        }
    }
    if (key >= kv.span) return;
    const size_t at = ((size_t)(kv.from + key) * a.K + kh) * D, all = (size_t)a.n_kv * a.K * D;
    float* const p = SPLIT ? b.part_dkv + part * all + at : nullptr;
    store_row<D, MT>(p, b.dk + at, dk, hf, b.scale, has);
    store_row<D, MT>(SPLIT ? p + b.row_parts * all : nullptr, b.dv + at, dv, hf, 1.0f, has);
}

// The same for 128 channels, where one wave's gradients of 32 keys take 128 registers. Eight waves, two to a SIMD: four tiles of keys by
// two tiles of rows of a stage, so that one wave's products run beside another's exponentials; V stays in LDS, what would be its registers
// make room for that. The two waves of a key tile add up at the end. 325 us at the sizes of the other kernel (395 with four waves of one
// tile of keys each, one to a SIMD).
template <bool SPLIT>
__global__ __launch_bounds__(512, 2) void k_cross_bwd_dkdv_wide(CrossBwdArgs b)
{
    constexpr int D = 128, ROWS = 64, NBUF = 3, BM = 128, SHIFT = 7;
    using T = Tile<D>;
    constexpr int KS = T::KS, MT = T::MT, BYTES = ROWS * T::ROWB, LPW = ROWS * T::NC / 512, VBYTES = BM * T::ROWB;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[VBYTES + NBUF * 2 * BYTES];
    __shared__ __attribute__((aligned(16))) float sl[NBUF][ROWS], sd[NBUF][ROWS];
    const CrossArgs& a = b.f;
    const uint32_t sV = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem, sQ = sV + VBYTES;
    constexpr uint32_t GQ = NBUF * BYTES;             // from a row of Q to the same of dO
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kt = wave & 3, group = wave >> 2;
    if (!SPLIT) {
        const int from = offset_of(a.kv_offsets, a.n_kv, 0), to = offset_of(a.kv_offsets, a.n_kv, a.segments);
        zero_rows(b.dk, a.n_kv, from, to, (uint32_t)a.K * T::ROWB);
        zero_rows(b.dv, a.n_kv, from, to, (uint32_t)a.K * T::ROWB);
    }
    const uint32_t u = piece_of(b.kv_turn);
    const uint32_t x = u / (uint32_t)a.K;
    const int kh = (int)(u - x * a.K), part = SPLIT ? (int)(x / (uint32_t)b.kv_slots) : 0, slot = (int)(x - (uint32_t)part * b.kv_slots);
    if (SPLIT ? part >= b.row_parts : slot >= b.kv_slots) return;
    const int seg = segment_of(a.kv_offsets, a.n_kv, a.segments, 1, SHIFT, slot);
    const Rows qs = rows_of(a.q_offsets, a.q_lens, a.n_q, seg), kv = rows_of(a.kv_offsets, a.kv_lens, a.n_kv, seg);
    const long long blk = slot - first_slot(a.kv_offsets, a.n_kv, seg, 1, SHIFT);
    if (blk < 0 || blk * BM >= kv.span) return;
    const int row0 = SPLIT ? part * b.row_chunk : 0, live = qs.len * a.G;
    const int nrows = blk * BM >= kv.len ? 0 : SPLIT ? min(max(live - row0, 0), b.row_chunk) : live;

    const uint32_t row_bytes = (uint32_t)a.H * T::ROWB;
    const float mul = a.s_mul, lmul = -LOG2E / a.s_mul;
    int srow[LPW];
    uint32_t scol[LPW];
#pragma unroll
    for (int i = 0; i < LPW; ++i) {
        const int p = (wave * LPW + i) * 64 + lane;
        srow[i] = p / T::NC;
        scol[i] = ((p % T::NC) ^ T::swizzle(srow[i])) << 4;
    }
    float nl = 0.f, nd = 0.f;                         // of row `tid` of the stage requested last
    auto request = [&](int st) __attribute__((always_inline)) {
        const uint32_t to = (st % NBUF) * BYTES;
        if (tid < ROWS) {
            const int r = st * ROWS + tid, rc = row0 + min(r, nrows - 1);
            const int q = divide(rc, a.G, a.by_g), g = rc - q * a.G;
            const size_t at = (size_t)(qs.from + q) * a.H + kh * a.G + g;
            const float l = a.lse[at], d = b.dsum[at];
            nl = r < nrows ? l * lmul : -INFINITY;
            nd = -d;
        }
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
            const int r = row0 + min(st * ROWS + srow[i], nrows - 1);
            const int q = divide(r, a.G, a.by_g), g = r - q * a.G;
            const uint64_t at = (uint64_t)(qs.from + q) * row_bytes + (uint32_t)(kh * a.G + g) * T::ROWB + scol[i];
            lds_dma16(reinterpret_cast<const char*>(a.q) + at, sQ + to + (wave * LPW + i) * 1024);
            lds_dma16(reinterpret_cast<const char*>(b.dout) + at, sQ + GQ + to + (wave * LPW + i) * 1024);
        }
    };
    auto keep_sums = [&](int st) __attribute__((always_inline)) {
        if (tid < ROWS) {
            sl[st % NBUF][tid] = nl;
            sd[st % NBUF][tid] = nd;
        }
    };
    const int nst = (nrows + ROWS - 1) / ROWS;
    const long long key = blk * BM + kt * 32 + l32;
    const bool busy = blk * BM + kt * 32 < kv.len;
    U4 kf[KS];
    f32x16 dk[MT], dv[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) dk[mt] = dv[mt] = f32x16{0};
    if (nst > 0) {
#pragma unroll
        for (int i = 0; i < VBYTES / 8192; ++i) {     // V: rows past the end repeat the last one
            const int p = (wave * (VBYTES / 8192) + i) * 64 + lane, r = p / T::NC;
            const long long k = min(blk * BM + r, (long long)kv.len - 1);
            const uint64_t at = ((uint64_t)(kv.from + k) * a.K + kh) * T::ROWB + (((p % T::NC) ^ T::swizzle(r & 31)) << 4);
            lds_dma16(reinterpret_cast<const char*>(a.v) + at, sV + (wave * (VBYTES / 8192) + i) * 1024);
        }
        request(0);
        keep_sums(0);
        if (nst > 1) {
            request(1);
            keep_sums(1);
        }
        const size_t at = ((size_t)(kv.from + min(key, (long long)kv.len - 1)) * a.K + kh) * D + hf * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[ks].u = *reinterpret_cast<const uint4*>(a.k + at + ks * 16);
    }
    uint32_t off[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) off[ks] = T::row_piece(lane, ks);
    const uint32_t tr = sQ + T::transposed(lane), sv = sV + kt * T::BYTES;

    for (int st = 0; st < nst; ++st) {
        // the stage is here once only what was asked for after it is outstanding
        if (st > 0 && st + 1 < nst) __builtin_amdgcn_s_waitcnt(vm_wait(2 * LPW));
        else __builtin_amdgcn_s_waitcnt(vm_wait(0));
        __syncthreads();                              // every wave's part of it is, and stage st - 1 has been read
        if (st + 2 < nst) request(st + 2);
        if (busy) {
            const int buf = st % NBUF;
            const uint32_t at = buf * BYTES + group * T::BYTES;
            f32x16 s, dp;
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const float4 l = *reinterpret_cast<const float4*>(&sl[buf][group * 32 + 8 * r4 + 4 * hf]);
                const float4 d = *reinterpret_cast<const float4*>(&sd[buf][group * 32 + 8 * r4 + 4 * hf]);
                s[4 * r4] = l.x, s[4 * r4 + 1] = l.y, s[4 * r4 + 2] = l.z, s[4 * r4 + 3] = l.w;
                dp[4 * r4] = d.x, dp[4 * r4 + 1] = d.y, dp[4 * r4 + 2] = d.z, dp[4 * r4 + 3] = d.w;
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                U4 qf, gf, vf;
                qf.u = lds_read16(sQ + at + off[ks]);
                gf.u = lds_read16(sQ + GQ + at + off[ks]);
                vf.u = lds_read16(sv + off[ks]);
                s = mfma(qf, kf[ks], s);
                dp = mfma(gf, vf, dp);
            }
            U4 p0, p1, d0, d1;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = __builtin_amdgcn_exp2f(s[r] * mul);
                dp[r] *= s[r];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                (&p0.u.x)[e] = pack_bf16(s[2 * e], s[2 * e + 1]);
                (&p1.u.x)[e] = pack_bf16(s[8 + 2 * e], s[8 + 2 * e + 1]);
                (&d0.u.x)[e] = pack_bf16(dp[2 * e], dp[2 * e + 1]);
                (&d1.u.x)[e] = pack_bf16(dp[8 + 2 * e], dp[8 + 2 * e + 1]);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                U4 g0, g1, q0, q1;
                read_transposed<D>(g0, g1, tr + GQ + at, (tr + GQ + at) ^ T::FLIP, mt);
                read_transposed<D>(q0, q1, tr + at, (tr + at) ^ T::FLIP, mt);
                dv[mt] = mfma(g0, p0, dv[mt]);
                dk[mt] = mfma(q0, d0, dk[mt]);
                dv[mt] = mfma(g1, p1, dv[mt]);
                dk[mt] = mfma(q1, d1, dk[mt]);
            }
        }
        if (st + 2 < nst) keep_sums(st + 2);
    }
    // ---- the second wave of every key tile hands its sums over: dk, then dv, [4][4][16][64]
    float* const meet = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        f32x16(&acc)[MT] = which ? dv : dk;
        __syncthreads();
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if (group == 1) meet[(kt * MT * 16 + mt * 16 + r) * 64 + lane] = acc[mt][r];
            }
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[mt][r] += meet[(kt * MT * 16 + mt * 16 + r) * 64 + lane];
            }
        }
    }
    if (group == 1 || key >= kv.span) return;
    const bool has = key < kv.len && nrows > 0;
    const size_t at = ((size_t)(kv.from + key) * a.K + kh) * D, all = (size_t)a.n_kv * a.K * D;
    float* const p = SPLIT ? b.part_dkv + part * all + at : nullptr;
    store_row<D, MT>(p, b.dk + at, dk, hf, b.scale, has);
    store_row<D, MT>(SPLIT ? p + b.row_parts * all : nullptr, b.dv + at, dv, hf, 1.0f, has);
}

// The parts of a gradient: GROUPS threads to four channels, each adds up every GROUPS-th part; rows that no segment owns get zeros. y: a
// second gradient, whose parts follow. Many parts are few rows: one thread to all of 192 parts took 17 us for 77 states of 64 channels,
// 16 of them take 5; three parts of 36 MB take 20 us with one and 76 with 16, most of which have none.
template <int GROUPS>
__global__ __launch_bounds__(256) void k_cross_bwd_join(const float* part, int parts, long long n, int row_pieces, const int32_t* offsets,
                                                        int segments, int n_rows, uint16_t* x, uint16_t* y)
{
    constexpr int PIECES = 256 / GROUPS;
    __shared__ float4 meet[GROUPS][PIECES + 1];
    const int c = threadIdx.x % PIECES, k = threadIdx.x / PIECES;
    long long i = (long long)blockIdx.x * PIECES + c;
    uint16_t* to = x;
    const bool second = i >= n;
    if (second) {
        i -= n;
        to = y;
        part += (size_t)parts * n * 4;
    }
    const bool has = i < n && (!second || y);
    const long long row = i / row_pieces;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (has && row >= offset_of(offsets, n_rows, 0) && row < offset_of(offsets, n_rows, segments)) {
#pragma unroll 4
        for (int p = k; p < parts; p += GROUPS) {
            const float4 f = reinterpret_cast<const float4*>(part)[p * n + i];
            s.x += f.x;
            s.y += f.y;
            s.z += f.z;
            s.w += f.w;
        }
    }
    if (GROUPS > 1) {
        meet[k][c] = s;
        __syncthreads();
        for (int g = 1; k == 0 && g < GROUPS; ++g) {
            const float4 f = meet[g][c];
            s.x += f.x;
            s.y += f.y;
            s.z += f.z;
            s.w += f.w;
        }
    }
    if (k != 0 || !has) return;
    reinterpret_cast<uint2*>(to)[i] = make_uint2(pack_bf16(s.x, s.y), pack_bf16(s.z, s.w));
}

hipError_t join(const float* part, int parts, long long n, long long all, int row_pieces, const int32_t* offsets, int segments, int n_rows,
                uint16_t* x, uint16_t* y, hipStream_t stream)
{
    if (parts >= 16) k_cross_bwd_join<16><<<(unsigned)((all + 15) / 16), 256, 0, stream>>>(part, parts, n, row_pieces, offsets, segments, n_rows, x, y);
    else k_cross_bwd_join<1><<<(unsigned)((all + 255) / 256), 256, 0, stream>>>(part, parts, n, row_pieces, offsets, segments, n_rows, x, y);
    return hipGetLastError();
}

template <int D>
hipError_t launch(const CrossBwdArgs& b, hipStream_t stream)
{
    const CrossArgs& a = b.f;
    hipError_t e;
    if (b.short_tiles > 0) {                          // one kernel for everything but the join
        e = cross_bwd_short_launch(b, D, b.short_tiles, stream);
        if (e != hipSuccess || b.row_parts == 1) return e;
        const long long n = (long long)a.n_kv * a.K * (D / 4);
        return join(b.part_dkv, b.row_parts, n, 2 * n, a.K * (D / 4), a.kv_offsets, a.segments, a.n_kv, b.dk, b.dv, stream);
    }
    if (a.n_q > 0) {
        const unsigned grid = cross_grid((long long)a.slots * a.parts, a.K, a.turn);
        if (a.parts > 1) k_cross_bwd_dq<D, true><<<grid, 256, 0, stream>>>(b);
        else k_cross_bwd_dq<D, false><<<grid, 256, 0, stream>>>(b);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (a.parts > 1) {
            const long long n = (long long)a.n_q * a.H * (D / 4);
            e = join(b.part_dq, a.parts, n, n, a.H * (D / 4), a.q_offsets, a.segments, a.n_q, b.dq, nullptr, stream);
            if (e != hipSuccess) return e;
        }
    }
    if (a.n_kv > 0) {
        const unsigned grid = cross_grid((long long)b.kv_slots * b.row_parts, a.K, b.kv_turn);
        if constexpr (D == 128) {
            if (b.row_parts > 1) k_cross_bwd_dkdv_wide<true><<<grid, 512, 0, stream>>>(b);
            else k_cross_bwd_dkdv_wide<false><<<grid, 512, 0, stream>>>(b);
        } else {
            if (b.row_parts > 1) k_cross_bwd_dkdv<D, true><<<grid, 256, 0, stream>>>(b);
            else k_cross_bwd_dkdv<D, false><<<grid, 256, 0, stream>>>(b);
        }
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (b.row_parts > 1) {
            const long long n = (long long)a.n_kv * a.K * (D / 4);
            e = join(b.part_dkv, b.row_parts, n, 2 * n, a.K * (D / 4), a.kv_offsets, a.segments, a.n_kv, b.dk, b.dv, stream);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace

hipError_t cross_bwd_launch(const CrossBwdArgs& b, int head_dim, hipStream_t stream)
{
    switch (head_dim) {
        case 16: return launch<16>(b, stream);
        case 32: return launch<32>(b, stream);
        case 64: return launch<64>(b, stream);
        case 128: return launch<128>(b, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace f3d
