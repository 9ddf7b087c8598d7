// Cross attention forward for gfx950 (Section 4.2's attention, with the keys of another set): the query rows of a segment (the points
// of a scan, the tokens of a sequence) attend to all states of the same segment, of which there are another number.
//
//   S = scale q k^T,  P = exp(S - lse),  lse = log sum exp S,  out = P v
//
// Heads that share a key/value head are rows below each other: row r of a (segment, key/value head) is query r / G and head r % G of
// the group, so a state is read once for all of them. A wave owns tiles of 32 such rows; keys and values stream through LDS in
// stages filled by global -> LDS loads ahead of their use, row-major, swizzled (cross_common.h). Per tile of 32 keys the TRANSPOSED
// score tile S^T = K Q^T comes from 32x32x16 MFMAs: a lane then owns 16 keys of ONE row, its exponentials are per-lane work, and the
// probabilities, rounded to 16 bits, are the B operand of O^T += V^T P^T as they lie. Two sums of the exponentials are kept in
// binary32: of the rounded ones, which the result is divided by (what rounding adds to a probability leaves with it: one key gives its value
// exactly), and, where lse is wanted, of the exponentials as they are.
//
// Two forms. ROWS (k_cross): every wave has rows of its own and all keys. FEW (k_cross_few): a (segment, key/value head) has one tile of
// rows or less, the waves take the key tiles of a stage and meet in LDS at the end; that form reads keys as fast as memory
// delivers them, which is all a call with single queries does. Where the launch would leave compute units idle the keys are split
// into parts, whose results (relative to the part's reference) a second kernel joins in a fixed order.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "cross_common.h"

namespace f3d {

namespace {

constexpr float LN2 = 0.6931471805599453f;

// Many query rows: a wave owns a tile of 32 of them at a time, a workgroup a run of row blocks, so that short keys are staged once for
// several of them (they stay in LDS) and the next block's rows are on their way during this one's work. The exponentials are taken against
// the fixed reference 0, without a maximum to find and to move; a block whose sums leave the safe range is done again with the running
// maximum (reference moved only by more than 2^8). Bound: the vector ALU's issue port. A tile of 32 channels has 16 exponentials (8
// cycles each), 34 other instructions and 4 MFMAs (16 cycles of the same port each), 16 more with lse. Measured: 914601 rows of 8 x 32
// channels, 256 keys a segment, lse: 467 us = 513 TFLOP/s; about 7000 keys: 635 TFLOP/s; 16 ragged segments of up to 2047 rows and 1500 keys,
// 12 heads of 64 channels on 4, binary16: 102 us = 730 TFLOP/s (121 with the running maximum in the first sweep, and 516 for the
// other); two segments of 60000 rows and 300 keys, 8 x 128 channels: 275 us = 536 TFLOP/s (322 with one workgroup on a compute unit).
template <int D, bool F16, bool SPLIT, bool LSE>
__global__ __launch_bounds__(256, 2) void k_cross(CrossArgs a)
{
    using T = Tile<D>;
    using S = RowStage<D>;
    using E = Half<F16>;
    constexpr int KS = T::KS, MT = T::MT, NBUF = S::NBUF;
    constexpr int BM = 128;                           // rows of a workgroup at a time
    __shared__ __attribute__((aligned(1024))) unsigned char smem[S::TOTAL];
    const uint32_t sK = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem, sV = sK + NBUF * S::BYTES;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // which (run of row blocks, part, key/value head): consecutive ids stay on one XCD, the heads of the same rows beside each other
    const uint32_t u = piece_of(a.turn);
    const uint32_t x = u / (uint32_t)a.K;
    const int kh = (int)(u - x * a.K), slot = (int)(SPLIT ? x / (uint32_t)a.parts : x), part = SPLIT ? (int)(x - (uint32_t)slot * a.parts) : 0;
    if (slot >= a.slots) return;
    const int b = segment_of(a.q_offsets, a.n_q, a.segments, a.G, a.run_shift, slot);
    const Rows qs = rows_of(a.q_offsets, a.q_lens, a.n_q, b), kv = rows_of(a.kv_offsets, a.kv_lens, a.n_kv, b);
    const long long run = slot - first_slot(a.q_offsets, a.n_q, b, a.G, a.run_shift);
    const int rows = qs.span * a.G, live = qs.len * a.G;   // n_q * heads is below 2^31 by more than a run
    if (run < 0 || (run << a.run_shift) >= rows) return;
    const int first_row = (int)(run << a.run_shift);
    const int blocks = (min(rows - first_row, 1 << a.run_shift) + BM - 1) / BM;
    const int key0 = SPLIT ? part * a.chunk : 0;
    const int nkeys = first_row >= live ? 0 : SPLIT ? min(max(kv.len - key0, 0), a.chunk) : kv.len;   // this workgroup's

    const uint32_t row_bytes = (uint32_t)a.K * T::ROWB;
    KeyRing<D> ring;
    ring.start(a.k, a.v, (uint64_t)(kv.from + key0) * row_bytes + (uint64_t)kh * T::ROWB, row_bytes, nkeys, blocks, sK, wave);

    uint32_t koff[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) koff[ks] = sK + T::row_piece(lane, ks);
    const uint32_t voff = sV + T::transposed(lane);
    const float mul = a.s_mul;

    // this lane's row: row l32 of the wave's tile
    U4 qf[KS], nq[KS];
    auto row_of = [&](int blk) __attribute__((always_inline)) { return first_row + blk * BM + wave * 32 + l32; };
    uint32_t place, next_place;                       // (query, head) of the tensor
    auto fetch_row = [&](int blk) __attribute__((always_inline)) {
        const int r = min(row_of(blk), rows - 1), i = divide(r, a.G, a.by_g), g = r - i * a.G;   // past the end: the last row
        next_place = (uint32_t)(qs.from + i) * (uint32_t)a.H + (uint32_t)(kh * a.G + g);
        const char* const from = reinterpret_cast<const char*>(a.q) + (uint64_t)next_place * T::ROWB + hf * 16;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) nq[ks].u = *reinterpret_cast<const uint4*>(from + ks * 32);
    };
    fetch_row(0);
    if (nkeys > 0) {
        __builtin_amdgcn_s_waitcnt(vm_wait(0));
        __syncthreads();                              // the stages asked for so far are here
    }

    f32x16 o[MT], sa, sb;
    float m, l, lr;                                   // reference of the exponentials (log2 units), sums over this lane's keys: as they are
    U4 kf[KS];                                        // (for the log-sum-exp) and rounded, as the product with v takes them
    auto read_k = [&](U4 (&f)[KS], uint32_t at) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) f[ks].u = lds_read16(koff[ks] + at);
    };
    // One unit of the pipeline: the softmax of the score tile `s` (keys from kbase on) and O^T += V^T P^T from the keys at
    // `at`, with the MFMAs of the NEXT score tile (`sn`, keys in kf) in between.
    bool robust = false;
    auto unit = [&](f32x16& s, uint32_t at, int kbase, f32x16& sn) __attribute__((always_inline)) {
        U4 p0, p1, v0[2], v1[2];
        if (kbase + 32 > nkeys) {                     // the last tile may be short
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (kbase + 8 * (r >> 2) + 4 * hf + (r & 3) >= nkeys) s[r] = -INFINITY;
        }
        if (robust) {                                 // the running maximum
            float mx = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
            for (int r = 3; r < 15; r += 2) mx = fmaxf(fmaxf(mx, s[r]), s[r + 1]);
            mx = fmaxf(mx, s[15]);
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_int(mx), __float_as_int(mx), false, false);   // the row's other keys
            mx = fmaxf(__int_as_float(sw[0]), __int_as_float(sw[1])) * mul;
            if (__builtin_amdgcn_ballot_w64(mx > m + 8.0f)) {
                const float top = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - top);   // the first time 2^-inf, onto zeros
                m = top;
                if (LSE) l *= alpha;
                lr *= alpha;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[mt][r] *= alpha;
                }
            }
        }
        const auto prob = [&](int r) __attribute__((always_inline)) { s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], mul, -m)); };
        constexpr int EP = 16 / KS;
        F3D_SB();
        read_transposed<D>(v0[0], v1[0], voff + at, (voff + at) ^ T::FLIP, 0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
            for (int e = 0; e < EP; ++e) prob(ks * EP + e);
            F3D_SB();
            sn = E::mfma(kf[ks], qf[ks], ks == 0 ? f32x16{0} : sn);
            F3D_SB();
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            (&p0.u.x)[e] = E::pack(s[2 * e], s[2 * e + 1]);
            lr = E::sum2((&p0.u.x)[e], lr);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt + 1 < MT) read_transposed<D>(v0[(mt + 1) & 1], v1[(mt + 1) & 1], voff + at, (voff + at) ^ T::FLIP, mt + 1);
            F3D_SB();
            o[mt] = E::mfma(v0[mt & 1], p0, o[mt]);
            F3D_SB();
            if (mt == 0) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    (&p1.u.x)[e] = E::pack(s[8 + 2 * e], s[8 + 2 * e + 1]);
                    lr = E::sum2((&p1.u.x)[e], lr);
                }
            }
            F3D_SB();
            o[mt] = E::mfma(v1[mt & 1], p1, o[mt]);
            F3D_SB();
#pragma unroll
            for (int r = mt * (16 / MT); LSE && r < (mt + 1) * (16 / MT); ++r) l += s[r];
        }
    };

    int buf = 0, read = 0;                            // read: stages over all row blocks
    // One sweep over the keys for the block of rows in qf. The optimistic one takes the exponentials against the fixed reference 0: exact
    // as long as the sum stays well inside the range of the formats, which is looked at afterwards.
    auto sweep = [&](bool busy) __attribute__((always_inline)) {
        m = robust ? -INFINITY : 0.f;
        l = lr = 0.f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) o[mt] = f32x16{0};
        if (ring.stays) buf = 0;
        read_k(kf, buf * S::BYTES);
        sa = f32x16{0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sa = E::mfma(kf[ks], qf[ks], sa);
        auto stage = [&](int st, auto first_tile) __attribute__((always_inline)) {
            const int bufn = buf + 1 == NBUF ? 0 : buf + 1;
            const uint32_t at0 = buf * S::BYTES, an0 = bufn * S::BYTES;
#pragma unroll
            for (int t4 = 0; t4 < S::TILES; ++t4) {
                if (t4 + 1 == S::TILES && !ring.stays) ring.hand_over(buf, ++read);
                const int kbase = st * S::ROWS + t4 * 32;
                if (!busy || kbase >= nkeys) continue;
                const uint32_t at = at0 + t4 * T::BYTES, an = t4 + 1 < S::TILES ? at + T::BYTES : an0;
                read_k(kf, an);                       // what is computed ahead of the last tile is never used
                if (((t4 + decltype(first_tile)::value) & 1) == 0) unit(sa, at, kbase, sb);
                else unit(sb, at, kbase, sa);
            }
            buf = bufn;
        };
        for (int st = 0; st < ring.nst; st += S::LOOP) {
            stage(st, std::integral_constant<int, 0>{});
            if (S::LOOP == 1) continue;
            if (st + 1 >= ring.nst) break;
            stage(st + 1, std::integral_constant<int, 1>{});
        }
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_int(lr), __float_as_int(lr), false, false);
        lr = __int_as_float(sw[0]) + __int_as_float(sw[1]);
        if (!LSE) return;
        const auto su = __builtin_amdgcn_permlane32_swap(__float_as_int(l), __float_as_int(l), false, false);
        l = __int_as_float(su[0]) + __int_as_float(su[1]);
    };
    for (int blk = 0; blk < blocks; ++blk) {
        const bool busy = first_row + blk * BM + wave * 32 < live;   // this wave has rows with results
        place = next_place;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = nq[ks];
        if (blk + 1 < blocks) fetch_row(blk + 1);
        robust = false;
        while (nkeys > 0) {
            sweep(busy);
            if (robust) break;
            const bool bad = row_of(blk) < live && !(lr > E::SUM_LO && lr < E::SUM_HI);
            // keys that stay: every wave for itself
            robust = ring.stays ? __builtin_amdgcn_ballot_w64(bad) != 0 : __syncthreads_or(bad) != 0;
            if (!robust) break;
            if (ring.stays) continue;
            // the same keys once more: what is on its way for the next block are their first stages
            ring.total += ring.nst;
            if (blk + 1 == blocks) {                  // nothing is: all stages asked for have been read
                ring.fill(buf, NBUF - 1);
                __builtin_amdgcn_s_waitcnt(vm_wait(0));
                __syncthreads();
            }
        }
        // ---- results
        const int row = row_of(blk);
        const bool has = row < live && nkeys > 0;
        const uint32_t at_q = place;
        if (row >= rows) continue;
        if (SPLIT) {
            const size_t pa = (size_t)part * a.n_q * a.H + at_q;
            if (hf == 0) a.part_ml[pa] = has ? make_float2(m, lr) : make_float2(-INFINITY, 0.f);
            if (LSE && hf == 0) a.part_l[pa] = has ? l : 0.f;
            if (!has) continue;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int r4 = 0; r4 < (D == 16 ? 2 : 4); ++r4)
                    *reinterpret_cast<float4*>(a.part_o + pa * D + mt * 32 + 8 * r4 + 4 * hf) =
                        make_float4(o[mt][4 * r4], o[mt][4 * r4 + 1], o[mt][4 * r4 + 2], o[mt][4 * r4 + 3]);
            }
            continue;
        }
        const float inv = 1.0f / lr;
        if (LSE && hf == 0) a.lse[at_q] = has ? (m + __log2f(l)) * LN2 : -INFINITY;
        uint16_t* const to = a.out + (size_t)at_q * D;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int r4 = 0; r4 < (D == 16 ? 2 : 4); ++r4) {
                uint2 y = make_uint2(0, 0);
                if (has) {
                    y.x = E::pack(o[mt][4 * r4] * inv, o[mt][4 * r4 + 1] * inv);
                    y.y = E::pack(o[mt][4 * r4 + 2] * inv, o[mt][4 * r4 + 3] * inv);
                }
                *reinterpret_cast<uint2*>(to + mt * 32 + 8 * r4 + 4 * hf) = y;
            }
        }
    }
}

// Few query rows: the tiles of a stage of keys are shared out to the waves. Bound: HBM, every key and value once. 32 single queries of 32
// heads over caches of up to 4096 states of 8 x 128 channels, 341 MB: 71 us = 4.8 TB/s, and 4.8 us for the join; with one workgroup of four
// waves on a compute unit instead of two of two waves, 77 us.
template <int D>
struct FewStage {
    using T = Tile<D>;
    static constexpr int WAVES = D == 128 ? 2 : 4;    // 128: two workgroups on a compute unit
    static constexpr int ROWS = 32 * WAVES;
    static constexpr int BYTES = ROWS * T::ROWB;      // of K, and of V
    static constexpr int NBUF = D >= 64 ? 2 : 3;
    static constexpr int LPW = ROWS * T::NC / (64 * WAVES);    // loads per lane, stage and tensor
    static constexpr int TOTAL = NBUF * 2 * BYTES;
};

template <int D, bool F16, bool SPLIT>
__global__ __launch_bounds__(64 * FewStage<D>::WAVES, D == 128 ? 1 : 2) void k_cross_few(CrossArgs a)
{
    using T = Tile<D>;
    using S = FewStage<D>;
    using E = Half<F16>;
    constexpr int KS = T::KS, MT = T::MT, LPW = S::LPW, NBUF = S::NBUF, NW = S::WAVES;
    constexpr int BM = 32, SHIFT = 5;                 // rows of a workgroup
    __shared__ __attribute__((aligned(1024))) unsigned char smem[S::TOTAL];
    const uint32_t sK = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem, sV = sK + NBUF * S::BYTES;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // which (row block, part, key/value head): consecutive ids stay on one XCD, the heads of the same rows beside each other
    const uint32_t u = piece_of(a.turn);
    const uint32_t x = u / (uint32_t)a.K;
    const int kh = (int)(u - x * a.K), slot = (int)(SPLIT ? x / (uint32_t)a.parts : x), part = SPLIT ? (int)(x - (uint32_t)slot * a.parts) : 0;
    if (slot >= a.slots) return;
    const int b = segment_of(a.q_offsets, a.n_q, a.segments, a.G, SHIFT, slot);
    const Rows qs = rows_of(a.q_offsets, a.q_lens, a.n_q, b), kv = rows_of(a.kv_offsets, a.kv_lens, a.n_kv, b);
    const long long blk = slot - first_slot(a.q_offsets, a.n_q, b, a.G, SHIFT);
    const long long rows = (long long)qs.span * a.G, live = (long long)qs.len * a.G;
    if (blk < 0 || blk * BM >= rows) return;
    const int key0 = SPLIT ? part * a.chunk : 0;
    const int nkeys = blk * BM >= live ? 0 : SPLIT ? min(max(kv.len - key0, 0), a.chunk) : kv.len;   // this workgroup's

    // ---- staging
    const uint32_t row_bytes = (uint32_t)a.K * T::ROWB;
    const uint64_t first = (uint64_t)(kv.from + key0) * row_bytes + (uint64_t)kh * T::ROWB;
    int srow[LPW];
    uint32_t scol[LPW];
#pragma unroll
    for (int i = 0; i < LPW; ++i) {
        const int p = (wave * LPW + i) * 64 + lane;
        srow[i] = p / T::NC;
        scol[i] = ((p % T::NC) ^ T::swizzle(srow[i])) << 4;
    }
    auto dma_stage = [&](int st) __attribute__((always_inline)) {
        const uint32_t to = (st % NBUF) * S::BYTES;
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
            const int key = min(st * S::ROWS + srow[i], nkeys - 1);   // past the end: the last key again, masked
            const uint64_t at = first + (uint64_t)(uint32_t)key * row_bytes + scol[i];
            lds_dma16(reinterpret_cast<const char*>(a.k) + at, sK + to + (wave * LPW + i) * 1024);
            lds_dma16(reinterpret_cast<const char*>(a.v) + at, sV + to + (wave * LPW + i) * 1024);
        }
    };
    const int nst = (nkeys + S::ROWS - 1) / S::ROWS;
    if (nst > 0) dma_stage(0);
    if (NBUF > 2 && nst > 1) dma_stage(1);

    // ---- this lane's row: row l32
    U4 qf[KS];
    {
        const int r = (int)min(blk * BM + l32, rows - 1), i = divide(r, a.G, a.by_g), g = r - i * a.G;   // past the end: the last row again
        const uint16_t* const from = a.q + ((size_t)(qs.from + i) * a.H + kh * a.G + g) * D + hf * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[ks].u = *reinterpret_cast<const uint4*>(from + ks * 16);
        }
    }
    uint32_t koff[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) koff[ks] = sK + T::row_piece(lane, ks);
    const uint32_t voff = sV + T::transposed(lane);
    const float mul = a.s_mul;

    f32x16 o[MT];
    float m = -INFINITY, l = 0.f, lr = 0.f;           // as in the other kernel
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[mt] = f32x16{0};

    auto tile = [&](uint32_t at, int kbase) __attribute__((always_inline)) {
        U4 kf[KS], p0, p1;
        f32x16 s = f32x16{0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[ks].u = lds_read16(koff[ks] + at);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = E::mfma(kf[ks], qf[ks], s);
        if (kbase + 32 > nkeys) {                     // the last tile may be short
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (kbase + 8 * (r >> 2) + 4 * hf + (r & 3) >= nkeys) s[r] = -INFINITY;
        }
        float mx = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
        for (int r = 3; r < 15; r += 2) mx = fmaxf(fmaxf(mx, s[r]), s[r + 1]);
        mx = fmaxf(mx, s[15]);
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_int(mx), __float_as_int(mx), false, false);   // the row's other keys
        mx = fmaxf(__int_as_float(sw[0]), __int_as_float(sw[1])) * mul;
        if (__builtin_amdgcn_ballot_w64(mx > m + 8.0f)) {
            const float top = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - top);   // the first time 2^-inf, onto zeros
            m = top;
            l *= alpha;
            lr *= alpha;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int r = 0; r < 16; ++r) o[mt][r] *= alpha;
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], mul, -m));
            l += s[r];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            (&p0.u.x)[e] = E::pack(s[2 * e], s[2 * e + 1]);
            (&p1.u.x)[e] = E::pack(s[8 + 2 * e], s[8 + 2 * e + 1]);
            lr = E::sum2((&p1.u.x)[e], E::sum2((&p0.u.x)[e], lr));
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            U4 v0, v1;
            read_transposed<D>(v0, v1, voff + at, (voff + at) ^ T::FLIP, mt);
            o[mt] = E::mfma(v0, p0, o[mt]);
            o[mt] = E::mfma(v1, p1, o[mt]);
        }
    };

    for (int st = 0; st < nst; ++st) {
        // this wave's loads of the stage are here: at most those of the next one are younger
        if (NBUF > 2 && st + 1 < nst) __builtin_amdgcn_s_waitcnt(vm_wait(2 * LPW));
        else __builtin_amdgcn_s_waitcnt(vm_wait(0));
        __syncthreads();                              // every wave's are, and the buffer of stage st - 1 has been read
        if (st + NBUF - 1 < nst) dma_stage(st + NBUF - 1);
        if (st * S::ROWS + wave * 32 < nkeys) tile((st % NBUF) * S::BYTES + wave * T::BYTES, st * S::ROWS + wave * 32);
    }
    {
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_int(l), __float_as_int(l), false, false);
        l = __int_as_float(sw[0]) + __int_as_float(sw[1]);
        const auto su = __builtin_amdgcn_permlane32_swap(__float_as_int(lr), __float_as_int(lr), false, false);
        lr = __int_as_float(su[0]) + __int_as_float(su[1]);
    }

    // ---- the waves' results meet in LDS: row by row, channels in order
    constexpr int P = D + 4;                      // floats from one row to the next
    static_assert(NW * 32 * P * 4 <= S::TOTAL, "room for the results");
    float* const meet = reinterpret_cast<float*>(smem);
    __shared__ float sm_[NW][32], sl_[NW][32], sr_[NW][32];
    __syncthreads();                              // the last stage has been read
    if (hf == 0) {
        sm_[wave][l32] = m;
        sl_[wave][l32] = l;
        sr_[wave][l32] = lr;
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int r4 = 0; r4 < (D == 16 ? 2 : 4); ++r4)
            *reinterpret_cast<float4*>(meet + (wave * 32 + l32) * P + mt * 32 + 8 * r4 + 4 * hf) =
                make_float4(o[mt][4 * r4], o[mt][4 * r4 + 1], o[mt][4 * r4 + 2], o[mt][4 * r4 + 3]);
    }
    __syncthreads();
    constexpr int TPR = 2 * NW, EACH = D / TPR;       // threads of a row, channels of a thread
    const int rr = tid / TPR, c0 = (tid % TPR) * EACH;
    const long long r = blk * BM + rr;
    if (r >= rows) return;
    const int i = divide((int)r, a.G, a.by_g), g = (int)r - i * a.G;
    const size_t at = (size_t)(qs.from + i) * a.H + kh * a.G + g;
    const bool counts = r < live;
    float top = sm_[0][rr];
#pragma unroll
    for (int k = 1; k < NW; ++k) top = fmaxf(top, sm_[k][rr]);
    float w[NW], sum = 0.f, rounded = 0.f;
#pragma unroll
    for (int k = 0; k < NW; ++k) {                // a wave without keys has -inf, and so has `top` where all have
        w[k] = sm_[k][rr] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm_[k][rr] - top);
        sum += w[k] * sl_[k][rr];
        rounded += w[k] * sr_[k][rr];
    }
    float y[EACH];
#pragma unroll
    for (int c = 0; c < EACH; ++c) {
        y[c] = 0.f;
#pragma unroll
        for (int k = 0; k < NW; ++k)
            if (w[k] != 0.f) y[c] += w[k] * meet[(k * 32 + rr) * P + c0 + c];
    }
    if (!counts) sum = 0.f;
    if (SPLIT) {
        const size_t pa = (size_t)part * a.n_q * a.H + at;
        if (tid % TPR == 0) a.part_ml[pa] = make_float2(sum > 0.f ? top : -INFINITY, rounded);
        if (a.lse && tid % TPR == 0) a.part_l[pa] = sum;
        if (sum > 0.f) {
#pragma unroll
            for (int c = 0; c < EACH; c += 2) *reinterpret_cast<float2*>(a.part_o + pa * D + c0 + c) = make_float2(y[c], y[c + 1]);
        }
        return;
    }
    const float inv = sum > 0.f ? 1.0f / rounded : 0.f;
    if (a.lse && tid % TPR == 0) a.lse[at] = sum > 0.f ? (top + __log2f(sum)) * LN2 : -INFINITY;
#pragma unroll
    for (int c = 0; c < EACH; c += 2) {
        const uint32_t pair = sum > 0.f ? E::pack(y[c] * inv, y[c + 1] * inv) : 0u;
        *reinterpret_cast<uint32_t*>(a.out + at * D + c0 + c) = pair;
    }
}

// The parts of every (row, head): D / 4 threads with four channels each, GROUPS times over where there are many parts: every group takes each
// GROUPS-th part and they meet in LDS. With the kernel in front, one query over 60000 states of 8 x 128 channels 55 us, 110 with one group;
// four queries over 3000 of 8 x 64 12 and 18.
template <int D, bool F16, int GROUPS>
__global__ __launch_bounds__(256) void k_cross_join(CrossArgs a)
{
    constexpr int TPR = D / 4, ROWS = 256 / (TPR * GROUPS);
    struct Sums {
        float top, sum, whole, y[4];                  // the parts' largest score, sums relative to it
    };
    __shared__ Sums meet[GROUPS > 1 ? GROUPS - 1 : 1][ROWS * TPR];
    const int x = threadIdx.x % (ROWS * TPR), k = threadIdx.x / (ROWS * TPR);
    const long long n = (long long)a.n_q * a.H, at = (long long)blockIdx.x * ROWS + x / TPR;
    const int c = (x % TPR) * 4;
    // rows behind the last segment, or before the first, belong to nobody: they stay as they were
    const long long q = min(at, n - 1) / a.H;
    const bool has = at < n && q >= offset_of(a.q_offsets, a.n_q, 0) && q < offset_of(a.q_offsets, a.n_q, a.segments);
    Sums s = {-INFINITY, 0.f, 0.f, {0.f, 0.f, 0.f, 0.f}};
    if (has) {
#pragma unroll 4
        for (int p = k; p < a.parts; p += GROUPS) s.top = fmaxf(s.top, a.part_ml[p * n + at].x);
#pragma unroll 4
        for (int p = k; p < a.parts; p += GROUPS) {
            const float2 ml = a.part_ml[p * n + at];
            if (ml.x == -INFINITY) continue;          // no keys in this part: nothing was stored
            const float w = __builtin_amdgcn_exp2f(ml.x - s.top);
            const float4 o = *reinterpret_cast<const float4*>(a.part_o + (p * n + at) * D + c);
            s.sum += w * ml.y;
            if (a.lse) s.whole += w * a.part_l[p * n + at];
            s.y[0] += w * o.x;
            s.y[1] += w * o.y;
            s.y[2] += w * o.z;
            s.y[3] += w * o.w;
        }
    }
    if (GROUPS > 1) {
        if (k > 0) meet[k - 1][x] = s;
        __syncthreads();
        if (k > 0) return;
        float top = s.top;
#pragma unroll
        for (int g = 0; g < GROUPS - 1; ++g) top = fmaxf(top, meet[g][x].top);
        Sums all = {top, 0.f, 0.f, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const Sums t = g == 0 ? s : meet[g > 0 ? g - 1 : 0][x];
            const float w = t.top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(t.top - top);
            all.sum += w * t.sum;
            all.whole += w * t.whole;
#pragma unroll
            for (int e = 0; e < 4; ++e) all.y[e] += w * t.y[e];
        }
        s = all;
    }
    if (!has) return;
    const float inv = s.sum > 0.f ? 1.0f / s.sum : 0.f;
    if (a.lse && c == 0) a.lse[at] = s.sum > 0.f ? (s.top + __log2f(s.whole)) * LN2 : -INFINITY;
    *reinterpret_cast<uint2*>(a.out + at * D + c) =
        make_uint2(Half<F16>::pack(s.y[0] * inv, s.y[1] * inv), Half<F16>::pack(s.y[2] * inv, s.y[3] * inv));
}

template <int D, bool F16, int GROUPS>
hipError_t join(const CrossArgs& a, hipStream_t stream)
{
    constexpr int ROWS = 256 / (D / 4 * GROUPS);
    k_cross_join<D, F16, GROUPS><<<(unsigned)(((long long)a.n_q * a.H + ROWS - 1) / ROWS), 256, 0, stream>>>(a);
    return hipGetLastError();
}

template <int D, bool F16>
hipError_t launch(const CrossArgs& a, hipStream_t stream)
{
    const unsigned grid = cross_grid((long long)a.slots * a.parts, a.K, a.turn), few_threads = 64 * FewStage<D>::WAVES;
    const bool split = a.parts > 1;
    if (a.few) {
        if (split) k_cross_few<D, F16, true><<<grid, few_threads, 0, stream>>>(a);
        else k_cross_few<D, F16, false><<<grid, few_threads, 0, stream>>>(a);
    } else if (split) {
        if (a.lse) k_cross<D, F16, true, true><<<grid, 256, 0, stream>>>(a);
        else k_cross<D, F16, true, false><<<grid, 256, 0, stream>>>(a);
    } else {
        if (a.lse) k_cross<D, F16, false, true><<<grid, 256, 0, stream>>>(a);
        else k_cross<D, F16, false, false><<<grid, 256, 0, stream>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !split) return e;
    return a.parts < 4 ? join<D, F16, 1>(a, stream) : join<D, F16, 8>(a, stream);
}

template <int D>
hipError_t launch_typed(const CrossArgs& a, hipStream_t stream)
{
    return a.f16 ? launch<D, true>(a, stream) : launch<D, false>(a, stream);
}

}  // namespace

CrossPlan cross_plan(long long n_q, long long n_kv, int segments, long long max_q, long long max_kv, int heads, int kv_heads, int head_dim, bool backward)
{
    constexpr long long CUS = 256;
    const int group = heads / kv_heads;
    CrossPlan p = {};
    const long long rows = n_q * group;               // of one key/value head
    p.few = max_q * group <= 32 && !backward;
    const int block_shift = p.few ? 5 : 7;            // the tile of one wave, or of four
    // Parts of 256 keys at least. Single rows: where there are fewer than two workgroups per compute unit, until there are about three (the
    // loads of a cache in flight). Rows' blocks: only until every compute unit has one: 4096 x 300 keys of 8 x 32 channels (256 blocks)
    // 8.0 us, 14.4 with three; 512 x 8000 of 8 x 128 (32 blocks) 37 and 56; 2000 x 4000 of 8 x 64 (128 blocks) 38 and 40.
    long long work = (rows + (1ll << block_shift) - 1) >> block_shift;
    if (work < segments) work = segments;
    const long long blocks = work * kv_heads;
    long long parts = 1;
    if (blocks < (p.few ? 2 * CUS : CUS)) {
        parts = ((p.few ? 3 * CUS : CUS) + blocks - 1) / blocks;
        const long long most = (max_kv + 255) / 256;
        if (parts > most) parts = most;
        if (parts < 1) parts = 1;
    }
    p.chunk = (int)(((max_kv + parts - 1) / parts + 127) / 128 * 128);
    if (p.chunk < 128) p.chunk = 128;
    p.parts = (int)((max_kv + p.chunk - 1) / p.chunk);
    if (p.parts < 1) p.parts = 1;
    // a workgroup takes a run of row blocks while that leaves a dozen of them per compute unit
    p.run_shift = block_shift;
    if (!p.few && p.parts == 1)
        while (p.run_shift < block_shift + 3 && (blocks >> (p.run_shift - block_shift + 1)) >= 12 * CUS) ++p.run_shift;
    p.slots = (int)((rows >> p.run_shift) + segments);
    if (!backward) return p;
    if (((head_dim == 16 && max_kv <= 128) || (head_dim == 32 && max_kv <= 96)) && n_q > 0 && n_kv > 0) {   // every key's gradients in registers: one kernel
        p.short_tiles = (int)((max_kv + 31) / 32);
        p.parts = 1;
        p.kv_slots = segments;
        // two workgroups per compute unit; 256 rows each, two tiles a wave, at least
        const long long all = (long long)segments * kv_heads, most = (max_q * group + 255) / 256;
        long long row_parts = (2 * CUS + all - 1) / all;
        if (row_parts > most) row_parts = most;
        p.row_chunk = (int)(((max_q * group + row_parts - 1) / row_parts + 127) / 128 * 128);
        p.row_parts = (int)((max_q * group + p.row_chunk - 1) / p.row_chunk);
        return p;
    }
    p.kv_slots = (int)(n_kv / 128 + segments);
    const long long kv_work = n_kv / 128 > segments ? n_kv / 128 : segments;
    long long row_parts = 1;
    // fewer than two workgroups per compute unit: until there are one and a half (two segments of 700 rows and 2000 keys, 32 heads of 128
    // channels on 8: 216 us for all gradients, 246 with three; 50000 rows and 500 keys, 8 of 128: 461 and 501)
    if (kv_work * kv_heads < 2 * CUS) {
        row_parts = (3 * CUS / 2 + kv_work * kv_heads - 1) / (kv_work * kv_heads);
        const long long most = (max_q * group + 255) / 256;
        if (row_parts > most) row_parts = most;
        if (row_parts < 1) row_parts = 1;
    }
    const long long chunk = ((max_q * group + row_parts - 1) / row_parts + 127) / 128 * 128;
    p.row_chunk = (int)(chunk < 128 ? 128 : chunk);
    p.row_parts = (int)((max_q * group + p.row_chunk - 1) / p.row_chunk);
    if (p.row_parts < 1) p.row_parts = 1;
    return p;
}

hipError_t cross_launch(const CrossArgs& a, int head_dim, hipStream_t stream)
{
    switch (head_dim) {
        case 16: return launch_typed<16>(a, stream);
        case 32: return launch_typed<32>(a, stream);
        case 64: return launch_typed<64>(a, stream);
        case 128: return launch_typed<128>(a, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace f3d
