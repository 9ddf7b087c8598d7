// Internal interface between the C ABI (flash3d_api.hip) and the cross attention kernels (cross.hip, cross_bwd.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn.h"

namespace f3d {

struct CrossArgs {
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    const int32_t* q_offsets;   // [segments + 1]
    const int32_t* kv_offsets;
    const int32_t* q_lens;      // null, or [segments]
    const int32_t* kv_lens;
    int n_q, n_kv;
    int segments;
    int H, K, G;                // heads, key/value heads, heads that share one of these
    Divide by_g;                // rows of a segment, heads that share keys counted one by one, by G
    float s_mul;                // softmax scale * log2(e), multiplied onto the product
    uint16_t* out;
    float* lse;                 // null, or [n_q, H]
    int f16;
    int few;                    // the form for few query rows
    int run_shift;              // a workgroup takes 2^run_shift rows of a segment
    int slots;                  // such runs over all segments (upper bound, surplus workgroups exit)
    int turn;                   // consecutive pieces of work that go to one XCD
    int parts;                  // parts the keys of a segment are split into
    int chunk;                  // keys of a part
    float* part_o;              // [parts][n_q * H][head_dim], sums of a part relative to its largest score
    float2* part_ml;            // [parts][n_q * H]: that score (log2 units), sum of the rounded exponentials
    float* part_l;              // [parts][n_q * H]: their sum as they are, where lse is wanted
};

// consecutive pieces (row blocks x parts x key/value heads) to an XCD: the heads of up to eight blocks; the grid is whole rounds of eight turns
inline int cross_turn(long long blocks, int kv_heads) { return kv_heads * (int)(blocks < 64 ? 1 : blocks < 512 ? blocks / 64 : 8); }
inline unsigned cross_grid(long long blocks, int kv_heads, int turn) { return (unsigned)((blocks * kv_heads + 8ll * turn - 1) / (8ll * turn) * 8 * turn); }

struct CrossBwdArgs {
    CrossArgs f;                // parts and chunk of the query gradient's kernel
    const uint16_t* dout;
    float* dsum;                // [n_q, H]: sum over the head's channels of dout * out
    uint16_t* dq;
    uint16_t* dk;
    uint16_t* dv;
    float scale;
    float* part_dq;             // [parts][n_q * H][head_dim], where parts > 1
    int short_tiles;            // 0: the two kernels; else one, for segments of up to 32 short_tiles keys
    int kv_turn;
    int kv_slots;               // blocks of 128 keys over all segments
    int row_parts;              // parts the query rows of a segment are split into
    int row_chunk;              // rows of a part
    float* part_dkv;            // [2][row_parts][n_kv * K][head_dim], where row_parts > 1
};

// What a call takes: a rule on sizes the host knows
struct CrossPlan {
    int few, run_shift, slots, parts, chunk;
    int short_tiles, kv_slots, row_parts, row_chunk;   // backward
};
CrossPlan cross_plan(long long n_q, long long n_kv, int segments, long long max_q, long long max_kv, int heads, int kv_heads, int head_dim, bool backward);

hipError_t cross_launch(const CrossArgs& a, int head_dim, hipStream_t stream);
hipError_t cross_bwd_short_launch(const CrossBwdArgs& a, int head_dim, int tiles, hipStream_t stream);
hipError_t cross_bwd_launch(const CrossBwdArgs& a, int head_dim, hipStream_t stream);

}  // namespace f3d
