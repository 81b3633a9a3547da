// What the kernels of ragged batches share: sequences of different lengths in one list of rows, pages of a cache that a table names.
#pragma once

#include "common.h"
#include "paged_ranges.h"

namespace sdv2 {

// Rows q_start[s] .. q_start[s + 1] - 1 are the new tokens of sequence s, the last of its kv_len[s] tokens; token j lies in page
// table[s * table_stride + (j >> page_shift)] at slot j & (P - 1).  An entry outside [0, n_pages) names no page.
struct RaggedArgs {
    const int* q_start;       // [n_seqs + 1]
    const int* kv_len;        // [n_seqs]
    const int* table;         // [n_seqs][table_stride]
    int n_seqs, n_tokens, table_stride;
    int page_shift, n_pages, kv_heads;
};

// First of n_seqs sequences whose end, ends(s + 1), is behind t (n_seqs: none), found by the whole wave; ends ascends.  Each round 64
// lanes look at the ends of 64 runs of sequences at once, so that 64 sequences take one load and 4096 two, one behind the other,
// where a bisection takes 6 and 12.
template <typename F>
__device__ __forceinline__ int find_sequence(int n_seqs, int t, F&& ends) {
    const int lane = threadIdx.x & 63;
    int first = 0, n = n_seqs;                               // it is one of first .. first + n, the last meaning "behind these"
    while (n > 0) {
        const int run = (n + 63) >> 6, behind = first + n;   // sequences per lane
        const int end = min(first + (lane + 1) * run, behind);
        const bool before = first + lane * run < behind && ends(end) <= t;        // t is behind this lane's run
        first = min(behind, first + __builtin_popcountll(__builtin_amdgcn_ballot_w64(before)) * run);
        n = run == 1 ? 0 : min(run, behind - first);
        if (n > 0) --n;                                      // that run's end is behind t: its last sequence needs no look
    }
    return __builtin_amdgcn_readfirstlane(first);
}

// That sequence with its rows and one more number of it.  Up to 64 sequences are looked at by a lane each, which fetches all of
// it at once: a second round of loads behind the first is 0.7 us of a launch of a few.
struct Sequence {
    int index, q0, n, more;
};
template <typename F>
__device__ __forceinline__ Sequence sequence_at(const int* q_start, const int* more, int n_seqs, int t, F&& ends) {
    Sequence s;
    if (n_seqs <= 64) {
        const int lane = threadIdx.x & 63, i = min(lane, n_seqs - 1);
        const int first = q_start[i], last = q_start[i + 1], other = more[i];
        s.index = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < n_seqs && ends(last, i + 1) <= t));
        const int at = min(s.index, n_seqs - 1);
        s.q0 = __builtin_amdgcn_readlane(first, at);
        s.n = __builtin_amdgcn_readlane(last, at) - s.q0;
        s.more = __builtin_amdgcn_readlane(other, at);
        return s;
    }
    s.index = find_sequence(n_seqs, t, [&](int i) { return ends(q_start[i], i); });
    const int at = min(s.index, n_seqs - 1);
    s.q0 = __builtin_amdgcn_readfirstlane(q_start[at]);
    s.n = __builtin_amdgcn_readfirstlane(q_start[at + 1]) - s.q0;
    s.more = __builtin_amdgcn_readfirstlane(more[at]);
    return s;
}

// Eight bf16 from eight e4m3 (exact).
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ bf16x8 widen_e4m3(u32x2 v) {
    bf16x8 out;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[w], 1.0f, false);
        const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[w], 1.0f, true);
        out[4 * w] = lo[0];
        out[4 * w + 1] = lo[1];
        out[4 * w + 2] = hi[0];
        out[4 * w + 3] = hi[1];
    }
    return out;
}

// ---------------------------------------------------------------- launchers (host side)
// Norm of each head and rotation of q and k, out of place or in place, or into pages together with v.
struct TurnArgs {
    const bf16 *q, *k, *v;            // rows of heads of 128; q or k may be null (no heads), v is null without pages
    bf16 *q_out, *k_out;              // k_out is null with pages
    long long q_stride, k_stride, v_stride, q_out_stride, k_out_stride;     // elements from row to row
    int rows, q_heads, k_heads;
    const float *g_q, *g_k;           // gains [128] of the norm; null: no norm
    float eps;
    int axes, halves;                 // axes 0: no rotation
    const int* pos;                   // [rows][axes]
    double turns[kHeadDim / 2];       // of each pair: revolutions per unit of its axis' position
    // with pages
    RaggedArgs batch;
    void *k_pages, *v_pages;          // [n_pages][kv_heads][P][128] bf16 or e4m3
    int e4m3;
    float k_inverse, v_inverse;       // 1 / scale (1 for bf16)
};
hipError_t launch_turn(const TurnArgs& a, hipStream_t s);

struct PagedAttnArgs {
    RaggedArgs batch;
    MaskArgs mask;
    const bf16* q;
    bf16* o;
    long long q_stride, o_stride;
    const void *k_pages, *v_pages;
    int q_heads, group;               // query heads, and those of one key head
    float v_scale;
    float* part_o;                    // [parts][n_tokens * q_heads][128]
    float* part_ml;                   // [parts][n_tokens * q_heads][2]
    int parts, part_tiles;            // key tiles of a part; the last part takes what is left
    FastDiv by_group, by_tiles, by_heads;     // set by the launcher, as is the number of row tiles
    int row_tiles;
    unsigned n_wg;
};
struct PagedAttnPlan {
    int rows;                         // rows (tokens times group) of a workgroup: 32, keys over its waves; 128 or 256, rows over its waves
    int parts, part_tiles;
};
PagedAttnPlan plan_paged_attention(const RaggedArgs& b, const MaskArgs& mask, int q_heads, int max_q_len, int max_kv_len, int e4m3);
// Tuning hooks: rows of a workgroup (32, 128, 256) and parts of the key range (0 = planner); -1 leaves a value as is.
void set_paged_overrides(int rows, int parts);
hipError_t launch_paged_attention(const PagedAttnArgs& a, const PagedAttnPlan& plan, int e4m3, hipStream_t s);

struct LoraArgs {
    const bf16* x;                    // [rows][x_stride], K of them
    const bf16* a;                    // [n_adapters][rank][K]
    const bf16* b;                    // [n_adapters][N][rank]
    const float* scale;               // [n_adapters] or null
    const int* adapter;               // [n_seqs]
    const int* q_start;               // [n_seqs + 1]
    const void* y;
    void* out;
    long long x_stride, y_stride, out_stride;
    int n_seqs, n_tokens, K, N, rank, n_adapters, fp32;
    float* u;                         // scale x A^T, K in parts: [parts][slots][u_ranks / 4][16 tokens][4]
    int u_ranks;                      // rank rounded up to 16
    int parts;
    int slots;                        // sixteens of tokens of one sequence each; 0: u is [parts][n_tokens][u_ranks]
};
// whether the second product takes a sequence's tokens one by one, and u has a row for each (slots = 0)
bool lora_by_tokens(int max_q_len);
// parts of K: n_seqs, n_tokens, max_q_len, K, rank
int lora_parts(int n_seqs, int n_tokens, int max_q_len, int K, int rank);
hipError_t launch_lora(const LoraArgs& a, int max_q_len, hipStream_t s);

}  // namespace sdv2
