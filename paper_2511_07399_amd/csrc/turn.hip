// Norms of queries and keys for each head with the position rotation, on their own and on the way into a paged cache.
//
//   y = x / sqrt(mean(x^2) + eps) g  over the 128 numbers of a head (no gain: y = x), then pair j of the head, numbers (2j, 2j + 1)
//   or (j, j + 64), turned by position times frequency.
//
// HBM bound: every number is read once and written once, some sixty vector instructions per eight of them in between.  Sixteen
// lanes hold a head (16 bytes each), so a wave load is four heads (1 KB); the sum of squares stays inside a row of sixteen lanes
// and is formed by cross-lane moves of the vector unit.  In the (j, j + 64) order a number's partner is eight lanes away in the
// same row, one such move.  4680 rows of 40 + 40 heads, three axes: 191.7 MB in 42.4 us, 4.5 TB/s (a copy's 4.2 to 4.5); 6240 rows of
// 12 heads of q, k and v to 8-bit pages: 95.8 MB in 23.2 us, 4.1 TB/s; one token 2.6 us, which is a launch.
//
// The angle is position x turns in double (32 bits lose it: at position 10^6 the fastest pair's angle would be off by 0.06), of which
// the fraction of a turn goes to a single-precision sine and cosine.  Lane j forms pair j; the lanes fetch theirs by shuffle.
#include "ragged.h"

namespace sdv2 {

namespace {

// Sum over the row of sixteen lanes that a head occupies, in all of them.
__device__ __forceinline__ float head_sum(float v) {
    v += dpp_f<0x128>(v);        // row_ror:8
    v += dpp_f<0x124>(v);        // row_ror:4
    v += dpp_f<0x4E>(v);         // quad_perm [2, 3, 0, 1]
    return v + dpp_f<0xB1>(v);   // quad_perm [1, 0, 3, 2]
}

// To e4m3, one rounding; beyond its range the largest number, NaN stays.
__device__ __forceinline__ u32x2 pack_e4m3(const float (&x)[8]) {
    float c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = x[e] != x[e] ? x[e] : fminf(fmaxf(x[e], -448.0f), 448.0f);
    u32x2 r;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(c[4 * w], c[4 * w + 1], 0, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(c[4 * w + 2], c[4 * w + 3], v, true);
        r[w] = (unsigned)v;
    }
    return r;
}

// Fours of heads of a row, in the order q, k, v; a wave takes QUADS of them.
template <int QUADS, bool PAGES, bool HALVES>
__global__ __launch_bounds__(256) void turn_kernel(TurnArgs a, int waves_per_row, int q_quads, int k_quads) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int row = wave / waves_per_row;
    if (row >= a.rows) return;
    const int quad0 = (wave - row * waves_per_row) * QUADS;
    const int n_quads = q_quads + k_quads * (PAGES ? 2 : 1);
    const int hl = lane >> 4, c = lane & 15;                   // head of the four, 16-byte piece of the head

    bf16x8 in[QUADS];
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int quad = min(quad0 + i, n_quads - 1);
        const int kind = quad < q_quads ? 0 : quad < q_quads + k_quads ? 1 : 2;
        const int h = (quad - (kind == 0 ? 0 : kind == 1 ? q_quads : q_quads + k_quads)) * 4 + hl;
        const bf16* base = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
        const long long stride = kind == 0 ? a.q_stride : kind == 1 ? a.k_stride : a.v_stride;
        const int heads = kind == 0 ? a.q_heads : a.k_heads;
        in[i] = *reinterpret_cast<const bf16x8*>(base + row * stride + min(h, heads - 1) * kHeadDim + c * 8);
    }

    // where the row's key and value go: its sequence, its place there, the page
    long long slot = -1;                                       // page * kv_heads * P + slot in the page
    if (PAGES) {
        const Sequence s = sequence_at(a.batch.q_start, a.batch.kv_len, a.batch.n_seqs, row, [](int end, int) { return end; });
        if (s.index >= a.batch.n_seqs) return;                 // behind the last sequence: nothing of it is written
        const int at = tokens_of(s.more, a.batch.table_stride, a.batch.page_shift) - s.n + row - s.q0;      // (as the attention reads it)
        const int entry = at >> a.batch.page_shift;
        if (at >= 0 && entry < a.batch.table_stride) {
            const int page = a.batch.table[(long long)s.index * a.batch.table_stride + entry];
            if ((unsigned)page < (unsigned)a.batch.n_pages)
                slot = (((long long)page * a.k_heads) << a.batch.page_shift) + (at & ((1 << a.batch.page_shift) - 1));
        }
    }

    constexpr int P = HALVES ? 8 : 4;                          // pairs of a lane: 8 (c % 8) + e, or 4 c + e
    float cs[P], sn[P];
    if (a.axes > 0) {
        const int axis = a.axes == 1 ? 0 : (lane >= 22) + (lane >= 43);
        const double turns = (double)a.pos[(long long)row * a.axes + axis] * a.turns[lane];
        float s_own, c_own;
        sincospif(2.0f * (float)(turns - rint(turns)), &s_own, &c_own);
#pragma unroll
        for (int e = 0; e < P; ++e) {
            const int pair = HALVES ? 8 * (c & 7) + e : 4 * c + e;
            cs[e] = __shfl(c_own, pair, kWave);
            sn[e] = __shfl(s_own, pair, kWave);
        }
    }

#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int quad = quad0 + i;
        if (quad >= n_quads) return;
        const int kind = quad < q_quads ? 0 : quad < q_quads + k_quads ? 1 : 2;
        const int h = (quad - (kind == 0 ? 0 : kind == 1 ? q_quads : q_quads + k_quads)) * 4 + hl;
        const bool live = h < (kind == 0 ? a.q_heads : a.k_heads);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)in[i][e];
        if (kind < 2) {
            const float* gain = kind == 0 ? a.g_q : a.g_k;
            if (gain != nullptr) {
                auto squares = [&]() {
                    float sq = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sq += x[e] * x[e];
                    return head_sum(sq) * (1.0f / kHeadDim);
                };
                float mean = squares(), eps = a.eps;
                if (__builtin_expect(mean == INFINITY, 0)) {                  // beyond 32 bits: the head times 2^-70, and eps with it
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= 0x1p-70f;
                    mean = squares();
                    eps *= 0x1p-140f;
                }
                const float r = rsqrtf(mean + eps);
                const f32x4 g0 = *reinterpret_cast<const f32x4*>(gain + c * 8), g1 = *reinterpret_cast<const f32x4*>(gain + c * 8 + 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= r * (e < 4 ? g0[e & 3] : g1[e & 3]);
            }
            if (a.axes > 0) {
                if (HALVES) {
                    // the first eight lanes of a head hold u of (u, v), the others v: u c - v s, and v c + u s
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float other = dpp_f<0x128>(x[e]);
                        x[e] = x[e] * cs[e] + (c < 8 ? -other : other) * sn[e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float u = x[2 * e], v = x[2 * e + 1];
                        x[2 * e] = u * cs[e] - v * sn[e];
                        x[2 * e + 1] = u * sn[e] + v * cs[e];
                    }
                }
            }
        }
        if (!live) continue;
        if (PAGES && kind > 0) {
            if (slot < 0) continue;
            const long long at = slot + ((long long)h << a.batch.page_shift);
            void* pages = kind == 1 ? a.k_pages : a.v_pages;
            if (a.e4m3) {
                const float inv = kind == 1 ? a.k_inverse : a.v_inverse;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= inv;
                *reinterpret_cast<u32x2*>(static_cast<unsigned char*>(pages) + at * kHeadDim + c * 8) = pack_e4m3(x);
                continue;
            }
            bf16x8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (bf16)x[e];
            *reinterpret_cast<bf16x8*>(static_cast<bf16*>(pages) + at * kHeadDim + c * 8) = o;
        } else {
            bf16x8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (bf16)x[e];
            bf16* dst = kind == 0 ? a.q_out + row * a.q_out_stride : a.k_out + row * a.k_out_stride;
            *reinterpret_cast<bf16x8*>(dst + h * kHeadDim + c * 8) = o;
        }
    }
}

}  // namespace

hipError_t launch_turn(const TurnArgs& a, hipStream_t s) {
    const bool pages = a.k_pages != nullptr;
    const int q_quads = (a.q_heads + 3) / 4, k_quads = (a.k_heads + 3) / 4;
    const int n = q_quads + k_quads * (pages ? 2 : 1);
    // A wave has four heads up to 16 waves a SIMD, from there on sixteen heads, which share the angles and
    // the look-up of the page.  One four | four of them, us: 48 rows appended 5.1 | 6.2, 333 6.0 | 6.6; rotated, 32 + 8 heads, 400 rows
    // 5.7 | 6.2, 1600 9.8 | 11.1; 3000 rows appended to 8-bit pages 21.5 | 19.1, 9360 of 40 heads 126 | 120; 20 000 rotated 38.7 | 37.7.
    const bool few = (long long)a.rows * n <= 16384;
    const int quads = few ? 1 : 4;
    const int waves_per_row = (n + quads - 1) / quads;
    const dim3 grid((unsigned)(((long long)a.rows * waves_per_row + 3) / 4));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, waves_per_row, q_quads, k_quads); };
    if (few) {
        if (pages) a.halves ? go(turn_kernel<1, true, true>) : go(turn_kernel<1, true, false>);
        else a.halves ? go(turn_kernel<1, false, true>) : go(turn_kernel<1, false, false>);
    } else {
        if (pages) a.halves ? go(turn_kernel<4, true, true>) : go(turn_kernel<4, true, false>);
        else a.halves ? go(turn_kernel<4, false, true>) : go(turn_kernel<4, false, false>);
    }
    return hipGetLastError();
}

}  // namespace sdv2
