// Low-rank adapters of many requests beside a shared projection:  out = y + scale (x A^T) B^T, each sequence with its own A [r, K],
// B [N, r] and scale, or none.
//
// Memory bound: x, y, out and the adapters' matrices once, 2 r (K + N) flops a row.  Two launches with u = scale x A^T between them; both
// are products on 16x16x32 matrix instructions whose fragments come straight from memory (sixteen rows, 64 bytes each), since
// nothing is used often enough to pay for its way through LDS.
//   u: computed transposed, ranks as rows and tokens as columns.  A workgroup has 16 or 32 tokens of one sequence and 16 RT ranks; its eight
//     waves take pieces of 64 of K in turn and add up through LDS.  u is left as two bf16 numbers per value, high and low (u = high + low
//     to 2^-17: as one bf16 its rounding would be the largest error of an fp32 result).
//   out: columns of out as rows, tokens as columns, y as the accumulator's start.  The rows of four instructions are interleaved so that a
//     lane ends up with sixteen columns next to each other of its token.
#include "ragged.h"

namespace sdv2 {

namespace {

// Tokens of one sequence that a workgroup has, and its adapter.  Tiles are numbered as the row tiles of the paged attention: those of
// sequence s start at floor(q_start[s] / tokens) + s.
struct Tile {
    int first, count, adapter;        // first row of the batch, rows (<= tokens), adapter or -1
};
template <int TOKENS>
__device__ __forceinline__ bool locate(const LoraArgs& a, int tile, Tile* t) {
    const int s = find_sequence(a.n_seqs, tile, [&](int i) { return a.q_start[i] / TOKENS + i; });
    if (s >= a.n_seqs) return false;
    const int q0 = __builtin_amdgcn_readfirstlane(a.q_start[s]), n = __builtin_amdgcn_readfirstlane(a.q_start[s + 1]) - q0;
    const int id = __builtin_amdgcn_readfirstlane(a.adapter[s]);
    if (q0 < 0 || n < 0 || n > a.n_tokens - q0) return false;         // not a batch: touch nothing
    const int at = (tile - q0 / TOKENS - s) * TOKENS;
    if (at >= n) return false;
    t->first = q0 + at;
    t->count = min(TOKENS, n - at);
    t->adapter = (unsigned)id < (unsigned)a.n_adapters ? id : -1;
    return true;
}

constexpr int kDownWaves = 8;

template <int NT, int RT>
__global__ __launch_bounds__(64 * kDownWaves) void lora_down_kernel(LoraArgs a, unsigned groups) {
    __shared__ f32x4 parts[kDownWaves][RT * NT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, lk = lane >> 4;
    const unsigned tile = blockIdx.x / groups;
    Tile t;
    if (!locate<16 * NT>(a, (int)tile, &t) || t.adapter < 0) return;
    const int rank0 = (int)(blockIdx.x - tile * groups) * (16 * RT);

    const bf16 *wp[RT], *xp[NT];
#pragma unroll
    for (int i = 0; i < RT; ++i) wp[i] = a.a + ((long long)t.adapter * a.rank + min(rank0 + 16 * i + l15, a.rank - 1)) * a.K + 8 * lk;
#pragma unroll
    for (int i = 0; i < NT; ++i) xp[i] = a.x + (long long)(t.first + min(16 * i + l15, t.count - 1)) * a.x_stride + 8 * lk;
    f32x4 acc[RT][NT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // pieces of 64 numbers (a line of 128 bytes in a row); several at once, so that their loads are in flight together
    constexpr int kAtOnce = RT * NT == 1 ? 5 : RT + NT <= 4 ? 3 : 2;
    const int pieces = a.K >> 6;
    for (int p0 = wave; p0 < pieces; p0 += kDownWaves * kAtOnce) {
        bf16x8 w[kAtOnce][2][RT], x[kAtOnce][2][NT];
#pragma unroll
        for (int c = 0; c < kAtOnce; ++c) {
            const int at = min(p0 + kDownWaves * c, pieces - 1) * 64;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < RT; ++i) w[c][h][i] = *reinterpret_cast<const bf16x8*>(wp[i] + at + 32 * h);
#pragma unroll
                for (int j = 0; j < NT; ++j) x[c][h][j] = *reinterpret_cast<const bf16x8*>(xp[j] + at + 32 * h);
            }
        }
#pragma unroll
        for (int c = 0; c < kAtOnce; ++c) {
            if (p0 + kDownWaves * c >= pieces) break;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[c][h][i], x[c][h][j], acc[i][j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) parts[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    const float scale = a.scale != nullptr ? a.scale[t.adapter] : 1.0f;
    for (int b = wave; b < RT * NT; b += kDownWaves) {
        f32x4 u = parts[0][b][lane];
#pragma unroll
        for (int k = 1; k < kDownWaves; ++k) u += parts[k][b][lane];
        const int rank = rank0 + 16 * (b / NT) + 4 * lk, token = 16 * (b % NT) + l15;      // four ranks of one token
        if (token >= t.count || rank >= a.u_ranks) continue;
        bf16x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float v = rank < a.rank ? u[e] * scale : 0.0f;
            hi[e] = (bf16)v;
            lo[e] = (bf16)(v - (float)hi[e]);
        }
        bf16* const to = a.u + (long long)(t.first + token) * 2 * a.u_ranks + rank;
        *reinterpret_cast<bf16x4*>(to) = hi;
        *reinterpret_cast<bf16x4*>(to + a.u_ranks) = lo;
    }
}

// Sixteen columns of y or out.
template <typename T>
struct Sixteen;
template <>
struct Sixteen<float> {
    f32x4 x[4];
    __device__ __forceinline__ void load(const float* p) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = reinterpret_cast<const f32x4*>(p)[i];
    }
    __device__ __forceinline__ f32x4 four(int i) const { return x[i]; }
    static __device__ __forceinline__ void store(float* p, const f32x4 (&v)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<f32x4*>(p)[i] = v[i];
    }
};
template <>
struct Sixteen<bf16> {
    bf16x8 x[2];
    __device__ __forceinline__ void load(const bf16* p) {
        x[0] = reinterpret_cast<const bf16x8*>(p)[0];
        x[1] = reinterpret_cast<const bf16x8*>(p)[1];
    }
    __device__ __forceinline__ f32x4 four(int i) const {
        f32x4 r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = (float)x[i >> 1][4 * (i & 1) + e];
        return r;
    }
    static __device__ __forceinline__ void store(bf16* p, const f32x4 (&v)[4]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (bf16)v[2 * h + (e >> 2)][e & 3];
            reinterpret_cast<bf16x8*>(p)[h] = o;
        }
    }
};

// KS: steps of 32 ranks.  A wave has NB blocks of 64 columns and the tile's tokens, sixteen at a time.
template <typename T, int KS, int NB, int TOKENS>
__global__ __launch_bounds__(256) void lora_up_kernel(LoraArgs a, unsigned groups) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, lk = lane >> 4;
    const unsigned tile = blockIdx.x / groups;
    const int block0 = ((int)(blockIdx.x - tile * groups) * 4 + wave) * NB, blocks = a.N >> 6;
    if (block0 >= blocks) return;
    Tile t;
    if (!locate<TOKENS>(a, (int)tile, &t)) return;
    const T* const y = static_cast<const T*>(a.y);
    T* const out = static_cast<T*>(a.out);
    if (t.adapter < 0) {
        if (a.y == a.out) return;
        for (int i = 0; i < t.count; i += 16)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int n = (block0 + b) * 64 + 16 * lk;
                if (i + l15 >= t.count || block0 + b >= blocks) continue;
                Sixteen<T> v;
                v.load(y + (long long)(t.first + i + l15) * a.y_stride + n);
                const f32x4 same[4] = {v.four(0), v.four(1), v.four(2), v.four(3)};
                Sixteen<T>::store(out + (long long)(t.first + i + l15) * a.out_stride + n, same);
            }
        return;
    }
    // row r of instruction m is column 16 (r / 4) + 4 m + r % 4 of the block
    const bf16x8 none = {};
    bf16x8 w[NB][4][KS];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const int n = min(block0 + b, blocks - 1) * 64 + 16 * (l15 >> 2) + 4 * m + (l15 & 3);
            const bf16* const p = a.b + ((long long)t.adapter * a.N + n) * a.rank;
#pragma unroll
            for (int k = 0; k < KS; ++k) w[b][m][k] = 32 * k + 8 * lk < a.rank ? *reinterpret_cast<const bf16x8*>(p + 32 * k + 8 * lk) : none;
        }
    for (int i = 0; i < t.count; i += 16) {
        const bool live = i + l15 < t.count;
        const long long row = t.first + min(i + l15, t.count - 1);
        Sixteen<T> v[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
            if (live) v[b].load(y + row * a.y_stride + min(block0 + b, blocks - 1) * 64 + 16 * lk);
        bf16x8 u[2][KS];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int k = 0; k < KS; ++k) u[h][k] = *reinterpret_cast<const bf16x8*>(a.u + (row * 2 + h) * a.u_ranks + 32 * k + 8 * lk);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            f32x4 acc[4];
#pragma unroll
            for (int m = 0; m < 4; ++m) acc[m] = v[b].four(m);
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int m = 0; m < 4; ++m) acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[b][m][k], u[h][k], acc[m], 0, 0, 0);
            if (live && block0 + b < blocks) Sixteen<T>::store(out + row * a.out_stride + (block0 + b) * 64 + 16 * lk, acc);
        }
    }
}

template <typename T, int NB, int TOKENS>
void launch_up(const LoraArgs& a, hipStream_t s) {
    const unsigned groups = (unsigned)(a.N / 64 + 4 * NB - 1) / (4 * NB);
    const dim3 grid(groups * (unsigned)(a.n_tokens / TOKENS + a.n_seqs));
    switch (a.u_ranks / 32) {
        case 1: hipLaunchKernelGGL((lora_up_kernel<T, 1, NB, TOKENS>), grid, dim3(256), 0, s, a, groups); break;
        case 2: hipLaunchKernelGGL((lora_up_kernel<T, 2, NB, TOKENS>), grid, dim3(256), 0, s, a, groups); break;
        case 3: hipLaunchKernelGGL((lora_up_kernel<T, 3, NB, TOKENS>), grid, dim3(256), 0, s, a, groups); break;
        default: hipLaunchKernelGGL((lora_up_kernel<T, 4, NB, TOKENS>), grid, dim3(256), 0, s, a, groups); break;
    }
}
template <int NT, int RT>
void launch_down(const LoraArgs& a, hipStream_t s) {
    const unsigned groups = (unsigned)(a.u_ranks + 16 * RT - 1) / (16 * RT);
    hipLaunchKernelGGL((lora_down_kernel<NT, RT>), dim3(groups * (unsigned)(a.n_tokens / (16 * NT) + a.n_seqs)), dim3(64 * kDownWaves), 0, s, a, groups);
}

}  // namespace

hipError_t launch_lora(const LoraArgs& a, int max_q_len, hipStream_t s) {
    const bool few = max_q_len <= 16;
    if (few) launch_down<1, 1>(a, s);
    else if (a.n_tokens < 4096 || a.u_ranks < 64) launch_down<2, 2>(a, s);
    else launch_down<2, 4>(a, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.fp32) few ? launch_up<float, 2, 16>(a, s) : launch_up<float, 1, 64>(a, s);
    else few ? launch_up<bf16, 2, 16>(a, s) : launch_up<bf16, 1, 64>(a, s);
    return hipGetLastError();
}

}  // namespace sdv2
