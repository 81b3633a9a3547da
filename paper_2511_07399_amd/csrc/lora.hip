// Low-rank adapters of many requests beside a shared projection:  out = y + scale (x A^T) B^T, each sequence with its own A [r, K],
// B [N, r] and scale, or none.
//
// Memory bound: x, y, out and the adapters' matrices once, 2 r (K + N) flops a row.  Two launches with u = scale x A^T between them; both
// are products on 16x16x32 matrix instructions whose fragments come straight from memory (sixteen rows, 64 bytes each), since
// nothing is used often enough to pay for its way through LDS.
//   u: computed transposed, ranks as rows and tokens as columns.  A workgroup has 16 or 32 tokens of one sequence and 16 RT ranks; its eight
//     waves take pieces of 64 of K in turn and add up through LDS.  u is left in 32 bits, and goes to the second product as two or three
//     bf16 numbers that add up to it (kPieces: as one, its rounding would be the result's largest error).
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
    const Sequence s = sequence_at(a.q_start, a.adapter, a.n_seqs, tile, [](int end, int i) { return end / TOKENS + i; });
    const int q0 = s.q0, n = s.n, id = s.more;
    if (s.index >= a.n_seqs || q0 < 0 || n < 0 || n > a.n_tokens - q0) return false;      // (not a batch: touch nothing)
    const int at = (tile - q0 / TOKENS - s.index) * TOKENS;
    if (at < 0 || at >= n) return false;
    t->first = q0 + at;
    t->count = min(TOKENS, n - at);
    t->adapter = (unsigned)id < (unsigned)a.n_adapters ? id : -1;
    return true;
}

constexpr int kDownWaves = 8;
// bf16 numbers that one of u goes to the second product as: each takes off eight bits, and an output of 32 bits shows the 17th
// (four frames of rank 64 against 64 bits: two pieces 1.9e-6 of the output, three 1.2e-7, which is the sum's own).
template <typename T>
constexpr int kPieces = sizeof(T) == 4 ? 3 : 2;

template <int NT, int RT>
__global__ __launch_bounds__(64 * kDownWaves) void lora_down_kernel(LoraArgs a, unsigned groups) {
    __shared__ f32x4 parts[kDownWaves][RT * NT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, lk = lane >> 4;
    const unsigned rest = blockIdx.x / a.parts, part = blockIdx.x - rest * a.parts, tile = rest / groups;
    Tile t;
    if (!locate<16 * NT>(a, (int)tile, &t) || t.adapter < 0) return;
    const int rank0 = (int)(rest - tile * groups) * (16 * RT);
    const float scale = a.scale != nullptr ? a.scale[t.adapter] : 1.0f;

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
    constexpr int kAtOnce = 3;
    const int all = a.K >> 6, pieces = (int)((long long)all * (part + 1) / a.parts);
    for (int p0 = (int)((long long)all * part / a.parts) + wave; p0 < pieces; p0 += kDownWaves * kAtOnce) {
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
        __builtin_amdgcn_sched_barrier(0);       // (left to itself, the compiler puts each load in front of its product)
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
    for (int b = wave; b < RT * NT; b += kDownWaves) {
        f32x4 u = parts[0][b][lane];
#pragma unroll
        for (int k = 1; k < kDownWaves; ++k) u += parts[k][b][lane];
        const int rank = rank0 + 16 * (b / NT) + 4 * lk, token = 16 * (b % NT) + l15;      // four ranks of one token
        if (token >= t.count || rank >= a.u_ranks) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = rank < a.rank ? u[e] * scale : 0.0f;
        *reinterpret_cast<f32x4*>(a.u + ((long long)part * a.n_tokens + t.first + token) * a.u_ranks + rank) = u;
    }
}

// A lane's sixteen columns of a block of 64 of y or out: pieces of 16 bytes such that the four lanes of a token have 64 bytes next to each
// other in each.  Which column of the block instruction m's row r is, goes by that: column(m, r).
template <typename T>
struct Sixteen;
template <>
struct Sixteen<float> {
    f32x4 x[4];
    static __device__ __forceinline__ int column(int m, int r) { return 16 * m + r; }
    __device__ __forceinline__ void load(const float* p, int lk) {
#pragma unroll
        for (int m = 0; m < 4; ++m) x[m] = *reinterpret_cast<const f32x4*>(p + 16 * m + 4 * lk);
    }
    __device__ __forceinline__ f32x4 four(int m) const { return x[m]; }
    static __device__ __forceinline__ void store(float* p, int lk, const f32x4 (&v)[4]) {
#pragma unroll
        for (int m = 0; m < 4; ++m) *reinterpret_cast<f32x4*>(p + 16 * m + 4 * lk) = v[m];
    }
};
template <>
struct Sixteen<bf16> {
    bf16x8 x[2];
    static __device__ __forceinline__ int column(int m, int r) { return 32 * (m >> 1) + 8 * (r >> 2) + 4 * (m & 1) + (r & 3); }
    __device__ __forceinline__ void load(const bf16* p, int lk) {
#pragma unroll
        for (int h = 0; h < 2; ++h) x[h] = *reinterpret_cast<const bf16x8*>(p + 32 * h + 8 * lk);
    }
    __device__ __forceinline__ f32x4 four(int m) const {
        f32x4 r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = (float)x[m >> 1][4 * (m & 1) + e];
        return r;
    }
    static __device__ __forceinline__ void store(bf16* p, int lk, const f32x4 (&v)[4]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (bf16)v[2 * h + (e >> 2)][e & 3];
            *reinterpret_cast<bf16x8*>(p + 32 * h + 8 * lk) = o;
        }
    }
};

// KS: steps of 32 ranks.  A wave has a block of 64 columns, whose rows of B it holds, and the tile's tokens, sixteen at a time: the next
// sixteen's y and u are on their way under this one's products.
template <typename T, int KS, int TOKENS>
__global__ __launch_bounds__(256) void lora_up_kernel(LoraArgs a, unsigned groups) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, lk = lane >> 4;
    const unsigned tile = blockIdx.x / groups;
    const int block = (int)(blockIdx.x - tile * groups) * 4 + wave;
    if (block >= (a.N >> 6)) return;
    Tile t;
    if (!locate<TOKENS>(a, (int)tile, &t)) return;
    const T* const y = static_cast<const T*>(a.y) + block * 64;
    T* const out = static_cast<T*>(a.out) + block * 64;
    auto row_of = [&](int g) { return (long long)t.first + min(16 * g + l15, t.count - 1); };
    constexpr int NG = TOKENS / 16, NP = kPieces<T>;
    if (t.adapter < 0) {
        if (a.y == a.out) return;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            if (16 * g + l15 >= t.count) continue;
            Sixteen<T> v;
            v.load(y + row_of(g) * a.y_stride, lk);
            const f32x4 same[4] = {v.four(0), v.four(1), v.four(2), v.four(3)};
            Sixteen<T>::store(out + row_of(g) * a.out_stride, lk, same);
        }
        return;
    }
    struct Group {
        Sixteen<T> v;
        f32x4 u[KS][2];
    };
    // ranks past the end, of which the products must see zeros on both sides (infinities and NaN), are copies of the last until then
    const bool cut = (a.rank & 31) != 0;
    auto fetch = [&](int g) {
        Group x;
        x.v.load(y + row_of(g) * a.y_stride, lk);
        const float* const p = a.u + row_of(g) * a.u_ranks;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) x.u[k][h] = *reinterpret_cast<const f32x4*>(p + min(32 * k + 8 * lk, a.u_ranks - 8) + 4 * h);
        if (NG == 1) {
            for (int part = 1; part < a.parts; ++part) {
                const float* const o = p + (long long)part * a.n_tokens * a.u_ranks;
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h) x.u[k][h] += *reinterpret_cast<const f32x4*>(o + min(32 * k + 8 * lk, a.u_ranks - 8) + 4 * h);
            }
        }
        return x;
    };
    Group next = fetch(0);
    bf16x8 w[4][KS];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const bf16* const p = a.b + ((long long)t.adapter * a.N + block * 64 + Sixteen<T>::column(m, l15)) * a.rank;
#pragma unroll
        for (int k = 0; k < KS; ++k) w[m][k] = *reinterpret_cast<const bf16x8*>(p + min(32 * k + 8 * lk, a.rank - 8));
    }
    __builtin_amdgcn_sched_barrier(0);
    const bf16x8 none = {};
    if (cut) {
#pragma unroll
        for (int m = 0; m < 4; ++m) w[m][KS - 1] = 32 * (KS - 1) + 8 * lk < a.rank ? w[m][KS - 1] : none;
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        if (16 * g >= t.count) break;
        Group now = next;
        if (g + 1 < NG && 16 * (g + 1) < t.count) next = fetch(g + 1);
        __builtin_amdgcn_sched_barrier(0);
        if (cut && 32 * (KS - 1) + 8 * lk >= a.rank) now.u[KS - 1][0] = now.u[KS - 1][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        f32x4 acc[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) acc[m] = now.v.four(m);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            bf16x8 piece[NP];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float rest = now.u[k][e >> 2][e & 3];
#pragma unroll
                for (int h = 0; h < NP; ++h) {
                    piece[h][e] = (bf16)rest;
                    rest -= (float)piece[h][e];
                }
            }
#pragma unroll
            for (int h = NP - 1; h >= 0; --h)
#pragma unroll
                for (int m = 0; m < 4; ++m) acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[m][k], piece[h], acc[m], 0, 0, 0);
        }
        if (16 * g + l15 < t.count) Sixteen<T>::store(out + row_of(g) * a.out_stride, lk, acc);
    }
}

// One token of a sequence: on the vector unit, where a tile would be empty but for one of sixteen tokens.  B's rows lie one behind the
// other, so lanes next to each other read pieces of eight ranks next to each other: P lanes have a column (P the power of two from the
// pieces of a row on), 64 / P columns a load, and add up by moves within the row of lanes; of the P loads that cover 64 columns a lane
// keeps the sum of one, its own.  B's bytes bound it: 64 tokens of 16 adapters beside 5120 x 15 360, both launches, rank 16 15.2 us, 64
// 31.2, 128 48.4 (by tiles 18.5, -, 59.5; a lane with columns of its own, 16 bytes of 64 lines a load, 15.0 and 48.6 at ranks 16 and 64).
template <int P>
__device__ __forceinline__ float piece_sum(float v) {
    if (P >= 2) v += dpp_f<0xB1>(v);         // quad_perm [1, 0, 3, 2]
    if (P >= 4) v += dpp_f<0x4E>(v);         // quad_perm [2, 3, 0, 1]
    if (P >= 8) v += dpp_f<0x141>(v);        // row_half_mirror
    if (P >= 16) v += dpp_f<0x140>(v);       // row_mirror
    return v;
}
template <typename T, int P>
__global__ __launch_bounds__(256) void lora_up_few_kernel(LoraArgs a, unsigned groups) {
    constexpr int kBlocks = P >= 4 ? 1 : 4 / P;                // blocks of 64 columns of a wave: four loads or more at once
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int piece = lane & (P - 1), c = lane / P;
    const unsigned tile = blockIdx.x / groups;
    const int block0 = ((int)(blockIdx.x - tile * groups) * 4 + wave) * kBlocks, blocks = a.N >> 6;
    if (block0 >= blocks) return;
    Tile t;
    if (!locate<16>(a, (int)tile, &t)) return;
    const T* const y = static_cast<const T*>(a.y);
    T* const out = static_cast<T*>(a.out);
    const bool adapted = t.adapter >= 0;
    if (!adapted && a.y == a.out) return;
    // the lane's column of a block, and its piece of the rows of the columns that it adds up for others
    const int own = piece * (64 / P) + c;
    const bool there = 8 * piece < a.rank;                     // (a row of pieces that is no power of two)
    bf16x8 w[kBlocks][P];
    if (adapted) {
        const bf16* const p = a.b + (long long)t.adapter * a.N * a.rank + min(8 * piece, a.rank - 8);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int g = 0; g < P; ++g)
                w[b][g] = *reinterpret_cast<const bf16x8*>(p + (long long)(min(block0 + b, blocks - 1) * 64 + g * (64 / P) + c) * a.rank);
    }
    for (int i = 0; i < t.count; ++i) {
        const long long row = t.first + i;
        T v[kBlocks];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) v[b] = y[row * a.y_stride + min(block0 + b, blocks - 1) * 64 + own];
        float x[kBlocks];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) x[b] = 0.0f;
        if (adapted) {
            f32x4 u[2] = {};
            if (there)
                for (int p = 0; p < a.parts; ++p) {
                    const f32x4* const up = reinterpret_cast<const f32x4*>(a.u + ((long long)p * a.n_tokens + row) * a.u_ranks + 8 * piece);
                    u[0] += up[0];
                    u[1] += up[1];
                }
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int g = 0; g < P; ++g) {
                    float sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum = fmaf(u[e >> 2][e & 3], (float)w[b][g][e], sum);
                    sum = there ? sum : 0.0f;
                    sum = piece_sum<P>(sum);
                    x[b] = piece == g ? sum : x[b];
                }
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
            if (block0 + b < blocks) out[row * a.out_stride + (block0 + b) * 64 + own] = adapted ? (T)((float)v[b] + x[b]) : v[b];
    }
}

template <typename T, int TOKENS>
void launch_up_tiles(const LoraArgs& a, hipStream_t s) {
    const unsigned groups = (unsigned)(a.N / 64 + 3) / 4;
    const dim3 grid(groups * (unsigned)(a.n_tokens / TOKENS + a.n_seqs));
    switch ((a.u_ranks + 31) / 32) {
        case 1: hipLaunchKernelGGL((lora_up_kernel<T, 1, TOKENS>), grid, dim3(256), 0, s, a, groups); break;
        case 2: hipLaunchKernelGGL((lora_up_kernel<T, 2, TOKENS>), grid, dim3(256), 0, s, a, groups); break;
        case 3: hipLaunchKernelGGL((lora_up_kernel<T, 3, TOKENS>), grid, dim3(256), 0, s, a, groups); break;
        default: hipLaunchKernelGGL((lora_up_kernel<T, 4, TOKENS>), grid, dim3(256), 0, s, a, groups); break;
    }
}
template <typename T>
void launch_up(const LoraArgs& a, int max_q_len, hipStream_t s) {
    if (max_q_len == 1) {
        auto go = [&](auto kernel, int blocks) {
            const unsigned groups = (unsigned)(a.N / 64 + 4 * blocks - 1) / (4 * blocks);
            hipLaunchKernelGGL(kernel, dim3(groups * (unsigned)(a.n_tokens / 16 + a.n_seqs)), dim3(256), 0, s, a, groups);
        };
        if (a.rank <= 8) go(lora_up_few_kernel<T, 1>, 4);
        else if (a.rank <= 16) go(lora_up_few_kernel<T, 2>, 2);
        else if (a.rank <= 32) go(lora_up_few_kernel<T, 4>, 1);
        else if (a.rank <= 64) go(lora_up_few_kernel<T, 8>, 1);
        else go(lora_up_few_kernel<T, 16>, 1);
        return;
    }
    if (max_q_len <= 16) launch_up_tiles<T, 16>(a, s);
    else launch_up_tiles<T, 32>(a, s);
}
template <int NT, int RT>
void launch_down(const LoraArgs& a, hipStream_t s) {
    const unsigned groups = (unsigned)(a.u_ranks + 16 * RT - 1) / (16 * RT);
    hipLaunchKernelGGL((lora_down_kernel<NT, RT>), dim3(groups * a.parts * (unsigned)(a.n_tokens / (16 * NT) + a.n_seqs)), dim3(64 * kDownWaves), 0, s, a, groups);
}

}  // namespace

int lora_parts(int n_seqs, int n_tokens, int max_q_len, int K, int rank) {
    if (max_q_len > 16) return 1;
    const int workgroups = max(n_tokens / 16, n_seqs) * ((rank + 15) / 16);
    return max(1, min(min(kUnits / workgroups, K / 1024), 4));
}

hipError_t launch_lora(const LoraArgs& a, int max_q_len, hipStream_t s) {
    const bool few = max_q_len <= 16;
    if (few) launch_down<1, 1>(a, s);
    else if (a.n_tokens < 4096 || a.u_ranks < 64) launch_down<2, 2>(a, s);
    else launch_down<2, 4>(a, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.fp32) launch_up<float>(a, max_q_len, s);
    else launch_up<bf16>(a, max_q_len, s);
    return hipGetLastError();
}

}  // namespace sdv2
