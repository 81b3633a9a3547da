// Low-rank adapters of many requests beside a shared projection:  out = y + scale (x A^T) B^T, each sequence with its own A [r, K],
// B [N, r] and scale, or none.
//
// Memory bound: x, y, out and the adapters' matrices once, 2 r (K + N) flops a row.  Two launches with u = scale x A^T between them, on
// 16x16x32 matrix instructions.  (One launch, in which each workgroup of the second product forms u for itself, reads A once per
// workgroup: when both were built, 64 tokens of rank 16, 5120 to 15 360, took 12.3 us instead of 13.2, but 8 of rank 64, 5120 x 5120, 36 instead
// of 12.)  Times below: a pass among others in a recorded graph.
//   u: computed transposed, ranks as rows and tokens as columns.  Few tokens: lora_down_kernel, 16 tokens and 16 ranks a workgroup, its
//     eight waves in turn over pieces of 64 of K, K in parts over workgroups.  Many: lora_down_tile_kernel, 32 tokens.  u stays in 32
//     bits, and goes to the second product as two or three bf16 numbers that add up to it (kPieces: as one, its rounding would be the
//     result's largest error).
//   out: lora_up_kernel, tokens as rows, y as the accumulator's start; one or two tokens a sequence: lora_up_few_kernel, on the vector unit.
// What the cache is asked for a load decides: 16 bytes of a lane are an access by themselves unless the lanes next to it are in the same
// line.  8800 tokens of four sequences, bf16, 5120 x 5120 of rank 64: fragments straight from memory 145 us, rows by lines through LDS 97
// (now 100: 270 MB, 2.7 TB/s); 1536 x 1536 45 -> 32 (now 33.5); 32 bits, 5120 x 5120, 175 -> 119 (now 121: 3.7 TB/s).
#include "ragged.h"

#include <type_traits>

namespace sdv2 {

namespace {

// Tokens of one sequence that a workgroup has, and its adapter.  Tiles are numbered as the row tiles of the paged attention: those of
// sequence s start at floor(q_start[s] / tokens) + s.
struct Tile {
    int first, count, adapter;        // first row of the batch, rows (<= tokens), adapter or -1
    int slot;                         // of u: sixteens of tokens, numbered as tiles of sixteen
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
    t->slot = q0 / 16 + s.index + at / 16;
    t->adapter = (unsigned)id < (unsigned)a.n_adapters ? id : -1;
    return true;
}

// u between the launches: by sixteens of tokens, and of those by fours of ranks, [slot][rank / 4][16 tokens][4], so that the sixteen
// lanes of a fragment's rows have 256 bytes next to each other; a row for a token where the second product has one token at a time.
__device__ __forceinline__ float* u_at(const LoraArgs& a, int part, int slot, int rank, int token) {
    return a.u + ((long long)part * a.slots + slot) * 16 * a.u_ranks + rank * 16 + token * 4;
}
__device__ __forceinline__ float* u_row(const LoraArgs& a, int part, int row, int rank) {
    return a.u + ((long long)part * a.n_tokens + row) * a.u_ranks + rank;
}

// What of x is rounded to bf16 first: a number beyond the largest of bf16 would become an infinity.
__device__ __forceinline__ float within_bf16(float x) {
    constexpr float kLargest = 0x1.fep127f;
    return __builtin_fabsf(x) < INFINITY ? __builtin_amdgcn_fmed3f(x, -kLargest, kLargest) : x;
}

// Zeros in the place of infinities and NaN.
__device__ __forceinline__ bf16x8 numbers_of(bf16x8 x) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __builtin_fabsf((float)x[e]) < INFINITY ? x[e] : (bf16)0.0f;
    return x;
}

constexpr int kDownWaves = 8;
// bf16 numbers that one of u goes to the second product as: each takes off eight bits, and an output of 32 bits shows the 17th
// (four frames of rank 64 against 64 bits: two pieces 1.9e-6 of the output, three 1.2e-7, which is the sum's own).
template <typename T>
constexpr int kPieces = sizeof(T) == 4 ? 3 : 2;

__global__ __launch_bounds__(64 * kDownWaves) void lora_down_kernel(LoraArgs a, unsigned groups) {
    __shared__ f32x4 parts[kDownWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, lk = lane >> 4;
    const unsigned rest = blockIdx.x / a.parts, part = blockIdx.x - rest * a.parts, tile = rest / groups;
    Tile t;
    if (!locate<16>(a, (int)tile, &t) || t.adapter < 0) return;
    const int rank0 = (int)(rest - tile * groups) * 16;
    const float scale = a.scale != nullptr ? a.scale[t.adapter] : 1.0f;

    const bf16* const wp = a.a + ((long long)t.adapter * a.rank + min(rank0 + l15, a.rank - 1)) * a.K + 8 * lk;
    const bf16* const xp = a.x + (long long)(t.first + min(l15, t.count - 1)) * a.x_stride + 8 * lk;
    f32x4 acc = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // pieces of 64 numbers (a line of 128 bytes in a row); several at once, so that their loads are in flight together
    constexpr int kAtOnce = 3;
    const int all = a.K >> 6, pieces = (int)((long long)all * (part + 1) / a.parts);
    for (int p0 = (int)((long long)all * part / a.parts) + wave; p0 < pieces; p0 += kDownWaves * kAtOnce) {
        bf16x8 w[kAtOnce][2], x[kAtOnce][2];
#pragma unroll
        for (int c = 0; c < kAtOnce; ++c) {
            const int at = min(p0 + kDownWaves * c, pieces - 1) * 64;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                w[c][h] = *reinterpret_cast<const bf16x8*>(wp + at + 32 * h);
                x[c][h] = *reinterpret_cast<const bf16x8*>(xp + at + 32 * h);
            }
        }
        __builtin_amdgcn_sched_barrier(0);       // (left to itself, the compiler puts each load in front of its product)
#pragma unroll
        for (int c = 0; c < kAtOnce; ++c) {
            if (p0 + kDownWaves * c >= pieces) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[c][h], x[c][h], acc, 0, 0, 0);
        }
    }
    parts[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
    f32x4 u = parts[0][lane];
#pragma unroll
    for (int k = 1; k < kDownWaves; ++k) u += parts[k][lane];
    const int rank = rank0 + 4 * lk;             // four ranks of one token
    if (l15 >= t.count) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = rank < a.rank ? u[e] * scale : 0.0f;
    *reinterpret_cast<f32x4*>(a.slots != 0 ? u_at(a, part, t.slot, rank, l15) : u_row(a, part, t.first + l15, rank)) = u;
}

// The same for 32 tokens and up to 64 ranks (16 RT), through LDS: a row's line of 128 bytes goes to eight lanes next
// to each other, where a fragment's lanes next to each other have different rows, each an access of the cache by itself.  Each wave has
// a stage of its own, and two pieces of 64 of K on their way to its registers.
template <int RT>
__global__ __launch_bounds__(256) void lora_down_tile_kernel(LoraArgs a, unsigned groups) {
    constexpr int kWaves = 4, kRows = 16 * RT + 32, kLoads = kRows / 8;
    __shared__ bf16x8 stage[kWaves][kRows * 8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, lk = lane >> 4;
    const unsigned tile = blockIdx.x / groups;
    Tile t;
    if (!locate<32>(a, (int)tile, &t) || t.adapter < 0) return;
    const int rank0 = (int)(blockIdx.x - tile * groups) * (16 * RT);
    const float scale = a.scale != nullptr ? a.scale[t.adapter] : 1.0f;

    // rows of the stage: the ranks, then the tokens; sixteen bytes c of row r lie at place c ^ (r / 2 & 7)
    const bf16* from[kLoads];
    int to[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int r = 8 * i + (lane >> 3), c = lane & 7;
        from[i] = 8 * i < 16 * RT ? a.a + ((long long)t.adapter * a.rank + min(rank0 + r, a.rank - 1)) * a.K + 8 * c
                                  : a.x + (long long)(t.first + min(r - 16 * RT, t.count - 1)) * a.x_stride + 8 * c;
        to[i] = r * 8 + (c ^ (r >> 1 & 7));
    }
    bf16x8* const mine = stage[wave];
    f32x4 acc[RT][2];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i][0] = acc[i][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int pieces = a.K >> 6;
    struct Piece {
        bf16x8 v[kLoads];
    };
    auto fetch = [&](int p) {
        Piece x;
        const int at = min(p, pieces - 1) * 64;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) x.v[i] = *reinterpret_cast<const bf16x8*>(from[i] + at);
        return x;
    };
    auto multiply = [&](const Piece& x) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) mine[to[i]] = x.v[i];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");         // (other lanes' writes)
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x8 w[RT], v[2];
            auto row = [&](int r) { return mine[(r + l15) * 8 + ((4 * h + lk) ^ (l15 >> 1))]; };
#pragma unroll
            for (int i = 0; i < RT; ++i) w[i] = row(16 * i);
#pragma unroll
            for (int j = 0; j < 2; ++j) v[j] = row(16 * RT + 16 * j);
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[i], v[j], acc[i][j], 0, 0, 0);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    Piece first = fetch(wave), second = fetch(wave + kWaves);
    for (int p = wave; p < pieces; p += 2 * kWaves) {
        multiply(first);
        first = fetch(p + 2 * kWaves);
        __builtin_amdgcn_sched_barrier(0);
        if (p + kWaves >= pieces) break;
        multiply(second);
        second = fetch(p + 3 * kWaves);
        __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
    f32x4* const parts = reinterpret_cast<f32x4*>(stage);              // [wave][block][lane]
    static_assert(kWaves * RT * 2 * 64 <= kWaves * kRows * 8, "the sums fit the stage");
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) parts[(wave * RT * 2 + i * 2 + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int b = wave; b < RT * 2; b += kWaves) {
        f32x4 u = parts[b * 64 + lane];
#pragma unroll
        for (int k = 1; k < kWaves; ++k) u += parts[(k * RT * 2 + b) * 64 + lane];
        const int rank = rank0 + 16 * (b >> 1) + 4 * lk;               // four ranks of one token
        if (16 * (b & 1) + l15 >= t.count || rank >= a.u_ranks) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = rank < a.rank ? u[e] * scale : 0.0f;
        *reinterpret_cast<f32x4*>(u_at(a, 0, t.slot + (b & 1), rank, l15)) = u;
    }
}

// KS: steps of 32 ranks.  A wave has a block of 64 columns and the tile's tokens, sixteen at a time: the next sixteen's y and u are on
// their way under this one's products.  Tokens are the rows of the result and lane l15 has columns 4 l15 .. + 3 (of four instructions),
// so a token's y and out are sixteen lanes next to each other; B's rows, of one piece of memory, are turned into fragments through LDS.
// Waves a SIMD: as many as the products and what is on its way need registers for.  The second pass over a group (below), which is
// hardly ever made, would take one of them (rank 64, 8800 rows, 5120 x 5120: 103.6 us instead of 100.3).
constexpr int lora_up_waves(int ks, int size) { return ks == 1 ? (size == 2 ? 5 : 4) : ks == 2 ? (size == 2 ? 4 : 3) : ks == 3 ? (size == 2 ? 3 : 2) : 2; }
template <typename T, int KS, int TOKENS>
__global__ __launch_bounds__(256, lora_up_waves(KS, sizeof(T))) void lora_up_kernel(LoraArgs a, unsigned groups) {
    typedef T four __attribute__((ext_vector_type(4)));
    __shared__ bf16x8 stage[4][64 * (4 * KS + 1)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, lk = lane >> 4;
    const unsigned tile = blockIdx.x / groups;
    const int block = (int)(blockIdx.x - tile * groups) * 4 + wave;
    if (block >= (a.N >> 6)) return;                           // (no barrier follows: a wave's stage is its own)
    Tile t;
    if (!locate<TOKENS>(a, (int)tile, &t)) return;
    const T* const y = static_cast<const T*>(a.y) + block * 64 + 4 * l15;
    T* const out = static_cast<T*>(a.out) + block * 64 + 4 * l15;
    constexpr int NG = TOKENS / 16, NP = kPieces<T>;
    auto token = [&](int g, int e) { return 16 * g + 4 * lk + e; };
    auto load = [&](int g, int e) { return *reinterpret_cast<const four*>(y + (long long)(t.first + min(token(g, e), t.count - 1)) * a.y_stride); };
    auto store = [&](int g, int e, four v) {
        if (token(g, e) < t.count) *reinterpret_cast<four*>(out + (long long)(t.first + token(g, e)) * a.out_stride) = v;
    };
    if (t.adapter < 0) {
        if (a.y == a.out) return;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            four v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = load(g, e);
#pragma unroll
            for (int e = 0; e < 4; ++e) store(g, e, v[e]);
        }
        return;
    }
    struct Group {
        four v[4];
        f32x4 u[KS][2];
    };
    // ranks past the end, of which the products must see zeros on both sides (infinities and NaN), are copies of the last until then
    const int pieces = a.rank >> 3;
    const bool cut = (pieces & 3) != 0;
    auto fetch = [&](int g) {
        Group x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x.v[e] = load(g, e);
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) x.u[k][h] = *reinterpret_cast<const f32x4*>(u_at(a, 0, t.slot + g, 8 * min(4 * k + lk, pieces - 1) + 4 * h, l15));
        if (NG == 1) {
            for (int part = 1; part < a.parts; ++part)
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h) x.u[k][h] += *reinterpret_cast<const f32x4*>(u_at(a, part, t.slot, 8 * min(4 * k + lk, pieces - 1) + 4 * h, l15));
        }
        return x;
    };
    // a row of B to row (column & 3) * 16 + column / 4 of the stage, whose rows are an odd number of pieces apart
    bf16x8 w[4][KS];
    bf16x8* const mine = stage[wave];
    const int apart = pieces | 1;
    {
        const bf16x8* const p = reinterpret_cast<const bf16x8*>(a.b + ((long long)t.adapter * a.N + block * 64) * a.rank);
        bf16x8 v[4 * KS];
#pragma unroll
        for (int j = 0; j < 4 * KS; ++j)
            if (j < pieces) v[j] = p[64 * j + lane];
        const int per = (65536 + pieces - 1) / pieces;         // (quotients of numbers under 1024 by at most 16 are exact so)
#pragma unroll
        for (int j = 0; j < 4 * KS; ++j)
            if (j < pieces) {
                const int i = 64 * j + lane, column = (i * per) >> 16;
                mine[((column & 3) * 16 + (column >> 2)) * apart + i - column * pieces] = v[j];
            }
    }
    Group next = fetch(0);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");     // (other lanes' writes)
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int k = 0; k < KS; ++k) w[m][k] = mine[(16 * m + l15) * apart + min(4 * k + lk, pieces - 1)];
    const bf16x8 none = {};
    if (cut) {
#pragma unroll
        for (int m = 0; m < 4; ++m) w[m][KS - 1] = 4 * (KS - 1) + lk < pieces ? w[m][KS - 1] : none;
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        if (16 * g >= t.count) break;
        Group now = next;
        if (g + 1 < NG && 16 * (g + 1) < t.count) next = fetch(g + 1);
        __builtin_amdgcn_sched_barrier(0);
        if (cut && 4 * (KS - 1) + lk >= pieces) now.u[KS - 1][0] = now.u[KS - 1][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        f32x4 acc[4];
        auto multiply = [&](auto careful) {
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[m][e] = (float)now.v[e][m];
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                bf16x8 piece[NP];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float rest = now.u[k][e >> 2][e & 3];
#pragma unroll
                    for (int h = 0; h < NP; ++h) {
                        piece[h][e] = (bf16)(h == 0 ? within_bf16(rest) : rest);
                        const float less = rest - (float)piece[h][e];
                        rest = less == less ? less : 0.0f;         // (of an infinity nothing is left)
                    }
                }
#pragma unroll
                for (int h = NP - 1; h >= 0; --h)
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        bf16x8 b = w[m][k];
                        if (careful.value && h > 0) {
                            asm volatile("" : "+v"(b));        // (here, not ahead of the loop)
                            b = numbers_of(b);
                        }
                        acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(piece[h], b, acc[m], 0, 0, 0);
                    }
            }
        };
        multiply(std::false_type());
        float broken = 0.0f;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) broken = __builtin_fmaf(acc[m][e], 0.0f, broken);
        // an infinity in B times a second piece of u, which may be zero or of the other sign, is in none of the sums of the formula
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(broken == 0.0f)) != 0, 0)) multiply(std::true_type());
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            four v;
#pragma unroll
            for (int m = 0; m < 4; ++m) v[m] = (T)acc[m][e];
            store(g, e, v);
        }
    }
}

// One or two tokens of a sequence: on the vector unit, where a tile would be empty but for those of sixteen tokens.  B's rows lie one behind the
// other, so lanes next to each other read pieces of eight ranks next to each other: P lanes have a column (P the power of two from the
// pieces of a row on), 64 / P columns a load, and add up by moves within the row of lanes; of the P loads that cover 64 columns a lane
// keeps the sum of one, its own.  B's bytes bound it: 64 tokens of 16 adapters beside 5120 x 15 360, both launches, rank 16 15.1 us, 64
// 30.9, 128 52.6 (by tiles 20.7, 39.9 and 66.4; a lane with columns of its own, 16 bytes of 64 lines a load, when this was 15.3 and 31.2 us, 15.0 and
// 48.6 at ranks 16 and 64).
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
            if (there) {
                auto at = [&](int p, int h) { return *reinterpret_cast<const f32x4*>(u_row(a, p, t.first + i, 8 * piece + 4 * h)); };
                u[0] = at(0, 0);
                u[1] = at(0, 1);
                for (int p = 1; p < a.parts; p += 2) {        // (two parts, or three, on their way at once)
                    const int q = min(p + 1, a.parts - 1);
                    const f32x4 x = at(p, 0), y = at(p, 1), v = at(q, 0), z = at(q, 1);
                    u[0] += x;
                    u[1] += y;
                    if (q > p) u[0] += v, u[1] += z;
                }
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

// Tiles of sixteen tokens and ranks, K in parts, for one or two tokens a sequence and wherever that is under half a workgroup a compute unit; else
// tiles of 32 tokens by lines.  Measured, by sixteens | by 32 in us, 5120 x 5120: 16 sequences of 4 tokens of rank 16 10.3 | 14.9, of 48
// 13.9 | 19.7; one of 1000 of rank 128 40.3 | 34.4; 128 of 16 of rank 16 30.3 | 26.2; 1536 x 4608: 100 of 4 15.1 | 16.2, of 16 17.9 | 17.8,
// 64 of 24 of rank 64 28.4 | 25.4, 64 of 16 20.6 | 21.5.
int sixteens(int n_seqs, int n_tokens, int rank) { return max(n_tokens / 16, n_seqs) * ((rank + 15) / 16); }
bool by_sixteens(int n_seqs, int n_tokens, int max_q_len, int rank) { return lora_by_tokens(max_q_len) || sixteens(n_seqs, n_tokens, rank) < kUnits / 2; }

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
    if (lora_by_tokens(max_q_len)) {
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
    if (by_sixteens(a.n_seqs, a.n_tokens, max_q_len, a.rank)) launch_up_tiles<T, 16>(a, s);
    else launch_up_tiles<T, 32>(a, s);
}
}  // namespace

// By lanes | by tiles, both launches, us: 64 sequences of one token, 5120 to 15 360, rank 16, 15.1 | 20.7, of two 18.6 | 21.7, of four 25.1 | 23.6;
// of rank 64 one 30.9 | 39.9, two 34.9 | 39.8; of rank 128 two 58.9 | 67.9; 16, 5120 x 5120, rank 16, one 8.9 | 9.7, two 9.6 | 9.9, four 11.5 | 10.2;
// 8 of three 10.7 | 9.7; 1000 of two, 1536 x 1536, rank 16, 25.9 | 31.2, 5120 x 5120, rank 128, 371 | 310.
bool lora_by_tokens(int max_q_len) { return max_q_len <= 2; }

int lora_parts(int n_seqs, int n_tokens, int max_q_len, int K, int rank) {
    if (!by_sixteens(n_seqs, n_tokens, max_q_len, rank)) return 1;
    // (1 part | these, 5120 x 5120 of rank 16: one token 12.7 | 8.6 us, 16 sequences of 8 15.6 | 9.9)
    return max(1, min(min(kUnits / sixteens(n_seqs, n_tokens, rank), K / 1024), 4));
}

hipError_t launch_lora(const LoraArgs& a, int max_q_len, hipStream_t s) {
    if (by_sixteens(a.n_seqs, a.n_tokens, max_q_len, a.rank)) {
        const unsigned groups = (unsigned)(a.u_ranks / 16);
        hipLaunchKernelGGL(lora_down_kernel, dim3(groups * a.parts * (unsigned)(a.n_tokens / 16 + a.n_seqs)), dim3(64 * kDownWaves), 0, s, a, groups);
    } else {
        auto go = [&](auto kernel, int ranks) {
            const unsigned groups = (unsigned)((a.u_ranks + ranks - 1) / ranks);
            hipLaunchKernelGGL(kernel, dim3(groups * (unsigned)(a.n_tokens / 32 + a.n_seqs)), dim3(256), 0, s, a, groups);
        };
        if (a.u_ranks <= 16) go(lora_down_tile_kernel<1>, 16);
        else if (a.u_ranks <= 32) go(lora_down_tile_kernel<2>, 32);
        else go(lora_down_tile_kernel<4>, 64);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.fp32) launch_up<float>(a, max_q_len, s);
    else launch_up<bf16>(a, max_q_len, s);
    return hipGetLastError();
}

}  // namespace sdv2
