// Attention of a ragged batch of new tokens over a paged cache.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j) over the keys j that the row may see; the zero row where there is none, and
//   where all their scores are minus infinity.
//
// A number of a key or value is two bytes and two flops a row: few rows are bound by memory, a few hundred that share the keys by the
// matrix cores.  Two kernels, each in one pass with the running reference point and sum of a softmax, and a third that
// joins parts of a key range.  Measured (32 query and 8 key heads unless said otherwise):
//   few rows: 64 tokens over 1 to 16 000 keys 1.99 GB in 365 us, 5.45 TB/s (reads of 8 KB at random places alone: 6.05); 8-bit pages,
//     0.99 GB, 194 us, 5.1 TB/s; one token over 9001 keys 14.9 us in two launches.
//   many rows: 2 x 4680 rows of 12 heads over 10 920 keys 628 GF in 694 us, 0.9 PF/s (the kernel over contiguous keys, whose values lie
//     transposed already and whose p is one bf16 number, 1.2); six prompts of 1 to 4096 tokens, causal, 234 GF in 298 us: the last
//     workgroups' tail; 333 rows over 32 700 keys of 8 bits 179 GF in 207 us, the join's reading included.
#include "ragged.h"

#include <climits>
#include <type_traits>

namespace sdv2 {

namespace {

constexpr int D = kHeadDim;
constexpr float kSumLimit = 16384.0f;     // a lane's sum of p over one tile (at most 32 keys) beyond this: move the reference
constexpr float kNoKey = -1.0e30f;   // reference point of a row that has seen no key yet: finite, so that -inf minus it is -inf

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Formats of a row of 128 numbers, in a page or in LDS.
enum Format { kBf16, kE4m3, kFp16 };

// p of eight keys on its way to the second product, whose other side is values: as one bf16 number it would add an error the size of
// the output's own rounding (2.3e-3 of the output against 64 bits, where the rounding alone is 1.66e-3).
//   With bf16 values: two bf16 numbers that add up to p but for 2^-16 of it, a product each.
//   With fp16 values: one fp16 number, p but for 2^-11.  What is under 2^-14 loses bits there, so the reference point of the exponents lies
//     kLift under the row's maximum: p of that is 2^8, and what a small one loses is 2^-33 of it at most.
template <int F>
struct Weights {
    f16x8 x;
    static constexpr float kLift = 8.0f, kSlack = 6.0f;      // kSlack: log2 units that the maximum may rise before the reference point is moved
    __device__ __forceinline__ void set(int e, float p) { x[e] = (_Float16)p; }
    __device__ __forceinline__ float get(int e) const { return (float)x[e]; }
    __device__ __forceinline__ void pin() { asm volatile("" : "+v"(x)); }
};
template <>
struct Weights<kBf16> {
    bf16x8 hi, lo;
    static constexpr float kLift = 0.0f, kSlack = 8.0f;
    __device__ __forceinline__ void set(int e, float p) {
        hi[e] = (bf16)p;
        lo[e] = (bf16)(p - (float)hi[e]);
    }
    __device__ __forceinline__ float get(int e) const { return (float)hi[e] + (float)lo[e]; }
    __device__ __forceinline__ void pin() { asm volatile("" : "+v"(hi), "+v"(lo)); }
};

// o[db] += values (32 channels x 16 keys of each db) times p.
__device__ __forceinline__ void add_values(f32x16 (&o)[4], const bf16x8 (&v)[4], const Weights<kBf16>& w) {
#pragma unroll
    for (int db = 0; db < 4; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[db], w.lo, o[db], 0, 0, 0);
#pragma unroll
    for (int db = 0; db < 4; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[db], w.hi, o[db], 0, 0, 0);
}
template <int F>
__device__ __forceinline__ void add_values(f32x16 (&o)[4], const f16x8 (&v)[4], const Weights<F>& w) {
#pragma unroll
    for (int db = 0; db < 4; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[db], w.x, o[db], 0, 0, 0);
}

// Eight fp16 from eight e4m3 (exact).
__device__ __forceinline__ f16x8 widen_to_fp16(u32x2 v) {
    f16x8 out;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const f16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[w], 1.0f, false);
        const f16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[w], 1.0f, true);
        out[4 * w] = lo[0];
        out[4 * w + 1] = lo[1];
        out[4 * w + 2] = hi[0];
        out[4 * w + 3] = hi[1];
    }
    return out;
}

// Eight fp16 from eight bf16 times kValueScale: exact where each of them is zero or of size 2^-25 up to 2^8, which `range` keeps account of.
constexpr float kValueScale = 256.0f;
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
struct Range {
    u16x2 least = {0xffff, 0xffff};          // twice the bits of the smallest but zero, less one (0xfe: 2^-17 in fp16)
    f16x2 large = {0, 0};                    // NaN: one was too large, infinite or NaN
    __device__ __forceinline__ bool left() const {
        return least[0] < 0xff || least[1] < 0xff || !(large[0] == (_Float16)0) || !(large[1] == (_Float16)0);
    }
};
__device__ __forceinline__ f16x8 scaled_to_fp16(uint4 x, Range& range) {
    uint4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned w = i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w;
        const float lo = __uint_as_float(w << 16) * kValueScale, hi = __uint_as_float(w & 0xffff0000u) * kValueScale;
        unsigned h = __builtin_bit_cast(unsigned, f16x2{(_Float16)lo, (_Float16)hi}), twice;
        asm("" : "+v"(h));                   // (or it is formed twice)
        asm("v_pk_mad_u16 %0, %1, 2, -1 op_sel_hi:[1,0,1]" : "=v"(twice) : "v"(h));
        range.least = __builtin_elementwise_min(range.least, __builtin_bit_cast(u16x2, twice));
        range.large = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, h), f16x2{0, 0}, range.large);
        (i == 0 ? out.x : i == 1 ? out.y : i == 2 ? out.z : out.w) = h;
    }
    return __builtin_bit_cast(f16x8, out);
}

// Whether any number is infinite or NaN.
__device__ __forceinline__ bool broken_sums(const f32x16 (&o)[4]) {
    float t[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) t[r & 3] = __builtin_fmaf(o[db][r], 0.0f, t[r & 3]);
    return !((t[0] + t[1]) + (t[2] + t[3]) == 0.0f);
}

typedef __attribute__((address_space(3))) void* lds_void_ptr;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4_ptr;
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2* lds_i32x2_ptr;

__device__ __forceinline__ void load_to_lds(const void* src, void* dst) { __builtin_amdgcn_global_load_lds(src, (lds_void_ptr)dst, 16, 0, 0); }

// The waits count loads, so loads stay where they are written, and reads of what they bring behind the wait.
__device__ __forceinline__ void hold_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ void reads_done() {
    hold_order();
    __builtin_amdgcn_s_waitcnt(0xC07F);          // lgkmcnt(0)
    hold_order();
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float max2(float a, float b) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
// Largest of a block's sixteen scores and of the partner lane's (the same row's other sixteen keys); NaN gives way.  (Written as
// instructions, which wait for no product: the caller has read the scores in ordinary code before.)
__device__ __forceinline__ float block_max(const f32x16& s) {
    float m[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) m[c] = max2(max3(s[4 * c], s[4 * c + 1], s[4 * c + 2]), s[4 * c + 3]);
    const float x = max2(max3(m[0], m[1], m[2]), m[3]);
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return max2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Two groups of four channels of a row as bf16: a lane has channels 4 lh .. + 3 of two blocks of eight; the halves of the wave trade
// words so that each lane stores eight channels in a row (lanes < 32 the first block, the others the second).
__device__ __forceinline__ uint4 eight_channels(const bf16x4& lo, const bf16x4& hi) {
    const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
    const auto x = __builtin_amdgcn_permlane32_swap(a.x, b.x, false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(a.y, b.y, false, false);
    return uint4{x[0], y[0], x[1], y[1]};
}

// ---------------------------------------------------------------------------------------------------
// What a workgroup works on: a run of rows of one sequence and key head, and a run of the key tiles that they see.  Row r of a sequence is
// its token r / group under query head r % group of the key head, so all rows share keys and values.
struct Work {
    int seq, hk, part;
    int q0, n, kv_len;        // first row of the sequence in the batch, its new tokens, its tokens
    int row0, rows;           // first row of this workgroup, and all of the sequence's
};

// Row tiles are numbered without a table: those of sequence s start at floor(q_start[s] group / tile) + s, which leaves each sequence
// at least as many numbers as it has tiles.  False: a number that no tile has.
__device__ __forceinline__ bool locate(const PagedAttnArgs& a, int tile_rows, int tile, Work* w) {
    const Sequence s = sequence_at(a.batch.q_start, a.batch.kv_len, a.batch.n_seqs, tile,
                                   [&](int end, int i) { return (int)((long long)end * a.group / tile_rows) + i; });
    w->seq = s.index;
    if (w->seq >= a.batch.n_seqs) return false;
    w->q0 = s.q0;
    w->n = s.n;
    w->kv_len = tokens_of(s.more, a.batch.table_stride, a.batch.page_shift);
    if (w->q0 < 0 || w->n < 0 || w->n > a.batch.n_tokens - w->q0) return false;      // not a batch: touch nothing
    w->rows = w->n * a.group;
    w->row0 = (tile - (int)((long long)w->q0 * a.group / tile_rows) - w->seq) * tile_rows;
    return w->row0 >= 0 && w->row0 < w->rows;
}

// ---------------------------------------------------------------------------------------------------
// Tiles of keys and values in LDS as they lie in a page, [key][128], a row's 16-byte chunks permuted so that fragment reads spread
// over the 64 banks.  A row: 256 bytes of bf16 or (values) fp16, or 128 of e4m3.
//   K fragment (32 keys x 16 numbers): a lane reads its key's row, 16 bytes at a time; chunk c of row r lies at c ^ (r % 16), e4m3:
//     c ^ (r / 2 % 8).  Of e4m3, 16 bytes are two steps' numbers: lane half lh of step s has numbers 32 (s / 2) + 16 lh + 8 (s % 2) .. + 7
//     where bf16 has 16 s + 8 lh .. + 7, and the query's fragments go by the same rule.
//   V fragment (32 channels x 16 keys) transposed: ds_read_b64_tr hands each of 16 lanes a column of the rows that the 16 lanes
//     address, four keys of 16 bits or eight of 8 bits, and the rows are picked in the order in which the scores' accumulators hold
//     the keys (4 lh .. + 3 and 8 + 4 lh .. + 3 of sixteen).  Chunk c of row r lies at c ^ (r % 4) * 4; e4m3: c ^ 2 (r / 2 % 2 + 2 (r / 8 % 2)).
template <int F>
struct Rows {
    static constexpr bool E4M3 = F == kE4m3;
    static constexpr int kRow = E4M3 ? 128 : 256;             // bytes
    typedef std::conditional_t<F == kBf16, bf16x8, f16x8> Values;
    static constexpr int kPerLoad = 1024 / kRow;              // rows of a wave load
    // byte within the rows of load number i that this lane fetches to its place (K, V)
    static __device__ __forceinline__ int k_source(int lane, int i) {
        if (E4M3) return (lane >> 3) * 128 + (((lane & 7) ^ (lane >> 4) ^ (4 * (i & 1))) << 4);
        return (lane >> 4) * 256 + (((lane & 15) ^ (lane >> 4) ^ (4 * (i & 3))) << 4);
    }
    static __device__ __forceinline__ int v_source(int lane, int i) {
        if (E4M3) return (lane >> 3) * 128 + (((lane & 7) ^ (((lane >> 4) & 1) << 1) ^ ((i & 1) << 2)) << 4);
        return (lane >> 4) * 256 + (((lane & 15) ^ ((lane >> 4) << 2)) << 4);
    }
    static __device__ __forceinline__ int v_position(int row, int chunk) {      // byte of a chunk
        if (E4M3) return row * 128 + ((chunk ^ ((((row >> 1) & 1) | (((row >> 3) & 1) << 1)) << 1)) << 4);
        return row * 256 + ((chunk ^ ((row & 3) << 2)) << 4);
    }
    // first number of this lane's eight in step s of the query
    static __device__ __forceinline__ int q_number(int s, int lh) { return E4M3 ? 32 * (s >> 1) + 16 * lh + 8 * (s & 1) : 16 * s + 8 * lh; }
    // the eight fragments of 32 keys
    static __device__ __forceinline__ void k_fragments(bf16x8 (&f)[8], const unsigned char* tile, int l31, int lh) {
        if (E4M3) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const uint4 x = *reinterpret_cast<const uint4*>(tile + l31 * 128 + (((2 * s + lh) ^ ((l31 >> 1) & 7)) << 4));
                f[2 * s] = widen_e4m3(u32x2{x.x, x.y});
                f[2 * s + 1] = widen_e4m3(u32x2{x.z, x.w});
            }
        } else {
#pragma unroll
            for (int s = 0; s < 8; ++s) f[s] = *reinterpret_cast<const bf16x8*>(tile + l31 * 256 + (((2 * s + lh) ^ (l31 & 15)) << 4));
        }
    }
    // this lane's byte of the reads of channels 32 db .. + 31 of the first sixteen keys
    static __device__ __forceinline__ int v_lane(int lane, int db) {
        const int lh = lane >> 5;
        if (E4M3) {
            const int j = (lane & 15) >> 1, g = ((j >> 1) & 1) | ((j >> 2) << 1);
            return (4 * lh + (j & 3) + 8 * (j >> 2)) * 128 + ((db ^ g) << 5) + ((lane >> 4) & 1) * 16 + (lane & 1) * 8;
        }
        const int x = (lane >> 2) & 3;
        return (4 * lh + x) * 256 + ((db ^ x) << 6) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
    }
    // fragment of sixteen keys whose rows start at `tile`
    static __device__ __forceinline__ Values v_fragment(const unsigned char* tile, int at) {
        if constexpr (E4M3) {
            const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2_ptr)(tile + at));
            return widen_to_fp16(__builtin_bit_cast(u32x2, x));
        }
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(tile + at));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(tile + at + 8 * 256));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        return __builtin_bit_cast(Values, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // whether these sixteen bytes of values hold an infinity or NaN
    static __device__ __forceinline__ bool broken(uint4 x) {
        unsigned hit = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned w = i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w;
            if (E4M3) hit |= ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;                    // 0x7f or 0xff
            else if (F == kFp16) hit |= ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u;
            else hit |= ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;                         // exponent of ones
        }
        return hit != 0;
    }
};

// Bit j: key j of the 32 whose value rows start at row `first` of the tile holds an infinity or NaN.
template <int F>
__device__ __forceinline__ unsigned broken_keys(const unsigned char* v, int first, int lane) {
    typedef Rows<F> R;
    const int row = first + (lane & 31);
    bool hit = false;
    constexpr int kChunks = R::kRow / 16 / 2;                 // of this lane: half a row
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        // each lane starts at another chunk, so that the lanes of a read do not all hit one bank
        const int chunk = (lane >> 5) * kChunks + ((c + lane) & (kChunks - 1));
        hit |= R::broken(*reinterpret_cast<const uint4*>(v + R::v_position(row, chunk)));
    }
    const unsigned long long b = __builtin_amdgcn_ballot_w64(hit);
    return (unsigned)(b | (b >> 32));
}

// Adds to O^T the keys in `broken` of 32 (rows `first` .. of the value tile), one by one and only to the rows that see them: in a product
// with the others, zero times their infinities or NaN would reach rows that do not, and an infinity times p's second piece would be
// NaN where p times it is not.  w0, w1: p of the 32 keys, s: their scores, minus infinity where the row does not see the key.  scratch: 2 KB of
// the wave's.  The caller then blanks these keys' values and goes on as ever.  Rare, so short, not fast.
constexpr int kApartBytes = 2048;
template <int F>
__device__ __forceinline__ void add_apart(f32x16 (&o)[4], const unsigned char* v, int first, const Weights<F>& w0, const Weights<F>& w1, const f32x16& s,
                                          unsigned broken, unsigned char* scratch, int lane) {
    typedef Rows<F> R;
    const int lh = lane >> 5;
    float* const own = reinterpret_cast<float*>(scratch);     // [eight keys of sixteen][64 lanes]; -1: not seen
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        unsigned left = broken >> (16 * half) & 0xffffu;
        if (left == 0) continue;
        reads_done();                                         // (of what lay there)
#pragma unroll
        for (int e = 0; e < 8; ++e) own[e * 64 + lane] = s[8 * half + e] == -INFINITY ? -1.0f : half == 0 ? w0.get(e) : w1.get(e);
        hold_order();
#pragma clang loop unroll(disable)
        while (left != 0) {
            const int j = __builtin_ctz(left), row = first + 16 * half + j;
            left &= left - 1;
            // key j of sixteen: element (j & 3) + 4 (j / 8) of lane half j / 4 % 2
            const float p = own[((j & 3) + 4 * (j >> 3)) * 64 + (lane & 31) + 32 * ((j >> 2) & 1)];
            const unsigned keep = p >= 0.0f ? ~0u : 0u;
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float x[4];
                    if (F == kE4m3) {
                        const unsigned w = *reinterpret_cast<const unsigned*>(v + R::v_position(row, 2 * db + (g >> 1)) + 8 * (g & 1) + 4 * lh);
                        const f16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
                        x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
                    } else {
                        const uint2 w = *reinterpret_cast<const uint2*>(v + R::v_position(row, 4 * db + g) + 8 * lh);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const unsigned short n = (unsigned short)((e < 2 ? w.x : w.y) >> (16 * (e & 1)));
                            x[e] = F == kFp16 ? (float)__builtin_bit_cast(_Float16, n) : (float)__builtin_bit_cast(bf16, n);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        // (p may be zero in 32 bits, and infinity times it is an infinity)
                        const float t = __builtin_fabsf(x[e]) < INFINITY ? p * x[e] : x[e];
                        o[db][4 * g + e] += __uint_as_float(__float_as_uint(t) & keep);
                    }
                }
        }
    }
}

// Output of a lane's row: 32 NDB channels from d0 on, value(db, g, e) = channel d0 + 32 db + 8 g + 4 lh + e before the division by the
// sum.  Whole key range: bf16 to o.  In parts: 32 bits and (m, l) to the workspace, for the join.
template <int NDB, typename F>
__device__ __forceinline__ void store_rows(const PagedAttnArgs& a, const Work& w, bool live, int token, int head, float m, float l, int d0,
                                           bool write_ml, int lh, F&& value) {
    const int t = w.q0 + token;
    if (a.parts == 1) {
        const float inv = l != 0.0f ? a.v_scale / l : 0.0f;
        bf16* const op = a.o + t * a.o_stride + head * D + d0 + 8 * lh;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int g = 0; g < 4; g += 2) {
                bf16x4 x[2];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[0][e] = (bf16)(value(db, g, e) * inv);
                    x[1][e] = (bf16)(value(db, g + 1, e) * inv);
                }
                const uint4 v = eight_channels(x[0], x[1]);
                if (live) *reinterpret_cast<uint4*>(op + 32 * db + 8 * g) = v;
            }
        return;
    }
    if (!live) return;
    const long long at = ((long long)w.part * a.batch.n_tokens + t) * a.q_heads + head;
    float* const op = a.part_o + at * D + d0 + 4 * lh;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = value(db, g, e);
            *reinterpret_cast<f32x4*>(op + 32 * db + 8 * g) = x;
        }
    if (write_ml) {
        a.part_ml[at * 2] = m;
        a.part_ml[at * 2 + 1] = l;
    }
}

// What a part that has no keys leaves for the join.
__device__ __forceinline__ void no_keys(const PagedAttnArgs& a, const Work& w, int token, int head) {
    float* const ml = a.part_ml + (((long long)w.part * a.batch.n_tokens + w.q0 + token) * a.q_heads + head) * 2;
    ml[0] = kNoKey;
    ml[1] = 0.0f;
}

// ---------------------------------------------------------------------------------------------------
// Few rows: the keys are what is read, and the memory what bounds it.  A workgroup has at most 32 rows; its four waves take the key
// tiles of 32 in turn, each with a buffer of its own in LDS that direct loads fill and no barrier guards: a wave waits for its own loads
// only, and fetches the next keys as soon as its fragments of these are in registers.  Two workgroups per compute unit, up to 128 KB of
// loads on their way.  The waves' outputs are joined through LDS, those of the key range's parts by a second launch.
constexpr int kTokenTile = 32, kTokenWaves = 4;
constexpr int kTokenStages = 65536, kTokenLds = kTokenStages + kTokenWaves * kApartBytes;      // bytes of LDS

template <bool E4M3>
__global__ __launch_bounds__(256, 2) void paged_attention_tokens_kernel(PagedAttnArgs a) {
    constexpr int F = E4M3 ? kE4m3 : kBf16;
    typedef Rows<F> R;
    typedef Weights<F> P;
    constexpr int KT = kTokenTile, NW = kTokenWaves;
    constexpr int kStages = E4M3 ? 2 : 1;
    constexpr int kTile = KT * R::kRow, kLoads = KT / R::kPerLoad;          // bytes and wave loads of a K or V tile
    static_assert(NW * kStages * 2 * kTile == kTokenStages, "and the waves' outputs fill it too");
    __shared__ __attribute__((aligned(16))) unsigned char smem[kTokenLds];      // (its size stated here, a launch sets no attribute: it may be the first, and recorded)
    unsigned char* const k_first = smem;
    unsigned char* const v_first = smem + NW * kTile;
    unsigned char* const k_second = smem + 2 * NW * kTile;
    unsigned char* const v_second = smem + 3 * NW * kTile;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l31 = lane & 31, lh = lane >> 5;
    // Workgroups go to the eight XCDs in turn, so the heads of a sequence come one after the other: with the sequences next to each
    // other, an XCD has every eighth of them where their number allows, and the XCD with the longest is waited for (64 sequences of
    // 1 to 16 000 keys: 395 us, this order 350).
    Work w;
    const unsigned rest = divide(blockIdx.x, a.by_heads), part = divide(rest, a.by_tiles);
    w.hk = (int)(blockIdx.x - rest * a.by_heads.d);
    w.part = (int)part;
    if (!locate(a, KT, (int)(rest - part * a.by_tiles.d), &w)) return;
    const int last_row = min(w.row0 + 32, w.rows) - 1;
    const Visited vis = visited_tiles<KT>(a.mask, w.row0 / a.group, last_row / a.group, w.n, w.kv_len);
    const int first = min(vis.count, w.part * a.part_tiles), end = w.part == a.parts - 1 ? vis.count : min(vis.count, first + a.part_tiles);
    const int count = max(0, (end - first - wave + NW - 1) / NW);           // tiles of this wave

    // this lane's row
    const int row = min(w.row0 + l31, w.rows - 1), token = (int)divide(row, a.by_group), head = w.hk * a.group + row - token * a.group;
    const bool live = w.row0 + l31 < w.rows;
    if (a.parts > 1 && first >= end) {
        if (wave == 0 && lh == 0 && live) no_keys(a, w, token, head);
        return;
    }
    const RowKeys keys = row_keys(a.mask, token, w.n, w.kv_len);
    bf16x8 qf[8];
    {
        const bf16* qp = a.q + (long long)(w.q0 + token) * a.q_stride + head * D;
#pragma unroll
        for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qp + R::q_number(s, lh));
    }

    const int* const table = a.batch.table + (long long)w.seq * a.batch.table_stride;
    const int slot_mask = (1 << a.batch.page_shift) - 1;

    // A wave whose sums have come out broken goes over its keys once more, with care: an infinite value that every row of a tile sees
    // belongs into the result, where the two pieces of p have made a NaN of it.  (e4m3 has no infinity.)
    f32x16 o[4];
    float m, l;
    bool careful = false;
again:
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] = 0.0f;
    m = kNoKey, l = 0.0f;

    // 32 tiles at a time, whose 64 pages of sixteen keys the lanes look up together
    for (int batch = 0; batch < count; batch += 32) {
        const int n = min(32, count - batch);
        int pages;
        {
            const int t = tile_of(vis, first + wave + NW * (batch + min(lane >> 1, n - 1)));
            pages = table[min((t * KT + 16 * (lane & 1)) >> a.batch.page_shift, a.batch.table_stride - 1)];
        }
        const bool gone = (unsigned)pages >= (unsigned)a.batch.n_pages;
        const unsigned long long holes = __builtin_amdgcn_ballot_w64(gone);
        if (gone) pages = 0;                                                 // fetched, not seen
        auto fetch = [&](const void* pool, int i, unsigned char* to, bool values) {
            const int t = tile_of(vis, first + wave + NW * (batch + i));
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const long long page = __builtin_amdgcn_readlane(pages, 2 * i + half);
                const unsigned char* src = static_cast<const unsigned char*>(pool) +
                    (((page * a.batch.kv_heads + w.hk) << a.batch.page_shift) + ((t * KT + 16 * half) & slot_mask)) * R::kRow;
#pragma unroll
                for (int x = 0; x < kLoads / 2; ++x) {
                    const int load = half * (kLoads / 2) + x;
                    load_to_lds(src + x * 1024 + (values ? R::v_source(lane, load) : R::k_source(lane, load)), to + load * 1024);
                }
            }
        };
        // (restrict: a transposing read is taken to wait for every load on its way to LDS that may alias it)
        auto step = [&](unsigned char* __restrict__ kt, unsigned char* __restrict__ vt, int i) __attribute__((always_inline)) {
            const int t = tile_of(vis, first + wave + NW * (batch + i)), key0 = t * KT;
            // these keys are there when no more loads are on their way than went out behind theirs
            if (i + kStages - 1 < n) __builtin_amdgcn_s_waitcnt(0x0F70 | (kLoads * (2 * kStages - 1)));
            else __builtin_amdgcn_s_waitcnt(0x0F70);
            hold_order();
            f32x16 s0, s1;
#pragma unroll
            for (int r = 0; r < 16; ++r) s0[r] = s1[r] = 0.0f;
            {
                bf16x8 kf[8];
                R::k_fragments(kf, kt, l31, lh);
#pragma unroll
                for (int s = 0; s < 8; s += 2) {
                    s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[s], s0, 0, 0, 0);
                    s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s + 1], qf[s + 1], s1, 0, 0, 0);
                }
            }
            if (i + kStages < n) {
                reads_done();                                                // the fragments are in registers
                fetch(a.k_pages, i + kStages, kt, false);
            }
            s0 += s1;
            const unsigned gaps = (unsigned)(holes >> (2 * i)) & 3u;
            const bool masked = gaps != 0 || !whole(vis, key0, key0 + KT);
            if (masked) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int j = 8 * (r >> 2) + 4 * lh + (r & 3);
                    if (!sees(keys, key0 + j) | (((gaps >> (r >> 3)) & 1) != 0)) s0[r] = -INFINITY;
                }
            }
            const float top = block_max(s0) * a.mask.scale_log2e;
            const bool moved = top > m + (P::kLift + P::kSlack);
            if (__builtin_amdgcn_ballot_w64(moved) != 0) {
                const float next = moved ? top - P::kLift : m, alpha = __builtin_amdgcn_exp2f(m - next);
                m = next;
                l *= alpha;
#pragma unroll
                for (int db = 0; db < 4; ++db)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
            }
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            P pf[2];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s0[r], a.mask.scale_log2e, -m));
                sum[r & 3] += p;
                pf[r >> 3].set(r & 7, p);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            // and these values: behind them went out kStages - 1 tiles and the keys just asked for
            if (i + kStages < n) __builtin_amdgcn_s_waitcnt(0x0F70 | (kLoads * (2 * kStages - 1)));
            else __builtin_amdgcn_s_waitcnt(0x0F70);
            hold_order();
            const unsigned broken = masked || careful ? broken_keys<F>(vt, 0, lane) : 0u;
            if (__builtin_expect(broken != 0, 0)) {
                add_apart<F>(o, vt, 0, pf[0], pf[1], s0, broken, smem + kTokenStages + wave * kApartBytes, lane);
                if ((broken >> l31) & 1)
                    for (int c = 0; c < R::kRow / 32; ++c) *reinterpret_cast<uint4*>(vt + l31 * R::kRow + lh * (R::kRow / 2) + c * 16) = uint4{0, 0, 0, 0};
                reads_done();
            }
#pragma unroll
            for (int ts = 0; ts < 2; ++ts) {
                typename R::Values v[4];
#pragma unroll
                for (int db = 0; db < 4; ++db) v[db] = R::v_fragment(vt + 16 * ts * R::kRow, R::v_lane(lane, db));
                add_values(o, v, pf[ts]);
            }
            if (i + kStages < n) {
                reads_done();
                fetch(a.v_pages, i + kStages, vt, true);
                hold_order();
            }
        };
        fetch(a.k_pages, 0, k_first + wave * kTile, false);
        hold_order();
        fetch(a.v_pages, 0, v_first + wave * kTile, true);
        hold_order();
        if (kStages == 2 && n > 1) {
            fetch(a.k_pages, 1, k_second + wave * kTile, false);
            hold_order();
            fetch(a.v_pages, 1, v_second + wave * kTile, true);
            hold_order();
        }
        for (int i = 0; i < n; ++i) {
            step(k_first + wave * kTile, v_first + wave * kTile, i);
            if (kStages == 2 && ++i < n) step(k_second + wave * kTile, v_second + wave * kTile, i);
        }
        reads_done();                                                        // the buffers are free for the next 32 tiles
    }
    if (!E4M3 && !careful && __builtin_expect(__builtin_amdgcn_ballot_w64(broken_sums(o)) != 0, 0)) {
        careful = true;
        goto again;
    }

    // ---- join the waves, in their order: wave w adds up and stores channels 32 w .. + 31
    {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    }
    // where a wave's four channels of one kind lie: [wave][4][64] of block db
    auto place = [&](int wv, int db, int g) {
        unsigned char* const part = kStages == 2 ? (db == 0 ? k_first : db == 1 ? k_second : db == 2 ? v_first : v_second)
                                                 : (db < 2 ? k_first : v_first) + (db & 1) * (NW * 4096);
        return reinterpret_cast<f32x4*>(part) + (wv * 4 + g) * 64 + lane;
    };
    __syncthreads();                                                         // everyone is done with the buffers
    float* const ml = reinterpret_cast<float*>(k_first);                     // [NW][2][32]
    if (lh == 0) {
        ml[wave * 64 + l31] = m;
        ml[wave * 64 + 32 + l31] = l;
    }
    __syncthreads();
    float top = kNoKey, total = 0.0f;
#pragma unroll
    for (int k = 0; k < NW; ++k) top = fmaxf(top, ml[k * 64 + l31]);
#pragma unroll
    for (int k = 0; k < NW; ++k) total += ml[k * 64 + 32 + l31] * __builtin_amdgcn_exp2f(ml[k * 64 + l31] - top);
    const float weight = __builtin_amdgcn_exp2f(m - top);
    __syncthreads();
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = o[db][4 * g + e] * weight;
            *place(wave, db, g) = x;
        }
    __syncthreads();
    f32x4 mine[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        mine[g] = *place(0, wave, g);
#pragma unroll
        for (int k = 1; k < NW; ++k) mine[g] += *place(k, wave, g);
    }
    store_rows<1>(a, w, live, token, head, top, total, 32 * wave, wave == 0 && lh == 0, lh, [&](int, int g, int e) { return mine[g][e]; });
}

// Second launch where the key range is in parts: out = sum_i 2^(m_i - max m) O_i / sum_i 2^(m_i - max m) l_i.  A part that saw no key of the
// row has left l = 0 and no O.  Sixteen lanes have eight channels each of a row and head, and GROUPS such groups take its parts in turn:
// one group, and the parts of a single token are a chain of loads (36 of them: 10.8 us, sixteen groups 4).
template <int GROUPS>
__global__ __launch_bounds__(256) void paged_attention_join_kernel(PagedAttnArgs a) {
    __shared__ f32x4 sums[GROUPS == 1 ? 1 : 256][2];
    __shared__ float ml[GROUPS == 1 ? 1 : 256][2];
    const long long row_heads = (long long)a.batch.n_tokens * a.q_heads;
    const int group = (threadIdx.x >> 4) % GROUPS, c = threadIdx.x & 15;
    const long long at = (long long)blockIdx.x * (16 / GROUPS) + threadIdx.x / (16 * GROUPS);
    const int t = (int)(at / a.q_heads), h = (int)(at - (long long)t * a.q_heads);
    const bool live = at < row_heads && t < a.batch.q_start[a.batch.n_seqs];        // behind the last sequence nothing is written
    float top = kNoKey, total = 0.0f;
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = x;
    if (live) {
        constexpr int kAtOnce = 4;
        for (int p0 = group; p0 < a.parts; p0 += GROUPS * kAtOnce) {
            float m[kAtOnce], l[kAtOnce];
            f32x4 u[kAtOnce], v[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const int p = p0 + GROUPS * i;
                const bool in = p < a.parts;
                const float* const q = a.part_ml + ((in ? p : p0) * row_heads + at) * 2;
                m[i] = q[0];
                l[i] = in ? q[1] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                if (l[i] == 0.0f) continue;
                const f32x4* const q = reinterpret_cast<const f32x4*>(a.part_o + ((p0 + GROUPS * i) * row_heads + at) * D + c * 8);
                u[i] = q[0];
                v[i] = q[1];
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                if (l[i] == 0.0f) continue;
                const float next = fmaxf(top, m[i]), keep = __builtin_amdgcn_exp2f(top - next), weight = __builtin_amdgcn_exp2f(m[i] - next);
                top = next;
                total = total * keep + l[i] * weight;
                x = x * keep + u[i] * weight;
                y = y * keep + v[i] * weight;
            }
        }
    }
    if (GROUPS > 1) {
        sums[threadIdx.x][0] = x;
        sums[threadIdx.x][1] = y;
        ml[threadIdx.x][0] = top;
        ml[threadIdx.x][1] = total;
        __syncthreads();
        if (group != 0 || !live) return;
#pragma unroll
        for (int g = 1; g < GROUPS; ++g) top = fmaxf(top, ml[threadIdx.x + 16 * g][0]);
        const float own = __builtin_amdgcn_exp2f(ml[threadIdx.x][0] - top);
        total *= own;
        x *= own;
        y *= own;
#pragma unroll
        for (int g = 1; g < GROUPS; ++g) {
            const float weight = __builtin_amdgcn_exp2f(ml[threadIdx.x + 16 * g][0] - top);
            total += weight * ml[threadIdx.x + 16 * g][1];
            x += weight * sums[threadIdx.x + 16 * g][0];
            y += weight * sums[threadIdx.x + 16 * g][1];
        }
    }
    if (!live) return;
    const float inv = total != 0.0f ? a.v_scale / total : 0.0f;
    bf16x8 out;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = (bf16)((e < 4 ? x[e & 3] : y[e & 3]) * inv);
    *reinterpret_cast<bf16x8*>(a.o + t * a.o_stride + h * D + c * 8) = out;
}

// ---------------------------------------------------------------------------------------------------
// Many rows: NW waves of 32 rows share tiles of 64 keys; the matrix cores bound it, with the vector unit's softmax close behind.
//   * Scores are computed transposed, S^T = K Q^T: a lane owns a row (column of S^T) with its partner lane + 32, keeps the row's sum and
//     reference point, and the accumulators are in the order that the second product O^T = V^T P^T takes its P in.
//   * Keys and values have two stages each.  While the vector unit forms p of tile n, the matrix unit forms S^T of tile n + 1; then
//     come the values of tile n.  The loads of keys and values n + 2 go out between the first products, those to LDS and these to
//     registers, from which they are put into LDS at the start of the next tile.
//   * The reference point of a row's exponents trails its maximum by up to kSumLimit's logarithm: a steady tile forms no maximum and
//     rescales nothing.
//   * Values pass through registers on their way to LDS and are fp16 there, so that p goes to the second product as one fp16 number: as two bf16
//     numbers beside bf16 values, twice the products, two chunks of 4680 rows took 938 us instead of 694, prompts 456 instead of 298 (one bf16
//     number: 622 and 271, and 1.4 times the error).  e4m3 and most bf16 are exact in fp16; a tile that holds others is left out by the loop
//     and taken afterwards as it is (every 40th page so 797 us instead of 707, all of them 2361).
//   * Keys of 8 bits are widened on the way too: every wave reads every fragment, and widening those would be eight times the
//     conversions.  8-bit tiles are fetched one tile earlier.
template <int NW>
constexpr int kRowsStages = 65536 + (NW == 8 ? 8 * 8192 : 0);
// Tiles that are taken apart from the loop and noted by their numbers; if there are more, all from the first to the last are looked at again.
constexpr int kApartTiles = 48;
template <int NW>
constexpr int kRowsLds = kRowsStages<NW> + NW * kApartBytes + 64 + 4 * kApartTiles;      // bytes of LDS

template <bool E4M3, int NW>
__global__ __launch_bounds__(64 * NW, NW == 4 ? 2 : 1) void paged_attention_rows_kernel(PagedAttnArgs a) {
    typedef Rows<kFp16> R;                                    // values in LDS; keys are bf16 there whatever the pages hold
    typedef Weights<kFp16> P;
    constexpr int KT = 64, kTile = KT * 256;
    constexpr int kRow = E4M3 ? 128 : 256;                    // bytes in a page
    constexpr int kLoads = KT * kRow / 1024 / NW;             // wave loads of a K or V tile by each wave
    constexpr int kLoadRows = 1024 / kRow;
    constexpr int kAhead = E4M3 ? 3 : 2;                      // tiles between the fetch of keys and their softmax
    __shared__ __attribute__((aligned(16))) unsigned char smem[kRowsLds<NW>];
    unsigned char* const k_stage = smem;                      // [2][64 keys][256 B]
    unsigned char* const v_stage = smem + 2 * kTile;          // [2][64 keys][256 B]
    constexpr int kStages = kRowsStages<NW>;                  // behind them eight waves' rows, then add_apart's scratch, two words per wave and a list of tiles
    unsigned* const flags = reinterpret_cast<unsigned*>(smem + kStages + NW * kApartBytes);
    int* const apart = reinterpret_cast<int*>(flags + 16);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l31 = lane & 31, lh = lane >> 5;
    // Workgroups are handed to the eight XCDs in turn; renumbered, each XCD (its own L2) works through a run of row tiles of the same keys,
    // the last tile first: under a causal mask it sees the most keys.
    const unsigned flat = blockIdx.x, xcd = flat & 7u, per = a.n_wg >> 3, rem = a.n_wg & 7u;
    const unsigned logical = xcd * per + min(xcd, rem) + (flat >> 3), rest = divide(logical, a.by_tiles), part = divide(rest, a.by_heads);
    Work w;
    w.hk = (int)(rest - part * a.by_heads.d);
    w.part = (int)part;
    if (!locate(a, 32 * NW, a.row_tiles - 1 - (int)(logical - rest * a.by_tiles.d), &w)) return;
    const int last_row = min(w.row0 + 32 * NW, w.rows) - 1;
    const int first_token = (int)divide(w.row0, a.by_group), last_token = (int)divide(last_row, a.by_group);
    const Visited vis = visited_tiles<KT>(a.mask, first_token, last_token, w.n, w.kv_len);
    const int first = min(vis.count, w.part * a.part_tiles), end = w.part == a.parts - 1 ? vis.count : min(vis.count, first + a.part_tiles);
    // this lane's row, formed anew where it is needed: kept across the loop it would be spilled
    auto own_row = [&]() {
        int t = threadIdx.x;
        asm volatile("" : "+v"(t));
        return w.row0 + 32 * (t >> 6) + (t & 31);
    };
    struct Place {
        int token, head;
        bool live;
    };
    auto place_of = [&](int row) {
        const int r = min(row, w.rows - 1), token = (int)divide(r, a.by_group);
        return Place{token, w.hk * a.group + r - token * a.group, row < w.rows};
    };
    if (a.parts > 1 && first >= end) {
        const Place x = place_of(own_row());
        if (lh == 0 && x.live) no_keys(a, w, x.token, x.head);
        return;
    }

    f32x16 o[4];                                              // (of bf16 pages: times kValueScale)
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] = 0.0f;
    float m = kNoKey, l = 0.0f;

    if (first < end) {
        // ---- pages.  Lane g of four looks up the page of sixteen keys of a tile; all four go to every wave, a tile before its keys are
        // fetched.
        const int* const table = a.batch.table + (long long)w.seq * a.batch.table_stride;
        const int slot_mask = (1 << a.batch.page_shift) - 1;
        auto key_of = [&](int n) { return tile_of(vis, min(n, end - 1)) * KT; };
        auto look_up = [&](int n) { return table[min((key_of(n) + 16 * (lane & 3)) >> a.batch.page_shift, a.batch.table_stride - 1)]; };
        struct Source {
            long long at[kLoads];                             // byte in the pools of this wave's loads of a tile
        };
        unsigned gaps_ahead = 0;                              // four bits a tile: sixteen keys without a page
        auto source_of = [&](int pages, int n, int tiles_ahead) {
            const bool gone = (unsigned)pages >= (unsigned)a.batch.n_pages;
            gaps_ahead |= ((unsigned)__builtin_amdgcn_ballot_w64(gone) & 15u) << (4 * tiles_ahead);
            if (gone) pages = 0;                              // fetched, not seen
            Source s;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int row = kLoadRows * (wave + NW * i);
                const long long page = __builtin_amdgcn_readlane(pages, row >> 4);
                s.at[i] = (((page * a.batch.kv_heads + w.hk) << a.batch.page_shift) + ((key_of(n) + row) & slot_mask)) * kRow;
            }
            return s;
        };
        // keys of bf16: straight to LDS
        const int k_lane = (lane >> 4) * 256 + (((lane & 15) ^ ((4 * wave + (lane >> 4)) & 15)) << 4);
        auto fetch = [&](const Source& s, unsigned char* stage) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                load_to_lds(static_cast<const unsigned char*>(a.k_pages) + s.at[i] + k_lane, stage + 1024 * (wave + NW * i));
        };
        // values, and keys of e4m3: to registers, and from there in the format of LDS
        struct Bytes {
            uint4 x[kLoads];
        };
        const int v_lane = E4M3 ? lane * 16 : R::v_source(lane, 0);
        auto take = [&](const void* pool, const Source& s) {
            Bytes b;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) b.x[i] = *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(pool) + s.at[i] + v_lane);
            return b;
        };
        auto put_keys = [&](const Bytes& b, unsigned char* stage) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int row = 8 * (wave + NW * i) + (lane >> 3), c = 2 * (lane & 7), turn = row & 15;
                *reinterpret_cast<bf16x8*>(stage + row * 256 + ((c ^ turn) << 4)) = widen_e4m3(u32x2{b.x[i].x, b.x[i].y});
                *reinterpret_cast<bf16x8*>(stage + row * 256 + (((c + 1) ^ turn) << 4)) = widen_e4m3(u32x2{b.x[i].z, b.x[i].w});
            }
        };
        // and a word of this wave's for the tile: whether its values need care, because of their range or an infinity or NaN
        auto put_values = [&](const Bytes& b, unsigned char* stage, unsigned* care_flags) {
            bool care = false;
            Range range;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if constexpr (E4M3) {
                    const int row = 8 * (wave + NW * i) + (lane >> 3), c = 2 * (lane & 7);
                    *reinterpret_cast<f16x8*>(stage + R::v_position(row, c)) = widen_to_fp16(u32x2{b.x[i].x, b.x[i].y});
                    *reinterpret_cast<f16x8*>(stage + R::v_position(row, c + 1)) = widen_to_fp16(u32x2{b.x[i].z, b.x[i].w});
                    care |= Rows<kE4m3>::broken(b.x[i]);
                } else {
                    *reinterpret_cast<f16x8*>(stage + 1024 * (wave + NW * i) + lane * 16) = scaled_to_fp16(b.x[i], range);
                }
            }
            if (!E4M3) care = range.left();
            const unsigned long long any = __builtin_amdgcn_ballot_w64(care);
            if (lane == 0) care_flags[wave] = any != 0;
        };

        // ---- the wave's 32 rows, through LDS: eight waves behind the stages; four in the second stages, which are free until then
        unsigned char* const q_stage = NW == 8 ? smem + 4 * kTile + wave * 8192 : (wave < 2 ? k_stage : v_stage) + kTile + (wave & 1) * 8192;
        int pages[kAhead + 1];
#pragma unroll
        for (int i = 0; i <= kAhead; ++i) pages[i] = look_up(first + i);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + (lane >> 4);
            const Place x = place_of(w.row0 + 32 * wave + r);
            const bf16* src = a.q + (long long)(w.q0 + x.token) * a.q_stride + x.head * D;
            load_to_lds(reinterpret_cast<const unsigned char*>(src) + (((lane & 15) ^ (r & 15)) << 4), q_stage + i * 1024);
        }
        hold_order();
        Source src0 = source_of(pages[0], first, 0), src1 = source_of(pages[1], first + 1, 1);
        Source ahead;                                         // e4m3: of the tile whose values are fetched next
        Bytes k_bytes, v_bytes, k_one;
        int next_pages;
        auto barrier = [&]() {
            hold_order();
            __builtin_amdgcn_s_barrier();
            hold_order();
        };
        if constexpr (E4M3) {
            const Source src2 = source_of(pages[2], first + 2, 2);
            k_bytes = take(a.k_pages, src0);
            v_bytes = take(a.v_pages, src0);
            k_one = take(a.k_pages, src1);
            const Bytes k_two = take(a.k_pages, src2), v_one = take(a.v_pages, src1);
            put_keys(k_bytes, k_stage);
            put_values(v_bytes, v_stage, flags);
            if (NW == 8) put_keys(k_one, k_stage + kTile);
            k_bytes = k_two;
            v_bytes = v_one;
            ahead = src2;
            next_pages = pages[3];
            __builtin_amdgcn_s_waitcnt(0x0070);               // all loads, and what was put
        } else {
            fetch(src0, k_stage);
            hold_order();
            v_bytes = take(a.v_pages, src0);
            hold_order();
            if (NW == 8) fetch(src1, k_stage + kTile);
            hold_order();
            const Bytes v_one = take(a.v_pages, src1);
            put_values(v_bytes, v_stage, flags);
            v_bytes = v_one;
            next_pages = pages[2];
            __builtin_amdgcn_s_waitcnt(0x0070 | ((NW == 8 ? 2 : 1) * kLoads));      // the rows, the first keys, and what was put
        }
        barrier();
        bf16x8 qf[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(q_stage + l31 * 256 + (((2 * s + lh) ^ (l31 & 15)) << 4));
        if (NW == 4) {
            reads_done();
            barrier();                                        // everyone has its rows: the second stages are free
            if constexpr (E4M3) put_keys(k_one, k_stage + kTile);
            else fetch(src1, k_stage + kTile);
        }

        const int k_first = l31 * 256 + ((lh ^ (l31 & 15)) << 4);            // this lane's byte of step 0; of step s: 32 s turned into it
        // Half of S^T of the tile at sk: steps 4 half .. + 3 of both 32-key blocks, the fragments first, the products in turn to the two
        // accumulators (one that waits for its own predecessor takes 12 clocks longer).
        auto qk_half = [&](f32x16 (&s)[2], const unsigned char* sk, int half, auto&& after_reads) {
            if (half == 0) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[kb][r] = 0.0f;
            }
            bf16x8 kf[4][2];
            int at = k_first;
            if (NW == 4) asm volatile("" : "+v"(at));         // (its eight places, kept across the loop, would cost the queries their registers)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) kf[i][kb] = *reinterpret_cast<const bf16x8*>(sk + kb * 32 * 256 + (at ^ (32 * (4 * half + i))));
            after_reads();
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i][kb], qf[4 * half + i], s[kb], 0, 0, 0);
        };
        int v_at[4];
#pragma unroll
        for (int db = 0; db < 4; ++db) v_at[db] = R::v_lane(lane, db);
        const float scale = a.mask.scale_log2e;

        int care_count = 0, care_first = 0, care_last = 0;    // tiles whose values are left out by the loop (below)
        auto nothing = []() {};
        f32x16 s_a[2], s_b[2];
        qk_half(s_a, k_stage, 0, nothing);
        qk_half(s_a, k_stage, 1, nothing);

        // One tile: s_cur holds S^T of tile n; S^T of tile n + 1 is formed into s_nxt on the way.  k_now: keys n + 1; k_fill: keys n + 2 go there;
        // v_now: values n; v_fill: values n + 1 go there (restrict: a transposing read is taken to wait for every load on its way to LDS
        // that may alias it); care_now, care_fill: the words of the values n and n + 1.  Past the last tile it is fetched again,
        // unconditionally, into a stage that nobody reads.
        auto tile_step = [&](const unsigned char* __restrict__ k_now, unsigned char* __restrict__ k_fill, unsigned char* __restrict__ v_now,
                             unsigned char* __restrict__ v_fill, f32x16 (&s_cur)[2], f32x16 (&s_nxt)[2], int n, const unsigned* __restrict__ care_now,
                             unsigned* __restrict__ care_fill) __attribute__((always_inline)) {
            __builtin_amdgcn_s_waitcnt(0x0070);
            barrier();                       // keys n + 1 and values n are there; everyone is done with keys n and values n - 1
            const unsigned gaps = gaps_ahead & 15u;
            gaps_ahead >>= 4;
            const int key0 = key_of(n);
            const bool masked = gaps != 0 || !whole(vis, key0, key0 + KT);
            if (masked) {
                const RowKeys keys = row_keys(a.mask, place_of(own_row()).token, w.n, w.kv_len);
                // bounds relative to this lane's first key; sixteen keys without a page are behind the end
                const int mine = key0 + 4 * lh, before = keys.end - mine, from = keys.low - mine, sink = keys.sink - mine;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int stop = (gaps >> (2 * kb + half)) & 1 ? INT_MIN : before;
#pragma unroll
                        for (int r = 8 * half; r < 8 * half + 8; ++r) {
                            const int j = kb * 32 + 8 * (r >> 2) + (r & 3);
                            if ((j >= stop) | ((j < from) & (j >= sink))) s_cur[kb][r] = -INFINITY;
                        }
                    }
            }
            const Source src = source_of(next_pages, n + kAhead, kAhead - 1);
            float sums[4];
            P pf[4];
            auto exps = [&](int kb) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s_cur[kb][r], scale, -m));
                    sums[r & 3] = (kb == 0 && r < 4) ? p : sums[r & 3] + p;     // four independent chains
                    pf[kb * 2 + (r >> 3)].set(r & 7, p);
                }
            };
            auto pin = [&]() {               // the fragments are formed here, among the products, not after the branch
#pragma unroll
                for (int i = 0; i < 4; ++i) pf[i].pin();
            };
            if constexpr (E4M3) put_keys(k_bytes, k_fill);
            put_values(v_bytes, v_fill, care_fill);
            if constexpr (E4M3) {
                k_bytes = take(a.k_pages, src);
                v_bytes = take(a.v_pages, ahead);
            }
            __builtin_amdgcn_sched_barrier(0);
            qk_half(s_nxt, k_now, 0, [&]() {
                if constexpr (!E4M3) {
                    fetch(src, k_fill);
                    v_bytes = take(a.v_pages, src);
                }
            });
            exps(0);
            __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);       // the eight fragment reads, then product | load | vector work
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (!E4M3 && i < 2 * kLoads) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
                __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            ahead = src;
            next_pages = look_up(n + kAhead + 1);
            bool care;                       // a wave's word of these values says so
            qk_half(s_nxt, k_now, 1, [&]() { care = __builtin_amdgcn_ballot_w64(care_now[lane & (NW - 1)] != 0) != 0; });
            exps(1);
            float lsum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
            pin();
            __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
                __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(lsum <= kSumLimit)) != 0, 0)) {
                // a row's scores have run ahead of its reference point (or it has seen no key yet): move it to their maximum, which is more than
                // log2(kSumLimit / 32) ahead
                const float top = max2(block_max(s_cur[0]), block_max(s_cur[1])) * scale;
                const float next = top > m + (P::kLift + 1.0f) ? top - P::kLift : m, alpha = __builtin_amdgcn_exp2f(m - next);
                m = next;
                l *= alpha;
#pragma unroll
                for (int db = 0; db < 4; ++db)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
                exps(0);
                exps(1);
                lsum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
                pin();
            }
            l += lsum;
            __builtin_amdgcn_sched_barrier(0);
            if (__builtin_expect(care, 0) && (!E4M3 || masked)) {        // (NaN that every row sees needs none)
                if (care_count < kApartTiles) apart[care_count] = n;
                if (care_count++ == 0) care_first = n;
                care_last = n;
                return;
            }
#pragma unroll
            for (int ts = 0; ts < 4; ++ts) {
                typename R::Values v[4];
#pragma unroll
                for (int db = 0; db < 4; ++db) v[db] = R::v_fragment(v_now + 16 * ts * 256, v_at[db]);
                add_values(o, v, pf[ts]);
            }
            __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);       // fragment reads (two each) run four ahead of the products
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        for (int n = first; n < end; n += 2) {
            tile_step(k_stage + kTile, k_stage, v_stage, v_stage + kTile, s_a, s_b, n, flags, flags + NW);
            if (n + 1 < end) tile_step(k_stage, k_stage + kTile, v_stage + kTile, v_stage, s_b, s_a, n + 1, flags + NW, flags);
        }
        __builtin_amdgcn_s_waitcnt(0x0070);      // no load may still be on its way to this LDS when the wave ends

        // ---- Tiles with values that do not go to the second product like others: bf16 beyond the range of fp16, which are taken as they are
        // here, with p as two bf16 numbers; infinities and NaN in either format, which are added key by key.  Their p is in l already;
        // their scores are formed once more, the same in the same order, and p at the last reference point.  Rare, so short, not fast.
        const bool listed = care_count <= kApartTiles;
        for (int i = 0; i < (listed ? care_count : care_last - care_first + 1); ++i) {
            constexpr int C = E4M3 ? kFp16 : kBf16;
            __syncthreads();                     // everyone is done with the stages
            const int n = listed ? __builtin_amdgcn_readfirstlane(apart[i]) : care_first + i, key0 = key_of(n);
            bool care = false;
            for (int x = threadIdx.x; x < KT * kRow / 16; x += 64 * NW) {
                const int r = x / (kRow / 16), c = x % (kRow / 16), key = key0 + r;
                long long page = table[min(key >> a.batch.page_shift, a.batch.table_stride - 1)];
                if ((unsigned long long)page >= (unsigned)a.batch.n_pages) page = 0;
                const long long at = (((page * a.batch.kv_heads + w.hk) << a.batch.page_shift) + (key & slot_mask)) * kRow + c * 16;
                const uint4 k = *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(a.k_pages) + at);
                const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(a.v_pages) + at);
                if constexpr (E4M3) {
                    *reinterpret_cast<bf16x8*>(k_stage + r * 256 + (((2 * c) ^ (r & 15)) << 4)) = widen_e4m3(u32x2{k.x, k.y});
                    *reinterpret_cast<bf16x8*>(k_stage + r * 256 + (((2 * c + 1) ^ (r & 15)) << 4)) = widen_e4m3(u32x2{k.z, k.w});
                    *reinterpret_cast<f16x8*>(v_stage + R::v_position(r, 2 * c)) = widen_to_fp16(u32x2{v.x, v.y});
                    *reinterpret_cast<f16x8*>(v_stage + R::v_position(r, 2 * c + 1)) = widen_to_fp16(u32x2{v.z, v.w});
                    care |= Rows<kE4m3>::broken(v);
                } else {
                    Range range;
                    scaled_to_fp16(v, range);
                    care |= range.left();
                    *reinterpret_cast<uint4*>(k_stage + r * 256 + ((c ^ (r & 15)) << 4)) = k;
                    *reinterpret_cast<uint4*>(v_stage + R::v_position(r, c)) = v;
                }
            }
            const unsigned long long cares = __builtin_amdgcn_ballot_w64(care);
            if (lane == 0) flags[wave] = cares != 0;
            const int page = look_up(n);
            const unsigned gaps = (unsigned)__builtin_amdgcn_ballot_w64((unsigned)page >= (unsigned)a.batch.n_pages) & 15u;
            __syncthreads();
            // (the loop has taken those out of e4m3 of which every row sees every key in)
            if (__builtin_amdgcn_ballot_w64(flags[lane & (NW - 1)] != 0) == 0 || (E4M3 && gaps == 0 && whole(vis, key0, key0 + KT))) continue;
            qk_half(s_a, k_stage, 0, nothing);
            qk_half(s_a, k_stage, 1, nothing);
            const RowKeys keys = row_keys(a.mask, place_of(own_row()).token, w.n, w.kv_len);
            Weights<C> p[4];
#pragma unroll
            for (int r = 0; r < 32; ++r) {
                const int j = 8 * (r >> 2) + (r & 3) + 4 * lh;
                const bool seen = sees(keys, key0 + j) & (((gaps >> (j >> 4)) & 1) == 0);
                const float x = s_a[r >> 4][r & 15] = seen ? s_a[r >> 4][r & 15] : -INFINITY;
                p[r >> 3].set(r & 7, __builtin_amdgcn_exp2f(__builtin_fmaf(x, scale, -m)) * (E4M3 ? 1.0f : kValueScale));
            }
            unsigned broken[2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                broken[kb] = broken_keys<C>(v_stage, 32 * kb, lane);
                add_apart<C>(o, v_stage, 32 * kb, p[2 * kb], p[2 * kb + 1], s_a[kb], broken[kb], smem + kStages + wave * kApartBytes, lane);
            }
            __syncthreads();                     // nobody needs those any more
            const unsigned long long all = broken[0] | ((unsigned long long)broken[1] << 32);
            for (int x = threadIdx.x; x < KT * 16; x += 64 * NW)
                if ((all >> (x >> 4)) & 1) *reinterpret_cast<uint4*>(v_stage + x * 16) = uint4{0, 0, 0, 0};
            __syncthreads();
#pragma unroll
            for (int ts = 0; ts < 4; ++ts) {
                typename Rows<C>::Values v[4];
#pragma unroll
                for (int db = 0; db < 4; ++db) v[db] = Rows<C>::v_fragment(v_stage + 16 * ts * 256, v_at[db]);
                add_values(o, v, p[ts]);
            }
        }
    }
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    const float total = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    const Place x = place_of(own_row());
    store_rows<4>(a, w, x.live, x.token, x.head, m, total, 0, lh == 0, lh,
                  [&](int db, int g, int e) { return E4M3 ? o[db][4 * g + e] : o[db][4 * g + e] * (1.0f / kValueScale); });
}

}  // namespace

// Overrides for tuning runs and tests (sdv2_tuning_set); 0 = the plan's own choice.
static int g_force_rows = 0, g_force_parts = 0;
void set_paged_overrides(int rows, int parts) {
    if (rows >= 0) g_force_rows = rows;
    if (parts >= 0) g_force_parts = parts;
}

// Parts of the key range where workgroups have 32 rows.  Memory serves the compute units alike, so a unit with two workgroups finishes
// after the units with one; many small parts even that out and even out the lengths, which only the device knows.  A part costs a
// workgroup's start (4 us) and the join's reading: it is worth 512 keys (8-bit pages, half the bytes: 1024).  With less than a
// workgroup per unit the chain of a workgroup's tiles is the time, and 128 keys, one tile a wave, are worth a part.  us, bf16, 8 key
// heads, equal lengths, this rule / best number of parts: 64 x 7584 keys 362 / 337 (one), 32 x 12 000 293 / 271 (three; one 349), 32 x 700 26.1 / 23.7
// (two), 12 x 3000 36.4 / 35.7, 4 x 3000 17.5 / 17.4 (eight; one 35.5), 4 x 700 12.7 / 11.9, 1 x 12 000 17.6 / 17.6 (32; one 117), 1 x 3000 13.4 / 12.7.
// 64 x 1 to 16 000: 385 / 366 (eight), one part 392; of 8 bits 205 / 199 (six), one 214.  Equal lengths want few parts and ragged ones more,
// and the host knows the longest only.
static int token_parts(long long workgroups, int keys, int e4m3) {
    const long long spread = min((4096 + workgroups - 1) / workgroups, (long long)(keys / (e4m3 ? 1024 : 512)));
    const long long chain = min(kUnits / workgroups, (long long)(keys / 128));
    return (int)max(max(spread, chain >= 4 ? chain : 1ll), 1ll);
}

// More rows than that: the form and the parts by an estimate of the time, us,
//   rounds (tiles per + start), rounds of `slots` workgroups, the last by how much of it is filled (two workgroups on a unit share it),
//   or the keys' bytes at `rate` where that is longer,  + join per part and its bytes.
// Fitted to 1056 launches of 38 shapes (100 to 9360 rows times 1 to 8 in a group, 700 to 33 000 keys, 1 to 40 key heads, both formats, every
// form in 1 to 32 parts) when p was one bf16 number: rms error 15 %, the form picked 2 % slower than the best of all in the mean.  Of the
// present kernels (bf16 pages 10 to 20 % slower in every form) over 98 shapes of both formats drawn afterwards, 12 to 2500 rows a sequence: 6.6 % slower
// in the mean; a new fit to those was no better on shapes of yet another draw.  The largest losses, up to 60 %, are where the estimate
// has the workgroups just fill the units: numbers that no row tile has take places too.  What it replaced, 128 rows up to 128 and
// 256 beyond in as many parts as fill the units (both then): 8 x 64 new tokens over 8000 keys 135.6 -> 103.3, 3 x 200 over 12 000 236.9 -> 146.4,
// of 8 bits 8 x 16 over 8000 79.0 -> 47.7, 333 over 33 000 333 -> 209.
struct FormCost {
    int rows, keys, slots;
    float two, one, start, rate;      // a tile of keys (of the four waves, where they share them out) with both slots of a unit taken and with one
};
static const FormCost kForms[2][3] = {{{32, 128, 512, 1.67f, 1.10f, 3.6f, 2.2e7f}, {128, 64, 512, 2.12f, 1.20f, 5.3f, 4.1e6f}, {256, 64, 256, 1.76f, 1.37f, 7.8f, 3.2e6f}},
                                      {{32, 128, 512, 1.35f, 0.80f, 3.7f, 1.3e7f}, {128, 64, 512, 2.26f, 1.50f, 5.9f, 2.5e6f}, {256, 64, 256, 1.80f, 1.55f, 10.f, 2.0e6f}}};
constexpr float kJoin = 9.0f, kJoinRate = 8e6f;      // us, bytes per us
constexpr int kMostParts = 32;
constexpr long long kMostWorkgroups = 1ll << 22;     // of up to 512 threads: a grid has fewer than 2^32

static float form_cost(const FormCost& f, const RaggedArgs& b, int group, int max_q_len, float keys, int e4m3, int parts) {
    const long long tiles_of_rows = min((long long)b.n_seqs * (((long long)max_q_len * group + f.rows - 1) / f.rows),
                                        (long long)b.n_tokens * group / f.rows + b.n_seqs);
    const long long wgs = tiles_of_rows * b.kv_heads * parts;
    const float tiles = ceilf(ceilf(keys / (float)f.keys) / (float)parts);
    const int rest = (int)(wgs % f.slots);
    float us = (float)(wgs / f.slots) * (tiles * f.two + f.start);
    if (rest > 0) {
        const float share = f.slots == kUnits ? (float)rest / kUnits : rest <= kUnits ? 0.0f : (float)(rest - kUnits) / kUnits;
        us += tiles * (f.one + (f.two - f.one) * share) + f.start;
    }
    const float bytes = (float)b.n_seqs * keys * b.kv_heads * (4.0f * D / (1 + e4m3)) * (f.rows == 32 ? fmaxf(1.0f, (float)max_q_len * group / 32) : 1.0f);
    us = fmaxf(us, bytes / f.rate);
    if (parts > 1) us += kJoin + (float)parts * b.n_tokens * b.kv_heads * group * (8.0f * D + 16.0f) / kJoinRate;
    return us;
}

PagedAttnPlan plan_paged_attention(const RaggedArgs& b, const MaskArgs& mask, int q_heads, int max_q_len, int max_kv_len, int e4m3) {
    const int group = q_heads / b.kv_heads;
    const long long rows = (long long)max_q_len * group;
    // keys that a workgroup's rows see at most
    long long keys = max_kv_len;
    if (mask.window > 0) keys = min(keys, (long long)mask.window + mask.sink + min(max_q_len, 256 / group + 1) + mask.block);
    int form = 32, parts = 1;
    if (rows <= 32 && (g_force_rows == 0 || g_force_rows == 32)) {
        parts = token_parts(max((long long)b.n_tokens * group / 32, (long long)b.n_seqs) * b.kv_heads, (int)keys, e4m3);
    } else {
        // under a causal mask rows see half of the new tokens in the mean
        const float mean = mask.block > 0 && mask.window == 0 ? fmaxf((float)keys - 0.5f * max_q_len, 64.0f) : (float)keys;
        float best = INFINITY;
        for (const FormCost& f : kForms[e4m3]) {
            if (g_force_rows > 0 && f.rows != g_force_rows) continue;
            for (int p = 1; p <= kMostParts && (p == 1 || (p - 1) * 2 * f.keys < keys); ++p) {
                const float us = form_cost(f, b, group, max_q_len, mean, e4m3, p);
                if (us < best) best = us, form = f.rows, parts = p;
                if (g_force_parts > 0) break;
            }
        }
    }
    const int key_tile = form == 32 ? 32 : 64, tiles = (int)((keys + key_tile - 1) / key_tile);
    if (g_force_parts > 0) parts = min(g_force_parts, max(tiles, 1));
    parts = (int)max(1ll, min((long long)parts, kMostWorkgroups / (((long long)b.n_tokens * group / form + b.n_seqs) * b.kv_heads)));
    PagedAttnPlan p{form, 1, max(1, (tiles + parts - 1) / parts)};
    p.parts = max(1, (tiles + p.part_tiles - 1) / p.part_tiles);
    return p;
}

hipError_t launch_paged_attention(const PagedAttnArgs& args, const PagedAttnPlan& plan, int e4m3, hipStream_t s) {
    typedef void (*Kernel)(PagedAttnArgs);
    PagedAttnArgs a = args;
    a.parts = plan.parts;
    a.part_tiles = plan.part_tiles;
    a.row_tiles = (int)((long long)a.batch.n_tokens * a.group / plan.rows) + a.batch.n_seqs;
    const long long n_wg = (long long)a.row_tiles * a.batch.kv_heads * plan.parts;
    a.n_wg = (unsigned)n_wg;
    a.by_tiles = fast_div((unsigned)a.row_tiles, (unsigned long long)n_wg);
    a.by_heads = fast_div((unsigned)a.batch.kv_heads, (unsigned long long)n_wg);
    a.by_group = fast_div((unsigned)a.group, (unsigned long long)a.batch.n_tokens * a.group);
    auto go = [&](Kernel k, int threads) { hipLaunchKernelGGL(k, dim3(a.n_wg), dim3(threads), 0, s, a); };
    if (plan.rows == 32) go(e4m3 ? paged_attention_tokens_kernel<true> : paged_attention_tokens_kernel<false>, 256);
    else if (plan.rows == 128) go(e4m3 ? paged_attention_rows_kernel<true, 4> : paged_attention_rows_kernel<false, 4>, 256);
    else go(e4m3 ? paged_attention_rows_kernel<true, 8> : paged_attention_rows_kernel<false, 8>, 512);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && plan.parts > 1) {
        const long long row_heads = (long long)a.batch.n_tokens * a.q_heads;
        // (1 | 4 | 16 groups, both launches: one token over 9000 keys 22.3 | 16.8 | 15.9 us, over 33 000 48.4 | 37.0 | 34.3; 4 over 3000
        // 17.9 | 16.9 | 17.3; 64 over 9000 425 | 421 | 424; 333 over 33 000 208 | 210 | 217)
        const int groups = plan.parts > 16 && row_heads <= 4096 ? 16 : plan.parts > 4 && row_heads <= 16384 ? 4 : 1;
        const dim3 grid((unsigned)((row_heads * groups + 15) / 16));
        if (groups == 16) hipLaunchKernelGGL(paged_attention_join_kernel<16>, grid, dim3(256), 0, s, a);
        else if (groups == 4) hipLaunchKernelGGL(paged_attention_join_kernel<4>, grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(paged_attention_join_kernel<1>, grid, dim3(256), 0, s, a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace sdv2
