// Attention of a ragged batch of new tokens over a paged cache.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j) over the keys j that the row may see; the zero row where there is none.
//
// One wave per row and query head, a key at a time, with the running maximum and sum of the softmax.
#include "ragged.h"

namespace sdv2 {

namespace {

constexpr int D = kHeadDim;

template <bool E4M3>
__global__ __launch_bounds__(256) void paged_attention_row_kernel(PagedAttnArgs a) {
    const int lane = threadIdx.x & 63;
    const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t = __builtin_amdgcn_readfirstlane((int)(wave / a.q_heads)), h = __builtin_amdgcn_readfirstlane((int)(wave % a.q_heads));
    if (t >= a.batch.n_tokens) return;
    const int s = sequence_of_row(a.batch, t);
    if (s >= a.batch.n_seqs) return;
    const int q0 = a.batch.q_start[s], n = a.batch.q_start[s + 1] - q0;
    const int kv_len = (int)min((long long)a.batch.kv_len[s], (long long)a.batch.table_stride << a.batch.page_shift);
    const RowKeys keys = row_keys(a.mask, t - q0, n, kv_len);
    const int hk = h / a.group;
    const bf16x2 q = *reinterpret_cast<const bf16x2*>(a.q + t * a.q_stride + h * D + lane * 2);
    float m = -INFINITY, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
    for (int j = 0; j < keys.end; ++j) {
        if (j >= keys.sink && j < keys.low) j = keys.low;
        const int page = a.batch.table[(long long)s * a.batch.table_stride + (j >> a.batch.page_shift)];
        if ((unsigned)page >= (unsigned)a.batch.n_pages) continue;
        const long long at =
            ((((long long)page * a.batch.kv_heads + hk) << a.batch.page_shift) + (j & ((1 << a.batch.page_shift) - 1))) * D + lane * 2;
        float k0, k1, v0, v1;
        if (E4M3) {
            const bf16x2 k = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(*reinterpret_cast<const unsigned short*>(static_cast<const unsigned char*>(a.k_pages) + at), 1.0f, false);
            const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(*reinterpret_cast<const unsigned short*>(static_cast<const unsigned char*>(a.v_pages) + at), 1.0f, false);
            k0 = (float)k[0], k1 = (float)k[1], v0 = (float)v[0], v1 = (float)v[1];
        } else {
            const bf16x2 k = *reinterpret_cast<const bf16x2*>(static_cast<const bf16*>(a.k_pages) + at);
            const bf16x2 v = *reinterpret_cast<const bf16x2*>(static_cast<const bf16*>(a.v_pages) + at);
            k0 = (float)k[0], k1 = (float)k[1], v0 = (float)v[0], v1 = (float)v[1];
        }
        const float x = wave_sum((float)q[0] * k0 + (float)q[1] * k1) * a.mask.scale_log2e;
        const float top = fmaxf(m, x);
        const float keep = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top), p = __builtin_amdgcn_exp2f(x - top);
        l = l * keep + p;
        o0 = o0 * keep + p * v0;
        o1 = o1 * keep + p * v1;
        m = top;
    }
    const float inv = l != 0.0f ? a.v_scale / l : 0.0f;
    *reinterpret_cast<bf16x2*>(a.o + t * a.o_stride + h * D + lane * 2) = bf16x2{(bf16)(o0 * inv), (bf16)(o1 * inv)};
}

}  // namespace

PagedAttnPlan plan_paged_attention(const RaggedArgs&, int, int, int, int) { return PagedAttnPlan{0, 1}; }

hipError_t launch_paged_attention(const PagedAttnArgs& a, const PagedAttnPlan&, int e4m3, hipStream_t s) {
    const long long waves = (long long)a.batch.n_tokens * a.q_heads;
    const dim3 grid((unsigned)((waves + 3) / 4));
    if (e4m3) hipLaunchKernelGGL(paged_attention_row_kernel<true>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(paged_attention_row_kernel<false>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace sdv2
