// Low-rank adapters of many requests beside a shared projection:  out = y + scale (x A^T) B^T, each sequence with its own A [r, K],
// B [N, r] and scale, or none.
//
// Two launches: u = x A^T in 32 bits, a wave per row and eight ranks, then the update, a thread per output.
#include "ragged.h"

namespace sdv2 {

namespace {

__device__ __forceinline__ int adapter_of_row(const LoraArgs& a, int t, int* seq) {
    RaggedArgs b{};
    b.q_start = a.q_start;
    b.n_seqs = a.n_seqs;
    *seq = sequence_of_row(b, t);
    if (*seq >= a.n_seqs) return -1;
    const int id = a.adapter[*seq];
    return (unsigned)id < (unsigned)a.n_adapters ? id : -1;
}

__global__ __launch_bounds__(256) void lora_down_kernel(LoraArgs a) {
    const int lane = threadIdx.x & 63, t = blockIdx.x;
    int seq;
    const int id = adapter_of_row(a, t, &seq);
    if (id < 0) return;
    for (int r = threadIdx.x >> 6; r < a.rank; r += 4) {
        const bf16* x = a.x + t * a.x_stride;
        const bf16* w = a.a + ((long long)id * a.rank + r) * a.K;
        float sum = 0.0f;
        for (int k = lane; k < a.K; k += 64) sum += (float)x[k] * (float)w[k];
        sum = wave_sum(sum);
        if (lane == 0) a.u[(long long)t * a.rank + r] = sum;
    }
}

__global__ __launch_bounds__(256) void lora_up_kernel(LoraArgs a) {
    const int t = blockIdx.x, n = blockIdx.y * 256 + threadIdx.x;
    int seq;
    const int id = adapter_of_row(a, t, &seq);
    if (seq >= a.n_seqs || n >= a.N) return;
    float sum = 0.0f;
    if (id >= 0) {
        const bf16* w = a.b + ((long long)id * a.N + n) * a.rank;
        for (int r = 0; r < a.rank; ++r) sum += a.u[(long long)t * a.rank + r] * (float)w[r];
        if (a.scale != nullptr) sum *= a.scale[id];
    }
    const long long from = t * a.y_stride + n, to = t * a.out_stride + n;
    if (a.fp32) static_cast<float*>(a.out)[to] = static_cast<const float*>(a.y)[from] + sum;
    else static_cast<bf16*>(a.out)[to] = (bf16)((float)static_cast<const bf16*>(a.y)[from] + sum);
}

}  // namespace

int lora_parts(int, int, int, int, int) { return 1; }

hipError_t launch_lora(const LoraArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(lora_down_kernel, dim3(a.n_tokens), dim3(256), 0, s, a);
    hipLaunchKernelGGL(lora_up_kernel, dim3(a.n_tokens, (a.N + 255) / 256), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace sdv2
