// Attention over the key/value cache: o_i = sum_j p_ij v_j, p_i = softmax over the visible entries of scale q_i . k_j.
// Simple form: one warp per query row (sequence, token, query head); 32 entries at a time, lane = entry for the dot
// products, lane = output columns for the sum, running maximum and sum of the softmax in between.
#include "si_kv.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// dot product of a 16-bit row in global memory with a float row in shared memory
template <int DT, int D> __device__ __forceinline__ float dot_row(const uint16_t *row, const float *q) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < D; c += 8) {
        const uint4 w = *reinterpret_cast<const uint4 *>(row + c);
        s = fmaf(si_cvt<DT>::lo(w.x), q[c], s); s = fmaf(si_cvt<DT>::hi(w.x), q[c + 1], s);
        s = fmaf(si_cvt<DT>::lo(w.y), q[c + 2], s); s = fmaf(si_cvt<DT>::hi(w.y), q[c + 3], s);
        s = fmaf(si_cvt<DT>::lo(w.z), q[c + 4], s); s = fmaf(si_cvt<DT>::hi(w.z), q[c + 5], s);
        s = fmaf(si_cvt<DT>::lo(w.w), q[c + 6], s); s = fmaf(si_cvt<DT>::hi(w.w), q[c + 7], s);
    }
    return s;
}

struct AttnArgs {
    si_kv_view kv;
    const uint16_t *q;
    long long q_ss, q_ts;
    int T, Hq, window, n_sink;
    float scale;
    uint16_t *out;
    float *lse;
    int32_t *status;
};

// weight[b, h, j] += sum over queries and the group's heads of exp(scale q . k_j - lse): one warp per entry, lane =
// query row.
template <int DT, int D>
__global__ void __launch_bounds__(128) attn_weights_kernel(const AttnArgs A, const float *__restrict__ lse) {
    __shared__ float sk[4][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, G = A.Hq / A.kv.H;
    const int j = blockIdx.x * 4 + warp, h = blockIdx.y, b = blockIdx.z;
    const int n = si_kv_len(A.kv, b, A.status);
    if (j >= n) return;
    for (int c = lane; c < D; c += 32) sk[warp][c] = si_cvt<DT>::lo(A.kv.k[A.kv.row(b, h, j) + c]);
    __syncwarp();
    float sum = 0.f;
    for (int r = lane; r < A.T * G; r += 32) {
        const int i = r / G, hq = h * G + r % G, s = n - A.T + i;
        if (!si_visible(j, s, si_window_lo(s, A.window), A.n_sink)) continue;
        const float x = dot_row<DT, D>(A.q + b * A.q_ss + i * A.q_ts + (long long)hq * D, sk[warp]) * A.scale;
        sum += exp2f((x - lse[((long long)b * A.T + i) * A.Hq + hq]) * kLog2e);
    }
    sum = warp_sum(sum);
    if (lane == 0) A.kv.weight[A.kv.meta(b, h) + j] += sum;
}

template <typename F> int by_type(int dtype, int D, F f) {
    if (dtype == SI_BF16) return D == 128 ? f.template operator()<SI_BF16, 128>() : f.template operator()<SI_BF16, 64>();
    return D == 128 ? f.template operator()<SI_F16, 128>() : f.template operator()<SI_F16, 64>();
}
struct Weights {
    const AttnArgs &A; const float *lse; cudaStream_t st;
    template <int DT, int D> int operator()() {
        attn_weights_kernel<DT, D><<<dim3((A.kv.cap + 3) / 4, A.kv.H, A.kv.B), 128, 0, st>>>(A, lse);
        SI_CUDA_TRY(cudaGetLastError());
        return SI_OK;
    }
};

}  // namespace

extern "C" int si_attn_weights(const si_kv_t *kv, const void *q, long long q_seq_stride, long long q_tok_stride, int T,
                               int n_q_heads, int window, int n_sink, float scale, const float *lse, void *workspace,
                               size_t ws_bytes, int32_t *status_dev, void *stream) {
    const int rc = si_attn_check(kv, n_q_heads, window, n_sink, scale);
    if (rc) return rc;
    if (T < 0) return SI_ERR_INVALID_ARG;
    if (kv->n_seqs == 0 || T == 0) return SI_OK;
    if (!q || !lse || !kv->weight || q_seq_stride < 0 || q_tok_stride < 0) return SI_ERR_INVALID_ARG;
    if (kv->pos) return SI_ERR_UNSUPPORTED;
    if (!si_aligned16(q) || ((q_seq_stride | q_tok_stride) & 7)) return SI_ERR_ALIGNMENT;
    const AttnArgs A{si_kv_view_of(kv), (const uint16_t *)q, q_seq_stride, q_tok_stride, T, n_q_heads, window, n_sink, scale,
                     nullptr, nullptr, status_dev};
    return by_type(kv->dtype, kv->head_dim, Weights{A, lse, (cudaStream_t)stream});
}
