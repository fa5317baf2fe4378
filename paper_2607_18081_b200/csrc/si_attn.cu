// Attention over the key/value cache: o_i = sum_j p_ij v_j, p_i = softmax over the visible entries of scale q_i . k_j.
// Simple form: one warp per query row (sequence, token, query head); 32 entries at a time, lane = entry for the dot
// products, lane = output columns for the sum, running maximum and sum of the softmax in between.
#include "si_kv.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}
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

template <int DT, int D>
__global__ void __launch_bounds__(128) attn_rows_kernel(const AttnArgs A) {
    __shared__ float sq[4][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long r = (long long)blockIdx.x * 4 + warp, rows = (long long)A.kv.B * A.T * A.Hq;
    if (r >= rows) return;
    const int hq = (int)(r % A.Hq), i = (int)(r / A.Hq % A.T), b = (int)(r / A.Hq / A.T), h = hq / (A.Hq / A.kv.H);
    const int n = si_kv_len(A.kv, b, A.status), s = n - A.T + i, lo = si_window_lo(s, A.window);
    const uint16_t *q = A.q + b * A.q_ss + i * A.q_ts + (long long)hq * D;
    for (int c = lane; c < D; c += 32) sq[warp][c] = si_cvt<DT>::lo(q[c]);
    __syncwarp();
    float m = -INFINITY, l = 0.f, o[D / 32] = {};
    for (int j0 = 0; j0 < n; j0 += 32) {
        const int j = j0 + lane;
        const bool vis = j < n && si_visible(j, s, lo, A.n_sink);
        if (!__any_sync(0xFFFFFFFFu, vis)) continue;
        const float x = vis ? dot_row<DT, D>(A.kv.k + A.kv.row(b, h, j), sq[warp]) * A.scale : -INFINITY;
        const float m2 = fmaxf(m, warp_max(x)), base = m2 == -INFINITY ? 0.f : m2;
        const float p = vis ? exp2f((x - base) * kLog2e) : 0.f, f = exp2f((m - base) * kLog2e);
        l = l * f + warp_sum(p);
        m = m2;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) o[c] *= f;
        for (int t = 0; t < 32; ++t) {
            if (!__shfl_sync(0xFFFFFFFFu, (int)vis, t)) continue;
            const float pt = __shfl_sync(0xFFFFFFFFu, p, t);
            const uint16_t *v = A.kv.v + A.kv.row(b, h, j0 + t);
#pragma unroll
            for (int c = 0; c < D / 32; ++c) o[c] = fmaf(pt, si_cvt<DT>::lo(v[c * 32 + lane]), o[c]);
        }
    }
    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);      // no visible entry: 0; NaN stays NaN
#pragma unroll
    for (int c = 0; c < D / 32; ++c) A.out[r * D + c * 32 + lane] = si_cvt<DT>::from_float(o[c] * inv);
    if (A.lse && lane == 0) A.lse[r] = l == 0.f ? -INFINITY : m + logf(l);
}

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
struct Rows {
    const AttnArgs &A; cudaStream_t st;
    template <int DT, int D> int operator()() {
        const long long rows = (long long)A.kv.B * A.T * A.Hq;
        attn_rows_kernel<DT, D><<<(unsigned)((rows + 3) / 4), 128, 0, st>>>(A);
        SI_CUDA_TRY(cudaGetLastError());
        return SI_OK;
    }
};
struct Weights {
    const AttnArgs &A; const float *lse; cudaStream_t st;
    template <int DT, int D> int operator()() {
        attn_weights_kernel<DT, D><<<dim3((A.kv.cap + 3) / 4, A.kv.H, A.kv.B), 128, 0, st>>>(A, lse);
        SI_CUDA_TRY(cudaGetLastError());
        return SI_OK;
    }
};

}  // namespace

extern "C" int si_attn_prefill(const si_kv_t *kv, const void *q, long long q_seq_stride, long long q_tok_stride, int T,
                               int n_q_heads, int window, int n_sink, float scale, void *out, float *lse, void *workspace,
                               size_t ws_bytes, int32_t *status_dev, void *stream) {
    const int rc = si_attn_check(kv, n_q_heads, window, n_sink, scale);
    if (rc) return rc;
    if (T < 0) return SI_ERR_INVALID_ARG;
    if (kv->n_seqs == 0 || T == 0) return SI_OK;
    if (!q || !out || q_seq_stride < 0 || q_tok_stride < 0) return SI_ERR_INVALID_ARG;
    if (kv->pos) return SI_ERR_UNSUPPORTED;
    if (!si_aligned16(q) || !si_aligned16(out) || ((q_seq_stride | q_tok_stride) & 7)) return SI_ERR_ALIGNMENT;
    const AttnArgs A{si_kv_view_of(kv), (const uint16_t *)q, q_seq_stride, q_tok_stride, T, n_q_heads, window, n_sink, scale,
                     (uint16_t *)out, lse, status_dev};
    return by_type(kv->dtype, kv->head_dim, Rows{A, (cudaStream_t)stream});
}

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
