// The key/value cache as the kernels see it, and what the calls on it share: argument checks, which entries a query
// sees, the status word.
#pragma once
#include <limits.h>

#include "si_common.cuh"

struct si_kv_view {
    uint16_t *k, *v;
    float *weight;
    int32_t *pos;
    const int32_t *len;
    long long ss, hs, rs;        // element strides: sequence, head, entry
    int B, H, D, cap;
    __host__ __device__ long long row(int b, int h, int j) const { return b * ss + h * hs + j * rs; }
    __host__ __device__ long long meta(int b, int h) const { return ((long long)b * H + h) * cap; }
};

inline si_kv_view si_kv_view_of(const si_kv_t *kv) {
    return {(uint16_t *)kv->k, (uint16_t *)kv->v, kv->weight, kv->pos, kv->len, kv->seq_stride, kv->head_stride,
            kv->row_stride, kv->n_seqs, kv->n_kv_heads, kv->head_dim, kv->capacity};
}

// 4-byte words (lengths, positions, weights, lse, status), any of them NULL.
template <typename... P> bool si_aligned4(const P *...p) { return (((uintptr_t)p | ...) & 3u) == 0; }

// Host checks common to all calls on a cache.
inline int si_kv_check(const si_kv_t *kv) {
    if (!kv || kv->n_seqs < 0 || kv->n_kv_heads < 1 || kv->capacity < 1 || kv->head_dim < 1) return SI_ERR_INVALID_ARG;
    if (kv->dtype != SI_F16 && kv->dtype != SI_BF16) return SI_ERR_INVALID_ARG;
    if (kv->n_kv_heads > 65535 || kv->n_seqs > 65535) return SI_ERR_INVALID_ARG;
    if (kv->head_dim != 64 && kv->head_dim != 128) return SI_ERR_UNSUPPORTED;
    if (kv->n_seqs == 0) return SI_OK;
    if (!kv->k || !kv->v || !kv->len) return SI_ERR_INVALID_ARG;
    if (kv->row_stride < kv->head_dim || kv->head_stride < 0 || kv->seq_stride < 0) return SI_ERR_INVALID_ARG;
    if (!si_aligned16(kv->k) || !si_aligned16(kv->v) || ((kv->row_stride | kv->head_stride | kv->seq_stride) & 7)) return SI_ERR_ALIGNMENT;
    if (!si_aligned4(kv->weight, kv->pos, kv->len)) return SI_ERR_ALIGNMENT;
    return SI_OK;
}

// Two rows of the cache share memory through a zero stride: it can be read, but not written.
inline bool si_kv_shared(const si_kv_t *kv) {
    return (kv->n_seqs > 1 && kv->seq_stride == 0) || (kv->n_kv_heads > 1 && kv->head_stride == 0);
}

// ... and of those that bring queries.
inline int si_attn_check(const si_kv_t *kv, int n_q_heads, int window, int n_sink, float scale) {
    const int rc = si_kv_check(kv);
    if (rc) return rc;
    if (n_q_heads < 1 || n_q_heads % kv->n_kv_heads || window < 0 || n_sink < 0) return SI_ERR_INVALID_ARG;
    if (!(scale > -2.0e38f && scale < 2.0e38f)) return SI_ERR_INVALID_ARG;      // scale log2(e) is finite too
    if (n_q_heads / kv->n_kv_heads > 128) return SI_ERR_UNSUPPORTED;
    return SI_OK;
}

// SMs of the current device when first asked (all devices of a machine are alike here)
int si_sm_count();

// Allows `kernel` that much dynamic shared memory, once per device (`done`: a bit per device).
template <typename K> int si_allow_smem(K kernel, int bytes, std::atomic<unsigned long long> &done) {
    int dev = 0;
    SI_CUDA_TRY(cudaGetDevice(&dev));
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(done.load() & bit)) {
        SI_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
        done.fetch_or(bit);
    }
    return SI_OK;
}

// Every kernel of these calls is a programmatic dependent that waits for the kernel ahead of it before it touches memory, and
// lets its own dependents start early; each call says so by si_mt_forget() before it launches.

// implemented in si_attn_decode.cu / si_attn_prefill.cu / si_attn_weights.cu
size_t si_attn_decode_ws_bytes(const si_kv_t *kv, int n_q_heads);
size_t si_attn_prefill_ws_bytes(const si_kv_t *kv, int n_q_heads, int T);
size_t si_attn_weights_ws_bytes(const si_kv_t *kv);

__device__ __forceinline__ void si_report(int32_t *status, int err) { if (status) atomicCAS(status, 0, err); }

// Entries in use, clamped to the capacity.
__device__ __forceinline__ int si_kv_len(const si_kv_view &kv, int b, int32_t *status) {
    const int n = __ldg(kv.len + b);
    if (n < 0 || n > kv.cap) { si_report(status, SI_ERR_OUT_OF_RANGE); return n < 0 ? 0 : kv.cap; }
    return n;
}

// Visibility of an entry at position p to a query at position s: p <= s and (p > lo or p < n_sink), where lo is the
// last position in front of the window (below every position when there is no window).
__device__ __forceinline__ int si_window_lo(int s, int window) {
    const long long lo = (long long)s - window;
    return window == 0 || lo < INT_MIN ? INT_MIN : (int)lo;
}
__device__ __forceinline__ bool si_visible(int p, int s, int lo, int n_sink) { return p <= s && (p > lo || p < n_sink || lo == INT_MIN); }

// Exclusive sum over the block in thread order; `sh`: THREADS / 32 + 1 ints, the last one receives the total.
template <int THREADS> __device__ __forceinline__ int si_block_scan(int v, int *sh) {
    constexpr int W = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xFFFFFFFFu, inc, o);
        if (lane >= o) inc += t;
    }
    if (lane == 31) sh[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        const int w = lane < W ? sh[lane] : 0;
        int winc = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xFFFFFFFFu, winc, o);
            if (lane >= o) winc += t;
        }
        __syncwarp();
        if (lane < W) sh[lane] = winc - w;
        if (lane == 31) sh[W] = winc;
    }
    __syncthreads();
    return sh[warp] + inc - v;
}
