// Eviction from the key/value cache by accumulated attention weight.
//
// Per (sequence, head) row: a radix select (digits of 11, 11 and 10 bits of an order-preserving 32-bit key; protected
// entries have the highest key, NaN the lowest) finds the key of the last kept entry and how many entries with that
// key are kept (the lower slots); one ordered scan then splits the slots into kept below the budget (they stay), freed
// slots and kept entries beyond the budget (the i-th of them goes to the i-th freed slot).  A second kernel moves the
// rows.  All decisions are integer, so the result is exact.
#include "si_kv.cuh"

namespace {

constexpr int kRowThreads = 1024;
constexpr int kBins = 2048;

struct EvictArgs {
    si_kv_view src, dst;
    const int32_t *q_pos;
    int n_new, budget, n_sink, n_recent, in_place;
    int stride;                          // min(budget, src.cap): slots that can be filled
    int32_t *kept, *len_out, *source;    // source: int32 [rows][stride]
    int32_t *freed, *movers;             // [rows][cap / 2 + 1] each
    int32_t *status;
};

__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    if (w == 0.f) w = 0.f;
    const uint32_t b = __float_as_uint(w);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

__device__ __forceinline__ int entries(const EvictArgs &A, int b) {
    const int n = si_kv_len(A.src, b, A.status) + A.n_new;
    if (n > A.src.cap) { si_report(A.status, SI_ERR_OUT_OF_RANGE); return A.src.cap; }
    return n;
}

// exclusive scan over the block of two counters packed in 64 bits; *total gets the sum
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long *tot, unsigned long long *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long t = __shfl_up_sync(0xFFFFFFFFu, inc, o);
        if (lane >= o) inc += t;
    }
    __syncthreads();
    if (lane == 31) tot[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        const unsigned long long w = tot[lane];
        unsigned long long winc = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long t = __shfl_up_sync(0xFFFFFFFFu, winc, o);
            if (lane >= o) winc += t;
        }
        tot[lane] = winc - w;
        if (lane == 31) *total = winc;
    }
    __syncthreads();
    return tot[warp] + inc - v;
}

__global__ void __launch_bounds__(kRowThreads) evict_select_kernel(const EvictArgs A) {
    __shared__ unsigned int hist[kBins];
    __shared__ unsigned long long tot[32], total;
    __shared__ uint32_t sh_prefix;
    __shared__ int sh_need;
    const int tid = threadIdx.x, b = blockIdx.y, h = blockIdx.x, row = b * A.src.H + h;
    const int n = entries(A, b), budget = A.budget;
    int32_t *source = A.source + (size_t)row * A.stride;
    if (n <= budget) {
        for (int j = tid; j < A.stride; j += kRowThreads) source[j] = j < n ? j : -1;
        return;
    }
    const float *w = A.src.weight + A.src.meta(b, h);
    const int32_t *pos = A.src.pos ? A.src.pos + A.src.meta(b, h) : nullptr;
    const int last = A.q_pos ? A.q_pos[b] : n - 1;
    auto key = [&](int j) -> uint32_t {
        const int p = pos ? pos[j] : j;
        return p < A.n_sink || (long long)p > (long long)last - A.n_recent ? 0xFFFFFFFFu : weight_key(w[j]);
    };
    // radix select of the budget-th largest key
    uint32_t prefix = 0, mask = 0;
    int need = budget;
    const int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
    for (int pass = 0; pass < 3; ++pass) {
        for (int i = tid; i < kBins; i += kRowThreads) hist[i] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kRowThreads) {
            const uint32_t k = key(j);
            if ((k & mask) == prefix) atomicAdd(&hist[(k >> shifts[pass]) & ((1u << bits[pass]) - 1)], 1u);
        }
        __syncthreads();
        // bins from the top down: two per thread
        const int hi = kBins - 1 - 2 * tid;
        const unsigned int c0 = hist[hi], c1 = hist[hi - 1];
        const int before = (int)block_scan(c0 + c1, tot, &total);
        if (before < need && before + (int)c0 >= need) { sh_prefix = prefix | ((uint32_t)hi << shifts[pass]); sh_need = need - before; }
        else if (before + (int)c0 < need && before + (int)(c0 + c1) >= need) { sh_prefix = prefix | ((uint32_t)(hi - 1) << shifts[pass]); sh_need = need - before - (int)c0; }
        __syncthreads();
        prefix = sh_prefix; need = sh_need;
        mask |= ((1u << bits[pass]) - 1) << shifts[pass];
        __syncthreads();
    }
    // ordered scan: ties with the last kept key go to the lower slots; freed slots and movers are listed in order
    int32_t *freed = A.freed + (size_t)row * (A.src.cap / 2 + 1), *movers = A.movers + (size_t)row * (A.src.cap / 2 + 1);
    int ties = 0, n_freed = 0, n_movers = 0;
    for (int j0 = 0; j0 < n; j0 += kRowThreads) {
        const int j = j0 + tid;
        const uint32_t k = j < n ? key(j) : 0u;
        const bool tie = j < n && k == prefix;
        const int tie_rank = ties + (int)block_scan(tie, tot, &total);
        ties += (int)total;
        const bool keep = j < n && (k > prefix || (tie && tie_rank < need));
        const bool is_freed = j < budget && !keep, is_mover = j >= budget && keep;
        const unsigned long long r = block_scan((unsigned long long)is_freed << 32 | (unsigned long long)is_mover, tot, &total);
        if (j < budget && keep) source[j] = j;
        if (is_freed) freed[n_freed + (int)(r >> 32)] = j;
        if (is_mover) movers[n_movers + (int)(r & 0xFFFFFFFFu)] = j;
        n_freed += (int)(total >> 32); n_movers += (int)(total & 0xFFFFFFFFu);
    }
    __syncthreads();
    for (int i = tid; i < n_freed; i += kRowThreads) source[freed[i]] = movers[i];
}

// One warp per kept slot: the key, the value, the position and the weight; nothing to do for an entry that stays.
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictArgs A) {
    const int b = blockIdx.z, h = blockIdx.y, row = b * A.src.H + h, lane = threadIdx.x & 31;
    if (h == 0 && blockIdx.x == 0 && threadIdx.x == 0 && A.len_out) A.len_out[b] = min(entries(A, b), A.budget);
    const int slot = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (slot >= A.budget) return;
    const int j = slot < A.stride ? A.source[(size_t)row * A.stride + slot] : -1;
    if (lane == 0 && A.kept) A.kept[(size_t)row * A.budget + slot] = j;
    if (j < 0 || (A.in_place && j == slot)) return;
    const long long from = A.src.row(b, h, j), to = A.dst.row(b, h, slot);
    for (int c = lane; c < A.src.D / 4; c += 32) {       // 16-byte pieces: the first half of the lanes K, the others V
        const bool is_v = c >= A.src.D / 8;
        const int at = (is_v ? c - A.src.D / 8 : c) * 8;
        *reinterpret_cast<uint4 *>((is_v ? A.dst.v : A.dst.k) + to + at) = *reinterpret_cast<const uint4 *>((is_v ? A.src.v : A.src.k) + from + at);
    }
    if (lane == 0) {
        A.dst.pos[A.dst.meta(b, h) + slot] = A.src.pos ? A.src.pos[A.src.meta(b, h) + j] : j;
        A.dst.weight[A.dst.meta(b, h) + slot] = A.src.weight[A.src.meta(b, h) + j];
    }
}

size_t evict_ws_bytes(const si_kv_t *kv) {
    const size_t rows = (size_t)kv->n_seqs * kv->n_kv_heads;
    return si_align_up(rows * kv->capacity * 4, 256) + 2 * si_align_up(rows * ((size_t)kv->capacity / 2 + 1) * 4, 256);
}

}  // namespace

int si_sm_count() {
    static std::atomic<int> known{0};
    int n = known.load();
    if (!n) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
            (void)cudaGetLastError();
            return SI_NUM_SMS_FALLBACK;
        }
        known.store(n);
    }
    return n;
}

extern "C" int si_kv_workspace_bytes(const si_kv_t *kv, int n_q_heads, int T, size_t *bytes_out) {
    const int rc = si_kv_check(kv);
    if (rc) return rc;
    if (!bytes_out || n_q_heads < 0 || T < 0 || n_q_heads % kv->n_kv_heads) return SI_ERR_INVALID_ARG;
    size_t most = kv->weight ? evict_ws_bytes(kv) : 0;
    if (n_q_heads && T) {
        if (n_q_heads / kv->n_kv_heads > 128) return SI_ERR_UNSUPPORTED;
        const size_t each[3] = {si_attn_decode_ws_bytes(kv, n_q_heads), si_attn_prefill_ws_bytes(kv, n_q_heads, T), kv->weight ? si_attn_weights_ws_bytes(kv) : 0};
        for (size_t b : each) most = b > most ? b : most;
    }
    *bytes_out = most;
    return SI_OK;
}

extern "C" int si_kv_evict(const si_kv_t *src, const si_kv_t *dst, const int32_t *q_pos, int n_new, int budget, int n_sink,
                           int n_recent, int32_t *kept, int32_t *len_out, void *workspace, size_t ws_bytes, int32_t *status_dev,
                           void *stream) {
    int rc = si_kv_check(src);
    if (rc) return rc;
    if ((rc = si_kv_check(dst))) return rc;
    if (budget < 1 || n_new < 0 || n_sink < 0 || n_recent < 0 || (long long)n_sink + n_recent > budget || budget > dst->capacity) return SI_ERR_INVALID_ARG;
    if (src->n_seqs != dst->n_seqs || src->n_kv_heads != dst->n_kv_heads || src->head_dim != dst->head_dim || src->dtype != dst->dtype) return SI_ERR_INVALID_ARG;
    if (src->n_seqs == 0) return SI_OK;
    const bool in_place = src->k == dst->k;
    if (!src->weight || !dst->weight || !dst->pos || (src->pos && !q_pos) || (in_place && !src->pos)) return SI_ERR_INVALID_ARG;
    if (in_place && (src->v != dst->v || src->pos != dst->pos || src->weight != dst->weight || src->seq_stride != dst->seq_stride ||
                     src->head_stride != dst->head_stride || src->row_stride != dst->row_stride || src->capacity != dst->capacity)) return SI_ERR_INVALID_ARG;
    if (ws_bytes < evict_ws_bytes(src)) return SI_ERR_NOMEM;
    if (!workspace) return SI_ERR_INVALID_ARG;
    if ((uintptr_t)workspace & 255) return SI_ERR_ALIGNMENT;
    const size_t rows = (size_t)src->n_seqs * src->n_kv_heads;
    char *ws = (char *)workspace;
    EvictArgs A{si_kv_view_of(src), si_kv_view_of(dst), q_pos, n_new, budget, n_sink, n_recent, in_place,
                budget < src->capacity ? budget : src->capacity, kept, len_out,
                (int32_t *)ws, nullptr, nullptr, status_dev};
    A.freed = (int32_t *)(ws + si_align_up(rows * src->capacity * 4, 256));
    A.movers = (int32_t *)((char *)A.freed + si_align_up(rows * ((size_t)src->capacity / 2 + 1) * 4, 256));
    const cudaStream_t st = (cudaStream_t)stream;
    evict_select_kernel<<<dim3(src->n_kv_heads, src->n_seqs), kRowThreads, 0, st>>>(A);
    SI_CUDA_TRY(cudaGetLastError());
    evict_move_kernel<<<dim3((budget + 7) / 8, src->n_kv_heads, src->n_seqs), 256, 0, st>>>(A);
    SI_CUDA_TRY(cudaGetLastError());
    return SI_OK;
}
