// Eviction from the key/value cache by accumulated attention weight.
//
// Per (sequence, head) row: a radix select (digits of 11, 11 and 10 bits of an order-preserving 32-bit key; protected
// entries have the highest key, NaN the lowest) finds the key of the last kept entry and how many entries with that
// key are kept (the lower slots); ordered counts then split the slots into kept ones below the budget (they stay), freed
// ones and kept entries beyond the budget (the i-th of them goes to the i-th freed slot).  All decisions are integer, so the
// result is exact.
//
// A row is worked on by a cluster of 1 to 8 CTAs, each with its slice of the keys in shared memory (read once from HBM);
// the CTAs add one another's histograms and counts through distributed shared memory.  Then the rows move: bound by HBM
// (4 * head_dim bytes read and written per moved entry) in a second kernel with eight rows in flight per warp, or, in
// place with few entries over the budget (a decode step), in the same kernel.
#include "si_kv.cuh"
#include "si_tc.cuh"

namespace {

constexpr int kRowThreads = 1024;
constexpr int kBins = 2048;
constexpr int kMaxCluster = 8;
constexpr int kSliceKeys = 48 * 1024;        // keys of a slice in shared memory; longer rows read their weights again instead
constexpr int kFewMoves = 256;               // in place with at most this many entries over the budget: one kernel
constexpr int kFewOver = 4;                  // at most this many entries over the budget are looked for one by one
constexpr int kMoveRows = 8;                 // rows in flight per warp of the moving kernel

struct EvictArgs {
    si_kv_view src, dst;
    const int32_t *q_pos;
    int n_new, budget, n_sink, n_recent, in_place, move_here;
    int slots;                           // slots that `source` describes: the budget, at most the capacity if it is scratch
    int32_t *source, *lists;             // [rows][slots]: source slot of every slot (the caller's `kept` or scratch); [rows][cap + 2]:
                                         // freed slots, then (from cap / 2 + 1) the entries that fill them, at most cap / 2 each
    int list_source;                     // 0: nobody reads `source` (moves of this kernel only, no `kept`)
    int32_t *len_out;
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

__device__ __forceinline__ unsigned int ld_cluster(const unsigned int *smem, int rank) {
    unsigned int v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(si_tc::map_to_cta(si_tc::smem_u32(smem), rank)) : "memory");
    return v;
}

template <bool SMEM>
__global__ void __launch_bounds__(kRowThreads, 2) evict_select_kernel(const EvictArgs A) {
    extern __shared__ uint32_t keys[];
    __shared__ unsigned int hist[3][kBins], share[3];        // share: counts for the CTAs behind this one
    __shared__ unsigned long long tot[32], total;
    __shared__ uint32_t sh_prefix;
    __shared__ int sh_need;
    const int C = gridDim.x, rank = blockIdx.x, tid = threadIdx.x, h = blockIdx.y, b = blockIdx.z, row = b * A.src.H + h;
    si_tc::pdl_wait();                                       // a programmatic dependent too
    const int n = entries(A, b), budget = A.budget;
    int32_t *source = A.source + (size_t)row * A.slots, *freed_slots = A.lists + (size_t)row * (A.src.cap + 2), *movers = freed_slots + A.src.cap / 2 + 1;
    if (A.move_here && A.len_out && h == 0 && rank == 0 && tid == 0) A.len_out[b] = min(n, budget);
    si_tc::pdl_launch();
    if (n <= budget) {                                       // the whole cluster alike
        if (A.list_source)
            for (int j = rank * kRowThreads + tid; j < A.slots; j += C * kRowThreads) source[j] = j < n ? j : -1;
        return;
    }
    const float *w = A.src.weight + A.src.meta(b, h);
    const int32_t *pos = A.src.pos ? A.src.pos + A.src.meta(b, h) : nullptr;
    const int last = A.q_pos ? A.q_pos[b] : n - 1;
    auto key_of = [&](int p, float x) -> uint32_t {
        return p < A.n_sink || (long long)p > (long long)last - A.n_recent ? 0xFFFFFFFFu : weight_key(x);
    };
    const int len = (n + C - 1) / C, s0 = min(n, rank * len), s1 = min(n, s0 + len);     // this CTA's slots
    if (SMEM) {
        constexpr int U = 4;                                 // loads of a thread in flight: U weights, U positions
        for (int q = s0 + tid; q < s1; q += U * kRowThreads) {
            float x[U];
            int p[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = q + u * kRowThreads;
                x[u] = j < s1 ? __ldg(w + j) : 0.f;
                p[u] = pos && j < s1 ? __ldg(pos + j) : j;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (q + u * kRowThreads < s1) keys[q + u * kRowThreads - s0] = key_of(p[u], x[u]);
        }
    }
    auto key = [&](int j) -> uint32_t { return SMEM ? keys[j - s0] : key_of(pos ? pos[j] : j, w[j]); };
    auto sync = [&]() { if (C > 1) si_tc::cluster_sync_all(); else __syncthreads(); };
    auto list_stayers = [&]() {                              // freed slots are overwritten later
        if (A.list_source) for (int j = s0 + tid; j < min(s1, budget); j += kRowThreads) source[j] = j;
    };
    int moves;
    if (SMEM && C == 1 && n - budget <= kFewOver) {
        // A decode step: the few that go are found one after the other, each by one maximum over the block -- the lowest key,
        // of equal ones the highest slot (16 x 8 rows of 2049 entries: 4.8 us a step, 9.3 by histograms).
        list_stayers();
        unsigned long long out = 0;                          // this thread's slots that go, a bit per round of kRowThreads
        int gone[kFewOver];
#pragma unroll
        for (int r = 0; r < kFewOver; ++r) {
            gone[r] = INT_MAX;
            if (r >= n - budget) continue;
            unsigned long long best = 0;
            for (int j = tid, i = 0; j < n; j += kRowThreads, ++i)
                if (!(out >> i & 1)) {
                    const unsigned long long v = (unsigned long long)~keys[j] << 32 | (unsigned int)j + 1;
                    best = v > best ? v : best;
                }
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                const unsigned long long v = __shfl_xor_sync(0xFFFFFFFFu, best, o);
                best = v > best ? v : best;
            }
            __syncthreads();
            if ((tid & 31) == 0) tot[tid >> 5] = best;
            __syncthreads();
            best = tot[tid & 31];
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                const unsigned long long v = __shfl_xor_sync(0xFFFFFFFFu, best, o);
                best = v > best ? v : best;
            }
            gone[r] = (int)(unsigned int)best - 1;
            if (gone[r] % kRowThreads == tid) out |= 1ull << (gone[r] / kRowThreads);
        }
        // freed slots in ascending order, and the entries beyond the budget that stay
        moves = 0;
        if (tid == 0) {
            int m = budget;
            while (true) {
                int next = INT_MAX;
#pragma unroll
                for (int r = 0; r < kFewOver; ++r)
                    if (gone[r] < budget && gone[r] < next && (moves == 0 || gone[r] > freed_slots[moves - 1])) next = gone[r];
                if (next == INT_MAX) break;
                while (true) {
                    bool is_gone = false;
#pragma unroll
                    for (int r = 0; r < kFewOver; ++r) is_gone |= gone[r] == m;
                    if (!is_gone) break;
                    ++m;
                }
                freed_slots[moves] = next;
                movers[moves++] = m++;
            }
            sh_need = moves;
        }
        __syncthreads();
        moves = sh_need;
    } else {
        for (int i = tid; i < 3 * kBins; i += kRowThreads) hist[0][i] = 0;
        __syncthreads();
        // radix select of the budget-th largest key
        uint32_t prefix = 0, mask = 0;
        int need = budget;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            constexpr int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
            for (int j = s0 + tid; j < s1; j += kRowThreads) {
                const uint32_t k = key(j);
                if ((k & mask) == prefix) atomicAdd(&hist[pass][(k >> shifts[pass]) & ((1u << bits[pass]) - 1)], 1u);
            }
            sync();
            // bins from the top down: two per thread
            const int hi = kBins - 1 - 2 * tid;
            unsigned int c0 = 0, c1 = 0;
            if (C == 1) { c0 = hist[pass][hi]; c1 = hist[pass][hi - 1]; }
            else for (int r = 0; r < C; ++r) { c0 += ld_cluster(&hist[pass][hi], r); c1 += ld_cluster(&hist[pass][hi - 1], r); }
            const int before = (int)block_scan(c0 + c1, tot, &total);
            if (before < need && before + (int)c0 >= need) { sh_prefix = prefix | ((uint32_t)hi << shifts[pass]); sh_need = need - before; }
            else if (before + (int)c0 < need && before + (int)(c0 + c1) >= need) { sh_prefix = prefix | ((uint32_t)(hi - 1) << shifts[pass]); sh_need = need - before - (int)c0; }
            __syncthreads();
            prefix = sh_prefix; need = sh_need;
            mask |= ((1u << bits[pass]) - 1) << shifts[pass];
        }
        // Ordered counts.  A thread has `per` neighbouring slots (an odd number: no bank conflicts; at most 63, so that a mask of
        // them is one register pair) of every round; slices in shared memory are one round, longer ones (one CTA) as many as it takes.
        const int per = min((s1 - s0 + kRowThreads - 1) / kRowThreads | 1, 63), rounds = (s1 - s0 + per * kRowThreads - 1) / (per * kRowThreads);
        auto before_me = [&](int which, unsigned int mine) {     // the sum of `mine` over the CTAs in front
            if (C == 1) return 0u;
            if (tid == 0) share[which] = mine;
            sync();
            unsigned int s = 0;
            for (int r = 0; r < rank; ++r) s += ld_cluster(&share[which], r);
            return s;
        };
        list_stayers();
        int ties = 0, freed = 0, moved = 0;                      // so far in this row
        // the slots of round r that are kept, ties to the lower ones; `below`: those of them under the budget
        auto kept_of = [&](int r, int &j0, unsigned long long &valid, unsigned long long &below) {
            j0 = s0 + r * per * kRowThreads + tid * per;
            const int cnt = max(0, min(per, s1 - j0)), low = max(0, min(cnt, budget - j0));
            valid = (1ull << cnt) - 1; below = (1ull << low) - 1;
            unsigned long long keep = 0, tie = 0;
            for (int i = 0; i < cnt; ++i) {
                const uint32_t k = key(j0 + i);
                keep |= (unsigned long long)(k > prefix) << i;
                tie |= (unsigned long long)(k == prefix) << i;
            }
            int t = ties + (int)block_scan((unsigned long long)__popcll(tie), tot, &total);
            const int all = (int)total;
            if (r == 0) { const int ahead = (int)before_me(0, all); t += ahead; ties += ahead; }
            ties += all;
            for (; tie && t < need; ++t) { keep |= tie & (0ull - tie); tie &= tie - 1; }
            return keep;
        };
        for (int r = 0; r < rounds; ++r) {
            int j0;
            unsigned long long valid, below;
            const unsigned long long keep = kept_of(r, j0, valid, below), gone = valid & below & ~keep, far = keep & ~below;
            const unsigned long long at = block_scan((unsigned long long)__popcll(gone) << 32 | (unsigned long long)__popcll(far), tot, &total);
            const unsigned long long all = total;
            if (r == 0) { freed += (int)before_me(1, (unsigned int)(all >> 32)); moved += (int)before_me(2, (unsigned int)all); }
            int f = freed + (int)(at >> 32), m = moved + (int)(at & 0xFFFFFFFFu);
            for (unsigned long long g = gone; g; g &= g - 1) freed_slots[f++] = j0 + __ffsll(g) - 1;
            for (unsigned long long g = far; g; g &= g - 1) movers[m++] = j0 + __ffsll(g) - 1;
            freed += (int)(all >> 32); moved += (int)(all & 0xFFFFFFFFu);
        }
        sync();                                                   // the lists are complete (global writes included); keys and weights are no longer read
        moves = freed;
        if (C > 1) { moves = 0; for (int r = 0; r < C; ++r) moves += (int)ld_cluster(&share[1], r); }
    }
    if (A.list_source)
        for (int i = rank * kRowThreads + tid; i < moves; i += C * kRowThreads) source[freed_slots[i]] = movers[i];
    if (A.move_here) {
        const int lanes = A.src.D / 4, groups = kRowThreads / lanes, lane = tid % lanes;
        const bool is_v = lane >= lanes / 2;
        const int c = (is_v ? lane - lanes / 2 : lane) * 8;
        for (int i = rank * groups + tid / lanes; i < moves; i += C * groups) {
            const int from = movers[i], slot = freed_slots[i];
            *reinterpret_cast<uint4 *>((is_v ? A.dst.v : A.dst.k) + A.dst.row(b, h, slot) + c) =
                *reinterpret_cast<const uint4 *>((is_v ? A.src.v : A.src.k) + A.src.row(b, h, from) + c);
            if (lane == 0) {                                  // in place: src is dst
                A.dst.pos[A.dst.meta(b, h) + slot] = pos[from];
                A.dst.weight[A.dst.meta(b, h) + slot] = w[from];
            }
        }
    }
    if (C > 1) si_tc::cluster_sync_all();                     // the counts of this CTA may still be read
}

// The rows of the kept entries to their slots; nothing to do for an entry that stays.  A group of D / 4 lanes per row, kMoveRows
// rows in flight per group.
template <int D>
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictArgs A) {
    constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
    // heads side by side in time: in a token-major cache they share the DRAM pages of a token
    const int b = blockIdx.z, h = blockIdx.x, row = b * A.src.H + h, lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    si_tc::pdl_wait();
    si_tc::pdl_launch();
    if (h == 0 && blockIdx.y == 0 && threadIdx.x == 0 && A.len_out) A.len_out[b] = min(entries(A, b), A.budget);
    const bool is_v = lane >= kLanes / 2;
    const int c = (is_v ? lane - kLanes / 2 : lane) * 8, slot0 = blockIdx.y * (kGroups * kMoveRows) + group;
    const uint16_t *from = (is_v ? A.src.v : A.src.k) + A.src.row(b, h, 0) + c;
    uint16_t *to = (is_v ? A.dst.v : A.dst.k) + A.dst.row(b, h, 0) + c;
    int j[kMoveRows];
#pragma unroll
    for (int k = 0; k < kMoveRows; ++k) {
        const int slot = slot0 + k * kGroups;
        j[k] = slot < A.slots ? A.source[(size_t)row * A.slots + slot] : -1;
        if (A.in_place && j[k] == slot) j[k] = -1;
    }
    // position and weight of row k: lane k, in one round of loads as well
    const int my_slot = slot0 + lane * kGroups;
    int my_j = lane < kMoveRows && my_slot < A.slots ? A.source[(size_t)row * A.slots + my_slot] : -1, my_pos = my_j;
    if (A.in_place && my_j == my_slot) my_j = -1;
    float my_weight = 0.f;
    if (my_j >= 0) {
        if (A.src.pos) my_pos = A.src.pos[A.src.meta(b, h) + my_j];
        my_weight = A.src.weight[A.src.meta(b, h) + my_j];
    }
    uint4 v[kMoveRows];
#pragma unroll
    for (int k = 0; k < kMoveRows; ++k)
        if (j[k] >= 0) v[k] = __ldcs(reinterpret_cast<const uint4 *>(from + j[k] * A.src.rs));
#pragma unroll
    for (int k = 0; k < kMoveRows; ++k)
        if (j[k] >= 0) __stcs(reinterpret_cast<uint4 *>(to + (slot0 + k * kGroups) * A.dst.rs), v[k]);
    if (my_j >= 0) {
        A.dst.pos[A.dst.meta(b, h) + my_slot] = my_pos;
        A.dst.weight[A.dst.meta(b, h) + my_slot] = my_weight;
    }
}

__global__ void evict_len_kernel(const EvictArgs A) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < A.src.B) A.len_out[b] = min(entries(A, b), A.budget);
}

size_t evict_ws_bytes(const si_kv_t *kv) {
    const size_t rows = (size_t)kv->n_seqs * kv->n_kv_heads;
    return si_align_up(rows * kv->capacity * 4, 256) + si_align_up(rows * ((size_t)kv->capacity + 2) * 4, 256);
}

// CTAs per row: more while the rows leave SMs idle and a slice stays long enough to be worth the exchanges (4096 keys), and
// as many as it takes for the slices to fit shared memory.
int cluster_size(const si_kv_t *kv) {
    const long long rows = (long long)kv->n_seqs * kv->n_kv_heads;
    int c = 1;
    while (c < kMaxCluster && rows * c * 2 <= si_sm_count() && kv->capacity / (c * 2) >= 4096) c *= 2;
    while (c < kMaxCluster && (kv->capacity + c - 1) / c > kSliceKeys) c *= 2;
    return c;
}

template <bool SMEM> int launch_select(const EvictArgs &A, int C, size_t smem, cudaStream_t st) {
    if (smem > 0) {
        static std::atomic<unsigned long long> allowed{0};
        const int rc = si_allow_smem(evict_select_kernel<SMEM>, kSliceKeys * 4, allowed);
        if (rc) return rc;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(C, A.src.H, A.src.B);
    cfg.blockDim = dim3(kRowThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = C; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = C > 1 ? 2 : 1;
    SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, evict_select_kernel<SMEM>, A));
    return SI_OK;
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
    if (budget < 1 || n_new < 0 || n_new > src->capacity || n_sink < 0 || n_recent < 0 || (long long)n_sink + n_recent > budget || budget > dst->capacity) return SI_ERR_INVALID_ARG;
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
    EvictArgs A{si_kv_view_of(src), si_kv_view_of(dst), q_pos, n_new, budget, n_sink, n_recent, in_place,
                in_place && src->capacity - budget <= kFewMoves, kept || budget < src->capacity ? budget : src->capacity, kept ? kept : (int32_t *)workspace,
                (int32_t *)((char *)workspace + si_align_up(rows * src->capacity * 4, 256)), 0, len_out, status_dev};
    A.list_source = kept || !A.move_here;
    const cudaStream_t st = (cudaStream_t)stream;
    const bool len_after = A.move_here && len_out == src->len;  // the rows of a sequence still read the old length
    if (len_after) A.len_out = nullptr;
    const int C = cluster_size(src), slice = (src->capacity + C - 1) / C;
    rc = slice <= kSliceKeys ? launch_select<true>(A, C, (size_t)slice * 4, st) : launch_select<false>(A, C, 0, st);
    if (rc) return rc;
    if (len_after) {
        A.len_out = len_out;
        evict_len_kernel<<<(src->n_seqs + 127) / 128, 128, 0, st>>>(A);
        SI_CUDA_TRY(cudaGetLastError());
    }
    if (A.move_here) return SI_OK;
    const int per_block = 256 / (src->head_dim / 4) * kMoveRows;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(src->n_kv_heads, (A.slots + per_block - 1) / per_block, src->n_seqs);
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at; cfg.numAttrs = 1;
    if (src->head_dim == 128) SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, evict_move_kernel<128>, A));
    else SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, evict_move_kernel<64>, A));
    return SI_OK;
}
