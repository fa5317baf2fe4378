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
#include "si_evict.cuh"
#include "si_tc.cuh"

namespace {

constexpr int kRowThreads = 1024;
constexpr int kBins = 2048;
constexpr int kMaxCluster = 8;
constexpr int kSliceKeys = 48 * 1024;        // keys of a slice in shared memory; longer rows read their weights again instead,
                                             // in rounds of so many slots
constexpr int kCandidates = 2048;            // keys of the first digit's bin that are listed for the last pass
constexpr int kFewMoves = 256;               // in place with at most this many entries over the budget: one kernel
constexpr int kFewOver = 4;                  // at most this many entries over the budget are looked for one by one
constexpr int kMoveRows = 8;                 // rows in flight per warp of the moving kernel
constexpr int kMaxGridY = 65535;

__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    if (w == 0.f) w = 0.f;
    const uint32_t b = __float_as_uint(w);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// The lowest n bits.
__device__ __forceinline__ unsigned int first_bits(int n) { return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1; }

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

template <bool SMEM, bool Q4>
__global__ void __launch_bounds__(kRowThreads, 2) evict_select_kernel(const EvictArgs A) {
    extern __shared__ uint32_t keys[];
    __shared__ unsigned int hist[3][kBins], share[3];        // share: counts for the CTAs behind this one
    __shared__ uint32_t cand[kCandidates];
    __shared__ int scan[kRowThreads / 32 + 1], n_cand;
    __shared__ unsigned long long tot[32], total;
    __shared__ uint32_t sh_prefix;
    __shared__ int sh_need;
    const int C = gridDim.x, rank = blockIdx.x, tid = threadIdx.x, h = blockIdx.y, b = blockIdx.z, row = b * A.src.H + h;
    si_tc::pdl_wait();                                       // a programmatic dependent too
    const int n = si_evict_entries(A, b), budget = A.budget;
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
    const int len = ((n + C - 1) / C + 3) & ~3, s0 = min(n, rank * len), s1 = min(n, s0 + len);     // this CTA's slots
    if (SMEM) {
        if (!(((uintptr_t)w | (uintptr_t)pos) & 15)) {       // (s0 is a multiple of 4, or nothing is left)
            constexpr int U = 2;                             // 16-byte loads of a thread in flight: U weights, U positions
            for (int q = s0 + 4 * tid; q < s1; q += 4 * U * kRowThreads) {
                float4 x[U];
                int4 p[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int j = q + u * 4 * kRowThreads;
                    const bool in = j + 3 < s1;              // the last, partial group entry by entry
                    x[u] = in ? __ldg(reinterpret_cast<const float4 *>(w + j)) : make_float4(j < s1 ? w[j] : 0.f, j + 1 < s1 ? w[j + 1] : 0.f, j + 2 < s1 ? w[j + 2] : 0.f, 0.f);
                    p[u] = !pos ? make_int4(j, j + 1, j + 2, j + 3) : in ? __ldg(reinterpret_cast<const int4 *>(pos + j))
                         : make_int4(j < s1 ? pos[j] : 0, j + 1 < s1 ? pos[j + 1] : 0, j + 2 < s1 ? pos[j + 2] : 0, 0);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int j = q + u * 4 * kRowThreads;
                    if (j < s1)                              // the slice has room for whole groups
                        *reinterpret_cast<uint4 *>(keys + (j - s0)) = make_uint4(key_of(p[u].x, x[u].x), key_of(p[u].y, x[u].y), key_of(p[u].z, x[u].z), key_of(p[u].w, x[u].w));
                }
            }
        } else {
            for (int j = s0 + tid; j < s1; j += kRowThreads) keys[j - s0] = key_of(pos ? pos[j] : j, w[j]);
        }
        __syncthreads();
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
        if (tid == 0) n_cand = 0;
        __syncthreads();
        auto each_key = [&](auto f) {
            if (SMEM) {
                for (int q = 4 * tid; q < s1 - s0; q += 4 * kRowThreads) {
                    const uint4 k = *reinterpret_cast<const uint4 *>(keys + q);
                    f(k.x);
                    if (q + 1 < s1 - s0) f(k.y);
                    if (q + 2 < s1 - s0) f(k.z);
                    if (q + 3 < s1 - s0) f(k.w);
                }
            } else {
                for (int j = s0 + tid; j < s1; j += kRowThreads) f(key(j));
            }
        };
        // radix select of the budget-th largest key; the second pass lists the keys of its bin for the third
        uint32_t prefix = 0;
        int need = budget;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            if (pass == 0) each_key([&](uint32_t k) { atomicAdd(&hist[0][k >> 21], 1u); });
            else if (pass == 1)
                each_key([&](uint32_t k) {
                    if ((k >> 21) != (prefix >> 21)) return;
                    atomicAdd(&hist[1][k >> 10 & 2047], 1u);
                    const int at = atomicAdd(&n_cand, 1);
                    if (at < kCandidates) cand[at] = k;
                });
            else {
                auto last_digit = [&](uint32_t k) { if ((k >> 10) == (prefix >> 10)) atomicAdd(&hist[2][k & 1023], 1u); };
                if (n_cand <= kCandidates) for (int i = tid; i < n_cand; i += kRowThreads) last_digit(cand[i]);
                else each_key(last_digit);
            }
            sync();
            // bins from the top down: two per thread
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, hi = kBins - 1 - 2 * tid;
            int c0 = 0, c1 = 0;
            if (C == 1) { c0 = hist[pass][hi]; c1 = hist[pass][hi - 1]; }
            else for (int r = 0; r < C; ++r) { c0 += ld_cluster(&hist[pass][hi], r); c1 += ld_cluster(&hist[pass][hi - 1], r); }
            const int before = si_block_scan<kRowThreads>(c0 + c1, scan);
            if (before < need && before + c0 >= need) { sh_prefix = prefix | ((uint32_t)hi << shift); sh_need = need - before; }
            else if (before + c0 < need && before + c0 + c1 >= need) { sh_prefix = prefix | ((uint32_t)(hi - 1) << shift); sh_need = need - before - c0; }
            __syncthreads();
            prefix = sh_prefix; need = sh_need;
        }
        // Ordered counts on bit maps, a bit per slot: keys above the last kept one, keys equal to it.  Their words take the place of
        // the first two histograms (no CTA of the cluster reads those after the last exchange).  Slices in shared memory are one
        // round; longer ones, of one CTA, as many as it takes.
        unsigned int *above = hist[0], *equal = hist[1];
        auto before_me = [&](int which, unsigned int mine) {     // the sum of `mine` over the CTAs in front
            if (C == 1) return 0;
            if (tid == 0) share[which] = mine;
            sync();
            int t = 0;
            for (int r = 0; r < rank; ++r) t += (int)ld_cluster(&share[which], r);
            return t;
        };
        list_stayers();
        int ties = 0, freed = 0, moved = 0;                      // so far in this row
        for (int base = s0; base < s1 || base == s0; base += kSliceKeys) {
            const int cnt = min(kSliceKeys, s1 - base), words = (cnt + 31) / 32, share_w = words > kRowThreads ? 2 : 1;
            for (int i = tid; i < words * 32; i += kRowThreads) {
                const uint32_t k = i < cnt ? key(base + i) : 0u;
                const unsigned int a = __ballot_sync(0xFFFFFFFFu, i < cnt && k > prefix), e = __ballot_sync(0xFFFFFFFFu, i < cnt && k == prefix);
                if ((tid & 31) == 0) { above[i / 32] = a; equal[i / 32] = e; }
            }
            __syncthreads();
            const int w0 = min(words, tid * share_w), w1 = min(words, w0 + share_w);
            int mine = 0;
            for (int q = w0; q < w1; ++q) mine += __popc(equal[q]);
            int t = ties + si_block_scan<kRowThreads>(mine, scan);
            const int all_ties = scan[kRowThreads / 32];
            if (base == s0) { const int ahead = before_me(0, all_ties); t += ahead; ties += ahead; }
            ties += all_ties;
            unsigned int keep[2], low[2], in[2];                 // of this thread's words: kept slots, slots under the budget, slots
            unsigned long long counts = 0;                       // freed slots above, movers below
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                keep[u] = low[u] = in[u] = 0;
                if (w0 + u >= w1) continue;
                const int slot = base + (w0 + u) * 32;
                unsigned int e = equal[w0 + u];
                in[u] = first_bits(s1 - slot); low[u] = first_bits(budget - slot);
                keep[u] = above[w0 + u];
                for (; e && t < need; ++t) { keep[u] |= e & (0u - e); e &= e - 1; }
                t += __popc(e);                                  // the rest of the ties goes
                counts += (unsigned long long)__popc(in[u] & low[u] & ~keep[u]) << 32 | (unsigned)__popc(keep[u] & ~low[u]);
            }
            const unsigned long long at = block_scan(counts, tot, &total), all = total;
            if (base == s0) { freed += before_me(1, (unsigned int)(all >> 32)); moved += before_me(2, (unsigned int)all); }
            int f = freed + (int)(at >> 32), m = moved + (int)(at & 0xFFFFFFFFu);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int slot = base + (w0 + u) * 32;
                for (unsigned int g = in[u] & low[u] & ~keep[u]; g; g &= g - 1) freed_slots[f++] = slot + __ffs(g) - 1;
                for (unsigned int g = keep[u] & ~low[u]; g; g &= g - 1) movers[m++] = slot + __ffs(g) - 1;
            }
            freed += (int)(all >> 32); moved += (int)(all & 0xFFFFFFFFu);
            __syncthreads();                                     // the maps may be written again
        }
        sync();                                                   // the lists are complete (global writes included); keys and weights are no longer read
        moves = freed;
        if (C > 1) { moves = 0; for (int r = 0; r < C; ++r) moves += (int)ld_cluster(&share[1], r); }
    }
    if (A.list_source)
        for (int i = rank * kRowThreads + tid; i < moves; i += C * kRowThreads) source[freed_slots[i]] = movers[i];
    if (Q4 && A.move_here) {
        for (int i = rank * (kRowThreads / kMoveLanes4) + tid / kMoveLanes4; i < moves; i += C * (kRowThreads / kMoveLanes4))
            si_move_entry4(A, b, h, movers[i], freed_slots[i], tid % kMoveLanes4);
    } else if (A.move_here) {
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
template <int D, bool FIRST>
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictArgs A) {
    constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
    // heads side by side in time: in a token-major cache they share the DRAM pages of a token
    const int b = blockIdx.z, h = blockIdx.x, block = FIRST ? blockIdx.y : A.block0 + blockIdx.y, row = b * A.src.H + h, lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    si_tc::pdl_wait();
    si_tc::pdl_launch();
    if (FIRST && h == 0 && blockIdx.y == 0 && threadIdx.x == 0 && A.len_out) A.len_out[b] = min(si_evict_entries(A, b), A.budget);
    const bool is_v = lane >= kLanes / 2;
    const int c = (is_v ? lane - kLanes / 2 : lane) * 8, slot0 = block * (kGroups * kMoveRows) + group;
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
    if (b < A.src.B) A.len_out[b] = min(si_evict_entries(A, b), A.budget);
}

// CTAs per row: more while the rows leave SMs idle and a slice stays long enough to be worth the exchanges (4096 keys), and
// as many as it takes for the slices to fit shared memory.
int cluster_size(long long rows, int capacity) {
    int c = 1;
    while (c < kMaxCluster && rows * c * 2 <= si_sm_count() && capacity / (c * 2) >= 4096) c *= 2;
    while (c < kMaxCluster && (capacity + c - 1) / c + 3 > kSliceKeys) c *= 2;
    return c;
}

template <bool SMEM, bool Q4> int launch_select(const EvictArgs &A, int C, size_t smem, cudaStream_t st) {
    if (smem > 0) {
        static std::atomic<unsigned long long> allowed{0};
        const int rc = si_allow_smem(evict_select_kernel<SMEM, Q4>, kSliceKeys * 4, allowed);
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
    SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, evict_select_kernel<SMEM, Q4>, A));
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

size_t si_evict_ws_bytes(int n_seqs, int n_kv_heads, int capacity) {
    const size_t rows = (size_t)n_seqs * n_kv_heads;
    return si_align_up(rows * capacity * 4, 256) + si_align_up(rows * ((size_t)capacity + 2) * 4, 256);
}

EvictArgs si_evict_args(const si_kv_view &src, const si_kv_view &dst, bool in_place, const int32_t *q_pos, int n_new, int budget, int n_sink, int n_recent,
                        int32_t *kept, int32_t *len_out, void *workspace, int32_t *status) {
    const size_t rows = (size_t)src.B * src.H;
    EvictArgs A{src, dst, q_pos, n_new, budget, n_sink, n_recent, in_place, in_place && src.cap - budget <= kFewMoves,
                kept || budget < src.cap ? budget : src.cap, kept ? kept : (int32_t *)workspace,
                (int32_t *)((char *)workspace + si_align_up(rows * src.cap * 4, 256)), 0, len_out, status};
    A.list_source = kept || !A.move_here;
    return A;
}

int si_evict_select(EvictArgs &A, cudaStream_t st) {
    int32_t *len_out = A.len_out;
    const bool len_after = A.move_here && len_out == A.src.len;  // the rows of a sequence still read the old length
    if (len_after) A.len_out = nullptr;
    const int C = cluster_size((long long)A.src.B * A.src.H, A.src.cap), slice = ((A.src.cap + C - 1) / C + 3) & ~3;
    const size_t smem = (size_t)slice * 4;
    const bool q4 = A.src4.data != nullptr;
    int rc;
    if (slice <= kSliceKeys) rc = q4 ? launch_select<true, true>(A, C, smem, st) : launch_select<true, false>(A, C, smem, st);
    else rc = q4 ? launch_select<false, true>(A, 1, 0, st) : launch_select<false, false>(A, 1, 0, st);     // in rounds: one CTA
    if (rc || !len_after) return rc;
    A.len_out = len_out;
    evict_len_kernel<<<(A.src.B + 127) / 128, 128, 0, st>>>(A);
    SI_CUDA_TRY(cudaGetLastError());
    return SI_OK;
}

extern "C" int si_kv_workspace_bytes(const si_kv_t *kv, int n_q_heads, int T, size_t *bytes_out) {
    const int rc = si_kv_check(kv);
    if (rc) return rc;
    if (!bytes_out || n_q_heads < 0 || T < 0 || n_q_heads % kv->n_kv_heads) return SI_ERR_INVALID_ARG;
    size_t most = kv->weight ? si_evict_ws_bytes(kv->n_seqs, kv->n_kv_heads, kv->capacity) : 0;
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
    // one row's entries would be read while another's are written there
    if (si_kv_shared(dst) || (!in_place && (src->v == dst->v || src->weight == dst->weight || src->pos == dst->pos))) return SI_ERR_INVALID_ARG;
    if (!si_aligned4(q_pos, kept, len_out, status_dev)) return SI_ERR_ALIGNMENT;
    if (ws_bytes < si_evict_ws_bytes(src->n_seqs, src->n_kv_heads, src->capacity)) return SI_ERR_NOMEM;
    if (!workspace) return SI_ERR_INVALID_ARG;
    if ((uintptr_t)workspace & 255) return SI_ERR_ALIGNMENT;
    EvictArgs A = si_evict_args(si_kv_view_of(src), si_kv_view_of(dst), in_place, q_pos, n_new, budget, n_sink, n_recent, kept, len_out, workspace, status_dev);
    si_mt_forget();
    const cudaStream_t st = (cudaStream_t)stream;
    if ((rc = si_evict_select(A, st))) return rc;
    if (A.move_here) return SI_OK;
    const int per_block = 256 / (src->head_dim / 4) * kMoveRows, blocks = (int)(((long long)A.slots + per_block - 1) / per_block);
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at; cfg.numAttrs = 1;
    // One launch up to the limit of a grid's second dimension (4 million slots of head size 128), more beyond, by a version of
    // their own: the number of the first block as one more operand everywhere costs 3 % (8 x 32 heads: 221 against 215 us), block
    // and head out of one grid dimension by a division 1 %.
    for (A.block0 = 0; A.block0 < blocks; A.block0 += kMaxGridY) {
        cfg.gridDim = dim3(src->n_kv_heads, blocks - A.block0 < kMaxGridY ? blocks - A.block0 : kMaxGridY, src->n_seqs);
        if (src->head_dim == 128) SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, A.block0 ? evict_move_kernel<128, false> : evict_move_kernel<128, true>, A));
        else SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, A.block0 ? evict_move_kernel<64, false> : evict_move_kernel<64, true>, A));
    }
    return SI_OK;
}
