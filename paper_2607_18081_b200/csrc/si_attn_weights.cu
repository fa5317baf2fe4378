// The attention every cache entry received from the last T queries:
//   weight[j] += sum_i sum_heads exp(scale q_i . k_j - lse_i)   over the queries i that see entry j.
//
// S^T = K Q^T with 128 keys as rows and 128 packed (query, head) rows as columns: a thread owns a key, so the
// sum over queries is a sum along its row of tensor memory and nothing is exchanged.  2 D flops and one exponential per
// pair; the exponential unit (16 per clock and SM: 1024 clocks per tile pair) is twice as slow as the matrix unit (512), so one
// of every eight pairs of exponentials goes to the multiply-add units (4096-token prompt: 113 us; none 117, three of eight
// 120: back to back the chip is at its power limit, and a polynomial costs more energy than it saves time).
//
// A key tile is 256 keys, two such products with the same query tile: with 128 the stream of query tiles out of L2 (32 KB per
// 1000 clocks and SM) was the bound.  Work is split in (key tile, query tile) pairs: all pairs of all sequences and heads in one row, cut into equal runs, one
// per CTA, so the triangle of a causal prompt and sequences of any lengths load all SMs alike.  A key tile whose pairs lie
// in one run is finished there; one that crosses CTAs leaves 256 partial sums per CTA, which a second kernel adds in the
// order of the CTAs -- no atomics, the same bits every time.
// All in fp32.  The caller's lse is rounded once more when it is turned to base 2, like the sum it is taken from; that and the scale
// cost 1.6e-7 of a weight.  The matrix unit cuts off its D / 16 partial sums: 1.6e-7 of a score (head size 128, f16), up to
// 1.5e-6 of a weight where the lse is exact and next to nothing where it is si_attn_prefill's, whose scores are cut off alike.
//   warps 0-15   exponentials and sums: a warpgroup per half of the keys and parity of the query tile (four warps per
//                scheduler partition cover one another's tensor-memory and exponential latencies)
//   warp 16      TMA loads of key tiles (two buffers) and query tiles (a ring)
//   warp 17      matrix products into four tensor-memory buffers
//   warp 18      the queries' lse into a ring of its own
#include <type_traits>

#include "si_attn_tc.cuh"

namespace {

using namespace si_attn;

constexpr int kGroups = 4, kThreads = kGroups * 128 + 128;
constexpr int kKeys = 2 * kTile;                     // keys of a key tile
constexpr int kBufs = 4, kLse = 4;                   // score tiles in tensor memory: [parity of the query tile][half of the keys]; ring of lse rows
constexpr int kPolyOf8 = 1;

template <int D> struct Cfg {
    static constexpr int kBytes = kTile * D * 2, kPanel = kTile * 128;
    static constexpr int kStages = D == 128 ? 2 : 4;     // ring of query tiles
    static constexpr int kSmem = (4 + kStages) * kBytes + 1024 + 512 + kLse * kTile * 4 + 2 * kKeys * 4;
};
struct Bars { uint64_t kfull[2], kempty[2], full[4], empty[4], s[kBufs], free[kBufs], lfull[kLse], lempty[kLse]; uint32_t tmem; int odd[kLse]; };

struct WeightArgs {
    const float *lse;
    float *part;        // [n_cta][2][kKeys]
    int2 *runs;         // [B][key tiles][H]: first and last CTA of a key tile
    int *part_first;    // [n_cta]: the item a CTA's run starts with
    int n_cta, nkt;     // key tiles of a full cache
};

// Query tiles that see key tile kt of a sequence with n entries: first, number.
struct Span { int first, n; };
__device__ __forceinline__ Span query_tiles(const TcArgs &A, int n, int kt) {
    const int k0 = kt * kKeys, shift = n - A.T;
    if (k0 >= n) return {0, 0};
    const int i0 = max(0, k0 - shift);
    long long i1 = A.T - 1;
    if (A.window && k0 >= A.n_sink) i1 = min(i1, (long long)min(k0 + kKeys, n) - 1 + A.window - 1 - shift);
    if (i1 < i0) return {0, 0};
    return {i0 / A.R, (int)i1 / A.R - i0 / A.R + 1};
}

// A place in the row of all pairs: item (sequence, key tile, head) with the heads of a tile side by side.
struct Cursor { int start, b, kt, h, len; Span q; };
__device__ __forceinline__ int item_of(const TcArgs &A, const WeightArgs &W, const Cursor &c) { return (c.b * W.nkt + c.kt) * A.kv.H + c.h; }
__device__ __forceinline__ void next_item(const TcArgs &A, const WeightArgs &W, Cursor &c) {     // the caller knows that there is one
    c.start += c.q.n;
    if (++c.h < A.kv.H) return;
    c.h = 0;
    do {
        if (++c.kt >= W.nkt || c.kt * kKeys >= c.len) { c.kt = 0; ++c.b; c.len = si_kv_len(A.kv, c.b, nullptr); }
        c.q = query_tiles(A, c.len, c.kt);
    } while (c.q.n == 0);
}

template <int DT, int D, bool NEG>
__global__ void __launch_bounds__(kThreads, 1)
weights_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap, const TcArgs A, const WeightArgs W) {
    using C = Cfg<D>;
    constexpr int kStages = C::kStages;
    extern __shared__ char smem_raw[];
    __shared__ int scan[kThreads / 32 + 1];
    __shared__ Cursor found;
    char *smem = (char *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    char *ring = smem + 4 * C::kBytes;
    Bars *B = (Bars *)(ring + kStages * C::kBytes);
    float *lse2 = (float *)((char *)B + 512), *other = lse2 + kLse * kTile;        // [stage][column], [exchange & 1][key]
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) { mbar_init(&B->kfull[i], 1); mbar_init(&B->kempty[i], 1); }
        for (int i = 0; i < kStages; ++i) { mbar_init(&B->full[i], 1); mbar_init(&B->empty[i], 1); }
        for (int i = 0; i < kLse; ++i) { mbar_init(&B->lfull[i], 1); mbar_init(&B->lempty[i], 8); }
        for (int i = 0; i < kBufs; ++i) { mbar_init(&B->s[i], 1); mbar_init(&B->free[i], 4); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 17) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&B->tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // rows of a query tile that no copy writes (G does not divide 128) are zero, so that their scores are numbers
    const int used = A.R * A.G;
    for (int i = tid; i < kStages * (D / 64) * (kTile - used) * 8; i += kThreads) {
        const int panel = i / ((kTile - used) * 8), at = i % ((kTile - used) * 8);
        *reinterpret_cast<uint4 *>(ring + panel * C::kPanel + used * 128 + at * 16) = make_uint4(0, 0, 0, 0);
    }
    fence_async_proxy();
    pdl_wait();                             // a programmatic dependent: up to here it ran beside the end of the kernel before it
    pdl_launch();

    // this CTA's run of pairs: thread t stands for (sequence, key tile) numbers t * per ..
    const int n_bk = A.kv.B * W.nkt, per = (n_bk + kThreads - 1) / kThreads;
    int sum = 0;
    for (int k = tid * per; k < min(n_bk, (tid + 1) * per); ++k)
        sum += query_tiles(A, si_kv_len(A.kv, k / W.nkt, blockIdx.x == 0 ? A.status : nullptr), k % W.nkt).n * A.kv.H;
    tc_fence_before();
    const int before = si_block_scan<kThreads>(sum, scan);
    tc_fence_after();
    const uint32_t tmem = B->tmem;
    const int total = scan[kThreads / 32], run = (total - 1) / W.n_cta + 1;
    const int g0 = (int)min((long long)total, (long long)blockIdx.x * run), g1 = total - g0 < run ? total : g0 + run;
    if (g0 < g1 && before <= g0 && g0 - before < sum) {      // one thread's share holds the run's first pair: it looks it up for all
        Cursor c;
        int k = tid * per, start = before;
        while (true) {
            c.b = k / W.nkt; c.kt = k % W.nkt;
            c.len = si_kv_len(A.kv, c.b, nullptr);
            c.q = query_tiles(A, c.len, c.kt);
            if (start + c.q.n * A.kv.H > g0) break;
            start += c.q.n * A.kv.H;
            ++k;
        }
        c.h = (g0 - start) / c.q.n;
        c.start = start + c.h * c.q.n;
        W.part_first[blockIdx.x] = item_of(A, W, c);
        found = c;
    }
    __syncthreads();
    Cursor cur = found;

    if (warp == 16) {
        if (elect_one()) {
            int it = 0, seg = 0;
            bool ok = true;
            for (int g = g0; g < g1 && ok; ++seg) {
                ok = mbar_wait(&B->kempty[seg & 1], (seg >> 1 & 1) ^ 1, kWait);
                if (!ok) break;
                mbar_arrive_expect_tx(&B->kfull[seg & 1], 2 * C::kBytes);
                for (int c = 0; c < 2 * (D / 64); ++c)
                    tma_load_4d(smem + (seg & 1) * 2 * C::kBytes + c * C::kPanel, &kmap, c % (D / 64) * 64, cur.kt * kKeys + c / (D / 64) * kTile, cur.h * A.kv_h, cur.b * A.kv_b, &B->kfull[seg & 1]);
                const int end = min(g1, cur.start + cur.q.n);
                for (; g < end; ++g, ++it) {
                    const int st = it % kStages;
                    ok = mbar_wait(&B->empty[st], (it / kStages & 1) ^ 1, kWait);
                    if (!ok) break;
                    mbar_arrive_expect_tx(&B->full[st], (D / 64) * 128 * used);
                    for (int c = 0; c < D / 64; ++c)
                        tma_load_4d(ring + st * C::kBytes + c * C::kPanel, &qmap, c * 64, cur.h * A.G, (cur.q.first + g - cur.start) * A.R, cur.b * A.q_b, &B->full[st]);
                }
                if (g < g1) next_item(A, W, cur);
            }
            if (!ok) {                           // a wait ran out: the copies already started must land before the CTA goes
                si_report(A.status, SI_ERR_TIMEOUT);
                for (int k = max(0, seg - 1); k <= seg; ++k) mbar_wait(&B->kfull[k & 1], k >> 1 & 1, kWait);
                for (int k = max(0, it - kStages); k < it; ++k) mbar_wait(&B->full[k % kStages], k / kStages & 1, kWait);
            }
        }
    } else if (warp == 17) {
        if (elect_one()) {
            const uint32_t id = make_idesc(DT == SI_BF16, 0, 0, 128, 128);
            const Desc q_desc = desc_of(smem_u32(ring), 16, 1024), k_desc = desc_of(smem_u32(smem), 16, 1024);
            int it = 0, seg = 0;
            bool ok = true;
            for (int g = g0; g < g1 && ok; ++seg) {
                ok = mbar_wait(&B->kfull[seg & 1], seg >> 1 & 1, kWait);
                const int end = min(g1, cur.start + cur.q.n);
                const uint32_t kb = (seg & 1) * (2 * C::kBytes / 16);
                for (; g < end && ok; ++g, ++it) {
                    const int st = it % kStages;
                    const uint32_t qb = st * (C::kBytes / 16);
                    ok = mbar_wait(&B->full[st], it / kStages & 1, kWait);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int buf = (it & 1) * 2 + half;
                        ok = ok && mbar_wait(&B->free[buf], (it >> 1 & 1) ^ 1, kWait);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint32_t off = ((k >> 2) * C::kPanel + (k & 3) * 32) / 16;
                            umma_ss(tmem + buf * kTile, k_desc, kb + half * (C::kBytes / 16) + off, q_desc, qb + off, id, k > 0);
                        }
                        umma_commit(&B->s[buf]);
                    }
                    if (ok) umma_commit(&B->empty[st]);
                }
                umma_commit(&B->kempty[seg & 1]);
                if (g < g1 && ok) next_item(A, W, cur);
            }
            if (!ok) si_report(A.status, SI_ERR_TIMEOUT);
        }
    } else if (warp == 18) {
        // lse of the 128 packed rows in base 2, negated; rows that do not exist or see nothing get -inf, so that they add
        // exp2(-inf) = 0.  Where an lse is neither a number nor -inf (a query or a key that is not a number: the scores are not
        // either), the tile says so and is left to the exponential unit, which keeps NaN.  The next tile's values are on their way while this one's place is waited for.
        int it = 0;
        bool ok = true;
        float v[4];
        auto fetch = [&](const Cursor &c, int g) {
            const int i0 = (c.q.first + g - c.start) * A.R;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = k * 32 + lane, i = i0 + r / A.G;
                v[k] = r < used && i < A.T ? W.lse[((long long)c.b * A.T + i) * A.Hq + c.h * A.G + r % A.G] : -INFINITY;
            }
        };
        if (g0 < g1) fetch(cur, g0);
        for (int g = g0; g < g1; ++g, ++it) {
            const int st = it % kLse;
            float w[4];
            bool odd = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                w[k] = v[k] == -INFINITY ? -INFINITY : -v[k] * kLog2e;
                odd |= !(v[k] < INFINITY);
            }
            odd = __any_sync(0xFFFFFFFFu, odd);
            if (g + 1 < g1) {
                if (g + 1 == cur.start + cur.q.n) next_item(A, W, cur);
                fetch(cur, g + 1);
            }
            ok = ok && mbar_wait(&B->lempty[st], (it / kLse & 1) ^ 1, kWait);
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 4; ++k) lse2[st * kTile + k * 32 + lane] = w[k];
            __syncwarp();
            if (lane == 0) { B->odd[st] = odd; mbar_arrive(&B->lfull[st]); }
        }
    } else if (warp < 16) {
        const int buf = warp >> 2, parity = buf >> 1, half = buf & 1, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const f32x2 sc = two(NEG ? -A.scale2 : A.scale2, NEG ? -A.scale2 : A.scale2);
        int it = 0, exchanges = 0;
        bool ok = true, first_segment = true;
        for (int g = g0; g < g1; ) {
            // a segment of one query tile belongs to the warpgroup of its parity alone; others are joined by the even one
            const int end = min(g1, cur.start + cur.q.n), key = cur.kt * kKeys + half * kTile + row, shift = cur.len - A.T;
            const bool single = end - g == 1, writer = single ? (it & 1) == parity : parity == 0;
            const bool whole = cur.start >= g0 && cur.start + cur.q.n <= g1;
            float *weight = A.kv.weight + A.kv.meta(cur.b, cur.h) + key;
            const float old = whole && writer && key < cur.len ? *weight : 0.f;      // needed at the end only
            float sum = 0.f, lost = 0.f;
            for (; g < end; ++g, ++it) {
                if ((it & 1) != parity) continue;
                const int st = it % kLse;
                // a wait that runs out is reported and the run goes on without waiting, to its end
                if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&B->s[buf], it >> 1 & 1, kWait) && mbar_wait(&B->lfull[st], it / kLse & 1, kWait));
                tc_fence_after();
                // column c is the query at position s0 + c / G: this key is seen by a range of columns
                const int s0 = shift + (cur.q.first + g - cur.start) * A.R;
                const bool sink = key < A.n_sink || !A.window;
                const int c_lo = min(max(key - s0, 0), kTile) * A.G, c_hi = sink ? kTile : (int)min(max((long long)key + A.window - s0, 0ll), (long long)kTile) * A.G;
                const bool open = __all_sync(0xFFFFFFFFu, c_lo == 0 && c_hi >= kTile) && !B->odd[st];
                f32x2 part[4] = {};
                auto quarter = [&](auto masked, int qq) {
                    constexpr bool MASKED = decltype(masked)::value;
                    uint32_t x[32];
                    tmem_ld32(tmem + lanes + buf * kTile + qq * 32, x);
                    tmem_wait_ld(x);
                    const float *ls = lse2 + st * kTile + qq * 32;
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        const float4 z = *reinterpret_cast<const float4 *>(ls + 2 * k);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            f32x2 p = fma2(two(x[2 * (k + e)], x[2 * (k + e) + 1]), sc, e ? two(z.z, z.w) : two(z.x, z.y));
                            float p0, p1;
                            if (!MASKED && (k + e) * kPolyOf8 % 8 < kPolyOf8) p = ex2_poly(p);
                            else {
                                untwo(p, p0, p1);
                                p0 = ex2(p0); p1 = ex2(p1);
                                if (MASKED) {
                                    const int c = qq * 32 + 2 * (k + e);
                                    if (c < c_lo || c >= c_hi) p0 = 0.f;
                                    if (c + 1 < c_lo || c + 1 >= c_hi) p1 = 0.f;
                                }
                                p = two(p0, p1);
                            }
                            part[(k + e) & 3] = add2(part[(k + e) & 3], p);
                        }
                    }
                };
                if (open) {
#pragma unroll
                    for (int qq = 0; qq < 4; ++qq) quarter(std::false_type(), qq);
                } else {
#pragma unroll
                    for (int qq = 0; qq < 4; ++qq) quarter(std::true_type(), qq);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) { mbar_arrive(&B->free[buf]); mbar_arrive(&B->lempty[st]); }
                float a, b;
                untwo(add2(add2(part[0], part[1]), add2(part[2], part[3])), a, b);
                // a long prompt's first entries collect thousands of tiles: the sum carries what its rounding lost
                const float add = (a + b) - lost, next = sum + add;
                lost = (next - sum) - add;
                sum = next;
            }
            if (!single) {
                float *xch = other + (exchanges++ & 1) * kKeys + half * kTile + row;
                if (parity) *xch = sum;
                asm volatile("bar.sync %0, 256;" ::"r"(1 + half) : "memory");
                if (!parity) sum += *xch;
            }
            if (writer) {
                if (!whole) W.part[((long long)blockIdx.x * 2 + (first_segment ? 0 : 1)) * kKeys + half * kTile + row] = sum;
                else if (key < cur.len) *weight = old + sum;
                if (half == 0 && row == 0 && cur.start >= g0) W.runs[item_of(A, W, cur)] = make_int2(cur.start / run, (cur.start + cur.q.n - 1) / run);
            }
            first_segment = false;
            if (g < g1) next_item(A, W, cur);
        }
        if (!ok && lane == 0) si_report(A.status, SI_ERR_TIMEOUT);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 17) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// Key tiles that crossed CTAs: their parts in order.
__global__ void __launch_bounds__(kKeys) weights_join_kernel(const TcArgs A, const WeightArgs W) {
    const int kt = blockIdx.x, h = blockIdx.y, b = blockIdx.z, row = threadIdx.x, key = kt * kKeys + row;
    pdl_wait();
    pdl_launch();
    const int n = si_kv_len(A.kv, b, nullptr);
    if (key >= n || query_tiles(A, n, kt).n == 0) return;
    const int item = (b * W.nkt + kt) * A.kv.H + h;
    const int2 run = W.runs[item];
    if (run.x == run.y) return;
    float sum = 0.f;
#pragma unroll 8
    for (int x = run.x; x <= run.y; ++x) sum += W.part[((long long)x * 2 + (x > run.x || W.part_first[x] == item ? 0 : 1)) * kKeys + row];
    A.kv.weight[A.kv.meta(b, h) + key] += sum;
}

struct Layout { int n_cta, nkt; size_t part, runs, first, total; };
Layout layout_of(const si_kv_t *kv) {
    Layout L;
    L.n_cta = si_sm_count();
    L.nkt = (kv->capacity + kKeys - 1) / kKeys;
    L.part = 0;
    L.runs = si_align_up((size_t)L.n_cta * 2 * kKeys * 4, 256);
    L.first = L.runs + si_align_up((size_t)kv->n_seqs * L.nkt * kv->n_kv_heads * 8, 256);
    L.total = L.first + si_align_up((size_t)L.n_cta * 4, 256);
    return L;
}

struct Call { const CUtensorMap &qm, &km; const TcArgs &A; const WeightArgs &W; cudaStream_t st; };
template <int DT, int D, bool NEG> int launch(const Call &c) {
    static std::atomic<unsigned long long> allowed{0};
    const int rc = si_allow_smem(weights_kernel<DT, D, NEG>, Cfg<D>::kSmem, allowed);
    if (rc) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at; cfg.numAttrs = 1;
    cfg.gridDim = dim3(c.W.n_cta);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Cfg<D>::kSmem;
    cfg.stream = c.st;
    SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, weights_kernel<DT, D, NEG>, c.qm, c.km, c.A, c.W));
    cfg.gridDim = dim3(c.W.nkt, c.A.kv.H, c.A.kv.B);
    cfg.blockDim = dim3(kKeys);
    cfg.dynamicSmemBytes = 0;
    SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, weights_join_kernel, c.A, c.W));
    return SI_OK;
}
template <int DT, int D> int launch_t(const Call &c, bool neg) { return neg ? launch<DT, D, true>(c) : launch<DT, D, false>(c); }

}  // namespace

size_t si_attn_weights_ws_bytes(const si_kv_t *kv) { return layout_of(kv).total; }

extern "C" int si_attn_weights(const si_kv_t *kv, const void *q, long long q_seq_stride, long long q_tok_stride, int T,
                               int n_q_heads, int window, int n_sink, float scale, const float *lse, void *workspace,
                               size_t ws_bytes, int32_t *status_dev, void *stream) {
    int rc = si_attn_check(kv, n_q_heads, window, n_sink, scale);
    if (rc) return rc;
    if (T < 0) return SI_ERR_INVALID_ARG;
    if (kv->n_seqs == 0 || T == 0) return SI_OK;
    if (!q || !lse || !kv->weight || q_seq_stride < 0 || q_tok_stride < 0) return SI_ERR_INVALID_ARG;
    if (kv->pos || (q_tok_stride == 0 && T > 1)) return SI_ERR_UNSUPPORTED;     // tensor copies have no zero stride
    if (!si_aligned16(q) || !si_aligned4(lse, status_dev) || ((q_seq_stride | q_tok_stride) & 7)) return SI_ERR_ALIGNMENT;
    const Layout L = layout_of(kv);
    const TcArgs A = tc_args(kv, q_seq_stride, T, n_q_heads, window, n_sink, scale, nullptr, nullptr, status_dev);
    // pairs are numbered in 32 bits
    if ((double)kv->n_seqs * kv->n_kv_heads * L.nkt * ((T + A.R - 1) / A.R + 1) > 2.0e9) return SI_ERR_TOO_LARGE;
    if (ws_bytes < L.total) return SI_ERR_NOMEM;
    if (!workspace) return SI_ERR_INVALID_ARG;
    if ((uintptr_t)workspace & 255) return SI_ERR_ALIGNMENT;
    char *ws = (char *)workspace;
    const WeightArgs W{lse, (float *)ws, (int2 *)(ws + L.runs), (int *)(ws + L.first), L.n_cta, L.nkt};
    CUtensorMap qm, km;
    if ((rc = make_q_map(&qm, q, kv, q_seq_stride, q_tok_stride, T, n_q_heads, A.G, A.R))) return rc;
    if ((rc = make_kv_map(&km, kv->k, kv))) return rc;
    const Call c{qm, km, A, W, (cudaStream_t)stream};
    const bool neg = scale < 0.f;
    si_mt_forget();
    if (kv->dtype == SI_BF16) return kv->head_dim == 128 ? launch_t<SI_BF16, 128>(c, neg) : launch_t<SI_BF16, 64>(c, neg);
    return kv->head_dim == 128 ? launch_t<SI_F16, 128>(c, neg) : launch_t<SI_F16, 64>(c, neg);
}
