// Prefill attention: o_i = sum_j p_ij v_j, p_i = softmax over the visible entries of scale q_i . k_j, for the last T positions
// of every sequence.  One pass over the keys with the running maximum and sum of the softmax.
//
// A CTA owns two tiles of 128 query rows.  A row is a (query, head of the group) pair, so the G heads that read one key head
// share its tiles, and the span of positions in a tile -- what the causal edge and the window cost -- is 128 / G.  Warps 0-3
// and 4-7 are the softmax warpgroups of the two tiles (one row per thread), warp 8 loads tiles by TMA, warp 9 issues the
// matrix products (10 and 11 idle: registers are handed over by whole warpgroups):
//   S_t = Q_t K_j^T      (operands in shared memory, S in tensor memory)
//   O_t += P_t V_j       (P in tensor memory, written over S_t by the softmax warps; V as it lies, MN-major)
// The products of one tile run while the softmax of the other does.  O stays in tensor memory; it is rescaled only when a
// row's maximum grows by more than 2^8 (then p may reach 2^8, which fp32 sums and 16-bit p carry without loss), by the
// softmax warps themselves: S_t(j) is complete only after O_t(j-1), so nothing else touches O_t at that time.
#include "si_attn_tc.cuh"

namespace {

using namespace si_attn;

constexpr int kThreads = 384;
// Registers: 384 threads start with 168 each; the four service warps give up 96 of theirs, the softmax warps take 48 more
// (2 x 216 + 72 = 3 x 168), so that a row's 128 scores stay in registers.
constexpr int kRegsSoft = 216, kRegsService = 72;
constexpr float kLazy = 8.f;

template <int D> struct Cfg {
    static constexpr int kBytes = kTile * D * 2;            // a tile of queries, keys or values
    static constexpr int kStages = D == 128 ? 5 : 8;
    static constexpr int kSmem = (2 + kStages) * kBytes + 1024 + 256;
    static constexpr int kPanel = kTile * 128;              // 64 columns of a tile
};

struct Bars { uint64_t q, full[8], empty[8], s[2], p[2], o[2]; uint32_t tmem; int failed; };

template <int DT, int D>
__global__ void __launch_bounds__(kThreads, 1)
prefill_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
               const TcArgs A) {
    using C = Cfg<D>;
    constexpr int NS = C::kStages;
    extern __shared__ char smem_raw[];
    char *smem = (char *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    char *ring = smem + 2 * C::kBytes;
    Bars *B = (Bars *)(ring + NS * C::kBytes);
    volatile int *failed = &B->failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        mbar_init(&B->q, 1);
        for (int s = 0; s < NS; ++s) { mbar_init(&B->full[s], 1); mbar_init(&B->empty[s], 1); }
        for (int t = 0; t < 2; ++t) { mbar_init(&B->s[t], 1); mbar_init(&B->p[t], 4); mbar_init(&B->o[t], 1); }
        B->failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&B->tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = B->tmem;

    // blocks of queries from the last (most keys) to the first, so that the long ones start first
    const int heads = A.kv.H * A.kv.B, nqb = gridDim.x / heads;
    const int qb = nqb - 1 - blockIdx.x / heads, h = blockIdx.x % heads % A.kv.H, b = blockIdx.x % heads / A.kv.H;
    const int n = si_kv_len(A.kv, b, A.status), i0 = qb * 2 * A.R, shift = n - A.T;       // query i is at position shift + i
    const int tiles = i0 + A.R < A.T ? 2 : 1;
    const KeyTiles keys = key_tiles(shift + i0, shift + min(A.T, i0 + 2 * A.R) - 1, A.window, A.n_sink);

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsService));
        if (warp == 8 && lane == 0 && keys.n > 0) {
            bool ok = true;
            mbar_arrive_expect_tx(&B->q, tiles * (D / 64) * 128 * A.G * A.R);
            for (int t = 0; t < tiles; ++t)
                for (int c = 0; c < D / 64; ++c)
                    tma_load_4d(smem + t * C::kBytes + c * C::kPanel, &qmap, c * 64, h * A.G, i0 + t * A.R, b * A.q_b, &B->q);
            int it = 0;
            for (; it < 2 * keys.n; ++it) {
                const int st = it % NS;
                if (!mbar_wait(&B->empty[st], (it / NS & 1) ^ 1, kWait) || *failed) { *failed = 1; ok = false; break; }
                mbar_arrive_expect_tx(&B->full[st], C::kBytes);
                for (int c = 0; c < D / 64; ++c)
                    tma_load_4d(ring + st * C::kBytes + c * C::kPanel, it & 1 ? &vmap : &kmap, c * 64, keys.key0(it >> 1), h * A.kv_h, b * A.kv_b, &B->full[st]);
            }
            if (!ok) {                       // a wait ran out: the copies already started must land before the CTA goes
                mbar_wait(&B->q, 0, kWait);
                for (int k = max(0, it - NS); k < it; ++k) mbar_wait(&B->full[k % NS], k / NS & 1, kWait);
            }
        } else if (warp == 9 && keys.n > 0) {
            const uint32_t id_s = make_idesc(DT == SI_BF16, 0, 0, 128, 128), id_o = make_idesc(DT == SI_BF16, 0, 1, 128, D);
            // descriptors: a base per operand, steps added in its 16-byte address field
            const uint64_t q_desc = make_desc(smem_u32(smem), 16, 1024), k_desc = make_desc(smem_u32(ring), 16, 1024),
                           v_desc = make_desc(smem_u32(ring), C::kPanel, 1024);
            auto qk = [&](int t, int st) {
                if (lane == 0) {
                    const uint64_t qd = q_desc + t * (C::kBytes / 16), kd = k_desc + st * (C::kBytes / 16);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint64_t off = ((k >> 2) * C::kPanel + (k & 3) * 32) / 16;
                        umma(tmem + t * 128, qd + off, kd + off, id_s, k > 0);
                    }
                    umma_commit(&B->s[t]);
                }
            };
            auto pv = [&](int t, int st, bool acc) {
                if (lane == 0) {
                    const uint64_t vd = v_desc + st * (C::kBytes / 16);
#pragma unroll
                    for (int k = 0; k < kTile / 16; ++k) umma_ts(tmem + 256 + t * D, tmem + t * 128 + k * 8, vd + k * 128, id_o, acc || k > 0);
                }
            };
            auto all = [](bool v) { return __all_sync(0xFFFFFFFFu, v) != 0; };     // the whole warp goes on or stops
            bool ok = all(mbar_wait(&B->q, 0, kWait) && mbar_wait(&B->full[0], 0, kWait));
            if (ok) {
                tc_fence_after();
                for (int t = 0; t < tiles; ++t) qk(t, 0);
                if (lane == 0) umma_commit(&B->empty[0]);
            }
            for (int j = 0; j < keys.n && ok; ++j) {
                const int iv = 2 * j + 1, sv = iv % NS, ik = 2 * j + 2, sk = ik % NS;
                const bool more = j + 1 < keys.n;
                ok = all(mbar_wait(&B->full[sv], iv / NS & 1, kWait) && !*failed);
                if (ok && keys.key0(j) + kTile > n) {
                    // entries from n on may hold anything, and 0 * NaN is NaN: their values are cleared (16-byte pieces of whole rows)
                    const int first = n - keys.key0(j);
                    for (int i = lane; i < (kTile - first) * 8 * (D / 64); i += 32) {
                        const int c = i / ((kTile - first) * 8), at = i % ((kTile - first) * 8);
                        *reinterpret_cast<uint4 *>(ring + sv * C::kBytes + c * C::kPanel + first * 128 + at * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_proxy();
                    __syncwarp();
                }
                for (int t = 0; t < tiles && ok; ++t) {
                    ok = all(mbar_wait(&B->p[t], j & 1, kWait) && !*failed);
                    if (ok && more && t == 0) ok = all(mbar_wait(&B->full[sk], ik / NS & 1, kWait));
                    if (!ok) break;
                    tc_fence_after();
                    pv(t, sv, j > 0);
                    if (t == tiles - 1 && lane == 0) umma_commit(&B->empty[sv]);
                    if (more) qk(t, sk);
                    else if (lane == 0) umma_commit(&B->o[t]);
                }
                if (ok && more && lane == 0) umma_commit(&B->empty[sk]);
            }
            if (!ok) {
                *failed = 1;
                if (lane == 0) { umma_commit(&B->o[0]); umma_commit(&B->o[1]); }    // the products already issued end before tensor memory is freed
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoft));
        const int t = warp >> 2, row = (warp & 3) * 32 + lane;
        const int i = i0 + t * A.R + row / A.G, hq = h * A.G + row % A.G, s = shift + i, lo = max(si_window_lo(s, A.window), -1);
        const bool valid = row < A.R * A.G && i < A.T;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = tmem + lane_base + t * 128, to = tmem + lane_base + 256 + t * D;
        // what every row of the tile sees
        const int smin = shift + i0 + t * A.R, smax = shift + min(A.T, i0 + (t + 1) * A.R) - 1, lo_max = max(si_window_lo(smax, A.window), -1);
        float m = -INFINITY, base2 = 0.f, l = 0.f;
        bool ok = true;
        if (t < tiles) {
            for (int j = 0; j < keys.n; ++j) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&B->s[t], j & 1, kWait) && !*failed);
                if (!ok) break;
                tc_fence_after();
                uint32_t x[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(ts + c * 32, x[c]);
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_wait_ld(x[c]);
                const int key0 = keys.key0(j);
                if (A.sign < 0.f) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) x[c / 32][c % 32] ^= 0x80000000u;
                }
                if (!(key0 + kTile - 1 <= smin && (key0 > lo_max || key0 + kTile <= A.n_sink))) {
                    const int hi_c = s - key0, lo_c = lo - key0, sink_c = A.n_sink - key0;
#pragma unroll
                    for (int c = 0; c < 128; ++c)
                        if (!(c <= hi_c && (c > lo_c || c < sink_c))) x[c / 32][c % 32] = 0xFF800000u;
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = __uint_as_float(x[c][0]);
#pragma unroll
                    for (int k = 1; k < 32; ++k) mx[c] = fmaxf(mx[c], __uint_as_float(x[c][k]));
                }
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                const bool grow = top > m && (top - m) * A.scale2 > kLazy;
                if (__any_sync(0xFFFFFFFFu, grow)) {
                    const float m2 = grow ? top : m, b2 = m2 == -INFINITY ? 0.f : m2 * A.scale2, f = grow ? ex2(m == -INFINITY ? -INFINITY : base2 - b2) : 1.f;
                    m = m2; base2 = b2; l *= f;
                    if (j > 0) {
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t o[32];
                            tmem_ld32(to + c * 32, o);
                            tmem_wait_ld(o);
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                            tmem_st32(to + c * 32, o);
                        }
                    }
                }
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t pk[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) {
                        const int c = half * 64 + 2 * k;
                        const float p0 = ex2(fmaf(__uint_as_float(x[c / 32][c % 32]), A.scale2, -base2));
                        const float p1 = ex2(fmaf(__uint_as_float(x[c / 32][c % 32 + 1]), A.scale2, -base2));
                        sum[k & 3] += p0 + p1;
                        pk[k] = pack2<DT>(p0, p1);
                    }
                    tmem_st32(ts + half * 32, pk);
                }
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&B->p[t]);
            }
            if (!ok) *failed = 1;
            if (keys.n > 0) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&B->o[t], 0, kWait) && ok);
                tc_fence_after();
            }
            const float inv = l == 0.f ? 0.f : 1.f / l;
            const long long r = ((long long)b * A.T + i) * A.Hq + hq;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                if (keys.n > 0) { tmem_ld32(to + c * 32, o); tmem_wait_ld(o); }
                if (!valid) continue;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint4 w = make_uint4(0, 0, 0, 0);
                    if (l != 0.f) {
                        const uint32_t *v = o + k * 8;
                        w.x = pack2<DT>(__uint_as_float(v[0]) * inv, __uint_as_float(v[1]) * inv);
                        w.y = pack2<DT>(__uint_as_float(v[2]) * inv, __uint_as_float(v[3]) * inv);
                        w.z = pack2<DT>(__uint_as_float(v[4]) * inv, __uint_as_float(v[5]) * inv);
                        w.w = pack2<DT>(__uint_as_float(v[6]) * inv, __uint_as_float(v[7]) * inv);
                    }
                    *reinterpret_cast<uint4 *>(A.out + r * D + c * 32 + k * 8) = w;
                }
            }
            if (valid && A.lse) A.lse[r] = l == 0.f ? -INFINITY : (base2 + log2f(l)) / kLog2e;
        }
        if (!ok && lane == 0) si_report(A.status, SI_ERR_TIMEOUT);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <int DT, int D> int launch(const CUtensorMap &qm, const CUtensorMap &km, const CUtensorMap &vm, const TcArgs &A, cudaStream_t st) {
    static std::atomic<int> ready{0};
    if (!ready.load()) {
        SI_CUDA_TRY(cudaFuncSetAttribute(prefill_kernel<DT, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::kSmem));
        ready.store(1);
    }
    const long long blocks = (long long)((A.T + 2 * A.R - 1) / (2 * A.R)) * A.kv.H * A.kv.B;
    if (blocks > INT_MAX) return SI_ERR_TOO_LARGE;
    prefill_kernel<DT, D><<<(unsigned)blocks, kThreads, Cfg<D>::kSmem, st>>>(qm, km, vm, A);
    SI_CUDA_TRY(cudaGetLastError());
    return SI_OK;
}

}  // namespace

extern "C" int si_attn_prefill(const si_kv_t *kv, const void *q, long long q_seq_stride, long long q_tok_stride, int T,
                               int n_q_heads, int window, int n_sink, float scale, void *out, float *lse, void *workspace,
                               size_t ws_bytes, int32_t *status_dev, void *stream) {
    (void)workspace; (void)ws_bytes;
    int rc = si_attn_check(kv, n_q_heads, window, n_sink, scale);
    if (rc) return rc;
    if (T < 0) return SI_ERR_INVALID_ARG;
    if (kv->n_seqs == 0 || T == 0) return SI_OK;
    if (!q || !out || q_seq_stride < 0 || q_tok_stride < 0) return SI_ERR_INVALID_ARG;
    if (kv->pos) return SI_ERR_UNSUPPORTED;
    if (!si_aligned16(q) || !si_aligned16(out) || ((q_seq_stride | q_tok_stride) & 7)) return SI_ERR_ALIGNMENT;
    const TcArgs A = tc_args(kv, q_seq_stride, T, n_q_heads, window, n_sink, scale, out, lse, status_dev);
    CUtensorMap qm, km, vm;
    if ((rc = make_q_map(&qm, q, kv, q_seq_stride, q_tok_stride, T, n_q_heads, A.G, A.R))) return rc;
    if ((rc = make_kv_map(&km, kv->k, kv)) || (rc = make_kv_map(&vm, kv->v, kv))) return rc;
    const cudaStream_t st = (cudaStream_t)stream;
    if (kv->dtype == SI_BF16) return kv->head_dim == 128 ? launch<SI_BF16, 128>(qm, km, vm, A, st) : launch<SI_BF16, 64>(qm, km, vm, A, st);
    return kv->head_dim == 128 ? launch<SI_F16, 128>(qm, km, vm, A, st) : launch<SI_F16, 64>(qm, km, vm, A, st);
}
