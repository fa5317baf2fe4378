// Prefill attention: o_i = sum_j p_ij v_j, p_i = softmax over the visible entries of scale q_i . k_j, for the last T positions
// of every sequence.  One pass over the keys with the running maximum and sum of the softmax.
//
// A CTA owns two tiles of 128 query rows.  A row is a (query, head of the group) pair, so the G heads that read one key head
// share its tiles, and the span of positions in a tile -- what the causal edge and the window cost -- is 128 / G.
//   warps 0-3, 4-7   softmax of the two tiles, a row per thread
//   warp 8           loads tiles by TMA
//   warp 9           issues the matrix products: S_t = Q_t K_j^T  (operands in shared memory, S in tensor memory)
//                                                O_t += P_t V_j   (P in tensor memory, written over S_t; V as it lies, MN-major)
//   warp 10          clears the values beyond the length in a sequence's last tile (11 idles)
// The products of one tile run while the softmax of the other does.  O stays in tensor memory; it is rescaled only when a
// row's maximum grows by more than 2^8 (then p may reach 2^8, which fp32 sums and 16-bit p carry without loss), by the
// softmax warps themselves: S_t(j) is complete only after O_t(j-1), so nothing else touches O_t at that time.
//
// Roundings below 32 bits: p goes into the product with V in the cache's type, as V has it (the matrix unit takes both operands
// alike; p in fp32 would be two or three products for one), the result is rounded once more; scores, the running maximum, the sum
// (of the unrounded p) and O are fp32.  Exponentials are the hardware's (2 ulp) of a base-2 argument.
//
// With few rows the keys are split over CTAs as well: each leaves its unnormalised O, maximum and sum, and a second kernel
// joins them in order.
#include <type_traits>

#include "si_attn_tc.cuh"

namespace {

using namespace si_attn;

constexpr int kThreads = 384;
// Registers: 384 threads start with 168 each; the four service warps give up 64 of theirs, the softmax warps take 32 more
// (2 x 200 + 104 = 3 x 168), so that a row's 128 scores stay in registers.
constexpr int kRegsSoft = 200, kRegsService = 104;
constexpr float kLazy = 8.f;
// An exponent is x * scale2 - base2 in one fused step, with base2 the rounded product of the maximum: all p of a row carry the
// same factor of 2^(what was rounded off), which cancels, and which is near 1 up to here.  Beyond, where it could reach any
// size (2^(+-4) at 2^27), the maximum is taken from the scores first.
constexpr float kFar = 65536.f;

template <int D> struct Cfg {
    static constexpr int kBytes = kTile * D * 2;            // a tile of queries, keys or values
    static constexpr int kStages = 4;                       // even ones hold keys, odd ones values
    static constexpr int kSmem = (2 + kStages) * kBytes + 1024 + 256;
    static constexpr int kPanel = kTile * 128;              // 64 columns of a tile
};

// The lowest n bits.
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1; }

struct Bars { uint64_t q, full[4], empty[4], s[2], p[2][2], o[2], dirty, clean; uint32_t tmem; int failed; };

// Keys split over P.n CTAs per block of queries (1: not split); parts: [split][block][tile][row], values and {maximum, sum}, the
// maximum unscaled.
struct SplitArgs { int n, blocks; float *o; float2 *ml; };

// NEG: the scale is negative; the scores are then turned around and |scale| is used.
template <int DT, int D, bool NEG>
__global__ void __launch_bounds__(kThreads, 1)
prefill_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
               const __grid_constant__ CUtensorMap omap, const TcArgs A, const SplitArgs P) {
    using C = Cfg<D>;
    constexpr int NS = C::kStages;
    extern __shared__ char smem_raw[];
    char *smem = (char *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    char *ring = smem + 2 * C::kBytes;
    Bars *B = (Bars *)(ring + NS * C::kBytes);
    volatile int *failed = &B->failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // blocks of queries from the last (most keys) to the first, so that the long ones start first
    const int heads = A.kv.H * A.kv.B, nqb = gridDim.x / heads;
    const int split = blockIdx.y, qb = nqb - 1 - blockIdx.x / heads, h = blockIdx.x % heads % A.kv.H, b = blockIdx.x % heads / A.kv.H;
    pdl_wait();                             // a programmatic dependent: its launch runs beside the end of the kernel before it
    const int n = si_kv_len(A.kv, b, A.status);      // on its way during the set-up

    if (threadIdx.x == 0) {
        prefetch_map(&qmap); prefetch_map(&kmap); prefetch_map(&vmap); prefetch_map(&omap);
        mbar_init(&B->q, 1);
        for (int s = 0; s < NS; ++s) { mbar_init(&B->full[s], 1); mbar_init(&B->empty[s], 1); }
        for (int t = 0; t < 2; ++t) { mbar_init(&B->s[t], 1); mbar_init(&B->p[t][0], 4); mbar_init(&B->p[t][1], 4); mbar_init(&B->o[t], 1); }
        mbar_init(&B->dirty, 1); mbar_init(&B->clean, 1);
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
    const int i0 = qb * 2 * A.R, shift = n - A.T;            // query i is at position shift + i
    const int tiles = i0 + A.R < A.T ? 2 : 1;
    KeyTiles keys = key_tiles(shift + i0, shift + min(A.T, i0 + 2 * A.R) - 1, A.window, A.n_sink);
    if (P.n > 1) {                          // the tiles of this CTA's share (far fewer than 2^31 / splits)
        keys.off = keys.n * split / P.n;
        keys.n = keys.n * (split + 1) / P.n - keys.off;
    }

    const bool tail = keys.n > 0 && keys.key0(keys.n - 1) + kTile > n;     // the last tile reaches beyond the entries in use
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
            // One elected thread issues everything, with the stages and tiles of a round of the ring unrolled: all addresses and
            // descriptors are then fixed offsets.  (The matrix unit takes a 128 x 128 x 16 product every 64 clocks and queues few
            // of them; address arithmetic between two products was 30 % of the time.)
            if (elect_one()) {
                const uint32_t id_s = make_idesc(DT == SI_BF16, 0, 0, 128, 128), id_o = make_idesc(DT == SI_BF16, 0, 1, 128, D);
                const Desc q_desc = desc_of(smem_u32(smem), 16, 1024), k_desc = desc_of(smem_u32(ring), 16, 1024),
                           v_desc = desc_of(smem_u32(ring), C::kPanel, 1024);
                auto qk = [&](int t, int st) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = ((k >> 2) * C::kPanel + (k & 3) * 32) / 16;
                        umma_ss(tmem + t * 128, q_desc, t * (C::kBytes / 16) + off, k_desc, st * (C::kBytes / 16) + off, id_s, k > 0);
                    }
                    umma_commit(&B->s[t]);
                };
                bool ok = mbar_wait(&B->q, 0, kWait) && mbar_wait(&B->full[0], 0, kWait);
                if (ok) {
                    tc_fence_after();
                    qk(0, 0);
                    if (tiles > 1) qk(1, 0);
                    umma_commit(&B->empty[0]);
                }
                constexpr int kRound = NS / 2;                // key tiles per round of the ring (keys in even stages, values in odd ones)
                for (int j0 = 0, round = 0; j0 < keys.n && ok; j0 += kRound, round ^= 1) {
#pragma unroll
                    for (int u = 0; u < kRound; ++u) {
                        const int j = j0 + u;
                        if (j >= keys.n || !ok) break;
                        const int sv = 2 * u + 1, sk = (2 * u + 2) % NS;
                        const bool more = j + 1 < keys.n;
                        ok = mbar_wait(&B->full[sv], round, kWait);
                        if (ok && more) ok = mbar_wait(&B->full[sk], u + 1 == kRound ? round ^ 1 : round, kWait);
                        if (ok && tail && !more) {            // another warp clears what lies beyond the length
                            mbar_arrive(&B->dirty);
                            ok = mbar_wait(&B->clean, 0, kWait);
                        }
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            if (t >= tiles || !ok) break;
                            ok = mbar_wait(&B->p[t][0], j & 1, kWait);       // the first half of P
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                umma_ts(tmem + 256 + t * D, tmem + t * 128 + k * 8, v_desc, sv * (C::kBytes / 16) + k * 128, id_o, j > 0 || k > 0);
                            ok = mbar_wait(&B->p[t][1], j & 1, kWait);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll
                            for (int k = 4; k < 8; ++k)
                                umma_ts(tmem + 256 + t * D, tmem + t * 128 + k * 8, v_desc, sv * (C::kBytes / 16) + k * 128, id_o, 1);
                            if (more) qk(t, sk);
                            else umma_commit(&B->o[t]);
                        }
                        if (!ok) break;
                        umma_commit(&B->empty[sv]);
                        if (more) umma_commit(&B->empty[sk]);
                    }
                }
                if (!ok) {
                    *failed = 1;
                    umma_commit(&B->o[0]);       // the products already issued end before tensor memory is freed
                    umma_commit(&B->o[1]);
                }
            }
        } else if (warp == 10 && tail) {
            // entries from n on may hold anything, and 0 * NaN is NaN: their values in the last tile are cleared
            const int iv = 2 * keys.n - 1, first = n - keys.key0(keys.n - 1);
            const bool ok = __all_sync(0xFFFFFFFFu, mbar_wait(&B->dirty, 0, kWait) && !*failed);
            if (ok) {
                for (int i = lane; i < (kTile - first) * 8 * (D / 64); i += 32) {
                    const int c = i / ((kTile - first) * 8), at = i % ((kTile - first) * 8);
                    *reinterpret_cast<uint4 *>(ring + iv % NS * C::kBytes + c * C::kPanel + first * 128 + at * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_async_proxy();
                __syncwarp();
                if (lane == 0) mbar_arrive(&B->clean);
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
            // what was rounded off m * scale2, as far as the p of the row carry it
            auto off_by = [&](float m, float base2) { return m == -INFINITY || fabsf(base2) > kFar ? 0.f : __fmaf_rn(m, A.scale2, -base2); };
            // one key tile; MASKED: some row of the tile does not see some key of it (a template argument: joining two versions of
            // a row's 128 registers after a branch costs more than the maximum).  FAR: some row's base2 may be beyond kFar; a step
            // of the near kind that comes to one leaves everything as it is and returns false, and the rest of the tiles is worked
            // on in a loop of its own (the third version inside the first loop: 3 % slower, 505 -> 521 us for 8192 tokens).
            auto step = [&](auto masked, auto farther, int j, int key0) {
                constexpr bool MASKED = decltype(masked)::value, FAR = decltype(farther)::value;
                uint32_t x[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(ts + c * 32, x[c]);
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_wait_ld(x[c]);
                if (NEG) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) x[c / 32][c % 32] ^= 0x80000000u;
                }
                if (MASKED) {
                    // the columns this row sees, a bit each; a hidden score becomes -inf by two logical operations
                    const int hi_c = s - key0, lo_c = lo - key0, sink_c = A.n_sink - key0;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint32_t seen = first_bits(hi_c + 1 - c * 32) & (~first_bits(lo_c + 1 - c * 32) | first_bits(sink_c - c * 32));
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            const uint32_t all = (uint32_t)((int)(seen << (31 - k)) >> 31);
                            x[c][k] = (x[c][k] & all) | (0xFF800000u & ~all);
                        }
                    }
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = max3(__uint_as_float(x[c][0]), __uint_as_float(x[c][1]), __uint_as_float(x[c][2]));
#pragma unroll
                    for (int k = 3; k < 31; k += 2) mx[c] = max3(mx[c], __uint_as_float(x[c][k]), __uint_as_float(x[c][k + 1]));
                    mx[c] = fmaxf(mx[c], __uint_as_float(x[c][31]));
                }
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                const bool grow = top > m && (top - m) * A.scale2 > kLazy;
                if (__any_sync(0xFFFFFFFFu, grow)) {
                    if (!FAR && __any_sync(0xFFFFFFFFu, grow && fabsf(top * A.scale2) > kFar)) return false;
                    const float m2 = grow ? top : m, b2 = m2 == -INFINITY ? 0.f : m2 * A.scale2;
                    const float f = !grow ? 1.f : m == -INFINITY ? 0.f : ex2((m - m2) * A.scale2 + (off_by(m2, b2) - off_by(m, base2)));
                    m = m2; base2 = b2; l *= f;
                    if (j > 0) {
#pragma unroll 1
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t o[16];
                            tmem_ld16(to + c * 16, o);
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                            tmem_st16(to + c * 16, o);
                        }
                    }
                }
                const bool far = FAR && fabsf(base2) > kFar;
                const f32x2 sc = two(A.scale2, A.scale2), bs = far ? two(0.f, 0.f) : two(-base2, -base2), top2 = far ? two(-m, -m) : two(0.f, 0.f);
                f32x2 sum[4] = {};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t pk[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) {
                        const int c = half * 64 + 2 * k;
                        f32x2 p = two(x[c / 32][c % 32], x[c / 32][c % 32 + 1]);
                        if (FAR) p = add2(p, top2);
                        p = fma2(p, sc, bs);
                        float p0, p1;
                        untwo(p, p0, p1);
                        p0 = ex2(p0); p1 = ex2(p1);
                        sum[k & 3] = add2(sum[k & 3], two(p0, p1));
                        pk[k] = pack2<DT>(p0, p1);
                    }
                    tmem_st32(ts + half * 32, pk);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&B->p[t][half]);
                }
                float s0, s1;
                untwo(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), s0, s1);
                l += s0 + s1;
                return true;
            };
            int j = 0;
            auto scores_of = [&](int j) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&B->s[t], j & 1, kWait));
                if (ok) tc_fence_after();
                return ok;
            };
            for (; j < keys.n && scores_of(j); ++j) {
                const int key0 = keys.key0(j);
                if (key0 + kTile - 1 <= smin && (key0 > lo_max || key0 + kTile <= A.n_sink)) { if (!step(std::false_type(), std::false_type(), j, key0)) break; }
                else if (!step(std::true_type(), std::false_type(), j, key0)) break;
            }
            if (ok && j < keys.n) {
                do step(std::true_type(), std::true_type(), j, keys.key0(j));
                while (++j < keys.n && scores_of(j));
            }
            pdl_launch();
            if (!ok) *failed = 1;
            if (keys.n > 0) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&B->o[t], 0, kWait) && ok && !*failed);
                tc_fence_after();
            }
            if (P.n > 1) {
                // parts are relative to the maximum itself
                const float c0 = ex2(-off_by(m, base2));
                const long long part = (((long long)split * P.blocks + blockIdx.x) * 2 + t) * kTile + row;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32] = {};
                    if (keys.n > 0) { tmem_ld32(to + c * 32, o); tmem_wait_ld(o); }
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        *reinterpret_cast<float4 *>(P.o + part * D + c * 32 + k) = make_float4(__uint_as_float(o[k]) * c0, __uint_as_float(o[k + 1]) * c0,
                                                                                              __uint_as_float(o[k + 2]) * c0, __uint_as_float(o[k + 3]) * c0);
                }
                P.ml[part] = make_float2(m, l * c0);
            } else {
                const float inv = l == 0.f ? 0.f : 1.f / l;
                const long long r = ((long long)b * A.T + i) * A.Hq + hq;
                // through the tile's query buffer (its last product is done), in the layout of the boxes the queries came in, and
                // out as the same boxes: rows of a thread are 2 D bytes apart, storing them directly took 4000 clocks
                char *stage = smem + t * C::kBytes + row * 128;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32] = {};
                    if (keys.n > 0) { tmem_ld32(to + c * 32, o); tmem_wait_ld(o); }
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
                        const int piece = c % 2 * 4 + k;
                        *reinterpret_cast<uint4 *>(stage + c / 2 * C::kPanel + ((piece ^ (row & 7)) << 4)) = w;
                    }
                }
                fence_async_proxy();
                asm volatile("bar.sync %0, 128;" ::"r"(1 + t) : "memory");
                if ((warp & 3) == 0 && elect_one()) {
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) tma_store_4d(&omap, smem + t * C::kBytes + c * C::kPanel, c * 64, h * A.G, i0 + t * A.R, b);
                    tma_store_wait();
                }
                if (valid && A.lse) A.lse[r] = l == 0.f ? -INFINITY : (base2 + log2f(l)) / kLog2e;
            }
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

// One warp per row: the parts of its splits, summed in order; four columns per lane, so that a warp reads 32 / (D / 4) splits at
// a time.  The values do not wait for the maxima.
constexpr int kMaxSplits = 160;
template <int DT, int D>
__global__ void __launch_bounds__(256) prefill_join_kernel(const TcArgs A, const SplitArgs P) {
    constexpr int kLanes = D / 4, kSide = 32 / kLanes, kAhead = 8;
    __shared__ float sh_f[8][kMaxSplits];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, side = lane / kLanes, col = lane % kLanes * 4;
    const long long r = (long long)blockIdx.x * 8 + warp;
    pdl_wait();
    pdl_launch();
    if (r >= (long long)A.kv.B * A.T * A.Hq) return;
    const unsigned rr = (unsigned)r;                          // rows of a split call are few
    const int hq = rr % A.Hq, i = rr / A.Hq % A.T, b = rr / A.Hq / A.T, h = hq / A.G;
    const int heads = A.kv.H * A.kv.B, nqb = P.blocks / heads, qb = i / (2 * A.R), t = i / A.R % 2;
    const long long block = (long long)(nqb - 1 - qb) * heads + b * A.kv.H + h, row = i % A.R * A.G + hq % A.G;
    const long long first = (block * 2 + t) * kTile + row, step = (long long)P.blocks * 2 * kTile;
    float4 v[kAhead];
    auto fetch = [&](int s0) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int s = s0 + k * kSide + side;
            v[k] = s < P.n ? *reinterpret_cast<const float4 *>(P.o + (first + s * step) * D + col) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    };
    fetch(0);
    float2 ml[kMaxSplits / 32];
    float top = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < kMaxSplits / 32; ++k) {
        const int s = k * 32 + lane;
        ml[k] = s < P.n ? P.ml[first + s * step] : make_float2(-INFINITY, 0.f);
        top = fmaxf(top, ml[k].x);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
#pragma unroll
    for (int k = 0; k < kMaxSplits / 32; ++k) {
        const float f = ml[k].x == -INFINITY ? 0.f : ex2((ml[k].x - top) * A.scale2);
        sh_f[warp][k * 32 + lane] = f;
        l += ml[k].y * f;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
    __syncwarp();
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < P.n; s0 += kAhead * kSide) {
        if (s0 > 0) fetch(s0);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int s = s0 + k * kSide + side;
            const float f = s < P.n ? sh_f[warp][s] : 0.f;
            if (f == 0.f) continue;                           // nothing seen in this part: its values are not used
            acc.x += v[k].x * f; acc.y += v[k].y * f; acc.z += v[k].z * f; acc.w += v[k].w * f;
        }
    }
#pragma unroll
    for (int o = kLanes; o < 32; o *= 2) {
        acc.x += __shfl_xor_sync(0xFFFFFFFFu, acc.x, o); acc.y += __shfl_xor_sync(0xFFFFFFFFu, acc.y, o);
        acc.z += __shfl_xor_sync(0xFFFFFFFFu, acc.z, o); acc.w += __shfl_xor_sync(0xFFFFFFFFu, acc.w, o);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (side == 0) *reinterpret_cast<uint2 *>(A.out + r * D + col) = make_uint2(pack2<DT>(acc.x * inv, acc.y * inv), pack2<DT>(acc.z * inv, acc.w * inv));
    if (lane == 0 && A.lse) A.lse[r] = l == 0.f ? -INFINITY : (top * A.scale2 + log2f(l)) / kLog2e;
}

// Blocks of queries, and over how many CTAs their keys are split: with fewer blocks than half the SMs as many as fit one
// wave, but no part of fewer than four key tiles (a part costs its start, 3 us, and its join).
struct Plan { long long blocks; int splits; };
int splits_of(long long blocks, long long tiles) {
    const int sms = si_sm_count();
    if (blocks * 2 > sms || tiles < 8) return 1;
    const long long n = sms / blocks < tiles / 4 ? sms / blocks : tiles / 4;
    return n < kMaxSplits ? (int)n : kMaxSplits;
}
Plan plan_of(const si_kv_t *kv, int n_q_heads, int T, int window, int n_sink) {
    const int G = n_q_heads / kv->n_kv_heads, R = kTile / G;
    Plan p{((long long)T + 2 * R - 1) / (2 * R) * kv->n_kv_heads * kv->n_seqs, 1};
    long long tiles = ((long long)kv->capacity + kTile - 1) / kTile;
    if (window) {
        const long long w = ((long long)window + 2 * R + n_sink) / kTile + 3;
        if (w < tiles) tiles = w;
    }
    p.splits = splits_of(p.blocks, tiles);
    return p;
}
size_t parts_o_bytes(const Plan &p, int D) { return p.splits > 1 ? si_align_up((size_t)p.splits * p.blocks * 2 * kTile * D * 4, 256) : 0; }
size_t parts_ml_bytes(const Plan &p) { return p.splits > 1 ? si_align_up((size_t)p.splits * p.blocks * 2 * kTile * 8, 256) : 0; }

struct Call { const CUtensorMap &qm, &km, &vm, &om; const TcArgs &A; const SplitArgs &P; cudaStream_t st; };
template <int DT, int D, bool NEG> int launch(const Call &c) {
    static std::atomic<unsigned long long> allowed{0};
    const int rc = si_allow_smem(prefill_kernel<DT, D, NEG>, Cfg<D>::kSmem, allowed);
    if (rc) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at; cfg.numAttrs = 1;
    cfg.gridDim = dim3(c.P.blocks, c.P.n);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Cfg<D>::kSmem;
    cfg.stream = c.st;
    SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, prefill_kernel<DT, D, NEG>, c.qm, c.km, c.vm, c.om, c.A, c.P));
    if (c.P.n > 1) {
        cfg.gridDim = dim3((unsigned)(((long long)c.A.kv.B * c.A.T * c.A.Hq + 7) / 8));
        cfg.blockDim = dim3(256);
        cfg.dynamicSmemBytes = 0;
        SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, prefill_join_kernel<DT, D>, c.A, c.P));
    }
    return SI_OK;
}
template <int DT, int D> int launch_t(const Call &c, bool neg) { return neg ? launch<DT, D, true>(c) : launch<DT, D, false>(c); }

}  // namespace

// For all calls with that many queries and heads or fewer: fewer rows are fewer blocks of queries, whose keys are split more
// often.  The most parts that any number of blocks leaves (a window only shortens the keys).
size_t si_attn_prefill_ws_bytes(const si_kv_t *kv, int n_q_heads, int T) {
    const long long per = (long long)kv->n_kv_heads * kv->n_seqs, tiles = ((long long)kv->capacity + kTile - 1) / kTile;
    const long long blocks = plan_of(kv, n_q_heads, T, 0, 0).blocks;
    Plan most{0, 1};
    for (long long n = per; n > 0 && n <= blocks && n * 2 <= si_sm_count(); n += per) {
        const Plan p{n, splits_of(n, tiles)};
        if (p.splits > 1 && p.blocks * p.splits > most.blocks * most.splits) most = p;
    }
    return most.splits > 1 ? parts_o_bytes(most, kv->head_dim) + parts_ml_bytes(most) : 0;
}

extern "C" int si_attn_prefill(const si_kv_t *kv, const void *q, long long q_seq_stride, long long q_tok_stride, int T,
                               int n_q_heads, int window, int n_sink, float scale, void *out, float *lse, void *workspace,
                               size_t ws_bytes, int32_t *status_dev, void *stream) {
    int rc = si_attn_check(kv, n_q_heads, window, n_sink, scale);
    if (rc) return rc;
    if (T < 0) return SI_ERR_INVALID_ARG;
    if (kv->n_seqs == 0 || T == 0) return SI_OK;
    if (!q || !out || q_seq_stride < 0 || q_tok_stride < 0) return SI_ERR_INVALID_ARG;
    if (kv->pos || (q_tok_stride == 0 && T > 1)) return SI_ERR_UNSUPPORTED;     // tensor copies have no zero stride
    if (!si_aligned16(q) || !si_aligned16(out) || !si_aligned4(lse, status_dev) || ((q_seq_stride | q_tok_stride) & 7)) return SI_ERR_ALIGNMENT;
    const Plan p = plan_of(kv, n_q_heads, T, window, n_sink);
    if (p.blocks > INT_MAX) return SI_ERR_TOO_LARGE;
    if (p.splits > 1) {
        if (ws_bytes < parts_o_bytes(p, kv->head_dim) + parts_ml_bytes(p)) return SI_ERR_NOMEM;
        if (!workspace) return SI_ERR_INVALID_ARG;
        if ((uintptr_t)workspace & 255) return SI_ERR_ALIGNMENT;
    }
    const SplitArgs P{p.splits, (int)p.blocks, (float *)workspace, (float2 *)((char *)workspace + parts_o_bytes(p, kv->head_dim))};
    const TcArgs A = tc_args(kv, q_seq_stride, T, n_q_heads, window, n_sink, scale, out, lse, status_dev);
    CUtensorMap qm, km, vm, om;
    if ((rc = make_q_map(&qm, q, kv, q_seq_stride, q_tok_stride, T, n_q_heads, A.G, A.R))) return rc;
    if ((rc = make_kv_map(&km, kv->k, kv)) || (rc = make_kv_map(&vm, kv->v, kv))) return rc;
    const long long row = (long long)n_q_heads * kv->head_dim;
    if ((rc = make_q_map(&om, out, kv, T * row, row, T, n_q_heads, A.G, A.R))) return rc;
    const Call c{qm, km, vm, om, A, P, (cudaStream_t)stream};
    const bool neg = scale < 0.f;
    si_mt_forget();
    if (kv->dtype == SI_BF16) return kv->head_dim == 128 ? launch_t<SI_BF16, 128>(c, neg) : launch_t<SI_BF16, 64>(c, neg);
    return kv->head_dim == 128 ? launch_t<SI_F16, 128>(c, neg) : launch_t<SI_F16, 64>(c, neg);
}
