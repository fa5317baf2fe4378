// Single-token attention over the key/value cache in 4 bits.
//
//   out_q = sum_j p_qj (s_j c_j + m_j),  p_q = softmax over the visible entries j of scale q . (s'_j c'_j + m'_j)
//
// with a step s and a lowest value m per entry and group of channels.  Nothing is unpacked to 16-bit values: per group,
//   q . k_j = s'_j (q . c'_j) + m'_j sum(q)        out = sum_j (p_j s_j) c_j + sum_j p_j m_j,
// so that the matrix products run on the codes themselves and the steps are applied to few numbers: to the scores (keys x
// heads) and to p.  A word of eight codes becomes matrix operands by one shift and four masks: a pair of nibbles in the low bits of two
// halves is a pair of f16 numbers c 2^-24 (subnormal, which the matrix unit multiplies exactly), sixteen times that one nibble
// further up, which the other operand (q / 16) or the end (out / 16) takes back.  The layout of a tile (si_kv4.cuh) makes them
// m16n8k16 operands as they lie there.
//   - q enters as f16, scaled per head by the power of two that brings its largest element to 2^14 .. 2^15 (exact but for elements below
//     2^-31 of it).
//   - p enters as f16(p s) relative to a base 2^(m + E - 6): m the running maximum of the scores, 2^E above all steps so far.  So p s is
//     below 2^14 and the largest of all is around 2^5, far from both ends of f16: rounded to 11 bits for every type.
// Everything else is fp32.
//
// Bound by HBM: D + 8 D / group bytes per entry, key head (16 query heads).  A warp keeps kStages - 1 tiles of 32 entries in flight, one bulk
// copy each.  Work is split as for the 16-bit cache: equal runs of tiles, parts joined in order.
#include "si_attn_split.cuh"
#include "si_kv4.cuh"

namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32, kPerSm = 2, kStages = 4;

template <int D, int NG, int NT> struct Cfg {
    static constexpr int kTile = si_tile4<D, NG>::kBytes, kStage = kTile + 128;      // ... and the entries' positions; a multiple of 128
    static constexpr int kRow = D + 4, kMerge = 8 * kRow;                            // merge buffer of a warp: eight heads at a time, rows padded
    static constexpr int kSmem = kWarps * kStages * kStage + kWarps * kMerge * 4 + kWarps * 8 * NT * 2 * 4;
};

struct Decode4Args {
    DecodeArgs d;
    si_kv4_view kv;
};

__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }          // -126 .. 127
__device__ __forceinline__ int exponent(float x) { return (int)(__float_as_uint(x) >> 23 & 255) - 127; }
template <int N> __device__ __forceinline__ void load_words(uint32_t (&r)[N], const char *at) {
    if constexpr (N == 4) { const uint4 v = *reinterpret_cast<const uint4 *>(at); r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w; }
    else if constexpr (N == 2) { const uint2 v = *reinterpret_cast<const uint2 *>(at); r[0] = v.x; r[1] = v.y; }
    else r[0] = *reinterpret_cast<const uint32_t *>(at);
}

// The queries of an item.  f: B operands, per word of codes the elements (0, 1), (2, 3) / 16, (4, 5), (6, 7) / 16 of head lane / 4;
// sum: of a group's elements, times 2^-24, and back: what a score is to be multiplied with, of heads 2 (lane % 4) + {0, 1}.
template <int D, int NG, int NT> struct Query { uint32_t f[NT][D / 32][4]; float sum[NT][NG][2], back[NT][2]; };
template <int DT, int D, int NG, int NT> __device__ __forceinline__ void load_q(const DecodeArgs &A, int b, int hh, Query<D, NG, NT> &Q) {
    using T = si_tile4<D, NG>;
    const int lane = threadIdx.x & 31, t = lane & 3, h = hh / A.GB, head0 = hh % A.GB * 8 * NT, heads = min(8 * NT, A.G - head0);
    uint4 raw[NT][T::W];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int head = nt * 8 + (lane >> 2);
        const uint16_t *q = A.q + b * A.q_ss + (long long)(h * A.G + head0 + (head < heads ? head : 0)) * D + 8 * t;
#pragma unroll
        for (int w = 0; w < T::W; ++w) raw[nt][w] = head < heads ? *reinterpret_cast<const uint4 *>(q + 32 * w) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float x[T::W][8], top = 0.f;
#pragma unroll
        for (int w = 0; w < T::W; ++w) {
            const uint32_t u[4] = {raw[nt][w].x, raw[nt][w].y, raw[nt][w].z, raw[nt][w].w};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                x[w][k] = k & 1 ? si_cvt<DT>::hi(u[k / 2]) : si_cvt<DT>::lo(u[k / 2]);
                top = fmaxf(top, fabsf(x[w][k]));
            }
        }
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const int e = top == 0.f ? 0 : min(exponent(top), 117), up = 14 - e;
        const float f0 = pow2(up / 2), f1 = pow2(up - up / 2);           // 2^up may be beyond fp32
        float sum[NG] = {};
#pragma unroll
        for (int w = 0; w < T::W; ++w) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                x[w][k] = fabsf(x[w][k]) <= 3.4e38f ? x[w][k] * f0 * f1 : NAN;      // infinity times a code of zero, minus itself: NaN in any case
                sum[T::group_of(w)] += x[w][k];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) Q.f[nt][w][k] = pack2<SI_F16>(x[w][2 * k] * (k & 1 ? 0.0625f : 1.f), x[w][2 * k + 1] * (k & 1 ? 0.0625f : 1.f));
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            sum[g] += __shfl_xor_sync(0xFFFFFFFFu, sum[g], 1);
            sum[g] += __shfl_xor_sync(0xFFFFFFFFu, sum[g], 2);
#pragma unroll
            for (int c = 0; c < 2; ++c) Q.sum[nt][g][c] = 0x1p-24f * __shfl_sync(0xFFFFFFFFu, sum[g], 8 * t + 4 * c);
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) Q.back[nt][c] = pow2(__shfl_sync(0xFFFFFFFFu, e, 8 * t + 4 * c) + 10);
    }
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar, uint64_t hint) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(si_tc::smem_u32(bar)), "l"(hint) : "memory");
}

template <int DT, int D, int NG, int NT>
__global__ void __launch_bounds__(kThreads, kPerSm) decode4_kernel(const Decode4Args A4) {
    using C = Cfg<D, NG, NT>;
    using T = si_tile4<D, NG>;
    constexpr int CH = kTileEntries, HB = 8 * NT, W = T::W;
    constexpr int kLowE = DT == SI_BF16 ? -90 : -14, kHighE = DT == SI_BF16 ? 90 : 16;
    const DecodeArgs &A = A4.d;
    extern __shared__ __align__(128) char smem[];
    __shared__ int sh_scan[kThreads / 32 + 1];
    __shared__ Cursor sh_at;
    __shared__ uint64_t full[kWarps][kStages];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lg = lane >> 2, lt = lane & 3;
    char *ring = smem + warp * kStages * C::kStage;
    float *merge_o = (float *)(smem + kWarps * kStages * C::kStage);
    float *ml = merge_o + kWarps * C::kMerge;
    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < kStages; ++s) si_tc::mbar_init(&full[warp][s], 1);
        si_tc::fence_async_proxy();
    }
    si_tc::pdl_wait();                     // a programmatic dependent too: its launch runs beside the end of the kernel before it
    si_tc::pdl_launch();
    // tiles pass through L2 once; the scores stay there for the joining kernel
    uint64_t once, stay;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(once));
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(stay));

    // this CTA's run of tiles
    const Run run = find_run<CH, kThreads>(A, &sh_at, sh_scan, blockIdx.x == 0 ? A.status : nullptr);
    const int per = run.per, g0 = run.g0, g1 = run.g1;
    Cursor cons = sh_at;

    // ---- loader side: tiles g0 + warp, + kWarps, ...
    Cursor load = cons;
    int load_id = g0 + warp, load_stage = 0;
    const uint32_t ring_addr = si_tc::smem_u32(ring);
    auto issue = [&]() {
        if (load_id >= g1) return;
        while (load_id >= load.start + load.w.nc) next_item<CH>(A, load);
        if (lane == 0) {
            const int t = load_id - load.start, c = t < load.w.c_sink ? t : load.w.c_win + t - load.w.c_sink, h = load.hh / A.GB;
            uint64_t *bar = &full[warp][load_stage];
            const uint32_t to = ring_addr + load_stage * C::kStage;
            si_tc::mbar_arrive_expect_tx(bar, C::kTile + (A.kv.pos ? CH * 4 : 0));
            bulk_load(to, A4.kv.row(load.b, h) + (long long)c * C::kTile, C::kTile, bar, once);
            if (A.kv.pos) bulk_load(to + C::kTile, A.kv.pos + A.kv.meta(load.b, h) + c * CH, CH * 4, bar, once);
        }
        load_id += kWarps;
        load_stage = load_stage + 1 == kStages ? 0 : load_stage + 1;
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) issue();

    // ---- consumer side
    int id = g0 + warp, stage = 0;
    uint32_t parity = 0;
    bool first_segment = true;
    Query<D, NG, NT> Q;
    if (g0 < g1) load_q<DT, D, NG, NT>(A, cons.b, cons.hh, Q);
    // A new entry is stored by the warp that works on it.  One that its query does not see (entries without positions, and a
    // query position given that lies before the entry or a window behind it) is stored here.
    if (A.kn && A.q_pos && !A.kv.pos)
        for (int r = blockIdx.x * kWarps + warp; r < A.kv.B * A.kv.H; r += gridDim.x * kWarps) {
            const int b = r / A.kv.H, h = r % A.kv.H;
            const SeqWork w = seq_work<CH>(A, b, nullptr);
            if (w.n_old == INT_MAX || si_visible(w.n_old, w.s, w.lo, A.n_sink)) continue;
            const long long from = b * A.new_ss + (long long)h * D;
            si_q4::store_entry<DT, D, NG>(A.kn + from, A.vn + from, w.n_old % CH, (char *)A4.kv.row(b, h) + (long long)(w.n_old / CH) * C::kTile, nullptr);
        }
    // sequences without a visible entry have no tile: their rows are zero
    if (run.empty)
        for (int b = blockIdx.x; b < A.kv.B; b += gridDim.x) {
            if (seq_work<CH>(A, b, nullptr).nc) continue;
            for (int i = tid; i < A.Hq * D; i += kThreads) A.out[(long long)b * A.Hq * D + i] = 0;
            if (A.lse) for (int i = tid; i < A.Hq; i += kThreads) A.lse[(long long)b * A.Hq + i] = -INFINITY;
        }
    if (g0 >= g1) return;
    while (true) {
        const int seg_end = min(g1, cons.start + cons.w.nc);
        const int h = cons.hh / A.GB, gb = cons.hh % A.GB, head0 = gb * HB, heads = min(HB, A.G - head0);
        const SeqWork w = cons.w;
        float o[NT][W][2][4] = {}, low[NT][NG][2] = {};    // sum p s c 2^-24 of a value's elements 32 w + 4 lg + .., sum p m of this lane's entries
        float m[NT][2], base[NT][2], l[NT][2];             // base: what p is relative to, 0 while there is no maximum
        int E = -1000;
        uint32_t most = 0;                                 // 2^E in 16 bits: no step so far is above
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) { m[nt][0] = m[nt][1] = -INFINITY; base[nt][0] = base[nt][1] = l[nt][0] = l[nt][1] = 0.f; }
        for (; id < seg_end; id += kWarps) {
            if (!si_tc::mbar_wait(&full[warp][stage], parity, si_tc::kSpinLimit)) si_report(A.status, SI_ERR_TIMEOUT);
            __syncwarp();
            issue();
            char *tile = ring + stage * C::kStage;
            const int t = id - cons.start, j0 = (t < w.c_sink ? t : w.c_win + t - w.c_sink) * CH;
            // which entries are visible; the steps of the others must not meet the products (0 * NaN)
            uint32_t vis;
            {
                const int j = j0 + lane;
                int p = j;
                if (A.kv.pos) p = j == w.n_old ? w.s : *reinterpret_cast<const int *>(tile + C::kTile + lane * 4);
                vis = __ballot_sync(0xFFFFFFFFu, j < w.n && si_visible(p, w.s, w.lo, A.n_sink));
            }
            const bool fresh = w.n_old >= j0 && w.n_old - j0 < CH && (vis >> (w.n_old - j0) & 1);
            if (vis != 0xFFFFFFFFu) {
                if (!(vis >> lane & 1))
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        *reinterpret_cast<uint32_t *>(tile + T::kKeyPar + (lane * NG + g) * 4) = 0;
                        *reinterpret_cast<uint32_t *>(tile + T::kValuePar + (lane * NG + g) * 4) = 0;
                    }
                __syncwarp();
            }
            if (fresh) {                       // the new entry, into the tile here and in the cache
                const long long from = cons.b * A.new_ss + (long long)h * D;
                si_q4::store_entry<DT, D, NG>(A.kn + from, A.vn + from, w.n_old - j0, tile, gb == 0 ? (char *)A4.kv.row(cons.b, h) + (long long)(j0 / CH) * C::kTile : nullptr);
                if (gb == 0 && A.kv.pos && lane == 0) A.kv.pos[A.kv.meta(cons.b, h) + w.n_old] = w.s;
                __syncwarp();
            }
            if (vis != 0xFFFFFFFFu || fresh) si_tc::fence_async_proxy();      // the next copy into this stage comes behind these writes
            float x[2][NT][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t ka[W], kb[W], pa[NG], pb[NG];
                load_words(ka, tile + u * 8 * D + lane * T::kCell);
                load_words(kb, tile + u * 8 * D + 4 * D + lane * T::kCell);
                load_words(pa, tile + T::kKeyPar + (u * 16 + lg) * NG * 4);
                load_words(pb, tile + T::kKeyPar + (u * 16 + 8 + lg) * NG * 4);
                float acc[NT][NG][4] = {};
#pragma unroll
                for (int i = 0; i < W; ++i) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t a[4] = {si_q4::low_codes(ka[i] >> 8 * half), si_q4::low_codes(kb[i] >> 8 * half), si_q4::high_codes(ka[i] >> 8 * half), si_q4::high_codes(kb[i] >> 8 * half)};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma<SI_F16>(acc[nt][T::group_of(i)], a, Q.f[nt][i][2 * half], Q.f[nt][i][2 * half + 1]);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float y = 0.f;
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            const uint32_t par = e >> 1 ? pb[g] : pa[g];
                            y = fmaf(acc[nt][g][e], si_cvt<DT>::lo(par), fmaf(Q.sum[nt][g][e & 1], si_cvt<DT>::hi(par), y));
                        }
                        x[u][nt][e] = y * Q.back[nt][e & 1] * A.scale2;
                    }
            }
            if (vis != 0xFFFFFFFFu) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!(vis >> (u * 16 + lg + (e >> 1) * 8) & 1)) x[u][nt][e] = -INFINITY;
            }
            uint32_t vp[2][2][NG], top16 = 0;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    load_words(vp[u][r], tile + T::kValuePar + (u * 16 + r * 8 + lg) * NG * 4);
#pragma unroll
                    for (int g = 0; g < NG; ++g) top16 = __vmaxu2(top16, vp[u][r][g]);
                }
            bool grow = (top16 & 0xFFFFu) > most;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) grow |= x[u][nt][e] > m[nt][e & 1] + kLazy;
            if (A.acc) {
                float *sc = A.scores + ((((long long)cons.b * A.kv.H + h) * A.GB + gb) * A.kv.cap + j0) * A.GS;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const int key = u * 16 + lg + (e >> 1) * 8, head = nt * 8 + 2 * lt;
                            if (head < A.GS && j0 + key < w.n)
                                asm volatile("st.global.L2::cache_hint.v2.f32 [%0], {%1, %2}, %3;"
                                             ::"l"(sc + (long long)key * A.GS + head), "f"(x[u][nt][e]), "f"(x[u][nt][e + 1]), "l"(stay) : "memory");
                        }
            }
            if (__any_sync(0xFFFFFFFFu, grow)) {
                uint32_t low16 = 0;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int g = 0; g < NG; ++g) low16 = max(low16, vp[u][r][g] >> 16 & 0x7FFFu);
                const uint32_t step = __reduce_max_sync(0xFFFFFFFFu, top16 & 0xFFFFu), size = __reduce_max_sync(0xFFFFFFFFu, low16);
                // above every step, and p m stays in fp32
                E = max(E, min(max(max(exponent(si_cvt<DT>::lo(step)) + 1, exponent(si_cvt<DT>::lo(size)) - 9), kLowE), kHighE));
                most = (uint32_t)(DT == SI_BF16 ? (E + 127) << 7 : (E + 15) << 10);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float mx = m[nt][c];
#pragma unroll
                        for (int u = 0; u < 2; ++u) mx = fmaxf(mx, fmaxf(x[u][nt][c], x[u][nt][c + 2]));
                        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 16));
                        const float to = mx == -INFINITY ? 0.f : mx + (float)(E - 6), f = m[nt][c] == -INFINITY ? 1.f : ex2(base[nt][c] - to);
                        m[nt][c] = mx;
                        base[nt][c] = to;
                        l[nt][c] *= f;
#pragma unroll
                        for (int g = 0; g < NG; ++g) low[nt][g][c] *= f;
#pragma unroll
                        for (int i = 0; i < W; ++i)
#pragma unroll
                            for (int half = 0; half < 2; ++half) { o[nt][i][half][c] *= f; o[nt][i][half][c + 2] *= f; }
                    }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t va[W], vb[W], pf[NT][NG][2];
                load_words(va, tile + T::kValues + u * 8 * D + lt * D + (lg ^ T::swizzle(lt)) * T::kCell);
                load_words(vb, tile + T::kValues + u * 8 * D + 4 * D + lt * D + (lg ^ T::swizzle(lt)) * T::kCell);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[u][nt][e] = ex2(x[u][nt][e] - base[nt][e & 1]);
                        l[nt][e & 1] += x[u][nt][e];
                    }
#pragma unroll
                    for (int g = 0; g < NG; ++g)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float s = si_cvt<DT>::lo(vp[u][r][g]), mn = si_cvt<DT>::hi(vp[u][r][g]);
                            pf[nt][g][r] = mov_trans(pack2<SI_F16>(x[u][nt][2 * r] * s, x[u][nt][2 * r + 1] * s));
                            low[nt][g][0] = fmaf(x[u][nt][2 * r], mn, low[nt][g][0]);
                            low[nt][g][1] = fmaf(x[u][nt][2 * r + 1], mn, low[nt][g][1]);
                        }
                }
#pragma unroll
                for (int i = 0; i < W; ++i)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t a[4] = {si_q4::low_codes(va[i] >> 8 * half), si_q4::high_codes(va[i] >> 8 * half), si_q4::low_codes(vb[i] >> 8 * half), si_q4::high_codes(vb[i] >> 8 * half)};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma<SI_F16>(o[nt][i][half], a, pf[nt][T::group_of(i)][0], pf[nt][T::group_of(i)][1]);
                    }
            }
            __syncwarp();                      // the stage may be loaded again
            if (++stage == kStages) { stage = 0; parity ^= 1; }
        }
        const Cursor seg = cons;
        if (seg_end < g1) next_item<CH>(A, cons);
        // the CTAs of this item, for the joining kernel: written by the one that has its first tile
        if (tid == 0 && seg.start >= g0)
            A.runs[(long long)seg.b * A.kv.H * A.GB + seg.hh] = make_int2(seg.start / per | (first_segment ? 0 : kSecondSlot), (seg.start + w.nc - 1) / per);
        // ---- the segment's warps joined: rows scaled to the common base, summed in warp order
        const bool whole = seg.start >= g0 && seg.start + w.nc <= g1;
        float *po = A.part_o + ((long long)blockIdx.x * 2 + (first_segment ? 0 : 1)) * HB * D;
        float *pml = A.part_ml + ((long long)blockIdx.x * 2 + (first_segment ? 0 : 1)) * HB * 2;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float *mine = merge_o + warp * C::kMerge;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int head = 2 * lt + c;
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int s = 4; s < 32; s <<= 1) low[nt][g][c] += __shfl_xor_sync(0xFFFFFFFFu, low[nt][g][c], s);
#pragma unroll
                for (int s = 4; s < 32; s <<= 1) l[nt][c] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][c], s);
                if (lane < 4) {
                    ml[(warp * HB + nt * 8 + head) * 2] = m[nt][c] == -INFINITY ? -INFINITY : base[nt][c];
                    ml[(warp * HB + nt * 8 + head) * 2 + 1] = l[nt][c];
                }
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float mn = low[nt][T::group_of(i)][c];
                    *reinterpret_cast<float4 *>(mine + head * C::kRow + 32 * i + 4 * lg) =
                        make_float4(fmaf(o[nt][i][0][c], 0x1p24f, mn), fmaf(o[nt][i][0][c + 2], 0x1p20f, mn), fmaf(o[nt][i][1][c], 0x1p24f, mn), fmaf(o[nt][i][1][c + 2], 0x1p20f, mn));
                }
            }
            __syncthreads();
            for (int i = tid; i < 8 * (D / 2); i += kThreads) {
                const int hd = i / (D / 2), d = i % (D / 2) * 2, head = nt * 8 + hd;
                if (head >= heads) continue;
                float top = -INFINITY, sum = 0.f;
#pragma unroll
                for (int v = 0; v < kWarps; ++v) top = fmaxf(top, ml[(v * HB + head) * 2]);
                float2 acc = make_float2(0.f, 0.f);
#pragma unroll
                for (int v = 0; v < kWarps; ++v) {
                    const float mv = ml[(v * HB + head) * 2], f = mv == -INFINITY ? 1.f : ex2(mv - top);     // without a maximum: 0, or NaN (NaN scores only)
                    const float2 y = *reinterpret_cast<const float2 *>(merge_o + v * C::kMerge + hd * C::kRow + d);
                    sum += ml[(v * HB + head) * 2 + 1] * f;
                    acc.x += y.x * f; acc.y += y.y * f;
                }
                const long long row = (long long)seg.b * A.Hq + h * A.G + head0 + head;
                if (whole) {
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    *reinterpret_cast<uint32_t *>(A.out + row * D + d) = pack2<DT>(acc.x * inv, acc.y * inv);
                    if (d == 0) {
                        const float l2 = sum == 0.f ? -INFINITY : top + log2f(sum);
                        if (A.lse) A.lse[row] = l2 / kLog2e;
                        if (A.acc) A.done[row] = make_float2(top == -INFINITY ? 0.f : top, inv);
                    }
                } else {
                    *reinterpret_cast<float2 *>(po + head * D + d) = acc;
                    if (d == 0) { pml[head * 2] = top; pml[head * 2 + 1] = sum; }
                }
            }
            __syncthreads();
        }
        first_segment = false;
        if (seg_end >= g1) return;
        load_q<DT, D, NG, NT>(A, cons.b, cons.hh, Q);
    }
}

template <int DT, int D, int NG, int NT> int launch(const Decode4Args &A, cudaStream_t st) {
    static std::atomic<unsigned long long> allowed{0};
    const int rc = si_allow_smem(decode4_kernel<DT, D, NG, NT>, (Cfg<D, NG, NT>::kSmem), allowed);
    if (rc) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at; cfg.numAttrs = 1;
    cfg.gridDim = dim3(A.d.n_cta);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Cfg<D, NG, NT>::kSmem;
    cfg.stream = st;
    SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, decode4_kernel<DT, D, NG, NT>, A));
    return launch_join<DT, D, NT, kTileEntries>(A.d, st);
}
template <int DT> int launch_t(const Decode4Args &A, int NG, int NT, cudaStream_t st) {
    if (A.d.kv.D == 128) {
        if (NT == 1) return NG == 4 ? launch<DT, 128, 4, 1>(A, st) : launch<DT, 128, 2, 1>(A, st);
        return NG == 4 ? launch<DT, 128, 4, 2>(A, st) : launch<DT, 128, 2, 2>(A, st);
    }
    if (NT == 1) return NG == 2 ? launch<DT, 64, 2, 1>(A, st) : launch<DT, 64, 1, 1>(A, st);
    return NG == 2 ? launch<DT, 64, 2, 2>(A, st) : launch<DT, 64, 1, 2>(A, st);
}

Layout layout_of(const si_kv4_t *kv, int n_q_heads, bool acc) {
    return layout_of(kPerSm * si_sm_count(), kv->n_seqs, kv->n_kv_heads, kv->head_dim, kv->capacity, n_q_heads, acc);
}

}  // namespace

size_t si_kv4_attn_decode_ws_bytes(const si_kv4_t *kv, int n_q_heads) { return layout_of(kv, n_q_heads, kv->weight != nullptr).total; }

extern "C" int si_kv4_attn_decode(const si_kv4_t *kv, const void *q, long long q_seq_stride, int n_q_heads, const int32_t *q_pos,
                                  const void *k_new, const void *v_new, long long new_seq_stride, int window, int n_sink,
                                  float scale, void *out, float *lse, unsigned flags, void *workspace, size_t ws_bytes,
                                  int32_t *status_dev, void *stream) {
    int rc = si_kv4_check(kv);
    if (rc || (rc = si_query_check(kv->n_kv_heads, n_q_heads, window, n_sink, scale))) return rc;
    if (flags & ~(unsigned)SI_FLAG_ACC_WEIGHT) return SI_ERR_INVALID_ARG;
    if (kv->n_seqs == 0) return SI_OK;
    const int acc = (flags & SI_FLAG_ACC_WEIGHT) != 0;
    if (!q || !out || q_seq_stride < 0 || !k_new != !v_new || new_seq_stride < 0) return SI_ERR_INVALID_ARG;
    if ((kv->pos && !q_pos) || (acc && !kv->weight) || (k_new && si_kv4_shared(kv))) return SI_ERR_INVALID_ARG;
    if (!si_aligned16(q) || !si_aligned16(out) || !si_aligned16(k_new) || !si_aligned16(v_new) || !si_aligned4(q_pos, lse, status_dev) ||
        ((q_seq_stride | new_seq_stride) & 7))
        return SI_ERR_ALIGNMENT;
    const Layout L = layout_of(kv, n_q_heads, acc);
    // tiles are numbered in 32 bits
    if ((double)kv->n_seqs * kv->n_kv_heads * L.GB * (kv->capacity / kTileEntries + 2) > 2.0e9) return SI_ERR_TOO_LARGE;
    if (ws_bytes < L.total) return SI_ERR_NOMEM;
    if (!workspace) return SI_ERR_INVALID_ARG;
    if ((uintptr_t)workspace & 255) return SI_ERR_ALIGNMENT;
    char *ws = (char *)workspace;
    const Decode4Args A{{si_kv4_meta_of(kv), (const uint16_t *)q, (const uint16_t *)k_new, (const uint16_t *)v_new, q_pos, q_seq_stride,
                         new_seq_stride, n_q_heads, n_q_heads / kv->n_kv_heads, L.GB, L.GS, window, n_sink, scale * kLog2e,
                         (uint16_t *)out, lse, status_dev, acc, L.n_cta, (float *)(ws + L.o), (float *)(ws + L.ml),
                         (float2 *)(ws + L.done), (float *)(ws + L.scores), (int2 *)(ws + L.runs)}, si_kv4_view_of(kv)};
    si_mt_forget();
    return kv->dtype == SI_BF16 ? launch_t<SI_BF16>(A, si_kv4_groups(kv), L.NT, (cudaStream_t)stream) : launch_t<SI_F16>(A, si_kv4_groups(kv), L.NT, (cudaStream_t)stream);
}
