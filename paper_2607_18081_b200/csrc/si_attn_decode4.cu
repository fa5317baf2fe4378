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

// Three CTAs of four warps per SM (registers allow no more; two of four: 69.8 against 63.5 us for one sequence of 260001, four of
// four with two tiles in flight: 66.8), two for sixteen heads.
#ifndef K_PER_SM
#define K_PER_SM 3
#define K_STAGES 3
#endif
constexpr int kWarps = 4, kThreads = kWarps * 32, kMergeWarps = 2;
template <int H> constexpr int kPerSmOf = H == 16 ? 2 : K_PER_SM;
template <int H> constexpr int kStagesOf = H == 16 ? 4 : K_STAGES;

// H: query heads of a pass, 4, 8 or 16.  Eight fill the eight columns of a product; 16 are two tiles of columns beside the same
// codes; with four the columns are two neighbouring groups side by side (a word of codes meets zeros in the columns of the
// other group), which halves the numbers that the steps are applied to.
template <int H> constexpr int kTilesOf = H == 16 ? 2 : 1;
template <int D, int NG, int H> struct Cfg {
    static constexpr int kTile = si_tile4<D, NG>::kBytes, kStage = kTile + 128;      // ... and the entries' positions; a multiple of 128
    static constexpr int kRow = D + 4, kMerge = 8 * kRow;                            // merge buffer of a warp: eight heads at a time, rows padded
    static constexpr int kSmem = kWarps * kStagesOf<H> * kStage + kMergeWarps * kMerge * 4 + kWarps * 8 * kTilesOf<H> * 2 * 4;
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

// The queries of an item as B operands (head lane / 4).  f: per word of codes the elements (0, 1), (2, 3) / 16, (4, 5), (6, 7) / 16.
// sum: the sums of the groups' elements, for the product with the words (step, lowest value) of the keys as they lie there: 0 beside
// the step, and beside the lowest value the sum in kParts 16-bit parts, 24 (f16: 22) bits together.  back: what a score is to be
// multiplied with, above 0 (the sign is in the others), of the lane's heads, 2 (lane % 4) + {0, 1} (H = 4: 2 (lane % 2) + {0, 1}).
template <int DT> constexpr int kParts = DT == SI_BF16 ? 3 : 2;
template <int DT> constexpr float kSumScale = DT == SI_BF16 ? 0x1p-24f : 0x1p-8f;       // f16 has no room for 2^-24
template <int DT, int NG> constexpr int kSumSteps = (kParts<DT> * NG + 7) / 8;           // products of eight words
template <int DT, int D, int NG, int H> struct Query { uint32_t f[kTilesOf<H>][D / 32][4], sum[kTilesOf<H>][kSumSteps<DT, NG>][2]; float back[kTilesOf<H>][2]; };
template <int DT, int D, int NG, int H> __device__ __forceinline__ void load_q(const DecodeArgs &A, int b, int hh, Query<DT, D, NG, H> &Q) {
    using T = si_tile4<D, NG>;
    constexpr int NT = kTilesOf<H>;
    constexpr bool PAIR = H == 4;
    const int lane = threadIdx.x & 31, t = lane & 3, h = hh / A.GB, head0 = hh % A.GB * 8 * NT, heads = min(8 * NT, A.G - head0);
    uint4 raw[NT][T::W];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int head = PAIR ? lane >> 2 & 3 : nt * 8 + (lane >> 2);
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
        const float f0 = pow2(up / 2), f1 = copysignf(pow2(up - up / 2), A.scale2);      // 2^up may be beyond fp32
        float sum[NG] = {};
#pragma unroll
        for (int w = 0; w < T::W; ++w) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                x[w][k] = fabsf(x[w][k]) <= 3.4e38f ? x[w][k] * f0 * f1 : NAN;      // infinity times a code of zero, minus itself: NaN in any case
                sum[T::group_of(w)] += x[w][k];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                Q.f[nt][w][k] = pack2<SI_F16>(x[w][2 * k] * (k & 1 ? 0.0625f : 1.f), x[w][2 * k + 1] * (k & 1 ? 0.0625f : 1.f));
                if (PAIR && (lane >> 4) != T::group_of(w) % 2) Q.f[nt][w][k] = 0;
            }
        }
        uint32_t part[kParts<DT>][NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            sum[g] += __shfl_xor_sync(0xFFFFFFFFu, sum[g], 1);
            sum[g] += __shfl_xor_sync(0xFFFFFFFFu, sum[g], 2);
            float rest = sum[g] * kSumScale<DT>;
#pragma unroll
            for (int i = 0; i < kParts<DT>; ++i) {
                part[i][g] = (uint32_t)si_cvt<DT>::from_float(rest) << 16;
                rest -= si_cvt<DT>::hi(part[i][g]);
            }
        }
        // word t (and t + 4) of a step of eight is part i / NG of group i % NG, i its number
#pragma unroll
        for (int i = 0; i < kSumSteps<DT, NG> * 8; ++i)
            if (i % 4 == 0) Q.sum[nt][i / 8][i / 4 % 2] = 0;
#pragma unroll
        for (int i = 0; i < kParts<DT> * NG; ++i)
            if (t == i % 4 && !(PAIR && lane >> 4)) Q.sum[nt][i / 8][i / 4 % 2] = part[i / NG][T::place_of(i % NG)];
#pragma unroll
        for (int c = 0; c < 2; ++c) Q.back[nt][c] = fminf(fmaxf(fabsf(A.scale2) * pow2(__shfl_sync(0xFFFFFFFFu, e, 8 * (PAIR ? t & 1 : t) + 4 * c) + 10), 1.2e-38f), 3.4e38f);
    }
}

// One product of 16 x 16 by 16 x 8.  Not volatile: the compiler may interleave those of different tiles.
template <int DT> __device__ __forceinline__ void product(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (DT == SI_BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) { uint32_t r; asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x)); return r; }

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar, uint64_t hint) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(si_tc::smem_u32(bar)), "l"(hint) : "memory");
}

template <int DT, int D, int NG, int H>
__global__ void __launch_bounds__(kThreads, kPerSmOf<H>) decode4_kernel(const Decode4Args A4) {
    using T = si_tile4<D, NG>;
    constexpr int NT = kTilesOf<H>, CH = kTileEntries, HB = 8 * NT, W = T::W;
    constexpr bool PAIR = H == 4;
    constexpr int L = PAIR ? NG / 2 : NG, GW = W / NG;      // groups of a lane (H = 4: the even or the odd ones), words of a group
    using C = Cfg<D, NG, H>;
    constexpr int kStages = kStagesOf<H>;
    constexpr int kLowE = DT == SI_BF16 ? -90 : -14, kHighE = DT == SI_BF16 ? 90 : 16;
    const DecodeArgs &A = A4.d;
    extern __shared__ __align__(128) char smem[];
    __shared__ int sh_scan[kThreads / 32 + 1];
    __shared__ Cursor sh_at;
    __shared__ uint64_t full[kWarps][kStages];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lg = lane >> 2, lt = lane & 3;
    const int head_of = PAIR ? 2 * (lt & 1) : 2 * lt, par_of = PAIR ? (lt >> 1) * L * 4 : 0;      // the lane's first head, where its groups' words are
    char *ring = smem + warp * kStages * C::kStage;
    float *merge_o = (float *)(smem + kWarps * kStages * C::kStage);
    float *ml = merge_o + kMergeWarps * C::kMerge;
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

    // ---- loader side: tiles g0 + warp, + kWarps, ..; load_left of them from load_from on lie at equal distances
    Cursor load = cons;
    int load_id = g0 + warp, load_stage = 0, load_left = 0;
    const uint8_t *load_from = nullptr;
    const int32_t *load_pos = nullptr;
    const uint32_t ring_addr = si_tc::smem_u32(ring);
    auto issue = [&]() {
        if (load_id >= g1) return;
        if (load_left == 0) {
            while (load_id >= load.start + load.w.nc) next_item<CH>(A, load);
            const int t = load_id - load.start, h = load.hh / A.GB;
            const bool sink = t < load.w.c_sink;
            const int c = sink ? t : load.w.c_win + t - load.w.c_sink;
            load_left = ((sink ? load.w.c_sink : load.w.nc) - t + kWarps - 1) / kWarps;
            load_from = A4.kv.row(load.b, h) + (long long)c * C::kTile;
            if (A.kv.pos) load_pos = A.kv.pos + A.kv.meta(load.b, h) + c * CH;
        }
        if (lane == 0) {
            uint64_t *bar = &full[warp][load_stage];
            const uint32_t to = ring_addr + load_stage * C::kStage;
            si_tc::mbar_arrive_expect_tx(bar, C::kTile + (A.kv.pos ? CH * 4 : 0));
            bulk_load(to, load_from, C::kTile, bar, once);
            if (A.kv.pos) bulk_load(to + C::kTile, load_pos, CH * 4, bar, once);
        }
        load_from += kWarps * C::kTile;
        if (A.kv.pos) load_pos += kWarps * CH;
        --load_left;
        load_id += kWarps;
        load_stage = load_stage + 1 == kStages ? 0 : load_stage + 1;
    };
#pragma unroll
    for (int s = 0; s < kStages; ++s) issue();

    // ---- consumer side
    int id = g0 + warp, stage = 0;
    uint32_t parity = 0;
    bool first_segment = true;
    Query<DT, D, NG, H> Q;
    if (g0 < g1) load_q<DT, D, NG, H>(A, cons.b, cons.hh, Q);
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
        // o: sum p s c 2^-24.  Word i: elements 4 lg + 2 n, 4 lg + 2 n + 1 (the latter times 16) in the two halves of quad 2 i + n.  H = 4: words k of
        // an even and an odd group, in the halves of four quads, one per element; those of the lane's own groups count.
        // low: sum p m of this lane's entries
        float o[NT][2 * W][4] = {}, low[NT][L][2] = {};
        // m: the maximum, raw: the same without the factor `back`, edge: the score that moves it; base: what p is relative to, 0 while there is none
        float m[NT][2], raw[NT][2], edge[NT][2], base[NT][2], l[NT][2];
        int E = -1000;
        uint32_t most = 0;                                 // 2^E in 16 bits: no step so far is above
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) { m[nt][0] = m[nt][1] = raw[nt][0] = raw[nt][1] = edge[nt][0] = edge[nt][1] = -INFINITY; base[nt][0] = base[nt][1] = l[nt][0] = l[nt][1] = 0.f; }
        // tiles whose first entry lies in all0 .. all1 are visible throughout and hold no new entry (without positions)
        const int all0 = w.lo == INT_MIN ? 0 : max(w.lo, -1) + 1, all1 = A.kv.pos ? -1 : min(min(w.n, w.n_old), w.s >= INT_MAX - 1 ? INT_MAX : w.s + 1) - CH;
        // The next tile in the ring: waits for it, clears the steps of hidden entries (they must not meet the products: 0 * NaN), puts the
        // new entry in its place.  Which entries are visible, and the number of the first.
        auto prepare = [&](int id, char *&tile, uint32_t &vis, int &j0) {
            if (!si_tc::mbar_wait(&full[warp][stage], parity, si_tc::kSpinLimit)) si_report(A.status, SI_ERR_TIMEOUT);
            tile = ring + stage * C::kStage;
            if (++stage == kStages) { stage = 0; parity ^= 1; }
            const int t = id - cons.start;
            j0 = (t < w.c_sink ? t : w.c_win + t - w.c_sink) * CH;
            vis = 0xFFFFFFFFu;
            if (j0 >= all0 && j0 <= all1) return;
            const int j = j0 + lane;
            int p = j;
            if (A.kv.pos) p = j == w.n_old ? w.s : *reinterpret_cast<const int *>(tile + C::kTile + lane * 4);
            vis = __ballot_sync(0xFFFFFFFFu, j < w.n && si_visible(p, w.s, w.lo, A.n_sink));
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
            if (fresh) {                       // into the tile here and in the cache
                const long long from = cons.b * A.new_ss + (long long)h * D;
                si_q4::store_entry<DT, D, NG>(A.kn + from, A.vn + from, w.n_old - j0, tile, gb == 0 ? (char *)A4.kv.row(cons.b, h) + (long long)(j0 / CH) * C::kTile : nullptr);
                if (gb == 0 && A.kv.pos && lane == 0) A.kv.pos[A.kv.meta(cons.b, h) + w.n_old] = w.s;
                __syncwarp();
            }
            if (vis != 0xFFFFFFFFu || fresh) si_tc::fence_async_proxy();      // the next copy into this stage comes behind these writes
        };
        // Scores of entries 16 u .. 16 u + 15 but for the factor `back`: rows lg and lg + 8, the lane's heads.
        auto scores = [&](const char *tile, int u, float (&x)[NT][4]) {
            uint32_t ka[W], kb[W], pa[L], pb[L];
            load_words(ka, tile + u * 8 * D + lane * T::kCell);
            load_words(kb, tile + u * 8 * D + 4 * D + lane * T::kCell);
            load_words(pa, tile + T::kKeyPar + (u * 16 + lg) * NG * 4 + par_of);
            load_words(pb, tile + T::kKeyPar + (u * 16 + 8 + lg) * NG * 4 + par_of);
            const uint32_t wa = *reinterpret_cast<const uint32_t *>(tile + T::kKeyPar + ((u * 16 + lg) * NG + lt % NG) * 4);
            const uint32_t wb = *reinterpret_cast<const uint32_t *>(tile + T::kKeyPar + ((u * 16 + 8 + lg) * NG + lt % NG) * 4);
            float acc[NT][L][4] = {}, sum[NT][4] = {};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < kSumSteps<DT, NG>; ++i) {
                    const uint32_t a[4] = {wa, wb, wa, wb};
                    product<DT>(sum[nt], a, Q.sum[nt][i][0], Q.sum[nt][i][1]);
                }
#pragma unroll
            for (int i = 0; i < W; ++i) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t a[4] = {si_q4::low_codes(ka[i] >> 8 * half), si_q4::low_codes(kb[i] >> 8 * half), si_q4::high_codes(ka[i] >> 8 * half), si_q4::high_codes(kb[i] >> 8 * half)};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) product<SI_F16>(acc[nt][PAIR ? T::group_of(i) / 2 : T::group_of(i)], a, Q.f[nt][i][2 * half], Q.f[nt][i][2 * half + 1]);
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float y = sum[nt][e] * (0x1p-24f / kSumScale<DT>);
#pragma unroll
                    for (int g = 0; g < L; ++g) y = fmaf(acc[nt][PAIR ? g : T::place_of(g)][e], si_cvt<DT>::lo(e >> 1 ? pb[g] : pa[g]), y);
                    x[nt][e] = PAIR ? y + __shfl_xor_sync(0xFFFFFFFFu, y, 2) : y;
                }
        };
        // p of the same entries, and their share of the sums.
        auto add = [&](const char *tile, int u, const float (&x)[NT][4], const uint32_t (&vp)[2][L]) {
            uint32_t va[W], vb[W], pf[NT][L][2];
            load_words(va, tile + T::kValues + u * 8 * D + lt * D + (lg ^ T::swizzle(lt)) * T::kCell);
            load_words(vb, tile + T::kValues + u * 8 * D + 4 * D + lt * D + (lg ^ T::swizzle(lt)) * T::kCell);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = ex2(fmaf(x[nt][e], Q.back[nt][e & 1], -base[nt][e & 1]));
                    l[nt][e & 1] += p[e];
                }
#pragma unroll
                for (int g = 0; g < L; ++g)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float s = si_cvt<DT>::lo(vp[r][g]), mn = si_cvt<DT>::hi(vp[r][g]);
                        pf[nt][g][r] = transposed(pack2<SI_F16>(p[2 * r] * s, p[2 * r + 1] * s));
                        low[nt][g][0] = fmaf(p[2 * r], mn, low[nt][g][0]);
                        low[nt][g][1] = fmaf(p[2 * r + 1], mn, low[nt][g][1]);
                    }
            }
            if constexpr (PAIR) {
#pragma unroll
                for (int i = 0; i < W / 2; ++i) {
                    const int even = i / GW * 2 * GW + i % GW, odd = even + GW;
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        auto codes = [&](uint32_t w) { return n & 1 ? si_q4::high_codes(w >> 8 * (n / 2)) : si_q4::low_codes(w >> 8 * (n / 2)); };
                        const uint32_t a[4] = {codes(va[even]), codes(va[odd]), codes(vb[even]), codes(vb[odd])};
                        product<SI_F16>(o[0][4 * i + n], a, pf[0][i / GW][0], pf[0][i / GW][1]);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < W; ++i)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t a[4] = {si_q4::low_codes(va[i] >> 8 * half), si_q4::high_codes(va[i] >> 8 * half), si_q4::low_codes(vb[i] >> 8 * half), si_q4::high_codes(vb[i] >> 8 * half)};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) product<SI_F16>(o[nt][2 * i + half], a, pf[nt][T::place_of(T::group_of(i))][0], pf[nt][T::place_of(T::group_of(i))][1]);
                    }
            }
        };
        float x[2][NT][4];
        uint32_t vp[2][2][L];
        // Hidden entries out of the scores; the scores out for the weights; steps of the values; whether the base has to move first.
        auto settle = [&](const char *tile, uint32_t vis, int j0) {
            if (vis != 0xFFFFFFFFu) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!(vis >> (u * 16 + lg + (e >> 1) * 8) & 1)) x[u][nt][e] = -INFINITY;
            }
            uint32_t top16 = 0;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    load_words(vp[u][r], tile + T::kValuePar + (u * 16 + r * 8 + lg) * NG * 4 + par_of);
#pragma unroll
                    for (int g = 0; g < L; ++g) top16 = __vmaxu2(top16, vp[u][r][g]);
                }
            bool grow = (top16 & 0xFFFFu) > most;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) grow |= x[u][nt][e] > edge[nt][e & 1];
            if (A.acc) {
                float *sc = A.scores + ((((long long)cons.b * A.kv.H + h) * A.GB + gb) * A.kv.cap + j0) * A.GS;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const int key = u * 16 + lg + (e >> 1) * 8, head = nt * 8 + head_of;
                            if (head < A.GS && j0 + key < w.n && !(PAIR && lt >> 1))
                                asm volatile("st.global.L2::cache_hint.v2.f32 [%0], {%1, %2}, %3;"
                                             ::"l"(sc + (long long)key * A.GS + head), "f"(x[u][nt][e] * Q.back[nt][0]), "f"(x[u][nt][e + 1] * Q.back[nt][1]), "l"(stay) : "memory");
                        }
            }
            if (!__any_sync(0xFFFFFFFFu, grow)) return;
            uint32_t low16 = 0;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int g = 0; g < L; ++g) low16 = max(low16, vp[u][r][g] >> 16 & 0x7FFFu);
            const uint32_t step = __reduce_max_sync(0xFFFFFFFFu, top16 & 0xFFFFu), size = __reduce_max_sync(0xFFFFFFFFu, low16);
            // above every step, and p m stays in fp32
            E = max(E, min(max(max(exponent(si_cvt<DT>::lo(step)) + 1, exponent(si_cvt<DT>::lo(size)) - 9), kLowE), kHighE));
            most = (uint32_t)(DT == SI_BF16 ? (E + 127) << 7 : (E + 15) << 10);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float mx = raw[nt][c];
#pragma unroll
                    for (int u = 0; u < 2; ++u) mx = fmaxf(mx, fmaxf(x[u][nt][c], x[u][nt][c + 2]));
                    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 4));
                    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 8));
                    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 16));
                    raw[nt][c] = mx;
                    edge[nt][c] = mx + kLazy / Q.back[nt][c];
                    mx *= Q.back[nt][c];
                    const float to = mx == -INFINITY ? 0.f : mx + (float)(E - 6), f = m[nt][c] == -INFINITY ? 1.f : ex2(base[nt][c] - to);
                    m[nt][c] = mx;
                    base[nt][c] = to;
                    l[nt][c] *= f;
#pragma unroll
                    for (int g = 0; g < L; ++g) low[nt][g][c] *= f;
#pragma unroll
                    for (int i = 0; i < 2 * W; ++i) { o[nt][i][c] *= f; o[nt][i][c + 2] *= f; }
                }
        };
        for (; id < seg_end; id += kWarps) {
            char *tile;
            uint32_t vis;
            int j0;
            prepare(id, tile, vis, j0);
            scores(tile, 0, x[0]);
            scores(tile, 1, x[1]);
            settle(tile, vis, j0);
            add(tile, 0, x[0], vp[0]);
            add(tile, 1, x[1], vp[1]);
            __syncwarp();                      // the stage may be loaded again
            issue();
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
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int s = 4; s < 32; s <<= 1) l[nt][c] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][c], s);
                if (lane < 4) *reinterpret_cast<float2 *>(ml + (warp * HB + nt * 8 + head_of + c) * 2) = make_float2(m[nt][c] == -INFINITY ? -INFINITY : base[nt][c], l[nt][c]);
            }
        __syncthreads();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float f[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float top = -INFINITY;
#pragma unroll
                for (int v = 0; v < kWarps; ++v) top = fmaxf(top, ml[(v * HB + nt * 8 + head_of + c) * 2]);
                f[c] = m[nt][c] == -INFINITY ? 1.f : ex2(base[nt][c] - top);
#pragma unroll
                for (int g = 0; g < L; ++g)
#pragma unroll
                    for (int s = 4; s < 32; s <<= 1) low[nt][g][c] += __shfl_xor_sync(0xFFFFFFFFu, low[nt][g][c], s);
            }
            float *mine = merge_o + warp % kMergeWarps * C::kMerge;
#pragma unroll
            for (int round = 0; round < kWarps; round += kMergeWarps) {
                if (warp / kMergeWarps * kMergeWarps == round)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int i = 0; i < (PAIR ? W / 2 : W); ++i) {
                            // the lane's words: all, or k of its own groups
                            const int word = PAIR ? i / GW * 2 * GW + i % GW + (lt >> 1) * GW : i;
                            const float mn = low[nt][PAIR ? i / GW : T::place_of(T::group_of(i))][c];
                            auto of = [&](int n) { return PAIR ? (lt >> 1 ? o[nt][(4 * i + n) % (2 * W)][c + 2] : o[nt][(4 * i + n) % (2 * W)][c]) : o[nt][2 * i + n / 2][c + 2 * (n & 1)]; };
                            float4 *to = reinterpret_cast<float4 *>(mine + (head_of + c) * C::kRow + 32 * word + 4 * lg);
                            float4 y = round == 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : *to;
                            y.x = fmaf(fmaf(of(0), 0x1p24f, mn), f[c], y.x);
                            y.y = fmaf(fmaf(of(1), 0x1p20f, mn), f[c], y.y);
                            y.z = fmaf(fmaf(of(2), 0x1p24f, mn), f[c], y.z);
                            y.w = fmaf(fmaf(of(3), 0x1p20f, mn), f[c], y.w);
                            *to = y;
                        }
                __syncthreads();
            }
            for (int i = tid; i < (PAIR ? 4 : 8) * (D / 2); i += kThreads) {
                const int hd = i / (D / 2), d = i % (D / 2) * 2, head = nt * 8 + hd;
                if (head >= heads) continue;
                float top = -INFINITY, sum = 0.f;
#pragma unroll
                for (int v = 0; v < kWarps; ++v) top = fmaxf(top, ml[(v * HB + head) * 2]);
#pragma unroll
                for (int v = 0; v < kWarps; ++v) {
                    const float2 y = *reinterpret_cast<const float2 *>(ml + (v * HB + head) * 2);
                    sum += y.y * (y.x == -INFINITY ? 1.f : ex2(y.x - top));     // without a maximum: 0, or NaN (NaN scores only)
                }
                float2 acc = make_float2(0.f, 0.f);
#pragma unroll
                for (int v = 0; v < kMergeWarps; ++v) {
                    const float2 y = *reinterpret_cast<const float2 *>(merge_o + v * C::kMerge + hd * C::kRow + d);
                    acc.x += y.x; acc.y += y.y;
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
        load_q<DT, D, NG, H>(A, cons.b, cons.hh, Q);
    }
}

template <int DT, int D, int NG, int H> int launch(const Decode4Args &A, cudaStream_t st) {
    using C = Cfg<D, NG, H>;
    static std::atomic<unsigned long long> allowed{0};
    const int rc = si_allow_smem(decode4_kernel<DT, D, NG, H>, C::kSmem, allowed);
    if (rc) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at; cfg.numAttrs = 1;
    cfg.gridDim = dim3(A.d.n_cta);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::kSmem;
    cfg.stream = st;
    SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, decode4_kernel<DT, D, NG, H>, A));
    return launch_join<DT, D, kTilesOf<H>, kTileEntries>(A.d, st);
}
template <int DT, int D, int NG> int launch_h(const Decode4Args &A, cudaStream_t st) {
    if (A.d.G > 8) return launch<DT, D, NG, 16>(A, st);
    if constexpr (NG > 1) if (A.d.G <= 4) return launch<DT, D, NG, 4>(A, st);
    return launch<DT, D, NG, 8>(A, st);
}
template <int DT> int launch_t(const Decode4Args &A, int NG, cudaStream_t st) {
    if (A.d.kv.D == 128) return NG == 4 ? launch_h<DT, 128, 4>(A, st) : launch_h<DT, 128, 2>(A, st);
    return NG == 2 ? launch_h<DT, 64, 2>(A, st) : launch_h<DT, 64, 1>(A, st);
}

Layout layout_of(const si_kv4_t *kv, int n_q_heads, bool acc) {
    return layout_of((n_q_heads / kv->n_kv_heads > 8 ? kPerSmOf<16> : kPerSmOf<8>) * si_sm_count(), kv->n_seqs, kv->n_kv_heads, kv->head_dim, kv->capacity, n_q_heads, acc);
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
    return kv->dtype == SI_BF16 ? launch_t<SI_BF16>(A, si_kv4_groups(kv), (cudaStream_t)stream) : launch_t<SI_F16>(A, si_kv4_groups(kv), (cudaStream_t)stream);
}
