// Single-token attention over the key/value cache in 4 bits.
//
//   out_q = sum_j p_qj (s_j c_j + m_j),  p_q = softmax over the visible entries j of scale q . (s'_j c'_j + m'_j)
//
// with a step s and a lowest value m per entry and group of channels.  Nothing is unpacked to 16-bit values: per group,
//   q . k_j = s'_j (q . c'_j) + m'_j sum(q)        out = sum_j (p_j s_j) (c_j - 8) + sum_j p_j (m_j + 8 s_j),
// so that the matrix products run on the codes themselves and the steps are applied to few numbers: to the scores (keys x
// heads) and to p.  A word of eight codes becomes matrix operands by one shift and four masks: a pair of nibbles in the low bits of two
// halves is a pair of f16 numbers c 2^-24 (subnormal, which the matrix unit multiplies exactly), sixteen times that one nibble
// further up, which the other operand (q / 16) or the end (out / 16) takes back.  The layout of a tile (si_kv4.cuh) makes them
// m16n8k16 operands as they lie there.
//   - q enters as f16, scaled per head by the power of two that brings its largest element to 2^14 .. 2^15.  Half of its elements are divided by
//     16 on top of it: exact but for elements below 2^-27 (bf16) or 2^-24 (f16) of the largest.
//   - p is 2^(score - m - 12), m the running maximum of the scores: whatever the values are, its sum and the weights do not depend
//     on them, and 2^12 below 1 it leaves room for sums of p times the largest bf16 numbers.  It enters as f16(p s up), `up` a scale per head and
//     group of channels that follows the largest p s so far and keeps it at 2^7 .. 2^15: rounded to 11 bits down to 2^-20 of that one, however
//     far apart the steps of groups, or of entries that matter and entries that do not, may be.
// Everything else is fp32.
//
// D + 8 D / group bytes per entry, key head (and 16 query heads) have to come from HBM, a third of what 16 bits take.  Neither they nor the
// issue slots bind: with some 650 instructions per tile of 32 entries and four heads (all included) half of the slots are used, a quarter of
// the matrix unit, 45 % of HBM.  Each of a scheduler's three warps waits for its own chain from shared memory through a product, the
// exponent, a pack, a transposition and a product (most stalls: fixed latencies, then loads and the busy matrix unit).  One sequence of
// 260001 entries, 32/8 heads, groups of 64: 63 us, 4.7 TB/s; 512 windows of 2052: 46 us, 3.7 TB/s; a call takes 9 us without any work (two
// kernels).  8 sequences of 15000 with two key heads: 8 query heads each 25 us (groups of 64: 22), 12 and 16 36 and 38 (groups of 64: 32).
// The scales per head and group cost 1 to 2 % of long caches, 5 % of the windows and 7 % of the step of 24 caches, whose runs of four tiles set
// them anew.
//
// A warp keeps kStages - 1 tiles in flight, one bulk copy each.  Work is cut into equal runs of tiles, one per warp, whatever the
// lengths; items that more than one run has leave parts that a second kernel joins in order: no atomics, the same bits every time.
#include "si_attn_split.cuh"
#include "si_kv4.cuh"

namespace {

// Three CTAs of four warps per SM, two for sixteen heads; three (four) tiles per warp in flight.  (Two 71 us for one sequence of 260001 entries,
// three 63, four 66, where 128 registers were too few and spilled; taken before the codes were shifted.)  168 and 255 registers are
// enough but for heads of 128 in four groups: with 5 to 8 query heads a thread spills 44 to 64 bytes, with more than 8 72 to 104, and in two
// groups with 5 to 8 8 bytes.  Every warp has a run of tiles of its own: joining the warps of a CTA at an item's end cost more than the
// additional parts do.
constexpr int kWarps = 4, kThreads = kWarps * 32;
template <int H> constexpr int kPerSmOf = H == 16 ? 2 : 3;
template <int H> constexpr int kStagesOf = H == 16 ? 4 : 3;
constexpr int kRoom = 12;              // p is at most 2^-12, but for scores that have not moved the maximum yet
constexpr float kOne = 1 << kRoom;
constexpr float kMostUp = 0x1p126f;    // scale of p s before anything was seen
constexpr int kPad = 3;                // an item's start and end take about as long as so many tiles (0: 47.7 us for 512 windows of 2052, 3: 41.7, 8: 44.4, before the codes were shifted)
// Units of a run: fewer would leave more parts than they save time (24 x 2 caches of 2049 entries and their eviction: two 28.7 us a
// step, four 27.3), but with little work the SMs come first (one cache of 1001, 8 heads: two 17.9, four 18.6).
constexpr int kFewUnits = 2, kManyUnits = 4;

// H: query heads of a pass, 4, 8 or 16.  Eight fill the eight columns of a product; 16 are two tiles of columns beside the same
// codes; with four the columns are two neighbouring groups side by side (a word of codes meets zeros in the columns of the
// other group), which halves the numbers that the steps are applied to.
template <int H> constexpr int kTilesOf = H == 16 ? 2 : 1;
template <int D, int NG, int H> struct Cfg {
    static constexpr int kTile = si_tile4<D, NG>::kBytes, kStage = kTile + 128;      // ... and the entries' positions; a multiple of 128
    static constexpr int kSmem = kWarps * kStagesOf<H> * kStage;
};

struct Decode4Args {
    DecodeArgs d;
    si_kv4_view kv;
};

// Runs: the tiles of all (sequence, head block) items in one row, in front of every item kPad units without a tile, which stand for
// the time an item's start and end take (short items are then not crowded into one run); run i of n has units total * i / n up to
// total * (i + 1) / n.  A.n_cta is the number of warps; there are fewer runs if they had less than kManyUnits.
struct Runs {
    int total, n;
    __device__ __forceinline__ int first(int i) const { return (int)((long long)total * i / n); }
    __device__ __forceinline__ int of(int unit) const { return (int)(((long long)n * (unit + 1) - 1) / total); }      // the run of a unit
};
__device__ __forceinline__ int units(const SeqWork &w) { return w.nc > 0 ? w.nc + kPad : 0; }
__device__ __forceinline__ void next_unit_item(const DecodeArgs &A, Cursor &c) {      // there is one
    c.start += units(c.w);
    if (++c.hh < A.kv.H * A.GB) return;
    c.hh = 0;
    do c.w = seq_work<kTileEntries>(A, ++c.b, nullptr); while (c.w.nc == 0);
}
// The item of the first unit of every warp's run, in `at` (where there is one).  Thread t stands for sequences t * share ..; the one
// that holds a run's first unit looks it up.
__device__ __forceinline__ Runs find_runs(const DecodeArgs &A, Cursor *at, int *sh, int32_t *status, bool *some_empty) {
    const int tid = threadIdx.x, share = (A.kv.B + kThreads - 1) / kThreads, items = A.kv.H * A.GB;
    const int b0 = min(A.kv.B, tid * share), b1 = min(A.kv.B, b0 + share);
    int sum = 0;
    bool empty = false;
    SeqWork w;
    for (int b = b0; b < b1; ++b) {
        w = seq_work<kTileEntries>(A, b, status);
        sum += units(w) * items;
        empty |= w.nc == 0;
    }
    const int before = si_block_scan<kThreads>(sum, sh);
    const int total = sh[kThreads / 32];
    const Runs r{total, min(A.n_cta, max((total + kManyUnits - 1) / kManyUnits, min((total + kFewUnits - 1) / kFewUnits, (int)gridDim.x)))};
    if (r.total > 0)
        for (int i = 0; i < kWarps; ++i) {
            const int run = i * gridDim.x + blockIdx.x;
            if (run >= r.n) break;
            const int g0 = r.first(run);
            if (before > g0 || g0 - before >= sum) continue;
            Cursor c;
            int start = before;
            c.b = b0;
            c.w = share > 1 ? seq_work<kTileEntries>(A, b0, nullptr) : w;      // with one sequence per thread it is at hand
            while (start + units(c.w) * items <= g0) { start += units(c.w) * items; c.w = seq_work<kTileEntries>(A, ++c.b, nullptr); }
            c.hh = (g0 - start) / units(c.w);
            c.start = start + c.hh * units(c.w);
            at[i] = c;
        }
    *some_empty = __syncthreads_or(empty);
    return r;
}

__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }          // -126 .. 127
__device__ __forceinline__ int exponent(float x) { return (int)(__float_as_uint(x) >> 23 & 255) - 127; }
template <int N> __device__ __forceinline__ void load_words(uint32_t (&r)[N], const char *at) {
    if constexpr (N == 4) { const uint4 v = *reinterpret_cast<const uint4 *>(at); r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w; }
    else if constexpr (N == 2) { const uint2 v = *reinterpret_cast<const uint2 *>(at); r[0] = v.x; r[1] = v.y; }
    else r[0] = *reinterpret_cast<const uint32_t *>(at);
}

// The queries of an item as B operands (head lane / 4).  f: per word of codes the elements (0, 1), (2, 3) / 16, (4, 5), (6, 7) / 16.
// sum: the sums of the groups' elements, for the product with the words (lowest value, step) of the keys as they lie there: 0 beside
// the step, and beside the lowest value the sum in kParts 16-bit parts, 24 (f16: 22) bits together.  Lane t of four has in its two
// registers the groups whose words lie at kOwn (t / 2) and kOwn (t / 2) + 1 (one register's only where kOwn is 1), and part t % 2 of
// them; the third part takes a product of its own, or the other register.
// back: what a score is to be multiplied with, above 0 (the sign is in the others), and lazy: how far one may be above the
// maximum, of the lane's heads, 2 (lane % 4) + {0, 1} (H = 4: 2 (lane % 2) + {0, 1}).
template <int DT> constexpr int kParts = DT == SI_BF16 ? 3 : 2;
template <int DT> constexpr float kSumScale = DT == SI_BF16 ? 0x1p-24f : 0x1p-8f;       // f16 has no room for 2^-24
template <int DT, int NG> constexpr int kSumSteps = NG == 4 ? kParts<DT> - 1 : 1;
template <int NG> constexpr int kOwn = NG == 4 ? 2 : 1;
template <int DT, int D, int NG, int H> struct Query { uint32_t f[kTilesOf<H>][D / 32][4], sum[kTilesOf<H>][kSumSteps<DT, NG>][2]; float back[kTilesOf<H>][2], lazy[kTilesOf<H>][2]; };
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
        const int e = exponent(top), up = 14 - e;
        auto back = [&](int n) { return fabsf(A.scale2) * pow2(n / 2) * pow2(n - n / 2); };      // 2^n may be beyond fp32
        // where `back` is below fp32 its rest goes into the query; where it is beyond, the scores are NaN
        const float f0 = pow2(up / 2) * fminf(back(min(e + 136, 200)), 1.f), f1 = copysignf(pow2(up - up / 2), A.scale2), most = back(e + 10) <= 3.4e38f ? 3.4e38f : -1.f;
        float sum[NG] = {};
#pragma unroll
        for (int w = 0; w < T::W; ++w) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                x[w][k] = fabsf(x[w][k]) <= most ? x[w][k] * f0 * f1 : NAN;      // infinity times a code of zero, minus itself: NaN in any case
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
                part[i][g] = si_cvt<DT>::from_float(rest);
                rest -= si_cvt<DT>::lo(part[i][g]);
            }
        }
#pragma unroll
        for (int i = 0; i < kSumSteps<DT, NG>; ++i)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                uint32_t v = 0;
#pragma unroll
                for (int k = 0; k < kParts<DT>; ++k)
#pragma unroll
                    for (int place = 0; place < NG; ++place) {
                        // NG = 4: part 2 i + t % 2 of place 2 (t / 2) + r; NG = 2: part 2 r + t % 2 of place t / 2; NG = 1: part 2 r + t % 2, t < 2
                        const bool here = NG == 4 ? k == 2 * i + t % 2 && place == 2 * (t / 2) + r : k == 2 * r + t % 2 && place == t / 2;
                        if (here && !(PAIR && lane >> 4)) v = part[k][T::place_of(place)];
                    }
                Q.sum[nt][i][r] = v;
            }
#pragma unroll
        for (int c = 0; c < 2; ++c) Q.back[nt][c] = fminf(fmaxf(back(__shfl_sync(0xFFFFFFFFu, e, 8 * (PAIR ? t & 1 : t) + 4 * c) + 10), 0x1p-126f), 3.4e38f);
#pragma unroll
        for (int c = 0; c < 2; ++c) Q.lazy[nt][c] = kLazy / Q.back[nt][c];
    }
}

// Two results.  Steps are rounded up, so that the highest code may stand for a little more than f16 holds: the largest number then, as
// when it is read back.  The lowest one too: what p s loses in rounding may lie beyond it.
template <int DT> __device__ __forceinline__ uint32_t result2(float a, float b) {
    auto in = [](float x) { return DT == SI_F16 ? si_q4::max_nan(si_q4::min_nan(x, 65504.f), -65504.f) : x; };
    return pack2<DT>(in(a), in(b));
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
// ... onto zeros.
template <int DT> __device__ __forceinline__ void first_product(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (DT == SI_BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void add2(float &a, float &b, float c, float d) {
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(a), "+f"(b) : "f"(c), "f"(d));
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
    constexpr bool kUpShared = NT * L >= 4, kShort = NT == 1 && L == 4;
    using C = Cfg<D, NG, H>;
    constexpr int kStages = kStagesOf<H>;
    const DecodeArgs &A = A4.d;
    extern __shared__ __align__(128) char smem[];
    __shared__ int sh_scan[kThreads / 32 + 1];
    __shared__ Cursor sh_item[kWarps], sh_load[kWarps];        // every warp's item to work on and to load from
    __shared__ uint64_t full[kWarps][kStages];
    __shared__ float2 sh_up[kUpShared ? kWarps : 1][NT * L][4];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lg = lane >> 2, lt = lane & 3;
    const int head_of = PAIR ? 2 * (lt & 1) : 2 * lt, par_of = PAIR ? (lt >> 1) * L * 4 : 0;      // the lane's first head, where its groups' words are
    char *ring = smem + warp * kStages * C::kStage;
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

    // this warp's run
    bool some_empty;
    const Runs runs = find_runs(A, sh_item, sh_scan, blockIdx.x == 0 ? A.status : nullptr, &some_empty);
    const int my_run = warp * gridDim.x + blockIdx.x;      // few runs: on all SMs alike
    const bool any = my_run < runs.n;
    const int g0 = any ? runs.first(my_run) : 0, g1 = any ? runs.first(my_run + 1) : 0;

    // ---- loader side: load_left tiles from load_from on lie one behind the other
    int load_id = g0, load_left = 0;
    const uint8_t *load_from = nullptr;
    const int32_t *load_pos = nullptr;
    if (lane == 0) sh_load[warp] = sh_item[warp];
    __syncwarp();
    const uint32_t ring_addr = si_tc::smem_u32(ring);
    auto issue = [&](int stage) {
        if (load_left == 0) {
            if (load_id >= g1) return;
            Cursor load = sh_load[warp];
            if (load_id >= load.start + kPad + load.w.nc) {
                next_unit_item(A, load);
                __syncwarp();
                if (lane == 0) sh_load[warp] = load;
                __syncwarp();
            }
            const int first = load.start + kPad;
            load_id = max(load_id, first);
            if (load_id >= g1) return;
            const int t = load_id - first, h = load.hh / A.GB;
            const bool sink = t < load.w.c_sink;
            const int c = sink ? t : load.w.c_win + t - load.w.c_sink;
            load_left = min(sink ? load.w.c_sink : load.w.nc, g1 - first) - t;
            load_from = A4.kv.row(load.b, h) + (long long)c * C::kTile;
            if (A.kv.pos) load_pos = A.kv.pos + A.kv.meta(load.b, h) + c * CH;
        }
        if (lane == 0) {
            uint64_t *bar = &full[warp][stage];
            const uint32_t to = ring_addr + stage * C::kStage;
            si_tc::mbar_arrive_expect_tx(bar, C::kTile + (A.kv.pos ? CH * 4 : 0));
            bulk_load(to, load_from, C::kTile, bar, once);
            if (A.kv.pos) bulk_load(to + C::kTile, load_pos, CH * 4, bar, once);
        }
        load_from += C::kTile;
        if (A.kv.pos) load_pos += CH;
        --load_left;
        ++load_id;
    };
#pragma unroll
    for (int s = 0; s < kStages; ++s) issue(s);

    // ---- consumer side
    int id = g0, stage = 0;
    uint32_t parity = 0;
    bool first_segment = true;
    Query<DT, D, NG, H> Q;
    if (any) load_q<DT, D, NG, H>(A, sh_item[warp].b, sh_item[warp].hh, Q);
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
    if (some_empty)
        for (int b = blockIdx.x; b < A.kv.B; b += gridDim.x) {
            if (seq_work<CH>(A, b, nullptr).nc) continue;
            for (int i = tid; i < A.Hq * D; i += kThreads) A.out[(long long)b * A.Hq * D + i] = 0;
            if (A.lse) for (int i = tid; i < A.Hq; i += kThreads) A.lse[(long long)b * A.Hq + i] = -INFINITY;
        }
    if (!any) return;
    while (true) {
        const Cursor &item = sh_item[warp];
        const int start = item.start + kPad, end = start + item.w.nc, c_sink = item.w.c_sink, c_skip = item.w.c_win - c_sink, seg_end = min(g1, end);
        if (start >= g1) return;               // nothing of this item is in the run
        const int h = item.hh / A.GB, gb = item.hh % A.GB, head0 = gb * HB, heads = min(HB, A.G - head0), seq = item.b;
        // tiles numbered whole0 .. whole0 + whole_n - 1 are visible throughout and hold no new entry (without positions)
        int whole0 = 0, whole_n = 0;
        if (!A.kv.pos) {
            const SeqWork &w = item.w;
            const int from = w.lo == INT_MIN ? 0 : max(w.lo, -1) + 1, to = min(min(w.n, w.n_old), w.s >= INT_MAX - 1 ? INT_MAX : w.s + 1);
            const int c0 = max((from + CH - 1) / CH, w.c_win);
            whole0 = start - c_skip + c0;
            whole_n = max(0, to / CH - c0);
        }
        id = max(id, start);
        float *scores_to = A.scores + (((long long)seq * A.kv.H + h) * A.GB + gb) * A.kv.cap * A.GS;
        // o: sum p s (c - 8) 2^-24.  Word i: elements 4 lg + 2 n, 4 lg + 2 n + 1 (the latter times 16) in the two halves of quad 2 i + n.
        // H = 4: words k of an even and an odd group, in the halves of four quads, one per element; those of the lane's own groups count.
        // low: sum p (m + 8 s) of this lane's entries
        float o[NT][2 * W][4] = {}, low[NT][L][2] = {};
        // the maximum (0 while there is none) and the score that moves it, both without the factor `back`.  p is 2^((x - m) back - 12), the
        // difference taken first: with m back rounded, scores beyond 2^24 would lose the 12, and at 2^30 p would be anything
        float m[NT][2], edge[NT][2], l[NT][2];
        // what p s is scaled with for f16, per group and the lane's heads; in shared memory where registers are short
        float2 up_reg[kUpShared ? 1 : NT * L] = {};
        auto up_of = [&](int nt, int g) { if constexpr (kUpShared) return sh_up[warp][nt * L + g][lt]; else return up_reg[nt * L + g]; };
        auto set_up = [&](int nt, int g, float2 y) {       // the eight lanes of these heads have the same
            if constexpr (kUpShared) { __syncwarp(); if (lg == 0) sh_up[warp][nt * L + g][lt] = y; __syncwarp(); }
            else up_reg[nt * L + g] = y;
        };
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) { edge[nt][0] = edge[nt][1] = -INFINITY; m[nt][0] = m[nt][1] = l[nt][0] = l[nt][1] = 0.f; }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int g = 0; g < L; ++g) set_up(nt, g, make_float2(kMostUp, kMostUp));
        // o of a group and head times f
        auto scale_o = [&](int nt, int g, int c, float f) {
#pragma unroll
            for (int i = 0; i < 2 * W; ++i)
                if ((PAIR ? i / 4 / GW : T::place_of(T::group_of(i / 2))) == g) { o[nt][i][c] *= f; o[nt][i][c + 2] *= f; }
        };
        // The next tile in the ring: waits for it, clears the steps of hidden entries (they must not meet the products: 0 * NaN), puts the
        // new entry in its place.  Which entries are visible.
        auto first_of = [&]() { const int t = id - start; return (t < c_sink ? t : t + c_skip) * CH; };
        auto prepare = [&](char *tile) -> uint32_t {
            if (!si_tc::mbar_wait(&full[warp][stage], parity, si_tc::kSpinLimit)) si_report(A.status, SI_ERR_TIMEOUT);
            if ((unsigned)(id - whole0) < (unsigned)whole_n) return 0xFFFFFFFFu;
            const int j0 = first_of();
            const SeqWork w = item.w;
            const int j = j0 + lane;
            int p = j;
            if (A.kv.pos) p = j == w.n_old ? w.s : *reinterpret_cast<const int *>(tile + C::kTile + lane * 4);
            const uint32_t vis = __ballot_sync(0xFFFFFFFFu, j < w.n && si_visible(p, w.s, w.lo, A.n_sink));
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
                const long long from = seq * A.new_ss + (long long)h * D;
                si_q4::store_entry<DT, D, NG>(A.kn + from, A.vn + from, w.n_old - j0, tile, gb == 0 ? (char *)A4.kv.row(seq, h) + (long long)(j0 / CH) * C::kTile : nullptr);
                if (gb == 0 && A.kv.pos && lane == 0) A.kv.pos[A.kv.meta(seq, h) + w.n_old] = w.s;
                __syncwarp();
            }
            if (vis != 0xFFFFFFFFu || fresh) si_tc::fence_async_proxy();      // the next copy into this stage comes behind these writes
            return vis;
        };
        // Scores but for the factor `back`: entries 16 u + lg and 16 u + lg + 8, the lane's heads.  The products of both halves of a tile take
        // turns: they wait for their own sums only.
        auto scores = [&](const char *tile, float (&x)[2][NT][4]) {
            uint32_t ka[2][W], kb[2][W], pa[2][L], pb[2][L];
            float acc[2][NT][L][4], sum[2][NT][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                load_words(ka[u], tile + u * 8 * D + lane * T::kCell);
                load_words(kb[u], tile + u * 8 * D + 4 * D + lane * T::kCell);
                load_words(pa[u], tile + T::kKeyPar + (u * 16 + lg) * NG * 4 + par_of);
                load_words(pb[u], tile + T::kKeyPar + (u * 16 + 8 + lg) * NG * 4 + par_of);
                uint32_t wa[kOwn<NG>], wb[kOwn<NG>];
                if constexpr (PAIR || NG == 1) {
#pragma unroll
                    for (int r = 0; r < kOwn<NG>; ++r) { wa[r] = pa[u][r]; wb[r] = pb[u][r]; }
                } else {
                    load_words(wa, tile + T::kKeyPar + (u * 16 + lg) * NG * 4 + (lt >> 1) * kOwn<NG> * 4);
                    load_words(wb, tile + T::kKeyPar + (u * 16 + 8 + lg) * NG * 4 + (lt >> 1) * kOwn<NG> * 4);
                }
                const uint32_t a[4] = {wa[0], wb[0], wa[kOwn<NG> - 1], wb[kOwn<NG> - 1]};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < kSumSteps<DT, NG>; ++i) {
                        if (i == 0) first_product<DT>(sum[u][nt], a, Q.sum[nt][i][0], Q.sum[nt][i][1]);
                        else product<DT>(sum[u][nt], a, Q.sum[nt][i][0], Q.sum[nt][i][1]);
                    }
            }
            constexpr int WL = W / L;          // words of a sum
#pragma unroll
            for (int k = 0; k < WL; ++k)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int g = 0; g < L; ++g)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const int i = g * WL + k;
                            const uint32_t a[4] = {si_q4::low_codes(ka[u][i] >> 8 * half), si_q4::low_codes(kb[u][i] >> 8 * half), si_q4::high_codes(ka[u][i] >> 8 * half), si_q4::high_codes(kb[u][i] >> 8 * half)};
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                if (k == 0 && half == 0) first_product<SI_F16>(acc[u][nt][g], a, Q.f[nt][i][0], Q.f[nt][i][1]);
                                else product<SI_F16>(acc[u][nt][g], a, Q.f[nt][i][2 * half], Q.f[nt][i][2 * half + 1]);
                            }
                        }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float y = sum[u][nt][e] * (0x1p-24f / kSumScale<DT>);
#pragma unroll
                        for (int g = 0; g < L; ++g) y = fmaf(acc[u][nt][PAIR ? g : T::place_of(g)][e], si_cvt<DT>::hi(e >> 1 ? pb[u][g] : pa[u][g]), y);
                        x[u][nt][e] = PAIR ? y + __shfl_xor_sync(0xFFFFFFFFu, y, 2) : y;
                    }
        };
        // p of the same entries, and their share of the sums.  One vote for all that seldom happens: the maximum and the scales move.
        auto add = [&](const char *tile, const float (&x)[2][NT][4], const uint32_t (&vp)[2][2][L]) {
            uint32_t va[2][W], vb[2][W], pf[2][NT][L][2];
            auto times_step = [&](float2 y, uint32_t word) { const float s = si_cvt<DT>::hi(word); return __fmul2_rn(y, make_float2(s, s)); };
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                bool grow = false;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) grow |= x[u][nt][e] > edge[nt][e & 1];
                float2 p[2][2];                            // entries 16 u + 8 r + lg, the lane's heads
                auto make_p = [&]() {
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float2 d = __fadd2_rn(make_float2(x[u][nt][2 * r], x[u][nt][2 * r + 1]), make_float2(-m[nt][0], -m[nt][1]));
                            const float2 y = __ffma2_rn(d, make_float2(Q.back[nt][0], Q.back[nt][1]), make_float2(-kRoom, -kRoom));
                            p[u][r] = make_float2(ex2(y.x), ex2(y.y));
                        }
                };
                make_p();
                auto pack = [&]() {
                    uint32_t top = 0;                      // the largest of each half (NaN above all)
#pragma unroll
                    for (int g = 0; g < L; ++g) {
                        const float2 f = up_of(nt, g);
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            uint32_t ps[2];
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                const float2 y = __fmul2_rn(times_step(p[u][r], vp[u][r][g]), f);
                                ps[r] = pack2<SI_F16>(y.x, y.y);
                                pf[u][nt][g][r] = transposed(ps[r]);
                            }
                            top = __vimax3_u16x2(top, ps[0], ps[1]);
                        }
                    }
                    return ((top + 0x08000800u) & 0x80008000u) != 0;
                };
                if (__builtin_expect(__any_sync(0xFFFFFFFFu, pack() | grow), 0)) {
                    float f[2] = {1.f, 1.f};
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const bool none = edge[nt][c] == -INFINITY;
                        float mx = none ? -INFINITY : m[nt][c];
#pragma unroll
                        for (int u = 0; u < 2; ++u) mx = fmaxf(mx, fmaxf(x[u][nt][c], x[u][nt][c + 2]));
                        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 16));
                        if (mx == -INFINITY) continue;         // all hidden or NaN
                        if (!none) f[c] = ex2((m[nt][c] - mx) * Q.back[nt][c]);
                        m[nt][c] = mx;
                        edge[nt][c] = mx + Q.lazy[nt][c];
                        l[nt][c] *= f[c];
                    }
                    make_p();
                    // a score far above the maximum, or a p s of 2^15 or more: the maximum moves, and the scale of every group and head
                    // whose largest p s is above 2^14 then goes down, so that it is 2^7 again
#pragma unroll
                    for (int g = 0; g < L; ++g) {
                        float2 most = make_float2(0.f, 0.f);
                        const float2 was = up_of(nt, g);
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                const float2 y = times_step(p[u][r], vp[u][r][g]);
                                most = make_float2(fmaxf(most.x, y.x), fmaxf(most.y, y.y));      // NaN does not count
                            }
#pragma unroll
                        for (int s = 4; s < 32; s <<= 1) most = make_float2(fmaxf(most.x, __shfl_xor_sync(0xFFFFFFFFu, most.x, s)), fmaxf(most.y, __shfl_xor_sync(0xFFFFFFFFu, most.y, s)));
                        float2 now;
                        auto move = [&](int c, float ps, float from, float &to) {
                            // p has fallen by f, so its scale rises by as much; but p s is to fit
                            to = f[c] == 1.f ? from : fminf(__fdividef(from, f[c]), kMostUp);
                            if (ps * to > 16384.f) to = __fdividef(128.f, ps);
                            if (f[c] != 1.f || to != from) scale_o(nt, g, c, __fdividef(f[c] * to, from));
                            low[nt][g][c] *= f[c];
                        };
                        move(0, most.x, was.x, now.x);
                        move(1, most.y, was.y, now.y);
                        set_up(nt, g, now);
                    }
                    pack();
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float2 y = p[u][r];
                        uint32_t word[L];                  // once more where registers are short
                        if constexpr (kShort) load_words(word, tile + T::kValuePar + (u * 16 + r * 8 + lg) * NG * 4 + par_of);
                        add2(l[nt][0], l[nt][1], y.x, y.y);
#pragma unroll
                        for (int g = 0; g < L; ++g) {
                            const uint32_t v = kShort ? word[g] : vp[u][r][g];
                            const float mn = fmaf(8.f, si_cvt<DT>::hi(v), si_cvt<DT>::lo(v));
                            const float2 z = __ffma2_rn(y, make_float2(mn, mn), make_float2(low[nt][g][0], low[nt][g][1]));
                            low[nt][g][0] = z.x; low[nt][g][1] = z.y;
                        }
                    }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                load_words(va[u], tile + T::kValues + u * 8 * D + lt * D + (lg ^ T::swizzle(lt)) * T::kCell);
                load_words(vb[u], tile + T::kValues + u * 8 * D + 4 * D + lt * D + (lg ^ T::swizzle(lt)) * T::kCell);
            }
            // Every sum also gets -8 times (upper nibbles: -128 times) the sum of its rounded p s, which a product with constants gives: with
            // codes around zero it stays small, and so do what the matrix unit cuts off of it and what the rounding of p s leaves
            // (2052 entries, f16: error 2.6e-4 instead of 4.7e-4; 260001, bf16: 1.7e-3 instead of 4.5e-3).  In the products
            // themselves, as one more each, it cost 5 us of 68 for one sequence of 260001.
            auto codes = [&](uint32_t w, int n) { return n & 1 ? si_q4::high_codes(w >> 4 * (n & 2)) : si_q4::low_codes(w >> 4 * (n & 2)); };
            constexpr uint32_t kEight = 0x80088008u;           // a pair of -8 2^-24
            const uint32_t eight[4] = {kEight, kEight, kEight, kEight};
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if constexpr (PAIR) {
#pragma unroll
                    for (int i = 0; i < W / 2; ++i) {
                        const int even = i / GW * 2 * GW + i % GW, odd = even + GW;
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            const uint32_t a[4] = {codes(va[u][even], n), codes(va[u][odd], n), codes(vb[u][even], n), codes(vb[u][odd], n)};
                            product<SI_F16>(o[0][4 * i + n], a, pf[u][0][i / GW][0], pf[u][0][i / GW][1]);
                        }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < W; ++i)
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const uint32_t a[4] = {codes(va[u][i], 2 * half), codes(va[u][i], 2 * half + 1), codes(vb[u][i], 2 * half), codes(vb[u][i], 2 * half + 1)};
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                const int g = T::place_of(T::group_of(i));
                                product<SI_F16>(o[nt][2 * i + half], a, pf[u][nt][g][0], pf[u][nt][g][1]);
                            }
                        }
                }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int g = 0; g < L; ++g) {
                    float e[4];
                    first_product<SI_F16>(e, eight, pf[0][nt][g][0], pf[0][nt][g][1]);
                    product<SI_F16>(e, eight, pf[1][nt][g][0], pf[1][nt][g][1]);
                    const float f0 = 16.f * e[0], f1 = 16.f * e[1];
                    if constexpr (PAIR) {
#pragma unroll
                        for (int i = g * GW; i < (g + 1) * GW; ++i)
#pragma unroll
                            for (int n = 0; n < 4; ++n) {
                                float (&q)[4] = o[nt][4 * i + n];
                                add2(q[0], q[1], n & 1 ? f0 : e[0], n & 1 ? f1 : e[1]);
                                add2(q[2], q[3], n & 1 ? f0 : e[0], n & 1 ? f1 : e[1]);
                            }
                    } else {
#pragma unroll
                        for (int i = 0; i < W; ++i)
                            if (T::place_of(T::group_of(i)) == g)
#pragma unroll
                                for (int half = 0; half < 2; ++half) {
                                    float (&q)[4] = o[nt][2 * i + half];
                                    add2(q[0], q[1], e[0], e[1]);
                                    add2(q[2], q[3], f0, f1);
                                }
                    }
                }
        };
        float x[2][NT][4];
        uint32_t vp[2][2][L];
        // Hidden entries out of the scores; the scores out for the weights; steps of the values.
        auto settle = [&](const char *tile, uint32_t vis) {
            if (vis != 0xFFFFFFFFu) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!(vis >> (u * 16 + lg + (e >> 1) * 8) & 1)) x[u][nt][e] = -INFINITY;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 2; ++r) load_words(vp[u][r], tile + T::kValuePar + (u * 16 + r * 8 + lg) * NG * 4 + par_of);
            if (A.acc) {
                const int j0 = first_of();
                float *sc = scores_to + (long long)j0 * A.GS;
                const int left = vis == 0xFFFFFFFFu ? CH : item.w.n - j0;         // entries of the tile
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const int key = u * 16 + lg + (e >> 1) * 8, head = nt * 8 + head_of;
                            if (head < A.GS && key < left && !(PAIR && lt >> 1))
                                asm volatile("st.global.L2::cache_hint.v2.f32 [%0], {%1, %2}, %3;"
                                             ::"l"(sc + key * A.GS + head), "f"(x[u][nt][e] * Q.back[nt][0]), "f"(x[u][nt][e + 1] * Q.back[nt][1]), "l"(stay) : "memory");
                        }
            }
        };
        for (; id < seg_end; ++id) {
            char *tile = ring + stage * C::kStage;
            const uint32_t vis = prepare(tile);
            scores(tile, x);
            settle(tile, vis);
            add(tile, x, vp);
            __syncwarp();                      // the stage may be loaded again
            issue(stage);
            if (++stage == kStages) { stage = 0; parity ^= 1; }
        }
        // ---- the item's end, or the run's: the lanes' sums joined; a result, or a part for the joining kernel
        const bool whole = start >= g0 && end <= g1;
        const long long slot = (long long)my_run * 2 + (first_segment ? 0 : 1), row = (long long)seq * A.Hq + h * A.G + head0;
        if (lane == 0 && start >= g0)          // the runs of this item, for the joining kernel: by the one that has its first tile
            A.runs[(long long)seq * A.kv.H * A.GB + item.hh] = make_int2(my_run | (first_segment ? 0 : kSecondSlot), whole ? my_run : runs.of(end - 1));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int head = nt * 8 + head_of + c;
#pragma unroll
                for (int s = 4; s < 32; s <<= 1) {
                    l[nt][c] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][c], s);
#pragma unroll
                    for (int g = 0; g < L; ++g) low[nt][g][c] += __shfl_xor_sync(0xFFFFFFFFu, low[nt][g][c], s);
                }
                if (head >= heads) continue;
                const float sum = l[nt][c], inv = sum == 0.f ? 0.f : 1.f / sum;
                // what the maximum loses as a score of its own goes into the sums (where a score has less than whole numbers, nothing is known of it)
                const float top = m[nt][c] * Q.back[nt][c], lost = fmaf(m[nt][c], Q.back[nt][c], -top), rest = fabsf(lost) < 1.f ? lost : 0.f, grow = ex2(rest);
                if (lg == 0 && !(PAIR && lt >> 1)) {
                    if (whole) {
                        if (A.lse) A.lse[row + head] = sum == 0.f ? -INFINITY : (top + (rest + log2f(sum * kOne))) / kLog2e;
                        if (A.acc) A.done[row + head] = make_float2(top, inv * ex2(-rest - (float)kRoom));
                    } else {
                        *reinterpret_cast<float2 *>(A.part_ml + (slot * HB + head) * 2) = make_float2(edge[nt][c] == -INFINITY ? -INFINITY : top, sum * grow);
                    }
                }
#pragma unroll
                for (int i = 0; i < (PAIR ? W / 2 : W); ++i) {
                    // the lane's words: all, or k of its own groups
                    const int word = PAIR ? i / GW * 2 * GW + i % GW + (lt >> 1) * GW : i;
                    const int g = PAIR ? i / GW : T::place_of(T::group_of(i));
                    const float mn = low[nt][g][c], f0 = __fdividef(0x1p24f, c ? up_of(nt, g).y : up_of(nt, g).x), f1 = f0 * 0.0625f;
                    auto of = [&](int n) { return PAIR ? (lt >> 1 ? o[nt][(4 * i + n) % (2 * W)][c + 2] : o[nt][(4 * i + n) % (2 * W)][c]) : o[nt][2 * i + n / 2][c + 2 * (n & 1)]; };
                    const float4 y = make_float4(fmaf(of(0), f0, mn), fmaf(of(1), f1, mn), fmaf(of(2), f0, mn), fmaf(of(3), f1, mn));
                    if (whole) *reinterpret_cast<uint2 *>(A.out + (row + head) * D + 32 * word + 4 * lg) = make_uint2(result2<DT>(y.x * inv, y.y * inv), result2<DT>(y.z * inv, y.w * inv));
                    else *reinterpret_cast<float4 *>(A.part_o + (slot * HB + head) * D + 32 * word + 4 * lg) = make_float4(y.x * grow, y.y * grow, y.z * grow, y.w * grow);
                }
            }
        first_segment = false;
        if (end >= g1) return;
        __syncwarp();
        if (lane == 0) { Cursor next = item; next_unit_item(A, next); sh_item[warp] = next; }
        __syncwarp();
        load_q<DT, D, NG, H>(A, sh_item[warp].b, sh_item[warp].hh, Q);
    }
}

// Joins the parts of items that more than one run has, and, where weights are wanted, adds them up.  The first n_out CTAs of a
// (sequence, key head) make the output: a thread per pair of channels of a head and slice of the parts, eight parts at a time,
// each slice relative to its own maximum; the slices are joined in order.  The others have U * 256 keys each and add their weights.
// Chains of short dependent loads: what does not depend on another load is asked for first (scores and weights beyond the length
// too: the memory is there, the values are not used).  GX: heads per key in `scores` at most.
constexpr int kJoin4 = 256, kMaxSlices = 16;
template <int DT, int D, int NT, int GX, int U>
__global__ void __launch_bounds__(kJoin4, 3) join4_kernel(const DecodeArgs A, const int n_out) {
    constexpr int HB = 8 * NT, CH = kTileEntries;
    __shared__ float2 sh_done[128];
    __shared__ float4 sh_part[kJoin4];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, h = blockIdx.y, b = blockIdx.z;
    si_tc::pdl_wait();
    si_tc::pdl_launch();
    const int2 *runs = A.runs + ((long long)b * A.kv.H + h) * A.GB;
    const long long row = (long long)b * A.Hq + h * A.G;
    const int2 run0 = runs[0];
    struct Parts { int first, n, slot0; };
    auto parts_of = [&](int gb) {
        const int2 r = gb == 0 ? run0 : runs[gb];
        return Parts{r.x & ~kSecondSlot, r.y - (r.x & ~kSecondSlot) + 1, r.x & kSecondSlot ? 1 : 0};      // later runs begin with the item
    };
    auto slot = [&](const Parts &p, int i) { return (long long)(p.first + i) * 2 + (i > 0 ? 0 : p.slot0); };
    auto part_ml = [&](const Parts &p, int i, int head) { return *reinterpret_cast<const float2 *>(A.part_ml + (slot(p, i) * HB + head) * 2); };
    // a part without a maximum has sums of 0, or NaN (NaN scores only)
    auto factor = [&](float v, float top) { return v == -INFINITY ? 1.f : ex2(v - top); };
    if ((int)blockIdx.x < n_out) {
        if (seq_work<CH>(A, b, nullptr).nc == 0) return;
        for (int gb = 0; gb < A.GB; ++gb) {
            const int head0 = gb * HB, heads = min(HB, A.G - head0), pairs = heads * (D / 2);
            const Parts p = parts_of(gb);
            if (p.n == 1) continue;                        // finished by one warp
            int slices = 1;
            while (slices < kMaxSlices && p.n > 8 * slices) slices *= 2;
            const int wide = kJoin4 / slices, slice = tid / wide;
            const int k0 = p.n * slice / slices, k1 = p.n * (slice + 1) / slices;
            for (int u = blockIdx.x; u * wide < pairs; u += n_out) {
                const int at = u * wide + tid % wide, head = at / (D / 2), pair = at % (D / 2);
                float4 sum = make_float4(0.f, 0.f, -INFINITY, 0.f);        // two channels, maximum, sum of p
                if (at < pairs)
                    for (int k = k0; k < k1; k += 8) {
                        float2 o[8], ml[8];
                        float top = sum.z;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const bool in = k + i < k1;
                            ml[i] = in ? part_ml(p, k + i, head) : make_float2(-INFINITY, 0.f);
                            o[i] = in ? *reinterpret_cast<const float2 *>(A.part_o + (slot(p, k + i) * HB + head) * D + 2 * pair) : make_float2(0.f, 0.f);
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) top = fmaxf(top, ml[i].x);
                        const float f = factor(sum.z, top);
                        sum = make_float4(sum.x * f, sum.y * f, top, sum.w * f);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float g = factor(ml[i].x, top);
                            sum.x += o[i].x * g; sum.y += o[i].y * g; sum.w += ml[i].y * g;
                        }
                    }
                if (slices > 1) {
                    __syncthreads();
                    sh_part[tid] = sum;
                    __syncthreads();
                    if (slice == 0) {
                        float top = sum.z;
                        for (int k = 1; k < slices; ++k) top = fmaxf(top, sh_part[k * wide + tid].z);
                        const float f = factor(sum.z, top);
                        sum = make_float4(sum.x * f, sum.y * f, top, sum.w * f);
                        for (int k = 1; k < slices; ++k) {
                            const float4 t = sh_part[k * wide + tid];
                            const float g = factor(t.z, top);
                            sum.x += t.x * g; sum.y += t.y * g; sum.w += t.w * g;
                        }
                    }
                }
                if (slice == 0 && at < pairs) {
                    const float inv = sum.w == 0.f ? 0.f : 1.f / sum.w;
                    *reinterpret_cast<uint32_t *>(A.out + (row + head0 + head) * D + 2 * pair) = result2<DT>(sum.x * inv, sum.y * inv);
                    if (pair == 0 && A.lse) A.lse[row + head0 + head] = sum.w == 0.f ? -INFINITY : ((sum.z == -INFINITY ? 0.f : sum.z) + log2f(sum.w * kOne)) / kLog2e;
                }
            }
        }
        return;
    }
    const int j0 = (blockIdx.x - n_out) * (U * kJoin4);
    SeqWork w;
    // few keys a thread: everything at once; many: not before it is known that the range has entries
    if (U > 1) { w = seq_work<CH>(A, b, nullptr); if (j0 >= w.n) return; }
    float *weight = A.kv.weight + A.kv.meta(b, h);
    const float *sc = A.scores + ((long long)b * A.kv.H + h) * A.GB * A.kv.cap * A.GS;
    float2 x[U][GX / 2];                   // the first head block's scores
    float old[U];
    const int most = U > 1 ? w.n : A.kv.cap;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int j = j0 + i * kJoin4 + tid;
        if (j >= most) continue;
        old[i] = weight[j];
#pragma unroll
        for (int g = 0; g < GX; g += 2)
            if (g < A.GS) x[i][g / 2] = *reinterpret_cast<const float2 *>(sc + (long long)j * A.GS + g);
    }
    const float2 whole = tid < A.G ? A.done[row + tid] : make_float2(0.f, 0.f);
    if (U == 1) { w = seq_work<CH>(A, b, nullptr); if (j0 >= w.n) return; }
    if (tid < A.G) sh_done[tid] = whole;
    __syncthreads();
    for (int gb = 0; gb < A.GB && w.nc > 0; ++gb) {
        const int head0 = gb * HB, heads = min(HB, A.G - head0);
        const Parts p = parts_of(gb);
        if (p.n == 1) continue;
        for (int head = warp; head < heads; head += kJoin4 / 32) {      // a warp per head, a lane per part
            float2 ml[4];                              // the first 128 parts stay in registers
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) ml[k] = k * 32 + lane < p.n ? part_ml(p, k * 32 + lane, head) : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int k = 0; k < 4; ++k) top = fmaxf(top, ml[k].x);
            for (int i = 128 + lane; i < p.n; i += 32) top = fmaxf(top, part_ml(p, i, head).x);
#pragma unroll
            for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
#pragma unroll
            for (int k = 0; k < 4; ++k) sum += ml[k].y * factor(ml[k].x, top);
            for (int i = 128 + lane; i < p.n; i += 32) { const float2 v = part_ml(p, i, head); sum += v.y * factor(v.x, top); }
#pragma unroll
            for (int s = 16; s; s >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, s);
            if (lane == 0) sh_done[head0 + head] = make_float2(top == -INFINITY ? 0.f : top, sum == 0.f ? 0.f : 1.f / (sum * kOne));
        }
    }
    __syncthreads();
    // the first block's heads: a hidden entry's score is -inf; it receives nothing, from a head whose sum is NaN neither
    float add[U] = {};
#pragma unroll
    for (int g = 0; g < GX; ++g) {
        if (g >= A.G) break;
        const float2 done = sh_done[g];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const float y = g & 1 ? x[i][g / 2].y : x[i][g / 2].x;
            if (y != -INFINITY) add[i] = fmaf(ex2(y - done.x), done.y, add[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int j = j0 + i * kJoin4 + tid, c = j / CH;
        if (j >= w.n) continue;
        if (!(c < w.c_sink || (c >= w.c_win && c < w.c_win + w.nc - w.c_sink))) { if (j == w.n_old) weight[j] = 0.f; continue; }
        float sum = add[i];
        for (int gb = 1; gb < A.GB; ++gb)
            for (int g = gb * HB; g < min(A.G, gb * HB + HB); ++g) {
                const float y = sc[((long long)gb * A.kv.cap + j) * A.GS + g - gb * HB];
                if (y != -INFINITY) sum = fmaf(ex2(y - sh_done[g].x), sh_done[g].y, sum);
            }
        weight[j] = j == w.n_old ? sum : old[i] + sum;
    }
}

template <int DT, int D, int NT, int GX> int launch_join4(const DecodeArgs &A, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at; cfg.numAttrs = 1;
    cfg.stream = st;
    cfg.blockDim = dim3(kJoin4);
    constexpr int kKeys = NT == 1 ? 4 : 2;
    const long long items = (long long)A.kv.H * A.kv.B;
    // CTAs for the output while they are resident at once (four per SM)
    const long long room = 4ll * si_sm_count() / items, most = (long long)(A.G < 8 * NT ? A.G : 8 * NT) * (D / 2) * kMaxSlices / kJoin4;
    const int n_out = (int)(room < 1 || most < 1 ? 1 : room < most ? room : most);
    // ranges of 256 keys while all their CTAs are resident at once (three per SM): the start of a CTA costs more than its keys
    const bool few = items * ((A.kv.cap + kJoin4 - 1) / kJoin4) <= 3ll * si_sm_count();
    const int keys = (few ? 1 : kKeys) * kJoin4;
    cfg.gridDim = dim3(n_out + (A.acc ? (A.kv.cap + keys - 1) / keys : 0), A.kv.H, A.kv.B);
    if (few || !A.acc) SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, join4_kernel<DT, D, NT, GX, 1>, A, n_out));
    else SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, join4_kernel<DT, D, NT, GX, kKeys>, A, n_out));
    return SI_OK;
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
    cfg.gridDim = dim3(A.d.n_cta / kWarps);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::kSmem;
    cfg.stream = st;
    SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, decode4_kernel<DT, D, NG, H>, A));
    if constexpr (H == 16) return launch_join4<DT, D, 2, 16>(A.d, st);
    else return A.d.GS <= 4 ? launch_join4<DT, D, 1, 4>(A.d, st) : launch_join4<DT, D, 1, 8>(A.d, st);
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
    return layout_of((n_q_heads / kv->n_kv_heads > 8 ? kPerSmOf<16> : kPerSmOf<8>) * kWarps * si_sm_count(), kv->n_seqs, kv->n_kv_heads, kv->head_dim, kv->capacity, n_q_heads, acc);
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
    if ((double)kv->n_seqs * kv->n_kv_heads * L.GB * (kv->capacity / kTileEntries + 2 + kPad) > 2.0e9) return SI_ERR_TOO_LARGE;
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
