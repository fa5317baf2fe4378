// What the single-token kernels over a key/value cache share, whatever its entries are held in: a call's arguments, the chunks of a
// sequence that hold visible entries, the workspace; and for 16-bit entries the row of all chunks, cut into equal runs, one per CTA, and
// the kernel that joins the parts of items that cross CTAs in their order and adds up the weights.  CH: entries of a chunk.
#pragma once
#include "si_kv.cuh"
#include "si_tc.cuh"

namespace {

constexpr int kJoinWarps = 8, kJoinThreads = kJoinWarps * 32;
constexpr int kMaxParts = 608;             // CTAs of a main kernel whose parts decode_join_kernel joins at most
constexpr int kSecondSlot = 1 << 30;       // in the table of runs: the item's first part is in the second slot of its CTA
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.f;               // the running maximum moves only when a score exceeds it by 2^8: p stays below 2^8, exact to fp32 all the same

struct DecodeArgs {
    si_kv_view kv;
    const uint16_t *q, *kn, *vn;
    const int32_t *q_pos;
    long long q_ss, new_ss;
    int Hq, G, GB, GS, window, n_sink;   // GB: blocks of 8 * NT heads per key head; GS: heads per key in `scores`
    float scale2;                        // scale * log2(e)
    uint16_t *out;
    float *lse;
    int32_t *status;
    int acc, n_cta;
    float *part_o, *part_ml;             // [n_cta][2][8 NT][D], [n_cta][2][8 NT][2]
    float2 *done;                        // [B][Hq]: maximum and 1 / sum of finished items (weights only: p = 2^(score - maximum) / sum, without
                                         // the rounding of a logarithm)
    float *scores;                       // [B][H][GB][cap][GS]
    int2 *runs;                          // [B][H][GB]: first and last CTA of an item
};

// The chunks of sequence b that hold visible entries: c_sink chunks from the front, then those from c_win to c_end.
struct SeqWork { int n, n_old, s, lo, c_sink, c_win, nc; };
template <int CH> __device__ __forceinline__ SeqWork seq_work(const DecodeArgs &A, int b, int32_t *status) {
    SeqWork w;
    w.n = si_kv_len(A.kv, b, status);
    w.n_old = INT_MAX;
    if (A.kn) {
        if (w.n < A.kv.cap) w.n_old = w.n++;
        else si_report(status, SI_ERR_OUT_OF_RANGE);
    }
    w.s = A.q_pos ? A.q_pos[b] : w.n - 1;
    w.lo = si_window_lo(w.s, A.window);
    w.c_sink = 0; w.c_win = 0;
    int end = w.n;
    if (!A.kv.pos) {                               // entry j is at position j
        end = max(0, min(w.n, w.s >= INT_MAX - 1 ? w.n : w.s + 1));
        if (w.lo >= 0) {
            const int first = min(w.lo + 1, end);
            w.c_win = first / CH;
            w.c_sink = min((min(A.n_sink, first) + CH - 1) / CH, w.c_win);
        }
    }
    w.nc = w.c_sink + (end + CH - 1) / CH - w.c_win;
    return w;
}

__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ uint32_t mov_trans(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
template <int DT> __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    if (DT == SI_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int DT> __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (DT == SI_BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Position in the row of all chunks: item = (sequence, head block), its first chunk and its number of chunks.
struct Cursor {
    int start;           // number of the item's first chunk among all
    int b, hh;           // hh = head * GB + head block
    SeqWork w;
};
template <int CH> __device__ __forceinline__ bool next_item(const DecodeArgs &A, Cursor &c) {   // false: past the last one
    c.start += c.w.nc;
    if (++c.hh < A.kv.H * A.GB && c.w.nc > 0) return true;
    c.hh = 0;
    do {
        if (++c.b >= A.kv.B) { c.w.nc = 0; return false; }
        c.w = seq_work<CH>(A, c.b, nullptr);
    } while (c.w.nc == 0);
    return true;
}

// Number of chunks of all items; the first chunk of this CTA's run is at `at` on return (of all threads, if there is one).  Thread t
// of the block stands for sequences t * per ..; the one that holds the run's first chunk looks it up.
struct Run { int g0, g1, per; bool empty; };
template <int CH, int kThreads> __device__ __forceinline__ Run find_run(const DecodeArgs &A, Cursor *at, int *sh, int32_t *status) {
    const int tid = threadIdx.x, share = (A.kv.B + kThreads - 1) / kThreads, items = A.kv.H * A.GB;
    const int b0 = min(A.kv.B, tid * share), b1 = min(A.kv.B, b0 + share);
    int sum = 0;
    bool empty = false;
    Cursor c;
    for (int b = b0; b < b1; ++b) {
        c.w = seq_work<CH>(A, b, status);
        sum += c.w.nc * items;
        empty |= c.w.nc == 0;
    }
    const int before = si_block_scan<kThreads>(sum, sh), total = sh[kThreads / 32];
    Run r;
    r.per = (total - 1) / A.n_cta + 1;
    r.g0 = (int)min((long long)total, (long long)blockIdx.x * r.per);
    r.g1 = total - r.g0 < r.per ? total : r.g0 + r.per;
    if (r.g0 < r.g1 && before <= r.g0 && r.g0 - before < sum) {
        int start = before;
        c.b = b0;
        if (share > 1) c.w = seq_work<CH>(A, b0, nullptr);    // with one sequence per thread it is at hand
        while (start + c.w.nc * items <= r.g0) { start += c.w.nc * items; c.w = seq_work<CH>(A, ++c.b, nullptr); }
        c.hh = (r.g0 - start) / c.w.nc;
        c.start = start + c.hh * c.w.nc;
        *at = c;
    }
    r.empty = __syncthreads_or(empty);                       // some sequence has nothing to see
    return r;
}

// Joins the parts of items that crossed CTAs and, where weights are wanted, adds them up.  One CTA per (sequence, key head)
// and range of U * 256 keys; the first range's writes the output.  A chain of short dependent loads: everything that does not
// depend on another load is asked for first (scores and weights beyond the length too: the memory is there, the values are
// not used).  At most 80 registers, so that the CTAs become resident beside the main kernel's and wait there for its end.
template <int DT, int D, int NT, int CH, int U>
__global__ void __launch_bounds__(kJoinThreads, 3) decode_join_kernel(const DecodeArgs A) {
    constexpr int HB = 8 * NT;
    __shared__ float sh_f[HB][kMaxParts];
    __shared__ float2 sh_done[128];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, h = blockIdx.y, b = blockIdx.z, j0 = blockIdx.x * (U * kJoinThreads);
    si_tc::pdl_wait();
    si_tc::pdl_launch();
    float *weight = A.kv.weight + A.kv.meta(b, h);
    const float *sc = A.scores + ((long long)b * A.kv.H + h) * A.GB * A.kv.cap * A.GS;
    float2 x[U][HB / 2];                   // the first head block's scores
    float old[U];
    if (A.acc) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int j = j0 + i * kJoinThreads + tid;
            if (j >= A.kv.cap) continue;
            old[i] = weight[j];
#pragma unroll
            for (int g = 0; g < HB; g += 2)
                if (g < A.GS) x[i][g / 2] = *reinterpret_cast<const float2 *>(sc + (long long)j * A.GS + g);
        }
    }
    const long long row = (long long)b * A.Hq + h * A.G;
    const float2 whole = A.acc && tid < A.G ? A.done[row + tid] : make_float2(0.f, 0.f);
    const SeqWork w = seq_work<CH>(A, b, nullptr);
    if (j0 >= w.n && (blockIdx.x > 0 || w.nc == 0)) return;
    if (A.acc && tid < A.G) sh_done[tid] = whole;
    for (int gb = 0; gb < A.GB && w.nc > 0; ++gb) {
        const int head0 = gb * HB, heads = min(HB, A.G - head0);
        int2 run = A.runs[((long long)b * A.kv.H + h) * A.GB + gb];
        const int first_slot = run.x & kSecondSlot ? 1 : 0;
        run.x &= ~kSecondSlot;
        if (run.x == run.y) continue;                  // finished by one CTA
        const int parts = run.y - run.x + 1;
        auto slot = [&](int i) { return (long long)(run.x + i) * 2 + (i > 0 ? 0 : first_slot); };     // later CTAs begin with the item
        __syncthreads();
        for (int head = warp; head < heads; head += kJoinWarps) {      // a warp per head, a lane per part: one round of loads
            float2 ml[4];                              // the first 128 parts stay in registers
            float top = -INFINITY, sum = 0.f;
            auto part = [&](int i) { return i < parts ? *reinterpret_cast<const float2 *>(A.part_ml + (slot(i) * HB + head) * 2) : make_float2(-INFINITY, 0.f); };
#pragma unroll
            for (int k = 0; k < 4; ++k) { ml[k] = part(k * 32 + lane); top = fmaxf(top, ml[k].x); }
            for (int i = 128 + lane; i < parts; i += 32) top = fmaxf(top, part(i).x);
#pragma unroll
            for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            auto add = [&](int i, float2 v) {
                if (i >= parts) return;
                const float f = v.x == -INFINITY ? 0.f : ex2(v.x - top);
                sh_f[head][i] = f;
                sum += v.y * f;
            };
#pragma unroll
            for (int k = 0; k < 4; ++k) add(k * 32 + lane, ml[k]);
            for (int i = 128 + lane; i < parts; i += 32) add(i, part(i));
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            if (lane == 0) {
                sh_done[head0 + head] = make_float2(top == -INFINITY ? 0.f : top, sum == 0.f ? 0.f : 1.f / sum);
                if (blockIdx.x == 0 && A.lse) A.lse[row + head0 + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) / kLog2e;
            }
        }
        __syncthreads();
        if (blockIdx.x == 0)
            for (int i = tid; i < heads * (D / 2); i += kJoinThreads) {
                const int head = i / (D / 2), d = i % (D / 2) * 2;
                float2 acc = make_float2(0.f, 0.f);
#pragma unroll 8
                for (int k = 0; k < parts; ++k) {
                    const float2 t = *reinterpret_cast<const float2 *>(A.part_o + (slot(k) * HB + head) * D + d);
                    acc.x += t.x * sh_f[head][k]; acc.y += t.y * sh_f[head][k];
                }
                *reinterpret_cast<uint32_t *>(A.out + (row + head0 + head) * D + d) = pack2<DT>(acc.x * sh_done[head0 + head].y, acc.y * sh_done[head0 + head].y);
            }
    }
    if (!A.acc) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int j = j0 + i * kJoinThreads + tid, c = j / CH;
        if (j >= w.n) continue;
        if (!(c < w.c_sink || (c >= w.c_win && c < w.c_win + w.nc - w.c_sink))) { if (j == w.n_old) weight[j] = 0.f; continue; }
        float sum = 0.f;
        for (int gb = 0; gb < A.GB; ++gb) {
            const float *more = sc + ((long long)gb * A.kv.cap + j) * A.GS;
#pragma unroll
            for (int g = 0; g < HB; g += 2) {
                if (g >= A.GS || gb * HB + g >= A.G) break;
                const float2 y = gb == 0 ? x[i][g / 2] : *reinterpret_cast<const float2 *>(more + g);
                // a hidden entry's score is -inf: it receives nothing, from a head whose sum is NaN neither
                if (y.x != -INFINITY) sum += ex2(y.x - sh_done[gb * HB + g].x) * sh_done[gb * HB + g].y;
                if (gb * HB + g + 1 < A.G && y.y != -INFINITY) sum += ex2(y.y - sh_done[gb * HB + g + 1].x) * sh_done[gb * HB + g + 1].y;
            }
        }
        weight[j] = j == w.n_old ? sum : old[i] + sum;
    }
}

struct Layout { int n_cta, NT, GB, GS; size_t o, ml, done, scores, runs, total; };
inline Layout layout_of(int n_cta, int n_seqs, int n_kv_heads, int head_dim, int capacity, int n_q_heads, bool acc) {
    Layout L;
    L.n_cta = n_cta;
    const int G = n_q_heads / n_kv_heads;
    L.NT = G <= 8 ? 1 : 2;
    L.GB = (G + 8 * L.NT - 1) / (8 * L.NT);
    L.GS = G >= 8 * L.NT ? 8 * L.NT : (G + 1) / 2 * 2;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off += si_align_up(bytes, 256); return at; };
    L.o = take((size_t)L.n_cta * 2 * 8 * L.NT * head_dim * 4);
    L.ml = take((size_t)L.n_cta * 2 * 8 * L.NT * 2 * 4);
    L.done = take(acc ? (size_t)n_seqs * n_q_heads * 8 : 0);
    L.scores = take(acc ? (size_t)n_seqs * n_kv_heads * L.GB * capacity * L.GS * 4 : 0);
    L.runs = take((size_t)n_seqs * n_kv_heads * L.GB * 8);
    L.total = off;
    return L;
}

template <int DT, int D, int NT, int CH> int launch_join(const DecodeArgs &A, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at; cfg.numAttrs = 1;
    cfg.stream = st;
    // ranges of 256 keys while all their CTAs are resident at once (three per SM), else of 1024: the start of a CTA costs more
    // than its keys (24 x 2 rows of 2112: 20.7 against 22.6 us a call; 32 x 8 rows of 8192: 130 against 116)
    const long long items = (long long)A.kv.H * A.kv.B;
    const bool few = items * ((A.kv.cap + kJoinThreads - 1) / kJoinThreads) <= 3ll * si_sm_count();
    const int keys = few ? kJoinThreads : (NT == 1 ? 4 : 2) * kJoinThreads;
    cfg.gridDim = dim3(A.acc ? (A.kv.cap + keys - 1) / keys : 1, A.kv.H, A.kv.B);
    cfg.blockDim = dim3(kJoinThreads);
    if (few) SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, decode_join_kernel<DT, D, NT, CH, 1>, A));
    else SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, decode_join_kernel<DT, D, NT, CH, NT == 1 ? 4 : 2>, A));
    return SI_OK;
}

}  // namespace
