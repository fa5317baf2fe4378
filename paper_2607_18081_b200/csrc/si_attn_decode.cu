// Single-token attention over the key/value cache.
//
//   out_q = sum_j p_qj v_j,  p_q = softmax over the visible entries j of scale q . k_j,   q = the G query heads of a key head
//
// Bound by HBM: every visible key and value is read once (once per 16 heads where G is larger; in a cache with positions every
// one, visible or not: a chunk's positions come beside its keys), G flops per byte.  So the kernel is a stream: each warp keeps
// two chunks of 4 KB of keys and 4 KB of values in flight (cp.async into a ring of its own, 128 KB per SM) while it works
// on a third (three in flight: 2 % slower).  The G heads make the second dimension of two small matrix products per chunk,
//   S^T [keys x heads] = K Q^T        O^T [head_dim x heads] += V^T P^T,
// with the keys on the long side of the m16n8k16 fragment, so that eight heads fill it (heads-first would waste half of
// it), K and V come from shared memory by ldmatrix as they lie there, and P^T gets from the accumulator layout to the
// operand layout by a transposing register move.  At 23 bytes per SM and clock the warp-level products are a tenth busy:
// a tcgen05 tile of 128 rows would be filled with G of them and gains nothing.
//
// Work is split in chunks, not in sequences: the chunks of all (sequence, head) items in one row, cut into equal runs, one
// per CTA, whatever the lengths.  An item that crosses CTAs leaves partial sums (one maximum, one sum and head_dim fp32
// values per head and CTA) that a second kernel joins in the order of the CTAs -- no atomics, the same bits every time.
// Roundings below 32 bits: p to the cache's type for the product with V (the warp-level product takes both operands in one
// 16-bit type), the result once; everything else is fp32.
// With weights wanted the scores go to the workspace (4 bytes per head beside 4 * head_dim bytes per key) and the second
// kernel, which knows the sums, adds exp(score - maximum) / sum.
#include "si_kv.cuh"
#include "si_tc.cuh"

namespace {

// Two CTAs of four warps per SM rather than one of eight: while one joins its warps' sums at the end of a sequence the other
// streams (batch of 32 ragged caches with weights 106 -> 105 us, 24 evicted caches of 2000 21.2 -> 19.7).  More runs than CTAs
// that are resident (3 or 4 per SM) even out the SMs' shares of the bandwidth, but cost as much in starts and parts.
constexpr int kWarps = 4, kThreads = kWarps * 32, kPerSm = 2;
constexpr int kJoinWarps = 8, kJoinThreads = kJoinWarps * 32;
constexpr int kStages = 3;
constexpr int kMaxParts = 608;             // CTAs of the main kernel at most
constexpr int kSecondSlot = 1 << 30;       // in the table of runs: the item's first part is in the second slot of its CTA
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.f;               // the running maximum moves only when a score exceeds it by 2^8: p stays below 2^8, exact to fp32 all the same

template <int D, int NT> struct Cfg {
    static constexpr int CH = 2048 / D;                  // keys per chunk: 4 KB of keys, 4 KB of values
    static constexpr int kStage = 8192 + 128;            // ... and the entries' positions; a multiple of 128 (swizzle)
    static constexpr int kRow = D + 4;                   // padded row of the merge buffer: conflict-free fragment writes
    static constexpr int kMerge = 8 * kRow;              // floats per warp: eight heads at a time
    static constexpr int kSmem = kWarps * kStages * kStage + kWarps / 2 * kMerge * 4 + kWarps * 8 * NT * 2 * 4;
};

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
template <int D> __device__ __forceinline__ SeqWork seq_work(const DecodeArgs &A, int b, int32_t *status) {
    constexpr int CH = 2048 / D;
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
__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
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
template <int D> __device__ __forceinline__ bool next_item(const DecodeArgs &A, Cursor &c) {   // false: past the last one
    c.start += c.w.nc;
    if (++c.hh < A.kv.H * A.GB && c.w.nc > 0) return true;
    c.hh = 0;
    do {
        if (++c.b >= A.kv.B) { c.w.nc = 0; return false; }
        c.w = seq_work<D>(A, c.b, nullptr);
    } while (c.w.nc == 0);
    return true;
}

// Number of chunks of all items; the first chunk of this CTA's run is at `at` on return (of all threads, if there is one).  Thread t
// of the block stands for sequences t * per ..; the one that holds the run's first chunk looks it up.
struct Run { int g0, g1, per; bool empty; };
template <int D> __device__ __forceinline__ Run find_run(const DecodeArgs &A, Cursor *at, int *sh, int32_t *status) {
    const int tid = threadIdx.x, share = (A.kv.B + kThreads - 1) / kThreads, items = A.kv.H * A.GB;
    const int b0 = min(A.kv.B, tid * share), b1 = min(A.kv.B, b0 + share);
    int sum = 0;
    bool empty = false;
    Cursor c;
    for (int b = b0; b < b1; ++b) {
        c.w = seq_work<D>(A, b, status);
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
        if (share > 1) c.w = seq_work<D>(A, b0, nullptr);    // with one sequence per thread it is at hand
        while (start + c.w.nc * items <= r.g0) { start += c.w.nc * items; c.w = seq_work<D>(A, ++c.b, nullptr); }
        c.hh = (r.g0 - start) / c.w.nc;
        c.start = start + c.hh * c.w.nc;
        *at = c;
    }
    r.empty = __syncthreads_or(empty);                       // some sequence has nothing to see
    return r;
}

// The queries of an item as B operands: head = lane / 4, two neighbouring elements per register.
template <int D, int NT> __device__ __forceinline__ void load_q(const DecodeArgs &A, int b, int hh, uint32_t (&qf)[NT][D / 16][2]) {
    const int lane = threadIdx.x & 31, h = hh / A.GB, head0 = hh % A.GB * 8 * NT, heads = min(8 * NT, A.G - head0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int head = nt * 8 + (lane >> 2);
        const uint16_t *q = A.q + b * A.q_ss + (long long)(h * A.G + head0 + (head < heads ? head : 0)) * D + 2 * (lane & 3);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            qf[nt][s][0] = head < heads ? *reinterpret_cast<const uint32_t *>(q + s * 16) : 0u;
            qf[nt][s][1] = head < heads ? *reinterpret_cast<const uint32_t *>(q + s * 16 + 8) : 0u;
        }
    }
}

template <int DT, int D, int NT>
__global__ void __launch_bounds__(kThreads, kPerSm) decode_kernel(const DecodeArgs A) {
    using C = Cfg<D, NT>;
    constexpr int CH = C::CH, HB = 8 * NT, PIECES = D / 8, SUB = CH / 16;
    extern __shared__ __align__(128) char smem[];
    __shared__ int sh_scan[kThreads / 32 + 1];
    __shared__ Cursor sh_at;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    char *ring = smem + warp * kStages * C::kStage;
    float *merge_o = (float *)(smem + kWarps * kStages * C::kStage);
    float *ml = merge_o + kWarps / 2 * C::kMerge;
    si_tc::pdl_wait();                     // a programmatic dependent too: its launch runs beside the end of the kernel before it
    si_tc::pdl_launch();
    // keys and values pass through L2 once; the scores stay there for the joining kernel
    uint64_t once, stay;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(once));
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(stay));

    // this CTA's run of chunks
    const Run run = find_run<D>(A, &sh_at, sh_scan, blockIdx.x == 0 ? A.status : nullptr);
    const int per = run.per, g0 = run.g0, g1 = run.g1;
    Cursor cons = sh_at;

    // ---- loader side: chunk ids g0 + warp, + kWarps, ...
    Cursor load = cons;
    int load_id = g0 + warp;
    int load_stage = 0;
    const uint32_t ring_addr = si_tc::smem_u32(ring);
    const int load_r = lane / PIECES, load_c = lane % PIECES * 8;
    const uint32_t load_at = load_r * (D * 2) + (((lane % PIECES) & 8) << 4) + (((lane ^ load_r) & 7) << 4);
    auto issue = [&]() {
        if (load_id < g1) {
            while (load_id >= load.start + load.w.nc) next_item<D>(A, load);
            const int t = load_id - load.start, c = t < load.w.c_sink ? t : load.w.c_win + t - load.w.c_sink;
            const int h = load.hh / A.GB, j0 = c * CH;
            const uint32_t kdst = ring_addr + load_stage * C::kStage;
            // row r of the chunk, 16-byte piece c of it, lies at r * 2 D + ((c ^ r) & 7) * 16 (+ 128 for c >= 8): the eight
            // rows of an ldmatrix tile are then in eight different banks groups.  A lane loads the same piece of rows r0, r0 + 32 / PIECES, ..
            const uint32_t at = (kdst + load_at);
            const long long step = (32 / PIECES) * A.kv.rs;
            if (j0 + CH <= min(load.w.n, load.w.n_old)) {
                const uint16_t *ks = A.kv.k + A.kv.row(load.b, h, j0 + load_r) + load_c, *vs = A.kv.v + (ks - A.kv.k);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t to = (at ^ ((i * (32 / PIECES) & 7) << 4)) + i * 512;
                    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(to), "l"(ks), "l"(once) : "memory");
                    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(to + 4096), "l"(vs), "l"(once) : "memory");
                    ks += step; vs += step;
                }
            } else {
#pragma unroll 1
                for (int i = 0; i < 8; ++i) {
                    const int j = j0 + load_r + i * (32 / PIECES);
                    const bool fresh = j == load.w.n_old;
                    const long long off = fresh ? load.b * A.new_ss + (long long)h * D + load_c : A.kv.row(load.b, h, j < load.w.n ? j : 0) + load_c;
                    const uint16_t *ks = (fresh ? A.kn : A.kv.k) + off, *vs = (fresh ? A.vn : A.kv.v) + off;
                    const int bytes = j < load.w.n ? 16 : 0;     // past the end: zeros, nothing is read
                    const uint32_t to = (at ^ ((i * (32 / PIECES) & 7) << 4)) + i * 512;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(ks), "r"(bytes) : "memory");
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + 4096), "l"(vs), "r"(bytes) : "memory");
                }
            }
            if (A.kv.pos && lane < CH) {
                const int j = j0 + lane;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(kdst + 8192 + lane * 4),
                             "l"(A.kv.pos + A.kv.meta(load.b, h) + (j < load.w.n ? j : 0)), "r"(j < load.w.n ? 4 : 0) : "memory");
            }
            load_id += kWarps;
            load_stage = load_stage + 1 == kStages ? 0 : load_stage + 1;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    issue();
    issue();

    // ---- consumer side
    int id = g0 + warp;
    int stage = 0;
    bool first_segment = true;
    uint32_t qf[NT][D / 16][2];
    if (g0 < g1) load_q<D, NT>(A, cons.b, cons.hh, qf);
    // A new entry is stored for later calls by the warp that works on it.  One that its query does not see (entries without
    // positions, and a query position given that lies before the entry or a window behind it) is stored here.
    if (A.kn && A.q_pos && !A.kv.pos)
        for (int r = blockIdx.x; r < A.kv.B * A.kv.H; r += gridDim.x) {
            const int b = r / A.kv.H, h = r % A.kv.H;
            const SeqWork w = seq_work<D>(A, b, nullptr);
            if (w.n_old == INT_MAX || si_visible(w.n_old, w.s, w.lo, A.n_sink)) continue;
            const long long to = A.kv.row(b, h, w.n_old), from = b * A.new_ss + (long long)h * D;
            if (tid < PIECES) *reinterpret_cast<uint4 *>(A.kv.k + to + tid * 8) = *reinterpret_cast<const uint4 *>(A.kn + from + tid * 8);
            else if (tid < 2 * PIECES) *reinterpret_cast<uint4 *>(A.kv.v + to + (tid - PIECES) * 8) = *reinterpret_cast<const uint4 *>(A.vn + from + (tid - PIECES) * 8);
        }
    // sequences without a visible entry have no chunk: their rows are zero
    if (run.empty)
        for (int b = blockIdx.x; b < A.kv.B; b += gridDim.x) {
            if (seq_work<D>(A, b, nullptr).nc) continue;
            for (int i = tid; i < A.Hq * D; i += kThreads) A.out[(long long)b * A.Hq * D + i] = 0;
            if (A.lse) for (int i = tid; i < A.Hq; i += kThreads) A.lse[(long long)b * A.Hq + i] = -INFINITY;
        }
    if (g0 >= g1) return;
    while (true) {
        const int seg_end = min(g1, cons.start + cons.w.nc);
        const int h = cons.hh / A.GB, gb = cons.hh % A.GB, head0 = gb * HB, heads = min(HB, A.G - head0);
        const SeqWork w = cons.w;
        float o[NT][D / 16][4] = {};
        float m[NT][2], base[NT][2], l[NT][2];      // base: the maximum, 0 while there is none
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) { m[nt][0] = m[nt][1] = -INFINITY; base[nt][0] = base[nt][1] = l[nt][0] = l[nt][1] = 0.f; }
        for (; id < seg_end; id += kWarps) {
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncwarp();
            issue();
            const uint32_t kbase = ring_addr + stage * C::kStage, vbase = kbase + 4096;
            const int t = id - cons.start, j0 = (t < w.c_sink ? t : w.c_win + t - w.c_sink) * CH;
            // which keys of the chunk are visible; the values of the others must not meet the product (0 * NaN)
            uint32_t vis;
            {
                const int j = j0 + lane;
                int p = j;
                if (A.kv.pos) p = j == w.n_old ? w.s : *reinterpret_cast<const int *>(ring + stage * C::kStage + 8192 + (lane & (CH - 1)) * 4);
                vis = __ballot_sync(0xFFFFFFFFu, lane < CH && j < w.n && si_visible(p, w.s, w.lo, A.n_sink));
            }
            constexpr uint32_t kAll = CH == 32 ? 0xFFFFFFFFu : (1u << (CH & 31)) - 1;
            if (vis != kAll) {
                for (int i = lane; i < CH * PIECES; i += 32)
                    if (!(vis >> (i / PIECES) & 1)) *reinterpret_cast<uint4 *>(ring + stage * C::kStage + 4096 + i * 16) = make_uint4(0, 0, 0, 0);
                __syncwarp();
            }
            if (w.n_old - j0 < CH && w.n_old >= j0 && gb == 0 && (vis >> (w.n_old - j0) & 1)) {       // the new entry, out of the stage
                const int r = w.n_old - j0, piece = lane % PIECES, at = r * (D * 2) + ((piece & 8) << 4) + (((piece ^ r) & 7) << 4);
                const char *st = ring + stage * C::kStage + at;
                const long long to = A.kv.row(cons.b, h, w.n_old) + piece * 8;
                if (lane < PIECES) *reinterpret_cast<uint4 *>(A.kv.k + to) = *reinterpret_cast<const uint4 *>(st);
                if (lane >= 32 - PIECES) *reinterpret_cast<uint4 *>(A.kv.v + to) = *reinterpret_cast<const uint4 *>(st + 4096);
                if (A.kv.pos && lane == 0) A.kv.pos[A.kv.meta(cons.b, h) + w.n_old] = w.s;
            }
            float x[SUB][NT][4] = {};
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                const uint32_t ka = kbase + u * 16 * D * 2 + (lane & 15) * (D * 2) + (((lane >> 4 ^ lane) & 7) << 4);
#pragma unroll
                for (int s = 0; s < D / 16; ++s) {
                    uint32_t a[4];
                    ldm4(a, (ka ^ ((2 * s & 7) << 4)) + (s >> 2) * 128);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma<DT>(x[u][nt], a, qf[nt][s][0], qf[nt][s][1]);
                }
            }
            bool grow = false;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[u][nt][e] *= A.scale2;
            if (vis != kAll) {
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!(vis >> (u * 16 + (lane >> 2) + (e >> 1) * 8) & 1)) x[u][nt][e] = -INFINITY;
            }
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) grow |= x[u][nt][e] > m[nt][e & 1] + kLazy;
            if (A.acc) {
                float *sc = A.scores + ((((long long)cons.b * A.kv.H + h) * A.GB + gb) * A.kv.cap + j0) * A.GS;
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const int key = u * 16 + (lane >> 2) + (e >> 1) * 8, head = nt * 8 + 2 * (lane & 3);
                            if (head < A.GS && j0 + key < w.n)
                                asm volatile("st.global.L2::cache_hint.v2.f32 [%0], {%1, %2}, %3;"
                                             ::"l"(sc + (long long)key * A.GS + head), "f"(x[u][nt][e]), "f"(x[u][nt][e + 1]), "l"(stay) : "memory");
                        }
            }
            if (__any_sync(0xFFFFFFFFu, grow)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float mx = m[nt][c];
#pragma unroll
                        for (int u = 0; u < SUB; ++u) mx = fmaxf(mx, fmaxf(x[u][nt][c], x[u][nt][c + 2]));
                        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 16));
                        const float f = mx == -INFINITY ? 1.f : ex2(m[nt][c] - mx);
                        m[nt][c] = mx;
                        base[nt][c] = mx == -INFINITY ? 0.f : mx;
                        l[nt][c] *= f;
#pragma unroll
                        for (int s = 0; s < D / 16; ++s) { o[nt][s][c] *= f; o[nt][s][c + 2] *= f; }
                    }
            }
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                uint32_t pb[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[u][nt][e] = ex2(x[u][nt][e] - base[nt][e & 1]);
                        l[nt][e & 1] += x[u][nt][e];
                    }
                    pb[nt][0] = mov_trans(pack2<DT>(x[u][nt][0], x[u][nt][1]));
                    pb[nt][1] = mov_trans(pack2<DT>(x[u][nt][2], x[u][nt][3]));
                }
                const uint32_t va = vbase + u * 16 * D * 2 + ((lane & 7) + ((lane >> 4) << 3)) * (D * 2) + ((((lane >> 3 & 1) ^ lane) & 7) << 4);
#pragma unroll
                for (int s = 0; s < D / 16; ++s) {
                    uint32_t a[4];
                    ldm4t(a, (va ^ ((2 * s & 7) << 4)) + (s >> 2) * 128);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma<DT>(o[nt][s], a, pb[nt][0], pb[nt][1]);
                }
            }
            __syncwarp();                      // the stage may be loaded again
            stage = stage + 1 == kStages ? 0 : stage + 1;
        }
        // the next item's queries are on their way while the warps are joined
        const Cursor seg = cons;
        if (seg_end < g1) {
            next_item<D>(A, cons);
            load_q<D, NT>(A, cons.b, cons.hh, qf);
        }
        // the CTAs of this item, for the joining kernel: written by the one that has its first chunk
        if (tid == 0 && seg.start >= g0)
            A.runs[(long long)seg.b * A.kv.H * A.GB + seg.hh] = make_int2(seg.start / per | (first_segment ? 0 : kSecondSlot), (seg.start + w.nc - 1) / per);
        // ---- the segment's warps joined: rows scaled to the common maximum, summed in warp order
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                l[nt][c] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][c], 4);
                l[nt][c] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][c], 8);
                l[nt][c] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][c], 16);
                if (lane < 4) {
                    ml[(warp * HB + nt * 8 + 2 * lane + c) * 2] = m[nt][c];
                    ml[(warp * HB + nt * 8 + 2 * lane + c) * 2 + 1] = l[nt][c];
                }
            }
        __syncthreads();
        const bool whole = seg.start >= g0 && seg.start + w.nc <= g1;
        float *po = A.part_o + ((long long)blockIdx.x * 2 + (first_segment ? 0 : 1)) * HB * D;
        float *pml = A.part_ml + ((long long)blockIdx.x * 2 + (first_segment ? 0 : 1)) * HB * 2;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            // eight heads at a time: the upper half of the warps through the buffer to the lower half, those to the threads that finish
            float f[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int head = nt * 8 + 2 * (lane & 3) + c;
                float top = -INFINITY;
#pragma unroll
                for (int v = 0; v < kWarps; ++v) top = fmaxf(top, ml[(v * HB + head) * 2]);
                f[c] = m[nt][c] == -INFINITY ? 0.f : ex2(m[nt][c] - top);
            }
            float *mine = merge_o + (warp % (kWarps / 2)) * C::kMerge + 2 * (lane & 3) * C::kRow + (lane >> 2);
#pragma unroll
            for (int s = 0; s < D / 16; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][s][e] *= f[e & 1];
            if (warp >= kWarps / 2) {
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e) mine[(e & 1) * C::kRow + s * 16 + (e >> 1) * 8] = o[nt][s][e];
            }
            __syncthreads();
            if (warp < kWarps / 2) {
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e) mine[(e & 1) * C::kRow + s * 16 + (e >> 1) * 8] += o[nt][s][e];
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
                    const float mv = ml[(v * HB + head) * 2];
                    sum += ml[(v * HB + head) * 2 + 1] * (mv == -INFINITY ? 1.f : ex2(mv - top));     // without a maximum: 0, or NaN (NaN scores only)
                }
#pragma unroll
                for (int v = 0; v < kWarps / 2; ++v) {
                    const float2 t = *reinterpret_cast<const float2 *>(merge_o + v * C::kMerge + hd * C::kRow + d);
                    acc.x += t.x; acc.y += t.y;
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
    }
}

// Joins the parts of items that crossed CTAs and, where weights are wanted, adds them up.  One CTA per (sequence, key head)
// and range of U * 256 keys; the first range's writes the output.  A chain of short dependent loads: everything that does not
// depend on another load is asked for first (scores and weights beyond the length too: the memory is there, the values are
// not used).  At most 80 registers, so that the CTAs become resident beside the main kernel's and wait there for its end.
template <int DT, int D, int NT, int U>
__global__ void __launch_bounds__(kJoinThreads, 3) decode_join_kernel(const DecodeArgs A) {
    constexpr int HB = 8 * NT, CH = 2048 / D;
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
    const SeqWork w = seq_work<D>(A, b, nullptr);
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
Layout layout_of(const si_kv_t *kv, int n_q_heads, bool acc) {
    Layout L;
    L.n_cta = kPerSm * si_sm_count() < kMaxParts ? kPerSm * si_sm_count() : kMaxParts;
    const int G = n_q_heads / kv->n_kv_heads;
    L.NT = G <= 8 ? 1 : 2;
    L.GB = (G + 8 * L.NT - 1) / (8 * L.NT);
    L.GS = G >= 8 * L.NT ? 8 * L.NT : (G + 1) / 2 * 2;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off += si_align_up(bytes, 256); return at; };
    L.o = take((size_t)L.n_cta * 2 * 8 * L.NT * kv->head_dim * 4);
    L.ml = take((size_t)L.n_cta * 2 * 8 * L.NT * 2 * 4);
    L.done = take(acc ? (size_t)kv->n_seqs * n_q_heads * 8 : 0);
    L.scores = take(acc ? (size_t)kv->n_seqs * kv->n_kv_heads * L.GB * kv->capacity * L.GS * 4 : 0);
    L.runs = take((size_t)kv->n_seqs * kv->n_kv_heads * L.GB * 8);
    L.total = off;
    return L;
}

template <int DT, int D, int NT> int launch(const DecodeArgs &A, cudaStream_t st) {
    static std::atomic<unsigned long long> allowed{0};
    const int rc = si_allow_smem(decode_kernel<DT, D, NT>, (Cfg<D, NT>::kSmem), allowed);
    if (rc) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at; cfg.numAttrs = 1;
    cfg.gridDim = dim3(A.n_cta);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Cfg<D, NT>::kSmem;
    cfg.stream = st;
    SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, decode_kernel<DT, D, NT>, A));
    // ranges of 256 keys while all their CTAs are resident at once (three per SM), else of 1024: the start of a CTA costs more
    // than its keys (24 x 2 rows of 2112: 20.7 against 22.6 us a call; 32 x 8 rows of 8192: 130 against 116)
    const long long items = (long long)A.kv.H * A.kv.B;
    const bool few = items * ((A.kv.cap + kJoinThreads - 1) / kJoinThreads) <= 3ll * si_sm_count();
    const int keys = few ? kJoinThreads : (NT == 1 ? 4 : 2) * kJoinThreads;
    cfg.gridDim = dim3(A.acc ? (A.kv.cap + keys - 1) / keys : 1, A.kv.H, A.kv.B);
    cfg.blockDim = dim3(kJoinThreads);
    cfg.dynamicSmemBytes = 0;
    if (few) SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, decode_join_kernel<DT, D, NT, 1>, A));
    else SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, decode_join_kernel<DT, D, NT, NT == 1 ? 4 : 2>, A));
    return SI_OK;
}
template <int DT> int launch_t(const DecodeArgs &A, int NT, cudaStream_t st) {
    if (A.kv.D == 128) return NT == 1 ? launch<DT, 128, 1>(A, st) : launch<DT, 128, 2>(A, st);
    return NT == 1 ? launch<DT, 64, 1>(A, st) : launch<DT, 64, 2>(A, st);
}

}  // namespace

size_t si_attn_decode_ws_bytes(const si_kv_t *kv, int n_q_heads) { return layout_of(kv, n_q_heads, kv->weight != nullptr).total; }

extern "C" int si_attn_decode(const si_kv_t *kv, const void *q, long long q_seq_stride, int n_q_heads, const int32_t *q_pos,
                              const void *k_new, const void *v_new, long long new_seq_stride, int window, int n_sink,
                              float scale, void *out, float *lse, unsigned flags, void *workspace, size_t ws_bytes,
                              int32_t *status_dev, void *stream) {
    const int rc = si_attn_check(kv, n_q_heads, window, n_sink, scale);
    if (rc) return rc;
    if (flags & ~(unsigned)SI_FLAG_ACC_WEIGHT) return SI_ERR_INVALID_ARG;
    if (kv->n_seqs == 0) return SI_OK;
    const int acc = (flags & SI_FLAG_ACC_WEIGHT) != 0;
    if (!q || !out || q_seq_stride < 0 || !k_new != !v_new || new_seq_stride < 0) return SI_ERR_INVALID_ARG;
    if ((kv->pos && !q_pos) || (acc && !kv->weight) || (k_new && si_kv_shared(kv))) return SI_ERR_INVALID_ARG;
    if (!si_aligned16(q) || !si_aligned16(out) || !si_aligned16(k_new) || !si_aligned16(v_new) || !si_aligned4(q_pos, lse, status_dev) ||
        ((q_seq_stride | new_seq_stride) & 7))
        return SI_ERR_ALIGNMENT;
    const Layout L = layout_of(kv, n_q_heads, acc);
    // chunks are numbered in 32 bits: 2^31 of them are 16 TB of keys and values unless sequences share memory by zero strides
    if ((double)kv->n_seqs * kv->n_kv_heads * L.GB * (kv->capacity / (2048 / kv->head_dim) + 2) > 2.0e9) return SI_ERR_TOO_LARGE;
    if (ws_bytes < L.total) return SI_ERR_NOMEM;
    if (!workspace) return SI_ERR_INVALID_ARG;
    if ((uintptr_t)workspace & 255) return SI_ERR_ALIGNMENT;
    char *ws = (char *)workspace;
    const DecodeArgs A{si_kv_view_of(kv), (const uint16_t *)q, (const uint16_t *)k_new, (const uint16_t *)v_new, q_pos, q_seq_stride,
                       new_seq_stride, n_q_heads, n_q_heads / kv->n_kv_heads, L.GB, L.GS, window, n_sink, scale * kLog2e,
                       (uint16_t *)out, lse, status_dev, acc, L.n_cta, (float *)(ws + L.o), (float *)(ws + L.ml),
                       (float2 *)(ws + L.done), (float *)(ws + L.scores), (int2 *)(ws + L.runs)};
    si_mt_forget();
    return kv->dtype == SI_BF16 ? launch_t<SI_BF16>(A, L.NT, (cudaStream_t)stream) : launch_t<SI_F16>(A, L.NT, (cudaStream_t)stream);
}
