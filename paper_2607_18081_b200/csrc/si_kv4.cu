// The key/value cache in 4 bits: quantising entries as they are stored, reading them back, eviction.  (Layout and format: si_kv4.cuh.)
//
// An entry is 4 D bytes in 16 bits and D + 8 D / group in 4.  Measured: 65000 entries of eight heads of 128 read back in 58 us (6.0 TB/s of the
// two sides together: bound by HBM); a prompt of 8192 tokens stored in 9 us (4.9 TB/s; the issue slots are two thirds busy, half of it the
// codes, and the warps are a wave and a half); 2048 of 16384 entries of 128 heads moved in 19 us (bound by the latency of scattered
// reads: a value's cell holds its neighbour too, so 256 bytes are read for 160).
#include "si_evict.cuh"
#include "si_tc.cuh"

namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32, kOctet = 8;

template <int DT> __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    if (DT == SI_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Pairs of 16-bit numbers; NaN if either is.
template <int DT> __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
    uint32_t r;
    if (DT == SI_BF16) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <int DT> __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    if (DT == SI_BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

struct StoreArgs {
    si_kv_view src, meta;            // meta: pos, weight, len, capacity of the cache in 4 bits
    si_kv4_view dst;
    const int32_t *first_pos;
    int32_t *status;
};

// A warp per eight entries, everything it reads asked for at once: 16-byte pieces of rows, eight elements a lane, which make one word
// of a key's codes and two half words of a value's (the two entries of a pair exchange a half each).  A warp's words of a store are
// 128 contiguous bytes, in the tile's order.  (A warp per tile, with the tile put together in shared memory, has a quarter of the
// loads in flight: 8192 tokens of eight heads 20 us instead of 12; 9 since the steps of the eight groups that a lane takes part in
// are dealt to the groups' lanes.)
template <int DT, int D, int NG>
__global__ void __launch_bounds__(kThreads) store_kernel(const StoreArgs A) {
    using T = si_tile4<D, NG>;
    constexpr int L = D / 8, ROWS = 32 / L, N = kOctet / ROWS, GL = D / NG / 8;     // lanes of a row, rows of a warp at a time, times, lanes of a group
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = blockIdx.x % A.src.H, b = blockIdx.z;
    const long long block = blockIdx.x / A.src.H;          // the heads of a token side by side in time: in a token-major source they share DRAM pages
    si_tc::pdl_wait();
    si_tc::pdl_launch();
    const bool tell = blockIdx.x == 0 && threadIdx.x == 0;
    const int start = si_kv_len(A.meta, b, tell ? A.status : nullptr);
    int n = si_kv_len(A.src, b, tell ? A.status : nullptr);
    if (n > A.meta.cap - start) { if (tell) si_report(A.status, SI_ERR_OUT_OF_RANGE); n = A.meta.cap - start; }
    const long long e0 = (start / kOctet + block * kWarps + warp) * kOctet;
    if (n <= 0 || e0 >= start + n) return;
    const int r0 = max(0, start - (int)e0), r1 = min(kOctet, start + n - (int)e0);     // rows of the eight that are stored
    const int c = lane % L, w = c / 4, t = c % 4, sub = lane / L;
    uint4 raw[N][2];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = i * ROWS + sub;
        const bool in = r >= r0 && r < r1;
        const long long at = A.src.row(b, h, in ? (int)e0 + r - start : 0) + c * 8;
        raw[i][0] = in ? __ldcs(reinterpret_cast<const uint4 *>(A.src.k + at)) : make_uint4(0, 0, 0, 0);
        raw[i][1] = in ? __ldcs(reinterpret_cast<const uint4 *>(A.src.v + at)) : make_uint4(0, 0, 0, 0);
    }
    // the eight entries' part of the tile, and of the steps
    uint8_t *tile = A.dst.row(b, h) + e0 / kTileEntries * T::kBytes + (int)(e0 % kTileEntries) * (D / 2);
    uint8_t *steps = A.dst.row(b, h) + e0 / kTileEntries * T::kBytes + (int)(e0 % kTileEntries) * NG * 4;
    // The extremes of every group, of keys then of values, are with all of its lanes; its step and reciprocal are found by one of them.
    constexpr int I = 2 * N, CALLS = (I + GL - 1) / GL;
    uint32_t lo2[I], hi2[I];
#pragma unroll
    for (int k = 0; k < I; ++k) {
        const uint4 u = raw[k % N][k / N];
        lo2[k] = min2<DT>(min2<DT>(u.x, u.y), min2<DT>(u.z, u.w));
        hi2[k] = max2<DT>(max2<DT>(u.x, u.y), max2<DT>(u.z, u.w));
#pragma unroll
        for (int o = 1; o < GL; o <<= 1) {
            lo2[k] = min2<DT>(lo2[k], __shfl_xor_sync(0xFFFFFFFFu, lo2[k], o));
            hi2[k] = max2<DT>(hi2[k], __shfl_xor_sync(0xFFFFFFFFu, hi2[k], o));
        }
    }
    uint32_t par[CALLS];
    float inverse[CALLS];
#pragma unroll
    for (int q = 0; q < CALLS; ++q) {
        const int mine = q * GL + c % GL;
        uint32_t lo = lo2[0], hi = hi2[0];
#pragma unroll
        for (int k = 1; k < I; ++k) if (mine == k) { lo = lo2[k]; hi = hi2[k]; }
        par[q] = si_q4::group_word<DT>(si_q4::min_nan(si_cvt<DT>::lo(lo), si_cvt<DT>::hi(lo)), si_q4::max_nan(si_cvt<DT>::lo(hi), si_cvt<DT>::hi(hi)), &inverse[q]);
        const int row = mine % N * ROWS + sub;
        if (mine < I && row >= r0 && row < r1)
            *reinterpret_cast<uint32_t *>(steps + (mine / N ? T::kValuePar : T::kKeyPar) + (row * NG + T::place_of(c / GL)) * 4) = par[q];
    }
#pragma unroll
    for (int k = 0; k < I; ++k) {
        const int i = k % N, row = i * ROWS + sub, other_row = row ^ 1, from = lane / GL * GL + k % GL;
        const bool in = row >= r0 && row < r1, both = in && other_row >= r0 && other_row < r1;
        const float low = si_cvt<DT>::lo(__shfl_sync(0xFFFFFFFFu, par[k / GL], from)), inv = __shfl_sync(0xFFFFFFFFu, inverse[k / GL], from);
        const uint32_t u[4] = {raw[i][k / N].x, raw[i][k / N].y, raw[i][k / N].z, raw[i][k / N].w};
        // a code's bits lie above those of 2^23 * 1.5, whose sum over eight places is taken off at the end
        auto code = [&](int e) { return si_q4::code_bits(e & 1 ? si_cvt<DT>::hi(u[e / 2]) : si_cvt<DT>::lo(u[e / 2]), low, inv); };
        auto joined = [&](int k7, int k6, int k5, int k4, int k3, int k2, int k1, int k0) {
            uint32_t x = code(k7);
            x = x * 16 + code(k6); x = x * 16 + code(k5); x = x * 16 + code(k4);
            x = x * 16 + code(k3); x = x * 16 + code(k2); x = x * 16 + code(k1);
            return x * 16 + code(k0) - 0x3F400000u;
        };
        if (k < N) {
            const uint32_t word = joined(7, 5, 3, 1, 6, 4, 2, 0);
            if (in) *reinterpret_cast<uint32_t *>(tile + T::key_word(row, w, t)) = word;
        } else {
            const uint32_t word = joined(7, 6, 5, 4, 3, 2, 1, 0);      // elements 0 .. 3 in the lower half
            const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, word, L);
            if (both) {
                *reinterpret_cast<uint32_t *>(tile + T::value_word(row, w, 2 * t + (row & 1))) = row & 1 ? __byte_perm(other, word, 0x7632) : __byte_perm(word, other, 0x5410);
            } else if (in) {
                *reinterpret_cast<uint16_t *>(tile + T::value_word(row, w, 2 * t) + 2 * (row & 1)) = (uint16_t)word;
                *reinterpret_cast<uint16_t *>(tile + T::value_word(row, w, 2 * t + 1) + 2 * (row & 1)) = (uint16_t)(word >> 16);
            }
        }
    }
    if (lane < r0 || lane >= r1) return;
    const int e = (int)e0 + lane, j = e - start;
    if (A.meta.pos) A.meta.pos[A.meta.meta(b, h) + e] = A.src.pos ? A.src.pos[A.src.meta(b, h) + j] : A.first_pos ? A.first_pos[b] + j : e;
    if (A.meta.weight) A.meta.weight[A.meta.meta(b, h) + e] = A.src.weight ? A.src.weight[A.src.meta(b, h) + j] : 0.f;
}

struct LoadArgs {
    si_kv_view meta, dst;
    si_kv4_view src;
    const int32_t *first;
    int n;
    int32_t *len_out, *status;
};

// m + s c.  The step is rounded up, so that the highest code may stand for a little more than the type holds: the largest number
// then (bf16: a range of 2^94 is far from its end).
template <int DT> __device__ __forceinline__ float value_of(float code, float step, float low) {
    const float x = fmaf(code, step, low);
    return DT == SI_F16 ? si_q4::min_nan(x, 65504.f) : x;
}

// The entries of sequence b that are read back: from *first up to the returned end.
__device__ __forceinline__ int load_span(const LoadArgs &A, int b, int32_t *status, int *first) {
    const int len = si_kv_len(A.meta, b, status), f = A.first ? A.first[b] : 0;
    if (f < 0) si_report(status, SI_ERR_OUT_OF_RANGE);
    *first = max(0, f);
    return *first + min(A.n, max(0, len - *first));
}

// A warp per eight entries, all words asked for at once; a lane makes eight neighbouring elements of a row.
template <int DT, int D, int NG>
__global__ void __launch_bounds__(kThreads) load_kernel(const LoadArgs A) {
    using T = si_tile4<D, NG>;
    constexpr int L = D / 8, ROWS = 32 / L, N = kOctet / ROWS;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = blockIdx.x % A.dst.H, b = blockIdx.z;
    const long long block = blockIdx.x / A.dst.H;
    si_tc::pdl_wait();
    si_tc::pdl_launch();
    const bool tell = blockIdx.x == 0 && threadIdx.x == 0;
    int first;
    const int end = load_span(A, b, tell ? A.status : nullptr, &first);
    if (tell && A.len_out) A.len_out[b] = end - first;
    const long long e0 = (first / kOctet + block * kWarps + warp) * kOctet;
    if (end <= first || e0 >= end) return;
    const int r0 = max(0, first - (int)e0), r1 = min(kOctet, end - (int)e0);
    const uint8_t *from = A.src.row(b, h) + e0 / kTileEntries * T::kBytes;
    const int c = lane % L, w = c / 4, t = c % 4, g = T::place_of(T::group_of(w)), sub = lane / L, in_tile = (int)(e0 % kTileEntries);
    uint32_t kw[N], v0[N], v1[N], kp[N], vp[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {              // the eight entries lie in one tile: all of it is there to be read
        const int r = in_tile + i * ROWS + sub;
        auto word = [&](int at) { return __ldcs(reinterpret_cast<const uint32_t *>(from + at)); };
        kw[i] = word(T::key_word(r, w, t));
        v0[i] = word(T::value_word(r, w, 2 * t)); v1[i] = word(T::value_word(r, w, 2 * t + 1));
        kp[i] = word(T::kKeyPar + (r * NG + g) * 4); vp[i] = word(T::kValuePar + (r * NG + g) * 4);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int row = i * ROWS + sub;
        // codes come as c 2^-24 and 16 c 2^-24
        float2 x[4];
        auto values = [&](uint32_t codes, uint32_t par) {
            const float s = si_cvt<DT>::hi(par), m = si_cvt<DT>::lo(par), s0 = s * 0x1p24f, s1 = s * 0x1p20f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[k] = si_q4::code_pair(k & 1 ? si_q4::high_codes(codes >> 4 * (k & 2)) : si_q4::low_codes(codes >> 4 * (k & 2)));
                x[k].x = value_of<DT>(x[k].x, k & 1 ? s1 : s0, m); x[k].y = value_of<DT>(x[k].y, k & 1 ? s1 : s0, m);
            }
        };
        if (row < r0 || row >= r1) continue;
        const long long at = A.dst.row(b, h, (int)e0 + row - first) + c * 8;
        values(kw[i], kp[i]);
        __stcs(reinterpret_cast<uint4 *>(A.dst.k + at), make_uint4(pack2<DT>(x[0].x, x[0].y), pack2<DT>(x[1].x, x[1].y), pack2<DT>(x[2].x, x[2].y), pack2<DT>(x[3].x, x[3].y)));
        values(__byte_perm(v0[i], v1[i], row & 1 ? 0x7632 : 0x5410), vp[i]);       // elements 0 .. 3 | 4 .. 7
        __stcs(reinterpret_cast<uint4 *>(A.dst.v + at), make_uint4(pack2<DT>(x[0].x, x[1].x), pack2<DT>(x[2].x, x[3].x), pack2<DT>(x[0].y, x[1].y), pack2<DT>(x[2].y, x[3].y)));
    }
    if (lane < r0 || lane >= r1) return;
    const int e = (int)e0 + lane;
    if (A.meta.pos && A.dst.pos) A.dst.pos[A.dst.meta(b, h) + e - first] = A.meta.pos[A.meta.meta(b, h) + e];
    if (A.meta.weight && A.dst.weight) A.dst.weight[A.dst.meta(b, h) + e - first] = A.meta.weight[A.meta.meta(b, h) + e];
}

// Numbers of entries that go where the lengths or the first entries are.
__global__ void load_len_kernel(const LoadArgs A) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= A.dst.B) return;
    int first;
    const int end = load_span(A, b, nullptr, &first);
    A.len_out[b] = end - first;
}

// The kept entries to their slots; nothing to do for an entry that stays.  A warp per sixteen slots, everything asked for before anything is
// written: eight lanes have the values' cells of both sources of a pair of slots (which hold a neighbour each) and put the two halves
// together, four the cells of a key, two the steps of an entry, two its position and weight.  (Sixteen lanes per pair with these
// roles side by side: a warp's lanes part ways, 21 us instead of 19 for 2048 of 16384 entries of 128 heads.)
constexpr int kMoveSlots = 16;                // of a warp
template <int D, int NG>
__global__ void __launch_bounds__(256) move4_kernel(const EvictArgs A) {
    using T = si_tile4<D, NG>;
    constexpr int W = T::W;
    const int h = blockIdx.x % A.src.H, b = blockIdx.z, lane = threadIdx.x % 32;
    const long long row = (long long)b * A.src.H + h, s0 = ((long long)(blockIdx.x / A.src.H) * 8 + threadIdx.x / 32) * kMoveSlots;
    si_tc::pdl_wait();
    si_tc::pdl_launch();
    if (blockIdx.x == 0 && threadIdx.x == 0 && A.len_out) A.len_out[b] = min(si_evict_entries(A, b), A.budget);
    if (s0 >= A.slots) return;
    int mine = -1;                            // the source of slot s0 + lane
    if (lane < kMoveSlots && s0 + lane < A.slots) mine = A.source[row * A.slots + s0 + lane];
    if (A.in_place && mine == s0 + lane) mine = -1;
    if (!__any_sync(0xFFFFFFFFu, mine >= 0)) return;
    const uint8_t *src = A.src4.row(b, h);
    uint8_t *dst = A.dst4.row(b, h) + s0 / kTileEntries * T::kBytes;             // sixteen slots lie in one tile
    const int r0 = (int)(s0 % kTileEntries);
    auto from = [&](int slot) { return __shfl_sync(0xFFFFFFFFu, mine, slot); };
    auto tile_of = [&](int j) { return src + (long long)(j / kTileEntries) * T::kBytes; };
    auto load = [](auto &to, const uint8_t *at) {
        constexpr int N = sizeof(to) / 4;
        if constexpr (N == 4) { const uint4 v = __ldcs(reinterpret_cast<const uint4 *>(at)); to[0] = v.x; to[1] = v.y; to[2] = v.z; to[3] = v.w; }
        else if constexpr (N == 2) { const uint2 v = __ldcs(reinterpret_cast<const uint2 *>(at)); to[0] = v.x; to[1] = v.y; }
        else to[0] = __ldcs(reinterpret_cast<const uint32_t *>(at));
    };
    auto store = [](uint8_t *at, const auto &x) {
        constexpr int N = sizeof(x) / 4;
        if constexpr (N == 4) *reinterpret_cast<uint4 *>(at) = make_uint4(x[0], x[1], x[2], x[3]);
        else if constexpr (N == 2) *reinterpret_cast<uint2 *>(at) = make_uint2(x[0], x[1]);
        else *reinterpret_cast<uint32_t *>(at) = x[0];
    };
    uint32_t even[2][W], odd[2][W], key[2][W], step[NG], word = 0;
    int v0[2], v1[2], k0[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int pair = i * 4 + lane / 8;
        v0[i] = from(2 * pair); v1[i] = from(2 * pair + 1); k0[i] = from(i * 8 + lane / 4);
        if (v0[i] >= 0) load(even[i], tile_of(v0[i]) + T::value_word(v0[i] % kTileEntries, 0, lane % 8));
        if (v1[i] >= 0) load(odd[i], tile_of(v1[i]) + T::value_word(v1[i] % kTileEntries, 0, lane % 8));
        if (k0[i] >= 0) load(key[i], tile_of(k0[i]) + T::key_word(k0[i] % kTileEntries, 0, lane % 4));
    }
    const int p0 = from(lane / 2), m0 = from(lane % 16), par = lane & 1 ? T::kValuePar : T::kKeyPar;
    if (p0 >= 0) load(step, tile_of(p0) + par + p0 % kTileEntries * NG * 4);
    if (m0 >= 0) {
        if (lane >= 16) word = __float_as_uint(A.src.weight[A.src.meta(b, h) + m0]);
        else word = A.src.pos ? A.src.pos[A.src.meta(b, h) + m0] : m0;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint8_t *at = dst + T::value_word(r0 + 2 * (i * 4 + lane / 8), 0, lane % 8);
        uint32_t both[W];
#pragma unroll
        for (int w = 0; w < W; ++w)            // the source's half into the slot's
            both[w] = (v0[i] & 1 ? even[i][w] >> 16 : even[i][w] & 0xFFFFu) | (v1[i] & 1 ? odd[i][w] & 0xFFFF0000u : odd[i][w] << 16);
        if (v0[i] >= 0 && v1[i] >= 0) store(at, both);
        else if (v0[i] >= 0 || v1[i] >= 0)
#pragma unroll
            for (int w = 0; w < W; ++w) reinterpret_cast<uint16_t *>(at)[2 * w + (v0[i] < 0)] = (uint16_t)(v0[i] < 0 ? both[w] >> 16 : both[w]);
        if (k0[i] >= 0) store(dst + T::key_word(r0 + i * 8 + lane / 4, 0, lane % 4), key[i]);
    }
    if (p0 >= 0) store(dst + par + (r0 + lane / 2) * NG * 4, step);
    if (m0 >= 0) {
        const long long to = A.dst.meta(b, h) + s0 + lane % 16;
        if (lane >= 16) A.dst.weight[to] = __uint_as_float(word);
        else A.dst.pos[to] = (int)word;
    }
}

cudaLaunchConfig_t config(dim3 grid, int threads, cudaStream_t st, cudaLaunchAttribute *at) {
    cudaLaunchConfig_t cfg = {};
    at->id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at->val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cfg.attrs = at; cfg.numAttrs = 1;
    return cfg;
}

template <template <int, int, int> class F, typename... P> int by_shape(int dtype, int D, int NG, P... p) {
    if (dtype == SI_BF16) {
        if (D == 128) return NG == 4 ? F<SI_BF16, 128, 4>::go(p...) : F<SI_BF16, 128, 2>::go(p...);
        return NG == 2 ? F<SI_BF16, 64, 2>::go(p...) : F<SI_BF16, 64, 1>::go(p...);
    }
    if (D == 128) return NG == 4 ? F<SI_F16, 128, 4>::go(p...) : F<SI_F16, 128, 2>::go(p...);
    return NG == 2 ? F<SI_F16, 64, 2>::go(p...) : F<SI_F16, 64, 1>::go(p...);
}
template <int DT, int D, int NG> struct Store {
    static int go(cudaLaunchConfig_t *cfg, const StoreArgs *A) { SI_CUDA_TRY(cudaLaunchKernelEx(cfg, store_kernel<DT, D, NG>, *A)); return SI_OK; }
};
template <int DT, int D, int NG> struct Load {
    static int go(cudaLaunchConfig_t *cfg, const LoadArgs *A) { SI_CUDA_TRY(cudaLaunchKernelEx(cfg, load_kernel<DT, D, NG>, *A)); return SI_OK; }
};

template <int DT, int D, int NG> struct Move {
    static int go(cudaLaunchConfig_t *cfg, const EvictArgs *A) { SI_CUDA_TRY(cudaLaunchKernelEx(cfg, move4_kernel<D, NG>, *A)); return SI_OK; }
};

// Blocks that cover n entries, wherever among eight the first one is, for every head.
long long octet_blocks(int n, int heads) { return (((long long)n + kOctet - 2) / kOctet + kWarps) / kWarps * heads; }

bool same_shape(const si_kv_t *a, const si_kv4_t *b) {
    return a->n_seqs == b->n_seqs && a->n_kv_heads == b->n_kv_heads && a->head_dim == b->head_dim && a->dtype == b->dtype;
}

}  // namespace

extern "C" int si_kv4_tile_bytes(int head_dim, int group, size_t *bytes_out) {
    if (!bytes_out) return SI_ERR_INVALID_ARG;
    if ((head_dim != 64 && head_dim != 128) || (group != 32 && group != 64)) return SI_ERR_UNSUPPORTED;
    *bytes_out = si_tile4_bytes(head_dim, group);
    return SI_OK;
}

extern "C" int si_kv4_workspace_bytes(const si_kv4_t *kv, int n_q_heads, size_t *bytes_out) {
    const int rc = si_kv4_check(kv);
    if (rc) return rc;
    if (!bytes_out || n_q_heads < 0 || n_q_heads % kv->n_kv_heads) return SI_ERR_INVALID_ARG;
    if (n_q_heads / kv->n_kv_heads > 128) return SI_ERR_UNSUPPORTED;
    const size_t evict = kv->weight ? si_evict_ws_bytes(kv->n_seqs, kv->n_kv_heads, kv->capacity) : 0, decode = n_q_heads ? si_kv4_attn_decode_ws_bytes(kv, n_q_heads) : 0;
    *bytes_out = evict > decode ? evict : decode;
    return SI_OK;
}

extern "C" int si_kv4_store(const si_kv_t *src, const si_kv4_t *dst, const int32_t *first_pos, int32_t *status_dev, void *stream) {
    int rc = si_kv_check(src);
    if (rc) return rc;
    if ((rc = si_kv4_check(dst))) return rc;
    if (!same_shape(src, dst)) return SI_ERR_INVALID_ARG;
    if (src->n_seqs == 0) return SI_OK;
    if (si_kv4_shared(dst)) return SI_ERR_INVALID_ARG;
    if (!si_aligned4(first_pos, status_dev)) return SI_ERR_ALIGNMENT;
    const StoreArgs A{si_kv_view_of(src), si_kv4_meta_of(dst), si_kv4_view_of(dst), first_pos, status_dev};
    si_mt_forget();
    cudaLaunchAttribute at;
    const long long blocks = octet_blocks(src->capacity < dst->capacity ? src->capacity : dst->capacity, dst->n_kv_heads);
    if (blocks > INT_MAX) return SI_ERR_TOO_LARGE;
    cudaLaunchConfig_t cfg = config(dim3((unsigned)blocks, 1, dst->n_seqs), kThreads, (cudaStream_t)stream, &at);
    return by_shape<Store>(dst->dtype, dst->head_dim, si_kv4_groups(dst), &cfg, &A);
}

extern "C" int si_kv4_load(const si_kv4_t *src, const si_kv_t *dst, const int32_t *first, int n, int32_t *len_out, int32_t *status_dev, void *stream) {
    int rc = si_kv4_check(src);
    if (rc) return rc;
    if ((rc = si_kv_check(dst))) return rc;
    if (!same_shape(dst, src) || n < 0 || n > dst->capacity) return SI_ERR_INVALID_ARG;
    if (src->n_seqs == 0) return SI_OK;
    if (si_kv_shared(dst)) return SI_ERR_INVALID_ARG;
    if (!si_aligned4(first, len_out, status_dev)) return SI_ERR_ALIGNMENT;
    // all blocks read the lengths and the first entries: a result in their place is written behind them
    const bool len_after = len_out && (len_out == src->len || len_out == first);
    for (const int32_t *in : {src->len, first})
        if (len_out && in && len_out != in && len_out < in + src->n_seqs && in < len_out + src->n_seqs) return SI_ERR_INVALID_ARG;
    LoadArgs A{si_kv4_meta_of(src), si_kv_view_of(dst), si_kv4_view_of(src), first, n, len_after ? nullptr : len_out, status_dev};
    si_mt_forget();
    const int most = n < src->capacity ? n : src->capacity;
    cudaLaunchAttribute at;
    const long long blocks = octet_blocks(most, src->n_kv_heads);
    if (blocks > INT_MAX) return SI_ERR_TOO_LARGE;
    cudaLaunchConfig_t cfg = config(dim3((unsigned)blocks, 1, src->n_seqs), kThreads, (cudaStream_t)stream, &at);
    rc = by_shape<Load>(src->dtype, src->head_dim, si_kv4_groups(src), &cfg, &A);
    if (rc || !len_after) return rc;
    A.len_out = len_out;
    load_len_kernel<<<(src->n_seqs + 127) / 128, 128, 0, (cudaStream_t)stream>>>(A);
    SI_CUDA_TRY(cudaGetLastError());
    return SI_OK;
}

extern "C" int si_kv4_evict(const si_kv4_t *src, const si_kv4_t *dst, const int32_t *q_pos, int n_new, int budget, int n_sink, int n_recent,
                            int32_t *kept, int32_t *len_out, void *workspace, size_t ws_bytes, int32_t *status_dev, void *stream) {
    int rc = si_kv4_check(src);
    if (rc) return rc;
    if ((rc = si_kv4_check(dst))) return rc;
    if (budget < 1 || n_new < 0 || n_new > src->capacity || n_sink < 0 || n_recent < 0 || (long long)n_sink + n_recent > budget || budget > dst->capacity) return SI_ERR_INVALID_ARG;
    if (src->n_seqs != dst->n_seqs || src->n_kv_heads != dst->n_kv_heads || src->head_dim != dst->head_dim || src->dtype != dst->dtype ||
        si_kv4_groups(src) != si_kv4_groups(dst)) return SI_ERR_INVALID_ARG;
    if (src->n_seqs == 0) return SI_OK;
    const bool in_place = src->data == dst->data;
    if (!src->weight || !dst->weight || !dst->pos || (src->pos && !q_pos) || (in_place && !src->pos)) return SI_ERR_INVALID_ARG;
    if (in_place && (src->pos != dst->pos || src->weight != dst->weight || src->seq_stride != dst->seq_stride || src->head_stride != dst->head_stride ||
                     src->capacity != dst->capacity)) return SI_ERR_INVALID_ARG;
    if (si_kv4_shared(dst) || (!in_place && (src->weight == dst->weight || src->pos == dst->pos))) return SI_ERR_INVALID_ARG;
    if (!si_aligned4(q_pos, kept, len_out, status_dev)) return SI_ERR_ALIGNMENT;
    if (ws_bytes < si_evict_ws_bytes(src->n_seqs, src->n_kv_heads, src->capacity)) return SI_ERR_NOMEM;
    if (!workspace) return SI_ERR_INVALID_ARG;
    if ((uintptr_t)workspace & 255) return SI_ERR_ALIGNMENT;
    EvictArgs A = si_evict_args(si_kv4_meta_of(src), si_kv4_meta_of(dst), in_place, q_pos, n_new, budget, n_sink, n_recent, kept, len_out, workspace, status_dev);
    if (((long long)A.slots / 128 + 1) * src->n_kv_heads > INT_MAX) return SI_ERR_TOO_LARGE;
    A.src4 = si_kv4_view_of(src); A.dst4 = si_kv4_view_of(dst); A.groups = si_kv4_groups(src);
    si_mt_forget();
    if ((rc = si_evict_select(A, (cudaStream_t)stream)) || A.move_here) return rc;
    cudaLaunchAttribute at;
    constexpr int kPerBlock = 8 * kMoveSlots;
    const long long blocks = ((long long)A.slots + kPerBlock - 1) / kPerBlock * src->n_kv_heads;
    cudaLaunchConfig_t cfg = config(dim3((unsigned)blocks, 1, src->n_seqs), 256, (cudaStream_t)stream, &at);
    return by_shape<Move>(src->dtype, src->head_dim, A.groups, &cfg, &A);
}
