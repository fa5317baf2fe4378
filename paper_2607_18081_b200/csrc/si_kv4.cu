// The key/value cache in 4 bits: quantising entries as they are stored, reading them back, eviction.  (Layout and format: si_kv4.cuh.)
//
// All three are bound by HBM: an entry is 4 D bytes in 16 bits and D + 8 D / group in 4.
#include "si_evict.cuh"
#include "si_tc.cuh"

namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;

struct StoreArgs {
    si_kv_view src, meta;            // meta: pos, weight, len, capacity of the cache in 4 bits
    si_kv4_view dst;
    const int32_t *first_pos;
    int32_t *status;
};

// A warp per tile: the entries' rows come in as 16-byte pieces (eight elements: one word of a key's codes, two half words of a
// value's), the tile is put together in shared memory and goes out in 16-byte pieces.
template <int DT, int D, int NG>
__global__ void __launch_bounds__(kThreads) store_kernel(const StoreArgs A) {
    using T = si_tile4<D, NG>;
    constexpr int L = D / 8, ROWS = 32 / L, GL = D / NG / 8;     // lanes of a row, rows of a warp, lanes of a group
    __shared__ __align__(16) char sh[kWarps][T::kBytes];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = blockIdx.y, b = blockIdx.z;
    si_tc::pdl_wait();
    si_tc::pdl_launch();
    const bool tell = h == 0 && blockIdx.x == 0 && threadIdx.x == 0;
    const int start = si_kv_len(A.meta, b, tell ? A.status : nullptr);
    int n = si_kv_len(A.src, b, tell ? A.status : nullptr);
    if (n > A.meta.cap - start) { if (tell) si_report(A.status, SI_ERR_OUT_OF_RANGE); n = A.meta.cap - start; }
    const int tile = start / kTileEntries + blockIdx.x * kWarps + warp, e0 = tile * kTileEntries;
    if (n <= 0 || e0 >= start + n) return;
    const int r0 = max(0, start - e0), r1 = min(kTileEntries, start + n - e0);
    char *sm = sh[warp];
    const int c = lane % L, w = c / 4, t = c % 4;
#pragma unroll 2
    for (int i = 0; i < kTileEntries; i += ROWS) {
        const int r = i + lane / L;
        const bool in = r >= r0 && r < r1;
        const long long at = A.src.row(b, h, in ? e0 + r - start : 0) + c * 8;
        uint4 raw[2];
        raw[0] = in ? *reinterpret_cast<const uint4 *>(A.src.k + at) : make_uint4(0, 0, 0, 0);
        raw[1] = in ? *reinterpret_cast<const uint4 *>(A.src.v + at) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const uint32_t u[4] = {raw[which].x, raw[which].y, raw[which].z, raw[which].w};
            float f[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) { f[2 * k] = si_cvt<DT>::lo(u[k]); f[2 * k + 1] = si_cvt<DT>::hi(u[k]); }
            float low = f[0], high = f[0];
#pragma unroll
            for (int k = 1; k < 8; ++k) { low = si_q4::min_nan(low, f[k]); high = si_q4::max_nan(high, f[k]); }
#pragma unroll
            for (int o = 1; o < GL; o <<= 1) {
                low = si_q4::min_nan(low, __shfl_xor_sync(0xFFFFFFFFu, low, o));
                high = si_q4::max_nan(high, __shfl_xor_sync(0xFFFFFFFFu, high, o));
            }
            float inverse;
            const uint32_t par = si_q4::group_word<DT>(low, high, &inverse);
            uint32_t code[8], word = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) code[k] = si_q4::code_bits(f[k], low, inverse) & 15u;
            if (which == 0) {
#pragma unroll
                for (int k = 0; k < 8; ++k) word |= code[k] << (4 * ((k >> 1) + (k & 1) * 4));
                *reinterpret_cast<uint32_t *>(sm + T::key_word(r, w, t)) = word;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) word |= code[k] << (4 * k);
                // elements 0 .. 3 in the lower half, 4 .. 7 in the upper: the two entries of a pair exchange a half each
                const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, word, L);
                const uint32_t both = r & 1 ? __byte_perm(other, word, 0x7632) : __byte_perm(word, other, 0x5410);
                *reinterpret_cast<uint32_t *>(sm + T::value_word(r, w, 2 * t + (r & 1))) = both;
            }
            if (c % GL == 0) *reinterpret_cast<uint32_t *>(sm + (which ? T::kValuePar : T::kKeyPar) + (r * NG + T::place_of(c / GL)) * 4) = par;
        }
    }
    __syncwarp();
    uint8_t *to = A.dst.row(b, h) + (long long)tile * T::kBytes;
    auto copy16 = [&](int from, int end) {
        for (int i = from + lane * 16; i < end; i += 512) *reinterpret_cast<uint4 *>(to + i) = *reinterpret_cast<const uint4 *>(sm + i);
    };
    if (r0 == 0 && r1 == kTileEntries) {
        copy16(0, T::kBytes);
    } else {
        copy16(r0 * (D / 2), r1 * (D / 2));
        const int p0 = (r0 + 1) / 2, p1 = r1 / 2;                // whole pairs of values, then the single ones
        copy16(T::kValues + p0 * D, T::kValues + p1 * D);
        auto single = [&](int r) {
            if (lane >= D / 4) return;
            const int at = T::kValues + (r >> 1) * D + lane * 4 + 2 * (r & 1);
            *reinterpret_cast<uint16_t *>(to + at) = *reinterpret_cast<const uint16_t *>(sm + at);
        };
        if (r0 & 1) single(r0);
        if (r1 & 1) single(r1 - 1);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const int par = which ? T::kValuePar : T::kKeyPar;
            for (int i = r0 * NG + lane; i < r1 * NG; i += 32) *reinterpret_cast<uint32_t *>(to + par + i * 4) = *reinterpret_cast<const uint32_t *>(sm + par + i * 4);
        }
    }
    if (lane < r0 || lane >= r1) return;
    const int e = e0 + lane, j = e - start;
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

template <int DT> __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    if (DT == SI_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// m + s c.  The step is rounded up, so that the highest code may stand for a little more than the type holds: the largest number
// then (bf16: a range of 2^94 is far from its end).
template <int DT> __device__ __forceinline__ float value_of(float code, float step, float low) {
    const float x = fmaf(code, step, low);
    return DT == SI_F16 ? si_q4::min_nan(x, 65504.f) : x;
}

// A warp per tile; a lane makes eight neighbouring elements of a row.
template <int DT, int D, int NG>
__global__ void __launch_bounds__(kThreads) load_kernel(const LoadArgs A) {
    using T = si_tile4<D, NG>;
    constexpr int L = D / 8, ROWS = 32 / L;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = blockIdx.y, b = blockIdx.z;
    si_tc::pdl_wait();
    si_tc::pdl_launch();
    const bool tell = h == 0 && blockIdx.x == 0 && threadIdx.x == 0;
    const int len = si_kv_len(A.meta, b, tell ? A.status : nullptr);
    int first = A.first ? A.first[b] : 0;
    if (first < 0) { if (tell) si_report(A.status, SI_ERR_OUT_OF_RANGE); first = 0; }
    const int end = first + min(A.n, max(0, len - first));
    if (tell && A.len_out) A.len_out[b] = end - first;
    if (end <= first) return;
    const int tile = first / kTileEntries + blockIdx.x * kWarps + warp, e0 = tile * kTileEntries;
    if (e0 >= end) return;
    const uint8_t *from = A.src.row(b, h) + (long long)tile * T::kBytes;
    const int c = lane % L, w = c / 4, t = c % 4, g = T::place_of(T::group_of(w));
#pragma unroll 4
    for (int i = 0; i < kTileEntries; i += ROWS) {
        const int r = i + lane / L;
        if (e0 + r < first || e0 + r >= end) continue;
        const uint32_t kw = *reinterpret_cast<const uint32_t *>(from + T::key_word(r, w, t));
        const uint32_t v0 = *reinterpret_cast<const uint32_t *>(from + T::value_word(r, w, 2 * t)), v1 = *reinterpret_cast<const uint32_t *>(from + T::value_word(r, w, 2 * t + 1));
        const uint32_t kp = *reinterpret_cast<const uint32_t *>(from + T::kKeyPar + (r * NG + g) * 4), vp = *reinterpret_cast<const uint32_t *>(from + T::kValuePar + (r * NG + g) * 4);
        // codes come as c 2^-24 and 16 c 2^-24
        float s = si_cvt<DT>::hi(kp), m = si_cvt<DT>::lo(kp), s0 = s * 0x1p24f, s1 = s * 0x1p20f;
        float2 x[4] = {si_q4::code_pair(si_q4::low_codes(kw)), si_q4::code_pair(si_q4::high_codes(kw)), si_q4::code_pair(si_q4::low_codes(kw >> 8)), si_q4::code_pair(si_q4::high_codes(kw >> 8))};
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = pack2<DT>(value_of<DT>(x[k].x, k & 1 ? s1 : s0, m), value_of<DT>(x[k].y, k & 1 ? s1 : s0, m));
        const long long at = A.dst.row(b, h, e0 + r - first) + c * 8;
        *reinterpret_cast<uint4 *>(A.dst.k + at) = make_uint4(o[0], o[1], o[2], o[3]);
        const uint32_t vw = __byte_perm(v0, v1, r & 1 ? 0x7632 : 0x5410);       // elements 0 .. 3 | 4 .. 7
        s = si_cvt<DT>::hi(vp); m = si_cvt<DT>::lo(vp); s0 = s * 0x1p24f; s1 = s * 0x1p20f;
        float2 y[4] = {si_q4::code_pair(si_q4::low_codes(vw)), si_q4::code_pair(si_q4::high_codes(vw)), si_q4::code_pair(si_q4::low_codes(vw >> 8)), si_q4::code_pair(si_q4::high_codes(vw >> 8))};
#pragma unroll
        for (int k = 0; k < 4; ++k) { y[k].x = value_of<DT>(y[k].x, k & 1 ? s1 : s0, m); y[k].y = value_of<DT>(y[k].y, k & 1 ? s1 : s0, m); }
        *reinterpret_cast<uint4 *>(A.dst.v + at) = make_uint4(pack2<DT>(y[0].x, y[1].x), pack2<DT>(y[2].x, y[3].x), pack2<DT>(y[0].y, y[1].y), pack2<DT>(y[2].y, y[3].y));
    }
    const int e = e0 + lane;
    if (e < first || e >= end) return;
    if (A.meta.pos && A.dst.pos) A.dst.pos[A.dst.meta(b, h) + e - first] = A.meta.pos[A.meta.meta(b, h) + e];
    if (A.meta.weight && A.dst.weight) A.dst.weight[A.dst.meta(b, h) + e - first] = A.meta.weight[A.meta.meta(b, h) + e];
}

// The kept entries to their slots; nothing to do for an entry that stays.
__global__ void __launch_bounds__(256) move4_kernel(const EvictArgs A) {
    constexpr int kSlots = 256 / kMoveLanes4;
    const int b = blockIdx.z, h = blockIdx.y, row = b * A.src.H + h, lane = threadIdx.x % kMoveLanes4;
    si_tc::pdl_wait();
    si_tc::pdl_launch();
    if (h == 0 && blockIdx.x == 0 && threadIdx.x == 0 && A.len_out) A.len_out[b] = min(si_evict_entries(A, b), A.budget);
    const int slot = blockIdx.x * kSlots + threadIdx.x / kMoveLanes4;
    if (slot >= A.slots) return;
    const int j = A.source[(size_t)row * A.slots + slot];
    if (j >= 0 && !(A.in_place && j == slot)) si_move_entry4(A, b, h, j, slot, lane);
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

// Blocks that cover n entries, wherever in a tile the first one is.
unsigned tile_blocks(int n) { return (unsigned)(((long long)n + kTileEntries - 2) / kTileEntries + kWarps) / kWarps; }

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
    cudaLaunchConfig_t cfg = config(dim3(tile_blocks(src->capacity), dst->n_kv_heads, dst->n_seqs), kThreads, (cudaStream_t)stream, &at);
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
    const LoadArgs A{si_kv4_meta_of(src), si_kv_view_of(dst), si_kv4_view_of(src), first, n, len_out, status_dev};
    si_mt_forget();
    const int most = n < src->capacity ? n : src->capacity;
    cudaLaunchAttribute at;
    cudaLaunchConfig_t cfg = config(dim3(tile_blocks(most), src->n_kv_heads, src->n_seqs), kThreads, (cudaStream_t)stream, &at);
    return by_shape<Load>(src->dtype, src->head_dim, si_kv4_groups(src), &cfg, &A);
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
    A.src4 = si_kv4_view_of(src); A.dst4 = si_kv4_view_of(dst); A.groups = si_kv4_groups(src);
    si_mt_forget();
    if ((rc = si_evict_select(A, (cudaStream_t)stream)) || A.move_here) return rc;
    cudaLaunchAttribute at;
    cudaLaunchConfig_t cfg = config(dim3((A.slots + 256 / kMoveLanes4 - 1) / (256 / kMoveLanes4), src->n_kv_heads, src->n_seqs), 256, (cudaStream_t)stream, &at);
    SI_CUDA_TRY(cudaLaunchKernelEx(&cfg, move4_kernel, A));
    return SI_OK;
}
