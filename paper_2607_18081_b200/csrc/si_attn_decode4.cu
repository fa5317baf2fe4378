// Single-token attention over the key/value cache in 4 bits.
//
//   out_q = sum_j p_qj (s_j c_j + m_j),  p_q = softmax over the visible entries j of scale q . (s'_j c'_j + m'_j)
//
// A warp per sequence and key head: it stores the new entry, then goes through its entries once per query head, and once more
// for the weights.
#include "si_attn_split.cuh"
#include "si_kv4.cuh"

namespace {

struct Decode4Args {
    DecodeArgs d;
    si_kv4_view kv;
};

// elements d, d + 1 of the key (value) in slot r of a tile
template <int DT, int D, int NG> __device__ __forceinline__ float2 two(const uint8_t *tile, int r, int d, bool value) {
    using T = si_tile4<D, NG>;
    const uint32_t par = *reinterpret_cast<const uint32_t *>(tile + (value ? T::kValuePar : T::kKeyPar) + (r * NG + d / (D / NG)) * 4);
    const int w = d / 32, in = d % 32;
    uint32_t c0, c1;
    if (value) {
        const uint32_t x = *reinterpret_cast<const uint32_t *>(tile + T::value_word(r, w, in / 4)) >> (16 * (r & 1) + 4 * (in % 4));
        c0 = x & 15; c1 = x >> 4 & 15;
    } else {
        const uint32_t x = *reinterpret_cast<const uint32_t *>(tile + T::key_word(r, w, in / 8)) >> (4 * (in % 8 / 2));
        c0 = x & 15; c1 = x >> 16 & 15;
    }
    const float s = si_cvt<DT>::lo(par), m = si_cvt<DT>::hi(par);
    return make_float2(fmaf(s, (float)c0, m), fmaf(s, (float)c1, m));
}

template <int DT, int D, int NG>
__global__ void __launch_bounds__(32) decode4_kernel(const Decode4Args A4) {
    const DecodeArgs &A = A4.d;
    constexpr int E = D / 64;              // pairs of elements per lane
    const int h = blockIdx.x, b = blockIdx.y, lane = threadIdx.x;
    si_tc::pdl_wait();
    si_tc::pdl_launch();
    const SeqWork w = seq_work<kTileEntries>(A, b, h == 0 && lane == 0 ? A.status : nullptr);
    uint8_t *row = A4.kv.row(b, h);
    const int32_t *pos = A.kv.pos ? A.kv.pos + A.kv.meta(b, h) : nullptr;
    if (w.n_old != INT_MAX) {
        const long long from = b * A.new_ss + (long long)h * D;
        si_q4::store_entry<DT, D, NG>(A.kn + from, A.vn + from, w.n_old % kTileEntries, (char *)row + (long long)(w.n_old / kTileEntries) * A4.kv.tile, nullptr);
        if (pos && lane == 0) A.kv.pos[A.kv.meta(b, h) + w.n_old] = w.s;
        __threadfence_block();
        __syncwarp();
    }
    auto sees = [&](int j) { return si_visible(pos ? pos[j] : j, w.s, w.lo, A.n_sink); };
    for (int g = 0; g < A.G; ++g) {
        const int head = h * A.G + g;
        float2 q[E], o[E];
        for (int i = 0; i < E; ++i) {
            const uint32_t u = *reinterpret_cast<const uint32_t *>(A.q + b * A.q_ss + (long long)head * D + 64 * i + 2 * lane);
            q[i] = make_float2(si_cvt<DT>::lo(u), si_cvt<DT>::hi(u));
            o[i] = make_float2(0.f, 0.f);
        }
        auto score = [&](int j) {
            const uint8_t *tile = row + (long long)(j / kTileEntries) * A4.kv.tile;
            float x = 0.f;
            for (int i = 0; i < E; ++i) {
                const float2 k = two<DT, D, NG>(tile, j % kTileEntries, 64 * i + 2 * lane, false);
                x = fmaf(q[i].x, k.x, fmaf(q[i].y, k.y, x));
            }
            for (int s = 16; s; s >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, s);
            return x * A.scale2;
        };
        float top = -INFINITY, sum = 0.f;
        for (int j = 0; j < w.n; ++j) {
            if (!sees(j)) continue;
            const float x = score(j), next = fmaxf(top, x), f = top == -INFINITY ? 1.f : ex2(top - next), p = ex2(x - (next == -INFINITY ? 0.f : next));
            top = next;
            sum = sum * f + p;
            const uint8_t *tile = row + (long long)(j / kTileEntries) * A4.kv.tile;
            for (int i = 0; i < E; ++i) {
                const float2 v = two<DT, D, NG>(tile, j % kTileEntries, 64 * i + 2 * lane, true);
                o[i].x = fmaf(p, v.x, o[i].x * f); o[i].y = fmaf(p, v.y, o[i].y * f);
            }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum, base = top == -INFINITY ? 0.f : top;
        const long long to = (long long)b * A.Hq + head;
        for (int i = 0; i < E; ++i) *reinterpret_cast<uint32_t *>(A.out + to * D + 64 * i + 2 * lane) = pack2<DT>(o[i].x * inv, o[i].y * inv);
        if (lane == 0 && A.lse) A.lse[to] = sum == 0.f ? -INFINITY : (top + log2f(sum)) / kLog2e;
        if (!A.acc) continue;
        for (int j = 0; j < w.n; ++j) {
            float *weight = A.kv.weight + A.kv.meta(b, h) + j;
            if (!sees(j)) { if (j == w.n_old && lane == 0) *weight = 0.f; continue; }
            const float p = ex2(score(j) - base) * inv;
            if (lane == 0) *weight = (j == w.n_old && g == 0 ? 0.f : *weight) + p;
        }
    }
}

template <int DT> int launch(const Decode4Args &A, int NG, cudaStream_t st) {
    const dim3 grid(A.d.kv.H, A.d.kv.B);
    if (A.d.kv.D == 128) {
        if (NG == 4) decode4_kernel<DT, 128, 4><<<grid, 32, 0, st>>>(A);
        else decode4_kernel<DT, 128, 2><<<grid, 32, 0, st>>>(A);
    } else {
        if (NG == 2) decode4_kernel<DT, 64, 2><<<grid, 32, 0, st>>>(A);
        else decode4_kernel<DT, 64, 1><<<grid, 32, 0, st>>>(A);
    }
    SI_CUDA_TRY(cudaGetLastError());
    return SI_OK;
}

Layout layout_of(const si_kv4_t *kv, int n_q_heads, bool acc) {
    return layout_of(2 * si_sm_count(), kv->n_seqs, kv->n_kv_heads, kv->head_dim, kv->capacity, n_q_heads, acc);
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
    return kv->dtype == SI_BF16 ? launch<SI_BF16>(A, si_kv4_groups(kv), (cudaStream_t)stream) : launch<SI_F16>(A, si_kv4_groups(kv), (cudaStream_t)stream);
}
