// The key/value cache held in 4 bits: layout, argument checks, quantisation.
//
// A group of 32 or 64 neighbouring values x of a key or value is held as its lowest value m and a step s, both of the cache's
// 16-bit type, and 4-bit codes c; it stands for m + s c:
//     s = fl((max x - min x) fl(1 / 15)) rounded up to the type,   c = nearest integer (ties to even) of fl(x - m) fl(1 / s)
// with fl = round to fp32 and the last product exact (one fused multiply-add).  m is one of the values, so it is exact; s is rounded
// up, so that no code is cut off at 15: |x - (m + s c)| <= s / 2 but for the fp32 roundings.  s below 2^-126 is 0.  A group that
// holds a NaN or an infinity, or whose range is beyond 2^94, has s = m = NaN.
//
// Entries lie in tiles of 32, each contiguous, in the order in which a warp's lane (g, t) = (lane / 4, lane % 4) works on them, so
// that every access to a tile in shared memory is one vector per lane without bank conflicts and the codes need no shuffle:
//   keys     entry r, D / 2 bytes at r D / 2; of its elements, lane t of four has 32 w + 8 t + e (w < D / 32, e < 8): D / 8 bytes at
//            t D / 8, word w.  Elements 2 i and 2 i + 1 are nibbles i and i + 4 of the word.
//   values   from 16 D: entries in pairs, pair r / 2 of D bytes at D (r / 2); lane g of eight has elements 32 w + 4 g + i (i < 4): D / 8
//            bytes, word w, the even entry in its lower half, the odd one in its upper half, element i in nibble i of the half.
//            The eight cells of a pair are permuted by an XOR of g (bank conflicts).
//   steps    from 32 D: per entry D / group words of lowest value (lower half) and step (upper half) of the keys, then of the values;
//            four groups in the order 0, 2, 1, 3 (two lanes of four work on the even groups, two on the odd ones)
// A word masked with 0x000F000F is then a pair of f16 numbers c 2^-24 (subnormal, and exact in a product with fp32 sums): two
// neighbouring elements of a key, or one element of two neighbouring entries; with 0x00F000F0, the next ones, times 16.
#pragma once
#include "si_kv.cuh"

constexpr int kTileEntries = 32;

// keys of all kernels: D = head_dim, NG = groups per entry
template <int D, int NG> struct si_tile4 {
    static constexpr int W = D / 32;                     // words of a lane's cell
    static constexpr int kCell = D / 8, kValues = 16 * D, kKeyPar = 32 * D, kPar = kTileEntries * NG * 4, kValuePar = kKeyPar + kPar;
    static constexpr int kBytes = kValuePar + kPar;
    __host__ __device__ static constexpr int group_of(int w) { return w * NG / W; }
    // bank conflicts: the sixteen-byte (D = 64: eight-byte) cells that lanes g = 2 a, 2 a + 1 (4 a .. 4 a + 3) of all four t read
    // in one access are then in different banks
    __host__ __device__ static constexpr int swizzle(int t) { return D == 128 ? 2 * t : (t >> 1) * 4; }
    __host__ __device__ static constexpr int place_of(int g) { return NG == 4 ? (g & 1) << 1 | g >> 1 : g; }      // its own inverse
    __host__ __device__ static constexpr int key_word(int r, int w, int t) { return r * (D / 2) + t * kCell + w * 4; }
    __host__ __device__ static constexpr int value_word(int r, int w, int g) { return kValues + (r >> 1) * D + (g ^ swizzle(r >> 1 & 3)) * kCell + w * 4; }
};
inline int si_tile4_bytes(int head_dim, int group) { return 32 * head_dim + 2 * kTileEntries * 4 * (head_dim / (group < head_dim ? group : head_dim)); }
inline int si_kv4_groups(const si_kv4_t *kv) { return kv->head_dim / (kv->group < kv->head_dim ? kv->group : kv->head_dim); }

struct si_kv4_view {
    uint8_t *data;
    long long ss, hs;                // bytes
    int tile;                        // bytes of a tile
    __host__ __device__ __forceinline__ uint8_t *row(int b, int h) const { return data + b * ss + h * hs; }
};
inline si_kv4_view si_kv4_view_of(const si_kv4_t *kv) { return {(uint8_t *)kv->data, kv->seq_stride, kv->head_stride, si_tile4_bytes(kv->head_dim, kv->group)}; }
// Everything but the entries themselves, as the kernels shared with the 16-bit cache see it.
inline si_kv_view si_kv4_meta_of(const si_kv4_t *kv) {
    return {nullptr, nullptr, kv->weight, kv->pos, kv->len, 0, 0, 0, kv->n_seqs, kv->n_kv_heads, kv->head_dim, kv->capacity};
}

inline int si_kv4_check(const si_kv4_t *kv) {
    if (!kv || kv->n_seqs < 0 || kv->n_kv_heads < 1 || kv->capacity < kTileEntries || kv->capacity % kTileEntries || kv->head_dim < 1) return SI_ERR_INVALID_ARG;
    if (kv->dtype != SI_F16 && kv->dtype != SI_BF16) return SI_ERR_INVALID_ARG;
    if (kv->n_kv_heads > 65535 || kv->n_seqs > 65535) return SI_ERR_INVALID_ARG;
    if ((kv->head_dim != 64 && kv->head_dim != 128) || (kv->group != 32 && kv->group != 64)) return SI_ERR_UNSUPPORTED;
    if (kv->n_seqs == 0) return SI_OK;
    if (!kv->data || !kv->len || kv->head_stride < 0 || kv->seq_stride < 0) return SI_ERR_INVALID_ARG;
    if (!si_aligned16(kv->data) || ((kv->head_stride | kv->seq_stride) & 15) || !si_aligned16(kv->pos) || !si_aligned16(kv->weight) || !si_aligned4(kv->len))
        return SI_ERR_ALIGNMENT;
    return SI_OK;
}
inline bool si_kv4_shared(const si_kv4_t *kv) {
    return (kv->n_seqs > 1 && kv->seq_stride == 0) || (kv->n_kv_heads > 1 && kv->head_stride == 0);
}

namespace si_q4 {

__device__ __forceinline__ float min_nan(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// lowest value | step << 16 of a group with these extremes; *inverse is what its codes are computed with
template <int DT> __device__ __forceinline__ uint32_t group_word(float low, float high, float *inverse) {
    const float range = high - low;
    *inverse = 0.f;
    if (!(range <= 0x1p94f)) return DT == SI_BF16 ? 0x7FC07FC0u : 0x7E007E00u;
    const float step = range * (1.0f / 15.0f);
    uint32_t s = si_cvt<DT>::from_float(step);
    if (si_cvt<DT>::lo(s) < step) ++s;
    const float sf = si_cvt<DT>::lo(s);
    if (sf < 0x1p-126f) s = 0;
    else *inverse = __frcp_rn(sf);
    return s << 16 | (uint32_t)si_cvt<DT>::from_float(low);
}
// 2^23 * 1.5 + code: the code is in the low bits
__device__ __forceinline__ uint32_t code_bits(float x, float low, float inverse) { return __float_as_uint(__fmaf_rn(__fsub_rn(x, low), inverse, 12582912.f)); }

// One entry's key and value (16-bit rows of D elements) into slot r of a tile, by a warp.  `tile` and `more` (either may be NULL):
// two places that get the same.
template <int DT, int D, int NG> __device__ __forceinline__ void store_entry(const uint16_t *k, const uint16_t *v, int r, char *tile, char *more) {
    using T = si_tile4<D, NG>;
    constexpr int E = D / 32, GL = 32 / NG;              // elements of a lane, lanes of a group
    const int lane = threadIdx.x & 31, d = lane * E, w = d / 32, in = d % 32;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const uint16_t *x = which ? v : k;
        float f[E];
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const uint32_t u = *reinterpret_cast<const uint32_t *>(x + d + i);
            f[i] = si_cvt<DT>::lo(u); f[i + 1] = si_cvt<DT>::hi(u);
        }
        float low = f[0], high = f[0];
#pragma unroll
        for (int i = 1; i < E; ++i) { low = min_nan(low, f[i]); high = max_nan(high, f[i]); }
#pragma unroll
        for (int o = 1; o < GL; o <<= 1) {
            low = min_nan(low, __shfl_xor_sync(0xFFFFFFFFu, low, o));
            high = max_nan(high, __shfl_xor_sync(0xFFFFFFFFu, high, o));
        }
        float inverse;
        const uint32_t par = group_word<DT>(low, high, &inverse);
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int e = in % 8 + i, nibble = which ? in % 4 + i : (e >> 1) + (e & 1) * 4;
            word |= (code_bits(f[i], low, inverse) & 15u) << (4 * nibble);
        }
        const int par_at = (which ? T::kValuePar : T::kKeyPar) + (r * NG + T::place_of(lane / GL)) * 4;
        if (which == 0) {
#pragma unroll
            for (int o = 1; o < 8 / E; o <<= 1) word |= __shfl_xor_sync(0xFFFFFFFFu, word, o);
            const int at = T::key_word(r, w, in / 8);
            if (in % 8 == 0 && tile) *reinterpret_cast<uint32_t *>(tile + at) = word;
            if (in % 8 == 0 && more) *reinterpret_cast<uint32_t *>(more + at) = word;
        } else {
#pragma unroll
            for (int o = 1; o < 4 / E; o <<= 1) word |= __shfl_xor_sync(0xFFFFFFFFu, word, o);
            const int at = T::value_word(r, w, in / 4) + 2 * (r & 1);
            if (in % 4 == 0 && tile) *reinterpret_cast<uint16_t *>(tile + at) = (uint16_t)word;
            if (in % 4 == 0 && more) *reinterpret_cast<uint16_t *>(more + at) = (uint16_t)word;
        }
        if (lane % GL == 0 && tile) *reinterpret_cast<uint32_t *>(tile + par_at) = par;
        if (lane % GL == 0 && more) *reinterpret_cast<uint32_t *>(more + par_at) = par;
    }
}

// Pairs of f16 numbers c 2^-24 to floats: exact.
__device__ __forceinline__ float2 code_pair(uint32_t w) {
    float2 f;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.f32.f16 %0, lo;\n\tcvt.f32.f16 %1, hi;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(w));
    return f;
}
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return w & 0x000F000Fu; }       // c 2^-24
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return w & 0x00F000F0u; }      // 16 c 2^-24

}  // namespace si_q4

// implemented in si_attn_decode4.cu
size_t si_kv4_attn_decode_ws_bytes(const si_kv4_t *kv, int n_q_heads);
