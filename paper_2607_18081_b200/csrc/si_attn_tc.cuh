// What the tensor-core attention kernels (prefill, accumulated weights) share: packed query tiles, the key tiles a block
// of queries sees, 4-D tensor maps, tensor-memory loads and stores.
#pragma once
#include "si_kv.cuh"
#include "si_tc.cuh"

namespace si_attn {

using namespace si_tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kTile = 128;                 // rows of a query tile, keys of a key tile
// Probes after which a wait gives up: a probe that fails takes 4 us, so after some 4 s; waits here are microseconds.  All are the
// suspending kind: polling without a pause takes the same time alone, but back to back the chip is at its power limit and polling warps cost 1-2 %.
constexpr int kWait = 1 << 20;

struct TcArgs {
    si_kv_view kv;
    int T, Hq, G, R;                       // G query heads per key head; R = kTile / G queries per tile: row r = query r / G, head r % G
    int window, n_sink;
    float scale2;                          // |scale| log2(e)
    int q_b, kv_b, kv_h;                   // 0 where sequences (heads) share memory through a zero stride, else 1
    uint16_t *out;
    float *lse;
    int32_t *status;
};

// The key tiles that queries at positions smin .. smax see: `sinks` tiles from the front, then tiles from entry `first` on; n in
// all.  With a window, `first` is the first entry in it, wherever that lies: a tile may start at any entry.
struct KeyTiles {
    int sinks, first, n, off;      // off: the first one of this CTA's share
    __device__ __forceinline__ int key0(int j) const { j += off; return j < sinks ? j * kTile : first + (j - sinks) * kTile; }
};
__device__ __forceinline__ KeyTiles key_tiles(int smin, int smax, int window, int n_sink) {
    KeyTiles k = {0, 0, 0, 0};
    if (smax < 0) return k;
    const int lo = window ? max(0, si_window_lo(smin, window) + 1) : 0, sinks = (min(n_sink, lo) + kTile - 1) / kTile;
    if (lo >= sinks * kTile) { k.sinks = sinks; k.first = lo; }      // else the two would overlap: everything from the front
    k.n = k.sinks + (smax + kTile - k.first) / kTile;
    return k;
}

__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
template <int DT> __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    if (DT == SI_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
// two fp32 values in a register pair: one instruction for both
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 two(float lo, float hi) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ f32x2 two(uint32_t lo, uint32_t hi) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi)); return r; }
__device__ __forceinline__ void untwo(f32x2 v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }

// 2^x for a pair on the multiply-add units: x = n + f with n the nearest integer (added to and taken from 1.5 * 2^23, whose low
// bits then hold n), 2^f by its polynomial of least relative error on [-1/2, 1/2] of degree 5 (2.1e-7 in fp32, computed for
// this file by a Remez exchange), n added to the exponent field.  x below -126 counts as -126, and so does NaN: it is for
// numbers only (a form that keeps NaN, with 2^n as a factor, made the weights of a prompt 112.6 -> 114.1 us).  The exponential unit does 16
// values per clock and SM, which a tile's softmax is otherwise bound by.
__device__ __forceinline__ f32x2 ex2_poly(f32x2 x) {
    float a, b;
    untwo(x, a, b);
    x = two(fmaxf(a, -126.f), fmaxf(b, -126.f));
    const f32x2 t = add2(x, two(12582912.f, 12582912.f)), f = add2(x, fma2(t, two(-1.f, -1.f), two(12582912.f, 12582912.f)));
    f32x2 p = two(0.0013276472454890609f, 0.0013276472454890609f);
    p = fma2(p, f, two(0.009675540961325169f, 0.009675540961325169f));
    p = fma2(p, f, two(0.05550713092088699f, 0.05550713092088699f));
    p = fma2(p, f, two(0.24022120237350464f, 0.24022120237350464f));
    p = fma2(p, f, two(0.6931469440460205f, 0.6931469440460205f));
    p = fma2(p, f, two(1.0000001192092896f, 1.0000001192092896f));
    float ta, tb, pa, pb;
    untwo(t, ta, tb);
    untwo(p, pa, pb);
    return two(__float_as_uint(pa) + (__float_as_uint(ta) << 23), __float_as_uint(pb) + (__float_as_uint(tb) << 23));
}

__device__ __forceinline__ void tma_load_4d(void *dst, const CUtensorMap *map, int x, int y, int z, int w, uint64_t *bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar)) : "memory");
}
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// A box out of shared memory; rows and columns beyond the tensor are not written.
__device__ __forceinline__ void tma_store_4d(const CUtensorMap *map, const void *src, int x, int y, int z, int w) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3, %4}], [%5];"
                 ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(src)) : "memory");
}
__device__ __forceinline__ void tma_store_wait() {
    asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group 0;" ::: "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// D[tmem] (+)= A . B with A in shared memory or (16-bit pairs) in tensor memory and B in shared memory.  Descriptors come as
// their two words: the upper one is the same for all steps of an operand, the lower one (address / 16) takes the offsets.
struct Desc { uint32_t lo, hi; };
__device__ __forceinline__ Desc desc_of(uint32_t smem_addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
    const uint64_t d = make_desc(smem_addr, lbo_bytes, sbo_bytes);
    return {(uint32_t)d, (uint32_t)(d >> 32)};
}
__device__ __forceinline__ void umma_ss(uint32_t d_tmem, Desc a, uint32_t a_off, Desc b, uint32_t b_off, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "mov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n\t}"
        ::"r"(d_tmem), "r"(a.lo + a_off), "r"(a.hi), "r"(b.lo + b_off), "r"(b.hi), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, Desc b, uint32_t b_off, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
        "mov.b64 b, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "r"(b.lo + b_off), "r"(b.hi), "r"(idesc), "r"(accumulate) : "memory");
}
#define SI_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define SI_P8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
#define SI_I8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of this warp's 32 lanes; the registers are valid after tmem_wait_ld on them
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : SI_R8(r, 0), SI_R8(r, 8), SI_R8(r, 16), SI_R8(r, 24) : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : SI_P8(r, 0), SI_P8(r, 8), SI_P8(r, 16), SI_P8(r, 24)::"memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
                 ::SI_I8(r, 0), SI_I8(r, 8), SI_I8(r, 16), SI_I8(r, 24), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::SI_I8(r, 0), SI_I8(r, 8), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint64_t *bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// Tensor map of a 16-bit array [d3][d2][d1][d0] with element strides s1, s2, s3 (multiples of 8), boxes of 64 x b1 x b2 x 1 with
// the 128-byte swizzle.  A dimension whose stride is 0 is encoded with extent 1.
inline int make_map_4d(CUtensorMap *map, const void *base, int d0, const long long (&d)[3], const long long (&s)[3], int b1, int b2) {
    typedef CUresult (*encode_fn_t)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                    const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                    CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<encode_fn_t> encode{nullptr};
    encode_fn_t f = encode.load();
    if (!f) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        SI_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q));
        if (!fn || q != cudaDriverEntryPointSuccess) return SI_ERR_CUDA;
        f = (encode_fn_t)fn;
        encode.store(f);
    }
    cuuint64_t dims[4] = {(cuuint64_t)d0, 1, 1, 1}, strides[3];
    for (int i = 0; i < 3; ++i) {
        const bool one = d[i] <= 1 || s[i] == 0;
        dims[i + 1] = one ? 1 : (cuuint64_t)d[i];
        strides[i] = one ? (cuuint64_t)d0 * 2 : (cuuint64_t)s[i] * 2;
        if (strides[i] >= 1ull << 40) return SI_ERR_UNSUPPORTED;
    }
    const cuuint32_t box[4] = {64, (cuuint32_t)b1, (cuuint32_t)b2, 1}, estr[4] = {1, 1, 1, 1};
    const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, const_cast<void *>(base), dims, strides, box, estr,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SI_OK : SI_ERR_CUDA;
}

// Maps of the queries (boxes of R tokens x G heads: one packed tile) and of the cache's keys or values (boxes of 128 entries).
inline int make_q_map(CUtensorMap *map, const void *q, const si_kv_t *kv, long long ss, long long ts, int T, int Hq, int G, int R) {
    const long long d[3] = {Hq, T, kv->n_seqs}, s[3] = {kv->head_dim, ts, ss};
    return make_map_4d(map, q, kv->head_dim, d, s, G, R);
}
inline int make_kv_map(CUtensorMap *map, const void *base, const si_kv_t *kv) {
    const long long d[3] = {kv->capacity, kv->n_kv_heads, kv->n_seqs}, s[3] = {kv->row_stride, kv->head_stride, kv->seq_stride};
    return make_map_4d(map, base, kv->head_dim, d, s, kTile, 1);
}
inline TcArgs tc_args(const si_kv_t *kv, long long q_ss, int T, int Hq, int window, int n_sink, float scale, void *out, float *lse, int32_t *status) {
    TcArgs A;
    A.kv = si_kv_view_of(kv);
    A.T = T; A.Hq = Hq; A.G = Hq / kv->n_kv_heads; A.R = kTile / A.G;
    A.window = window; A.n_sink = n_sink;
    // a scale of zero makes all weights equal; the smallest steps keep -inf * scale from becoming NaN
    A.scale2 = scale == 0.f ? 1e-30f : (scale < 0.f ? -scale : scale) * kLog2e;
    A.q_b = kv->n_seqs > 1 && q_ss != 0; A.kv_b = kv->n_seqs > 1 && kv->seq_stride != 0; A.kv_h = kv->n_kv_heads > 1 && kv->head_stride != 0;
    A.out = (uint16_t *)out; A.lse = lse; A.status = status;
    return A;
}

}  // namespace si_attn
