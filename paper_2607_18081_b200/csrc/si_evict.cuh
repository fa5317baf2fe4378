// Eviction, as shared by the cache in 16 bits and the one in 4: what the selecting kernel (si_kv.cu) decides with and leaves.
#pragma once
#include "si_kv4.cuh"

struct EvictArgs {
    si_kv_view src, dst;
    const int32_t *q_pos;
    int n_new, budget, n_sink, n_recent, in_place, move_here;
    int slots;                           // slots that `source` describes: the budget, at most the capacity if it is scratch
    int32_t *source, *lists;             // [rows][slots]: source slot of every slot (the caller's `kept` or scratch); [rows][cap + 2]:
                                         // freed slots, then (from cap / 2 + 1) the entries that fill them, at most cap / 2 each
    int list_source;                     // 0: nobody reads `source` (moves of this kernel only, no `kept`)
    int32_t *len_out;
    int32_t *status;
    int block0;                          // moving kernel: number of the grid's first block of slots
    si_kv4_view src4, dst4;              // the entries of caches in 4 bits (src.k, src.v, .. are NULL then)
    int groups;                          // ... and their groups per entry
};

size_t si_evict_ws_bytes(int n_seqs, int n_kv_heads, int capacity);
EvictArgs si_evict_args(const si_kv_view &src, const si_kv_view &dst, bool in_place, const int32_t *q_pos, int n_new, int budget, int n_sink,
                        int n_recent, int32_t *kept, int32_t *len_out, void *workspace, int32_t *status);
// Launches the selection; with A.move_here on return, everything is done.
int si_evict_select(EvictArgs &A, cudaStream_t st);

__device__ __forceinline__ int si_evict_entries(const EvictArgs &A, int b) {
    const int n = si_kv_len(A.src, b, A.status) + A.n_new;
    if (n > A.src.cap) { si_report(A.status, SI_ERR_OUT_OF_RANGE); return A.src.cap; }
    return n;
}

constexpr int kMoveLanes4 = 16;
// Entry `from` of a 4-bit row to slot `to`, by kMoveLanes4 lanes: eight for the values, four for the key, two for the steps, one for
// position and weight.
__device__ __forceinline__ void si_move_entry4(const EvictArgs &A, int b, int h, int from, int to, int lane) {
    const uint8_t *s = A.src4.row(b, h) + (long long)(from / kTileEntries) * A.src4.tile;
    uint8_t *d = A.dst4.row(b, h) + (long long)(to / kTileEntries) * A.dst4.tile;
    const int D = A.src.D, W = D / 32, NG = A.groups, f = from % kTileEntries, t = to % kTileEntries;
    if (lane < 8) {
        auto at = [&](int r) { return D == 128 ? si_tile4<128, 4>::value_word(r, 0, lane) : si_tile4<64, 2>::value_word(r, 0, lane); };   // the same for any group
        const uint16_t *x = reinterpret_cast<const uint16_t *>(s + at(f)) + (f & 1);
        uint16_t *y = reinterpret_cast<uint16_t *>(d + at(t)) + (t & 1), v[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) if (w < W) v[w] = x[2 * w];
#pragma unroll
        for (int w = 0; w < 4; ++w) if (w < W) y[2 * w] = v[w];
    } else if (lane < 14) {
        const int n = lane < 12 ? W : NG, par = 32 * D + (lane == 13 ? kTileEntries * NG * 4 : 0);
        const uint32_t *x = reinterpret_cast<const uint32_t *>(s + (lane < 12 ? f * (D / 2) + (lane - 8) * (D / 8) : par + f * NG * 4));
        uint32_t *y = reinterpret_cast<uint32_t *>(d + (lane < 12 ? t * (D / 2) + (lane - 8) * (D / 8) : par + t * NG * 4)), v[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) if (w < n) v[w] = x[w];
#pragma unroll
        for (int w = 0; w < 4; ++w) if (w < n) y[w] = v[w];
    } else if (lane == 14) {
        const int p = A.src.pos ? A.src.pos[A.src.meta(b, h) + from] : from;
        const float w = A.src.weight[A.src.meta(b, h) + from];
        A.dst.pos[A.dst.meta(b, h) + to] = p;
        A.dst.weight[A.dst.meta(b, h) + to] = w;
    }
}
