// A paged K/V cache in bf16, in the layout of the pass's own pool (kv_index in common.cuh):
//   [layer][page][K, V][KV head][position / 8][column / 8][position % 8][column % 8]
// A (page, K or V, head) block is contiguous, 128 bytes of it are an 8 x 8 core matrix of the tensor cores' shared-memory operands: eight positions
// by eight columns.  Copied as it is, a block serves as the K-major operand of Q K^T and as the MN-major operand of P V alike.
#pragma once
#include "where.cuh"

namespace pipesd {

// A call's requests (Kv4Where, kv4_rows) and the pool.
struct Kv16Pool {
    uint16_t* pool;
    int n_layers, layer, hd;
};

__device__ __forceinline__ size_t kv16_block_elems(const Kv4Where& w, int hd) { return (size_t)w.page_size * hd; }
// Block of (layer, page, K or V, head).
__device__ __forceinline__ uint16_t* kv16_block(const Kv16Pool& p, const Kv4Where& w, int layer, int page, int kv, int head) {
    return p.pool + ((((size_t)layer * w.n_pages + page) * 2 + kv) * w.Hkv + head) * kv16_block_elems(w, p.hd);
}
// Element (slot, 8 c) of a block: 16 bytes of it are consecutive.
__device__ __forceinline__ uint32_t kv16_piece(int slot, int c, int hd) { return (uint32_t)((slot >> 3) * 8 * hd + c * 64 + (slot & 7) * 8); }
// The page that holds a position of request r, or -1.
__device__ __forceinline__ int kv16_page(const Kv4Where& w, int r, int pos) {
    const int page = w.table[(size_t)r * w.max_pages + pos / w.page_size];
    return page >= 0 && page < w.n_pages ? page : -1;
}
// Request that row belongs to, the first one that claims it, its base and its first row (whole warp; -1: none).
__device__ __forceinline__ int kv16_request_of(const Kv4Where& w, int row, int& first, int& base) {
    const int lane = threadIdx.x & 31;
    for (int r0 = 0; r0 < w.n_req; r0 += 32) {
        int f = 0, b = 0, n = 0;
        if (r0 + lane < w.n_req) n = kv4_rows(w, r0 + lane, f, b);
        const unsigned hit = __ballot_sync(0xffffffffu, n > 0 && row >= f && row - f < n);
        if (hit) {
            const int l = __ffs(hit) - 1;
            first = __shfl_sync(0xffffffffu, f, l);
            base = __shfl_sync(0xffffffffu, b, l);
            return r0 + l;
        }
    }
    return -1;
}

}  // namespace pipesd
