// What moves rows and pages of the bf16 cache: append and read, reserve, fork, compact and release, and a tree's ancestors.
//
// All of it is copying, bound by HBM where there is much of it and by a chain of dependent loads (request, table, row) where there is little.
// Pages are handed out by a table of references alone (refs[page], 0: free): the lowest free ids, in the order of the requests, so that what a
// call hands out does not depend on the calls before it beyond what they still hold, and nothing has to be kept in step with the tables.
#pragma once
#include "kv16.cuh"

namespace pipesd {

struct Kv16RowsArgs {
    Kv4Where w;
    Kv16Pool p;
    const void *k, *v;          // append: rows in; read: rows out (bf16)
    long long k_stride, v_stride;
    int wide;                   // rows can be loaded in 16-byte pieces
};

__device__ __forceinline__ uint4 kv16_load8(const uint16_t* p, bool wide) {
    if (wide) return *reinterpret_cast<const uint4*>(p);
    return make_uint4(pack2(p[0], p[1]), pack2(p[2], p[3]), pack2(p[4], p[5]), pack2(p[6], p[7]));
}
__device__ __forceinline__ uint4 kv16_load8(const float* p, bool wide) {
    float x[8];
    if (wide) {
        *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(p);
        *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(p + 4);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = p[i];
    }
    return bf16x8(x);
}

constexpr int kKv16RowWarps = 4;

// A warp per (row, KV head): eight columns of K or of V a lane.  grid: rows / 4, KV heads.
template <int HD, typename T>
__global__ void __launch_bounds__(32 * kKv16RowWarps) kv16_append_kernel(const Kv16RowsArgs a) {
    constexpr int kPieces = HD / 8;
    const int row = blockIdx.x * kKv16RowWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31, kv = lane / kPieces, c = lane % kPieces;
    if (row >= a.w.rows) return;
    int first, base;
    const int r = kv16_request_of(a.w, row, first, base);
    if (r < 0) return;
    const int pos = base + row - first, page = kv16_page(a.w, r, pos);
    if (page < 0 || kv >= 2) return;
    const int head = blockIdx.y;
    const T* src = kv == 0 ? static_cast<const T*>(a.k) + row * a.k_stride : static_cast<const T*>(a.v) + row * a.v_stride;
    *reinterpret_cast<uint4*>(kv16_block(a.p, a.w, a.p.layer, page, kv, head) + kv16_piece(pos % a.w.page_size, c, HD)) = kv16_load8(src + head * HD + c * 8, a.wide);
}

// The same the other way; 0 where no page is and for rows of no request.
template <int HD>
__global__ void __launch_bounds__(32 * kKv16RowWarps) kv16_read_kernel(const Kv16RowsArgs a) {
    constexpr int kPieces = HD / 8;
    const int row = blockIdx.x * kKv16RowWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31, kv = lane / kPieces, c = lane % kPieces;
    if (row >= a.w.rows) return;
    int first, base, pos = 0, page = -1;
    const int r = kv16_request_of(a.w, row, first, base);
    if (r >= 0) {
        pos = base + row - first;
        page = kv16_page(a.w, r, pos);
    }
    if (kv >= 2) return;
    const int head = blockIdx.y;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (page >= 0) x = *reinterpret_cast<const uint4*>(kv16_block(a.p, a.w, a.p.layer, page, kv, head) + kv16_piece(pos % a.w.page_size, c, HD));
    uint16_t* dst = static_cast<uint16_t*>(const_cast<void*>(kv == 0 ? a.k : a.v)) + ((size_t)row * a.w.Hkv + head) * HD + c * 8;
    *reinterpret_cast<uint4*>(dst) = x;
}

// ---- the ancestors of a tree's nodes
constexpr int kTreeWords = 256;                    // of a row's mask at most: 8192 nodes

// A CTA per request: its parents in shared memory, a thread per node that walks up.  A parent has a lower index than its child, so every walk ends.
// Bound by launch, loads and the longest path: 4.7 us for 8 requests of 64 nodes, of which none is 10 deep.
// One CTA more: rows in front of the first request and behind the last.
__global__ void __launch_bounds__(256) tree_mask_kernel(const int32_t* row0, const int32_t* parent, int n_req, int rows, int words, uint32_t* mask,
                                                         int32_t* depth) {
    __shared__ int32_t up[32 * kTreeWords];
    const int r = blockIdx.x;
    if (r == n_req) {
        const int from = max(0, min(row0[0], rows)), to = max(from, min(row0[n_req], rows));
        for (size_t i = threadIdx.x; i < (size_t)from * words; i += blockDim.x) mask[i] = 0;
        for (size_t i = (size_t)to * words + threadIdx.x; i < (size_t)rows * words; i += blockDim.x) mask[i] = 0;
        for (int i = threadIdx.x; i < from; i += blockDim.x) depth[i] = 0;
        for (int i = to + threadIdx.x; i < rows; i += blockDim.x) depth[i] = 0;
        return;
    }
    const int first = row0[r], end = row0[r + 1];
    if (first < 0 || end < first || end > rows) return;
    const int n = end - first, held = min(n, 32 * words);
    for (int i = threadIdx.x; i < held; i += blockDim.x) up[i] = parent[first + i];
    uint32_t* const mine = mask + (size_t)first * words;
    for (size_t i = threadIdx.x; i < (size_t)n * words; i += blockDim.x) mine[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        int d = -1, node = i < held ? i : -1, word = node >> 5;
        uint32_t bits = 0;
        while (node >= 0) {
            ++d;
            if (node >> 5 != word) {
                mine[(size_t)i * words + word] = bits;
                word = node >> 5;
                bits = 0;
            }
            bits |= 1u << (node & 31);
            const int p = up[node];
            node = p < node ? p : -1;
        }
        if (i < held) mine[(size_t)i * words + word] = bits;
        depth[first + i] = d;
    }
}

// ---- compaction
struct Kv16CompactArgs {
    Kv4Where w;                 // row0 and rows are not used
    Kv16Pool p;
    const uint32_t* keep;       // [n_req][words]
    int words;
    int32_t* kept;
};
constexpr int kCompactMoves = 256;                 // rows that are listed at a time

// Rows base + j with bit j of the request's keep go to base + (number of bits below j).  A warp per (layer, K or V, head) block, which loads sixteen
// rows before it stores them; targets lie in front of their sources and both ascend, so that no row is overwritten before it is
// read.  Eight lanes have the same columns of eight rows: rows that lie side by side share their sectors (32 forks of 64 nodes in 32 layers of 8 heads,
// 20 rows each: 55 us with the lanes along a row, 41 so).  grid: requests, blocks / 8.
template <int HD>
__global__ void __launch_bounds__(256) kv16_compact_kernel(const Kv16CompactArgs a) {
    constexpr int kPieces = HD / 8, kGroups = kPieces / 4;                     // of 4 pieces by 8 rows
    __shared__ uint32_t src[kCompactMoves], dst[kCompactMoves];      // page * page_size + slot
    __shared__ int s_n, s_word, s_rank;
    const int r = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int base = a.w.base[r], limit = base < 0 ? 0 : max(0, a.w.max_pages * a.w.page_size - base);
    const uint32_t* keep = a.keep + (size_t)r * a.words;
    const int blocks = a.p.n_layers * 2 * a.w.Hkv;
    const size_t elems = kv16_block_elems(a.w, HD);
    if (tid == 0) s_word = s_rank = 0;
    __syncthreads();
    for (;;) {
        // the next words' moves, 32 rows a word, listed by one warp
        if (warp == 0) {
            int n = 0, word = s_word, rank = s_rank;
            for (; word < a.words && n <= kCompactMoves - 32; ++word) {
                const int j = word * 32 + lane;
                const bool on = j < limit && (keep[word] >> lane & 1u);
                const unsigned all = __ballot_sync(0xffffffffu, on);
                const int to = rank + __popc(all & ((1u << lane) - 1));
                bool move = on && to != j;
                int p0 = -1, p1 = -1;
                if (move) {
                    p0 = kv16_page(a.w, r, base + j);
                    p1 = kv16_page(a.w, r, base + to);
                    move = p0 >= 0 && p1 >= 0;
                }
                const unsigned moves = __ballot_sync(0xffffffffu, move);
                if (move) {
                    const int at = n + __popc(moves & ((1u << lane) - 1));
                    src[at] = (uint32_t)p0 * a.w.page_size + (base + j) % a.w.page_size;
                    dst[at] = (uint32_t)p1 * a.w.page_size + (base + to) % a.w.page_size;
                }
                n += __popc(moves);
                rank += __popc(all);
            }
            if (lane == 0) { s_n = n; s_word = word; s_rank = rank; }
        }
        __syncthreads();
        const int n = s_n;
        const bool last = s_word >= a.words;
        for (int b = blockIdx.y * 8 + warp; b < blocks; b += gridDim.y * 8) {
            const int layer = b / (2 * a.w.Hkv), rest = b % (2 * a.w.Hkv);
            uint16_t* const at = a.p.pool + ((size_t)layer * a.w.n_pages * 2 * a.w.Hkv + rest) * elems;
            auto row_of = [&](uint32_t where) {
                const uint32_t page = where / a.w.page_size, slot = where % a.w.page_size;
                return at + (size_t)page * 2 * a.w.Hkv * elems + kv16_piece(slot, lane >> 3, HD);
            };
            for (int i0 = 0; i0 < n; i0 += 16) {
                uint4 x[2][kGroups];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int i = i0 + 8 * u + (lane & 7);
                    if (i < n) {
                        const uint16_t* const from = row_of(src[i]);
#pragma unroll
                        for (int c = 0; c < kGroups; ++c) x[u][c] = *reinterpret_cast<const uint4*>(from + c * 4 * 64);
                    }
                }
                __syncwarp();
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int i = i0 + 8 * u + (lane & 7);
                    if (i < n) {
                        uint16_t* const to = row_of(dst[i]);
#pragma unroll
                        for (int c = 0; c < kGroups; ++c) *reinterpret_cast<uint4*>(to + c * 4 * 64) = x[u][c];
                    }
                }
                __syncwarp();
            }
        }
        if (last) break;
        __syncthreads();
    }
    if (blockIdx.y == 0 && tid == 0) a.kept[r] = s_rank;
}

// ---- handing out pages
struct Kv16PlanArgs {
    const int32_t *src, *dst;   // fork: slots of the table; reserve: null, request i is slot i
    const int32_t *length, *own;
    int32_t *table, *refs, *pages;
    int n, n_slots, n_pages, max_pages, page_size;
    int32_t* scratch;           // [0] copies; then need[n], at[n]; free[cap]; copies [cap][2]
    int cap;
};
constexpr int kPlanThreads = 1024;

// Sum in front of the thread's v; whole CTA.  N: int where the sum of all threads' fits, else long long.
template <typename N>
__device__ __forceinline__ N block_scan(N v, N* s_warp, N& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    N inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const N t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = inc;
    __syncthreads();
    N w = s_warp[lane], s = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const N t = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += t;
    }
    total = __shfl_sync(0xffffffffu, s, 31);
    return __shfl_sync(0xffffffffu, s - w, warp) + inc - v;
}

// One CTA.  Pages [share, end) of request i are its own new ones: fork: copies of the source's pages there; reserve: those that are not there yet.
// Bound by its chain of loads and barriers: 7.6 us for 32 requests over 2048 pages, hidden by nothing; one CTA, since ids go out in order.
__global__ void __launch_bounds__(kPlanThreads) kv16_plan_kernel(const Kv16PlanArgs a) {
    __shared__ int s_warp[32];
    __shared__ long long s_wide[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t* const need = a.scratch + 1;
    int32_t* const at = need + a.n;
    int32_t* const free_ids = at + a.n;
    int32_t* const copies = free_ids + a.cap;
    auto there = [&](int id) { return id >= 0 && id < a.n_pages; };
    auto range = [&](int i, int& from, int& to, int& share, int& end) {          // false: the request's numbers make no sense
        from = a.src ? a.src[i] : i;
        to = a.dst ? a.dst[i] : i;
        const int length = a.length[i];
        if (from < 0 || from >= a.n_slots || to < 0 || to >= a.n_slots || length < 0 || (long long)length > (long long)a.max_pages * a.page_size) return false;
        if (a.src && from == to) return false;
        end = (length + a.page_size - 1) / a.page_size;
        share = 0;
        if (a.own) {
            const int own = a.own[i];
            if (own < 0) return false;
            share = min(own / a.page_size, end);
        }
        return true;
    };
    auto wants = [&](int from, int c) { return there(a.table[(size_t)from * a.max_pages + c]) == (a.src != nullptr); };
    // pages that every request needs, counted no further than the pool could serve; their sum is one of 64 bits
    for (int i = warp; i < a.n; i += kPlanThreads / 32) {
        int from, to, share, end, n = -1;
        if (range(i, from, to, share, end)) {
            n = 0;
            for (int c0 = share; c0 < end && n <= a.n_pages; c0 += 32) n += __popc(__ballot_sync(0xffffffffu, c0 + lane < end && wants(from, c0 + lane)));
        }
        if (lane == 0) need[i] = n;
    }
    __syncthreads();
    long long all = 0;
    for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
        long long total;
        const long long before = block_scan<long long>(i0 + tid < a.n ? max(need[i0 + tid], 0) : 0, s_wide, total);
        if (i0 + tid < a.n) at[i0 + tid] = (int)min(all + before, (long long)INT32_MAX);
        all += total;
    }
    const int wanted = (int)min(all, (long long)a.cap);
    // the lowest free ids, as many as are wanted
    int found = 0;
    for (int p0 = 0; p0 < a.n_pages && found < wanted; p0 += 4 * kPlanThreads) {
        const int p = p0 + 4 * tid;
        bool f[4];
        int mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = p + i < a.n_pages && a.refs[p + i] == 0;
            mine += f[i];
        }
        int total, to = found + block_scan<int>(mine, s_warp, total);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (f[i] && to < wanted) {
                copies[2 * to + 1] = -1;           // (none yet)
                free_ids[to++] = p + i;
            }
        found += total;
    }
    found = min(found, wanted);
    __syncthreads();
    if (found < all && tid == 0) {                 // not enough for all: in order, who still fits
        int used = 0;
        for (int i = 0; i < a.n; ++i) {
            const int n = need[i];
            if (n < 0) continue;
            if (n > found - used) { need[i] = -1; continue; }
            at[i] = used;
            used += n;
        }
        all = used;
    }
    __syncthreads();
    for (int i = warp; i < a.n; i += kPlanThreads / 32) {
        int from, to, share, end;
        const bool ok = need[i] >= 0;
        if (ok) {
            range(i, from, to, share, end);
            int32_t* const row = a.table + (size_t)to * a.max_pages;
            int next = at[i];
            const int stop = next + need[i];       // (a table that changes meanwhile -- a slot that is both source and target -- hands out no more)
            for (int c0 = 0; c0 < (a.src ? a.max_pages : end); c0 += 32) {
                const int c = c0 + lane;
                const bool in = c >= share && c < end, mine = in && wants(from, c);
                const unsigned votes = __ballot_sync(0xffffffffu, mine);
                const int k = next + __popc(votes & ((1u << lane) - 1));
                if (mine && k < stop) {
                    const int id = free_ids[k];
                    if (a.src) {
                        copies[2 * k] = a.table[(size_t)from * a.max_pages + c];
                        copies[2 * k + 1] = id;
                    }
                    a.refs[id] = 1;
                    row[c] = id;
                } else if (a.src && c < a.max_pages) {
                    int id = c < share ? a.table[(size_t)from * a.max_pages + c] : -1;
                    if (!there(id)) id = -1;
                    if (id >= 0) atomicAdd(a.refs + id, 1);
                    row[c] = id;
                }
                next += __popc(votes);
            }
        }
        if (lane == 0) a.pages[i] = ok ? end : -1;
    }
    if (tid == 0) a.scratch[0] = a.src ? (int)all : 0;
}

struct Kv16CopyArgs {
    uint4* pool;
    const int32_t* scratch;
    int n, cap, n_layers, n_pages;
    long long page_pieces;      // 16-byte pieces of a page's layer
};
constexpr int kCopyThreads = 256, kCopyUnroll = 4;

// The planned copies, in all layers.  Four pieces of 16 bytes a thread on their way at once, eight CTAs an SM: 76 us for 200 MB read and written
// (5.1 TB/s, behind the plan), read past the L2's order (__ldcs), since forks are written next, not their sources.
__global__ void __launch_bounds__(kCopyThreads) kv16_copy_kernel(const Kv16CopyArgs a) {
    pdl_wait();
    const int count = a.scratch[0];
    const int32_t* const copies = a.scratch + 1 + 2 * (size_t)a.n + a.cap;
    constexpr int kStep = kCopyThreads * kCopyUnroll;
    const long long chunks = (a.page_pieces + kStep - 1) / kStep, items = chunks * a.n_layers * count;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const long long chunk = it % chunks, rest = it / chunks;
        const int layer = (int)(rest % a.n_layers), e = (int)(rest / a.n_layers), from = copies[2 * e], to = copies[2 * e + 1];
        if (to < 0 || from < 0 || from >= a.n_pages) continue;       // (a table that changed under the plan)
        const uint4* src = a.pool + ((long long)layer * a.n_pages + from) * a.page_pieces;
        uint4* dst = a.pool + ((long long)layer * a.n_pages + to) * a.page_pieces;
        uint4 x[kCopyUnroll];
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u) {
            const long long i = chunk * kStep + u * kCopyThreads + threadIdx.x;
            if (i < a.page_pieces) x[u] = __ldcs(src + i);
        }
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u) {
            const long long i = chunk * kStep + u * kCopyThreads + threadIdx.x;
            if (i < a.page_pieces) dst[i] = x[u];
        }
    }
}

// Pages wholly behind a request's length are let go.  grid: requests.
__global__ void __launch_bounds__(128) kv16_release_kernel(const int32_t* length, int32_t* table, int32_t* refs, int n_pages, int max_pages, int page_size) {
    const int len = length[blockIdx.x];
    if (len < 0) return;
    int32_t* const row = table + (size_t)blockIdx.x * max_pages;
    for (int c = (len > 0 ? (len - 1) / page_size + 1 : 0) + threadIdx.x; c < max_pages; c += blockDim.x) {
        const int id = row[c];
        if (id >= 0 && id < n_pages) {
            atomicAdd(refs + id, -1);
            row[c] = -1;
        }
    }
}

}  // namespace pipesd
