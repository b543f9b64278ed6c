// Attention of every request's new rows over its pages: positions in front of base, and of the new rows those that the row's mask names.
//
// Rows of a tile are (new row, query head of the KV head's group) pairs.  Work: the key tiles of all (request, KV head, row group) triples in a
// row, cut into equal ranges, one per CTA (one CTA per SM).  A triple that one CTA has whole is finished there; of others each CTA leaves its sums, which
// pages_merge_kernel adds up in CTA order.  No atomics, no state between calls.
// A row group has up to 256 rows in bf16.  More than 128: the CTA's two streams (attend16_tile.cuh) have 128 rows each and go through the same
// tiles; fewer: both have the same rows and take the tiles in turn, and their sums are joined at the end -- by the merge, or, where the CTA has all of
// the triple, in tensor memory, where each stream reads the other's, half of the columns each.  fp32: q and weights as three bf16 terms, groups of 128
// rows and tiles of 64 keys, since the terms of q fill shared memory and those of the weights tensor memory.
// Blocks of pages are operands of the products as they are (kv16.cuh): a bulk copy per page and tile, by the lanes of a warp for keys and one for values.
//
// Bound by the cache's bytes where rows are few and caches long: 32 rows behind 131040 positions (128 query rows by KV head) 108 us, 5.0 TB/s; by the chain
// of a triple's beginning and end where they are short: until the first scores 9000 clocks, 4500 from the last weights to the sums' end, 3300 to 3900 a tile of
// 256 rows between them (16 requests of 8 to 64 nodes behind 256 to 8192 positions: 118 us, 52 of bytes).  The merge adds 6 to 10.
#pragma once
#include <type_traits>

#include "attend16_tile.cuh"
#include "kv16.cuh"

namespace pipesd {

constexpr int kPagesSms = 148;
// What a triple counts in the ranges: a lead, and every tile; a tile whose rows fill both streams counts more.  As measured: 13000 clocks, 2200 and 3900.
// (No lead: 32 single tokens behind up to 4096 positions took 117 us instead of 83; 12 or 24 instead of 18: 16 ragged trees 122 instead of 120.)
constexpr int kPagesLead = 18, kPagesTile = 3, kPagesWideTile = 5;

template <int HD, typename T>
struct PagesShape {
    static constexpr bool kWide = sizeof(T) == 4;
    static constexpr int kTerms = kWide ? 3 : 1, kHalves = kWide ? 1 : 2, kKeys = kWide ? 64 : 128, kRows = kWide ? 128 : 256;
    static constexpr int kQTile = 128 * HD * 2, kQ = (kWide ? 3 : 2) * kQTile, kTile = kKeys * HD * 2;
    // A wait for a place's turn returns while the turn before it is still to come, too: who waits has to know that one to be over.  Keys: an even number of
    // places gives each stream places of its own where the streams take a job's tiles in turn, and behind a job all its keys have come before the next
    // one's queries are given.  Values, which a job's rows need not have waited for: each stream waits for all of them in order, the other stream's too,
    // and gives a place back when it has seen that it came, so that no place is two turns ahead of a wait.
    static constexpr int kKSlots = kWide ? (HD == 128 ? 4 : 8) : (HD == 128 ? 2 : 4), kVSlots = kWide ? (HD == 128 ? 4 : 8) : (HD == 128 ? 2 : 6);
    static_assert(kKSlots % 2 == 0, "");
    static constexpr int kSlots = kKSlots + kVSlots;
};
struct PagesArgs {
    Kv4Where w;
    Kv16Pool p;
    const void* q;
    void* out;
    long long q_stride, out_stride;
    int Hq, q_wide, out_wide;   // wide: 16-byte loads and stores
    float scale;                // times log2(e)
    const uint32_t* mask;       // [rows][words], null: a row sees the new rows up to itself
    int words;
    struct PagesSplit* splits;  // [ranges]
    float* parts;               // [own_shares * ranges] of {sums [HD / 4][cap][4], references [cap], denominators [cap]}: of a range's first triple and of a later one, by stream
    uint32_t page_mul, page_shift;                       // position / page_size = position * page_mul >> page_shift, for positions below 2^30
    int tile_pages, tile_over;  // keys / page_size and the remainder
    int G, cap;                 // query heads per KV head; query rows that a share has room for
    int log_keys, log_rows;     // of a tile and a row group
    int ranges, lead;           // into which the tiles are cut; what a triple counts beside its tiles
    int own_shares;             // of a range: two for each stream that goes through it
    int gives_up;               // a CTA that has given up from the start (tests; -1: none)
};
// The triple that goes on behind a range, as the merge needs it (rows 0: none).
struct PagesSplit {
    int first, head, rho0, rows, last, share, both, pad;     // last: its last range; share: where this one's sums are
};
struct PagesJob {
    int req, n, first, base, head, rho0, n_rows, tiles;      // tiles: 0 = no more jobs
    int whole, share;           // whole: all of the triple's; share: where its sums go else
    int u0;                     // the first of its tiles
    int pad;
};
struct PagesControl {
    unsigned long long job_full[2], job_read[2], q_full, q_empty, k_full[8], k_empty[8], v_full[8], v_empty[8], s_full[2], p_full[2][2], o_full[2], joint, done[2];
    PagesJob jobs[4];           // the slot of job i is said again for job i + 4, when everyone has read job i + 2
    int bad_lo[4], bad_hi[4];   // tiles in which a value was not finite
    uint32_t present[32];       // eight positions a bit
    float ref[2][128], sum[2][128];
    uint32_t tmem;
    int dead;
};
template <int HD, typename T>
constexpr int pages_smem() { return PagesShape<HD, T>::kQ + PagesShape<HD, T>::kSlots * PagesShape<HD, T>::kTile + (int)sizeof(PagesControl); }

// What a request adds to the sequence: tiles per triple, row groups, and what a triple counts.
struct PagesRequest {
    int n, first, base, units, groups;
};
__device__ __forceinline__ int pages_weight(int rows) { return rows > 128 ? kPagesWideTile : kPagesTile; }
__device__ __forceinline__ long long pages_count(const PagesArgs& a, int units, int rows) { return a.lead + (long long)units * pages_weight(rows); }
__device__ __forceinline__ PagesRequest pages_load(const PagesArgs& a, int r) {
    PagesRequest q = {0, 0, 0, 0, 0};
    if (r >= a.w.n_req) return q;
    q.n = kv4_rows(a.w, r, q.first, q.base);
    if (q.n <= 0) { q.n = 0; return q; }
    q.units = (q.base + q.n + (1 << a.log_keys) - 1) >> a.log_keys;
    q.groups = (q.n * a.G + (1 << a.log_rows) - 1) >> a.log_rows;
    return q;
}
__device__ __forceinline__ int pages_group_rows(const PagesArgs& a, const PagesRequest& q, int group) { return min(1 << a.log_rows, q.n * a.G - (group << a.log_rows)); }
// All heads' triples of a request: group by group within a head.
__device__ __forceinline__ long long pages_head(const PagesArgs& a, const PagesRequest& q) {
    if (q.groups == 0) return 0;
    return (q.groups - 1) * pages_count(a, q.units, 1 << a.log_rows) + pages_count(a, q.units, pages_group_rows(a, q, q.groups - 1));
}
__device__ __forceinline__ long long pages_scan(long long v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}
__device__ __forceinline__ long long pages_share(const PagesArgs& a, long long all) {
    return max((all + a.ranges - 1) / a.ranges, a.log_rows > 7 ? (long long)kPagesWideTile : (long long)kPagesTile);      // (every range within a triple has a tile of it)
}
// a / b of whole numbers, a >= 0, b > 0: the fp32 quotient is off by 2^-21 of itself and one, so that the loops run once at most below two
// million.  (A division of 64-bit integers takes several times as long, and this is what everyone waits for first.)
__device__ __forceinline__ long long pages_div(long long a, long long b) {
    long long q = (long long)__fdividef((float)a, (float)b), r = a - q * b;
    for (; r < 0; r += b) --q;
    for (; r >= b; r -= b) ++q;
    return q;
}
// The way through a range (whole warp).
struct PagesWalk {
    long long f, f0, f_end, share, off;
    int req, range;
    PagesSplit split;

    __device__ __forceinline__ void begin(const PagesArgs& a, int which) {
        const int lane = threadIdx.x & 31, per = (a.w.n_req + 31) / 32;        // a lane adds up `per` neighbouring requests
        long long mine = pages_head(a, pages_load(a, lane * per));
#pragma unroll 4
        for (int x = 1; x < per; ++x) mine += pages_head(a, pages_load(a, lane * per + x));
        mine *= a.w.Hkv;
        long long inc = pages_scan(mine);
        const long long all = __shfl_sync(0xffffffffu, inc, 31);
        share = pages_share(a, all);
        range = which;
        f = f0 = (long long)which * share;
        f_end = min(f + share, all);
        split = {};
        off = f;
        req = a.w.n_req;
        if (f >= f_end) return;
        int l = __ffs(__ballot_sync(0xffffffffu, off < inc)) - 1;
        off -= __shfl_sync(0xffffffffu, inc - mine, l);
        req = l * per;
        for (int x = 0; per > 1 && x < per; x += 32) {                         // among that lane's
            mine = x + lane < per ? pages_head(a, pages_load(a, l * per + x + lane)) * a.w.Hkv : 0;
            inc = pages_scan(mine);
            const unsigned hit = __ballot_sync(0xffffffffu, off < inc);
            if (hit) {
                const int h = __ffs(hit) - 1;
                off -= __shfl_sync(0xffffffffu, inc - mine, h);
                req = l * per + x + h;
                break;
            }
            off -= __shfl_sync(0xffffffffu, inc, 31);
        }
    }
    // The next triple of which the range has tiles; tiles 0: there is none.
    __device__ __forceinline__ PagesJob next(const PagesArgs& a) {
        PagesJob job = {};
        while (f < f_end && req < a.w.n_req) {
            const PagesRequest q = pages_load(a, req);
            const long long head = pages_head(a, q);
            if (off >= head * a.w.Hkv) { ++req; off = 0; continue; }           // (requests without rows have nothing)
            job.head = (int)pages_div(off, head);
            const long long full = pages_count(a, q.units, 1 << a.log_rows), in_head = off - job.head * head;
            const int group = (int)min(pages_div(in_head, full), (long long)q.groups - 1);
            job.n_rows = pages_group_rows(a, q, group);
            const int weight = pages_weight(job.n_rows);
            const long long start = f - (in_head - group * full), count = pages_count(a, q.units, job.n_rows);      // of the triple
            // tile t of it is the range's that start + lead + t * weight lies in
            auto tiles_before = [&](long long at) {
                const unsigned long long x = max(0ll, at - start - a.lead);
                return (int)min((unsigned long long)q.units, weight == kPagesTile ? (x + kPagesTile - 1) / kPagesTile : (x + kPagesWideTile - 1) / kPagesWideTile);
            };
            const int u0 = f > start ? tiles_before(f) : 0, u1 = tiles_before(f_end);
            const long long step = min(start + count, f_end) - f;
            off += step;
            f += step;
            if (u0 >= u1) continue;
            job.req = req; job.n = q.n; job.first = q.first; job.base = q.base;
            job.rho0 = group << a.log_rows;
            job.u0 = u0;
            job.whole = u0 == 0 && u1 == q.units;
            job.share = a.own_shares * range + (start > f0 ? a.own_shares / 2 : 0);
            // without a mask no row of the group sees what lies behind its last one
            const int seen = a.mask ? q.units : min(q.units, ((q.base + (job.rho0 + job.n_rows - 1) / a.G) >> a.log_keys) + 1);
            job.tiles = max(1, min(u1, seen) - u0);                            // (a tile at least: the others' sums are none)
            if (u0 == 0 && !job.whole)
                split = {q.first, job.head, job.rho0, job.n_rows, (int)pages_div(start + a.lead + (long long)(q.units - 1) * weight, share), job.share, job.n_rows > 128, 0};
            return job;
        }
        job.tiles = 0;
        return job;
    }
};

// Which of the 32 positions from `start` on row i of a request sees (bit 0: the first).
__device__ __forceinline__ uint32_t pages_see(const PagesArgs& a, const PagesJob& job, int i, int start) {
    const int total = job.base + job.n;
    auto below = [](int n) { return n >= 32 ? 0xffffffffu : (n <= 0 ? 0u : (1u << n) - 1u); };
    if (!a.mask) return below(min(job.base + i + 1, total) - start);
    const int j = start - job.base;                // the first's new row; below 0: the prefix
    if (j <= -32) return 0xffffffffu;
    const uint32_t* const m = a.mask + (size_t)(job.first + i) * a.words;
    const int w = j >> 5, sh = j & 31;             // (w is -1 where the border lies within)
    const uint32_t lo = w < 0 ? 0xffffffffu : (w < a.words ? m[w] : 0u), hi = w + 1 < a.words ? m[w + 1] : 0u;
    return __funnelshift_r(lo, hi, sh) & below(total - start);
}

// Eight neighbouring values of a query row as they are (wide: aligned to 16 bytes), and as the products take them.
template <int n, typename T>
__device__ __forceinline__ void pages_load8(const T* p, bool wide, uint4 (&x)[n]) {
    if (wide) {
#pragma unroll
        for (int h = 0; h < n; ++h) x[h] = reinterpret_cast<const uint4*>(p)[h];
    } else if constexpr (n == 1) {
        x[0] = make_uint4(pack2(p[0], p[1]), pack2(p[2], p[3]), pack2(p[4], p[5]), pack2(p[6], p[7]));
    } else {
        const uint32_t* const w = reinterpret_cast<const uint32_t*>(p);
#pragma unroll
        for (int h = 0; h < n; ++h) x[h] = make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]);
    }
}
__device__ __forceinline__ void pages_terms(const uint4 (&x)[1], uint4 (&terms)[1]) { terms[0] = x[0]; }
// Three terms of fp32 values: what a term leaves is exact.
__device__ __forceinline__ void pages_terms(const uint4 (&x)[2], uint4 (&terms)[3]) {
    float v[8] = {__uint_as_float(x[0].x), __uint_as_float(x[0].y), __uint_as_float(x[0].z), __uint_as_float(x[0].w),
                  __uint_as_float(x[1].x), __uint_as_float(x[1].y), __uint_as_float(x[1].z), __uint_as_float(x[1].w)};
#pragma unroll
    for (int t = 0; t < 3; ++t) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            v[2 * i] -= __uint_as_float(w[i] << 16);
            v[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
        }
        terms[t] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
// 16 neighbouring outputs.
__device__ __forceinline__ void pages_store16(uint16_t* p, bool wide, const float* y) {
    if (wide) {
#pragma unroll
        for (int x = 0; x < 16; x += 8) *reinterpret_cast<uint4*>(p + x) = bf16x8(y + x);
    } else {
#pragma unroll
        for (int x = 0; x < 16; ++x) p[x] = f32_to_bf16_bits(y[x]);
    }
}
__device__ __forceinline__ void pages_store16(float* p, bool wide, const float* y) {
    if (wide) {
#pragma unroll
        for (int x = 0; x < 16; x += 4) *reinterpret_cast<float4*>(p + x) = make_float4(y[x], y[x + 1], y[x + 2], y[x + 3]);
    } else {
#pragma unroll
        for (int x = 0; x < 16; ++x) p[x] = y[x];
    }
}
__device__ __forceinline__ void pages_store(uint16_t* p, float y) { *p = f32_to_bf16_bits(y); }
__device__ __forceinline__ void pages_store(float* p, float y) { *p = y; }

// Which of the 16 columns from d on hold something that is not finite in the values of tiles lo .. hi that row i sees (0 in shared memory, where these
// tiles were cleaned).  Tiles without a border and with all of their pages were not, and their products have it.  Eight positions at once: they are of
// one page, and lie side by side.  (Others wait meanwhile, two seconds at most: two tiles two million positions apart, 128 columns: 0.13.)
template <int HD, int kKeys>
__device__ __noinline__ uint32_t pages_bad(const PagesArgs& a, const PagesJob& job, int i, int lo, int hi, int d) {
    uint32_t bad = 0;
    for (int u = lo; u <= hi; ++u) {
        const int u0 = u * kKeys;
        bool cleaned = u0 + kKeys > job.base;
        for (int g = 0; !cleaned && g < kKeys; g += 8) cleaned = kv16_page(a.w, job.req, u0 + g) < 0;
        if (!cleaned) continue;
        for (int p0 = u0; p0 < u0 + kKeys; p0 += 32) {
            const uint32_t bits = pages_see(a, job, i, p0);
#pragma unroll 1
            for (int g = 0; g < 32; g += 8) {
                const int page = bits >> g & 0xffu ? kv16_page(a.w, job.req, p0 + g) : -1;
                if (page < 0) continue;
                const uint16_t* const at = kv16_block(a.p, a.w, a.p.layer, page, 1, job.head) + kv16_piece((p0 + g) % a.w.page_size, d / 8, HD);
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const uint32_t here = not_finite16(at + 8 * x, 64);
                    if (bits >> (g + x) & 1u) bad |= here;
                }
            }
        }
    }
    return bad;
}

// A warp's copies of one kind (kv 0: keys, 1: values) into a ring of its own, tile after tile over all jobs.  A lane per page that a tile touches; page
// ids come by windows of 32, looked up a window ahead.
struct PagesFetch {
    const uint16_t* block;      // of the pool's first page
    const int32_t* table;
    int total8, pages, p0, page0, off0, window, ids, ids_next;      // p0, page0, off0: the next tile's first position, its page, and where it lies in it

    __device__ __forceinline__ int look(int c) const { return c < pages ? table[c] : -1; }
    __device__ __forceinline__ void begin(const PagesArgs& a, const PagesJob& job, int kv) {
        const int lane = threadIdx.x & 31;
        auto page_of = [&](int pos) { return (int)((unsigned long long)(uint32_t)pos * a.page_mul >> a.page_shift); };
        table = a.w.table + (size_t)job.req * a.w.max_pages;
        block = kv16_block(a.p, a.w, a.p.layer, 0, kv, job.head);
        total8 = (job.base + job.n + 7) & ~7;
        pages = page_of(total8 - 1) + 1;
        p0 = job.u0 << a.log_keys;
        page0 = window = page_of(p0);
        off0 = p0 - page0 * a.w.page_size;
        ids = look(window + lane);
        ids_next = look(window + 32 + lane);
    }
    // The next tile's pages, one per lane: positions start .. end of the tile, and which groups of eight of the tile are there at all.
    struct Piece {
        int start, end;
        bool there;
        const uint16_t* src;
        uint32_t present;
    };
    template <int HD, int kKeys>
    __device__ __forceinline__ Piece look_up(const PagesArgs& a) const {
        const int lane = threadIdx.x & 31, ps = a.w.page_size;
        Piece t;
        t.start = max(0, lane * ps - off0);
        t.end = min(min(kKeys, (lane + 1) * ps - off0), total8 - p0);
        const int at = page0 - window + lane;
        const int x = __shfl_sync(0xffffffffu, ids, at & 31), y = __shfl_sync(0xffffffffu, ids_next, at & 31), id = at < 32 ? x : y;
        t.there = t.start < t.end && id >= 0 && id < a.w.n_pages;
        t.src = block + (t.there ? id * ((size_t)2 * a.w.Hkv * kv16_block_elems(a.w, HD)) + (size_t)(t.start + off0 - lane * ps) * HD : 0);
        t.present = __reduce_or_sync(0xffffffffu, t.there ? ((1u << ((t.end - t.start) >> 3)) - 1u) << (t.start >> 3) : 0u);
        return t;
    }
    template <int kKeys>
    __device__ __forceinline__ void go_on(const PagesArgs& a) {
        p0 += kKeys;
        page0 += a.tile_pages;
        off0 += a.tile_over;
        if (off0 >= a.w.page_size) { off0 -= a.w.page_size; ++page0; }
        if (page0 - window >= 32) {
            window += 32;
            ids = ids_next;
            ids_next = look(window + 32 + (threadIdx.x & 31));
        }
    }
};
// The count-th tile that comes into a ring, when its place is free.  False: given up.
template <int HD, int kKeys, int kSlots>
__device__ __forceinline__ bool pages_copy(const PagesFetch::Piece& t, const uint16_t* src, uint32_t count, unsigned char* ring, unsigned long long* full,
                                           unsigned long long* empty, volatile int* dead) {
    const RingPlace<kSlots> place(count);
    if (count >= kSlots && !warp_wait(smem_u32(&empty[place.slot]), place.phase ^ 1, dead)) return false;
    const uint32_t bar = smem_u32(&full[place.slot]);
    if ((threadIdx.x & 31) == 0) mbar_expect_tx(bar, (uint32_t)__popc(t.present) * (HD * 16));
    __syncwarp();
    if (t.there) bulk_g2s(smem_u32(ring + place.slot * (kKeys * HD * 2)) + (uint32_t)t.start * (HD * 2), src, (uint32_t)(t.end - t.start) * (HD * 2), bar);
    return true;
}
// Given up: the copies in flight are waited for.
template <int kSlots>
__device__ __forceinline__ void pages_drain(uint32_t count, unsigned long long* full) {
    for (uint32_t i = count > kSlots ? count - kSlots : 0; i < count; ++i) mbar_wait(smem_u32(&full[i % kSlots]), i / kSlots & 1);
}

// Keys of pages that are not there are not seen.
template <int kWords>
__device__ __forceinline__ void pages_present(uint32_t present, bool masked, uint32_t (&see)[kWords]) {
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        const uint32_t x = present >> (4 * w);
        const uint32_t there = (x & 1u ? 0xffu : 0u) | (x & 2u ? 0xff00u : 0u) | (x & 4u ? 0xff0000u : 0u) | (x & 8u ? 0xff000000u : 0u);
        see[w] = (masked ? see[w] : 0xffffffffu) & there;
    }
}
template <int kWords>
__device__ __forceinline__ bool pages_any(bool masked, const uint32_t (&see)[kWords]) {
    uint32_t any = 0;
#pragma unroll
    for (int w = 0; w < kWords; ++w) any |= see[w];
    return !masked || any;
}
// The reference of a row that has seen scores of minus infinity alone, with a sum of 0: any other reference outweighs it, and where there is none the row
// is a NaN.  (A row that has seen nothing has minus infinity, and gives 0.)
constexpr float kBlind = -3.402823466e38f;
template <int HD, int kKeys, typename Found>
__device__ __forceinline__ void pages_clean(unsigned char* tile, int row, int keys, uint32_t present, Found found) {
    clean_values<kKeys * HD / 8>(
        tile, row,
        [&](int p) {
            const int key = p / HD * 8 + p % 8;    // (a group of eight keys: HD pieces)
            return key < keys && (present >> (key >> 3) & 1u) ? kSeenBySome : kNoKey;    // (who sees all is not worth asking here)
        },
        found);
}

// A job's queries in the products' order, by kWarps warps: 8 x 4 pieces of 8 columns a warp and step.  Row r comes to row r ^ turn of the operand (turn: 0 or 64).
// empty, wait(): the place is free, wait for that.
template <int HD, typename T, int kWarps, typename Wait>
__device__ __forceinline__ bool pages_queries(const PagesArgs& a, const PagesJob& job, int warp, unsigned char* place, int turn, bool empty, Wait wait) {
    // A thread has a piece of every kRowStep-th row, several of them on their way at once.
    constexpr int kPieces = HD / 8, kTerms = PagesShape<HD, T>::kTerms, kQTile = PagesShape<HD, T>::kQTile, kRowStep = 32 * kWarps / kPieces;
    const int lane = threadIdx.x & 31, piece = warp % (kPieces / 4) * 4 + (lane >> 3), r0 = warp / (kPieces / 4) * 8 + (lane & 7);
    int node = (job.rho0 + r0) / a.G, g = (job.rho0 + r0) % a.G;
    const int node_step = kRowStep / a.G, g_step = kRowStep % a.G;
    const T* const q = static_cast<const T*>(a.q) + (size_t)job.head * a.G * HD + piece * 8;
    unsigned char* const to = place + piece * 128 + (r0 & 7) * 16;
    auto rows = [&](auto batch, bool wide) {
        constexpr int kBatch = decltype(batch)::value;
#pragma unroll 1
        for (int r = r0; r - r0 < job.n_rows; r += kBatch * kRowStep) {        // (as often for all of a warp)
            uint4 v[kBatch][sizeof(T) / 2];
#pragma unroll
            for (int y = 0; y < kBatch; ++y) {
                if (r + y * kRowStep < job.n_rows) pages_load8(q + (job.first + node) * a.q_stride + (size_t)g * HD, wide, v[y]);
                node += node_step;
                g += g_step;
                if (g >= a.G) { g -= a.G; ++node; }
            }
            if (!empty && !(empty = wait())) return;
#pragma unroll
            for (int y = 0; y < kBatch; ++y) {
                const int at = r + y * kRowStep;
                if (at < job.n_rows) {
                    uint4 terms[kTerms];
                    pages_terms(v[y], terms);
#pragma unroll
                    for (int t = 0; t < kTerms; ++t) *reinterpret_cast<uint4*>(to + (t + (at >> 7)) * kQTile + (((at & 127) ^ turn) >> 3) * HD * 16) = terms[t];
                }
            }
        }
    };
    if (a.q_wide) rows(std::integral_constant<int, 4>{}, true);                // (eight at once: more code to fetch, 32 single tokens behind up to 4096 positions 79 -> 84 us)
    else rows(std::integral_constant<int, 1>{}, false);
    return empty;
}

// A CTA that gave up has no results: NaN for all that its range holds, what was finished among it, and as the references of its shares, so that the
// merge gives NaN too.  By the streams' warps, when all roles have ended.
template <int HD, typename T>
__device__ __noinline__ void pages_gave_up(const PagesArgs& a, int range) {
    PagesWalk walk;
    walk.begin(a, range);
    for (;;) {
        const PagesJob job = walk.next(a);
        if (job.tiles == 0) break;
        for (int local = threadIdx.x; local < job.n_rows; local += 256) {
            const int rho = job.rho0 + local, slot = job.n_rows > 128 ? local & 127 : local;
            if (job.whole) {
                T* const out = static_cast<T*>(a.out) + (job.first + rho / a.G) * a.out_stride + (size_t)(job.head * a.G + rho % a.G) * HD;
                for (int d = 0; d < HD; ++d) pages_store(out + d, NAN);
            } else {
                for (int s = 0; s < a.own_shares / 2; ++s) a.parts[(size_t)(job.share + s) * a.cap * (HD + 2) + a.cap * HD + slot] = NAN;
            }
        }
    }
    if (threadIdx.x == 0) a.splits[range] = walk.split;
}

template <int HD, typename T>
__global__ void __launch_bounds__(kAttendThreads16, 1) pages_attend_kernel(const __grid_constant__ PagesArgs a) {
    using Shape = PagesShape<HD, T>;
    constexpr int kKeys = Shape::kKeys, kTile = Shape::kTile, kKSlots = Shape::kKSlots, kVSlots = Shape::kVSlots, kTerms = Shape::kTerms;
    constexpr int kHalves = Shape::kHalves;        // in which a tile's weights go over
    constexpr bool kOwn = Shape::kWide;            // the threads add up the tiles' sums
    constexpr uint32_t kIdescS = umma_idesc_bf16(128, kKeys, 0, 0), kIdescO = umma_idesc_bf16(128, HD, 0, 1);
    extern __shared__ __align__(128) unsigned char pages_memory[];
    unsigned char* const smem = pages_memory;
    unsigned char* const k_ring = smem + Shape::kQ;
    unsigned char* const v_ring = k_ring + kKSlots * kTile;
    PagesControl& c = *reinterpret_cast<PagesControl*>(v_ring + kVSlots * kTile);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = a.G;
    volatile int* const dead = &c.dead;
    pdl_launch_dependents();

    PagesWalk walk;
    if (warp == 8) walk.begin(a, blockIdx.x);                  // (while the others set up)
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&c.job_full[i]), 1);
            mbar_init(smem_u32(&c.job_read[i]), 11);       // all other roles' warps
        }
        mbar_init(smem_u32(&c.q_full), 8);
        mbar_init(smem_u32(&c.q_empty), 2);
        mbar_init(smem_u32(&c.joint), 8);
        for (int i = 0; i < kKSlots; ++i) {
            mbar_init(smem_u32(&c.k_full[i]), 1);
            mbar_init(smem_u32(&c.k_empty[i]), 2);
        }
        for (int i = 0; i < kVSlots; ++i) {
            mbar_init(smem_u32(&c.v_full[i]), 1);
            mbar_init(smem_u32(&c.v_empty[i]), 2);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_u32(&c.s_full[s]), 1);
            for (int h = 0; h < 2; ++h) mbar_init(smem_u32(&c.p_full[s][h]), 4);
            mbar_init(smem_u32(&c.o_full[s]), 1);
            mbar_init(smem_u32(&c.done[s]), 1);
        }
        c.dead = blockIdx.x == a.gives_up;
        fence_mbar_init();
    }
    if (warp == 9) tmem_alloc(smem_u32(&c.tmem), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = c.tmem;                  // stream s: scores and weights at 128 s, sums at 256 + HD s

    if (warp >= 8) {
        registers_fewer();
        if (warp == 8) {                               // ---- what there is to do, and keys
            uint32_t count = 0;                    // tiles of all jobs
            bool ok = true;
            auto say = [&](int i, const PagesJob& job) {
                if (i >= 2) ok = warp_wait(smem_u32(&c.job_read[i & 1]), (i >> 1 & 1) ^ 1, dead);
                if (ok && lane == 0) {
                    c.jobs[i & 3] = job;
                    c.bad_lo[i & 3] = INT32_MAX;
                    c.bad_hi[i & 3] = -1;
                    mbar_arrive(smem_u32(&c.job_full[i & 1]));
                }
                __syncwarp();
            };
            // A job is found and said while the tiles of the one before are fetched.
            PagesJob ahead;
            PagesFetch fetch, fetch_next;
            bool find = true;
            for (int i = 0, j = 0, n = 0; ok;) {
                if (find) {
                    ahead = walk.next(a);
                    say(i++, ahead);
                    if (ahead.tiles) fetch_next.begin(a, ahead, 0);
                    find = false;
                }
                if (j == n) {
                    n = ahead.tiles;
                    if (!ok || n == 0) break;
                    fetch = fetch_next;
                    j = 0;
                }
                const PagesFetch::Piece t = fetch.look_up<HD, kKeys>(a);
                if (lane == 0) c.present[count & 31] = t.present;
                ok = ok && pages_copy<HD, kKeys, kKSlots>(t, t.src, count, k_ring, c.k_full, c.k_empty, dead);
                fetch.go_on<kKeys>(a);
                count += ok;
                find = ++j == min(2, n);
            }
            if (!ok) pages_drain<kKSlots>(count, c.k_full);
            if (lane == 0) a.splits[blockIdx.x] = walk.split;
        } else if (warp == 10) {                   // ---- values
            uint32_t count = 0;
            bool ok = true;
            for (int i = 0; ok; ++i) {
                ok = warp_wait(smem_u32(&c.job_full[i & 1]), i >> 1 & 1, dead);
                if (!ok) break;
                const PagesJob& job = c.jobs[i & 3];
                const int n = job.tiles;
                PagesFetch fetch;
                if (n) fetch.begin(a, job, 1);
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c.job_read[i & 1]));
                if (n == 0) break;
                for (int j = 0; j < n && ok; ++j) {
                    const PagesFetch::Piece t = fetch.look_up<HD, kKeys>(a);
                    ok = pages_copy<HD, kKeys, kVSlots>(t, t.src, count, v_ring, c.v_full, c.v_empty, dead);
                    fetch.go_on<kKeys>(a);
                    count += ok;
                }
            }
            if (!ok) pages_drain<kVSlots>(count, c.v_full);
        } else if (warp == 9 || warp == 11) {      // ---- a stream's products
            if (elect_one()) {
                const int s = warp == 9 ? 0 : 1;
                using KPlace = RingPlace<kKSlots>;
                using VPlace = RingPlace<kVSlots>;
                uint32_t tile_no = 0;              // tiles of the jobs before
                bool ok = true;
                const uint64_t q_desc = umma_desc(smem_u32(smem), 128, HD * 16), k_desc = umma_desc(smem_u32(k_ring), 128, HD * 16),
                               v_desc = umma_desc(smem_u32(v_ring), HD * 16, 128);
                uint32_t p_phase = 0;              // of both halves
                auto k_there = [&](const KPlace& k) {
                    ok = ok && role_wait(smem_u32(&c.k_full[k.slot]), k.phase, dead);
                    if (ok) tc_fence_after();
                    return ok;
                };
                auto v_there = [&](const VPlace& v) { return ok = ok && role_wait(smem_u32(&c.v_full[v.slot]), v.phase, dead); };
                auto scores = [&](const KPlace& k, int q_tile) {
                    const uint64_t q = q_desc + (uint32_t)(q_tile * (Shape::kQTile >> 4)), tile = k_desc + k.slot * (kTile >> 4);
#pragma unroll
                    for (int t = 0; t < kTerms; ++t)
#pragma unroll
                        for (int x = 0; x < HD / 16; ++x)
                            umma_bf16(tmem + 128 * s, q + ((kTerms - 1 - t) * (Shape::kQTile >> 4) + x * 16), tile + x * 16, kIdescS, t + x > 0);
                    umma_commit(smem_u32(&c.s_full[s]));
                };
                auto see = [&](const VPlace& v) {          // a tile that the other stream takes
                    if (v_there(v)) mbar_arrive(smem_u32(&c.v_empty[v.slot]));
                };
                auto sums = [&](const VPlace& v, bool first) {
                    const uint64_t tile = v_desc + v.slot * (kTile >> 4);
                    for (int h = 0; h < kHalves; ++h) {
                        ok = ok && role_wait(smem_u32(&c.p_full[s][h]), p_phase, dead);
                        if (!ok) return false;
                        tc_fence_after();
#pragma unroll
                        for (int t = 0; t < kTerms; ++t)
#pragma unroll
                            for (int x = 0; x < 4; ++x)
                                umma_bf16_ta(tmem + 256 + HD * s, tmem + 128 * s + (kTerms - 1 - t) * (kKeys / 2) + 32 * h + 8 * x, tile + (4 * h + x) * HD * 2, kIdescO,
                                             (!kOwn && !first) || t + h + x > 0);
                    }
                    p_phase ^= 1;
                    return true;
                };
                for (int i = 0; ok; ++i) {
                    ok = role_wait(smem_u32(&c.job_full[i & 1]), i >> 1 & 1, dead);
                    if (!ok) break;
                    const int n = c.jobs[i & 3].tiles;
                    const bool both = c.jobs[i & 3].n_rows > 128;
                    mbar_arrive(smem_u32(&c.job_read[i & 1]));
                    if (n == 0) break;
                    // both: rows of q tile s, every tile of keys; else the same rows, tiles in turn
                    const int step = both ? 1 : 2, q_tile = both ? s : 0, j0 = both ? 0 : s;
                    // A place is free when what was issued so far is done, for both streams: of keys, the only one that uses it says so twice.
                    auto release_keys = [&](const KPlace& k) {
                        umma_commit(smem_u32(&c.k_empty[k.slot]));
                        if (!both) umma_commit(smem_u32(&c.k_empty[k.slot]));
                    };
                    ok = role_wait(smem_u32(&c.q_full), i & 1, dead);
                    if (!ok) break;
                    if (j0 < n) {
                        const KPlace k(tile_no + j0);
                        if (!k_there(k)) break;
                        scores(k, q_tile);
                        release_keys(k);
                    }
                    if (j0 + step >= n) umma_commit(smem_u32(&c.q_empty));
                    for (int j = j0; j < n; j += step) {
                        const bool more = j + step < n;
                        const KPlace k(tile_no + j + step);
                        const VPlace v(tile_no + j);
                        if (!both && j > 0) see(VPlace(tile_no + j - 1));
                        if (!v_there(v) || (more && !k_there(k))) break;
                        if (!sums(v, j == j0)) break;
                        if (more) scores(k, q_tile);
                        else umma_commit(smem_u32(&c.o_full[s]));
                        umma_commit(smem_u32(&c.v_empty[v.slot]));
                        if (more) release_keys(k);
                        if (more && j + 2 * step >= n) umma_commit(smem_u32(&c.q_empty));
                        if (!both && j + 2 == n) see(VPlace(tile_no + j + 1));
                    }
                    if (!both && j0 >= n) see(VPlace(tile_no));
                    tile_no += n;
                }
                // What was issued ends, and has arrived at its barriers, before the CTA goes.
                umma_commit(smem_u32(&c.done[s]));
                mbar_wait(smem_u32(&c.done[s]), 0);
            }
            __syncwarp();
        }
    } else {                                       // ---- a stream's rows
        registers_more();
        const int s = warp >> 2, row = tid & 127;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16, s_tmem = tmem + 128 * s + lanes, o_tmem = tmem + 256 + HD * s + lanes;
        using VPlace = RingPlace<kVSlots>;
        uint32_t tile_no = 0, s_phase = 0, full_phase = 0, joint_phase = 0;    // tile_no: tiles of the jobs before
        auto joint = [&] {                         // both streams' warps
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&c.joint));
            const bool there = warp_wait(smem_u32(&c.joint), joint_phase, dead);
            joint_phase ^= 1;
            return there;
        };
        // The queries of job i, in the products' order: 8 x 4 pieces of 8 columns a warp and step.  1: they are there, 0: there is no such job, -1: given up.
        auto queries = [&](int i) {
            if (!warp_wait(smem_u32(&c.job_full[i & 1]), i >> 1 & 1, dead)) return -1;
            const PagesJob& job = c.jobs[i & 3];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&c.job_read[i & 1]));
            if (job.tiles == 0) return 0;
            if (!pages_queries<HD, T, 8>(a, job, warp, smem, 0, i == 0, [&] { return warp_wait(smem_u32(&c.q_empty), (i - 1) & 1, dead); })) return -1;
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&c.q_full));
            return 1;
        };
        int next = 1;                              // of the job behind the present one
        for (int i = -1; next == 1; ++i) {         // (-1: nothing yet)
            const PagesJob& job = c.jobs[i & 3];
            const int n = i < 0 ? 0 : job.tiles;
            const bool both = job.n_rows > 128;
            bool ok = true;
            const int local = both ? 128 * s + row : row;                      // of the group's rows
            const bool mine = local < job.n_rows, any = (both ? 128 * s : 0) + 32 * (warp & 3) < job.n_rows;
            const int rho = job.rho0 + (mine ? local : 0), node = rho / G;
            // positions that every row of the stream sees
            const int clear = a.mask ? job.base : job.base + (job.rho0 + (both ? 128 * s : 0)) / G + 1;
            float ref = -INFINITY, sum = 0.f, own[kOwn ? HD : 1] = {};
            bool saw = false;                      // the row has seen a position
            for (int j = both ? 0 : s; j < n; j += both ? 1 : 2) {
                const int u = job.u0 + j, p0 = u * kKeys;
                uint32_t see[kKeys / 32];
                bool masked = p0 + kKeys > clear;
                if (masked) {
#pragma unroll
                    for (int w = 0; w < kKeys / 32; ++w) see[w] = pages_see(a, job, node, p0 + 32 * w);
                }
                ok = ok && warp_wait(smem_u32(&c.s_full[s]), s_phase, dead);
                s_phase ^= 1;
                if (!ok) break;
                tc_fence_after();
                const uint32_t present = c.present[(tile_no + j) & 31];        // eight positions a bit
                if (present != (kKeys == 128 ? 0xffffu : 0xffu)) {
                    pages_present(present, masked, see);
                    masked = true;
                }
                saw = saw || pages_any(masked, see);
                if (masked) {
                    const VPlace v(tile_no + j);
                    ok = warp_wait(smem_u32(&c.v_full[v.slot]), v.phase, dead);
                    if (!ok) break;
                    const int keys = job.base + job.n - p0;
                    pages_clean<HD, kKeys>(v_ring + v.slot * kTile, row, keys, present, [&] {
                        atomicMin(&c.bad_lo[i & 3], u);
                        atomicMax(&c.bad_hi[i & 3], u);
                    });
                }
                auto given = [&](int h) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&c.p_full[s][h]));
                    __syncwarp();
                };
                if (any) {
                    softmax_tile<HD, kKeys, kTerms, kOwn>(s_tmem, o_tmem, a.scale, both ? j == 0 : j < 2, masked, see, ref, sum, own, given);
                } else {
#pragma unroll
                    for (int h = 0; h < kHalves; ++h) given(h);
                }
            }
            // ---- the next job's queries, whose products begin while this one's sums are read
            next = ok ? queries(i + 1) : -1;
            if (i < 0) continue;
            ok = next >= 0;
            // ---- the range's sums
            const bool mine_has = both || s < n;
            if (ok && mine_has) ok = warp_wait(smem_u32(&c.o_full[s]), full_phase, dead);
            if (mine_has) full_phase ^= 1;
            tile_no += n;
            tc_fence_after();
            const bool whole = job.whole, join = whole && !both;               // join: both streams' sums are the triple's
            if constexpr (kOwn)
                if (ok && any && mine_has) {
                    own_sums<HD>(o_tmem, own);
#pragma unroll
                    for (int d = 0; d < HD; d += 16) tmem_st16(o_tmem + d, *reinterpret_cast<const float(*)[16]>(own + d));
                    tmem_st_wait();
                }
            if (sum != sum) ref = INFINITY;        // (not what a row that sees nothing has: every factor of it is then a NaN)
            if (saw) ref = fmaxf(ref, kBlind);
            if (ok && join) {
                c.ref[s][row] = ref;
                c.sum[s][row] = sum;
                tc_fence_before();
                ok = joint();
                tc_fence_after();
            }
            T* const out = static_cast<T*>(a.out) + (job.first + node) * a.out_stride + (size_t)(job.head * G + rho % G) * HD;
            float* const part = a.parts + (size_t)(job.share + s) * a.cap * (HD + 2);
            const int slot = both ? row : local;   // (a stream's rows: of 128)
            if (!ok) break;                        // a copy or a product that never came
            float f0 = 1.f, f1 = 1.f;              // what stream 0's and stream 1's sums are multiplied with
            bool none0 = ref == -INFINITY, none1 = true;                       // a stream that has seen nothing has none
            if (join) {
                const float r0 = c.ref[0][row], r1 = c.ref[1][row];
                none0 = r0 == -INFINITY;
                none1 = r1 == -INFINITY;
                ref = fmaxf(r0, r1);
                f0 = none0 ? 0.f : exp2_approx(r0 - ref);
                f1 = none1 ? 0.f : exp2_approx(r1 - ref);
                sum = c.sum[0][row] * f0 + c.sum[1][row] * f1;
            }
            const int lo = *(volatile int*)&c.bad_lo[i & 3], hi = *(volatile int*)&c.bad_hi[i & 3];
            if (whole) {
                const float inv = sum > 0.f ? 1.f / sum : ref == -INFINITY ? 0.f : NAN;
                f0 *= inv;
                f1 *= inv;
            }
            const int d0 = join ? s * (HD / 2) : 0, d1 = join ? d0 + HD / 2 : HD;
            const uint32_t from = tmem + 256 + HD * (join ? 0 : s) + lanes;
            if (any)
#pragma unroll 1
                for (int d = d0; d < d1; d += 16) {
                    float y[16], o[16];
                    tmem_ld16(from + d, y);
                    tmem_ld_wait16(y);
#pragma unroll
                    for (int x = 0; x < 16; ++x) y[x] = none0 ? 0.f : y[x] * f0;
                    if (join && n > 1) {
                        tmem_ld16(from + HD + d, o);
                        tmem_ld_wait16(o);
#pragma unroll
                        for (int x = 0; x < 16; ++x) y[x] = none1 ? y[x] : fmaf(o[x], f1, y[x]);
                    }
                    if (mine) {
                        if (lo <= hi) {
                            const uint32_t bad = pages_bad<HD, kKeys>(a, job, node, lo, hi, d);
#pragma unroll
                            for (int x = 0; x < 16; ++x)
                                if (bad >> x & 1u) y[x] = NAN;
                        }
                        if (whole) {
                            pages_store16(out + d, a.out_wide, y);
                        } else {
#pragma unroll
                            for (int x = 0; x < 16; x += 4)
                                *reinterpret_cast<float4*>(part + ((size_t)(d + x) * a.cap + 4 * slot)) = make_float4(y[x], y[x + 1], y[x + 2], y[x + 3]);
                        }
                    }
                    __syncwarp();
                }
            if (mine && !whole) {
                part[a.cap * HD + slot] = ref;
                part[a.cap * (HD + 1) + slot] = sum;
            }
            tc_fence_before();
            if (join && !joint()) break;           // both streams' sums have been read
        }
    }
    __syncthreads();
    if (warp < 8 && *dead) pages_gave_up<HD, T>(a, blockIdx.x);
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Adds up the shares of triples that several ranges had.  A CTA per (range that ends within a triple, 32 columns), rows by 32: a warp per eighth of the
// shares, a lane per row, whose shares lie side by side; each warp keeps a maximum of its own, and their sums are added in order.  grid: ranges, HD / 32, 1 to 4.  A
// chain of loads (record, shares) behind the last range: 6 to 10 us.  A warp per 32 rows where shares are few: 113 registers instead of 80, 3 to 8 us slower.
constexpr int kPagesMergeWarps = 8;
template <int HD, typename T>
__global__ void __launch_bounds__(32 * kPagesMergeWarps) pages_merge_kernel(const __grid_constant__ PagesArgs a) {
    __shared__ float s_top[kPagesMergeWarps][32], s_sum[kPagesMergeWarps][32];
    __shared__ float s_v[kPagesMergeWarps][32][33];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = a.G;
    // Launched with programmatic serialisation: behind this the shares are complete.  Every thread waits, those without work too.
    pdl_wait();
    // rows of requests that have no position: nothing to see
    if (blockIdx.y == 0 && blockIdx.z == 0)
        for (int r0 = blockIdx.x * 32; r0 < a.w.n_req; r0 += gridDim.x * 32) {
            int first = 0, base, n = 0, end = 0;
            if (r0 + lane < a.w.n_req) {
                n = kv4_rows(a.w, r0 + lane, first, base);
                end = min(a.w.row0[r0 + lane + 1], a.w.rows);
            }
            first = max(first, 0) + n;
            for (unsigned some = __ballot_sync(0xffffffffu, first < end); some; some &= some - 1) {
                const int l = __ffs(some) - 1, from = __shfl_sync(0xffffffffu, first, l), to = __shfl_sync(0xffffffffu, end, l);
                for (int row = from + warp; row < to; row += kPagesMergeWarps)
                    for (int d = lane; d < a.Hq * HD; d += 32) pages_store(static_cast<T*>(a.out) + row * a.out_stride + d, 0.f);
            }
        }
    const PagesSplit split = a.splits[blockIdx.x];
    const int c0 = blockIdx.x, streams = split.both ? 1 : a.own_shares / 2, shares = (split.last - c0 + 1) * streams, d0 = blockIdx.y * 32;
    for (int r0 = blockIdx.z * 32; r0 < split.rows; r0 += 32 * gridDim.z) {
        const int local = r0 + lane;
        const bool mine = local < split.rows;
        // A row's shares: of every CTA, and, unless each has rows of its own, of both streams.
        const int slot = mine ? (split.both ? local & 127 : local) : 0;
        auto share = [&](int i) {
            const int c = i / streams, s = split.both ? local >> 7 : i % streams;
            return a.parts + (size_t)((c == 0 ? split.share : a.own_shares * (c0 + c)) + s) * a.cap * (HD + 2);
        };
        float top = -INFINITY, sum = 0.f, v[32] = {};
#pragma unroll 2
        for (int i = warp; i < shares; i += kPagesMergeWarps) {
            const float* const p = share(i);
            const float r = p[a.cap * HD + slot], part = p[a.cap * (HD + 1) + slot];
            float4 y[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) y[x] = *reinterpret_cast<const float4*>(p + (size_t)(d0 + 4 * x) * a.cap + 4 * slot);
            if (r == -INFINITY) continue;          // a share that has seen nothing
            const float next = r == r ? fmaxf(top, r) : INFINITY;              // (a NaN where a share never came)
            const float keep = top == -INFINITY ? 0.f : exp2_approx(top - next), factor = exp2_approx(r - next);
            top = next;
            sum = fmaf(factor, part, sum * keep);
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                v[4 * x] = fmaf(factor, y[x].x, v[4 * x] * keep);
                v[4 * x + 1] = fmaf(factor, y[x].y, v[4 * x + 1] * keep);
                v[4 * x + 2] = fmaf(factor, y[x].z, v[4 * x + 2] * keep);
                v[4 * x + 3] = fmaf(factor, y[x].w, v[4 * x + 3] * keep);
            }
        }
        s_top[warp][lane] = top;
        s_sum[warp][lane] = sum;
#pragma unroll
        for (int x = 0; x < 32; ++x) s_v[warp][lane][x] = v[x];
        __syncthreads();
        // four rows a warp, a lane per column
        for (int r = warp; r < 32 && r0 + r < split.rows; r += kPagesMergeWarps) {
            float most = -INFINITY, y = 0.f, total = 0.f;
#pragma unroll
            for (int w = 0; w < kPagesMergeWarps; ++w) most = fmaxf(most, s_top[w][r]);
#pragma unroll
            for (int w = 0; w < kPagesMergeWarps; ++w) {
                const float factor = s_top[w][r] == -INFINITY ? 0.f : exp2_approx(s_top[w][r] - most);
                y = fmaf(factor, s_v[w][r][lane], y);
                total = fmaf(factor, s_sum[w][r], total);
            }
            const int rho = split.rho0 + r0 + r;
            const float inv = total > 0.f ? 1.f / total : most == -INFINITY ? 0.f : NAN;
            pages_store(static_cast<T*>(a.out) + (split.first + rho / G) * a.out_stride + (size_t)(split.head * G + rho % G) * HD + d0 + lane, y * inv);
        }
        __syncthreads();
    }
}

}  // namespace pipesd
