// Attention over pages where row groups are small: the two streams of a CTA go through ranges of their own.
//
// The same products, tiles, ranges and shares as in attend16_pages.cuh, for bf16 and groups of at most 128 rows, which is what single tokens, chains and small
// trees have.  There both streams have the same triple and end it together; with few rows and short caches a CTA then spends more time between triples (sums
// read, joined and written, the next queries) than on tiles.  Here a stream has a range, a ring and a warp that fetches for it, and nothing to
// wait for in the other, so that one stream's tiles come in while the other ends a triple.
// Warps: 0-3 and 4-7 the streams' rows, 8 and 10 fetch a stream's keys and values, 9 and 11 issue its products.
//
// Bound by the cache's bytes behind long contexts (32 single tokens behind 256 to 4096 positions 71 us, 4.7 TB/s, 6.9 while tiles flow; one behind 131072 93 us,
// 5.8 TB/s), else by a stream's own chain: 2000 to 2700 clocks of one warp for a tile's 128 exponentials a row and what goes with them, 4500 for the one with the
// border, 1000 to 3000 until the next scores (heads of 128 leave a stream one place for keys), 6000 for a triple's end and the next one's beginning (256 behind 512: 128 us, 4.2 TB/s).
#pragma once
#include "attend16_pages.cuh"

namespace pipesd {

// A triple counts as much as three tiles beside its tiles (two to seven: within 3 us of 74 for 32 single tokens behind up to 4096 positions).
constexpr int kApartLead = 3 * kPagesTile;

template <int HD>
struct ApartShape {
    static constexpr int kKeys = 128, kTile = kKeys * HD * 2;
    static constexpr int kKSlots = HD == 128 ? 1 : 2, kVSlots = HD == 128 ? 1 : 3;       // of a stream
    static constexpr int kStream = (1 + kKSlots + kVSlots) * kTile;            // queries, keys, values
};
struct ApartStream {
    unsigned long long job_full[2], job_read[2], q_full, q_empty, k_full[2], k_empty[2], v_full[3], v_empty[3], s_full, p_full[2], o_full, done;
    PagesJob jobs[4];           // as in PagesControl
    int bad_lo[4], bad_hi[4];
    uint32_t present[32];
};
struct ApartControl {
    ApartStream stream[2];
    uint32_t tmem;
    int dead;
};
template <int HD>
constexpr int apart_smem() { return 2 * ApartShape<HD>::kStream + (int)sizeof(ApartControl); }

template <int HD>
__global__ void __launch_bounds__(kAttendThreads16, 1) pages_apart_kernel(const __grid_constant__ PagesArgs a) {
    using Shape = ApartShape<HD>;
    constexpr int kKeys = Shape::kKeys, kTile = Shape::kTile, kKSlots = Shape::kKSlots, kVSlots = Shape::kVSlots;
    constexpr uint32_t kIdescS = umma_idesc_bf16(128, kKeys, 0, 0), kIdescO = umma_idesc_bf16(128, HD, 0, 1);
    using KPlace = RingPlace<kKSlots>;
    using VPlace = RingPlace<kVSlots>;
    extern __shared__ __align__(128) unsigned char apart_memory[];
    ApartControl& control = *reinterpret_cast<ApartControl*>(apart_memory + 2 * Shape::kStream);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int s = warp < 8 ? warp >> 2 : (warp >> 1) & 1;                      // 8, 9: stream 0; 10, 11: stream 1
    unsigned char* const queries = apart_memory + s * Shape::kStream;
    unsigned char* const k_ring = queries + kTile;
    unsigned char* const v_ring = k_ring + kKSlots * kTile;
    ApartStream& c = control.stream[s];
    volatile int* const dead = &control.dead;
    pdl_launch_dependents();

    const bool fetches = warp == 8 || warp == 10, issues = warp == 9 || warp == 11;
    const int range = 2 * blockIdx.x + s;
    PagesWalk walk;
    if (fetches) walk.begin(a, range);             // (while the others set up)
    if (tid == 0) {
        for (int x = 0; x < 2; ++x) {
            ApartStream& b = control.stream[x];
            for (int i = 0; i < 2; ++i) {
                mbar_init(smem_u32(&b.job_full[i]), 1);
                mbar_init(smem_u32(&b.job_read[i]), 5);
                mbar_init(smem_u32(&b.p_full[i]), 4);
            }
            mbar_init(smem_u32(&b.q_full), 4);
            mbar_init(smem_u32(&b.q_empty), 1);
            for (int i = 0; i < kKSlots; ++i) {
                mbar_init(smem_u32(&b.k_full[i]), 1);
                mbar_init(smem_u32(&b.k_empty[i]), 1);
            }
            for (int i = 0; i < kVSlots; ++i) {
                mbar_init(smem_u32(&b.v_full[i]), 1);
                mbar_init(smem_u32(&b.v_empty[i]), 1);
            }
            mbar_init(smem_u32(&b.s_full), 1);
            mbar_init(smem_u32(&b.o_full), 1);
            mbar_init(smem_u32(&b.done), 1);
        }
        control.dead = blockIdx.x == a.gives_up;
        fence_mbar_init();
    }
    if (warp == 9) tmem_alloc(smem_u32(&control.tmem), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t s_tile = control.tmem + 128 * s, o_tile = control.tmem + 256 + HD * s;

    if (warp >= 8) {
        registers_fewer();
        if (fetches) {                             // ---- what there is to do; keys and values
            uint32_t count = 0;                    // tiles of all jobs whose keys were fetched, and whose values
            uint32_t values = 0;
            bool ok = true;
            // A job is found and said while the tiles of the one before are fetched.
            PagesJob ahead;
            PagesFetch fetch, fetch_next;
            bool find = true;
            for (int i = 0, j = 0, n = 0; ok;) {
                if (find) {
                    ahead = walk.next(a);
                    if (i >= 2) ok = warp_wait(smem_u32(&c.job_read[i & 1]), (i >> 1 & 1) ^ 1, dead);
                    if (ok && lane == 0) {
                        c.jobs[i & 3] = ahead;
                        c.bad_lo[i & 3] = INT32_MAX;
                        c.bad_hi[i & 3] = -1;
                        mbar_arrive(smem_u32(&c.job_full[i & 1]));
                    }
                    __syncwarp();
                    ++i;
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
                count += ok;
                const uint16_t* const v = t.src + a.w.Hkv * kv16_block_elems(a.w, HD);   // a page's values lie behind its keys
                ok = ok && pages_copy<HD, kKeys, kVSlots>(t, v, values, v_ring, c.v_full, c.v_empty, dead);
                values += ok;
                fetch.go_on<kKeys>(a);
                find = ++j == min(2, n);
            }
            if (!ok) {
                pages_drain<kKSlots>(count, c.k_full);
                pages_drain<kVSlots>(values, c.v_full);
            }
            if (lane == 0) a.splits[range] = walk.split;
        } else if (issues) {                       // ---- a stream's products
            if (elect_one()) {
                uint32_t k_no = 0, v_no = 0, p_phase = 0;
                bool ok = true;
                const uint64_t q_desc = umma_desc(smem_u32(queries), 128, HD * 16), k_desc = umma_desc(smem_u32(k_ring), 128, HD * 16),
                               v_desc = umma_desc(smem_u32(v_ring), HD * 16, 128);
                for (int i = 0; ok; ++i) {
                    ok = role_wait(smem_u32(&c.job_full[i & 1]), i >> 1 & 1, dead);
                    if (!ok) break;
                    const int n = c.jobs[i & 3].tiles;
                    mbar_arrive(smem_u32(&c.job_read[i & 1]));
                    if (n == 0) break;
                    ok = role_wait(smem_u32(&c.q_full), i & 1, dead);
                    auto scores = [&] {
                        const KPlace k(k_no++);
                        ok = ok && role_wait(smem_u32(&c.k_full[k.slot]), k.phase, dead);
                        if (!ok) return;
                        tc_fence_after();
                        const uint64_t tile = k_desc + k.slot * (kTile >> 4);
#pragma unroll
                        for (int x = 0; x < HD / 16; ++x) umma_bf16(s_tile, q_desc + x * 16, tile + x * 16, kIdescS, x > 0);
                        umma_commit(smem_u32(&c.s_full));
                        umma_commit(smem_u32(&c.k_empty[k.slot]));
                    };
                    for (int j = -1; j < n; ++j) {                             // a tile's sums, then the next one's scores
                        if (j >= 0) {
                            const VPlace v(v_no++);
                            const uint64_t tile = v_desc + v.slot * (kTile >> 4);
                            ok = ok && role_wait(smem_u32(&c.v_full[v.slot]), v.phase, dead);
                            for (int h = 0; h < 2; ++h) {
                                ok = ok && role_wait(smem_u32(&c.p_full[h]), p_phase, dead);
                                if (!ok) break;
                                tc_fence_after();
#pragma unroll
                                for (int x = 0; x < 4; ++x)
                                    umma_bf16_ta(o_tile, s_tile + 32 * h + 8 * x, tile + (4 * h + x) * HD * 2, kIdescO, j + h + x > 0);
                            }
                            p_phase ^= 1;
                            if (!ok) break;
                            umma_commit(smem_u32(&c.v_empty[v.slot]));
                        }
                        if (j + 1 < n) scores();
                        else umma_commit(smem_u32(&c.o_full));
                        if (!ok) break;
                        if (j + 2 == n) umma_commit(smem_u32(&c.q_empty));
                    }
                }
                // What was issued ends, and has arrived at its barriers, before the CTA goes.
                umma_commit(smem_u32(&c.done));
                mbar_wait(smem_u32(&c.done), 0);
            }
            __syncwarp();
        }
    } else {                                       // ---- a stream's rows
        registers_more();
        // Few rows are one warp's work: those of stream 1 lie 64 lanes further on, so that it is a warp of another scheduler
        // (256 single tokens behind 512 positions 146 -> 128 us).
        const int turn = 64 * s, row = (tid & 127) ^ turn;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16, s_tmem = s_tile + lanes, o_tmem = o_tile + lanes;
        uint32_t tile_no = 0, s_phase = 0, full_phase = 0;                     // tile_no: tiles of the jobs before
        int next = 1;                              // of the job behind the present one: 1: its queries are there, 0: there is none, -1: given up
        for (int i = -1; next == 1; ++i) {         // (-1: nothing yet)
            const PagesJob& job = c.jobs[i & 3];
            const int n = i < 0 ? 0 : job.tiles;
            const bool mine = row < job.n_rows, any = (row & ~31) < job.n_rows;
            const int rho = job.rho0 + (mine ? row : 0), node = rho / a.G;
            const int clear = a.mask ? job.base : job.base + job.rho0 / a.G + 1;         // positions that every row sees
            float ref = -INFINITY, sum = 0.f, none[1];
            bool ok = true, saw = false;           // saw: the row has seen a position
            for (int j = 0; j < n; ++j) {
                const int u = job.u0 + j, p0 = u * kKeys;
                uint32_t see[kKeys / 32];
                bool masked = p0 + kKeys > clear;
                if (masked) {
#pragma unroll
                    for (int w = 0; w < kKeys / 32; ++w) see[w] = pages_see(a, job, node, p0 + 32 * w);
                }
                ok = warp_wait(smem_u32(&c.s_full), s_phase, dead);
                s_phase ^= 1;
                if (!ok) break;
                tc_fence_after();
                const uint32_t present = c.present[(tile_no + j) & 31];        // eight positions a bit
                if (present != 0xffffu) {
                    pages_present(present, masked, see);
                    masked = true;
                }
                saw = saw || pages_any(masked, see);
                if (masked) {
                    const VPlace v(tile_no + j);
                    ok = warp_wait(smem_u32(&c.v_full[v.slot]), v.phase, dead);
                    if (!ok) break;
                    pages_clean<HD, kKeys>(v_ring + v.slot * kTile, row, job.base + job.n - p0, present, [&] {
                        atomicMin(&c.bad_lo[i & 3], u);
                        atomicMax(&c.bad_hi[i & 3], u);
                    });
                }
                auto given = [&](int h) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&c.p_full[h]));
                    __syncwarp();
                };
                if (any) {
                    softmax_tile<HD, kKeys, 1, false>(s_tmem, o_tmem, a.scale, j == 0, masked, see, ref, sum, none, given);
                } else {
                    given(0);
                    given(1);
                }
            }
            // ---- the next job's queries, whose scores are made while this one's sums are read
            if (ok) {
                next = -1;
                if (warp_wait(smem_u32(&c.job_full[(i + 1) & 1]), (i + 1) >> 1 & 1, dead)) {
                    const PagesJob& then = c.jobs[(i + 1) & 3];
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&c.job_read[(i + 1) & 1]));
                    if (then.tiles == 0) {
                        next = 0;
                    } else if (pages_queries<HD, uint16_t, 4>(a, then, warp & 3, queries, turn, i < 0, [&] { return warp_wait(smem_u32(&c.q_empty), i & 1, dead); })) {
                        next = 1;
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&c.q_full));
                    }
                }
            } else {
                next = -1;
            }
            if (i < 0) continue;
            // ---- the range's sums
            ok = next >= 0;
            if (ok) ok = warp_wait(smem_u32(&c.o_full), full_phase, dead);
            full_phase ^= 1;
            tile_no += n;
            tc_fence_after();
            const bool whole = job.whole;
            if (sum != sum) ref = INFINITY;        // (not what a row that sees nothing has: every factor of it is then a NaN)
            if (saw) ref = fmaxf(ref, kBlind);
            uint16_t* const out = static_cast<uint16_t*>(a.out) + (job.first + node) * a.out_stride + (size_t)(job.head * a.G + rho % a.G) * HD;
            float* const part = a.parts + (size_t)job.share * a.cap * (HD + 2);
            if (!ok) break;                        // a copy or a product that never came
            const int lo = *(volatile int*)&c.bad_lo[i & 3], hi = *(volatile int*)&c.bad_hi[i & 3];
            const bool nothing = ref == -INFINITY;
            const float factor = !whole ? 1.f : sum > 0.f ? 1.f / sum : NAN;
            if (any)
#pragma unroll 1
                for (int d = 0; d < HD; d += 32) {
                    uint32_t u[32];
                    tmem_ld32(o_tmem + d, u);
                    tmem_ld_wait32(u);
                    if (mine) {
                        float y[32];
#pragma unroll
                        for (int x = 0; x < 32; ++x) y[x] = nothing ? 0.f : __uint_as_float(u[x]) * factor;
                        if (lo <= hi)
#pragma unroll 1
                            for (int h = 0; h < 32; h += 16) {
                                const uint32_t bad = pages_bad<HD, kKeys>(a, job, node, lo, hi, d + h);
#pragma unroll
                                for (int x = 0; x < 32; ++x)
                                    if (x / 16 == h / 16 && (bad >> (x % 16) & 1u)) y[x] = NAN;
                            }
                        if (whole) {
                            pages_store16(out + d, a.out_wide, y);
                            pages_store16(out + d + 16, a.out_wide, y + 16);
                        } else {
#pragma unroll
                            for (int x = 0; x < 32; x += 4)
                                *reinterpret_cast<float4*>(part + ((size_t)(d + x) * a.cap + 4 * row)) = make_float4(y[x], y[x + 1], y[x + 2], y[x + 3]);
                        }
                    }
                    __syncwarp();
                }
            if (mine && !whole) {
                part[a.cap * HD + row] = ref;
                part[a.cap * (HD + 1) + row] = sum;
            }
            tc_fence_before();
        }
    }
    __syncthreads();
    if (warp < 8 && *dead)
        for (int x = 0; x < 2; ++x) pages_gave_up<HD, uint16_t>(a, 2 * blockIdx.x + x);
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(control.tmem, 512);
    }
}

}  // namespace pipesd
