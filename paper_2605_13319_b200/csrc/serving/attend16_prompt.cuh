// Causal attention of prompts packed one behind the other: out[i] = sum over j <= i of the prompt of softmax_j(scale q_i.k_j) v_j.
//
// Rows of a tile are (token, query head of the KV head's group) pairs, so that every tile reads one KV head's keys once for all of the group: T = 128 / G
// tokens by G heads, rounded down (G = 3: 126 rows of 128).  A job is two such tiles, 2 T consecutive tokens of a prompt by one KV head, each with a
// stream of its own (attend16_tile.cuh); both go through the same keys, 128 at a time, from the first up to their last token.
// A CTA per SM takes jobs in turn: sorted by length (block of tokens, last first; then prompts, then heads), dealt out back and forth, so that the CTAs'
// sums differ by less than a job.  Nothing is shared between CTAs: no atomics, no scratch.
// Warps: 0-3 and 4-7 the streams' rows, 8 fetches (copy engine, 128-byte swizzle), 9 and 11 issue the streams' products.
//
// Bound by the products and the exponentials alike (attend16_tile.cuh): 16384 tokens, 32 heads over 8 of 128, 2.2 TFLOP: 1.74 ms (1.26 PFLOP/s) in a
// short run, 2.0 under the power limit, the tensor pipe 62 % busy; 2048 tokens 45 us (0.76 PFLOP/s), of which 4 until the first tile and, for every job, 2000
// clocks for its outputs and 1300 more for the tile with the border; 8 prompts of 100 to 2000 tokens in heads of 64 166 us, where the exponentials weigh twice
// as much against the products.  Jobs of 2 T tokens: both streams share what is fetched, 128 bytes a clock and SM of shared memory are what
// S = Q K^T takes already.  Finding a job goes through all prompts' lengths some ten times: beside the tiles of the job before up to some
// hundred prompts, but 2000 prompts of three tokens take 1.3 ms.
#pragma once
#include "attend16_tile.cuh"

namespace pipesd {

struct PromptArgs {
    const int32_t* row0;
    const uint16_t* v;
    uint16_t* out;
    long long v_stride, out_stride;
    int n_req, rows, Hq, Hkv;
    float scale;                // times log2(e)
    int ctas;
    int gives_up;               // a CTA that has given up from the start (tests; -1: none)
};
struct PromptJob {
    int first, n, t0, head;     // the prompt's first row and length (0: no more jobs), the job's first token
};
constexpr int kPromptJobs = 2;

struct PromptControl {
    unsigned long long q_full, q_empty, full[16], empty[16], s_full[2], p_full[2][2], o_full[2], done[2];
    PromptJob jobs[kPromptJobs];
    int flags[kPromptJobs];     // a value of the job's last tiles was not finite
    uint32_t tmem;
    int dead;
};
template <int HD>
struct PromptShape {
    static constexpr int kTile = 128 * HD * 2, kStages = HD == 128 ? 5 : 8;
    static constexpr int kSmem = (2 + kStages) * kTile + (int)sizeof(PromptControl);
};

__device__ __forceinline__ void tensor3_g2s(uint32_t dst_smem, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst_smem), "l"(map),
                 "r"(bar), "r"(x), "r"(y), "r"(z)
                 : "memory");
}

// Tokens of prompt r (0 where its entries make no sense).
__device__ __forceinline__ int prompt_len(const PromptArgs& a, int r, int& first) {
    first = a.row0[r];
    const int end = a.row0[r + 1];
    return first < 0 || end < first || end > a.rows ? 0 : end - first;
}
// Blocks of `block` tokens with an index of `level` or more, over all prompts (whole warp; mine: of the lane's own prompt, r = lane).
__device__ __forceinline__ int prompt_blocks_from(const PromptArgs& a, int level, int block, int mine) {
    int sum = max(0, mine - level);
    for (int r = 32 + (threadIdx.x & 31); r < a.n_req; r += 32) {
        int first;
        const int b = (prompt_len(a, r, first) + block - 1) / block;
        sum += max(0, b - level);
    }
    return __reduce_add_sync(0xffffffffu, sum);
}
// Levels that there are, and the length and first row of prompt `lane` (whole warp).
__device__ __forceinline__ int prompt_levels(const PromptArgs& a, int block, int& n0, int& first0) {
    const int lane = threadIdx.x & 31;
    n0 = first0 = 0;
    if (lane < a.n_req) n0 = prompt_len(a, lane, first0);
    int longest = n0;
    for (int r = 32 + lane; r < a.n_req; r += 32) {
        int first;
        longest = max(longest, prompt_len(a, r, first));
    }
    return (__reduce_max_sync(0xffffffffu, longest) + block - 1) / block;
}
// A CTA's i-th job: the jobs, longest first, are dealt out back and forth (whole warp).  n = 0: there are not as many.
__device__ __forceinline__ PromptJob prompt_job(const PromptArgs& a, int i, int block, int levels, int n0, int first0) {
    const int mine = (n0 + block - 1) / block;
    const long long round = (long long)i * a.ctas, rank = i & 1 ? round + a.ctas - 1 - blockIdx.x : round + blockIdx.x;
    PromptJob job = {0, 0, 0, 0};
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = levels;                       // the largest level that at least rank + 1 jobs reach
    if ((long long)prompt_blocks_from(a, 0, block, mine) * a.Hkv <= rank) return job;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((long long)prompt_blocks_from(a, mid, block, mine) * a.Hkv > rank) lo = mid;
        else hi = mid;
    }
    const int index = (int)(rank - (long long)prompt_blocks_from(a, lo + 1, block, mine) * a.Hkv);
    int left = index / a.Hkv;
    job.head = index % a.Hkv;
    for (int r0 = 0; r0 < a.n_req; r0 += 32) {
        int first = first0, n = n0;
        if (r0 > 0) n = r0 + lane < a.n_req ? prompt_len(a, r0 + lane, first) : 0;
        const unsigned reach = __ballot_sync(0xffffffffu, n > lo * block);
        if (left < __popc(reach)) {
            const unsigned it = __ballot_sync(0xffffffffu, (reach >> lane & 1u) && __popc(reach & ((1u << lane) - 1)) == left);
            const int l = __ffs(it) - 1;
            job.first = __shfl_sync(0xffffffffu, first, l);
            job.n = __shfl_sync(0xffffffffu, n, l);
            job.t0 = lo * block;
            return job;
        }
        left -= __popc(reach);
    }
    return job;
}
// Tiles of 128 keys that stream s of a job goes through.
__device__ __forceinline__ int prompt_tiles(const PromptJob& job, int s, int T) {
    const int t = job.t0 + s * T;
    return t >= job.n ? 0 : (min(t + T, job.n) + 127) >> 7;
}

// Which of 16 columns hold something that is not finite in n rows of v (0 in shared memory, where the job's last tiles had it).
template <int HD>
__device__ __noinline__ uint32_t prompt_bad(const uint16_t* v, long long stride, int n) {
    uint32_t bad = 0;
    for (int i = 0; i < n; ++i) bad |= not_finite16(v + i * stride, 8);
    return bad;
}

// A CTA that gave up has no results: NaN for all of its jobs, those that were finished among them.  By the streams' warps, when all roles have ended.
template <int HD>
__device__ __noinline__ void prompt_gave_up(const PromptArgs& a) {
    const int G = a.Hq / a.Hkv, block = 2 * (128 / G);
    int n0, first0;
    const int levels = prompt_levels(a, block, n0, first0);
    for (int i = 0;; ++i) {
        const PromptJob job = prompt_job(a, i, block, levels, n0, first0);
        if (job.n == 0) break;
        for (int x = threadIdx.x; x < min(block, job.n - job.t0) * G; x += 256) {
            uint16_t* const out = a.out + (long long)(job.first + job.t0 + x / G) * a.out_stride + (job.head * G + x % G) * HD;
            for (int d = 0; d < HD; ++d) out[d] = 0x7fff;
        }
    }
}

template <int HD>
__global__ void __launch_bounds__(kAttendThreads16, 1)
    prompt_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ PromptArgs a) {
    using Shape = PromptShape<HD>;
    constexpr int kTile = Shape::kTile, kStages = Shape::kStages, kAtom = 128 * 128;      // an atom: 128 rows of 64 columns
    constexpr uint32_t kIdescS = umma_idesc_bf16(128, 128, 0, 0), kIdescO = umma_idesc_bf16(128, HD, 0, 1);
    extern __shared__ __align__(1024) unsigned char prompt_memory[];
    unsigned char* const smem = prompt_memory;
    unsigned char* const ring = smem + 2 * kTile;
    PromptControl& c = *reinterpret_cast<PromptControl*>(ring + kStages * kTile);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = a.Hq / a.Hkv, T = 128 / G;
    volatile int* const dead = &c.dead;

    PromptJob ahead;
    int levels = 0, n0 = 0, first0 = 0;            // n0, first0: of prompt `lane`
    if (warp == 8) {                               // (while the others set up)
        if (lane < 3) tensor_map_prefetch(lane == 0 ? &map_q : lane == 1 ? &map_k : &map_v);
        levels = prompt_levels(a, 2 * T, n0, first0);
        ahead = prompt_job(a, 0, 2 * T, levels, n0, first0);
    }
    if (tid == 0) {
        mbar_init(smem_u32(&c.q_full), 1);
        mbar_init(smem_u32(&c.q_empty), 10);     // both streams' products, and their warps when they have read the job
        for (int i = 0; i < kStages; ++i) {
            mbar_init(smem_u32(&c.full[i]), 1);
            mbar_init(smem_u32(&c.empty[i]), 2);
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
        if (warp == 8) {                               // ---- fetches
            uint32_t entry = 0;                        // of the ring, over all jobs
            bool ok = true;
            for (int i = 0; ok; ++i) {
                const PromptJob job = ahead;
                if (i > 0) ok = warp_wait(smem_u32(&c.q_empty), (i - 1) & 1, dead);
                if (!ok) break;
                const int tiles[2] = {prompt_tiles(job, 0, T), prompt_tiles(job, 1, T)}, n = max(tiles[0], tiles[1]);
                if (lane == 0) {
                    const uint32_t bar = smem_u32(&c.q_full);
                    c.jobs[i % kPromptJobs] = job;
                    c.flags[i % kPromptJobs] = 0;
                    if (job.n == 0) {
                        mbar_arrive(bar);
                    } else {
                        mbar_expect_tx(bar, (uint32_t)((tiles[1] ? 2 : 1) * (HD / 64) * T * G * 128));
                        for (int s = 0; s < 2; ++s)
                            for (int x = 0; tiles[s] && x < HD / 64; ++x)
                                tensor3_g2s(smem_u32(smem + s * kTile + x * kAtom), &map_q, 64 * x, job.head * G, job.first + job.t0 + s * T, bar);
                    }
                }
                __syncwarp();
                if (job.n == 0) break;
                for (int e = 0; e < 2 * n && ok; ++e) {
                    const RingPlace<kStages> place(entry);
                    if (entry >= kStages) ok = warp_wait(smem_u32(&c.empty[place.slot]), place.phase ^ 1, dead);
                    if (!ok) break;
                    if (lane == 0) {
                        const uint32_t full = smem_u32(&c.full[place.slot]);
                        mbar_expect_tx(full, kTile);
                        for (int x = 0; x < HD / 64; ++x)
                            tensor3_g2s(smem_u32(ring + place.slot * kTile + x * kAtom), e & 1 ? &map_v : &map_k, 64 * x, job.head, job.first + (e >> 1) * 128, full);
                    }
                    __syncwarp();
                    ++entry;
                }
                if (ok) ahead = prompt_job(a, i + 1, 2 * T, levels, n0, first0);        // (while the ring's tiles are gone through)
            }
            if (!ok && lane == 0) {                    // given up: the copies in flight are waited for
                for (uint32_t e = entry > kStages ? entry - kStages : 0; e < entry; ++e) mbar_wait(smem_u32(&c.full[e % kStages]), (e / kStages) & 1);
            }
            __syncwarp();
        } else if (warp == 9 || warp == 11) {      // ---- a stream's products
            if (elect_one()) {
                const int s = warp == 9 ? 0 : 1;
                using Place = RingPlace<kStages>;
                uint32_t entry = 0;                // of the ring, over all jobs: tile t's keys at entry + 2 t, its values behind them
                bool ok = true;
                const uint64_t q_desc = umma_desc_swizzled(smem_u32(smem + s * kTile), 16, 1024), k_desc = umma_desc_swizzled(smem_u32(ring), 16, 1024),
                               v_desc = umma_desc_swizzled(smem_u32(ring), kAtom, 1024);
                uint32_t p_phase = 0;              // of both halves
                auto arrived = [&](const Place& at) { return ok = ok && role_wait(smem_u32(&c.full[at.slot]), at.phase, dead); };
                auto release = [&](const Place& at) { umma_commit(smem_u32(&c.empty[at.slot])); };      // free when what was issued so far is done
                auto scores = [&](const Place& k) {
                    const uint64_t tile = k_desc + k.slot * (kTile >> 4);
#pragma unroll
                    for (int x = 0; x < HD / 16; ++x) {
                        const uint32_t at = ((x >> 2) * kAtom + (x & 3) * 32) >> 4;
                        umma_bf16(tmem + 128 * s, q_desc + at, tile + at, kIdescS, x > 0);
                    }
                    umma_commit(smem_u32(&c.s_full[s]));
                };
                auto sums = [&](const Place& v, bool first) {
                    const uint64_t tile = v_desc + v.slot * (kTile >> 4);
                    for (int h = 0; h < 2; ++h) {
                        ok = ok && role_wait(smem_u32(&c.p_full[s][h]), p_phase, dead);
                        if (!ok) return false;
                        tc_fence_after();
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            umma_bf16_ta(tmem + 256 + HD * s, tmem + 128 * s + 32 * h + 8 * x, tile + (4 * h + x) * (2048 >> 4), kIdescO, !first || h + x > 0);
                    }
                    p_phase ^= 1;
                    return true;
                };
                for (int i = 0; ok; ++i) {
                    ok = role_wait(smem_u32(&c.q_full), i & 1, dead);
                    if (!ok) break;
                    const PromptJob job = c.jobs[i % kPromptJobs];
                    if (job.n == 0) break;
                    const int n = prompt_tiles(job, s, T), tiles = max(n, prompt_tiles(job, 1 - s, T));
                    if (n > 0) {
                        const Place k(entry);
                        if (!arrived(k)) break;
                        tc_fence_after();
                        scores(k);
                        release(k);
                        if (n == 1) umma_commit(smem_u32(&c.q_empty));
                    } else {
                        mbar_arrive(smem_u32(&c.q_empty));
                    }
                    for (int j = 0; j < n; ++j) {
                        const Place v(entry + 2 * j + 1), k(entry + 2 * j + 2);
                        const bool more = j + 1 < n;
                        if (!arrived(v) || (more && !arrived(k))) break;
                        if (!sums(v, j == 0)) break;
                        if (more) scores(k);
                        else umma_commit(smem_u32(&c.o_full[s]));
                        release(v);
                        if (more) release(k);
                        if (j + 2 == n) umma_commit(smem_u32(&c.q_empty));
                    }
                    for (int e = 2 * n; e < 2 * tiles && ok; ++e) {            // what the other stream alone goes through
                        const Place at(entry + e);
                        if (arrived(at)) mbar_arrive(smem_u32(&c.empty[at.slot]));
                    }
                    entry += 2 * tiles;
                }
                // What was issued ends, and has arrived at its barriers, before the CTA goes.
                umma_commit(smem_u32(&c.done[s]));
                mbar_wait(smem_u32(&c.done[s]), 0);
            }
            __syncwarp();
        }
    } else {                                       // ---- a stream's rows
        registers_more();
        const int s = warp >> 2, row = tid & 127, token = row / G, g = row % G;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16, s_tmem = tmem + 128 * s + lanes, o_tmem = tmem + 256 + HD * s + lanes;
        uint32_t entry = 0, s_phase = 0, full_phase = 0;
        for (int i = 0;; ++i) {
            if (!warp_wait(smem_u32(&c.q_full), i & 1, dead)) break;
            const PromptJob job = c.jobs[i % kPromptJobs];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&c.q_empty));
            if (job.n == 0) break;
            const int tiles = prompt_tiles(job, s, T), all = max(prompt_tiles(job, 0, T), prompt_tiles(job, 1, T));
            const int t = job.t0 + s * T + token;  // this row's token
            const int clear = (job.t0 + s * T + 1) >> 7;                       // tiles that every row sees whole
            float ref = -INFINITY, sum = 0.f, none[1];
            bool ok = true;
            for (int j = 0; j < tiles; ++j) {
                uint32_t see[4];
                const bool masked = j >= clear;
                if (masked) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int n = t + 1 - (j * 128 + 32 * w);
                        see[w] = n >= 32 ? 0xffffffffu : (n <= 0 ? 0u : (1u << n) - 1u);
                    }
                    const uint32_t ev = entry + 2 * j + 1;
                    ok = warp_wait(smem_u32(&c.full[ev % kStages]), (ev / kStages) & 1, dead);
                    if (!ok) break;
                    const int all = job.t0 + s * T - j * 128;                  // the last key that every row sees
                    clean_values<kTile / 16>(
                        ring + ev % kStages * kTile, row,
                        [&](int p) {
                            const int key = p >> 3 & 127;
                            return key <= all ? kSeenByAll : j * 128 + key < job.n ? kSeenBySome : kNoKey;
                        },
                        [&] { *(volatile int*)&c.flags[i % kPromptJobs] = 1; });
                }
                ok = warp_wait(smem_u32(&c.s_full[s]), s_phase, dead);
                s_phase ^= 1;
                if (!ok) break;
                tc_fence_after();
                softmax_tile<HD, 128, 1, false>(s_tmem, o_tmem, a.scale, j == 0, masked, see, ref, sum, none, [&](int h) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&c.p_full[s][h]));
                    __syncwarp();
                });
            }
            entry += 2 * all;
            if (tiles == 0) continue;
            const bool mine = token < T && t < job.n;
            uint16_t* const out = a.out + (long long)(job.first + t) * a.out_stride + (job.head * G + g) * HD;
            if (ok) ok = warp_wait(smem_u32(&c.o_full[s]), full_phase, dead);
            full_phase ^= 1;
            if (!ok) break;                        // a copy or a product that never came
            tc_fence_after();
            const bool fix = *(volatile int*)&c.flags[i % kPromptJobs];
            const float inv = sum > 0.f ? 1.f / sum : NAN;      // (0: every score that the row sees is minus infinity; it sees itself)
            // 64 bytes of each of four rows by four lanes: a store of a piece by every row's own lane would cost a pass per row (a job of 64 columns
            // ends 1000 clocks sooner for it)
            const unsigned rows = __ballot_sync(0xffffffffu, mine);
            uint4* to[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) to[y] = reinterpret_cast<uint4*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(out), (lane & 28) + y)) + (lane & 3);
#pragma unroll 1
            for (int d = 0; d < HD; d += 32) {
                uint32_t u[32];
                tmem_ld32(o_tmem + d, u);
                tmem_ld_wait32(u);
                float o[32];
#pragma unroll
                for (int x = 0; x < 32; ++x) o[x] = __uint_as_float(u[x]) * inv;
                if (fix && mine) {
                    const int p = job.t0 >> 7 << 7;
#pragma unroll
                    for (int h = 0; h < 32; h += 16) {
                        const uint32_t bad = prompt_bad<HD>(a.v + (long long)(job.first + p) * a.v_stride + job.head * HD + d + h, a.v_stride, t + 1 - p);
#pragma unroll
                        for (int x = 0; x < 16; ++x)
                            if (bad >> x & 1u) o[h + x] = NAN;
                    }
                }
                __syncwarp();
                uint4 x[4] = {bf16x8(o), bf16x8(o + 8), bf16x8(o + 16), bf16x8(o + 24)};
                exchange_pieces(x);
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    if (rows >> ((lane & 28) + y) & 1u) to[y][d / 8] = x[y];
            }
            tc_fence_before();
        }
    }
    __syncthreads();
    if (warp < 8 && *dead) prompt_gave_up<HD>(a);
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

}  // namespace pipesd
