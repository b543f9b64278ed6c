// Attention of a chunk of query rows per request over its 4-bit pages (kv4.cuh):
//   out[row] = sum_j softmax_j(scale q.k_j) v_j over the positions j <= base + i of row i of its request.
//
// All query rows that share a KV head form one narrow operand (row = chunk row * G + query head of the group; 8 NT of them at a time).
// Per unit of 16 positions, with keys and then value columns on the M side of mma.m16n8k16 (fp16 operands, fp32 sums):
//   S^T[16 keys x rows] = sum over groups of s_key,group * (codes . Q_group), and, by one more product (bf16), zeros . (sums of Q
//                         over the groups, as three bf16 terms)
//   O^T[HD x rows]     += (codes - 8)^T . (P * s_key,group),   and one more product [z + 8 s of the groups; ones] . P, which is the
//                         middles' share of the output and the denominators, both of the very P (rounded) that P * s is made of.
// No value is ever dequantised.  A key's code goes into the tensor cores as the subnormal that its bits are, n * 2^-24; Q is
// scaled by a power of two per row (largest entry near 2^15).  A value's code is centred on the way, by one fused multiply-add per
// two codes (exact): outputs are means of many values, whose sum of uncentred codes would be hundreds of times the result and
// its rounding as well.  fp16 keeps 11 bits of P, of P * s and of the middles (bf16 outputs: an eighth of them one step beside the nearest,
// error against 64 bits 1.68e-3 where rounding alone has 1.67e-3; a second term of P would double the values' products); the scales
// and middles are taken relative to a power of two that fits the warp's first unit, and rescaled (like a row's exponentials, which are
// relative to a score of that unit) when one exceeds it by 2^6 (2^4).
// fp32 queries and outputs (kSplit): Q, P, P * s and the middles as two fp16 terms each, 22 bits of mantissa; a unit's products go to the
// running sums by ordinary additions, which round to nearest, and keys' codes are centred too, middles times sums of Q (fp32) added beside
// (the tensor pipe truncates where it adds: error 2.1e-6 over long caches without either, 1.2e-6 with the additions, 2.5e-7 with both;
// 155 ragged rows take 9 us of 206 more for the one, 3 of 201 for the other).  An exponential's argument stays near 0, P's power of two comes after.
// Work: the units of all (request, KV head, row group) triples in a row, cut into equal ranges, one per CTA; the warps of a CTA take
// its units in turn.  A triple that one CTA has whole is finished there; of others each CTA leaves (O, reference, denominator),
// which kv4_merge_kernel adds up in CTA order.  No atomics, no state between calls.
// Every warp has a ring of kAttendStages units of its own, filled by one bulk copy per unit: nothing synchronises the warps of a CTA
// until its range, or a triple in it, ends.
//
// What bounds it.  Few query rows: instructions, 370 a unit and tile (80 of them the codes' unpacking, on a pipe of half rate), at 2.4 a cycle
// of four; 1 row of 131072 positions over 8 heads 53 us, 168 MB, 3.2 TB/s (0.48 of the measured copy).  Short caches: a chain of 12 us (tables,
// copies, queries, products, exchange, merge).  Many query rows: what every score costs in instructions, and the warp-level products.  The
// same on tcgen05 -- a tile of 128 positions unpacked into tensor memory for 64 rows, a thread per key -- was slower at every number of
// rows (9 rows of 32 heads 170 us for 66, 68 rows over 8 heads 117 for 80, 160 rows 193 for 151): its products take a tenth of the time, and
// scores, exponentials and both unpackings, with barriers between them, more than here.
#pragma once
#include "kv4.cuh"

namespace pipesd {

// Row tiles of a CTA (NT), and what fits an SM: sixteen warps of 128 registers with one, twelve of 168 with two (which unpack a unit's codes
// for twice the rows).  More, at one CTA of eight warps per SM, were slower at every number of rows.
__host__ __device__ constexpr int attend_warps(int nt) { return nt == 1 ? 8 : 4; }
__host__ __device__ constexpr int attend_ctas_per_sm(int nt) { return nt == 1 ? 2 : 3; }
constexpr int kAttendSms = 148;
constexpr int kAttendMinUnits = 8;                 // of a CTA
constexpr float kAttendNone = -3.3e38f;            // reference of a row that has seen nothing: below every score
constexpr float kAttendExcess = 4.f;               // log2 units by which a score may exceed its row's reference: P <= 16
constexpr float kAttendScaleExcess = 64.f;         // factor by which a scale may exceed its warp's unit
// fp16 has 40 binades for a number and its second term: P is taken times 2^6 (up to 2^10), scales times 1 / 4 (up to 2^5: their 8 bits are exact
// down to 2^-16 of the first unit's; products up to 2^15), middles times 2^8 (up to 2^15).
constexpr float kAttendUpP = 6.f, kAttendUpPFactor = 64.f, kAttendUpScale = 0.25f, kAttendUpMiddle = 256.f;
constexpr int kAttendStages = 4;
constexpr float kTwo9 = 512.f, kTwoM24 = 5.9604644775390625e-8f;

struct Kv4AttendArgs {
    Kv4Where w;
    unsigned char* pool;
    const void* q;
    void* out;
    long long q_stride, out_stride;
    int Hq;
    float scale;               // times log2(e)
    float* parts;              // [2 * CTAs][8 NT (HD + 2)]
    int ctas, rows_cap, heads; // rows_cap: query rows of a triple; heads: of a row that a warp or CTA of the merge takes
};

// What a request adds to the flat sequence of units: units per triple and triples.
__device__ __forceinline__ void attend_load(const Kv4AttendArgs& a, int r, int& n, int& first, int& base, int& units, int& groups) {
    n = first = base = units = groups = 0;
    if (r >= a.w.n_req) return;
    n = kv4_rows(a.w, r, first, base);
    if (n <= 0) { n = 0; return; }
    units = (base + n + kKv4Unit - 1) / kKv4Unit;
    groups = (n * (a.Hq / a.w.Hkv) + a.rows_cap - 1) / a.rows_cap;
}
__device__ __forceinline__ long long warp_scan_i64(long long v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}
// Units of all requests, and of those before request `upto` (whole warp).
__device__ __forceinline__ long long attend_total(const Kv4AttendArgs& a, int upto, long long& before) {
    const int lane = threadIdx.x & 31;
    long long all = 0;
    before = 0;
    for (int r0 = 0; r0 < a.w.n_req; r0 += 32) {
        int n, first, base, units, groups;
        attend_load(a, r0 + lane, n, first, base, units, groups);
        const long long mine = (long long)units * groups * a.w.Hkv, inc = warp_scan_i64(mine);
        if (upto >= r0 && upto < r0 + 32) before = all + __shfl_sync(0xffffffffu, inc - mine, upto - r0);
        all += __shfl_sync(0xffffffffu, inc, 31);
    }
    return all;
}
// Units of a CTA: an equal share, at least kAttendMinUnits.
__device__ __forceinline__ long long attend_share(const Kv4AttendArgs& a, long long all) {
    const long long per = (all + a.ctas - 1) / a.ctas;
    return per < kAttendMinUnits ? kAttendMinUnits : per;
}
// This CTA's range [f, f_end) of the flat sequence, and where it begins: `off` units into request `req`.  False: it has none.  (Whole
// warps; the sums over the first 32 requests are kept for the search.)
__device__ __forceinline__ bool attend_begin(const Kv4AttendArgs& a, long long& f, long long& f_end, int& req, long long& off) {
    const int lane = threadIdx.x & 31;
    auto chunk = [&](int r0, long long& mine) {
        int n, first, base, units, groups;
        attend_load(a, r0 + lane, n, first, base, units, groups);
        mine = (long long)units * groups * a.w.Hkv;
        return warp_scan_i64(mine);
    };
    long long mine0;
    const long long inc0 = chunk(0, mine0);
    long long all = __shfl_sync(0xffffffffu, inc0, 31);
    for (int r0 = 32; r0 < a.w.n_req; r0 += 32) {
        long long mine;
        all += __shfl_sync(0xffffffffu, chunk(r0, mine), 31);
    }
    const long long share = attend_share(a, all);
    f = (long long)blockIdx.x * share;
    f_end = f + share < all ? f + share : all;
    if (f >= f_end) return false;
    long long left = f;
    for (int r0 = 0;; r0 += 32) {
        long long mine = mine0, inc = inc0;
        if (r0 > 0) inc = chunk(r0, mine);
        const unsigned hit = __ballot_sync(0xffffffffu, left < inc);
        if (hit) {
            const int l = __ffs(hit) - 1;
            req = r0 + l;
            off = left - __shfl_sync(0xffffffffu, inc - mine, l);
            return true;
        }
        left -= __shfl_sync(0xffffffffu, inc, 31);
    }
}

template <int HD, int NT, bool kSplit>
struct AttendSmem {
    static constexpr int kRows = 8 * NT, kGroups = HD / kKv4Group, kTerms = kSplit ? 2 : 1, kAttendWarps = attend_warps(NT);
    uint2 q[HD / 16][NT][kTerms][32];              // B fragments
    uint2 qsum[NT][32];                            // sums of the groups' (scaled) entries as a B fragment, bf16: k = 4 term + group; kSplit: fp32 [group][row]
    float qc[kRows];                               // what a row's scores are multiplied with
    int horizon[kRows];                            // last visible position; -1 for a row that is none
    float ref[kAttendWarps][kRows], sum[kAttendWarps][kRows];
    unsigned long long bars[kAttendWarps][kAttendStages];
    union alignas(16) {                            // the ring is empty when the warps' shares are added up
        unsigned char ring[kAttendWarps][kAttendStages][20 * HD];
        float o[kAttendWarps][kRows][HD + 4];      // padded: the fragments' stores then hit 32 banks
    };
};

__device__ __forceinline__ float warp_max_f32(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float attend_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t attend_transpose(uint32_t v) {       // 8 x 8 of 16 bits across the warp
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t attend_mul2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t attend_fma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t attend_pack(float x, float y) {      // fp16 pair, the first in the low half
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
    return r;
}
__device__ __forceinline__ float f16_lo(uint32_t v) {
    float r;
    asm("{.reg .b16 l, h; mov.b32 {l, h}, %1; cvt.f32.f16 %0, l;}" : "=f"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ float f16_hi(uint32_t v) {
    float r;
    asm("{.reg .b16 l, h; mov.b32 {l, h}, %1; cvt.f32.f16 %0, h;}" : "=f"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void attend_split(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = attend_pack(x, y);
    lo = attend_pack(x - f16_lo(hi), y - f16_hi(hi));
}
// (codes - 8) / 512 of a register of codes * 2^-24 (even nibbles) or 16 codes * 2^-24 (odd ones); exact.
template <bool kOdd>
__device__ __forceinline__ uint32_t attend_centre(uint32_t n) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(n), "r"(kOdd ? 0x68006800u : 0x78007800u), "r"(0xa400a400u));
    return r;
}
// D(16 x 8, fp32) += A(16 x 16, fp16, row) . B(16 x 8, fp16, col)
__device__ __forceinline__ void attend_mma(float (&c)[4], const uint4& a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ float attend_in(float v) { return v; }
__device__ __forceinline__ float attend_in(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ void attend_out(float* p, float v) { *p = v; }
__device__ __forceinline__ void attend_out(uint16_t* p, float v) { *p = f32_to_bf16_bits(v); }

template <bool kBf16>
__device__ __forceinline__ void attend_mma_first(float (&c)[4], const uint4& a, uint32_t b0, uint32_t b1) {      // D = A . B
    if (kBf16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
                     : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                     : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
                     : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                     : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1), "f"(0.f));
}
// Power of two (as its float) that a unit's scales and middles up to m are taken relative to.
__device__ __forceinline__ float attend_unit_scale(float m) { return __uint_as_float(max(__float_as_uint(m) & 0x7f800000u, 27u << 23)); }

// grid: a.ctas, block 32 attend_warps(NT), dynamic shared memory: one AttendSmem.
template <int HD, int NT, typename T>
__global__ void __launch_bounds__(32 * attend_warps(NT), attend_ctas_per_sm(NT)) kv4_attend_kernel(const Kv4AttendArgs a) {
    constexpr bool kSplit = sizeof(T) == 4;
    using SM = AttendSmem<HD, NT, kSplit>;
    constexpr int kGroups = SM::kGroups, kRows = SM::kRows, kTerms = SM::kTerms, kTiles = HD / 16;
    constexpr int kAttendWarps = SM::kAttendWarps, kAttendThreads = 32 * kAttendWarps;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SM& sm = *reinterpret_cast<SM*>(smem_raw);
    float* const qsums = reinterpret_cast<float*>(sm.qsum);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int G = a.Hq / a.w.Hkv;
    pdl_launch_dependents();

    if (lane == 0)
        for (int i = 0; i < kAttendStages; ++i) mbar_init(smem_u32(&sm.bars[warp][i]), 1);
    fence_mbar_init();
    __syncwarp();
    uint32_t parity = 0, mapped = 0;               // of the ring's barriers; which of its units are there
    bool failed = false;
    long long f, f_end, off;
    int req;
    if (!attend_begin(a, f, f_end, req, off)) return;
    const long long f_cta = f;
    while (f < f_end) {
        int n, first, base, units, groups;
        attend_load(a, req, n, first, base, units, groups);
        if (off >= (long long)units * groups * a.w.Hkv) { ++req; off = 0; continue; }      // (requests without rows have no units)
        const int triple = (int)(off / units), u0 = (int)(off % units);
        const int u1 = (int)((long long)units - u0 < f_end - f ? units : u0 + (f_end - f));
        const int head = triple / groups, rho0 = triple % groups * kRows;
        const int n_rows = min(kRows, n * G - rho0);

        const int seen_all = base + rho0 / G;                                // positions up to here are visible to every row
        const int seen_any = base + (rho0 + n_rows - 1) / G;
        float unit_scale = 0.f;                    // 0: nothing seen yet
        const int ulast = min(u1, seen_any / kKv4Unit + 1);                  // units from here on are hidden from every row
        const unsigned char* mine = nullptr;       // lane i: where the unit (it & ~31) + i of this warp is
        auto locate = [&](int it) {
            const int u = u0 + warp + kAttendWarps * (it + lane);
            mine = u < ulast ? kv4_unit(a.pool, a.w, req, head, u, HD) : nullptr;
        };
        const int n_it = ulast - u0 - warp > 0 ? (ulast - u0 - warp + kAttendWarps - 1) / kAttendWarps : 0;
        auto request = [&](int it) {               // whole warp; it < n_it
            if ((it & 31) == 0) locate(it);
            const unsigned char* src = reinterpret_cast<const unsigned char*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), it & 31));
            const int st = it % kAttendStages;
            if (lane == 0) {
                const uint32_t bar = smem_u32(&sm.bars[warp][st]);
                if (src) {
                    mbar_expect_tx(bar, 20 * HD);
                    bulk_g2s(smem_u32(sm.ring[warp][st]), src, 20 * HD, bar);
                } else {
                    mbar_arrive(bar);
                }
            }
            mapped = (mapped & ~(1u << st)) | (src ? 1u << st : 0u);
        };
        for (int it = 0; it < min(n_it, kAttendStages); ++it) request(it);       // (on their way while the queries are laid out)
        // ---- queries of the triple: normalised, split, in fragment order; one warp per row
        for (int row = warp; row < kRows; row += kAttendWarps) {
            constexpr int kE = HD / 32;            // neighbouring columns of a lane
            float x[kE];
            float mx = 0.f;
            const int rho = rho0 + row;
            if (row < n_rows) {
                const T* src = static_cast<const T*>(a.q) + (size_t)(first + rho / G) * a.q_stride + (size_t)(head * G + rho % G) * HD + lane * kE;
#pragma unroll
                for (int i = 0; i < kE; ++i) { x[i] = attend_in(src[i]); mx = fmaxf(mx, fabsf(x[i])); }
            } else {
#pragma unroll
                for (int i = 0; i < kE; ++i) x[i] = 0.f;
            }
            mx = warp_max_f32(mx);
            int e = 0;
            if (mx > 0.f && mx < INFINITY) e = ilogbf(mx) + 1;                // |q| < 2^e
            // 2^(15 - e), which may leave fp32's range, as two factors
            const int half = (15 - e) / 2;
            const float up0 = __int_as_float((127 + half) << 23), up1 = __int_as_float((127 + 15 - e - half) << 23);
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < kE; ++i) {
                const int d = lane * kE + i, grp = d / 32, tt = d % 32 / 8, p = d % 8;
                // the odd nibbles come in as 16 codes, unless codes are centred
                uint32_t hi, lo;
                const float qs = x[i] * up0 * up1, down = !kSplit && (p & 1) ? 0.0625f : 1.f;
                attend_split(qs * down, 0.f, hi, lo);
                part += kSplit ? f16_lo(hi) + f16_lo(lo) : f16_lo(hi) * (p & 1 ? 16.f : 1.f);
                uint16_t* dst = reinterpret_cast<uint16_t*>(&sm.q[2 * grp + (p >> 1 & 1)][row / 8][0][row % 8 * 4 + tt]) + 2 * (p & 1) + (p >> 2);
                dst[0] = (uint16_t)hi;
                if (kSplit) dst[32 * 4] = (uint16_t)lo;
            }
#pragma unroll
            for (int o = 1; o < 32 / kGroups; o <<= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
            if (kSplit) {
                if (lane % (32 / kGroups) == 0) qsums[lane / (32 / kGroups) * kRows + row] = part * (1.f / kTwo9);       // (as the centred codes are)
            } else if (lane % (32 / kGroups) == 0) {
                // k = 4 term + group sits in lane 4 (row % 8) + k % 8 / 2, register k / 8, half k % 2; groups that are none and the
                // fourth term are 0
                const int grp = lane / (32 / kGroups);
                float rest = part * kTwoM24;       // (as the products with codes * 2^-24 are)
#pragma unroll
                for (int term = 0; term < 4; ++term) {
                    const uint16_t h = term < 3 ? f32_to_bf16_bits(rest) : (uint16_t)0;
                    rest -= bf16_bits_to_f32(h);
#pragma unroll
                    for (int k = 4 * term + grp; k < 4 * term + 4; k += kGroups) {
                        uint16_t* dst = reinterpret_cast<uint16_t*>(&sm.qsum[row / 8][row % 8 * 4 + k % 8 / 2]) + 2 * (k / 8) + k % 2;
                        *dst = k % 4 < kGroups ? h : (uint16_t)0;
                    }
                }
            }
            if (lane == 0) {
                sm.qc[row] = ldexpf(a.scale, e - 15 + (kSplit ? 9 : 24));
                sm.horizon[row] = row < n_rows ? base + rho / G : -1;
            }
        }
        __syncthreads();
        float o[kTiles][NT][4], zl[NT][4], ref[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int m = 0; m < kTiles; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[m][nt][i] = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) zl[nt][i] = 0.f;
            ref[nt][0] = ref[nt][1] = 0.f;
        }
#pragma unroll 1
        for (int it = 0; it < n_it; ++it) {
            const int st = it % kAttendStages, u = u0 + warp + kAttendWarps * it;
            const unsigned char* up = sm.ring[warp][st];
            const bool there = mapped >> st & 1u;
            failed = failed || !mbar_wait(smem_u32(&sm.bars[warp][st]), parity >> st & 1u);
            parity ^= 1u << st;
            if (!there) {
                if (it + kAttendStages < n_it) request(it + kAttendStages);
                continue;
            }
            const bool edge = u * kKv4Unit + kKv4Unit - 1 > seen_all;
            uint32_t kw[2][kGroups], ksz[2][kGroups];      // keys g and g + 8: 8 columns of each group; (s, z) of each group
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const unsigned char* kp = up + (g + 8 * i) * (HD / 2) + t * (4 * kGroups);
                const unsigned char* sp = up + kv4_k_scales(HD) + (g + 8 * i) * (4 * kGroups);
                if (HD == 128) {
                    *reinterpret_cast<uint4*>(kw[i]) = *reinterpret_cast<const uint4*>(kp);
                    *reinterpret_cast<uint4*>(ksz[i]) = *reinterpret_cast<const uint4*>(sp);
                } else {
                    *reinterpret_cast<uint2*>(kw[i]) = *reinterpret_cast<const uint2*>(kp);
                    *reinterpret_cast<uint2*>(ksz[i]) = *reinterpret_cast<const uint2*>(sp);
                }
            }
            // V's scales and middles: lane l takes positions 2 (l % 8), + 1 of group l / 8
            float vs[2], vm[2];
            {
                const int l = lane % (8 * kGroups);
                uint32_t sw = *reinterpret_cast<const uint32_t*>(up + kv4_v_scales(HD) + l * 4), zw = *reinterpret_cast<const uint32_t*>(up + kv4_v_scales(HD) + HD + l * 4);
                if (edge) {                        // what lies behind the last position is not part of the cache: any bits
                    const int p0 = u * kKv4Unit + 2 * (l & 7);
                    const uint32_t keep = (p0 <= seen_any ? 0xffffu : 0u) | (p0 + 1 <= seen_any ? 0xffff0000u : 0u);
                    sw &= keep;
                    zw &= keep;
                }
                vs[0] = bf16_lo(sw); vs[1] = bf16_hi(sw);
                vm[0] = fmaf(8.f, vs[0], bf16_lo(zw)); vm[1] = fmaf(8.f, vs[1], bf16_hi(zw));
            }
            const float vmax = fmaxf(fmaxf(fabsf(vs[0]), fabsf(vs[1])), fmaxf(fabsf(vm[0]), fabsf(vm[1])));
            // ---- scores relative to the rows' references: [2 keys][2 rows] of each tile of 8 rows
            uint4 zf;                              // zeros of both keys: groups 2 (t % 2), + 1
            if (!kSplit) {
                const bool odd = kGroups == 4 && (t & 1);
                zf.x = __byte_perm(odd ? ksz[0][kGroups - 2] : ksz[0][0], odd ? ksz[0][kGroups - 1] : ksz[0][1], 0x7632);
                zf.y = __byte_perm(odd ? ksz[1][kGroups - 2] : ksz[1][0], odd ? ksz[1][kGroups - 1] : ksz[1][1], 0x7632);
                if (kGroups == 2 && (t & 1)) zf.x = zf.y = 0u;
                zf.z = t < 2 ? zf.x : 0u;          // (k from 12 on: nothing)
                zf.w = t < 2 ? zf.y : 0u;
            }
            float s[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (kSplit) {
                    s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
                } else {
                    const uint2 b = sm.qsum[nt][lane];
                    attend_mma_first<true>(s[nt], zf, b.x, b.y);
                }
#pragma unroll
                for (int grp = 0; grp < kGroups; ++grp) {
                    float acc[4];
                    uint4 af[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t w0 = kw[0][grp] >> (8 * h), w1 = kw[1][grp] >> (8 * h);
                        af[h] = make_uint4(w0 & 0x000f000fu, w1 & 0x000f000fu, w0 & 0x00f000f0u, w1 & 0x00f000f0u);
                        if (kSplit) af[h] = make_uint4(attend_centre<false>(af[h].x), attend_centre<false>(af[h].y), attend_centre<true>(af[h].z), attend_centre<true>(af[h].w));
                    }
#pragma unroll
                    for (int i = 0; i < 2 * kTerms; ++i) {     // the small terms first: the sum is truncated at every step
                        const uint2 b = sm.q[2 * grp + i % 2][nt][kTerms - 1 - i / 2][lane];
                        if (i == 0) attend_mma_first<false>(acc, af[0], b.x, b.y);
                        else attend_mma(acc, af[i % 2], b.x, b.y);
                    }
                    const float s0 = bf16_lo(ksz[0][grp]), s1 = bf16_lo(ksz[1][grp]);
                    if (kSplit) {                  // the middles, z + 8 s
                        const float2 b = *reinterpret_cast<const float2*>(&qsums[grp * kRows + nt * 8 + 2 * t]);
                        const float m0 = fmaf(8.f, s0, bf16_hi(ksz[0][grp])), m1 = fmaf(8.f, s1, bf16_hi(ksz[1][grp]));
                        s[nt][0] = fmaf(m0, b.x, s[nt][0]); s[nt][1] = fmaf(m0, b.y, s[nt][1]);
                        s[nt][2] = fmaf(m1, b.x, s[nt][2]); s[nt][3] = fmaf(m1, b.y, s[nt][3]);
                    }
                    s[nt][0] = fmaf(s0, acc[0], s[nt][0]); s[nt][1] = fmaf(s0, acc[1], s[nt][1]);
                    s[nt][2] = fmaf(s1, acc[2], s[nt][2]); s[nt][3] = fmaf(s1, acc[3], s[nt][3]);
                }
                const float2 qc = *reinterpret_cast<const float2*>(&sm.qc[nt * 8 + 2 * t]);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[nt][i] = fmaf(s[nt][i], i & 1 ? qc.y : qc.x, -ref[nt][i & 1]);
                if (edge) {
                    const int2 hz = *reinterpret_cast<const int2*>(&sm.horizon[nt * 8 + 2 * t]);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (u * kKv4Unit + g + 8 * (i >> 1) > (i & 1 ? hz.y : hz.x)) s[nt][i] = -INFINITY;
                }
            }
            // ---- references
            bool over = vmax > unit_scale * kAttendScaleExcess || unit_scale == 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) over |= s[nt][i] > kAttendExcess;
            if (__any_sync(0xffffffffu, over)) {
                const float fit = attend_unit_scale(warp_max_f32(vmax));
                const float to = fmaxf(fit, unit_scale), shrink = unit_scale / to;
                const bool first_unit = unit_scale == 0.f;
                unit_scale = to;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float m = fmaxf(s[nt][c], s[nt][2 + c]);
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
                        // how far the reference moves: up, or (of the first unit) to the unit's maximum
                        m = first_unit && m > -INFINITY ? m : fmaxf(m, 0.f);
                        const float factor = first_unit ? 1.f : attend_exp2(-m);
                        ref[nt][c] += m;
                        s[nt][c] -= m;
                        s[nt][2 + c] -= m;
                        zl[nt][c] *= g == 4 ? factor : factor * shrink;      // (row 4: the denominators; rows from 8 on are not used)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int mt = 0; mt < kTiles; ++mt) o[mt][nt][2 * i + c] *= factor * shrink;
                    }
            }
            // ---- V's scales and middles relative to that, fp16
            uint32_t s16, m16, m16_lo = 0u, s16w[kGroups][2];
            {
                const float inv = __uint_as_float((254u << 23) - __float_as_uint(unit_scale));       // 1 / unit_scale
                const float inv_s = inv * kAttendUpScale, inv_m = inv * kAttendUpMiddle;
                s16 = attend_pack(vs[0] * inv_s, vs[1] * inv_s);                                      // (8 bits: exact)
                if (kSplit) attend_split(vm[0] * inv_m, vm[1] * inv_m, m16, m16_lo);
                else m16 = attend_pack(vm[0] * inv_m, vm[1] * inv_m);
            }
#pragma unroll
            for (int grp = 0; grp < kGroups; ++grp)
#pragma unroll
                for (int i = 0; i < 2; ++i) s16w[grp][i] = __shfl_sync(0xffffffffu, s16, grp * 8 + t + 4 * i);
            // ---- probabilities, as the B operand: rounded, then transposed
            float p[NT][4];
            uint32_t ph[NT][2], pl[kSplit ? NT : 1][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int i = 0; i < 4; ++i) p[nt][i] = kSplit ? attend_exp2(s[nt][i]) * kAttendUpPFactor : attend_exp2(s[nt][i] + kAttendUpP);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t hi = attend_pack(p[nt][2 * i], p[nt][2 * i + 1]);
                    if (kSplit) pl[nt][i] = attend_transpose(attend_pack(p[nt][2 * i] - f16_lo(hi), p[nt][2 * i + 1] - f16_hi(hi)));
                    ph[nt][i] = attend_transpose(hi);
                }
            }
            // ---- the middles' share and the denominators
            uint4 az = make_uint4(0u, 0u, 0u, 0u), azl = az;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t v = __shfl_sync(0xffffffffu, m16, g % kGroups * 8 + t + 4 * i);
                const uint32_t w = g < kGroups ? v : g == 4 ? 0x3c003c00u : 0u;
                if (i == 0) az.x = w;
                else az.z = w;
                if (kSplit) {
                    const uint32_t x = __shfl_sync(0xffffffffu, m16_lo, g % kGroups * 8 + t + 4 * i);
                    if (i == 0) azl.x = g < kGroups ? x : 0u;
                    else azl.z = g < kGroups ? x : 0u;
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (kSplit) {
                    float x[4];
                    attend_mma_first<false>(x, az, pl[nt][0], pl[nt][1]);
                    attend_mma(x, azl, ph[nt][0], ph[nt][1]);
                    attend_mma(x, az, ph[nt][0], ph[nt][1]);
                    zl[nt][0] += x[0];
                    zl[nt][1] += x[1];
                } else {
                    attend_mma(zl[nt], az, ph[nt][0], ph[nt][1]);
                }
            }
            uint32_t vw[kTiles];                   // a word per tile
#pragma unroll
            for (int c = 0; c < HD / 64; ++c) *reinterpret_cast<uint4*>(vw + 4 * c) = *reinterpret_cast<const uint4*>(up + kv4_v_codes(HD) + (c * 32 + lane) * 16);
            __syncwarp();                          // the unit has been read: its place in the ring is free
            if (it + kAttendStages < n_it) request(it + kAttendStages);
#pragma unroll
            for (int grp = 0; grp < kGroups; ++grp) {
                uint32_t b[NT][kTerms][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (kSplit) {              // (hi + lo) * s: what the product rounds off goes to the second term
                            uint32_t hi, lo;
                            hi = attend_mul2(ph[nt][i], s16w[grp][i]);
                            lo = attend_fma2(ph[nt][i], s16w[grp][i], hi ^ 0x80008000u);
                            b[nt][0][i] = hi;
                            b[nt][kTerms - 1][i] = attend_fma2(pl[nt][i], s16w[grp][i], lo);
                        } else {
                            b[nt][0][i] = attend_mul2(ph[nt][i], s16w[grp][i]);
                        }
                    }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t w0 = vw[2 * grp + h], w1 = w0 >> 8;
                    const uint4 af = make_uint4(attend_centre<false>(w0 & 0x000f000fu), attend_centre<true>(w0 & 0x00f000f0u),
                                                attend_centre<false>(w1 & 0x000f000fu), attend_centre<true>(w1 & 0x00f000f0u));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if (kSplit) {
                            float x[4];
                            attend_mma_first<false>(x, af, b[nt][kTerms - 1][0], b[nt][kTerms - 1][1]);
                            attend_mma(x, af, b[nt][0][0], b[nt][0][1]);
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[2 * grp + h][nt][i] += x[i];
                        } else {
                            attend_mma(o[2 * grp + h][nt], af, b[nt][0][0], b[nt][0][1]);
                        }
                    }
                }
            }
        }
        if (failed) {                              // a copy that never came: no result
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) zl[nt][0] = zl[nt][1] = NAN;
        }
        __syncthreads();                           // the rings are empty
        // ---- the warps' shares: outputs with the middles' part, references, denominators
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (g == 4) {
                *reinterpret_cast<float2*>(&sm.ref[warp][nt * 8 + 2 * t]) =
                    make_float2(zl[nt][0] == 0.f ? kAttendNone : ref[nt][0], zl[nt][1] == 0.f ? kAttendNone : ref[nt][1]);
                *reinterpret_cast<float2*>(&sm.sum[warp][nt * 8 + 2 * t]) = make_float2(zl[nt][0], zl[nt][1]);
            }
#pragma unroll
            for (int grp = 0; grp < kGroups; ++grp) {
                const float z[2] = {__shfl_sync(0xffffffffu, zl[nt][0], grp * 4 + t), __shfl_sync(0xffffffffu, zl[nt][1], grp * 4 + t)};
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sm.o[warp][nt * 8 + 2 * t + (i & 1)][(2 * grp + h) * 16 + g + 8 * (i >> 1)] =
                            fmaf(o[2 * grp + h][nt][i], kTwo9 * kAttendUpMiddle / kAttendUpScale, z[i & 1]) * (unit_scale / kAttendUpMiddle);
            }
        }
        __syncthreads();
        const bool whole = u0 == 0 && u1 == units;
        float* part = a.parts + (size_t)(2 * blockIdx.x + (f - u0 > f_cta ? 1 : 0)) * (kRows * (HD + 2));
        for (int i = tid; i < n_rows * (HD / 4); i += kAttendThreads) {
            const int row = i / (HD / 4), c = i % (HD / 4) * 4;
            float top = kAttendNone;
#pragma unroll
            for (int w = 0; w < kAttendWarps; ++w) top = fmaxf(top, sm.ref[w][row]);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < kAttendWarps; ++w) {
                const float factor = attend_exp2(sm.ref[w][row] - top);
                const float4 x = *reinterpret_cast<const float4*>(&sm.o[w][row][c]);
                v.x = fmaf(factor, x.x, v.x); v.y = fmaf(factor, x.y, v.y); v.z = fmaf(factor, x.z, v.z); v.w = fmaf(factor, x.w, v.w);
                sum = fmaf(factor, sm.sum[w][row], sum);
            }
            if (whole) {
                const int rho = rho0 + row;
                const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
                T* dst = static_cast<T*>(a.out) + (size_t)(first + rho / G) * a.out_stride + (size_t)(head * G + rho % G) * HD + c;
                attend_out(dst, v.x * inv); attend_out(dst + 1, v.y * inv); attend_out(dst + 2, v.z * inv); attend_out(dst + 3, v.w * inv);
            } else {
                *reinterpret_cast<float4*>(part + row * HD + c) = v;
                if (c == 0) { part[kRows * HD + row] = top; part[kRows * (HD + 1) + row] = sum; }
            }
        }
        fence_proxy_async_smem();                  // (the next copies go where these values were)
        __syncthreads();
        f += u1 - u0;
        off += u1 - u0;
    }
}

// Adds up the shares of triples that several CTAs had, per (row, query head).  W warps each: a CTA per job, of which warp w takes the shares w,
// w + 4, ..., and the warps' sums are added in their order (a warp for a row alone waits for the L2 once per four shares: 12 us for 37 of them).
// W = 1: beyond a wave of such CTAs a warp per a.heads heads of a row, since what finds a job's shares costs more than the few that each then
// has (us with four and one, CTAs of one row tile, heads of 128: 32 rows of 32 heads in bf16, one wave, 52.5 52.6; 64 rows 63.7 60; 155 rows
// in fp32 206 198; a prompt of 2000 rows in bf16 705 606).
constexpr int kMergeWarps = 4;
constexpr int kMergeWave = 148 * 9;                // CTAs of it that the device holds (56 registers)
template <int HD, int W, typename T>
__global__ void __launch_bounds__(32 * kMergeWarps) kv4_merge_kernel(const Kv4AttendArgs a) {
    constexpr int kE = HD / 32;
    __shared__ float s_v[W][HD], s_sum[W];
    const int lane = threadIdx.x & 31, warp = W == 1 ? 0 : threadIdx.x >> 5;
    const long long job = W == 1 ? (long long)blockIdx.x * kMergeWarps + (threadIdx.x >> 5) : (long long)blockIdx.x;
    const int blocks = (a.Hq + a.heads - 1) / a.heads, G = a.Hq / a.w.Hkv;       // (of heads)
    const int row = (int)(job / blocks), q0 = (int)(job % blocks) * a.heads, q1 = min(a.Hq, q0 + a.heads);
    int req = -1;
    for (int r0 = 0; row < a.w.rows && r0 < a.w.n_req && req < 0; r0 += 32) {    // (the last CTA's warps may have no row)
        const int r = min(r0 + lane, a.w.n_req - 1);
        const unsigned hit = __ballot_sync(0xffffffffu, a.w.row0[r] <= row && row < a.w.row0[r + 1]);
        if (hit) req = min(r0 + __ffs(hit) - 1, a.w.n_req - 1);
    }
    int n, first, base, units, groups;
    attend_load(a, req < 0 ? a.w.n_req : req, n, first, base, units, groups);
    long long before;
    const long long all = attend_total(a, req, before), share = attend_share(a, all);
    // Launched with programmatic serialisation: behind this the shares are complete.  Every thread waits, those without work too: a grid that
    // ended without could let its successor begin before its predecessor has ended.
    pdl_wait();
    if (req < 0) return;
    const size_t slot_size = (size_t)a.rows_cap * (HD + 2);
    for (int qh = q0; qh < q1; ++qh) {
        T* out = static_cast<T*>(a.out) + (size_t)row * a.out_stride + (size_t)qh * HD + lane * kE;
        if (row - first >= n) {                    // a row without a position: nothing to see
            if (warp == 0)
#pragma unroll
                for (int i = 0; i < kE; ++i) attend_out(out + i, 0.f);
            continue;
        }
        const int rho = (row - first) * G + qh % G;
        const long long start = before + (long long)(qh / G * groups + rho / a.rows_cap) * units;
        const int c0 = (int)(start / share), c1 = (int)((start + units - 1) / share);
        if (c0 == c1) continue;
        const int local = rho % a.rows_cap;
        auto slot = [&](int c) { return a.parts + (size_t)(2 * c + (start > (long long)c * share ? 1 : 0)) * slot_size; };
        float top = kAttendNone;
        for (int c = c0 + lane; c <= c1; c += 32) top = fmaxf(top, slot(c)[a.rows_cap * HD + local]);
        top = warp_max_f32(top);
        float v[kE] = {}, sum = 0.f;
#pragma unroll 4
        for (int c = c0 + warp; c <= c1; c += W) {
            const float* p = slot(c);
            const float factor = attend_exp2(p[a.rows_cap * HD + local] - top);
#pragma unroll
            for (int i = 0; i < kE; ++i) v[i] = fmaf(factor, p[local * HD + lane * kE + i], v[i]);
            sum = fmaf(factor, p[a.rows_cap * (HD + 1) + local], sum);
        }
        if (W > 1) {                               // (one head: a.heads is 1)
#pragma unroll
            for (int i = 0; i < kE; ++i) s_v[warp][lane * kE + i] = v[i];
            if (lane == 0) s_sum[warp] = sum;
            __syncthreads();
            if (warp) return;
#pragma unroll
            for (int w = 1; w < W; ++w) {
                sum += s_sum[w];
#pragma unroll
                for (int i = 0; i < kE; ++i) v[i] += s_v[w][lane * kE + i];
            }
        }
        const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
#pragma unroll
        for (int i = 0; i < kE; ++i) attend_out(out + i, v[i] * inv);
    }
}

}  // namespace pipesd
