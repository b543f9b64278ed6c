// Shaped next-token distributions: temperature, top-k, top-p and min-p on rows of logits, and the two things that are done with
// them, drawing a token (sample) and the acceptance rule of speculative sampling (accept).
//
// A row's ids are ordered by logit, highest first, equal ones by id, lowest first.  With w_j = exp((l_j - max) / T) (T = 0: 1 for
// the first of the order, 0 for the others) the settings keep
//   top-k   the first k ids of the order (k <= 0: all),
//   top-p   of these the shortest prefix that holds at least p of their mass: an id stays while the mass before it is < p * Z,
//   min-p   of these the ids with w_j >= min_p,
// and P_j = w_j / (sum of the kept w).  All three cut the order somewhere, so that a row's outcome is one bound: the last kept logit
// and id.
//
// Masses are 64-bit whole numbers, w * 2^45 rounded to nearest: sums do not depend on their order, a prefix never decreases, and no
// result changes between runs, cluster sizes or passes.  At most 2^18 ids, so a sum is at most 2^63; what rounding moves is
// 2^-46 of the most likely id's weight per id, and an id below that has no mass at all.  Weights are evaluated in fp64: thresholds and
// draws are whole decisions, and one in a few thousand of a flat row would fall on the other side of a border with fp32 weights.
//
// What bounds it.  One row: the chain of passes and barriers (32000 ids: greedy 4.5 us, unshaped 10, top-k 12, top-p 20).  Many rows: fp64 and
// 32-bit instructions of the weights, 43 a logit, and the second read of a row that L2 no longer holds.  256 rows of 128256 fp32, 131 MB:
// greedy 28 us (4.7 TB/s), min-p 55, top-k 50 70, unshaped 84, top-p 0.9 134 (0.98 TB/s; five passes and an exponential of CUDA's in every
// one 386).
#pragma once
#include "../common.cuh"

namespace pipesd {

constexpr int kShapeThreads = 512;
constexpr int kShapeWarps = kShapeThreads / 32;
constexpr int kShapeBins = 4096, kShapeFine = 1024, kShapeDigit = 2048, kShapeSegs = 64;
constexpr int kSegBins = kShapeBins / kShapeSegs, kSegFine = 32;      // bins of a segment
constexpr int kShapeMaxVocab = 1 << 18;
constexpr float kShapeMaxT = 1e30f;                // beyond, even the lowest logit would have to be weighed against -inf
constexpr double kMassOne = 35184372088832.0;      // 2^45

struct Shaping { float t; int k; float p, mp; };   // pipesd_shaping

// What the rest of a call needs to know about a row: P_id = exp2((l - m) * c) / (total * 2^-45) where the id's key is >= bound, that is
// where l > cut or l = cut and id <= cut_id.  total = 0: the row has no distribution (no finite logit, a NaN or +inf among them,
// settings out of range).
struct RowShape {
    double m, c;
    unsigned long long total;
    float cut;
    int cut_id;
};

__device__ __forceinline__ float logit_f32(float v) { return v; }
__device__ __forceinline__ float logit_f32(uint16_t v) { return bf16_bits_to_f32(v); }
template <typename T> __device__ __forceinline__ T logit_none();
template <> __device__ __forceinline__ float logit_none<float>() { return -INFINITY; }
template <> __device__ __forceinline__ uint16_t logit_none<uint16_t>() { return 0xff80; }

// Position in the order as a number: larger = earlier.  The addition makes -0 a +0, so that the two tie.
__device__ __forceinline__ unsigned long long order_key(float l, int id) {
    const uint32_t b = __float_as_uint(l + 0.f);
    const uint32_t s = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return (unsigned long long)s << 32 | (uint32_t)~id;
}

__device__ __forceinline__ float key_logit(unsigned long long key) {
    const uint32_t b = (uint32_t)(key >> 32);
    return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}

// Exponent of the weight of a logit that r keeps (which has one of at least -1000).
__device__ __forceinline__ double shape_exponent(float l, const RowShape& r) { return ((double)l - r.m) * r.c; }
// The lowest logit with an exponent of about -990 or more.  What lies below has no mass, whatever the settings keep of it: the bound
// of a row is never lower.
__device__ __forceinline__ float shape_low(double m, double c) {
    const float l = (float)fmax(m - 990.0 / c, -3.4028234e38);
    return ((double)l - m) * c < -1000.0 ? nextafterf(l, INFINITY) : l;
}
// 2^y for -1000 <= y <= 0: whole part into the exponent, the rest by a polynomial of degree 9 (interpolation at the Chebyshev
// nodes of [-1/2, 1/2], coefficients computed in 70 digits: relative error 1.8e-14, less than a step of the masses).  Coefficients
// are read as constant operands: as literals each costs two moves.
__constant__ double kExp2Poly[10] = {1.0000000000000135, 0.6931471805599462, 0.2402265069564034, 0.05550410866465167, 0.009618129193934313,
                                     0.0013333558200794592, 0.0001540343375125101, 1.5252672924850737e-05, 1.325964524488711e-06, 1.0205905413765595e-07};
__device__ __forceinline__ double shape_exp2(double y) {
    const double big = 6755399441055744.0;         // 1.5 * 2^52: the sum's low bits are the rounded y
    const double n = y + big, r = y - (n - big);
    double p = kExp2Poly[9];
#pragma unroll
    for (int i = 8; i >= 0; --i) p = fma(p, r, kExp2Poly[i]);
    return __hiloint2double(__double2hiint(p) + (__double2loint(n) << 20), __double2loint(p));
}
// A weight as a whole number of 2^-45: 128 + w has exactly those last bits.  (Sums may add the bits as they are and take the 128s away
// in the end: whole numbers modulo 2^64.)
constexpr unsigned long long kMassBase = 0x4060000000000000ull;          // 128.0
__device__ __forceinline__ unsigned long long shape_mass_bits(double y) { return (unsigned long long)__double_as_longlong(shape_exp2(y) + 128.0); }
__device__ __forceinline__ unsigned long long shape_mass(double y) { return shape_mass_bits(y) - kMassBase; }
__device__ __forceinline__ bool shape_keeps(float l, int id, const RowShape& r) { return l > r.cut || (l == r.cut && id <= r.cut_id); }

__device__ __forceinline__ unsigned long long warp_sum_u64(unsigned long long v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ unsigned long long warp_max_u64(unsigned long long v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long t = __shfl_xor_sync(0xffffffffu, v, o);
        v = t > v ? t : v;
    }
    return v;
}
// Inclusive prefix over the lanes.
__device__ __forceinline__ unsigned long long warp_scan_u64(unsigned long long v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}

template <int C>
__device__ __forceinline__ void shape_sync() {
    if (C > 1) cluster_sync_all();
    else __syncthreads();
}
template <int C>
__device__ __forceinline__ int shape_rank() { return C > 1 ? (int)cluster_ctarank() : 0; }
template <int C>
__device__ __forceinline__ unsigned long long shape_peer(const unsigned long long* p, int rank) {
    if (C == 1) return *p;
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(dsmem_addr(smem_u32(p), (uint32_t)rank)) : "memory");
    return v;
}
template <int C>
__device__ __forceinline__ int shape_peer_i32(const int* p, int rank) {
    if (C == 1) return *p;
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(dsmem_addr(smem_u32(p), (uint32_t)rank)) : "memory");
    return v;
}

constexpr int kShapeList = 1024;                   // ids that are dealt with one by one
struct ShapeSmem {
    union {                                        // bins of a row, or of a digit
        uint32_t coarse[kShapeBins];
        unsigned long long digit[kShapeDigit];
    };
    union {
        unsigned long long fine[kShapeFine];       // bins of a window
        unsigned long long mass[kShapeList];       // masses of `keys`
    };
    unsigned long long own[kShapeList];            // keys that this CTA collected
    unsigned long long keys[kShapeList];           // the cluster's
    unsigned long long part[kShapeWarps], part2[kShapeWarps];
    unsigned long long seg[kShapeSegs];            // sums of neighbouring bins: counts, or masses as doubles
    unsigned long long fine_seg[kShapeFine / kSegFine];
    unsigned long long cta[4];                     // what the other CTAs of the cluster read: key maximum, kept mass, masses of a window
    unsigned long long found[3];
    int n_own, n_keys, window[2];
};

// Walks this warp's ids of the row, VEC neighbours per lane and group: f(logits, first id) for groups of ids first + [0, VEC), several
// groups' loads in flight together.  All lanes call f together; what lies at or behind j1 comes as -inf.
template <typename T, int VEC, typename F>
__device__ __forceinline__ void shape_groups(const T* row, int j0, int j1, F&& f) {
    constexpr int kBatch = VEC == 1 ? 8 : 4;
    const int lane = threadIdx.x & 31;
    for (int j = j0; j < j1; j += 32 * VEC * kBatch) {
        T v[kBatch][VEC];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int i = j + (b * 32 + lane) * VEC;
            if (VEC > 1 && i + VEC <= j1) {
                *reinterpret_cast<uint4*>(v[b]) = *reinterpret_cast<const uint4*>(row + i);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[b][e] = i + e < j1 ? row[i + e] : logit_none<T>();
            }
        }
        if (VEC == 1) {                            // eight groups of one: as one group of eight, of ids 32 apart
            float l[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) l[b] = logit_f32(v[b][0]);
            f(l, j + lane);
        } else {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                if (j + b * 32 * VEC >= j1) break;
                float l[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) l[e] = logit_f32(v[b][e]);
                f(l, j + (b * 32 + lane) * VEC);
            }
        }
    }
}
// The ids of a group are first + kApart * e.
template <int VEC>
__device__ __forceinline__ constexpr int group_apart() { return VEC == 1 ? 32 : 1; }

// The same id by id (lanes may diverge in f).
template <typename T, int VEC, typename F>
__device__ __forceinline__ void shape_walk(const T* row, int j0, int j1, F&& f) {
    shape_groups<T, VEC>(row, j0, j1, [&](const auto& l, int first) {
        constexpr int kN = sizeof(l) / 4;
        const int lane = threadIdx.x & 31;
        if (first - lane * (VEC == 1 ? 1 : VEC) + 32 * kN <= j1) {           // the whole warp's group is inside
#pragma unroll
            for (int e = 0; e < kN; ++e) f(l[e], first + e * group_apart<VEC>());
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const int id = first + e * group_apart<VEC>();
                if (id < j1) f(l[e], id);
            }
        }
    });
}

// Whether r keeps an id; kTies: of the ids with just the cut's logit some may be cut (else cut_id is behind all ids).
template <bool kTies>
__device__ __forceinline__ bool shape_kept(float l, int id, const RowShape& r) { return kTies ? shape_keeps(l, id, r) : l >= r.cut; }

// Masses of the ids that r keeps, as shape_mass_bits: f(bits, kept, logit, id); what is not kept is weighed as the maximum.  All of a
// group's exponentials side by side, without a branch between them (one by one they are chains of fifteen dependent fp64 operations);
// groups of which the warp keeps nothing are skipped.
template <bool kTies, typename T, int VEC, typename F>
__device__ __forceinline__ void shape_masses(const T* row, int j0, int j1, const RowShape& r, F&& f) {
    const float m = (float)r.m;
    shape_groups<T, VEC>(row, j0, j1, [&](const auto& l, int first) {
        constexpr int kN = sizeof(l) / 4;
        bool keep[kN], any = false;
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            keep[e] = shape_kept<kTies>(l[e], first + e * group_apart<VEC>(), r);
            any |= keep[e];
        }
        if (!__any_sync(0xffffffffu, any)) return;
        unsigned long long w[kN];
#pragma unroll
        for (int e = 0; e < kN; ++e) w[e] = shape_mass_bits(shape_exponent(keep[e] ? l[e] : m, r));
#pragma unroll
        for (int e = 0; e < kN; ++e) f(w[e], keep[e], l[e], first + e * group_apart<VEC>());
    });
}
// A sum of them: the 128s, and the 2^45 of the others, are taken away in the end.
struct MassSum {
    unsigned long long bits = 0;
    unsigned n = 0, others = 0;
    __device__ __forceinline__ unsigned long long total() const { return bits - n * kMassBase - ((unsigned long long)others << 45); }
};
// This lane's sum.
template <bool kTies, typename T, int VEC>
__device__ __forceinline__ unsigned long long shape_mass_sum_of(const T* row, int j0, int j1, const RowShape& r) {
    MassSum sum;
    shape_masses<kTies, T, VEC>(row, j0, j1, r, [&](unsigned long long w, bool keep, float, int) {
        sum.bits += w;
        ++sum.n;
        sum.others += !keep;
    });
    return sum.total();
}
template <typename T, int VEC>
__device__ __forceinline__ unsigned long long shape_mass_sum(const T* row, int j0, int j1, const RowShape& r, int V) {
    return r.cut_id < V ? shape_mass_sum_of<true, T, VEC>(row, j0, j1, r) : shape_mass_sum_of<false, T, VEC>(row, j0, j1, r);
}

// Sum (kMax: maximum) over the CTA; every thread gets it.  `part` is not used again before the next barrier but one.
template <bool kMax>
__device__ __forceinline__ unsigned long long cta_reduce_u64(unsigned long long v, unsigned long long* part) {
    v = kMax ? warp_max_u64(v) : warp_sum_u64(v);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < kShapeWarps; ++w) v = kMax ? (part[w] > v ? part[w] : v) : v + part[w];
    return v;
}

// Finding the bound.  A cut of the order is the key at which a running sum over it (of ones: top-k; of masses: top-p) first reaches
// `need`; everything from there upwards is kept.
//
// The usual way has two passes over the row.  The first one, which also finds the maximum, counts bins of equal width in the logit with
// 32-bit atomics, from kShapeUp units above the largest of the row's first ids downwards; for masses a bin adds up
// w / (weight of its middle), which lies within 1 / 128 of 1, as whole numbers of 2^-13: its mass is then known to kShapeSlack.
// That settles a window of bins that holds the cut for certain, mostly one; for top-k the bin itself.  Top-k's second pass collects the
// ids of that bin, with those above it where they are few: these rows are finished from that list.  Top-p's computes the masses
// proper: their sums above and in the window, and in kShapeFine finer bins of it (64-bit atomics, few of them), and keeps the window's
// ids (more than the list holds: a third pass collects those of one fine bin).  Those of the fine bin with the cut are compared with
// each other.  Where even they are more than the lists hold (thousands of equal logits, a cut in the far tail) shape_select_digits
// takes over, which needs no luck: digit by digit over the whole key.
constexpr double kShapeSlack = 1.1e-4;             // half a step of 2^-13 (6.1e-5), the quarter step that shape_count's constant is rounded by
                                                   // (3.1e-5), and what fp32 loses of the places of bin and maximum (8e-6 each)
constexpr float kShapeWidth = 64.f;                // bins per unit of the exponent (top-p) or of the logit (top-k)
constexpr float kShapeUp = 20.f;                   // units: 44 remain below, e^-44 of the maximum over 2^18 ids is nothing

template <int C, bool kMass, typename T, int VEC>
__device__ __noinline__ unsigned long long shape_select_digits(const T* row, int j0, int j1, const RowShape& r, unsigned long long need, double need_share,
                                                               ShapeSmem& sm) {
    const int tid = threadIdx.x;
    unsigned long long prefix = 0;
    int known = 0;                                 // leading bits of the key that are settled
#pragma unroll 1
    for (int level = 0; level < 5; ++level) {      // 32 bits of logit: 11, 11, 10; ids: 11, 11, above them ten ones
        if (level == 3) {
            prefix = prefix << 10 | 1023u;
            known += 10;
        }
        const int bits = level == 2 ? 10 : 11, shift = 64 - known - bits;
        unsigned long long* hist = sm.digit;
        shape_sync<C>();                           // nobody reads what was here before
        for (int b = tid; b < kShapeDigit; b += kShapeThreads) hist[b] = 0;
        __syncthreads();
        shape_walk<T, VEC>(row, j0, j1, [&](float l, int id) {
            const unsigned long long key = order_key(l, id);
            if (!shape_keeps(l, id, r) || (known && key >> (64 - known) != prefix)) return;
            const unsigned long long add = kMass ? shape_mass(shape_exponent(l, r)) : 1ull;
            if (add) atomicAdd(hist + (size_t)((key >> shift) & ((1u << bits) - 1)), add);
        });
        shape_sync<C>();
        // bins from the top: thread t takes four neighbours; all CTAs add up the same numbers
        unsigned long long mine[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = kShapeDigit - 1 - (tid * 4 + i);
            mine[i] = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) mine[i] += shape_peer<C>(hist + b, c);
            sum += mine[i];
        }
        const unsigned long long incl = warp_scan_u64(sum);
        if ((tid & 31) == 31) sm.part[tid >> 5] = incl;
        __syncthreads();
        unsigned long long above = incl - sum, all = 0;
#pragma unroll
        for (int w = 0; w < kShapeWarps; ++w) {
            if (w < tid >> 5) above += sm.part[w];
            all += sm.part[w];
        }
        if (level == 0 && kMass) need = (unsigned long long)ceil(need_share * (double)all);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (above < need && need <= above + mine[i]) {
                sm.found[0] = (unsigned long long)(kShapeDigit - 1 - (tid * 4 + i));
                sm.found[1] = above;
            }
            above += mine[i];
        }
        __syncthreads();
        prefix = prefix << bits | sm.found[0];
        need -= sm.found[1];
        known += bits;
    }
    shape_sync<C>();
    return prefix;
}

// The row's place among bins of equal width from `from` downwards; the first bin takes everything above, the last everything below.  No
// contraction: every pass has to come to the same place.
struct ShapeBins {
    float from, inv;                               // bins per unit of the logit
    __device__ __forceinline__ float at(float l) const { return __fmul_rn(__fsub_rn(from, l), inv); }
    __device__ __forceinline__ float clamped(float l) const { return fminf(fmaxf(at(l), 0.f), (float)(kShapeBins - 1)); }
};
// (The place's whole part by an addition that rounds towards zero, the weight's whole steps by one that rounds to nearest: the converters
// take a quarter of the rate.)
template <bool kMass>
__device__ __forceinline__ void shape_count(const ShapeBins& bins, float l, uint32_t* coarse) {
    const float big = 8388608.f, x = bins.clamped(l), b = __fadd_rz(x, big);
    uint32_t add = 1;
    if (kMass) {                                   // exp(-d) to the second order, d = (f - 1/2) / 64, |d| <= 1 / 128, in steps of 2^-13
        constexpr float d0 = 0.5f / kShapeWidth;
        const float f = x - (b - big);
        add = __float_as_uint(fmaf(f, fmaf(f, 4096.f / (kShapeWidth * kShapeWidth), -(8192.f + 8192.f * d0) / kShapeWidth), big + 8192.f * (1.f + d0 + 0.5f * d0 * d0))) - 0x4b000000u;
    }
    atomicAdd(coarse + (__float_as_uint(b) - 0x4b000000u), add);
}

// Behind the pass and a barrier of the CTA: its bins' sums by segment, so that a cluster exchanges 64 numbers and then the bins of
// one segment (all bins of all CTAs read by all of them take 20 us in a cluster of eight).  Masses are relative to a weight of 1 at the
// first bin's upper end.
constexpr double kBinShrink = 0.98449643700540845;       // exp(-1 / kShapeWidth)
__device__ __forceinline__ double shape_bin_weight(int b) { return shape_exp2(((double)b + 0.5) * (-1.4426950408889634 / kShapeWidth)) * (1.0 / 8192.0); }
template <bool kMass>
__device__ __forceinline__ void shape_segments(ShapeSmem& sm) {
    const int tid = threadIdx.x;
    constexpr int kEach = kShapeBins / kShapeThreads;
    uint32_t n[kEach];
#pragma unroll
    for (int i = 0; i < kEach; i += 4) *reinterpret_cast<uint4*>(n + i) = *reinterpret_cast<const uint4*>(sm.coarse + tid * kEach + i);
    if (kMass) {
        double w = shape_bin_weight(tid * kEach), sum = 0.0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) { sum += (double)n[i] * w; w *= kBinShrink; }
#pragma unroll
        for (int o = 1; o < kSegBins / kEach; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (tid % (kSegBins / kEach) == 0) sm.seg[tid / (kSegBins / kEach)] = (unsigned long long)__double_as_longlong(sum);
    } else {
        unsigned sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) sum += n[i];
#pragma unroll
        for (int o = 1; o < kSegBins / kEach; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (tid % (kSegBins / kEach) == 0) sm.seg[tid / (kSegBins / kEach)] = sum;
    }
}
// Pass over the ids that r keeps for their bins alone: where the first pass began too low, or a second cut follows.
template <bool kMass, typename T, int VEC>
__device__ __noinline__ void shape_coarse(const T* row, int j0, int j1, const ShapeBins bins, const RowShape& r, ShapeSmem& sm) {
    for (int b = threadIdx.x; b < kShapeBins; b += kShapeThreads) sm.coarse[b] = 0;
    __syncthreads();
    shape_walk<T, VEC>(row, j0, j1, [&](float l, int id) {
        if (shape_keeps(l, id, r)) shape_count<kMass>(bins, l, sm.coarse);
    });
    __syncthreads();
    shape_segments<kMass>(sm);
}

template <int C>
__device__ __forceinline__ unsigned shape_bin(const ShapeSmem& sm, int b) {
    unsigned n = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) n += (unsigned)shape_peer_i32<C>(reinterpret_cast<const int*>(sm.coarse + b), c);
    return n;
}
__device__ __forceinline__ double warp_scan_f64(double v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}
// The neighbours 2 lane, 2 lane + 1 among 64 counts in which the running sum first reaches need (whole warp; it does): their place and the sum
// before it.
__device__ __forceinline__ int shape_find2(unsigned long long a, unsigned long long b, unsigned long long need, unsigned long long& before, unsigned long long& in) {
    const int lane = threadIdx.x & 31;
    const unsigned long long incl = before + warp_scan_u64(a + b), start = incl - a - b;
    const unsigned hit = __ballot_sync(0xffffffffu, need <= incl);
    const int l = hit ? __ffs(hit) - 1 : 31;
    const bool second = need > start + a;
    const int at = __shfl_sync(0xffffffffu, 2 * lane + second, l);
    before = __shfl_sync(0xffffffffu, second ? start + a : start, l);
    in = __shfl_sync(0xffffffffu, second ? b : a, l);
    return at;
}

// The CTAs' own lists, put together in all of them as far as `wanted` says so (order arbitrary; ends with a barrier of the CTA).
// Returns the number in sm.keys; more than kShapeList: not all of them are there.
template <int C, typename F>
__device__ __forceinline__ int shape_gather(ShapeSmem& sm, F&& wanted) {
    if (threadIdx.x == 0) sm.n_keys = 0;
    __syncthreads();
    bool over = false;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int theirs = shape_peer_i32<C>(&sm.n_own, c);
        over |= theirs > kShapeList;
        for (int i = threadIdx.x; i < min(theirs, kShapeList); i += kShapeThreads) {
            const unsigned long long key = shape_peer<C>(sm.own + i, c);
            if (!wanted(key)) continue;
            const int at = atomicAdd(&sm.n_keys, 1);
            if (at < kShapeList) sm.keys[at] = key;
        }
    }
    __syncthreads();
    return over ? kShapeList + 1 : sm.n_keys;
}
__device__ __forceinline__ void shape_keep_key(ShapeSmem& sm, float l, int id) {
    const int i = atomicAdd(&sm.n_own, 1);
    if (i < kShapeList) sm.own[i] = order_key(l, id);
}

// Top-k, k < V, behind the first pass and a barrier of the cluster: the bound, or (few enough) the list of at least all kept keys in
// sm.keys, *listed of them.  sm.n_own = 0 at the start.
template <int C, typename T, int VEC>
__device__ unsigned long long shape_top_k(const T* row, int j0, int j1, const RowShape& r, const ShapeBins& bins, int k, ShapeSmem& sm, int* listed) {
    const int tid = threadIdx.x, lane = tid & 31;
    *listed = 0;
    if (tid < 32) {                                // the segment, then its bin
        unsigned long long n[2] = {0, 0}, above = 0, in;
#pragma unroll
        for (int c = 0; c < C; ++c) { n[0] += shape_peer<C>(sm.seg + 2 * lane, c); n[1] += shape_peer<C>(sm.seg + 2 * lane + 1, c); }
        int at = shape_find2(n[0], n[1], (unsigned)k, above, in) * kSegBins;
        at += shape_find2(shape_bin<C>(sm, at + 2 * lane), shape_bin<C>(sm, at + 2 * lane + 1), (unsigned)k, above, in);
        if (lane == 0) {
            sm.found[0] = (unsigned long long)at;
            sm.found[1] = above;
            sm.found[2] = in;
        }
    }
    __syncthreads();
    const int cut = (int)sm.found[0], before = (int)sm.found[1], in = (int)sm.found[2];
    const bool all = before + in <= kShapeList;    // all that may be kept
    if (in > kShapeList) return shape_select_digits<C, false, T, VEC>(row, j0, j1, r, (unsigned long long)k, 0.0, sm);
    shape_walk<T, VEC>(row, j0, j1, [&](float l, int id) {
        const int b = (int)bins.clamped(l);
        if (all ? b <= cut : b == cut) shape_keep_key(sm, l, id);
    });
    shape_sync<C>();
    const int n = shape_gather<C>(sm, [](unsigned long long) { return true; });
    if (all) {
        *listed = n;
        return 0ull;
    }
    unsigned long long last = 0;                   // inverted: the smallest kept key as a maximum
    for (int i = tid; i < n; i += kShapeThreads) {
        int rank = before;
        for (int j = 0; j < n; ++j) rank += sm.keys[j] > sm.keys[i];
        if (rank < k && ~sm.keys[i] > last) last = ~sm.keys[i];
    }
    const unsigned long long bound = ~cta_reduce_u64<true>(last, sm.part2);
    shape_sync<C>();
    return bound;
}

// Top-p, 0 < p < 1, among the ids that r keeps, behind the first pass and a barrier of the cluster: the bound.  *parts: sm.part holds
// the kept masses of this CTA's warps (whose ids are `per` each).  sm.n_own = 0 at the start.
template <int C, typename T, int VEC>
__device__ unsigned long long shape_top_p(const T* row, int j0, int j1, const RowShape& r, const ShapeBins& bins, float share, ShapeSmem& sm, int V, int per, bool* parts) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const double p = (double)share;
    *parts = false;
    for (int i = tid; i < kShapeFine; i += kShapeThreads) sm.fine[i] = 0;
    // The cut is in bin b if prefix(b - 1) < p Z <= prefix(b); what is known of a prefix is off by kShapeSlack of itself, and so is what
    // is known of a suffix (plus what the last bin holds, below 2^18 e^-44 of the maximum), so that a p close to 1 is as sharp as one
    // close to 0.  The same for segments of bins.
    if (warp == 0) {
        constexpr double kUp = 1.0 + 3.0 * kShapeSlack, kDown = 1.0 - 3.0 * kShapeSlack;
        const double tail = 1e-9 * shape_exp2((double)bins.at((float)r.m) * (-1.4426950408889634 / kShapeWidth));
        double n[2] = {0.0, 0.0};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) n[i] += __longlong_as_double((long long)shape_peer<C>(sm.seg + 2 * lane + i, c));
        const double incl = warp_scan_f64(n[0] + n[1]), all = __shfl_sync(0xffffffffu, incl, 31), cut_above = p * all, cut_below = (1.0 - p) * all;
        auto may = [&](double above, double upto) {
            const double below = fmax(all - above, 0.0), after = fmax(all - upto, 0.0);
            return above * kDown - tail < cut_above && upto * kUp + tail >= cut_above && below * kUp + tail > cut_below && after * kDown - tail <= cut_below;
        };
        auto widest = [&](int& lo, int& hi) {
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
        };
        const double s0 = incl - n[0] - n[1], s1 = incl - n[1];
        int lo = kShapeBins, hi = -1;
        if (may(s0, s1)) { lo = 2 * lane; hi = 2 * lane; }
        if (may(s1, incl)) { lo = min(lo, 2 * lane + 1); hi = 2 * lane + 1; }
        widest(lo, hi);
        if (hi >= lo && hi - lo < 4) {             // its bins: 2, 4, ... neighbours a lane
            double run = __shfl_sync(0xffffffffu, lo & 1 ? s1 : s0, lo >> 1);
            const int first = lo * kSegBins, segs = hi - lo + 1;
            int blo = kShapeBins, bhi = -1;
            for (int q = 0; q < segs; ++q) {
                const int b = first + q * kSegBins + 2 * lane;
                const double w = shape_bin_weight(b), a0 = (double)shape_bin<C>(sm, b) * w, a1 = (double)shape_bin<C>(sm, b + 1) * (w * kBinShrink);
                const double up = run + warp_scan_f64(a0 + a1), b0 = up - a0 - a1, b1 = up - a1;
                if (may(b0, b1)) { blo = min(blo, b); bhi = max(bhi, b); }
                if (may(b1, up)) { blo = min(blo, b + 1); bhi = max(bhi, b + 1); }
                run = __shfl_sync(0xffffffffu, up, 31);
            }
            widest(blo, bhi);
            lo = blo;
            hi = bhi;
        } else if (hi >= lo) {
            lo *= kSegBins;
            hi = hi * kSegBins + kSegBins - 1;
        }
        if (lane == 0) { sm.window[0] = lo; sm.window[1] = hi; }
    }
    __syncthreads();
    const int lo = sm.window[0], hi = sm.window[1];
    if (hi < 0) return shape_select_digits<C, true, T, VEC>(row, j0, j1, r, 0ull, p, sm);
    // ---- the masses proper: above the window, all, and by fine bins of the window
    const float from = lo == 0 ? -INFINITY : (float)lo, to = hi == kShapeBins - 1 ? INFINITY : (float)(hi + 1);
    const float steps = (float)kShapeFine / (float)(hi + 1 - lo);
    auto fine_of = [&](float x) { return (int)fminf(fmaxf(__fmul_rn(__fsub_rn(x, (float)lo), steps), 0.f), (float)(kShapeFine - 1)); };
    MassSum s_all, s_above;
    auto weigh = [&](unsigned long long w, bool keep, float l, int id) {
        const float x = bins.at(l);
        s_all.bits += w;
        ++s_all.n;
        s_all.others += !keep;
        if (x < from) {                            // (kept, or it would not be above a kept one)
            s_above.bits += w;
            ++s_above.n;
        } else if (x < to && keep && w > kMassBase) {
            atomicAdd(sm.fine + fine_of(x), w - kMassBase);
            shape_keep_key(sm, l, id);
        }
    };
    if (r.cut_id < V) shape_masses<true, T, VEC>(row, j0, j1, r, weigh);
    else shape_masses<false, T, VEC>(row, j0, j1, r, weigh);
    unsigned long long m_all = s_all.total(), m_above = s_above.total();
    m_all = warp_sum_u64(m_all);
    m_above = warp_sum_u64(m_above);
    if (lane == 0) { sm.part[warp] = m_all; sm.part2[warp] = m_above; }
    __syncthreads();
    {
        unsigned long long t = sm.fine[2 * tid] + sm.fine[2 * tid + 1];
#pragma unroll
        for (int o = 1; o < kSegFine / 2; o <<= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        if (tid % (kSegFine / 2) == 0) sm.fine_seg[tid / (kSegFine / 2)] = t;
    }
    if (warp == 0) {
        m_all = warp_sum_u64(lane < kShapeWarps ? sm.part[lane] : 0ull);
        m_above = warp_sum_u64(lane < kShapeWarps ? sm.part2[lane] : 0ull);
        if (lane == 0) { sm.cta[2] = m_all; sm.cta[3] = m_above; }
    }
    shape_sync<C>();
    m_all = 0;
    unsigned long long run = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) { m_all += shape_peer<C>(&sm.cta[2], c); run += shape_peer<C>(&sm.cta[3], c); }
    const unsigned long long need = (unsigned long long)ceil(p * (double)m_all);
    if (warp == 0) {                               // the segment of fine bins, then the bin
        auto sum_of = [&](const unsigned long long* at) {
            unsigned long long t = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) t += shape_peer<C>(at, c);
            return t;
        };
        int at = 0;
        bool in = run < need;
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            const unsigned long long mine = sum_of(step == 0 ? sm.fine_seg + lane : sm.fine + at * kSegFine + lane), incl = run + warp_scan_u64(mine);
            const unsigned hit = __ballot_sync(0xffffffffu, need <= incl);
            in = in && hit;
            const int l = hit ? __ffs(hit) - 1 : 0;
            at = at * kSegFine + l;
            run = __shfl_sync(0xffffffffu, incl - mine, l);
        }
        if (lane == 0) {
            sm.found[0] = in ? (unsigned long long)at : ~0ull;
            sm.found[1] = run;
        }
    }
    __syncthreads();
    const unsigned long long before = sm.found[1];
    const int cut = (int)sm.found[0];
    if (sm.found[0] == ~0ull) return shape_select_digits<C, true, T, VEC>(row, j0, j1, r, 0ull, p, sm);
    int n = shape_gather<C>(sm, [&](unsigned long long key) { return fine_of(bins.at(key_logit(key))) == cut; });
    shape_sync<C>();                               // the fine bins and the lists have been read
    const bool whole = n <= kShapeList;            // the window's ids are all in the lists
    if (!whole) {                                  // another pass, for the fine bin's alone
        if (tid == 0) sm.n_own = 0;
        __syncthreads();
        shape_walk<T, VEC>(row, j0, j1, [&](float l, int id) {
            const float x = bins.at(l);
            if (x >= from && x < to && fine_of(x) == cut && shape_keeps(l, id, r)) shape_keep_key(sm, l, id);
        });
        shape_sync<C>();
        n = shape_gather<C>(sm, [](unsigned long long) { return true; });
        shape_sync<C>();
    }
    if (n > kShapeList) return shape_select_digits<C, true, T, VEC>(row, j0, j1, r, 0ull, p, sm);
    for (int i = tid; i < n; i += kShapeThreads) sm.mass[i] = shape_mass(shape_exponent(key_logit(sm.keys[i]), r));
    if (lane == 0) sm.part[warp] = 0;
    __syncthreads();
    unsigned long long last = 0;                   // inverted: the smallest kept key as a maximum
    for (int i = tid; i < n; i += kShapeThreads) {
        unsigned long long t = before;
        for (int j = 0; j < n; ++j) t += sm.keys[j] > sm.keys[i] ? sm.mass[j] : 0ull;
        if (t < need && ~sm.keys[i] > last) last = ~sm.keys[i];
    }
    __syncthreads();
    unsigned long long high = warp_max_u64(last);
    if (lane == 0 && high) atomicMax(&sm.found[2], high);
    // the window's kept ids, by the warps that they belong to
    __syncthreads();
    const unsigned long long bound = ~sm.found[2];
    if (!whole) return bound;
    const int first = shape_rank<C>() * kShapeWarps * per;
    for (int i = tid; i < sm.n_own; i += kShapeThreads) {
        const unsigned long long key = sm.own[i];
        if (key >= bound) atomicAdd(&sm.part[((int)~(uint32_t)key - first) / per], shape_mass(shape_exponent(key_logit(key), r)));
    }
    __syncthreads();
    if (lane == 0) sm.part[warp] += sm.part2[warp];
    *parts = true;
    return bound;
}

// The rest of a row whose kept ids are all among sm.keys[0 .. n): top-k by rank, top-p, min-p, and the token (-1: no u).  Every CTA of
// the cluster computes the same.
__device__ __forceinline__ int shape_from_list(RowShape& r, const Shaping& s, int n, float u, ShapeSmem& sm, unsigned long long& total) {
    const float low = shape_low(r.m, r.c);
    const int tid = threadIdx.x;
    constexpr int kMine = kShapeList / kShapeThreads;
    for (int i = tid; i < n; i += kShapeThreads) {
        const float l = key_logit(sm.keys[i]);
        sm.mass[i] = l >= low ? shape_mass(shape_exponent(l, r)) : 0ull;
    }
    __syncthreads();
    unsigned long long before[kMine], sum = 0;
    bool kept[kMine];
#pragma unroll
    for (int e = 0; e < kMine; ++e) {
        const int i = tid + e * kShapeThreads;
        int rank = 0;
        before[e] = 0;
        kept[e] = false;
        if (i < n) {
            const unsigned long long key = sm.keys[i];
            for (int j = 0; j < n; ++j) {
                const bool up = sm.keys[j] > key;
                rank += up;
                before[e] += up ? sm.mass[j] : 0ull;
            }
            kept[e] = rank < s.k;
            if (kept[e]) sum += sm.mass[i];
        }
    }
    if (s.p < 1.f) {
        const unsigned long long all = cta_reduce_u64<false>(sum, sm.part);
        const unsigned long long need = (unsigned long long)ceil((double)s.p * (double)all);
#pragma unroll
        for (int e = 0; e < kMine; ++e) kept[e] = kept[e] && before[e] < need;
    }
    sum = 0;
    unsigned long long last = 0;                   // inverted: the smallest kept key as a maximum
#pragma unroll
    for (int e = 0; e < kMine; ++e) {
        const int i = tid + e * kShapeThreads;
        kept[e] = kept[e] && key_logit(sm.keys[i]) >= r.cut;      // (min-p, and what has no mass)
        if (kept[e]) {
            sum += sm.mass[i];
            last = ~sm.keys[i] > last ? ~sm.keys[i] : last;
        }
    }
    const unsigned long long bound = ~cta_reduce_u64<true>(last, sm.part2);
    r.cut = key_logit(bound);
    r.cut_id = (int)~(uint32_t)bound;
    __syncthreads();
    total = cta_reduce_u64<false>(sum, sm.part);
    if (tid == 0) sm.window[0] = -1;
    __syncthreads();
    if (!(u >= 0.f)) return -1;
    // in id order: an id's low key bits are its complement
    const unsigned long long target = (unsigned long long)floor((double)u * (double)total);
#pragma unroll
    for (int e = 0; e < kMine; ++e) {
        const int i = tid + e * kShapeThreads;
        if (!kept[e]) continue;
        const uint32_t id = (uint32_t)sm.keys[i];
        unsigned long long run = 0;
        for (int j = 0; j < n; ++j) run += sm.keys[j] >= bound && (uint32_t)sm.keys[j] > id ? sm.mass[j] : 0ull;
        if (run <= target && target < run + sm.mass[i]) sm.window[0] = (int)~id;
    }
    __syncthreads();
    return sm.window[0];
}

// The lowest logit whose weight is at least min_p: log2(min_p) is met or not met by an exponent as it is computed, so the quotient is
// only a first guess.
__device__ __forceinline__ float shape_min_p(float m, double c, double min_p) {
    const double y = log2(min_p), guess = (double)m + y / c;
    auto meets = [&](float l) { return ((double)l - (double)m) * c >= y; };
    if (!(guess > -3.4e38)) return -INFINITY;
    float l = (float)guess;
    for (int i = 0; i < 4 && !meets(l); ++i) l = nextafterf(l, INFINITY);
    for (int i = 0; i < 4 && meets(nextafterf(l, -INFINITY)); ++i) l = nextafterf(l, -INFINITY);
    return l;
}

// One row: its shape, and with kDraw its token and, where asked for, its probabilities.
template <int C, bool kDraw, typename T, int VEC>
__device__ void shape_row(const T* row, int V, const Shaping s, float u, int32_t* token, float* probs, RowShape* out, ShapeSmem& sm) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = shape_rank<C>();
    constexpr int kStep = 32 * VEC;
    const int per = ((V + C * kShapeWarps - 1) / (C * kShapeWarps) + kStep - 1) / kStep * kStep;     // ids of a warp
    const int j0 = min(V, (rank * kShapeWarps + warp) * per), j1 = min(V, j0 + per);

    const bool sane = s.t >= 0.f && s.t <= kShapeMaxT && s.p > 0.f && s.mp >= 0.f && s.mp <= 1.f && (!kDraw || (u >= 0.f && u < 1.f));
    const bool cut_k = sane && s.t > 0.f && s.k > 0 && s.k < V, cut_p = sane && s.t > 0.f && s.p < 1.f;
    if (tid == 0) { sm.n_own = 0; sm.found[2] = 0; }
    ShapeBins bins = {0.f, cut_k ? kShapeWidth : kShapeWidth / s.t};
    if (cut_k || cut_p) {
        for (int b = tid; b < kShapeBins; b += kShapeThreads) sm.coarse[b] = 0;
        float first = -INFINITY;                   // of the row's first ids, the same in all CTAs
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (tid + i * kShapeThreads < V) first = fmaxf(first, logit_f32(row[tid + i * kShapeThreads]));
        const unsigned long long f = cta_reduce_u64<true>(first > -INFINITY && first < INFINITY ? order_key(first, 0) : 0ull, sm.part2);
        bins.from = (f ? key_logit(f) : 0.f) + (cut_k ? kShapeUp : kShapeUp * s.t);
        if (!(bins.inv < 1e30f)) bins.inv = 1e30f; // (a tiny temperature: the bins are of no use, and found to be so)
    }
    // ---- first pass: the first of the order (a NaN or +inf anywhere shows as the largest key there is), and the bins
    float best = -INFINITY;
    int best_id = 0;                               // (only looked for where it is the row's token)
    bool bad = false;
    auto look = [&](float l) {
        bad |= !(l < INFINITY);
        best = fmaxf(best, l);
    };
    if (cut_k) shape_walk<T, VEC>(row, j0, j1, [&](float l, int) { look(l); shape_count<false>(bins, l, sm.coarse); });
    else if (cut_p) shape_walk<T, VEC>(row, j0, j1, [&](float l, int) { look(l); shape_count<true>(bins, l, sm.coarse); });
    else if (s.t > 0.f) shape_walk<T, VEC>(row, j0, j1, [&](float l, int) { look(l); });
    else
        shape_walk<T, VEC>(row, j0, j1, [&](float l, int id) {
            bad |= !(l < INFINITY);
            if (l > best) { best = l; best_id = id; }
        });
    unsigned long long top = cta_reduce_u64<true>(bad ? ~0ull : best > -INFINITY ? order_key(best, best_id) : 0ull, sm.part);
    if (cut_k) shape_segments<false>(sm);
    else if (cut_p) shape_segments<true>(sm);
    if (tid == 0) sm.cta[0] = top;
    shape_sync<C>();
    if (C > 1) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const unsigned long long t = shape_peer<C>(&sm.cta[0], c);
            top = t > top ? t : top;
        }
    }

    RowShape r;
    r.m = r.c = 0.0;
    r.cut = -INFINITY;                             // keeps everything
    r.cut_id = V;
    const bool empty = top == 0ull || top == ~0ull || !sane;          // uniform over the cluster
    unsigned long long total = 0;
    int drawn = -1, listed = 0;
    bool parts = false;                            // sm.part holds the kept masses of this CTA's warps
    bool done = empty;                             // token and total are known (to every CTA)
    if (!empty) {
        const float m = key_logit(top);
        r.m = (double)m;
        r.c = s.t > 0.f ? 1.4426950408889634074 / (double)s.t : 0.0;
        if (s.t == 0.f) {
            r.cut = m;
            r.cut_id = drawn = (int)~(uint32_t)top;
            total = 1ull << 45;
            done = true;
        } else {
            float floor_ = shape_low(r.m, r.c);
            if (s.mp > 0.f) floor_ = fmaxf(floor_, shape_min_p(m, r.c, (double)s.mp));
            // the first pass' bins, unless the maximum lies above them
            auto again = [&](float from, float inv) {
                bins.from = from;
                bins.inv = inv;
            };
            unsigned long long bound = 0;
            if (cut_k) {
                if (!(m <= bins.from)) {
                    again(m, kShapeWidth);
                    shape_coarse<false, T, VEC>(row, j0, j1, bins, r, sm);
                    shape_sync<C>();
                }
                bound = shape_top_k<C, T, VEC>(row, j0, j1, r, bins, s.k, sm, &listed);
            }
            if (listed) {
                r.cut = floor_;
                drawn = shape_from_list(r, s, listed, kDraw ? u : -1.f, sm, total);
                done = true;
            } else {
                auto keep_from = [&](float cut, int id) {
                    if (cut > r.cut) { r.cut = cut; r.cut_id = id; }
                };
                auto keep_key = [&](unsigned long long b) { keep_from(key_logit(b), (int)~(uint32_t)b); };
                if (bound) keep_key(bound);
                keep_from(shape_low(r.m, r.c), V);
                if (cut_p) {
                    unsigned long long b;
                    if (!(kShapeWidth / s.t < 1e30f)) {
                        b = shape_select_digits<C, true, T, VEC>(row, j0, j1, r, 0ull, (double)s.p, sm);
                    } else {
                        if (cut_k || !(m <= bins.from)) {
                            if (cut_k) {
                                shape_sync<C>();   // (the lists of the first cut have been read)
                                if (tid == 0) { sm.n_own = 0; sm.found[2] = 0; }
                            }
                            again(m, kShapeWidth / s.t);
                            shape_coarse<true, T, VEC>(row, j0, j1, bins, r, sm);
                            shape_sync<C>();
                        }
                        b = shape_top_p<C, T, VEC>(row, j0, j1, r, bins, s.p, sm, V, per, &parts);
                    }
                    r.cut = key_logit(b);          // (among what was kept: never lower)
                    r.cut_id = (int)~(uint32_t)b;
                }
                if (floor_ > r.cut) parts = false;
                keep_from(floor_, V);
            }
        }
    }
    if (!done) {
        // ---- mass of what is kept: this warp's, the CTA's, the row's
        unsigned long long mass = 0;
        if (!parts) {
            mass = warp_sum_u64(shape_mass_sum<T, VEC>(row, j0, j1, r, V));
            __syncthreads();
            if (lane == 0) sm.part[warp] = mass;
        }
        __syncthreads();
        unsigned long long mine = 0, before = 0;   // this CTA's mass, and that of the ids before its own
#pragma unroll
        for (int w = 0; w < kShapeWarps; ++w) mine += sm.part[w];
        total = mine;
        if (C > 1) {
            if (tid == 0) sm.cta[1] = mine;
            cluster_sync_all();
            total = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const unsigned long long t = shape_peer<C>(&sm.cta[1], c);
                if (c < rank) before += t;
                total += t;
            }
        }
        if (kDraw) {
            // First id whose running mass exceeds u * total.  It is among the ids of the one warp whose share of the sum holds the target; all
            // warps of its CTA add those up once more, a part each, and one of them walks its part (a warp alone takes 50 us for a sixteenth
            // of 128256 ids).
            const unsigned long long target = (unsigned long long)floor((double)u * (double)total);
            if (before <= target && target < before + mine) {
                auto owner = [&](const unsigned long long* part, int& w) {
                    for (w = 0; w < kShapeWarps - 1 && target >= before + part[w]; ++w) before += part[w];
                };
                int w;
                owner(sm.part, w);
                int o0 = min(V, (rank * kShapeWarps + w) * per), o1 = min(V, o0 + per);
                const int sub = ((o1 - o0 + kShapeWarps - 1) / kShapeWarps + 31) / 32 * 32;
                const int s0 = min(o1, o0 + warp * sub), s1 = min(o1, s0 + sub);
                const unsigned long long some = warp_sum_u64(shape_mass_sum<T, 1>(row, s0, s1, r, V));
                if (lane == 0) sm.part2[warp] = some;
                __syncthreads();
                owner(sm.part2, w);
                if (w == warp) {
                    unsigned long long run = before;
                    for (int j = s0; j < s1; j += 32) {
                        const int id = j + lane;
                        const float l = id < s1 ? logit_f32(row[id]) : -INFINITY;
                        const unsigned long long mass_ = shape_keeps(l, id, r) ? shape_mass(shape_exponent(l, r)) : 0ull;
                        const unsigned long long incl = run + warp_scan_u64(mass_);
                        const unsigned over = __ballot_sync(0xffffffffu, incl > target);
                        if (over) {
                            if (lane == 0) *token = j + __ffs(over) - 1;
                            break;
                        }
                        run = __shfl_sync(0xffffffffu, incl, 31);
                    }
                }
            }
        }
    }
    if (out && rank == 0 && tid == 0) {
        r.total = total;
        *out = r;
    }
    if (kDraw) {
        if (done && rank == 0 && tid == 0) *token = drawn;
        if (probs) {
            const double scale = done && empty ? 0.0 : kMassOne / (double)total;
            if (done) {                            // few ids, or none: zeros first
                if (VEC > 1 && ((uintptr_t)probs & 15) == 0)
                    for (int j = j0 + lane * 4; j < j1; j += 128) {
                        if (j + 4 <= j1) *reinterpret_cast<float4*>(probs + j) = make_float4(0.f, 0.f, 0.f, 0.f);
                        else
                            for (int i = j; i < j1; ++i) probs[i] = 0.f;
                    }
                else
                    for (int j = j0 + lane; j < j1; j += 32) probs[j] = 0.f;
                __syncthreads();
                const int c0 = min(V, rank * kShapeWarps * per), c1 = min(V, c0 + kShapeWarps * per);     // this CTA's ids
                if (listed) {
                    for (int i = tid; i < listed; i += kShapeThreads) {
                        const unsigned long long key = sm.keys[i];
                        const int id = (int)~(uint32_t)key;
                        if (shape_keeps(key_logit(key), id, r) && id >= c0 && id < c1) probs[id] = (float)(shape_exp2(shape_exponent(key_logit(key), r)) * scale);
                    }
                } else if (!empty && tid == 0 && drawn >= c0 && drawn < c1) {
                    probs[drawn] = 1.f;
                }
            } else {
                shape_groups<T, VEC>(row, j0, j1, [&](const auto& l, int first) {
                    constexpr int kN = sizeof(l) / 4;
                    float p[kN];
                    bool any = false;
#pragma unroll
                    for (int e = 0; e < kN; ++e) {
                        p[e] = 0.f;
                        any |= shape_keeps(l[e], first + e * group_apart<VEC>(), r);
                    }
                    if (__any_sync(0xffffffffu, any)) {
#pragma unroll
                        for (int e = 0; e < kN; ++e) p[e] = (float)(shape_exp2(shape_exponent(l[e], r)) * scale);
#pragma unroll
                        for (int e = 0; e < kN; ++e) p[e] = shape_keeps(l[e], first + e * group_apart<VEC>(), r) ? p[e] : 0.f;
                    }
                    if (VEC > 1 && ((uintptr_t)probs & 15) == 0 && first + kN <= j1) {
#pragma unroll
                        for (int e = 0; e < kN; e += 4) *reinterpret_cast<float4*>(probs + first + e) = make_float4(p[e], p[e + 1 < kN ? e + 1 : e], p[e + 2 < kN ? e + 2 : e], p[e + 3 < kN ? e + 3 : e]);
                    } else {
#pragma unroll
                        for (int e = 0; e < kN; ++e) {
                            const int id = first + e * group_apart<VEC>();
                            if (id < j1) probs[id] = p[e];
                        }
                    }
                });
            }
        }
    }
    if (C > 1) cluster_sync_all();                 // nobody leaves while another one still reads its shared memory
}

struct ShapeArgs {
    const void* logits;
    long long stride;          // elements between rows
    int V, first, rows;        // rows first .. first + rows - 1
    bool more;                 // the grid behind this one has the rest of the rows
    const Shaping* shaping;    // of all rows, or [n_req] with row0
    const int32_t* row0;       // nullable: [n_req + 1]
    int n_req;
    const float* u;
    int32_t* tokens;
    float* probs;
    long long probs_stride;
    RowShape* shapes;
};

// grid rows * C, cluster C.
template <int C, bool kDraw, typename T, int VEC>
__global__ void __launch_bounds__(kShapeThreads, 2) shape_kernel(const ShapeArgs a) {
    __shared__ ShapeSmem sm;
    if (a.more) pdl_launch_dependents();
    const int row = a.first + blockIdx.x / C;
    const T* lr = static_cast<const T*>(a.logits) + (size_t)row * a.stride;
    if (kDraw) {
        shape_row<C, true, T, VEC>(lr, a.V, a.shaping[row], a.u[row], a.tokens + row, a.probs ? a.probs + (size_t)row * a.probs_stride : nullptr,
                                   nullptr, sm);
    } else {
        // The lowest of the requests that claim the row (several may, where entries of row0 make no sense): the one that acceptance looks at,
        // if there is one, and the same in all CTAs of the cluster, whose barriers go by its settings.
        __shared__ int s_req;
        if (threadIdx.x == 0) s_req = a.n_req;
        __syncthreads();
        for (int i = threadIdx.x; i < a.n_req; i += kShapeThreads)
            if (a.row0[i] <= row && row < a.row0[i + 1]) {
                atomicMin(&s_req, i);
                break;
            }
        __syncthreads();
        const int req = s_req;                     // (n_req: a row that is no request's)
        if (req < a.n_req) shape_row<C, false, T, VEC>(lr, a.V, a.shaping[req], 0.f, nullptr, nullptr, a.shapes + row, sm);
    }
    // What follows may begin to launch, and waits for this grid before it reads.  (A grid of the rest of a call's rows runs beside the one
    // before it, and ends after it.)
    pdl_launch_dependents();
    pdl_wait();
}

// ---- acceptance -----------------------------------------------------------------------------------------------------------
struct AcceptArgs {
    const void* logits;
    long long stride;
    int V, rows;
    const int32_t* row0;
    int n_req;
    const float* q;            // [rows - n_req][V]: row i of request r at row0[r] - r + i
    long long q_stride;
    const int32_t* drafts;     // [rows - n_req]
    const float* u;            // [rows]: k + 1 per request, the last one for the final draw
    const RowShape* shapes;
    int32_t *n_accepted, *next_token;
};

constexpr int kAcceptThreads = 512;
constexpr int kAcceptBatch = 8;                    // steps of 32 ids whose loads are in flight together

// A cluster of kCluster CTAs per request, grid (kCluster, n_req).  The tests are independent of one another: thread i takes draft i, the first
// failure counts.  The draw is an inverse CDF in id order over fp64 terms, max(0, P - q) or P: warp w of CTA r adds the ids
// [(r * 16 + w) * R, + R) batch by batch of 256, the totals are added in warp and rank order, and the one warp whose range
// holds u * total goes through the batch that does again.  Bound by the latencies of five dependent loads and by the fp64 terms: with 1024 threads
// a CTA, one to an SM, and the whole range walked again, 310 rows of 128256 ids for 32 requests took 151 us, rows included; so 143.
template <int kAcceptCluster, typename T>
__global__ void __launch_bounds__(kAcceptThreads, 2) accept_shaped_kernel(const AcceptArgs a) {
    cluster_started_arrive();                      // (totals are stored into the other CTAs below)
    pdl_wait();                                    // launched with programmatic serialisation: the shapes must be there
    cluster_started_wait();
    constexpr int kWarps = kAcceptThreads / 32;
    const int req = blockIdx.y, rank = (int)cluster_ctarank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ int s_first;
    __shared__ double s_warp[kWarps], s_incl[kWarps], s_cta[2][kAcceptCluster], s_base, s_total;
    const int first = a.row0[req], end = a.row0[req + 1];
    // A request whose entries make sense: rows and drafts that are there, and no entry of an earlier request behind its first row, so that no
    // two such requests share a row.
    bool later = false;
    for (int i = tid; i < req; i += kAcceptThreads) later |= a.row0[i] > first;
    if (tid == 0) s_first = a.rows;
    const bool sane = !__syncthreads_or(later) && first >= req && end > first && end <= a.rows && end - req - 1 <= a.rows - a.n_req;
    const int k = sane ? end - first - 1 : 0, slot0 = sane ? first - req : 0;     // slot0: of the request's first draft
    if (!sane) {                                   // no such rows (the whole cluster leaves)
        if (rank == 0 && tid == 0) { a.n_accepted[req] = 0; a.next_token[req] = -1; }
        return;
    }
    const T* logits = static_cast<const T*>(a.logits) + (size_t)first * a.stride;
    auto prob = [&](const T* row, const RowShape& r, int id, double scale) {
        const float l = logit_f32(row[id]);
        return shape_keeps(l, id, r) ? __dmul_rn(shape_exp2(shape_exponent(l, r)), scale) : 0.0;       // (no contraction: the same in every pass)
    };
    for (int i = tid; i < k; i += kAcceptThreads) {
        const RowShape r = a.shapes[first + i];
        const int x = a.drafts[slot0 + i];
        bool ok = false;
        if (r.total && x >= 0 && x < a.V) {
            const double p = prob(logits + (size_t)i * a.stride, r, x, kMassOne / (double)r.total);
            const double q = (double)a.q[(size_t)(slot0 + i) * a.q_stride + x];
            const double ratio = q > 0.0 ? p / q : (p > 0.0 ? INFINITY : 0.0), ui = (double)a.u[first + i];
            ok = q >= 0.0 && ui >= 0.0 && ui < fmin(ratio, 1.0);         // (no NaN, and nothing below 0)
        }
        if (!ok) atomicMin(&s_first, i);
    }
    __syncthreads();
    const int n = min(s_first, k);
    const RowShape r = a.shapes[first + n];
    const float uk = a.u[first + k];
    if (r.total == 0 || !(uk >= 0.f && uk < 1.f)) {
        if (rank == 0 && tid == 0) { a.n_accepted[req] = n; a.next_token[req] = -1; }
        return;
    }
    const T* lr = logits + (size_t)n * a.stride;
    const double scale = kMassOne / (double)r.total;
    constexpr int kAllWarps = kAcceptCluster * kWarps;
    const int R = ((a.V + kAllWarps - 1) / kAllWarps + 31) / 32 * 32;
    static_assert(kShapeMaxVocab <= kAllWarps * 32 * 32 * kAcceptBatch, "a lane per batch");
    const int j0 = min(a.V, (rank * kWarps + warp) * R), j1 = min(a.V, j0 + R);
    bool use_q = n < k;
    const float* qr = a.q + (size_t)(slot0 + (use_q ? n : 0)) * a.q_stride;
    // The terms of kAcceptBatch steps of 32 ids, this lane's.  (One step at a time, each waits for the L2: 20 us for a walk of 16.)
    auto terms = [&](int j, double (&t)[kAcceptBatch]) {
        float l[kAcceptBatch], q[kAcceptBatch];
#pragma unroll
        for (int i = 0; i < kAcceptBatch; ++i) {
            const bool in = j + 32 * i < j1;
            l[i] = in ? logit_f32(lr[j + 32 * i]) : -INFINITY;
            q[i] = in && use_q ? qr[j + 32 * i] : 0.f;
        }
        bool keep[kAcceptBatch], any = false;
#pragma unroll
        for (int i = 0; i < kAcceptBatch; ++i) {
            keep[i] = shape_keeps(l[i], j + 32 * i, r);
            any |= keep[i];
            t[i] = 0.0;
        }
        if (!__any_sync(0xffffffffu, any)) return;
        double w[kAcceptBatch];                    // side by side, without a branch between them
#pragma unroll
        for (int i = 0; i < kAcceptBatch; ++i) w[i] = __dmul_rn(shape_exp2(shape_exponent(keep[i] ? l[i] : r.cut, r)), scale);
#pragma unroll
        for (int i = 0; i < kAcceptBatch; ++i)     // (a q that is no probability makes the sum a NaN)
            t[i] = !keep[i] ? 0.0 : q[i] >= 0.f ? fmax(0.0, w[i] - (double)q[i]) : (double)NAN;
    };
    for (int attempt = 0; attempt < 2; ++attempt) {
        double sum = 0.0, batch_sum = 0.0;         // lane b: the sum of batch b
        int n_batch = 0;
        for (int j = j0; j < j1; j += 32 * kAcceptBatch, ++n_batch) {     // (all lanes together)
            double t[kAcceptBatch], part = 0.0;
            terms(j + lane, t);
#pragma unroll
            for (int i = 0; i < kAcceptBatch; ++i) part += t[i];
            part = warp_sum_d(part);
            if (lane == n_batch) batch_sum = part;
            sum += part;
        }
        if (lane == 0) s_warp[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            double inc = 0.0, before = 0.0, all = 0.0;       // in order: a warp without mass ends where it starts, exactly
#pragma unroll
            for (int i = 0; i < kWarps; ++i) {
                if (i == lane) before = all;
                all += s_warp[i];
                if (i == lane) inc = all;
            }
            __syncwarp();
            if (lane < kWarps) {
                s_warp[lane] = before;
                s_incl[lane] = inc;
            }
            if (lane < kAcceptCluster)
                asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(dsmem_addr(smem_u32(&s_cta[attempt][rank]), (uint32_t)lane)), "d"(all) : "memory");
        }
        cluster_sync_all();
        if (tid == 0) {
            double run = 0.0;
            for (int c = 0; c < kAcceptCluster; ++c) {
                if (c == rank) s_base = run;
                run += s_cta[attempt][c];
            }
            s_total = run;
        }
        __syncthreads();
        const double total = s_total;
        if (!(total < INFINITY)) {                 // a NaN, or below 0, among the q of the row: nothing to draw from
            if (rank == 0 && tid == 0) { a.n_accepted[req] = n; a.next_token[req] = -1; }
            return;
        }
        if (use_q && !(total > 0.0)) {             // P <= q everywhere: the draw is from P
            use_q = false;
            __syncthreads();
            continue;
        }
        const double target = (double)uk * total, start = s_base + s_warp[warp];
        if (s_base + s_incl[warp] > target && !(start > target)) {        // one warp of the cluster
            // its batch with the target (or, where rounding falls short of that, the last one with mass), then the id
            double run = start, before = start;
            int at = 0;
            for (int i = 0; i < n_batch; ++i) {
                const double part = __shfl_sync(0xffffffffu, batch_sum, i);
                if (part > 0.0) { at = i; before = run; }
                run += part;
                if (part > 0.0 && run > target) break;
            }
            int token = -1, last = -1;
            const int j = j0 + at * 32 * kAcceptBatch;
            double own[kAcceptBatch];
            terms(j + lane, own);
            run = before;
#pragma unroll
            for (int i = 0; i < kAcceptBatch; ++i) {
                if (token >= 0) continue;
                double inc = own[i];
                const unsigned mass = __ballot_sync(0xffffffffu, inc > 0.0);
                if (!mass) continue;
                last = j + 32 * i + 31 - __clz(mass);
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double t = __shfl_up_sync(0xffffffffu, inc, o);
                    if (lane >= o) inc += t;
                }
                const unsigned hit = __ballot_sync(0xffffffffu, own[i] > 0.0 && run + inc > target);
                if (hit) token = j + 32 * i + __ffs(hit) - 1;
                run += __shfl_sync(0xffffffffu, inc, 31);
            }
            if (token < 0) token = last;           // the walk's rounding fell short of the batch's total
            if (lane == 0) { a.n_accepted[req] = n; a.next_token[req] = token; }
        }
        break;
    }
}

}  // namespace pipesd
