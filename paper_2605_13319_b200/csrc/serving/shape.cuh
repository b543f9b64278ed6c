// Shaped next-token distributions: temperature, top-k, top-p and min-p on rows of logits, and the two things that are done with
// them, drawing a token (sample) and the acceptance rule of speculative sampling (accept).
//
// A row's ids are ordered by logit, highest first, equal ones by id, lowest first.  With w_j = exp((l_j - max) / T) (T = 0: 1 for
// the first of the order, 0 for the others) the settings keep
//   top-k   the first k ids of the order (k <= 0: all),
//   top-p   of these the shortest prefix that holds at least p of their mass: an id stays while the mass before it is < p * Z,
//   min-p   of these the ids with w_j >= min_p,
// and P_j = w_j / (sum of the kept w).  All three cut the order somewhere, so that a row's outcome is one 64-bit bound: the key of
// the last kept id (sortable logit bits, then inverted id), plus the min-p bound on the exponent.
//
// Masses are 64-bit whole numbers, w * 2^45 rounded to nearest: sums do not depend on their order, a prefix never decreases, and no
// result changes between runs, cluster sizes or passes.  At most 2^18 ids, so a sum stays below 2^63; what rounding moves is
// 2^-46 of the most likely id's weight per id, and an id below that has no mass at all.  Weights are evaluated in fp64.
#pragma once
#include "../common.cuh"

namespace pipesd {

constexpr int kShapeThreads = 512;
constexpr int kShapeWarps = kShapeThreads / 32;
constexpr int kShapeBins = 2048;
constexpr int kShapeMaxVocab = 1 << 18;
constexpr double kMassOne = 35184372088832.0;      // 2^45

struct Shaping { float t; int k; float p, mp; };   // pipesd_shaping

// What the rest of a call needs to know about a row: P_id = exp2((l - m) * c) / (total * 2^-45) where key >= bound and the exponent
// is >= y_min.  total = 0: the row has no distribution (no finite logit, a NaN or +inf among them, settings out of range).
struct RowShape {
    double m, c, y_min;
    unsigned long long bound, total;
};

__device__ __forceinline__ float logit_f32(float v) { return v; }
__device__ __forceinline__ float logit_f32(uint16_t v) { return bf16_bits_to_f32(v); }

// Position in the order as a number: larger = earlier.  The addition makes -0 a +0, so that the two tie.
__device__ __forceinline__ unsigned long long order_key(float l, int id) {
    const uint32_t b = __float_as_uint(l + 0.f);
    const uint32_t s = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return (unsigned long long)s << 32 | (uint32_t)~id;
}

__device__ __forceinline__ double shape_exponent(float l, const RowShape& r) { return fmax(((double)l - r.m) * r.c, -1000.0); }
__device__ __forceinline__ unsigned long long shape_mass(double y) { return (unsigned long long)__double2ull_rn(exp2(y) * kMassOne); }
__device__ __forceinline__ bool shape_keeps(float l, int id, const RowShape& r) {
    return order_key(l, id) >= r.bound && shape_exponent(l, r) >= r.y_min;
}

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

struct ShapeSmem {
    unsigned long long hist[2][kShapeBins];        // a level's bins; levels take turns, so that one barrier per level is enough
    unsigned long long part[kShapeWarps];
    unsigned long long cta[2];                     // what the other CTAs of the cluster read: key maximum, kept mass
    unsigned long long found[3];                   // bin, sum above it, level's sum
};

// Walks this warp's ids of the row, VEC neighbours per lane and step, kBatch steps' loads in flight together.
template <typename T, int VEC, typename F>
__device__ __forceinline__ void shape_walk(const T* row, int j0, int j1, F&& f) {
    constexpr int kBatch = VEC == 1 ? 8 : 4;
    const int lane = threadIdx.x & 31;
    for (int j = j0 + lane * VEC; j < j1; j += 32 * VEC * kBatch) {
        T v[kBatch][VEC];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int i = j + b * 32 * VEC;
            if (i >= j1) continue;
            if (VEC == 1) v[b][0] = row[i];
            else if (i + VEC <= j1) *reinterpret_cast<uint4*>(v[b]) = *reinterpret_cast<const uint4*>(row + i);
            else
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (i + e < j1) v[b][e] = row[i + e];
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (j + b * 32 * VEC + e < j1) f(logit_f32(v[b][e]), j + b * 32 * VEC + e);
    }
}

// The key at which a running sum over the order, of ones (kMass false) or of masses, first reaches `need`: everything from it upwards
// is kept.  Radix descent over the key's digits (32 bits of logit, 22 of id), among keys >= floor_.  Returns floor_ if the whole sum stays
// below `need`.
template <int C, bool kMass, typename T, int VEC>
__device__ unsigned long long shape_select(const T* row, int j0, int j1, const RowShape& r, unsigned long long floor_, unsigned long long need,
                                           double need_share, ShapeSmem& sm, int& turn) {
    const int tid = threadIdx.x;
    unsigned long long prefix = 0;
    int known = 0;                                 // leading bits of the key that are settled
    constexpr int kBits[5] = {11, 11, 10, 11, 11};
#pragma unroll 1
    for (int level = 0; level < 5; ++level) {
        if (level == 3) {                          // ids are below 2^22: ten more bits are ones
            prefix = prefix << 10 | 1023u;
            known += 10;
        }
        const int bits = kBits[level], shift = 64 - known - bits;
        unsigned long long* hist = sm.hist[turn & 1];
        for (int b = tid; b < kShapeBins; b += kShapeThreads) hist[b] = 0;
        __syncthreads();
        shape_walk<T, VEC>(row, j0, j1, [&](float l, int id) {
            const unsigned long long key = order_key(l, id);
            if (key < floor_ || (known && key >> (64 - known) != prefix)) return;
            const unsigned long long add = kMass ? shape_mass(shape_exponent(l, r)) : 1ull;
            if (add) atomicAdd(hist + (size_t)((key >> shift) & ((1u << bits) - 1)), add);
        });
        shape_sync<C>();
        // bins from the top: thread t takes four neighbours; all CTAs add up the same numbers
        unsigned long long mine[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = kShapeBins - 1 - (tid * 4 + i);
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
        if (level == 0 && (all < need || need == 0)) return floor_;     // the same in every thread of the cluster
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (above < need && need <= above + mine[i]) {
                sm.found[0] = (unsigned long long)(kShapeBins - 1 - (tid * 4 + i));
                sm.found[1] = above;
            }
            above += mine[i];
        }
        __syncthreads();
        prefix = prefix << bits | sm.found[0];
        need -= sm.found[1];
        known += bits;
        ++turn;
        __syncthreads();
    }
    return prefix;
}

// One row: its shape, and with kDraw its token and, where asked for, its probabilities.
template <int C, bool kDraw, typename T, int VEC>
__device__ void shape_row(const T* row, int V, const Shaping s, float u, int32_t* token, float* probs, RowShape* out, ShapeSmem& sm) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = shape_rank<C>();
    constexpr int kStep = 32 * VEC;
    const int per = ((V + C * kShapeWarps - 1) / (C * kShapeWarps) + kStep - 1) / kStep * kStep;     // ids of a warp
    const int j0 = min(V, (rank * kShapeWarps + warp) * per), j1 = min(V, j0 + per);

    // ---- the first of the order; a NaN or +inf anywhere shows as the largest key there is
    float best = -INFINITY;
    int best_id = V;
    bool bad = false;
    shape_walk<T, VEC>(row, j0, j1, [&](float l, int id) {
        bad |= !(l < INFINITY);
        if (l > best) { best = l; best_id = id; }
    });
    unsigned long long top = bad ? ~0ull : best_id < V ? order_key(best, best_id) : 0ull;
    top = warp_max_u64(top);
    if (lane == 0) sm.part[warp] = top;
    __syncthreads();
    if (warp == 0) {
        top = warp_max_u64(lane < kShapeWarps ? sm.part[lane] : 0ull);
        if (lane == 0) sm.cta[0] = top;
    }
    shape_sync<C>();
    top = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const unsigned long long t = shape_peer<C>(&sm.cta[0], c);
        top = t > top ? t : top;
    }

    RowShape r;
    const bool sane = s.t >= 0.f && s.t < INFINITY && s.p > 0.f && s.mp >= 0.f && s.mp <= 1.f && (!kDraw || (u >= 0.f && u < 1.f));
    const bool empty = top == 0ull || top == ~0ull || !sane;          // uniform over the cluster
    unsigned long long mass = 0;
    if (!empty) {
        const uint32_t b = (uint32_t)(top >> 32);
        r.m = (double)__uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
        r.c = s.t > 0.f ? 1.4426950408889634074 / (double)s.t : 0.0;
        r.y_min = s.mp > 0.f ? log2((double)s.mp) : -INFINITY;
        r.bound = 0;
        if (s.t == 0.f) {
            r.bound = top;
        } else {
            int turn = 0;
            if (s.k > 0 && s.k < V) r.bound = shape_select<C, false, T, VEC>(row, j0, j1, r, 0ull, (unsigned long long)s.k, 0.0, sm, turn);
            if (s.p < 1.f) r.bound = shape_select<C, true, T, VEC>(row, j0, j1, r, r.bound, 0ull, (double)s.p, sm, turn);
        }
        // ---- mass of what is kept: this warp's, the CTA's, the row's
        shape_walk<T, VEC>(row, j0, j1, [&](float l, int id) {
            if (shape_keeps(l, id, r)) mass += shape_mass(shape_exponent(l, r));
        });
        mass = warp_sum_u64(mass);
    }
    __syncthreads();
    if (lane == 0) sm.part[warp] = mass;
    __syncthreads();
    if (tid == 0) {
        unsigned long long t = 0;
        for (int w = 0; w < kShapeWarps; ++w) t += sm.part[w];
        sm.cta[1] = t;
    }
    shape_sync<C>();
    unsigned long long total = 0, before = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const unsigned long long t = shape_peer<C>(&sm.cta[1], c);
        if (c < rank) before += t;
        total += t;
    }
    for (int w = 0; w < warp; ++w) before += sm.part[w];
    if (out && rank == 0 && tid == 0) {
        r.total = empty ? 0ull : total;
        *out = r;
    }
    if (kDraw) {
        if (empty) {
            if (rank == 0 && tid == 0) *token = -1;
            if (probs)
                for (int j = j0 + lane; j < j1; j += 32) probs[j] = 0.f;
        } else {
            // first id whose running mass exceeds u * total: in the one warp whose share of the sum holds it
            const unsigned long long target = (unsigned long long)floor((double)u * (double)total);
            if (before <= target && target < before + mass) {
                unsigned long long run = before;
                for (int j = j0; j < j1; j += 32) {
                    const int id = j + lane;
                    const float l = id < j1 ? logit_f32(row[id]) : -INFINITY;
                    const unsigned long long w = id < j1 && shape_keeps(l, id, r) ? shape_mass(shape_exponent(l, r)) : 0ull;
                    const unsigned long long incl = run + warp_scan_u64(w);
                    const unsigned hit = __ballot_sync(0xffffffffu, incl > target);
                    if (hit) {
                        if (lane == 0) *token = j + __ffs(hit) - 1;
                        break;
                    }
                    run = __shfl_sync(0xffffffffu, incl, 31);
                }
            }
            if (probs) {
                const double scale = kMassOne / (double)total;
                shape_walk<T, VEC>(row, j0, j1, [&](float l, int id) {
                    probs[id] = shape_keeps(l, id, r) ? (float)(exp2(shape_exponent(l, r)) * scale) : 0.f;
                });
            }
        }
    }
    if (C > 1) cluster_sync_all();                 // nobody leaves while another one still reads its shared memory
}

struct ShapeArgs {
    const void* logits;
    long long stride;          // elements between rows
    int V, rows;
    const Shaping* shaping;    // [rows], or [n_req] with row0
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
    const int row = blockIdx.x / C;
    const T* lr = static_cast<const T*>(a.logits) + (size_t)row * a.stride;
    if (kDraw) {
        shape_row<C, true, T, VEC>(lr, a.V, a.shaping[row], a.u[row], a.tokens + row, a.probs ? a.probs + (size_t)row * a.probs_stride : nullptr,
                                   nullptr, sm);
    } else {
        __shared__ int s_req;
        if (threadIdx.x == 0) s_req = -1;
        __syncthreads();
        for (int i = threadIdx.x; i < a.n_req; i += kShapeThreads)
            if (a.row0[i] <= row && row < a.row0[i + 1]) s_req = i;
        __syncthreads();
        const int req = s_req;
        if (req < 0) return;                       // a row that is no request's (the whole cluster leaves)
        shape_row<C, false, T, VEC>(lr, a.V, a.shaping[req], 0.f, nullptr, nullptr, a.shapes + row, sm);
    }
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

constexpr int kAcceptThreads = 1024;
constexpr int kAcceptCluster = 8;

// A cluster per request, grid (kAcceptCluster, n_req).  The tests are independent of one another: thread i takes draft i, the first
// failure counts.  The draw is an inverse CDF in id order over fp64 terms, max(0, P - q) or P: warp w of CTA r adds the ids
// [(r * 32 + w) * R, + R) lane by lane, the totals are added in warp and rank order, and the one warp whose range
// holds u * total walks it again.
template <typename T>
__global__ void __launch_bounds__(kAcceptThreads) accept_shaped_kernel(const AcceptArgs a) {
    constexpr int kWarps = kAcceptThreads / 32;
    const int req = blockIdx.y, rank = (int)cluster_ctarank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ int s_first;
    __shared__ double s_warp[kWarps], s_incl[kWarps], s_cta[2][kAcceptCluster], s_base, s_total;
    const int first = a.row0[req], k = a.row0[req + 1] - first - 1;
    const int slot0 = first - req;                 // of the request's first draft
    if (k < 0 || first < 0 || first + k >= a.rows || slot0 < 0 || slot0 + k > a.rows - a.n_req) {     // no such rows (the whole cluster leaves)
        if (rank == 0 && tid == 0) { a.n_accepted[req] = 0; a.next_token[req] = -1; }
        return;
    }
    const T* logits = static_cast<const T*>(a.logits) + (size_t)first * a.stride;
    auto prob = [&](const T* row, const RowShape& r, int id, double scale) {
        const float l = logit_f32(row[id]);
        return shape_keeps(l, id, r) ? exp2(shape_exponent(l, r)) * scale : 0.0;
    };
    if (tid == 0) s_first = k;
    __syncthreads();
    for (int i = tid; i < k; i += kAcceptThreads) {
        const RowShape r = a.shapes[first + i];
        const int x = a.drafts[slot0 + i];
        bool ok = false;
        if (r.total && x >= 0 && x < a.V) {
            const double p = prob(logits + (size_t)i * a.stride, r, x, kMassOne / (double)r.total);
            const double q = (double)a.q[(size_t)(slot0 + i) * a.q_stride + x];
            const double ratio = q > 0.0 ? p / q : (p > 0.0 ? INFINITY : 0.0);
            ok = (double)a.u[first + i] < fmin(ratio, 1.0);
        }
        if (!ok) atomicMin(&s_first, i);
    }
    __syncthreads();
    const int n = s_first;
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
    const int j0 = min(a.V, (rank * kWarps + warp) * R), j1 = min(a.V, j0 + R);
    bool use_q = n < k;
    const float* qr = a.q + (size_t)(slot0 + (use_q ? n : 0)) * a.q_stride;
    auto term = [&](int j) {
        if (j >= j1) return 0.0;
        const double p = prob(lr, r, j, scale);
        return use_q ? fmax(0.0, p - (double)qr[j]) : p;
    };
    for (int attempt = 0; attempt < 2; ++attempt) {
        double sum = 0.0;
#pragma unroll 4
        for (int j = j0 + lane; j < j1; j += 32) sum += term(j);
        sum = warp_sum_d(sum);
        if (lane == 0) s_warp[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            double inc = s_warp[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double t = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += t;
            }
            const double before = __shfl_up_sync(0xffffffffu, inc, 1), all = __shfl_sync(0xffffffffu, inc, 31);
            s_warp[lane] = lane ? before : 0.0;    // a warp's start is the previous one's end, exactly
            s_incl[lane] = inc;
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
        if (use_q && !(total > 0.0)) {             // P <= q everywhere: the draw is from P
            use_q = false;
            __syncthreads();
            continue;
        }
        const double target = (double)uk * total, start = s_base + s_warp[warp];
        if (s_base + s_incl[warp] > target && !(start > target)) {        // one warp of the cluster
            double run = start;
            int token = -1, last = -1;
            for (int j = j0; j < j1 && token < 0; j += 32) {
                const double own = term(j + lane);
                double inc = own;
                const unsigned mass = __ballot_sync(0xffffffffu, inc > 0.0);
                if (mass) last = j + 31 - __clz(mass);
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double t = __shfl_up_sync(0xffffffffu, inc, o);
                    if (lane >= o) inc += t;
                }
                const unsigned hit = __ballot_sync(0xffffffffu, own > 0.0 && run + inc > target);
                if (hit) token = j + __ffs(hit) - 1;
                run += __shfl_sync(0xffffffffu, inc, 31);
            }
            if (token < 0) token = last;           // the walk's rounding fell short of the range's total
            if (lane == 0) { a.n_accepted[req] = n; a.next_token[req] = token; }
        }
        break;
    }
}

}  // namespace pipesd
