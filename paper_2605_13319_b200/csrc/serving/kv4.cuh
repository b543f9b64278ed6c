// A paged K/V cache held in 4 bits, and the attention of short chunks of query rows over it.
//
// Values: the columns of a (position, head) row are cut into groups of 32 that share a zero z = bf16(min) and a scale
// s = bf16((max - z) / 15); a value is held as the code c = clamp(rint((x - z) / s), 0, 15) and stands for s * c + z (s <= 0: c = 0).
//
// Layout of one layer: [page][KV head][unit], a unit being 16 positions of one head in 20 * HD contiguous bytes:
//   K codes   8 HD   [position 16][t 4][group]      32-bit words, nibble p = column 32 group + 8 t + p
//   K s, z    2 HD   [position 16][group]           bf16 pairs
//   V codes   8 HD   [tile / 4][g 8][t 4][tile % 4] words, tile = 16 columns; nibble p = column 16 tile + g + 8 (p & 1) of position
//                                                   2 t + (p >> 2) + 8 (p >> 1 & 1)
//   V s       HD     [group][position 16]           bf16
//   V z       HD     [group][position 16]           bf16
// Both code orders are those of the A operand of mma.m16n8k16 (lane 4 g + t): a word ANDed with 0x000f000f is a register of
// the operand, the same after shifts by 8, and with 0x00f000f0 another one.  Read as fp16 such a register holds whole numbers (n < 2048)
// times 2^-24 (subnormals: the exponent fields 0 and 1 are one linear range), so that a code needs one AND (and a shift for
// every second one) and no conversion.  The factor 16 of the odd nibbles goes into Q, or into the step that centres V's codes.
#pragma once
#include "../common.cuh"

namespace pipesd {

constexpr int kKv4Unit = 16;                       // positions of a unit
constexpr int kKv4Group = 32;                      // columns of a scale
constexpr float kKv4Limit = 281474976710656.f;     // 2^48: larger values are held as this; a NaN as 0

__host__ __device__ constexpr int kv4_unit_bytes(int hd) { return 20 * hd; }
__host__ __device__ constexpr int kv4_k_scales(int hd) { return 8 * hd; }
__host__ __device__ constexpr int kv4_v_codes(int hd) { return 10 * hd; }
__host__ __device__ constexpr int kv4_v_scales(int hd) { return 18 * hd; }

// Where the requests of a call are: request r has the rows row0[r] .. row0[r + 1] - 1, at the positions base[r] ... of its pages.
struct Kv4Where {
    const int32_t *row0, *base, *table;
    int n_req, rows, n_pages, max_pages, page_size, Hkv;
};

// New rows and base of a request; a request whose numbers make no sense has none.
__device__ __forceinline__ int kv4_rows(const Kv4Where& w, int r, int& first, int& base) {
    first = w.row0[r];
    base = w.base[r];
    const int end = w.row0[r + 1];
    if (first < 0 || end < first || end > w.rows || base < 0) return 0;
    return min(end - first, max(0, w.max_pages * w.page_size - base));      // rows behind the table's last position are dropped
}

// Address of a unit of a request, or null where no page is mapped.
__device__ __forceinline__ unsigned char* kv4_unit(unsigned char* pool, const Kv4Where& w, int r, int head, int unit, int hd) {
    const int pos = unit * kKv4Unit, page = w.table[(size_t)r * w.max_pages + pos / w.page_size];
    if (page < 0 || page >= w.n_pages) return nullptr;
    return pool + (((size_t)page * w.Hkv + head) * (w.page_size / kKv4Unit) + pos % w.page_size / kKv4Unit) * kv4_unit_bytes(hd);
}

// Eight neighbouring values as they come (wide: in 16-byte pieces), and put within the limits: a NaN as 0.
__device__ __forceinline__ void kv4_load8(const float* p, bool wide, float (&x)[8]) {
    if (wide) {
        *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(p);
        *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(p + 4);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = p[i];
    }
}
__device__ __forceinline__ void kv4_load8(const uint16_t* p, bool wide, float (&x)[8]) {
    uint32_t h[4];
    if (wide) {
        *reinterpret_cast<uint4*>(h) = *reinterpret_cast<const uint4*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = pack2(p[2 * i], p[2 * i + 1]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(h[i] << 16); x[2 * i + 1] = __uint_as_float(h[i] & 0xffff0000u); }
}
__device__ __forceinline__ void kv4_limit8(float (&x)[8]) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
    if (most <= __float_as_uint(kKv4Limit)) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] == x[i] ? fminf(fmaxf(x[i], -kKv4Limit), kKv4Limit) : 0.f;
}

// The n-th of the units that the requests' rows touch, in order (one warp; -1: there are not as many), and its number.
__device__ __forceinline__ int kv4_nth_unit(const Kv4Where& w, int nth, int& unit) {
    const int lane = threadIdx.x & 31;
    unit = 0;
    for (int r0 = 0; r0 < w.n_req; r0 += 32) {
        int first, base = 0, n = 0;
        if (r0 + lane < w.n_req) n = kv4_rows(w, r0 + lane, first, base);
        const int u0 = base / kKv4Unit, cnt = n > 0 ? (base + n - 1) / kKv4Unit - u0 + 1 : 0;
        int inc = cnt;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += t;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, nth < inc);
        if (hit) {
            const int l = __ffs(hit) - 1;
            unit = __shfl_sync(0xffffffffu, u0 + nth - (inc - cnt), l);
            return r0 + l;
        }
        nth -= __shfl_sync(0xffffffffu, inc, 31);
    }
    return -1;
}

// Scale of a group and codes of eight of its values, as the definition has them in exact arithmetic.  fp32 decides where it can: the
// quotients are off by 2^-20 at most, so that only those within 1e-5 of a border, and a scale within four steps of one between two
// bf16 values, need more.
__device__ __forceinline__ uint16_t kv4_scale(float mx, float z) {
    const float q = (mx - z) * (1.f / 15.f);
    const uint32_t low = __float_as_uint(q) & 0xffffu;
    if (low - 0x7ffcu > 8u && fabsf(q) > 1e-30f) return f32_to_bf16_bits(q);
    return f32_to_bf16_bits((float)(((double)mx - (double)z) / 15.0));
}
// A quotient near a border m + 1/2 (values of 8 bits fall on one every few hundred times): the sign of x - z - (m + 1/2) s, with the
// difference's rounding error; the product is exact, 13 bits.
__device__ __noinline__ float kv4_at_border(float x, float z, float s, float m) {
    const float d = __fsub_rn(x, z), zz = __fsub_rn(d, x), err = __fadd_rn(__fsub_rn(x, __fsub_rn(d, zz)), -__fadd_rn(z, zz));
    const float over = __fadd_rn(__fsub_rn(d, __fmul_rn(m + 0.5f, s)), err);
    return over > 0.f || (over == 0.f && ((int)m & 1)) ? m + 1.f : m;
}
__device__ __forceinline__ uint32_t kv4_codes(const float (&x)[8], float s, float z) {
    if (!(s > 0.f)) return 0u;
    uint32_t word = 0;
    if (s < 1e-30f) {                              // its reciprocal, or the quotient's steps, may leave fp32's range
#pragma unroll
        for (int i = 0; i < 8; ++i) word |= (uint32_t)fmin(fmax(rint(((double)x[i] - (double)z) / (double)s), 0.0), 15.0) << (4 * i);
        return word;
    }
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    const float big = 12582912.f;                  // 1.5 * 2^23: the sum's last bits are the rounded quotient
    uint32_t near = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = fminf(fmaxf((x[i] - z) * inv, 0.f), 15.f), n = t + big;
        if (fabsf(t - (n - big)) > 0.49999f) near |= 1u << i;
        word += __float_as_uint(n) << (4 * i);
    }
    if (near) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (near >> i & 1u) {
                const float t = fminf(fmaxf((x[i] - z) * inv, 0.f), 15.f), n = kv4_at_border(x[i], z, s, floorf(t));
                word += (uint32_t)((int)n - (int)rintf(t)) << (4 * i);
            }
    }
    return word - 0x4b400000u * 0x11111111u;       // the big ones' bits, shifted like the codes
}

struct Kv4AppendArgs {
    Kv4Where w;
    const void *k, *v;
    long long k_stride, v_stride;      // elements between rows
    unsigned char* pool;
    bool wide;                         // rows and heads begin at multiples of 16 bytes
};

// An 8 x 8 transpose of nibbles over the lanes whose numbers differ in the bits 0, 3 and 2: lane j of them (j made of these bits, in this
// order) gets the j-th nibbles of all eight.
__device__ __forceinline__ uint32_t kv4_transpose(uint32_t x) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const int bit = k == 0 ? 1 : k == 1 ? 8 : 4, shift = 4 << k;
        const uint32_t even = k == 0 ? 0x0f0f0f0fu : k == 1 ? 0x00ff00ffu : 0x0000ffffu;     // nibbles whose number has the bit k clear
        const uint32_t y = __shfl_xor_sync(0xffffffffu, x, bit);
        x = lane & bit ? (x & ~even) | ((y & ~even) >> shift) : (x & even) | ((y & even) << shift);
    }
    return x;
}

// A CTA takes a unit that gets new rows, and KV heads blockIdx.y, + gridDim.y, ...  A warp has one group of columns and eight of the unit's
// positions (2t, 2t + 1, 2t + 8, 2t + 9 for two t), four lanes to a group, 8 columns each: what the words of V are made of, so that
// nibbles change places within the warp and no barrier is needed.  V's words hold several positions: those that are not new keep theirs.
// Bound: the latency of finding the unit and its page (three dependent loads) at few rows, instructions (some 30 a value, most of them the
// 32-bit pipes') at many.  32 requests of one row (8 heads of 128, bf16): 4.7 us; 2048 rows of 32 heads: 26 us, 44 MB in and out, 1.7 TB/s
// (through shared memory and two barriers, a division in fp64 near borders: 39 us; three CTAs to an SM instead of four: 28).
constexpr int kKv4AppendThreads = 256;
template <int HD, typename T>
__global__ void __launch_bounds__(kKv4AppendThreads, 4) kv4_append_kernel(const Kv4AppendArgs a) {
    constexpr int kGroups = HD / kKv4Group, kCombos = 2 * kGroups, kWarps = kKv4AppendThreads / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int unit;
    const int req = kv4_nth_unit(a.w, blockIdx.x, unit);
    if (req < 0) return;
    int first, base;
    const int n = kv4_rows(a.w, req, first, base);
    const int lo = max(0, base - unit * kKv4Unit), hi = min(kKv4Unit, base + n - unit * kKv4Unit);     // new positions of the unit
    const int combo = warp % kCombos, group = combo / 2;
    const int piece = lane & 3, t = 2 * (combo & 1) + (lane >> 4), slot = 2 * t + (lane >> 2 & 1) + 8 * (lane >> 3 & 1);
    const bool mine = slot >= lo && slot < hi;
    const size_t row = (size_t)(first + unit * kKv4Unit + slot - base);
    unsigned char* const unit0 = kv4_unit(a.pool, a.w, req, 0, unit, HD);
    if (!unit0) return;                                    // no page there: the rows are dropped
    const size_t head_bytes = (size_t)(a.w.page_size / kKv4Unit) * kv4_unit_bytes(HD);
    constexpr int kKinds = kCombos == kWarps ? 2 : 1;      // of K and V, one warp does both or one
    const int kind0 = kKinds == 2 ? 0 : warp / kCombos;
    const size_t col = group * kKv4Group + piece * 8;
    float next[kKinds][8];
    auto fetch = [&](int head) {
#pragma unroll
        for (int i = 0; i < kKinds; ++i) {
            const int kv = kind0 + i;
            if (mine) kv4_load8(static_cast<const T*>(kv ? a.v : a.k) + row * (kv ? a.v_stride : a.k_stride) + (size_t)head * HD + col, a.wide, next[i]);
        }
    };
    fetch(blockIdx.y);
    for (int head = blockIdx.y; head < a.w.Hkv; head += gridDim.y) {
        float x[kKinds][8];
#pragma unroll
        for (int i = 0; i < kKinds; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = mine ? next[i][e] : 0.f;
        if (head + (int)gridDim.y < a.w.Hkv) fetch(head + gridDim.y);
        unsigned char* dst = unit0 + head * head_bytes;
#pragma unroll
        for (int i = 0; i < kKinds; ++i) {
            const int kv = kind0 + i;
            kv4_limit8(x[i]);
            float mn = x[i][0], mx = x[i][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) { mn = fminf(mn, x[i][e]); mx = fmaxf(mx, x[i][e]); }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            }
            const uint16_t zb = f32_to_bf16_bits(mn);
            const float z = bf16_bits_to_f32(zb);
            const uint16_t sb = kv4_scale(mx, z);
            const uint32_t word = kv4_codes(x[i], bf16_bits_to_f32(sb), z);
            if (kv == 0) {
                if (mine) {
                    *reinterpret_cast<uint32_t*>(dst + slot * (HD / 2) + (piece * kGroups + group) * 4) = word;
                    if (piece == 0) *reinterpret_cast<uint32_t*>(dst + kv4_k_scales(HD) + (slot * kGroups + group) * 4) = pack2(sb, zb);
                }
            } else {
                if (mine && piece == 0) {
                    uint16_t* sz = reinterpret_cast<uint16_t*>(dst + kv4_v_scales(HD)) + group * kKv4Unit + slot;
                    sz[0] = sb;
                    sz[HD / 2] = zb;
                }
                const uint32_t turned = kv4_transpose(word);
                const int g = (lane & 1) | (lane >> 2 & 2) | (lane & 4), tile = 2 * group + (piece >> 1);
                uint32_t fresh = 0;
#pragma unroll
                for (int nib = 0; nib < 8; ++nib) {
                    const int at = 2 * t + (nib >> 2) + 8 * (nib >> 1 & 1);
                    if (at >= lo && at < hi) fresh |= 15u << (4 * nib);
                }
                uint32_t* p = reinterpret_cast<uint32_t*>(dst + kv4_v_codes(HD)) + (tile / 4 * 32 + g * 4 + t) * 4 + tile % 4;
                if (fresh) *p = fresh == 0xffffffffu ? turned : (*p & ~fresh) | (turned & fresh);
            }
        }
    }
}

struct Kv4ReadArgs {
    Kv4Where w;
    unsigned char* pool;
    float *k, *v;              // [rows][Hkv][HD]
    int units;
};

// The values of the rows' positions; bound by its stores: 2048 rows of 32 heads 18 us, 78 MB in and out, 4.3 TB/s.  The first units * Hkv CTAs: one (unit, KV head) each, 8 columns of a row per thread.  The others look for rows
// that have no position in any unit (no page, behind the table's end, no request): zeros.
template <int HD>
__global__ void __launch_bounds__(kKv4AppendThreads) kv4_read_kernel(const Kv4ReadArgs a) {
    constexpr int kPieces = HD / 8, kGroups = HD / kKv4Group, kTasks = kKv4Unit * kPieces;
    __shared__ int s_req, s_unit;
    __shared__ __align__(16) uint32_t words[20 * HD / 4];
    const int tid = threadIdx.x, nth = blockIdx.x / a.w.Hkv, head = blockIdx.x % a.w.Hkv;
    auto put = [&](int kv, size_t row, int h, int piece, const float (&x)[8]) {
        float4* out = reinterpret_cast<float4*>((kv ? a.v : a.k) + (row * a.w.Hkv + h) * HD + piece * 8);
        out[0] = make_float4(x[0], x[1], x[2], x[3]);
        out[1] = make_float4(x[4], x[5], x[6], x[7]);
    };
    const float none[8] = {};
    if (nth >= a.units) {                          // sixteen rows, sixteen threads each
        __shared__ int has[kKv4Unit];
        const int local = tid / kKv4Unit, row = ((int)blockIdx.x - a.units * a.w.Hkv) * kKv4Unit + local;
        if (tid < kKv4Unit) has[tid] = 0;
        __syncthreads();
        for (int r = tid % kKv4Unit; r < a.w.n_req; r += kKv4Unit) {
            int first, base;
            const int n = kv4_rows(a.w, r, first, base);
            if (n > 0 && row >= first && row < first + n) has[local] = 1;
        }
        __syncthreads();
        if (row < a.w.rows && !has[local])
            for (int i = tid % kKv4Unit; i < 2 * a.w.Hkv * kPieces; i += kKv4Unit) put(i & 1, row, i / 2 / kPieces, i / 2 % kPieces, none);
        return;
    }
    if (tid < 32) {
        int unit;
        const int req = kv4_nth_unit(a.w, nth, unit);
        if (tid == 0) { s_req = req; s_unit = unit; }
    }
    __syncthreads();
    const int req = s_req, unit = s_unit;
    if (req < 0) return;
    int first, base;
    const int n = kv4_rows(a.w, req, first, base);
    const int lo = max(0, base - unit * kKv4Unit), hi = min(kKv4Unit, base + n - unit * kKv4Unit);
    const unsigned char* u = kv4_unit(a.pool, a.w, req, head, unit, HD);
    if (u)
        for (int i = tid; i < 20 * HD / 16; i += kKv4AppendThreads) reinterpret_cast<uint4*>(words)[i] = reinterpret_cast<const uint4*>(u)[i];
    __syncthreads();
    for (int task = tid; task < 2 * kTasks; task += kKv4AppendThreads) {
        const int kv = task / kTasks, slot = task % kTasks / kPieces, piece = task % kPieces, group = piece >> 2;
        if (slot < lo || slot >= hi) continue;
        const size_t row = (size_t)(first + unit * kKv4Unit + slot - base);
        float x[8];
        if (!u) {
            put(kv, row, head, piece, none);
            continue;
        }
        if (kv == 0) {
            const uint32_t word = words[slot * (HD / 8) + (piece & 3) * kGroups + group], sz = words[kv4_k_scales(HD) / 4 + slot * kGroups + group];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = fmaf((float)(word >> (4 * i) & 15u), __uint_as_float(sz << 16), __uint_as_float(sz & 0xffff0000u));
        } else {
            const uint16_t* sz = reinterpret_cast<const uint16_t*>(words) + kv4_v_scales(HD) / 2 + group * kKv4Unit + slot;
            const float s = bf16_bits_to_f32(sz[0]), z = bf16_bits_to_f32(sz[HD / 2]);
            const int tile = piece >> 1, nib = (piece & 1) + 2 * (slot >> 3) + 4 * (slot & 1), t = slot % 8 / 2;
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                const uint32_t word = words[kv4_v_codes(HD) / 4 + (tile / 4 * 32 + g * 4 + t) * 4 + tile % 4];
                x[g] = fmaf((float)(word >> (4 * nib) & 15u), s, z);
            }
        }
        put(kv, row, head, piece, x);
    }
}

}  // namespace pipesd
