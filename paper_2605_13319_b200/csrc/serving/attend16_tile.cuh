// What the bf16 attention kernels (prompts; pages, together and apart) do with a tile of 128 query rows by kKeys keys on the 5th-generation tensor cores.
//
//   S[128 x kKeys] = Q K^T        both operands in shared memory, fp32 scores in tensor memory, a lane per query row
//   P = exp2(scale S - ref)       one thread per row: its scores in registers, no exchange between threads.  ref is the row's running
//                                 maximum as of the last time it rose by more than 2^8 in weight: O and the sum are rescaled only then, so that
//                                 P <= 2^8, and hardly ever behind a row's first tile
//   O[128 x HD] += P V            P as bf16 in tensor memory (over the scores it was made of), V in shared memory, fp32 sums in tensor memory
//
// P is rounded to bf16 because a product's operands are of one type and V is bf16: half a step, at most 2^-8 of a weight; their sum is of the unrounded ones,
// in fp32.  Against 64 bits the outputs' error, 1.6e-3 by their own rounding, becomes 2.2e-3 (of the norm).  A second term of P, as fp32 queries take three,
// would double these products, half of what bounds a long prompt.
//
// Two such streams per CTA, each with four warps of its own and a thread that issues its products: while one stream's exponentials are taken the tensor
// cores do the other's products.  P goes over in halves, so that the first half's products run beside the second's exponentials.
//
// What bounds it, for two streams of 128 rows by 128 keys with heads of 128: the products 2048 clocks (S = Q K^T of 64 clocks a k16 step, P V the same), the
// exponentials 2048 clocks too (the special-function units take 16 a clock), 3500 measured in a long prompt: the hand-over from one to the other, some
// 1000 clocks a tile and stream, is covered by the other stream only in part.  A tile of one stream with few rows, so with one warp at work, takes that warp
// 2000 to 2700 clocks, 3300 with the other stream's on the same scheduler.  Steps of 64 keys with two places for the scores: a prompt of 16384 2133 us
// instead of 1984; two threads a row: 2222; a quarter of the exponentials as polynomials on the FMA pipe: 1830 instead of 1728 (short runs).
#pragma once
#include "../tcgen05.cuh"

namespace pipesd {

// ---- instructions that tcgen05.cuh does not have
// Shared-memory operand descriptor of tiles in the copy engine's 128-byte swizzle: rows of 128 bytes in groups of eight (1024 bytes), 16-byte pieces
// exchanged by the row's number in its group.  K-major: sbo = bytes between groups of eight rows (lbo is not used).  MN-major: a row holds
// 64 neighbouring columns of one k; lbo = bytes between blocks of 64 columns, sbo = between groups of eight k.
__device__ __forceinline__ uint64_t umma_desc_swizzled(uint32_t saddr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
    return umma_desc(saddr, lbo_bytes, sbo_bytes) | (2ull << 61);
}
// D[tmem] (+)= A[tmem] . B[smem], one k16 step (A: 8 columns of bf16 pairs); issued by ONE thread.
__device__ __forceinline__ void umma_bf16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
        "}\n"
        :
        : "r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
#define PIPESD_R8(u, i) "=r"(u[i]), "=r"(u[i + 1]), "=r"(u[i + 2]), "=r"(u[i + 3]), "=r"(u[i + 4]), "=r"(u[i + 5]), "=r"(u[i + 6]), "=r"(u[i + 7])
#define PIPESD_IN8(u, i) "r"(u[i]), "r"(u[i + 1]), "r"(u[i + 2]), "r"(u[i + 3]), "r"(u[i + 4]), "r"(u[i + 5]), "r"(u[i + 6]), "r"(u[i + 7])
#define PIPESD_RW8(u, i) "+r"(u[i]), "+r"(u[i + 1]), "+r"(u[i + 2]), "+r"(u[i + 3]), "+r"(u[i + 4]), "+r"(u[i + 5]), "+r"(u[i + 6]), "+r"(u[i + 7])
// 32 consecutive columns of this thread's lane, as bits; whole warp, same address.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* u) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
        "%23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : PIPESD_R8(u, 0), PIPESD_R8(u, 8), PIPESD_R8(u, 16), PIPESD_R8(u, 24)
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* u) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
        "%23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        PIPESD_IN8(u, 0), PIPESD_IN8(u, 8), PIPESD_IN8(u, 16), PIPESD_IN8(u, 24)
        : "memory");
}
// Waits for the loads before it; u names registers of theirs, so that no use of these moves ahead of the wait.
__device__ __forceinline__ void tmem_ld_wait32(uint32_t* u) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : PIPESD_RW8(u, 0), PIPESD_RW8(u, 8), PIPESD_RW8(u, 16), PIPESD_RW8(u, 24)::"memory");
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {      // the first in the low half
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Two fp32 values in one register pair, and what is done with both at once.
__device__ __forceinline__ uint64_t pair_of(uint32_t x, uint32_t y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(x), "r"(y));
    return r;
}
__device__ __forceinline__ uint64_t pair_of(float x, float y) { return pair_of(__float_as_uint(x), __float_as_uint(y)); }
__device__ __forceinline__ void pair_split(uint64_t v, float& x, float& y) {
    uint32_t a, b;
    asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(v));
    x = __uint_as_float(a);
    y = __uint_as_float(b);
}
__device__ __forceinline__ uint64_t pair_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t pair_add(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// ---- waits: bounded, and given up at once when another role of the CTA has given up
__device__ __forceinline__ bool role_wait(uint32_t bar, uint32_t parity, volatile int* dead) {
    uint64_t t0 = 0;
    for (uint32_t it = 0;; ++it) {
        uint32_t ok;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok)
                     : "r"(bar), "r"(parity)
                     : "memory");
        if (ok) return true;
        if ((it & 255u) == 255u) {
            if (*dead) return false;
            const uint64_t now = global_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > 2000000000ull) {
                *dead = 1;
                return false;
            }
        }
    }
}

// The same for a whole warp, which goes on together.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* dead) { return __all_sync(0xffffffffu, role_wait(bar, parity, dead)); }

// Warps 0-3 and 4-7: the streams'; 8-11 fetch and issue.  Twelve warps are launched with 168 registers each; the last four hand over to the others
// (8 x 208 + 4 x 88 = 12 x 168).
constexpr int kAttendThreads16 = 384, kLaunchRegisters = 168;
__device__ __forceinline__ void registers_more() { asm volatile("setmaxnreg.inc.sync.aligned.u32 208;"); }
__device__ __forceinline__ void registers_fewer() { asm volatile("setmaxnreg.dec.sync.aligned.u32 88;"); }

// Slot and phase of the at-th entry of a ring of n slots.
template <int n>
struct RingPlace {
    uint32_t slot, phase;
    __device__ __forceinline__ explicit RingPlace(uint32_t at) : slot(at % n), phase(at / n & 1u) {}
};

constexpr float kRefExcess = 8.f;                  // log2 units by which a weight may exceed 1

// Adds a tile's sums to a row's.
template <int HD>
__device__ __forceinline__ void own_sums(uint32_t o_tmem, float (&own)[HD]) {
#pragma unroll
    for (int c = 0; c < HD; c += 16) {
        float o[16];
        tmem_ld16(o_tmem + c, o);
        tmem_ld_wait16(o);
#pragma unroll
        for (int i = 0; i < 16; ++i) own[c + i] += o[i];
    }
}

// One row's share of a tile, whose scores have come (and the products of the tile before are done).  `first`: there are no sums yet.  masked: bit c of
// `see` says whether key c is seen; the others' scores are replaced, whatever they are.  given(h): half h of the weights is where the products read it.
// kOwn: the products of a tile are sums of their own, which the thread adds to `own`: the tensor cores' additions truncate, which in bf16 does not
// count, but would cost fp32 two bits over a long row.
template <int HD, int kKeys, int kTerms, bool kOwn, typename Given>
__device__ __forceinline__ void softmax_tile(uint32_t s_tmem, uint32_t o_tmem, float scale, bool first, bool masked, const uint32_t (&see)[kKeys / 32], float& ref,
                                             float& sum, float (&own)[kOwn ? HD : 1], Given given) {
    constexpr int kHalf = kTerms == 1 ? kKeys / 2 : kKeys;
    uint32_t s[kKeys];
#pragma unroll
    for (int i = 0; i < kKeys; i += 32) tmem_ld32(s_tmem + i, s + i);
    if constexpr (kOwn)
        if (!first) own_sums<HD>(o_tmem, own);
#pragma unroll
    for (int i = 0; i < kKeys; i += 32) tmem_ld_wait32(s + i);
    if (masked) {
#pragma unroll
        for (int i = 0; i < kKeys; ++i)
            if (!(see[i / 32] >> (i % 32) & 1u)) s[i] = 0xff800000u;
    }
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < kKeys; i += 2) mx[(i >> 1) & 3] = max3(mx[(i >> 1) & 3], __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
    const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * scale;
    const bool up = top > ref + kRefExcess || (ref == -INFINITY && top > ref);
    if (__any_sync(0xffffffffu, up)) {
        const float next = up ? top : ref, factor = up ? exp2_approx(ref - next) : 1.f;
        ref = next;
        sum *= factor;
        if constexpr (kOwn) {
#pragma unroll
            for (int i = 0; i < HD; ++i) own[i] *= factor;
        } else if (!first) {
#pragma unroll 1
            for (int c = 0; c < HD; c += 16) {
                float o[16];
                tmem_ld16(o_tmem + c, o);
                tmem_ld_wait16(o);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] *= factor;
                tmem_st16(o_tmem + c, o);
            }
        }
    }
    const float shift = ref == -INFINITY ? 0.f : -ref;
    const uint64_t scale2 = pair_of(scale, scale), shift2 = pair_of(shift, shift);
    uint64_t part[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < kKeys / kHalf; ++h) {
        uint32_t* const x = s + h * kHalf;
#pragma unroll
        for (int i = 0; i < kHalf; i += 2) {
            const uint64_t p = pair_fma(pair_of(x[i], x[i + 1]), scale2, shift2);
            float a, b;
            pair_split(p, a, b);
            a = exp2_approx(a);
            b = exp2_approx(b);
            part[(i >> 1) & 1] = pair_add(part[(i >> 1) & 1], pair_of(a, b));
            x[i] = __float_as_uint(a);
            x[i + 1] = __float_as_uint(b);
        }
#pragma unroll
        for (int t = 0; t < kTerms; ++t) {
            uint32_t p[kHalf / 2];
#pragma unroll
            for (int i = 0; i < kHalf / 2; ++i) {
                const float a = __uint_as_float(x[2 * i]), b = __uint_as_float(x[2 * i + 1]);
                p[i] = pack_bf16(a, b);
                if (t + 1 < kTerms) {              // what the term leaves, exactly
                    x[2 * i] = __float_as_uint(a - __uint_as_float(p[i] << 16));
                    x[2 * i + 1] = __float_as_uint(b - __uint_as_float(p[i] & 0xffff0000u));
                }
            }
            tmem_st32(s_tmem + t * (kKeys / 2) + h * (kHalf / 2), p);
        }
        tmem_st_wait();
        given(h);
    }
    float even, odd;
    pair_split(pair_add(part[0], part[1]), even, odd);
    sum += even + odd;
}

// Values of a tile that no row may take into its products: pieces that are no key's, and what is not finite where not every row sees it.  A weight of 0
// does not keep them out, so they become 0 in shared memory.  Done by the 128 threads of a stream; kPieces pieces of 16 bytes.  kind(piece): what the
// piece's key is.  found(): something is not finite, said before it goes, so that who reads the 0 instead finds it said.
enum { kSeenByAll, kSeenBySome, kNoKey };
template <int kPieces, typename Kind, typename Found>
__device__ __forceinline__ void clean_values(unsigned char* tile, int tid, Kind kind, Found found) {
    constexpr int kBatch = 4;                      // loads at once
    static_assert(kPieces % (128 * kBatch) == 0, "");
#pragma unroll 1
    for (int i = tid; i < kPieces; i += 128 * kBatch) {
        uint4* const at = reinterpret_cast<uint4*>(tile) + i;
        uint4 x[kBatch];
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
            const int k = kind(i + 128 * y);
            x[y] = make_uint4(0, 0, 0, 0);
            if (k == kSeenBySome) x[y] = at[128 * y];
            if (k == kNoKey) at[128 * y] = x[y];
        }
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
            uint32_t w[4] = {x[y].x, x[y].y, x[y].z, x[y].w}, bad = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) bad |= ((w[j] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
            if (bad) {
                found();
                __threadfence_block();
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t b = ((w[j] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                    if (b & 0x8000u) w[j] &= 0xffff0000u;
                    if (b & 0x80000000u) w[j] &= 0x0000ffffu;
                }
                at[128 * y] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
    fence_proxy_async_smem();
    __syncwarp();
}
// Four lanes have four pieces each, of a row each: afterwards piece `lane & 3` of each of the four rows.
__device__ __forceinline__ void exchange_pieces(uint4 (&x)[4]) {
    auto swap = [](uint4& a, uint4& b, bool odd, int lanes) {                  // a stays where odd is false, b where it is true; the other goes
        uint4 go = odd ? a : b;
        go.x = __shfl_xor_sync(0xffffffffu, go.x, lanes);
        go.y = __shfl_xor_sync(0xffffffffu, go.y, lanes);
        go.z = __shfl_xor_sync(0xffffffffu, go.z, lanes);
        go.w = __shfl_xor_sync(0xffffffffu, go.w, lanes);
        if (odd) a = go;
        else b = go;
    };
    const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
    swap(x[0], x[1], odd, 1);
    swap(x[2], x[3], odd, 1);
    swap(x[0], x[2], high, 2);
    swap(x[1], x[3], high, 2);
}
// Bits of the 16 columns behind p whose value is not finite.
__device__ __forceinline__ uint32_t not_finite16(const uint16_t* p, int piece_stride) {
    uint32_t bits = 0;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const uint4 x = *reinterpret_cast<const uint4*>(p + c * piece_stride);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if ((w[j] & 0x7f80u) == 0x7f80u) bits |= 1u << (8 * c + 2 * j);
            if ((w[j] & 0x7f800000u) == 0x7f800000u) bits |= 2u << (8 * c + 2 * j);
        }
    }
    return bits;
}

}  // namespace pipesd
