// Attention in bf16: whole prompts packed one behind the other, and new rows (a tree of drafts, a chain, a token) over the pages of kv16.cuh.
#pragma once
#include "kv16.cuh"

namespace pipesd {

struct Attend16Args {
    Kv4Where w;                 // prompts: row0, n_req, rows, Hkv
    Kv16Pool p;                 // pages
    const uint16_t *k, *v;      // prompts: packed rows
    long long k_stride, v_stride;
    const void* q;
    void* out;
    long long q_stride, out_stride;
    int Hq;
    float scale;                // times log2(e)
    const uint32_t* mask;       // [rows][words], null: a row sees the new rows up to itself
    int words;
};

__device__ __forceinline__ float attend16_in(float v) { return v; }
__device__ __forceinline__ float attend16_in(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ void attend16_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void attend16_store(uint16_t* p, float v) { *p = f32_to_bf16_bits(v); }

// A warp per (row, query head).
template <int HD, typename T, bool kPaged>
__global__ void __launch_bounds__(128) attend16_simple_kernel(const Attend16Args a) {
    constexpr int kE = HD / 32;
    const int lane = threadIdx.x & 31;
    const long long job = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int row = (int)(job / a.Hq), qh = (int)(job % a.Hq), head = qh / (a.Hq / a.w.Hkv);
    if (row >= a.w.rows) return;
    int first = 0, base = 0, r = -1, n = 0;
    if (kPaged) {
        r = kv16_request_of(a.w, row, first, base);
    } else {
        for (int i = 0; i < a.w.n_req && r < 0; ++i)
            if (a.w.row0[i] >= 0 && a.w.row0[i] <= row && row < a.w.row0[i + 1] && a.w.row0[i + 1] <= a.w.rows) { r = i; first = a.w.row0[i]; }
    }
    T* const out = static_cast<T*>(a.out) + row * a.out_stride + qh * HD + lane * kE;
    if (r < 0) {                                   // a request's row that has no position sees nothing
        for (int i = 0; kPaged && i < a.w.n_req && r < 0; ++i)
            if (a.w.row0[i] <= row && row < a.w.row0[i + 1]) r = i;
        for (int e = 0; r >= 0 && e < kE; ++e) attend16_store(out + e, 0.f);
        return;
    }
    n = row - first;
    float q[kE], o[kE] = {}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < kE; ++e) q[e] = attend16_in((static_cast<const T*>(a.q) + row * a.q_stride + qh * HD + lane * kE)[e]) * a.scale;
    const int total = kPaged ? base + (a.mask ? min(a.w.row0[r + 1] - first, 32 * a.words) : n + 1) : n + 1;
    for (int pos = 0; pos < total; ++pos) {
        const uint16_t *k, *v;
        if (kPaged) {
            const int j = pos - base;
            if (j >= 0 && a.mask && !(a.mask[(size_t)row * a.words + j / 32] >> (j & 31) & 1)) continue;
            if (pos / a.w.page_size >= a.w.max_pages) break;
            const int page = kv16_page(a.w, r, pos), slot = pos % a.w.page_size;
            if (page < 0) continue;
            const uint32_t at = kv16_piece(slot, lane * kE / 8, HD) + lane * kE % 8;
            k = kv16_block(a.p, a.w, a.p.layer, page, 0, head) + at;
            v = kv16_block(a.p, a.w, a.p.layer, page, 1, head) + at;
        } else {
            k = a.k + (first + pos) * a.k_stride + head * HD + lane * kE;
            v = a.v + (first + pos) * a.v_stride + head * HD + lane * kE;
        }
        float s = 0.f;
        for (int e = 0; e < kE; ++e) s = fmaf(q[e], bf16_bits_to_f32(k[e]), s);
        s = warp_sum(s);
        const float mn = fmaxf(m, s), f = exp2f(m - mn), p = exp2f(s - mn);
        m = mn;
        l = l * f + p;
        for (int e = 0; e < kE; ++e) o[e] = fmaf(p, bf16_bits_to_f32(v[e]), o[e] * f);
    }
    for (int e = 0; e < kE; ++e) attend16_store(out + e, l > 0.f ? o[e] / l : (l == 0.f ? 0.f : l));
}

}  // namespace pipesd
