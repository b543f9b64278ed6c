// C entries of the 4-bit K/V cache.
#include <algorithm>
#include <mutex>

#include "../../../include/pipesd.h"
#include "kv4.cuh"
#include "kv4_attend.cuh"

using namespace pipesd;

namespace {

bool cfg_ok(const pipesd_kv4_cfg* c) {
    return c && (c->head_dim == 64 || c->head_dim == 128) && c->n_kv_heads >= 1 && c->n_kv_heads <= 65535 && c->page_size >= kKv4Unit &&
           c->page_size % kKv4Unit == 0 && c->page_size <= 4096 && c->n_pages >= 1 && c->max_pages >= 1 &&
           (int64_t)c->max_pages * c->page_size <= (1 << 30) && c->reserved == 0;
}
bool where_ok(const pipesd_kv4_cfg* c, const void* pool, int32_t n_req, int32_t rows, const int32_t* row0, const int32_t* base, const int32_t* table) {
    return cfg_ok(c) && pool && (uintptr_t)pool % 16 == 0 && n_req >= 1 && rows >= 1 && row0 && base && table;
}
Kv4Where where_of(const pipesd_kv4_cfg* c, int n_req, int rows, const int32_t* row0, const int32_t* base, const int32_t* table) {
    return Kv4Where{row0, base, table, n_req, rows, c->n_pages, c->max_pages, c->page_size, c->n_kv_heads};
}
bool dtype_ok(int32_t dtype) { return dtype == PIPESD_F32 || dtype == PIPESD_BF16; }
bool aligned(const void* p, int32_t dtype) { return (uintptr_t)p % (dtype == PIPESD_F32 ? 4 : 2) == 0; }
bool wide(const void* p, int64_t stride, int32_t rows, int32_t dtype) {
    return (uintptr_t)p % 16 == 0 && (rows == 1 || stride * (dtype == PIPESD_F32 ? 4 : 2) % 16 == 0);
}
// n rows behind any base touch at most n / 16 + 2 units, and no more than n.
int most_units(int32_t n_req, int32_t rows) { return (int)std::min<int64_t>(rows, rows / kKv4Unit + 2ll * n_req); }
int32_t launched() { return cudaGetLastError() == cudaSuccess ? PIPESD_OK : PIPESD_E_CUDA; }

using AttendFn = void (*)(Kv4AttendArgs);
template <int HD, typename T>
AttendFn attend_fn(int nt) {
    return nt == 1 ? kv4_attend_kernel<HD, 1, T> : kv4_attend_kernel<HD, 2, T>;
}
template <int HD, typename T>
size_t attend_smem(int nt) {
    constexpr bool s = sizeof(T) == 4;
    return nt == 1 ? sizeof(AttendSmem<HD, 1, s>) : sizeof(AttendSmem<HD, 2, s>);
}

// Shared-memory limits belong to a device: set once for each, with that device current.
constexpr int kDevices = 64;
std::mutex g_mu;
bool g_ready[kDevices] = {false};
template <int HD, typename T>
bool attend_attrs() {
    for (int nt : {1, 2})
        if (cudaFuncSetAttribute((const void*)attend_fn<HD, T>(nt), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)attend_smem<HD, T>(nt)) != cudaSuccess)
            return false;
    return true;
}
bool device_ready() {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return false;
    std::lock_guard<std::mutex> lock(g_mu);
    if (!g_ready[dev]) g_ready[dev] = attend_attrs<64, float>() && attend_attrs<64, uint16_t>() && attend_attrs<128, float>() && attend_attrs<128, uint16_t>();
    return g_ready[dev];
}

// Tiles of eight query rows that a CTA takes of a KV head's: two unless that pads the rows by a fifth and more.  us with one and two (8
// requests of 2000 to 4000 positions, 32 heads of 128; bf16, fp32): 4 rows 45 58, 56 80; 9 rows 77 66, 99 87; 17 rows 110 115, 142 158; over 8 KV
// heads: 36 rows 54 53, 68 70; 68 rows 87 80, 112 107.
int attend_row_tiles(int64_t rows) { return (rows + 15) / 16 * 16 * 5 <= (rows + 7) / 8 * 8 * 6 ? 2 : 1; }
// That where there is work for the CTAs of two: `units` of the page table (what the host knows of the lengths) times the row groups that read each,
// `rows` of a KV head in the mean.  us with one and two tiles, bf16, one request, by units * groups: 9 rows of 32 heads behind 2048 positions
// (8 thousand) 25 29; behind 8192 (33) 39 39; behind 16384 (66) 57 51; 9 rows over 8 heads behind 16384 (41) 43 47; 64 rows of 32 heads behind
// 2048 (34) 39 41; 128 rows (70) 61 55; prompts of 64 rows (1) 18 25, of 512 (66) 78 68, of 2000 (1000) 620 430.  (A prompt of 128 rows (4) 25 18,
// whose triples of eight units need no merge with either.)
constexpr int64_t kAttendTwoTiles = 49152;
int attend_tiles(int64_t units, int64_t rows) { return units * ((rows + 7) / 8) < kAttendTwoTiles ? 1 : attend_row_tiles(rows); }

template <int HD, typename T>
int32_t attend_run(Kv4AttendArgs& a, int nt, cudaStream_t st) {
    attend_fn<HD, T>(nt)<<<a.ctas, 32 * attend_warps(nt), attend_smem<HD, T>(nt), st>>>(a);
    if (cudaGetLastError() != cudaSuccess) return PIPESD_E_CUDA;
    const long long jobs = (long long)a.w.rows * a.Hq;
    const bool many = jobs > kMergeWave;
    a.heads = many ? (int)std::min<long long>(a.Hq, (jobs + kMergeWave * kMergeWarps - 1) / (kMergeWave * kMergeWarps)) : 1;
    const long long blocks = (long long)a.w.rows * ((a.Hq + a.heads - 1) / a.heads);
    if (launch_pdl(many ? kv4_merge_kernel<HD, 1, T> : kv4_merge_kernel<HD, kMergeWarps, T>, dim3((unsigned)(many ? (blocks + kMergeWarps - 1) / kMergeWarps : blocks)),
                   dim3(32 * kMergeWarps), 0, st, a) != cudaSuccess)
        return PIPESD_E_CUDA;
    return launched();
}

}  // namespace

extern "C" {

uint64_t pipesd_kv4_pool_bytes(const pipesd_kv4_cfg* cfg) {
    if (!cfg_ok(cfg)) return 0;
    return (uint64_t)cfg->n_pages * cfg->n_kv_heads * (cfg->page_size / kKv4Unit) * kv4_unit_bytes(cfg->head_dim);
}

int32_t pipesd_kv4_append(const pipesd_kv4_cfg* cfg, void* pool, const void* k, const void* v, int32_t dtype, int64_t k_stride, int64_t v_stride,
                          int32_t n_req, int32_t rows, const int32_t* row0, const int32_t* base, const int32_t* table, void* cuda_stream) {
    if (!where_ok(cfg, pool, n_req, rows, row0, base, table) || !k || !v || !dtype_ok(dtype) || !aligned(k, dtype) || !aligned(v, dtype)) return PIPESD_E_INVALID;
    const int64_t width = (int64_t)cfg->n_kv_heads * cfg->head_dim;
    if (rows > 1 && (k_stride < width || v_stride < width)) return PIPESD_E_INVALID;
    const Kv4AppendArgs a = {where_of(cfg, n_req, rows, row0, base, table), k, v, k_stride, v_stride, static_cast<unsigned char*>(pool),
                             wide(k, k_stride, rows, dtype) && wide(v, v_stride, rows, dtype)};
    // CTAs for one wave and a half (four to an SM), beyond which a CTA takes several heads of its unit.  us with one wave, one and a half, and two:
    // 2048 rows of 32 heads of 128 in bf16 27.1, 25.9, 24.4; 5 requests of 100 to 700 rows of 8 heads of 64 in fp32 7.4, 7.2, 7.9; of 32 heads of
    // 128 in bf16 (by graph, cold) 1000 rows 22.5, 22.5, 20.5, 4096 57, 59, 53, 8192 107, 107, 94; of 8 heads of 64 2048 rows 10, 12, 12,
    // 4096 14, 16, 14.  Two waves gain a tenth at the largest and lose as much at the smaller ones.
    const int units = most_units(n_req, rows);
    const dim3 grid((unsigned)units, (unsigned)std::min(cfg->n_kv_heads, std::max(1, 6 * 148 / units)));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (cfg->head_dim == 128) {
        if (dtype == PIPESD_F32) kv4_append_kernel<128, float><<<grid, kKv4AppendThreads, 0, st>>>(a);
        else kv4_append_kernel<128, uint16_t><<<grid, kKv4AppendThreads, 0, st>>>(a);
    } else {
        if (dtype == PIPESD_F32) kv4_append_kernel<64, float><<<grid, kKv4AppendThreads, 0, st>>>(a);
        else kv4_append_kernel<64, uint16_t><<<grid, kKv4AppendThreads, 0, st>>>(a);
    }
    return launched();
}

int32_t pipesd_kv4_read(const pipesd_kv4_cfg* cfg, const void* pool, float* k, float* v, int32_t n_req, int32_t rows, const int32_t* row0,
                        const int32_t* base, const int32_t* table, void* cuda_stream) {
    if (!where_ok(cfg, pool, n_req, rows, row0, base, table) || !k || !v || (uintptr_t)k % 16 || (uintptr_t)v % 16) return PIPESD_E_INVALID;
    const Kv4ReadArgs a = {where_of(cfg, n_req, rows, row0, base, table), static_cast<unsigned char*>(const_cast<void*>(pool)), k, v,
                           most_units(n_req, rows)};
    const int64_t ctas = (int64_t)a.units * cfg->n_kv_heads + (rows + kKv4Unit - 1) / kKv4Unit;
    if (ctas > INT32_MAX) return PIPESD_E_INVALID;
    const dim3 grid((unsigned)ctas);
    if (cfg->head_dim == 128) kv4_read_kernel<128><<<grid, kKv4AppendThreads, 0, (cudaStream_t)cuda_stream>>>(a);
    else kv4_read_kernel<64><<<grid, kKv4AppendThreads, 0, (cudaStream_t)cuda_stream>>>(a);
    return launched();
}

uint64_t pipesd_kv4_attend_scratch_bytes(const pipesd_kv4_cfg* cfg) {
    if (!cfg_ok(cfg)) return 0;
    // two shares per CTA, each of 8 rows per tile
    return (uint64_t)2 * kAttendSms * std::max(8 * attend_ctas_per_sm(1), 16 * attend_ctas_per_sm(2)) * (cfg->head_dim + 2) * 4;
}

int32_t pipesd_kv4_attend(const pipesd_kv4_cfg* cfg, const void* pool, const void* q, void* out, int32_t dtype, int64_t q_stride, int64_t out_stride,
                          int32_t n_q_heads, float scale, int32_t n_req, int32_t rows, const int32_t* row0, const int32_t* base, const int32_t* table,
                          void* scratch, void* cuda_stream) {
    if (!where_ok(cfg, pool, n_req, rows, row0, base, table) || !q || !out || !scratch || (uintptr_t)scratch % 16 || !dtype_ok(dtype) || !aligned(q, dtype) ||
        !aligned(out, dtype) || n_q_heads < 1 || n_q_heads % cfg->n_kv_heads || !(scale > 0.f && scale < INFINITY))
        return PIPESD_E_INVALID;
    const int64_t width = (int64_t)n_q_heads * cfg->head_dim;
    if (rows > 1 && (q_stride < width || out_stride < width)) return PIPESD_E_INVALID;
    if ((int64_t)rows * n_q_heads > INT32_MAX) return PIPESD_E_INVALID;
    if (!device_ready()) return PIPESD_E_CUDA;
    Kv4AttendArgs a = {};
    a.w = where_of(cfg, n_req, rows, row0, base, table);
    a.pool = static_cast<unsigned char*>(const_cast<void*>(pool));
    a.q = q;
    a.out = out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.Hq = n_q_heads;
    a.scale = scale * 1.4426950408889634f;
    a.parts = static_cast<float*>(scratch);
    const int nt = attend_tiles((int64_t)n_req * cfg->max_pages * (cfg->page_size / kKv4Unit) * cfg->n_kv_heads,
                                (int64_t)(rows + n_req - 1) / n_req * (n_q_heads / cfg->n_kv_heads));
    a.rows_cap = 8 * nt;
    a.ctas = kAttendSms * attend_ctas_per_sm(nt);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (cfg->head_dim == 128) return dtype == PIPESD_F32 ? attend_run<128, float>(a, nt, st) : attend_run<128, uint16_t>(a, nt, st);
    return dtype == PIPESD_F32 ? attend_run<64, float>(a, nt, st) : attend_run<64, uint16_t>(a, nt, st);
}

}  // extern "C"
