// C entries of the bf16 K/V cache, its pages, and attention in bf16.
#include <algorithm>
#include <atomic>
#include <mutex>

#include "../../../include/pipesd.h"
#include "attend16_apart.cuh"
#include "attend16_pages.cuh"
#include "attend16_prompt.cuh"
#include "kv16_pages.cuh"

using namespace pipesd;

namespace {

std::atomic<int32_t> g_gives_up{-1};               // pipesd_debug_attend_gives_up

bool cfg_ok(const pipesd_kv16_cfg* c) {
    return c && (c->head_dim == 64 || c->head_dim == 128) && c->n_kv_heads >= 1 && c->n_kv_heads <= 65535 && c->page_size >= 8 && c->page_size % 8 == 0 &&
           c->page_size <= 4096 && c->n_pages >= 1 && (int64_t)c->n_pages * c->page_size <= INT32_MAX && c->max_pages >= 1 &&
           (int64_t)c->max_pages * c->page_size <= (1 << 30) && c->n_layers >= 1 && c->n_layers <= 65535 && c->reserved == 0 &&
           (double)c->n_layers * c->n_pages * c->page_size * c->n_kv_heads * c->head_dim < 0x1p60;
}
bool pool_ok(const pipesd_kv16_cfg* c, const void* pool) { return cfg_ok(c) && pool && (uintptr_t)pool % 16 == 0; }
bool where_ok(const pipesd_kv16_cfg* c, const void* pool, int32_t layer, int32_t n_req, int32_t rows, const int32_t* row0, const int32_t* base,
              const int32_t* table) {
    return pool_ok(c, pool) && layer >= 0 && layer < c->n_layers && n_req >= 1 && rows >= 1 && row0 && base && table;
}
Kv4Where where_of(const pipesd_kv16_cfg* c, int n_req, int rows, const int32_t* row0, const int32_t* base, const int32_t* table) {
    return Kv4Where{row0, base, table, n_req, rows, c->n_pages, c->max_pages, c->page_size, c->n_kv_heads};
}
Kv16Pool pool_of(const pipesd_kv16_cfg* c, const void* pool, int layer) {
    return Kv16Pool{static_cast<uint16_t*>(const_cast<void*>(pool)), c->n_layers, layer, c->head_dim};
}
int size_of(int32_t dtype) { return dtype == PIPESD_F32 ? 4 : 2; }
bool dtype_ok(int32_t dtype) { return dtype == PIPESD_F32 || dtype == PIPESD_BF16; }
bool aligned(const void* p, int32_t dtype) { return (uintptr_t)p % size_of(dtype) == 0; }
bool wide(const void* p, int64_t stride, int32_t rows, int32_t dtype) { return (uintptr_t)p % 16 == 0 && (rows == 1 || stride * size_of(dtype) % 16 == 0); }
// The kernels take it times log2(e).
bool scale_ok(float scale) { return scale > 0.f && scale * 1.4426950408889634f < INFINITY; }
int32_t launched() { return cudaGetLastError() == cudaSuccess ? PIPESD_OK : PIPESD_E_CUDA; }

// Query rows that a share (of a stream) has room for.
int pages_cap(const pipesd_kv16_cfg* c, int32_t rows, int32_t n_q_heads) {
    return (int)std::min<int64_t>(128, ((int64_t)rows * (n_q_heads / c->n_kv_heads) + 3) / 4 * 4);
}
template <int HD, typename T>
int32_t pages_run(PagesArgs& a, cudaStream_t st) {
    constexpr int keys = PagesShape<HD, T>::kKeys, rows = PagesShape<HD, T>::kRows;
    a.log_keys = keys == 128 ? 7 : 6;
    a.log_rows = rows == 256 ? 8 : 7;
    a.ranges = kPagesSms;
    a.lead = kPagesLead;
    a.own_shares = 4;
    a.gives_up = g_gives_up.load(std::memory_order_relaxed);
    a.tile_pages = keys / a.w.page_size;
    a.tile_over = keys % a.w.page_size;
    // ceil(2^(30 + L) / page_size) with 2^L >= page_size is off by less than page_size <= 2^L, so that the quotient of a position below 2^30 is exact
    int log = 0;
    while ((1 << log) < a.w.page_size) ++log;
    a.page_shift = 30 + log;
    a.page_mul = (uint32_t)(((1ull << a.page_shift) + a.w.page_size - 1) / a.w.page_size);
    bool apart = false;
    if constexpr (keys == 128) {
        // Streams with triples of their own where requests have up to 64 query rows by KV head on average.  Together and apart, us, 8 KV heads of 128:
        // 4 rows, 256 requests behind 512 positions 203 and 128, 8 behind 16384 95 and 91; 32 rows, 8 behind 4096 39.5 and 36.5; 64 rows, 4 behind
        // 8192 41 and 41.5, one behind 2048 (32 KV heads) 25 and 23; 128 rows, 16 behind 2048 58 and 62.
        apart = (int64_t)a.w.rows * a.G <= 64 * (int64_t)a.w.n_req;
        if (apart) {
            a.log_rows = 7;
            a.ranges = 2 * kPagesSms;
            a.lead = kApartLead;
            a.own_shares = 2;
            pages_apart_kernel<HD><<<kPagesSms, kAttendThreads16, apart_smem<HD>(), st>>>(a);
        }
    }
    if (!apart) pages_attend_kernel<HD, T><<<kPagesSms, kAttendThreads16, pages_smem<HD, T>(), st>>>(a);
    if (cudaGetLastError() != cudaSuccess) return PIPESD_E_CUDA;
    if (launch_pdl(pages_merge_kernel<HD, T>, dim3(a.ranges, HD / 32, std::min<int64_t>(4, ((int64_t)a.w.rows * a.G + 31) / 32)), dim3(32 * kPagesMergeWarps), 0, st, a) != cudaSuccess) return PIPESD_E_CUDA;
    return launched();
}

constexpr int32_t kPlanRequests = 1 << 30;         // (indices that step by a CTA's threads are 32-bit)
int plan_cap(const pipesd_kv16_cfg* c, int32_t n) { return (int)std::min<int64_t>((int64_t)n * c->max_pages, c->n_pages); }

// [rows, heads, head_dim] with `stride` elements between rows, fetched in boxes of 64 columns x box_heads x box_rows; rows behind the last read as 0.
bool rows_map(CUtensorMap* m, const void* base, int hd, int heads, int64_t rows, int64_t stride, int box_heads, int box_rows) {
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
        return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? (Encode)fn : (Encode) nullptr;
    }();
    if (!encode) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)hd, (cuuint64_t)heads, (cuuint64_t)rows}, strides[2] = {(cuuint64_t)hd * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows}, ones[3] = {1, 1, 1};
    return encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Shared-memory limits belong to a device: set once for each, with that device current.
constexpr int kDevices = 64, kSms = 148;
std::mutex g_mu;
bool g_ready[kDevices] = {false};
// The kernels' warps exchange registers: what they take together must be what they are launched with.
bool attend_ready(const void* kernel, int smem) {
    cudaFuncAttributes at;
    return cudaFuncGetAttributes(&at, kernel) == cudaSuccess && at.numRegs == kLaunchRegisters &&
           cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess;
}
static_assert(apart_smem<64>() <= 232448 && apart_smem<128>() <= 232448 && PromptShape<128>::kSmem <= 232448 && PromptShape<64>::kSmem <= 232448, "a CTA's shared memory");
template <int HD, typename T>
bool pages_ready() {
    static_assert(pages_smem<HD, T>() <= 232448, "a CTA's shared memory");
    return attend_ready((const void*)pages_attend_kernel<HD, T>, pages_smem<HD, T>());
}
bool device_ready() {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return false;
    std::lock_guard<std::mutex> lock(g_mu);
    if (!g_ready[dev])
        g_ready[dev] = attend_ready((const void*)prompt_kernel<64>, PromptShape<64>::kSmem) && attend_ready((const void*)prompt_kernel<128>, PromptShape<128>::kSmem) &&
                       pages_ready<64, float>() && pages_ready<64, uint16_t>() && pages_ready<128, float>() && pages_ready<128, uint16_t>() &&
                       attend_ready((const void*)pages_apart_kernel<64>, apart_smem<64>()) && attend_ready((const void*)pages_apart_kernel<128>, apart_smem<128>());
    return g_ready[dev];
}

}  // namespace

extern "C" {

int32_t pipesd_debug_attend_gives_up(int32_t cta) {
    if (cta < -1 || cta >= kSms) return PIPESD_E_INVALID;
    g_gives_up.store(cta, std::memory_order_relaxed);
    return PIPESD_OK;
}

uint64_t pipesd_kv16_pool_bytes(const pipesd_kv16_cfg* cfg) {
    if (!cfg_ok(cfg)) return 0;
    return (uint64_t)cfg->n_layers * cfg->n_pages * 2 * cfg->n_kv_heads * cfg->page_size * cfg->head_dim * 2;
}

int32_t pipesd_kv16_append(const pipesd_kv16_cfg* cfg, void* pool, int32_t layer, const void* k, const void* v, int32_t dtype, int64_t k_stride,
                           int64_t v_stride, int32_t n_req, int32_t rows, const int32_t* row0, const int32_t* base, const int32_t* table,
                           void* cuda_stream) {
    if (!where_ok(cfg, pool, layer, n_req, rows, row0, base, table) || !k || !v || !dtype_ok(dtype) || !aligned(k, dtype) || !aligned(v, dtype))
        return PIPESD_E_INVALID;
    const int64_t width = (int64_t)cfg->n_kv_heads * cfg->head_dim;
    if (rows > 1 && (k_stride < width || v_stride < width)) return PIPESD_E_INVALID;
    const Kv16RowsArgs a = {where_of(cfg, n_req, rows, row0, base, table), pool_of(cfg, pool, layer), k, v, k_stride, v_stride,
                            wide(k, k_stride, rows, dtype) && wide(v, v_stride, rows, dtype)};
    const dim3 grid((unsigned)((rows + kKv16RowWarps - 1) / kKv16RowWarps), (unsigned)cfg->n_kv_heads);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (cfg->head_dim == 128) {
        if (dtype == PIPESD_F32) kv16_append_kernel<128, float><<<grid, 32 * kKv16RowWarps, 0, st>>>(a);
        else kv16_append_kernel<128, uint16_t><<<grid, 32 * kKv16RowWarps, 0, st>>>(a);
    } else {
        if (dtype == PIPESD_F32) kv16_append_kernel<64, float><<<grid, 32 * kKv16RowWarps, 0, st>>>(a);
        else kv16_append_kernel<64, uint16_t><<<grid, 32 * kKv16RowWarps, 0, st>>>(a);
    }
    return launched();
}

int32_t pipesd_kv16_read(const pipesd_kv16_cfg* cfg, const void* pool, int32_t layer, void* k, void* v, int32_t n_req, int32_t rows, const int32_t* row0,
                         const int32_t* base, const int32_t* table, void* cuda_stream) {
    if (!where_ok(cfg, pool, layer, n_req, rows, row0, base, table) || !k || !v || (uintptr_t)k % 16 || (uintptr_t)v % 16) return PIPESD_E_INVALID;
    const Kv16RowsArgs a = {where_of(cfg, n_req, rows, row0, base, table), pool_of(cfg, pool, layer), k, v, 0, 0, 1};
    const dim3 grid((unsigned)((rows + kKv16RowWarps - 1) / kKv16RowWarps), (unsigned)cfg->n_kv_heads);
    if (cfg->head_dim == 128) kv16_read_kernel<128><<<grid, 32 * kKv16RowWarps, 0, (cudaStream_t)cuda_stream>>>(a);
    else kv16_read_kernel<64><<<grid, 32 * kKv16RowWarps, 0, (cudaStream_t)cuda_stream>>>(a);
    return launched();
}

int32_t pipesd_tree_mask(int32_t n_req, int32_t rows, const int32_t* row0, const int32_t* parent, int32_t words, uint32_t* mask, int32_t* depth,
                         void* cuda_stream) {
    if (n_req < 1 || rows < 1 || !row0 || !parent || !mask || !depth || words < 1 || words > kTreeWords) return PIPESD_E_INVALID;
    tree_mask_kernel<<<n_req + 1u, 256, 0, (cudaStream_t)cuda_stream>>>(row0, parent, n_req, rows, words, mask, depth);
    return launched();
}

int32_t pipesd_kv16_compact(const pipesd_kv16_cfg* cfg, void* pool, int32_t n_req, const uint32_t* keep, int32_t words, const int32_t* base,
                            const int32_t* table, int32_t* kept, void* cuda_stream) {
    if (!pool_ok(cfg, pool) || n_req < 1 || !keep || words < 1 || words > (1 << 25) || !base || !table || !kept) return PIPESD_E_INVALID;
    const Kv16CompactArgs a = {where_of(cfg, n_req, 0, nullptr, base, table), pool_of(cfg, pool, 0), keep, words, kept};
    const int64_t blocks = (int64_t)cfg->n_layers * 2 * cfg->n_kv_heads;
    if (blocks > INT32_MAX) return PIPESD_E_INVALID;
    const dim3 grid((unsigned)n_req, (unsigned)std::min<int64_t>((blocks + 7) / 8, 65535));
    if (cfg->head_dim == 128) kv16_compact_kernel<128><<<grid, 256, 0, (cudaStream_t)cuda_stream>>>(a);
    else kv16_compact_kernel<64><<<grid, 256, 0, (cudaStream_t)cuda_stream>>>(a);
    return launched();
}

uint64_t pipesd_kv16_plan_scratch_bytes(const pipesd_kv16_cfg* cfg, int32_t n) {
    if (!cfg_ok(cfg) || n < 1 || n > kPlanRequests) return 0;
    return 4 * (1 + 2 * (uint64_t)n + 3 * (uint64_t)plan_cap(cfg, n));
}

int32_t pipesd_kv16_reserve(const pipesd_kv16_cfg* cfg, int32_t n_req, const int32_t* length, int32_t* table, int32_t* refs, int32_t* pages, void* scratch,
                            void* cuda_stream) {
    if (!cfg_ok(cfg) || n_req < 1 || n_req > kPlanRequests || !length || !table || !refs || !pages || !scratch || (uintptr_t)scratch % 4) return PIPESD_E_INVALID;
    const Kv16PlanArgs a = {nullptr, nullptr, length, nullptr, table, refs, pages, n_req, n_req, cfg->n_pages, cfg->max_pages, cfg->page_size,
                            static_cast<int32_t*>(scratch), plan_cap(cfg, n_req)};
    kv16_plan_kernel<<<1, kPlanThreads, 0, (cudaStream_t)cuda_stream>>>(a);
    return launched();
}

int32_t pipesd_kv16_fork(const pipesd_kv16_cfg* cfg, void* pool, int32_t n, const int32_t* src, const int32_t* dst, const int32_t* length,
                         const int32_t* own, int32_t n_slots, int32_t* table, int32_t* refs, int32_t* pages, void* scratch, void* cuda_stream) {
    if (!pool_ok(cfg, pool) || n < 1 || n > kPlanRequests || n_slots < 1 || !src || !dst || !length || !own || !table || !refs || !pages || !scratch || (uintptr_t)scratch % 4)
        return PIPESD_E_INVALID;
    const Kv16PlanArgs a = {src, dst, length, own, table, refs, pages, n, n_slots, cfg->n_pages, cfg->max_pages, cfg->page_size,
                            static_cast<int32_t*>(scratch), plan_cap(cfg, n)};
    kv16_plan_kernel<<<1, kPlanThreads, 0, (cudaStream_t)cuda_stream>>>(a);
    if (cudaGetLastError() != cudaSuccess) return PIPESD_E_CUDA;
    const Kv16CopyArgs c = {static_cast<uint4*>(pool), a.scratch, n, a.cap, cfg->n_layers, cfg->n_pages,
                            (long long)cfg->n_kv_heads * cfg->page_size * cfg->head_dim / 4};
    if (launch_pdl(kv16_copy_kernel, dim3(148 * 8), dim3(kCopyThreads), 0, (cudaStream_t)cuda_stream, c) != cudaSuccess) return PIPESD_E_CUDA;
    return launched();
}

int32_t pipesd_kv16_release(const pipesd_kv16_cfg* cfg, int32_t n_req, const int32_t* length, int32_t* table, int32_t* refs, void* cuda_stream) {
    if (!cfg_ok(cfg) || n_req < 1 || !length || !table || !refs) return PIPESD_E_INVALID;
    kv16_release_kernel<<<n_req, 128, 0, (cudaStream_t)cuda_stream>>>(length, table, refs, cfg->n_pages, cfg->max_pages, cfg->page_size);
    return launched();
}

uint64_t pipesd_kv16_attend_scratch_bytes(const pipesd_kv16_cfg* cfg, int32_t rows, int32_t n_q_heads) {
    if (!cfg_ok(cfg) || rows < 1 || n_q_heads < 1 || n_q_heads % cfg->n_kv_heads || n_q_heads / cfg->n_kv_heads > 128) return 0;
    return kPagesSms * (2 * sizeof(PagesSplit) + (uint64_t)4 * pages_cap(cfg, rows, n_q_heads) * (cfg->head_dim + 2) * 4);
}

int32_t pipesd_kv16_attend(const pipesd_kv16_cfg* cfg, const void* pool, int32_t layer, const void* q, void* out, int32_t dtype, int64_t q_stride,
                           int64_t out_stride, int32_t n_q_heads, float scale, int32_t n_req, int32_t rows, const int32_t* row0, const int32_t* base,
                           const int32_t* table, const uint32_t* mask, int32_t words, void* scratch, void* cuda_stream) {
    if (!where_ok(cfg, pool, layer, n_req, rows, row0, base, table) || !q || !out || !scratch || (uintptr_t)scratch % 16 || !dtype_ok(dtype) ||
        !aligned(q, dtype) || !aligned(out, dtype) || n_q_heads < 1 || n_q_heads % cfg->n_kv_heads || n_q_heads / cfg->n_kv_heads > 128 ||
        !scale_ok(scale) || (mask && (words < 1 || words > kTreeWords)))
        return PIPESD_E_INVALID;
    const int64_t width = (int64_t)n_q_heads * cfg->head_dim;
    if (rows > 1 && (q_stride < width || out_stride < width)) return PIPESD_E_INVALID;
    if ((int64_t)rows * n_q_heads > INT32_MAX) return PIPESD_E_INVALID;
    if (!device_ready()) return PIPESD_E_CUDA;
    PagesArgs a = {};
    a.w = where_of(cfg, n_req, rows, row0, base, table);
    a.p = pool_of(cfg, pool, layer);
    a.q = q;
    a.out = out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.Hq = n_q_heads;
    a.q_wide = wide(q, q_stride, rows, dtype);
    a.out_wide = wide(out, out_stride, rows, dtype);
    a.scale = scale * 1.4426950408889634f;
    a.mask = mask;
    a.words = mask ? words : 0;
    a.splits = static_cast<PagesSplit*>(scratch);
    a.parts = reinterpret_cast<float*>(a.splits + 2 * kPagesSms);
    a.G = n_q_heads / cfg->n_kv_heads;
    a.cap = pages_cap(cfg, rows, n_q_heads);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (cfg->head_dim == 128) return dtype == PIPESD_F32 ? pages_run<128, float>(a, st) : pages_run<128, uint16_t>(a, st);
    return dtype == PIPESD_F32 ? pages_run<64, float>(a, st) : pages_run<64, uint16_t>(a, st);
}

int32_t pipesd_attend_packed(const void* q, const void* k, const void* v, void* out, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                             int64_t out_stride, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float scale, int32_t n_req, int32_t rows,
                             const int32_t* row0, void* cuda_stream) {
    if (!q || !k || !v || !out || !row0 || (head_dim != 64 && head_dim != 128) || n_kv_heads < 1 || n_kv_heads > 65535 || n_q_heads < 1 ||
        n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > 128 || !scale_ok(scale) || n_req < 1 || rows < 1)
        return PIPESD_E_INVALID;
    const int64_t wq = (int64_t)n_q_heads * head_dim, wkv = (int64_t)n_kv_heads * head_dim;
    if ((int64_t)rows * n_q_heads > INT32_MAX) return PIPESD_E_INVALID;
    for (const void* p : {q, k, v, (const void*)out})
        if ((uintptr_t)p % 16) return PIPESD_E_INVALID;
    if (rows > 1 && (q_stride < wq || k_stride < wkv || v_stride < wkv || out_stride < wq || q_stride % 8 || k_stride % 8 || v_stride % 8 || out_stride % 8))
        return PIPESD_E_INVALID;
    if (!device_ready()) return PIPESD_E_CUDA;
    if (rows == 1) { q_stride = out_stride = wq; k_stride = v_stride = wkv; }
    const int G = n_q_heads / n_kv_heads, T = 128 / G;
    CUtensorMap mq, mk, mv;
    if (!rows_map(&mq, q, head_dim, n_q_heads, rows, q_stride, G, T) || !rows_map(&mk, k, head_dim, n_kv_heads, rows, k_stride, 1, 128) ||
        !rows_map(&mv, v, head_dim, n_kv_heads, rows, v_stride, 1, 128))
        return PIPESD_E_INVALID;
    // the jobs there can be: a prompt's last one may be short
    const int64_t jobs = ((int64_t)rows / (2 * T) + std::min(n_req, rows)) * n_kv_heads;
    const PromptArgs a = {row0,    static_cast<const uint16_t*>(v), static_cast<uint16_t*>(out), v_stride, out_stride, n_req, rows, n_q_heads, n_kv_heads,
                          scale * 1.4426950408889634f, (int)std::min<int64_t>(jobs, kSms), g_gives_up.load(std::memory_order_relaxed)};
    if (head_dim == 128) prompt_kernel<128><<<a.ctas, kAttendThreads16, PromptShape<128>::kSmem, (cudaStream_t)cuda_stream>>>(mq, mk, mv, a);
    else prompt_kernel<64><<<a.ctas, kAttendThreads16, PromptShape<64>::kSmem, (cudaStream_t)cuda_stream>>>(mq, mk, mv, a);
    return launched();
}

}  // extern "C"
