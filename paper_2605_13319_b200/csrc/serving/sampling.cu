// C entries of shaped sampling and shaped acceptance.
#include <algorithm>

#include "../../../include/pipesd.h"
#include "shape.cuh"

using namespace pipesd;

namespace {

static_assert(sizeof(Shaping) == sizeof(pipesd_shaping), "pipesd_shaping is read as it is");

// CTAs of a row: as many as leave every CTA an SM of its own and 8000 ids.  us, top-p 0.9, by CTAs per row (1, 2, 4, 8): 1 row of 128256
// 89, 55, 37, 29; 32 rows 94, 58, 39, 39; 16 rows of 32000 31, 25, 21, 25; of 8192 15, 17, 17, 22.  Two CTAs on an SM pay or cost as the settings have
// it, which the host does not know: 128 rows of 128256 with one and two CTAs (cold) unshaped 63 57, top-p 104 86, top-k 50 55 47, but top-k 1000
// with top-p 158 256, since every CTA of a cluster ranks the whole list of kept ids.  (Clusters do not fill every group of SMs either: 37 rows of four
// such CTAs take 236 where 24 rows take 133.)
int shape_cluster(int rows, int V) {
    int c = 8;
    while (c > 1 && ((long long)rows * c > 148 || V < c * 8000)) c /= 2;
    return c;
}

bool rows_ok(const void* p, int32_t dtype, int64_t stride, int32_t rows, int32_t vocab) {
    return p && (dtype == PIPESD_F32 || dtype == PIPESD_BF16) && rows >= 1 && vocab >= 1 && vocab <= kShapeMaxVocab && stride >= vocab &&
           (uintptr_t)p % (dtype == PIPESD_F32 ? 4 : 2) == 0;
}

// Clusters of C CTAs, with programmatic serialisation (`early`) or without.
template <typename Args>
cudaError_t launch_cluster(void (*kernel)(Args), dim3 grid, int threads, int C, bool early, cudaStream_t st, const Args& a) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (C > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = C;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (early) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
    if (e != cudaSuccess) (void)cudaGetLastError();          // (reported here, not by the next call)
    return e;
}

template <bool kDraw, typename T, int VEC>
cudaError_t launch_rows(const ShapeArgs& a, bool early, cudaStream_t st) {
    const int c = shape_cluster(a.rows, a.V);
    const auto kernel = c == 8 ? shape_kernel<8, kDraw, T, VEC> : c == 4 ? shape_kernel<4, kDraw, T, VEC> : c == 2 ? shape_kernel<2, kDraw, T, VEC> : shape_kernel<1, kDraw, T, VEC>;
    return launch_cluster(kernel, dim3((unsigned)a.rows * c), kShapeThreads, c, early, st, a);
}

// Rows that would begin another wave of one CTA each, a few of them, go by clusters beside the end of the wave before (128256 ids, top-p: 296
// rows 133 us, 310 rows 197 in two waves).
template <bool kDraw, typename T, int VEC>
cudaError_t launch_shape_c(const ShapeArgs& a, cudaStream_t st) {
    const int wave = 2 * 148, rest = a.rows % wave;
    if (a.rows <= wave || rest == 0 || shape_cluster(rest, a.V) == 1) return launch_rows<kDraw, T, VEC>(a, false, st);
    ShapeArgs part = a;
    part.rows = a.rows - rest;
    part.more = true;
    const cudaError_t e = launch_rows<kDraw, T, VEC>(part, false, st);
    if (e != cudaSuccess) return e;
    part.first = a.first + part.rows;
    part.rows = rest;
    part.more = false;
    return launch_rows<kDraw, T, VEC>(part, true, st);
}

template <bool kDraw>
cudaError_t launch_shape_any(const ShapeArgs& a, int dtype, cudaStream_t st) {
    const size_t size = dtype == PIPESD_F32 ? 4 : 2;
    const bool wide = (uintptr_t)a.logits % 16 == 0 && (a.rows == 1 || (size_t)a.stride * size % 16 == 0);
    if (dtype == PIPESD_F32) return wide ? launch_shape_c<kDraw, float, 4>(a, st) : launch_shape_c<kDraw, float, 1>(a, st);
    return wide ? launch_shape_c<kDraw, uint16_t, 8>(a, st) : launch_shape_c<kDraw, uint16_t, 1>(a, st);
}

}  // namespace

extern "C" {

int32_t pipesd_sample(const void* logits, int32_t dtype, int64_t row_stride, int32_t rows, int32_t vocab, const pipesd_shaping* shaping,
                      const float* u, int32_t* tokens, float* probs, int64_t probs_stride, void* cuda_stream) {
    if (!rows_ok(logits, dtype, row_stride, rows, vocab) || !shaping || !u || !tokens || (probs && (probs_stride < vocab || probs == logits)))
        return PIPESD_E_INVALID;
    ShapeArgs a = {};
    a.logits = logits;
    a.stride = row_stride;
    a.V = vocab;
    a.rows = rows;
    a.shaping = reinterpret_cast<const Shaping*>(shaping);
    a.u = u;
    a.tokens = tokens;
    a.probs = probs;
    a.probs_stride = probs_stride;
    return launch_shape_any<true>(a, dtype, (cudaStream_t)cuda_stream) == cudaSuccess ? PIPESD_OK : PIPESD_E_CUDA;
}

uint64_t pipesd_accept_scratch_bytes(int32_t rows) { return rows < 1 ? 0 : (uint64_t)rows * sizeof(RowShape); }

int32_t pipesd_accept(const void* logits, int32_t dtype, int64_t row_stride, int32_t n_req, int32_t rows, int32_t vocab, const int32_t* row0,
                      const pipesd_shaping* shaping, const float* q, int64_t q_stride, const int32_t* drafts, const float* u, int32_t* n_accepted,
                      int32_t* next_token, void* scratch, void* cuda_stream) {
    if (!rows_ok(logits, dtype, row_stride, rows, vocab) || n_req < 1 || n_req > rows || n_req > 65535 || !row0 || !shaping || !u || !n_accepted ||
        !next_token || !scratch || (uintptr_t)scratch % 8)
        return PIPESD_E_INVALID;
    if (rows > n_req && (!q || !drafts || q_stride < vocab)) return PIPESD_E_INVALID;       // (no drafts at all: neither is read)
    cudaStream_t st = (cudaStream_t)cuda_stream;
    ShapeArgs s = {};
    s.logits = logits;
    s.stride = row_stride;
    s.V = vocab;
    s.rows = rows;
    s.shaping = reinterpret_cast<const Shaping*>(shaping);
    s.row0 = row0;
    s.n_req = n_req;
    s.shapes = static_cast<RowShape*>(scratch);
    if (launch_shape_any<false>(s, dtype, st) != cudaSuccess) return PIPESD_E_CUDA;
    AcceptArgs a = {logits, row_stride, vocab, rows, row0, n_req, q, q_stride, drafts, u, s.shapes, n_accepted, next_token};
    // CTAs of a request: as many as fit the device together, two to an SM
    const int c = n_req * 8 <= 2 * 148 ? 8 : n_req * 4 <= 2 * 148 ? 4 : 2;
    const bool f32 = dtype == PIPESD_F32;
    const auto kernel = c == 8 ? (f32 ? accept_shaped_kernel<8, float> : accept_shaped_kernel<8, uint16_t>)
                      : c == 4 ? (f32 ? accept_shaped_kernel<4, float> : accept_shaped_kernel<4, uint16_t>)
                               : (f32 ? accept_shaped_kernel<2, float> : accept_shaped_kernel<2, uint16_t>);
    const cudaError_t e = launch_cluster(kernel, dim3((unsigned)c, (unsigned)n_req), kAcceptThreads, c, true, st, a);
    return e == cudaSuccess ? PIPESD_OK : PIPESD_E_CUDA;
}

}  // extern "C"
