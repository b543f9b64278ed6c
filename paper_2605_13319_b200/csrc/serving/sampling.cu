// C entries of shaped sampling and shaped acceptance.
#include <algorithm>

#include "../../../include/pipesd.h"
#include "shape.cuh"

using namespace pipesd;

namespace {

static_assert(sizeof(Shaping) == sizeof(pipesd_shaping), "pipesd_shaping is read as it is");

// CTAs of a row: as many as leave every CTA an SM of its own and 8000 ids.  us, top-p 0.9, by CTAs per row (1, 2, 4, 8): 1 row of 128256
// 89, 55, 37, 29; 32 rows 94, 58, 39, 39; 128 rows 95, 85, 102, 147 (two CTAs fit an SM, but share its fp64 pipes, and clusters do not
// fill every group of SMs to its last place); 16 rows of 32000 31, 25, 21, 25; of 8192 15, 17, 17, 22.
int shape_cluster(int rows, int V) {
    int c = 8;
    while (c > 1 && ((long long)rows * c > 148 || V < c * 8000)) c /= 2;
    return c;
}

bool rows_ok(const void* p, int32_t dtype, int64_t stride, int32_t rows, int32_t vocab) {
    return p && (dtype == PIPESD_F32 || dtype == PIPESD_BF16) && rows >= 1 && vocab >= 1 && vocab <= kShapeMaxVocab && stride >= vocab &&
           (uintptr_t)p % (dtype == PIPESD_F32 ? 4 : 2) == 0;
}

template <int C, bool kDraw, typename T, int VEC>
cudaError_t launch_shape(const ShapeArgs& a, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.rows * C);
    cfg.blockDim = dim3(kShapeThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = C > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, shape_kernel<C, kDraw, T, VEC>, a);
}

template <bool kDraw, typename T, int VEC>
cudaError_t launch_shape_c(const ShapeArgs& a, cudaStream_t st) {
    switch (shape_cluster(a.rows, a.V)) {
        case 8: return launch_shape<8, kDraw, T, VEC>(a, st);
        case 4: return launch_shape<4, kDraw, T, VEC>(a, st);
        case 2: return launch_shape<2, kDraw, T, VEC>(a, st);
        default: return launch_shape<1, kDraw, T, VEC>(a, st);
    }
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
    if (!rows_ok(logits, dtype, row_stride, rows, vocab) || !shaping || !u || !tokens || (probs && probs_stride < vocab)) return PIPESD_E_INVALID;
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
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kAcceptCluster, (unsigned)n_req);
    cfg.blockDim = dim3(kAcceptThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kAcceptCluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = dtype == PIPESD_F32 ? cudaLaunchKernelEx(&cfg, accept_shaped_kernel<float>, a)
                                              : cudaLaunchKernelEx(&cfg, accept_shaped_kernel<uint16_t>, a);
    return e == cudaSuccess ? PIPESD_OK : PIPESD_E_CUDA;
}

}  // extern "C"
