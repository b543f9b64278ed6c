// Where the requests of a call on a paged cache are.
#pragma once
#include "../common.cuh"

namespace pipesd {

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

}  // namespace pipesd
