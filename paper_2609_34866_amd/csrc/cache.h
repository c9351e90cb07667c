// cache.h -- the paged cache of quantized keys and values, as its kernels see it (cache.hip, attn_cache.hip).
//
// A page holds page_size tokens of every key/value head:
//   keys    [page][head][token][DHB]          values [page][head][token / 32][DHB][token % 32]
//   scales, zero-points [page][head][token]
// with DHB = dh bits / 8 bytes; at 4 bits a byte holds elements i (low) and i + dh / 2 (high).  Values
// lie transposed in blocks of 32 tokens, so that a matrix-core operand over the tokens is one load.
#pragma once

#include "kernels.h"

namespace jab {
namespace {

// The tables are read at wave-uniform places and never written by these kernels: scalar loads, which leave the
// vector loads in flight alone.
__device__ inline int table(const int32_t *p, int64_t i) {
    typedef const __attribute__((address_space(4))) int32_t *scalar;
    return ((scalar)(uintptr_t)p)[i];
}

// the new tokens of a sequence: rows row .. row + n of the batch, at positions past .. past + n
struct SeqRows {
    int row, n, past;
};
// Counts that do not fit the buffers are cut to what does: no access depends on them being right.
__device__ inline SeqRows seq_rows(const CacheArgs &g, int s) {
    SeqRows r;
    r.row = min(max(table(g.start, s), 0), g.M);
    r.n = min(max(table(g.start, s + 1), r.row), g.M) - r.row;
    r.past = min(max(table(g.past, s), 0), g.cap);
    return r;
}
// the page that holds position pos (below cap) of sequence s, or -1
__device__ inline int page_of(const CacheArgs &g, int s, int pos) {
    const int p = table(g.pages, (int64_t)s * g.max_pages + (pos >> g.page_shift));
    return p >= 0 && p < g.n_pages ? p : -1;
}

}  // namespace
}  // namespace jab
