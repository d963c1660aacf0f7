// Which cached rows a query sees and where they lie, for the kernels that read a cache in pages or a tree of drafted tokens.
//   pages: row j of a sequence is plane row  table[j / page] * page + j % page  (pages of a power of two rows, sixteen at least,
//          so that a tile of sixteen cached tokens lies inside one)
//   trees: a query sees the first `prefix` rows of its sequence and, behind them, the rows of the drafted tokens whose bits its
//          mask row has
// Everything here is the same in every lane of a work-group: the loads go through the scalar cache.  The host can run it too.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define EKV_ROWS_FN __host__ __device__ __forceinline__
#else
#include <algorithm>
#define EKV_ROWS_FN inline
using std::max;
using std::min;
#endif

namespace ekv {

struct RowMap {
  const int32_t* table;                     // [sequences, cols]; nullptr: a sequence's rows back to back
  int32_t cols, shift;                      // pages of 1 << shift rows
  int32_t n_pages;                          // pages in the planes: an entry outside [0, n_pages) counts as page 0
  const int32_t* nodes;                     // [sequences] drafted tokens; nullptr: no trees
  const uint32_t* mask;                     // [sequences, q_per_seq, words]
  int32_t words;
};

// A load whose address is the same in every lane, of memory that no kernel of the launch writes: through the scalar cache, so that
// no wait for it is one for the vector loads in flight.
template <typename T>
EKV_ROWS_FN T uniform_load(const T* p) {
#if defined(__HIP_DEVICE_COMPILE__)
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
#else
  return *p;
#endif
}

struct SeenRows {
  const int32_t* table;                     // the sequence's row of the table; without one, something that may be read, and a shift that
  bool paged;                               // has every row on "page" 0 (a page is looked up without a branch, which would split the
                                            // loop of the matrix-core kernels: their accumulators then leave the accumulation registers)
  const uint32_t* mask;                     // the query's row of the masks
  int prefix, len;                          // rows ahead of the tree; one past the last row that is seen (0: nothing is)
  int64_t row0;                             // rows back to back: the sequence's first
  int shift, n_pages, words;

  // seq_len: of every query, or the rows ahead of every sequence's tree; cap: rows of a sequence that may be read at all
  EKV_ROWS_FN SeenRows(const RowMap& m, const int32_t* seq_len, int b, int q_per_seq, int64_t stride, int64_t cap64) {
    const int seq = b / q_per_seq, t = b - seq * q_per_seq;
    const int cap = (int)max(min(cap64, (int64_t)(INT32_MAX - 256)), (int64_t)0);    // (room for sums of a row and a tile or a tree)
    paged = m.table != nullptr;
    shift = paged ? m.shift : 31; n_pages = m.n_pages; words = m.words;
    row0 = seq * stride;
    table = paged ? m.table + (int64_t)seq * m.cols : seq_len;
    mask = m.nodes ? m.mask + ((int64_t)seq * q_per_seq + t) * m.words : nullptr;
    prefix = len = min(max(uniform_load(seq_len + (mask ? seq : b)), 0), cap);
    if (mask) {
      const int nodes = min(uniform_load(m.nodes + seq), q_per_seq);
      const int room = min(nodes, cap - prefix);                 // drafted tokens whose rows may be read
      for (int w = 0; w < words; ++w) {
        uint32_t bits = uniform_load(mask + w);
        if (room < 32 * w + 32) bits = room > 32 * w ? bits & ((1u << (room - 32 * w)) - 1u) : 0u;
        if (bits) len = prefix + 32 * w + 32 - __builtin_clz(bits);
      }
      if (t >= nodes) len = 0;
    }
  }

  // the page of a tile that begins at row j < len
  EKV_ROWS_FN int page(int j) const { return uniform_load(table + (j >> shift)); }
  // the plane row of row j, whose page that is
  EKV_ROWS_FN int64_t row(int j, int page) const {
    if (!paged) return row0 + j;
    const int p = (uint32_t)page < (uint32_t)n_pages ? page : 0;
    return ((int64_t)p << shift) + (j & ((1 << shift) - 1));
  }

  // which of the rows j .. j + 15 are seen (j < len): bit i for row j + i
  EKV_ROWS_FN uint32_t tile(int j) const {
    uint32_t seen = len - j >= 16 ? 0xffffu : (1u << (len - j)) - 1u;
    if (mask && j + 16 > prefix) {
      const int node = j - prefix, lo = max(node, 0), w = lo >> 5;           // (-15 at least)
      uint64_t bits = w < words ? uniform_load(mask + w) : 0u;
      if (w + 1 < words) bits |= (uint64_t)uniform_load(mask + w + 1) << 32;
      bits >>= lo & 31;
      if (node < 0) bits = (bits << -node) | ((1u << -node) - 1u);
      seen &= (uint32_t)bits;
    }
    return seen;
  }
  EKV_ROWS_FN bool sees(int j) const {
    if (j >= len) return false;
    if (!mask || j < prefix) return true;
    return (mask[(j - prefix) >> 5] >> ((j - prefix) & 31)) & 1u;
  }
};

}  // namespace ekv
