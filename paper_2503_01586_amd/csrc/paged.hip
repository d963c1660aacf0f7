// What a server keeps a cache in pages with, and what it does around the attention of a drafted tree: pages handed out and taken
// back (page_plan), masks and positions of the trees (tree_plan), the accepted path's rows moved up (tree_commit).
// All of it is whole numbers and copies; every kernel is bound by a launch and one or two trips to memory, not by its bytes.
#include "common.hpp"
#include "launch.hpp"

namespace ekv {

// ---- pages ----
// Request b holds the first held[b] pages of its row of the table and needs  want = ceil((cached + new) / page).  The pages it
// lacks come from the front of a ring of free ones, the ones it no longer needs go to the ring's end, all in the order of the
// requests, so two running sums over the requests say where everything lies and nothing depends on the order of execution.
// The ring never holds more entries than there are pages, so what is read of it (the front) and what is written (behind the
// end) never share a place: a call does not hand out again what it takes back.
struct PageRecord {
  int64_t held_want;                        // held | want << 32
  int32_t front, granted;                   // place in the ring of the first page handed out, and how many are
  int32_t back;                             // place in the ring of the first page that goes back
};

__device__ __forceinline__ int page_held(const PageRecord& r) { return (int)(uint32_t)r.held_want; }
__device__ __forceinline__ int page_want(const PageRecord& r) { return (int)(r.held_want >> 32); }
__device__ __forceinline__ int ring_place(int base, int off, int n) {
  const uint32_t i = (uint32_t)base + (uint32_t)off;
  return (int)(i < (uint32_t)n ? i : i % (uint32_t)n);
}

constexpr int kPlanThreads = 1024;

// Phase one, by one work-group: the records of up to 1024 requests from b0 on; grown and back: the sums over the requests ahead,
// carried from call to call in every thread.
__device__ __forceinline__ void page_records(const PagePlanArgs& a, int64_t b0, int64_t taken, int64_t given, int64_t& grown,
                                             int64_t& back, PageRecord* rec, int64_t* sums) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = b0 + tid;
  int held = 0, want = 0;
  if (b < a.B) {
    held = min(max(a.held[b], 0), a.cols);
    const int64_t tokens = (int64_t)max(a.cached_len[b], 0) + min(max(a.new_len[b], 0), a.T);
    want = (int)min((tokens + (1 << a.shift) - 1) >> a.shift, (int64_t)a.cols);
  }
  const int64_t grow = max(want - held, 0), less = max(held - want, 0);
  int64_t g = grow, l = less;               // inclusive sums over the wave, then over the waves ahead
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t gu = __shfl_up(g, o, kWave), lu = __shfl_up(l, o, kWave);
    if (lane >= o) { g += gu; l += lu; }
  }
  if (lane == 63) { sums[2 * wave] = g; sums[2 * wave + 1] = l; }
  __syncthreads();
  int64_t all_g = 0, all_l = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) { g += sums[2 * w]; l += sums[2 * w + 1]; }
    all_g += sums[2 * w];
    all_l += sums[2 * w + 1];
  }
  __syncthreads();
  if (b < a.B) {
    const int64_t before = grown + g - grow;
    const int64_t avail = min(max(given - taken, (int64_t)0), (int64_t)a.n_pages);
    PageRecord r;
    r.held_want = (int64_t)(uint32_t)held | (int64_t)want << 32;
    r.granted = (int)min(max(avail - before, (int64_t)0), grow);
    r.front = (int)((uint64_t)(taken + before) % (uint32_t)a.n_pages);
    r.back = (int)((uint64_t)(given + back + l - less) % (uint32_t)a.n_pages);
    *rec = r;
  }
  grown += all_g;
  back += all_l;
}

// what all requests were granted, and the counts of the ring after the call
__device__ __forceinline__ void page_totals(const PagePlanArgs& a, int64_t taken, int64_t given, int64_t grown, int64_t back) {
  const int64_t avail = min(max(given - taken, (int64_t)0), (int64_t)a.n_pages);
  a.span_out[0] = taken + min(grown, avail);
  a.span_out[1] = given + back;
}

// Phase two for one request: its pages, by `n` threads
__device__ __forceinline__ void page_moves(const PagePlanArgs& a, int64_t b, const PageRecord& r, int i, int n) {
  int32_t* row = a.table + b * a.cols;
  const int held = page_held(r), want = page_want(r);
  if (i == 0) a.held_out[b] = held > want ? want : held + r.granted;
  for (int k = i; k < r.granted; k += n) row[held + k] = a.ring[ring_place(r.front, k, a.n_pages)];
  for (int k = i; k < held - want; k += n) a.ring[ring_place(r.back, k, a.n_pages)] = row[want + k];
}
// ... and for one new token t of it.  (A page handed out in this call is taken from the ring, not from the table's row, which
// another thread is about to write.)
__device__ __forceinline__ void page_token(const PagePlanArgs& a, int64_t b, int t, const PageRecord& r) {
  const int64_t pos = (int64_t)max(a.cached_len[b], 0) + t, at = pos >> a.shift;
  const int held = page_held(r), want = page_want(r);
  const bool real = t < a.new_len[b];
  int64_t slot = -1;
  if (real && at < (held > want ? want : held + r.granted)) {
    const int page = at < held ? a.table[b * a.cols + at] : a.ring[ring_place(r.front, (int)at - held, a.n_pages)];
    if ((uint32_t)page < (uint32_t)a.n_pages) slot = ((int64_t)page << a.shift) + (pos & ((1 << a.shift) - 1));
  }
  const int64_t e = b * a.T + t;
  a.pos[e] = real ? (int32_t)pos : 0;
  a.slot[e] = slot;
  a.kv_len[e] = slot >= 0 ? (int32_t)pos + 1 : 0;
}

// Few requests and tokens: both phases in one launch of one work-group, the records in LDS.  64 requests of one token: 4.6 us, a launch
// and three trips to memory one behind the other (lengths and counts, ring, table and tokens).
__global__ __launch_bounds__(kPlanThreads) void page_plan_small_kernel(const PagePlanArgs a) {
  __shared__ int64_t sums[2 * kPlanThreads / 64];
  __shared__ PageRecord rec[kPlanThreads];
  const int tid = threadIdx.x;
  const int64_t taken = a.span[0], given = a.span[1];
  int64_t grown = 0, back = 0;
  page_records(a, 0, taken, given, grown, back, rec + tid, sums);
  __syncthreads();                          // (held and span have been read: their outputs may be the same arrays)
  if (tid == 0) page_totals(a, taken, given, grown, back);
  const int n = (int)a.B, per = kPlanThreads / n > 64 ? 64 : kPlanThreads / n;     // threads for a request's pages
  if (tid < n * per) page_moves(a, tid / per, rec[tid / per], tid % per, per);
  const int tokens = n * a.T;
  for (int e = tid; e < tokens; e += kPlanThreads) page_token(a, e / a.T, e % a.T, rec[e / a.T]);
}

// The others.  Up to 1024 requests whose counts are not updated in place: every work-group forms all records for itself and fills its
// share.  Else the records first, then a wave for every request's pages and a thread for every token.  256 requests of up to 2048 tokens:
// 8.3 us for the 8.4 MB of positions, slots and lengths (in two launches the call takes 9.6 us instead of 7.7).
constexpr int kFillTokens = 4096;            // tokens of a work-group
__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(const PagePlanArgs a, int token_groups) {
  __shared__ int64_t sums[2 * kPlanThreads / 64];
  __shared__ PageRecord rec[kPlanThreads];
  const int tid = threadIdx.x;
  const int64_t taken = a.span[0], given = a.span[1];
  int64_t grown = 0, back = 0;
  page_records(a, 0, taken, given, grown, back, rec + tid, sums);
  __syncthreads();
  if ((int)blockIdx.x < token_groups) {
    const int64_t end = min((int64_t)(blockIdx.x + 1) * kFillTokens, a.B * a.T);
    for (int64_t e = (int64_t)blockIdx.x * kFillTokens + tid; e < end; e += kPlanThreads) {
      const int b = (int)(e / a.T);
      page_token(a, b, (int)(e - (int64_t)b * a.T), rec[b]);
    }
  } else {
    const int g = blockIdx.x - token_groups, b = g * (kPlanThreads / 64) + (tid >> 6);
    if (b < a.B) page_moves(a, b, rec[b], tid & 63, 64);
    if (g == 0 && tid == 0) page_totals(a, taken, given, grown, back);
  }
}

__global__ __launch_bounds__(kPlanThreads) void page_records_kernel(const PagePlanArgs a) {
  __shared__ int64_t sums[2 * kPlanThreads / 64];
  const int64_t taken = a.span[0], given = a.span[1];
  int64_t grown = 0, back = 0;
  for (int64_t b0 = 0; b0 < a.B; b0 += kPlanThreads)
    page_records(a, b0, taken, given, grown, back, reinterpret_cast<PageRecord*>(a.ws) + b0 + threadIdx.x, sums);
  __syncthreads();
  if (threadIdx.x == 0) page_totals(a, taken, given, grown, back);
}
__global__ __launch_bounds__(256) void page_fill_kernel(const PagePlanArgs a, int token_groups) {
  const PageRecord* rec = reinterpret_cast<const PageRecord*>(a.ws);
  if ((int)blockIdx.x < token_groups) {
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e < a.B * a.T) {
      const int64_t b = e / a.T;
      page_token(a, b, (int)(e - b * a.T), rec[b]);
    }
  } else {
    const int64_t b = (int64_t)(blockIdx.x - token_groups) * 4 + (threadIdx.x >> 6);
    if (b < a.B) page_moves(a, b, rec[b], threadIdx.x & 63, 64);
  }
}

size_t page_plan_workspace(int64_t B) { return (size_t)B * sizeof(PageRecord); }

hipError_t launch_page_plan(const PagePlanArgs& a, hipStream_t stream) {
  if (a.B <= kPlanThreads && a.B * a.T <= 4 * kPlanThreads) {
    page_plan_small_kernel<<<1, kPlanThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  if (a.B <= kPlanThreads && a.held_out != a.held && a.span_out != a.span) {
    const int64_t groups = (a.B * a.T + kFillTokens - 1) / kFillTokens;
    page_plan_kernel<<<(unsigned)(groups + (a.B + kPlanThreads / 64 - 1) / (kPlanThreads / 64)), kPlanThreads, 0, stream>>>(a, (int)groups);
    return hipGetLastError();
  }
  page_records_kernel<<<1, kPlanThreads, 0, stream>>>(a);
  const int64_t token_groups = (a.B * a.T + 255) / 256;
  page_fill_kernel<<<(unsigned)(token_groups + (a.B + 3) / 4), 256, 0, stream>>>(a, (int)token_groups);
  return hipGetLastError();
}

// ---- a prompt's rows ----
// The first S rows of every sequence, from its pages to planes in which they lie back to back: what the rebuild of keys and values for
// many queries reads (elitekv_prefill_attn's kernels).  A work-group copies a tile of sixteen rows, which lies inside one page, of both
// planes.  2 x 4000 rows of 7B 25 %: 12.5 us for 33 MB read and as much written, 5.2 TB/s (a copy of 4 GiB: 4.75).
__global__ __launch_bounds__(256) void gather_pages_kernel(const RowMap map, const ekv_u32x4* __restrict__ ke_plane,
                                                           const ekv_u32x4* __restrict__ c_plane, int ke_units, int c_units, int64_t S,
                                                           ekv_u32x4* __restrict__ ke_out, ekv_u32x4* __restrict__ c_out) {
  const int64_t b = blockIdx.y, j = (int64_t)blockIdx.x * 16, to = b * S + j;
  const int rows = (int)min((int64_t)16, S - j);
  const int page = uniform_load(map.table + b * map.cols + (j >> map.shift));
  const int64_t from = ((int64_t)((uint32_t)page < (uint32_t)map.n_pages ? page : 0) << map.shift) + (j & ((1 << map.shift) - 1));
  auto copy = [&](const ekv_u32x4* src, ekv_u32x4* dst, int n) {
    int i = threadIdx.x;
    for (; i + 3 * 256 < n; i += 4 * 256) {                // four pieces under way
      ekv_u32x4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = src[i + u * 256];
#pragma unroll
      for (int u = 0; u < 4; ++u) dst[i + u * 256] = v[u];
    }
    for (; i < n; i += 256) dst[i] = src[i];
  };
  copy(c_plane + from * c_units, c_out + to * c_units, rows * c_units);
  copy(ke_plane + from * ke_units, ke_out + to * ke_units, rows * ke_units);
}

hipError_t launch_gather_pages(const elitekv_dims& d, const RowMap& map, const void* ke_plane, const void* c_plane, int64_t B, int64_t S,
                               void* ke_out, void* c_out, hipStream_t stream) {
  gather_pages_kernel<<<dim3((unsigned)((S + 15) / 16), (unsigned)B), 256, 0, stream>>>(
      map, (const ekv_u32x4*)ke_plane, (const ekv_u32x4*)c_plane, 2 * d.r * d.n_heads * 2 / 16, d.d_c * 2 / 16, S, (ekv_u32x4*)ke_out,
      (ekv_u32x4*)c_out);
  return hipGetLastError();
}

// ---- trees ----
// A work-group per sequence, a thread per node.  A node sees itself and what its parent sees: the masks and the nodes that the
// chains have reached double in every round (mask |= the reached node's mask), seven rounds for a chain of 128; the depth is the
// number of bits less one.  One tree of 8 nodes 2.0 us, 256 of 128 4.3 (a launch, and a trip to memory for lengths and parents).
constexpr int kTreeNodes = ELITEKV_TREE_MAX_NODES, kTreeWords = kTreeNodes / 32;

__global__ __launch_bounds__(kTreeNodes) void tree_plan_kernel(const int32_t* __restrict__ parent,
                                                               const int32_t* __restrict__ prefix_len,
                                                               const int32_t* __restrict__ n_nodes, int T,
                                                               int32_t* __restrict__ pos, uint32_t* __restrict__ mask) {
  __shared__ uint32_t seen[kTreeNodes][kTreeWords + 1];
  __shared__ int up[kTreeNodes];
  const int t = threadIdx.x;
  const int64_t b = blockIdx.x;
  const int nodes = min(n_nodes[b], T), words = (T + 31) >> 5;
  const bool real = t < nodes;
  int at = t < T ? parent[b * T + t] : -1;
  if ((uint32_t)at >= (uint32_t)t || !real) at = -1;           // (an entry that is no earlier node: a root)
  uint32_t m[kTreeWords];
#pragma unroll
  for (int w = 0; w < kTreeWords; ++w) m[w] = real && t >> 5 == w ? 1u << (t & 31) : 0u;
  bool more = __syncthreads_or(at >= 0);
  while (more) {
#pragma unroll
    for (int w = 0; w < kTreeWords; ++w) seen[t][w] = m[w];
    up[t] = at;
    __syncthreads();
    if (at >= 0) {
#pragma unroll
      for (int w = 0; w < kTreeWords; ++w) m[w] |= seen[at][w];
      at = up[at];
    }
    more = __syncthreads_or(at >= 0);
  }
  if (t >= T) return;
  int depth = -1;
#pragma unroll
  for (int w = 0; w < kTreeWords; ++w) {
    depth += __popc(m[w]);
    if (w < words) mask[(b * T + t) * words + w] = m[w];
  }
  pos[b * T + t] = real ? prefix_len[b] + depth : 0;
}

hipError_t launch_tree_plan(const int32_t* parent, const int32_t* prefix_len, const int32_t* n_nodes, int64_t B, int64_t T,
                            int32_t* pos, uint32_t* mask, hipStream_t stream) {
  tree_plan_kernel<<<(unsigned)B, T <= 64 ? 64 : kTreeNodes, 0, stream>>>(parent, prefix_len, n_nodes, (int)T, pos, mask);
  return hipGetLastError();
}

// ---- the accepted path ----
// Row prefix + k takes what row prefix + path[k] holds, k <= path[k], for both planes; a rotated key stays as it is: a node's
// position is prefix + its depth, and the k-th node of a path has depth k.  A thread owns a piece of the row for every k, so no
// two threads touch the same bytes: rows that are sources of later copies lie at or behind the rows written so far, and 16
// copies are loaded ahead of the first of them being stored.  One path of up to 8 nodes, 7B 25 %: 2.7 us; 128 of up to 26, 13B 25 %: 7.2 us,
// the trips for lengths and path, table, rows, one behind the other.
constexpr int kCommitAhead = 16;

template <typename U>
__global__ __launch_bounds__(256) void tree_commit_kernel(const int32_t* __restrict__ path, const int32_t* __restrict__ path_len,
                                                          const int32_t* __restrict__ prefix_len, int T, int64_t stride,
                                                          int64_t plane_rows, int64_t cap, const RowMap map, U* ke_plane, U* c_plane, int ke_units,
                                                          int c_units) {
  __shared__ int64_t from[kTreeNodes], to[kTreeNodes];
  __shared__ int first[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = blockIdx.y;
  const int n = min(path_len[b], T);
  const int64_t prefix = prefix_len[b];
  int64_t f = -1, t = -1;
  if (tid < n) {
    const int node = path[b * T + tid];
    if (prefix >= 0 && node > tid && node < T && prefix + node < cap) {
      auto row = [&](int64_t j) -> int64_t {
        if (!map.table) return b * stride + j < plane_rows ? b * stride + j : -1;
        const int page = map.table[b * map.cols + (j >> map.shift)];
        return (uint32_t)page < (uint32_t)map.n_pages ? ((int64_t)page << map.shift) + (j & ((1 << map.shift) - 1)) : -1;
      };
      f = row(prefix + node);
      t = row(prefix + tid);
    }
  }
  // the copies there are, in their order
  const bool real = f >= 0 && t >= 0;
  const uint64_t all = __ballot(real);
  if (lane == 0 && wave < 2) first[wave] = __popcll(all);
  __syncthreads();
  if (real) {
    const int at = __popcll(all & ((1ull << lane) - 1ull)) + (wave > 0 ? first[0] : 0);
    from[at] = f;
    to[at] = t;
  }
  const int m = __builtin_amdgcn_readfirstlane(first[0] + first[1]);
  __syncthreads();
  const int u = blockIdx.x * 256 + tid;
  if (m == 0 || u >= ke_units + c_units) return;
  U* plane = u < ke_units ? ke_plane + u : c_plane + (u - ke_units);
  const int64_t row_units = u < ke_units ? ke_units : c_units;
  for (int k0 = 0; k0 < m; k0 += kCommitAhead) {
    U v[kCommitAhead];
#pragma unroll
    for (int i = 0; i < kCommitAhead; ++i) v[i] = plane[from[min(k0 + i, m - 1)] * row_units];   // (past the last: the last again)
#pragma unroll
    for (int i = 0; i < kCommitAhead; ++i)
      if (k0 + i < m) plane[to[k0 + i] * row_units] = v[i];
  }
}

hipError_t launch_tree_commit(const elitekv_dims& d, const int32_t* path, const int32_t* path_len, const int32_t* prefix_len,
                              int64_t B, int64_t T, int64_t stride, int64_t plane_rows, int64_t cap, const RowMap& map, void* ke_plane, void* c_plane,
                              hipStream_t stream) {
  const int e = d.dtype == ELITEKV_FP32 ? 4 : 2;
  const int64_t ke = (int64_t)2 * d.r * d.n_heads * e, c = (int64_t)d.d_c * e;
  // 16 bytes a thread where both rows are whole pieces of them, an element otherwise
  const int unit = ke % 16 == 0 && c % 16 == 0 ? 16 : e;
  const dim3 grid((unsigned)(((ke + c) / unit + 255) / 256), (unsigned)B);
#define EKV_COMMIT(U)                                                                                                          \
  tree_commit_kernel<U><<<grid, 256, 0, stream>>>(path, path_len, prefix_len, (int)T, stride, plane_rows, cap, map, (U*)ke_plane, (U*)c_plane, \
                                                  (int)(ke / unit), (int)(c / unit))
  if (unit == 16) EKV_COMMIT(ekv_u32x4);
  else if (unit == 4) EKV_COMMIT(uint32_t);
  else EKV_COMMIT(uint16_t);
#undef EKV_COMMIT
  return hipGetLastError();
}

}  // namespace ekv
