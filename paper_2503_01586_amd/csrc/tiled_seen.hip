// The decode kernels in fp32 arithmetic (tiled_f32.hip) for caches in pages and for trees of drafted tokens, and what stands around
// their attention for many rows.
#include "tiled_f32.hpp"
#include "reader_map.hpp"
#include <type_traits>

namespace ekv {

// ---- split attention ----
// The products of attn_tiled_kernel: work-group (8 waves) = (split, 16 heads, query row), per tile of 16 cached tokens every wave takes CPW
// blocks of 16 latent columns; scores, maxima, sums and accumulators in fp32.  A tile of 16 rows lies inside one page.  What differs:
//   * A row that is not seen is not loaded: its lanes load the last one of the tile that is, or, where a tile has none, the last of all.
//   * A wave takes CPW whole blocks without a branch: where the blocks do not suffice its window is moved back, with zeros for the query of
//     blocks that are another wave's (SEP, separated latents: a wave without score or value blocks leaves out those products).  A branch a
//     block has the compiler wait for every LDS read and for all loads under way.
//   * A block's registers are loaded again right behind its score products, so that a row has a whole tile's time to come; its page and
//     address are looked up during the value products of the tile before.
//   * Column block g of GW blocks holds columns GW i + e, so that a lane's GW columns are one LDS read: A operand of GW products.
//   * The work-groups that read the same rows follow each other on an XCD (reader_map.hpp), as for several queries in bf16.
// 2 x 12 nodes behind 1000 and 567 tokens, 7B 25 %: 75 us (attn_tiled_kernel with a table and masks, branches and all: 97); 2 x 24 behind
// 2000 the whole call 371 -> 293.  Bound by the fp32 matrix cores and, between two tiles' products, the exchange of the scores' parts: of
// 75 us the products are 33 in the work-groups with most tiles (13 of 16 tokens), 23 on average; a work-group's start takes 8.
// (Scores of the next tile formed while the parts of this one are exchanged: 82, the rows then have too little time to come.)
template <typename T, int CPW, bool SEP>
__global__ __launch_bounds__(kTtWaves * 64) void attn_seen_tiled_kernel(
    const T* __restrict__ ke_plane, const T* __restrict__ c_plane, const float* __restrict__ qe,
    const float* __restrict__ qt, const int32_t* __restrict__ seq_len, float* __restrict__ part_m,
    float* __restrict__ part_l, float* __restrict__ part_u, int n_h, int two_r, int d_c, int d_q, int d_u,
    int64_t max_seq_len, int64_t batch_stride_rows, int64_t plane_rows, int n_splits, int q_per_seq, int batch, int reader_run,
    int reader_turns, const RowMap map) {
  constexpr int CS = CPW * 16 + 4;                        // row of a wave's slice in LDS: conflict-free both ways
  constexpr int KE = CPW < 12 ? 4 : 2;                    // elite pieces of a lane requested ahead (registers)
  constexpr int GW = CPW % 4 == 0 ? 4 : CPW % 2 == 0 ? 2 : 1, GROUPS = CPW / GW;
  typedef __attribute__((ext_vector_type(GW))) float vec;
  extern __shared__ __align__(16) float smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  float* cs = smem + wave * kTtTok * CS;                  // [wave][16 tokens][CS]
  tf_f32x4* sp = reinterpret_cast<tf_f32x4*>(smem + kTtWaves * kTtTok * CS);   // [2][8 waves + elite][64 lanes]
  float* qe_s = smem + kTtWaves * kTtTok * CS + 2 * (kTtWaves + 1) * 64 * 4;   // [16 heads][two_r]

  // (every argument is fetched in one trip of the scalar cache)
  asm volatile("" ::"s"(ke_plane), "s"(c_plane), "s"(qe), "s"(qt), "s"(seq_len), "s"(n_h), "s"(two_r), "s"(d_c), "s"(d_q), "s"(d_u),
               "s"(max_seq_len), "s"(batch_stride_rows), "s"(plane_rows), "s"(n_splits), "s"(q_per_seq), "s"(batch), "s"(reader_run),
               "s"(reader_turns));
  asm volatile("" ::"s"(map.table), "s"(map.cols), "s"(map.shift), "s"(map.n_pages), "s"(map.nodes), "s"(map.mask), "s"(map.words));
  const int groups = (n_h + 15) / 16, readers = q_per_seq * groups;
  const int place = reader_place(blockIdx.x, n_splits * batch * groups, reader_run, reader_turns);
  if (place < 0) return;
  const int item = place / readers, reader = place % readers;
  const int split = __builtin_amdgcn_readfirstlane(item % n_splits), h0 = __builtin_amdgcn_readfirstlane(reader % groups * 16);
  const int b = __builtin_amdgcn_readfirstlane(item / n_splits * q_per_seq + reader / groups);
  const int i16 = lane & 15, quad = lane >> 4;
  const int head = h0 + i16;
  const int head_ld = min(head, n_h - 1);                 // lanes past the last head repeat it and store nothing
  const int64_t pi = ((int64_t)b * n_splits + split) * n_h + head;

  // this wave's blocks are [blk0, blk0 + CPW) as far as they exist; it loads those from win on
  const int n_blks = d_c / 16, q_blks = d_q / 16, v_blk0 = (d_c - d_u) / 16;
  const int blk0 = wave * CPW, win = min(blk0, n_blks - CPW);
  const bool does_q = blk0 < q_blks, does_v = blk0 < n_blks && win + CPW > v_blk0;

  // elite term: this lane's (token, head) pair is token 2 wave + quad / 2, head i16; quad & 1 takes every other 4 values
  const int ke_units = two_r / 4, ke_par = quad & 1, ke_tok = 2 * wave + (quad >> 1);

  // (requested ahead of everything that waits for a length or a page)
  tf_f32x4 acc[CPW], cv[CPW], qv[CPW], kv[KE], qev[KE];
  const float* qrow = qt + ((int64_t)b * n_h + head_ld) * d_q + quad * 4;
  const float* qe_row = qe + ((int64_t)b * n_h + head_ld) * two_r;
#pragma unroll
  for (int u = 0; u < KE; ++u) qev[u] = ld4(qe_row + max(min(2 * u + ke_par, ke_units - 1), 0) * 4);   // (r = 0: not used)
#pragma unroll
  for (int i = 0; i < CPW; ++i) qv[i] = ld4(qrow + min(win + i, q_blks - 1) * 16);

  const int64_t room = plane_rows - (int64_t)(b / q_per_seq) * batch_stride_rows;
  const SeenRows seen(map, seq_len, b, q_per_seq, batch_stride_rows, map.table ? max_seq_len : min(max_seq_len, room));
  const int len = seen.len, n_tiles = (len + kTtTok - 1) / kTtTok;
  if (split >= n_tiles) {
    if (wave == 0 && quad == 0 && head < n_h) {
      part_m[pi] = -INFINITY;
      part_l[pi] = 0.f;
    }
    return;
  }

  auto page_at = [&](int tile) { return seen.page(min(tile, n_tiles - 1) * kTtTok); };
  int tile = split;
  const int end_page = seen.page(len - 1), page0 = page_at(tile), page1 = page_at(tile + n_splits);
  int page = page_at(tile + 2 * n_splits);
  const int64_t end_row = seen.row(len - 1, end_page);
  const T *krow = ke_plane, *crow = c_plane;
  uint32_t sees = 0;
  auto aim = [&](int j, int page) {                       // at the tile that begins at row j
    sees = seen.tile(j);
    const int64_t row = sees ? seen.row(j, page) : end_row;
    const int last = sees ? 31 - __builtin_clz(sees) : 0;
    const int c_tok = (sees >> i16) & 1u ? i16 : last, k_tok = (sees >> ke_tok) & 1u ? ke_tok : last;
    krow = ke_plane + ((row + k_tok) * n_h + head_ld) * two_r;
    crow = c_plane + (row + c_tok) * d_c + win * 16 + quad * 4;
  };
  const T* kmore = ke_plane;                              // the same keys' row, for the pieces that are not requested ahead
  auto load_keys = [&]() {
    kmore = krow;
#pragma unroll
    for (int u = 0; u < KE; ++u)
      if (2 * u < ke_units) kv[u] = ld4(krow + min(2 * u + ke_par, ke_units - 1) * 4);
  };

  aim(tile * kTtTok, page0);
  load_keys();
#pragma unroll
  for (int i = 0; i < CPW; ++i) cv[i] = ld4(crow + i * 16);
  const uint32_t first = sees;
  if (ke_units > 2 * KE) {                         // elite rows of more than 8 KE values
    for (int e = tid; e < 16 * two_r; e += kTtWaves * 64)
      qe_s[e] = qe[((int64_t)b * n_h + min(h0 + e / two_r, n_h - 1)) * two_r + e % two_r];
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < CPW; ++i) acc[i] = (tf_f32x4)(0.f);
  float m = -INFINITY, l = 0.f;
  // everything requested so far has landed: a wait for it inside the loop would be one for the next tile's rows, every time
  __builtin_amdgcn_s_waitcnt(0x0f70);
  if (win < blk0 || win + CPW > q_blks) {                  // blocks that are another wave's, or values only
#pragma unroll
    for (int i = 0; i < CPW; ++i)
      if (win + i < blk0 || win + i >= q_blks) qv[i] = (tf_f32x4)(0.f);
  }

  // a tile's rows are aimed at while the tile two before it is in its value products
  uint32_t now = first;
  aim(min(tile + n_splits, n_tiles - 1) * kTtTok, page1);
  int buf = 0;
  for (; tile < n_tiles; tile += n_splits, buf ^= 1) {
    float es = 0.f;
#pragma unroll
    for (int u = 0; u < KE; ++u)
      if (2 * u < ke_units) {
        const bool in = 2 * u + ke_par < ke_units;
#pragma unroll
        for (int e = 0; e < 4; ++e) es = fmaf(in ? kv[u][e] : 0.f, qev[u][e], es);
      }
    for (int u = KE; 2 * u + ke_par < ke_units; ++u) {
      const tf_f32x4 kx = ld4(kmore + (2 * u + ke_par) * 4);
      const float* qp = qe_s + i16 * two_r + (2 * u + ke_par) * 4;
#pragma unroll
      for (int e = 0; e < 4; ++e) es = fmaf(kx[e], qp[e], es);
    }
    es += __shfl_xor(es, 16, kWave);

    // the scores, and the next tile's rows behind every block's products: in flight until its turn a tile later
    tf_f32x4 s4[2] = {(tf_f32x4)(0.f), (tf_f32x4)(0.f)};
    auto scores = [&](auto product, auto more) {
#pragma unroll
      for (int i = 0; i < CPW; ++i) {
        *reinterpret_cast<tf_f32x4*>(cs + i16 * CS + i * 16 + quad * 4) = cv[i];
        if constexpr (decltype(product)::value) {
#pragma unroll
          for (int e = 0; e < 4; ++e) s4[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(cv[i][e], qv[i][e], s4[e & 1], 0, 0, 0);
        }
        if constexpr (decltype(more)::value) cv[i] = ld4(crow + i * 16);
      }
    };
    if (tile + n_splits < n_tiles) {
      load_keys();
      if (!SEP || does_q) scores(std::true_type{}, std::true_type{});
      else scores(std::false_type{}, std::true_type{});
    } else {
      if (!SEP || does_q) scores(std::true_type{}, std::false_type{});
      else scores(std::false_type{}, std::false_type{});
    }
    tf_f32x4* spb = sp + buf * (kTtWaves + 1) * 64;
    spb[wave * 64 + lane] = s4[0] + s4[1];
    if (ke_par == 0) reinterpret_cast<float*>(spb + kTtWaves * 64 + (ke_tok >> 2) * 16 + i16)[ke_tok & 3] = es;
    __syncthreads();

    tf_f32x4 s = spb[kTtWaves * 64 + lane];
#pragma unroll
    for (int w = 0; w < kTtWaves; ++w) s += spb[w * 64 + lane];
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (!((now >> (quad * 4 + v)) & 1u)) s[v] = -INFINITY;
    float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    mx = max_of_quads(mx);
    const float m_new = fmaxf(m, mx);
    const float m_sub = m_new == -INFINITY ? 0.f : m_new;  // nothing seen yet: weights and sum stay 0
    const float alpha = exp2f(m - m_sub);                  // m = -inf on the first tile gives 0
    tf_f32x4 p;
#pragma unroll
    for (int v = 0; v < 4; ++v) p[v] = exp2f(s[v] - m_sub);
    l = l * alpha + ((p[0] + p[1]) + (p[2] + p[3]));       // (of this lane's tokens)
    m = m_new;
    now = sees;
    if (tile + 2 * n_splits < n_tiles) {
      aim((tile + 2 * n_splits) * kTtTok, page);
      page = page_at(tile + 3 * n_splits);
    }
    if (SEP && !does_v) continue;
    if (__any(alpha != 1.f)) {
#pragma unroll
      for (int i = 0; i < CPW; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] *= alpha;
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      vec a[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) a[v] = *reinterpret_cast<const vec*>(cs + (quad * 4 + v) * CS + g * 16 * GW + GW * i16);
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int e = 0; e < GW; ++e)
          acc[g * GW + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[v][e], p[v], acc[g * GW + e], 0, 0, 0);
    }
  }

  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  if (head >= n_h) return;
  if (wave == 0 && quad == 0) {
    part_m[pi] = m;
    part_l[pi] = l;
  }
  if (l == 0.f || !does_v) return;                         // nothing seen: the merge does not read the accumulators
  float* u_row = part_u + pi * d_u - v_blk0 * 16;
#pragma unroll
  for (int g = 0; g < GROUPS; ++g)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int col = win * 16 + g * 16 * GW + GW * (quad * 4 + v);
      vec o;
#pragma unroll
      for (int e = 0; e < GW; ++e) o[e] = acc[g * GW + e][v];
      if (col >= max(blk0, v_blk0) * 16) *reinterpret_cast<vec*>(u_row + col) = o;
    }
}

template <typename T, int CPW, bool SEP>
static hipError_t launch_seen(const DecodeArgs& a, const DecodePlan& p, const float* qe, const float* qt, float* pm, float* pl, float* pu,
                              hipStream_t stream) {
  static LdsLimit limit;
  const elitekv_dims& d = a.dims;
  const size_t lds = sizeof(float) * (size_t)(kTtWaves * kTtTok * (CPW * 16 + 4) + 2 * (kTtWaves + 1) * 256 + 32 * d.r);
  const hipError_t e = raise_lds_limit(limit, (const void*)attn_seen_tiled_kernel<T, CPW, SEP>, lds);
  if (e != hipSuccess) return e;
  const int readers = a.q_per_seq * ((d.n_heads + 15) / 16), all = (int)(p.n_splits * (a.B / a.q_per_seq) * readers);
  const int run = reader_run(readers, all), turns = reader_turns(all, run);
  const int grid = 8 * (turns * run + (all - turns * 8 * run + 7) / 8);
  attn_seen_tiled_kernel<T, CPW, SEP><<<grid, kTtWaves * 64, lds, stream>>>(
      (const T*)a.ke_plane, (const T*)a.c_plane, qe, qt, a.seq_len, pm, pl, pu, d.n_heads, 2 * d.r, d.d_c, p.d_q, p.d_u,
      a.max_seq_len, a.batch_stride_rows, a.plane_rows, p.n_splits, a.q_per_seq, (int)a.B, run, turns, a.map);
  return hipGetLastError();
}
template <typename T>
static hipError_t launch_seen_t(const DecodeArgs& a, const DecodePlan& p, const float* qe, const float* qt, float* pm, float* pl, float* pu,
                                hipStream_t stream) {
  const bool sep = p.d_q != a.dims.d_c;
  const int cpw = (a.dims.d_c / 16 + kTtWaves - 1) / kTtWaves;       // (of every size taken there are CPW blocks at least)
#define EKV_SEEN(C) \
  if (cpw <= C) return sep ? launch_seen<T, C, true>(a, p, qe, qt, pm, pl, pu, stream) : launch_seen<T, C, false>(a, p, qe, qt, pm, pl, pu, stream);
  EKV_SEEN(1) EKV_SEEN(2) EKV_SEEN(4) EKV_SEEN(6) EKV_SEEN(8) EKV_SEEN(12) EKV_SEEN(16)
#undef EKV_SEEN
  return hipErrorInvalidValue;
}
hipError_t launch_attn_seen_tiled(const DecodeArgs& a, const DecodePlan& p, const float* qe, const float* qt, float* pm, float* pl,
                                  float* pu, hipStream_t stream) {
  return a.dims.dtype == ELITEKV_FP32 ? launch_seen_t<float>(a, p, qe, qt, pm, pl, pu, stream)
                                      : launch_seen_t<bf16_t>(a, p, qe, qt, pm, pl, pu, stream);
}

// ---- query preparation of many rows ----
// qt[b, k] = sum_j W_uk[k, h, j] q_ne[b, j]  on the fp32 matrix cores: work-group = (64 latent columns, head, 32 rows), a wave's 16 rows of
// W_uk as the A operand, all of them in flight at once; four consecutive j of a lane are those of four products, so both operands are 16
// bytes a lane.  W_uk is read once per 32 rows (qprep_tiled_kernel: per 4).  KS: contraction steps of 16.  Bound by the bytes of W_uk and
// the trips in front of the products (elite indices, queries): 24 rows, 7B 25 %, 22 MB: 12.4 us (qprep_tiled_kernel 21.4).
constexpr int kTqRows = 32;

template <typename T, int KS>
__global__ __launch_bounds__(256) void qprep_many_tiled_kernel(const T* __restrict__ q, const int32_t* __restrict__ q_pos,
                                                               const T* __restrict__ W_uk, const int32_t* __restrict__ elite_idx,
                                                               float* __restrict__ qe, float* __restrict__ qt, int B, int n_h, int d_h, int r,
                                                               int d_q, const RopeTable rope, float scale_log2e) {
  constexpr int QS = KS * 16 + 4;
  __shared__ __align__(16) float q_ne[kTqRows][QS];
  __shared__ unsigned long long elite[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i16 = lane & 15, quad = lane >> 4;
  const int nd = d_h - 2 * r, half = d_h / 2;
  const int h = blockIdx.y, b0 = blockIdx.z * kTqRows, k0 = blockIdx.x * 64 + wave * 16;

  const T* w = W_uk + ((int64_t)min(k0 + i16, d_q - 1) * n_h + h) * nd;
  tf_f32x4 wv[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) wv[s] = ld4(w + min(4 * s + quad, nd / 4 - 1) * 4);

  if (tid < 2) elite[tid] = 0ull;
  for (int e = tid; e < kTqRows * QS; e += 256) (&q_ne[0][0])[e] = 0.f;
  __syncthreads();
  for (int j = tid; j < r; j += 256) {
    const int i = elite_idx[h * r + j];
    if (i >= 0 && i < half) atomicOr(&elite[i >> 6], 1ull << (i & 63));
  }
  __syncthreads();
  // a thread takes chunk i of every `per`th row; the non-elite chunks keep their order
  const int per = 256 / half, i = tid % half, row = tid / half;
  const unsigned long long e0 = elite[0], e1 = elite[1], below = (1ull << (i & 63)) - 1ull;
  const int before = i < 64 ? __popcll(~e0 & below) : __popcll(~e0) + __popcll(~e1 & below);
  if (row < per && !(((i < 64 ? e0 : e1) >> (i & 63)) & 1ull) && 2 * before + 1 < nd) {   // (not so only with repeated indices)
#pragma unroll 8
    for (int bt = row; bt < kTqRows; bt += per) {
      const T* qrow = q + ((int64_t)min(b0 + bt, B - 1) * n_h + h) * d_h;
      q_ne[bt][2 * before] = ld(qrow, 2 * i) * scale_log2e;
      q_ne[bt][2 * before + 1] = ld(qrow, 2 * i + 1) * scale_log2e;
    }
  }
  if (blockIdx.x == 0) {
    for (int e = tid; e < kTqRows * r; e += 256) {
      const int b = b0 + e / r, j = e % r;
      if (b >= B) continue;
      const int c = min(max(elite_idx[h * r + j], 0), half - 1);
      float sn, cs;
      rope_sincos(q_pos[b], rope.theta[c], &sn, &cs);
      const T* qrow = q + ((int64_t)b * n_h + h) * d_h;
      const float u = ld(qrow, 2 * c), v = ld(qrow, 2 * c + 1);
      float* o = qe + ((int64_t)b * n_h + h) * 2 * r;
      o[2 * j] = (u * cs - v * sn) * scale_log2e;
      o[2 * j + 1] = (u * sn + v * cs) * scale_log2e;
    }
  }
  __syncthreads();
  tf_f32x4 acc[2] = {(tf_f32x4)(0.f), (tf_f32x4)(0.f)};
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const bool in = 4 * s + quad < nd / 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const tf_f32x4 qv = ld4(&q_ne[16 * t + i16][16 * s + 4 * quad]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(in ? wv[s][e] : 0.f, qv[e], acc[t], 0, 0, 0);
    }
  }
  // D[k, b]: this lane holds row i16 and latent columns 4 quad .. 4 quad + 3
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int b = b0 + 16 * t + i16;
    if (b < B && k0 < d_q) *reinterpret_cast<tf_f32x4*>(qt + ((int64_t)b * n_h + h) * d_q + k0 + 4 * quad) = acc[t];
  }
}

template <typename T, int KS>
static hipError_t launch_qprep_many(const DecodeArgs& a, const DecodePlan& p, float* qe, float* qt, hipStream_t stream) {
  const elitekv_dims& d = a.dims;
  const dim3 grid((p.d_q + 63) / 64, d.n_heads, (unsigned)((a.B + kTqRows - 1) / kTqRows));
  qprep_many_tiled_kernel<T, KS><<<grid, 256, 0, stream>>>((const T*)a.q, a.q_pos, (const T*)a.W_uk, a.elite_idx, qe, qt, (int)a.B, d.n_heads,
                                                           d.head_dim, d.r, p.d_q, rope_table(d.rope_base, d.head_dim),
                                                           kLog2e / sqrtf((float)d.head_dim));
  return hipGetLastError();
}
hipError_t launch_qprep_many_tiled(const DecodeArgs& a, const DecodePlan& p, float* qe, float* qt, hipStream_t stream) {
  const bool narrow = a.dims.head_dim - 2 * a.dims.r <= 128;
  if (a.dims.dtype == ELITEKV_FP32) return narrow ? launch_qprep_many<float, 8>(a, p, qe, qt, stream) : launch_qprep_many<float, 16>(a, p, qe, qt, stream);
  return narrow ? launch_qprep_many<bf16_t, 8>(a, p, qe, qt, stream) : launch_qprep_many<bf16_t, 16>(a, p, qe, qt, stream);
}

// ---- up-projection of many rows ----
// out[b, j] = sum_k ubar[b, k] W_uv[k, h, j]: work-group (16 waves) = (32 output columns of a head, 16 rows), the waves share out the
// contraction in steps of 16 and their sums meet in LDS.  A lane's two columns of a row of W_uv are the A operands of two products (columns
// 2 i and 2 i + 1), its four consecutive latents of a row of ubar the B operands of four steps.  W_uv is read once per 16 rows
// (upproj_tiled_kernel: per 4).  24 rows, 7B 25 %, 25 MB: 11.4 us (upproj_tiled_kernel 22.7).
constexpr int kTuRows = 16, kTuWaves = 16, kTuRed = kTuCols + 4;

__device__ __forceinline__ float2 ld2(const float* p) { return *reinterpret_cast<const float2*>(p); }
__device__ __forceinline__ float2 ld2(const bf16_t* p) {
  const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

template <typename T>
__global__ __launch_bounds__(kTuWaves * 64) void upproj_many_tiled_kernel(const float* __restrict__ ubar, int ubar_rows,
                                                                          const T* __restrict__ W_uv, T* __restrict__ out, int B, int n_h,
                                                                          int d_h, int d_u) {
  __shared__ __align__(16) float red[kTuWaves][kTuRows][kTuRed];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i16 = lane & 15, quad = lane >> 4;
  const int h = blockIdx.y, j0 = blockIdx.x * kTuCols, b0 = blockIdx.z * kTuRows;
  const float* u = ubar + ((int64_t)min(b0 + i16, B - 1) * ubar_rows * n_h + h) * d_u + 4 * quad;
  const T* w = W_uv + ((int64_t)4 * quad * n_h + h) * d_h + j0 + 2 * i16;
  const int64_t w_row = (int64_t)n_h * d_h;
  tf_f32x4 acc[2] = {(tf_f32x4)(0.f), (tf_f32x4)(0.f)};
  constexpr int AHEAD = 6;                                 // steps of a wave whose operands are requested together
  const int steps = d_u / 16;
  for (int g0 = wave; g0 < steps; g0 += AHEAD * kTuWaves) {
    tf_f32x4 uv[AHEAD];
    float2 wv[AHEAD][4];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int g = min(g0 + i * kTuWaves, steps - 1);
      uv[i] = ld4(u + 16 * g);
#pragma unroll
      for (int v = 0; v < 4; ++v) wv[i][v] = ld2(w + (16 * g + v) * w_row);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (g0 + i * kTuWaves < steps) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          acc[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[i][v].x, uv[i][v], acc[0], 0, 0, 0);
          acc[1] = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[i][v].y, uv[i][v], acc[1], 0, 0, 0);
        }
      }
  }
  // D[j, b]: this lane holds row i16 and columns 2 (4 quad + v) + {0, 1}
#pragma unroll
  for (int v = 0; v < 4; ++v) *reinterpret_cast<float2*>(&red[wave][i16][8 * quad + 2 * v]) = make_float2(acc[0][v], acc[1][v]);
  __syncthreads();
  if (tid >= kTuRows * kTuCols) return;
  const int row = tid / kTuCols, col = tid % kTuCols;
  if (b0 + row >= B) return;
  float a = 0.f;
#pragma unroll
  for (int g = 0; g < kTuWaves; ++g) a += red[g][row][col];
  st(out, ((int64_t)(b0 + row) * n_h + h) * d_h + j0 + col, a);
}

template <typename T>
static hipError_t launch_upproj_many(const DecodeArgs& a, const DecodePlan& p, const float* ubar, hipStream_t stream) {
  const elitekv_dims& d = a.dims;
  const dim3 grid(d.head_dim / kTuCols, d.n_heads, (unsigned)((a.B + kTuRows - 1) / kTuRows));
  upproj_many_tiled_kernel<T><<<grid, kTuWaves * 64, 0, stream>>>(ubar, p.ubar_rows, (const T*)a.W_uv, (T*)a.out, (int)a.B, d.n_heads,
                                                                 d.head_dim, p.d_u);
  return hipGetLastError();
}
hipError_t launch_upproj_many_tiled(const DecodeArgs& a, const DecodePlan& p, const float* ubar, hipStream_t stream) {
  return a.dims.dtype == ELITEKV_FP32 ? launch_upproj_many<float>(a, p, ubar, stream) : launch_upproj_many<bf16_t>(a, p, ubar, stream);
}

}  // namespace ekv
