// The bf16 attention of many queries that share their rows (trees of drafted tokens, drafted chains over pages), two queries a work-group.
//
// Work-group (four waves, one per SIMD) = (split, two queries of a sequence, 32 heads); per step a tile of 32 cached rows, of which every
// wave has its quarter of the latent columns and eight heads' elite keys in LDS:
//   scores   D[token, head] = C Q^T + K_e Q_e^T     32x32x16 MFMA, A = the tile's rows, B = a query (registers).  The elite keys differ from
//            head to head: they are more columns of the tile, and the elite query has zeros there for the other heads.
//   softmax  the waves' parts are added, in their order, by the wave that has a query's 16 heads; a lane has eight tokens of a head
//   values   U[column, head] += C^T P^T             the same tile read transposed, B = the probabilities of one query and of the other
// An operand from LDS serves both queries, and the chain scores -> sum -> maximum -> probabilities -> values, which bounds the kernel of one
// query and sixteen rows (decode_mfma_kernel.hpp), is passed a quarter as often.  The accumulators of two queries and the queries fill the
// registers (768 columns: 192 + 104 of 512), so there is one wave per SIMD, rows come through registers (requested between the score
// products, stored between the value products), and wider latents are left to the other kernel.
//
// Rounded to bf16, as there: the absorbed query, the probabilities (their sums are fp32) and a split's accumulators on their way out; here
// the rotated elite query too.  Products of the elite columns of other heads are zeros times their keys: a row that holds an infinity or
// NaN in one head's elite key has none but NaN scores in the heads of the same wave, for the queries that see it.
//
// 8 trees of 64 nodes behind 2048 to 512 tokens, 7B 12.5 %: 167 us, 460 TFLOP/s (one query a work-group: 192); a step takes 2.5 us: 0.75
// of products, the rest the chain and a wave's own instructions, 320 vector ones a step, with no second wave to fill in.  With the rows
// requested ahead of all products and stored behind them 200; with exp2f, which also takes care of denormals, 179.  3 trees of 26 behind
// 5001 to 2833 tokens, latents of 768 + 768: 104 us, 300 TFLOP/s (one query a work-group 193).
#include "decode_mfma_kernel.hpp"

namespace ekv {

// LDS: every wave's slice of a tile [32 tokens][DC_W latent columns | 8 heads' elite keys], rows an odd multiple of 32 bytes apart (eight
// rows at one column, and the four rows of 32 bytes of a transposed read, lie in different banks); the score parts, the probabilities
template <int DC_W, int TWO_R>
struct PairsLayout {
  static constexpr int ROW = DC_W * 2 + 16 * TWO_R, RS = ROW / 32 % 2 ? ROW : ROW + 32;
  static constexpr int SLICE = 32 * RS;                     // one wave's
  static constexpr int X = 4 * SLICE, P = X + 4 * 4 * 8 * 256, ALPHA = P + 2 * 4 * 32 * 16, RAISED = ALPHA + 2 * 32 * 4;
  static constexpr int BYTES = RAISED + 16;
  static constexpr int TSTR = DC_W * 2 + 16;                // head rows of the result on its way out, in the wave's slice
  static_assert(32 * TSTR <= SLICE && BYTES <= 160 * 1024 && DC_W % 64 == 0, "");
};

// SEP: separated latents of two halves.  A wave has a quarter of the key latents' columns and one of the value latents', which take the
// former's place in LDS behind the score products: value latents are on their way during the scores, the next tile's key latents and elite
// keys from there on.
template <int DC_W, int TWO_R, bool SEP>
__global__ __launch_bounds__(256, 1) void attn_pairs_kernel(const AttnMfmaMappedParams p) {
  using L = PairsLayout<DC_W, TWO_R>;
  constexpr int KS = DC_W / 16, ES = TWO_R / 2, CT = DC_W / 32, CB = DC_W / 64;
  constexpr int KL = TWO_R / 2;                             // loads of elite keys (8 heads, 32 tokens)
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hi = lane >> 5, i16 = lane & 15, q16 = lane >> 4;

  const int pairs = (p.q_per_seq + 1) / 2, readers = pairs * p.head_groups, seqs = p.batch / p.q_per_seq;
  const int place = reader_place(blockIdx.x, p.n_splits * seqs * readers, p.reader_run, p.reader_turns);
  if (place < 0) return;
  const int item = place / readers, reader = place % readers;
  const int split = __builtin_amdgcn_readfirstlane(item % p.n_splits), seq = __builtin_amdgcn_readfirstlane(item / p.n_splits);
  const int hg = __builtin_amdgcn_readfirstlane(reader % p.head_groups);
  const int t0 = __builtin_amdgcn_readfirstlane(reader / p.head_groups * 2);
  const int ba = seq * p.q_per_seq + t0;
  const bool two = t0 + 1 < p.q_per_seq;
  const int bb = two ? ba + 1 : ba;
  if (split == 0 && hg == 0) {
    for (int h = tid; h < p.n_h; h += 256) {
      p.chunk_counters[(int64_t)ba * p.n_h + h] = 0;
      p.chunk_counters[(int64_t)bb * p.n_h + h] = 0;
    }
  }

  // the absorbed queries of this wave's columns (B operands: lane <-> head n, eight columns from 8 hi on), the elite ones in bf16
  const int head = min(hg * 32 + n, p.n_h - 1);            // heads past the last repeat it and are not stored
  bf16x8 qa[KS], qb[KS], ea, eb;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const int k = wave * DC_W + ks * 16 + hi * 8;
    qa[ks] = *reinterpret_cast<const bf16x8*>(p.qt + qt_packed_index(ba, head, k, p.head_groups, p.d_q, p.q_slice));
    qb[ks] = *reinterpret_cast<const bf16x8*>(p.qt + qt_packed_index(bb, head, k, p.head_groups, p.d_q, p.q_slice));
  }
  {
    const int at = TWO_R == 8 ? 0 : hi * 8;
    const float* fa = p.qe + ((int64_t)ba * p.n_h + head) * TWO_R + at;
    const float* fb = p.qe + ((int64_t)bb * p.n_h + head) * TWO_R + at;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      ea[j] = (__bf16)fa[j];
      eb[j] = (__bf16)fb[j];
    }
  }

  const int64_t row0 = (int64_t)seq * p.batch_stride_rows;
  const int64_t cap = min(p.max_seq_len, rows_left(p, row0));
  const SeenRows sa = rows_seen(p, ba, cap), sb = rows_seen(p, bb, cap);
  const int len_b = two ? sb.len : 0, len = max(sa.len, len_b);

  // Tiles of 32 rows that both queries see alike are taken for both at once.  A tile that they see differently is taken for each alone,
  // behind all of the others, so that a row which one of them does not see is never multiplied for it.  (Three loops, and not branches in
  // one: around those the compiler copies the accumulators.)
  auto bits = [](const SeenRows& s, int end, int j) {
    uint32_t v = j < end ? s.tile(j) : 0u;
    if (j + 16 < end) v |= s.tile(j + 16) << 16;
    return v;
  };
  struct Step { int j; uint32_t u; int page0, page1; };     // j < 0: none; u: the rows that are seen; the pages of its halves
  const int tiles = (len + 31) >> 5;
  const int same = sa.len == 0 || len_b == 0 ? 0 : (sa.mask ? sa.prefix : min(sa.len, len_b)) >> 5;      // tiles that both see whole
  int at = 0;
  auto step_at = [&](int j, uint32_t u) { return Step{j, u, sa.page(u & 0xffffu ? j : j + 16), sa.page(u >> 16 ? j + 16 : j)}; };
  auto next = [&](auto with_a, auto with_b) {
    constexpr bool A = decltype(with_a)::value, B = decltype(with_b)::value;
    if (A && B && at < same) {
      const int j = at * 32;
      at += p.n_splits;
      return step_at(j, 0xffffffffu);
    }
    for (; at < tiles; at += p.n_splits) {
      const uint32_t a = bits(sa, sa.len, at * 32), b = bits(sb, len_b, at * 32);
      if (A && B ? a == b && a : A ? a && a != b : b && a != b) {
        const int j = at * 32;
        at += p.n_splits;
        return step_at(j, A ? a : b);
      }
    }
    return Step{-1, 0, 0, 0};
  };

  // A step's rows, on their way through registers into the wave's slice.  An unseen row's lanes load the last seen one of its half of the
  // tile, or of the other half.
  constexpr int NL = 4 * CB + KL;
  static_assert(NL == KS + ES, "a piece behind every score product");
  u32x4 stage[NL];
  const int64_t crow = (int64_t)p.d_c * 2, krow = (int64_t)p.n_h * TWO_R * 2;
  const char* cbase = reinterpret_cast<const char*>(p.c_plane) + wave * DC_W * 2;
  const int64_t v_off = SEP ? (int64_t)p.d_q * 2 : 0;       // bytes from the key latents of a row to its value latents
  const char* kbase = reinterpret_cast<const char*>(p.ke_plane);
  // 16-byte piece of the eight heads' keys that this lane loads
  const uint32_t kpiece = lane & (TWO_R - 1);
  const uint32_t kcol = TWO_R == 8 ? (uint32_t)min(hg * 32 + wave * 8 + (int)kpiece, p.n_h - 1) * 16
                                   : (uint32_t)(min(hg * 32 + wave * 8 + (int)(kpiece >> 1), p.n_h - 1) * 2 + (kpiece & 1)) * 16;
  const char *c0 = cbase, *c1 = cbase, *k0 = kbase, *k1 = kbase;      // the halves' rows
  uint32_t rows[4], seen_u = 0, e0 = 0, e1 = 0;             // of this lane: row of its half, for the pieces of 8 rows each
  auto row_of = [&](int r) {                                // r < 32: its row, or the one that stands for it
    const uint32_t h = r & 15;
    return (seen_u >> r) & 1u ? h : r < 16 ? e0 : e1;
  };
  auto aim = [&](const Step& s) {
    const uint32_t u0 = s.u & 0xffffu, u1 = s.u >> 16;
    const int64_t b0 = sa.row(u0 ? s.j : s.j + 16, s.page0), b1 = sa.row(u1 ? s.j + 16 : s.j, s.page1);
    seen_u = s.u;
    e0 = 31 - __builtin_clz(u0 ? u0 : u1); e1 = 31 - __builtin_clz(u1 ? u1 : u0);
    c0 = cbase + b0 * crow; c1 = cbase + b1 * crow; k0 = kbase + b0 * krow; k1 = kbase + b1 * krow;
#pragma unroll
    for (int rg = 0; rg < 4; ++rg) rows[rg] = s.u == 0xffffffffu ? (uint32_t)((rg & 1) * 8 + (lane >> 3)) : row_of(rg * 8 + (lane >> 3));
  };
  // piece i of a step: the elite keys' first, then the column blocks, four pieces of eight rows each
  auto fetch = [&](int i, int64_t off = 0) {
    if (i < KL) {
      constexpr int RPL = 64 / TWO_R;                       // rows of a piece
      const uint32_t r = TWO_R == 8 ? rows[i & 3] : row_of(i * RPL + lane / TWO_R);
      stage[i] = *reinterpret_cast<const u32x4*>((i * RPL < 16 ? k0 : k1) + r * (uint32_t)krow + kcol);
    } else {
      const int cb = (i - KL) >> 2, rg = (i - KL) & 3;
      stage[i] = *reinterpret_cast<const u32x4*>((rg < 2 ? c0 : c1) + off + cb * 128 + (rows[rg] * (uint32_t)crow + (lane & 7) * 16));
    }
  };
  char* slice = smem + wave * L::SLICE;
  auto settle = [&](int i) {
    if (i < KL) {
      *reinterpret_cast<u32x4*>(slice + (i * (64 / TWO_R) + lane / TWO_R) * L::RS + DC_W * 2 + kpiece * 16) = stage[i];
    } else {
      const int cb = (i - KL) >> 2, rg = (i - KL) & 3;
      *reinterpret_cast<u32x4*>(slice + (rg * 8 + (lane >> 3)) * L::RS + cb * 128 + (lane & 7) * 16) = stage[i];
    }
  };

  f32x16 ua[CT], ub[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) { ua[ct] = (f32x16)(0.f); ub[ct] = (f32x16)(0.f); }
  // of the rows this wave finalises: query wave / 2, heads 16 (wave & 1) + i16; a lane has tokens 8 q16 .. 8 q16 + 7
  float m_run = -INFINITY, l_run = 0.f;
  float* alphas = reinterpret_cast<float*>(smem + L::ALPHA);
  int* raised = reinterpret_cast<int*>(smem + L::RAISED);

  // the accumulators, and one query, stay in the accumulation registers
  auto pin = [&]() {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) asm volatile("" : "+a"(ua[ct]), "+a"(ub[ct]));
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+a"(qb[ks]));
  };
  auto compute = [&](const Step& s, auto with_a, auto with_b) {
    constexpr bool A = decltype(with_a)::value, B = decltype(with_b)::value;
    pin();
    // ---- this wave's part of the scores: D[token, head]
    f32x16 da = (f32x16)(0.f), db = (f32x16)(0.f);
    const char* arow = slice + n * L::RS + hi * 16;
    int own_n = n;                                           // (formed anew every time: the selected queries do not stay in registers)
    asm volatile("" : "+v"(own_n));
    {
      constexpr int LOOK = 3;                                // operands read ahead: more of them would push the accumulators out
      bf16x8 c[LOOK];
#pragma unroll
      for (int ks = 0; ks < LOOK; ++ks) c[ks] = *reinterpret_cast<const bf16x8*>(arow + ks * 32);
#pragma unroll
      for (int ks = 0; ks < KS + ES; ++ks) {
        bf16x8 fa, fb;
        if (ks < KS) {
          fa = qa[ks < KS ? ks : 0];
          fb = qb[ks < KS ? ks : 0];
        } else {
          // elite keys: column j of the step is a dim of one head, and only that head's query has it
          const bool own = own_n == 8 * wave + (TWO_R == 8 ? 2 * (ks - KS) + hi : ks - KS);
          const bf16x8 none = (bf16x8)((__bf16)0.f);
          fa = own ? ea : none;
          fb = own ? eb : none;
        }
        if constexpr (A) da = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[ks % LOOK], fa, da, 0, 0, 0);
        if constexpr (B) db = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[ks % LOOK], fb, db, 0, 0, 0);
        if (ks + LOOK < KS + ES) c[ks % LOOK] = *reinterpret_cast<const bf16x8*>(arow + (ks + LOOK) * 32);
        if constexpr (!SEP) fetch(ks);                       // (as many pieces as products)
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    auto part = [&](const f32x16& d, int q) {
      char* x = smem + L::X + (((2 * q + (n >> 4)) * 4 + wave) * 8 + hi) * 256 + i16 * 16;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = d[4 * g + e];
        *reinterpret_cast<f32x4*>(x + g * 512) = v;
      }
    };
    if constexpr (A) part(da, 0);
    if constexpr (B) part(db, 1);
    if constexpr (SEP) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        if (i >= KL) settle(i);                              // the value latents (the key latents have been read)
        fetch(i);
      }
    }
    __syncthreads();

    // ---- the rows of this wave: sum of the parts, maximum, probabilities
    const uint32_t mine = s.u;
    if (wave < 2 ? A : B) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const char* x = smem + L::X + ((wave * 4 + w) * 8 + 2 * q16) * 256 + i16 * 16;
        const f32x4 lo = *reinterpret_cast<const f32x4*>(x), up = *reinterpret_cast<const f32x4*>(x + 256);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] += lo[e]; v[4 + e] += up[e]; }
      }
      float mx = -INFINITY;
      if (mine != 0xffffffffu) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!((mine >> (8 * q16 + e)) & 1u)) v[e] = -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) mx = fmaxf(mx, v[e]);
      mx = max_of_quads(mx);
      const float m_new = mx > m_run + kRescaleSlack ? mx : m_run;
      const float m_sub = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = m_new != m_run ? exp2f(m_run - m_sub) : 1.f;
      m_run = m_new;
      float sum = 0.f;
      bf16x8 pr;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = __builtin_amdgcn_exp2f(v[e] - m_sub);   // (below 2^-126: 0)
        sum += x;
        pr[e] = (__bf16)x;
      }
      l_run = l_run * alpha + sum;
      const int q = wave >> 1, h = 16 * (wave & 1) + i16;
      *reinterpret_cast<bf16x8*>(smem + L::P + ((q * 4 + q16) * 32 + h) * 16) = pr;
      const bool up = __any(alpha != 1.f);
      if (up && q16 == 0) alphas[q * 32 + h] = alpha;
      if (lane == 0) raised[wave] = up;
    }
    __syncthreads();

    pin();
    // ---- values: U[column, head] += C^T P^T, the tile read transposed
    auto rescale = [&](f32x16 (&u)[CT], int q) {
      const int any = __builtin_amdgcn_readfirstlane(raised[2 * q] | raised[2 * q + 1] << 1);
      if (any) {
        const float al = (any >> (n >> 4)) & 1 ? alphas[q * 32 + n] : 1.f;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            float y, z;
            asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(y) : "a"(u[ct][j]));
            y *= al;
            asm volatile("v_accvgpr_write_b32 %0, %1\n\ts_nop 2" : "=a"(z) : "v"(y));   // + wait states before an MFMA reads it
            u[ct][j] = z;
          }
      }
    };
    if constexpr (A) rescale(ua, 0);
    if constexpr (B) rescale(ub, 1);
    const char* tr = slice + (8 * hi + (i16 >> 2)) * L::RS + (16 * (q16 & 1) + 4 * (i16 & 3)) * 2;
    auto columns = [&](int i) {                              // block i / 2, tokens 16 (i % 2) ..
      const char* at = tr + 16 * (i & 1) * L::RS + (i >> 1) * 64;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)at);
      const s16x4 up = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at + 4 * L::RS));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto weights = [&](int q, int h) { return *reinterpret_cast<const bf16x8*>(smem + L::P + ((4 * q + 2 * h + hi) * 32 + n) * 16); };
    bf16x8 pa[2], pb[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (A) pa[h] = weights(0, h);
      if constexpr (B) pb[h] = weights(1, h);
    }
    constexpr int LOOK = 3;
    bf16x8 c[LOOK];
#pragma unroll
    for (int i = 0; i < LOOK; ++i) c[i] = columns(i);
#pragma unroll
    for (int i = 0; i < 2 * CT; ++i) {
      if constexpr (A) ua[i >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[i % LOOK], pa[i & 1], ua[i >> 1], 0, 0, 0);
      if constexpr (B) ub[i >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[i % LOOK], pb[i & 1], ub[i >> 1], 0, 0, 0);
      if (i + LOOK < 2 * CT) c[i % LOOK] = columns(i + LOOK);
      if (i == 0) {
#pragma unroll
        for (int k = 0; k < KL; ++k) settle(k);
      }
      if ((i & 3) == 3) {                                    // (the block's columns have been read)
#pragma unroll
        for (int k = 0; k < 4; ++k) settle(KL + (i >> 2) * 4 + k);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (SEP) {
#pragma unroll
      for (int i = KL; i < NL; ++i) fetch(i, v_off);
    }
    pin();
  };

  // A step's rows are requested between the score products of the step before it, and take its rows' place in LDS between the value
  // products (behind the last step: the last rows again).
  auto run = [&](int from, auto with_a, auto with_b) {
    at = from;
    Step cur = next(with_a, with_b);
    if (cur.j < 0) return;
    aim(cur);
#pragma unroll
    for (int i = 0; i < NL; ++i) fetch(i);
#pragma unroll
    for (int i = 0; i < NL; ++i) settle(i);
    if constexpr (SEP) {
#pragma unroll
      for (int i = KL; i < NL; ++i) fetch(i, v_off);
    }
    while (cur.j >= 0) {
      const Step ahead = next(with_a, with_b);
      if (ahead.j >= 0) aim(ahead);
      compute(cur, with_a, with_b);
      cur = ahead;
    }
  };
  run(split, std::true_type{}, std::true_type{});
  // (the first tile of this split that the two may see differently)
  const int tail = same <= split ? split : split + (same - split + p.n_splits - 1) / p.n_splits * p.n_splits;
  run(tail, std::true_type{}, std::false_type{});
  run(tail, std::false_type{}, std::true_type{});

  // ---- the split's partials: maxima and sums, and the accumulators head-major in bf16, transposed through the wave's slice
  l_run += __shfl_xor(l_run, 16, kWave);
  l_run += __shfl_xor(l_run, 32, kWave);
  const int64_t slots = (int64_t)p.head_groups * 32;
  const int64_t ia = ((int64_t)ba * p.n_part + split) * slots + hg * 32, ib = ((int64_t)bb * p.n_part + split) * slots + hg * 32;
  if (q16 == 0 && (wave < 2 || two)) {
    const int h = 16 * (wave & 1) + i16;
    const int64_t i = (wave < 2 ? ia : ib) + h;
    p.part_m[i] = m_run;
    p.part_l[i] = hg * 32 + h < p.n_h ? l_run : 0.f;
  }
  auto store = [&](const f32x16 (&u)[CT], int64_t pi) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint2 pk;
        pk.x = pack_bf16x2(u[ct][4 * g], u[ct][4 * g + 1]);
        pk.y = pack_bf16x2(u[ct][4 * g + 2], u[ct][4 * g + 3]);
        *reinterpret_cast<uint2*>(slice + n * L::TSTR + (ct * 32 + 8 * g + 4 * hi) * 2) = pk;
      }
    constexpr int CPR = DC_W / 8;
    char* base = reinterpret_cast<char*>(p.part_u) + (pi * p.d_u + wave * DC_W) * 2;
#pragma unroll
    for (int i = 0; i < 32 * CPR / 64; ++i) {
      const int idx = i * 64 + lane, row = idx / CPR, ch = idx % CPR;
      const u32x4 v = *reinterpret_cast<const u32x4*>(slice + row * L::TSTR + ch * 16);
      if (hg * 32 + row < p.n_h) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(base + (int64_t)row * p.d_u * 2 + ch * 16));
    }
  };
  store(ua, ia);
  if (two) store(ub, ib);
}

template <int DC_W, int TWO_R, bool SEP>
static hipError_t launch_pairs(AttnMfmaMappedParams& prm, hipStream_t stream) {
  using L = PairsLayout<DC_W, TWO_R>;
  static LdsLimit limit;
  const hipError_t e = raise_lds_limit(limit, reinterpret_cast<const void*>(&attn_pairs_kernel<DC_W, TWO_R, SEP>), L::BYTES);
  if (e != hipSuccess) return e;
  const int readers = (prm.q_per_seq + 1) / 2 * prm.head_groups, all = prm.n_splits * (prm.batch / prm.q_per_seq) * readers;
  prm.reader_run = reader_run(readers, all);
  prm.reader_turns = reader_turns(all, prm.reader_run);
  const int grid = 8 * (prm.reader_turns * prm.reader_run + (all - prm.reader_turns * 8 * prm.reader_run + 7) / 8);
  attn_pairs_kernel<DC_W, TWO_R, SEP><<<grid, 256, L::BYTES, stream>>>(prm);
  return hipGetLastError();
}

// groups: (pair of queries, group of 32 heads) of all sequences.  A work-group's start, two queries' with one wave per SIMD, takes 7 us more
// than one query's, so there have to be enough tiles a compute unit: four where the kernel of one query has a compute unit to itself, eight
// where two of its work-groups share one.  Trees or drafted chains, queries x rows (tiles a compute unit), us, one query a work-group / two:
//                      1 x 8 x 6000 (2.9)  2 x 16 x 2000 (3.9)  4 x 5 x 4096 (6)  16 x 4 x 2000 (7.9)  4 x 26 x 2000 (13)  8 x 64 x 2048 (64)
//   768 + 768, r = 8     50.5 / 54.3         60.2 / 58.4          68.2 / 63.4       94.6 / 79.3          142.8 / 94.8        496 / 270
//   512 + 512, r = 8     47.2 / 45.9         54.1 / 47.5          61.7 / 52.2       82.3 / 60.9          128.3 / 75.7        461 / 215
//   768, r = 8           46.0 / 52.1         52.5 / 55.0          58.1 / 58.8       75.4 / 67.8          118.0 / 87.5        394 / 225
//   256 + 256, r = 4     39.7 / 39.2         38.0 / 37.7          40.5 / 40.2       51.5 / 46.5          63.6 / 55.4         203 / 144
//   768, r = 4           43.7 / 50.2         47.5 / 53.5          49.8 / 55.8       64.6 / 65.4          82.2 / 83.0         241 / 209
//   512, r = 8           40.4 / 44.4         42.1 / 45.2          44.9 / 48.6       56.5 / 55.9          70.8 / 69.2         228 / 187
//   256, r = 4           36.5 / 38.5         35.6 / 37.1          37.3 / 39.1       47.1 / 45.6          57.5 / 54.3         177 / 138
bool attn_pairs_pays(const elitekv_dims& d, int d_ck, int64_t groups, int64_t max_seq) {
  const int half = d_ck ? d.d_c - d_ck : d.d_c;
  return decode_mfma_supported(d, d_ck) && (d_ck == 0 || d_ck == half) && (d.r == 4 || d.r == 8) &&
         (half == 768 || half == 512 || half == 256) &&
         groups * ((max_seq + 31) / 32) >= (decode_mfma_groups_per_cu(d) == 1 ? 4 : 8) * 256;
}

hipError_t launch_attn_pairs(const AttnMfmaParams& prm, const DecodeArgs& a, hipStream_t stream) {
  AttnMfmaMappedParams p;
  static_cast<AttnMfmaParams&>(p) = prm;
  p.map = a.map;
  const elitekv_dims& d = a.dims;
#define EKV_PAIRS(W) \
  if (prm.d_u == 4 * W)                                                                                                       \
    return a.d_ck ? (d.r == 4 ? launch_pairs<W, 8, true>(p, stream) : launch_pairs<W, 16, true>(p, stream))                    \
                  : d.r == 4 ? launch_pairs<W, 8, false>(p, stream) : launch_pairs<W, 16, false>(p, stream);
  EKV_PAIRS(64) EKV_PAIRS(128) EKV_PAIRS(192)
#undef EKV_PAIRS
  return hipErrorInvalidValue;
}

}  // namespace ekv
