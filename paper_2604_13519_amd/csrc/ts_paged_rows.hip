// Attention of chunks of rows over a paged cache of any type: causal chunks, windows, draft trees, single tokens.
#include <type_traits>

#include "ts_paged.h"
#include "ts_rows_tiles.h"

// ---------------------------------------------------------------------------------
// The rows of a chunk and the query heads that share a KV head are the columns of one problem: column m of (sequence, KV head) is
// row m / group, head m % group, and all columns go over the same keys and values.  One pass with a running maximum and sum, the
// cache's length split over workgroups and joined where the tiles of columns alone do not fill the card.
//
// This kernel: few columns (single tokens), fp32 rows or pages, a scale of zero.  Tiles of 16 NT columns, four waves that take blocks of 32 keys in
// turn, straight from memory: bound by the bytes of the cache, each read once for a tile.
//
// Matrix instructions without any exchange between lanes: S^T = K Q^T puts 16 columns on the lanes (lane l: column l % 16) and four keys
// of a tile in a lane's registers; O^T = V^T P^T wants eight (fp32: one) consecutive keys of a column in a lane.
// Which key is which row of K's tile is free: row m of tile t takes key 8 (m / 4) + 4 t + m % 4, and the probabilities that a
// lane has computed are, in place, the operand it needs next.  8-bit keys are widened to bf16 times their scales (exact), 8-bit values
// without, their scales go onto the probabilities: eight keys of a lane are eight scales.  In blocks with a scale below 2^-63 or from 2^113 on
// the values are widened times theirs: an infinite one is so whatever its probability, a tiny one costs no bits of it.
//
// Where rows see different keys of a block, probabilities of unseen ones are zero, and zero times an infinite or NaN value
// is not: such blocks are looked through, and values that are not finite are replaced by zeros and counted by indicator products,
// so that they reach the rows that see them and no other.
//
// 8-bit pages, 8 KV heads of 128, 64 query heads: a token for each of 8 sequences up to 32768 (387 MB) 82 us in a kernel trace, 4.7 TB/s.
// 32 query heads over 8, one token over 8192 positions, in a captured graph with its join: bf16 12.5 us (ts_kv_attend 10.6), 8-bit 12.0.
// fp32 pages, 32 query heads over 8 of 128, 300 rows over 4000: 356 us, 57 TFLOP/s of the 157 that fp32 matrix
// instructions have.
// ---------------------------------------------------------------------------------
constexpr int RO_WAVES = 4;
constexpr int RO_CUS = 256, RO_UNIT = 128, RO_MOST = 2;    // RO_MOST: workgroups a CU that a call is split into, at most

struct RowsArgs {
  ts_kv_attend_rows_args a;
  float scale_log2;                      // scores enter 2^x
  int group, chunk, splits;              // query heads per KV head, keys per workgroup, workgroups per tile at most
  int seq_tiles;                         // without offsets: tiles of a sequence's one row
  float* part_o;                         // [n_rows][n_q_heads][splits][head_dim], relative to 2^m
  float* part_ml;                        // [n_rows][n_q_heads][splits][2]
};

// positions [lo, hi) that a row can see (with ancestors: some of them)
__device__ __forceinline__ int2 row_range(const ts_kv_attend_rows_args& a, const RowSeq& s, int row) {
  const int64_t p = s.zero + row, up = a.ancestors ? s.zero + s.end : p + 1;
  const int hi = (int)max((int64_t)0, min((int64_t)s.cap, up));
  const int lo = a.window > 0 ? (int)max((int64_t)0, min((int64_t)hi, p + 1 - a.window)) : 0;
  return make_int2(lo, hi);
}

// whether one of four scales is below 2^-63, or from 2^113 on (NaN too)
__device__ __forceinline__ bool far_scale(uint32_t w) { return (((((w & 0x7f7f7f7fu) + 0x10101010u) & w) | ~(w | w << 1)) & 0x80808080u) != 0; }
__device__ __forceinline__ bool not_finite(uint32_t bf16_pair) {
  return (bf16_pair & 0x7f80u) == 0x7f80u || (bf16_pair & 0x7f800000u) == 0x7f800000u;
}
// 0: +infinity, 1: -infinity, 2: NaN
__device__ __forceinline__ bool of_class(uint32_t f32_bits, int cls) {
  return cls == 0 ? f32_bits == 0x7f800000u : cls == 1 ? f32_bits == 0xff800000u : (f32_bits & 0x7fffffffu) > 0x7f800000u;
}
__device__ __forceinline__ float class_value(int cls) { return __uint_as_float(cls == 0 ? 0x7f800000u : cls == 1 ? 0xff800000u : 0x7fc00000u); }

template <typename T, typename TQ, int HD, int NT>
__global__ __launch_bounds__(RO_WAVES * 64, NT == 1 ? 2 : 1) void k_kv_attend_rows(RowsArgs g) {
  constexpr bool F32 = sizeof(T) == 4, E8 = sizeof(T) == 1;
  constexpr int KB = 32, KT = KB / 16, KL = KB / 4;                            // keys of a block, tiles of them, keys of a lane
  constexpr int QP = !F32 && sizeof(TQ) == 4 ? 3 : 1;                          // terms of a query
  constexpr int PP = !F32 && (sizeof(TQ) == 4 || NT == 1) ? 3 : 1;             // terms of a probability
  constexpr int KC = (HD * (int)sizeof(T) + 63) / 64;                          // 16-byte pieces of a key per lane
  constexpr int QS = F32 ? KC : HD / 32;                                       // steps of the products with a query
  constexpr int DT = (HD + 15) / 16;                                           // tiles of 16 dimensions
  constexpr int TM = 16 * NT, OS = DT * 16 + 4;
  __shared__ float so[RO_WAVES * 16 * OS];
  __shared__ float sm[RO_WAVES][16], sl[RO_WAVES][16];
  __shared__ int2 where[TM];                                  // row and head of a column
  const ts_kv_attend_rows_args& a = g.a;
  const ts_kv_pages& pages = a.cache.pages;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, n = lane % 16, lg = lane / 16;
  int id = blockIdx.x;
  const int hkv = pages.n_kv_heads, kvh = id % hkv; id /= hkv;
  const int split = id % g.splits, t = id / g.splits, G = g.group;
  int m0, cols;
  RowSeq rs;
  const int seq = tile_of<TM, 16>(a, G, g.seq_tiles, t, m0, cols, rs);
  if (seq < 0) return;
  const int row0 = rs.first + m0 / G, rem = m0 % G;
  const int2 low = row_range(a, rs, row0), high = row_range(a, rs, row0 + (rem + cols - 1) / G);
  const int lo = low.x, hi = high.y;                         // what any column sees, and what all do
  const int all_lo = high.x, all_hi = a.ancestors ? min(max(rs.start + 1, 0), low.y) : low.y;
  const int64_t from = ((int64_t)(lo / g.chunk) + split) * g.chunk;
  if (split > 0 && from >= hi) return;
  const int k0 = (int)max(from, (int64_t)(lo & ~(KB - 1))), k1 = (int)min((int64_t)hi, from + g.chunk);

  // columns: lane n of tile j
  int c_lo[NT], c_hi[NT];
  uint64_t c_set[NT];
  ts_u32x4 q[NT][QP][QS];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int m = rem + min(j * 16 + n, cols - 1), row = row0 + m / G, head = kvh * G + m % G;
    if (tid < 16) where[j * 16 + n] = make_int2(row, head);
    const int2 range = row_range(a, rs, row);
    c_lo[j] = range.x; c_hi[j] = range.y;
    c_set[j] = a.ancestors ? a.ancestors[row] : 0;
    const TQ* src = (const TQ*)a.q + (int64_t)row * a.q_stride + (int64_t)head * HD;
#pragma unroll
    for (int c = 0; c < QS; ++c) {
      constexpr int E = F32 ? 4 : 8;
      float x[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = E8 ? (c / 2 * 4 + lg) * 16 + c % 2 * 8 + e : (c * 4 + lg) * E + e;
        x[e] = d < HD ? widen(src[d < HD ? d : 0]) : 0.f;
      }
      if constexpr (!F32) {
        uint32_t u[QP][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          ts_bf16x2 w[QP];
          split_bf16x2_nonzero<QP>(x[2 * e], x[2 * e + 1], w);
#pragma unroll
          for (int p = 0; p < QP; ++p) u[p][e] = __builtin_bit_cast(uint32_t, w[p]);
        }
#pragma unroll
        for (int p = 0; p < QP; ++p) q[j][p][c] = ts_u32x4{u[p][0], u[p][1], u[p][2], u[p][3]};
      } else {
        q[j][0][c] = ts_u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
      }
    }
  }

  ts_f32x4 o[NT][DT];
  float m[NT], l[NT];                                        // l: of this lane's keys only
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    m[j] = -INFINITY; l[j] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[j][d] = ts_f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const TS_CONSTANT int32_t* table = (const TS_CONSTANT int32_t*)(a.table + (int64_t)seq * a.table_stride);
  const char* kp = (const char*)pages.k;
  const char* vp = (const char*)pages.v;
  const int64_t head_bytes = (int64_t)16 * HD * sizeof(T), page_bytes = hkv * head_bytes;

  typedef typename std::conditional<E8, ts_u32x2, ts_u32x4>::type Vals;        // four (fp32) or eight consecutive keys of a dimension
  struct Block { ts_u32x4 k[KT][KC]; Vals v[F32 ? 2 : 1][DT]; ts_u32x2 ks, vs; bool ok0, ok1; };
  auto pages_of = [&](int kb) {                              // the second may lie behind the last position
    return make_int2(kb < hi ? table[kb / 16] : -1, kb + 16 < hi ? table[kb / 16 + 1] : -1);
  };
  auto fetch = [&](Block& f, int2 pg) __attribute__((always_inline)) {         // pages that do not exist: another is read, and masked
    f.ok0 = pg.x >= 0 && pg.x < pages.n_pages;
    f.ok1 = pg.y >= 0 && pg.y < pages.n_pages;
    const int p0 = f.ok0 ? pg.x : 0, p1 = f.ok1 ? pg.y : p0;
    const int64_t at0 = p0 * page_bytes + kvh * head_bytes, at1 = p1 * page_bytes + kvh * head_bytes;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      const int key = F32 ? 16 * t + n : KL * (n / 4) + 4 * t + n % 4;
      const char* row = kp + (key < 16 ? at0 : at1) + key % 16 * HD * (int)sizeof(T);
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const int b = (c * 4 + lg) * 16;
        if (HD * (int)sizeof(T) % 64 == 0 || b < HD * (int)sizeof(T)) f.k[t][c] = *reinterpret_cast<const ts_u32x4*>(row + b);
        else f.k[t][c] = ts_u32x4{0, 0, 0, 0};
      }
    }
    if constexpr (F32) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          if (HD % 16 == 0 || d * 16 + n < HD) f.v[t][d] = *reinterpret_cast<const ts_u32x4*>(vp + (t ? at1 : at0) + (d * 16 + n) * 64 + lg * 16);
          else f.v[t][d] = ts_u32x4{0, 0, 0, 0};
        }
    } else {
      constexpr int HALF = 8 * (int)sizeof(T);               // bytes of eight keys
      const char* col = vp + (lg < 2 ? at0 : at1) + (lg & 1) * HALF;
#pragma unroll
      for (int d = 0; d < DT; ++d) f.v[0][d] = *reinterpret_cast<const Vals*>(col + (d * 16 + n) * 2 * HALF);
      if constexpr (E8) {                                    // 16 HD bytes of codes to 16 of scales: of this lane's rows of K's tiles, of its keys
        f.ks = *reinterpret_cast<const ts_u32x2*>(a.cache.k_scales + (n < 8 ? at0 : at1) / HD + (n / 4 & 1) * 8);
        f.vs = *reinterpret_cast<const ts_u32x2*>(a.cache.v_scales + (lg < 2 ? at0 : at1) / HD + (lg & 1) * 8);
      }
    }
  };
  auto use = [&](Block& f, int kb) __attribute__((always_inline)) {
    ts_f32x4 s[NT][KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
#pragma unroll
      for (int j = 0; j < NT; ++j) s[j][t] = ts_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < QS; ++c) {
        if constexpr (F32) {
          const ts_f32x4 kx = __builtin_bit_cast(ts_f32x4, f.k[t][c]);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const ts_f32x4 qx = __builtin_bit_cast(ts_f32x4, q[j][0][c]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[j][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[e], qx[e], s[j][t], 0, 0, 0);
          }
        } else {
          ts_u32x4 kx;
          if constexpr (E8) kx = e4m3_to_bf16(f.k[t][c / 2][c % 2 * 2], f.k[t][c / 2][c % 2 * 2 + 1], __uint_as_float(f.ks[t] >> n % 4 * 8 << 23));
          else kx = f.k[t][c];
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int p = QP - 1; p >= 0; --p)
              s[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(ts_bf16x8, kx), __builtin_bit_cast(ts_bf16x8, q[j][p][c]), s[j][t], 0, 0, 0);
        }
      }
    }
    auto key_of = [&](int i) { return kb + (F32 ? 16 * (i / 4) + 4 * lg + i % 4 : KL * lg + i); };      // a lane's i-th key
    const bool whole = kb >= all_lo && kb + KB <= min(all_hi, k1) && f.ok0 && f.ok1;
    bool far = false;                                        // a value's scale goes onto its probability where that neither overflows nor loses bits
    if constexpr (E8) far = __ballot(far_scale(f.vs[0]) || far_scale(f.vs[1])) != 0;
    uint32_t keep[NT];
    uint32_t pk[NT][PP][KL / 2];                             // probabilities as pairs of bf16 terms
    float px[F32 ? NT : 1][F32 ? KL : 1];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      float x[KL];
#pragma unroll
      for (int i = 0; i < KL; ++i) {
        x[i] = s[j][i / 4][i % 4] * g.scale_log2;
      }
      if (!whole) {
        keep[j] = 0;
#pragma unroll
        for (int i = 0; i < KL; ++i) {
          const int key = key_of(i), own = key - rs.start;
          bool in = (key >= c_lo[j]) & (key < min(c_hi[j], k1)) & (F32 ? (i < 4 ? f.ok0 : f.ok1) : (lg < 2 ? f.ok0 : f.ok1));
          if (a.ancestors) in = in & ((own <= 0) | ((own <= 64) & ((int)(c_set[j] >> (own - 1 & 63)) & 1)));
          x[i] = in ? x[i] : -INFINITY;
          keep[j] |= in ? 1u << i : 0;
        }
      }
      float top = x[0];
#pragma unroll
      for (int i = 1; i < KL; ++i) top = fmaxf(top, x[i]);
      top = fmaxf(max_over_lane_groups(top), m[j]);
      if (__ballot(top > m[j])) {                            // the sums so far move to the new reference
        const float w = m[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[j] - top);
        l[j] *= w;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[j][d] *= w;
        m[j] = top;
      }
      const float ref = m[j] == -INFINITY ? 0.f : m[j];
#pragma unroll
      for (int i = 0; i < KL; ++i) {
        x[i] = __builtin_amdgcn_exp2f(x[i] - ref);
        l[j] += x[i];
      }
      if constexpr (E8) {
        if (!far) {
#pragma unroll
          for (int i = 0; i < KL; ++i) x[i] = __builtin_amdgcn_ldexpf(x[i], (int)(f.vs[i / 4] >> i % 4 * 8 & 255) - 127);
        }
      }
      if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < KL; ++i) px[j][i] = x[i];
      } else {
#pragma unroll
        for (int i = 0; i < KL / 2; ++i) {
          ts_bf16x2 w[PP];
          if constexpr (PP == 1) w[0] = to_bf16x2(x[2 * i], x[2 * i + 1]);
          else split_bf16x2_nonzero<PP>(x[2 * i], x[2 * i + 1], w);
#pragma unroll
          for (int p = 0; p < PP; ++p) pk[j][p][i] = __builtin_bit_cast(uint32_t, w[p]);
        }
      }
    }
    if constexpr (F32) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          ts_u32x4 v = f.v[t][d];
          if (!whole && __ballot((v[0] & 0x7f800000u) == 0x7f800000u || (v[1] & 0x7f800000u) == 0x7f800000u || (v[2] & 0x7f800000u) == 0x7f800000u ||
                                 (v[3] & 0x7f800000u) == 0x7f800000u)) {
            for (int cls = 0; cls < 3; ++cls)
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                ts_f32x4 hit = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int r = 0; r < 4; ++r)
                  hit = __builtin_amdgcn_mfma_f32_16x16x4f32(of_class(v[r], cls) ? 1.f : 0.f, keep[j] >> (4 * t + r) & 1 ? 1.f : 0.f, hit, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[j][d][r] += hit[r] > 0.f ? class_value(cls) : 0.f;
              }
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = (v[r] & 0x7f800000u) == 0x7f800000u ? 0 : v[r];
          }
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[j][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[r]), px[j][4 * t + r], o[j][d], 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          ts_u32x4 w;
          if constexpr (E8) {
            if (far) w = e4m3_to_bf16(f.v[0][d][0], f.v[0][d][1], f.vs[0], f.vs[1]);
            else w = e4m3_to_bf16(f.v[0][d][0], f.v[0][d][1], 1.f);
          } else {
            w = f.v[0][d];
          }
          if (!whole && __ballot(not_finite(w[0]) || not_finite(w[1]) || not_finite(w[2]) || not_finite(w[3]))) {
            for (int cls = 0; cls < 3; ++cls) {
              ts_u32x4 is;
#pragma unroll
              for (int e = 0; e < 4; ++e) is[e] = (of_class(w[e] << 16, cls) ? 0x3f80u : 0) | (of_class(w[e] & 0xffff0000u, cls) ? 0x3f800000u : 0);
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                ts_u32x4 in;
#pragma unroll
                for (int e = 0; e < 4; ++e) in[e] = (keep[j] >> (2 * e) & 1 ? 0x3f80u : 0) | (keep[j] >> (2 * e + 1) & 1 ? 0x3f800000u : 0);
                const ts_f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(ts_bf16x8, is),
                                                                              __builtin_bit_cast(ts_bf16x8, in), ts_f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[j][d][r] += hit[r] > 0.f ? class_value(cls) : 0.f;
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] &= ((w[e] & 0x7f80u) == 0x7f80u ? 0 : 0xffffu) | ((w[e] & 0x7f800000u) == 0x7f800000u ? 0 : 0xffff0000u);
          }
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int p = PP - 1; p >= 0; --p)
              o[j][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(ts_bf16x8, w),
                                                                __builtin_bit_cast(ts_bf16x8, ts_u32x4{pk[j][p][0], pk[j][p][1], pk[j][p][2], pk[j][p][3]}), o[j][d], 0, 0, 0);
        }
    }
  };
  // The next block is requested before one is used; past the end the last is requested again, since the waits count the loads
  // behind the ones they wait for.
  constexpr int STEP = RO_WAVES * KB;
  const int kw = k0 + wave * KB;
  if (kw + STEP >= k1) {
    if (kw < k1) {
      Block f;
      fetch(f, pages_of(kw));
      use(f, kw);
    }
  } else if constexpr (NT * HD <= 256 && !(F32 && HD == 128)) {
    const int last = kw + (k1 - 1 - kw) / STEP * STEP;
    Block fa, fb;
    fetch(fa, pages_of(kw));
    int2 next = pages_of(kw + STEP);
    for (int kb = kw; kb < k1; kb += 2 * STEP) {
      fetch(fb, next);
      next = pages_of(min(kb + 2 * STEP, last));
      use(fa, kb);
      if (kb + STEP >= k1) break;
      fetch(fa, next);
      next = pages_of(min(kb + 3 * STEP, last));
      use(fb, kb + STEP);
    }
  } else {
    int2 next = pages_of(kw);
    for (int kb = kw; kb < k1; kb += STEP) {
      Block f;
      fetch(f, next);
      next = pages_of(kb + STEP);
      use(f, kb);
    }
  }

  // the four waves' parts, a tile of columns at a time
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    if (j * 16 >= cols) break;
    if (j) __syncthreads();
    l[j] += __shfl_xor(l[j], 16, 64);
    l[j] += __shfl_xor(l[j], 32, 64);
    if (lane < 16) { sm[wave][n] = m[j]; sl[wave][n] = l[j]; }
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<ts_f32x4*>(&so[(wave * 16 + n) * OS + d * 16 + lg * 4]) = o[j][d];
    __syncthreads();
    for (int i = tid; i < min(16, cols - j * 16) * HD; i += RO_WAVES * 64) {
      const int c = i / HD, d = i % HD, row = where[j * 16 + c].x, head = where[j * 16 + c].y;
      float top = sm[0][c];
#pragma unroll
      for (int w = 1; w < RO_WAVES; ++w) top = fmaxf(top, sm[w][c]);
      const float ref = top == -INFINITY ? 0.f : top;
      float sum = 0.f, val = 0.f;
#pragma unroll
      for (int w = 0; w < RO_WAVES; ++w) {
        const float x = __builtin_amdgcn_exp2f(sm[w][c] - ref);
        sum += x * sl[w][c];
        val += x * so[(w * 16 + c) * OS + d];
      }
      const int64_t at = (int64_t)row * a.n_q_heads + head;
      if (g.splits == 1) {
        st_from_f32((TQ*)a.out + (int64_t)row * a.out_stride + (int64_t)head * HD + d, sum == 0.f ? 0.f : val / sum);
        if (a.lse && d == 0) a.lse[at] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
      } else {
        const int64_t part = at * g.splits + (lo / g.chunk + split) % g.splits;
        g.part_o[part * HD + d] = val;
        if (d == 0) *reinterpret_cast<float2*>(g.part_ml + part * 2) = make_float2(top, sum);
      }
    }
  }
}

// ---------------------------------------------------------------------------------
// Many columns over bf16 and 8-bit pages, bf16 rows: bound by the matrix pipes and by the soft-max beside them.  W waves of 32
// columns share the keys and values of a block of 64 through the LDS.  The running maximum is a reference that moves only when a
// score passes it by more than 2^8, so that sums are rarely rescaled.  The matrix layout is the one above in tiles of 32 x 32: row m of K's
// tile is key m with its bits 2 and 3 swapped.  Blocks go through registers (8-bit ones are widened there, times their scales,
// once for all waves) into two LDS slots: while block b is used, b + 1 waits in registers and is written behind it, then b + 2 is
// requested; one barrier a block.  Probabilities are rounded to bf16 for the product with the values, a rounding as large as the output's own:
// 0.0023 of the outputs' norm from 64 bits, where the output's alone is 0.0017.  A second term, which takes that away, is half as many matrix
// instructions again: prompts 286 -> 367 us, 8-bit chunks below 972 -> 1244, the tree 36.2 -> 40.1; 412, 1463 and 44.6 where the second term may not be zero, so that
// an infinite value stays so.
//
// bf16, 32 query heads over 8 of 128: three prompts, 9012 rows (237 GFLOP as counted) 290 - 305 us, 0.80 PFLOP/s, matrix pipes busy 40 %;
// a tree of 65 rows over 8192 positions 28 us and 7 of the join; 16 x 33 rows over up to 4096 66 and 12.  8-bit, 64 heads over 8:
// 4 x 512 rows over up to 16384 (881 GFLOP) 975 - 985 us, 0.90 PFLOP/s.  What a block's time goes into, by leaving pieces out (the last
// case, 1193 us then): products alone 531, without staging 872, without staging and LDS reads 640, without staging and soft-max 730.
// Measured and not kept (prompts and last case, microseconds, beside this kernel of the same day): four waves of 64 columns, half the
// LDS reads, a phase's soft-max between its neighbours' products by hand, one wave a SIMD: 406 and 2247 : 332 and 1261.  Two groups of
// waves half a step apart, one multiplying while the other works out probabilities: 319 - 356 and 1365 - 1895.  Two blocks on their way, a
// barrier for 128 keys, wave priorities, fragments read ahead: no gain.
// ---------------------------------------------------------------------------------
typedef float ts_f32x16 __attribute__((ext_vector_type(16)));

template <typename T, int HD, int RW_WAVES>
__global__ __launch_bounds__(RW_WAVES * 64, 2) void k_kv_attend_wide(RowsArgs g) {
  constexpr bool E8 = sizeof(T) == 1;
  constexpr int RW_TM = RW_WAVES * 32;
  constexpr int DT = HD / 32, KS = HD / 16, PAGE = 16 * HD;               // tiles of 32 dimensions, steps of 16, elements of a page and head
  constexpr int RING = 2, LOADS = (4 * PAGE * (int)sizeof(T) + 16 * RW_WAVES * 64 - 1) / (16 * RW_WAVES * 64);      // 16-byte loads of a thread for keys, and for values
  constexpr int PER_PAGE = PAGE * (int)sizeof(T) / 16;                    // 16-byte pieces of a page
  constexpr float LAZY = 8.f;
  __shared__ int dirty;
  __shared__ ts_u32x4 sk[RING][4 * PAGE / 8], sv[RING][4 * PAGE / 8];
  const ts_kv_attend_rows_args& a = g.a;
  const ts_kv_pages& pages = a.cache.pages;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, n = lane % 32, h = lane / 32;
  int id = blockIdx.x;
  const int hkv = pages.n_kv_heads, kvh = id % hkv; id /= hkv;
  const int split = id % g.splits, t = id / g.splits, G = g.group;
  int m0, cols;
  RowSeq rs;
  const int seq = tile_of<RW_TM, 32>(a, G, g.seq_tiles, t, m0, cols, rs);
  if (seq < 0) return;
  const int row0 = rs.first + m0 / G, rem = m0 % G;
  const int lo = row_range(a, rs, row0).x, hi = row_range(a, rs, row0 + (rem + cols - 1) / G).y;
  const int64_t from = ((int64_t)(lo / g.chunk) + split) * g.chunk;
  if (split > 0 && from >= hi) return;
  const int k0 = (int)max(from, (int64_t)(lo & ~63)), k1 = (int)min((int64_t)hi, from + g.chunk);
  const int blocks = k1 > k0 ? (k1 - k0 + 63) / 64 : 0;
  // this wave's columns
  const int mine0 = min(wave * 32, cols - 1), mine1 = min(wave * 32 + 32, cols) - 1;     // one of them again where there is none
  const bool active = wave * 32 < cols;
  const int2 w_low = row_range(a, rs, row0 + (rem + mine0) / G), w_high = row_range(a, rs, row0 + (rem + max(mine1, mine0)) / G);
  const int all_lo = w_high.x, all_hi = min(a.ancestors ? min(max(rs.start + 1, 0), w_low.y) : w_low.y, k1);

  const int tile_lo = row_range(a, rs, row0 + (rem + cols - 1) / G).x;
  const int tile_hi = min(a.ancestors ? min(max(rs.start + 1, 0), row_range(a, rs, row0).y) : row_range(a, rs, row0).y, k1);

  const float scale = g.scale_log2 == 0.f ? 0x1p-149f : fabsf(g.scale_log2);       // zero only where the host flushes subnormal numbers, see rows_cut
  int c_lo, c_hi;
  uint64_t c_set;
  ts_u32x4 q[KS];
  {
    const int m = rem + min(wave * 32 + n, cols - 1), row = row0 + m / G, head = kvh * G + m % G;
    const int2 range = row_range(a, rs, row);
    c_lo = range.x; c_hi = min(range.y, k1);
    c_set = a.ancestors ? a.ancestors[row] : 0;
    const bf16_t* src = (const bf16_t*)a.q + (int64_t)row * a.q_stride + (int64_t)head * HD;
    const uint32_t sign = g.scale_log2 < 0.f ? 0x80008000u : 0;      // a negative scale turns the query, exactly
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      const uint4 w = load16(src + c * 16 + h * 8);
      q[c] = ts_u32x4{w.x ^ sign, w.y ^ sign, w.z ^ sign, w.w ^ sign};
    }
  }
  ts_f32x16 o[DT];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

  // ---- blocks: pages, registers, LDS
  const int32_t* table = a.table + (int64_t)seq * a.table_stride + k0 / 16 + lane % 4;
  auto pages_of = [&](int b) __attribute__((always_inline)) {  // lane i: page i % 4 of the block, -1 behind the last position
    return b < blocks && k0 + b * 64 + lane % 4 * 16 < hi ? table[b * 4] : -1;
  };
  auto good_bits = [&](int pg) __attribute__((always_inline)) { return (int)__ballot((uint32_t)pg < (uint32_t)pages.n_pages) & 15; };
  struct Stage { ts_u32x4 k[LOADS], v[LOADS], vs[E8 ? LOADS : 1]; uint32_t ks[E8 ? LOADS : 1]; };
  const uint32_t piece_at = tid % PER_PAGE * 16;             // this thread's piece of a page
  auto request = [&](Stage& st, int pg, int ok) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int which = min(__builtin_amdgcn_readfirstlane((i * RW_WAVES * 64 + tid) / PER_PAGE), 3);
      const int page = ok >> which & 1 ? __builtin_amdgcn_readlane(pg, which) : 0;
      const int64_t head = (int64_t)page * hkv + kvh;
      st.k[i] = *reinterpret_cast<const ts_u32x4*>((const char*)pages.k + head * (PAGE * (int)sizeof(T)) + piece_at);
      st.v[i] = *reinterpret_cast<const ts_u32x4*>((const char*)pages.v + head * (PAGE * (int)sizeof(T)) + piece_at);
      if constexpr (E8) {
        st.ks[i] = (a.cache.k_scales + head * 16)[piece_at / HD];
        st.vs[i] = *reinterpret_cast<const ts_u32x4*>(a.cache.v_scales + head * 16);
      }
    }
  };
  // LDS places of 16-byte pieces: of sixteen lanes that read or write together, each meets a sixteenth of 256 bytes of its own.  Sixteen
  // lanes read one piece of sixteen keys, or one half (eight keys) of sixteen dimensions; they write the pieces of one or two
  // keys (widened: every other one of two or four), or both halves of eight dimensions (widened: one of sixteen).
  auto key_place = [&](int key, int piece) __attribute__((always_inline)) { return key * (HD / 8) + (piece ^ (HD == 128 ? key & 15 : key >> 1 & 7)); };
  auto value_place = [&](int page, int dim, int half) __attribute__((always_inline)) { return ((page * DT + dim / 32) * 2 + half) * 32 + (dim % 32 ^ half * 8); };
  // values that are not finite become zeros where not every column sees them
  auto clean = [&](ts_u32x4 v) __attribute__((always_inline)) {
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool x = (v[e] & 0x7f80u) == 0x7f80u, y = (v[e] & 0x7f800000u) == 0x7f800000u;
      bad |= x | y;
      v[e] &= (x ? 0 : 0xffffu) | (y ? 0 : 0xffff0000u);
    }
    if (bad) dirty = 1;
    return v;
  };
  auto write = [&](Stage& st, int slot, bool all_see) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int piece = i * RW_WAVES * 64 + tid, pg = piece / PER_PAGE, in = piece % PER_PAGE;
      if (LOADS * RW_WAVES * 64 > 4 * PER_PAGE && piece >= 4 * PER_PAGE) break;      // of small blocks the other waves have no part
      ts_u32x4 v[E8 ? 2 : 1];
      if constexpr (E8) {
        const int key = pg * 16 + in * 16 / HD, c = in % (HD / 16) * 2;
        const float ks = scale_at<0>(st.ks[i]);
        sk[slot][key_place(key, c)] = e4m3_to_bf16(st.k[i][0], st.k[i][1], ks);
        sk[slot][key_place(key, c + 1)] = e4m3_to_bf16(st.k[i][2], st.k[i][3], ks);
        v[0] = e4m3_to_bf16(st.v[i][0], st.v[i][1], st.vs[i][0], st.vs[i][1]);
        v[1] = e4m3_to_bf16(st.v[i][2], st.v[i][3], st.vs[i][2], st.vs[i][3]);
      } else {
        sk[slot][key_place(pg * 16 + in / (HD / 8), in % (HD / 8))] = st.k[i];
        v[0] = st.v[i];
      }
#pragma unroll
      for (int e = 0; e < (E8 ? 2 : 1); ++e) {
        if (!all_see) v[e] = clean(v[e]);
        sv[slot][E8 ? value_place(pg, in, e) : value_place(pg, in / 2, in % 2)] = v[e];
      }
    }
  };

  const int kn = (n & ~12) | (n & 4) << 1 | (n & 8) >> 1;    // the key that is row n of K's tile
  // truth values without branches
  auto sees = [&](int key, bool ok) __attribute__((always_inline)) { return (key >= c_lo) & (key < c_hi) & ok; };
  auto sees_tree = [&](int key) __attribute__((always_inline)) {
    const int own = key - rs.start;
    return (own <= 0) | ((own <= 64) & ((int)(c_set >> ((own - 1) & 63)) & 1));
  };
  auto use = [&](int slot, int kb, int ok) __attribute__((always_inline)) {
    ts_f32x16 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
#pragma unroll
      for (int c = 0; c < KS; ++c)
        s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(ts_bf16x8, sk[slot][key_place(t * 32 + kn, c * 2 + h)]), __builtin_bit_cast(ts_bf16x8, q[c]), s[t], 0, 0, 0);
    }
    if (!(kb >= all_lo && kb + 64 <= all_hi && ok == 15)) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = sees(kb + 32 * t + 16 * (i / 8) + 8 * h + i % 8, (ok >> (2 * t + i / 8) & 1) != 0) ? s[t][i] : -INFINITY;
      if (a.ancestors) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[t][i] = sees_tree(kb + 32 * t + 16 * (i / 8) + 8 * h + i % 8) ? s[t][i] : -INFINITY;
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) top = fmaxf(top, s[i / 16][i % 16]);
    const uint32_t u = __float_as_uint(top);
    const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * scale;
    if (__ballot(top > m + LAZY)) {                          // the sums so far move to the new reference
      const float next = top > m + LAZY ? top : m, w = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - next);
      l *= w;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= w;
      m = next;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      ts_u32x4 p[2];
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], scale, -ref)), y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i + 1], scale, -ref));
        l += x;
        l += y;
        p[i / 8][i / 2 % 4] = __builtin_bit_cast(uint32_t, to_bf16x2(x, y));
      }
#pragma unroll
      for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int d = 0; d < DT; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(ts_bf16x8, sv[slot][value_place(t * 2 + v, d * 32 + n, h)]), __builtin_bit_cast(ts_bf16x8, p[v]), o[d], 0, 0, 0);
    }
  };
  auto whole = [&](int b, int ok) { return k0 + b * 64 >= tile_lo && k0 + b * 64 + 64 <= tile_hi && ok == 15; };

  if (tid == 0) dirty = 0;
  __syncthreads();
  if (blocks) {
    // Block b + 1 is on its way or in registers while block b is used, and the pages of b + 2 are known.
    int next = pages_of(0), ok = good_bits(next), ok_next;
    Stage st;
    request(st, next, ok);
    next = pages_of(1);
    write(st, 0, whole(0, ok));
    ok_next = good_bits(next);
    request(st, next, ok_next);
    next = pages_of(2);
    __syncthreads();
    for (int b = 0; b < blocks; ++b) {
      if (active) use(b & 1, k0 + b * 64, ok);
      if (b + 1 < blocks) write(st, b + 1 & 1, whole(b + 1, ok_next));
      ok = ok_next;
      ok_next = good_bits(next);
      request(st, next, ok_next);
      next = pages_of(b + 3);
      wait_lds();
    }
  }
  // Values that are not finite, in blocks whose keys not every column sees, were left out: here they reach those that do.
  if (blocks && dirty) {
    for (int b = 0; b < blocks; ++b) {
      const int pg = pages_of(b), ok = good_bits(pg);
      if (whole(b, ok)) continue;
      for (int u = 0; u < 4; ++u) {
        if (!(ok >> u & 1)) continue;
        const int page = __builtin_amdgcn_readlane(pg, u);
        const int kb = k0 + b * 64 + u * 16 + 8 * h;
        const int64_t head = (int64_t)page * hkv + kvh;
        ts_u32x4 in;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool one = sees(kb + e, true) & (!a.ancestors | sees_tree(kb + e));
          in[e / 2] = (e & 1 ? in[e / 2] : 0) | (one ? (e & 1 ? 0x3f800000u : 0x3f80u) : 0);
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          ts_u32x4 v;
          if constexpr (E8) {
            const uint2 w = *reinterpret_cast<const uint2*>((const char*)pages.v + (head * HD + d * 32 + n) * 16 + 8 * h), sc = *reinterpret_cast<const uint2*>(a.cache.v_scales + head * 16 + 8 * h);
            v = e4m3_to_bf16(w.x, w.y, sc.x, sc.y);
          } else {
            v = *reinterpret_cast<const ts_u32x4*>((const char*)pages.v + (head * HD + d * 32 + n) * 32 + 16 * h);
          }
          for (int cls = 0; cls < 3; ++cls) {
            ts_u32x4 is;
#pragma unroll
            for (int e = 0; e < 4; ++e) is[e] = (of_class(v[e] << 16, cls) ? 0x3f80u : 0) | (of_class(v[e] & 0xffff0000u, cls) ? 0x3f800000u : 0);
            ts_f32x16 hit;
#pragma unroll
            for (int i = 0; i < 16; ++i) hit[i] = 0.f;
            hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(ts_bf16x8, is), __builtin_bit_cast(ts_bf16x8, in), hit, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] += hit[i] > 0.f ? class_value(cls) : 0.f;
          }
        }
      }
    }
  }
  if (!active) return;
  const uint32_t u = __float_as_uint(l);
  const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const float sum = __uint_as_float(both[0]) + __uint_as_float(both[1]);
  if (wave * 32 + n >= cols) return;
  const int mc = rem + wave * 32 + n, row = row0 + mc / G, head = kvh * G + mc % G;
  const int64_t at = (int64_t)row * a.n_q_heads + head;
  if (g.splits == 1) {
    const float inv = 1.f / sum;
    bf16_t* dst = (bf16_t*)a.out + (int64_t)row * a.out_stride + (int64_t)head * HD;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = sum == 0.f ? 0.f : o[d][i + e] * inv;
        store_n<4>(dst + d * 32 + 2 * i + 4 * h, x);
      }
    if (a.lse && h == 0) a.lse[at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.69314718055994531f;
  } else {
    const int64_t part = at * g.splits + (lo / g.chunk + split) % g.splits;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(g.part_o + part * HD + d * 32 + 2 * i + 4 * h) = make_float4(o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]);
    if (h == 0) *reinterpret_cast<float2*>(g.part_ml + part * 2) = make_float2(m, sum);
  }
}

// The join of a row's splits: chunk c of the cache's positions lies at place c % splits.  Few splits: a wave per (row, head), four
// dimensions a lane, the splits dealt to the lane groups of a head's length.  Bound by trips to memory in turn: the sequence, its length, the parts.
// One token over 8192 positions (33 splits, the kernel below) 5.0 - 5.6 us in a trace, 65 rows x 32 heads of 17 splits (18 MB) 6.8 - 7.0.  Weights and
// parts asked for before the row's sequence is known gained 0.2 - 0.5 us of a call (17.1 : 16.6, 35.6 : 35.3, 75.6 : 75.4): not kept.
template <typename TQ, int HD>
__global__ __launch_bounds__(256) void k_kv_attend_rows_join_few(RowsArgs g) {
  constexpr int COLS = HD / 4, GROUPS = 64 / COLS;
  const ts_kv_attend_rows_args& a = g.a;
  const int64_t at = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64);
  const int lane = threadIdx.x % 64, row = (int)(at / a.n_q_heads), h = (int)(at % a.n_q_heads);
  if (row >= a.n_rows) return;
  int seq = row;
  if (a.row_offsets) {
    seq = seq_of_row(a.row_offsets, a.n_seqs + 1, row);
    if (seq < 0 || seq >= a.n_seqs || row >= a.row_offsets[seq + 1]) return;
  } else if (row >= a.n_seqs) {
    return;
  }
  const int2 range = row_range(a, row_seq(a, seq), row);
  const int c0 = range.x / g.chunk, used = range.y > range.x ? (range.y + g.chunk - 1) / g.chunk - c0 : 0;      // a row that sees nothing has no parts
  const float2* ml = reinterpret_cast<const float2*>(g.part_ml) + at * g.splits;
  const float4* part = reinterpret_cast<const float4*>(g.part_o) + at * g.splits * COLS + lane % COLS;
  float top = -INFINITY;
  for (int i = lane; i < used; i += 64) top = fmaxf(top, ml[(c0 + i) % g.splits].x);
  top = wave_max(top);
  const float ref = top == -INFINITY ? 0.f : top;
  float sum = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = lane / COLS; i < used; i += GROUPS) {
    const int place = (c0 + i) % g.splits;
    const float2 p = ml[place];
    const float4 v = part[(int64_t)place * COLS];
    const float f = __builtin_amdgcn_exp2f(p.x - ref);
    sum += f * p.y;
    x[0] += f * v.x; x[1] += f * v.y; x[2] += f * v.z; x[3] += f * v.w;
  }
#pragma unroll
  for (int o = COLS; o < 64; o *= 2) {
    sum += __shfl_xor(sum, o, 64);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], o, 64);
  }
  if (lane >= COLS) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = sum == 0.f ? 0.f : x[e] / sum;
  store_n<4>((TQ*)a.out + (int64_t)row * a.out_stride + (int64_t)h * HD + lane * 4, x);
  if (a.lse && lane == 0) a.lse[at] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
}

// Many splits: a workgroup per (row, head), four dimensions a thread, the splits dealt to the rows of threads.
constexpr int RO_SPLITS = RO_MOST * RO_CUS;                  // at most, see rows_cut; a window may add one
template <typename TQ, int HD>
__global__ __launch_bounds__(256) void k_kv_attend_rows_join(RowsArgs g) {
  constexpr int COLS = HD / 4, ROWS = 256 / COLS;
  __shared__ float sw[RO_SPLITS + 1];
  __shared__ float4 sv[256];
  __shared__ float red[2][4];
  const ts_kv_attend_rows_args& a = g.a;
  const int tid = threadIdx.x, wave = tid / 64, h = blockIdx.x % a.n_q_heads, row = blockIdx.x / a.n_q_heads;
  int seq = row;
  if (a.row_offsets) {
    seq = seq_of_row(a.row_offsets, a.n_seqs + 1, row);
    if (seq < 0 || seq >= a.n_seqs || row >= a.row_offsets[seq + 1]) return;
  } else if (row >= a.n_seqs) {
    return;
  }
  const RowSeq rs = row_seq(a, seq);
  const int2 range = row_range(a, rs, row);
  const int c0 = range.x / g.chunk, used = range.y > range.x ? (range.y + g.chunk - 1) / g.chunk - c0 : 0;      // a row that sees nothing has no parts
  const int64_t at = (int64_t)row * a.n_q_heads + h;
  const float2* ml = reinterpret_cast<const float2*>(g.part_ml) + at * g.splits;
  float top = -INFINITY;
  for (int i = tid; i < used; i += 256) top = fmaxf(top, ml[(c0 + i) % g.splits].x);
  top = wave_max(top);
  if (tid % 64 == 0) red[0][wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  const float ref = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  for (int i = tid; i < used; i += 256) {
    const float2 p = ml[(c0 + i) % g.splits];
    const float f = __builtin_amdgcn_exp2f(p.x - ref);
    sw[i] = f;
    sum += f * p.y;
  }
  sum = wave_sum(sum);
  if (tid % 64 == 0) red[1][wave] = sum;
  __syncthreads();
  sum = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  const int d = tid % COLS, r = tid / COLS;
  const float4* part = reinterpret_cast<const float4*>(g.part_o) + at * g.splits * COLS + d;
  float4 val = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int i = r; i < used; i += ROWS) {
    const float4 v = part[(int64_t)((c0 + i) % g.splits) * COLS];
    const float f = sw[i];
    val.x += f * v.x; val.y += f * v.y; val.z += f * v.z; val.w += f * v.w;
  }
  sv[tid] = val;
  __syncthreads();
  if (tid >= HD) return;
  const float* sc = reinterpret_cast<const float*>(sv);
  float out = 0.f;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) out += sc[i * HD + tid];
  st_from_f32((TQ*)a.out + (int64_t)row * a.out_stride + (int64_t)h * HD + tid, sum == 0.f ? 0.f : out / sum);
  if (a.lse && tid == 0) a.lse[at] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------------

struct RowsCut { int nt, chunk, splits; int64_t slots; };    // tiles of 16 a workgroup (8 and 16: the wide kernel), keys of a split, splits, tile slots per KV head

// Columns of a workgroup, from those a sequence has on average: 16; then, of fp32 rows or pages, 32; of others 128 and, from 512 on, 256.
// bf16, 32 query heads over 8, microseconds: 8 rows over 8192 (32 columns) 128 a workgroup 20.3, tiles of 64 straight from memory 29.3;
// 16 x 12 rows over 4096 (48) 57 and 157; 16 x 33 over up to 4096 (132) 76, and 256 a workgroup 88; 8-bit chunks of 4 x 512 rows
// (4096) 1217 and 1127.  All of these have about as many rows a sequence.  Where they differ the average serves neither kind: 7 tokens over 32768 positions and a chunk
// of 512 rows over 8192, bf16, 64 heads over 8, 674 in one call and 166 + 168 in two; a token over 32768 beside 63 over 200, 32 heads, 284 and 30 + 16.
static int rows_nt(int64_t n_seqs, int64_t n_rows, int group, bool f32) { return n_rows * group <= n_seqs * 16 ? 1 : f32 ? 2 : n_rows * group <= n_seqs * 512 ? 8 : 16; }
static int64_t rows_units(int max_len, int window) {         // of 128 keys, in what one tile sees
  const int64_t span = window > 0 && (int64_t)window + 256 < max_len ? window + 256 : max_len;
  return std::max<int64_t>(1, (span + RO_UNIT - 1) / RO_UNIT);
}
// workgroups without a split
static int64_t rows_whole(int64_t n_seqs, int64_t n_rows, int group, int hkv, int nt) {
  return std::max<int64_t>(n_seqs, (n_rows * group + 16 * nt - 1) / (16 * nt)) * hkv;
}
static int64_t rows_room(int64_t n_seqs, int64_t n_rows, int group, int hkv, int max_len, int window) {
  int64_t room = 1;
  for (int nt : {1, 2, 8, 16}) room = std::max(room, std::min(rows_units(max_len, window), RO_MOST * RO_CUS / std::max<int64_t>(1, rows_whole(n_seqs, n_rows, group, hkv, nt))));
  return room > 1 && window > 0 ? room + 1 : room;
}
static RowsCut rows_cut(const ts_kv_attend_rows_args& a) {
  const int group = a.n_q_heads / a.cache.pages.n_kv_heads, hkv = a.cache.pages.n_kv_heads;
  RowsCut c;
  // The wide kernel masks products before it scales them, and zero times the -infinity of what is not seen is not -infinity: a scale of zero is
  // the other kernel's, where a seen infinite product makes its head NaN.
  c.nt = a.scale == 0.f ? 1 : rows_nt(a.n_seqs, a.n_rows, group, a.cache.pages.dtype == TS_DTYPE_F32 || a.dtype == TS_DTYPE_F32);
  const int tm = 16 * c.nt;
  c.slots = a.row_offsets ? (int64_t)a.n_rows * group / tm + a.n_seqs : (int64_t)a.n_seqs * ((group + tm - 1) / tm);
  const int64_t whole = rows_whole(a.n_seqs, a.n_rows, group, hkv, c.nt), units = rows_units(a.max_len, a.window);
  int64_t per = 1;
  // Workgroups a CU: two of the smaller wide ones (16 x 33 rows 105 -> 86 us, 8 x 33 rows over 16384 8-bit positions 237 -> 143; three or four
  // no faster) and of single tokens over 8-bit pages (8 sequences up to 32768 133 -> 88, four 93).
  const int a_cu = (c.nt == 1 && a.cache.pages.dtype == TS_DTYPE_E4M3) || c.nt == 8 ? 2 : 1;
  if (units * whole > RO_MOST * RO_CUS) {
    const int64_t want = std::max<int64_t>(1, std::min(a_cu, RO_MOST) * RO_CUS / whole);
    per = (units + want - 1) / want;
  }
  if (units <= 2) per = units;
  c.chunk = (int)(per * RO_UNIT);
  c.splits = (int)((units + per - 1) / per);
  if (c.splits == 1) c.chunk = 1 << 30;                      // one chunk, wherever a window lies
  else if (a.window > 0) ++c.splits;
  return c;
}

static ts_status check_rows(const char* call, int32_t n_seqs, int32_t n_rows, int32_t hq, int32_t hkv, int32_t max_len, int32_t window) {
  if (n_seqs < 1 || n_seqs > (1 << 20)) return ts_fail(TS_ERR_INVALID_ARG, "%s: n_seqs %d outside [1, 2^20]", call, n_seqs);
  if (n_rows < 0 || n_rows > (1 << 23)) return ts_fail(TS_ERR_INVALID_ARG, "%s: %d rows outside [0, 2^23]", call, n_rows);
  if (hkv < 1 || hkv > 65536 || hq < 1 || hq > 65536 || hq % hkv) return ts_fail(TS_ERR_INVALID_ARG, "%s: %d query heads over %d KV heads", call, hq, hkv);
  if (max_len < 0 || max_len > (1 << 30)) return ts_fail(TS_ERR_INVALID_ARG, "%s: max_len %d outside [0, 2^30]", call, max_len);
  if (window < 0) return ts_fail(TS_ERR_INVALID_ARG, "%s: window %d is negative", call, window);
  const int64_t slots = (int64_t)n_rows * (hq / hkv) / 16 + (int64_t)n_seqs * ((hq / hkv + 15) / 16);
  constexpr int64_t kMost = (1 << 24) - 1;                   // workgroups of 256 whose threads a launch can count
  if (slots * hkv * rows_room(n_seqs, n_rows, hq / hkv, hkv, max_len, window) > kMost || (int64_t)n_rows * hq > kMost)
    return ts_fail(TS_ERR_INVALID_ARG, "%s: %d rows of %d sequences and %d heads are too many for one call", call, n_rows, n_seqs, hq);
  return TS_OK;
}

extern "C" ts_status ts_kv_attend_rows_workspace(int32_t n_seqs, int32_t n_rows, int32_t hq, int32_t hkv, int32_t head_dim, int32_t max_len, int32_t window,
                                                 uint64_t* bytes) {
  const char* call = "ts_kv_attend_rows_workspace";
  if (!bytes) return ts_fail(TS_ERR_INVALID_ARG, "%s: null argument", call);
  ts_status st = check_rows(call, n_seqs, n_rows, hq, hkv, max_len, window);
  if (st) return st;
  if (head_dim < 8 || head_dim > 128) return ts_fail(TS_ERR_INVALID_ARG, "%s: head_dim %d", call, head_dim);
  const int64_t room = rows_room(n_seqs, n_rows, hq / hkv, hkv, max_len, window);
  *bytes = room > 1 ? (uint64_t)n_rows * hq * room * (head_dim + 2) * 4 : 0;
  return TS_OK;
}

template <typename TQ, int HD>
static void launch_join(const RowsArgs& g, hipStream_t s) {
  const int64_t n = (int64_t)g.a.n_rows * g.a.n_q_heads;
  if (g.splits <= (n >= 1024 ? 64 : 16)) k_kv_attend_rows_join_few<TQ, HD><<<(uint32_t)((n + 3) / 4), 256, 0, s>>>(g);
  else k_kv_attend_rows_join<TQ, HD><<<(uint32_t)n, 256, 0, s>>>(g);
}
template <typename T, typename TQ, int HD>
static void launch_rows(const RowsArgs& g, const RowsCut& c, hipStream_t s) {
  const uint32_t grid = (uint32_t)(c.slots * g.a.cache.pages.n_kv_heads * c.splits);
  if (c.nt == 1) k_kv_attend_rows<T, TQ, HD, 1><<<grid, RO_WAVES * 64, 0, s>>>(g);
  else if constexpr (sizeof(T) == 4 || sizeof(TQ) == 4) k_kv_attend_rows<T, TQ, HD, 2><<<grid, RO_WAVES * 64, 0, s>>>(g);
  else if (c.nt == 8) k_kv_attend_wide<T, HD, 4><<<grid, 256, 0, s>>>(g);
  else k_kv_attend_wide<T, HD, 8><<<grid, 512, 0, s>>>(g);
  if (c.splits > 1) launch_join<TQ, HD>(g, s);
}
template <typename TQ>
static void launch_rows_q(const RowsArgs& g, const RowsCut& c, hipStream_t s) {
  const ts_kv_pages& p = g.a.cache.pages;
#define TS_ROWS(T, HD) if (p.head_dim == HD) return launch_rows<T, TQ, HD>(g, c, s)
  if (p.dtype == TS_DTYPE_E4M3) { TS_ROWS(e4m3_t, 64); TS_ROWS(e4m3_t, 128); }
  else if (p.dtype == TS_DTYPE_BF16) { TS_ROWS(bf16_t, 64); TS_ROWS(bf16_t, 128); }
  else { TS_ROWS(float, 8); TS_ROWS(float, 16); TS_ROWS(float, 32); TS_ROWS(float, 64); TS_ROWS(float, 128); }
#undef TS_ROWS
}

extern "C" ts_status ts_kv_attend_rows(const ts_kv_attend_rows_args* args, ts_stream stream) {
  const char* call = "ts_kv_attend_rows";
  if (!args) return ts_fail(TS_ERR_INVALID_ARG, "%s: null argument", call);
  const ts_kv_attend_rows_args& a = *args;
  const ts_kv_pages& p = a.cache.pages;
  ts_status st = check_kv_pages_any(call, a.cache, a.table, a.table_stride, a.table_width, a.lengths, a.n_seqs, a.dtype);
  if (st) return st;
  if ((st = check_rows(call, a.n_seqs, a.n_rows, a.n_q_heads, p.n_kv_heads, a.max_len, a.window))) return st;
  if (!a.row_offsets && a.n_rows < a.n_seqs) return ts_fail(TS_ERR_INVALID_ARG, "%s: %d rows for %d sequences", call, a.n_rows, a.n_seqs);
  if (!aligned_to(a.row_offsets, 4)) return ts_fail(TS_ERR_INVALID_ARG, "%s: misaligned row_offsets", call);
  if (!aligned_to(a.ancestors, 8)) return ts_fail(TS_ERR_INVALID_ARG, "%s: misaligned ancestors", call);
  if (a.ancestors && a.window) return ts_fail(TS_ERR_INVALID_ARG, "%s: window and ancestors exclude each other", call);
  if (!(fabsf(a.scale) < INFINITY)) return ts_fail(TS_ERR_INVALID_ARG, "%s: scale must be finite", call);
  if (a.n_rows == 0) return TS_OK;
  if (!a.q || !a.out) return ts_fail(TS_ERR_INVALID_ARG, "%s: null argument", call);
  const int64_t q_row = (int64_t)a.n_q_heads * p.head_dim;
  if (a.q_stride < q_row || a.out_stride < q_row) return ts_fail(TS_ERR_INVALID_ARG, "%s: a row stride is below its row", call);
  const int esz = ops_esz(a.dtype);
  if (!aligned_to(a.q, esz) || !aligned_to(a.out, esz) || !aligned_to(a.lse, 4)) return ts_fail(TS_ERR_INVALID_ARG, "%s: rows are not aligned to their type", call);
  const RowsCut c = rows_cut(a);
  if (c.splits > 1) {
    uint64_t need = 0;
    if ((st = ts_kv_attend_rows_workspace(a.n_seqs, a.n_rows, a.n_q_heads, p.n_kv_heads, p.head_dim, a.max_len, a.window, &need))) return st;
    need = std::max(need, (uint64_t)a.n_rows * a.n_q_heads * c.splits * (p.head_dim + 2) * 4);           // what the kernels write: never beyond the bytes given
    if (!a.workspace || a.workspace_bytes < need || !aligned_to(a.workspace, 16))
      return ts_fail(TS_ERR_INVALID_ARG, "%s: needs a 16-byte aligned workspace of %llu bytes, got %llu", call, (unsigned long long)need, (unsigned long long)a.workspace_bytes);
  }
  int dev;
  if ((st = ops_device(call, {p.k, p.v, a.cache.k_scales, a.cache.v_scales, a.table, a.lengths, a.row_offsets, a.ancestors, a.q, a.out, a.lse, c.splits > 1 ? a.workspace : nullptr},
                       stream, &dev))) return st;
  DeviceGuard on(dev);
  RowsArgs g{};
  g.a = a;
  g.scale_log2 = a.scale * 1.4426950408889634f;
  g.group = a.n_q_heads / p.n_kv_heads;
  g.chunk = c.chunk;
  g.splits = c.splits;
  g.seq_tiles = (g.group + 16 * c.nt - 1) / (16 * c.nt);
  g.part_o = (float*)a.workspace;
  g.part_ml = g.part_o + (int64_t)a.n_rows * a.n_q_heads * c.splits * p.head_dim;
  if (a.dtype == TS_DTYPE_BF16) launch_rows_q<bf16_t>(g, c, (hipStream_t)stream);
  else launch_rows_q<float>(g, c, (hipStream_t)stream);
  TS_HIP(hipGetLastError());
  return TS_OK;
}
