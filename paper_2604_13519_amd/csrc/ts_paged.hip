// One layer's step over a paged cache: rows appended with the rotary embedding applied on the way, and attention of one
// new token per sequence, split over the cache's length and joined.
#include <math.h>

#include "ts_ops.h"

// ---------------------------------------------------------------------------------
// append
//
// A workgroup takes the rows that share a page (a single row in a decoding step, up to 16 of a context) and a few
// heads: the values are transposed within a page, so a page's 16 positions of a dimension are one 32-byte (fp32: 64)
// piece, written whole.  The angle of position p and pair j is p theta^(-2 j / hd); as a number of turns it is formed and
// reduced to [-1/2, 1/2] in 64 bits, so that far positions keep their phase, and sine and cosine are taken in fp32: what is left is
// rounded to 2^-26 of a turn there, 9e-8 radians, as much as a step of fp32 sines.
//
// Bound by the start of a launch for a step's rows (one row, 8 + 32 heads of 128: 3.9 us, of which starting a launch is 2 to 3) and by HBM
// for contexts: 2040 rows of 8 + 64 heads move 80 MB (as counted) in 21.2 us, 3.8 TB/s; 2048 rows of 8 + 32 heads on whole pages 50 MB
// in 10.2 us, 4.9 TB/s.
// ---------------------------------------------------------------------------------
constexpr int APPEND_THREADS = 256, APPEND_HEADS = 32;     // heads of a workgroup at most

template <typename T> __device__ __forceinline__ float widen(T v) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(v);
  else return v;
}
// N consecutive elements in vectors
template <int N, typename T>
__device__ __forceinline__ void load_n(const T* p, float (&v)[N]) {
  uint32_t u[N * sizeof(T) / 4];
  if constexpr (N * sizeof(T) == 4) u[0] = load4(p);
  else if constexpr (N * sizeof(T) == 8) { const uint2 w = load8(p); u[0] = w.x; u[1] = w.y; }
  else
#pragma unroll
    for (int i = 0; i < (int)(N * sizeof(T) / 16); ++i) {
      const uint4 w = load16((const char*)p + 16 * i);
      u[4 * i] = w.x; u[4 * i + 1] = w.y; u[4 * i + 2] = w.z; u[4 * i + 3] = w.w;
    }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (sizeof(T) == 2) v[i] = __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
    else v[i] = __uint_as_float(u[i]);
  }
}
template <int N, typename T>
__device__ __forceinline__ void store_n(T* p, const float (&v)[N]) {
  uint32_t u[N * sizeof(T) / 4];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (sizeof(T) == 2) { if (!(i & 1)) u[i / 2] = __builtin_bit_cast(uint32_t, to_bf16x2(v[i], v[i + 1])); }
    else u[i] = __float_as_uint(v[i]);
  }
  if constexpr (N * sizeof(T) == 4) store4(p, u[0]);
  else if constexpr (N * sizeof(T) == 8) store8(p, make_uint2(u[0], u[1]));
  else
#pragma unroll
    for (int i = 0; i < (int)(N * sizeof(T) / 16); ++i) store16((char*)p + 16 * i, make_uint4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]));
}

// those of positions p0 .. p0 + N - 1 that lie in [lo, hi), in as few pieces as there are
template <int N, typename T>
__device__ __forceinline__ void store_some(T* p, int p0, int lo, int hi, const float* v) {
  if (lo <= p0 && p0 + N <= hi) {
    if constexpr (N == 1) st_from_f32(p, v[0]);
    else {
      float w[N];
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = v[i];
      store_n<N>(p, w);
    }
  } else if constexpr (N > 1) {
    if (lo < p0 + N / 2) store_some<N / 2>(p, p0, lo, hi, v);
    if (hi > p0 + N / 2) store_some<N / 2>(p + N / 2, p0 + N / 2, lo, hi, v + N / 2);
  }
}

struct AppendArgs {
  ts_kv_append_args a;
  double log2_theta;                     // rope_theta > 0
  int window, heads;                     // of a workgroup: rows it looks for pages in, heads
};

// the last sequence whose first row is not behind `row`, -1 if none: 64 offsets at a time, one per lane
__device__ __forceinline__ int seq_of_row(const int32_t* offsets, int n, int row) {
  const int lane = threadIdx.x % 64;
  int lo = 0, left = n;                  // offsets [lo, lo + left) are open; all before lo are <= row
  for (;;) {
    const int step = (left + 63) / 64;
    const int i = lane * step;
    const int c = __popcll(__ballot(i < left && offsets[lo + (i < left ? i : 0)] <= row));
    if (c == 0) return lo - 1;
    if (step == 1) return lo + c - 1;
    lo += (c - 1) * step + 1;
    left = min(step - 1, left - (c - 1) * step - 1);
    if (left <= 0) return lo - 1;
  }
}

// `cnt` rows from `row` on into slots `slot`, ... of a page, heads [head0, head1) of (queries, keys, values)
struct AppendPage { int row, cnt, slot, page, head0, head1, hq, hkv; int64_t pos; };

// Queries and keys, in pieces of VE pairs.  A thread requests all its pieces (more than four: in batches) before it stores
// one - the stores may alias the loads for all the compiler knows - and the sines are worked out while they come.
template <typename TI, typename TC, int HD>
__device__ __forceinline__ void append_turned(const AppendArgs& g, const AppendPage& at, const double* freq, float2* cs) {
  constexpr int VE = HD >= 32 && sizeof(TI) == 2 && sizeof(TC) == 2 ? 8 : 4, HALF = HD / 2, PIECES = HALF / VE, BATCH = 4;
  const ts_kv_append_args& a = g.a;
  const int tid = threadIdx.x, cnt = at.cnt, n = (min(at.head1, at.hq + at.hkv) - at.head0) * cnt * PIECES;
  const int by_cnt = (65536 + cnt - 1) / cnt;                // divides what is below 16 * APPEND_HEADS by cnt
  const bool turn = a.rope_theta > 0.f;
  for (int i0 = 0; i0 < n; i0 += BATCH * APPEND_THREADS) {
    float x[BATCH][VE], y[BATCH][VE];
    int rr[BATCH], hh[BATCH];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      if (i0 + b * APPEND_THREADS >= n) break;
      const int i = min(i0 + b * APPEND_THREADS + tid, n - 1), c = i % PIECES, hr = i / PIECES;
      hh[b] = hr * by_cnt >> 16;
      rr[b] = hr - hh[b] * cnt;
      hh[b] += at.head0;
      const int64_t row = at.row + rr[b];
      const TI* src = hh[b] < at.hq ? (const TI*)a.q + row * a.q_stride + hh[b] * HD : (const TI*)a.k + row * a.k_stride + (hh[b] - at.hq) * HD;
      load_n<VE>(src + c * VE, x[b]);
      load_n<VE>(src + HALF + c * VE, y[b]);
    }
    if (turn && i0 == 0) {
      for (int i = tid; i < cnt * HALF; i += APPEND_THREADS) {
        const double t = freq[i % HALF] * (double)(at.pos + i / HALF), rest = t - rint(t);
        float sn, c;
        sincospif(2.f * (float)rest, &sn, &c);
        cs[i] = make_float2(c, sn);
      }
      __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = i0 + b * APPEND_THREADS + tid, c = i % PIECES;
      if (i >= n) continue;
      if (turn) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float2 w = cs[rr[b] * HALF + c * VE + e];
          const float u = x[b][e] * w.x - y[b][e] * w.y;
          y[b][e] = y[b][e] * w.x + x[b][e] * w.y;
          x[b][e] = u;
        }
      }
      if (hh[b] < at.hq) {
        TI* dst = (TI*)a.q_out + (int64_t)(at.row + rr[b]) * a.q_out_stride + hh[b] * HD;
        store_n<VE>(dst + c * VE, x[b]);
        store_n<VE>(dst + HALF + c * VE, y[b]);
      } else {
        TC* dst = (TC*)a.pages.k + (((int64_t)at.page * at.hkv + (hh[b] - at.hq)) * 16 + at.slot + rr[b]) * HD;
        store_n<VE>(dst + c * VE, x[b]);
        store_n<VE>(dst + HALF + c * VE, y[b]);
      }
    }
  }
}

template <typename TI, typename TC, int HD>
__device__ __forceinline__ void append_values(const AppendArgs& g, const AppendPage& at) {
  const ts_kv_append_args& a = g.a;
  const int tid = threadIdx.x, cnt = at.cnt, slot = at.slot, row = at.row, page = at.page, hkv = at.hkv, turned = at.hq + at.hkv, head0 = at.head0, head1 = at.head1;
  // values: a thread writes the positions of a dimension, of two for rows of bf16.  All rows are requested at once (what
  // lies outside the new ones is the nearest of them, not stored); they go in vectors, cut at the ends.
  constexpr int DV = 4 / sizeof(TI), SV = 16 / sizeof(TC);
  const int val0 = max(head0, turned), end = slot + cnt;
  for (int i = tid; i < (head1 - val0) * HD / DV; i += APPEND_THREADS) {
    const int h = val0 - turned + i * DV / HD, d = i * DV % HD;
    const TI* src = (const TI*)a.v + (int64_t)row * a.v_stride + h * HD + d;
    TC* dst = (TC*)a.pages.v + (((int64_t)page * hkv + h) * HD + d) * 16;
    if (cnt == 1) {
      float w[DV];
      load_n<DV>(src, w);
#pragma unroll
      for (int e = 0; e < DV; ++e) st_from_f32(dst + e * 16 + slot, w[e]);
      continue;
    }
    float v[DV][16];
#pragma unroll
    for (int p = 0; p < 16; ++p) {
      float w[DV];
      load_n<DV>(src + (int64_t)min(max(p - slot, 0), cnt - 1) * a.v_stride, w);
#pragma unroll
      for (int e = 0; e < DV; ++e) v[e][p] = w[e];
    }
#pragma unroll
    for (int p0 = 0; p0 < 16; p0 += SV)
#pragma unroll
      for (int e = 0; e < DV; ++e) store_some<SV>(dst + e * 16 + p0, p0, slot, end, &v[e][p0]);
  }
}

// TI rows' element, TC cache's element
template <typename TI, typename TC, int HD>
__global__ __launch_bounds__(APPEND_THREADS) void k_kv_append(AppendArgs g) {
  constexpr int HALF = HD / 2;
  __shared__ float2 cs[16 * HALF];
  __shared__ double freq[HALF];
  const ts_kv_append_args& a = g.a;
  const int tid = threadIdx.x, hkv = a.pages.n_kv_heads, hq = a.q ? a.n_q_heads : 0;
  const int head0 = blockIdx.y * g.heads, turned = hq + hkv, head1 = min(head0 + g.heads, turned + hkv);
  const bool turn = a.rope_theta > 0.f && head0 < turned;
  if (turn && tid < HALF) freq[tid] = exp2(g.log2_theta * (-2.0 * tid / HD)) * 0.15915494309189535;      // turns per position

  // The page's first new row takes the others along; a workgroup takes the pages whose first new row is in its window.
  const int window1 = min((int)(blockIdx.x + 1) * g.window, a.n_rows);
  for (int row = blockIdx.x * g.window, cnt; row < window1; row += cnt) {
    cnt = 1;
    const int seq = seq_of_row(a.row_offsets, a.n_seqs + 1, row);
    if (seq < 0 || seq >= a.n_seqs) continue;
    const int first = a.row_offsets[seq], end = min(a.row_offsets[seq + 1], a.n_rows);
    const int64_t pos = (int64_t)a.lengths[seq] + row - first;
    if (pos < 0 || row >= end) continue;
    const int slot = (int)(pos & 15);
    cnt = min(16 - slot, end - row);
    if ((row != max(first, 0) && slot != 0) || pos >= (int64_t)a.table_width * 16) continue;
    const int page = a.table[(int64_t)seq * a.table_stride + pos / 16];
    if (page < 0 || page >= a.pages.n_pages) continue;
    const AppendPage at{row, cnt, slot, page, head0, head1, hq, hkv, pos};
    __syncthreads();                                         // freq is there, the last page's cs no longer read
    if (head0 < turned) append_turned<TI, TC, HD>(g, at, freq, cs);
    if (head1 > turned) append_values<TI, TC, HD>(g, at);
  }
}

// ---------------------------------------------------------------------------------
// attention of one token
//
// out = sum_p w_p v_p with w the softmax of scale (q . k_p): one pass over the keys and values with a running maximum m
// and sum l; what was accumulated is multiplied by 2^(m_old - m_new) when the maximum rises.  Bound by the bytes of the
// cache: 2 head_dim elements per position and KV head, read once for all query heads of the group.
//
// Matrix instructions without any exchange between lanes: S^T = K Q^T puts the 16 query heads of a tile on the lanes
// (lane l: head l % 16) and four keys in a lane's registers, and O^T = V^T P^T wants, as its second operand, eight
// (fp32: one) consecutive keys of a head in a lane.  Which key is which row of K's tile is free, so tile t of a block of 32 keys
// takes key 8 (m / 4) + 4 t + m % 4 as its row m: then the probabilities a lane has computed are, in place, the operand
// it needs, and the matching values are 16 contiguous bytes of the transposed page.  Maximum and sum of a head lie in
// four lanes (l, l + 16, l + 32, l + 48); nothing passes through the LDS before the waves of a workgroup are joined.
//
// bf16, 8 KV heads of 128: 8 sequences of up to 32768 tokens, 64 query heads (727 MB, as counted): 125.7 us in a kernel trace, 5.8 TB/s,
// a kernel that only reads the same bytes takes 123; one sequence of 8192, 32 query heads (34 MB): 10.6 us and 4.0 of the join in
// the trace, 12.3 both in a captured graph.  fp32, 8 sequences of 8192, 8 KV heads of 128 (537 MB): 103.6 us, 5.2 TB/s.
// ---------------------------------------------------------------------------------
constexpr int ATT_WAVES = 4, ATT_KB = 32;

struct AttendArgs {
  ts_kv_attend_args a;
  float scale_log2;                      // scores enter 2^x
  int group, tiles, chunk, splits;       // query heads per KV head, tiles of 16 of them, keys per workgroup, workgroups per sequence at most
  float* part_o;                         // [n_seqs][n_q_heads][splits][head_dim], relative to 2^m
  float* part_ml;                        // [n_seqs][n_q_heads][splits][2]
};

// positions seen by a sequence's token: [lo, hi), and where its chunks start (a block boundary)
__device__ __forceinline__ void seen_range(const ts_kv_attend_args& a, int seq, int& lo, int& hi, int& base) {
  const int64_t room = (int64_t)a.table_width * 16;
  const int len = max(0, a.lengths[seq]);                    // the window is the last of these, seen or not
  hi = min(len, a.max_len);
  if (hi > room) hi = (int)room;
  lo = a.window > 0 && len > a.window ? min(len - a.window, hi) : 0;
  base = lo & ~(ATT_KB - 1);
}

template <typename T, typename TQ, int HD>
__global__ __launch_bounds__(ATT_WAVES * 64, 2) void k_kv_attend(AttendArgs g) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int QP = BF && sizeof(TQ) == 4 ? 3 : 1;          // terms of a query
  constexpr int PP = 3;                                      // terms of a probability (bf16 caches): all of its 24 bits
  constexpr int KC = BF ? HD / 32 : (HD + 15) / 16;          // 16-byte pieces of a key per lane
  constexpr int DT = (HD + 15) / 16;                         // tiles of 16 dimensions
  constexpr int OS = DT * 16 + 4;                            // floats of a head's row in the LDS
  __shared__ float so[ATT_WAVES * 16 * OS];
  __shared__ float sm[ATT_WAVES][16], sl[ATT_WAVES][16];
  const ts_kv_attend_args& a = g.a;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, n = lane % 16, lg = lane / 16;
  // neighbours take the KV heads of the same positions: a page's heads lie side by side in memory and are read together
  int id = blockIdx.x, tile = 0;
  // Tiles of the same keys are 8 apart (fewer at the end), on one XCD, whose cache serves all but the first: 8 sequences of 8192,
  // 64 heads over one KV head 19.7 us, as neighbours 27.3.
  if (g.tiles > 1) {
    const int u0 = id / (8 * g.tiles) * 8, width = min(8, (int)(gridDim.x / g.tiles) - u0), in = id - u0 * g.tiles;
    tile = in / width;
    id = u0 + in % width;
  }
  const int hkv = a.pages.n_kv_heads, kvh = id % hkv; id /= hkv;
  const int split = id % g.splits, seq = id / g.splits;
  int lo, hi, base;
  seen_range(a, seq, lo, hi, base);
  const int64_t from = base + (int64_t)split * g.chunk;      // base and the launch's span may both be near 2^30
  if (split > 0 && from >= hi) return;                       // the join knows which splits there are
  const int k0 = (int)from, k1 = (int)min((int64_t)hi, from + g.chunk);
  const int heads = min(16, g.group - tile * 16), head0 = kvh * g.group + tile * 16;

  // the queries: lane (head n, group lg) holds the dimensions it multiplies with its keys' pieces
  uint4 q[QP][KC];
  {
    const TQ* src = (const TQ*)a.q + (int64_t)seq * a.q_stride + (int64_t)(head0 + min(n, heads - 1)) * HD;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      constexpr int E = BF ? 8 : 4;
      float x[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = (c * 4 + lg) * E + e;
        x[e] = d < HD ? widen(src[d < HD ? d : 0]) : 0.f;
      }
      if constexpr (BF) {
        uint32_t u[QP][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          ts_bf16x2 t[QP];
          split_bf16x2_nonzero<QP>(x[2 * e], x[2 * e + 1], t);
#pragma unroll
          for (int p = 0; p < QP; ++p) u[p][e] = __builtin_bit_cast(uint32_t, t[p]);
        }
#pragma unroll
        for (int p = 0; p < QP; ++p) q[p][c] = make_uint4(u[p][0], u[p][1], u[p][2], u[p][3]);
      } else {
        q[0][c] = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
      }
    }
  }

  ts_f32x4 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = ts_f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;                              // l: of this lane's keys only

  const int32_t* table = a.table + (int64_t)seq * a.table_stride;
  const char* kp = (const char*)a.pages.k;
  const char* vp = (const char*)a.pages.v;
  const int64_t head_bytes = (int64_t)16 * HD * sizeof(T), page_bytes = hkv * head_bytes;

  // A block of 32 keys: its two pages, and what a lane holds of its keys and values.
  struct Block { uint4 k[2][KC], v[BF ? 1 : 2][DT]; bool ok0, ok1; };
  auto pages_of = [&](int kb) {                              // the second may lie behind the last position
    return make_int2(kb < hi ? table[kb / 16] : -1, kb + 16 < hi ? table[kb / 16 + 1] : -1);
  };
  auto fetch = [&](Block& f, int2 pg) {                      // pages that do not exist: another is read, and masked
    f.ok0 = pg.x >= 0 && pg.x < a.pages.n_pages;
    f.ok1 = pg.y >= 0 && pg.y < a.pages.n_pages;
    const int p0 = f.ok0 ? pg.x : 0, p1 = f.ok1 ? pg.y : p0;
    const int64_t off0 = p0 * page_bytes + kvh * head_bytes, off1 = p1 * page_bytes + kvh * head_bytes;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int key = BF ? 8 * (n / 4) + 4 * t + n % 4 : 16 * t + n;
      const char* row = kp + (key < 16 ? off0 : off1) + (key % 16) * HD * (int)sizeof(T);
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const int at = (c * 4 + lg) * 16;
        if (HD * (int)sizeof(T) % 64 == 0 || at < HD * (int)sizeof(T)) f.k[t][c] = *reinterpret_cast<const uint4*>(row + at);
        else f.k[t][c] = make_uint4(0, 0, 0, 0);
      }
    }
    if constexpr (BF) {
      const char* col = vp + (lg < 2 ? off0 : off1) + (lg & 1) * 16;
#pragma unroll
      for (int d = 0; d < DT; ++d) f.v[0][d] = *reinterpret_cast<const uint4*>(col + (d * 16 + n) * 32);
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          if (HD % 16 == 0 || d * 16 + n < HD) f.v[t][d] = *reinterpret_cast<const uint4*>(vp + (t ? off1 : off0) + (d * 16 + n) * 64 + lg * 16);
          else f.v[t][d] = make_uint4(0, 0, 0, 0);
        }
    }
  };
  auto use = [&](Block& f, int kb) {
    ts_f32x4 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = ts_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        if constexpr (BF) {
#pragma unroll
          for (int p = QP - 1; p >= 0; --p)
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(ts_bf16x8, f.k[t][c]), __builtin_bit_cast(ts_bf16x8, q[p][c]), s[t], 0, 0, 0);
        } else {
          const ts_f32x4 kx = __builtin_bit_cast(ts_f32x4, f.k[t][c]), qx = __builtin_bit_cast(ts_f32x4, q[0][c]);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[e], qx[e], s[t], 0, 0, 0);
        }
      }
    }
    // this lane's keys: 8 lg + 4 t + r (fp32: 16 t + 4 lg + r) of the block
    float x[8];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[4 * t + r] = s[t][r] * g.scale_log2;
    if (!(kb >= lo && kb + ATT_KB <= k1 && f.ok0 && f.ok1)) {
      auto seen = [&](int i) {
        const int key = BF ? 8 * lg + i : 16 * (i / 4) + 4 * lg + i % 4;
        return kb + key >= lo && kb + key < k1 && (key < 16 ? f.ok0 : f.ok1);
      };
      uint32_t keep[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool in = seen(i);
        x[i] = in ? x[i] : -INFINITY;
        keep[i] = in ? 0xffffffffu : 0;
      }
      // 0 times whatever an unseen place holds is not 0
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        if constexpr (BF) {
          uint4& v = f.v[0][d];
          v.x &= (keep[0] & 0xffff) | (keep[1] & 0xffff0000u);
          v.y &= (keep[2] & 0xffff) | (keep[3] & 0xffff0000u);
          v.z &= (keep[4] & 0xffff) | (keep[5] & 0xffff0000u);
          v.w &= (keep[6] & 0xffff) | (keep[7] & 0xffff0000u);
        } else {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            uint4& v = f.v[t][d];
            v.x &= keep[4 * t]; v.y &= keep[4 * t + 1]; v.z &= keep[4 * t + 2]; v.w &= keep[4 * t + 3];
          }
        }
      }
    }
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    top = fmaxf(max_over_lane_groups(top), m);
    if (__ballot(top > m)) {                                 // the sums so far move to the new reference
      const float w = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
      l *= w;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= w;
      m = top;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = __builtin_amdgcn_exp2f(x[i] - ref);
      l += x[i];
    }
    if constexpr (BF) {
      uint32_t u[PP][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ts_bf16x2 t[PP];
        split_bf16x2_nonzero<PP>(x[2 * e], x[2 * e + 1], t);
#pragma unroll
        for (int p = 0; p < PP; ++p) u[p][e] = __builtin_bit_cast(uint32_t, t[p]);
      }
#pragma unroll
      for (int p = PP - 1; p >= 0; --p)
#pragma unroll
        for (int d = 0; d < DT; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(ts_bf16x8, f.v[0][d]),
                                                         __builtin_bit_cast(ts_bf16x8, make_uint4(u[p][0], u[p][1], u[p][2], u[p][3])), o[d], 0, 0, 0);
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int d = 0; d < DT; ++d) o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(ts_f32x4, f.v[t][d])[r], x[4 * t + r], o[d], 0, 0, 0);
    }
  };
  // One block's keys and values are on their way while another is used (two or three were no faster: 8 sequences of 8192 tokens
  // 45.0, 46.0 and 47.4 us), and the pages of the one after are known.  The
  // request is made on every path - past the end for the last block again - because the waits count the loads behind
  // the ones they wait for: with a path that requests nothing they would wait for the request as well.
  constexpr int STEP = ATT_WAVES * ATT_KB;
  const int kw = k0 + wave * ATT_KB;
  if (kw + STEP >= k1) {
    if (kw < k1) {
      Block f;
      fetch(f, pages_of(kw));
      use(f, kw);
    }
  } else if constexpr (BF || HD < 128) {
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
  } else {                                                   // 128 fp32 dimensions do not fit twice; 5.2 TB/s as it is, see above
    int2 next = pages_of(kw);
    for (int kb = kw; kb < k1; kb += STEP) {
      Block f;
      fetch(f, next);
      next = pages_of(kb + STEP);
      use(f, kb);
    }
  }

  // the four waves' parts
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (lane < 16) { sm[wave][n] = m; sl[wave][n] = l; }
#pragma unroll
  for (int d = 0; d < DT; ++d) *reinterpret_cast<ts_f32x4*>(&so[(wave * 16 + n) * OS + d * 16 + lg * 4]) = o[d];
  __syncthreads();
  for (int i = tid; i < heads * HD; i += ATT_WAVES * 64) {
    const int h = i / HD, d = i % HD;
    float top = sm[0][h];
#pragma unroll
    for (int w = 1; w < ATT_WAVES; ++w) top = fmaxf(top, sm[w][h]);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, val = 0.f;
#pragma unroll
    for (int w = 0; w < ATT_WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm[w][h] - ref);
      sum += f * sl[w][h];
      val += f * so[(w * 16 + h) * OS + d];
    }
    const int64_t row = (int64_t)seq * a.n_q_heads + head0 + h;
    if (g.splits == 1) {
      st_from_f32((TQ*)a.out + (int64_t)seq * a.out_stride + (int64_t)(head0 + h) * HD + d, sum == 0.f ? 0.f : val / sum);
      if (a.lse && d == 0) a.lse[row] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
    } else {
      g.part_o[(row * g.splits + split) * HD + d] = val;
      if (d == 0) *reinterpret_cast<float2*>(g.part_ml + (row * g.splits + split) * 2) = make_float2(top, sum);
    }
  }
}

// The join of a sequence's splits: out = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i.  A workgroup per (sequence, head):
// the weights of the splits first, into the LDS, then four dimensions a thread and the splits dealt to the 1024 / HD rows
// of threads, so that a row's reads are few and all in flight at once.  A launch of its own, 4.0 us in a kernel trace: joining in the
// last workgroup to end needs the parts written through to memory by every workgroup, and one sequence of 8192 took 62 us so, not 12.5.
constexpr int ATT_SPLITS = 512;                              // at most, see attend_cut
template <typename TQ, int HD>
__global__ __launch_bounds__(256) void k_kv_attend_join(AttendArgs g) {
  constexpr int COLS = HD / 4, ROWS = 256 / COLS;
  __shared__ float sw[ATT_SPLITS];
  __shared__ float4 sv[256];
  __shared__ float red[2][4];
  const ts_kv_attend_args& a = g.a;
  const int64_t row = blockIdx.x;
  const int seq = (int)(row / a.n_q_heads), h = (int)(row % a.n_q_heads), tid = threadIdx.x, wave = tid / 64;
  int lo, hi, base;
  seen_range(a, seq, lo, hi, base);
  const int used = max(1, min(g.splits, (hi - base + g.chunk - 1) / g.chunk));
  const float2* ml = reinterpret_cast<const float2*>(g.part_ml) + row * g.splits;
  float2 p[ATT_SPLITS / 256];
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < ATT_SPLITS / 256; ++i) {
    const int j = i * 256 + tid;
    p[i] = j < used ? ml[j] : make_float2(-INFINITY, 0.f);
    top = fmaxf(top, p[i].x);
  }
  top = wave_max(top);
  if (tid % 64 == 0) red[0][wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  const float ref = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < ATT_SPLITS / 256; ++i) {
    const int j = i * 256 + tid;
    const float f = __builtin_amdgcn_exp2f(p[i].x - ref);
    if (j < used) { sw[j] = f; sum += f * p[i].y; }
  }
  sum = wave_sum(sum);
  if (tid % 64 == 0) red[1][wave] = sum;
  __syncthreads();
  sum = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  const int d = tid % COLS, r = tid / COLS;
  const float4* part = reinterpret_cast<const float4*>(g.part_o) + row * g.splits * COLS + d;
  float4 val = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int i = r; i < used; i += ROWS) {
    const float4 v = part[(int64_t)i * COLS];
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
  st_from_f32((TQ*)a.out + (int64_t)seq * a.out_stride + (int64_t)h * HD + tid, sum == 0.f ? 0.f : out / sum);
  if (a.lse && tid == 0) a.lse[row] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------------
static ts_status check_pages(const char* call, const ts_kv_pages& p, const int32_t* table, int64_t table_stride, int32_t table_width, const int32_t* lengths,
                             int32_t n_seqs, int32_t dtype) {
  if (!p.k || !p.v || !table || !lengths) return ts_fail(TS_ERR_INVALID_ARG, "%s: null argument", call);
  if (!ops_dtype_ok(p.dtype) || !ops_dtype_ok(dtype)) return ts_fail(TS_ERR_INVALID_ARG, "%s: dtype must be TS_DTYPE_F32 or TS_DTYPE_BF16", call);
  if (p.n_pages < 1 || p.n_kv_heads < 1 || p.n_kv_heads > 65536) return ts_fail(TS_ERR_INVALID_ARG, "%s: %d pages of %d KV heads", call, p.n_pages, p.n_kv_heads);
  const int hd = p.head_dim;
  if (p.dtype == TS_DTYPE_BF16 ? hd != 64 && hd != 128 : hd != 8 && hd != 16 && hd != 32 && hd != 64 && hd != 128)
    return ts_fail(TS_ERR_INVALID_ARG, "%s: head_dim %d (bf16: 64 or 128; fp32: a power of two in [8,128])", call, hd);
  if (!aligned_to(p.k, 16) || !aligned_to(p.v, 16)) return ts_fail(TS_ERR_INVALID_ARG, "%s: pages must be 16-byte aligned", call);
  if (n_seqs < 1 || n_seqs > (1 << 20)) return ts_fail(TS_ERR_INVALID_ARG, "%s: n_seqs %d outside [1, 2^20]", call, n_seqs);
  if (table_width < 1 || table_stride < table_width) return ts_fail(TS_ERR_INVALID_ARG, "%s: page table of width %d, stride %lld", call, table_width, (long long)table_stride);
  if (!aligned_to(table, 4) || !aligned_to(lengths, 4)) return ts_fail(TS_ERR_INVALID_ARG, "%s: misaligned table or lengths", call);
  return TS_OK;
}

template <typename TI, typename TC>
static bool launch_append(const AppendArgs& g, int hd, dim3 grid, hipStream_t s) {
  switch (hd) {
    case 64: k_kv_append<TI, TC, 64><<<grid, APPEND_THREADS, 0, s>>>(g); return true;
    case 128: k_kv_append<TI, TC, 128><<<grid, APPEND_THREADS, 0, s>>>(g); return true;
  }
  if constexpr (sizeof(TC) == 4) {
    switch (hd) {
      case 8: k_kv_append<TI, TC, 8><<<grid, APPEND_THREADS, 0, s>>>(g); return true;
      case 16: k_kv_append<TI, TC, 16><<<grid, APPEND_THREADS, 0, s>>>(g); return true;
      case 32: k_kv_append<TI, TC, 32><<<grid, APPEND_THREADS, 0, s>>>(g); return true;
    }
  }
  return false;
}

extern "C" ts_status ts_kv_append(const ts_kv_append_args* args, ts_stream stream) {
  if (!args) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_append: null argument");
  const ts_kv_append_args& a = *args;
  ts_status st = check_pages("ts_kv_append", a.pages, a.table, a.table_stride, a.table_width, a.lengths, a.n_seqs, a.dtype);
  if (st) return st;
  const int hd = a.pages.head_dim, esz = ops_esz(a.dtype);
  if (a.n_rows < 0 || a.n_rows > (1 << 23)) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_append: %d rows outside [0, 2^23]", a.n_rows);
  if (!a.row_offsets || !aligned_to(a.row_offsets, 4)) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_append: null or misaligned row_offsets");
  if (!(a.rope_theta >= 0.f) || !(a.rope_theta < INFINITY)) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_append: rope_theta %g must be zero or positive", a.rope_theta);
  if ((a.q != nullptr) != (a.q_out != nullptr)) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_append: q and q_out belong together");
  if (a.q && (a.n_q_heads < 1 || a.n_q_heads > 65536)) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_append: %d query heads", a.n_q_heads);
  if (a.n_rows == 0) return TS_OK;
  if (!a.k || !a.v) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_append: null argument");
  const int64_t kv_row = (int64_t)a.pages.n_kv_heads * hd, q_row = (int64_t)a.n_q_heads * hd;
  if (a.k_stride < kv_row || a.v_stride < kv_row || (a.q && (a.q_stride < q_row || a.q_out_stride < q_row)))
    return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_append: a row stride is below its row");
  if (!aligned_to(a.k, esz) || !aligned_to(a.v, esz) || !aligned_to(a.q, esz) || !aligned_to(a.q_out, esz))
    return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_append: rows are not aligned to their type");
  int dev;
  if ((st = ops_device("ts_kv_append", {a.pages.k, a.pages.v, a.table, a.lengths, a.row_offsets, a.q, a.k, a.v, a.q_out}, stream, &dev))) return st;
  DeviceGuard on(dev);
  AppendArgs g{};
  g.a = a;
  g.log2_theta = a.rope_theta > 0.f ? log2((double)a.rope_theta) : 0.0;
  const int heads = (a.q ? a.n_q_heads : 0) + 2 * a.pages.n_kv_heads;
  // A workgroup's window, from the rows a sequence has on average: pages of one window are written one after the other, but
  // the more windows, the more workgroups only find that another takes their rows along.  bf16, 8 KV heads of 128, 32 query
  // heads, microseconds at windows 1 / 2 / 4 / 8 / 16: 512 sequences of 1 row 15 / 16 / 18 / 28 / 46, of 2 rows 29 / 20 / 23 / 26
  // / 44; 64 of 8 rows 20 / 15 / 13 / 17 / 19, of 20 rows 24 / 18 / 17 / 15 / 18; 1 of 128 rows 7.4 / 6.8 / 5.4 / 5.4 / 7.7,
  // of 512 rows 17.5 / 13.9 / 9.0 / 6.9 / 8.1, of 2048 rows 55 / 38 / 22 / 14.5 / 11.3.
  const int each = a.n_rows / a.n_seqs;
  g.window = each < 2 ? 1 : each < 8 ? 2 : each < 256 ? 4 : each < 1024 ? 8 : 16;
  // Its heads: many sequences with a few rows each are many pages with little on them, and where a page's rows go and their
  // sines are the work: 8 / 32 heads, 64 sequences of 1 row 4.8 / 5.3 us, 128 5.8 / 6.0, 256 9.2 / 7.6, 1024 29 / 20; 64 of 4
  // rows 9.7 / 10.3, 128 17 / 14, 512 43 / 32; contexts 2040 rows of 5 21 / 23, 2048 of 1 12 / 18.
  g.heads = a.n_seqs >= 128 && each < 16 ? APPEND_HEADS : 8;
  const dim3 grid((a.n_rows + g.window - 1) / g.window, (heads + g.heads - 1) / g.heads);
  hipStream_t s = (hipStream_t)stream;
  const bool in16 = a.dtype == TS_DTYPE_BF16, c16 = a.pages.dtype == TS_DTYPE_BF16;
  in16 ? c16 ? launch_append<bf16_t, bf16_t>(g, hd, grid, s) : launch_append<bf16_t, float>(g, hd, grid, s)
       : c16 ? launch_append<float, bf16_t>(g, hd, grid, s) : launch_append<float, float>(g, hd, grid, s);
  TS_HIP(hipGetLastError());
  return TS_OK;
}

// How a call is cut.  The longest sequences give a workgroup a CU: two a CU, in shorter chunks, are slower (bf16, 8 KV heads of
// 128, 4 query heads each, microseconds: 8 sequences of 2048 keys 18.1, one a CU 16.8; of 32768 191 and 183; ragged ones, up to
// 32768, 134 and 117; 16 ragged ones up to 2048 20.5 and 18.9), and so is less than one (8 ragged up to 2048: 16.8, not 12.7).
// Only where they leave chunks of 128 keys, two a CU are as fast or faster: 8 of 1024 10.0 and 10.5, one of 8192 12.5 and 14.0.
// A sequence of few keys is not cut, whose join (3 to 4) takes longer than what it saves, 1.05 per 128 keys of 256 bytes: 256 keys
// whole 6.2, cut 7.5; 384 7.3 and 7.6; 512 8.4 and 7.4; of 128 bytes 512 keys 5.8 and 7.1, 1024 7.9 and 7.0; of 512 bytes 256 keys
// 10.9 and 9.5.
// Where the keys do not divide among the CUs in units of 128, fewer workgroups than CUs are left: one sequence of 8192 keys 512
// workgroups of 128, 12.3 us, of 8193 176 of 384, 13.7; between 129 and 255 sequences x KV heads each sequence is whole, 16 of 4096 keys
// 54.8 us (4.9 TB/s), 17 64.2 (4.4), 24 74.4 (5.4), 32 96.9 (5.5).
constexpr int ATT_CUS = 256;
static int64_t attend_units(int max_len, int window) {       // of 128 keys, in the longest sequence
  const int64_t span = window > 0 && window < max_len ? (int64_t)window + ATT_KB - 1 : max_len;
  return std::max<int64_t>(1, (span + ATT_WAVES * ATT_KB - 1) / (ATT_WAVES * ATT_KB));
}
static int64_t attend_whole(int64_t n_seqs, int hq, int hkv) { return n_seqs * hkv * ((hq / hkv + 15) / 16); }
static void attend_cut(int64_t n_seqs, int hq, int hkv, int key_bytes, int max_len, int window, int* chunk, int* splits) {
  const int64_t whole = attend_whole(n_seqs, hq, hkv), units = attend_units(max_len, window);
  int64_t per = 1;                                           // units a chunk
  if (units <= (key_bytes <= 128 ? 4 : key_bytes <= 256 ? 3 : 1)) per = units;
  else if (units * whole > 2 * ATT_CUS) {
    const int64_t want = std::max<int64_t>(1, ATT_CUS / whole);
    per = (units + want - 1) / want;
  }
  *chunk = (int)(per * ATT_WAVES * ATT_KB);
  *splits = (int)((units + per - 1) / per);
}
// the most splits that this max_len or a smaller one gets
static int64_t attend_splits_room(int64_t n_seqs, int hq, int hkv, int max_len, int window) {
  return std::min(attend_units(max_len, window), std::max<int64_t>(1, 2 * ATT_CUS / attend_whole(n_seqs, hq, hkv)));
}

static ts_status check_attend(const char* call, int32_t n_seqs, int32_t hq, int32_t hkv, int32_t max_len, int32_t window) {
  if (n_seqs < 1 || n_seqs > (1 << 20)) return ts_fail(TS_ERR_INVALID_ARG, "%s: n_seqs %d outside [1, 2^20]", call, n_seqs);
  if (hkv < 1 || hkv > 65536 || hq < 1 || hq > 65536 || hq % hkv) return ts_fail(TS_ERR_INVALID_ARG, "%s: %d query heads over %d KV heads", call, hq, hkv);
  if (max_len < 0 || max_len > (1 << 30)) return ts_fail(TS_ERR_INVALID_ARG, "%s: max_len %d outside [0, 2^30]", call, max_len);
  if (window < 0) return ts_fail(TS_ERR_INVALID_ARG, "%s: window %d is negative", call, window);
  const int64_t groups = attend_whole(n_seqs, hq, hkv) * attend_splits_room(n_seqs, hq, hkv, max_len, window);
  constexpr int64_t kMost = (1 << 24) - 1;                   // workgroups of 256 whose threads a launch can count
  if (groups > kMost || (int64_t)n_seqs * hq > kMost) return ts_fail(TS_ERR_INVALID_ARG, "%s: %d sequences of %d heads are too many for one call", call, n_seqs, hq);
  return TS_OK;
}

extern "C" ts_status ts_kv_attend_workspace(int32_t n_seqs, int32_t hq, int32_t hkv, int32_t head_dim, int32_t max_len, int32_t window, uint64_t* bytes) {
  if (!bytes) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_attend_workspace: null argument");
  ts_status st = check_attend("ts_kv_attend_workspace", n_seqs, hq, hkv, max_len, window);
  if (st) return st;
  if (head_dim < 8 || head_dim > 128) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_attend_workspace: head_dim %d", head_dim);
  const int64_t room = attend_splits_room(n_seqs, hq, hkv, max_len, window);
  *bytes = room > 1 ? (uint64_t)n_seqs * hq * room * (head_dim + 2) * 4 : 0;
  return TS_OK;
}

template <typename T, typename TQ, int HD>
static void launch_attend(const AttendArgs& g, hipStream_t s) {
  const ts_kv_attend_args& a = g.a;
  k_kv_attend<T, TQ, HD><<<(uint32_t)((int64_t)a.n_seqs * a.pages.n_kv_heads * g.tiles * g.splits), ATT_WAVES * 64, 0, s>>>(g);
  if (g.splits > 1) k_kv_attend_join<TQ, HD><<<(uint32_t)((int64_t)a.n_seqs * a.n_q_heads), 256, 0, s>>>(g);
}
template <typename TQ>
static void launch_attend_q(const AttendArgs& g, hipStream_t s) {
  const int hd = g.a.pages.head_dim;
  if (g.a.pages.dtype == TS_DTYPE_BF16) {
    if (hd == 64) launch_attend<bf16_t, TQ, 64>(g, s);
    else launch_attend<bf16_t, TQ, 128>(g, s);
  } else {
    if (hd == 8) launch_attend<float, TQ, 8>(g, s);
    else if (hd == 16) launch_attend<float, TQ, 16>(g, s);
    else if (hd == 32) launch_attend<float, TQ, 32>(g, s);
    else if (hd == 64) launch_attend<float, TQ, 64>(g, s);
    else launch_attend<float, TQ, 128>(g, s);
  }
}

extern "C" ts_status ts_kv_attend(const ts_kv_attend_args* args, ts_stream stream) {
  if (!args) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_attend: null argument");
  const ts_kv_attend_args& a = *args;
  ts_status st = check_pages("ts_kv_attend", a.pages, a.table, a.table_stride, a.table_width, a.lengths, a.n_seqs, a.dtype);
  if (st) return st;
  if ((st = check_attend("ts_kv_attend", a.n_seqs, a.n_q_heads, a.pages.n_kv_heads, a.max_len, a.window))) return st;
  if (!a.q || !a.out) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_attend: null argument");
  const int64_t q_row = (int64_t)a.n_q_heads * a.pages.head_dim;
  if (a.q_stride < q_row || a.out_stride < q_row) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_attend: a row stride is below its row");
  const int esz = ops_esz(a.dtype);
  if (!aligned_to(a.q, esz) || !aligned_to(a.out, esz) || !aligned_to(a.lse, 4)) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_attend: rows are not aligned to their type");
  if (!(fabsf(a.scale) < INFINITY)) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_attend: scale must be finite");
  AttendArgs g{};
  g.a = a;
  attend_cut(a.n_seqs, a.n_q_heads, a.pages.n_kv_heads, a.pages.head_dim * ops_esz(a.pages.dtype), a.max_len, a.window, &g.chunk, &g.splits);
  if (g.splits > 1) {
    uint64_t need = 0;
    if ((st = ts_kv_attend_workspace(a.n_seqs, a.n_q_heads, a.pages.n_kv_heads, a.pages.head_dim, a.max_len, a.window, &need))) return st;
    if (!a.workspace || a.workspace_bytes < need || !aligned_to(a.workspace, 16))
      return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_attend: needs a 16-byte aligned workspace of %llu bytes, got %llu", (unsigned long long)need, (unsigned long long)a.workspace_bytes);
  }
  int dev;
  if ((st = ops_device("ts_kv_attend", {a.pages.k, a.pages.v, a.table, a.lengths, a.q, a.out, a.lse, g.splits > 1 ? a.workspace : nullptr}, stream, &dev))) return st;
  DeviceGuard on(dev);
  g.scale_log2 = a.scale * 1.4426950408889634f;
  g.group = a.n_q_heads / a.pages.n_kv_heads;
  g.tiles = (g.group + 15) / 16;
  g.part_o = (float*)a.workspace;
  g.part_ml = g.part_o + (int64_t)a.n_seqs * a.n_q_heads * g.splits * a.pages.head_dim;
  if (a.dtype == TS_DTYPE_BF16) launch_attend_q<bf16_t>(g, (hipStream_t)stream);
  else launch_attend_q<float>(g, (hipStream_t)stream);
  TS_HIP(hipGetLastError());
  return TS_OK;
}
