// Rows into and out of a paged cache of any type: appended with a norm of each head and a rotation of any layout in the same
// pass, quantised to 8 bits where the pages are, and read back.
#include "ts_paged.h"

// ---------------------------------------------------------------------------------
// append
//
// A workgroup takes the rows that share a page (up to 16) and a few heads.  LPV lanes hold a head's row, VE values each: the mean of
// squares, and the largest magnitude for 8 bits, are sums and maxima over them.  A value's partner of the rotation is its
// neighbour, in the lane, or half of rope_dim away, in another lane: normed rows pass through the LDS of their wave.  Angles are
// formed and reduced in 64 bits as turns, sine and cosine taken in fp32, once per row and pair for all heads of the workgroup.
// Values are transposed within a page; 8-bit ones are first quantised by rows, into the LDS, since a row's scale is needed
// before its first byte.
//
// 8 + 32 heads of 128, bf16: a token's row 4.5 us, with norms 5.1, into 8-bit pages 4.9 (ts_kv_append 3.9): the launch and three dependent trips to
// memory; 2048 rows on whole pages 13.0, 16.1 and 16.0 (10.4): 50 MB at 3.1 TB/s.  1938 rows of 5 sequences, 8 + 64 heads, 8-bit: 32.5 us for
// 76 MB, 2.3 TB/s.  ts_kv_append moves 79 MB of the same rows in 21.2, with the same pages begun and ended by parts and the same trips for offsets, length,
// page and rows, so these are not what makes the difference.  What it has beside them: pieces of at most four heads on their way in place of all,
// a pair's sines read one by one (conflicts are half of the LDS cycles), and for 8 bits two barriers and a pass through the
// LDS.  Their shares were not measured.  Four, eight and sixteen heads a workgroup, with the reading back:
// 49.7, 40.8 and 45.0; rows reduced through the LDS 37 for 33.
// ---------------------------------------------------------------------------------
constexpr int RA_THREADS = 256, RA_HEADS = 8;

struct AppendAnyArgs {
  ts_kv_append_norm_rope_args a;
  double log2_theta;
  int window;                            // rows a workgroup looks for pages in
  bool turn;                             // rope_dim > 0 and frequencies that are not all zero
};

// Rows of LPV lanes (2 .. 32) are reduced without the LDS: within four lanes, within 8 and 16 by their mirrors, and 32 by a swap.
template <int CTRL> __device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t other_16(uint32_t v) {    // of lane l ^ 16
  const auto x = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return threadIdx.x & 16 ? x[0] : x[1];
}
template <int LPV, typename F>
__device__ __forceinline__ uint32_t over(uint32_t v, F join) {
  if constexpr (LPV > 1) v = join(v, moved<0xb1>(v));
  if constexpr (LPV > 2) v = join(v, moved<0x4e>(v));
  if constexpr (LPV > 4) v = join(v, moved<0x141>(v));
  if constexpr (LPV > 8) v = join(v, moved<0x140>(v));
  if constexpr (LPV > 16) v = join(v, other_16(v));
  return v;
}
template <int LPV>
__device__ __forceinline__ float sum_over(float v) {
  return __uint_as_float(over<LPV>(__float_as_uint(v), [](uint32_t x, uint32_t y) { return __float_as_uint(__uint_as_float(x) + __uint_as_float(y)); }));
}
template <int LPV>
__device__ __forceinline__ uint32_t max_over(uint32_t v) {
  return over<LPV>(v, [](uint32_t x, uint32_t y) { return max(x, y); });
}
// the bits of the largest magnitude of a row: magnitudes order like their bits, NaN above infinity
template <int LPV, int VE>
__device__ __forceinline__ uint32_t top_bits(const float (&x)[VE]) {
  uint32_t t = 0;
#pragma unroll
  for (int e = 0; e < VE; ++e) t = max(t, __float_as_uint(x[e]) & 0x7fffffffu);
  return max_over<LPV>(t);
}
template <int VE>
__device__ __forceinline__ void to_codes(const float (&x)[VE], uint32_t byte, uint32_t (&w)[VE / 4]) {
  const float inv = __uint_as_float((254u - min(byte, 253u)) << 23);
#pragma unroll
  for (int e = 0; e < VE; e += 4) w[e / 4] = byte == 255 ? 0x7f7f7f7fu : f32_to_e4m3(x[e] * inv, x[e + 1] * inv, x[e + 2] * inv, x[e + 3] * inv);
}

// the value of the lane half a row of LPV lanes away
template <int LPV>
__device__ __forceinline__ float other_half(float v) {
  const uint32_t u = __float_as_uint(v);
  if constexpr (LPV == 32) return __uint_as_float(other_16(u));
  else if constexpr (LPV == 16) return __uint_as_float(moved<0x128>(u));             // rotated by 8 within 16
  else if constexpr (LPV == 8) return __uint_as_float(moved<0x1b>(moved<0x141>(u))); // mirrored within 8, and back within 4
  else if constexpr (LPV == 4) return __uint_as_float(moved<0x4e>(u));
  else return __uint_as_float(moved<0xb1>(u));
}

template <typename TI, typename TC, int HD>
struct AppendAny {
  static constexpr int VE = sizeof(TI) == 2 ? 8 : 4, LPV = HD / VE, VECS = RA_THREADS / LPV, BATCH = 4, HALF = HD / 2;
  static constexpr bool E8 = sizeof(TC) == 1;
  float2 cs[16 * HALF];
  double freq[HALF];
  union {
    float x[RA_THREADS / 64][64 * VE];           // normed rows of a wave
    uint8_t v[E8 ? RA_HEADS * 16 * HD : 1];      // quantised values, [head][position][dimension]
  };
};

// Queries and keys.  A thread keeps its row of the page and its place in the head and goes through the heads, so that its sines are
// read once; several heads' pieces are requested before the first is worked on.
template <typename TI, typename TC, int HD>
__device__ __forceinline__ void any_turned(const AppendAnyArgs& g, const AppendPage& at, AppendAny<TI, TC, HD>& s) {
  typedef AppendAny<TI, TC, HD> S;
  constexpr int VE = S::VE, LPV = S::LPV, HALF = S::HALF, BATCH = S::BATCH, VECS = S::VECS;
  const ts_kv_append_norm_rope_args& a = g.a;
  const int tid = threadIdx.x, cnt = at.cnt, n = min(at.head1, at.hq + at.hkv) - at.head0;
  const int lane = tid % 64, c = tid % LPV, d0 = c * VE, rd = a.rope_dim, rh = rd / 2, vec = tid / LPV;
  const bool whole = rd % (2 * VE) == 0;                     // a lane's partners are one lane's
  float* mine = s.x[tid / 64] + lane / LPV * HD;
  auto gains = [&](const void* p, float (&v)[VE]) {
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] = a.norm_dtype == TS_DTYPE_BF16 ? bf16_to_f32(((const bf16_t*)p)[d0 + e]) : ((const float*)p)[d0 + e];
  };
  float gq[VE], gk[VE];
  if (a.q_norm && at.head0 < at.hq) gains(a.q_norm, gq);
  if (a.k_norm && at.head1 > at.hq) gains(a.k_norm, gk);
  const int row_step = min(cnt, VECS), head_step = VECS / row_step;                   // rows and heads at once
  const int r0 = vec % row_step, h0 = vec / row_step;
  bool first = true;
  for (int rb = 0; rb < cnt; rb += row_step) {
    const int r = min(rb + r0, cnt - 1);
    const int64_t row = at.row + r;
    float cs[VE], sn[VE];
    for (int hb = 0; hb < n; hb += BATCH * head_step) {
      float x[BATCH][VE];
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        if (hb + b * head_step >= n) break;
        const int h = at.head0 + min(hb + b * head_step + h0, n - 1);
        load_n<VE>((h < at.hq ? (const TI*)a.q + row * a.q_stride + (int64_t)h * HD : (const TI*)a.k + row * a.k_stride + (int64_t)(h - at.hq) * HD) + d0, x[b]);
      }
      if (g.turn && first) {                                 // while the first pieces come
        for (int i = tid; i < cnt * rh; i += RA_THREADS) {
          const int ri = i / rh, j = i - ri * rh;
          const int64_t p = a.positions ? a.positions[at.row + ri] : at.pos + ri;
          const double t = s.freq[j] * (double)p, rest = t - rint(t);
          float si, co;
          sincospif(2.f * (float)rest, &si, &co);
          s.cs[ri * HALF + j] = make_float2(co * a.rope_magnitude, si * a.rope_magnitude);
        }
        __syncthreads();
      }
      first = false;
      if (g.turn && hb == 0) {                               // y = x cs + partner sn
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const int d = d0 + e, j = a.rope_pairs ? d / 2 : d < rh ? d : d - rh;
          const float2 w = d < rd ? s.cs[r * HALF + j] : make_float2(1.f, 0.f);
          cs[e] = w.x;
          sn[e] = (a.rope_pairs ? e % 2 == 0 : d < rh) ? -w.y : w.y;
        }
      }
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        if (hb + b * head_step >= n) break;
        const int hi = hb + b * head_step + h0, h = at.head0 + min(hi, n - 1);
        const bool is_q = h < at.hq, there = hi < n && rb + r0 < cnt && h0 < head_step;
        float (&v)[VE] = x[b];
        if (a.q_norm || a.k_norm) {
          const bool normed = is_q ? a.q_norm != nullptr : a.k_norm != nullptr;      // all lanes of a row go one way
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < VE; ++e) ss += v[e] * v[e];
          const float rs = rsqrtf(sum_over<LPV>(ss) * (1.f / HD) + a.norm_eps);
          if (normed) {
#pragma unroll
            for (int e = 0; e < VE; ++e) v[e] = v[e] * rs * (is_q ? gq[e] : gk[e]);
          }
        }
        if (g.turn) {
          float o[VE];                                       // the partners
          if (a.rope_pairs) {
#pragma unroll
            for (int e = 0; e < VE; ++e) o[e] = v[e ^ 1];
          } else if (whole && rd == HD && LPV > 1) {
#pragma unroll
            for (int e = 0; e < VE; ++e) o[e] = other_half<LPV>(v[e]);
          } else {
            // one wave writes and reads here, and its LDS accesses are done in order
#pragma unroll
            for (int e = 0; e < VE; e += 4) *reinterpret_cast<float4*>(mine + d0 + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
            __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int e = 0; e < VE; ++e) {
              const int d = d0 + e;
              o[e] = d < rd ? mine[d < rh ? d + rh : d - rh] : 0.f;
            }
            __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");
          }
#pragma unroll
          for (int e = 0; e < VE; ++e)                       // beyond rope_dim the value itself, whatever lies in the other lane
            v[e] = d0 + e < rd ? v[e] * cs[e] + o[e] * sn[e] : v[e];
        }
        if constexpr (S::E8) {
          const uint32_t byte = scale_byte(top_bits<LPV>(v));
          if (there && !is_q) {
            const int64_t at16 = ((int64_t)at.page * at.hkv + (h - at.hq)) * 16 + at.slot + r;
            uint32_t w[VE / 4];
            to_codes(v, byte, w);
            uint8_t* dst = (uint8_t*)a.cache.pages.k + at16 * HD + d0;
            if constexpr (VE == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t*>(dst) = w[0];
            if (c == 0) a.cache.k_scales[at16] = (uint8_t)byte;
          }
        } else if (there && !is_q) {
          store_n<VE>((TC*)a.cache.pages.k + (((int64_t)at.page * at.hkv + (h - at.hq)) * 16 + at.slot + r) * HD + d0, v);
        }
        if (there && is_q) store_n<VE>((TI*)a.q_out + row * a.q_out_stride + (int64_t)h * HD + d0, v);
      }
    }
  }
}

// bytes [lo, hi) of the sixteen in w, in as few pieces as there are
template <int N>
__device__ __forceinline__ void store_bytes(uint8_t* p, int p0, int lo, int hi, const uint32_t* w) {
  if (hi <= p0 || lo >= p0 + N) return;
  if (lo <= p0 && p0 + N <= hi) {
    if constexpr (N == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (N == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else if constexpr (N == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else if constexpr (N == 2) *reinterpret_cast<uint16_t*>(p) = (uint16_t)(w[0] >> p0 % 4 * 8);
    else *p = (uint8_t)(w[0] >> p0 % 4 * 8);
  } else if constexpr (N > 1) {
    store_bytes<N / 2>(p, p0, lo, hi, w);
    store_bytes<N / 2>(p + N / 2, p0 + N / 2, lo, hi, N >= 8 ? w + N / 8 : w);
  }
}

// values into 8-bit pages
template <typename TI, int HD>
__device__ __forceinline__ void any_values8(const AppendAnyArgs& g, const AppendPage& at, AppendAny<TI, e4m3_t, HD>& s) {
  typedef AppendAny<TI, e4m3_t, HD> S;
  constexpr int VE = S::VE, LPV = S::LPV, BATCH = S::BATCH;
  const ts_kv_append_norm_rope_args& a = g.a;
  const int tid = threadIdx.x, cnt = at.cnt, turned = at.hq + at.hkv, val0 = max(at.head0, turned), n = (at.head1 - val0) * cnt;
  const int d0 = tid % LPV * VE;
  uint8_t* vp = (uint8_t*)a.cache.pages.v;
  __syncthreads();                                           // the normed rows' place is no longer read
  for (int i0 = 0; i0 < n; i0 += BATCH * S::VECS) {
    float x[BATCH][VE];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      if (i0 + b * S::VECS >= n) break;
      const int i = min(i0 + b * S::VECS + tid / LPV, n - 1), h = i / cnt;
      load_n<VE>((const TI*)a.v + (int64_t)(at.row + i - h * cnt) * a.v_stride + (int64_t)(val0 - turned + h) * HD + d0, x[b]);
    }
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = i0 + b * S::VECS + tid / LPV, h = i / cnt, r = i - h * cnt;
      if (i0 + b * S::VECS >= n) break;
      const uint32_t byte = scale_byte(top_bits<LPV>(x[b]));
      if (i >= n) continue;
      uint32_t w[VE / 4];
      to_codes(x[b], byte, w);
      const int64_t head = (int64_t)at.page * at.hkv + (val0 - turned + h);
      if (d0 == 0) a.cache.v_scales[head * 16 + at.slot + r] = (uint8_t)byte;
      if (cnt == 1) {
#pragma unroll
        for (int e = 0; e < VE; ++e) vp[(head * HD + d0 + e) * 16 + at.slot] = (uint8_t)(w[e / 4] >> e % 4 * 8);
      } else {
        uint8_t* to = s.v + (h * 16 + at.slot + r) * HD + d0;
        if constexpr (VE == 8) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(to) = w[0];
      }
    }
  }
  if (cnt == 1) return;
  __syncthreads();
  // four dimensions a thread: sixteen positions of them, transposed by bytes
  for (int i = tid; i < (at.head1 - val0) * HD / 4; i += RA_THREADS) {
    const int h = i * 4 / HD, d = i * 4 % HD;
    uint32_t w[4][4];
#pragma unroll
    for (int p = 0; p < 16; p += 4) {
      const uint8_t* from = s.v + (h * 16 + p) * HD + d;
      const uint32_t r0 = *(const uint32_t*)from, r1 = *(const uint32_t*)(from + HD), r2 = *(const uint32_t*)(from + 2 * HD), r3 = *(const uint32_t*)(from + 3 * HD);
      const uint32_t lo01 = __builtin_amdgcn_perm(r1, r0, 0x05010400u), hi01 = __builtin_amdgcn_perm(r1, r0, 0x07030602u);      // bytes 0 0 1 1, 2 2 3 3
      const uint32_t lo23 = __builtin_amdgcn_perm(r3, r2, 0x05010400u), hi23 = __builtin_amdgcn_perm(r3, r2, 0x07030602u);
      w[0][p / 4] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u);
      w[1][p / 4] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
      w[2][p / 4] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u);
      w[3][p / 4] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
    }
    uint8_t* dst = vp + (((int64_t)at.page * at.hkv + (val0 - turned + h)) * HD + d) * 16;
#pragma unroll
    for (int e = 0; e < 4; ++e) store_bytes<16>(dst + 16 * e, 0, at.slot, at.slot + cnt, w[e]);
  }
}

template <typename TI, typename TC, int HD>
__global__ __launch_bounds__(RA_THREADS) void k_kv_append_any(AppendAnyArgs g) {
  __shared__ AppendAny<TI, TC, HD> s;
  const ts_kv_append_norm_rope_args& a = g.a;
  const int tid = threadIdx.x, hkv = a.cache.pages.n_kv_heads, hq = a.q ? a.n_q_heads : 0;
  const int head0 = blockIdx.y * RA_HEADS, turned = hq + hkv, head1 = min(head0 + RA_HEADS, turned + hkv);
  if (g.turn && head0 < turned && tid < a.rope_dim / 2)      // turns per position
    s.freq[tid] = (a.rope_freqs ? (double)a.rope_freqs[tid] : exp2(g.log2_theta * (-2.0 * tid / a.rope_dim))) * 0.15915494309189535;

  // the page's first new row takes the others along; a workgroup takes the pages whose first new row is in its window
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
    if (page < 0 || page >= a.cache.pages.n_pages) continue;
    const AppendPage at{row, cnt, slot, page, head0, head1, hq, hkv, pos};
    __syncthreads();                                         // freq is there, the last page's LDS contents no longer read
    if (head0 < turned) any_turned<TI, TC, HD>(g, at, s);
    if (head1 > turned) {
      if constexpr (sizeof(TC) == 1) any_values8<TI, HD>(g, at, s);
      else append_values<TI, TC, HD>(a.v, a.v_stride, a.cache.pages.v, at);
    }
  }
}

// ---------------------------------------------------------------------------------
// read: the way back.  A workgroup takes the positions of a page and a few heads, keys first; a thread of the values takes all positions
// of a few dimensions, so that a wave's rows are written in long pieces.  Bound by HBM: 16000 positions of 8 8-bit heads of 128 (99 MB)
// 19.6 us, 5.0 TB/s, a copy's rate.
// ---------------------------------------------------------------------------------
struct ReadArgs {
  ts_kv_read_args a;
  int window;
};

template <typename TC, typename TO, int HD>
__global__ __launch_bounds__(RA_THREADS) void k_kv_read(ReadArgs g) {
  constexpr int VE = sizeof(TC) == 1 && sizeof(TO) == 2 ? 8 : 4, PIECES = HD / VE, DV = 4 / sizeof(TC);
  const ts_kv_read_args& a = g.a;
  const int tid = threadIdx.x, hkv = a.cache.pages.n_kv_heads;
  const int head0 = blockIdx.y * RA_HEADS, head1 = min(head0 + RA_HEADS, 2 * hkv);
  const int window1 = min((int)(blockIdx.x + 1) * g.window, a.n_rows);
  auto none = [&](int row0, int rows) {                      // rows that are no position
    if (!a.zero_rest) return;
    for (int i = tid; i < rows * (head1 - head0) * HD; i += RA_THREADS) {
      const int d = i % HD, hr = i / HD, h = head0 + hr % (head1 - head0), r = hr / (head1 - head0);
      if (h < hkv) { if (a.k_out) st_from_f32((TO*)a.k_out + (int64_t)(row0 + r) * a.k_stride + (int64_t)h * HD + d, 0.f); }
      else if (a.v_out) st_from_f32((TO*)a.v_out + (int64_t)(row0 + r) * a.v_stride + (int64_t)(h - hkv) * HD + d, 0.f);
    }
  };
  for (int row = blockIdx.x * g.window, cnt; row < window1; row += cnt) {
    cnt = 1;
    const int seq = seq_of_row(a.row_offsets, a.n_seqs + 1, row);
    if (seq < 0 || seq >= a.n_seqs) { none(row, 1); continue; }
    const int first = a.row_offsets[seq], end = min(a.row_offsets[seq + 1], a.n_rows);
    const int64_t pos = (a.starts ? (int64_t)a.starts[seq] : 0) + row - first;
    if (pos < 0 || row >= end) { none(row, 1); continue; }
    const int slot = (int)(pos & 15);
    cnt = min(16 - slot, end - row);
    if (row != max(first, 0) && slot != 0) continue;         // another window's
    if (pos >= (int64_t)a.table_width * 16) { none(row, cnt); continue; }
    const int page = a.table[(int64_t)seq * a.table_stride + pos / 16];
    if (page < 0 || page >= a.cache.pages.n_pages) { none(row, cnt); continue; }
    if (a.k_out && head0 < hkv) {
      const int n = (min(head1, hkv) - head0) * cnt * PIECES;
      for (int i = tid; i < n; i += RA_THREADS) {
        const int c = i % PIECES, hr = i / PIECES, h = head0 + hr / cnt, r = hr % cnt;
        const int64_t at16 = ((int64_t)page * hkv + h) * 16 + slot + r;
        float v[VE];
        if constexpr (sizeof(TC) == 1) {
          const uint8_t* src = (const uint8_t*)a.cache.pages.k + at16 * HD + c * VE;
          const float scale = scale_at<0>(a.cache.k_scales[at16]);
#pragma unroll
          for (int e = 0; e < VE; e += 4) e4m3_to_f32(*(const uint32_t*)(src + e), scale, v + e);
        } else {
          load_n<VE>((const TC*)a.cache.pages.k + at16 * HD + c * VE, v);
        }
        store_n<VE>((TO*)a.k_out + (int64_t)(row + r) * a.k_stride + (int64_t)h * HD + c * VE, v);
      }
    }
    if (a.v_out && head1 > hkv) {
      const int val0 = max(head0, hkv) - hkv;
      for (int i = tid; i < (head1 - hkv - val0) * HD / DV; i += RA_THREADS) {
        const int h = val0 + i * DV / HD, d = i * DV % HD;
        const int64_t head = (int64_t)page * hkv + h;
        float v[DV][16];
        ts_u32x4 sc = {0, 0, 0, 0};
        if constexpr (sizeof(TC) == 1) sc = *reinterpret_cast<const ts_u32x4*>(a.cache.v_scales + head * 16);
#pragma unroll
        for (int e = 0; e < DV; ++e) {
          if constexpr (sizeof(TC) == 1) {
            const ts_u32x4 w = *reinterpret_cast<const ts_u32x4*>((const char*)a.cache.pages.v + (head * HD + d + e) * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) e4m3_to_f32(w[i], sc[i], v[e] + 4 * i);
          } else {
            load_n<16>((const TC*)a.cache.pages.v + (head * HD + d + e) * 16, v[e]);
          }
        }
        TO* dst = (TO*)a.v_out + (int64_t)row * a.v_stride + (int64_t)h * HD + d;
#pragma unroll
        for (int p = 0; p < 16; ++p) {
          if (p < slot || p >= slot + cnt) continue;
          float w[DV];
#pragma unroll
          for (int e = 0; e < DV; ++e) w[e] = v[e][p];
          TO* to = dst + (int64_t)(p - slot) * a.v_stride;
          if constexpr (DV * sizeof(TO) >= 4) store_n<DV>(to, w);
          else st_from_f32(to, w[0]);
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------------
// Rows of a window.  One sequence of 512 rows, 8 + 32 heads of 128: windows of 8 10.1 us, of 16 8.7; of 2048 rows the same.
static int window_of(int n_rows, int n_seqs) {
  const int each = n_rows / n_seqs;
  return each < 2 ? 1 : each < 8 ? 2 : each < 256 ? 4 : 16;
}

template <typename TI>
static void launch_append_any(const AppendAnyArgs& g, dim3 grid, hipStream_t s) {
  const ts_kv_pages& p = g.a.cache.pages;
#define TS_APPEND_ANY(TC, HD) if (p.head_dim == HD) return k_kv_append_any<TI, TC, HD><<<grid, RA_THREADS, 0, s>>>(g)
  if (p.dtype == TS_DTYPE_E4M3) { TS_APPEND_ANY(e4m3_t, 64); TS_APPEND_ANY(e4m3_t, 128); }
  else if (p.dtype == TS_DTYPE_BF16) { TS_APPEND_ANY(bf16_t, 64); TS_APPEND_ANY(bf16_t, 128); }
  else { TS_APPEND_ANY(float, 8); TS_APPEND_ANY(float, 16); TS_APPEND_ANY(float, 32); TS_APPEND_ANY(float, 64); TS_APPEND_ANY(float, 128); }
#undef TS_APPEND_ANY
}

extern "C" ts_status ts_kv_append_norm_rope(const ts_kv_append_norm_rope_args* args, ts_stream stream) {
  const char* call = "ts_kv_append_norm_rope";
  if (!args) return ts_fail(TS_ERR_INVALID_ARG, "%s: null argument", call);
  const ts_kv_append_norm_rope_args& a = *args;
  const ts_kv_pages& p = a.cache.pages;
  ts_status st = check_kv_pages_any(call, a.cache, a.table, a.table_stride, a.table_width, a.lengths, a.n_seqs, a.dtype);
  if (st) return st;
  const int hd = p.head_dim, esz = ops_esz(a.dtype);
  if (a.n_rows < 0 || a.n_rows > (1 << 23)) return ts_fail(TS_ERR_INVALID_ARG, "%s: %d rows outside [0, 2^23]", call, a.n_rows);
  if (!a.row_offsets || !aligned_to(a.row_offsets, 4)) return ts_fail(TS_ERR_INVALID_ARG, "%s: null or misaligned row_offsets", call);
  if (!aligned_to(a.positions, 4)) return ts_fail(TS_ERR_INVALID_ARG, "%s: misaligned positions", call);
  if (!(a.rope_theta >= 0.f) || !(a.rope_theta < INFINITY)) return ts_fail(TS_ERR_INVALID_ARG, "%s: rope_theta %g must be zero or positive", call, a.rope_theta);
  if (a.rope_dim < 0 || a.rope_dim > hd || a.rope_dim % 2) return ts_fail(TS_ERR_INVALID_ARG, "%s: rope_dim %d must be even and in [0, %d]", call, a.rope_dim, hd);
  if (!aligned_to(a.rope_freqs, 4)) return ts_fail(TS_ERR_INVALID_ARG, "%s: misaligned rope_freqs", call);
  if (!(fabsf(a.rope_magnitude) < INFINITY)) return ts_fail(TS_ERR_INVALID_ARG, "%s: rope_magnitude must be finite", call);
  if (a.q_norm || a.k_norm) {
    if (!ops_dtype_ok(a.norm_dtype)) return ts_fail(TS_ERR_INVALID_ARG, "%s: norm_dtype must be TS_DTYPE_F32 or TS_DTYPE_BF16", call);
    if (!(a.norm_eps >= 0.f) || !(a.norm_eps < INFINITY)) return ts_fail(TS_ERR_INVALID_ARG, "%s: norm_eps %g must be zero or positive", call, a.norm_eps);
    if (!aligned_to(a.q_norm, ops_esz(a.norm_dtype)) || !aligned_to(a.k_norm, ops_esz(a.norm_dtype))) return ts_fail(TS_ERR_INVALID_ARG, "%s: gains are not aligned to their type", call);
  }
  if ((a.q != nullptr) != (a.q_out != nullptr)) return ts_fail(TS_ERR_INVALID_ARG, "%s: q and q_out belong together", call);
  if (a.q && (a.n_q_heads < 1 || a.n_q_heads > 65536)) return ts_fail(TS_ERR_INVALID_ARG, "%s: %d query heads", call, a.n_q_heads);
  if (a.n_rows == 0) return TS_OK;
  if (!a.k || !a.v) return ts_fail(TS_ERR_INVALID_ARG, "%s: null argument", call);
  const int64_t kv_row = (int64_t)p.n_kv_heads * hd, q_row = (int64_t)a.n_q_heads * hd;
  if (a.k_stride < kv_row || a.v_stride < kv_row || (a.q && (a.q_stride < q_row || a.q_out_stride < q_row)))
    return ts_fail(TS_ERR_INVALID_ARG, "%s: a row stride is below its row", call);
  if (!aligned_to(a.k, esz) || !aligned_to(a.v, esz) || !aligned_to(a.q, esz) || !aligned_to(a.q_out, esz))
    return ts_fail(TS_ERR_INVALID_ARG, "%s: rows are not aligned to their type", call);
  int dev;
  if ((st = ops_device(call, {p.k, p.v, a.cache.k_scales, a.cache.v_scales, a.table, a.lengths, a.row_offsets, a.positions, a.q, a.k, a.v, a.q_out, a.q_norm, a.k_norm, a.rope_freqs},
                       stream, &dev))) return st;
  DeviceGuard on(dev);
  AppendAnyArgs g{};
  g.a = a;
  g.turn = a.rope_dim > 0 && (a.rope_freqs || a.rope_theta > 0.f);
  g.log2_theta = a.rope_theta > 0.f ? log2((double)a.rope_theta) : 0.0;
  g.window = window_of(a.n_rows, a.n_seqs);
  const int heads = (a.q ? a.n_q_heads : 0) + 2 * p.n_kv_heads;
  const dim3 grid((a.n_rows + g.window - 1) / g.window, (heads + RA_HEADS - 1) / RA_HEADS);
  if (a.dtype == TS_DTYPE_BF16) launch_append_any<bf16_t>(g, grid, (hipStream_t)stream);
  else launch_append_any<float>(g, grid, (hipStream_t)stream);
  TS_HIP(hipGetLastError());
  return TS_OK;
}

template <typename TO>
static void launch_read(const ReadArgs& g, dim3 grid, hipStream_t s) {
  const ts_kv_pages& p = g.a.cache.pages;
#define TS_READ(TC, HD) if (p.head_dim == HD) return k_kv_read<TC, TO, HD><<<grid, RA_THREADS, 0, s>>>(g)
  if (p.dtype == TS_DTYPE_E4M3) { TS_READ(e4m3_t, 64); TS_READ(e4m3_t, 128); }
  else if (p.dtype == TS_DTYPE_BF16) { TS_READ(bf16_t, 64); TS_READ(bf16_t, 128); }
  else { TS_READ(float, 8); TS_READ(float, 16); TS_READ(float, 32); TS_READ(float, 64); TS_READ(float, 128); }
#undef TS_READ
}

extern "C" ts_status ts_kv_read(const ts_kv_read_args* args, ts_stream stream) {
  const char* call = "ts_kv_read";
  if (!args) return ts_fail(TS_ERR_INVALID_ARG, "%s: null argument", call);
  const ts_kv_read_args& a = *args;
  const ts_kv_pages& p = a.cache.pages;
  ts_status st = check_kv_pages_any(call, a.cache, a.table, a.table_stride, a.table_width, a.row_offsets, a.n_seqs, a.dtype);
  if (st) return st;
  if (a.n_rows < 0 || a.n_rows > (1 << 23)) return ts_fail(TS_ERR_INVALID_ARG, "%s: %d rows outside [0, 2^23]", call, a.n_rows);
  if (!aligned_to(a.starts, 4)) return ts_fail(TS_ERR_INVALID_ARG, "%s: misaligned starts", call);
  if (a.n_rows == 0 || (!a.k_out && !a.v_out)) return TS_OK;
  const int64_t kv_row = (int64_t)p.n_kv_heads * p.head_dim;
  if ((a.k_out && a.k_stride < kv_row) || (a.v_out && a.v_stride < kv_row)) return ts_fail(TS_ERR_INVALID_ARG, "%s: a row stride is below its row", call);
  const int esz = ops_esz(a.dtype);
  if (!aligned_to(a.k_out, esz) || !aligned_to(a.v_out, esz)) return ts_fail(TS_ERR_INVALID_ARG, "%s: rows are not aligned to their type", call);
  int dev;
  if ((st = ops_device(call, {p.k, p.v, a.cache.k_scales, a.cache.v_scales, a.table, a.starts, a.row_offsets, a.k_out, a.v_out}, stream, &dev))) return st;
  DeviceGuard on(dev);
  ReadArgs g{};
  g.a = a;
  g.window = window_of(a.n_rows, a.n_seqs);
  const dim3 grid((a.n_rows + g.window - 1) / g.window, (2 * p.n_kv_heads + RA_HEADS - 1) / RA_HEADS);
  if (a.dtype == TS_DTYPE_BF16) launch_read<bf16_t>(g, grid, (hipStream_t)stream);
  else launch_read<float>(g, grid, (hipStream_t)stream);
  TS_HIP(hipGetLastError());
  return TS_OK;
}
