// Shared by the calls over a paged cache: rows and pages in vectors, the sequence of a row, values transposed into pages, and the checks
// that the calls have in common.
#pragma once
#include <math.h>

#include "ts_ops.h"

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

template <typename TI, typename TC, int HD>
__device__ __forceinline__ void append_values(const void* v_rows, int64_t v_stride, void* v_pages, const AppendPage& at) {
  const int tid = threadIdx.x, cnt = at.cnt, slot = at.slot, row = at.row, page = at.page, hkv = at.hkv, turned = at.hq + at.hkv, head0 = at.head0, head1 = at.head1;
  // values: a thread writes the positions of a dimension, of two for rows of bf16.  All rows are requested at once (what
  // lies outside the new ones is the nearest of them, not stored); they go in vectors, cut at the ends.
  constexpr int DV = 4 / sizeof(TI), SV = 16 / sizeof(TC);
  const int val0 = max(head0, turned), end = slot + cnt;
  for (int i = tid; i < (head1 - val0) * HD / DV; i += APPEND_THREADS) {
    const int h = val0 - turned + i * DV / HD, d = i * DV % HD;
    const TI* src = (const TI*)v_rows + (int64_t)row * v_stride + h * HD + d;
    TC* dst = (TC*)v_pages + (((int64_t)page * hkv + h) * HD + d) * 16;
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
      load_n<DV>(src + (int64_t)min(max(p - slot, 0), cnt - 1) * v_stride, w);
#pragma unroll
      for (int e = 0; e < DV; ++e) v[e][p] = w[e];
    }
#pragma unroll
    for (int p0 = 0; p0 < 16; p0 += SV)
#pragma unroll
      for (int e = 0; e < DV; ++e) store_some<SV>(dst + e * 16 + p0, p0, slot, end, &v[e][p0]);
  }
}

// ---- 8-bit pages ------------------------------------------------------------------
struct e4m3_t { uint8_t b; };

// The conversions of gfx950 take a scale as the exponent field of an fp32, its other bits ignored: 2^(field - 127), 255 is NaN; exactly what
// a scale byte says.  scale_at<I>(w): the operand for byte I of w.
template <int I> __device__ __forceinline__ float scale_at(uint32_t w) { return __uint_as_float(I == 3 ? w >> 1 : w << (23 - 8 * I)); }
// four values, the bits of one dword, times the scale
__device__ __forceinline__ void e4m3_to_f32(uint32_t w, float scale, float* v) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
  v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
}
// four values of one dword times four scales, the bytes of another
__device__ __forceinline__ void e4m3_to_f32(uint32_t w, uint32_t scales, float* v) {
  v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale_at<0>(scales), false)[0];
  v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale_at<1>(scales), false)[1];
  v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale_at<2>(scales), true)[0];
  v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale_at<3>(scales), true)[1];
}
// eight values of one scale as bf16, rounded only where bf16 is subnormal
__device__ __forceinline__ ts_u32x4 e4m3_to_bf16(uint32_t a, uint32_t b, float scale) {
  return ts_u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true)),
                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true))};
}
// eight values of one scale each: the bytes of two dwords, their scales those of two others
__device__ __forceinline__ ts_u32x4 e4m3_to_bf16(uint32_t a, uint32_t b, uint32_t s_a, uint32_t s_b) {
  float x[4], y[4];
  e4m3_to_f32(a, s_a, x);
  e4m3_to_f32(b, s_b, y);
  return ts_u32x4{__builtin_bit_cast(uint32_t, to_bf16x2(x[0], x[1])), __builtin_bit_cast(uint32_t, to_bf16x2(x[2], x[3])),
                  __builtin_bit_cast(uint32_t, to_bf16x2(y[0], y[1])), __builtin_bit_cast(uint32_t, to_bf16x2(y[2], y[3]))};
}
__device__ __forceinline__ uint32_t f32_to_e4m3(float a, float b, float c, float d) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
// The scale byte of a row from its largest magnitude's bits (those of infinity and NaN are above all others): magnitude
// m 2^x, 1 <= m < 2, fits 448 = 1.75 * 2^8 with e = x - 8, or one more where m is beyond 1.75.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  return top >= 0x7f800000u ? 255u : (uint32_t)max(0, (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u));
}

// ---- checks that the calls have in common ---------------------------------------------
inline ts_status check_kv_pages(const char* call, const ts_kv_pages& p, const int32_t* table, int64_t table_stride, int32_t table_width, const int32_t* lengths,
                                int32_t n_seqs, int32_t dtype) {
  if (!p.k || !p.v || !table || !lengths) return ts_fail(TS_ERR_INVALID_ARG, "%s: null argument", call);
  if (!ops_dtype_ok(dtype)) return ts_fail(TS_ERR_INVALID_ARG, "%s: dtype must be TS_DTYPE_F32 or TS_DTYPE_BF16", call);
  if (p.n_pages < 1 || p.n_kv_heads < 1 || p.n_kv_heads > 65536) return ts_fail(TS_ERR_INVALID_ARG, "%s: %d pages of %d KV heads", call, p.n_pages, p.n_kv_heads);
  const int hd = p.head_dim;
  if (p.dtype != TS_DTYPE_F32 ? hd != 64 && hd != 128 : hd != 8 && hd != 16 && hd != 32 && hd != 64 && hd != 128)
    return ts_fail(TS_ERR_INVALID_ARG, "%s: head_dim %d (fp32 pages: a power of two in [8,128], others: 64 or 128)", call, hd);
  if (!aligned_to(p.k, 16) || !aligned_to(p.v, 16)) return ts_fail(TS_ERR_INVALID_ARG, "%s: pages must be 16-byte aligned", call);
  if (n_seqs < 1 || n_seqs > (1 << 20)) return ts_fail(TS_ERR_INVALID_ARG, "%s: n_seqs %d outside [1, 2^20]", call, n_seqs);
  if (table_width < 1 || table_stride < table_width) return ts_fail(TS_ERR_INVALID_ARG, "%s: page table of width %d, stride %lld", call, table_width, (long long)table_stride);
  if (!aligned_to(table, 4) || !aligned_to(lengths, 4)) return ts_fail(TS_ERR_INVALID_ARG, "%s: misaligned table or lengths", call);
  return TS_OK;
}
// pages of any type, with the scales that 8-bit ones need and others do not have
inline ts_status check_kv_pages_any(const char* call, const ts_kv_pages_any& c, const int32_t* table, int64_t table_stride, int32_t table_width,
                                    const int32_t* lengths, int32_t n_seqs, int32_t dtype) {
  const bool eight = c.pages.dtype == TS_DTYPE_E4M3;
  if (!eight && !ops_dtype_ok(c.pages.dtype)) return ts_fail(TS_ERR_INVALID_ARG, "%s: dtype of the pages must be TS_DTYPE_F32, TS_DTYPE_BF16 or TS_DTYPE_E4M3", call);
  if (eight ? !c.k_scales || !c.v_scales : c.k_scales || c.v_scales) return ts_fail(TS_ERR_INVALID_ARG, "%s: scales belong to TS_DTYPE_E4M3 pages, and both of them", call);
  if (!aligned_to(c.k_scales, 16) || !aligned_to(c.v_scales, 16)) return ts_fail(TS_ERR_INVALID_ARG, "%s: scales must be 16-byte aligned", call);
  return check_kv_pages(call, c.pages, table, table_stride, table_width, lengths, n_seqs, dtype);
}
