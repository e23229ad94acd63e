// 4-bit microscaled values: quantisation, the values back, weights laid out for the product, and the product.
//
// A block of 32 values has a scale 2^e, e = floor(log2 max|x|) - 2, so that the largest lies in [4, 8) of the 4-bit
// grid 0, 1/2, 1, 3/2, 2, 3, 4, 6.  e is read off the exponent field of the largest magnitude; dividing by a power of
// two is exact, so the rounding of v_cvt_scalef32_pk_fp4_f32 (to nearest, ties to even, saturating) is the only one.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "ts_ops.h"

// ---------------------------------------------------------------------------------
// quantisation: 16 bytes of values a lane, four lanes a block (fp32: eight).  Bound by HBM: it reads the values and writes 17 bytes a block.
// 14336 x 4096 bf16 (117 MB read, 31 MB written, as counted), four matrices in turn: 28.5 us and the values back 28.8, 5.2 TB/s
// both; fp32 46.8 and 52.3 us, 5.7 and 5.1 TB/s; a copy of 1 GiB moves 5.1.  Two pieces a thread, a workgroup's width apart:
// four 31.4 and 29.2 us (65 rows 3.4 and 2.6, with two 2.6 and 2.3), one 30.9 and 33.1.  A wave's loads and stores are whole lines:
// eight fp32 values a lane, stored in two halves, 64.5 us.
// ---------------------------------------------------------------------------------
constexpr int QT = 256, QU = 2;           // threads of a workgroup, pieces per thread
template <typename T> struct MxPiece {     // 16 bytes of values
  static constexpr int V = 16 / sizeof(T), LANES = 32 / V;           // values, pieces of a block
  typedef typename std::conditional<V == 8, uint32_t, uint16_t>::type Codes;
};

template <typename T, int V>
__device__ __forceinline__ void mx_values(const T* p, int n, float (&v)[V]) {
  if (n >= V) {
    const uint4 w = load16(p);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if constexpr (sizeof(T) == 2) v[i] = __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
      else v[i] = __uint_as_float(u[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[i] = 0.f;
      if (i < n) {
        if constexpr (sizeof(T) == 2) v[i] = bf16_to_f32(p[i]);
        else v[i] = p[i];
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(QT) void k_mx_quantize(const T* x, uint32_t rows, uint32_t cols, int64_t stride,
                                                    uint8_t* codes, uint8_t* scales) {
  typedef MxPiece<T> P;
  constexpr int V = P::V, LANES = P::LANES;
  const uint32_t blocks = (cols + 31) / 32, row_pieces = blocks * LANES;
  const uint64_t pieces = (uint64_t)rows * row_pieces;                     // < 2^32, see the launch
  float v[QU][V];
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    const uint64_t at = (uint64_t)blockIdx.x * (QT * QU) + u * QT + threadIdx.x;
    const uint32_t piece = (uint32_t)(at < pieces ? at : 0), r = piece / row_pieces, c = (piece - r * row_pieces) * V;
    mx_values(x + (int64_t)r * stride + c, (int)cols - (int)c, v[u]);
  }
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    const uint64_t at = (uint64_t)blockIdx.x * (QT * QU) + u * QT + threadIdx.x;
    uint32_t top = 0;                                                      // magnitudes order like their bit patterns, NaN last
#pragma unroll
    for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(v[u][i]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < LANES; o *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    const uint32_t ef = top >> 23, s = ef == 255 ? 255 : ef > 2 ? ef - 2 : 0;
    const float inv = __uint_as_float((254 - min(s, 253u)) << 23);         // 2^(127 - s)
    uint32_t w = 0;
    if (s != 255) {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][0] * inv, v[u][1] * inv, 1.f, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][2] * inv, v[u][3] * inv, 1.f, 1);
      if constexpr (V == 8) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][4] * inv, v[u][5] * inv, 1.f, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][6] * inv, v[u][7] * inv, 1.f, 3);
      }
    }
    if (at < pieces) {
      reinterpret_cast<typename P::Codes*>(codes)[at] = (typename P::Codes)w;
      if (at % LANES == 0) scales[at / LANES] = (uint8_t)s;
    }
  }
}

// scale byte -> 2^(s - 127); 255 -> NaN
__device__ __forceinline__ float mx_scale(uint32_t s) {
  return __uint_as_float(s == 255 ? 0x7fc00000u : s == 0 ? 0x00400000u : s << 23);
}

template <typename T>
__global__ __launch_bounds__(QT) void k_mx_dequantize(const uint8_t* codes, const uint8_t* scales, uint32_t rows, uint32_t cols,
                                                      T* x, int64_t stride) {
  typedef MxPiece<T> P;
  constexpr int V = P::V, LANES = P::LANES;
  const uint32_t blocks = (cols + 31) / 32, row_pieces = blocks * LANES;
  const uint64_t pieces = (uint64_t)rows * row_pieces;
  uint32_t w[QU], s[QU];
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    const uint64_t at = (uint64_t)blockIdx.x * (QT * QU) + u * QT + threadIdx.x, a = at < pieces ? at : 0;
    w[u] = reinterpret_cast<const typename P::Codes*>(codes)[a];
    s[u] = scales[a / LANES];
  }
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    const uint64_t at = (uint64_t)blockIdx.x * (QT * QU) + u * QT + threadIdx.x;
    if (at >= pieces) continue;
    const uint32_t r = (uint32_t)at / row_pieces, c = ((uint32_t)at - r * row_pieces) * V;
    const float f = mx_scale(s[u]);
    float v[V];
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.f, 1);
    v[0] = a[0] * f; v[1] = a[1] * f; v[2] = b[0] * f; v[3] = b[1] * f;
    if constexpr (V == 8) {
      const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.f, 3);
      v[4] = d[0] * f; v[5] = d[1] * f; v[6] = e[0] * f; v[7] = e[1] * f;
    }
    T* p = x + (int64_t)r * stride + c;
    const int n = (int)cols - (int)c;
    if (n >= V) {
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (V == 8) o[i] = __float_as_uint(v[2 * i]) >> 16 | (__float_as_uint(v[2 * i + 1]) & 0xffff0000u);     // two significant bits: cutting is exact
        else o[i] = __float_as_uint(v[i]);
      }
      store16(p, make_uint4(o[0], o[1], o[2], o[3]));
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < n) {
          if constexpr (sizeof(T) == 2) p[i] = (bf16_t)(__float_as_uint(v[i]) >> 16);
          else p[i] = v[i];
        }
    }
  }
}

// rows of one launch: pieces within 32 bits
static int64_t mx_slab(int64_t cols) { return ((int64_t)1 << 31) / ((cols + 31) / 32 * 8); }
template <typename T> static uint32_t mx_pieces_groups(int64_t rows, int64_t cols) {
  constexpr int N = QT * QU;
  return (uint32_t)((rows * ((cols + 31) / 32 * MxPiece<T>::LANES) + N - 1) / N);
}

void launch_mx_quantize(hipStream_t s, const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t stride, uint8_t* codes, uint8_t* scales) {
  const int64_t blocks = (cols + 31) / 32, slab = mx_slab(cols);
  const int esz = ops_esz(dtype);
  for (int64_t r = 0; r < rows; r += slab) {
    const int64_t n = std::min(slab, rows - r);
    const void* xs = (const char*)x + r * stride * esz;
    uint8_t *cs = codes + r * blocks * 16, *ss = scales + r * blocks;
    if (dtype == TS_DTYPE_BF16) k_mx_quantize<bf16_t><<<mx_pieces_groups<bf16_t>(n, cols), QT, 0, s>>>((const bf16_t*)xs, (uint32_t)n, (uint32_t)cols, stride, cs, ss);
    else k_mx_quantize<float><<<mx_pieces_groups<float>(n, cols), QT, 0, s>>>((const float*)xs, (uint32_t)n, (uint32_t)cols, stride, cs, ss);
  }
}

static void launch_mx_dequantize(hipStream_t s, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* x, int32_t dtype, int64_t stride) {
  const int64_t blocks = (cols + 31) / 32, slab = mx_slab(cols);
  const int esz = ops_esz(dtype);
  for (int64_t r = 0; r < rows; r += slab) {
    const int64_t n = std::min(slab, rows - r);
    void* xs = (char*)x + r * stride * esz;
    const uint8_t *cs = codes + r * blocks * 16, *ss = scales + r * blocks;
    if (dtype == TS_DTYPE_BF16) k_mx_dequantize<bf16_t><<<mx_pieces_groups<bf16_t>(n, cols), QT, 0, s>>>(cs, ss, (uint32_t)n, (uint32_t)cols, (bf16_t*)xs, stride);
    else k_mx_dequantize<float><<<mx_pieces_groups<float>(n, cols), QT, 0, s>>>(cs, ss, (uint32_t)n, (uint32_t)cols, (float*)xs, stride);
  }
}

// ---------------------------------------------------------------------------------
// weights laid out for the product: records of (16 rows, 128 columns), chunk after chunk of a row tile.  A record is
// what one wave loads for one chunk, contiguous: 16 bytes of codes per lane - lane l = 16 g + n: of row n, codes
// 8 g .. + 7 of each of the chunk's four blocks, the operand of four matrix instructions - then the four scales of each
// row.  Rows and blocks beyond the matrix hold zeros.  Done once, when a matrix is loaded: 14336 x 4096 28 us, 2.2 TB/s read and
// written (codes are gathered in 4-byte pieces).
// ---------------------------------------------------------------------------------
constexpr int MX_REC = 1024 + 64;
static int64_t mx_chunks(int64_t n_in) { return (n_in + 127) / 128; }
size_t mx_packed_bytes(int64_t n_out, int64_t n_in) { return (size_t)((n_out + 15) / 16) * mx_chunks(n_in) * MX_REC; }

__global__ __launch_bounds__(256) void k_mx_pack(const uint8_t* codes, const uint8_t* scales, int n_out, int n_in, uint8_t* packed,
                                                 int n_tile0, int n_tile_stride, int chunks, int64_t records, int* range_flag) {
  const int64_t rec = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (rec >= records) return;
  const int lane = threadIdx.x % 64, tile = (int)(rec / chunks), c = (int)(rec % chunks);
  const int n = tile * 16 + lane % 16, lg = lane / 16, blocks = (n_in + 31) / 32;
  const int64_t row = (int64_t)min(n, n_out - 1) * blocks;
  uint32_t w[4], s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = c * 4 + i;
    const bool in = n < n_out && b < blocks;
    w[i] = in ? reinterpret_cast<const uint32_t*>(codes)[(row + b) * 4 + lg] : 0;
    s[i] = in ? scales[row + b] : 127;
  }
  uint8_t* p = packed + ((int64_t)(n_tile0 + tile * n_tile_stride) * chunks + c) * MX_REC;
  reinterpret_cast<uint4*>(p)[lane] = make_uint4(w[0], w[1], w[2], w[3]);
  // a block's largest value is at least 4 times its scale (a code below that would not be of this scale): 4 * 2^14 is
  // beyond half's largest number, 6 * 2^13 is not
  if (range_flag && lg == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) if (s[i] > 127 + 13 && s[i] != 255) *range_flag = 1;
  }
  if (lg == 0) reinterpret_cast<uint32_t*>(p + 1024)[lane] = s[0] | s[1] << 8 | s[2] << 16 | s[3] << 24;
}

void launch_mx_pack(hipStream_t s, const uint8_t* codes, const uint8_t* scales, int n_out, int n_in, void* packed, int n_tile0, int n_tile_stride,
                    int* range_flag) {
  const int64_t chunks = mx_chunks(n_in), blocks = (n_in + 31) / 32, slab = ((int64_t)1 << 25) / chunks * 16;     // rows: threads within 32 bits
  for (int64_t r = 0; r < n_out; r += slab) {
    const int n = (int)std::min(slab, n_out - r);
    const int64_t records = (n + 15) / 16 * chunks;
    k_mx_pack<<<(uint32_t)((records + 3) / 4), 256, 0, s>>>(codes + r * blocks * 16, scales + r * blocks, n, n_in, (uint8_t*)packed, n_tile0 + (int)(r / 16) * n_tile_stride,
                                                            n_tile_stride, (int)chunks, records, range_flag);
  }
}

// ---------------------------------------------------------------------------------
// the product
//
// The weights go from memory straight into the registers of the matrix instructions; a pair of codes is widened with its
// scale by one conversion instruction.  Two significant bits and eight of exponent fit bf16, so nothing is rounded.
// (Models' rows are halves: see the range of the scales at their loading.)
// ---------------------------------------------------------------------------------
template <int IN> struct MxIn { static constexpr int planes = IN == MX_IN_BF16 ? 1 : IN == MX_IN_F32 ? 3 : 2; };

template <int IN>
__device__ __forceinline__ ts_f32x4 mx_mfma(uint4 w, uint4 x, ts_f32x4 acc) {
  if constexpr (IN == MX_IN_PLANES) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(ts_f16x8, w), __builtin_bit_cast(ts_f16x8, x), acc, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(ts_bf16x8, w), __builtin_bit_cast(ts_bf16x8, x), acc, 0, 0, 0);
}

// eight 4-bit codes of block i of a chunk -> eight halves or bf16 values times its scale, of which the instruction reads the exponent
template <int IN>
__device__ __forceinline__ uint4 mx_widen(uint32_t w, uint32_t scales, int i) {
  const float s = __uint_as_float((scales >> 8 * i & 255) << 23);
  uint4 o;
  if constexpr (IN == MX_IN_PLANES) {
    o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0));
    o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1));
    o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2));
    o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3));
  } else {
    o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
    o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
    o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
    o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
  }
  return o;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// eight inputs of a row as they come from memory
template <int IN> struct MxRaw { uint4 a[IN == MX_IN_BF16 ? 1 : 2]; };

template <int IN> struct MxElem { typedef bf16_t T; };
template <> struct MxElem<MX_IN_F32> { typedef float T; };
// Byte offset of element k of row r from row `row0`, within 32 bits (see the limit of the stride): added to a uniform
// base by the load itself.  Rows past the last: the last again, never stored.  The empty asm keeps the compiler from
// forming 64-bit lane addresses ahead of the loop, two registers and two additions a load.
template <int IN>
__device__ __forceinline__ uint32_t mx_x_offset(const MxArgs& g, int row0, int r, int k) {
  return ((uint32_t)(min(row0 + r, g.rows - 1) - row0) * (uint32_t)g.x_stride + k) * (uint32_t)sizeof(typename MxElem<IN>::T);
}
template <int IN>
__device__ __forceinline__ MxRaw<IN> mx_fetch(const MxArgs& g, const char* base, uint32_t off) {
  MxRaw<IN> o;
  asm("" : "+v"(off));
  o.a[0] = load16(base + off);
  if constexpr (IN == MX_IN_F32) o.a[1] = load16(base + off + 16);
  if constexpr (IN == MX_IN_PLANES) o.a[1] = load16(base + g.x_plane * 2 + off);
  return o;
}
__device__ __forceinline__ uint4 mx_fetch_w(const uint8_t* base, uint32_t off) {
  asm("" : "+v"(off));
  return *reinterpret_cast<const uint4*>(base + off);
}
__device__ __forceinline__ uint32_t mx_fetch_s(const uint8_t* base, uint32_t off) {
  asm("" : "+v"(off));
  return *reinterpret_cast<const uint32_t*>(base + 1024 + off);
}
// the first n of them, zeros behind (models' rows are whole chunks)
template <int IN>
__device__ __forceinline__ MxRaw<IN> mx_fetch_some(const char* base, uint32_t off, int n) {
  const typename MxElem<IN>::T* p = (const typename MxElem<IN>::T*)(base + off);
  MxRaw<IN> o;
  if constexpr (IN != MX_IN_PLANES) {
    constexpr int W = IN == MX_IN_BF16 ? 4 : 8;
    uint32_t u[W];
#pragma unroll
    for (int i = 0; i < W; ++i) u[i] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) {
        if constexpr (IN == MX_IN_BF16) u[i / 2] |= (uint32_t)p[i] << 16 * (i & 1);
        else u[i] = __float_as_uint(p[i]);
      }
#pragma unroll
    for (int i = 0; i < W / 4; ++i) o.a[i] = make_uint4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]);
  }
  return o;
}

// the planes that enter the matrix instructions
template <int IN>
__device__ __forceinline__ void mx_planes(const MxRaw<IN>& v, uint4 (&o)[MxIn<IN>::planes]) {
  if constexpr (IN == MX_IN_F32) {
    const uint32_t u[8] = {v.a[0].x, v.a[0].y, v.a[0].z, v.a[0].w, v.a[1].x, v.a[1].y, v.a[1].z, v.a[1].w};
    uint32_t t3[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ts_bf16x2 t[3];
      split_bf16x2<3>(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]), t);
#pragma unroll
      for (int p = 0; p < 3; ++p) t3[p][i] = __builtin_bit_cast(uint32_t, t[p]);
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) o[p] = make_uint4(t3[p][0], t3[p][1], t3[p][2], t3[p][3]);
  } else {
#pragma unroll
    for (int p = 0; p < MxIn<IN>::planes; ++p) o[p] = v.a[p];
  }
}

// four neighbouring columns of one row
__device__ __forceinline__ void mx_emit(const MxArgs& g, int row, int n, const ts_f32x4& v) {
  if (row >= g.rows || n >= g.n_out) return;
  if (g.y_f32) {
    float* p = (float*)g.y + blockIdx.z * g.y_part + (int64_t)row * g.y_stride + n;
    if (n + 4 <= g.n_out) store16(p, __builtin_bit_cast(uint4, v));
    else
#pragma unroll
      for (int j = 0; j < 4; ++j) if (n + j < g.n_out) p[j] = v[j];
  } else {
    bf16_t* p = (bf16_t*)g.y + (int64_t)row * g.y_stride + n;
    const uint32_t a = __builtin_bit_cast(uint32_t, to_bf16x2(v[0], v[1])), b = __builtin_bit_cast(uint32_t, to_bf16x2(v[2], v[3]));
    if (n + 4 <= g.n_out) store8(p, make_uint2(a, b));
    else
#pragma unroll
      for (int j = 0; j < 4; ++j) if (n + j < g.n_out) p[j] = (bf16_t)((j < 2 ? a : b) >> 16 * (j & 1));
  }
}
// SwiGLU of four neighbouring features
__device__ __forceinline__ void mx_emit_swiglu(const MxArgs& g, int row, int f, const ts_f32x4& gate, const ts_f32x4& up) {
  if (row >= g.rows || 2 * f >= g.n_out) return;
  float p[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) p[j] = gate[j] / (1.f + __expf(-gate[j])) * up[j];
  st_act_planes4((f16_t*)g.y + (int64_t)row * g.y_stride + f, g.y_plane, p[0], p[1], p[2], p[3], g.sat);
}

// Few rows or few columns: KW waves share 16 rows by CT column tiles (of 16), wave w takes chunks w, w + KW, ..., one in use
// and one on its way.  An input is used by one wave only, so a lane reads its pieces of its row itself: for
// instruction i of a chunk, 64 neighbouring bytes of each of 16 rows.  The waves' sums meet in the LDS, added in their
// order.  Bound by the start of the launch and one trip to memory: one bf16 row, 4096 x 4096 (9 MB): 3.7 us, of which 1.8 at
// a copy's rate; 37 fp32 rows, 1001 x 1031: 4.9 us.
template <int IN, int OUT, int CT, int KW>
__global__ __launch_bounds__(KW * 64) void k_mx_few(MxArgs g) {
  typedef typename MxElem<IN>::T E;
  constexpr int NP = MxIn<IN>::planes;
  __shared__ __align__(16) ts_f32x4 red[KW][CT][64];
  const int kw = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, lm = lane % 16, lg = lane / 16;
  const int row0 = blockIdx.y * 16, tile0 = blockIdx.x * CT, n_tiles = (g.n_out + 15) / 16;
  const uint8_t* wp[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) wp[c] = g.w + (int64_t)min(tile0 + c, n_tiles - 1) * g.chunks * MX_REC;
  const char* xp = (const char*)((const E*)g.x + (int64_t)row0 * g.x_stride);
  const uint32_t xo = mx_x_offset<IN>(g, row0, lm, lg * 8);
  ts_f32x4 acc[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) acc[c] = ts_f32x4{0.f, 0.f, 0.f, 0.f};

  struct Chunk { uint4 w[CT]; uint32_t s[CT]; MxRaw<IN> x[4]; };
  auto fetch_w = [&](Chunk& q, int64_t cc) {
#pragma unroll
    for (int c = 0; c < CT; ++c) { q.w[c] = mx_fetch_w(wp[c] + cc * MX_REC, lane * 16); q.s[c] = mx_fetch_s(wp[c] + cc * MX_REC, lm * 4); }
  };
  const int full = g.n_in / 128;                             // chunks without an end in them
  auto fetch = [&](Chunk& q, int chunk) {
    const int64_t cc = min(chunk, full - 1);                 // past the end: requested, not used
    fetch_w(q, cc);
#pragma unroll
    for (int i = 0; i < 4; ++i) q.x[i] = mx_fetch<IN>(g, xp + (cc * 128 + i * 32) * (int)sizeof(E), xo);
  };
  auto multiply = [&](const Chunk& q) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint4 xf[NP];
      mx_planes<IN>(q.x[i], xf);
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const uint4 wf = mx_widen<IN>(word(q.w[c], i), q.s[c], i);
#pragma unroll
        for (int p = NP - 1; p >= 0; --p) acc[c] = mx_mfma<IN>(wf, xf[p], acc[c]);      // the smaller terms first
      }
    }
  };
  if (kw < full) {
    Chunk a, b;
    fetch(a, kw);
    for (int c = kw; c < full; c += 2 * KW) {
      fetch(b, c + KW);
      multiply(a);
      if (c + KW >= full) break;
      fetch(a, c + 2 * KW);
      multiply(b);
    }
  }
  if (IN != MX_IN_PLANES && full < g.chunks && kw == full % KW) {         // the last chunk ends early
    Chunk q;
    fetch_w(q, full);
#pragma unroll
    for (int i = 0; i < 4; ++i) q.x[i] = mx_fetch_some<IN>(xp + ((int64_t)full * 128 + i * 32) * (int)sizeof(E), xo, g.n_in - (full * 128 + i * 32 + lg * 8));
    multiply(q);
  }
#pragma unroll
  for (int c = 0; c < CT; ++c) red[kw][c][lane] = acc[c];
  __syncthreads();
  auto sum = [&](int t) {
    ts_f32x4 v = red[0][t][lane];
#pragma unroll
    for (int o = 1; o < KW; ++o) v += red[o][t][lane];
    return v;
  };
  if constexpr (OUT == MX_OUT_SWIGLU) {                      // tiles alternate: gate and up of the same 16 features
    if (kw < CT / 2) mx_emit_swiglu(g, row0 + lm, (tile0 / 2 + kw) * 16 + 4 * lg, sum(2 * kw), sum(2 * kw + 1));
  } else {
    if (kw < CT) mx_emit(g, row0 + lm, (tile0 + kw) * 16 + 4 * lg, sum(kw));
  }
}

// More rows.  A workgroup computes RT row tiles by WC x CT column tiles (of T x T, T = 16 or 32) over all of K; KW
// groups of its waves take every KW-th chunk and are added up in the LDS at the end, in the order of the groups.  The
// rows go through the LDS (16-byte pieces, their place in a row of 256 bytes exclusive-or'ed with the row number: the
// rows that a read of 16 lanes covers lie in different banks: no conflicts counted), in two buffers, one barrier a step; rows
// and weights are requested a step ahead.
// bf16 rows, 4096 inputs: 2048 rows x 14336 columns 200 us, 1.2 PFLOP/s, what the library's product of bf16 matrices of these
// sizes takes (199); the matrix pipes are busy 65 % of the time, the rest is issuing the widening of the codes, the
// reads of the LDS and the barrier.  65 rows x 28672 columns 22 - 25 us: its 67 MB need 13 at a copy's rate, its
// 65 rows 13 at the library's rate, the 80 it multiplies 16, and 224 workgroups leave an eighth of the CUs without work.  Rows or weights requested two or three steps ahead are no
// faster (25 - 26 us), nor are waves of 64 columns, which read half as much from the LDS (28 us with KW 2, 36 with 4).
template <int T> struct MxTile;
template <> struct MxTile<16> { typedef ts_f32x4 Acc; };
template <> struct MxTile<32> { typedef float Acc __attribute__((ext_vector_type(16))); };
template <int IN, int T>
__device__ __forceinline__ typename MxTile<T>::Acc mx_mfma_t(uint4 w, uint4 x, typename MxTile<T>::Acc acc) {
  if constexpr (T == 16) return mx_mfma<IN>(w, x, acc);
  else if constexpr (IN == MX_IN_PLANES) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(ts_f16x8, w), __builtin_bit_cast(ts_f16x8, x), acc, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(ts_bf16x8, w), __builtin_bit_cast(ts_bf16x8, x), acc, 0, 0, 0);
}

constexpr int MX_AHEAD = 4;
template <int IN, int OUT, int T, int RT, int CT, int WC, int KW>
__global__ __launch_bounds__(WC * KW * 64) void k_mx_rows(MxArgs g) {
  typedef typename MxTile<T>::Acc Acc;
  typedef typename MxElem<IN>::T E;
  constexpr int NP = MxIn<IN>::planes, MT = RT * T, GT = WC * 64, XU = MT * 16 / GT, AQ = T * T / 256;
  constexpr int BL = T / 16, KS = 4 * BL;                    // 16-byte pieces of a record per lane, instructions of a chunk
  static_assert(XU * GT == MT * 16, "pieces of a chunk divide among the threads of a group");
  constexpr int PLANE = MT * 256, BUF = NP * KW * PLANE, RED = (KW - 1) * WC * CT * RT * AQ * 1024;
  static_assert(2 * BUF <= 160 * 1024 && RED <= 160 * 1024, "LDS of a CU");
  __shared__ __align__(16) char smem[2 * BUF > RED ? 2 * BUF : RED];
  const int tid = threadIdx.x, kw = __builtin_amdgcn_readfirstlane(tid / GT), gt = tid % GT, lane = tid % 64;
  const int wc = __builtin_amdgcn_readfirstlane(gt / 64), lm = lane % T, lg = lane / T;
  const int row0 = blockIdx.y * MT, tile0 = (blockIdx.x * WC + wc) * CT, n_tiles = (g.n_out + 15) / 16;
  char* xs = smem + kw * (NP * PLANE);
  const int chunk0 = blockIdx.z * g.per;

  // Weights: instruction i of a chunk takes inputs (64 / T) 8 i + 8 lg .. + 7.  With T = 32 a lane's row lies in one of
  // two records, and its inputs are those of lane groups lg and lg + 2 of the record.
  const uint8_t* wp[CT];
  uint32_t wo[CT], so[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int first = min((tile0 + c) * BL, n_tiles - 1);
    const uint32_t second = lm >= 16 && first + 1 < n_tiles ? (uint32_t)g.chunks * MX_REC : 0;
    wp[c] = g.w + ((int64_t)first * g.chunks + chunk0) * MX_REC;
    wo[c] = second + (lg * 16 + lm % 16) * 16;
    so[c] = second + lm % 16 * 4;
  }

  Acc acc[RT][CT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int q = 0; q < 4 * AQ; ++q) acc[r][c][q] = 0.f;

  const char* xp = (const char*)((const E*)g.x + (int64_t)row0 * g.x_stride + (int64_t)chunk0 * 128);
  uint32_t xo[XU], xl[XU];
#pragma unroll
  for (int u = 0; u < XU; ++u) {
    const int r = (gt + u * GT) / 16;
    xo[u] = mx_x_offset<IN>(g, row0, r, gt % 16 * 8);
    xl[u] = r * 256 + ((gt % 16) ^ (r & 15)) * 16;
  }
  auto put = [&](char* buf, const MxRaw<IN> (&x)[XU]) {
#pragma unroll
    for (int u = 0; u < XU; ++u) {
      uint4 o[NP];
      mx_planes<IN>(x[u], o);
#pragma unroll
      for (int p = 0; p < NP; ++p) *reinterpret_cast<uint4*>(buf + p * PLANE + xl[u]) = o[p];
    }
  };
  struct Weights { uint4 w[CT][BL]; uint32_t s[CT]; };
  auto fetch_w = [&](Weights& q, int64_t cc) {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
#pragma unroll
      for (int b = 0; b < BL; ++b) q.w[c][b] = mx_fetch_w(wp[c] + cc * MX_REC + b * 512, wo[c]);
      q.s[c] = mx_fetch_s(wp[c] + cc * MX_REC, so[c]);
    }
  };
  // Fragments of the rows are read MX_AHEAD before their products and the next step's weights are widened among them:
  // left to itself the compiler reads each into the same registers right before its use and waits for the LDS every time.
  auto multiply = [&](const char* buf, const Weights& q) {
    constexpr int NF = KS * RT * NP, FD = MX_AHEAD;
    auto frag = [&](int f) {                                 // instruction, row tile, term: the smaller terms first
      const int i = f / (RT * NP), r = f / NP % RT, p = NP - 1 - f % NP;
      return *reinterpret_cast<const uint4*>(buf + p * PLANE + (r * T + lm) * 256 + (((64 / T * i + lg) ^ (lm & 15)) * 16));
    };
    auto widen = [&](int c, int i) { return mx_widen<IN>(word(q.w[c][i % BL], i / BL), q.s[c], i / BL); };
    uint4 xa[FD + 1], wf[2][CT];
#pragma unroll
    for (int f = 0; f < FD; ++f) xa[f] = frag(f);
#pragma unroll
    for (int c = 0; c < CT; ++c) wf[0][c] = widen(c, 0);
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      const int i = f / (RT * NP), r = f / NP % RT, at = f % (RT * NP);
      if (f + FD < NF) xa[(f + FD) % (FD + 1)] = frag(f + FD);
      if (i + 1 < KS) {
#pragma unroll
        for (int c = 0; c < CT; ++c)
          if (c * (RT * NP) / CT == at) wf[(i + 1) & 1][c] = widen(c, i + 1);
      }
#pragma unroll
      for (int c = 0; c < CT; ++c) acc[r][c] = mx_mfma_t<IN, T>(wf[i & 1][c], xa[f % (FD + 1)], acc[r][c]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  MxRaw<IN> xn[XU];
  const int full = min(g.n_in / 128 - chunk0, g.per), trips = (full + KW - 1) / KW;     // chunks without an end in them
  auto fetch = [&](Weights& q, int chunk) {
    const int64_t cc = min(chunk, full - 1);                              // past the end: requested, not used
#pragma unroll
    for (int u = 0; u < XU; ++u) xn[u] = mx_fetch<IN>(g, xp + cc * (128 * (int)sizeof(E)), xo[u]);
    fetch_w(q, cc);
  };
  auto step = [&](char* buf, const Weights& now, Weights& next, int t) {
    put(buf, xn);
    fetch(next, (t + 1) * KW + kw);
    wait_lds();
    if (KW == 1 || t * KW + kw < full) multiply(buf, now);
  };
  int t = 0;
  if (full > 0) {
    Weights a, b;
    fetch(a, kw);
    for (; t + 2 <= trips; t += 2) {
      step(xs, a, b, t);
      step(xs + BUF, b, a, t + 1);
    }
    if (t < trips) { step(xs, a, b, t); ++t; }
  }
  if (IN != MX_IN_PLANES && full < g.chunks) {               // the last chunk ends early (K is not split then)
    char* buf = xs + (t & 1) * BUF;
    Weights q;
    if (kw == 0) {
#pragma unroll
      for (int u = 0; u < XU; ++u) xn[u] = mx_fetch_some<IN>(xp + (int64_t)full * (128 * (int)sizeof(E)), xo[u], g.n_in - full * 128 - gt % 16 * 8);
      put(buf, xn);
      fetch_w(q, full);
    }
    wait_lds();
    if (kw == 0) multiply(buf, q);
  }

  if constexpr (KW > 1) {                                  // the groups' sums, added in their order
    ts_f32x4* red = reinterpret_cast<ts_f32x4*>(smem);
    constexpr int PER = WC * CT * RT * AQ * 64;
    auto part = [&](int r, int c, int q) { return ((wc * RT + r) * CT + c) * AQ * 64 + q * 64 + lane; };
    __syncthreads();
    if (kw > 0) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int q = 0; q < AQ; ++q) red[(kw - 1) * PER + part(r, c, q)] = ts_f32x4{acc[r][c][4 * q], acc[r][c][4 * q + 1], acc[r][c][4 * q + 2], acc[r][c][4 * q + 3]};
    }
    __syncthreads();
    if (kw > 0) return;
#pragma unroll
    for (int o = 0; o < KW - 1; ++o)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int q = 0; q < AQ; ++q) {
            const ts_f32x4 v = red[o * PER + part(r, c, q)];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[r][c][4 * q + j] += v[j];
          }
  }
  // a lane holds, of row lm of each row tile, columns 8 q + 4 lg .. + 3 of each column tile (T = 16: q = 0, four groups)
  auto four = [](const Acc& a, int q) { return ts_f32x4{a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]}; };
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = row0 + r * T + lm;
    if constexpr (OUT == MX_OUT_SWIGLU) {                    // tiles of 16 alternate: gate and up of the same features
      if constexpr (T == 16) {
#pragma unroll
        for (int c = 0; c < CT; c += 2) mx_emit_swiglu(g, row, (tile0 + c) * 8 + 4 * lg, acc[r][c], acc[r][c + 1]);
      } else {
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int q = 0; q < 2; ++q) mx_emit_swiglu(g, row, (tile0 + c) * 16 + 8 * q + 4 * lg, four(acc[r][c], q), four(acc[r][c], q + 2));
      }
    } else {
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int q = 0; q < AQ; ++q) mx_emit(g, row, (tile0 + c) * T + 8 * q + 4 * lg, four(acc[r][c], q));
    }
  }
}

template <int IN, int OUT, int CT, int KW>
static void mx_launch_few(hipStream_t s, const MxArgs& g) {
  k_mx_few<IN, OUT, CT, KW><<<dim3((g.n_out + 16 * CT - 1) / (16 * CT), (g.rows + 15) / 16), KW * 64, 0, s>>>(g);
}
template <int IN, int OUT, int T, int RT, int CT, int WC, int KW>
static void mx_launch(hipStream_t s, const MxArgs& g) {
  constexpr int MT = RT * T, NT = WC * CT * T;
  k_mx_rows<IN, OUT, T, RT, CT, WC, KW><<<dim3((g.n_out + NT - 1) / NT, (g.rows + MT - 1) / MT, (g.chunks + g.per - 1) / g.per), WC * KW * 64, 0, s>>>(g);
}

// Which shape a call takes: the one whose rounds of workgroups (256 CUs) times the time of a round is least.  The times are
// microseconds of one round at 4096 inputs, measured between events with an eighth of the CUs to all of them at work; what is
// beyond a start of 2.2 (direct) or 2.6 scales with the inputs.  Several blocks of fewer rows are offered as well as one: 64 rows
// x 14336 inputs, 4096 columns: two blocks of 32 rows 17.9 us, one of 64 on half the CUs 30.8; 128 fp32 rows, 6144 columns 36.7, 45.6
// (35.3 since the rows' terms are cut, not rounded; the fp32 times below are those of before).
// For 2, 3, 4, 5 row tiles of 16, columns a workgroup:
//   bf16 rows   32:  6.8   8.7  12.1  13.0     64:  7.9  10.0  12.8  14.7     128: 11.5  14.8  17.3  20.8
//   fp32 rows                                  64: 24.8  35.3  45.8  52       128: 35    47    61.6  73
//   planes                                     64: 12.8  16.9  21.9  26.8     128: 23.1  29.5  37    44.2
// 64 rows x 256 columns, T = 32: 30.5, 84, 52.6.  The shapes without LDS staging, 16 rows x 16 or 32 columns, are bound by
// the rows' way through the caches: a round takes a time for r rows, more rounds one each (direct_us below).  One row of
// 4096 inputs, 4096 columns: 3.8 and 4.3 us (32 columns staged 6.7); 28672 columns: 13.8 and 12.0 us, 128 columns staged 12.5;
// 16 rows: 4096 columns 7.0, 7.3, 6.9 us, 28672 columns 36.3, 22.7, 13.1 us.
// 65 rows x 4096 inputs, 28672 columns: 128 columns wide 22.3 us, 64 wide 29.8, 32 wide 47.4, 256 wide 31.6; 4096
// columns: 32 wide 13.0, 64 wide 14.7, 128 wide 20.9.
static constexpr float mx_round_us[3][3][4] = {{{6.8f, 8.7f, 12.1f, 13.0f}, {7.9f, 10.0f, 12.8f, 14.7f}, {11.5f, 14.8f, 17.3f, 20.8f}},
                                               {{0, 0, 0, 0}, {24.8f, 35.3f, 45.8f, 52.f}, {35.f, 47.f, 61.6f, 73.f}},
                                               {{0, 0, 0, 0}, {12.8f, 16.9f, 21.9f, 26.8f}, {23.1f, 29.5f, 37.f, 44.2f}}};
static constexpr float mx_wide_us[3] = {30.5f, 84.f, 52.6f};
static float mx_groups(int rows, int n_out, int mt, int nt) { return (float)((rows + mt - 1) / mt) * (float)((n_out + nt - 1) / nt); }
static int mx_row_tiles(int rows) { return std::clamp((rows + 15) / 16, 2, 5); }       // at most, of 16
// Several blocks of planes hold their times only in blocks of 64 rows, or up to three smaller ones: 520 rows x 4096 inputs, 4096
// columns in blocks of 48 or 80 53 us, not 48 and 42, 64 rows by 256 columns 43; 132 rows, 28672 columns, two blocks of 80 rows
// 76 us, three of 48 68, of 64 91.
template <int IN> static bool mx_blocks_hold(int rows, int rt) {
  return IN != MX_IN_PLANES || rt == 4 || (rt == 5 ? rows <= 80 : rows <= 48 * rt);
}

template <int IN, int OUT>
static MxPlan mx_plan_of(int rows, int n_out, int chunks) {
  // one round: [0] + [1] r, of several each: [2] + [3] r
  static constexpr float direct_us[3][2][4] = {{{3.6f, 0.22f, 2.4f, 0.21f}, {4.0f, 0.2f, 2.8f, 0.2f}},
                                               {{7.2f, 0.29f, 4.6f, 0.31f}, {7.6f, 0.25f, 5.6f, 0.28f}},
                                               {{4.9f, 0.42f, 2.6f, 0.4f}, {5.0f, 0.42f, 3.7f, 0.42f}}};
  const int rts = mx_row_tiles(rows);
  const float r = (float)std::min(rows, 16);
  auto share = [&](int mt, int nt) { return mx_groups(rows, n_out, mt, nt) / 256.f; };
  auto scaled = [&](float start, float us) { return start + (us - start) * (float)chunks / 32.f; };
  MxPlan best{MX_N256, 0, scaled(2.6f, ceilf(share(64, 256)) * mx_wide_us[IN])};
  auto offer = [&](int shape, int rt, float cost) { if (cost < best.us) best = MxPlan{shape, rt, cost}; };
  for (int w = IN == MX_IN_BF16 ? 0 : 1; w < 3; ++w)
    if (OUT == MX_OUT_ROWS || w == 2)
      for (int rt = rts; rt >= 2; --rt)
        if (mx_blocks_hold<IN>(rows, rt)) offer(MX_N32 + w, rt, scaled(2.6f, ceilf(share(16 * rt, 32 << w)) * mx_round_us[IN][w][rt - 2]));
  for (int w = OUT == MX_OUT_ROWS ? 0 : 1; w < 2; ++w) {
    const float* us = direct_us[IN][w];
    const float rounds = share(16, 16 << w);                 // past two they run into each other
    offer(MX_DIRECT + w, 0, scaled(2.2f, std::max(us[0] + us[1] * r, (rounds > 2.f ? rounds : ceilf(rounds)) * (us[2] + us[3] * r))));
  }
  return best;
}

// Splits of K for a model's projection, whose sums the next kernel adds up: what a shape takes for its share of the
// chunks, 2.5 us for starting and the sums' way to memory and back at 4 TB/s.  (65 rows x 14336 inputs, 4096 columns:
// 128 columns in 1 split 147 us, as chosen here 28.)
static MxPlan mx_plan_splits(int rows, int n_out, int chunks, int most, int* splits) {
  const int rts = mx_row_tiles(rows);
  MxPlan best{MX_N256, 0, 1e30f};
  for (int s = 1; s <= most; ++s) {
    const int per = (chunks + s - 1) / s;
    if ((chunks + per - 1) / per != s) continue;
    for (int w = 1; w <= 3; ++w)
      for (int rt = rts; rt >= (w < 3 ? 2 : rts); --rt) {
        if (w < 3 && !mx_blocks_hold<MX_IN_PLANES>(rows, rt)) continue;
        const float round = w < 3 ? mx_round_us[MX_IN_PLANES][w][rt - 2] : mx_wide_us[MX_IN_PLANES];
        const float rounds = ceilf(mx_groups(rows, n_out, w < 3 ? 16 * rt : 64, 32 << w) * s / 256.f);
        const float us = 2.5f + rounds * (round - 2.5f) * per / 32.f + (s > 1 ? s : 0) * (float)rows * n_out * 8 / 4e6f;
        if (us < best.us) { best = MxPlan{MX_N32 + w, rt, us}; *splits = s; }
      }
  }
  return best;
}

template <int IN, int OUT, int RT>
static void mx_project_tiles(hipStream_t s, const MxArgs& g, int shape) {
  constexpr int K64 = IN == MX_IN_BF16 ? 4 : IN == MX_IN_F32 ? 1 : 2, K128 = IN == MX_IN_BF16 ? 2 : 1;
  if constexpr (OUT == MX_OUT_ROWS && IN == MX_IN_BF16) if (shape == MX_N32) return mx_launch<IN, OUT, 16, RT, 1, 2, 4>(s, g);
  if constexpr (OUT == MX_OUT_ROWS) if (shape == MX_N64) return mx_launch<IN, OUT, 16, RT, 1, 4, K64>(s, g);
  mx_launch<IN, OUT, 16, RT, 2, 4, K128>(s, g);
}

template <int IN, int OUT>
static void mx_project_by(hipStream_t s, const MxArgs& g, const MxPlan& p) {
  if constexpr (OUT == MX_OUT_ROWS) if (p.shape == MX_DIRECT) return mx_launch_few<IN, OUT, 1, 8>(s, g);
  if (p.shape == MX_DIRECT2) return mx_launch_few<IN, OUT, 2, 8>(s, g);
  if (p.shape == MX_N256) return mx_launch<IN, OUT, 32, 2, 2, 4, 1>(s, g);
  if (p.rt == 2) mx_project_tiles<IN, OUT, 2>(s, g, p.shape);
  else if (p.rt == 3) mx_project_tiles<IN, OUT, 3>(s, g, p.shape);
  else if (p.rt == 4) mx_project_tiles<IN, OUT, 4>(s, g, p.shape);
  else mx_project_tiles<IN, OUT, 5>(s, g, p.shape);
}

MxPlan mx_plan(int in, int out, int rows, int n_out, int chunks) {
  if (in == MX_IN_BF16) return mx_plan_of<MX_IN_BF16, MX_OUT_ROWS>(rows, n_out, chunks);
  if (in == MX_IN_F32) return mx_plan_of<MX_IN_F32, MX_OUT_ROWS>(rows, n_out, chunks);
  if (out == MX_OUT_ROWS) return mx_plan_of<MX_IN_PLANES, MX_OUT_ROWS>(rows, n_out, chunks);
  return mx_plan_of<MX_IN_PLANES, MX_OUT_SWIGLU>(rows, n_out, chunks);
}
MxPlan mx_plan_model(int rows, int n_out, int chunks, size_t out_elems, int* splits) {
  const int most = (int)std::min<size_t>(16, out_elems / ((size_t)rows * n_out));
  *splits = 1;
  MxPlan p = mx_plan_splits(rows, n_out, chunks, std::max(most, 1), splits);
  if (const MxPlan one = mx_plan(MX_IN_PLANES, MX_OUT_ROWS, rows, n_out, chunks); one.us < p.us) { p = one; *splits = 1; }
  return p;
}
void launch_mx_by(hipStream_t s, int in, int out, const MxArgs& g, const MxPlan& p) {
  if (in == MX_IN_BF16) mx_project_by<MX_IN_BF16, MX_OUT_ROWS>(s, g, p);
  else if (in == MX_IN_F32) mx_project_by<MX_IN_F32, MX_OUT_ROWS>(s, g, p);
  else if (out == MX_OUT_ROWS) mx_project_by<MX_IN_PLANES, MX_OUT_ROWS>(s, g, p);
  else mx_project_by<MX_IN_PLANES, MX_OUT_SWIGLU>(s, g, p);
}

// ---------------------------------------------------------------------------------
// a model's projections
// ---------------------------------------------------------------------------------
static MxArgs mx_model_args(const ts_model* m, const f16_t* X, const void* W, int R, int N, int K) {
  MxArgs g{};
  g.w = (const uint8_t*)W;
  g.x = X;
  g.x_stride = act_ld(K);
  g.x_plane = (size_t)(m->ws_rows + TS_MROWS_PER_BLOCK) * act_ld(K);
  g.rows = R; g.n_out = N; g.n_in = K; g.chunks = g.per = (int)mx_chunks(K);
  g.sat = m->sat_count;
  return g;
}
int launch_mx_model(ts_model* m, const f16_t* X, const void* W, float* out, size_t out_elems, int R, int N, int K) {
  MxArgs g = mx_model_args(m, X, W, R, N, K);
  g.y = out; g.y_stride = N; g.y_f32 = 1;
  int splits;
  const MxPlan p = mx_plan_model(R, N, g.chunks, out_elems, &splits);
  g.per = (g.chunks + splits - 1) / splits;
  g.y_part = (size_t)R * N;
  launch_mx_by(m->stream, MX_IN_PLANES, MX_OUT_ROWS, g, p);
  return splits;
}
void launch_mx_model_swiglu(ts_model* m, const f16_t* X, const void* W, f16_t* act_out, int R, int F, int K) {
  MxArgs g = mx_model_args(m, X, W, R, 2 * F, K);
  g.y = act_out; g.y_stride = act_ld(F); g.y_plane = (size_t)(m->ws_rows + TS_MROWS_PER_BLOCK) * act_ld(F);
  launch_mx_by(m->stream, MX_IN_PLANES, MX_OUT_SWIGLU, g, mx_plan(MX_IN_PLANES, MX_OUT_SWIGLU, R, 2 * F, g.chunks));
}

// ---------------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------------
static ts_status mx_check(const char* call, const void* codes, const void* scales, const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t stride) {
  if (!ops_dtype_ok(dtype)) return ts_fail(TS_ERR_INVALID_ARG, "%s: dtype must be TS_DTYPE_F32 or TS_DTYPE_BF16", call);
  if (rows < 0 || cols < 0 || rows > ((int64_t)1 << 40) || cols > ((int64_t)1 << 30))
    return ts_fail(TS_ERR_INVALID_ARG, "%s: %lld rows of %lld columns", call, (long long)rows, (long long)cols);
  if (rows == 0 || cols == 0) return TS_OK;
  if (!codes || !scales || !x) return ts_fail(TS_ERR_INVALID_ARG, "%s: null argument", call);
  if (stride < cols) return ts_fail(TS_ERR_INVALID_ARG, "%s: row stride %lld below the %lld columns", call, (long long)stride, (long long)cols);
  if (!aligned_to(codes, 16)) return ts_fail(TS_ERR_INVALID_ARG, "%s: codes must be 16-byte aligned", call);
  if (!aligned_to(x, ops_esz(dtype))) return ts_fail(TS_ERR_INVALID_ARG, "%s: values are not aligned to their type", call);
  return TS_OK;
}

extern "C" ts_status ts_mx_quantize(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t row_stride, uint8_t* codes, uint8_t* scales,
                                    ts_stream stream) {
  ts_status st = mx_check("ts_mx_quantize", codes, scales, x, dtype, rows, cols, row_stride);
  if (st || rows == 0 || cols == 0) return st;
  int dev;
  if ((st = ops_device("ts_mx_quantize", {x, codes, scales}, stream, &dev))) return st;
  DeviceGuard on(dev);
  launch_mx_quantize((hipStream_t)stream, x, dtype, rows, cols, row_stride, codes, scales);
  TS_HIP(hipGetLastError());
  return TS_OK;
}

extern "C" ts_status ts_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* x, int32_t dtype, int64_t row_stride,
                                      ts_stream stream) {
  ts_status st = mx_check("ts_mx_dequantize", codes, scales, x, dtype, rows, cols, row_stride);
  if (st || rows == 0 || cols == 0) return st;
  int dev;
  if ((st = ops_device("ts_mx_dequantize", {x, codes, scales}, stream, &dev))) return st;
  DeviceGuard on(dev);
  launch_mx_dequantize((hipStream_t)stream, codes, scales, rows, cols, x, dtype, row_stride);
  TS_HIP(hipGetLastError());
  return TS_OK;
}

static ts_status mx_check_shape(const char* call, int32_t n_out, int32_t n_in) {
  if (n_out < 1 || n_in < 1 || n_out > (1 << 24) || n_in > (1 << 22))
    return ts_fail(TS_ERR_INVALID_ARG, "%s: a matrix of %d x %d (at least 1 x 1, at most 2^24 x 2^22)", call, n_out, n_in);
  return TS_OK;
}

extern "C" ts_status ts_mx_packed_bytes(int32_t n_out, int32_t n_in, uint64_t* bytes) {
  if (!bytes) return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_packed_bytes: null argument");
  ts_status st = mx_check_shape("ts_mx_packed_bytes", n_out, n_in);
  if (st) return st;
  *bytes = mx_packed_bytes(n_out, n_in);
  return TS_OK;
}

extern "C" ts_status ts_mx_pack(const uint8_t* codes, const uint8_t* scales, int32_t n_out, int32_t n_in, void* packed, ts_stream stream) {
  ts_status st = mx_check_shape("ts_mx_pack", n_out, n_in);
  if (st) return st;
  if (!codes || !scales || !packed) return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_pack: null argument");
  if (!aligned_to(codes, 16) || !aligned_to(packed, 16)) return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_pack: codes and packed must be 16-byte aligned");
  int dev;
  if ((st = ops_device("ts_mx_pack", {codes, scales, packed}, stream, &dev))) return st;
  DeviceGuard on(dev);
  launch_mx_pack((hipStream_t)stream, codes, scales, n_out, n_in, packed, 0, 1, nullptr);
  TS_HIP(hipGetLastError());
  return TS_OK;
}

extern "C" ts_status ts_mx_project(const void* packed, int32_t n_out, int32_t n_in, const void* x, int32_t dtype, int64_t rows, int64_t x_stride, void* y,
                                   int64_t y_stride, ts_stream stream) {
  ts_status st = mx_check_shape("ts_mx_project", n_out, n_in);
  if (st) return st;
  if (!ops_dtype_ok(dtype)) return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_project: dtype must be TS_DTYPE_F32 or TS_DTYPE_BF16");
  if (rows < 0 || rows > (1 << 19)) return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_project: %lld rows outside [0, 2^19]", (long long)rows);
  if (rows == 0) return TS_OK;
  if (!packed || !x || !y) return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_project: null argument");
  if (rows > 1 && x_stride > (1 << 22)) return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_project: rows %lld values apart (at most 2^22)", (long long)x_stride);
  if (x_stride < n_in || y_stride < n_out)
    return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_project: row strides %lld, %lld below the rows of %d, %d", (long long)x_stride, (long long)y_stride, n_in, n_out);
  const int esz = ops_esz(dtype);
  if (!aligned_to(packed, 16) || !aligned_to(x, esz) || !aligned_to(y, esz))
    return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_project: packed must be 16-byte aligned, rows to their type");
  int dev;
  if ((st = ops_device("ts_mx_project", {packed, x, y}, stream, &dev))) return st;
  DeviceGuard on(dev);
  MxArgs g{};
  g.w = (const uint8_t*)packed;
  g.x = x; g.x_stride = x_stride;
  g.y = y; g.y_stride = y_stride; g.y_f32 = dtype == TS_DTYPE_F32;
  g.n_out = n_out; g.n_in = n_in; g.chunks = g.per = (int)mx_chunks(n_in);
  g.rows = (int)rows;
  const int in = dtype == TS_DTYPE_BF16 ? MX_IN_BF16 : MX_IN_F32;
  launch_mx_by((hipStream_t)stream, in, MX_OUT_ROWS, g, mx_plan(in, MX_OUT_ROWS, g.rows, n_out, g.chunks));
  TS_HIP(hipGetLastError());
  return TS_OK;
}
