// 4-bit microscaled values: quantisation, the values back, weights laid out for the product, and the product.
//
// A block of 32 values has a scale 2^e, e = floor(log2 max|x|) - 2, so that the largest lies in [4, 8) of the 4-bit
// grid 0, 1/2, 1, 3/2, 2, 3, 4, 6.  e is read off the exponent field of the largest magnitude; dividing by a power of
// two is exact, so the rounding of v_cvt_scalef32_pk_fp4_f32 (to nearest, ties to even, saturating) is the only one.
#include "ts_ops.h"

// ---------------------------------------------------------------------------------
// quantisation: four lanes a block, eight values a lane.  Bound by HBM: it reads the values and writes 17 bytes a block.
// ---------------------------------------------------------------------------------
constexpr int QT = 256, QU = 4;           // threads of a workgroup, pieces of eight values per thread

template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, bool vec, float (&v)[8]) {
  if (vec && n >= 8) {
    if constexpr (sizeof(T) == 2) {
      const uint4 w = *reinterpret_cast<const uint4*>(p);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
    } else {
      const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = 0.f;
      if (i < n) {
        if constexpr (sizeof(T) == 2) v[i] = bf16_to_f32(p[i]);
        else v[i] = p[i];
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(QT) void k_mx_quantize(const T* x, uint32_t rows, uint32_t cols, int64_t stride, bool vec,
                                                    uint8_t* codes, uint8_t* scales) {
  const uint32_t blocks = (cols + 31) / 32, row_pieces = blocks * 4;
  const uint64_t pieces = (uint64_t)rows * row_pieces;                     // < 2^32, see the launch
  float v[QU][8];
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    const uint64_t at = (uint64_t)blockIdx.x * (QT * QU) + u * QT + threadIdx.x;
    const uint32_t piece = (uint32_t)(at < pieces ? at : 0), r = piece / row_pieces, c = (piece - r * row_pieces) * 8;
    load8(x + (int64_t)r * stride + c, (int)cols - (int)c, vec, v[u]);
  }
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    const uint64_t at = (uint64_t)blockIdx.x * (QT * QU) + u * QT + threadIdx.x;
    uint32_t top = 0;                                                      // magnitudes order like their bit patterns, NaN last
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[u][i]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    const uint32_t ef = top >> 23, s = ef == 255 ? 255 : ef > 2 ? ef - 2 : 0;
    const float inv = __uint_as_float((254 - min(s, 253u)) << 23);         // 2^(127 - s)
    uint32_t w = 0;
    if (s != 255) {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][0] * inv, v[u][1] * inv, 1.f, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][2] * inv, v[u][3] * inv, 1.f, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][4] * inv, v[u][5] * inv, 1.f, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][6] * inv, v[u][7] * inv, 1.f, 3);
    }
    if (at < pieces) {
      reinterpret_cast<uint32_t*>(codes)[at] = w;
      if ((at & 3) == 0) scales[at >> 2] = (uint8_t)s;
    }
  }
}

// scale byte -> 2^(s - 127); 255 -> NaN
__device__ __forceinline__ float mx_scale(uint32_t s) {
  return __uint_as_float(s == 255 ? 0x7fc00000u : s == 0 ? 0x00400000u : s << 23);
}

template <typename T>
__global__ __launch_bounds__(QT) void k_mx_dequantize(const uint8_t* codes, const uint8_t* scales, uint32_t rows, uint32_t cols,
                                                      T* x, int64_t stride, bool vec) {
  const uint32_t blocks = (cols + 31) / 32, row_pieces = blocks * 4;
  const uint64_t pieces = (uint64_t)rows * row_pieces;
  uint32_t w[QU], s[QU];
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    const uint64_t at = (uint64_t)blockIdx.x * (QT * QU) + u * QT + threadIdx.x, a = at < pieces ? at : 0;
    w[u] = reinterpret_cast<const uint32_t*>(codes)[a];
    s[u] = scales[a >> 2];
  }
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    const uint64_t at = (uint64_t)blockIdx.x * (QT * QU) + u * QT + threadIdx.x;
    if (at >= pieces) continue;
    const uint32_t r = (uint32_t)at / row_pieces, c = ((uint32_t)at - r * row_pieces) * 8;
    const float f = mx_scale(s[u]);
    float v[8];
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.f, 1);
    const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.f, 3);
    v[0] = a[0] * f; v[1] = a[1] * f; v[2] = b[0] * f; v[3] = b[1] * f; v[4] = d[0] * f; v[5] = d[1] * f; v[6] = e[0] * f; v[7] = e[1] * f;
    T* p = x + (int64_t)r * stride + c;
    const int n = (int)cols - (int)c;
    if (vec && n >= 8) {
      if constexpr (sizeof(T) == 2) {                                       // two significant bits: cutting is exact
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __float_as_uint(v[2 * i]) >> 16 | (__float_as_uint(v[2 * i + 1]) & 0xffff0000u);
        *reinterpret_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
      } else {
        reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) {
          if constexpr (sizeof(T) == 2) p[i] = (bf16_t)(__float_as_uint(v[i]) >> 16);
          else p[i] = v[i];
        }
    }
  }
}

// rows of one launch: pieces within 32 bits
static int64_t mx_slab(int64_t cols) { return ((int64_t)1 << 31) / ((cols + 31) / 32 * 4); }
static uint32_t mx_groups(int64_t rows, int64_t cols) { return (uint32_t)((rows * ((cols + 31) / 32 * 4) + QT * QU - 1) / (QT * QU)); }

void launch_mx_quantize(hipStream_t s, const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t stride, uint8_t* codes, uint8_t* scales) {
  const int64_t blocks = (cols + 31) / 32, slab = mx_slab(cols);
  const int esz = ops_esz(dtype);
  const bool vec = aligned_to(x, 16) && stride * esz % 16 == 0;
  for (int64_t r = 0; r < rows; r += slab) {
    const int64_t n = std::min(slab, rows - r);
    const void* xs = (const char*)x + r * stride * esz;
    uint8_t *cs = codes + r * blocks * 16, *ss = scales + r * blocks;
    if (dtype == TS_DTYPE_BF16) k_mx_quantize<bf16_t><<<mx_groups(n, cols), QT, 0, s>>>((const bf16_t*)xs, (uint32_t)n, (uint32_t)cols, stride, vec, cs, ss);
    else k_mx_quantize<float><<<mx_groups(n, cols), QT, 0, s>>>((const float*)xs, (uint32_t)n, (uint32_t)cols, stride, vec, cs, ss);
  }
}

static void launch_mx_dequantize(hipStream_t s, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* x, int32_t dtype, int64_t stride) {
  const int64_t blocks = (cols + 31) / 32, slab = mx_slab(cols);
  const int esz = ops_esz(dtype);
  const bool vec = aligned_to(x, 16) && stride * esz % 16 == 0;
  for (int64_t r = 0; r < rows; r += slab) {
    const int64_t n = std::min(slab, rows - r);
    void* xs = (char*)x + r * stride * esz;
    const uint8_t *cs = codes + r * blocks * 16, *ss = scales + r * blocks;
    if (dtype == TS_DTYPE_BF16) k_mx_dequantize<bf16_t><<<mx_groups(n, cols), QT, 0, s>>>(cs, ss, (uint32_t)n, (uint32_t)cols, (bf16_t*)xs, stride, vec);
    else k_mx_dequantize<float><<<mx_groups(n, cols), QT, 0, s>>>(cs, ss, (uint32_t)n, (uint32_t)cols, (float*)xs, stride, vec);
  }
}

// ---------------------------------------------------------------------------------
// weights laid out for the product: records of (16 rows, 128 columns), chunk after chunk of a row tile.  A record is
// what one wave loads for one chunk, contiguous: 16 bytes of codes per lane (lane l: row l % 16, block l / 16 of the
// chunk), then a scale byte per lane.  Rows and blocks beyond the matrix hold zeros.
// ---------------------------------------------------------------------------------
constexpr int MX_REC = 1024 + 64;
static int64_t mx_chunks(int64_t n_in) { return (n_in + 127) / 128; }
size_t mx_packed_bytes(int64_t n_out, int64_t n_in) { return (size_t)((n_out + 15) / 16) * mx_chunks(n_in) * MX_REC; }

__global__ __launch_bounds__(256) void k_mx_pack(const uint8_t* codes, const uint8_t* scales, int n_out, int n_in, uint8_t* packed,
                                                 int n_tile0, int n_tile_stride, int chunks, int64_t records) {
  const int64_t rec = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (rec >= records) return;
  const int lane = threadIdx.x % 64, tile = (int)(rec / chunks), c = (int)(rec % chunks);
  const int n = tile * 16 + lane % 16, b = c * 4 + lane / 16, blocks = (n_in + 31) / 32;
  uint4 w = make_uint4(0, 0, 0, 0);
  uint8_t s = 127;
  if (n < n_out && b < blocks) {
    w = reinterpret_cast<const uint4*>(codes)[(int64_t)n * blocks + b];
    s = scales[(int64_t)n * blocks + b];
  }
  uint8_t* p = packed + ((int64_t)(n_tile0 + tile * n_tile_stride) * chunks + c) * MX_REC;
  reinterpret_cast<uint4*>(p)[lane] = w;
  p[1024 + lane] = s;
}

void launch_mx_pack(hipStream_t s, const uint8_t* codes, const uint8_t* scales, int n_out, int n_in, void* packed, int n_tile0, int n_tile_stride) {
  const int64_t records = (int64_t)((n_out + 15) / 16) * mx_chunks(n_in);
  k_mx_pack<<<(uint32_t)((records + 3) / 4), 256, 0, s>>>(codes, scales, n_out, n_in, (uint8_t*)packed, n_tile0, n_tile_stride, (int)mx_chunks(n_in), records);
}

// ---------------------------------------------------------------------------------
// the product
//
// A workgroup computes WR x RT row tiles by WC x CT column tiles (of 16) over all of K; KW groups of its waves take
// every KW-th chunk of 128 inputs and are added up in the LDS at the end, in the order of the groups.  The weights go
// from memory straight into the registers of the matrix instructions: a lane's 16 bytes are one block of one row, and
// since a sum over k may be taken in any order as long as both operands agree on it, the four instructions of a chunk
// take inputs 32 g + 8 i .. + 7 from lane group g.  The rows go through the LDS (16-byte pieces, their place in a row
// of 256 bytes exclusive-or'ed with the row number: the 16 rows a quarter wave reads lie in different banks).
// ---------------------------------------------------------------------------------
enum { MX_IN_BF16 = 0, MX_IN_F32 = 1, MX_IN_PLANES = 2 };   // rows: bf16; fp32 as three bf16 terms; a model's hi and lo halves
enum { MX_OUT_ROWS = 0, MX_OUT_SWIGLU = 1 };

struct MxArgs {
  const uint8_t* w;
  const void* x; int64_t x_stride; size_t x_plane;        // elements between the hi and the lo plane
  void* y; int64_t y_stride; size_t y_plane; int32_t y_f32;
  unsigned long long* sat;
  int rows, n_out, n_in, chunks;
  int vec_x, vec_y;
};

template <int IN> struct MxIn { static constexpr int planes = IN == MX_IN_BF16 ? 1 : IN == MX_IN_F32 ? 3 : 2; };

template <int IN>
__device__ __forceinline__ ts_f32x4 mx_mfma(uint4 w, uint4 x, ts_f32x4 acc) {
  if constexpr (IN == MX_IN_PLANES) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(ts_f16x8, w), __builtin_bit_cast(ts_f16x8, x), acc, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(ts_bf16x8, w), __builtin_bit_cast(ts_bf16x8, x), acc, 0, 0, 0);
}

// eight 4-bit codes -> eight halves or bf16 values times the scale (both exact: see the callers for the ranges)
template <int IN>
__device__ __forceinline__ uint4 mx_widen(uint32_t w, float s) {
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

// one 16-byte piece (eight inputs) of a row as it comes from memory
template <int IN> struct MxRaw { uint4 a[IN == MX_IN_BF16 ? 1 : 2]; };

template <int IN>
__device__ __forceinline__ MxRaw<IN> mx_fetch(const MxArgs& g, int r, int k) {
  MxRaw<IN> o;
#pragma unroll
  for (uint4& v : o.a) v = make_uint4(0, 0, 0, 0);
  if (r >= g.rows || k >= g.n_in) return o;
  if constexpr (IN == MX_IN_PLANES) {                        // n_in is a multiple of 128, rows are padded
    const f16_t* p = (const f16_t*)g.x + (int64_t)r * g.x_stride + k;
    o.a[0] = *reinterpret_cast<const uint4*>(p);
    o.a[1] = *reinterpret_cast<const uint4*>(p + g.x_plane);
  } else if constexpr (IN == MX_IN_BF16) {
    const bf16_t* p = (const bf16_t*)g.x + (int64_t)r * g.x_stride + k;
    if (g.vec_x && k + 8 <= g.n_in) o.a[0] = *reinterpret_cast<const uint4*>(p);
    else {
      uint32_t u[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i) if (k + i < g.n_in) u[i / 2] |= (uint32_t)p[i] << 16 * (i & 1);
      o.a[0] = make_uint4(u[0], u[1], u[2], u[3]);
    }
  } else {
    const float* p = (const float*)g.x + (int64_t)r * g.x_stride + k;
    if (g.vec_x && k + 8 <= g.n_in) { o.a[0] = reinterpret_cast<const uint4*>(p)[0]; o.a[1] = reinterpret_cast<const uint4*>(p)[1]; }
    else {
      uint32_t u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = k + i < g.n_in ? __float_as_uint(p[i]) : 0;
      o.a[0] = make_uint4(u[0], u[1], u[2], u[3]);
      o.a[1] = make_uint4(u[4], u[5], u[6], u[7]);
    }
  }
  return o;
}

// into the LDS as one piece per plane, `plane` bytes apart
template <int IN>
__device__ __forceinline__ void mx_put(char* at, int plane, const MxRaw<IN>& v) {
  if constexpr (IN == MX_IN_F32) {
    const uint32_t u[8] = {v.a[0].x, v.a[0].y, v.a[0].z, v.a[0].w, v.a[1].x, v.a[1].y, v.a[1].z, v.a[1].w};
    uint32_t o[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ts_bf16x2 t[3];
      split_bf16x2<3>(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]), t);
#pragma unroll
      for (int p = 0; p < 3; ++p) o[p][i] = __builtin_bit_cast(uint32_t, t[p]);
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(at + p * plane) = make_uint4(o[p][0], o[p][1], o[p][2], o[p][3]);
  } else {
#pragma unroll
    for (int p = 0; p < MxIn<IN>::planes; ++p) *reinterpret_cast<uint4*>(at + p * plane) = v.a[p];
  }
}

template <int IN, int OUT, int RT, int CT, int WR, int WC, int KW>
__global__ __launch_bounds__(WR * WC * KW * 64) void k_mx_project(MxArgs g) {
  constexpr int NP = MxIn<IN>::planes, MT = WR * RT * 16, GT = WR * WC * 64, XU = MT * 16 / GT;
  static_assert(XU * GT == MT * 16, "pieces of a chunk divide among the threads of a group");
  constexpr int PLANE = MT * 256, LDS = NP * KW * PLANE, RED = (KW - 1) * WR * WC * CT * RT * 1024;
  static_assert(LDS <= 160 * 1024 && RED <= 160 * 1024, "LDS of a CU");
  __shared__ __align__(16) char smem[LDS > RED ? LDS : RED];
  const int tid = threadIdx.x, kw = tid / GT, gt = tid % GT, lane = tid % 64, wave = gt / 64;
  const int wr = wave / WC, wc = wave % WC, lm = lane % 16, lg = lane / 16;
  const int row0 = blockIdx.y * MT, tile0 = (blockIdx.x * WC + wc) * CT, n_tiles = (g.n_out + 15) / 16;
  char* xs = smem + kw * (NP * PLANE);

  const uint8_t* wp[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) wp[c] = g.w + (int64_t)min(tile0 + c, n_tiles - 1) * g.chunks * MX_REC;

  ts_f32x4 acc[CT][RT];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[c][r] = ts_f32x4{0.f, 0.f, 0.f, 0.f};

  uint4 wn[CT];
  uint32_t sn[CT];
  MxRaw<IN> xn[XU];
  auto fetch = [&](int chunk) {
    const int cc = min(chunk, g.chunks - 1);                              // past the end: loaded, never used
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      wn[c] = *reinterpret_cast<const uint4*>(wp[c] + (int64_t)cc * MX_REC + lane * 16);
      sn[c] = wp[c][(int64_t)cc * MX_REC + 1024 + lane];
    }
#pragma unroll
    for (int u = 0; u < XU; ++u) {
      const int piece = gt + u * GT, r = piece / 16, k = chunk * 128 + (piece % 16) * 8;
      xn[u] = mx_fetch<IN>(g, row0 + r, k);
    }
  };
  fetch(kw);
  const int trips = (g.chunks + KW - 1) / KW;
  for (int t = 0; t < trips; ++t) {
    const int chunk = t * KW + kw;
#pragma unroll
    for (int u = 0; u < XU; ++u) {
      const int piece = gt + u * GT, r = piece / 16, q = piece % 16;
      mx_put<IN>(xs + r * 256 + ((q ^ (r & 15)) * 16), PLANE, xn[u]);
    }
    uint4 w[CT];
    float s[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) { w[c] = wn[c]; s[c] = mx_scale(sn[c]); }
    __syncthreads();
    if (t + 1 < trips) fetch(chunk + KW);
    if (chunk < g.chunks) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint4 wf[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) wf[c] = mx_widen<IN>(i == 0 ? w[c].x : i == 1 ? w[c].y : i == 2 ? w[c].z : w[c].w, s[c]);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const int row = (wr * RT + r) * 16 + lm;
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const uint4 xf = *reinterpret_cast<const uint4*>(xs + p * PLANE + row * 256 + (((4 * lg + i) ^ lm) * 16));
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[c][r] = mx_mfma<IN>(wf[c], xf, acc[c][r]);
          }
        }
      }
    }
    __syncthreads();
  }

  if constexpr (KW > 1) {                                  // the groups' sums, added in their order
    ts_f32x4* red = reinterpret_cast<ts_f32x4*>(smem);
    constexpr int PER = WR * WC * CT * RT * 64;
    if (kw > 0) {
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int r = 0; r < RT; ++r) red[(kw - 1) * PER + ((wave * CT + c) * RT + r) * 64 + lane] = acc[c][r];
    }
    __syncthreads();
    if (kw > 0) return;
    for (int o = 0; o < KW - 1; ++o)
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[c][r] += red[o * PER + ((wave * CT + c) * RT + r) * 64 + lane];
  }

  // a lane holds columns 4 lg .. + 3 of each column tile, of row lm of each row tile
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = row0 + (wr * RT + r) * 16 + lm;
    if (row >= g.rows) continue;
    if constexpr (OUT == MX_OUT_SWIGLU) {
#pragma unroll
      for (int c = 0; c < CT; c += 2) {                    // tiles alternate: gate and up of the same 16 features
        if (tile0 + c >= n_tiles) continue;
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float gate = acc[c][r][j];
          v[j] = gate / (1.f + __expf(-gate)) * acc[c + 1][r][j];
        }
        st_act_planes4((f16_t*)g.y + (int64_t)row * g.y_stride + (tile0 + c) * 8 + 4 * lg, g.y_plane, v[0], v[1], v[2], v[3], g.sat);
      }
    } else {
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const int n = (tile0 + c) * 16 + 4 * lg;
        const ts_f32x4 v = acc[c][r];
        if (n >= g.n_out) continue;
        if (g.y_f32) {
          float* p = (float*)g.y + (int64_t)row * g.y_stride + n;
          if (g.vec_y && n + 4 <= g.n_out) *reinterpret_cast<ts_f32x4*>(p) = v;
          else
#pragma unroll
            for (int j = 0; j < 4; ++j) if (n + j < g.n_out) p[j] = v[j];
        } else {
          bf16_t* p = (bf16_t*)g.y + (int64_t)row * g.y_stride + n;
          const uint32_t a = __builtin_bit_cast(uint32_t, to_bf16x2(v[0], v[1])), b = __builtin_bit_cast(uint32_t, to_bf16x2(v[2], v[3]));
          if (g.vec_y && n + 4 <= g.n_out) *reinterpret_cast<uint2*>(p) = make_uint2(a, b);
          else
#pragma unroll
            for (int j = 0; j < 4; ++j) if (n + j < g.n_out) p[j] = (bf16_t)((j < 2 ? a : b) >> 16 * (j & 1));
        }
      }
    }
  }
}

template <int IN, int OUT, int RT, int CT, int WR, int WC, int KW>
static void mx_launch(hipStream_t s, const MxArgs& g) {
  constexpr int MT = WR * RT * 16, NT = WC * CT * 16;
  k_mx_project<IN, OUT, RT, CT, WR, WC, KW><<<dim3((g.n_out + NT - 1) / NT, (g.rows + MT - 1) / MT), WR * WC * KW * 64, 0, s>>>(g);
}

template <int IN, int OUT>
static void mx_project(hipStream_t s, const MxArgs& g) {
  if (g.rows <= 16) mx_launch<IN, OUT, 1, 2, 1, 1, 4>(s, g);
  else if (g.rows <= 48) mx_launch<IN, OUT, 3, 2, 1, 2, 2>(s, g);
  else if (g.rows <= 80) mx_launch<IN, OUT, 5, 2, 1, 2, 2>(s, g);
  else mx_launch<IN, OUT, 4, 4, 2, 2, 1>(s, g);
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
  if (n_out < 1 || n_in < 1 || n_out > (1 << 24) || n_in > (1 << 24))
    return ts_fail(TS_ERR_INVALID_ARG, "%s: a matrix of %d x %d (both must lie in [1, 2^24])", call, n_out, n_in);
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
  launch_mx_pack((hipStream_t)stream, codes, scales, n_out, n_in, packed, 0, 1);
  TS_HIP(hipGetLastError());
  return TS_OK;
}

extern "C" ts_status ts_mx_project(const void* packed, int32_t n_out, int32_t n_in, const void* x, int32_t dtype, int64_t rows, int64_t x_stride, void* y,
                                   int64_t y_stride, ts_stream stream) {
  ts_status st = mx_check_shape("ts_mx_project", n_out, n_in);
  if (st) return st;
  if (!ops_dtype_ok(dtype)) return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_project: dtype must be TS_DTYPE_F32 or TS_DTYPE_BF16");
  if (rows < 0 || rows > (1 << 22)) return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_project: %lld rows outside [0, 2^22]", (long long)rows);
  if (rows == 0) return TS_OK;
  if (!packed || !x || !y) return ts_fail(TS_ERR_INVALID_ARG, "ts_mx_project: null argument");
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
  g.n_out = n_out; g.n_in = n_in; g.chunks = (int)mx_chunks(n_in);
  g.vec_x = aligned_to(x, 16) && x_stride * esz % 16 == 0;
  g.vec_y = aligned_to(y, 4 * esz) && y_stride % 4 == 0;
  g.rows = (int)rows;
  if (dtype == TS_DTYPE_BF16) mx_project<MX_IN_BF16, MX_OUT_ROWS>((hipStream_t)stream, g);
  else mx_project<MX_IN_F32, MX_OUT_ROWS>((hipStream_t)stream, g);
  TS_HIP(hipGetLastError());
  return TS_OK;
}
