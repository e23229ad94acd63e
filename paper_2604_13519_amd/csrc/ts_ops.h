// Shared by the device-tensor operators (include/toolspec_ops.h): pointer checks, device switching, element types.
#pragma once
#include <initializer_list>

#include "../../include/toolspec_ops.h"
#include "ts_device_utils.h"
#include "ts_internal.h"

typedef __bf16 ts_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 ts_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 ts_f16x8 __attribute__((ext_vector_type(8)));
typedef float ts_f32x4 __attribute__((ext_vector_type(4)));

// Every pointer that is not null has to be memory of one GPU, the stream's: what a kernel would fault on becomes an error here.
// Returns that GPU in *device.
ts_status ops_device(const char* call, std::initializer_list<const void*> pointers, ts_stream stream, int* device);

// Makes `device` current for a launch and gives the caller its own back.
struct DeviceGuard {
  int back;
  explicit DeviceGuard(int device) : back(-1) {
    int now = -1;
    if (hipGetDevice(&now) == hipSuccess && now != device && hipSetDevice(device) == hipSuccess) back = now;
  }
  ~DeviceGuard() { if (back >= 0) (void)hipSetDevice(back); }
};

inline bool ops_dtype_ok(int32_t dtype) { return dtype == TS_DTYPE_F32 || dtype == TS_DTYPE_BF16; }
inline int ops_esz(int32_t dtype) { return dtype == TS_DTYPE_BF16 ? 2 : 4; }
inline bool aligned_to(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// 16, 8 and 4 bytes from or to the place of any element: the vector accesses of gfx950 need no more alignment than that
typedef uint32_t ts_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t ts_u32x2 __attribute__((ext_vector_type(2)));
typedef ts_u32x4 ts_u32x4_any __attribute__((aligned(2)));
typedef ts_u32x2 ts_u32x2_any __attribute__((aligned(2)));
__device__ __forceinline__ uint4 load16(const void* p) { return __builtin_bit_cast(uint4, (ts_u32x4)*reinterpret_cast<const ts_u32x4_any*>(p)); }
__device__ __forceinline__ uint2 load8(const void* p) { return __builtin_bit_cast(uint2, (ts_u32x2)*reinterpret_cast<const ts_u32x2_any*>(p)); }
typedef uint32_t ts_u32_any __attribute__((aligned(2)));
__device__ __forceinline__ uint32_t load4(const void* p) { return *reinterpret_cast<const ts_u32_any*>(p); }
__device__ __forceinline__ void store4(void* p, uint32_t v) { *reinterpret_cast<ts_u32_any*>(p) = v; }
__device__ __forceinline__ void store16(void* p, uint4 v) { *reinterpret_cast<ts_u32x4_any*>(p) = __builtin_bit_cast(ts_u32x4, v); }
__device__ __forceinline__ void store8(void* p, uint2 v) { *reinterpret_cast<ts_u32x2_any*>(p) = __builtin_bit_cast(ts_u32x2, v); }

// Barrier that waits for the LDS alone: global loads stay in flight across it.
__device__ __forceinline__ void wait_lds() { wait_loads<63>(); }

// One conversion instruction of gfx950 per pair of values.
__device__ __forceinline__ ts_bf16x2 to_bf16x2(float a, float b) {
  const ts_f32x2 v = {a, b};
  return __builtin_convertvector(v, ts_bf16x2);
}
// fp32 as a sum of bf16 terms of one sign: each is the rest so far cut to bf16, the last rounded to nearest, so three carry all
// 24 significant bits (a rest below bf16's smallest subnormal, 2^-133, is lost).  Cut, not rounded: the first term of a number next
// to the largest would round to infinity, and a product that overflows in the first term would meet another of the opposite sign.
// Infinities stay in the first term, NaN in the last.
template <int N>
__device__ __forceinline__ void split_bf16x2(float a, float b, ts_bf16x2 (&t)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i + 1 == N) { t[i] = to_bf16x2(a, b); break; }
    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
    t[i] = __builtin_bit_cast(ts_bf16x2, __builtin_amdgcn_perm(ub, ua, 0x07060302u));        // the high halves of both
    const float ra = a - __uint_as_float(ua & 0xffff0000u), rb = b - __uint_as_float(ub & 0xffff0000u);
    a = i == 0 && fabsf(a) == INFINITY ? 0.f : ra;
    b = i == 0 && fabsf(b) == INFINITY ? 0.f : rb;
  }
}

// Terms that meet infinities: 0 times infinity is NaN, so where the first term is not zero no other is either, the least that
// bf16 holds (2^-133, as much as a term's rest may lose) in its place, of the same sign.
typedef uint16_t ts_u16x2 __attribute__((ext_vector_type(2)));
template <int N>
__device__ __forceinline__ void split_bf16x2_nonzero(float a, float b, ts_bf16x2 (&t)[N]) {
  split_bf16x2<N>(a, b, t);
  const ts_u16x2 first = __builtin_bit_cast(ts_u16x2, t[0]), sign = first & (uint16_t)0x8000;
  const ts_u16x2 least = __builtin_elementwise_min((ts_u16x2)(first & (uint16_t)0x7fff), (ts_u16x2)(uint16_t)1) | sign;
#pragma unroll
  for (int i = 1; i < N; ++i)                                    // magnitudes order like their bit patterns, and all have one sign
    t[i] = __builtin_bit_cast(ts_bf16x2, __builtin_elementwise_max(__builtin_bit_cast(ts_u16x2, t[i]) | sign, least));
}

// the weights of a model with 4-bit projections (ts_mx.hip), used by the passes of toolspec.h
size_t mx_packed_bytes(int64_t n_out, int64_t n_in);
void launch_mx_quantize(hipStream_t s, const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t row_stride, uint8_t* codes, uint8_t* scales);
// tiles of 16 rows go to tile n_tile0 + i * n_tile_stride of `packed`; range_flag (may be null) is set where a value would not
// fit IEEE half
void launch_mx_pack(hipStream_t s, const uint8_t* codes, const uint8_t* scales, int n_out, int n_in, void* packed, int n_tile0, int n_tile_stride,
                    int* range_flag);
