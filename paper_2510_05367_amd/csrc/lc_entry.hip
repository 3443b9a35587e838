// Cache entries that are quantised as they are written and read back: groups of 32 values of a row share a power of two.
#include "../../include/lightcache.h"
#include "lc_internal.h"

namespace lc {
namespace {

constexpr int kGroup = 32;

// What a code counts: value = code * 2^e with e + 127 in the scale byte. 2^e has a bit pattern of its own at e = -127 (the
// one denormal among them), and 255 marks a group that is no number.
__device__ __forceinline__ float scale_up(int byte) {
  return __uint_as_float(byte == 255 ? 0x7fc00000u : byte ? (uint32_t)byte << 23 : 0x00400000u);
}
__device__ __forceinline__ float scale_down(int byte) {  // 2^-e; byte <= 254
  return __uint_as_float(byte == 254 ? 0x00400000u : (uint32_t)(254 - byte) << 23);
}

// Per format: codes of N neighbouring values in a packet of N * kBits / 8 bytes. kLast is the largest magnitude below 2^(kTopExp): in
// groups of the largest scale that a float can ask for, 2^(128 - kTopExp), the codes from there on stand for 2^128 and more, which
// no float holds.
template <int F> struct Code;
template <> struct Code<LC_ENTRY_INT8> {
  static constexpr int kBits = 8, kTopExp = 6;
  static constexpr float kLast = 63.f;
  static constexpr uint32_t kTopFrac = 0x7e0000u;  // 127 = 1.984375 * 2^6
  static __device__ __forceinline__ uint32_t pack4(const float (&u)[4]) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= ((uint32_t)(int)rintf(u[e]) & 0xffu) << (8 * e);
    return w;
  }
  static __device__ __forceinline__ void unpack4(uint32_t w, float (&u)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = (float)(int)(int8_t)(w >> (8 * e));
  }
};
template <> struct Code<LC_ENTRY_FP8> {
  static constexpr int kBits = 8, kTopExp = 8;
  static constexpr float kLast = 240.f;
  static constexpr uint32_t kTopFrac = 0x600000u;  // 448 = 1.75 * 2^8
  static __device__ __forceinline__ uint32_t pack4(const float (&u)[4]) {
    int w = 0;
#ifdef __HIP_DEVICE_COMPILE__
    w = __builtin_amdgcn_cvt_pk_fp8_f32(u[0], u[1], w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(u[2], u[3], w, true);
#endif
    return (uint32_t)w;
  }
  static __device__ __forceinline__ void unpack4(uint32_t w, float (&u)[4]) {
#ifdef __HIP_DEVICE_COMPILE__
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    u[0] = a[0]; u[1] = a[1]; u[2] = b[0]; u[3] = b[1];
#endif
  }
};
template <> struct Code<LC_ENTRY_FP4> {
  static constexpr int kBits = 4, kTopExp = 2;
  static constexpr float kLast = 3.f;
  static constexpr uint32_t kTopFrac = 0x400000u;  // 6 = 1.5 * 2^2
  static __device__ __forceinline__ uint32_t pack4(const float (&u)[4]) {
    uint32_t w = 0;
#ifdef __HIP_DEVICE_COMPILE__
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, u[0], u[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, u[2], u[3], 1.f, 1);
#endif
    return w & 0xffffu;
  }
  static __device__ __forceinline__ void unpack4(uint32_t w, float (&u)[4]) {
#ifdef __HIP_DEVICE_COMPILE__
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1);
    u[0] = a[0]; u[1] = a[1]; u[2] = b[0]; u[3] = b[1];
#endif
  }
};

// Four neighbouring values of a row as floats: whole and aligned packets in one load, others one by one (columns beyond the
// row are zeros).
template <class T, bool WHOLE> __device__ __forceinline__ void load4(const T* p, int left, float (&v)[4]) {
  if constexpr (WHOLE) {
    if constexpr (sizeof(T) == 4) {
      const f32x4 t = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = t[e];
    } else {
      const bf16x4 t = *reinterpret_cast<const bf16x4*>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = static_cast<float>(t[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < left ? to_f32(p[e]) : 0.f;
  }
}
template <class T, bool WHOLE> __device__ __forceinline__ void store4(T* p, int left, const float (&v)[4]) {
  if constexpr (WHOLE) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    } else {
      bf16x4 t;
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = static_cast<bf16_t>(v[e]);
      *reinterpret_cast<bf16x4*>(p) = t;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = from_f32<T>(v[e]);
  }
}
template <int F> __device__ __forceinline__ void put_codes(unsigned char* p, uint32_t w) {
  if constexpr (Code<F>::kBits == 8) *reinterpret_cast<uint32_t*>(p) = w;
  else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w;
}
template <int F> __device__ __forceinline__ uint32_t get_codes(const unsigned char* p) {
  if constexpr (Code<F>::kBits == 8) return *reinterpret_cast<const uint32_t*>(p);
  else return *reinterpret_cast<const uint16_t*>(p);
}

// A thread holds four values of a row, eight neighbouring threads a group. Rows are cut into ppr = 8 * groups packets of four. Bound by
// the bytes: 8192 x 1024 floats to 8-bit codes with a sum 21.4 us = 5.1 TB/s (a large copy 5.2), 33001 x 1000 bf16 to 4 bits with a float sum 68.8 us = 5.1.
// Rows that are not whole aligned packets load and store value by value: 8192 x 1024 floats, with a sum, in rows of 1024 and of 1025 16.6 and 25.2 us, read back
// with a sum 12.8 and 18.8 (partly out of the last-level cache).
template <int F, class X, class Y, bool WHOLE>
__global__ __launch_bounds__(256) void entry_pack_kernel(const X* x, int64_t x_ld, unsigned char* __restrict__ codes,
                                                         unsigned char* __restrict__ scales, const Y* base, Y* y, int64_t y_ld,
                                                         uint32_t packets, uint32_t ppr, int cols) {
  typedef Code<F> C;
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  const bool live = i < packets;  // (the eight threads of a group are all alive or all not)
  const int64_t row = live ? i / ppr : 0;
  const int c0 = live ? (int)(i % ppr) * 4 : 0;
  const int left = live ? cols - c0 : 0;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (left > 0) load4<X, WHOLE>(x + row * x_ld + c0, left, v);
  // magnitudes compare like their bit patterns, infinities above all numbers and NaNs above them
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  const bool number = top < 0x7f800000u;
  const int byte = number ? max((int)(top >> 23) - C::kTopExp + ((top & 0x7fffffu) > C::kTopFrac), 0) : 255;
  const float down = number ? scale_down(byte) : 0.f;
  const float most = byte == 255 - C::kTopExp ? C::kLast : INFINITY;  // (a finite value stays one)
  float u[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = number ? fminf(fmaxf(v[e] * down, -most), most) : 0.f;
  const uint32_t w = C::pack4(u);
  if (!live) return;
  put_codes<F>(codes + (int64_t)i * (C::kBits / 2), w);
  if ((threadIdx.x & 7) == 0) scales[i >> 3] = (unsigned char)byte;
  if (y != nullptr && left > 0) {
    const float up = scale_up(byte);
    float b[4] = {0.f, 0.f, 0.f, 0.f};
    if (base != nullptr) load4<Y, WHOLE>(base + row * y_ld + c0, left, b);
    C::unpack4(w, u);
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] += u[e] * up;
    store4<Y, WHOLE>(y + row * y_ld + c0, left, b);
  }
}

// The same cut; 8192 x 1024 from 8-bit codes 7.9 us, with a sum 11.6 (42 and 76 MB, partly out of the last-level cache).
template <int F, class Y, bool WHOLE>
__global__ __launch_bounds__(256) void entry_unpack_kernel(const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales,
                                                           const Y* base, Y* y, int64_t y_ld, uint32_t packets, uint32_t ppr, int cols) {
  typedef Code<F> C;
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= packets) return;
  const int64_t row = i / ppr;
  const int c0 = (int)(i % ppr) * 4, left = cols - c0;
  if (left <= 0) return;
  float u[4], b[4] = {0.f, 0.f, 0.f, 0.f};
  if (base != nullptr) load4<Y, WHOLE>(base + row * y_ld + c0, left, b);
  C::unpack4(get_codes<F>(codes + (int64_t)i * (C::kBits / 2)), u);
  const float up = scale_up(scales[i >> 3]);
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] += u[e] * up;
  store4<Y, WHOLE>(y + row * y_ld + c0, left, b);
}

struct EntryShape { int64_t groups, packets, code_bytes, total; };
// false where format or sizes are out of range
bool entry_shape(const lc_entry_args* a, EntryShape* s) {
  if (!a || a->format < LC_ENTRY_INT8 || a->format > LC_ENTRY_FP4 || a->rows <= 0 || a->cols <= 0) return false;
  const int64_t groups = ((int64_t)a->cols + kGroup - 1) / kGroup;
  if (a->rows > (((int64_t)1 << 29) - 64) / groups) return false;  // (packets of four values are counted, and launched, in 32 bits)
  s->groups = groups;
  s->packets = a->rows * groups * (kGroup / 4);
  s->code_bytes = a->rows * groups * (a->format == LC_ENTRY_FP4 ? kGroup / 2 : kGroup);
  s->total = s->code_bytes + a->rows * groups;
  return true;
}
inline bool aligned_for4(const void* p, int64_t ld, int dt) {
  const size_t b = 4 * dtype_size(dt);
  return (uintptr_t)p % b == 0 && ld % 4 == 0;
}
inline bool is_dtype(int dt) { return dt == LC_F32 || dt == LC_BF16; }

lc_status bad(int status, const char* what) { return (lc_status)op_fail(status, "%s", what); }

lc_status check_entry(const lc_entry_args* a, const void* entry, EntryShape* s) {
  if (!a) return bad(LC_ERR_ARG, "args is NULL");
  if (a->format < LC_ENTRY_INT8 || a->format > LC_ENTRY_FP4) return bad(LC_ERR_ARG, "format must be one of LC_ENTRY_INT8, LC_ENTRY_FP8, LC_ENTRY_FP4");
  if (!entry_shape(a, s)) return bad(LC_ERR_SHAPE, "rows and cols must be positive, and of less than 2^34 values in all");
  if (!entry) return bad(LC_ERR_ARG, "entry is NULL");
  if ((uintptr_t)entry % 16) return bad(LC_ERR_ARG, "entry must be 16-byte aligned");
  return LC_OK;
}

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" {

size_t lc_entry_packed_bytes(const lc_entry_args* a) {
  EntryShape s;
  return entry_shape(a, &s) ? (size_t)s.total : 0;
}

lc_status lc_op_entry_pack(const lc_entry_args* a, const void* x, void* entry, const void* base, void* y, void* stream) {
  EntryShape s;
  const lc_status st = check_entry(a, entry, &s);
  if (st != LC_OK) return st;
  if (!x) return bad(LC_ERR_ARG, "x is NULL");
  if (!is_dtype(a->x_dtype)) return bad(LC_ERR_ARG, "x_dtype must be LC_F32 or LC_BF16");
  if (a->x_ld < a->cols && a->rows > 1) return bad(LC_ERR_SHAPE, "x_ld must be at least cols");
  if (base && !y) return bad(LC_ERR_ARG, "base without y");
  if (y) {
    if (!is_dtype(a->y_dtype)) return bad(LC_ERR_ARG, "y_dtype must be LC_F32 or LC_BF16");
    if (a->y_ld < a->cols && a->rows > 1) return bad(LC_ERR_SHAPE, "y_ld must be at least cols");
    if (x == y && (a->x_dtype != a->y_dtype || (a->x_ld != a->y_ld && a->rows > 1)))
      return bad(LC_ERR_SHAPE, "in place, x and y have the same type and rows");
  }
  const int ydt = y ? a->y_dtype : LC_F32;
  const bool whole = a->cols % 4 == 0 && aligned_for4(x, a->x_ld, a->x_dtype) && (!y || aligned_for4(y, a->y_ld, ydt)) &&
                     (!base || aligned_for4(base, a->y_ld, ydt));
  unsigned char* const codes = (unsigned char*)entry;
  const unsigned blocks = (unsigned)((s.packets + 255) / 256);
#define LC_GO(F, X, Y, W)                                                                                                            \
  entry_pack_kernel<F, X, Y, W><<<blocks, 256, 0, (hipStream_t)stream>>>((const X*)x, a->x_ld, codes, codes + s.code_bytes, (const Y*)base, \
                                                                         (Y*)y, a->y_ld, (uint32_t)s.packets, (uint32_t)(s.groups * (kGroup / 4)), a->cols)
#define LC_W(F, X, Y) do { if (whole) LC_GO(F, X, Y, true); else LC_GO(F, X, Y, false); } while (0)
#define LC_T(F)                                                                                   \
  do {                                                                                            \
    if (a->x_dtype == LC_F32) { if (ydt == LC_F32) LC_W(F, float, float); else LC_W(F, float, bf16_t); }    \
    else { if (ydt == LC_F32) LC_W(F, bf16_t, float); else LC_W(F, bf16_t, bf16_t); }             \
  } while (0)
  switch (a->format) {
    case LC_ENTRY_INT8: LC_T(LC_ENTRY_INT8); break;
    case LC_ENTRY_FP8: LC_T(LC_ENTRY_FP8); break;
    default: LC_T(LC_ENTRY_FP4); break;
  }
#undef LC_T
#undef LC_W
#undef LC_GO
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LC_OK : (lc_status)op_fail(LC_ERR_HIP, "entry_pack: %s", hipGetErrorString(e));
}

lc_status lc_op_entry_unpack(const lc_entry_args* a, const void* entry, const void* base, void* y, void* stream) {
  EntryShape s;
  const lc_status st = check_entry(a, entry, &s);
  if (st != LC_OK) return st;
  if (!y) return bad(LC_ERR_ARG, "y is NULL");
  if (!is_dtype(a->y_dtype)) return bad(LC_ERR_ARG, "y_dtype must be LC_F32 or LC_BF16");
  if (a->y_ld < a->cols && a->rows > 1) return bad(LC_ERR_SHAPE, "y_ld must be at least cols");
  const bool whole = a->cols % 4 == 0 && aligned_for4(y, a->y_ld, a->y_dtype) && (!base || aligned_for4(base, a->y_ld, a->y_dtype));
  const unsigned char* const codes = (const unsigned char*)entry;
  const unsigned blocks = (unsigned)((s.packets + 255) / 256);
#define LC_GO(F, Y, W)                                                                                                                   \
  entry_unpack_kernel<F, Y, W><<<blocks, 256, 0, (hipStream_t)stream>>>(codes, codes + s.code_bytes, (const Y*)base, (Y*)y, a->y_ld, (uint32_t)s.packets, \
                                                                        (uint32_t)(s.groups * (kGroup / 4)), a->cols)
#define LC_W(F, Y) do { if (whole) LC_GO(F, Y, true); else LC_GO(F, Y, false); } while (0)
#define LC_T(F) do { if (a->y_dtype == LC_F32) LC_W(F, float); else LC_W(F, bf16_t); } while (0)
  switch (a->format) {
    case LC_ENTRY_INT8: LC_T(LC_ENTRY_INT8); break;
    case LC_ENTRY_FP8: LC_T(LC_ENTRY_FP8); break;
    default: LC_T(LC_ENTRY_FP4); break;
  }
#undef LC_T
#undef LC_W
#undef LC_GO
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LC_OK : (lc_status)op_fail(LC_ERR_HIP, "entry_unpack: %s", hipGetErrorString(e));
}

}  // extern "C"
