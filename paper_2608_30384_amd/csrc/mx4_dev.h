// Device helpers of the microscaled 4-bit (MX4) rows: E2M1 codes, two to a
// byte with the lower coordinate in the low nibble, and one E8M0 scale
// 2^(s - 127) for every 32 coordinates (s = 255: NaN).  A row of D coordinates
// takes steps = ceil(D / 128) groups of 64 bytes of codes and 4 scales, zero
// past D, so that every group of 128 coordinates is one operand of the scaled
// matrix instruction and starts on a 64-byte boundary.  And of the 8-bit (MX8)
// rows: E4M3 codes, a byte each, 128 bytes to a group, with the same scales.
#pragma once

#include "rslm_internal.h"

namespace rslm {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kMx4MaxDim = 65536;
constexpr int64_t kMx4MaxRows = 0x7fffff00;   // workgroups of 128 rows, 256 threads each, stay below 2^32 threads

__host__ __device__ inline int mx4_steps(int dim) { return (dim + 127) / 128; }

// Elements of float rows at any element alignment.
struct __attribute__((packed, aligned(4))) F32x8u {
  float v[8];
};
struct __attribute__((packed, aligned(2))) H16x8u {
  uint16_t v[8];
};

template <int T>
struct FloatType;
template <>
struct FloatType<RSLM_F32> {
  typedef float type;
};
template <>
struct FloatType<RSLM_F16> {
  typedef _Float16 type;
};
template <>
struct FloatType<RSLM_BF16> {
  typedef __bf16 type;
};

__host__ __device__ inline int float_bytes(int dtype) { return dtype == RSLM_F32 ? 4 : 2; }

template <int T>
__device__ __forceinline__ float h16_to_float(uint16_t u) {
  if constexpr (T == RSLM_F16) return float(__builtin_bit_cast(_Float16, u));
  else return __uint_as_float(uint32_t(u) << 16);
}
// to 16 bits, to nearest even
template <int T>
__device__ __forceinline__ uint16_t float_to_h16(float f) {
  if constexpr (T == RSLM_F16) return __builtin_bit_cast(uint16_t, _Float16(f));
  else return __builtin_bit_cast(uint16_t, __bf16(f));
}

// One element of a float row.
template <int T>
__device__ __forceinline__ float load_float(const void *p, int64_t i) {
  if constexpr (T == RSLM_F32) return static_cast<const float *>(p)[i];
  else return h16_to_float<T>(static_cast<const uint16_t *>(p)[i]);
}
template <int T>
__device__ __forceinline__ void store_float(void *p, int64_t i, float f) {
  if constexpr (T == RSLM_F32) static_cast<float *>(p)[i] = f;
  else static_cast<uint16_t *>(p)[i] = float_to_h16<T>(f);
}

// row[c .. c + 7] as they are stored, 0 at and past dim.  Kept so until every
// load of a thread is out: a conversion beside its load would wait for it.
template <int T>
struct Raw8 {
  typename FloatType<T>::type v[8];
};
template <int T>
__device__ __forceinline__ void load_raw8(Raw8<T> &p, const void *row, int c, int dim) {
  typedef typename FloatType<T>::type F;
  const F *x = static_cast<const F *>(row) + c;
  if (c + 8 <= dim) {
    if constexpr (T == RSLM_F32) {
      const F32x8u a = *reinterpret_cast<const F32x8u *>(x);
      __builtin_memcpy(&p, &a, sizeof(a));
    } else {
      const H16x8u a = *reinterpret_cast<const H16x8u *>(x);
      __builtin_memcpy(&p, &a, sizeof(a));
    }
  } else if (c < dim) {
    F e[8];   // a branch for each would wait for each
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = x[min(i, dim - 1 - c)];
#pragma unroll
    for (int i = 0; i < 8; ++i) p.v[i] = c + i < dim ? e[i] : F(0.f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p.v[i] = F(0.f);
  }
}
template <int T>
__device__ __forceinline__ void raw_values(float (&v)[8], const Raw8<T> &p) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = float(p.v[i]);
}

// v[i] = row[c + i], 0 at and past dim.
template <int T>
__device__ __forceinline__ void load_float8(float (&v)[8], const void *row, int c, int dim) {
  Raw8<T> p;
  load_raw8<T>(p, row, c, dim);
  raw_values<T>(v, p);
}
template <int T>
__device__ __forceinline__ void store_float8(const float (&v)[8], void *row, int c, int dim) {
  if (c + 8 <= dim) {
    if constexpr (T == RSLM_F32) {
      F32x8u a;
#pragma unroll
      for (int i = 0; i < 8; ++i) a.v[i] = v[i];
      *reinterpret_cast<F32x8u *>(static_cast<float *>(row) + c) = a;
    } else {
      H16x8u a;
#pragma unroll
      for (int i = 0; i < 8; ++i) a.v[i] = float_to_h16<T>(v[i]);
      *reinterpret_cast<H16x8u *>(static_cast<uint16_t *>(row) + c) = a;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < dim) store_float<T>(row, c + i, v[i]);
  }
}

struct __attribute__((packed, aligned(4))) F32x4u {
  float v[4];
};
struct __attribute__((packed, aligned(2))) H16x4u {
  uint16_t v[4];
};

// row[c .. c + 3] = v of a row that ends at n.
template <int T>
__device__ __forceinline__ void store_float4(void *row, int64_t c, int64_t n, f32x4 v) {
  if (c + 4 <= n) {
    if constexpr (T == RSLM_F32) {
      *reinterpret_cast<F32x4u *>(static_cast<float *>(row) + c) = F32x4u{{v[0], v[1], v[2], v[3]}};
    } else {
      *reinterpret_cast<H16x4u *>(static_cast<uint16_t *>(row) + c) =
          H16x4u{{float_to_h16<T>(v[0]), float_to_h16<T>(v[1]), float_to_h16<T>(v[2]), float_to_h16<T>(v[3])}};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < n) store_float<T>(row, c + i, v[i]);
  }
}

// The scale of an E8M0 code as the conversions take it: they read the float's
// exponent field alone, as such a code (field 0 is 2^-127, field 255 NaN).
__device__ __forceinline__ float e8m0_arg(uint32_t s) { return __uint_as_float(s << 23); }

// E8M0 code of a block whose largest magnitude has the float32 bits `top`
// (sign cleared): 2^(floor(log2 top) - 2), so that the largest coordinate
// falls in [4, 8) of the codes' range of 6; a block with an infinity or a NaN
// takes the NaN scale, which E2M1 itself cannot express.
__device__ __forceinline__ uint32_t e8m0_code(uint32_t top) {
  const uint32_t e = top >> 23;
  return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}

// Codes of 8 coordinates at the scale s: to nearest, ties to the even code,
// saturated at 6 (v_cvt_scalef32_pk_fp4_f32).
__device__ __forceinline__ uint32_t mx4_codes8(const float (&v)[8], uint32_t s) {
  const float a = e8m0_arg(s);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], a, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], a, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], a, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], a, 3);
  return s == 255u ? 0u : w;
}

// Values of the 8 codes of w at the scale s.
__device__ __forceinline__ void mx4_values8(float (&v)[8], uint32_t w, uint32_t s) {
  const float a = e8m0_arg(s);
  const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, a, 0);
  const f32x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, a, 1);
  const f32x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, a, 2);
  const f32x2 p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, a, 3);
  v[0] = p0.x, v[1] = p0.y, v[2] = p1.x, v[3] = p1.y;
  v[4] = p2.x, v[5] = p2.y, v[6] = p3.x, v[7] = p3.y;
}
// Of the 4 codes of w's lower half.
__device__ __forceinline__ f32x4 mx4_values4(uint32_t w, uint32_t s) {
  const float a = e8m0_arg(s);
  const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, a, 0);
  const f32x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, a, 1);
  return f32x4{p0.x, p0.y, p1.x, p1.y};
}
// 8 codes' values in bfloat16, which holds every such value exactly.
__device__ __forceinline__ uint4 mx4_bf16x8(uint32_t w, float a) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, a, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, a, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, a, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, a, 3)));
}

// E8M0 code of a block of E4M3 codes, of the largest magnitude's bits: the least
// scale that keeps it within their 448 = 1.75 2^8, so that no code saturates and
// every rounding is by half a unit (2^-4 of a value) at most.
__device__ __forceinline__ uint32_t e8m0_code8(uint32_t top) {
  const uint32_t e = (top >> 23) + ((top & 0x7fffffu) > 0x600000u);
  return top >= 0x7f800000u ? 255u : e > 8u ? e - 8u : 0u;
}

typedef short i16x2 __attribute__((ext_vector_type(2)));

// E4M3 codes of 8 coordinates at the scale s, to nearest, ties to the even code.
__device__ __forceinline__ uint2 mx8_codes8(const float (&v)[8], uint32_t s) {
  const float a = e8m0_arg(s);
  i16x2 lo = {0, 0}, hi = {0, 0};
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, v[0], v[1], a, false);
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, v[2], v[3], a, true);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, v[4], v[5], a, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, v[6], v[7], a, true);
  return s == 255u ? make_uint2(0u, 0u)
                   : make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}
// Values of the 4 codes of w at the scale s.
__device__ __forceinline__ f32x4 mx8_values4(uint32_t w, uint32_t s) {
  const float a = e8m0_arg(s);
  const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(int(w), a, false);
  const f32x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(int(w), a, true);
  return f32x4{p0.x, p0.y, p1.x, p1.y};
}
__device__ __forceinline__ void mx8_values8(float (&v)[8], uint2 w, uint32_t s) {
  const f32x4 a = mx8_values4(w.x, s), b = mx8_values4(w.y, s);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
}
// 8 codes' values in bfloat16, which holds every one of 2^-130 and more exactly.
__device__ __forceinline__ uint4 mx8_bf16x8(uint2 w, float a) {
  return make_uint4(
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(w.x), a, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(w.x), a, true)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(w.y), a, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(w.y), a, true)));
}

// ---- loads from memory to LDS, which go past the registers

__device__ __forceinline__ i32x4 buffer_of(const uint8_t *p, int64_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  i32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane(int(a));
  r[1] = __builtin_amdgcn_readfirstlane(int(a >> 32) & 0xffff);
  r[2] = __builtin_amdgcn_readfirstlane(int(bytes > 0xffffffffll ? 0xffffffffll : bytes));
  r[3] = 0x00020000;   // raw, 32-bit; reads past the end give 0
  return r;
}
// 64 lanes x 16 (or 4) bytes from the buffer to LDS, lane l's at lds + 16 (4) l.  The LDS
// address goes in m0, which the compiler writes, as it may hold a value of its own
// there; one instruction has to come between (it may be the s_nop).
// The whole offset is the lane's, which the end of the buffer is checked against.
template <int BYTES = 16>
__device__ __forceinline__ void load_to_lds(i32x4 buf, uint32_t lds, uint32_t offset) {
  static_assert(BYTES == 16 || BYTES == 4);
  asm volatile("s_nop 0\n\t"
               ".if %3 == 16\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds\n\t"
               ".else\n\tbuffer_load_dword %1, %2, 0 offen lds\n\t.endif"
               :
               : "{m0}"(lds), "v"(offset), "s"(buf), "n"(BYTES)
               : "memory");
}
// The same from 64 addresses, one of each lane.
__device__ __forceinline__ void load_to_lds(const void *p, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "{m0}"(lds), "v"(p) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char *)p));
}
// At most N of the wavefront's loads are still out, and its LDS reads are done;
// then every wavefront's.
template <int N>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
// The wavefront's LDS writes and reads are done; then every wavefront's.
__device__ __forceinline__ void arrive_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

inline bool float_type_ok(int dtype) {
  return dtype == RSLM_F32 || dtype == RSLM_F16 || dtype == RSLM_BF16;
}
inline bool aligned_to(const void *p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace rslm
