// Device helpers of the operators: typed access to 8 consecutive elements that
// start on any element, and the 8-bit rounding.
#pragma once

#include "ops_internal.h"
#include "prm_device.h"

namespace prm {

typedef unsigned u32x4e_t __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes, 2-byte alignment
typedef unsigned u32x4b_t __attribute__((ext_vector_type(4), aligned(1)));   // 16 bytes, any alignment
typedef unsigned u32x2e_t __attribute__((ext_vector_type(2), aligned(2)));   // 8 bytes, 2-byte alignment
typedef unsigned u32x2b_t __attribute__((ext_vector_type(2), aligned(1)));   // 8 bytes, any alignment

struct TF32 {
  using S = float;
  struct Raw { f32x4u_t a, b; };
  __device__ __forceinline__ static Raw load8(const S* p) {
    return {*(const PRM_GLOBAL f32x4u_t*)p, *(const PRM_GLOBAL f32x4u_t*)(p + 4)};
  }
  __device__ __forceinline__ static void expand(const Raw& r, float v[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) { v[k] = r.a[k]; v[4 + k] = r.b[k]; }
  }
  __device__ __forceinline__ static Raw pack(const float v[8]) {
    return {f32x4u_t{v[0], v[1], v[2], v[3]}, f32x4u_t{v[4], v[5], v[6], v[7]}};
  }
  __device__ __forceinline__ static void store8(S* p, const Raw& r) {
    *(PRM_GLOBAL f32x4u_t*)p = r.a;
    *(PRM_GLOBAL f32x4u_t*)(p + 4) = r.b;
  }
  __device__ __forceinline__ static void store4(S* p, const float v[4]) { *(PRM_GLOBAL f32x4u_t*)p = f32x4u_t{v[0], v[1], v[2], v[3]}; }
  __device__ __forceinline__ static float load1(const S* p) { return *gptr(p); }
  __device__ __forceinline__ static void store1(S* p, float v) { *gptr(p) = v; }
};

struct TBF16 {
  using S = uint16_t;
  using Raw = u32x4e_t;
  __device__ __forceinline__ static Raw load8(const S* p) { return *(const PRM_GLOBAL Raw*)p; }
  __device__ __forceinline__ static void expand(const Raw& r, float v[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(r[k] << 16);
      v[2 * k + 1] = __uint_as_float(r[k] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ static Raw pack(const float v[8]) {
    return Raw{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]), pack_bf2(v[4], v[5]), pack_bf2(v[6], v[7])};
  }
  __device__ __forceinline__ static void store8(S* p, const Raw& r) { *(PRM_GLOBAL Raw*)p = r; }
  __device__ __forceinline__ static void store4(S* p, const float v[4]) {
    *(PRM_GLOBAL u32x2e_t*)p = u32x2e_t{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
  }
  __device__ __forceinline__ static float load1(const S* p) { return bf2f(*gptr(p)); }
  __device__ __forceinline__ static void store1(S* p, float v) { *gptr(p) = (uint16_t)f2bf(v); }
};

struct TF16 {
  using S = uint16_t;
  using Raw = u32x4e_t;
  __device__ __forceinline__ static float up(uint32_t h) { return (float)__builtin_bit_cast(_Float16, (uint16_t)h); }
  __device__ __forceinline__ static uint32_t down(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
  __device__ __forceinline__ static Raw load8(const S* p) { return *(const PRM_GLOBAL Raw*)p; }
  __device__ __forceinline__ static void expand(const Raw& r, float v[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = up(r[k] & 0xffffu);
      v[2 * k + 1] = up(r[k] >> 16);
    }
  }
  __device__ __forceinline__ static Raw pack(const float v[8]) {
    Raw r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = down(v[2 * k]) | (down(v[2 * k + 1]) << 16);
    return r;
  }
  __device__ __forceinline__ static void store8(S* p, const Raw& r) { *(PRM_GLOBAL Raw*)p = r; }
  __device__ __forceinline__ static void store4(S* p, const float v[4]) {
    *(PRM_GLOBAL u32x2e_t*)p = u32x2e_t{down(v[0]) | (down(v[1]) << 16), down(v[2]) | (down(v[3]) << 16)};
  }
  __device__ __forceinline__ static float load1(const S* p) { return up(*gptr(p)); }
  __device__ __forceinline__ static void store1(S* p, float v) { *gptr(p) = (uint16_t)down(v); }
};

// 8 elements of a row at column c < cols: whole, or the row's last ones with zeros behind
template <class E>
__device__ __forceinline__ typename E::Raw load_row8(const typename E::S* row, int64_t c, int64_t cols) {
  if (c + 8 <= cols) return E::load8(row + c);
  float v[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = c + k < cols ? E::load1(row + c + k) : 0.f;
  return E::pack(v);  // exact: the values are of the type
}
template <class E>
__device__ __forceinline__ void store_row8(typename E::S* row, int64_t c, int64_t cols, const typename E::Raw& r) {
  if (c + 8 <= cols) {
    E::store8(row + c, r);
    return;
  }
  float v[8];
  E::expand(r, v);
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (c + k < cols) E::store1(row + c + k, v[k]);
}
__device__ __forceinline__ void store_q8(int8_t* row, int64_t c, int64_t cols, const u32x2b_t& r) {
  if (c + 8 <= cols) {
    *(PRM_GLOBAL u32x2b_t*)(row + c) = r;
    return;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (c + k < cols) *gptr(row + c + k) = (int8_t)((r[k >> 2] >> (8 * (k & 3))) & 0xffu);
}

// ---- 8 bits ----------------------------------------------------------------------
// q = the whole number nearest to 127 u / top, ties to even, decided exactly: in fp32
// where the quotient lies clear of a border of two whole numbers, and otherwise (about
// one value in 5000) by comparing 254 |u| with (2 k + 1) top in fp64, which holds both
// (fp32 products u: to its last bit).  The fp32 quotient is off by at most five
// roundings of 2^-24, 127 * 5 * 2^-24 = 3.8e-5, so 1e-4 is clear.  u and top are first
// scaled by a power of two that brings top near 1: no row is too small or too large.
__device__ __forceinline__ int ilogb_(float t) { return __builtin_amdgcn_frexp_expf(t); }
__device__ __forceinline__ int ilogb_(double t) { return __builtin_amdgcn_frexp_exp(t); }

template <typename U>
struct Eight {
  U top;      // max |u| of the row; 0, or not finite: every q is 0
  U pw;       // the power of two
  float inv;  // 127 / (top pw)
  bool some;
  __device__ __forceinline__ explicit Eight(U t) : top(t) {
    some = t > (U)0 && finite();
    int e = 0;
    if constexpr (sizeof(U) == 8) {
      e = some ? ilogb_(t) : 0;
      pw = __builtin_ldexp(1.0, -e);
    } else {
      e = some ? ilogb_(t) : 0;
      pw = __builtin_ldexpf(1.f, min(max(-e, -126), 120));
    }
    inv = some ? 127.f / (float)(t * pw) : 0.f;
  }
  __device__ __forceinline__ bool finite() const { return top < (U)__builtin_huge_valf(); }
  __device__ __forceinline__ float quotient(U u) const { return some ? (float)(u * pw) * inv : 0.f; }
  __device__ __forceinline__ static bool close(float f) { return fabsf(fabsf(f - rintf(f)) - 0.5f) < 1e-4f; }
  __device__ __forceinline__ int decide(U u, float f) const {
    const int k = (int)floorf(fabsf(f));
    const double l = 254.0 * fabs((double)u), r = (2 * k + 1) * (double)top;
    const int q = l > r ? k + 1 : l < r ? k : k + (k & 1);
    return f < 0.f ? -q : q;
  }
  __device__ __forceinline__ int operator()(U u) const {
    const float f = quotient(u);
    return close(f) ? decide(u, f) : (int)rintf(f);
  }
  // the scale: factor * top / 127; a row with a value that is not finite has NaN
  __device__ __forceinline__ float scale(float factor) const {
    return finite() ? (float)((double)factor * (double)top / 127.0) : __builtin_nanf("");
  }
};

}  // namespace prm
