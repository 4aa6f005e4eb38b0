// Device helpers of the operators: typed access to 8 consecutive elements that
// start on any element, and the 8-bit rounding.
#pragma once

#include <type_traits>

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

// 16-bit elements moved down by n of 8, zeros behind
__device__ __forceinline__ u32x4e_t moved_down(const u32x4e_t& r, int n) {
  const uint64_t lo = (uint64_t)r[1] << 32 | r[0], hi = (uint64_t)r[3] << 32 | r[2];
  const int b = 16 * n;
  const uint64_t l = b == 0 ? lo : b < 64 ? lo >> b | hi << (64 - b) : hi >> (b - 64);
  const uint64_t h = b < 64 ? hi >> b : 0;
  return u32x4e_t{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
}
__device__ __forceinline__ TF32::Raw moved_down(const TF32::Raw& r, int n) {
  float v[8];
  TF32::expand(r, v);
#pragma unroll
  for (int step = 1; step < 8; step <<= 1) {
    const bool on = n & step;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = on ? (k + step < 8 ? v[k + step] : 0.f) : v[k];
  }
  return TF32::pack(v);
}
// 8 elements of a row at column c < cols: whole, or the row's last ones with zeros behind
template <class E>
__device__ __forceinline__ typename E::Raw load_row8(const typename E::S* row, int64_t c, int64_t cols) {
  if (c + 8 <= cols) return E::load8(row + c);
  float v[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = c + k < cols ? E::load1(row + c + k) : 0.f;
  return E::pack(v);  // exact: the values are of the type
}
// The same in one load: at the row's end its last 8 elements, moved down.  For sweeps that
// wait for each load (statistics of 1024 x 645: 12 us, with the other 14); it costs
// registers that the kernels of whole rows need (gradient of 8192 x 4096: 69 us, 55).
template <class E>
__device__ __forceinline__ typename E::Raw load_end8(const typename E::S* row, int64_t c, int64_t cols) {
  if (cols < 8) return load_row8<E>(row, c, cols);
  const int64_t from = min(c, cols - 8);
  const typename E::Raw r = E::load8(row + from);
  return c == from ? r : moved_down(r, (int)(c - from));
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
// q = the whole number nearest to 127 u / top, ties to even, decided exactly.  In fp32,
// adding 1.5 * 2^23 to u inv (inv = 127 / top) rounds the product, unrounded before, to a
// whole number, which the sum's low byte holds.  inv alone is inexact, and where that
// could move a value over a border of two whole numbers depends on what u is:
//
// VALUES: u and top are values of a 16-bit type, U 2^a and T 2^b with whole U, T < 2^11.
// The quotient is 127 U / (T 2^j), and off a border k + 1/2 by a whole multiple of
// 1 / (2 T 2^j), which is (k + 1/2) / 254 U or more: at least 1.9e-6 of the border.  With inv
// rounded UP (an error of less than 2^-23 = 1.2e-7) only values ON a border can fall
// wrong.  There 127 U = T 2^(j-1) (2 k + 1), so the prime 127 divides 2 k + 1, which is
// k = 63 alone, where the upwards error gives the even 64; or it divides T, one number
// for the whole row, whose values are then decided by themselves.
//
// PRODUCT32, WIDE: u is a product of bf16 values (16 bits), or any fp32 or fp64 value.  What
// the rounding leaves over says how far from the border it fell.  inv is off by 3 * 2^-24 at
// most, and u by 2^-24 (fp32 products: none): 127 * 4 * 2^-24 = 3.1e-5, so where the
// remainder stays 4e-5 clear of 1/2 the number is right.
//
// Otherwise comparing 254 |u| with (2 k + 1) top decides, in a type that holds both exactly:
// fp32 (24 bits; 255 top is in its range up to 1.3e36) but for WIDE and rows too small or too
// large for that, which take fp64 (products of fp32 values: to its last bit).
// 16384 x 4096 bf16 rows: 34 us; with a check for each value 38, for each 8 values 45
// (values on a border, half the largest above all, are common there).
enum EightKind { VALUES, PRODUCT32, WIDE };
template <typename U, EightKind K>
struct Eight {
  using X = std::conditional_t<K == WIDE, double, float>;
  U top;      // max |u| of the row
  float inv;  // 0: every q is 0 (a row of zeros, or one with a value that is not finite)
  bool fp32;  // fp32 decides: always (VALUES), or where it can
  Eight() = default;
  __device__ __forceinline__ explicit Eight(U t) : top(t) {
    fp32 = t > (U)1e-35f && t < (U)1e36f;
    inv = fp32 ? 127.f / (float)t : 0.f;
    if (fmaf(inv, (float)t, -127.f) < 0.f && fp32) inv = __uint_as_float(__float_as_uint(inv) + 1);
    if constexpr (K == VALUES) fp32 = fp32 && ((__float_as_uint(t) & 0x7fffffu) | 0x800000u) % 127u != 0;
  }
  __device__ __forceinline__ bool finite() const { return top < (U)__builtin_huge_valf(); }
  // k or k + 1 of |u|
  template <typename Y>
  __device__ __forceinline__ int side(U u, int k) const {
    const Y l = (Y)254 * (Y)(u < 0 ? -u : u), r = (Y)(2 * k + 1) * (Y)top;
    const int q = l > r ? k + 1 : l < r ? k : k + (k & 1);
    return u < 0 ? -q : q;
  }
  // From the floor of the quotient; next to a whole number that may be the one below, with
  // the same q.
  __device__ __forceinline__ int exactly(U u) const {
    if (inv > 0.f) return side<X>(u, (int)floorf(fabsf((float)u * inv)));
    if (!(top > (U)0) || !finite()) return 0;
    return side<double>(u, (int)floor(127.0 * (fabs((double)u) / (double)top)));
  }
  // q of one value in the low byte; `rest`: the largest |remainder| so far
  __device__ __forceinline__ uint32_t fast(U u, float& rest) const {
    constexpr float kMagic = 12582912.f;
    const float n = fmaf((float)u, inv, kMagic);
    if constexpr (K != VALUES) rest = fmaxf(rest, fabsf(fmaf((float)u, inv, kMagic - n)));
    return __float_as_uint(n);
  }
  __device__ __forceinline__ bool sure(float rest) const { return K == VALUES ? fp32 : fp32 && rest < 0.49996f; }
  // the scale: factor * top / 127; a row with a value that is not finite has NaN
  __device__ __forceinline__ float scale(double factor) const {
    return finite() ? (float)(factor * (double)top / 127.0) : __builtin_nanf("");
  }
};
// the rounding of a type's own values
template <class E> using EightOf = Eight<float, std::is_same_v<typename E::S, float> ? WIDE : VALUES>;
// the low bytes of four words
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

// Largest magnitude, as the bits of a float, that keeps a NaN: of 16-bit values two at a
// time on their bits as stored (NaN above infinity above the finite ones).
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
template <class E> struct TopRaw {
  u16x2_t m = {0, 0};
  __device__ __forceinline__ void add(const typename E::Raw& r) {
#pragma unroll
    for (int k = 0; k < 4; ++k) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, r[k] & 0x7fff7fffu));
  }
  __device__ __forceinline__ uint32_t bits() const {
    const uint16_t h = m[0] > m[1] ? m[0] : m[1];
    float v[8];
    typename E::Raw r = {h, 0u, 0u, 0u};
    E::expand(r, v);
    return __float_as_uint(v[0]);
  }
};
template <> struct TopRaw<TF32> {
  uint32_t m = 0;
  __device__ __forceinline__ void add(const TF32::Raw& r) {
#pragma unroll
    for (int k = 0; k < 4; ++k) m = max(max(m, __float_as_uint(r.a[k]) & 0x7fffffffu), __float_as_uint(r.b[k]) & 0x7fffffffu);
  }
  __device__ __forceinline__ uint32_t bits() const { return m; }
};

}  // namespace prm
