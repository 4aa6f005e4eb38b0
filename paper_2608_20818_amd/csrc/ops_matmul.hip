// 8-bit product of the linear layer on gfx950:
//
//   out[i][j] = a_scale[i] b_scale[j] sum_k a[i][k] b[j][k]  (+ bias[j])
//
// a (tokens) and b (output channels) both have k along their rows.  The sums are exact
// in 32-bit whole numbers (v_mfma_i32_32x32x32_i8, v_mfma_i32_16x16x64_i8), so neither
// the order of the sum nor how it is split changes a bit of the result; the scales are
// applied in fp32 and the result is rounded once.
#include <type_traits>

#include "ops_device.h"

namespace prm {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));

// 16 bytes of a row from k, which may start on any byte; zeros behind the row's end
__device__ __forceinline__ u32x4_t load_k16(const int8_t* row, int64_t k, int64_t klen) {
  if (k + 16 <= klen) {
    const u32x4b_t x = *(const PRM_GLOBAL u32x4b_t*)(row + k);
    return u32x4_t{x[0], x[1], x[2], x[3]};
  }
  u32x4_t v = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (k + i < klen) v[i >> 2] |= (uint32_t)(uint8_t)*gptr(row + k + i) << (8 * (i & 3));
  return v;
}

template <class E> struct Out4;  // four consecutive outputs

template <class E>
__device__ __forceinline__ void store4(typename E::S* row, int64_t c, int64_t n, const float v[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (c + k < n) E::store1(row + c + k, v[k]);
}

// ---------------------------------------------------------------------------
// tiles: four waves, 64 x 64 outputs each or 32 x 32, operands staged through
// registers into shared memory, any alignment
// ---------------------------------------------------------------------------
template <class E, int BM, int BN>
__global__ __launch_bounds__(256) void tile_kernel(ProductArgs p, int tiles_m) {
  constexpr int BK = 128;            // bytes of k a stage
  constexpr int WM = BM / 2, WN = BN / 2, MI = WM / 32, NI = WN / 32;
  constexpr int LA = BM * 8 / 256, LB = BN * 8 / 256;  // 16-byte pieces a thread loads
  __shared__ __attribute__((aligned(16))) char sa[2][BM * BK];
  __shared__ __attribute__((aligned(16))) char sb[2][BN * BK];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int64_t row0 = (int64_t)(blockIdx.x % tiles_m) * BM, col0 = (int64_t)(blockIdx.x / tiles_m) * BN;
  // piece ch of row r lies at ch ^ (r / 2 % 8): rows read together hit distinct banks
  auto at = [](int r, int ch) __attribute__((always_inline)) { return r * BK + ((ch ^ ((r >> 1) & 7)) << 4); };
  u32x4_t ra[LA], rb[LB];
  const int ch = tid & 7, r0 = tid >> 3;
  auto fetch = [&](int64_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LA; ++i) ra[i] = load_k16(p.a + min(row0 + r0 + 32 * i, p.m - 1) * p.lda, k + 16 * ch, p.k);
#pragma unroll
    for (int i = 0; i < LB; ++i) rb[i] = load_k16(p.b + min(col0 + r0 + 32 * i, p.n - 1) * p.ldb, k + 16 * ch, p.k);
  };
  auto put = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LA; ++i) *reinterpret_cast<u32x4_t*>(sa[s] + at(r0 + 32 * i, ch)) = ra[i];
#pragma unroll
    for (int i = 0; i < LB; ++i) *reinterpret_cast<u32x4_t*>(sb[s] + at(r0 + 32 * i, ch)) = rb[i];
  };
  i32x16_t acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = i32x16_t{};
  fetch(0);
  put(0);
  __syncthreads();
  int s = 0;
  for (int64_t k = 0; k < p.k; k += BK) {
    const bool more = k + BK < p.k;
    if (more) fetch(k + BK);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      i32x4_t fa[MI], fb[NI];
#pragma unroll
      for (int i = 0; i < MI; ++i)
        fa[i] = *reinterpret_cast<const i32x4_t*>(sa[s] + at(wm * WM + 32 * i + (lane & 31), 2 * ks + (lane >> 5)));
#pragma unroll
      for (int j = 0; j < NI; ++j)
        fb[j] = *reinterpret_cast<const i32x4_t*>(sb[s] + at(wn * WN + 32 * j + (lane & 31), 2 * ks + (lane >> 5)));
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
    if (more) put(s ^ 1);
    __syncthreads();
    s ^= 1;
  }
  // lane L holds output row 32 i + L % 32 and, of each block of columns, 8 q + 4 (L / 32) + 0..3
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int64_t r = row0 + wm * WM + 32 * i + (lane & 31);
    if (r >= p.m) continue;
    const float as = *gptr(p.a_scale + r);
    typename E::S* out = (typename E::S*)p.out + r * p.ldo;
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t c = col0 + wn * WN + 32 * j + 8 * q + 4 * (lane >> 5);
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t cc = min(c + e, p.n - 1);
          v[e] = (float)acc[i][j][4 * q + e] * as * *gptr(p.b_scale + cc);
          if (p.bias) v[e] += E::load1((const typename E::S*)p.bias + cc);
        }
        store4<E>(out, c, p.n, v);
      }
  }
}

// ---------------------------------------------------------------------------
// few tokens: 16 channels a block, read once and straight into registers; the
// block's waves split k and join their sums in shared memory
// ---------------------------------------------------------------------------
template <class E, int MT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(ProductArgs p) {
  __shared__ __attribute__((aligned(16))) i32x4_t part[WAVES][MT][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int kg = 16 * (lane >> 4);
  const int8_t* b = p.b + min(n0 + (lane & 15), p.n - 1) * p.ldb;
  const int8_t* a[MT];
  i32x4_t acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    a[t] = p.a + min((int64_t)(16 * t + (lane & 15)), p.m - 1) * p.lda;
    acc[t] = i32x4_t{};
  }
  // wave w takes the pieces of 256 bytes of k w, w + WAVES, ...
  for (int64_t k = 256 * wave; k < p.k; k += 256 * WAVES) {
    u32x4_t fb[4], fa[4][MT];
#pragma unroll
    for (int u = 0; u < 4; ++u) fb[u] = load_k16(b, k + 64 * u + kg, p.k);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int t = 0; t < MT; ++t) fa[u][t] = load_k16(a[t], k + 64 * u + kg, p.k);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int t = 0; t < MT; ++t)
        acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, fb[u]), __builtin_bit_cast(i32x4_t, fa[u][t]),
                                                       acc[t], 0, 0, 0);
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) part[wave][t][lane] = acc[t];
  __syncthreads();
  // lane L of tile t: token 16 t + L % 16, channels 4 (L / 16) + 0..3
  for (int t = wave; t < MT; t += WAVES) {
    i32x4_t sum = part[0][t][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += part[w][t][lane];
    const int64_t r = 16 * t + (lane & 15), c = n0 + 4 * (lane >> 4);
    if (r >= p.m) continue;
    const float as = *gptr(p.a_scale + r);
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t cc = min(c + e, p.n - 1);
      v[e] = (float)sum[e] * as * *gptr(p.b_scale + cc);
      if (p.bias) v[e] += E::load1((const typename E::S*)p.bias + cc);
    }
    store4<E>((typename E::S*)p.out + r * p.ldo, c, p.n, v);
  }
}

template <class E>
hipError_t launch(const ProductArgs& p, hipStream_t s) {
  if (p.m == 0 || p.n == 0) return hipSuccess;
  if (p.m <= 64) {
    const unsigned g = (unsigned)((p.n + 15) / 16);
    if (p.m <= 16) few_kernel<E, 1, 8><<<g, 512, 0, s>>>(p);
    else if (p.m <= 32) few_kernel<E, 2, 8><<<g, 512, 0, s>>>(p);
    else few_kernel<E, 4, 8><<<g, 512, 0, s>>>(p);
    return hipGetLastError();
  }
  const int64_t tm = (p.m + 127) / 128, tn = (p.n + 127) / 128;
  if (tm * tn >= 256) {
    tile_kernel<E, 128, 128><<<(unsigned)(tm * tn), 256, 0, s>>>(p, (int)tm);
  } else {
    const int64_t um = (p.m + 63) / 64, un = (p.n + 63) / 64;
    tile_kernel<E, 64, 64><<<(unsigned)(um * un), 256, 0, s>>>(p, (int)um);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_int8_matmul(OpType t, const ProductArgs& p, hipStream_t s) {
  return t == OP_F32 ? launch<TF32>(p, s) : t == OP_BF16 ? launch<TBF16>(p, s) : launch<TF16>(p, s);
}

}  // namespace prm
