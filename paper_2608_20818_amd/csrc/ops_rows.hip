// Row operators of the 8-bit linear layer on gfx950: the quantiser, and the
// root-mean-square norm with the residual's addition and its gradients.
//
//   quantize    s = max |x| / 127 of the row,  q = rn(127 x / max |x|)
//   rms_norm    h = x + res (kept in the storage type),  r = (mean h^2 + eps)^(-1/2)
//               y = h r w, or y in 8 bits: as r is one number for the row, it cancels
//               from q = rn(127 h w / max |h w|) and stays in the scale r max |h w| / 127
//   gradient    n = h r, g = gy w:  dx = r (g - n mean(g n)) + gh,  dw = sum over rows of gy n
//
// All are bound by HBM.  The norm, its gradient and the quantiser of rows read each element once
// and hold it in registers as stored until the row's statistics are there (rows of at most
// 32768 elements, in the layer's launch of several quantisers 16384; longer ones are swept again);
// the quantiser of columns reads a matrix twice.  A thread holds pieces of 8 elements, so that an
// access of 16-bit values is 16 bytes a lane and one contiguous span a wave, at any alignment.
// bf16, bytes moved: norm with the residual 8192 x 5120 61 us (5.5 TB/s), with 8-bit output 58 us
// (5.0 TB/s; fp16 56, fp32 106 us), its gradient 8192 x 4096 54 us (5.0 TB/s), rows in 8 bits
// 10240 x 2560 15 us (5.4 TB/s), columns 4096 x 5120 25 us; a copy of 4 GiB reaches 6.5 TB/s, three
// streams in and two out 5.65.
#include <type_traits>

#include "ops_device.h"

namespace prm {
namespace {

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, off, 64));
  return v;
}
__device__ __forceinline__ double wave_max(double v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = fmax(v, __shfl_xor(v, off, 64));
  return v;
}
using prm::wave_sum;  // of floats
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// The largest |u|, that keeps a NaN: fp32 magnitudes as their bits (NaN above infinity
// above the finite ones), fp64 ones with a flag in the place of NaN (infinity).
template <typename U> struct Top;
template <> struct Top<float> {
  uint32_t m = 0;
  __device__ __forceinline__ void add(float u) { m = max(m, __float_as_uint(u) & 0x7fffffffu); }
  __device__ __forceinline__ float value() const { return __uint_as_float(m); }
};
template <> struct Top<double> {
  double m = 0;
  __device__ __forceinline__ void add(double u) { m = u == u ? fmax(m, fabs(u)) : (double)__builtin_huge_valf(); }
  __device__ __forceinline__ double value() const { return m; }
};

// Sum, and largest, over the threads of a row: a wave, or the whole block.
template <int TPR, typename T, typename U>
__device__ __forceinline__ void row_reduce(T& ss, Top<U>& top, bool with_sum, bool with_top, T* rs, decltype(Top<U>::m)* rt) {
  if (with_sum) ss = wave_sum(ss);
  if (with_top) top.m = wave_max(top.m);
  if constexpr (TPR > 64) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      rs[w] = ss;
      if (with_top) rt[w] = top.m;
    }
    __syncthreads();
    ss = 0;
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i) {
      ss += rs[i];
      if (with_top) top.m = max(top.m, rt[i]);
    }
  }
}

template <class U, EightKind K>
__device__ __forceinline__ u32x2b_t eight8(const Eight<U, K>& e, const U u[8]) {
  uint32_t n[8];
  float rest = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) n[k] = e.fast(u[k], rest);
  if (!e.sure(rest)) {
#pragma unroll
    for (int k = 0; k < 8; ++k) n[k] = (uint32_t)e.exactly(u[k]);
  }
  return u32x2b_t{low_bytes(n[0], n[1], n[2], n[3]), low_bytes(n[4], n[5], n[6], n[7])};
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
// TPR threads a row (64: four rows a block of 256), NCH pieces of 8 elements a
// thread; NCH 0: the row is swept twice, from memory.  MODE 0: the norm, 1: the norm
// in 8 bits, 2: the quantiser alone.
enum { NORM = 0, NORM8 = 1, QUANT = 2 };

template <class E, int TPR, int NCH, int MODE, bool RES>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void rows_kernel(NormArgs a) {
  using S = typename E::S;
  // the product h w of two 16-bit values is exact in fp32 (of bf16: within its range), that of fp32
  // values in fp64
  using U = std::conditional_t<MODE == NORM8 && sizeof(S) == 4, double, float>;
  constexpr int WPB = TPR == 64 ? 1 : TPR / 64;
  __shared__ float rs[WPB];
  __shared__ decltype(Top<U>::m) rt[WPB];
  const int t = TPR == 64 ? (threadIdx.x & 63) : threadIdx.x;
  const int64_t row = TPR == 64 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : (int64_t)blockIdx.x;
  if (TPR == 64 && row >= a.rows) return;  // whole waves, and no barrier below
  const S* x = (const S*)a.x + row * a.ldx;
  const S* res = RES ? (const S*)a.res + row * a.ldres : nullptr;
  S* hrow = RES ? (S*)a.h + row * a.ldh : nullptr;
  const S* w = (const S*)a.w;
  const int64_t cols = a.cols;
  auto weight8 = [&](int64_t c, float v[8]) __attribute__((always_inline)) {
    if (MODE == QUANT || !w) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 1.f;
    } else {
      E::expand(load_row8<E>(w, c, cols), v);
    }
  };
  // h of a piece, written where the sum is kept
  auto sum8 = [&](int64_t c) __attribute__((always_inline)) {
    typename E::Raw r = load_row8<E>(x, c, cols);
    if constexpr (RES) {
      float v[8], u[8];
      E::expand(r, v);
      E::expand(load_row8<E>(res, c, cols), u);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += u[k];
      r = E::pack(v);
      store_row8<E>(hrow, c, cols, r);
    }
    return r;
  };
  float ss = 0.f;
  Top<U> top;
  TopRaw<E> raw_top;
  auto stats = [&](int64_t c, const typename E::Raw& r) __attribute__((always_inline)) {
    float v[8];
    if (MODE != QUANT) {
      E::expand(r, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) ss += v[k] * v[k];
    }
    if (MODE == NORM8) {
      float f[8];
      weight8(c, f);
#pragma unroll
      for (int k = 0; k < 8; ++k) top.add((U)v[k] * (U)f[k]);
    }
    if (MODE == QUANT) raw_top.add(r);
  };
  constexpr int N = NCH ? NCH : 1;
  typename E::Raw held[N];
  if constexpr (NCH) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = 8 * ((int64_t)i * TPR + t);
      if (c < cols) held[i] = sum8(c);
    }
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = 8 * ((int64_t)i * TPR + t);
      if (c < cols) stats(c, held[i]);
    }
  } else {
    for (int64_t c = 8 * t; c < cols; c += 8 * TPR) stats(c, sum8(c));
  }
  if constexpr (MODE == QUANT) top.m = raw_top.bits();
  row_reduce<TPR>(ss, top, MODE != QUANT, MODE != NORM, rs, rt);
  // Rows whose squares leave fp32's range, or whose products of bf16 values do, at either end:
  // once more in fp64, from memory (the kept sum is read back by the thread that wrote it), so
  // that the other rows' registers hold none of it.
  if constexpr (MODE != QUANT && !std::is_same_v<E, TF16>) {
    bool far = !(ss < __builtin_huge_valf());
    if (MODE == NORM8 && sizeof(S) == 2) far |= !(top.value() > (U)1e-35f && top.value() < (U)1e36f);
    if (far) {
      __shared__ double ds[WPB], dt[WPB];
      const S* h = RES ? hrow : x;
      if (MODE == NORM8 && top.value() == (U)0) {
        // a row of zeros, as padding is (8192 x 5120: 57 us; through the products 72), or products
        // below fp32's range
        TopRaw<E> some;
#pragma clang loop unroll(disable)
        for (int64_t c = 8 * t; c < cols; c += 8 * TPR) some.add(load_row8<E>(h, c, cols));
        if (!(TPR == 64 ? __any(some.bits() != 0) : __syncthreads_or(some.bits() != 0))) {
#pragma clang loop unroll(disable)
          for (int64_t c = 8 * t; c < cols; c += 8 * TPR) store_q8(a.q + row * a.ldq, c, cols, u32x2b_t{0u, 0u});
          if (t == 0) a.scale[row] = 0.f;
          return;
        }
      }
      double sum = 0;
      Top<double> most;
#pragma clang loop unroll(disable)
      for (int64_t c = 8 * t; c < cols; c += 8 * TPR) {
        float v[8], f[8];
        E::expand(load_row8<E>(h, c, cols), v);
        weight8(c, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          sum += (double)v[k] * v[k];
          if (MODE == NORM8) most.add((double)v[k] * f[k]);
        }
      }
      row_reduce<TPR>(sum, most, true, MODE == NORM8, ds, dt);
      const double root = 1.0 / sqrt(sum / (double)cols + (double)a.eps);
      const Eight<double, WIDE> eight(most.value());
      if (MODE == NORM8 && t == 0) a.scale[row] = eight.scale(root);
#pragma clang loop unroll(disable)
      for (int64_t c = 8 * t; c < cols; c += 8 * TPR) {
        float v[8], f[8];
        E::expand(load_row8<E>(h, c, cols), v);
        weight8(c, f);
        if constexpr (MODE == NORM) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = (float)((double)v[k] * root * f[k]);
          store_row8<E>((S*)a.y + row * a.ldy, c, cols, E::pack(v));
        } else {
          double u[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) u[k] = (double)v[k] * f[k];
          store_q8(a.q + row * a.ldq, c, cols, eight8(eight, u));
        }
      }
      return;
    }
  }
  const float r = MODE == QUANT ? 1.f : 1.f / sqrtf(ss / (float)cols + a.eps);
  using R = std::conditional_t<MODE == QUANT, EightOf<E>, Eight<U, std::is_same_v<E, TBF16> ? PRODUCT32 : WIDE>>;
  const R eight(top.value());
  if (MODE != NORM && t == 0) a.scale[row] = eight.scale(r);
  auto out = [&](int64_t c, const typename E::Raw& raw) __attribute__((always_inline)) {
    float v[8], f[8];
    E::expand(raw, v);
    weight8(c, f);
    if constexpr (MODE == NORM) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = v[k] * r * f[k];
      store_row8<E>((S*)a.y + row * a.ldy, c, cols, E::pack(v));
    } else {
      U u[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) u[k] = (U)v[k] * (U)f[k];
      store_q8(a.q + row * a.ldq, c, cols, eight8(eight, u));
    }
  };
  if constexpr (NCH) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = 8 * ((int64_t)i * TPR + t);
      if (c < cols) out(c, held[i]);
    }
  } else {
    // the kept sum is read back by the thread that wrote it
    for (int64_t c = 8 * t; c < cols; c += 8 * TPR) out(c, load_row8<E>(RES ? hrow : x, c, cols));
  }
}

template <class E, int MODE, bool RES>
hipError_t launch_rows(const NormArgs& a, hipStream_t s) {
  // a grid holds less than 2^32 threads: more rows go in slices
  constexpr int64_t kSlice = 1 << 21;
  if (a.rows > kSlice) {
    NormArgs b = a;
    for (int64_t r = 0; r < a.rows; r += kSlice) {
      using S = typename E::S;
      b.rows = a.rows - r < kSlice ? a.rows - r : kSlice;
      b.x = (const S*)a.x + r * a.ldx;
      if (RES) {
        b.res = (const S*)a.res + r * a.ldres;
        b.h = (S*)a.h + r * a.ldh;
      }
      if (MODE == NORM) {
        b.y = (S*)a.y + r * a.ldy;
      } else {
        b.q = a.q + r * a.ldq;
        b.scale = a.scale + r;
      }
      const hipError_t e = launch_rows<E, MODE, RES>(b, s);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  if (a.rows == 0) return hipSuccess;
  const int64_t pieces = (a.cols + 7) / 8;
  const dim3 per_wave((unsigned)((a.rows + 3) / 4)), per_block((unsigned)a.rows);
#define PRM_ROWS(TPR, NCH) rows_kernel<E, TPR, NCH, MODE, RES><<<TPR == 64 ? per_wave : per_block, TPR == 64 ? 256 : TPR, 0, s>>>(a)
  if (pieces <= 64) PRM_ROWS(64, 1);
  else if (a.rows >= 2048 && pieces <= 128) PRM_ROWS(64, 2);
  else if (pieces <= 256) PRM_ROWS(256, 1);
  else if (a.rows < 512 && pieces <= 1024) PRM_ROWS(1024, 1);
  else if (pieces <= 512) PRM_ROWS(256, 2);
  else if (pieces <= 1024) PRM_ROWS(256, 4);
  else if (pieces <= 2048) PRM_ROWS(1024, 2);
  else if (pieces <= 4096) PRM_ROWS(1024, 4);
  else PRM_ROWS(1024, 0);
#undef PRM_ROWS
  return hipGetLastError();
}

template <class E>
hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  if (a.y) return a.res ? launch_rows<E, NORM, true>(a, s) : launch_rows<E, NORM, false>(a, s);
  return a.res ? launch_rows<E, NORM8, true>(a, s) : launch_rows<E, NORM8, false>(a, s);
}

// ---------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------
// A row's threads (TPR; 64: four rows a block of 256) keep their columns' share of dw over
// all the rows that they take (row, row + step, ...), and a block leaves it as one row of
// `part`; a second kernel adds those rows in order.  The next row is on its way while one
// is summed.  NCH 0 (rows over 32768): two sweeps a row, and dw in `part` itself.
template <class E, int TPR, int NCH>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void norm_grad_kernel(NormGradArgs a) {
  using S = typename E::S;
  constexpr int WPB = TPR == 64 ? 4 : TPR / 64;
  __shared__ float red[2][2][WPB];
  __shared__ float share[TPR == 64 ? 4 : 1][TPR == 64 ? 512 : 1];
  static_assert(TPR > 64 || NCH == 1, "the share of a wave");
  int t = TPR == 64 ? (threadIdx.x & 63) : threadIdx.x;
  const int wave = threadIdx.x >> 6;
  const int64_t cols = a.cols;
  const int64_t step = (int64_t)gridDim.x * (TPR == 64 ? 4 : 1);
  const S* w = (const S*)a.w;
  constexpr int N = NCH ? NCH : 1;
  float dw[N][8];
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) dw[i][k] = 0.f;
  auto weight8 = [&](int64_t c, float v[8]) __attribute__((always_inline)) {
    if (w) E::expand(load_row8<E>(w, c, cols), v);
    else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 1.f;
    }
  };
  float* const mine = a.part + (int64_t)blockIdx.x * cols;
  bool first = true;
  int flip = 0;
  // the registers of a block of 1024 hold no second row of two pieces of fp32, or of four
  constexpr bool AHEAD = NCH > 0 && (TPR < 1024 || NCH * sizeof(S) <= 4);
  typename E::Raw rh[N], rg[N], rs[N];
  auto fetch = [&](int64_t row) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = 8 * ((int64_t)i * TPR + t);
      if (c < cols) {
        rh[i] = load_row8<E>((const S*)a.h + row * a.ldh, c, cols);
        rg[i] = load_row8<E>((const S*)a.gy + row * a.ldgy, c, cols);
        if (a.gh) rs[i] = load_row8<E>((const S*)a.gh + row * a.ldgh, c, cols);
      }
    }
  };
  // sums of h^2 and of g h of a piece, h scaled by `down`; fma by name, as both loops below have
  // to come to the same bits
  auto stats = [&](int64_t c, const typename E::Raw& xh, const typename E::Raw& xg, float down, float& ss, float& sg) __attribute__((always_inline)) {
    float v[8], g[8], f[8];
    E::expand(xh, v);
    E::expand(xg, g);
    weight8(c, f);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] *= down;
      ss = fmaf(v[k], v[k], ss);
      sg = fmaf(g[k] * f[k], v[k], sg);
    }
  };
  auto swept = [&](int64_t row, float down, float& ss, float& sg) __attribute__((always_inline)) {
    ss = sg = 0.f;
#pragma clang loop unroll(disable)
    for (int64_t c = 8 * t; c < cols; c += 8 * TPR)
      stats(c, load_row8<E>((const S*)a.h + row * a.ldh, c, cols), load_row8<E>((const S*)a.gy + row * a.ldgy, c, cols), down, ss, sg);
  };
  auto joined = [&](float& ss, float& sg) __attribute__((always_inline)) {
    ss = wave_sum(ss);
    sg = wave_sum(sg);
    if constexpr (TPR > 64) {
      // two sets of slots in turn: a wave writes the next sums behind one barrier only
      if ((threadIdx.x & 63) == 0) {
        red[flip][0][wave] = ss;
        red[flip][1][wave] = sg;
      }
      __syncthreads();
      ss = sg = 0.f;
#pragma unroll
      for (int i = 0; i < WPB; ++i) {
        ss += red[flip][0][i];
        sg += red[flip][1][i];
      }
      flip ^= 1;
    }
  };
  // a piece of dx, and its share of dw (`with_dw`); r and coef = mean(g n) r are those of h scaled
  auto out = [&](int64_t row, int64_t c, const typename E::Raw& xh, const typename E::Raw& xg, const typename E::Raw& xs, float r, float coef, float down,
                 bool with_dw, float d[8]) __attribute__((always_inline)) {
    float v[8], g[8], f[8], o[8];
    E::expand(xh, v);
    E::expand(xg, g);
    weight8(c, f);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] *= down;
      d[k] = with_dw ? d[k] + g[k] * (v[k] * r) : d[k];
      o[k] = r * (g[k] * f[k] - v[k] * coef) * down;
    }
    if (a.gh) {
      E::expand(xs, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] += v[k];
    }
    store_row8<E>((S*)a.dx + row * a.lddx, c, cols, E::pack(o));
  };
  auto out_swept = [&](int64_t row, int64_t c, float r, float coef, float down, bool with_dw, float d[8]) __attribute__((always_inline)) {
    const typename E::Raw xh = load_row8<E>((const S*)a.h + row * a.ldh, c, cols);
    out(row, c, xh, load_row8<E>((const S*)a.gy + row * a.ldgy, c, cols), a.gh ? load_row8<E>((const S*)a.gh + row * a.ldgh, c, cols) : xh, r, coef, down,
        with_dw, d);
  };
  // NCH 0: dw of the row's pieces in `part` itself
  auto out_long = [&](int64_t row, float r, float coef, float down, bool with_dw) __attribute__((always_inline)) {
    for (int64_t c = 8 * t; c < cols; c += 8 * TPR) {
      float d[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) d[k] = first || c + k >= cols || !a.dw ? 0.f : mine[c + k];
      out_swept(row, c, r, coef, down, with_dw, d);
      if (a.dw)
        for (int k = 0; k < 8 && c + k < cols; ++k) mine[c + k] = d[k];
    }
    first = false;
  };
  const int64_t row0 = TPR == 64 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  int64_t row = row0;
  float far = 0.f;  // NaN once a row's sums have left fp32's range
  if (AHEAD && row < a.rows) fetch(row);
  for (; row < a.rows; row += step) {
    float ss = 0.f, sg = 0.f;
    typename E::Raw ch[N], cg[N], cs[N];
    if constexpr (NCH) {
      if (!AHEAD) fetch(row);
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        ch[i] = rh[i];
        cg[i] = rg[i];
        if (a.gh) cs[i] = rs[i];
      }
      if (AHEAD && row + step < a.rows) fetch(row + step);
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int64_t c = 8 * ((int64_t)i * TPR + t);
        if (c < cols) stats(c, ch[i], cg[i], 1.f, ss, sg);
      }
    } else {
      swept(row, 1.f, ss, sg);
    }
    joined(ss, sg);
    if (!std::is_same_v<E, TF16>) far = fmaf(ss, 0.f, fmaf(sg, 0.f, far));
    const float r = 1.f / sqrtf(ss / (float)cols + a.eps);
    const float coef = r * r * (sg / (float)cols);
    if constexpr (NCH) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int64_t c = 8 * ((int64_t)i * TPR + t);
        if (c < cols) out(row, c, ch[i], cg[i], cs[i], r, coef, 1.f, true, dw[i]);
      }
    } else {
      out_long(row, r, coef, 1.f, true);
    }
  }
  // Rows whose sums left fp32's range, once more, h scaled by a power of two: an infinite sum of
  // squares gave r = 0, so such a row has no share of dw yet, one that has an infinite sum of g h
  // alone has.  A loop of its own, as in the first one its registers cost the others a wave of four,
  // and a branch 8% (8192 x 1024 bf16: 20.8 us, 22.4).
  if (!std::is_same_v<E, TF16> && !(far == 0.f)) {
    constexpr float inf = __builtin_huge_valf();
    asm volatile("" : "+v"(t));  // nothing that is computed from it is held through the first loop
#pragma clang loop unroll(disable)
    for (row = row0; row < a.rows; row += step) {
      float ss, sg;
      swept(row, 1.f, ss, sg);
      joined(ss, sg);
      if (ss < inf && fabsf(sg) < inf) continue;
      const bool with_dw = !(ss < inf);
      constexpr float down = 0x1p-80f;  // 2^24 squares of 2^128 come to 2^120
      swept(row, down, ss, sg);
      joined(ss, sg);
      const float r = 1.f / sqrtf(ss / (float)cols + a.eps * down * down);
      const float coef = r * r * (sg / (float)cols);
      if constexpr (NCH) {
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
          const int64_t c = 8 * ((int64_t)i * TPR + t);
          if (c < cols) out_swept(row, c, r, coef, down, with_dw, dw[i]);
        }
      } else {
        out_long(row, r, coef, down, with_dw);
      }
    }
  }
  if (!a.dw) return;
  if constexpr (TPR == 64) {
    // the block's four waves, added in order
#pragma unroll
    for (int k = 0; k < 8; ++k) share[wave][8 * t + k] = dw[0][k];
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += 256) mine[c] = (share[0][c] + share[1][c]) + (share[2][c] + share[3][c]);
  } else if constexpr (NCH) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = 8 * ((int64_t)i * TPR + t);
      if (c >= cols) continue;
      if (c + 8 <= cols) {
        TF32::store8(mine + c, TF32::pack(dw[i]));
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (c + k < cols) mine[c + k] = dw[i][k];
      }
    }
  }
}

// dw[c] = sum over parts, in order: 32 threads a column take each 32nd part, and their
// sums are added in order.
template <class E>
__global__ __launch_bounds__(1024) void part_sum_kernel(const float* part, int nparts, int64_t cols, typename E::S* out) {
  __shared__ float red[32][33];
  const int tc = threadIdx.x & 31, tr = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + tc;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int i = tr; i < nparts; i += 32) s += *gptr(part + (int64_t)i * cols + c);
  }
  red[tr][tc] = s;
  __syncthreads();
  if (tr == 0 && c < cols) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += red[i][tc];
    E::store1(out + c, s);
  }
}

template <class E>
hipError_t launch_grad(const NormGradArgs& a, hipStream_t s) {
  const int64_t pieces = (a.cols + 7) / 8;
  if (a.rows > 0) {
    const unsigned blocks = (unsigned)a.nparts;
#define PRM_GRAD(TPR, NCH) norm_grad_kernel<E, TPR, NCH><<<blocks, TPR == 64 ? 256 : TPR, 0, s>>>(a)
    if (pieces <= 64) PRM_GRAD(64, 1);
    else if (pieces <= 256) PRM_GRAD(256, 1);
    else if (pieces <= 512) PRM_GRAD(256, 2);
    else if (pieces <= 1024) PRM_GRAD(1024, 1);
    else if (pieces <= 2048) PRM_GRAD(1024, 2);
    else if (pieces <= 4096) PRM_GRAD(1024, 4);
    else PRM_GRAD(1024, 0);
#undef PRM_GRAD
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dw)
    part_sum_kernel<E><<<(unsigned)((a.cols + 31) / 32), 1024, 0, s>>>(a.part, a.rows > 0 ? a.nparts : 0, a.cols, (typename E::S*)a.dw);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// quantiser of columns, transposed
// ---------------------------------------------------------------------------
// Largest magnitudes (as bits) and sums of the columns over a block of rows: 32 lanes
// of 8 columns, 8 rows at a time.
struct ColStatsShared {
  uint32_t rm[8][256];
  float rs[8][256];
};
template <class E, bool SUM>
__device__ __forceinline__ void col_stats(const QuantArgs& a, int bx, int by, ColStatsShared& sh) {
  using S = typename E::S;
  auto& rm = sh.rm;
  auto& rs = sh.rs;
  const int tc = threadIdx.x & 31, tr = threadIdx.x >> 5;
  const int64_t c = (int64_t)bx * 256 + 8 * tc;
  const int64_t r0 = (int64_t)by * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  uint32_t m[8];
  float sum[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) { m[k] = 0; sum[k] = 0.f; }
  if (c < a.cols) {
    const auto add = [&](const typename E::Raw& raw) __attribute__((always_inline)) {
      float v[8];
      E::expand(raw, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        m[k] = max(m[k], __float_as_uint(v[k]) & 0x7fffffffu);
        if (SUM) sum[k] += v[k];
      }
    };
    int64_t r = r0 + tr;
    for (; r + 24 < r1; r += 32) {  // four rows' loads together
      typename E::Raw raw[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[i] = load_end8<E>((const S*)a.x + (r + 8 * i) * a.ldx, c, a.cols);
#pragma unroll
      for (int i = 0; i < 4; ++i) add(raw[i]);
    }
    for (; r < r1; r += 8) add(load_end8<E>((const S*)a.x + r * a.ldx, c, a.cols));
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    rm[tr][8 * tc + k] = m[k];
    if (SUM) rs[tr][8 * tc + k] = sum[k];
  }
  __syncthreads();
  const int64_t cc = (int64_t)bx * 256 + threadIdx.x;
  if (cc >= a.cols) return;
  uint32_t top = 0;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    top = max(top, rm[i][threadIdx.x]);
    if (SUM) s += rs[i][threadIdx.x];
  }
  a.part_max[(int64_t)by * a.cols + cc] = top;
  if (SUM) a.part_sum[(int64_t)by * a.cols + cc] = s;
}

// A tile of 128 rows x 64 columns: a thread quantises 4 rows of 8 columns, and the tile
// leaves through shared memory as 128 bytes of each of its columns, 8 lanes a column.
template <class E>
struct ColQuantShared {
  static constexpr int LD = 33;  // words of a column: rows and columns on distinct banks
  uint32_t tile[64 * LD];
  uint32_t pm[4][64];
  float ps[4][64];
  EightOf<E> eights[64];
};
// OWN: a job may have no statistics laid out (its registers cost the others three waves of eight).
template <class E, bool SUM, bool OWN>
__device__ __forceinline__ void col_quant(const QuantArgs& a, int64_t bx, int64_t by, ColQuantShared<E>& sh) {
  using S = typename E::S;
  using E8 = EightOf<E>;
  constexpr int LD = ColQuantShared<E>::LD;
  auto& tile = sh.tile;
  auto& pm = sh.pm;
  auto& ps = sh.ps;
  auto& eights = sh.eights;
  const int64_t c0 = bx * 64, r0 = by * 128;
  const bool first = by == 0;
  const int tc = threadIdx.x & 7, tr = threadIdx.x >> 3;
  const int64_t c = c0 + 8 * tc;
  // the tile is on its way while the columns' statistics are joined
  typename E::Raw raw[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = r0 + 4 * tr + i;
    raw[i] = r < a.rows && c < a.cols ? load_row8<E>((const S*)a.x + r * a.ldx, c, a.cols) : typename E::Raw{};
  }
  {
    const int jc = threadIdx.x & 63, jr = threadIdx.x >> 6;
    if (OWN && a.nrb == 0) {
      // few rows: the block's own statistics, 32 rows at a time, joined over the wave
      uint32_t m[8];
      float s[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) { m[k] = 0; s[k] = 0.f; }
      if (c < a.cols) {
#pragma unroll 4
        for (int64_t r = tr; r < a.rows; r += 32) {
          float v[8];
          E::expand(load_end8<E>((const S*)a.x + r * a.ldx, c, a.cols), v);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            m[k] = max(m[k], __float_as_uint(v[k]) & 0x7fffffffu);
            if (SUM) s[k] += v[k];
          }
        }
      }
#pragma unroll
      for (int off = 8; off <= 32; off <<= 1)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          m[k] = max(m[k], (uint32_t)__shfl_xor((int)m[k], off, 64));
          if (SUM) s[k] += __shfl_xor(s[k], off, 64);
        }
      if (jc < 8) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          pm[jr][8 * tc + k] = m[k];
          if (SUM) ps[jr][8 * tc + k] = s[k];
        }
      }
    } else {
      uint32_t m = 0;
      float s = 0.f;
      if (c0 + jc < a.cols) {
#pragma unroll 4
        for (int i = jr; i < a.nrb; i += 4) {
          m = max(m, *gptr(a.part_max + (int64_t)i * a.cols + c0 + jc));
          if (SUM && first) s += *gptr(a.part_sum + (int64_t)i * a.cols + c0 + jc);
        }
      }
      pm[jr][jc] = m;
      if (SUM) ps[jr][jc] = s;
    }
    __syncthreads();
    if (jr == 0) {
      const uint32_t m = max(max(pm[0][jc], pm[1][jc]), max(pm[2][jc], pm[3][jc]));
      const E8 e(__uint_as_float(m));
      eights[jc] = e;
      if (first && c0 + jc < a.cols) {
        a.scale[c0 + jc] = e.scale(1.f);
        if (SUM) E::store1((S*)a.sum + c0 + jc, (ps[0][jc] + ps[1][jc]) + (ps[2][jc] + ps[3][jc]));
      }
    }
    __syncthreads();
  }
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) E::expand(raw[i], v[i]);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const E8 e = eights[8 * tc + k];
    uint32_t n[4];
    float rest = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) n[i] = e.fast(v[i][k], rest);
    if (!e.sure(rest)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) n[i] = (uint32_t)e.exactly(v[i][k]);
    }
    tile[(8 * tc + k) * LD + tr] = low_bytes(n[0], n[1], n[2], n[3]);
  }
  __syncthreads();
  const int piece = threadIdx.x & 7;  // 16 bytes of a column each
  const int64_t r = r0 + 16 * piece;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int col = 32 * i + (threadIdx.x >> 3);
    if (c0 + col >= a.cols || r >= a.rows) continue;
    int8_t* out = a.q + (c0 + col) * a.ldq;
    const uint32_t* src = tile + col * LD + 4 * piece;
    const u32x4b_t w = {src[0], src[1], src[2], src[3]};
    if (r + 16 <= a.rows) {
      *(PRM_GLOBAL u32x4b_t*)(out + r) = w;
    } else {
      store_q8(out, r, a.rows, u32x2b_t{w[0], w[1]});
      if (r + 8 < a.rows) store_q8(out, r + 8, a.rows, u32x2b_t{w[2], w[3]});
    }
  }
}

// ---------------------------------------------------------------------------
// several quantisers in one launch: what a layer's pass needs of its operands at once.
// The launches of small matrices, not their bytes, are what such a pass waits for.
// ---------------------------------------------------------------------------
// Rows of at most 8 NCH 256 elements (NCH 0: any), a block a row, or a wave where they are
// short; blocks take rows in turn, the next one on its way while one is rounded.
template <class E, int NCH>
__device__ __forceinline__ void quant_rows(const QuantArgs& a, int64_t block, int64_t blocks, uint32_t* red) {
  using S = typename E::S;
  constexpr int N = NCH ? NCH : 1;
  const bool wide = a.cols > 512;
  const int width = wide ? 256 : 64, t = wide ? threadIdx.x : threadIdx.x & 63;
  const int64_t cols = a.cols, step = wide ? blocks : 4 * blocks;
  typename E::Raw next[N];
  auto fetch = [&](int64_t row) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int64_t c = 8 * ((int64_t)i * width + t);
      if (c < cols) next[i] = load_row8<E>((const S*)a.x + row * a.ldx, c, cols);
    }
  };
  int64_t row = wide ? block : 4 * block + (threadIdx.x >> 6);
  if (NCH && row < a.rows) fetch(row);
  int flip = 0;
  for (; row < a.rows; row += step) {
    const S* x = (const S*)a.x + row * a.ldx;
    typename E::Raw held[N];
    TopRaw<E> top;
    if constexpr (NCH) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) held[i] = next[i];
      if (row + step < a.rows) fetch(row + step);
#pragma unroll
      for (int i = 0; i < NCH; ++i)
        if (8 * ((int64_t)i * width + t) < cols) top.add(held[i]);
    } else {
      for (int64_t c = 8 * t; c < cols; c += 8 * width) top.add(load_row8<E>(x, c, cols));
    }
    uint32_t m = wave_max(top.bits());
    if (wide) {
      // two sets of slots in turn: a wave writes the next row's behind one barrier only
      if ((threadIdx.x & 63) == 0) red[flip + (threadIdx.x >> 6)] = m;
      __syncthreads();
      m = max(max(red[flip], red[flip + 1]), max(red[flip + 2], red[flip + 3]));
      flip ^= 4;
    }
    const EightOf<E> e(__uint_as_float(m));
    if (t == 0) a.scale[row] = e.scale(1.f);
    auto out = [&](int64_t c, const typename E::Raw& raw) __attribute__((always_inline)) {
      float v[8];
      E::expand(raw, v);
      store_q8(a.q + row * a.ldq, c, cols, eight8(e, v));
    };
    if constexpr (NCH) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int64_t c = 8 * ((int64_t)i * width + t);
        if (c < cols) out(c, held[i]);
      }
    } else {
      for (int64_t c = 8 * t; c < cols; c += 8 * width) out(c, load_row8<E>(x, c, cols));
    }
  }
}

template <class E, int NCH>
__global__ __launch_bounds__(256) void quant_first_kernel(QuantJobs jobs) {
  __shared__ union {
    uint32_t red[8];
    ColStatsShared stats;
  } sh;
  int j = 0, b = blockIdx.x;
  while (j + 1 < jobs.n && b >= jobs.blocks[j]) b -= jobs.blocks[j++];
  const QuantArgs& a = jobs.a[j];
  if (!jobs.columns[j]) {
    quant_rows<E, NCH>(a, b, jobs.blocks[j], sh.red);
  } else {
    const int gx = (int)((a.cols + 255) / 256);
    if (a.sum) col_stats<E, true>(a, b % gx, b / gx, sh.stats);
    else col_stats<E, false>(a, b % gx, b / gx, sh.stats);
  }
}

template <class E, bool OWN>
__global__ __launch_bounds__(256) void quant_columns_kernel(QuantJobs jobs) {
  __shared__ ColQuantShared<E> sh;
  int j = 0, b = blockIdx.x;
  while (j + 1 < jobs.n && b >= jobs.blocks[j]) b -= jobs.blocks[j++];
  const QuantArgs& a = jobs.a[j];
  const int gx = (int)((a.cols + 63) / 64);
  if (a.sum) col_quant<E, true, OWN>(a, b % gx, b / gx, sh);
  else col_quant<E, false, OWN>(a, b % gx, b / gx, sh);
}

int64_t column_tiles(const QuantArgs& a) { return (a.cols + 63) / 64 * ((a.rows + 127) / 128); }

// Blocks that take rows: eight a CU, as many as it holds.
constexpr int64_t kRowBlocks = 2048;

template <class E>
hipError_t launch_jobs(const QuantJobs& jobs, hipStream_t s) {
  QuantJobs first = jobs, second = {};
  int64_t blocks = 0, pieces = 0, rows = 0;
  const auto groups = [](const QuantArgs& a) { return a.cols > 512 ? a.rows : (a.rows + 3) / 4; };
  for (int j = 0; j < jobs.n; ++j)
    if (!jobs.columns[j]) rows += groups(jobs.a[j]);
  const int64_t per_block = (rows + kRowBlocks - 1) / kRowBlocks;
  for (int j = 0; j < jobs.n; ++j) {
    const QuantArgs& a = jobs.a[j];
    int64_t n;
    if (jobs.columns[j]) {
      n = (a.cols + 255) / 256 * a.nrb;  // none, where the tiles do it themselves
      const int k = second.n++;
      second.a[k] = a;
      second.blocks[k] = (int32_t)column_tiles(a);
    } else {
      n = (groups(a) + per_block - 1) / per_block;
      const int64_t p = (a.cols + 7) / 8, per = a.cols > 512 ? (p + 255) / 256 : 1;
      pieces = per > pieces ? per : pieces;
    }
    first.blocks[j] = (int32_t)n;
    blocks += n;
  }
  if (blocks > 0) {  // rows, or statistics
    const unsigned g = (unsigned)blocks;
    if (pieces <= 1) quant_first_kernel<E, 1><<<g, 256, 0, s>>>(first);
    else if (pieces <= 2) quant_first_kernel<E, 2><<<g, 256, 0, s>>>(first);
    else if (pieces <= 4) quant_first_kernel<E, 4><<<g, 256, 0, s>>>(first);
    else if (pieces <= 8) quant_first_kernel<E, 8><<<g, 256, 0, s>>>(first);
    else quant_first_kernel<E, 0><<<g, 256, 0, s>>>(first);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (second.n) {
    int64_t g = 0;
    bool own = false;
    for (int j = 0; j < second.n; ++j) {
      g += second.blocks[j];
      own |= second.a[j].nrb == 0;
    }
    if (own) quant_columns_kernel<E, true><<<(unsigned)g, 256, 0, s>>>(second);
    else quant_columns_kernel<E, false><<<(unsigned)g, 256, 0, s>>>(second);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rms_norm(OpType t, const NormArgs& a, hipStream_t s) {
  return t == OP_F32 ? launch_norm<TF32>(a, s) : t == OP_BF16 ? launch_norm<TBF16>(a, s) : launch_norm<TF16>(a, s);
}

hipError_t launch_quantize_rows(OpType t, const QuantArgs& q, hipStream_t s) {
  NormArgs a = {};
  a.x = q.x;
  a.q = q.q;
  a.scale = q.scale;
  a.rows = q.rows;
  a.cols = q.cols;
  a.ldx = q.ldx;
  a.ldq = q.ldq;
  return t == OP_F32    ? launch_rows<TF32, QUANT, false>(a, s)
         : t == OP_BF16 ? launch_rows<TBF16, QUANT, false>(a, s)
                        : launch_rows<TF16, QUANT, false>(a, s);
}

// No row blocks where a matrix is laid out alone and has few rows: each tile of 128 rows then
// takes the statistics itself, reading all rows, and a launch is saved (512 x 8192 bf16: 8.8
// us, before 11.4; among others, whose first launch is there anyway, it would cost time).
// Otherwise, row blocks of the columns' statistics: of at least 64 rows, at most 64, and no more than
// fill the card (kStatBlocks of 256 columns), as each tile of the second kernel reads the
// statistics of all.
constexpr int64_t kOwnRows = 512;
constexpr int64_t kStatBlocks = 1024;  // 8192 x 16384 bf16: 135 us; 512 135, 2048 139, no bound 148
void quantize_cols_blocks(int64_t rows, int64_t cols, bool alone, int32_t* nrb, int32_t* rows_per_block) {
  if (alone && rows <= kOwnRows) {
    *nrb = *rows_per_block = 0;
    return;
  }
  const int64_t most = kStatBlocks / ((cols + 255) / 256), n = most < 1 ? 1 : most > 64 ? 64 : most;
  int64_t per = (rows + n - 1) / n;
  per = per < 64 ? 64 : per;
  *rows_per_block = (int32_t)per;
  *nrb = (int32_t)((rows + per - 1) / per);
}

int64_t quantize_tiles(const QuantJobs& jobs) {
  int64_t n = 0;
  for (int j = 0; j < jobs.n; ++j)
    if (jobs.columns[j]) n += column_tiles(jobs.a[j]);
  return n;
}

hipError_t launch_quantize(OpType t, const QuantJobs& jobs, hipStream_t s) {
  return t == OP_F32 ? launch_jobs<TF32>(jobs, s) : t == OP_BF16 ? launch_jobs<TBF16>(jobs, s) : launch_jobs<TF16>(jobs, s);
}

// Blocks, each of which leaves a row of partial dw: as many as the card holds at once (of
// 256 threads four a CU, two with two pieces of fp32; of 1024 one), so that none waits for
// another to end.  A block of short rows takes four at a time.  8192 x 4096 bf16: 55 us
// with 1024, 62 with 512; fp32 117 and 105; 2048 x 16384 bf16 59 us with 256, 68 with 512.
int32_t rms_norm_grad_parts(OpType t, int64_t rows, int64_t cols) {
  const int64_t most = cols > 4096 ? 256 : cols > 2048 && t == OP_F32 ? 512 : 1024, groups = cols <= 512 ? (rows + 3) / 4 : rows;
  return (int32_t)(groups < most ? (groups < 1 ? 1 : groups) : most);
}

hipError_t launch_rms_norm_grad(OpType t, const NormGradArgs& a, hipStream_t s) {
  return t == OP_F32 ? launch_grad<TF32>(a, s) : t == OP_BF16 ? launch_grad<TBF16>(a, s) : launch_grad<TF16>(a, s);
}

}  // namespace prm
