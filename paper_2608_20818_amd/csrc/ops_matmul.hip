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
// large tiles: 256 x 256 outputs, four waves of 128 x 128 (256 sums a lane), k in
// stages of 128 bytes through two shared-memory buffers.  Stage t + 1 flows into one
// by direct global-to-LDS loads while stage t is read from the other; the last row
// blocks of a stage run behind its barrier, while the next one's first operands load.
// Rows start on 16-byte boundaries (the direct loads' granule); k may end anywhere: what
// is over 128 bytes goes first, through registers, with zeros behind the end (the sum's
// order is free).  Rows past the matrix read its last row and are not stored.
// ---------------------------------------------------------------------------
namespace big {
constexpr int BM = 256, BK = 128, NWAVES = 4, NTHREADS = 256;
constexpr int W = 128, MI = 4;                        // a wave's block, in pieces of 32
constexpr int OPERAND = BM * BK, STAGE = 2 * OPERAND;  // 32 KB, 64 KB
constexpr int DMA = BM / 8 / NWAVES, NDMA = 2 * DMA;  // 1 KB wave loads of an operand, and of a stage
// 16-byte piece ch of row r lies at ch ^ (r / 2 % 8): 16 rows read at one piece hit 16
// distinct 16-byte groups of banks
__device__ __forceinline__ int at(int r, int ch) { return r * BK + ((ch ^ ((r >> 1) & 7)) << 4); }
typedef __attribute__((address_space(3))) void* lds_ptr;
}  // namespace big

template <class E>
__global__ __launch_bounds__(big::NTHREADS, 1) void big_kernel(ProductArgs p, int tiles_m, int tiles_n) {
  using namespace big;
  __shared__ __attribute__((aligned(16))) char smem[2 * STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  // Work groups go to the 8 XCDs in turn: each gets a run of tiles of its own, in columns
  // of 8 tile rows, so that the 32 tiles an XCD works on share 8 + 4 panels in its L2.
  int tm, tn;
  {
    const int total = tiles_m * tiles_n, per = total >> 3, rest = total & 7;
    const int x = blockIdx.x & 7, i = blockIdx.x >> 3;
    const int t = x * per + min(x, rest) + i;
    const int group = t / (8 * tiles_n), first = 8 * group, high = min(8, tiles_m - first);
    const int in = t - 8 * group * tiles_n;
    tm = first + in % high;
    tn = in / high;
  }
  const int64_t row0 = (int64_t)tm * BM, col0 = (int64_t)tn * BM;

  // Wave load q of an operand covers tile rows 64 wave + 8 q + lane / 8, and lane fills
  // the piece at place lane % 8.  A load is a scalar base (operand, tile, k) plus a
  // 32-bit offset of the lane; rows are clamped to the matrix.
  const char* const baseA = (const char*)p.a + row0 * p.lda;
  const char* const baseB = (const char*)p.b + col0 * p.ldb;
  const int lastA = (int)min((int64_t)BM, p.m - row0) - 1, lastB = (int)min((int64_t)BM, p.n - col0) - 1;
  uint32_t offA[DMA], offB[DMA];
#pragma unroll
  for (int q = 0; q < DMA; ++q) {
    const int r = 64 * wave + 8 * q + (lane >> 3);
    const uint32_t piece = (uint32_t)(((lane & 7) ^ ((r >> 1) & 7)) << 4);
    offA[q] = (uint32_t)(min(r, lastA) * p.lda) + piece;
    offB[q] = (uint32_t)(min(r, lastB) * p.ldb) + piece;
  }
  // As assembly, because the compiler folds the lane's offset into a 64-bit vector
  // address before adding k.  It does not see these writes to shared memory: every wait
  // for a stage is explicit.  M0 holds the destination; the compiler reserves it and
  // uses it for nothing else in this kernel.  The s_nop is the wait state between its
  // write and the load.
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr)smem;
  auto dma1 = [&](int stage, int64_t k, int q) __attribute__((always_inline)) {
    const bool isb = q >= DMA;
    const int qq = isb ? q - DMA : q;
    const char* base = (isb ? baseB : baseA) + k;
    const uint32_t lds = lds0 + stage + (isb ? OPERAND : 0) + (DMA * wave + qq) * 1024;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // the M0 clobber
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(isb ? offB[qq] : offA[qq]), "s"(base), "s"(lds) : "m0");
#pragma clang diagnostic pop
  };
  auto landed = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };

  i32x16_t acc[MI][MI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < MI; ++j) acc[i][j] = i32x16_t{};
  const int arow = wm * W + (lane & 31), brow = wn * W + (lane & 31), khalf = lane >> 5;
  // set 1 of the operands outlives a stage: its last row block is multiplied behind the
  // barrier (zeros before the first stage)
  i32x4_t fa[2][MI], fb[2][MI];
#pragma unroll
  for (int i = 0; i < MI; ++i) fa[1][i] = fb[1][i] = i32x4_t{};
  // operands swapped: a lane's sums are four consecutive outputs of one row
  auto mul = [&](int set, int i) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < MI; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[set][j], fa[set][i], acc[i][j], 0, 0, 0);
  };
  // where the lane's operands of k-step ks lie, but for the buffer and 32 rows times i
  int pa[4], pb[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    pa[ks] = at(arow, 2 * ks + khalf);
    pb[ks] = OPERAND + at(brow, 2 * ks + khalf);
  }
  // one stage from the buffer at `cur` while the one at `knext` flows into the other (MORE)
  auto stage = [&](int cur, int64_t knext, auto morec) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(morec)::value;
    const int nxt = cur ^ STAGE;
    auto read = [&](int set, int i, int ks) __attribute__((always_inline)) {
      fa[set][i] = *reinterpret_cast<const i32x4_t*>(smem + (cur + pa[ks]) + 32 * BK * i);
      fb[set][i] = *reinterpret_cast<const i32x4_t*>(smem + (cur + pb[ks]) + 32 * BK * i);
    };
    // a quarter of the loads at once, the rest between the products of the first two k-steps
    constexpr int D0 = NDMA / 4, REST = NDMA - D0, SLOTS = 2 * MI;
    if (MORE) {
#pragma unroll
      for (int q = 0; q < D0; ++q) dma1(nxt, knext, q);
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) read(0, i, 0);
    mul(1, MI - 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
      for (int i = 0; i < (ks == 3 ? MI - 1 : MI); ++i) {
        if (ks < 2 && MORE) {
          const int slot = ks * MI + i;
#pragma unroll
          for (int q = D0 + REST * slot / SLOTS; q < D0 + REST * (slot + 1) / SLOTS; ++q) dma1(nxt, knext, q);
        }
        if (ks < 3) read((ks + 1) & 1, i, ks + 1);
        mul(ks & 1, i);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  constexpr std::integral_constant<bool, true> yes{};
  constexpr std::integral_constant<bool, false> no{};

  const int64_t full = p.k / BK;
  const bool odd = p.k % BK != 0;
  const int64_t n = full + odd;  // stages; with `odd`, stage 0 is the end of k and stage t the piece t - 1
  const int64_t shift = odd ? BK : 0;
  if (odd) {
    u32x4_t r[2][OPERAND / 16 / NTHREADS];
    const int ch = tid & 7, r0 = tid >> 3;
#pragma unroll
    for (int i = 0; i < OPERAND / 16 / NTHREADS; ++i) {
      r[0][i] = load_k16((const int8_t*)baseA + min(r0 + 32 * i, lastA) * p.lda, full * BK + 16 * ch, p.k);
      r[1][i] = load_k16((const int8_t*)baseB + min(r0 + 32 * i, lastB) * p.ldb, full * BK + 16 * ch, p.k);
    }
#pragma unroll
    for (int i = 0; i < OPERAND / 16 / NTHREADS; ++i) {
      *reinterpret_cast<u32x4_t*>(smem + at(r0 + 32 * i, ch)) = r[0][i];
      *reinterpret_cast<u32x4_t*>(smem + OPERAND + at(r0 + 32 * i, ch)) = r[1][i];
    }
  } else {
#pragma unroll
    for (int q = 0; q < NDMA; ++q) dma1(0, 0, q);
    landed();
  }
  __syncthreads();
  int cur = 0;
  for (int64_t k = BK - shift; k < n * BK - shift; k += BK) {
    stage(cur, k, yes);
    landed();
    __syncthreads();  // the next stage has landed, and every wave is done with this one's buffer
    cur ^= STAGE;
  }
  stage(cur, 0, no);
  mul(1, MI - 1);
  __syncthreads();

  // Lane L holds output row 32 i + L % 32 of the wave's block and, of its columns, 32 j +
  // 8 q + 4 (L / 32) + 0..3.  32 rows at a time pass through a part of shared memory of the
  // wave's own (16-byte piece c of row r at c ^ r), from which a lane takes 8 columns, the
  // same for every row: 4 rows of 128 outputs a store.
  int* const mine = reinterpret_cast<int*>(smem + wave * OPERAND);
  const int c8 = lane & 15, r4 = lane >> 4;
  const int64_t c = col0 + wn * W + 8 * c8;
  const bool whole = c + 8 <= p.n;
  float bs[8], bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int64_t cc = min(c + e, p.n - 1);
    bs[e] = *gptr(p.b_scale + cc);
    bias[e] = p.bias ? E::load1((const typename E::S*)p.bias + cc) : 0.f;
  }
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = lane & 31;
#pragma unroll
    for (int j = 0; j < MI; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const i32x4_t v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        *reinterpret_cast<i32x4_t*>(mine + 128 * r + 4 * ((8 * j + 2 * q + khalf) ^ r)) = v;
      }
    __builtin_amdgcn_wave_barrier();  // the wave's own part: its accesses to shared memory are in order
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int rr = 4 * k + r4;
      const int64_t row = row0 + wm * W + 32 * i + rr;
      const i32x4_t lo = *reinterpret_cast<const i32x4_t*>(mine + 128 * rr + 4 * ((2 * c8) ^ rr));
      const i32x4_t hi = *reinterpret_cast<const i32x4_t*>(mine + 128 * rr + 4 * ((2 * c8 + 1) ^ rr));
      if (row < p.m) {
        const float as = *gptr(p.a_scale + row);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)(e < 4 ? lo[e & 3] : hi[e & 3]) * as * bs[e] + bias[e];
        typename E::S* out = (typename E::S*)p.out + row * p.ldo;
        if (whole) {
          E::store8(out + c, E::pack(v));
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + e < p.n) E::store1(out + c + e, v[e]);
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
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
hipError_t launch(const ProductArgs& p, ProductKind kind, hipStream_t s) {
  const int64_t b = kind == PRODUCT_BIG ? 256 : kind == PRODUCT_MID ? 128 : 64;
  const int64_t tm = (p.m + b - 1) / b, tn = (p.n + b - 1) / b;
  const unsigned tiles = (unsigned)(tm * tn), few = (unsigned)((p.n + 15) / 16);
  switch (kind) {
    case PRODUCT_FEW:
      if (p.m <= 16) few_kernel<E, 1, 8><<<few, 512, 0, s>>>(p);
      else if (p.m <= 32) few_kernel<E, 2, 8><<<few, 512, 0, s>>>(p);
      else few_kernel<E, 4, 8><<<few, 512, 0, s>>>(p);
      break;
    case PRODUCT_SMALL: tile_kernel<E, 64, 64><<<tiles, 256, 0, s>>>(p, (int)tm); break;
    case PRODUCT_MID: tile_kernel<E, 128, 128><<<tiles, 256, 0, s>>>(p, (int)tm); break;
    default: big_kernel<E><<<tiles, 256, 0, s>>>(p, (int)tm, (int)tn);
  }
  return hipGetLastError();
}

}  // namespace

bool product_takes(const ProductArgs& p, ProductKind kind) {
  if (kind == PRODUCT_FEW) return p.m <= 64;
  if (kind == PRODUCT_SMALL || kind == PRODUCT_MID) return true;
  // direct loads need their 16-byte granule, and 32-bit offsets within a tile
  return p.lda % 16 == 0 && p.ldb % 16 == 0 && (uintptr_t)p.a % 16 == 0 && (uintptr_t)p.b % 16 == 0 && p.lda < (1 << 23) &&
         p.ldb < (1 << 23);
}

ProductKind product_kind(const ProductArgs& p) {
  if (p.m <= 64) return PRODUCT_FEW;
  const auto tiles = [&](int64_t b) { return ((p.m + b - 1) / b) * ((p.n + b - 1) / b); };
  if (product_takes(p, PRODUCT_BIG) && tiles(256) >= 64) return PRODUCT_BIG;
  return tiles(128) >= 256 ? PRODUCT_MID : PRODUCT_SMALL;
}

hipError_t launch_int8_matmul(OpType t, const ProductArgs& p, ProductKind kind, hipStream_t s) {
  if (p.m == 0 || p.n == 0) return hipSuccess;
  return t == OP_F32 ? launch<TF32>(p, kind, s) : t == OP_BF16 ? launch<TBF16>(p, kind, s) : launch<TF16>(p, kind, s);
}

}  // namespace prm
