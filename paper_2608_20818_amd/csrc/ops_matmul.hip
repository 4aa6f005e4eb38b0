// 8-bit product of the linear layer on gfx950:
//
//   out[i][j] = a_scale[i] b_scale[j] sum_k a[i][k] b[j][k]  (+ bias[j])
//
// a (tokens) and b (output channels) both have k along their rows.  The sums are exact
// in 32-bit whole numbers (v_mfma_i32_32x32x32_i8, v_mfma_i32_16x16x64_i8), so neither
// the order of the sum nor how it is split changes a bit of the result; the scales are
// applied in fp32 and the result is rounded once.
#include <cmath>
#include <type_traits>

#include "ops_device.h"

namespace prm {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));

// 16 bytes of a row from k, at any address
__device__ __forceinline__ u32x4_t load16(const int8_t* p) {
  const u32x4b_t x = *(const PRM_GLOBAL u32x4b_t*)p;
  return u32x4_t{x[0], x[1], x[2], x[3]};
}
// The same with zeros behind the row's end: the row's last 16 bytes, moved down.
__device__ __forceinline__ u32x4_t load_k16(const int8_t* row, int64_t k, int64_t klen) {
  if (klen >= 16) {
    const int64_t from = min(k, klen - 16);
    const u32x4_t v = load16(row + from);
    const int sh = (int)min(k - from, (int64_t)16) * 8;
    const uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
    const uint64_t l = sh == 0 ? lo : sh < 64 ? lo >> sh | hi << (64 - sh) : sh < 128 ? hi >> (sh - 64) : 0;
    const uint64_t h = sh < 64 ? hi >> sh : 0;
    return u32x4_t{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
  }
  u32x4_t v = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (k + i < klen) v[i >> 2] |= (uint32_t)(uint8_t)*gptr(row + k + i) << (8 * (i & 3));
  return v;
}

template <class E>
__device__ __forceinline__ void store4(typename E::S* row, int64_t c, int64_t n, const float v[4]) {
  if (c + 4 <= n) {
    E::store4(row + c, v);
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (c + k < n) E::store1(row + c + k, v[k]);
}

// The epilogue of a wave's block of 32 MI x 32 NI sums.  The matrix instruction leaves lane
// L output row 32 i + L % 32 and, of each piece of 32 columns, 8 q + 4 (L / 32) + 0..3.  32
// rows at a time pass through a part of shared memory of the wave's own, from which a lane
// takes 8 columns, the same for every row.  All scales are fetched up front (the first
// part): a load behind a store would wait for the store.
template <class E, int MI, int NI>
struct Epilogue {
  static constexpr int LPR = 4 * NI, RPI = 64 / LPR, IT = 32 / RPI;  // lanes a row, rows a store, stores of 32 rows
  float as[(MI + 1) / 2], bs[8], bias[8];  // as: row 64 h + lane of the block
  int64_t r0, c;
  __device__ __forceinline__ void at_block(int64_t row, int64_t col) {
    const int lane = threadIdx.x & 63;
    r0 = row + lane / LPR;
    c = col + 8 * (lane & (LPR - 1));
  }
  __device__ __forceinline__ void fetch(const ProductArgs& p, int64_t row, int64_t col) {
    const int lane = threadIdx.x & 63;
    at_block(row, col);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t cc = min(c + e, p.n - 1);
      bs[e] = *gptr(p.b_scale + cc);
      bias[e] = p.bias ? E::load1((const typename E::S*)p.bias + cc) : 0.f;
    }
#pragma unroll
    for (int h = 0; h < (MI + 1) / 2; ++h) as[h] = *gptr(p.a_scale + min(row + 64 * h + lane, p.m - 1));
  }
  // 16-byte piece ch of row r: rows written, and read, together hit distinct banks
  __device__ __forceinline__ static int at(int r, int ch) { return 32 * NI * r + 4 * (ch ^ ((NI == 1 ? r >> 1 : r) & (8 * NI - 1))); }
  // SPLIT: the sums themselves, to the split's rows of p.part (ceil(n / 8) times 8 columns)
  template <bool SPLIT = false>
  __device__ __forceinline__ void store(const ProductArgs& p, const i32x16_t (&acc)[MI][NI], int* mine) {
    const int lane = threadIdx.x & 63;
    const bool whole = c + 8 <= p.n;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const i32x4_t v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          *reinterpret_cast<i32x4_t*>(mine + at(lane & 31, 8 * j + 2 * q + (lane >> 5))) = v;
        }
      __builtin_amdgcn_wave_barrier();  // a wave's accesses to shared memory are in order
#pragma unroll
      for (int k = 0; k < IT; ++k) {
        const int rr = RPI * k + lane / LPR;
        const int64_t row = r0 + RPI * (IT * i + k);
        const i32x4_t lo = *reinterpret_cast<const i32x4_t*>(mine + at(rr, 2 * (lane & (LPR - 1))));
        const i32x4_t hi = *reinterpret_cast<const i32x4_t*>(mine + at(rr, 2 * (lane & (LPR - 1)) + 1));
        if constexpr (SPLIT) {
          if (row < p.m && c < p.n) {
            PRM_GLOBAL i32x4_t* dst = (PRM_GLOBAL i32x4_t*)(p.part + ((int64_t)blockIdx.y * p.m + row) * ((p.n + 7) / 8 * 8) + c);
            dst[0] = lo;
            dst[1] = hi;
          }
          continue;
        }
        const float scale = __shfl(as[i / 2], 32 * (i & 1) + rr, 64);
        if (row < p.m) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = (float)(e < 4 ? lo[e & 3] : hi[e & 3]) * scale * bs[e] + bias[e];
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
};

// ---------------------------------------------------------------------------
// tiles: four waves, 64 x 64 outputs each or 32 x 32, operands staged through
// registers into shared memory, any alignment
// ---------------------------------------------------------------------------
template <class E, int BM, int BN, int P>
__global__ __launch_bounds__(256) void tile_kernel(ProductArgs p, int tiles_m) {
  constexpr int BK = 128;            // bytes of k a stage
  constexpr int WM = BM / 2, WN = BN / 2, MI = WM / 32, NI = WN / 32;
  constexpr int LA = BM * 8 / 256, LB = BN * 8 / 256;  // 16-byte pieces a thread loads
  __shared__ __attribute__((aligned(16))) char smem[2][(BM + BN) * BK];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int64_t row0 = (int64_t)(blockIdx.x % tiles_m) * BM, col0 = (int64_t)(blockIdx.x / tiles_m) * BN;
  // piece ch of row r lies at ch ^ (r / 2 % 8): rows read together hit distinct banks
  auto at = [](int r, int ch) __attribute__((always_inline)) { return r * BK + ((ch ^ ((r >> 1) & 7)) << 4); };
  const int ch = tid & 7, r0 = tid >> 3;
  const int8_t *rowa[LA], *rowb[LB];
#pragma unroll
  for (int i = 0; i < LA; ++i) rowa[i] = p.a + min(row0 + r0 + 32 * i, p.m - 1) * p.lda;
#pragma unroll
  for (int i = 0; i < LB; ++i) rowb[i] = p.b + min(col0 + r0 + 32 * i, p.n - 1) * p.ldb;
  // P stages are on their way in registers while one is multiplied
  u32x4_t ra[P][LA], rb[P][LB];
  auto fetch = [&](int s, int64_t k) __attribute__((always_inline)) {
    if (k >= p.k) return;
    if (k + BK <= p.k) {
#pragma unroll
      for (int i = 0; i < LA; ++i) ra[s][i] = load16(rowa[i] + k + 16 * ch);
#pragma unroll
      for (int i = 0; i < LB; ++i) rb[s][i] = load16(rowb[i] + k + 16 * ch);
    } else {
#pragma unroll
      for (int i = 0; i < LA; ++i) ra[s][i] = load_k16(rowa[i], k + 16 * ch, p.k);
#pragma unroll
      for (int i = 0; i < LB; ++i) rb[s][i] = load_k16(rowb[i], k + 16 * ch, p.k);
    }
  };
  i32x16_t acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = i32x16_t{};
#pragma unroll
  for (int s = 0; s < P; ++s) fetch(s, s * BK);
  int buf = 0;
  for (int64_t k0 = 0; k0 < p.k; k0 += P * BK) {
#pragma unroll
    for (int s = 0; s < P; ++s) {
      const int64_t k = k0 + s * BK;
      if (k >= p.k) break;
      char *const sa = smem[buf], *const sb = sa + BM * BK;
#pragma unroll
      for (int i = 0; i < LA; ++i) *reinterpret_cast<u32x4_t*>(sa + at(r0 + 32 * i, ch)) = ra[s][i];
#pragma unroll
      for (int i = 0; i < LB; ++i) *reinterpret_cast<u32x4_t*>(sb + at(r0 + 32 * i, ch)) = rb[s][i];
      fetch(s, k + P * BK);
      __syncthreads();  // the other buffer's readers are past the barrier before this one
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        i32x4_t fa[MI], fb[NI];
#pragma unroll
        for (int i = 0; i < MI; ++i)
          fa[i] = *reinterpret_cast<const i32x4_t*>(sa + at(wm * WM + 32 * i + (lane & 31), 2 * ks + (lane >> 5)));
#pragma unroll
        for (int j = 0; j < NI; ++j)
          fb[j] = *reinterpret_cast<const i32x4_t*>(sb + at(wn * WN + 32 * j + (lane & 31), 2 * ks + (lane >> 5)));
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
      }
      buf ^= 1;
    }
  }
  __syncthreads();
  Epilogue<E, MI, NI> ep;
  ep.fetch(p, row0 + wm * WM, col0 + wn * WN);
  ep.store(p, acc, reinterpret_cast<int*>(smem[0]) + wave * 1024 * NI);
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
// a pointer that is the same for the whole wave, in scalar registers
__device__ __forceinline__ const char* scalar(const char* p) {
  const uint64_t u = (uint64_t)(uintptr_t)p;
  return (const char*)(uintptr_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32) |
                                  (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u));
}

namespace big {
constexpr int BM = 256, BK = 128, NWAVES = 4, NTHREADS = 256;
constexpr int W = 128, MI = 4;                        // a wave's block, in pieces of 32
constexpr int OPERAND = BM * BK, STAGE = 2 * OPERAND;  // 32 KB, 64 KB
constexpr int DMA = BM / 8 / NWAVES, NDMA = 2 * DMA;  // 1 KB wave loads of an operand, and of a stage
// 16-byte piece ch of row r lies at ch ^ (r / 2 % 8): 16 rows read at one piece hit 16
// distinct 16-byte groups of banks
__device__ __forceinline__ int at(int r, int ch) { return r * BK + ((ch ^ ((r >> 1) & 7)) << 4); }
typedef __attribute__((address_space(3))) void* lds_ptr;
// Work groups go to the 8 XCDs in turn: each gets a run of tiles of its own, in columns
// of 8 tile rows, so that the 32 tiles an XCD works on share 8 + 4 panels in its L2.
__device__ __forceinline__ void tile_of(int tiles_m, int tiles_n, int& tm, int& tn) {
  const int total = tiles_m * tiles_n, per = total >> 3, rest = total & 7;
  const int x = blockIdx.x & 7, t = x * per + min(x, rest) + (blockIdx.x >> 3);
  const int group = t / (8 * tiles_n), first = 8 * group, high = min(8, tiles_m - first);
  const int in = t - 8 * group * tiles_n;
  tm = first + in % high;
  tn = in / high;
}
}  // namespace big

template <class E>
__global__ __launch_bounds__(big::NTHREADS, 1) void big_kernel(ProductArgs p, int tiles_m, int tiles_n) {
  using namespace big;
  __shared__ __attribute__((aligned(16))) char smem[2 * STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  int tm, tn;
  tile_of(tiles_m, tiles_n, tm, tn);
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
    const char* base = scalar((isb ? baseB : baseA) + k);
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
  Epilogue<E, MI, MI> ep;
  ep.fetch(p, row0 + wm * W, col0 + wn * W);
  stage(cur, 0, no);
  mul(1, MI - 1);
  __syncthreads();
  ep.store(p, acc, reinterpret_cast<int*>(smem) + wave * 1024 * MI);
}

// ---------------------------------------------------------------------------
// piped tiles: BM x BN outputs, four waves of half of each, k in stages of BK bytes
// through NBUF shared-memory buffers.  All operands of a stage lie in registers: while
// k-step s is multiplied, its registers are free to take the next stage's.  In the middle
// of stage t, its operands all read, one barrier says that stage t + 1 has landed for every
// wave and that the buffer of stage t is free; the loads of stage t + NBUF go there, and
// are waited for NBUF - 1 stages later.
// ---------------------------------------------------------------------------
template <class E, int BM, int BN, int BK, int NBUF, bool SPLIT>
__global__ __launch_bounds__(256) void piped_kernel(ProductArgs p, int tiles_m, int tiles_n) {
  using big::lds_ptr;
  constexpr int STAGE = (BM + BN) * BK, KS = BK / 32, CH = BK / 16;
  constexpr int WM = BM / 2, WN = BN / 2, MI = WM / 32, NI = WN / 32;
  constexpr int RPL = 1024 / BK;                            // rows of one 1 KB wave load
  constexpr int LA = BM / RPL / 4, LB = BN / RPL / 4, LPS = LA + LB;  // loads of a wave a stage
  constexpr int SH = CH == 8 ? 1 : 2;                       // 16 rows read at one piece hit 16 groups of banks
  static_assert((NBUF - 1) * LPS < 64, "the wait counter's range");
  __shared__ __attribute__((aligned(16))) char smem[NBUF * STAGE];
  auto at = [](int r, int ch) __attribute__((always_inline)) { return r * BK + ((ch ^ ((r >> SH) & (CH - 1))) << 4); };
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  int tm, tn;
  big::tile_of(tiles_m, tiles_n, tm, tn);
  const int64_t row0 = (int64_t)tm * BM, col0 = (int64_t)tn * BN;
  const char* const baseA = (const char*)p.a + row0 * p.lda;
  const char* const baseB = (const char*)p.b + col0 * p.ldb;
  const int lastA = (int)min((int64_t)BM, p.m - row0) - 1, lastB = (int)min((int64_t)BN, p.n - col0) - 1;
  uint32_t off[LPS];
#pragma unroll
  for (int q = 0; q < LPS; ++q) {
    const int r = (q < LA ? BM / 4 * wave + RPL * q : BN / 4 * wave + RPL * (q - LA)) + lane / CH;
    const uint32_t piece = (uint32_t)(((lane & (CH - 1)) ^ ((r >> SH) & (CH - 1))) << 4);
    off[q] = (q < LA ? (uint32_t)(min(r, lastA) * p.lda) : (uint32_t)(min(r, lastB) * p.ldb)) + piece;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr)smem;
  auto load1 = [&](int buf, int64_t k, int q) __attribute__((always_inline)) {
    const char* base = scalar((q < LA ? baseA : baseB) + k);
    const uint32_t lds = lds0 + buf + (q < LA ? (LA * wave + q) * 1024 : BM * BK + (LB * wave + q - LA) * 1024);
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // the M0 clobber
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off[q]), "s"(base), "s"(lds) : "m0");
#pragma clang diagnostic pop
  };
  auto load = [&](int buf, int64_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < LPS; ++q) load1(buf, k, q);
  };
  i32x16_t acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = i32x16_t{};
  int pa[KS], pb[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    pa[ks] = at(wm * WM + (lane & 31), 2 * ks + (lane >> 5));
    pb[ks] = BM * BK + at(wn * WN + (lane & 31), 2 * ks + (lane >> 5));
  }
  i32x4_t fa[KS][MI], fb[KS][NI];
  auto read = [&](int buf, int ks) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MI; ++i) fa[ks][i] = *reinterpret_cast<const i32x4_t*>(smem + (buf + pa[ks]) + 32 * BK * i);
#pragma unroll
    for (int j = 0; j < NI; ++j) fb[ks][j] = *reinterpret_cast<const i32x4_t*>(smem + (buf + pb[ks]) + 32 * BK * j);
  };
  auto mul = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[ks][j], fa[ks][i], acc[i][j], 0, 0, 0);
  };
  // This block's stages: pieces first .. last - 1 of BK bytes and, where k ends within a
  // piece, the first split takes that end (`odd`) as its stage 0, before its pieces.
  const int full = (int)(p.k / BK), splits = SPLIT ? (int)gridDim.y : 1, split = SPLIT ? (int)blockIdx.y : 0;
  const int first = (int)((int64_t)full * split / splits), last = (int)((int64_t)full * (split + 1) / splits);
  const int odd = split == 0 && p.k % BK != 0;
  const int n = last - first + odd;
  if (odd) {
    u32x4_t r[LPS];
    const int ch = tid & (CH - 1), r0 = tid / CH;
#pragma unroll
    for (int q = 0; q < LPS; ++q)
      r[q] = q < LA ? load_k16((const int8_t*)baseA + min(r0 + 4 * RPL * q, lastA) * p.lda, (int64_t)full * BK + 16 * ch, p.k)
                    : load_k16((const int8_t*)baseB + min(r0 + 4 * RPL * (q - LA), lastB) * p.ldb, (int64_t)full * BK + 16 * ch, p.k);
#pragma unroll
    for (int q = 0; q < LPS; ++q)
      *reinterpret_cast<u32x4_t*>(smem + (q < LA ? at(r0 + 4 * RPL * q, ch) : BM * BK + at(r0 + 4 * RPL * (q - LA), ch))) = r[q];
  }
#pragma unroll
  for (int t = 0; t < NBUF; ++t)
    if (t >= odd && t < n) load(t * STAGE, (int64_t)(first + t - odd) * BK);
  if (n >= NBUF) asm volatile("s_waitcnt vmcnt(%0)" ::"i"((NBUF - 1) * LPS) : "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) read(0, ks);
  int cur = 0;
  auto half = [&](int from) __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < KS / 2; ++ks) mul(from + ks);
  };
  for (int t = 0; t + 1 < n; ++t) {
    half(0);
    // of the NBUF stages loaded, t + 1 may be the first to be waited for; where no full
    // set is behind it, all are
    if (t + NBUF <= n) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"((NBUF - 2) * LPS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int nxt = cur == (NBUF - 1) * STAGE ? 0 : cur + STAGE;
    const bool more = t + NBUF < n;
    const int64_t k = (int64_t)(first + t + NBUF - odd) * BK;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < KS / 2; ++ks) read(nxt, ks);
#pragma unroll
    for (int ks = KS / 2; ks < KS; ++ks) {
      if (more) {
#pragma unroll
        for (int q = 0; q < LPS; ++q)
          if (q * (KS / 2) / LPS == ks - KS / 2) load1(cur, k, q);
      }
      mul(ks);
      __builtin_amdgcn_sched_barrier(0);
      read(nxt, ks);
    }
    cur = nxt;
  }
  Epilogue<E, MI, NI> ep;
  if constexpr (SPLIT) ep.at_block(row0 + wm * WM, col0 + wn * WN);
  else ep.fetch(p, row0 + wm * WM, col0 + wn * WN);
  half(0);
  half(KS / 2);
  __syncthreads();
  ep.template store<SPLIT>(p, acc, reinterpret_cast<int*>(smem) + wave * 1024 * NI);
}

// ---------------------------------------------------------------------------
// few tokens (at most 16): 16 channels a block, read once and straight into registers;
// the block's waves split k and join their sums in shared memory.  One token through 20480
// x 5120: 20 us (5.2 TB/s; bound by reading the weight), 8 tokens 26.  Every block reads the tokens
// from its L2, which 16 of them feel (31 us; two or four times the channels a block were
// no faster).
// ---------------------------------------------------------------------------
template <class E, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(ProductArgs p) {
  __shared__ __attribute__((aligned(16))) i32x4_t part[WAVES][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int kg = 16 * (lane >> 4);
  const int8_t* a = p.a + min((int64_t)(lane & 15), p.m - 1) * p.lda;
  const int8_t* b = p.b + min(n0 + (lane & 15), p.n - 1) * p.ldb;
  i32x4_t acc = {};
  // wave w takes the pieces of 256 bytes of k w, w + WAVES, ...
  for (int64_t k = 256 * wave; k < p.k; k += 256 * WAVES) {
    u32x4_t fa[4], fb[4];
    if (k + 256 <= p.k) {
#pragma unroll
      for (int u = 0; u < 4; ++u) fb[u] = load16(b + k + 64 * u + kg);
#pragma unroll
      for (int u = 0; u < 4; ++u) fa[u] = load16(a + k + 64 * u + kg);
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) fb[u] = load_k16(b, k + 64 * u + kg, p.k);
#pragma unroll
      for (int u = 0; u < 4; ++u) fa[u] = load_k16(a, k + 64 * u + kg, p.k);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, fb[u]), __builtin_bit_cast(i32x4_t, fa[u]), acc, 0, 0, 0);
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave != 0) return;
  // lane L: token L % 16, channels 4 (L / 16) + 0..3
#pragma unroll
  for (int w = 1; w < WAVES; ++w) acc += part[w][lane];
  const int64_t r = lane & 15, c = n0 + 4 * (lane >> 4);
  if (r >= p.m) return;
  const float as = *gptr(p.a_scale + r);
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t cc = min(c + e, p.n - 1);
    v[e] = (float)acc[e] * as * *gptr(p.b_scale + cc);
    if (p.bias) v[e] += E::load1((const typename E::S*)p.bias + cc);
  }
  store4<E>((typename E::S*)p.out + r * p.ldo, c, p.n, v);
}

// The sums of the splits, joined (in 64 bits: a sum longer than one piece may pass 2^31) and
// scaled: 8 columns a thread.
template <class E>
__global__ __launch_bounds__(256) void join_kernel(ProductArgs p, int splits) {
  const int64_t piece = (int64_t)blockIdx.x * 256 + threadIdx.x, per = (p.n + 7) / 8;
  const int64_t row = piece / per, c = 8 * (piece - row * per);
  if (row >= p.m) return;
  const int64_t ldp = 8 * per;
  int64_t sum[8] = {};
  for (int s = 0; s < splits; ++s) {
    const PRM_GLOBAL i32x4_t* src = (const PRM_GLOBAL i32x4_t*)(p.part + ((int64_t)s * p.m + row) * ldp + c);
    const i32x4_t lo = src[0], hi = src[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sum[e] += lo[e];
      sum[4 + e] += hi[e];
    }
  }
  const float as = *gptr(p.a_scale + row);
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int64_t cc = min(c + e, p.n - 1);
    v[e] = (float)sum[e] * as * *gptr(p.b_scale + cc);
    if (p.bias) v[e] += E::load1((const typename E::S*)p.bias + cc);
  }
  store_row8<E>((typename E::S*)p.out + row * p.ldo, c, p.n, E::pack(v));
}

// Operands whose rows start on any byte, laid out for the direct loads: rows of kp (a
// multiple of 128) bytes, zeros behind the end.  16 bytes a thread.
__global__ __launch_bounds__(256) void pack_kernel(PackArgs g) {
  int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int which = i >= g.rows[0] * (g.kp / 16);
  if (which) i -= g.rows[0] * (g.kp / 16);
  const int64_t per = g.kp / 16, row = i / per, k = 16 * (i - row * per);
  if (row >= g.rows[which]) return;
  const int8_t* src = g.src[which] + row * g.ld[which];
  u32x4_t v = {0u, 0u, 0u, 0u};
  if (k + 16 <= g.k) v = load16(src + k);
  else if (k < g.k) v = load_k16(src, k, g.k);
  *(PRM_GLOBAL u32x4_t*)(g.dst[which] + row * g.kp + k) = v;
}

template <class E, int BM>
void launch_piped(const ProductArgs& p, int splits, hipStream_t s) {
  const int tm = (int)((p.m + BM - 1) / BM), tn = (int)((p.n + BM - 1) / BM);
  if (splits == 1) {
    piped_kernel<E, BM, BM, 128, 4, false><<<(unsigned)(tm * tn), 256, 0, s>>>(p, tm, tn);
    return;
  }
  piped_kernel<E, BM, BM, 128, 4, true><<<dim3((unsigned)(tm * tn), (unsigned)splits), 256, 0, s>>>(p, tm, tn);
  join_kernel<E><<<(unsigned)((p.m * ((p.n + 7) / 8) + 255) / 256), 256, 0, s>>>(p, splits);
}

int64_t tile_size(ProductKind kind) { return kind == PRODUCT_256 ? 256 : kind == PRODUCT_ANY64 || kind == PRODUCT_64 ? 64 : 128; }

template <class E>
hipError_t launch(ProductArgs p, const ProductPlan& plan, hipStream_t s) {
  if (plan.pack) {
    PackArgs g = {};
    g.k = p.k;
    g.kp = (p.k + 127) / 128 * 128;
    int8_t* at = (int8_t*)p.part;
    const auto lay = [&](const int8_t*& operand, int64_t& ld, int64_t rows, int which) {
      g.src[which] = operand;
      g.ld[which] = ld;
      g.dst[which] = at;
      g.rows[which] = rows;
      operand = at;
      ld = g.kp;
      at += rows * g.kp;
    };
    if (plan.pack & 1) lay(p.a, p.lda, p.m, 0);
    if (plan.pack & 2) lay(p.b, p.ldb, p.n, 1);
    const int64_t pieces = (g.rows[0] + g.rows[1]) * (g.kp / 16);
    pack_kernel<<<(unsigned)((pieces + 255) / 256), 256, 0, s>>>(g);
    if (plan.pack == 3) p.k = g.kp;  // zeros behind both ends: no end within a piece
    p.part = (int32_t*)at;
  }
  const int64_t b = tile_size(plan.kind);
  const int64_t tm = (p.m + b - 1) / b, tn = (p.n + b - 1) / b;
  const unsigned tiles = (unsigned)(tm * tn);
  switch (plan.kind) {
    case PRODUCT_FEW: few_kernel<E, 8><<<(unsigned)((p.n + 15) / 16), 512, 0, s>>>(p); break;
    case PRODUCT_ANY64: tile_kernel<E, 64, 64, 4><<<tiles, 256, 0, s>>>(p, (int)tm); break;
    case PRODUCT_ANY128: tile_kernel<E, 128, 128, 2><<<tiles, 256, 0, s>>>(p, (int)tm); break;
    case PRODUCT_64: launch_piped<E, 64>(p, plan.splits, s); break;
    case PRODUCT_128: launch_piped<E, 128>(p, plan.splits, s); break;
    case PRODUCT_128_PAIRED: piped_kernel<E, 128, 128, 128, 2, false><<<tiles, 256, 0, s>>>(p, (int)tm, (int)tn); break;
    default: big_kernel<E><<<tiles, 256, 0, s>>>(p, (int)tm, (int)tn);
  }
  return hipGetLastError();
}

}  // namespace

// the direct loads' 16-byte granule, and 32-bit offsets within a tile
static bool direct(const int8_t* p, int64_t ld) { return ld % 16 == 0 && (uintptr_t)p % 16 == 0 && ld < (1 << 23); }

bool product_takes(const ProductArgs& p, const ProductPlan& plan) {
  const ProductKind kind = plan.kind;
  const int64_t pieces = p.k / 128;
  if (plan.pack && (kind < PRODUCT_64 || plan.pack > 3)) return false;
  if (plan.splits == 1 ? p.k > kMaxPieceK : plan.splits > 1 && ((pieces + plan.splits - 1) / plan.splits + 1) * 128 > kMaxPieceK)
    return false;  // a piece's sum has to fit 32 bits
  if (plan.splits != 1 && ((kind != PRODUCT_64 && kind != PRODUCT_128) || plan.splits < 1 || plan.splits > pieces || plan.splits > 64))
    return false;
  if (kind == PRODUCT_FEW) return p.m <= 16;
  // the launches' grids: tiles, the sums joined and the operands laid out anew
  const int64_t b = tile_size(kind), packed = (plan.pack & 1 ? p.m : 0) + (plan.pack & 2 ? p.n : 0);
  if (((p.m + b - 1) / b) * ((p.n + b - 1) / b) >= kMaxTiles) return false;
  if (plan.splits > 1 && (p.m * ((p.n + 7) / 8) + 255) / 256 >= kMaxTiles) return false;
  if ((packed * ((p.k + 127) / 128 * 8) + 255) / 256 >= kMaxTiles) return false;
  if (kind == PRODUCT_ANY64 || kind == PRODUCT_ANY128) return true;
  // operands that are laid out anew, or that the direct loads take as they are
  return ((plan.pack & 1) || direct(p.a, p.lda)) && ((plan.pack & 2) || direct(p.b, p.ldb));
}

uint64_t product_workspace(const ProductArgs& p, const ProductPlan& plan) {
  const uint64_t kp = (uint64_t)((p.k + 127) / 128 * 128);
  return (plan.pack & 1 ? (uint64_t)p.m * kp : 0) + (plan.pack & 2 ? (uint64_t)p.n * kp : 0) +
         (plan.splits > 1 ? (uint64_t)plan.splits * (uint64_t)p.m * (uint64_t)((p.n + 7) / 8 * 8) * 4 : 0);
}

// The least of the kernels' estimated times, in microseconds: rounds of tiles over the 256
// CUs, stages of 128 bytes of k in a round, and what a round and a call cost beside them.
// A stage gets dearer as the card fills (shared L2, and for the large tile the clock
// under load).  Measured / estimated, bf16 out:
//                          64          128        128 paired   256
//    512 x 4096 x 4096    16 / 19      20 / 21      28 / 45     45 / 47
//   1024 x 4096 x 4096    29 / 38      24 / 24      31 / 45     47 / 49
//   4096 x 4096 x  128    22 / 16      20 / 19      14 / 14     16 / 16
//    256 x 20480 x 5120   62 / 58      62 / 57      57 / 54     77 / 60
//   4096 x 4096 x 4096   136 / 145    100 / 93      84 / 86     65 / 64
//   8192 x 20480 x 5120 1459 / 1763  1120 / 1121   998 / 1004  736 / 715
// Splitting k costs a second launch and the sums' way through memory at about 2 TB/s:
// 64 x 4096 x 16384 takes 37.7 us in one piece (64), 21.6 in 4; 1024 x 1024 x 65536
// 147 (64) and 99 (128 in 4); 64 x 4096 x 4096 9.4, and 10.7 in 2.
// Rows that start anywhere are read as they are (ANY64, ANY128), or laid out anew first (a
// launch, and both ways through memory at about 4 TB/s): 4096 x 4096 x 4097 takes 244 us
// on ANY64, 177 on ANY128, and 81 laid out for 256; 64 x 6144 x 2047 12 us on ANY64, 17 laid
// out.  Few tokens' kernel reads any rows at one speed.
ProductPlan product_plan(const ProductArgs& p, bool workspace) {
  if (p.m <= 8 && p.k <= kMaxPieceK) return {PRODUCT_FEW, 1, 0};
  const int pack = (direct(p.a, p.lda) ? 0 : 1) | (direct(p.b, p.ldb) ? 0 : 2);
  if (pack && p.m <= 16 && p.k <= kMaxPieceK) return {PRODUCT_FEW, 1, 0};
  const auto tiles = [&](int64_t b) { return (double)((p.m + b - 1) / b) * (double)((p.n + b - 1) / b); };
  const double stages = (double)((p.k + 127) / 128);
  const auto rounds = [](double t, double at_once) { return std::ceil(t / at_once); };
  const auto fill = [](double t) { return t < 256 ? t / 256 : 1.0; };
  double best = 1e30;
  ProductPlan plan = {PRODUCT_64, 64, pack};
  const auto take = [&](ProductKind kind, int splits, int packed, double t) {
    const ProductPlan q = {kind, splits, packed};
    if (t < best && (workspace || !product_workspace(p, q)) && product_takes(p, q)) {
      best = t;
      plan = q;
    }
  };
  if (pack) {
    take(PRODUCT_ANY64, 1, 0, 3.5 + rounds(tiles(64), 256) * stages * (tiles(64) <= 256 ? 0.65 : 0.43));
    take(PRODUCT_ANY128, 1, 0, 4.5 + rounds(tiles(128), 256) * (stages * 1.1 + 2));
  }
  const double laid = pack ? 3.5 + ((pack & 1 ? (double)p.m : 0) + (pack & 2 ? (double)p.n : 0)) * stages * 128 * 2 / 4e6 : 0;
  take(PRODUCT_256, 1, pack, laid + 14 + rounds(tiles(256), 256) * (stages * (0.95 + 0.6 * fill(tiles(256))) + 9) - 9);
  take(PRODUCT_128_PAIRED, 1, pack, laid + 4 + rounds(tiles(128), 512) * (stages * 1.15 + 4));
  for (int s = 1; s == 1 || (s <= 16 && stages >= 8 * s); s *= 2) {
    const double n = std::ceil(stages / s);
    const double join = laid + (s == 1 ? 0 : 3.5 + s * (double)p.m * (double)p.n * 4 / 2e6);
    take(PRODUCT_128, s, pack, 4.5 + rounds(s * tiles(128), 256) * (n * (0.45 + 0.15 * fill(s * tiles(128))) + 4) - 4 + join);
    take(PRODUCT_64, s, pack, 3.2 + rounds(s * tiles(64), 256) * (n * (0.2 + 0.06 * fill(s * tiles(64) / 4)) + 0.6) - 0.6 + join);
  }
  return plan;
}

hipError_t launch_int8_matmul(OpType t, const ProductArgs& p, const ProductPlan& plan, hipStream_t s) {
  if (p.m == 0 || p.n == 0) return hipSuccess;
  return t == OP_F32 ? launch<TF32>(p, plan, s) : t == OP_BF16 ? launch<TBF16>(p, plan, s) : launch<TF16>(p, plan, s);
}

}  // namespace prm
