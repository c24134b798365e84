// 8-bit products: e4m3 operands with a power-of-two scale for each 128 values along the reduction, their quantiser, and the
// linear layer with its gradients (include/sparse_block.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>
#include <utility>

#include "sparse_attn.h"
#include "sparse_attn_internal.h"
#include "sparse_block.h"
#include "sparse_block_internal.h"

namespace {

using namespace sa_block;

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;

constexpr int kGroup = 128;     // values that share a scale

__host__ __device__ constexpr long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------------------------------
// Quantiser
// ---------------------------------------------------------------------------------------
struct QuantParams {
  const __bf16* x;
  uint8_t *q, *q_scales, *qt, *qt_scales;
  float* col_part;              // [row tiles][cols]: sums of each tile's columns, or NULL
  long long rows, cols, qt_pitch;
};

// eight values times 2^-e as e4m3 bytes
__device__ __forceinline__ int2 e4m3x8(const float (&v)[8], float down) {
  float t[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = e4m3_input(v[e] * down);
  int2 r;
  r.x = e4m3x4(t[0], t[1], t[2], t[3]);
  r.y = e4m3x4(t[4], t[5], t[6], t[7]);
  return r;
}

__device__ __forceinline__ void store_bytes(uint8_t* p, int2 v, int n, bool whole) {
  if (whole) {
    *(int2*)p = v;
    return;
  }
  for (int i = 0; i < n; ++i) p[i] = (uint8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
}

// Eight columns of a row from column c on; those past the end are anything.  Loads stand under no condition that differs from row to
// row, which would make each wait for the one before.  VEC: rows are whole runs of eight on 16 bytes.
template <bool VEC>
__device__ __forceinline__ bf16x8 columns8(const __bf16* row, long long c, long long cols) {
  if constexpr (VEC) return __builtin_nontemporal_load((const bf16x8*)(row + (c < cols ? c : 0)));
  bf16x8 t;
  if (c + 8 <= cols) {
    t = *(const any_bf16x8*)(row + c);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = row[min(c + e, cols - 1)];
  }
  return t;
}

// Rows only: 16 neighbouring lanes hold the 128 columns of a group.  HBM-bound, one pass: 33024 x 3072 60 us, 5.1 TB/s;
// 33024 x 3073 85 us.
template <bool VEC>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const QuantParams p) {
  const long long groups = ceil_div(p.cols, kGroup);
  const long long total = p.rows * groups;
  const int j = threadIdx.x & 15;
  for (long long i = (long long)blockIdx.x * 16 + (threadIdx.x >> 4); i - (threadIdx.x >> 4) < total; i += (long long)gridDim.x * 16) {
    const bool live = i < total;
    const long long row = live ? i / groups : 0, group = live ? i % groups : 0, c = group * kGroup + j * 8;
    const int n = live ? (int)max(0LL, min(8LL, p.cols - c)) : 0;
    float v[8] = {};
    if (n > 0) {
      const bf16x8 t = columns8<VEC>(p.x + row * p.cols, c, p.cols);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = VEC || e < n ? (float)t[e] : 0.f;
    }
    float amax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, finite_abs(v[e]));
    const int ex = e4m3_exponent(group16_max(amax));
    if (n > 0) store_bytes(p.q + row * p.cols + c, e4m3x8(v, power_of_two(-ex)), n, VEC);
    if (live && j == 0) p.q_scales[i] = (uint8_t)(ex + 127);
  }
}

// A tile of 128 x 128, each thread with a patch of 8 x 8: scales along the rows and / or along the columns (BLOCK: one for the
// tile), the transposed bytes through LDS so that both forms are written in whole lines, and the tile's column sums.  HBM-bound:
// 33024 x 3072 into both forms 83 us, 4.9 TB/s; 9001 x 3072 35 us, 3.1 TB/s, as its 1704 tiles are two rounds of the four workgroups
// that the registers, which hold the patch, allow on a CU.
template <bool VEC, bool BLOCK>
__global__ void __launch_bounds__(256) quantize_tile_kernel(const QuantParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[kGroup][kGroup + 16];
  __shared__ float red[4][kGroup];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, cc = threadIdx.x & 15, rr = threadIdx.x >> 4;
  const long long r0 = (long long)blockIdx.y * kGroup, c0 = (long long)blockIdx.x * kGroup;
  const long long row = r0 + rr * 8, col = c0 + cc * 8;
  const int nr = (int)max(0LL, min(8LL, p.rows - row)), nc = (int)max(0LL, min(8LL, p.cols - col));
  bf16x8 held[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) held[i] = columns8<VEC>(p.x + min(row + i, p.rows - 1) * p.cols, col, p.cols);
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = i < nr && e < nc ? (float)held[i][e] : 0.f;
  int tile_e = 0;
  if (BLOCK) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(v[i][e]));
    m = group16_max(m);
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    if (lane == 0) red[wave][0] = m;
    __syncthreads();
    tile_e = e4m3_exponent(fmaxf(fmaxf(red[0][0], red[1][0]), fmaxf(red[2][0], red[3][0])));
    __syncthreads();
    if (threadIdx.x == 0) {
      if (p.q_scales) p.q_scales[blockIdx.y * (long long)gridDim.x + blockIdx.x] = (uint8_t)(tile_e + 127);
      if (p.qt_scales) p.qt_scales[blockIdx.x * (long long)gridDim.y + blockIdx.y] = (uint8_t)(tile_e + 127);
    }
  }
  if (p.q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      int ex = tile_e;
      if (!BLOCK) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(v[i][e]));
        ex = e4m3_exponent(group16_max(m));
        if (i < nr && cc == 0) p.q_scales[(row + i) * gridDim.x + blockIdx.x] = (uint8_t)(ex + 127);
      }
      if (i < nr && nc > 0) store_bytes(p.q + (row + i) * p.cols + col, e4m3x8(v[i], power_of_two(-ex)), nc, VEC);
    }
  }
  // over the rows of the tile: the thread's eight, the wave's other three patches, the other waves
  auto columns = [&](float (&m)[8], auto&& join) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      m[e] = join(m[e], __shfl_xor(m[e], 16));
      m[e] = join(m[e], __shfl_xor(m[e], 32));
    }
    if (lane < 16) {
#pragma unroll
      for (int e = 0; e < 8; ++e) red[wave][cc * 8 + e] = m[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] = join(join(red[0][cc * 8 + e], red[1][cc * 8 + e]), join(red[2][cc * 8 + e], red[3][cc * 8 + e]));
    __syncthreads();
  };
  if (p.col_part) {
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s[e] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s[e] += v[i][e];
    }
    columns(s, [](float a, float b) { return a + b; });
    if (rr == 0)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < nc) p.col_part[blockIdx.y * p.cols + col + e] = s[e];
  }
  if (!p.qt) return;
  float down[8];
  if (BLOCK) {
#pragma unroll
    for (int e = 0; e < 8; ++e) down[e] = power_of_two(-tile_e);
  } else {
    float m[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      m[e] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) m[e] = fmaxf(m[e], finite_abs(v[i][e]));
    }
    columns(m, [](float a, float b) { return fmaxf(a, b); });
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int ex = e4m3_exponent(m[e]);
      down[e] = power_of_two(-ex);
      if (rr == 0 && e < nc) p.qt_scales[(col + e) * gridDim.y + blockIdx.y] = (uint8_t)(ex + 127);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = v[i][e];
    *(int2*)&turned[cc * 8 + e][rr * 8] = e4m3x8(t, down[e]);
  }
  __syncthreads();
  // rows of the transposed tile: eight lanes with 16 bytes each; rows past the end hold zeros, which pad to 16
  const long long pad = ceil_div(p.rows, 16) * 16;
  for (int k = threadIdx.x; k < kGroup * 8; k += 256) {
    const int c = k >> 3, r = (k & 7) * 16;
    if (c0 + c < p.cols && r0 + r < pad) *(i32x4*)(p.qt + (c0 + c) * p.qt_pitch + r0 + r) = *(const i32x4*)&turned[c][r];
  }
}

// column sums of the tiles: out[c] = sum over tiles of part[tile][c], a thread's tiles and then the threads in order
__global__ void __launch_bounds__(1024) column_parts_kernel(const float* part, long long n, long long cols, float* out) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6;
  const long long c = (long long)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < cols)
    for (long long i = slice; i < n; i += 16) s += part[i * cols + c];
  red[slice][lane] = s;
  __syncthreads();
  if (slice || c >= cols) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s += red[i][lane];
  out[c] = s;
}

// ---------------------------------------------------------------------------------------
// Product
// ---------------------------------------------------------------------------------------
struct GemmParams {
  const uint8_t *a, *a_scales, *b, *b_scales;
  const __bf16* bias;
  void* out;
  long long M, N, a_pitch, b_pitch;
  int K, groups, a_shift, b_shift;    // groups: scales per row; shift: 7 where 128 rows share them, else 0
  int out_f32;
};

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

// Buffer descriptor of `bytes` bytes at `base` (both wave-uniform): lanes that read past the end get zeros.
__device__ __forceinline__ u32x4 buffer_of(const uint8_t* base, unsigned bytes) {
  const unsigned long long a = (unsigned long long)base;
  u32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane((unsigned)a);
  r[1] = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32)) & 0xffffu;
  r[2] = __builtin_amdgcn_readfirstlane(bytes);
  r[3] = 0x00020000u;
  return r;
}
// 16 bytes a lane from lane_off + tile_off of the buffer to consecutive LDS (see sa_load_to_lds_16B).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int LDS0>
__device__ __forceinline__ void buffer_to_lds(const u32x4& buffer, unsigned lane_off, unsigned tile_off, unsigned lds_addr) {
  asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(lds_addr), "v"(lane_off), "s"(buffer), "s"(tile_off), "i"(LDS0)
               : "memory", "m0", "scc");
}
// 4 bytes a lane, 256 in all
__device__ __forceinline__ void scale_to_lds(const u32x4& buffer, unsigned lane_off, unsigned tile_off, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
               :
               : "s"(lds_addr), "v"(lane_off), "s"(buffer), "s"(tile_off)
               : "memory", "m0");
}
#pragma clang diagnostic pop

template <int N, class F, int... I>
__device__ __forceinline__ void all_of_impl(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
// f(0), f(1), ... f(N - 1) with the number as a type
template <int N, class F>
__device__ __forceinline__ void all_of(F&& f) {
  all_of_impl<N>(f, std::make_integer_sequence<int, N>{});
}

// N neighbouring results, of which `left` exist.  Rows may start at any element: the memory instructions take addresses that are
// no multiple of their size.  PAST sends them past the caches; see past_caches().
template <bool PAST, int N>
__device__ __forceinline__ void store_run(float* out, const float (&v)[N], long long left) {
  if (left >= N) {
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      const f32x4 r = {v[e], v[e + 1], v[e + 2], v[e + 3]};
      if constexpr (PAST)
        __builtin_nontemporal_store(r, (any_f32x4*)(out + e));
      else
        *(any_f32x4*)(out + e) = r;
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < left) out[e] = v[e];
}
template <bool PAST, int N>
__device__ __forceinline__ void store_run(__bf16* out, const float (&v)[N], long long left) {
  typedef __attribute__((ext_vector_type(N))) __bf16 run;
  typedef run __attribute__((aligned(2))) any_run;
  if (left >= N) {
    run r;
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = (__bf16)v[e];
    if constexpr (PAST)
      __builtin_nontemporal_store(r, (any_run*)out);
    else
      *(any_run*)out = r;
    return;
  }
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < left) out[e] = (__bf16)v[e];
}
// Results go past the caches where every row starts on 64 bytes: no tile then leaves a part of such a piece to its neighbour, and
// the operands keep the cache (1126 x 9216 x 3072: 35.9 us, through the cache 38.7; 14720 x 4768 x 128: 49 and 60).  Other rows
// share pieces, which the cache has to put together (2249 x 6924 x 1392: 38.4 us through it, 52.6 past it; 21006 x 889 x 480: 33
// and 49).
__host__ __device__ __forceinline__ bool past_caches(const GemmParams& p) { return (p.N * (p.out_f32 ? 4 : 2) & 63) == 0 && ((uintptr_t)p.out & 63) == 0; }

// ---------------------------------------------------------------------------------------
// Products that do not fill the chip with large tiles, down to a single row: TM x TN tiles, WM x WN waves, operands streamed
// through a ring of kRing stages in LDS (128 channels each), the reduction split over blockIdx.z where the tiles alone are few
// and it is long.  What bounds it is reading the operands: kRing - 1 stages are on their way while one is worked on, up to three
// workgroups to a CU.  One row times 18432 x 3072: 13.6 us, 4.2 TB/s of weights that are in no cache (registers instead of LDS, a
// wave for 16 columns and a share of the groups, the row quantised in each: 26 us); 200 rows times 9216 x 3072: 17.4 us,
// 0.65 PFLOP/s, a stage's way through barrier, LDS and MFMAs being as long as its loads' there.  Three stages of 64 x 64 rather
// than four, so that three workgroups fit a CU: 17.4 and 22 us for these 200 rows, 13.0 and 14.3 for the one.
// Rows of 128 bytes whose 16-byte chunks are permuted (row_swizzle) so that operand reads spread over all banks.
// v_mfma_scale_f32_16x16x128_f8f6f4 takes a whole group per instruction and applies both scales.  b rows are the instruction's
// first operand, so that a lane ends with four neighbouring columns, or eight where a wave has several fragments of them.
// ---------------------------------------------------------------------------------------
struct SplitParams {
  GemmParams g;
  float* part;                 // [splits][M][N] with more than one split
  int per_split;               // groups of a split
  int tiles, tiles_m, tiles_n, per_xcd;
  int by_rows;                 // tiles that share rows behind each other, not those that share columns
};

constexpr int kScaleSpan = 32;     // groups whose scales are in LDS at a time

template <int TM, int TN, int WM, int WN, int kRing>
__global__ void __launch_bounds__(64 * WM * WN) fp8_gemm_kernel(const SplitParams q) {
  const GemmParams& p = q.g;
  constexpr int kWaves = WM * WN, kM = TM / WM / 16, kN = TN / WN / 16;
  constexpr int kRows = TM + TN, kStage = kRows * 128, kA = TM / 8 / kWaves, kB = TN / 8 / kWaves, kLoads = kA + kB;
  static_assert(TM / 8 % kWaves == 0 && TN / 8 % kWaves == 0, "stage loads must split evenly over the waves");
  extern __shared__ __attribute__((aligned(1024))) char smem_all[];
  uint8_t* scale_lds = (uint8_t*)smem_all;                         // [kRows][kScaleSpan], a rows in front
  const char* smem = smem_all + kRows * kScaleSpan;                // as many stages as the reduction has, kRing at most
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;
  // Workgroups go to the XCDs in turn; an XCD gets neighbouring tiles, those that share columns (or rows, see launch_split) behind
  // each other, so that its cache fetches them once.
  const int id = blockIdx.x, tile = (id & 7) * q.per_xcd + (id >> 3);
  if (tile >= q.tiles) return;
  const long long m0 = (long long)(q.by_rows ? tile / q.tiles_n : tile % q.tiles_m) * TM, n0 = (long long)(q.by_rows ? tile % q.tiles_n : tile / q.tiles_m) * TN;
  const int l16 = lane & 15, quad = lane >> 4;
  const int first = blockIdx.z * q.per_split, stages = min(p.groups, first + q.per_split) - first;

  // Requests: wave w brings the rows 8 (u kWaves + w) + lane / 8 of each operand; rows and channels past the end are zeros.
  const u32x4 a_buf = buffer_of(p.a + m0 * p.a_pitch, (unsigned)(min((long long)TM, p.M - m0) * p.a_pitch));
  // Where a wave has several column fragments, two of them step through 32 columns so that a lane ends with eight neighbours; the
  // chunks of their rows are then permuted by the bits that the rows of a fragment differ in.
  constexpr bool kPaired = kN >= 2;
  auto b_swizzle = [](int row) __attribute__((always_inline)) { return kPaired ? (row >> 1 & 1) | (row >> 2 & 6) : sa_gemm::row_swizzle(row); };
  auto b_row = [&](int j) __attribute__((always_inline)) { return wn * (TN / WN) + (kPaired ? (j >> 1) * 32 + (l16 >> 2) * 8 + (j & 1) * 4 + (l16 & 3) : j * 16 + l16); };
  const u32x4 b_buf = buffer_of(p.b + n0 * p.b_pitch, (unsigned)(min((long long)TN, p.N - n0) * p.b_pitch));
  unsigned off[kLoads];
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int r = ((u < kA ? u : u - kA) * kWaves + wave) * 8 + lane / 8;
    off[u] = (unsigned)(r * (u < kA ? p.a_pitch : p.b_pitch)) + (((lane & 7) ^ (u < kA ? sa_gemm::row_swizzle(r) : b_swizzle(r))) << 4);
  }
  const unsigned lds = (unsigned)(size_t)smem + wave * 1024;
  auto request = [&](int stage, int buf) __attribute__((always_inline)) {
    const int k0 = (first + stage) * kGroup;
    if (p.K - k0 < kGroup) {                       // the last group: its stage is requested last
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int r = ((u < kA ? u : u - kA) * kWaves + wave) * 8 + lane / 8;
        if ((((lane & 7) ^ (u < kA ? sa_gemm::row_swizzle(r) : b_swizzle(r))) << 4) >= p.K - k0) off[u] = 0x80000000u;
      }
    }
    all_of<kLoads>([&](auto u_c) __attribute__((always_inline)) {
      constexpr int u = decltype(u_c)::value;
      buffer_to_lds<(u < kA ? u * kWaves : TM / 8 + (u - kA) * kWaves) * 1024>(u < kA ? a_buf : b_buf, off[u], (unsigned)k0, lds + buf * kStage);
    });
  };
  // scales of stages s .. s + kScaleSpan - 1, four to a word; all earlier reads of the scales are behind a barrier
  auto stage_scales = [&](int s) __attribute__((always_inline)) {
    const int n = min(kScaleSpan, stages - s);
    for (int t = threadIdx.x; t < kRows * (kScaleSpan / 4); t += 64 * kWaves) {
      const int row = t / (kScaleSpan / 4), g = t % (kScaleSpan / 4) * 4;
      if (g >= n) continue;
      const long long r = row < TM ? min(p.M - 1, m0 + row) : min(p.N - 1, n0 + row - TM);
      const uint8_t* from = (row < TM ? p.a_scales + (r >> p.a_shift) * p.groups : p.b_scales + (r >> p.b_shift) * p.groups) + first + s + g;
      unsigned v = 0;
      if (g + 4 <= n) {
        __builtin_memcpy(&v, from, 4);
      } else {
        for (int e = 0; e < n - g; ++e) v |= (unsigned)from[e] << (8 * e);
      }
      *(unsigned*)(scale_lds + row * kScaleSpan + g) = v;
    }
  };
  f32x4 acc[kN][kM] = {};
  const int ra = wm * (TM / WM) + l16;
  // this lane's row in fragment 0 of each operand and its first chunk; the second is 64 bytes away by XOR
  const unsigned a_read = (unsigned)(ra * 128 + ((quad ^ sa_gemm::row_swizzle(ra)) << 4)), b_read = (unsigned)((TM + b_row(0)) * 128 + ((quad ^ b_swizzle(b_row(0))) << 4));
  auto operand = [&](const char* at, unsigned o) __attribute__((always_inline)) {
    const i32x4 lo = *(const i32x4*)(at + o), hi = *(const i32x4*)(at + (o ^ 64));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  for (int s0 = 0; s0 < stages; s0 += kScaleSpan) {
    const int span = min(kScaleSpan, stages - s0);
    if (s0) sa_gemm::lds_barrier();                  // every wave has read its last operands and scales
#pragma unroll
    for (int r = 0; r < kRing - 1; ++r)
      if (r < span) request(s0 + r, r);
    stage_scales(s0);
    int buf = 0;
    unsigned ea[kM], eb[kN];
    for (int s = 0; s < span; ++s) {
      // everything but the requests of the stages behind this one has landed
      if (s + kRing - 2 < span)
        sa_wait_vmem_but<(kRing - 2) * kLoads>();
      else
        sa_wait_vmem();
      sa_gemm::lds_barrier();
      const char* at = smem + buf * kStage;
      i32x8 xa[kM], wb[kN];
      if (s % 4 == 0) {
#pragma unroll
        for (int i = 0; i < kM; ++i) ea[i] = *(const unsigned*)(scale_lds + (ra + i * 16) * kScaleSpan + s);
#pragma unroll
        for (int j = 0; j < kN; ++j) eb[j] = *(const unsigned*)(scale_lds + (TM + b_row(j)) * kScaleSpan + s);
      }
#pragma unroll
      for (int i = 0; i < kM; ++i) xa[i] = operand(at, a_read + i * 2048);
#pragma unroll
      for (int j = 0; j < kN; ++j) wb[j] = operand(at, b_read + (kPaired ? (j >> 1) * 4096 + (j & 1) * 512 : j * 2048));
      __builtin_amdgcn_sched_barrier(0);
      if (s + kRing - 1 < span) request(s0 + s + kRing - 1, buf == 0 ? kRing - 1 : buf - 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < kN; ++j)
#pragma unroll
        for (int i = 0; i < kM; ++i) acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wb[j], xa[i], acc[j][i], 0, 0, 0, eb[j], 0, ea[i]);
#pragma unroll
      for (int i = 0; i < kM; ++i) ea[i] >>= 8;
#pragma unroll
      for (int j = 0; j < kN; ++j) eb[j] >>= 8;
      buf = buf == kRing - 1 ? 0 : buf + 1;
    }
  }
  const bool split = gridDim.z > 1, to_f32 = split || p.out_f32, past = !split && past_caches(p);
  float* f32_out = split ? q.part + (size_t)blockIdx.z * p.M * p.N : (float*)p.out;
  constexpr int kRun = kPaired ? 2 : 1;            // fragments whose results are neighbours
#pragma unroll
  for (int j = 0; j < kN; j += kRun) {
    const long long n = n0 + wn * (TN / WN) + (kPaired ? (j >> 1) * 32 + quad * 8 : j * 16 + quad * 4);
    float bias[4 * kRun] = {};
    if (p.bias && !split) {
#pragma unroll
      for (int e = 0; e < 4 * kRun; ++e) bias[e] = n + e < p.N ? (float)p.bias[n + e] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kM; ++i) {
      const long long m = m0 + wm * (TM / WM) + i * 16 + l16;
      if (m >= p.M || n >= p.N) continue;
      float v[4 * kRun];
#pragma unroll
      for (int e = 0; e < 4 * kRun; ++e) v[e] = acc[j + e / 4][i][e & 3] + bias[e];
      if (to_f32) {
        if (past)
          store_run<true>(f32_out + m * p.N + n, v, p.N - n);
        else
          store_run<false>(f32_out + m * p.N + n, v, p.N - n);
      } else {
        if (past)
          store_run<true>((__bf16*)p.out + m * p.N + n, v, p.N - n);
        else
          store_run<false>((__bf16*)p.out + m * p.N + n, v, p.N - n);
      }
    }
  }
}

// Sum of the splits in their order, plus the bias; eight results a thread.  Where 100 x 304 x 9008 fills five CUs, four splits
// and this take 13.8 us, the product in one piece 25.8.
__global__ void __launch_bounds__(256) join_splits_kernel(const float* part, int splits, const __bf16* bias, void* out, int out_f32, long long M, long long N) {
  const long long total = M * N, i = ((long long)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= total) return;
  const int n = (int)min(8LL, total - i);
  float v[8] = {};
  if (n == 8 && total % 4 == 0) {
    for (int s = 0; s < splits; ++s) {
      const f32x4 a = *(const f32x4*)(part + s * total + i), b = *(const f32x4*)(part + s * total + i + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] += a[e];
        v[e + 4] += b[e];
      }
    }
  } else {
    for (int s = 0; s < splits; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) v[e] += part[s * total + i + e];
  }
  if (bias)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) v[e] += (float)bias[(i + e) % N];
  if (n == 8 && ((uintptr_t)out & 15) == 0) {
    if (out_f32) {
      *(f32x4*)((float*)out + i) = f32x4{v[0], v[1], v[2], v[3]};
      *(f32x4*)((float*)out + i + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
      bf16x8 r;
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = (__bf16)v[e];
      *(bf16x8*)((__bf16*)out + i) = r;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) {
        if (out_f32)
          ((float*)out)[i + e] = v[e];
        else
          ((__bf16*)out)[i + e] = (__bf16)v[e];
      }
  }
}

// ---------------------------------------------------------------------------------------
// Large products: tiles of 128 to 256 rows and 256 columns, four waves with a quarter each, one workgroup per CU that walks over
// its share of the tiles.  33024 x 9216 x 3072 735 to 810 us over several chips, 2.3 to 2.5 PFLOP/s, 33024 x 3072 x 3072 into float32
// 306 us, 2.0 PFLOP/s.  In the first the matrix pipes are busy 63 % of the time, at 1.74 GHz (the instruction alone, from registers:
// 4.3 PFLOP/s), and a wave waits 37 % of its own; how much of the rest is the clock under this load and how much the waits has not been
// taken apart.  Tiles of 224 and 256 rows keep four registers in scratch memory.
//
// What the tile is chosen by is LDS traffic: per 128 channels a wave of 128 x 128 reads 32 KiB for 64 MFMAs of 32 cycles, so
// the four waves and the arriving 64 KiB take about 1500 of the 2048 cycles that the matrix pipes work; 64 x 64 to a wave would
// take 3072.  The accumulators then fill half of the register file, one wave runs on each SIMD, and nothing hides a wait: so
// operands are read from LDS ahead of their MFMAs, and requested from memory a stage (128 channels = one scale group) earlier:
//     eight steps j of eight MFMAs: column fragment j of stage s against the eight row fragments, which are in registers
//     steps 0 .. 5: column fragments 2 .. 7 and the row fragments of stage s + 1 are read
//     in front of step 6: rows of stage s + 2 and columns of stage s + 1 have landed, all waves' reads have returned: barrier
//     steps 6, 7, and 0, 1 of the next stage: rows of stage s + 3 and columns of stage s + 2 are requested, over the rows of
//     stage s + 1 and the columns of stage s, whose last reads were in front of the barrier; fragments 0, 1 of stage s + 1
// The stages of a workgroup's tiles are one stream: the last ones of a tile request and read the first of the next.
// Column fragments step through the columns so that a lane ends with runs of eight neighbouring results, 64 bytes for four lanes.
// Scale bytes come the same way, in an order in which a lane finds those of its eight fragments in eight bytes
// (pack_scales_kernel); the MFMAs take each from its byte.
// ---------------------------------------------------------------------------------------
constexpr int kBig = 256, kBigBuffer = kBig * 128;             // columns of a tile, bytes of a stage of them
constexpr int kScaleRing = 4;                                  // pairs of stages whose scales have room in LDS
constexpr int kScaleBytes = 256;                               // of one operand half and two stages
constexpr int kBigLds = 4 * kBigBuffer + 4 * kScaleRing * kScaleBytes;
constexpr int kBand = 8;                                       // tiles that share columns and run together on an XCD

// rows: rows of a tile.  The last tile starts early enough to be whole: it computes and stores some rows again, the same way.
__host__ __device__ constexpr long long row_of_tile(long long tile, int rows, long long M) { return tile * rows < M - rows ? tile * rows : M - rows; }

// Scales for the kernel below: [half tile][stage, an even number][16 lanes][8 fragments] bytes, rows first, then columns.
// Stages past the last group and columns past the end get 2^0.
struct PackParams {
  const uint8_t *a_scales, *b_scales;
  uint8_t* out;
  long long M, N, a_bytes, bytes;
  int groups, stages, a_shift, b_shift, tile_rows;
};
__global__ void __launch_bounds__(256) pack_scales_kernel(const PackParams p) {
  const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 8;       // eight fragments of a lane
  if (at >= p.bytes) return;
  const bool rows = at < p.a_bytes;
  const long long in = rows ? at : at - p.a_bytes;
  const int lane = (int)(in / 8 % 16), stage = (int)(in / 128 % p.stages);
  const long long half = in / 128 / p.stages;
  const uint8_t* scales = rows ? p.a_scales : p.b_scales;
  const int shift = rows ? p.a_shift : p.b_shift;
  const long long last = (rows ? p.M : p.N) - 1, first = rows ? row_of_tile(half >> 1, p.tile_rows, p.M) + (half & 1) * (p.tile_rows / 2) : half * 128;
  uint8_t v[8];
#pragma unroll
  for (int f = 0; f < 8; ++f) {                // no load under a condition, which would make it wait for the one before
    const long long r = first + (rows ? f * 16 + lane : (f >> 1) * 32 + (lane >> 2) * 8 + (f & 1) * 4 + (lane & 3));
    v[f] = scales[(min(r, last) >> shift) * p.groups + min(stage, p.groups - 1)];
    if (stage >= p.groups || (!rows && r > last)) v[f] = 127;
  }
  __builtin_memcpy(p.out + at, v, 8);
}

template <int KI, bool OUT_F32>
__global__ void __launch_bounds__(256, 1) fp8_gemm_big_kernel(const GemmParams p, const uint8_t* scales, int tiles_m, int tiles_n, int per_xcd) {
  constexpr int kRows = 32 * KI, kRowBuffer = kRows * 128, kCol0 = 2 * kRowBuffer;     // LDS: two stages of rows, of columns, scales
  constexpr int kScale0 = kCol0 + 2 * kBigBuffer, kStores = 4 * KI;                    // stores of a whole tile by a wave, at least
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave & 1, wn = wave >> 1, l16 = lane & 15, quad = lane >> 4;
  const unsigned lds = (unsigned)(size_t)smem;
  const int stages = (p.groups + 1) & ~1;                       // an odd number of groups is filled up by one of zeros

  // Requests: wave w brings the rows 8 (4 u + w) + lane / 8, u = 0, 1, ..., of each operand.  Chunks are permuted so that the
  // sixteen lanes that read the same chunk of a fragment's rows find them in distinct banks: by bits 1-3 of the row for the
  // rows, whose fragments are sixteen neighbours, and by bits 1, 3 and 4 for the columns, whose fragments are four times four.
  const int lr = lane >> 3, lc = lane & 7;
  const unsigned a_chunk = (lc ^ (((wave & 1) << 2) | (lr >> 1))) << 4;
  const unsigned b_chunk = (lc ^ (((lr >> 1) & 1) | (wave << 1))) << 4;
  const unsigned a_row = (unsigned)((8 * wave + lr) * p.a_pitch), b_row = (unsigned)((8 * wave + lr) * p.b_pitch);
  const unsigned a_step = (unsigned)(32 * p.a_pitch), b_step = (unsigned)(32 * p.b_pitch);

  // operand reads: this lane's row in fragment 0, its first chunk; the second is 64 bytes away by XOR
  const unsigned x_read = (unsigned)((wm * (kRows / 2) + l16) * 128 + ((quad ^ (l16 >> 1)) << 4));
  const unsigned w_read = (unsigned)(kCol0 + (wn * 128 + (l16 >> 2) * 8 + (l16 & 3)) * 128 + ((quad ^ (((l16 >> 1) & 1) | ((l16 >> 2) << 1))) << 4));
  // scales in LDS: [operand][half][ring][stage of the pair][lane][fragment]; wave w brings those of operand w / 2, half w % 2
  const unsigned s_base = kScale0, s_to = lds + s_base + wave * kScaleRing * kScaleBytes;
  const unsigned ea_read = s_base + wm * kScaleRing * kScaleBytes + l16 * 8, eb_read = s_base + (2 + wn) * kScaleRing * kScaleBytes + l16 * 8;

  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, slots = gridDim.x >> 3;
  const int total = tiles_m * tiles_n, last_tile = min(total, (xcd + 1) * per_xcd);
  int tile = xcd * per_xcd + slot;
  if (tile >= last_tile) return;

  const bool past = past_caches(p);
  struct Tile {
    long long m0, n0;
    u32x4 a, b, s;
    int valid;
  };
  auto tile_at = [&](int t) __attribute__((always_inline)) {
    Tile r;
    r.valid = t < last_tile;
    if (!r.valid) t = last_tile - 1;
    const int band = t / (kBand * tiles_n), in = t - band * kBand * tiles_n;
    const int high = min(kBand, tiles_m - band * kBand);
    const int tm = band * kBand + in % high, tn = in / high;
    r.m0 = row_of_tile(tm, kRows, p.M);
    r.n0 = (long long)tn * kBig;
    r.a = buffer_of(p.a + r.m0 * p.a_pitch, r.valid ? (unsigned)(kRows * p.a_pitch) : 0u);
    r.b = buffer_of(p.b + r.n0 * p.b_pitch, r.valid ? (unsigned)(min((long long)kBig, p.N - r.n0) * p.b_pitch) : 0u);   // columns past the end are zeros
    const long long half = wave < 2 ? 2 * tm + wave : 2LL * tiles_m + 2 * tn + (wave - 2);
    r.s = buffer_of(scales + half * stages * 128, r.valid ? (unsigned)stages * 128 : 0u);
    return r;
  };
  Tile now = tile_at(tile), next = tile_at(tile + slots);
  auto pick = [](bool first, const u32x4& a, const u32x4& b) __attribute__((always_inline)) {
    return u32x4{first ? a[0] : b[0], first ? a[1] : b[1], first ? a[2] : b[2], a[3]};
  };
  // One request of rows (u = 0 .. KI - 1) or columns (0 .. 7), in order.  Offsets run along in one register each; they are
  // kept from the compiler, which would hold all of them.  s: stage, counted from the current tile's first.
  unsigned a_off = a_row, b_off = b_row;
  auto request = [&](auto rows_c, auto u_c, int s, unsigned to) __attribute__((always_inline)) {
    constexpr bool rows = decltype(rows_c)::value;
    constexpr int u = decltype(u_c)::value;
    unsigned& row = rows ? a_off : b_off;
    if constexpr (u == 0) row = rows ? a_row : b_row;
    const bool here = s < stages;
    const int k0 = (here ? s : s - stages) * kGroup, left = p.K - k0;
    const unsigned chunk = rows ? a_chunk : b_chunk;
    const unsigned off = (int)chunk < left ? row + chunk : 0x80000000u;         // channels past the end are zeros
    // the scalar offset has to lie inside the buffer: the range check subtracts it
    buffer_to_lds<u * 4096>(rows ? pick(here, now.a, next.a) : pick(here, now.b, next.b), off, left > 0 && (here || next.valid) ? (unsigned)k0 : 0u,
                            to + wave * 1024);
    row += rows ? a_step : b_step;
    asm volatile("" : "+v"(row));
  };
  using T = std::true_type;
  using F = std::false_type;
  auto request_rows = [&](int s) __attribute__((always_inline)) {
    all_of<KI>([&](auto u) __attribute__((always_inline)) { request(T{}, u, s, lds + (s & 1) * kRowBuffer); });
  };
  auto request_columns = [&](int s) __attribute__((always_inline)) {
    all_of<8>([&](auto u) __attribute__((always_inline)) { request(F{}, u, s, lds + kCol0 + (s & 1) * kBigBuffer); });
  };
  // the scales of stages s and s + 1 (s even): four bytes a lane
  auto request_scales = [&](int s, int ring) __attribute__((always_inline)) {
    const bool here = s < stages;
    const unsigned at = (unsigned)(here ? s : s - stages) * 128;
    scale_to_lds(pick(here, now.s, next.s), (unsigned)lane * 4, here || next.valid ? at : 0u, s_to + ring * kScaleBytes);
  };
  struct Fragment {
    i32x4 lo, hi;
    __device__ __forceinline__ i32x8 all() const { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }
  };
  auto chunk_at = [&](unsigned at) __attribute__((always_inline)) { return *(const i32x4*)(smem + at); };
  auto scale_of = [&](unsigned at) __attribute__((always_inline)) { return *(const int2*)(smem + at); };

  Fragment x[2][KI], w[4];
  int2 ea[2], eb[2];
  request_rows(0);
  request_columns(0);
  request_rows(1);
  request_scales(0, 0);
  request_scales(2, 1);
  sa_wait_vmem();
  sa_gemm::lds_barrier();
#pragma unroll
  for (int i = 0; i < KI; ++i) x[0][i] = {chunk_at(x_read + i * 2048), chunk_at((x_read ^ 64) + i * 2048)};
#pragma unroll
  for (int j = 0; j < 2; ++j) w[j] = {chunk_at(w_read + j * 512), chunk_at((w_read ^ 64) + j * 512)};
  ea[0] = scale_of(ea_read);
  eb[0] = scale_of(eb_read);
  __builtin_amdgcn_s_waitcnt(0xC07F);
  sa_gemm::lds_barrier();
  request_rows(2);
  request_columns(1);
  sa_wait_vmem();

  f32x4 acc[8][KI];
  unsigned ring = 0;                   // where the scales of this pair of stages are
  for (;;) {
    int s = 0;
    auto stage = [&](auto odd_c, auto first_c) __attribute__((always_inline)) {
      constexpr int odd = decltype(odd_c)::value;
      constexpr bool first = decltype(first_c)::value;
      const unsigned x_base = x_read + (1 - odd) * kRowBuffer, w_base = w_read + odd * kBigBuffer, w_base_next = w_read + (1 - odd) * kBigBuffer;
      const unsigned scales_next = odd ? ((ring + 1) & (kScaleRing - 1)) * kScaleBytes : ring * kScaleBytes + 128;
      all_of<8 * KI>([&](auto t_c) __attribute__((always_inline)) {
        constexpr int t = decltype(t_c)::value, j = t / KI, i = t % KI;
        if constexpr (t == 6 * KI) {
          // The first stage of a tile waits for its predecessor's loads but not for the stores of the results behind them.
          __builtin_amdgcn_s_waitcnt(0xC07F);
          if constexpr (first)
            sa_wait_vmem_but<kStores>();
          else
            sa_wait_vmem();
          sa_gemm::lds_barrier();
        }
        const int es_b = j < 4 ? eb[odd].x : eb[odd].y, es_a = i < 4 ? ea[odd].x : ea[odd].y;
        const f32x4 c = first ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[j][i];
        acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[j & 3].all(), x[odd][i].all(), c, 0, 0, j & 3, es_b, i & 3, es_a);
        __builtin_amdgcn_sched_barrier(0);
        // behind each MFMA at most one LDS read and one request
        constexpr int kHalves = (2 * KI + 3) / 4, h = (j - 1) * kHalves + i - 2;      // halves of row fragments, over steps 1 .. 4
        if constexpr (i < 2) {
          constexpr int f = j < 6 ? j + 2 : j - 6;
          const unsigned at = ((j < 6 ? w_base : w_base_next) ^ (i * 64)) + (f >> 1) * 4096 + (f & 1) * 512;
          if constexpr (i == 0)
            w[f & 3].lo = chunk_at(at);
          else
            w[f & 3].hi = chunk_at(at);
        } else if constexpr (j >= 1 && j < 5 && i < 2 + kHalves && h < 2 * KI) {
          const unsigned at = (x_base ^ (h % 2 * 64)) + h / 2 * 2048;
          if constexpr (h % 2 == 0)
            x[1 - odd][h / 2].lo = chunk_at(at);
          else
            x[1 - odd][h / 2].hi = chunk_at(at);
        } else if constexpr (j == 0 && i == 2) {
          ea[1 - odd] = scale_of(ea_read + scales_next);
        } else if constexpr (j == 0 && i == 3) {
          eb[1 - odd] = scale_of(eb_read + scales_next);
        }
        constexpr int kRowsPerStep = (KI + 1) / 2;
        if constexpr (j >= 6)                          // rows of stage s + 3 behind the barrier,
          all_of<kRowsPerStep>([&](auto r) __attribute__((always_inline)) {
            constexpr int n = decltype(r)::value, u = (j - 6) * kRowsPerStep + n;
            if constexpr (i == (n * KI + KI / 2) / kRowsPerStep && u < KI) request(T{}, std::integral_constant<int, u>{}, s + 3, lds + (1 - odd) * kRowBuffer);
          });
        if constexpr (j < 2 && !first)                 // columns of stage s + 1 behind that of the stage before
          all_of<4>([&](auto r) __attribute__((always_inline)) {
            constexpr int n = decltype(r)::value, u = j * 4 + n;
            if constexpr (i == (n * KI + KI / 2) / 4) request(F{}, std::integral_constant<int, u>{}, s + 1, lds + kCol0 + (1 - odd) * kBigBuffer);
          });
        if constexpr (t == 8 * KI - 1 && !odd) request_scales(s + 4, (ring + 2) & (kScaleRing - 1));
        __builtin_amdgcn_sched_barrier(0);
      });
      if (odd) ring = (ring + 1) & (kScaleRing - 1);
      ++s;
    };
    using Even = std::integral_constant<int, 0>;
    using Odd = std::integral_constant<int, 1>;
    stage(Even{}, T{});
    stage(Odd{}, F{});
    while (s < stages) {
      stage(Even{}, F{});
      stage(Odd{}, F{});
    }
    // the results are formed here: the compiler would move MFMAs behind the branches below, and operands to memory for it
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < KI; ++i) asm volatile("" : "+a"(acc[j][i]));

    request_columns(stages + 1);         // in front of the stores, which nothing waits for before the next tile's second stage
    const long long n = now.n0 + wn * 128 + quad * 8;
    const bool whole = now.n0 + kBig <= p.N;
    using Out = std::conditional_t<OUT_F32, float, __bf16>;
    Out* const out = (Out*)p.out + (now.m0 + wm * (kRows / 2) + l16) * p.N + n;
    auto store_all = [&](auto whole_c, auto past_c) __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const long long left = whole_c.value ? 8 : p.N - n - q * 32;
        float bias[8] = {};
        if (p.bias) {
#pragma unroll
          for (int e = 0; e < 8; ++e) bias[e] = e < left ? (float)p.bias[n + q * 32 + e] : 0.f;
        }
        Out* at = out + q * 32;
#pragma unroll
        for (int i = 0; i < KI; ++i) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = acc[q * 2 + e / 4][i][e & 3] + bias[e];
          store_run<past_c.value>(at, v, left);
          at += 16 * p.N;
        }
      }
    };
    if (whole && past)
      store_all(T{}, T{});
    else if (whole)
      store_all(T{}, F{});
    else
      store_all(F{}, F{});
    if (!whole) sa_wait_vmem();          // fewer stores than kStores: nothing is left for the wait that counts on them
    tile += slots;
    if (!next.valid) break;
    now = next;
    next = tile_at(tile + slots);
  }
  sa_wait_vmem();                      // nothing may still be on its way to LDS when the workgroup ends
}

// ---------------------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------------------
int launched(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? 0 : sa_fail(SPARSE_ATTN_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
}

void launch_quantize(const QuantParams& p, bool block, hipStream_t stream) {
  const bool vec = p.cols % 8 == 0;
  if (!block && !p.qt && !p.col_part) {
    const long long want = ceil_div(p.rows * ceil_div(p.cols, kGroup), 16);
    const unsigned grid = (unsigned)(want < 16384 ? want : 16384);
    if (vec)
      hipLaunchKernelGGL(quantize_rows_kernel<true>, dim3(grid), dim3(256), 0, stream, p);
    else
      hipLaunchKernelGGL(quantize_rows_kernel<false>, dim3(grid), dim3(256), 0, stream, p);
    return;
  }
  const dim3 grid((unsigned)ceil_div(p.cols, kGroup), (unsigned)ceil_div(p.rows, kGroup));
  if (block) {
    if (vec)
      hipLaunchKernelGGL((quantize_tile_kernel<true, true>), grid, dim3(256), 0, stream, p);
    else
      hipLaunchKernelGGL((quantize_tile_kernel<false, true>), grid, dim3(256), 0, stream, p);
  } else {
    if (vec)
      hipLaunchKernelGGL((quantize_tile_kernel<true, false>), grid, dim3(256), 0, stream, p);
    else
      hipLaunchKernelGGL((quantize_tile_kernel<false, false>), grid, dim3(256), 0, stream, p);
  }
}

// How a product is computed, and the scratch that takes.
struct Route {
  int ki;                      // large kernel: rows of a tile / 32; 0: the kernel for the others, with
  int tile;                    // one of kTiles, and
  int splits, per_split;       // parts of the reduction, groups in each
};

// rows, columns, what a stage costs a CU (us / 100), and how many thirds of a workgroup's time n of them take on one CU:
// max(3, rate n - less), as they overlap where several fit its LDS
struct TileCost {
  int m, n, stage, rate, less, threads;
};
constexpr TileCost kTiles[] = {{128, 128, 64, 3, 0, 512}, {64, 64, 27, 2, 0, 256}, {32, 64, 24, 3, 1, 256}};

constexpr long long kMostSplitTiles = 512;     // tiles times splits, at most
constexpr int kLeastSplit = 16;                // groups of a split, about

// Scratch memory that a product of these sizes may take, whichever its route: the splits' sums or the packed scales.  It does not
// grow when a size shrinks, unlike what the routes need (of 3072 columns and 12288 channels: one row 48 KiB, in four splits, 400
// rows nothing), so that no later and smaller call finds too little: such a call may be under capture.
size_t scratch_of(long long M, long long N, int groups) {
  size_t sums = 0, scales = 0;
  if (groups >= 2 * kLeastSplit) sums = (size_t)std::min(groups / kLeastSplit * M * N, kMostSplitTiles * kTiles[0].m * kTiles[0].n) * 4;
  if (M >= 128 && groups >= 3) scales = (size_t)(ceil_div(M, 128) + ceil_div(N, kBig)) * 2 * ((groups + 1) & ~1) * 128;
  return sums > scales ? sums : scales;
}

// Takes the route that a small model of the times calls the fastest.  Its constants are measured (us / 100), over 1 to 33024
// rows, 300 to 18432 columns and 128 to 9008 channels; what it is right to within (15 %) is less than what the routes differ by
// where the choice matters, for instance (us):
//     rows x columns x channels   32 x 64   64 x 64   128 x 128   large
//     1 x 18432 x 3072             15.2      13.5       18.3       -
//     100 x 9216 x 3072            18.8      12.7       18.0       -
//     200 x 9216 x 3072            21.9      17.4       18.9      31
//     1000 x 9216 x 3072           84        46         51        35 (160 rows; 256: 41, 128: 53)
//     2000 x 9216 x 3072          190       111         84        60 (160 rows; 256: 78)
//     9001 x 3072 x 256            50        36         28         -
//     100 x 304 x 9008             22.7      25.8       44         -   in 4 splits 13.6, 13.8, 18.5
// splits is 0 where there is none, with more results than fit any memory.  A large tile's stage does not get cheaper in proportion with its rows (256: 143, 128: 95): below some 200 rows it waits for memory.
Route route_of(long long M, long long N, int groups) {
  Route best = {};
  long long best_cost = 1LL << 60;
  auto consider = [&](const Route& r, long long cost) {
    if (cost < best_cost) best = r, best_cost = cost;
  };
  for (int t = 0; t < 3; ++t) {
    const TileCost& c = kTiles[t];
    const long long tiles = ceil_div(M, c.m) * ceil_div(N, c.n);
    if ((tiles + 7) * c.threads > 0xffffffffLL) continue;          // threads of a launch
    // the reduction is split where it is long and the tiles are few: joining costs a launch and the sums' traffic
    const long long most = tiles < 256 ? std::min(kMostSplitTiles / tiles, (long long)groups / kLeastSplit) : 1;
    for (long long splits = 1; splits <= std::max(1LL, most); splits *= 2) {
      Route r = {0, t, 1, (int)ceil_div(groups, splits)};
      r.splits = (int)ceil_div(groups, r.per_split);
      const long long per_cu = ceil_div(tiles * r.splits, 256);
      // sums are written and read at 4 TB/s
      long long cost = 200 + std::max(3LL, c.rate * per_cu - c.less) * (r.per_split * (long long)c.stage + 200) / 3;
      if (r.splits > 1) cost += 400 + (long long)r.splits * M * N * 8 / 40000;
      consider(r, cost);
    }
  }
  constexpr int stage[] = {95, 108, 120, 140, 143};            // of tiles of 128, 160, 192, 224, 256 rows
  // the stream of requests runs up to four stages ahead, into the next tile but not past it: three groups at least
  for (int ki = 8; ki >= 4 && groups >= 3; --ki) {
    if (M < 32 * ki) continue;
    const long long tiles_m = ceil_div(M, 32 * ki), tiles = tiles_m * ceil_div(N, kBig);
    if (tiles > 0x3fffffff) continue;
    const int stages = (groups + 1) & ~1;
    const long long rounds = ceil_div(ceil_div(tiles, 8), 32);
    consider({ki, 0, 1, 0}, 600 + rounds * ((long long)stages * stage[ki - 4] + 350));
  }
  return best;
}

template <int KI, bool OUT_F32>
int launch_big(const char* who, const GemmParams& p, uint8_t* packed, hipStream_t stream) {
  if (p.M < 32 * KI || p.groups < 3) return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: tiles of %d rows do not fit %lld rows of %d groups", who, 32 * KI, p.M, p.groups);
  constexpr int lds = kBigLds - (8 - KI) * 2 * 4096;
  static const hipError_t attr_err = hipFuncSetAttribute((const void*)fp8_gemm_big_kernel<KI, OUT_F32>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (attr_err != hipSuccess) return sa_fail(SPARSE_ATTN_ERR_HIP, "%s: hipFuncSetAttribute failed: %s", who, hipGetErrorString(attr_err));
  const int tiles_m = (int)ceil_div(p.M, 32 * KI), tiles_n = (int)ceil_div(p.N, kBig), stages = (p.groups + 1) & ~1;
  const long long a_bytes = (long long)tiles_m * 2 * stages * 128, bytes = a_bytes + (long long)tiles_n * 2 * stages * 128;
  const PackParams pack = {p.a_scales, p.b_scales, packed, p.M, p.N, a_bytes, bytes, p.groups, stages, p.a_shift, p.b_shift, 32 * KI};
  hipLaunchKernelGGL(pack_scales_kernel, dim3((unsigned)ceil_div(bytes / 8, 256)), dim3(256), 0, stream, pack);
  const int per_xcd = (int)ceil_div((long long)tiles_m * tiles_n, 8);
  const int slots = per_xcd < 32 ? per_xcd : 32;
  hipLaunchKernelGGL((fp8_gemm_big_kernel<KI, OUT_F32>), dim3(8 * slots), dim3(256), lds, stream, p, packed, tiles_m, tiles_n, per_xcd);
  return launched(who);
}

template <int TM, int TN, int WM, int WN, int RING>
int launch_split(const char* who, const GemmParams& p, const Route& r, float* part, hipStream_t stream) {
  constexpr int most = RING * (TM + TN) * 128 + (TM + TN) * kScaleSpan;
  const int lds = (r.per_split < RING ? r.per_split : RING) * (TM + TN) * 128 + (TM + TN) * kScaleSpan;
  static const hipError_t attr_err = hipFuncSetAttribute((const void*)fp8_gemm_kernel<TM, TN, WM, WN, RING>, hipFuncAttributeMaxDynamicSharedMemorySize, most);
  if (attr_err != hipSuccess) return sa_fail(SPARSE_ATTN_ERR_HIP, "%s: hipFuncSetAttribute failed: %s", who, hipGetErrorString(attr_err));
  const int tiles_m = (int)ceil_div(p.M, TM), tiles_n = (int)ceil_div(p.N, TN), tiles = tiles_m * tiles_n, per_xcd = (tiles + 7) / 8;
  // Where neighbours in a row share pieces of memory, they follow each other if all columns fit a cache of 4 MB next to the rest
  // (14719 x 4758 x 128: 52 us, the other way 85); else columns are fetched once (300 x 9216 x 3072: 18.5 us, by rows 21.7).
  const int by_rows = !past_caches(p) && p.N * p.K <= 2 << 20;
  hipLaunchKernelGGL((fp8_gemm_kernel<TM, TN, WM, WN, RING>), dim3(8 * per_xcd, 1, (unsigned)r.splits), dim3(64 * WM * WN), lds, stream,
                     SplitParams{p, part, r.per_split, tiles, tiles_m, tiles_n, per_xcd, by_rows});
  if (r.splits > 1)
    hipLaunchKernelGGL(join_splits_kernel, dim3((unsigned)ceil_div(ceil_div(p.M * p.N, 8), 256)), dim3(256), 0, stream, part, r.splits, p.bias, p.out,
                       p.out_f32, p.M, p.N);
  return launched(who);
}

// scratch: scratch_of() bytes, 256-byte aligned
int launch_gemm(const char* who, const GemmParams& p, const Route& r, uint8_t* scratch, hipStream_t stream) {
  if (r.splits == 0) return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: too many results, %lld x %lld", who, p.M, p.N);
  if (r.ki == 0)
    switch (r.tile) {
      case 0: return launch_split<128, 128, 4, 2, 3>(who, p, r, (float*)scratch, stream);
      case 1: return launch_split<64, 64, 2, 2, 3>(who, p, r, (float*)scratch, stream);
      default: return launch_split<32, 64, 1, 4, 6>(who, p, r, (float*)scratch, stream);
    }
  auto big = [&](auto ki) {
    return p.out_f32 ? launch_big<decltype(ki)::value, true>(who, p, scratch, stream) : launch_big<decltype(ki)::value, false>(who, p, scratch, stream);
  };
  switch (r.ki) {
    case 8: return big(std::integral_constant<int, 8>{});
    case 7: return big(std::integral_constant<int, 7>{});
    case 6: return big(std::integral_constant<int, 6>{});
    case 5: return big(std::integral_constant<int, 5>{});
    default: return big(std::integral_constant<int, 4>{});
  }
}

int check_product(const char* who, long long M, long long N, long long K, int out_dtype) {
  if (M <= 0 || N <= 0 || K <= 0) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: M=%lld, N=%lld, K=%lld must be positive", who, M, N, K);
  // rows of a tile are addressed with 32 bits, tiles and their rows by the grid
  if (M > (1LL << 22) || N > (1LL << 22) || K > (1LL << 22))
    return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: at most 2^22 rows and channels, got M=%lld, N=%lld, K=%lld", who, M, N, K);
  if (K % 16) return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: K=%lld must be a multiple of 16", who, K);
  if (out_dtype != SPARSE_BLOCK_BF16 && out_dtype != SPARSE_BLOCK_F32)
    return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: the result's type %d must be BF16 or F32", who, out_dtype);
  return 0;
}

struct Range {
  const char* name;
  const void* p;
  size_t bytes;
};
int check_result(const char* who, const Range& out, std::initializer_list<Range> ins) {
  for (const Range& in : ins)
    if (overlap(out.p, out.bytes, in.p, in.bytes)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: %s must not overlap %s", who, out.name, in.name);
  return 0;
}
int check_elements(const char* who, const void* p, int size, const char* name) {
  return (uintptr_t)p & (size - 1) ? sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: %s must be aligned to its elements", who, name) : 0;
}

size_t rounded(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

extern "C" {

int sparse_fp8_quantize(const void* x, void* q, uint8_t* q_scales, void* qt, uint8_t* qt_scales, long long qt_pitch, long long rows,
                        long long cols, int block, void* hip_stream) {
  const char* who = "fp8_quantize";
  if (rows <= 0 || cols <= 0) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: rows=%lld and cols=%lld must be positive", who, rows, cols);
  if (rows > (1LL << 22) || cols > (1LL << 22)) return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: at most 2^22 rows and columns, got %lld and %lld", who, rows, cols);
  if (!x || (!q && !qt) || !q != !q_scales || !qt != !qt_scales)
    return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: x and one of q, qt must not be NULL, each with its scales", who);
  if (!aligned16(x) || (q && (uintptr_t)q & (cols % 8 ? 0 : 7))) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: x must be 16-byte, q 8-byte aligned", who);
  if (qt && (!aligned16(qt) || qt_pitch % 16 || qt_pitch < rows))
    return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: qt must be 16-byte aligned, with a pitch (%lld) that is a multiple of 16 and holds %lld rows", who, qt_pitch, rows);
  const size_t groups_c = (size_t)ceil_div(cols, kGroup), groups_r = (size_t)ceil_div(rows, kGroup);
  const Range in = {"x", x, (size_t)rows * cols * 2};
  const Range outs[] = {{"q", q, (size_t)rows * cols}, {"q_scales", q_scales, (block ? groups_r : rows) * groups_c},
                        {"qt", qt, qt ? (size_t)(cols - 1) * qt_pitch + ceil_div(rows, 16) * 16 : 0}, {"qt_scales", qt_scales, (block ? groups_c : cols) * groups_r}};
  for (int i = 0; i < 4; ++i) {
    if (int rc = check_result(who, outs[i], {in})) return rc;
    for (int j = 0; j < i; ++j)
      if (int rc = check_result(who, outs[i], {outs[j]})) return rc;
  }
  const QuantParams p = {(const __bf16*)x, (uint8_t*)q, q_scales, (uint8_t*)qt, qt_scales, nullptr, rows, cols, qt_pitch};
  launch_quantize(p, block != 0, (hipStream_t)hip_stream);
  return launched(who);
}

int sparse_fp8_gemm(const void* a, const uint8_t* a_scales, int a_block, const void* b, const uint8_t* b_scales, int b_block, const void* bias,
                    void* out, int out_dtype, long long M, long long N, long long K, void* hip_stream) {
  const char* who = "fp8_gemm";
  if (int rc = check_product(who, M, N, K, out_dtype)) return rc;
  if (!a || !a_scales || !b || !b_scales || !out) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: a, b, their scales and out must not be NULL", who);
  if (!aligned16(a) || !aligned16(b)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: a and b must be 16-byte aligned", who);
  const int size = out_dtype == SPARSE_BLOCK_F32 ? 4 : 2, groups = (int)ceil_div(K, kGroup);
  if (int rc = check_elements(who, out, size, "out")) return rc;
  if (int rc = check_elements(who, bias, 2, "bias")) return rc;
  if (int rc = check_result(who, {"out", out, (size_t)M * N * size},
                            {{"a", a, (size_t)M * K}, {"b", b, (size_t)N * K}, {"bias", bias, (size_t)N * 2},
                             {"a_scales", a_scales, (size_t)(a_block ? ceil_div(M, kGroup) : M) * groups},
                             {"b_scales", b_scales, (size_t)(b_block ? ceil_div(N, kGroup) : N) * groups}}))
    return rc;
  const GemmParams p = {(const uint8_t*)a, a_scales, (const uint8_t*)b, b_scales, (const __bf16*)bias, out, M, N, K, K, (int)K, groups,
                        a_block ? 7 : 0, b_block ? 7 : 0, size == 4};
  const Route r = route_of(M, N, groups);
  sa_scratch scratch;
  if (const size_t need = scratch_of(M, N, groups))
    if (int rc = scratch.get(need, (hipStream_t)hip_stream)) return rc;
  return launch_gemm(who, p, r, (uint8_t*)scratch.data(), (hipStream_t)hip_stream);
}

int sparse_fp8_linear(const void* x, const void* w, const uint8_t* w_scales, const void* bias, void* out, int out_dtype, long long M, long long N,
                      long long K, void* hip_stream) {
  const char* who = "fp8_linear";
  if (int rc = check_product(who, M, N, K, out_dtype)) return rc;
  if (!x || !w || !w_scales || !out) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: x, w, w_scales and out must not be NULL", who);
  if (!aligned16(x) || !aligned16(w)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: x and w must be 16-byte aligned", who);
  const int size = out_dtype == SPARSE_BLOCK_F32 ? 4 : 2, groups = (int)ceil_div(K, kGroup);
  if (int rc = check_elements(who, out, size, "out")) return rc;
  if (int rc = check_elements(who, bias, 2, "bias")) return rc;
  if (int rc = check_result(who, {"out", out, (size_t)M * N * size},
                            {{"x", x, (size_t)M * K * 2}, {"w", w, (size_t)N * K}, {"bias", bias, (size_t)N * 2},
                             {"w_scales", w_scales, (size_t)ceil_div(N, kGroup) * groups}}))
    return rc;
  hipStream_t stream = (hipStream_t)hip_stream;
  sa_scratch scratch;
  const Route r = route_of(M, N, groups);
  const size_t held = rounded((size_t)M * K), scaled = rounded((size_t)M * groups);
  if (int rc = scratch.get(held + scaled + scratch_of(M, N, groups), stream)) return rc;
  uint8_t *x8 = (uint8_t*)scratch.data(), *xs = x8 + held;
  launch_quantize({(const __bf16*)x, x8, xs, nullptr, nullptr, nullptr, M, K, 0}, false, stream);
  const GemmParams p = {x8, xs, (const uint8_t*)w, w_scales, (const __bf16*)bias, out, M, N, K, K, (int)K, groups, 0, 7, size == 4};
  return launch_gemm(who, p, r, xs + scaled, stream);
}

int sparse_fp8_linear_backward(const void* dy, const void* x, const void* wt, const uint8_t* wt_scales, void* dx, void* dw, int dw_dtype,
                               float* dbias, long long M, long long N, long long K, void* hip_stream) {
  const char* who = "fp8_linear_backward";
  if (int rc = check_product(who, M, N, K, dw_dtype)) return rc;
  if (N % 16) return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: N=%lld must be a multiple of 16", who, N);
  if (!dy || (!dx && !dw && !dbias) || (dx && (!wt || !wt_scales)) || (dw && !x))
    return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: dy and a result must not be NULL, nor wt and wt_scales with dx, nor x with dw", who);
  if (!aligned16(dy) || (dx && !aligned16(wt)) || (dw && !aligned16(x))) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: dy, x and wt must be 16-byte aligned", who);
  const int size = dw_dtype == SPARSE_BLOCK_F32 ? 4 : 2;
  if (int rc = check_elements(who, dx, 2, "dx")) return rc;
  if (int rc = check_elements(who, dw, size, "dw")) return rc;
  if (int rc = check_elements(who, dbias, 4, "dbias")) return rc;
  const int groups_n = (int)ceil_div(N, kGroup), groups_m = (int)ceil_div(M, kGroup);
  const Range in_dy = {"dy", dy, (size_t)M * N * 2}, in_x = {"x", dw ? x : nullptr, (size_t)M * K * 2}, in_w = {"wt", dx ? wt : nullptr, (size_t)N * K},
              in_s = {"wt_scales", dx ? wt_scales : nullptr, (size_t)ceil_div(K, kGroup) * groups_n};
  const Range out_x = {"dx", dx, (size_t)M * K * 2}, out_w = {"dw", dw, (size_t)N * K * size}, out_b = {"dbias", dbias, (size_t)N * 4};
  if (int rc = check_result(who, out_x, {in_dy, in_x, in_w, in_s})) return rc;
  if (int rc = check_result(who, out_w, {in_dy, in_x, in_w, in_s, out_x})) return rc;
  if (int rc = check_result(who, out_b, {in_dy, in_x, in_w, in_s, out_x, out_w})) return rc;

  hipStream_t stream = (hipStream_t)hip_stream;
  const long long pitch = ceil_div(M, 16) * 16;
  const Route rx = route_of(M, K, groups_n), rw = route_of(N, K, groups_m);
  size_t need = 0;
  auto take = [&](bool want, size_t bytes) {
    const size_t at = need;
    if (want) need += rounded(bytes);
    return at;
  };
  const size_t at_dy = take(dx, (size_t)M * N), at_dys = take(dx, (size_t)M * groups_n), at_dyt = take(dw, (size_t)N * pitch),
               at_dyts = take(dw, (size_t)N * groups_m), at_xt = take(dw, (size_t)K * pitch), at_xts = take(dw, (size_t)K * groups_m),
               at_part = take(dbias, (size_t)groups_m * N * 4), at_x = take(dx, scratch_of(M, K, groups_n)), at_w = take(dw, scratch_of(N, K, groups_m));
  sa_scratch scratch;
  if (int rc = scratch.get(need, stream)) return rc;
  uint8_t* base = (uint8_t*)scratch.data();
  float* part = dbias ? (float*)(base + at_part) : nullptr;
  launch_quantize({(const __bf16*)dy, dx ? base + at_dy : nullptr, dx ? base + at_dys : nullptr, dw ? base + at_dyt : nullptr,
                   dw ? base + at_dyts : nullptr, part, M, N, pitch}, false, stream);
  if (dbias) hipLaunchKernelGGL(column_parts_kernel, dim3((unsigned)ceil_div(N, 64)), dim3(1024), 0, stream, part, (long long)groups_m, N, dbias);
  if (dx) {
    const GemmParams p = {base + at_dy, base + at_dys, (const uint8_t*)wt, wt_scales, nullptr, dx, M, K, N, N, (int)N, groups_n, 0, 7, 0};
    if (int rc = launch_gemm(who, p, rx, base + at_x, stream)) return rc;
  }
  if (dw) {
    launch_quantize({(const __bf16*)x, nullptr, nullptr, base + at_xt, base + at_xts, nullptr, M, K, pitch}, false, stream);
    const GemmParams p = {base + at_dyt, base + at_dyts, base + at_xt, base + at_xts, nullptr, dw, N, K, pitch, pitch, (int)pitch, groups_m, 0, 0, size == 4};
    if (int rc = launch_gemm(who, p, rw, base + at_w, stream)) return rc;
  }
  return launched(who);
}

}  // extern "C"
