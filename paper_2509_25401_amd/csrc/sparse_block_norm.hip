// Block norm: gated addition to the residual stream and modulated norm, forward and backward (include/sparse_block.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>

#include "sparse_attn.h"
#include "sparse_attn_internal.h"
#include "sparse_block.h"
#include "sparse_block_internal.h"

namespace {

using namespace sa_block;

constexpr int kMaxChannels = 16384;

// How the rows lie: whole units on 16 bytes; or from any element on, where the last unit of a row may have fewer channels.  Its
// thread then either reads the row's last eight channels and moves those that are its own to their places, so that no load stands
// under a condition and waits for the one before; or reads its channels one by one, the others' runs standing under the condition.
enum Rows { kWhole, kTailMoved, kTailApart };

// Where the values of a row lie among the threads that share it: unit u of thread t is eight consecutive channels.
template <Rows ROWS>
struct Place {
  int t, threads, C;
  __device__ __forceinline__ int channel(int u, int e) const { return (u * threads + t) * 8 + e; }
  __device__ __forceinline__ bool has(int u, int e) const { return channel(u, ROWS == kWhole ? 0 : e) < C; }
  // Behind Unit::load(), before the first use: values of channels that do not exist become zeros.  The last unit of a row holds the
  // row's last eight channels until then, and moves down those that are its own.
  template <class... F>
  __device__ __forceinline__ void settle(int u, F&... f) const {
    if constexpr (ROWS == kTailMoved) {
      if (has(u, 7)) return;
      const int away = has(u, 0) && C >= 8 ? 8 - (C & 7) : 0;
#pragma unroll
      for (int by = 1; by < 8; by *= 2)
        if (away & by) {
#pragma unroll
          for (int e = 0; e + by < 8; ++e) ((f[e] = f[e + by]), ...);
        }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (!has(u, e)) ((f[e] = 0.f), ...);
    }
  }
};

template <class T, Rows ROWS>
struct Unit {
  Pack8<T> v;
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int e = 0; e < 8; ++e) v.set(e, 0.f);
  }
  template <bool ONCE>
  __device__ __forceinline__ void load(const T* row, const Place<ROWS>& p, int u) {
    if constexpr (ROWS == kWhole) {
      if (!p.has(u, 0)) return zero();
      if (ONCE)
        v.load_once(row + p.channel(u, 0));
      else
        v.load(row + p.channel(u, 0));
    } else if constexpr (ROWS == kTailApart) {
      if (p.has(u, 7)) {
        v.load_any(row + p.channel(u, 0));
      } else if (p.has(u, 0)) {
        T one[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) one[e] = row[min(p.channel(u, e), p.C - 1)];     // all on their way together
#pragma unroll
        for (int e = 0; e < 8; ++e) v.set(e, p.has(u, e) ? (float)one[e] : 0.f);
      } else {
        zero();
      }
    } else if (p.C >= 8) {
      v.load_any(row + min(p.channel(u, 0), p.C - 8));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v.set(e, (float)row[min(p.channel(u, e), p.C - 1)]);
    }
  }
  __device__ __forceinline__ void store(T* row, const Place<ROWS>& p, int u) const {
    if constexpr (ROWS == kWhole) {
      if (p.has(u, 0)) v.store_once(row + p.channel(u, 0));
    } else if (p.has(u, 7)) {
      v.store_any(row + p.channel(u, 0));          // through the cache: rows share its lines
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (p.has(u, e)) row[p.channel(u, e)] = (T)v.get(e);
    }
  }
  __device__ __forceinline__ float get(int e) const { return v.get(e); }
  __device__ __forceinline__ void set(int e, float f) { v.set(e, f); }
};

// Sums over the threads of a row: the wave's own, then across the waves through LDS.  Consecutive calls of a kernel take
// turns between two slots, so that one barrier per call is enough.
template <bool ONE, int N>
struct RowSum {
  float (*slot)[16][N];     // [2][wave][value]
  int wave, waves, turn = 0;
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
    if (ONE || waves == 1) return;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) slot[turn][wave][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float s = 0.f;
      for (int w = 0; w < waves; ++w) s += slot[turn][w][k];
      v[k] = s;
    }
    turn ^= 1;
  }
};

struct NormParams {
  const void *x, *y, *weight, *scale, *shift, *gate, *post_weight;
  void *x_out, *h;
  uint8_t* h_scales;
  long long rows, rows_per_vector, scale_stride, shift_stride, gate_stride;
  int C, layer;
  float alpha, eps, post_eps;
};

// One pass per row: x (and y) are read once, stay in registers through the reductions, x' and h are written once.  Bound by the
// memory: 33024 x 3072 bf16 with y, gate, scale and shift 150 us, 5.4 TB/s; with float32 x 223 us, 5.5 TB/s; 17 x 3072 3.7 us.
// 9001 x 3073 69 us, 3.2 TB/s: its rows' 16-byte accesses straddle lines and its stores go through the cache; how much of it either
// costs has not been measured.  All sums and all values in between are float32; what is rounded are
// the results: x' to its type, and h, which is of the x' before that, to bf16 or to its e4m3 form.
// ONE: a wave per row, four rows per workgroup, no barrier; else all waves of the workgroup share a row.
template <class TX, class TV, int NV, bool VEC, bool ONE, bool F8>
__global__ void __launch_bounds__(ONE ? 256 : 1024) block_norm_kernel(const NormParams p) {
  // us, tail moved / apart.  Eight units to a thread of one wave: bf16 9001 x 3073 84.5 / 69.0, float32 11776 x 2109 122.6 / 108.5.  One
  // unit to a thread of several waves: 9001 x 4099 108.7 / 96.8, 9001 x 7001 196 / 182, 300 x 7001 11.4 / 10.0, but 1500 x 4001 16.0 /
  // 17.3.  Else moved: 40000 x 333 43.5 / 47.8, 30000 x 1001 54.4 / 60.6, 18002 x 2001 67.3 / 72.7 (though 18002 x 1161 61.0 / 56.4),
  // 9001 x 9001 177 / 182 (though 9001 x 16001 315 / 301).
  constexpr Rows ROWS = VEC ? kWhole : (ONE ? NV == 8 : NV == 1) ? kTailApart : kTailMoved;
  __shared__ float slots[2][16][1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long row = ONE ? block_of() * 4 + wave : block_of();
  if (row >= p.rows) return;                                  // whole waves, and without ONE whole workgroups; with it no barrier follows
  const Place<ROWS> at{ONE ? lane : (int)threadIdx.x, ONE ? 64 : (int)blockDim.x, p.C};
  RowSum<ONE, 1> sum{slots, wave, (int)blockDim.x >> 6};
  const float inv_c = 1.f / (float)p.C;
  const long long g = row / p.rows_per_vector;
  const TX* x = (const TX*)p.x + row * p.C;

  float v[NV][8];
  Unit<TX, ROWS> xu[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) xu[u].template load<true>(x, at, u);
  if (p.y) {
    const __bf16* y = (const __bf16*)p.y + row * p.C;
    const TV* gate = p.gate ? (const TV*)p.gate + g * p.gate_stride : nullptr;
    const TV* wp = (const TV*)p.post_weight;
    Unit<__bf16, ROWS> yu[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) yu[u].template load<true>(y, at, u);
    float rp = 1.f;
    if (wp) {
      float s[1] = {0.f};
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = yu[u].get(e);
        at.settle(u, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] = fmaf(f[e], f[e], s[0]);
      }
      sum(s);
      rp = 1.f / sqrtf(s[0] * inv_c + p.post_eps);
    }
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      Unit<TV, ROWS> gu, wu;
      if (gate) gu.template load<false>(gate, at, u);
      if (wp) wu.template load<false>(wp, at, u);
      Unit<TX, ROWS> o;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float t = yu[u].get(e) * rp;
        if (wp) t *= wu.get(e);
        if (gate) t *= gu.get(e);
        v[u][e] = fmaf(p.alpha, xu[u].get(e), t);
      }
      at.settle(u, v[u]);
#pragma unroll
      for (int e = 0; e < 8; ++e) o.set(e, v[u][e]);
      o.store((TX*)p.x_out + row * p.C, at, u);
    }
  } else {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] = p.alpha * xu[u].get(e);
      at.settle(u, v[u]);
    }
  }
  if (!p.h) return;

  float mean = 0.f;
  if (p.layer) {
    float s[1] = {0.f};
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += v[u][e];            // channels that do not exist hold zeros
    sum(s);
    mean = s[0] * inv_c;
  }
  float s[1] = {0.f};
#pragma unroll
  for (int u = 0; u < NV; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[u][e] -= mean;
      if (at.has(u, e)) s[0] = fmaf(v[u][e], v[u][e], s[0]);
    }
  sum(s);
  const float r = 1.f / sqrtf(s[0] * inv_c + p.eps);
  const TV* w = (const TV*)p.weight;
  const TV* scale = p.scale ? (const TV*)p.scale + g * p.scale_stride : nullptr;
  const TV* shift = p.shift ? (const TV*)p.shift + g * p.shift_stride : nullptr;
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    Unit<TV, ROWS> wu, su, bu;
    if (w) wu.template load<false>(w, at, u);
    if (scale) su.template load<false>(scale, at, u);
    if (shift) bu.template load<false>(shift, at, u);
    float up[8], add[8], h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      up[e] = w ? wu.get(e) : 1.f;
      if (scale) up[e] *= 1.f + su.get(e);
      add[e] = shift ? bu.get(e) : 0.f;
    }
    at.settle(u, up, add);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = fmaf(v[u][e] * r, up[e], add[e]);
    if constexpr (F8) {
      // 128 channels are 16 neighbouring lanes of one unit
      const bool has = at.has(u, 0);
      float amax = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, has ? finite_abs(h[e]) : 0.f);
      const int ex = e4m3_exponent(group16_max(amax));
      const float down = power_of_two(-ex);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = e4m3_input(h[e] * down);
      if (has) {
        const int c = at.channel(u, 0);
        int2 q;
        q.x = e4m3x4(h[0], h[1], h[2], h[3]);
        q.y = e4m3x4(h[4], h[5], h[6], h[7]);
        *(int2*)((uint8_t*)p.h + row * p.C + c) = q;
        if ((lane & 15) == 0) p.h_scales[row * ((p.C + 127) / 128) + c / 128] = (uint8_t)(ex + 127);
      }
    } else {
      Unit<__bf16, ROWS> o;
#pragma unroll
      for (int e = 0; e < 8; ++e) o.set(e, h[e]);
      o.store((__bf16*)p.h + row * p.C, at, u);
    }
  }
}

// ---------------------------------------------------------------------------------------
// Backward.  With n the normalised row, m = y / rms(y) (y without a post norm), u = weight (1 + scale):
//     dn  = dh u;                dx' = dx_out + r (dn - [mean(dn)] - n mean(dn n))          ([]: layer norm only)
//     dm  = dx' gate post_weight;  dy = rp (dm - m mean(dm m))                              (dm without a post norm)
// and the sums over the rows of a vector g:  A = sum dh n,  E = sum dx' m,  S = sum dh, from which
//     dshift = S, dscale = weight A, dgate = post_weight E, dweight = sum_g (1 + scale_g) A_g, dpost = sum_g gate_g E_g.
// So three sums are kept per channel, in registers: a workgroup walks over a chunk of the rows of one vector with every
// thread at its own channels, and writes its sums once; a second kernel adds the chunks in order.
// ---------------------------------------------------------------------------------------
struct BackParams {
  const void *dh, *dx_out, *x, *y, *weight, *scale, *gate, *post_weight;
  void *dx, *dy;
  float* part[3];         // S, A, E, each [vectors * chunks][C], or NULL where nobody asks for it
  long long rows, rows_per_vector, vectors, scale_stride, gate_stride;
  int C, layer, chunks, rows_per_chunk, row_waves;
  float alpha, eps, post_eps;
};

// What bounds it beside the memory is that the sums of a row have to be known before its results: one trip through LDS and a
// barrier for each row (two of them with a post norm), while the next two rows are on their way.  A workgroup
// is as many teams of waves as make twelve, each with a chunk of its own: the register file holds three waves on each SIMD, and
// workgroups of six waves, which the SIMDs get as 2, 2, 1, 1, left half of it empty.  Each wave sums around its own
// mean and the waves' sums are put together for the row's mean: with wave w's n_w channels, mean m_w and d_w = m_w - mean,
//     sum (x - mean)^2 = sum_w [ sum (x - m_w)^2 + n_w d_w^2 ],   sum dn (x - mean) = sum_w [ sum dn (x - m_w) + d_w sum dn ].
// 33024 x 3072 bf16 in 16 vectors, with y and dx_out: 253 us, 4.8 TB/s of the six tensors; 9001 x 3072 80 us, 4.1 TB/s; 512 x 3072
// 24 us, mostly the way to the first row and the sums'.  18002 x 1160 with a post norm 75 us, 3.3 TB/s: three waves to a row, the
// last with 17 lanes of work, and two barriers; there the vector instructions bound it.  Rows at any alignment (9001 x 3073, 98 us)
// keep one row on its way instead of two, and even so hold 26 to 42 registers' worth in scratch memory (with the tail apart 10 to 20, and
// 142 us); so do whole rows of more than 6144 channels, 6 to 28 (4000 x 7000 93 us, 3.6 TB/s), and far more beyond 8192.  Sums and values in between are float32; dx and dy are
// rounded once, to their types.
template <class TX, class TV, int NV, bool VEC, int THREADS>
__global__ void __launch_bounds__(THREADS) block_norm_backward_kernel(const BackParams p) {
  constexpr Rows ROWS = VEC ? kWhole : kTailMoved;
  __shared__ __attribute__((aligned(16))) float slots[2][16][4];
  __shared__ float post_slots[2][16][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = p.row_waves, l16 = lane & 15;
  const int team = wave / waves, base = team * waves;          // the team's first wave
  const Place<ROWS> at{(int)threadIdx.x - base * 64, waves * 64, p.C};
  const float inv_c = 1.f / (float)p.C;
  const long long chunk = block_of() * (blockDim.x / 64 / waves) + team, all = p.vectors * p.chunks;
  const long long g = min(chunk, all - 1) / p.chunks;
  const long long first = g * p.rows_per_vector + (min(chunk, all - 1) % p.chunks) * p.rows_per_chunk;
  const long long end_g = min(p.rows, (g + 1) * p.rows_per_vector);
  const long long end = chunk < all ? min(end_g, first + p.rows_per_chunk) : first;      // a team without a chunk goes along
  const bool post = p.post_weight != nullptr, with_y = p.y != nullptr;

  constexpr int kAhead = VEC ? 2 : 1;          // rows on their way
  struct Row {
    Unit<TX, ROWS> x[NV], dxo[NV];
    Unit<__bf16, ROWS> dh[NV], y[NV];
  } buffer[kAhead];
  auto load = [&](Row& b, long long row) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      b.x[u].template load<true>((const TX*)p.x + row * p.C, at, u);
      b.dh[u].template load<true>((const __bf16*)p.dh + row * p.C, at, u);
      if (p.dx_out)
        b.dxo[u].template load<true>((const TX*)p.dx_out + row * p.C, at, u);
      else
        b.dxo[u].zero();
      if (with_y)
        b.y[u].template load<true>((const __bf16*)p.y + row * p.C, at, u);
      else
        b.y[u].zero();
    }
  };
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (first + k < end) load(buffer[k], first + k);

  float up[NV][8], gp[NV][8];                  // weight (1 + scale), gate post_weight
  float count = 0.f;
  {
    // all on their way before the first is used
    Unit<TV, ROWS> w[NV], sc[NV], ga[NV], pw[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (p.weight) w[u].template load<false>((const TV*)p.weight, at, u);
      if (p.scale) sc[u].template load<false>((const TV*)p.scale + g * p.scale_stride, at, u);
      if (p.gate) ga[u].template load<false>((const TV*)p.gate + g * p.gate_stride, at, u);
      if (post) pw[u].template load<false>((const TV*)p.post_weight, at, u);
    }
#pragma unroll
    for (int u = 0; u < NV; ++u) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        up[u][e] = (p.weight ? w[u].get(e) : 1.f) * (p.scale ? 1.f + sc[u].get(e) : 1.f);
        gp[u][e] = (p.gate ? ga[u].get(e) : 1.f) * (post ? pw[u].get(e) : 1.f);
        count += at.has(u, e) ? 1.f : 0.f;
      }
      at.settle(u, up[u], gp[u]);
    }
  }
  count = wave_sum(count);                     // channels of this wave
  if (lane == 0) post_slots[0][wave][0] = count;
  __syncthreads();
  const float n_w = l16 < waves ? post_slots[0][base + l16][0] : 0.f;       // of the team's wave l16
  __syncthreads();
  const float inv_count = count > 0.f ? 1.f / count : 0.f, inv_n_w = n_w > 0.f ? 1.f / n_w : 0.f;
  float S[NV][8] = {}, A[NV][8] = {}, E[NV][8] = {};

  int turn = 0;
  auto process = [&](Row& b, long long row) __attribute__((always_inline)) {
    float n[NV][8], d[NV][8], yf[NV][8], o[NV][8];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[u][e] = b.x[u].get(e);
        d[u][e] = b.dh[u].get(e);
        o[u][e] = b.dxo[u].get(e);
        yf[u][e] = b.y[u].get(e);
      }
      at.settle(u, n[u], d[u], o[u], yf[u]);
    }
    if (row + kAhead < end) load(b, row + kAhead);
    float sum_x = 0.f, m_w = 0.f;
    if (p.layer) {
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum_x += n[u][e];          // channels that do not exist hold zeros
      sum_x = wave_sum(sum_x);
      m_w = sum_x * inv_count;
    }
    float sq = 0.f, sd = 0.f, sdn = 0.f, sy = 0.f;
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = at.has(u, e) ? n[u][e] - m_w : 0.f, dn = d[u][e] * up[u][e];
        sq = fmaf(v, v, sq);
        sd += dn;
        sdn = fmaf(dn, v, sdn);
        sy = fmaf(yf[u][e], yf[u][e], sy);
      }
    sq = wave_sum(sq);
    sdn = wave_sum(sdn);
    sd = p.layer ? wave_sum(sd) : 0.f;
    if (post) sy = wave_sum(sy);
    if (lane == 0) {
      *(f32x4*)slots[turn][wave] = f32x4{sum_x, sq, sd, sdn};
      if (post) post_slots[turn][wave][0] = sy;
    }
    __syncthreads();
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (l16 < waves) v = *(const f32x4*)slots[turn][base + l16];
    const float mean = p.layer ? group_sum<16>(v[0]) * inv_c : 0.f;
    const float away = p.layer ? v[0] * inv_n_w - mean : 0.f;
    const float r = 1.f / sqrtf(group_sum<16>(fmaf(n_w * away, away, v[1])) * inv_c + p.eps);
    const float mean_dnn = group_sum<16>(fmaf(v[2], away, v[3])) * r * inv_c;
    const float mean_dn = p.layer ? group_sum<16>(v[2]) * inv_c : 0.f;
    float rp = 1.f;
    if (post) rp = 1.f / sqrtf(group_sum<16>(l16 < waves ? post_slots[turn][base + l16][0] : 0.f) * inv_c + p.post_eps);
    float dot = 0.f;
    if (row < end) {
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float nn = at.has(u, e) ? (n[u][e] - mean) * r : 0.f, dn = d[u][e];
          o[u][e] += r * (dn * up[u][e] - mean_dn - nn * mean_dnn);
          yf[u][e] *= rp;
          S[u][e] += dn;
          A[u][e] = fmaf(dn, nn, A[u][e]);
          E[u][e] = fmaf(o[u][e], yf[u][e], E[u][e]);
          dot = fmaf(o[u][e] * gp[u][e], yf[u][e], dot);
        }
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        Unit<TX, ROWS> r8;
#pragma unroll
        for (int e = 0; e < 8; ++e) r8.set(e, p.alpha * o[u][e]);
        r8.store((TX*)p.dx + row * p.C, at, u);
      }
    }
    if (p.dy) {
      float mean_dmm = 0.f;
      if (post) {
        dot = wave_sum(dot);
        if (lane == 0) post_slots[turn][wave][1] = dot;
        __syncthreads();
        mean_dmm = group_sum<16>(l16 < waves ? post_slots[turn][base + l16][1] : 0.f) * inv_c;
      }
      if (row < end) {
#pragma unroll
        for (int u = 0; u < NV; ++u) {
          Unit<__bf16, ROWS> r8;
#pragma unroll
          for (int e = 0; e < 8; ++e) r8.set(e, rp * (o[u][e] * gp[u][e] - yf[u][e] * mean_dmm));
          r8.store((__bf16*)p.dy + row * p.C, at, u);
        }
      }
    }
    turn ^= 1;                                 // the other slots: written again behind the next barrier, read in front of it
  };
  // every team makes as many turns as the longest chunk has rows: the barriers are the workgroup's
  for (long long i = 0; i < p.rows_per_chunk; i += kAhead)
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + k < p.rows_per_chunk) process(buffer[k], first + i + k);
  if (chunk >= all) return;
  auto store = [&](float* to, const float (&v)[NV][8]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < NV; ++u)
      if (at.has(u, 7)) {
        *(any_f32x4*)(to + at.channel(u, 0)) = f32x4{v[u][0], v[u][1], v[u][2], v[u][3]};
        *(any_f32x4*)(to + at.channel(u, 4)) = f32x4{v[u][4], v[u][5], v[u][6], v[u][7]};
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at.has(u, e)) to[at.channel(u, e)] = v[u][e];
      }
  };
  const size_t own = (size_t)chunk * p.C;
  if (p.part[0]) store(p.part[0] + own, S);
  if (p.part[1]) store(p.part[1] + own, A);
  if (p.part[2]) store(p.part[2] + own, E);
}

// Sums of the chunks of a vector, a column to a thread, in their order but kAtOnce strands at a time so that the loads overlap.
// Where there are more than kFold of them, a first pass folds runs of kFold into one: 5 us for 512 chunks of 3072 channels, and
// 5 for the rest; one pass over all of them 40 us.
struct FinishParams {
  const float* part[3];   // S, A, E, each [vectors * chunks][C]; what nobody asks for is one of the others
  float* folded[3];       // each [vectors * runs][C], or NULL
  const void *weight, *scale, *gate, *post_weight;
  float *dscale, *dshift, *dgate;
  float *wa, *we;         // [vectors][C]: what dweight and dpost_weight are the sums of (the results themselves with one vector), or NULL
  long long vectors, scale_stride, gate_stride;
  int C, chunks;
};

constexpr int kFold = 32;

// Sums of n >= 1 rows of `pitch` floats, from column `at` of N planes.  Loads are not put under conditions, which would make each
// wait for the one before: rows past the end repeat the last one.
template <int N>
__device__ __forceinline__ void column_sums(const float* const (&p)[N], size_t at, long long n, size_t pitch, float (&out)[N]) {
  constexpr int kAtOnce = 8;
  float s[kAtOnce][N] = {};
  for (long long i = 0; i < n; i += kAtOnce) {
    float v[kAtOnce][N];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
      for (int a = 0; a < N; ++a) v[k][a] = p[a][at + min(i + k, n - 1) * pitch];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
      for (int a = 0; a < N; ++a) s[k][a] += i + k < n ? v[k][a] : 0.f;
  }
#pragma unroll
  for (int a = 0; a < N; ++a) out[a] = ((s[0][a] + s[1][a]) + (s[2][a] + s[3][a])) + ((s[4][a] + s[5][a]) + (s[6][a] + s[7][a]));
}

__global__ void __launch_bounds__(256) block_norm_fold_kernel(const FinishParams p) {
  const int c = blockIdx.x * 256 + threadIdx.x, run = blockIdx.z, runs = gridDim.z;
  if (c >= p.C) return;
  for (long long g = blockIdx.y; g < p.vectors; g += gridDim.y) {
    float s[3];
    column_sums(p.part, ((size_t)g * p.chunks + run * kFold) * p.C + c, min(kFold, p.chunks - run * kFold), p.C, s);
#pragma unroll
    for (int a = 0; a < 3; ++a)
      if (p.folded[a]) p.folded[a][((size_t)g * runs + run) * p.C + c] = s[a];
  }
}

template <class TV>
__global__ void __launch_bounds__(256) block_norm_finish_kernel(const FinishParams p) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= p.C) return;
  for (long long g = blockIdx.y; g < p.vectors; g += gridDim.y) {
    float s[3];
    column_sums(p.part, (size_t)g * p.chunks * p.C + c, p.chunks, p.C, s);
    const long long at = g * p.C + c;
    // with one chunk to a vector these may be the results' own places, where they stay if no factor follows
    if (p.dshift && p.dshift != p.part[0]) p.dshift[at] = s[0];
    if (p.dscale && (p.weight || p.dscale != p.part[1])) p.dscale[at] = p.weight ? s[1] * (float)((const TV*)p.weight)[c] : s[1];
    if (p.wa) p.wa[at] = p.scale ? s[1] * (1.f + (float)((const TV*)p.scale)[g * p.scale_stride + c]) : s[1];
    if (p.dgate && (p.post_weight || p.dgate != p.part[2])) p.dgate[at] = p.post_weight ? s[2] * (float)((const TV*)p.post_weight)[c] : s[2];
    if (p.we) p.we[at] = p.gate ? s[2] * (float)((const TV*)p.gate)[g * p.gate_stride + c] : s[2];
  }
}

// wa, we [n][C]: what the two weights' gradients are the sums of; 64 columns and sixteen shares of the vectors to a workgroup
__global__ void __launch_bounds__(1024) column_sum_kernel(const float* wa, const float* we, float* dweight, float* dpost, long long n, int C) {
  __shared__ float red[16][2][64];
  const int lane = threadIdx.x & 63, share = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  const long long per = (n + 15) / 16, first = share * per, count = min(per, n - first);
  float s[2] = {0.f, 0.f};
  const float* const part[2] = {wa, we};
  if (c < C && count > 0) column_sums(part, first * C + c, count, C, s);
  red[share][0][lane] = s[0];
  red[share][1][lane] = s[1];
  __syncthreads();
  if (share || c >= C) return;
  s[0] = s[1] = 0.f;
  for (int i = 0; i < 16; ++i) {
    s[0] += red[i][0][lane];
    s[1] += red[i][1][lane];
  }
  if (dweight) dweight[c] = s[0];
  if (dpost) dpost[c] = s[1];
}

// ---------------------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------------------
size_t type_size(int t) { return t == SPARSE_BLOCK_F32 ? 4 : t == SPARSE_BLOCK_E4M3 ? 1 : 2; }

int launched(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? 0 : sa_fail(SPARSE_ATTN_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
}

int check_sizes(const char* who, long long rows, long long rows_per_vector, int C, int norm, int x_dtype, int vector_dtype,
                float alpha, float eps, float post_eps) {
  if (rows <= 0 || C <= 0 || rows_per_vector <= 0)
    return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: rows=%lld, channels=%d and rows_per_vector=%lld must be positive", who, rows, C, rows_per_vector);
  if (C > kMaxChannels || rows > 0x7fffffffLL)
    return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: at most %d channels and 2^31 - 1 rows, got %d and %lld", who, kMaxChannels, C, rows);
  if (norm != SPARSE_BLOCK_NORM_RMS && norm != SPARSE_BLOCK_NORM_LAYER)
    return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: norm=%d is none of SPARSE_BLOCK_NORM_*", who, norm);
  if ((x_dtype != SPARSE_BLOCK_BF16 && x_dtype != SPARSE_BLOCK_F32) || (vector_dtype != SPARSE_BLOCK_BF16 && vector_dtype != SPARSE_BLOCK_F32))
    return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: x_dtype=%d and vector_dtype=%d must be BF16 or F32", who, x_dtype, vector_dtype);
  if (!finite_nonnegative(eps) || !finite_nonnegative(post_eps) || alpha - alpha != 0.f)
    return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: eps and post_eps must be finite and >= 0, alpha finite", who);
  return 0;
}

struct Range {
  const char* name;
  const void* p;
  size_t bytes;
};
// every `out` against every `in` and every other `out`; results may share an address with the input `same` (in place)
int check_overlaps(const char* who, const Range* outs, int n_out, const Range* ins, int n_in, const void* same, const void* same_out) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (overlap(outs[i].p, outs[i].bytes, ins[j].p, ins[j].bytes) && !(ins[j].p == same && outs[i].p == same && same == same_out))
        return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: %s must not overlap %s", who, outs[i].name, ins[j].name);
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes))
        return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: %s must not overlap %s", who, outs[i].name, outs[j].name);
  }
  return 0;
}

int check_elements(const char* who, std::initializer_list<const void*> tensors, size_t size) {
  for (const void* p : tensors)
    if ((uintptr_t)p & (size - 1)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: tensors must be aligned to their elements", who);
  return 0;
}

template <class TX, class TV>
void launch_norm(const NormParams& p, bool vec, bool f8, hipStream_t stream) {
  const int vectors = (p.C + 7) / 8;
  // A wave per row needs no barrier and keeps many rows in flight; a row's threads are spread over more waves where a
  // wave would hold more than eight units, and for few rows, where a row's own time is the call's.  One wave against more, us,
  // C 3072: 17 rows 8.3 / 3.7, 512 rows 9.1 / 5.4, 1126 rows 10.3 / 8.1, 2000 rows 10.8 / 12.7, 33024 rows 156 / 162.
  const bool one = vectors <= 512 && (p.rows >= 1536 || vectors <= 64);
  auto go = [&](auto nv, auto v, auto o, auto f) {
    constexpr int NV = decltype(nv)::value;
    constexpr bool VEC = decltype(v)::value, ONE = decltype(o)::value, F8 = decltype(f)::value;
    if constexpr (!(F8 && !VEC)) {
      const unsigned block = ONE ? 256 : 64 * ((vectors + 64 * NV - 1) / (64 * NV));
      hipLaunchKernelGGL((block_norm_kernel<TX, TV, NV, VEC, ONE, F8>), grid_of(ONE ? (p.rows + 3) / 4 : p.rows), dim3(block), 0, stream, p);
    }
  };
  using T = std::true_type;
  using F = std::false_type;
  auto units = [&](auto v, auto f) {
    if (one) {
      if (vectors <= 64) go(std::integral_constant<int, 1>{}, v, T{}, f);
      else if (vectors <= 128) go(std::integral_constant<int, 2>{}, v, T{}, f);
      else if (vectors <= 256) go(std::integral_constant<int, 4>{}, v, T{}, f);
      else go(std::integral_constant<int, 8>{}, v, T{}, f);
    } else if (vectors <= 1024) go(std::integral_constant<int, 1>{}, v, F{}, f);
    else go(std::integral_constant<int, 2>{}, v, F{}, f);
  };
  if (f8) units(T{}, T{});
  else if (vec) units(T{}, F{});
  else units(F{}, F{});
}

int row_waves(int C) { return C <= 8192 ? (C + 511) / 512 : (C + 1023) / 1024; }     // of the backward kernel: one or two units a thread
int teams_of(int waves) { return waves <= 12 ? 12 / waves : 1; }

template <class TX, class TV>
void launch_backward(BackParams& p, bool vec, hipStream_t stream) {
  p.row_waves = row_waves(p.C);
  const int teams = teams_of(p.row_waves);
  const dim3 grid = grid_of((p.vectors * p.chunks + teams - 1) / teams);
  const unsigned block = 64 * teams * p.row_waves;
  auto go = [&](auto nv, auto v, auto threads) {
    constexpr int NV = decltype(nv)::value, THREADS = decltype(threads)::value;
    constexpr bool VEC = decltype(v)::value;
    hipLaunchKernelGGL((block_norm_backward_kernel<TX, TV, NV, VEC, THREADS>), grid, dim3(block), 0, stream, p);
  };
  using T = std::true_type;
  using F = std::false_type;
  using N1 = std::integral_constant<int, 1>;
  using N2 = std::integral_constant<int, 2>;
  using Twelve = std::integral_constant<int, 768>;
  using Full = std::integral_constant<int, 1024>;
  if (p.C > 8192) vec ? go(N2{}, T{}, Full{}) : go(N2{}, F{}, Full{});
  else if (p.row_waves > 12) vec ? go(N1{}, T{}, Full{}) : go(N1{}, F{}, Full{});
  else vec ? go(N1{}, T{}, Twelve{}) : go(N1{}, F{}, Twelve{});
}

// Chunks of a vector's rows: their teams run in rounds of as many as fit the chip, and each has about six rows' worth of
// work of its own (vectors to read, sums to write and to add up): the number with the shortest rounds.  33024 x 3072 in 129
// vectors 275 us; with chunks for one round of all slots, whatever is left over, 408, and without the six rows 1263.
struct ChunkPlan {
  int chunks, rows;
};
ChunkPlan chunks_of(long long rpv, long long vectors, int C) {
  const long long slots = 256 * teams_of(row_waves(C));
  long long best = 1LL << 62;
  ChunkPlan plan = {1, (int)rpv};
  for (long long n = 1; n <= 1024 && n <= rpv; ++n) {
    const long long per = (rpv + n - 1) / n, cost = (vectors * n + slots - 1) / slots * (per + 6);
    if (cost < best) best = cost, plan = {(int)((rpv + per - 1) / per), (int)per};
  }
  return plan;
}

template <class F>
void by_types(int x_dtype, int vector_dtype, F&& f) {
  if (x_dtype == SPARSE_BLOCK_F32)
    vector_dtype == SPARSE_BLOCK_F32 ? f(float{}, float{}) : f(float{}, __bf16{});
  else
    vector_dtype == SPARSE_BLOCK_F32 ? f(__bf16{}, float{}) : f(__bf16{}, __bf16{});
}

}  // namespace

extern "C" {

int sparse_block_norm(const sparse_block_norm_args* a, void* hip_stream) {
  const char* who = "block_norm";
  if (!a) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: args must not be NULL", who);
  if (int rc = check_sizes(who, a->rows, a->rows_per_vector, a->channels, a->norm, a->x_dtype, a->vector_dtype, a->alpha, a->eps, a->post_eps)) return rc;
  const bool f8 = a->h && a->h_dtype == SPARSE_BLOCK_E4M3;
  if (a->h && !f8 && a->h_dtype != SPARSE_BLOCK_BF16)
    return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: h_dtype=%d must be BF16 or E4M3", who, a->h_dtype);
  if (!a->x || (a->y && !a->x_out) || (!a->y && !a->h)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: x, x_out (with y) and h or y must not be NULL", who);
  if (!a->y && (a->post_weight || a->gate)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: gate and post_weight need y", who);
  if (f8 != (a->h_scales != nullptr)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: h_scales goes with an E4M3 h", who);
  const long long vectors = (a->rows - 1) / a->rows_per_vector + 1;
  if (a->scale_stride < 0 || a->shift_stride < 0 || a->gate_stride < 0) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: strides must not be negative", who);
  const size_t n = (size_t)a->rows * a->channels, xs = type_size(a->x_dtype), vs = type_size(a->vector_dtype);
  auto vec_bytes = [&](long long stride) { return ((size_t)(vectors - 1) * stride + a->channels) * vs; };
  const Range outs[] = {{"x_out", a->y ? a->x_out : nullptr, n * xs}, {"h", a->h, n * (f8 ? 1 : 2)},
                        {"h_scales", a->h_scales, (size_t)a->rows * ((a->channels + 127) / 128)}};
  const Range ins[] = {{"x", a->x, n * xs}, {"y", a->y, n * 2}, {"weight", a->weight, (size_t)a->channels * vs},
                       {"post_weight", a->post_weight, (size_t)a->channels * vs}, {"scale", a->scale, vec_bytes(a->scale_stride)},
                       {"shift", a->shift, vec_bytes(a->shift_stride)}, {"gate", a->gate, vec_bytes(a->gate_stride)}};
  if (int rc = check_overlaps(who, outs, 3, ins, 7, a->x, a->x_out)) return rc;
  if (int rc = check_elements(who, {a->x, a->x_out}, xs)) return rc;
  if (int rc = check_elements(who, {a->y, f8 ? nullptr : a->h}, 2)) return rc;
  if (int rc = check_elements(who, {a->weight, a->post_weight, a->scale, a->shift, a->gate}, vs)) return rc;
  bool vec = a->channels % 8 == 0 && aligned16(a->x) && aligned16(a->x_out) && aligned16(a->y) && aligned16(a->weight) &&
             aligned16(a->post_weight) && aligned16(a->scale) && aligned16(a->shift) && aligned16(a->gate) &&
             (a->scale_stride | a->shift_stride | a->gate_stride) % 8 == 0;
  if (f8 && (!vec || a->channels % 16 || ((uintptr_t)a->h & 7)))
    return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: an E4M3 h needs a multiple of 16 channels and 16-byte aligned tensors and strides", who);
  vec = vec && (f8 || aligned16(a->h));
  NormParams p = {a->x, a->y, a->weight, a->scale, a->shift, a->gate, a->post_weight, a->x_out, a->h, a->h_scales, a->rows,
                  a->rows_per_vector, a->scale_stride, a->shift_stride, a->gate_stride, a->channels,
                  a->norm == SPARSE_BLOCK_NORM_LAYER, a->y ? a->alpha : 1.f, a->eps, a->post_eps};
  by_types(a->x_dtype, a->vector_dtype, [&](auto tx, auto tv) { launch_norm<decltype(tx), decltype(tv)>(p, vec, f8, (hipStream_t)hip_stream); });
  return launched(who);
}

int sparse_block_norm_backward(const sparse_block_norm_backward_args* a, void* hip_stream) {
  const char* who = "block_norm_backward";
  if (!a) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: args must not be NULL", who);
  if (int rc = check_sizes(who, a->rows, a->rows_per_vector, a->channels, a->norm, a->x_dtype, a->vector_dtype, a->alpha, a->eps, a->post_eps)) return rc;
  if (!a->dh || !a->x_out || !a->dx) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: dh, x_out and dx must not be NULL", who);
  if (!a->y && (a->gate || a->post_weight || a->dy || a->dgate || a->dpost_weight))
    return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: gate, post_weight, dy, dgate and dpost_weight need y", who);
  if ((a->dpost_weight && !a->post_weight) || (a->dweight && !a->weight))
    return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: a weight's gradient needs the weight", who);
  if (a->scale_stride < 0 || a->gate_stride < 0) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: strides must not be negative", who);
  const int C = a->channels;
  const long long vectors = (a->rows - 1) / a->rows_per_vector + 1;
  const size_t n = (size_t)a->rows * C, xs = type_size(a->x_dtype), vs = type_size(a->vector_dtype);
  auto vec_bytes = [&](long long stride) { return ((size_t)(vectors - 1) * stride + C) * vs; };
  const size_t sums = (size_t)vectors * C * 4;
  const Range outs[] = {{"dx", a->dx, n * xs}, {"dy", a->dy, n * 2}, {"dweight", a->dweight, (size_t)C * 4}, {"dscale", a->dscale, sums},
                        {"dshift", a->dshift, sums}, {"dgate", a->dgate, sums}, {"dpost_weight", a->dpost_weight, (size_t)C * 4}};
  const Range ins[] = {{"dh", a->dh, n * 2}, {"dx_out", a->dx_out, n * xs}, {"x_out", a->x_out, n * xs}, {"y", a->y, n * 2},
                       {"weight", a->weight, (size_t)C * vs}, {"post_weight", a->post_weight, (size_t)C * vs},
                       {"scale", a->scale, vec_bytes(a->scale_stride)}, {"gate", a->gate, vec_bytes(a->gate_stride)}};
  if (int rc = check_overlaps(who, outs, 7, ins, 8, a->dx_out, a->dx)) return rc;
  if (int rc = check_elements(who, {a->dx_out, a->x_out, a->dx}, xs)) return rc;
  if (int rc = check_elements(who, {a->dh, a->y, a->dy}, 2)) return rc;
  if (int rc = check_elements(who, {a->weight, a->scale, a->gate, a->post_weight}, vs)) return rc;
  if (int rc = check_elements(who, {a->dweight, a->dscale, a->dshift, a->dgate, a->dpost_weight}, 4)) return rc;
  const bool vec = C % 8 == 0 && aligned16(a->dh) && aligned16(a->dx_out) && aligned16(a->x_out) && aligned16(a->y) && aligned16(a->dx) &&
                   aligned16(a->dy) && aligned16(a->weight) && aligned16(a->scale) && aligned16(a->gate) && aligned16(a->post_weight) &&
                   (a->scale_stride | a->gate_stride) % 8 == 0;
  hipStream_t stream = (hipStream_t)hip_stream;
  const ChunkPlan plan = chunks_of(std::min(a->rows_per_vector, a->rows), vectors, C);
  if (vectors * plan.chunks > 0x7fffffffLL) return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: too many modulation vectors", who);
  const size_t VC = (size_t)vectors * C, plane = VC * plan.chunks;
  const int runs = plan.chunks > kFold ? (plan.chunks + kFold - 1) / kFold : 0;
  const bool want[3] = {a->dshift != nullptr, a->dscale || a->dweight, a->dgate || a->dpost_weight};
  float* const result[3] = {a->dshift, a->dscale, a->dgate};
  // Scratch memory: the chunks' sums, then those of the runs.  With one chunk to a vector they are the results up to a factor
  // and are kept there.  What the weights' gradients are the sums of: their own places with one vector.
  size_t need = 0, planes = 0;
  auto take = [&](bool wanted, size_t floats) {
    const size_t at = need;
    if (wanted) need += floats;
    return at;
  };
  size_t at_part[3], at_folded[3];
  for (int i = 0; i < 3; ++i) {
    planes += want[i];
    at_part[i] = take(want[i] && (plan.chunks > 1 || !result[i]), plane);
    at_folded[i] = take(want[i] && runs, VC * runs);
  }
  const size_t at_wa = take(a->dweight && vectors > 1, VC), at_we = take(a->dpost_weight && vectors > 1, VC);
  sa_scratch scratch;
  if (need)
    if (int rc = scratch.get(need * 4, stream)) return rc;
  float* const base = (float*)scratch.data();
  BackParams p = {a->dh, a->dx_out, a->x_out, a->y, a->weight, a->scale, a->gate, a->post_weight, a->dx, a->dy, {}, a->rows,
                  a->rows_per_vector, vectors, a->scale_stride, a->gate_stride, C, a->norm == SPARSE_BLOCK_NORM_LAYER, plan.chunks, plan.rows, 0,
                  a->y ? a->alpha : 1.f, a->eps, a->post_eps};
  for (int i = 0; i < 3; ++i) p.part[i] = !want[i] ? nullptr : plan.chunks == 1 && result[i] ? result[i] : base + at_part[i];
  by_types(a->x_dtype, a->vector_dtype, [&](auto tx, auto tv) { launch_backward<decltype(tx), decltype(tv)>(p, vec, stream); });
  if (int rc = launched(who)) return rc;
  if (!planes) return 0;
  float* wa = !a->dweight ? nullptr : vectors > 1 ? base + at_wa : a->dweight;
  float* we = !a->dpost_weight ? nullptr : vectors > 1 ? base + at_we : a->dpost_weight;
  FinishParams f = {{}, {}, a->weight, a->scale, a->gate, a->post_weight, a->dscale, a->dshift, a->dgate, wa, we, vectors,
                    a->scale_stride, a->gate_stride, C, plan.chunks};
  const int some = want[0] ? 0 : want[1] ? 1 : 2;
  for (int i = 0; i < 3; ++i) {
    f.part[i] = p.part[want[i] ? i : some];
    f.folded[i] = want[i] && runs ? base + at_folded[i] : nullptr;
  }
  const unsigned blocks = (unsigned)((C + 255) / 256), y = (unsigned)std::min(vectors, 65535LL);
  if (runs) {
    hipLaunchKernelGGL(block_norm_fold_kernel, dim3(blocks, y, (unsigned)runs), dim3(256), 0, stream, f);
    for (int i = 0; i < 3; ++i) f.part[i] = f.folded[want[i] ? i : some];
    f.chunks = runs;
  }
  if (a->vector_dtype == SPARSE_BLOCK_F32)
    hipLaunchKernelGGL(block_norm_finish_kernel<float>, dim3(blocks, y), dim3(256), 0, stream, f);
  else
    hipLaunchKernelGGL(block_norm_finish_kernel<__bf16>, dim3(blocks, y), dim3(256), 0, stream, f);
  const unsigned columns = (unsigned)((C + 63) / 64);
  if (vectors > 1 && (wa || we))
    hipLaunchKernelGGL(column_sum_kernel, dim3(columns), dim3(1024), 0, stream, wa ? wa : we, we ? we : wa, a->dweight, a->dpost_weight, vectors, C);
  return launched(who);
}

}  // extern "C"
