// Rotary heads: the rows of a fused projection split into heads, RMSNorm per head, rotation by the token's position on up to
// four axes, and the gradients (include/sparse_block.h).
//
// HBM-bound: every channel is read once and written once (backward: gradient and input read, one written).  A head's D
// channels are D / 8 neighbouring lanes with eight channels each, a wave holds 512 / D tokens and walks over heads: a lane
// stays at its channels, so it takes the sine and cosine of its four pairs once for all heads of its token.  With halves the
// members of a pair are R / 2 channels apart; a lane then holds four channels from each half instead of eight neighbours, so
// that a pair still lies in one lane.  33024 tokens of 24 + 24 + 24 heads of 128 with the norm of q and k: 245 us, 5.0 TB/s;
// backward with the weights' gradients 326 us, 5.6 TB/s; eight tokens 4 us.  Angles are reduced in 64 bits; norms,
// rotations and sums are float32, and each result is rounded once, to bf16.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "sparse_attn.h"
#include "sparse_attn_internal.h"
#include "sparse_block.h"
#include "sparse_block_internal.h"

namespace {

using namespace sa_block;

constexpr int kMaxAxes = 4, kMaxPairs = 128;
constexpr int kMaxHeads = 1 << 20;     // so that their channels are counted in 32 bits
constexpr long long kMostGroups = (1 << 24) - 1;     // workgroups of 256 threads: fewer than 2^32 of these

struct RotaryParams {
  const __bf16* qkv;
  const void* positions;
  __bf16 *Q, *K, *V;                 // backward: read
  __bf16* dqkv;                      // backward: written
  const __bf16 *q_weight, *k_weight;
  float* part;                       // backward: [workgroups][2][D] sums for the weights' gradients, or NULL
  long long qkv_b, qkv_l, dqkv_b, dqkv_l, q_b, q_h, q_l, k_b, k_h, k_l, v_b, v_h, v_l;
  long long tokens;                  // B * L
  int L, heads_q, heads_kv, axes, halves, per_batch, int_positions, pairs, heads_per_part;
  float eps;
  double turns[kMaxPairs];           // revolutions per unit of position
  uint8_t axis[kMaxPairs];
};

// One lane's eight channels of a head: two runs of four (neighbours, or from the two halves of the rotated channels).
struct Lane {
  int c0, c1;                        // first channels of the runs
  int turned;                        // its pairs below this are turned, the others pass as they are
  float cs[4], sn[4];
};

template <int D>
__device__ __forceinline__ Lane lane_of(const RotaryParams& p, int j, const void* pos_row) {
  Lane l;
  const int half = p.pairs;          // R / 2
  const bool split = p.halves && 4 * j < half;
  l.c0 = split ? 4 * j : 8 * j;
  l.c1 = split ? half + 4 * j : 8 * j + 4;
  l.turned = half - 4 * j;
  // All positions of the token are read, and the lane's pairs pick theirs: no read waits for another.
  double at[kMaxAxes];
#pragma unroll
  for (int a = 0; a < kMaxAxes; ++a) {
    const int i = min(a, p.axes - 1);
    at[a] = p.int_positions ? (double)((const int*)pos_row)[i] : (double)((const float*)pos_row)[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int pair = min(4 * j + i, kMaxPairs - 1), a = p.axis[pair];
    const double here = a == 0 ? at[0] : a == 1 ? at[1] : a == 2 ? at[2] : at[3];
    // whole revolutions are dropped in 64 bits: positions are few bits, so the angle is as exact as its frequency
    const double rev = here * p.turns[pair];
    sincospif(2.f * (float)(rev - rint(rev)), &l.sn[i], &l.cs[i]);
  }
  return l;
}

template <bool HALVES>
__device__ __forceinline__ bf16x8 load_runs(const __bf16* head, const Lane& l) {
  if constexpr (!HALVES) return __builtin_nontemporal_load((const bf16x8*)(head + l.c0));
  const bf16x4 a = __builtin_nontemporal_load((const bf16x4*)(head + l.c0)), b = __builtin_nontemporal_load((const bf16x4*)(head + l.c1));
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <bool HALVES>
__device__ __forceinline__ void store_runs(__bf16* head, const Lane& l, const float (&v)[8]) {
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (__bf16)v[e];
  if constexpr (!HALVES) {
    __builtin_nontemporal_store(r, (bf16x8*)(head + l.c0));
  } else {
    __builtin_nontemporal_store(__builtin_shufflevector(r, r, 0, 1, 2, 3), (bf16x4*)(head + l.c0));
    __builtin_nontemporal_store(__builtin_shufflevector(r, r, 4, 5, 6, 7), (bf16x4*)(head + l.c1));
  }
}
__device__ __forceinline__ void load_weight(const __bf16* w, const Lane& l, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = (float)w[l.c0 + e];
    v[e + 4] = (float)w[l.c1 + e];
  }
}
// rotation by +1 or -1 times the angle; a channel that is not turned takes nothing from its neighbour, which may be infinite
__device__ __forceinline__ void turn(const Lane& l, bool halves, float sign, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = halves ? v[i] : v[2 * i], b = halves ? v[i + 4] : v[2 * i + 1];
    const float s = sign * l.sn[i], x = a * l.cs[i] - b * s, y = a * s + b * l.cs[i];
    const bool on = i < l.turned;
    v[halves ? i : 2 * i] = on ? x : a;
    v[halves ? i + 4 : 2 * i + 1] = on ? y : b;
  }
}

constexpr int kAhead = 4;            // heads whose loads are on their way together (33024 tokens, 72 heads: 1: 295 us, 4: 249, 8: 259)

// Which heads of the row this workgroup walks over: [lo, hi) of heads_q + 2 heads_kv.
template <int D, bool HALVES>
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryParams p) {
  constexpr int kLanes = D / 8, kTokens = 64 / kLanes;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long token = ((long long)blockIdx.x * 4 + wave) * kTokens + lane / kLanes;
  const bool live = token < p.tokens;
  const long long at = live ? token : p.tokens - 1;          // idle lanes repeat the last token, their stores are left out
  const long long b = at / p.L, l = at % p.L;
  const void* pos = (const char*)p.positions + ((p.per_batch ? at : l) * p.axes) * 4;
  const Lane me = lane_of<D>(p, lane % kLanes, pos);
  const int hq = p.heads_q, hkv = p.heads_kv, lo = blockIdx.y * p.heads_per_part, hi = min(hq + 2 * hkv, lo + p.heads_per_part);
  const __bf16* row = p.qkv + b * p.qkv_b + l * p.qkv_l;

  auto walk = [&](int from, int to, const __bf16* w, __bf16* out, long long stride_h, bool rotate) __attribute__((always_inline)) {
    if (!out) return;
    float wf[8];
    if (w) load_weight(w, me, wf);
    const int last = min(to, hi);
    for (int h0 = max(from, lo); h0 < last; h0 += kAhead) {
      bf16x8 t[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) t[k] = load_runs<HALVES>(row + (long long)min(h0 + k, last - 1) * D, me);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (h0 + k >= last) break;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)t[k][e];
        if (w) {
          float s = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) s = fmaf(v[e], v[e], s);
          const float r = 1.f / sqrtf(group_sum<kLanes>(s) * (1.f / D) + p.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = v[e] * r * wf[e];
        }
        if (rotate) turn(me, HALVES, 1.f, v);
        if (live) store_runs<HALVES>(out + (h0 + k - from) * stride_h, me, v);
      }
    }
  };
  walk(0, hq, p.q_weight, p.Q ? p.Q + b * p.q_b + l * p.q_l : nullptr, p.q_h, true);
  walk(hq, hq + hkv, p.k_weight, p.K ? p.K + b * p.k_b + l * p.k_l : nullptr, p.k_h, true);
  walk(hq + hkv, hq + 2 * hkv, nullptr, p.V ? p.V + b * p.v_b + l * p.v_l : nullptr, p.v_h, false);
}

// d = rotation back of the gradient; with a norm, n = v / rms(v): dv = r (d w - n mean(d w n)), dw = sum d n.
template <int D, bool HALVES>
__global__ void __launch_bounds__(256) rotary_backward_kernel(const RotaryParams p) {
  constexpr int kLanes = D / 8, kTokens = 64 / kLanes;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int hq = p.heads_q, hkv = p.heads_kv, lo = blockIdx.y * p.heads_per_part, hi = min(hq + 2 * hkv, lo + p.heads_per_part);
  float sums[2][8] = {};
  int c0 = 0, c1 = 0;
  for (long long t0 = ((long long)blockIdx.x * 4 + wave) * kTokens; t0 < p.tokens; t0 += (long long)gridDim.x * 4 * kTokens) {
    const long long token = t0 + lane / kLanes;
    const bool live = token < p.tokens;
    const long long at = live ? token : p.tokens - 1;
    const long long b = at / p.L, l = at % p.L;
    const void* pos = (const char*)p.positions + ((p.per_batch ? at : l) * p.axes) * 4;
    const Lane me = lane_of<D>(p, lane % kLanes, pos);
    c0 = me.c0;
    c1 = me.c1;
    const __bf16* row = p.qkv ? p.qkv + b * p.qkv_b + l * p.qkv_l : nullptr;
    __bf16* drow = p.dqkv + b * p.dqkv_b + l * p.dqkv_l;

    auto walk = [&](int from, int to, const __bf16* w, const __bf16* grad, long long stride_h, bool rotate, float (&sum)[8]) __attribute__((always_inline)) {
      float wf[8];
      if (w) load_weight(w, me, wf);
      // one head at a time: two or four of them take registers that cost more waves than their loads gain (36.5, 38, 44 us
      // with 9001 tokens, 32 heads of 64)
      for (int h = max(from, lo); h < min(to, hi); ++h) {
        const bf16x8 td = load_runs<HALVES>(grad + (h - from) * stride_h, me);
        bf16x8 tv;
        if (w) tv = load_runs<HALVES>(row + (long long)h * D, me);
        float d[8], v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = (float)td[e];
        if (rotate) turn(me, HALVES, -1.f, d);
        if (w) {
          float s = 0.f, dot = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[e] = (float)tv[e];
            s = fmaf(v[e], v[e], s);
            dot = fmaf(d[e] * wf[e], v[e], dot);
          }
          const float r = 1.f / sqrtf(group_sum<kLanes>(s) * (1.f / D) + p.eps);
          const float mean = group_sum<kLanes>(dot) * r * (1.f / D);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float n = v[e] * r;
            if (live) sum[e] = fmaf(d[e], n, sum[e]);
            d[e] = r * (d[e] * wf[e] - n * mean);
          }
        }
        if (live) store_runs<HALVES>(drow + (long long)h * D, me, d);
      }
    };
    walk(0, hq, p.q_weight, p.Q + b * p.q_b + l * p.q_l, p.q_h, true, sums[0]);
    walk(hq, hq + hkv, p.k_weight, p.K + b * p.k_b + l * p.k_l, p.k_h, true, sums[1]);
    float none[8];
    walk(hq + hkv, hq + 2 * hkv, nullptr, p.V + b * p.v_b + l * p.v_l, p.v_h, false, none);
  }
  if (!p.part) return;
  // the workgroup's sums: over its token groups through LDS, in a fixed order
  __shared__ float red[4 * kTokens][D];
  float* part = p.part + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 2 * D;
  if (c1 == 0) {                       // a wave without a token still has its place in the sums below
    const int j = lane % kLanes;
    const bool split = HALVES && 4 * j < p.pairs;
    c0 = split ? 4 * j : 8 * j;
    c1 = split ? p.pairs + 4 * j : 8 * j + 4;
  }
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      red[wave * kTokens + lane / kLanes][c0 + e] = sums[k][e];
      red[wave * kTokens + lane / kLanes][c1 + e] = sums[k][e + 4];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < D; c += 256) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 4 * kTokens; ++i) s += red[i][c];
      part[k * D + c] = s;
    }
    __syncthreads();
  }
}

// [n][2][D] -> the two weights' gradients: a workgroup per channel pair of columns, its threads' strides added in order
__global__ void __launch_bounds__(256) rotary_weight_kernel(const float* part, int n, int D, float* dq, float* dk) {
  __shared__ float red[256];
  const int col = blockIdx.x;                 // 0 .. 2 D - 1
  float s = 0.f;
  for (int i = threadIdx.x; i < n; i += 256) s += part[(long long)i * 2 * D + col];
  red[threadIdx.x] = s;
  __syncthreads();
  for (int step = 128; step > 0; step >>= 1) {
    if ((int)threadIdx.x < step) red[threadIdx.x] += red[threadIdx.x + step];
    __syncthreads();
  }
  float* out = col < D ? dq : dk;
  if (threadIdx.x == 0 && out) out[col % D] = red[0];
}

// ---------------------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------------------
struct View {
  const char* name;
  const void* p;
  long long b, h, l;
  int heads;
};

// first and one past the last byte of a view of B x heads x L rows of D channels
size_t view_bytes(const View& v, int B, int L, int D) {
  return ((size_t)(B - 1) * v.b + (size_t)(v.heads - 1) * v.h + (size_t)(L - 1) * v.l + D) * 2;
}

int check_view(const char* who, const View& v) {
  if (!v.p) return 0;
  if (!aligned16(v.p) || (v.b | v.h | v.l) % 8 || v.b < 0 || v.h < 0 || v.l < 0)
    return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: %s must be 16-byte aligned, with strides that are multiples of 8 and not negative", who, v.name);
  return 0;
}

// Steps of one loop over the rows of two views: `range` values from 0 on, each `step` elements further (from `at` on, over all steps).
struct Walk {
  long long step, range;
};

// Whether a value of  at + sum of steps  lies in (-D, D), that is, whether two rows of D channels share an element.  The walks are
// sorted by their span; what the later ones can still add bounds the values of the first, so that few are looked at in views that
// are slices of one another.  `tries` bounds the others: without an answer by then the views count as overlapping.
bool meets(const Walk* w, int n, long long at, int D, long long rest, int& tries) {
  if (n == 0) return at > -D && at < D;
  const long long step = w->step, after = rest - step * (w->range - 1);
  // the values v with  -D < at + v step + [0, after] < D
  const long long low = -D - at - after, high = D - at;                     // of v step, both excluded
  const long long v0 = low < 0 ? 0 : low / step + 1, v1 = high <= 0 ? -1 : (high - 1) / step;
  for (long long v = v0; v <= v1 && v < w->range; ++v) {
    if (--tries < 0 || meets(w + 1, n - 1, at + v * step, D, after, tries)) return true;
  }
  return false;
}

// The differences of rows of views: walks in the order that meets() wants.
struct Walks {
  Walk w[6];
  int n = 0;
  void add(long long step, long long range) {
    if (range <= 1 || !step) return;
    int i = n++;
    for (; i > 0 && w[i - 1].step < step; --i) w[i] = w[i - 1];
    w[i] = {step, range};
  }
  bool meet(long long at, int D) const {
    long long reach = 0;
    for (int i = 0; i < n; ++i) reach += w[i].step * (w[i].range - 1);
    int tries = 1 << 16;
    return meets(w, n, at, D, reach, tries);
  }
};

// a written view must not hold an element twice
int check_written(const char* who, const View& v, int B, int L, int D) {
  const long long s[3] = {v.b, v.h, v.l}, n[3] = {B, v.heads, L};
  for (int i = 0; i < 3; ++i) {                  // two rows that differ in dimension i, maybe in those behind it, in none before it
    if (n[i] <= 1) continue;
    Walks d;
    long long at = s[i];
    d.add(s[i], n[i] - 1);
    for (int j = i + 1; j < 3; ++j) {
      at -= s[j] * (n[j] - 1);
      d.add(s[j], 2 * n[j] - 1);
    }
    if (d.meet(at, D)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: rows of %s overlap each other", who, v.name);
  }
  return 0;
}

// Two written views may be interleaved (slices of one tensor): whether a row of one shares elements with a row of the other.
bool rows_clash(const View& a, const View& b, int B, int L, int D) {
  if (!a.p || !b.p || !overlap(a.p, view_bytes(a, B, L, D), b.p, view_bytes(b, B, L, D))) return false;
  Walks d;
  long long at = (long long)((intptr_t)b.p - (intptr_t)a.p) / 2;
  const long long sa[3] = {a.b, a.h, a.l}, sb[3] = {b.b, b.h, b.l};
  const long long na[3] = {B, a.heads, L}, nb[3] = {B, b.heads, L};
  for (int i = 0; i < 3; ++i) {                  // row of b minus row of a: na - 1 steps down, nb - 1 steps up
    at -= sa[i] * (na[i] - 1);
    if (sa[i] == sb[i]) {
      d.add(sa[i], na[i] + nb[i] - 1);
    } else {
      d.add(sa[i], na[i]);
      d.add(sb[i], nb[i]);
    }
  }
  return d.meet(at, D);
}

int check_rotary(const char* who, const sparse_rotary_args* a, RotaryParams& p) {
  if (!a) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: args must not be NULL", who);
  if (a->B <= 0 || a->L <= 0 || a->heads_q < 0 || a->heads_kv < 0 || (a->heads_q == 0 && a->heads_kv == 0))
    return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: B=%d, L=%d must be positive, heads_q=%d and heads_kv=%d not negative nor both 0", who, a->B, a->L,
                   a->heads_q, a->heads_kv);
  if (a->heads_q > kMaxHeads || a->heads_kv > kMaxHeads)
    return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: at most %d heads of a kind, got %d and %d", who, kMaxHeads, a->heads_q, a->heads_kv);
  if (a->D != 32 && a->D != 64 && a->D != 128 && a->D != 256) return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: D=%d must be 32, 64, 128 or 256", who, a->D);
  if (a->axes < 1 || a->axes > kMaxAxes) return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: axes=%d must be between 1 and %d", who, a->axes, kMaxAxes);
  if (!a->positions || !a->axis_channels) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: positions and axis_channels must not be NULL", who);
  if (!a->inv_freq && !(a->theta > 0.0 && a->theta - a->theta == 0.0)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: theta must be finite and > 0 where inv_freq is NULL", who);
  if ((uintptr_t)a->positions & 3) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: positions must be 4-byte aligned", who);
  if (a->position_dtype != SPARSE_BLOCK_I32 && a->position_dtype != SPARSE_BLOCK_F32)
    return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: position_dtype=%d must be I32 or F32", who, a->position_dtype);
  if (!finite_nonnegative(a->eps)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: eps must be finite and >= 0", who);
  long long R = 0;
  for (int i = 0; i < a->axes; ++i) {
    if (a->axis_channels[i] < 0 || a->axis_channels[i] % 2)
      return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: axis_channels[%d]=%d must be even and not negative", who, i, a->axis_channels[i]);
    R += a->axis_channels[i];
  }
  if (R > a->D) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: the axes take %lld channels, a head has %d", who, R, a->D);
  if (a->halves && R % 8) return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: with halves the axes must take a multiple of 8 channels, got %lld", who, R);
  double from_theta[kMaxPairs];
  if (!a->inv_freq) sparse_rotary_frequencies(a->axes, a->axis_channels, a->theta, from_theta);
  const double* freq = a->inv_freq ? a->inv_freq : from_theta;
  for (int i = 0, k = 0; i < a->axes; ++i)
    for (int j = 0; j < a->axis_channels[i] / 2; ++j, ++k) {
      if (freq[k] - freq[k] != 0.0) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: inv_freq[%d] must be finite", who, k);
      p.turns[k] = freq[k] / 6.283185307179586476925286766559;
      p.axis[k] = (uint8_t)i;
    }
  for (const void* w : {a->q_weight, a->k_weight})
    if ((uintptr_t)w & 1) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: weights must be aligned to their elements", who);
  p.qkv = (const __bf16*)a->qkv;
  p.positions = a->positions;
  p.Q = (__bf16*)a->Q;
  p.K = (__bf16*)a->K;
  p.V = (__bf16*)a->V;
  p.q_weight = (const __bf16*)a->q_weight;
  p.k_weight = (const __bf16*)a->k_weight;
  p.qkv_b = a->qkv_stride_b, p.qkv_l = a->qkv_stride_l;
  p.q_b = a->q_stride_b, p.q_h = a->q_stride_h, p.q_l = a->q_stride_l;
  p.k_b = a->k_stride_b, p.k_h = a->k_stride_h, p.k_l = a->k_stride_l;
  p.v_b = a->v_stride_b, p.v_h = a->v_stride_h, p.v_l = a->v_stride_l;
  p.tokens = (long long)a->B * a->L;
  p.L = a->L, p.heads_q = a->heads_q, p.heads_kv = a->heads_kv, p.axes = a->axes, p.halves = a->halves != 0;
  p.per_batch = a->positions_per_batch != 0, p.int_positions = a->position_dtype == SPARSE_BLOCK_I32, p.pairs = (int)(R / 2);
  p.eps = a->eps;
  return 0;
}

// Few tokens: their heads are dealt to several workgroups, so that the call fills the chip and a wave's walk is short.  72 heads
// of 128, forward, against one workgroup for all heads: 64 tokens 4.6 us / 21, 512 tokens 7 / 23, 4608 tokens 36 / 47, from some
// 8192 tokens on the same.
constexpr int kFewParts = 512;
int head_parts(long long groups, int heads) {
  long long parts = (kFewParts + groups - 1) / groups;
  return (int)(parts < 1 ? 1 : parts > heads ? heads : parts);
}

template <class F>
void by_shape(int D, bool halves, F&& f) {
  auto h = [&](auto d) { halves ? f(d, std::true_type{}) : f(d, std::false_type{}); };
  switch (D) {
    case 32: h(std::integral_constant<int, 32>{}); break;
    case 64: h(std::integral_constant<int, 64>{}); break;
    case 128: h(std::integral_constant<int, 128>{}); break;
    default: h(std::integral_constant<int, 256>{}); break;
  }
}

}  // namespace

extern "C" {

int sparse_rotary_heads(const sparse_rotary_args* a, void* hip_stream) {
  const char* who = "rotary_heads";
  RotaryParams p = {};
  if (int rc = check_rotary(who, a, p)) return rc;
  if (!a->qkv || (!a->Q && !a->K && !a->V)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: qkv and one of Q, K, V must not be NULL", who);
  const int heads = a->heads_q + 2 * a->heads_kv;
  const View in = {"qkv", a->qkv, a->qkv_stride_b, a->D, a->qkv_stride_l, heads};
  View out[3] = {{"Q", a->Q, a->q_stride_b, a->q_stride_h, a->q_stride_l, a->heads_q},
                 {"K", a->K, a->k_stride_b, a->k_stride_h, a->k_stride_l, a->heads_kv},
                 {"V", a->V, a->v_stride_b, a->v_stride_h, a->v_stride_l, a->heads_kv}};
  if (int rc = check_view(who, in)) return rc;
  for (View& v : out) {
    if (v.heads == 0) v.p = nullptr;
    if (!v.p) continue;
    if (int rc = check_view(who, v)) return rc;
    if (int rc = check_written(who, v, a->B, a->L, a->D)) return rc;
    if (overlap(v.p, view_bytes(v, a->B, a->L, a->D), in.p, view_bytes(in, a->B, a->L, a->D)))
      return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: %s must not overlap qkv", who, v.name);
  }
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < i; ++j)
      if (rows_clash(out[i], out[j], a->B, a->L, a->D)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: %s must not overlap %s", who, out[i].name, out[j].name);
  const int per_group = 4 * 512 / a->D;
  const long long groups = (p.tokens + per_group - 1) / per_group;
  if (groups > kMostGroups) return sa_fail(SPARSE_ATTN_ERR_UNSUPPORTED, "%s: too many tokens", who);
  const int parts = head_parts(groups, heads);
  p.heads_per_part = (heads + parts - 1) / parts;
  const dim3 grid((unsigned)groups, (unsigned)((heads + p.heads_per_part - 1) / p.heads_per_part));
  by_shape(a->D, p.halves, [&](auto d, auto h) {
    hipLaunchKernelGGL((rotary_kernel<decltype(d)::value, decltype(h)::value>), grid, dim3(256), 0, (hipStream_t)hip_stream, p);
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? 0 : sa_fail(SPARSE_ATTN_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
}

int sparse_rotary_heads_backward(const sparse_rotary_args* a, void* dqkv, long long dqkv_stride_b, long long dqkv_stride_l,
                                 float* dq_weight, float* dk_weight, void* hip_stream) {
  const char* who = "rotary_heads_backward";
  RotaryParams p = {};
  if (int rc = check_rotary(who, a, p)) return rc;
  if (!dqkv || (a->heads_q && !a->Q) || (a->heads_kv && (!a->K || !a->V)))
    return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: dqkv and the gradients Q, K, V must not be NULL", who);
  if ((a->q_weight || a->k_weight) && !a->qkv) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: with a norm weight qkv must not be NULL", who);
  if ((dq_weight && !a->q_weight) || (dk_weight && !a->k_weight)) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: a weight's gradient needs the weight", who);
  for (const void* w : {dq_weight, dk_weight})
    if ((uintptr_t)w & 3) return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: the weights' gradients must be aligned to their elements", who);
  const int heads = a->heads_q + 2 * a->heads_kv;
  const View out = {"dqkv", dqkv, dqkv_stride_b, a->D, dqkv_stride_l, heads};
  const View in[4] = {{"qkv", a->qkv, a->qkv_stride_b, a->D, a->qkv_stride_l, heads},
                      {"Q", a->heads_q ? a->Q : nullptr, a->q_stride_b, a->q_stride_h, a->q_stride_l, a->heads_q},
                      {"K", a->heads_kv ? a->K : nullptr, a->k_stride_b, a->k_stride_h, a->k_stride_l, a->heads_kv},
                      {"V", a->heads_kv ? a->V : nullptr, a->v_stride_b, a->v_stride_h, a->v_stride_l, a->heads_kv}};
  if (int rc = check_view(who, out)) return rc;
  if (int rc = check_written(who, out, a->B, a->L, a->D)) return rc;
  for (const View& v : in) {
    if (int rc = check_view(who, v)) return rc;
    if (v.p && overlap(out.p, view_bytes(out, a->B, a->L, a->D), v.p, view_bytes(v, a->B, a->L, a->D)))
      return sa_fail(SPARSE_ATTN_ERR_INVALID, "%s: dqkv must not overlap %s", who, v.name);
  }
  p.dqkv = (__bf16*)dqkv;
  p.dqkv_b = dqkv_stride_b, p.dqkv_l = dqkv_stride_l;
  const int per_group = 4 * 512 / a->D;
  const long long all = (p.tokens + per_group - 1) / per_group;
  const bool sums = dq_weight || dk_weight;
  // with sums a workgroup takes several token groups, so that there are few of them to add and to keep (33024 tokens, 72 heads
  // of 128: 326 us, with 512 workgroups 364, with one for each group 328)
  const long long most = sums ? 2048 : kMostGroups;
  const long long groups = all < most ? all : most;
  const int parts = head_parts(groups, heads);
  p.heads_per_part = (heads + parts - 1) / parts;
  const dim3 grid((unsigned)groups, (unsigned)((heads + p.heads_per_part - 1) / p.heads_per_part));
  hipStream_t stream = (hipStream_t)hip_stream;
  const size_t n = (size_t)grid.x * grid.y;
  sa_scratch scratch;
  if (sums) {
    // as many as there are workgroups with these sizes or smaller ones: a smaller call has then what it needs
    const long long most_n = std::min(groups * heads, groups + kFewParts - 1);
    if (int rc = scratch.get(most_n * 2 * a->D * 4, stream)) return rc;
    p.part = (float*)scratch.data();
  }
  by_shape(a->D, p.halves, [&](auto d, auto h) {
    hipLaunchKernelGGL((rotary_backward_kernel<decltype(d)::value, decltype(h)::value>), grid, dim3(256), 0, stream, p);
  });
  if (sums) hipLaunchKernelGGL(rotary_weight_kernel, dim3(2 * a->D), dim3(256), 0, stream, p.part, (int)n, a->D, dq_weight, dk_weight);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? 0 : sa_fail(SPARSE_ATTN_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
}

void sparse_rotary_frequencies(int axes, const int* axis_channels, double theta, double* inv_freq) {
  for (int a = 0, k = 0; a < axes; ++a) {
    const double step = axis_channels[a] > 0 ? pow(theta, -2.0 / axis_channels[a]) : 1.0;
    double f = 1.0;                    // a product of at most 127 steps: a few parts in 10^14
    for (int i = 0; i < axis_channels[a] / 2; ++i, ++k, f *= step) inv_freq[k] = f;
  }
}

}  // extern "C"
