// Router of the routed-expert layer: top-k selection and routing weights, per-expert counts and
// the balance loss, and their gradients (formulas in tq.h).
//
// One wave holds one token's logits, NV consecutive experts a lane, as 32-bit keys whose unsigned
// order is the logits' order. Lanes and positions ascend with the expert id, so among equal keys
// the first lane's first position is the lowest id. A token's steps (maxima, sums) depend on each other, so its time is
// that of their chain: 2048 tokens of 256 experts, 8 slots 4.9 us, 1 token 3.0, an empty launch about 2.5.
#include <algorithm>

#include "tq_ops.hpp"

namespace tq {

constexpr int kRouteWaves = 4;
constexpr int kRouteMaxExperts = 4096;
constexpr int kRouteMaxTopk = 64;  // lane j of the wave keeps slot j
constexpr int kRouteMaxGroups = 256;
constexpr int kRouteTokensPerWave = 2;
constexpr int kJoinCols = 16;  // experts per workgroup of the join
constexpr int kJoinRows = 32;  // workgroups' sums that are read at once

// Waves of a workgroup of the balance pass (fewer where a lane's experts fill the registers).
__host__ __device__ constexpr int balance_waves(int nv) { return nv <= 8 ? 16 : 4; }
static int lane_experts(int E) { return E <= 64 ? 1 : E <= 128 ? 2 : E <= 256 ? 4 : E <= 512 ? 8 : E <= 1024 ? 16 : 64; }

// A logit as an ordered key: 0 for an expert that cannot be chosen (-inf, or none there). -0 and
// +0 are one value; a NaN of either sign comes first, so that it shows in the weights.
__device__ __forceinline__ uint32_t route_key(float l) {
  if (l == -__builtin_huge_valf()) return 0;
  if (l != l) return 0xffffffffu;
  const uint32_t u = __float_as_uint(l + 0.0f);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float route_value(uint32_t key) {
  return __uint_as_float(key ^ ((key & 0x80000000u) ? 0x80000000u : 0xffffffffu));
}

// The 12 lowest bits of a bfloat16's or fp16's fp32 key carry nothing (all zeros or all ones) and can take the expert.
constexpr uint32_t kTag = 0xfff;
static_assert(kRouteMaxExperts <= kTag + 1, "an expert fits a tag");
__device__ __forceinline__ uint32_t tag_of(int e) { return kTag - (uint32_t)e; }
template <bool TAGGED>
__device__ __forceinline__ float value_of(uint32_t key) {
  return TAGGED ? __uint_as_float(__float_as_uint(route_value(key)) & ~kTag) : route_value(key);
}

// A lane's logits of one token, NV consecutive ones, as they lie in memory (a token's loads are under way while the one before
// it is worked on).
template <int ROW, typename T, int NV>
struct Logits {
  static constexpr int C = NV < 4 ? NV : 4;
  typename VecOf<T, C>::type v[NV / C];

  __device__ __forceinline__ static uint32_t start(int lane, int c, int E) {  // (E >= C)
    return min((uint32_t)(lane * NV + c * C), (uint32_t)(E - C));
  }
  __device__ __forceinline__ void load(const T* row, int lane, int E) {
#pragma unroll
    for (int c = 0; c < NV / C; ++c) v[c] = *reinterpret_cast<const typename VecOf<T, C>::type*>(row + start(lane, c, E));
  }
  // TAGGED: with tag_of(expert) below the value, so that no two keys of a token are equal and the larger one has the lower id
  template <bool TAGGED>
  __device__ __forceinline__ void keys(int lane, int E, bool on, uint32_t (&key)[NV]) const {
#pragma unroll
    for (int c = 0; c < NV / C; ++c) {
      float f[C];
#pragma unroll
      for (int i = 0; i < C; ++i) f[i] = (float)v[c][i];
      if constexpr (ROW == kRowTail) rotate(f, lane * NV + c * C - start(lane, c, E));
#pragma unroll
      for (int i = 0; i < C; ++i) {
        uint32_t k = route_key(f[i]);
        if constexpr (TAGGED) k = k ? (k & ~kTag) | tag_of(lane * NV + c * C + i) : 0;
        key[c * C + i] = on && lane * NV + c * C + i < E ? k : 0;
      }
    }
  }
};

// exp(x) for x <= 0: 2^(x log2 e) by the exponential unit, with what the product's rounding left out brought in to first order.
// Below -200 (and NaN) as -200, whose exponential fp32 holds as 0.
__device__ __forceinline__ float exp_below(float x) {
  x = fmaxf(x, -200.0f);
  const float t = x * 0x1.715476p+0f;
  const float r = fmaf(x, 0x1.4ae0bep-26f, fmaf(x, 0x1.715476p+0f, -t));
  const float p = __builtin_amdgcn_exp2f(t);
  return fmaf(p, r * 0x1.62e430p-1f, p);
}

template <int NV>
__device__ __forceinline__ void local_best(const uint32_t (&key)[NV], uint32_t& bk, int& bp) {
  bk = key[0];
  bp = 0;
#pragma unroll
  for (int i = 1; i < NV; ++i)
    if (key[i] > bk) {
      bk = key[i];
      bp = i;
    }
}

// Slots from which select_bits finds them, rather than one maximum after another: its time hardly depends on topk, theirs
// does. Router with balance sums and gradients, bits against maxima: 16381 tokens of 64 experts, 8 slots 22.2 us against 23.4,
// 4 slots 21.0 against 20.5; 256 experts, 16 slots 41.2 against 43.2, 12 slots 39.4 against 38.5; 4096 of 1024 experts, 12 slots
// 54 against 61, 4 slots 51 against 45. Router alone, 64 tokens of 1024 experts, 8 slots 7.7 against 9.0; of 4096, 32 slots 30
// against 94.
// Tagged keys make a maximum cheaper: in bfloat16 with gradients, bits against maxima at 8192 tokens of 64 experts, 32 slots 20.4
// and 24.1 us, of 256 experts, 32 slots 28.5 and 30.8, 16 slots 26.0 and 24.0; 1024 tokens of 4096 experts, 64 slots 128 and 140,
// 32 slots 125 and 106.
constexpr int select_bits_from(int nv, bool tagged) { return tagged ? (nv <= 8 ? 32 : 64) : nv == 4 || nv == 8 ? 16 : 8; }

// The topk largest keys of a wave, and which experts have them: lane j < topk ends with one (key 0, id -1 for none) and its rank
// in `slot`. The topk-th largest key is found bit by bit from the top (a comparison a key and bit, counts in scalar registers; it
// ends as soon as exactly topk keys are left); those from it on go to the first lanes in the order of their ids, through LDS, and each
// counts the ones before it.
template <int NV>
__device__ __forceinline__ void select_bits(const uint32_t (&key)[NV], int topk, int lane, uint2* s_top, uint32_t& sel, int& id,
                                            int& slot) {
  uint32_t low = 0;
  int have = 0;  // keys >= low, once counted
  for (uint32_t bit = 0x80000000u; bit != 0; bit >>= 1) {
    const uint32_t c = low | bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) n += __builtin_popcountll(__ballot(key[i] >= c));
    if (n >= topk) {
      low = c;
      have = n;
      if (n == topk) break;
    }
  }
  low = max(low, 1u);  // (fewer than topk can be chosen: all of them)
  int spare = 0;       // equal keys that are too many, the last ids first
  if (have > topk) spare = have - topk;
  int at = 0;  // of the lane's first chosen one
  uint64_t on[NV];
  if (spare == 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) on[i] = __ballot(key[i] >= low);
  } else {
    int above = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) above += __builtin_popcountll(__ballot(key[i] > low));
    int eq = 0;  // equal ones before the lane's
#pragma unroll
    for (int i = 0; i < NV; ++i) eq += lanes_below(__ballot(key[i] == low));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      on[i] = __ballot(key[i] > low || (key[i] == low && eq < topk - above));
      eq += key[i] == low;
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) at += lanes_below(on[i]);
  if (lane < topk) s_top[lane] = uint2{0u, ~0u};
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (on[i] >> lane & 1) s_top[at++] = uint2{key[i], (uint32_t)(lane * NV + i)};
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const uint2 v = lane < topk ? s_top[lane] : uint2{0u, ~0u};
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  sel = v.x;
  id = (int)v.y;
  slot = 0;
  for (int j = 0; j < topk; ++j) {
    const uint32_t k = (uint32_t)readlane_i((int)sel, j);
    slot += k > sel || (k == sel && j < lane);
  }
}

// Workspace of the balance pass: ticket, token counts and probability sums and expert counts per
// workgroup, loss parts per join workgroup.
struct RouteWs {
  size_t parts, live, psum, cnt, total;
};
static int route_groups(int64_t t, int E) {
  const int per = balance_waves(lane_experts(E)) * kRouteTokensPerWave;
  const int64_t g = (t + per - 1) / per;
  return (int)(g < 1 ? 1 : g > kRouteMaxGroups ? kRouteMaxGroups : g);
}
static RouteWs route_ws(int64_t t, int E) {
  const size_t g = (size_t)route_groups(t, E);
  RouteWs w;
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  w.parts = 256;
  w.live = w.parts + up((size_t)((E + kJoinCols - 1) / kJoinCols) * 8);
  w.psum = w.live + up(g * 4);
  w.cnt = w.psum + up(g * E * 4);
  w.total = w.cnt + up(g * E * 4);
  return w;
}

// BAL: a workgroup's probability and slot counts stay in registers and LDS over all its tokens, and at most kRouteMaxGroups workgroups
// leave them to the join: 16381 tokens of 256 experts in bfloat16, 8 slots (17 MB with the gradient, 3.4 us of memory time) 17 us
// (19.4 with untagged keys, 1.2 of them a slot); the join 4.7, the gradient 10.8.
template <typename T, int NV, int ROW, bool BAL>
__global__ __launch_bounds__((BAL ? balance_waves(NV) : kRouteWaves) * 64) void k_route(const T* __restrict__ logits, int64_t t, int E,
                                                            const uint8_t* __restrict__ mask, bool masked, int topk,
                                                            int renorm, int32_t* __restrict__ idx, float* __restrict__ w,
                                                            uint8_t* __restrict__ ws, RouteWs L) {
  constexpr int WV = BAL ? balance_waves(NV) : kRouteWaves;
  constexpr bool kTagged = sizeof(T) == 2;
  __shared__ uint2 s_top[WV][kRouteMaxTopk];
  __shared__ float s_p[BAL ? NV * 64 : 1];
  __shared__ int s_c[BAL ? NV * 64 : 1];
  __shared__ int s_live;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float psum[BAL ? NV : 1];
  int live = 0;
  if constexpr (BAL) {
    for (int i = threadIdx.x; i < NV * 64; i += WV * 64) s_c[i] = 0;
    if (threadIdx.x == 0) s_live = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) psum[i] = 0.0f;
    __syncthreads();
  }
  Logits<ROW, T, NV> row;
  uint8_t here;
  const int64_t first = (int64_t)blockIdx.x * WV + wave, step = (int64_t)gridDim.x * WV;
  if (first < t) {
    row.load(logits + first * E, lane, E);
    here = mask[first];
  }
  for (int64_t tok = first; tok < t; tok += step) {
    uint32_t key[NV];
    const bool on = here != 0 || !masked;
    row.template keys<kTagged>(lane, E, on, key);
    if constexpr (BAL) {  // (without a branch, at which the compiler would wait for them: the last token's again at the end)
      const int64_t next = tok + step < t ? tok + step : tok;
      row.load(logits + next * E, lane, E);
      here = mask[next];
    }
    uint32_t bk;  // the lane's candidate
    int bp;
    local_best(key, bk, bp);
    const uint32_t top = wave_max_u32(bk);
    const float m = value_of<kTagged>(top);
    float z = 1.0f;
    if (top != 0 && (BAL || !renorm)) {
      float ex[NV], s = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        ex[i] = key[i] ? exp_below(value_of<kTagged>(key[i]) - m) : 0.0f;
        s += ex[i];
      }
      z = wave_sum_f32(s);
      if (!(fabsf(m) < __builtin_huge_valf())) z = __builtin_nanf("");
      if constexpr (BAL) {
        const float inv = 1.0f / z;
#pragma unroll
        for (int i = 0; i < NV; ++i) psum[i] = fmaf(ex[i], inv, psum[i]);
      }
    }
    live += on;
    uint32_t sel = 0;
    int id = -1, slot = lane;
    if (topk >= select_bits_from(NV, kTagged) && top != 0) {
      select_bits(key, topk, lane, s_top[wave], sel, id, slot);
    } else if constexpr (kTagged) {
      for (int r = 0; r < topk; ++r) {
        const uint32_t best = r == 0 ? top : wave_max_u32(bk);
        if (best == 0) break;
        sel = lane == r ? best : sel;
        bk = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          key[i] = key[i] == best ? 0 : key[i];
          bk = max(bk, key[i]);
        }
      }
      id = sel ? (int)(kTag - (sel & kTag)) : -1;
    } else {
      for (int r = 0; r < topk; ++r) {
        const uint32_t best = r == 0 ? top : wave_max_u32(bk);
        if (best == 0) break;
        const int from = __builtin_ctzll(__ballot(bk == best));
        const int at = readlane_i(bp, from);
        if (lane == r) {
          sel = best;
          id = from * NV + at;
        }
        if (lane == from) {
#pragma unroll
          for (int i = 0; i < NV; ++i)
            if (i == at) key[i] = 0;
          local_best(key, bk, bp);
        }
      }
    }
    float p = sel ? exp_below(value_of<kTagged>(sel) - m) : 0.0f;
    if (renorm) {
      z = top ? wave_sum_f32(p) : 1.0f;
      if (top && !(fabsf(m) < __builtin_huge_valf())) z = __builtin_nanf("");
    }
    p = sel ? p / z : 0.0f;
    if (lane < topk) {
      idx[tok * topk + slot] = id;
      w[tok * topk + slot] = p;
    }
    if constexpr (BAL) {
      if (id >= 0) atomicAdd(&s_c[id], 1);
    }
  }
  if constexpr (BAL) {
    // the waves' sums one after the other: their order does not change
    for (int v = 0; v < WV; ++v) {
      if (wave == v) {
#pragma unroll
        for (int i = 0; i < NV; ++i) s_p[lane * NV + i] = v == 0 ? psum[i] : s_p[lane * NV + i] + psum[i];
        if (lane == 0) s_live += live;
      }
      __syncthreads();
    }
    float* gp = reinterpret_cast<float*>(ws + L.psum) + (int64_t)blockIdx.x * E;
    int* gc = reinterpret_cast<int*>(ws + L.cnt) + (int64_t)blockIdx.x * E;
    for (int i = threadIdx.x; i < E; i += WV * 64) {
      gp[i] = s_p[i];
      gc[i] = s_c[i];
    }
    if (threadIdx.x == 0) {
      reinterpret_cast<int*>(ws + L.live)[blockIdx.x] = s_live;
      if (blockIdx.x == 0) *reinterpret_cast<uint32_t*>(ws) = 0;  // the join's ticket
    }
  }
}

// Joins the workgroups' sums, 16 experts a workgroup, in fp64 in a fixed order. The workgroup that
// takes the last ticket adds the loss parts (in order, whichever workgroup it is).
__global__ __launch_bounds__(kJoinCols * kJoinRows) void k_route_join(uint8_t* __restrict__ ws, RouteWs L, int groups, int E,
                                                                      int topk, float alpha,
                                                                      int32_t* __restrict__ counts,
                                                                      float* __restrict__ p_mean,
                                                                      float* __restrict__ coef, float* __restrict__ loss) {
  constexpr int N = kJoinCols * kJoinRows;
  __shared__ double s_p[N];
  __shared__ int s_c[N];
  __shared__ int s_l[N];
  __shared__ bool s_last;
  const int tid = threadIdx.x, col = blockIdx.x * kJoinCols + tid % kJoinCols, row = tid / kJoinCols;
  const float* gp = reinterpret_cast<const float*>(ws + L.psum);
  const int* gc = reinterpret_cast<const int*>(ws + L.cnt);
  double p = 0.0;
  int c = 0;
  if (col < E) {
#pragma unroll
    for (int k = 0; k < kRouteMaxGroups / kJoinRows; ++k) {
      const int g = row + k * kJoinRows;
      const int64_t at = (int64_t)min(g, groups - 1) * E + col;
      const float pv = gp[at];
      const int cv = gc[at];
      p += g < groups ? (double)pv : 0.0;
      c += g < groups ? cv : 0;
    }
  }
  s_p[tid] = p;
  s_c[tid] = c;
  s_l[tid] = tid < groups ? reinterpret_cast<const int*>(ws + L.live)[tid] : 0;  // (at most kRouteMaxGroups <= N of them)
  __syncthreads();
  for (int h = N / 2; h >= 1; h >>= 1) {  // columns join down to 16 lanes, the token count to one
    if (tid < h) {
      s_l[tid] += s_l[tid + h];
      if (h >= kJoinCols) {
        s_p[tid] += s_p[tid + h];
        s_c[tid] += s_c[tid + h];
      }
    }
    __syncthreads();
  }
  const double tv = (double)s_l[0];
  double part = 0.0;
  if (tid < kJoinCols && col < E) {
    const double f = tv > 0.0 ? (double)alpha * E * s_c[tid] / (topk * tv * tv) : 0.0;
    counts[col] = s_c[tid];
    p_mean[col] = tv > 0.0 ? (float)(s_p[tid] / tv) : 0.0f;
    coef[col] = (float)f;
    part = f * s_p[tid];
  }
  __syncthreads();
  s_p[tid] = part;  // (0 past the columns)
  __syncthreads();
  double* parts = reinterpret_cast<double*>(ws + L.parts);
  if (tid == 0) {
    double v = 0.0;
    for (int i = 0; i < kJoinCols; ++i) v += s_p[i];
    __hip_atomic_store(parts + blockIdx.x, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = __hip_atomic_fetch_add(reinterpret_cast<uint32_t*>(ws), 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 == gridDim.x;
  }
  __syncthreads();
  if (!s_last) return;
  // (at most 256 parts: read at once, added in order)
  s_p[tid] = tid < (int)gridDim.x ? __hip_atomic_load(parts + tid, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
  __syncthreads();
  if (tid == 0) {
    double sum = 0.0;
    for (unsigned i = 0; i < gridDim.x; ++i) sum += s_p[i];
    *loss = (float)sum;
  }
}

// Gradient by the logits: the probabilities again from the logits (cheaper than a [t][E] tensor written and read). The slots' terms
// reach their experts' lanes through LDS. A wave per token. dlogits may be logits: neither is restrict, and the wave has read its
// row before it writes it.
template <typename T, int NV, int ROW>
__global__ __launch_bounds__(kRouteWaves * 64) void k_route_bwd(const T* logits, int64_t t, int E,
                                                                const uint8_t* mask, bool masked, int topk, int renorm,
                                                                const int32_t* __restrict__ idx,
                                                                const float* __restrict__ w, const float* dw, bool slots,
                                                                const float* coef, int coefs, const float* dloss,
                                                                T* dlogits) {
  __shared__ float s_g[kRouteWaves][NV * 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t tok = (int64_t)blockIdx.x * kRouteWaves + wave;
  if (tok >= t) return;
  float* g = s_g[wave];
#pragma unroll
  for (int i = 0; i < NV; ++i) g[lane * NV + i] = 0.0f;
  const float dl = coefs ? dloss[0] : 0.0f;
  uint32_t key[NV];
  Logits<ROW, T, NV> row;
  row.load(logits + tok * E, lane, E);
  const int64_t slot = tok * topk + min(lane, topk - 1);
  int e = idx[slot];
  float wj = w[slot], dj = dw[slot], c[NV];
  auto load_coef = [&] {
#pragma unroll
    for (int i = 0; i < NV; ++i) c[i] = coef[max(min(lane * NV + i, coefs - 1), 0)];
  };
  if constexpr (NV <= 16) load_coef();  // (registers)
  row.template keys<false>(lane, E, mask[tok] != 0 || !masked, key);
  uint32_t bk = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) bk = max(bk, key[i]);
  const uint32_t top = wave_max_u32(bk);
  const float m = route_value(top);
  if (!slots || lane >= topk || e < 0 || e >= E || top == 0) e = -1;
  wj = e >= 0 ? wj : 0.0f;
  dj = e >= 0 ? dj : 0.0f;
  float p[NV], s = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    p[i] = key[i] ? exp_below(route_value(key[i]) - m) : 0.0f;
    s += p[i];
  }
  float inv = top ? 1.0f / wave_sum_f32(s) : 0.0f;
  if (top && !(fabsf(m) < __builtin_huge_valf())) inv = __builtin_nanf("");
  const float sw = wave_sum_f32(wj * dj);
  if (e >= 0) atomicAdd(&g[e], renorm ? wj * (dj - sw) : dj);
  s = 0.0f;
  if constexpr (NV > 16) load_coef();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    p[i] *= inv;
    c[i] = lane * NV + i < coefs ? dl * c[i] : 0.0f;
    s = fmaf(p[i], c[i], s);
  }
  const float sc = wave_sum_f32(s);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const float r = g[lane * NV + i];
    c[i] = renorm ? fmaf(p[i], c[i] - sc, r) : p[i] * (c[i] + r - (sc + sw));
    if (!key[i]) c[i] = 0.0f;
  }
  constexpr int C = NV < 4 ? NV : 4;
#pragma unroll
  for (int i = 0; i < NV; i += C) {
    float o[C];
#pragma unroll
    for (int k = 0; k < C; ++k) o[k] = c[i + k];
    store_row<ROW, C>(dlogits + tok * E, lane * NV + i, E, o);
  }
}

// Gradient of the layer's output by the routing weights: dw[s] = <dout[token of s], yd[s]>.
// A wave per slot; where that leaves compute units without a workgroup, the four waves of one share a slot. Bound by the
// read of yd: 2048 tokens of 8 slots, hidden 4096 (302 MB) 50 us, 6.1 TB/s. Shared against not, yd not in a cache, hidden 7168: 128
// slots 3.9 and 4.7 us, 512 7.2 and 7.7, 768 8.9 and 8.7, 1024 10.8 and 8.8; hidden 4096: 128 3.1 and 3.6, 512 5.3 both, 1024 7.6 and
// 6.3; hidden 1024: 128 2.6 and 2.3, 512 3.0 and 2.7.
constexpr int kSharedSlots = 512;
template <bool SHARE>
__global__ __launch_bounds__(256) void k_weight_grad(const float* __restrict__ yd, const float* __restrict__ dout,
                                                     const int32_t* __restrict__ idx, int64_t slot0, int64_t slots, int topk,
                                                     int H, int E, float* __restrict__ dw) {
  __shared__ float s_v[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t slot = slot0 + (SHARE ? blockIdx.x : (int64_t)blockIdx.x * 4 + wave);
  if (slot >= slots) return;
  const int e = idx[slot];
  const float* row = yd + slot * H;
  const float* d = dout + slot / topk * H;
  // (sums a lane, at 4096 columns: two, an error against 64 bits of 1.3e-7; one 1.6e-7; four 1.1e-7 in 1 % more time)
  float part[2] = {};
  if (e >= 0 && e < E) {  // an unrouted slot's row is never read
#pragma unroll 4
    for (int c = (SHARE ? wave * 256 : 0) + lane * 4; c < H; c += SHARE ? 1024 : 256) {  // (H is a multiple of 256)
      float a[4], b[4];
      load_n<4>(d + c, a);
      load_n<4>(row + c, b);
#pragma unroll
      for (int i = 0; i < 4; ++i) part[i & 1] = fmaf(a[i], b[i], part[i & 1]);
    }
  }
  float acc = wave_sum_f32(part[0] + part[1]);
  if constexpr (SHARE) {
    if (lane == 0) s_v[wave] = acc;
    __syncthreads();
    acc = (s_v[0] + s_v[1]) + (s_v[2] + s_v[3]);
    if (threadIdx.x == 0) dw[slot] = acc;
  } else if (lane == 0) {
    dw[slot] = acc;
  }
}

// Calls f with the experts a lane holds and how its vectors (of up to four) lie in a row.
template <typename F>
static void with_experts(int E, F f) {
  auto go = [&](auto nv) {
    constexpr int C = decltype(nv)::value < 4 ? decltype(nv)::value : 4;  // (C = 1, or E > 64)
    if (E % C == 0) f(nv, std::integral_constant<int, kRowWhole>{});
    else if constexpr (C > 1) f(nv, std::integral_constant<int, kRowTail>{});
  };
  switch (lane_experts(E)) {
    case 1: return go(std::integral_constant<int, 1>{});
    case 2: return go(std::integral_constant<int, 2>{});
    case 4: return go(std::integral_constant<int, 4>{});
    case 8: return go(std::integral_constant<int, 8>{});
    case 16: return go(std::integral_constant<int, 16>{});
    default: return go(std::integral_constant<int, 64>{});
  }
}

static tq_status check_route(const char* fn, const void* logits, int32_t type, int64_t t, int32_t E, int32_t topk,
                             int32_t flags, const void* idx, const void* w) {
  if (!known_type(type)) return fail(TQ_ERR_INVALID, "%s: unknown type %d", fn, type);
  if (t < 0 || t > (1 << 24)) return fail(TQ_ERR_INVALID, "%s: t = %lld outside [0, 2^24]", fn, (long long)t);
  if (E < 1 || E > kRouteMaxExperts) return fail(TQ_ERR_INVALID, "%s: n_experts = %d outside [1, %d]", fn, E, kRouteMaxExperts);
  if (topk < 1 || topk > kRouteMaxTopk || topk > E)
    return fail(TQ_ERR_INVALID, "%s: topk = %d outside [1, min(%d, n_experts)]", fn, topk, kRouteMaxTopk);
  if (flags & ~TQ_ROUTE_RENORM) return fail(TQ_ERR_INVALID, "%s: bad flags 0x%x", fn, flags);
  if (t == 0) return TQ_OK;
  if (!logits || !idx || !w) return fail(TQ_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(logits, type_bytes(type)) || !aligned(idx, 4) || !aligned(w, 4))
    return fail(TQ_ERR_ALIGN, "%s: logits must be aligned to their type, topk_idx and topk_w 4-byte aligned", fn);
  return TQ_OK;
}

template <bool BAL>
static void launch_route(const void* logits, int32_t type, int64_t t, int32_t E, const uint8_t* mask, int32_t topk,
                         int32_t flags, int32_t* idx, float* w, void* ws, unsigned groups, hipStream_t st) {
  with_type(type, [&](auto tv) {
    using T = decltype(tv);
    with_experts(E, [&](auto nv, auto row) {
      hipLaunchKernelGGL((k_route<T, decltype(nv)::value, decltype(row)::value, BAL>), dim3(groups),
                         dim3((BAL ? balance_waves(decltype(nv)::value) : kRouteWaves) * 64), 0, st,
                         static_cast<const T*>(logits), t, E, mask ? mask : reinterpret_cast<const uint8_t*>(logits), mask != nullptr,
                         topk, flags & TQ_ROUTE_RENORM, idx, w,
                         static_cast<uint8_t*>(ws), BAL ? route_ws(t, E) : RouteWs{});
    });
  });
}

}  // namespace tq

extern "C" tq_status tq_route(const void* logits, int32_t type, int64_t t, int32_t n_experts,
                              const uint8_t* token_mask, int32_t topk, int32_t flags, int32_t* topk_idx,
                              float* topk_w, void* stream) {
  using namespace tq;
  clear_error();
  tq_status st = check_route("tq_route", logits, type, t, n_experts, topk, flags, topk_idx, topk_w);
  if (st != TQ_OK || t == 0) return st;
  (void)hipGetLastError();
  const unsigned wgs = (unsigned)((t + kRouteWaves - 1) / kRouteWaves);
  launch_route<false>(logits, type, t, n_experts, token_mask, topk, flags, topk_idx, topk_w, nullptr, wgs,
                      (hipStream_t)stream);
  return check_launch("tq_route");
}

extern "C" size_t tq_route_workspace_bytes(int64_t t, int32_t n_experts) {
  if (t < 0 || t > (1 << 24) || n_experts < 1 || n_experts > tq::kRouteMaxExperts) return 0;
  return tq::route_ws(t, n_experts).total;
}

extern "C" tq_status tq_route_balance(const void* logits, int32_t type, int64_t t, int32_t n_experts,
                                      const uint8_t* token_mask, int32_t topk, int32_t flags, float alpha,
                                      int32_t* topk_idx, float* topk_w, int32_t* counts, float* p_mean, float* coef,
                                      float* loss, void* ws, size_t ws_bytes, void* stream) {
  using namespace tq;
  clear_error();
  const char* fn = "tq_route_balance";
  tq_status st = check_route(fn, logits, type, t, n_experts, topk, flags, topk_idx, topk_w);
  if (st != TQ_OK) return st;
  if (!counts || !p_mean || !coef || !loss || !ws) return fail(TQ_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(counts, 4) || !aligned(p_mean, 4) || !aligned(coef, 4) || !aligned(loss, 4) || !aligned(ws, 256))
    return fail(TQ_ERR_ALIGN, "%s: outputs must be 4-byte aligned, ws 256-byte aligned", fn);
  const RouteWs L = route_ws(t, n_experts);
  if (ws_bytes < L.total)
    return fail(TQ_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, L.total);
  (void)hipGetLastError();
  const int groups = route_groups(t, n_experts);
  launch_route<true>(logits, type, t, n_experts, token_mask, topk, flags, topk_idx, topk_w, ws, (unsigned)groups,
                     (hipStream_t)stream);
  hipLaunchKernelGGL(k_route_join, dim3((unsigned)((n_experts + kJoinCols - 1) / kJoinCols)), dim3(kJoinCols * kJoinRows),
                     0, (hipStream_t)stream, static_cast<uint8_t*>(ws), L, groups, n_experts, topk, alpha, counts, p_mean,
                     coef, loss);
  return check_launch(fn);
}

extern "C" tq_status tq_route_bwd(const void* logits, int32_t type, int64_t t, int32_t n_experts,
                                  const uint8_t* token_mask, int32_t topk, int32_t flags, const int32_t* topk_idx,
                                  const float* topk_w, const float* dtopk_w, const float* coef, const float* dloss,
                                  void* dlogits, void* stream) {
  using namespace tq;
  clear_error();
  const char* fn = "tq_route_bwd";
  tq_status st = check_route(fn, logits, type, t, n_experts, topk, flags, topk_idx, topk_w);
  if (st != TQ_OK || t == 0) return st;
  if (!dlogits || (!dtopk_w && !coef) || !coef != !dloss)
    return fail(TQ_ERR_INVALID, "%s: null dlogits, no gradient given, or one of coef and dloss alone", fn);
  if (!aligned(dlogits, type_bytes(type)) || !aligned(dtopk_w, 4) || !aligned(coef, 4) || !aligned(dloss, 4))
    return fail(TQ_ERR_ALIGN, "%s: dlogits must be aligned to its type, the others 4-byte aligned", fn);
  (void)hipGetLastError();
  const unsigned wgs = (unsigned)((t + kRouteWaves - 1) / kRouteWaves);
  // what is not there takes another address of at least its bytes: the kernel loads it and drops it
  const uint8_t* mask = token_mask ? token_mask : reinterpret_cast<const uint8_t*>(topk_idx);
  with_type(type, [&](auto tv) {
    using T = decltype(tv);
    with_experts(n_experts, [&](auto nv, auto row) {
      hipLaunchKernelGGL((k_route_bwd<T, decltype(nv)::value, decltype(row)::value>), dim3(wgs), dim3(kRouteWaves * 64), 0,
                         (hipStream_t)stream, static_cast<const T*>(logits), t, n_experts, mask, token_mask != nullptr, topk,
                         flags & TQ_ROUTE_RENORM, topk_idx, topk_w, dtopk_w ? dtopk_w : topk_w, dtopk_w != nullptr,
                         coef ? coef : topk_w, coef ? n_experts : 0, dloss, static_cast<T*>(dlogits));
    });
  });
  return check_launch(fn);
}

extern "C" tq_status tq_moe_weight_grad(const float* yd, const float* dout, int64_t t, int32_t hidden,
                                        const int32_t* topk_idx, int32_t topk, int32_t n_experts, float* dtopk_w,
                                        void* stream) {
  using namespace tq;
  clear_error();
  const char* fn = "tq_moe_weight_grad";
  if (t < 0 || t > (1 << 20)) return fail(TQ_ERR_INVALID, "%s: t = %lld outside [0, 2^20]", fn, (long long)t);
  if (hidden <= 0 || hidden % 256 != 0 || hidden > kMaxK)
    return fail(TQ_ERR_INVALID, "%s: hidden = %d must be a multiple of 256 in [256, %d]", fn, hidden, kMaxK);
  if (topk < 1 || topk > kRouteMaxTopk) return fail(TQ_ERR_INVALID, "%s: topk = %d outside [1, %d]", fn, topk, kRouteMaxTopk);
  if (n_experts < 1 || n_experts > kRouteMaxExperts)
    return fail(TQ_ERR_INVALID, "%s: n_experts = %d outside [1, %d]", fn, n_experts, kRouteMaxExperts);
  if (t == 0) return TQ_OK;
  if (!yd || !dout || !topk_idx || !dtopk_w) return fail(TQ_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(yd, 16) || !aligned(dout, 16) || !aligned(topk_idx, 4) || !aligned(dtopk_w, 4))
    return fail(TQ_ERR_ALIGN, "%s: yd and dout must be 16-byte aligned", fn);
  (void)hipGetLastError();
  const int64_t slots = t * topk;
  if (slots <= kSharedSlots) {
    hipLaunchKernelGGL(k_weight_grad<true>, dim3((unsigned)slots), dim3(256), 0, (hipStream_t)stream, yd, dout, topk_idx, (int64_t)0, slots,
                       topk, hidden, n_experts, dtopk_w);
    return check_launch(fn);
  }
  const int64_t most = items_per_launch(64);  // (a multiple of four)
  for (int64_t slot0 = 0; slot0 < slots; slot0 += most)
    hipLaunchKernelGGL(k_weight_grad<false>, dim3((unsigned)((std::min(most, slots - slot0) + 3) / 4)), dim3(256), 0, (hipStream_t)stream,
                       yd, dout, topk_idx, slot0, slots, topk, hidden, n_experts, dtopk_w);
  return check_launch(fn);
}
