// Router of the routed-expert layer: top-k selection and routing weights, per-expert counts and
// the balance loss, and their gradients (formulas in tq.h).
//
// One wave holds one token's logits, NV consecutive experts a lane, as 32-bit keys whose unsigned
// order is the logits' order. Lanes and positions ascend with the expert id, so among equal keys
// the first lane's first position is the lowest id.
#include "tq_ops.hpp"

namespace tq {

constexpr int kRouteWaves = 4;
constexpr int kRouteMaxExperts = 4096;
constexpr int kRouteMaxTopk = 64;  // lane j of the wave keeps slot j
constexpr int kRouteMaxGroups = 512;
constexpr int kRouteTokensPerWave = 4;
constexpr int kJoinCols = 16;  // experts per workgroup of the join

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

template <typename T, int NV>
__device__ __forceinline__ void load_keys(const T* row, int lane, int E, uint32_t (&key)[NV]) {
  constexpr int C = NV < 4 ? NV : 4;
#pragma unroll
  for (int c = 0; c < NV; c += C) {
    float v[C];
    load_row<C>(row, lane * NV + c, E, v, -__builtin_huge_valf());
#pragma unroll
    for (int i = 0; i < C; ++i) key[c + i] = route_key(v[i]);
  }
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

// Workspace of the balance pass: ticket, token counts and probability sums and expert counts per
// workgroup, loss parts per join workgroup.
struct RouteWs {
  size_t parts, live, psum, cnt, total;
};
static int route_groups(int64_t t) {
  const int64_t g = (t + kRouteWaves * kRouteTokensPerWave - 1) / (kRouteWaves * kRouteTokensPerWave);
  return (int)(g < 1 ? 1 : g > kRouteMaxGroups ? kRouteMaxGroups : g);
}
static RouteWs route_ws(int64_t t, int E) {
  const size_t g = (size_t)route_groups(t);
  RouteWs w;
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  w.parts = 256;
  w.live = w.parts + up((size_t)((E + kJoinCols - 1) / kJoinCols) * 8);
  w.psum = w.live + up(g * 4);
  w.cnt = w.psum + up(g * E * 4);
  w.total = w.cnt + up(g * E * 4);
  return w;
}

template <typename T, int NV, bool BAL>
__global__ __launch_bounds__(kRouteWaves * 64) void k_route(const T* __restrict__ logits, int64_t t, int E,
                                                            const uint8_t* __restrict__ mask, int topk, int renorm,
                                                            int32_t* __restrict__ idx, float* __restrict__ w,
                                                            uint8_t* __restrict__ ws, RouteWs L) {
  __shared__ float s_p[BAL ? NV * 64 : 1];
  __shared__ int s_c[BAL ? NV * 64 : 1];
  __shared__ int s_live;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float psum[BAL ? NV : 1];
  int live = 0;
  if constexpr (BAL) {
    for (int i = threadIdx.x; i < NV * 64; i += kRouteWaves * 64) s_c[i] = 0;
    if (threadIdx.x == 0) s_live = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) psum[i] = 0.0f;
    __syncthreads();
  }
  for (int64_t tok = (int64_t)blockIdx.x * kRouteWaves + wave; tok < t; tok += (int64_t)gridDim.x * kRouteWaves) {
    uint32_t key[NV];
    const bool on = !mask || mask[tok] != 0;
    load_keys<T, NV>(logits + tok * E, lane, E, key);
    if (!on) {
#pragma unroll
      for (int i = 0; i < NV; ++i) key[i] = 0;
    }
    uint32_t bk;
    int bp;
    local_best(key, bk, bp);
    const uint32_t top = wave_max_u32(bk);
    const float m = route_value(top);
    float z = 1.0f;
    if (top != 0 && (BAL || !renorm)) {
      float ex[NV], s = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        ex[i] = key[i] ? expf(route_value(key[i]) - m) : 0.0f;
        s += ex[i];
      }
      z = wave_sum_f32(s);
      if constexpr (BAL) {
        const float inv = 1.0f / z;
#pragma unroll
        for (int i = 0; i < NV; ++i) psum[i] = fmaf(ex[i], inv, psum[i]);
      }
    }
    live += on;
    uint32_t sel = 0;
    int id = -1;
    for (int r = 0; r < topk; ++r) {
      const uint32_t best = r == 0 ? top : wave_max_u32(bk);
      if (best == 0) break;
      const int from = __builtin_ctzll(__ballot(bk == best));
      const int pos = readlane_i(bp, from);
      if (lane == r) {
        sel = best;
        id = from * NV + pos;
      }
      if (lane == from) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (i == pos) key[i] = 0;
        local_best(key, bk, bp);
      }
    }
    float p = sel ? expf(route_value(sel) - m) : 0.0f;
    if (renorm) z = top ? wave_sum_f32(p) : 1.0f;
    p = sel ? p / z : 0.0f;
    if (lane < topk) {
      idx[tok * topk + lane] = id;
      w[tok * topk + lane] = p;
    }
    if constexpr (BAL) {
      if (id >= 0) atomicAdd(&s_c[id], 1);
    }
  }
  if constexpr (BAL) {
    // the waves' sums one after the other: their order does not change
    for (int v = 0; v < kRouteWaves; ++v) {
      if (wave == v) {
#pragma unroll
        for (int i = 0; i < NV; ++i) s_p[lane * NV + i] = v == 0 ? psum[i] : s_p[lane * NV + i] + psum[i];
        if (lane == 0) s_live += live;
      }
      __syncthreads();
    }
    float* gp = reinterpret_cast<float*>(ws + L.psum) + (int64_t)blockIdx.x * E;
    int* gc = reinterpret_cast<int*>(ws + L.cnt) + (int64_t)blockIdx.x * E;
    for (int i = threadIdx.x; i < E; i += kRouteWaves * 64) {
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
__global__ __launch_bounds__(256) void k_route_join(uint8_t* __restrict__ ws, RouteWs L, int groups, int E, int topk,
                                                    float alpha, int32_t* __restrict__ counts,
                                                    float* __restrict__ p_mean, float* __restrict__ coef,
                                                    float* __restrict__ loss) {
  __shared__ double s_p[256];
  __shared__ int s_c[256];
  __shared__ int s_l[256];
  __shared__ bool s_last;
  const int tid = threadIdx.x, col = blockIdx.x * kJoinCols + (tid & 15), row = tid >> 4;
  const float* gp = reinterpret_cast<const float*>(ws + L.psum);
  const int* gc = reinterpret_cast<const int*>(ws + L.cnt);
  const int* gl = reinterpret_cast<const int*>(ws + L.live);
  double p = 0.0;
  int c = 0, l = 0;
  if (col < E) {
#pragma unroll 8
    for (int g = row; g < groups; g += 16) {
      p += (double)gp[(int64_t)g * E + col];
      c += gc[(int64_t)g * E + col];
    }
  }
  for (int g = tid; g < groups; g += 256) l += gl[g];
  s_p[tid] = p;
  s_c[tid] = c;
  s_l[tid] = l;
  __syncthreads();
  for (int h = 128; h >= 1; h >>= 1) {  // columns join down to 16 lanes, the token count to one
    if (tid < h) {
      s_l[tid] += s_l[tid + h];
      if (h >= 16) {
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
  s_p[tid] = part;
  __syncthreads();
  double* parts = reinterpret_cast<double*>(ws + L.parts);
  if (tid == 0) {
    double v = 0.0;
    for (int i = 0; i < kJoinCols; ++i) v += s_p[i];
    __hip_atomic_store(parts + blockIdx.x, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const uint32_t k = __hip_atomic_fetch_add(reinterpret_cast<uint32_t*>(ws), 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    s_last = k + 1 == gridDim.x;
    if (s_last) {
      double sum = 0.0;
      for (unsigned i = 0; i < gridDim.x; ++i)
        sum += __hip_atomic_load(parts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      *loss = (float)sum;
    }
  }
}

// Gradient by the logits. The slots' terms reach their experts' lanes through LDS, whose entries
// are zero again before the next token.
template <typename T, int NV>
__global__ __launch_bounds__(kRouteWaves * 64) void k_route_bwd(const T* __restrict__ logits, int64_t t, int E,
                                                                const uint8_t* __restrict__ mask, int topk, int renorm,
                                                                const int32_t* __restrict__ idx,
                                                                const float* __restrict__ w,
                                                                const float* __restrict__ dw,
                                                                const float* __restrict__ coef,
                                                                const float* __restrict__ dloss,
                                                                T* __restrict__ dlogits) {
  __shared__ float s_g[kRouteWaves][NV * 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* g = s_g[wave];
#pragma unroll
  for (int i = 0; i < NV; ++i) g[lane * NV + i] = 0.0f;
  const float dl = coef ? dloss[0] : 0.0f;
  for (int64_t tok = (int64_t)blockIdx.x * kRouteWaves + wave; tok < t; tok += (int64_t)gridDim.x * kRouteWaves) {
    uint32_t key[NV];
    const bool on = !mask || mask[tok] != 0;
    load_keys<T, NV>(logits + tok * E, lane, E, key);
    uint32_t bk = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!on) key[i] = 0;
      bk = max(bk, key[i]);
    }
    const uint32_t top = wave_max_u32(bk);
    const float m = route_value(top);
    int e = -1;
    float wj = 0.0f, dj = 0.0f;
    if (dw && lane < topk) {
      e = idx[tok * topk + lane];
      if (e < 0 || e >= E || top == 0) e = -1;
      if (e >= 0) {
        wj = w[tok * topk + lane];
        dj = dw[tok * topk + lane];
      }
    }
    float p[NV], s = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      p[i] = key[i] ? expf(route_value(key[i]) - m) : 0.0f;
      s += p[i];
    }
    const float inv = top ? 1.0f / wave_sum_f32(s) : 0.0f;
    const float sw = wave_sum_f32(wj * dj);
    if (e >= 0) atomicAdd(&g[e], renorm ? wj * (dj - sw) : dj);
    float c[NV];
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      p[i] *= inv;
      c[i] = coef && lane * NV + i < E ? dl * coef[lane * NV + i] : 0.0f;
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
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (e >= 0) g[e] = 0.0f;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    constexpr int C = NV < 4 ? NV : 4;
#pragma unroll
    for (int i = 0; i < NV; i += C) {
      float o[C];
#pragma unroll
      for (int k = 0; k < C; ++k) o[k] = c[i + k];
      store_row<C>(dlogits + tok * E, lane * NV + i, E, o);
    }
  }
}

// Gradient of the layer's output by the routing weights: dw[s] = <dout[token of s], yd[s]>.
// Many slots: a wave takes SL slots of a token, so that a piece of dout read once serves them.
template <int SL>
__global__ __launch_bounds__(256) void k_weight_grad(const float* __restrict__ yd, const float* __restrict__ dout,
                                                     const int32_t* __restrict__ idx, int64_t t, int topk, int H,
                                                     int E, float* __restrict__ dw) {
  const int lane = threadIdx.x & 63;
  const int per = (topk + SL - 1) / SL;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t tok = unit / per;
  if (tok >= t) return;
  const int j0 = (int)(unit - tok * per) * SL;
  bool on[SL];
  float acc[SL];
  const float* row[SL];
#pragma unroll
  for (int s = 0; s < SL; ++s) {
    const int64_t slot = tok * topk + min(j0 + s, topk - 1);
    const int e = idx[slot];
    on[s] = j0 + s < topk && e >= 0 && e < E;
    acc[s] = 0.0f;
    row[s] = yd + slot * H;
  }
  const float* d = dout + tok * H;
  for (int c = lane * 4; c < H; c += 256) {  // (H is a multiple of 256: no lane leaves early)
    float a[4];
    load_n<4>(d + c, a);
#pragma unroll
    for (int s = 0; s < SL; ++s)
      if (on[s]) {  // an unrouted slot's row is never read
        float b[4];
        load_n<4>(row[s] + c, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[s] = fmaf(a[i], b[i], acc[s]);
      }
  }
#pragma unroll
  for (int s = 0; s < SL; ++s) {
    const float v = wave_sum_f32(acc[s]);
    if (lane == 0 && j0 + s < topk) dw[tok * topk + j0 + s] = on[s] ? v : 0.0f;
  }
}

// Calls f with the experts a lane holds (as a constant).
template <typename F>
static void with_experts(int E, F f) {
  if (E <= 64) f(std::integral_constant<int, 1>{});
  else if (E <= 128) f(std::integral_constant<int, 2>{});
  else if (E <= 256) f(std::integral_constant<int, 4>{});
  else if (E <= 512) f(std::integral_constant<int, 8>{});
  else if (E <= 1024) f(std::integral_constant<int, 16>{});
  else f(std::integral_constant<int, 64>{});
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
    with_experts(E, [&](auto nv) {
      hipLaunchKernelGGL((k_route<T, decltype(nv)::value, BAL>), dim3(groups), dim3(kRouteWaves * 64), 0, st,
                         static_cast<const T*>(logits), t, E, mask, topk, flags & TQ_ROUTE_RENORM, idx, w,
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
  const int groups = route_groups(t);
  launch_route<true>(logits, type, t, n_experts, token_mask, topk, flags, topk_idx, topk_w, ws, (unsigned)groups,
                     (hipStream_t)stream);
  hipLaunchKernelGGL(k_route_join, dim3((unsigned)((n_experts + kJoinCols - 1) / kJoinCols)), dim3(256), 0,
                     (hipStream_t)stream, static_cast<uint8_t*>(ws), L, groups, n_experts, topk, alpha, counts, p_mean,
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
  with_type(type, [&](auto tv) {
    using T = decltype(tv);
    with_experts(n_experts, [&](auto nv) {
      hipLaunchKernelGGL((k_route_bwd<T, decltype(nv)::value>), dim3(wgs), dim3(kRouteWaves * 64), 0,
                         (hipStream_t)stream, static_cast<const T*>(logits), t, n_experts, token_mask, topk,
                         flags & TQ_ROUTE_RENORM, topk_idx, topk_w, dtopk_w, coef, dloss, static_cast<T*>(dlogits));
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
  const int64_t units = t * topk;
  hipLaunchKernelGGL(k_weight_grad<1>, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, (hipStream_t)stream, yd, dout,
                     topk_idx, t, topk, hidden, n_experts, dtopk_w);
  return check_launch(fn);
}
