// Low-rank adapters of many requests beside a shared projection (formulas in tq.h).
//
// Few tokens: each token's adapter is read by waves of its own (k_lora_shrink_row, then
// k_lora_expand_row). Many: a plan sorts the tokens by adapter, and tiles of 16 tokens of one
// adapter run on the fp32 matrix instruction 16x16x4, whose products and sums are those of fp32
// arithmetic for every adapter type.
//
// Matrix instruction operands (wave64): A row = lane & 15, B column = lane & 15, both k = lane >> 4;
// the result's column = lane & 15, its rows 4 * (lane >> 4) + j. The order of k is free as long as A and
// B agree: lane group q takes the four consecutive k's 4q .. 4q+3 of sixteen, one vector load each,
// and instruction j multiplies the j-th of them.
#include "tq_ops.hpp"

namespace tq {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kLoraMaxAdapters = 1024;
constexpr int kLoraMaxRank = 128;
constexpr int kLoraTile = 16;      // tokens of a tile
constexpr int kLoraRowTokens = 64; // up to so many tokens the row kernels run
constexpr int kPlanWaves = 8;

// What a call keeps in its workspace: the low-rank values, and the plan of its tokens. Group
// n_adapters holds the tokens without an adapter.
struct LoraWs {
  size_t low, off, order, tile_group, tile_at, total;
  int64_t tiles;  // at most
};
static LoraWs lora_ws(int n_adapters, int rank, int64_t t) {
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  LoraWs L;
  L.tiles = (t + kLoraTile - 1) / kLoraTile + (t < n_adapters + 1 ? t : n_adapters + 1);
  L.low = 0;
  L.off = up((size_t)t * rank * 4);
  L.order = L.off + up((size_t)(n_adapters + 2) * 4);
  L.tile_group = L.order + up((size_t)t * 4);
  L.tile_at = L.tile_group + up((size_t)L.tiles * 4);
  L.total = L.tile_at + up((size_t)L.tiles * 4);
  if (L.total < 256) L.total = 256;
  return L;
}

// The plan as the kernels see it.
struct LoraPlan {
  int32_t *off, *order, *tile_group, *tile_at;
};
static LoraPlan plan_of(void* ws, const LoraWs& L) {
  auto* b = static_cast<uint8_t*>(ws);
  return {reinterpret_cast<int32_t*>(b + L.off), reinterpret_cast<int32_t*>(b + L.order),
          reinterpret_cast<int32_t*>(b + L.tile_group), reinterpret_cast<int32_t*>(b + L.tile_at)};
}

__device__ __forceinline__ int adapter_of(int id, int na) { return id < 0 || id >= na ? na : id; }
__device__ __forceinline__ int live_rank(const int32_t* ranks, int a, int R) {
  return ranks ? min(max(ranks[a], 0), R) : R;
}

// Stable sort of the tokens by adapter in one workgroup: each wave counts a contiguous part of the
// tokens, the counts (group major, wave minor) become first positions, and each wave places its
// part in order. No position depends on the order of the atomics. Unused tiles get group -1.
__global__ __launch_bounds__(kPlanWaves * 64) void k_lora_plan(const int32_t* __restrict__ ids, int t, int na,
                                                               LoraPlan P, int tiles) {
  __shared__ int s_at[kPlanWaves][kLoraMaxAdapters + 1];
  __shared__ int s_tile[kLoraMaxAdapters + 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ng = na + 1;
  for (int i = tid; i < kPlanWaves * (kLoraMaxAdapters + 1); i += kPlanWaves * 64) (&s_at[0][0])[i] = 0;
  __syncthreads();
  const int chunks = (t + 63) / 64, per = (chunks + kPlanWaves - 1) / kPlanWaves;
  const int c0 = wave * per, c1 = min(c0 + per, chunks);
  for (int c = c0; c < c1; ++c)
    if (c * 64 + lane < t) atomicAdd(&s_at[wave][adapter_of(ids[c * 64 + lane], na)], 1);
  __syncthreads();
  if (wave == 0) {
    const int each = (ng + 63) / 64, g0 = lane * each, g1 = min(g0 + each, ng);
    int sum = 0, tsum = 0;
    for (int g = g0; g < g1; ++g) {
      int n = 0;
      for (int w = 0; w < kPlanWaves; ++w) n += s_at[w][g];
      sum += n;
      tsum += (n + kLoraTile - 1) / kLoraTile;
    }
    int before = sum, tbefore = tsum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int u = __shfl_up(before, d), v = __shfl_up(tbefore, d);
      if (lane >= d) before += u, tbefore += v;
    }
    before -= sum;
    tbefore -= tsum;
    for (int g = g0; g < g1; ++g) {
      P.off[g] = before;
      s_tile[g] = tbefore;
      int n = 0;
      for (int w = 0; w < kPlanWaves; ++w) {
        const int k = s_at[w][g];
        s_at[w][g] = before + n;
        n += k;
      }
      before += n;
      tbefore += (n + kLoraTile - 1) / kLoraTile;
    }
    if (lane == 63) {
      P.off[ng] = t;
      s_tile[ng] = tbefore;
    }
  }
  __syncthreads();
  // s_at[0][g] is the first position of group g until wave 0 places its part
  for (int g = tid; g < ng; g += kPlanWaves * 64) {
    const int at = s_at[0][g];
    for (int k = s_tile[g]; k < s_tile[g + 1]; ++k) {
      P.tile_group[k] = g;
      P.tile_at[k] = at + (k - s_tile[g]) * kLoraTile;
    }
  }
  for (int k = s_tile[ng] + tid; k < tiles; k += kPlanWaves * 64) P.tile_group[k] = -1;
  __syncthreads();
  for (int c = c0; c < c1; ++c) {
    const int tok = c * 64 + lane;
    const int g = tok < t ? adapter_of(ids[tok], na) : -1;
    uint64_t left = __ballot(tok < t);
    while (left) {
      const int gl = readlane_i(g, __builtin_ctzll(left));
      const uint64_t same = __ballot(g == gl);
      const int base = s_at[wave][gl];
      if (g == gl) P.order[base + __popcll(same & ((1ull << lane) - 1))] = tok;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (lane == 0) s_at[wave][gl] = base + __popcll(same);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      left &= ~same;
    }
  }
}

// ---- many tokens -----------------------------------------------------------------------------

// low[token][r] = scale * sum_c P[token][c] * M[r][c] for a tile's tokens. TR: M is stored [width][R].
// The waves split the columns in runs of 16; their sums join in LDS in order.
constexpr int kShrinkWaves = 8;
template <typename W, int RT, bool TR>
__global__ __launch_bounds__(kShrinkWaves * 64) void k_lora_shrink(const float* __restrict__ p, int width,
                                                                   const W* __restrict__ mat, int R, int na,
                                                                   const int32_t* __restrict__ ranks,
                                                                   const float* __restrict__ scale, LoraPlan P,
                                                                   float* __restrict__ low) {
  __shared__ float s_v[kShrinkWaves][16][RT * 16 + 1];
  const int g = P.tile_group[blockIdx.x];
  if (g < 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
  const int at = P.tile_at[blockIdx.x], cnt = min(P.off[g + 1] - at, kLoraTile);
  const int rl = g < na ? live_rank(ranks, g, R) : 0;
  const float sc = scale && g < na ? scale[g] : 1.0f;
  if (g < na) {
    const float* row = p + (int64_t)P.order[at + min(i, cnt - 1)] * width;  // rows past the tile's end: dropped below
    const W* m = mat + (int64_t)g * R * width;
    f32x4 acc[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) acc[rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int c = wave * 16; c < width; c += kShrinkWaves * 16) {
      float a[4], b[RT][4];
      load_row<4>(row, c + 4 * q, width, a);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int r = min(rt * 16 + i, R - 1);  // ranks past the stored ones: dropped below
        if constexpr (TR) {
#pragma unroll
          for (int j = 0; j < 4; ++j) b[rt][j] = c + 4 * q + j < width ? (float)m[(int64_t)(c + 4 * q + j) * R + r] : 0.0f;
        } else {
          load_n<4>(m + (int64_t)r * width + c + 4 * q, b[rt]);  // (width is a multiple of 256)
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[rt][j], acc[rt], 0, 0, 0);
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int j = 0; j < 4; ++j) s_v[wave][4 * q + j][rt * 16 + i] = acc[rt][j];
  }
  __syncthreads();
  for (int o = threadIdx.x; o < 16 * R; o += kShrinkWaves * 64) {
    const int tk = o / R, r = o - tk * R;
    if (tk >= cnt) break;
    float v = 0.0f;
    if (r < rl) {  // (a tile without an adapter has none)
#pragma unroll
      for (int w = 0; w < kShrinkWaves; ++w) v += s_v[w][tk][r];
      v *= sc;
    }
    low[(int64_t)P.order[at + tk] * R + r] = v;
  }
}

// out[token][c] = in[token][c] + scale * sum_r low[token][r] * M[c][r] for a tile's tokens and 64 columns a wave.
// TR: M is stored [R][width]. Row i of result tile u is column 16 (i >> 2) + 4 u + (i & 3) of the 64 (TR: 4 i + u), so that a
// lane ends with 16 consecutive columns of one token.
template <typename W, bool TR>
__global__ __launch_bounds__(256) void k_lora_expand(const float* __restrict__ low, const W* __restrict__ mat, int R,
                                                     int width, int na, const int32_t* __restrict__ ranks,
                                                     const float* __restrict__ scale, LoraPlan P, const float* in,
                                                     float* out) {
  const int g = P.tile_group[blockIdx.x];
  if (g < 0 || (g == na && in == out)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
  const int at = P.tile_at[blockIdx.x], cnt = min(P.off[g + 1] - at, kLoraTile);
  const int c0 = (blockIdx.y * 4 + wave) * 64;
  if (c0 >= width) return;
  const int64_t tok = P.order[at + min(i, cnt - 1)];
  float v[4][4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[u][j] = 0.0f;
    if (in && i < cnt) load_row<4>(in + tok * width, c0 + 16 * q + 4 * u, width, v[u]);
  }
  if (g < na) {
    const int rl = live_rank(ranks, g, R);
    const float sc = scale ? scale[g] : 1.0f;
    const W* m = mat + (int64_t)g * R * width;
    f32x4 acc[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) acc[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int r0 = 0; r0 < rl; r0 += 16) {
      const int r = r0 + 4 * q;
      float l[4], b[4][4];  // b[u][j]: rank r + j of the lane's column of tile u
      load_row<4>(low + tok * R, r, rl, l);
      if constexpr (TR) {
        const int c = min(c0 + 4 * i, width - 4);  // (width is a multiple of 256)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float w[4] = {};
          if (r + j < rl) load_n<4>(m + (int64_t)(r + j) * width + c, w);
#pragma unroll
          for (int u = 0; u < 4; ++u) b[u][j] = w[u];
        }
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int c = min(c0 + 16 * (i >> 2) + 4 * u + (i & 3), width - 1);
          load_row<4>(m + (int64_t)c * R, r, rl, b[u]);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[u][j], l[j], acc[u], 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float& o = TR ? v[j][u] : v[u][j];
        o = fmaf(sc, acc[u][j], o);
      }
  }
  if (i < cnt) {
#pragma unroll
    for (int u = 0; u < 4; ++u) store_row<4>(out + tok * width, c0 + 16 * q + 4 * u, width, v[u]);
  }
}

// G = scale * sum over an adapter's tokens of P[token][c] * low[token][r], 64 columns a workgroup, written [width][R] (TR) or
// [R][width]. The waves take the tokens in turns of four; their sums join in LDS in order. Column 4 i + u
// of the 64 is row i of result tile u. An adapter without tokens gets zeros.
constexpr int kOuterWaves = 8;
template <int RT, bool TR>
__global__ __launch_bounds__(kOuterWaves * 64) void k_lora_outer(const float* __restrict__ p, int width,
                                                                 const float* __restrict__ low, int R,
                                                                 const int32_t* __restrict__ ranks,
                                                                 const float* __restrict__ scale, LoraPlan P,
                                                                 float* __restrict__ grad) {
  __shared__ float s_g[RT * 16][65];
  const int g = blockIdx.y, c0 = blockIdx.x * 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
  const int at = P.off[g], cnt = P.off[g + 1] - at;
  const int rl = cnt > 0 ? live_rank(ranks, g, R) : 0;
  f32x4 acc[4][RT];
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) acc[u][rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (rl > 0) {
#pragma unroll 2
    for (int k = wave * 4; k < cnt; k += kOuterWaves * 4) {
      const bool on = k + q < cnt;
      const int64_t tok = P.order[at + min(k + q, cnt - 1)];
      float a[4], b[RT];
      load_row<4>(p + tok * width, c0 + 4 * i, width, a);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) b[rt] = on && rt * 16 + i < rl ? low[tok * R + rt * 16 + i] : 0.0f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float au = on ? a[u] : 0.0f;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[u][rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(au, b[rt], acc[u][rt], 0, 0, 0);
      }
    }
  }
  for (int w = 0; w < kOuterWaves; ++w) {
    if (wave == w) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float& s = s_g[rt * 16 + i][16 * q + 4 * j + u];
            s = w == 0 ? acc[u][rt][j] : s + acc[u][rt][j];
          }
    }
    __syncthreads();
  }
  const float sc = scale ? scale[g] : 1.0f;
  grad += (int64_t)g * R * width;
  for (int o = threadIdx.x; o < 64 * R; o += kOuterWaves * 64) {
    const int r = TR ? o % R : o >> 6, c = TR ? o / R : o & 63;
    if (c0 + c < width) grad[TR ? (int64_t)(c0 + c) * R + r : (int64_t)r * width + c0 + c] = r < rl ? sc * s_g[r][c] : 0.0f;
  }
}

// ---- few tokens ------------------------------------------------------------------------------

// low[token][r] = A[r] x[token]: a wave takes two ranks of a token, 8 columns a lane and step.
template <typename W>
__global__ __launch_bounds__(256) void k_lora_shrink_row(const float* __restrict__ x, int k, const W* __restrict__ a,
                                                         int R, int na, const int32_t* __restrict__ ids,
                                                         const int32_t* __restrict__ ranks, float* __restrict__ low) {
  const int lane = threadIdx.x & 63, r0 = (blockIdx.y * 4 + (threadIdx.x >> 6)) * 2;
  const int64_t tok = blockIdx.x;
  if (r0 >= R) return;
  const int g = adapter_of(ids[tok], na);
  const int rl = g < na ? live_rank(ranks, g, R) : 0;
  float s0 = 0.0f, s1 = 0.0f;
  if (r0 < rl) {
    const W* m = a + ((int64_t)g * R + r0) * k;  // (R is even: row r0 + 1 is stored)
    const float* row = x + tok * k;
#pragma unroll 4
    for (int c = lane * 8; c < k; c += 512) {
      float xv[8], w0[8], w1[8];
      load_n<8>(row + c, xv);
      load_n<8>(m + c, w0);
      load_n<8>(m + k + c, w1);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s0 = fmaf(xv[i], w0[i], s0);
        s1 = fmaf(xv[i], w1[i], s1);
      }
    }
  }
  s0 = wave_sum_f32(s0);
  s1 = wave_sum_f32(s1);
  if (lane == 0) {
    low[tok * R + r0] = r0 < rl ? s0 : 0.0f;
    low[tok * R + r0 + 1] = r0 + 1 < rl ? s1 : 0.0f;
  }
}

// out[token][c] = in[token][c] + scale * <low[token], B[c]>: a thread per column.
template <typename W>
__global__ __launch_bounds__(256) void k_lora_expand_row(const float* __restrict__ low, const W* __restrict__ b, int R,
                                                         int n, int na, const int32_t* __restrict__ ids,
                                                         const int32_t* __restrict__ ranks,
                                                         const float* __restrict__ scale, const float* in, float* out) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  const int64_t tok = blockIdx.y;
  const int g = adapter_of(ids[tok], na);
  if (c >= n || (g == na && in == out)) return;
  float v = in ? in[tok * n + c] : 0.0f;
  if (g < na) {
    const int rl = live_rank(ranks, g, R);
    const float sc = scale ? scale[g] : 1.0f;
    const W* m = b + ((int64_t)g * n + c) * R;
    const float* l = low + tok * R;
    float s = 0.0f;
#pragma unroll 2
    for (int r = 0; r < rl; r += 8) {
      float w[8];
      load_n<8>(m + r, w);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r + i < rl) s = fmaf(l[r + i], w[i], s);
    }
    v = fmaf(sc, s, v);
  }
  out[tok * n + c] = v;
}

template <typename F>
static void with_rank(int R, F f) {
  if (R <= 16) f(std::integral_constant<int, 1>{});
  else if (R <= 32) f(std::integral_constant<int, 2>{});
  else if (R <= 64) f(std::integral_constant<int, 4>{});
  else f(std::integral_constant<int, 8>{});
}

static tq_status check_adapters(const char* fn, const tq_adapters* ad, int64_t t) {
  if (!ad) return fail(TQ_ERR_INVALID, "%s: null adapters descriptor", fn);
  if (!known_type(ad->type)) return fail(TQ_ERR_INVALID, "%s: unknown type %d", fn, ad->type);
  if (ad->n_adapters < 1 || ad->n_adapters > kLoraMaxAdapters)
    return fail(TQ_ERR_INVALID, "%s: n_adapters = %d outside [1, %d]", fn, ad->n_adapters, kLoraMaxAdapters);
  if (ad->rank < 8 || ad->rank % 8 != 0 || ad->rank > kLoraMaxRank)
    return fail(TQ_ERR_INVALID, "%s: rank = %d must be a multiple of 8 in [8, %d]", fn, ad->rank, kLoraMaxRank);
  if (ad->n < 1 || ad->n > (1 << 20)) return fail(TQ_ERR_INVALID, "%s: n = %d outside [1, 2^20]", fn, ad->n);
  if (ad->k <= 0 || ad->k % 256 != 0 || ad->k > kMaxK)
    return fail(TQ_ERR_INVALID, "%s: k = %d must be a multiple of 256 in [256, %d]", fn, ad->k, kMaxK);
  if (t < 0 || t > (1 << 20)) return fail(TQ_ERR_INVALID, "%s: t = %lld outside [0, 2^20]", fn, (long long)t);
  return TQ_OK;
}

static tq_status check_tensors(const char* fn, const tq_adapters* ad, const void* ws, size_t ws_bytes, int64_t t) {
  if (!ad->a || !ad->b || !ws) return fail(TQ_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(ad->a, 16) || !aligned(ad->b, 16) || !aligned(ad->scale, 4) || !aligned(ad->ranks, 4) || !aligned(ws, 256))
    return fail(TQ_ERR_ALIGN, "%s: a and b must be 16-byte aligned, scale and ranks 4-byte, ws 256-byte aligned", fn);
  const LoraWs L = lora_ws(ad->n_adapters, ad->rank, t);
  if (ws_bytes < L.total)
    return fail(TQ_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, L.total);
  return TQ_OK;
}

static void launch_plan(const int32_t* ids, int64_t t, int na, const LoraPlan& P, const LoraWs& L, hipStream_t st) {
  hipLaunchKernelGGL(k_lora_plan, dim3(1), dim3(kPlanWaves * 64), 0, st, ids, (int)t, na, P, (int)L.tiles);
}

}  // namespace tq

extern "C" size_t tq_lora_workspace_bytes(const tq_adapters* ad, int64_t t) {
  using namespace tq;
  if (check_adapters("tq_lora_workspace_bytes", ad, t) != TQ_OK) return 0;
  return lora_ws(ad->n_adapters, ad->rank, t).total;
}

extern "C" tq_status tq_lora(const tq_adapters* ad, const float* x, int64_t t, const int32_t* ids, const float* y,
                             float* out, float* v, void* ws, size_t ws_bytes, void* stream) {
  using namespace tq;
  clear_error();
  const char* fn = "tq_lora";
  tq_status st = check_adapters(fn, ad, t);
  if (st != TQ_OK || t == 0) return st;
  if (!x || !ids || !out) return fail(TQ_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(x, 16) || !aligned(ids, 4) || !aligned(y, 4) || !aligned(out, 4) || !aligned(v, 4))
    return fail(TQ_ERR_ALIGN, "%s: x must be 16-byte aligned, the others 4-byte aligned", fn);
  if ((st = check_tensors(fn, ad, ws, ws_bytes, t)) != TQ_OK) return st;
  (void)hipGetLastError();
  const hipStream_t hs = (hipStream_t)stream;
  const LoraWs L = lora_ws(ad->n_adapters, ad->rank, t);
  const LoraPlan P = plan_of(ws, L);
  float* low = v ? v : reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + L.low);
  const int R = ad->rank, n = ad->n, k = ad->k, na = ad->n_adapters;
  with_type(ad->type, [&](auto wv) {
    using W = decltype(wv);
    const W *a = static_cast<const W*>(ad->a), *b = static_cast<const W*>(ad->b);
    if (t <= kLoraRowTokens) {
      hipLaunchKernelGGL(k_lora_shrink_row<W>, dim3((unsigned)t, (unsigned)((R + 7) / 8)), dim3(256), 0, hs, x, k, a, R,
                         na, ids, ad->ranks, low);
      hipLaunchKernelGGL(k_lora_expand_row<W>, dim3((unsigned)((n + 255) / 256), (unsigned)t), dim3(256), 0, hs, low, b,
                         R, n, na, ids, ad->ranks, ad->scale, y, out);
      return;
    }
    launch_plan(ids, t, na, P, L, hs);
    with_rank(R, [&](auto rt) {
      hipLaunchKernelGGL((k_lora_shrink<W, decltype(rt)::value, false>), dim3((unsigned)L.tiles),
                         dim3(kShrinkWaves * 64), 0, hs, x, k, a, R, na, ad->ranks, nullptr, P, low);
    });
    hipLaunchKernelGGL((k_lora_expand<W, false>), dim3((unsigned)L.tiles, (unsigned)((n + 255) / 256)), dim3(256), 0, hs,
                       low, b, R, n, na, ad->ranks, ad->scale, P, y, out);
  });
  return check_launch(fn);
}

extern "C" tq_status tq_lora_bwd(const tq_adapters* ad, const float* x, const float* v, const float* dy, int64_t t,
                                 const int32_t* ids, const float* dx, float* out, float* da, float* db, void* ws,
                                 size_t ws_bytes, void* stream) {
  using namespace tq;
  clear_error();
  const char* fn = "tq_lora_bwd";
  tq_status st = check_adapters(fn, ad, t);
  if (st != TQ_OK) return st;
  if (!da || !db || (t > 0 && (!x || !v || !dy || !ids)) || (dx && !out && t > 0))
    return fail(TQ_ERR_INVALID, "%s: null pointer, or dx without out", fn);
  if (!aligned(x, 16) || !aligned(v, 4) || !aligned(dy, 4) || !aligned(ids, 4) || !aligned(dx, 4) || !aligned(out, 4) ||
      !aligned(da, 4) || !aligned(db, 4))
    return fail(TQ_ERR_ALIGN, "%s: x must be 16-byte aligned, the others 4-byte aligned", fn);
  if ((st = check_tensors(fn, ad, ws, ws_bytes, t)) != TQ_OK) return st;
  (void)hipGetLastError();
  const hipStream_t hs = (hipStream_t)stream;
  const LoraWs L = lora_ws(ad->n_adapters, ad->rank, t);
  const LoraPlan P = plan_of(ws, L);
  float* u = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + L.low);
  const int R = ad->rank, n = ad->n, k = ad->k, na = ad->n_adapters;
  launch_plan(ids, t, na, P, L, hs);
  with_type(ad->type, [&](auto wv) {
    using W = decltype(wv);
    const W *a = static_cast<const W*>(ad->a), *b = static_cast<const W*>(ad->b);
    with_rank(R, [&](auto rt) {
      constexpr int RT = decltype(rt)::value;
      if (t > 0)
        hipLaunchKernelGGL((k_lora_shrink<W, RT, true>), dim3((unsigned)L.tiles), dim3(kShrinkWaves * 64), 0, hs, dy, n,
                           b, R, na, ad->ranks, ad->scale, P, u);
      hipLaunchKernelGGL((k_lora_outer<RT, true>), dim3((unsigned)((n + 63) / 64), (unsigned)na), dim3(kOuterWaves * 64), 0, hs,
                         dy, n, v, R, ad->ranks, ad->scale, P, db);
      hipLaunchKernelGGL((k_lora_outer<RT, false>), dim3((unsigned)((k + 63) / 64), (unsigned)na), dim3(kOuterWaves * 64), 0, hs,
                         x, k, u, R, ad->ranks, nullptr, P, da);
    });
    if (out && t > 0)
      hipLaunchKernelGGL((k_lora_expand<W, true>), dim3((unsigned)L.tiles, (unsigned)((k + 255) / 256)), dim3(256), 0, hs,
                         u, a, R, k, na, ad->ranks, nullptr, P, dx, out);
  });
  return check_launch(fn);
}
