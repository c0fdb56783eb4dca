// Products of MXFP4 rows with MXFP4 weights, y = X W^T, and the gated block's two products with activation
// and elementwise product in the same pass, on the scaled fp4 matrix instructions.
//
// A lane of an instruction holds one block of 32 of one row with its scale byte, which is how the layout stores them: 16
// contiguous bytes a block, a row's blocks one after another. The order of elements within a block does not matter, both
// operands having the same. The weights are the first operand, so that a lane's results are consecutive outputs of one token.
#include <algorithm>

#include "tq_mx.hpp"

namespace tq {

// What a product writes, and the gated block's parts. gated: h, and g, u where not null.
struct MxOut {
  void *y, *g, *u;
  const float *g_add, *u_add;
  int type, act;
};

struct MxArgs {
  const uint8_t *wc[2], *ws[2];  // weights (gate, up)
  const uint8_t *xc, *xs;
  int n, t, kb;
  MxOut out;
};

// Four consecutive outputs r .. r+3 of token `tok` (those below n).
template <bool GATED>
__device__ __forceinline__ void mx_finish(const MxArgs& a, int64_t tok, int r, const float (&v)[4], const float (&w)[4]) {
  const int m = a.n - r;
  if (m <= 0) return;
  const int64_t i = tok * a.n + r;
  if constexpr (!GATED) {
    store4(a.out.type, a.out.y, i, v, m);
  } else {
    float g[4], u[4], h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      g[j] = v[j];
      u[j] = w[j];
      if (a.out.g_add && j < m) g[j] += a.out.g_add[i + j];
      if (a.out.u_add && j < m) u[j] += a.out.u_add[i + j];
      h[j] = act_fwd(a.out.act, g[j]) * u[j];
    }
    store4(a.out.type, a.out.y, i, h, m);
    if (a.out.g) {
      store4(a.out.type, a.out.g, i, g, m);
      store4(a.out.type, a.out.u, i, u, m);
    }
  }
}

// ---- few tokens: bound by the weights' bytes. A workgroup takes MT tiles of 16 rows (GATED: gate and up rows of
// the same outputs) and NT * 16 tokens; its waves share k and join through LDS, in order.
template <int MT, int NT, int NW, bool GATED>
__global__ __launch_bounds__(NW * 64) void k_mx_few(const MxArgs a) {
  static_assert(!GATED || MT == 2, "gate and up");
  __shared__ f32x4 red[NW][MT * NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int row0 = blockIdx.x * (GATED ? 16 : 16 * MT);
  const int tok0 = blockIdx.y * (NT * 16);
  const int kb = a.kb;
  // rows past the last read as zeros
  __amdgpu_buffer_rsrc_t wc[MT], ws[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int r = GATED ? row0 : row0 + 16 * m, rows = max(0, min(16, a.n - r)), s = GATED ? m : 0;
    wc[m] = make_rsrc(a.wc[s] + (int64_t)r * kb * 128, (uint32_t)(rows * kb * 128));
    ws[m] = make_rsrc(a.ws[s] + (int64_t)r * kb * 8, (uint32_t)(rows * kb * 8));
  }
  const int toks = min(NT * 16, a.t - tok0);
  const __amdgpu_buffer_rsrc_t xc = make_rsrc(a.xc + (int64_t)tok0 * kb * 128, (uint32_t)(toks * kb * 128));
  const __amdgpu_buffer_rsrc_t xs = make_rsrc(a.xs + (int64_t)tok0 * kb * 8, (uint32_t)(toks * kb * 8));

  f32x4 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const uint32_t rc = (uint32_t)(l16 * kb) * 128u + (uint32_t)g * 32u, rs = (uint32_t)(l16 * kb) * 8u + (uint32_t)g * 2u;
  for (int c = wave; c < kb; c += NW) {
    uint4 w[MT][2], x[NT][2];
    int sw[MT], sx[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      w[m][0] = buf_load16(wc[m], rc + c * 128u, 0, 0);
      w[m][1] = buf_load16(wc[m], rc + c * 128u + 16u, 0, 0);
      sw[m] = buf_load_u16(ws[m], rs + c * 8u, 0);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      x[n][0] = buf_load16(xc, rc + (uint32_t)(n * 16 * kb) * 128u + c * 128u, 0, 0);
      x[n][1] = buf_load16(xc, rc + (uint32_t)(n * 16 * kb) * 128u + c * 128u + 16u, 0, 0);
      sx[n] = buf_load_u16(xs, rs + (uint32_t)(n * 16 * kb) * 8u + c * 8u, 0);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        acc[m][n] = mfma_fp4_16<0>(w[m][0], x[n][0], acc[m][n], sw[m], sx[n]);
        acc[m][n] = mfma_fp4_16<1>(w[m][1], x[n][1], acc[m][n], sw[m], sx[n]);
      }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) red[wave][m * NT + n][lane] = acc[m][n];
  __syncthreads();
  constexpr int OUT = GATED ? NT : MT * NT;
  for (int o = wave; o < OUT; o += NW) {
    const int n = o % NT, m = o / NT;
    f32x4 s = red[0][o][lane], u = {};
    if constexpr (GATED) u = red[0][NT + o][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      s += red[w][o][lane];
      if constexpr (GATED) u += red[w][NT + o][lane];
    }
    const int tok = tok0 + 16 * n + l16, r = row0 + 16 * m + 4 * g;
    if (tok < a.t) {
      const float v[4] = {s[0], s[1], s[2], s[3]}, w[4] = {u[0], u[1], u[2], u[3]};
      mx_finish<GATED>(a, tok, r, v, w);
    }
  }
}

// ---- many tokens: tiles of BM weight rows (GATED: BM / 2 gate rows, then the up rows of the same outputs) by BN tokens,
// staged through LDS 256 elements of k at a time, two stages. A stage's row is 128 bytes, its 16-byte pieces exchanged by the
// row's low bits, so that eight rows' reads of one piece meet all banks. Scales are staged for four steps at once.
template <int BM, int BN, int WM, int WN, bool GATED>
__global__ __launch_bounds__(WM * WN * 64) void k_mx_tile(const MxArgs a) {
  constexpr int NTHR = WM * WN * 64, MT = BM / WM / 32, NT = BN / WN / 32, ROWS = BM + BN;
  constexpr int PC = ROWS * 8 / NTHR, PS = ROWS * 4 / NTHR;  // pieces a thread moves: codes (16 bytes), scales (8)
  static_assert(ROWS * 8 % NTHR == 0 && ROWS * 4 % NTHR == 0 && (!GATED || MT % 2 == 0), "tile");
  __shared__ __attribute__((aligned(16))) uint8_t sc[2][ROWS * 128];
  __shared__ __attribute__((aligned(16))) uint8_t ss[2][ROWS * 32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN, l32 = lane & 31, half = lane >> 5;
  const int kb = a.kb;
  constexpr int OUTS = GATED ? BM / 2 : BM;  // outputs of a tile
  const int row0 = blockIdx.x * OUTS, tok0 = blockIdx.y * BN;
  const int rows = min(OUTS, a.n - row0), toks = min(BN, a.t - tok0);

  // The tile row q lies in: part 0 gate (or all weights), 1 up, 2 tokens.
  const auto part = [&](int r) { return r >= BM ? 2 : GATED && r >= BM / 2 ? 1 : 0; };
  const auto first = [&](int p) { return p == 2 ? BM : p == 1 ? BM / 2 : 0; };
  const uint8_t *cb[3] = {a.wc[0] + (int64_t)row0 * kb * 128, GATED ? a.wc[1] + (int64_t)row0 * kb * 128 : nullptr,
                          a.xc + (int64_t)tok0 * kb * 128};
  const uint8_t *sb[3] = {a.ws[0] + (int64_t)row0 * kb * 8, GATED ? a.ws[1] + (int64_t)row0 * kb * 8 : nullptr,
                          a.xs + (int64_t)tok0 * kb * 8};
  const int cnt[3] = {rows, rows, toks};

  uint4 pc[PC];
  uint2 ps[PS];
  const auto load_codes = [&](int c) {
#pragma unroll
    for (int s = 0; s < PC; ++s) {
      const int q = tid + s * NTHR, r = q >> 3;
      const int p = part(__builtin_amdgcn_readfirstlane(r));
      const __amdgpu_buffer_rsrc_t rs = make_rsrc(cb[p] + c * 128, (uint32_t)((cnt[p] * kb - c) * 128));
      pc[s] = buf_load16(rs, (uint32_t)((r - first(p)) * kb) * 128u + (uint32_t)(q & 7) * 16u, 0, 0);
    }
  };
  const auto store_codes = [&](int b) {
#pragma unroll
    for (int s = 0; s < PC; ++s) {
      const int q = tid + s * NTHR, r = q >> 3;
      *reinterpret_cast<uint4*>(&sc[b][r * 128 + (((q & 7) ^ (r & 7)) << 4)]) = pc[s];
    }
  };
  const auto load_scales = [&](int grp) {
#pragma unroll
    for (int s = 0; s < PS; ++s) {
      const int q = tid + s * NTHR, r = q >> 2;
      const int p = part(__builtin_amdgcn_readfirstlane(r));
      const __amdgpu_buffer_rsrc_t rs = make_rsrc(sb[p] + grp * 32, (uint32_t)(cnt[p] * kb * 8 - grp * 32));
      const auto v = __builtin_amdgcn_raw_buffer_load_b64(rs, (uint32_t)((r - first(p)) * kb) * 8u + (uint32_t)(q & 3) * 8u, 0, 0);
      ps[s] = make_uint2(v[0], v[1]);
    }
  };
  const auto store_scales = [&](int b) {
#pragma unroll
    for (int s = 0; s < PS; ++s) *reinterpret_cast<uint2*>(&ss[b][(tid + s * NTHR) * 8]) = ps[s];
  };

  f32x16 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.0f;

  // this lane's row of each of the wave's tiles (GATED: the first half of its tiles gate, the others up)
  int ar[MT], br[NT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    constexpr int H = MT / 2;
    ar[m] = GATED ? (m / H) * (BM / 2) + wm * (H * 32) + (m % H) * 32 + l32 : wm * (MT * 32) + m * 32 + l32;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) br[n] = BM + wn * (NT * 32) + n * 32 + l32;

  load_codes(0);
  load_scales(0);
  store_codes(0);
  store_scales(0);
  __syncthreads();
  for (int c = 0; c < kb; ++c) {
    const int b = c & 1, sbuf = (c >> 2) & 1;
    const bool more = c + 1 < kb, scales_too = more && (c & 3) == 3;
    if (more) load_codes(c + 1);
    if (scales_too) load_scales((c >> 2) + 1);
    int sa[MT], sx[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m) sa[m] = *reinterpret_cast<const int*>(&ss[sbuf][ar[m] * 32 + (c & 3) * 8 + half * 4]);
#pragma unroll
    for (int n = 0; n < NT; ++n) sx[n] = *reinterpret_cast<const int*>(&ss[sbuf][br[n] * 32 + (c & 3) * 8 + half * 4]);
    const auto step = [&](auto jc) {
      constexpr int J = decltype(jc)::value;
      uint4 w[MT], x[NT];
#pragma unroll
      for (int m = 0; m < MT; ++m) w[m] = *reinterpret_cast<const uint4*>(&sc[b][ar[m] * 128 + (((4 * half + J) ^ (ar[m] & 7)) << 4)]);
#pragma unroll
      for (int n = 0; n < NT; ++n) x[n] = *reinterpret_cast<const uint4*>(&sc[b][br[n] * 128 + (((4 * half + J) ^ (br[n] & 7)) << 4)]);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = mfma_fp4_32<J>(w[m], x[n], acc[m][n], sa[m], sx[n]);
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
    if (more) store_codes(b ^ 1);
    if (scales_too) store_scales(sbuf ^ 1);
    __syncthreads();
  }

#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int tok = tok0 + br[n] - BM;
    if (tok >= a.t) continue;
#pragma unroll
    for (int m = 0; m < (GATED ? MT / 2 : MT); ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int r = row0 + ar[m] - l32 + 8 * q + 4 * half;
        float v[4], w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[j] = acc[m][n][4 * q + j];
          w[j] = GATED ? acc[(GATED ? MT / 2 : 0) + m][n][4 * q + j] : 0.0f;
        }
        mx_finish<GATED>(a, tok, r, v, w);
      }
  }
}

template <bool GATED>
static void launch_mx(const MxArgs& a, hipStream_t st) {
  const auto up = [](int64_t x, int64_t y) { return (unsigned)((x + y - 1) / y); };
  if (a.t <= 64) {
    const auto few = [&](auto nt) {
      constexpr int NT = decltype(nt)::value, MT = GATED ? 2 : 1;
      hipLaunchKernelGGL((k_mx_few<MT, NT, 8, GATED>), dim3(up(a.n, 16), up(a.t, NT * 16)), dim3(512), 0, st, a);
    };
    if (a.t <= 16) few(std::integral_constant<int, 1>{});
    else if (a.t <= 32) few(std::integral_constant<int, 2>{});
    else few(std::integral_constant<int, 4>{});
    return;
  }
  constexpr int BM = 128, BN = 128, OUTS = GATED ? BM / 2 : BM;
  hipLaunchKernelGGL((k_mx_tile<BM, BN, 2, 2, GATED>), dim3(up(a.n, OUTS), up(a.t, BN)), dim3(256), 0, st, a);
}

// Bytes of a matrix's codes and scales.
static size_t codes_bytes(const tq_mat_mx* m) { return (size_t)m->n * m->k / 2; }
static size_t mx_scales_bytes(const tq_mat_mx* m) { return (size_t)m->n * m->k / 32; }

// An output lies on none of a matrix's planes.
static bool on_matrix(const void* p, size_t n, const tq_mat_mx* m) {
  return overlap(p, n, m->codes, codes_bytes(m)) || overlap(p, n, m->scales, mx_scales_bytes(m));
}

}  // namespace tq

extern "C" tq_status tq_gemm_mx(const tq_mat_mx* w, const tq_mat_mx* x, int32_t type, void* y, void* stream) {
  using namespace tq;
  clear_error();
  if (tq_status st = check_mx_weights("tq_gemm_mx", "w", w)) return st;
  if (tq_status st = check_mx_rows("tq_gemm_mx", x, w->k)) return st;
  if (!known_type(type)) return fail(TQ_ERR_INVALID, "tq_gemm_mx: unknown type %d", type);
  if (x->n == 0) return TQ_OK;
  if (!y) return fail(TQ_ERR_INVALID, "tq_gemm_mx: null pointer");
  if (!aligned(y, type_bytes(type))) return fail(TQ_ERR_ALIGN, "tq_gemm_mx: y must be aligned to its type");
  const size_t ny = (size_t)x->n * w->n * type_bytes(type);
  if (on_matrix(y, ny, w) || on_matrix(y, ny, x)) return fail(TQ_ERR_INVALID, "tq_gemm_mx: y lies on an input");
  MxArgs a{{w->codes, nullptr}, {w->scales, nullptr}, x->codes, x->scales, w->n, x->n, w->k / 256, {y, nullptr, nullptr, nullptr, nullptr, type, 0}};
  (void)hipGetLastError();
  launch_mx<false>(a, (hipStream_t)stream);
  return check_launch("tq_gemm_mx");
}

extern "C" tq_status tq_gated_mx(const tq_mat_mx* gate, const tq_mat_mx* up, const tq_mat_mx* x, int32_t act, const float* g_add,
                                 const float* u_add, int32_t type, void* h, void* g, void* u, void* stream) {
  using namespace tq;
  clear_error();
  if (tq_status st = check_mx_weights("tq_gated_mx", "gate", gate)) return st;
  if (tq_status st = check_mx_weights("tq_gated_mx", "up", up)) return st;
  if (gate->n != up->n || gate->k != up->k)
    return fail(TQ_ERR_INVALID, "tq_gated_mx: gate is %d x %d, up %d x %d", gate->n, gate->k, up->n, up->k);
  if (tq_status st = check_mx_rows("tq_gated_mx", x, gate->k)) return st;
  if (act != TQ_ACT_SILU && act != TQ_ACT_GELU) return fail(TQ_ERR_INVALID, "tq_gated_mx: unknown activation %d", act);
  if (!known_type(type)) return fail(TQ_ERR_INVALID, "tq_gated_mx: unknown type %d", type);
  if (x->n == 0) return TQ_OK;
  if (!h || (!g != !u)) return fail(TQ_ERR_INVALID, "tq_gated_mx: null pointer");
  const size_t b = type_bytes(type);
  if (!aligned(h, b) || !aligned(g, b) || !aligned(u, b) || !aligned(g_add, 4) || !aligned(u_add, 4))
    return fail(TQ_ERR_ALIGN, "tq_gated_mx: tensors must be aligned to their types");
  const size_t ne = (size_t)x->n * gate->n, no = ne * b;
  const void* outs[3] = {h, g, u};
  for (int i = 0; i < 3; ++i) {
    const void* o = outs[i];
    if (on_matrix(o, no, gate) || on_matrix(o, no, up) || on_matrix(o, no, x) || overlap(o, no, g_add, ne * 4) ||
        overlap(o, no, u_add, ne * 4) || overlap(o, no, outs[(i + 1) % 3], no))
      return fail(TQ_ERR_INVALID, "tq_gated_mx: an output lies on an input or another output");
  }
  MxArgs a{{gate->codes, up->codes}, {gate->scales, up->scales}, x->codes, x->scales, gate->n, x->n, gate->k / 256,
           {h, g, u, g_add, u_add, type, act}};
  (void)hipGetLastError();
  launch_mx<true>(a, (hipStream_t)stream);
  return check_launch("tq_gated_mx");
}
