// Gradients through MXFP4 weights: dx = dy W^, and the gated block's dg, du and dx = dg Wg^ + du Wu^.
//
// The weights' scales run along k, the outputs here, so a sum over n meets another scale at every term and the fp4
// matrix instruction cannot take it. The weights are turned into bfloat16 (exact: e2m1 has 2 significant bits) on the
// way into LDS, by the scaled conversion, and read back transposed; products run on the bfloat16 matrix instruction.
// An fp32 (fp16) gradient is the exact sum of three (two) bfloat16 parts, each a pass of its own over the weights.
#include <algorithm>

#include "tq_mx.hpp"

namespace tq {

constexpr int kStep = 64;  // rows of the weights a step

// One pass: a [t][lda] bfloat16 (columns n .. lda hold zeros or are not there) against one weight matrix.
struct MxSeg {
  const bf16_t* a;
  const uint8_t *codes, *scales;
  int64_t lda;
};
struct MxBwdArgs {
  MxSeg seg[6];
  int nseg, n, t, kb, type, splits;
  void* out;   // dx, or with splits > 1 the partial sums [splits][t][k] fp32
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

// Four rows' elements of this lane's column: lane i of 16 passes the address of row i / 4, columns 4 (i % 4) ...
__device__ __forceinline__ s16x4 read_columns(const void* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(const_cast<void*>(p)));
}

// Tiles of BC columns of k by BN tokens, kStep rows of the weights a step through two LDS stages.
//   a stage's tokens: 128 bytes a row, 16-byte pieces exchanged by the row's low bits;
//   its weights: BC bfloat16 a row, 32-byte units exchanged likewise.
template <int BC, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64) void k_mx_bwd(const MxBwdArgs a) {
  constexpr int NTHR = WM * WN * 64, MT = BC / WM / 32, NT = BN / WN / 32;
  constexpr int WP = BC / 32;                      // pieces (blocks of 32) of a weight row
  constexpr int PW = kStep * WP / NTHR, PA = BN * 8 / NTHR;
  static_assert(PW >= 1 && kStep * WP % NTHR == 0 && PA >= 1 && BN * 8 % NTHR == 0, "tile");
  __shared__ __attribute__((aligned(16))) uint8_t sa[2][BN * 128];
  __shared__ __attribute__((aligned(16))) uint8_t sw[2][kStep * BC * 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN, l32 = lane & 31, half = lane >> 5;
  const int kb = a.kb, col0 = blockIdx.x * BC, tok0 = blockIdx.y * BN, toks = min(BN, a.t - tok0);
  const int per = (a.n + kStep - 1) / kStep, all = per * a.nseg;
  const int s0 = (int)((int64_t)all * blockIdx.z / a.splits), s1 = (int)((int64_t)all * (blockIdx.z + 1) / a.splits);

  uint4 pw[PW], pa[PA];
  uint32_t pe[PW];
  const auto load = [&](int s) {
    const int g = s / per, n0 = (s - g * per) * kStep;
    const MxSeg& sg = a.seg[g];
    const int rows = min(kStep, a.n - n0);
    const __amdgpu_buffer_rsrc_t rc = make_rsrc(sg.codes + (int64_t)n0 * kb * 128 + col0 / 2, (uint32_t)(rows * kb * 128 - col0 / 2));
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(sg.scales + (int64_t)n0 * kb * 8 + col0 / 32, (uint32_t)(rows * kb * 8 - col0 / 32));
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(sg.a + (int64_t)tok0 * sg.lda + n0, (uint32_t)((toks * sg.lda - n0) * 2));
    const uint32_t cols = (uint32_t)(sg.lda - n0);
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      const int q = tid + i * NTHR, r = q % kStep, p = q / kStep;
      pw[i] = buf_load16(rc, (uint32_t)(r * kb) * 128u + (uint32_t)p * 16u, 0, 0);
      pe[i] = __builtin_amdgcn_raw_buffer_load_b8(rs, (uint32_t)(r * kb) * 8u + (uint32_t)p, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < PA; ++i) {
      const int q = tid + i * NTHR, r = q >> 3, p = q & 7;
      // (past the row's end lies the next token's row, whose infinities must not meet the weights' zeros)
      const uint32_t at = (uint32_t)p * 8u < cols ? (uint32_t)r * (uint32_t)sg.lda * 2u + (uint32_t)p * 16u : 0xfffffff0u;
      pa[i] = buf_load16(ra, r < toks ? at : 0xfffffff0u, 0, 0);
    }
  };
  const auto store = [&](int b) {
#pragma unroll
    for (int i = 0; i < PA; ++i) {
      const int q = tid + i * NTHR, r = q >> 3, p = q & 7;
      *reinterpret_cast<uint4*>(&sa[b][r * 128 + ((p ^ (r & 7)) << 4)]) = pa[i];
    }
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      const int q = tid + i * NTHR, r = q % kStep, p = q / kStep;
      const float s = e8m0_f32(pe[i] & 255u);
      const uint32_t w[4] = {pw[i].x, pw[i].y, pw[i].z, pw[i].w};
      uint32_t lo[8], hi[8];  // elements 0..15 and 16..31 of the block, two a dword
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const uint32_t c0 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], s, 0));
        const uint32_t c1 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], s, 1));
        const uint32_t c2 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], s, 2));
        const uint32_t c3 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], s, 3));
        lo[2 * d] = __builtin_amdgcn_perm(c1, c0, 0x05040100u);
        lo[2 * d + 1] = __builtin_amdgcn_perm(c3, c2, 0x05040100u);
        hi[2 * d] = __builtin_amdgcn_perm(c1, c0, 0x07060302u);
        hi[2 * d + 1] = __builtin_amdgcn_perm(c3, c2, 0x07060302u);
      }
      uint8_t* row = &sw[b][r * BC * 2];
      uint4* u0 = reinterpret_cast<uint4*>(row + (((2 * p) ^ (r & 7)) << 5));
      uint4* u1 = reinterpret_cast<uint4*>(row + (((2 * p + 1) ^ (r & 7)) << 5));
      u0[0] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      u0[1] = make_uint4(lo[4], lo[5], lo[6], lo[7]);
      u1[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      u1[1] = make_uint4(hi[4], hi[5], hi[6], hi[7]);
    }
  };

  f32x16 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.0f;

  const int i16 = lane & 15, g16 = lane >> 4;
  if (s0 < s1) {
    load(s0);
    store(0);
  }
  __syncthreads();
  for (int s = s0; s < s1; ++s) {
    const int b = (s - s0) & 1;
    const bool more = s + 1 < s1;
    if (more) load(s + 1);
#pragma unroll
    for (int k = 0; k < kStep / 16; ++k) {
      bf16x8 w[MT], x[NT];
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int unit = (wm * MT + m) * 2 + (g16 & 1);
        const int r0 = 16 * k + 8 * (g16 >> 1) + i16 / 4, r1 = r0 + 4;
        const s16x4 v0 = read_columns(&sw[b][r0 * BC * 2 + ((unit ^ (r0 & 7)) << 5) + 8 * (i16 & 3)]);
        const s16x4 v1 = read_columns(&sw[b][r1 * BC * 2 + ((unit ^ (r1 & 7)) << 5) + 8 * (i16 & 3)]);
        w[m] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int r = (wn * NT + n) * 32 + l32;
        x[n] = *reinterpret_cast<const bf16x8*>(&sa[b][r * 128 + (((2 * k + half) ^ (r & 7)) << 4)]);
      }
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[m], x[n], acc[m][n], 0, 0, 0);
    }
    if (more) store(b ^ 1);
    __syncthreads();
  }

  const int64_t k = (int64_t)kb * 256;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int tok = tok0 + (wn * NT + n) * 32 + l32;
    if (tok >= a.t) continue;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = col0 + (wm * MT + m) * 32 + 8 * q + 4 * half;
        const float v[4] = {acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
        if (a.splits > 1) store4(TQ_F32, a.out, ((int64_t)blockIdx.z * a.t + tok) * k + c, v, 4);
        else store4(a.type, a.out, tok * k + c, v, 4);
      }
  }
}

// The partial sums of `splits` parts, in order; four elements a thread.
__global__ __launch_bounds__(256) void k_mx_bwd_join(const float* __restrict__ part, int splits, int64_t quads, int type, void* out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= quads) return;
  f32x4 s = *reinterpret_cast<const f32x4*>(part + 4 * i);
  for (int p = 1; p < splits; ++p) s += *reinterpret_cast<const f32x4*>(part + 4 * (p * quads + i));
  const float v[4] = {s[0], s[1], s[2], s[3]};
  store4(type, out, 4 * i, v, 4);
}

// The exact bfloat16 parts of a value: its leading 8 bits, the next 8, the rest.
__device__ __forceinline__ void bf16_parts(float x, bf16_t (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const float h = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    p[i] = __builtin_bit_cast(bf16_t, (uint16_t)(__float_as_uint(x) >> 16));
    x -= h;
  }
}

// Rows of n values to NP planes [t][pad] of bfloat16 parts, the last ones first (pad - n zeros a row).
template <typename T, int NP>
__device__ __forceinline__ void put_parts(float x, bf16_t* planes, int64_t plane, int64_t at) {
  bf16_t p[3];
  bf16_parts(x, p);
#pragma unroll
  for (int i = 0; i < NP; ++i) planes[(NP - 1 - i) * plane + at] = p[i];
}

template <typename T, int NP>
__global__ __launch_bounds__(256) void k_mx_parts(const T* __restrict__ x, int64_t t, int n, int pad, bf16_t* __restrict__ planes) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < t * pad; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / pad;
    const int c = (int)(i - r * pad);
    put_parts<T, NP>(c < n ? (float)x[r * n + c] : 0.0f, planes, t * pad, i);
  }
}

// dg = dh u act'(g), du = dh act(g), and where `planes` is given their parts ([2][NP][t][pad]).
template <typename T, int NP>
__global__ __launch_bounds__(256) void k_gated_bwd(const T* g, const T* u, const T* dh, int act, int64_t t, int n, int pad, T* dg, T* du,
                                                   bf16_t* __restrict__ planes) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < t * pad; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / pad;
    const int c = (int)(i - r * pad);
    float vg = 0.0f, vu = 0.0f;
    if (c < n) {
      const int64_t j = r * n + c;
      const float d = (float)dh[j], uu = (float)u[j];
      float a, da;
      act_both(act, (float)g[j], a, da);
      const T tg = (T)(d * uu * da), tu = (T)(d * a);
      dg[j] = tg;
      du[j] = tu;
      vg = (float)tg;
      vu = (float)tu;
    }
    if (planes) {
      put_parts<T, NP>(vg, planes, t * pad, i);
      put_parts<T, NP>(vu, planes + NP * t * pad, t * pad, i);
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------

static int parts_of(int32_t type) { return type == TQ_F32 ? 3 : type == TQ_F16 ? 2 : 1; }
static int64_t pad_of(int n) { return ((int64_t)n + 63) / 64 * 64; }
static int tokens_a_tile(int64_t t) { return t <= 32 ? 32 : t <= 64 ? 64 : 128; }
constexpr int64_t kTargetWgs = 512;

// Parts the sum over the rows of the weights is split into where there are few tiles.
static int splits_of(int64_t t, int kb, int steps) {
  const int bn = tokens_a_tile(t);
  const int64_t tiles = (t + bn - 1) / bn * kb * (bn == 128 ? 2 : 1);
  return (int)std::max<int64_t>(1, std::min<int64_t>(kTargetWgs / tiles, steps / 2));
}

static size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Room for the parts of `mats` gradients, then for the partial sums: at most kTargetWgs tiles of 256 columns, their tokens.
static size_t bwd_bytes(int n, int32_t type, int64_t t, int mats) {
  const size_t planes = (size_t)mats * parts_of(type) * t * pad_of(n) * 2;
  return up256(planes) + (size_t)kTargetWgs * 256 * 4 * std::min<int64_t>(t, tokens_a_tile(t)) + 256;
}

// Workgroups of 256 for `n` elements, whose threads go on to further ones.
static unsigned blocks_for(int64_t n) { return (unsigned)std::min<int64_t>((n + 255) / 256, 1 << 18); }

template <typename F>
static void with_parts(int32_t type, F f) {
  if (type == TQ_F32) f(float{}, std::integral_constant<int, 3>{});
  else if (type == TQ_BF16) f(bf16_t{}, std::integral_constant<int, 1>{});
  else f(f16_t{}, std::integral_constant<int, 2>{});
}

static void launch_bwd(MxBwdArgs a, void* dx, int32_t type, float* part, hipStream_t st) {
  const int steps = (a.n + kStep - 1) / kStep * a.nseg, bn = tokens_a_tile(a.t);
  a.splits = splits_of(a.t, a.kb, steps);
  a.type = type;
  a.out = a.splits > 1 ? part : dx;
  const unsigned ty = (unsigned)((a.t + bn - 1) / bn), kb = (unsigned)a.kb, z = (unsigned)a.splits;
  if (bn == 32) hipLaunchKernelGGL((k_mx_bwd<256, 32, 4, 1>), dim3(kb, ty, z), dim3(256), 0, st, a);
  else if (bn == 64) hipLaunchKernelGGL((k_mx_bwd<256, 64, 4, 1>), dim3(kb, ty, z), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_mx_bwd<128, 128, 2, 2>), dim3(kb * 2, ty, z), dim3(256), 0, st, a);
  if (a.splits > 1) {
    const int64_t quads = (int64_t)a.t * a.kb * 64;
    hipLaunchKernelGGL(k_mx_bwd_join, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, part, a.splits, quads, type, dx);
  }
}

static bool rows_in_range(int64_t t) { return t >= 0 && t <= kMxMaxRows; }

static bool weights_in_range(const tq_mat_mx* w) {
  return w && w->n >= 1 && w->n <= kMxMaxRows && w->k > 0 && w->k % 256 == 0 && w->k <= kMaxK;
}

static bool on_matrix(const void* p, size_t n, const tq_mat_mx* m) {
  return overlap(p, n, m->codes, (size_t)m->n * m->k / 2) || overlap(p, n, m->scales, (size_t)m->n * m->k / 32);
}

}  // namespace tq

extern "C" size_t tq_gemm_mx_bwd_workspace_bytes(const tq_mat_mx* w, int32_t type, int64_t t) {
  using namespace tq;
  return weights_in_range(w) && known_type(type) && rows_in_range(t) ? bwd_bytes(w->n, type, t, 1) : 0;
}

extern "C" tq_status tq_gemm_mx_bwd(const tq_mat_mx* w, const void* dy, int32_t type, int64_t t, void* dx, void* ws, size_t ws_bytes,
                                    void* stream) {
  using namespace tq;
  clear_error();
  if (tq_status st = check_mx_weights("tq_gemm_mx_bwd", "w", w)) return st;
  if (!known_type(type)) return fail(TQ_ERR_INVALID, "tq_gemm_mx_bwd: unknown type %d", type);
  if (!rows_in_range(t)) return fail(TQ_ERR_INVALID, "tq_gemm_mx_bwd: t = %lld out of range", (long long)t);
  if (t == 0) return TQ_OK;
  if (!dy || !dx || !ws) return fail(TQ_ERR_INVALID, "tq_gemm_mx_bwd: null pointer");
  const size_t b = type_bytes(type);
  if (!aligned(dy, b) || !aligned(dx, b) || !aligned(ws, 256))
    return fail(TQ_ERR_ALIGN, "tq_gemm_mx_bwd: ws must be 256-byte aligned, tensors to their types");
  const size_t need = bwd_bytes(w->n, type, t, 1), ny = (size_t)t * w->n * b, nx = (size_t)t * w->k * b;
  if (ws_bytes < need) return fail(TQ_ERR_WORKSPACE, "tq_gemm_mx_bwd: workspace of %zu bytes, %zu needed", ws_bytes, need);
  if (overlap(dx, nx, dy, ny) || on_matrix(dx, nx, w) || overlap(ws, ws_bytes, dx, nx) || overlap(ws, ws_bytes, dy, ny) ||
      on_matrix(ws, ws_bytes, w))
    return fail(TQ_ERR_INVALID, "tq_gemm_mx_bwd: overlapping tensors");
  (void)hipGetLastError();
  const int np = parts_of(type);
  const int64_t pad = pad_of(w->n);
  MxBwdArgs a{};
  a.nseg = np;
  a.n = w->n;
  a.t = (int)t;
  a.kb = w->k / 256;
  bf16_t* planes = (bf16_t*)ws;
  // (bfloat16 rows whose 16-byte pieces are whole are read where they are)
  const bool direct = type == TQ_BF16 && w->n % 8 == 0 && aligned(dy, 16);
  for (int i = 0; i < np; ++i)
    a.seg[i] = direct ? MxSeg{(const bf16_t*)dy, w->codes, w->scales, w->n} : MxSeg{planes + i * t * pad, w->codes, w->scales, pad};
  if (!direct)
    with_parts(type, [&](auto z, auto npc) {
      using T = decltype(z);
      hipLaunchKernelGGL((k_mx_parts<T, decltype(npc)::value>), dim3(blocks_for(t * pad)), dim3(256), 0, (hipStream_t)stream,
                         (const T*)dy, t, w->n, (int)pad, planes);
    });
  launch_bwd(a, dx, type, (float*)((uint8_t*)ws + up256((size_t)np * t * pad * 2)), (hipStream_t)stream);
  return check_launch("tq_gemm_mx_bwd");
}

extern "C" size_t tq_gated_mx_bwd_workspace_bytes(const tq_mat_mx* gate, const tq_mat_mx* up, int32_t type, int64_t t) {
  using namespace tq;
  return weights_in_range(gate) && weights_in_range(up) && gate->n == up->n && gate->k == up->k && known_type(type) && rows_in_range(t)
             ? bwd_bytes(gate->n, type, t, 2) : 0;
}

extern "C" tq_status tq_gated_mx_bwd(const tq_mat_mx* gate, const tq_mat_mx* up, int32_t act, int32_t type, int64_t t, const void* g,
                                     const void* u, const void* dh, void* dg, void* du, void* dx, void* ws, size_t ws_bytes,
                                     void* stream) {
  using namespace tq;
  clear_error();
  if (tq_status st = check_mx_weights("tq_gated_mx_bwd", "gate", gate)) return st;
  if (tq_status st = check_mx_weights("tq_gated_mx_bwd", "up", up)) return st;
  if (gate->n != up->n || gate->k != up->k)
    return fail(TQ_ERR_INVALID, "tq_gated_mx_bwd: gate is %d x %d, up %d x %d", gate->n, gate->k, up->n, up->k);
  if (act != TQ_ACT_SILU && act != TQ_ACT_GELU) return fail(TQ_ERR_INVALID, "tq_gated_mx_bwd: unknown activation %d", act);
  if (!known_type(type)) return fail(TQ_ERR_INVALID, "tq_gated_mx_bwd: unknown type %d", type);
  if (!rows_in_range(t)) return fail(TQ_ERR_INVALID, "tq_gated_mx_bwd: t = %lld out of range", (long long)t);
  if (t == 0) return TQ_OK;
  if (!g || !u || !dh || !dg || !du || (dx && !ws)) return fail(TQ_ERR_INVALID, "tq_gated_mx_bwd: null pointer");
  const size_t b = type_bytes(type);
  if (!aligned(g, b) || !aligned(u, b) || !aligned(dh, b) || !aligned(dg, b) || !aligned(du, b) || !aligned(dx, b) || !aligned(ws, 256))
    return fail(TQ_ERR_ALIGN, "tq_gated_mx_bwd: ws must be 256-byte aligned, tensors to their types");
  const int n = gate->n, np = parts_of(type);
  const size_t need = bwd_bytes(n, type, t, 2), nh = (size_t)t * n * b, nx = (size_t)t * gate->k * b;
  if (dx && ws_bytes < need) return fail(TQ_ERR_WORKSPACE, "tq_gated_mx_bwd: workspace of %zu bytes, %zu needed", ws_bytes, need);
  const void* in[3] = {g, u, dh};
  bool bad = overlap(dg, nh, du, nh) || overlap(dx, nx, dg, nh) || overlap(dx, nx, du, nh);
  for (const void* p : in)
    bad = bad || (dg != p && overlap(dg, nh, p, nh)) || (du != p && overlap(du, nh, p, nh)) || overlap(dx, nx, p, nh) ||
          (dx && overlap(ws, ws_bytes, p, nh));
  for (const tq_mat_mx* m : {gate, up})
    bad = bad || on_matrix(dg, nh, m) || on_matrix(du, nh, m) || on_matrix(dx, nx, m) || (dx && on_matrix(ws, ws_bytes, m));
  bad = bad || (dx && (overlap(ws, ws_bytes, dg, nh) || overlap(ws, ws_bytes, du, nh) || overlap(ws, ws_bytes, dx, nx)));
  if (bad) return fail(TQ_ERR_INVALID, "tq_gated_mx_bwd: overlapping tensors");
  (void)hipGetLastError();
  const int64_t pad = pad_of(n);
  const bool direct = type == TQ_BF16 && n % 8 == 0 && aligned(dg, 16) && aligned(du, 16);
  bf16_t* planes = dx && !direct ? (bf16_t*)ws : nullptr;
  const int64_t width = planes ? pad : n;
  with_parts(type, [&](auto z, auto npc) {
    using T = decltype(z);
    hipLaunchKernelGGL((k_gated_bwd<T, decltype(npc)::value>), dim3(blocks_for(t * width)), dim3(256), 0, (hipStream_t)stream,
                       (const T*)g, (const T*)u, (const T*)dh, act, t, n, (int)width, (T*)dg, (T*)du, planes);
  });
  if (dx) {
    MxBwdArgs a{};
    a.nseg = 2 * np;
    a.n = n;
    a.t = (int)t;
    a.kb = gate->k / 256;
    for (int m = 0; m < 2; ++m)
      for (int i = 0; i < np; ++i) {
        const tq_mat_mx* w = m ? up : gate;
        a.seg[m * np + i] = direct ? MxSeg{(const bf16_t*)(m ? du : dg), w->codes, w->scales, n}
                                   : MxSeg{planes + (m * np + i) * t * pad, w->codes, w->scales, pad};
      }
    launch_bwd(a, dx, type, (float*)((uint8_t*)ws + up256((size_t)2 * np * t * pad * 2)), (hipStream_t)stream);
  }
  return check_launch("tq_gated_mx_bwd");
}
