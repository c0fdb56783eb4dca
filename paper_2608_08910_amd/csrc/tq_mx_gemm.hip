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

// The first m of 8 consecutive elements from i of a [type] tensor.
__device__ __forceinline__ void store8(int type, void* p, int64_t i, const float (&v)[8], int m) {
  if (m >= 8 && type != TQ_F32) {
    if (type == TQ_BF16) store_n<8>((bf16_t*)p + i, v);
    else store_n<8>((f16_t*)p + i, v);
    return;
  }
  const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
  store4(type, p, i, a, m);
  store4(type, p, i + 4, b, m - 4);
}

// v += the first m of N elements.
template <int N>
__device__ __forceinline__ void add_n(const float* p, float (&v)[N], int m) {
  if (m >= N) {
    float a[N];
    load_n<N>(p, a);
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] += a[j];
  } else {
#pragma unroll
    for (int j = 0; j < N - 1; ++j)
      if (j < m) v[j] += p[j];
  }
}

template <int N>
__device__ __forceinline__ void put(int type, void* p, int64_t i, const float (&v)[N], int m) {
  if constexpr (N == 4) store4(type, p, i, v, m);
  else store8(type, p, i, v, m);
}

// N consecutive outputs r .. of token `tok` (those below n), from the sums of the weights' (gate's) and, GATED, up's rows.
template <bool GATED, int N>
__device__ __forceinline__ void mx_finish(const MxArgs& a, int64_t tok, int r, float (&g)[N], float (&u)[N]) {
  const int m = a.n - r;
  if (m <= 0) return;
  const int64_t i = tok * a.n + r;
  if constexpr (!GATED) {
    put<N>(a.out.type, a.out.y, i, g, m);
  } else {
    if (a.out.g_add) add_n<N>(a.out.g_add + i, g, m);
    if (a.out.u_add) add_n<N>(a.out.u_add + i, u, m);
    float h[N];
#pragma unroll
    for (int j = 0; j < N; ++j) h[j] = act_fwd(a.out.act, g[j]) * u[j];
    put<N>(a.out.type, a.out.y, i, h, m);
    if (a.out.g) {
      put<N>(a.out.type, a.out.g, i, g, m);
      put<N>(a.out.type, a.out.u, i, u, m);
    }
  }
}

// ---- few tokens: bound by the weights' bytes, or by the time to the first of them. A workgroup takes MT tiles of 16 rows
// (GATED: the first half of its rows gate, the others up of the same outputs) and NT * 16 tokens; its waves share k, 256
// elements at a time, and join through LDS, in order. Operands come straight from memory: lanes l, l + 16, l + 32, l + 48
// take four consecutive blocks of a row, 64 bytes of it (with two blocks each, 32 bytes apart: 4096 x 2048 one token 3.7 us, 3.0 so). GATED with
// one tile issues each load of weights for gate and for up, half of the lanes past the buffer (2 x (2048 x 7168) one token 6.1 us a call, its bytes 3.1).
template <int MT, int NT, int NW, bool GATED>
__global__ __launch_bounds__(NW * 64) void k_mx_few(const MxArgs a) {
  __shared__ f32x4 red[NW][MT * NT][64];
  constexpr int OUTS = GATED ? 8 * MT : 16 * MT;  // outputs of a workgroup
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int row0 = blockIdx.x * OUTS, tok0 = blockIdx.y * (NT * 16), kb = a.kb;
  const int rows = min(OUTS, a.n - row0), toks = min(NT * 16, a.t - tok0);
  // Rows past the last read as zeros. MT = 1 and GATED: lanes 8 .. 15 of each 16 read up's rows, the others gate's.
  const auto rsrc = [&](const uint8_t* p, int first, int count, int bytes) {
    return make_rsrc(p + (int64_t)first * kb * bytes, (uint32_t)(count * kb * bytes));
  };
  const __amdgpu_buffer_rsrc_t wc0 = rsrc(a.wc[0], row0, rows, 128), ws0 = rsrc(a.ws[0], row0, rows, 8);
  const __amdgpu_buffer_rsrc_t wc1 = rsrc(a.wc[GATED], row0, rows, 128), ws1 = rsrc(a.ws[GATED], row0, rows, 8);
  const __amdgpu_buffer_rsrc_t xc = rsrc(a.xc, tok0, toks, 128), xs = rsrc(a.xs, tok0, toks, 8);

  f32x4 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  constexpr uint32_t kNone = 0xf0000000u;  // past every buffer
  const auto load2 = [&](__amdgpu_buffer_rsrc_t rs, uint32_t at) {
    const auto v = __builtin_amdgcn_raw_buffer_load_b64(rs, at, 0, 0);
    return make_uint2(v[0], v[1]);
  };
  for (int c = wave; c < kb; c += NW) {
    uint4 w[MT][2], x[NT][2];
    uint2 sw[MT], sx[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      if constexpr (GATED && MT == 1) {
        const uint32_t r = (uint32_t)((l16 & 7) * kb + c), at = r * 128u + (uint32_t)g * 16u, no = kNone;
        const uint32_t a0 = l16 < 8 ? at : no, a1 = l16 < 8 ? no : at;
        const uint4 p0 = buf_load16(wc0, a0, 0), p1 = buf_load16(wc0, a0 + 64u, 0), q0 = buf_load16(wc1, a1, 0), q1 = buf_load16(wc1, a1 + 64u, 0);
        const uint2 e0 = load2(ws0, l16 < 8 ? r * 8u : no), e1 = load2(ws1, l16 < 8 ? no : r * 8u);
        w[m][0] = make_uint4(p0.x | q0.x, p0.y | q0.y, p0.z | q0.z, p0.w | q0.w);
        w[m][1] = make_uint4(p1.x | q1.x, p1.y | q1.y, p1.z | q1.z, p1.w | q1.w);
        sw[m] = make_uint2(e0.x | e1.x, e0.y | e1.y);
      } else {
        constexpr int H = GATED ? MT / 2 : MT;
        const uint32_t r = (uint32_t)((m % H * 16 + l16) * kb + c);
        w[m][0] = buf_load16(m < H ? wc0 : wc1, r * 128u + (uint32_t)g * 16u, 0);
        w[m][1] = buf_load16(m < H ? wc0 : wc1, r * 128u + (uint32_t)g * 16u + 64u, 0);
        sw[m] = load2(m < H ? ws0 : ws1, r * 8u);
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint32_t r = (uint32_t)((n * 16 + l16) * kb + c);
      x[n][0] = buf_load16(xc, r * 128u + (uint32_t)g * 16u, 0, 0);
      x[n][1] = buf_load16(xc, r * 128u + (uint32_t)g * 16u + 64u, 0, 0);
      sx[n] = load2(xs, r * 8u);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        acc[m][n] = mfma_fp4_16<0>(w[m][0], x[n][0], acc[m][n], (int)(sw[m].x >> (8 * g)), (int)(sx[n].x >> (8 * g)));
        acc[m][n] = mfma_fp4_16<0>(w[m][1], x[n][1], acc[m][n], (int)(sw[m].y >> (8 * g)), (int)(sx[n].y >> (8 * g)));
      }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) red[wave][m * NT + n][lane] = acc[m][n];
  __syncthreads();
  // Four outputs of a token a thread (4 g of 16 rows; GATED with one tile: of 8, g < 2, up's sums 32 lanes on).
  constexpr bool MIX = GATED && MT == 1;
  constexpr int OT = MIX ? NT : OUTS / 16 * NT;
  for (int o = wave; o < OT; o += NW) {
    const int n = o % NT, m = o / NT;
    f32x4 s = red[0][o][lane], u = {};
    if constexpr (GATED) u = MIX ? red[0][o][lane ^ 32] : red[0][OT + o][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      s += red[w][o][lane];
      if constexpr (GATED) u += MIX ? red[w][o][lane ^ 32] : red[w][OT + o][lane];
    }
    const int tok = tok0 + 16 * n + l16, r = row0 + 16 * m + 4 * g;
    if (tok < a.t && (!MIX || g < 2)) {
      float v[4] = {s[0], s[1], s[2], s[3]}, w[4] = {u[0], u[1], u[2], u[3]};
      mx_finish<GATED, 4>(a, tok, r, v, w);
    }
  }
}

// ---- many tokens: tiles of BM weight rows (GATED: BM / 2 gate rows, then the up rows of the same outputs) by BN tokens,
// 256 elements of k (whole 128-byte lines) at a time, through S LDS stages that the loads fill without passing through
// registers. In a stage a row's 16-byte pieces are exchanged by the row's number, so that the 16 rows whose pieces
// one LDS access takes lie in different banks; likewise the dwords of the scales, staged for four steps at once.
// The operands of one quarter of a step are read while the matrix unit works on the quarter before, across the barrier too.
// Results pass through LDS on their way out: stored from the lanes that hold them, 16 bytes of a row at a time, they cost
// as much as the products (16384 x 7168 gated, 4096 tokens, h alone: 775 us, 516 so when measured, 489 by now; with adapters' parts and g and u
// kept 655: little of the way out overlaps the products, a compute unit holding one tile). The products are bound by clocks, 54% of them the matrix
// unit's, and by power: 861 thousand clocks at 1.72 GHz on random codes, 882 at 2.37 on zeros.
// WK = 2: two groups of waves share the four quarters of a step (where tiles are few), and their sums join on the way out.
template <int BM, int BN, int WM, int WN, int WK, int S, bool GATED>
__global__ __launch_bounds__(WM * WN * WK * 64) void k_mx_tile(const MxArgs a) {
  constexpr int NW = WM * WN * WK, Q = 4 / WK, MT = BM / WM / 32, NT = BN / WN / 32, ROWS = BM + BN;
  constexpr int OUTS = GATED ? BM / 2 : BM;  // outputs of a tile
  constexpr int PL = ROWS / 8 / NW;          // load instructions of a wave, 8 rows each
  static_assert((S - 2) * PL < 64 && (WK == 1 || WK == 2), "stages");
  constexpr bool FIXED = OUTS % (8 * NW) == 0 && BN % (8 * NW) == 0;  // a load instruction's part does not depend on the wave
  static_assert(ROWS % (8 * NW) == 0 && (!GATED || MT % 2 == 0), "tile");
  __shared__ __attribute__((aligned(16))) uint8_t sc[S * ROWS * 128];
  __shared__ __attribute__((aligned(16))) uint8_t ss[2 * ROWS * 32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wk = wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN, l32 = lane & 31, half = lane >> 5, l8 = lane >> 3;
  const int kb = a.kb;
  // Consecutive workgroups go to the eight dies in turn: each die takes a run of tiles, four token tiles at a time, so that
  // its L2 serves them (16384 x 7168 gated, 4096 tokens: 815 us in plain order, 699 so, before the other steps).
  const int nx = gridDim.x, ny = gridDim.y, tile = die_order(blockIdx.y * nx + blockIdx.x, nx * ny);
  const int g0 = tile / (4 * nx) * 4, gs = min(4, ny - g0), in = tile - g0 * nx;
  const int row0 = in / gs * OUTS, tok0 = (g0 + in % gs) * BN;
  const int rows = min(OUTS, a.n - row0), toks = min(BN, a.t - tok0);

  // Rows of a stage: part 0 the weights (gate), 1 up, 2 the tokens; rows past the last read as zeros.
  const uint8_t *c0 = a.wc[0] + (int64_t)row0 * kb * 128, *c1 = GATED ? a.wc[1] + (int64_t)row0 * kb * 128 : nullptr,
                *c2 = a.xc + (int64_t)tok0 * kb * 128;
  const uint8_t *e0 = a.ws[0] + (int64_t)row0 * kb * 8, *e1 = GATED ? a.ws[1] + (int64_t)row0 * kb * 8 : nullptr,
                *e2 = a.xs + (int64_t)tok0 * kb * 8;
  const auto part = [](int r) { return r >= BM ? 2 : r >= OUTS ? 1 : 0; };
  const auto first = [](int p) { return p == 2 ? BM : p * OUTS; };
  // Step c (past the last one the next rows' codes, or zeros, that nothing uses).
  const auto load_codes = [&](int c) {
    const uint32_t dst = lds_address(sc) + (uint32_t)(c % S) * (ROWS * 128);
#pragma unroll
    for (int s = 0; s < PL; ++s) {
      const int r0 = (wave + s * NW) * 8, p = part(FIXED ? s * NW * 8 : r0);
      const int count = p == 2 ? toks : rows;
      const i32x4 rs = rsrc_words((p == 2 ? c2 : p == 1 ? c1 : c0) + c * 128, (uint32_t)max(0, (count * kb - c) * 128));
      const uint32_t at = (uint32_t)((r0 - first(p) + l8) * kb) * 128u + (uint32_t)(((lane & 7) ^ (((r0 + l8) >> 1) & 7)) * 16);
      load_lds<16>(rs, dst + r0 * 128, at);
    }
  };
  // Scales of steps 4 grp .. 4 grp + 3 (past a row's end the next row's, unused).
  const auto load_scales = [&](int grp) {
    const uint32_t dst = lds_address(ss) + (uint32_t)(grp & 1) * (ROWS * 32);
#pragma unroll
    for (int s = 0; s < PL; ++s) {
      const int r0 = (wave + s * NW) * 8, p = part(FIXED ? s * NW * 8 : r0);
      const int count = p == 2 ? toks : rows;
      const i32x4 rs = rsrc_words((p == 2 ? e2 : p == 1 ? e1 : e0) + grp * 32, (uint32_t)max(0, count * kb * 8 - grp * 32));
      const uint32_t at = (uint32_t)((r0 - first(p) + l8) * kb) * 8u + (uint32_t)((lane & 7) ^ ((r0 >> 3) & 3)) * 4u;
      load_lds<4>(rs, dst + r0 * 32, at);
    }
  };

  f32x16 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.0f;

  // This lane's rows: ra and rb, and a constant for each of the wave's tiles (GATED: the first half of them gate, the others up).
  constexpr int H = GATED ? MT / 2 : MT;
  const int ra = wm * (H * 32) + l32, rb = BM + wn * (NT * 32) + l32;
  const auto tile_row = [](int m) { return m / H * OUTS + m % H * 32; };
  int piece[Q];
#pragma unroll
  for (int j = 0; j < Q; ++j) piece[j] = ((4 * half + wk * Q + j) ^ ((l32 >> 1) & 7)) << 4;

  uint4 w0[MT], x0[NT], w1[MT], x1[NT];  // two quarters' operands
  int sa[MT], sx[NT], sp1[MT], sp2[NT];  // scales of the step, and of the one before for its last quarter
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    w1[m] = make_uint4(0, 0, 0, 0);
    sp1[m] = 0;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    x1[n] = make_uint4(0, 0, 0, 0);
    sp2[n] = 0;
  }
  const auto read = [&](const uint8_t* cur, int j, uint4 (&w)[MT], uint4 (&x)[NT]) {
#pragma unroll
    for (int n = 0; n < NT; ++n) x[n] = *reinterpret_cast<const uint4*>(cur + rb * 128 + piece[j] + n * 4096);
#pragma unroll
    for (int m = 0; m < MT; ++m) w[m] = *reinterpret_cast<const uint4*>(cur + ra * 128 + piece[j] + tile_row(m) * 128);
    __builtin_amdgcn_sched_barrier(0);
  };
  const auto multiply = [&](auto jc, const uint4 (&w)[MT], const uint4 (&x)[NT], const int (&p)[MT], const int (&q)[NT]) {
    constexpr int J = decltype(jc)::value;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[m][n] = mfma_fp4_32<J>(w[m], x[n], acc[m][n], p[m], q[n]);
    __builtin_amdgcn_sched_barrier(0);
  };
  const std::integral_constant<int, 0> q0;
  const std::integral_constant<int, 1> q1;
  const std::integral_constant<int, 2> q2;
  const std::integral_constant<int, Q - 1> last;
  // This wave's loads of the next step have arrived and its reads of this one are done; then everyone's.
  const auto step_end = [] {
    asm volatile("" ::: "memory");  // (the barrier alone does not keep the compiler from moving reads across)
    __builtin_amdgcn_s_waitcnt(wait_loads((S - 2) * PL));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  typedef typename std::conditional<Q == 4, int, uint16_t>::type scales_t;
  const auto turn = [&](int c) {
    const uint8_t* cur = sc + (c % S) * (ROWS * 128);
    read(cur, 0, w0, x0);
    const uint8_t* sp = ss + ((c >> 2) & 1) * (ROWS * 32) + (((c & 3) * 2 + half) ^ (l32 >> 3)) * 4 + wk * Q;
#pragma unroll
    for (int m = 0; m < MT; ++m) sa[m] = *reinterpret_cast<const scales_t*>(sp + ra * 32 + tile_row(m) * 32);
#pragma unroll
    for (int n = 0; n < NT; ++n) sx[n] = *reinterpret_cast<const scales_t*>(sp + rb * 32 + n * 1024);
    __builtin_amdgcn_sched_barrier(0);
    load_codes(c + S - 1);
    if ((c & 3) == 0) load_scales((c >> 2) + 1);  // (older than the S - 2 steps in flight when that group begins)
    multiply(last, w1, x1, sp1, sp2);
    read(cur, 1, w1, x1);
    multiply(q0, w0, x0, sa, sx);
    if constexpr (Q == 4) {
      read(cur, 2, w0, x0);
      multiply(q1, w1, x1, sa, sx);
      read(cur, 3, w1, x1);
      multiply(q2, w0, x0, sa, sx);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) sp1[m] = sa[m];
#pragma unroll
    for (int n = 0; n < NT; ++n) sp2[n] = sx[n];
    step_end();
  };
  load_scales(0);
#pragma unroll
  for (int c = 0; c < S - 1; ++c) load_codes(c);
  step_end();
  for (int c = 0; c < kb; ++c) turn(c);
  multiply(last, w1, x1, sp1, sp2);
  __builtin_amdgcn_s_waitcnt(wait_loads(0));  // nothing may arrive in the LDS that the results take
  __syncthreads();

  // Out: each group's sums of TB tokens to a stage's LDS (16-byte units exchanged by the token's number), then eight outputs a
  // thread. A group has S / WK stages.
  constexpr int SG = S / WK, RB = BM * 4, TB = ROWS * 128 / RB / 32 * 32, TP = BN < SG * TB ? BN : SG * TB, GR = OUTS / 8;
  constexpr int XM = BM / 4 < 32 ? BM / 4 - 1 : 31;  // units of a row are exchanged among themselves
  static_assert(SG >= 1 && TB >= 32, "out");
  const auto at = [&](int grp, int tk) {  // token tk's row in a group's stages; the stage is wave-uniform where tk is a tile's
    const int s = grp * SG + (SG > 1 ? tk / TB : 0), r = SG > 1 ? tk % TB : tk;
    return sc + s * (ROWS * 128) + r * RB;
  };
#pragma unroll
  for (int t0 = 0; t0 < BN; t0 += TP) {
    if (t0) __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int tk = wn * (NT * 32) + n * 32 - t0;  // of the tile's first token
      if (tk >= 0 && tk < TP) {
        uint8_t* row = at(wk, tk) + l32 * RB;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int unit = (ra - l32 + tile_row(m)) / 4 + 2 * q + half;
            const f32x4 v = {acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
            *reinterpret_cast<f32x4*>(row + ((unit ^ (l32 & XM)) << 4)) = v;
          }
      }
    }
    __syncthreads();
#pragma unroll 2
    for (int e = tid; e < TP * GR; e += NW * 64) {
      const int tk = e / GR, j = e % GR, x = tk & XM;
      if (t0 + tk >= toks) continue;
      const auto eight = [&](int unit, float (&v)[8]) {
#pragma unroll
        for (int grp = 0; grp < WK; ++grp) {
          const uint8_t* row = at(grp, tk);
          const f32x4 lo = *reinterpret_cast<const f32x4*>(row + ((unit ^ x) << 4)), hi = *reinterpret_cast<const f32x4*>(row + (((unit + 1) ^ x) << 4));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = grp ? v[i] + lo[i] : lo[i];
            v[4 + i] = grp ? v[4 + i] + hi[i] : hi[i];
          }
        }
      };
      float g[8], u[8];
      eight(2 * j, g);
      if constexpr (GATED) eight(OUTS / 4 + 2 * j, u);
      mx_finish<GATED, 8>(a, tok0 + t0 + tk, row0 + 8 * j, g, u);
    }
  }
}

// The tile by the number of 16 x 16 squares of rows of the weights (both matrices' if GATED) and tokens. us, k = 4096 unless
// said, rows x tokens: up to four squares a workgroup, straight from memory, while that makes at most 256 workgroups
// (4096 x 32 few<1,2> 6.5, few<1,1> 7.9, 64 x 32 tiles 7.9; 4096 x 64 few<2,2> 8.0, few<1,2> 11.3, 64 x 64 tiles 9.3; of more
// tokens, each reading the weights again, 1049 x 173 at k = 8704 few<2,2> 18.8, 64 x 64 tiles 12.7; of many rows 32768 x 8 few<1,1> 20.8,
// 64 x 32 tiles 15.2); then tiles through LDS: 64 x 64 up to 512 of them (4096 x 256 9.2, 128 x 128 14.6; 4096 x 512 13.5, 15.0;
// 4096 x 1024 24.6, 16.4), 128 x 128 in four stages where each has a compute unit of its own (4096 x 1024 16.4, in two stages
// 20.1), in two where two share one (4096 x 2048 28.4, 31.7), and 256 x 256 where the chip's places are as full with them
// (4096 x 4096 at k = 2048 22.4, 128 x 128 27.7; 4096 x 1500 at 7168 57.7, 39.0).
template <bool GATED>
static void launch_mx(const MxArgs& a, hipStream_t st) {
  const auto up = [](int64_t x, int64_t y) { return (unsigned)((x + y - 1) / y); };
  const int64_t rows = (int64_t)a.n * (GATED ? 2 : 1);
  const auto count = [&](int64_t bm, int64_t bn) { return up(rows, bm) * (int64_t)up(a.t, bn); };
  const auto few = [&](auto mt, auto nt) {
    constexpr int MT = decltype(mt)::value, NT = decltype(nt)::value;
    hipLaunchKernelGGL((k_mx_few<MT, NT, 8, GATED>), dim3(up(a.n, (GATED ? 8 : 16) * MT), up(a.t, NT * 16)), dim3(512), 0, st, a);
  };
  const auto tile = [&](auto kernel, int bm, int bn, int threads) {
    hipLaunchKernelGGL(kernel, dim3(up(a.n, GATED ? bm / 2 : bm), up(a.t, bn)), dim3(threads), 0, st, a);
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  const int64_t squares = count(16, 16);
  if (a.t == 1 || squares <= 256 || (a.t <= 16 && squares <= 1536)) few(one, one);
  else if (squares <= 512) few(one, two);
  else if (squares <= 1024 && a.t <= 64) few(two, two);
  else if (a.t <= 32) tile(k_mx_tile<64, 32, GATED ? 1 : 2, 1, 1, 4, GATED>, 64, 32, GATED ? 64 : 128);
  else if (count(64, 64) <= 512) tile(k_mx_tile<64, 64, GATED ? 1 : 2, 2, 2, 4, GATED>, 64, 64, GATED ? 256 : 512);
  else if (20 * ((count(256, 256) + 255) / 256) <= 11 * ((count(128, 128) + 511) / 512)) tile(k_mx_tile<256, 256, 4, 4, 1, 2, GATED>, 256, 256, 1024);
  else if (count(128, 128) <= 256) tile(k_mx_tile<128, 128, 2, 4, 1, 4, GATED>, 128, 128, 512);
  else tile(k_mx_tile<128, 128, 2, 4, 1, 2, GATED>, 128, 128, 512);
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
