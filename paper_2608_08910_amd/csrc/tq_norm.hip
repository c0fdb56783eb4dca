// Norms around a block, fused with the block's gate and the scaled residual (formulas in tq.h).
//
// A row is held in registers by one workgroup of TPR threads, 4 * NR elements a thread: every
// tensor is read once and written once, and the row's mean squares are the only exchange. Bound by memory: 2048 rows of 4096 in
// fp32 (134 MB) 29 us, 4.6 TB/s (a copy: 5.1); one row of 7168 4.2 us. Gradients of 2047 rows of 4096, stream in bfloat16 (151 MB)
// 33 us, and 4.8 for the join.
#include <algorithm>

#include "tq_ops.hpp"

namespace tq {

constexpr int kNormMaxHidden = 16384;

struct NormArgs {
  const float *g_post, *gate, *g_pre;
  int gate_kind, hidden;
  float res_scale, eps;
  const float* gate_tok;  // (backward: a token's gate; gate is then a channel's)
};

// Sums over the TPR threads of a workgroup; all threads receive them. `buf` holds N * TPR / 64
// floats that no earlier exchange still reads.
template <int TPR, int N>
__device__ __forceinline__ void block_sum(float (&v)[N], float* buf) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = wave_sum_f32(v[n]);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) buf[n * W + (threadIdx.x >> 6)] = v[n];
    }
    __syncthreads();
    const int w = threadIdx.x & 15;  // (16 lanes add the waves' sums up: one read each)
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = row_sum_f32(w < W ? buf[n * W + min(w, W - 1)] : 0.0f);
  }
}

// How a row's n columns meet the fours that threads take. Rows of a width that is no multiple of four start at any element:
// there the fours are those of the whole tensor, so that its loads and stores stay whole and aligned, and element c of them is
// column c - m of the row. (Fours of the row itself: 2048 rows of 4093 in fp32 39 us, these 31; elements one by one: 1650 rows of 5077
// 68 us, these 35, their gradients 117 and 64.) A thread past the row, and the
// last four of the tensor, read an earlier four that ends with the tensor, rotated.
template <int ROW>
struct Span {
  uint32_t m, n, end;  // end: elements that may be read (another row follows: three more than the row's)
  __device__ __forceinline__ Span(int64_t row, int64_t t, uint32_t width) : n(width) {
    // (the widest rows take their own fours: with others before and after, they would not fit a workgroup)
    m = ROW == kRowTail && width <= kNormMaxHidden - 3 ? (uint32_t)row * width & 3 : 0;
    end = ROW == kRowTail && row + 1 < t ? m + n + 3 : m + n;
  }
  __device__ __forceinline__ bool has(uint32_t c, int i) const {
    return ROW == kRowWhole ? c < n : c + i - m < n;  // (before the row: a large number)
  }
  template <typename T>
  __device__ __forceinline__ void raw(const T* from, uint32_t c, typename VecOf<T, 4>::type& v) const {
    if constexpr (ROW != kRowShort) {
      v = *reinterpret_cast<const typename VecOf<T, 4>::type*>(at_element(from, min(c, end - 4)));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *at_element(from, min(c + i, n - 1));
    }
  }
  // a row's elements as fp32, `fill` outside it (`from`: m elements before the row)
  template <typename V>
  __device__ __forceinline__ void get(const V& v, uint32_t c, float (&f)[4], bool there = true, float fill = 0.0f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)v[i];
    if constexpr (ROW == kRowTail) rotate(f, c - min(c, end - 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = there && has(c, i) ? f[i] : fill;
  }
  template <typename T>
  __device__ __forceinline__ void load(const T* from, uint32_t c, float (&f)[4]) const {
    typename VecOf<T, 4>::type v;
    raw(from, c, v);
    get(v, c, f);
  }
  // by column, from an array of n
  __device__ __forceinline__ void column(const float* w, uint32_t c, float (&f)[4]) const {
    if constexpr (ROW == kRowTail) {
      const uint32_t s = min(max(c, m), m + n - 4) - m;
      load_n<4>(at_element(w, s), f);
      rotate(f, c - m - s);
    } else {
      load_row<ROW, 4>(w, c, n, f);
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* to, uint32_t c, const float (&f)[4]) const {
    if (ROW == kRowWhole ? c < n : ROW == kRowTail && c >= m && c + 4 <= m + n) {
      store_n<4>(at_element(to, c), f);
    } else if (ROW != kRowWhole) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (has(c, i)) *at_element(to, c + i) = (T)f[i];
    }
  }
};

template <typename X, typename Y, int TPR, int NR, int ROW>
__global__ __launch_bounds__(TPR) void k_block_norm(const X* x, const Y* y, int64_t row0, int64_t t, NormArgs A, X* x_out, Y* h) {
  __shared__ float s_buf[2][TPR / 64];
  const int H = A.hidden, tid = threadIdx.x;
  const int64_t row = row0 + blockIdx.x;
  const Span<ROW> S(row, t, H);
  const int64_t off = row * H - S.m;
  float xv[NR][4], yv[NR][4], gp[NR][4], ga[NR][4];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int c = (r * TPR + tid) * 4;
    S.load(x + off, c, xv[r]);
    if (y) S.load(y + off, c, yv[r]);
  }
  const float n = 1.0f / (float)H;
  if (y) {
    const float gt = A.gate_kind == TQ_GATE_TOKEN ? A.gate[row] : 1.0f;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const int c = (r * TPR + tid) * 4;
#pragma unroll
      for (int i = 0; i < 4; ++i) gp[r][i] = 1.0f, ga[r][i] = gt;
      if (A.g_post) S.column(A.g_post, c, gp[r]);
      if (A.gate_kind == TQ_GATE_CHANNEL) S.column(A.gate, c, ga[r]);
    }
    float r2 = 1.0f;
    if (A.g_post) {
      float s[1] = {0.0f};
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[0] = fmaf(yv[r][i], yv[r][i], s[0]);
      block_sum<TPR>(s, s_buf[0]);
      r2 = 1.0f / sqrtf(fmaf(s[0], n, A.eps));
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) {
#pragma unroll
      for (int i = 0; i < 4; ++i) xv[r][i] = fmaf(ga[r][i], yv[r][i] * r2 * gp[r][i], A.res_scale * xv[r][i]);
      S.store(x_out + off, (r * TPR + tid) * 4, xv[r]);
    }
  }
  if (!h) return;
  // the norm of the unrounded stream: its rounding to the stream's type does not reach h
  float s[1] = {0.0f};
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    S.column(A.g_pre, (r * TPR + tid) * 4, gp[r]);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[0] = fmaf(xv[r][i], xv[r][i], s[0]);
  }
  block_sum<TPR>(s, s_buf[1]);
  const float r1 = 1.0f / sqrtf(fmaf(s[0], n, A.eps));
#pragma unroll
  for (int r = 0; r < NR; ++r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) xv[r][i] = xv[r][i] * r1 * gp[r][i];
    S.store(h + off, (r * TPR + tid) * 4, xv[r]);
  }
}

// The start of a row, kept in scalar registers (else a loop over rows carries a vector address per tensor and piece, and the
// weights themselves where they are to be read again each time).
template <typename T>
__device__ __forceinline__ T* row_at(T* p, int64_t off) {
  p += off;
  asm volatile("" : "+s"(p));
  return p;
}

// Four consecutive elements of each of a row's tensors as they lie in memory (their conversion waits for them, the loads do not).
template <typename X, typename Y, int ROW>
struct RowRaw {
  typename VecOf<X, 4>::type x, d;
  typename VecOf<Y, 4>::type y, q;

  __device__ __forceinline__ void load(const X* xo, const Y* yi, const X* dxo, const Y* dh, int64_t row, uint32_t c, const Span<ROW>& S) {
    const int64_t off = row * S.n - S.m;
    S.raw(row_at(xo, off), c, x);
    S.raw(row_at(dh, off), c, q);
    S.raw(row_at(dxo, off), c, d);
    S.raw(row_at(yi, off), c, y);
  }
};

// What of a backward call is there (a tensor that is not has another's address, so that the loads need no branch).
constexpr int kHasPost = 1, kHasGate = 2, kHasPre = 4, kHasStream = 8, kHasBlock = 16;

// Backward: workgroup b takes rows b, b + G, ... and keeps its sums by column in registers; they go
// to part[b][3][hidden] (g_post, gate, g_pre), which k_norm_join adds in a fixed order. Rows of up to 4096: the next
// row's loads are under way while a row is worked on. Rows past 8192 do not fit into registers: they are read twice, the second
// time from the cache, and two of the three sums stay in LDS.
template <typename X, typename Y, int TPR, int NR, int ROW>
__global__ __launch_bounds__(TPR) void k_block_norm_bwd(const X* xo, const Y* y, int64_t t, NormArgs A, const X* dxo,
                                                        const Y* dh, X* dx, Y* dy, float* dgate_tok, int has,
                                                        float* part) {
  constexpr bool kHold = NR <= 2, kAhead = NR == 1;  // (registers)
  constexpr int NA = kHold ? NR : 1;
  typedef RowRaw<X, Y, ROW> Raw;
  __shared__ float s_buf[2][3 * (TPR / 64)];
  const uint32_t H = A.hidden, tid = threadIdx.x;
  const float n = 1.0f / (float)H;
  const bool pre_on = has & kHasPre, post_on = has & kHasPost, gate_on = has & kHasGate, d_on = has & kHasStream, y_on = has & kHasBlock;
  float a_post[NA][4] = {}, a_gate[NA][4] = {}, a_pre[NR][4] = {};
  __shared__ f32x4 s_sum[kHold ? 1 : 2][kHold ? 1 : NR * TPR];  // (each thread its own)
  if constexpr (!kHold) {
#pragma unroll
    for (int r = 0; r < NR; ++r) s_sum[0][r * TPR + tid] = s_sum[1][r * TPR + tid] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  int64_t row = blockIdx.x;
  Span<ROW> S(row, t, H);  // (m is that of all the workgroup's rows: they lie a multiple of four apart)
  auto weights = [&](int r, float (&pre)[4], float (&post)[4], float (&ga)[4]) {
    const uint32_t c = (r * TPR + tid) * 4;
    S.column(row_at(A.g_pre, 0), c, pre);
    S.column(row_at(A.g_post, 0), c, post);
    S.column(row_at(A.gate, 0), c, ga);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      pre[i] = pre_on ? pre[i] : 0.0f;
      post[i] = post_on ? post[i] : 1.0f;
      ga[i] = gate_on ? ga[i] : 1.0f;
    }
  };
  float gpre[4], gpost[4], gate[4];
  if constexpr (kAhead) weights(0, gpre, gpost, gate);
  Raw raw[kHold ? NR : 1];
  if constexpr (kAhead) {
#pragma unroll
    for (int r = 0; r < NR; ++r) raw[r].load(xo, y, dxo, dh, row, (r * TPR + tid) * 4, S);
  }
  for (; row < t; row += gridDim.x) {
    S = Span<ROW>(row, t, H);
    const int64_t off = row * H - S.m;
    float xv[kHold ? NR : 1][4], dv[kHold ? NR : 1][4], yv[NR][4], q[NR][4];
    float s[3] = {0.0f, 0.0f, 0.0f};  // <x', x'>, <dh g_pre, x'>, <y, y>
    if constexpr (kHold && !kAhead) {
#pragma unroll
      for (int r = 0; r < NR; ++r) raw[r].load(xo, y, dxo, dh, row, (r * TPR + tid) * 4, S);
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const uint32_t c = (r * TPR + tid) * 4;
      const int k = kHold ? r : 0;
      float pre[4];
      if constexpr (!kHold) {
        asm volatile("" ::: "memory");  // (one piece at a time: together they would not fit)
        raw[0].load(xo, y, dxo, dh, row, c, S);
      }
      if constexpr (kAhead) {
#pragma unroll
        for (int i = 0; i < 4; ++i) pre[i] = gpre[i];
      } else {
        S.column(row_at(A.g_pre, 0), c, pre);
#pragma unroll
        for (int i = 0; i < 4; ++i) pre[i] = pre_on ? pre[i] : 0.0f;
      }
      S.get(raw[k].x, c, xv[k], pre_on);
      S.get(raw[k].y, c, yv[r], y_on);
      S.get(raw[k].q, c, q[r], pre_on);
      if constexpr (kHold) S.get(raw[k].d, c, dv[k], d_on);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[0] = fmaf(xv[k][i], xv[k][i], s[0]);
        s[1] = fmaf(q[r][i] * pre[i], xv[k][i], s[1]);
        s[2] = fmaf(yv[r][i], yv[r][i], s[2]);
      }
    }
    if constexpr (kAhead) {  // (the last one's again at the end)
      const int64_t next = row + gridDim.x < t ? row + gridDim.x : row;
      const Span<ROW> N(next, t, H);
#pragma unroll
      for (int r = 0; r < NR; ++r) raw[r].load(xo, y, dxo, dh, next, (r * TPR + tid) * 4, N);
    }
    block_sum<TPR>(s, s_buf[0]);
    const float r1 = pre_on ? 1.0f / sqrtf(fmaf(s[0], n, A.eps)) : 0.0f;
    // (two of the three factors on the mean, one after the other, and one on the sum: their cube leaves the range of fp32 for rows of
    // root mean square past 1e15, and for rows of zeros with eps below 2e-26. 690 rows of 12004 88 us, with the cube 90, with the
    // second factor on the row's values 111.)
    const float k1 = r1 * (r1 * (s[1] * n));
    const float r2 = post_on ? 1.0f / sqrtf(fmaf(s[2], n, A.eps)) : 1.0f;
    const float gt = A.gate_kind == TQ_GATE_TOKEN ? A.gate_tok[row] : 1.0f;
    float u[2] = {0.0f, 0.0f};  // <dn g_post, y>, <D, n>
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const uint32_t c = (r * TPR + tid) * 4;
      const int k = kHold ? r : 0;
      float pre[4], post[4], ga[4], o[4];
      if constexpr (!kHold) {
        asm volatile("" ::: "memory");
        raw[0].load(xo, y, dxo, dh, row, c, S);
        S.get(raw[0].x, c, xv[0], pre_on);
        S.get(raw[0].d, c, dv[0], d_on);
        S.get(raw[0].y, c, yv[r], y_on);
        S.get(raw[0].q, c, q[r], pre_on);
      }
      if constexpr (kAhead) {
#pragma unroll
        for (int i = 0; i < 4; ++i) pre[i] = gpre[i], post[i] = gpost[i], ga[i] = gate[i];
      } else {
        weights(r, pre, post, ga);
      }
      f32x4 sp, sg;
      if constexpr (!kHold) sp = s_sum[0][r * TPR + tid], sg = s_sum[1][r * TPR + tid];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float D = fmaf(r1, fmaf(-k1, xv[k][i], q[r][i] * pre[i]), dv[k][i]);
        a_pre[r][i] = fmaf(q[r][i], xv[k][i] * r1, a_pre[r][i]);
        o[i] = A.res_scale * D;
        const float yn = yv[r][i] * r2, dn = ga[i] * gt * D;
        if constexpr (kHold) {
          a_gate[r][i] = fmaf(D, yn * post[i], a_gate[r][i]);
          a_post[r][i] = fmaf(dn, yn, a_post[r][i]);
        } else {
          sg[i] = fmaf(D, yn * post[i], sg[i]);
          sp[i] = fmaf(dn, yn, sp[i]);
        }
        u[0] = fmaf(dn * post[i], yv[r][i], u[0]);
        u[1] = fmaf(D, yn * post[i], u[1]);
        q[r][i] = dn * post[i];
      }
      if constexpr (!kHold) s_sum[0][r * TPR + tid] = sp, s_sum[1][r * TPR + tid] = sg;
      S.store(row_at(dx, off), c, o);
    }
    block_sum<TPR>(u, s_buf[1]);
    if (!y_on) continue;
    if (dgate_tok && tid == 0) dgate_tok[row] = u[1];
    const float k2 = r2 * (r2 * (u[0] * n));
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = post_on ? r2 * fmaf(-k2, yv[r][i], q[r][i]) : q[r][i];  // (an infinite y: 0 * inf)
      S.store(row_at(dy, off), (r * TPR + tid) * 4, o);
    }
  }
  float* p = part + (int64_t)blockIdx.x * 3 * H - S.m;
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const uint32_t c = (r * TPR + tid) * 4;
    if constexpr (!kHold) {
#pragma unroll
      for (int i = 0; i < 4; ++i) a_post[0][i] = s_sum[0][r * TPR + tid][i], a_gate[0][i] = s_sum[1][r * TPR + tid][i];
    }
    if (post_on) S.store(p, c, a_post[kHold ? r : 0]);
    if (gate_on) S.store(p + H, c, a_gate[kHold ? r : 0]);
    if (pre_on) S.store(p + 2 * H, c, a_pre[r]);
  }
}

// Column sums of part[groups][3][H]: 64 columns and 16 groups of rows a workgroup, in order.
__global__ __launch_bounds__(1024) void k_norm_join(const float* part, int groups, int H, float* dg_post, float* dgate,
                                                    float* dg_pre) {
  __shared__ float s_v[16][64];
  float* out = blockIdx.y == 0 ? dg_post : blockIdx.y == 1 ? dgate : dg_pre;
  if (!out) return;
  const int lane = threadIdx.x & 63, row = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float v = 0.0f;
  if (c < H) {
    const float* p = part + (int64_t)blockIdx.y * H + c;
#pragma unroll 8
    for (int g = row; g < groups; g += 16) v += p[(int64_t)g * 3 * H];
  }
  s_v[row][lane] = v;
  __syncthreads();
  if (row == 0 && c < H) {
#pragma unroll
    for (int k = 1; k < 16; ++k) v += s_v[k][lane];
    out[c] = v;
  }
}

// Columns that a row's threads have to span: up to three before or after it, where its fours are the tensor's.
static int norm_span(int H) { return H % 4 == 0 || H < 4 || H > kNormMaxHidden - 3 ? H : H + 3; }
static int norm_tpr(int H) {  // threads of a row in the backward pass
  const int w = norm_span(H);
  return w <= 256 ? 64 : w <= 1024 ? 256 : w <= 2048 ? 512 : 1024;
}
// About two thousand threads a compute unit, but eight rows a workgroup where there are enough (each workgroup leaves parts
// to join). A multiple of four where a workgroup has several rows, for Span.
static int norm_groups(int64_t t, int H) {
  const int64_t most = 256 * 2048 / norm_tpr(H), g = std::max<int64_t>(256, (t + 31) / 32 * 4);
  return (int)std::min(t, std::min(g, most));
}
static size_t norm_ws(int64_t t, int H) {
  const size_t b = (size_t)norm_groups(t, H) * 3 * H * 4;
  return b < 256 ? 256 : (b + 255) / 256 * 256;
}

// Calls f(X, Y) with the stream's and the block's element types.
template <typename F>
static void with_types(int32_t xt, int32_t yt, F f) {
  with_type(xt, [&](auto x) {
    if (yt == xt) f(x, x);
    else f(x, float{});
  });
}
template <int TPR, int NR>
struct RowShape {
  static constexpr int tpr = TPR, nr = NR;
};
// (rows shorter than a vector run on 64 threads only)
template <int TPR, int ROW>
constexpr int row_end() { return TPR > 64 && ROW == kRowShort ? kRowTail : ROW; }
// Gradients of rows past 8192 take the code of odd widths for every width, for which the compiler finds a better use of the few
// registers left (29 to 37 of them spill all the same): 511 rows of 16384 84 us against 105, 690 of 12004 94 against 124.
template <typename S, int ROW>
constexpr int bwd_row_end() { return S::nr > 2 ? kRowTail : row_end<S::tpr, ROW>(); }

static tq_status check_norm(const char* fn, int32_t xt, int32_t yt, int64_t t, int32_t H, const float* g_post,
                            const float* gate, int32_t gate_kind, const float* g_pre, float eps, bool has_y) {
  if (!known_type(xt) || !known_type(yt) || (yt != xt && yt != TQ_F32))
    return fail(TQ_ERR_INVALID, "%s: types %d, %d: the block's type must be the stream's or fp32", fn, xt, yt);
  if (t < 0 || t > (1 << 24)) return fail(TQ_ERR_INVALID, "%s: t = %lld outside [0, 2^24]", fn, (long long)t);
  if (H < 1 || H > kNormMaxHidden) return fail(TQ_ERR_INVALID, "%s: hidden = %d outside [1, %d]", fn, H, kNormMaxHidden);
  if (gate_kind < TQ_GATE_NONE || gate_kind > TQ_GATE_TOKEN || (t > 0 && (gate_kind != TQ_GATE_NONE) != (gate != nullptr)))
    return fail(TQ_ERR_INVALID, "%s: gate kind %d %s a gate", fn, gate_kind, gate ? "with" : "without");
  if (!(eps > 0.0f) || eps > 1.0f) return fail(TQ_ERR_INVALID, "%s: eps = %g outside (0, 1]", fn, (double)eps);
  if (t > 0 && !has_y && (g_post || gate)) return fail(TQ_ERR_INVALID, "%s: g_post or gate without y", fn);
  if (!aligned(g_post, 4) || !aligned(gate, 4) || !aligned(g_pre, 4))
    return fail(TQ_ERR_ALIGN, "%s: g_post, gate and g_pre must be 4-byte aligned", fn);
  return TQ_OK;
}

}  // namespace tq

extern "C" tq_status tq_block_norm(const void* x, int32_t x_type, const void* y, int32_t y_type, int64_t t,
                                   int32_t hidden, const float* g_post, const float* gate, int32_t gate_kind,
                                   float res_scale, const float* g_pre, float eps, void* x_out, void* h, void* stream) {
  using namespace tq;
  clear_error();
  const char* fn = "tq_block_norm";
  tq_status st = check_norm(fn, x_type, y_type, t, hidden, g_post, gate, gate_kind, g_pre, eps, y != nullptr);
  if (st != TQ_OK || t == 0) return st;
  if (!x || (!y && !h) || !y != !x_out || !h != !g_pre)
    return fail(TQ_ERR_INVALID, "%s: null x, neither y nor h, y and x_out not together, or h and g_pre not together", fn);
  if (!aligned(x, type_bytes(x_type)) || !aligned(x_out, type_bytes(x_type)) || !aligned(y, type_bytes(y_type)) ||
      !aligned(h, type_bytes(y_type)))
    return fail(TQ_ERR_ALIGN, "%s: x, y, x_out and h must be aligned to their types", fn);
  (void)hipGetLastError();
  const int span = norm_span(hidden);
  const NormArgs A = {g_post, gate, g_pre, gate_kind, hidden, res_scale, eps, nullptr};
  with_types(x_type, y_type, [&](auto xv, auto yv) {
    using X = decltype(xv);
    using Y = decltype(yv);
    auto go = [&](auto shape) {
      using S = decltype(shape);
      with_row(hidden, [&](auto end) {
        const int64_t most = items_per_launch(S::tpr);
        for (int64_t row0 = 0; row0 < t; row0 += most)
          hipLaunchKernelGGL((k_block_norm<X, Y, S::tpr, S::nr, row_end<S::tpr, decltype(end)::value>()>),
                             dim3((unsigned)std::min(most, t - row0)), dim3(S::tpr), 0, (hipStream_t)stream,
                             static_cast<const X*>(x), static_cast<const Y*>(y), row0, t, A, static_cast<X*>(x_out), static_cast<Y*>(h));
      });
    };
    if (span <= 256) go(RowShape<64, 1>{});
    else if (span <= 1024) go(RowShape<256, 1>{});
    else if (span <= 2048) go(RowShape<256, 2>{});
    else if (span <= 4096) go(RowShape<256, 4>{});
    else if (span <= 8192) go(RowShape<512, 4>{});
    else go(RowShape<1024, 4>{});
  });
  return check_launch(fn);
}

extern "C" size_t tq_block_norm_workspace_bytes(int64_t t, int32_t hidden) {
  if (t < 0 || t > (1 << 24) || hidden < 1 || hidden > tq::kNormMaxHidden) return 0;
  return tq::norm_ws(t, hidden);
}

extern "C" tq_status tq_block_norm_bwd(const void* x_out, int32_t x_type, const void* y, int32_t y_type, int64_t t,
                                       int32_t hidden, const float* g_post, const float* gate, int32_t gate_kind,
                                       float res_scale, const float* g_pre, float eps, const void* dx_out,
                                       const void* dh, void* dx, void* dy, float* dg_post, float* dgate, float* dg_pre,
                                       void* ws, size_t ws_bytes, void* stream) {
  using namespace tq;
  clear_error();
  const char* fn = "tq_block_norm_bwd";
  const bool has_y = dy != nullptr;
  tq_status st = check_norm(fn, x_type, y_type, t, hidden, g_post, gate, gate_kind, g_pre, eps, has_y);
  if (st != TQ_OK) return st;
  if (!dg_pre != !g_pre || !dg_post != !g_post || (gate_kind != TQ_GATE_TOKEN && !dgate != !gate) || !ws)
    return fail(TQ_ERR_INVALID, "%s: null ws, or dg_post, dgate or dg_pre without its input (or the reverse)", fn);
  if (t > 0 && (!dx || (dh && !x_out) || !y != !dy || !dh != !g_pre || (!dx_out && !dh) || (!y && !dh) || !dgate != !gate))
    return fail(TQ_ERR_INVALID,
                "%s: null dx, dh without x_out, no incoming gradient, neither y nor dh, or not together: y and dy, dh and g_pre, "
                "gate and dgate",
                fn);
  for (const void* p : {x_out, dx_out, (const void*)dx})
    if (!aligned(p, type_bytes(x_type))) return fail(TQ_ERR_ALIGN, "%s: the stream's tensors must be aligned to their type", fn);
  for (const void* p : {y, dh, (const void*)dy})
    if (!aligned(p, type_bytes(y_type))) return fail(TQ_ERR_ALIGN, "%s: the block's tensors must be aligned to their type", fn);
  if (!aligned(dg_post, 4) || !aligned(dgate, 4) || !aligned(dg_pre, 4) || !aligned(ws, 256))
    return fail(TQ_ERR_ALIGN, "%s: gradients must be 4-byte aligned, ws 256-byte aligned", fn);
  if (ws_bytes < norm_ws(t, hidden))
    return fail(TQ_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, norm_ws(t, hidden));
  (void)hipGetLastError();
  const int span = norm_span(hidden);
  const int groups = norm_groups(t, hidden);
  float* part = static_cast<float*>(ws);
  float* dg_ch = gate_kind == TQ_GATE_CHANNEL ? dgate : nullptr;
  float* dg_tok = gate_kind == TQ_GATE_TOKEN ? dgate : nullptr;
  const int want = (dg_post ? kHasPost : 0) | (dg_ch ? kHasGate : 0) | (dg_pre ? kHasPre : 0);
  const int has = want | (dx_out ? kHasStream : 0) | (has_y ? kHasBlock : 0);
  // what is not there takes an address of its type and size that is: the kernel loads it and drops it
  const NormArgs A = {g_post ? g_post : part, dg_ch ? gate : part, g_pre ? g_pre : part, gate_kind, hidden,
                      has_y ? res_scale : 1.0f, eps, gate};
  if (!dh) x_out = dx_out, dh = y;
  if (!dx_out) dx_out = x_out;
  if (!y) y = dh;
  if (t > 0)
    with_types(x_type, y_type, [&](auto xv, auto yv) {
      using X = decltype(xv);
      using Y = decltype(yv);
      auto go = [&](auto shape) {
        using S = decltype(shape);
        with_row(hidden, [&](auto end) {
          hipLaunchKernelGGL((k_block_norm_bwd<X, Y, S::tpr, S::nr, bwd_row_end<S, decltype(end)::value>()>), dim3((unsigned)groups),
                             dim3(S::tpr), 0, (hipStream_t)stream, static_cast<const X*>(x_out), static_cast<const Y*>(y), t,
                             A, static_cast<const X*>(dx_out), static_cast<const Y*>(dh), static_cast<X*>(dx),
                             static_cast<Y*>(dy), dg_tok, has, part);
        });
      };
      switch (norm_tpr(hidden)) {
        case 64: go(RowShape<64, 1>{}); break;
        case 256: go(RowShape<256, 1>{}); break;
        case 512:
          go(RowShape<512, 1>{});
          break;
        default:
          if (span <= 4096) go(RowShape<1024, 1>{});
          else if (span <= 8192) go(RowShape<1024, 2>{});
          else go(RowShape<1024, 4>{});
      }
    });
  if (want)
    hipLaunchKernelGGL(k_norm_join, dim3((unsigned)((hidden + 63) / 64), 3), dim3(1024), 0, (hipStream_t)stream, part,
                       groups, hidden, dg_post, dg_ch, dg_pre);
  return check_launch(fn);
}
