// Low-rank adapters of many requests beside a shared projection (formulas in tq.h).
//
// Few tokens: each token's adapter is read by waves of its own (k_lora_shrink_row, then
// k_lora_expand_row, or k_lora_row for both). Many: a plan sorts the tokens by adapter, and tiles of 32 tokens of one
// adapter run on the matrix unit, with products and sums of fp32 arithmetic for every adapter type.
//
// Times at 4096 x 4096 in bfloat16: 2043 tokens of 8 adapters of rank 64 (109 MB, 21 us of memory time) plan 6.1 us, first product
// 14.5, second 23.4; 1 token of rank 16 4.8 us a call. Gradients of 2048 tokens of 8 adapters of rank 16 beside 2048 x 4096
// (122 MB, 24 us): plan 6, first product 8, second 18.4, db 8.8, da 13.6.
//
// Operands of the fp32 matrix instruction 16x16x4 (wave64): A row = lane & 15, B column = lane & 15, both k = lane >> 4;
// the result's column = lane & 15, its rows 4 * (lane >> 4) + j. The order of k is free as long as A and
// B agree: lane group q takes the four consecutive k's 4q .. 4q+3 of sixteen, one vector load each,
// and instruction j multiplies the j-th of them.
#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "tq_ops.hpp"

namespace tq {

constexpr int kLoraMaxAdapters = 1024;
constexpr int kLoraMaxRank = 128;
constexpr int kLoraTile = 32;      // tokens of a tile: two halves, which share what is loaded of an adapter
constexpr int kLoraMaxSplit = 16;  // workgroups that share a tile's columns in the first product
constexpr int kLoraJoin = 4;       // parts of theirs that the second product reads at once
constexpr int kPlanWaves = 16;

// What a call keeps in its workspace. low: the first product's parts [split][tile][32][rank]; sum: the
// gradient's u [t][rank]. The plan: tile_group[tile] and
// slots[tile][32], the tokens of a tile (-1 past its end); an adapter's tiles are consecutive, from tile
// first[g] on, and count[g] tokens fill them. Group n_adapters holds the tokens without an adapter; tiles
// that no group needs have group -1.
struct LoraWs {
  size_t low, sum, first, count, tile_group, slots, total;
  int64_t tiles;  // at most
};
// Workgroups that share a tile's columns in the first product, at most: four, or fewer where there are four workgroups a compute unit
// without; of few tiles more, 128 workgroups in all (gradients of 120 tokens of rank 32 beside 16001 x 256, 16 splits 33 us, 4 53;
// 256 workgroups: 1000 tokens of rank 128 beside 4096 x 4096 46 us against 42 for the longer join).
static int lora_splits(int64_t tiles) {
  return (int)std::min<int64_t>(kLoraMaxSplit, std::max(std::min<int64_t>(4, std::max<int64_t>(1, 1024 / tiles)), 128 / tiles));
}
// The most parts [32][rank] that the first product of at most `tiles` tiles writes, so that the workspace of a batch holds that of
// every smaller one: lora_splits(i) * i grows to 128 parts at 8 tiles, from 32 tiles on to 1024 at 256, and is at most 1024 or i past them.
static int64_t lora_parts(int64_t tiles) {
  return std::max(tiles, std::min<int64_t>(1024, std::max(4 * tiles, std::min<int64_t>(128, kLoraMaxSplit * tiles))));
}
static LoraWs lora_ws(int n_adapters, int rank, int64_t t) {
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  LoraWs L;
  L.tiles = (t + kLoraTile - 1) / kLoraTile + (t < n_adapters + 1 ? t : n_adapters + 1);
  L.low = 0;
  L.sum = up((size_t)lora_parts(L.tiles) * kLoraTile * rank * 4);
  L.first = L.sum + up((size_t)t * rank * 4);
  L.count = L.first + up((size_t)(n_adapters + 1) * 4);
  L.tile_group = L.count + up((size_t)(n_adapters + 1) * 4);
  L.slots = L.tile_group + up((size_t)L.tiles * 4);
  L.total = L.slots + up((size_t)L.tiles * kLoraTile * 4);
  return L;
}

// The plan as the kernels see it.
struct LoraPlan {
  int32_t *first, *count, *tile_group, *slots;
};
static LoraPlan plan_of(void* ws, const LoraWs& L) {
  auto* b = static_cast<uint8_t*>(ws);
  auto at = [&](size_t o) { return reinterpret_cast<int32_t*>(b + o); };
  return {at(L.first), at(L.count), at(L.tile_group), at(L.slots)};
}

// An adapter set's arrays as the kernels see them (W: the element type).
template <typename W>
struct LoraSet {
  const W* mat;  // a [na][R][width], or b [na][width][R]
  const int32_t* ranks;
  const float* scale;
  int na, R, width;
};

__device__ __forceinline__ int adapter_of(int id, int na) { return id < 0 || id >= na ? na : id; }
__device__ __forceinline__ int live_rank(const int32_t* ranks, int a, int R) {
  return ranks ? min(max(ranks[a], 0), R) : R;
}

// Stable sort of the tokens by adapter in one workgroup: each wave counts a contiguous part of the
// tokens, the counts (group major, wave minor) become first positions, and each wave places its
// part in order. No position depends on the order of the atomics.
__global__ __launch_bounds__(kPlanWaves * 64) void k_lora_plan(const int32_t* __restrict__ ids, int t, int na,
                                                               LoraPlan P, int tiles) {
  __shared__ int s_at[kPlanWaves][kLoraMaxAdapters + 1];
  __shared__ int s_scan[kPlanWaves];
  constexpr int kThreads = kPlanWaves * 64, kKept = 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ng = na + 1;
  const int chunks = (t + 63) / 64, per = (chunks + kPlanWaves - 1) / kPlanWaves;
  const int c0 = wave * per, c1 = min(c0 + per, chunks);
  // the first chunks' groups stay in registers, loaded at once (up to 4096 tokens: all of them)
  int kept[kKept];
#pragma unroll
  for (int k = 0; k < kKept; ++k) kept[k] = c0 + k < c1 && (c0 + k) * 64 + lane < t ? ids[(c0 + k) * 64 + lane] : 0;
  for (int w = 0; w < kPlanWaves; ++w)
    for (int g = tid; g < ng; g += kThreads) s_at[w][g] = 0;
  __syncthreads();
  for (int c = c0; c < c1; ++c) {
    const int tok = c * 64 + lane;
    if (tok < t) {
      int id = kept[0];
#pragma unroll
      for (int k = 1; k < kKept; ++k)
        if (c - c0 == k) id = kept[k];
      if (c - c0 >= kKept) id = ids[tok];
      atomicAdd(&s_at[wave][adapter_of(id, na)], 1);
    }
  }
  __syncthreads();
  // a thread per group: tokens, tiles, first tile (group 1024, where there is one, comes last and by itself)
  int cnt[kPlanWaves], sum = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    cnt[w] = tid < ng ? s_at[w][tid] : 0;
    sum += cnt[w];
  }
  const int own = (sum + kLoraTile - 1) / kLoraTile;
  int before = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(before, d);
    if (lane >= d) before += u;
  }
  if (lane == 63) s_scan[wave] = before;
  before -= own;
  __syncthreads();
  int used = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    if (w < wave) before += s_scan[w];
    used += s_scan[w];
  }
  auto place = [&](int g, const int (&n)[kPlanWaves], int tokens, int tile) {
    P.first[g] = tile;
    P.count[g] = tokens;
    int at = tile * kLoraTile;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
      s_at[w][g] = at;
      at += n[w];
    }
    for (int k = tokens; k % kLoraTile != 0; ++k) P.slots[tile * kLoraTile + k] = -1;
  };
  if (tid < ng) place(tid, cnt, sum, before);
  if (ng > kThreads) {
    sum = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
      cnt[w] = s_at[w][kThreads];
      sum += cnt[w];
    }
    __syncthreads();
    if (tid == 0) place(kThreads, cnt, sum, used);
    used += (sum + kLoraTile - 1) / kLoraTile;
  }
  for (int k = used + tid; k < tiles; k += kThreads) P.tile_group[k] = -1;
  __syncthreads();
  for (int c = c0; c < c1; ++c) {
    const int tok = c * 64 + lane;
    int id = kept[0];
#pragma unroll
    for (int k = 1; k < kKept; ++k)
      if (c - c0 == k) id = kept[k];
    if (c - c0 >= kKept && tok < t) id = ids[tok];
    const int g = tok < t ? adapter_of(id, na) : -1;
    const int base = g >= 0 ? s_at[wave][g] : 0;  // (read by all before the last of a group moves it on)
    int at = 0, next = -1;
    uint64_t left = __ballot(tok < t);
    while (left) {
      const int gl = readlane_i(g, __builtin_ctzll(left));
      const uint64_t same = __ballot(g == gl);
      if (g == gl) {
        at = base + __popcll(same & ((1ull << lane) - 1));
        if ((same >> lane) == 1) next = at + 1;
      }
      left &= ~same;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (next >= 0) s_at[wave][g] = next;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (g >= 0) {
      P.slots[at] = tok;
      if (at % kLoraTile == 0) P.tile_group[at / kLoraTile] = g;  // (every tile's first slot is filled)
    }
  }
}

// ---- many tokens -----------------------------------------------------------------------------

// bfloat16 adapters take the bf16 matrix instruction 16x16x32 (lane group q: k 8q .. 8q+7): an fp32 value is the exact sum
// of three bfloat16 (8 of its 24 significant bits each, cut off, so that nothing overflows), the products are
// exact in fp32 and the three go into the same fp32 sums. fp16 and fp32 adapters take the fp32 instruction, a sixteenth of
// the rate.
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));

struct Split3 {
  bf16x8 part[3];
  Split3() = default;
  __device__ __forceinline__ explicit Split3(const float (&v)[8]) {
    u32x4 w[3];
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      float a = v[j], b = v[j + 1];
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
        w[p][j / 2] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);  // the high halves of both
        a -= __uint_as_float(ua & 0xffff0000u);
        b -= __uint_as_float(ub & 0xffff0000u);
      }
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) part[p] = __builtin_bit_cast(bf16x8, w[p]);
  }
};

__device__ __forceinline__ f32x4 mfma3(const Split3& x, bf16x8 w, f32x4 acc) {
#pragma unroll
  for (int p = 2; p >= 0; --p) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.part[p], w, acc, 0, 0, 0);
  return acc;
}

// The end of a first product in a workgroup whose waves' sums lie in LDS, s[wave][slot][RT * 16]: they are added up in order, and
// go to the split's part of the tile.
struct LoraOut {
  float* low;
  int splits;
  int64_t tiles;
};
template <int RT, int WAVES>
__device__ __forceinline__ void finish_low(const float* s, const int32_t* slots, int tile, int split, int R, int rl, float sc,
                                           const LoraOut& O) {
  float* part = O.low + ((int64_t)split * O.tiles + tile) * kLoraTile * R;
  for (int o = threadIdx.x; o < kLoraTile * R; o += WAVES * 64) {
    const int tk = o / R, r = o - tk * R;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += s[(w * kLoraTile + tk) * (RT * 16) + r];
    part[o] = r < rl && slots[tk] >= 0 ? sc * v : 0.0f;
  }
}

// The first product, low[token][r] = scale * sum over the columns, a split of them a workgroup, of P[token][c] * M[r][c] for a
// tile's tokens. The waves share the columns and join their sums in LDS in order; workgroups that run together
// take neighbouring columns, not one column range of many rows.
//
// Adjacent lanes of a matrix operand are different rows of P and of M (stored [R][width]), so that loads straight
// into operands touch 64 pieces of 16 bytes (R = 64, 2043 tokens: 19 us, through LDS 13). Each wave therefore
// reads whole 128-byte lines, 8 or 16 lanes a row, and turns them in a part of LDS of its own. The next turn's lines are
// under way meanwhile. A row's 16-byte pieces lie rotated by the row's number, since the operand reads 16 rows at once.
constexpr int kShrinkWaves = 4;

// 16-byte piece p (of 2^L a row) of row r, in a wave's LDS
template <int L>
__device__ __forceinline__ int piece_at(int r, int p) { return (r << L) + ((p + r) & ((1 << L) - 1)); }

// the lane's pieces of rows [0, N) of 128 << D bytes each, whole lines a row
template <int N, int D>
struct RowPieces {
  static constexpr int L = 3 + D, kLoads = N >> (6 - L);
  uint4 v[kLoads];
  __device__ __forceinline__ void load(const uint8_t* base, int64_t stride, int last, int lane) {
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      v[k] = ld16(base + min((k << (6 - L)) + (lane >> L), last) * stride + ((lane & ((1 << L) - 1)) << 4));
  }
  __device__ __forceinline__ void put(uint4* lds, int lane) const {
#pragma unroll
    for (int k = 0; k < kLoads; ++k) lds[piece_at<L>((k << (6 - L)) + (lane >> L), lane & ((1 << L) - 1))] = v[k];
  }
};

template <typename W, int RT>
__global__ __launch_bounds__(kShrinkWaves * 64) void k_lora_shrink(const float* __restrict__ p, LoraSet<W> S,
                                                                   LoraPlan P, int cols, LoraOut O) {
  constexpr int CT = 128 / sizeof(W);      // columns a turn: a line of M's row
  constexpr int XD = sizeof(W) == 2 ? 1 : 0;  // P's row piece is two lines or one
  constexpr int XL = 3 + XD, XK = 16 >> (6 - XL);  // 2^XL pieces of a row; loads of a lane for 16 rows
  __shared__ uint4 s_m[kShrinkWaves][RT * 16 << 3];
  __shared__ uint4 s_x[kShrinkWaves][kLoraTile << XL];
  __shared__ int s_tok[kLoraTile];
  const int tile = blockIdx.x / O.splits, split = blockIdx.x - tile * O.splits;
  const int g = P.tile_group[tile];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
  const int32_t* slots = P.slots + (int64_t)tile * kLoraTile;
  int tok[2][XK];  // the tokens whose pieces the lane loads
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int k = 0; k < XK; ++k) tok[h][k] = slots[h * 16 + (k << (6 - XL)) + (lane >> XL)];
  const int own = slots[lane & (kLoraTile - 1)];
  if (g < 0) return;
  const int R = S.R, width = S.width, rl = g < S.na ? live_rank(S.ranks, g, R) : 0;
  if (rl == 0) return;  // (nobody reads the tile's values)
  if (threadIdx.x < kLoraTile) s_tok[lane] = own;
  const bool two = readlane_i(own, 16) >= 0;  // the second half has tokens
  const float* row[2][XK];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int k = 0; k < XK; ++k)  // (an empty slot reads the first slot's row; its results are dropped)
      row[h][k] = p + (int64_t)(tok[h][k] < 0 ? readlane_i(own, 0) : tok[h][k]) * width + ((lane & ((1 << XL) - 1)) << 2);
  const uint8_t* m = reinterpret_cast<const uint8_t*>(S.mat + (int64_t)g * R * width);
  const int c1 = min((split + 1) * cols, width);
  constexpr int kTurn = kShrinkWaves * CT;
  RowPieces<RT * 16, 0> w;
  uint4 x[2][XK];
  auto load = [&](int c) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (h == 0 || two) {
#pragma unroll
        for (int k = 0; k < XK; ++k) x[h][k] = ld16(row[h][k] + c);
      }
    w.load(m + (int64_t)c * sizeof(W), (int64_t)width * sizeof(W), R - 1, lane);  // (ranks past the stored ones: dropped below)
  };
  f32x4 acc[2][RT];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) acc[h][rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  // 32 columns (16 of fp32): piece 4 c + q of a row of M
  auto multiply = [&](int h, int c) {
    const uint4* xs = s_x[wave];
    const uint4* ms = s_m[wave];
    if constexpr (sizeof(W) == 2) {
      float xv[8];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const f32x4 f = __builtin_bit_cast(f32x4, xs[piece_at<XL>(h * 16 + i, 8 * c + 2 * q + k)]);
#pragma unroll
        for (int j = 0; j < 4; ++j) xv[4 * k + j] = f[j];
      }
      typedef W w8 __attribute__((ext_vector_type(8)));
      if constexpr (std::is_same<W, bf16_t>::value) {
        const Split3 sx(xv);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          acc[h][rt] = mfma3(sx, __builtin_bit_cast(w8, ms[piece_at<3>(rt * 16 + i, 4 * c + q)]), acc[h][rt]);
      } else {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const w8 b = __builtin_bit_cast(w8, ms[piece_at<3>(rt * 16 + i, 4 * c + q)]);
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[h][rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(xv[j], (float)b[j], acc[h][rt], 0, 0, 0);
        }
      }
    } else {
      const f32x4 xv = __builtin_bit_cast(f32x4, xs[piece_at<XL>(h * 16 + i, 4 * c + q)]);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const f32x4 b = __builtin_bit_cast(f32x4, ms[piece_at<3>(rt * 16 + i, 4 * c + q)]);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[h][rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(xv[j], b[j], acc[h][rt], 0, 0, 0);
      }
    }
  };
  int c = split * cols + wave * CT;  // (width is a multiple of 256, cols of kTurn: a turn lies inside)
  if (c < c1) load(c);
  for (; c < c1; c += kTurn) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    w.put(s_m[wave], lane);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (h == 0 || two) {
#pragma unroll
        for (int k = 0; k < XK; ++k)
          s_x[wave][piece_at<XL>(h * 16 + (k << (6 - XL)) + (lane >> XL), lane & ((1 << XL) - 1))] = x[h][k];
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (c + kTurn < c1) load(c + kTurn);
    multiply(0, 0);
    multiply(0, 1);
    if (two) {
      multiply(1, 0);
      multiply(1, 1);
    }
  }
  // result column i of tile rt is rank 16 rt + i; the wave's part of LDS, read to the end, takes its sums
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  float* own_v = reinterpret_cast<float*>(s_m[wave]);
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int j = 0; j < 4; ++j) own_v[(h * 16 + 4 * q + j) * (RT * 16) + rt * 16 + i] = acc[h][rt][j];
  __syncthreads();
  finish_low<RT, kShrinkWaves>(reinterpret_cast<const float*>(&s_m[0][0]), s_tok, tile, split, R, rl, S.scale ? S.scale[g] : 1.0f, O);
}

// The same where M is stored [width][R]: neighbouring lanes' ranks lie side by side there, and rank RT * i + rt is
// column i of result tile rt, so that a lane loads RT of them at once. A wave takes 32 columns a step, eight consecutive ones a lane
// group. ROW: how fours lie in P's rows.
template <typename W, int RT, int ROW>
struct ShrinkStep {
  typedef typename VecOf<W, RT>::type vr;
  float x[2][8];
  vr w[8];

  // (columns from `end` on are zeros of x, times the weights of the last one)
  __device__ __forceinline__ void load(const float* const (&row)[2], bool two, const W* m, int c, int q, int r0, int R, int end) {
    const int e = c + 8 * q;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const vr*>(m + (int64_t)min(e + j, end - 1) * R + r0);
    load_x(0, row[0], e, end);
    if (two) load_x(1, row[1], e, end);
  }
  __device__ __forceinline__ void load_x(int h, const float* row, int e, int end) {
    float a[4], b[4];
    load_row<ROW, 4>(row, e, end, a);
    load_row<ROW, 4>(row, e + 4, end, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[h][j] = a[j], x[h][4 + j] = b[j];
  }
  __device__ __forceinline__ void multiply(f32x4 (&acc)[2][RT], bool two) const {
    half(acc[0], x[0]);
    if (two) half(acc[1], x[1]);
  }
  __device__ __forceinline__ void half(f32x4 (&acc)[RT], const float (&xh)[8]) const {
    if constexpr (std::is_same<W, bf16_t>::value && RT > 1) {  // (one rank a load: packing costs more than it saves, 20 us and 7)
      const Split3 s(xh);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        bf16x8 b;
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = w[j][rt];
        acc[rt] = mfma3(s, b, acc[rt]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(xh[j], (float)w[j][rt], acc[rt], 0, 0, 0);
    }
  }
};

template <typename W, int RT, int ROW>
__global__ __launch_bounds__(kShrinkWaves * 64) void k_lora_shrink_t(const float* __restrict__ p, LoraSet<W> S,
                                                                     LoraPlan P, int cols, LoraOut O) {
  __shared__ float s_v[kShrinkWaves][kLoraTile * RT * 16];
  __shared__ int s_tok[kLoraTile];
  const int tile = blockIdx.x / O.splits, split = blockIdx.x - tile * O.splits;
  const int g = P.tile_group[tile];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
  const int32_t* slots = P.slots + (int64_t)tile * kLoraTile;
  const int tok[2] = {slots[i], slots[16 + i]}, own = slots[lane & (kLoraTile - 1)];
  if (g < 0) return;
  const int R = S.R, width = S.width, rl = g < S.na ? live_rank(S.ranks, g, R) : 0;
  if (rl == 0) return;  // (nobody reads the tile's values)
  if (threadIdx.x < kLoraTile) s_tok[lane] = own;
  const bool two = readlane_i(own, 16) >= 0;  // the second half has tokens
  const int c1 = min((split + 1) * cols, width);
  const float* row[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) row[h] = p + (int64_t)(tok[h] < 0 ? readlane_i(own, 0) : tok[h]) * width;  // (slot 0 is never empty)
  const W* m = S.mat + (int64_t)g * R * width;
  const int r0 = min(RT * i, R - RT);  // (ranks past the stored ones: dropped below)
  f32x4 acc[2][RT];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) acc[h][rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int kTurn = kShrinkWaves * 32;
  ShrinkStep<W, RT, ROW> s0, s1;
  int c = split * cols + wave * 32;
  if (c < c1) s0.load(row, two, m, c, q, r0, R, c1);
  while (c < c1) {
    if (c + kTurn < c1) s1.load(row, two, m, c + kTurn, q, r0, R, c1);
    s0.multiply(acc, two);
    c += kTurn;
    if (c >= c1) break;
    if (c + kTurn < c1) s0.load(row, two, m, c + kTurn, q, r0, R, c1);
    s1.multiply(acc, two);
    c += kTurn;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int j = 0; j < 4; ++j) s_v[wave][(h * 16 + 4 * q + j) * (RT * 16) + RT * i + rt] = acc[h][rt][j];
  __syncthreads();
  finish_low<RT, kShrinkWaves>(&s_v[0][0], s_tok, tile, split, R, rl, S.scale ? S.scale[g] : 1.0f, O);
}

// The columns of a row that lane i of 16 has in the four result tiles of 64 columns from c0 on: fours in order, or every 16th. Those
// past the row hold anything.
template <bool FOURS, int UT = 4>
__device__ __forceinline__ void load_columns(const float* row, int c0, int i, int width, float (&v)[UT]) {
  if constexpr (FOURS) {
    load_n<UT>(at_element(row, min(c0 + UT * i, width - UT)), v);
  } else {
#pragma unroll
    for (int u = 0; u < UT; ++u) v[u] = *at_element(row, min(c0 + 16 * u + i, width - 1));
  }
}

// out[token][c] = in[token][c] + scale * sum_r low[token][r] * M[c][r] for a tile's tokens, 64 columns a wave
// and turn. Column c0 + 4 i + u is column i of result tile u: a lane ends with four consecutive columns of each of four
// tokens, and 16 lanes read and write 256 consecutive bytes of a row. The low-rank values, summed over the splits in order, stay in
// registers as operands (KQ ranks a lane group and matrix instruction, 8 on the bf16 one, 4 on the fp32 one); `sum` (may be null)
// receives them. FOURS: width is a multiple of four. Else rows start anywhere and column c0 + 16 u + i takes that place: 16 lanes then
// take 64 consecutive bytes, one element each at a time (2043 tokens of rank 64 on 4001 columns, whole call: fours read element by
// element 55 us, this 46).
// TR: M is stored [R][width], and neighbouring lanes' columns lie side by side. Else the 64 columns' ranks are one run of
// memory, which the wave reads in order and turns in LDS as the first product does (the column of lane i in tile u in row
// 16 u + i; a power of two pieces lie turned by the row's number, else rows an odd number of pieces apart).
template <typename W, int RT, bool TR, bool FOURS>
__global__ __launch_bounds__(256) void k_lora_expand(LoraSet<W> S, LoraPlan P, LoraOut O, int slabs, int each, float* sum,
                                                     const float* in, float* out) {
  constexpr bool kBf = std::is_same<W, bf16_t>::value;
  constexpr int KQ = kBf ? 8 : 4, NK = kBf ? (RT + 1) / 2 : RT, NF = kBf ? 3 * NK : NK;
  constexpr int NP = RT * 16 * (int)sizeof(W) / 16;  // 16-byte pieces of a column of M, at most; also loads of a lane
  typedef typename VecOf<W, KQ>::type vk;
  typedef typename VecOf<W, 4>::type v4;
  __shared__ uint4 s_m[TR ? 1 : 4][TR ? 1 : 64 * NP];  // (64 rows of NP, or of at most NP - 1 pieces)
  __shared__ __attribute__((aligned(16))) float s_l[kLoraTile][RT * 16 + 4];
  const int tile = blockIdx.x / slabs, slab = blockIdx.x - tile * slabs;
  const int g = P.tile_group[tile];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
  const int32_t* slots = P.slots + (int64_t)tile * kLoraTile;
  int row[2][4];  // the tokens of the lane's results; an empty slot's are the first slot's, and not stored
  const int first = slots[0];
  const bool two = slots[16] >= 0;  // the second half has tokens
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int j = 0; j < 4; ++j) row[h][j] = slots[h * 16 + 4 * q + j];
  const bool rows = sum && slab == 0;
  if (g < 0 || (g == S.na && in == out && !rows)) return;
  constexpr int turn = 256;
  const int R = S.R, width = S.width;
  int c0 = slab * each * turn + wave * 64;
  const int end = min((slab + 1) * each * turn, width);
  uint4 raw[TR ? 1 : NP];
  v4 wt[TR ? NK : 1][TR ? KQ : 1];
  const W* m = S.mat + (int64_t)(g < S.na ? g : 0) * R * width;
  const int np = R * (int)sizeof(W) / 16;  // pieces of a column, and of its row in LDS
  const bool pow2 = (np & (np - 1)) == 0;
  const int pitch = pow2 ? np : np | 1;
  const uint32_t inv = 65536u / np + 1;  // piece / np = piece * inv >> 16 for the 64 np <= 2048 pieces of a turn
  auto turned = [&](int piece, int r) { return pow2 ? (piece + r) & (np - 1) : piece; };
  auto load_mat = [&](int c) {
    if constexpr (TR) {
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int j = 0; j < KQ; ++j)  // (width is a multiple of 256)
          wt[k][j] = *reinterpret_cast<const v4*>(m + (int64_t)min((k * 4 + q) * KQ + j, R - 1) * width + c + 4 * i);
    } else {
      const uint8_t* run = reinterpret_cast<const uint8_t*>(m + (int64_t)c * R);
      const int last = min(64, width - c) * np - 1;
#pragma unroll
      for (int k = 0; k < NP; ++k) raw[k] = ld16(run + min(k * 64 + lane, last) * 16);
    }
  };
  if (c0 < end) load_mat(c0);
  const int rl = g < S.na ? live_rank(S.ranks, g, R) : 0;
  for (int o = threadIdx.x; o < kLoraTile * (R / 4); o += 256) {
    const int tk = o / (R / 4), r = (o - tk * (R / 4)) * 4;
    float l[4] = {};
    for (int s0 = 0; s0 < (rl > 0 ? O.splits : 0); s0 += kLoraJoin) {
      float v[kLoraJoin][4];
#pragma unroll
      for (int s = 0; s < kLoraJoin; ++s)  // (a split that is not there: the last one's again, and not added)
        load_n<4>(O.low + (((int64_t)min(s0 + s, O.splits - 1) * O.tiles + tile) * kLoraTile + tk) * R + r, v[s]);
#pragma unroll
      for (int s = 0; s < kLoraJoin; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) l[j] += s0 + s < O.splits ? v[s][j] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) s_l[tk][r + j] = l[j];
    if (rows && slots[tk] >= 0) store_n<4>(sum + (int64_t)slots[tk] * R + r, l);
  }
  __syncthreads();
  if (c0 >= end || (g == S.na && in == out)) return;
  uint4 l[2][NF];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const int r = (k * 4 + q) * KQ;
      float x[KQ];
#pragma unroll
      for (int j = 0; j < KQ; ++j) x[j] = r < R ? s_l[h * 16 + i][min(r, R - KQ) + j] : 0.0f;  // (R is a multiple of 8)
      if constexpr (kBf) {
        const Split3 x3(x);
#pragma unroll
        for (int p = 0; p < 3; ++p) l[h][3 * k + p] = __builtin_bit_cast(uint4, x3.part[p]);
      } else {
        l[h][k] = __builtin_bit_cast(uint4, f32x4{x[0], x[1], x[2], x[3]});
      }
    }
  const float sc = S.scale && g < S.na ? S.scale[g] : 1.0f;
  bool has[2][4];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      has[h][j] = row[h][j] >= 0;
      row[h][j] = has[h][j] ? row[h][j] : first;
    }
  for (; c0 < end; c0 += turn) {
    const uint4* ms = s_m[TR ? 0 : wave];
    float y[2][4][4];  // [half][token][column]
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u) y[h][j][u] = 0.0f;
      if (in && (h == 0 || two)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) load_columns<FOURS>(in + (int64_t)row[h][j] * width, c0, i, width, y[h][j]);
      }
    }
    if constexpr (!TR) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int k = 0; k < NP; ++k) {
        const int pc = k * 64 + lane, col = (int)((uint32_t)pc * inv >> 16), r = FOURS ? (col & 3) * 16 + (col >> 2) : col;
        if (pc < 64 * np) s_m[wave][r * pitch + turned(pc - col * np, r)] = raw[k];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (c0 + turn < end) load_mat(c0 + turn);
    }
    f32x4 acc[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int u = 0; u < 4; ++u) acc[h][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](auto masked) {
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        const int r = (k * 4 + q) * KQ, rc = min(r, R - KQ);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          vk b;
          if constexpr (TR) {
#pragma unroll
            for (int j = 0; j < KQ; ++j) b[j] = wt[k][j][u];
          } else {
            constexpr int kPer = 16 / sizeof(W);  // ranks of a piece
            b = *reinterpret_cast<const vk*>(reinterpret_cast<const W*>(ms + (u * 16 + i) * pitch + turned(rc / kPer, u * 16 + i)) +
                                             rc % kPer);
          }
          if constexpr (decltype(masked)::value) {  // zeros past the live ranks
#pragma unroll
            for (int j = 0; j < KQ; ++j) b[j] = r + j < rl ? b[j] : (W)0.0f;
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {  // (an empty second half is multiplied too: its operands are zeros)
            if constexpr (kBf) {
#pragma unroll
              for (int p = 2; p >= 0; --p)
                acc[h][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, l[h][3 * k + p]), b, acc[h][u], 0, 0, 0);
            } else {
              const f32x4 lk = __builtin_bit_cast(f32x4, l[h][k]);
#pragma unroll
              for (int j = 0; j < KQ; ++j)
                acc[h][u] = __builtin_amdgcn_mfma_f32_16x16x4f32(lk[j], (float)b[j], acc[h][u], 0, 0, 0);
            }
          }
        }
      }
    };
    if (rl == NK * 4 * KQ) multiply(std::false_type{});
    else if (rl > 0) multiply(std::true_type{});
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int u = 0; u < 4; ++u) y[h][j][u] = fmaf(sc, acc[h][u][j], y[h][j][u]);
        if (has[h][j]) {
          float* o = out + (int64_t)row[h][j] * width;
          if constexpr (FOURS) {
            store_row<kRowWhole, 4>(o, c0 + 4 * i, width, y[h][j]);
          } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
              if (c0 + 16 * u + i < width) o[c0 + 16 * u + i] = y[h][j][u];
          }
        }
      }
    if constexpr (TR)
      if (c0 + turn < end) load_mat(c0 + turn);
  }
}

// Rows of `sum` alone, as k_lora_expand writes them (those that no reader looks at hold anything).
__global__ __launch_bounds__(256) void k_lora_sum(LoraPlan P, int R, LoraOut O, float* __restrict__ sum) {
  const int tile = blockIdx.x;
  if (P.tile_group[tile] < 0) return;
  for (int o = threadIdx.x; o < kLoraTile * R; o += 256) {
    const int tok = P.slots[tile * kLoraTile + o / R];
    if (tok < 0) break;
    float v = O.low[(int64_t)tile * kLoraTile * R + o];
    for (int s = 1; s < O.splits; ++s) v += O.low[((int64_t)s * O.tiles + tile) * kLoraTile * R + o];
    sum[(int64_t)tok * R + o % R] = v;
  }
}

// G = scale * sum over an adapter's tokens of P[token][c] * low[token][r], 32 columns a workgroup, written [width][R]
// (TR) or [R][width]. The waves take the halves of the adapter's tiles in turns, four tokens a matrix instruction, with the next
// one's loads under way; their sums join in LDS in order. Column c0 + 2 i + u (FOURS; else c0 + 16 u + i) is row i of result tile u,
// rank RT * i + rt its column. An adapter without tokens gets zeros.
//
// Bound by the loads of the workgroups of the adapter with most tokens, which share P's columns among too few compute units: 32 columns
// and 8 waves rather than 64 and 16 spread them over twice as many. Whole backward calls, 64 columns and 32: 2048 tokens of rank 16
// on 8 adapters 56 and 51 us; 3000 of rank 8 on one adapter 98 and 86, on 64 adapters in fp32 100 and 78; 1000 of rank 128 on 4
// adapters 156 and 83 (but 600 of rank 40 on 16 adapters in fp32 79 and 87). The matrix product is fp32 for every type of
// adapter: both factors are fp32 values here.
constexpr int kOuterTiles = 2, kOuterWaves = 8;
template <int RT, bool FOURS>
struct OuterStep {
  static constexpr int UT = kOuterTiles;
  float a[4][UT], b[4][RT];
  bool on[4];
  // (an empty slot's tokens are the first slot's, times zero)
  __device__ __forceinline__ void load(const int32_t* slots, const float* p, const float* low, int q, int i, int c0, int width, int r0,
                                       int R) {
    int tok[4];
    const int first = slots[0];
#pragma unroll
    for (int s = 0; s < 4; ++s) tok[s] = slots[4 * s + q];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      on[s] = tok[s] >= 0;
      tok[s] = on[s] ? tok[s] : first;
      load_columns<FOURS, UT>(p + (int64_t)tok[s] * width, c0, i, width, a[s]);
      load_n<RT>(low + (int64_t)tok[s] * R + min(r0, R - RT), b[s]);
    }
  }
  __device__ __forceinline__ void multiply(f32x4 (&acc)[UT][RT], int r0, int rl) const {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float v = on[s] && r0 + rt < rl ? b[s][rt] : 0.0f;
#pragma unroll
        for (int u = 0; u < UT; ++u) acc[u][rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s][u], v, acc[u][rt], 0, 0, 0);
      }
  }
};

template <int RT, bool TR, bool FOURS>
__global__ __launch_bounds__(kOuterWaves * 64) void k_lora_outer(const float* __restrict__ p, int width,
                                                                       const float* __restrict__ low, int R,
                                                                       const int32_t* __restrict__ ranks,
                                                                       const float* __restrict__ scale, LoraPlan P,
                                                                       float* __restrict__ grad) {
  constexpr int WV = kOuterWaves, UT = kOuterTiles, CW = 16 * UT;
  __shared__ float s_g[RT * 16][CW + 1];
  const int g = blockIdx.y, c0 = blockIdx.x * CW;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
  const int cnt = P.count[g], nt = (cnt + 15) / 16;  // (halves of tiles)
  const int rl = cnt > 0 ? live_rank(ranks, g, R) : 0;
  f32x4 acc[UT][RT];
#pragma unroll
  for (int u = 0; u < UT; ++u)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) acc[u][rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (rl > 0) {
    const int32_t* slots = P.slots + P.first[g] * kLoraTile;
    OuterStep<RT, FOURS> s0, s1;
    int k = wave;
    if constexpr (RT == 8) {  // (one tile in flight: two do not fit beside the sums)
      for (; k < nt; k += WV) {
        s0.load(slots + k * 16, p, low, q, i, c0, width, RT * i, R);
        s0.multiply(acc, RT * i, rl);
      }
    } else {
      if (k < nt) s0.load(slots + k * 16, p, low, q, i, c0, width, RT * i, R);
      while (k < nt) {
        if (k + WV < nt) s1.load(slots + (k + WV) * 16, p, low, q, i, c0, width, RT * i, R);
        s0.multiply(acc, RT * i, rl);
        k += WV;
        if (k >= nt) break;
        if (k + WV < nt) s0.load(slots + (k + WV) * 16, p, low, q, i, c0, width, RT * i, R);
        s1.multiply(acc, RT * i, rl);
        k += WV;
      }
    }
  }
  const int live = min(nt, WV);  // waves that had a tile
  for (int w = 0; w < live; ++w) {
    if (wave == w) {
#pragma unroll
      for (int u = 0; u < UT; ++u)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float& s = s_g[RT * i + rt][FOURS ? UT * (4 * q + j) + u : 16 * u + 4 * q + j];
            s = w == 0 ? acc[u][rt][j] : s + acc[u][rt][j];
          }
    }
    __syncthreads();
  }
  const float sc = scale ? scale[g] : 1.0f;
  grad += (int64_t)g * R * width;
  for (int o = threadIdx.x; o < CW * R; o += WV * 64) {
    const int r = TR ? o % R : o / CW, c = TR ? o / R : o % CW;
    if (c0 + c < width) grad[TR ? (int64_t)(c0 + c) * R + r : (int64_t)r * width + c0 + c] = r < rl ? sc * s_g[r][c] : 0.0f;
  }
}

// ---- few tokens ------------------------------------------------------------------------------

// low[token][r] = A[r] x[token]: a wave takes two ranks of a token, 8 columns a lane and step.
template <typename W>
__global__ __launch_bounds__(256) void k_lora_shrink_row(const float* __restrict__ x, LoraSet<W> S,
                                                         const int32_t* __restrict__ ids, float* __restrict__ low) {
  const int lane = threadIdx.x & 63, r0 = (blockIdx.y * 4 + (threadIdx.x >> 6)) * 2;
  const int64_t tok = blockIdx.x;
  const int R = S.R, k = S.width;
  if (r0 >= R) return;
  const int g = adapter_of(ids[tok], S.na);
  const int rl = g < S.na ? live_rank(S.ranks, g, R) : 0;
  float s0 = 0.0f, s1 = 0.0f;
  if (r0 < rl) {
    const W* m = S.mat + ((int64_t)g * R + r0) * k;  // (R is even: row r0 + 1 is stored)
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
__global__ __launch_bounds__(256) void k_lora_expand_row(const float* __restrict__ low, LoraSet<W> S,
                                                         const int32_t* __restrict__ ids, const float* in, float* out) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  const int64_t tok = blockIdx.y;
  const int R = S.R, n = S.width;
  const int g = adapter_of(ids[tok], S.na);
  if (c >= n || (g == S.na && in == out)) return;
  float v = in ? in[tok * n + c] : 0.0f;
  if (g < S.na) {
    const int rl = live_rank(S.ranks, g, R);
    const float sc = S.scale ? S.scale[g] : 1.0f;
    const W* m = S.mat + ((int64_t)g * n + c) * R;
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

// Both products of a token in one launch: a workgroup computes the token's low-rank values by itself (a wave per rank) and then 1024
// of its columns, whose first ranks were loaded meanwhile. Every workgroup of a token reads the adapter's A again.
template <typename W>
__global__ __launch_bounds__(1024) void k_lora_row(const float* __restrict__ x, LoraSet<W> A, LoraSet<W> B,
                                                   const int32_t* __restrict__ ids, float* __restrict__ v, const float* in,
                                                   float* out) {
  constexpr int kFirst = 2;  // pieces of 8 ranks loaded ahead
  __shared__ float s_v[kLoraMaxRank];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t tok = blockIdx.y;
  const int R = A.R, k = A.width, n = B.width, c = blockIdx.x * 1024 + threadIdx.x;
  const int g = adapter_of(ids[tok], A.na);
  const float* yi = in + tok * n;
  float* yo = out + tok * n;
  if (g == A.na) {
    if (in != out && c < n) yo[c] = in ? yi[c] : 0.0f;
    if (v && blockIdx.x == 0 && threadIdx.x < R) v[tok * R + threadIdx.x] = 0.0f;
    return;
  }
  const int rl = live_rank(A.ranks, g, R);
  const float sc = B.scale ? B.scale[g] : 1.0f;
  const W* b = B.mat + (int64_t)g * n * R;
  typedef typename VecOf<W, 8>::type w8;
  w8 first[kFirst];
  const int cc = min(c, n - 1);
#pragma unroll
  for (int j = 0; j < kFirst; ++j) first[j] = *reinterpret_cast<const w8*>(b + (int64_t)cc * R + min(8 * j, R - 8));
  const float y = in ? yi[cc] : 0.0f;
  const float* row = x + tok * k;
  for (int r = wave; r < R; r += 16) {
    float s = 0.0f;
    if (r < rl) {
      const W* m = A.mat + ((int64_t)g * R + r) * k;
#pragma unroll 4
      for (int j = lane * 8; j < k; j += 512) {  // (k is a multiple of 256)
        float xv[8], w[8];
        load_n<8>(row + j, xv);
        load_n<8>(m + j, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(xv[i], w[i], s);
      }
    }
    s = wave_sum_f32(s);
    if (lane == 0) s_v[r] = s;
  }
  __syncthreads();
  if (v && blockIdx.x == 0 && threadIdx.x < R) v[tok * R + threadIdx.x] = s_v[threadIdx.x];
  if (c >= n) return;
  float s = 0.0f;
  for (int j = 0; 8 * j < rl; ++j) {
    const w8 w = j < kFirst ? (j == 0 ? first[0] : first[1]) : *reinterpret_cast<const w8*>(b + (int64_t)c * R + 8 * j);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (8 * j + i < rl) s = fmaf(s_v[8 * j + i], (float)w[i], s);
  }
  yo[c] = fmaf(sc, s, y);
}

template <typename F>
static void with_rank(int R, F f) {
  if (R <= 16) f(std::integral_constant<int, 1>{});
  else if (R <= 32) f(std::integral_constant<int, 2>{});
  else if (R <= 64) f(std::integral_constant<int, 4>{});
  else f(std::integral_constant<int, 8>{});
}

template <typename F>
static void with_fours(int width, F f) {
  if (width % 4 == 0) f(std::true_type{});
  else f(std::false_type{});
}

// The row kernels read an adapter once for each of its tokens, the tiles once for 32, after a plan (about 14 us at least). Rows up to
// 160 MB of reads: 400 tokens of rank 32 beside 2048 x 4096 (157 MB) 16.7 us against 20.4, 1000 of rank 8 (98 MB) 15.7 against 20.1,
// 400 of rank 16 in fp32 beside 4096 x 4096 (210 MB) 18.8 against 19.9. And up to 1024 tokens, since the rows' workgroups,
// some for each token, come to cost more than the plan: rank 8 beside 64 x 256, 1024 tokens 6.9 us against 13.9, 2048 11.8 and 15.3,
// 4096 23.2 and 18.4; beside 1024 x 1024, 1024 11.2 and 16.6, 2048 20.3 and 20.6; rank 16 beside 2048 x 2048, 512 13.7 and 17.3, 1024
// 20.4 and 20.1.
static bool takes_rows(const tq_adapters* ad, int64_t t) {
  return t <= 1024 && t * ad->rank * ((int64_t)ad->k + ad->n) * (int64_t)type_bytes(ad->type) <= 160 << 20;
}
// Both products in one launch, where its workgroups' repeated reads of A are small: each at most 256 KB and two ranks a wave, 32 MB in
// all. Beside 4096 x 4096 in bfloat16, one launch against two: 1 token of rank 16 4.8 us against 6.5, of rank 24 6.2 against 6.9, of
// rank 32 7.8 against 7.2; 64 tokens of rank 16 (32 MB) 6.5 against 7.2, 128 (64 MB) 11.4 against 10.6.
static bool takes_one_launch(const tq_adapters* ad, int64_t t) {
  const int64_t bytes = (int64_t)ad->rank * ad->k * (int64_t)type_bytes(ad->type);
  return ad->rank <= 24 && bytes <= 256 << 10 && bytes * t * ((ad->n + 1023) / 1024) <= 32 << 20;
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

// A tensor's bytes (none where p is null or n is 0), and whether any of them are another's.
struct Bytes {
  const void* p;
  int64_t n;
};
static bool meets(Bytes a, std::initializer_list<Bytes> others) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p);
  for (const Bytes& b : others) {
    const uintptr_t b0 = reinterpret_cast<uintptr_t>(b.p);
    if (a.p && b.p && a.n && b.n && a0 < b0 + b.n && b0 < a0 + a.n) return true;
  }
  return false;
}

static void launch_plan(const int32_t* ids, int64_t t, int na, const LoraPlan& P, const LoraWs& L, hipStream_t st) {
  hipLaunchKernelGGL(k_lora_plan, dim3(1), dim3(kPlanWaves * 64), 0, st, ids, (int)t, na, P, (int)L.tiles);
}

// The first product over `width` columns, split where there are few tiles.
template <typename W, int RT, bool TR>
static LoraOut launch_shrink(const float* p, const LoraSet<W>& S, const LoraPlan& P, const LoraWs& L, void* ws, hipStream_t st) {
  int splits = lora_splits(L.tiles);
  const int step = kShrinkWaves * 64;
  const int cols = ((S.width + splits - 1) / splits + step - 1) / step * step;
  splits = (S.width + cols - 1) / cols;
  const LoraOut O = {reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + L.low), splits, L.tiles};
  const dim3 grid((unsigned)(L.tiles * splits)), wg(kShrinkWaves * 64);
  if constexpr (TR)
    with_row(S.width, [&](auto row) {
      hipLaunchKernelGGL((k_lora_shrink_t<W, RT, decltype(row)::value>), grid, wg, 0, st, p, S, P, cols, O);
    });
  else
    hipLaunchKernelGGL((k_lora_shrink<W, RT>), grid, wg, 0, st, p, S, P, cols, O);
  return O;
}

template <typename W, int RT, bool TR>
static void launch_expand(const LoraSet<W>& S, const LoraPlan& P, const LoraOut& O, float* sum, const float* in, float* out,
                          hipStream_t st) {
  // a workgroup takes as many turns as leave about four workgroups a compute unit
  const int turns = (S.width + 255) / 256, each = (int)std::max<int64_t>(1, turns * O.tiles / 1024);
  const int slabs = (turns + each - 1) / each;
  with_fours(S.width, [&](auto fours) {
    hipLaunchKernelGGL((k_lora_expand<W, RT, TR, decltype(fours)::value || TR>), dim3((unsigned)(O.tiles * slabs)), dim3(256), 0, st,
                       S, P, O, slabs, each, sum, in, out);
  });
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
  const Bytes bx = {x, t * ad->k * 4}, bi = {ids, t * 4}, by = {y, t * ad->n * 4}, bo = {out, by.n}, bv = {v, t * ad->rank * 4};
  if (meets(bv, {bx, bi, by, bo}) || meets(bo, {bx, bi}) || (out != y && meets(bo, {by})))
    return fail(TQ_ERR_INVALID, "%s: out and v must not lie on x, ids, y (but out may be y) or each other", fn);
  (void)hipGetLastError();
  const hipStream_t hs = (hipStream_t)stream;
  const LoraWs L = lora_ws(ad->n_adapters, ad->rank, t);
  const LoraPlan P = plan_of(ws, L);
  float* low = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + L.low);
  const int R = ad->rank, n = ad->n, na = ad->n_adapters;
  with_type(ad->type, [&](auto wv) {
    using W = decltype(wv);
    const LoraSet<W> A = {static_cast<const W*>(ad->a), ad->ranks, nullptr, na, R, ad->k};
    const LoraSet<W> B = {static_cast<const W*>(ad->b), ad->ranks, ad->scale, na, R, n};
    if (takes_rows(ad, t)) {
      if (takes_one_launch(ad, t)) {
        hipLaunchKernelGGL(k_lora_row<W>, dim3((unsigned)((n + 1023) / 1024), (unsigned)t), dim3(1024), 0, hs, x, A, B, ids, v, y, out);
        return;
      }
      if (v) low = v;
      hipLaunchKernelGGL(k_lora_shrink_row<W>, dim3((unsigned)t, (unsigned)((R + 7) / 8)), dim3(256), 0, hs, x, A, ids, low);
      hipLaunchKernelGGL(k_lora_expand_row<W>, dim3((unsigned)((n + 255) / 256), (unsigned)t), dim3(256), 0, hs, low, B,
                         ids, y, out);
      return;
    }
    launch_plan(ids, t, na, P, L, hs);
    with_rank(R, [&](auto rt) {
      constexpr int RT = decltype(rt)::value;
      const LoraOut O = launch_shrink<W, RT, false>(x, A, P, L, ws, hs);
      launch_expand<W, RT, false>(B, P, O, v, y, out, hs);
    });
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
  const int R = ad->rank, n = ad->n, k = ad->k, na = ad->n_adapters;
  const Bytes bx = {x, t * k * 4}, bi = {ids, t * 4}, bv = {v, t * R * 4}, bdy = {dy, t * n * 4}, bdx = {dx, bx.n}, bo = {out, bx.n},
              ba = {da, (int64_t)na * R * k * 4}, bb = {db, (int64_t)na * n * R * 4};
  if (meets(bo, {bx, bi, bv, bdy}) || (out != dx && meets(bo, {bdx})) || meets(ba, {bx, bi, bv, bdy, bdx, bo, bb}) ||
      meets(bb, {bx, bi, bv, bdy, bdx, bo}))
    return fail(TQ_ERR_INVALID, "%s: out, da and db must not lie on x, ids, v, dy, dx (but out may be dx) or each other", fn);
  (void)hipGetLastError();
  const hipStream_t hs = (hipStream_t)stream;
  const LoraWs L = lora_ws(ad->n_adapters, ad->rank, t);
  const LoraPlan P = plan_of(ws, L);
  float* u = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + L.sum);
  launch_plan(ids, t, na, P, L, hs);
  with_type(ad->type, [&](auto wv) {
    using W = decltype(wv);
    const LoraSet<W> A = {static_cast<const W*>(ad->a), ad->ranks, nullptr, na, R, k};
    const LoraSet<W> B = {static_cast<const W*>(ad->b), ad->ranks, ad->scale, na, R, n};
    with_rank(R, [&](auto rt) {
      constexpr int RT = decltype(rt)::value;
      if (t > 0) {
        const LoraOut O = launch_shrink<W, RT, true>(dy, B, P, L, ws, hs);
        if (out)
          launch_expand<W, RT, true>(A, P, O, u, dx, out, hs);
        else
          hipLaunchKernelGGL(k_lora_sum, dim3((unsigned)L.tiles), dim3(256), 0, hs, P, R, O, u);
      }
      const dim3 wg(kOuterWaves * 64);
      auto grid = [&](int width) { return dim3((unsigned)((width + 16 * kOuterTiles - 1) / (16 * kOuterTiles)), (unsigned)na); };
      with_fours(n, [&](auto fours) {
        hipLaunchKernelGGL((k_lora_outer<RT, true, decltype(fours)::value>), grid(n), wg, 0, hs, dy, n, v, R, ad->ranks, ad->scale, P, db);
      });
      hipLaunchKernelGGL((k_lora_outer<RT, false, true>), grid(k), wg, 0, hs, x, k, u, R,
                         ad->ranks, nullptr, P, da);
    });
  });
  return check_launch(fn);
}
