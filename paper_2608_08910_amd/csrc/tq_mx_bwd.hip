// Gradients through MXFP4 weights: dx = dy W^, and the gated block's dg, du and dx = dg Wg^ + du Wu^.
//
// The weights' scales run along k, the outputs here, so a sum over n meets another scale at every term and the fp4
// matrix instruction cannot take it. The weights are turned into bfloat16 (exact: e2m1 has 2 significant bits) on the
// way into LDS, by the scaled conversion, and read back transposed; products run on the bfloat16 matrix instruction.
// An fp32 (fp16) gradient is the exact sum of three (two) bfloat16 parts: passes of their own, rows below each other, or split off in the tile.
#include <algorithm>

#include "tq_mx.hpp"
#include "tq_mx_plan.hpp"

namespace tq {

// One pass: a [t][lda] (columns n .. lda hold zeros or are not there) against one weight matrix.
struct MxSeg {
  const void* a;
  const uint8_t *codes, *scales;
  int64_t lda;
};
struct MxBwdArgs {
  MxSeg seg[6];
  int nseg, n, t, kb, type;
  int nx, ny;         // tiles
  int whole, splits;  // tiles that one workgroup does alone, in the order of place_of; workgroups of each of the others
  void* out;          // dx
  float* part;        // partial sums of the others: whole == 0: [splits][t][k]; else [splits][others][BN][BC]
};

// Tile number `tile` of nx by ny: four rows of tiles at a time.
__device__ __forceinline__ void place_of(int tile, int nx, int ny, int& x, int& y) {
  const int y0 = tile / (4 * nx) * 4, height = min(4, ny - y0), in = tile - y0 * nx;
  x = in / height;
  y = y0 + in % height;
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

// Four rows' elements of this lane's column: lane i of 16 passes the address of row i / 4, columns 4 (i % 4) ...
__device__ __forceinline__ s16x4 read_columns(const void* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(const_cast<void*>(p)));
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

// What a unit's number in 256 bytes of row r is exchanged by.
__device__ __forceinline__ int unit_place(int r) { return (r & 1) << 2 | (r & 2) << 2 | (r & 2) | ((r >> 2) & 1); }

// Tiles of BC columns of k by BN tokens, kStep rows of the weights a step. Codes, scales and the tokens' rows come through S LDS
// stages that the loads fill without passing through registers; while the matrix unit works on a step, the next one's codes
// become bfloat16 in LDS, once for the workgroup (each wave for itself would take as long as the products).
//   a stage's tokens: 128 bytes a row, 16-byte pieces exchanged by the row's number (16 rows' pieces in different banks);
//   weights: BC bfloat16 a row, 16-byte units exchanged by the row's number, so that the reads of 64 bytes of four rows and the
//   writes of one unit of eight rows meet all banks.
// The operands of a quarter step are read while the matrix unit works on the quarter before, across the barrier too.
// Bound by LDS at size: a 256 x 256 step reads and writes 280 KB of it, 2200 clocks at 128 bytes each, beside 2048 of products.
// Measured, 2 x (2048 x 7168) and 8192 rows in bfloat16: 430 us with the joining, 1.1 PFLOP/s; 4096 x 2048, 2048 rows: 49 us, 0.70 PFLOP/s. Without
// its loads a 256 x 256 tile takes 0.78 of its time, without conversions 0.88, without products 0.78. A 128 x 128 step (120 KB of LDS, 512 clocks of products,
// 0.75 us) waits for its loads instead, with eight waves a compute unit: at 55 us for 4096 x 2048, 2048 rows, it took 35 without loads, 46 where all
// missed the buffer, 45 without conversions, 53 without reads of operands, 54 without products.
// Up to 128 columns a wave takes 32 of them and all tokens (transposed reads take 8 bytes a lane, the tokens' 16: 128 x 64 82 us at
// 4096 x 2048, 2048 rows, with 64 x 32 a wave 85; 128 x 128 49.3, 64 x 64 a wave 49.9), at 128 x 128 two waves half of every step's rows
// each, whose sums join at the end (WK = 2; one wave each 58).
// T fp32 or fp16: dy comes in its own type, and its parts are split off in registers (5.5 vector instructions a value and wave) behind
// the last products of a quarter, so that a wave takes as many columns as it can; one reading of the weights serves all parts and
// nothing is written ahead. A step of 256 x 128 then takes 2.4 us in fp32 (three passes of parts 3.2), 1.75 in fp16 (2.1).
template <typename T, int BC, int BN, int WM, int WN, int WK, int S, int SPREAD>
__global__ __launch_bounds__(WM * WN * WK * 64) void k_mx_bwd(const MxBwdArgs a) {
  constexpr int EB = sizeof(T), NP = std::is_same<T, bf16_t>::value ? 1 : EB == 2 ? 2 : 3;  // parts of a value
  constexpr int TB = kStep * EB, UR = TB / 16, RI = 1024 / TB;  // a token's bytes in a stage, its units, rows a load instruction
  typedef typename VecOf<T, 8>::type T8;
  constexpr int NW = WM * WN * WK, QK = 4 / WK, NTHR = NW * 64, MT = BC / WM / 32, NT = BN / WN / 32;
  constexpr int RB = BC / 2, RS = BC / 32;             // bytes of a row's codes and scales in a tile
  // Load instructions of 1024 bytes: PA of each wave for the tokens, one for the codes of CW waves; SN of 256 bytes, from wave SF on, for
  // the scales (each wave its rows' codes and scales were half again as many: 55.6 us against 54.4 at 4096 x 2048, 2048 rows).
  constexpr int PA = BN / RI / NW, CW = kStep * RB / 1024, SN = kStep * RS / 256, SF = CW == NW ? 0 : CW, PL = PA + 2;
  constexpr int EACH = PA + (CW == NW);  // of each wave; of waves 0 .. SF + SN - 1 one more
  constexpr int HP = kStep * RB / 8 / NTHR;            // 8-byte pieces of codes that a thread turns into bfloat16
  static_assert(PA >= 1 && BN % (RI * NW) == 0 && HP >= 1 && CW <= NW && SF + SN <= NW && (S - 2) * PL < 64, "tile");
  constexpr int LA = BN * TB, LR = kStep * RB, LS = kStep * RS, LW = kStep * BC * 2;
  __shared__ __attribute__((aligned(16))) uint8_t lds[S * (LA + LR + LS) + 2 * LW];
  uint8_t *const sa = lds, *const sw = lds + S * LA, *const sr = sw + 2 * LW, *const ss = sr + S * LR;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wk = WK == 1 ? 0 : wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN, l32 = lane & 31, half = lane >> 5;
  const int kb = a.kb, n = a.n;
  // (whole == 0: blockIdx.x the tile, blockIdx.z the share; else one after another, the shares of the others behind the whole ones.
  // Both by one division more each cost 0.6 us of 16.)
  const int all_tiles = a.nx * a.ny, others = all_tiles - a.whole;
  int tile, z = blockIdx.z, splits = a.splits;
  if (a.whole == 0) {
    tile = die_order(blockIdx.x, all_tiles);
  } else if ((int)blockIdx.x < a.whole) {
    tile = die_order(blockIdx.x, a.whole);
    splits = 1;
  } else {
    const int o = die_order(blockIdx.x - a.whole, others * splits);
    z = __builtin_amdgcn_readfirstlane(o / others);
    tile = a.whole + o - z * others;
  }
  int tx, ty;
  place_of(tile, a.nx, a.ny, tx, ty);
  const int col0 = __builtin_amdgcn_readfirstlane(tx * BC), tok0 = __builtin_amdgcn_readfirstlane(ty * BN), toks = min(BN, a.t - tok0);
  const int per = (n + kStep - 1) / kStep, all = per * a.nseg;
  // (at most 6 * 2^14 steps and 32 splits)
  const int s0 = __builtin_amdgcn_readfirstlane(all * z / splits);
  const int s1 = __builtin_amdgcn_readfirstlane(all * (z + 1) / splits);

  // Where the next step's tokens and weights are loaded from: its pass and first row, and what follows from them. They go on by
  // constants; a pass's own values are read from the arguments where it begins (each step that wait cost as much as its loads).
  const int pass0 = __builtin_amdgcn_readfirstlane(s0 / per), row00 = (s0 - pass0 * per) * kStep;
  int ts = s0, tg = pass0, tn = row00, ws = s0, wg = pass0, wn0 = row00;
  const uint8_t *tp, *cp, *ep;
  uint32_t lda, tbytes;
  const auto pass_tokens = [&] {
    const MxSeg& sg = a.seg[tg];
    lda = (uint32_t)sg.lda;
    tp = (const uint8_t*)sg.a + ((int64_t)tok0 * sg.lda + tn) * EB;
    tbytes = ((uint32_t)toks * lda - (uint32_t)tn) * EB;
  };
  const auto pass_weights = [&] {
    const MxSeg& sg = a.seg[wg];
    cp = sg.codes + (int64_t)wn0 * kb * 128 + col0 / 2;
    ep = sg.scales + (int64_t)wn0 * kb * 8 + col0 / 32;
  };
  pass_tokens();
  pass_weights();
  const auto token_place = [](int r) { return UR == 8 ? (r >> 1) & 7 : r & 15; };
  const auto code_place = [](int r) { return RB == 64 ? (r >> 2) & 3 : (r >> 1) & 7; };
  // Loads of step s: the tokens' rows, and the codes and scales (past the last step: nothing).
  i32x4 rt, rc, re;  // a step's resources: tokens, codes, scales (past the last step nothing is read)
  uint32_t cols, dt, dc, de;
  const auto tokens_of = [&] {
    rt = rsrc_words(tp, ts < s1 ? tbytes : 0u);
    cols = lda - (uint32_t)tn;
    dt = lds_address(sa) + (uint32_t)(ts - s0) % S * LA;
    if (++ts >= s1) return;
    tn += kStep;
    tp += TB;
    tbytes -= TB;
    if (tn >= n) {
      tn = 0;
      ++tg;
      pass_tokens();
    }
  };
  const auto weights_of = [&] {
    const int rows = ws < s1 ? min(kStep, n - wn0) : 0;
    const uint32_t slot = (uint32_t)(ws - s0) % S;
    rc = rsrc_words(cp, (uint32_t)max(0, rows * kb * 128 - col0 / 2));
    re = rsrc_words(ep, (uint32_t)max(0, rows * kb * 8 - col0 / 32));
    dc = lds_address(sr) + slot * LR;
    de = lds_address(ss) + slot * LS;
    if (++ws >= s1) return;
    wn0 += kStep;
    cp += kStep * 128 * kb;
    ep += kStep * 8 * kb;
    if (wn0 >= n) {
      wn0 = 0;
      ++wg;
      pass_weights();
    }
  };
  // Load instruction i of those that tokens_of and weights_of have set up: PA of tokens, codes, scales.
  const auto load = [&](int i) {
    if (i < PA) {
      const int r0 = (wave + i * NW) * RI, r = r0 + lane / UR, p = (lane % UR) ^ token_place(r);
      // (past a row's end lies the next token's, whose infinities must not meet the weights' zeros)
      load_lds<16>(rt, dt + r0 * TB, (uint32_t)p * (16u / EB) < cols ? (uint32_t)r * lda * EB + (uint32_t)p * 16u : 0xf0000000u);
    } else if (i == PA) {
      const int q = wave * 64 + lane, r = q / (RB / 16), p = (q % (RB / 16)) ^ code_place(r);
      if (wave < CW) load_lds<16>(rc, dc + wave * 1024, (uint32_t)(r * kb) * 128u + (uint32_t)p * 16u);
    } else {
      const int q = (wave - SF) * 64 + lane, r = q / (RS / 4), p = q % (RS / 4);
      if (wave >= SF && wave < SF + SN) load_lds<4>(re, de + (wave - SF) * 256, (uint32_t)(r * kb) * 8u + (uint32_t)p * 4u);
    }
  };
  // Step s's codes to bfloat16: 8 bytes a thread and piece. A byte's two elements stay together: place 2 i of a block of 32
  // holds its column i, place 2 i + 1 its column 16 + i.
  uint2 raw[HP];
  uint32_t ex[HP];
  const auto read_codes = [&](int s) {
    const int slot = (uint32_t)(s - s0) % S;
#pragma unroll
    for (int i = 0; i < HP; ++i) {
      const int q = tid + i * NTHR, r = q % kStep, p = q / kStep;
      raw[i] = *reinterpret_cast<const uint2*>(sr + slot * LR + r * RB + (((p / 2) ^ code_place(r)) << 4) + ((p & 1) << 3));
      ex[i] = ss[slot * LS + r * RS + p / 2];
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  const auto convert = [&](int s, int i) {
    {
      const int q = tid + i * NTHR, r = q % kStep, p = q / kStep;
      const float e = e8m0_f32(ex[i]);
      const uint32_t w[2] = {raw[i].x, raw[i].y};
      uint32_t v[8];
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        v[4 * d] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], e, 0));
        v[4 * d + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], e, 1));
        v[4 * d + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], e, 2));
        v[4 * d + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], e, 3));
      }
      uint8_t* row = sw + ((s - s0) & 1) * LW + r * BC * 2;
      *reinterpret_cast<uint4*>(row + (((2 * p) ^ unit_place(r)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<uint4*>(row + (((2 * p + 1) ^ unit_place(r)) << 4)) = make_uint4(v[4], v[5], v[6], v[7]);
    }
  };

  f32x16 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[m][c][i] = 0.0f;

  // Quarter k of a step: 16 rows of the weights. Lanes 16 g .. 16 g + 15 read rows 8 (g / 2) .. + 7 of columns 16 (g % 2) .. + 15.
  const int i16 = lane & 15, g16 = lane >> 4;
  const int rw = 8 * (g16 >> 1) + i16 / 4, uw = 2 * (g16 & 1) + ((i16 >> 1) & 1);  // and 4 rows on; the unit in a block of 32 columns
  struct Tokens {
    bf16x8 part[NT][NP];
  };
  bf16x8 w0[MT], w1[MT];
  Tokens x0, x1;
#pragma unroll
  for (int m = 0; m < MT; ++m) w1[m] = bf16x8{};
#pragma unroll
  for (int c = 0; c < NT; ++c)
#pragma unroll
    for (int p = 0; p < NP; ++p) x1.part[c][p] = bf16x8{};
  // Reads of quarter k's operands, one instruction at a time: of the tokens, then two for each tile of columns.
  constexpr int XR = EB / 2, RD = NT * XR + 2 * MT, QP = MT * NT * NP;
  s16x4 part;
  T8 raw_x[NT];
  const auto read = [&](int s, int k, int i, bf16x8 (&w)[MT]) {
    if (i < NT * XR) {
      const int c = i / XR, u = ((wk * QK + k) * 2 + half) * XR + i % XR;
      const uint4 v = *reinterpret_cast<const uint4*>(sa + (uint32_t)(s - s0) % S * LA + (wn * NT * 32 + l32) * TB + ((u ^ token_place(l32)) << 4) + c * 32 * TB);
      if constexpr (EB == 2) {
        raw_x[c] = __builtin_bit_cast(T8, v);
      } else {
        const f32x4 f = __builtin_bit_cast(f32x4, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) raw_x[c][i % XR * 4 + j] = f[j];
      }
    } else {
      const int m = (i - NT * XR) / 2, r = (i - NT * XR) % 2, u = (wm * MT + m) * 4 + uw;
      const uint8_t* at = sw + ((s - s0) & 1) * LW + (16 * (wk * QK + k) + rw + 4 * r) * BC * 2 + 8 * (i16 & 1) + ((u ^ unit_place(rw + 4 * r)) << 4);
      if (r == 0) part = read_columns(at);
      else w[m] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(part, read_columns(at), 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };
  // A quarter's products, and what goes between them, so that neither holds the other: the next quarter's reads after the
  // first products, then `also` after each (loads issued together would hold the wave until the memory unit has taken them); and
  // after the last ones the parts of the values read, a few each.
  const auto multiply = [&](const bf16x8 (&w)[MT], const Tokens& x, int s, int k, bf16x8 (&nw)[MT], Tokens& nx, auto also) {
    constexpr int R = (RD + QP - 1) / QP > 2 ? (RD + QP - 1) / QP : 2;
    constexpr int after = (NT * XR + R - 1) / R, pairs = NP == 1 ? 1 : (4 * NT + QP - after - 1) / (QP - after), first = QP - (4 * NT + pairs - 1) / pairs;
    static_assert(NP == 1 || (QP > after && first >= after), "parts behind the reads");
#pragma unroll
    for (int i = 0; i < QP; ++i) {
      const int p = NP - 1 - i / (MT * NT), m = i / NT % MT, c = i % NT;
      acc[m][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[m], x.part[c][p], acc[m][c], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (k >= 0) {
#pragma unroll
        for (int j = 0; j < R; ++j)
          if (i * R + j < RD) read(s, k, i * R + j, nw);
        if constexpr (NP > 1) {
#pragma unroll
          for (int h = 0; h < 2 * pairs; ++h) {
            const int e = (i - first) * 2 * pairs + h, c8 = e / 8, j = e % 8;
            if (i >= first && c8 < NT) {
              bf16_t v[3];
              bf16_parts((float)raw_x[c8][j], v);
#pragma unroll
              for (int o = 0; o < NP; ++o) nx.part[c8][o][j] = v[o];
            }
          }
        } else if (i == QP - 1) {
#pragma unroll
          for (int j = 0; j < NT; ++j) nx.part[j][0] = __builtin_bit_cast(bf16x8, raw_x[j]);
        }
      }
      also(i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const auto step_end = [&] {
    asm volatile("" ::: "memory");  // (the barrier alone does not keep the compiler from moving reads across)
    if (S > 2 && wave < SF + SN) __builtin_amdgcn_s_waitcnt(wait_loads((S - 2) * (EACH + 1)));
    else __builtin_amdgcn_s_waitcnt(wait_loads((S - 2) * EACH));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // (a step's codes are needed one step before its tokens' rows, and are loaded so much earlier)
  weights_of();
#pragma unroll
  for (int i = PA; i < PL; ++i) load(i);
#pragma unroll
  for (int j = 0; j < S - 1; ++j) {
    tokens_of();
    weights_of();
#pragma unroll
    for (int i = 0; i < PL; ++i) load(i);
  }
  step_end();
  read_codes(s0);
#pragma unroll
  for (int i = 0; i < HP; ++i) convert(s0, i);
  __syncthreads();
  // After product i of quarter q (0 .. 3 of a step's products, the first the step before's last): every SPREAD-th a load, and with two
  // stages, where a load has one step to arrive in, behind the last what the next step's are to be (80 scalar instructions: ahead of the
  // step's first load they cost 2 x (2048 x 7168) with 8192 rows 500 us against 478).
  constexpr bool AHEAD = S == 2;
  const auto load_after = [&](int q, int i) {
    constexpr int last = (PL - 1) * SPREAD;
    static_assert(last + (AHEAD ? 2 : 0) < QK * QP, "loads among a step's products");
    const int at = q * QP + i;
    if (at % SPREAD == 0 && at / SPREAD < PL) load(at / SPREAD);
    if (AHEAD && at == last + 1) tokens_of();
    if (AHEAD && at == last + 2) weights_of();
  };
  if (AHEAD) {
    tokens_of();
    weights_of();
  }
  for (int s = s0; s < s1; ++s) {
    if (!AHEAD) {
      tokens_of();
      weights_of();
    }
    read_codes(s + 1);
    // (the codes that were read at the step's beginning are there in its second half)
#pragma unroll
    for (int q = 0; q < QK; q += 2) {
      multiply(w1, x1, s, q, w0, x0, [&](int i) {
        load_after(q, i);
        if (q >= QK / 2 && (q - QK / 2) * QP + i < HP) convert(s + 1, (q - QK / 2) * QP + i);
      });
      multiply(w0, x0, s, q + 1, w1, x1, [&](int i) {
        load_after(q + 1, i);
        if (q + 1 >= QK / 2 && (q + 1 - QK / 2) * QP + i < HP) convert(s + 1, (q + 1 - QK / 2) * QP + i);
      });
    }
    step_end();
  }
  static_assert(HP <= QK / 2 * QP, "conversions among a half step's products");
  multiply(w1, x1, 0, -1, w0, x0, [](int) {});
  __builtin_amdgcn_s_waitcnt(wait_loads(0));  // nothing may arrive in the LDS that the results take
  __syncthreads();

  // Out: TP tokens' sums to LDS (16-byte units exchanged by the token's number), then four columns a thread.
  constexpr int TF = (int)sizeof(lds) / (BC * 4) / 32 * 32, TP = TF < BN ? TF : BN, GR = BC / 4;
  static_assert(TP >= 32, "out");
  const int64_t k = (int64_t)kb * 256;
  float* const sums = a.whole ? a.part + ((int64_t)z * others + tile - a.whole) * (BN * BC) : a.part + ((int64_t)z * a.t + tok0) * k + col0;
  const int64_t pitch = a.whole ? BC : k;
#pragma unroll
  for (int t0 = 0; t0 < BN; t0 += TP) {
    if (t0) __syncthreads();
#pragma unroll
    for (int p = 0; p < WK; ++p) {
      if (p) __syncthreads();
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        const int tk = (wn * NT + c) * 32 - t0;
        if (tk >= 0 && tk < TP && (WK == 1 || wk == p)) {
          uint8_t* row = lds + (tk + l32) * (BC * 4);
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              // places 8 q + 4 half .. + 3: columns i, 16 + i, i + 1, 17 + i
              const int u = (wm * MT + m) * 8 + q, at = half * 8;
              const f32x16& v = acc[m][c];
              f32x2& lo = *reinterpret_cast<f32x2*>(row + ((u ^ l32) << 4) + at);
              f32x2& hi = *reinterpret_cast<f32x2*>(row + (((u + 4) ^ l32) << 4) + at);
              const f32x2 l = {v[4 * q], v[4 * q + 2]}, h = {v[4 * q + 1], v[4 * q + 3]};
              lo = p ? lo + l : l;
              hi = p ? hi + h : h;
            }
        }
      }
    }
    __syncthreads();
#pragma unroll 4
    for (int e = tid; e < TP * GR; e += NTHR) {
      const int tk = e / GR, j = e % GR;
      if (t0 + tk >= toks) continue;
      const f32x4 r = *reinterpret_cast<const f32x4*>(lds + tk * (BC * 4) + ((j ^ (tk & 31)) << 4));
      const float v[4] = {r[0], r[1], r[2], r[3]};
      if (a.part && tile >= a.whole) store_n<4>(sums + (t0 + tk) * pitch + 4 * j, v);
      else store4(a.type, a.out, (tok0 + t0 + tk) * k + col0 + 4 * j, v, 4);
    }
  }
}

// `sums` partial sums, in order; four elements a thread.
__global__ __launch_bounds__(256) void k_mx_bwd_join(const float* __restrict__ part, int sums, int64_t quads, int type, void* out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= quads) return;
  f32x4 s = *reinterpret_cast<const f32x4*>(part + 4 * i);
#pragma unroll 8
  for (int p = 1; p < sums; ++p) s += *reinterpret_cast<const f32x4*>(part + 4 * (p * quads + i));
  const float v[4] = {s[0], s[1], s[2], s[3]};
  store4(type, out, 4 * i, v, 4);
}

// The same for tiles of bc columns by bn tokens from number `whole` on, whose partial sums stand by tiles. Bound by memory (128 tiles
// of 256 x 256 in two shares, 84 MB: 13 us).
__global__ __launch_bounds__(256) void k_mx_bwd_join_tiles(const float* __restrict__ part, int sums, int whole, int nx, int ny, int bc, int bn, int t, int type,
                                                           void* out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, quads = (int64_t)(nx * ny - whole) * (bc * bn / 4);
  if (i >= quads) return;
  const int in = (int)(i % (bc * bn / 4)) * 4;
  int x, y;
  place_of(whole + (int)(i / (bc * bn / 4)), nx, ny, x, y);
  const int64_t tok = (int64_t)y * bn + in / bc;
  if (tok >= t) return;
  f32x4 s = *reinterpret_cast<const f32x4*>(part + 4 * i);
  for (int p = 1; p < sums; ++p) s += *reinterpret_cast<const f32x4*>(part + 4 * (p * quads + i));
  const float v[4] = {s[0], s[1], s[2], s[3]};
  store4(type, out, tok * ((int64_t)nx * bc) + x * bc + in % bc, v, 4);
}

// Eight values' NP parts to planes of `plane` elements, the last parts first.
template <int NP>
__device__ __forceinline__ void put_parts(const float (&v)[8], bf16_t* planes, int64_t plane, int64_t at) {
  typedef bf16_t bf16x8v __attribute__((ext_vector_type(8)));
  bf16x8v w[NP];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    bf16_t p[3];
    bf16_parts(v[j], p);
#pragma unroll
    for (int i = 0; i < NP; ++i) w[i][j] = p[i];
  }
#pragma unroll
  for (int i = 0; i < NP; ++i) *reinterpret_cast<bf16x8v*>(planes + (NP - 1 - i) * plane + at) = w[i];
}

// The first m of eight consecutive values, zeros after them.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int m, float (&v)[8]) {
  if (m >= 8) {
    load_n<8>(p, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < m ? (float)p[j] : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void save8(T* p, int m, const float (&v)[8]) {
  if (m >= 8) {
    store_n<8>(p, v);
  } else {
#pragma unroll
    for (int j = 0; j < 7; ++j)
      if (j < m) p[j] = (T)v[j];
  }
}

// Few rows: a workgroup takes 32 columns of k by 32 rows of dy, and its waves share the rows of the weights, 64 a step, with
// nothing to wait for between them until the sums. A lane loads 16 bytes of codes of one row of the weights, writes its 32 bfloat16 to
// the wave's own LDS and reads them back by columns; dy comes straight from memory in its type and is split into its
// bfloat16 parts in registers, so that there is one launch. Bound by the first cache, which takes 128 bytes for each 16 of codes and
// for each scale (a step 0.24 us, of one row of dy 0.17; 0.15 with both packed), and below that by the launch and one wait for memory.
// Measured: 512 x 1024, 8 rows: bfloat16 3.2 us, fp32 3.8 us; 900 x 2048, 60 rows: 6.0 and 7.5 us. Not kept: 16 waves (equal), 64 rows a
// wave (registers), codes four steps ahead (equal), loads past the first cache (1.5 times slower: 8 workgroups share a line), waves
// beside each other in a line and the rows split further (2048 x 4096, 33 rows, fp32 16.4; of two a line 1536 columns, 300 rows 16.7, 19.7 so).
struct MxFewArgs {
  const void* dy[2];  // of type T, [t][n]
  const uint8_t *codes[2], *scales[2];
  int mats, n, t, kb, type, splits;
  void* out;
  float* part;
};
template <typename T, int NP>
__global__ __launch_bounds__(kFewWaves * 64) void k_mx_bwd_few(const MxFewArgs a) {
  typedef typename VecOf<T, 8>::type T8;
  constexpr int NW = kFewWaves;
  __shared__ __attribute__((aligned(16))) uint8_t lds[NW * 4096];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
  const int nx = gridDim.x, tile = die_order(blockIdx.y * nx + blockIdx.x, nx * gridDim.y);
  const int col0 = tile % nx * 32, tok0 = tile / nx * 32, n = a.n;
  const int per = (n + 63) / 64, all = per * a.mats;
  const int s0 = all * (int)blockIdx.z / a.splits, s1 = all * (int)(blockIdx.z + 1) / a.splits;
  uint8_t* const own = lds + wave * 4096;
  const int i16 = lane & 15, g16 = lane >> 4, rw = 8 * (g16 >> 1) + i16 / 4, uw = 2 * (g16 & 1) + ((i16 >> 1) & 1);

  // Steps s of 64 rows of the weights: 32 codes and their scale of the lane's row, zeros past the last.
  struct Codes {
    uint4 c;
    uint32_t e;
  };
  const auto load_codes = [&](int s, Codes& w) {
    const int m = s >= per, row = (s - m * per) * 64 + lane, r = min(row, n - 1);
    w.c = *reinterpret_cast<const uint4*>((m ? a.codes[1] : a.codes[0]) + (int64_t)r * a.kb * 128 + col0 / 2);
    w.e = (m ? a.scales[1] : a.scales[0])[(int64_t)r * a.kb * 8 + col0 / 32];
  };
  // The same rows of the gradient, 8 a lane and quarter. (Rows of dy past the last are a copy of it; nothing of them is stored.)
  const auto load_rows = [&](int s, T8 (&x)[4]) {
    const int m = s >= per, r0 = (s - m * per) * 64;
    const T* row = (const T*)(m ? a.dy[1] : a.dy[0]) + (int64_t)min(tok0 + l32, a.t - 1) * n + r0 + 8 * half;
    if (r0 + 64 <= n) {
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = *reinterpret_cast<const T8*>(row + 16 * q);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) x[q][j] = r0 + 8 * half + 16 * q + j < n ? row[16 * q + j] : (T)0.0f;
    }
  };

  f32x16 acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
  const auto work = [&](int s, const Codes& cw, const T8 (&x)[4]) {
    const bool there = (s - (s >= per ? per : 0)) * 64 + lane < n;
    const float e = e8m0_f32(there ? cw.e : 0u);
    const uint32_t w[4] = {there ? cw.c.x : 0u, there ? cw.c.y : 0u, there ? cw.c.z : 0u, there ? cw.c.w : 0u};
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      uint4 v;
      v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], e, 0));
      v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], e, 1));
      v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], e, 2));
      v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[d], e, 3));
      *reinterpret_cast<uint4*>(own + lane * 64 + ((d ^ ((lane >> 1) & 3)) << 4)) = v;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");  // (a wave's accesses to LDS keep their order)
    bf16x8 wq[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      s16x4 p[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int rr = 16 * q + rw + 4 * r;
        p[r] = read_columns(own + rr * 64 + 8 * (i16 & 1) + ((uw ^ ((rr >> 1) & 3)) << 4));
      }
      wq[q] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(p[0], p[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      bf16x8 b[NP];
      if constexpr (NP == 1) {
        b[0] = __builtin_bit_cast(bf16x8, x[q]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          bf16_t p[3];
          bf16_parts((float)x[q][j], p);
#pragma unroll
          for (int i = 0; i < NP; ++i) b[i][j] = p[i];
        }
      }
#pragma unroll
      for (int i = NP - 1; i >= 0; --i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wq[q], b[i], acc, 0, 0, 0);
    }
  };

  // (two steps' codes are loaded two steps ahead, the rows of dy one)
  Codes now[2], next[2];
  T8 x[2][4];
  const int first = s0 + wave;
#pragma unroll
  for (int d = 0; d < 2; ++d)
    if (first + d * NW < s1) load_codes(first + d * NW, now[d]);
  if (first < s1) load_rows(first, x[0]);
  for (int s = first; s < s1; s += 2 * NW) {
#pragma unroll
    for (int d = 0; d < 2; ++d)
      if (s + (2 + d) * NW < s1) load_codes(s + (2 + d) * NW, next[d]);
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const int at = s + d * NW;
      if (at + NW < s1) load_rows(at + NW, x[1 - d]);
      if (at < s1) work(at, now[d], x[d]);
    }
#pragma unroll
    for (int d = 0; d < 2; ++d) now[d] = next[d];
  }

  // The waves' sums to LDS, 16-byte units of a row of 32 columns exchanged by the row's number; then added in order.
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    // places 8 q + 4 half .. + 3: columns i, 16 + i, i + 1, 17 + i
    uint8_t* row = own + l32 * 128 + half * 8;
    *reinterpret_cast<f32x2*>(row + ((q ^ (l32 & 7)) << 4)) = f32x2{acc[4 * q], acc[4 * q + 2]};
    *reinterpret_cast<f32x2*>(row + (((q + 4) ^ (l32 & 7)) << 4)) = f32x2{acc[4 * q + 1], acc[4 * q + 3]};
  }
  __syncthreads();
  const int64_t k = (int64_t)a.kb * 256, tok = tok0 + tid / 8;
  if (tid >= 256 || tok >= a.t) return;
  const uint8_t* at = lds + tid / 8 * 128 + ((tid ^ (tid >> 3)) & 7) * 16;
  f32x4 r = *reinterpret_cast<const f32x4*>(at);
#pragma unroll
  for (int p = 1; p < NW; ++p) r += *reinterpret_cast<const f32x4*>(at + p * 4096);
  const float v[4] = {r[0], r[1], r[2], r[3]};
  const int64_t c = col0 + 4 * (tid & 7);
  if (a.part) store4(TQ_F32, a.part, ((int64_t)blockIdx.z * a.t + tok) * k + c, v, 4);
  else store4(a.type, a.out, tok * k + c, v, 4);
}

// Rows of n values to NP planes [rows][8 * groups] of bfloat16 parts, zeros past n. Eight values a thread.
template <typename T, int NP>
__global__ __launch_bounds__(256) void k_mx_parts(const T* __restrict__ x, int64_t rows, int n, int groups, bf16_t* __restrict__ planes) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * groups; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / groups;
    const int c = (int)(i - r * groups) * 8;
    float v[8];
    load8(x + r * n + c, n - c, v);
    put_parts<NP>(v, planes, rows * groups * 8, i * 8);
  }
}

// Four values a thread (of rows of whole 16-byte pieces).
template <typename T>
__global__ __launch_bounds__(256) void k_mx_copy(const T* __restrict__ x, int64_t fours, T* __restrict__ out) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < fours; i += (int64_t)gridDim.x * 256) {
    float v[4];
    load_n<4>(x + 4 * i, v);
    store_n<4>(out + 4 * i, v);
  }
}

// dg = dh u act'(g), du = dh act(g), and where PLANES their parts ([2][NP][rows][8 * groups]; else rows is 1). Eight values a
// thread: bound by memory (8192 x 2048 in bfloat16: 168 MB, 31 us).
template <typename T, int NP, bool PLANES>
__global__ __launch_bounds__(256) void k_gated_bwd(const T* g, const T* u, const T* dh, int act, int64_t rows, int64_t n, int64_t groups, T* dg,
                                                   T* du, bf16_t* __restrict__ planes) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * groups; i += (int64_t)gridDim.x * 256) {
    const int64_t r = PLANES ? i / groups : 0, c = (i - r * groups) * 8, j0 = r * n + c;
    const int m = (int)min(n - c, (int64_t)8);
    float vg[8], vu[8], vd[8];
    load8(g + j0, m, vg);
    load8(u + j0, m, vu);
    load8(dh + j0, m, vd);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float a, da;
      act_both(act, vg[j], a, da);
      // (rounded to the type here: the products below take the same values)
      vg[j] = (float)(T)(vd[j] * vu[j] * da);
      vu[j] = (float)(T)(vd[j] * a);
    }
    save8(dg + j0, m, vg);
    save8(du + j0, m, vu);
    if constexpr (PLANES) {
      put_parts<NP>(vg, planes, rows * groups * 8, i * 8);
      put_parts<NP>(vu, planes + NP * rows * groups * 8, rows * groups * 8, i * 8);
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------

// Workgroups of 256 for `n` items, whose threads go on to further ones.
static unsigned blocks_for(int64_t n) { return (unsigned)std::min<int64_t>((n + 255) / 256, 1 << 16); }

// What one call multiplies: dx [t][256 kb] = the sum of dy[m] [t][n] W[m]^ over its `mats` gradients.
struct BwdCall {
  const tq_mat_mx* w[2];
  const void* dy[2];
  int mats, n, kb, type;
  int64_t t;
  bool lined;  // the tensors start at 16-byte pieces

  // Tiles that take dy in its type, and which calls need no parts of it. (The plan knows of sizes alone: where a tensor lies changes no bit.)
  bool in_type(const BwdPlan& p) const { return p.tile >= 0 && kBwdTiles[p.tile].in_type; }
  bool in_place(const BwdPlan& p) const { return p.tile < 0 || in_type(p) || (type == TQ_BF16 && whole_rows(n, type) && lined); }
};

template <typename F>
static void with_parts(int32_t type, F f) {
  if (type == TQ_F32) f(float{}, std::integral_constant<int, 3>{});
  else if (type == TQ_BF16) f(bf16_t{}, std::integral_constant<int, 1>{});
  else f(f16_t{}, std::integral_constant<int, 2>{});
}

// The product as planned, of dy in place or of its parts in `planes` (or of a copy there, for tiles that need its pieces lined up).
static void launch_bwd(BwdCall b, const BwdPlan& p, bf16_t* planes, float* part, void* dx, hipStream_t st) {
  if (b.in_type(p) && !b.lined)
    with_parts(b.type, [&](auto z, auto) {
      using T = decltype(z);
      for (int m = 0; m < b.mats; ++m) {
        T* copy = (T*)planes + m * b.t * b.n;
        hipLaunchKernelGGL(k_mx_copy<T>, dim3(blocks_for(b.t * b.n / 4)), dim3(256), 0, st, (const T*)b.dy[m], b.t * b.n / 4, copy);
        b.dy[m] = copy;
      }
    });
  const int np = parts_of(b.type);
  const int64_t quads = b.t * b.kb * 64, pad = pad_of(b.n);
  int sums = p.splits;
  if (p.tile < 0) {
    MxFewArgs a{};
    for (int m = 0; m < b.mats; ++m) a.dy[m] = b.dy[m], a.codes[m] = b.w[m]->codes, a.scales[m] = b.w[m]->scales;
    a.mats = b.mats, a.n = b.n, a.t = (int)b.t, a.kb = b.kb, a.type = b.type, a.splits = p.splits, a.out = dx;
    a.part = sums > 1 ? part : nullptr;
    const dim3 grid((unsigned)b.kb * 8, (unsigned)((b.t + 31) / 32), (unsigned)p.splits);
    with_parts(b.type, [&](auto z, auto npc) {
      hipLaunchKernelGGL((k_mx_bwd_few<decltype(z), decltype(npc)::value>), grid, dim3(kFewWaves * 64), 0, st, a);
    });
  } else {
    MxBwdArgs a{};
    const bool in_place = b.in_place(p);
    for (int m = 0; m < b.mats; ++m)
      for (int i = 0; i < (p.stacked || in_place ? 1 : np); ++i)  // (a gradient's parts follow each other)
        a.seg[a.nseg++] = in_place ? MxSeg{b.dy[m], b.w[m]->codes, b.w[m]->scales, b.n}
                                   : MxSeg{planes + (m * np + i) * b.t * pad, b.w[m]->codes, b.w[m]->scales, pad};
    if (p.stacked) sums *= np;
    a.n = b.n, a.t = (int)b.t * (p.stacked ? np : 1), a.kb = b.kb, a.type = b.type, a.splits = p.splits, a.out = dx;
    a.whole = (int)p.whole;
    a.part = sums > 1 ? part : nullptr;
    const BwdTile& c = kBwdTiles[p.tile];
    const int nx = a.nx = b.kb * (256 / c.bc), ny = a.ny = (a.t + c.bn - 1) / c.bn;
    const unsigned tiles = (unsigned)((int64_t)nx * ny);
    const dim3 grid = p.whole ? dim3((unsigned)(p.whole + (tiles - p.whole) * p.splits)) : dim3(tiles, 1, (unsigned)p.splits);
    switch (p.tile) {
      case 0: hipLaunchKernelGGL((k_mx_bwd<bf16_t, 128, 32, 4, 1, 1, 4, 1>), grid, dim3(256), 0, st, a); break;
      case 1: hipLaunchKernelGGL((k_mx_bwd<bf16_t, 128, 64, 4, 1, 1, 4, 1>), grid, dim3(256), 0, st, a); break;
      case 2: hipLaunchKernelGGL((k_mx_bwd<bf16_t, 128, 128, 4, 1, 2, 4, 1>), grid, dim3(512), 0, st, a); break;
      case 3: hipLaunchKernelGGL((k_mx_bwd<bf16_t, 256, 128, 4, 2, 1, 2, 2>), grid, dim3(512), 0, st, a); break;
      case 4: hipLaunchKernelGGL((k_mx_bwd<bf16_t, 256, 256, 2, 4, 1, 2, 2>), grid, dim3(512), 0, st, a); break;
      case 5:
        if (np == 2) hipLaunchKernelGGL((k_mx_bwd<f16_t, 128, 64, 2, 2, 1, 3, 1>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((k_mx_bwd<float, 128, 64, 2, 2, 1, 3, 1>), grid, dim3(256), 0, st, a);
        break;
      default:
        if (np == 2) hipLaunchKernelGGL((k_mx_bwd<f16_t, 256, 128, 2, 4, 1, 2, 4>), grid, dim3(512), 0, st, a);
        else hipLaunchKernelGGL((k_mx_bwd<float, 256, 128, 2, 4, 1, 2, 4>), grid, dim3(512), 0, st, a);
    }
    if (p.whole) {
      const int64_t tile_quads = ((int64_t)nx * ny - p.whole) * (c.bc * c.bn / 4);
      hipLaunchKernelGGL(k_mx_bwd_join_tiles, dim3((unsigned)((tile_quads + 255) / 256)), dim3(256), 0, st, part, sums, a.whole, nx, ny, c.bc, c.bn, a.t,
                         b.type, dx);
      return;
    }
  }
  if (sums > 1)
    hipLaunchKernelGGL(k_mx_bwd_join, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, part, sums, quads, b.type, dx);
}

static bool rows_in_range(int64_t t) { return t >= 0 && t <= kMxMaxRows; }

static bool weights_in_range(const tq_mat_mx* w) {
  return w && w->n >= 1 && w->n <= kMxMaxRows && w->k > 0 && w->k % 256 == 0 && w->k <= kMaxK;
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
  const BwdCall call{{w}, {dy}, 1, w->n, w->k / 256, type, t, aligned(dy, 16)};
  const BwdPlan plan = plan_bwd(t, call.kb, w->n, 1, type);
  bf16_t* planes = (bf16_t*)ws;
  if (!call.in_place(plan))
    with_parts(type, [&](auto z, auto npc) {
      using T = decltype(z);
      hipLaunchKernelGGL((k_mx_parts<T, decltype(npc)::value>), dim3(blocks_for(t * pad / 8)), dim3(256), 0, (hipStream_t)stream,
                         (const T*)dy, t, w->n, (int)(pad / 8), planes);
    });
  launch_bwd(call, plan, planes, (float*)((uint8_t*)ws + up256((size_t)np * t * pad * 2)), dx, (hipStream_t)stream);
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
  const BwdCall call{{gate, up}, {dg, du}, 2, n, gate->k / 256, type, t, aligned(dg, 16) && aligned(du, 16)};
  const BwdPlan plan = plan_bwd(t, call.kb, n, 2, type);
  bf16_t* planes = dx && !call.in_place(plan) ? (bf16_t*)ws : nullptr;  // (read and written with dg and du)
  with_parts(type, [&](auto z, auto npc) {
    using T = decltype(z);
    constexpr int NP = decltype(npc)::value;
    const int64_t groups = planes ? pad / 8 : (t * n + 7) / 8;
    if (planes)
      hipLaunchKernelGGL((k_gated_bwd<T, NP, true>), dim3(blocks_for(t * groups)), dim3(256), 0, (hipStream_t)stream, (const T*)g, (const T*)u,
                         (const T*)dh, act, t, (int64_t)n, groups, (T*)dg, (T*)du, planes);
    else
      hipLaunchKernelGGL((k_gated_bwd<T, NP, false>), dim3(blocks_for(groups)), dim3(256), 0, (hipStream_t)stream, (const T*)g, (const T*)u,
                         (const T*)dh, act, (int64_t)1, t * n, groups, (T*)dg, (T*)du, planes);
  });
  if (dx) launch_bwd(call, plan, (bf16_t*)ws, (float*)((uint8_t*)ws + up256((size_t)2 * np * t * pad * 2)), dx, (hipStream_t)stream);
  return check_launch("tq_gated_mx_bwd");
}
