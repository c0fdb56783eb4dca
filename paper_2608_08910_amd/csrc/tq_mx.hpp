// What the MXFP4 feed-forward operators share: argument checks, activation functions, matrix
// instruction operands.
#pragma once

#include "tq_ops.hpp"

namespace tq {

constexpr int64_t kMxMaxRows = int64_t{1} << 20;

// True where two byte ranges share a byte.
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
  return a && b && na && nb && p < q + nb && q < p + na;
}
// A tensor that lies on one of a matrix's planes.
inline bool on_matrix(const void* p, size_t n, const tq_mat_mx* m) {
  return overlap(p, n, m->codes, (size_t)m->n * m->k / 2) || overlap(p, n, m->scales, (size_t)m->n * m->k / 32);
}

// A weight matrix of these calls.
inline tq_status check_mx_weights(const char* what, const char* name, const tq_mat_mx* w) {
  if (!w) return fail(TQ_ERR_INVALID, "%s: null descriptor of %s", what, name);
  if (w->n < 1 || w->n > kMxMaxRows) return fail(TQ_ERR_INVALID, "%s: %s: n = %d out of range", what, name, w->n);
  if (w->k <= 0 || w->k % 256 != 0 || w->k > kMaxK)
    return fail(TQ_ERR_INVALID, "%s: %s: k = %d must be a positive multiple of 256 <= %d", what, name, w->k, kMaxK);
  if (!w->codes || !w->scales) return fail(TQ_ERR_INVALID, "%s: %s: null pointer", what, name);
  if (!aligned(w->codes, 128) || !aligned(w->scales, 8))
    return fail(TQ_ERR_ALIGN, "%s: %s: codes must be 128-byte, scales 8-byte aligned", what, name);
  return TQ_OK;
}

// The quantized rows of a batch (none: nothing of them is read).
inline tq_status check_mx_rows(const char* what, const tq_mat_mx* x, int32_t k) {
  if (!x) return fail(TQ_ERR_INVALID, "%s: null descriptor of x", what);
  if (x->n < 0 || x->n > kMxMaxRows) return fail(TQ_ERR_INVALID, "%s: x: %d rows out of range", what, x->n);
  if (x->k != k) return fail(TQ_ERR_INVALID, "%s: x has k = %d, the weights %d", what, x->k, k);
  if (x->n == 0) return TQ_OK;
  if (!x->codes || !x->scales) return fail(TQ_ERR_INVALID, "%s: x: null pointer", what);
  if (!aligned(x->codes, 128) || !aligned(x->scales, 8))
    return fail(TQ_ERR_ALIGN, "%s: x: codes must be 128-byte, scales 8-byte aligned", what);
  return TQ_OK;
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A lane's 32 e2m1 values as an operand of the scaled matrix instructions (fp4 operands fill the first 16 bytes).
__device__ __forceinline__ i32x8 fp4_operand(const uint4 w) {
  const i32x8 v = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
  return v;
}

// acc += A B over 64 elements of k: lane l holds row (column) l % 32 and one block of 32, with its scale byte J of sa (sb).
template <int J>
__device__ __forceinline__ f32x16 mfma_fp4_32(const uint4 a, const uint4 b, f32x16 acc, int sa, int sb) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fp4_operand(a), fp4_operand(b), acc, 4, 4, J, sa, J, sb);
}
// The same over 128 elements, rows (columns) l % 16.
template <int J>
__device__ __forceinline__ f32x4 mfma_fp4_16(const uint4 a, const uint4 b, f32x4 acc, int sa, int sb) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fp4_operand(a), fp4_operand(b), acc, 4, 4, J, sa, J, sb);
}

typedef int i32x4 __attribute__((ext_vector_type(4)));
// The words of make_rsrc's resource.
__device__ __forceinline__ i32x4 rsrc_words(const void* base, uint32_t bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  return i32x4{(int)(uint32_t)p, (int)(uint32_t)(p >> 32) & 0xffff, (int)bytes, 0x00020000};
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
// N bytes a lane from offset `at` to consecutive LDS addresses from dst (wave-uniform). Written out, so that the compiler
// does not wait for loads under way before each read of LDS; the kernel waits where it needs them (step_end). Writes m0 alone. The
// compiler keeps no distances into the block: s_mov and s_nop are the five wait states that a vector instruction's write of rs needs.
template <int N>
__device__ __forceinline__ void load_lds(i32x4 rs, uint32_t dst, uint32_t at) {
  static_assert(N == 16 || N == 4, "bytes a lane");
  if constexpr (N == 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(dst), "v"(at), "s"(rs) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(dst), "v"(at), "s"(rs) : "memory", "m0");
}
// s_waitcnt: all but the last `loads` loads have arrived, and all reads of LDS.
constexpr int wait_loads(int loads) { return (loads & 15) | (loads >> 4) << 14 | 0x0070; }

// Consecutive workgroups go to the eight dies in turn: the place of workgroup id of `all` in an order in which each die takes a run.
__device__ __forceinline__ int die_order(int id, int all) {
  const int die = id & 7;
  return die * (all / 8) + min(die, all % 8) + (id >> 3);
}

// An fp32 of the value 2^(E-127) for the scaled conversions (E = 255: an infinity, which they take for NaN).
__device__ __forceinline__ float e8m0_f32(uint32_t e) { return __uint_as_float(max(e << 23, 0x00400000u)); }

constexpr float kGeluA = 0.7978845608028654f, kGeluB = 0.044715f;  // sqrt(2 / pi)

// act(z) = z p, p the logistic function of a = z, or of a = 2 kGeluA (z + kGeluB z^3). exp of a large argument is an
// infinity and p then 0.
__device__ __forceinline__ float gelu_clamp(float z) { return z > 30.0f ? 30.0f : z < -30.0f ? -30.0f : z; }  // (p is 0 or 1 there; NaN stays)
__device__ __forceinline__ float act_argument(int act, float z) {
  if (act != TQ_ACT_GELU) return z;
  const float c = gelu_clamp(z);
  return 2.0f * kGeluA * (c + kGeluB * c * c * c);
}

// p = 1 / (1 + exp(-a)) and q = 1 - p, the larger from the smaller, which is right to a few of its own half steps: from a = 0 on q = exp(-a) / (1 + exp(-a)), p = 1 - q.
// (1 - p would be off by half a step of p, times z a': GELU's act' at z = 5 by 35 half steps; on random z of 4 to 6 11.1 on average, 0.7 so. 1 / (1 + exp(-a))
// for p is up to three times as far off as its one rounding, which turned bfloat16 ties of z times another value the wrong way.)
__device__ __forceinline__ void logistic(float a, float& p, float& q) {
  const float e = expf(-a), r = 1.0f / (1.0f + e);
  q = a >= 0.0f ? e * r : 1.0f - r;
  p = a >= 0.0f ? 1.0f - q : r;
}
__device__ __forceinline__ float act_fwd(int act, float z) {
  float p, q;
  logistic(act_argument(act, z), p, q);
  return z * p;
}

// act(z) and act'(z) = p + z p q a', a' = 1 or 2 kGeluA (1 + 3 kGeluB z^2).
__device__ __forceinline__ void act_both(int act, float z, float& a, float& da) {
  float p, q;
  logistic(act_argument(act, z), p, q);
  a = z * p;
  if (act == TQ_ACT_GELU) {
    const float c = gelu_clamp(z);
    da = p + c * p * q * (2.0f * kGeluA * (1.0f + 3.0f * kGeluB * c * c));
  } else {
    da = p * (1.0f + z * q);
  }
}

// The first `m` of four consecutive elements from i of a [type] tensor; m >= 4: all, in one access.
__device__ __forceinline__ void store4(int type, void* p, int64_t i, const float (&v)[4], int m) {
  if (m >= 4) {
    if (type == TQ_F32) store_n<4>((float*)p + i, v);
    else if (type == TQ_BF16) store_n<4>((bf16_t*)p + i, v);
    else store_n<4>((f16_t*)p + i, v);
    return;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (j < m) {
      if (type == TQ_F32) ((float*)p)[i + j] = v[j];
      else if (type == TQ_BF16) ((bf16_t*)p)[i + j] = (bf16_t)v[j];
      else ((f16_t*)p)[i + j] = (f16_t)v[j];
    }
}

}  // namespace tq
