// Rows to MXFP4: blocks of 32 with one power-of-two scale, e2m1 codes in the layout of the MXFP4 arm.
//
// A block's largest magnitude is the largest of its bit patterns without the sign, as an integer; its exponent
// field less 2 is the scale byte, with no logarithm. The conversion instruction rounds x / scale to e2m1 (nearest even,
// magnitudes past 6 to 6; equal to the definition on every fp16 and bfloat16 value and at and beside every fp32 tie, scales from 2^-127 on).
#include "tq_mx.hpp"

namespace tq {

// The values of a block that a lane holds: H from element 16 / L * q, H from element 16 higher, L lanes a block.
template <typename T>
struct MxLane {
  static constexpr int H = 16 / (int)sizeof(T);  // 16 bytes each
  static constexpr int L = 16 / H;
};

template <typename T>
__global__ __launch_bounds__(256) void k_quantize_mx(const T* x, int64_t blocks, int noclip, uint8_t* __restrict__ codes,
                                                     uint8_t* __restrict__ scales, T* values) {
  constexpr int H = MxLane<T>::H, L = MxLane<T>::L;
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, b = i / L;
  const int q = (int)(i % L);
  if (b >= blocks) return;  // (the lanes of a block leave together)
  float v[2][H];
  load_n<H>(x + b * 32 + q * H, v[0]);
  load_n<H>(x + b * 32 + 16 + q * H, v[1]);
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < H; ++j) top = max(top, max(__float_as_uint(v[0][j]) & 0x7fffffffu, __float_as_uint(v[1][j]) & 0x7fffffffu));
  top = max(top, (uint32_t)dpp_i<kDppXor1>((int)top));
  if constexpr (L == 4) top = max(top, (uint32_t)dpp_i<kDppXor2>((int)top));
  const bool finite = top < 0x7f800000u;
  const int e = (int)(top >> 23) - 2 + (noclip && (top & 0x7fffffu) > 0x400000u);
  const uint32_t byte = finite ? (uint32_t)max(e, 0) : 255u;
  const float s = e8m0_f32(byte);
  uint32_t c[H / 4];
#pragma unroll
  for (int d = 0; d < H / 4; ++d) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0][4 * d + 0], v[1][4 * d + 0], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0][4 * d + 1], v[1][4 * d + 1], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0][4 * d + 2], v[1][4 * d + 2], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0][4 * d + 3], v[1][4 * d + 3], s, 3);
    c[d] = finite ? w : 0u;
  }
  if (codes) {
    typedef uint32_t piece __attribute__((ext_vector_type(H / 4)));
    piece w;
#pragma unroll
    for (int d = 0; d < H / 4; ++d) w[d] = c[d];
    *reinterpret_cast<piece*>(codes + b * 16 + q * H) = w;
    if (q == 0) scales[b] = (uint8_t)byte;
  }
  if (values) {
#pragma unroll
    for (int d = 0; d < H / 4; ++d) {
      const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[d], s, 0);
      const auto p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[d], s, 1);
      const auto p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[d], s, 2);
      const auto p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[d], s, 3);
      v[0][4 * d + 0] = p0[0]; v[1][4 * d + 0] = p0[1];
      v[0][4 * d + 1] = p1[0]; v[1][4 * d + 1] = p1[1];
      v[0][4 * d + 2] = p2[0]; v[1][4 * d + 2] = p2[1];
      v[0][4 * d + 3] = p3[0]; v[1][4 * d + 3] = p3[1];
    }
    store_n<H>(values + b * 32 + q * H, v[0]);
    store_n<H>(values + b * 32 + 16 + q * H, v[1]);
  }
}

}  // namespace tq

extern "C" tq_status tq_quantize_mx(const void* x, int32_t type, int64_t t, int32_t k, int32_t flags, uint8_t* codes,
                                    uint8_t* scales, void* values, void* stream) {
  using namespace tq;
  clear_error();
  if (!known_type(type)) return fail(TQ_ERR_INVALID, "tq_quantize_mx: unknown type %d", type);
  if (t < 0 || t > kMxMaxRows) return fail(TQ_ERR_INVALID, "tq_quantize_mx: t = %lld out of range", (long long)t);
  if (k <= 0 || k % 256 != 0 || k > kMaxK)
    return fail(TQ_ERR_INVALID, "tq_quantize_mx: k = %d must be a positive multiple of 256 <= %d", k, kMaxK);
  if (flags & ~TQ_MX_NOCLIP) return fail(TQ_ERR_INVALID, "tq_quantize_mx: unknown flags %d", flags);
  if (t == 0) return TQ_OK;
  if (!x || (!codes && !values) || (!codes != !scales)) return fail(TQ_ERR_INVALID, "tq_quantize_mx: null pointer");
  if (!aligned(x, 16) || !aligned(codes, 128) || !aligned(scales, 8) || !aligned(values, 16))
    return fail(TQ_ERR_ALIGN, "tq_quantize_mx: x and values must be 16-byte, codes 128-byte, scales 8-byte aligned");
  const size_t nx = (size_t)t * k * type_bytes(type), nc = (size_t)t * k / 2, ns = (size_t)t * k / 32;
  if (overlap(codes, nc, x, nx) || overlap(scales, ns, x, nx) || overlap(codes, nc, scales, ns) ||
      (values != x && overlap(values, nx, x, nx)) || overlap(values, nx, codes, nc) || overlap(values, nx, scales, ns))
    return fail(TQ_ERR_INVALID, "tq_quantize_mx: overlapping tensors");
  (void)hipGetLastError();
  with_type(type, [&](auto z) {
    using T = decltype(z);
    static_assert(kMxMaxRows * (kMaxK / 32) * MxLane<T>::L <= int64_t{1} << 31, "threads of a launch");
    const int64_t blocks = t * (k / 32), all = blocks * MxLane<T>::L;
    const int wg = all <= 256 * 64 ? 64 : 256;
    hipLaunchKernelGGL(k_quantize_mx<T>, dim3((unsigned)((all + wg - 1) / wg)), dim3(wg), 0, (hipStream_t)stream, (const T*)x, blocks,
                       flags & TQ_MX_NOCLIP, codes, scales, (T*)values);
  });
  return check_launch("tq_quantize_mx");
}
