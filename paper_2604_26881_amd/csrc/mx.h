// 8-bit rows with a power-of-two scale per 32 neighbours (the microscaling format that the gfx950 matrix cores take):
// value = e4m3 byte * 2^(scale byte - 127).
//
// The scale of a block with largest magnitude a is the smallest power of two, at least 2^-126, with a <= 448 * scale (448:
// the largest e4m3), so no value saturates: a value is off by at most half a step, 2^-4 of itself (values more than 2^15
// below the largest of their block: of 2^-6 * scale).  A block that holds an infinity or a NaN is NaN in scale and values.
// Both follow from the bits of a alone (its exponent, and one more where its mantissa is above that of 448), and the
// multiplication by the inverse scale is exact, so the only rounding is the conversion's, to nearest even.
#pragma once
#include "common.h"
#include <type_traits>

namespace moe {

template <int N>
using number = std::integral_constant<int, N>;

constexpr int MX = 32;                 // values per scale
constexpr int MX_DIM_MAX = 16384;     // H and I of an expert block: the scales of a workgroup's rows fit LDS beside its rings
constexpr uint32_t MX_NAN4 = 0x7f7f7f7fu;

// Scale byte of a block from the largest of its magnitudes' bits (as integers they order like the values, NaN above all)
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return 255u;
  const int b = (int)((amax_bits + 0x1fffffu) >> 23) - 8;     // mantissa above 1.75: the next power
  return (uint32_t)max(b, 1);
}
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return __uint_as_float((254u - min(byte, 253u)) << 23); }
// Four values to four e4m3 bytes; inv is the exact inverse of the block's scale
__device__ __forceinline__ uint32_t mx_pack4(float a, float b, float c, float d, float inv, uint32_t byte) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, v, true);
  return byte == 255u ? MX_NAN4 : (uint32_t)v;
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// Maximum over the four lanes of a quad
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));
}

// 32 bytes of a lane as the matrix instruction's operand
typedef __attribute__((ext_vector_type(8))) int i32x8;
__device__ __forceinline__ i32x8 mx_operand(u32x4 lo, u32x4 hi) {
  return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}
// Eight e4m3 bytes times their scale, in bf16: exact, NaN for a scale byte of 255
__device__ __forceinline__ bf16x8 mx_to_bf16(uint32_t lo, uint32_t hi, int scale_byte) {
  const float s = __uint_as_float((uint32_t)scale_byte << 23);
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// silu(g) * u with the reciprocal instruction, off by 2^-23 or so before the rounding to bf16 (below g = -87 the quotient is 0).  A
// division is eleven instructions: the tile kernel took 6 % longer with it.
__device__ __forceinline__ float silu_times(float g, float u) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u; }

// Arguments of the expert kernels on 8-bit weights: C[r, n] over the rows r of experts [lo, hi).
struct MxArgs {
  const uint8_t *A, *As;       // gate/up: token rows [rows, Kdim] and their scales [rows, Kdim / 32]; down: hidden rows, bf16 [rows, Kdim]
  const uint8_t *B0, *B0s;     // weights [E, N, Kdim] (gate branch, or the down projection), scales [E, N, Kdim / 32]
  const uint8_t *B1, *B1s;     // up branch (gate/up), else unused
  bf16_t* C;                   // hidden rows, or output rows, [rows, N]
  const int32_t* offsets;      // expert_offsets on the device
  int lo, hi;
  int rows_total;              // rows of all experts of the layer
  int mean_rows;               // rows_total / experts of the layer, rounded up: picks kernels
  int N, Kdim;
  const int32_t* gather;       // not nullptr: row r of A is A[gather[r] / gather_div]
  int gather_div;
};
int launch_stream_mx_gateup(const MxArgs& a, hipStream_t st);
int launch_stream_mx_down(const MxArgs& a, hipStream_t st);
// Tiles: more than 24 rows per expert, and a contraction long enough for their scales to come 16 bytes of a row at a time.
// (60 experts, H 2048, I 1408, gate/up + down, tiles and streamed: 17 rows 75 + 45 and 72 + 42 us, 27 rows 76 + 46 and 80 + 47,
// 40 rows 78 + 48 and 128 + 65.)
inline bool mx_in_tiles(const MxArgs& a) { return a.mean_rows > 24 && a.Kdim >= 512; }
int launch_tile_mx_gateup(const MxArgs& a, hipStream_t st);
int launch_tile_mx_down(const MxArgs& a, hipStream_t st);

int launch_quantize_mx(const void* x, int rows, int H, void* q, void* scales, hipStream_t st);
int launch_residual_norm_mx(const void* x, const void* y, const void* weight, int T, int H, float eps, void* sum, void* out,
                            void* q, void* scales, hipStream_t st);

struct RouteScored {
  const bf16_t *x, *Wr;
  const float* balance;
  int T, H, E, K, sigmoid, groups, top_groups, best, renorm;
  float scale;
  int32_t* ids;
  float* w;
};
int launch_route_scored(const RouteScored& a, hipStream_t st);

}  // namespace moe
