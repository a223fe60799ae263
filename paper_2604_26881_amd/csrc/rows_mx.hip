// Rows of bf16 to 8-bit rows with scales, alone and behind the residual norm that precedes an MoE layer.
//
// Both are streams: every input is read once, every output written once, the row stays in registers in between.  A lane
// holds 8 neighbours (one 16-byte load, one 8-byte store), so the 32 values of a scale are the four lanes of a quad and
// their maximum is two lane exchanges.
#include "fold.h"
#include "mx.h"
#include <algorithm>

namespace moe {

// Eight values of this lane, a quarter of a block: their bytes to q[0 .. 8), the scale by the quad's first lane to *scale
__device__ __forceinline__ void store_mx8(const float (&v)[8], uint8_t* __restrict__ q, uint8_t* __restrict__ scale) {
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, magnitude(v[i]));
  const uint32_t byte = mx_scale_byte(quad_max(a));
  const float inv = mx_inverse(byte);
  uint2 o;
  o.x = mx_pack4(v[0], v[1], v[2], v[3], inv, byte);
  o.y = mx_pack4(v[4], v[5], v[6], v[7], inv, byte);
  *reinterpret_cast<uint2*>(q) = o;
  if ((threadIdx.x & 3) == 0) *scale = (uint8_t)byte;
}

// n8: eighths, rows * H / 8 (the rows are contiguous, and H is whole blocks)
__global__ __launch_bounds__(256) void quantize_mx_kernel(const bf16_t* __restrict__ x, size_t n8, uint8_t* __restrict__ q,
                                                          uint8_t* __restrict__ scales) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n8) return;     // (n8 is a multiple of 8: quads leave together)
  float v[8];
  widen8(reinterpret_cast<const u32x4*>(x)[i], v);
  store_mx8(v, q + 8 * i, scales + i / 4);
}

int launch_quantize_mx(const void* x, int rows, int H, void* q, void* scales, hipStream_t st) {
  const size_t n8 = (size_t)rows * (size_t)(H / 8);
  constexpr size_t most = (size_t)1 << 31;      // eighths of a launch (a grid has less than 2^32 threads)
  for (size_t at = 0; at < n8; at += most) {
    const size_t n = std::min(most, n8 - at);
    hipLaunchKernelGGL(quantize_mx_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, (const bf16_t*)x + 8 * at, n,
                       (uint8_t*)q + 8 * at, (uint8_t*)scales + at / 4);
    if (hipGetLastError() != hipSuccess) return -4;
  }
  return 0;
}

// Sum of the lanes' values in fp64; every lane returns it
__device__ __forceinline__ double fold_sum_f64(double a) {
  auto step = [&](auto ctrl_, auto rows_) {
    const unsigned long long b = __builtin_bit_cast(unsigned long long, a);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, decltype(ctrl_)::value, decltype(rows_)::value, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), decltype(ctrl_)::value, decltype(rows_)::value, 0xf, false);
    a += __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
  };
  step(number<0xB1>{}, number<0xf>{});       // strides 1, 2, 4, 8 within rows of 16
  step(number<0x4E>{}, number<0xf>{});
  step(number<0x141>{}, number<0xf>{});
  step(number<0x140>{}, number<0xf>{});
  step(number<0x142>{}, number<0xa>{});      // rows 1 and 3 take in the row before them, then the upper half the lower
  step(number<0x143>{}, number<0xc>{});
  const unsigned long long b = __builtin_bit_cast(unsigned long long, a);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
  return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}

// u = x + y; n = u / sqrt(mean(u^2) + eps) * weight.  One workgroup per token row, up to 4 x 8 values per lane (H <= 8192).
// The sum of squares is fp64 (no square of a bf16 overflows there), and so are 1 / sqrt and its products with u and the weight,
// rounded once to fp32: n is the nearest fp32 wherever it is one, though 1 / sqrt alone may lie beyond the range of fp32 (eps 0
// and rows of subnormals, large weights), and as few 8-bit values as can be land on the wrong side of a border.  sum and out
// are rounded once from fp32, and so are the 8-bit rows (from n itself, not from out).  What bounds it is the bytes: 16 384 rows
// of 2048, all outputs, 55 us, 5.5 TB/s; 777 rows of 4096, 8-bit rows alone, 4.8 us (with the factor as the sum of two fp32, which
// overflowed, 55 and 4.6).
__global__ __launch_bounds__(256) void residual_norm_mx_kernel(const bf16_t* x, const bf16_t* y, const bf16_t* __restrict__ weight,
                                                               int H, float eps, bf16_t* sum, bf16_t* out,
                                                               uint8_t* __restrict__ q, uint8_t* __restrict__ scales) {
  const size_t t = blockIdx.x;
  __shared__ double s_part[4];
  float u[4][8];
  double ss = 0.0;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int c = threadIdx.x + 256 * r;
    if (c < H / 8) {
      widen8(reinterpret_cast<const u32x4*>(x + t * H)[c], u[r]);
      if (y != nullptr) {
        float v[8];
        widen8(reinterpret_cast<const u32x4*>(y + t * H)[c], v);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[r][i] += v[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fma((double)u[r][i], (double)u[r][i], ss);
    }
  }
  const double wave_total = fold_sum_f64(ss);
  if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = wave_total;
  __syncthreads();
  const double scale = 1.0 / sqrt(((s_part[0] + s_part[1]) + (s_part[2] + s_part[3])) / (double)H + (double)eps);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int c = threadIdx.x + 256 * r;
    if (c < H / 8) {
      if (sum != nullptr)
        reinterpret_cast<u32x4*>(sum + t * H)[c] = u32x4{pack_bf16x2(u[r][0], u[r][1]), pack_bf16x2(u[r][2], u[r][3]),
                                                         pack_bf16x2(u[r][4], u[r][5]), pack_bf16x2(u[r][6], u[r][7])};
      float n[8], v[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
      if (weight != nullptr) widen8(reinterpret_cast<const u32x4*>(weight)[c], v);
#pragma unroll
      for (int i = 0; i < 8; ++i) n[i] = (float)((double)u[r][i] * (scale * (double)v[i]));
      if (out != nullptr)
        reinterpret_cast<u32x4*>(out + t * H)[c] = u32x4{pack_bf16x2(n[0], n[1]), pack_bf16x2(n[2], n[3]),
                                                         pack_bf16x2(n[4], n[5]), pack_bf16x2(n[6], n[7])};
      if (q != nullptr) store_mx8(n, q + t * H + 8 * c, scales + t * (H / MX) + c / 4);
    }
  }
}

int launch_residual_norm_mx(const void* x, const void* y, const void* weight, int T, int H, float eps, void* sum, void* out,
                            void* q, void* scales, hipStream_t st) {
  constexpr int most = 1 << 23;                 // rows of a launch (a grid has less than 2^32 threads)
  auto from = [](auto* p, size_t n) { return p != nullptr ? p + n : p; };
  for (int t = 0; t < T; t += std::min(most, T - t)) {
    const size_t at = (size_t)t * H;
    hipLaunchKernelGGL(residual_norm_mx_kernel, dim3(std::min(most, T - t)), dim3(256), 0, st, (const bf16_t*)x + at,
                       from((const bf16_t*)y, at), (const bf16_t*)weight, H, eps, from((bf16_t*)sum, at), from((bf16_t*)out, at),
                       from((uint8_t*)q, at), from((uint8_t*)scales, at / MX));
    if (hipGetLastError() != hipSuccess) return -4;
  }
  return 0;
}

}  // namespace moe
