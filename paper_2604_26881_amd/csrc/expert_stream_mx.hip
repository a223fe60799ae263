// Expert blocks on 8-bit weights, weights streamed: for experts with few rows, where the work is reading the weights once
// from HBM.
//
//   gate/up : h[r, n]  = bf16( silu(<A[r,:], Wg[e][n,:]>) * <A[r,:], Wu[e][n,:]> )     rows and weights in 8 bits
//   down    : Yp[r, n] = bf16( <h[r,:], Wd[e][n,:]> )                                  bf16 rows, 8-bit weights
//
// Matrix instructions, per K step of 128.  Gate/up: 16x16x128 on 8-bit values with a scale byte per lane: a lane holds, of row
// lane % 16, bytes 16 g .. + 15 and 64 + 16 g .. + 15 of the step (g = lane / 16), and gives the scale of the step's g-th
// block.  Down: the same bytes of the weights become bf16, exactly (4 significant bits, the exponent range of fp32; one
// instruction converts two and applies their scale), eight at a time for four 16x16x32 steps; the hidden rows are read in that
// order of K too.
//
// A workgroup is four waves that share 16 * WB weight rows (gate/up: half of them gate rows, half the matching up rows) and
// MT tiles of 16 token rows, and cut K into four parts of whole steps: with one token's experts there are few column blocks,
// and four times the waves have four times the requests in flight.  Each wave copies its steps global -> LDS (whole 128-byte
// lines) into a ring of its own, as the bf16 streaming kernels do; the four partial sums meet in LDS and are added in the
// order of the parts.  The cut depends on the contraction alone, so a row's bits do not depend on the block cut.
// The scales (1/32 of the bytes) of a workgroup's rows are staged once, before the first step.
// A last step of 64 (contractions that are not whole steps) copies its bytes twice and multiplies zeros in the second half.
#include "mx.h"
#include <algorithm>

namespace moe {
namespace {

template <int MT, int WB, bool GATEUP, int NST>
struct StreamMxShape {
  static constexpr int WROWS = 16 * WB;
  static constexpr int PASS = 16 * MT;                      // token rows of a pass
  static constexpr int XROW = GATEUP ? 128 : 256;           // bytes of a token row per step
  static constexpr int XC = XROW / 64;                      // 1 KB copies per tile of 16 token rows
  static constexpr int STAGE = WROWS * 128 + PASS * XROW;
  static constexpr int NI = 2 * WB + XC * MT;               // 1 KB copies per stage
  static constexpr int RING = NST * STAGE;                  // of one wave
  static constexpr int SROWS = WROWS + (GATEUP ? PASS : 0); // rows with scales
  static constexpr int LDP = PASS + 1;                      // partial sums: [WROWS][LDP], a padding word per row
  static_assert(NST >= 2 && NST * NI < 64, "the wait counter holds 6 bits");
  static_assert(RING >= WROWS * LDP * 4, "a wave's partial sums take the place of its ring");
};

template <int MT, int WB, bool GATEUP, int NST>
__global__ __launch_bounds__(256) void expert_stream_mx_kernel(MxArgs a) {
  using S = StreamMxShape<MT, WB, GATEUP, NST>;
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NPER = GATEUP ? S::WROWS / 2 : S::WROWS;    // output columns of a workgroup
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int eg = a.lo + (int)blockIdx.y;
  const int rb = a.offsets[eg], Me = a.offsets[eg + 1] - rb;
  if (Me <= (int)blockIdx.z * S::PASS) return;
  const int N = a.N, Kdim = a.Kdim, kb32 = Kdim / MX;
  const int n0 = (int)blockIdx.x * NPER;
  const int nk = (Kdim + 127) / 128;
  const bool half_last = (Kdim & 127) != 0;
  // this wave's part of K: steps [k0, k0 + kn); its walk starts at a step of its own and wraps around (waves that start
  // together would otherwise ask the same memory channels, see expert_stream_lds.hip)
  const int k0 = nk * wave / 4, kn = nk * (wave + 1) / 4 - k0;
  const int rot = kn > 0 ? (int)((blockIdx.x * 3u + (unsigned)eg * 5u) % (unsigned)kn) : 0;
  auto step_of = [&](int s) { return k0 + (s + rot >= kn ? s + rot - kn : s + rot); };

  const size_t wrow = (size_t)eg * N + n0;
  const uint8_t* W0 = a.B0 + wrow * Kdim;                   // the first WROWS / 2 rows, and the others
  const uint8_t* W1 = GATEUP ? a.B1 + wrow * Kdim : W0 + (size_t)(S::WROWS / 2) * Kdim;
  unsigned char* const ring = smem + wave * S::RING;
  unsigned char* const scales = smem + 4 * S::RING;         // [SROWS][kb32]: the weight rows, then the token rows
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)ring;
  // copies of weights: lane -> row lane/8 of an 8-row group, slot lane%8 holding chunk slot xor row%8
  const int crow = lane >> 3, cchunk = (lane & 7) ^ crow;
  uint32_t coffW[WB];
#pragma unroll
  for (int i = 0; i < WB; ++i) coffW[i] = (uint32_t)(i * 8 + crow) * (uint32_t)Kdim + (uint32_t)cchunk * 16u;
  // of token rows, 8-bit: alike; bf16: row lane/16 of a 4-row group, slot lane%16 holding chunk slot xor row%16
  auto xrow = [&](int i) { return GATEUP ? i * 8 + crow : i * 4 + (lane >> 4); };
  auto xchunk = [&](int i) { return GATEUP ? cchunk : (lane & 15) ^ (i * 4 + (lane >> 4)); };
  const int r16 = lane & 15, g = lane >> 4, swz = r16 & 7;

  // scales of the weight rows: two contiguous runs of WROWS / 2 rows
  {
    const uint8_t* S0 = a.B0s + wrow * kb32;
    const uint8_t* S1 = GATEUP ? a.B1s + wrow * kb32 : S0 + (size_t)(S::WROWS / 2) * kb32;
    const int run = S::WROWS / 2 * kb32;                    // a multiple of 16 bytes (kb32 is even, WROWS / 2 of 16)
    for (int i = tid; i < run / 16; i += 256) {
      *reinterpret_cast<u32x4*>(scales + 16 * i) = reinterpret_cast<const u32x4*>(S0)[i];
      *reinterpret_cast<u32x4*>(scales + run + 16 * i) = reinterpret_cast<const u32x4*>(S1)[i];
    }
  }

  for (int m0 = (int)blockIdx.z * S::PASS; m0 < Me; m0 += S::PASS * (int)gridDim.z) {
    auto token_row = [&](int m) -> int {                    // rows past the end repeat the last row
      const int r = rb + min(m, Me - 1);
      return a.gather != nullptr ? a.gather[r] / a.gather_div : r;
    };
    uint32_t coffX[MT][S::XC];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < S::XC; ++i)
        coffX[mt][i] = (uint32_t)token_row(m0 + mt * 16 + xrow(i)) * (uint32_t)(GATEUP ? Kdim : 2 * Kdim) + (uint32_t)xchunk(i) * 16u;
    if (GATEUP) {
      for (int i = tid; i < S::PASS * (kb32 / 2); i += 256) {   // (rows of an even number of bytes)
        const int m = i / (kb32 / 2), j = i - m * (kb32 / 2);
        *reinterpret_cast<uint16_t*>(scales + (S::WROWS + m) * kb32 + 2 * j) =
            *reinterpret_cast<const uint16_t*>(a.As + (size_t)token_row(m0 + m) * kb32 + 2 * j);
      }
    }
    __syncthreads();

    f32x4 acc[WB][MT];
#pragma unroll
    for (int b = 0; b < WB; ++b)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) acc[b][mt] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto issue = [&](int s, int slot) {
      const uint32_t l = lds0 + (uint32_t)slot * S::STAGE;
      const int k = step_of(s);
      const size_t kb = (size_t)k * 128;
      const bool tail = half_last && k == nk - 1;           // chunks of the missing half come from the half that is there
      const uint32_t back = tail && cchunk >= 4 ? 64u : 0u;
#pragma unroll
      for (int i = 0; i < WB; ++i) copy_to_lds_16(W0 + kb, coffW[i] - back, l + (uint32_t)i * 1024u, true);
#pragma unroll
      for (int i = 0; i < WB; ++i) copy_to_lds_16(W1 + kb, coffW[i] - back, l + (uint32_t)(WB + i) * 1024u, true);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < S::XC; ++i) {
          const uint32_t xback = GATEUP ? back : tail && xchunk(i) >= 8 ? 128u : 0u;
          copy_to_lds_16(a.A + (GATEUP ? kb : 2 * kb), coffX[mt][i] - xback, l + (uint32_t)(2 * WB + mt * S::XC + i) * 1024u);
        }
    };
    auto consume = [&](int s, int slot, auto&& then) {
      const int k = step_of(s);
      const bool tail = half_last && k == nk - 1;
      const unsigned char* st = ring + slot * S::STAGE;
      const unsigned char* sw0 = scales + r16 * kb32;
      u32x4 w[WB][2], x[MT][S::XC];
      int sw[WB][GATEUP ? 1 : 2], sx[MT];
#pragma unroll
      for (int b = 0; b < WB; ++b) {
#pragma unroll
        for (int p = 0; p < 2; ++p) w[b][p] = *reinterpret_cast<const u32x4*>(st + b * 2048 + r16 * 128 + (((4 * p + g) ^ swz) << 4));
        if (GATEUP) {
          sw[b][0] = sw0[b * 16 * kb32 + min(4 * k + g, kb32 - 1)];
        } else {
#pragma unroll
          for (int p = 0; p < 2; ++p) sw[b][p] = sw0[b * 16 * kb32 + min(4 * k + 2 * p + (g >> 1), kb32 - 1)];
        }
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const unsigned char* sx0 = st + S::WROWS * 128 + mt * 16 * S::XROW + r16 * S::XROW;
#pragma unroll
        for (int i = 0; i < S::XC; ++i)
          x[mt][i] = *reinterpret_cast<const u32x4*>(
              sx0 + (GATEUP ? ((4 * i + g) ^ swz) << 4 : ((8 * (i >> 1) + 2 * g + (i & 1)) ^ r16) << 4));
        sx[mt] = GATEUP ? sw0[(S::WROWS + mt * 16) * kb32 + min(4 * k + g, kb32 - 1)] : 0;
      }
      // the empty asm makes the compiler wait for the LDS reads here: after it the slot may be overwritten
#pragma unroll
      for (int b = 0; b < WB; ++b) {
        asm volatile("" : "+v"(w[b][0]), "+v"(w[b][1]), "+v"(sw[b][0]));
        if (!GATEUP) asm volatile("" : "+v"(sw[b][GATEUP ? 0 : 1]));
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int i = 0; i < S::XC; ++i) asm volatile("" : "+v"(x[mt][i]));
        if (GATEUP) asm volatile("" : "+v"(sx[mt]));
      }
      then();
      if (tail) {                                           // zeros in the half that is not there, and any finite scale
        const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int b = 0; b < WB; ++b) {
          w[b][1] = zero;
          if (GATEUP && g >= 2) sw[b][0] = 127;
          if (!GATEUP) sw[b][GATEUP ? 0 : 1] = 127;
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
          for (int i = S::XC / 2; i < S::XC; ++i) x[mt][i] = zero;
          if (GATEUP && g >= 2) sx[mt] = 127;
        }
      }
      if constexpr (GATEUP) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int b = 0; b < WB; ++b)
            acc[b][mt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(w[b][0], w[b][1]), mx_operand(x[mt][0], x[mt][1]),
                                                                          acc[b][mt], 0, 0, 0, sw[b][0], 0, sx[mt]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int b = 0; b < WB; ++b) {
            const bf16x8 wf = mx_to_bf16(w[b][i >> 1][2 * (i & 1)], w[b][i >> 1][2 * (i & 1) + 1], sw[b][GATEUP ? 0 : i >> 1]);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
              acc[b][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, as_bf16x8(x[mt][GATEUP ? 0 : i]), acc[b][mt], 0, 0, 0);
          }
      }
    };
    if (kn > NST) {
#pragma unroll
      for (int s = 0; s < NST - 1; ++s) issue(s, s);
      int slot = 0;
      for (int s = 0; s < kn; ++s) {
        if (s + NST - 1 <= kn) wait_copies_but<(NST - 2) * S::NI>(); else wait_copies_but<0>();
        const int free_slot = slot == 0 ? NST - 1 : slot - 1;
        consume(s, slot, [&] { if (s + NST - 1 < kn) issue(s + NST - 1, free_slot); });
        slot = slot + 1 == NST ? 0 : slot + 1;
      }
    } else {
      for (int s = 0; s < kn; ++s) issue(s, s);
      wait_copies_but<0>();
      for (int s = 0; s < kn; ++s) consume(s, s, [] {});
    }

    // The partial sums meet in LDS, in the rings.  Accumulator element j of block b, tile mt: weight row 16 b + 4 g + j, token
    // row 16 mt + lane % 16.
    float* const part = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int b = 0; b < WB; ++b)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[(b * 16 + 4 * g + j) * S::LDP + mt * 16 + r16] = acc[b][mt][j];
    __syncthreads();
    auto total = [&](int row, int m) -> float {
      const float* p = reinterpret_cast<const float*>(smem) + row * S::LDP + m;
      constexpr int next = S::RING / 4;
      return ((p[0] + p[next]) + p[2 * next]) + p[3 * next];
    };
    constexpr int CG = NPER / 4;                            // groups of four output columns
    for (int i = tid; i < S::PASS * CG; i += 256) {
      const int m = i / CG, c = 4 * (i % CG);
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = total(c + j, m);
        if (GATEUP) v[j] = __fdividef(v[j], 1.0f + __expf(-v[j])) * total(S::WROWS / 2 + c + j, m);
      }
      if (m0 + m < Me)
        *reinterpret_cast<uint2*>(a.C + (size_t)(rb + m0 + m) * N + n0 + c) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
    __syncthreads();     // the next pass's copies and scales take the place of what was read here
  }
}

template <int MT, int WB, bool GATEUP, int NST>
int launch_stream_mx_t(const MxArgs& a, hipStream_t st) {
  using S = StreamMxShape<MT, WB, GATEUP, NST>;
  auto kern = expert_stream_mx_kernel<MT, WB, GATEUP, NST>;
  constexpr int lds_max = 160 * 1024;
  static_assert(4 * S::RING + S::SROWS * (MX_DIM_MAX / MX) <= lds_max, "the longest contraction's scales fit beside the rings");
  const int lds = 4 * S::RING + S::SROWS * (a.Kdim / MX);
  static std::atomic<uint64_t> lds_raised{0};
  if (raise_lds_limit((const void*)kern, lds_max, lds_raised) != 0) return -4;
  const int passes_max = (a.rows_total + S::PASS - 1) / S::PASS;
  const int gz = std::max(1, std::min(8, passes_max / 2));
  hipLaunchKernelGGL(kern, dim3(a.N / (GATEUP ? S::WROWS / 2 : S::WROWS), a.hi - a.lo, gz), dim3(256), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : -4;
}

}  // namespace

int launch_stream_mx_gateup(const MxArgs& a, hipStream_t st) { return launch_stream_mx_t<1, 4, true, 2>(a, st); }
int launch_stream_mx_down(const MxArgs& a, hipStream_t st) { return launch_stream_mx_t<1, 4, false, 2>(a, st); }

}  // namespace moe
