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
// A workgroup is four waves that share 16 * WB weight rows (gate/up: half of them gate rows, half the matching up rows) and up
// to 16 * MT token rows of one expert, and cut K into four parts of whole steps: with one token's experts there are few column
// blocks, and four times the waves have four times the requests in flight.  A wave copies a step global -> LDS (whole
// 128-byte lines), takes it into registers, and asks for a later one into the same place before it multiplies.  One stage per
// wave: what keeps the memory busy is workgroups side by side, whose first and last steps overlap (60 experts, 8.5 rows each on
// average, H 2048, I 1408, gate/up and down: two stages 83 + 48 us, one 59 + 34); where there are no others, two.  The four
// partial sums meet in LDS and are added in the order of the parts.  The parts depend on the contraction alone, and where a wave
// starts in its part on the output column and the expert alone, so a row's bits do not depend on the block cut.
// Only the 1 KB pieces that hold token rows of the expert are copied (8 rows of 8 bits, 4 of bf16; for one row of bf16 four
// pieces would be half as many bytes as the weights).
// The first weights are requested before anything else; the scales of the rows (1/32 of the bytes) come next to them, once.
//
// The workgroups are column blocks by tiles of token rows of the experts that have any; a tile is found in registers
// from the row bounds on the device (a wave holds all of them, four experts per lane): experts without rows cost no workgroup
// (one token, 8 of 256 experts, H 4096, I 2048: 24 + 13 us; with a workgroup for every expert 39 + 28).
//
// Measured, gate/up + down (the weights at the 5.06 TB/s of a large copy in brackets): H 2048, I 1408, one token's 4 experts
// 8.3 + 5.2 us (4.7 + 2.4), 60 experts of 8.5 rows 58 + 33 (70 + 35); H 4096, I 2048, 160 experts of 1.6 rows 398 + 200
// (547 + 274).  With many experts the weights come at 6 to 7 TB/s; with one token's experts what is left is the chain of
// latencies: row bounds, sort, first lines, two more, the sum, the store.
//
// A last step of 64 (contractions that are not whole steps) copies its bytes twice and multiplies zeros in the second half.
#include "fold.h"
#include "mx.h"
#include <algorithm>
#include <type_traits>

namespace moe {
namespace {

template <int MT, int WB, bool GATEUP, int NST>
struct StreamMxShape {
  static constexpr int WROWS = 16 * WB;
  static constexpr int ROWS = 16 * MT;                      // token rows of a workgroup
  static constexpr int XROW = GATEUP ? 128 : 256;           // bytes of a token row per step
  static constexpr int XPIECE = 1024 / XROW;                // token rows of a 1 KB copy
  static constexpr int STAGE = WROWS * 128 + ROWS * XROW;   // of one wave
  static constexpr int RING = NST * STAGE;
  static constexpr int SROWS = WROWS + (GATEUP ? ROWS : 0); // rows with scales
  static constexpr int LDP = ROWS + 1;                      // partial sums: [WROWS][LDP], a padding word per row
  static constexpr int START = GATEUP ? 32 : 64;            // output columns that share their start in K, in every form
  static_assert(START % (GATEUP ? WROWS / 2 : WROWS) == 0, "a workgroup has one start");
  static_assert(STAGE >= WROWS * LDP * 4, "a wave's partial sums take the place of its stage");
};

template <int MT, int WB, bool GATEUP, int NST>
__global__ __launch_bounds__(256) void expert_stream_mx_kernel(MxArgs a) {
  using S = StreamMxShape<MT, WB, GATEUP, NST>;
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NPER = GATEUP ? S::WROWS / 2 : S::WROWS;    // output columns of a workgroup
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // workgroups go through the columns of a tile of token rows, then to the next tile (one dimension: a grid's others end at 65535)
  const unsigned column_blocks = (unsigned)(a.N / NPER), column = blockIdx.x % column_blocks;
  // the tile's expert and its rows
  int eg, m0, rb, Me;
  {
    const int nexp = a.hi - a.lo, want = (int)(blockIdx.x / column_blocks);
    int off[5], tiles[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 5; ++i) off[i] = a.offsets[a.lo + min(lane * 4 + i, nexp)];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += tiles[i] = (max(off[i + 1] - off[i], 0) + S::ROWS - 1) / S::ROWS;
    int before = wave_scan(sum) - sum;
    const unsigned long long mine = __ballot(before <= want && want < before + sum);
    if (mine == 0ull) return;
    const int owner = __builtin_ctzll(mine);
    int i = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      const bool on = i == j && want >= before + tiles[j];
      before += on ? tiles[j] : 0;
      i += on;
    }
    int at = off[0], end = off[1];
#pragma unroll
    for (int j = 1; j < 4; ++j) {
      at = i == j ? off[j] : at;
      end = i == j ? off[j + 1] : end;
    }
    eg = a.lo + owner * 4 + __builtin_amdgcn_readlane(i, owner);
    rb = __builtin_amdgcn_readlane(at, owner);
    Me = __builtin_amdgcn_readlane(end, owner) - rb;
    m0 = (want - __builtin_amdgcn_readlane(before, owner)) * S::ROWS;
  }
  const int rows = min(S::ROWS, Me - m0);
  const int N = a.N, Kdim = a.Kdim, kb32 = Kdim / MX;
  const int n0 = (int)column * NPER;
  const int nk = (Kdim + 127) / 128;
  const bool half_last = (Kdim & 127) != 0;
  // this wave's part of K: steps [k0, k0 + kn); its walk starts at a step of its own and wraps around (waves that start
  // together would otherwise ask the same memory channels, see expert_stream_lds.hip).  The start goes by the output columns in
  // units that every form has, never by the block of columns: how wide that is depends on the block cut (launch_stream_mx).
  const int k0 = nk * wave / 4, kn = nk * (wave + 1) / 4 - k0;
  const int rot = kn > 0 ? (int)(((unsigned)n0 / S::START * 3u + (unsigned)eg * 5u) % (unsigned)kn) : 0;
  auto step_of = [&](int s) { return k0 + (s + rot >= kn ? s + rot - kn : s + rot); };

  const size_t wrow = (size_t)eg * N + n0;
  const uint8_t* W0 = a.B0 + wrow * Kdim;                   // the first WROWS / 2 rows, and the others
  const uint8_t* W1 = GATEUP ? a.B1 + wrow * Kdim : W0 + (size_t)(S::WROWS / 2) * Kdim;
  unsigned char* const ring = smem + wave * S::RING;
  unsigned char* const scales = smem + 4 * S::RING;         // [SROWS][kb32]: the weight rows, then the token rows
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem, lds0 = lds_base + (uint32_t)(wave * S::RING);
  // copies of weights: lane -> row lane/8 of an 8-row group, slot lane%8 holding chunk slot xor row%8
  const int crow = lane >> 3, cchunk = (lane & 7) ^ crow;
  uint32_t coffW[WB];
#pragma unroll
  for (int i = 0; i < WB; ++i) coffW[i] = (uint32_t)(i * 8 + crow) * (uint32_t)Kdim + (uint32_t)cchunk * 16u;
  // of token rows, 8-bit: alike; bf16: row lane/16 of a 4-row group, slot lane%16 holding chunk slot xor row%16
  auto xrow = [&](int i) { return GATEUP ? i * 8 + crow : i * 4 + (lane >> 4); };
  auto xchunk = [&](int i) { return GATEUP ? cchunk : (lane & 15) ^ ((i * 4 + (lane >> 4)) & 15); };
  const int r16 = lane & 15, g = lane >> 4, swz = r16 & 7;

  auto issue_weights = [&](int s, uint32_t slot) {
    const uint32_t l = lds0 + slot * S::STAGE;
    const int k = step_of(s);
    const uint32_t back = half_last && k == nk - 1 && cchunk >= 4 ? 64u : 0u;     // the missing half from the half that is there
    const size_t kb = (size_t)k * 128;
#pragma unroll
    for (int i = 0; i < WB; ++i) copy_to_lds_16(W0 + kb, coffW[i] - back, l + (uint32_t)i * 1024u, true);
#pragma unroll
    for (int i = 0; i < WB; ++i) copy_to_lds_16(W1 + kb, coffW[i] - back, l + (uint32_t)(WB + i) * 1024u, true);
  };

  f32x4 acc[WB][MT];
#pragma unroll
  for (int b = 0; b < WB; ++b)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[b][mt] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto walk = [&](auto xn_) {
    constexpr int XN = decltype(xn_)::value;                // 1 KB pieces of token rows
    constexpr int MTX = (XN * S::XPIECE + 15) / 16;         // tiles of 16 token rows
    constexpr int NI = 2 * WB + XN;                         // copies of a stage
    for (int s = 0; s < min(kn, NST); ++s) issue_weights(s, (uint32_t)s);
    auto token_row = [&](int m) -> int {                    // rows past the end repeat the last row
      const int r = rb + m0 + min(m, rows - 1);
      return a.gather != nullptr ? a.gather[r] / a.gather_div : r;
    };
    uint32_t coffX[XN];
#pragma unroll
    for (int i = 0; i < XN; ++i) coffX[i] = (uint32_t)token_row(xrow(i)) * (uint32_t)(GATEUP ? Kdim : 2 * Kdim) + (uint32_t)xchunk(i) * 16u;
    auto issue_tokens = [&](int s, uint32_t slot) {
      const int k = step_of(s);
      const bool tail = half_last && k == nk - 1;
#pragma unroll
      for (int i = 0; i < XN; ++i) {
        const uint32_t back = tail && xchunk(i) >= (GATEUP ? 4 : 8) ? (uint32_t)S::XROW / 2u : 0u;
        copy_to_lds_16(a.A + (size_t)k * S::XROW, coffX[i] - back, lds0 + slot * S::STAGE + (uint32_t)(S::WROWS * 128 + i * 1024));
      }
    };
    // scales of the weight rows: two contiguous runs of WROWS / 2 rows
    {
      const uint8_t* S0 = a.B0s + wrow * kb32;
      const uint8_t* S1 = GATEUP ? a.B1s + wrow * kb32 : S0 + (size_t)(S::WROWS / 2) * kb32;
      const int run = S::WROWS / 2 * kb32;                  // a multiple of 16 bytes (kb32 is even, WROWS / 2 of 8)
      const uint32_t l = lds_base + 4u * S::RING;
      for (int i = wave * 64; i < run / 16; i += 256) {
        if (i + lane < run / 16) {
          copy_to_lds_16(S0, (uint32_t)(i + lane) * 16u, l + (uint32_t)i * 16u);
          copy_to_lds_16(S1, (uint32_t)(i + lane) * 16u, l + (uint32_t)(run + i * 16));
        }
      }
    }
    if (GATEUP) {
      for (int i = tid; i < rows * (kb32 / 2); i += 256) {  // (rows of an even number of bytes)
        const int m = i / (kb32 / 2), j = i - m * (kb32 / 2);
        *reinterpret_cast<uint16_t*>(scales + (S::WROWS + m) * kb32 + 2 * j) =
            *reinterpret_cast<const uint16_t*>(a.As + (size_t)token_row(m) * kb32 + 2 * j);
      }
      wait_lds_reads();                                     // (these writes)
    }
    for (int s = 0; s < min(kn, NST); ++s) issue_tokens(s, (uint32_t)s);
    wait_copies_but<0>();
    __syncthreads();

    uint32_t slot = 0;
    for (int s = 0; s < kn; ++s) {
      const int k = step_of(s);
      const bool tail = half_last && k == nk - 1;
      const unsigned char* const stage = ring + slot * S::STAGE;
      const unsigned char* sw0 = scales + r16 * kb32;
      u32x4 w[WB][2], x[MTX][S::XROW / 64];
      int sw[WB][GATEUP ? 1 : 2], sx[MTX];
#pragma unroll
      for (int b = 0; b < WB; ++b) {
#pragma unroll
        for (int p = 0; p < 2; ++p) w[b][p] = *reinterpret_cast<const u32x4*>(stage + b * 2048 + r16 * 128 + (((4 * p + g) ^ swz) << 4));
        if (GATEUP) {
          sw[b][0] = sw0[b * 16 * kb32 + min(4 * k + g, kb32 - 1)];
        } else {
#pragma unroll
          for (int p = 0; p < 2; ++p) sw[b][p] = sw0[b * 16 * kb32 + min(4 * k + 2 * p + (g >> 1), kb32 - 1)];
        }
      }
#pragma unroll
      for (int mt = 0; mt < MTX; ++mt) {
        const int row = min(mt * 16 + r16, XN * S::XPIECE - 1);     // (rows that were not copied repeat one that was)
        const unsigned char* at = stage + S::WROWS * 128 + row * S::XROW;
#pragma unroll
        for (int i = 0; i < S::XROW / 64; ++i)
          x[mt][i] = *reinterpret_cast<const u32x4*>(
              at + (GATEUP ? ((4 * i + g) ^ (row & 7)) << 4 : ((8 * (i >> 1) + 2 * g + (i & 1)) ^ (row & 15)) << 4));
        sx[mt] = GATEUP ? scales[(S::WROWS + min(mt * 16 + r16, rows - 1)) * kb32 + min(4 * k + g, kb32 - 1)] : 0;
      }
      // the empty asm makes the compiler wait for the LDS reads here: after it the stage may be overwritten
#pragma unroll
      for (int b = 0; b < WB; ++b) {
        asm volatile("" : "+v"(w[b][0]), "+v"(w[b][1]), "+v"(sw[b][0]));
        if (!GATEUP) asm volatile("" : "+v"(sw[b][GATEUP ? 0 : 1]));
      }
#pragma unroll
      for (int mt = 0; mt < MTX; ++mt) {
#pragma unroll
        for (int i = 0; i < S::XROW / 64; ++i) asm volatile("" : "+v"(x[mt][i]));
        if (GATEUP) asm volatile("" : "+v"(sx[mt]));
      }
      if (s + NST < kn) {
        issue_weights(s + NST, slot);
        issue_tokens(s + NST, slot);
      }
      slot = NST == 1 || slot + 1 == NST ? 0u : slot + 1u;
      if (tail) {                                           // zeros in the half that is not there, and any finite scale
        const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int b = 0; b < WB; ++b) {
          w[b][1] = zero;
          if (GATEUP && g >= 2) sw[b][0] = 127;
          if (!GATEUP) sw[b][GATEUP ? 0 : 1] = 127;
        }
#pragma unroll
        for (int mt = 0; mt < MTX; ++mt) {
#pragma unroll
          for (int i = S::XROW / 128; i < S::XROW / 64; ++i) x[mt][i] = zero;
          if (GATEUP && g >= 2) sx[mt] = 127;
        }
      }
      if constexpr (GATEUP) {
#pragma unroll
        for (int mt = 0; mt < MTX; ++mt)
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
            for (int mt = 0; mt < MTX; ++mt)
              acc[b][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, as_bf16x8(x[mt][GATEUP ? 0 : i]), acc[b][mt], 0, 0, 0);
          }
      }
      if (NST > 1 && s + NST < kn) wait_copies_but<(NST - 1) * NI>(); else wait_copies_but<0>();      // the next step has landed
    }
  };
  if (rows <= S::XPIECE) walk(std::integral_constant<int, 1>{});
  else if (rows <= 2 * S::XPIECE) walk(std::integral_constant<int, 2>{});
  else if (4 * S::XPIECE <= S::ROWS && rows <= 4 * S::XPIECE) walk(std::integral_constant<int, 4 * S::XPIECE <= S::ROWS ? 4 : 2>{});
  else walk(std::integral_constant<int, S::ROWS / S::XPIECE>{});

  // The partial sums meet in LDS, in the stages.  Accumulator element j of block b, tile mt: weight row 16 b + 4 g + j, token row
  // 16 mt + lane % 16.
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
  constexpr int CG = NPER / 4;                              // groups of four output columns
  for (int i = tid; i < rows * CG; i += 256) {
    const int m = i / CG, c = 4 * (i % CG);
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = total(c + j, m);
      if (GATEUP) v[j] = silu_times(v[j], total(S::WROWS / 2 + c + j, m));
    }
    *reinterpret_cast<uint2*>(a.C + (size_t)(rb + m0 + m) * N + n0 + c) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  }
}

template <int MT, int WB, bool GATEUP, int NST>
int launch_stream_mx_t(const MxArgs& a, hipStream_t st) {
  using S = StreamMxShape<MT, WB, GATEUP, NST>;
  auto kern = expert_stream_mx_kernel<MT, WB, GATEUP, NST>;
  constexpr int lds_max = 160 * 1024;
  static_assert(4 * S::RING + S::SROWS * (MX_DIM_MAX / MX) <= lds_max, "the longest contraction's scales fit beside the stages");
  const int lds = 4 * S::RING + S::SROWS * (a.Kdim / MX);
  static std::atomic<uint64_t> lds_raised{0};
  const int nexp = a.hi - a.lo;
  if (nexp > 256) return -2;
  if (raise_lds_limit((const void*)kern, lds_max, lds_raised) != 0) return -4;
  // tiles of 16 rows: at most one per expert that has rows, and one per 16 rows besides
  const int active = std::min(nexp, a.rows_total), tiles = active + (a.rows_total - active) / S::ROWS;
  hipLaunchKernelGGL(kern, dim3((unsigned)(a.N / (GATEUP ? S::WROWS / 2 : S::WROWS)) * (unsigned)tiles), dim3(256), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : -4;
}

template <bool GATEUP>
int launch_stream_mx(const MxArgs& a, hipStream_t st) {
  // 32 token rows per workgroup where many experts have more than 16: 60 experts (H 2048, I 1408) of 12 rows 68 + 38 us, with
  // 16 rows 66 + 36; of 17 rows 72 + 42, with 16 rows 88 + 45.
  if (a.mean_rows > 12) return launch_stream_mx_t<2, 4, GATEUP, 1>(a, st);
  // Few workgroups, one to a compute unit: a second stage per wave, and for down, whose blocks are the longer ones, blocks of 32
  // columns (H 2048, I 1408: one token's 4 experts 13.2 us both, with one stage 14.2, with that and 64 columns 15; two tokens' 8
  // experts, down alone, 6.5 and 7.4; two of 8 experts, H 4096, I 7168, down alone, 12 and 16.  With 660 and 480 workgroups, 15
  // experts, 19 + 12 with one stage, 24 + 14 with two.)
  if ((long)std::min(a.hi - a.lo, a.rows_total) * (a.N / (GATEUP ? 32 : 64)) <= 256)
    return launch_stream_mx_t<1, GATEUP ? 4 : 2, GATEUP, 2>(a, st);
  return launch_stream_mx_t<1, 4, GATEUP, 1>(a, st);
}

}  // namespace

int launch_stream_mx_gateup(const MxArgs& a, hipStream_t st) { return launch_stream_mx<true>(a, st); }
int launch_stream_mx_down(const MxArgs& a, hipStream_t st) { return launch_stream_mx<false>(a, st); }

}  // namespace moe
