// Expert blocks on 8-bit weights in MFMA tiles: for experts with many rows.
//
//   gate/up : h[r, n]  = bf16( silu(<A[r,:], Wg[e][n,:]>) * <A[r,:], Wu[e][n,:]> )     rows and weights in 8 bits
//   down    : Yp[r, n] = bf16( <h[r,:], Wd[e][n,:]> )                                  bf16 rows, 8-bit weights
//
// A tile is BM token rows of one expert by 256 weight rows (gate/up: 128 gate rows and the matching 128 up rows), eight waves
// as 2 x 4, each on BM / 2 token rows by 64 weight rows (a gate block of 32 and its up block).  The kernel is persistent: every
// wave forms the tiles of the experts in registers from the row bounds on the device and walks tile numbers with a fixed
// stride, as the bf16 tile kernels do (expert_tile.hip has the measurements behind that walk: XCDs take runs of neighbouring
// tiles, experts with few and with many tiles are drawn in turn).
//
// K steps of 128 (gate/up) or 64 (down: a bf16 row has as many bytes) through a ring of NS LDS stages filled by asynchronous
// copies, a row's 16-byte chunks xor-swizzled against bank conflicts; one barrier per step.  The scales of a step come with
// it, one 4-byte slot per row: gate/up four scale bytes (a contraction that is not whole steps has rows of scales on odd
// multiples of two bytes: then two slots of two bytes), down two.
//
// Gate/up multiplies with 32x32x64 on 8-bit values: a lane holds of row lane % 32 the chunks 4m + h and 4m + 2 + h of the
// step's half m (h = lane / 32) and gives the scale of block 2m + h: the row's slot, shifted by h bytes, and a byte select.
// Down turns weights into bf16 on their way from LDS to the matrix cores, exactly, 16 neighbours per lane, for two
// 32x32x16 steps; the hidden rows are read in that order of K.  The conversions (32 per wave and step of 1024 MFMA clocks)
// run beside the other wave's matrix instructions.
//
// Rows past the end of an expert repeat its last row and are not stored; 32-row blocks of nothing but such rows are not
// multiplied.  Experts whose rows fit one tile read every weight once: their tiles ask for weights with the read-once hint and
// start their walk over K at a step of their own.  A row's bits depend on the tile height (picked from layer-wide sizes) and
// that start (from expert and column), never on the block cut.
#include <math.h>
#include <algorithm>
#include <type_traits>
#include "mx.h"

namespace moe {
namespace {

constexpr int TILE_MX_EMAX = 256;

template <int BM, bool GATEUP, int NS, bool PAIR>
struct TileMxShape {
  static constexpr int BN = 256, WAVES_M = 2, WAVES_N = 4, NW = 8;
  static constexpr int TB = BM / 64, NB = 2;                // 32-row blocks of a wave: tokens, weights
  static constexpr int NOUT = GATEUP ? BN / 2 : BN;         // output columns of a tile
  static constexpr int BK = GATEUP ? 128 : 64;              // K values per step
  static constexpr int WROWB = GATEUP ? 128 : 64;           // bytes per staged weight row (token rows: 128)
  static constexpr int SROWS = GATEUP ? BM + BN : BN;       // rows with scales
  static constexpr int TOKENS = BM * 128, WEIGHTS = BN * WROWB;
  static constexpr int STAGE = TOKENS + WEIGHTS + SROWS * 4 * (PAIR ? 2 : 1);
  static constexpr int NLA = BM / 64;                       // 1 KB copies per wave and stage: token rows,
  static constexpr int NLB = GATEUP ? 4 : 2;                // weight rows,
  static constexpr int NLS = PAIR ? 2 : 1;                  // scales (64 rows each)
  static constexpr int NL = NLA + NLB + NLS;
  static constexpr int GM = 4;                              // token tiles per locality group of the walk
  static_assert(GATEUP || !PAIR, "the down projection's steps have two scale bytes");
  static_assert(NS >= 2 && NS * NL < 64 && NS * STAGE <= 160 * 1024, "wait counter and LDS");
};

// One value of SZ bytes per lane into LDS, four bytes apart (zero-extended)
template <int SZ>
__device__ __forceinline__ void copy_to_lds_small(const void* base, uint32_t voff, uint32_t lds) {
  if constexpr (SZ == 2)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_ushort %0, %1" ::"v"(voff), "s"(base), "s"(lds) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(voff), "s"(base), "s"(lds) : "memory", "m0");
}

template <int BM, bool GATEUP, int NS, bool PAIR, bool SINGLE>
__global__ __launch_bounds__(512, 2) void expert_tile_mx_kernel(MxArgs a) {
  using S = TileMxShape<BM, GATEUP, NS, PAIR>;
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int HEAVY_MIN = 3;       // token tiles from which an expert counts as bound by the matrix cores
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / S::WAVES_N, wn = wave % S::WAVES_N;
  const int nexp = a.hi - a.lo;

  // rows [rb, re) and tiles [first, last) (in its class's list) of four experts per lane
  int first[4], last[4], rb[4], re[4], cnt[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = lane * 4 + i;
    rb[i] = e < nexp ? a.offsets[a.lo + e] : 0;
    re[i] = e < nexp ? a.offsets[a.lo + e + 1] : 0;
    last[i] = (max(re[i] - rb[i], 0) + BM - 1) / BM;
    cnt[last[i] >= HEAVY_MIN] += last[i];
  }
  int total[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    int incl = cnt[c];
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int o = __shfl_up(incl, s, WAVE);
      if (lane >= s) incl += o;
    }
    total[c] = __builtin_amdgcn_readlane(incl, 63);
    cnt[c] = incl - cnt[c];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool heavy = last[i] >= HEAVY_MIN;
    first[i] = heavy ? cnt[1] : cnt[0];
    last[i] += first[i];
    cnt[0] = heavy ? cnt[0] : last[i];
    cnt[1] = heavy ? last[i] : cnt[1];
  }
  const int total0 = total[0], total1 = total[1];
  const int grp0 = (total0 + S::GM - 1) / S::GM, grp1 = (total1 + S::GM - 1) / S::GM;   // locality groups per class
  const int ngrp = grp0 + grp1;
  const int N = a.N, Kdim = a.Kdim, kb32 = Kdim / MX;
  const int NT = (N + S::NOUT - 1) / S::NOUT;
  const int nk = (Kdim + S::BK - 1) / S::BK;
  const int groupTiles = S::GM * NT;
  const int Lend = grp0 == 0 || grp1 == 0 ? (total0 + total1) * NT : ngrp * groupTiles;
  // light groups among the first g of the merged walk: (g * light_ratio) >> 32, exactly grp0 at g = ngrp
  const unsigned long long light_ratio = ngrp > 0 ? ((((unsigned long long)grp0) << 32) + (unsigned)ngrp - 1ull) / (unsigned)ngrp : 0ull;

  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int crow = lane >> 3, cchunk = (lane & 7) ^ crow;   // copies of 128-byte rows: row lane/8, slot lane%8 holding chunk slot xor row%8
  const int r32 = lane & 31, half = lane >> 5, swz = lane & 7;
  const uint32_t tail_back = GATEUP && cchunk >= 4 ? 64u : 0u;

  const int G = gridDim.x;
  const bool xcd_walk = (G % 8) == 0;
  const int slot = xcd_walk ? (int)(blockIdx.x >> 3) : 0;
  const int run = xcd_walk ? max(1, min(G >> 3, (Lend + 7) >> 3)) : 1;
  if (xcd_walk && slot >= run) return;

  struct Tile { int row0, rowEnd, tbv, n0; bool once, valid; };
  const uint8_t *Ag = nullptr, *Bg0 = nullptr, *Bg1 = nullptr, *Sg = nullptr;
  uint32_t coff[S::NLA + S::NLB], soff = 0;     // byte offsets of this lane's parts of a stage's copies, at K step 0
  int krot = 0;
  auto kstep = [&](int kt) -> int { const int k = kt + krot; return k >= nk ? k - nk : k; };
  auto issue = [&](int kt, int st, auto once_) {
    const int k = kstep(min(kt, nk - 1));       // (past the end the last step again: the wait counts stay constant)
    const uint32_t l = lds0 + (uint32_t)st * S::STAGE + (uint32_t)wave * 1024u;
    const uint32_t back = PAIR && k == nk - 1 ? tail_back : 0u;     // the missing half from the half that is there
#pragma unroll
    for (int i = 0; i < S::NLA; ++i) copy_to_lds_16(Ag + (size_t)k * 128, coff[i] - back, l + (uint32_t)i * 8192u);
#pragma unroll
    for (int i = 0; i < S::NLB; ++i)
      copy_to_lds_16((GATEUP && i >= 2 ? Bg1 : Bg0) + (size_t)k * S::WROWB, coff[S::NLA + i] - back, l + (uint32_t)(S::TOKENS + i * 8192),
                     decltype(once_)::value);
    const uint32_t ls = lds0 + (uint32_t)st * S::STAGE + (uint32_t)(S::TOKENS + S::WEIGHTS) + (uint32_t)(wave % (S::SROWS / 64)) * 256u;
    if constexpr (!GATEUP) {
      copy_to_lds_small<2>(Sg + 2 * (size_t)k, soff, ls);
    } else if constexpr (PAIR) {
      copy_to_lds_small<2>(Sg + 4 * (size_t)k, soff, ls);
      copy_to_lds_small<2>(Sg + 4 * (size_t)k + (k == nk - 1 ? 0 : 2), soff, ls + (uint32_t)S::SROWS * 4u);
    } else {
      copy_to_lds_small<4>(Sg + 4 * (size_t)k, soff, ls);
    }
  };

  int it = 0;
  auto next_tile = [&]() -> Tile {
    Tile t{};
    int mrow = 0, nt = 0, cls = 0;
    for (;; ++it) {
      const int L = xcd_walk ? ((it * 8 + (int)(blockIdx.x & 7)) * run + slot) : (it * G + (int)blockIdx.x);
      if (L >= Lend) return t;
      const int grp = L / groupTiles, rem = L - grp * groupTiles;
      const int before = (int)(((unsigned long long)(unsigned)grp * light_ratio) >> 32);
      cls = (int)(((unsigned long long)(unsigned)(grp + 1) * light_ratio) >> 32) > before ? 0 : 1;
      const int g0 = (cls == 0 ? before : grp - before) * S::GM;
      const int size = min(S::GM, (cls == 0 ? total0 : total1) - g0);
      nt = rem / size;
      mrow = g0 + rem - nt * size;
      if (nt < NT) break;
    }
    ++it;
    t.valid = true;
    int at = 0, vf = 0, vb = 0, ve = 0;
    unsigned long long found = 0ull;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool mine = (last[i] - first[i] >= HEAVY_MIN) == (cls == 1) && first[i] <= mrow && mrow < last[i];
      found |= __ballot(mine);
      at = mine ? i : at;
      vf = mine ? first[i] : vf;
      vb = mine ? rb[i] : vb;
      ve = mine ? re[i] : ve;
    }
    const int owner = __builtin_ctzll(found);
    const int eg = a.lo + owner * 4 + __builtin_amdgcn_readlane(at, owner);
    const int rb_e = __builtin_amdgcn_readlane(vb, owner);
    t.row0 = rb_e + (mrow - __builtin_amdgcn_readlane(vf, owner)) * BM;
    t.rowEnd = __builtin_amdgcn_readlane(ve, owner);
    const int rows = min(BM, t.rowEnd - t.row0);
    t.tbv = min(S::TB, max(1, (((rows + 31) >> 5) - wm + S::WAVES_M - 1) / S::WAVES_M));
    t.n0 = nt * S::NOUT;
    t.once = SINGLE && t.rowEnd - rb_e <= BM;
    auto token = [&](int r) -> int {
      const int row = t.row0 + min(r, rows - 1);
      return GATEUP && a.gather != nullptr ? a.gather[row] / a.gather_div : row;
    };
    auto column = [&](int r) { return min(t.n0 + r, N - 1); };
    Ag = a.A;
    const size_t wrow = (size_t)eg * N;
    Bg0 = a.B0 + wrow * Kdim;
    Bg1 = GATEUP ? a.B1 + wrow * Kdim : nullptr;
#pragma unroll
    for (int i = 0; i < S::NLA; ++i)
      coff[i] = (uint32_t)token((i * S::NW + wave) * 8 + crow) * (uint32_t)(GATEUP ? Kdim : 2 * Kdim) + (uint32_t)cchunk * 16u;
#pragma unroll
    for (int i = 0; i < S::NLB; ++i) {
      if (GATEUP)        // copies of 8 rows; the second half of the rows: the up branch
        coff[S::NLA + i] = (uint32_t)column(((i & 1) * S::NW + wave) * 8 + crow) * (uint32_t)Kdim + (uint32_t)cchunk * 16u;
      else               // of 16 rows: row lane/4, slot lane%4 holding chunk slot xor (row/4)%4
        coff[S::NLA + i] = (uint32_t)column((i * S::NW + wave) * 16 + (lane >> 2)) * (uint32_t)Kdim + (uint32_t)((lane & 3) ^ ((lane >> 4) & 3)) * 16u;
    }
    const int sgrp = wave % (S::SROWS / 64);     // 64 rows of scales (waves past the last group copy one a second time)
    if (GATEUP && sgrp < BM / 64) {
      Sg = a.As;
      soff = (uint32_t)token(sgrp * 64 + lane) * (uint32_t)kb32;
    } else {
      const int w = sgrp - (GATEUP ? BM / 64 : 0);
      Sg = (GATEUP && w >= 2 ? a.B1s : a.B0s) + wrow * kb32;
      soff = (uint32_t)column((GATEUP ? w & 1 : w) * 64 + lane) * (uint32_t)kb32;
    }
    krot = SINGLE && t.once ? (int)((unsigned)(eg * 5 + t.n0 / S::NOUT * 3) % (unsigned)nk) : 0;
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) {
      if (SINGLE && t.once) issue(s, s, std::true_type{}); else issue(s, s, std::false_type{});
    }
    return t;
  };

  Tile cur = next_tile();
  while (cur.valid) {
    f32x16 acc[S::NB][S::TB];
#pragma unroll
    for (int nb = 0; nb < S::NB; ++nb)
#pragma unroll
      for (int tb = 0; tb < S::TB; ++tb)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[nb][tb][i] = 0.0f;

    auto pipeline = [&](auto tbc_, auto once_) {
      constexpr int TBc = decltype(tbc_)::value;
      auto scale_of = [&](const unsigned char* sc, int row) -> uint32_t {
        const uint32_t lo = *reinterpret_cast<const uint32_t*>(sc + row * 4);
        return PAIR ? lo | *reinterpret_cast<const uint32_t*>(sc + (S::SROWS + row) * 4) << 16 : lo;
      };
      auto wrow = [&](int nb) { return (GATEUP ? nb * 128 + wn * 32 : wn * 64 + nb * 32) + r32; };
      auto trow = [&](int tb) { return (tb * S::WAVES_M + wm) * 32 + r32; };
      int st = 0;
      for (int kt = 0; kt < nk; ++kt) {
        wait_lds_reads();                         // (of stage kt - 1)
        wait_copies_but<(NS - 2) * S::NL>();      // stage kt has landed
        workgroup_barrier();                      // for everyone; and everyone has read stage kt - 1, whose buffer is free
        issue(kt + NS - 1, st == 0 ? NS - 1 : st - 1, once_);
        const unsigned char* base = smem + st * S::STAGE;
        const unsigned char* sc = base + S::TOKENS + S::WEIGHTS;
        if constexpr (GATEUP) {
          int sw[S::NB], sx[TBc];
#pragma unroll
          for (int nb = 0; nb < S::NB; ++nb) sw[nb] = (int)(scale_of(sc, BM + wrow(nb)) >> (8 * half));
#pragma unroll
          for (int tb = 0; tb < TBc; ++tb) sx[tb] = (int)(scale_of(sc, trow(tb)) >> (8 * half));
          const bool whole = !PAIR || kstep(kt) != nk - 1;
          auto half_step = [&](auto m_) {
            constexpr int m = decltype(m_)::value;
            auto chunks = [&](const unsigned char* row) {
              return mx_operand(*reinterpret_cast<const u32x4*>(row + (((4 * m + half) ^ swz) << 4)),
                                *reinterpret_cast<const u32x4*>(row + (((4 * m + 2 + half) ^ swz) << 4)));
            };
            i32x8 w[S::NB];
#pragma unroll
            for (int nb = 0; nb < S::NB; ++nb) w[nb] = chunks(base + S::TOKENS + wrow(nb) * 128);
#pragma unroll
            for (int tb = 0; tb < TBc; ++tb) {
              const i32x8 x = chunks(base + trow(tb) * 128);
#pragma unroll
              for (int nb = 0; nb < S::NB; ++nb)
                acc[nb][tb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[nb], x, acc[nb][tb], 0, 0, 2 * m, sw[nb], 2 * m, sx[tb]);
            }
          };
          half_step(std::integral_constant<int, 0>{});
          if (whole) half_step(std::integral_constant<int, 1>{});
        } else {
          uint32_t sw[S::NB];
#pragma unroll
          for (int nb = 0; nb < S::NB; ++nb) sw[nb] = scale_of(sc, wrow(nb));
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            u32x4 w[S::NB];
#pragma unroll
            for (int nb = 0; nb < S::NB; ++nb)
              w[nb] = *reinterpret_cast<const u32x4*>(base + S::TOKENS + wrow(nb) * 64 + (((2 * p + half) ^ ((lane >> 2) & 3)) << 4));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              bf16x8 wf[S::NB];
#pragma unroll
              for (int nb = 0; nb < S::NB; ++nb) wf[nb] = mx_to_bf16(w[nb][2 * j], w[nb][2 * j + 1], (int)((sw[nb] >> (8 * p)) & 255u));
#pragma unroll
              for (int tb = 0; tb < TBc; ++tb) {
                const bf16x8 x = as_bf16x8(*reinterpret_cast<const u32x4*>(base + trow(tb) * 128 + (((4 * p + 2 * half + j) ^ swz) << 4)));
#pragma unroll
                for (int nb = 0; nb < S::NB; ++nb)
                  acc[nb][tb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[nb], x, acc[nb][tb], 0, 0, 0);
              }
            }
          }
        }
        st = st + 1 == NS ? 0 : st + 1;
      }
      wait_lds_reads();
      wait_copies_but<0>();      // the repeated copies of the last steps: none may outlive the tile
      workgroup_barrier();       // the next tile's first copies overwrite stages that other waves may still read
    };
    auto run_pipeline = [&](auto once_) {
      switch (cur.tbv) {
        case 1: pipeline(std::integral_constant<int, 1>{}, once_); break;
        case 2: if constexpr (S::TB >= 2) pipeline(std::integral_constant<int, 2>{}, once_); break;
        case 3: if constexpr (S::TB >= 3) pipeline(std::integral_constant<int, 3>{}, once_); break;
        default: if constexpr (S::TB >= 4) pipeline(std::integral_constant<int, 4>{}, once_); break;
      }
    };
    if (SINGLE && cur.once) run_pipeline(std::true_type{}); else run_pipeline(std::false_type{});

    const Tile nxt = next_tile();      // its first copies fly while this tile is stored

    // accumulator element i of block (nb, tb): column 8 (i / 4) + 4 half + i % 4 of the block, token row lane % 32; lanes l and
    // l + 32 trade four columns each, so that each stores 16 bytes
#pragma unroll
    for (int tb = 0; tb < S::TB; ++tb) {
      const int m = cur.row0 + (tb * S::WAVES_M + wm) * 32 + r32;
      if (m < cur.rowEnd) {
        bf16_t* const out = a.C + (size_t)m * N;
#pragma unroll
        for (int nb = 0; nb < (GATEUP ? 1 : S::NB); ++nb) {
          const int n = cur.n0 + (GATEUP ? wn * 32 : wn * 64 + nb * 32);
          if (n < N) {           // (N is whole blocks of 32)
#pragma unroll
            for (int q = 0; q < 4; q += 2) {
              float v[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float g = acc[nb][tb][4 * q + i];
                v[i] = GATEUP ? __fdividef(g, 1.0f + __expf(-g)) * acc[S::NB - 1][tb][4 * q + i] : g;
              }
              uint32_t ox = pack_bf16x2(v[0], v[1]), oy = pack_bf16x2(v[2], v[3]);
              uint32_t oz = pack_bf16x2(v[4], v[5]), ow = pack_bf16x2(v[6], v[7]);
              trade_halves(ox, oz);
              trade_halves(oy, ow);
              *reinterpret_cast<u32x4*>(out + n + 8 * (q + half)) = u32x4{ox, oy, oz, ow};
            }
          }
        }
      }
    }
    cur = nxt;
  }
}

int num_cus() {
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 256;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) return 256;
  return n;
}

template <int BM, bool GATEUP, int NS, bool PAIR, bool SINGLE>
int launch_tile_mx_t(const MxArgs& a, hipStream_t st) {
  using S = TileMxShape<BM, GATEUP, NS, PAIR>;
  auto kern = expert_tile_mx_kernel<BM, GATEUP, NS, PAIR, SINGLE>;
  constexpr int lds = NS * S::STAGE;
  static std::atomic<uint64_t> lds_raised{0};
  const int nexp = a.hi - a.lo;
  if (nexp > TILE_MX_EMAX) return -2;
  if (raise_lds_limit((const void*)kern, lds, lds_raised) != 0) return -4;
  const long NT = (a.N + S::NOUT - 1) / S::NOUT;
  const long bound = (((long)a.rows_total / BM + nexp + S::GM - 1) / S::GM) * S::GM * NT;
  const int grid = (int)std::min(bound, (long)num_cus());      // as many workgroups as are resident at once
  if (grid <= 0) return 0;
  hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * S::NW), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : -4;
}

template <int BM, bool GATEUP, int NS, bool SINGLE>
int launch_tile_mx_any(const MxArgs& a, hipStream_t st) {
  if constexpr (GATEUP) {
    if (a.Kdim % 128 != 0) return launch_tile_mx_t<BM, true, NS, true, SINGLE>(a, st);
  }
  return launch_tile_mx_t<BM, GATEUP, NS, false, SINGLE>(a, st);
}

// Tile height from the layer-wide mean (never from the block bounds).
int tile_height(const MxArgs& a) {
  const double m = a.mean_rows + 1.5 * sqrt((double)a.mean_rows);
  return m <= 64.0 ? 64 : m <= 128.0 ? 128 : 256;
}

}  // namespace

int launch_tile_mx_gateup(const MxArgs& a, hipStream_t st) {
  switch (tile_height(a)) {
    case 64: return launch_tile_mx_any<64, true, 3, true>(a, st);
    case 128: return launch_tile_mx_any<128, true, 3, true>(a, st);
    default: return launch_tile_mx_any<256, true, 2, false>(a, st);
  }
}
int launch_tile_mx_down(const MxArgs& a, hipStream_t st) {
  switch (tile_height(a)) {
    case 64: return launch_tile_mx_any<64, false, 5, true>(a, st);
    case 128: return launch_tile_mx_any<128, false, 4, true>(a, st);
    default: return launch_tile_mx_any<256, false, 3, false>(a, st);
  }
}

}  // namespace moe
