// Expert blocks on 8-bit weights in MFMA tiles: for experts with many rows.
//
//   gate/up : h[r, n]  = bf16( silu(<A[r,:], Wg[e][n,:]>) * <A[r,:], Wu[e][n,:]> )     rows and weights in 8 bits
//   down    : Yp[r, n] = bf16( <h[r,:], Wd[e][n,:]> )                                  bf16 rows, 8-bit weights
//
// A tile is up to 256 token rows of one expert by 256 weight rows (gate/up: 128 gate rows and the matching 128 up rows), eight
// waves as 2 x 4, each on half of the token rows by 64 weight rows (a gate block of 32 and its up block).  Its height is whole
// blocks of 64 rows.  (Tiles of at most 128 rows, with as many stages, were up to 6 % faster for experts of 50 to 120 rows, and
// far slower for more.)
//
// The kernel is persistent: every wave forms the tiles of the experts in registers from the row bounds on the device and walks
// tile numbers with a fixed stride; XCDs take runs of neighbouring tiles.  The numbers go from the highest tiles to the lowest,
// so every workgroup gets as many of each height as the others but for one, and every other XCD walks backwards, so that high
// tiles (bound by the matrix cores) and low ones (by the weights' bytes) run side by side.  With the experts in order and those
// of few rows strewn in, some workgroups had half again as much as others: 4096 tokens drawn by rank (E 60, H 2048, I 1408)
// 173 + 152 us, this way 162 + 137; 2000 such tokens (E 128, H 1024, I 768) 66 + 72, 60 + 60.  With many rows everywhere the
// order by expert was the better one, by the weights that an expert's last tile shares with its others: 16 384 tokens
// 440 + 380 us, 463 + 381.  (Builds that differed in the order alone, means of 20 passes on a card not yet warm.)
//
// K steps of 128 (gate/up) or 64 (down: a bf16 row has as many bytes) through a ring of LDS stages filled by asynchronous
// copies, more of them the lower the tile, a row's 16-byte chunks xor-swizzled against bank conflicts; one barrier per step.
// Scales come 16 bytes of a row at a time, those of 4 (gate/up) or 8 steps, into two buffers of their own: every row is another
// cache line, and fetched step by step they cost as many line requests as the rows themselves (one expert of 16 384 rows,
// H 8192, I 4096, gate/up: 1004 us, this way 916, without any scales 872).
//
// Gate/up multiplies with 32x32x64 on 8-bit values: a lane holds of row lane % 32 the chunks 4m + h and 4m + 2 + h of the
// step's half m (h = lane / 32) and gives the scale of block 2m + h: the row's slot, shifted by h bytes, and a byte select.
// Down turns weights into bf16 on their way from LDS to the matrix cores, exactly, 16 neighbours per lane, for two
// 32x32x16 steps; the hidden rows are read in that order of K.  The conversions (32 per wave and step of 1024 MFMA clocks)
// run beside the other wave's matrix instructions.
//
// Rows past the end of an expert repeat its last row and are not stored; 64-row blocks of nothing but such rows are neither
// copied nor multiplied.  Weights are copied without a read-once hint: down reads a 128-byte line in two steps, and a hinted
// line was fetched twice (60 experts of 64 rows, H 2048, I 1408: 66 us with it, 55 without).  A row's bits do not depend on the
// tile's height.
//
// Measured: one expert of 16 384 rows, H 8192, I 4096: gate/up 895 us, 2.46 PFLOP/s, down 805, 1.37.  16 384 tokens on 60
// experts, H 2048, I 1408: 427 + 369 us, 4096 drawn by rank 154 + 130, the 2000 of E 128 73 + 65 (medians of 40 passes on a warm
// card).  What is lost against the former's rates are the first and last steps of tiles of 16 and 22 steps, the sigmoid and the
// stores (65 us of gate/up), and 5 % to workgroups that wait for the last ones.  Gate/up runs at 1.8 GHz, the card's power limit, so
// fewer waits alone make it no faster: another barrier per step that let copies start half a step earlier changed nothing.
#include <algorithm>
#include "fold.h"
#include "mx.h"

namespace moe {
namespace {

constexpr int TILE_MX_EMAX = 256;

template <bool GATEUP, bool TAIL>
struct TileMxShape {
  static constexpr int BM = 256, BN = 256, WAVES_M = 2, WAVES_N = 4, NW = 8;
  static constexpr int TB = BM / 64, NB = 2;                // 32-row blocks of a wave: tokens, weights
  static constexpr int NOUT = GATEUP ? BN / 2 : BN;         // output columns of a tile
  static constexpr int BK = GATEUP ? 128 : 64;              // K values per step
  static constexpr int WROWB = GATEUP ? 128 : 64;           // bytes per staged weight row (token rows: 128)
  static constexpr int SROWS = GATEUP ? BM + BN : BN;       // rows with scales
  static constexpr int SB = GATEUP ? 4 : 2, GS = 16 / SB;   // scale bytes per row and step, steps per group of 16 bytes
  static constexpr int SCALES = SROWS * 16;                 // a group; two of them lie in front of the stages
  // copies of 1 KB per wave and stage: 64 token rows each, weight rows (and, once per group, scales of 64 rows)
  static constexpr int NLA = TB, NLB = GATEUP ? 4 : 2;
  // for a tile of 64 h rows: bytes of a stage's tokens and of a stage, and how many stages fit
  static constexpr int tokens(int h) { return h * 8192; }
  static constexpr int stage(int h) { return tokens(h) + BN * WROWB; }
  static constexpr int ring(int h) { return std::min(GS, (160 * 1024 - 2 * SCALES) / stage(h)); }
  static constexpr int lds() {
    int most = 0;
    for (int h = 1; h <= TB; ++h) most = std::max(most, ring(h) * stage(h));
    return 2 * SCALES + most;
  }
  static constexpr int GM = 4;                              // token tiles per locality group of the walk
  static_assert(GATEUP || !TAIL, "the down projection's steps are half as long");
  static_assert(ring(TB) >= 2 && ring(1) * (1 + NLB) < 60 && ring(TB) * (TB + NLB) < 60 && SROWS / 64 <= NW,
                "two stages at least, the wait counter, a copy of scales per wave");
};
constexpr int TILE_MX_MIN_K = 512;       // a row has 16 scale bytes

template <int FROM, int TO, class F>
__device__ __forceinline__ void for_range(F&& f) {
  if constexpr (FROM < TO) {
    f(number<FROM>{});
    for_range<FROM + 1, TO>(f);
  }
}

template <bool GATEUP, bool TAIL>
__global__ __launch_bounds__(512, 2) void expert_tile_mx_kernel(MxArgs a) {
  using S = TileMxShape<GATEUP, TAIL>;
  constexpr int BM = S::BM;
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / S::WAVES_N, wn = wave % S::WAVES_N;
  const int nexp = a.hi - a.lo;

  // Tiles by their height in blocks of 64 rows, 1 .. TB: of every expert the whole ones, and what is left over.  Four experts per
  // lane: rows [rb, re), the place of the first whole tile among those of height TB, of the rest among those of its height.
  int rb[4], re[4], whole[4], rest[4], total[S::TB];
  auto whole_tiles = [&](int i) { return (re[i] - rb[i]) / BM; };
  auto rest_height = [&](int i) { return ((re[i] - rb[i]) % BM + 63) >> 6; };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = lane * 4 + i;
    rb[i] = e < nexp ? a.offsets[a.lo + e] : 0;
    re[i] = max(rb[i], e < nexp ? a.offsets[a.lo + e + 1] : 0);
    whole[i] = rest[i] = 0;
  }
#pragma unroll
  for (int h = 1; h <= S::TB; ++h) {
    int n[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += n[i] = (h == S::TB ? whole_tiles(i) : 0) + (rest_height(i) == h ? 1 : 0);
    const int upto = wave_scan(sum);
    total[h - 1] = __builtin_amdgcn_readlane(upto, 63);
    int at = upto - sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (h == S::TB) whole[i] = at;
      else rest[i] = rest_height(i) == h ? at : rest[i];
      at += n[i];
    }
  }
  const int N = a.N, Kdim = a.Kdim, kb32 = Kdim / MX;
  const int NT = (N + S::NOUT - 1) / S::NOUT;
  const int nk = (Kdim + S::BK - 1) / S::BK;
  int Lend = 0;
#pragma unroll
  for (int h = 0; h < S::TB; ++h) Lend += total[h] * NT;

  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int crow = lane >> 3, cchunk = (lane & 7) ^ crow;   // copies of 128-byte rows: row lane/8, slot lane%8 holding chunk slot xor row%8
  const int r32 = lane & 31, half = lane >> 5, swz = lane & 7;
  const int sgrp = wave % (S::SROWS / 64);                  // 64 rows of scales (waves past the last group have none)
  const uint32_t tail_back = GATEUP && cchunk >= 4 ? 64u : 0u;

  const int G = gridDim.x;
  const bool xcd_walk = (G % 8) == 0;
  const int slot = xcd_walk ? (int)(blockIdx.x >> 3) : 0;
  const int run = xcd_walk ? max(1, min(G >> 3, (Lend + 7) >> 3)) : 1;
  if (xcd_walk && slot >= run) return;
  // Rounds of `step` tiles, one for every workgroup; the last, not a whole one, begins at the workgroups that had the lower tiles
  // of the rounds before.
  const int step = xcd_walk ? 8 * run : G, mine = xcd_walk ? (int)(blockIdx.x & 7) * run + slot : (int)blockIdx.x;
  const int rounds = (Lend + step - 1) / step;
  const bool back = xcd_walk && (blockIdx.x & 1) != 0;      // half of the XCDs begin with the low tiles

  struct Tile { int row0, rowEnd, eg, rows, tbv, n0; bool valid; };
  const uint8_t *Ag = nullptr, *Bg0 = nullptr, *Bg1 = nullptr, *Sg = nullptr;
  uint32_t coff[S::NLA + S::NLB], soff = 0;     // byte offsets of this lane's parts of a stage's copies, at K step 0
  // copies [FROM, TO) of K step k into stage buffer st of a tile of TBc * 64 rows: its token rows, then the weights
  auto issue_step = [&](auto tbc_, int k, int st, auto from_, auto to_) {
    constexpr int TBc = decltype(tbc_)::value;
    const uint32_t l = lds0 + (uint32_t)(2 * S::SCALES + wave * 1024) + (uint32_t)st * S::stage(TBc);
    const uint32_t back = TAIL && k == nk - 1 ? tail_back : 0u;     // the missing half from the half that is there
    for_range<decltype(from_)::value, decltype(to_)::value>([&](auto i_) {
      constexpr int i = decltype(i_)::value, w = i - TBc;
      if constexpr (w < 0) copy_to_lds_16(Ag + (size_t)k * 128, coff[i] - back, l + (uint32_t)i * 8192u);
      else copy_to_lds_16((GATEUP && w >= 2 ? Bg1 : Bg0) + (size_t)k * S::WROWB, coff[S::NLA + w] - back, l + (uint32_t)(S::tokens(TBc) + w * 8192));
    });
  };
  // of K step kt; past the end the last step again: the wait counts stay constant
  auto issue = [&](auto tbc_, int kt, int st, auto from_, auto to_) { issue_step(tbc_, min(kt, nk - 1), st, from_, to_); };
  // Scales: 16 bytes of a row are GS steps.  The last group of a row that is not whole groups starts earlier instead, so that it
  // ends with the row.
  auto group_start = [&](int k) { return min(k / S::GS * 16, kb32 - 16); };
  int group_in = 0, group_out = 0;       // the buffers of the next group to be requested, and of the one that is read
  // before the copies of K step kt the scales, if a group begins there.  (The copy is not counted in the waits, which makes them
  // wait for one copy more than they must.)
  auto issue_scales = [&](int kt) {
    const int k = min(kt, nk - 1);
    if (k % S::GS == 0 && kt < nk) {
      if (wave < S::SROWS / 64)
        copy_to_lds_16(Sg + group_start(k), soff, lds0 + (uint32_t)(group_in * S::SCALES) + (uint32_t)wave * 1024u);
      group_in ^= 1;
    }
  };

  int it = 0;
  // The next tile of this workgroup and, in gathered[], the token rows that this lane copies of it (requested while the current
  // tile is multiplied: its first copies then wait for nothing).
  int gathered[S::NLA + 1];
  auto find_tile = [&]() -> Tile {
    Tile t{};
    int at, h = S::TB;
    do {
      if (it == rounds) return t;
      const int r = back ? rounds - 1 - it : it;
      at = r * step + (r == rounds - 1 ? step - 1 - mine : mine);
      ++it;
    } while (at >= Lend);
    int tiles = total[S::TB - 1];
#pragma unroll
    for (int i = S::TB - 1; i >= 1; --i)
      if (h == i + 1 && at >= tiles * NT) {
        at -= tiles * NT;
        h = i;
        tiles = total[i - 1];
      }
    // groups of GM tiles of token rows go through the columns together
    const int g0 = at / (S::GM * NT) * S::GM, size = min(S::GM, tiles - g0);
    const int rem = at - g0 * NT, nt = rem / size, mrow = g0 + rem - nt * size;
    t.valid = true;
    int slot_of = 0, r0 = 0, r1 = 0;
    unsigned long long found = 0ull;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = whole_tiles(i), low = rest_height(i);
      const bool mine = h == S::TB ? mrow >= whole[i] && mrow < whole[i] + n + (low == S::TB ? 1 : 0) : low == h && mrow == rest[i];
      found |= __ballot(mine);
      slot_of = mine ? i : slot_of;
      r0 = mine ? rb[i] + (h == S::TB ? mrow - whole[i] : n) * BM : r0;
      r1 = mine ? re[i] : r1;
    }
    const int owner = __builtin_ctzll(found);
    t.eg = a.lo + owner * 4 + __builtin_amdgcn_readlane(slot_of, owner);
    t.row0 = __builtin_amdgcn_readlane(r0, owner);
    t.rowEnd = __builtin_amdgcn_readlane(r1, owner);
    t.rows = min(BM, t.rowEnd - t.row0);
    t.tbv = (t.rows + 63) >> 6;
    t.n0 = nt * S::NOUT;
    if (GATEUP && a.gather != nullptr) {
#pragma unroll
      for (int i = 0; i < S::NLA; ++i) gathered[i] = a.gather[t.row0 + min((i * S::NW + wave) * 8 + crow, t.rows - 1)];
      gathered[S::NLA] = a.gather[t.row0 + min(sgrp * 64 + lane, t.rows - 1)];
    }
    return t;
  };
  auto request_tile = [&](const Tile& t) {
    if (!t.valid) return;
    // row r of the tile, the i-th this lane copies
    auto token = [&](int r, int i) -> int { return GATEUP && a.gather != nullptr ? gathered[i] / a.gather_div : t.row0 + min(r, t.rows - 1); };
    auto column = [&](int r) { return min(t.n0 + r, N - 1); };
    const int eg = t.eg;
    Ag = a.A;
    const size_t wrow = (size_t)eg * N;
    Bg0 = a.B0 + wrow * Kdim;
    Bg1 = GATEUP ? a.B1 + wrow * Kdim : nullptr;
#pragma unroll
    for (int i = 0; i < S::NLA; ++i)
      coff[i] = (uint32_t)token((i * S::NW + wave) * 8 + crow, i) * (uint32_t)(GATEUP ? Kdim : 2 * Kdim) + (uint32_t)cchunk * 16u;
#pragma unroll
    for (int i = 0; i < S::NLB; ++i) {
      if (GATEUP)        // copies of 8 rows; the second half of the rows: the up branch
        coff[S::NLA + i] = (uint32_t)column(((i & 1) * S::NW + wave) * 8 + crow) * (uint32_t)Kdim + (uint32_t)cchunk * 16u;
      else               // of 16 rows: row lane/4, slot lane%4 holding chunk slot xor (row/4)%4
        coff[S::NLA + i] = (uint32_t)column((i * S::NW + wave) * 16 + (lane >> 2)) * (uint32_t)Kdim + (uint32_t)((lane & 3) ^ ((lane >> 4) & 3)) * 16u;
    }
    if (GATEUP && sgrp < BM / 64) {
      Sg = a.As;
      soff = (uint32_t)token(sgrp * 64 + lane, S::NLA) * (uint32_t)kb32;
    } else {
      const int w = sgrp - (GATEUP ? BM / 64 : 0);
      Sg = (GATEUP && w >= 2 ? a.B1s : a.B0s) + wrow * kb32;
      soff = (uint32_t)column((GATEUP ? w & 1 : w) * 64 + lane) * (uint32_t)kb32;
    }
    for_range<1, S::TB + 1>([&](auto h_) {
      constexpr int h = decltype(h_)::value;
      if (t.tbv == h) {
        for (int st = 0; st < S::ring(h); ++st) {
          issue_scales(st);
          issue(h_, st, st, number<0>{}, number<h + S::NLB>{});
        }
      }
    });
  };

  Tile cur = find_tile();
  request_tile(cur);
  while (cur.valid) {
    const Tile nxt = find_tile();
    f32x16 acc[S::NB][S::TB];
#pragma unroll
    for (int nb = 0; nb < S::NB; ++nb)
#pragma unroll
      for (int tb = 0; tb < S::TB; ++tb)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[nb][tb][i] = 0.0f;

    // Software pipeline.  All NS stages of the tile have been requested (request_tile).  A step is cut into slots of matrix
    // instructions; a slot's operands are read from LDS during the slot before, those of a step's first slot during the last slot of
    // the step before, behind the barrier that publishes the step's stage.  That barrier also says that everybody has the step
    // before it in registers, so its buffer takes the copies of the stage NS steps ahead: a part in that slot, the rest in the
    // first two slots of the next step (at the first step they repeat copies of the prologue: the same bytes to the same place).
    auto pipeline = [&](auto tbc_) {
      constexpr int TBc = decltype(tbc_)::value;
      constexpr int SLOTS = GATEUP ? 2 * TBc : 4;
      constexpr int NS = S::ring(TBc), STAGE = S::stage(TBc), TOKENS = S::tokens(TBc), NL = TBc + S::NLB;      // (NL: copies per wave and stage)
      const unsigned char* const stages = smem + 2 * S::SCALES;
      constexpr int PART0 = NL - 2 * (NL / 3), PART1 = SLOTS > 2 ? PART0 + NL / 3 : NL;
      auto wrow = [&](int nb) { return (GATEUP ? nb * 128 + wn * 32 : wn * 64 + nb * 32) + r32; };
      auto trow = [&](int tb) { return (tb * S::WAVES_M + wm) * 32 + r32; };
      auto slot_copies = [&](auto s_, int kt, int st) {
        constexpr int s = decltype(s_)::value;
        const int before = st == 0 ? NS - 1 : st - 1;
        if constexpr (s == SLOTS - 1) issue(tbc_, kt + NS, st, number<0>{}, number<PART0>{});
        if constexpr (s == 0) issue(tbc_, kt - 1 + NS, before, number<PART0>{}, number<PART1>{});
        if constexpr (s == 1 && SLOTS > 2) issue(tbc_, kt - 1 + NS, before, number<PART1>{}, number<NL>{});
      };
      auto publish = [&]() {                      // before a step's last slot
        wait_lds_reads();
        wait_copies_but<(NS - 2) * NL>();      // the next stage has landed
        workgroup_barrier();
        __builtin_amdgcn_sched_barrier(0);
      };
      // at the top of a step: the scales of the stage requested next, and where those of the next step (byte `scale_at` of each
      // row's 16, in LDS at `scales`) will be
      const unsigned char* scales = smem + group_out * S::SCALES;
      int scale_at = -group_start(0);
      auto scales_top = [&](int kt) {
        issue_scales(kt + NS);
        const int k = min(kt + 1, nk - 1);
        if (kt + 1 < nk && k % S::GS == 0) group_out ^= 1;
        scales = smem + group_out * S::SCALES;
        scale_at = S::SB * k - group_start(k);
      };
      wait_copies_but<(NS - 1) * NL>();
      workgroup_barrier();
      int st = 0;
      if constexpr (GATEUP) {
        u32x4 w[2][S::NB][2], x[2][2];            // weights of the step's two halves; token blocks of this slot and the next
        uint32_t sw[S::NB], sx[TBc];              // scale slots, shifted to the lane's block
        auto read_row = [&](u32x4 (&v)[2], const unsigned char* row, auto m_) {
          constexpr int m = decltype(m_)::value;
          v[0] = *reinterpret_cast<const u32x4*>(row + (((4 * m + half) ^ swz) << 4));
          v[1] = *reinterpret_cast<const u32x4*>(row + (((4 * m + 2 + half) ^ swz) << 4));
        };
        auto read_w = [&](const unsigned char* base, auto m_) {
#pragma unroll
          for (int nb = 0; nb < S::NB; ++nb) read_row(w[decltype(m_)::value][nb], base + TOKENS + wrow(nb) * 128, m_);
        };
        auto read_x = [&](const unsigned char* base, auto s_) {
          constexpr int s = decltype(s_)::value;
          read_row(x[s & 1], base + trow(s % TBc) * 128, number<s / TBc>{});
        };
        auto read_scales = [&]() {
          const unsigned char* sc = scales + (scale_at & ~3);
          const uint32_t scale_mask = scale_at == 14 ? 0xffffu : ~0u;
          auto one = [&](int row) -> uint32_t {
            const uint32_t lo = *reinterpret_cast<const uint32_t*>(sc + row * 16);
            if constexpr (!TAIL) return lo >> (8 * half);
            // (in the last group of a row of an odd number of pairs the step's bytes begin at an odd pair)
            return __builtin_amdgcn_alignbit(*reinterpret_cast<const uint32_t*>(sc + row * 16 + 4), lo, (scale_at & 2) * 8) >> (8 * half) & scale_mask;
          };
#pragma unroll
          for (int nb = 0; nb < S::NB; ++nb) sw[nb] = one(BM + wrow(nb));
#pragma unroll
          for (int tb = 0; tb < TBc; ++tb) sx[tb] = one(trow(tb));
        };
        read_scales();
        read_w(stages, number<0>{});
        read_x(stages, number<0>{});
        for (int kt = 0; kt < nk; ++kt) {
          const unsigned char* base = stages + st * STAGE;
          const int st1 = st + 1 == NS ? 0 : st + 1;
          scales_top(kt);
          const uint32_t there = !TAIL || kt != nk - 1 ? ~0u : 0u;      // a step's second half
          for_range<0, SLOTS>([&](auto s_) {
            constexpr int s = decltype(s_)::value, m = s / TBc, tb = s % TBc;
            uint32_t sw0[S::NB], sx0 = sx[tb];
#pragma unroll
            for (int nb = 0; nb < S::NB; ++nb) sw0[nb] = sw[nb];
            if constexpr (s == SLOTS - 1) publish();
            auto multiply = [&](int nb) {
              if constexpr (TAIL && m == 1 && tb == 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  w[1][nb][0][i] &= there;
                  w[1][nb][1][i] &= there;
                }
              }
              acc[nb][tb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_operand(w[m][nb][0], w[m][nb][1]), mx_operand(x[s & 1][0], x[s & 1][1]),
                                                                            acc[nb][tb], 0, 0, 2 * m, (int)sw0[nb], 2 * m, (int)sx0);
            };
            multiply(0);
            __builtin_amdgcn_sched_barrier(0x6);
            if constexpr (s < SLOTS - 1) {
              read_x(base, number<s + 1>{});
              if constexpr (s == (TBc > 1 ? TBc - 2 : 0)) read_w(base, number<1>{});
            } else {
              const unsigned char* next = stages + st1 * STAGE;
              read_x(next, number<0>{});
              read_w(next, number<0>{});
              read_scales();
            }
            slot_copies(s_, kt, st);
            __builtin_amdgcn_sched_barrier(0x6);
            multiply(1);
            __builtin_amdgcn_sched_barrier(0x6);
          });
          st = st1;
        }
      } else {
        u32x4 raw[2][S::NB];                      // weights as they are, of the step's two halves
        bf16x8 wf[2][S::NB], x[2][TBc];           // operands of this slot and the next
        uint32_t sw[S::NB];
        auto read_raw = [&](const unsigned char* base, auto p_) {
          constexpr int p = decltype(p_)::value;
#pragma unroll
          for (int nb = 0; nb < S::NB; ++nb)
            raw[p][nb] = *reinterpret_cast<const u32x4*>(base + TOKENS + wrow(nb) * 64 + (((2 * p + half) ^ ((lane >> 2) & 3)) << 4));
        };
        auto read_scales = [&]() {
#pragma unroll
          for (int nb = 0; nb < S::NB; ++nb) sw[nb] = *reinterpret_cast<const uint16_t*>(scales + scale_at + wrow(nb) * 16);
        };
        auto read_x1 = [&](const unsigned char* base, auto s_, int tb) {
          constexpr int s = decltype(s_)::value;
          x[s & 1][tb] = as_bf16x8(*reinterpret_cast<const u32x4*>(base + trow(tb) * 128 + (((4 * (s >> 1) + 2 * half + (s & 1)) ^ swz) << 4)));
        };
        auto convert = [&](auto s_) {
          constexpr int s = decltype(s_)::value, p = s >> 1, j = s & 1;
#pragma unroll
          for (int nb = 0; nb < S::NB; ++nb) wf[j][nb] = mx_to_bf16(raw[p][nb][2 * j], raw[p][nb][2 * j + 1], (int)((sw[nb] >> (8 * p)) & 255u));
        };
        read_scales();
        read_raw(stages, number<0>{});
#pragma unroll
        for (int tb = 0; tb < TBc; ++tb) read_x1(stages, number<0>{}, tb);
        convert(number<0>{});
        for (int kt = 0; kt < nk; ++kt) {
          const unsigned char* base = stages + st * STAGE;
          const int st1 = st + 1 == NS ? 0 : st + 1;
          scales_top(kt);
          for_range<0, SLOTS>([&](auto s_) {
            constexpr int s = decltype(s_)::value;
            if constexpr (s == SLOTS - 1) publish();
            const unsigned char* from = s < SLOTS - 1 ? base : stages + st1 * STAGE;
            constexpr int NM = S::NB * TBc;       // matrix instructions of the slot: behind the first ones the reads, then the copies
#pragma unroll
            for (int j = 0; j < NM; ++j) {
              acc[j % S::NB][j / S::NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[s & 1][j % S::NB], x[s & 1][j / S::NB], acc[j % S::NB][j / S::NB], 0, 0, 0);
              if (j == 0) {
                if constexpr (s == 0) read_raw(base, number<1>{});
                if constexpr (s == SLOTS - 1) {
                  read_raw(from, number<0>{});
                  read_scales();
                }
              }
              if (j < TBc) read_x1(from, number<(s + 1) % SLOTS>{}, j);
              if (j == (TBc < NM - 1 ? TBc : NM - 1)) slot_copies(s_, kt, st);
              __builtin_amdgcn_sched_barrier(0x6);
            }
            convert(number<(s + 1) % SLOTS>{});
          });
          st = st1;
        }
      }
      group_out ^= 1;      // (the next tile begins a group)
      wait_lds_reads();
      wait_copies_but<0>();      // the repeated copies of the last steps: none may outlive the tile
      workgroup_barrier();       // the next tile's first copies overwrite stages that other waves may still read
    };
    switch (cur.tbv) {
      case 1: pipeline(number<1>{}); break;
      case 2: if constexpr (S::TB >= 2) pipeline(number<2>{}); break;
      case 3: if constexpr (S::TB >= 3) pipeline(number<3>{}); break;
      default: if constexpr (S::TB >= 4) pipeline(number<4>{}); break;
    }

    request_tile(nxt);      // its first copies fly while this tile is stored

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
                v[i] = GATEUP ? silu_times(g, acc[S::NB - 1][tb][4 * q + i]) : g;
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

template <bool GATEUP, bool TAIL>
int launch_tile_mx_t(const MxArgs& a, hipStream_t st) {
  using S = TileMxShape<GATEUP, TAIL>;
  auto kern = expert_tile_mx_kernel<GATEUP, TAIL>;
  constexpr int lds = S::lds();
  if (a.Kdim < TILE_MX_MIN_K) return -2;
  static std::atomic<uint64_t> lds_raised{0};
  const int nexp = a.hi - a.lo;
  if (nexp > TILE_MX_EMAX) return -2;
  if (raise_lds_limit((const void*)kern, lds, lds_raised) != 0) return -4;
  const long NT = (a.N + S::NOUT - 1) / S::NOUT;
  const long bound = (((long)a.rows_total / S::BM + nexp + S::GM - 1) / S::GM) * S::GM * NT;
  const int grid = (int)std::min(bound, (long)num_cus());      // as many workgroups as are resident at once
  if (grid <= 0) return 0;
  hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * S::NW), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : -4;
}

}  // namespace

int launch_tile_mx_gateup(const MxArgs& a, hipStream_t st) {
  return a.Kdim % 128 != 0 ? launch_tile_mx_t<true, true>(a, st) : launch_tile_mx_t<true, false>(a, st);
}
int launch_tile_mx_down(const MxArgs& a, hipStream_t st) { return launch_tile_mx_t<false, false>(a, st); }

}  // namespace moe
