// Gating by scores: softmax or sigmoid of the router logits, an optional bias that takes part in the choice alone, experts
// in groups of which only the best are considered, top-k, renormalised and scaled weights.
//
//   l[t,e] = <x[t,:], Wr[e,:]>   in the order of additions of route.hip, so both calls choose from the same logits
//   s[t,e] = softmax_e(l) or sigmoid(l), formed in 64 bits and rounded once to fp32 where the choice depends on it;   c = s + balance
//   value of a group = its largest c, or the sum of its two largest;  the top_groups best groups are kept
//   ids = the K largest c among the kept groups' experts;  w = s[id] (over their sum + 1e-20 with renorm) * scale
// NaN orders below everything, so the ids are K different experts whatever the rows hold.
//
// What bounds it: the products.  In the defined order they are one vector multiply-add each; on the matrix cores they are almost free,
// but add up in another order, and ids must not depend on that.  So: logits from the matrix cores with a bound of their
// error, the choice from those; and where two candidates lie closer than the bound allows, the logits of just these are formed
// again in the defined order (and their scores in 64 bits) and the choice is repeated: an id is always the definition's.
// (Weights are formed in fp32, from the logits at hand, whose last bits are either evaluation's: off by less than 32 roundings and
// what is lost in the difference to the largest logit, on top of the logits' own error.)  About one token in eighteen is looked at
// twice (256 experts in 8 groups, H 2048).
//
// Measured (H 2048): 13 tokens, 60 experts 8.6 us, 3 of them the products and 4 the choice; 301 tokens, 256 experts in 8 groups
// 28.6 us (8 products: every workgroup reads the router's 1 MB; 2.5 their sum; 7 the choice, and 9 to 10 more where near ties are
// formed again); 8192 such tokens 48.5 us (15 + 5 + 9, and up to 18); 16 384 tokens, 60 experts, sigmoid 32 us.  2000 tokens of 160
// experts in 8 groups, softmax, H 4096: 33 us, with a balance 71 (best 1) and 75 (best 2): groups that are near to each other have
// all of the token's logits formed again.
//
// The bound of the error is derived in score_margin.h from how often a term is rounded in either order, up to some 60 times
// (H 2048), and so does not rest on how large errors usually are (1.3 * 2^-24 of the magnitudes' sum).
#include "fold.h"
#include "mx.h"
#include "score_margin.h"
#include <algorithm>
#include <type_traits>

namespace moe {
namespace {

// Whole numbers that order like the values: -0 as +0, NaN as 1, below -infinity; 0 is left for "no expert"
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return v != v ? 1u : (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return k <= 1u ? __uint_as_float(0x7fc00000u) : __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ double sigmoid64(float l) { return 1.0 / (1.0 + exp(-(double)l)); }

// Folds over a row of LANES (16 or 32) lanes; every lane has the result
template <int LANES, class T, class F>
__device__ __forceinline__ T row_fold(T v, F&& f) {
  auto other = [](T x, auto ctrl) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, false));
  };
  v = f(v, other(v, std::integral_constant<int, 0xB1>{}));
  v = f(v, other(v, std::integral_constant<int, 0x4E>{}));
  v = f(v, other(v, std::integral_constant<int, 0x141>{}));
  v = f(v, other(v, std::integral_constant<int, 0x140>{}));
  if constexpr (LANES == 32) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, v);
    const auto both = __builtin_amdgcn_permlane16_swap(bits, bits, false, false);      // the even 16 lanes' value, and the odd ones'
    const uint32_t even = both[0], odd = both[1];
    v = f(__builtin_bit_cast(T, even), __builtin_bit_cast(T, odd));
  }
  return v;
}
template <int LANES>
__device__ __forceinline__ uint32_t row_max(uint32_t v) { return row_fold<LANES>(v, [](uint32_t a, uint32_t b) { return max(a, b); }); }
template <int LANES>
__device__ __forceinline__ uint32_t row_min(uint32_t v) { return row_fold<LANES>(v, [](uint32_t a, uint32_t b) { return min(a, b); }); }
template <int LANES>
__device__ __forceinline__ float row_max(float v) { return row_fold<LANES>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int LANES>
__device__ __forceinline__ float row_sum(float v) { return row_fold<LANES>(v, [](float a, float b) { return a + b; }); }

// N logits by one wave, of token rows x[n] (or one for all) and router rows w[n], in the defined order.  Four chunks of 512 at a time
// are requested before they are used.
template <int NX, int N>
__device__ __forceinline__ void defined_logits(const bf16_t* const (&x)[NX], const bf16_t* const (&w)[N], int H, int lane, float (&l)[N]) {
  static_assert(NX == 1 || NX == N, "one row for all, or one each");
  float acc[N];
#pragma unroll
  for (int n = 0; n < N; ++n) acc[n] = 0.0f;
  for (int h0 = 8 * lane; h0 < H; h0 += 2048) {
    u32x4 xv[NX][4], wv[N][4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const bool in = h0 + 512 * c < H;      // (a product of zeros leaves a sum as it is)
#pragma unroll
      for (int n = 0; n < NX; ++n) xv[n][c] = in ? *reinterpret_cast<const u32x4*>(x[n] + h0 + 512 * c) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int n = 0; n < N; ++n) wv[n][c] = in ? *reinterpret_cast<const u32x4*>(w[n] + h0 + 512 * c) : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        float xf[8], wf[8];
        widen8(xv[NX == 1 ? 0 : n][c], xf);
        widen8(wv[n][c], wf);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[n] = __builtin_fmaf(xf[i], wf[i], acc[n]);
      }
  }
#pragma unroll
  for (int n = 0; n < N; ++n) l[n] = fold_sum(acc[n]);
}

constexpr int GROUPS_MAX = 64;

// 64 / LANES tokens by one wave, one per row of LANES lanes; lane j of a row owns experts EPL j .. EPL j + EPL - 1.  What belongs to
// a token is the same in the lanes of its row.
//   t, want: the token and whether its row of results is asked for;  whole: the logits are the defined ones (in all rows);
//   s_logit: its logits in LDS (by expert; exact ones are written back);  s_bal: the balance, by expert, at most bal_most;
//   doubt: what a logit may be off by, negative if that is not known;  s_key, s_thr: EPL * LANES and 64 words of the row.
// True where the choice cannot be made without all of the token's logits in the defined order; then nothing is written.
template <int EPL, int LANES>
__device__ __forceinline__ bool choose(const RouteScored& a, int t, bool want, bool whole, float* s_logit, const float* s_bal, float bal_most,
                                       float doubt, int lane, uint32_t* s_key, float* s_thr) {
  static_assert(LANES == 16 || LANES == 32, "rows");
  const int jl = lane & (LANES - 1), row0 = lane & (64 - LANES), e0 = EPL * jl;
  const int size = a.E / a.groups;
  const uint32_t per_group = 65536u / (uint32_t)size + 1u;                   // e / size = e * per_group >> 16 for e < 256
  auto group_of = [&](int e) { return __umul24((uint32_t)e, per_group) >> 16; };
  const bool grouped = a.groups > a.top_groups;
  // softmax without extras orders like its logits
  const bool by_logit = !whole && !a.sigmoid && a.balance == nullptr && (!grouped || a.best == 1);
  const bool by_score = !a.sigmoid && !by_logit;
  auto row_any = [&](bool v) { return ((__ballot(v) >> row0) & ((1ull << LANES) - 1ull)) != 0ull; };

  // Sum over the experts, in an order that does not depend on LANES: rows of 16 lanes add what rows of 32 have in two lanes as
  // those do, one by one and then the two.
  constexpr int HALF = LANES == 16 ? EPL / 2 : EPL;
  auto sum_of = [&](const float (&v)[EPL]) {
    float part[EPL / HALF];
#pragma unroll
    for (int h = 0; h < EPL / HALF; ++h) {
      part[h] = 0.0f;
#pragma unroll
      for (int i = 0; i < HALF; ++i) part[h] += v[HALF * h + i];
    }
    return row_sum<LANES>(EPL / HALF == 2 ? part[0] + part[EPL / HALF - 1] : part[0]);
  };

  uint32_t key[EPL];         // what is compared, 0 beyond E
  float m = 0.0f;
  double z = 1.0;
  unsigned exact = whole ? ~0u : 0u;       // this lane's experts whose logit (and key) is the defined one
  bool redo = false;
  {
    float l[EPL];
#pragma unroll
    for (int i = 0; i < EPL; i += 2) {
      const float2 v = *reinterpret_cast<const float2*>(s_logit + e0 + i);
      l[i] = e0 + i < a.E ? v.x : 0.0f;
      l[i + 1] = e0 + i + 1 < a.E ? v.y : 0.0f;
    }
    float magnitudes = 0.0f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) magnitudes += fabsf(l[i]);
    if (row_any(magnitudes != 0.0f))
      redo = !whole && (doubt < 0.0f || (by_score && doubt > LOGIT_ERROR_MOST) || row_any(!(magnitudes < INFINITY)));
    else doubt = 0.0f;       // (a row of zeros: 0 in any order)
    if (!a.sigmoid) {
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < EPL; ++i) top = e0 + i < a.E ? fmaxf(top, l[i]) : top;
      m = row_max<LANES>(top);
    }
    if (whole) {             // scores in 64 bits
      if (!a.sigmoid) {
        double sum = 0.0, part = 0.0;
#pragma unroll 1
        for (int i = 0; i < EPL; ++i) {
          if (i == HALF) {
            sum = part;
            part = 0.0;
          }
          if (e0 + i < a.E) part += exp((double)s_logit[e0 + i] - (double)m);
        }
        sum += part;
#pragma unroll
        for (int w = 1; w < LANES; w <<= 1) sum += __shfl_xor(sum, w, WAVE);
        z = sum;
      }
#pragma unroll 1
      for (int i = 0; i < EPL; ++i) {
        const double v = (double)s_logit[e0 + i];
        s_key[e0 + i] = __float_as_uint((float)(a.sigmoid ? 1.0 / (1.0 + exp(-v)) : exp(v - (double)m) / z));
      }
#pragma unroll
      for (int i = 0; i < EPL; ++i) l[i] = __uint_as_float(s_key[e0 + i]);
    } else if (a.sigmoid) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) l[i] = __builtin_amdgcn_rcpf(1.0f + __expf(-l[i]));
    } else if (!by_logit) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) l[i] = e0 + i < a.E ? expf(l[i] - m) : 0.0f;
      const float sum = sum_of(l);
      z = sum;
      const float inverse = 1.0f / sum;
#pragma unroll
      for (int i = 0; i < EPL; ++i) l[i] *= inverse;
    }
    if (a.balance != nullptr) {
#pragma unroll
      for (int i = 0; i < EPL; i += 2) {
        const float2 v = *reinterpret_cast<const float2*>(s_bal + e0 + i);
        l[i] += v.x;
        l[i + 1] += v.y;
      }
    }
#pragma unroll
    for (int i = 0; i < EPL; ++i) key[i] = e0 + i < a.E ? order_key(l[i]) : 0u;
  }
  const ScoreMargin margin = a.sigmoid ? margin_of_sigmoids(doubt) : by_logit ? margin_of_logits(doubt) : margin_of_softmax(doubt, 1.0f / (float)z, bal_most);
  int my_id = 0;
  for (;;) {
    unsigned again = 0u;     // this lane's experts whose logit the choice needs exactly
    bool alike = false;      // softmax: so close, or so far below the largest, that scores may round alike
    uint32_t cur[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) cur[i] = key[i];

    if (grouped) {
      // lane j of a row takes groups j, j + LANES, ..: their two largest keys, then the best groups one by one
#pragma unroll
      for (int i = 0; i < EPL; i += 2) *reinterpret_cast<uint2*>(s_key + e0 + i) = uint2{key[i], key[i + 1]};
      __builtin_amdgcn_wave_barrier();
      constexpr int GPL = GROUPS_MAX / LANES;
      uint32_t value[GPL], left[GPL];
      float low[GPL], size_of[GPL];    // the smallest c that counts in a group's value, and how large those are
#pragma unroll
      for (int gi = 0; gi < GPL; ++gi) {
        value[gi] = left[gi] = 0u;
        low[gi] = size_of[gi] = 0.0f;
        const int g = jl + LANES * gi;
        if (LANES * gi < a.groups && g < a.groups) {
          uint32_t k1 = 0u, k2 = 0u;
          auto take = [&](uint32_t k) {
            k2 = max(k2, min(k1, k));
            k1 = max(k1, k);
          };
          if ((size & 3) == 0) {       // (each group from a place of its own on: other LDS banks)
            int at = 4 * (g % (size / 4));
#pragma unroll 4
            for (int j = 0; j < size; j += 4) {
              const u32x4 k = *reinterpret_cast<const u32x4*>(s_key + g * size + at);
              take(k.x); take(k.y); take(k.z); take(k.w);
              at = at + 4 == size ? 0 : at + 4;
            }
          } else {
            for (int j = 0; j < size; ++j) take(s_key[g * size + j]);
          }
          const float v1 = key_value(k1), v2 = key_value(k2);
          value[gi] = left[gi] = a.best == 1 ? k1 : order_key(v1 + v2);
          low[gi] = a.best == 1 ? v1 : v2;
          size_of[gi] = fabsf(v1) + (a.best == 1 ? 0.0f : fabsf(v2));
        }
      }
      auto most_left = [&]() {
        uint32_t v = left[0];
#pragma unroll
        for (int gi = 1; gi < GPL; ++gi) v = max(v, left[gi]);
        return row_max<LANES>(v);
      };
      __builtin_amdgcn_wave_barrier();
      uint32_t last = 0u;
      unsigned long long kept = 0ull;
      for (int j = 0; j < a.top_groups; ++j) {
        last = most_left();
        uint32_t g = GROUPS_MAX;
#pragma unroll
        for (int gi = GPL - 1; gi >= 0; --gi)
          if (left[gi] == last) g = jl + LANES * gi;                        // (last is not 0: more groups than are kept)
        g = row_min<LANES>(g);
        kept |= 1ull << g;
#pragma unroll
        for (int gi = 0; gi < GPL; ++gi) left[gi] = jl + LANES * gi == (int)g ? 0u : left[gi];
      }
      // the border between the last group kept and the best one left: who may be on either side of it
      const float vk = key_value(last), vn = key_value(most_left());
      bool close = false;
      float thr[GPL];
#pragma unroll
      for (int gi = 0; gi < GPL; ++gi) {
        const float v = key_value(value[gi]);
        const float moved = margin.between_groups(a.best, size_of[gi]);
        const bool in = !whole && value[gi] != 0u && size_of[gi] < INFINITY && vk - vn <= moved && v >= vk - moved && v <= vn + moved;
        thr[gi] = in ? low[gi] - moved : INFINITY;
        close |= in;
      }
      if (__any(close)) {
#pragma unroll
        for (int gi = 0; gi < GPL; ++gi) s_thr[jl + LANES * gi] = thr[gi];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          const float c = key_value(key[i]);
          if (key[i] != 0u && ((exact >> i) & 1u) == 0u && fabsf(c) < INFINITY && c >= s_thr[group_of(e0 + i)]) again |= 1u << i;
        }
        __builtin_amdgcn_wave_barrier();
      }
      if (by_logit) {        // against the best value that differs: groups with the last one's own stand in their order already
        uint32_t differs = 0u;
#pragma unroll
        for (int gi = 0; gi < GPL; ++gi) differs = left[gi] != last ? max(differs, left[gi]) : differs;
        alike = vk - key_value(row_max<LANES>(differs)) <= 2e-6f * fmaxf(1.0f, fabsf(vk)) || vk - m < -70.0f;      // (none: NaN)
      } else if (!a.sigmoid) {
        alike = close;
      }
#pragma unroll
      for (int i = 0; i < EPL; ++i) cur[i] = (kept >> group_of(e0 + i)) & 1ull ? cur[i] : 0u;
    }
    unsigned allowed = 0u;
#pragma unroll
    for (int i = 0; i < EPL; ++i) allowed |= cur[i] != 0u ? 1u << i : 0u;

    auto best_left = [&]() {
      uint32_t k = cur[0];
#pragma unroll
      for (int i = 1; i < EPL; ++i) k = max(k, cur[i]);
      return row_max<LANES>(k);
    };
    auto expert_of = [&](uint32_t k) {       // the first one left with this key
      uint32_t e = 256u;
#pragma unroll
      for (int i = EPL - 1; i >= 0; --i) e = cur[i] == k ? (uint32_t)(e0 + i) : e;
      return (int)row_min<LANES>(e);
    };
    uint32_t my_key = 0u, last_key = 0u;     // lane j < K: the j-th choice
    for (int j = 0; j < a.K; ++j) {
      const uint32_t k = last_key = best_left();
      const int e = expert_of(k);
#pragma unroll
      for (int i = 0; i < EPL; ++i) cur[i] = e == e0 + i ? 0u : cur[i];
      my_key = jl == j ? k : my_key;
      my_id = jl == j ? e : my_id;
    }
    const uint32_t border = best_left();     // the best one that is not chosen (none is left: 0)
    const float my_c = key_value(my_key), next = key_value(border);
    bool close;
    float most;
    {
      // every choice with the one after it, the last with the border (a NaN or an infinite one is what it is)
      auto following = [&](float v, float last) {
        const float w = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x101, 0xF, 0xF, false));     // row_shl 1
        return jl == a.K - 1 ? last : w;
      };
      const float after = following(my_c, next), d = my_c - after, large = fmaxf(fabsf(my_c), fabsf(after));
      const bool both = (jl < a.K - 1 || (jl == a.K - 1 && border != 0u)) && large < INFINITY;
      close = both && d <= 2.0f * margin.off(large);
      most = row_max<LANES>(fmaxf(jl < a.K && fabsf(my_c) < INFINITY ? fabsf(my_c) : 0.0f, fabsf(next) < INFINITY ? fabsf(next) : 0.0f));
      if (by_logit) {        // again the best one left whose value differs from the last choice's
        uint32_t differs = 0u;
#pragma unroll
        for (int i = 0; i < EPL; ++i) differs = cur[i] != last_key ? max(differs, cur[i]) : differs;
        const float e = my_c - following(my_c, key_value(row_max<LANES>(differs)));
        alike |= jl < a.K && ((e > 0.0f && e <= 4e-7f * fmaxf(1.0f, fabsf(my_c))) || my_c - m < -70.0f);
      } else if (!a.sigmoid) {               // between exact logits what is left is the denominator's error
        float score = my_c, score_next = next;
        if (a.balance != nullptr) {
          score -= s_bal[my_id];
          score_next -= s_bal[min(expert_of(border), a.E - 1)];
        }
        const float s_after = following(score, score_next);
        alike |= both && d <= 2.1f * doubt * fabsf(score - s_after) + 5e-7f * (large + fabsf(s_after));
      }
    }
    close = !whole && row_any(close);
    if (__any(close)) {      // whose logits lie that near to another's, at or above the border of the choice
      const float width = 2.0f * margin.off(most);
      unsigned one = 0u, two = 0u;           // experts with a chosen value, or two, that near (a chosen one's own counts)
      for (int j = 0; j <= a.K; ++j) {
        const float c = j < a.K ? __shfl(my_c, row0 + j, WAVE) : next;
        unsigned hit = 0u;
#pragma unroll
        for (int i = 0; i < EPL; ++i) hit |= fabsf(key_value(key[i]) - c) <= width ? 1u << i : 0u;
        two |= one & hit;
        one |= j < a.K ? hit : 0u;           // (the border concerns the chosen alone)
      }
      unsigned chosen = 0u;
#pragma unroll
      for (int i = 0; i < EPL; ++i) chosen |= cur[i] == 0u ? 1u << i : 0u;
      if (close) again |= (chosen & two & allowed) | (~chosen & one & allowed);
      again &= ~exact;
    }
    if (!whole && !redo) redo = !row_any(again != 0u) && row_any(alike);
    if (redo || !want) again = 0u;
    unsigned long long todo = __ballot(again != 0u);
    if (todo == 0ull) break;
    exact |= again;
    unsigned bits = 0u;
    int owner = 0;
    while (todo != 0ull || bits != 0u) {     // two logits at a time
      int at[2], slot[2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        if (bits == 0u && todo != 0ull) {
          owner = __builtin_ctzll(todo);
          todo &= todo - 1ull;
          bits = (unsigned)__builtin_amdgcn_readlane((int)again, owner);
        }
        at[n] = owner;
        slot[n] = bits != 0u ? __builtin_ctz(bits) : slot[0];                // (none left: the first one once more)
        bits &= bits - 1u;
      }
      const bf16_t *xs[2], *ws[2];
      float v[2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        xs[n] = a.x + (size_t)__builtin_amdgcn_readlane(t, at[n]) * a.H;
        ws[n] = a.Wr + (size_t)(EPL * (at[n] & (LANES - 1)) + slot[n]) * a.H;
      }
      defined_logits(xs, ws, a.H, lane, v);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int e = EPL * (at[n] & (LANES - 1)) + slot[n];
        const float score = a.sigmoid ? (float)sigmoid64(v[n]) : by_logit ? v[n] : (float)(exp((double)v[n] - (double)m) / z);
        const uint32_t k = order_key(a.balance != nullptr ? score + s_bal[e] : score);     // (of the owner's token: the owner's)
        if (lane == at[n]) {
          s_logit[e] = v[n];
#pragma unroll
          for (int q = 0; q < EPL; ++q) key[q] = q == slot[n] ? k : key[q];
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  if (by_logit) {            // the weights' denominator
    float p[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) p[i] = e0 + i < a.E ? expf(s_logit[e0 + i] - m) : 0.0f;
    z = sum_of(p);
  }
  float s = 0.0f;
  if (jl < a.K) {
    const float l = s_logit[my_id];
    s = a.sigmoid ? 1.0f / (1.0f + expf(-l)) : expf(l - m) / (float)z;
  }
  if (a.renorm) s = s / (row_sum<LANES>(s) + 1e-20f);
  if (jl < a.K && want && !redo) {
    a.ids[(size_t)t * a.K + jl] = my_id;
    a.w[(size_t)t * a.K + jl] = s * a.scale;
  }
  return redo;
}

// A workgroup of eight waves takes 16 * TT tokens and all experts (NBLK blocks of 16); each wave an eighth of K, so that every
// byte of the router and of the rows is read once per workgroup, with no barrier on the way.  16 rows by 128 bytes are two
// copies of 1 KB straight into the wave's own ring in LDS, whole lines with eight lanes side by side on a row, and come back
// as operands from there.  (Loaded as operands, 16 rows by 16 bytes per 16 lanes, they took four times as long: 0.35 us per
// block and wave, of the address unit.)  The eight partial sums meet in LDS, eight tiles at a time, and are added in the order
// of the parts: a logit's bits depend on H alone.  The squares for the error bound are summed from the same operands, weighted
// by how often their terms are rounded.
// The choice is a chain of small steps, bound by their latency: all eight waves share the tokens, 32 lanes for each of 16 (half as
// many experts per lane as with 16 lanes: 301 tokens 4 us less than with 16 lanes and half of the waves idle), 16 lanes for each of 32.
constexpr int ROUTE_WAVES = 8, ROUTE_RING = 8;                               // items of 2 KB in a wave's ring
template <int NBLK, int TT>
struct RouteShape {
  static constexpr int TOKENS = 16 * TT, EP = 16 * NBLK, LDL = EP + 4;       // logits [TOKENS][LDL]
  static constexpr int LANES = 64 * ROUTE_WAVES / TOKENS;                    // that choose for a token
  static constexpr int RINGS = ROUTE_WAVES * ROUTE_RING * 2048;              // then: parts (later keys and thresholds), logits behind them
  static constexpr int PARTS = ROUTE_WAVES * 8 * 1024, LOGITS = TOKENS * LDL * 4, NORMS = ROUTE_WAVES * 4 * (1 + TOKENS) * 4, BAL = EP * 4;
  static constexpr int LDS = RINGS + NORMS + BAL;
  static_assert(RINGS >= PARTS + LOGITS && PARTS >= TOKENS * (EP + GROUPS_MAX) * 4 && LDS <= 160 * 1024, "LDS");
};

template <int NBLK, int TT>
__global__ __launch_bounds__(64 * ROUTE_WAVES) void route_scored_kernel(RouteScored a) {
  using S = RouteShape<NBLK, TT>;
  extern __shared__ __align__(16) unsigned char smem[];
  float* const s_logit = reinterpret_cast<float*>(smem + S::PARTS);
  float* const s_wn = reinterpret_cast<float*>(smem + S::RINGS);             // [wave][g], then [TOKENS][wave][g]
  float* const s_xn = s_wn + ROUTE_WAVES * 4;
  float* const s_bal = s_xn + ROUTE_WAVES * 4 * S::TOKENS;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int t0 = blockIdx.x * S::TOKENS;
  const int H = a.H, nk = H / 64;
  const int k0 = nk * wave / ROUTE_WAVES, k1 = nk * (wave + 1) / ROUTE_WAVES;

  // A block's first expert: the last ones start early enough to have 16 rows (the overlap is formed twice, alike); with fewer
  // than 16 experts, and for the last tokens, the last row is read again.
  auto first = [&](int b) { return max(0, min(16 * b, a.E - 16)); };
  const int crow = lane >> 3, cchunk = (lane & 7) ^ crow;                    // slot lane%8 of row lane/8 holds chunk slot xor row%8
  uint32_t woff[2], xoff[TT][2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    woff[i] = (uint32_t)min(8 * i + crow, a.E - 1) * (uint32_t)H * 2u + 16u * cchunk;
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) xoff[tt][i] = (uint32_t)min(16 * tt + 8 * i + crow, a.T - 1 - t0) * (uint32_t)H * 2u + 16u * cchunk;
  }
  unsigned char* const ring = smem + wave * ROUTE_RING * 2048;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)ring;
  const bf16_t* const x0 = a.x + (size_t)t0 * H;
  constexpr int NQ = TT + NBLK;                                              // items of a K step: token tiles, then experts
  auto issue = [&](int j, int k, int slot) {                                 // item j of step k
    const unsigned char* base = reinterpret_cast<const unsigned char*>((j < TT ? x0 : a.Wr + (size_t)first(j - TT) * H) + 64 * min(k, k1 - 1));
#pragma unroll
    for (int i = 0; i < 2; ++i) copy_to_lds_16(base, j < TT ? xoff[j < TT ? j : 0][i] : woff[i], lds0 + (uint32_t)slot * 2048u + (uint32_t)i * 1024u);
  };
  auto squares = [&](u32x4 v, float s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t pair = v[i];      // (a bit cast of the element itself takes the vector's first)
      const bf16x2 p = __builtin_bit_cast(bf16x2, pair);
      s = __builtin_amdgcn_fdot2_f32_bf16(p, p, s, false);
    }
    return s;
  };
  f32x4 acc[NBLK][TT];
  float wn[NBLK], xn[TT];
#pragma unroll
  for (int b = 0; b < NBLK; ++b) {
    wn[b] = 0.0f;
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) acc[b][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
#pragma unroll
  for (int tt = 0; tt < TT; ++tt) xn[tt] = 0.0f;
  if (k0 < k1) {
    constexpr int AHEAD = ROUTE_RING - 1;                                    // items in flight
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) issue(q % NQ, k0 + q / NQ, q);
    int slot = 0;
    u32x4 xa[TT][2];
    for (int k = k0; k < k1; ++k) {
      const float roundings = (float)logit_roundings(k, k1, nk);
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        wait_copies_but<2 * (AHEAD - 1)>();
        const unsigned char* st = ring + slot * 2048 + r16 * 128;
        u32x4 v0 = *reinterpret_cast<const u32x4*>(st + ((g ^ (r16 & 7)) << 4));
        u32x4 v1 = *reinterpret_cast<const u32x4*>(st + (((4 + g) ^ (r16 & 7)) << 4));
        asm volatile("" : "+v"(v0), "+v"(v1));                               // in registers: the slot read before may be filled again
        issue((j + AHEAD) % NQ, k + (j + AHEAD) / NQ, slot == 0 ? ROUTE_RING - 1 : slot - 1);
        slot = slot + 1 == ROUTE_RING ? 0 : slot + 1;
        if (j < TT) {
          xa[j < TT ? j : 0][0] = v0;
          xa[j < TT ? j : 0][1] = v1;
          xn[j < TT ? j : 0] = __builtin_fmaf(roundings, squares(v1, squares(v0, 0.0f)), xn[j < TT ? j : 0]);
        } else {
          const int b = j < TT ? 0 : j - TT;
          wn[b] = __builtin_fmaf(roundings, squares(v1, squares(v0, 0.0f)), wn[b]);
#pragma unroll
          for (int tt = 0; tt < TT; ++tt) {
            acc[b][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v0), as_bf16x8(xa[tt][0]), acc[b][tt], 0, 0, 0);
            acc[b][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v1), as_bf16x8(xa[tt][1]), acc[b][tt], 0, 0, 0);
          }
        }
      }
    }
  }
  wait_copies_but<0>();
  // squares: of each part of K the largest expert's (their sum is at least the largest sum), and every token's
  float wpart = wn[0];
#pragma unroll
  for (int b = 1; b < NBLK; ++b) wpart = fmaxf(wpart, wn[b]);
  wpart = row_max<16>(wpart);
  if (r16 == 0) s_wn[wave * 4 + g] = wpart;
#pragma unroll
  for (int tt = 0; tt < TT; ++tt) s_xn[(16 * tt + r16) * (ROUTE_WAVES * 4) + wave * 4 + g] = xn[tt];
  for (int e = tid; e < S::EP; e += 64 * ROUTE_WAVES) s_bal[e] = a.balance != nullptr && e < a.E ? a.balance[e] : 0.0f;
  // tile v = b * TT + tt of a round of eight is summed by wave v % 8; the parts take the place of the rings
  f32x4* const s_part = reinterpret_cast<f32x4*>(smem);                      // [wave][8][lane]
#pragma unroll
  for (int r = 0; r < NBLK * TT; r += 8) {
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 8; ++v)
      if (r + v < NBLK * TT) s_part[(wave * 8 + v) * 64 + lane] = acc[(r + v) / TT][(r + v) % TT];
    __syncthreads();
    const int v = r + wave;
    if (v < NBLK * TT) {
      f32x4 sum = s_part[wave * 64 + lane];
#pragma unroll
      for (int w = 1; w < ROUTE_WAVES; ++w) sum += s_part[(w * 8 + wave) * 64 + lane];
      // element j: expert first + 4 g + j of token r16
#pragma unroll
      for (int j = 0; j < 4; ++j) s_logit[(16 * (v % TT) + r16) * S::LDL + first(v / TT) + 4 * g + j] = sum[j];
    }
  }
  __syncthreads();
  float bal_most = 0.0f;
  if (a.balance != nullptr && !a.sigmoid) {
#pragma unroll
    for (int e = lane; e < S::EP; e += 64) bal_most = fmaxf(bal_most, fabsf(s_bal[e]) < INFINITY ? fabsf(s_bal[e]) : 0.0f);
    bal_most = fold_max(bal_most);
  }
  const int tk = (wave * 64 + lane) / S::LANES, t = t0 + tk;
  const float w2 = row_sum<16>(s_wn[r16] + s_wn[16 + r16]), x2 = row_sum<16>(s_xn[tk * 32 + r16] + s_xn[tk * 32 + 16 + r16]);
  const bool known = x2 >= 1e-28f && x2 < INFINITY && w2 >= 1e-28f && w2 < INFINITY;     // (squares that did not vanish or overflow)
  uint32_t* const s_key = reinterpret_cast<uint32_t*>(smem) + tk * (S::EP + GROUPS_MAX);
  const float doubt = known ? LOGIT_ERROR_UNIT * sqrtf(x2) * sqrtf(w2) : -1.0f;
  int* const s_redo = reinterpret_cast<int*>(s_wn);                          // (every wave has read the norms before the barrier below)
  bool redo = false;
  for (int pass = 0; pass < 2; ++pass) {
    redo = choose<S::EP / S::LANES, S::LANES>(a, min(t, a.T - 1), t < a.T && (pass == 0 || redo), pass > 0, s_logit + tk * S::LDL, s_bal,
                                              bal_most, doubt, lane, s_key, reinterpret_cast<float*>(s_key + S::EP)) && t < a.T;
    if (pass > 0 || !__syncthreads_or(redo)) break;
    // the tokens that need all of their logits in the defined order (values that are not finite, softmax scores too close to
    // tell apart by a denominator that is not exact): by all waves
    if ((lane & (S::LANES - 1)) == 0) s_redo[tk] = redo;
    __syncthreads();
    for (int i = 0; i < S::TOKENS; ++i) {
      if (s_redo[i] == 0) continue;
      for (int e = 4 * wave; e < a.E; e += 4 * ROUTE_WAVES) {
        const bf16_t *xs[1] = {x0 + (size_t)i * H}, *ws[4];
        float v[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) ws[n] = a.Wr + (size_t)min(e + n, a.E - 1) * H;
        defined_logits(xs, ws, H, lane, v);
        if (lane == 0) *reinterpret_cast<f32x4*>(s_logit + i * S::LDL + e) = f32x4{v[0], v[1], v[2], v[3]};
      }
    }
    __syncthreads();
  }
}

template <int NBLK, int TT>
int launch_route_scored_t(const RouteScored& a, hipStream_t st) {
  using S = RouteShape<NBLK, TT>;
  auto kern = route_scored_kernel<NBLK, TT>;
  static std::atomic<uint64_t> lds_raised{0};
  if (raise_lds_limit((const void*)kern, S::LDS, lds_raised) != 0) return -4;
  constexpr int most = 1 << 24;          // tokens of a launch (a grid has less than 2^32 threads)
  for (int t0 = 0; t0 < a.T; t0 += std::min(most, a.T - t0)) {
    RouteScored part = a;
    part.x += (size_t)t0 * a.H;
    part.ids += (size_t)t0 * a.K;
    part.w += (size_t)t0 * a.K;
    part.T = std::min(most, a.T - t0);
    hipLaunchKernelGGL(kern, dim3((part.T + S::TOKENS - 1) / S::TOKENS), dim3(64 * ROUTE_WAVES), S::LDS, st, part);
    if (hipGetLastError() != hipSuccess) return -4;
  }
  return 0;
}

}  // namespace

int launch_route_scored(const RouteScored& a, hipStream_t st) {
  const bool many = a.T > 16 * 256;      // more than a workgroup of 16 tokens per compute unit
  if (a.E <= 64) return many ? launch_route_scored_t<4, 2>(a, st) : launch_route_scored_t<4, 1>(a, st);
  if (a.E <= 128) return many ? launch_route_scored_t<8, 2>(a, st) : launch_route_scored_t<8, 1>(a, st);
  if (a.E <= 192) return many ? launch_route_scored_t<12, 2>(a, st) : launch_route_scored_t<12, 1>(a, st);
  return many ? launch_route_scored_t<16, 2>(a, st) : launch_route_scored_t<16, 1>(a, st);
}

}  // namespace moe
