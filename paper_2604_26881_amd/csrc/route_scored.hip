// Gating by scores: softmax or sigmoid of the router logits, an optional bias that takes part in the choice alone, experts
// in groups of which only the best are considered, top-k, renormalised and scaled weights.
//
//   l[t,e] = <x[t,:], Wr[e,:]>   in the order of additions of route.hip, so both calls see the same logits
//   s[t,e] = softmax_e(l) or sigmoid(l), formed in 64 bits and rounded once to fp32;   c = s + balance
//   value of a group = its largest c, or the sum of its two largest;  the top_groups best groups are kept
//   ids = the K largest c among the kept groups' experts;  w = s[id] (over their sum + 1e-20 with renorm) * scale
//
// Why 64 bits: the choice compares scores, and a score's last bit would otherwise be the library exponential's business.
// With the rounding of an exact value, every implementation of the formula chooses alike.
// NaN orders below everything, so the ids are K different experts whatever the rows hold.
#include "fold.h"
#include "mx.h"

namespace moe {

constexpr int SCORED_EMAX = 256;

__device__ __forceinline__ uint32_t fold_umax(uint32_t a) {
  auto step = [&](auto ctrl, auto rmask) {
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp((int)a, (int)a, decltype(ctrl)::value, decltype(rmask)::value, 0xF, false));
  };
  step(std::integral_constant<int, 0xB1>{}, std::integral_constant<int, 0xF>{});
  step(std::integral_constant<int, 0x4E>{}, std::integral_constant<int, 0xF>{});
  step(std::integral_constant<int, 0x141>{}, std::integral_constant<int, 0xF>{});
  step(std::integral_constant<int, 0x140>{}, std::integral_constant<int, 0xF>{});
  step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});
  step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});
  return (uint32_t)__builtin_amdgcn_readlane((int)a, 63);
}
// Whole numbers that order like the values: -0 as +0, NaN as 0, below -infinity
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return v != v ? 0u : (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return k == 0u ? __uint_as_float(0x7fc00000u) : __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k);
}

// Scores of one token by one wave: l[i] is the logit of expert lane + 64 i
__device__ __forceinline__ void form_scores(const RouteScored& a, const float (&l)[4], int lane, float (&s)[4]) {
  if (a.sigmoid) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = (float)(1.0 / (1.0 + exp(-(double)l[i])));
    return;
  }
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane + 64 * i < a.E) m = fmaxf(m, l[i]);
  m = fold_max(m);
  double p[4], z = 0.0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p[i] = lane + 64 * i < a.E ? exp((double)l[i] - (double)m) : 0.0;
    z += p[i];
  }
#pragma unroll
  for (int w = 1; w < 64; w <<= 1) z += __shfl_xor(z, w, WAVE);
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = (float)(p[i] / z);
}

// Choice and weights of one token by one wave; key[i] and s[i] belong to expert lane + 64 i, s_key holds 256 keys of the wave.
__device__ __forceinline__ void choose(const RouteScored& a, const uint32_t (&key)[4], const float (&s)[4], int lane,
                                       uint32_t* s_key, int t) {
  bool out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = lane + 64 * i >= a.E;
  if (a.groups > a.top_groups) {
    const int size = a.E / a.groups;
#pragma unroll
    for (int i = 0; i < 4; ++i) s_key[lane + 64 * i] = key[i];
    __builtin_amdgcn_wave_barrier();
    uint32_t k1 = 0, k2 = 0;       // the two largest keys of group `lane`
    if (lane < a.groups) {
      for (int j = 0; j < size; ++j) {
        const uint32_t k = s_key[lane * size + j];
        k2 = max(k2, min(k1, k));
        k1 = max(k1, k);
      }
    }
    const uint32_t value = a.best == 1 ? k1 : order_key(key_value(k1) + key_value(k2));
    bool left = lane < a.groups;
    unsigned long long kept = 0ull;
    for (int j = 0; j < a.top_groups; ++j) {
      const uint32_t best = fold_umax(left ? value : 0u);
      const int g = __builtin_ctzll(__ballot(left && value == best));
      kept |= 1ull << g;
      if (lane == g) left = false;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!out[i]) out[i] = ((kept >> ((lane + 64 * i) / size)) & 1ull) == 0ull;
  }
  int my_id = 0;
  float my_s = 0.0f, run = 0.0f;
  for (int j = 0; j < a.K; ++j) {
    uint32_t k = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!out[i]) k = max(k, key[i]);
    k = fold_umax(k);
    int e = -1;
    float mine = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned long long hit = __ballot(!out[i] && key[i] == k);
      if (e < 0 && hit != 0ull) {
        e = __builtin_ctzll(hit) + 64 * i;
        mine = s[i];
      }
    }
    const float sj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), e & 63));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (e == lane + 64 * i) out[i] = true;
    run += sj;
    if (lane == j) { my_id = e; my_s = sj; }
  }
  if (a.renorm) my_s = my_s / (run + 1e-20f);
  if (lane < a.K) {
    a.ids[(size_t)t * a.K + lane] = my_id;
    a.w[(size_t)t * a.K + lane] = my_s * a.scale;
  }
}

// The logit of one (token, expert) pair by one wave, in the defined order
__device__ __forceinline__ float defined_logit(const bf16_t* x, const bf16_t* w, int H, int lane) {
  float acc = 0.0f;
  for (int h = 8 * lane; h < H; h += 512) {
    float xf[8], wf[8];
    widen8(*reinterpret_cast<const u32x4*>(x + h), xf);
    widen8(*reinterpret_cast<const u32x4*>(w + h), wf);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc = __builtin_fmaf(xf[i], wf[i], acc);
  }
  return fold_sum(acc);
}

__global__ __launch_bounds__(256) void route_scored_kernel(RouteScored a) {
  __shared__ float s_logit[SCORED_EMAX];
  __shared__ uint32_t s_key[SCORED_EMAX];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = blockIdx.x;
  for (int e = wave; e < a.E; e += 4) {
    const float l = defined_logit(a.x + (size_t)t * a.H, a.Wr + (size_t)e * a.H, a.H, lane);
    if (lane == 0) s_logit[e] = l;
  }
  __syncthreads();
  if (wave != 0) return;
  float l[4], s[4];
  uint32_t key[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) l[i] = lane + 64 * i < a.E ? s_logit[lane + 64 * i] : 0.0f;
  form_scores(a, l, lane, s);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = lane + 64 * i;
    key[i] = order_key(a.balance != nullptr && e < a.E ? s[i] + a.balance[e] : s[i]);
  }
  choose(a, key, s, lane, s_key, t);
}

int launch_route_scored(const RouteScored& a, hipStream_t st) {
  hipLaunchKernelGGL(route_scored_kernel, dim3(a.T), dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? 0 : -4;
}

}  // namespace moe
