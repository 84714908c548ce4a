// Device code of the policy's side: actions drawn from logits, the policy loss with its gradient, and the
// advantages of a rollout.
//
// A row of logits belongs to a team of TEAM threads (one lane, a part of a wavefront, a wavefront, a
// workgroup), which holds all of it in registers, PER classes a thread: one read of HBM, whatever is
// computed of it.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <cstdint>

namespace pcgrl {

struct F32 {
  using raw = float;
  static constexpr int kKeyShift = 0;  // low bits of the ordered key that no two values differ in
  static __device__ float load(raw r) { return r; }
  static __device__ raw store(float f) { return f; }
};
struct F16 {
  using raw = uint16_t;
  static constexpr int kKeyShift = 13;
  static __device__ float load(raw r) { return __half2float(__ushort_as_half(r)); }
  static __device__ raw store(float f) { return __half_as_ushort(__float2half_rn(f)); }
};
struct BF16 {
  using raw = uint16_t;
  static constexpr int kKeyShift = 16;
  static __device__ float load(raw r) { return __uint_as_float((uint32_t)r << 16); }
  static __device__ raw store(float f) {  // to nearest, ties to even; a NaN stays one
    const uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (raw)((u >> 16) | 0x40u);
    return (raw)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
  }
};

constexpr float kNone = -__builtin_huge_valf();  // the logit of a class that may not be chosen

// 2^z for z <= 0 (0 below -1000, NaN for NaN), to about 2^-52: the powers of f in [-1/2, 1/2] with ln(2)^k / k!.
__device__ inline double pow2(double z) {
  z = z < -1000. ? -1000. : z;
  const double n = __builtin_rint(z), f = z - n;
  double p = 2.5678435993488196e-11;   // ln(2)^12 / 12!
  p = __builtin_fma(p, f, 4.44553827187081e-10);  // 11
  p = __builtin_fma(p, f, 7.054911620801121e-09);  // 10
  p = __builtin_fma(p, f, 1.0178086009239696e-07);  // 9
  p = __builtin_fma(p, f, 1.3215486790144305e-06);  // 8
  p = __builtin_fma(p, f, 1.5252733804059838e-05);  // 7
  p = __builtin_fma(p, f, 0.00015403530393381606);  // 6
  p = __builtin_fma(p, f, 0.0013333558146428441);  // 5
  p = __builtin_fma(p, f, 0.009618129107628477);  // 4
  p = __builtin_fma(p, f, 0.055504108664821576);  // 3
  p = __builtin_fma(p, f, 0.2402265069591007);  // 2
  p = __builtin_fma(p, f, 0.6931471805599453);  // 1
  p = __builtin_fma(p, f, 1.);
  return __builtin_ldexp(p, (int)n);
}

// Floats in their order as unsigned integers.
__device__ inline uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// What the threads of a team know together.
template <int TEAM> struct Team {
  static constexpr int kWaves = TEAM > 64 ? TEAM / 64 : 1;
  double* room;  // LDS: two sets of a double for each wavefront, used in turn, so that one barrier a sum is enough
  int turn = 0;
  __device__ static int rank() { return TEAM == 1 ? 0 : (int)(threadIdx.x & (TEAM - 1)); }
  template <typename V, typename Op> __device__ V all(V v, Op op) {
    constexpr int kIn = TEAM < 64 ? TEAM : 64;
#pragma unroll
    for (int d = 1; d < kIn; d <<= 1) v = op(v, __shfl_xor(v, d));
    if constexpr (TEAM > 64) {
      V* at = reinterpret_cast<V*>(room + turn * kWaves);
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
      __syncthreads();
      v = at[0];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) v = op(v, at[i]);
    }
    return v;
  }
  __device__ double sum(double v) {
    return all(v, [](double a, double b) { return a + b; });
  }
  __device__ int sum(int v) {
    return all(v, [](int a, int b) { return a + b; });
  }
  __device__ int least(int v) {
    return all(v, [](int a, int b) { return a < b ? a : b; });
  }
  __device__ float most(float v) {
    return all(v, [](float a, float b) { return a > b ? a : b; });
  }
};

// The classes of a thread: pieces of VEC neighbouring ones; each wavefront of a team has one stretch of the
// row, in which its lanes' pieces lie side by side, so that running sums go from wavefront to wavefront.
template <typename T, int TEAM, int PER> struct Row {
  static constexpr int VEC = PER < 16 / (int)sizeof(typename T::raw) ? PER : 16 / (int)sizeof(typename T::raw);
  static constexpr int PIECES = PER / VEC;
  static constexpr int LANES = TEAM < 64 ? TEAM : 64;
  // first class of piece c
  static __device__ int at(int c) {
    const int r = Team<TEAM>::rank();
    return (r / LANES) * (LANES * PER) + (c * LANES + r % LANES) * VEC;
  }
  // Logits of the classes that may be chosen, kNone for the others.  (+0 for -0: they are equal.)
  static __device__ void load(const typename T::raw* row, const uint8_t* mask, int n, float (&x)[PER]) {
#pragma unroll
    for (int c = 0; c < PIECES; ++c) {
      const int at0 = at(c);
      typename T::raw v[VEC];
      uint8_t m[VEC];
      if (at0 + VEC <= n) {
        __builtin_memcpy(v, row + at0, sizeof(v));
        if (mask) __builtin_memcpy(m, mask + at0, sizeof(m));
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[c * VEC + e] = mask && m[e] == 0 ? kNone : T::load(v[e]) + 0.f;
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int i = at0 + e;
          x[c * VEC + e] = i < n && (!mask || mask[i] != 0) ? T::load(row[i]) + 0.f : kNone;
        }
      }
    }
  }
  static __device__ void store(typename T::raw* row, int n, const float (&g)[PER]) {
#pragma unroll
    for (int c = 0; c < PIECES; ++c) {
      const int at0 = at(c);
      if (at0 + VEC <= n) {
        typename T::raw v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = T::store(g[c * VEC + e]);
        __builtin_memcpy(row + at0, v, sizeof(v));
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (at0 + e < n) row[at0 + e] = T::store(g[c * VEC + e]);
      }
    }
  }
};

template <int TEAM> constexpr int team_block() { return TEAM > 64 ? TEAM : 256; }

// ---- actions drawn from logits

struct SampleArgs {
  const void* logits;
  const uint8_t* mask;
  const float* uniform;
  int32_t* actions;
  float* log_probs;
  int64_t n_rows, logits_stride, mask_stride;
  int32_t n, top_k;     // (top_k: 0 or 1..n-1)
  double slope;         // log2(e) / temperature
  double inv_temperature, top_p, min_p;
};

constexpr int kSampleBest = 0, kSamplePlain = 1, kSampleCut = 2;

// Weights are held as whole numbers of 2^-bits in doubles, with as many bits as leave every sum of a row
// below 2^53: sums are exact, whatever their order, so that a running sum cut up over lanes and wavefronts is the
// same number as the sum of the parts.  (A weight is off by half a unit, at the most 2^-39 of the
// largest one.)
template <int CLASSES> constexpr double weight_unit() {
  int bits = 53;
  for (int c = 1; c < CLASSES; c <<= 1) --bits;
  return (double)(1ll << bits);
}

template <typename T, int TEAM, int PER, int HOW> __global__ __launch_bounds__(team_block<TEAM>()) void sample_kernel(SampleArgs a) {
  using R = Row<T, TEAM, PER>;
  __shared__ double room[TEAM > 64 ? 2 * TEAM / 64 : 1];
  __shared__ double wave_sums[TEAM > 64 ? TEAM / 64 : 1];
  __shared__ int found;
  Team<TEAM> team{room};
  constexpr int kTeams = team_block<TEAM>() / TEAM;
  constexpr double kUnit = weight_unit<TEAM * PER>();
  for (int64_t row = (int64_t)blockIdx.x * kTeams + threadIdx.x / TEAM; row < a.n_rows; row += (int64_t)gridDim.x * kTeams) {
    float x[PER];
    R::load(static_cast<const typename T::raw*>(a.logits) + row * a.logits_stride, a.mask ? a.mask + row * a.mask_stride : nullptr, a.n, x);
    float top = kNone;
    int odd = 0;  // a NaN or +infinity
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      top = x[j] > top ? x[j] : top;
      odd |= !(x[j] < __builtin_huge_valf());
    }
    top = team.most(top);
    odd = team.sum(odd);
    if (odd != 0 || top == kNone) {
      if (team.rank() == 0) {
        a.actions[row] = -1;
        if (a.log_probs) a.log_probs[row] = odd == 0 ? 0.f : __builtin_nanf("");
      }
      continue;
    }
    if constexpr (HOW == kSampleBest) {
      int best = a.n;
#pragma unroll
      for (int j = PER - 1; j >= 0; --j)
        if (x[j] == top) best = R::at(j / R::VEC) + j % R::VEC;
      best = team.least(best);
      if (team.rank() == 0) {
        a.actions[row] = best;
        if (a.log_probs) a.log_probs[row] = 0.f;
      }
      continue;
    }
    double w[PER], whole = 0.;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      w[j] = __builtin_rint(kUnit * pow2(((double)x[j] - (double)top) * a.slope));
      whole += w[j];
    }
    whole = team.sum(whole);
    double kept = whole;
    if constexpr (HOW == kSampleCut) {
      // The classes kept are those of a larger key than `edge` and the first `ties` of that key.
      uint32_t edge = 0;
      int ties = 0x7fffffff;
      constexpr int kBits = 32 - T::kKeyShift;
      auto key = [&](int j) { return key_of(x[j]) >> T::kKeyShift; };
      auto count_from = [&](uint32_t k) {
        int c = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) c += key(j) >= k;
        return team.sum(c);
      };
      auto sum_from = [&](uint32_t k) {
        double s = 0.;
#pragma unroll
        for (int j = 0; j < PER; ++j) s += key(j) >= k ? w[j] : 0.;
        return team.sum(s);
      };
      auto weight_at = [&](uint32_t k) {
        float v = kNone;
#pragma unroll
        for (int j = 0; j < PER; ++j) v = key(j) == k ? x[j] : v;
        v = team.most(v);
        return __builtin_rint(kUnit * pow2(((double)v - (double)top) * a.slope));
      };
      if (a.top_k > 0 && count_from((key_of(kNone) >> T::kKeyShift) + 1) > a.top_k) {
        for (int b = kBits - 1; b >= 0; --b) {
          const uint32_t k = edge | (1u << b);
          if (count_from(k) >= a.top_k) edge = k;
        }
        ties = a.top_k - count_from(edge + 1);
        kept = sum_from(edge + 1) + ties * weight_at(edge);
      }
      if (a.top_p < 1.) {
        const double share = a.top_p * kept;
        uint32_t k2 = 0;
        for (int b = kBits - 1; b >= 0; --b) {
          const uint32_t k = k2 | (1u << b);
          if (sum_from(k) >= share) k2 = k;
        }
        if (k2 >= edge) {
          const double above = sum_from(k2 + 1), one = weight_at(k2);
          int more = 1;                                      // classes of this key while the sum before them is below the share
          if (one > 0.) more = (int)__builtin_fmin(__builtin_ceil((share - above) / one), 32768.);
          ties = k2 == edge && ties < more ? ties : more;
          edge = k2;
        }
      }
      // the last class, by index, of those of the key `edge` that are kept
      int last = 0x7fffffff;
      auto count_at = [&](int until) {
        int c = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) c += key(j) == edge && R::at(j / R::VEC) + j % R::VEC <= until;
        return team.sum(c);
      };
      if (ties < 32768 && count_at(a.n) > ties) {
        int low = -1, high = a.n - 1;                        // count_at(low) < ties <= count_at(high)
        while (high - low > 1) {
          const int mid = (low + high) >> 1;
          if (count_at(mid) < ties) low = mid; else high = mid;
        }
        last = high;
      }
      kept = 0.;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const bool in = key(j) > edge || (key(j) == edge && R::at(j / R::VEC) + j % R::VEC <= last);
        const bool enough = pow2(((double)x[j] - (double)top) * a.slope) >= a.min_p;
        w[j] = in && enough ? w[j] : 0.;
        kept += w[j];
      }
      kept = team.sum(kept);
    }
    // the first class whose running sum exceeds the target
    double u = (double)a.uniform[row];
    u = u >= 0. ? u : 0.;
    const double target = (u < 1. ? u : 1. - 0x1p-24) * kept;
    int chosen = a.n;
    double before = 0.;
    bool here = true;
    if constexpr (TEAM > 64) {
      double mine = 0.;
#pragma unroll
      for (int j = 0; j < PER; ++j) mine += w[j];
      for (int d = 1; d < 64; d <<= 1) mine += __shfl_xor(mine, d);
      if ((threadIdx.x & 63) == 0) wave_sums[threadIdx.x >> 6] = mine;
      __syncthreads();
      for (int i = 0; i < (int)(threadIdx.x >> 6); ++i) before += wave_sums[i];
      here = before <= target && target < before + mine;
    }
    if (here) {
#pragma unroll
      for (int c = 0; c < R::PIECES; ++c) {
        double mine = 0.;
#pragma unroll
        for (int e = 0; e < R::VEC; ++e) mine += w[c * R::VEC + e];
        double until = mine;                                 // running sum over the lanes of a team
        for (int d = 1; d < R::LANES; d <<= 1) {
          const double o = __shfl_up(until, d, R::LANES);
          until += (Team<TEAM>::rank() % R::LANES) >= d ? o : 0.;
        }
        double run = before + until - mine;
        if (run <= target && target < before + until) {
#pragma unroll
          for (int e = 0; e < R::VEC; ++e) {
            run += w[c * R::VEC + e];
            if (run > target && chosen == a.n) chosen = R::at(c) + e;
          }
        }
        before += __shfl(until, R::LANES - 1, R::LANES);
      }
    }
    if constexpr (TEAM > 64) {
      if (chosen < a.n) found = chosen;
      __syncthreads();
      chosen = found;
    } else {
      chosen = team.least(chosen);
    }
    chosen = (uint32_t)chosen < (uint32_t)a.n ? chosen : a.n - 1;
    if (team.rank() == 0) {
      a.actions[row] = chosen;
      if (a.log_probs) {
        const typename T::raw* at = static_cast<const typename T::raw*>(a.logits) + row * a.logits_stride;
        a.log_probs[row] = (float)(((double)T::load(at[chosen]) - (double)top) * a.inv_temperature - log(whole / kUnit));
      }
    }
  }
}

// ---- the policy loss

struct LossArgs {
  const void* logits;
  const uint8_t* mask;
  const int32_t* actions;
  const float* advantages;
  const float* old;
  const void* values;
  const float* returns;
  void* grad_logits;
  void* grad_values;
  float* log_probs;
  float* entropies;
  double* partial;      // kLossSums doubles of each workgroup, or NULL
  int64_t n_rows, logits_stride, mask_stride, grad_stride;
  int32_t n;
  double slope, inv_temperature, low, high;  // the ratio is clipped to [low, high]
  double entropy_coef, value_coef, scale;
};

constexpr int kLossSums = 6;  // rows, policy loss, entropy, value loss, divergence, clipped rows
constexpr int kLossBlocks = 2048;

template <typename T, int TEAM, int PER> __global__ __launch_bounds__(team_block<TEAM>()) void loss_kernel(LossArgs a) {
  using R = Row<T, TEAM, PER>;
  using raw = typename T::raw;
  __shared__ double room[TEAM > 64 ? 2 * TEAM / 64 : 1];
  __shared__ double sums[kLossSums][team_block<TEAM>() / 64];
  Team<TEAM> team{room};
  constexpr int kTeams = team_block<TEAM>() / TEAM;
  double part[kLossSums] = {};
  for (int64_t row = (int64_t)blockIdx.x * kTeams + threadIdx.x / TEAM; row < a.n_rows; row += (int64_t)gridDim.x * kTeams) {
    const raw* logits = static_cast<const raw*>(a.logits) + row * a.logits_stride;
    const uint8_t* mask = a.mask ? a.mask + row * a.mask_stride : nullptr;
    const int action = a.actions[row];
    const bool inside = action >= 0 && action < a.n;
    float x[PER];
    R::load(logits, mask, a.n, x);
    const float mine = inside && (!mask || mask[action] != 0) ? T::load(logits[action]) : kNone;
    float top = kNone;
#pragma unroll
    for (int j = 0; j < PER; ++j) top = x[j] > top ? x[j] : top;
    top = team.most(top);
    const bool use = mine != kNone;       // (then something may be chosen)
    float w[PER];
    double whole = 0., spread = 0.;       // sums of the weights, and of the weights times their log2
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const double y = ((double)x[j] - (double)top) * a.slope, e = pow2(y);
      w[j] = x[j] == kNone ? 0.f : (float)e;
      whole += x[j] == kNone ? 0. : e;
      spread += x[j] == kNone ? 0. : e * y;
    }
    whole = team.sum(whole);
    spread = team.sum(spread);
    const double log_whole = log(whole);
    const double entropy = log_whole - 0.69314718055994530942 * (spread / whole);
    const double logp = ((double)mine - (double)top) * a.inv_temperature - log_whole;
    double pull = 0.;                     // the policy loss's derivative by the log-probability
    if (use) {
      const double adv = (double)a.advantages[row];
      const double change = a.old ? logp - (double)a.old[row] : 0.;
      const double ratio = exp(change);
      const bool clipped = a.old && ((adv > 0. && ratio > a.high) || (adv < 0. && ratio < a.low));
      pull = clipped ? 0. : -adv * ratio;
      if (team.rank() == 0) {
        part[0] += 1.;
        part[1] += !a.old ? -adv * logp : clipped ? -adv * (adv > 0. ? a.high : a.low) : -adv * ratio;
        part[2] += entropy;
        part[4] += ratio - 1. - change;
        part[5] += clipped ? 1. : 0.;
      }
    }
    if (team.rank() == 0) {
      if (a.values) {
        const double off = use ? (double)T::load(static_cast<const raw*>(a.values)[row]) - (double)a.returns[row] : 0.;
        part[3] += .5 * off * off;
        if (a.grad_values) static_cast<raw*>(a.grad_values)[row] = T::store((float)(a.value_coef * a.scale * off));
      }
      if (a.log_probs) a.log_probs[row] = use ? (float)logp : 0.f;
      if (a.entropies) a.entropies[row] = use ? (float)entropy : 0.f;
    }
    if (a.grad_logits) {
      const double by = a.scale * a.inv_temperature;
      const float k1 = (float)(by * pull), k2 = (float)(by * a.entropy_coef);
      const float inv = (float)(1. / whole), h = (float)(entropy - log_whole), slope = (float)a.inv_temperature;
      float g[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const float p = w[j] * inv;
        const float around = (x[j] - top) * slope + h;      // log p + entropy
        const bool chosen = R::at(j / R::VEC) + j % R::VEC == action;
        g[j] = !use || x[j] == kNone ? 0.f : k2 * p * around + (chosen ? k1 - k1 * p : -(k1 * p));
      }
      R::store(static_cast<raw*>(a.grad_logits) + row * a.grad_stride, a.n, g);
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < kLossSums; ++i) {
    double v = part[i];
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) sums[i][threadIdx.x >> 6] = v;
  }
  __syncthreads();
  if (threadIdx.x < kLossSums) {
    double v = 0.;
    for (int i = 0; i < team_block<TEAM>() / 64; ++i) v += sums[threadIdx.x][i];
    a.partial[(size_t)blockIdx.x * kLossSums + threadIdx.x] = v;
  }
}

// Joins the workgroups' sums, always in the same order.
__global__ __launch_bounds__(64 * kLossSums) void loss_sums_kernel(const double* partial, int blocks, double entropy_coef, double value_coef,
                                                                  double scale, float* stats) {
  __shared__ double sums[kLossSums];
  const int which = threadIdx.x >> 6;
  double v = 0.;
  for (int b = threadIdx.x & 63; b < blocks; b += 64) v += partial[(size_t)b * kLossSums + which];
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) sums[which] = v;
  __syncthreads();
  if (threadIdx.x == 0) stats[0] = (float)(scale * (sums[1] - entropy_coef * sums[2] + value_coef * sums[3]));
  if (threadIdx.x < kLossSums) stats[1 + threadIdx.x] = (float)sums[threadIdx.x];
}

// ---- advantages

struct AdvantageArgs {
  const float* reward;
  const uint8_t* done;
  const void* values;
  float* advantages;
  float* returns;
  int32_t n_steps, n_envs;
  double discount, trace;
};

// One lane an environment, backwards over its steps.
template <typename T> __global__ __launch_bounds__(256) void advantages_kernel(AdvantageArgs a) {
  const int64_t env = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (env >= a.n_envs) return;
  const typename T::raw* values = static_cast<const typename T::raw*>(a.values);
  double next = (double)T::load(values[(int64_t)a.n_steps * a.n_envs + env]), after = 0.;
  for (int t = a.n_steps - 1; t >= 0; --t) {
    const int64_t at = (int64_t)t * a.n_envs + env;
    const double v = (double)T::load(values[at]);
    const bool goes_on = a.done[at] == 0;
    const double error = (double)a.reward[at] + (goes_on ? a.discount * next : 0.) - v;
    after = error + (goes_on ? a.discount * a.trace * after : 0.);
    a.advantages[at] = (float)after;
    if (a.returns) a.returns[at] = (float)(after + v);
    next = v;
  }
}

}  // namespace pcgrl
