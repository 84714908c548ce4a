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
  int32_t envs_log2;  // environments of a workgroup
  int32_t group;      // steps of a workgroup: a multiple of what it takes at a time, or all
  double discount, decay;  // decay: discount * trace
};

constexpr int kAdvantageThreads = 256, kAdvantageSteps = 8;
// workgroups that share the steps of their environments out: one launch sums up what each group of steps makes
// of the advantage behind it (a factor and a term), one turns these into the advantage behind each group,
// one computes the advantages
constexpr int kAdvantageAll = 0, kAdvantageSum = 1, kAdvantageApply = 2;
constexpr int kAdvantageEach = 8;  // groups of a thread of the launch in the middle

// (a factor of 0 is the end of an episode: what is behind it does not count, be it infinite or no number)
__device__ inline double after_it(double factor, double term, double behind) { return factor == 0. ? term : __builtin_fma(factor, behind, term); }

// Between the launches the factor and the term of group g + 1, and then the advantage behind group g, lie in the
// first rows of group g's own advantages, which the last launch reads before it writes them.
__device__ inline void put(float* at, int64_t n, double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  at[0] = __uint_as_float((uint32_t)u);
  at[n] = __uint_as_float((uint32_t)(u >> 32));
}
__device__ inline double take(const float* at, int64_t n) {
  return __longlong_as_double((long long)((uint64_t)__float_as_uint(at[0]) | (uint64_t)__float_as_uint(at[n]) << 32));
}

// What the threads of a workgroup behind this one make of the advantage behind them all: thread c E + e has steps behind
// those of thread (c - 1) E + e.  Sets `behind` to the advantage behind this thread's steps and returns that before the
// workgroup's first; `factor_all`, if asked for, is multiplied by all factors.
template <bool ALL> __device__ inline double join_steps(int envs_log2, double factor, double term, double& behind, double& factor_all, double (*factors)[64],
                                                        double (*terms)[64]) {
  constexpr int kWaves = kAdvantageThreads / 64;
  const int E = 1 << envs_log2, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // within a wavefront: this thread's steps and all behind them
  double f = factor, t = term;
  for (int d = E; d < 64; d <<= 1) {
    const double f2 = __shfl_down(f, d), t2 = __shfl_down(t, d);
    if (lane + d < 64) {
      t = after_it(f, t, t2);
      f *= f2;
    }
  }
  const int per = E < 64 ? 1 : E >> 6;      // wavefronts side by side on the same steps
  __syncthreads();
  if (lane < E) {
    factors[wave][lane] = f;
    terms[wave][lane] = t;
  }
  __syncthreads();
  double mine = behind;
  const int col = lane & (E - 1);
#pragma unroll
  for (int w = kWaves - 1; w >= 0; --w) {
    if (per > 1 && (w & (per - 1)) != (wave & (per - 1))) continue;
    if (w == wave) mine = behind;
    behind = after_it(factors[w][col], terms[w][col], behind);
    if (ALL) factor_all *= factors[w][col];
  }
  // behind this thread's steps are those of the lanes behind it, and then what is behind the wavefront
  const double f2 = E < 64 ? __shfl_down(f, E) : 1., t2 = E < 64 ? __shfl_down(t, E) : 0.;
  const bool last = lane + E >= 64;
  const double all = behind;
  behind = last ? mine : after_it(f2, t2, mine);
  return all;
}

// A thread takes kAdvantageSteps steps of one environment at a time: neighbouring lanes have neighbouring
// environments, and the threads left over go along the steps.  Each sums its steps up as a factor and a term;
// joined from the last to the first they give every thread the advantage behind its steps.  Every input
// is read once into registers, and the next steps are asked for before these are joined, which is worth a third to
// a half (128 steps of 65 536 environments 41 -> 22 us, 10 000 of 800 71 -> 46).
// Bound by memory for many environments: 32 steps of 262 144 with bfloat16 values, 126 MB, 21 us (6.0 TB/s of 5.4 that a large
// copy reaches, as part of it stays in the last-level cache); by the latency of a load and a join, 2.5 us, and of a launch
// for few.  Four environments a thread with 16-byte loads were not faster (26.5 against 21.6 us), nor workgroups of 1024 threads
// (2000 steps of 64 9.1 against 9.9, 64 steps of 64 5.4 against 3.5).
template <typename T, int MODE> __global__ __launch_bounds__(kAdvantageThreads) void advantages_kernel(AdvantageArgs a) {
  __shared__ double factors[kAdvantageThreads / 64][64], terms[kAdvantageThreads / 64][64];
  constexpr int L = kAdvantageSteps;
  const int E = 1 << a.envs_log2, C = kAdvantageThreads >> a.envs_log2;
  const int e = threadIdx.x & (E - 1), c = threadIdx.x >> a.envs_log2;
  const int64_t n = a.n_envs, env = (int64_t)blockIdx.x * E + e;
  const bool live = env < n;
  const typename T::raw* values = static_cast<const typename T::raw*>(a.values);
  const int g = MODE == kAdvantageSum ? blockIdx.y + 1 : blockIdx.y;
  const int lo = g * a.group, hi = a.n_steps - lo < a.group ? a.n_steps : lo + a.group;
  double behind = 0., factor_all = 1.;
  if (MODE == kAdvantageApply && hi < a.n_steps) {
    if (live) behind = take(a.advantages + (int64_t)lo * n + env, n);
    __syncthreads();
  }
  typename T::raw v[L + 1];
  float r[L];
  uint8_t d[L];
  auto fetch = [&](int base) {
#pragma unroll
    for (int i = 0; i <= L; ++i)
      if (live && base + i >= lo && base + L > lo) v[i] = values[(int64_t)(base + i) * n + env];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      if (live && base + i >= lo) {
        r[i] = a.reward[(int64_t)(base + i) * n + env];
        d[i] = a.done[(int64_t)(base + i) * n + env];
      }
    }
  };
  fetch(hi - (C - c) * L);
  for (int top = hi; top > lo; top -= C * L) {
    const int base = top - (C - c) * L;
    double error[L], factor = 1., term = 0., mine = behind;
    float value[L];
    uint32_t ends = 0;
#pragma unroll
    for (int i = L - 1; i >= 0; --i) {
      if (live && base + i >= lo) {
        const bool end = d[i] != 0;
        value[i] = T::load(v[i]);
        error[i] = (double)r[i] + (end ? 0. : a.discount * (double)T::load(v[i + 1])) - (double)value[i];
        term = end ? error[i] : __builtin_fma(a.decay, term, error[i]);
        factor = end ? 0. : factor * a.decay;
        ends |= end ? 1u << i : 0u;
      }
    }
    if (top - C * L > lo) fetch(base - C * L);
    if (C > 1) {
      behind = join_steps<MODE == kAdvantageSum>(a.envs_log2, factor, term, mine, factor_all, factors, terms);
    } else {
      behind = after_it(factor, term, behind);
      factor_all *= factor;
    }
    if (MODE != kAdvantageSum) {
#pragma unroll
      for (int i = L - 1; i >= 0; --i) {
        if (live && base + i >= lo) {
          mine = ends >> i & 1u ? error[i] : __builtin_fma(a.decay, mine, error[i]);
          const int64_t at = (int64_t)(base + i) * n + env;
          a.advantages[at] = (float)mine;
          if (a.returns) a.returns[at] = (float)(mine + (double)value[i]);
        }
      }
    }
  }
  if (MODE == kAdvantageSum && live && c == 0) {
    float* at = a.advantages + (int64_t)(lo - a.group) * n + env;
    put(at, n, factor_all);
    put(at + 2 * n, n, behind);
  }
}

__global__ __launch_bounds__(kAdvantageThreads) void advantages_join_kernel(AdvantageArgs a, int groups) {
  __shared__ double factors[kAdvantageThreads / 64][64], terms[kAdvantageThreads / 64][64];
  const int E = 1 << a.envs_log2, C = kAdvantageThreads >> a.envs_log2;
  const int e = threadIdx.x & (E - 1), c = threadIdx.x >> a.envs_log2;
  const int64_t n = a.n_envs, env = (int64_t)blockIdx.x * E + e;
  const int each = (groups + C - 1) / C, first = c * each;      // groups first .. first + each - 1, the last one's end is the end
  double f[kAdvantageEach], t[kAdvantageEach];
  const bool live = env < n;
#pragma unroll
  for (int i = 0; i < kAdvantageEach; ++i) {
    const bool in = live && i < each && first + i < groups - 1;
    const float* at = a.advantages + (int64_t)(first + i) * a.group * n + env;
    f[i] = in ? take(at, n) : 1.;
    t[i] = in ? take(at + 2 * n, n) : 0.;
  }
  double factor = 1., term = 0.;
#pragma unroll
  for (int i = kAdvantageEach - 1; i >= 0; --i) {
    term = after_it(f[i], t[i], term);
    factor *= f[i];
  }
  double behind = 0., unused = 1.;
  join_steps<false>(a.envs_log2, factor, term, behind, unused, factors, terms);
#pragma unroll
  for (int i = kAdvantageEach - 1; i >= 0; --i) {
    if (live && i < each && first + i < groups - 1) {
      behind = after_it(f[i], t[i], behind);
      put(a.advantages + (int64_t)(first + i) * a.group * n + env, n, behind);
    }
  }
}

}  // namespace pcgrl
