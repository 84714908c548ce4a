// Host side of the policy's entry points in include/pcgrl.h: argument checks and launches.
#include "../../include/pcgrl.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "pcgrl_host.h"
#include "pcgrl_policy.hip.h"

using namespace pcgrl;

namespace {

int size_of(int type) { return type == PCGRL_UNPACK_F32 ? 4 : type == PCGRL_UNPACK_F16 || type == PCGRL_UNPACK_BF16 ? 2 : 0; }
bool misaligned(const void* p, int size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) != 0; }
constexpr int64_t kMostRows = 0x7fffffff;  // (and most elements between two)
// Rows of n elements, `stride` apart.
bool bad_rows(int64_t rows, int64_t stride, int n) { return rows > 1 && (stride < n || stride > kMostRows); }
bool bad_count(int64_t rows) { return rows < 0 || rows > kMostRows; }

// Bytes of `rows` rows, and whether two stretches of memory share any.
size_t span(int64_t rows, int64_t stride, int64_t n, int size) { return rows < 1 ? 0 : (size_t)((rows - 1) * stride + n) * size; }
bool overlap(const void* p, size_t np, const void* q, size_t nq) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return p && q && a < b + nq && b < a + np;
}
struct Memory {
  const void* at;
  size_t bytes;
};
// Whether any of the outputs shares memory with an input or with another output.
template <size_t O, size_t I> bool any_overlap(const Memory (&out)[O], const Memory (&in)[I]) {
  for (size_t o = 0; o < O; ++o) {
    for (const Memory& i : in)
      if (overlap(out[o].at, out[o].bytes, i.at, i.bytes)) return true;
    for (size_t p = 0; p < o; ++p)
      if (overlap(out[o].at, out[o].bytes, out[p].at, out[p].bytes)) return true;
  }
  return false;
}

int launched() { return hipGetLastError() == hipSuccess ? PCGRL_OK : PCGRL_E_HIP; }

// By type, and by the team and the classes a thread that hold a row of n classes.
template <int TEAM, int PER> struct Shape {
  static constexpr int kTeam = TEAM, kPer = PER;
};
template <typename F> int by_type(int type, F&& f) {
  if (type == PCGRL_UNPACK_F32) return f(F32{});
  if (type == PCGRL_UNPACK_F16) return f(F16{});
  return f(BF16{});
}
// (up to 8 classes: a lane that holds exactly as many.  Beyond that as many lanes as have 8 to 32 classes each: what a row costs besides
// its classes is shared by the rows of a wavefront.  Measured, us for losses: 20 000 rows of 500 in a wavefront / sixteen lanes 30 / 21, 5000 of 2000 in 256
// threads / a wavefront 28 / 19, 3000 of 4000 in 256 / 128 26 / 22.)
template <typename F> int by_few_classes(int n, F&& f) {
  switch (n) {
    case 1: return f(Shape<1, 1>{});
    case 2: return f(Shape<1, 2>{});
    case 3: return f(Shape<1, 3>{});
    case 4: return f(Shape<1, 4>{});
    case 5: return f(Shape<1, 5>{});
    case 6: return f(Shape<1, 6>{});
    case 7: return f(Shape<1, 7>{});
    default: return f(Shape<1, 8>{});
  }
}
template <typename F> int by_classes(int n, F&& f) {
  if (n <= 8) return by_few_classes(n, f);
  if (n <= 64) return f(Shape<8, 8>{});
  if (n <= 128) return f(Shape<8, 16>{});
  if (n <= 256) return f(Shape<16, 16>{});
  if (n <= 512) return f(Shape<16, 32>{});
  if (n <= 1024) return f(Shape<64, 16>{});
  if (n <= 2048) return f(Shape<64, 32>{});
  if (n <= 4096) return f(Shape<128, 32>{});
  if (n <= 8192) return f(Shape<256, 32>{});
  if (n <= 16384) return f(Shape<512, 32>{});
  return f(Shape<1024, 32>{});
}
// Workgroups of a loss that the machine holds at once, each of which then takes several rows: four wavefronts a SIMD, five of
// the smallest teams.  Measured, us for 512 / 1024 / 1280 / 2048 workgroups: 2 097 152 rows of 7 classes 47 / 37 / 35 / 35, 300 000 of 50
// 62 / 46 / 44 / 43, 20 000 of 500 23 / 20 / 21 / 21; for 256 / 512 / 1024 (of 512 threads) 1024 of 16 384 42 / 31.5 / 32.
template <int TEAM> constexpr int64_t resident() {
  constexpr int64_t most = (TEAM <= 8 ? 5 : 4) * (int64_t)65536 / team_block<TEAM>();
  static_assert(most <= kLossBlocks, "");
  return most;
}
// Workgroups for so many rows, and no more than `most` of them, which then take rows in turn.
template <int TEAM> unsigned groups_for(int64_t rows, int64_t most) {
  const int64_t each = team_block<TEAM>() / TEAM, want = (rows + each - 1) / each;
  return (unsigned)(want < most ? want : most);
}

// How advantages are shared out over workgroups: sets the environments and steps of one, and returns the groups
// that the steps are cut into.  Measured, us:
//   Few environments: as many threads along the steps as take all of them at once, 64 steps of 64 environments
//   with 4 / 16 / 32 environments a workgroup 4.4 / 3.8 / 3.5, 2000 of 64 with 1 / 4 / 8 9.9 / 12.0 / 20.2.
//   Where that takes several turns of 2.5 us the steps are cut into groups, at the price of two more launches and
//   of reading the inputs twice: 10 000 steps of 16 10.5 against 32, of 1 14.9 against 23.4, but 3000 of 1 13.2 against
//   9.5, 1000 of 4096 21.5 against 23.6 and 300 of 4096 12.6 against 10.3.
//   Many: rows of a workgroup as wide as leave enough workgroups, 300 steps of 8000 with 16 / 32 / 64
//   environments 16.2 / 14.0 / 15.8, 128 of 65 536 with 32 / 64 / 256 27.4 / 21.8 / 27.7, 32 of 262 145 with 64 / 256 31 / 24.
int share_steps(AdvantageArgs* a) {
  const int n = a->n_envs, T = a->n_steps;
  const bool cut = n < 4096 && T > (n <= 64 ? 4096 : 2048);
  int fit = 0, lg = n >= 131072 ? 8 : n >= 32768 ? 6 : n >= 8000 ? 5 : n >= 4096 ? 4 : 0;
  while (fit < 6 && (T << (fit + 1)) <= kAdvantageThreads * kAdvantageSteps) ++fit;
  if (cut) lg = n > 2048 ? 6 : n > 512 ? 5 : 4;
  else if (fit > lg) lg = fit;
  while (lg > 0 && (1 << (lg - 1)) >= n) --lg;
  a->envs_log2 = lg;
  if (!cut) return 1;
  const int at_once = (kAdvantageThreads >> lg) * kAdvantageSteps;
  const int across = (n + (1 << lg) - 1) >> lg, pieces = (T + at_once - 1) / at_once, room = kAdvantageEach * (kAdvantageThreads >> lg);
  int groups = 1600 / across;
  groups = groups < pieces ? groups : pieces;
  groups = groups < room ? groups : room;
  if (groups < 2) return 1;
  const int each = (pieces + groups - 1) / groups;
  a->group = each * at_once;
  return (pieces + each - 1) / each;
}

}  // namespace

extern "C" {

int pcgrl_sample(const pcgrl_ctx* ctx, const pcgrl_sampling* how, const void* logits, const uint8_t* mask, const float* uniform,
                 int64_t n_rows, int32_t* actions, float* log_probs, void* stream) {
  if (!ctx || !how) return PCGRL_E_NULL;
  const int size = size_of(how->type);
  if (size == 0 || how->n_classes < 1 || how->n_classes > PCGRL_MAX_CLASSES || bad_count(n_rows)) return PCGRL_E_CONFIG;
  if (!(how->temperature >= 0.) || !(how->temperature <= 3e38) || !(how->top_p > 0.) || !(how->min_p >= 0. && how->min_p <= 1.) ||
      how->top_k < 0)
    return PCGRL_E_CONFIG;
  if (how->temperature > 0. && how->temperature < 1e-30) return PCGRL_E_CONFIG;
  if (n_rows == 0) return PCGRL_OK;
  const bool best = how->temperature == 0.;
  if (!logits || !actions || (!uniform && !best)) return PCGRL_E_NULL;
  if (misaligned(logits, size) || misaligned(uniform, 4) || misaligned(actions, 4) || misaligned(log_probs, 4)) return PCGRL_E_CONFIG;
  if (bad_rows(n_rows, how->logits_stride, how->n_classes)) return PCGRL_E_CONFIG;
  if (mask && how->mask_stride != 0 && bad_rows(n_rows, how->mask_stride, how->n_classes)) return PCGRL_E_CONFIG;
  const size_t each = (size_t)n_rows * 4;
  const Memory in[] = {{logits, span(n_rows, how->logits_stride, how->n_classes, size)}, {mask, span(n_rows, how->mask_stride, how->n_classes, 1)}, {uniform, each}};
  const Memory out[] = {{actions, each}, {log_probs, each}};
  if (any_overlap(out, in)) return PCGRL_E_CONFIG;
  DeviceGuard guard(device_of(ctx));
  if (!guard.ok) return PCGRL_E_DEVICE;
  SampleArgs a{};
  a.logits = logits;
  a.mask = mask;
  a.uniform = uniform;
  a.actions = actions;
  a.log_probs = log_probs;
  a.n_rows = n_rows;
  a.logits_stride = how->logits_stride;
  a.mask_stride = how->mask_stride;
  a.n = how->n_classes;
  a.top_k = how->top_k < how->n_classes ? how->top_k : 0;
  a.inv_temperature = best ? 0. : 1. / how->temperature;
  a.slope = 64. * 1.44269504088896340736 * a.inv_temperature;
  const int bits = weight_bits(a.n);
  a.unit = std::ldexp(1., bits);
  a.inv_unit = std::ldexp(1., -bits);
  a.reach = (float)((bits + 2) * 0.69314718055994530942 * how->temperature);
  a.top_p = how->top_p;
  a.least = how->min_p * a.unit;
  const bool cut = a.top_k > 0 || a.top_p < 1. || a.least > 0.;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return by_type(how->type, [&](auto type) {
    using T = decltype(type);
    if (best) {
      return by_classes(a.n, [&](auto shape) {
        using S = decltype(shape);
        hipLaunchKernelGGL((best_kernel<T, S::kTeam, S::kPer>), dim3(groups_for<S::kTeam>(n_rows, 1 << 20)), dim3(team_block<S::kTeam>()), 0, st, a);
        return launched();
      });
    }
    auto few = [&](auto shape, auto kernel) {
      using S = decltype(shape);
      hipLaunchKernelGGL(kernel, dim3(groups_for<S::kTeam>(n_rows, 1 << 20)), dim3(256), 0, st, a);
      return launched();
    };
    auto either = [&](auto shape) {
      using S = decltype(shape);
      return few(shape, cut ? &sample_few_kernel<T, S::kTeam, S::kPer, kSampleCut> : &sample_few_kernel<T, S::kTeam, S::kPer, kSamplePlain>);
    };
    if (a.n <= 8) return by_few_classes(a.n, either);
    if (a.n <= 64) return either(Shape<8, 8>{});
    // Beyond that, registers for plain draws and where there are enough rows to hide the steps of the halving behind each other, LDS
    // for the rest.  Measured, us for registers / LDS: 4096 rows of 200 classes in bfloat16 3.7 / 7.4, with top_p 12.2 / 15.2, with top_k
    // and top_p 15.0 / 13.6; in float32, with its twice as many bits, with top_p 12.8 / 10.1, 60 000 rows 88 / 106; 16 rows 11.0 / 9.3; 60 000 rows of
    // 500 in bfloat16 35 / 76, with top_p 201 / 169.
    if (cut ? a.n <= 256 && n_rows >= (sizeof(typename T::raw) == 2 ? 2048 : 8192) : a.n <= 512) {
      if (a.n <= 128) return either(Shape<8, 16>{});
      if (a.n <= 256) return either(Shape<16, 16>{});
      return few(Shape<16, 32>{}, &sample_few_kernel<T, 16, 32, kSamplePlain>);
    }
    auto many = [&](auto shape) {
      using S = decltype(shape);
      constexpr int kVec = Stretch<T, S::kTeam>::VEC;
      a.lds_row = (uint32_t)((a.n + 64 * kVec - 1) / (64 * kVec) * 1024);
      const uint32_t lds = a.lds_row * (team_block<S::kTeam>() / S::kTeam);
      auto* kernel = cut ? &sample_many_kernel<T, S::kTeam, kSampleCut> : &sample_many_kernel<T, S::kTeam, kSamplePlain>;
      hipLaunchKernelGGL(kernel, dim3(groups_for<S::kTeam>(n_rows, 1 << 20)), dim3(team_block<S::kTeam>()), lds, st, a);
      return launched();
    };
    // A wavefront a row where it is short; then a workgroup of 256 or 512 threads, of which a compute unit has room for more than one,
    // 512 where there are no more than two rows for each of them; 1024 where one row is as much LDS as there is, and for the longest of
    // rows that have a compute unit each.  Measured, us for 64 / 256 / 512 / 1024 threads a row, with top_p: 4096 rows of 1024 classes 22 /
    // 41 / 82 / 189, 2000 of 4000 47 / 39 / 51 / 115, 1000 of 8000 - / 33 / 39 / 61, 512 of 8000 - / 25 / 22 / 31, 257 of 12 000 - / 32 / 25 / 39,
    // 1024 of 28 672 - / 137 / 91 / 131, 257 - / 64 / 45 / 62, 256 - / 59 / 36 / 34; in float32 256 of 28 672 - / - / 33 / 28, 512 - / - / 67 / 57.
    if (a.n <= 1024) return many(Shape<64, 1>{});
    if (a.n * (int)sizeof(typename T::raw) > 61440 || (n_rows <= 256 && a.n > 16384)) return many(Shape<1024, 1>{});
    if (a.n <= 4096 || (a.n <= 8192 && n_rows > 512)) return many(Shape<256, 1>{});
    return many(Shape<512, 1>{});
  });
}

int pcgrl_step_logits(pcgrl_ctx* ctx, const pcgrl_sampling* how, const void* logits, const uint8_t* mask, const float* uniform,
                      int32_t* actions, float* log_probs, uint8_t* obs, float* reward, uint8_t* done, void* stream) {
  if (!ctx || !how) return PCGRL_E_NULL;
  if (how->n_classes != tiles_in(ctx)) return PCGRL_E_CONFIG;
  // (the step reads actions while it writes, and would write over the log-probabilities)
  const size_t n = (size_t)levels_of(ctx);
  const Memory drawn[] = {{actions, n * 4}, {log_probs, n * 4}}, stepped[] = {{obs, n * (size_t)pcgrl_obs_stride(ctx)}, {reward, n * 4}, {done, n}};
  for (const Memory& d : drawn)
    for (const Memory& s : stepped)
      if (overlap(d.at, d.bytes, s.at, s.bytes)) return PCGRL_E_CONFIG;
  const int rc = pcgrl_sample(ctx, how, logits, mask, uniform, levels_of(ctx), actions, log_probs, stream);
  return rc == PCGRL_OK ? pcgrl_step(ctx, actions, obs, reward, done, stream) : rc;
}

int pcgrl_advantages(const pcgrl_ctx* ctx, const float* reward, const uint8_t* done, const void* values, int32_t values_type,
                     int32_t n_steps, int32_t n_envs, double discount, double trace, float* advantages, float* returns, void* stream) {
  if (!ctx) return PCGRL_E_NULL;
  const int size = size_of(values_type);
  if (size == 0 || n_steps < 0 || n_steps > (1 << 20) || n_envs < 0 || n_envs > (1 << 24)) return PCGRL_E_CONFIG;
  if (!(discount >= 0. && discount <= 1.) || !(trace >= 0. && trace <= 1.)) return PCGRL_E_CONFIG;
  if (n_steps == 0 || n_envs == 0) return PCGRL_OK;
  if (!reward || !done || !values || !advantages) return PCGRL_E_NULL;
  if (misaligned(reward, 4) || misaligned(values, size) || misaligned(advantages, 4) || misaligned(returns, 4)) return PCGRL_E_CONFIG;
  const size_t steps = (size_t)n_steps * n_envs;
  const Memory in[] = {{reward, steps * 4}, {done, steps}, {values, (steps + n_envs) * size}}, out[] = {{advantages, steps * 4}, {returns, steps * 4}};
  if (any_overlap(out, in)) return PCGRL_E_CONFIG;
  DeviceGuard guard(device_of(ctx));
  if (!guard.ok) return PCGRL_E_DEVICE;
  AdvantageArgs a{reward, done, values, advantages, returns, n_steps, n_envs, 0, n_steps, discount, discount * trace, discount * trace > 0. ? 1e-300 : 0.};
  const int groups = share_steps(&a);
  const dim3 block(kAdvantageThreads), grid((unsigned)((n_envs + (1 << a.envs_log2) - 1) >> a.envs_log2), (unsigned)groups);
  hipStream_t st = static_cast<hipStream_t>(stream);
  return by_type(values_type, [&](auto type) {
    using T = decltype(type);
    if (groups == 1) {
      hipLaunchKernelGGL((advantages_kernel<T, kAdvantageAll>), grid, block, 0, st, a);
      return launched();
    }
    hipLaunchKernelGGL((advantages_kernel<T, kAdvantageSum>), dim3(grid.x, grid.y - 1), block, 0, st, a);
    hipLaunchKernelGGL(advantages_join_kernel, dim3(grid.x), block, 0, st, a, groups);
    hipLaunchKernelGGL((advantages_kernel<T, kAdvantageApply>), grid, block, 0, st, a);
    return launched();
  });
}

int64_t pcgrl_policy_loss_workspace(void) { return (int64_t)kLossBlocks * kLossSums * (int64_t)sizeof(double); }

int pcgrl_policy_loss(const pcgrl_ctx* ctx, const pcgrl_loss* l, void* stream) {
  if (!ctx || !l) return PCGRL_E_NULL;
  const int size = size_of(l->type);
  if (size == 0 || l->n_classes < 1 || l->n_classes > PCGRL_MAX_CLASSES || bad_count(l->n_rows)) return PCGRL_E_CONFIG;
  if (!(l->temperature >= 1e-30 && l->temperature <= 3e38) || !(l->clip_low >= 0. && l->clip_low <= 1.) || !(l->clip_high >= 0.) ||
      !std::isfinite(l->clip_high) || !std::isfinite(l->entropy_coef) || !std::isfinite(l->value_coef) || !std::isfinite(l->scale))
    return PCGRL_E_CONFIG;
  // (what gradients are multiplied by, with room for a sum of products in 64 bits)
  constexpr double kMostFactor = 1e300;
  const double by = l->scale / l->temperature;
  if (!(std::fabs(by) <= kMostFactor && std::fabs(by * l->entropy_coef) <= kMostFactor && std::fabs(l->scale * l->value_coef) <= kMostFactor)) return PCGRL_E_CONFIG;
  if (l->stats && !l->workspace) return PCGRL_E_NULL;
  if (misaligned(l->stats, 4) || misaligned(l->workspace, 8)) return PCGRL_E_CONFIG;
  if (l->n_rows > 0) {
    if (!l->logits || !l->actions || !l->advantages || (l->values && !l->returns)) return PCGRL_E_NULL;
    if (misaligned(l->logits, size) || misaligned(l->actions, 4) || misaligned(l->advantages, 4) || misaligned(l->old_log_probs, 4) ||
        misaligned(l->values, size) || misaligned(l->returns, 4) || misaligned(l->grad_logits, size) || misaligned(l->grad_values, size) ||
        misaligned(l->log_probs, 4) || misaligned(l->entropies, 4))
      return PCGRL_E_CONFIG;
    if (l->grad_values && !l->values) return PCGRL_E_NULL;
    if (bad_rows(l->n_rows, l->logits_stride, l->n_classes)) return PCGRL_E_CONFIG;
    if (l->mask && l->mask_stride != 0 && bad_rows(l->n_rows, l->mask_stride, l->n_classes)) return PCGRL_E_CONFIG;
    if (l->grad_logits && bad_rows(l->n_rows, l->grad_stride, l->n_classes)) return PCGRL_E_CONFIG;
    // (the gradients may lie where what they are of is: nothing else of it is read after them)
    const int64_t n = l->n_rows;
    const bool in_place = l->grad_logits == l->logits && (n == 1 || l->grad_stride == l->logits_stride);
    const size_t row = (size_t)n * 4, value = (size_t)n * size, logits = span(n, l->logits_stride, l->n_classes, size);
    const Memory in[] = {{in_place ? nullptr : l->logits, logits}, {l->mask, span(n, l->mask_stride, l->n_classes, 1)},
                         {l->actions, row}, {l->advantages, row}, {l->old_log_probs, row},
                         {l->grad_values == l->values ? nullptr : l->values, value}, {l->values ? l->returns : nullptr, row}};
    const Memory out[] = {{l->grad_logits, span(n, l->grad_stride, l->n_classes, size)}, {l->grad_values, value}, {l->log_probs, row},
                          {l->entropies, row}, {l->stats, PCGRL_LOSS_STATS * 4}, {l->stats ? l->workspace : nullptr, (size_t)pcgrl_policy_loss_workspace()}};
    if (any_overlap(out, in)) return PCGRL_E_CONFIG;
  }
  if (l->n_rows == 0 && !l->stats) return PCGRL_OK;
  DeviceGuard guard(device_of(ctx));
  if (!guard.ok) return PCGRL_E_DEVICE;
  LossArgs a{};
  a.logits = l->logits;
  a.mask = l->mask;
  a.actions = l->actions;
  a.advantages = l->advantages;
  a.old = l->old_log_probs;
  a.values = l->values;
  a.returns = l->returns;
  a.grad_logits = l->grad_logits;
  a.grad_values = l->grad_values;
  a.log_probs = l->log_probs;
  a.entropies = l->entropies;
  a.partial = l->stats ? static_cast<double*>(l->workspace) : nullptr;
  a.n_rows = l->n_rows;
  a.logits_stride = l->logits_stride;
  a.mask_stride = l->mask_stride;
  a.grad_stride = l->grad_stride;
  a.n = l->n_classes;
  a.inv_temperature = 1. / l->temperature;
  a.slope = 64. * 1.44269504088896340736 * a.inv_temperature;
  a.low = 1. - l->clip_low;
  a.high = 1. + l->clip_high;
  a.by = l->scale * a.inv_temperature;
  a.bonus = a.by * l->entropy_coef;
  a.value_by = l->value_coef * l->scale;
  // (gradients in 32 bits: if all factors are in reach, and that of the logits' distances keeps all its bits)
  const double bonus = std::fabs(a.bonus);
  const bool narrow = l->temperature >= 1. / kWidest && l->temperature <= kWidest && bonus < kWidest && (bonus == 0. || bonus / l->temperature > 0x1p-100);
  a.widest = narrow ? kWidest : -1.;
  a.bonus_off = narrow ? (float)(a.bonus * a.inv_temperature) : 0.f;
  a.least = narrow ? (float)(-1000. / a.inv_temperature) : 0.f;
  hipStream_t st = static_cast<hipStream_t>(stream);
  unsigned blocks = 0;
  if (l->n_rows > 0) {
    const int rc = by_type(l->type, [&](auto type) {
      return by_classes(a.n, [&](auto shape) {
        using S = decltype(shape);
        blocks = groups_for<S::kTeam>(l->n_rows, resident<S::kTeam>());
        hipLaunchKernelGGL((loss_kernel<decltype(type), S::kTeam, S::kPer>), dim3(blocks), dim3(team_block<S::kTeam>()), 0, st, a);
        return launched();
      });
    });
    if (rc != PCGRL_OK) return rc;
  }
  if (!l->stats) return PCGRL_OK;
  hipLaunchKernelGGL(loss_sums_kernel, dim3(1), dim3(kSumThreads), 0, st, static_cast<const double*>(l->workspace), (int)blocks,
                     l->entropy_coef, l->value_coef, l->scale, l->stats);
  return launched();
}

}  // extern "C"
