// Device code of the policy's side: actions drawn from logits, the policy loss with its gradient, and the
// advantages of a rollout.
//
// A row of logits belongs to a team of TEAM threads (one lane, a part of a wavefront, a wavefront, a
// workgroup), which holds all of it in registers, PER classes a thread, or in LDS: one read of HBM, whatever is
// computed of it.  What an action or the clipping of a ratio depends on is computed in 64 bits, which this part does at the rate
// of 32; it is what most of these kernels are bound by.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/pcgrl.h"

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
  static __device__ raw store(float f) { return __builtin_bit_cast(raw, (__bf16)f); }  // (one instruction, to nearest even)
};

constexpr float kNone = -__builtin_huge_valf();  // the logit of a class that may not be chosen

// 2^z for z <= 0 (0 below -1000, NaN for NaN), to about 2^-52: the powers of f in [-1/2, 1/2] with ln(2)^k / k!.
__device__ __forceinline__ double pow2(double z) {
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
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// Lets the compiler forget what it has computed from the classes of a thread: what it would keep from one pass over them to
// the next takes more registers than there are.
template <int TEAM, int PER> __device__ __forceinline__ void forget_classes(float (&x)[PER], int& first) {
  if constexpr (PER >= 16 || TEAM >= 64) {
#pragma unroll
    for (int j = 0; j < PER; ++j) asm volatile("" : "+v"(x[j]));
    asm volatile("" : "+v"(first));
  }
}

// Values of other lanes.
template <int CTRL> __device__ __forceinline__ int moved(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
template <int CTRL> __device__ __forceinline__ float moved(float v) { return __int_as_float(moved<CTRL>(__float_as_int(v))); }
template <int CTRL> __device__ __forceinline__ double moved(double v) { return __hiloint2double(moved<CTRL>(__double2hiint(v)), moved<CTRL>(__double2loint(v))); }
__device__ __forceinline__ int of_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ float of_lane(float v, int lane) { return __int_as_float(of_lane(__float_as_int(v), lane)); }
__device__ __forceinline__ double of_lane(double v, int lane) { return __hiloint2double(of_lane(__double2hiint(v), lane), of_lane(__double2loint(v), lane)); }

// op over the first LANES lanes of every LANES, in all of them.
template <int LANES, typename V, typename Op> __device__ __forceinline__ V over_lanes(V v, Op op) {
  static_assert(LANES == 1 || LANES == 8 || LANES == 16 || LANES == 64, "");
  if constexpr (LANES >= 8) {
    v = op(v, moved<0xB1>(v));   // the other of a pair
    v = op(v, moved<0x4E>(v));   // the other pair of four
    v = op(v, moved<0x141>(v));  // the other four of eight
  }
  if constexpr (LANES >= 16) v = op(v, moved<0x140>(v));  // the other eight of sixteen
  if constexpr (LANES == 64) {
    v = op(op(of_lane(v, 0), of_lane(v, 16)), op(of_lane(v, 32), of_lane(v, 48)));
  }
  return v;
}
// Sum over the lanes before and including this one, of every LANES: within rows of 16 lanes by shifts that bring in zeros, then
// with what the rows before have.
template <int LANES, typename V> __device__ __forceinline__ V sum_until(V v) {
  if constexpr (LANES == 8) {
    const int lane = threadIdx.x & 7;
    V o = moved<0x111>(v);
    v += lane >= 1 ? o : (V)0;
    o = moved<0x112>(v);
    v += lane >= 2 ? o : (V)0;
    o = moved<0x114>(v);
    v += lane >= 4 ? o : (V)0;
  }
  if constexpr (LANES >= 16) {
    v += moved<0x111>(v);
    v += moved<0x112>(v);
    v += moved<0x114>(v);
    v += moved<0x118>(v);
  }
  if constexpr (LANES == 64) {
    const V a = of_lane(v, 15), b = a + of_lane(v, 31), c = b + of_lane(v, 47);
    const int row = (threadIdx.x & 63) >> 4;
    v += row == 0 ? (V)0 : row == 1 ? a : row == 2 ? b : c;
  }
  return v;
}

// Whether logits have a NaN or +infinity among them: those are the largest of all bit patterns, with the sign or without it.
// (A comparison for each logit takes three times as many instructions.)
struct Oddity {
  int most = (int)0x80000000;
  uint32_t most_signed = 0;
  __device__ __forceinline__ void look(float x) {
    most = max(most, __float_as_int(x));
    most_signed = max(most_signed, __float_as_uint(x));
  }
  __device__ __forceinline__ bool seen() const { return most >= 0x7f800000 || most_signed > 0xff800000u; }
};

// What the threads of a team know together.
template <int TEAM> struct Team {
  static constexpr int kWaves = TEAM > 64 ? TEAM / 64 : 1, kLanes = TEAM < 64 ? TEAM : 64;
  double* room;  // LDS: two sets of a double for each wavefront, used in turn, so that one barrier a sum is enough
  int turn = 0;
  __device__ static int rank() { return TEAM == 1 ? 0 : (int)(threadIdx.x & (TEAM - 1)); }
  // (what follows from it is computed for each row: kept from row to row it takes more registers than there are)
  __device__ __forceinline__ static int rank_anew() {
    int r = rank();
    asm volatile("" : "+v"(r));
    return r;
  }
  // Orders what a team has written to LDS before what it reads afterwards.
  __device__ static void sync() {
    if constexpr (TEAM > 64) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  }
  template <typename V, typename Op> __device__ __forceinline__ V all(V v, Op op) {
    v = over_lanes<kLanes>(v, op);
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
  // The sum, and what of it is in the wavefronts before this one and in this one, to which each may have something to add.
  __device__ __forceinline__ double sum(double v, double& before, double& here, const double* extra = nullptr) {
    here = over_lanes<kLanes>(v, [](double a, double b) { return a + b; });
    if (extra) here += extra[TEAM > 64 ? rank() >> 6 : 0];
    before = 0.;
    if constexpr (TEAM > 64) {
      double *at = room + turn * kWaves, all = 0.;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = here;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        before = i == (int)(threadIdx.x >> 6) ? all : before;
        all += at[i];
      }
      return all;
    }
    return here;
  }
  __device__ __forceinline__ void sum_both(double& v, double& w) {
    v = over_lanes<kLanes>(v, [](double a, double b) { return a + b; });
    w = over_lanes<kLanes>(w, [](double a, double b) { return a + b; });
    if constexpr (TEAM > 64) {  // (with room for two doubles a wavefront in each of the two sets)
      double2* at = reinterpret_cast<double2*>(room) + turn * kWaves;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = double2{v, w};
      __syncthreads();
      v = w = 0.;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        v += at[i].x;
        w += at[i].y;
      }
    }
  }
  __device__ int least(int v) {
    return all(v, [](int a, int b) { return a < b ? a : b; });
  }
  // The largest of one and the smallest of the other, at once; orders LDS.
  __device__ __forceinline__ void most_and_least(float& most, float& least) {
    most = over_lanes<kLanes>(most, [](float a, float b) { return a > b ? a : b; });
    least = over_lanes<kLanes>(least, [](float a, float b) { return a < b ? a : b; });
    if constexpr (TEAM > 64) {
      float2* at = reinterpret_cast<float2*>(room + turn * kWaves);
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = float2{most, least};
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        most = __builtin_fmaxf(most, at[i].x);
        least = __builtin_fminf(least, at[i].y);
      }
    } else {
      sync();
    }
  }
  __device__ float most(float v) {
    return all(v, [](float a, float b) { return a > b ? a : b; });
  }
};

// Powers of two by a table of 2^(i / 64), 64 doubles in LDS, times `unit`: power() is unit * 2^(z / 64) to 2^-44 (what the fifth term
// could add, (ln(2) / 128)^5 / 120), with four terms of the series of what is left of z, 17 instructions; with five to 2^-51.
template <int TEAM> __device__ __forceinline__ void fill_powers(double* table, double unit) {
  if (threadIdx.x < 64) table[threadIdx.x] = unit * 2. * pow2((double)threadIdx.x / 64. - 1.);
  if (TEAM <= 64) __syncthreads();  // (larger teams have a barrier for their largest logit before they read it)
}
template <int TERMS = 4> __device__ __forceinline__ double power_from(const double* table, double z) {  // (z >= -64000, or NaN)
  const double t = z + 0x1.8p52, r = z - (t - 0x1.8p52);  // the nearest whole number, in the low word of t
  const int n = __double2loint(t);
  double q = 5.732851688640402e-10;                       // (ln(2) / 64)^4 / 4!
  if constexpr (TERMS == 5) q = __builtin_fma(1.2417843701716925e-12, r, q);  // 5
  q = __builtin_fma(q, r, 2.1173137155464774e-07);        // 3
  q = __builtin_fma(q, r, 5.864904955056169e-05);         // 2
  q = __builtin_fma(q, r, 0.010830424696249145) * r;      // 1
  const double of = table[n & 63];
  return __builtin_ldexp(__builtin_fma(of, q, of), n >> 6);
}
template <int TERMS = 4> __device__ __forceinline__ double power(const double* table, double z) { return power_from<TERMS>(table, __builtin_fmax(z, -64000.)); }

// The natural logarithm of v >= 1 (NaN for infinity and NaN), to about 2^-44, with `inv_unit` one over the table's unit: what the one in
// single precision leaves, some 1e-7, by the series.  The library's takes a hundred registers of constants out of a loop.  It goes into
// log-probabilities, which are float32, and into the ratio to such a one: 2^-24 of them is what there is.
__device__ __forceinline__ double log_of(const double* table, double inv_unit, double v) {
  const double about = (double)__builtin_amdgcn_logf((float)v);
  const double rest = v * (power(table, -64. * about) * inv_unit) - 1.;
  return __builtin_fma(about, 0.69314718055994530942, rest - .5 * rest * rest);
}

// The classes of a thread: pieces of VEC neighbouring ones; each wavefront of a team has one stretch of the
// row, in which its lanes' pieces lie side by side, so that running sums go from wavefront to wavefront.  The stretches are as
// long as the row needs, to one piece, whatever the team could hold.  A piece is read at once, whatever its
// alignment; the one that the row ends in is read as the last VEC classes, of which those of the piece before are left out.
// A lane that holds a row holds exactly its classes: what it computes for others in vain is as dear as for these (2 097 152 losses of
// 7 classes in eight places 43.9 us, in seven 39.0).
template <typename T, int TEAM, int PER> struct Row {
  static constexpr int VEC = TEAM == 1 || PER < 16 / (int)sizeof(typename T::raw) ? PER : 16 / (int)sizeof(typename T::raw);
  static constexpr int AT_ONCE = VEC <= 1 ? 1 : VEC <= 2 ? 2 : VEC <= 4 ? 4 : 8;  // classes that a lane with a row reads at once
  static constexpr int PIECES = PER / VEC;
  static constexpr int LANES = TEAM < 64 ? TEAM : 64;
  int first, pieces;  // the thread's first class, and the pieces of its wavefront
  int n;
  __device__ __forceinline__ Row(int rank, int n_classes) : n(n_classes) {
    if constexpr (TEAM < 64) {
      first = rank * VEC;
      pieces = PIECES;
    } else {
      constexpr int W = TEAM / 64;
      const int all = (n + 64 * VEC - 1) / (64 * VEC), w = __builtin_amdgcn_readfirstlane(rank >> 6), from = w * all / W;
      pieces = (w + 1) * all / W - from;
      first = (from * 64 + (rank & 63)) * VEC;
    }
  }
  __device__ __forceinline__ bool has(int c) const { return TEAM < 64 || c < pieces; }  // (the same for a wavefront)
  __device__ __forceinline__ int begin(int c) const { return first + c * LANES * VEC; }
  __device__ __forceinline__ bool owns(int c, int i) const { return i >= begin(c) && i < begin(c) + VEC; }
  // the class of element e of piece c
  __device__ __forceinline__ int at(int c, int e) const {
    const int b = begin(c);
    return (TEAM > 1 && b > n - VEC ? n - VEC : b) + e;
  }
  // Logits of the classes that may be chosen, kNone for the others.  For a lane that holds a row, `ahead` and `mask_ahead` are the
  // elements from the row's first to the end of all rows: where there are as many as AT_ONCE, it reads so many
  // at once, the next row's first ones among them, and not each class by itself.
  __device__ __forceinline__ void load(const typename T::raw* row, const uint8_t* mask, int64_t ahead, int64_t mask_ahead, float (&x)[PER]) const {
    if constexpr (TEAM == 1) {
      typename T::raw v[AT_ONCE] = {};
      uint8_t m[AT_ONCE];
      if (ahead >= AT_ONCE) {
        __builtin_memcpy(v, row, sizeof(v));
      } else {
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] = row[e];
      }
#pragma unroll
      for (int e = 0; e < PER; ++e) x[e] = T::load(v[e]);
      if (!mask) return;
      if (mask_ahead >= AT_ONCE) {
        __builtin_memcpy(m, mask, sizeof(m));
      } else {  // (the last rows, and one row for all)
#pragma unroll
        for (int e = 0; e < PER; ++e) m[e] = mask[e];
      }
#pragma unroll
      for (int e = 0; e < PER; ++e) x[e] = m[e] == 0 ? kNone : x[e];
      return;
    }
#pragma unroll
    for (int c = 0; c < PIECES; ++c) {
      const int b = begin(c), from = b > n - VEC ? n - VEC : b;
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[c * VEC + e] = kNone;
      if (has(c) && b < n) {
        typename T::raw v[VEC];
        __builtin_memcpy(v, row + from, sizeof(v));
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[c * VEC + e] = T::load(v[e]);
        if (mask) {
          uint8_t m[VEC];
          __builtin_memcpy(m, mask + from, sizeof(m));
#pragma unroll
          for (int e = 0; e < VEC; ++e) x[c * VEC + e] = m[e] == 0 ? kNone : x[c * VEC + e];
        }
        if (from < b) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) x[c * VEC + e] = from + e < b ? kNone : x[c * VEC + e];
        }
      }
    }
  }
  __device__ __forceinline__ void store(typename T::raw* row, int c, const float (&g)[VEC]) const {
    const int b = begin(c), from = b > n - VEC ? n - VEC : b;
    typename T::raw v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = T::store(g[e]);
    if (TEAM == 1 || b + VEC <= n) {
      __builtin_memcpy(row + b, v, sizeof(v));
    } else if (b < n) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (from + e >= b) row[from + e] = v[e];
    }
  }
};

// Keeps the compiler from taking more than four classes of a thread through a loop at once, by having the sums over them
// done: what more take in registers costs more than it hides (28 672 classes a row went through scratch memory; no loss does now).
template <typename V> __device__ __forceinline__ void done(V& v) { asm volatile("" : "+v"(v)); }
template <typename... V> __device__ __forceinline__ void part_end(int j, V&... sums) {
  if (j % 4 == 3) {
    (done(sums), ...);
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <int TEAM> constexpr int team_block() { return TEAM > 64 ? TEAM : 256; }

// Elements from row `row` to the end of `rows` rows of n.
__device__ __forceinline__ int64_t from_row(int64_t row, int64_t rows, int64_t stride, int n) { return (rows - 1 - row) * stride + n; }

// ---- actions drawn from logits

struct SampleArgs {
  const void* logits;
  const uint8_t* mask;
  const float* uniform;
  int32_t* actions;
  float* log_probs;
  int64_t n_rows, logits_stride, mask_stride;
  int32_t n, top_k;     // (top_k: 0 or 1..n-1)
  double slope;         // 64 * log2(e) / temperature
  float reach;          // below the largest logit by more than this there are no weights
  double inv_temperature, top_p, least;  // least: min_p, as a weight
  double unit, inv_unit;  // the largest weight, 2^weight_bits(n)
  uint32_t lds_row;     // bytes of LDS that a row takes
};

constexpr int kSampleBest = 0, kSamplePlain = 1, kSampleCut = 2;

// Weights are held in doubles as whole numbers, the largest as 2^weight_bits(n): the sums of n of them do not exceed 2^53 and are
// exact, whatever their order, so that a running sum cut up over lanes and wavefronts is the same number as the sum of the parts.
// Up to 64 classes that is the only bound (2^50 for 8 classes, 2^47 for 64), and powers have the fifth term for it.  Beyond, where
// instructions a class are what a draw costs, powers to 2^-44 are good for 2^42; from 2048 classes the sums bind again, to 2^38 for 32 768.
__host__ __device__ constexpr int weight_bits(int n) {
  int sums = 53;
  while ((1 << (53 - sums)) < n) --sums;
  return n <= 8 ? 50 : n <= 64 ? 47 : sums < 42 ? sums : 42;
}
static_assert(weight_bits(8) == 50 && weight_bits(64) == 47 && weight_bits(1000) == 42 && weight_bits(4097) == 40 && weight_bits(PCGRL_MAX_CLASSES) == 38, "");

// The last of the classes that top_k and top_p keep, in the order of falling logits and rising indices.
struct Cutoff {
  uint32_t key;
  int index;
};

// How a row's weights follow from its logits.
template <int TERMS> struct Weigh {
  const double* table;
  float top;
  double slope;
  __device__ __forceinline__ double operator()(float x) const { return __builtin_rint(power<TERMS>(table, ((double)x - (double)top) * slope)); }
};
// (the two zeros are equal)
template <typename T> __device__ __forceinline__ uint32_t class_key(float x) { return key_of(x + 0.f) >> T::kKeyShift; }

__device__ __forceinline__ void put_draw(const SampleArgs& a, int64_t row, int action, float logit, float top, double whole, const double* table) {
  a.actions[row] = action;
  if (a.log_probs) a.log_probs[row] = (float)(((double)logit - (double)top) * a.inv_temperature - log_of(table, a.inv_unit, whole * a.inv_unit));
}
__device__ __forceinline__ void put_nothing(const SampleArgs& a, int64_t row, float top) {
  a.actions[row] = -1;
  if (a.log_probs) a.log_probs[row] = top == kNone ? 0.f : __builtin_nanf("");
}
__device__ __forceinline__ double uniform_of(const SampleArgs& a, int64_t row) {
  const double u = (double)a.uniform[row];
  return u >= 0. ? u < 1. ? u : 1. - 0x1p-24 : 0.;
}

// The largest logit by itself, the lowest index of equal ones, for any team: bound by memory (1000 rows of 8000 in bfloat16 4.9 us, 3.3
// TB/s).
template <typename T, int TEAM, int PER> __global__ __launch_bounds__(team_block<TEAM>()) void best_kernel(SampleArgs a) {
  using R = Row<T, TEAM, PER>;
  constexpr int kTeams = team_block<TEAM>() / TEAM;
  __shared__ double room[TEAM > 64 ? 2 * TEAM / 64 : 1];
  Team<TEAM> team{room};
  for (int64_t row = (int64_t)blockIdx.x * kTeams + threadIdx.x / TEAM; row < a.n_rows; row += (int64_t)gridDim.x * kTeams) {
    const int rank = team.rank_anew();
    const R of(rank, a.n);
    float x[PER], top = kNone;
    of.load(static_cast<const typename T::raw*>(a.logits) + row * a.logits_stride, a.mask ? a.mask + row * a.mask_stride : nullptr,
            from_row(row, a.n_rows, a.logits_stride, a.n), from_row(row, a.n_rows, a.mask_stride, a.n), x);
    Oddity odd;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      top = __builtin_fmaxf(top, x[j]);
      odd.look(x[j]);
    }
    top = team.most(odd.seen() ? __builtin_huge_valf() : top);
    if (!(top < __builtin_huge_valf()) || top == kNone) {
      if (rank == 0) put_nothing(a, row, top);
      continue;
    }
    int best = a.n;
#pragma unroll
    for (int j = PER - 1; j >= 0; --j)
      if (x[j] == top) best = of.at(j / R::VEC, j % R::VEC);
    best = team.least(best);
    if (rank == 0) {
      a.actions[row] = best;
      if (a.log_probs) a.log_probs[row] = 0.f;
    }
  }
}

// ---- few classes: a row in the registers of a lane or of eight or sixteen

// A lane that holds a whole row: each class against every other one.
template <typename T, int PER> __device__ __forceinline__ Cutoff cut_lane(const float (&x)[PER], const double (&w)[PER], const SampleArgs& a) {
  int before[PER];
  double mass[PER], whole = 0.;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    before[j] = 0;
    mass[j] = 0.;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (i == j) continue;
      const bool first = x[i] > x[j] || (i < j && x[i] == x[j]);
      before[j] += first;
      mass[j] += first ? w[i] : 0.;
    }
  }
  const int k = a.top_k > 0 ? a.top_k : PER;
#pragma unroll
  for (int j = 0; j < PER; ++j) whole += before[j] < k ? w[j] : 0.;
  const double share = a.top_p < 1. ? a.top_p * whole : __builtin_huge_val();
  Cutoff cut{0, 0x7fffffff};
  int most = -1;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const bool last = before[j] < k && mass[j] < share && before[j] > most;
    most = last ? before[j] : most;
    cut.key = last ? class_key<T>(x[j]) : cut.key;
    cut.index = last ? j : cut.index;
  }
  return cut;
}

// By halving the range of keys, and where a key is kept in part that of the indices: a sum over the team for each bit.
template <typename T, int TEAM, int PER>
__device__ __forceinline__ Cutoff cut_by_halves(const float (&x)[PER], const double (&w)[PER], const Row<T, TEAM, PER>& of, Team<TEAM>& team, const SampleArgs& a,
                                                double whole) {
  using R = Row<T, TEAM, PER>;
  constexpr int kBits = 32 - T::kKeyShift;
  uint32_t key[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) key[j] = class_key<T>(x[j]);
  auto count_from = [&](uint32_t k) {
    int c = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) c += key[j] >= k;
    return team.sum(c);
  };
  auto sum_from = [&](uint32_t k) {
    double s = 0.;
#pragma unroll
    for (int j = 0; j < PER; ++j) s += key[j] >= k ? w[j] : 0.;
    return team.sum(s);
  };
  auto weight_at = [&](uint32_t k) {  // of a class with this key
    double v = 0.;
#pragma unroll
    for (int j = 0; j < PER; ++j) v = key[j] == k ? w[j] : v;
    return team.all(v, [](double a, double b) { return a > b ? a : b; });
  };
  uint32_t edge = 0;
  int ties = 0x7fffffff;  // classes of the key `edge` that are kept
  if (a.top_k > 0 && count_from(class_key<T>(kNone) + 1) > a.top_k) {
#pragma unroll 1
    for (int b = kBits - 1; b >= 0; --b) {
      const uint32_t k = edge | (1u << b);
      if (count_from(k) >= a.top_k) edge = k;
    }
    ties = a.top_k - count_from(edge + 1);
    whole = sum_from(edge + 1) + ties * weight_at(edge);
  }
  if (a.top_p < 1.) {
    const double share = a.top_p * whole;
    uint32_t low = 0;
#pragma unroll 1
    for (int b = kBits - 1; b >= 0; --b) {
      const uint32_t k = low | (1u << b);
      if (sum_from(k) >= share) low = k;
    }
    // (not below `edge`: all of its classes together reach the share)
    const double above = sum_from(low + 1), one = weight_at(low);
    const int more = one > 0. ? (int)__builtin_fmin(__builtin_ceil((share - above) / one), (double)PCGRL_MAX_CLASSES) : 1;
    ties = low == edge && ties < more ? ties : more;
    edge = low;
  }
  auto count_until = [&](int until) {
    int c = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) c += key[j] == edge && of.at(j / R::VEC, j % R::VEC) <= until;
    return team.sum(c);
  };
  Cutoff cut{edge, 0x7fffffff};
  if (ties < PCGRL_MAX_CLASSES && count_until(a.n) > ties) {
    int low = -1, high = a.n - 1;  // count_until(low) < ties <= count_until(high)
    while (high - low > 1) {
      const int mid = (low + high) >> 1;
      if (count_until(mid) < ties) low = mid; else high = mid;
    }
    cut.index = high;
  }
  return cut;
}

// Draws of few classes, a row in the registers of one lane, of eight or of sixteen.  With w = 2^((x - top) / (temperature ln 2)), as
// whole numbers in doubles, every sum of them is exact (weight_bits): the order in which threads add them up does not
// matter, and an action depends on the numbers given alone.  A row is read once; then come the largest logit, the weights
// and their sum, the cutoff, what is kept, and the running sum to the target.  One lane holds up to 8 classes: a
// reduction over lanes is a dozen instructions for each row, and none of these need any; it finds each class's place by
// comparing all pairs.  Eight or sixteen lanes use DPP moves, and halve the range of keys for the cutoff, 16 or 32 sums.
// Bound by a launch up to some 20 000 rows (16 384 rows of 7 classes in bfloat16 3.4 us), then by 64-bit instructions: 262 144 rows of
// 7 4.2 us, with top_p or top_k 8.2, 1 000 000 of 4 8.2 us (2.4 TB/s), 100 000 of 64 9.2, 4096 of 200 3.6, with top_p 12.2.  Cutoffs of
// 65 to 256 classes keep 20 to 76 bytes a thread in scratch memory, draws of 257 to 512 without one up to 32: a row there is 16 or 32 classes a
// thread, with a weight of 64 bits each, in 128 registers; with twice as many half the rows would be there to hide each other's waits.
template <typename T, int TEAM, int PER, int HOW> __global__ __launch_bounds__(256, PER >= 16 ? 4 : 1) void sample_few_kernel(SampleArgs a) {
  static_assert(TEAM <= 16 && HOW != kSampleBest, "");
  using R = Row<T, TEAM, PER>;
  constexpr int kTeams = 256 / TEAM;
  __shared__ double table[64];
  Team<TEAM> team{nullptr};
  fill_powers<TEAM>(table, a.unit);
  for (int64_t row = (int64_t)blockIdx.x * kTeams + threadIdx.x / TEAM; row < a.n_rows; row += (int64_t)gridDim.x * kTeams) {
    const int rank = team.rank_anew();
    const R of(rank, a.n);
    float x[PER], top = kNone;
    of.load(static_cast<const typename T::raw*>(a.logits) + row * a.logits_stride, a.mask ? a.mask + row * a.mask_stride : nullptr,
            from_row(row, a.n_rows, a.logits_stride, a.n), from_row(row, a.n_rows, a.mask_stride, a.n), x);
    Oddity odd;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      top = __builtin_fmaxf(top, x[j]);
      odd.look(x[j]);
    }
    top = team.most(odd.seen() ? __builtin_huge_valf() : top);
    if (!(top < __builtin_huge_valf()) || top == kNone) {
      if (rank == 0) put_nothing(a, row, top);
      continue;
    }
    const Weigh<TEAM * PER <= 64 ? 5 : 4> weigh{table, top, a.slope};
    double w[PER], whole = 0.;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      w[j] = weigh(x[j]);
      whole += w[j];
    }
    whole = team.sum(whole);
    double kept = whole;
    if constexpr (HOW == kSampleCut) {
      Cutoff cut{0, 0x7fffffff};
      if (a.top_k > 0 || a.top_p < 1.) {
        if constexpr (TEAM == 1) cut = cut_lane<T, PER>(x, w, a);
        else cut = cut_by_halves<T, TEAM, PER>(x, w, of, team, a, whole);
      }
      kept = 0.;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const uint32_t key = class_key<T>(x[j]);
        w[j] = (key > cut.key || (key == cut.key && of.at(j / R::VEC, j % R::VEC) <= cut.index)) && w[j] >= a.least ? w[j] : 0.;
        kept += w[j];
      }
      kept = team.sum(kept);
    }
    // the first class whose running sum exceeds the target
    const double target = uniform_of(a, row) * kept;
    double before = 0.;
#pragma unroll
    for (int c = 0; c < R::PIECES; ++c) {
      double piece = 0.;
#pragma unroll
      for (int e = 0; e < R::VEC; ++e) piece += w[c * R::VEC + e];
      const double until = before + sum_until<TEAM>(piece);
      double run = until - piece;
      if (run <= target && target < until) {
        int chosen = -1;
        float logit = 0.f;
#pragma unroll
        for (int e = 0; e < R::VEC; ++e) {
          run += w[c * R::VEC + e];
          float v = x[c * R::VEC + e];
          asm("" : "+v"(v));  // (else it becomes an address chosen among the classes, and they go to memory)
          const bool it = chosen < 0 && run > target;
          chosen = it ? of.at(c, e) : chosen;
          logit = it ? v : logit;
        }
        put_draw(a, row, chosen, logit, top, whole, table);
      }
      if (c + 1 < R::PIECES) before = __shfl(until, TEAM - 1, TEAM);
    }
  }
}

// ---- many classes: a row in the LDS of a wavefront or a workgroup

// LDS of a team that looks for a cutoff: weights and numbers of classes in bins of falling logits, and the classes of one bin.
template <int TEAM> struct CutRoom {
  static constexpr int kBins = TEAM == 64 ? 256 : TEAM == 256 ? 512 : 1024, kList = TEAM == 64 ? 128 : 256;
  struct alignas(16) Entry {
    uint64_t order;  // the key, and below it the index turned round: what is kept first is larger
    double weight;
  };
  Entry list[kList];
  double mass[kBins];
  int count[kBins];
  double extra[TEAM / 64];
  double wave_mass[TEAM / 64];
  int wave_count[TEAM / 64];
  double mass_before, mass_until;
  int bin, count_before, listed;
  Cutoff found;
  __device__ __forceinline__ void put(uint32_t key, int index, double weight) {
    const int at = atomicAdd(&listed, 1);
    if (at < kList) list[at] = Entry{(uint64_t)key << 32 | (uint32_t)~index, weight};
  }
  static __device__ __forceinline__ Cutoff cutoff(uint64_t order) { return Cutoff{(uint32_t)(order >> 32), (int)~(uint32_t)order}; }
  // Weights and number of the listed classes before the one given.
  __device__ __forceinline__ void rank_of(uint64_t order, double& before, int& first) const {
#pragma unroll 8
    for (int i = 0; i < listed; ++i) {
      const Entry e = list[i];
      before += e.order > order ? e.weight : 0.;
      first += e.order > order;
    }
  }
  __device__ __forceinline__ void clear(int rank) {
    for (int b = rank; b < kBins; b += TEAM) {
      mass[b] = 0.;
      count[b] = 0;
    }
  }
  // of a class so far below the largest logit (a NaN, of 0 times infinity, goes to the last bin, with all others)
  static __device__ __forceinline__ int bin_of(float below, float scale) { return (int)__builtin_fminf(below * scale, (float)(kBins - 1)); }
};

// A row in LDS: each thread has written, and reads, its own pieces of it, of VEC neighbouring classes, so that no barrier is
// needed; each wavefront has one stretch of the row, in which its lanes' pieces lie side by side, so that running sums go
// from wavefront to wavefront.  What masks leave out, and what is behind the last class, is -infinity.
template <typename T, int TEAM> struct Stretch {
  using raw = typename T::raw;
  static constexpr int VEC = 16 / (int)sizeof(raw), W = TEAM / 64;
  raw* row;
  int n, all, first, pieces;  // pieces of a row and of this wavefront (each of 64 lanes); this thread's first class
  __device__ __forceinline__ Stretch(raw* lds, int rank, int classes) : row(lds), n(classes) {
    all = (n + 64 * VEC - 1) / (64 * VEC);
    const int w = __builtin_amdgcn_readfirstlane(rank >> 6), from = w * all / W;
    pieces = (w + 1) * all / W - from;
    first = (from * 64 + (rank & 63)) * VEC;
  }
  // the wavefront of a class: the last one that begins at its piece or before
  __device__ __forceinline__ int wave_of(int index) const { return ((index / (64 * VEC) + 1) * W - 1) / all; }
  // Reads the row, several pieces at a time, and shows every logit to `look`.
  template <typename F> __device__ __forceinline__ void fill(const raw* from, const uint8_t* mask, F look) {
    constexpr int kAtOnce = 4;
#pragma unroll 1
    for (int c0 = 0; c0 < pieces; c0 += kAtOnce) {
      raw v[kAtOnce][VEC];
      uint8_t m[kAtOnce][VEC];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int b = first + (c0 + i) * 64 * VEC;
        if (c0 + i < pieces && b + VEC <= n) {
          __builtin_memcpy(v[i], from + b, sizeof(v[i]));
          if (mask) __builtin_memcpy(m[i], mask + b, sizeof(m[i]));
        }
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int b = first + (c0 + i) * 64 * VEC;
        if (c0 + i >= pieces) break;
        if (b + VEC <= n) {
          if (mask) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[i][e] = m[i][e] == 0 ? T::store(kNone) : v[i][e];
          }
          __builtin_memcpy(__builtin_assume_aligned(row + b, 16), v[i], sizeof(v[i]));
#pragma unroll
          for (int e = 0; e < VEC; ++e) look(T::load(v[i][e]));
        } else {  // (behind the row, or the end of it)
#pragma unroll 1
          for (int e = 0; e < VEC; ++e) {
            const raw r = b + e < n && (!mask || mask[b + e] != 0) ? from[b + e] : T::store(kNone);
            row[b + e] = r;
            look(T::load(r));
          }
        }
      }
    }
  }
  template <typename F> __device__ __forceinline__ void piece(int c, F f) const {
    raw v[VEC];
    const int b = first + c * 64 * VEC;
    __builtin_memcpy(v, __builtin_assume_aligned(row + b, 16), sizeof(v));
#pragma unroll
    for (int e = 0; e < VEC; ++e) f(T::load(v[e]), b + e);
  }
  // (four at a time, which are as many as there are registers for)
  template <typename F> __device__ __forceinline__ void each(F f) const {
#pragma unroll 1
    for (int q = 0; q < pieces * (VEC / 4); ++q) {
      const int b = first + q / (VEC / 4) * 64 * VEC + q % (VEC / 4) * 4;
      raw v[4];
      __builtin_memcpy(v, __builtin_assume_aligned(row + b, 4 * sizeof(raw)), sizeof(v));
#pragma unroll
      for (int e = 0; e < 4; ++e) f(T::load(v[e]), b + e);
    }
  }
  // The class at which the running sum of `value` first exceeds `target`, in the wavefront that `before` and `here` say has it:
  // calls `found` in its lane.
  template <typename V, typename F> __device__ __forceinline__ void find(double before, double here, double target, V value, F found) const {
    if (!(before <= target && target < before + here)) return;
#pragma unroll 1
    for (int c = 0; c < pieces; ++c) {
      double sum = 0.;
      piece(c, [&](float x, int index) { sum += value(x, index); });
      const double until = before + sum_until<64>(sum);
      double run = until - sum;
      if (run <= target && target < until) {
        int chosen = -1;
        float logit = 0.f;
        piece(c, [&](float x, int index) {
          run += value(x, index);
          const bool it = chosen < 0 && run > target;
          chosen = it ? index : chosen;
          logit = it ? x : logit;
        });
        found(chosen, logit);
      }
      before = of_lane(until, 63);
      if (target < before) break;
    }
  }
  // The same with the wavefronts of a team sharing the pieces of that one out, where it has more than two: the pieces' sums are added
  // up by all, the one that has the class goes through its piece.  Measured, us by itself / together: 1024 rows of 28 672 classes (7
  // pieces) with top_p 101 / 90, without 39 / 36, 1000 of 8000 (4) 14.7 / 13.4, but 2000 of 4000 (2) 15.6 / 16.7, of 2000 (1) 10.8 / 12.0.
  __device__ __forceinline__ bool many_pieces() const { return TEAM > 64 && all > 2 * W; }
  struct Search {
    double sums[16];  // of the wavefront's pieces, at most 8
    int wave;         // -1 at the start
  };
  template <typename V, typename F>
  __device__ __forceinline__ void find_together(Team<TEAM>& team, Search& search, double before, double here, double target, V value, F found) const {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const bool mine = before <= target && target < before + here;
    if (mine && lane == 0) search.wave = wave;
    team.sync();
    const int who = __builtin_amdgcn_readfirstlane(search.wave);
    const int from = who * all / W, count = who < 0 ? 0 : (who + 1) * all / W - from;
    Stretch of = *this;
    of.first = (from * 64 + lane) * VEC;
#pragma unroll 1
    for (int c = wave; c < count; c += W) {
      double sum = 0.;
      of.piece(c, [&](float x, int index) { sum += value(x, index); });
      sum = over_lanes<64>(sum, [](double a, double b) { return a + b; });
      if (lane == 0) search.sums[c] = sum;
    }
    team.sync();
    if (!mine) return;
    int c = 0;
    for (; c < count - 1 && before + search.sums[c] <= target; ++c) before += search.sums[c];
    double run = 0.;
    double w[VEC];
    int e = 0;
    piece(c, [&](float x, int index) { run += w[e++] = value(x, index); });
    const double until = before + sum_until<64>(run);
    run = until - run;
    if (run <= target && target < until) {
      int chosen = -1;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        run += w[i];
        chosen = chosen < 0 && run > target ? i : chosen;
      }
      const int index = first + c * 64 * VEC + chosen;
      found(index, T::load(row[index]));
    }
  }
};

// The sums before a thread's bins.
template <int TEAM> struct BinSums {
  double run;
  int seen, all;
  __device__ __forceinline__ BinSums(Team<TEAM>& team, CutRoom<TEAM>& m, int rank, bool counted) {
    constexpr int kOwn = CutRoom<TEAM>::kBins / TEAM;
    const int lane = threadIdx.x & 63, wave = rank >> 6;
    double mass = 0.;
    int count = 0;
    all = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      mass += m.mass[rank * kOwn + i];
      if (counted) count += m.count[rank * kOwn + i];
    }
    run = sum_until<64>(mass);
    seen = counted ? sum_until<64>(count) : 0;
    if constexpr (TEAM > 64) {
      if (lane == 63) {
        m.wave_mass[wave] = run;
        m.wave_count[wave] = seen;
      }
      team.sync();
      double behind = 0.;
      int passed = 0;
#pragma unroll
      for (int i = 0; i < TEAM / 64; ++i) {
        behind += i < wave ? m.wave_mass[i] : 0.;
        if (counted) {
          passed += i < wave ? m.wave_count[i] : 0;
          all += m.wave_count[i];
        }
      }
      run += behind;
      seen += passed;
    } else {
      all = of_lane(seen, 63);
    }
    run -= mass;
    seen -= count;
  }
};

// By bins: the weights (for top_k the numbers) of a row's classes are added up in LDS in bins of equal width from the
// largest logit down to the smallest one, or to where weights vanish; the bin in which the sum from the
// top reaches what is looked for is listed, and each of its few classes is ranked against the others.  Three passes over the
// row, whatever the types.  A bin with more classes than the list holds is binned again by itself, unless they are
// all equal: then they are counted off by index.
template <typename T, int TEAM>
__device__ __forceinline__ Cutoff cut_by_bins(const Stretch<T, TEAM>& in, const Weigh<4>& weigh, Team<TEAM>& team, const SampleArgs& a, CutRoom<TEAM>& m, double whole,
                                              float low, float scale) {
  using C = CutRoom<TEAM>;
  constexpr int kOwn = C::kBins / TEAM;
  const int rank = Team<TEAM>::rank();
  Cutoff cut{0, 0x7fffffff};
  bool by_mass = a.top_k == 0, binned = by_mass, whole_row = true;  // (for top_k the numbers are there, but not the weights)
  // the logits that are binned, and how: the whole row by their distances, part of it by their keys, of which two that differ can
  // always be told apart
  float from = weigh.top, to = low;
  uint64_t by = 0;
  double mass_before = 0.;                       // of the logits above them
  int count_before = 0;
  auto inside = [&](float x) { return x <= from && x >= to && x != kNone; };
  auto bin_of = [&](float x) { return whole_row ? C::bin_of(from - x, scale) : (int)((uint64_t)(class_key<T>(from) - class_key<T>(x)) * by >> 32); };
#pragma unroll 1
  for (;; binned = false) {
    if (!binned) {
      team.sync();
      m.clear(rank);
      team.sync();
      in.each([&](float x, int) {
        if (inside(x)) {
          const int b = bin_of(x);
          unsafeAtomicAdd(&m.mass[b], weigh(x));
          if (a.top_k > 0) atomicAdd(&m.count[b], 1);
        }
      });
      team.sync();
    }
    const BinSums<TEAM> sums(team, m, rank, a.top_k > 0);
    double run = sums.run + mass_before;
    int seen = sums.seen + count_before;
    if (!by_mass && whole_row && sums.all <= a.top_k) by_mass = true;  // top_k keeps all
    if (by_mass && !(a.top_p < 1.)) break;
    const double share = a.top_p * whole;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int b = rank * kOwn + i;
      const double one = m.mass[b];
      const int n = a.top_k > 0 ? m.count[b] : 0;
      if (by_mass ? run < share && share <= run + one : seen < a.top_k && a.top_k <= seen + n) {
        m.bin = b;
        m.mass_before = run;
        m.count_before = seen;
        m.listed = 0;
      }
      run += one;
      seen += n;
    }
    team.sync();
    const int bin = m.bin;
    in.each([&](float x, int index) {
      if (inside(x) && bin_of(x) == bin) m.put(class_key<T>(x), index, weigh(x));
    });
    team.sync();
    const int listed = m.listed;
    mass_before = m.mass_before;
    count_before = m.count_before;
    if (listed > C::kList) {
      float most = kNone, least = -kNone;
      in.each([&](float x, int) {
        if (inside(x) && bin_of(x) == bin) {
          most = __builtin_fmaxf(most, x);
          least = __builtin_fminf(least, x);
        }
      });
      team.most_and_least(most, least);
      from = most;
      to = least;
      if (to < from) {
        by = ((uint64_t)C::kBins << 32) / ((uint64_t)(class_key<T>(from) - class_key<T>(to)) + 1);
        whole_row = false;
        continue;
      }
      // all equal: the first few by index, as many as it takes
      const double one = m.list[0].weight;
      const int ties = by_mass ? (int)__builtin_fmin(__builtin_ceil((share - mass_before) / one), (double)PCGRL_MAX_CLASSES) : a.top_k - count_before;
      auto equal = [&](float x, int) { return x == from ? 1. : 0.; };
      double mine = 0., before, here;
      in.each([&](float x, int index) { mine += equal(x, index); });
      team.sum(mine, before, here);
      in.find(before, here, (double)(ties - 1), equal, [&](int index, float x) { m.found = Cutoff{class_key<T>(x), index}; });
      team.sync();
      cut = m.found;
      whole = mass_before + (double)ties * one;
    } else {
      for (int i = rank; i < listed; i += TEAM) {
        const typename C::Entry e = m.list[i];
        double before = mass_before;
        int first = count_before;
        m.rank_of(e.order, before, first);
        const double until = before + e.weight;
        if (by_mass ? before < share && share <= until : first == a.top_k - 1) {
          m.found = C::cutoff(e.order);
          m.mass_until = until;
        }
      }
      team.sync();
      cut = m.found;
      whole = m.mass_until;
    }
    if (by_mass || !(a.top_p < 1.)) break;
    by_mass = true;  // top_p, of what top_k has left
    from = weigh.top;
    to = low;
    mass_before = 0.;
    count_before = 0;
    whole_row = true;
  }
  return cut;
}

// The same for top_p alone, which has the classes of the bins above added up in the pass that lists the bin: sets `mine` to what
// of this thread's classes is kept outside that bin, m.extra to what each wavefront has in it.  False if the list does not
// hold the bin.
template <typename T, int TEAM>
__device__ __forceinline__ bool share_by_bins(const Stretch<T, TEAM>& in, const Weigh<4>& weigh, Team<TEAM>& team, CutRoom<TEAM>& m, double share, double least, float scale,
                                              double& mine) {
  using C = CutRoom<TEAM>;
  constexpr int kOwn = C::kBins / TEAM;
  const int rank = Team<TEAM>::rank();
  const BinSums<TEAM> sums(team, m, rank, false);
  double run = sums.run;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const double one = m.mass[rank * kOwn + i];
    if (run < share && share <= run + one) {
      m.bin = rank * kOwn + i;
      m.mass_before = run;
      m.listed = 0;
    }
    run += one;
  }
  if (rank < TEAM / 64) m.extra[rank] = 0.;
  team.sync();
  const int bin = m.bin;
  mine = 0.;
  in.each([&](float x, int index) {
    const int b = C::bin_of(weigh.top - x, scale);
    const double w = weigh(x);
    mine += b < bin && w >= least ? w : 0.;
    if (b == bin && x != kNone) m.put(class_key<T>(x), index, w);
  });
  team.sync();
  const int listed = m.listed;
  if (listed > C::kList) return false;
  for (int i = rank; i < listed; i += TEAM) {
    const typename C::Entry e = m.list[i];
    double before = m.mass_before;
    int first = 0;
    m.rank_of(e.order, before, first);
    if (before < share) {
      const Cutoff it = C::cutoff(e.order);
      if (share <= before + e.weight) m.found = it;
      if (e.weight >= least) unsafeAtomicAdd(&m.extra[in.wave_of(it.index)], e.weight);
    }
  }
  team.sync();
  return true;
}

// For a top_k that the list holds, with the rest of the bin that it ends in: every class that may be kept is listed, ranked once by its
// logit, for top_k and top_p, and once by its index, for the draw.  False if the list does not hold them, or if top_k keeps all.
template <typename T, int TEAM>
__device__ __forceinline__ bool draw_from_list(const Stretch<T, TEAM>& in, const Weigh<4>& weigh, Team<TEAM>& team, const SampleArgs& a, CutRoom<TEAM>& m, double least,
                                               float scale, double whole, int64_t row) {
  using C = CutRoom<TEAM>;
  constexpr int kOwn = C::kBins / TEAM, kMost = C::kList < TEAM ? C::kList : TEAM;
  const int rank = Team<TEAM>::rank();
  if (rank == 0) m.listed = m.bin = 0;
  const BinSums<TEAM> sums(team, m, rank, true);
  if (sums.all <= a.top_k) return false;
  if (TEAM == 64) team.sync();
  int seen = sums.seen;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int n = m.count[rank * kOwn + i];
    if (seen < a.top_k && a.top_k <= seen + n) m.bin = seen + n <= kMost ? rank * kOwn + i : -1;
    seen += n;
  }
  team.sync();
  const int bin = m.bin;
  if (bin < 0) return false;
  in.each([&](float x, int index) {
    if (x != kNone && C::bin_of(weigh.top - x, scale) <= bin) m.put(class_key<T>(x), index, weigh(x));
  });
  team.sync();
  const int listed = m.listed;
  typename C::Entry e{0, 0.};
  double before = 0.;
  int first = a.top_k;
  if (rank < listed) {
    e = m.list[rank];
    first = 0;
    m.rank_of(e.order, before, first);
    if (first == a.top_k - 1) m.mass_until = before + e.weight;
  }
  team.sync();
  const bool keep = first < a.top_k && (!(a.top_p < 1.) || before < a.top_p * m.mass_until) && e.weight >= least;
  if (rank < listed) m.list[rank].weight = keep ? e.weight : 0.;
  team.sync();
  if (keep) {
    const Cutoff it = C::cutoff(e.order);
    double until = 0., all = 0.;
#pragma unroll 8
    for (int i = 0; i < listed; ++i) {
      const typename C::Entry o = m.list[i];
      until += (uint32_t)o.order >= (uint32_t)e.order ? o.weight : 0.;  // (turned round: an index no larger)
      all += o.weight;
    }
    const double target = uniform_of(a, row) * all;
    if (until > target && until - e.weight <= target) put_draw(a, row, it.index, T::load(in.row[it.index]), weigh.top, whole, weigh.table);
  }
  return true;
}

// Draws of many classes: the row goes to LDS on its way in, where every pass after that reads it, four classes a thread at a time, and
// weights are computed again in each rather than kept: registers for 32 doubles a thread would leave a compute unit room for one row, and
// the phases in which threads wait for each other are what a second row hides.  Without truncations one pass sums the
// weights, and the draw goes through the wavefront that has it.  For top_p the same pass bins them, a second lists the bin
// in which the share is reached and sums what is above it.  For a top_k it counts them, and lists what may be kept.
// Bound by 64-bit instructions, 34 a class in one pass and 87 in the two for top_p (1024 rows of 28 672 in bfloat16, masked: floor of the bytes
// 16.3 us, one pass 37, of which 26 are instructions, with top_p 92, of which 65 are, with a top_k of 50 66, with one of 1000, which is counted
// and then binned, 138), and by waits where rows are few: one row of 16 384 in float32 with top_k 15 us, one of 28 672 with top_p 27.  Cutoffs
// of 16-bit types in 256 and 512 threads keep 8 to 12 bytes a thread in scratch memory.
template <typename T, int TEAM, int HOW> __global__ __launch_bounds__(team_block<TEAM>(), 4) void sample_many_kernel(SampleArgs a) {
  static_assert(TEAM >= 64 && HOW != kSampleBest, "");
  using S = Stretch<T, TEAM>;
  constexpr int kTeams = team_block<TEAM>() / TEAM;
  extern __shared__ __attribute__((aligned(16))) char rows_lds[];
  __shared__ double table[64], room[TEAM > 64 ? 2 * TEAM / 64 : 1];
  __shared__ CutRoom<TEAM> cut_room[HOW == kSampleCut ? kTeams : 1];
  Team<TEAM> team{room};
  CutRoom<TEAM>& m = cut_room[HOW == kSampleCut ? threadIdx.x / TEAM % kTeams : 0];
  fill_powers<TEAM>(table, a.unit);
  __shared__ typename S::Search search;
  const bool searched = HOW == kSampleCut && (a.top_k > 0 || a.top_p < 1.);
  for (int64_t row = (int64_t)blockIdx.x * kTeams + threadIdx.x / TEAM; row < a.n_rows; row += (int64_t)gridDim.x * kTeams) {
    const int rank = team.rank_anew();
    S in(reinterpret_cast<typename T::raw*>(rows_lds + (size_t)(threadIdx.x / TEAM % kTeams) * a.lds_row), rank, a.n);
    float top = kNone, low = -kNone;
    Oddity odd;
    in.fill(static_cast<const typename T::raw*>(a.logits) + row * a.logits_stride, a.mask ? a.mask + row * a.mask_stride : nullptr, [&](float x) {
      top = __builtin_fmaxf(top, x);
      if (HOW == kSampleCut) low = __builtin_fminf(low, x == kNone ? -kNone : x);
      odd.look(x);
    });
    top = odd.seen() ? __builtin_huge_valf() : top;
    if (TEAM > 64 && rank == 0) search.wave = -1;
    if constexpr (HOW == kSampleCut) {
      if (searched) m.clear(rank);
      team.most_and_least(top, low);
    } else {
      top = team.most(top);
    }
    if (!(top < __builtin_huge_valf()) || top == kNone) {
      if (rank == 0) put_nothing(a, row, top);
      continue;
    }
    const Weigh<4> weigh{table, top, a.slope};
    const float range = __builtin_fminf(top - low, a.reach), scale = HOW == kSampleCut && range > 0.f ? (float)CutRoom<TEAM>::kBins / range : 0.f;
    double mine = 0., before, here;
    in.each([&](float x, int) {
      const double w = weigh(x);
      mine += w;
      if (HOW == kSampleCut && searched) {
        const int b = m.bin_of(top - x, scale);
        if (a.top_k == 0) {
          if (w > 0.) unsafeAtomicAdd(&m.mass[b], w);
        } else if (x != kNone) {
          atomicAdd(&m.count[b], 1);
        }
      }
    });
    const double whole = team.sum(mine, before, here);
    double kept = whole;
    const double least = HOW == kSampleCut ? a.least : 0.;
    Cutoff cut{0, 0x7fffffff};
    // what is kept of a class's weight
    auto kept_of = [&](float x, int index) {
      const double v = weigh(x);
      const uint32_t key = class_key<T>(x);
      return HOW != kSampleCut || ((key > cut.key || (key == cut.key && index <= cut.index)) && v >= least) ? v : 0.;
    };
    if constexpr (HOW == kSampleCut) {
      bool summed = false;
      if (searched) {
        if (TEAM == 64) team.sync();
        if (a.top_k > 0 && draw_from_list<T, TEAM>(in, weigh, team, a, m, least, scale, whole, row)) {
          team.sync();
          continue;
        }
        if (a.top_k == 0) {
          summed = share_by_bins<T, TEAM>(in, weigh, team, m, a.top_p * whole, least, scale, mine);
          if (summed) {
            cut = m.found;
            kept = team.sum(mine, before, here, m.extra);
          }
        }
        if (!summed) cut = cut_by_bins<T, TEAM>(in, weigh, team, a, m, whole, low, scale);
      }
      if (!summed) {
        mine = 0.;
        in.each([&](float x, int index) {
          const uint32_t key = class_key<T>(x);  // (top_k may leave none in most places)
          if (__builtin_amdgcn_ballot_w64(key >= cut.key) != 0) mine += kept_of(x, index);
        });
        kept = team.sum(mine, before, here);
      }
    }
    auto found = [&](int index, float logit) { put_draw(a, row, index, logit, top, whole, table); };
    if (in.many_pieces()) in.find_together(team, search, before, here, uniform_of(a, row) * kept, kept_of, found);
    else in.find(before, here, uniform_of(a, row) * kept, kept_of, found);
    if (TEAM > 64 && HOW == kSampleCut) team.sync();  // (the next row's bins are cleared before its first barrier)
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
  double widest;        // rows whose factors are not below it have their gradients in 64 bits: kWidest, or -1, all
  double slope, inv_temperature, low, high;  // the ratio is clipped to [low, high]
  double by, bonus, value_by;  // scale / temperature, that times the entropy's coefficient; scale times the value's
  float bonus_off, least;      // bonus / temperature; -1000 temperatures
};

constexpr int kLossSums = 6;  // rows, policy loss, entropy, value loss, divergence, clipped rows
constexpr int kLossBlocks = 2048;
// The classes' gradients are computed in 32 bits where what they are multiplied by is below this: then a probability may lose what 32
// bits do not hold of it, 2^-150, and the gradient is off by no more than 2^-110.
constexpr double kWidest = 0x1p40;

// The loss and its gradients, a row in the registers of a team: read once, written once.  With y = (x - top) / temperature,
// w = e^y and W the sum of w, log p = y - log W and the entropy is log W - (sum of w y) / W: one pass for both sums, in 64 bits.  The second
// pass needs w, kept in 32 bits, whose rounding is that of the gradient, and log p from x: p (entropy_coef (log p + H) - pull),
// one fused multiply-add and two products a class.  For the class that was chosen 1 - p loses what p has in 32 bits, so that its
// gradient is computed in 64 and written over.  Rows whose factors 32 bits do not hold (very low and very high temperatures, large coefficients,
// ratios beyond e^28 with an advantage below 0, advantages and ratios that are infinite or no number) have all of theirs
// computed in 64 bits, from the logits again.  Sums of rows go to a workgroup's partials, which a second launch joins, in
// the same order always (atomics would not, and have to be cleared first); that launch is 4 us of each figure below.
// Bound by instructions, about 45 a class and 110 a row, which for one lane a row are shared by 64 rows: 2 097 152 rows of
// 7 in bfloat16 35 us (floor of the bytes 18.6), 300 000 of 50 44, 20 000 of 500 20, 1001 of 8505 in float16 23 (7.9), 1024 of 16 384, masked,
// 31.5 (15.5), 500 of 28 672 in float32 35.5 (21.2).  Rows of a wavefront put together in LDS for full stores were not faster (31 to 32 us for the
// gradients alone), nor were eight places for 7 classes (43.9, when seven took 39).
template <typename T, int TEAM, int PER> __global__ __launch_bounds__(team_block<TEAM>(), PER >= 16 || TEAM >= 64 ? 4 : 1) void loss_kernel(LossArgs a) {
  using R = Row<T, TEAM, PER>;
  using raw = typename T::raw;
  __shared__ alignas(16) double room[TEAM > 64 ? 4 * TEAM / 64 : 1];
  __shared__ double table[64], sums[TEAM > 64 ? 1 : kLossSums][4];
  Team<TEAM> team{room};
  fill_powers<TEAM>(table, 1.);
  constexpr int kTeams = team_block<TEAM>() / TEAM;
  double part[kLossSums] = {};
  for (int64_t row = (int64_t)blockIdx.x * kTeams + threadIdx.x / TEAM; row < a.n_rows; row += (int64_t)gridDim.x * kTeams) {
    const raw* logits = static_cast<const raw*>(a.logits) + row * a.logits_stride;
    const uint8_t* mask = a.mask ? a.mask + row * a.mask_stride : nullptr;
    const int action = a.actions[row];
    const bool inside = action >= 0 && action < a.n;
    float x[PER];
    const int rank = team.rank_anew();
    R of(rank, a.n);
    of.load(logits, mask, from_row(row, a.n_rows, a.logits_stride, a.n), from_row(row, a.n_rows, a.mask_stride, a.n), x);
    const float mine = inside && (!mask || mask[action] != 0) ? T::load(logits[action]) : kNone;
    float top = kNone;
    Oddity odd;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      top = __builtin_fmaxf(top, x[j]);
      odd.look(x[j]);
    }
    top = team.most(odd.seen() ? __builtin_huge_valf() : top);
    const bool use = mine != kNone;       // (then something may be chosen)
    float w[PER];
    double whole = 0., spread = 0.;       // sums of the weights, and of the weights times their log2
    forget_classes<TEAM, PER>(x, of.first);
#pragma unroll
    for (int c = 0; c < R::PIECES; ++c) {
      if (!of.has(c)) continue;
#pragma unroll
      for (int i = 0; i < R::VEC; ++i) {
        const int j = c * R::VEC + i;
        // (a class that may not be chosen has the weight of 2^-1000, nothing)
        const double y = __builtin_fmax(((double)x[j] - (double)top) * a.slope, -64000.), e = power_from(table, y);
        w[j] = (float)e;
        done(w[j]);
        whole += e;
        spread = __builtin_fma(e, y, spread);
        part_end(j, whole, spread);
      }
    }
    team.sum_both(whole, spread);
    if (!(top < __builtin_huge_valf())) whole = __builtin_nan("");
    const double log_whole = log_of(table, 1., whole);
    const double part_of = 1. / whole, entropy = log_whole - 0.69314718055994530942 / 64. * (spread * part_of);
    const double logp = ((double)mine - (double)top) * a.inv_temperature - log_whole;
    double pull = 0.;                     // the policy loss's derivative by the log-probability
    if (use) {
      const double adv = (double)a.advantages[row];
      const double change = a.old ? logp - (double)a.old[row] : 0.;
      const double ratio = change == change ? power(table, __builtin_fmin(change * (64. * 1.44269504088896340736), 128000.)) : change;
      const bool clipped = a.old && ((adv > 0. && ratio > a.high) || (adv < 0. && ratio < a.low));
      pull = clipped ? 0. : -adv * ratio;
      if (rank == 0) {
        part[0] += 1.;
        part[1] += !a.old ? -adv * logp : clipped ? -adv * (adv > 0. ? a.high : a.low) : -adv * ratio;
        part[2] += entropy;
        part[4] += ratio - 1. - change;
        part[5] += clipped ? 1. : 0.;
      }
    }
    if (rank == 0) {
      if (a.values) {
        const double off = use ? (double)T::load(static_cast<const raw*>(a.values)[row]) - (double)a.returns[row] : 0.;
        part[3] += .5 * off * off;
        if (a.grad_values) static_cast<raw*>(a.grad_values)[row] = T::store((float)(a.value_by * off));
      }
      if (a.log_probs) a.log_probs[row] = use ? (float)logp : 0.f;
      if (a.entropies) a.entropies[row] = use ? (float)entropy : 0.f;
    }
    if (a.grad_logits) {
      // scale / temperature * p (entropy_coef (log p + entropy) - pull) for each class; the lane of the one chosen, which has
      // pull added, writes it once more
      const double push = a.bonus * (entropy - log_whole) - a.by * pull;
      const double p = power(table, ((double)mine - (double)top) * a.slope) * part_of;
      const float chosen = (float)(a.bonus * p * (logp + entropy) + a.by * pull * (1. - p));
      raw* grad = static_cast<raw*>(a.grad_logits) + row * a.grad_stride;
      if (__builtin_expect(use && !(__builtin_fabs(push) < a.widest), 0)) {
        // (one class after the other, each read once more, so that nothing of this takes registers from the other rows)
        int64_t again = row;
        asm volatile("" : "+v"(again));
        const raw* from = static_cast<const raw*>(a.logits) + again * a.logits_stride;
        const uint8_t* may = a.mask ? a.mask + again * a.mask_stride : nullptr;
#pragma unroll 1
        for (int k = 0; k < of.pieces * R::VEC; ++k) {
          const int j = of.begin(k / R::VEC) + k % R::VEC;
          if (j >= a.n) continue;
          const double off = (double)(may && may[j] == 0 ? kNone : T::load(from[j])) - (double)top, z = off * a.slope;
          const double e = z < -64000. ? 0. : power_from(table, z);
          // (what has no probability has no gradient, whatever it would be times; in a row with a NaN that is one)
          const double g = e > 0. ? e * part_of * (a.bonus * (off * a.inv_temperature) + push) : e * part_of;
          grad[j] = T::store(j == action ? chosen : (float)g);
        }
      } else {
        const float inv = (float)part_of, k4 = (float)push;
        forget_classes<TEAM, PER>(x, of.first);
#pragma unroll
        for (int c = 0; c < R::PIECES; ++c) {
          if (!of.has(c)) continue;
          float g[R::VEC];
#pragma unroll
          for (int e = 0; e < R::VEC; ++e) {
            const int j = c * R::VEC + e;
            // (of a class that may not be chosen w is 0, and the rest is a number)
            g[e] = w[j] * inv * __builtin_fmaf(a.bonus_off, __builtin_fmaxf(x[j] - top, a.least), k4);
            if (!use) g[e] = 0.f;
          }
          of.store(grad, c, g);
          if (use && of.owns(c, action)) grad[action] = T::store(chosen);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  // (the first lane of each team has the sums of its rows)
  if (!a.partial) return;
  double* out = a.partial + (size_t)blockIdx.x * kLossSums;
  if constexpr (TEAM > 64) {
    if (threadIdx.x == 0) {
#pragma unroll
      for (int i = 0; i < kLossSums; ++i) out[i] = part[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kLossSums; ++i) {
      const double v = TEAM == 64 ? part[i] : over_lanes<64>(part[i], [](double a, double b) { return a + b; });
      if ((threadIdx.x & 63) == 0) sums[i][threadIdx.x >> 6] = v;
    }
    __syncthreads();
    if (threadIdx.x < kLossSums) {
      double v = 0.;
      for (int i = 0; i < 4; ++i) v += sums[threadIdx.x][i];
      out[threadIdx.x] = v;
    }
  }
}

// Joins the workgroups' sums, always in the same order: thread t has every 768th of them, all of one kind, read at once (a loop
// that waits for each, a wavefront a kind, took 8 us more for 1280 workgroups).
constexpr int kSumThreads = 128 * kLossSums, kSumsEach = kLossBlocks * kLossSums / kSumThreads;
__global__ __launch_bounds__(kSumThreads) void loss_sums_kernel(const double* partial, int blocks, double entropy_coef, double value_coef,
                                                               double scale, float* stats) {
  __shared__ double some[kSumThreads], sums[kLossSums];
  double v[kSumsEach];
#pragma unroll
  for (int i = 0; i < kSumsEach; ++i) {
    const int at = threadIdx.x + i * kSumThreads;
    v[i] = at < blocks * kLossSums ? partial[at] : 0.;
  }
#pragma unroll
  for (int d = kSumsEach / 2; d > 0; d /= 2) {
#pragma unroll
    for (int i = 0; i < d; ++i) v[i] += v[i + d];
  }
  some[threadIdx.x] = v[0];
  __syncthreads();
  const int which = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (which < kLossSums) {
    const double both = some[which + kLossSums * lane] + some[which + kLossSums * (lane + 64)];
    const double sum = over_lanes<64>(both, [](double a, double b) { return a + b; });
    if (lane == 0) sums[which] = sum;
  }
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
  double discount, decay, least;  // decay: discount * trace; least: of a product of them
};

constexpr int kAdvantageThreads = 256, kAdvantageSteps = 8;
// workgroups that share the steps of their environments out: one launch sums up what each group of steps makes
// of the advantage behind it (a factor and a term), one turns these into the advantage behind each group,
// one computes the advantages
constexpr int kAdvantageAll = 0, kAdvantageSum = 1, kAdvantageApply = 2;
constexpr int kAdvantageEach = 8;  // groups of a thread of the launch in the middle

// A stretch of steps makes term + factor * behind of the advantage behind it.  A factor of -1 is the end of an episode in it:
// what is behind that does not count, be it infinite or no number.  Products stop at `least`, 1e-300, so that what is infinite
// stays so over however many steps (a finite advantage times that is nothing); with a decay of 0 they are 0.
__device__ __forceinline__ double after_it(double factor, double term, double behind) { return factor < 0. ? term : __builtin_fma(factor, behind, term); }
__device__ __forceinline__ double both_factors(double front, double back, double least) {
  return front < 0. || back < 0. ? -1. : __builtin_fmax(front * back, least);
}

// Between the launches the factor and the term of group g + 1, and then the advantage behind group g, lie in the
// first rows of group g's own advantages, which the last launch reads before it writes them.
__device__ __forceinline__ void put(float* at, int64_t n, double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  at[0] = __uint_as_float((uint32_t)u);
  at[n] = __uint_as_float((uint32_t)(u >> 32));
}
__device__ __forceinline__ double take(const float* at, int64_t n) {
  return __longlong_as_double((long long)((uint64_t)__float_as_uint(at[0]) | (uint64_t)__float_as_uint(at[n]) << 32));
}

// What the threads of a workgroup behind this one make of the advantage behind them all: thread c E + e has steps behind
// those of thread (c - 1) E + e.  Sets `behind` to the advantage behind this thread's steps and returns that before the
// workgroup's first; `factor_all`, if asked for, is multiplied by all factors.
template <bool ALL> __device__ __forceinline__ double join_steps(int envs_log2, double least, double factor, double term, double& behind, double& factor_all,
                                                                   double (*factors)[64], double (*terms)[64]) {
  constexpr int kWaves = kAdvantageThreads / 64;
  const int E = 1 << envs_log2, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // within a wavefront: this thread's steps and all behind them
  double f = factor, t = term;
  for (int d = E; d < 64; d <<= 1) {
    const double f2 = __shfl_down(f, d), t2 = __shfl_down(t, d);
    if (lane + d < 64) {
      t = after_it(f, t, t2);
      f = both_factors(f, f2, least);
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
    if (ALL) factor_all = both_factors(factors[w][col], factor_all, least);
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
// Bound by memory for many environments: 32 steps of 262 144 with bfloat16 values, 126 MB, 22.5 us where its arrays stay the same from call to
// call (5.6 TB/s; a large copy reaches 5.4, as none of it stays in the last-level cache); by the latency of a load and a join, 2.5 us, and of a launch
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
        factor = end ? -1. : both_factors(a.decay, factor, a.least);
        ends |= end ? 1u << i : 0u;
      }
    }
    if (top - C * L > lo) fetch(base - C * L);
    if (C > 1) {
      behind = join_steps<MODE == kAdvantageSum>(a.envs_log2, a.least, factor, term, mine, factor_all, factors, terms);
    } else {
      behind = after_it(factor, term, behind);
      factor_all = both_factors(factor, factor_all, a.least);
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
    factor = both_factors(f[i], factor, a.least);
  }
  double behind = 0., unused = 1.;
  join_steps<false>(a.envs_log2, a.least, factor, term, behind, unused, factors, terms);
#pragma unroll
  for (int i = kAdvantageEach - 1; i >= 0; --i) {
    if (live && i < each && first + i < groups - 1) {
      behind = after_it(f[i], t[i], behind);
      put(a.advantages + (int64_t)(first + i) * a.group * n + env, n, behind);
    }
  }
}

}  // namespace pcgrl
