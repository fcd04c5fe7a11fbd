// The next token of every sequence from its logits: temperature, top-k, top-p and min-p, drawn by a given random number.
//
// Tokens stand in order of falling logit, equal ones in order of their ids.  Token v weighs w_v = exp((z_v - max) / temperature); what the
// filters keep are first parts of that order, and the draw takes the first token at which the sum of the weights so far exceeds u
// times the sum of all that is kept.  Sums have to be right to the last token: a row may hold 150,000 tokens of like weight, and
// an error of 1e-7 of the sum would draw another one now and then.  Weights are therefore whole multiples of 2^-42 of the largest one
// (from a series in 64 bits, weight_of()), and every sum is one of integers: exact, and the same in any order, atomics
// included.  A token below 2^-43 of the largest weight weighs nothing.
//
// A workgroup of 1024 threads has a row:
//   A  the maximum; of the threads' own maxima the k-th largest (without top-k the 400th) gives a line above which all tokens
//      that matter usually lie, and not many more than that;
//   B  a second pass lists the tokens above the line (in LDS, 1024 at most) and sums all weights where they are asked for;
//   C  the list is sorted and its sums formed: counts, masses and the draw are looked up.
// Rows that this does not settle (nearly flat ones, where hundreds of tokens are kept, or many equal ones) go by
//   D  a histogram of counts and masses over 2048 equal steps of (max - z) / temperature.  Where a count or mass falls, the
//      step's tokens are listed and sorted as in C, after further histograms of it where there are too many.
#include "bc_common.h"

namespace bc {
namespace {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kListed = 1024;              // tokens a sorted list holds
constexpr int kSteps = 2048;               // of a histogram
constexpr int kWeightBits = 42;            // the largest token weighs 2^42
constexpr float kSpan = 43.5f;             // base-2 exponents a histogram covers: weights below 2^-43 round to nothing
constexpr int kUsualLine = 400;            // thread maxima above the line without top-k: 0.5 tokens a thread, 512 in all

struct SampleParams {
  const char* z;
  int64_t row_bytes;
  const float* temperature;    // [B], each nullable but u
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  const uint8_t* active;
  int32_t* token;
  float* logprob;
  int32_t V;
};

typedef unsigned long long u64;

__device__ __forceinline__ float sample_value(uint32_t bits, float) { return __uint_as_float(bits); }
__device__ __forceinline__ float sample_value(uint32_t bits, bf16_t) { return __uint_as_float(bits << 16); }

// f(z, token) of every logit of a row, which may start at any element: those in front of the first 16-byte boundary and behind the last are
// taken one by one, the others by 16 bytes, four loads of a thread at a time.
template <typename T, typename F>
__device__ __forceinline__ void each_logit(const char* row, int32_t V, const F& f) {
  constexpr int EPU = Elem<T>::per16, ES = Elem<T>::size, BATCH = 4;
  const int head = min(((16 - (int)(reinterpret_cast<uintptr_t>(row) & 15u)) & 15) / ES, V);
  const int units = (V - head) / EPU, tail = V - head - units * EPU, tid = threadIdx.x;
  if (tid < head + tail) {
    const int i = tid < head ? tid : V - tail + tid - head;
    uint32_t bits;
    if constexpr (ES == 4) bits = reinterpret_cast<const uint32_t*>(row)[i];
    else bits = reinterpret_cast<const uint16_t*>(row)[i];
    f(sample_value(bits, T{}), i);
  }
  const uint4* at = reinterpret_cast<const uint4*>(row + head * ES);
  for (int base = 0; base < units; base += BATCH * kSampleThreads) {
    uint4 r[BATCH];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int unit = base + b * kSampleThreads + tid;
      if (unit < units) r[b] = at[unit];
    }
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int unit = base + b * kSampleThreads + tid;
      if (unit < units) {
        float x[EPU];
        unpack16(r[b], x, T{});
#pragma unroll
        for (int e = 0; e < EPU; ++e) f(x[e], head + unit * EPU + e);
      }
    }
  }
}

// What the threads share.
struct SampleLds {
  uint32_t count[kSteps];
  u64 mass[kSteps];
  u64 list[kListed];
  u64 wave64[kSampleWaves];
  uint32_t wave32[kSampleWaves];
  float wavef[kSampleWaves];
  uint32_t n;
  u64 found_mass, found_item, found_first, found_last;
  uint32_t found_count;
};

__device__ __forceinline__ u64 shuffle_up(u64 x, int by) {
  const uint32_t lo = __shfl_up((uint32_t)x, by, 64), hi = __shfl_up((uint32_t)(x >> 32), by, 64);
  return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 shuffle_xor(u64 x, int by) {
  const uint32_t lo = __shfl_xor((uint32_t)x, by, 64), hi = __shfl_xor((uint32_t)(x >> 32), by, 64);
  return (u64)hi << 32 | lo;
}
template <typename N>
__device__ __forceinline__ N wave_scan(N x) {          // sum of this lane's and all before it
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    N y;
    if constexpr (sizeof(N) == 8) y = shuffle_up(x, o); else y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  return x;
}
// The same over the workgroup; `waves`: kSampleWaves in LDS.
template <typename N>
__device__ __forceinline__ N block_scan(N x, N* waves) {
  x = wave_scan(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  N before = 0;
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) before += w < (int)(threadIdx.x >> 6) ? waves[w] : 0;
  return x + before;
}
template <typename N>
__device__ __forceinline__ N block_sum(N x, N* waves) {
  x = wave_scan(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  N all = 0;
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) all += waves[w];
  return all;
}
__device__ __forceinline__ float block_max(float x, float* waves) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  float all = waves[0];
#pragma unroll
  for (int w = 1; w < kSampleWaves; ++w) all = fmaxf(all, waves[w]);
  return all;
}

// Place of a token in the order as one number, smaller in front: the logit's bits turned so that they fall with it, then the id.
__device__ __forceinline__ u64 item_of(float z, int token) {
  const uint32_t b = __float_as_uint(z + 0.f);                // (-0 is 0)
  const uint32_t falling = b & 0x80000000u ? b : ~b & 0x7fffffffu;
  return (u64)falling << 32 | (uint32_t)token;
}
__device__ __forceinline__ float logit_of(u64 item) {
  const uint32_t f = (uint32_t)(item >> 32);
  return __uint_as_float(f & 0x80000000u ? f : ~f & 0x7fffffffu);
}

// One row's scale.
struct Scale {
  float max;
  double rate;                 // log2(e) / temperature
  float steps;                 // steps of the histogram per unit of (max - z) / 2
  double temperature;
  __device__ __forceinline__ Scale(float m, double t) : max(m), rate(1.4426950408889634074 / t), temperature(t) {
    steps = (float)fmin(rate * (2 * kSteps / kSpan), 1e30);       // (finite: max - z may be zero)
  }
  // step of a logit; kSteps and more: it weighs nothing (-inf too).  Rises with max - z whatever is rounded.
  __device__ __forceinline__ int step(float z) const { return (int)fminf((0.5f * max - 0.5f * z) * steps, (float)kSteps); }
  // 2^42 exp((z - max) / temperature) to the nearest integer: 2^(whole + part) with the series of 2^part (next term 2^-47)
  __device__ __forceinline__ u64 weight(float z) const {
    const double e = kWeightBits - ((double)max - (double)z) * rate;
    if (!(e > -2.0)) return 0;
    const double whole = __builtin_rint(e), x = (e - whole) * 0.69314718055994530942;
    double y = 1.0 / 39916800;
    y = __builtin_fma(y, x, 1.0 / 3628800);
    y = __builtin_fma(y, x, 1.0 / 362880);
    y = __builtin_fma(y, x, 1.0 / 40320);
    y = __builtin_fma(y, x, 1.0 / 5040);
    y = __builtin_fma(y, x, 1.0 / 720);
    y = __builtin_fma(y, x, 1.0 / 120);
    y = __builtin_fma(y, x, 1.0 / 24);
    y = __builtin_fma(y, x, 1.0 / 6);
    y = __builtin_fma(y, x, 0.5);
    y = __builtin_fma(y, x, 1.0);
    y = __builtin_fma(y, x, 1.0);
    // y * 2^whole + 2^52: the integer in the low bits
    const double two = __longlong_as_double((long long)(1023 + (int)whole) << 52);
    return (u64)__double_as_longlong(__builtin_fma(y, two, 4503599627370496.0)) & 0xfffffffffffffull;
  }
  __device__ __forceinline__ bool above(float z, double log_min) const { return ((double)z - (double)max) / temperature >= log_min; }
};

// The listed items in order, one a thread; `n` of them.
__device__ __forceinline__ u64 sort_list(SampleLds& s, int n) {
  const int tid = threadIdx.x;
  u64 x = tid < n ? s.list[tid] : ~0ull;
  int size = 64;
  while (size < n) size <<= 1;
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j >= 1; j >>= 1) {
      u64 y;
      if (j >= 64) {
        __syncthreads();
        s.list[tid] = x;
        __syncthreads();
        y = s.list[tid ^ j];
      } else {
        y = shuffle_xor(x, j);
      }
      const bool keep_small = ((tid & j) == 0) == ((tid & k) == 0);
      x = (y < x) == keep_small ? y : x;
    }
  return x;
}

// A sorted list with its sums.
struct Sorted {
  int n;
  u64 item, weight, upto;      // this thread's; upto: weights of the list up to and with it
  u64 all;
  __device__ __forceinline__ Sorted(SampleLds& s, int count, const Scale& sc) : n(count) {
    item = sort_list(s, n);
    weight = (int)threadIdx.x < n ? sc.weight(logit_of(item)) : 0;
    upto = block_scan(weight, s.wave64);
    all = 0;
#pragma unroll
    for (int w = 0; w < kSampleWaves; ++w) all += s.wave64[w];
  }
  // how many items end at or before a mass
  __device__ __forceinline__ int until(u64 mass) const { return __syncthreads_count((int)threadIdx.x < n && upto <= mass); }
  // the item at a place and the mass up to and with it, for every thread
  __device__ __forceinline__ void at(SampleLds& s, int place, u64& the_item, u64& the_mass) const {
    __syncthreads();
    if ((int)threadIdx.x == place) { s.found_item = item; s.found_mass = upto; }
    __syncthreads();
    the_item = s.found_item;
    the_mass = s.found_mass;
  }
};

__device__ __forceinline__ void clear_steps(SampleLds& s, bool masses) {
  __syncthreads();
  for (int i = threadIdx.x; i < kSteps; i += kSampleThreads) {
    s.count[i] = 0;
    if (masses) s.mass[i] = 0;
  }
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
}
// Counts and masses of the steps -> those in front of each step (the totals in the return value).
struct Totals { uint32_t count; u64 mass; };
__device__ __forceinline__ Totals sum_steps(SampleLds& s) {
  __syncthreads();
  const int i = 2 * threadIdx.x;
  const uint32_t c0 = s.count[i], c1 = s.count[i + 1];
  const u64 m0 = s.mass[i], m1 = s.mass[i + 1];
  const uint32_t c = block_scan(c0 + c1, s.wave32);
  const u64 m = block_scan(m0 + m1, s.wave64);
  Totals t{0, 0};
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) { t.count += s.wave32[w]; t.mass += s.wave64[w]; }
  s.count[i] = c - c0 - c1; s.count[i + 1] = c - c1;
  s.mass[i] = m - m0 - m1; s.mass[i + 1] = m - m1;
  __syncthreads();
  return t;
}

// What is looked for in the order: the first token at which the count so far reaches `count` (mass: the weights so far exceed it).
struct Target { bool by_count; uint32_t count; u64 mass; };
// The step in which it lies; steps hold what is in front of them.  The caller has made sure that it lies in one.
struct Place { int step; uint32_t before_count, count; u64 before_mass; };
__device__ __forceinline__ Place step_of(SampleLds& s, const Target& t, const Totals& all, uint32_t base_count, u64 base_mass) {
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int i = 2 * threadIdx.x + e;
    const bool last = i == kSteps - 1;
    const uint32_t c0 = s.count[i], c1 = last ? all.count : s.count[i + 1];
    const u64 m0 = s.mass[i], m1 = last ? all.mass : s.mass[i + 1];
    const bool here = t.by_count ? base_count + c0 < t.count && t.count <= base_count + c1
                                 : base_mass + m0 <= t.mass && t.mass < base_mass + m1;
    if (here) { s.found_first = i; s.found_count = c0; s.n = c1 - c0; s.found_mass = m0; }
  }
  __syncthreads();
  Place p{(int)s.found_first, base_count + s.found_count, s.n, base_mass + s.found_mass};
  __syncthreads();
  return p;
}

struct Found { u64 item, mass; };       // mass: up to and with it

// Looks a target up in a row whose first histogram (sc.step()) is in `s`, as sum_steps() leaves it, and keeps it there.
template <typename T>
__device__ __noinline__ Found look_up(SampleLds& s, const char* row, int32_t V, const Scale& sc, const Totals& all, const Target& t) {
  // the first histogram is put by: two counts and masses a thread
  Place at = step_of(s, t, all, 0, 0);
  const int i = 2 * threadIdx.x;
  const uint32_t keep_c0 = s.count[i], keep_c1 = s.count[i + 1];
  const u64 keep_m0 = s.mass[i], keep_m1 = s.mass[i + 1];
  u64 lo = 0, hi = ~0ull;
  const int step = at.step;
  if (at.count > kListed) {             // its items' ends, from which further histograms cut
    u64 first = ~0ull, last = 0;
    each_logit<T>(row, V, [&](float z, int token) {
      if (sc.step(z) == step) {
        const u64 x = item_of(z, token);
        first = x < first ? x : first;
        last = x > last ? x : last;
      }
    });
    __syncthreads();
    if (threadIdx.x == 0) { s.found_first = ~0ull; s.found_last = 0; }
    __syncthreads();
    atomicMin(&s.found_first, first);
    atomicMax(&s.found_last, last);
    __syncthreads();
    lo = s.found_first;
    hi = s.found_last;
  }
  for (int level = 0; level < 7 && at.count > kListed; ++level) {      // (11 bits of 64 each)
    const int bits = 64 - __clzll((long long)(hi - lo)), shift = bits > 11 ? bits - 11 : 0;
    clear_steps(s, true);
    each_logit<T>(row, V, [&](float z, int token) {
      if (sc.step(z) != step) return;
      const u64 x = item_of(z, token);
      if (x < lo || x > hi) return;
      const int n = (int)((x - lo) >> shift);
      atomicAdd(&s.count[n], 1u);
      atomicAdd(&s.mass[n], sc.weight(z));
    });
    const Totals sub = sum_steps(s);
    at = step_of(s, t, sub, at.before_count, at.before_mass);
    lo += (u64)at.step << shift;
    const u64 end = lo + ((1ull << shift) - 1);
    hi = end < hi ? end : hi;
  }
  __syncthreads();
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
  each_logit<T>(row, V, [&](float z, int token) {
    if (sc.step(z) != step) return;
    const u64 x = item_of(z, token);
    if (x < lo || x > hi) return;
    const uint32_t n = atomicAdd(&s.n, 1u);
    if (n < kListed) s.list[n] = x;
  });
  __syncthreads();
  const Sorted list(s, (int)at.count, sc);
  const int place = t.by_count ? (int)(t.count - at.before_count) - 1 : list.until(t.mass - at.before_mass);
  Found f;
  list.at(s, place, f.item, f.mass);
  f.mass += at.before_mass;
  __syncthreads();
  s.count[i] = keep_c0; s.count[i + 1] = keep_c1;
  s.mass[i] = keep_m0; s.mass[i + 1] = keep_m1;
  __syncthreads();
  return f;
}

// floor(u * mass), below it
__device__ __forceinline__ u64 part_of(float u, u64 mass) {
  const double x = (double)u * (double)mass;
  const u64 y = x > 0.0 ? (u64)x : 0;
  return y < mass ? y : mass - 1;
}
// The mass that a kept token ends beyond first: tokens whose mass in front is below p * mass are kept.
__device__ __forceinline__ u64 cut_of(float p, u64 mass) {
  const double x = ceil((double)p * (double)mass);
  const u64 y = x >= 1.0 ? (u64)x : 1;
  return (y < mass ? y : mass) - 1;
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(SampleParams p) {
  __shared__ SampleLds s;
  const int b = blockIdx.x;
  if (p.active && !p.active[b]) return;
  const char* row = p.z + (int64_t)b * p.row_bytes;
  float t = p.temperature ? p.temperature[b] : 1.f;
  int k = p.top_k ? p.top_k[b] : 0;
  const float top_p = p.top_p ? p.top_p[b] : 1.f, min_p = p.min_p ? p.min_p[b] : 0.f, u = p.u[b];
  if (t == 0.f) { t = 1.f; k = 1; }                    // the largest alone

  // A
  float mine = -__builtin_inff();
  bool bad = !(t > 0.f && t < __builtin_inff()) || u != u;
  each_logit<T>(row, p.V, [&](float z, int) {
    mine = fmaxf(mine, z);
    bad = bad || !(z < __builtin_inff());
  });
  const float max = block_max(mine, s.wavef);
  if (__syncthreads_or(bad) || !(max > -__builtin_inff())) {
    if (threadIdx.x == 0) {
      p.token[b] = -1;
      if (p.logprob) p.logprob[b] = __builtin_nanf("");
    }
    return;
  }
  const Scale sc(max, (double)t);
  const bool by_k = k > 0 && k < p.V, by_p = top_p < 1.f, by_m = min_p > 0.f;
  const double log_min = by_m ? log((double)min_p) : 0.0;

  // the line: the step in which the wanted number of thread maxima is reached
  const uint32_t wanted = by_k ? (uint32_t)k : (uint32_t)kUsualLine;
  clear_steps(s, false);
  {
    const int step = sc.step(mine);
    if (step < kSteps) atomicAdd(&s.count[step], 1u);
  }
  __syncthreads();
  if (threadIdx.x == 0) s.found_first = kSteps - 1;
  const uint32_t c0 = s.count[2 * threadIdx.x], c1 = s.count[2 * threadIdx.x + 1], upto = block_scan(c0 + c1, s.wave32);
  if (upto >= wanted && upto - c0 - c1 < wanted) s.found_first = 2 * threadIdx.x + (upto - c1 >= wanted ? 0 : 1);
  __syncthreads();
  const int line = (int)s.found_first;

  // B
  const bool sum_all = !by_k && (by_p || !by_m);
  u64 sum = 0;
  each_logit<T>(row, p.V, [&](float z, int token) {
    const int step = sc.step(z);
    if (step <= line) {
      const uint32_t n = atomicAdd(&s.n, 1u);
      if (n < kListed) s.list[n] = item_of(z, token);
    }
    if (sum_all && step < kSteps) sum += sc.weight(z);
  });
  u64 all = sum_all ? block_sum(sum, s.wave64) : 0;
  __syncthreads();
  const int listed = (int)s.n;
  const bool complete = line == kSteps - 1;            // all that weighs anything is listed

  // C
  u64 item = 0, kept = 0;
  bool settled = false;
  if (listed <= kListed) {
    const Sorted list(s, listed, sc);
    u64 other;
    if (complete) all = list.all;
    bool known = true;
    kept = all;
    if (by_k) {
      if (k <= listed) list.at(s, k - 1, other, kept);
      else if (complete) kept = list.all;
      else known = false;
    }
    if (known && by_p) {
      const u64 cut = cut_of(top_p, kept);
      if (cut < list.all) list.at(s, list.until(cut), other, kept);
      else known = false;
    }
    if (by_m) {
      const int above = __syncthreads_count((int)threadIdx.x < listed && sc.above(logit_of(list.item), log_min));
      u64 m = 1ull << kWeightBits;                     // (the largest is always kept)
      if (above > 0) list.at(s, above - 1, other, m);
      const bool alone = !by_k && !by_p;
      if (above < listed || complete) {
        // (what lies behind the list is lower still, and a cut by top-p that is not settled lies behind it)
        kept = !alone && known && kept < m ? kept : m;
        known = true;
      } else if (alone || !known || kept > list.all) {
        known = false;
      }
    }
    if (known) {
      const u64 mass = part_of(u, kept);
      if (mass < list.all) {
        list.at(s, list.until(mass), item, other);
        settled = true;
      }
    }
  }

  // D
  if (!settled) {
    clear_steps(s, true);
    each_logit<T>(row, p.V, [&](float z, int) {
      const int step = sc.step(z);
      if (step < kSteps) {
        atomicAdd(&s.count[step], 1u);
        atomicAdd(&s.mass[step], sc.weight(z));
      }
    });
    const Totals total = sum_steps(s);
    kept = total.mass;
    if (by_k && (uint32_t)k < total.count) kept = look_up<T>(s, row, p.V, sc, total, Target{true, (uint32_t)k, 0}).mass;
    if (by_p) kept = look_up<T>(s, row, p.V, sc, total, Target{false, 0, cut_of(top_p, kept)}).mass;
    if (by_m) {
      // whole steps in front of the one the limit falls into, give or take one, and what of those three is above it
      const double limit = -0.5 * log_min * sc.temperature * (double)sc.steps;
      const int near = (int)fmin(fmax(limit, 0.0), (double)kSteps), from = near > 0 ? near - 1 : 0;
      u64 m = 0;
      each_logit<T>(row, p.V, [&](float z, int) {
        const int step = sc.step(z);
        if (step >= from && step <= near + 1 && step < kSteps && sc.above(z, log_min)) m += sc.weight(z);
      });
      m = block_sum(m, s.wave64) + (from < kSteps ? s.mass[from] : total.mass);
      m = m < 1ull << kWeightBits ? 1ull << kWeightBits : m;
      kept = m < kept ? m : kept;
    }
    item = look_up<T>(s, row, p.V, sc, total, Target{false, 0, part_of(u, kept)}).item;
  }
  if (threadIdx.x == 0) {
    p.token[b] = (int32_t)(uint32_t)item;
    if (p.logprob)
      p.logprob[b] = (float)(((double)logit_of(item) - (double)max) / sc.temperature - log((double)kept * (1.0 / (1ull << kWeightBits))));
  }
}

}  // namespace
}  // namespace bc

using namespace bc;

extern "C" int32_t bc_sample_tokens(int32_t B, int32_t V, const void* logits, int32_t logits_dtype, int64_t row_stride, const float* temperature,
                                    const int32_t* top_k, const float* top_p, const float* min_p, const float* u, const uint8_t* active,
                                    int32_t* tokens, float* logprob, void* stream) {
  if (logits_dtype != BC_F32 && logits_dtype != BC_BF16) return BC_ERR_SHAPE;
  if (B < 0 || V < 1 || V > (1 << 20)) return BC_ERR_SHAPE;
  if (B == 0) return BC_OK;
  const int es = elem_size(logits_dtype);
  if (!logits || !u || !tokens || (reinterpret_cast<uintptr_t>(logits) & (es - 1))) return BC_ERR_ARG;
  if (row_stride < V && B > 1) return BC_ERR_ARG;
  if (row_stride > (1LL << 40)) return BC_ERR_ARG;
  SampleParams p{static_cast<const char*>(logits), row_stride * es, temperature, top_k, top_p, min_p, u, active, tokens, logprob, V};
  if (logits_dtype == BC_BF16) sample_kernel<bf16_t><<<B, kSampleThreads, 0, as_stream(stream)>>>(p);
  else sample_kernel<float><<<B, kSampleThreads, 0, as_stream(stream)>>>(p);
  return launch_status();
}
