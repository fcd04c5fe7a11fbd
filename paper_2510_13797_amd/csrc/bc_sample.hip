// The next token of every sequence from its logits: temperature, top-k, top-p and min-p, drawn by a given random number.
//
// Tokens stand in order of falling logit, equal ones in order of their ids.  Token v weighs w_v = exp((z_v - max) / temperature); what the
// filters keep are first parts of that order, and the draw takes the first token at which the sum of the weights so far exceeds u
// times the sum of all that is kept.  Sums have to be right to the last token: a row may hold 150,000 tokens of like weight, and
// an error of 1e-7 of the sum would draw another one now and then.  Weights are therefore whole multiples of 2^-42 of the largest one
// (from a series in 64 bits, Scale::weight()), and every sum is one of integers: exact, and the same in any order, atomics
// included.  A token below 2^-43 of the largest weight weighs nothing.
//
// A workgroup of 1024 threads has a row:
//   A  the maximum; of the threads' own maxima the k-th largest (without top-k the 200th) gives a line above which all tokens
//      that matter usually lie, and not many more than that;
//   B  a second pass lists the tokens above the line (in LDS, 1024 at most).  Where the sum of all weights is asked for, it adds up those below
//      the line in 32 bits, with a bound on how far off that is (Scale::tail_sum());
//   C  the list is sorted and its sums formed: counts, masses and the draw are looked up, at both ends of the bound where there is one.
// Rows that this does not settle (nearly flat ones, where hundreds of tokens are kept, many equal ones, a border inside the bound) go by
//   D  sums of whole rows.  bf16 logits have few values: their counts are taken in LDS, and a value weighs its count times its weight (151,936 equal logits
//      131 us, zeros 87; zeros by the fp32 way 377).  fp32 logits go by a
//      histogram of counts and masses over 2048 equal steps of (max - z) / temperature; where a count or mass falls, the step's
//      tokens are listed and sorted as in C, after further histograms of it where there are too many.
//
// What bounds it is the vector work of a compute unit that has a row to itself, 148 logits a thread at V = 151,936: passes A and B look at 16
// bytes at a time by packed 16-bit comparisons (bf16; 32-bit ones for fp32) and at single logits only where one is above the line.
#include "bc_common.h"

namespace bc {
namespace {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kAtOnce = 10;                // loads of a thread that are waited for together
constexpr int kListed = 1024;              // tokens a sorted list holds
constexpr int kSteps = 2048;               // of a histogram
constexpr int kWeightBits = 42;            // the largest token weighs 2^42
constexpr float kSpan = 43.5f;             // base-2 exponents a histogram covers: weights below 2^-43 round to nothing
constexpr int kUsualLine = 200;            // thread maxima above the line without top-k: some 220 tokens
constexpr int kValues = 4096;              // bf16 values counted: 16 binades of either sign,
constexpr int kCopies = 2;                 // odd and even lanes apart, so that fewer meet at a count
constexpr int kZeros = kValues + 1;         // (a place in name alone)
constexpr int kNowhere = 64;               // counts for logits of no place, a lane's own each

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
constexpr double kTailBound = 1.0 / (1 << 17);

__device__ __forceinline__ float sample_value(uint32_t bits, float) { return __uint_as_float(bits); }
__device__ __forceinline__ float sample_value(uint32_t bits, bf16_t) { return __uint_as_float(bits << 16); }

// A row, which may start at any element: those in front of the first 16-byte boundary and behind the last are taken one by one (single(bits,
// token)), the others by 16 bytes (unit(words, first token)), BATCH loads of a thread at a time: kAtOnce where there is little to do
// with them; fewer where there is more, with the next ones on their way meanwhile (AHEAD).
template <typename T, int BATCH, bool AHEAD, typename FS, typename FU>
__device__ __forceinline__ void each_unit(const char* row, int32_t V, const FS& single, const FU& unit_of) {
  constexpr int EPU = Elem<T>::per16, ES = Elem<T>::size;
  const int head = min(((16 - (int)(reinterpret_cast<uintptr_t>(row) & 15u)) & 15) / ES, V);
  const int units = (V - head) / EPU, tail = V - head - units * EPU, tid = threadIdx.x;
  if (tid < head + tail) {
    const int i = tid < head ? tid : V - tail + tid - head;
    if constexpr (ES == 4) single(reinterpret_cast<const uint32_t*>(row)[i], i);
    else single((uint32_t)reinterpret_cast<const uint16_t*>(row)[i], i);
  }
  // (every load is made, that of the last unit behind the row's end: where they were conditional, each waited for the one before it)
  typedef __attribute__((address_space(1))) const u32x4_t global_unit_t;
  const global_unit_t* at = (const global_unit_t*)(row + head * ES);
  const auto load = [&](uint4 (&r)[BATCH], int base) {
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const u32x4_t x = at[min(base + b * kSampleThreads + tid, units - 1)];
      r[b] = make_uint4(x.x, x.y, x.z, x.w);
    }
  };
  const auto work = [&](const uint4 (&r)[BATCH], int base) {
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int unit = base + b * kSampleThreads + tid;
      if (unit < units) unit_of(r[b], head + unit * EPU);
    }
  };
  constexpr int STEP = BATCH * kSampleThreads;
  if (units == 0) return;
  if constexpr (!AHEAD) {
    for (int base = 0; base < units; base += STEP) {
      uint4 r[BATCH];
      load(r, base);
      work(r, base);
    }
  } else {
    uint4 r[BATCH], n[BATCH];
    load(r, 0);
    for (int base = 0; base < units; base += 2 * STEP) {
      load(n, base + STEP);
      work(r, base);
      load(r, base + 2 * STEP);
      work(n, base + STEP);
    }
  }
}
// f(z, token) of every logit
template <typename T, typename F>
__device__ __forceinline__ void each_logit(const char* row, int32_t V, const F& f) {
  each_unit<T, 4, false>(row, V, [&](uint32_t bits, int token) { f(sample_value(bits, T{}), token); }, [&](const uint4& r, int token) {
    float x[Elem<T>::per16];
    unpack16(r, x, T{});
#pragma unroll
    for (int e = 0; e < Elem<T>::per16; ++e) f(x[e], token + e);
  });
}

// Logits as signed integers: not negative ones rise with the value, negative ones fall.  The largest and smallest integer of some logits tell their
// maximum, the largest unsigned one whether a NaN with a sign is among them, and the lowest if one has a sign.
typedef __attribute__((ext_vector_type(2))) short pair16_t;
typedef __attribute__((ext_vector_type(2))) unsigned short upair16_t;
struct Ends16 {                // of bf16, packed
  pair16_t most = {-32768, -32768}, least = {32767, 32767};
  upair16_t umost = {0, 0};
  __device__ __forceinline__ void add(uint32_t w) {
    const pair16_t x = __builtin_bit_cast(pair16_t, w);
    most = __builtin_elementwise_max(most, x);
    least = __builtin_elementwise_min(least, x);
    umost = __builtin_elementwise_max(umost, __builtin_bit_cast(upair16_t, w));
  }
  __device__ __forceinline__ void add(const uint4& r) { add(r.x); add(r.y); add(r.z); add(r.w); }
  __device__ __forceinline__ void one(uint32_t bits) { add(bits * 0x10001u); }
  __device__ __forceinline__ void finish(float& max, float& low, bool& bad) const {
    const int hi = most.x > most.y ? most.x : most.y, lo = least.x < least.y ? least.x : least.y;
    const uint32_t u = umost.x > umost.y ? umost.x : umost.y;
    const bool any = hi >= lo;
    max = any ? __uint_as_float((uint32_t)(hi >= 0 ? hi : lo & 0xffff) << 16) : -__builtin_inff();
    low = any ? __uint_as_float((u >= 0x8000u ? u : (uint32_t)lo) << 16) : __builtin_inff();
    bad = any && (hi >= 0x7f80 || u > 0xff80u);
  }
};
struct Ends32 {
  int32_t most = INT32_MIN, least = INT32_MAX;
  uint32_t umost = 0;
  __device__ __forceinline__ void one(uint32_t bits) {
    most = max(most, (int32_t)bits);
    least = min(least, (int32_t)bits);
    umost = max(umost, bits);
  }
  __device__ __forceinline__ void add(const uint4& r) { one(r.x); one(r.y); one(r.z); one(r.w); }
  __device__ __forceinline__ void finish(float& max, float& low, bool& bad) const {
    const bool any = most >= least;
    max = any ? __uint_as_float((uint32_t)(most >= 0 ? most : least)) : -__builtin_inff();
    low = any ? __uint_as_float(umost >= 0x80000000u ? umost : (uint32_t)least) : __builtin_inff();
    bad = any && (most >= 0x7f800000 || umost > 0xff800000u);
  }
};
template <typename T> using Ends = std::conditional_t<std::is_same<T, float>::value, Ends32, Ends16>;

// Whether one of the logits of 16 bytes may be at or above a line, given as its integer (rounded down): exact for fp32.
struct Line {
  float z;
  int32_t i;
  __device__ __forceinline__ Line(float z_, float) : z(z_), i((int32_t)__float_as_uint(z_)) {}
  __device__ __forceinline__ Line(float z_, bf16_t) : z(z_) {
    const uint32_t b = __float_as_uint(z_);
    i = (int16_t)((b >> 16) + ((b & 0x80000000u) && (b & 0xffffu) ? 1 : 0));
  }
  template <typename N> __device__ __forceinline__ bool reached(N most, N least) const {
    return i >= 0 ? most >= i : most >= 0 || least <= i;
  }
  __device__ __forceinline__ bool reached(const uint4& r, float) const {
    const int32_t a = (int32_t)r.x, b = (int32_t)r.y, c = (int32_t)r.z, d = (int32_t)r.w;
    const int32_t most = max(max(a, b), max(c, d));
    return reached(most, i >= 0 ? most : min(min(a, b), min(c, d)));
  }
  __device__ __forceinline__ bool reached(const uint4& r, bf16_t) const {
    const pair16_t a = __builtin_bit_cast(pair16_t, r.x), b = __builtin_bit_cast(pair16_t, r.y), c = __builtin_bit_cast(pair16_t, r.z),
                   d = __builtin_bit_cast(pair16_t, r.w);
    const pair16_t most = __builtin_elementwise_max(__builtin_elementwise_max(a, b), __builtin_elementwise_max(c, d));
    const int32_t hi = most.x > most.y ? most.x : most.y;
    if (i >= 0) return hi >= i;
    const pair16_t least = __builtin_elementwise_min(__builtin_elementwise_min(a, b), __builtin_elementwise_min(c, d));
    return reached(hi, (int32_t)(least.x < least.y ? least.x : least.y));
  }
};

// What the threads share.
struct SampleLds {
  union {
    struct { u64 mass[kSteps]; uint32_t count[kSteps]; };
    float lows[kSampleThreads];                          // (in place of masses)
    uint32_t value_count[(kValues + kNowhere) * kCopies];
  };
  u64 list[kListed];
  u64 wave64[kSampleWaves];
  uint32_t wave32[kSampleWaves];
  float wavef[kSampleWaves];
  double waved[kSampleWaves];
  uint32_t n;
  u64 found_mass, found_item, found_first, found_last, found_weight;
  uint32_t found_count, found_kind;
};

// x of the lane whose number differs in bit J (of 64 lanes), by the vector units: through LDS (two shuffles for 64 bits) a sort of 512 took 10 us, 3 so.
template <int J>
__device__ __forceinline__ uint32_t across(uint32_t x) {
  if constexpr (J == 1) return __builtin_amdgcn_update_dpp(x, x, kDppXor1, 0xf, 0xf, true);
  else if constexpr (J == 2) return __builtin_amdgcn_update_dpp(x, x, kDppXor2, 0xf, 0xf, true);
  else if constexpr (J == 4) {           // 7 - i, then 3 - i inside a quad
    const uint32_t y = __builtin_amdgcn_update_dpp(x, x, kDppHalfMirror, 0xf, 0xf, true);
    return __builtin_amdgcn_update_dpp(y, y, 0x1B, 0xf, 0xf, true);
  } else if constexpr (J == 8) return __builtin_amdgcn_update_dpp(x, x, 0x128, 0xf, 0xf, true);      // turned by eight of sixteen
  else if constexpr (J == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  }
}
template <int J>
__device__ __forceinline__ u64 across64(u64 x) { return (u64)across<J>((uint32_t)(x >> 32)) << 32 | across<J>((uint32_t)x); }
// x of another lane, zero where there is none (row: 16 lanes; mask: rows that take it)
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t from_before(uint32_t x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 from_before(u64 x) {
  return (u64)from_before<CTRL, ROWS>((uint32_t)(x >> 32)) << 32 | from_before<CTRL, ROWS>((uint32_t)x);
}
template <typename N>
__device__ __forceinline__ N wave_scan(N x) {          // sum of this lane's and all before it
  x += from_before<0x111, 0xf>(x);                      // 1, 2, 4, 8 lanes back inside a row,
  x += from_before<0x112, 0xf>(x);
  x += from_before<0x114, 0xf>(x);
  x += from_before<0x118, 0xf>(x);
  x += from_before<0x142, 0xa>(x);                      // the last of a row to the next, of two rows to the next two
  x += from_before<0x143, 0xc>(x);
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
__device__ __forceinline__ double block_sum_double(double x, double* waves) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  double all = 0.0;
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

// The row's lowest logit.
__device__ __forceinline__ float lowest_of(SampleLds& s) { return -block_max(-s.lows[threadIdx.x], s.wavef); }

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
  float rate_hi, offset;       // the rate in 32 bits, max times it
  // low: the row's lowest logit, below which steps need not reach (151,936 normal logits of 0.001, which are within a few steps of kSpan: 610 us, 127 so)
  __device__ __forceinline__ Scale(float m, double t, float low = -__builtin_inff()) : max(m), rate(1.4426950408889634074 / t), temperature(t) {
    rate_hi = (float)rate;
    offset = max * rate_hi;
    steps = (float)fmin(fmax(rate * (2 * kSteps / kSpan), 0.999 * 2 * kSteps / ((double)m - (double)low)), 1e30);       // (finite: max - z may be zero)
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
  // exp((z - max) / temperature) in 32 bits, but for factors that all have in common: its exponent is z * rate_hi - offset, rounded once
  // (half a step of less than 2^6, 2^-19 * ln 2), and tail_sum() puts right what the rounding of rate and offset did to it, the former (kSpan * 2^-24 * ln 2 at most) from
  // some of the exponents.  With the instruction's 2^-23 and sums of eight, 3 * 2^-24, below 2^-18: kTailBound is twice that.  (Weights beyond kSpan, which round to
  // nothing, stay in: less than V altogether.)  The offset's rounding moves all exponents by half a step of it: where that is more than a half, as for logits
  // of 20 and a temperature of 1e-6, rows are left to D (beyond offsets of 2^31 it was more than 126, and weights and their sums not finite).
  // A token is right whatever the bound; the share of one drawn from a row that no filter cuts is as good as this sum.  What counts of that lies above
  // 2^-32 (V of them are 2^-12 of the largest): half a step of less than 2^5 and the rate's, (2^-20 + 2^-19) ln 2, 2^-23 and 3 * 2^-24 are 2.3e-6 of it; 6e-7
  // measured, 300 tokens over 151,635 of one value, where roundings do not even out.  (All weights in 64 bits instead, where a share is asked for:
  // one such row 28 -> 51 us, 64 rows of mixed settings 30.5 -> 53.)
  __device__ __forceinline__ float tail_exponent(float z) const { return __builtin_fmaf(z, rate_hi, -offset); }
  __device__ __forceinline__ bool tail_fits() const { return fabsf(offset) < 16777216.f; }
  __device__ __forceinline__ double tail_sum(double weights, double mean_exponent) const {
    return weights * exp2((double)offset - (double)max * (double)rate_hi) * (1.0 + 0.69314718055994531 * mean_exponent * ((rate - (double)rate_hi) / rate));
  }
  __device__ __forceinline__ bool above(float z, double log_min) const { return ((double)z - (double)max) / temperature >= log_min; }
};

// The listed items in order, one a thread: bitonic, in registers inside a wave.  Waves without items keep to the barriers.
template <int J>
__device__ __forceinline__ void sort_step(u64& x, bool falling) {
  const u64 y = across64<J>(x);
  const bool keep_small = ((threadIdx.x & J) == 0) != falling;
  x = (y < x) == keep_small ? y : x;
}
template <int J>
__device__ __forceinline__ void sort_steps(u64& x, bool falling) {      // J, J / 2 ... 1
  sort_step<J>(x, falling);
  if constexpr (J > 1) sort_steps<J / 2>(x, falling);
}
template <bool WAVE>
__device__ __forceinline__ u64 sort_list(SampleLds& s, int n) {
  const int tid = threadIdx.x;
  u64 x = tid < n ? s.list[tid] : ~0ull;
  int size = 64;
  if constexpr (!WAVE)
    while (size < n) size <<= 1;
  const bool mine = (tid & ~63) < size;                  // (a wave's)
  if (mine) {
    sort_steps<1>(x, tid & 2);
    sort_steps<2>(x, tid & 4);
    sort_steps<4>(x, tid & 8);
    sort_steps<8>(x, tid & 16);
    sort_steps<16>(x, tid & 32);
    sort_steps<32>(x, !WAVE && (tid & 64));
  }
  if constexpr (!WAVE) {
    for (int k = 128; k <= size; k <<= 1) {
      for (int j = k >> 1; j >= 64; j >>= 1) {
        __syncthreads();
        s.list[tid] = x;
        __syncthreads();
        const u64 y = s.list[tid ^ j];
        x = (y < x) == (((tid & j) == 0) == ((tid & k) == 0)) ? y : x;
      }
      if (mine) sort_steps<32>(x, tid & k);
    }
  }
  return x;
}

// A sorted list with its sums.  WAVE: of 64 items at most, by the first wave alone, without barriers.
template <bool WAVE>
struct Sorted {
  SampleLds& s;
  int n;
  u64 item, weight, upto;      // this thread's; upto: weights of the list up to and with it
  u64 all;
  __device__ __forceinline__ Sorted(SampleLds& lds, int count, const Scale& sc) : s(lds), n(count) {
    item = sort_list<WAVE>(s, n);
    weight = (int)threadIdx.x < n ? sc.weight(logit_of(item)) : 0;
    if constexpr (WAVE) {
      upto = wave_scan(weight);
      all = from_lane(upto, 63);
    } else {
      upto = block_scan(weight, s.wave64);
      all = 0;
#pragma unroll
      for (int w = 0; w < kSampleWaves; ++w) all += s.wave64[w];
    }
  }
  static __device__ __forceinline__ u64 from_lane(u64 x, int lane) {
    const uint32_t lo = __shfl((uint32_t)x, lane, 64), hi = __shfl((uint32_t)(x >> 32), lane, 64);
    return (u64)hi << 32 | lo;
  }
  __device__ __forceinline__ int how_many(bool mine) const {
    if constexpr (WAVE) return __popcll(__ballot(mine));
    else return __syncthreads_count(mine);
  }
  // how many items end at or before a mass
  __device__ __forceinline__ int until(u64 mass) const { return how_many((int)threadIdx.x < n && upto <= mass); }
  // the item at a place and the mass up to and with it, for every thread
  __device__ __forceinline__ void at(int place, u64& the_item, u64& the_mass) const {
    if constexpr (WAVE) {
      the_item = from_lane(item, place & 63);
      the_mass = from_lane(upto, place & 63);
    } else {
      __syncthreads();
      if ((int)threadIdx.x == place) { s.found_item = item; s.found_mass = upto; }
      __syncthreads();
      the_item = s.found_item;
      the_mass = s.found_mass;
    }
  }
  __device__ __forceinline__ u64 mass_at(int place) const {
    u64 i, m;
    at(place, i, m);
    return m;
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
__device__ __noinline__ Found look_up(SampleLds& s, const char* row, int32_t V, float max, float low, double temperature, Totals all, Target t) {
  const Scale sc(max, temperature, low);
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
  const Sorted<false> list(s, (int)at.count, sc);
  const int place = t.by_count ? (int)(t.count - at.before_count) - 1 : list.until(t.mass - at.before_mass);
  Found f;
  list.at(place, f.item, f.mass);
  f.mass += at.before_mass;
  __syncthreads();
  s.count[i] = keep_c0; s.count[i + 1] = keep_c1;
  s.mass[i] = keep_m0; s.mass[i + 1] = keep_m1;
  __syncthreads();
  return f;
}

// a / b of a quotient below 2^32, by 64-bit floating point and what that is off
__device__ __forceinline__ u64 quotient(u64 a, u64 b) {
  u64 q = (u64)((double)a / (double)b);
  if (q * b > a) --q;
  return (q + 1) * b <= a ? q + 1 : q;
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

// What a row asks for.
struct Wish {
  bool by_k, by_p, by_m;
  int k;
  float top_p, u;
  double log_min;
};
struct Drawn { u64 item, kept; bool settled; };

// C: from the list of all tokens above a line.  complete: all that weigh anything.  tail: what the others weigh, in 32 bits.
template <bool WAVE>
__device__ __forceinline__ Drawn draw_from_list(SampleLds& s, int listed, const Scale& sc, const Wish& w, bool complete, double tail, int V) {
  const Sorted<WAVE> list(s, listed, sc);
  Drawn d{0, 0, false};
  u64 other;
  // the mass of all lies from lo to hi
  u64 lo = list.all, hi = list.all;
  if (!complete) {
    // (and the weights' rounding to integers, and sums of eight that held listed ones)
    const u64 off = (u64)(tail * kTailBound) + (list.all >> 21) + (u64)V;
    d.kept = list.all + (u64)tail;
    lo = d.kept > list.all + off ? d.kept - off : list.all;
    hi = d.kept + off;
  } else {
    d.kept = list.all;
  }
  bool known = true;           // what is kept, but for all of lo to hi
  u64 least = 0;               // ... and if not, at least so much
  if (w.by_k) {
    if (w.k <= listed) { d.kept = list.mass_at(w.k - 1); lo = hi = d.kept; }
    else if (!complete) { known = false; least = list.all; }
  }
  if (known && w.by_p) {
    const int place = list.until(cut_of(w.top_p, lo));
    const u64 upto = place < listed ? list.mass_at(place) : list.all;
    if (place < listed && (lo == hi || place == list.until(cut_of(w.top_p, hi)))) d.kept = lo = hi = upto;
    else { known = false; least = upto; }
  }
  if (w.by_m) {
    const int above = list.how_many((int)threadIdx.x < listed && sc.above(logit_of(list.item), w.log_min));
    const u64 m = above > 0 ? list.mass_at(above - 1) : 1ull << kWeightBits;       // (the largest is always kept)
    const bool all_known = above < listed || complete;                              // (what lies behind the list is lower still)
    if (all_known && (known ? lo != hi || m < lo : m <= least)) { d.kept = lo = hi = m; known = true; }
    else if (!all_known) known = known && lo == hi && hi <= list.all;
  }
  if (known) {
    const int place = list.until(part_of(w.u, lo));
    if (place < listed && (lo == hi || place == list.until(part_of(w.u, hi)))) {
      list.at(place, d.item, other);
      d.settled = true;
    }
  }
  return d;
}

// D for bf16 logits.  Values of 16 binades of either sign stand in falling order at 4096 places; those nearer to zero, which come between the signs, in
// a list, and zeros, between its signs, as a count.  Not settled: too many in the list.
struct ValueSums {
  SampleLds& s;
  uint32_t c[4];               // this thread's four places
  u64 w[4];
  uint32_t before_count, near_count, all_count;        // near: list and zeros
  u64 before_mass, near_mass, all_mass, half_mass;
  uint32_t half_count;
  uint32_t zeros, over_count;  // over: of the list, above zero
  u64 zero_weight, over_mass;
  // place, its first token's count and mass, and what each of its tokens weighs, for every thread; kValues: the list near zero (zeros in front of what is below
  // them), kZeros
  struct At { uint32_t place, before_count; u64 before_mass, weight; };
  __device__ __forceinline__ At find(const Target& t) {
    __syncthreads();
    uint32_t cc = before_count;
    u64 m = before_mass;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool here = t.by_count ? cc < t.count && t.count <= cc + c[e] : m <= t.mass && t.mass < m + c[e] * w[e];
      if (here) { s.found_kind = 4 * threadIdx.x + e; s.found_count = cc; s.found_mass = m; s.found_weight = w[e]; }
      cc += c[e];
      m += c[e] * w[e];
    }
    if (threadIdx.x == 0) {
      const auto within = [&](uint32_t c0, uint32_t c1, u64 m0, u64 m1) {
        return t.by_count ? c0 < t.count && t.count <= c1 : m0 <= t.mass && t.mass < m1;
      };
      const u64 zero_mass = zeros * zero_weight;
      if (within(half_count, half_count + near_count, half_mass, half_mass + near_mass)) {
        const uint32_t c0 = half_count + over_count;
        const u64 m0 = half_mass + over_mass;
        const bool zero = within(c0, c0 + zeros, m0, m0 + zero_mass), over = within(half_count, c0, half_mass, m0);
        s.found_kind = zero ? kZeros : kValues;
        s.found_count = zero ? c0 : half_count + (over ? 0 : zeros);
        s.found_mass = zero ? m0 : half_mass + (over ? 0 : zero_mass);
        s.found_weight = zero ? zero_weight : 0;
      }
    }
    __syncthreads();
    return At{s.found_kind, s.found_count, s.found_mass, s.found_weight};
  }
};
__device__ __forceinline__ Drawn draw_from_values(SampleLds& s, const char* row, int32_t V, const Scale& sc, float low, const Wish& w) {
  const float max = sc.max;
  const int tid = threadIdx.x;
  Drawn d{0, 0, false};
  // the lowest logit that weighs anything (or that there is: 151,936 normal ones of 0.001 would not fit the list, 622 us for 60), and the binades: down from the larger magnitude of it and the largest
  const float lowest = fmaxf((float)fmax((double)max - (double)kSpan / sc.rate, -3.4028234663852886e38), low);
  const uint32_t top = __float_as_uint(fmaxf(fabsf(max), fabsf(lowest))) >> 23, a0 = top > 15 ? (top - 15) << 7 : 1;        // (zeros are equal whatever their sign: never a place of their own)
  __syncthreads();
  for (int i = tid; i < (kValues + kNowhere) * kCopies; i += kSampleThreads) s.value_count[i] = 0;
  if (tid == 0) s.n = s.found_count = 0;
  __syncthreads();
  // place of a value, less than kValues for one of the binades and only for those: magnitude less a0, turned for a positive one, then the lane's count there as
  // bytes (two values at a time).  Places below the lowest logit are counted, and weigh nothing.
  const auto packed = [](int x) { return (uint32_t)x * 0x10001u; };
  const upair16_t from = __builtin_bit_cast(upair16_t, packed(a0)), nowhere = __builtin_bit_cast(upair16_t, packed(kValues + (tid & (kNowhere - 1))));
  const uint32_t copy = packed(4 * (tid & (kCopies - 1)));
  const auto places = [&](uint32_t x, uint32_t magnitude) {
    const upair16_t v = __builtin_bit_cast(upair16_t, magnitude) - from;
    const uint32_t sign = __builtin_bit_cast(uint32_t, __builtin_bit_cast(pair16_t, x) >> 15);
    const upair16_t turned = __builtin_bit_cast(upair16_t, __builtin_bit_cast(uint32_t, v) ^ (~sign & 0x07ff07ffu));
    const upair16_t at = __builtin_elementwise_min(__builtin_elementwise_add_sat(turned, __builtin_bit_cast(upair16_t, sign & 0x08000800u)), nowhere);
    static_assert((kValues + kNowhere) * kCopies * 4 <= 65536 && kCopies == 2, "bytes of a place");
    return __builtin_bit_cast(uint32_t, at << (unsigned short)3) | copy;
  };
  char* const counts = reinterpret_cast<char*>(s.value_count);
  const auto count = [&](uint32_t at) { atomicAdd(reinterpret_cast<uint32_t*>(counts + at), 1u); };
  uint32_t zero = 0;
  const auto near_zero = [&](uint32_t h, int token) {
    if ((h & 0x7fffu) < a0) {
      const float z = __uint_as_float(h << 16);
      if (z == 0.f) {
        ++zero;
      } else if (z >= lowest) {
        const uint32_t n = atomicAdd(&s.n, 1u);
        if (n < kListed) s.list[n] = item_of(z, token);
      }
    }
  };
  each_unit<bf16_t, 5, true>(row, V, [&](uint32_t h, int token) {
    count(places(h, h & 0x7fffu) & 0xffffu);
    near_zero(h, token);
  }, [&](const uint4& r, int token) {
    const uint32_t x[4] = {r.x, r.y, r.z, r.w};
    upair16_t least = {0xffff, 0xffff};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t magnitude = x[e] & 0x7fff7fffu, at = places(x[e], magnitude);
      least = __builtin_elementwise_min(least, __builtin_bit_cast(upair16_t, magnitude));
      count(at & 0xffffu);
      count(at >> 16);
    }
    if (least.x < a0 || least.y < a0)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        near_zero(x[e] & 0xffffu, token + 2 * e);
        near_zero(x[e] >> 16, token + 2 * e + 1);
      }
  });
  if (zero != 0) atomicAdd(&s.found_count, zero);
  __syncthreads();
  const int listed = (int)s.n;
  const uint32_t zeros = lowest <= 0.f ? s.found_count : 0;
  if (listed > kListed) return d;
  const Sorted<false> near(s, listed, sc);
  const auto value_at = [&](int place) {
    const uint32_t v = place < kValues / 2 ? (uint32_t)place ^ 0x7ffu : (uint32_t)place ^ 0x800u;
    return __uint_as_float(((v + a0) | (place < kValues / 2 ? 0u : 0x8000u)) << 16);
  };
  ValueSums x{s};
  uint32_t cc = 0;
  u64 m = 0, above = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int place = 4 * tid + e;
    x.c[e] = 0;
#pragma unroll
    for (int n = 0; n < kCopies; ++n) x.c[e] += s.value_count[place * kCopies + n];
    x.w[e] = x.c[e] ? sc.weight(value_at(place)) : 0;
    cc += x.c[e];
    m += x.c[e] * x.w[e];
    if (w.by_m && x.c[e] && sc.above(value_at(place), w.log_min)) above += x.c[e] * x.w[e];
  }
  x.zeros = zeros;
  x.zero_weight = x.zeros ? sc.weight(0.f) : 0;
  x.over_count = x.zeros ? (uint32_t)near.how_many(tid < listed && logit_of(near.item) > 0.f) : (uint32_t)listed;
  x.over_mass = !x.zeros ? near.all : x.over_count ? near.mass_at((int)x.over_count - 1) : 0;
  x.near_count = (uint32_t)listed + x.zeros;
  x.near_mass = near.all + x.zeros * x.zero_weight;
  const uint32_t upto_count = block_scan(cc, s.wave32);
  x.half_count = 0; x.all_count = x.near_count;
#pragma unroll
  for (int i = 0; i < kSampleWaves; ++i) {
    if (i < kSampleWaves / 2) x.half_count += s.wave32[i];
    x.all_count += s.wave32[i];
  }
  const u64 upto_mass = block_scan(m, s.wave64);
  x.half_mass = 0; x.all_mass = x.near_mass;
#pragma unroll
  for (int i = 0; i < kSampleWaves; ++i) {
    if (i < kSampleWaves / 2) x.half_mass += s.wave64[i];
    x.all_mass += s.wave64[i];
  }
  const bool behind = tid >= kSampleThreads / 2;
  x.before_count = upto_count - cc + (behind ? x.near_count : 0);
  x.before_mass = upto_mass - m + (behind ? x.near_mass : 0);

  // up to and with what a target finds
  const auto mass_at = [&](const Target& t) {
    const ValueSums::At at = x.find(t);
    if (at.place == kValues) {
      const int place = t.by_count ? (int)(t.count - at.before_count) - 1 : near.until(t.mass - at.before_mass);
      return at.before_mass + near.mass_at(place);
    }
    return t.by_count ? at.before_mass + (u64)(t.count - at.before_count) * at.weight
                      : at.before_mass + (quotient(t.mass - at.before_mass, at.weight) + 1) * at.weight;
  };
  d.kept = x.all_mass;
  if (w.by_k && (uint32_t)w.k < x.all_count) d.kept = mass_at(Target{true, (uint32_t)w.k, 0});
  if (w.by_p) d.kept = mass_at(Target{false, 0, cut_of(w.top_p, d.kept)});
  if (w.by_m) {
    if (tid < listed && sc.above(logit_of(near.item), w.log_min)) above += near.weight;
    if (tid == 0 && x.zeros && sc.above(0.f, w.log_min)) above += x.zeros * x.zero_weight;
    u64 least = block_sum(above, s.wave64);
    least = least < 1ull << kWeightBits ? 1ull << kWeightBits : least;
    d.kept = least < d.kept ? least : d.kept;
  }
  const u64 mass = part_of(w.u, d.kept);
  const ValueSums::At at = x.find(Target{false, 0, mass});
  u64 other;
  if (at.place == kValues) {
    near.at(near.until(mass - at.before_mass), d.item, other);
    d.settled = true;
    return d;
  }
  // which of the equal ones: by id
  const bool is_zero = at.place == kZeros;
  uint32_t equal = is_zero ? x.zeros : 0;
  if (!is_zero)
#pragma unroll
    for (int n = 0; n < kCopies; ++n) equal += s.value_count[at.place * kCopies + n];
  const uint32_t h = is_zero ? 0u : __float_as_uint(value_at((int)at.place)) >> 16, both = h * 0x10001u;
  const uint32_t bits_of = is_zero ? 0x7fff7fffu : ~0u;        // (a zero's sign does not count)
  uint32_t rank = (uint32_t)quotient(mass - at.before_mass, at.weight);
  // f(a token, or the first of a unit that has some; how many; the unit) of those
  const auto each_equal = [&](const auto& single, const auto& some) {
    each_unit<bf16_t, kAtOnce, false>(row, V, [&](uint32_t bits, int token) {
      if ((bits & bits_of) == h) single(token);
    }, [&](const uint4& r, int token) {
      const uint32_t x[4] = {r.x & bits_of, r.y & bits_of, r.z & bits_of, r.w & bits_of};
      // (a half that is equal is zero: the smaller ones of two and two)
      const auto diff = [&](int e) { return __builtin_bit_cast(upair16_t, x[e] ^ both); };
      const upair16_t least = __builtin_elementwise_min(__builtin_elementwise_min(diff(0), diff(1)), __builtin_elementwise_min(diff(2), diff(3)));
      if (least.x == 0 || least.y == 0) some(x, token);
    });
  };
  __syncthreads();
  int stretch = -1;
  if (equal > kListed) {       // too many for the list: those of the 512 tokens among which it is (a unit goes by its first)
    for (int i = tid; i < kSteps; i += kSampleThreads) s.count[i] = 0;
    __syncthreads();
    each_equal([&](int token) { atomicAdd(&s.count[token >> 9], 1u); }, [&](const uint32_t (&x)[4], int token) {
      uint32_t n = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) n += ((x[e] & 0xffffu) == h) + (x[e] >> 16 == h);
      atomicAdd(&s.count[token >> 9], n);
    });
    __syncthreads();
    const uint32_t c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1], upto = block_scan(c0 + c1, s.wave32), before = upto - c0 - c1;
    if (before <= rank && rank < upto) {
      const bool second = rank >= before + c0;
      s.found_kind = 2 * tid + (second ? 1 : 0);
      s.found_count = before + (second ? c0 : 0);
    }
    __syncthreads();
    stretch = (int)s.found_kind;
    rank -= s.found_count;
  }
  if (tid == 0) s.n = 0;
  __syncthreads();
  const auto note = [&](int token) {
    const uint32_t n = atomicAdd(&s.n, 1u);
    if (n < kListed) s.list[n] = item_of(__uint_as_float(h << 16), token);
  };
  each_equal([&](int token) { if (stretch < 0 || token >> 9 == stretch) note(token); }, [&](const uint32_t (&x)[4], int token) {
    if (stretch < 0 || token >> 9 == stretch)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if ((x[e] & 0xffffu) == h) note(token + 2 * e);
        if (x[e] >> 16 == h) note(token + 2 * e + 1);
      }
  });
  __syncthreads();
  const u64 items = sort_list<false>(s, (int)s.n);
  __syncthreads();
  if (tid == (int)rank) s.found_item = items;
  __syncthreads();
  d.item = s.found_item;
  d.settled = true;
  return d;
}

// D for any logits.  It and look_up() are functions of their own: inline, their registers cost the other ways (one row 12.8 -> 14.8 us) and each other (a
// flat fp32 row 109 -> 129); a call saves a hundred registers a thread in memory, which is little beside their passes (and was a third of draw_from_values()).
template <typename T>
__device__ __noinline__ Drawn draw_from_steps(SampleLds& s, const char* row, int32_t V, float max, double temperature, Wish w) {
  // (bf16: draw_from_values() has written over them)
  const float low = std::is_same<T, float>::value ? lowest_of(s) : -__builtin_inff();
  const Scale sc(max, temperature, low);
  clear_steps(s, true);
  each_logit<T>(row, V, [&](float z, int) {
    const int step = sc.step(z);
    if (step < kSteps) {
      const u64 same = __ballot(z == __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(z)))), all = __ballot(true);
      if (same == all) {       // (one value throughout: once for all lanes, which would meet at one step)
        if ((threadIdx.x & 63) == __builtin_ctzll(all)) {
          const uint32_t n = (uint32_t)__popcll(all);
          atomicAdd(&s.count[step], n);
          atomicAdd(&s.mass[step], sc.weight(z) * n);
        }
      } else {
        atomicAdd(&s.count[step], 1u);
        atomicAdd(&s.mass[step], sc.weight(z));
      }
    }
  });
  const Totals total = sum_steps(s);
  Drawn d{0, total.mass, true};
  // top-k's last token, top-p's, the draw: one after the other
#pragma clang loop unroll(disable)
  for (int stage = 0; stage < 3; ++stage) {
    Target t{stage == 0, (uint32_t)w.k, 0};
    if (stage == 0) {
      if (!w.by_k || (uint32_t)w.k >= total.count) continue;
    } else if (stage == 1) {
      if (!w.by_p) continue;
      t.mass = cut_of(w.top_p, d.kept);
    } else {
      if (w.by_m) {
        // whole steps in front of the one the limit falls into, give or take one, and what of those three is above it
        const double limit = -0.5 * w.log_min * sc.temperature * (double)sc.steps;
        const int near = (int)fmin(fmax(limit, 0.0), (double)kSteps), from = near > 0 ? near - 1 : 0;
        u64 m = 0;
        each_logit<T>(row, V, [&](float z, int) {
          const int step = sc.step(z);
          if (step >= from && step <= near + 1 && step < kSteps && sc.above(z, w.log_min)) m += sc.weight(z);
        });
        m = block_sum(m, s.wave64) + (from < kSteps ? s.mass[from] : total.mass);
        m = m < 1ull << kWeightBits ? 1ull << kWeightBits : m;
        d.kept = m < d.kept ? m : d.kept;
      }
      t.mass = part_of(w.u, d.kept);
    }
    const Found f = look_up<T>(s, row, V, max, low, temperature, total, t);
    if (stage < 2) d.kept = f.mass; else d.item = f.item;
  }
  return d;
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(SampleParams p) {
  __shared__ SampleLds s;
  const int b = blockIdx.x;
  if (p.active && !p.active[b]) return;
  const char* row = p.z + (int64_t)b * p.row_bytes;
  float t = p.temperature ? p.temperature[b] : 1.f;
  Wish w;
  w.k = p.top_k ? p.top_k[b] : 0;
  w.top_p = p.top_p ? p.top_p[b] : 1.f;
  const float min_p = p.min_p ? p.min_p[b] : 0.f;
  w.u = p.u[b];
  for (int i = threadIdx.x; i < kSteps; i += kSampleThreads) s.count[i] = 0;
  if (threadIdx.x == 0) { s.n = 0; s.found_first = kSteps - 1; }
  if (t >= 0.f && t < 1.17549435e-38f) { t = 1.f; w.k = 1; }      // the largest alone (log2(e) / t fits 32 bits otherwise)

  // A
  float mine, low;
  bool bad;
  Ends<T> ends;
  each_unit<T, kAtOnce, false>(row, p.V, [&](uint32_t bits, int) { ends.one(bits); }, [&](const uint4& r, int) { ends.add(r); });
  ends.finish(mine, low, bad);
  s.lows[threadIdx.x] = low;                             // (of use to D alone: kept in a register, 17.6 us of an fp32 row were 18.7)
  bad = bad || !(t > 0.f && t < __builtin_inff()) || w.u != w.u;
  const float max = block_max(mine, s.wavef) + 0.f;      // (-0 is 0)
  if (__syncthreads_or(bad) || !(max > -__builtin_inff())) {
    if (threadIdx.x == 0) {
      p.token[b] = -1;
      if (p.logprob) p.logprob[b] = __builtin_nanf("");
    }
    return;
  }
  const Scale sc(max, (double)t);
  w.by_k = w.k > 0 && w.k < p.V;
  w.by_p = w.top_p < 1.f;
  w.by_m = min_p > 0.f;
  w.log_min = w.by_m ? log((double)min_p) : 0.0;

  // the line: the step in which the wanted number of thread maxima is reached
  const uint32_t wanted = w.by_k ? (uint32_t)w.k : (uint32_t)kUsualLine;
  {
    const int step = sc.step(mine);
    if (step < kSteps) atomicAdd(&s.count[step], 1u);
  }
  __syncthreads();
  const uint32_t c0 = s.count[2 * threadIdx.x], c1 = s.count[2 * threadIdx.x + 1], upto = block_scan(c0 + c1, s.wave32);
  if (upto >= wanted && upto - c0 - c1 < wanted) s.found_first = 2 * threadIdx.x + (upto - c1 >= wanted ? 0 : 1);
  __syncthreads();
  const int step = (int)s.found_first;
  const bool complete = step == kSteps - 1;              // all that weighs anything is above the line
  // (its lower end, and what is rounded in it)
  const float depth = 2.f * (float)(step + 1) / sc.steps;
  const Line line(fmaxf(max - depth - 1e-6f * (fabsf(max) + depth), -3.4028235e38f), T{});

  // Rows so flat that the list would not hold what is drawn from: left to D.  The threads' maxima above the line say about what it holds (half
  // as much again), 16 bytes a thread from the middle of the row what lies below.  (A wrong guess costs time alone.)
  const bool sum = !w.by_k && (w.by_p || !w.by_m) && !complete;
  bool flat = sum && !sc.tail_fits();
  if (sum && !w.by_m && !flat) {
    float in = mine >= line.z ? fast_exp2(sc.tail_exponent(mine)) : 0.f, out = 0.f;
    constexpr int EPU = Elem<T>::per16;
    const int units = (p.V - EPU) / EPU;                 // (whole ones there are wherever the row starts)
    if (units >= kSampleThreads) {
      const char* at = row + ((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) + (int64_t)((units - kSampleThreads) / 2 + threadIdx.x) * 16;
      float x[EPU];
      unpack16(*reinterpret_cast<const uint4*>(at), x, T{});
#pragma unroll
      for (int e = 0; e < EPU; ++e) out += x[e] < line.z ? fast_exp2(sc.tail_exponent(x[e])) : 0.f;
      const double above = 1.5 * block_sum_double((double)in, s.waved);
      const double below = block_sum_double((double)out, s.waved) * ((double)units / kSampleThreads);
      flat = above < 0.85 * (w.by_p ? w.top_p : w.u) * (above + below);
    }
  }

  // B
  double tail = 0.0;
  const auto note = [&](float z, int token) {
    if (z >= line.z) {
      const uint32_t n = atomicAdd(&s.n, 1u);
      if (n < kListed) s.list[n] = item_of(z, token);
    }
  };
  if (flat) {
  } else if (sum) {
    double part = 0.0;
    float some = 0.f, weighted = 0.f;                    // of every unit's first: weight, weight times exponent
    const auto listed_too = [&](float z, int token) {    // (its weight has been added: taken away as it was)
      if (z >= line.z) {
        part -= (double)fast_exp2(sc.tail_exponent(z));
        note(z, token);
      }
    };
    each_unit<T, 5, true>(row, p.V, [&](uint32_t bits, int token) {
      const float z = sample_value(bits, T{});
      part += (double)fast_exp2(sc.tail_exponent(z));
      listed_too(z, token);
    }, [&](const uint4& r, int token) {
      float z[Elem<T>::per16], x[Elem<T>::per16];
      unpack16(r, z, T{});
#pragma unroll
      for (int e = 0; e < Elem<T>::per16; ++e) x[e] = fast_exp2(sc.tail_exponent(z[e]));
      some += x[0];
      weighted = __builtin_fmaf(x[0], fmaxf(sc.tail_exponent(z[0]), -1000.f), weighted);      // (-inf: no NaN)
      if constexpr (Elem<T>::per16 == 8) part += (double)(((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])));
      else part += (double)((x[0] + x[1]) + (x[2] + x[3]));
      if (line.reached(r, T{}))
#pragma unroll
        for (int e = 0; e < Elem<T>::per16; ++e) listed_too(z[e], token + e);
    });
    const double weights = block_sum_double(part, s.waved);
    const double of = block_sum_double((double)some, s.waved), exponents = block_sum_double((double)weighted, s.waved);
    tail = fmax(sc.tail_sum(weights, of > 0.0 ? exponents / of : 0.0), 0.0) * (double)(1ull << kWeightBits);
  } else {
    each_unit<T, kAtOnce, false>(row, p.V, [&](uint32_t bits, int token) { note(sample_value(bits, T{}), token); }, [&](const uint4& r, int token) {
      if (line.reached(r, T{})) {
        float x[Elem<T>::per16];
        unpack16(r, x, T{});
#pragma unroll
        for (int e = 0; e < Elem<T>::per16; ++e) note(x[e], token + e);
      }
    });
  }
  __syncthreads();
  const int listed = (int)s.n;

  // C
  Drawn d{0, 0, false};
  if (flat) {
  } else if (listed <= 64) {
    if (threadIdx.x < 64) {
      d = draw_from_list<true>(s, listed, sc, w, complete, tail, p.V);
      if (threadIdx.x == 0) { s.found_item = d.item; s.found_mass = d.kept; s.found_kind = d.settled; }
    }
    __syncthreads();
    d = Drawn{s.found_item, s.found_mass, s.found_kind != 0};
  } else if (listed <= kListed) {
    d = draw_from_list<false>(s, listed, sc, w, complete, tail, p.V);
  }
  if constexpr (std::is_same<T, bf16_t>::value) {
    if (!d.settled) {
      d = draw_from_values(s, row, p.V, sc, lowest_of(s), w);
      if (!d.settled) d = draw_from_steps<T>(s, row, p.V, max, (double)t, w);
    }
  } else {
    if (!d.settled) d = draw_from_steps<T>(s, row, p.V, max, (double)t, w);
  }
  if (threadIdx.x == 0) {
    p.token[b] = (int32_t)(uint32_t)d.item;
    if (p.logprob)
      p.logprob[b] = (float)(((double)logit_of(d.item) - (double)max) / sc.temperature - log((double)d.kept * (1.0 / (1ull << kWeightBits))));
  }
}

}  // namespace
}  // namespace bc

using namespace bc;

extern "C" int32_t bc_sample_tokens(int32_t B, int32_t V, const void* logits, int32_t logits_dtype, int64_t row_stride, const float* temperature,
                                    const int32_t* top_k, const float* top_p, const float* min_p, const float* u, const uint8_t* active,
                                    int32_t* tokens, float* logprob, void* stream) {
  if (logits_dtype != BC_F32 && logits_dtype != BC_BF16) return BC_ERR_SHAPE;
  if (B < 0 || (int64_t)B * kSampleThreads > 0xffffffffLL || V < 1 || V > (1 << 20)) return BC_ERR_SHAPE;      // (threads of a grid: 32 bits)
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
