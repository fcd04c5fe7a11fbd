// A lane's share of a head under norm and rotation: d / 8 lanes have a head, eight elements a lane, in two pieces of four that are each
// other's partners in the rotation.  Shared by the kernels that turn packed projections into q, k and v (bc_rope.hip) and into entries of a
// cache (bc_paged_append.hip).
#pragma once
#include "bc_common.h"

namespace bc {

// four elements <-> floats.  STREAM: past the caches
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
template <bool STREAM, typename V>
__device__ __forceinline__ V load_from(const char* at) {
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const V*>(at));
  else return *reinterpret_cast<const V*>(at);
}
template <bool STREAM, typename V>
__device__ __forceinline__ void store_to(char* at, const V& x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<V*>(at));
  else *reinterpret_cast<V*>(at) = x;
}
template <bool STREAM = false>
__device__ __forceinline__ void load4(const char* at, float (&x)[4], float) {
  const f32x4_t r = load_from<STREAM, f32x4_t>(at);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = r[e];
}
template <bool STREAM = false>
__device__ __forceinline__ void load4(const char* at, float (&x)[4], bf16_t) {
  const u32x2_t r = load_from<STREAM, u32x2_t>(at);
  x[0] = __uint_as_float(r.x << 16); x[1] = __uint_as_float(r.x & 0xffff0000u);
  x[2] = __uint_as_float(r.y << 16); x[3] = __uint_as_float(r.y & 0xffff0000u);
}
template <bool STREAM>
__device__ __forceinline__ void store4(char* at, const float (&x)[4], float) {
  store_to<STREAM>(at, f32x4_t{x[0], x[1], x[2], x[3]});
}
template <bool STREAM>
__device__ __forceinline__ void store4(char* at, const float (&x)[4], bf16_t) {
  store_to<STREAM>(at, u32x2_t{pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3])});
}

// cos and sin of position * inv_freq.  The product and its remainder of quarter turns in 64 bits: a position of a million times a
// frequency near one is off by 0.03 in 32.  What is left, at most an eighth of a turn, by the series in 32 bits (next term
// below 2e-9).
__device__ __forceinline__ void angle_of(int32_t position, float inv_freq, float& c, float& s) {
  const double quarters = (double)position * ((double)inv_freq * 0.63661977236758134308);      // 2 / pi
  const double whole = __builtin_rint(quarters);
  const float x = (float)(quarters - whole) * 1.57079632679489661923f, xx = x * x;
  const int n = (int)(int64_t)whole;
  const float sn = x + x * xx * (-1.f / 6 + xx * (1.f / 120 + xx * (-1.f / 5040 + xx * (1.f / 362880))));
  const float cs = 1.f + xx * (-0.5f + xx * (1.f / 24 + xx * (-1.f / 720 + xx * (1.f / 40320 + xx * (-1.f / 3628800)))));
  const float a = n & 1 ? sn : cs, b = n & 1 ? cs : sn;
  c = (n + 1) & 2 ? -a : a;
  s = n & 2 ? -b : b;
}

// Where a lane's two pieces of a head stand, and its angles.
template <int D>
struct RopeLane {
  int o1, o2;                  // elements
  bool turns;
  float c[4], s[4];
  __device__ __forceinline__ RopeLane(int half, const float* inv_freq, int lane, int32_t position) {
    const int at = 4 * lane;
    turns = at < half;
    o1 = turns ? at : 2 * at;               // (behind the rotated part eight in a row: 2 * half + 8 * (lane - half / 4))
    o2 = turns ? half + at : o1 + 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      c[e] = 1.f; s[e] = 0.f;
      if (turns) angle_of(position, inv_freq[at + e], c[e], s[e]);
    }
  }
  // by the angles, or (BACK) against them
  template <bool BACK>
  __device__ __forceinline__ void turn(float (&a)[4], float (&b)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float sn = BACK ? -s[e] : s[e], x = fmaf(a[e], c[e], -b[e] * sn), y = fmaf(b[e], c[e], a[e] * sn);
      a[e] = turns ? x : a[e];              // (not by a product with zero: the partner may be infinite)
      b[e] = turns ? y : b[e];
    }
  }
};

}  // namespace bc
