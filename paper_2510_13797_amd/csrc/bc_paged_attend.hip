// bc_paged_attend: attention of every sequence's newest rows over its entries in 8-bit pages (Sec. 2's attention; rows of a decode step,
// drafted tokens that are checked, chunks of a prompt).
//
//   out[i, h] = sum_j softmax_j(scale q[i, h] . K_j) V_j,  j over entries 0 .. L - n + i of the L there are, n of them the rows' own
//   K_j = key bytes * their block's scale, V_j likewise
//
// The query heads of a KV head see the same entries, so (row, head) pairs are the columns of the products: column i * g + h.  A tile is two
// blocks of 16 entries, which come from memory as operands (bc_paged.h) and become bf16 or half precision by the hardware's conversions,
// exactly: S^T = K.Q^T by 16x16x32 MFMA, whose result has four entries of a column in a lane; a word of values is those four entries of one
// element, so O^T += V^T.P^T takes both as they are.  A key scale that is a power of two goes along with the conversion, exactly; others
// are factors of their block's scores.  Values become half precision without their scale, which is a factor of the weights; those enter
// their product in two half-precision parts (22 bits) at a level that goes with the products (kLevelMost).  Softmax online, sums in fp32.
//
// Two kernels:
//   up to 32 columns: bound by memory, and by latency at both ends.  A row over 16,000, 32/8 heads, d = 128 (33 MB): 12.6 us; 64 rows over
//   4352 to 8704, 12/2 heads (216 MB): 38.7 (6.3 TB/s while it streams, as 1.07 GB in 171 us; a large read reaches 6.5); 1 to 8 rows of 16
//   sequences over 900 to 6000, 32/8 heads (121 MB): 28.2 to 29.3;
//   more: bound by the matrix cores, large ones by the power limit.  4 x 2048 rows over 30,000, 32/8 heads: 4.9 to 5.2 ms from card to
//   card, 0.79 to 0.74 PFLOP/s of the definition's products and 1.2 to 1.1 of those issued (a library product of 16384^3 reaches 1.39 to
//   1.32), matrix pipe busy 59 % of the cycles at 1.9 to 1.8 GHz; 512 rows over 7680: 103 to 108 us.
#include "bc_paged.h"

namespace bc {
namespace {

constexpr float kRedo = 256.f;                 // a lane's weights of a tile may sum to this before the reference moves,
constexpr float kLazy = 2.f;                   // and then it moves where a column's maximum is this much (log2) above it

struct AttendParams {
  PagedTables t;
  const char* q;               // [rows, Hq, d] bf16
  float* out;                  // [rows, Hq, d]
  const uint8_t* k;            // [pages, Hkv, page_rows, d]
  const uint8_t* v;
  const float* ks;             // [pages, Hkv, page_rows / 16]
  const float* vs;
  int32_t* arrivals;           // [B * Hkv] zero between launches
  float* part;                 // sums of parts; many columns: [parts][rows * Hq][d], and
  float2* part_ml;             // [parts][rows * Hq] their maximum (log2) and sum
  int32_t Hq, Hkv, g, max_len;
  uint32_t max_chunks, chunk_tiles;     // few columns
  int32_t blocks, parts;       // many: workgroups along a pair's columns, parts of its entries,
  uint32_t base;               // the launch's first workgroup
  float qs;                    // scale * log2 e
};

// Partial results go past the caches in both directions (the L2s of the XCDs do not see each other's lines): buffer accesses of system scope.
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_v;
typedef __attribute__((ext_vector_type(2))) float f32x2_v;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_v;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_v;
constexpr int kPast = 1 | 16;                  // sc0, sc1
__device__ __forceinline__ __amdgpu_buffer_rsrc_t parts_of(float* part) { return __builtin_amdgcn_make_buffer_rsrc(part, 0, 0x7fffffff, 0x27000); }
__device__ __forceinline__ void store16_past(__amdgpu_buffer_rsrc_t parts, uint32_t at, const f32x4_t& x) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, x), parts, at, 0, kPast);
}
__device__ __forceinline__ void store8_past(__amdgpu_buffer_rsrc_t parts, uint32_t at, float x, float y) {
  __builtin_amdgcn_raw_buffer_store_b64(u32x2_v{__float_as_uint(x), __float_as_uint(y)}, parts, at, 0, kPast);
}
__device__ __forceinline__ f32x4_t load16_past(__amdgpu_buffer_rsrc_t parts, uint32_t at) {
  return __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(parts, at, 0, kPast));
}
__device__ __forceinline__ u32x2_v load8_past(__amdgpu_buffer_rsrc_t parts, uint32_t at) { return __builtin_amdgcn_raw_buffer_load_b64(parts, at, 0, kPast); }

// A scale as the conversion's factor and what is left of it: one for a power of two.
__device__ __forceinline__ bool power_of_two_scale(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u & 0x807fffffu) == 0 && u - 0x00800000u < 0x7f000000u;
}
__device__ __forceinline__ uint32_t scaled_bf16(uint32_t w, float scale, bool high) {
  return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
}
__device__ __forceinline__ u32x4_t scaled_operand(uint32_t a, uint32_t b, float scale) {
  return u32x4_t{scaled_bf16(a, scale, false), scaled_bf16(a, scale, true), scaled_bf16(b, scale, false), scaled_bf16(b, scale, true)};
}

// eight e4m3 values (two words) as an operand in half precision: exact
__device__ __forceinline__ u32x4_t half_operand(uint32_t a, uint32_t b) {
  return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true))};
}
// f u, f v -> two pairs in half precision, the second one what the first leaves (22 bits together; the least step is 2^-24)
__device__ __forceinline__ void split_halves(float u, float v, float f, uint32_t& hi, uint32_t& lo) {
  const f16x2_v h = __builtin_convertvector(f32x2_v{u * f, v * f}, f16x2_v);
  hi = __builtin_bit_cast(uint32_t, h);
  lo = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_v{fmaf(u, f, -(float)h[0]), fmaf(v, f, -(float)h[1])}, f16x2_v));
}
// Bit 7 of the bytes that are no number (0x7f or 0xff), other bits anything; and a word with those bytes zero.
__device__ __forceinline__ uint32_t no_numbers(uint32_t w) { return (w & 0x7f7f7f7fu) + 0x01010101u; }
__device__ __forceinline__ uint32_t only_numbers(uint32_t w) { return w & ~((no_numbers(w) >> 7 & 0x01010101u) * 0xffu); }
// A NaN that the compiler, which is told that there are none, does not see.
__device__ __forceinline__ float no_number() {
  float x;
  asm volatile("v_mov_b32 %0, 0x7fc00000" : "=v"(x));
  return x;
}
// The level of a column's values.  Weights times their block's value scale enter products in half precision, so what they are brought to
// has to go with the product: sums are kept as `f` times what they are, f a power of two, so that no factor passes 2^14 and the largest
// came to 2^8 when f was last set.  What was small beside that is as small in the result.  f starts where nothing is too large and sums are
// zero.
constexpr int kLevelTop = 119;                 // log2
constexpr float kLevelMost = 16384.f, kLevelStart = 0x1p119f;
__device__ __forceinline__ float level_for(float largest) {      // 2^8 over it, as a power of two (up to 2^kLevelTop)
  return __uint_as_float(min(127u + kLevelTop, 254u + 8u - (__float_as_uint(largest) >> 23)) << 23);
}
// What a reference that moves up by `by` (log2, a whole number, or anything beyond 2^23) does to them: the level goes up with it, as far as
// it goes; from there on the sums come down by the factor that is returned, to nothing where there are none yet.  (By exponents: as a
// product level and move may pass what 32 bits hold where neither does.)
__device__ __forceinline__ float raise_level(float& level, float by) {
  const float up = (float)((int)(__float_as_uint(level) >> 23) - 127) + by, most = fminf(up, (float)kLevelTop);
  level = __uint_as_float((uint32_t)(127 + (int)most) << 23);
  return fast_exp2(most - up);
}
// A scale times the level passes what 32 bits hold where the scale is 2^9 or more, the level high and the weights next to nothing (or none
// that the column sees): such a scale leaves its exponent beyond 2^8 to the weights, which are 2^8 at most.
constexpr uint32_t kFarScale = (127 + 9) << 23;                  // (bits)
__device__ __forceinline__ float far_scale(float& scale) {
  const uint32_t u = __float_as_uint(scale), e = max((u >> 23 & 255u), 127u + 8u) - (127u + 8u);
  scale = __uint_as_float(u - (e << 23));
  return __uint_as_float((127u + e) << 23);
}
// What waves, halves of a workgroup, parts and teams hand over: sums of weights times values, their reference and their sum of weights.
// Sums of up to 2^39 may pass what 32 bits hold where their mean, the result, does not: those at a level below 2^-40 (of values above 2^48
// or so) are in a unit of 2^-40, for which their sum of weights is negative.  Where only some are, the others come to that unit.
constexpr float kUnit = 0x1p-40f;
__device__ __forceinline__ float inverse_power(float x) { return __uint_as_float((254u << 23) - __float_as_uint(x)); }      // 1 / x of a power of two
__device__ __forceinline__ float unit_at(float level) { return level < kUnit ? kUnit : 1.f; }
__device__ __forceinline__ float in_unit(float weights, float unit) { return unit < 1.f ? -weights : weights; }
// The unit for sums of one and another (of which the least sum of weights is enough), and what brings those of `weights` to it.
__device__ __forceinline__ float unit_for(float unit, float least_weights) { return least_weights < 0.f ? kUnit : unit; }
__device__ __forceinline__ float to_unit(float weights, float unit) { return weights < 0.f ? 1.f : unit; }
// The result: a sum over its weights, out of its unit.  (The hardware's reciprocal is off by 2^-23 at most, as sums of some weights are.)
template <typename V>
__device__ __forceinline__ V mean_of(const V& sum, float weights, float unit) { return sum * __builtin_amdgcn_rcpf(weights) * inverse_power(unit); }
__device__ __forceinline__ f32x4_t mfma16(const bf16x8_t& a, const bf16x8_t& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t lane_value(uint32_t x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// Waves a SIMD has room for.
constexpr int few_waves(int ct, int nw) { return ct == 1 && nw == 4 ? 4 : 2; }

// What a sequence of the call is, the same wherever it is asked for.
struct AttendSpan { int64_t row; int n, L; bool bad; };
__device__ __forceinline__ AttendSpan attend_span(const AttendParams& p, int s) {
  const PagedSpan span = paged_span(p.t, s);
  const int L = span.len;
  const bool bad = span.n < 0 || (span.n > 0 && (L < span.n || L > p.max_len));
  return {span.row, bad ? 0 : span.n, L, bad};
}

// Up to 16 * CT columns a KV head.  The waves of a workgroup have the tiles of its chunk of a (sequence, KV head) pair by turns.  Where a
// pair has several chunks, each leaves its sums in the workspace, and the workgroup that is the last to arrive adds them up in their order.
template <int D, int CT, int NW, bool STREAM>
__global__ void __launch_bounds__(64 * NW, few_waves(CT, NW)) paged_few_kernel(AttendParams p) {
  constexpr int H = D / 64, COLS = 16 * CT, PITCH = D + 4, BLOCK_BYTES = kPagedBlock * D, SUMS = COLS * (D + 2);
  __shared__ __attribute__((aligned(16))) float s_o[NW][COLS][PITCH];
  __shared__ float s_ml[NW][COLS][2];
  __shared__ float s_team[256 * NW / D][2];      // (a team and a column: d / 4 threads)
  __shared__ int s_last;
  const auto parts = parts_of(p.part);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, g4 = lane >> 4;
  const int per_page = p.t.page_shift - 4;

  const uint32_t pairs = (uint32_t)p.t.B * p.Hkv, chunk = blockIdx.x / pairs;
  const int pair = blockIdx.x - chunk * pairs, s = pair / p.Hkv, kvh = pair - s * p.Hkv;
  // 32 tiles of the wave at a time: lane 2 i + b has block b of the i-th.  (Which ones they are follows from the chunk's number alone: the
  // table is asked for together with the length.)
  const uint32_t t0 = chunk * p.chunk_tiles;
  const int most = (p.t.table_pages << per_page) - 1;
  auto page_of = [&](uint32_t tb) { return p.t.table[(int64_t)s * p.t.table_pages + (min(2 * (int)(tb + NW * (lane >> 1)) + (lane & 1), most) >> per_page)]; };
  int page = page_of(t0 + wave);
  const AttendSpan span = attend_span(p, s);
  if (span.bad && chunk == 0 && kvh == 0 && tid == 0) atomicOr(p.t.err, BC_ERRBIT_STATE);
  const uint32_t tiles = span.n > 0 ? (uint32_t)(span.L + 31) >> 5 : 0, chunks = (tiles + p.chunk_tiles - 1) / p.chunk_tiles;
  if (chunk >= chunks) return;
  const uint32_t t1 = min(t0 + p.chunk_tiles, tiles);
  const int n = span.n, L = span.L, own = n * p.g, seen_by_all = L - n + 1;

  bf16x8_t q[CT][2 * H];
  int key_lim[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int col = min(16 * ct + c16, own - 1), i = col / p.g;
    key_lim[ct] = L - n + 1 + i;
    const char* at = p.q + ((span.row + i) * p.Hq + kvh * p.g + (col - i * p.g)) * (2 * D) + 32 * g4;
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) q[ct][2 * h + e] = *reinterpret_cast<const bf16x8_t*>(at + 128 * h + 16 * e);
  }
  f32x4_t o[CT][4 * H];
  float m[CT], l[CT], level[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    m[ct] = kNegBig; l[ct] = 0.f; level[ct] = kLevelStart;
#pragma unroll
    for (int i = 0; i < 4 * H; ++i) o[ct][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  const uint32_t k_lane = (c16 >> 2) * 4 * D + (c16 & 3) * 64 + g4 * 16, v_lane = g4 * 4 * D + c16 * 16;
  for (uint32_t tb = t0 + wave; tb < t1; tb += 32 * NW) {
    const int count = min(32, (int)(t1 - tb + NW - 1) / NW), block = 2 * (int)(tb + NW * (lane >> 1)) + (lane & 1), last = (L - 1) >> 4;
    if (tb != t0 + wave) page = page_of(tb);
    // (a tile's second block may lie behind the last one: the first in its place; other lanes' blocks are nobody's)
    const int first_of = __builtin_amdgcn_update_dpp(page, page, 0xA0, 0xf, 0xf, true);        // quad_perm [0, 0, 2, 2]
    const int at_block = block > last ? block & ~1 : block;
    if (block > last) page = first_of;
    if (page < 0 || page >= p.t.pages) {
      if (at_block <= last && (lane >> 1) < count) atomicOr(p.t.err, BC_ERRBIT_STATE);
      page = 0;
    }
    const uint32_t unit = (((uint32_t)page * p.Hkv + kvh) << per_page) + (at_block & ((1 << per_page) - 1));
    const float qs = CT == 1 ? 1.f : p.qs, k_scale = CT == 1 ? p.ks[unit] * p.qs : p.ks[unit], v_scale = p.vs[unit];
    // (With one tile of columns key scales are always factors of the scores: two ways through the code cost a short step half a
    // microsecond, 9.7 -> 10.3 us.)
    const bool uneven = CT == 1 || __any(at_block <= last && (lane >> 1) < count && !power_of_two_scale(k_scale));

    // A tile's keys and values have their registers to themselves: the next tile's keys are asked for as soon as this one's scores are
    // formed, its values behind the weights' product.
    u32x4_t key[2][H], value[2][H];
    // (Behind the last tile one 16-byte piece of it in every lane's place: with a branch about the loads the compiler did not know how many
    // were on their way, and waited for all of them in front of the scores: 14.1 us for a row over 16,000, 13.3 so.)
    auto load = [&](u32x4_t (&x)[2][H], const uint8_t* pool, uint32_t at_lane, int i) {
      const uint32_t lane_at = i < count ? at_lane : 0;
      i = min(i, count - 1);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint8_t* at = pool + (uint64_t)lane_value(unit, 2 * i + b) * BLOCK_BYTES;
#pragma unroll
        for (int h = 0; h < H; ++h) {
          const u32x4_t* from = reinterpret_cast<const u32x4_t*>(at + (lane_at + 256 * h));
          x[b][h] = STREAM ? __builtin_nontemporal_load(from) : *from;
        }
      }
    };
    load(key, p.k, k_lane, 0);
    load(value, p.v, v_lane, 0);
    for (int i = 0; i < count; ++i) {
      const int key0 = 32 * (tb + NW * i);
      f32x4_t sc[CT][2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const float scale = uneven ? 1.f : __uint_as_float(lane_value(__float_as_uint(k_scale), 2 * i + b));
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) sc[ct][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const bf16x8_t a = __builtin_bit_cast(bf16x8_t, scaled_operand(key[b][h][2 * e], key[b][h][2 * e + 1], scale));
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) sc[ct][b] = mfma16(a, q[ct][2 * h + e], sc[ct][b]);
          }
      }
      load(key, p.k, k_lane, i + 1);
      if (uneven) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) sc[ct][b] *= __uint_as_float(lane_value(__float_as_uint(k_scale), 2 * i + b));
      }
      const bool ends = key0 + 32 > seen_by_all;                   // some columns do not see all of it
      if (CT == 1 && ends) {
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if (key0 + 16 * (r >> 2) + 4 * g4 + (r & 3) >= key_lim[0]) sc[0][r >> 2][r & 3] = 2.f * kNegBig;
      }
      f16x8_v part[CT][2];
      const uint32_t u0 = lane_value(__float_as_uint(v_scale), 2 * i), u1 = lane_value(__float_as_uint(v_scale), 2 * i + 1);
      const float v0 = __uint_as_float(u0), v1 = __uint_as_float(u1);
      const bool far = max(u0 & 0x7fffffffu, u1 & 0x7fffffffu) >= kFarScale;        // (by the scalar unit)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float w[8], sums[2], sum;
        const int there = key_lim[ct] - key0 - 4 * g4;
        auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
          for (int r = 0; r < 8; ++r) w[r] = fast_exp2(fmaf(sc[ct][r >> 2][r & 3], qs, -m[ct]));
          if (CT > 1 && ends) {
#pragma unroll
            for (int r = 0; r < 8; ++r) w[r] = 16 * (r >> 2) + (r & 3) < there ? w[r] : 0.f;
          }
          sums[0] = (w[0] + w[1]) + (w[2] + w[3]); sums[1] = (w[4] + w[5]) + (w[6] + w[7]);
          sum = sums[0] + sums[1];
        };
        auto move = [&]() __attribute__((always_inline)) {   // the reference, to the column's maximum
          float top = kNegBig;
#pragma unroll
          for (int r = 0; r < 8; ++r) top = fmaxf(top, CT == 1 || 16 * (r >> 2) + (r & 3) < there ? sc[ct][r >> 2][r & 3] * qs : kNegBig);
          top = rows_allreduce_max(top);
          const float to = top > m[ct] + (CT == 1 ? 0.f : kLazy) ? ceilf(top) : m[ct];
          if (!__any(to > m[ct])) return;
          const float down = raise_level(level[ct], to - m[ct]);
          l[ct] *= fast_exp2(m[ct] - to);
          m[ct] = to;
          if (down != 1.f) {
#pragma unroll
            for (int j = 0; j < 4 * H; ++j) o[ct][j] *= down;
          }
        };
        // With two tiles of columns vector work counts: the maximum is formed only where weights get large (38.7 -> 35.3 us for 16 x 1-8
        // rows over 900 to 6000, 32/8 heads).  With one, a wave's two or three tiles would pay for forming the first one's weights twice.
        if constexpr (CT == 1) {
          move();
          weights();
        } else {
          weights();
          if (__builtin_expect(__any(sum > kRedo), 0)) {
            move();
            weights();
          }
        }
        l[ct] += sum;
        const float largest = fmaxf(sums[0] * fabsf(v0), sums[1] * fabsf(v1));     // (block by block: a heavy key has nothing to do with another block's scale)
        if (__builtin_expect(__any(largest * level[ct] > kLevelMost), 0)) {
          const float all = rows_allreduce_max(largest), to = all * level[ct] > kLevelMost ? level_for(all) : level[ct], was = to / level[ct];
#pragma unroll
          for (int j = 0; j < 4 * H; ++j) o[ct][j] *= was;
          level[ct] = to;
        }
        float s0 = v0, s1 = v1;
        if (__builtin_expect(far, 0)) {
          const float f0 = far_scale(s0), f1 = far_scale(s1);
#pragma unroll
          for (int r = 0; r < 8; ++r) w[r] *= r < 4 ? f0 : f1;
        }
        u32x4_t hi, lo;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          uint32_t h, x;
          split_halves(w[2 * r], w[2 * r + 1], (r < 2 ? s0 : s1) * level[ct], h, x);
          hi[r] = h; lo[r] = x;
        }
        part[ct][0] = __builtin_bit_cast(f16x8_v, hi);
        part[ct][1] = __builtin_bit_cast(f16x8_v, lo);
      }
      if (key0 + 32 > L) {                     // bytes behind the last entry may be anything: zeros, not a product with a weight of zero
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int there = L - (key0 + 16 * b + 4 * g4);
          const uint32_t mask = there >= 4 ? 0xffffffffu : there <= 0 ? 0u : (1u << (8 * there)) - 1;
#pragma unroll
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) value[b][h][j] &= mask;
        }
      }
      // A value that is no number would reach the columns that do not see it, by a weight of zero: its bytes become zeros, and the columns
      // that do see it get a sum of weights that is no number.
      if (__builtin_expect(n > 1 && ends, 0)) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          uint32_t nans = 0;
#pragma unroll
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) nans |= no_numbers(value[b][h][j]);
          if (__builtin_expect(__any((nans & 0x80808080u) != 0), 0)) {
#pragma unroll 1
            for (int r = 0; r < 4; ++r, nans >>= 8) {
              const bool here = (__ballot(nans >> 7 & 1) >> (16 * g4) & 0xffff) != 0;      // entry key0 + 16 b + 4 g4 + r
#pragma unroll
              for (int ct = 0; ct < CT; ++ct)
                if (here && key0 + 16 * b + 4 * g4 + r < key_lim[ct]) l[ct] = no_number();
            }
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                value[b][h][j] = only_numbers(value[b][h][j]);
                __builtin_amdgcn_sched_barrier(0);
              }
          }
        }
      }
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f16x8_v a = __builtin_bit_cast(f16x8_v, half_operand(value[0][h][j], value[1][h][j]));
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int k = 0; k < 2; ++k)
              o[ct][4 * h + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, part[ct][k], o[ct][4 * h + j], 0, 0, 0);
        }
      load(value, p.v, v_lane, i + 1);
    }
  }

  // the waves' sums: a lane has elements 64 h + 16 g4 + 4 r + j of its column
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const float sum = rows_allreduce_sum(l[ct]);
    const float unit = unit_at(level[ct]), f = unit * inverse_power(level[ct]);
    if (g4 == 0) { s_ml[wave][16 * ct + c16][0] = m[ct]; s_ml[wave][16 * ct + c16][1] = in_unit(sum, unit); }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f32x4_t*>(&s_o[wave][16 * ct + c16][64 * h + 16 * g4 + 4 * r]) =
            f32x4_t{o[ct][4 * h][r], o[ct][4 * h + 1][r], o[ct][4 * h + 2][r], o[ct][4 * h + 3][r]} * f;
  }
  __syncthreads();
  const bool whole = chunks == 1;
  const uint32_t mine = (pair * p.max_chunks + chunk) * (SUMS * 4);
  auto result = [&](int c, int x) {            // where element x of a column goes
    const int i = c / p.g;
    return reinterpret_cast<f32x4_t*>(p.out + ((span.row + i) * p.Hq + kvh * p.g + (c - i * p.g)) * D + x);
  };
  for (int at = tid; at < own * (D / 4); at += 64 * NW) {
    const int c = at / (D / 4), x = 4 * (at % (D / 4));
    float top = kNegBig, least = 0.f, sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) { top = fmaxf(top, s_ml[w][c][0]); least = fminf(least, s_ml[w][c][1]); }
    const float unit = unit_for(1.f, least);
    f32x4_t r{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = fast_exp2(s_ml[w][c][0] - top), l = s_ml[w][c][1];
      sum += f * fabsf(l);
      r += f * to_unit(l, unit) * *reinterpret_cast<const f32x4_t*>(&s_o[w][c][x]);
    }
    if (whole) *result(c, x) = mean_of(r, sum, unit);
    else {
      store16_past(parts, mine + 4 * (c * D + x), r);
      if (x == 0) store8_past(parts, mine + 4 * (COLS * D + 2 * c), top, in_unit(sum, unit));
    }
  }
  if (whole) return;
  // the workgroup that arrives last adds the parts up, in their order
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) s_last = __hip_atomic_fetch_add(p.arrivals + pair, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (s_last != (int)chunks - 1) return;
  if (tid == 0) __hip_atomic_store(p.arrivals + pair, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // A column's piece of four elements is a thread's, or (few columns) several threads' by turns; their sums meet in LDS.
  const int pieces = own * (D / 4);
  int teams = 1;
  while (2 * teams * pieces <= 64 * NW) teams *= 2;
  const int team = teams > 1 ? tid / pieces : 0;             // (threads behind the last team have nothing to do)
  auto add_up = [&](auto together) {
    constexpr int N = decltype(together)::value;             // parts that a thread asks for at once
    for (int at = tid - team * pieces; at < pieces && team < teams; at += 64 * NW) {
      const int c = at / (D / 4), x = 4 * (at % (D / 4));
      float top = kNegBig, sum = 0.f, unit = 1.f;
      f32x4_t r{0.f, 0.f, 0.f, 0.f};
      for (uint32_t k0 = team; k0 < chunks; k0 += N * teams) {
        u32x2_v ml[N];
        f32x4_t part[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const uint32_t place = (pair * p.max_chunks + min(k0 + k * teams, chunks - 1)) * (SUMS * 4);
          ml[k] = load8_past(parts, place + 4 * (COLS * D + 2 * c));
          part[k] = load16_past(parts, place + 4 * (c * D + x));
        }
        float high = top, least = 0.f;
#pragma unroll
        for (int k = 0; k < N; ++k) { high = fmaxf(high, __uint_as_float(ml[k][0])); least = fminf(least, __uint_as_float(ml[k][1])); }
        const float was = fast_exp2(top - high), to = unit_for(unit, least);
        top = high; sum *= was; r *= to < unit ? was * kUnit : was;
        unit = to;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float f = k0 + k * teams < chunks ? fast_exp2(__uint_as_float(ml[k][0]) - top) : 0.f, l = __uint_as_float(ml[k][1]);
          sum += f * fabsf(l);
          r += f * to_unit(l, unit) * part[k];
        }
      }
      if (teams == 1) *result(c, x) = mean_of(r, sum, unit);
      else {
        *reinterpret_cast<f32x4_t*>(&s_o[0][0][0] + (team * pieces + at) * 4) = r;
        if (x == 0) { s_team[team * own + c][0] = top; s_team[team * own + c][1] = in_unit(sum, unit); }
      }
    }
  };
  if (chunks <= 4u * teams) add_up(std::integral_constant<int, 4>{});
  else if (chunks <= 8u * teams) add_up(std::integral_constant<int, 8>{});
  else add_up(std::integral_constant<int, 16>{});
  if (teams > 1) {
    __syncthreads();
    if (tid < pieces) {
      const int c = tid / (D / 4), x = 4 * (tid % (D / 4));
      float top = kNegBig, least = 0.f, sum = 0.f;
      for (int k = 0; k < teams; ++k) { top = fmaxf(top, s_team[k * own + c][0]); least = fminf(least, s_team[k * own + c][1]); }
      const float unit = unit_for(1.f, least);
      f32x4_t r{0.f, 0.f, 0.f, 0.f};
      for (int k = 0; k < teams; ++k) {
        const float f = fast_exp2(s_team[k * own + c][0] - top), l = s_team[k * own + c][1];
        sum += f * fabsf(l);
        r += f * to_unit(l, unit) * *reinterpret_cast<const f32x4_t*>(&s_o[0][0][0] + (k * pieces + tid) * 4);
      }
      *result(c, x) = mean_of(r, sum, unit);
    }
  }
}

// ---------------------------------------------------------------------------
// Many columns: 32 a wave, the workgroup's four share tiles of 64 entries.  A wave brings the bytes of one of a tile's four blocks,
// converts them (keys to bf16, values to half precision) and leaves them in LDS as the operands of 32x32x16 products, 16 bytes a lane: keys
// [32 entries][d / 16][half][entry], element 16 i + 8 half + e of a key (its place among the 32 turned by i, so that the writes meet no
// bank twice); values [16 entries][j][half][row], element (d / 32) row + j: a word's four keys are half of an operand, the lane's other
// word the other half, and results have d / 32 elements in a row.
// ---------------------------------------------------------------------------
constexpr int kManyWaves = 4, kManyColumns = 32 * kManyWaves, kManyTile = 16 * kManyWaves;
// Tiles of a block of columns, and those of one of its parts.
struct ManyCut { int tiles, t0, t1, parts; };
__device__ __forceinline__ ManyCut many_cut(int parts, int lim, int part) {
  const int tiles = (lim + kManyTile - 1) / kManyTile, n = min(parts, max(1, tiles >> 2));      // (no part of fewer than four tiles)
  return {tiles, (int)((int64_t)tiles * part / n), (int)((int64_t)tiles * (part + 1) / n), n};
}

// Up to 64 columns (HALVES): two waves have a column, and of every tile half of the entries each; their sums meet in LDS at the end.  (With
// two of the four waves idle, the same SIMDs had all the work of both workgroups: 18 x 2-5 rows over 10,000-30,000, 16/2 heads, 93 -> 71.5
// us; 100 x 16 over 500-2000, 32/8, 135 -> 104.)
template <int D, bool HALVES>
__global__ void __launch_bounds__(64 * kManyWaves, 2) paged_many_kernel(AttendParams p) {
  constexpr int NX = HALVES ? 1 : 2, KS = D / 16, NJ = D / 32, K_BYTES = kManyTile * D * 2, STAGE = 2 * K_BYTES, BLOCK_BYTES = kPagedBlock * D;
  __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];
  __shared__ float s_rest[2][kManyWaves];                        // what the conversion left of a block's key scale,
  __shared__ int s_odd;                                          // 1: that has been something but ones; 2: a value scale has been beyond kFarScale
  __shared__ __attribute__((aligned(16))) float s_value[2][kManyWaves];                                 // value scales,
  __shared__ __attribute__((aligned(8))) uint16_t s_no_number[2][kManyWaves];      // entries with a value that is no number
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
  const uint32_t pairs = (uint32_t)p.t.B * p.Hkv;
  uint32_t id = p.base + blockIdx.x;
  const int pair = id % pairs; id /= pairs;
  const int part = id % p.parts, block = p.blocks - 1 - id / p.parts;          // (the longest ones first)
  const int s = pair / p.Hkv, kvh = pair - s * p.Hkv;
  const AttendSpan span = attend_span(p, s);
  if (span.bad && block == 0 && part == 0 && kvh == 0 && tid == 0) atomicOr(p.t.err, BC_ERRBIT_STATE);
  const int n = span.n, L = span.L, columns = n * p.g, first = block * kManyColumns;
  if (first >= columns) return;
  const int last_row = (min(first + kManyColumns, columns) - 1) / p.g;
  const ManyCut cut = many_cut(p.parts, L - n + 1 + last_row, part);
  if (part >= cut.parts) return;

  const int x0 = HALVES ? wave >> 1 : 0;                         // (the wave's half)
  const int mine = first + 32 * (HALVES ? wave & 1 : wave), c = min(mine + col, columns - 1), i = c / p.g;
  const int lim = L - n + 1 + i;                                 // entries that this lane's column sees
  const int all_free = (L - n + 1 + first / p.g) / kManyTile;    // tiles that all columns of the workgroup see whole
  const int free_tiles = (L - n + 1 + min(mine, columns - 1) / p.g) / kManyTile;        // tiles that all of the wave's columns see whole
  const int seen = mine < columns ? (L - n + (min(mine + 32, columns) - 1) / p.g) / kManyTile + 1 : 0;         // tiles that the wave works on
  bf16x8_t qb[KS];
  {
    const char* at = p.q + ((span.row + i) * p.Hq + kvh * p.g + (c - i * p.g)) * (2 * D) + 16 * half;
#pragma unroll
    for (int k = 0; k < KS; ++k) qb[k] = *reinterpret_cast<const bf16x8_t*>(at + 32 * k);
  }
  f32x16_t O[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) O[j] = f32x16_t{0.f};
  float m = kNegBig, l = 0.f, level = kLevelStart;               // m: a whole number, once it has moved

  // A tile's bytes on their way: the wave's block of it.
  const int per_page = p.t.page_shift - 4, last_block = (L - 1) >> 4;
  u32x4_t kb[D / 64], vb[D / 64];                                // (d = 64: two words of each of two groups of values)
  float k_scale = 1.f, v_scale = 1.f;
  auto fetch = [&](int t) {
    const int b = min(4 * t + wave, last_block);
    int page = p.t.table[(int64_t)s * p.t.table_pages + (b >> per_page)];
    if ((uint32_t)page >= (uint32_t)p.t.pages) {
      if (lane == 0) atomicOr(p.t.err, BC_ERRBIT_STATE);
      page = 0;
    }
    const uint32_t unit = (((uint32_t)page * p.Hkv + kvh) << per_page) + (b & ((1 << per_page) - 1));
    const uint8_t *k = p.k + (uint64_t)unit * BLOCK_BYTES, *v = p.v + (uint64_t)unit * BLOCK_BYTES;
    k_scale = p.ks[unit]; v_scale = p.vs[unit];
#pragma unroll
    for (int x = 0; x < D / 64; ++x) kb[x] = *reinterpret_cast<const u32x4_t*>(k + (1024 * x + 16 * lane));
    if constexpr (D == 128) {
#pragma unroll
      for (int x = 0; x < D / 64; ++x) vb[x] = *reinterpret_cast<const u32x4_t*>(v + (1024 * x + 16 * lane));
    } else {
      const u32x2_v a = *reinterpret_cast<const u32x2_v*>(v + (256 * half + 8 * col)), b = *reinterpret_cast<const u32x2_v*>(v + (512 + 256 * half + 8 * col));
      vb[0] = u32x4_t{a[0], a[1], b[0], b[1]};
    }
  };
  auto put = [&](int t, int stage) {
    char* to = lds + stage * STAGE;
    const bool ke = power_of_two_scale(k_scale);
    const float kf = ke ? k_scale : 1.f;
    if (lane == 0) {
      s_rest[stage][wave] = ke ? 1.f : k_scale;
      s_value[stage][wave] = v_scale;
      const bool far = (__float_as_uint(v_scale) & 0x7fffffffu) >= kFarScale;
      if (__builtin_expect(!ke || far, 0)) atomicOr(&s_odd, (ke ? 0 : 1) | (far ? 2 : 0));
    }
#pragma unroll
    for (int x = 0; x < D / 64; ++x) {                           // rows of the block: 4 * group + (lane / 4) % 4
      const int at = 64 * x + lane, group = at / (D / 4), h = at / 16 % (D / 64), k = 4 * h + lane % 4, row = 16 * (wave & 1) + 4 * group + lane / 4 % 4;
      char* place = to + (wave >> 1) * (K_BYTES / 2) + k * 1024 + ((row ^ (2 * (k & 3))) * 16);
      *reinterpret_cast<u32x4_t*>(place) = scaled_operand(kb[x][0], kb[x][1], kf);
      *reinterpret_cast<u32x4_t*>(place + 512) = scaled_operand(kb[x][2], kb[x][3], kf);
    }
    // values: words w of group `half` and of group `half + 2`
    char* place = to + K_BYTES + wave * (NJ * 1024) + half * 512 + col * 16;
    uint32_t keep[2] = {0xffffffffu, 0xffffffffu};
    if (kManyTile * (t + 1) > L) {                               // bytes behind the last entry may be anything
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int there = L - kManyTile * t - 16 * wave - 4 * (half + 2 * x);
        keep[x] = there >= 4 ? 0xffffffffu : there <= 0 ? 0u : (1u << (8 * there)) - 1;
      }
    }
    if (__builtin_expect(t >= all_free, 0)) {                                         // (as with few columns)
      uint32_t nans[2] = {0, 0}, entries = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (D == 128) { nans[0] |= no_numbers(vb[0][j] & keep[0]); nans[1] |= no_numbers(vb[D / 64 - 1][j] & keep[1]); }
        else nans[j >> 1] |= no_numbers(vb[0][j] & keep[j >> 1]);
      }
      if (__builtin_expect(__any(((nans[0] | nans[1]) & 0x80808080u) != 0), 0)) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint64_t have = __ballot(nans[x] >> (8 * r + 7) & 1);
            entries |= ((uint32_t)have != 0 ? 1u : 0u) << (8 * x + r) | ((have >> 32) != 0 ? 1u : 0u) << (8 * x + 4 + r);
          }
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
#pragma unroll
          for (int j = 0; j < 4; ++j) vb[x][j] = only_numbers(vb[x][j]);
      }
      if (lane == 0) s_no_number[stage][wave] = (uint16_t)entries;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const uint32_t a = D == 128 ? vb[0][j] : vb[0][j & 1], b = D == 128 ? vb[D / 64 - 1][j] : vb[0][2 + (j & 1)];
      *reinterpret_cast<u32x4_t*>(place + j * 1024) = half_operand(a & keep[0], b & keep[1]);
    }
  };

  fetch(cut.t0);
  if (tid == 0) s_odd = 0;
  __syncthreads();
  put(cut.t0, 0);
  if (cut.t0 + 1 < cut.t1) fetch(cut.t0 + 1);
  __syncthreads();
  for (int t = cut.t0, stage = 0; t < cut.t1; ++t, stage ^= 1) {
    if (t + 1 < cut.t1) put(t + 1, stage ^ 1);
    if (t + 2 < cut.t1) fetch(t + 2);
    if (t < seen) {
      const char* tile = lds + stage * STAGE;
      // (The wave that has products to issue goes first: the other of its SIMD forms weights meanwhile.  5.15 -> 4.81 ms; with the weights
      // first 5.16.)
      __builtin_amdgcn_s_setprio(1);
      f32x16_t sc[NX];
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        sc[x] = f32x16_t{0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k)
          sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              *reinterpret_cast<const bf16x8_t*>(tile + (x0 + x) * (K_BYTES / 2) + k * 1024 + half * 512 + ((col ^ (2 * (k & 3))) * 16)), qb[k], sc[x], 0, 0, 0);
      }
      __builtin_amdgcn_s_setprio(0);
      // (A block's values are read in front of the block before it: 111 us for 512 rows over 7680, 110 so.)
      f16x8_v a[2][NJ];
      auto values = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) a[b & 1][j] = *reinterpret_cast<const f16x8_v*>(tile + K_BYTES + (2 * x0 + b) * (NJ * 1024) + j * 1024 + half * 512 + col * 16);
      };
      values(0);
      const int odd = __builtin_amdgcn_readfirstlane(s_odd);
      // result e of sc[x]: entry 32 (x0 + x) + 8 (e / 4) + 4 half + e % 4 of the tile, of its block 2 (x0 + x) + e / 8
      if (__builtin_expect(odd & 1, 0)) {
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) sc[x][e] *= s_rest[stage][2 * (x0 + x) + e / 8];
      }
      const bool ends = t >= free_tiles;                         // some columns do not see all of it
      const int there = lim - kManyTile * t - 32 * x0 - 4 * half;
      float pe[NX][16], sums[2 * NX], psum;                            // sums: of blocks
      auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < NX; ++x) {
#pragma unroll
          for (int e = 0; e < 16; ++e) pe[x][e] = fast_exp2(fmaf(sc[x][e], p.qs, -m));
          if (ends) {
#pragma unroll
            for (int e = 0; e < 16; ++e) pe[x][e] = 32 * x + 8 * (e >> 2) + (e & 3) < there ? pe[x][e] : 0.f;
          }
          sums[2 * x] = ((pe[x][0] + pe[x][1]) + (pe[x][2] + pe[x][3])) + ((pe[x][4] + pe[x][5]) + (pe[x][6] + pe[x][7]));
          sums[2 * x + 1] = ((pe[x][8] + pe[x][9]) + (pe[x][10] + pe[x][11])) + ((pe[x][12] + pe[x][13]) + (pe[x][14] + pe[x][15]));
        }
        psum = sums[0] + sums[1];
        if constexpr (NX == 2) psum += sums[2] + sums[3];
      };
      weights();
      if (__builtin_expect(__any(psum > kRedo), 0)) {
        float top = kNegBig;
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) top = fmaxf(top, 32 * x + 8 * (e >> 2) + (e & 3) < there ? sc[x][e] * p.qs : kNegBig);
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float to = top > m + kLazy ? ceilf(top) : m, was = fast_exp2(m - to), down = raise_level(level, to - m);
        m = to; l *= was;
        if (down != 1.f) {
#pragma unroll
          for (int j = 0; j < NJ; ++j) O[j] *= down;
        }
        weights();
      }
      l += psum;
      if (__builtin_expect(t >= all_free, 0)) {
        const uint64_t entries = *reinterpret_cast<const uint64_t*>(s_no_number[stage]);
        const int sees = lim - kManyTile * t;
        if (sees > 0 && (entries & (sees >= 64 ? ~0ull : (1ull << sees) - 1)) != 0) l = no_number();
      }
      float scales[2 * NX], largest = 0.f;
#pragma unroll
      for (int b = 0; b < 2 * NX; ++b) {
        scales[b] = s_value[stage][2 * x0 + b];
        largest = fmaxf(largest, sums[b] * fabsf(scales[b]));
      }
      if (__builtin_expect(__any(largest * level > kLevelMost), 0)) {
        const float both = fmaxf(largest, __shfl_xor(largest, 32, 64)), to = both * level > kLevelMost ? level_for(both) : level, was = to / level;
#pragma unroll
        for (int j = 0; j < NJ; ++j) O[j] *= was;
        level = to;
      }
      if (__builtin_expect(odd & 2, 0)) {
#pragma unroll
        for (int b = 0; b < 2 * NX; ++b) {
          const float f = far_scale(scales[b]);
#pragma unroll
          for (int y = 0; y < 8; ++y) pe[b >> 1][8 * (b & 1) + y] *= f;
        }
      }
#pragma unroll
      for (int b = 0; b < 2 * NX; ++b) {
        u32x4_t hi, lo;
        if (b == 0) __builtin_amdgcn_s_setprio(1);
        const float f = scales[b] * level;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          uint32_t h, r;
          split_halves(pe[b >> 1][8 * (b & 1) + 2 * y], pe[b >> 1][8 * (b & 1) + 2 * y + 1], f, h, r);
          hi[y] = h; lo[y] = r;
        }
        if (b + 1 < 2 * NX) values(b + 1);
#pragma unroll
        for (int j = 0; j < NJ; ++j) O[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[b & 1][j], __builtin_bit_cast(f16x8_v, hi), O[j], 0, 0, 0);
#pragma unroll
        for (int j = 0; j < NJ; ++j) O[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[b & 1][j], __builtin_bit_cast(f16x8_v, lo), O[j], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    __syncthreads();
  }
  l += __shfl_xor(l, 32, 64);
  float unit = unit_at(level), f = unit * inverse_power(level);
  if constexpr (HALVES) {                                        // (all have left the last tile behind)
    float* other = reinterpret_cast<float*>(lds) + (wave & 1) * (NJ * 16 + 2) * 64 + lane;
    if (wave >= 2) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) other[(16 * j + e) * 64] = O[j][e] * f;
      other[NJ * 16 * 64] = m; other[(NJ * 16 + 1) * 64] = in_unit(l, unit);
    }
    __syncthreads();
    if (wave >= 2) return;
    const float its = other[NJ * 16 * 64], weights = other[(NJ * 16 + 1) * 64], top = fmaxf(m, its), f0 = fast_exp2(m - top), f1 = fast_exp2(its - top);
    const float both = unit_for(unit, weights), u0 = both < unit ? f0 * kUnit : f0, u1 = f1 * to_unit(weights, both);
    l = l * f0 + fabsf(weights) * f1;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) O[j][e] = O[j][e] * f * u0 + other[(16 * j + e) * 64] * u1;
    m = top; unit = both; f = 1.f;
  }
  if (mine + col >= columns) return;
  const int64_t at = (span.row + i) * p.Hq + kvh * p.g + (c - i * p.g);
  const bool whole = cut.parts == 1;
  float* to = whole ? p.out + at * D : p.part + (part * (p.t.rows * p.Hq) + at) * D;
  const float mean = whole ? __builtin_amdgcn_rcpf(l) : 1.f, out = whole ? f * inverse_power(unit) : f;      // (one after the other: either may leave the range that both together keep)
  if (!whole && half == 0) p.part_ml[part * (p.t.rows * p.Hq) + at] = make_float2(m, in_unit(l, unit));
  // result e of block j: its row 8 (e / 4) + 4 half + e % 4
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int row = 8 * (e >> 2) + 4 * half + (e & 3);
    if constexpr (D == 128) *reinterpret_cast<f32x4_t*>(to + 4 * row) = f32x4_t{O[0][e] * mean * out, O[1][e] * mean * out, O[NJ - 2][e] * mean * out, O[NJ - 1][e] * mean * out};
    else *reinterpret_cast<f32x2_v*>(to + 2 * row) = f32x2_v{O[0][e] * mean * out, O[1][e] * mean * out};
  }
}

// The parts of many columns: a column's pieces of four elements a thread each.
template <int D>
__global__ void __launch_bounds__(256) paged_fold_kernel(AttendParams p) {
  constexpr int UNITS = D / 4, PER = 256 / UNITS;
  const int64_t pairs = (int64_t)p.t.B * p.Hkv;
  const uint32_t id = p.base + blockIdx.x;
  const int pair = id % pairs, s = pair / p.Hkv, kvh = pair - s * p.Hkv;
  const int c = (int)(id / pairs) * PER + threadIdx.x / UNITS, unit = threadIdx.x % UNITS;
  const AttendSpan span = attend_span(p, s);
  const int columns = span.n * p.g;
  if (c >= columns) return;
  const int i = c / p.g, last_row = (min(c / kManyColumns * kManyColumns + kManyColumns, columns) - 1) / p.g;
  const ManyCut cut = many_cut(p.parts, span.L - span.n + 1 + last_row, 0);
  if (cut.parts == 1) return;
  const int64_t at = (span.row + i) * p.Hq + kvh * p.g + (c - i * p.g), step = p.t.rows * p.Hq;
  float top = kNegBig, sum = 0.f, in = 1.f;
  f32x4_t r{0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < cut.parts; k0 += 8) {
    float2 ml[8];
    f32x4_t x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t from = min(k0 + k, cut.parts - 1) * step + at;
      ml[k] = p.part_ml[from];
      x[k] = *reinterpret_cast<const f32x4_t*>(p.part + from * D + 4 * unit);
    }
    float high = top, least = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) { high = fmaxf(high, ml[k].x); least = fminf(least, ml[k].y); }
    const float was = fast_exp2(top - high), to = unit_for(in, least);
    top = high; sum *= was; r *= to < in ? was * kUnit : was;
    in = to;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float f = k0 + k < cut.parts ? fast_exp2(ml[k].x - top) : 0.f;
      sum += f * fabsf(ml[k].y); r += f * to_unit(ml[k].y, in) * x[k];
    }
  }
  *reinterpret_cast<f32x4_t*>(p.out + at * D + 4 * unit) = mean_of(r, sum, in);
}

struct AttendLaunch {
  int ct, waves, max_chunks, chunk_tiles;      // few columns
  bool stream;
  int blocks, parts;           // many
  size_t part_bytes, ml_at;
  bool fits;
};
// How a call is cut.  Lengths are on the device; the longest that there can be stands for them.
// Few columns, four waves a workgroup in up to 512 or eight in up to 256 (us, one row a sequence, d = 128):
//   1 x 16,000 rows, 32/8 heads          17.0, 13.3     64 x 300-1500 (eight share a prompt), 12/2   10.6, 11.2
//   4 x 2000, 32/8                       11.0, 10.2     1 x 500, 32/8                                 6.4,  7.4
//   128 x 300-3000, 12/2                 26.0, 24.0     64 x 400, 12/2                                8.4,  8.9
//   32 x 4000, 32/8                      48.9, 46.9     64 x 1000, 32/8 (more pairs than 256)        26.0, 27.6
// and two to eight rows: 1 x 8000, 32/8 28.1, 19.1; 64 x 1000, 12/2 16.9, 15.5; 1 x 500, 32/8 9.6, 10.7; 128 x 300, 32/8 26.8, 38.4.  More
// and smaller workgroups (four waves, 768): 19.8 for the first.  Two tiles of columns leave twice the sums to add up: chunks of at least
// sixteen tiles (1 x 8000: 19.1 -> 15.9, others as they were).
// Caches beyond some 100 MB go past the caches: 64 x 1000 rows, 32/8 heads (131 MB) 30.2 -> 26.7; 128 x 300 (79 MB) 17.5 -> 18.3.
// (Chunks of equal size for all sequences of a batch, worked out by every workgroup from the lengths: 2.3 us more for one tile of columns,
// nothing gained with two.)
// Workgroups that run at once are those of d = 128, by registers and LDS.  With d = 64 there is room for more, 768 of many columns, 512 of
// eight waves and one tile; cuts for it have not been measured.
// Many columns: as many parts as cost least, in tiles of 64: rounds of the workgroups that run at once (two a compute unit), a workgroup's
// tiles and its two ends, and parts written and read again.  512 rows over 7680, 32/8 heads, in three, four, five parts 135, 115, 153 us.
// One round of workgroups at most, and so:
//   69 x 15 rows over 1400-27,900, 14/2 heads, d = 64   237, 184     8 x 50-500 over 300-20,000, 12/2   555, 438     9 x 256 over 4000, 32/8   298, 273
//   the same, all over 27,900                           270, 258     3 x 400 over 6000, 32/8            208, 190     20 x 64 over 3000, 32/8   119, 119 (ends of three tiles: 132)
// Where a call fills the chip several times over, another part saves little of its time and takes as much memory as its outputs
// (17 x 8200 rows, 32/8 heads, over a table of 2^20 entries: 7 GB in three parts for 0.8 % of the count above): no more parts
// than 256 MB hold, seven for 2048 rows of 32 heads, two for three rounds of workgroups.
constexpr int kMostParts = 16, kManyGroups = 512;
constexpr int64_t kPartBytes = 256 << 20;
constexpr double kEndTiles = 5, kFoldTiles = 0.012;
constexpr int64_t kStreamBytes = 96 << 20;
AttendLaunch plan_attend(const bc_shape* sh, int64_t rows, int64_t max_new, int64_t max_len) {
  AttendLaunch a{};
  const int64_t g = sh->Hq / sh->Hkv, columns = max_new * g, pairs = (int64_t)sh->B * sh->Hkv, tiles = (max_len + 31) / 32;
  if (columns > 0x7fffffff) return a;
  if (columns <= 32) {
    a.ct = columns <= 16 ? 1 : 2;
    a.waves = pairs <= 256 && tiles >= (a.ct == 1 ? 62 : 32) ? 8 : 4;
    a.stream = pairs * max_len * 2 * sh->d > kStreamBytes;
    const int64_t groups = a.waves == 8 ? 256 : 512, most = groups / pairs < 1 ? 1 : groups / pairs, each = (tiles + most - 1) / most;
    const int least = a.ct == 1 ? a.waves : 16;
    a.chunk_tiles = (int)(each < least ? least : each);
    a.max_chunks = (int)((tiles + a.chunk_tiles - 1) / a.chunk_tiles);
    a.part_bytes = a.max_chunks > 1 ? (size_t)(pairs * a.max_chunks) * 16 * a.ct * (sh->d + 2) * 4 : 0;
    a.fits = true;
    return a;
  }
  a.blocks = (int)((columns + kManyColumns - 1) / kManyColumns);
  const int64_t groups = pairs * a.blocks;
  double least = 0;
  const int64_t part_bytes = rows * sh->Hq * (sh->d + 2) * 4;
  for (int64_t parts = 1; parts <= kMostParts && (parts == 1 || (parts <= tiles / 8 && parts * part_bytes <= kPartBytes)); ++parts) {
    const double rounds = (double)((groups * parts + kManyGroups - 1) / kManyGroups), fold = parts > 1 ? kFoldTiles * (double)(groups * parts) : 0;
    const double cost = rounds * ((double)tiles / 2 / (double)parts + kEndTiles) + fold;
    if (parts == 1 || cost < least) { least = cost; a.parts = (int)parts; }
  }
  const int64_t parts = a.parts;
  const int64_t fold = pairs * ((columns + 1024 / sh->d - 1) / (1024 / sh->d));
  a.fits = groups * parts <= 0x7fffffff && fold <= 0x7fffffff;
  if (parts > 1) {
    a.ml_at = (size_t)(parts * rows * sh->Hq) * sh->d * 4;
    a.part_bytes = a.ml_at + (size_t)(parts * rows * sh->Hq) * 8;
  }
  return a;
}

template <int D, int CT, int NW>
void launch_few(const AttendParams& p, const AttendLaunch& a, hipStream_t s) {
  const unsigned groups = (unsigned)((int64_t)p.t.B * p.Hkv * a.max_chunks);
  if (a.stream) paged_few_kernel<D, CT, NW, true><<<groups, 64 * NW, 0, s>>>(p);
  else paged_few_kernel<D, CT, NW, false><<<groups, 64 * NW, 0, s>>>(p);
}
template <int D>
void launch_attend(AttendParams& p, const AttendLaunch& a, hipStream_t s) {
  if (a.ct) {
    if (a.ct == 1) { if (a.waves == 8) launch_few<D, 1, 8>(p, a, s); else launch_few<D, 1, 4>(p, a, s); }
    else { if (a.waves == 8) launch_few<D, 2, 8>(p, a, s); else launch_few<D, 2, 4>(p, a, s); }
    return;
  }
  const int64_t pairs = (int64_t)p.t.B * p.Hkv, columns = (int64_t)p.t.max_new * p.g, per = 1024 / D;
  in_launches(pairs * a.blocks * a.parts, 64 * kManyWaves, [&](uint32_t base, unsigned groups) {
    p.base = base;
    if (columns <= kManyColumns / 2) paged_many_kernel<D, true><<<groups, 64 * kManyWaves, 0, s>>>(p);
    else paged_many_kernel<D, false><<<groups, 64 * kManyWaves, 0, s>>>(p);
  });
  if (a.parts == 1) return;
  in_launches(pairs * ((columns + per - 1) / per), 256, [&](uint32_t base, unsigned groups) {
    p.base = base;
    paged_fold_kernel<D><<<groups, 256, 0, s>>>(p);
  });
}

int64_t longest(const bc_pages* pg) {
  const int64_t all = (int64_t)pg->table_pages * pg->page_rows;
  return pg->max_len > 0 && pg->max_len < all ? pg->max_len : all;
}

}  // namespace
}  // namespace bc

using namespace bc;

extern "C" size_t bc_paged_workspace_bytes(const bc_shape* shape, int64_t rows, int32_t max_new, int32_t max_len) {
  if (check_shape(shape) != BC_OK || rows < 0 || rows > 0x7fffffff || max_new < 0 || max_len < 1 || (int64_t)shape->B * shape->Hkv > (1 << 23)) return 0;
  const int64_t most = max_new < rows ? max_new : rows;
  const AttendLaunch a = plan_attend(shape, rows, most < max_len ? most : max_len, max_len);
  return a.fits ? a.part_bytes + 16 : 0;
}

extern "C" int32_t bc_paged_attend(const bc_shape* shape, const bc_pages* pages, int64_t rows, const int64_t* row_offsets, int32_t max_new,
                                   const void* q, float* out, const uint8_t* active, void* workspace, size_t workspace_bytes, void* stream) {
  const int32_t st = check_pages(shape, pages, rows, row_offsets, max_new);
  if (st != BC_OK) return st;
  if (!nonnegative_finite(shape->scale)) return BC_ERR_ARG;
  if (rows == 0 || max_new == 0) return BC_OK;
  if (!q || !out || !aligned16(q) || !aligned16(out) || !pages->arrivals) return BC_ERR_ARG;
  const int64_t max_len = longest(pages);
  // (a sequence cannot have more new rows than there are, nor than entries)
  int64_t most = max_new < rows ? max_new : rows;
  if (most > max_len) most = max_len;
  const AttendLaunch a = plan_attend(shape, rows, most, max_len);
  if (!a.fits) return BC_ERR_SHAPE;
  if (a.part_bytes && (!workspace || !aligned16(workspace) || workspace_bytes < a.part_bytes)) return BC_ERR_WORKSPACE;
  AttendParams p{};
  p.t = paged_tables(shape, pages, rows, row_offsets, (int32_t)most, active);
  p.q = static_cast<const char*>(q); p.out = out;
  p.k = static_cast<const uint8_t*>(pages->k); p.v = static_cast<const uint8_t*>(pages->v); p.ks = pages->k_scale; p.vs = pages->v_scale;
  p.arrivals = pages->arrivals; p.part = static_cast<float*>(workspace);
  p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + a.ml_at);
  p.Hq = shape->Hq; p.Hkv = shape->Hkv; p.g = shape->Hq / shape->Hkv; p.max_len = (int32_t)max_len;
  p.max_chunks = a.max_chunks; p.chunk_tiles = a.chunk_tiles; p.blocks = a.blocks; p.parts = a.parts;
  p.qs = shape->scale * kLog2e;
  if (shape->d == 128) launch_attend<128>(p, a, as_stream(stream)); else launch_attend<64>(p, a, as_stream(stream));
  return launch_status();
}
