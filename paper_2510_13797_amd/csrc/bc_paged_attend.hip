// bc_paged_attend: attention of every sequence's newest rows over its entries in 8-bit pages (Sec. 2's attention; rows of a decode step, drafted tokens that are
// checked, chunks of a prompt).
//
//   out[i, h] = sum_j softmax_j(scale q[i, h] . K_j) V_j,  j over entries 0 .. L - n + i of the L there are, n of them the rows' own
//   K_j = key bytes * their block's scale, V_j likewise
//
// The query heads of a KV head see the same entries, so (row, head) pairs are the columns of the products: column i * g + h.  A tile is two blocks of 16 entries, which
// come from memory as operands (bc_paged.h) and become bf16 by the hardware's conversion, exactly: S^T = K.Q^T by 16x16x32 MFMA, whose result has four entries of a
// column in a lane; a word of values is those four entries of one element, so O^T += V^T.P^T takes both as they are.  A block's key scale is a factor of its scores, its
// value scale one of its weights (in fp32, in front of their split into two bf16 parts, 17 bits).  Softmax online, sums in fp32.
#include "bc_paged.h"

namespace bc {
namespace {

constexpr float kMasked = 2.f * kNegBig;       // a score that no maximum is below

struct AttendParams {
  PagedTables t;
  const char* q;               // [rows, Hq, d] bf16
  float* out;                  // [rows, Hq, d]
  const uint8_t* k;            // [pages, Hkv, page_rows, d]
  const uint8_t* v;
  const float* ks;             // [pages, Hkv, page_rows / 16]
  const float* vs;
  int32_t* arrivals;           // [B * Hkv] zero between launches
  float* part;                 // [pair][chunk][columns][d + 2]
  int32_t Hq, Hkv, g, max_len;
  int32_t column_blocks, max_chunks, chunk_tiles;
  float qs;                    // scale * log2 e
};

// Partial results go past the caches in both directions: the L2s of the XCDs do not see each other's lines.
__device__ __forceinline__ void store2_past(float* a, float x, float y) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(a), (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}
__device__ __forceinline__ uint64_t load2_past(const float* a) {
  return __hip_atomic_load(reinterpret_cast<const uint64_t*>(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}
__device__ __forceinline__ float low_of(uint64_t x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float high_of(uint64_t x) { return __uint_as_float((uint32_t)(x >> 32)); }

__device__ __forceinline__ uint32_t bf16_of(uint32_t w, bool high) {
  return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
}
// eight e4m3 values (two words) as an operand
__device__ __forceinline__ bf16x8_t operand_of(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(bf16x8_t, u32x4_t{bf16_of(a, false), bf16_of(a, true), bf16_of(b, false), bf16_of(b, true)});
}
__device__ __forceinline__ f32x4_t mfma16(const bf16x8_t& a, const bf16x8_t& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t lane_value(uint32_t x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// A tile as it comes from memory: 16 bytes a lane for 64 elements of a block of keys, and of values.
template <int D> struct Tile { u32x4_t k[2][D / 64], v[2][D / 64]; };

template <int D, int CT, int NW>
__global__ void __launch_bounds__(64 * NW) paged_few_kernel(AttendParams p) {
  constexpr int H = D / 64, COLS = 16 * CT, PITCH = D + 4, BLOCK_BYTES = kPagedBlock * D;
  __shared__ __attribute__((aligned(16))) float s_o[NW][COLS][PITCH];
  __shared__ float s_ml[NW][COLS][2];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, g4 = lane >> 4;
  uint32_t id = blockIdx.x;
  const int kvh = id % p.Hkv; id /= p.Hkv;
  const int s = id % p.t.B; id /= p.t.B;
  const int cb = id % p.column_blocks, chunk = id / p.column_blocks;
  const bool herald = chunk == 0 && cb == 0 && kvh == 0 && tid == 0;
  const PagedSpan span = paged_span(p.t, s);
  if (span.n == 0) return;
  const int n = span.n, L = p.t.len[s];
  if (n < 0 || L < n || L > p.max_len) {
    if (herald) atomicOr(p.t.err, BC_ERRBIT_STATE);
    return;
  }
  const int columns = n * p.g, col0 = cb * COLS;                       // (host: no more than 2^31)
  if (col0 >= columns) return;
  const int own = min(COLS, columns - col0);
  const int first_row = col0 / p.g, last_row = (col0 + own - 1) / p.g;
  const int seen_by_all = L - n + 1 + first_row, lim = L - n + 1 + last_row;
  const int tiles = (lim + 31) >> 5;
  const int want = min(p.max_chunks, (tiles + p.chunk_tiles - 1) / p.chunk_tiles), per = (tiles + want - 1) / want, chunks = (tiles + per - 1) / per;
  if (chunk >= chunks) return;
  const int t0 = chunk * per, t1 = min(tiles, t0 + per);

  bf16x8_t q[CT][2 * H];
  int key_lim[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int col = min(col0 + 16 * ct + c16, columns - 1), i = col / p.g;
    key_lim[ct] = L - n + 1 + i;
    const char* at = p.q + ((span.row + i) * p.Hq + kvh * p.g + (col - i * p.g)) * (2 * D) + 32 * g4;
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) q[ct][2 * h + e] = *reinterpret_cast<const bf16x8_t*>(at + 128 * h + 16 * e);
  }
  f32x4_t o[CT][4 * H];
  float m[CT], l[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    m[ct] = kNegBig; l[ct] = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * H; ++i) o[ct][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  const uint32_t k_lane = (c16 >> 2) * 4 * D + (c16 & 3) * 64 + g4 * 16, v_lane = g4 * 4 * D + c16 * 16;
  // 32 tiles of the wave at a time: lane 2 i + b has block b of the i-th
  for (int tb = t0 + wave; tb < t1; tb += 32 * NW) {
    const int count = min(32, (t1 - tb + NW - 1) / NW);
    const int block = min(2 * (tb + NW * min(lane >> 1, count - 1)) + (lane & 1), (lim - 1) >> 4);   // (one behind the last is the last)
    int page = p.t.table[(int64_t)s * p.t.table_pages + (block >> (p.t.page_shift - 4))];
    if (page < 0 || page >= p.t.pages) {
      atomicOr(p.t.err, BC_ERRBIT_STATE);
      page = 0;
    }
    const int per_page = p.t.page_shift - 4;
    const uint32_t unit = (((uint32_t)page * p.Hkv + kvh) << per_page) + (block & ((1 << per_page) - 1));
    const float k_scale = p.ks[unit] * p.qs, v_scale = p.vs[unit];

    auto load = [&](Tile<D>& x, int i) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint64_t at = (uint64_t)lane_value(unit, 2 * i + b) * BLOCK_BYTES;
#pragma unroll
        for (int h = 0; h < H; ++h) x.k[b][h] = *reinterpret_cast<const u32x4_t*>(p.k + at + (k_lane + 256 * h));
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint64_t at = (uint64_t)lane_value(unit, 2 * i + b) * BLOCK_BYTES;
#pragma unroll
        for (int h = 0; h < H; ++h) x.v[b][h] = *reinterpret_cast<const u32x4_t*>(p.v + at + (v_lane + 256 * h));
      }
    };
    auto work = [&](Tile<D>& x, int i) {
      const int key0 = 32 * (tb + NW * i);
      f32x4_t sc[CT][2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) sc[ct][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const bf16x8_t a = operand_of(x.k[b][h][2 * e], x.k[b][h][2 * e + 1]);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) sc[ct][b] = mfma16(a, q[ct][2 * h + e], sc[ct][b]);
          }
      }
      const bool ends = key0 + 32 > seen_by_all;
      bf16x8_t hi[CT], lo[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float z[8];
        float top = kMasked;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const float f = __uint_as_float(lane_value(__float_as_uint(k_scale), 2 * i + b));
#pragma unroll
          for (int r = 0; r < 4; ++r) z[4 * b + r] = sc[ct][b][r] * f;
        }
        if (ends) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (key0 + 16 * b + 4 * g4 + r >= key_lim[ct]) z[4 * b + r] = kMasked;
        }
#pragma unroll
        for (int r = 0; r < 8; ++r) top = fmaxf(top, z[r]);
        top = fmaxf(rows_allreduce_max(top), m[ct]);
        if (__any(top > m[ct])) {
          const float was = fast_exp2(m[ct] - top);
          l[ct] *= was;
#pragma unroll
          for (int j = 0; j < 4 * H; ++j) o[ct][j] *= was;
          m[ct] = top;
        }
        float w[8];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const float f = __uint_as_float(lane_value(__float_as_uint(v_scale), 2 * i + b));
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float e = fast_exp2(z[4 * b + r] - m[ct]);
            l[ct] += e;
            w[4 * b + r] = e * f;
          }
        }
        u32x4_t wh, wl;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          wh[r] = pack2_bf16(w[2 * r], w[2 * r + 1]);
          wl[r] = pack2_bf16(w[2 * r] - __uint_as_float(wh[r] << 16), w[2 * r + 1] - __uint_as_float(wh[r] & 0xffff0000u));
        }
        hi[ct] = __builtin_bit_cast(bf16x8_t, wh);
        lo[ct] = __builtin_bit_cast(bf16x8_t, wl);
      }
      if (key0 + 32 > L) {                     // bytes behind the last entry may be anything: zeros, not a product with a weight of zero
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int there = L - (key0 + 16 * b + 4 * g4);
          const uint32_t mask = there >= 4 ? 0xffffffffu : there <= 0 ? 0u : (1u << (8 * there)) - 1;
#pragma unroll
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) x.v[b][h][j] &= mask;
        }
      }
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x8_t a = operand_of(x.v[0][h][j], x.v[1][h][j]);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            o[ct][4 * h + j] = mfma16(a, hi[ct], o[ct][4 * h + j]);
            o[ct][4 * h + j] = mfma16(a, lo[ct], o[ct][4 * h + j]);
          }
        }
    };
    Tile<D> a, b;
    load(a, 0);
    for (int i = 0; i < count; i += 2) {
      load(b, min(i + 1, count - 1));
      work(a, i);
      if (i + 1 >= count) break;
      load(a, min(i + 2, count - 1));
      work(b, i + 1);
    }
  }

  // the waves' sums: a lane has elements 64 h + 16 g4 + 4 r + j of its column
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const float sum = rows_allreduce_sum(l[ct]);
    if (g4 == 0) { s_ml[wave][16 * ct + c16][0] = m[ct]; s_ml[wave][16 * ct + c16][1] = sum; }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f32x4_t*>(&s_o[wave][16 * ct + c16][64 * h + 16 * g4 + 4 * r]) =
            f32x4_t{o[ct][4 * h][r], o[ct][4 * h + 1][r], o[ct][4 * h + 2][r], o[ct][4 * h + 3][r]};
  }
  __syncthreads();
  const int pair = s * p.Hkv + kvh;
  float* mine = p.part + ((int64_t)pair * p.max_chunks + chunk) * COLS * (D + 2);
  for (int at = tid; at < own * (D / 4); at += 64 * NW) {
    const int c = at / (D / 4), x = 4 * (at % (D / 4));
    float top = kNegBig;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, s_ml[w][c][0]);
    float sum = 0.f;
    f32x4_t r{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = fast_exp2(s_ml[w][c][0] - top);
      sum += f * s_ml[w][c][1];
      r += f * *reinterpret_cast<const f32x4_t*>(&s_o[w][c][x]);
    }
    if (chunks == 1) {
      const int i = (col0 + c) / p.g;
      float* to = p.out + ((span.row + i) * p.Hq + kvh * p.g + (col0 + c - i * p.g)) * D + x;
      *reinterpret_cast<f32x4_t*>(to) = r * (1.f / sum);
    } else {
      store2_past(mine + c * D + x, r[0], r[1]);
      store2_past(mine + c * D + x + 2, r[2], r[3]);
      if (x == 0) store2_past(mine + COLS * D + 2 * c, top, sum);
    }
  }
  if (chunks == 1) return;
  // the workgroup that arrives last adds the parts up, in their order
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) s_last = __hip_atomic_fetch_add(p.arrivals + pair, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (s_last != chunks - 1) return;
  if (tid == 0) __hip_atomic_store(p.arrivals + pair, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const float* parts = p.part + (int64_t)pair * p.max_chunks * COLS * (D + 2);
  for (int at = tid; at < own * (D / 2); at += 64 * NW) {
    const int c = at / (D / 2), x = 2 * (at % (D / 2));
    float top = kNegBig, sum = 0.f, r0 = 0.f, r1 = 0.f;
    for (int k0 = 0; k0 < chunks; k0 += 8) {
      uint64_t ml[8], r[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float* one = parts + (int64_t)min(k0 + k, chunks - 1) * COLS * (D + 2);
        ml[k] = load2_past(one + COLS * D + 2 * c);
        r[k] = load2_past(one + c * D + x);
      }
      float high = top;
#pragma unroll
      for (int k = 0; k < 8; ++k) high = fmaxf(high, low_of(ml[k]));
      const float was = fast_exp2(top - high);
      top = high; sum *= was; r0 *= was; r1 *= was;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float f = k0 + k < chunks ? fast_exp2(low_of(ml[k]) - top) : 0.f;
        sum += f * high_of(ml[k]); r0 += f * low_of(r[k]); r1 += f * high_of(r[k]);
      }
    }
    const int i = (col0 + c) / p.g;
    float* to = p.out + ((span.row + i) * p.Hq + kvh * p.g + (col0 + c - i * p.g)) * D + x;
    const float f = 1.f / sum;
    to[0] = r0 * f; to[1] = r1 * f;
  }
}

struct AttendLaunch {
  int ct, waves, column_blocks, max_chunks, chunk_tiles;
  size_t part_bytes;
  bool fits;
};
AttendLaunch plan_attend(const bc_shape* sh, int64_t max_new, int64_t max_len) {
  AttendLaunch a{};
  const int64_t g = sh->Hq / sh->Hkv, columns = max_new * g, pairs = (int64_t)sh->B * sh->Hkv;
  a.ct = columns <= 16 ? 1 : 2;
  a.waves = 4;
  const int64_t blocks = (columns + 16 * a.ct - 1) / (16 * a.ct), tiles = (max_len + 31) / 32;
  int64_t chunks = 1;
  a.chunk_tiles = 4;
  if (blocks == 1) {
    chunks = (1024 + pairs - 1) / pairs;
    if (chunks > 64) chunks = 64;
    if (chunks > (tiles + 3) / 4) chunks = (tiles + 3) / 4;
    if (chunks < 1) chunks = 1;
  }
  a.max_chunks = (int)chunks;
  a.fits = columns <= 0x7fffffff && pairs * blocks * chunks <= 0x7fffffff;
  a.column_blocks = (int)blocks;
  a.part_bytes = chunks > 1 ? (size_t)(pairs * chunks * 16 * a.ct * (sh->d + 2)) * 4 : 0;
  return a;
}

template <int D>
void launch_attend(const AttendParams& p, const AttendLaunch& a, hipStream_t s) {
  const unsigned grid = (unsigned)((int64_t)p.t.B * p.Hkv * a.column_blocks * a.max_chunks);
  if (a.ct == 1) paged_few_kernel<D, 1, 4><<<grid, 256, 0, s>>>(p);
  else paged_few_kernel<D, 2, 4><<<grid, 256, 0, s>>>(p);
}

int64_t longest(const bc_pages* pg) {
  const int64_t all = (int64_t)pg->table_pages * pg->page_rows;
  return pg->max_len > 0 && pg->max_len < all ? pg->max_len : all;
}

}  // namespace
}  // namespace bc

using namespace bc;

extern "C" size_t bc_paged_workspace_bytes(const bc_shape* shape, int32_t max_new, int32_t max_len) {
  if (check_shape(shape) != BC_OK || max_new < 0 || max_len < 1 || (int64_t)shape->B * shape->Hkv > (1 << 23)) return 0;
  if (!plan_attend(shape, max_new, max_len).fits) return 0;
  // (fewer rows may be cut where more are not)
  size_t most = 0;
  const int64_t g = shape->Hq / shape->Hkv;
  for (int64_t n : {(int64_t)1, 16 / g, 32 / g, (int64_t)max_new}) {
    const AttendLaunch a = plan_attend(shape, n < max_new ? n : max_new, max_len);
    if (a.fits && a.part_bytes > most) most = a.part_bytes;
  }
  return most + 16;
}

extern "C" int32_t bc_paged_attend(const bc_shape* shape, const bc_pages* pages, int64_t rows, const int64_t* row_offsets, int32_t max_new,
                                   const void* q, float* out, const uint8_t* active, void* workspace, size_t workspace_bytes, void* stream) {
  const int32_t st = check_pages(shape, pages, rows, row_offsets, max_new);
  if (st != BC_OK) return st;
  if (!nonnegative_finite(shape->scale)) return BC_ERR_ARG;
  if (rows == 0 || max_new == 0) return BC_OK;
  if (!row_offsets) max_new = 1;
  if (!q || !out || !aligned16(q) || !aligned16(out) || !pages->arrivals) return BC_ERR_ARG;
  const int64_t max_len = longest(pages);
  // (a sequence cannot have more new rows than there are, nor than entries)
  int64_t most = max_new < rows ? max_new : rows;
  if (most > max_len) most = max_len;
  const AttendLaunch a = plan_attend(shape, most, max_len);
  if (!a.fits) return BC_ERR_SHAPE;
  if (a.part_bytes && (!workspace || !aligned16(workspace) || workspace_bytes < a.part_bytes)) return BC_ERR_WORKSPACE;
  AttendParams p{};
  p.t = paged_tables(shape, pages, rows, row_offsets, (int32_t)most, active);
  p.q = static_cast<const char*>(q); p.out = out;
  p.k = static_cast<const uint8_t*>(pages->k); p.v = static_cast<const uint8_t*>(pages->v); p.ks = pages->k_scale; p.vs = pages->v_scale;
  p.arrivals = pages->arrivals; p.part = static_cast<float*>(workspace);
  p.Hq = shape->Hq; p.Hkv = shape->Hkv; p.g = shape->Hq / shape->Hkv; p.max_len = (int32_t)max_len;
  p.column_blocks = a.column_blocks; p.max_chunks = a.max_chunks; p.chunk_tiles = a.chunk_tiles;
  p.qs = shape->scale * kLog2e;
  if (shape->d == 128) launch_attend<128>(p, a, as_stream(stream)); else launch_attend<64>(p, a, as_stream(stream));
  return launch_status();
}
