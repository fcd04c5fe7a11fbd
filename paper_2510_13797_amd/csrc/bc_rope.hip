// The packed output of a layer's projections -> the q, k and v that the attention calls take: RMS norm of every query and key head,
// rotation by position, v copied; and the gradient of that, behind bc_prefill_attn_bwd.
//
//   r = 1 / sqrt(mean(x^2) + eps),  y = w * x * r  (without a weight y = x),  a_i = position * inv_freq_i,  h = rot / 2
//   o_i = y_i cos a_i - y_{i+h} sin a_i,  o_{i+h} = y_{i+h} cos a_i + y_i sin a_i  (i < h),  o_i = y_i  (i >= rot)
//   gradient: dy = o's rotated back,  dw = sum dy x r,  dx = r (w dy - x r^2 mean(w dy x))
//
// Bound by memory: every element in and out once.  139,008 rows of 12/2 heads, d = 128, bf16: 1.14 GB in 203 us, the gradient's 2.21 GB in 420 (5.6 and 5.3 TB/s; torch's copy of
// 2 GiB reaches 4.9); a token of 32/8 heads 3 us beside the call's 13.  d / 8 lanes work on a head, eight elements a lane, in two pieces of four that
// are each other's partners in the rotation: both halves of a pair are in one lane, and an instruction still asks for whole
// 128-byte lines.  A lane's four angles serve all heads of its row that are its item.  All arithmetic in fp32, rounded once
// (angles: angle_of()).
#include "bc_common.h"

namespace bc {
namespace {

constexpr int kRopeThreads = 256;

struct RopeParams {
  const char* qkv;             // [rows, Hq + 2 Hkv, d], rows row_bytes apart
  int64_t row_bytes;
  const int32_t* positions;    // [rows]
  const float* inv_freq;       // [rot / 2]
  const char* qw;              // [d] or null
  const char* kw;
  char* q;                     // [rows, Hq, d], [rows, Hkv, d] (v: or null)
  char* k;
  char* v;
  const float* dq;             // gradients of those (dv: or null)
  const float* dk;
  const float* dv;
  char* dqkv;                  // gradient of qkv, rows drow_bytes apart
  int64_t drow_bytes;
  float* partial;              // [workgroups][2][d] sums of dw, or null
  int64_t rows;
  int32_t Hq, Hkv, half;       // half: rot / 2
  int32_t heads;               // worked on: Hq + Hkv, and Hkv more where v is
  int32_t chunks, per_item;    // a row's heads as `chunks` items of per_item
  float eps;
};

// four elements <-> floats.  STREAM: past the caches (rope_streams())
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
  __device__ __forceinline__ RopeLane(const RopeParams& p, int lane, int32_t position) {
    const int at = 4 * lane;
    turns = at < p.half;
    o1 = turns ? at : 2 * at;               // (behind the rotated part eight in a row: 2 * half + 8 * (lane - half / 4))
    o2 = turns ? p.half + at : o1 + 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      c[e] = 1.f; s[e] = 0.f;
      if (turns) angle_of(position, p.inv_freq[at + e], c[e], s[e]);
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

template <typename T, int D, bool NORM, bool STREAM, int U>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_kernel(RopeParams p) {
  constexpr int LPH = D / 8, ES = Elem<T>::size, HEAD = D * ES;
  const int lane = threadIdx.x % LPH;
  const uint32_t item = blockIdx.x * (kRopeThreads / LPH) + threadIdx.x / LPH, at = item / (uint32_t)p.chunks;
  const int64_t row = at;
  if (row >= p.rows) return;
  const int first = (int)(item - at * p.chunks) * p.per_item, last = min(first + p.per_item, p.heads);
  const RopeLane<D> ln(p, lane, p.positions[row]);
  float wq[2][4], wk[2][4];
  const bool nq = NORM && p.qw != nullptr, nk = NORM && p.kw != nullptr;
  if (nq) { load4(p.qw + ln.o1 * ES, wq[0], T{}); load4(p.qw + ln.o2 * ES, wq[1], T{}); }
  if (nk) { load4(p.kw + ln.o1 * ES, wk[0], T{}); load4(p.kw + ln.o2 * ES, wk[1], T{}); }
  const char* in = p.qkv + row * p.row_bytes;
  for (int h0 = first; h0 < last; h0 += U) {
    float x[U][2][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = min(h0 + u, last - 1);
      load4<STREAM>(in + (int64_t)h * HEAD + ln.o1 * ES, x[u][0], T{});
      load4<STREAM>(in + (int64_t)h * HEAD + ln.o2 * ES, x[u][1], T{});
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u;
      if (h >= last) break;
      char* out = h < p.Hq ? p.q + (row * p.Hq + h) * HEAD
                           : h < p.Hq + p.Hkv ? p.k + (row * p.Hkv + h - p.Hq) * HEAD : p.v + (row * p.Hkv + h - p.Hq - p.Hkv) * HEAD;
      if (h < p.Hq + p.Hkv) {
        if (NORM && (h < p.Hq ? nq : nk)) {
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) sum += x[u][0][e] * x[u][0][e] + x[u][1][e] * x[u][1][e];
          const float r = 1.f / sqrtf(group_allreduce_sum<LPH>(sum) * (1.f / D) + p.eps);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[u][0][e] *= r * (h < p.Hq ? wq[0][e] : wk[0][e]);
            x[u][1][e] *= r * (h < p.Hq ? wq[1][e] : wk[1][e]);
          }
        }
        ln.template turn<false>(x[u][0], x[u][1]);
      }
      store4<STREAM>(out + ln.o1 * ES, x[u][0], T{});
      store4<STREAM>(out + ln.o2 * ES, x[u][1], T{});
    }
  }
}

// (The sums of dw are of 32 bits over a lane's items and a workgroup's lanes, some hundred terms, and of 64 behind that: 360,000 rows of four heads, whose sums are about a
// thousand, are off by 5e-4 at most.)
template <typename T, int D, bool NORM, bool STREAM>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_bwd_kernel(RopeParams p) {
  constexpr int LPH = D / 8, ES = Elem<T>::size, HEAD = D * ES, GROUPS = kRopeThreads / LPH;
  __shared__ float sums[NORM ? GROUPS : 1][NORM ? D : 1];
  const int lane = threadIdx.x % LPH, group = threadIdx.x / LPH;
  float aq[2][4] = {}, ak[2][4] = {};
  int o1 = 0, o2 = 0;
  const bool nq = NORM && p.qw != nullptr, nk = NORM && p.kw != nullptr;
  for (uint32_t item = blockIdx.x * GROUPS + group;; item += gridDim.x * GROUPS) {
    const uint32_t at = item / (uint32_t)p.chunks;
    const int64_t row = at;
    if (row >= p.rows) break;
    const int first = (int)(item - at * p.chunks) * p.per_item, last = min(first + p.per_item, p.heads);
    const RopeLane<D> ln(p, lane, p.positions[row]);
    o1 = ln.o1; o2 = ln.o2;
    float wq[2][4], wk[2][4];
    if (nq) { load4(p.qw + o1 * ES, wq[0], T{}); load4(p.qw + o2 * ES, wq[1], T{}); }
    if (nk) { load4(p.kw + o1 * ES, wk[0], T{}); load4(p.kw + o2 * ES, wk[1], T{}); }
    for (int h = first; h < last; ++h) {
      const bool isq = h < p.Hq, norm = NORM && h < p.Hq + p.Hkv && (isq ? nq : nk);
      const float* g = isq ? p.dq + (row * p.Hq + h) * D
                           : h < p.Hq + p.Hkv ? p.dk + (row * p.Hkv + h - p.Hq) * D : p.dv + (row * p.Hkv + h - p.Hq - p.Hkv) * D;
      float dy[2][4], x[2][4];
      load4<STREAM>(reinterpret_cast<const char*>(g + o1), dy[0], 0.f);
      load4<STREAM>(reinterpret_cast<const char*>(g + o2), dy[1], 0.f);
      if (norm) {
        const char* in = p.qkv + row * p.row_bytes + (int64_t)h * HEAD;
        load4<STREAM>(in + o1 * ES, x[0], T{});
        load4<STREAM>(in + o2 * ES, x[1], T{});
      }
      if (h < p.Hq + p.Hkv) ln.template turn<true>(dy[0], dy[1]);
      if (norm) {
        float sum = 0.f, dot = 0.f;
        float wdy[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            wdy[i][e] = dy[i][e] * (isq ? wq[i][e] : wk[i][e]);
            sum += x[i][e] * x[i][e];
            dot += wdy[i][e] * x[i][e];
          }
        const float r = 1.f / sqrtf(group_allreduce_sum<LPH>(sum) * (1.f / D) + p.eps);
        const float m = group_allreduce_sum<LPH>(dot) * (1.f / D) * r * r;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float dw = dy[i][e] * x[i][e] * r;
            if (isq) aq[i][e] += dw; else ak[i][e] += dw;
            dy[i][e] = r * (wdy[i][e] - x[i][e] * m);
          }
      }
      char* out = p.dqkv + row * p.drow_bytes + (int64_t)h * HEAD;
      store4<STREAM>(out + o1 * ES, dy[0], T{});
      store4<STREAM>(out + o2 * ES, dy[1], T{});
    }
  }
  if constexpr (NORM) {
    if (p.partial == nullptr) return;
    // (a group without an item has zeros, and its lanes' places from no item: those of a position's own)
    const int at = 4 * lane;
    o1 = at < p.half ? at : 2 * at;
    o2 = at < p.half ? p.half + at : o1 + 4;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sums[group][o1 + e] = which ? ak[0][e] : aq[0][e];
        sums[group][o2 + e] = which ? ak[1][e] : aq[1][e];
      }
      __syncthreads();
      if (threadIdx.x < D) {
        float t = 0.f;
        for (int g = 0; g < GROUPS; ++g) t += sums[g][threadIdx.x];
        p.partial[((int64_t)blockIdx.x * 2 + which) * D + threadIdx.x] = t;
      }
    }
  }
}

// dw from the workgroups' sums, in a fixed order: 16 columns a workgroup, 64 slices of the workgroups, whose sums a thread asks for all together
// (16 slices, one load after the other: 22 us for 1024 workgroups, 3 so).
constexpr int kRopeBwdMost = 1024;       // workgroups of the gradient, each with its sums of dw
template <int D>
__global__ void __launch_bounds__(1024) rope_weight_sum_kernel(const float* partial, int n, float* dqw, float* dkw) {
  constexpr int SLICES = 64, EACH = kRopeBwdMost / SLICES;
  __shared__ double part[SLICES][17];
  const int c = threadIdx.x & 15, slice = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  float x[EACH];
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    const int i = slice + k * SLICES;
    x[k] = partial[(int64_t)(i < n ? i : 0) * 2 * D + col];
  }
  double t = 0.0;
#pragma unroll
  for (int k = 0; k < EACH; ++k) t += slice + k * SLICES < n ? (double)x[k] : 0.0;
  part[slice][c] = t;
  for (int half = SLICES / 2; half >= 1; half >>= 1) {
    __syncthreads();
    if (slice < half) part[slice][c] += part[slice + half][c];
  }
  if (slice == 0) {
    float* to = col < D ? dqw : dkw;
    if (to) to[col & (D - 1)] = (float)part[0][c];
  }
}

// Heads of an item: one, so that few rows spread over the chip, and a whole row (its angles worked out once) where there are
// more heads than lanes to work on them.  (With fewer than 32768 rows an item number fits 32 bits as 65536 heads at most do; with
// more, a row is an item.)
void deal_heads(RopeParams& p) {
  constexpr int64_t kItems = 32768;
  const int64_t n = p.rows * p.heads / kItems;
  p.per_item = (int)(n < 1 ? 1 : n < p.heads ? n : p.heads);
  p.chunks = (p.heads + p.per_item - 1) / p.per_item;
}
int64_t rope_groups(const RopeParams& p, int d) {
  const int64_t per = kRopeThreads / (d / 8);
  return (p.rows * p.chunks + per - 1) / per;
}

int32_t check_rope(const bc_shape* sh, int64_t rows, int64_t stride, const int32_t* positions, const float* inv_freq, int32_t rot,
                   const void* qw, const void* kw, float eps) {
  const int32_t st = check_shape(sh);
  if (st != BC_OK) return st;
  if (rows < 0 || rows > 0x7fffffff || (int64_t)sh->Hq + 2 * (int64_t)sh->Hkv > 65536 || rot < 0 || rot > sh->d || rot % 8 != 0) return BC_ERR_SHAPE;
  if (!nonnegative_finite(eps)) return BC_ERR_ARG;
  if (rows == 0) return BC_OK;
  if (!positions || (rot > 0 && !inv_freq)) return BC_ERR_ARG;
  if (stride < (int64_t)(sh->Hq + 2 * (int64_t)sh->Hkv) * sh->d || stride > (1LL << 31) || stride * elem_size(sh->kv_dtype) % 16 != 0) return BC_ERR_ARG;
  if ((qw && !aligned16(qw)) || (kw && !aligned16(kw))) return BC_ERR_ARG;
  return BC_OK;
}
void fill_rope(RopeParams& p, const bc_shape* sh, int64_t rows, const void* qkv, int64_t stride, const int32_t* positions,
               const float* inv_freq, int32_t rot, const void* qw, const void* kw, float eps) {
  p.qkv = static_cast<const char*>(qkv);
  p.row_bytes = stride * elem_size(sh->kv_dtype);
  p.positions = positions; p.inv_freq = inv_freq;
  p.qw = static_cast<const char*>(qw); p.kw = static_cast<const char*>(kw);
  p.rows = rows; p.Hq = sh->Hq; p.Hkv = sh->Hkv; p.half = rot / 2; p.eps = eps;
}

// Packed rows beyond the 256 MB of the Infinity Cache go past it, in and out: 139,008 rows of 12/2 heads, d = 128, forward and gradients 678 -> 633 us.  Smaller ones
// leave their results there for the attention that reads them next: forward and attention of 24,000 rows 113 us, streamed 133 (139,008: 772 and 766).
bool rope_streams(const RopeParams& p, int d, int es) { return p.rows * (p.Hq + 2 * (int64_t)p.Hkv) * d * es > (256LL << 20); }

template <typename T, int D, bool STREAM>
void launch_rope(const RopeParams& p, hipStream_t s) {
  const dim3 grid((unsigned)rope_groups(p, D));
  if (p.qw || p.kw) qk_norm_rope_kernel<T, D, true, STREAM, 4><<<grid, kRopeThreads, 0, s>>>(p);
  else qk_norm_rope_kernel<T, D, false, STREAM, 4><<<grid, kRopeThreads, 0, s>>>(p);
}
template <typename T, int D>
void launch_rope(const RopeParams& p, hipStream_t s) {
  if (rope_streams(p, D, Elem<T>::size)) launch_rope<T, D, true>(p, s);
  else launch_rope<T, D, false>(p, s);
}
template <typename T, int D, bool STREAM>
void launch_rope_bwd(const RopeParams& p, float* dqw, float* dkw, hipStream_t s) {
  const int64_t want = rope_groups(p, D);
  const int n = (int)(want < kRopeBwdMost ? want : kRopeBwdMost);
  if (n == 0) {                            // (no rows: dw is zero)
  } else if (p.qw || p.kw) qk_norm_rope_bwd_kernel<T, D, true, STREAM><<<n, kRopeThreads, 0, s>>>(p);
  else qk_norm_rope_bwd_kernel<T, D, false, STREAM><<<n, kRopeThreads, 0, s>>>(p);
  if (p.partial) rope_weight_sum_kernel<D><<<2 * D / 16, 1024, 0, s>>>(p.partial, n, dqw, dkw);
}
template <typename T, int D>
void launch_rope_bwd(const RopeParams& p, float* dqw, float* dkw, hipStream_t s) {
  if (rope_streams(p, D, Elem<T>::size)) launch_rope_bwd<T, D, true>(p, dqw, dkw, s);
  else launch_rope_bwd<T, D, false>(p, dqw, dkw, s);
}

}  // namespace
}  // namespace bc

using namespace bc;

extern "C" int32_t bc_qk_norm_rope(const bc_shape* shape, int64_t rows, const void* qkv, int64_t qkv_row_stride, const int32_t* positions,
                                   const float* inv_freq, int32_t rot, const void* q_weight, const void* k_weight, float eps, void* q,
                                   void* k, void* v, void* stream) {
  const int32_t st = check_rope(shape, rows, qkv_row_stride, positions, inv_freq, rot, q_weight, k_weight, eps);
  if (st != BC_OK || rows == 0) return st;
  if (q == qkv || k == qkv || v == qkv) return BC_ERR_ARG;
  if (!qkv || !q || !k || !aligned16(qkv) || !aligned16(q) || !aligned16(k) || !aligned16(v)) return BC_ERR_ARG;
  RopeParams p{};
  fill_rope(p, shape, rows, qkv, qkv_row_stride, positions, inv_freq, rot, q_weight, k_weight, eps);
  p.q = static_cast<char*>(q); p.k = static_cast<char*>(k); p.v = static_cast<char*>(v);
  p.heads = p.Hq + (v ? 2 : 1) * p.Hkv;
  deal_heads(p);
  hipStream_t s = as_stream(stream);
  if (shape->kv_dtype == BC_BF16) {
    if (shape->d == 128) launch_rope<bf16_t, 128>(p, s); else launch_rope<bf16_t, 64>(p, s);
  } else {
    if (shape->d == 128) launch_rope<float, 128>(p, s); else launch_rope<float, 64>(p, s);
  }
  return launch_status();
}

extern "C" size_t bc_qk_norm_rope_bwd_workspace_bytes(const bc_shape* shape) {
  if (check_shape(shape) != BC_OK) return 0;
  return (size_t)kRopeBwdMost * 2 * shape->d * sizeof(float);
}

extern "C" int32_t bc_qk_norm_rope_bwd(const bc_shape* shape, int64_t rows, const void* qkv, int64_t qkv_row_stride, const int32_t* positions,
                                       const float* inv_freq, int32_t rot, const void* q_weight, const void* k_weight, float eps,
                                       const float* dq, const float* dk, const float* dv, void* dqkv, int64_t dqkv_row_stride,
                                       float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes, void* stream) {
  int32_t st = check_rope(shape, rows, qkv_row_stride, positions, inv_freq, rot, q_weight, k_weight, eps);
  if (st != BC_OK) return st;
  if ((dq_weight && !q_weight) || (dk_weight && !k_weight)) return BC_ERR_ARG;
  const bool sums = dq_weight || dk_weight;
  if (sums && (!workspace || !aligned16(workspace) || workspace_bytes < bc_qk_norm_rope_bwd_workspace_bytes(shape))) return BC_ERR_WORKSPACE;
  if (rows > 0) {
    st = check_rope(shape, rows, dqkv_row_stride, positions, inv_freq, rot, q_weight, k_weight, eps);
    if (st != BC_OK) return st;
    if (!dq || !dk || !dqkv || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) || !aligned16(dqkv)) return BC_ERR_ARG;
    if ((q_weight || k_weight) && (!qkv || !aligned16(qkv))) return BC_ERR_ARG;
    if (dqkv == qkv && dqkv_row_stride != qkv_row_stride) return BC_ERR_ARG;
  }
  RopeParams p{};
  fill_rope(p, shape, rows, qkv, qkv_row_stride, positions, inv_freq, rot, q_weight, k_weight, eps);
  p.dq = dq; p.dk = dk; p.dv = dv;
  p.dqkv = static_cast<char*>(dqkv); p.drow_bytes = dqkv_row_stride * elem_size(shape->kv_dtype);
  p.partial = sums ? static_cast<float*>(workspace) : nullptr;
  p.heads = p.Hq + (dv ? 2 : 1) * p.Hkv;
  if (rows == 0 && !sums) return BC_OK;
  deal_heads(p);
  hipStream_t s = as_stream(stream);
  if (shape->kv_dtype == BC_BF16) {
    if (shape->d == 128) launch_rope_bwd<bf16_t, 128>(p, dq_weight, dk_weight, s); else launch_rope_bwd<bf16_t, 64>(p, dq_weight, dk_weight, s);
  } else {
    if (shape->d == 128) launch_rope_bwd<float, 128>(p, dq_weight, dk_weight, s); else launch_rope_bwd<float, 64>(p, dq_weight, dk_weight, s);
  }
  return launch_status();
}
