// bc_paged_append: rows of packed projections -> queries in bf16, and keys and values as entries of a cache in 8-bit pages (Alg. 1's "KV is updated
// internally", "encode b" and "encode the prompt", over pages): RMS norm of the query and key heads, rotation by position, and e4m3 with a
// scale for each block of 16 entries and head.
//
//   y, o: as in bc_rope.hip.  Block scale s = 2^e, the least one (e >= -120) with |x| <= 448 s for every finite x written to the block
//   since its first entry; an entry's byte is e4m3(x / s).  A block's scale only grows while it holds entries; those that stay then become
//   e4m3(old * old s / s).
//
// A power of two: dividing by it is exact, so an e4m3 value keeps its bits when a block's scale grows (but for the few below 2^-6), and an
// entry's error is the one rounding, 2^-4 of its value, that any scale would leave.
//
// Bound by memory where rows are many (139,008 rows of 12/2 heads, d = 128, bf16: 1.07 GB in 186 us, 5.7 TB/s; torch's copy of 2 GiB
// reaches 5.1), by the latency of tables and loads where they are few (24 chunks of up to 130 rows, 14/2 heads, d = 64, fp32: 8.8 us; a row
// of 32/8 heads: 4.2, beside 9 of the call).  Two kernels:
//   a block of 16 entries a workgroup (few rows: several, which share the heads), d / 8 lanes a row: the block's largest magnitude goes through LDS;
//   one new row a sequence at most (a decode step): a workgroup a sequence, a wave for the key or the value of a head; the rest of the
//   block is touched only where its scale grows.
#include "bc_paged.h"
#include "bc_rope_lane.h"

namespace bc {
namespace {

struct AppendParams {
  PagedTables t;
  const char* qkv;             // [rows, Hq + 2 Hkv, d], rows row_bytes apart
  int64_t row_bytes;
  const int32_t* positions;    // [rows]
  const float* inv_freq;       // [half]
  const char* qw;              // [d] or null
  const char* kw;
  const int32_t* keep;         // [B] or null
  char* q;                     // [rows, Hq, d] bf16, or null
  uint8_t* k;                  // [pages, Hkv, page_rows, d]
  uint8_t* v;
  float* ks;                   // [pages, Hkv, page_rows / 16]
  float* vs;
  int32_t Hq, Hkv, half;
  int32_t* arrivals;           // [B * Hkv] zero between launches
  uint32_t base;               // block kernel: the launch's first workgroup,
  uint32_t blocks, turns;      // blocks of a sequence, workgroups of a block,
  int32_t kv_turns, kv_share;  // those that share its keys and values, and heads of either that each has;
  int32_t q_from, q_share;     // the first one that has queries, and heads that each has
  float eps;
};

__device__ __forceinline__ bool finite_bits(float x) { return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u; }

// The exponent of the least power of two s with most <= 448 s: 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(float most) {
  return max((int)((__float_as_uint(most) + 0x1fffffu) >> 23) - 127 - 8, -120);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// 1 / s of a scale that is one (2^-120 .. 2^120: both are normal)
__device__ __forceinline__ float inverse_of(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

// What is not finite is stored as a NaN.
__device__ __forceinline__ float storable(float x) { return finite_bits(x) ? x : __uint_as_float(0x7fc00000u); }
__device__ __forceinline__ uint32_t quantise(const float (&x)[4], float inv) {
  return pack_e4m3(storable(x[0]) * inv, storable(x[1]) * inv, storable(x[2]) * inv, storable(x[3]) * inv);
}
__device__ __forceinline__ float largest(const float (&x)[2][4]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) m = fmaxf(m, finite_bits(x[i][e]) ? fabsf(x[i][e]) : 0.f);
  return m;
}

// Where row r of a page's head has element o (bytes from the head's first): keys, values.
template <int D> __device__ __forceinline__ int key_at(int r, int o) { return (r >> 2) * 4 * D + (o >> 6) * 256 + (r & 3) * 64 + (o & 63); }
template <int D> __device__ __forceinline__ int value_at(int r, int o) { return (r >> 2) * 4 * D + o * 4 + (r & 3); }

// What a call does to a sequence, the same for every wave that asks (all 64 lanes together): nothing where n == 0.
struct AppendPlan { int64_t row; int n, start; };
__device__ __forceinline__ AppendPlan append_plan(const AppendParams& p, int s, int lane, bool herald) {
  const PagedSpan span = paged_span(p.t, s);
  const int L = span.len, start = p.keep ? p.keep[s] : L;
  if (span.n == 0) return {0, 0, 0};
  int bad = span.n < 0 || L < 0 || start < 0 || start > L ? BC_ERRBIT_STATE : 0;
  if (!bad && (int64_t)start + span.n > (int64_t)p.t.table_pages << p.t.page_shift) bad = BC_ERRBIT_CAPACITY;
  if (!bad) {
    const int first = start >> p.t.page_shift, last = (start + span.n - 1) >> p.t.page_shift;
    bool out = false;
    for (int i = first + lane; i <= last; i += 64) {
      const int page = p.t.table[(int64_t)s * p.t.table_pages + i];
      out |= page < 0 || page >= p.t.pages;
    }
    if (__ballot(out)) bad = BC_ERRBIT_STATE;
  }
  if (bad) {
    if (herald && lane == 0) atomicOr(p.t.err, bad);
    return {0, 0, 0};
  }
  return {span.row, span.n, start};
}

template <typename T, int D, bool NORM>
__device__ __forceinline__ void norm_head(float (&x)[2][4], const float (&w)[2][4], float eps) {
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) sum += x[0][e] * x[0][e] + x[1][e] * x[1][e];
  const float r = 1.f / sqrtf(group_allreduce_sum<D / 8>(sum) * (1.f / D) + eps);
#pragma unroll
  for (int e = 0; e < 4; ++e) { x[0][e] *= r * w[0][e]; x[1][e] *= r * w[1][e]; }
}

// 16 rows' lanes: 256 threads, 128 for d = 64.  A block has p.turns workgroups: the first kv_turns share the heads of keys and of values,
// the others those of queries; one alone has all.  (Five waves a SIMD: 256 x 2-4 rows 29.6 us with four, 28.0.  In fp32 with norms that is
// two registers short.)
template <typename T, int D, bool NORM, bool STREAM>
__global__ void __launch_bounds__(2 * D, Elem<T>::size == 2 ? 5 : 4) paged_append_kernel(AppendParams p) {
  constexpr int LPH = D / 8, ES = Elem<T>::size, HEAD = D * ES, U = 4;
  __shared__ float s_most[U][kPagedBlock];
  const int lane = threadIdx.x % LPH, mine = threadIdx.x / LPH;      // a row of the block
  const uint32_t of_sequence = p.blocks * p.turns, id = p.base + blockIdx.x;
  const int s = id / of_sequence, at_block = id - s * of_sequence, j = at_block / p.turns, turn = at_block - j * p.turns;
  const AppendPlan plan = append_plan(p, s, threadIdx.x & 63, at_block == 0 && threadIdx.x < 64);
  if (plan.n == 0) return;
  const int start = plan.start, end = start + plan.n;
  // The length moves when all of the sequence's workgroups have read it, those without rows among them: counted behind the work (in front
  // of it the loads behind the count, which come back in order, waited for its answer: 2 us).
  auto leave = [&] {
    __syncthreads();
    if (threadIdx.x != 0 || __hip_atomic_fetch_add(p.arrivals + s * p.Hkv, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != (int)of_sequence - 1) return;
    __hip_atomic_store(p.arrivals + s * p.Hkv, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    p.t.len[s] = end;
  };
  if (j > ((end - 1) >> 4) - (start >> 4)) return leave();            // (counted in blocks: places behind the last one may pass 31 bits)
  const int first = ((start >> 4) + j) << 4, slot = first + mine;
  const bool fresh = slot >= start && slot < end, stays = slot < start, staying = first < start;
  const int64_t row = plan.row + (fresh ? slot - start : 0);         // (other rows' lanes look at the first one)
  const char* in = p.qkv + row * p.row_bytes;
  const RopeLane<D> ln(p.half, p.inv_freq, lane, p.positions[row]);
  if (p.q && fresh && turn >= p.q_from) {
    float w[2][4];
    const bool norm = NORM && p.qw != nullptr;
    if (norm) { load4(p.qw + ln.o1 * ES, w[0], T{}); load4(p.qw + ln.o2 * ES, w[1], T{}); }
    const int h_first = (turn - p.q_from) * p.q_share, h_end = min(h_first + p.q_share, p.Hq);
    for (int h0 = h_first; h0 < h_end; h0 += U) {
      float x[U][2][4];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = min(h0 + u, h_end - 1);
        load4<STREAM>(in + (int64_t)h * HEAD + ln.o1 * ES, x[u][0], T{});
        load4<STREAM>(in + (int64_t)h * HEAD + ln.o2 * ES, x[u][1], T{});
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h0 + u >= h_end) break;
        if (norm) norm_head<T, D, NORM>(x[u], w, p.eps);
        ln.template turn<false>(x[u][0], x[u][1]);
        char* out = p.q + (row * p.Hq + h0 + u) * (D * 2);
        store4<STREAM>(out + ln.o1 * 2, x[u][0], bf16_t{});
        store4<STREAM>(out + ln.o2 * 2, x[u][1], bf16_t{});
      }
    }
  }
  if (turn >= p.kv_turns) return leave();
  const int page = p.t.table[(int64_t)s * p.t.table_pages + (first >> p.t.page_shift)];
  const int r = slot & ((1 << p.t.page_shift) - 1), per_page = 1 << (p.t.page_shift - 4), block = (first >> 4) & (per_page - 1);
  // keys, then values
  float w[2][4];
  const bool norm = NORM && p.kw != nullptr;
  if (norm) { load4(p.kw + ln.o1 * ES, w[0], T{}); load4(p.kw + ln.o2 * ES, w[1], T{}); }
  const int it_end = min((turn + 1) * p.kv_share, 2 * p.Hkv);
  for (int it = turn * p.kv_share; it < it_end; it += U) {
    float x[U][2][4], was[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int item = min(it + u, it_end - 1), value = item >= p.Hkv, h = item - value * p.Hkv;
      const int o1 = value ? 8 * lane : ln.o1, o2 = value ? 8 * lane + 4 : ln.o2;       // (values are not turned: eight in a row)
      load4<STREAM>(in + (int64_t)(p.Hq + item) * HEAD + o1 * ES, x[u][0], T{});
      load4<STREAM>(in + (int64_t)(p.Hq + item) * HEAD + o2 * ES, x[u][1], T{});
      was[u] = staying ? (value ? p.vs : p.ks)[((int64_t)page * p.Hkv + h) * per_page + block] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int item = min(it + u, it_end - 1), value = item >= p.Hkv, h = item - value * p.Hkv;
      if (stays) {                         // what it holds, for the case that the scale grows (half of it: 256 * 2^120 is no number of 32 bits)
        const uint8_t* old = (value ? p.v : p.k) + ((((int64_t)page * p.Hkv + h) << p.t.page_shift) * D);
        if (value) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float a[4], b[4];
            unpack_e4m3(old[value_at<D>(r, 8 * lane + e)], a);
            unpack_e4m3(old[value_at<D>(r, 8 * lane + 4 + e)], b);
            x[u][0][e] = a[0]; x[u][1][e] = b[0];
          }
        } else {
          unpack_e4m3(*reinterpret_cast<const uint32_t*>(old + key_at<D>(r, ln.o1)), x[u][0]);
          unpack_e4m3(*reinterpret_cast<const uint32_t*>(old + key_at<D>(r, ln.o2)), x[u][1]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[u][0][e] *= 0.5f * was[u]; x[u][1][e] *= 0.5f * was[u]; }
      } else if (!value) {
        if (norm) norm_head<T, D, NORM>(x[u], w, p.eps);
        ln.template turn<false>(x[u][0], x[u][1]);
      }
      const float most = group_allreduce_max<LPH>(fresh ? largest(x[u]) : 0.f);
      if (lane == 0) s_most[u][mine] = most;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int item = it + u, value = item >= p.Hkv, h = item - value * p.Hkv;
      if (item >= it_end) break;
      float most = 0.f;
#pragma unroll
      for (int i = 0; i < kPagedBlock; ++i) most = fmaxf(most, s_most[u][i]);
      const float scale = fmaxf(power_of_two(scale_exponent(most)), was[u]), inv = inverse_of(scale) * (stays ? 2.f : 1.f);
      const int64_t head = (int64_t)page * p.Hkv + h;
      if (threadIdx.x == 0) (value ? p.vs : p.ks)[head * per_page + block] = scale;
      uint8_t* to = (value ? p.v : p.k) + (head << p.t.page_shift) * D;
      uint32_t a = quantise(x[u][0], inv), b = quantise(x[u][1], inv);
      if (!value) {
        if (fresh || (stays && scale != was[u])) {
          *reinterpret_cast<uint32_t*>(to + key_at<D>(r, ln.o1)) = a;
          *reinterpret_cast<uint32_t*>(to + key_at<D>(r, ln.o2)) = b;
        }
      } else {
        // four rows' words of four elements each -> four elements' words of four rows each: rows r ^ 1, then r ^ 2 (v_perm: bytes 0..3 of the second
        // operand, 4..7 of the first)
        const bool odd = r & 1, high = r & 2;
        auto turned = [&](uint32_t x0) {
          const uint32_t y = __shfl_xor(x0, LPH, 64);
          const uint32_t x1 = odd ? __builtin_amdgcn_perm(x0, y, 0x07030501) : __builtin_amdgcn_perm(y, x0, 0x06020400);
          const uint32_t z = __shfl_xor(x1, 2 * LPH, 64);
          return high ? __builtin_amdgcn_perm(x1, z, 0x07060302) : __builtin_amdgcn_perm(z, x1, 0x05040100);
        };
        a = turned(a); b = turned(b);
        // entries behind the last one keep their bytes
        const int group = slot & ~3, whole = end - group;             // rows of the group in front of the end
        if (whole > 0 && (group + 4 > start || scale != was[u])) {
          uint32_t* wa = reinterpret_cast<uint32_t*>(to + value_at<D>(r & ~3, 8 * lane + (r & 3)));
          uint32_t* wb = reinterpret_cast<uint32_t*>(to + value_at<D>(r & ~3, 8 * lane + 4 + (r & 3)));
          if (whole < 4) {
            const uint32_t ours = (1u << (8 * whole)) - 1;
            a = (a & ours) | (*wa & ~ours);
            b = (b & ours) | (*wb & ~ours);
          }
          *wa = a; *wb = b;
        }
      }
    }
    __syncthreads();
  }
  leave();
}

// One new row at most: a workgroup a sequence, whose waves take the keys' and values' heads and then the queries' by turns, and at the end
// the length.
template <typename T, int D, bool NORM>
__global__ void __launch_bounds__(1024) paged_append_one_kernel(AppendParams p) {
  constexpr int LPH = D / 8, ES = Elem<T>::size, HEAD = D * ES, PER = 64 / LPH;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int s = blockIdx.x, in_head = lane % LPH, part = lane / LPH;
  const AppendPlan plan = append_plan(p, s, lane, wave == 0);
  if (plan.n == 0) return;
  const int start = plan.start, in_page = start & ((1 << p.t.page_shift) - 1), kept = start & 15, first = in_page & ~15;
  const int page = p.t.table[(int64_t)s * p.t.table_pages + (start >> p.t.page_shift)];
  const char* in = p.qkv + plan.row * p.row_bytes;
  const RopeLane<D> ln(p.half, p.inv_freq, in_head, p.positions[plan.row]);
  const int tasks = 2 * p.Hkv + (p.q ? (p.Hq + PER - 1) / PER : 0);
  for (int task = wave; task < tasks; task += waves) {
    float x[2][4];
    if (task >= 2 * p.Hkv) {
      const int h = (task - 2 * p.Hkv) * PER + part;
      if (h < p.Hq) {
        load4(in + (int64_t)h * HEAD + ln.o1 * ES, x[0], T{});
        load4(in + (int64_t)h * HEAD + ln.o2 * ES, x[1], T{});
        if (NORM && p.qw != nullptr) {
          float w[2][4];
          load4(p.qw + ln.o1 * ES, w[0], T{}); load4(p.qw + ln.o2 * ES, w[1], T{});
          norm_head<T, D, NORM>(x, w, p.eps);
        }
        ln.template turn<false>(x[0], x[1]);
        char* out = p.q + (plan.row * p.Hq + h) * (D * 2);
        store4<false>(out + ln.o1 * 2, x[0], bf16_t{});
        store4<false>(out + ln.o2 * 2, x[1], bf16_t{});
      }
      continue;
    }
    const bool value = task >= p.Hkv;
    const int h = value ? task - p.Hkv : task;
    const int64_t head = (int64_t)page * p.Hkv + h;
    float* scales = (value ? p.vs : p.ks) + (head << (p.t.page_shift - 4)) + (first >> 4);
    uint8_t* to = (value ? p.v : p.k) + (head << p.t.page_shift) * D;
    const float was = kept ? *scales : 0.f;
    const int o1 = value ? 8 * in_head : ln.o1, o2 = value ? o1 + 4 : ln.o2;
    const char* at = in + (int64_t)(p.Hq + task) * HEAD;              // (every group of lanes has the whole head)
    load4(at + o1 * ES, x[0], T{});
    load4(at + o2 * ES, x[1], T{});
    if (!value) {
      if (NORM && p.kw != nullptr) {
        float w[2][4];
        load4(p.kw + o1 * ES, w[0], T{}); load4(p.kw + o2 * ES, w[1], T{});
        norm_head<T, D, NORM>(x, w, p.eps);
      }
      ln.template turn<false>(x[0], x[1]);
    }
    const float most = group_allreduce_max<LPH>(largest(x));
    const float scale = fmaxf(power_of_two(scale_exponent(most)), was), inv = inverse_of(scale);
    if (lane == 0) *scales = scale;
    if (kept && __builtin_amdgcn_readfirstlane(__float_as_uint(scale)) != __builtin_amdgcn_readfirstlane(__float_as_uint(was))) {
      // the entries that stay: words of four bytes, of the keys one row's, of the values four rows'; stored byte by byte, those of the new
      // row not at all
      const float ratio = was * inv;
      for (int i = lane; i < ((kept + 3) >> 2) * D; i += 64) {
        uint8_t* word = to + first * D + 4 * i;
        const int row = 4 * (i / D) + ((i >> 4) & 3);                  // a key's (words of a group: [d / 64][4][16])
        if (!value && row >= kept) continue;
        float y[4];
        unpack_e4m3(*reinterpret_cast<const uint32_t*>(word), y);
        const uint32_t z = pack_e4m3(y[0] * ratio, y[1] * ratio, y[2] * ratio, y[3] * ratio);
        if (!value) *reinterpret_cast<uint32_t*>(word) = z;
        else
#pragma unroll
          for (int b = 0; b < 4; ++b)
            if (4 * (i / D) + b < kept) word[b] = (uint8_t)(z >> (8 * b));
      }
    }
    const uint32_t a = quantise(x[0], inv), b = quantise(x[1], inv);
    if (!value) {
      if (part == 0) {
        *reinterpret_cast<uint32_t*>(to + key_at<D>(in_page, o1)) = a;
        *reinterpret_cast<uint32_t*>(to + key_at<D>(in_page, o2)) = b;
      }
    } else {
      // eight bytes four apart, dealt to the groups of lanes
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e % PER == part) to[value_at<D>(in_page, o1 + e)] = (uint8_t)((e < 4 ? a : b) >> (8 * (e & 3)));
    }
  }
  __syncthreads();                       // every wave has read the length
  if (threadIdx.x == 0) p.t.len[s] = start + 1;
}

// Workgroups of a block: more where there are few rows, of keys and values as of queries.  (us, 32/8 heads, bf16: keys and values all in
// one workgroup, and shared out)
//   5 x 1-15 rows 18.0, 8.9     64 x 2-8 19.9, 13.1     1 x 2000 28.7, 19.0     256 x 2-4 27.6, 28.0
// 1024, 1536, 2048, 4096 workgroups: 1 x 2000 rows 23.3, 28.0, 28.0, 28.0; 400 x 2-4 43.5, 39.5, 72, 80.
// (Into empty sequences.  Behind 300 to 1500 entries, where most blocks hold some that are read and looked at again: 256 x 2-4 rows 36, 400 x
// 2-4 65.)
constexpr int64_t kAppendGroups = 1024;
void deal_blocks(AppendParams& p, int64_t rows) {
  const int64_t blocks = (rows + kPagedBlock - 1) / kPagedBlock + p.t.B, of_q = p.q ? (p.Hq + 3) / 4 : 0, of_kv = (2 * (int64_t)p.Hkv + 3) / 4;      // (four heads at a time)
  const int64_t want = kAppendGroups / blocks;
  // groups of four as `turns` workgroups share them: groups of each; and how many workgroups then have some
  auto each = [](int64_t of, int64_t turns) { return turns < 2 ? of : turns < of ? (of + turns - 1) / turns : 1; };
  auto having = [](int64_t of, int64_t each) { return of ? (of + each - 1) / each : 0; };
  const int64_t kv = each(of_kv, want * of_kv / (of_kv + of_q));
  p.kv_share = (int32_t)(4 * kv);
  p.kv_turns = (int32_t)having(of_kv, kv);
  const int64_t q = each(of_q, want - p.kv_turns);
  p.q_share = (int32_t)(4 * q);
  p.q_from = want < 2 ? 0 : p.kv_turns;
  p.turns = (uint32_t)(want < 2 ? 1 : p.kv_turns + having(of_q, q));
}
// Packed rows beyond the 256 MB of the Infinity Cache go past it, as in bc_qk_norm_rope.
template <typename T, int D, bool NORM>
void launch_append(AppendParams& p, int64_t rows, hipStream_t s) {
  if (p.t.max_new <= 1) {
    constexpr int PER = 64 / (D / 8);
    const int tasks = 2 * p.Hkv + (p.q ? (p.Hq + PER - 1) / PER : 0);
    paged_append_one_kernel<T, D, NORM><<<p.t.B, 64 * (tasks < 16 ? tasks : 16), 0, s>>>(p);
    return;
  }
  const bool past = rows * (p.Hq + 2 * (int64_t)p.Hkv) * D * Elem<T>::size > (256LL << 20);
  in_launches((int64_t)p.t.B * p.blocks * p.turns, 2 * D, [&](uint32_t base, unsigned groups) {
    p.base = base;
    if (past) paged_append_kernel<T, D, NORM, true><<<groups, 2 * D, 0, s>>>(p);
    else paged_append_kernel<T, D, NORM, false><<<groups, 2 * D, 0, s>>>(p);
  });
}
template <typename T>
void launch_append(AppendParams& p, int64_t rows, int d, hipStream_t s) {
  const bool norm = p.qw || p.kw;
  if (d == 128) { if (norm) launch_append<T, 128, true>(p, rows, s); else launch_append<T, 128, false>(p, rows, s); }
  else { if (norm) launch_append<T, 64, true>(p, rows, s); else launch_append<T, 64, false>(p, rows, s); }
}

}  // namespace
}  // namespace bc

using namespace bc;

extern "C" int32_t bc_paged_append(const bc_shape* shape, const bc_pages* pages, int64_t rows, const int64_t* row_offsets, int32_t max_new,
                                   const void* qkv, int64_t qkv_row_stride, const int32_t* positions, const float* inv_freq, int32_t rot,
                                   const void* q_weight, const void* k_weight, float eps, const int32_t* keep, const uint8_t* active,
                                   void* q, void* stream) {
  const int32_t st = check_pages(shape, pages, rows, row_offsets, max_new);
  if (st != BC_OK) return st;
  if ((int64_t)shape->Hq + 2 * (int64_t)shape->Hkv > 65536 || rot < 0 || rot > shape->d || rot % 8 != 0) return BC_ERR_SHAPE;
  if (!nonnegative_finite(eps)) return BC_ERR_ARG;
  if (rows == 0 || max_new == 0) return BC_OK;
  // (a sequence cannot have more new rows than there are)
  const int64_t most = max_new < rows ? max_new : rows, blocks = (most + 14) / kPagedBlock + 1;
  if (shape->B * blocks > 0x7fffffff) return BC_ERR_SHAPE;
  if (!qkv || !positions || (rot > 0 && !inv_freq) || !aligned16(qkv) || !aligned16(q) || !aligned16(q_weight) || !aligned16(k_weight) || !pages->arrivals) return BC_ERR_ARG;
  if (qkv_row_stride < (int64_t)(shape->Hq + 2 * (int64_t)shape->Hkv) * shape->d || qkv_row_stride > (1LL << 31) ||
      qkv_row_stride * elem_size(shape->kv_dtype) % 16 != 0 || q == qkv)
    return BC_ERR_ARG;
  AppendParams p{};
  p.t = paged_tables(shape, pages, rows, row_offsets, max_new, active);
  p.qkv = static_cast<const char*>(qkv); p.row_bytes = qkv_row_stride * elem_size(shape->kv_dtype);
  p.positions = positions; p.inv_freq = inv_freq; p.half = rot / 2;
  p.qw = static_cast<const char*>(q_weight); p.kw = static_cast<const char*>(k_weight); p.eps = eps;
  p.keep = keep; p.q = static_cast<char*>(q);
  p.k = static_cast<uint8_t*>(pages->k); p.v = static_cast<uint8_t*>(pages->v); p.ks = pages->k_scale; p.vs = pages->v_scale;
  p.Hq = shape->Hq; p.Hkv = shape->Hkv; p.blocks = (uint32_t)blocks; p.arrivals = pages->arrivals;
  deal_blocks(p, rows);
  if (shape->B * blocks * p.turns > 0x7fffffff) return BC_ERR_SHAPE;
  hipStream_t s = as_stream(stream);
  if (shape->kv_dtype == BC_BF16) launch_append<bf16_t>(p, rows, shape->d, s); else launch_append<float>(p, rows, shape->d, s);
  return launch_status();
}
