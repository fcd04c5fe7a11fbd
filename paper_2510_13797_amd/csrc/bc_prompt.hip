// bc_prompt_step: a chunk of new prompt rows for every sequence of a cache - their attention over what is resident and over each
// other, and their append (Sec. 2's attention; Alg. 1's "encode the prompt", in pieces or over a cache that has decoded).
//
//   out[i, h] = sum_j softmax_j(scale q[i, h] . K_j) V_j,  j over the L resident rows and new rows 0 .. i
//
// The query heads of a KV head see the same keys, so (row, head) pairs are the columns of the products: column i * g + h, with the
// causal limit by i alone.  Tiles of 32 keys come from two places, first the slab's rows [0, L), then the new rows as the call got
// them (the append need not be over), and go through LDS into 32x32x16 MFMA as in the prefill kernels: S^T = K.Q^T, O^T += V^T.P^T
// with P in two bf16 parts (17 bits: what a decode step over the same rows gives; in fp32 sums) or three, softmax online in registers.
//
// Two kernels share a wave's work on a tile:
//   many columns: a workgroup's four waves have 32 columns each and share the tiles (3-stage ring, a barrier a tile).  Bound by the matrix cores:
//   4 x 2048 rows over 30,000, 32/8 heads, d = 128, 5.25 to 5.5 ms, 4.16 TFLOP of the definition (0.77 PFLOP/s), 6.25 of products issued (1.16; a library
//   product of 16384^3 reaches 1.35).  Weights in three parts would leave 2.4e-7 of an output's error in place of 2.2e-6 to 3.0e-6 (plain fp32: 0.5e-6 to
//   2.1e-6) and take 7.9 ms; 512 rows over 7680, which take 107 us, went from 118 to 163 in an earlier session;
//   32 columns or fewer: all four waves have the same columns and every fourth tile each, in a ring of their own without barriers, and are merged through
//   LDS.  Bound by memory: 7 rows over 16,000, 65 MB, 17.5 us (3.7 TB/s) and 4 for the fold; there the third part costs nothing, and is taken.
// Where that leaves compute units idle the keys are cut into parts, each of which leaves its sums in the workspace (plan_prompt()).
// A second launch folds the parts in order, appends the rows to the slab and moves the tables: the first launch reads them.
#include <vector>

#include "bc_prefill_tiles.h"

namespace bc {
namespace {

// Where the chunks' rows are: in the kernel arguments for up to 128 sequences (a launch that stored them took 4.5 us).
constexpr int kInlineChunks = 128;
struct InlineOffsets {
  int64_t first;
  int32_t from[kInlineChunks + 1];        // less `first`
};

struct PromptParams {
  const char* q;               // [total, Hq, d]
  const char* k;               // [total, Hkv, d]
  const char* v;
  char* k_slab;
  char* v_slab;
  const int64_t* base;
  const int32_t* cap;
  int32_t* cacheP;
  const int32_t* cachec;
  int32_t* nb;
  int32_t* w;
  int32_t* err;
  const uint8_t* active;
  float* out;                  // [total, Hq, d]
  int32_t* resident;           // [B] rows in front of the chunk, -1: the sequence takes no part
  float2* ml;                  // [parts][rows * Hq] maximum (log2) and sum of a part: a sequence's columns behind those of the ones in front
  float* sums;                 // [parts][rows * Hq][d]                                of it, in it a pair's behind the pair's in front of it
  const int64_t* row_off;      // [B + 1], null: `inl`
  int32_t B, Hq, Hkv, g;
  int32_t npairs, pstride, turn, parts;      // as in the prefill kernels
  int64_t first_row, slots;    // the first sequence's first row; columns of a part
  int32_t table_blocks, copy_blocks;      // of the second launch
  float qscale;
  InlineOffsets inl;
};

#define BC_INLINE __attribute__((always_inline))

constexpr float kRedo = 256.f;      // a lane's 16 weights may sum to this before the reference moves
constexpr float kLazy = 2.0f;       // ... and then it moves where a column's maximum is this much (log2) above it
constexpr int kColumns = 32 * kTileWaves;
constexpr int kFewStages = 2;
constexpr int kMostParts = 64;      // a lane each in the fold
constexpr int kFoldGroups = 4;      // of threads that share a column's parts,
constexpr int kFoldAtOnce = 8;      // each asking for eight together
constexpr int kFoldLoads = 16;      // of a thread where there are up to eight parts

struct Chunk { int64_t off0; int rows; };
__device__ __forceinline__ Chunk chunk_of(const PromptParams& p, int s) {        // (p: the kernel's only argument)
  if (p.row_off != nullptr) return {p.row_off[s], (int)(p.row_off[s + 1] - p.row_off[s])};
  typedef __attribute__((address_space(4))) const char const_char_t;
  typedef __attribute__((address_space(4))) const InlineOffsets const_offsets_t;
  const_offsets_t* in = (const_offsets_t*)((const_char_t*)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(PromptParams, inl));
  const int at = in->from[s];
  return {in->first + at, in->from[s + 1] - at};
}

// Where a pair's sums start inside a part's: columns take the room of the rows that there are (a pair's place by the longest chunk's columns took
// gigabytes where one chunk was long and many short).
__device__ __forceinline__ int64_t first_slot(const PromptParams& p, const Chunk& c, int kvh) {
  return (c.off0 - p.first_row) * p.Hq + (int64_t)kvh * c.rows * p.g;
}

// What a sequence's tables say: rows in front of the chunk, or -1 and the error bit to set.
struct Resident { int rows, bit; };
__device__ __forceinline__ Resident resident_rows(const PromptParams& p, int s, int n) {
  if (n <= 0 || (p.active && !p.active[s])) return {-1, 0};
  const int c = p.cachec[s], w = p.w[s], L = p.cacheP[s] + p.nb[s] + w;
  if (c > 0 && w > c) return {-1, BC_ERRBIT_STATE};            // a beacon at the tail that has not been compacted
  if ((int64_t)L + n > p.cap[s]) return {-1, BC_ERRBIT_CAPACITY};
  return {L, 0};
}

// The keys of a workgroup's columns as a list of tiles: the slab's full ones (F), the new rows' that all of the columns see
// (F1: nothing is masked up to here), what is left of the slab, the new rows' others.  (Values that differ between slab and new rows are held
// as one and what is added for the other: chosen between two members of the structure, the compiler kept all of it in memory.)
struct PromptTiles {
  const char* k0;              // slab: the pair's first row
  const char* v0;
  int64_t dk, dv;              // from there to the pair's first new row
  uint32_t row, drow;          // bytes from row to row of the slab, and more from new row to new row
  int L, dL, F, F1, rest;      // rows of the slab; new rows less that; rest: 1 where a part of a tile of the slab is left
  struct At { bool fresh; int row0; };
  __device__ __forceinline__ int dense() const { return F + F1; }
  __device__ __forceinline__ At at(int t) const {
    const int u = t - F - F1;
    const bool left = u >= 0 && u < rest;                     // the slab's last tile
    const bool fresh = t >= F && !left;
    return {fresh, (t - (fresh ? F + (u >= rest ? rest : 0) : left ? F1 : 0)) * kTileRows};
  }
  struct Load { const char* k; const char* v; uint32_t step; int valid; };
  __device__ __forceinline__ Load load(int t) const {
    const At a = at(t);
    const uint32_t step = row + (a.fresh ? drow : 0u);
    const int64_t off = (int64_t)a.row0 * step;
    return {k0 + (a.fresh ? dk : 0) + off, v0 + (a.fresh ? dv : 0) + off, step, L + (a.fresh ? dL : 0) - a.row0};
  }
  // bit x: new row i may see key x of tile t
  __device__ __forceinline__ uint32_t visible(int t, int i) const {
    const At a = at(t);
    const int upto = (a.fresh ? i : L - 1) - a.row0;
    return upto < 0 ? 0u : upto >= 31 ? ~0u : (2u << upto) - 1u;
  }
};

// A wave's 32 columns: accumulators and the running softmax, whose reference m is lazy (it moves only where a lane's weights
// pass kRedo; a column's first visible tile always goes that way, its weights against -1e30 being infinite).
template <int D>
struct Columns {
  static constexpr int KS = D / 16, NJ = D / 32;
  bf16x8_t qb[KS];
  f32x16_t O[NJ];
  float m, l;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < NJ; ++j) O[j] = f32x16_t{0.f};
    m = kNegBig; l = 0.f;
  }
  // One tile (K, then V behind it).  `next` asks for further tiles, behind the scores' products.  The order is written out as in
  // the prefill kernels: operands are asked for several instructions ahead.
  // THIRD: what two parts of a weight leave (below 2^-17 of it) is a third one, half as many products again.
  template <bool MASKED, bool THIRD, typename F>
  __device__ __forceinline__ void tile(const char* tile, int koff, int voff, uint32_t see, float qscale, const F& next) {
    float pe[16], psum;
    auto weights = [&](const f32x16_t& s) BC_INLINE {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        pe[e] = fast_exp2(fmaf(s[e], qscale, -m));
        if constexpr (MASKED) pe[e] = keep_if_visible(pe[e], see, e);
      }
      psum = (((pe[0] + pe[1]) + (pe[2] + pe[3])) + ((pe[4] + pe[5]) + (pe[6] + pe[7]))) +
             (((pe[8] + pe[9]) + (pe[10] + pe[11])) + ((pe[12] + pe[13]) + (pe[14] + pe[15])));
    };
    bf16x8_t r[KS], c[2 * NJ];
    auto col_of = [&](int n) BC_INLINE { return cols_operand<D>(tile + voff, n % NJ, n / NJ); };
#pragma unroll
    for (int i = 0; i < KS; ++i) r[i] = *reinterpret_cast<const bf16x8_t*>(tile + koff + rows_read_imm<D>(i));
    step_fence();
    {
      f32x16_t s = f32x16_t{0.f};
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(r[i], qb[i], s, 0, 0, 0);
        if (i >= KS - NJ) c[i - KS + NJ] = col_of(i - KS + NJ);
        step_fence();
      }
      next();
      weights(s);
    }
    if (__builtin_expect(__any(psum > kRedo), 0)) {
      f32x16_t s = f32x16_t{0.f};
      const char* ka = tile + opaque(koff);                  // (reads the operands again)
#pragma unroll
      for (int i = 0; i < KS; ++i)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8_t*>(ka + rows_read_imm<D>(i)), qb[i], s, 0, 0, 0);
      float tmax = kNegBig;
#pragma unroll
      for (int e = 0; e < 16; ++e) tmax = fmaxf(tmax, !MASKED || visible_bit(see, e) ? s[e] : kNegBig);
      const float cand = halves_max(tmax) * qscale;
      const float to = cand > m + kLazy ? cand : m;
      const float alpha = fast_exp2(m - to);
      m = to;
      l *= alpha;
#pragma unroll
      for (int j = 0; j < NJ; ++j) O[j] *= alpha;
      weights(s);
    }
    l += psum;
    Parts y;
#pragma unroll
    for (int g = 0; g < 4; ++g) y.split(g, pe[2 * g], pe[2 * g + 1]);
    step_fence();
#pragma unroll
    for (int k = 0; k < 4 * NJ; ++k) {
      const int n = k / 2;
      O[n % NJ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[n], y.operand(k & 1, n / NJ), O[n % NJ], 0, 0, 0);
      if (!THIRD && k % 2 == 0 && n + NJ < 2 * NJ) c[n + NJ] = col_of(n + NJ);
      if (THIRD && k % 2 == 0 && n < NJ) c[n + NJ] = col_of(n + NJ);
#pragma unroll
      for (int g = 4; g < 8; ++g)
        if (k == (g - 4) * NJ / 2) y.split(g, pe[2 * g], pe[2 * g + 1]);
      step_fence();
    }
    if constexpr (THIRD) {
      uint32_t rest[8];
#pragma unroll
      for (int g = 0; g < 8; ++g)
        rest[g] = pack2_bf16(pe[2 * g] - __uint_as_float(y.h[g] << 16) - __uint_as_float(y.l[g] << 16),
                             pe[2 * g + 1] - __uint_as_float(y.h[g] & 0xffff0000u) - __uint_as_float(y.l[g] & 0xffff0000u));
#pragma unroll
      for (int n = 0; n < 2 * NJ; ++n) {
        const uint32_t* r = rest + 4 * (n / NJ);
        O[n % NJ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[n], __builtin_bit_cast(bf16x8_t, make_uint4(r[0], r[1], r[2], r[3])), O[n % NJ], 0, 0, 0);
      }
    }
  }
};

// A wave's 32 query columns from column `first` on (the last one repeated behind it) -> a tile of its own in LDS.
template <int D>
__device__ __forceinline__ void issue_columns(const PromptParams& p, int64_t off0, int kvh, int first, int columns, int lane,
                                              uint32_t lds_addr) {
  constexpr int ROWB = D * 2;
  const int i0 = min(first, columns - 1) / p.g;
  const char* at = p.q + ((off0 + i0) * p.Hq + kvh * p.g) * ROWB;
#pragma unroll
  for (int rg = 0; rg < kTileRows / 8; ++rg) {
    const TileLane t = rows_tile_lane(lane, rg);
    const int x = min(first + t.row, columns - 1), i = x / p.g;
    const uint32_t o = (uint32_t)((i - i0) * p.Hq + x - i * p.g) * ROWB + t.in_row;
#pragma unroll
    for (int n = 0; n < D / 64; ++n) issue_block<false>(at + 128 * n, o, lds_addr + n * 4096 + rg * 1024);
  }
}

// The workgroup's place and its sequence; false: nothing to do.
struct PromptWork {
  int part, pair, kvh, s, n, columns, first;
  int64_t off0, slot0;
  PromptTiles tiles;
  int t0, t1;                  // tiles of this part
  template <int D, int WIDE>
  __device__ __forceinline__ bool start(const PromptParams& p) {
    constexpr int ROWB = D * 2;
    part = blockIdx.x / p.pstride;
    pair = pair_in_turn(blockIdx.x - part * p.pstride, p.pstride, p.turn, blockIdx.y * p.parts + part);
    if (pair >= p.npairs) return false;
    kvh = pair % p.Hkv;
    s = pair / p.Hkv;
    const Chunk chunk = chunk_of(p, s);
    off0 = chunk.off0;
    n = chunk.rows;
    slot0 = part * p.slots + first_slot(p, chunk, kvh);
    const int block = gridDim.y - 1 - blockIdx.y;              // long ones first
    const Resident r = resident_rows(p, s, n);
    if (block == 0 && part == 0 && kvh == 0 && threadIdx.x == 0) {
      p.resident[s] = r.rows;
      if (r.bit) atomicOr(p.err, r.bit);
    }
    columns = n * p.g;
    first = block * WIDE;
    if (r.rows < 0 || first >= columns) return false;
    const int cap = p.cap[s];
    const int64_t slab = (p.base[s] * p.Hkv + (int64_t)kvh * cap) * ROWB, fresh = (off0 * p.Hkv + kvh) * ROWB;
    tiles.L = r.rows; tiles.dL = n - r.rows;
    tiles.F = r.rows / kTileRows;
    tiles.rest = r.rows % kTileRows ? 1 : 0;
    tiles.F1 = (first / p.g + 1) / kTileRows;
    tiles.k0 = p.k_slab + slab; tiles.v0 = p.v_slab + slab;
    tiles.row = ROWB; tiles.drow = (uint32_t)(p.Hkv - 1) * ROWB;
    tiles.dk = p.k + fresh - tiles.k0; tiles.dv = p.v + fresh - tiles.v0;
    const int last = (min(first + WIDE, columns) - 1) / p.g;                     // row of the last column
    const int NT = tiles.F + tiles.rest + last / kTileRows + 1;
    t0 = (int)((int64_t)NT * part / p.parts);
    t1 = (int)((int64_t)NT * (part + 1) / p.parts);
    return true;
  }
  // where a column's sums of this part go
  __device__ __forceinline__ int64_t slot(int column) const { return slot0 + column; }
};

template <int D> constexpr int prompt_lds() { return kTileStages * 2 * kTileRows * D * 2; }

// 128 columns: 32 a wave, tiles shared.
template <int D>
__global__ __launch_bounds__(kTileWaves * 64, 3) void prompt_attn_kernel(PromptParams p) {
  constexpr int ROWB = D * 2, TILE = kTileRows * ROWB, NLD = TILE / 1024 / kTileWaves, OW = D / 2;
  __shared__ __attribute__((aligned(1024))) char lds[prompt_lds<D>()];
  static_assert(prompt_lds<D>() >= kTileWaves * 32 * OW * 4 && prompt_lds<D>() >= (2 + kTileWaves) * TILE, "LDS");
  PromptWork wk;
  if (!wk.start<D, kColumns>(p)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int first = wk.first + 32 * wave;
  const int i = min(first + col, wk.columns - 1) / p.g;                                   // new row of this lane's column
  const int i_last = (min(first + 32, wk.columns) - 1) / p.g;
  // tiles this wave works on; the others it loads and passes with the workgroup
  const int mine = first < wk.columns ? min(wk.t1, wk.tiles.F + wk.tiles.rest + i_last / kTileRows + 1) : 0;
  const PromptTiles& tiles = wk.tiles;

  const uint32_t lds0 = lds_address(lds) + wave * 1024;
  const TileLane klane = rows_tile_lane(lane, wave), vlane = cols_tile_lane(lane, wave);
  auto issue_tile = [&](int t, int stage) BC_INLINE {
    const PromptTiles::Load ld = tiles.load(t);
    const uint32_t ko = (uint32_t)(klane.row < ld.valid ? klane.row : 0) * ld.step + klane.in_row;
    const uint32_t vo = (uint32_t)(vlane.row < ld.valid ? vlane.row : 0) * ld.step + vlane.in_row;
#pragma unroll
    for (int n = 0; n < NLD; ++n) {
      issue_block<false>(ld.k + 128 * n, ko, lds0 + stage * (2 * TILE) + n * 4096);
      issue_block<false>(ld.v + 128 * n, vo, lds0 + stage * (2 * TILE) + TILE + n * 4096);
    }
  };
  Columns<D> x;
  x.clear();
  if (wk.t0 < wk.t1) {
    issue_tile(wk.t0, 0);
    issue_columns<D>(p, wk.off0, wk.kvh, first, wk.columns, lane, lds_address(lds) + (2 + wave) * TILE);
    wait_vmcnt<0>();
    read_wave_rows<D>(lds + (2 + wave) * TILE, lane, x.qb);
    landed_operands(x.qb);
    lds_barrier();
    if (wk.t0 + 1 < wk.t1) issue_tile(wk.t0 + 1, 1);
  }
  const int koff = rows_read_offset(lane), voff = TILE + cols_read_offset(lane);
  int stage = 0, t = wk.t0;
  // tile t has landed and everyone has finished t - 1, whose stage t + 2 goes into
  auto begin_pass = [&]() BC_INLINE {
    if (t + 1 < wk.t1) wait_vmcnt<2 * NLD>();
    else wait_vmcnt<0>();
    lds_barrier();
  };
  auto next = [&]() BC_INLINE { if (t + 2 < wk.t1) issue_tile(t + 2, stage >= 1 ? stage - 1 : kTileStages - 1); };
  auto end_pass = [&]() BC_INLINE { stage = stage + 1 == kTileStages ? 0 : stage + 1; };
  for (const int dense = min(tiles.dense(), mine); t < dense; ++t) {
    begin_pass();
    x.template tile<false, false>(lds + stage * (2 * TILE), koff, voff, ~0u, p.qscale, next);
    end_pass();
  }
  for (; t < mine; ++t) {
    begin_pass();
    x.template tile<true, false>(lds + stage * (2 * TILE), koff, voff, tiles.visible(t, i) >> (4 * half), p.qscale, next);
    end_pass();
  }
  for (; t < wk.t1; ++t) {
    begin_pass();
    next();
    end_pass();
  }
  lds_barrier();          // the stages are free: the results go through them
  if (first >= wk.columns) return;
  const float l = halves_sum(x.l);
  float* my = reinterpret_cast<float*>(lds + wave * (32 * OW * 4));
  const int left = wk.columns - first;
  if (p.parts == 1) {
    const float inv = 1.0f / l;
    float* out = p.out + (wk.off0 * p.Hq + wk.kvh * p.g) * D;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass)
      store_rows<D>(my, x.O, inv, pass, lane, out, D, [&](int t) {
        const int c = first + t, r = c / p.g;
        return t < left ? r * p.Hq + c - r * p.g : -1;
      });
  } else {
    if (half == 0 && col < left) p.ml[wk.slot(first + col)] = make_float2(x.m, l);
    if (wk.t0 >= wk.t1) return;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass)
      store_rows<D, false>(my, x.O, 1.f, pass, lane, p.sums + wk.slot(first) * D, D, [&](int t) { return t < left ? t : -1; });
  }
}

template <int D> constexpr int prompt_few_lds() { return kTileWaves * kFewStages * 2 * kTileRows * D * 2; }

// 32 columns: the same for every wave, which has every fourth tile.
template <int D>
__global__ __launch_bounds__(kTileWaves * 64, 1) void prompt_few_kernel(PromptParams p) {
  constexpr int ROWB = D * 2, TILE = kTileRows * ROWB, RG = kTileRows / 8, NLD = 2 * RG * (D / 64), MINE = kFewStages * 2 * TILE;
  __shared__ __attribute__((aligned(1024))) char lds[prompt_few_lds<D>()];
  __shared__ float2 wave_ml[kTileWaves][32];
  PromptWork wk;
  if (!wk.start<D, 32>(p)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int i = min(col, wk.columns - 1) / p.g;
  const PromptTiles& tiles = wk.tiles;
  char* own = lds + wave * MINE;
  const uint32_t own_at = lds_address(lds) + wave * MINE;
  auto issue_tile = [&](int t, int stage) BC_INLINE {
    const PromptTiles::Load ld = tiles.load(t);
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
      const TileLane kl = rows_tile_lane(lane, rg), vl = cols_tile_lane(lane, rg);
      const uint32_t ko = (uint32_t)(kl.row < ld.valid ? kl.row : 0) * ld.step + kl.in_row;
      const uint32_t vo = (uint32_t)(vl.row < ld.valid ? vl.row : 0) * ld.step + vl.in_row;
#pragma unroll
      for (int n = 0; n < D / 64; ++n) {
        // (read once: out of the way of the caches)
        lds_dma16_s<true>(ko, (uint64_t)(ld.k + 128 * n), own_at + stage * (2 * TILE) + n * 4096 + rg * 1024);
        lds_dma16_s<true>(vo, (uint64_t)(ld.v + 128 * n), own_at + stage * (2 * TILE) + TILE + n * 4096 + rg * 1024);
      }
    }
  };
  Columns<D> x;
  x.clear();
  const int first = wk.t0 + wave;
  if (first < wk.t1) {
    issue_tile(first, 0);
    issue_columns<D>(p, wk.off0, wk.kvh, 0, wk.columns, lane, own_at + 2 * TILE);
    wait_vmcnt<0>();
    read_wave_rows<D>(own + 2 * TILE, lane, x.qb);
    landed_operands(x.qb);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (first + kTileWaves < wk.t1) issue_tile(first + kTileWaves, 1);
  }
  const int koff = rows_read_offset(lane), voff = TILE + cols_read_offset(lane);
  int stage = 0;
  for (int t = first; t < wk.t1; t += kTileWaves) {
    if (t + kTileWaves < wk.t1) wait_vmcnt<NLD>();
    else wait_vmcnt<0>();
    const char* at = own + stage * (2 * TILE);
    auto nothing = [] {};
    if (t < tiles.dense())
      x.template tile<false, true>(at, koff, voff, ~0u, p.qscale, nothing);
    else
      x.template tile<true, true>(at, koff, voff, tiles.visible(t, i) >> (4 * half), p.qscale, nothing);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // the stage has been read
    if (t + 2 * kTileWaves < wk.t1) issue_tile(t + 2 * kTileWaves, stage);
    stage ^= 1;
  }
  // merge: every wave's sums at the start of its own stages
  constexpr int UNITS = D / 4;
  const float l = halves_sum(x.l);
  float* mine = reinterpret_cast<float*>(own);
#pragma unroll
  for (int j = 0; j < D / 32; ++j)
#pragma unroll
    for (int u = 0; u < 4; ++u)
      *reinterpret_cast<f32x4_t*>(mine + col * D + (((8 * j + 2 * u + half) ^ (col & (UNITS - 1))) << 2)) =
          f32x4_t{x.O[j][4 * u], x.O[j][4 * u + 1], x.O[j][4 * u + 2], x.O[j][4 * u + 3]};
  if (half == 0) wave_ml[wave][col] = make_float2(x.m, l);
  __syncthreads();
  for (int at = threadIdx.x; at < 32 * UNITS; at += kTileWaves * 64) {
    const int c = at / UNITS, unit = at % UNITS;
    if (c >= wk.columns) break;
    float M = kNegBig, sum = 0.f;
#pragma unroll
    for (int wv = 0; wv < kTileWaves; ++wv) M = fmaxf(M, wave_ml[wv][c].x);
    f32x4_t o = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int wv = 0; wv < kTileWaves; ++wv) {
      const float f = fast_exp2(wave_ml[wv][c].x - M);
      sum += wave_ml[wv][c].y * f;
      o += *reinterpret_cast<const f32x4_t*>(reinterpret_cast<const float*>(lds + wv * MINE) + c * D + ((unit ^ (c & (UNITS - 1))) << 2)) * f;
    }
    if (p.parts == 1) {
      const int r = c / p.g;
      float* to = p.out + ((wk.off0 + r) * p.Hq + wk.kvh * p.g + c - r * p.g) * D;
      *reinterpret_cast<f32x4_t*>(to + 4 * unit) = o * (1.0f / sum);
    } else {
      const int64_t slot = wk.slot(c);
      if (unit == 0) p.ml[slot] = make_float2(M, sum);
      if (wk.t0 < wk.t1) *reinterpret_cast<f32x4_t*>(p.sums + slot * D + 4 * unit) = o;
    }
  }
}

// Weights of a column's parts from their maxima and sums, a lane each.
struct PartWeight { float f, inv; };
template <int LANES>
__device__ __forceinline__ PartWeight part_weight(float2 ml) {
  float M = ml.x;
#pragma unroll
  for (int o = LANES / 2; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  const float f = ml.y > 0.f ? fast_exp2(ml.x - M) : 0.f;         // (0: the part had no tiles and left no sums)
  float sum = ml.y * f;
#pragma unroll
  for (int o = LANES / 2; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
  return {f, 1.0f / sum};
}

// Many parts of few columns: four groups of threads share a column's parts, eight loads of each together (one column's parts one after the other by
// 32 threads: 7 rows over 16,000, 32 parts, 26 us; 4 so).
template <int D>
__device__ __forceinline__ void fold_many_parts(const PromptParams& p, int block) {
  constexpr int UNITS = D / 4, COLS = 256 / UNITS / kFoldGroups;
  const int pair = block % p.npairs, s = pair / p.Hkv;
  if (p.resident[s] < 0) return;
  const Chunk chunk = chunk_of(p, s);
  const int columns = chunk.rows * p.g, first = block / p.npairs * COLS;
  if (first >= columns) return;
  __shared__ float weight[COLS][kMostParts];
  __shared__ float inv[COLS];
  __shared__ f32x4_t some[kFoldGroups][COLS * UNITS];
  const int64_t slot0 = first_slot(p, chunk, pair % p.Hkv) + first, step = p.slots;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (wave < COLS) {
    const int64_t slot = slot0 + min(wave, columns - 1 - first);
    const PartWeight w = part_weight<64>(lane < p.parts ? p.ml[slot + lane * step] : make_float2(kNegBig, 0.f));
    weight[wave][lane] = w.f;
    if (lane == 0) inv[wave] = w.inv;
  }
  __syncthreads();
  const int group = threadIdx.x / (COLS * UNITS), at = threadIdx.x % (COLS * UNITS), c = at / UNITS, unit = at % UNITS;
  const float* sums = p.sums + (slot0 + min(c, columns - 1 - first)) * D + 4 * unit;
  f32x4_t o = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int n0 = group; n0 < p.parts; n0 += kFoldGroups * kFoldAtOnce) {
    f32x4_t x[kFoldAtOnce];
#pragma unroll
    for (int e = 0; e < kFoldAtOnce; ++e) {
      const int n = n0 + e * kFoldGroups;
      if (n < p.parts) x[e] = *reinterpret_cast<const f32x4_t*>(sums + n * step * D);
    }
#pragma unroll
    for (int e = 0; e < kFoldAtOnce; ++e) {
      const int n = n0 + e * kFoldGroups;
      const float f = n < p.parts ? weight[c][n] : 0.f;
      if (f > 0.f) o += x[e] * f;
    }
  }
  some[group][at] = o;
  __syncthreads();
  if (group != 0 || first + c >= columns) return;
#pragma unroll
  for (int n = 1; n < kFoldGroups; ++n) o += some[n][at];
  const int col = first + c, r = col / p.g;
  float* to = p.out + ((chunk.off0 + r) * p.Hq + pair % p.Hkv * p.g + col - r * p.g) * D;
  *reinterpret_cast<f32x4_t*>(to + 4 * unit) = o * inv[c];
}

// Up to eight parts of many columns: D / 4 threads a column, each with kFoldLoads loads on their way (PARTS for each of several
// columns; one column and two loads a thread: 4 x 2048 rows of 32 heads in two parts 252 us, 88 with eight loads), columns by their place in the
// output.  Sequence s has the workgroups from fold_start(s) on, at least
// as many as its columns take, so that there are next to none for rows that shorter chunks do not have.  (The sequence is found for the
// workgroup, by scalar loads: by every thread for its own column, its chunk came from the kernel's arguments by vector loads.)
template <int D, int PARTS> constexpr int fold_columns() { return 256 / (D / 4) * (kFoldLoads / PARTS); }
template <int PER>
__host__ __device__ __forceinline__ int64_t fold_start(int64_t rows, int s, int Hq) { return rows * Hq / PER + s; }
template <int D, int PARTS>
__device__ __forceinline__ void fold_few_parts(const PromptParams& p, int block) {
  constexpr int UNITS = D / 4, PER = fold_columns<D, PARTS>(), COLS = kFoldLoads / PARTS, APART = 256 / UNITS;
  const int64_t off = chunk_of(p, 0).off0;
  int s = 0, end = p.B;
  while (end - s > 1) {
    const int mid = (s + end) >> 1;
    if (fold_start<PER>(chunk_of(p, mid).off0 - off, mid, p.Hq) <= block) s = mid; else end = mid;
  }
  if (p.resident[s] < 0) return;
  const Chunk chunk = chunk_of(p, s);
  const int first = (int)(block - fold_start<PER>(chunk.off0 - off, s, p.Hq)) * PER + threadIdx.x / UNITS, unit = threadIdx.x % UNITS;
  const int last = chunk.rows * p.Hq - 1;
  const int64_t step = p.slots;
  int64_t slot[COLS];
  f32x4_t x[COLS][PARTS];
  float2 ml[COLS];
  const int lane = threadIdx.x & (PARTS - 1);
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    const int at = min(first + c * APART, last), i = at / p.Hq, head = at - i * p.Hq, kvh = head / p.g;
    slot[c] = first_slot(p, chunk, kvh) + i * p.g + head - kvh * p.g;
    ml[c] = lane < p.parts ? p.ml[slot[c] + lane * step] : make_float2(kNegBig, 0.f);
#pragma unroll
    for (int n = 0; n < PARTS; ++n)
      if (n < p.parts) x[c][n] = *reinterpret_cast<const f32x4_t*>(p.sums + (slot[c] + n * step) * D + 4 * unit);
  }
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    const PartWeight w = part_weight<PARTS>(ml[c]);
    f32x4_t o = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < PARTS; ++n) {
      const float f = __shfl(w.f, (threadIdx.x & (64 - PARTS)) + n, 64);
      if (n < p.parts && f > 0.f) o += x[c][n] * f;
    }
    const int at = first + c * APART;
    if (at <= last) __builtin_nontemporal_store(o * w.inv, reinterpret_cast<f32x4_t*>(p.out + (chunk.off0 * p.Hq + at) * D + 4 * unit));
  }
}

// The second launch: tables, append, and the fold of the parts.  What the first one decided is in p.resident.
// PARTS: at most, 0: more.
template <int D, int PARTS>
__global__ __launch_bounds__(256) void prompt_finish_kernel(PromptParams p) {
  constexpr int ROWB = D * 2, RU = ROWB / 16;
  int block = blockIdx.x;
  if (block < p.table_blocks) {
    const int s = block * 256 + threadIdx.x;
    if (s < p.B && p.resident[s] >= 0) {
      const Chunk chunk = chunk_of(p, s);
      p.cacheP[s] = p.resident[s] + chunk.rows;
      p.nb[s] = 0;
      p.w[s] = 0;
    }
    return;
  }
  block -= p.table_blocks;
  if (block < p.copy_blocks * p.B) {
    const int s = block / p.copy_blocks, slice = block - s * p.copy_blocks, L = p.resident[s];
    if (L < 0) return;
    const Chunk chunk = chunk_of(p, s);
    const int cap = p.cap[s];
    const int64_t slab = p.base[s] * p.Hkv, units = (int64_t)chunk.rows * p.Hkv * RU;
    for (int64_t u = (int64_t)slice * 256 + threadIdx.x; u < units; u += (int64_t)p.copy_blocks * 256) {
      const int64_t row = u / RU;                               // (new row, KV head)
      const int i = (int)(row / p.Hkv), h = (int)(row - (int64_t)i * p.Hkv), at = (int)(u - row * RU);
      const int64_t from = (chunk.off0 * p.Hkv + row) * ROWB + 16 * at, to = (slab + (int64_t)h * cap + L + i) * ROWB + 16 * at;
      *reinterpret_cast<uint4*>(p.k_slab + to) = *reinterpret_cast<const uint4*>(p.k + from);
      *reinterpret_cast<uint4*>(p.v_slab + to) = *reinterpret_cast<const uint4*>(p.v + from);
    }
    return;
  }
  block -= p.copy_blocks * p.B;
  if constexpr (PARTS == 0) fold_many_parts<D>(p, block);
  else fold_few_parts<D, PARTS>(p, block);
}

// How a call is cut.  Lengths of the caches are on the device; the capacity stands for them.  Many columns: as many workgroups as run at once (three
// a compute unit), half as many again for several sequences, whose lengths differ, in parts of 16 tiles and more; 32 columns: one a
// compute unit (its LDS), four tiles and more.  One, two, three, four, six, eight parts in us, with the rule's in brackets:
//   (one earlier session; the first line's six parts now take 107)
//   512 rows over 7680, 32/8 heads      242 151 141 124 [120] 127
//   700 over 3000, 12/2                 112  67  55  55 [46] 47
//   8 x 64 over 2000, 32/8               74  52  52 [49] 51  61
//   8 x 10-200 over 100-6000, 32/8      219 132 129 [123] 123 129
//   64 x 5-120 over 0-3000, 12/2        145 [129] 124 125 141 159
//   128 x 10-100 over 0-2000, 4/1        92  74 [67] 69  75  82
struct PromptPlan {
  bool few;
  int blocks;                  // workgroups along a pair's columns
  int parts;
  int64_t columns;             // of a pair, at most
  size_t bytes, ml_at, sums_at, tables_at;
};
// What the kernels and their grids hold: offsets inside a tile of 32 rows and a sequence's (row, head) pairs are of 32 bits, and so are the threads of a
// grid's row; its rows are 65535 blocks of columns at most.
bool prompt_fits(const bc_shape* sh, int64_t max_new, int64_t total) {
  if (sh->kv_dtype != BC_BF16 || sh->Hq > 65536 || (int64_t)sh->B * sh->Hkv > (1 << 23)) return false;
  if (max_new >= (1LL << 31) || max_new * sh->Hq >= (1LL << 31) || total >= (1LL << 31)) return false;
  return max_new * (sh->Hq / sh->Hkv) <= 65535LL * kColumns;
}
PromptPlan plan_prompt(const bc_shape* sh, int64_t max_new, int64_t total, int32_t max_cap) {
  const int64_t g = sh->Hq / sh->Hkv, npairs = (int64_t)sh->B * sh->Hkv;
  PromptPlan pl;
  pl.few = max_new * g <= 32;
  const int64_t wide = pl.few ? 32 : kColumns;
  pl.blocks = (int)((max_new * g + wide - 1) / wide);
  if (pl.blocks < 1) pl.blocks = 1;
  pl.columns = pl.blocks * wide;
  // workgroups there will be about, and as many as run at once
  const int64_t all = (total * g / wide + sh->B) * sh->Hkv, most = npairs * pl.blocks, work = all < most ? all : most;
  const int64_t room = pl.few ? 256 : sh->B > 1 ? 1152 : 768, tiles = (max_cap + kTileRows - 1) / kTileRows;
  int64_t parts = work > 0 ? room / work : 1;
  const int64_t enough = tiles / (pl.few ? 4 : 16);
  if (parts > enough) parts = enough;
  pl.parts = (int)(parts < 1 ? 1 : parts > kMostParts ? kMostParts : parts);
  size_t at = ((size_t)sh->B * 4 + 15) & ~(size_t)15;
  pl.tables_at = at;
  if (sh->B > kInlineChunks) at += ((size_t)sh->B * 16 + 8 + 15) & ~(size_t)15;
  pl.ml_at = at;
  const size_t slots = pl.parts > 1 ? (size_t)pl.parts * total * sh->Hq : 0;
  at += (slots * sizeof(float2) + 15) & ~(size_t)15;
  pl.sums_at = at;
  at += slots * sh->d * sizeof(float);
  pl.bytes = at;
  return pl;
}

template <int D, int PARTS>
void launch_finish(const PromptParams& p, const PromptPlan& pl, int64_t total, hipStream_t s) {
  constexpr int PER = 256 / (D / 4) / kFoldGroups;
  int64_t fold = 0;
  if constexpr (PARTS == 0) fold = p.npairs * ((pl.columns + PER - 1) / PER);
  else if (p.parts > 1) fold = fold_start<fold_columns<D, PARTS>()>(total, p.B, p.Hq);
  prompt_finish_kernel<D, PARTS><<<(unsigned)(p.table_blocks + (int64_t)p.copy_blocks * p.B + fold), 256, 0, s>>>(p);
}
template <int D>
int32_t launch_prompt(const PromptParams& p, const PromptPlan& pl, int64_t total, hipStream_t s) {
  const dim3 grid(p.pstride * p.parts, pl.blocks);
  if (pl.few) prompt_few_kernel<D><<<grid, kTileWaves * 64, 0, s>>>(p);
  else prompt_attn_kernel<D><<<grid, kTileWaves * 64, 0, s>>>(p);
  const int32_t st = launch_status();       // (the second launch goes by what the first one leaves)
  if (st != BC_OK) return st;
  if (p.parts <= 2) launch_finish<D, 2>(p, pl, total, s);
  else if (p.parts <= 4) launch_finish<D, 4>(p, pl, total, s);
  else if (p.parts <= 8) launch_finish<D, 8>(p, pl, total, s);
  else launch_finish<D, 0>(p, pl, total, s);
  return launch_status();
}

}  // namespace
}  // namespace bc

using namespace bc;

extern "C" size_t bc_prompt_workspace_bytes(const bc_shape* shape, int32_t max_new, int64_t total_new, int32_t max_cap) {
  if (check_shape(shape) != BC_OK || max_new < 0 || total_new < 0 || max_cap < 1 || !prompt_fits(shape, max_new, total_new)) return 0;
  return plan_prompt(shape, max_new, total_new, max_cap).bytes;
}

extern "C" int32_t bc_prompt_step(const bc_shape* shape, const bc_cache* cache, const void* k, const void* v, const void* q,
                                  const int64_t* row_offsets, float* out, const uint8_t* active, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  int32_t st = check_shape(shape);
  if (st != BC_OK) return st;
  if (shape->kv_dtype != BC_BF16) return BC_ERR_SHAPE;
  st = check_cache(cache);
  if (st != BC_OK) return st;
  if (!row_offsets || !positive_finite(shape->scale)) return BC_ERR_ARG;
  int64_t max_new = 0;
  if (row_offsets[0] < 0) return BC_ERR_ARG;
  for (int b = 0; b < shape->B; ++b) {
    const int64_t n = row_offsets[b + 1] - row_offsets[b];
    if (n < 0) return BC_ERR_ARG;
    if (n > max_new) max_new = n;
  }
  const int64_t total = row_offsets[shape->B] - row_offsets[0];
  if (total == 0) return BC_OK;
  if (!k || !v || !q || !out || !aligned16(k) || !aligned16(v) || !aligned16(q) || !aligned16(out)) return BC_ERR_ARG;
  if (!prompt_fits(shape, max_new, total)) return BC_ERR_SHAPE;
  const PromptPlan pl = plan_prompt(shape, max_new, total, cache->max_cap);
  if (!workspace || !aligned16(workspace) || workspace_bytes < pl.bytes) return BC_ERR_WORKSPACE;
  PromptParams p{};
  char* ws = static_cast<char*>(workspace);
  if (shape->B <= kInlineChunks) {
    p.inl.first = row_offsets[0];
    for (int b = 0; b <= shape->B; ++b) p.inl.from[b] = (int32_t)(row_offsets[b] - row_offsets[0]);
  } else {                                                     // (offsets, and in place of the other tables zeros)
    std::vector<int64_t> words;
    try {
      words.assign((size_t)2 * shape->B + 1, 0);
    } catch (...) {
      return BC_ERR_WORKSPACE;
    }
    for (int b = 0; b <= shape->B; ++b) words[b] = row_offsets[b];
    const int32_t* none = reinterpret_cast<const int32_t*>(words.data() + shape->B + 1);
    st = bc_trajectory_tables(words.data(), none, none + shape->B, shape->B, ws + pl.tables_at, stream);
    if (st != BC_OK) return st;
    p.row_off = reinterpret_cast<const int64_t*>(ws + pl.tables_at);
  }
  p.q = static_cast<const char*>(q); p.k = static_cast<const char*>(k); p.v = static_cast<const char*>(v);
  p.k_slab = static_cast<char*>(cache->k_slab); p.v_slab = static_cast<char*>(cache->v_slab);
  p.base = cache->base; p.cap = cache->cap; p.cacheP = cache->P; p.cachec = cache->c;
  p.nb = cache->nb; p.w = cache->w; p.err = cache->err;
  p.active = active; p.out = out;
  p.resident = reinterpret_cast<int32_t*>(ws);
  p.ml = reinterpret_cast<float2*>(ws + pl.ml_at);
  p.sums = reinterpret_cast<float*>(ws + pl.sums_at);
  p.B = shape->B; p.Hq = shape->Hq; p.Hkv = shape->Hkv; p.g = shape->Hq / shape->Hkv;
  p.npairs = shape->B * shape->Hkv;
  // All of a pair's workgroups on one XCD, as in the prefill kernels - but where the heads of a sequence do not take all XCDs alike, pairs of long and
  // short sequences would weigh on some XCDs more than on others: there a pair moves on by one XCD from row to row of the grid.  (24 sequences of
  // up to 300 rows over up to 3500, 12/2 heads: 102 us so, 123 on one XCD; 64 of up to 120 over 3000, 124 and 138; 32/8 heads, 8 sequences of up to 200
  // over 6000, 131 and 123; 16 fresh ones of up to 1500, 248 and 220.)
  const bool roam = shape->B > 1 && shape->Hkv % 8 != 0;
  p.pstride = roam ? p.npairs | 1 : pair_stride(p.npairs);
  p.turn = roam ? 0 : pair_turn(p.pstride);
  p.parts = pl.parts;
  p.first_row = row_offsets[0];
  p.slots = total * shape->Hq;
  p.table_blocks = (shape->B + 255) / 256;
  const int64_t units = max_new * shape->Hkv * (shape->d / 8);
  const int64_t copies = (units + 1023) / 1024, share = 4096 / shape->B + 1;
  p.copy_blocks = (int32_t)(copies < share ? copies : share);
  p.qscale = shape->scale * kLog2e;
  hipStream_t s = as_stream(stream);
  return shape->d == 128 ? launch_prompt<128>(p, pl, total, s) : launch_prompt<64>(p, pl, total, s);
}
