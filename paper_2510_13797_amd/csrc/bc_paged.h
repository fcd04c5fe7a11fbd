// The cache in pages of 8-bit entries, as its two calls see it (bc_paged_append.hip writes, bc_paged_attend.hip reads).
//
// An entry is a key and a value in e4m3, d bytes each, and a block of 16 entries of a head has one scale, a power of two.  Entries lie in
// groups of four: keys [d / 64][4][64], values [d][4].  So sixteen keys of a head are the first operand of a matrix product as they come
// from memory, 16 bytes a lane and 256 in a row, and a word of values holds the four keys that a lane has weights of: neither goes through
// LDS, and nothing is transposed.
#pragma once
#include "bc_common.h"
#include "bc_paged_grid.h"

namespace bc {

constexpr int kPagedBlock = 16;          // entries that share a scale, and the rows of a matrix operand

// Tables and limits of a call: bc_pages and the rows' arguments.
struct PagedTables {
  const int32_t* table;        // [B, table_pages]
  int32_t* len;                // [B]
  int32_t* err;
  const int64_t* off;          // [B + 1] or null: a row a sequence
  const uint8_t* active;       // [B] or null
  int64_t rows;                // that the call's tensors have
  int32_t B, pages, page_shift, table_pages, max_new;
};

// New rows of a sequence: [row, row + n), and its length.  n = 0: left alone; n < 0: not a span of the call (the caller sets the state bit).
// (All that the tables say is asked for together.)
struct PagedSpan { int64_t row; int n, len; };
__device__ __forceinline__ PagedSpan paged_span(const PagedTables& t, int s) {
  const int64_t a = t.off ? t.off[s] : s, b = t.off ? t.off[s + 1] : s + 1;
  const int len = t.len[s];
  const bool active = t.active ? t.active[s] != 0 : true;
  const bool bad = a < 0 || b < a || b > t.rows || b - a > t.max_new;
  return {a, !active ? 0 : bad ? -1 : (int)(b - a), len};
}

// the four e4m3 values of a word
__device__ __forceinline__ void unpack_e4m3(uint32_t w, float (&x)[4]) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

inline int32_t check_pages(const bc_shape* sh, const bc_pages* pg, int64_t rows, const int64_t* off, int32_t max_new) {
  const int32_t st = check_shape(sh);
  if (st != BC_OK) return st;
  if (!pg || !pg->k || !pg->v || !pg->k_scale || !pg->v_scale || !pg->table || !pg->len || !pg->err) return BC_ERR_ARG;
  if (!aligned16(pg->k) || !aligned16(pg->v)) return BC_ERR_ARG;
  if (pg->pages < 1 || pg->table_pages < 1) return BC_ERR_SHAPE;
  if (pg->page_rows < kPagedBlock || pg->page_rows > 1024 || (pg->page_rows & (pg->page_rows - 1))) return BC_ERR_SHAPE;
  // (blocks and entries are counted in 32 bits)
  if ((int64_t)pg->pages * sh->Hkv * (pg->page_rows / kPagedBlock) > 0x7fffffff || (int64_t)pg->table_pages * pg->page_rows > 0x7fffff00) return BC_ERR_SHAPE;
  if (rows < 0 || rows > 0x7fffffff || max_new < 0 || (int64_t)sh->B * sh->Hkv > (1 << 23)) return BC_ERR_SHAPE;
  if (!off && (rows != sh->B || max_new != 1)) return BC_ERR_ARG;
  return BC_OK;
}

inline PagedTables paged_tables(const bc_shape* sh, const bc_pages* pg, int64_t rows, const int64_t* off, int32_t max_new, const uint8_t* active) {
  PagedTables t{};
  t.table = pg->table; t.len = pg->len; t.err = pg->err; t.off = off; t.active = active; t.rows = rows;
  t.B = sh->B; t.pages = pg->pages; t.table_pages = pg->table_pages; t.max_new = max_new;
  t.page_shift = __builtin_ctz(pg->page_rows);
  return t;
}

}  // namespace bc
