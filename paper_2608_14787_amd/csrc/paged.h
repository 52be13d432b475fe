// Paged KV cache: device descriptor and stored order, shared by the operators on it (internal to libsdd).
#pragma once

#include "model.h"

namespace sdd {

// Division by a number known on the host: the kernels' indices come apart by a few of them before the first load, and a
// division is some twenty instructions here.  n / d = n m >> (31 + s) for 0 <= n < 2^31, with s = ceil(log2 d) and m =
// ceil(2^(31 + s) / d) < 2^32 (the rounding of m moves the quotient by less than n / 2^(31 + s) < 1 / d).
struct FastDiv {
  uint32_t d, m, s;
  FastDiv() : d(1), m(1u << 31), s(0) {}
  explicit FastDiv(uint32_t by) : d(by), s(0) {
    while ((1u << s) < by) ++s;
    m = (uint32_t)((((uint64_t)1 << (31 + s)) + by - 1) / by);
  }
  __host__ __device__ inline int div(int n) const { return (int)((uint64_t)(uint32_t)n * m >> (31 + s)); }
};

// Sticky bits of the operators' error word (those of sdd_kv_state).
constexpr int kErrCapacity = 1, kErrId = 4;

// A pool of pages as the kernels see it.  The bytes of head h of page p start at (p * hkv + h) * head_bytes: K, V (side
// bytes each), then for e4m3 a scale byte per position of K and of V.
struct PageDesc {
  char* base;
  const int32_t* table;  // [B][width] page of positions page_size i ..
  int width, n_pages, hkv, log_page;
  int side;        // page_size * head_dim * element size
  int head_bytes;  // 2 side, + 2 page_size for e4m3
};

// Checks a pool's description; fills everything but the table.
int page_desc(const sdd_pages* pg, PageDesc* d);

__device__ inline char* page_head(const PageDesc& d, int page, int h) {
  return d.base + ((int64_t)page * d.hkv + h) * d.head_bytes;
}

// Stored order of a side of a page: steps of 32 positions, each the list of 1 KiB blocks that one attention step loads
// with one 16-byte load per lane.  Position p, dimension c (offsets in bytes from the side's start):
//   bf16  K block b * hd/32 + kk, lane 16 g + rho: dimensions 32 kk + 8 g .. + 7 of position kv_row(rho, b)
//         V block db,             lane 16 g + rho: positions 8 g .. 8 g + 7 of dimension 16 db + rho
//   e4m3  K block b * hd/64 + j,  lane 16 g + rho: dimensions 64 j + 16 g .. + 15 of position kv_row(rho, b)
//         V block jj,             lane 16 g + rho: positions 8 g .. 8 g + 7 of dimension 32 jj + rho, then of 32 jj + 16 + rho
// where kv_row(rho, b) = 8 (rho / 4) + 4 b + rho % 4 is the position that K sub-tile b feeds to MFMA row rho: the scores
// then leave lane group g on the positions 8 g .. 8 g + 7 of its V entries.
template <bool E4, int HD>
__device__ inline int page_k_offset(int p, int c) {
  const int i = p % 32, rho = 4 * (i / 8) + i % 4, b = (i / 4) % 2;
  if constexpr (E4) return p / 32 * 32 * HD + (b * (HD / 64) + c / 64) * 1024 + (16 * (c % 64 / 16) + rho) * 16 + c % 16;
  return p / 32 * 64 * HD + (b * (HD / 32) + c / 32) * 1024 + (16 * (c % 32 / 8) + rho) * 16 + c % 8 * 2;
}
template <bool E4, int HD>
__device__ inline int page_v_offset(int p, int c) {
  const int i = p % 32;
  if constexpr (E4) return p / 32 * 32 * HD + c / 32 * 1024 + (16 * (i / 8) + c % 16) * 16 + c % 32 / 16 * 8 + i % 8;
  return p / 32 * 64 * HD + c / 16 * 1024 + (16 * (i / 8) + c % 16) * 16 + i % 8 * 2;
}

// e4m3 rows are stored as codes of y 2^-e and a scale byte e + 127, e the smallest exponent with max |y| <= 448 2^e
// (1 <= e + 127 <= 254; a row of zeros has 127).  A power of two, so that the only rounding is the codes'.  A row that
// holds an infinity or a NaN is stored as NaN codes (0x7f) with byte 127.
__device__ inline int scale_byte(float amax) {
  if (!(amax > 0.f)) return 127;
  const uint32_t u = __builtin_bit_cast(uint32_t, amax);
  // amax = f 2^x, f in [1, 2); 448 = 1.75 2^8
  const int x = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  return max(1, min(254, x + 127));
}
__device__ inline float scale_value(int byte) { return __builtin_bit_cast(float, (uint32_t)byte << 23); }

// ---- new rows into a pool (paged.hip) -------------------------------------------------------------------
struct AppendArgs {
  PageDesc pg;
  const int32_t* len;
  const RowInfo* rows;  // instead of len: row b R holds the sequence (its table row), position and validity
  const char* qkv;
  int64_t row_stride;  // elements
  const float *q_gain, *k_gain, *rope;
  uint16_t* q_out;
  int32_t* err;
  int B, R, hq, max_pos;
  float eps;
  int n_qk;       // workgroups of the q/k part
  int per_wave;   // head sets that a wave takes one after the other
  int v_groups;   // 8-position groups that R rows can touch
  FastDiv by_waves, by_r, by_hkv, by_groups;  // (set by the launch; by_waves: waves of a row)
};

int launch_paged_append(AppendArgs a, int head_dim, bool e4, bool f32, hipStream_t st);

// ---- attention over a pool (paged_attn.hip) ------------------------------------------------------------
struct PagedAttnArgs {
  PageDesc pg;
  const int32_t* len;   // [B] positions before the rows; < 0: the sequence is skipped
  const RowInfo* rows;  // instead of len, as above
  const uint16_t* q;    // [B][R][hq][hd]
  uint16_t* out;        // the same, or fragment-major rows (frag)
  int frag;
  int B, R, hq, grp, max_len;
  // A chunk of a prompt, whose cut is the workspace's affair and may not show in the results: the many-vector kernel with every
  // sequence in one part, where a vector's sums depend on its own position and the cache alone.  No partial results.
  bool uncut;
  // |scale| of the scores, times log2(e) (1 for a scale of 0); the queries' bits are masked and flipped for its sign
  float scale;
  uint32_t q_and, q_xor;
  void set_scale(float x) {
    scale = x == 0.f ? 1.f : __builtin_fabsf(x) * 1.44269504088896340736f;
    q_and = x == 0.f ? 0u : ~0u;
    q_xor = x < 0.f ? 0x80008000u : 0u;
  }
  int32_t* err;
  // The cut of a call for each of the kernels: blocks of query vectors, chunks that a sequence of max_len positions has, chunks
  // at most and positions of one at least, positions up to which a sequence is not cut.
  struct Cut {
    int qtiles, splits, max_splits, min_chunk, whole;
    FastDiv by_qtiles;  // (set by the launch, as those below)
  } few, many;
  int many_from;     // positions from which a sequence is the many-vector kernel's
  int splits, qpad;  // of a sequence's partial results: chunks, and query vectors of one
  FastDiv by_grp, by_hkv, by_b, by_qv;
  float* part;  // partial results
};
// Bytes of partial results that a call needs that is not `uncut` (B, R, hq, grp, max_len and pg.hkv are read).
size_t paged_attn_workspace(PagedAttnArgs a, int head_dim);
int launch_paged_attn(PagedAttnArgs a, int head_dim, bool e4, hipStream_t st);

}  // namespace sdd
