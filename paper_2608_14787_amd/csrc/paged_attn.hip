// Attention of new rows over a paged KV cache (gfx950): R rows of each of B sequences, the sequence's own K/V of those
// rows already in its pages (bf16 or e4m3), row r at position len + r and seeing the positions up to its own.
//
// For a query vector q (row, head) over the visible positions p: s_p = scale q.k_p, w_p = e^(s_p - m), o = sum w_p v_p / sum w_p,
// in one pass with the running maximum m, sum and accumulator in fp32 (exponentials of base 2, scale holding log2 e).  The
// weights are rounded to bf16 for the second product, as V is held in bf16 or less; their sum takes them before that rounding.
// A second product with what the rounding leaves would make outputs exact to their own rounding, for 9 to 33% of the time (32
// decode rows 65 us for 56, 1024 prompt rows 91 for 68).  With few rows a row's largest weight is exactly 1 and outputs are off by
// 0.00175 of their size (28/4 heads, 513 positions), 0.00165 of it their own rounding.
//
// Two kernels.  paged_attn_kernel: a workgroup takes 16 query vectors of one KV head (rows x the heads that share it) over one
// chunk of the sequence; its four waves take the chunk's 32-position steps round-robin, each step's K and V straight into the
// wave's registers, and are joined through LDS in wave order.  paged_attn_wide_kernel, for calls with many query vectors: 128
// of them a workgroup, sharing each step through a ring in LDS.  A third joins the chunks' results in chunk order.  The cut of
// a sequence into chunks depends on its own length and the call's shape, not on what the others hold.
//
// The rows of a tile see different parts of its last steps, where a hidden position's weight of 0 does not keep out a V value that
// is not finite.  Both kernels zero such values there and add them behind the loop to the vectors that see them: 1024 rows of 64/8
// heads behind 3000 positions 143 us, with a NaN in the last position 151, in every row 175; 33 rows behind 1000 17 and 28.
//
// Bound, for 64/8 heads of 128: with few rows the stream of K and V (32 ragged sequences in bf16 53 us, 5.4 TB/s; 229000
// positions in e4m3 80 us, 5.9 TB/s) or, short, the chain of page id, loads, products and joins (one row, 513 positions 6.9 us);
// with many the softmax's instructions beside the products (1024 rows behind 1055 positions 65 us, 0.81 PFLOP/s; 4096 rows
// from 0 on 268, 1.0 PFLOP/s).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "gemm.h"
#include "paged.h"

namespace sdd {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;
// A chunk is at least two steps a wave, and a sequence is cut into no more workgroups than kTargetItems.  Measured with chunks
// of at least 128, 256 and 512 (attention alone): 32 ragged decode sequences 64, 53, 52 us; one of 513 positions 5.1, 5.5, 6.4.
constexpr int kMinChunk = 256;
constexpr int kTargetItems = 512;
// A short sequence is one chunk, so that its parts need no second kernel to join them: up to kWhole positions, or kWholeMany
// where its heads and rows are kManyItems workgroups as it is.  Measured, 64/8 heads, bf16, one chunk against several and
// the join: one row, 300 positions 5.8 / 8.1 us, 700 7.5 / 8.2, 1000 8.6 / 8.3, 1300 12.0 / 8.6; 33 rows (136 workgroups), 1300
// 11.6 / 14.6, 1600 12.8 / 15.5, and from e4m3 pages 15.0 / 15.1, 2000 17.3 / 16.2.
constexpr int kWhole = 768, kWholeMany = 1536, kManyItems = 64;

// The many-vector kernel: a workgroup's waves, a tile of 32 query vectors each; the number of such workgroups (before the cut
// into chunks) from which a call takes it; its chunks and items.  Measured, 64/8 heads of 128, bf16, this kernel against the
// other, both with the join: eight sequences of 284-3761 positions, 33 rows (192 workgroups) 57 / 76 us; six of 2000 (144) 45 /
// 50; four of 1000 (96) 30 / 19; one sequence, 1024 rows behind 1024 positions (512) 73 / 127; 256 rows (128) 38 / 27.
// Chunks of 256, 512, 768, 1024 with the first of these: 63, 57.5, 57, 61 us (longer ones leave compute units idle, shorter
// ones write more partial results).  A call has kWideItems workgroups at most: with many sequences partial results would cost
// more than they give (64 sequences, 33 rows: 279 us, and 366 where a sequence's chunks did not depend on the batch), with one
// sequence 512 fill the device (kWideFew; 1024 workgroups of 1024 rows behind 1024 positions: 102 instead of 69 us).
constexpr int kWideWaves = 4;
constexpr int kWideBlocks = 160;
constexpr int kWideChunk = 512, kWideItems = 2048, kWideFew = 4;
// Below kWideBlocks the two cross where a sequence is long: both are launched, and a sequence's positions say whose it is.
// Measured, one sequence, this kernel against the other: 256 rows of 28/4 heads (1792 vectors), behind 1000 positions 28.5 / 26,
// 8000 59 / 138; 400 rows behind 4000 57 / 107; 256 rows of 64/8 (2048) 38 / 27 and 101 / 154, from e4m3 pages 41 / 26 and 116 /
// 142; 65 rows (520) 27 / 13 and 47 / 68; 128 rows (1024) behind 3000 38 / 33.5, 8000 57 / 79, from e4m3 pages 66 / 77.
constexpr int kManyVectors = 1536, kManyFrom = 2560;
constexpr int kSomeVectors = 512, kSomeFrom = 6144;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Positions of a chunk of a sequence of total positions.
__host__ __device__ inline int chunk_of(const PagedAttnArgs::Cut& t, int total) {
  if (total <= t.whole) return t.whole;
  const int c = (total + t.max_splits - 1) / t.max_splits;
  return max(t.min_chunk, (c + 127) / 128 * 128);
}

struct Seq {
  int pos, row;  // position of the block's row 0 (-1: nothing to do), row of the table
};
__device__ inline Seq attn_seq(const PagedAttnArgs& a, int b, bool report) {
  int p, row = b, ok = 1;
  if (a.rows) {
    const RowInfo* ri = a.rows + (int64_t)b * a.R;
    p = ri->pos, row = ri->seq, ok = ri->valid;
  } else {
    p = a.len[b];
  }
  // (uniform values, in scalar registers: what is addressed with them stays there)
  p = __builtin_amdgcn_readfirstlane(p), row = __builtin_amdgcn_readfirstlane(row), ok = __builtin_amdgcn_readfirstlane(ok);
  const bool fits = (int64_t)p + a.R <= a.max_len;
  if (report && !fits && a.err && !a.rows) atomicOr(a.err, kErrCapacity);
  return Seq{ok && fits && p >= 0 ? p : -1, row};
}

// Partial results: rows of HD values, then a (maximum, sum) pair for each row; row (sequence x KV head, chunk, query vector).
__host__ __device__ inline int64_t part_rows(const PagedAttnArgs& a) { return (int64_t)a.B * a.pg.hkv * a.splits * a.qpad; }
__device__ inline int64_t part_row(const PagedAttnArgs& a, int bh, int c, int qv) {
  return ((int64_t)bh * a.splits + c) * a.qpad + qv;
}

__device__ inline int64_t out_index(const PagedAttnArgs& a, int b, int r, int h, int HD, int dim) {
  const int row = b * a.R + r;
  return a.frag ? xfrag_index<uint16_t>(row, h * HD + dim, a.hq * HD / 32) : ((int64_t)row * a.hq + h) * HD + dim;
}
__device__ inline void store_out4(const PagedAttnArgs& a, int b, int r, int h, int HD, int dim, const float* y) {
  *reinterpret_cast<uint2*>(a.out + out_index(a, b, r, h, HD, dim)) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
}

// Eight e4m3 codes to bf16, times a power of two (exact).
__device__ inline bf16x8 e4m3_frag(uint32_t x, uint32_t y, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)y, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)y, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// A query fragment as the products take it: scores are scaled by a.scale > 0 alone, so a negative scale's sign is the query's,
// and a scale of 0 a query of zeros.
__device__ inline uint4 load_q(const PagedAttnArgs& a, const uint16_t* q) {
  uint4 v = load16(q);
  v.x = (v.x & a.q_and) ^ a.q_xor, v.y = (v.y & a.q_and) ^ a.q_xor;
  v.z = (v.z & a.q_and) ^ a.q_xor, v.w = (v.w & a.q_and) ^ a.q_xor;
  return v;
}
__device__ inline uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Adds what is not finite among the V values of positions p .. p + 7 (a group of a step) and of dimension dim to y, as far as a
// vector at position qpos sees them: an infinity or NaN, times a positive weight, is itself.
template <bool E4, int HD>
__device__ inline float add_wild(const PagedAttnArgs& a, int page, int kvh, int p, int dim, int qpos, float y) {
  const char* v = page_head(a.pg, page, kvh) + a.pg.side + page_v_offset<E4, HD>(p & ((1 << a.pg.log_page) - 1), dim);
  if constexpr (E4) {
    const uint2 w = *reinterpret_cast<const uint2*>(v);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (p + i <= qpos && ((i < 4 ? w.x : w.y) >> (8 * (i % 4)) & 0x7f) == 0x7f) y = NAN;
  } else {
    const uint4 w = load16(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = bf16_to_f32((uint16_t)((i / 2 == 0 ? w.x : i / 2 == 1 ? w.y : i / 2 == 2 ? w.z : w.w) >> (16 * (i % 2))));
      if (p + i <= qpos && !__builtin_isfinite(x)) y += x;
    }
  }
  return y;
}

template <bool E4, int HD, bool ONCE>
__global__ void __launch_bounds__(kThreads, 3) paged_attn_kernel(PagedAttnArgs a) {
  constexpr int KK = HD / 32, DB = HD / 16;
  constexpr int NK = E4 ? HD / 64 : HD / 32, NV = E4 ? HD / 32 : HD / 16;  // 16-byte loads of a step: 2 NK of K, NV of V
  __shared__ __align__(16) float s_o[kWaves][16][HD + 4];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  __shared__ __align__(16) char s_q[KK * 1024];
  touch_kernargs<PagedAttnArgs>();
  const int hkv = a.pg.hkv;
  // workgroups go to the XCDs round-robin by id: the query tiles of one (chunk, sequence, head) share an XCD's L2
  const int low = blockIdx.x % kXcds, rest = blockIdx.x / kXcds;
  const int group = a.few.by_qtiles.div(rest), qt = rest - group * a.few.qtiles, item = group * kXcds + low;
  if (item >= a.few.splits * a.B * hkv) return;
  const int bc = a.by_hkv.div(item), kvh = item - bc * hkv, c = a.by_b.div(bc), b = bc - c * a.B;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const Seq sq = attn_seq(a, b, threadIdx.x == 0 && c == 0 && kvh == 0 && qt == 0);
  if (sq.pos < 0) return;
  const int total = sq.pos + a.R, chunk = chunk_of(a.few, total), n_chunks = (total + chunk - 1) / chunk;
  if (c >= n_chunks || total >= a.many_from) return;
  const int QV = a.R * a.grp, qv = qt * 16 + lane % 16;
  const bool qok = qv < QV;
  const int r = qok ? a.by_grp.div(qv) : 0, hh = qok ? qv - r * a.grp : 0;
  const int qpos = qok ? sq.pos + r : -1;
  const int lo = __builtin_amdgcn_readfirstlane(sq.pos + a.by_grp.div(qt * 16));  // position of the tile's first row
  const int tile_end = __builtin_amdgcn_readfirstlane(sq.pos + min(a.R - 1, a.by_grp.div(qt * 16 + 15)) + 1);
  const int p_begin = c * chunk, p_end = min(tile_end, p_begin + chunk);
  const int g8 = 8 * (lane / 16);

  // the chunk's page ids, 64 at a time across the lanes
  const int lg = a.pg.log_page;
  int page0 = p_begin >> lg, ids = 0;
  auto load_ids = [&]() { ids = a.pg.table[(int64_t)sq.row * a.pg.width + min(page0 + lane, a.pg.width - 1)]; };
  load_ids();
  // Query fragments (fragment i: the 8 dimensions that the i-th K operand of a step holds) sit in LDS.
  uint4 q_frag = make_uint4(0, 0, 0, 0);
  if (wave < KK) {
    const uint16_t* Q = a.q + ((int64_t)(b * a.R + r) * a.hq + kvh * a.grp + hh) * HD;
    q_frag = load_q(a, Q + (E4 ? 64 * (wave / 2) + 16 * (lane / 16) + 8 * (wave % 2) : 32 * wave + g8));
  }
  bool bad_page = false;
  // Where a step lies: the head's part of its page as a descriptor (one address register for all of a step's loads), the
  // position in the page, and whether the page exists.  Past the wave's last step the descriptor is of size zero and loads by
  // it touch no memory: every path through the loop has the same loads in flight, so each wait is for what it needs alone.
  struct Place {
    __amdgpu_buffer_rsrc_t page;
    int in;
    bool ok;
  };
  auto place = [&](int p) {
    const bool in_range = p < p_end;
    const int i = in_range ? (p >> lg) - page0 : 0;
    int id;
    if (i < kWave) {
      id = __builtin_amdgcn_readlane(ids, i);
    } else {  // (read here as well, so that only this path waits for the load)
      page0 += kWave;
      load_ids();
      id = __builtin_amdgcn_readlane(ids, i - kWave);
    }
    const bool ok = (unsigned)id < (unsigned)a.pg.n_pages;
    bad_page |= in_range && !ok;
    return Place{__builtin_amdgcn_make_buffer_rsrc(page_head(a.pg, ok ? id : 0, kvh), 0, in_range ? a.pg.head_bytes : 0,
                                                   kBufferRsrcWord3),
                 p & ((1 << lg) - 1), ok};
  };
  uint4 kr[2][NK], vr[NV];
  uint8_t ks[2] = {0, 0};  // e4m3: scale byte of the lane's K row of each sub-tile
  uint2 vs = {0, 0};      // and those of its 8 positions of V
  auto load = [&](const Place& pl, int off) {
    // (ONCE: one query tile, which reads a position once: non-temporal)
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(pl.page, lane * 16, off, ONCE ? kNtCpol : 0));
  };
  auto load_k = [&](const Place& pl) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < NK; ++j) kr[s][j] = load(pl, pl.in * HD * (E4 ? 1 : 2) + (s * NK + j) * 1024);
    if constexpr (E4)
#pragma unroll
      for (int s = 0; s < 2; ++s)
        ks[s] = __builtin_amdgcn_raw_buffer_load_b8(pl.page, kv_row(lane % 16, s), 2 * a.pg.side + pl.in, 0);
  };
  auto load_v = [&](const Place& pl) {
#pragma unroll
    for (int j = 0; j < NV; ++j) vr[j] = load(pl, a.pg.side + pl.in * HD * (E4 ? 1 : 2) + j * 1024);
    if constexpr (E4) {
      const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(pl.page, g8, 2 * a.pg.side + (1 << lg) + pl.in, 0);
      vs = make_uint2(v[0], v[1]);
    }
  };

  f32x4 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;  // (m: of the scores before the scale)
  float ref = 0.f;               // -m scale (0 for no m)
  // the step from which some of the tile's vectors see less than others (a single row's: none)
  const int own_rows = tile_end == lo + 1 ? INT32_MAX : max(p_begin, (lo + 1) & ~31);
  bool wild = false;  // the lane has zeroed a value there
  // V operand of 16 dimensions.  Of a step that not every vector sees whole, positions outside `mask` (a bit for each of the
  // lane's 8) are zeroed: their weights are 0, and 0 times a stale or foreign non-finite value would not be.  So is what is not
  // finite among the tile's own rows, to be added behind the loop.
  auto v_frag = [&](auto part, auto own, int db, uint32_t mask) {
    constexpr bool PART = decltype(part)::value, OWN = decltype(own)::value;
    if constexpr (E4) {
      uint32_t w[2] = {word(vr[db / 2], db % 2 * 2), word(vr[db / 2], db % 2 * 2 + 1)};
      if constexpr (PART) {
        uint32_t keep[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) keep[i / 4] |= (mask >> i & 1) ? 0xffu << (8 * (i % 4)) : 0u;
        w[0] &= keep[0], w[1] &= keep[1];
      }
      if constexpr (OWN)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t bad = ((w[k] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;  // (the NaN codes)
          w[k] &= ~((bad << 1) - (bad >> 7));
          wild |= bad != 0;
        }
      return e4m3_frag(w[0], w[1], 1.f);
    } else {
      uint32_t w[4] = {vr[db].x, vr[db].y, vr[db].z, vr[db].w};
      if constexpr (PART)
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] &= ((mask >> (2 * k) & 1) ? 0xffffu : 0u) | ((mask >> (2 * k + 1) & 1) ? 0xffff0000u : 0u);
      if constexpr (OWN)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t bad = ((w[k] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;  // (exponents of all ones)
          w[k] &= ~((bad << 1) - (bad >> 15));
          wild |= bad != 0;
        }
      return __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
    }
  };
  auto below = [&](int p, int end) {  // mask of the lane's positions of step p that lie before end
    const int n = max(0, min(8, end - (p + g8)));
    return (1u << n) - 1u;
  };
  constexpr int kStride = 32 * kWaves;
  const int p0 = p_begin + 32 * wave;
  Place pl;
  // Step p, whose place is pl; issues the next one's loads.
  auto step = [&](int p) {
    const bool ok = pl.ok;
    f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < KK; ++i) {
      const bf16x8 q = *reinterpret_cast<const bf16x8*>(s_q + i * 1024 + lane * 16);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        bf16x8 k;
        if constexpr (E4)
          k = e4m3_frag(word(kr[t][i / 2], i % 2 * 2), word(kr[t][i / 2], i % 2 * 2 + 1), scale_value(ks[t]));
        else
          k = __builtin_bit_cast(bf16x8, kr[t][i]);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q, s[t], 0, 0, 0);
      }
    }
    // s[i / 4][i % 4]: position p + g8 + i, query vector lane % 16
    float sv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sv[i] = s[i / 4][i % 4];
    // K's registers are free: the next step's loads go out ahead of this one's softmax, V's after its product
    pl = place(p + kStride);
    load_k(pl);
    __builtin_amdgcn_sched_barrier(0);
    const bool inner = p + 31 <= lo && p + 32 <= p_end && ok;  // every query vector sees the whole step
    if (!inner) {
      const int end = ok ? min(qpos + 1, p_end) : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) sv[i] = p + g8 + i < end ? sv[i] : -INFINITY;
    }
    float top = sv[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, sv[i]);
    top = xor16_op(top, [](float x, float y) { return fmaxf(x, y); });
    top = xor32_op(top, [](float x, float y) { return fmaxf(x, y); });
    if (__any(top > m)) {
      const float mn = fmaxf(m, top), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * a.scale);
      l *= f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= f;
      m = mn;
      ref = m == -INFINITY ? 0.f : -m * a.scale;  // (a hidden score's weight is then exp2(-inf) = 0)
    }
    float e[8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[i], a.scale, ref));
      sum += e[i];
    }
    l += sum;
    if constexpr (E4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] *= scale_value(((i < 4 ? vs.x : vs.y) >> (8 * (i % 4))) & 255);
      if (!inner) {  // (a position that was never written may have any scale byte)
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = sv[i] == -INFINITY ? 0.f : e[i];
      }
    }
    const bf16x8 pf = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]),
                                                            pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])));
    auto values = [&](auto part, auto own, uint32_t mask) {
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_frag(part, own, db, mask), pf, o[db], 0, 0, 0);
    };
    if (inner)
      values(std::false_type(), std::false_type(), 0);
    else if (p < own_rows)
      values(std::true_type(), std::false_type(), below(p, ok ? p_end : 0));
    else
      values(std::true_type(), std::true_type(), below(p, ok ? p_end : 0));
  };
  pl = place(p0);
  load_k(pl);
  load_v(pl);
  if (wave < KK) *reinterpret_cast<uint4*>(s_q + wave * 1024 + lane * 16) = q_frag;
  __syncthreads();  // the queries are in LDS
#pragma unroll 1
  for (int p = p0; p < p_end; p += kStride) {
    step(p);
    __builtin_amdgcn_sched_barrier(0);
    load_v(pl);
  }
  // what the wave zeroed of its steps (48 positions at most, in two of them)
  if (__any(wild)) {
#pragma unroll 1
    for (int p = own_rows; p < min(p_end, tile_end); p += 8) {
      const int id = a.pg.table[(int64_t)sq.row * a.pg.width + (p >> lg)];
      if ((p - p_begin) / 32 % kWaves != wave || (unsigned)id >= (unsigned)a.pg.n_pages) continue;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[db][i] = add_wild<E4, HD>(a, id, kvh, p, 16 * db + 4 * (lane / 16) + i, qpos, o[db][i]);
    }
  }
  m *= a.scale;  // (-inf stays: the scale is positive)
  if (a.err && bad_page && lane == 0) atomicOr(a.err, kErrId);
  l = xor16_op(l, [](float x, float y) { return x + y; });
  l = xor32_op(l, [](float x, float y) { return x + y; });
#pragma unroll
  for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(&s_o[wave][lane % 16][16 * db + 4 * (lane / 16)]) = o[db];
  if (lane < 16) {
    s_m[wave][lane] = m;
    s_l[wave][lane] = l;
  }
  __syncthreads();
  const int64_t at = part_row(a, b * hkv + kvh, c, qt * 16);
  float* part_o = a.part + at * HD;
  float* part_ml = a.part + part_rows(a) * HD + at * 2;
  for (int e = threadIdx.x; e < 16 * HD / 4; e += kThreads) {
    const int q = e / (HD / 4), d = e % (HD / 4) * 4;
    if (qt * 16 + q >= QV) continue;
    float M = s_m[0][q];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][q]);
    float y[4] = {0.f, 0.f, 0.f, 0.f}, L = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      // (a wave whose visible scores are all NaN has m = -inf and a NaN sum)
      const float f = s_m[w][q] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(s_m[w][q] - M);
      L += f * s_l[w][q];
      const f32x4 v = *reinterpret_cast<const f32x4*>(&s_o[w][q][d]);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] += f * v[i];
    }
    if (n_chunks == 1) {
      const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = L == 0.f ? 0.f : y[i] * inv;
      const int qq = qt * 16 + q;
      store_out4(a, b, a.by_grp.div(qq), kvh * a.grp + qq - a.by_grp.div(qq) * a.grp, HD, d, y);
    } else {
      *reinterpret_cast<f32x4*>(part_o + q * HD + d) = f32x4{y[0], y[1], y[2], y[3]};
      if (d == 0) {
        part_ml[2 * q] = M;
        part_ml[2 * q + 1] = L;
      }
    }
  }
}

// ---- many query vectors ---------------------------------------------------------------------------------
//
// A workgroup takes NW tiles of 32 query vectors of one KV head, a wave each (queries and accumulators in registers), over one
// chunk.  The steps of K and V pass through a ring in LDS, loaded there directly (no registers, several steps in flight) and
// read by every wave; e4m3 operands are converted on their way from LDS to the products.  S^T = K Q^T and O^T = V^T P^T by
// 32x32x16 products: a lane holds 16 scores of one query vector, which are its operand of the second product as they stand
// (the stored order of K's rows sees to that).  At 168 registers three workgroups share a compute unit (bf16 with 128 dimensions
// keeps two values of its end in scratch for that), and 36 or 48 KiB of LDS each.

// Four reads of 16 (8) bytes a lane from addr + off(i), and their wait, in one block: the compiler would hold every LDS read back
// until all direct loads into LDS, those of later steps too, have landed.
template <int DIV, int HI, int LO>  // off(i) = i / DIV * HI + i % DIV * LO
__device__ inline void lds_read16(u32x4* f, uint32_t addr) {
  constexpr auto off = [](int i) { return i / DIV * HI + i % DIV * LO; };
  asm volatile("ds_read_b128 %0, %4 offset:%5\n\tds_read_b128 %1, %4 offset:%6\n\tds_read_b128 %2, %4 offset:%7\n\t"
               "ds_read_b128 %3, %4 offset:%8\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
               : "v"(addr), "i"(off(0)), "i"(off(1)), "i"(off(2)), "i"(off(3)) : "memory");
}
template <int STEP>
__device__ inline void lds_read8(u32x2* f, uint32_t addr) {
  asm volatile("ds_read_b64 %0, %4\n\tds_read_b64 %1, %4 offset:%5\n\tds_read_b64 %2, %4 offset:%6\n\t"
               "ds_read_b64 %3, %4 offset:%7\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
               : "v"(addr), "i"(STEP), "i"(2 * STEP), "i"(3 * STEP) : "memory");
}

// An e4m3 step's K operands (N reads of 16 bytes, 512 apart) and scale bytes, as above.
template <int N>
__device__ inline void lds_read_e4(u32x4* k, u32x2* sb, uint32_t ak, uint32_t aks, uint32_t avs) {
  static_assert(N == 2 || N == 4, "reads of a block");
  uint32_t ks;
  if constexpr (N == 2) {
    asm volatile("ds_read_u8 %2, %6\n\tds_read_b128 %0, %5\n\tds_read_b128 %1, %5 offset:512\n\tds_read_b64 %3, %7\n\t"
                 "ds_read_b64 %4, %7 offset:16\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(k[0]), "=&v"(k[1]), "=&v"(ks), "=&v"(sb[1]), "=&v"(sb[2]) : "v"(ak), "v"(aks), "v"(avs) : "memory");
  } else {
    asm volatile("ds_read_u8 %4, %8\n\tds_read_b128 %0, %7\n\tds_read_b128 %1, %7 offset:512\n\tds_read_b128 %2, %7 offset:1024\n\t"
                 "ds_read_b128 %3, %7 offset:1536\n\tds_read_b64 %5, %9\n\tds_read_b64 %6, %9 offset:16\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(k[0]), "=&v"(k[1]), "=&v"(k[2]), "=&v"(k[3]), "=&v"(ks), "=&v"(sb[1]), "=&v"(sb[2])
                 : "v"(ak), "v"(aks), "v"(avs) : "memory");
  }
  sb[0][0] = ks;
}

// The weights' reference m need not be the maximum here: it moves, and with it the accumulators, only where a score passes it by
// kFar (weights up to 2^kFar; sums are fp32).  With 32 query vectors some maximum rises in most steps: rescaled at each rise, a
// third of the step's vector instructions were the accumulators'.  The price is that a row's largest weight, 1 where it is the
// reference, is rounded to bf16 too.  Rescaled at each rise, 1024 rows of 64/8 heads behind 1055 positions take 76 us for 68 and
// eight blocks of 33 rows 60 for 55; outputs are off by 0.0018 of their size then, 0.0023 so, and 0.0017 where only they are
// rounded.
constexpr float kFar = 8.f;

template <bool E4, int HD>
__global__ void __launch_bounds__(kWideWaves * kWave, 3) paged_attn_wide_kernel(PagedAttnArgs a) {
  constexpr int NW = kWideWaves;
  constexpr int KS = HD / 16, DB = HD / 32;   // products of a tile and step: KS for the scores, 2 DB for the values
  constexpr int NB = (E4 ? 2 : 4) * HD / 32;  // 1 KiB blocks of a step, K's then V's
  constexpr int L = NB / NW + (E4 ? 1 : 0);   // loads that a wave issues for a step (e4m3: its own copy of the scale bytes)
  constexpr int kStage = NB * 1024 + (E4 ? NW * 256 : 0);
  constexpr int RS = E4 ? 4 : 3;              // ring stages: RS - 1 steps in flight, of 8 or 16 KiB
  static_assert(NB % NW == 0, "a step's blocks over the waves");
  __shared__ __align__(16) char s_ring[RS * kStage];
  touch_kernargs<PagedAttnArgs>();
  const int hkv = a.pg.hkv;
  const int low = blockIdx.x % kXcds, rest = blockIdx.x / kXcds;
  const int group = a.many.by_qtiles.div(rest), qb = a.many.qtiles - 1 - (rest - group * a.many.qtiles), item = group * kXcds + low;
  if (item >= a.many.splits * a.B * hkv) return;
  const int bc = a.by_hkv.div(item), kvh = item - bc * hkv, c = a.by_b.div(bc), b = bc - c * a.B;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, half = lane / 32;
  const Seq sq = attn_seq(a, b, threadIdx.x == 0 && c == 0 && kvh == 0 && qb == 0);
  if (sq.pos < 0) return;
  const int total = sq.pos + a.R, chunk = chunk_of(a.many, total), n_chunks = (total + chunk - 1) / chunk;
  if (c >= n_chunks || total < a.many_from) return;
  const int QV = a.R * a.grp, q_block = qb * NW * 32, q0 = q_block + wave * 32, qv = q0 + lane % 32;
  const int block_end = __builtin_amdgcn_readfirstlane(sq.pos + min(a.R - 1, a.by_grp.div(q_block + NW * 32 - 1)) + 1);
  const int p_begin = c * chunk, p_end = min(block_end, p_begin + chunk);
  // the lane's query's position (-1: none; its column of the products is computed as any other and not stored); the tile's first
  // position, which all its vectors see, and the one past its last (0: no queries)
  const bool qok = qv < QV;
  const int r = qok ? a.by_grp.div(qv) : 0, hh = qok ? qv - r * a.grp : 0;
  const int qpos = qok ? sq.pos + r : -1;
  const int first = __builtin_amdgcn_readfirstlane(sq.pos + a.by_grp.div(q0));
  const int tile_end = __builtin_amdgcn_readfirstlane(q0 < QV ? sq.pos + min(a.R - 1, a.by_grp.div(q0 + 31)) + 1 : 0);
  const int lg = a.pg.log_page;
  int page0 = p_begin >> lg, ids = 0;  // the chunk's page ids, 64 at a time across the lanes
  auto load_ids = [&]() { ids = a.pg.table[(int64_t)sq.row * a.pg.width + min(page0 + lane, a.pg.width - 1)]; };
  load_ids();
  bf16x8 qf[KS];  // fragment i: the dimensions of the i-th K operand
  {
    const uint16_t* Q = a.q + ((int64_t)(b * a.R + r) * a.hq + kvh * a.grp + hh) * HD;
#pragma unroll
    for (int i = 0; i < KS; ++i)
      qf[i] = __builtin_bit_cast(bf16x8, load_q(a, Q + (E4 ? 64 * (i / 4) + 32 * (i / 2 % 2) + 16 * half + 8 * (i % 2) : 16 * i + 8 * half)));
  }
  bool bad_page = false;
  int p_load = p_begin, slot = 0;  // next step to load, its byte offset in the ring
  uint32_t ok_bits = 0;            // whether the pages of the steps in flight exist, the oldest in bit RS - 2
  // the page of the next step: its head's bytes, their number (0 for a missing page)
  char* page_at = nullptr;
  int page_bytes = 0;
  const int in_mask = (1 << lg) - 1;
  auto turn_page = [&]() {
    const int i = min(p_load, max(p_end - 1, p_begin)) >> lg;
    int id;
    if (i - page0 < kWave) {
      id = __builtin_amdgcn_readlane(ids, i - page0);
    } else {  // (read here as well, so that only this path waits for the load)
      page0 += kWave;
      load_ids();
      id = __builtin_amdgcn_readlane(ids, i - page0);
    }
    const bool ok = (unsigned)id < (unsigned)a.pg.n_pages;
    bad_page |= !ok && p_load < p_end;
    page_at = page_head(a.pg, ok ? id : 0, kvh);
    page_bytes = ok ? a.pg.head_bytes : 0;
  };
  auto issue = [&]() {
    const int in = p_load & in_mask, at = in * HD * (E4 ? 1 : 2);
    if (in == 0) turn_page();
    ok_bits = ok_bits << 1 | (page_bytes ? 1u : 0u);
    // (past the end, and for a missing page, loads of no memory: the count in flight stays the same)
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(page_at, 0, p_load < p_end ? page_bytes : 0, kBufferRsrcWord3);
    char* st = s_ring + slot;
#pragma unroll
    for (int j = 0; j < NB / NW; ++j) {
      const int blk = wave + NW * j;
      load_lds16<0>(rs, st + blk * 1024, lane * 16, blk < NB / 2 ? at + blk * 1024 : a.pg.side + at + (blk - NB / 2) * 1024);
    }
    if constexpr (E4)  // 16 lanes of 4 bytes: K's 32 scale bytes, V's
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(st + NB * 1024 + wave * 256), 4,
                                               lane < 16 ? lane % 8 * 4 + (lane / 8 << lg) : 0x7ffffff0, 2 * a.pg.side + in, 0, 0);
    p_load += 32;
    slot = slot + kStage == RS * kStage ? 0 : slot + kStage;
  };

  const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(s_ring);
  const int rho = lane % 16, b16 = lane % 32 / 16;
  const uint32_t rd_k = ring + b16 * (NB / 4) * 1024 + (16 * half + rho) * 16;
  const uint32_t rd_v = ring + NB / 2 * 1024 + (E4 ? (16 * half + rho) * 16 + 8 * b16 : b16 * 1024 + (16 * half + rho) * 16);
  const uint32_t rd_ks = ring + NB * 1024 + wave * 256 + kv_row(rho, b16), rd_vs = ring + NB * 1024 + wave * 256 + 32 + 8 * half;
  f32x16 o[DB];
  float m = -INFINITY, l = 0.f;           // (m: of the scores before the scale)
  float ref = 0.f, m_far = -INFINITY;     // -m scale (0 for no m), and the score from which m moves
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  turn_page();
#pragma unroll
  for (int i = 0; i < RS - 1; ++i) issue();
  uint32_t so = 0;  // this step's byte offset in the ring
  auto next_step = [&]() {
    __builtin_amdgcn_s_waitcnt(wait_vmcnt((RS - 2) * L));
    phase_barrier();  // the step is whole, and the slot of the step before it has been read by every wave
    issue();
  };
  const int own_rows = max(p_begin, (first + 1) & ~31);  // the step from which some of the tile's vectors see less than others
  bool wild = false;                                     // the lane has zeroed a value there
  // Step p, at so in the ring.  INNER: every query vector sees the whole of it.
  auto step = [&](auto inner_c, int p, bool ok) {
    constexpr bool inner = decltype(inner_c)::value;
    const uint32_t at_step = so;
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
    u32x2 vs[2] = {u32x2{0, 0}, u32x2{0, 0}};  // e4m3: V's scale bytes of positions 8 half .. and 16 + 8 half ..
    auto at = [&](int i) { return 16 * (i / 4 % 2) + 8 * half + 4 * (i / 8) + i % 4; };  // position of s[i]
    if constexpr (E4) {
      u32x4 kr[KS / 2];
      u32x2 sb[3];  // scale bytes: of the lane's K row, V's
      lds_read_e4<KS / 2>(kr, sb, rd_k + at_step, rd_ks + at_step, rd_vs + at_step);
      const float ks = scale_value((int)sb[0][0]);
#pragma unroll
      for (int i = 0; i < KS; ++i)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(e4m3_frag(kr[i / 2][i % 2 * 2], kr[i / 2][i % 2 * 2 + 1], ks), qf[i], s, 0, 0, 0);
      vs[0] = sb[1], vs[1] = sb[2];
    } else {
#pragma unroll
      for (int h = 0; h < KS; h += 4) {
        u32x4 kr[4];
        lds_read16<4, 0, 512>(kr, rd_k + at_step + h * 512);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr[i]), qf[h + i], s, 0, 0, 0);
      }
    }
    float sv[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sv[i] = s[i];
    if constexpr (!inner) {
      const int e = ok ? min(qpos + 1, p_end) : 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) sv[i] = p + at(i) < e ? sv[i] : -INFINITY;
    }
    float top = sv[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, sv[i]);
    top = xor32_op(top, [](float x, float y) { return fmaxf(x, y); });
    // (each vector's reference moves by its own scores: what it gives does not depend on the others of its tile)
    const bool far = top * a.scale > m_far;
    if (__any(far)) {
      const float mn = far ? fmaxf(m, top) : m;
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * a.scale);
      l *= f;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= f;
      m = mn;
      ref = m == -INFINITY ? 0.f : -m * a.scale;
      ref = __builtin_isfinite(ref) ? ref : NAN;  // (scores past the range have no weights; minus infinity would make all of them 0)
      m_far = m == -INFINITY ? -INFINITY : kFar - ref;
    }
    float e[16], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[i], a.scale, ref));
      sum += e[i];
    }
    l += sum;
    if constexpr (E4) {
#pragma unroll
      for (int i = 0; i < 16; ++i)  // byte 4 (i / 8) + i % 4 of the eight from 16 (i / 4 % 2) + 8 half
        e[i] *= scale_value((vs[i / 4 % 2][i / 8] >> (8 * (i % 4))) & 255);
      if constexpr (!inner) {  // (a position that was never written may have any scale byte)
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = sv[i] == -INFINITY ? 0.f : e[i];
      }
    }
    bf16x8 pf[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)  // positions 16 h + 8 half .. + 7: registers 4 h .. and 8 + 4 h ..
      pf[h] = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16x2(e[4 * h], e[4 * h + 1]), pack_bf16x2(e[4 * h + 2], e[4 * h + 3]),
                                                    pack_bf16x2(e[8 + 4 * h], e[9 + 4 * h]),
                                                    pack_bf16x2(e[10 + 4 * h], e[11 + 4 * h])));
    // V operands, 64 dimensions at a time: operand 2 db + h holds dimension 32 db + lane % 32, positions 16 h + 8 half .. + 7
#pragma unroll
    for (int g = 0; g < DB; g += 2) {
      bf16x8 v[4];
      // Positions from p_end on are zeroed: their weights are 0, and 0 times a stale non-finite value would not be.  The tile's own
      // rows see different parts of a step: what is not finite there is zeroed too, and added behind the loop to those that see it.
      auto seen = [&](int i) { return (ok ? p_end : 0) - (p + 16 * (i % 2) + 8 * half); };  // positions of operand i
      if constexpr (E4) {
        u32x2 vr[4];
        lds_read8<512>(vr, rd_v + at_step + g * 1024);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (!inner)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int n = max(0, min(4, seen(i) - 4 * k));
              uint32_t w = vr[i][k] & (uint32_t)((uint64_t(1) << (8 * n)) - 1);
              const uint32_t bad = ((w & 0x7f7f7f7fu) + 0x01010101u) & (p >= own_rows ? 0x80808080u : 0u);  // (the NaN codes)
              w &= ~((bad << 1) - (bad >> 7));
              wild |= bad != 0;
              vr[i][k] = w;
            }
          v[i] = e4m3_frag(vr[i][0], vr[i][1], 1.f);
        }
      } else {
        u32x4 vr[4];
        lds_read16<2, 2048, 512>(vr, rd_v + at_step + g * 2048);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (!inner)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint32_t w = vr[i][k] & ((2 * k < seen(i) ? 0xffffu : 0u) | (2 * k + 1 < seen(i) ? 0xffff0000u : 0u));
              const uint32_t bad = ((w & 0x7f807f80u) + 0x00800080u) & (p >= own_rows ? 0x80008000u : 0u);  // (exponents of all ones)
              w &= ~((bad << 1) - (bad >> 15));
              wild |= bad != 0;
              vr[i][k] = w;
            }
          v[i] = __builtin_bit_cast(bf16x8, vr[i]);
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int db = 0; db < 2; ++db) o[g + db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[2 * db + h], pf[h], o[g + db], 0, 0, 0);
    }
  };
  int p = p_begin;
  // the steps that every query vector sees whole, up to a missing page; then the others (one loop after the other: as the two
  // sides of a branch in one loop they would each copy the accumulators)
  const int p_inner = min(min(first - 31, p_end - 32), tile_end - 1);
#pragma unroll 1
  for (; p <= p_inner && (ok_bits >> (RS - 2) & 1); p += 32) {
    next_step();
    step(std::true_type{}, p, true);
    so = so + kStage == (uint32_t)(RS * kStage) ? 0 : so + kStage;
  }
#pragma unroll 1
  for (; p < min(p_end, tile_end); p += 32) {
    const bool ok = ok_bits >> (RS - 2) & 1;
    next_step();
    step(std::false_type{}, p, ok);
    so = so + kStage == (uint32_t)(RS * kStage) ? 0 : so + kStage;
  }
  for (; p < p_end; p += 32) next_step();  // (steps behind the tile's last position: the other waves')
  __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));  // (the loads past the end: they clear LDS)
  if (a.err && bad_page && threadIdx.x == 0) atomicOr(a.err, kErrId);
  // what the wave zeroed (64 positions at most)
  if (__any(wild)) {
#pragma unroll 1
    for (int p = own_rows; p < min(p_end, tile_end); p += 8) {
      const int id = a.pg.table[(int64_t)sq.row * a.pg.width + (p >> lg)];
      if ((unsigned)id >= (unsigned)a.pg.n_pages) continue;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i)  // dimension 32 db + 8 (i / 4) + 4 half + i % 4
          o[db][i] = add_wild<E4, HD>(a, id, kvh, p, 32 * db + 8 * (i / 4) + 4 * half + i % 4, qpos, o[db][i]);
    }
  }
  const float lsum = xor32_op(l, [](float x, float y) { return x + y; });
  if (!qok) return;
  const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
  const int64_t row = part_row(a, b * hkv + kvh, c, qv);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // dimensions 32 db + 8 i + 4 half .. + 3
      const int d = 32 * db + 8 * i + 4 * half;
      float y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = o[db][4 * i + k];
      if (n_chunks == 1) {
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = lsum == 0.f ? 0.f : y[k] * inv;
        store_out4(a, b, r, kvh * a.grp + hh, HD, d, y);
      } else {
        *reinterpret_cast<f32x4*>(a.part + row * HD + d) = f32x4{y[0], y[1], y[2], y[3]};
      }
    }
  if (n_chunks > 1 && half == 0) {
    float* ml = a.part + part_rows(a) * HD + row * 2;
    ml[0] = m * a.scale;
    ml[1] = lsum;
  }
}

// Joins the chunks of a query vector, 4 dimensions a lane: four sums, of the chunks c = g mod 4 in order, added in order of g.
// A call whose sequences have few chunks takes one group of HD / 4 lanes for all four (SMALL: up to kSmallJoin chunks, all of a
// vector's loads in flight at once); others a group for each.  The sums are the same.
constexpr int kJoin = 4, kSmallJoin = 16;
template <int HD, bool SMALL>
__global__ void __launch_bounds__(kThreads) paged_combine_kernel(PagedAttnArgs a) {
  constexpr int LN = HD / 4, VEC = kThreads / (SMALL ? LN : LN * kJoin);
  __shared__ __align__(16) float s_y[SMALL ? 1 : kThreads][4];
  __shared__ float s_l[kThreads / LN];
  const int grp = threadIdx.x / LN, ln = threadIdx.x % LN, d = 4 * ln, QV = a.R * a.grp;
  const int idx = (int)blockIdx.x * VEC + (SMALL ? grp : grp / kJoin);
  const int bh = a.by_qv.div(idx), qv = idx - bh * QV, b = a.by_hkv.div(bh), kvh = bh - b * a.pg.hkv;
  int n = 1;
  if (b < a.B) {
    int p = a.rows ? a.rows[(int64_t)b * a.R].pos : a.len[b];
    const bool ok = (!a.rows || a.rows[(int64_t)b * a.R].valid) && p >= 0 && (int64_t)p + a.R <= a.max_len;
    const int total = p + a.R;
    const int chunk = chunk_of(total < a.many_from ? a.few : a.many, total);
    if (ok) n = (total + chunk - 1) / chunk;
  }
  const int64_t at = part_row(a, bh, 0, qv), stride = a.qpad;  // (of a chunk)
  const float* o = a.part + at * HD + d;
  const float* ml = a.part + part_rows(a) * HD + at * 2;
  f32x4 y[kJoin];
  float L[kJoin], M = -INFINITY;
#pragma unroll
  for (int g = 0; g < kJoin; ++g) y[g] = f32x4{0.f, 0.f, 0.f, 0.f}, L[g] = 0.f;
  auto add = [&](int g, float mc, float lc, const f32x4& v) {
    const float f = mc == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mc - M);  // (no maximum: a sum of 0, or of NaN scores)
    L[g] += f * lc;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[g][i] += f * v[i];
  };
  if constexpr (SMALL) {
    if (n == 1) return;
    constexpr int U = 8;
    float2 p[kSmallJoin];
    f32x4 v[U];
#pragma unroll
    for (int c = 0; c < kSmallJoin; ++c) p[c] = *reinterpret_cast<const float2*>(ml + 2 * stride * min(c, n - 1));
#pragma unroll
    for (int c = 0; c < U; ++c) v[c] = *reinterpret_cast<const f32x4*>(o + stride * min(c, n - 1) * HD);
#pragma unroll
    for (int c = 0; c < kSmallJoin; ++c) M = fmaxf(M, p[c].x);
#pragma unroll
    for (int c = 0; c < U; ++c)
      if (c < n) add(c % kJoin, p[c].x, p[c].y, v[c]);
    if (n > U) {
#pragma unroll
      for (int c = 0; c < U; ++c) v[c] = *reinterpret_cast<const f32x4*>(o + stride * min(U + c, n - 1) * HD);
#pragma unroll
      for (int c = 0; c < U; ++c)
        if (U + c < n) add(c % kJoin, p[U + c].x, p[U + c].y, v[c]);
    }
  } else {
    constexpr int U = 8;
    const int g = grp % kJoin;
    if (n > 1) {
      for (int c = ln; c < n; c += LN) M = fmaxf(M, ml[2 * stride * c]);
#pragma unroll
      for (int k = 1; k < LN; k *= 2) M = fmaxf(M, __shfl_xor(M, k));
      for (int c0 = g; c0 < n; c0 += kJoin * U) {
        f32x4 v[U];
        float2 p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int c = min(c0 + kJoin * u, n - 1);
          p[u] = *reinterpret_cast<const float2*>(ml + 2 * stride * c);
          v[u] = *reinterpret_cast<const f32x4*>(o + stride * c * HD);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c0 + kJoin * u < n) add(0, p[u].x, p[u].y, v[u]);
      }
    }
    *reinterpret_cast<f32x4*>(s_y[threadIdx.x]) = y[0];
    if (ln == 0) s_l[grp] = L[0];
    __syncthreads();
    if (g != 0 || n == 1) return;
#pragma unroll
    for (int k = 1; k < kJoin; ++k) {
      L[k] = s_l[grp + k];
      y[k] = *reinterpret_cast<const f32x4*>(s_y[threadIdx.x + k * LN]);
    }
  }
#pragma unroll
  for (int k = 1; k < kJoin; ++k) {
    L[0] += L[k];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[0][i] += y[k][i];
  }
  const float inv = 1.f / L[0];
  float out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = L[0] == 0.f ? 0.f : y[0][i] * inv;
  const int r = a.by_grp.div(qv);
  store_out4(a, b, r, kvh * a.grp + qv - r * a.grp, HD, d, out);
}

template <bool E4, int HD>
void launch_t(const PagedAttnArgs& a, hipStream_t st) {
  auto grid = [&](const PagedAttnArgs::Cut& t) { return dim3((unsigned)(ceil_div((int64_t)t.splits * a.B * a.pg.hkv, kXcds) * kXcds * t.qtiles)); };
  if (a.many_from <= a.max_len)
    hipLaunchKernelGGL((paged_attn_wide_kernel<E4, HD>), grid(a.many), dim3(kWideWaves * kWave), 0, st, a);
  if (a.many_from > 0 && a.few.qtiles == 1)
    hipLaunchKernelGGL((paged_attn_kernel<E4, HD, true>), grid(a.few), dim3(kThreads), 0, st, a);
  else if (a.many_from > 0)
    hipLaunchKernelGGL((paged_attn_kernel<E4, HD, false>), grid(a.few), dim3(kThreads), 0, st, a);
  if (a.splits > 1) {
    const int64_t vecs = (int64_t)a.B * a.pg.hkv * a.R * a.grp;
    if (a.splits <= kSmallJoin)
      hipLaunchKernelGGL((paged_combine_kernel<HD, true>), dim3((unsigned)ceil_div(vecs * (HD / 4), kThreads)), dim3(kThreads), 0, st, a);
    else
      hipLaunchKernelGGL((paged_combine_kernel<HD, false>), dim3((unsigned)ceil_div(vecs * (HD / 4) * kJoin, kThreads)), dim3(kThreads), 0, st, a);
  }
}

}  // namespace

static void cut_call(PagedAttnArgs* a) {
  const int QV = a->R * a->grp;
  const int64_t blocks = ceil_div(QV, 32 * kWideWaves);
  const bool all = a->uncut || (QV > 16 && a->B * a->pg.hkv * blocks >= kWideBlocks);
  a->many_from = all ? 0 : QV >= kManyVectors ? kManyFrom : QV >= kSomeVectors ? kSomeFrom : INT32_MAX;
  auto cut = [&](int64_t qtiles, int64_t items, int min_chunk, int whole, int longest) {
    PagedAttnArgs::Cut t{};
    t.qtiles = (int)qtiles;
    t.max_splits = (int)std::max<int64_t>(1, items / (a->pg.hkv * qtiles));
    t.min_chunk = min_chunk;
    t.whole = whole;
    t.splits = longest <= whole ? 1 : std::min(t.max_splits, (int)ceil_div(longest, min_chunk));
    return t;
  };
  const int64_t tiles = ceil_div(QV, 16);
  a->few = cut(tiles, kTargetItems, kMinChunk, a->pg.hkv * tiles >= kManyItems ? kWholeMany : kWhole, std::min(a->max_len, a->many_from));
  a->many = cut(blocks, a->uncut ? 1 : kWideItems / (all ? std::max(a->B, kWideFew) : kWideFew), kWideChunk, kWideChunk, a->max_len);
  a->splits = std::max(a->many_from > 0 ? a->few.splits : 1, a->many_from <= a->max_len ? a->many.splits : 1);
  a->qpad = (int)align_up(QV, 16);
}

// Enough for a call of a->B sequences, a->R rows and a->max_len positions and for each with fewer of any of them, whichever
// kernel takes it and however it is cut.  A sequence has no more chunks than kSizeStep positions each, and where it has more
// than one kTargetItems workgroups of 16 vectors at most; or kWideItems / kWideFew of 128, of which a call has kWideItems where
// the many-vector kernel takes all, and elsewhere less than kWideBlocks times a sequence's chunks.
size_t paged_attn_workspace(PagedAttnArgs a, int hd) {
  constexpr int kSizeStep = 128, kBlock = 32 * kWideWaves;
  static_assert(kSizeStep <= kMinChunk && kSizeStep <= kWideChunk, "");
  if (a.max_len <= kSizeStep) return 0;
  cut_call(&a);
  const int64_t most = a.pg.hkv * ceil_div(a.max_len, kSizeStep) * a.qpad;  // of a sequence (below 2^61)
  int64_t rows = a.B * std::min<int64_t>(most, kTargetItems * 16);
  if (a.many_from == 0) rows = std::max(rows, std::min<int64_t>(a.B * std::min<int64_t>(most, kWideItems * kBlock), kWideItems * kBlock));
  if (a.R * a.grp >= kSomeVectors) {
    const int64_t one = kWideItems / kWideFew * kBlock, call = kWideBlocks * kBlock * ceil_div(kWideItems / kWideFew, a.pg.hkv * (kSomeVectors / kBlock));
    rows = std::max(rows, std::min(a.B * std::min(most, one), call));
  }
  return (size_t)rows * (hd + 2) * 4;
}

int launch_paged_attn(PagedAttnArgs a, int hd, bool e4, hipStream_t st) {
  cut_call(&a);
  a.by_grp = FastDiv(a.grp), a.by_hkv = FastDiv(a.pg.hkv), a.by_b = FastDiv(a.B), a.by_qv = FastDiv(a.R * a.grp);
  a.few.by_qtiles = FastDiv(a.few.qtiles), a.many.by_qtiles = FastDiv(a.many.qtiles);
  const int64_t blocks = align_up((int64_t)a.splits * a.B * a.pg.hkv, kXcds) * a.few.qtiles;  // (of either kernel at most)
  if (blocks >= (int64_t(1) << 31) || (int64_t)a.B * a.R * a.hq >= (int64_t(1) << 31))  // (the join's index is of 32 bits)
    return fail(SDD_EUNSUPPORTED, "%d x %d rows in one call", a.B, a.R);
  prof_begin(PROF_ATTN, st);
  if (e4) {
    if (hd == 128) launch_t<true, 128>(a, st);
    else launch_t<true, 64>(a, st);
  } else {
    if (hd == 128) launch_t<false, 128>(a, st);
    else launch_t<false, 64>(a, st);
  }
  prof_end(PROF_ATTN, st);
  return check_launch("paged_attn_kernel");
}

}  // namespace sdd

using namespace sdd;

static int attn_args(const sdd_pages* pg, int width, int B, int R, int n_q_heads, int max_len, PagedAttnArgs* a) {
  int rc = page_desc(pg, &a->pg);
  if (rc) return rc;
  SDD_REQUIRE(B > 0 && R > 0 && R <= (1 << 20) && (int64_t)B * R <= (1 << 24), "bad shape B=%d rows=%d", B, R);
  SDD_REQUIRE(n_q_heads > 0 && n_q_heads <= 65536 && n_q_heads % pg->n_kv_heads == 0, "%d query heads over %d KV heads", n_q_heads, pg->n_kv_heads);
  SDD_REQUIRE(max_len > 0 && max_len <= (1 << 30), "bad max_len %d", max_len);
  a->B = B;
  a->R = R;
  a->hq = n_q_heads;
  a->grp = n_q_heads / pg->n_kv_heads;
  a->max_len = max_len;
  SDD_REQUIRE((int64_t)R * a->grp < (1 << 28), "%d rows of %d heads", R, n_q_heads);
  return SDD_OK;
}

extern "C" int sdd_paged_attention_workspace_bytes(const sdd_pages* pg, int B, int R, int n_q_heads, int max_len, size_t* bytes) {
  SDD_REQUIRE(bytes != nullptr, "bytes is NULL");
  PagedAttnArgs a{};
  int rc = attn_args(pg, 0, B, R, n_q_heads, max_len, &a);
  if (rc) return rc;
  *bytes = paged_attn_workspace(a, pg->head_dim);
  return SDD_OK;
}

extern "C" int sdd_paged_attention(const sdd_pages* pg, const int32_t* table, int table_width, const int32_t* len, int B, int R,
                                   int n_q_heads, const uint16_t* q, float scale, int max_len, uint16_t* out, int32_t* err,
                                   void* ws, size_t ws_bytes, sdd_stream_t stream) {
  PagedAttnArgs a{};
  int rc = attn_args(pg, table_width, B, R, n_q_heads, max_len, &a);
  if (rc) return rc;
  SDD_REQUIRE(pg->pages && table && len && q && out, "NULL pointer");
  SDD_REQUIRE((uintptr_t)pg->pages % 256 == 0, "pages must be 256-byte aligned");
  SDD_REQUIRE((uintptr_t)q % 16 == 0 && (uintptr_t)out % 16 == 0, "q and out must be 16-byte aligned");
  SDD_REQUIRE(table_width > 0 && std::isfinite(scale), "bad table_width %d or scale", table_width);
  if ((int64_t)table_width * pg->page_size < max_len) a.max_len = table_width * pg->page_size;
  const size_t need = paged_attn_workspace(a, pg->head_dim);
  if (ws_bytes < need) return fail(SDD_ENOMEM, "attention workspace needs %zu bytes, got %zu", need, ws_bytes);
  SDD_REQUIRE(need == 0 || (ws && (uintptr_t)ws % 256 == 0), "workspace must be 256-byte aligned");
  a.pg.table = table;
  a.pg.width = table_width;
  a.len = len;
  a.q = q;
  a.out = out;
  a.err = err;
  a.set_scale(scale);
  a.part = reinterpret_cast<float*>(ws);
  return launch_paged_attn(a, pg->head_dim, pg->dtype == SDD_E4M3, reinterpret_cast<hipStream_t>(stream));
}
