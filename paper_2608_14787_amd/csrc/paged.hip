// Paged KV cache (gfx950): new rows into the pages (per-head RMSNorm of q and k, rotation, storage in bf16 or e4m3) and
// cached rows read back.  Stored order: paged.h.
//
// Both are streams: a row's (n_q + 2 n_kv) heads are read once, q is written once and K/V once in the cache's type; the
// rotation's cosines and sines are read from a table (angles in 64 bits when it is made: in 32 bits, position 10^5 would be
// off by 4e-3 rad at the first frequency).  Bound: the memory.  64/8 heads of 128: 4095 rows appended (168 MB, norms and
// rotation) 38 us, 4.4 TB/s where a copy of torch's runs at 4.9, and rows in fp32 (252 MB) 53 us; eight prefixes of 4001
// positions read from e4m3 pages (197 MB) 34 us, 5.8 TB/s, from bf16 (262 MB) 45 (in- and outputs changing from call to call); one
// row appended 4.4 us, read 3.2.
#include <algorithm>
#include <cmath>

#include "gemm.h"
#include "paged.h"

namespace sdd {

typedef float f32x2 __attribute__((ext_vector_type(2)));

int page_desc(const sdd_pages* pg, PageDesc* d) {
  SDD_REQUIRE(pg != nullptr, "pages description is NULL");
  SDD_REQUIRE(pg->dtype == SDD_BF16 || pg->dtype == SDD_E4M3, "paged caches hold bf16 or e4m3 (dtype %d)", pg->dtype);
  SDD_REQUIRE(pg->n_kv_heads > 0 && pg->n_kv_heads <= 1024 && pg->n_pages > 0, "bad n_kv_heads %d or n_pages %d", pg->n_kv_heads, pg->n_pages);
  if (pg->head_dim != 64 && pg->head_dim != 128) return fail(SDD_EUNSUPPORTED, "head_dim %d (64 and 128 are built)", pg->head_dim);
  int lg = 5;
  while (lg < 10 && (1 << lg) != pg->page_size) ++lg;
  SDD_REQUIRE((1 << lg) == pg->page_size, "page_size %d is no power of two in [32, 1024]", pg->page_size);
  const bool e4 = pg->dtype == SDD_E4M3;
  d->base = reinterpret_cast<char*>(pg->pages);
  d->hkv = pg->n_kv_heads;
  d->n_pages = pg->n_pages;
  d->log_page = lg;
  d->side = pg->page_size * pg->head_dim * (e4 ? 1 : 2);
  d->head_bytes = 2 * d->side + (e4 ? 2 * pg->page_size : 0);
  return SDD_OK;
}

namespace {

// A sequence's first position of this call, or -1: nothing to do (padding, or a block that does not fit).  The refusal
// is reported by the threads that ask for it.
__device__ inline int64_t block_start(const int32_t* len, int b, int R, int64_t cap, int32_t* err, bool report) {
  const int64_t p = len[b];
  if (p < 0) return -1;
  if (p + R <= cap) return p;
  if (report && err) atomicOr(err, kErrCapacity);
  return -1;
}

__device__ inline int page_of(const PageDesc& d, int row, int64_t pos, int32_t* err) {
  const int pg = d.table[(int64_t)row * d.width + (pos >> d.log_page)];
  if ((unsigned)pg < (unsigned)d.n_pages) return pg;
  if (err) atomicOr(err, kErrId);
  return -1;
}

// ---- append ----------------------------------------------------------------------------------------------

struct Start {
  int64_t pos;
  int row;
};
__device__ inline Start append_start(const AppendArgs& a, int b, bool report) {
  const int64_t cap = min((int64_t)a.pg.width << a.pg.log_page, a.rope ? (int64_t)a.max_pos : INT64_MAX);
  if (a.rows) {
    const RowInfo ri = a.rows[(int64_t)b * a.R];
    if (!ri.valid || ri.pos + (int64_t)a.R > cap) return Start{-1, 0};
    return Start{ri.pos, ri.seq};
  }
  return Start{block_start(a.len, b, a.R, cap, a.err, report), b};
}

// 8 consecutive elements of a row from element i
template <typename T>
__device__ inline void load8(const char* base, int64_t i, float* y) {
  const T* p = reinterpret_cast<const T*>(base) + i;
  if constexpr (sizeof(T) == 2) {
    unpack16(load16(p), y, T());
  } else {
    unpack16(load16(p), y, T());
    unpack16(load16(p + 4), y + 4, T());
  }
}

// 16 bytes past the caches
__device__ inline void store_nt(void* p, uint4 v) {
  __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(p));
}

// Four values already within +-448 to their nearest e4m3 codes (ties to even), value i in byte i.
__device__ inline uint32_t pack_e4m3x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// max |y|, or infinity where a value is not finite
__device__ inline float amax8(const float* y) {
  float m = 0.f, z = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    m = fmaxf(m, fabsf(y[i]));
    z = __builtin_fmaf(y[i], 0.f, z);  // 0 for finite values, NaN otherwise
  }
  return z == 0.f ? m : INFINITY;
}

// Sums / maxima over the LN lanes (4, 8 or 16, aligned) that share a head.
template <int LN, typename Op>
__device__ inline float lanes_op(float v, Op op) {
  v = op(v, dpp_f<kDppXor1>(v));
  v = op(v, dpp_f<kDppXor2>(v));
  if constexpr (LN >= 8) v = op(v, dpp_f<kDppHalfMirror>(v));
  if constexpr (LN >= 16) v = op(v, dpp_f<kDppMirror>(v));
  return v;
}

// q and k: LN = HD / 16 lanes a head, lane i holding dimensions 8 i .. 8 i + 7 and, HD / 2 further, their partners in the
// rotation, so that every access to rows, gains, table and pages is 16 bytes wide and no value changes lanes.  v: the
// lane's 8 dimensions of 8 consecutive positions, turned in registers so that its stores are 16 bytes (e4m3: 8) as well;
// groups of positions that the rows cover in part are stored position by position, their neighbours left alone.
template <typename T, bool E4, int HD>
__global__ void __launch_bounds__(256) append_kernel(AppendArgs a) {
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  constexpr auto add = [](float x, float y) { return x + y; };
  constexpr auto mx = [](float x, float y) { return fmaxf(x, y); };
  const int H = a.hq + a.pg.hkv;
  if ((int)blockIdx.x < a.n_qk) {
    constexpr int LN = HD / 16, HS = kWave / LN;  // heads of a set: one wave's
    const int sets = (H + HS - 1) / HS;
    const int item = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + wave);
    const int row = a.by_waves.div(item);
    if (row >= a.B * a.R) return;
    const int64_t m = row;
    const int b = a.by_r.div(row), r = row - b * a.R, s0 = (item - row * (int)a.by_waves.d) * a.per_wave, s1 = min(sets, s0 + a.per_wave);
    // (raw elements of the set after the one at work, so that its loads run meanwhile)
    constexpr int NV = sizeof(T) / 2;
    uint4 raw[2][NV];
    auto load_set = [&](int s) {
      const int h = min(s * HS + lane / LN, H - 1);
      const T* x = reinterpret_cast<const T*>(a.qkv) + m * a.row_stride + (int64_t)h * HD + 8 * (lane % LN);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[j][i] = load_nt16(x + j * (HD / 2) + i * 16 / (int)sizeof(T));
    };
    load_set(s0);
    const Start st = append_start(a, b, lane == 0 && s0 == 0);
    if (st.pos < 0) return;
    const int64_t pos = st.pos + r;
    const int d = 8 * (lane % LN);
    float cs[8], sn[8];
    if (a.rope) {
      const float* t = a.rope + (pos * (HD / 2) + d) * 2;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(t + 4 * i);
        cs[2 * i] = v[0], sn[2 * i] = v[1], cs[2 * i + 1] = v[2], sn[2 * i + 1] = v[3];
      }
    }
    const int page = page_of(a.pg, st.row, pos, lane == 0 && s0 == 0 ? a.err : nullptr);
    const int in_page = (int)(pos & ((1 << a.pg.log_page) - 1));
    for (int s = s0; s < s1; ++s) {
      const int h = s * HS + lane / LN;
      const bool on = h < H;  // (lanes past the last head work on it too and store nothing)
      const bool is_q = h < a.hq;
      float y[16];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < NV; ++i) unpack16(raw[j][i], y + 8 * j + i * 16 / (int)sizeof(T), T());
      load_set(min(s + 1, s1 - 1));
      const float* gain = is_q ? a.q_gain : a.k_gain;
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) ss = __builtin_fmaf(y[i], y[i], ss);
      ss = lanes_op<LN>(ss, add);
      if (gain) {
        const float inv = 1.f / sqrtf(ss / (float)HD + a.eps);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 g = *reinterpret_cast<const f32x4*>(gain + d + (j / 2) * (HD / 2) + 4 * (j % 2));
#pragma unroll
          for (int i = 0; i < 4; ++i) y[4 * j + i] *= inv * g[i];
        }
      }
      if (a.rope) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float lo = y[i], hi = y[8 + i];
          y[i] = lo * cs[i] - hi * sn[i];
          y[8 + i] = hi * cs[i] + lo * sn[i];
        }
      }
      uint4 w[2];
#pragma unroll
      for (int j = 0; j < 2; ++j)
        w[j] = make_uint4(pack_bf16x2(y[8 * j], y[8 * j + 1]), pack_bf16x2(y[8 * j + 2], y[8 * j + 3]),
                          pack_bf16x2(y[8 * j + 4], y[8 * j + 5]), pack_bf16x2(y[8 * j + 6], y[8 * j + 7]));
      if (E4 && (s + 1) * HS > a.hq) {  // a set with a k head (all its lanes take part in the exchange)
        const float am = lanes_op<LN>(fmaxf(amax8(y), amax8(y + 8)), mx);
        const bool bad = !(am < INFINITY);
        const int sb = bad ? 127 : scale_byte(am);
        const float inv = scale_value(254 - sb);
        uint2 c[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float* z = y + 8 * j;
          c[j] = bad ? make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu)
                     : make_uint2(pack_e4m3x4(z[0] * inv, z[1] * inv, z[2] * inv, z[3] * inv),
                                  pack_e4m3x4(z[4] * inv, z[5] * inv, z[6] * inv, z[7] * inv));
        }
        if (on && !is_q && page >= 0) {
          char* k = page_head(a.pg, page, h - a.hq);
          *reinterpret_cast<uint2*>(k + page_k_offset<E4, HD>(in_page, d)) = c[0];
          *reinterpret_cast<uint2*>(k + page_k_offset<E4, HD>(in_page, d + HD / 2)) = c[1];
          if (d == 0) k[2 * a.pg.side + in_page] = (char)sb;
        }
      } else if (!E4 && on && !is_q && page >= 0) {
        char* k = page_head(a.pg, page, h - a.hq);
        *reinterpret_cast<uint4*>(k + page_k_offset<E4, HD>(in_page, d)) = w[0];
        *reinterpret_cast<uint4*>(k + page_k_offset<E4, HD>(in_page, d + HD / 2)) = w[1];
      }
      if (on && is_q) {
        uint16_t* q = a.q_out + (m * a.hq + h) * HD + d;
        *reinterpret_cast<uint4*>(q) = w[0];
        *reinterpret_cast<uint4*>(q + HD / 2) = w[1];
      }
    }
    return;
  }
  // v: an item is (sequence, group of 8 positions, head), LN lanes of 8 dimensions each
  constexpr int LN = HD / 8, IT = kWave / LN;
  const int item = (((int)blockIdx.x - a.n_qk) * 4 + wave) * IT + lane / LN;
  const int bg = a.by_hkv.div(item), h = item - bg * a.pg.hkv;
  const int b = a.by_groups.div(bg), grp = bg - b * a.v_groups, d = 8 * (lane % LN);
  Start st{-1, 0};
  if (b < a.B) st = append_start(a, b, false);
  const int64_t g0 = st.pos / 8 * 8 + 8 * (int64_t)grp;  // the group's first position
  const bool on = st.pos >= 0 && g0 < st.pos + a.R;
  int page = -1;
  if (on) page = page_of(a.pg, st.row, g0, nullptr);  // (a group lies within one page)
  float y[8][8];
  int lo = 8, hi = 0;  // the group's positions that are rows of this call
  if (page >= 0) {
    lo = (int)max((int64_t)0, st.pos - g0), hi = (int)min((int64_t)8, st.pos + a.R - g0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t m = (int64_t)b * a.R + (g0 + min(max(i, lo), hi - 1) - st.pos);
      load8<T>(a.qkv, m * a.row_stride + (int64_t)(H + h) * HD + d, y[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) y[i][e] = 0.f;
  }
  const int in_page = (int)(g0 & ((1 << a.pg.log_page) - 1));
  char* v = page_head(a.pg, max(page, 0), h);
  if constexpr (E4) {
    int sb[8];
    uint32_t nan = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float am = lanes_op<LN>(amax8(y[i]), mx);
      const bool bad = !(am < INFINITY);
      sb[i] = bad ? 127 : scale_byte(am);
      nan |= bad ? 1u << i : 0u;
      const float inv = scale_value(254 - sb[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[i][e] = bad ? 0.f : y[i][e] * inv;
    }
    if (page < 0) return;
    uint32_t keep[2] = {0, 0};  // bytes of NaN rows
#pragma unroll
    for (int i = 0; i < 8; ++i) keep[i / 4] |= (nan >> i & 1) ? 0x7fu << (8 * (i % 4)) : 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t c0 = pack_e4m3x4(y[0][e], y[1][e], y[2][e], y[3][e]) | keep[0];
      const uint32_t c1 = pack_e4m3x4(y[4][e], y[5][e], y[6][e], y[7][e]) | keep[1];
      char* dst = v + a.pg.side + page_v_offset<E4, HD>(in_page, d + e);
      if (lo == 0 && hi == 8) {
        *reinterpret_cast<uint2*>(dst) = make_uint2(c0, c1);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i >= lo && i < hi) dst[i] = (char)((i < 4 ? c0 : c1) >> (8 * (i % 4)));
      }
    }
    if (d == 0)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i >= lo && i < hi) v[2 * a.pg.side + (1 << a.pg.log_page) + in_page + i] = (char)sb[i];
  } else {
    if (page < 0) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint16_t* dst = reinterpret_cast<uint16_t*>(v + a.pg.side + page_v_offset<E4, HD>(in_page, d + e));
      if (lo == 0 && hi == 8) {
        *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16x2(y[0][e], y[1][e]), pack_bf16x2(y[2][e], y[3][e]),
                                                    pack_bf16x2(y[4][e], y[5][e]), pack_bf16x2(y[6][e], y[7][e]));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i >= lo && i < hi) dst[i] = f32_to_bf16(y[i][e]);
      }
    }
  }
}

// ---- read ------------------------------------------------------------------------------------------------

struct ReadArgs {
  PageDesc pg;
  const int32_t* start;
  uint16_t *k, *v;  // [B][n][hkv][HD]
  int32_t* err;
  int B, n, groups;
};

// 8 codes to 8 floats, times s
__device__ inline void unpack_e4m3x8(uint2 c, float s, float* y) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int w = (int)(j ? c.y : c.x);
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    y[4 * j] = lo[0] * s, y[4 * j + 1] = lo[1] * s, y[4 * j + 2] = hi[0] * s, y[4 * j + 3] = hi[1] * s;
  }
}

// An item is (sequence, group of 8 positions, head); LN = HD / 8 lanes, 8 dimensions each.  K: position by position, 16
// bytes out of (e4m3: 8) and into place.  V: the lane's 8 dimensions of all 8 positions, turned in registers.  Stored past the
// caches (eight prefixes of 4001 positions, bf16: 45 us, 52 with ordinary stores).
template <bool E4, int HD>
__global__ void __launch_bounds__(256) read_kernel(ReadArgs a) {
  constexpr int LN = HD / 8;
  const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LN;
  const int lane = threadIdx.x % LN, d = 8 * lane;
  const int h = (int)(item % a.pg.hkv);
  const int64_t bg = item / a.pg.hkv;
  const int b = (int)(bg / a.groups), grp = (int)(bg % a.groups);
  if (b >= a.B) return;
  const int64_t pos = block_start(a.start, b, a.n, (int64_t)a.pg.width << a.pg.log_page, a.err, lane == 0 && h == 0 && grp == 0);
  if (pos < 0) return;
  const int64_t g0 = pos / 8 * 8 + 8 * (int64_t)grp;
  if (g0 >= pos + a.n) return;
  const int lo = (int)max((int64_t)0, pos - g0), hi = (int)min((int64_t)8, pos + a.n - g0);
  const int page = page_of(a.pg, b, g0, lane == 0 && h == 0 ? a.err : nullptr);
  const int in_page = (int)(g0 & ((1 << a.pg.log_page) - 1));
  const int64_t o0 = (((int64_t)b * a.n + (g0 - pos)) * a.pg.hkv + h) * HD + d;  // of position g0 (may lie before the output)
  const int64_t ostep = (int64_t)a.pg.hkv * HD;
  if (page < 0) {
    for (int i = lo; i < hi; ++i) {
      *reinterpret_cast<uint4*>(a.k + o0 + i * ostep) = make_uint4(0, 0, 0, 0);
      *reinterpret_cast<uint4*>(a.v + o0 + i * ostep) = make_uint4(0, 0, 0, 0);
    }
    return;
  }
  const char* p = page_head(a.pg, page, h);
  const int PS = 1 << a.pg.log_page;
  auto pack = [](const float* y) {
    return make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
  };
  if constexpr (E4) {
    uint2 kc[8], vc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) kc[i] = *reinterpret_cast<const uint2*>(p + page_k_offset<E4, HD>(in_page + i, d));
#pragma unroll
    for (int e = 0; e < 8; ++e) vc[e] = *reinterpret_cast<const uint2*>(p + a.pg.side + page_v_offset<E4, HD>(in_page, d + e));
    const uint2 ks = *reinterpret_cast<const uint2*>(p + 2 * a.pg.side + in_page);
    const uint2 vs = *reinterpret_cast<const uint2*>(p + 2 * a.pg.side + PS + in_page);
    float vt[8][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) unpack_e4m3x8(vc[e], 1.f, vt[e]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int sh = 8 * (i % 4);
      float y[8];
      unpack_e4m3x8(kc[i], scale_value(((i < 4 ? ks.x : ks.y) >> sh) & 255), y);
      const float s = scale_value(((i < 4 ? vs.x : vs.y) >> sh) & 255);
      float z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = vt[e][i] * s;
      if (i >= lo && i < hi) {
        store_nt(a.k + o0 + i * ostep, pack(y));
        store_nt(a.v + o0 + i * ostep, pack(z));
      }
    }
  } else {
    uint4 kc[8], vc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) kc[i] = load16(p + page_k_offset<E4, HD>(in_page + i, d));
#pragma unroll
    for (int e = 0; e < 8; ++e) vc[e] = load16(p + a.pg.side + page_v_offset<E4, HD>(in_page, d + e));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint4 &x = vc[2 * j], &y = vc[2 * j + 1];
        const uint32_t xw = i / 2 == 0 ? x.x : i / 2 == 1 ? x.y : i / 2 == 2 ? x.z : x.w;
        const uint32_t yw = i / 2 == 0 ? y.x : i / 2 == 1 ? y.y : i / 2 == 2 ? y.z : y.w;
        w[j] = i % 2 ? (xw >> 16) | (yw & 0xffff0000u) : (xw & 0xffffu) | (yw << 16);
      }
      if (i >= lo && i < hi) {
        store_nt(a.k + o0 + i * ostep, kc[i]);
        store_nt(a.v + o0 + i * ostep, make_uint4(w[0], w[1], w[2], w[3]));
      }
    }
  }
}

__global__ void rope_table_kernel(float* t, int64_t n, int half, double theta) {
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
    const double ang = (double)(i / half) * pow(theta, -2.0 * (double)(i % half) / (2.0 * half));
    t[2 * i] = (float)cos(ang);
    t[2 * i + 1] = (float)sin(ang);
  }
}

template <typename T, bool E4>
void launch_append_t(const AppendArgs& a, int hd, int blocks, hipStream_t st) {
  if (hd == 128)
    hipLaunchKernelGGL((append_kernel<T, E4, 128>), dim3(blocks), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((append_kernel<T, E4, 64>), dim3(blocks), dim3(256), 0, st, a);
}

}  // namespace

int launch_paged_append(AppendArgs a, int hd, bool e4, bool f32, hipStream_t st) {
  const int H = a.hq + a.pg.hkv, hs = kWave / (hd / 16), sets = (int)ceil_div(H, hs);
  const int64_t rows = (int64_t)a.B * a.R;
  // one set of heads per wave while the waves are few (latency); three, the table's loads serving them all, up to what fills
  // the device; all of a row's beyond.  Measured, 64/8 heads of 128 (9 sets), bf16, sets a wave 1, 3, 9: 264 rows 6.8, 5.7, 6.6 us;
  // 1024 rows 15.1, 15.2, 17.6 (e4m3 pages 15.3, 11.8, 16.9); 4095 rows 48, 40, 38
  a.per_wave = rows * sets <= 1024 ? 1 : std::min(sets, rows <= 2560 ? 3 : sets);
  const int64_t waves = rows * ceil_div(sets, a.per_wave);
  a.v_groups = (int)((a.R + 14) / 8);
  const int64_t v_items = (int64_t)a.B * a.v_groups * a.pg.hkv, per = kWave / (hd / 8);
  const int64_t nqk = ceil_div(waves, 4), nv = ceil_div(v_items, 4 * per);
  if (std::max(4 * nqk, nv * 4 * per) >= (int64_t(1) << 31)) return fail(SDD_EUNSUPPORTED, "%lld rows in one call", (long long)rows);
  a.n_qk = (int)nqk;
  a.by_waves = FastDiv((uint32_t)ceil_div(sets, a.per_wave)), a.by_r = FastDiv(a.R);
  a.by_hkv = FastDiv(a.pg.hkv), a.by_groups = FastDiv(a.v_groups);
  const int blocks = (int)(nqk + nv);
  prof_begin(PROF_PAGES, st);
  if (f32) {
    if (e4) launch_append_t<float, true>(a, hd, blocks, st);
    else launch_append_t<float, false>(a, hd, blocks, st);
  } else {
    if (e4) launch_append_t<uint16_t, true>(a, hd, blocks, st);
    else launch_append_t<uint16_t, false>(a, hd, blocks, st);
  }
  prof_end(PROF_PAGES, st);
  return check_launch("append_kernel");
}

}  // namespace sdd

using namespace sdd;

extern "C" int sdd_pages_bytes(const sdd_pages* pg, size_t* bytes) {
  SDD_REQUIRE(bytes != nullptr, "bytes is NULL");
  PageDesc d;
  int rc = page_desc(pg, &d);
  if (rc) return rc;
  *bytes = (size_t)d.n_pages * d.hkv * d.head_bytes;
  return SDD_OK;
}

extern "C" int sdd_rope_table(float* table, int max_pos, int head_dim, float theta, sdd_stream_t stream) {
  SDD_REQUIRE(table != nullptr, "table is NULL");
  SDD_REQUIRE(max_pos > 0 && head_dim > 0 && head_dim % 2 == 0 && theta > 0.f && std::isfinite(theta),
              "bad max_pos %d, head_dim %d or theta", max_pos, head_dim);
  const int64_t n = (int64_t)max_pos * (head_dim / 2);
  hipLaunchKernelGGL(rope_table_kernel, dim3((int)std::min<int64_t>(ceil_div(n, 256), 8192)), dim3(256), 0,
                     reinterpret_cast<hipStream_t>(stream), table, n, head_dim / 2, (double)theta);
  return check_launch("rope_table_kernel");
}

// What every operator on a pool asks of its arguments.
static int pool_args(const sdd_pages* pg, const int32_t* table, int width, const int32_t* len, int B, int R, PageDesc* d) {
  int rc = page_desc(pg, d);
  if (rc) return rc;
  SDD_REQUIRE(pg->pages && table && len, "NULL pointer");
  SDD_REQUIRE((uintptr_t)pg->pages % 256 == 0, "pages must be 256-byte aligned");
  SDD_REQUIRE(B > 0 && R > 0 && R <= (1 << 24) && (int64_t)B * R <= (1 << 30) && width > 0, "bad shape B=%d rows=%d table_width=%d", B, R, width);
  d->table = table;
  d->width = width;
  return SDD_OK;
}

extern "C" int sdd_paged_append(const sdd_pages* pg, const int32_t* table, int table_width, const int32_t* len, int B,
                                int R, int n_q_heads, const void* qkv, int qkv_dtype, size_t row_stride,
                                const float* q_gain, const float* k_gain, float eps, const float* rope, int max_pos,
                                uint16_t* q_out, int32_t* err, sdd_stream_t stream) {
  AppendArgs a{};
  int rc = pool_args(pg, table, table_width, len, B, R, &a.pg);
  if (rc) return rc;
  SDD_REQUIRE(qkv && q_out, "NULL pointer");
  SDD_REQUIRE(qkv_dtype == SDD_F32 || qkv_dtype == SDD_BF16, "bad qkv dtype %d", qkv_dtype);
  SDD_REQUIRE(n_q_heads > 0 && n_q_heads <= 65536 && n_q_heads % pg->n_kv_heads == 0, "%d query heads over %d KV heads", n_q_heads, pg->n_kv_heads);
  SDD_REQUIRE(row_stride >= (size_t)(n_q_heads + 2 * pg->n_kv_heads) * pg->head_dim, "row_stride %zu is shorter than a row", row_stride);
  const size_t es = qkv_dtype == SDD_F32 ? 4 : 2;
  SDD_REQUIRE((uintptr_t)qkv % 16 == 0 && row_stride * es % 16 == 0, "qkv rows must be 16-byte aligned");
  SDD_REQUIRE((uintptr_t)q_out % 16 == 0 && (uintptr_t)q_gain % 16 == 0 && (uintptr_t)k_gain % 16 == 0 && (uintptr_t)rope % 16 == 0,
              "q_out, gains and rope must be 16-byte aligned");
  SDD_REQUIRE((q_gain == nullptr) == (k_gain == nullptr), "gains of q and k come together");
  SDD_REQUIRE(!q_gain || eps >= 0.f, "bad eps");
  SDD_REQUIRE(!rope || max_pos > 0, "a rotation table of %d positions", max_pos);
  a.len = len;
  a.qkv = reinterpret_cast<const char*>(qkv);
  a.row_stride = (int64_t)row_stride;
  a.q_gain = q_gain;
  a.k_gain = k_gain;
  a.rope = rope;
  a.q_out = q_out;
  a.err = err;
  a.B = B;
  a.R = R;
  a.hq = n_q_heads;
  a.max_pos = max_pos;
  a.eps = eps;
  return launch_paged_append(a, pg->head_dim, pg->dtype == SDD_E4M3, qkv_dtype == SDD_F32, reinterpret_cast<hipStream_t>(stream));
}

extern "C" int sdd_paged_read(const sdd_pages* pg, const int32_t* table, int table_width, const int32_t* start, int B, int n,
                              uint16_t* k, uint16_t* v, int32_t* err, sdd_stream_t stream) {
  ReadArgs a{};
  int rc = pool_args(pg, table, table_width, start, B, n, &a.pg);
  if (rc) return rc;
  SDD_REQUIRE(k && v, "NULL pointer");
  SDD_REQUIRE((uintptr_t)k % 16 == 0 && (uintptr_t)v % 16 == 0, "k and v must be 16-byte aligned");
  a.start = start;
  a.k = k;
  a.v = v;
  a.err = err;
  a.B = B;
  a.n = n;
  a.groups = (int)(((int64_t)n + 14) / 8);
  const int hd = pg->head_dim;
  const int64_t blocks = ceil_div((int64_t)B * a.groups * pg->n_kv_heads * (hd / 8), 256);
  if (blocks >= (int64_t(1) << 31)) return fail(SDD_EUNSUPPORTED, "%d x %d positions in one call", B, n);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)blocks);
  prof_begin(PROF_PAGES, st);
  if (pg->dtype == SDD_E4M3) {
    if (hd == 128) hipLaunchKernelGGL((read_kernel<true, 128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((read_kernel<true, 64>), grid, dim3(256), 0, st, a);
  } else {
    if (hd == 128) hipLaunchKernelGGL((read_kernel<false, 128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((read_kernel<false, 64>), grid, dim3(256), 0, st, a);
  }
  prof_end(PROF_PAGES, st);
  return check_launch("read_kernel");
}
