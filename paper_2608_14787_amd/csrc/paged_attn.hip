// Attention of new rows over a paged KV cache (gfx950): R rows of each of B sequences, the sequence's own K/V of those
// rows already in its pages (bf16 or e4m3), row r at position len + r and seeing the positions up to its own.
//
// For a query vector q (row, head) over the visible positions p: s_p = scale q.k_p, w_p = e^(s_p - m), o = sum w_p v_p / sum w_p,
// in one pass with the running maximum m, sum and accumulator in fp32 (exponentials of base 2, scale holding log2 e).  The
// weights are rounded to bf16 for the second product, as V is held in bf16 or less; their sum takes them before that rounding.
//
// A workgroup takes 16 query vectors of one KV head (rows x the heads that share it) over one chunk of the sequence; its
// four waves take the chunk's 32-position steps round-robin and are joined through LDS in wave order, and the chunks'
// results by combine_kernel in chunk order.  The cut into chunks depends on the sequence's own length alone.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "gemm.h"
#include "paged.h"

namespace sdd {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kMinChunk = 256;      // positions: two steps a wave
constexpr int kTargetItems = 512;   // workgroups a sequence is cut into at most

__host__ __device__ inline int chunk_of(int total, int max_splits) {
  const int c = (total + max_splits - 1) / max_splits;
  return max(kMinChunk, (c + 127) / 128 * 128);
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

__device__ inline void store_out4(const PagedAttnArgs& a, int b, int r, int h, int HD, int dim, const float* y) {
  const int row = b * a.R + r;
  const int64_t at = a.frag ? xfrag_index<uint16_t>(row, h * HD + dim, a.hq * HD / 32) : ((int64_t)row * a.hq + h) * HD + dim;
  *reinterpret_cast<uint2*>(a.out + at) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
}

// Four e4m3 codes of a word to bf16.
__device__ inline void unpack_e4m3(uint32_t w, bf16x2& lo, bf16x2& hi) {
  lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, true);
}
__device__ inline bf16x8 e4m3_frag(uint32_t x, uint32_t y) {
  bf16x2 a, b, c, d;
  unpack_e4m3(x, a, b);
  unpack_e4m3(y, c, d);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ inline uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

template <bool E4, int HD>
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
  const int group = a.by_qtiles.div(rest), qt = rest - group * a.qtiles, item = group * kXcds + low;
  if (item >= a.splits * a.B * hkv) return;
  const int bc = a.by_hkv.div(item), kvh = item - bc * hkv, c = a.by_b.div(bc), b = bc - c * a.B;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const Seq sq = attn_seq(a, b, threadIdx.x == 0 && c == 0 && kvh == 0 && qt == 0);
  if (sq.pos < 0) return;
  const int total = sq.pos + a.R, chunk = chunk_of(total, a.max_splits), n_chunks = (total + chunk - 1) / chunk;
  if (c >= n_chunks) return;
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
    q_frag = load16(Q + (E4 ? 64 * (wave / 2) + 16 * (lane / 16) + 8 * (wave % 2) : 32 * wave + g8));
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
  uint2 ks = {0, 0}, vs = {0, 0};
  auto load = [&](const Place& pl, int off) {
    // (non-temporal: a decode step reads a position once)
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(pl.page, lane * 16, off, kNtCpol));
  };
  auto load_scales = [&](const Place& pl, int off) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(pl.page, g8, off, 0);
    return make_uint2(v[0], v[1]);
  };
  auto load_k = [&](const Place& pl) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < NK; ++j) kr[s][j] = load(pl, pl.in * HD * (E4 ? 1 : 2) + (s * NK + j) * 1024);
    if constexpr (E4) ks = load_scales(pl, 2 * a.pg.side + pl.in);
  };
  auto load_v = [&](const Place& pl) {
#pragma unroll
    for (int j = 0; j < NV; ++j) vr[j] = load(pl, a.pg.side + pl.in * HD * (E4 ? 1 : 2) + j * 1024);
    if constexpr (E4) vs = load_scales(pl, 2 * a.pg.side + (1 << lg) + pl.in);
  };

  f32x4 o[DB];
  float m, l;
  bool wild;
  auto reset = [&]() {
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY, l = 0.f, wild = false;
  };
  reset();
  // V operand of 16 dimensions, positions outside `mask` (a bit for each of the lane's 8) zeroed: their weights are 0, and 0
  // times a stale or foreign non-finite value would not be
  auto v_frag = [&](int db, uint32_t mask) {
    if constexpr (E4) {
      uint32_t x = word(vr[db / 2], db % 2 * 2), y = word(vr[db / 2], db % 2 * 2 + 1);
      if (mask != 255) {  // (lane by lane: no product in here)
        uint32_t mx = 0, my = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          mx |= (mask >> i & 1) ? 0xffu << (8 * i) : 0u;
          my |= (mask >> (4 + i) & 1) ? 0xffu << (8 * i) : 0u;
        }
        x &= mx, y &= my;
      }
      return e4m3_frag(x, y);
    } else {
      uint4 w = vr[db];
      if (mask != 255) {
        uint32_t k[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          k[i] = ((mask >> (2 * i) & 1) ? 0xffffu : 0u) | ((mask >> (2 * i + 1) & 1) ? 0xffff0000u : 0u);
        w.x &= k[0], w.y &= k[1], w.z &= k[2], w.w &= k[3];
      }
      return __builtin_bit_cast(bf16x8, w);
    }
  };
  auto below = [&](int p, int end) {  // mask of the lane's positions of step p that lie before end
    const int n = max(0, min(8, end - (p + g8)));
    return (1u << n) - 1u;
  };
  constexpr int kStride = 32 * kWaves;
  const int p0 = p_begin + 32 * wave;
  Place pl;
  // Step p, whose place is pl; issues the next one's loads.  ONE: every query vector's product by itself, V zeroed where it is
  // hidden from it.
  auto step = [&](auto one, int p) {
    const bool ok = pl.ok;
    f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < KK; ++i) {
      const bf16x8 q = *reinterpret_cast<const bf16x8*>(s_q + i * 1024 + lane * 16);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        bf16x8 k;
        if constexpr (E4)
          k = e4m3_frag(word(kr[t][i / 2], i % 2 * 2), word(kr[t][i / 2], i % 2 * 2 + 1));
        else
          k = __builtin_bit_cast(bf16x8, kr[t][i]);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q, s[t], 0, 0, 0);
      }
    }
    // s[i / 4][i % 4]: position p + g8 + i, query vector lane % 16
    float sv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sv[i] = s[i / 4][i % 4] * a.scale;
      if constexpr (E4) sv[i] *= scale_value(((i < 4 ? ks.x : ks.y) >> (8 * (i % 4))) & 255);
    }
    // K's registers are free: the next step's loads go out ahead of this one's softmax, V's after its product
    pl = place(p + kStride);
    load_k(pl);
    __builtin_amdgcn_sched_barrier(0);
    const bool whole = p + 32 <= p_end && ok;  // (the same in every lane: products run with all of them)
    if (p + 31 > lo || !whole) {
      const int end = ok ? min(qpos + 1, p_end) : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) sv[i] = p + g8 + i < end ? sv[i] : -INFINITY;
    }
    float top = sv[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, sv[i]);
    top = xor16_op(top, [](float x, float y) { return fmaxf(x, y); });
    top = xor32_op(top, [](float x, float y) { return fmaxf(x, y); });
    const float mn = fmaxf(m, top);
    if (__any(mn != m)) {
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      l *= f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= f;
      m = mn;
    }
    const float ref = m == -INFINITY ? 0.f : m;  // (a hidden score's weight is then exp2(-inf) = 0)
    float e[8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e[i] = __builtin_amdgcn_exp2f(sv[i] - ref);
      sum += e[i];
    }
    l += sum;
    if constexpr (E4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = e[i] * scale_value(((i < 4 ? vs.x : vs.y) >> (8 * (i % 4))) & 255);
        e[i] = sv[i] == -INFINITY ? 0.f : x;  // (a position that was never written may have any scale byte)
      }
    }
    const bf16x8 pf = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]),
                                                            pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])));
    if constexpr (decltype(one)::value) {
#pragma unroll 1
      for (int q = 0; q < 16; ++q) {
        const uint32_t seen = below(p, ok ? min(p_end, __builtin_amdgcn_readlane(qpos, q) + 1) : 0);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_frag(db, seen), pf, o[db], 0, 0, 0);
          if (lane % 16 == q) o[db] = y;  // (a product's columns are independent: the others are not taken)
        }
      }
    } else if (whole && p + 31 <= lo) {
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_frag(db, 255), pf, o[db], 0, 0, 0);
    } else {
      const uint32_t mask = below(p, ok ? p_end : 0);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 v = v_frag(db, mask);
#pragma unroll
        for (int i = 0; i < 8; ++i) wild |= !__builtin_isfinite((float)v[i]);
        o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf, o[db], 0, 0, 0);
      }
    }
  };
  auto steps = [&](auto one) {
    pl = place(p0);
    load_k(pl);
    load_v(pl);
    if constexpr (!decltype(one)::value) {
      if (wave < KK) *reinterpret_cast<uint4*>(s_q + wave * 1024 + lane * 16) = q_frag;
      __syncthreads();  // the queries are in LDS
    }
#pragma unroll 1
    for (int p = p0; p < p_end; p += kStride) {
      step(one, p);
      __builtin_amdgcn_sched_barrier(0);
      load_v(pl);
    }
  };
  steps(std::false_type{});
  // On the tile's diagonal a position may be hidden from some of the query vectors only.  Where a V value there is not finite,
  // the zero weight of those vectors has not kept it out: the wave's steps again, each vector's product by itself.
  if (lo + 1 < tile_end && __any(wild)) {
    reset();
    page0 = p_begin >> lg;
    load_ids();
    steps(std::true_type{});
  }
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
  const int64_t slot = ((int64_t)(b * hkv + kvh) * a.qtiles + qt) * a.splits + c;
  float* part_o = a.part + slot * 16 * HD;
  float* part_ml = a.part + (int64_t)a.B * hkv * a.qtiles * a.splits * 16 * HD + slot * 32;
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

// Joins the chunks of a query vector: kJoin groups of HD / 4 lanes (4 dimensions a lane) take the chunks g, g + kJoin, ... in
// order, several loads in flight, and are added in order of g.  A workgroup holds kThreads / (kJoin HD / 4) query vectors.
constexpr int kJoin = 4;
template <int HD>
__global__ void __launch_bounds__(kThreads) paged_combine_kernel(PagedAttnArgs a) {
  constexpr int LN = HD / 4, VEC = kThreads / (LN * kJoin), U = 4;
  __shared__ __align__(16) float s_y[kThreads][4];
  __shared__ float s_l[kThreads / LN];
  const int grp = threadIdx.x / LN, g = grp % kJoin, ln = threadIdx.x % LN, d = 4 * ln, QV = a.R * a.grp;
  const int64_t idx = (int64_t)blockIdx.x * VEC + grp / kJoin, bh = idx / QV;
  const int qv = (int)(idx % QV), b = (int)(bh / a.pg.hkv), kvh = (int)(bh % a.pg.hkv);
  Seq sq{-1, 0};
  if (b < a.B) sq = attn_seq(a, b, false);
  const int total = sq.pos + a.R, chunk = chunk_of(total, a.max_splits), n = sq.pos < 0 ? 1 : (total + chunk - 1) / chunk;
  float y[4] = {0.f, 0.f, 0.f, 0.f}, L = 0.f;
  if (n > 1) {
    const int64_t slot = (bh * a.qtiles + qv / 16) * a.splits;
    const float* o = a.part + (slot * 16 + qv % 16) * HD + d;
    const float* ml = a.part + (int64_t)a.B * a.pg.hkv * a.qtiles * a.splits * 16 * HD + (slot * 16 + qv % 16) * 2;
    float M = -INFINITY;
    for (int c = ln; c < n; c += LN) M = fmaxf(M, ml[32 * c]);
#pragma unroll
    for (int k = 1; k < LN; k *= 2) M = fmaxf(M, __shfl_xor(M, k));
    for (int c0 = g; c0 < n; c0 += kJoin * U) {
      f32x4 v[U];
      float mc[U], lc[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = min(c0 + kJoin * u, n - 1);
        mc[u] = ml[32 * c], lc[u] = ml[32 * c + 1];
        v[u] = *reinterpret_cast<const f32x4*>(o + (int64_t)c * 16 * HD);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (c0 + kJoin * u >= n) break;
        const float f = mc[u] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mc[u] - M);
        L += f * lc[u];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] += f * v[u][i];
      }
    }
  }
  *reinterpret_cast<f32x4*>(s_y[threadIdx.x]) = f32x4{y[0], y[1], y[2], y[3]};
  if (ln == 0) s_l[grp] = L;
  __syncthreads();
  if (g != 0 || n == 1) return;
#pragma unroll
  for (int k = 1; k < kJoin; ++k) {
    L += s_l[grp + k];
    const f32x4 v = *reinterpret_cast<const f32x4*>(s_y[threadIdx.x + k * LN]);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] += v[i];
  }
  const float inv = 1.f / L;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = L == 0.f ? 0.f : y[i] * inv;
  store_out4(a, b, qv / a.grp, kvh * a.grp + qv % a.grp, HD, d, y);
}

template <bool E4, int HD>
void launch_t(const PagedAttnArgs& a, hipStream_t st) {
  const int64_t items = (int64_t)a.splits * a.B * a.pg.hkv;
  hipLaunchKernelGGL((paged_attn_kernel<E4, HD>), dim3((unsigned)(ceil_div(items, kXcds) * kXcds * a.qtiles)), dim3(kThreads), 0, st, a);
  if (a.splits > 1) {
    const int64_t vecs = (int64_t)a.B * a.pg.hkv * a.R * a.grp;
    hipLaunchKernelGGL((paged_combine_kernel<HD>), dim3((unsigned)ceil_div(vecs * (HD / 4) * kJoin, kThreads)), dim3(kThreads), 0, st, a);
  }
}

}  // namespace

// The cut of a call: chunks per sequence at most, and those that a sequence of max_len positions has.
static void attn_splits(PagedAttnArgs* a) {
  a->qtiles = (int)ceil_div((int64_t)a->R * a->grp, 16);
  a->max_splits = std::max(1, kTargetItems / std::max(1, std::min(kTargetItems, a->pg.hkv * a->qtiles)));
  a->splits = std::min(a->max_splits, (int)ceil_div(a->max_len, kMinChunk));
}

size_t paged_attn_workspace(PagedAttnArgs a, int hd) {
  attn_splits(&a);
  if (a.splits == 1) return 0;
  return (size_t)a.B * a.pg.hkv * a.qtiles * a.splits * 16 * (hd + 2) * 4;
}

int launch_paged_attn(PagedAttnArgs a, int hd, bool e4, hipStream_t st) {
  attn_splits(&a);
  a.by_grp = FastDiv(a.grp), a.by_hkv = FastDiv(a.pg.hkv), a.by_b = FastDiv(a.B), a.by_qtiles = FastDiv(a.qtiles);
  const int64_t blocks = (ceil_div((int64_t)a.splits * a.B * a.pg.hkv, kXcds) * kXcds) * a.qtiles;
  if (blocks >= (int64_t(1) << 31) || (int64_t)a.B * a.R * a.hq * hd / 4 * 4 / 256 >= (int64_t(1) << 31))
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
  a.scale = scale * kLog2e;
  a.part = reinterpret_cast<float*>(ws);
  return launch_paged_attn(a, pg->head_dim, pg->dtype == SDD_E4M3, reinterpret_cast<hipStream_t>(stream));
}
