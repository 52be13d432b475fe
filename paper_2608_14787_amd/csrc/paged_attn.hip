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

#include "gemm.h"
#include "paged.h"

namespace sdd {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kMinChunk = 128;      // positions: one step a wave
constexpr int kTargetItems = 512;   // workgroups a sequence is cut into at most

__host__ __device__ inline int chunk_of(int total, int max_splits) {
  const int c = (total + max_splits - 1) / max_splits;
  return max(kMinChunk, (c + kMinChunk - 1) / kMinChunk * kMinChunk);
}

struct Seq {
  int pos, row;  // position of the block's row 0 (-1: nothing to do), row of the table
};
__device__ inline Seq attn_seq(const PagedAttnArgs& a, int b, bool report) {
  if (a.rows) {
    const RowInfo ri = a.rows[(int64_t)b * a.R];
    return Seq{ri.valid && ri.pos + a.R <= a.max_len ? ri.pos : -1, ri.seq};
  }
  const int p = a.len[b];
  if (p >= 0 && (int64_t)p + a.R > a.max_len) {
    if (report && a.err) atomicOr(a.err, kErrCapacity);
    return Seq{-1, b};
  }
  return Seq{p < 0 ? -1 : p, b};
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

// One step's operands (32 positions): K blocks, V blocks, e4m3 scale bytes of the lane's 8 positions.
template <bool E4, int HD>
struct StepRegs {
  static constexpr int NK = E4 ? HD / 64 : HD / 32, NV = E4 ? HD / 32 : HD / 16;
  uint4 k[2][NK], v[NV];
  uint2 ks, vs;
  bool ok;  // the page exists
};

template <bool E4, int HD>
__global__ void __launch_bounds__(kThreads) paged_attn_kernel(PagedAttnArgs a) {
  constexpr int KK = HD / 32, DB = HD / 16;
  using Regs = StepRegs<E4, HD>;
  __shared__ __align__(16) float s_o[kWaves][16][HD + 4];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  const int hkv = a.pg.hkv;
  // workgroups go to the XCDs round-robin by id: the query tiles of one (chunk, sequence, head) share an XCD's L2
  const int low = blockIdx.x % kXcds, rest = blockIdx.x / kXcds;
  const int qt = rest % a.qtiles, item = rest / a.qtiles * kXcds + low;
  if (item >= a.splits * a.B * hkv) return;
  const int kvh = item % hkv, b = item / hkv % a.B, c = item / hkv / a.B;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const Seq sq = attn_seq(a, b, threadIdx.x == 0 && c == 0 && kvh == 0 && qt == 0);
  if (sq.pos < 0) return;
  const int total = sq.pos + a.R, chunk = chunk_of(total, a.max_splits), n_chunks = (total + chunk - 1) / chunk;
  if (c >= n_chunks) return;
  const int QV = a.R * a.grp, qv = qt * 16 + lane % 16;
  const bool qok = qv < QV;
  const int r = qok ? qv / a.grp : 0, hh = qok ? qv % a.grp : 0;
  const int qpos = qok ? sq.pos + r : -1;
  const int lo = sq.pos + qt * 16 / a.grp;  // position of the tile's first row
  const int tile_end = sq.pos + min(a.R - 1, (qt * 16 + 15) / a.grp) + 1;
  const int p_begin = c * chunk, p_end = min(tile_end, p_begin + chunk);

  uint4 qf[KK];  // fragment i: the 8 dimensions that the i-th K operand of a step holds
  {
    const uint16_t* Q = a.q + ((int64_t)(b * a.R + r) * a.hq + kvh * a.grp + hh) * HD;
#pragma unroll
    for (int i = 0; i < KK; ++i)
      qf[i] = load16(Q + (E4 ? 64 * (i / 2) + 16 * (lane / 16) + 8 * (i % 2) : 32 * i + 8 * (lane / 16)));
  }
  const int g8 = 8 * (lane / 16);
  // the chunk's page ids, 64 at a time across the lanes
  const int lg = a.pg.log_page;
  int page0 = p_begin >> lg, ids = 0;
  auto load_ids = [&]() { ids = a.pg.table[(int64_t)sq.row * a.pg.width + min(page0 + lane, a.pg.width - 1)]; };
  load_ids();
  bool bad_page = false;
  auto load_step = [&](int p, Regs& st) {
    int i = (p >> lg) - page0;
    if (i >= kWave) {
      page0 += kWave;
      load_ids();
      i -= kWave;
    }
    const int id = __builtin_amdgcn_readlane(ids, i);
    st.ok = (unsigned)id < (unsigned)a.pg.n_pages;
    bad_page |= !st.ok;
    const int in = p & ((1 << lg) - 1);
    const char* base = page_head(a.pg, st.ok ? id : 0, kvh);
    const char* k = base + in * HD * (E4 ? 1 : 2) + lane * 16;
    const char* v = k + a.pg.side;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < Regs::NK; ++j) st.k[s][j] = load16(k + (s * Regs::NK + j) * 1024);
#pragma unroll
    for (int j = 0; j < Regs::NV; ++j) st.v[j] = load16(v + j * 1024);
    if constexpr (E4) {
      st.ks = *reinterpret_cast<const uint2*>(base + 2 * a.pg.side + in + g8);
      st.vs = *reinterpret_cast<const uint2*>(base + 2 * a.pg.side + (1 << lg) + in + g8);
    }
  };

  f32x4 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  // V operand of 16 dimensions, positions outside `mask` (a bit for each of the lane's 8) zeroed: their weights are 0, and 0
  // times a stale or foreign non-finite value would not be
  auto v_frag = [&](const Regs& st, int db, uint32_t mask) {
    if constexpr (E4) {
      uint32_t x = word(st.v[db / 2], db % 2 * 2), y = word(st.v[db / 2], db % 2 * 2 + 1);
      if (mask != 255) {
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
      uint4 v = st.v[db];
      if (mask != 255) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = ((mask >> (2 * i) & 1) ? 0xffffu : 0u) | ((mask >> (2 * i + 1) & 1) ? 0xffff0000u : 0u);
        v.x &= w[0], v.y &= w[1], v.z &= w[2], v.w &= w[3];
      }
      return __builtin_bit_cast(bf16x8, v);
    }
  };
  auto below = [&](int p, int end) {  // mask of the lane's positions of step p that lie before end
    const int n = max(0, min(8, end - (p + g8)));
    return (1u << n) - 1u;
  };
  auto step = [&](int p, const Regs& st) {
    f32x4 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KK; ++i) {
        bf16x8 k;
        if constexpr (E4)
          k = e4m3_frag(word(st.k[t][i / 2], i % 2 * 2), word(st.k[t][i / 2], i % 2 * 2 + 1));
        else
          k = __builtin_bit_cast(bf16x8, st.k[t][i]);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, __builtin_bit_cast(bf16x8, qf[i]), s[t], 0, 0, 0);
      }
    }
    // s[i / 4][i % 4]: position p + g8 + i, query vector lane % 16
    float sv[8];
    float top = -INFINITY;
    const int end = st.ok ? min(qpos + 1, p_end) : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v = s[i / 4][i % 4] * a.scale;
      if constexpr (E4) v *= scale_value(((i < 4 ? st.ks.x : st.ks.y) >> (8 * (i % 4))) & 255);
      sv[i] = p + g8 + i < end ? v : -INFINITY;
      top = fmaxf(top, sv[i]);
    }
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
    float e[8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e[i] = sv[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sv[i] - mn);
      sum += e[i];
      if constexpr (E4) e[i] *= sv[i] == -INFINITY ? 0.f : scale_value(((i < 4 ? st.vs.x : st.vs.y) >> (8 * (i % 4))) & 255);
    }
    l += sum;
    const bf16x8 pf = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]),
                                                            pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])));
    const uint32_t mask = below(p, st.ok ? p_end : 0);
    bf16x8 vf[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) vf[db] = v_frag(st, db, mask);
    // Steps on the tile's diagonal: a position may be hidden from some of the query vectors only.  Where its V is not finite,
    // their zero weights would not keep it out; then every query vector's product leaves out what is hidden from it.
    if (p + 31 > lo && lo + 1 < tile_end) {
      bool wild = false;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 8; ++i) wild |= !__builtin_isfinite((float)vf[db][i]);
      if (__any(wild)) {
        for (int q = 0; q < 16; ++q) {
          const uint32_t seen = mask & below(p, __builtin_amdgcn_readlane(qpos, q) + 1);
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_frag(st, db, seen), pf, o[db], 0, 0, 0);
            if (lane % 16 == q) o[db] = y;  // (a product's columns are independent: the others are not taken)
          }
        }
        return;
      }
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[db], pf, o[db], 0, 0, 0);
  };
  const int p_first = p_begin + 32 * wave;
  constexpr int kStride = 32 * kWaves;
  if (p_first < p_end) {
    Regs s0, s1;
    load_step(p_first, s0);
    for (int p = p_first;; p += 2 * kStride) {
      const bool more = p + kStride < p_end;
      if (more) load_step(p + kStride, s1);
      step(p, s0);
      if (!more) break;
      const bool again = p + 2 * kStride < p_end;
      if (again) load_step(p + 2 * kStride, s0);
      step(p + kStride, s1);
      if (!again) break;
    }
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
      store_out4(a, b, qq / a.grp, kvh * a.grp + qq % a.grp, HD, d, y);
    } else {
      *reinterpret_cast<f32x4*>(part_o + q * HD + d) = f32x4{y[0], y[1], y[2], y[3]};
      if (d == 0) {
        part_ml[2 * q] = M;
        part_ml[2 * q + 1] = L;
      }
    }
  }
}

// Joins the chunks of one query vector per HD / 4 lanes, in chunk order.
template <int HD>
__global__ void __launch_bounds__(256) paged_combine_kernel(PagedAttnArgs a) {
  constexpr int LN = HD / 4;
  const int64_t idx = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LN;
  const int d = 4 * (threadIdx.x % LN), QV = a.R * a.grp;
  const int64_t bh = idx / QV;
  const int qv = (int)(idx % QV), b = (int)(bh / a.pg.hkv), kvh = (int)(bh % a.pg.hkv);
  if (b >= a.B) return;
  const Seq sq = attn_seq(a, b, false);
  if (sq.pos < 0) return;
  const int total = sq.pos + a.R, chunk = chunk_of(total, a.max_splits), n = (total + chunk - 1) / chunk;
  if (n == 1) return;
  const int64_t slot = (bh * a.qtiles + qv / 16) * a.splits;
  const float* o = a.part + (slot * 16 + qv % 16) * HD + d;
  const float* ml = a.part + (int64_t)a.B * a.pg.hkv * a.qtiles * a.splits * 16 * HD + (slot * 16 + qv % 16) * 2;
  float M = -INFINITY;
  for (int c = 0; c < n; ++c) M = fmaxf(M, ml[32 * c]);
  float y[4] = {0.f, 0.f, 0.f, 0.f}, L = 0.f;
  for (int c = 0; c < n; ++c) {
    const float mc = ml[32 * c], lc = ml[32 * c + 1];
    const float f = mc == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mc - M);
    L += f * lc;
    const f32x4 v = *reinterpret_cast<const f32x4*>(o + (int64_t)c * 16 * HD);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] += f * v[i];
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
    hipLaunchKernelGGL((paged_combine_kernel<HD>), dim3((unsigned)ceil_div(vecs * (HD / 4), 256)), dim3(256), 0, st, a);
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
  const int64_t blocks = (ceil_div((int64_t)a.splits * a.B * a.pg.hkv, kXcds) * kXcds) * a.qtiles;
  if (blocks >= (int64_t(1) << 31) || (int64_t)a.B * a.R * a.hq * hd / 4 / 256 >= (int64_t(1) << 31))
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
