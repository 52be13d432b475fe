// Log probabilities of given tokens, with each row's entropy and its n most likely tokens (gfx950).
//
// Row z of V logits, m = max z, S = sum e^(z - m), T = sum e^(z - m) (z - m):
//   log p(t) = z_t - m - ln S,   H = -sum p ln p = ln S - T / S.
// One pass over the logits.  Every thread keeps (m, S, T) of what it has seen (a growing m rescales: T <- f (T + S d),
// S <- f S with d = m_old - m_new, f = e^d) and every wave its n largest tokens, the order being by logit and then by
// lower index, as one 64-bit integer key a token.  A wave holds its best 64 keys sorted across its lanes; the n-th is a
// threshold that a vector of logits passes or not with one comparison of its maximum, and the few keys that pass
// gather in LDS until 64 are sorted and merged.  The first threshold is the n-th largest of the lanes' maxima over the
// wave's first vectors: at least n tokens reach it.
// Rows are cut into C chunks of whole 16-byte vectors (C from the row count and V alone); a row's last workgroup to
// finish joins the chunks' records in chunk order, so results do not depend on the order of arrival.
#include <algorithm>

#include "sdd_internal.h"

namespace sdd {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kMaxTop = 32, kMaxChunks = 64;
constexpr int kUnroll = 4;             // vectors in flight per thread
constexpr int kCounters = 1024;        // rows that may be cut into chunks
constexpr int kCntStride = 16;         // ints between two rows' arrival counters (a 64-byte line each)
constexpr size_t kCounterBytes = (size_t)kCounters * kCntStride * 4;
constexpr int kResident = 2048;        // workgroups on the device at once, at 8 a compute unit

struct Job {
  const char* z;
  size_t seq_stride;  // elements
  const int32_t* tokens;
  float *logprob, *entropy, *top_logprob;
  int32_t* top;
  int R, V, n_top, C, chunk;  // chunk: vectors
  int* counters;
  float* recs;     // [rows][C][4]: m, S, T
  uint64_t* keys;  // [rows][C][n_top], best first
};

// Orders floats as unsigned integers (-0 as 0); invertible.
__device__ inline uint32_t ordered(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ inline float unordered(uint32_t o) {
  return __builtin_bit_cast(float, o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ inline uint64_t make_key(float v, int idx) { return (uint64_t)ordered(v) << 32 | (uint32_t)~idx; }
constexpr uint64_t kFloor = (uint64_t)0x007fffffu << 32 | 0xffffffffu;  // no token at -inf is above it

// v of lane l ^ J
template <int J>
__device__ inline int xor_lane(int v) {
  if constexpr (J == 1) return dpp_i<kDppXor1>(v);
  if constexpr (J == 2) return dpp_i<kDppXor2>(v);
  if constexpr (J == 4) return dpp_i<0x1B>(dpp_i<kDppHalfMirror>(v));  // l ^ 7, then l ^ 3 (quad_perm [3,2,1,0])
  if constexpr (J == 8) return dpp_i<kDppRor8>(v);
  unsigned a = (unsigned)v, b = a;
  if constexpr (J == 16) {
    permlane16_swap(a, b);
    return (int)(threadIdx.x & 16 ? a : b);
  } else {
    permlane32_swap(a, b);
    return (int)(threadIdx.x & 32 ? a : b);
  }
}
template <int J>
__device__ inline uint64_t xor_lane64(uint64_t v) {
  return (uint64_t)(uint32_t)xor_lane<J>((int)(v >> 32)) << 32 | (uint32_t)xor_lane<J>((int)v);
}
template <int J, int K>  // one step of a bitonic sort, largest first, of runs of K
__device__ inline void sort_step(uint64_t& v) {
  const uint64_t o = xor_lane64<J>(v);
  const int lane = threadIdx.x % kWave;
  const bool first = ((lane & J) == 0) == ((lane & K) == 0);
  v = (v > o) == first ? v : o;
}
__device__ inline void merge64(uint64_t& v) {  // a bitonic run of 64
  sort_step<32, 64>(v), sort_step<16, 64>(v), sort_step<8, 64>(v), sort_step<4, 64>(v), sort_step<2, 64>(v), sort_step<1, 64>(v);
}
__device__ inline void sort64(uint64_t& v) {
  sort_step<1, 2>(v);
  sort_step<2, 4>(v), sort_step<1, 4>(v);
  sort_step<4, 8>(v), sort_step<2, 8>(v), sort_step<1, 8>(v);
  sort_step<8, 16>(v), sort_step<4, 16>(v), sort_step<2, 16>(v), sort_step<1, 16>(v);
  sort_step<16, 32>(v), sort_step<8, 32>(v), sort_step<4, 32>(v), sort_step<2, 32>(v), sort_step<1, 32>(v);
  merge64(v);
}
__device__ inline uint64_t lane_key(uint64_t v, int l) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, l);
}
__device__ inline uint64_t reversed(uint64_t v) {  // lane l gets lane 63 - l's
  return xor_lane64<32>(xor_lane64<16>((uint64_t)(uint32_t)dpp_i<kDppMirror>((int)(v >> 32)) << 32 | (uint32_t)dpp_i<kDppMirror>((int)v)));
}

__device__ inline void wave_sync() {  // LDS accesses of one wave stay in program order
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A wave's best keys: best[lane] sorted (zero: none), and fewer than 64 more in buf.
struct Best {
  uint64_t best, thr;  // thr: only keys above it count
  float thr_f;         // its logit
  int cnt;
  uint64_t* buf;  // LDS, 128 keys
};
__device__ inline void set_thr(Best& b, uint64_t thr) {
  b.thr = thr;
  b.thr_f = unordered((uint32_t)(thr >> 32));
}
__device__ inline void flush(Best& b, int n) {
  const int lane = threadIdx.x % kWave;
  wave_sync();
  uint64_t v = lane < b.cnt ? b.buf[lane] : 0;
  const uint64_t rest = b.buf[kWave + lane];
  wave_sync();
  b.buf[lane] = rest;
  wave_sync();
  b.cnt = max(0, b.cnt - kWave);
  sort64(v);
  v = reversed(v);
  b.best = v > b.best ? v : b.best;
  merge64(b.best);
  const uint64_t t = lane_key(b.best, n - 1);
  if (t > b.thr) set_thr(b, t);
}
__device__ inline void push(Best& b, uint64_t key, bool pass, int n) {
  const uint64_t mask = __builtin_amdgcn_ballot_w64(pass);
  if (mask == 0) return;
  const int at = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
  if (pass) b.buf[b.cnt + at] = key;
  b.cnt += __builtin_popcountll(mask);
  if (b.cnt >= kWave) flush(b, n);
}

struct Stats {
  float m, s, t;
};
// (m, s, t) of both; commutative.  A part with m = -inf holds s and t of 0, or NaN where a logit was NaN.
__device__ inline Stats join(const Stats& a, const Stats& b) {
  const float m = fmaxf(a.m, b.m);
  const float da = a.m == -INFINITY ? 0.f : a.m - m, db = b.m == -INFINITY ? 0.f : b.m - m;
  // (-88: beyond it e^d is 0 and d s must not become 0 times infinity)
  const float fa = __expf(da), fb = __expf(db);
  return Stats{m, a.s * fa + b.s * fb, fa * (a.t + a.s * fmaxf(da, -1e4f)) + fb * (b.t + b.s * fmaxf(db, -1e4f))};
}
template <int CTRL>
__device__ inline Stats join_dpp(const Stats& a) {
  return join(a, Stats{dpp_f<CTRL>(a.m), dpp_f<CTRL>(a.s), dpp_f<CTRL>(a.t)});
}
__device__ inline Stats join_wave(Stats a) {
  a = join_dpp<kDppXor1>(a);
  a = join_dpp<kDppXor2>(a);
  a = join_dpp<kDppHalfMirror>(a);
  a = join_dpp<kDppMirror>(a);
#pragma unroll
  for (int o = 16; o < kWave; o *= 2) a = join(a, Stats{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.t, o)});
  return a;
}

// Wave 0 writes a row's results from its statistics and sorted keys.
template <typename T>
__device__ inline void write_row(const Job& j, int row, const T* z, const Stats& st, uint64_t best) {
  const int lane = threadIdx.x % kWave;
  // no distribution: a NaN or +inf among the logits, or none above -inf
  const bool bad = !(st.s > 0.f && st.s < INFINITY && st.m < INFINITY);
  const float nan = __builtin_nanf(""), ls = __logf(st.s);
  if (lane == 0) {
    if (j.tokens) {
      const int t = j.tokens[row];
      j.logprob[row] = bad || (unsigned)t >= (unsigned)j.V ? nan : (Elem<T>::to_f32(z[t]) - st.m) - ls;
    }
    if (j.entropy) j.entropy[row] = bad ? nan : fmaxf(ls - st.t / st.s, 0.f);
  }
  if (lane < j.n_top) {
    const bool none = bad || best <= kFloor;
    j.top[(int64_t)row * j.n_top + lane] = none ? -1 : (int)~(uint32_t)best;
    j.top_logprob[(int64_t)row * j.n_top + lane] = bad ? nan : none ? -INFINITY : (unordered((uint32_t)(best >> 32)) - st.m) - ls;
  }
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(Job j) {
  constexpr int VEC = 16 / (int)sizeof(T);
  __shared__ uint64_t s_buf[TOP ? kWaves : 1][TOP ? 2 * kWave : 1];
  __shared__ Stats s_st[kWaves];
  __shared__ int s_flag;
  const int row = blockIdx.x / j.C, c = blockIdx.x % j.C;
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const T* z = reinterpret_cast<const T*>(j.z) + (int64_t)(row / j.R) * j.seq_stride + (int64_t)(row % j.R) * j.V;
  // vectors lie on 16-byte borders: the row's first and last may hold fewer of its elements
  const int shift = (int)((uintptr_t)z % 16 / sizeof(T));
  const int v_end = min((j.V + shift + VEC - 1) / VEC, (c + 1) * j.chunk);
  Stats st{-INFINITY, 0.f, 0.f};
  Best b;
  if constexpr (TOP) {
    b.best = 0;
    b.cnt = 0;
    b.buf = s_buf[wave];
    set_thr(b, kFloor);
  }
  bool first = true;
  for (int v0 = c * j.chunk; v0 < v_end; v0 += kUnroll * kThreads) {
    float x[kUnroll][VEC];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int v = v0 + u * kThreads + (int)threadIdx.x, e0 = v * VEC - shift;
      if (v < v_end && e0 >= 0 && e0 + VEC <= j.V) {
        unpack16(load_nt16(z + e0), x[u], T());
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][e] = v < v_end && e0 + e >= 0 && e0 + e < j.V ? Elem<T>::to_f32(z[e0 + e]) : -INFINITY;
      }
    }
    float hi[kUnroll], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      hi[u] = x[u][0];
#pragma unroll
      for (int e = 1; e < VEC; ++e) hi[u] = fmaxf(hi[u], x[u][e]);
      top = fmaxf(top, hi[u]);
    }
    if (top > st.m) {
      const float d = st.m == -INFINITY ? 0.f : st.m - top, f = __expf(d);
      st.t = f * (st.t + st.s * fmaxf(d, -1e4f));
      st.s *= f;
      st.m = top;
    }
    const float ref = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float s = 0.f, t = 0.f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float d = x[u][e] - ref, p = __expf(d);
        s += p;
        t = __builtin_fmaf(p, fmaxf(d, -1e4f), t);  // (a masked token adds 0 times a finite number)
      }
      st.s += s;
      st.t += t;
    }
    if constexpr (TOP) {
      if (first) {
        first = false;
        uint64_t v = (uint64_t)ordered(top) << 32;
        sort64(v);
        const uint64_t t = lane_key(v, j.n_top - 1);
        if (t > kFloor) set_thr(b, t - 1);  // (any index at that logit passes)
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (!__builtin_amdgcn_ballot_w64(hi[u] >= b.thr_f)) continue;
        const int e0 = (v0 + u * kThreads + (int)threadIdx.x) * VEC - shift;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          if (!__builtin_amdgcn_ballot_w64(x[u][e] >= b.thr_f)) continue;
          const uint64_t key = make_key(x[u][e], e0 + e);
          push(b, key, key > b.thr && x[u][e] > -INFINITY, j.n_top);
        }
      }
    }
  }
  if constexpr (TOP) {
    if (b.cnt > 0) flush(b, j.n_top);
    wave_sync();
    b.buf[lane] = b.best;
  }
  st = join_wave(st);
  if (lane == 0) s_st[wave] = st;
  __syncthreads();
  uint64_t best = 0;
  if (wave == 0) {
    st = join(join(s_st[0], s_st[1]), join(s_st[2], s_st[3]));
    if constexpr (TOP) {
      best = b.best;
#pragma unroll
      for (int w = 1; w < kWaves; ++w) {
        const uint64_t o = s_buf[w][kWave - 1 - lane];
        best = o > best ? o : best;
        merge64(best);
      }
    }
    if (j.C == 1) {
      write_row<T>(j, row, z, st, best);
    } else {
      const int64_t at = (int64_t)row * j.C + c;
      if (lane == 0) {
        st_coherent(j.recs + 4 * at, st.m);
        st_coherent(j.recs + 4 * at + 1, st.s);
        st_coherent(j.recs + 4 * at + 2, st.t);
      }
      if constexpr (TOP)
        if (lane < j.n_top) st_coherent(j.keys + at * j.n_top + lane, best);
    }
  }
  if (j.C == 1) return;
  if (!arrive_last(j.counters + row * kCntStride, j.C, &s_flag) || wave != 0) return;
  // this row's chunks, lane l chunk l's statistics
  const int64_t r0 = (int64_t)row * j.C;
  Stats p{-INFINITY, 0.f, 0.f};
  if (lane < j.C) p = Stats{ld_coherent(j.recs + 4 * (r0 + lane)), ld_coherent(j.recs + 4 * (r0 + lane) + 1), ld_coherent(j.recs + 4 * (r0 + lane) + 2)};
  p = join_wave(p);
  if constexpr (TOP) {
    b.best = 0;
    b.cnt = 0;
    set_thr(b, kFloor);
    // n chunks or more: the n-th largest of their best keys is reached by n keys at least
    uint64_t head = lane < j.C ? ld_coherent(j.keys + (r0 + lane) * j.n_top) : 0, v = head;
    sort64(v);
    const uint64_t t = lane_key(v, j.n_top - 1);
    if (t > kFloor) set_thr(b, t - 1);
    for (int i = 0; i < j.n_top; ++i) {
      const bool pass = lane < j.C && head > b.thr && head > kFloor;
      if (!__builtin_amdgcn_ballot_w64(pass)) break;  // (lists are sorted)
      push(b, head, pass, j.n_top);
      if (i + 1 < j.n_top && lane < j.C) head = ld_coherent(j.keys + (r0 + lane) * j.n_top + i + 1);
    }
    if (b.cnt > 0) flush(b, j.n_top);
    best = b.best;
  }
  write_row<T>(j, row, z, p, best);
}

// Chunks of a row: as many as fill the device once, none under 4 vectors a thread, at most a wave's lanes.
int chunks_for(int64_t rows, int64_t vectors) {
  if (rows > kCounters) return 1;
  const int64_t c = std::min<int64_t>({kResident / rows, ceil_div(vectors, kUnroll * kThreads), kMaxChunks});
  return (int)std::max<int64_t>(1, c);
}
size_t workspace(int64_t rows, int n_top) {
  // rows x chunks is at most kResident, or a row's one chunk needs no record
  return kCounterBytes + (size_t)std::max<int64_t>(kResident, kMaxChunks) * (16 + 8 * (size_t)n_top);
}

template <typename T>
int launch(Job j, int64_t rows, hipStream_t st) {
  const int64_t vectors = ceil_div((int64_t)j.V + 16 / sizeof(T) - 1, 16 / sizeof(T));  // of a row at any alignment
  j.C = chunks_for(rows, vectors);
  j.chunk = (int)ceil_div(vectors, j.C);
  j.C = (int)ceil_div(vectors, j.chunk);
  const dim3 grid((unsigned)(rows * j.C));
  prof_begin(PROF_LOGP, st);
  if (j.n_top > 0)
    hipLaunchKernelGGL((logprobs_kernel<T, true>), grid, dim3(kThreads), 0, st, j);
  else
    hipLaunchKernelGGL((logprobs_kernel<T, false>), grid, dim3(kThreads), 0, st, j);
  prof_end(PROF_LOGP, st);
  return check_launch("logprobs_kernel");
}

}  // namespace
}  // namespace sdd

using namespace sdd;

static int logprobs_shape(int B, int R, int V, int n_top) {
  SDD_REQUIRE(B > 0 && R > 0 && V > 0 && V <= (1 << 28) && (int64_t)B * R <= (1 << 24), "bad shape B=%d rows=%d V=%d", B, R, V);
  SDD_REQUIRE(n_top >= 0 && n_top <= kMaxTop, "n_top must be in [0, %d] (%d)", kMaxTop, n_top);
  return SDD_OK;
}

extern "C" int sdd_logprobs_workspace_bytes(int n_rows, int V, int n_top, size_t* bytes) {
  SDD_REQUIRE(bytes != nullptr, "bytes is NULL");
  int rc = logprobs_shape(1, n_rows, V, n_top);
  if (rc) return rc;
  *bytes = workspace(n_rows, n_top);
  return SDD_OK;
}

extern "C" int sdd_token_logprobs(const void* logits, int dtype, size_t seq_stride, int B, int R, int V, const int32_t* tokens,
                                  int n_top, float* logprob, float* entropy, int32_t* top, float* top_logprob, void* ws,
                                  size_t ws_bytes, sdd_stream_t stream) {
  int rc = logprobs_shape(B, R, V, n_top);
  if (rc) return rc;
  SDD_REQUIRE(logits && ws, "NULL pointer");
  SDD_REQUIRE(dtype == SDD_F32 || dtype == SDD_BF16, "bad logits dtype %d", dtype);
  SDD_REQUIRE((tokens == nullptr) == (logprob == nullptr), "tokens and logprob come together");
  SDD_REQUIRE(n_top == 0 || (top && top_logprob), "n_top > 0 needs top and top_logprob");
  SDD_REQUIRE(B == 1 || seq_stride >= (size_t)R * V, "seq_stride too small");
  SDD_REQUIRE((uintptr_t)logits % (dtype == SDD_F32 ? 4 : 2) == 0, "misaligned logits");
  const int64_t rows = (int64_t)B * R;
  const size_t need = workspace(rows, n_top);
  if (ws_bytes < need) return fail(SDD_ENOMEM, "logprobs workspace needs %zu bytes, got %zu", need, ws_bytes);
  SDD_REQUIRE((uintptr_t)ws % 16 == 0, "workspace must be 16-byte aligned");
  Job j{};
  j.z = reinterpret_cast<const char*>(logits);
  j.seq_stride = seq_stride;
  j.tokens = tokens;
  j.logprob = logprob;
  j.entropy = entropy;
  j.top = top;
  j.top_logprob = top_logprob;
  j.R = R;
  j.V = V;
  j.n_top = n_top;
  j.counters = reinterpret_cast<int*>(ws);
  char* rest = reinterpret_cast<char*>(ws) + kCounterBytes;
  j.keys = reinterpret_cast<uint64_t*>(rest);
  j.recs = reinterpret_cast<float*>(rest + (size_t)kResident * 8 * n_top);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  return dtype == SDD_BF16 ? launch<uint16_t>(j, rows, st) : launch<float>(j, rows, st);
}
