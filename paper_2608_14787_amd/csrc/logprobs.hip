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
//
// Bound: the arithmetic, close to the memory.  A bf16 logit costs 11 instructions of which the exponential counts
// four times; 528 rows of 151936 (160 MB, 22.6 us at the copy's 7.1 TB/s) take 35 us without alternatives, 43 with one, 45
// with 5, 50 with 20 (57 where each token that passed was picked out of its vector at once); one row of 152064 floats takes 5.0
// and 9.5 with 20.  The time above that of no alternatives goes to the sorts (a fixed cost of a workgroup) and to the tokens
// that pass: so few workgroups with long chunks, 2048 at most.  528 rows, 20 alternatives: in 3696 workgroups 7 us more than in
// 1584, in 8448 38.  With two vectors in flight instead of four the same rows take 9 us more (the first threshold comes from
// half as many tokens), one row of 4096 twice as long.
#include <algorithm>
#include <type_traits>

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

// The same for 32-bit values.
template <int J, int K>
__device__ inline void sort_step32(uint32_t& v) {
  const uint32_t o = (uint32_t)xor_lane<J>((int)v);
  const int lane = threadIdx.x % kWave;
  v = ((lane & J) == 0) == ((lane & K) == 0) ? max(v, o) : min(v, o);
}
__device__ inline void sort64_32(uint32_t& v) {
  sort_step32<1, 2>(v);
  sort_step32<2, 4>(v), sort_step32<1, 4>(v);
  sort_step32<4, 8>(v), sort_step32<2, 8>(v), sort_step32<1, 8>(v);
  sort_step32<8, 16>(v), sort_step32<4, 16>(v), sort_step32<2, 16>(v), sort_step32<1, 16>(v);
  sort_step32<16, 32>(v), sort_step32<8, 32>(v), sort_step32<4, 32>(v), sort_step32<2, 32>(v), sort_step32<1, 32>(v);
  sort_step32<32, 64>(v), sort_step32<16, 64>(v), sort_step32<8, 64>(v), sort_step32<4, 64>(v), sort_step32<2, 64>(v), sort_step32<1, 64>(v);
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
  bool held;      // best holds keys
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
  if (b.held) {
    v = reversed(v);
    b.best = v > b.best ? v : b.best;
    merge64(b.best);
  } else {
    b.best = v;
    b.held = true;
  }
  const uint64_t t = lane_key(b.best, n - 1);
  if (t > b.thr) set_thr(b, t);
}
__device__ inline int lanes_below(uint64_t mask) {  // lanes of the mask before this one
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
__device__ inline void push(Best& b, uint64_t key, bool pass, int n) {
  const uint64_t mask = __builtin_amdgcn_ballot_w64(pass);
  if (mask == 0) return;
  if (pass) b.buf[b.cnt + lanes_below(mask)] = key;
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

// Wave 0 writes a row's results from its statistics, its token's logit and its sorted keys.
__device__ inline void write_row(const Job& j, int row, int token, float zt, const Stats& st, uint64_t best) {
  const int lane = threadIdx.x % kWave;
  // no distribution: a NaN or +inf among the logits, or none above -inf
  const bool bad = !(st.s > 0.f && st.s < INFINITY && st.m < INFINITY);
  const float nan = __builtin_nanf(""), ls = __logf(st.s);
  if (lane == 0) {
    if (j.tokens) j.logprob[row] = bad || (unsigned)token >= (unsigned)j.V ? nan : (zt - st.m) - ls;
    if (j.entropy) j.entropy[row] = bad ? nan : fmaxf(ls - st.t / st.s, 0.f);
  }
  if (lane < j.n_top) {
    const bool none = bad || best <= kFloor;
    j.top[(int64_t)row * j.n_top + lane] = none ? -1 : (int)~(uint32_t)best;
    j.top_logprob[(int64_t)row * j.n_top + lane] = bad ? nan : none ? -INFINITY : (unordered((uint32_t)(best >> 32)) - st.m) - ls;
  }
}

// VEC elements from p, which need only be aligned as an element is (this GPU's global loads need no more).
template <typename T, int VEC>
__device__ inline uint4 load_any(const T* p) {
  if constexpr (VEC == 1) {
    return make_uint4(__builtin_bit_cast(uint32_t, Elem<T>::to_f32(*p)), 0, 0, 0);
  } else {
    typedef u32x4 any2 __attribute__((aligned(2)));
    typedef u32x4 any4 __attribute__((aligned(4)));
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const std::conditional_t<sizeof(T) == 2, any2, any4>*>(p));
    return make_uint4(v.x, v.y, v.z, v.w);
  }
}

// A vector's 16 bytes again from its values (which are the type's own).
__device__ inline uint4 repack(const float (&x)[8], uint16_t) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, x[2 * i]) >> 16 | (__builtin_bit_cast(uint32_t, x[2 * i + 1]) & 0xffff0000u);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ inline uint4 repack(const float (&x)[4], float) {
  return make_uint4(__builtin_bit_cast(uint32_t, x[0]), __builtin_bit_cast(uint32_t, x[1]), __builtin_bit_cast(uint32_t, x[2]),
                    __builtin_bit_cast(uint32_t, x[3]));
}
template <typename T>
__device__ inline uint4 repack(const float (&x)[1], T) {
  return make_uint4(__builtin_bit_cast(uint32_t, x[0]), 0, 0, 0);
}

template <typename T, bool TOP, int VEC>  // VEC: 16 bytes' elements, or 1 for rows of fewer
__global__ void __launch_bounds__(kThreads) logprobs_kernel(Job j) {
  __shared__ uint64_t s_buf[TOP ? kWaves : 1][TOP ? 2 * kWave : 1];
  __shared__ uint32_t s_first[TOP ? kWaves : 1][TOP ? kWave : 1];
  __shared__ Stats s_st[kWaves];
  __shared__ int s_flag;
  touch_kernargs<Job>();
  const int row = blockIdx.x / j.C, c = blockIdx.x % j.C;
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const T* z = reinterpret_cast<const T*>(j.z) + (int64_t)(row / j.R) * j.seq_stride + (int64_t)(row % j.R) * j.V;
  int token = -1;
  float zt = 0.f;
  if (j.tokens) {
    token = j.tokens[row];
    zt = Elem<T>::to_f32(z[min(max(token, 0), j.V - 1)]);
  }
  const int v_end = min((j.V + VEC - 1) / VEC, (c + 1) * j.chunk);
  Stats st{-INFINITY, 0.f, 0.f};
  Best b;
  if constexpr (TOP) {
    b.best = 0;
    b.cnt = 0;
    b.held = false;
    b.buf = s_buf[wave];
    set_thr(b, kFloor);
  }
  // A vector with a logit that may count is put aside whole; kGroup of them are opened at once, a lane a logit.
  constexpr int kGroup = kWave / VEC;
  __shared__ uint4 s_vec[TOP ? kWaves : 1][TOP ? kWave + kGroup : 1];
  __shared__ int s_at[TOP ? kWaves : 1][TOP ? kWave + kGroup : 1];  // its first index
  int n_vec = 0;
  auto open_vectors = [&](int at, int n) {
    wave_sync();
    using E = std::conditional_t<VEC == 1, float, T>;
    const int i = lane / VEC, e = lane % VEC, in = at + min(i, n - 1);
    const float x = Elem<E>::to_f32(reinterpret_cast<const E*>(&s_vec[wave][in])[e]);
    const uint64_t key = make_key(x, s_at[wave][in] + e);
    push(b, key, i < n && key > b.thr && x > -INFINITY, j.n_top);
    wave_sync();
  };
  const int first = c * j.chunk;
  auto step = [&](auto unroll, int v0) {
    constexpr int U = decltype(unroll)::value;  // vectors of a thread
    // (the row's last vector begins early enough to end with the row, threads past the chunk take it too: every load is in the
    // row, none is conditional; what is not a thread's own is set to -inf)
    uint4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      raw[u] = load_any<T, VEC>(z + min((v0 + u * kThreads + (int)threadIdx.x) * VEC, j.V - VEC));
    float x[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (VEC == 1)
        x[u][0] = __builtin_bit_cast(float, raw[u].x);
      else
        unpack16(raw[u], x[u], T());
    }
    const int v1 = v0 + U * kThreads;
    if (v1 > v_end || (int64_t)v1 * VEC > j.V) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int v = v0 + u * kThreads + (int)threadIdx.x, own = v < v_end ? v * VEC - min(v * VEC, j.V - VEC) : VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][e] = e >= own ? x[u][e] : -INFINITY;
      }
    }
    float hi[U], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      hi[u] = x[u][0];
#pragma unroll
      for (int e = 1; e < VEC; ++e) hi[u] = fmaxf(hi[u], x[u][e]);
      top = fmaxf(top, hi[u]);
    }
    if (__any(top > st.m)) {
      const float mn = fmaxf(st.m, top), d = st.m == -INFINITY ? 0.f : st.m - mn, f = __expf(d);
      st.t = f * (st.t + st.s * fmaxf(d, -1e4f));
      st.s *= f;
      st.m = mn;
    }
    const float ref = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
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
      if (v0 == first) {
        s_first[wave][lane] = ordered(top);
        __syncthreads();
        uint32_t v = s_first[0][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v = max(v, s_first[w][lane]);
        sort64_32(v);
        const uint64_t t = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)v, j.n_top - 1) << 32;
        if (t > kFloor) set_thr(b, t - 1);  // (any index at that logit passes)
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint64_t mask = __builtin_amdgcn_ballot_w64(hi[u] >= b.thr_f);
        if (!mask) continue;
        if (hi[u] >= b.thr_f) {
          const int at = n_vec + lanes_below(mask);
          s_vec[wave][at] = repack(x[u], T());
          s_at[wave][at] = min((v0 + u * kThreads + (int)threadIdx.x) * VEC, j.V - VEC);
        }
        n_vec += __builtin_popcountll(mask);
        while (n_vec >= kGroup) {
          n_vec -= kGroup;
          open_vectors(n_vec, kGroup);
        }
      }
    }
  };
  // (one vector a thread or less at the end: not a step of four)
  int v0 = first;
  for (; v0 + kThreads < v_end; v0 += kUnroll * kThreads) step(std::integral_constant<int, kUnroll>(), v0);
  if (v0 < v_end) step(std::integral_constant<int, 1>(), v0);
  if constexpr (TOP) {
    if (n_vec > 0) open_vectors(0, n_vec);
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
      write_row(j, row, token, zt, st, best);
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
  // this row's chunks, lane l chunk l's statistics and first keys
  const int64_t r0 = (int64_t)row * j.C;
  Stats p{-INFINITY, 0.f, 0.f};
  constexpr int kAhead = 4;  // keys of a chunk that are loaded at once
  uint64_t head[kAhead] = {0, 0, 0, 0};
  if (lane < j.C) {
    p = Stats{ld_coherent(j.recs + 4 * (r0 + lane)), ld_coherent(j.recs + 4 * (r0 + lane) + 1), ld_coherent(j.recs + 4 * (r0 + lane) + 2)};
    if constexpr (TOP)
#pragma unroll
      for (int i = 0; i < kAhead; ++i) head[i] = ld_coherent(j.keys + (r0 + lane) * j.n_top + min(i, j.n_top - 1));
  }
  p = join_wave(p);
  if constexpr (TOP) {
    b.best = 0;
    b.cnt = 0;
    b.held = false;
    set_thr(b, kFloor);
    // n chunks or more: the n-th largest of their best logits is reached by n keys at least
    uint32_t v = (uint32_t)(head[0] >> 32);
    sort64_32(v);
    const uint64_t t = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)v, j.n_top - 1) << 32;
    if (t > kFloor) set_thr(b, t - 1);
    // (lists are sorted)
    bool more = true;
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (more && i < j.n_top) {
        const bool pass = lane < j.C && head[i] > b.thr && head[i] > kFloor;
        more = __builtin_amdgcn_ballot_w64(pass) != 0;
        push(b, head[i], pass, j.n_top);
      }
    for (int i = kAhead; more && i < j.n_top; ++i) {
      const uint64_t k = lane < j.C ? ld_coherent(j.keys + (r0 + lane) * j.n_top + i) : 0;
      const bool pass = k > b.thr && k > kFloor;
      more = __builtin_amdgcn_ballot_w64(pass) != 0;
      push(b, k, pass, j.n_top);
    }
    if (b.cnt > 0) flush(b, j.n_top);
    best = b.best;
  }
  write_row(j, row, token, zt, p, best);
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
  constexpr int VEC = 16 / (int)sizeof(T);
  const int64_t vectors = j.V < VEC ? j.V : ceil_div((int64_t)j.V, VEC);
  j.C = chunks_for(rows, vectors);
  j.chunk = (int)ceil_div(vectors, j.C);
  j.C = (int)ceil_div(vectors, j.chunk);
  const dim3 grid((unsigned)(rows * j.C));
  prof_begin(PROF_LOGP, st);
  auto with = [&](auto top) {
    constexpr bool TOP = decltype(top)::value;
    if (j.V < VEC)
      hipLaunchKernelGGL((logprobs_kernel<T, TOP, 1>), grid, dim3(kThreads), 0, st, j);
    else
      hipLaunchKernelGGL((logprobs_kernel<T, TOP, VEC>), grid, dim3(kThreads), 0, st, j);
  };
  if (j.n_top > 0)
    with(std::true_type());
  else
    with(std::false_type());
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
