// Matrix product in 8 bits (gfx950): out[r][n] = sum_j xs[j][r] ws[n / 128][j] sum_{k in block j} x[r][k] w[n][k].
//
// The matrix's rows are the first operand of the products, the activations' the second, so that a lane's four results are
// four columns of one output row and need one activation scale.  A block's 128 products are summed by the matrix cores from
// zero and added to the accumulators in fp32 with the block's two scales.
#include <algorithm>

#include "e4m3.h"
#include "gemm.h"

namespace sdd {
namespace {

struct MatArgs {
  const char* w;     // stored tiles
  const float* ws;   // [ceil(N / 128)][KB]
  const uint8_t* x;  // [M][K]
  const void* xs;    // [KB][M]
  int M, N, K, KB, NT;  // NT: row tiles of the matrix
  char* out;
  int64_t stride;  // elements of out
  int vec;         // rows of out take stores of four elements
  // sums cut over K: `splits` parts of `per` blocks, each to part [split][M][16 NT] in fp32 (splits > 1)
  int splits, per;
  float* part;
};

template <bool E8>
__device__ inline float x_scale(const MatArgs& a, int kb, int m) {
  const int64_t i = (int64_t)kb * a.M + m;
  return E8 ? e8m0_value(reinterpret_cast<const uint8_t*>(a.xs)[i]) : reinterpret_cast<const float*>(a.xs)[i];
}

// Eight codes to bf16, exactly.
__device__ inline bf16x8 widen(uint32_t lo, uint32_t hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Four consecutive columns from n of row m.
template <bool F32>
__device__ inline void store4(const MatArgs& a, int m, int n, const f32x4& v) {
  if (m >= a.M) return;
  if constexpr (F32) {
    float* o = reinterpret_cast<float*>(a.out) + (int64_t)m * a.stride + n;
    if (a.vec && n + 4 <= a.N) {
      *reinterpret_cast<f32x4*>(o) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < a.N) o[i] = v[i];
    }
  } else {
    uint16_t* o = reinterpret_cast<uint16_t*>(a.out) + (int64_t)m * a.stride + n;
    if (a.vec && n + 4 <= a.N) {
      *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < a.N) o[i] = f32_to_bf16(v[i]);
    }
  }
}

// ---- few rows ---------------------------------------------------------------------------------------------
//
// A workgroup takes NT row tiles of the matrix and all (up to 16 MT) rows; its eight waves take every eighth block of 128
// columns, each its own loads (no barrier in the loop), and join in LDS in wave order.

constexpr int kFewWaves = 8;

template <int NT>
struct WStep {
  u32x4 w[NT][2];
  float ws[NT];
};
template <int MT>
struct XStep {
  u32x4 x[MT][2];
  uint32_t xs[MT];
};

// widened on its way to the products; p: a block's sums
template <int MT, int NT, bool E8>
__device__ inline void multiply(const WStep<NT>& s, const XStep<MT>& r, f32x4 (*acc)[NT]) {
  f32x4 p[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) p[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      bf16x8 w[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j] = widen(s.w[j][h][2 * c], s.w[j][h][2 * c + 1]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const bf16x8 x = widen(r.x[i][h][2 * c], r.x[i][h][2 * c + 1]);
#pragma unroll
        for (int j = 0; j < NT; ++j) p[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j], x, p[i][j], 0, 0, 0);
      }
    }
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const float xs = E8 ? e8m0_value(r.xs[i]) : __builtin_bit_cast(float, r.xs[i]);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const float sc = xs * s.ws[j];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(p[i][j][e], sc, acc[i][j][e]);
    }
  }
}

constexpr int kNowhere = 0x7ffffff0;  // an offset past every descriptor's end: zeros, and no memory is read

template <int MT, int NT, bool E8, bool F32>
__global__ void __launch_bounds__(kFewWaves * kWave, 2) few_rows_kernel(MatArgs a) {
  constexpr int WS = 2, XS = 2;
  __shared__ __align__(16) f32x4 s_part[kFewWaves][MT * NT][kWave];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int t0 = blockIdx.x * NT;
  const int steps = (a.KB - wave + kFewWaves - 1) / kFewWaves;  // (KB < wave: none)
  __amdgpu_buffer_rsrc_t rw[NT], rws[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int tile = min(t0 + t, a.NT - 1);
    rw[t] = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w + (int64_t)tile * a.KB * kTile8), 0, a.KB * kTile8, kBufferRsrcWord3);
    rws[t] = __builtin_amdgcn_make_buffer_rsrc((void*)(a.ws + (int64_t)(tile / 8) * a.KB), 0, a.KB * 4, kBufferRsrcWord3);
  }
  const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)a.x, 0, a.M * a.K, kBufferRsrcWord3);
  const __amdgpu_buffer_rsrc_t rxs = __builtin_amdgcn_make_buffer_rsrc((void*)a.xs, 0, a.KB * a.M * (E8 ? 1 : 4), kBufferRsrcWord3);
  int row[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) row[t] = min(t * 16 + lane % 16, a.M - 1);
  auto load_w = [&](WStep<NT>& s, int step) {
    const int kb = wave + kFewWaves * step;  // past KB: past the descriptors' ends
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int h = 0; h < 2; ++h) s.w[t][h] = __builtin_amdgcn_raw_buffer_load_b128(rw[t], kb * kTile8 + h * 1024 + lane * 16, 0, kNtCpol);
      s.ws[t] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rws[t], kb * 4, 0, 0));
    }
  };
  auto load_x = [&](XStep<MT>& s, int step) {
    const int kb = wave + kFewWaves * step;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = kb * kBlock8 + h * 64 + lane / 16 * 16;
        s.x[t][h] = __builtin_amdgcn_raw_buffer_load_b128(rx, k < a.K ? row[t] * a.K + k : kNowhere, 0, 0);
      }
      const int at = kb < a.KB ? kb * a.M + row[t] : kNowhere / 4;
      s.xs[t] = E8 ? (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rxs, at, 0, 0) : __builtin_amdgcn_raw_buffer_load_b32(rxs, at * 4, 0, 0);
    }
  };
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  WStep<NT> w[WS];
  XStep<MT> x[XS];
  static_assert(WS % XS == 0, "rings turn together");
#pragma unroll
  for (int i = 0; i < WS - 1; ++i) {
    load_w(w[i], i);
    if (i >= WS - XS) load_x(x[i - (WS - XS)], i - (WS - XS));
    __builtin_amdgcn_sched_barrier(0);
  }
  for (int i = 0; i < steps; i += WS) {
#pragma unroll
    for (int j = 0; j < WS; ++j) {
      load_x(x[(j + XS - 1) % XS], i + j + XS - 1);
      load_w(w[(j + WS - 1) % WS], i + j + WS - 1);
      __builtin_amdgcn_sched_barrier(0);  // (loads stay in their order: the waits count them)
      multiply<MT, NT, E8>(w[j], x[j % XS], acc);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) s_part[wave][i * NT + j][lane] = acc[i][j];
  __syncthreads();
  for (int item = threadIdx.x; item < MT * NT * kWave; item += kFewWaves * kWave) {
    const int t = item / kWave, l = item % kWave, i = t / NT, j = t % NT;
    f32x4 v = s_part[0][t][l];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) v += s_part[w][t][l];
    if (t0 + j < a.NT) store4<F32>(a, i * 16 + l % 16, (t0 + j) * 16 + l / 16 * 4, v);
  }
}

// ---- rows shared through LDS ------------------------------------------------------------------------------
//
// A workgroup takes 8 NT row tiles of the matrix, NT a wave, up to 16 MT rows, and a part of K.  The rows' codes pass through
// LDS, CB blocks at a time in two buffers, so that they are read from L2 once a workgroup; a wave's own tiles go from memory to
// registers, R - 1 blocks ahead.

typedef int i32x8 __attribute__((ext_vector_type(8)));

template <int MT, int NT, int R, bool FP8, bool E8, bool F32>
__global__ void __launch_bounds__(512, MT * NT <= 4 ? 4 : 2) shared_rows_kernel(MatArgs a) {
  constexpr int CB = R, kThreads = 512, kRows = 16 * MT;
  constexpr int PIECES = kRows * CB * 8 / kThreads;  // 16-byte pieces of a chunk a thread moves
  static_assert(kRows * CB * 8 % kThreads == 0, "pieces of a chunk over the threads");
  __shared__ __align__(16) u32x4 s_x[2][MT][CB][2][kWave];
  __shared__ float s_xs[2][CB][kRows];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int groups = (a.NT + 8 * NT - 1) / (8 * NT);
  const int group = blockIdx.x % groups, rest = blockIdx.x / groups, split = rest % a.splits, m0 = rest / a.splits * kRows;
  const int k0 = split * a.per, n = min(a.KB, k0 + a.per) - k0;  // blocks of this part
  __amdgpu_buffer_rsrc_t rw[NT], rws[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int tile = min((group * 8 + wave) * NT + t, a.NT - 1);
    rw[t] = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w + ((int64_t)tile * a.KB + k0) * kTile8), 0, n * kTile8, kBufferRsrcWord3);
    rws[t] = __builtin_amdgcn_make_buffer_rsrc((void*)(a.ws + (int64_t)(tile / 8) * a.KB + k0), 0, n * 4, kBufferRsrcWord3);
  }
  const int rows = min(kRows, a.M - m0);
  const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + (int64_t)m0 * a.K), 0, rows * a.K, kBufferRsrcWord3);
  struct W {
    u32x4 w[NT][2];
    float ws[NT];
  };
  auto load_w = [&](W& s, int i) {  // (blocks from n on: past the descriptors' ends)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int h = 0; h < 2; ++h) s.w[t][h] = __builtin_amdgcn_raw_buffer_load_b128(rw[t], i * kTile8 + h * 1024 + lane * 16, 0, kNtCpol);
      s.ws[t] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rws[t], i * 4, 0, 0));
    }
  };
  // A chunk's codes: CB * 8 neighbouring threads take a row's 16-byte pieces; piece c of row r lies in its half's column c % 4
  // of the fragment, at place r ^ c % 8, which spreads a row's pieces over the banks.
  const int pc = threadIdx.x % (CB * 8), pr = threadIdx.x / (CB * 8);
  constexpr int STEP = kThreads / (CB * 8);
  u32x4 piece[PIECES];
  float xscale[(CB * kRows + kThreads - 1) / kThreads];
  auto load_x = [&](int i) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int r = pr + p * STEP, k = (k0 + i) * kBlock8 + pc * 16;
      piece[p] = __builtin_amdgcn_raw_buffer_load_b128(rx, i * 8 + pc < n * 8 && k < a.K && r < rows ? r * a.K + k : kNowhere, 0, 0);
    }
#pragma unroll
    for (int p = 0; p < (CB * kRows + kThreads - 1) / kThreads; ++p) {
      const int at = threadIdx.x + p * kThreads, kb = at / kRows, r = at % kRows;
      const bool ok = kb < CB && i + kb < n;
      xscale[p] = x_scale<E8>(a, ok ? k0 + i + kb : k0, m0 + min(r, rows - 1));
    }
  };
  auto store_x = [&](int buf) {
    const int kb = pc / 8, h = pc / 4 % 2, g = pc % 4;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int r = pr + p * STEP;
      s_x[buf][r / 16][kb][h][16 * g + ((r % 16) ^ (pc % 8))] = piece[p];
    }
#pragma unroll
    for (int p = 0; p < (CB * kRows + kThreads - 1) / kThreads; ++p) {
      const int at = threadIdx.x + p * kThreads;
      if (at < CB * kRows) s_xs[buf][at / kRows][at % kRows] = xscale[p];
    }
  };
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int g4 = lane / 16, r16 = lane % 16;
  auto multiply = [&](const W& s, int buf, int kb) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      u32x4 x[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) x[h] = s_x[buf][i][kb][h][16 * g4 + (r16 ^ (4 * h + g4))];
      const float xs = s_xs[buf][kb][i * 16 + r16];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        f32x4 p = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (FP8) {
          const i32x8 wf = {(int)s.w[j][0][0], (int)s.w[j][0][1], (int)s.w[j][0][2], (int)s.w[j][0][3],
                            (int)s.w[j][1][0], (int)s.w[j][1][1], (int)s.w[j][1][2], (int)s.w[j][1][3]};
          const i32x8 xf = {(int)x[0][0], (int)x[0][1], (int)x[0][2], (int)x[0][3], (int)x[1][0], (int)x[1][1], (int)x[1][2], (int)x[1][3]};
          p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf, xf, p, 0, 0, 0, 127, 0, 127);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < 2; ++c)
              p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(s.w[j][h][2 * c], s.w[j][h][2 * c + 1]),
                                                          widen(x[h][2 * c], x[h][2 * c + 1]), p, 0, 0, 0);
        }
        const float sc = xs * s.ws[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(p[e], sc, acc[i][j][e]);
      }
    }
  };
  auto turn = [&]() {  // a buffer is written, the other has been read
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    phase_barrier();
  };
  W w[R];
  load_x(0);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < R - 1; ++i) {
    load_w(w[i], i);
    __builtin_amdgcn_sched_barrier(0);
  }
  store_x(0);
  turn();
  int buf = 0;
  for (int i = 0; i < n; i += CB) {
    load_x(i + CB);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      load_w(w[(j + R - 1) % R], i + j + R - 1);
      __builtin_amdgcn_sched_barrier(0);
      if (i + j < n) multiply(w[j], buf, j);
      __builtin_amdgcn_sched_barrier(0);
    }
    store_x(buf ^ 1);
    turn();
    buf ^= 1;
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int tile = (group * 8 + wave) * NT + j, m = m0 + i * 16 + r16;
      asm volatile("" : "+v"(acc[i][j]));
      if (tile >= a.NT) continue;
      if (a.splits > 1) {
        if (m < a.M) *reinterpret_cast<f32x4*>(a.part + ((int64_t)split * a.M + m) * (a.NT * 16) + tile * 16 + g4 * 4) = acc[i][j];
      } else {
        store4<F32>(a, m, tile * 16 + g4 * 4, acc[i][j]);
      }
    }
}

// Parts of sums, added in their order: a thread takes four columns of a row.
template <bool F32>
__global__ void __launch_bounds__(256) join_kernel(MatArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t m = i / (a.NT * 4);
  if (m >= a.M) return;
  const int n = (int)(i - m * (a.NT * 4)) * 4;
  const float* p = a.part + m * (a.NT * 16) + n;
  const int64_t step = (int64_t)a.M * (a.NT * 16);
  f32x4 v = *reinterpret_cast<const f32x4*>(p);
  for (int s = 1; s < a.splits; ++s) v += *reinterpret_cast<const f32x4*>(p + s * step);
  if (n < a.N) store4<F32>(a, (int)m, n, v);
}

// ---- many rows --------------------------------------------------------------------------------------------
//
// A workgroup takes 128 rows of the matrix and 128 of the activations, through LDS a block of columns at a time; four waves
// of 64 x 64.

template <bool E8, bool F32>
__global__ void __launch_bounds__(256) many_rows_kernel(MatArgs a) {
  __shared__ __align__(16) uint4 s_w[8][2][kWave], s_x[8][2][kWave];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int n_blocks = (a.NT + 7) / 8;
  const int bn = blockIdx.x % n_blocks, bm = blockIdx.x / n_blocks;
  const int wn = wave % 2 * 4, wm = wave / 2 * 4;
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kb = 0; kb < a.KB; ++kb) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = wave * 2 + i / 2, h = i % 2;
      const int nt = min(bn * 8 + t, a.NT - 1);
      s_w[t][h][lane] = load16(a.w + ((int64_t)nt * a.KB + kb) * kTile8 + h * 1024 + lane * 16);
      const int m = min(bm * 128 + t * 16 + lane % 16, a.M - 1), k = kb * kBlock8 + h * 64 + lane / 16 * 16;
      s_x[t][h][lane] = load16(a.x + (int64_t)m * a.K + (k < a.K ? k : 0));
    }
    __syncthreads();
    const float ws = a.ws[(int64_t)bn * a.KB + kb];
    f32x4 p[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) p[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 w[4], x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = s_w[wn + i][h][lane], x[i] = s_x[wm + i][h][lane];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          p[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w[j].x, w[j].y), widen(x[i].x, x[i].y), p[i][j], 0, 0, 0);
          p[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w[j].z, w[j].w), widen(x[i].z, x[i].w), p[i][j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float sc = ws * x_scale<E8>(a, kb, min(bm * 128 + (wm + i) * 16 + lane % 16, a.M - 1));
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(p[i][j][e], sc, acc[i][j][e]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int nt = bn * 8 + wn + j;
      if (nt < a.NT) store4<F32>(a, bm * 128 + (wm + i) * 16 + lane % 16, nt * 16 + lane / 16 * 4, acc[i][j]);
    }
}

// How a product is computed: by the call's shape alone.
struct Plan {
  int kind;  // 0: few rows, 1: shared rows, 2: many rows
  int mt, nt, splits, per;
};
Plan plan_of(int M, int NT, int KB) {
  Plan p = {2, 8, 8, 1, KB};
  if (M <= 16) {
    p.kind = 0, p.mt = 1, p.nt = NT >= 512 ? 2 : 1;
  } else if (M <= 256) {
    p.kind = 1;
    p.mt = M <= 32 ? 2 : M <= 48 ? 3 : M <= 64 ? 4 : M <= 128 ? 8 : 16;
    p.nt = p.mt >= 8 || NT >= 2048 ? 2 : 1;
    const int groups = (int)ceil_div(NT, 8 * p.nt);
    p.splits = std::max(1, std::min(256 / groups, KB / 4));
    p.per = (int)ceil_div(KB, p.splits);
    p.splits = (int)ceil_div(KB, p.per);
  }
  return p;
}
size_t plan_bytes(const Plan& p, int M, int NT) { return p.splits > 1 ? (size_t)p.splits * M * NT * 16 * 4 : 0; }

template <int MT, int NT, bool E8, bool F32>
void launch_shared(const MatArgs& a, hipStream_t st) {
  constexpr int R = MT >= 8 ? 2 : 4;
  const unsigned grid = (unsigned)(ceil_div(a.NT, 8 * NT) * a.splits * ceil_div(a.M, 16 * MT));
  hipLaunchKernelGGL((shared_rows_kernel<MT, NT, R, !F32, E8, F32>), dim3(grid), dim3(512), 0, st, a);
}
template <bool E8, bool F32>
int launch_matmul(MatArgs a, const Plan& p, hipStream_t st) {
  a.splits = p.splits;
  a.per = p.per;
  if (p.kind == 0) {
    if (p.nt == 2)
      hipLaunchKernelGGL((few_rows_kernel<1, 2, E8, F32>), dim3((a.NT + 1) / 2), dim3(kFewWaves * kWave), 0, st, a);
    else
      hipLaunchKernelGGL((few_rows_kernel<1, 1, E8, F32>), dim3(a.NT), dim3(kFewWaves * kWave), 0, st, a);
  } else if (p.kind == 1) {
    switch (p.mt * 4 + p.nt) {
      case 9: launch_shared<2, 1, E8, F32>(a, st); break;
      case 13: launch_shared<3, 1, E8, F32>(a, st); break;
      case 17: launch_shared<4, 1, E8, F32>(a, st); break;
      case 33: launch_shared<8, 1, E8, F32>(a, st); break;
      case 65: launch_shared<16, 1, E8, F32>(a, st); break;
      case 10: launch_shared<2, 2, E8, F32>(a, st); break;
      case 14: launch_shared<3, 2, E8, F32>(a, st); break;
      case 18: launch_shared<4, 2, E8, F32>(a, st); break;
      case 34: launch_shared<8, 2, E8, F32>(a, st); break;
      default: launch_shared<16, 2, E8, F32>(a, st);
    }
    if (p.splits > 1)
      hipLaunchKernelGGL((join_kernel<F32>), dim3((unsigned)ceil_div((int64_t)a.M * a.NT * 4, 256)), dim3(256), 0, st, a);
  } else {
    hipLaunchKernelGGL((many_rows_kernel<E8, F32>), dim3((a.NT + 7) / 8 * (unsigned)ceil_div(a.M, 128)), dim3(256), 0, st, a);
  }
  return check_launch("matmul");
}

}  // namespace
}  // namespace sdd

using namespace sdd;

extern "C" int sdd_e4m3_matmul_workspace_bytes(const sdd_e4m3_matrix* m, int M, size_t* bytes) {
  SDD_REQUIRE(bytes != nullptr, "bytes is NULL");
  if (int rc = check_matrix(m)) return rc;
  SDD_REQUIRE(M > 0 && M <= kMaxM8, "bad row count %d", M);
  // (fewer rows may be cut into more parts)
  const int NT = (int)ceil_div(m->N, 16), KB = (int)ceil_div(m->K, kBlock8);
  *bytes = plan_bytes(plan_of(M, NT, KB), M, NT);
  for (int rows = 16; rows < M && rows <= 4096; rows += 16) *bytes = std::max(*bytes, plan_bytes(plan_of(rows, NT, KB), rows, NT));
  return SDD_OK;
}

extern "C" int sdd_e4m3_matmul(const sdd_e4m3_matrix* m, const uint8_t* x, const void* x_scales, int scale_dtype, int M, void* out,
                               int out_dtype, size_t out_stride, void* ws, size_t ws_bytes, sdd_stream_t stream) {
  if (int rc = check_matrix(m)) return rc;
  SDD_REQUIRE(m->data && x && x_scales && out, "NULL pointer");
  SDD_REQUIRE(M > 0 && M <= kMaxM8, "bad row count %d", M);
  SDD_REQUIRE(scale_dtype == SDD_F32 || scale_dtype == SDD_E8M0, "scales must be fp32 or E8M0 (dtype %d)", scale_dtype);
  SDD_REQUIRE(out_dtype == SDD_F32 || out_dtype == SDD_BF16, "out must be bf16 or fp32 (dtype %d)", out_dtype);
  const size_t es = out_dtype == SDD_F32 ? 4 : 2;
  SDD_REQUIRE(out_stride >= (size_t)m->N && out_stride <= ((size_t)1 << 32), "out stride %zu for rows of %d", out_stride, m->N);
  SDD_REQUIRE((uintptr_t)m->data % 256 == 0 && (uintptr_t)x % 16 == 0, "the matrix must be 256-byte aligned, codes 16-byte");
  SDD_REQUIRE((uintptr_t)out % es == 0 && (scale_dtype == SDD_E8M0 || (uintptr_t)x_scales % 4 == 0), "misaligned out or scales");
  MatArgs a = {};
  a.w = reinterpret_cast<const char*>(m->data);
  a.ws = reinterpret_cast<const float*>(a.w + matrix_code_bytes(m));
  a.x = x;
  a.xs = x_scales;
  a.M = M;
  a.N = m->N;
  a.K = m->K;
  a.KB = (int)ceil_div(m->K, kBlock8);
  a.NT = (int)ceil_div(m->N, 16);
  a.out = reinterpret_cast<char*>(out);
  a.stride = (int64_t)out_stride;
  a.vec = (uintptr_t)out % (4 * es) == 0 && out_stride % 4 == 0;
  SDD_REQUIRE(ceil_div(a.NT, 8) * ceil_div(M, 128) < ((int64_t)1 << 31), "too many rows (%d of %d)", M, m->N);
  const Plan p = plan_of(M, a.NT, a.KB);
  const size_t need = plan_bytes(p, M, a.NT);
  if (need) {
    SDD_REQUIRE(ws && (uintptr_t)ws % 16 == 0, "workspace is NULL or not 16-byte aligned");
    if (ws_bytes < need) return fail(SDD_ENOMEM, "workspace of %zu bytes, %zu needed", ws_bytes, need);
  }
  a.part = reinterpret_cast<float*>(ws);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  prof_begin(PROF_GEMM8, st);
  int rc;
  if (scale_dtype == SDD_E8M0)
    rc = out_dtype == SDD_F32 ? launch_matmul<true, true>(a, p, st) : launch_matmul<true, false>(a, p, st);
  else
    rc = out_dtype == SDD_F32 ? launch_matmul<false, true>(a, p, st) : launch_matmul<false, false>(a, p, st);
  prof_end(PROF_GEMM8, st);
  return rc;
}
