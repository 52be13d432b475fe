// Matrix product in 8 bits (gfx950): out[r][n] = sum_j xs[j][r] ws[n / 128][j] sum_{k in block j} x[r][k] w[n][k].
//
// The matrix's rows are the first operand of the products, the activations' the second, so that a lane's four results are
// four columns of one output row and need one activation scale.  A block's 128 products are summed by the matrix cores from
// zero and added to the accumulators in fp32 with the block's two scales.
#include <algorithm>

#include "e4m3.h"

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

template <int MT, int NT>
struct Step {
  uint4 w[NT][2], x[MT][2];
  float xs[MT], ws[NT];
};

template <int MT, int NT, bool E8>
__device__ inline void load_step(const MatArgs& a, Step<MT, NT>& s, int kb, const int* tile, const int* row) {
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const char* p = a.w + ((int64_t)tile[t] * a.KB + kb) * kTile8 + lane * 16;
#pragma unroll
    for (int h = 0; h < 2; ++h) s.w[t][h] = load_nt16(p + h * 1024);
    s.ws[t] = a.ws[(int64_t)(tile[t] / 8) * a.KB + kb];
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // behind a row's end: codes of the same row again, which the matrix's stored zeros take out
      const int k = kb * kBlock8 + h * 64 + lane / 16 * 16;
      s.x[t][h] = load16(a.x + (int64_t)row[t] * a.K + (k < a.K ? k : 0));
    }
    s.xs[t] = x_scale<E8>(a, kb, row[t]);
  }
}

template <int MT, int NT>
__device__ inline void multiply(const Step<MT, NT>& s, f32x4 (*acc)[NT]) {
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
      for (int j = 0; j < NT; ++j) w[j] = c ? widen(s.w[j][h].z, s.w[j][h].w) : widen(s.w[j][h].x, s.w[j][h].y);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const bf16x8 x = c ? widen(s.x[i][h].z, s.x[i][h].w) : widen(s.x[i][h].x, s.x[i][h].y);
#pragma unroll
        for (int j = 0; j < NT; ++j) p[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j], x, p[i][j], 0, 0, 0);
      }
    }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const float sc = s.xs[i] * s.ws[j];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(p[i][j][e], sc, acc[i][j][e]);
    }
}

template <int MT, int NT, bool E8, bool F32>
__global__ void __launch_bounds__(kFewWaves * kWave) few_rows_kernel(MatArgs a) {
  __shared__ __align__(16) f32x4 s_part[kFewWaves][MT * NT][kWave];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  int tile[NT], row[MT];
#pragma unroll
  for (int t = 0; t < NT; ++t) tile[t] = min((int)blockIdx.x * NT + t, a.NT - 1);
#pragma unroll
  for (int t = 0; t < MT; ++t) row[t] = min(t * 16 + lane % 16, a.M - 1);
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  Step<MT, NT> s0, s1;
  int kb = wave;
  if (kb < a.KB) load_step<MT, NT, E8>(a, s0, kb, tile, row);
  for (; kb < a.KB; kb += 2 * kFewWaves) {
    const bool more = kb + kFewWaves < a.KB;
    if (more) load_step<MT, NT, E8>(a, s1, kb + kFewWaves, tile, row);
    multiply<MT, NT>(s0, acc);
    if (kb + 2 * kFewWaves < a.KB) load_step<MT, NT, E8>(a, s0, kb + 2 * kFewWaves, tile, row);
    if (more) multiply<MT, NT>(s1, acc);
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
    const int nt = (int)blockIdx.x * NT + j;
    if (nt < a.NT) store4<F32>(a, i * 16 + l % 16, nt * 16 + l / 16 * 4, v);
  }
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

template <int MT, bool E8, bool F32>
void launch_few(const MatArgs& a, hipStream_t st) {
  if (a.NT >= 1024)
    hipLaunchKernelGGL((few_rows_kernel<MT, 2, E8, F32>), dim3((a.NT + 1) / 2), dim3(kFewWaves * kWave), 0, st, a);
  else
    hipLaunchKernelGGL((few_rows_kernel<MT, 1, E8, F32>), dim3(a.NT), dim3(kFewWaves * kWave), 0, st, a);
}
template <bool E8, bool F32>
int launch_matmul(const MatArgs& a, hipStream_t st) {
  if (a.M <= 16)
    launch_few<1, E8, F32>(a, st);
  else if (a.M <= 32)
    launch_few<2, E8, F32>(a, st);
  else if (a.M <= 48)
    launch_few<3, E8, F32>(a, st);
  else if (a.M <= 64)
    launch_few<4, E8, F32>(a, st);
  else
    hipLaunchKernelGGL((many_rows_kernel<E8, F32>), dim3((a.NT + 7) / 8 * (unsigned)ceil_div(a.M, 128)), dim3(256), 0, st, a);
  return check_launch("matmul");
}

}  // namespace
}  // namespace sdd

using namespace sdd;

extern "C" int sdd_e4m3_matmul_workspace_bytes(const sdd_e4m3_matrix* m, int M, size_t* bytes) {
  SDD_REQUIRE(bytes != nullptr, "bytes is NULL");
  if (int rc = check_matrix(m)) return rc;
  SDD_REQUIRE(M > 0 && M <= kMaxM8, "bad row count %d", M);
  *bytes = 0;
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
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  prof_begin(PROF_GEMM8, st);
  int rc;
  if (scale_dtype == SDD_E8M0)
    rc = out_dtype == SDD_F32 ? launch_matmul<true, true>(a, st) : launch_matmul<true, false>(a, st);
  else
    rc = out_dtype == SDD_F32 ? launch_matmul<false, true>(a, st) : launch_matmul<false, false>(a, st);
  prof_end(PROF_GEMM8, st);
  return rc;
}
