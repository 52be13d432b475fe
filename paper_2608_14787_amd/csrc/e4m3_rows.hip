// Rows and matrices into 8 bits (gfx950): e4m3 codes with a scale for each block of 128 columns, of rows as they are, after
// a residual's addition and an RMS norm, or after SwiGLU, and of matrices in blocks of 128 x 128.
//
// A block y with a = max |y|: s = max(a / 448, 2^-126), or the least power of two with a <= 448 s; codes = e4m3(y / s).  The
// quotient is fp32's.
// Bound: the memory, and for few rows the chain load, sum, maximum, store.  A lane holds 16 or 8 consecutive columns, 8 or 16
// lanes a block: its maximum is a few steps inside a row of lanes, and no value changes lanes.  Read and written together (a
// copy reaches 4.8 TB/s, a read stream 6.3 to 6.8): matrix 10240 x 5120 of bf16 24 us (6.6 TB/s), rows 2047 x 18944 after SwiGLU 33 (5.9),
// 4095 x 5120 with an fp32 residual and y 49 (5.6); one row 2.8, 33 x 8192 2.9 (a kernel's own time, each launch standing alone).
#include <algorithm>

#include "e4m3.h"

namespace sdd {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Columns of a lane.  16: its codes are 16 bytes; rows of quantize and SwiGLU, matrices.  8: its bf16 values are, and its fp32
// values 32; the norm, which moves up to four times the codes' bytes in other types.
constexpr int kMaxNormThreads = 1024, kMaxNormK = 65536;

template <typename T, int P>
struct Raw {  // P elements as they lie in memory
  static constexpr int N = P * (int)sizeof(T) / 16;
  uint4 v[N];
  __device__ inline void load(const T* p) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = load16(reinterpret_cast<const char*>(p) + 16 * i);
  }
  __device__ inline void zero() {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ inline void values(float* y) const {
#pragma unroll
    for (int i = 0; i < N; ++i) unpack16(v[i], y + i * (16 / sizeof(T)), T());
  }
};
template <typename T, int P>
__device__ inline void store_values(T* p, const float* y) {
  constexpr int E = 16 / sizeof(T);
#pragma unroll
  for (int i = 0; i < P / E; ++i) {
    const float* v = y + i * E;
    uint4 w;
    if constexpr (sizeof(T) == 2)
      w = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    else
      w = make_uint4(__builtin_bit_cast(uint32_t, v[0]), __builtin_bit_cast(uint32_t, v[1]), __builtin_bit_cast(uint32_t, v[2]),
                     __builtin_bit_cast(uint32_t, v[3]));
    reinterpret_cast<uint4*>(p)[i] = w;
  }
}

// max |y|, or infinity where a value is not finite
template <int P>
__device__ inline float amax_of(const float* y) {
  float m = 0.f, z = 0.f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    m = fmaxf(m, fabsf(y[i]));
    z = __builtin_fmaf(y[i], 0.f, z);  // 0 for finite values, NaN otherwise
  }
  return z == 0.f ? m : INFINITY;
}
template <int P>
__device__ inline float amax_block(float m) {  // over the 128 / P lanes of a block
  m = fmaxf(m, dpp_f<kDppXor1>(m));
  m = fmaxf(m, dpp_f<kDppXor2>(m));
  m = fmaxf(m, dpp_f<kDppHalfMirror>(m));
  return P == 16 ? m : fmaxf(m, dpp_f<kDppMirror>(m));
}

constexpr float kTinyScale = 0x1p-90f;
struct Scale {
  float inv;    // 1 / by; NaN: the block is not finite
  float by;     // what the values are divided by: s, or 2^64 s (and they are taken times 2^64)
  float s;
  int byte;     // of a power of two
};
__device__ inline Scale scale_of(float a, bool e8) {
  if (a == INFINITY) return Scale{__builtin_nanf(""), 1.f, 1.f, 127};
  if (a == 0.f) return Scale{1.f, 1.f, 1.f, 127};
  if (e8) {
    // a = f 2^x, f in [1, 2); 448 = 1.75 2^8
    const uint32_t u = __builtin_bit_cast(uint32_t, a);
    const int x = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
    const int byte = max(1, min(254, x + 127));
    const float s = __builtin_bit_cast(float, (uint32_t)byte << 23);
    return Scale{__builtin_bit_cast(float, byte == 254 ? 0x00400000u : (uint32_t)(254 - byte) << 23), s, s, byte};
  }
  const float s = fmaxf(a / 448.f, 0x1p-126f);
  const float by = s < kTinyScale ? s * 0x1p64f : s;
  return Scale{1.f / by, by, s, 0};
}
// P codes of y / s, stored past the caches (100 to 300 MB of rows take 5 to 15% less time so).  The quotient is a product with
// 1 / s corrected by its remainder, as fp32's division rounds it.  The lowest border between two codes is 2^-10, so that a remainder
// that matters is a multiple of 2^-33 2^-23 s: below kTinyScale it could be lost under 2^-149, and the block is divided times 2^64.
template <int P>
__device__ inline void store_codes(uint8_t* to, const float* y, const Scale& sc) {
  uint32_t w[P / 4];
  float v[P];
#pragma unroll
  for (int i = 0; i < P; ++i) v[i] = y[i];
  if (sc.by != sc.s) {
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] *= 0x1p64f;
  }
#pragma unroll
  for (int i = 0; i < P / 4; ++i) {
    float q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      q[j] = v[4 * i + j] * sc.inv;
      q[j] = __builtin_fmaf(-__builtin_fmaf(q[j], sc.by, -v[4 * i + j]), sc.inv, q[j]);  // (in this form -0 stays -0)
    }
    w[i] = sc.inv != sc.inv ? 0x7f7f7f7fu : codes4(q[0], q[1], q[2], q[3]);
  }
  if constexpr (P == 16)
    __builtin_nontemporal_store(u32x4{w[0], w[1], w[2], w[3]}, reinterpret_cast<u32x4*>(to));
  else
    __builtin_nontemporal_store(u32x2{w[0], w[1]}, reinterpret_cast<u32x2*>(to));
}
__device__ inline void store_scale(void* scales, bool e8, int64_t i, const Scale& sc) {
  if (e8)
    reinterpret_cast<uint8_t*>(scales)[i] = (uint8_t)sc.byte;
  else
    reinterpret_cast<float*>(scales)[i] = sc.s;
}

struct RowsArgs {
  const char* x;
  int64_t stride;  // elements
  int M, K;
  uint8_t* codes;
  void* scales;
  int e8;
  // rmsnorm
  const char* res;
  char* res_out;
  const float* gain;
  uint16_t* y;
  float eps;
};

// The lane's P columns from `col` of row m, y, to codes; the first lane of a block stores its scale.
template <int P>
__device__ inline void store_rows(const RowsArgs& a, int64_t m, int col, const float* y) {
  const Scale sc = scale_of(amax_block<P>(amax_of<P>(y)), a.e8);
  if (col >= a.K) return;
  store_codes<P>(a.codes + m * a.K + col, y, sc);
  if (col % kBlock8 == 0) store_scale(a.scales, a.e8, (int64_t)(col / kBlock8) * a.M + m, sc);
}

// Rows as they are, or after SwiGLU: a wave takes 1024 columns of a row.
template <typename T, bool SWIGLU>
__global__ void __launch_bounds__(256) rows_kernel(RowsArgs a, int segs) {
  constexpr int P = 16;
  const int lane = threadIdx.x % kWave;
  const int64_t item = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  const int64_t m = item / segs;
  if (m >= a.M) return;
  const int col = ((int)(item - m * segs) * kWave + lane) * P;
  const T* x = reinterpret_cast<const T*>(a.x) + m * a.stride + col;
  Raw<T, P> r, u;
  r.zero(), u.zero();
  if (col < a.K) {
    r.load(x);
    if constexpr (SWIGLU) u.load(x + a.K);
  }
  float y[P];
  r.values(y);
  if constexpr (SWIGLU) {
    float up[P];
    u.values(up);
    // (the reciprocal of a quarter of 1 + e^-g, and a quarter of that: the instruction gives 0 for 1 / (1 + e^-g) below 2^-126, g < -87.3)
#pragma unroll
    for (int i = 0; i < P; ++i) y[i] = y[i] * (0.25f * __builtin_amdgcn_rcpf(__builtin_fmaf(__expf(-y[i]), 0.25f, 0.25f))) * up[i];
  }
  store_rows<P>(a, m, col, y);
}

// A workgroup takes a row, C vectors of 8 columns a thread, kept in registers between the sum and the conversion.
template <typename T, typename RT, bool RES, int C>
__global__ void __launch_bounds__(kMaxNormThreads) norm_kernel(RowsArgs a) {
  constexpr int P = 8;
  __shared__ float s_sum[kMaxNormThreads / kWave], s_max[kMaxNormThreads / kWave];
  const int64_t m = blockIdx.x;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
  const T* x = reinterpret_cast<const T*>(a.x) + m * a.stride;
  float y[C][P];
  float sum = 0.f;
  Raw<T, P> r[C];
  Raw<RT, P> q[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * (int)blockDim.x + (int)threadIdx.x) * P;
    r[c].zero();
    q[c].zero();
    if (col < a.K) {
      r[c].load(x + col);
      if constexpr (RES) q[c].load(reinterpret_cast<const RT*>(a.res) + m * a.K + col);
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * (int)blockDim.x + (int)threadIdx.x) * P;
    r[c].values(y[c]);
    if constexpr (RES) {
      float z[P];
      q[c].values(z);
#pragma unroll
      for (int i = 0; i < P; ++i) y[c][i] += z[i];
      if (col < a.K) store_values<RT, P>(reinterpret_cast<RT*>(a.res_out) + m * a.K + col, y[c]);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) sum = __builtin_fmaf(y[c][i], y[c][i], sum);
  }
  sum = wave_sum(sum);
  if (lane == 0) s_sum[wave] = sum;
  __syncthreads();
  sum = 0.f;
  for (int w = 0; w < waves; ++w) sum += s_sum[w];
  float eps = a.eps;
  // Squares out of fp32's range (the whole workgroup sees the same sum): above, or so far below that those lost count.  At most
  // 65536 squares lose 2^-150 each, 2^-34 of a sum of 2^-100; a mean below that is 2^-40 of an eps of 2^-60.  The row then starts
  // again times a power of two that brings the larger of its maximum and sqrt(eps) to 1: y = r f / sqrt(mean (r f)^2 + eps f^2).
  if (sum == INFINITY || (sum < 0x1p-100f && eps < 0x1p-60f)) {
    float mx = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < P; ++i) mx = fmaxf(mx, fabsf(y[c][i]));
    mx = wave_max(mx);
    if (lane == 0) s_max[wave] = mx;
    __syncthreads();  // (s_sum has been read, too)
    for (int w = 0; w < waves; ++w) mx = fmaxf(mx, s_max[w]);
    mx = fmaxf(mx, sqrtf(eps));
    if (mx > 0.f && mx < INFINITY) {
      const float f = __builtin_bit_cast(float, (uint32_t)(127 - max(-126, min(126, __builtin_amdgcn_frexp_expf(mx)))) << 23);
      sum = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < P; ++i) {
          y[c][i] *= f;
          sum = __builtin_fmaf(y[c][i], y[c][i], sum);
        }
      sum = wave_sum(sum);
      if (lane == 0) s_sum[wave] = sum;
      __syncthreads();
      sum = 0.f;
      for (int w = 0; w < waves; ++w) sum += s_sum[w];
      eps = eps * f * f;
    }
  }
  const float rs = 1.f / sqrtf(sum / (float)a.K + eps);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * (int)blockDim.x + (int)threadIdx.x) * P;
    if (col < a.K) {
      Raw<float, P> g;
      g.load(a.gain + col);
      float gv[P];
      g.values(gv);
#pragma unroll
      for (int i = 0; i < P; ++i) y[c][i] = y[c][i] * rs * gv[i];
      if (a.y) store_values<uint16_t, P>(a.y + m * a.K + col, y[c]);
    } else {  // (zeros times a norm that is not finite)
#pragma unroll
      for (int i = 0; i < P; ++i) y[c][i] = 0.f;
    }
    store_rows<P>(a, m, col, y[c]);
  }
}

// A workgroup takes a block of 128 x 128, four vectors of 16 columns a thread.
template <typename T>
__global__ void __launch_bounds__(256) matrix_kernel(RowsArgs a, int KB) {
  constexpr int P = 16, kLanes = kBlock8 / P;
  __shared__ float s_max[4];
  const int nb = blockIdx.x / KB, kb = blockIdx.x - nb * KB;
  const int col = kb * kBlock8 + threadIdx.x % kLanes * P;
  Raw<T, P> r[4];
  float mx = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = (int64_t)nb * kBlock8 + i * 32 + threadIdx.x / kLanes;
    r[i].zero();
    if (row < a.M && col < a.K) r[i].load(reinterpret_cast<const T*>(a.x) + row * a.stride + col);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[P];
    r[i].values(y);
    mx = fmaxf(mx, amax_of<P>(y));
  }
  mx = wave_max(mx);
  if (threadIdx.x % kWave == 0) s_max[threadIdx.x / kWave] = mx;
  __syncthreads();
  const Scale sc = scale_of(fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3])), a.e8);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = (int64_t)nb * kBlock8 + i * 32 + threadIdx.x / kLanes;
    if (row >= a.M || col >= a.K) continue;
    float y[P];
    r[i].values(y);
    store_codes<P>(a.codes + row * a.K + col, y, sc);
  }
  if (threadIdx.x == 0) store_scale(a.scales, a.e8, (int64_t)nb * KB + kb, sc);
}

// Row-major codes and scales to the stored order: a thread moves 16 bytes at a time.  51200 x 5120 98 us, 5.4 TB/s read and written,
// where a copy of the codes takes 99.
__global__ void __launch_bounds__(256) load_codes_kernel(const uint8_t* codes, uint4* to, int N, int K, int KB, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int lane = (int)(i % kWave), half = (int)(i / kWave % 2);
    const int64_t tile = i / (2 * kWave);
    const int64_t nt = tile / KB, row = nt * 16 + lane % 16;
    const int col = (int)(tile - nt * KB) * kBlock8 + half * 64 + lane / 16 * 16;
    to[i] = row < N && col < K ? load16(codes + row * K + col) : make_uint4(0, 0, 0, 0);
  }
}
__global__ void __launch_bounds__(256) load_scales_kernel(const void* scales, int e8, float* to, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  to[i] = e8 ? e8m0_value(reinterpret_cast<const uint8_t*>(scales)[i]) : reinterpret_cast<const float*>(scales)[i];
}

bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

// The arguments that every conversion has.
int check_rows(const void* x, int dtype, size_t stride, int M, int K, int width, const void* codes, const void* scales, int scale_dtype) {
  SDD_REQUIRE(x && codes && scales, "NULL pointer");
  SDD_REQUIRE(dtype == SDD_BF16 || dtype == SDD_F32, "rows must be bf16 or fp32 (dtype %d)", dtype);
  SDD_REQUIRE(scale_dtype == SDD_F32 || scale_dtype == SDD_E8M0, "scales must be fp32 or E8M0 (dtype %d)", scale_dtype);
  SDD_REQUIRE(M > 0 && M <= kMaxM8 && K > 0 && K <= kMaxK8 && K % 16 == 0, "bad shape [%d][%d] (K a multiple of 16, at most 2^20)", M, K);
  const size_t es = dtype == SDD_F32 ? 4 : 2;
  SDD_REQUIRE(stride >= (size_t)width && stride <= ((size_t)1 << 32), "row stride %zu for rows of %d", stride, width);
  SDD_REQUIRE(aligned16(x) && stride * es % 16 == 0 && aligned16(codes), "rows and codes must be 16-byte aligned");
  SDD_REQUIRE(scale_dtype == SDD_E8M0 || (uintptr_t)scales % 4 == 0, "scales must be 4-byte aligned");
  return SDD_OK;
}

RowsArgs rows_args(const void* x, size_t stride, int M, int K, uint8_t* codes, void* scales, int scale_dtype) {
  RowsArgs a = {};
  a.x = reinterpret_cast<const char*>(x);
  a.stride = (int64_t)stride;
  a.M = M;
  a.K = K;
  a.codes = codes;
  a.scales = scales;
  a.e8 = scale_dtype == SDD_E8M0;
  return a;
}

template <bool SWIGLU>
int launch_rows(const RowsArgs& a, int dtype, hipStream_t st) {
  const int segs = (int)ceil_div(a.K, 16 * kWave);
  const int64_t blocks = ceil_div((int64_t)a.M * segs, 4);
  if (int rc = check_grid((double)blocks, 256)) return rc;
  prof_begin(PROF_ROWS8, st);
  if (dtype == SDD_F32)
    hipLaunchKernelGGL((rows_kernel<float, SWIGLU>), dim3((unsigned)blocks), dim3(256), 0, st, a, segs);
  else
    hipLaunchKernelGGL((rows_kernel<uint16_t, SWIGLU>), dim3((unsigned)blocks), dim3(256), 0, st, a, segs);
  prof_end(PROF_ROWS8, st);
  return check_launch("rows_kernel");
}

template <typename T, typename RT, bool RES>
void launch_norm(const RowsArgs& a, hipStream_t st) {
  const int vecs = a.K / 8;
  const int threads = (int)std::min<int64_t>(kMaxNormThreads, ceil_div(vecs, kWave) * kWave);
  const int c = (int)ceil_div(vecs, threads);
  if (c == 1)
    hipLaunchKernelGGL((norm_kernel<T, RT, RES, 1>), dim3(a.M), dim3(threads), 0, st, a);
  else if (c == 2)
    hipLaunchKernelGGL((norm_kernel<T, RT, RES, 2>), dim3(a.M), dim3(threads), 0, st, a);
  else if (c <= 4)
    hipLaunchKernelGGL((norm_kernel<T, RT, RES, 4>), dim3(a.M), dim3(threads), 0, st, a);
  else
    hipLaunchKernelGGL((norm_kernel<T, RT, RES, 8>), dim3(a.M), dim3(threads), 0, st, a);
}
template <typename T>
void launch_norm(const RowsArgs& a, int residual_dtype, hipStream_t st) {
  if (!a.res) return launch_norm<T, float, false>(a, st);
  if (residual_dtype == SDD_F32) return launch_norm<T, float, true>(a, st);
  launch_norm<T, uint16_t, true>(a, st);
}

}  // namespace

int check_grid(double blocks, int threads) {
  SDD_REQUIRE(blocks * threads < 4294967296.0, "%.0f workgroups of %d threads are too many for a launch", blocks, threads);
  return SDD_OK;
}

int check_matrix(const sdd_e4m3_matrix* m) {
  SDD_REQUIRE(m != nullptr, "matrix description is NULL");
  SDD_REQUIRE(m->N > 0 && m->N <= kMaxN8 && m->K > 0 && m->K <= kMaxK8 && m->K % 16 == 0,
              "bad matrix [%d][%d] (K a multiple of 16, at most 2^20; N at most 2^24)", m->N, m->K);
  SDD_REQUIRE(m->scale_dtype == SDD_F32 || m->scale_dtype == SDD_E8M0, "a matrix's scales must be fp32 or E8M0 (dtype %d)", m->scale_dtype);
  return SDD_OK;
}

}  // namespace sdd

using namespace sdd;

extern "C" int sdd_e4m3_quantize(const void* x, int dtype, size_t row_stride, int M, int K, uint8_t* codes, void* scales,
                                 int scale_dtype, sdd_stream_t stream) {
  if (int rc = check_rows(x, dtype, row_stride, M, K, K, codes, scales, scale_dtype)) return rc;
  return launch_rows<false>(rows_args(x, row_stride, M, K, codes, scales, scale_dtype), dtype, reinterpret_cast<hipStream_t>(stream));
}

extern "C" int sdd_e4m3_swiglu(const void* x, int dtype, size_t row_stride, int M, int K, uint8_t* codes, void* scales,
                               int scale_dtype, sdd_stream_t stream) {
  SDD_REQUIRE(K <= kMaxK8, "K %d", K);
  if (int rc = check_rows(x, dtype, row_stride, M, K, 2 * K, codes, scales, scale_dtype)) return rc;
  return launch_rows<true>(rows_args(x, row_stride, M, K, codes, scales, scale_dtype), dtype, reinterpret_cast<hipStream_t>(stream));
}

extern "C" int sdd_e4m3_quantize_matrix(const void* x, int dtype, size_t row_stride, int N, int K, uint8_t* codes, void* scales,
                                        int scale_dtype, sdd_stream_t stream) {
  if (int rc = check_rows(x, dtype, row_stride, N, K, K, codes, scales, scale_dtype)) return rc;
  const int KB = (int)ceil_div(K, kBlock8);
  const int64_t blocks = ceil_div(N, kBlock8) * KB;
  if (int rc = check_grid((double)blocks, 256)) return rc;
  const RowsArgs a = rows_args(x, row_stride, N, K, codes, scales, scale_dtype);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  prof_begin(PROF_ROWS8, st);
  if (dtype == SDD_F32)
    hipLaunchKernelGGL((matrix_kernel<float>), dim3((unsigned)blocks), dim3(256), 0, st, a, KB);
  else
    hipLaunchKernelGGL((matrix_kernel<uint16_t>), dim3((unsigned)blocks), dim3(256), 0, st, a, KB);
  prof_end(PROF_ROWS8, st);
  return check_launch("matrix_kernel");
}

extern "C" int sdd_e4m3_rmsnorm(const void* x, int dtype, size_t row_stride, const void* residual, void* residual_out,
                                int residual_dtype, const float* gain, float eps, int M, int K, uint8_t* codes, void* scales,
                                int scale_dtype, uint16_t* y_out, sdd_stream_t stream) {
  if (int rc = check_rows(x, dtype, row_stride, M, K, K, codes, scales, scale_dtype)) return rc;
  SDD_REQUIRE(gain && aligned16(gain), "gain is NULL or not 16-byte aligned");
  SDD_REQUIRE(!residual == !residual_out, "residual and residual_out come together");
  SDD_REQUIRE(!residual || residual_dtype == SDD_BF16 || residual_dtype == SDD_F32, "residual must be bf16 or fp32 (dtype %d)", residual_dtype);
  SDD_REQUIRE(aligned16(residual) && aligned16(residual_out) && aligned16(y_out), "residual and y must be 16-byte aligned");
  SDD_REQUIRE(eps >= 0.f && eps < INFINITY, "eps %g", (double)eps);
  if (K > kMaxNormK) return fail(SDD_EUNSUPPORTED, "rows of %d (at most %d are built)", K, kMaxNormK);
  if (int rc = check_grid(M, (int)std::min<int64_t>(kMaxNormThreads, ceil_div(K / 8, kWave) * kWave))) return rc;
  RowsArgs a = rows_args(x, row_stride, M, K, codes, scales, scale_dtype);
  a.res = reinterpret_cast<const char*>(residual);
  a.res_out = reinterpret_cast<char*>(residual_out);
  a.gain = gain;
  a.eps = eps;
  a.y = y_out;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  prof_begin(PROF_ROWS8, st);
  if (dtype == SDD_F32)
    launch_norm<float>(a, residual_dtype, st);
  else
    launch_norm<uint16_t>(a, residual_dtype, st);
  prof_end(PROF_ROWS8, st);
  return check_launch("norm_kernel");
}

extern "C" int sdd_e4m3_matrix_bytes(const sdd_e4m3_matrix* m, size_t* bytes) {
  SDD_REQUIRE(bytes != nullptr, "bytes is NULL");
  if (int rc = check_matrix(m)) return rc;
  *bytes = (size_t)(matrix_code_bytes(m) + ceil_div(ceil_div(m->N, kBlock8) * ceil_div(m->K, kBlock8) * 4, 256) * 256);
  return SDD_OK;
}

extern "C" int sdd_e4m3_matrix_load(const sdd_e4m3_matrix* m, const uint8_t* codes, const void* scales, sdd_stream_t stream) {
  if (int rc = check_matrix(m)) return rc;
  SDD_REQUIRE(m->data && codes && scales, "NULL pointer");
  SDD_REQUIRE((uintptr_t)m->data % 256 == 0 && aligned16(codes), "the matrix must be 256-byte aligned, its codes 16-byte");
  SDD_REQUIRE(m->scale_dtype == SDD_E8M0 || (uintptr_t)scales % 4 == 0, "scales must be 4-byte aligned");
  const int KB = (int)ceil_div(m->K, kBlock8);
  const int64_t n = matrix_code_bytes(m) / 16, ns = ceil_div(m->N, kBlock8) * KB;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  prof_begin(PROF_ROWS8, st);
  hipLaunchKernelGGL(load_codes_kernel, dim3((unsigned)std::min<int64_t>(ceil_div(n, 256), 1 << 20)), dim3(256), 0, st, codes, reinterpret_cast<uint4*>(m->data),
                     m->N, m->K, KB, n);
  hipLaunchKernelGGL(load_scales_kernel, dim3((unsigned)ceil_div(ns, 256)), dim3(256), 0, st, scales, m->scale_dtype == SDD_E8M0,
                     reinterpret_cast<float*>(reinterpret_cast<char*>(m->data) + matrix_code_bytes(m)), ns);
  prof_end(PROF_ROWS8, st);
  return check_launch("load_codes_kernel");
}
