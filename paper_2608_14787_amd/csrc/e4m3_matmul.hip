// Matrix product in 8 bits (gfx950): out[r][n] = sum_j xs[j][r] ws[n / 128][j] sum_{k in block j} x[r][k] w[n][k].
//
// The matrix's rows are the first operand of the products, the activations' the second, so that a lane's four results are
// four columns of one output row and need one activation scale.  A block's 128 products are summed by the matrix cores from
// zero and added to the accumulators in fp32 with the block's two scales (their product in fp32).
//
// Which instructions.  The fp8 products (16x16x128) align the eight products of 8 consecutive columns to the largest sum of two
// exponents among them, E, and cut what lies under 2^(E - 13) toward zero; the groups' sums are added in 24 bits or more.  That is an
// error of the products' size, not of the result's: up to 7 2^-13 of a group's largest, as root mean squares 4.2e-5 to 4.5e-5 of
// such sums (K of 5120 and 25600, 2% of the columns loud), where codes themselves are 2^-4 off and a sum's rounding to bf16 up to 2^-8 of
// it.  bf16 results of more than 16 rows take them, at half the time of bf16 products.  fp32 results, and those of up to 16 rows, which
// wait for memory anyway, widen the codes to bf16, exactly, and sum in fp32.
// Where both scales are powers of two the fp8 instruction takes them; in tiles of many rows it then also adds to the accumulators,
// and no fp32 work is left beside the products (4095 x 51200 x 5120 916 us, 1051 with fp32 scales).  Widened codes take the
// matrix's scale with them.
//
// Bound: up to about 300 rows the matrix's bytes (6.3 to 6.8 TB/s of a plain read stream on this card), then the products (2.5
// PFLOP/s in a library product of fp8 of 8192^3, 3.1 of 16384^3).
//
// Times in this file: a call among others in a captured graph, matrices in turn that together pass the caches; "alone" a kernel's
// own time where each launch stands alone.  Where the matrices lie in memory makes up to a fifth: 33 x 51200 x 5120 takes 43 us from
// some buffers and 54 from others, so that only times of one sentence compare.
#include <algorithm>
#include <cmath>
#include <type_traits>

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

// A power of two w as a product of two, b in 2^-100 .. 2^100 and a = w / b (NaN where w is).  Where both scales are powers of two
// xs ws may lie outside fp32's range and the result not: the matrix's codes are then widened times b, and a block's sum is
// multiplied by xs a.  Up to xs ws = 2^200 neither overflows before the result does (128 x 448^2 is less than 2^25).
struct Factors {
  float a, b;
};
__device__ inline Factors factors(float w) {
  const float b = fminf(fmaxf(w, 0x1p-100f), 0x1p100f);
  return Factors{w * __builtin_bit_cast(float, 0x7f000000u - __builtin_bit_cast(uint32_t, b)), b};
}
__device__ inline int byte_of(float power) { return (int)(__builtin_bit_cast(uint32_t, power) >> 23 & 255); }

// Eight codes times a power of two (2^-100 .. 2^100) to bf16, exactly.
__device__ inline bf16x8 widen(uint32_t lo, uint32_t hi, float by = 1.f) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, by, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, by, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, by, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, by, true);
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
// A workgroup takes NT row tiles of the matrix and all (up to 16) rows; its eight waves take every eighth block of 128
// columns, each its own loads (no barrier in the loop), and join in LDS in wave order.  Bound by the matrix's bytes: each is read
// once, 1 KiB of a wave at a time, past the caches (nothing else reads them).  1 x 51200 x 5120 45 us (5.8 TB/s), 1 x 18944 x 3584 16
// (4.3), 1 x 4608 x 3584 7.0 (5.8 alone).  Two blocks of a wave in registers: 46, 15 and 6.5 against 47, 17 and 7.3 with three and 58, 18
// and 7.7 with four.

constexpr int kFewWaves = 8, kFewRows = 4;

template <int NT>
struct Few {  // a wave's codes and scales of one block of columns
  u32x4 w[NT][2], x[2];
  float ws[NT];
  uint32_t xs;
};

constexpr int kNowhere = 0x7ffffff0;  // an offset past every descriptor's end: zeros, and no memory is read

template <int NT, bool E8, bool BOTH, bool F32>
__global__ void __launch_bounds__(kFewWaves * kWave, 2) few_rows_kernel(MatArgs a) {
  __shared__ __align__(16) f32x4 s_part[kFewWaves][NT][kWave];
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
  const int row = min(lane % 16, a.M - 1);
  auto load = [&](Few<NT>& s, int step) {
    const int kb = wave + kFewWaves * step;  // past KB: past the descriptors' ends
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = kb * kBlock8 + h * 64 + lane / 16 * 16;
      s.x[h] = __builtin_amdgcn_raw_buffer_load_b128(rx, k < a.K ? row * a.K + k : kNowhere, 0, 0);
    }
    const int at = kb < a.KB ? kb * a.M + row : kNowhere / 4;
    s.xs = E8 ? (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rxs, at, 0, 0) : __builtin_amdgcn_raw_buffer_load_b32(rxs, at * 4, 0, 0);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int h = 0; h < 2; ++h) s.w[t][h] = __builtin_amdgcn_raw_buffer_load_b128(rw[t], kb * kTile8 + h * 1024 + lane * 16, 0, kNtCpol);
      s.ws[t] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rws[t], kb * 4, 0, 0));
    }
    __builtin_amdgcn_sched_barrier(0);  // (loads stay in their order: the waits count them)
  };
  f32x4 acc[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](const Few<NT>& s) {
    const float xs = E8 ? e8m0_value(s.xs) : __builtin_bit_cast(float, s.xs);
    Factors ws[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) ws[j] = BOTH ? factors(s.ws[j]) : Factors{s.ws[j], 1.f};
    f32x4 p[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) p[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const bf16x8 x = widen(s.x[h][2 * c], s.x[h][2 * c + 1]);
#pragma unroll
        for (int j = 0; j < NT; ++j)
          p[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(s.w[j][h][2 * c], s.w[j][h][2 * c + 1], ws[j].b), x, p[j], 0, 0, 0);
      }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const float sc = xs * ws[j].a;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] = __builtin_fmaf(p[j][e], sc, acc[j][e]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  Few<NT> s[2];
  load(s[0], 0);
  for (int i = 0; i < steps; i += 2) {
    load(s[1], i + 1);
    multiply(s[0]);
    load(s[0], i + 2);
    multiply(s[1]);  // (behind the last block: zeros)
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) s_part[wave][j][lane] = acc[j];
  __syncthreads();
  for (int item = threadIdx.x; item < NT * kWave; item += kFewWaves * kWave) {
    const int j = item / kWave, l = item % kWave;
    f32x4 v = s_part[0][j][l];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) v += s_part[w][j][l];
    if (t0 + j < a.NT) store4<F32>(a, l % 16, (t0 + j) * 16 + l / 16 * 4, v);
  }
}

// ---- rows shared through LDS ------------------------------------------------------------------------------
//
// A workgroup of 8 / GK x GK waves takes NT row tiles of the matrix a wave, all of up to 16 MT rows, and a part of K.  The rows'
// codes pass through LDS, CB blocks of columns at a time in two buffers, so that they are read from L2 once a workgroup (loaded in
// the operands' order, 16 rows of 64 bytes a load, a compute unit gets 15 bytes a clock from L2; whole lines 50); a
// wave's own tiles go from memory to registers, R - 1 blocks ahead.  33 x 51200 x 5120 42 us alone (6.2 TB/s of the matrix; rows read
// by each wave 74), 43 to 54 among others; 33 x 5120 x 25600 in fp32 27 and 4.5 in the join alone (62 with the columns in one part), 34 among
// others; 33 x 10240 x 5120 17, 33 x 5120 x 8192 15, of 16 rows 15 and 13.  Of a chunk's blocks each of the GK waves of a tile takes
// every GK-th; they join in LDS, in their order.

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kSharedThreads = 512;

template <int MT, int NT, int GK, bool FP8, bool E8, bool BOTH, bool F32>
__global__ void __launch_bounds__(kSharedThreads, 2) shared_rows_kernel(MatArgs a) {
  constexpr int R = MT >= 8 ? 2 : 4;           // blocks of a wave in registers
  constexpr int CB = MT >= 8 ? 2 : 4;          // blocks of a chunk
  constexpr int SPC = CB / GK;                 // of them a wave's
  constexpr int U = R / SPC;                   // chunks until a wave's registers come round
  constexpr int GN = 8 / GK, kRows = 16 * MT;
  constexpr bool AHEAD = U % 2 == 0;           // codes are asked for two chunks ahead, not one
  static_assert(SPC >= 1 && SPC * U == R && (AHEAD || U == 1), "a wave's registers turn with the chunks");
  constexpr int PIECES = kRows * CB * 8 / kSharedThreads;  // 16-byte pieces of a chunk a thread moves
  static_assert(kRows * CB * 8 % kSharedThreads == 0, "pieces of a chunk over the threads");
  constexpr int XS = (CB * kRows + kSharedThreads - 1) / kSharedThreads;
  constexpr bool SCALED = BOTH && FP8;  // the instruction takes the scales
  union Shared {
    struct {
      u32x4 x[2][MT][CB][2][kWave];
      uint32_t xs[2][CB][kRows];  // the scales, fp32 (SCALED: their bytes)
    } in;
    f32x4 part[GK > 1 ? 8 : 1][MT * NT][kWave];
  };
  __shared__ __align__(16) Shared s;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int wn = wave % GN, wk = wave / GN;
  const int groups = (a.NT + GN * NT - 1) / (GN * NT);
  const int group = blockIdx.x % groups, split = blockIdx.x / groups;
  const int k0 = split * a.per, n = min(a.KB, k0 + a.per) - k0;  // blocks of this part
  __amdgpu_buffer_rsrc_t rw[NT], rws[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int tile = min((group * GN + wn) * NT + t, a.NT - 1);
    rw[t] = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w + ((int64_t)tile * a.KB + k0) * kTile8), 0, n * kTile8, kBufferRsrcWord3);
    rws[t] = __builtin_amdgcn_make_buffer_rsrc((void*)(a.ws + (int64_t)(tile / 8) * a.KB + k0), 0, n * 4, kBufferRsrcWord3);
  }
  const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)a.x, 0, a.M * a.K, kBufferRsrcWord3);
  struct W {
    u32x4 w[NT][2];
    float ws[NT];
  };
  auto load_w = [&](W& r, int step) {  // (blocks from n on: past the descriptors' ends)
    const int i = step * GK + wk;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int h = 0; h < 2; ++h) r.w[t][h] = __builtin_amdgcn_raw_buffer_load_b128(rw[t], i * kTile8 + h * 1024 + lane * 16, 0, kNtCpol);
      r.ws[t] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rws[t], i * 4, 0, 0));
    }
  };
  // A chunk's codes: CB * 8 neighbouring threads take a row's 16-byte pieces; piece c of row r lies in its half's column c % 4
  // of the fragment, at place r ^ c % 8, which spreads a row's pieces over the banks.
  const int pc = threadIdx.x % (CB * 8), pr = threadIdx.x / (CB * 8);
  constexpr int STEP = kSharedThreads / (CB * 8);
  struct X {
    u32x4 piece[PIECES];
    uint32_t scale[XS];  // as in memory; behind the part's end 0
  };
  auto load_x = [&](X& v, int i) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int r = pr + p * STEP, k = (k0 + i) * kBlock8 + pc * 16;
      int at = r * a.K + k;
      at = i * 8 + pc < n * 8 && k < a.K && r < a.M ? at : kNowhere;
      asm volatile("" : "+v"(at));  // (a select, not a branch around the load)
      v.piece[p] = __builtin_amdgcn_raw_buffer_load_b128(rx, at, 0, 0);
    }
#pragma unroll
    for (int p = 0; p < XS; ++p) {
      const int at = threadIdx.x + p * kSharedThreads, kb = at / kRows, r = at % kRows;
      const bool ok = kb < CB && i + kb < n;
      const int64_t from = (int64_t)(ok ? k0 + i + kb : k0) * a.M + min(r, a.M - 1);
      if constexpr (E8)
        v.scale[p] = ok ? reinterpret_cast<const uint8_t*>(a.xs)[from] : 0u;
      else
        v.scale[p] = ok ? reinterpret_cast<const uint32_t*>(a.xs)[from] : 0u;
    }
  };
  auto store_x = [&](const X& v, int buf) {
    const int kb = pc / 8, h = pc / 4 % 2, g = pc % 4;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int r = pr + p * STEP;
      s.in.x[buf][r / 16][kb][h][16 * g + ((r % 16) ^ (pc % 8))] = v.piece[p];
    }
#pragma unroll
    for (int p = 0; p < XS; ++p) {
      const int at = threadIdx.x + p * kSharedThreads;
      if (at >= CB * kRows) continue;
      s.in.xs[buf][at / kRows][at % kRows] = E8 && !SCALED ? __builtin_bit_cast(uint32_t, e8m0_value(v.scale[p])) : v.scale[p];
    }
  };
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int g4 = lane / 16, r16 = lane % 16;
  // Row tiles go in groups of G: a group's fragments are read while the one before it is multiplied.
  constexpr int G = MT <= 4 ? MT : 4;
  static_assert(MT % G == 0, "whole groups");
  struct F {
    u32x4 x[G][2];
    uint32_t xs[G];
  };
  auto read_x = [&](F& f, int buf, int kb, int g) {
#pragma unroll
    for (int i = 0; i < G; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) f.x[i][h] = s.in.x[buf][g * G + i][kb][h][16 * g4 + (r16 ^ (4 * h + g4))];
      f.xs[i] = s.in.xs[buf][kb][(g * G + i) * 16 + r16];
    }
  };
  auto multiply = [&](const W& r, int buf, int kb) {
    Factors ws[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) ws[j] = BOTH && !SCALED ? factors(r.ws[j]) : Factors{r.ws[j], 1.f};
    F f[2];
    read_x(f[0], buf, kb, 0);
#pragma unroll
    for (int g = 0; g < MT / G; ++g) {
      if (g + 1 < MT / G) read_x(f[(g + 1) % 2], buf, kb, g + 1);
      const F& v = f[g % 2];
      f32x4 p[G][NT];
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          p[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
          if constexpr (FP8) {
            const i32x8 wf = {(int)r.w[j][0][0], (int)r.w[j][0][1], (int)r.w[j][0][2], (int)r.w[j][0][3],
                              (int)r.w[j][1][0], (int)r.w[j][1][1], (int)r.w[j][1][2], (int)r.w[j][1][3]};
            const i32x8 xf = {(int)v.x[i][0][0], (int)v.x[i][0][1], (int)v.x[i][0][2], (int)v.x[i][0][3],
                              (int)v.x[i][1][0], (int)v.x[i][1][1], (int)v.x[i][1][2], (int)v.x[i][1][3]};
            if constexpr (SCALED)
              p[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf, xf, p[i][j], 0, 0, 0, byte_of(r.ws[j]), 0, (int)v.xs[i]);
            else
              p[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf, xf, p[i][j], 0, 0, 0, 127, 0, 127);
          }
        }
      if constexpr (!FP8) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            bf16x8 wf[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) wf[j] = widen(r.w[j][h][2 * c], r.w[j][h][2 * c + 1], ws[j].b);
#pragma unroll
            for (int i = 0; i < G; ++i) {
              const bf16x8 xf = widen(v.x[i][h][2 * c], v.x[i][h][2 * c + 1]);
#pragma unroll
              for (int j = 0; j < NT; ++j) p[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[j], xf, p[i][j], 0, 0, 0);
            }
          }
      }
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          f32x4& c = acc[g * G + i][j];
          if constexpr (SCALED) {
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] += p[i][j][e];
          } else {
            const float sc = __builtin_bit_cast(float, v.xs[i]) * ws[j].a;
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] = __builtin_fmaf(p[i][j][e], sc, c[e]);
          }
        }
    }
    // (the products stay in their step: unpinned, they are moved behind the loads and barriers of later ones)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) asm volatile("" : "+v"(acc[i][j]));
  };
  auto turn = [&]() {  // a buffer is written, the other has been read
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    phase_barrier();
  };
  // Loads return in their order, so that waiting for a chunk's codes means waiting for every tile that was asked for before
  // them: AHEAD has more than a chunk of tiles in flight.
  W w[R];
  X xr[AHEAD ? 2 : 1];
  load_x(xr[0], 0);
  if constexpr (AHEAD) load_x(xr[1], CB);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < R - 1; ++i) {
    load_w(w[i], i);
    __builtin_amdgcn_sched_barrier(0);
  }
  store_x(xr[0], 0);
  turn();
  const int chunks = (n + CB - 1) / CB;
  for (int c = 0;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int buf = AHEAD ? u % 2 : c % 2;
      load_x(xr[AHEAD ? u % 2 : 0], (c + (AHEAD ? 2 : 1)) * CB);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < SPC; ++j) {
        const int slot = u * SPC + j;
        load_w(w[(slot + R - 1) % R], c * SPC + j + R - 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(w[slot], buf, j * GK + wk);  // (behind the part's end: zeros times scales of zero)
        __builtin_amdgcn_sched_barrier(0);
      }
      store_x(xr[AHEAD ? (u + 1) % 2 : 0], buf ^ 1);
      turn();
      if (++c >= chunks) goto done;
    }
  }
done:
  if constexpr (GK > 1) {  // (the buffers have been read: a barrier lies behind the last chunk)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) s.part[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
  }
  auto put = [&](int i, int tile, int l, f32x4 v) {
    const int m = i * 16 + l % 16, col = tile * 16 + l / 16 * 4;
    if (tile >= a.NT) return;
    if (a.splits > 1) {
      if (m < a.M) *reinterpret_cast<f32x4*>(a.part + ((int64_t)split * a.M + m) * (a.NT * 16) + col) = v;
    } else {
      store4<F32>(a, m, col, v);
    }
  };
  if constexpr (GK > 1) {
    for (int item = threadIdx.x; item < GN * MT * NT * kWave; item += kSharedThreads) {
      const int l = item % kWave, t = item / kWave % (MT * NT), g = item / (kWave * MT * NT);
      f32x4 v = s.part[g][t][l];
#pragma unroll
      for (int k = 1; k < GK; ++k) v += s.part[k * GN + g][t][l];
      put(t / NT, (group * GN + g) * NT + t % NT, l, v);
    }
  } else {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        asm volatile("" : "+v"(acc[i][j]));
        put(i, (group * GN + wn) * NT + j, lane, acc[i][j]);
      }
  }
}

// Parts of sums, added in their order: a thread takes four columns of a row, eight parts in flight at a time (one after the
// other, six parts of 33 x 5120 took 4.8 us).
template <bool F32>
__global__ void __launch_bounds__(256) join_kernel(MatArgs a) {
  const int n = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 4, m = blockIdx.y;
  if (n >= a.N) return;
  const int width = a.NT * 16;
  const float* p = a.part + (int64_t)m * width + n;
  const int64_t step = (int64_t)a.M * width;
  f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.splits; s += 8) {
    f32x4 q[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) q[u] = *reinterpret_cast<const f32x4*>(p + min(s + u, a.splits - 1) * step);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (s + u < a.splits) v += q[u];
  }
  store4<F32>(a, m, n, v);
}

// ---- many rows --------------------------------------------------------------------------------------------
//
// A workgroup of GN x GM waves takes 16 WN GN rows of the matrix and 16 WM GM of the activations; both pass through LDS a block
// of columns at a time, in a ring of RS that is loaded directly.  Scales come eight blocks at a time.
// Bound by the products: 256 x 256 reads LDS 96 KiB for 256 products of 16x16x128, 32 clocks each on four cores, half of what LDS
// could give meanwhile, and L2 64 KiB at 55 bytes a clock.  4095 x 51200 x 5120 1051 us (2.0 PFLOP/s), with powers of two as scales
// 916 (2.3; 4096 x 8192 x 8192 216, 2.5), fp32 results 4095 x 5120 x 25600 915 (1.17: bf16 products).  At 128 x 128 loads, LDS
// and products take about as long each and overlap only in part: 511 x 3584 x 18944 with powers of two 56 us, alone 40 and 6.5 in the
// join; 264 x 10240 x 5120 31.

// 16 bytes a lane from descriptor rs at voffset + soffset to LDS at `to` + 16 lane.  Not the builtin: behind that the compiler
// holds every LDS read back until all such loads have landed, those of the other buffer too.  m0 is the compiler's own register: it sets
// it for each use of its own, and has to hear that it changes here (that is what it warns of).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void load_direct(u32x4 rs, uint32_t to, int voffset, int soffset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(voffset), "s"(rs), "s"(soffset)
               : "memory", "m0");
}
template <bool BYTE>  // a word a lane to `to` + 4 lane: four bytes of memory, or one
__device__ inline void load_direct_word(u32x4 rs, uint32_t to, int voffset, int soffset) {
  if constexpr (BYTE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_ubyte %1, %2, %3 offen lds" ::"s"(to), "v"(voffset), "s"(rs), "s"(soffset)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(to), "v"(voffset), "s"(rs), "s"(soffset)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ inline u32x4 descriptor(const void* p, int bytes) {
  const uint64_t at = (uint64_t)p;
  return u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, (uint32_t)bytes, (uint32_t)kBufferRsrcWord3};
}
template <typename T>
__device__ inline T uniform(T v) {
  static_assert(sizeof(T) % 4 == 0, "words");
  union {
    T t;
    int w[sizeof(T) / 4];
  } u = {v};
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 4; ++i) u.w[i] = __builtin_amdgcn_readfirstlane(u.w[i]);
  return u.t;
}
__device__ inline uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }
__device__ inline i32x8 fragment(const u32x4& a, const u32x4& b) {
  return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

constexpr int kStripe = 12;
constexpr int kScaleSteps = 8;  // blocks whose scales lie in LDS at a time (in two halves)

template <int WN, int WM, int GN, int GM, int RS, bool FP8, bool E8, bool BOTH, bool F32>
__global__ void __launch_bounds__(kWave * GN * GM, 2) many_rows_kernel(MatArgs a) {
  constexpr bool SCALED = BOTH && FP8;  // the instruction takes the scales
  constexpr int kWaves = GN * GM, kThreads = kWave * kWaves, BN = 16 * WN * GN, BM = 16 * WM * GM;
  constexpr int LW = BN / 16 / kWaves, LX = BM / 8 / kWaves;  // KiB of a step that a wave loads, of each half of the tiles and of the rows
  constexpr int HALF = WN / 2;                                // a wave's tiles of a half
  static_assert(BN / 16 % kWaves == 0 && BM / 8 % kWaves == 0 && BN % 128 == 0 && WN % 2 == 0 && LX % 2 == 0, "a step's loads over the waves");
  constexpr int kStage = (BN + BM) * kBlock8;
  constexpr int LS = BM * kScaleSteps / kThreads;  // scale loads of a wave, for kScaleSteps blocks
  static_assert(BM * kScaleSteps % kThreads == 0 && BM % 64 == 0 && BN / 128 * kScaleSteps <= kWave, "scales over the waves");
  __shared__ __align__(16) char s_ring[RS * kStage];
  __shared__ uint32_t s_xs[2][kScaleSteps][BM];
  __shared__ float s_ws[2][kWave];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int n_blocks = (a.NT * 16 + BN - 1) / BN, m_blocks = (a.M + BM - 1) / BM;
  // Workgroups go to the XCDs in turn.  One XCD's, in their order: kStripe blocks of the matrix's rows, all blocks of the
  // activations in turn, so that the 32 at work together share both in its L2 (4095 x 51200 x 5120: stripes of 2 1101 us, 4 1061,
  // 6 to 16 1045 to 1052).
  const int low = blockIdx.x % kXcds, at = blockIdx.x / kXcds;
  const int stripe = at / (kStripe * m_blocks), in = at - stripe * kStripe * m_blocks;
  const int wide = min(kStripe, (n_blocks * a.splits + kXcds - 1) / kXcds - stripe * kStripe);
  const int bm = in / wide, item = (stripe * kStripe + in - bm * wide) * kXcds + low;
  if (item >= n_blocks * a.splits) return;
  const int bn = item % n_blocks, split = item / n_blocks;
  const int k0 = split * a.per, n = min(a.KB, k0 + a.per) - k0;
  const int t0 = bn * (BN / 16), m0 = bm * BM;
  const int tiles = min(BN / 16, a.NT - t0), rows = min(BM, a.M - m0);
  const int w_blocks = (a.NT + 7) / 8;
  const u32x4 rw = uniform(descriptor(a.w + (int64_t)t0 * a.KB * kTile8, tiles * a.KB * kTile8));
  const u32x4 rx = uniform(descriptor(a.x + (int64_t)m0 * a.K, rows * a.K));
  const uint32_t ring = lds_address(s_ring), at_xs = lds_address(s_xs), at_ws = lds_address(s_ws);
  // rows of the activations lie in LDS as in memory, 128 bytes each, 16-byte piece c at place c ^ row % 8
  int xrow[LX];
  const int xpiece = (lane % 8) ^ (lane / 8);
#pragma unroll
  for (int i = 0; i < LX; ++i) xrow[i] = min((wave * LX + i) * 8 + lane / 8, rows - 1) * a.K;
  // The part's blocks behind its last one are loaded as the last again, so that the loads in flight are always as many.
  auto issue_w = [&](int i, int half, int j) {  // load j of the first or the second half of each wave column's tiles
    const int kb = k0 + min(i, n - 1);
    const int b = wave * LW + j, t = b / 2 / HALF * WN + half * HALF + b / 2 % HALF;
    load_direct(rw, ring + i % RS * kStage + t * kTile8 + b % 2 * 1024, lane * 16, (min(t, tiles - 1) * a.KB + kb) * kTile8 + b % 2 * 1024);
  };
  auto issue_x = [&](int i, int j) {
    const int kb = k0 + min(i, n - 1);
    // behind a row's end: its first codes again, which the matrix's stored zeros take out
    const int k = kb * kBlock8 + xpiece * 16, kk = k < a.K ? k : 0;
    load_direct(rx, ring + i % RS * kStage + BN * kBlock8 + (wave * LX + j) * 1024, xrow[j] + kk, 0);
  };
  // Loads of a half step, in their order: half of the rows of step i + RS, and the second tiles of step i + RS - 1 or the first
  // ones of step i + RS, whose places have been read when the half step begins.
  constexpr int LH = LX / 2 + LW;
  auto issue = [&](int i, int half, int q) {
    if (q < LX / 2)
      issue_x(i + RS, half * (LX / 2) + q);
    else
      issue_w(i + RS - 1 + half, 1 - half, q - LX / 2);
  };
  auto issue_scales = [&](int i) {  // of blocks i .. i + kScaleSteps - 1
    const int to = i / kScaleSteps % 2;
#pragma unroll
    for (int p = 0; p < LS; ++p) {
      const int q = (wave * LS + p) * kWave, kb = min(k0 + i + q / BM, a.KB - 1);
      const u32x4 rs = uniform(descriptor(reinterpret_cast<const char*>(a.xs) + ((int64_t)kb * a.M + m0) * (E8 ? 1 : 4), rows * (E8 ? 1 : 4)));
      load_direct_word<E8>(rs, at_xs + (to * kScaleSteps * BM + q) * 4, min(q % BM + lane, rows - 1) * (E8 ? 1 : 4), 0);
    }
    if (wave == 0) {
      const int kb = min(k0 + i + lane / (BN / 128), a.KB - 1), nb = min(t0 / 8 + lane % (BN / 128), w_blocks - 1);
      const u32x4 rs = uniform(descriptor(a.ws + (int64_t)(t0 / 8) * a.KB, min(w_blocks - t0 / 8, BN / 128) * a.KB * 4));
      load_direct_word<false>(rs, at_ws + to * kWave * 4, ((nb - t0 / 8) * a.KB + kb) * 4, 0);
    }
  };
  const int wn = wave % GN, wm = wave / GN, g4 = lane / 16, r16 = lane % 16;
  f32x4 acc[WN][WM];
#pragma unroll
  for (int i = 0; i < WN; ++i)
#pragma unroll
    for (int j = 0; j < WM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  struct Rows {  // fragments of a wave's rows for a step, and the products of their scales with the matrix's
    u32x4 x[WM][2];
    float sc[WM];
    float wb;        // (BOTH: what the matrix's codes are widened times)
    int xs[WM], ws;  // (SCALED: their bytes)
  };
  const int p0 = (g4 ^ (r16 % 8)) * 16, p1 = ((4 + g4) ^ (r16 % 8)) * 16;
  auto read_row = [&](Rows& r, int i, int j) {
    const char* sx = s_ring + i % RS * kStage + BN * kBlock8 + ((wm * WM + j) * 16 + r16) * kBlock8;
    r.x[j][0] = *reinterpret_cast<const u32x4*>(sx + p0);
    r.x[j][1] = *reinterpret_cast<const u32x4*>(sx + p1);
  };
  auto read_scales = [&](Rows& r, int i) {
    const int half = i / kScaleSteps % 2, step = i % kScaleSteps;
    const float w1 = s_ws[half][step * (BN / 128) + wn * WN / 8];
    if constexpr (SCALED) r.ws = byte_of(w1);
    const Factors w = BOTH && !SCALED ? factors(w1) : Factors{w1, 1.f};
    r.wb = w.b;
#pragma unroll
    for (int j = 0; j < WM; ++j) {
      const uint32_t xs = s_xs[half][step][(wm * WM + j) * 16 + r16];
      if constexpr (SCALED)
        r.xs[j] = (int)xs;
      else
        r.sc[j] = (E8 ? e8m0_value(xs) : __builtin_bit_cast(float, xs)) * w.a;
    }
  };
  // tiles read ahead, and the registers that they turn through (256 x 256 has none left for more)
  constexpr int LOOK = WN * WM <= 16 ? 2 : 1, WR = LOOK > 1 ? 4 : 2;
  static_assert(WN % WR == 0 && HALF >= LOOK, "a step's tiles in whole turns, a half step's landed tiles ahead at most");
  u32x4 w[WR][2];
  auto read_tile = [&](u32x4* f, int i, int t) {
    const u32x4* sw = reinterpret_cast<const u32x4*>(s_ring + i % RS * kStage) + (wn * WN + t) * 128 + lane;
    f[0] = sw[0], f[1] = sw[64];
  };
  // The half of a step's products that the tiles I0 .. I0 + HALF - 1 have with its rows; meanwhile the next tiles' fragments are
  // read (those of the next half too), and in the second half the next step's rows.  A product's sums are added two
  // products later: a wave issues in order, and would wait for the products just asked for.
  constexpr int kLag = 2;
  auto multiply = [&](int step, const Rows& r, Rows& next, auto half_c) {
    constexpr int I0 = decltype(half_c)::value * HALF;
    constexpr int EVERY = HALF * WM / LH;  // products between two loads
    static_assert(EVERY >= 1, "loads between the products");
    f32x4 p[kLag + 1];
    auto add = [&](int t) {
      f32x4& c = acc[I0 + t / WM][t % WM];
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = __builtin_fmaf(p[t % (kLag + 1)][e], r.sc[t % WM], c[e]);
      asm volatile("" : "+v"(c));
    };
#pragma unroll
    for (int t = 0; t < HALF * WM; ++t) {
      const int i = I0 + t / WM, j = t % WM;
      if (j == 0) read_tile(w[(i + LOOK) % WR], step + (i + LOOK) / WN, (i + LOOK) % WN);
      if (I0 > 0 && t % HALF == 0 && t / HALF < WM) read_row(next, step + 1, t / HALF);
      if (I0 > 0 && t == HALF * WM / 2) read_scales(next, step + 1);
      // (one at a time: together they fill the queue to memory, and the products behind them wait)
      if (t % EVERY == EVERY / 2 && t / EVERY < LH) issue(step, I0 > 0, t / EVERY);
      const u32x4* f = w[i % WR];
      if constexpr (SCALED) {
        f32x4& c = acc[i][j];
        c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(f[0], f[1]), fragment(r.x[j][0], r.x[j][1]), c, 0, 0, 0, r.ws, 0, r.xs[j]);
        asm volatile("" : "+v"(c));
        __builtin_amdgcn_sched_barrier(0);
        continue;
      }
      f32x4& q = p[t % (kLag + 1)];
      q = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (FP8) {
        q = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(f[0], f[1]), fragment(r.x[j][0], r.x[j][1]), q, 0, 0, 0, 127, 0, 127);
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int c = 0; c < 2; ++c)
            q = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(f[h][2 * c], f[h][2 * c + 1], BOTH ? r.wb : 1.f),
                                                        widen(r.x[j][h][2 * c], r.x[j][h][2 * c + 1]), q, 0, 0, 0);
      }
      if (t >= kLag) add(t - kLag);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (SCALED) return;
#pragma unroll
    for (int t = HALF * WM - kLag; t < HALF * WM; ++t) add(t);
  };
  // All but a wave's newest `left` loads have landed, in every wave, and what was read before has been read; the compiler learns
  // that LDS changed.
  auto turn = [&](auto left_c) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%1) lgkmcnt(0)\n\ts_barrier" ::"v"(ring), "i"(decltype(left_c)::value) : "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // A step in two halves of the tiles, a barrier before each.  What a half reads ahead has to have landed by its own barrier: the
  // second half's first tile by that before the first half, the next step's rows and first tile by that before the second; each
  // time that leaves the loads of 2 RS - 3 half steps on their way.
  constexpr int kLeft = (2 * RS - 3) * LH;
  static_assert(kLeft + LH < 64, "loads that the counter holds");
  issue_scales(0);
#pragma unroll
  for (int i = 0; i < RS; ++i) {
#pragma unroll
    for (int q = 0; q < (i ? LH : LX / 2); ++q) issue(i - RS, 0, q);
#pragma unroll
    for (int q = 0; q < LH; ++q) issue(i - RS, 1, q);
  }
  Rows r0, r1;
  turn(std::integral_constant<int, kLeft + LH>());
#pragma unroll
  for (int i = 0; i < LOOK; ++i) read_tile(w[i], 0, i);
  read_scales(r0, 0);
#pragma unroll
  for (int j = 0; j < WM; ++j) read_row(r0, 0, j);
  auto one_step = [&](int i, Rows& r, Rows& next) {
    turn(std::integral_constant<int, kLeft>());
    multiply(i, r, next, std::integral_constant<int, 0>());
    turn(std::integral_constant<int, kLeft>());
    if (i % kScaleSteps == 0) issue_scales(i + kScaleSteps);
    multiply(i, r, next, std::integral_constant<int, 1>());
  };
  for (int i = 0;;) {
    one_step(i, r0, r1);
    if (++i >= n) break;
    one_step(i, r1, r0);
    if (++i >= n) break;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::"v"(ring) : "memory");  // (nothing is on its way to LDS that the next workgroup has)
#pragma unroll
  for (int i = 0; i < WN; ++i)
#pragma unroll
    for (int j = 0; j < WM; ++j) {
      const int tile = t0 + wn * WN + i, m = m0 + (wm * WM + j) * 16 + r16, col = tile * 16 + g4 * 4;
      if (tile >= a.NT) continue;
      if (a.splits > 1) {
        if (m < a.M) *reinterpret_cast<f32x4*>(a.part + ((int64_t)split * a.M + m) * (a.NT * 16) + col) = acc[i][j];
      } else {
        store4<F32>(a, m, col, acc[i][j]);
      }
    }
}

// How a product is computed: by the call's shape alone.
struct Plan {
  enum Kind { kFew, kShared, kTile128, kTile128Deep, kTile256 } kind;
  int mt, nt, gk;   // kFew, kShared: row tiles of the activations, of the matrix a wave, waves that share a tile
  int splits, per;  // parts of K, blocks of one
};

// Rows of which all calls up to here are computed alike.
int row_class(int M) {
  if (M <= kFewRows) return kFewRows;
  return M <= 64 ? (int)ceil_div(M, 16) * 16 : (int)std::min<int64_t>(ceil_div(M, 128) * 128, kMaxM8);
}

// Many rows: the tile and the parts of K with the least time by the steps that the busiest compute unit takes.  Measured, us a
// step of 128 columns: tiles of 256 x 256 1.35 alone and 2.0 on a full device; of 128 x 128 with four waves (two workgroups a
// compute unit) 0.80 alone, 0.88 with one everywhere, 1.17 with two; with eight waves and a deep ring 0.53 alone and 0.72.  The
// matrix at 6 TB/s, parts written and read at 4.5, 4 us a launch.  Over 24 shapes of 200 to 1023 rows the choice is
// the best or within 1% of it at 17; 5% from it on average and 56% at the most (264 x 3584 x 18944 66 us for 42.5, 700 x 3584 x 18944 92 for
// 71): where the parts do not divide by the XCDs, some get a workgroup more than they have places, which is not counted here.  Of fp32
// results, whose steps take longer, over 10 shapes of 100 to 2048 rows 0.8% on average and 4% at the most.
Plan plan_many(int M, int NT, int KB, bool f32) {
  Plan best = {Plan::kTile128, 0, 0, 0, 1, KB};
  double least = 1e30;
  const double stream = (double)NT * 16 * KB * kBlock8 / 6.0e6;
  for (int kind = Plan::kTile128; kind <= Plan::kTile256; ++kind) {
    const bool big = kind == Plan::kTile256, deep = kind == Plan::kTile128Deep;
    if (big && f32) continue;
    const double blocks = (double)ceil_div(NT, big ? 16 : 8) * ceil_div(M, big ? 256 : 128);
    const double slots = big || deep ? 256 : 512, t1 = big ? 1.35 : deep ? 0.53 : 0.80, t2 = big ? 2.0 : deep ? 0.72 : 1.17;
    for (int s = 1; s <= 8 && (s == 1 || (M <= 4096 && KB / s >= 4)); ++s) {
      const int per = (int)ceil_div(KB, s), parts = (int)ceil_div(KB, per);
      if (parts != s) continue;
      const double wgs = blocks * parts, full = std::floor(wgs / slots), rest = wgs - full * slots;
      const double last = big || deep ? t1 + (t2 - t1) * rest / slots : rest <= 128 ? t1 : rest <= 256 ? 0.88 : t2;
      double t = std::max(per * (full * t2 + (rest > 0 ? last : 0)), stream) + 4;
      if (parts > 1) t += 3 + (double)parts * M * NT * 16 * 8 / 4.5e6;
      if (t < least) least = t, best = Plan{(Plan::Kind)kind, 0, 0, 0, parts, per};
    }
  }
  return best;
}
// Up to 128 rows, measured in us:
// Up to 4 rows: no barrier and no second launch, but a workgroup has its tiles to itself: 1 x 4608 x 3584 7.0 (shared 8.1),
// 1 x 8192 x 5120 9.8 (11.3), 1 x 3584 x 18944 13.5 (15.1).  Not between 256 and 512 tiles, where some compute units get two
// workgroups and others one, and a long row: 1 x 5120 x 25600 30.6 (25.3).  Above 4 the rows are read too often:
// 16 x 51200 x 5120 51.3 (46.9), 16 x 5120 x 25600 37.3 (29.6).
// Tiles a wave of shared rows: two from 2048 row tiles on (33 x 51200 x 5120 48.0, with one 52.7); at 2048 one tile a wave makes 256
// workgroups (33 x 32768 x 4096 28.6, with two 34.2).
// Waves on one tile: four where there are few tiles and blocks (33 x 8192 x 4096 12.0, cut over K and joined 14.7; 33 x 5120 x 8192
// 16.8 and 15.3).
// 65 to 128 rows: shared where that is one launch of two tiles a wave (128 x 51200 x 5120 62, many rows' kernel 74); else many
// rows' (128 x 10240 x 5120 25.2, shared 29.5; fp32 results 128 x 51200 x 5120 83 and 115).
Plan plan_of(int M, int NT, int KB, bool f32) {
  M = row_class(M);
  if (M <= kFewRows && !(NT > 256 && NT < 512 && KB > 64)) return Plan{Plan::kFew, 1, NT >= 512 ? 2 : 1, 1, 1, KB};
  if (M > 128 || (M > 64 && (NT <= 2048 || f32))) return plan_many(M, NT, KB, f32);
  Plan p = {Plan::kShared, (int)ceil_div(M, 16), NT > 2048 ? 2 : 1, 1, 1, KB};
  if (M <= 64 && NT <= 512 && KB <= 32) {
    p.gk = 4;
  } else {
    const int groups = (int)ceil_div(NT, 8 * p.nt);
    p.per = (int)ceil_div(KB, std::max(1, std::min(256 / groups, KB / 4)));
    p.splits = (int)ceil_div(KB, p.per);
  }
  return p;
}
size_t plan_bytes(const Plan& p, int M, int NT) { return p.splits > 1 ? (size_t)p.splits * M * NT * 16 * 4 : 0; }

template <int MT, int NT, int GK, bool E8, bool BOTH, bool F32>
void launch_shared(const MatArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)(ceil_div(a.NT, 8 / GK * NT) * a.splits);
  hipLaunchKernelGGL((shared_rows_kernel<MT, NT, GK, !F32 && (MT > 1), E8, BOTH, F32>), dim3(grid), dim3(kSharedThreads), 0, st, a);
}
template <int MT, bool E8, bool BOTH, bool F32>
void launch_shared(const MatArgs& a, const Plan& p, hipStream_t st) {
  if (p.nt == 2) return launch_shared<MT, 2, 1, E8, BOTH, F32>(a, st);
  if (p.gk == 4) return launch_shared<MT, 1, 4, E8, BOTH, F32>(a, st);
  launch_shared<MT, 1, 1, E8, BOTH, F32>(a, st);
}
template <int WN, int WM, int GN, int GM, int RS, bool E8, bool BOTH, bool F32>
void launch_many(const MatArgs& a, hipStream_t st) {
  const int64_t items = ceil_div(a.NT, WN * GN) * a.splits, m_blocks = ceil_div(a.M, 16 * WM * GM);
  hipLaunchKernelGGL((many_rows_kernel<WN, WM, GN, GM, RS, !F32, E8, BOTH, F32>), dim3((unsigned)(ceil_div(items, kXcds) * kXcds * m_blocks)),
                     dim3(kWave * GN * GM), 0, st, a);
}
template <bool E8, bool BOTH, bool F32>
int launch_matmul(MatArgs a, const Plan& p, hipStream_t st) {
  a.splits = p.splits;
  a.per = p.per;
  switch (p.kind) {
    case Plan::kFew:
      if (p.nt == 2)
        hipLaunchKernelGGL((few_rows_kernel<2, E8, BOTH, F32>), dim3((a.NT + 1) / 2), dim3(kFewWaves * kWave), 0, st, a);
      else
        hipLaunchKernelGGL((few_rows_kernel<1, E8, BOTH, F32>), dim3(a.NT), dim3(kFewWaves * kWave), 0, st, a);
      break;
    case Plan::kShared:
      switch (p.mt) {
        case 1: launch_shared<1, E8, BOTH, F32>(a, p, st); break;
        case 2: launch_shared<2, E8, BOTH, F32>(a, p, st); break;
        case 3: launch_shared<3, E8, BOTH, F32>(a, p, st); break;
        case 4: launch_shared<4, E8, BOTH, F32>(a, p, st); break;
        default:
          if constexpr (!F32) launch_shared<8, 2, 1, E8, BOTH, F32>(a, st);
      }
      break;
    case Plan::kTile128: launch_many<4, 4, 2, 2, 2, E8, BOTH, F32>(a, st); break;
    case Plan::kTile128Deep: launch_many<4, 2, 2, 4, 4, E8, BOTH, F32>(a, st); break;
    case Plan::kTile256:
      if constexpr (!F32) launch_many<8, 4, 2, 4, 2, E8, BOTH, F32>(a, st);
  }
  if (p.splits > 1)
    hipLaunchKernelGGL((join_kernel<F32>), dim3((unsigned)ceil_div(a.NT, 64), (unsigned)a.M), dim3(256), 0, st, a);
  return check_launch("matmul");
}

}  // namespace
}  // namespace sdd

using namespace sdd;

extern "C" int sdd_e4m3_matmul_workspace_bytes(const sdd_e4m3_matrix* m, int M, size_t* bytes) {
  SDD_REQUIRE(bytes != nullptr, "bytes is NULL");
  if (int rc = check_matrix(m)) return rc;
  SDD_REQUIRE(M > 0 && M <= kMaxM8, "bad row count %d", M);
  // (fewer rows may be cut into more parts; over 4096 are in one)
  const int NT = (int)ceil_div(m->N, 16), KB = (int)ceil_div(m->K, kBlock8);
  *bytes = 0;
  for (int rows = kFewRows;; rows = row_class(rows + 1)) {
    const int r = std::min(rows, M);
    for (int f32 = 0; f32 < 2; ++f32) *bytes = std::max(*bytes, plan_bytes(plan_of(r, NT, KB, f32), r, NT));
    if (rows >= M || rows > 4096) break;
  }
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
  const Plan p = plan_of(M, a.NT, a.KB, out_dtype == SDD_F32);
  if (p.kind >= Plan::kTile128) {
    const bool big = p.kind == Plan::kTile256;
    const double blocks = (double)ceil_div(ceil_div(a.NT, big ? 16 : 8) * p.splits, kXcds) * kXcds * ceil_div(M, big ? 256 : 128);
    if (int rc = check_grid(blocks, p.kind == Plan::kTile128 ? 256 : 512)) return rc;
  }
  const size_t need = plan_bytes(p, M, a.NT);
  if (need) {
    SDD_REQUIRE(ws && (uintptr_t)ws % 16 == 0, "workspace is NULL or not 16-byte aligned");
    if (ws_bytes < need) return fail(SDD_ENOMEM, "workspace of %zu bytes, %zu needed", ws_bytes, need);
  }
  a.part = reinterpret_cast<float*>(ws);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  prof_begin(PROF_GEMM8, st);
  int rc;
  const bool f32 = out_dtype == SDD_F32;
  if (scale_dtype == SDD_F32)
    rc = f32 ? launch_matmul<false, false, true>(a, p, st) : launch_matmul<false, false, false>(a, p, st);
  else if (m->scale_dtype == SDD_E8M0)
    rc = f32 ? launch_matmul<true, true, true>(a, p, st) : launch_matmul<true, true, false>(a, p, st);
  else
    rc = f32 ? launch_matmul<true, false, true>(a, p, st) : launch_matmul<true, false, false>(a, p, st);
  prof_end(PROF_GEMM8, st);
  return rc;
}
