// Products of few tokens (at most 64): C(m, n) = sum_k W(m, k) X(n, k), W and X with K
// inner.  Bound by the bytes of W, which go from memory straight to the registers of the
// matrix instructions: a wave reads 16 rows of W (of each of its matrices) and the tokens'
// rows, a work-group's waves take the K of the same rows in turn and join their sums in LDS
// in wave order.  A lane's two loads of a row take 32 bytes in one piece (the order of K
// within a step is free as long as both operands follow it), so the 128-byte lines of a row
// are read whole by two instructions that go out together.
#pragma once

#include "common.h"

namespace pspo {

constexpr int kSkinnyTokens = 64;
constexpr int kSkinnyK = 64;   // K entries of a step: 4 lane groups x 2 x 8

struct SkinnyArgs {
  const uint16_t* w[2];   // row-major [M][K]; the second matrix with kPair
  const uint16_t* x;      // row-major [N][K]
  int M, N, K;
};

// A thread's 8 entries of a row from k on; zeros past the end (K % 8 == 0).
__device__ __forceinline__ bf16x8 skinny_load(const uint16_t* row, int k, int K, bool live) {
  u32x4 v = {0, 0, 0, 0};
  if (live && k < K) v = *reinterpret_cast<const u32x4*>(row + k);
  return __builtin_bit_cast(bf16x8, v);
}

// kMats matrices, NB blocks of 16 tokens, kAhead steps loaded before the first is used.
// epi(m, n, sums): the entry's sum of each matrix.  At most 16 waves, 8 with more than one
// block (twice the registers).
template <int kMats, int NB, int kAhead, class Epi>
__global__ __launch_bounds__(NB > 1 ? 512 : 1024) void skinny_kernel(SkinnyArgs a, Epi epi) {
  extern __shared__ float partial[];   // [waves][kMats][NB * 16][16]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int m0 = blockIdx.x * 16, r = lane & 15, g = lane >> 4;
  const int64_t pitch = a.K;
  const uint16_t* w[kMats];
#pragma unroll
  for (int p = 0; p < kMats; ++p) w[p] = a.w[p] + (int64_t)(m0 + r) * pitch + g * 16;
  const bool row = m0 + r < a.M;
  const uint16_t* x[NB];
  bool tok[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    x[b] = a.x + (int64_t)(b * 16 + r) * pitch + g * 16;
    tok[b] = b * 16 + r < a.N;
  }
  f32x4 acc[kMats][NB] = {};
  const int steps = (a.K + kSkinnyK - 1) / kSkinnyK, left = a.K - g * 16;
  for (int s0 = wave; s0 < steps; s0 += waves * kAhead) {
    bf16x8 fw[kAhead][kMats][2], fx[kAhead][NB][2];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int k = (s0 + s * waves) * kSkinnyK;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int p = 0; p < kMats; ++p) fw[s][p][h] = skinny_load(w[p], k + h * 8, left, row);
#pragma unroll
        for (int b = 0; b < NB; ++b) fx[s][b][h] = skinny_load(x[b], k + h * 8, left, tok[b]);
      }
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int p = 0; p < kMats; ++p)
#pragma unroll
          for (int b = 0; b < NB; ++b)
            acc[p][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[s][p][h], fx[s][b][h], acc[p][b], 0, 0, 0);
  }
  constexpr int kWave = kMats * NB * 256;
#pragma unroll
  for (int p = 0; p < kMats; ++p)
#pragma unroll
    for (int b = 0; b < NB; ++b)
      *reinterpret_cast<f32x4*>(partial + wave * kWave + ((p * NB + b) * 16 + r) * 16 + g * 4) = acc[p][b];
  __syncthreads();
  for (int i = threadIdx.x; i < NB * 256; i += blockDim.x) {
    const int m = m0 + (i & 15), n = i >> 4;
    if (m >= a.M || n >= a.N) continue;
    float sum[kMats];
#pragma unroll
    for (int p = 0; p < kMats; ++p) {
      sum[p] = 0.f;
      for (int q = 0; q < waves; ++q) sum[p] += partial[q * kWave + p * (NB * 256) + i];
    }
    epi(m, n, sum);
  }
}

}  // namespace pspo
