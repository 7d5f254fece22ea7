// Dropout from the counter-based generator, with the residual sum; forward and
// backward draw the same mask from (row, column, seed, offset) and store none.
//
// Per eight consecutive elements of a row one Philox4x32-10 evaluation gives
// 8 x 16 bits.  Bound: HBM (6 bytes an element with a bf16 residual), with the
// generator's 20 32 x 32 -> 64 multiplies per eight elements close behind (at a
// quarter of the vector rate); 16 bits an element rather than 32 halve those.
#include <cmath>

#include "pspo_layer.h"
#include "token_plan.h"
#include "vec8.h"

namespace pspo {
namespace {

// The four output words of Philox4x32-10 (Salmon et al., SC'11).
__device__ __forceinline__ u32x4 philox_words(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0,
                                              uint32_t k1) {
#pragma unroll
  for (int round = 0; round < 10; ++round) {
    const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)p1;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

struct DropArgs {
  const unsigned char *x, *residual;
  const int32_t* row_ids;
  unsigned char* y;
  int32_t N, vecs;      // rows, groups of eight per row
  int32_t per_part;     // groups of one row that one work-group row takes
  uint32_t k0, k1, off_lo, off_hi, T;
  float scale;
};

// 256 threads as (256 / kLanes) rows x kLanes lanes; a row's lanes walk its
// groups in steps of kLanes, up to kStep of them loaded before the first is used.
constexpr int kStep = 4;

template <class Tin, class Tout, bool kResidual, int kLanes, bool kPast>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs a) {
  const int lane = threadIdx.x % kLanes;
  const int64_t n = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  if (n >= a.N) return;
  const uint32_t row = a.row_ids ? (uint32_t)a.row_ids[n] : (uint32_t)n;
  const unsigned char* x = a.x + n * a.vecs * (8 * Tin::kBytes);
  const unsigned char* res = kResidual ? a.residual + n * a.vecs * (8 * Tin::kBytes) : nullptr;
  unsigned char* y = a.y + n * a.vecs * (8 * Tout::kBytes);
  const int begin = blockIdx.y * a.per_part, end = min(begin + a.per_part, a.vecs);
  for (int v0 = begin + lane; v0 < end; v0 += kStep * kLanes) {
    Raw8<Tin> xr[kStep], rr[kStep];
#pragma unroll
    for (int s = 0; s < kStep; ++s)
      if (v0 + s * kLanes < end) {
        xr[s] = load8<Tin, kPast>(x, v0 + s * kLanes);
        if constexpr (kResidual) rr[s] = load8<Tin, kPast>(res, v0 + s * kLanes);
      }
#pragma unroll
    for (int s = 0; s < kStep; ++s) {
      const int v = v0 + s * kLanes;
      if (v >= end) break;
      const u32x4 w = philox_words(row, (uint32_t)v + 1u, a.off_lo, a.off_hi, a.k0, a.k1);
      const Vec8 xv = unpack8(xr[s]);
      Vec8 o;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint32_t h = c & 1 ? w[c / 2] >> 16 : w[c / 2] & 0xFFFFu;
        o.v[c] = h < a.T ? xv.v[c] * a.scale : 0.f;   // a select: a dropped NaN or Inf leaves 0
      }
      if constexpr (kResidual) {
        const Vec8 rv = unpack8(rr[s]);
#pragma unroll
        for (int c = 0; c < 8; ++c) o.v[c] += rv.v[c];
      }
      store8<Tout, kPast>(y, v, o);
    }
  }
}

template <class Tin, class Tout, bool kResidual>
int launch(DropArgs a, hipStream_t stream) {
  const DropPlan p = drop_plan(a.N, a.vecs, Tin::kBytes * (kResidual ? 2 : 1) + Tout::kBytes);
  // a launch holds less than 2^32 threads along x
  PSPO_REQUIRE(p.gx < (int64_t(1) << 24), PSPO_ERR_UNSUPPORTED, "dropout supports at most 2^26 long rows per call");
  a.per_part = p.per_part;
  const dim3 grid((uint32_t)p.gx, (uint32_t)p.parts);
  if (p.past) {
    hipLaunchKernelGGL((dropout_kernel<Tin, Tout, kResidual, 64, true>), grid, dim3(256), 0, stream, a);
    PSPO_LAUNCHED("dropout_kernel", stream);
    return PSPO_OK;
  }
#define PSPO_DROP(L) \
  hipLaunchKernelGGL((dropout_kernel<Tin, Tout, kResidual, L, false>), grid, dim3(256), 0, stream, a)
  switch (p.lanes) {
    case 64: PSPO_DROP(64); break;
    case 32: PSPO_DROP(32); break;
    case 16: PSPO_DROP(16); break;
    case 8: PSPO_DROP(8); break;
    case 4: PSPO_DROP(4); break;
    case 2: PSPO_DROP(2); break;
    default: PSPO_DROP(1); break;
  }
#undef PSPO_DROP
  PSPO_LAUNCHED("dropout_kernel", stream);
  return PSPO_OK;
}

int run(const void* x, const void* residual, const int32_t* row_ids, int32_t N, int32_t d, double p, uint64_t seed,
        uint64_t offset, int32_t tin, int32_t tout, void* y, hipStream_t stream) {
  PSPO_REQUIRE(N >= 0, PSPO_ERR_INVALID_ARG, "N must be >= 0");
  PSPO_REQUIRE(d > 0 && d % 8 == 0, PSPO_ERR_UNSUPPORTED, "dropout needs d > 0 and d % 8 == 0");
  PSPO_REQUIRE(p >= 0.0 && p < 1.0, PSPO_ERR_INVALID_ARG, "p must lie in [0, 1)");
  PSPO_REQUIRE((tin == PSPO_TYPE_BF16 || tin == PSPO_TYPE_F32) && (tout == PSPO_TYPE_BF16 || tout == PSPO_TYPE_F32),
               PSPO_ERR_INVALID_ARG, "unknown element type");
  if (N == 0) return PSPO_OK;
  PSPO_REQUIRE(x && y, PSPO_ERR_INVALID_ARG, "null pointer argument");
  PSPO_REQUIRE(aligned(x, 16) && aligned(residual, 16) && aligned(y, 16) && aligned(row_ids, 4),
               PSPO_ERR_INVALID_ARG, "misaligned pointer argument");
  if (int rc = require_gfx950()) return rc;
  double t = std::floor((1.0 - p) * 65536.0 + 0.5);
  t = t < 1.0 ? 1.0 : (t > 65536.0 ? 65536.0 : t);
  DropArgs a{};
  a.x = static_cast<const unsigned char*>(x);
  a.residual = static_cast<const unsigned char*>(residual);
  a.row_ids = row_ids;
  a.y = static_cast<unsigned char*>(y);
  a.N = N;
  a.vecs = d / 8;
  a.k0 = (uint32_t)seed;
  a.k1 = (uint32_t)(seed >> 32);
  a.off_lo = (uint32_t)offset;
  a.off_hi = (uint32_t)(offset >> 32);
  a.T = (uint32_t)t;
  a.scale = (float)(65536.0 / t);
  const bool fi = tin == PSPO_TYPE_F32, fo = tout == PSPO_TYPE_F32;
  if (residual) return fi ? launch<F32, F32, true>(a, stream) : launch<Bf16, Bf16, true>(a, stream);
  if (fi) return fo ? launch<F32, F32, false>(a, stream) : launch<F32, Bf16, false>(a, stream);
  return fo ? launch<Bf16, F32, false>(a, stream) : launch<Bf16, Bf16, false>(a, stream);
}

}  // namespace
}  // namespace pspo

extern "C" {

int pspo_dropout_add_fwd(const void* x, const void* residual, const int32_t* row_ids, int32_t N, int32_t d, double p,
                         uint64_t seed, uint64_t offset, int32_t type, void* y, hipStream_t stream) {
  using namespace pspo;
  clear_last_error();
  TraceRange trace_range("pspo_dropout_add_fwd");
  return run(x, residual, row_ids, N, d, p, seed, offset, type, type, y, stream);
}

int pspo_dropout_bwd(const void* dy, const int32_t* row_ids, int32_t N, int32_t d, double p, uint64_t seed,
                     uint64_t offset, int32_t dy_type, int32_t dx_type, void* dx, hipStream_t stream) {
  using namespace pspo;
  clear_last_error();
  TraceRange trace_range("pspo_dropout_bwd");
  return run(dy, nullptr, row_ids, N, d, p, seed, offset, dy_type, dx_type, dx, stream);
}

}  // extern "C"
