// The gated feed-forward block y = (act(x Wg^T) * (x Wu^T)) Wd^T and its gradient.
//
// Forward, two products: gate and up together (their weight rows interleaved by
// blocks of 16 in the tile, so a lane holds both pre-activations of an entry and
// the activation and the product are the epilogue; h is the only intermediate
// that is written, in bf16), then the down projection.  Backward, four products:
// dh = dy Wd with the activation's gradient as its epilogue (reads the kept float32
// pre-activations, writes dg, du and h), dx = [dg du] [Wg; Wu], [dWg; dWu] =
// [dg du]^T x, dWd = dy^T h.  Roundings: h, dg and du to bf16 (the matrix cores'
// operand type; each adds 2^-9 relative rms or less to a sum of f or N terms), the
// outputs once; the pre-activations stay float32, because an error of theirs
// enters the gradient twice (through act and act').
#include <algorithm>
#include <cmath>

#include "pspo_layer.h"
#include "rowgemm.h"
#include "vec8.h"

namespace pspo {
namespace {

// act(g) = g s(a(g)), s the logistic function: a(g) = g (silu), or
// 2 sqrt(2/pi) (g + 0.044715 g^3) (gelu_tanh, as 1 + tanh(v) = 2 s(2 v)).
__device__ __forceinline__ float logistic(float a) { return 1.f / (1.f + __expf(-a)); }

constexpr float kGelu = 1.5957691216057308f;   // 2 sqrt(2 / pi)

__device__ __forceinline__ float act_value(float g, int kind) {
  if (kind == PSPO_ACT_SILU) return g * logistic(g);
  // beyond 16 the logistic is 0 or 1; the bound keeps the cube finite
  const float b = fminf(fmaxf(g, -16.f), 16.f);
  return g * logistic(kGelu * (b + 0.044715f * b * b * b));
}
__device__ __forceinline__ void act_both(float g, int kind, float& a, float& da) {
  if (kind == PSPO_ACT_SILU) {
    const float s = logistic(g);
    a = g * s;
    da = s + a * (1.f - s);
    return;
  }
  const float b = fminf(fmaxf(g, -16.f), 16.f);
  const float s = logistic(kGelu * (b + 0.044715f * b * b * b));
  a = g * s;
  da = s + b * s * (1.f - s) * (kGelu * (1.f + 0.134145f * b * b));
}

__device__ __forceinline__ u32x2 pack4(const float* v) { return u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}; }

// ---- epilogues -----------------------------------------------------------------
// The tile goes out in steps of kCols columns (tokens) through the wave's LDS, so
// that every store writes whole lines of one row.
constexpr int kCols = 16;

// C(m, n) -> out[n * ld + m] in bf16; rows n >= split belong to a second matrix.
struct EpiBf16 {
  uint16_t *out, *out2;
  int64_t ld;
  int M, N, split;
  template <int BM, int BN>
  __device__ __forceinline__ void apply(f32x4 (&acc)[BM][BN], int tm, int tn, int wm, int wn, int lane,
                                        unsigned char* lds, int) const {
    constexpr int kRow = BM * 32;
    const int m0 = (tm * 2 + wm) * BM * 16;
    repeat<BN>([&](auto jc) {   // constant indices into the accumulators, whatever the unroller decides
      constexpr int j = decltype(jc)::value;
#pragma unroll
      for (int i = 0; i < BM; ++i) {
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = acc[i][j][r];
        *reinterpret_cast<u32x2*>(lds + (lane & 15) * (kRow + 16) + i * 32 + (lane >> 4) * 8) = pack4(v);
      }
      wave_lds_fence();
      constexpr int kPer = kRow / 16;
#pragma unroll
      for (int x = 0; x < kCols * kPer; x += 64) {
        const int r = (x + lane) / kPer, c = (x + lane) % kPer * 8;
        const int n = ((tn * 2 + wn) * BN + j) * 16 + r;
        if (n < N && m0 + c < M) {
          uint16_t* row = n < split ? out + (int64_t)n * ld : out2 + (int64_t)(n - split) * ld;
          *reinterpret_cast<u32x4*>(row + m0 + c) = *reinterpret_cast<const u32x4*>(lds + r * (kRow + 16) + c * 2);
        }
      }
      wave_lds_fence();
    });
  }
};

// C(m, n) -> out[part][n * ld + m] in float32, or added to it.
struct EpiF32 {
  float *out, *out2;
  int64_t ld, part_stride;
  int M, N, split, add;
  template <int BM, int BN>
  __device__ __forceinline__ void apply(f32x4 (&acc)[BM][BN], int tm, int tn, int wm, int wn, int lane,
                                        unsigned char*, int part) const {
    const int m0 = (tm * 2 + wm) * BM * 16 + (lane >> 4) * 4;
    repeat<BN>([&](auto jc) {   // constant indices into the accumulators, whatever the unroller decides
      constexpr int j = decltype(jc)::value;
      const int n = ((tn * 2 + wn) * BN + j) * 16 + (lane & 15);
      if (n >= N) return;
      float* row = (n < split ? out + (int64_t)n * ld : out2 + (int64_t)(n - split) * ld) + part * part_stride;
#pragma unroll
      for (int i = 0; i < BM; ++i)
        if (m0 + i * 16 < M) {   // M % 8 == 0
          f32x4* p = reinterpret_cast<f32x4*>(row + m0 + i * 16);
          f32x4 v;
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = acc[i][j][r];
          *p = add ? *p + v : v;
        }
    });
  }
};

// Row blocks in pairs (gate, up): h[n][j] = act(g) u, and the pre-activations if kept.
struct EpiGateUp {
  uint16_t* h;
  float* pre;     // [N][2 f] or NULL
  int f, N, act;
  template <int BM, int BN>
  __device__ __forceinline__ void apply(f32x4 (&acc)[BM][BN], int tm, int tn, int wm, int wn, int lane,
                                        unsigned char* lds, int) const {
    constexpr int kRow = BM * 16;   // BM * 8 entries of h a token
    const int m0 = (tm * 2 + wm) * BM * 8;
    repeat<BN>([&](auto jc) {   // constant indices into the accumulators, whatever the unroller decides
      constexpr int j = decltype(jc)::value;
      const int n0 = ((tn * 2 + wn) * BN + j) * 16, n = n0 + (lane & 15);
#pragma unroll
      for (int i = 0; i < BM; i += 2) {
        f32x4 g, u;
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          g[r] = acc[i][j][r];
          u[r] = acc[i + 1][j][r];
          v[r] = act_value(g[r], act) * u[r];
        }
        const int m = m0 + i * 8 + (lane >> 4) * 4;
        if (pre != nullptr && n < N && m < f) {
          float* row = pre + (int64_t)n * 2 * f + m;
          *reinterpret_cast<f32x4*>(row) = g;
          *reinterpret_cast<f32x4*>(row + f) = u;
        }
        *reinterpret_cast<u32x2*>(lds + (lane & 15) * (kRow + 16) + i * 16 + (lane >> 4) * 8) = pack4(v);
      }
      wave_lds_fence();
      put_rows<kRow, kCols>(lds, reinterpret_cast<unsigned char*>(h + (int64_t)n0 * f + m0), (int64_t)f * 2, N - n0,
                            (f - m0) * 2, lane);
      wave_lds_fence();
    });
  }
};

// C(j, n) = dh: dgu[n] = (dh u act'(g), dh act(g)), h[n] = act(g) u.
struct EpiDh {
  const float* pre;   // [N][2 f]
  uint16_t *dgu, *h;  // [N][2 f], [N][f]
  int f, N, act;
  template <int BM, int BN>
  __device__ __forceinline__ void apply(f32x4 (&acc)[BM][BN], int tm, int tn, int wm, int wn, int lane,
                                        unsigned char* lds, int) const {
    constexpr int kRow = BM * 32, kOne = kCols * (kRow + 16);
    const int m0 = (tm * 2 + wm) * BM * 16;
    repeat<BN>([&](auto jc) {   // constant indices into the accumulators, whatever the unroller decides
      constexpr int j = decltype(jc)::value;
      const int n0 = ((tn * 2 + wn) * BN + j) * 16, n = n0 + (lane & 15);
#pragma unroll
      for (int i = 0; i < BM; ++i) {
        const int m = m0 + i * 16 + (lane >> 4) * 4;
        f32x4 g = {0.f, 0.f, 0.f, 0.f}, u = g;
        if (n < N && m < f) {
          const float* row = pre + (int64_t)n * 2 * f + m;
          g = *reinterpret_cast<const f32x4*>(row);
          u = *reinterpret_cast<const f32x4*>(row + f);
        }
        float dg[4], du[4], hv[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float a, da;
          act_both(g[r], act, a, da);
          const float dh = acc[i][j][r];
          dg[r] = dh * u[r] * da;
          du[r] = dh * a;
          hv[r] = a * u[r];
        }
        unsigned char* at = lds + (lane & 15) * (kRow + 16) + i * 32 + (lane >> 4) * 8;
        *reinterpret_cast<u32x2*>(at) = pack4(dg);
        *reinterpret_cast<u32x2*>(at + kOne) = pack4(du);
        *reinterpret_cast<u32x2*>(at + 2 * kOne) = pack4(hv);
      }
      wave_lds_fence();
      unsigned char* o = reinterpret_cast<unsigned char*>(dgu + (int64_t)n0 * 2 * f + m0);
      put_rows<kRow, kCols>(lds, o, (int64_t)f * 4, N - n0, (f - m0) * 2, lane);
      put_rows<kRow, kCols>(lds + kOne, o + (int64_t)f * 2, (int64_t)f * 4, N - n0, (f - m0) * 2, lane);
      put_rows<kRow, kCols>(lds + 2 * kOne, reinterpret_cast<unsigned char*>(h + (int64_t)n0 * f + m0), (int64_t)f * 2,
                            N - n0, (f - m0) * 2, lane);
      wave_lds_fence();
    });
  }
};

// ---- parts of K joined ------------------------------------------------------------
// out = sum over parts of slab[part][i], in order, for 8 entries a thread; float32 or
// bf16, or added to float32.  The entries from `split` on belong to a second matrix.
struct JoinArgs {
  const float* slab;
  int64_t total, split;
  int parts;
  unsigned char *out, *out2;
  int f32, add;
};
__global__ __launch_bounds__(256) void ffn_join_kernel(JoinArgs a) {
  const int64_t v = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (v >= a.total) return;
  Vec8 s{};
  for (int p = 0; p < a.parts; ++p) {
    const Vec8 x = unpack8(load8<F32>(reinterpret_cast<const unsigned char*>(a.slab + p * a.total), v / 8));
#pragma unroll
    for (int i = 0; i < 8; ++i) s.v[i] += x.v[i];
  }
  const bool second = v >= a.split;   // split % 8 == 0
  unsigned char* out = second ? a.out2 : a.out;
  const int64_t at = (second ? v - a.split : v) / 8;
  if (a.f32) {
    if (a.add) {
      const Vec8 x = unpack8(load8<F32>(out, at));
#pragma unroll
      for (int i = 0; i < 8; ++i) s.v[i] += x.v[i];
    }
    store8<F32>(out, at, s);
  } else {
    store8<Bf16>(out, at, s);
  }
}

// ---- plan ---------------------------------------------------------------------------
// Tile and K parts of a product of M x N entries over nk stages.  fused: the epilogue
// needs whole sums, so K is not split.
struct Plan {
  int big;       // 256 x 256 tiles (one work-group to a CU), else 128 x 128 (two)
  int tiles_m, tiles_n, parts;
};
constexpr int64_t kSlabBytes = int64_t(256) << 20;   // most that the parts of one product take

Plan plan_of(int64_t M, int64_t N, int nk, bool fused) {
  auto tiles = [&](int t) { return ((M + t - 1) / t) * ((N + t - 1) / t); };
  Plan p{};
  p.big = tiles(256) >= 224;
  const int t = p.big ? 256 : 128;
  p.tiles_m = (int)((M + t - 1) / t);
  p.tiles_n = (int)((N + t - 1) / t);
  p.parts = 1;
  if (!fused) {
    const int64_t have = tiles(t), slots = p.big ? 256 : 512;
    int64_t s = slots / std::max<int64_t>(have, 1);
    s = std::min<int64_t>(s, nk / 4);                          // four stages at least per part
    s = std::min<int64_t>(s, kSlabBytes / std::max<int64_t>(M * N * 4, 1));
    s = std::min<int64_t>(s, 64);
    p.parts = (int)std::max<int64_t>(s, 1);
  }
  return p;
}

template <bool kOuterA, bool kOuterB, bool kPairA, class Epi>
int launch(RowShape g, const Plan& p, const Epi& epi, const char* name, hipStream_t stream) {
  g.tiles_m = p.tiles_m;
  g.tiles_n = p.tiles_n;
  g.parts = p.parts;
  const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
  PSPO_REQUIRE(total < (int64_t(1) << 23), PSPO_ERR_UNSUPPORTED, "the product has more tiles than a launch holds");
  const dim3 grid((uint32_t)((total + kNumXcd - 1) / kNumXcd * kNumXcd), (uint32_t)p.parts);
  if (total == 0) return PSPO_OK;
  if (p.big)
    hipLaunchKernelGGL((row_gemm_kernel<8, 8, kOuterA, kOuterB, kPairA, Epi>), grid, dim3(256), 0, stream, g, epi);
  else
    hipLaunchKernelGGL((row_gemm_kernel<4, 4, kOuterA, kOuterB, kPairA, Epi>), grid, dim3(256), 0, stream, g, epi);
  PSPO_LAUNCHED(name, stream);
  return PSPO_OK;
}

// A product whose output is stored as it is: out[n][m], bf16 or float32 (or added to
// it); rows n >= split go to out2.  The slabs of K parts lie in `slab`.
struct Out {
  void *out, *out2;
  int split;
  bool f32, add;
};
template <bool kOuterA, bool kOuterB>
int product(RowShape g, int M, int N, const Out& o, float* slab, const char* name, hipStream_t stream) {
  const int nk = (g.K + kRowK - 1) / kRowK * g.segs;
  const Plan p = plan_of(M, N, nk, false);
  if (p.parts > 1) {
    EpiF32 e{slab, slab, M, (int64_t)M * N, M, N, N, 0};
    if (int rc = launch<kOuterA, kOuterB, false>(g, p, e, name, stream)) return rc;
    JoinArgs j{slab, (int64_t)M * N, (int64_t)M * o.split, p.parts, static_cast<unsigned char*>(o.out),
               static_cast<unsigned char*>(o.out2), o.f32, o.add};
    hipLaunchKernelGGL(ffn_join_kernel, dim3((uint32_t)((j.total / 8 + 255) / 256)), dim3(256), 0, stream, j);
    PSPO_LAUNCHED("ffn_join_kernel", stream);
    return PSPO_OK;
  }
  if (o.f32) {
    EpiF32 e{static_cast<float*>(o.out), static_cast<float*>(o.out2), M, 0, M, N, o.split, o.add};
    return launch<kOuterA, kOuterB, false>(g, p, e, name, stream);
  }
  EpiBf16 e{static_cast<uint16_t*>(o.out), static_cast<uint16_t*>(o.out2), M, M, N, o.split};
  return launch<kOuterA, kOuterB, false>(g, p, e, name, stream);
}

int64_t slab_bytes(int64_t M, int64_t N, int K, int segs) {
  const Plan p = plan_of(M, N, (K + kRowK - 1) / kRowK * segs, false);
  return p.parts > 1 ? p.parts * M * N * 4 : 0;
}

// Workspace layout of one call.
struct Space {
  int64_t h, dgu, pre, slab, total;
};
Space space_of(int64_t N, int64_t d, int64_t f, bool backward, bool kept) {
  Space s{};
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t a = at;
    at = round_up(at + bytes, 256);
    return a;
  };
  s.h = take(N * f * 2);
  int64_t slab = 0;
  if (backward) {
    s.dgu = take(N * 2 * f * 2);
    if (!kept) s.pre = take(N * 2 * f * 4);
    slab = std::max({slab_bytes(d, N, (int)f, 2), slab_bytes(d, 2 * f, (int)N, 1), slab_bytes(f, d, (int)N, 1)});
  } else {
    slab = slab_bytes(d, N, (int)f, 1);
  }
  s.slab = take(slab);
  s.total = at;
  return s;
}

constexpr int kMaxWidth = 1 << 20;   // d and f: a tile's rows stay below 2^31 bytes

int check_sizes(int32_t N, int32_t d, int32_t f, int32_t act) {
  PSPO_REQUIRE(N >= 0, PSPO_ERR_INVALID_ARG, "N must be >= 0");
  PSPO_REQUIRE(d > 0 && f > 0 && d % 8 == 0 && f % 8 == 0, PSPO_ERR_UNSUPPORTED,
               "the block needs d > 0, f > 0, d % 8 == 0 and f % 8 == 0");
  PSPO_REQUIRE(d <= kMaxWidth && f <= kMaxWidth, PSPO_ERR_UNSUPPORTED, "d and f are at most 2^20");
  PSPO_REQUIRE(act == PSPO_ACT_SILU || act == PSPO_ACT_GELU_TANH, PSPO_ERR_INVALID_ARG, "unknown activation");
  return PSPO_OK;
}

RowShape shape(const uint16_t* a, const uint16_t* a2, int64_t lda, int rows_a, const uint16_t* b, int64_t ldb, int rows_b,
               int K, int segs = 1, int64_t seg_b = 0) {
  RowShape g{};
  g.a = RowOperand{{a, a2}, lda, rows_a, 0};
  g.b = RowOperand{{b, b}, ldb, rows_b, seg_b};
  g.K = K;
  g.segs = segs;
  return g;
}

// h (and the pre-activations, if `pre`) of the first N tokens.
int gate_up(const uint16_t* x, const uint16_t* wg, const uint16_t* wu, int N, int d, int f, int act, uint16_t* h,
            float* pre, hipStream_t stream) {
  const RowShape g = shape(wg, wu, d, f, x, d, N, d);
  const Plan p = plan_of(2 * (int64_t)f, N, (d + kRowK - 1) / kRowK, true);
  return launch<false, false, true>(g, p, EpiGateUp{h, pre, f, N, act}, "ffn_gate_up", stream);
}

}  // namespace
}  // namespace pspo

extern "C" {

size_t pspo_gated_ffn_workspace_bytes(int32_t N, int32_t d, int32_t f, uint32_t flags) {
  using namespace pspo;
  if (N < 0 || d <= 0 || f <= 0 || d > kMaxWidth || f > kMaxWidth) return 0;
  const bool bwd = (flags & PSPO_FFN_BACKWARD) != 0;
  return (size_t)space_of(N, d, f, bwd, (flags & PSPO_FFN_PREACT) != 0).total;
}

int pspo_gated_ffn_fwd(const uint16_t* x, const uint16_t* w_gate, const uint16_t* w_up, const uint16_t* w_down, int32_t N,
                       int32_t d, int32_t f, int32_t act, uint16_t* y, float* preact, void* workspace,
                       size_t workspace_bytes, hipStream_t stream) {
  using namespace pspo;
  clear_last_error();
  TraceRange trace_range("pspo_gated_ffn_fwd");
  if (int rc = check_sizes(N, d, f, act)) return rc;
  if (N == 0) return PSPO_OK;
  PSPO_REQUIRE(x && w_gate && w_up && w_down && y && workspace, PSPO_ERR_INVALID_ARG, "null pointer argument");
  PSPO_REQUIRE(aligned(x, 16) && aligned(w_gate, 16) && aligned(w_up, 16) && aligned(w_down, 16) && aligned(y, 16) &&
                   aligned(preact, 16) && aligned(workspace, 256),
               PSPO_ERR_INVALID_ARG, "misaligned pointer argument");
  const Space s = space_of(N, d, f, false, false);
  PSPO_REQUIRE((int64_t)workspace_bytes >= s.total, PSPO_ERR_WORKSPACE,
               "workspace is smaller than pspo_gated_ffn_workspace_bytes()");
  if (int rc = require_gfx950()) return rc;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  uint16_t* h = reinterpret_cast<uint16_t*>(ws + s.h);
  float* slab = reinterpret_cast<float*>(ws + s.slab);
  if (int rc = gate_up(x, w_gate, w_up, N, d, f, act, h, preact, stream)) return rc;
  return product<false, false>(shape(w_down, w_down, f, d, h, f, N, f), d, N, Out{y, y, N, false, false}, slab,
                               "ffn_down", stream);
}

int pspo_gated_ffn_bwd(const uint16_t* dy, const uint16_t* x, const uint16_t* w_gate, const uint16_t* w_up,
                       const uint16_t* w_down, const float* preact, int32_t N, int32_t d, int32_t f, int32_t act,
                       uint32_t flags, uint16_t* dx, void* dw_gate, void* dw_up, void* dw_down, void* workspace,
                       size_t workspace_bytes, hipStream_t stream) {
  using namespace pspo;
  clear_last_error();
  TraceRange trace_range("pspo_gated_ffn_bwd");
  if (int rc = check_sizes(N, d, f, act)) return rc;
  PSPO_REQUIRE((flags & ~(PSPO_FFN_DW_F32 | PSPO_ACCUMULATE_DW)) == 0, PSPO_ERR_INVALID_ARG, "unknown flag bits");
  const bool f32 = (flags & PSPO_FFN_DW_F32) != 0, add = (flags & PSPO_ACCUMULATE_DW) != 0;
  PSPO_REQUIRE(f32 || !add, PSPO_ERR_INVALID_ARG, "accumulating needs float32 weight gradients");
  PSPO_REQUIRE(w_gate && w_up && w_down && dw_gate && dw_up && dw_down && workspace, PSPO_ERR_INVALID_ARG,
               "null pointer argument");
  PSPO_REQUIRE(N == 0 || (dy && x && dx), PSPO_ERR_INVALID_ARG, "null pointer argument");
  PSPO_REQUIRE(aligned(dy, 16) && aligned(x, 16) && aligned(w_gate, 16) && aligned(w_up, 16) && aligned(w_down, 16) &&
                   aligned(preact, 16) && aligned(dx, 16) && aligned(dw_gate, 16) && aligned(dw_up, 16) &&
                   aligned(dw_down, 16) && aligned(workspace, 256),
               PSPO_ERR_INVALID_ARG, "misaligned pointer argument");
  const Space s = space_of(N, d, f, true, preact != nullptr);
  PSPO_REQUIRE((int64_t)workspace_bytes >= s.total, PSPO_ERR_WORKSPACE,
               "workspace is smaller than pspo_gated_ffn_workspace_bytes()");
  if (int rc = require_gfx950()) return rc;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  uint16_t *h = reinterpret_cast<uint16_t*>(ws + s.h), *dgu = reinterpret_cast<uint16_t*>(ws + s.dgu);
  float* slab = reinterpret_cast<float*>(ws + s.slab);
  if (N > 0) {
    const float* pre = preact;
    if (pre == nullptr) {
      float* own = reinterpret_cast<float*>(ws + s.pre);
      if (int rc = gate_up(x, w_gate, w_up, N, d, f, act, h, own, stream)) return rc;
      pre = own;
    }
    const Plan p = plan_of(f, N, (d + kRowK - 1) / kRowK, true);
    if (int rc = launch<true, false, false>(shape(w_down, w_down, f, f, dy, d, N, d), p, EpiDh{pre, dgu, h, f, N, act},
                                            "ffn_dh", stream))
      return rc;
    if (int rc = product<true, false>(shape(w_gate, w_up, d, d, dgu, 2 * (int64_t)f, N, f, 2, f), d, N,
                                      Out{dx, dx, N, false, false}, slab, "ffn_dx", stream))
      return rc;
  }
  if (int rc = product<true, true>(shape(x, x, d, d, dgu, 2 * (int64_t)f, 2 * f, N), d, 2 * f,
                                   Out{dw_gate, dw_up, f, f32, add}, slab, "ffn_dw_gate_up", stream))
    return rc;
  return product<true, true>(shape(h, h, f, f, dy, d, d, N), f, d, Out{dw_down, dw_down, d, f32, add}, slab,
                             "ffn_dw_down", stream);
}

}  // extern "C"
