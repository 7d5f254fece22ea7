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
#include <cmath>
#include <type_traits>

#include "ffn_plan.h"
#include "pspo_layer.h"
#include "rowproduct.h"

namespace pspo {
namespace {

// act(g) = g s(a(g)), s the logistic function: a(g) = g (silu), or
// 2 sqrt(2/pi) (g + 0.044715 g^3) (gelu_tanh, as 1 + tanh(v) = 2 s(2 v)).
// The exponential and the reciprocal are the instructions (both good to an ulp or so of
// float32): with an IEEE division the dh product of 8192 tokens, one wave to a SIMD in its
// epilogue, took 992 us instead of 956.
__device__ __forceinline__ float logistic(float a) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(a * -1.4426950408889634f));
}

constexpr float kGelu = 1.5957691216057308f;   // 2 sqrt(2 / pi)

// Beyond 16 the logistic is 0 or 1; the bound keeps the cube finite (and a NaN a NaN).
__device__ __forceinline__ float gelu_bound(float g) { return g > 16.f ? 16.f : (g < -16.f ? -16.f : g); }

__device__ __forceinline__ float act_value(float g, int kind) {
  if (kind == PSPO_ACT_SILU) return g * logistic(g);
  const float b = gelu_bound(g);
  return g * logistic(kGelu * (b + 0.044715f * b * b * b));
}
__device__ __forceinline__ void act_both(float g, int kind, float& a, float& da) {
  if (kind == PSPO_ACT_SILU) {
    const float s = logistic(g);
    a = g * s;
    da = s + a * (1.f - s);
    return;
  }
  const float b = gelu_bound(g);
  const float s = logistic(kGelu * (b + 0.044715f * b * b * b));
  a = g * s;
  da = s + b * s * (1.f - s) * (kGelu * (1.f + 0.134145f * b * b));
}

// ---- epilogues -----------------------------------------------------------------
// Loads and stores go through the caches: where what a product writes fits them the next one finds it there (1443
// tokens, d = 88, f = 3768: the dh product 35.8 -> 20.9 us against accesses past the caches; 777
// tokens, d = 1000, f = 4104: 30.0 -> 23.6, the products behind it 66.5 -> 62.2), and at 8192 tokens,
// d = 3584, f = 14336, where nothing fits, the two differ by 1.4% at most.
// Row blocks in pairs (gate, up): h[n][m] = act(g) u, and the pre-activations if kept.
struct EpiGateUp {
  static constexpr bool kPair = true;
  uint16_t* h;
  float* pre;     // [N][2 f] or NULL
  int f, N, act;
  using Fetched = Nothing;
  __device__ __forceinline__ Nothing fetch(int64_t, int64_t) const { return {}; }
  __device__ __forceinline__ void piece(int64_t n, int64_t m, const f32x4* v, Nothing) const {
    if (n >= N || m >= f) return;
    if (pre != nullptr) {
      float* row = pre + n * 2 * f + m;
      put_f32(row, v);
      put_f32(row + f, v + 2);
    }
    const float *g = reinterpret_cast<const float*>(v), *u = g + 8;
    float o[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = act_value(g[k], act) * u[k];
    put_bf16(h + n * f + m, o);
  }
};

// C(m, n) = dh: dgu[n] = (dh u act'(g), dh act(g)), h[n] = act(g) u.
struct EpiDh {
  static constexpr bool kPair = false;
  const float* pre;   // [N][2 f]
  uint16_t *dgu, *h;  // [N][2 f], [N][f]
  int f, N, act;
  struct Fetched {
    f32x4 g[2], u[2];
  };
  __device__ __forceinline__ Fetched fetch(int64_t n, int64_t m) const {
    Fetched x{};
    if (n < N && m < f) {
      const f32x4* row = reinterpret_cast<const f32x4*>(pre + n * 2 * f + m);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        x.g[k] = row[k];
        x.u[k] = row[f / 4 + k];
      }
    }
    return x;
  }
  __device__ __forceinline__ void piece(int64_t n, int64_t m, const f32x4* v, const Fetched& x) const {
    if (n >= N || m >= f) return;
    float dg[8], du[8], hv[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float a, da;
      act_both(x.g[k / 4][k % 4], act, a, da);
      const float dh = v[k / 4][k % 4], u = x.u[k / 4][k % 4];
      dg[k] = dh * u * da;
      du[k] = dh * a;
      hv[k] = a * u;
    }
    uint16_t* row = dgu + n * 2 * f + m;
    put_bf16(row, dg);
    put_bf16(row + f, du);
    put_bf16(h + n * f + m, hv);
  }
};

// One product with its epilogue.
template <bool kOuterA, bool kOuterB, class Op>
int product(const RowShape& g, int64_t M, int64_t N, const Op& op, float* slab, const char* name, hipStream_t stream) {
  if (M == 0 || N == 0) return PSPO_OK;
  return product<kOuterA, kOuterB>(g, plan_of(M, N, (g.K + kRowK - 1) / kRowK, std::is_same_v<Op, EpiDh>), N, op, slab,
                                   name, stream);
}

struct SkinnyGateUp {
  uint16_t* h;
  float* pre;
  int f, act;
  __device__ __forceinline__ void operator()(int m, int n, const float (&s)[2]) const {
    if (pre != nullptr) {
      pre[(int64_t)n * 2 * f + m] = s[0];
      pre[(int64_t)n * 2 * f + f + m] = s[1];
    }
    h[(int64_t)n * f + m] = (uint16_t)pack_bf16(act_value(s[0], act) * s[1], 0.f);
  }
};
struct SkinnyStore {
  uint16_t* y;
  int ld;
  __device__ __forceinline__ void operator()(int m, int n, const float (&s)[1]) const {
    y[(int64_t)n * ld + m] = (uint16_t)pack_bf16(s[0], 0.f);
  }
};

constexpr int kMaxWidth = 1 << 20;   // d and f: a tile's rows stay below 2^31 bytes

int check_sizes(int32_t N, int32_t d, int32_t f, int32_t act) {
  PSPO_REQUIRE(N >= 0, PSPO_ERR_INVALID_ARG, "N must be >= 0");
  PSPO_REQUIRE(d > 0 && f > 0 && d % 8 == 0 && f % 8 == 0, PSPO_ERR_UNSUPPORTED,
               "the block needs d > 0, f > 0, d % 8 == 0 and f % 8 == 0");
  PSPO_REQUIRE(d <= kMaxWidth && f <= kMaxWidth, PSPO_ERR_UNSUPPORTED, "d and f are at most 2^20");
  PSPO_REQUIRE(act == PSPO_ACT_SILU || act == PSPO_ACT_GELU_TANH, PSPO_ERR_INVALID_ARG, "unknown activation");
  return PSPO_OK;
}

// h (and the pre-activations, if `pre`) of the first N tokens.
int gate_up(const uint16_t* x, const uint16_t* wg, const uint16_t* wu, int N, int d, int f, int act, uint16_t* h,
            float* pre, float* slab, hipStream_t stream) {
  if (few_tokens(N, d, f))
    return skinny<2>(SkinnyArgs{{wg, wu}, x, f, N, d}, SkinnyGateUp{h, pre, f, act}, "ffn_gate_up", stream);
  return product<false, false>(shape(wg, wu, d, f, x, d, N, d), 2 * (int64_t)f, N, EpiGateUp{h, pre, f, N, act}, slab,
                               "ffn_gate_up", stream);
}

}  // namespace
}  // namespace pspo

extern "C" {

size_t pspo_gated_ffn_workspace_bytes(int32_t N, int32_t d, int32_t f, uint32_t flags) {
  using namespace pspo;
  if (N < 0 || d <= 0 || f <= 0 || d % 8 != 0 || f % 8 != 0 || d > kMaxWidth || f > kMaxWidth) return 0;
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
  if (int rc = gate_up(x, w_gate, w_up, N, d, f, act, h, preact, slab, stream)) return rc;
  if (few_tokens(N, d, f))
    return skinny<1>(SkinnyArgs{{w_down, w_down}, h, d, N, f}, SkinnyStore{y, d}, "ffn_down", stream);
  return product<false, false>(shape(w_down, w_down, f, d, h, f, N, f), d, N, EpiStore{y, y, d, d, N, N, 0, 0}, slab,
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
  PSPO_REQUIRE(w_gate && w_up && w_down && dw_gate && dw_up && dw_down, PSPO_ERR_INVALID_ARG,
               "null pointer argument");
  PSPO_REQUIRE(N == 0 || (dy && x && dx && workspace), PSPO_ERR_INVALID_ARG, "null pointer argument");
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
      if (int rc = gate_up(x, w_gate, w_up, N, d, f, act, h, own, slab, stream)) return rc;
      pre = own;
    }
    if (int rc = product<true, false>(shape(w_down, w_down, f, f, dy, d, N, d), f, N, EpiDh{pre, dgu, h, f, N, act}, slab,
                                      "ffn_dh", stream))
      return rc;
  }
  const RowShape g[3] = {shape(w_gate, w_up, d, d, dgu, 2 * (int64_t)f, N, f, 2, f),
                         shape(x, x, d, d, dgu, 2 * (int64_t)f, 2 * f, N), shape(h, h, f, f, dy, d, d, N)};
  const EpiStore o[3] = {{dx, dx, d, d, N, N, 0, 0},
                         {dw_gate, dw_up, d, d, 2 * f, f, f32, add},
                         {dw_down, dw_down, f, f, d, d, f32, add}};
  return run_jobs(plan_backward(N, d, f), g, o, reinterpret_cast<unsigned char*>(slab), "ffn_gradients", stream);
}

}  // extern "C"
