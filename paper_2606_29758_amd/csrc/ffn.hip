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
#include "vec8.h"

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
// What becomes of eight entries (m .. m + 7, n) of a product; the same for a tile's
// accumulators (apply) and for the joined sums of its K parts (ffn_join_kernel).  Loads and stores
// go through the caches: where what a product writes fits them the next one finds it there (1443
// tokens, d = 88, f = 3768: the dh product 35.8 -> 20.9 us against accesses past the caches; 777
// tokens, d = 1000, f = 4104: 30.0 -> 23.6, the products behind it 66.5 -> 62.2), and at 8192 tokens,
// d = 3584, f = 14336, where nothing fits, the two differ by 1.4% at most.
struct Nothing {};

__device__ __forceinline__ void put_f32(float* to, const f32x4* v) {
  reinterpret_cast<f32x4*>(to)[0] = v[0];
  reinterpret_cast<f32x4*>(to)[1] = v[1];
}
__device__ __forceinline__ void put_bf16(uint16_t* to, const float* v) {
  u32x4 p;
#pragma unroll
  for (int k = 0; k < 4; ++k) p[k] = pack_bf16(v[2 * k], v[2 * k + 1]);
  *reinterpret_cast<u32x4*>(to) = p;
}

// C(m, n) -> out[n * ld + m], bf16 or float32 (or added to it); rows n >= split belong to a
// second matrix.
struct EpiStore {
  static constexpr bool kPair = false;
  void *out, *out2;
  int64_t ld;
  int M, N, split, f32, add;
  using Fetched = Nothing;
  __device__ __forceinline__ Nothing fetch(int64_t, int64_t) const { return {}; }
  __device__ __forceinline__ void piece(int64_t n, int64_t m, const f32x4* v, Nothing) const {
    if (n >= N || m >= M) return;   // M % 8 == 0
    void* base = n < split ? out : out2;
    const int64_t at = (n < split ? n : n - split) * ld + m;
    if (f32) {
      float* to = static_cast<float*>(base) + at;
      f32x4 s[2] = {v[0], v[1]};
      if (add) {
        s[0] += reinterpret_cast<const f32x4*>(to)[0];
        s[1] += reinterpret_cast<const f32x4*>(to)[1];
      }
      put_f32(to, s);
    } else {
      put_bf16(static_cast<uint16_t*>(base) + at, reinterpret_cast<const float*>(v));
    }
  }
};

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

// A K part's whole tile in float32 to slab number `slab`: the 16 x 16 blocks one after
// another (those of a column of blocks together), each as its lanes hold it, so that a store
// writes 1 KB in one piece.  slab_piece says where four entries lie.
struct Slab {
  float* base;
  int N;
};
template <int BM, int BN>
__device__ __forceinline__ void put_slab(const f32x4 (&acc)[BM][BN], int tn, int wm, int wn, int lane, int slab,
                                         const Slab& s) {
  float* to = s.base + (int64_t)slab * (1024 * BM * BN) + (wn * BN * 2 * BM + wm * BM) * 256 + lane * 4;
  repeat<BN>([&](auto jc) {
    constexpr int j = decltype(jc)::value;
    if (((tn * 2 + wn) * BN + j) * 16 >= s.N) return;   // nobody joins columns that do not exist
#pragma unroll
    for (int i = 0; i < BM; ++i) {
      f32x4 v;
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = acc_read(acc[i][j][r]);
      *reinterpret_cast<f32x4*>(to + (j * 2 * BM + i) * 256) = v;
    }
  });
}
// Offset of entries (m .. m + 3, n) of a tile of `tile` rows, m % 4 == 0.
__device__ __forceinline__ int slab_piece(int tile, int m, int n) {
  return ((n >> 4) * (tile >> 4) + (m >> 4)) * 256 + (((m >> 2) & 3) * 16 + (n & 15)) * 4;
}

// The epilogue of a launch: slabs where the tiles are parts, else `op`.
template <class Op>
struct Epi {
  Op op;
  Slab slab;
  template <int BM, int BN>
  __device__ __forceinline__ void apply(f32x4 (&acc)[BM][BN], int tm, int tn, int wm, int wn, int lane,
                                        unsigned char* lds, int index) const {
    if (slab.base != nullptr) put_slab(acc, tn, wm, wn, lane, index, slab);
    else row_pieces<BM, BN, Op::kPair>(acc, tm, tn, wm, wn, lane, lds, op);
  }
};

// ---- parts of K joined ------------------------------------------------------------
// The slabs of a tile's parts added in order and given to the product's epilogue.
struct JoinShape {
  const float* slab;
  RowShape g;
  int tile, tile_n;
};
template <class Op>
__device__ __forceinline__ void join_tile(const JoinShape& a, const Op& op, int index, int block) {
  int tm, tn;
  row_tile_at(a.g, a.g.tile0 + index, tm, tn);
  // a wave takes 8 columns x 64 entries: whole lines of the output, 128-byte pieces of the slabs
  const int width = Op::kPair ? a.tile / 2 : a.tile;
  const int w = block * 4 + threadIdx.x / 64, lane = threadIdx.x % 64;
  const int col = w / (width / 64) * 8 + lane / 8, m0 = w % (width / 64) * 64 + lane % 8 * 8;
  if (col >= a.tile_n) return;
  const int64_t n = (int64_t)tn * a.tile_n + col, m = (int64_t)tm * width + m0;
  if (n >= op.N) return;   // its slab columns are not written
  // gate and up in turn, 16 rows each; the next four entries of a piece lie 64 floats on
  const int row = Op::kPair ? m0 / 16 * 32 + m0 % 16 : m0;
  const int64_t size = (int64_t)a.tile * a.tile_n;
  const float* from = a.slab + index * size;
  const int p0 = slab_piece(a.tile, row, col), p1 = Op::kPair ? slab_piece(a.tile, row + 16, col) : 0;
  const typename Op::Fetched x = op.fetch(n, m);
  f32x4 v[Op::kPair ? 4 : 2] = {};
  // four parts' loads out before the first is added; the sums in the parts' order
  const int64_t next = a.g.count * size;
  constexpr int kV = Op::kPair ? 4 : 2;
  for (int p = 0; p < a.g.parts; p += 4) {
    f32x4 t[4][kV];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (p + q < a.g.parts) {
        const float* at = from + (p + q) * next;
        t[q][0] = *reinterpret_cast<const f32x4*>(at + p0);
        t[q][1] = *reinterpret_cast<const f32x4*>(at + p0 + 64);
        if constexpr (Op::kPair) {
          t[q][2] = *reinterpret_cast<const f32x4*>(at + p1);
          t[q][3] = *reinterpret_cast<const f32x4*>(at + p1 + 64);
        }
      }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (p + q < a.g.parts)
#pragma unroll
        for (int k = 0; k < kV; ++k) v[k] += t[q][k];
  }
  op.piece(n, m, v, x);
}
// Work-groups for a tile's join: a wave for 8 columns x 64 entries.
inline int join_blocks(int width, int tile_n) { return (width / 64 * (tile_n / 8) + 3) / 4; }

template <class Op>
__global__ __launch_bounds__(256) void ffn_join_kernel(JoinShape a, Op op) {
  join_tile(a, op, blockIdx.x, blockIdx.y);
}
// The joins of several products in one launch (grid x: their tiles one after another).
struct JoinJobs {
  JoinShape a[3];
  EpiStore op[3];
};
__global__ __launch_bounds__(256) void ffn_join_jobs_kernel(JoinJobs j) {
  int index = blockIdx.x, job = 0;
  while (index >= j.a[job].g.count) index -= j.a[job++].g.count;   // the counts add up to the grid
  join_tile(j.a[job], j.op[job], index, blockIdx.y);
}
template <class Op>
int join_parts(const Op& op, const RowShape& g, int tile, int tile_n, const float* slab, hipStream_t stream) {
  hipLaunchKernelGGL((ffn_join_kernel<Op>),
                     dim3((uint32_t)g.count, (uint32_t)join_blocks(Op::kPair ? tile / 2 : tile, tile_n)), dim3(256), 0,
                     stream, JoinShape{slab, g, tile, tile_n}, op);
  PSPO_LAUNCHED("ffn_join_kernel", stream);
  return PSPO_OK;
}

template <bool kOuterA, bool kOuterB, class Op>
int launch(const RowShape& g, const Plan& p, const Epi<Op>& epi, const char* name, hipStream_t stream) {
  const dim3 grid((uint32_t)round_up(g.count, kNumXcd), (uint32_t)g.parts);
  const bool deep = deep_ring((int64_t)g.count * g.parts);
#define PSPO_ROW(BM, BN, RING)                                                                                    \
  hipLaunchKernelGGL((row_gemm_kernel<BM, BN, RING, kOuterA, kOuterB, Op::kPair, Epi<Op>>), grid, dim3(256), 0, \
                     stream, g, epi)
  if (p.tile == 256) {
    PSPO_ROW(8, 8, 2);
  } else if (p.tile_n == 128) {
    if (deep) PSPO_ROW(4, 4, kDeep);
    else PSPO_ROW(4, 4, 2);
  } else if constexpr (!kOuterA) {
    if (deep) PSPO_ROW(4, 2, kDeep);
    else PSPO_ROW(4, 2, 2);
  }
#undef PSPO_ROW
  PSPO_LAUNCHED(name, stream);
  return PSPO_OK;
}

// One product with its epilogue: the whole tiles, then the rest in parts and their join.
template <bool kOuterA, bool kOuterB, class Op>
int product(RowShape g, int64_t M, int64_t N, const Op& op, float* slab, const char* name, hipStream_t stream) {
  if (M == 0 || N == 0) return PSPO_OK;
  const Plan p = plan_of(M, N, (g.K + kRowK - 1) / kRowK, std::is_same_v<Op, EpiDh>);
  const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
  PSPO_REQUIRE(total < (int64_t(1) << 23), PSPO_ERR_UNSUPPORTED, "the product has more tiles than a launch holds");
  g.tiles_m = p.tiles_m;
  g.tiles_n = p.tiles_n;
  g.tile0 = 0;
  g.count = p.whole;
  g.parts = 1;
  if (g.count > 0)
    if (int rc = launch<kOuterA, kOuterB>(g, p, Epi<Op>{op, {nullptr, 0}}, name, stream)) return rc;
  g.tile0 = p.whole;
  g.count = (int)(total - p.whole);
  if (g.count == 0) return PSPO_OK;
  g.parts = p.parts;
  if (int rc = launch<kOuterA, kOuterB>(g, p, Epi<Op>{op, {slab, (int)N}}, name, stream)) return rc;
  return join_parts(op, g, p.tile, p.tile_n, slab, stream);
}

int run_jobs(const JobPlan& p, const RowShape (&g)[3], const EpiStore (&o)[3], unsigned char* slabs,
             hipStream_t stream) {
  RowJobs<Epi<EpiStore>> jobs{};
  int64_t blocks = 0;
  for (int i = 0; i < 3; ++i) {
    const int64_t tiles = (int64_t)p.tiles_m[i] * p.tiles_n[i];
    PSPO_REQUIRE(tiles < (int64_t(1) << 23), PSPO_ERR_UNSUPPORTED, "the product has more tiles than a launch holds");
    RowShape& r = jobs.g[i];
    r = g[i];
    r.tiles_m = p.tiles_m[i];
    r.tiles_n = p.tiles_n[i];
    r.tile0 = 0;
    r.count = (int)tiles;
    r.parts = p.parts[i];
    jobs.blocks[i] = (int)(round_up(tiles, kNumXcd) * p.parts[i]);
    blocks += jobs.blocks[i];
    jobs.epi[i] = {o[i], {p.parts[i] > 1 ? reinterpret_cast<float*>(slabs + p.slab[i]) : nullptr, o[i].N}};
  }
  PSPO_REQUIRE(blocks < (int64_t(1) << 24), PSPO_ERR_UNSUPPORTED, "the products have more tiles than a launch holds");
  if (p.tile == 256)
    hipLaunchKernelGGL((row_jobs_kernel<8, 8, 2, Epi<EpiStore>>), dim3((uint32_t)blocks), dim3(256), 0, stream, jobs);
  else if (deep_ring(blocks))
    hipLaunchKernelGGL((row_jobs_kernel<4, 4, kDeep, Epi<EpiStore>>), dim3((uint32_t)blocks), dim3(256), 0, stream, jobs);
  else
    hipLaunchKernelGGL((row_jobs_kernel<4, 4, 2, Epi<EpiStore>>), dim3((uint32_t)blocks), dim3(256), 0, stream, jobs);
  PSPO_LAUNCHED("ffn_gradients", stream);
  JoinJobs join{};
  int split = 0;
  int64_t tiles = 0;
  for (int i = 0; i < 3; ++i)
    if (p.parts[i] > 1 && jobs.g[i].count > 0) {
      join.a[split] = JoinShape{reinterpret_cast<float*>(slabs + p.slab[i]), jobs.g[i], p.tile, p.tile};
      join.op[split++] = o[i];
      tiles += jobs.g[i].count;
    }
  if (split > 0) {
    hipLaunchKernelGGL(ffn_join_jobs_kernel, dim3((uint32_t)tiles, (uint32_t)join_blocks(p.tile, p.tile)), dim3(256), 0,
                       stream, join);
    PSPO_LAUNCHED("ffn_join_jobs_kernel", stream);
  }
  return PSPO_OK;
}

// ---- few tokens -----------------------------------------------------------------------
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

// Waves of a work-group: enough that the chip holds some 4,096, at most one for each
// step of K and 64 KB of sums.
template <int kMats, class Epi>
int skinny(const SkinnyArgs& a, const Epi& epi, const char* name, hipStream_t stream) {
  const int groups = (a.M + 15) / 16, blocks = (a.N + 15) / 16, steps = (a.K + kSkinnyK - 1) / kSkinnyK;
  int waves = 1;
  while (waves < (blocks > 1 ? 8 : 16) && waves * 2 <= steps && (int64_t)groups * waves < 4096 &&
         waves * 2 * kMats * blocks * 1024 <= 65536)
    waves *= 2;
  const size_t lds = (size_t)waves * kMats * blocks * 1024;
#define PSPO_SKINNY(NB, AHEAD)   hipLaunchKernelGGL((skinny_kernel<kMats, NB, AHEAD, Epi>), dim3(groups), dim3(64 * waves), lds, stream, a, epi)
  switch (blocks) {
    case 1: PSPO_SKINNY(1, 4); break;
    case 2: PSPO_SKINNY(2, 2); break;
    case 3: PSPO_SKINNY(3, 2); break;
    default: PSPO_SKINNY(4, 1); break;
  }
#undef PSPO_SKINNY
  PSPO_LAUNCHED(name, stream);
  return PSPO_OK;
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
  return run_jobs(plan_backward(N, d, f), g, o, reinterpret_cast<unsigned char*>(slab), stream);
}

}  // extern "C"
