// Launches of the row-major products (rowgemm.h, skinny.h): the epilogue that stores, K parts and
// their joins, one product as its plan (row_plan.h) covers it.  The names are internal to each source
// file that includes this.
#pragma once

#include <type_traits>

#include "row_plan.h"
#include "skinny.h"
#include "vec8.h"

namespace pspo {
namespace {

// ---- epilogues -----------------------------------------------------------------
// What becomes of eight entries (m .. m + 7, n) of a product; the same for a tile's accumulators
// (Epi::apply) and for the joined sums of its K parts (row_join_kernel).
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

// The epilogue of a launch: slabs where the tiles are parts, else `op`, by its own way from the
// accumulators (tile, kTile true) or piece by piece.
template <class Op, class = void>
struct HasTile : std::false_type {};
template <class Op>
struct HasTile<Op, std::enable_if_t<Op::kTile>> : std::true_type {};

template <class Op, class = void>
struct HasExtra : std::false_type {};
template <class Op>
struct HasExtra<Op, std::enable_if_t<Op::kExtra>> : std::true_type {};

// Two row blocks of a column (packed bf16: rows 4 g .. 4 g + 3 of lane group g = lane / 16) to eight
// consecutive rows a lane, from row 16 (g % 2) + 8 (g / 2) of the pair on.
__device__ __forceinline__ u32x4 eight_rows(const u32x2& a, const u32x2& b) {
  const auto x = __builtin_amdgcn_permlane16_swap(a.x, b.x, false, false);
  const auto y = __builtin_amdgcn_permlane16_swap(a.y, b.y, false, false);
  return u32x4{x[0], y[0], x[1], y[1]};
}
__device__ __forceinline__ int eight_rows_at(int lane) { return ((lane >> 4) & 1) * 16 + (lane >> 5) * 8; }

template <class Op>
struct Epi {
  static constexpr bool kExtra = HasExtra<Op>::value;
  Op op;
  Slab slab;
  __device__ __forceinline__ void extra(unsigned char* lds) const {
    if constexpr (kExtra) op.extra(lds);
  }
  template <int BM, int BN>
  __device__ __forceinline__ void direct(f32x4 (&acc)[BM][BN], int tm, int tn, int wm, int wn, int lane) const {
    op.template tile<BM, BN>(acc, tm, tn, wm, wn, lane);
  }
  template <int BM, int BN>
  __device__ __forceinline__ void apply(f32x4 (&acc)[BM][BN], int tm, int tn, int wm, int wn, int lane,
                                        unsigned char* lds, int index) const {
    if (slab.base != nullptr) put_slab(acc, tn, wm, wn, lane, index, slab);
    else if constexpr (HasTile<Op>::value) op.template tile<BM, BN>(acc, tm, tn, wm, wn, lane);
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
__global__ __launch_bounds__(256) void row_join_kernel(JoinShape a, Op op) {
  join_tile(a, op, blockIdx.x, blockIdx.y);
}
// The joins of several products in one launch (grid x: their tiles one after another).
template <class Op>
struct JoinJobs {
  JoinShape a[3];
  Op op[3];
};
template <class Op>
__global__ __launch_bounds__(256) void row_join_jobs_kernel(JoinJobs<Op> j) {
  int index = blockIdx.x, job = 0;
  while (index >= j.a[job].g.count) index -= j.a[job++].g.count;   // the counts add up to the grid
  join_tile(j.a[job], j.op[job], index, blockIdx.y);
}
template <class Op>
int join_parts(const Op& op, const RowShape& g, int tile, int tile_n, const float* slab, hipStream_t stream) {
  hipLaunchKernelGGL((row_join_kernel<Op>),
                     dim3((uint32_t)g.count, (uint32_t)join_blocks(Op::kPair ? tile / 2 : tile, tile_n)), dim3(256), 0,
                     stream, JoinShape{slab, g, tile, tile_n}, op);
  PSPO_LAUNCHED("row_join_kernel", stream);
  return PSPO_OK;
}

constexpr int kChainK = 32 * kRowK;   // longest K of the products that go in chains of tiles
template <bool kOuterA, bool kOuterB, class Op>
int launch(const RowShape& g, const Plan& p, const Epi<Op>& epi, const char* name, hipStream_t stream) {
  const dim3 grid((uint32_t)round_up(g.count, kNumXcd), (uint32_t)g.parts);
  const bool deep = deep_ring((int64_t)g.count * g.parts);
  if constexpr (HasTile<Op>::value) {
    // A work-group to a CU with tiles in turn, for the K where their way in and out counts: whole calls at
    // 7,400 rows, d = 416, V = 21520 412 -> 393 us, 777, 1536, 151936 1,250 -> 1,240; with 56 stages work-groups
    // of a tile each, taken when a CU is free, are better (4,096, 3584, 152064: 10,364 against 10,440).
    if (p.tile == 256 && g.parts == 1 && g.count > 256 && g.segs == 1 && g.K > kRowK && g.K <= kChainK) {
#define PSPO_CHAIN(BN)                                                                                     \
  hipLaunchKernelGGL((row_chain_kernel<8, BN, 2, kOuterA, kOuterB, Epi<Op>>), dim3(256), dim3(256), 0, stream, g, epi)
      if constexpr (!kOuterA) {
        if (p.tile_n == 160) PSPO_CHAIN(5);
        if (p.tile_n == 192) PSPO_CHAIN(6);
        if (p.tile_n == 224) PSPO_CHAIN(7);
      }
      if (p.tile_n == 256) PSPO_CHAIN(8);
#undef PSPO_CHAIN
      PSPO_LAUNCHED(name, stream);
      return PSPO_OK;
    }
  }
#define PSPO_ROW(BM, BN, RING)                                                                                    \
  hipLaunchKernelGGL((row_gemm_kernel<BM, BN, RING, kOuterA, kOuterB, Op::kPair, Epi<Op>>), grid, dim3(256), 0, \
                     stream, g, epi)
  if (p.tile == 256) {
    if constexpr (!kOuterA && HasTile<Op>::value) {   // (the pieces of row_pieces take 128 columns at a time)
      if (p.tile_n == 160) PSPO_ROW(8, 5, 2);
      if (p.tile_n == 192) PSPO_ROW(8, 6, 2);
      if (p.tile_n == 224) PSPO_ROW(8, 7, 2);
    }
    if (p.tile_n == 256) PSPO_ROW(8, 8, 2);
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

// One product with its epilogue, covered as `p` says: the whole tiles, then the rest in parts and their join.
template <bool kOuterA, bool kOuterB, class Op>
int product(RowShape g, const Plan& p, int64_t N, const Op& op, float* slab, const char* name, hipStream_t stream) {
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

// Up to three products in one launch and their joins in another.
template <class Op>
int run_jobs(const JobPlan& p, const RowShape (&g)[3], const Op (&o)[3], unsigned char* slabs, const char* name,
             hipStream_t stream) {
  RowJobs<Epi<Op>> jobs{};
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
  if (Epi<Op>::kExtra) ++blocks;
  const dim3 threads(256);
  bool chained = false;
  if constexpr (HasTile<Op>::value) {
    // The second of two products in chains of four tiles, all but its last two rounds (which fill the chip):
    // whole calls at 777 rows, d = 1536, V = 151936 1,240 -> 1,229 us, 1,999 rows 2,591 -> 2,568 (chains of two
    // 1,238 and 2,581).
    constexpr int kLinks = 4, kBehind = 512;
    RowShape &r = jobs.g[1], &rest = jobs.g[2];
    if (p.tile == 256 && p.parts[1] == 1 && rest.count == 0 && r.count > 2 * kBehind && r.segs == 1 && r.K > kRowK &&
        r.K <= kChainK) {
      chained = true;
      rest = r;
      r.count -= kBehind;
      rest.tile0 = r.count;
      rest.count = kBehind;
      jobs.epi[2] = jobs.epi[1];
      blocks -= jobs.blocks[1];
      jobs.blocks[1] = (int)round_up((r.count + kLinks - 1) / kLinks, kNumXcd);
      jobs.blocks[2] = kBehind;
      blocks += jobs.blocks[1] + jobs.blocks[2];
      hipLaunchKernelGGL((row_jobs_kernel<8, 8, 2, true, Epi<Op>>), dim3((uint32_t)blocks), threads, 0, stream, jobs);
    }
  }
  const dim3 grid((uint32_t)blocks);
  if (chained) {   // launched above
  } else if (p.tile == 256) {
    hipLaunchKernelGGL((row_jobs_kernel<8, 8, 2, false, Epi<Op>>), grid, threads, 0, stream, jobs);
  } else if (deep_ring(blocks)) {
    hipLaunchKernelGGL((row_jobs_kernel<4, 4, kDeep, false, Epi<Op>>), grid, threads, 0, stream, jobs);
  } else {
    hipLaunchKernelGGL((row_jobs_kernel<4, 4, 2, false, Epi<Op>>), grid, threads, 0, stream, jobs);
  }
  PSPO_LAUNCHED(name, stream);
  JoinJobs<Op> join{};
  int split = 0;
  int64_t tiles = 0;
  for (int i = 0; i < 3; ++i)
    if (p.parts[i] > 1 && jobs.g[i].count > 0) {
      join.a[split] = JoinShape{reinterpret_cast<float*>(slabs + p.slab[i]), jobs.g[i], p.tile, p.tile};
      join.op[split++] = o[i];
      tiles += jobs.g[i].count;
    }
  if (split > 0) {
    hipLaunchKernelGGL(row_join_jobs_kernel<Op>, dim3((uint32_t)tiles, (uint32_t)join_blocks(p.tile, p.tile)), dim3(256), 0,
                       stream, join);
    PSPO_LAUNCHED("row_join_jobs_kernel", stream);
  }
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

// ---- few tokens -----------------------------------------------------------------------
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

}  // namespace
}  // namespace pspo
