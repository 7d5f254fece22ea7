// Training objectives through the LM head: the policy loss with a reference penalty, the
// preference loss on pairs, distillation from top logits; forward and gradient in one call.
//
// All three have the same shape.  With z_i = W h_i, s = 1 / temperature and p_i = softmax(s z_i),
// the loss depends on row i through log p_i at a few ids (one, or a teacher's list), so its logit
// gradient is G_i = a_i p_i with those entries replaced:
//   log-prob l_i of one id o, delta_i = d loss / d l_i:  a_i = -s delta_i,
//       G_io = s delta_i (1 - p_io);
//   divergence from q_i with weight c_i:  a_i = s c_i,  G_ij = s c_i (p_ij - q_ij).
// The entries at the ids stay out of the softmax sums: finalize adds them, in float64 and from the logits that
// the log-probs take, so that with r the others' sum over the entry at o, l_i = -log1p(r) is never positive and
// 1 - p_io = r / (1 + r) keeps its digits as p -> 1.  (Added in float32 from the product's own logit, the target's
// share would differ from its log-prob's by 1e-6 to 1e-5, more than all the others of a peaked row.)
//
// Schedule:
//   1. gather: the rows that take part, copied (zeros for the others: a NaN there must not reach a
//      sum over rows), the logits at the ids, summed in float64, and from them the row's
//      reference c, the nearest integer to the largest of them times s log2(e);
//   2. product Z^T = W H^T; its epilogue writes E = 2^(s log2(e) z - c) in bf16 and, for each group
//      of 64 vocabulary entries, the sum of the unrounded values (zeros for the entries at the ids);
//   3. finalize: the sums and the entries at the ids merged into log sum exp, the objective's terms, the
//      entries at the ids put into E (the preference loss takes three small steps more: sequences, pairs, rows);
//   4. products dH = f E W and dW = E^T (f H): a row's factor f = a 2^(c - lse log2(e)) goes into the
//      epilogue of the first and into the copied hidden rows of the second (of up to 64 rows, whose
//      roundings average out in no sum, into E, in two bf16 parts).
// The matrix-core work is that of the formulas, 6 N d V: no logit is computed twice, and between the
// forward and the gradient products nothing passes over the N V entries (a conversion of them to G,
// with a maximum of each group as reference, took 634 of 13,320 us at 4,999 rows, d = 3584,
// V = 152064, and 142 of 585 at 2,501, 520, 32003).  c is a logit of the row, so its largest E is
// 2^-1/2 at least; a group that would pass 2^32 takes its own reference, and its row is brought to
// one reference in finalize (a power of two: exact).
#include <cfloat>
#include <cmath>

#include "objective_plan.h"
#include "pspo_objective.h"
#include "rowproduct.h"

namespace pspo {
namespace {

constexpr int kMostIds = 64;

// ---- lane exchanges within 8 lanes ------------------------------------------------
__device__ __forceinline__ float lane_move(float x, int which) {
  const int v = __float_as_int(x);
  const int r = which == 0   ? __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true)     // lane ^ 1
                : which == 1 ? __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true)     // lane ^ 2
                             : __builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, true);   // 7 - lane, of 8
  return __int_as_float(r);
}
__device__ __forceinline__ float max_of_8_lanes(float x) {
  x = fmaxf(x, lane_move(x, 0));
  x = fmaxf(x, lane_move(x, 1));
  return fmaxf(x, lane_move(x, 2));
}
__device__ __forceinline__ float sum_of_8_lanes(float x) {
  x += lane_move(x, 0);
  x += lane_move(x, 1);
  return x + lane_move(x, 2);
}

// Sum over the four lanes l % 16, the same in all of them.
__device__ __forceinline__ float across_rows(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// ---- forward product ---------------------------------------------------------------
// 2^(z t - c) with t = log2(e) / temperature in two parts: rounded to float32 alone, t would move
// every exponent of a row by up to 2^-24 of it the same way, 1e-6 of the sum.
struct Exponent {
  float t, t_low;
  __device__ __forceinline__ float operator()(float z, float c) const {
    return __builtin_amdgcn_exp2f(fmaf(z, t_low, fmaf(z, t, -c)));
  }
};
constexpr float kFar = 4294967296.f;   // largest sum of a group in its row's reference

// Eight logits (vocabulary entries m .. m + 7 of row n); the 8 lanes of a group of 64 entries
// hold it together, in a tile's epilogue and in a join alike.
struct EpiSoftmax {
  static constexpr bool kPair = false, kTile = true;
  uint16_t* e;       // [N][ld]
  f32x2* part;       // [N][ld / 64]: reference, sum (a wave that writes a group's has read its bits before)
  const float* c;    // [N]
  const int32_t* id; // [N]: the row's only id, or NULL: a group's part holds the bits of its entries at ids
  int64_t ld;
  int V, N;
  Exponent exponent;
  struct Fetched {
    float c;
    uint32_t at_ids;   // of the eight entries
  };
  static __device__ __forceinline__ uint64_t bit_of(int32_t id, int64_t m) {   // of the group from entry m on
    const uint32_t off = (uint32_t)(id - (int32_t)m);
    return off < (uint32_t)kGroup ? uint64_t(1) << off : 0;
  }
  __device__ __forceinline__ uint64_t listed_at(int64_t n, int64_t m) const {   // of a group's 64 entries
    return n < N && m < ld ? __builtin_bit_cast(uint64_t, part[n * (ld / kGroup) + m / kGroup]) : 0;
  }
  __device__ __forceinline__ Fetched fetch(int64_t n, int64_t m) const {
    const int64_t from = m / kGroup * kGroup;
    const uint64_t at = id == nullptr ? listed_at(n, from) : n < N ? bit_of(id[n], from) : 0;
    return {n < N ? c[n] : 0.f, (uint32_t)(at >> (m - from)) & 255u};
  }
  __device__ __forceinline__ float values(float (&x)[8], const f32x4* v, int64_t m, float ref, uint32_t at_ids) const {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = exponent(v[k / 4][k % 4], ref);
    if (m + 8 > V) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = m + k < V ? x[k] : 0.f;
    }
    if (at_ids != 0) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = at_ids >> k & 1 ? 0.f : x[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += x[k];
    return sum_of_8_lanes(sum);
  }
  __device__ __forceinline__ void piece(int64_t n, int64_t m, const f32x4* v, const Fetched& row) const {
    float x[8], ref = row.c;
    float sum = values(x, v, m, ref, row.at_ids);
    if (sum > kFar) {   // the same in the 8 lanes
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < 8; ++k) top = fmaxf(top, m + k < V ? v[k / 4][k % 4] : -INFINITY);
      ref = rintf(max_of_8_lanes(top) * exponent.t);
      sum = values(x, v, m, ref, row.at_ids);
    }
    if (n >= N || m >= ld) return;
    put_bf16(e + n * ld + m, x);
    if (m % kGroup == 0) part[n * (ld / kGroup) + m / kGroup] = f32x2{ref, sum};
  }
  // A wave's accumulators, a group of 64 entries of 16 rows at a time (four row blocks of a column
  // block: a lane holds 16 values of one row), without the LDS.
  template <int BM, int BN>
  __device__ __forceinline__ void tile(f32x4 (&acc)[BM][BN], int tm, int tn, int wm, int wn, int lane) const {
    const int64_t n0 = (int64_t)(tn * 2 + wn) * BN * 16 + (lane & 15);
    const int m0 = (tm * 2 + wm) * BM * 16, g4 = (lane >> 4) * 4;
    float ref[BN];
    int32_t only[BN];
    uint64_t lists[BN][BM / 4] = {};
    repeat<BN>([&](auto jc) {
      constexpr int j = decltype(jc)::value;
      const int64_t n = n0 + j * 16;
      ref[j] = n < N ? c[n] : 0.f;
      only[j] = id != nullptr && n < N ? id[n] : -1;
    });
    if (id == nullptr) {
      repeat<BN>([&](auto jc) {
        repeat<BM / 4>([&](auto gc) {
          constexpr int j = decltype(jc)::value, g = decltype(gc)::value;
          lists[j][g] = listed_at(n0 + j * 16, m0 + g * kGroup);
        });
      });
    }
    repeat<BN>([&](auto jc) {
      constexpr int j = decltype(jc)::value;
      const int64_t n = n0 + j * 16;
      repeat<BM / 4>([&](auto gc) {
        constexpr int i0 = decltype(gc)::value * 4;
        const int m = m0 + i0 * 16;
        float x[16];
        auto total = [&] {   // over the group
          float sum[4] = {};
#pragma unroll
          for (int q = 0; q < 16; ++q) sum[q % 4] += x[q];
          return across_rows((sum[0] + sum[1]) + (sum[2] + sum[3]));
        };
        auto values = [&](float from) {
#pragma unroll
          for (int q = 0; q < 16; ++q) x[q] = exponent(acc_read(acc[i0 + q / 4][j][q % 4]), from);
          if (m + kGroup > V) {   // the same in all lanes
#pragma unroll
            for (int q = 0; q < 16; ++q) x[q] = m + q / 4 * 16 + g4 + q % 4 < V ? x[q] : 0.f;
          }
          return total();
        };
        float from = ref[j], sum = values(from);
        const bool some = id == nullptr ? lists[j][i0 / 4] != 0 : (uint32_t)(only[j] - m) < (uint32_t)kGroup;
        if (__any(some || sum > kFar)) {
          const uint64_t at_ids = id == nullptr ? lists[j][i0 / 4] : bit_of(only[j], m);
          const uint32_t low = (uint32_t)at_ids >> g4, high = (uint32_t)(at_ids >> 32) >> g4;
          auto drop = [&] {   // the entries at ids
#pragma unroll
            for (int q = 0; q < 16; ++q) x[q] = (q < 8 ? low : high) >> (q / 4 % 2 * 16 + q % 4) & 1 ? 0.f : x[q];
            return total();
          };
          sum = drop();
          if (__any(sum > kFar)) {
            float top = -INFINITY;
#pragma unroll
            for (int q = 0; q < 16; ++q)
              top = fmaxf(top, m + q / 4 * 16 + g4 + q % 4 < V ? acc_read(acc[i0 + q / 4][j][q % 4]) : -INFINITY);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (sum > kFar) from = rintf(top * exponent.t);
            values(from);
            sum = drop();
          }
        }
        const bool on = n < N && m < ld;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float* v = x + h * 8;
          const u32x4 o = eight_rows(u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])},
                                     u32x2{pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])});
          if (on) *reinterpret_cast<u32x4*>(e + n * ld + m + h * 32 + eight_rows_at(lane)) = o;
        }
        if (on && lane < 16) part[n * (ld / kGroup) + m / kGroup] = f32x2{from, sum};
      });
    });
  }
};

// Few rows: the logits as they are.
struct SkinnyLogits {
  float* z;   // [N][ld]
  int64_t ld;
  __device__ __forceinline__ void operator()(int m, int n, const float (&s)[1]) const { z[n * ld + m] = s[0]; }
};

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
template <class T>
__device__ __forceinline__ T wave_sum(T x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
// The threads that take a row: a work-group of 256, or, from kTeamRows rows on, a wave (a work-group of
// four): 2,438 rows, d = 816, V = 1915 79 -> 72 us a call, 764 rows, 1656, 3661 78 -> 82 by waves.  Results
// of max and sum are the same in all threads, in a fixed order.
constexpr int64_t kTeamRows = 2048;
template <int kThreads>
struct Team {
  float maxima[4];
  double sums[4];
  static __device__ __forceinline__ int row() { return blockIdx.x * (256 / kThreads) + threadIdx.x / kThreads; }
  static __device__ __forceinline__ int thread() { return threadIdx.x % kThreads; }
  __device__ __forceinline__ void sync() const {
    if constexpr (kThreads == 256) __syncthreads();
    else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  __device__ __forceinline__ bool any(bool x) const {
    if constexpr (kThreads == 256) return __syncthreads_or(x);
    else return __any(x);
  }
  __device__ __forceinline__ float max(float x) {
    x = wave_max(x);
    if constexpr (kThreads == 64) return x;
    __syncthreads();
    if (threadIdx.x % 64 == 0) maxima[threadIdx.x / 64] = x;
    __syncthreads();
    return fmaxf(fmaxf(maxima[0], maxima[1]), fmaxf(maxima[2], maxima[3]));
  }
  __device__ __forceinline__ double sum(double x) {
    x = wave_sum(x);
    if constexpr (kThreads == 64) return x;
    __syncthreads();
    if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = x;
    __syncthreads();
    return (sums[0] + sums[1]) + (sums[2] + sums[3]);
  }
};
// Over the 256 threads of a work-group.
__device__ __forceinline__ double block_total(double x, double* sh) {
  x = wave_sum(x);
  __syncthreads();
  if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = x;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// (Reference, sum) of the groups of 2,048 logits of a row, without those at its ids.  Grid (N, groups).
__global__ __launch_bounds__(256) void few_groups_kernel(const float* __restrict__ z, int64_t ld, int V,
                                                         const int32_t* __restrict__ ids, int ids_of_row,
                                                         Exponent exponent, f32x2* __restrict__ part) {
  __shared__ Team<256> team;
  const int v0 = blockIdx.y * kFewGroup + threadIdx.x * 8;
  const float* row = z + (int64_t)blockIdx.x * ld;
  uint32_t in = v0 + 8 <= V ? 255u : v0 < V ? (1u << (V - v0)) - 1u : 0u;
  for (int j = 0; j < ids_of_row; ++j) {
    const uint32_t off = (uint32_t)(ids[(int64_t)blockIdx.x * ids_of_row + j] - v0);
    in &= off < 8u ? ~(1u << off) : 255u;
  }
  float x[8], top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    x[k] = in >> k & 1 ? row[v0 + k] : -INFINITY;
    top = fmaxf(top, x[k]);
  }
  const float ref = rintf(team.max(top) * exponent.t);
#pragma unroll
  for (int k = 0; k < 8; ++k) sum += in >> k & 1 ? exponent(x[k], ref) : 0.f;
  sum = (float)team.sum(sum);
  if (threadIdx.x == 0) part[(int64_t)blockIdx.x * gridDim.y + blockIdx.y] = f32x2{ref, sum};
}

constexpr int kRescaled = 2;   // of Rows::use

// ---- what a call's kernels share ------------------------------------------------------
// An id of a row (lane j has the j-th): its log-prob and probability, and the sum of all others' (1 - p,
// without its cancellation).
struct Listed {
  int id;          // -1: none
  bool first;      // the list has it at no place before
  double lp, p, left;
};
struct Rows {
  int N, d, V, k;          // k ids a row
  int way, grads;          // kTiles, kFew or kOnePass; gradients wanted
  int64_t ld, groups;      // entries between softmax rows; groups of a row
  int group;               // entries of a group
  double inv_t;
  int32_t* use;            // 1: takes part (kRescaled: with E brought to another reference than it was
                           // written in), 0: left out, -1: left out for an invalid id
  double* zs;              // [N][k] logits at the ids
  float* c;                // reference of the row
  f32x2* part;
  float* f;                // factor of E
  int32_t* ids;            // [N][k] places of the entries set apart (-1: none) and their values
  float* g;
  double* terms;           // [4][N] of the loss
  uint16_t *copy, *e;      // [N][d], [N][ld]
  int32_t* err;
};

__device__ __forceinline__ void raise(int32_t* err, int bit) {
  if (err != nullptr) atomicOr(err, bit);
}

// ---- 1. gather -------------------------------------------------------------------------
// A team per row; kLanes lanes take an id each in turn, whose row of W is read beside the hidden
// row.  Op::use(i, lane, r): as Rows::use, the same in all lanes; Op::id(i, j, r): the row's
// j-th id or -1.  Lists go 16 lanes to an id (2,501 rows of 50 ids, d = 520 25 us; 32 lanes 28, a wave
// for four ids together 50; 29 since the bits of the ids' places are written), one to four ids a wave each.
template <int kThreads, int kLanes, class Op>
__global__ __launch_bounds__(256) void gather_kernel(Rows r, Op op, const uint16_t* __restrict__ hidden,
                                                     const uint16_t* __restrict__ w) {
  __shared__ Team<kThreads> team;
  const int i = team.row(), t = team.thread();
  if (i >= r.N) return;
  const int use = op.use(i, t % 64, r);
  if (t == 0) r.use[i] = use;
  if (t < r.k) {   // (finalize writes what becomes of them)
    const int64_t at = (int64_t)i * r.k + t;
    r.ids[at] = use == 1 ? op.id(i, t, r) : -1;
  }
  if (r.way == kTiles && r.k > 1) {   // the bits of each group's entries at ids, where its sum will stand
    const int lane = t % 64, my = use == 1 && lane < r.k ? op.id(i, lane, r) : -1;
    f32x2* bits = r.part + (int64_t)i * r.groups;
    for (int g0 = t - lane; g0 < r.groups; g0 += kThreads) {
      uint64_t mine = 0;
      for (uint64_t here = __ballot(my >= 0 && my / (64 * kGroup) == g0 / 64); here != 0; here &= here - 1) {
        const int id = __builtin_amdgcn_readlane(my, __builtin_ctzll(here));
        if (id / kGroup == g0 + lane) mine |= uint64_t(1) << id % kGroup;
      }
      if (g0 + lane < r.groups) bits[g0 + lane] = __builtin_bit_cast(f32x2, mine);
    }
  }
  const u32x4* from = reinterpret_cast<const u32x4*>(hidden + (int64_t)i * r.d);
  u32x4* to = reinterpret_cast<u32x4*>(r.copy + (int64_t)i * r.d);
  const int pieces = r.d / 8;
  for (int p = t; p < pieces; p += kThreads) {
    u32x4 x = {0, 0, 0, 0};
    if (use == 1) x = from[p];
    to[p] = x;
  }
  if (use != 1) {
    if (t == 0) r.c[i] = 0.f;
    return;
  }
  float top = -INFINITY;
  for (int j = t / kLanes; j < r.k; j += kThreads / kLanes) {
    const int id = op.id(i, j, r);
    double sum = 0.0;
    if (id >= 0) {   // the same in the kLanes
      const u32x4* row = reinterpret_cast<const u32x4*>(w + (int64_t)id * r.d);
#pragma unroll 8
      for (int p = t % kLanes; p < pieces; p += kLanes) {
        const u32x4 hv = from[p], wv = row[p];
        float eight = 0.f;   // of exact products, their sums go on in float64: log-probs are summed over sequences
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          eight = fmaf(__uint_as_float(hv[q] << 16), __uint_as_float(wv[q] << 16), eight);
          eight = fmaf(__uint_as_float(hv[q] & 0xFFFF0000u), __uint_as_float(wv[q] & 0xFFFF0000u), eight);
        }
        sum += eight;
      }
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
      top = fmaxf(top, (float)sum);
    }
    if (t % kLanes == 0) r.zs[(int64_t)i * r.k + j] = sum;
  }
  top = team.max(top);
  if (t == 0) r.c[i] = rintf(top * (float)(r.inv_t * 1.4426950408889634));
}

// The row's hidden entries times its factor, the second operand of dW in tiles.
template <int kThreads>
__device__ __forceinline__ void scale_copy(const Rows& r, int i, float f) {
  if (r.way == kOnePass) return;   // (its head kernels take the rows as they are)
  u32x4* row = reinterpret_cast<u32x4*>(r.copy + (int64_t)i * r.d);
#pragma unroll 4
  for (int p = Team<kThreads>::thread(); p < r.d / 8; p += kThreads) {
    u32x4 x = row[p];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      x[q] = f == 0.f ? 0u : pack_bf16(f * __uint_as_float(x[q] << 16), f * __uint_as_float(x[q] & 0xFFFF0000u));
    row[p] = x;
  }
}

// ---- 3. finalize -----------------------------------------------------------------------
__device__ __forceinline__ double lane_value(double x, int lane) {   // lane: the same in all lanes
  const uint64_t v = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, lane), hi = __builtin_amdgcn_readlane((uint32_t)(v >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// What a lane's value x leaves of the whole, `others` and the wave's sum of `once` (x, or 0 where another lane has
// the same key): the whole less x, but where x is more than half of it (one key at most) the sum of all the rest.
__device__ __forceinline__ double without(double x, double once, double others, int key, double& whole) {
  whole = others + wave_sum(once);
  double rest = whole - x;
  const uint64_t most = __ballot(once > 0.5 * whole);
  if (most != 0) {
    const int at = __builtin_amdgcn_readlane(key, __builtin_ctzll(most));
    const double all = others + wave_sum(key == at ? 0.0 : once);
    if (key == at) rest = all;
  }
  return rest;
}
// Of a wave's lanes with the row's ids: own is an entry's 2^(z t - c), z its logit, others the sum over all
// entries that stand at no id.  An id that a list has twice counts once.  lse2: log2 of the whole sum, and c.
__device__ __forceinline__ Listed listed(int id, double own, double z, double others, float c, int lane, int k, double& lse2) {
  Listed x{id, id >= 0, 0.0, 0.0, 0.0};
  for (int j = 0; j < k; ++j) x.first = x.first && !(j < lane && __builtin_amdgcn_readlane(id, j) == id);
  double total;
  const double rest = without(own, x.first ? own : 0.0, others, id, total);
  lse2 = (double)c + log2(total);
  x.lp = own > rest ? -log1p(rest / own) : z - lse2 * 0.6931471805599453;
  x.p = own / total;
  x.left = rest / total;
  return x;
}

// A team per row: log2 of the sum over its groups and the entries at its ids, in a fixed order (a row whose
// groups have several references brought to the largest one); then op.row, called by the first wave, gives the
// terms, the row's factor a of p and, in r.ids and r.g, the entries G / a at the ids.  E's own scale
// is 2^(lse2 - c): the entries go in with it and the factor takes its inverse.  A row's gradient is
// mostly that of its largest entry at an id, so this one is made exact: all entries there take the
// factor that carries it to a value of bf16, and the row's factor its inverse.  (What this moves, the
// softmax entries, by 2^-8 at most, is what their own rounding moves them by; d_w_head of 777 rows was
// 0.0029 off float64 in the relative 2-norm without it, 0.0023 with it, 0.0017 of which is its own
// rounding to bf16.)  Below the normal numbers bf16 is too coarse for that, and no entry matters.
template <int kThreads, class Op>
__global__ __launch_bounds__(256) void finalize_kernel(Rows r, Op op) {
  __shared__ Team<kThreads> team;
  __shared__ float factors[256 / kThreads];
  const int i = team.row(), t = team.thread();
  if (i >= r.N) return;
  float& factor = factors[threadIdx.x / kThreads];
  const int use = r.use[i];
  uint16_t* row = r.e + (int64_t)i * r.ld;
  double others = 0.0;   // the sum without the entries at the row's ids, in units of 2^c
  float c = 0.f;
  if (use == 1) {
    const f32x2* part = r.part + (int64_t)i * r.groups;
    c = r.c[i];
    float top = -INFINITY;
    double sum = 0.0;
    bool far = false;
#pragma unroll 8
    for (int g = t; g < r.groups; g += kThreads) {
      const f32x2 p = part[g];
      sum += p.y;
      top = fmaxf(top, p.x);
      far = far || p.x != c;
    }
    if (team.any(far)) {
      top = fmaxf(team.max(top), c);
      sum = 0.0;
      for (int g = t; g < r.groups; g += kThreads) {
        const f32x2 p = part[g];
        if (p.x != -INFINITY || p.y != 0.f) sum += (double)p.y * (double)__builtin_amdgcn_exp2f(p.x - top);
      }
      if (r.way != kFew && r.grads)
        for (int64_t v0 = t * 8; v0 < r.groups * r.group; v0 += kThreads * 8) {
          const float down = __builtin_amdgcn_exp2f(part[v0 / r.group].x - top);
          u32x4 x = *reinterpret_cast<const u32x4*>(row + v0);
#pragma unroll
          for (int q = 0; q < 4; ++q)
            x[q] = pack_bf16(down * __uint_as_float(x[q] << 16), down * __uint_as_float(x[q] & 0xFFFF0000u));
          *reinterpret_cast<u32x4*>(row + v0) = x;
        }
      c = top;
      if (t == 0) r.use[i] = kRescaled;
    }
    others = team.sum(sum);
  }
  if (t < 64) {
    const int64_t at = (int64_t)i * r.k + t;   // this lane's, here and in op.row
    double lse2 = 0.0;
    Listed mine{-1, false, 0.0, 0.0, 0.0};
    if (use == 1) {
      const bool there = t < r.k && r.ids[at] >= 0;
      const double z = there ? r.zs[at] * r.inv_t : 0.0;
      double own = there ? exp2(z * 1.4426950408889634 - (double)c) : 0.0;
      own = own < FLT_MIN ? 0.0 : own;   // as the other entries, which are float32
      mine = listed(there ? r.ids[at] : -1, own, z, others, c, t, r.k, lse2);
    }
    if (r.way == kFew) c = (float)lse2;   // E is written from the logits, relative to the sum
    const float a = op.row(i, t, use, lse2 * 0.6931471805599453, mine, r);
    const bool entry = use == 1 && t < r.k && r.ids[at] >= 0;
    const float e = entry ? (float)((double)r.g[at] * exp2(lse2 - (double)c)) : 0.f;
    const float most = wave_max(fabsf(e));
    const float there = __uint_as_float((uint32_t)pack_bf16(most, 0.f) << 16);
    const float carry = most >= FLT_MIN && std::isfinite(there) ? there / most : 1.f;
    if (entry) r.g[at] = e * carry;
    if (t == 0) {
      r.c[i] = c;
      // (an objective that knows a later on multiplies by it)
      factor = use == 1 && a != 0.f ? a * (float)exp2((double)c - lse2) / carry : 0.f;
      r.f[i] = factor;
    }
  }
  if (!r.grads) return;
  team.sync();   // also: the rescaled row, r.ids and r.g are written
  if (r.way != kFew && use == 1 && t < r.k) {
    const int64_t at = (int64_t)i * r.k + t;
    const int id = r.ids[at];
    if (id >= 0) row[id] = (uint16_t)pack_bf16(r.g[at], 0.f);
  }
  if (Op::kFactor) scale_copy<kThreads>(r, i, factor);
}

// The loss from the rows' terms, in a fixed order: terms [kinds][n], loss = times[0] sum 0 + times[1]
// sum 1, stats the sums.  One work-group, of any size; it goes along with the launch of the gradients.
struct LossSum {
  const double* terms;
  int64_t n;
  int kinds;             // 1 or 4
  float times[2];
  double *loss, *stats;  // loss NULL: nothing to do

  template <int kKinds>
  __device__ __forceinline__ void sum(double (&out)[4], double* sh) const {
    double x[kKinds] = {};
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < n; i += blockDim.x)
#pragma unroll
      for (int q = 0; q < kKinds; ++q) x[q] += terms[q * n + i];
#pragma unroll
    for (int q = 0; q < kKinds; ++q) {
      x[q] = wave_sum(x[q]);
      if (threadIdx.x % 64 == 0) sh[q * 16 + threadIdx.x / 64] = x[q];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kKinds; ++q) {
      out[q] = 0.0;
      for (unsigned w = 0; w < blockDim.x / 64; ++w) out[q] += sh[q * 16 + w];
    }
  }
  __device__ __forceinline__ void run(double* sh) const {   // 64 doubles of LDS
    if (loss == nullptr) return;
    double s[4] = {};
    if (kinds == 4) sum<4>(s, sh);
    else sum<1>(s, sh);
    if (threadIdx.x != 0) return;
    *loss = times[1] != 0.f ? (double)times[0] * s[0] + (double)times[1] * s[1] : (double)times[0] * s[0];
    if (stats != nullptr)
      for (int q = 0; q < 4; ++q) stats[q] = s[q];
  }
};
__global__ __launch_bounds__(1024) void loss_sum_kernel(LossSum s) {
  __shared__ double sh[64];
  s.run(sh);
}

// ---- policy loss ---------------------------------------------------------------------------
// One id a row, its use checked by the objectives of a target.
__device__ __forceinline__ int target_use(int i, const int32_t* target, const float* weight, const Rows& r, int lane) {
  if (weight != nullptr && weight[i] == 0.f) return 0;
  const int o = target[i];
  if (o >= 0 && o < r.V) return 1;
  if (lane == 0) raise(r.err, PSPO_DEVERR_TARGET);
  return -1;
}

struct Policy {
  static constexpr bool kFactor = true;   // row() knows the row's factor
  const int32_t* target;
  const float *logp_old, *logp_ref, *weight;
  const int32_t* seq_id;
  const float* advantage;
  int R;
  float eps_low, eps_high, kl_coef, scale;
  int kl;
  float* logp_new;

  __device__ __forceinline__ int use(int i, int lane, const Rows& r) const {
    const int u = target_use(i, target, weight, r, lane);
    if (u != 1) return u;
    const int s = seq_id[i];
    if (s >= 0 && s < R) return 1;
    if (lane == 0) raise(r.err, PSPO_DEVERR_SEQ_ID);
    return -1;
  }
  __device__ __forceinline__ int id(int i, int, const Rows&) const { return target[i]; }
  __device__ __forceinline__ float row(int i, int lane, int use, double lse, const Listed& mine, const Rows& r) const {
    if (lane != 0) return 0.f;
    double gain = 0.0, div = 0.0, clipped = 0.0, delta = 0.0, l = 0.0;
    if (use == 1) {
      l = mine.lp;
      const double c = (double)weight[i] * (double)scale, A = advantage[seq_id[i]];
      const double rho = exp(l - (double)logp_old[i]);
      const double lo = 1.0 - (double)eps_low, hi = 1.0 + (double)eps_high;
      const double in = rho < lo ? lo : (rho > hi ? hi : rho);   // (a NaN stays)
      gain = c * (rho * A < in * A ? rho * A : in * A);
      const bool pass = (A > 0.0 && rho <= hi) || (A < 0.0 && rho >= lo);
      clipped = A != 0.0 && !pass ? 1.0 : 0.0;
      delta = pass ? -c * rho * A : 0.0;
      if (logp_ref != nullptr) {
        const double u = l - (double)logp_ref[i];
        div = c * (kl == PSPO_KL_K1 ? u : kl == PSPO_KL_K2 ? 0.5 * u * u : expm1(-u) + u);
        if (kl_coef != 0.f) delta += (double)kl_coef * c * (kl == PSPO_KL_K1 ? 1.0 : kl == PSPO_KL_K2 ? u : -expm1(-u));
      }
      const double loss = kl_coef != 0.f ? (double)kl_coef * div - gain : -gain;
      if (!(std::isfinite(lse) && std::isfinite((float)rho) && std::isfinite(loss) &&
            std::isfinite((float)(delta * r.inv_t))))
        raise(r.err, PSPO_DEVERR_NONFINITE);
    }
    const int64_t n = r.N;
    r.terms[i] = gain;
    r.terms[n + i] = div;
    r.terms[2 * n + i] = clipped;
    r.terms[3 * n + i] = use == 1 ? 1.0 : 0.0;
    r.ids[i] = use == 1 ? target[i] : -1;
    r.g[i] = use == 1 ? (float)-mine.left : 0.f;
    if (logp_new != nullptr) logp_new[i] = use < 0 ? NAN : (float)l;
    return (float)(-delta * r.inv_t);
  }
};

// ---- preference loss ------------------------------------------------------------------------
struct Preference {
  static constexpr bool kFactor = false;   // pref_rows_kernel does
  const int32_t* target;
  const float *logp_ref, *weight;
  float* logp_new;

  __device__ __forceinline__ int use(int i, int lane, const Rows& r) const {
    return target_use(i, target, weight, r, lane);
  }
  __device__ __forceinline__ int id(int i, int, const Rows&) const { return target[i]; }
  // terms: the log-prob, the row's part of its sequence's log ratio, its weight
  __device__ __forceinline__ float row(int i, int lane, int use, double lse, const Listed& mine, const Rows& r) const {
    if (lane != 0) return 0.f;
    double l = 0.0, part = 0.0, c = 0.0;
    if (use == 1) {
      l = mine.lp;
      c = weight != nullptr ? (double)weight[i] : 1.0;
      part = c * (logp_ref != nullptr ? l - (double)logp_ref[i] : l);   // its sequence looks whether it is finite
    }
    const int64_t n = r.N;
    r.terms[i] = l;
    r.terms[n + i] = part;
    r.terms[2 * n + i] = c;
    r.ids[i] = use == 1 ? target[i] : -1;
    r.g[i] = use == 1 ? (float)-mine.left : 0.f;
    if (logp_new != nullptr) logp_new[i] = use < 0 ? NAN : (float)l;
    return 1.f;   // pref_rows_kernel multiplies by what it is
  }
};

struct Pairs {
  const int32_t *cu, *chosen, *rejected;
  int R, P, kind, average;
  float beta, smoothing, scale;
  double *ratio, *norm, *coef;   // [R]
  double *pair, *pair_loss;      // [P]
  float *seq_ratio, *margin;
  int32_t* err;
};

// Sequence r's rows, clamped to [0, N].
__device__ __forceinline__ bool sequence_rows(const Pairs& q, int r, int N, int& lo, int& hi) {
  const int a = q.cu[r], b = q.cu[r + 1];
  lo = min(max(a, 0), N);
  hi = min(max(b, lo), N);
  return a >= 0 && b >= a && b <= N;
}

// Its log ratio and the factor that its rows' terms enter it with, from their sum and their weights'.
__device__ __forceinline__ void sequence_ratio(const Pairs& q, int r, double part, double c, bool write) {
  if (!write) return;
  const double norm = q.average ? (c != 0.0 ? 1.0 / c : 0.0) : 1.0;
  const double ratio = norm != 0.0 ? part * norm : 0.0;
  q.norm[r] = norm;
  q.ratio[r] = ratio;
  if (q.seq_ratio != nullptr) q.seq_ratio[r] = (float)ratio;
}

// A work-group per sequence.
__global__ __launch_bounds__(256) void pref_sequences_kernel(Pairs q, int N, const double* __restrict__ terms) {
  __shared__ double sh[4];
  const int r = blockIdx.x;
  int lo, hi;
  const bool fine = sequence_rows(q, r, N, lo, hi);
  if (!fine && threadIdx.x == 0) raise(q.err, PSPO_DEVERR_SEQ_ID);
  double part = 0.0, c = 0.0;
  for (int i = lo + threadIdx.x; i < hi; i += 256) {
    part += terms[(int64_t)N + i];
    c += terms[2 * (int64_t)N + i];
    if (!std::isfinite(terms[(int64_t)N + i])) raise(q.err, PSPO_DEVERR_NONFINITE);
  }
  part = block_total(part, sh);
  c = block_total(c, sh);
  sequence_ratio(q, r, part, c, threadIdx.x == 0);
}

// d loss / d u of a pair, and its part of the loss.
__device__ __forceinline__ void pair_terms(const Pairs& q, int p) {
  const int a = q.chosen[p], b = q.rejected[p];
  double loss = 0.0, du = 0.0, m = NAN;
  if (a >= 0 && a < q.R && b >= 0 && b < q.R) {
    const double u = q.ratio[a] - q.ratio[b], beta = q.beta, eps = q.smoothing;
    m = beta * u;
    if (q.kind == PSPO_PREF_SIGMOID) {
      // -log s(x) = max(-x, 0) + log1p(exp(-|x|)), s(-x) = exp(-x) s(x)
      const double e = exp(-fabs(m)), tail = log1p(e);
      const double up = m > 0.0 ? tail : tail - m, down = m > 0.0 ? tail + m : tail;   // -log s(m), -log s(-m)
      const double s = m > 0.0 ? 1.0 / (1.0 + e) : e / (1.0 + e), s_neg = m > 0.0 ? e / (1.0 + e) : 1.0 / (1.0 + e);
      loss = eps != 0.0 ? (1.0 - eps) * up + eps * down : up;
      du = beta * (eps * s - (1.0 - eps) * s_neg);
    } else {
      const double x = u - 0.5 / beta;
      loss = x * x;
      du = 2.0 * x;
    }
    if (!std::isfinite(loss)) raise(q.err, PSPO_DEVERR_NONFINITE);
  } else {
    raise(q.err, PSPO_DEVERR_SEQ_ID);
  }
  q.pair[p] = du * (double)q.scale;
  q.pair_loss[p] = loss * (double)q.scale;
  if (q.margin != nullptr) q.margin[p] = (float)m;
}
__global__ __launch_bounds__(256) void pref_pairs_kernel(Pairs q) {
  const int p = blockIdx.x * 256 + threadIdx.x;
  if (p < q.P) pair_terms(q, p);
}

// What pair p gives sequence r.
__device__ __forceinline__ double pair_part(const Pairs& q, int r, int p) {
  const int a = q.chosen[p], b = q.rejected[p];
  if (a == b || (a != r && b != r) || a < 0 || a >= q.R || b < 0 || b >= q.R) return 0.0;
  return a == r ? q.pair[p] : -q.pair[p];
}

// A work-group per sequence: what its pairs give it, in the pairs' order within each thread's share.
// The last one sums the loss.
__global__ __launch_bounds__(256) void pref_coef_kernel(Pairs q, double* __restrict__ loss) {
  __shared__ double sh[4], sum[64];
  const int r = blockIdx.x;
  if (r == q.R) {
    LossSum{q.pair_loss, q.P, 1, {1.f, 0.f}, loss, nullptr}.run(sum);
    return;
  }
  double c = 0.0;
  for (int p = threadIdx.x; p < q.P; p += 256) c += pair_part(q, r, p);
  c = block_total(c, sh);
  if (threadIdx.x == 0) q.coef[r] = q.norm[r] != 0.0 ? c * q.norm[r] : 0.0;
}

// All three of the above for a few thousand rows and few pairs, in one work-group: a wave per
// sequence in turn (8 completions of 257 rows, 4 pairs: two launches less, 8 us a call).
constexpr int kPrefWaves = 16;
constexpr int64_t kPrefRows = 16384, kPrefLooks = 1 << 18;   // rows; sequences times pairs
__global__ __launch_bounds__(64 * kPrefWaves) void pref_all_kernel(Pairs q, int N, const double* __restrict__ terms,
                                                                   double* __restrict__ loss) {
  __shared__ double sh[kPrefWaves];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  for (int r = wave; r < q.R; r += kPrefWaves) {
    int lo, hi;
    if (!sequence_rows(q, r, N, lo, hi) && lane == 0) raise(q.err, PSPO_DEVERR_SEQ_ID);
    double part = 0.0, c = 0.0;
#pragma unroll 4
    for (int i = lo + lane; i < hi; i += 64) {
      part += terms[(int64_t)N + i];
      c += terms[2 * (int64_t)N + i];
      if (!std::isfinite(terms[(int64_t)N + i])) raise(q.err, PSPO_DEVERR_NONFINITE);
    }
    sequence_ratio(q, r, wave_sum(part), wave_sum(c), lane == 0);
  }
  __syncthreads();
  for (int p = threadIdx.x; p < q.P; p += 64 * kPrefWaves) pair_terms(q, p);
  __syncthreads();
  for (int r = wave; r < q.R; r += kPrefWaves) {
    double c = 0.0;
    for (int p = lane; p < q.P; p += 64) c += pair_part(q, r, p);
    c = wave_sum(c);
    if (lane == 0) q.coef[r] = q.norm[r] != 0.0 ? c * q.norm[r] : 0.0;
  }
  double x = 0.0;
  for (int p = threadIdx.x; p < q.P; p += 64 * kPrefWaves) x += q.pair_loss[p];
  x = wave_sum(x);
  if (lane == 0) sh[wave] = x;
  __syncthreads();
  if (threadIdx.x != 0) return;
  x = 0.0;
  for (int k = 0; k < kPrefWaves; ++k) x += sh[k];
  *loss = x;
}

// The row's factor, from its sequence's; a team per row.  A row that no sequence holds may hold anything: where
// its entries are not finite they become zeros, which a factor of 0 makes of the others in d_w_head.
template <int kThreads>
__global__ __launch_bounds__(256) void pref_rows_kernel(Rows r, Pairs q) {
  const int i = Team<kThreads>::row();
  if (i >= r.N) return;
  int s = 0, e = q.R;   // the last sequence that starts at or before row i
  while (s < e) {
    const int mid = s + (e - s) / 2;
    if (q.cu[mid + 1] > i) e = mid;
    else s = mid + 1;
  }
  const bool held = s < q.R && q.cu[s] <= i, on = held && r.use[i] > 0;
  if (!held && r.use[i] > 0 && r.way != kFew && !std::isfinite(r.terms[i]))   // (the entries of few rows are written later)
    for (int64_t v0 = Team<kThreads>::thread() * 8; v0 < r.ld; v0 += kThreads * 8)
      *reinterpret_cast<u32x4*>(r.e + (int64_t)i * r.ld + v0) = u32x4{0, 0, 0, 0};
  const double delta = on ? q.coef[s] * r.terms[2 * (int64_t)r.N + i] : 0.0;
  const float a = (float)(-delta * r.inv_t);
  const float f = on && a != 0.f ? a * r.f[i] : 0.f;
  if constexpr (kThreads == 256) __syncthreads();   // f is read before it is written
  if (Team<kThreads>::thread() == 0) {
    if (on && !std::isfinite(a)) raise(r.err, PSPO_DEVERR_NONFINITE);
    r.f[i] = f;
  }
  scale_copy<kThreads>(r, i, f);
}

// ---- distillation -----------------------------------------------------------------------------
struct Distill {
  static constexpr bool kFactor = true;
  const int32_t* topk_ids;
  const float* topk;
  const float* weight;
  float scale;
  float* kl;

  // An entry: an id that is not negative with a teacher value above -inf (or NaN, which shows).
  __device__ __forceinline__ bool entry(int64_t at) const {
    return topk_ids[at] >= 0 && !(topk[at] == -INFINITY);
  }
  __device__ __forceinline__ int use(int i, int lane, const Rows& r) const {
    if (weight != nullptr && weight[i] == 0.f) return 0;
    const int64_t at = (int64_t)i * r.k + lane;
    const bool on = lane < r.k && entry(at);
    if (__any(on && topk_ids[at] >= r.V)) {
      if (lane == 0) raise(r.err, PSPO_DEVERR_TARGET);
      return -1;
    }
    return __any(on) ? 1 : 0;
  }
  __device__ __forceinline__ int id(int i, int j, const Rows& r) const {
    const int64_t at = (int64_t)i * r.k + j;
    return entry(at) ? topk_ids[at] : -1;
  }
  // Lane j has the list's entry j.
  __device__ __forceinline__ float row(int i, int lane, int use, double lse, const Listed& mine, const Rows& r) const {
    const int64_t at = (int64_t)i * r.k + lane;
    const bool on = mine.id >= 0, first = mine.first;
    double div = 0.0, c = 0.0, g = 0.0;
    if (use == 1) {
      const double x = on ? (double)topk[at] * r.inv_t : -INFINITY;
      double top = x;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {   // (a NaN stays)
        const double y = __shfl_xor(top, o);
        top = y > top || y != y ? y : top;
      }
      const double e = on ? exp(x - top) : 0.0;
      const double q = e / wave_sum(e);
      double same = 0.0, all;   // the probability of this lane's id
      for (int j = 0; j < r.k; ++j) {
        const double qj = lane_value(q, j);
        same += __builtin_amdgcn_readlane(mine.id, j) == mine.id ? qj : 0.0;
      }
      const double away = without(same, first ? same : 0.0, 0.0, mine.id, all);   // of the others
      c = (weight != nullptr ? (double)weight[i] : 1.0) * (double)scale;
      const double each = first && !(same == 0.0) ? same * ((same > 0.5 ? log1p(-away) : log(same)) - mine.lp) : 0.0;
      div = wave_sum(each);
      g = mine.p > 0.5 ? away - mine.left : mine.p - same;   // (1 - q) - (1 - p) where p is near 1
      if (lane == 0 && !(std::isfinite(lse) && std::isfinite(c * div) && std::isfinite((float)(c * r.inv_t))))
        raise(r.err, PSPO_DEVERR_NONFINITE);
    }
    if (lane < r.k) {
      r.ids[at] = first ? mine.id : -1;
      r.g[at] = first ? (float)g : 0.f;
    }
    if (lane != 0) return 0.f;
    r.terms[i] = use == 1 ? c * div : 0.0;
    if (kl != nullptr) kl[i] = use < 0 ? NAN : (float)div;
    return (float)(c * r.inv_t);
  }
};

// ---- E of few rows ---------------------------------------------------------------------------
// From the float32 logits, relative to the row's sum, eight entries a thread; zeros where the factor
// is 0.  Grid (N, ceil(ld / 2048)).
__global__ __launch_bounds__(256) void few_entries_kernel(Rows r, const float* __restrict__ z, Exponent exponent) {
  const int i = blockIdx.x, v0 = (blockIdx.y * 256 + threadIdx.x) * 8;
  if (v0 >= r.ld) return;
  uint16_t* row = r.e + (int64_t)i * r.ld;
  float x[8] = {};
  const bool on = r.f[i] != 0.f;
  if (on) {
    const float c = r.c[i];
    const f32x4* from = reinterpret_cast<const f32x4*>(z + (int64_t)i * r.ld + v0);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (v0 + k < r.V) x[k] = exponent(from[k / 4][k % 4], c);
  }
  put_bf16(row + v0, x);
  if (!on) return;
  const int32_t* ids = r.ids + (int64_t)i * r.k;
  for (int j = 0; j < r.k; ++j) {
    const int id = ids[j];
    if ((uint32_t)(id - v0) < 8u) row[id] = (uint16_t)pack_bf16(r.g[(int64_t)i * r.k + j], 0.f);
  }
}

// ---- up to 64 rows: one pass over W ------------------------------------------------------------
// A work-group takes blocks of 16 vocabulary entries in turn; its 4 waves, one to a SIMD with all of
// its registers (8 waves of half of them spilled from d = 2,560 on), split the hidden width, 32 F columns
// each.  A wave's part of the block comes to registers (the next block's while this one is
// worked on), goes from there into the matrix instructions of the logits and into its own LDS; the
// waves' sums are exchanged, every wave forms the block's 16 x 16 softmax entries, and reads its part
// again, transposed, for their product with it, which stays in its accumulators: W is read once for
// the logits and d_hidden.  Entries at the rows' ids are left out (they are added at the end, to the sums as
// they are and to the product with what becomes of them).  The entries of a block that pass 2^32 take their own
// reference, as in the tiles; their row's accumulators are then of no use (no other row's are touched),
// and its d_hidden is formed from E (one_pass_hidden_kernel; W read again by few work-groups: one such row costs
// about 2 ms, 553 -> 2,580 us at 16 rows, d = 3584, V = 152064).  16 rows to a work-group, those of the others
// in grid y, which meet W's blocks in the same L2 at about the same time (gridDim.x % 8 == 0 then).
// Bound by W's bytes: 16 rows, d = 3584, V = 152064 292 us, 1 row, d = 1536, V = 151936 127, 3.7 TB/s
// each (torch's sum over as many bytes reads 4.0).
constexpr int kHeadWaves = 8, kHiddenWaves = 16;

// Four rows (4 g .. 4 g + 3) of column 16 b + lane % 16 of a wave's rows of bf16 in LDS, `pitch` bytes
// apart: the matrix instruction's operand with the rows as K.
__device__ __forceinline__ s16x4 transposed(const unsigned char* rows, int pitch, int b, int lane) {
  const int p = lane & 15;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_s16x4*)(rows + ((lane >> 4) * 4 + (p >> 2)) * pitch + b * 32 + (p & 3) * 8));
}

template <int F>
__global__ __attribute__((amdgpu_flat_work_group_size(64 * kPassWaves, 64 * kPassWaves),
                          amdgpu_waves_per_eu(pass_per_cu(F), pass_per_cu(F))))
void one_pass_kernel(Rows r, const uint16_t* __restrict__ w, Exponent exponent, float* __restrict__ slab) {
  constexpr int kPitch = 64 * F + 16;   // odd in 16 bytes: a column's 16 rows lie in different banks
  __shared__ __attribute__((aligned(16))) unsigned char rows[kPassWaves][kPassRows * kPitch];
  __shared__ f32x4 sums[2][kPassWaves][64];
  __shared__ int ids[kPassRows * kMostIds], count;   // those in this work-group's blocks: id + 2^21 (row of the 16)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int p = lane & 15, g = lane >> 4, col0 = wave * 32 * F + g * 8;
  const int i0 = blockIdx.y * kPassRows, n = min(r.N - i0, kPassRows), i = i0 + p;   // this work-group's rows, this lane's
  const int blocks = (r.V + kPassRows - 1) / kPassRows;
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  for (int t = threadIdx.x; t < n * r.k; t += 64 * kPassWaves) {
    const int id = r.ids[(int64_t)i0 * r.k + t];
    if (id >= 0 && id / kPassRows % (int)gridDim.x == (int)blockIdx.x) ids[atomicAdd(&count, 1)] = id | t / r.k << 21;
  }
  // 16 rows of a matrix that has `have` left, as buffer loads (one address register for all; what lies
  // past the rows reads as zeros, and so does what lies past the width, by an offset out of range)
  const uint32_t at = (uint32_t)(p * r.d + col0) * 2u;
  auto rows_of = [&](const uint16_t* first, int have) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(first), 0, min(max(have, 0), kPassRows) * r.d * 2,
                                             0x00020000);
  };
  auto piece = [&](auto from, int f, int left) {   // left: columns from col0 to the width
    return __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(
                                          from, f * 32 < left ? at : 0x80000000u, f * 64, 0));
  };
  auto block = [&](int b) { return rows_of(w + (int64_t)b * kPassRows * r.d, r.V - b * kPassRows); };
  bf16x8 h[F], x[F];
  {
    const auto from = rows_of(r.copy + (int64_t)i0 * r.d, n), first = block(blockIdx.x);
#pragma unroll
    for (int f = 0; f < F; ++f) h[f] = piece(from, f, r.d - col0);
#pragma unroll
    for (int f = 0; f < F; ++f) x[f] = piece(first, f, r.d - col0);
  }
  const float ref = p < n ? r.c[i] : 0.f;
  f32x4 acc[2 * F];
#pragma unroll
  for (int b = 0; b < 2 * F; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  int buf = 0;
  __syncthreads();
  const int own = count;
  for (int b = blockIdx.x; b < blocks; b += gridDim.x) {
    // each piece makes room for the next block's at once, so that a block's worth of loads stays in flight
    const auto next = block(b + (int)gridDim.x);
    int left = r.d - col0;
    asm volatile("" : "+v"(left));   // formed again at every block: kept, the F offsets take F registers
    f32x4 z = {0.f, 0.f, 0.f, 0.f};
    wave_lds_fence();
#pragma unroll
    for (int f = 0; f < F; ++f) {
      *reinterpret_cast<u32x4*>(rows[wave] + p * kPitch + f * 64 + g * 16) = __builtin_bit_cast(u32x4, x[f]);
      z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[f], h[f], z, 0, 0, 0);
      x[f] = piece(next, f, left);
      if (f % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    sums[buf][wave][lane] = z;
    stage_barrier<63>();   // (the loads stay in flight)
    z = sums[buf][0][lane];
#pragma unroll
    for (int k = 1; k < kPassWaves; ++k) z += sums[buf][k][lane];
    buf ^= 1;   // a wave writes it again behind the next barrier, which every reader has then passed
    // entries v0 .. v0 + 3 of row p
    const int v0 = b * kPassRows + g * 4;
    float y[4], from = ref, sum = 0.f;
    auto values = [&] {
      sum = 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) y[q] = v0 + q < r.V ? exponent(z[q], from) : 0.f;
      for (int j = 0; j < own; ++j) {
        const int at = ids[j] - (v0 | p << 21);
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] = at == q ? 0.f : y[q];
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) sum += y[q];
      sum = across_rows(sum);
    };
    values();
    if (__any(sum > kFar)) {
      float top = -INFINITY;
#pragma unroll
      for (int q = 0; q < 4; ++q) top = fmaxf(top, v0 + q < r.V ? z[q] : -INFINITY);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (sum > kFar) from = rintf(top * exponent.t);
      values();
    }
    const u32x2 e = {pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
    if (wave == (b / (int)gridDim.x) % kPassWaves && p < n) {
      *reinterpret_cast<u32x2*>(r.e + (int64_t)i * r.ld + v0) = e;
      if (g == 0) r.part[(int64_t)i * r.groups + b] = f32x2{from, sum};
    }
    const s16x4 ev = __builtin_bit_cast(s16x4, e);
#pragma unroll
    for (int k = 0; k < 2 * F; ++k) {
      acc[k] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(transposed(rows[wave], kPitch, k, lane), ev, acc[k], 0, 0, 0);
      if (k % 8 == 7) __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (p >= n) return;
  float* out = slab + ((int64_t)blockIdx.x * r.N + i) * r.d;
#pragma unroll
  for (int k = 0; k < 2 * F; ++k) {
    const int col = wave * 32 * F + k * 16 + g * 4;
    if (col < r.d) *reinterpret_cast<f32x4*>(out + col) = acc[k];
  }
}

// d_hidden of a row from the work-groups' sums and the rows of W at its ids, in a fixed order; of a row
// with entries past its reference from its E.  Grid (ceil(d / 256), N): 4 columns a thread, each wave a
// sixteenth of the terms.
__global__ __launch_bounds__(64 * kHiddenWaves) void one_pass_hidden_kernel(
    Rows r, const uint16_t* __restrict__ w, const float* __restrict__ slab, int groups, void* out, int f32) {
  __shared__ f32x4 sh[kHiddenWaves][64];
  const int i = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 256 + lane * 4;
  const float f = r.f[i];
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](float e, int64_t v) {
    const u32x2 x = *reinterpret_cast<const u32x2*>(w + v * r.d + col);
    sum += e * f32x4{__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u), __uint_as_float(x.y << 16),
                     __uint_as_float(x.y & 0xFFFF0000u)};
  };
  if (f != 0.f && col < r.d) {
    if (r.use[i] == kRescaled) {
#pragma unroll 4
      for (int v = wave; v < r.V; v += kHiddenWaves) add(__uint_as_float((uint32_t)r.e[(int64_t)i * r.ld + v] << 16), v);
    } else {
#pragma unroll 8
      for (int k = wave; k < groups; k += kHiddenWaves)
        sum += *reinterpret_cast<const f32x4*>(slab + ((int64_t)k * r.N + i) * r.d + col);
      for (int j = wave; j < r.k; j += kHiddenWaves) {
        const int64_t at = (int64_t)i * r.k + j;
        if (r.ids[at] >= 0) add(r.g[at], r.ids[at]);
      }
    }
  }
  sh[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || col >= r.d) return;
#pragma unroll
  for (int k = 1; k < kHiddenWaves; ++k) sum += sh[k][lane];
  sum *= f;
  if (f == 0.f) sum = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t at = (int64_t)i * r.d + col;
  if (f32) *reinterpret_cast<f32x4*>(static_cast<float*>(out) + at) = sum;
  else
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(out) + at) = u32x2{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
}

// dW = (f E)^T H of up to 16 rows: the rows as they are in LDS, a wave 16 vocabulary entries at a time, whose
// rows of dW it writes from end to end.  The roundings of so few rows average out in no sum, so f E goes in
// rounded to bf16 and what that leaves, two matrix instructions on one operand of rows (with f H rounded
// instead d_w_head of 16 rows, d = 3584, V = 152064, lists of 16 was 0.0024 off float64 in the relative 2-norm,
// so it is 0.0017).  Bound by dW's bytes: the same rows 214 us, 5.1 TB/s; 1 row, d = 1536, V = 151936 78,
// 6.0 TB/s.  The last work-group sums the loss.
template <int F>
__global__ __launch_bounds__(64 * kHeadWaves) void one_pass_head_kernel(Rows r, void* out, int f32, int add,
                                                                        LossSum loss) {
  constexpr int kPitch = 512 * F + 16;   // F parts of 256 columns
  __shared__ __attribute__((aligned(16))) unsigned char rows[kPassRows * kPitch];
  __shared__ double sh[64];
  if (blockIdx.x == gridDim.x - 1) {
    loss.run(sh);
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, p = lane & 15, g = lane >> 4;
  for (int t = threadIdx.x; t < kPassRows * 32 * F; t += 64 * kHeadWaves) {
    const int i = t / (32 * F), col = t % (32 * F) * 8;
    u32x4 x = {0, 0, 0, 0};
    if (i < r.N && col < r.d && r.f[i] != 0.f) x = *reinterpret_cast<const u32x4*>(r.copy + (int64_t)i * r.d + col);
    *reinterpret_cast<u32x4*>(rows + i * kPitch + col * 2) = x;
  }
  __syncthreads();
  const int blocks = (r.V + 15) / 16, step = ((int)gridDim.x - 1) * kHeadWaves;
  float f[4];   // of rows 4 g .. 4 g + 3
#pragma unroll
  for (int q = 0; q < 4; ++q) f[q] = g * 4 + q < r.N ? r.f[g * 4 + q] : 0.f;
  auto entries = [&](int b) {   // of vocabulary entry 16 b + p and these rows
    s16x4 y = {0, 0, 0, 0};
    const int v = b * 16 + p;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (f[q] != 0.f && v < r.V) y[q] = (short)r.e[(int64_t)(g * 4 + q) * r.ld + v];
    return y;
  };
  int b = blockIdx.x * kHeadWaves + wave;
  s16x4 next = b < blocks ? entries(b) : s16x4{0, 0, 0, 0};
  for (; b < blocks; b += step) {
    float y[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] = f[q] * __uint_as_float((uint32_t)(uint16_t)next[q] << 16);
    if (b + step < blocks) next = entries(b + step);
    const u32x2 high = {pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] -= __uint_as_float(q % 2 ? high[q / 2] & 0xFFFF0000u : high[q / 2] << 16);
    const s16x4 yh = __builtin_bit_cast(s16x4, high),
                yl = __builtin_bit_cast(s16x4, u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])});
    const int v = b * 16 + p;
    for (int k = 0; k * 32 < r.d; ++k) {
      const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
      const s16x4 h0 = transposed(rows, kPitch, 2 * k, lane), h1 = transposed(rows, kPitch, 2 * k + 1, lane);
      f32x4 c0 = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(h0, yl, zero, 0, 0, 0);
      f32x4 c1 = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(h1, yl, zero, 0, 0, 0);
      c0 = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(h0, yh, c0, 0, 0, 0);
      c1 = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(h1, yh, c1, 0, 0, 0);
      if (f32) {
        const int col = k * 32 + g * 4;
        float* to = static_cast<float*>(out) + (int64_t)v * r.d + col;
        if (v < r.V && col < r.d) *reinterpret_cast<f32x4*>(to) = add ? *reinterpret_cast<f32x4*>(to) + c0 : c0;
        if (v < r.V && col + 16 < r.d)
          *reinterpret_cast<f32x4*>(to + 16) = add ? *reinterpret_cast<f32x4*>(to + 16) + c1 : c1;
      } else {
        const u32x4 o = eight_rows(u32x2{pack_bf16(c0[0], c0[1]), pack_bf16(c0[2], c0[3])},
                                   u32x2{pack_bf16(c1[0], c1[1]), pack_bf16(c1[2], c1[3])});
        const int col = k * 32 + eight_rows_at(lane);
        if (v < r.V && col < r.d)
          *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + (int64_t)v * r.d + col) = o;
      }
    }
  }
}

// Both gradients: out[n][m] = f[n] C(m, n), or C alone (f NULL), bf16 or float32 (or added to it).
struct EpiGrad {
  static constexpr bool kPair = false, kTile = true;
  static constexpr bool kExtra = true;
  void* out;
  const float* f;
  int64_t ld;
  int M, N, f32, add;
  LossSum loss;
  __device__ __forceinline__ void extra(unsigned char* lds) const { loss.run(reinterpret_cast<double*>(lds)); }
  struct Fetched {
    float f;
  };
  __device__ __forceinline__ Fetched fetch(int64_t n, int64_t) const { return {f != nullptr && n < N ? f[n] : 1.f}; }
  __device__ __forceinline__ void piece(int64_t n, int64_t m, const f32x4* v, const Fetched& x) const {
    if (n >= N || m >= M) return;   // M % 8 == 0
    f32x4 s[2];
#pragma unroll
    for (int k = 0; k < 8; ++k) s[k / 4][k % 4] = x.f == 0.f ? 0.f : x.f * v[k / 4][k % 4];   // a row left out is zeros
    if (f32) {
      float* to = static_cast<float*>(out) + n * ld + m;
      if (add) {
        s[0] += reinterpret_cast<const f32x4*>(to)[0];
        s[1] += reinterpret_cast<const f32x4*>(to)[1];
      }
      put_f32(to, s);
    } else {
      put_bf16(static_cast<uint16_t*>(out) + n * ld + m, reinterpret_cast<const float*>(s));
    }
  }
  // The accumulators as they lie: a lane has four consecutive entries of a row, 16 bytes of float32,
  // or eight after a swap with the next row block, 16 bytes of bf16.
  template <int BM, int BN>
  __device__ __forceinline__ void tile(f32x4 (&acc)[BM][BN], int tm, int tn, int wm, int wn, int lane) const {
    const int64_t n0 = (int64_t)(tn * 2 + wn) * BN * 16 + (lane & 15);
    const int64_t m0 = (int64_t)(tm * 2 + wm) * BM * 16;
    repeat<BN>([&](auto jc) {
      constexpr int j = decltype(jc)::value;
      const int64_t n = n0 + j * 16;
      const float x = fetch(n, 0).f;
      auto value = [&](auto ic) {
        constexpr int i = decltype(ic)::value;
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = acc_read(acc[i][j][r]);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = x == 0.f ? 0.f : x * v[r];
        return v;
      };
      if (f32) {
        float* to = static_cast<float*>(out) + n * ld + m0 + (lane >> 4) * 4;
        f32x4 old[BM] = {};
        if (add) {
#pragma unroll
          for (int i = 0; i < BM; ++i)
            if (n < N && m0 + i * 16 + (lane >> 4) * 4 < M) old[i] = *reinterpret_cast<const f32x4*>(to + i * 16);
        }
        repeat<BM>([&](auto ic) {
          constexpr int i = decltype(ic)::value;
          const f32x4 v = value(ic);
          if (n < N && m0 + i * 16 + (lane >> 4) * 4 < M) *reinterpret_cast<f32x4*>(to + i * 16) = old[i] + v;
        });
      } else {
        uint16_t* to = static_cast<uint16_t*>(out) + n * ld + m0 + eight_rows_at(lane);
        repeat<BM / 2>([&](auto ic) {
          constexpr int i = decltype(ic)::value * 2;
          const f32x4 a = value(std::integral_constant<int, i>{}), b = value(std::integral_constant<int, i + 1>{});
          const u32x4 o = eight_rows(u32x2{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])},
                                     u32x2{pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3])});
          if (n < N && m0 + i * 16 + eight_rows_at(lane) < M) *reinterpret_cast<u32x4*>(to + i * 16) = o;
        });
      }
    });
  }
};

// dW = (f E)^T H of 17 to 64 rows, whose tiles would be all way in and out (one stage of K): a work-group
// keeps 256 columns of the rows in its registers, 64 to a wave as the matrix instructions take them, and goes
// over its share of the vocabulary, 64 entries a step; their f E comes through LDS, the next step's E on the way
// meanwhile.  f E in two parts as above (24 rows, d = 1536, V = 21936, lists of 16: 0.0025 off float64 with f H
// rounded, 0.0018 so; 24 rows, d = 3584, V = 152064 721 -> 728 us a call).  KS: steps of 32 rows.  The last row of
// the grid sums the loss.  Whole calls against tiles: 24 rows of the same 770 / 728, 160, 46996 52 / 48.  (From 65
// rows on both gradients' tiles in one launch are as good or better: 160 rows, d = 3584 1,106 / 1,183.)
constexpr int kStreamPerCu = 2;
template <int KS>
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(kStreamPerCu, kStreamPerCu)))
void stream_head_kernel(Rows r, EpiGrad out) {
  constexpr int kPitch = 64 * 2 + 16;   // odd in 16 bytes
  __shared__ __attribute__((aligned(16))) unsigned char tile[2][2 * KS * 32 * kPitch];   // f E, and what its rounding leaves
  __shared__ double sh[64];
  if (blockIdx.y == gridDim.y - 1) {
    if (blockIdx.x == 0) out.loss.run(sh);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p = lane & 15, g = lane >> 4;
  const int col0 = (blockIdx.y * 4 + wave) * 64;   // this wave's columns of H
  // eight rows (8 g .. 8 g + 7 of step ks) of column 16 b + p
  auto operand = [&](const unsigned char* rows, int ks, int b) {
    union {
      s16x4 half[2];
      bf16x8 v;
    } u;
#pragma unroll
    for (int q = 0; q < 2; ++q)
      u.half[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_s16x4*)(rows + (ks * 32 + g * 8 + q * 4 + (p >> 2)) * kPitch + b * 32 + (p & 3) * 8));
    return u.v;
  };
  // the rows' columns to registers, a wave's 64 at a time through the tile
  bf16x8 h[KS][4];
  for (int turn = 0; turn < 4; ++turn) {
    for (int t = threadIdx.x; t < KS * 32 * 8; t += 256) {
      const int i = t / 8, col = (blockIdx.y * 4 + turn) * 64 + t % 8 * 8;
      u32x4 x = {0, 0, 0, 0};
      if (i < r.N && col < r.d && r.f[i] != 0.f) x = *reinterpret_cast<const u32x4*>(r.copy + (int64_t)i * r.d + col);
      *reinterpret_cast<u32x4*>(tile[0] + i * kPitch + t % 8 * 16) = x;
    }
    __syncthreads();
    if (turn == wave) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int b = 0; b < 4; ++b) h[ks][b] = operand(tile[0], ks, b);
    }
    __syncthreads();
  }
  const int tiles = (r.V + 63) / 64, step = gridDim.x;
  u32x4 e[KS];   // this thread's pieces of the next tile
  float f[KS];   // and their rows' factors
#pragma unroll
  for (int q = 0; q < KS; ++q) f[q] = q * 32 + (int)threadIdx.x / 8 < r.N ? r.f[q * 32 + threadIdx.x / 8] : 0.f;
  auto load = [&](int at) {
#pragma unroll
    for (int q = 0; q < KS; ++q) {
      const int i = q * 32 + threadIdx.x / 8;
      e[q] = u32x4{0, 0, 0, 0};
      if (f[q] != 0.f) e[q] = *reinterpret_cast<const u32x4*>(r.e + (int64_t)i * r.ld + at * 64 + threadIdx.x % 8 * 8);
    }
  };
  int buf = 0;
  if ((int)blockIdx.x < tiles) load(blockIdx.x);
  for (int at = blockIdx.x; at < tiles; at += step) {
#pragma unroll
    for (int q = 0; q < KS; ++q) {
      u32x4 high, low;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x = f[q] * __uint_as_float(e[q][k] << 16), y = f[q] * __uint_as_float(e[q][k] & 0xFFFF0000u);
        high[k] = pack_bf16(x, y);
        low[k] = pack_bf16(x - __uint_as_float(high[k] << 16), y - __uint_as_float(high[k] & 0xFFFF0000u));
      }
      unsigned char* to = tile[buf] + (q * 32 + threadIdx.x / 8) * kPitch + threadIdx.x % 8 * 16;
      *reinterpret_cast<u32x4*>(to) = high;
      *reinterpret_cast<u32x4*>(to + KS * 32 * kPitch) = low;
    }
    if (at + step < tiles) load(at + step);
    stage_barrier<63>();   // (the loads stay in flight; a wave writes this half again behind the next barrier)
    f32x4 acc[4][4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int b = 0; b < 4; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const bf16x8 y = operand(tile[buf], ks, b), rest = operand(tile[buf], KS + ks, b);
#pragma unroll
        for (int a = 0; a < 4; ++a) acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h[ks][a], rest, acc[a][b], 0, 0, 0);
#pragma unroll
        for (int a = 0; a < 4; ++a) acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h[ks][a], y, acc[a][b], 0, 0, 0);
      }
    buf ^= 1;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int v = at * 64 + b * 16 + p;
      if (out.f32) {
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int col = col0 + a * 16 + g * 4;
          if (v >= r.V || col >= r.d) continue;
          f32x4* to = reinterpret_cast<f32x4*>(static_cast<float*>(out.out) + (int64_t)v * r.d + col);
          *to = out.add ? *to + acc[a][b] : acc[a][b];
        }
      } else {
#pragma unroll
        for (int a = 0; a < 4; a += 2) {
          const f32x4 x = acc[a][b], y = acc[a + 1][b];
          const u32x4 o = eight_rows(u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])},
                                     u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])});
          const int col = col0 + a * 16 + eight_rows_at(lane);
          if (v < r.V && col < r.d)
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out.out) + (int64_t)v * r.d + col) = o;
        }
      }
    }
  }
}

__global__ __launch_bounds__(256) void fill_zero_kernel(u32x4* __restrict__ p, int64_t n) {
  for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = u32x4{0, 0, 0, 0};
}

// ---- host ------------------------------------------------------------------------------------------
struct Call {
  const uint16_t *hidden, *w;
  int32_t N, d, V, k;
  float temperature, scale;
  uint32_t flags, allowed;
  void *dh, *dw;
  double* loss;
  int32_t* err;
  void* workspace;
  size_t workspace_bytes;
  hipStream_t stream;
  bool grads() const { return dh != nullptr || dw != nullptr; }
};

// The checks that the three calls share.
int check(const Call& c) {
  PSPO_REQUIRE(c.N >= 0, PSPO_ERR_INVALID_ARG, "N must be >= 0");
  PSPO_REQUIRE(c.d > 0 && c.V > 0, PSPO_ERR_INVALID_ARG, "d and V must be > 0");
  PSPO_REQUIRE(c.d % 8 == 0, PSPO_ERR_UNSUPPORTED, "d must be a multiple of 8");
  PSPO_REQUIRE(sizes_fit(c.N, c.d, c.V), PSPO_ERR_UNSUPPORTED,
               "N is at most 2^23, d 2^20, V 2^21, and N d, N V and V d 2^36");
  PSPO_REQUIRE((c.flags & ~c.allowed) == 0, PSPO_ERR_INVALID_ARG, "unknown flag bits");
  PSPO_REQUIRE((c.flags & PSPO_ACCUMULATE_DW) == 0 || (c.flags & PSPO_OBJ_DW_F32) != 0, PSPO_ERR_INVALID_ARG,
               "accumulating needs a float32 d_w_head");
  PSPO_REQUIRE(std::isfinite(c.temperature) && c.temperature > 0.f && std::isfinite(1.f / c.temperature),
               PSPO_ERR_INVALID_ARG, "temperature must be positive and finite");
  PSPO_REQUIRE(std::isfinite(c.scale), PSPO_ERR_INVALID_ARG, "loss_scale must be finite");
  PSPO_REQUIRE(c.loss != nullptr && aligned(c.loss, 8), PSPO_ERR_INVALID_ARG, "loss must be given, 8-byte aligned");
  PSPO_REQUIRE(aligned(c.dh, 16) && aligned(c.dw, 16), PSPO_ERR_INVALID_ARG,
               "d_hidden and d_w_head must be 16-byte aligned");
  PSPO_REQUIRE(aligned(c.err, 4), PSPO_ERR_INVALID_ARG, "misaligned err_flag");
  PSPO_REQUIRE(aligned(c.workspace, 256), PSPO_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (c.N > 0) {
    PSPO_REQUIRE(c.hidden && c.w, PSPO_ERR_INVALID_ARG, "null input pointer");
    PSPO_REQUIRE(aligned(c.hidden, 16) && aligned(c.w, 16), PSPO_ERR_INVALID_ARG,
                 "hidden and w_head must be 16-byte aligned");
  }
  return PSPO_OK;
}
int check_workspace(const Call& c, int64_t need) {
  PSPO_REQUIRE(need == 0 || c.workspace != nullptr, PSPO_ERR_INVALID_ARG, "workspace must be given");
  PSPO_REQUIRE((int64_t)c.workspace_bytes >= need, PSPO_ERR_WORKSPACE,
               "workspace too small: need " + std::to_string(need) + " bytes");
  return require_gfx950();
}

Rows rows_of(const Call& c, const Layout& s) {
  unsigned char* ws = static_cast<unsigned char*>(c.workspace);
  Rows r{};
  r.N = c.N;
  r.d = c.d;
  r.V = c.V;
  r.k = c.k;
  r.ld = s.ld;
  r.groups = s.groups;
  r.way = way_of(c.N, c.d, c.grads());
  r.grads = c.grads();
  r.group = s.group;
  r.inv_t = 1.0 / (double)c.temperature;
  r.use = reinterpret_cast<int32_t*>(ws + s.use);
  r.zs = reinterpret_cast<double*>(ws + s.zs);
  r.c = reinterpret_cast<float*>(ws + s.c);
  r.part = reinterpret_cast<f32x2*>(ws + s.part);
  r.f = reinterpret_cast<float*>(ws + s.f);
  r.ids = reinterpret_cast<int32_t*>(ws + s.ids);
  r.g = reinterpret_cast<float*>(ws + s.g);
  r.terms = reinterpret_cast<double*>(ws + s.terms);
  r.copy = reinterpret_cast<uint16_t*>(ws + s.copy);
  r.e = reinterpret_cast<uint16_t*>(ws + s.e);
  r.err = c.err;
  return r;
}

Exponent exponent_of(const Rows& r) {
  const double t = r.inv_t * 1.4426950408889634;
  return Exponent{(float)t, (float)(t - (double)(float)t)};
}

// The kernels of one pass by the width that they are built for.
template <int F, int... More, class Run>
int pass_width(int parts, const Run& run) {
  if (parts <= F) return run(std::integral_constant<int, F>{});
  if constexpr (sizeof...(More) > 0) return pass_width<More...>(parts, run);
  return fail(PSPO_ERR_UNSUPPORTED, "d is too wide for one pass");
}
int one_pass(const Call& c, const Rows& r, float* slab) {
  return pass_width<2, 4, 8, 12, 16, 20, 24, 28>((c.d + 32 * kPassWaves - 1) / (32 * kPassWaves), [&](auto f) {
    hipLaunchKernelGGL(one_pass_kernel<f.value>,
                       dim3((unsigned)pass_groups(c.N, c.d, c.V), (unsigned)((c.N + kPassRows - 1) / kPassRows)),
                       dim3(64 * kPassWaves), 0, c.stream, r, c.w, exponent_of(r), slab);
    PSPO_LAUNCHED("one_pass_kernel", c.stream);
    return (int)PSPO_OK;
  });
}
int one_pass_head(const Call& c, const Rows& r, const LossSum& loss) {
  const int64_t blocks = ((int64_t)c.V + 15) / 16;
  const int groups = (int)std::min<int64_t>((blocks + kHeadWaves - 1) / kHeadWaves, 256);
  return pass_width<1, 2, 4, 6, 10, 14>((c.d + 255) / 256, [&](auto f) {
    hipLaunchKernelGGL(one_pass_head_kernel<f.value>, dim3((unsigned)groups + 1), dim3(64 * kHeadWaves), 0, c.stream, r,
                       c.dw, (c.flags & PSPO_OBJ_DW_F32) != 0, (c.flags & PSPO_ACCUMULATE_DW) != 0, loss);
    PSPO_LAUNCHED("one_pass_head_kernel", c.stream);
    return (int)PSPO_OK;
  });
}

int stream_head(const Call& c, const Rows& r, const EpiGrad& out) {
  const int64_t tiles = ((int64_t)c.V + 63) / 64, chunks = (c.d + 255) / 256;
  return pass_width<1, 2>((c.N + 31) / 32, [&](auto ks) {
    // as many work-groups as run at once, those of one share of the vocabulary on one XCD
    const int64_t most = std::max<int64_t>(256 * kStreamPerCu / chunks / kNumXcd * kNumXcd, kNumXcd);
    hipLaunchKernelGGL(stream_head_kernel<ks.value>, dim3((unsigned)std::min(tiles, most), (unsigned)chunks + 1), dim3(256),
                       0, c.stream, r, out);
    PSPO_LAUNCHED("stream_head_kernel", c.stream);
    return (int)PSPO_OK;
  });
}

// Steps 1 to 3 (N > 0).
template <class Op>
int forward(const Call& c, const Layout& s, const Rows& r, const Op& op) {
  unsigned char* ws = static_cast<unsigned char*>(c.workspace);
  float *z = reinterpret_cast<float*>(ws + s.z), *slab = reinterpret_cast<float*>(ws + s.slab);
  auto gather = [&](auto threads, auto lanes) {
    constexpr int kThreads = decltype(threads)::value, kLanes = decltype(lanes)::value;
    hipLaunchKernelGGL((gather_kernel<kThreads, kLanes, Op>), dim3((unsigned)(((int64_t)c.N * kThreads + 255) / 256)),
                       dim3(256), 0, c.stream, r, op, c.hidden, c.w);
  };
  if (c.k > 4) gather(std::integral_constant<int, 256>{}, std::integral_constant<int, 16>{});
  else if (c.N < kTeamRows) gather(std::integral_constant<int, 256>{}, std::integral_constant<int, 64>{});
  else gather(std::integral_constant<int, 64>{}, std::integral_constant<int, 64>{});
  PSPO_LAUNCHED("gather_kernel", c.stream);
  if (r.way == kOnePass) {
    if (int rc = one_pass(c, r, slab)) return rc;
  } else if (r.way == kFew) {
    if (int rc = skinny<1>(SkinnyArgs{{c.w, c.w}, r.copy, c.V, c.N, c.d}, SkinnyLogits{z, s.ld}, "objective_logits",
                           c.stream))
      return rc;
    hipLaunchKernelGGL(few_groups_kernel, dim3((unsigned)c.N, (unsigned)s.groups), dim3(256), 0, c.stream, z, s.ld,
                       c.V, (const int32_t*)r.ids, c.k, exponent_of(r), r.part);
    PSPO_LAUNCHED("few_groups_kernel", c.stream);
  } else {
    const Plan p = plan_forward(c.V, c.N, c.d);
    if (int rc = product<false, false>(shape(c.w, c.w, c.d, c.V, r.copy, c.d, c.N, c.d), p, c.N,
                                       EpiSoftmax{r.e, r.part, r.c, c.k == 1 ? r.ids : nullptr, s.ld, c.V, c.N, exponent_of(r)},
                                       slab, "objective_logits", c.stream))
      return rc;
  }
  if (c.N < kTeamRows)
    hipLaunchKernelGGL((finalize_kernel<256, Op>), dim3((unsigned)c.N), dim3(256), 0, c.stream, r, op);
  else
    hipLaunchKernelGGL((finalize_kernel<64, Op>), dim3((unsigned)((c.N + 3) / 4)), dim3(256), 0, c.stream, r, op);
  PSPO_LAUNCHED("finalize_kernel", c.stream);
  return PSPO_OK;
}

// Step 4.
int backward(const Call& c, const Layout& s, const Rows& r, const LossSum& loss) {
  const bool both = c.dh != nullptr && c.dw != nullptr;
  const bool along = c.N > 0 && (r.way == kOnePass ? c.dw != nullptr : both);   // the loss's sum, with a launch below
  if (loss.loss != nullptr && !along) {
    hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(1024), 0, c.stream, loss);
    PSPO_LAUNCHED("loss_sum_kernel", c.stream);
  }
  if (!c.grads()) return PSPO_OK;
  unsigned char* ws = static_cast<unsigned char*>(c.workspace);
  float *z = reinterpret_cast<float*>(ws + s.z), *slab = reinterpret_cast<float*>(ws + s.slab);
  const bool f32 = (c.flags & PSPO_OBJ_DW_F32) != 0, add = (c.flags & PSPO_ACCUMULATE_DW) != 0;
  if (c.N == 0) {
    if (c.dw == nullptr || add) return PSPO_OK;
    hipLaunchKernelGGL(fill_zero_kernel, dim3(1024), dim3(256), 0, c.stream, static_cast<u32x4*>(c.dw),
                       (int64_t)c.V * c.d / (f32 ? 4 : 8));
    PSPO_LAUNCHED("fill_zero_kernel", c.stream);
    return PSPO_OK;
  }
  if (r.way == kOnePass && c.dh != nullptr) {
    hipLaunchKernelGGL(one_pass_hidden_kernel, dim3((unsigned)((c.d + 255) / 256), (unsigned)c.N),
                       dim3(64 * kHiddenWaves), 0, c.stream, r, c.w, (const float*)slab,
                       (int)pass_groups(c.N, c.d, c.V), c.dh, (c.flags & PSPO_OBJ_DH_F32) != 0);
    PSPO_LAUNCHED("one_pass_hidden_kernel", c.stream);
  }
  if (r.way == kOnePass && c.dw == nullptr) return PSPO_OK;
  if (r.way == kOnePass && c.N <= kPassRows) return one_pass_head(c, r, loss);
  if (r.way == kFew) {
    hipLaunchKernelGGL(few_entries_kernel, dim3((unsigned)c.N, (unsigned)((s.ld + 2047) / 2048)), dim3(256), 0,
                       c.stream, r, (const float*)z, exponent_of(r));
    PSPO_LAUNCHED("few_entries_kernel", c.stream);
  }
  const RowShape g[3] = {shape(c.w, c.w, c.d, c.d, r.e, s.ld, c.N, c.V),
                         shape(r.copy, r.copy, c.d, c.d, r.e, s.ld, c.V, c.N), RowShape{}};
  const EpiGrad o[3] = {{c.dh, r.f, c.d, c.d, c.N, (c.flags & PSPO_OBJ_DH_F32) != 0, 0, loss},
                        {c.dw, nullptr, c.d, c.d, c.V, f32, add, LossSum{}}, EpiGrad{}};
  if (r.way == kOnePass) {
    EpiGrad head = o[1];
    head.loss = loss;
    return stream_head(c, r, head);
  }
  if (both)
    return run_jobs(plan_gradients(c.N, c.d, c.V), g, o, reinterpret_cast<unsigned char*>(slab), "objective_gradients",
                    c.stream);
  if (c.dh != nullptr)
    return product<true, false>(g[0], plan_square(c.d, c.N, c.V), c.N, o[0], slab, "objective_dh", c.stream);
  return product<true, true>(g[1], plan_square(c.d, c.V, c.N), c.V, o[1], slab, "objective_dw", c.stream);
}

}  // namespace
}  // namespace pspo

extern "C" {

size_t pspo_policy_loss_workspace_bytes(int32_t N, int32_t d, int32_t V, int32_t grads) {
  return pspo::workspace_size(N, d, V, 1, 0, 0, grads != 0);
}
size_t pspo_preference_workspace_bytes(int32_t N, int32_t d, int32_t V, int32_t R, int32_t P, int32_t grads) {
  if (R < 0 || P < 0 || !pspo::pairs_fit(R, P)) return 0;
  return pspo::workspace_size(N, d, V, 1, R, P, grads != 0);
}
size_t pspo_distill_workspace_bytes(int32_t N, int32_t d, int32_t V, int32_t k, int32_t grads) {
  if (k < 1 || k > pspo::kMostIds) return 0;
  return pspo::workspace_size(N, d, V, k, 0, 0, grads != 0);
}

int pspo_policy_loss_fwd_bwd(const uint16_t* hidden, const uint16_t* w_head, const int32_t* target,
                             const float* logp_old, const float* logp_ref, const float* weight, const int32_t* seq_id,
                             const float* advantage, int32_t N, int32_t d, int32_t V, int32_t R, float eps_low,
                             float eps_high, float kl_coef, int32_t kl_kind, float temperature, float loss_scale,
                             uint32_t flags, double* loss, void* d_hidden, void* d_w_head, float* logp_new,
                             double* stats, int32_t* err_flag, void* workspace, size_t workspace_bytes,
                             hipStream_t stream) {
  using namespace pspo;
  clear_last_error();
  TraceRange trace_range("pspo_policy_loss_fwd_bwd");
  const Call c{hidden, w_head, N, d, V, 1, temperature, loss_scale, flags,
               PSPO_OBJ_DH_F32 | PSPO_OBJ_DW_F32 | PSPO_ACCUMULATE_DW, d_hidden, d_w_head, loss, err_flag, workspace,
               workspace_bytes, stream};
  if (int rc = check(c)) return rc;
  PSPO_REQUIRE(R >= 0 && (N == 0 || R > 0), PSPO_ERR_INVALID_ARG, "R must be > 0 when N > 0");
  PSPO_REQUIRE(std::isfinite(eps_low) && eps_low >= 0.f && eps_low < 1.f && std::isfinite(eps_high) &&
                   eps_high >= 0.f && eps_high < 1.f,
               PSPO_ERR_INVALID_ARG, "eps_low and eps_high must lie in [0, 1)");
  PSPO_REQUIRE(std::isfinite(kl_coef), PSPO_ERR_INVALID_ARG, "kl_coef must be finite");
  PSPO_REQUIRE(kl_kind >= PSPO_KL_K1 && kl_kind <= PSPO_KL_K3, PSPO_ERR_INVALID_ARG, "unknown kl_kind");
  PSPO_REQUIRE(kl_coef == 0.f || N == 0 || logp_ref != nullptr, PSPO_ERR_INVALID_ARG, "kl_coef needs logp_ref");
  PSPO_REQUIRE(aligned(logp_new, 4) && aligned(stats, 8), PSPO_ERR_INVALID_ARG, "misaligned output pointer");
  if (N > 0) {
    PSPO_REQUIRE(target && logp_old && weight && seq_id && advantage, PSPO_ERR_INVALID_ARG, "null input pointer");
    PSPO_REQUIRE(aligned(target, 4) && aligned(logp_old, 4) && aligned(logp_ref, 4) && aligned(weight, 4) &&
                     aligned(seq_id, 4) && aligned(advantage, 4),
                 PSPO_ERR_INVALID_ARG, "misaligned per-token pointer");
  }
  const Layout s = layout_of(N, d, V, 1, 0, 0, c.grads());
  if (int rc = check_workspace(c, N > 0 ? s.total : 0)) return rc;
  const Rows r = rows_of(c, s);
  if (N > 0)
    if (int rc = forward(c, s, r,
                         Policy{target, logp_old, logp_ref, weight, seq_id, advantage, R, eps_low, eps_high, kl_coef,
                                loss_scale, kl_kind, logp_new}))
      return rc;
  return backward(c, s, r, LossSum{r.terms, N, 4, {-1.f, kl_coef}, loss, stats});
}

int pspo_preference_fwd_bwd(const uint16_t* hidden, const uint16_t* w_head, const int32_t* target,
                            const float* logp_ref, const float* weight, const int32_t* cu_seqlens,
                            const int32_t* chosen, const int32_t* rejected, int32_t N, int32_t d, int32_t V, int32_t R,
                            int32_t P, int32_t kind, float beta, float smoothing, float temperature, float loss_scale,
                            uint32_t flags, double* loss, void* d_hidden, void* d_w_head, float* logp_new,
                            float* seq_ratio, float* margin, int32_t* err_flag, void* workspace,
                            size_t workspace_bytes, hipStream_t stream) {
  using namespace pspo;
  clear_last_error();
  TraceRange trace_range("pspo_preference_fwd_bwd");
  const Call c{hidden, w_head, N, d, V, 1, temperature, loss_scale, flags,
               PSPO_OBJ_DH_F32 | PSPO_OBJ_DW_F32 | PSPO_ACCUMULATE_DW | PSPO_PREF_AVERAGE, d_hidden, d_w_head, loss,
               err_flag, workspace, workspace_bytes, stream};
  if (int rc = check(c)) return rc;
  PSPO_REQUIRE(R >= 0 && P >= 0, PSPO_ERR_INVALID_ARG, "R and P must be >= 0");
  PSPO_REQUIRE(pairs_fit(R, P), PSPO_ERR_UNSUPPORTED, "R is at most 2^23, R P 2^36");
  PSPO_REQUIRE(kind == PSPO_PREF_SIGMOID || kind == PSPO_PREF_SQUARED, PSPO_ERR_INVALID_ARG, "unknown kind");
  PSPO_REQUIRE(std::isfinite(beta) && beta > 0.f && std::isfinite(1.f / beta), PSPO_ERR_INVALID_ARG,
               "beta must be positive and finite");
  PSPO_REQUIRE(std::isfinite(smoothing) && smoothing >= 0.f && smoothing <= 1.f, PSPO_ERR_INVALID_ARG,
               "smoothing must lie in [0, 1]");
  PSPO_REQUIRE(kind == PSPO_PREF_SIGMOID || smoothing == 0.f, PSPO_ERR_INVALID_ARG,
               "smoothing belongs to PSPO_PREF_SIGMOID");
  PSPO_REQUIRE(cu_seqlens != nullptr && (P == 0 || (chosen && rejected)), PSPO_ERR_INVALID_ARG, "null input pointer");
  PSPO_REQUIRE(N == 0 || target, PSPO_ERR_INVALID_ARG, "null input pointer");
  PSPO_REQUIRE(aligned(target, 4) && aligned(logp_ref, 4) && aligned(weight, 4) && aligned(cu_seqlens, 4) &&
                   aligned(chosen, 4) && aligned(rejected, 4) && aligned(logp_new, 4) && aligned(seq_ratio, 4) &&
                   aligned(margin, 4),
               PSPO_ERR_INVALID_ARG, "misaligned pointer");
  const Layout s = layout_of(N, d, V, 1, R, P, c.grads());
  if (int rc = check_workspace(c, s.total)) return rc;
  const Rows r = rows_of(c, s);
  double* seqs = reinterpret_cast<double*>(static_cast<unsigned char*>(workspace) + s.seqs);
  double* pairs = reinterpret_cast<double*>(static_cast<unsigned char*>(workspace) + s.pairs);
  const Pairs q{cu_seqlens, chosen, rejected, R, P, kind, (flags & PSPO_PREF_AVERAGE) != 0, beta, smoothing, loss_scale,
                seqs, seqs + R, seqs + 2 * (int64_t)R, pairs, pairs + P, seq_ratio, margin, err_flag};
  if (N > 0)
    if (int rc = forward(c, s, r, Preference{target, logp_ref, weight, logp_new})) return rc;
  if (N <= kPrefRows && (int64_t)R * P <= kPrefLooks) {
    hipLaunchKernelGGL(pref_all_kernel, dim3(1), dim3(64 * kPrefWaves), 0, stream, q, N, (const double*)r.terms, loss);
    PSPO_LAUNCHED("pref_all_kernel", stream);
  } else {
    if (R > 0) {
      hipLaunchKernelGGL(pref_sequences_kernel, dim3((unsigned)R), dim3(256), 0, stream, q, N, (const double*)r.terms);
      PSPO_LAUNCHED("pref_sequences_kernel", stream);
    }
    if (P > 0) {
      hipLaunchKernelGGL(pref_pairs_kernel, dim3((unsigned)(((int64_t)P + 255) / 256)), dim3(256), 0, stream, q);
      PSPO_LAUNCHED("pref_pairs_kernel", stream);
    }
    hipLaunchKernelGGL(pref_coef_kernel, dim3((unsigned)R + 1), dim3(256), 0, stream, q, loss);
    PSPO_LAUNCHED("pref_coef_kernel", stream);
  }
  if (N > 0 && c.grads()) {
    if (N < kTeamRows) hipLaunchKernelGGL(pref_rows_kernel<256>, dim3((unsigned)N), dim3(256), 0, stream, r, q);
    else hipLaunchKernelGGL(pref_rows_kernel<64>, dim3((unsigned)((N + 3) / 4)), dim3(256), 0, stream, r, q);
    PSPO_LAUNCHED("pref_rows_kernel", stream);
  }
  return backward(c, s, r, LossSum{});
}

int pspo_distill_fwd_bwd(const uint16_t* hidden, const uint16_t* w_head, const int32_t* topk_ids,
                         const float* topk_logit, const float* weight, int32_t N, int32_t d, int32_t V, int32_t k,
                         float temperature, float loss_scale, uint32_t flags, double* loss, void* d_hidden,
                         void* d_w_head, float* kl, int32_t* err_flag, void* workspace, size_t workspace_bytes,
                         hipStream_t stream) {
  using namespace pspo;
  clear_last_error();
  TraceRange trace_range("pspo_distill_fwd_bwd");
  const Call c{hidden, w_head, N, d, V, k, temperature, loss_scale, flags,
               PSPO_OBJ_DH_F32 | PSPO_OBJ_DW_F32 | PSPO_ACCUMULATE_DW, d_hidden, d_w_head, loss, err_flag, workspace,
               workspace_bytes, stream};
  if (int rc = check(c)) return rc;
  PSPO_REQUIRE(k >= 1 && k <= kMostIds, PSPO_ERR_UNSUPPORTED, "k must lie in 1 .. 64");
  PSPO_REQUIRE(N == 0 || (topk_ids && topk_logit), PSPO_ERR_INVALID_ARG, "null input pointer");
  PSPO_REQUIRE(aligned(topk_ids, 4) && aligned(topk_logit, 4) && aligned(weight, 4) && aligned(kl, 4),
               PSPO_ERR_INVALID_ARG, "misaligned pointer");
  const Layout s = layout_of(N, d, V, k, 0, 0, c.grads());
  if (int rc = check_workspace(c, N > 0 ? s.total : 0)) return rc;
  const Rows r = rows_of(c, s);
  if (N > 0)
    if (int rc = forward(c, s, r, Distill{topk_ids, topk_logit, weight, loss_scale, kl})) return rc;
  return backward(c, s, r, LossSum{r.terms, N, 1, {1.f, 0.f}, loss, nullptr});
}

}  // extern "C"
