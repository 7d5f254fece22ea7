// Norms of queries and keys for each head with the position rotation in the
// same pass, and their gradient.
//
// Bound: HBM (each element read once and written once; the backward reads the
// input and the output's gradient).  A head's D entries lie on L lanes (D / 8
// rounded up to a power of two) with eight consecutive entries each, so the
// mean is log2 L exchanges within the wave, the partner of an entry in the
// half-split rotation sits in the same place of another lane (rot_dim is a
// multiple of 16), and a neighbouring pair in the same lane.  A wave takes one
// token at a time: the token's rot_dim / 2 angles are formed once (in float64:
// a float32 product pos * inv_freq is off by 0.004 rad at position 65,536) and
// serve all of its heads, 64 / L heads at once.
#include "pspo_layer.h"
#include "token_plan.h"
#include "vec8.h"

namespace pspo {
namespace {

constexpr int kMaxDim = 512;
constexpr int kWaves = kQkWaves;

struct QkArgs {
  const unsigned char *q, *k;        // inputs
  int64_t q_row, k_row;              // bytes between tokens
  const unsigned char *qw, *kw;      // NULL: ones
  const float* inv_freq;
  const int32_t *positions, *seq_id, *cu, *first;
  int32_t N, R, Hq, Hk, D, rot;
  float eps, inv_d;
  int interleaved, norm;
  unsigned char *q_out, *k_out;      // forward: outputs; backward: dq, dk
  const unsigned char *dq_out, *dk_out;
  float* partials;                   // backward: [work-groups][2][D], or NULL
  int32_t* err_flag;
  int32_t per_part;                  // passes of 64 / L heads that one grid row takes (forward)
};

__device__ __forceinline__ int64_t position_of(const QkArgs& a, int n, bool report) {
  if (a.positions) return a.positions[n];
  const int32_t r = a.seq_id[n];
  if (r < 0 || r >= a.R) {
    if (report && a.err_flag) atomicOr(a.err_flag, PSPO_DEVERR_SEQ_ID);
    return 0;
  }
  return (int64_t)(a.first ? a.first[r] : 0) + n - a.cu[r];
}

// The token's cosines and sines, rot / 2 of each, by the wave's lanes.
__device__ __forceinline__ void angles(const QkArgs& a, int n, int lane, float* cs, float* sn) {
  const double turns = (double)position_of(a, n, lane == 0) * 0.15915494309189533577;
  for (int i = lane; i < a.rot / 2; i += 64) {
    double t = turns * (double)a.inv_freq[i];
    t -= rint(t);                     // whole turns drop out exactly
    float s, c;
    sincospif(2.f * (float)t, &s, &c);
    cs[i] = c;
    sn[i] = s;
  }
}

// What a lane needs of the angles: for its entries 8 c .. 8 c + 7 of a head the
// cosine and the factor of the partner entry, and which lane holds the partner
// (itself: neighbouring pairs, or entries that are not turned).
struct LaneTurn {
  float c[8], s[8];
  int partner;      // lane offset to the partner's lane
  bool half_row;    // the same in every lane: the partner sits across the row of 16 lanes
};

// dir: +1 forward, -1 back (the transpose).
__device__ __forceinline__ LaneTurn lane_turn(const QkArgs& a, int chunk, const float* cs, const float* sn, float dir) {
  LaneTurn t;
  t.partner = 0;
  t.half_row = a.D == 128 && a.rot == 128;
  const int e0 = chunk * 8;
  if (e0 >= a.rot) {   // not turned (rot is a multiple of 16, so a lane's entries agree)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      t.c[j] = 1.f;
      t.s[j] = 0.f;
    }
    return t;
  }
  if (a.interleaved) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      t.c[j] = cs[(e0 + j) / 2];
      t.s[j] = (j & 1 ? dir : -dir) * sn[(e0 + j) / 2];
    }
    return t;
  }
  const int half = a.rot / 2;
  const bool low = e0 < half;
  t.partner = low ? half / 8 : -(half / 8);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int i = low ? e0 + j : e0 + j - half;
    t.c[j] = cs[i];
    t.s[j] = (low ? -dir : dir) * sn[i];
  }
  return t;
}

template <int kCtrl>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kCtrl, 0xF, 0xF, true));
}

// Sum over the head's L lanes, in each of them: up to 16 lanes by moves within a row of 16
// (quads, then mirrored halves), which go at the vector rate, beyond by exchanges through LDS.
template <int L>
__device__ __forceinline__ float head_sum(float x) {
  if constexpr (L >= 2) x += dpp<0xB1>(x);    // quad_perm 1, 0, 3, 2
  if constexpr (L >= 4) x += dpp<0x4E>(x);    // quad_perm 2, 3, 0, 1
  if constexpr (L >= 8) x += dpp<0x141>(x);   // row_half_mirror: the other quad of eight
  if constexpr (L >= 16) x += dpp<0x140>(x);  // row_mirror: the other half of sixteen
#pragma unroll
  for (int m = 16; m < L; m <<= 1) x += __shfl_xor(x, m);
  return x;
}

__device__ __forceinline__ Vec8 turn(const Vec8& z, const LaneTurn& t, int interleaved, int lane) {
  Vec8 o;
  if (interleaved) {   // uniform over the call
#pragma unroll
    for (int j = 0; j < 8; ++j) o.v[j] = z.v[j] * t.c[j] + z.v[j ^ 1] * t.s[j];
  } else if (t.half_row) {   // uniform: heads of 16 lanes turned whole, the partner 8 lanes on
#pragma unroll
    for (int j = 0; j < 8; ++j) o.v[j] = z.v[j] * t.c[j] + dpp<0x128>(z.v[j]) * t.s[j];   // row_ror:8
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) o.v[j] = z.v[j] * t.c[j] + __shfl(z.v[j], lane + t.partner) * t.s[j];
  }
  // an entry that is not turned is passed on as it is (0 * Inf would make a NaN of it)
  return o;
}

template <class T>
__device__ __forceinline__ Vec8 weight8(const unsigned char* w, int chunk, bool use) {
  if (w != nullptr && use) return unpack8(load8<T>(w, chunk));
  Vec8 o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o.v[j] = 1.f;
  return o;
}

// One wave per token (and per grid row, a span of its passes), heads in the
// order queries, keys; a pass takes 64 / L heads.
template <class T, int L, bool kPast>
__global__ __launch_bounds__(64 * kWaves) void qk_fwd_kernel(QkArgs a) {
  constexpr int kHeads = 64 / L;
  __shared__ float cs[kWaves][kMaxDim / 2], sn[kWaves][kMaxDim / 2];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t n = (int64_t)blockIdx.x * kWaves + wave;
  const bool live = n < a.N;
  if (live && a.rot) angles(a, (int)n, lane, cs[wave], sn[wave]);
  __syncthreads();
  if (!live) return;
  const int chunk = lane % L, sub = lane / L;
  const bool inside = chunk * 8 < a.D;
  const LaneTurn t = lane_turn(a, chunk, cs[wave], sn[wave], 1.f);
  const bool turned = chunk * 8 < a.rot;
  const Vec8 qw = weight8<T>(a.qw, chunk, inside), kw = weight8<T>(a.kw, chunk, inside);
  const int64_t head_bytes = (int64_t)a.D * T::kBytes;
  const int passes_q = (a.Hq + kHeads - 1) / kHeads, passes_k = (a.Hk + kHeads - 1) / kHeads;
  const int p0 = blockIdx.y * a.per_part, p1 = min(p0 + a.per_part, passes_q + passes_k);
  constexpr int kAhead = 4;   // passes loaded before the first is used
  for (int pb = p0; pb < p1; pb += kAhead) {
    Raw8<T> raw[kAhead];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int p = pb + s;
      const bool is_q = p < passes_q;
      const int h = (is_q ? p : p - passes_q) * kHeads + sub;
      raw[s] = Raw8<T>{};
      if (p < p1 && inside && h < (is_q ? a.Hq : a.Hk))
        raw[s] = load8<T>((is_q ? a.q + n * a.q_row : a.k + n * a.k_row) + h * head_bytes, chunk);
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int p = pb + s;
      if (p >= p1) break;
      const bool is_q = p < passes_q;
      const int h = (is_q ? p : p - passes_q) * kHeads + sub;
      Vec8 z = unpack8(raw[s]);
      if (a.norm) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) ss += z.v[j] * z.v[j];
        const float rstd = 1.f / sqrtf(head_sum<L>(ss) * a.inv_d + a.eps);
#pragma unroll
        for (int j = 0; j < 8; ++j) z.v[j] = z.v[j] * rstd * (is_q ? qw.v[j] : kw.v[j]);
      }
      const Vec8 o = turn(z, t, a.interleaved, lane);
      if (inside && h < (is_q ? a.Hq : a.Hk))
        store8<T, kPast>((is_q ? a.q_out + n * a.Hq * head_bytes : a.k_out + n * a.Hk * head_bytes) + h * head_bytes, chunk,
                  turned ? o : z);
    }
  }
}

// Grid y: queries, keys.  Waves walk the tokens in steps of grid x and keep their sums of
// dz * xhat in registers; a work-group's sums are joined in LDS, in wave order, and left in
// `partials`.  (One work-group for both sides held two sets of sums and weights: 196 registers,
// two waves to a SIMD: 138 us against 131 at 28,481 tokens of 28 + 4 heads of 128.)
template <class T, int L, bool kPast>
__global__ __launch_bounds__(64 * kWaves) void qk_bwd_kernel(QkArgs a) {
  constexpr int kHeads = 64 / L;
  __shared__ float cs[kWaves][kMaxDim / 2], sn[kWaves][kMaxDim / 2];
  __shared__ float sums[kWaves][kMaxDim];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int chunk = lane % L, sub = lane / L;
  const bool inside = chunk * 8 < a.D, turned = chunk * 8 < a.rot;
  const bool keys = blockIdx.y != 0;
  const Vec8 w = weight8<T>(keys ? a.kw : a.qw, chunk, inside);
  const int H = keys ? a.Hk : a.Hq;
  const int64_t head_bytes = (int64_t)a.D * T::kBytes, row_in = keys ? a.k_row : a.q_row, row_out = H * head_bytes;
  const unsigned char *in = keys ? a.k : a.q, *grad = keys ? a.dk_out : a.dq_out;
  unsigned char* out = keys ? a.k_out : a.q_out;
  float acc[8] = {};
  // every wave of a work-group runs the same count of steps (the barriers)
  for (int64_t n0 = (int64_t)blockIdx.x * kWaves; H > 0 && n0 < a.N; n0 += (int64_t)gridDim.x * kWaves) {
    const int64_t n = n0 + wave;
    const bool live = n < a.N;
    __syncthreads();
    if (live && a.rot) angles(a, (int)n, lane, cs[wave], sn[wave]);
    __syncthreads();
    if (!live) continue;
    const LaneTurn t = lane_turn(a, chunk, cs[wave], sn[wave], -1.f);
    const unsigned char *xin = in + n * row_in, *din = grad + n * row_out;
    unsigned char* dst = out + n * row_out;
    constexpr int kAhead = 2;
    for (int hb = 0; hb < H; hb += kAhead * kHeads) {
      Raw8<T> xr[kAhead], dr[kAhead];
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        const int h = hb + s * kHeads + sub;
        xr[s] = Raw8<T>{};
        dr[s] = Raw8<T>{};
        if (inside && h < H) {
          xr[s] = load8<T, kPast>(xin + h * head_bytes, chunk);
          dr[s] = load8<T, kPast>(din + h * head_bytes, chunk);
        }
      }
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        if (hb + s * kHeads >= H) break;
        const int h = hb + s * kHeads + sub;
        const Vec8 x = unpack8(xr[s]), d = unpack8(dr[s]);
        Vec8 dz = turn(d, t, a.interleaved, lane);
        if (!turned) dz = d;
        if (a.norm) {
          float ss = 0.f, dot = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            ss += x.v[j] * x.v[j];
            dot += dz.v[j] * w.v[j] * x.v[j];
          }
          const float rstd = 1.f / sqrtf(head_sum<L>(ss) * a.inv_d + a.eps);
          const float m = head_sum<L>(dot) * a.inv_d * rstd * rstd;   // mean(dz w xhat) / rms
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            acc[j] += dz.v[j] * (x.v[j] * rstd);
            dz.v[j] = rstd * (dz.v[j] * w.v[j] - x.v[j] * m);
          }
        }
        if (inside && h < H) store8<T, kPast>(dst + h * head_bytes, chunk, dz);
      }
    }
  }
  if (a.partials == nullptr) return;   // uniform: no weight gradient is wanted
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float x = acc[j];
#pragma unroll
    for (int m = L; m < 64; m <<= 1) x += __shfl_xor(x, m);
    if (sub == 0 && inside) sums[wave][chunk * 8 + j] = x;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.D; e += 64 * kWaves) {
    float x = 0.f;
#pragma unroll
    for (int w4 = 0; w4 < kWaves; ++w4) x += sums[w4][e];
    a.partials[((int64_t)blockIdx.x * 2 + (keys ? 1 : 0)) * a.D + e] = x;
  }
}

// dw[e] = the work-groups' partial sums added in order: 64 threads take every
// 64th of them, joined by halves.
__global__ __launch_bounds__(1024) void qk_dweight_kernel(const float* partials, int groups, int D, float* dqw,
                                                          float* dkw) {
  __shared__ float s[64][16];
  const int c = threadIdx.x % 16, r = threadIdx.x / 16;
  const int i = blockIdx.x * 16 + c;   // < 2 D: 2 D is a multiple of 16
  float x = 0.f;
  for (int g = r; g < groups; g += 64) x += partials[(int64_t)g * 2 * D + i];
  s[r][c] = x;
  __syncthreads();
  for (int m = 32; m > 0; m >>= 1) {
    if (r < m) s[r][c] += s[r + m][c];
    __syncthreads();
  }
  if (r == 0) {
    float* dst = i < D ? dqw : dkw;
    if (dst) dst[i % D] = s[0][c];
  }
}

template <class T, bool kPast>
void launch_fwd(const QkArgs& a, int L, dim3 grid, hipStream_t stream) {
#define PSPO_QK(W) \
  case W: hipLaunchKernelGGL((qk_fwd_kernel<T, W, kPast>), grid, dim3(64 * kWaves), 0, stream, a); break
  switch (L) { PSPO_QK(1); PSPO_QK(2); PSPO_QK(4); PSPO_QK(8); PSPO_QK(16); PSPO_QK(32); PSPO_QK(64); }
#undef PSPO_QK
}
template <class T, bool kPast>
void launch_bwd(const QkArgs& a, int L, dim3 grid, hipStream_t stream) {
#define PSPO_QK(W) \
  case W: hipLaunchKernelGGL((qk_bwd_kernel<T, W, kPast>), grid, dim3(64 * kWaves), 0, stream, a); break
  switch (L) { PSPO_QK(1); PSPO_QK(2); PSPO_QK(4); PSPO_QK(8); PSPO_QK(16); PSPO_QK(32); PSPO_QK(64); }
#undef PSPO_QK
}
template <class T>
void launch(const QkArgs& a, int L, dim3 grid, bool backward, hipStream_t stream) {
  const bool p = qk_past(a.N, a.Hq + a.Hk, a.D, T::kBytes, backward);
  if (backward) p ? launch_bwd<T, true>(a, L, grid, stream) : launch_bwd<T, false>(a, L, grid, stream);
  else p ? launch_fwd<T, true>(a, L, grid, stream) : launch_fwd<T, false>(a, L, grid, stream);
}

bool head_dim_fits(int32_t D) { return D >= 8 && D % 8 == 0 && D <= kMaxDim; }
// A launch holds less than 2^32 threads along x.
bool tokens_fit(int32_t N) { return token_groups(N) < (int64_t(1) << 24); }

// Checks shared by both directions; fills the common arguments.
int check(const void* q, const void* k, int64_t q_stride, int64_t k_stride, const void* qw, const void* kw,
          const float* inv_freq, const int32_t* positions, const int32_t* seq_id, const int32_t* cu,
          const int32_t* first, int32_t N, int32_t R, int32_t Hq, int32_t Hk, int32_t D, int32_t rot, float eps,
          int32_t type, uint32_t flags, int32_t* err_flag, QkArgs& a) {
  PSPO_REQUIRE(N >= 0 && R >= 0, PSPO_ERR_INVALID_ARG, "N and R must be >= 0");
  PSPO_REQUIRE(Hq >= 1 && Hk >= 0, PSPO_ERR_INVALID_ARG, "heads_q must be >= 1 and heads_k >= 0");
  PSPO_REQUIRE(Hq <= 65536 && Hk <= 65536, PSPO_ERR_UNSUPPORTED, "at most 65536 heads");
  PSPO_REQUIRE(head_dim_fits(D), PSPO_ERR_UNSUPPORTED,
               "head_dim must be a multiple of 8, at most 512");
  PSPO_REQUIRE(rot >= 0 && rot % 16 == 0 && rot <= D, PSPO_ERR_UNSUPPORTED,
               "rot_dim must be a multiple of 16, at most head_dim");
  PSPO_REQUIRE((flags & ~(PSPO_ROPE_INTERLEAVED | PSPO_QK_NO_NORM)) == 0, PSPO_ERR_INVALID_ARG, "unknown flag bits");
  PSPO_REQUIRE(type == PSPO_TYPE_BF16 || type == PSPO_TYPE_F32, PSPO_ERR_INVALID_ARG, "unknown element type");
  const bool norm = (flags & PSPO_QK_NO_NORM) == 0;
  PSPO_REQUIRE(!norm || (eps > 0.f && eps < 1e30f), PSPO_ERR_INVALID_ARG, "eps must be positive and finite");
  PSPO_REQUIRE(norm || (qw == nullptr && kw == nullptr), PSPO_ERR_INVALID_ARG, "weights need the norm");
  const int64_t b = type == PSPO_TYPE_F32 ? 4 : 2;
  PSPO_REQUIRE(q_stride >= (int64_t)Hq * D && (Hk == 0 || k_stride >= (int64_t)Hk * D), PSPO_ERR_INVALID_ARG,
               "row strides must be at least heads * head_dim");
  PSPO_REQUIRE(q_stride * b % 16 == 0 && (Hk == 0 || k_stride * b % 16 == 0), PSPO_ERR_INVALID_ARG,
               "rows must be 16-byte aligned");
  PSPO_REQUIRE(q_stride < (int64_t(1) << 40) && (Hk == 0 || k_stride < (int64_t(1) << 40)), PSPO_ERR_INVALID_ARG,
               "row stride out of range");
  PSPO_REQUIRE(tokens_fit(N), PSPO_ERR_UNSUPPORTED, "at most 2^26 tokens per call");
  if (N > 0) {
    PSPO_REQUIRE(q && (k || Hk == 0), PSPO_ERR_INVALID_ARG, "null input pointer");
    PSPO_REQUIRE(aligned(q, 16) && aligned(k, 16) && aligned(qw, 16) && aligned(kw, 16) && aligned(inv_freq, 4) &&
                     aligned(positions, 4) && aligned(seq_id, 4) && aligned(cu, 4) && aligned(first, 4),
                 PSPO_ERR_INVALID_ARG, "misaligned pointer argument");
    if (rot > 0) {
      PSPO_REQUIRE(inv_freq, PSPO_ERR_INVALID_ARG, "inv_freq is NULL");
      PSPO_REQUIRE(positions || (seq_id && cu), PSPO_ERR_INVALID_ARG,
                   "positions, or seq_id and cu_seqlens, must be given");
    }
  }
  a.q = static_cast<const unsigned char*>(q);
  a.k = static_cast<const unsigned char*>(k);
  a.q_row = q_stride * b;
  a.k_row = k_stride * b;
  a.qw = static_cast<const unsigned char*>(qw);
  a.kw = static_cast<const unsigned char*>(kw);
  a.inv_freq = inv_freq;
  a.positions = positions;
  a.seq_id = seq_id;
  a.cu = cu;
  a.first = first;
  a.N = N;
  a.R = R;
  a.Hq = Hq;
  a.Hk = Hk;
  a.D = D;
  a.rot = rot;
  a.eps = eps;
  a.inv_d = 1.f / (float)D;
  a.interleaved = (flags & PSPO_ROPE_INTERLEAVED) != 0;
  a.norm = norm;
  a.err_flag = err_flag;
  return PSPO_OK;
}

}  // namespace
}  // namespace pspo

extern "C" {

int pspo_qk_norm_rope_fwd(const void* q, const void* k, int64_t q_stride, int64_t k_stride, const void* q_weight,
                          const void* k_weight, const float* inv_freq, const int32_t* positions,
                          const int32_t* seq_id, const int32_t* cu_seqlens, const int32_t* first_pos, int32_t N,
                          int32_t R, int32_t heads_q, int32_t heads_k, int32_t head_dim, int32_t rot_dim, float eps,
                          int32_t type, uint32_t flags, void* q_out, void* k_out, int32_t* err_flag,
                          hipStream_t stream) {
  using namespace pspo;
  clear_last_error();
  TraceRange trace_range("pspo_qk_norm_rope_fwd");
  QkArgs a{};
  if (int rc = check(q, k, q_stride, k_stride, q_weight, k_weight, inv_freq, positions, seq_id, cu_seqlens, first_pos,
                     N, R, heads_q, heads_k, head_dim, rot_dim, eps, type, flags, err_flag, a))
    return rc;
  if (N == 0) return PSPO_OK;
  PSPO_REQUIRE(q_out && (k_out || heads_k == 0), PSPO_ERR_INVALID_ARG, "null output pointer");
  PSPO_REQUIRE(aligned(q_out, 16) && aligned(k_out, 16), PSPO_ERR_INVALID_ARG, "misaligned pointer argument");
  if (int rc = require_gfx950()) return rc;
  a.q_out = static_cast<unsigned char*>(q_out);
  a.k_out = static_cast<unsigned char*>(k_out);
  const int L = lanes_of(head_dim);
  const QkForward p = qk_forward(N, heads_q, heads_k, head_dim);
  a.per_part = p.per_part;
  const dim3 grid((uint32_t)p.gx, (uint32_t)p.parts);
  if (type == PSPO_TYPE_F32) launch<F32>(a, L, grid, false, stream);
  else launch<Bf16>(a, L, grid, false, stream);
  PSPO_LAUNCHED("qk_fwd_kernel", stream);
  return PSPO_OK;
}

size_t pspo_qk_norm_rope_workspace_bytes(int32_t N, int32_t head_dim) {
  if (N < 0 || !pspo::tokens_fit(N) || !pspo::head_dim_fits(head_dim)) return 0;
  return (size_t)pspo::bwd_groups(N) * 2 * (size_t)head_dim * sizeof(float);
}

int pspo_qk_norm_rope_bwd(const void* dq_out, const void* dk_out, const void* q, const void* k, int64_t q_stride,
                          int64_t k_stride, const void* q_weight, const void* k_weight, const float* inv_freq,
                          const int32_t* positions, const int32_t* seq_id, const int32_t* cu_seqlens,
                          const int32_t* first_pos, int32_t N, int32_t R, int32_t heads_q, int32_t heads_k,
                          int32_t head_dim, int32_t rot_dim, float eps, int32_t type, uint32_t flags, void* dq,
                          void* dk, float* dq_weight, float* dk_weight, int32_t* err_flag, void* workspace,
                          size_t workspace_bytes, hipStream_t stream) {
  using namespace pspo;
  clear_last_error();
  TraceRange trace_range("pspo_qk_norm_rope_bwd");
  QkArgs a{};
  if (int rc = check(q, k, q_stride, k_stride, q_weight, k_weight, inv_freq, positions, seq_id, cu_seqlens, first_pos,
                     N, R, heads_q, heads_k, head_dim, rot_dim, eps, type, flags, err_flag, a))
    return rc;
  PSPO_REQUIRE((q_weight || !dq_weight) && (k_weight || !dk_weight), PSPO_ERR_INVALID_ARG,
               "a weight's gradient needs the weight");
  PSPO_REQUIRE(aligned(dq_weight, 4) && aligned(dk_weight, 4), PSPO_ERR_INVALID_ARG, "misaligned pointer argument");
  const bool want = dq_weight || dk_weight;
  if (N > 0) {
    PSPO_REQUIRE(dq_out && dq && ((dk_out && dk) || heads_k == 0), PSPO_ERR_INVALID_ARG, "null pointer argument");
    PSPO_REQUIRE(aligned(dq_out, 16) && aligned(dk_out, 16) && aligned(dq, 16) && aligned(dk, 16),
                 PSPO_ERR_INVALID_ARG, "misaligned pointer argument");
    if (want) {
      PSPO_REQUIRE(workspace && aligned(workspace, 16), PSPO_ERR_INVALID_ARG, "workspace is NULL or misaligned");
      PSPO_REQUIRE(workspace_bytes >= pspo_qk_norm_rope_workspace_bytes(N, head_dim), PSPO_ERR_WORKSPACE,
                   "workspace is smaller than pspo_qk_norm_rope_workspace_bytes()");
    }
  }
  if (N == 0 && !want) return PSPO_OK;
  if (int rc = require_gfx950()) return rc;
  const int groups = bwd_groups(N);
  if (N > 0) {
    a.dq_out = static_cast<const unsigned char*>(dq_out);
    a.dk_out = static_cast<const unsigned char*>(dk_out);
    a.q_out = static_cast<unsigned char*>(dq);
    a.k_out = static_cast<unsigned char*>(dk);
    a.partials = want ? static_cast<float*>(workspace) : nullptr;
    const int L = lanes_of(head_dim);
    if (type == PSPO_TYPE_F32) launch<F32>(a, L, dim3(groups, 2), true, stream);
    else launch<Bf16>(a, L, dim3(groups, 2), true, stream);
    PSPO_LAUNCHED("qk_bwd_kernel", stream);
  }
  if (want) {
    hipLaunchKernelGGL(qk_dweight_kernel, dim3(2 * head_dim / 16), dim3(1024), 0, stream,
                       static_cast<const float*>(workspace), groups, head_dim, dq_weight, dk_weight);
    PSPO_LAUNCHED("qk_dweight_kernel", stream);
  }
  return PSPO_OK;
}

}  // extern "C"
