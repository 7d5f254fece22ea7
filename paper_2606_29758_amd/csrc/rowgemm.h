// Tiled bf16 x bf16 -> float32 matrix-core product on operands as they lie in
// row-major memory, with a pluggable epilogue:
//
//   C(m, n) = sum_k A(m, k) B(n, k),
//
// each operand either K-inner (rows of K entries: A[m * ld + k]) or K-outer
// (rows of M entries: A[k * ld + m]), so that the forward (weights and tokens
// K-inner), the input gradients (weights K-outer) and the weight gradients (both
// K-outer) of a linear layer need no transposed copy of anything.
//
// Tile: a 256-thread work-group (2 x 2 wave64s) owns (32 BM) x (32 BN) entries of
// C, each wave BM x BN blocks of v_mfma_f32_16x16x32_bf16 in the accumulator
// registers.  K advances in stages of 64 through a ring of two or four LDS buffers
// filled by buffer loads that write LDS directly; the buffer descriptor's range check
// turns rows and K past the operand's end into zeros, so no size need be a
// multiple of the tile.
//  * K-inner stages hold rows of 64 K entries (128 bytes): row r keeps its
//    16-byte chunk c at place c ^ (r & 7), so the 16-row operand reads (16 bytes
//    a lane) meet every bank once.
//  * K-outer stages hold one row of the tile's M entries per k, read through the
//    LDS transpose read (16 lanes take 4 rows x 16 entries, 8 bytes each, and
//    get 4 rows of one entry); the 32-byte pieces of row k sit at place
//    p ^ x(k), x(k) = (k & 3) | (k >> 3 & 3) << 2, so the 16 rows that one read
//    of a wave touches lie in 16 (8 on a 128-entry row) different places.
// Schedule: while the MFMAs of one half stage (32 K) run on one set of operand
// registers the other set is read, at most one LDS read or load after each MFMA;
// one barrier per stage, in its middle, behind which the stage's buffer is free
// for the loads of the stage that takes its place in the ring (two or four on).
#pragma once

#include "gemm.h"

namespace pspo {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kRowK = 64;                 // K entries per stage

struct RowOperand {
  const uint16_t* p[2];    // p[1]: second K segment (or the second half of interleaved rows)
  int64_t ld;              // entries between rows in memory
  int rows;                // M (or N) entries that exist
  int64_t seg_off;         // K-inner: entries from one K segment to the next within a row
};

struct RowShape {
  RowOperand a, b;
  int K, segs;             // K per segment, number of segments (1 or 2)
  int tiles_m, tiles_n;
  int tile0, count;        // this launch's tiles: positions [tile0, tile0 + count) of the order below
  int parts;               // K parts (grid y)
};

constexpr int kGroupRows = 4;   // row tiles x all column tiles per group of the tile order

// Position t of the tile order: groups of 4 row tiles x all column tiles, so that 4 x 8
// neighbours run together.
__device__ __forceinline__ void row_tile_at(const RowShape& g, int t, int& tm, int& tn) {
  const int width = kGroupRows * g.tiles_n;
  const int first = t / width * kGroupRows, rem = t % width;
  const int gs = min(g.tiles_m - first, kGroupRows);
  tm = first + rem % gs;
  tn = rem / gs;
}
// Work-group -> index among the launch's tiles (-1: none): work-groups b, b + 8, ... share an
// XCD and its L2; each XCD takes a contiguous run of the order.
__device__ __forceinline__ int row_index(const RowShape& g, int bid) {
  const int per = (g.count + kNumXcd - 1) / kNumXcd;
  const int x = bid % kNumXcd, k = bid / kNumXcd, t = x * per + k;
  return k < per && t < g.count ? t : -1;
}

// One operand's side of the pipeline.  kOuter: K-outer layout.  kPair: K-inner
// rows of two matrices interleaved by blocks of 16 (even blocks p[0], odd p[1]).
template <int Blocks, bool kOuter, bool kPair>
struct RowSide {
  static constexpr int kTile = 32 * Blocks;          // entries of M (or N) per tile
  static constexpr int kBytes = kTile * kRowK * 2;   // per stage
  static constexpr int kLoads = kTile / 32;          // 1 KB loads per wave per stage
  static constexpr int kReads = kOuter ? 2 * Blocks : Blocks;   // per half stage
  static constexpr int kLanesPerK = kTile * 2 / 16, kKPerLoad = 64 / kLanesPerK;
  static constexpr int kPlaces = kTile / 16;         // 32-byte pieces of a K-outer row

  uint32_t voff[kLoads];
  uint32_t tail;        // K-inner: added in the last stage of a segment (out of range for the lanes past K)
  uint32_t rd[2];       // LDS byte offset of the lane's reads in half stage 0 / 1
  const unsigned char* base[2];
  uint32_t range;       // K-inner: bytes of the tile's rows
  int64_t rows_bytes;   // bytes between rows in memory
  int64_t seg_bytes;
  int64_t col;          // K-outer: bytes from a row's start to the tile

  static __device__ __forceinline__ int place(int k) { return ((k & 3) | ((k >> 3) & 3) << 2) & (kPlaces - 1); }

  __device__ __forceinline__ void init(const RowOperand& o, int tile, int K, int wave, int side, int lane) {
    rows_bytes = o.ld * 2;
    seg_bytes = o.seg_off * 2;
    if constexpr (kOuter) {
      col = (int64_t)tile * kTile * 2;
      base[0] = reinterpret_cast<const unsigned char*>(o.p[0]) + col;
      base[1] = reinterpret_cast<const unsigned char*>(o.p[1]) + col;
#pragma unroll
      for (int q = 0; q < kLoads; ++q) {
        const int k = (q * 4 + wave) * kKPerLoad + lane / kLanesPerK;
        voff[q] = (uint32_t)(k * rows_bytes) + (uint32_t)(((lane % kLanesPerK) ^ (2 * place(k))) << 4);
      }
      // lane's row of the 4 x 16 piece: k = 8 (lane / 16) + (lane % 16) / 4, 8 bytes (lane % 4)
      const int k = (lane >> 4) * 8 + ((lane & 15) >> 2);
      rd[0] = (uint32_t)(k * (kTile * 2) + (((side * Blocks) ^ place(k)) << 5) + (lane & 3) * 8);
      rd[1] = rd[0] + 32 * (kTile * 2);
    } else {
      constexpr int kRows = kPair ? kTile / 2 : kTile;   // rows of one matrix
      const int64_t row0 = (int64_t)tile * kRows;
      const int64_t have = min((int64_t)o.rows - row0, (int64_t)kRows);
      range = (uint32_t)(have * rows_bytes);
      base[0] = reinterpret_cast<const unsigned char*>(kPair && (wave >> 1) ? o.p[1] : o.p[0]) + row0 * rows_bytes;
      const int chunk = (lane & 7) ^ (lane >> 3);
#pragma unroll
      for (int q = 0; q < kLoads; ++q) {
        // LDS row (4 q + wave) 8 + lane / 8; of a pair, block 2 q + wave / 2 is rows 16 q .. of matrix wave / 2
        const int row = kPair ? q * 16 + (wave & 1) * 8 + (lane >> 3) : (q * 4 + wave) * 8 + (lane >> 3);
        voff[q] = (uint32_t)(row * rows_bytes) + (uint32_t)(chunk << 4);
      }
      const int last = (K + kRowK - 1) / kRowK - 1;
      tail = last * kRowK + chunk * 8 < K ? 0u : 0x80000000u;
      const int row = side * Blocks * 16 + (lane & 15);
      rd[0] = (uint32_t)(row * (kRowK * 2) + (((lane >> 4) ^ (row & 7)) << 4));
      rd[1] = rd[0] ^ 64u;
    }
  }

  // Descriptor, scalar offset and lane addend of the stage to load next.
  struct Stage {
    u32x4 rsrc;
    uint32_t soff, add;
    uint64_t at;      // K-outer: address of the stage's first row
  };
  __device__ __forceinline__ void describe(Stage& st, uint64_t at, uint32_t num) const {
    // raw buffer descriptor: 48-bit base, no stride, bytes in range, 32-bit data format
    st.rsrc = u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, num, 0x00020000u};
  }
  // `left`: K entries of the segment from the stage's first on; live false: an empty range,
  // so the loads read nothing and write zeros.
  __device__ __forceinline__ void set(Stage& st, int left, bool live) const {
    if constexpr (kOuter) {
      // rows of this stage; the last one ends with the matrix's row, not past it
      const uint32_t num = (uint32_t)min(left, kRowK) * (uint32_t)rows_bytes - (uint32_t)col;
      describe(st, st.at, live ? num : 0u);
      st.soff = st.add = 0;
    } else {
      describe(st, reinterpret_cast<uint64_t>(base[0]), live ? range : 0u);
      st.add = left < kRowK ? tail : 0u;
    }
  }
  __device__ __forceinline__ void first(Stage& st, int seg, int s, int left, bool live) const {
    if constexpr (kOuter) st.at = reinterpret_cast<uint64_t>((seg ? base[1] : base[0]) + (int64_t)s * kRowK * rows_bytes);
    else st.soff = live ? (uint32_t)(seg * seg_bytes) + (uint32_t)s * (kRowK * 2) : 0u;
    set(st, left, live);
  }
  // From one stage to the next; `over`: it is the second segment's first.
  __device__ __forceinline__ void next(Stage& st, bool over, int left, bool live) const {
    if constexpr (kOuter) {
      st.at += (uint64_t)(kRowK * rows_bytes);
      if (over) st.at = reinterpret_cast<uint64_t>(base[1]);
    } else {
      st.soff = over ? (uint32_t)seg_bytes : st.soff + kRowK * 2;
      st.soff = live ? st.soff : 0u;
    }
    set(st, left, live);
  }
  // Load Q of the stage, to its 1 KB of the LDS buffer at byte offset `lds`.  Written as
  // asm, which has no output register: beside the builtin the compiler waits for every
  // load in flight before each transpose read.  It knows nothing of these loads:
  // row_barrier waits for them, and settle() keeps the wait states that a vector write
  // of a scalar register needs before a load reads it.  The LDS place goes in as an operand
  // in m0, so that the compiler knows that it is written.
  template <int Q>
  __device__ __forceinline__ void load(const Stage& st, uint32_t lds, int wave) const {
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "{m0}"(lds + (Q * 4 + wave) * 1024), "v"(voff[Q] + st.add), "s"(st.rsrc), "s"(st.soff)
                 : "memory");
  }
  // Read R of half stage `Half` into f (K-outer: two reads make one block).
  template <int R, int Half>
  __device__ __forceinline__ void read(bf16x8* f, const unsigned char* lds) const {
    if constexpr (kOuter) {
      constexpr int i = R / 2;
      // the read goes out as the pair's first half, its second 4 rows of K further
      union {
        s16x4 h[2];
        bf16x8 v;
      } u;
      u.v = f[i];
      u.h[R & 1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_s16x4*)(lds + ((rd[Half] ^ (i << 5)) + (R & 1) * 4 * (kTile * 2))));
      f[i] = u.v;
    } else {
      f[R] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(lds + rd[Half] + R * 16 * (kRowK * 2)));
    }
  }
};

// Five wait states between whatever wrote the descriptors and the loads that read them.
template <class SA, class SB>
__device__ __forceinline__ void settle(SA& a, SB& b) {
  asm volatile("s_nop 4" : "+s"(a.rsrc), "+s"(a.soff), "+s"(b.rsrc), "+s"(b.soff));
}

// stage_barrier whose wait for the asm loads is asm too.
template <int Vm>
__device__ __forceinline__ void row_barrier() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(Vm) : "memory");
  stage_barrier<63>();
}

template <int BM, int BN, int kRing>
constexpr int kRowLds = kRing * (32 * BM + 32 * BN) * kRowK * 2;

// One tile of a product: work-group `bid` of the launch's tiles, K part `part`.
// Epilogue: epi.apply<BM, BN>(acc, tm, tn, wm, wn, lane, wave_lds, slab); a wave has its own part
// of the LDS; slab = part * (tiles of the launch) + tile.  Lane l's accumulator [i][j][r] is
// C(tm 32 BM + (wm BM + i) 16 + (l / 16) 4 + r, tn 32 BN + (wn BN + j) 16 + l % 16).
template <int BM, int BN, int kRing, bool kOuterA, bool kOuterB, bool kPairA, class Epi>
__device__ __forceinline__ void row_gemm_tile(const RowShape& g, const Epi& epi, int bid, int part,
                                              unsigned char* lds) {
  using A = RowSide<BM, kOuterA, kPairA>;
  using B = RowSide<BN, kOuterB, false>;
  constexpr int kStage = A::kBytes + B::kBytes;

  const int index = row_index(g, bid);
  if (index < 0) return;
  int tm, tn;
  row_tile_at(g, g.tile0 + index, tm, tn);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  A sa;
  B sb;
  sa.init(g.a, tm, g.K, wave, wm, lane);
  sb.init(g.b, tn, g.K, wave, wn, lane);

  const int per_seg = (g.K + kRowK - 1) / kRowK, nk_all = per_seg * g.segs;
  const int kb = (int)((int64_t)part * nk_all / g.parts), ke = (int)((int64_t)(part + 1) * nk_all / g.parts);

  f32x4 acc[BM][BN];
#pragma unroll
  for (int i = 0; i < BM; ++i)
#pragma unroll
    for (int j = 0; j < BN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  bf16x8 fa[2][BM] = {}, fb[2][BN] = {};   // operand registers of the two half stages

  // The loads run kRing stages ahead; past the end they are empty.
  typename A::Stage ga;
  typename B::Stage gb;
  int ahead = kb, left;
  {
    const int seg = kb >= per_seg ? 1 : 0;
    left = g.K - (kb - seg * per_seg) * kRowK;
    sa.first(ga, seg, kb - seg * per_seg, left, kb < ke);
    sb.first(gb, seg, kb - seg * per_seg, left, kb < ke);
  }
  bool over = false;
  auto step = [&] {   // the next stage's place; its two sides follow
    ++ahead;
    left -= kRowK;
    over = left <= 0;
    left = over ? g.K : left;
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void*)lds;
#pragma unroll
  for (int st = 0; st < kRing; ++st) {
    settle(ga, gb);
    repeat<A::kLoads>([&](auto q) { sa.template load<decltype(q)::value>(ga, lds0 + st * kStage, wave); });
    repeat<B::kLoads>([&](auto q) { sb.template load<decltype(q)::value>(gb, lds0 + st * kStage + A::kBytes, wave); });
    if (st + 1 < kRing) {
      step();
      sa.next(ga, over, left, ahead < ke);
      sb.next(gb, over, left, ahead < ke);
    }
  }
  row_barrier<(kRing - 1) * (A::kLoads + B::kLoads)>();
  repeat<A::kReads>([&](auto r) { sa.template read<decltype(r)::value, 0>(fa[0], lds); });
  repeat<B::kReads>([&](auto r) { sb.template read<decltype(r)::value, 0>(fb[0], lds + A::kBytes); });

  constexpr int kMfma = BM * BN, kReads = A::kReads + B::kReads, kLoads = A::kLoads + B::kLoads;
  constexpr int kEvery = kMfma / kLoads, kApart = kMfma / kReads;   // MFMAs per load, per read
  static_assert(kReads <= kMfma && kLoads <= kMfma, "one read and one load at most after each MFMA");
  uint32_t cur = 0;
  for (int t = kb; t < ke; ++t) {
    const uint32_t nxt = cur == (kRing - 1) * kStage ? 0u : cur + kStage;
    // first half: K 0 .. 31 of this stage; its other half is read
    repeat<kMfma>([&](auto ic) {
      constexpr int i = decltype(ic)::value, m = i / BN, n = i % BN;
      mfma_agpr(acc[m][n], fa[0][m], fb[0][n]);
      if constexpr (i % kApart == 0 && i / kApart < kReads) {
        constexpr int r = i / kApart;
        if constexpr (r < B::kReads) sb.template read<r, 1>(fb[1], lds + cur + A::kBytes);
        else sa.template read<r - B::kReads, 1>(fa[1], lds + cur);
      }
      // where the next stage to load lies
      if constexpr (i == kMfma - 6) step();
      if constexpr (i == kMfma - 5) sa.next(ga, over, left, ahead < ke);
      if constexpr (i == kMfma - 3) sb.next(gb, over, left, ahead < ke);
      __builtin_amdgcn_sched_barrier(0);
    });
    // every wave is done with this stage's buffer, and the next stage has landed
    row_barrier<(kRing - 2) * kLoads>();
    settle(ga, gb);
    repeat<kMfma>([&](auto ic) {
      constexpr int i = decltype(ic)::value, m = i / BN, n = i % BN;
      mfma_agpr(acc[m][n], fa[1][m], fb[1][n]);
      if constexpr (i % kApart == 0 && i / kApart < kReads) {
        constexpr int r = i / kApart;
        if constexpr (r < B::kReads) sb.template read<r, 0>(fb[0], lds + nxt + A::kBytes);
        else sa.template read<r - B::kReads, 0>(fa[0], lds + nxt);
      }
      if constexpr (i % kEvery == kEvery - 1 && i / kEvery < kLoads) {
        constexpr int q = i / kEvery;
        if constexpr (q < A::kLoads) sa.template load<q>(ga, lds0 + cur, wave);
        else sb.template load<q - A::kLoads>(gb, lds0 + cur + A::kBytes, wave);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    cur = nxt;
    // The accumulators are readable some passes after the last MFMA, which the compiler
    // does not know of: the wait stands inside the loop, before any copy that it makes of
    // them on the way out.
    if (t + 1 == ke) mfma_drain();
    __builtin_amdgcn_sched_barrier(0);
  }

  row_barrier<0>();   // the last (empty) loads have landed, every wave is done with the buffers
  epi.template apply<BM, BN>(acc, tm, tn, wm, wn, lane, lds + wave * (kRing * kStage / 4),
                              part * g.count + index);
}

// Work-groups of a CU (waves of a SIMD): what the LDS holds.
template <int BM, int BN, int kRing>
constexpr int kRowGroups = 163840 / kRowLds<BM, BN, kRing> < 3 ? 163840 / kRowLds<BM, BN, kRing> : 3;

template <int BM, int BN, int kRing, bool kOuterA, bool kOuterB, bool kPairA, class Epi>
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(kRowGroups<BM, BN, kRing>)))
void row_gemm_kernel(RowShape g, Epi epi) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kRowLds<BM, BN, kRing>];
  row_gemm_tile<BM, BN, kRing, kOuterA, kOuterB, kPairA>(g, epi, blockIdx.x, blockIdx.y, lds);
}

// Independent products in one launch, the first with A K-outer and B K-inner, the others with
// both K-outer: their work-groups fill the chip together, so that only the last tiles of all
// leave part of it idle.  A job's work-groups: its parts one after another, the tiles of a
// part rounded up to whole rounds of the XCDs.
template <class Epi>
struct RowJobs {
  static constexpr int kJobs = 3;
  RowShape g[kJobs];
  Epi epi[kJobs];
  int blocks[kJobs];
};
template <int BM, int BN, int kRing, class Epi>
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(kRowGroups<BM, BN, kRing>)))
void row_jobs_kernel(RowJobs<Epi> jobs) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kRowLds<BM, BN, kRing>];
  int bid = blockIdx.x;
  if (bid < jobs.blocks[0]) {
    const int per = (jobs.g[0].count + kNumXcd - 1) / kNumXcd * kNumXcd;
    row_gemm_tile<BM, BN, kRing, true, false, false>(jobs.g[0], jobs.epi[0], bid % per, bid / per, lds);
    return;
  }
  bid -= jobs.blocks[0];
  const int job = bid < jobs.blocks[1] ? 1 : 2;
  if (job == 2) bid -= jobs.blocks[1];
  const int per = (jobs.g[job].count + kNumXcd - 1) / kNumXcd * kNumXcd;
  row_gemm_tile<BM, BN, kRing, true, true, false>(jobs.g[job], jobs.epi[job], bid % per, bid / per, lds);
}

// One accumulator, read where it is needed: as a plain value the compiler copies the
// whole tile to vector registers at the loop's end, and spills.
__device__ __forceinline__ float acc_read(float a) {
  float x;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(a));
  return x;
}

// A wave's own LDS: what its lanes wrote before is seen by its lanes' reads after.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Hands a wave's accumulators to `op` eight entries of a column at a time, whole lines of a
// row of the output together: op.fetch(n, m) for kAhead pieces (what they need from memory),
// then op.piece(n, m, values, fetched) for each.  With kPair the row blocks come in pairs (even:
// first matrix, odd: second) and a piece is eight entries of both.  The accumulators go through
// the wave's LDS, up to 64 columns at once, 16-byte chunk c of column n at place c ^ (n & 15);
// the work on them is a loop over whole lines of the output (against straight-line code with
// three staged stores per block column: dh product of 8192 tokens 956 -> 918 us).
template <int BM, int BN, bool kPair, class Op>
__device__ __forceinline__ void row_pieces(const f32x4 (&acc)[BM][BN], int tm, int tn, int wm, int wn, int lane,
                                           unsigned char* lds, const Op& op) {
  constexpr int kM = BM * 16, kPasses = BN > 4 ? BN / 4 : 1, kB = BN / kPasses;   // column blocks per pass
  constexpr int kWidth = kPair ? kM / 2 : kM, kPer = kWidth / 8;                  // entries, pieces of a column
  constexpr int kSteps = kB * 16 * kPer / 64, kAhead = kSteps < 4 ? kSteps : 4;
  static_assert(kSteps % kAhead == 0 && 64 % kPer == 0, "whole steps");
  const int g = lane >> 4, c0 = lane & 15;
  repeat<kPasses>([&](auto pc) {   // constant indices into the accumulators, whatever the unroller decides
    constexpr int pass = decltype(pc)::value;
    wave_lds_fence();
    repeat<kB>([&](auto jc) {
      constexpr int j = decltype(jc)::value;
#pragma unroll
      for (int i = 0; i < BM; ++i) {
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = acc_read(acc[i][pass * kB + j][r]);
        *reinterpret_cast<f32x4*>(lds + (j * 16 + c0) * (kM * 4) + (((i * 4 + g) ^ c0) << 4)) = v;
      }
    });
    wave_lds_fence();
    const int64_t n0 = ((int64_t)(tn * 2 + wn) * BN + pass * kB) * 16;
    const int64_t m0 = (int64_t)(tm * 2 + wm) * kWidth + lane % kPer * 8;
    const int k = lane % kPer;
    // chunk of the piece's first four entries: of the row, or of the first of a pair of blocks
    const int at = kPair ? k / 2 * 8 + k % 2 * 2 : k * 2;
    auto four = [&](int col, int chunk) -> f32x4 {
      return *reinterpret_cast<const f32x4*>(lds + col * (kM * 4) + ((chunk ^ (col & 15)) << 4));
    };
#pragma unroll 1
    for (int s = 0; s < kSteps; s += kAhead) {
      typename Op::Fetched f[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) f[u] = op.fetch(n0 + (s + u) * (64 / kPer) + lane / kPer, m0);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int col = (s + u) * (64 / kPer) + lane / kPer;
        f32x4 v[kPair ? 4 : 2];
        v[0] = four(col, at);
        v[1] = four(col, at + 1);
        if constexpr (kPair) {
          v[2] = four(col, at + 4);
          v[3] = four(col, at + 5);
        }
        op.piece(n0 + col, m0, v, f[u]);
      }
    }
  });
}

}  // namespace pspo
