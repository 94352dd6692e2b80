// Log-probabilities of target tokens over a vocabulary, and their gradient, without the logits in memory.
//
// z = s X W^T; forward: a tile of logits leaves its maximum and its sum of exponentials for every row, which a second
// kernel joins into the LSE; the targets' own logits are dot products of that kernel.  Backward: the logits of a piece of the
// vocabulary are formed again, dz = s (scatter(dlogp) - G exp(z - LSE)) is written for the piece, and two products read it:
// dX += dz W and dW = dz^T X.
//
// fp32 operands are three bf16 planes each, x = x1 + x2 + x3 exactly; a product takes the six pairs of planes whose
// indices add up to at most 4, smallest first.  What is left out is below 2^-23 of a term, and 2^-25 of it on average.
#include <algorithm>
#include <type_traits>

#include "psattn_device.h"

namespace psattn {
namespace {

using namespace dev;

// The workgroups' shapes: WM x WN wavefronts, each with FM x FN tiles of 32 x 32; stages of BK elements of the summed dimension
// of each of P planes, RING of them in LDS.
//
// Large, 8192 x 128256 logits of 4096: 6.30 ms, 1366 TFLOP/s (a library product of this kind: 1480).  Two wavefronts per SIMD, so
// that one's products cover the other's waits.  Bound by power: the matrix cores are busy 71-77% of the cycles at 1.74-1.52 GHz
// (2.13 with nothing else to do); without the copies 80% at 1.81, with data that is always in L2 73% at 1.78.  Tried and
// slower: four wavefronts of 128 x 128 (7.07 ms, nothing covers a wait), stages of 32 in rings of 4 and 5 (6.8: twice the
// barriers), raised wave priorities (no change).
template <int WM_, int WN_, int FM_, int FN_, int BK_, int RING_, int P_>
struct Tiling {
  static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_, WAVES = WM * WN, THREADS = 64 * WAVES, M = 32 * WM * FM, N = 32 * WN * FN;
  static constexpr int BK = BK_, RING = RING_, P = P_, PLANE = (M + N) * BK * 2, STAGE = P * PLANE, LDS = RING * STAGE;
};
template <int P>
struct Tilings;
template <>
struct Tilings<1> {
  using Large = Tiling<2, 4, 4, 2, 64, 2, 1>;    // 256 x 256, one workgroup per CU
  using Small = Tiling<2, 2, 2, 2, 64, 2, 1>;    // 128 x 128, two
  using Deep = Tiling<2, 2, 2, 2, 64, 4, 1>;     // 128 x 128, one, three stages ahead
  using Thin = Tiling<4, 1, 1, 1, 64, 6, 1>;     // 128 x 32, one: 100 KB of copies on their way.  Bound by W's bytes: one row
                                                 // x 4096 x 128256 171 us, 6.1 TB/s (two stages, four workgroups: 178)
};
// All planes of a stage lie in LDS together, so that each is copied, and read into registers, once for its products with three,
// two or one of the other operand's: half the copies and reads of a pass per pair of planes (513 rows x 1024 x 16001: logits
// 150 us that way, 127 so; 1024 rows x 1024 x 16000 155 us, 1300 TFLOP/s of bf16 products).  One workgroup per CU.
template <>
struct Tilings<3> {
  using Large = Tiling<4, 2, 2, 2, 32, 2, 3>;    // 256 x 128
  using Small = Tiling<2, 2, 2, 2, 32, 2, 3>;    // 128 x 128
  using Deep = Small;
  using Thin = Tiling<4, 1, 1, 1, 64, 2, 3>;     // 128 x 32
};

// An operand of a product: element (i, k) of plane q at p + q plane + i ld + k, or + k ld + i where K is the outer dimension.
// Reads of i >= rows and k >= ks give some element of the operand in their place: such i are not stored, and at
// such k the other operand holds zeros.
struct Operand {
  const bf16_t* p;
  int64_t ld, plane;
  int rows, ks;
};

// a pointer that is the same in every lane, in scalar registers
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t u = (uint64_t)(uintptr_t)p;
  return (const char*)(uintptr_t)((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(u >> 32)) << 32 |
                                  (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)u));
}

// One operand's share of a stage, copied to LDS without registers.  A copy instruction moves 1 KB.
// K inner: rows of BK elements (BK / 8 chunks of 16 bytes), chunk c of row i at position c ^ swz(i): 16 rows read at one column
// hit distinct banks.  K outer: rows of I elements, chunk c of row k at position c ^ ((k & 3) << 2): the transposing reads
// take 4 rows x 4 chunks, distinct banks again.
template <int BK>
__device__ __forceinline__ int kswz(int i) { return BK == 64 ? (i >> 1) & 7 : (i >> 2) & 3; }
template <int I, int BK, int WAVES, bool KOUTER>
struct Loader {
  static constexpr int ALL = I * BK * 2 / 1024, COUNT = ALL < WAVES ? 1 : ALL / WAVES;   // instructions: of all wavefronts, of one
  static_assert(ALL * 1024 == I * BK * 2 && (ALL < WAVES ? WAVES % ALL : ALL % WAVES) == 0, "whole instructions");
  // the first one of a wavefront (where there are fewer than wavefronts, several copy the same)
  static __device__ __forceinline__ int first(int wave) { return wave * COUNT % ALL; }
  const bf16_t* p;       // element (i0, 0) of the first plane
  int64_t step;          // bytes from one stage to the next
  uint32_t off[COUNT];   // of each instruction's lane, from the stage's first element
  __device__ __forceinline__ Loader(const Operand& o, int64_t i0) : p(o.p + (KOUTER ? i0 : i0 * o.ld)), step(KOUTER ? BK * o.ld * 2 : BK * 2) {}
  // offsets for stages of which klim elements (1 .. BK) lie inside the operand
  __device__ __forceinline__ void aim(const Operand& o, int64_t i0, int klim, int wave, int lane) {
    const int ilim = (int)min((int64_t)I, o.rows - i0);
#pragma unroll
    for (int j = 0; j < COUNT; ++j) {
      const int u = first(wave) + j;
      if (KOUTER) {
        constexpr int per = I / 8;
        const int k = u * (64 / per) + lane / per;
        int c = (lane % per) ^ ((k & 3) << 2);
        if (8 * c >= ilim) c = 0;
        off[j] = (uint32_t)(min(k, klim - 1) * (int)o.ld * 2 + 16 * c);
      } else {
        constexpr int per = BK / 8;
        const int i = u * (64 / per) + lane / per;
        int c = (lane % per) ^ kswz<BK>(i);
        if (8 * c >= klim) c = 0;
        off[j] = (uint32_t)(min(i, ilim - 1) * (int)o.ld * 2 + 16 * c);
      }
    }
  }
  // instruction J of a stage: base its first element, lds the wavefront's part of the tile
  template <int J>
  __device__ __forceinline__ void issue(const char* base, uint32_t lds) const {
    copy16_to_lds_off(base, off[J], lds + J * 1024);
  }
};

// A wavefront's reads of an operand's tile: FRAGS tiles of 32 rows from row i on, elements 16 KK .. 16 KK + 15 of the stage.
template <int I, int BK, int FRAGS, bool KOUTER>
struct Reader {
  uint32_t at[KOUTER ? FRAGS : BK / 16];
  __device__ __forceinline__ Reader(int i, int lane) {
    if (KOUTER) {
      const int l = lane & 15, k = 8 * (lane >> 5) + (l >> 2);
#pragma unroll
      for (int f = 0; f < FRAGS; ++f) {
        const int c = (i + 32 * f) / 8 + 2 * ((lane >> 4) & 1) + ((l & 3) >> 1);
        at[f] = k * I * 2 + ((c ^ ((k & 3) << 2)) << 4) + (l & 1) * 8;
      }
    } else {
      const int r = i + (lane & 31);
#pragma unroll
      for (int kk = 0; kk < BK / 16; ++kk) at[kk] = r * BK * 2 + (((2 * kk + (lane >> 5)) ^ kswz<BK>(r)) << 4);
    }
  }
  template <int KK, int F>
  __device__ __forceinline__ bf16x8 read(const uint8_t* tile) const {
    if constexpr (KOUTER) {
      const uint8_t* p = tile + at[F] + KK * 16 * I * 2;
      return as_bf(lds_tr(p), lds_tr(p + 4 * I * 2));
    } else {
      return as_bf(ld16(tile + at[KK] + F * 32 * BK * 2));
    }
  }
};

// acc = A rows i0 .. i0 + M - 1 (down the tiles) x B rows j0 .. j0 + N - 1 (across) over ks elements (all there are, padded to
// a multiple of 64).  RING stages in LDS: while one is multiplied, the next RING - 1 are on their way.  The barrier
// between two stages stands before the last of a stage's products, whose operands are in registers by then, so
// that they cover the first reads of the next stage.
template <class S, bool KA, bool KB>
__device__ __forceinline__ void product(f32x16 (&acc)[S::FM][S::FN], const Operand& A, const Operand& B, int64_t i0, int64_t j0, int ks,
                                        uint8_t* lds) {
  constexpr int BK = S::BK, QS = BK / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int f = 0; f < S::FM; ++f)
#pragma unroll
    for (int g = 0; g < S::FN; ++g)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[f][g][e] = 0.f;
  constexpr int P = S::P;
  const int steps = max(0, ks + 63) / 64 * (64 / BK);
  if (steps == 0) return;
  using LA = Loader<S::M, BK, S::WAVES, KA>;
  using LB = Loader<S::N, BK, S::WAVES, KB>;
  LA la(A, i0);
  LB lb(B, j0);
  const Reader<S::M, BK, S::FM, KA> ra(wave / S::WN * S::FM * 32, lane);
  const Reader<S::N, BK, S::FN, KB> rb(wave % S::WN * S::FN * 32, lane);
  const uint32_t at = __builtin_amdgcn_readfirstlane(lds_addr(lds));
  const int whole = min(A.ks, B.ks) / BK;   // stages that lie wholly inside both operands
  la.aim(A, i0, BK, wave, lane);
  lb.aim(B, j0, BK, wave, lane);
  int kt = 0, fill = 0;
  const char *qa[P], *qb[P];   // the planes of the stage that is being copied, and where to
  uint32_t da, db;
  auto point = [&] {
    int ta = kt, tb = kt;
    if (kt >= whole) {   // (the last stages)
      int ka = A.ks - kt * BK, kb = B.ks - kt * BK;
      if (ka <= 0) ta = 0, ka = A.ks;   // wholly behind the operand's end: its first stage again
      if (kb <= 0) tb = 0, kb = B.ks;
      la.aim(A, i0, min(BK, ka), wave, lane);
      lb.aim(B, j0, min(BK, kb), wave, lane);
    }
#pragma unroll
    for (int q = 0; q < P; ++q) {
      qa[q] = uniform((const char*)(la.p + q * A.plane) + ta * la.step);
      qb[q] = uniform((const char*)(lb.p + q * B.plane) + tb * lb.step);
    }
    da = at + fill * S::STAGE + LA::first(wave) * 1024;
    db = at + fill * S::STAGE + S::M * BK * 2 + LB::first(wave) * 1024;
    if (++fill == S::RING) fill = 0;
    ++kt;
  };
  constexpr int COPIES = P * (LA::COUNT + LB::COUNT);
  auto copy = [&](auto j) {
    constexpr int Q = decltype(j)::value / (LA::COUNT + LB::COUNT), J = decltype(j)::value % (LA::COUNT + LB::COUNT);
    if constexpr (J < LA::COUNT) la.template issue<J>(qa[Q], da + Q * S::PLANE);
    else lb.template issue<J - LA::COUNT>(qb[Q], db + Q * S::PLANE);
  };
  auto issue = [&] {
    point();
    static_for<COPIES>(copy);
  };
  // waits until the next stage is in LDS (ahead: RING - 2 later ones have been issued)
  auto landed = [&](bool ahead) {
    if (ahead) wait_vmem<(S::RING - 2) * COPIES>();
    else wait_vmem<0>();
    barrier_only();
  };
  bf16x8 fa[2][P][S::FM], fb[2][P][S::FN];
  for (int s = 0; s < S::RING - 1 && s < steps; ++s) issue();
  landed(S::RING - 1 <= steps);
  if (S::RING - 1 < steps) issue();
  // fragment F of the operands' P (FM + FN), elements 16 KK .. of a stage: B's first, which every product takes, then A's in the
  // order in which they are taken
  constexpr int READS = P * (S::FM + S::FN);
  auto read = [&](auto kk, auto frag, const uint8_t* tile) {
    constexpr int KK = decltype(kk)::value, I = decltype(frag)::value;
    if constexpr (I < P * S::FN) {
      constexpr int Q = I / S::FN, F = I % S::FN;
      fb[KK & 1][Q][F] = rb.template read<KK, F>(tile + Q * S::PLANE + S::M * BK * 2);
    } else {
      constexpr int Q = P - 1 - (I - P * S::FN) / S::FM, F = (I - P * S::FN) % S::FM;
      fa[KK & 1][Q][F] = ra.template read<KK, F>(tile + Q * S::PLANE);
    }
  };
  static_for<READS>([&](auto f) { read(IntC<0>{}, f, lds); });
  int use = 0;
  // One stage: COPY: a later stage is copied meanwhile, into this one's place; NEXT: a stage follows.  Between two products of
  // a wavefront stands one read of the operands of the products behind this quarter, or a copy.
  auto stage = [&](auto copy_flag, auto next_flag) {
    constexpr bool COPY = decltype(copy_flag)::value, NEXT = decltype(next_flag)::value;
    constexpr int PRODUCTS = (P == 3 ? 6 : 1) * S::FM * S::FN;
    const uint8_t* tile = lds + use * S::STAGE;
    if (++use == S::RING) use = 0;
    const uint8_t* next = lds + use * S::STAGE;
    static_for<QS>([&](auto q) {
      constexpr int KK = decltype(q)::value;
      constexpr bool LAST = KK == QS - 1;
      constexpr int ACTIONS = (LAST && !NEXT ? 0 : READS) + (LAST && COPY ? COPIES : 0);
      constexpr int PER = (ACTIONS + PRODUCTS - 1) / PRODUCTS;
      if constexpr (LAST && NEXT) {
        wait_lds<0>();
        landed(COPY);
        if constexpr (COPY) point();
      }
      sched_fence();
      static_for<PRODUCTS>([&](auto m) {
        constexpr int I = decltype(m)::value, F = I / S::FN % S::FM, G = I % S::FN, PAIR = I / (S::FM * S::FN);
        // the planes of A and B: (2, 0) (1, 1) (0, 2) (1, 0) (0, 1) (0, 0)
        constexpr int QA = P == 1 ? 0 : PAIR == 0 ? 2 : PAIR == 1 || PAIR == 3 ? 1 : 0, QB = P == 1 ? 0 : PAIR == 2 ? 2 : PAIR == 1 || PAIR == 4 ? 1 : 0;
        acc[F][G] = mfma(fa[KK & 1][QA][F], fb[KK & 1][QB][G], acc[F][G]);
        sched_fence();
        static_for<PER>([&](auto j) {
          constexpr int A = I * PER + decltype(j)::value;
          if constexpr (A < ACTIONS) {
            if constexpr (A >= READS) copy(IntC<A - READS>{});
            else if constexpr (LAST) read(IntC<0>{}, IntC<A>{}, next);
            else read(IntC<(KK + 1) % QS>{}, IntC<A>{}, tile);
          }
        });
        sched_fence();
      });
    });
  };
  int s = 0;
  for (; s < steps - S::RING; ++s) stage(Flag<true>{}, Flag<true>{});
  // (the last RING stages: every one of them has been issued)
  for (; s < steps - 1; ++s) stage(Flag<false>{}, Flag<true>{});
  stage(Flag<false>{}, Flag<false>{});
  wait_lds<0>();
  barrier_only();   // (the LDS is the caller's again)
}
// The row down the 32 x 32 tile of element e of a lane is down(e) + 4 (lane >> 5).
__device__ __forceinline__ constexpr int down(int e) { return 8 * (e / 4) + e % 4; }
// The four dwords of bf16 that lanes l and l + 32 hold of tile rows 16 h .. 16 h + 15, as 8 consecutive rows each: lanes below
// 32 get rows 16 h .., the others 16 h + 8 ..
__device__ __forceinline__ u32x4 rows8(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
  const auto x = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);
  const auto y = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
  return u32x4{(uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1]};
}

// A workgroup's tile as bf16 to the rows out(0) .. out(lim_across - 1) [elements down], through LDS, so that whole rows of
// it leave together: eight(f, g, h) are the 8 elements that rows8 gives the lane for rows 16 h of tile (f, g).  lim_across
// and lim_down (a multiple of 8): what there is of the tile.
template <class S, class F, class O>
__device__ __forceinline__ void store_tile(F&& eight, O&& out, int64_t lim_across, int64_t lim_down, uint8_t* lds) {
  constexpr int CH = S::M / 8;   // chunks of 16 bytes in a row, at position c ^ (row mod CH): no two lanes of a write in one bank
  static_assert(S::M * S::N * 2 <= S::LDS, "the tile fits");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int g = 0; g < S::FN; ++g)
#pragma unroll
    for (int f = 0; f < S::FM; ++f)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int j = (wave % S::WN * S::FN + g) * 32 + (lane & 31), c = (wave / S::WN * S::FM + f) * 4 + 2 * h + (lane >> 5);
        *(u32x4*)(lds + j * S::M * 2 + ((c ^ (j % CH)) << 4)) = eight(f, g, h);
      }
  __syncthreads();
#pragma unroll 4
  for (int k = threadIdx.x; k < S::N * CH; k += S::THREADS) {
    const int j = k / CH, c = (k % CH) ^ (j % CH);
    if (j < lim_across && 8 * c < lim_down) *(u32x4*)(out(j) + 8 * c) = ld16(lds + k * 16);
  }
}

// Which part of the sum and which tile a workgroup takes.  Workgroups go to the 8 XCDs in turn; those of one XCD take
// consecutive ones, part by part, and in a part in bands of 4 tiles down by all tiles across, so that the 32 that run on
// it at a time share rows of both operands in its L2.  (dX of 513 fp32 rows x 1024 x 16001, 12 parts of 40 tiles: 172 us
// with each part's tiles spread over the XCDs, 121 so.)
struct Tile { int part, down, across; };
__device__ __forceinline__ Tile tile_of(unsigned block, unsigned blocks, int downs, int acrosses) {
  const int each = blocks / 8, rest = blocks % 8, x = block % 8;
  const int all = x * each + min(x, rest) + block / 8, tiles = downs * acrosses;
  const int part = all / tiles, t = all - part * tiles;
  const int first = t / (4 * acrosses) * 4, high = min(4, downs - first), in = t - first * acrosses;
  // (divisions leave uniform values in vector registers)
  return {__builtin_amdgcn_readfirstlane(part), __builtin_amdgcn_readfirstlane(first + in % high), __builtin_amdgcn_readfirstlane(in / high)};
}

__device__ __forceinline__ int up64(int n) { return (n + 63) / 64 * 64; }
// X's rows: in the backward the live ones, np of them with the empty ones behind
__device__ __forceinline__ Operand x_operand(const LogprobArgs& a, int np) {
  if (a.xc) return {a.xc, a.hp, (int64_t)a.np * a.hp, np, a.hp};
  return {(const bf16_t*)a.X, a.h, 0, a.n, a.h};
}
__device__ __forceinline__ Operand w_operand(const LogprobArgs& a, int piece) {
  const int v0 = piece * a.piece_v, rows = min(a.piece_v, a.v - v0);
  if (a.wc) return {a.wc, a.hp, (int64_t)a.piece_v * a.hp, rows, a.hp};
  return {(const bf16_t*)a.W + (int64_t)v0 * a.h, a.h, 0, rows, a.h};
}
// elements k0 .. k0 + k - 1 of the summed dimension alone
__device__ __forceinline__ Operand part_of(Operand o, bool kouter, int64_t k0, int k) {
  o.p += kouter ? k0 * o.ld : k0;
  o.ks = (int)min((int64_t)k, o.ks - k0);
  return o;
}
__device__ __forceinline__ Operand swapped(const Operand& o) { return {o.p, o.ld, o.plane, o.ks, o.rows}; }

// the statistics of two sets of logits together
__device__ __forceinline__ LogprobStat join(const LogprobStat& p, const LogprobStat& q) {
  const float top = fmaxf(p.top, q.top), ref = top == kNegInf ? 0.f : top;
  // (fmaxf leaves a NaN out: it comes through the sums)
  return {top, p.sum * fast_exp2(p.top - ref) + q.sum * fast_exp2(q.top - ref)};
}

// bounds of a row's targets, whatever tgt_ptr holds
__device__ __forceinline__ void targets_of(const LogprobArgs& a, int r, int& e0, int& e1) {
  e0 = min(max(a.tgt_ptr[r], 0), a.e);
  e1 = min(max(a.tgt_ptr[r + 1], e0), a.e);
}

// ---- rows as the products take them.  Bound by the rows' bytes, a workgroup per row.
// row r of X, or zeros, to row i of xc
template <bool FP32>
__device__ __forceinline__ void copy_row(const LogprobArgs& a, int r, bool in_row, int64_t i) {
  for (int c = 8 * threadIdx.x; c < a.hp; c += 8 * 256) {
    const bool in = in_row && c < a.h;
    if (!FP32) {
      u32x4 x = {0, 0, 0, 0};
      if (in) x = ld16((const bf16_t*)a.X + (int64_t)r * a.h + c);
      *(u32x4*)(a.xc + i * a.hp + c) = x;
    } else {
      for (int k = 0; k < 8; k += 4) {
        f32x4 x = {0, 0, 0, 0};
        if (in) x = *(const f32x4*)((const float*)a.X + (int64_t)r * a.h + c + k);
        put_planes(x, a.xc, (int64_t)a.np * a.hp, i * a.hp + c + k);
      }
    }
  }
}
template <bool FP32>
__global__ __launch_bounds__(256) void prep_kernel(LogprobArgs a) {
  copy_row<FP32>(a, blockIdx.x, (int)blockIdx.x < a.n, blockIdx.x);
}

// The backward multiplies only rows that have a gradient: the others' part of either result is zero, whatever they hold.  They are
// packed in their order, so that sums keep theirs: each 256 rows count their own (rows_kernel), the counts are added up
// (before_kernel), and each row finds its place (gather_kernel).  Up to 256 rows every workgroup counts for itself.  A
// third of 2047 rows masked, in all two fifths without gradient: 2047 x 1544 x 50257 forward and backward 1.42 ms with all rows
// multiplied, 1.11 so.
__device__ __forceinline__ LogprobRow row_of(const LogprobArgs& a, int r, bool& live) {
  LogprobRow row = {0.f, 0.f, 0.f, -1, 0, 0, r, -1};
  live = false;
  if (r >= a.n) return row;
  targets_of(a, r, row.e0, row.e1);
  for (int e = row.e0; e < row.e1; ++e) {
    const int t = a.tgt[e];
    const float g = a.dlogp[e];
    if (t < 0 || t >= a.v) continue;
    row.total += g;
    live = live || g != 0.f;
    if (e == row.e0) row.t0 = t, row.g0 = g;
  }
  row.lse2 = a.lse[r] * kLog2e;
  return row;
}
// the place of each thread's row among the live ones of the workgroup's 256, and their number
__device__ __forceinline__ int rank_of(bool live, int& count) {
  __shared__ int s_count[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t mask = __ballot(live);
  if (lane == 0) s_count[wave] = __builtin_popcountll(mask);
  __syncthreads();
  int at = __builtin_popcountll(mask & ((1ull << lane) - 1));
  count = 0;
  for (int w = 0; w < 4; ++w) {
    if (w < wave) at += s_count[w];
    count += s_count[w];
  }
  return live ? at : -1;
}
__global__ __launch_bounds__(256) void rows_kernel(LogprobArgs a) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  bool live;
  LogprobRow row = row_of(a, r, live);
  int count;
  row.at = rank_of(live, count);
  if (r < a.n) a.info[r] = row;
  if (threadIdx.x == 0) a.before[blockIdx.x] = count;
}
__global__ __launch_bounds__(1024) void before_kernel(LogprobArgs a) {
  __shared__ int s_sum[1024];
  const int groups = (a.n + 255) / 256, each = (groups + 1023) / 1024, first = threadIdx.x * each, end = min(groups, first + each);
  int sum = 0;
  for (int k = first; k < end; ++k) sum += a.before[k];
  s_sum[threadIdx.x] = sum;
  for (int d = 1; d < 1024; d *= 2) {
    __syncthreads();
    const int x = (int)threadIdx.x >= d ? s_sum[threadIdx.x - d] : 0;
    __syncthreads();
    s_sum[threadIdx.x] += x;
  }
  int at = s_sum[threadIdx.x] - sum;
  for (int k = first; k < end; ++k) {
    const int n = a.before[k];
    a.before[k] = at;
    at += n;
  }
  if (threadIdx.x == 1023) *a.live = at;
}
// Workgroup r < n: row r; behind them those that fill the last 64 live rows up with empty ones.
template <bool FP32, bool ALONE>
__global__ __launch_bounds__(256) void gather_kernel(LogprobArgs a) {
  __shared__ LogprobRow s_me;
  const int r = blockIdx.x;
  int count, before = 0;
  if (ALONE) {
    bool live;
    LogprobRow row = row_of(a, threadIdx.x, live);
    row.at = rank_of(live, count);
    if ((int)threadIdx.x == r) s_me = row;
    if (r == 0 && threadIdx.x == 0) *a.live = count;
  } else {
    count = *a.live;
    if (r < a.n) before = a.before[r / 256];
    if (r < a.n && threadIdx.x == 0) s_me = a.info[r];
  }
  __syncthreads();
  if (r >= a.n) {
    const int i = count + r - a.n;
    if (i >= up64(count)) return;
    if (threadIdx.x == 0) a.row[i] = {0.f, 0.f, 0.f, -1, 0, 0, -1, -1};
    copy_row<FP32>(a, 0, false, i);
    return;
  }
  const LogprobRow me = s_me;
  const int i = me.at < 0 ? -1 : before + me.at;
  if (!FP32)
    for (int e = me.e0 + threadIdx.x; e < me.e1; e += 256) {
      a.ent_row[e] = i;
      a.ent_rem[e] = 0.f;
    }
  if (i >= 0) {
    if (threadIdx.x == 0) a.row[i] = me;
    copy_row<FP32>(a, r, true, i);
  } else if (a.dX) {
    const int64_t bytes = (int64_t)a.h * (FP32 ? 4 : 2);
    for (int64_t x = 16 * threadIdx.x; x < bytes; x += 16 * 256) *(u32x4*)((uint8_t*)a.dX + r * bytes + x) = u32x4{0, 0, 0, 0};
  }
}

__global__ __launch_bounds__(256) void wplanes_kernel(LogprobArgs a, int piece) {
  const int v = piece * a.piece_v + blockIdx.x;
  for (int c = 4 * threadIdx.x; c < a.hp; c += 4 * 256) {
    f32x4 x = {0, 0, 0, 0};
    if (v < a.v && c < a.h) x = *(const f32x4*)((const float*)a.W + (int64_t)v * a.h + c);
    put_planes(x, a.wc, (int64_t)a.piece_v * a.hp, (int64_t)blockIdx.x * a.hp + c);
  }
}

// ---- a tile of logits: M entries of the piece down, N rows across, so that a lane holds 16 FM entries of each of its FN rows.
// Forward: the maximum and the sum of exponentials of the tile's entries leave for each row, one fma, one exponential, one
// addition and half a maximum per logit; nothing else is written.  Backward: dz of the tile, scaled, as bf16 or as
// planes: 6.84 ms for 8192 x 128256 x 4096 (every row live) against the forward's 6.30, for the same product and 2 GB written.
template <class S, bool BACKWARD>
__device__ __forceinline__ void logits_tile(const LogprobArgs& a, int piece, int np, int down_tile, int64_t j0, uint8_t* lds, LogprobRow* s_row) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t i0 = (int64_t)down_tile * S::M;
  const int iw = (int)i0 + wave / S::WN * S::FM * 32, jw = wave % S::WN * S::FN * 32;   // the wavefront's first entry and row of the tile
  f32x16 acc[S::FM][S::FN];
  const Operand W = w_operand(a, piece);
  if constexpr (BACKWARD)   // (here so that its reads' time passes under the products)
    for (int j = threadIdx.x; j < S::N; j += S::THREADS)
      if (j0 + j < np) s_row[j] = a.row[j0 + j];
  product<S, false, false>(acc, W, x_operand(a, np), i0, j0, a.hp, lds);
  const float c = a.scale * kLog2e;
  const int left = W.rows - iw - 4 * (lane >> 5);   // element (f, e) is an entry where 32 f + down(e) is below
  if constexpr (!BACKWARD) {
    LogprobStat* part = (LogprobStat*)lds;                 // [WM][N]
    if (left < 32 * S::FM) {
#pragma unroll
      for (int g = 0; g < S::FN; ++g)
#pragma unroll
        for (int f = 0; f < S::FM; ++f)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[f][g][e] = 32 * f + down(e) < left ? acc[f][g][e] : kNegInf;
    }
#pragma unroll
    for (int g = 0; g < S::FN; ++g) {
      float top = kNegInf, sum = 0.f;
#pragma unroll
      for (int f = 0; f < S::FM; ++f)
#pragma unroll
        for (int e = 0; e < 16; e += 2) top = max3f(top, acc[f][g][e], acc[f][g][e + 1]);
      top = pair_max(top) * c;                             // (c > 0)
      const float ref = top == kNegInf ? 0.f : top;
#pragma unroll
      for (int f = 0; f < S::FM; ++f)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += fast_exp2(fmaf(acc[f][g][e], c, -ref));
      sum = pair_sum(sum);
      if (lane < 32) part[wave / S::WN * S::N + jw + 32 * g + lane] = {top, sum};
    }
    __syncthreads();
    for (int j = threadIdx.x; j < S::N; j += S::THREADS) {
      constexpr int PART = S::P == 3 ? 128 : S::M, WAVES = S::WM * PART / S::M;   // entries of a part, wavefronts down it
#pragma unroll
      for (int k = 0; k < S::M / PART; ++k) {
        LogprobStat p = part[k * WAVES * S::N + j];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) p = join(p, part[(k * WAVES + w) * S::N + j]);
        if (j0 + j < a.n && i0 + k * PART < W.rows) a.part[((piece * (int64_t)a.piece_v + i0) / PART + k) * a.n + j0 + j] = p;
      }
    }
    return;
  } else {
    const int v0 = piece * a.piece_v;
#pragma unroll
    for (int g = 0; g < S::FN; ++g) {
      sched_fence();
      LogprobRow row = {0.f, 0.f, 0.f, -1, 0, 0, -1, -1};
      if (j0 + jw + 32 * g < np) row = s_row[jw + 32 * g + (lane & 31)];
      // (a row whose G is 0 takes 2^-inf: nothing, whatever its LSE)
      const float k = -row.total * a.scale, ref = k == 0.f ? -kNegInf : row.lse2;
#pragma unroll
      for (int f = 0; f < S::FM; ++f)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[f][g][e] = k * fast_exp2(fmaf(acc[f][g][e], c, -ref));
      // The targets among the wavefront's entries: few, so each is looked for in the registers.  place: where target e is.
      auto place = [&](int e) {
        const int t = e == row.e0 ? row.t0 : e < row.e1 ? a.tgt[e] : -1;
        return t < 0 || t >= a.v ? -64 : t - v0 - iw - 4 * (lane >> 5);
      };
      auto here = [&](int at) { return at >= -4 && at < 32 * S::FM; };
      for (int t = row.e0; __any(t < row.e1); ++t) {
        const int at = place(t);
        if (!__any(here(at))) continue;
        const float d = a.scale * (t == row.e0 ? row.g0 : t < row.e1 ? a.dlogp[t] : 0.f);
#pragma unroll
        for (int f = 0; f < S::FM; ++f)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (at == 32 * f + down(e)) acc[f][g][e] += d;
      }
      if (left < 32 * S::FM) {
#pragma unroll
        for (int f = 0; f < S::FM; ++f)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[f][g][e] = 32 * f + down(e) < left ? acc[f][g][e] : 0.f;
      }
      if (S::P == 1) {
        // A target's dz is most of its row's, so its rounding would be most of the gradients' error: what it leaves out
        // goes into them by itself.
        for (int t = row.e0; __any(t < row.e1); ++t) {
          int at = place(t);
          if (!__any(here(at))) continue;
          if (here(at))
            for (int u = row.e0; u < t; ++u)
              if (place(u) == at) at = -64;
          float x = 0.f;
          bool mine = false;
#pragma unroll
          for (int f = 0; f < S::FM; ++f)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (at == 32 * f + down(e)) x = acc[f][g][e], mine = true;
          if (mine) a.ent_rem[t] = is_finite(x) ? x - bf2f(pack2(x, 0.f) & 0xffffu) : 0.f;
        }
      }
    }
    bf16_t* out = a.dl + j0 * a.piece_v + i0;
    const int64_t lim_across = np - j0, lim_down = a.piece_v - i0;
    if constexpr (S::P == 1) {
      store_tile<S>(
          [&](int f, int g, int h) {
            const f32x16& x = acc[f][g];
            return rows8(pack2(x[8 * h], x[8 * h + 1]), pack2(x[8 * h + 2], x[8 * h + 3]), pack2(x[8 * h + 4], x[8 * h + 5]),
                         pack2(x[8 * h + 6], x[8 * h + 7]));
          },
          [&](int j) { return out + (int64_t)j * a.piece_v; }, lim_across, lim_down, lds);
    } else {
      static_for<3>([&](auto q) {
        constexpr int Q = decltype(q)::value;
        if (Q) __syncthreads();
        store_tile<S>(
            [&](int f, int g, int h) {
              uint32_t w[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                uint32_t lo[3], hi[3];
                split3(acc[f][g][8 * h + 2 * k], lo[0], lo[1], lo[2]);
                split3(acc[f][g][8 * h + 2 * k + 1], hi[0], hi[1], hi[2]);
                w[k] = lo[Q] | hi[Q] << 16;
              }
              return rows8(w[0], w[1], w[2], w[3]);
            },
            [&](int j) { return out + ((int64_t)Q * a.np + j) * a.piece_v; }, lim_across, lim_down, lds);
      });
    }
  }
}

// Up to 64 rows behind the whole tiles of the largest kind have narrow ones, which start last and fill the compute units that
// the whole ones leave idle: logits of 777 rows x 1000 x 50257 126 us with whole tiles for the last 9 rows, 102 so; 320 rows 52
// and 44; 513 fp32 rows x 1024 x 16001 134 and 104; 64 rows x 4096 x 128256, bound by W's bytes, 227 and 222 (298 with each XCD's
// tiles spread over all of W).  The same for dX: both gradients of 2080 rows x 1544 x 50257 696 us, 654 so.  Smaller tiles gain
// nothing (logits of 129 rows x 1024 x 32000 20 us, 23 so).  fp32 logits: half as many entries, twice as long stages, so that
// whole 128 bytes of a row are copied at a time (513 rows: 118 us otherwise).
template <class S, int M, int BK>
using Narrow = Tiling<S::WAVES / 2, 2, M / (16 * S::WAVES), 1, BK, S::LDS / ((M + 64) * BK * 2 * S::P), S::P>;
template <class S>
using LogitsTail = Narrow<S, S::P == 3 ? 128 : S::M, 64>;
template <class S>
using GradsTail = Narrow<S, S::M, S::BK>;
template <class S>
inline constexpr bool HasTail = S::WAVES == 8;
// whole tiles of a row of them: the narrow one takes what is left
template <class S>
__device__ __forceinline__ int whole_tiles(int rows) {
  const int n = (rows + S::N - 1) / S::N;
  return HasTail<S> && n && rows - (n - 1) * S::N <= 64 ? n - 1 : n;
}
template <class S, bool BACKWARD>
__global__ __launch_bounds__(S::THREADS) void logits_kernel(LogprobArgs a, int piece, int downs, int tails) {
  constexpr bool TAIL = HasTail<S>;
  using T = std::conditional_t<TAIL, LogitsTail<S>, S>;
  static_assert(T::THREADS == S::THREADS && T::LDS <= S::LDS, "in its place");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[S::LDS];
  __shared__ LogprobRow s_row[BACKWARD ? S::N : 1];
  const int np = BACKWARD ? up64(*a.live) : a.n;   // (fewer rows are live than the launch has room for)
  const int whole = whole_tiles<S>(np), block = blockIdx.x, blocks = downs * whole;
  if (block < blocks) {
    const Tile tile = tile_of(block, blocks, downs, whole);
    logits_tile<S, BACKWARD>(a, piece, np, tile.down, (int64_t)tile.across * S::N, lds, s_row);
  } else if (TAIL && block < blocks + tails && whole * S::N < np) {
    logits_tile<T, BACKWARD>(a, piece, np, tile_of(block - blocks, tails, tails, 1).down, (int64_t)whole * S::N, lds, s_row);
  }
}

// ---- LSE and logp from the tiles' parts: 16 rows per workgroup, 64 threads for each row's parts (so that 128 bytes of them
// are read together), then a wavefront per row for its targets' dot products, in fp32 from X and W themselves.  Bound by the
// latency of four dependent reads where there are few rows (one row: 6 us), else by the rows' bytes (20480 x 4096: 82 us, 4.3 TB/s).
template <bool FP32>
__global__ __launch_bounds__(1024) void finish_kernel(LogprobArgs a) {
  __shared__ LogprobStat s_part[16][65];
  const int r0 = blockIdx.x * 16, lane = threadIdx.x & 63, i = threadIdx.x >> 6, r = r0 + i;
  {
    const int j = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int parts = (a.v + a.part_v - 1) / a.part_v;
    LogprobStat p = {kNegInf, 0.f};
    if (r0 + j < a.n) {
#pragma unroll 4
      for (int t = slice; t < parts; t += 64) p = join(p, a.part[(int64_t)t * a.n + r0 + j]);
    }
    s_part[j][slice] = p;
  }
  __syncthreads();
  if (r < a.n) {
    LogprobStat p = s_part[i][lane];
#pragma unroll
    for (int w = 32; w >= 1; w >>= 1) p = join(p, {__shfl_xor(p.top, w), __shfl_xor(p.sum, w)});
    const float lse = ((p.top == kNegInf ? 0.f : p.top) + log2f(p.sum)) * (1.f / kLog2e);
    if (lane == 0) a.lse_out[r] = lse;
    int e0, e1;
    targets_of(a, r, e0, e1);
    for (int e = e0; e < e1; ++e) {
      const int t = a.tgt[e];
      float z = 0.f;
      if (t >= 0 && t < a.v) {
        constexpr int V = FP32 ? 4 : 8;   // elements in 16 bytes
        const uint8_t* x = (const uint8_t*)elem_ptr<!FP32>(a.X, (size_t)r * a.h);
        const uint8_t* w = (const uint8_t*)elem_ptr<!FP32>(a.W, (size_t)t * a.h);
#pragma unroll 4
        for (int c = lane * V; c < a.h; c += 64 * V) {
          const u32x4 p = ld16(x + c * (16 / V)), q = ld16(w + c * (16 / V));
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (FP32) {
              z = fmaf(__uint_as_float(p[k]), __uint_as_float(q[k]), z);
            } else {
              z = fmaf(bf2f(p[k] & 0xffffu), bf2f(q[k] & 0xffffu), z);
              z = fmaf(__uint_as_float(p[k] & 0xffff0000u), __uint_as_float(q[k] & 0xffff0000u), z);
            }
          }
        }
#pragma unroll
        for (int w2 = 32; w2 >= 1; w2 >>= 1) z += __shfl_xor(z, w2);
        z = z * a.scale - lse;
      }
      if (lane == 0) a.logp[e] = z;
    }
  }
}

// 32 rows of the tile, 4 consecutive ones at a time, as fp32 to p + i .. (those below limit)
__device__ __forceinline__ void put_rows(float* p, int i, int limit, const f32x16& x, int lane) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int at = i + 8 * q + 4 * (lane >> 5);
    if (at < limit) *(f32x4*)(p + at) = f32x4{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
  }
}
// One of the terms rem(k) row(k) (down) at column col(k) (across) that are added to a tile; no row: nothing.
struct Term { const bf16_t* row; int32_t col; float rem; };
// acc += the terms, as products like any other: 64 at a time are a stage whose B is rem (as bf16, which leaves 2^-9 of what is
// itself below 2^-9 of the term it belongs to) at the term's column and zero elsewhere.  Elements i0 .. of the rows
// (below limit) go down the tile.
template <class S, class F>
__device__ __forceinline__ void add_terms(f32x16 (&acc)[S::FM][S::FN], int count, F&& term, int64_t i0, int limit, uint8_t* lds) {
  constexpr int CM = S::M / 8, CN = S::N / 8;
  static_assert((S::M + S::N) * 128 <= S::LDS, "a stage of 64 fits");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint8_t* b = lds + S::M * 128;
  const Reader<S::M, 64, S::FM, true> ra(wave / S::WN * S::FM * 32, lane);
  const Reader<S::N, 64, S::FN, true> rb(wave % S::WN * S::FN * 32, lane);
#pragma unroll 1
  for (int first = 0; first < count; first += 64) {
    __syncthreads();
#pragma unroll 2
    for (int x = threadIdx.x; x < 64 * CM; x += S::THREADS) {
      const int k = x / CM, c = (x % CM) ^ ((k & 3) << 2);
      const bf16_t* row = first + k < count ? term(first + k).row : nullptr;
      u32x4 y = {0, 0, 0, 0};
      if (row && i0 + 8 * c < limit) y = ld16(row + i0 + 8 * c);
      *(u32x4*)(lds + x * 16) = y;
    }
    for (int x = threadIdx.x; x < 64 * CN; x += S::THREADS) *(u32x4*)(b + x * 16) = u32x4{0, 0, 0, 0};
    __syncthreads();
    if (threadIdx.x < 64 && first + (int)threadIdx.x < count) {
      const int k = threadIdx.x;
      const Term t = term(first + k);
      if (t.row) *(bf16_t*)(b + k * S::N * 2 + (((t.col >> 3) ^ ((k & 3) << 2)) << 4) + (t.col & 7) * 2) = (bf16_t)pack2(t.rem, 0.f);
    }
    __syncthreads();
    static_for<4>([&](auto q) {
      constexpr int KK = decltype(q)::value;
      bf16x8 fa[S::FM], fb[S::FN];
      static_for<S::FM>([&](auto f) { fa[decltype(f)::value] = ra.template read<KK, decltype(f)::value>(lds); });
      static_for<S::FN>([&](auto f) { fb[decltype(f)::value] = rb.template read<KK, decltype(f)::value>(b); });
#pragma unroll
      for (int f = 0; f < S::FM; ++f)
#pragma unroll
        for (int g = 0; g < S::FN; ++g) acc[f][g] = mfma(fa[f], fb[g], acc[f][g]);
    });
  }
  __syncthreads();
}
// Target e as a term of live row i: what the rounding of its dz left out, 0 if that row does not list it.
__device__ __forceinline__ float rem_of(const LogprobArgs& a, int e, int i, int live) {
  if (i < 0 || i >= live) return 0.f;
  return e >= a.row[i].e0 && e < a.row[i].e1 ? a.ent_rem[e] : 0.f;
}
// the workgroup's tile to a result of the inputs' type, rows row(0) .. row(lim_across - 1) of h elements, elements i0 .. of them
template <class S, class R>
__device__ __forceinline__ void put_tile(const f32x16 (&acc)[S::FM][S::FN], void* out, R&& row, int h, int64_t i0, int64_t lim_across, uint8_t* lds) {
  if constexpr (S::P == 1) {
    store_tile<S>(
        [&](int f, int g, int k) {
          const f32x16& x = acc[f][g];
          return rows8(pack2(x[8 * k], x[8 * k + 1]), pack2(x[8 * k + 2], x[8 * k + 3]), pack2(x[8 * k + 4], x[8 * k + 5]),
                       pack2(x[8 * k + 6], x[8 * k + 7]));
        },
        [&](int j) { return (bf16_t*)out + (int64_t)row(j) * h + i0; }, lim_across, h - i0, lds);
  } else {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int g = 0; g < S::FN; ++g) {
      const int j = (wave % S::WN * S::FN + g) * 32 + (lane & 31);
      if (j >= lim_across) continue;
      float* p = (float*)out + (int64_t)row(j) * h;
#pragma unroll
      for (int f = 0; f < S::FM; ++f) put_rows(p, (int)i0 + (wave / S::WN * S::FM + f) * 32, h, acc[f][g], lane);
    }
  }
}

// dX: M of the hidden dimension down, N rows across, summed over the piece's entries or a part of them; W is read across its rows by
// the transposing loads.  Pieces add to fp32 sums in memory, the last one leaves the result.  8192 x 4096 x 128256 by itself, every
// row live: 6.57 ms in four pieces, 1310 TFLOP/s.
template <class S>
__device__ __forceinline__ void dx_tile(const LogprobArgs& a, int piece, const Tile& tile, uint8_t* lds) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = tile.part, k = a.stages_dx * 64;
  const int64_t i0 = (int64_t)tile.down * S::M, j0 = (int64_t)tile.across * S::N;
  const int iw = (int)i0 + wave / S::WN * S::FM * 32, jw = wave % S::WN * S::FN * 32;
  const int live = *a.live, np = up64(live);
  f32x16 acc[S::FM][S::FN];
  const bool last = piece == a.pieces - 1, rest = S::P == 1 && last && split == 0;   // rest: what the targets' dz left out is added
  // (the tile's rows have their targets one behind the other, with those of rows that are not live between them: LIST at a time, the first ones ahead of the products)
  constexpr int LIST = S::P == 1 ? 2 * S::N : 1;
  __shared__ struct { float rem; int32_t tgt, col; } s_list[LIST];
  int e_lo = 0, e_hi = 0;
  auto list = [&] {
    for (int k = threadIdx.x; k < LIST && e_lo + k < e_hi; k += S::THREADS) {
      const int e = e_lo + k, r = a.ent_row[e], t = a.tgt[e];
      const bool in = r >= j0 && r < j0 + S::N && t >= 0 && t < a.v;
      s_list[k] = {in ? rem_of(a, e, r, live) : 0.f, t, (int)(r - j0)};
    }
  };
  if (rest) {
    e_lo = a.row[j0].e0, e_hi = max(e_lo, a.row[min(j0 + S::N, (int64_t)live) - 1].e1);
    list();
  }
  const Operand W = part_of(swapped(w_operand(a, piece)), true, (int64_t)split * k, k);
  const Operand D = part_of({a.dl, a.piece_v, (int64_t)a.np * a.piece_v, np, a.piece_v}, false, (int64_t)split * k, k);
  product<S, true, false>(acc, W, D, i0, j0, W.ks, lds);
  float* sums = a.dx_acc + (int64_t)split * a.n * a.h;
#pragma unroll
  for (int g = 0; g < S::FN; ++g) {
    const int64_t r = j0 + jw + 32 * g + (lane & 31);
    const int limit = r < live ? a.h : 0;
    if (piece) {
#pragma unroll
      for (int f = 0; f < S::FM; ++f)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int at = iw + 32 * f + 8 * q + 4 * (lane >> 5);
          if (at >= limit) continue;
          const f32x4 y = *(const f32x4*)(sums + r * a.h + at);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[f][g][4 * q + e] += y[e];
        }
    }
  }
  if (rest) {
    while (e_lo < e_hi) {
      add_terms<S>(
          acc, min(LIST, e_hi - e_lo),
          [&](int k) { return Term{s_list[k].rem != 0.f ? (const bf16_t*)a.W + (int64_t)s_list[k].tgt * a.h : nullptr, s_list[k].col, s_list[k].rem}; }, i0, a.h, lds);
      e_lo += LIST;
      list();
    }
  }
  if (!last || a.splits_dx > 1) {
#pragma unroll
    for (int g = 0; g < S::FN; ++g) {
      const int64_t r = j0 + jw + 32 * g + (lane & 31);
      const int limit = r < live ? a.h : 0;
#pragma unroll
      for (int f = 0; f < S::FM; ++f) put_rows(sums + r * a.h, iw + 32 * f, limit, acc[f][g], lane);
    }
  }
  if (last && a.splits_dx == 1) put_tile<S>(acc, a.dX, [&](int j) { return a.row[j0 + j].r; }, a.h, i0, live - j0, lds);
}

// dW: M of the hidden dimension down, N entries across, summed over the rows; both operands are read by the transposing loads.
// 8192 x 4096 x 128256 by itself: 6.64 ms, 1297 TFLOP/s (a library product with such operands: 1180).  Few rows: bound by dW's bytes
// (64 rows: 377 us for 1.05 GB).
template <class S>
__device__ __forceinline__ void dw_tile(const LogprobArgs& a, int piece, const Tile& tile, uint8_t* lds) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int live = *a.live, np = up64(live);
  const int split = tile.part, k = (np / 64 + a.splits_dw - 1) / a.splits_dw * 64;
  const int64_t i0 = (int64_t)tile.down * S::M, j0 = (int64_t)tile.across * S::N;
  const int iw = (int)i0 + wave / S::WN * S::FM * 32, jw = wave % S::WN * S::FN * 32;
  f32x16 acc[S::FM][S::FN];
  const int v0 = piece * a.piece_v + (int)j0, vn = min(S::N, min(a.piece_v - (int)j0, a.v - v0));   // the tile's entries
  // What the targets' dz left out (rest): the targets are looked through for this tile's entries, 64 per wavefront and turn,
  // and those found are listed in their order, as many at a time as the list holds in any case.
  constexpr int TURNS = 8, LIST = S::P == 1 ? 256 * S::WAVES : 1;
  __shared__ struct { float rem; int32_t row, col; } s_list[LIST];
  __shared__ int s_count[S::WAVES];
  const bool rest = S::P == 1 && split == 0;
  int listed = 0, seen = 0, taken = 0;   // of the batch from seen on, `taken` have been listed before
  auto collect = [&] {
    listed = 0;
    while (seen < a.e && listed < LIST) {
      uint64_t mask[TURNS];
      int t[TURNS], mine = 0;
#pragma unroll
      for (int u = 0; u < TURNS; ++u) {
        const int e = seen + (wave * TURNS + u) * 64 + lane;
        t[u] = e < a.e ? a.tgt[e] - v0 : -1;
      }
#pragma unroll
      for (int u = 0; u < TURNS; ++u) {
        mask[u] = __ballot(t[u] >= 0 && t[u] < vn);
        mine += __builtin_popcountll(mask[u]);
      }
      __syncthreads();
      if (lane == 0) s_count[wave] = mine;
      __syncthreads();
      int at = listed - taken, all = -taken;
#pragma unroll
      for (int w = 0; w < S::WAVES; ++w) {
        const int n = s_count[w];
        if (w < wave) at += n;
        all += n;
      }
#pragma unroll
      for (int u = 0; u < TURNS; ++u) {
        const int k = at + __builtin_popcountll(mask[u] & ((1ull << lane) - 1));
        if ((mask[u] >> lane & 1) && k >= listed && k < LIST) s_list[k] = {0.f, seen + (wave * TURNS + u) * 64 + lane, t[u]};
        at += __builtin_popcountll(mask[u]);
      }
      if (listed + all > LIST) {
        taken += LIST - listed;
        listed = LIST;
        break;
      }
      listed += all;
      taken = 0;
      seen += 64 * TURNS * S::WAVES;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < listed; k += S::THREADS) {
      const int e = s_list[k].row, r = a.ent_row[e];
      s_list[k].rem = rem_of(a, e, r, live);
      s_list[k].row = r;
    }
  };
  if (rest) collect();
  const Operand X = part_of({a.xc, a.hp, (int64_t)a.np * a.hp, a.hp, np}, true, (int64_t)split * k, k);
  const Operand D = part_of({a.dl, a.piece_v, (int64_t)a.np * a.piece_v, a.piece_v, np}, true, (int64_t)split * k, k);
  product<S, true, true>(acc, X, D, i0, j0, X.ks, lds);
  if (rest) {
    for (;;) {
      add_terms<S>(
          acc, listed,
          [&](int k) { return Term{s_list[k].rem != 0.f ? a.xc + (int64_t)s_list[k].row * a.hp : nullptr, s_list[k].col, s_list[k].rem}; }, i0, a.h, lds);
      if (seen >= a.e) break;
      collect();
    }
  }
  if (a.splits_dw > 1) {
    float* sums = a.dw_acc + (int64_t)split * a.piece_v * a.h;
#pragma unroll
    for (int g = 0; g < S::FN; ++g) {
      const int j = jw + 32 * g + (lane & 31);
#pragma unroll
      for (int f = 0; f < S::FM; ++f) put_rows(sums + (j0 + j) * a.h, iw + 32 * f, j < vn ? a.h : 0, acc[f][g], lane);
    }
  } else {
    put_tile<S>(acc, a.dW, [&](int j) { return v0 + j; }, a.h, i0, vn, lds);
  }
}

// Both gradients of a piece in one launch where their tiles are of one shape: dX has few and long ones, whose last round would leave most
// of the chip idle, the more so as it is not known ahead how many rows are live; dW's fill it.  (The live tiles are the first ones, so
// that every XCD gets its share of them.)  2047 rows x 1544 x 50257, two fifths of the rows without gradient: 551 us one after the
// other, 460 so; 8192 x 4096 x 128256, a fifth: 11.96 and 10.97 ms.
template <class S>
__global__ __launch_bounds__(S::THREADS) void grads_kernel(LogprobArgs a, int piece, int downs, int dx_blocks, int dw_acrosses, int dw_blocks) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[S::LDS];
  const int block = blockIdx.x;
  if (block < dx_blocks) {
    constexpr bool TAIL = HasTail<S>;
    using T = std::conditional_t<TAIL, GradsTail<S>, S>;
    static_assert(T::THREADS == S::THREADS && T::LDS <= S::LDS, "in its place");
    const int live = *a.live, whole = whole_tiles<S>(live), blocks = downs * a.splits_dx * whole, parts = downs * a.splits_dx;
    if (block < blocks) {
      dx_tile<S>(a, piece, tile_of(block, blocks, downs, whole), lds);
    } else if (TAIL && block < blocks + parts && whole * S::N < live) {
      Tile tile = tile_of(block - blocks, parts, downs, 1);
      tile.across = whole * (S::N / T::N);
      dx_tile<T>(a, piece, tile, lds);
    }
  } else {
    dw_tile<S>(a, piece, tile_of(block - dx_blocks, dw_blocks, downs, dw_acrosses), lds);
  }
}

// Rows of h elements: the sum of their fp32 slabs, first to last.  ROWS: of the live rows, to where they come from.
template <bool FP32, bool ROWS>
__global__ __launch_bounds__(256) void slabs_kernel(LogprobArgs a, const float* slab, int64_t stride, int count, void* out, int rows) {
  const int64_t n = (int64_t)(ROWS ? *a.live : rows) * a.h;
  for (int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x); i < n; i += 4 * (int64_t)gridDim.x * 256) {
    f32x4 x = *(const f32x4*)(slab + i);
#pragma unroll 4
    for (int k = 1; k < count; ++k) x += *(const f32x4*)(slab + k * stride + i);
    int64_t at = i;
    if (ROWS) {
      const int64_t row = i / a.h;
      at = (int64_t)a.row[row].r * a.h + (i - row * a.h);
    }
    if (FP32) *(f32x4*)((float*)out + at) = x;
    else *(u32x2*)((bf16_t*)out + at) = u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
  }
}

int tiles(int64_t n, int tile) { return (int)((n + tile - 1) / tile); }
int piece_rows(const LogprobArgs& a, int piece) { return std::min(a.piece_v, a.v - piece * a.piece_v); }

}  // namespace

hipError_t launch_logprob_prep(const LogprobArgs& a, hipStream_t st) {
  if (a.planes == 3) hipLaunchKernelGGL(prep_kernel<true>, dim3((unsigned)a.np), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(prep_kernel<false>, dim3((unsigned)a.np), dim3(256), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_logprob_rows(const LogprobArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.n + 64), wg(256);
  if (a.n <= 256) {
    if (a.planes == 3) hipLaunchKernelGGL((gather_kernel<true, true>), grid, wg, 0, st, a);
    else hipLaunchKernelGGL((gather_kernel<false, true>), grid, wg, 0, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(rows_kernel, dim3((unsigned)((a.n + 255) / 256)), wg, 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(before_kernel, dim3(1), dim3(1024), 0, st, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.planes == 3) hipLaunchKernelGGL((gather_kernel<true, false>), grid, wg, 0, st, a);
  else hipLaunchKernelGGL((gather_kernel<false, false>), grid, wg, 0, st, a);
  return hipGetLastError();
}
hipError_t launch_logprob_wplanes(const LogprobArgs& a, int piece, hipStream_t st) {
  hipLaunchKernelGGL(wplanes_kernel, dim3((unsigned)a.piece_v), dim3(256), 0, st, a, piece);
  return hipGetLastError();
}
namespace {
// narrow tiles that cover n down
template <class S>
int tail_tiles(int64_t n) {
  if constexpr (HasTail<S>) return tiles(n, LogitsTail<S>::M);
  return 0;
}
// One workgroup per tile of down x across; of narrow ones there may be more down.
template <class S, bool BACKWARD>
void launch_logits(const LogprobArgs& a, int piece, hipStream_t st) {
  const int d = tiles(piece_rows(a, piece), S::M), c = tiles(BACKWARD ? a.np : a.n, S::N), tails = tail_tiles<S>(piece_rows(a, piece));
  hipLaunchKernelGGL((logits_kernel<S, BACKWARD>), dim3((unsigned)d * (unsigned)c + (unsigned)std::max(0, tails - d)), dim3(S::THREADS), 0, st, a, piece, d, tails);
}
template <int P, bool BACKWARD>
void logits(const LogprobArgs& a, int piece, hipStream_t st) {
  using T = Tilings<P>;
  if (a.shape == LP_LARGE) launch_logits<typename T::Large, BACKWARD>(a, piece, st);
  else if (a.shape == LP_SMALL) launch_logits<typename T::Small, BACKWARD>(a, piece, st);
  else if (a.shape == LP_DEEP) launch_logits<typename T::Deep, BACKWARD>(a, piece, st);
  else launch_logits<typename T::Thin, BACKWARD>(a, piece, st);
}
// One workgroup per tile and part of the sum, of either gradient or of both.
template <class S>
void launch_grads(const LogprobArgs& a, int piece, bool dx, bool dw, hipStream_t st) {
  const int downs = tiles(a.h, S::M), xc = tiles(a.n, S::N), wc = tiles(piece_rows(a, piece), S::N);
  const int xn = dx ? downs * xc * a.splits_dx : 0, wn = dw ? downs * wc * a.splits_dw : 0;
  hipLaunchKernelGGL(grads_kernel<S>, dim3((unsigned)xn + (unsigned)wn), dim3(S::THREADS), 0, st, a, piece, downs, xn, wc, wn);
}
template <int P>
void grads(const LogprobArgs& a, int piece, int shape, bool dx, bool dw, hipStream_t st) {
  using T = Tilings<P>;
  if (shape == LP_LARGE) launch_grads<typename T::Large>(a, piece, dx, dw, st);
  else if (shape == LP_SMALL) launch_grads<typename T::Small>(a, piece, dx, dw, st);
  else launch_grads<typename T::Deep>(a, piece, dx, dw, st);
}
template <bool ROWS>
void sum_slabs(const LogprobArgs& a, const float* slab, int64_t stride, int count, void* out, int rows, hipStream_t st) {
  const dim3 grid((unsigned)std::min<int64_t>(((int64_t)rows * a.h / 4 + 255) / 256, 8192));
  if (a.planes == 3) hipLaunchKernelGGL((slabs_kernel<true, ROWS>), grid, dim3(256), 0, st, a, slab, stride, count, out, rows);
  else hipLaunchKernelGGL((slabs_kernel<false, ROWS>), grid, dim3(256), 0, st, a, slab, stride, count, out, rows);
}
}  // namespace

hipError_t launch_logprob_logits(const LogprobArgs& a, int piece, bool backward, hipStream_t st) {
  if (backward) a.planes == 3 ? logits<3, true>(a, piece, st) : logits<1, true>(a, piece, st);
  else a.planes == 3 ? logits<3, false>(a, piece, st) : logits<1, false>(a, piece, st);
  return hipGetLastError();
}
hipError_t launch_logprob_finish(const LogprobArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)tiles(a.n, 16));
  if (a.planes == 3) hipLaunchKernelGGL(finish_kernel<true>, grid, dim3(1024), 0, st, a);
  else hipLaunchKernelGGL(finish_kernel<false>, grid, dim3(1024), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_logprob_grads(const LogprobArgs& a, int piece, bool dx, bool dw, hipStream_t st) {
  const int shape = dx ? a.shape_dx : a.shape_dw;
  a.planes == 3 ? grads<3>(a, piece, shape, dx, dw, st) : grads<1>(a, piece, shape, dx, dw, st);
  return hipGetLastError();
}
hipError_t launch_logprob_dx_sum(const LogprobArgs& a, hipStream_t st) {
  sum_slabs<true>(a, a.dx_acc, (int64_t)a.n * a.h, a.splits_dx, a.dX, a.n, st);
  return hipGetLastError();
}
hipError_t launch_logprob_dw_sum(const LogprobArgs& a, int piece, hipStream_t st) {
  const int64_t at = (int64_t)piece * a.piece_v * a.h * (a.planes == 3 ? 4 : 2);
  sum_slabs<false>(a, a.dw_acc, (int64_t)a.piece_v * a.h, a.splits_dw, (uint8_t*)a.dW + at, piece_rows(a, piece), st);
  return hipGetLastError();
}

}  // namespace psattn
