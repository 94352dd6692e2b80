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

#include "psattn_device.h"

namespace psattn {
namespace {

using namespace dev;

constexpr int TM = 128, TN = 128, BK = 64, LDK = BK + 8;

// An operand of a product: element (i, k) of plane q at p + q plane + i ld + k, or + k ld + i where K is the outer dimension.
// Elements of i >= rows or k >= ks are 0.
struct Operand {
  const bf16_t* p;
  int64_t ld, plane;
  int rows, ks;
};
__constant__ const int kPairA[6] = {2, 1, 0, 1, 0, 0}, kPairB[6] = {0, 1, 2, 0, 1, 0};

template <bool KOUTER>
__device__ __forceinline__ void load_tile(bf16_t (*lds)[LDK], const Operand& o, int q, int64_t i0, int64_t k0) {
  const bf16_t* p = o.p + q * o.plane;
  for (int c = threadIdx.x; c < TM * BK / 8; c += 256) {
    u32x4 x = {0, 0, 0, 0};
    if (!KOUTER) {
      const int i = c / (BK / 8), k = c % (BK / 8) * 8;
      if (i0 + i < o.rows && k0 + k < o.ks) x = ld16(p + (i0 + i) * o.ld + k0 + k);
      *(u32x4*)&lds[i][k] = x;
    } else {
      const int k = c / (TM / 8), i = c % (TM / 8) * 8;
      if (i0 + i < o.rows && k0 + k < o.ks) x = ld16(p + (k0 + k) * o.ld + i0 + i);
#pragma unroll
      for (int e = 0; e < 8; ++e) lds[i + e][k] = (bf16_t)(x[e / 2] >> (16 * (e & 1)));
    }
  }
}

// acc[f] = A rows i0 + 32 f .. (down the 32 x 32 tile) x B rows j0 + 32 wave .. (across) over k < ks
template <bool KA, bool KB>
__device__ __forceinline__ void product(f32x16 (&acc)[4], const Operand& A, const Operand& B, int planes, int64_t i0, int64_t j0, int ks) {
  __shared__ __attribute__((aligned(16))) bf16_t sa[TM][LDK], sb[TN][LDK];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[f][e] = 0.f;
  for (int q = planes == 3 ? 0 : 5; q < 6; ++q)
    for (int k0 = 0; k0 < ks; k0 += BK) {
      __syncthreads();
      load_tile<KA>(sa, A, kPairA[q], i0, k0);
      load_tile<KB>(sb, B, kPairB[q], j0, k0);
      __syncthreads();
#pragma unroll
      for (int k = 0; k < BK; k += 16) {
        const bf16x8 b = as_bf(ld16(&sb[32 * wave + (lane & 31)][k + 8 * (lane >> 5)]));
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[f] = mfma(as_bf(ld16(&sa[32 * f + (lane & 31)][k + 8 * (lane >> 5)])), b, acc[f]);
      }
    }
}
// the row down the 32 x 32 tile of element e of a lane
__device__ __forceinline__ int down(int e, int lane) { return 8 * (e / 4) + 4 * (lane >> 5) + e % 4; }

__device__ __forceinline__ Operand x_operand(const LogprobArgs& a) {
  if (a.xc) return {a.xc, a.hp, (int64_t)a.np * a.hp, a.np, a.hp};
  return {(const bf16_t*)a.X, a.h, 0, a.n, a.h};
}
__device__ __forceinline__ Operand w_operand(const LogprobArgs& a, int piece) {
  const int v0 = piece * a.piece_v, rows = min(a.piece_v, a.v - v0);
  if (a.wc) return {a.wc, a.hp, (int64_t)a.piece_v * a.hp, rows, a.hp};
  return {(const bf16_t*)a.W + (int64_t)v0 * a.h, a.h, 0, rows, a.h};
}
__device__ __forceinline__ Operand swapped(const Operand& o) { return {o.p, o.ld, o.plane, o.ks, o.rows}; }

// bounds of a row's targets, whatever tgt_ptr holds
__device__ __forceinline__ void targets_of(const LogprobArgs& a, int r, int& e0, int& e1) {
  e0 = min(max(a.tgt_ptr[r], 0), a.e);
  e1 = min(max(a.tgt_ptr[r + 1], e0), a.e);
}

// ---- rows as the products take them
template <bool FP32>
__global__ __launch_bounds__(256) void prep_kernel(LogprobArgs a, int backward) {
  const int r = blockIdx.x;
  __shared__ int s_live;
  if (threadIdx.x == 0) {
    bool live = !backward;
    float total = 0.f;
    if (backward && r < a.n) {
      int e0, e1;
      targets_of(a, r, e0, e1);
      for (int e = e0; e < e1; ++e) {
        const int t = a.tgt[e];
        const float g = a.dlogp[e];
        if (t >= 0 && t < a.v) {
          total += g;
          live = live || g != 0.f;
        }
      }
      a.total[r] = total;
    }
    s_live = live && r < a.n;
  }
  __syncthreads();
  const bool live = s_live;
  for (int c = 8 * threadIdx.x; c < a.hp; c += 8 * 256) {
    const bool in = live && c < a.h;
    if (!FP32) {
      u32x4 x = {0, 0, 0, 0};
      if (in) x = ld16((const bf16_t*)a.X + (int64_t)r * a.h + c);
      *(u32x4*)(a.xc + (int64_t)r * a.hp + c) = x;
    } else {
      for (int k = 0; k < 8; k += 4) {
        f32x4 x = {0, 0, 0, 0};
        if (in) x = *(const f32x4*)((const float*)a.X + (int64_t)r * a.h + c + k);
        put_planes(x, a.xc, (int64_t)a.np * a.hp, (int64_t)r * a.hp + c + k);
      }
    }
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

// ---- a tile of logits: 128 entries of the piece down, 128 rows across
template <bool BACKWARD>
__global__ __launch_bounds__(256) void logits_kernel(LogprobArgs a, int piece) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i0 = (int64_t)blockIdx.x * TM, j0 = (int64_t)blockIdx.y * TN;
  f32x16 acc[4];
  const Operand W = w_operand(a, piece);
  product<false, false>(acc, W, x_operand(a), a.planes, i0, j0, a.hp);
  const int64_t r = j0 + 32 * wave + (lane & 31);
  const float c = a.scale * kLog2e;
  if (!BACKWARD) {
    float top = kNegInf, sum = 0.f;
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const bool in = i0 + 32 * f + down(e, lane) < W.rows;
        acc[f][e] = in ? acc[f][e] * c : kNegInf;
        top = fmaxf(top, acc[f][e]);
      }
    top = pair_max(top);
    const float ref = top == kNegInf ? 0.f : top;
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum += fast_exp2(acc[f][e] - ref);
    sum = pair_sum(sum);
    if (r < a.n && lane < 32 && i0 < W.rows) a.part[((int64_t)piece * (a.piece_v / LP_PART) + blockIdx.x) * a.n + r] = {top, sum};
    return;
  }
  if (r >= a.np) return;
  const bool in_row = r < a.n;
  const float total = in_row ? a.total[r] : 0.f, lse2 = in_row ? a.lse[r] * kLog2e : 0.f;
  int e0 = 0, e1 = 0;
  if (in_row) targets_of(a, (int)r, e0, e1);
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t i = i0 + 32 * f + down(e, lane);
      float d = i < W.rows && total != 0.f ? -total * fast_exp2(acc[f][e] * c - lse2) : 0.f;
      for (int t = e0; t < e1; ++t)
        if (a.tgt[t] == piece * a.piece_v + i && i < W.rows) d += a.dlogp[t];
      d *= a.scale;
      if (i >= a.piece_v) continue;
      const int64_t at = r * a.piece_v + i, plane = (int64_t)a.np * a.piece_v;
      if (a.planes == 1) {
        a.dl[at] = (bf16_t)pack2(d, 0.f);
      } else {
        put_plane1(d, a.dl, plane, at);
      }
    }
}

// ---- LSE and logp from the tiles' parts: a wavefront per row
template <bool FP32>
__global__ __launch_bounds__(64) void finish_kernel(LogprobArgs a) {
  const int r = blockIdx.x, lane = threadIdx.x;
  const int parts = (a.v + LP_PART - 1) / LP_PART;
  float top = kNegInf, sum = 0.f;
  for (int t = lane; t < parts; t += 64) top = fmaxf(top, a.part[(int64_t)t * a.n + r].top);
  for (int w = 32; w >= 1; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
  const float ref = top == kNegInf ? 0.f : top;
  for (int t = lane; t < parts; t += 64) {
    const LogprobStat p = a.part[(int64_t)t * a.n + r];
    sum += p.sum * fast_exp2(p.top - ref);
  }
  for (int w = 32; w >= 1; w >>= 1) sum += __shfl_xor(sum, w);
  const float lse = (ref + log2f(sum)) * (1.f / kLog2e);
  if (lane == 0) a.lse_out[r] = lse;
  int e0, e1;
  targets_of(a, r, e0, e1);
  const void* x = elem_ptr<!FP32>(a.X, (size_t)r * a.h);
  for (int e = e0; e < e1; ++e) {
    const int t = a.tgt[e];
    float z = 0.f;
    if (t >= 0 && t < a.v) {
      for (int c = lane; c < a.h; c += 64) z = fmaf(elem<!FP32>(x, c), elem<!FP32>(elem_ptr<!FP32>(a.W, (size_t)t * a.h), c), z);
      for (int w = 32; w >= 1; w >>= 1) z += __shfl_xor(z, w);
      z = z * a.scale - lse;
    }
    if (lane == 0) a.logp[e] = z;
  }
}

// one element of a result of the inputs' type
__device__ __forceinline__ void put(void* p, int64_t i, float x, bool fp32) {
  if (fp32) ((float*)p)[i] = x;
  else ((bf16_t*)p)[i] = (bf16_t)pack2(x, 0.f);
}

// dX: 128 of the hidden dimension down, 128 rows across
__global__ __launch_bounds__(256) void dx_kernel(LogprobArgs a, int piece) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i0 = (int64_t)blockIdx.x * TM, j0 = (int64_t)blockIdx.y * TN;
  f32x16 acc[4];
  const Operand W = swapped(w_operand(a, piece));
  const Operand D = {a.dl, a.piece_v, (int64_t)a.np * a.piece_v, a.np, a.piece_v};
  product<true, false>(acc, W, D, a.planes, i0, j0, W.ks);
  const int64_t r = j0 + 32 * wave + (lane & 31);
  if (r >= a.n) return;
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t i = i0 + 32 * f + down(e, lane);
      if (i >= a.h) continue;
      float x = acc[f][e];
      if (piece) x += a.dx_acc[r * a.h + i];
      if (piece < a.pieces - 1) a.dx_acc[r * a.h + i] = x;
      else put(a.dX, r * a.h + i, x, a.planes == 3);
    }
}

// dW: 128 of the hidden dimension down, 128 entries across
__global__ __launch_bounds__(256) void dw_kernel(LogprobArgs a, int piece) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i0 = (int64_t)blockIdx.x * TM, j0 = (int64_t)blockIdx.y * TN;
  f32x16 acc[4];
  const Operand X = {a.xc, a.hp, (int64_t)a.np * a.hp, a.hp, a.np};
  const Operand D = {a.dl, a.piece_v, (int64_t)a.np * a.piece_v, a.piece_v, a.np};
  product<true, true>(acc, X, D, a.planes, i0, j0, a.np);
  const int64_t v = j0 + 32 * wave + (lane & 31), at = (int64_t)piece * a.piece_v + v;
  if (v >= a.piece_v || at >= a.v) return;
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t i = i0 + 32 * f + down(e, lane);
      if (i < a.h) put(a.dW, at * a.h + i, acc[f][e], a.planes == 3);
    }
}

unsigned tiles(int64_t n) { return (unsigned)((n + 127) / 128); }
int piece_rows(const LogprobArgs& a, int piece) { return std::min(a.piece_v, a.v - piece * a.piece_v); }

}  // namespace

hipError_t launch_logprob_prep(const LogprobArgs& a, bool backward, hipStream_t st) {
  if (a.planes == 3) hipLaunchKernelGGL(prep_kernel<true>, dim3((unsigned)a.np), dim3(256), 0, st, a, backward ? 1 : 0);
  else hipLaunchKernelGGL(prep_kernel<false>, dim3((unsigned)a.np), dim3(256), 0, st, a, backward ? 1 : 0);
  return hipGetLastError();
}
hipError_t launch_logprob_wplanes(const LogprobArgs& a, int piece, hipStream_t st) {
  hipLaunchKernelGGL(wplanes_kernel, dim3((unsigned)a.piece_v), dim3(256), 0, st, a, piece);
  return hipGetLastError();
}
hipError_t launch_logprob_logits(const LogprobArgs& a, int piece, bool backward, hipStream_t st) {
  const dim3 grid(tiles(backward ? a.piece_v : piece_rows(a, piece)), tiles(backward ? a.np : a.n));
  if (backward) hipLaunchKernelGGL(logits_kernel<true>, grid, dim3(256), 0, st, a, piece);
  else hipLaunchKernelGGL(logits_kernel<false>, grid, dim3(256), 0, st, a, piece);
  return hipGetLastError();
}
hipError_t launch_logprob_finish(const LogprobArgs& a, hipStream_t st) {
  if (a.planes == 3) hipLaunchKernelGGL(finish_kernel<true>, dim3((unsigned)a.n), dim3(64), 0, st, a);
  else hipLaunchKernelGGL(finish_kernel<false>, dim3((unsigned)a.n), dim3(64), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_logprob_dx(const LogprobArgs& a, int piece, hipStream_t st) {
  hipLaunchKernelGGL(dx_kernel, dim3(tiles(a.h), tiles(a.n)), dim3(256), 0, st, a, piece);
  return hipGetLastError();
}
hipError_t launch_logprob_dx_sum(const LogprobArgs&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_logprob_dw(const LogprobArgs& a, int piece, hipStream_t st) {
  hipLaunchKernelGGL(dw_kernel, dim3(tiles(a.h), tiles(piece_rows(a, piece))), dim3(256), 0, st, a, piece);
  return hipGetLastError();
}

}  // namespace psattn
