// AdamW over many tensors at once, its states in fp32 or in 8 bits, with clipping by the global norm.
//
// Every element takes, in fp32 with each product and sum rounded by itself (so that the results do not depend on the
// compiler's choice of fused operations):
//   g = gs grad,  m' = m b1 + g (1 - b1),  v' = v b2 + g^2 (1 - b2),  r = sqrt(v')
//   w' = w (1 - lr wd) - m' / (r / sqrt(1 - b2^t) + eps) * lr / (1 - b1^t)
// A workgroup takes ADAMW_CHUNK elements of one tensor (one record of the uploaded table), so any number of tensors of any
// size is one launch, and no tensor waits for another.  The kernels are bound by their bytes: 218 million bf16 weights with
// masters and fp32 gradients, 32-bit states 1218 us (30 bytes each, 5.4 TB/s), 8-bit states 797 us (18 bytes, 4.9 TB/s, with
// three quarters of the vector instructions' time behind it), the norm 187 us (4.7 TB/s; a large copy: 4.8).  Chunks of 8192 elements: 1243 and 783
// us, but 37 us instead of 31 for 300 tensors of 20000 on average and 12.4 instead of 9.5 for a tiny layer's nine.
//
// 8-bit states: a wavefront's turn is 256 elements, four per lane, which is one block of the states: its largest
// magnitude comes from the wavefront's own lanes, without LDS.  The power of two of a block moves the
// codes' grid by whole binades, so that an unchanged value stays on a code and is not rounded again.
#include <algorithm>

#include "psattn_device.h"

namespace psattn {
namespace {

using namespace dev;

constexpr int TURN = 1024;   // elements of a workgroup's turn: 4 per lane

// four elements at i of a gradient or a weight (their number in n: those behind it are 0)
__device__ __forceinline__ f32x4 load4(const float* p, int64_t i, int n) {
  if (n >= 4) return *(const f32x4*)(p + i);
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < n) x[k] = p[i + k];
  return x;
}
__device__ __forceinline__ f32x4 load4(const bf16_t* p, int64_t i, int n) {
  if (n >= 4) {
    const u32x2 b = ld8(p + i);
    return f32x4{bf2f(b[0] & 0xffffu), __uint_as_float(b[0] & 0xffff0000u), bf2f(b[1] & 0xffffu), __uint_as_float(b[1] & 0xffff0000u)};
  }
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < n) x[k] = bf2f(p[i + k]);
  return x;
}
__device__ __forceinline__ f32x4 load_grad(const void* g, bool bf16, int64_t i, int n) {
  return bf16 ? load4((const bf16_t*)g, i, n) : load4((const float*)g, i, n);
}
__device__ __forceinline__ void store4(float* p, int64_t i, int n, const f32x4& x) {
  if (n >= 4) {
    *(f32x4*)(p + i) = x;
    return;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < n) p[i + k] = x[k];
}
__device__ __forceinline__ void store4(bf16_t* p, int64_t i, int n, const f32x4& x) {
  const u32x2 b = {pack2(x[0], x[1]), pack2(x[2], x[3])};
  if (n >= 4) {
    *(u32x2*)(p + i) = b;
    return;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < n) p[i + k] = (bf16_t)(b[k / 2] >> (16 * (k & 1)));
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t i, int n) {
  if (n >= 4) return *(const uint32_t*)(p + i);
  uint32_t x = 0;
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < n) x |= (uint32_t)p[i + k] << (8 * k);
  return x;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t i, int n, uint32_t x) {
  if (n >= 4) {
    *(uint32_t*)(p + i) = x;
    return;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < n) p[i + k] = (uint8_t)(x >> (8 * k));
}

__device__ __forceinline__ f32x4 decode(uint32_t codes, int e) {
  const float p = __uint_as_float((uint32_t)e << 23);
  // (2^-127 and below are no powers that the encoder writes; 0 decodes to zeros)
  return f32x4{__builtin_amdgcn_cvt_f32_fp8(codes, 0) * p, __builtin_amdgcn_cvt_f32_fp8(codes, 1) * p,
               __builtin_amdgcn_cvt_f32_fp8(codes, 2) * p, __builtin_amdgcn_cvt_f32_fp8(codes, 3) * p};
}

// biased exponent of x, 0 if x is not finite
__device__ __forceinline__ uint32_t exponent(float x) {
  const uint32_t e = __float_as_uint(x) >> 23 & 0xffu;
  return e == 0xffu ? 0u : e;
}
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
__device__ __forceinline__ u16x2 max2(u16x2 a, u16x2 b) { return __builtin_elementwise_max(a, b); }
template <int ROTATE>
__device__ __forceinline__ u16x2 max_rotated(u16x2 x) {   // with the lane ROTATE further among 16
  const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x120 + ROTATE, 0xf, 0xf, true);
  return max2(x, __builtin_bit_cast(u16x2, y));
}
// both halves' max over the wavefront's 64 lanes, the same in every lane
__device__ __forceinline__ u16x2 wave_max(u16x2 x) {
  x = max_rotated<1>(max_rotated<2>(max_rotated<4>(max_rotated<8>(x))));
  const int y = __builtin_bit_cast(int, x);
  auto row = [&](int lane) { return __builtin_bit_cast(u16x2, __builtin_amdgcn_readlane(y, lane)); };
  return max2(max2(row(0), row(16)), max2(row(32), row(48)));
}

// x to its e4m3 value on the block's grid (as a float), up or down by the 16 random bits; above 2^-6 of the grid its codes
// have 3 bits behind the leading one (the low 20 bits of an fp32 are cut), below they are 2^-9 apart, as those
// behind 2^-6 are, to which such a value is moved and back.
template <bool FLOOR>
__device__ __forceinline__ float to_code(float x, float inv, uint32_t rnd) {
  const float a = fabsf(x) * inv;
  const float low = a < 0x1p-6f ? 0x1p-6f : 0.f;
  float y = __uint_as_float((__float_as_uint(a + low) + (rnd * 16u + 8u)) & 0xfff00000u) - low;
  if (FLOOR && x > 0.f && y == 0.f) y = 0x1p-9f;
  if (!is_finite(x)) y = __builtin_nanf("");
  return copysignf(y, x);
}
__device__ __forceinline__ uint32_t pack_codes(const f32x4& y) {
  int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  c = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
  return (uint32_t)c;
}

template <int BITS, class P>
__device__ __forceinline__ void step_chunk(const AdamwTensor& t, P* weights, const void* grad, bool grad_bf16, const AdamwScalars& s,
                                           int64_t base, uint32_t key, int tid) {
  PSATTN_NO_CONTRACT
  const float keep = (float)(1.0 - s.lr_decay * (double)t.decay);
  const int64_t end = min(t.n, base + ADAMW_CHUNK);
#pragma unroll 1
  for (int64_t at = base; at < end; at += TURN) {
    const int64_t i = at + 4 * tid;
    const int n = (int)min((int64_t)4, end - i);   // (0 or less: nothing, but the lane takes part in its block)
    const f32x4 gr = load_grad(grad, grad_bf16, i, n);
    f32x4 w = load4(weights, i, n), m, v;
    const int64_t blk = at / ADAMW_BLOCK + tid / 64;
    const bool held = blk * ADAMW_BLOCK < end;     // (uniform over the wavefront)
    if (BITS == 8) {
      const int em = held ? t.m_exp[blk] : 1, er = held ? t.v_exp[blk] : 1;
      m = decode(load_codes((const uint8_t*)t.m, i, n), em);
      const f32x4 r = decode(load_codes((const uint8_t*)t.v, i, n), er);
      v = r * r;
    } else {
      m = load4((const float*)t.m, i, n);
      v = load4((const float*)t.v, i, n);
    }
    f32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float g = gr[k] * s.gs;
      m[k] = m[k] * s.b1 + g * s.ob1;
      v[k] = v[k] * s.b2 + (g * g) * s.ob2;
      r[k] = sqrtf(v[k]);
      w[k] = w[k] * keep - (m[k] / (r[k] * s.inv_sb2 + s.eps)) * s.lr_t;
    }
    store4(weights, i, n, w);
    if (t.bf16) store4((bf16_t*)t.param, i, n, w);
    if (BITS == 8) {
      f32x4 ym, yr;
      u16x2 top = {0, 0};   // (elements behind the tensor's end have m = v = 0)
#pragma unroll
      for (int k = 0; k < 4; ++k) top = max2(top, u16x2{(uint16_t)exponent(m[k]), (uint16_t)exponent(r[k])});
      top = wave_max(top);
      const int em = max((int)top[0] - 7, 1), er = max((int)top[1] - 7, 1);
      const float im = __uint_as_float((uint32_t)(254 - em) << 23), ir = __uint_as_float((uint32_t)(254 - er) << 23);
      const uint32_t h0 = (uint32_t)i * 0x9E3779B1u;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t h = adamw_mix((h0 + k * 0x9E3779B1u) ^ key);
        ym[k] = to_code<false>(m[k], im, h >> 16);
        yr[k] = to_code<true>(r[k], ir, h & 0xffffu);
      }
      store_codes((uint8_t*)t.m, i, n, pack_codes(ym));
      store_codes((uint8_t*)t.v, i, n, pack_codes(yr));
      if (held && tid % 64 == 0) {
        t.m_exp[blk] = (uint8_t)em;
        t.v_exp[blk] = (uint8_t)er;
      }
    } else {
      store4((float*)t.m, i, n, m);
      store4((float*)t.v, i, n, v);
    }
  }
}

template <int BITS>
__global__ __launch_bounds__(256) void adamw_step_kernel(AdamwArgs a, AdamwGrads g) {
  const AdamwItem it = a.items[a.item0 + blockIdx.x];
  const int gi = it.tensor - a.tensor0;
  const void* grad = g.g[gi];
  if (!grad) return;
  const AdamwScalars s = a.dev ? *a.dev : a.s;
  if (s.skip) return;
  const AdamwTensor t = a.tensors[it.tensor];
  const bool gb = g.bf16[gi / 32] >> (gi % 32) & 1;
  const int64_t base = (int64_t)it.chunk * ADAMW_CHUNK;
  const uint32_t key = adamw_mix(s.key + (uint32_t)it.tensor);
  step_chunk<BITS, float>(t, t.bf16 ? t.master : (float*)t.param, grad, gb, s, base, key, threadIdx.x);
}

// sum of x over the workgroup in a fixed order; every thread calls it, thread 0 gets it
template <int THREADS>
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double part[THREADS / 64];
#pragma unroll
  for (int w = 32; w >= 1; w >>= 1) x += __shfl_xor(x, w);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
  __syncthreads();
  double r = 0;
  for (int k = 0; k < THREADS / 64; ++k) r += part[k];
  return r;
}

// Sum of squares of a chunk's gradients, in fp64: a square of fp32 is exact there, and no sum overflows.
__global__ __launch_bounds__(256) void adamw_norm_kernel(AdamwArgs a, AdamwGrads g) {
  const AdamwItem it = a.items[a.item0 + blockIdx.x];
  const int gi = it.tensor - a.tensor0;
  const void* grad = g.g[gi];
  const bool gb = g.bf16[gi / 32] >> (gi % 32) & 1;
  const int64_t base = (int64_t)it.chunk * ADAMW_CHUNK, end = min(a.tensors[it.tensor].n, base + ADAMW_CHUNK);
  double x = 0;
  if (grad) {
#pragma unroll 4
    for (int64_t i = base + 4 * threadIdx.x; i < end; i += TURN) {
      const f32x4 v = load_grad(grad, gb, i, (int)min((int64_t)4, end - i));
#pragma unroll
      for (int k = 0; k < 4; ++k) x = fma((double)v[k], (double)v[k], x);
    }
  }
  x = block_sum<256>(x);
  if (threadIdx.x == 0) a.part[a.item0 + blockIdx.x] = x;
}

// The step's scalars: the norm of the chunks' sums, the clipping factor, what dyn holds.
__global__ __launch_bounds__(1024) void adamw_scalars_kernel(AdamwArgs a, int with_norm) {
  PSATTN_NO_CONTRACT
  double x = 0;
  if (with_norm)
#pragma unroll 16
    for (int i = threadIdx.x; i < a.total_items; i += 1024) x += a.part[i];
  x = block_sum<1024>(x);
  if (threadIdx.x) return;
  double lr = a.hyper.lr, gs = a.hyper.grad_scale;
  int64_t step = a.hyper.step;
  uint32_t seed = a.hyper.seed;
  if (a.dyn) {
    lr = a.dyn->lr;
    gs = a.dyn->grad_scale;
    step = max(a.dyn->step, 1);
    seed = a.dyn->seed;
  }
  const double norm = fabs(gs) * sqrt(x);
  const bool clip = a.hyper.max_norm > 0;
  if (with_norm && clip) gs = gs * fmin(1.0, a.hyper.max_norm / (norm + 1e-6));
  AdamwScalars s = adamw_scalars(a.hyper, lr, gs, step, seed);
  s.skip = with_norm && clip && !(norm < __builtin_inf());
  *a.dev_out = s;
  if (a.norm) *a.norm = (float)norm;
}

}  // namespace

hipError_t launch_adamw_norm(const AdamwArgs& a, const AdamwGrads& g, hipStream_t st) {
  hipLaunchKernelGGL(adamw_norm_kernel, dim3((unsigned)a.n_items), dim3(256), 0, st, a, g);
  return hipGetLastError();
}
hipError_t launch_adamw_scalars(const AdamwArgs& a, bool with_norm, hipStream_t st) {
  hipLaunchKernelGGL(adamw_scalars_kernel, dim3(1), dim3(1024), 0, st, a, with_norm ? 1 : 0);
  return hipGetLastError();
}
hipError_t launch_adamw_step(const AdamwArgs& a, const AdamwGrads& g, hipStream_t st) {
  if (a.bits == 8) hipLaunchKernelGGL(adamw_step_kernel<8>, dim3((unsigned)a.n_items), dim3(256), 0, st, a, g);
  else hipLaunchKernelGGL(adamw_step_kernel<32>, dim3((unsigned)a.n_items), dim3(256), 0, st, a, g);
  return hipGetLastError();
}

}  // namespace psattn
