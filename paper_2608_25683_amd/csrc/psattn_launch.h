// Kernel launchers (defined in psattn_fwd.hip, psattn_bwd.hip, psattn_f32.hip and psattn_layer.hip, called by the C ABI).
#pragma once
#include <hip/hip_runtime.h>

#include "psattn.h"
#include "psattn_plan.h"

namespace psattn {

struct FwdArgs {
  PlanView plan;
  Shape s;
  int32_t n_items, n_merge;
  int32_t max_merge_rows;   // rows of the largest merge record
  int32_t siblings;         // the plan has items of packed siblings (PART_SIBLINGS)
  const void* Q;
  const void* K;
  const void* V;
  void* O;
  void* O_lo;       // bf16: residual O - bf16(O) of the fp32 result [Ns][Hq][d], or null
  float* LSE;
  float* part_o;    // [partial rows][Hq][d]
  float* part_lse;  // [partial rows][Hq]
  int64_t pool_slots;  // rows of the K and V pools
};

struct BwdArgs {
  PlanView plan;
  Shape s;
  int32_t n_fwd, n_merge, n_bkv, n_reduce, n_pad;
  int32_t max_merge_rows;   // rows of the largest merge record
  int32_t siblings;         // the plan has items of packed siblings (PART_SIBLINGS)
  const void* Q;
  const void* K;
  const void* V;
  const void* O;
  const void* O_lo; // bf16: residual of O (Delta from O + O_lo), or null
  const float* LSE;
  const void* dO;
  float* dQ;
  float* dK;
  float* dV;
  float* delta;    // [Ns][Hq]
  float* lse2;     // [Ns][Hq] LSE * log2(e)
  float* kv_nls;   // [Ns][Hq] -LSE / scale   (start of the dK/dV kernels' S accumulators)
  float* kv_nd;    // [Ns][Hq] -Delta         (start of their dP accumulators; bf16: the exact
                   //                          Delta' from the dQ pass, which runs first)
  float* part_dq;  // [partial rows][Hq][d]
  float* part_eps; // [partial rows][Hq] row sums of dS' of each piece (bf16)
  float* part_dk;  // [partial tiles][BKV_TILE][d]; each tile belongs to one kv head
  float* part_dv;
  int64_t pool_slots;  // rows of the K and V pools
};

// Log-probabilities over a vocabulary (psattn_logprob.hip).  The vocabulary is taken in pieces of piece_v
// entries (the forward of bf16 in one); buffers in the workspace:
struct LogprobStat { float top, sum; };   // max of z log2(e) and the sum of exp2(z log2(e) - max)
// What the backward's tiles take of a row r: its G, its LSE log2(e), its targets e0 .. e1 - 1 and the first of them (-1: not one
// of the vocabulary); at: its place among the live rows of its 256, -1 if none of its adjoints is other than 0.
struct LogprobRow { float total, lse2, g0; int32_t t0, e0, e1, r, at; };
struct LogprobArgs {
  int32_t n, h, v, e;        // rows, hidden, vocabulary, targets
  int32_t shape, shape_dx, shape_dw;   // LP_THIN .. LP_LARGE: of the logits' tiles, of the gradients'
  int32_t part_v;            // forward: entries per part, those of a tile
  int32_t planes;            // 1: bf16.  3: fp32 as three bf16 planes
  int32_t hp, np;            // h and n rounded up to 64: the padding of xc and dl holds zeros
  int32_t piece_v;           // entries per piece, a multiple of 256
  int32_t pieces;
  int32_t splits_dx, stages_dx;   // parts of a piece's entries in the dX product, each with its own fp32 sums, of so many
  int32_t splits_dw;              //   stages of 64; parts of the live rows in the dW product likewise
  float scale;
  const void* X;
  const void* W;
  const int32_t* tgt_ptr;
  const int32_t* tgt;
  const float* lse;
  const float* dlogp;
  float* logp;
  float* lse_out;
  void* dX;
  void* dW;
  LogprobStat* part;         // forward: [parts of the vocabulary][n]
  // backward: only rows that have a gradient are multiplied, packed in their order; how many there are is known on the GPU alone
  LogprobRow* info;          // [n] of every row (more than 256 rows)
  int32_t* before;           // [n / 256 + 1] live rows ahead of each 256
  int32_t* live;             // their number
  LogprobRow* row;           // [np] of the live rows, and up to a multiple of 64 of them empty ones
  int32_t* ent_row;          // backward, bf16: [e] the live row of each target, by its place
  float* ent_rem;            //   and what the rounding of its dz to bf16 left out (at a row's first target of the token; else 0)
  uint16_t* xc;              // [planes][np][hp]: X as the products take it, backward: of the live rows
  uint16_t* wc;              // fp32: [planes][piece_v][hp] planes of the piece
  uint16_t* dl;              // backward: [planes][np][piece_v] dz of the piece
  float* dx_acc;             // backward: [splits_dx][n][h] sums over the pieces, where there is more than one piece or part
  float* dw_acc;             // backward: [splits_dw][piece_v][h] of a piece, where there is more than one part
};
// tiles of 128 x 32, 128 x 128 (one workgroup per CU with more stages in flight, or two), 256 x 256
enum { LP_THIN, LP_DEEP, LP_SMALL, LP_LARGE };

// AdamW (psattn_adamw.hip)
struct AdamwTensor {
  void* param;
  float* master;
  void* m;
  void* v;
  uint8_t* m_exp;
  uint8_t* v_exp;
  int64_t n;
  float decay;
  int32_t bf16;
};
struct AdamwItem { int32_t tensor, chunk; };      // elements chunk * ADAMW_CHUNK ... of a tensor
constexpr int ADAMW_CHUNK = 4096, ADAMW_BLOCK = 256;
constexpr int ADAMW_GRADS = 320;                  // gradient pointers of a launch, in its 4 KB of arguments
struct AdamwGrads {
  const void* g[ADAMW_GRADS];
  uint32_t bf16[ADAMW_GRADS / 32];
};
struct AdamwScalars {                             // what one step's elements take, rounded once from fp64
  double lr_decay;                                // lr * weight_decay
  float gs, b1, ob1, b2, ob2, inv_sb2, eps, lr_t;
  uint32_t key;
  int32_t skip;
};
#ifdef __HIPCC__
#define PSATTN_HD __host__ __device__
#define PSATTN_NO_CONTRACT _Pragma("clang fp contract(off)")   // products and sums rounded one by one
#else
#define PSATTN_HD
#define PSATTN_NO_CONTRACT
#endif
// the hash behind the random rounding: 32 bits to 32 bits, every input bit reaching every output bit
PSATTN_HD inline uint32_t adamw_mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9E3779B1u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}
// b^n by squaring, the same on the host and on the device
PSATTN_HD inline double adamw_pow(double b, int64_t n) {
  double r = 1.0;
  for (; n; n >>= 1, b *= b)
    if (n & 1) r *= b;
  return r;
}
PSATTN_HD inline AdamwScalars adamw_scalars(const psattn_adamw_hyper& h, double lr, double gs, int64_t step, uint32_t seed) {
  PSATTN_NO_CONTRACT
  AdamwScalars s;
  s.lr_decay = lr * h.weight_decay;
  s.gs = (float)gs;
  s.b1 = (float)h.beta1;
  s.ob1 = (float)(1.0 - h.beta1);
  s.b2 = (float)h.beta2;
  s.ob2 = (float)(1.0 - h.beta2);
  s.inv_sb2 = (float)(1.0 / __builtin_sqrt(1.0 - adamw_pow(h.beta2, step)));
  s.eps = (float)h.eps;
  s.lr_t = (float)(lr / (1.0 - adamw_pow(h.beta1, step)));
  s.key = adamw_mix(adamw_mix(seed) + (uint32_t)step);
  s.skip = 0;
  return s;
}
struct AdamwArgs {
  const AdamwTensor* tensors;
  const AdamwItem* items;
  int32_t item0, n_items;     // of this launch
  int32_t tensor0;
  int32_t total_items;
  int32_t bits;
  const AdamwScalars* dev;    // scalars formed on the device, or null: those below
  AdamwScalars s;
  double* part;               // per item sum of squares
  const psattn_adamw_dyn* dyn;
  float* norm;
  psattn_adamw_hyper hyper;
  AdamwScalars* dev_out;
};

// Each launcher enqueues one kernel on stream and returns the launch status.
hipError_t launch_fwd_main(const FwdArgs& a, bool bf16, hipStream_t st);
hipError_t launch_fwd_merge(const FwdArgs& a, bool bf16, hipStream_t st);
hipError_t launch_bwd_pre(const BwdArgs& a, bool bf16, hipStream_t st);
hipError_t launch_bwd_kv(const BwdArgs& a, bool bf16, hipStream_t st);
hipError_t launch_bwd_dq(const BwdArgs& a, bool bf16, hipStream_t st);
hipError_t launch_bwd_reduce_kv(const BwdArgs& a, hipStream_t st);
hipError_t launch_bwd_reduce_dq(const BwdArgs& a, bool bf16, hipStream_t st);
// the fp32 kernels (psattn_f32.hip), called by the launchers above
hipError_t launch_fwd_f32(const FwdArgs& a, hipStream_t st);
hipError_t launch_bwd_dq_f32(const BwdArgs& a, hipStream_t st);
hipError_t launch_bwd_kv_f32(const BwdArgs& a, hipStream_t st);
// layer steps around the attention (psattn_layer.hip)
hipError_t launch_rope(const PlanView& plan, int32_t ns, int32_t heads, int32_t d, float theta, bool inverse, bool bf16,
                       void* X, hipStream_t st);
hipError_t launch_kv_move(const PlanView& plan, int32_t ns, int32_t row_bytes, bool to_pool, const void* a0,
                          const void* a1, void* b0, void* b1, hipStream_t st);
hipError_t launch_split_planes(const float* x, void* planes, int64_t n, hipStream_t st);
hipError_t launch_silu_bwd(const float* dm, const void* a, const void* b, void* da, void* db, int64_t n, hipStream_t st);
// The training step behind the layers.  Weak: a host-only build links without these kernels, and its calls fail.
#define PSATTN_WEAK __attribute__((weak))
PSATTN_WEAK hipError_t launch_logprob_prep(const LogprobArgs& a, hipStream_t st);
PSATTN_WEAK hipError_t launch_logprob_rows(const LogprobArgs& a, hipStream_t st);
PSATTN_WEAK hipError_t launch_logprob_wplanes(const LogprobArgs& a, int piece, hipStream_t st);
PSATTN_WEAK hipError_t launch_logprob_logits(const LogprobArgs& a, int piece, bool backward, hipStream_t st);
PSATTN_WEAK hipError_t launch_logprob_finish(const LogprobArgs& a, hipStream_t st);
PSATTN_WEAK hipError_t launch_logprob_grads(const LogprobArgs& a, int piece, bool dx, bool dw, hipStream_t st);
PSATTN_WEAK hipError_t launch_logprob_dx_sum(const LogprobArgs& a, hipStream_t st);
PSATTN_WEAK hipError_t launch_logprob_dw_sum(const LogprobArgs& a, int piece, hipStream_t st);
PSATTN_WEAK hipError_t launch_adamw_norm(const AdamwArgs& a, const AdamwGrads& g, hipStream_t st);
PSATTN_WEAK hipError_t launch_adamw_scalars(const AdamwArgs& a, bool with_norm, hipStream_t st);
PSATTN_WEAK hipError_t launch_adamw_step(const AdamwArgs& a, const AdamwGrads& g, hipStream_t st);

}  // namespace psattn
