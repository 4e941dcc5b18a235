// lm.hpp -- launch interface of the operators for language-model learners
// (gfx950): the loss over a large vocabulary, the norms around a block, and
// activations kept in 8 bits.
//
// As in kernels.hpp, replica j of k owns rows [j*n, (j+1)*n) of every
// activation and its parameters start pstride elements after those of
// replica j-1.  Launchers enqueue on the given stream and return the
// hipError_t of their launches; arguments have been checked by the caller.
#pragma once
#include "kernels.hpp"

namespace cbk {

enum { LM_F32 = 0, LM_F16 = 1, LM_BF16 = 2 };
inline int lm_size(int type) { return type == LM_F32 ? 4 : 2; }

// Softmax cross-entropy of h W^T (vocab_xent.hip).
struct XentArgs {
  int type, k, n, d, v;
  const void* h;          // [k*n] rows of d elements, ldh apart
  int64_t ldh;
  const void* w;          // [k] matrices [v][d], pstride elements apart
  int64_t pstride;
  const int32_t* labels;  // [k*n]
  int ignore;
  float* loss;            // [k] (forward)
  float* lse;             // [k*n] (written by the forward, read by the backward)
  float grad_scale;
  void* dh;               // [k*n][d]
  void* dw;               // [k] matrices [v][d], dstride elements apart
  int64_t dstride;
  void* ws;
};
size_t xent_ws_bytes(const XentArgs& a, bool backward);  // 0: too large for a launch
hipError_t xent_fwd(const XentArgs& a, hipStream_t s);
hipError_t xent_bwd(const XentArgs& a, hipStream_t s);

// The norms around a block with its gate and residual scale (gated_norm.hip).
struct NormArgs {
  int type, k, n, d;
  const void* x;          // forward: the stream before the block; backward: after it
  const void* block;      // or nullptr
  const void* gate;       // [k][ceil(n/gate_rows)][d], or nullptr
  int gate_rows;          // rows that share a row of the gate
  float res_scale, eps;
  const float* post;      // gamma of the norm after the block, or nullptr
  const float* pre;       // gamma of the norm before the next one, or nullptr
  int64_t post_stride, pre_stride;
  void* x_out;            // forward
  void* y;
  void* y_kept;           // y in 8 bits, or nullptr
  const void* dy;         // backward
  const void* dres;       // or nullptr
  void *dx, *dblock, *dgate;
  float *dpost, *dpre;
  int64_t dpost_stride, dpre_stride;
  void* ws;
};
constexpr int NORM_MAX_D = 16384;
size_t norm_ws_bytes(int type, int k, int n, int d, int gate_rows);
hipError_t norm_fwd(const NormArgs& a, hipStream_t s);
hipError_t norm_bwd(const NormArgs& a, hipStream_t s);

// Activations in 8 bits (ckpt.hip).
size_t kept_bytes(int64_t rows, int d);
hipError_t kept_pack(int type, int64_t rows, int d, const void* x, void* kept, hipStream_t s);
hipError_t kept_unpack(int type, int64_t rows, int d, const void* kept, void* x, hipStream_t s);
struct KeptGradArgs {
  int type, k, n, d, out;
  const void* kept;       // [k*n] rows of d in 8 bits
  const void* dy;         // [k*n][out]
  void* dw;               // [k] matrices [out][d], dstride elements apart
  int64_t dstride;
  void* ws;
};
size_t kept_grad_ws_bytes(const KeptGradArgs& a);  // 0: too large for a launch
hipError_t kept_grad(const KeptGradArgs& a, hipStream_t s);

}  // namespace cbk
