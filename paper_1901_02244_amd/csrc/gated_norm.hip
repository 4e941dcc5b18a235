// gated_norm.hip -- the seam between two blocks of a residual network in one
// pass: the norm after a block, its gate and residual scale, the addition to
// the stream, and the norm before the next block.  With r(v) =
// 1/sqrt(mean(v^2) + eps) over a row of d values and all arithmetic in fp32:
//
//   x' = x + s g (post o r(o))        y = pre x' r(x')
//
// g is one row of the gate for `gate_rows` rows of the learner.  Backward,
// from the stored x' (the statistics are taken again: the row is read anyway)
// with u = x' r(x'), w = o r(o):
//
//   a = pre dy          dx = dres + r(x') (a - u mean(a u))
//   b = s g dx post     do = r(o) (b - w mean(b w))
//   dpre = sum dy u     dpost = sum s g dx w     dg = sum s dx post w
//
// Bound by memory: a row is read once and lives in the registers of TPR
// threads, eight neighbouring columns at a time; the row sums go through lane
// shuffles (and LDS above one wave).  Every worker (TPR threads) walks
// consecutive rows, so that the gammas and the gate stay in registers, and in
// the backward pass the three column sums do too; each worker leaves one row
// of partial sums, which norm_sums adds in a fixed order.  Workers are laid
// out so that none has rows of two gate rows unless it has all rows of each.
// 16,384 rows of 4096, bf16: forward 104 us (5.2 TB/s of the four tensors that
// it moves; 129 us a call with the 8-bit form of y, where packing y in a call
// of its own takes 33 more), backward 174 us (4.6 TB/s of six) and 9 us for the
// column sums.  8192 rows of 4096, fp32: 110 and 169 us a call (4.9 and 4.8
// TB/s).  Two sizes stay far from that: some thousand rows, where every worker
// has one row and its partial sums are as much again (2 x 1000 x 1001, fp16:
// 13 and 6 us, the tensors alone would take 6), and workers of 1024 threads.
#include "kept.hpp"

#include <algorithm>
#include <type_traits>

namespace cbk {
namespace {

// Workers of a learner: `per` for each of `spans` spans of `rows` rows (a
// gate row's, or several whole ones'), each taking `each` rows.
struct Split {
  int span, spans, per, each;
  __host__ __device__ int workers() const { return spans * per; }
};

// The shape of a worker for rows of d: TPR threads of U * 8 columns.  Of the
// 16-bit types a thread takes two eights from 512 columns on: the backward
// kernel's registers allow two waves a SIMD either way, and twice as much is
// in flight; of fp32, which would spill, only above 8192.  1024 threads leave a
// lane 128 registers, which the backward passes: fp32 spills 41 (d a multiple
// of 8) to 74 registers from 4097 columns on, 405 to 572 above 8192, fp16
// there 209 to 276 and bf16 349 to 423 (4096 rows, backward: fp32 of 8192
// columns 366 us, 2.2 TB/s; of 16,384 columns fp32 1520, fp16 965 and bf16 1185
// us, 0.7 to 1.1 TB/s).
struct Shape {
  int tpr, u;
};
Shape shape_of(int type, int d) {
  if (d <= 512) return {d <= 64 ? 8 : d <= 128 ? 16 : d <= 256 ? 32 : 64, 1};
  const int eights = (d + 7) / 8;
  for (int tpr = 64; tpr < 1024; tpr *= 2)
    if (eights <= tpr * (type == LM_F32 ? 1 : 2)) return {tpr, type == LM_F32 ? 1 : 2};
  return {1024, eights <= 1024 ? 1 : 2};
}
constexpr int threads_of(int tpr) { return tpr < 128 ? 256 : tpr; }

// Forward: 1024 threads for every CU.  Backward: 512, the two waves a SIMD
// that its registers let be resident; and up to four rows a worker, so that
// the partial sums stay a small part of what is read, as long as each SIMD has
// a wave (4096 x 1024, bf16: 22.4 us against 24.9 with two rows; 2 x 1000 x
// 1001, fp16: 22.7 with one row against 29.6 with four on half the SIMDs).
Split split_rows(int type, int k, int n, int d, int gate_rows, bool backward) {
  const int per_learner = std::max(1, 256 * 256 / shape_of(type, d).tpr / k);
  const int target = per_learner * (backward ? 2 : 4);
  const int least = backward ? std::clamp(n / per_learner, 1, 4) : 1;
  const int each = std::max(least, (n + target - 1) / target);
  Split s;
  if (gate_rows <= each) {
    s.span = (each + gate_rows - 1) / gate_rows * gate_rows;
    s.per = 1;
  } else {
    s.span = std::min(gate_rows, n);
    s.per = (s.span + each - 1) / each;
  }
  s.spans = (n + s.span - 1) / s.span;
  s.each = (s.span + s.per - 1) / s.per;
  return s;
}

struct Dev {
  NormArgs a;
  Split s;
  float* part;    // [k][workers][3][d] partial sums of dpre, dpost, dgate
};

// Sums over a worker's threads, to all of them.  A wave that is ahead may be
// at its next call while another still reads the sums of this one, but not two
// calls ahead, for the barrier between: two buffers in turn need no second one.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*both)[TPR / 64 + 1][3], int& turn) {
  constexpr int LANES = TPR < 64 ? TPR : 64;
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], o);
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6;
    turn ^= 1;
    float(*lds)[3] = both[turn];
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[wave][i] = v[i];
    __syncthreads();
    constexpr int W = TPR / 64;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = lds[threadIdx.x % W][i];
#pragma unroll
      for (int o = W / 2; o; o >>= 1) v[i] += __shfl_xor(v[i], o);
    }
  }
}

template <int U>
using Row = float[U][8];

// Keeps x' an fp32 value until it is stored: the compiler may fold the
// addition and the rounding to fp16 into one instruction with one rounding,
// and the stored x' would then differ from its fp32 sum's in a last place (one
// in some 25,000), by how the code around it was compiled.
template <class T>
__device__ __forceinline__ void stay_f32(float (&x)[8]) {
  if constexpr (std::is_same_v<T, _Float16>) {
#pragma unroll
    for (int i = 0; i < 8; ++i) asm("" : "+v"(x[i]));
  }
}

template <int TPR, int U, bool WHOLE, class T>
__device__ __forceinline__ void load_row(const T* row, int t, int d, Row<U>& x) {
#pragma unroll
  for (int u = 0; u < U; ++u) load8<T, WHOLE>(row, (u * TPR + t) * 8, d, x[u]);
}
template <int U>
__device__ __forceinline__ void fill_row(Row<U>& x, float v) {
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[u][i] = v;
}
// gamma of this learner, or ones
template <int TPR, int U, bool WHOLE>
__device__ __forceinline__ void load_gamma(const float* g, int64_t stride, int j, int t, int d,
                                           Row<U>& x) {
  fill_row<U>(x, 1.f);
  if (g) load_row<TPR, U, WHOLE, float>(g + j * stride, t, d, x);
}
// A row as it lies in memory (zeros without one), to be converted where it is
// used: half the registers, for 16-bit types, of the floats.
template <class T, int U>
struct RawRow {
  Raw8<T> u[U];
};
template <int TPR, int U, bool WHOLE, class T>
__device__ __forceinline__ void load_raw(const void* base, int64_t at, int t, int d,
                                         RawRow<T, U>& x) {
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (base)
      x.u[u] = load_raw8<T, WHOLE>((const T*)base + at, (u * TPR + t) * 8, d);
    else
      x.u[u] = Raw8<T>{};
  }
}

// The rows of this worker: false if it has none.
template <int TPR>
__device__ __forceinline__ bool my_rows(const Dev& v, int& worker, int& r0, int& r1) {
  worker = blockIdx.x * (threads_of(TPR) / TPR) + threadIdx.x / TPR;
  if (worker >= v.s.workers()) return false;
  const int span = worker / v.s.per, part = worker % v.s.per;
  r0 = span * v.s.span + part * v.s.each;
  r1 = min(min(r0 + v.s.each, (span + 1) * v.s.span), v.a.n);
  return true;
}

template <class T, int TPR, int U, bool WHOLE>
__global__ __launch_bounds__(threads_of(TPR)) void norm_forward(Dev v) {
  const NormArgs& a = v.a;
  const int j = blockIdx.y, t = threadIdx.x % TPR, d = a.d;
  __shared__ float lds[2][TPR / 64 + 1][3];
  int turn = 0;
  int worker, r0, r1;
  if (!my_rows<TPR>(v, worker, r0, r1)) return;
  Row<U> post, pre, gate;
  load_gamma<TPR, U, WHOLE>(a.post, a.post_stride, j, t, d, post);
  load_gamma<TPR, U, WHOLE>(a.pre, a.pre_stride, j, t, d, pre);
  fill_row<U>(gate, 1.f);
  const int groups = (a.n + a.gate_rows - 1) / a.gate_rows;
  int group = -1;
  const float inv_d = 1.f / d;
  for (int r = r0; r < r1; ++r) {
    const int64_t at = ((int64_t)j * a.n + r) * d;
    Row<U> x;
    load_row<TPR, U, WHOLE>((const T*)a.x + at, t, d, x);
    if (a.block) {
      Row<U> o;
      load_row<TPR, U, WHOLE>((const T*)a.block + at, t, d, o);
      if (a.gate && group != r / a.gate_rows) {
        group = r / a.gate_rows;
        load_row<TPR, U, WHOLE>((const T*)a.gate + ((int64_t)j * groups + group) * d, t, d, gate);
      }
      float ro = 1.f;
      if (a.post) {
        float s[1] = {0.f};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < 8; ++i) s[0] += o[u][i] * o[u][i];
        row_sums<TPR, 1>(s, lds, turn);
        ro = 1.f / sqrtf(s[0] * inv_d + a.eps);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[u][i] += a.res_scale * gate[u][i] * (post[u][i] * (o[u][i] * ro));
        stay_f32<T>(x[u]);
        store8<T, WHOLE>((T*)a.x_out + at, (u * TPR + t) * 8, d, x[u]);
      }
    }
    if (!a.pre) continue;
    float s[1] = {0.f};
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += x[u][i] * x[u][i];
    row_sums<TPR, 1>(s, lds, turn);
    const float rx = 1.f / sqrtf(s[0] * inv_d + a.eps);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = (u * TPR + t) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[u][i] = pre[u][i] * (x[u][i] * rx);
      store8<T, WHOLE>((T*)a.y + at, c, d, x[u]);
      if (a.y_kept) {
        // the 8-bit form of y as stored: four lanes hold a group
        const int64_t dp = kept_dp(d), row = (int64_t)j * a.n + r;
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[u][i] = c + i < d ? to_f32((T)x[u][i]) : 0.f;
          most = max(most, abs_bits(x[u][i]));
        }
        most = max(most, (uint32_t)__shfl_xor((int)most, 1));
        most = max(most, (uint32_t)__shfl_xor((int)most, 2));
        const int byte = kept_byte<T>(most);
        if (c < dp) {
          *(uint64_t*)((char*)a.y_kept + row * dp + c) = kept_pack8<T>(x[u], byte);
          if ((t & 3) == 0)
            ((uint8_t*)a.y_kept)[(int64_t)a.k * a.n * dp + row * (dp / 32) + c / 32] = byte;
        }
      }
    }
  }
}

template <class T, int TPR, int U, bool WHOLE>
__global__ __launch_bounds__(threads_of(TPR), TPR > 512 ? 4 : 2) void norm_backward(Dev v) {
  const NormArgs& a = v.a;
  const int j = blockIdx.y, t = threadIdx.x % TPR, d = a.d;
  __shared__ float lds[2][TPR / 64 + 1][3];
  int turn = 0;
  int worker, r0, r1;
  if (!my_rows<TPR>(v, worker, r0, r1)) return;
  Row<U> post, pre, gate, dpre, dpost, dgate;
  load_gamma<TPR, U, WHOLE>(a.post, a.post_stride, j, t, d, post);
  load_gamma<TPR, U, WHOLE>(a.pre, a.pre_stride, j, t, d, pre);
  fill_row<U>(gate, 1.f);
  fill_row<U>(dpre, 0.f);
  fill_row<U>(dpost, 0.f);
  fill_row<U>(dgate, 0.f);
  const int groups = (a.n + a.gate_rows - 1) / a.gate_rows;
  int group = -1;
  const float inv_d = 1.f / d;
  // The next row's loads are in flight while a row is worked on.
  struct Rows {
    RawRow<T, U> x, dy, dres, o;
  };
  Rows next;
  auto fetch = [&](int r) {
    const int64_t at = ((int64_t)j * a.n + r) * d;
    load_raw<TPR, U, WHOLE, T>(a.x, at, t, d, next.x);
    load_raw<TPR, U, WHOLE, T>(a.dy, at, t, d, next.dy);
    load_raw<TPR, U, WHOLE, T>(a.dres, at, t, d, next.dres);
    load_raw<TPR, U, WHOLE, T>(a.block, at, t, d, next.o);
  };
  if (r0 < r1) fetch(r0);
  for (int r = r0; r < r1; ++r) {
    const int64_t at = ((int64_t)j * a.n + r) * d;
    Row<U> x, dy, dx, o;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[u][i] = next.x.u[u].at(i);
        dy[u][i] = next.dy.u[u].at(i);
        dx[u][i] = next.dres.u[u].at(i);
        o[u][i] = next.o.u[u].at(i);
      }
    if (r + 1 < r1) fetch(r + 1);
    if (a.gate && group != r / a.gate_rows) {
      group = r / a.gate_rows;
      load_row<TPR, U, WHOLE>((const T*)a.gate + ((int64_t)j * groups + group) * d, t, d, gate);
    }
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[0] += x[u][i] * x[u][i];
        s[1] += pre[u][i] * dy[u][i] * x[u][i];
        s[2] += o[u][i] * o[u][i];
      }
    row_sums<TPR, 3>(s, lds, turn);
    if (a.pre) {
      const float rx = 1.f / sqrtf(s[0] * inv_d + a.eps);
      const float m = s[1] * rx * inv_d;  // mean(a u)
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float unit = x[u][i] * rx;
          dx[u][i] += rx * (pre[u][i] * dy[u][i] - unit * m);
          dpre[u][i] += dy[u][i] * unit;
        }
    }
    if (a.dx)
#pragma unroll
      for (int u = 0; u < U; ++u)
        store8<T, WHOLE>((T*)a.dx + at, (u * TPR + t) * 8, d, dx[u]);
    if (!a.block) continue;
    const float ro = a.post ? 1.f / sqrtf(s[2] * inv_d + a.eps) : 1.f;
    float q[1] = {0.f};
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float w = o[u][i] * ro, sdx = a.res_scale * dx[u][i], b = gate[u][i] * sdx;
        dgate[u][i] += sdx * post[u][i] * w;
        dpost[u][i] += b * w;
        dx[u][i] = b * post[u][i];
        o[u][i] = w;
        q[0] += dx[u][i] * w;
      }
    if (a.post) {
      row_sums<TPR, 1>(q, lds, turn);
      q[0] *= inv_d;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) dx[u][i] = ro * (dx[u][i] - o[u][i] * q[0]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      store8<T, WHOLE>((T*)a.dblock + at, (u * TPR + t) * 8, d, dx[u]);
    // a gate row whose rows are all this worker's is done with its last one
    if (a.gate && v.s.per == 1 && ((r + 1) % a.gate_rows == 0 || r + 1 == a.n)) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        store8<T, WHOLE>((T*)a.dgate + ((int64_t)j * groups + group) * d, (u * TPR + t) * 8, d,
                  dgate[u]);
      fill_row<U>(dgate, 0.f);
    }
  }
  float* p = v.part + ((int64_t)j * v.s.workers() + worker) * 3 * d;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = (u * TPR + t) * 8;
    if (a.pre) store8<float, WHOLE>(p, c, d, dpre[u]);
    if (a.post) store8<float, WHOLE>(p + d, c, d, dpost[u]);
    if (a.gate && v.s.per > 1) store8<float, WHOLE>(p + 2 * d, c, d, dgate[u]);
  }
}

// Column sums over the workers' partial rows: 32 columns a workgroup, 32
// threads a column.  blockIdx.y: 0 dpre, 1 dpost, 2 + g the gate row g.
template <class T>
__global__ __launch_bounds__(1024) void norm_sums(Dev v) {
  const NormArgs& a = v.a;
  const int j = blockIdx.z, what = blockIdx.y, x = threadIdx.x & 31, sl = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + x, d = a.d;
  if ((what == 0 && !a.pre) || (what == 1 && !a.post)) return;
  const int W = v.s.workers();
  const int w0 = what < 2 ? 0 : (what - 2) * v.s.per, w1 = what < 2 ? W : w0 + v.s.per;
  const float* p = v.part + ((int64_t)j * W * 3 + min(what, 2)) * d + c;
  float s = 0.f;
  if (c < d) {
#pragma unroll 4
    for (int w = w0 + sl; w < w1; w += 32) s += p[(int64_t)w * 3 * d];
  }
  __shared__ float sum[32][33];
  sum[sl][x] = s;
  __syncthreads();
  // a column's 32 sums to 32 neighbouring lanes
  s = sum[x][sl];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor(s, o);
  const int col = blockIdx.x * 32 + sl;
  if (x || col >= d) return;
  if (what == 0)
    a.dpre[j * a.dpre_stride + col] = s;
  else if (what == 1)
    a.dpost[j * a.dpost_stride + col] = s;
  else
    ((T*)a.dgate)[((int64_t)j * v.s.spans + what - 2) * d + col] = (T)s;
}

template <class T, int TPR, int U>
void launch(const Dev& v, bool backward, hipStream_t s) {
  const int per = threads_of(TPR) / TPR;
  const dim3 grid((v.s.workers() + per - 1) / per, v.a.k), block(threads_of(TPR));
  const bool whole = v.a.d % 8 == 0;
  if (backward)
    klaunch(whole ? norm_backward<T, TPR, U, true> : norm_backward<T, TPR, U, false>, grid, block,
            0, s, v);
  else
    klaunch(whole ? norm_forward<T, TPR, U, true> : norm_forward<T, TPR, U, false>, grid, block, 0,
            s, v);
}

template <class T>
hipError_t run(const Dev& v, bool backward, hipStream_t s) {
  const int d = v.a.d;
  const Shape sh = shape_of(v.a.type, d);
  constexpr int U = sizeof(T) == 4 ? 1 : 2;
  if (sh.tpr == 8) launch<T, 8, 1>(v, backward, s);
  else if (sh.tpr == 16) launch<T, 16, 1>(v, backward, s);
  else if (sh.tpr == 32) launch<T, 32, 1>(v, backward, s);
  else if (sh.tpr == 64 && sh.u == 1) launch<T, 64, 1>(v, backward, s);
  else if (sh.tpr == 64) launch<T, 64, U>(v, backward, s);
  else if (sh.tpr == 128) launch<T, 128, U>(v, backward, s);
  else if (sh.tpr == 256) launch<T, 256, U>(v, backward, s);
  else if (sh.tpr == 512) launch<T, 512, U>(v, backward, s);
  else if (sizeof(T) == 4 && sh.u == 1) launch<T, 1024, sizeof(T) == 4 ? 1 : 2>(v, backward, s);
  else launch<T, 1024, 2>(v, backward, s);
  if (hipError_t e = hipGetLastError()) return e;
  if (!backward || (!v.a.pre && !v.a.post && !v.a.gate)) return hipSuccess;
  const int rows = 2 + (v.a.gate && v.s.per > 1 ? v.s.spans : 0);
  klaunch(norm_sums<T>, dim3((d + 31) / 32, rows, v.a.k), dim3(1024), 0, s, v);
  return hipGetLastError();
}

Dev dev_of(const NormArgs& a, bool backward) {
  Dev v;
  v.a = a;
  if (!a.gate) v.a.gate_rows = a.n;
  v.s = split_rows(a.type, a.k, a.n, a.d, v.a.gate_rows, backward);
  v.part = (float*)a.ws;
  return v;
}

hipError_t dispatch(const NormArgs& a, bool backward, hipStream_t s) {
  const Dev v = dev_of(a, backward);
  return a.type == LM_F32 ? run<float>(v, backward, s)
         : a.type == LM_F16 ? run<_Float16>(v, backward, s)
                            : run<__bf16>(v, backward, s);
}

}  // namespace

size_t norm_ws_bytes(int type, int k, int n, int d, int gate_rows) {
  return (size_t)k * split_rows(type, k, n, d, gate_rows, true).workers() * 3 * d * sizeof(float);
}
hipError_t norm_fwd(const NormArgs& a, hipStream_t s) { return dispatch(a, false, s); }
hipError_t norm_bwd(const NormArgs& a, hipStream_t s) { return dispatch(a, true, s); }

}  // namespace cbk
