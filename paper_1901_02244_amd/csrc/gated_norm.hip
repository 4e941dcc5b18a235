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
#include "kept.hpp"

#include <algorithm>

namespace cbk {
namespace {

// Workers of a learner: `per` for each of `spans` spans of `rows` rows (a
// gate row's, or several whole ones'), each taking `each` rows.
struct Split {
  int span, spans, per, each;
  __host__ __device__ int workers() const { return spans * per; }
};

// About 1024 workers in all: four workgroups for every CU where a worker is
// one, with few enough rows of partial sums.
Split split_rows(int k, int n, int gate_rows) {
  const int target = std::max(1, 1024 / k);
  const int each = std::max(1, (n + target - 1) / target);
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
  bool vec;
  float* part;    // [k][workers][3][d] partial sums of dpre, dpost, dgate
};

template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*lds)[N]) {
  constexpr int LANES = TPR < 64 ? TPR : 64;
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], o);
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[wave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < TPR / 64; ++w) v[i] += lds[w][i];
    }
  }
}

template <int U>
using Row = float[U][8];

template <int TPR, int U, class T>
__device__ __forceinline__ void load_row(const T* row, int t, int d, bool vec, Row<U>& x) {
#pragma unroll
  for (int u = 0; u < U; ++u) load8<T>(row, (u * TPR + t) * 8, d, vec, x[u]);
}
template <int U>
__device__ __forceinline__ void fill_row(Row<U>& x, float v) {
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[u][i] = v;
}
// gamma of this learner, or ones
template <int TPR, int U>
__device__ __forceinline__ void load_gamma(const float* g, int64_t stride, int j, int t, int d,
                                           Row<U>& x) {
  fill_row<U>(x, 1.f);
  const float* row = g + j * stride;
  if (g) load_row<TPR, U, float>(row, t, d, d % 8 == 0 && (uintptr_t)row % 16 == 0, x);
}

constexpr int threads_of(int tpr) { return tpr < 256 ? 256 : tpr; }

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

template <class T, int TPR, int U>
__global__ __launch_bounds__(threads_of(TPR)) void norm_forward(Dev v) {
  const NormArgs& a = v.a;
  const int j = blockIdx.y, t = threadIdx.x % TPR, d = a.d;
  __shared__ float lds[2][TPR / 64 + 1][1];
  int worker, r0, r1;
  if (!my_rows<TPR>(v, worker, r0, r1)) return;
  Row<U> post, pre, gate;
  load_gamma<TPR, U>(a.post, a.post_stride, j, t, d, post);
  load_gamma<TPR, U>(a.pre, a.pre_stride, j, t, d, pre);
  fill_row<U>(gate, 1.f);
  const int groups = (a.n + a.gate_rows - 1) / a.gate_rows;
  int group = -1;
  const float inv_d = 1.f / d;
  for (int r = r0; r < r1; ++r) {
    const int64_t at = ((int64_t)j * a.n + r) * d;
    Row<U> x;
    load_row<TPR, U>((const T*)a.x + at, t, d, v.vec, x);
    if (a.block) {
      Row<U> o;
      load_row<TPR, U>((const T*)a.block + at, t, d, v.vec, o);
      if (a.gate && group != r / a.gate_rows) {
        group = r / a.gate_rows;
        load_row<TPR, U>((const T*)a.gate + ((int64_t)j * groups + group) * d, t, d, v.vec, gate);
      }
      float ro = 1.f;
      if (a.post) {
        float s[1] = {0.f};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < 8; ++i) s[0] += o[u][i] * o[u][i];
        row_sums<TPR, 1>(s, lds[0]);
        ro = 1.f / sqrtf(s[0] * inv_d + a.eps);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[u][i] += a.res_scale * gate[u][i] * (post[u][i] * (o[u][i] * ro));
        store8<T>((T*)a.x_out + at, (u * TPR + t) * 8, d, v.vec, x[u]);
      }
    }
    if (!a.pre) continue;
    float s[1] = {0.f};
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += x[u][i] * x[u][i];
    row_sums<TPR, 1>(s, lds[1]);
    const float rx = 1.f / sqrtf(s[0] * inv_d + a.eps);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = (u * TPR + t) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[u][i] = pre[u][i] * (x[u][i] * rx);
      store8<T>((T*)a.y + at, c, d, v.vec, x[u]);
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

template <class T, int TPR, int U>
__global__ __launch_bounds__(threads_of(TPR)) void norm_backward(Dev v) {
  const NormArgs& a = v.a;
  const int j = blockIdx.y, t = threadIdx.x % TPR, d = a.d;
  __shared__ float lds_a[TPR / 64 + 1][3], lds_b[TPR / 64 + 1][1];
  int worker, r0, r1;
  if (!my_rows<TPR>(v, worker, r0, r1)) return;
  Row<U> post, pre, gate, dpre, dpost, dgate;
  load_gamma<TPR, U>(a.post, a.post_stride, j, t, d, post);
  load_gamma<TPR, U>(a.pre, a.pre_stride, j, t, d, pre);
  fill_row<U>(gate, 1.f);
  fill_row<U>(dpre, 0.f);
  fill_row<U>(dpost, 0.f);
  fill_row<U>(dgate, 0.f);
  const int groups = (a.n + a.gate_rows - 1) / a.gate_rows;
  int group = -1;
  const float inv_d = 1.f / d;
  for (int r = r0; r < r1; ++r) {
    const int64_t at = ((int64_t)j * a.n + r) * d;
    Row<U> x, dy, dx, o;
    fill_row<U>(dx, 0.f);
    fill_row<U>(dy, 0.f);
    fill_row<U>(o, 0.f);
    if (a.pre) {
      load_row<TPR, U>((const T*)a.x + at, t, d, v.vec, x);
      load_row<TPR, U>((const T*)a.dy + at, t, d, v.vec, dy);
    } else {
      fill_row<U>(x, 0.f);
    }
    if (a.block) load_row<TPR, U>((const T*)a.block + at, t, d, v.vec, o);
    if (a.dres) load_row<TPR, U>((const T*)a.dres + at, t, d, v.vec, dx);
    if (a.gate && group != r / a.gate_rows) {
      group = r / a.gate_rows;
      load_row<TPR, U>((const T*)a.gate + ((int64_t)j * groups + group) * d, t, d, v.vec, gate);
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
    row_sums<TPR, 3>(s, lds_a);
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
        store8<T>((T*)a.dx + at, (u * TPR + t) * 8, d, v.vec, dx[u]);
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
      row_sums<TPR, 1>(q, lds_b);
      q[0] *= inv_d;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) dx[u][i] = ro * (dx[u][i] - o[u][i] * q[0]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      store8<T>((T*)a.dblock + at, (u * TPR + t) * 8, d, v.vec, dx[u]);
    // a gate row whose rows are all this worker's is done with its last one
    if (a.gate && v.s.per == 1 && ((r + 1) % a.gate_rows == 0 || r + 1 == a.n)) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        store8<T>((T*)a.dgate + ((int64_t)j * groups + group) * d, (u * TPR + t) * 8, d, v.vec,
                  dgate[u]);
      fill_row<U>(dgate, 0.f);
    }
  }
  float* p = v.part + ((int64_t)j * v.s.workers() + worker) * 3 * d;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = (u * TPR + t) * 8;
    if (a.pre) store8<float>(p, c, d, d % 8 == 0, dpre[u]);
    if (a.post) store8<float>(p + d, c, d, d % 8 == 0, dpost[u]);
    if (a.gate && v.s.per > 1) store8<float>(p + 2 * d, c, d, d % 8 == 0, dgate[u]);
  }
}

// Column sums over the workers' partial rows: 32 columns a workgroup, eight
// threads a column.  blockIdx.y: 0 dpre, 1 dpost, 2 + g the gate row g.
template <class T>
__global__ __launch_bounds__(256) void norm_sums(Dev v) {
  const NormArgs& a = v.a;
  const int j = blockIdx.z, what = blockIdx.y, x = threadIdx.x & 31, sl = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + x, d = a.d;
  if ((what == 0 && !a.pre) || (what == 1 && !a.post)) return;
  const int W = v.s.workers();
  const int w0 = what < 2 ? 0 : (what - 2) * v.s.per, w1 = what < 2 ? W : w0 + v.s.per;
  const float* p = v.part + ((int64_t)j * W * 3 + min(what, 2)) * d + c;
  float s = 0.f;
  if (c < d)
    for (int w = w0 + sl; w < w1; w += 8) s += p[(int64_t)w * 3 * d];
  __shared__ float sum[8][32];
  sum[sl][x] = s;
  __syncthreads();
  if (sl || c >= d) return;
  for (int i = 1; i < 8; ++i) s += sum[i][x];
  if (what == 0)
    a.dpre[j * a.dpre_stride + c] = s;
  else if (what == 1)
    a.dpost[j * a.dpost_stride + c] = s;
  else
    ((T*)a.dgate)[((int64_t)j * v.s.spans + what - 2) * d + c] = (T)s;
}

template <class T, int TPR, int U>
void launch(const Dev& v, bool backward, hipStream_t s) {
  const int per = threads_of(TPR) / TPR;
  const dim3 grid((v.s.workers() + per - 1) / per, v.a.k);
  if (backward)
    klaunch(norm_backward<T, TPR, U>, grid, dim3(threads_of(TPR)), 0, s, v);
  else
    klaunch(norm_forward<T, TPR, U>, grid, dim3(threads_of(TPR)), 0, s, v);
}

// TPR threads of U*8 columns reach d.
template <class T>
hipError_t run(const Dev& v, bool backward, hipStream_t s) {
  const int d = v.a.d;
  if (d <= 64) launch<T, 8, 1>(v, backward, s);
  else if (d <= 128) launch<T, 16, 1>(v, backward, s);
  else if (d <= 256) launch<T, 32, 1>(v, backward, s);
  else if (d <= 512) launch<T, 64, 1>(v, backward, s);
  else if (d <= 1024) launch<T, 64, 2>(v, backward, s);
  else if (d <= 2048) launch<T, 256, 1>(v, backward, s);
  else if (d <= 4096) launch<T, 256, 2>(v, backward, s);
  else if (d <= 8192) launch<T, 512, 2>(v, backward, s);
  else launch<T, 1024, 2>(v, backward, s);
  if (hipError_t e = hipGetLastError()) return e;
  if (!backward || (!v.a.pre && !v.a.post && !v.a.gate)) return hipSuccess;
  const int rows = 2 + (v.a.gate && v.s.per > 1 ? v.s.spans : 0);
  klaunch(norm_sums<T>, dim3((d + 31) / 32, rows, v.a.k), dim3(256), 0, s, v);
  return hipGetLastError();
}

bool on_16(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if ((uintptr_t)p % 16) return false;
  return true;
}

Dev dev_of(const NormArgs& a) {
  Dev v;
  v.a = a;
  if (!a.gate) v.a.gate_rows = a.n;
  v.s = split_rows(a.k, a.n, v.a.gate_rows);
  v.vec = a.d % 8 == 0 && on_16({a.x, a.block, a.gate, a.x_out, a.y, a.dy, a.dres, a.dx, a.dblock,
                                 a.dgate});
  v.part = (float*)a.ws;
  return v;
}

hipError_t dispatch(const NormArgs& a, bool backward, hipStream_t s) {
  const Dev v = dev_of(a);
  return a.type == LM_F32 ? run<float>(v, backward, s)
         : a.type == LM_F16 ? run<_Float16>(v, backward, s)
                            : run<__bf16>(v, backward, s);
}

}  // namespace

size_t norm_ws_bytes(int k, int n, int d, int gate_rows) {
  return (size_t)k * split_rows(k, n, gate_rows).workers() * 3 * d * sizeof(float);
}
hipError_t norm_fwd(const NormArgs& a, hipStream_t s) { return dispatch(a, false, s); }
hipError_t norm_bwd(const NormArgs& a, hipStream_t s) { return dispatch(a, true, s); }

}  // namespace cbk
