// vocab_xent.hip -- softmax cross-entropy of a projection onto a large
// vocabulary, and its gradient, without the logits ever being kept.
//
// For the counted rows r (label not `ignore`) of a learner, C of them:
//   l[r][v] = sum_d h[r][d] W[v][d]        lse[r] = log sum_v exp l[r][v]
//   loss    = 1/C sum_r (lse[r] - l[r][y_r])
//   g[r][v] = exp(l[r][v] - lse[r]) - [v = y_r]
//   dh[r]   = s/C sum_v g[r][v] W[v]       dW[v] = s/C sum_r g[r][v] h[r]
//
// Forward: the counted rows are gathered (xent_rows), so that ignored rows
// cost nothing and whatever they hold stays out of the products; a matrix
// product with vocabulary tiles as P and rows as Q leaves a row's logits of
// one tile in few lanes, which reduce them to (max, sum of exponentials) per
// wave's share of the tile (xent_logits); xent_join joins those and xent_mean
// takes the mean.  Backward: for each piece of the vocabulary the logits are
// computed again, g of the piece is stored in the input type, and two
// products add its share of dh (fp32 sums across pieces) and write its rows
// of dW; xent_dh scales and scatters dh.  The sums run in a fixed order: no
// atomics.
//
// g is stored times 2^14 in fp16, so that probabilities down to 2^-28 are
// normal numbers and -1 is still in range; the scale is taken out, with s/C,
// from the fp32 sums.  That store is the only rounding before the results'
// own.
#include "lm.hpp"
#include "lm_tile.hpp"

#include <algorithm>

namespace cbk {
namespace {

constexpr float NEG_INF = -__builtin_inff();

template <class T>
constexpr float g_scale() {
  return __is_same(T, _Float16) ? 16384.f : 1.f;
}

__host__ __device__ constexpr int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// Places in the workspace, in bytes.
struct Layout {
  int cap;       // rows of a learner, up to a multiple of 64
  int dp;        // columns of the gathered rows, up to a multiple of 128 bytes
  int parts;     // vocabulary shares with a (max, sum) of their own
  int piece;     // vocabulary rows of one piece of the backward pass
  int splits;    // shares of a piece's vocabulary that sum dh on their own
  bool copy_w;
  size_t cnt, pos, row, lab, hc, wc, part, plog, rloss, g, dh, total;
};

// Tile shapes: BIG from 256 workgroups of it on, else MID; THIN for up to
// 32 rows of a learner.
enum { BIG, MID, THIN };

int64_t tiles(int64_t a, int64_t b, int ba, int bb) { return up(a, ba) / ba * (up(b, bb) / bb); }

int shape_of(int k, int64_t p, int64_t q) {
  if (q <= 32) return THIN;
  return k * tiles(p, q, 256, 256) >= 256 ? BIG : MID;
}
int bp_of(int shape) { return shape == MID ? 128 : 256; }
int bq_of(int shape) { return shape == BIG ? 256 : shape == MID ? 128 : 32; }
int wp_of(int shape) { return shape == THIN ? 4 : 2; }

Layout layout(const XentArgs& a, bool backward) {
  const int k = a.k, n = a.n, d = a.d, v = a.v, sz = lm_size(a.type);
  Layout l;
  l.cap = (int)up(n, 64);
  l.dp = (int)up(d, 128 / sz);
  // the rows of W are read 16 bytes at a time
  l.copy_w = (uintptr_t)a.w % 16 || (int64_t)d * sz % 16 || (k > 1 && a.pstride * sz % 16);
  const int64_t rows = (int64_t)k * l.cap;
  const int sh = shape_of(k, v, n);
  l.parts = (int)(up(v, bp_of(sh)) / bp_of(sh) * wp_of(sh));
  // A piece's g takes up to 256 MB, which the memory-side cache holds between
  // the products, but at least 4096 words, so that reading and writing the
  // fp32 sums of dh once a piece stays small beside the products.
  const int64_t fit = (int64_t(256) << 20) / (rows * sz) / 256 * 256;
  l.piece = (int)std::min<int64_t>(up(v, 256), std::max<int64_t>(4096, fit));
  const int sd = shape_of(k, d, n);
  const int64_t td = k * tiles(d, n, bp_of(sd), bq_of(sd));
  const int64_t steps = up(std::min(l.piece, v), 128 / sz) / (128 / sz);
  l.splits = (int)std::max<int64_t>(1, std::min<int64_t>(512 / std::max<int64_t>(td, 1), steps / 8));
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)up(std::max<int64_t>(bytes, 1), 256);
    return here;
  };
  l.cnt = take(k * 4);
  l.pos = take((int64_t)k * n * 4);
  l.row = take(rows * 4);
  l.lab = take(rows * 4);
  l.hc = take(rows * l.dp * sz);
  l.wc = l.copy_w ? take((int64_t)k * v * l.dp * sz) : 0;
  l.part = l.plog = l.rloss = l.g = l.dh = 0;
  if (backward) {
    l.g = take(rows * l.piece * sz);
    l.dh = take((int64_t)l.splits * rows * l.dp * 4);
  } else {
    l.part = take((int64_t)l.parts * rows * 8);
    l.plog = take(rows * 4);
    l.rloss = take((int64_t)k * n * 4);
  }
  l.total = at;
  return l;
}

// --- the counted rows ----------------------------------------------------------

constexpr int ROWS_PER_BLOCK = 16;

struct RowsArgs {
  const void* h;
  int64_t ldh;
  const int32_t* labels;
  int ignore, n, d, dp, cap;
  int *cnt, *pos, *row, *lab;
  void* hc;
};

// Gathers the counted rows of a learner, in order: every workgroup counts the
// labels before its own 16 rows (n/16 workgroups reading up to n labels from
// L2 cost less than a second launch), then copies its rows, padded with zeros
// to dp columns.  pos[r] is the gathered place of row r or -1, row[] and
// lab[] its inverse and the labels there.
template <class T, bool VEC>
__global__ __launch_bounds__(256) void xent_rows(RowsArgs a) {
  const int j = blockIdx.y, r0 = blockIdx.x * ROWS_PER_BLOCK, tid = threadIdx.x;
  const int32_t* lab = a.labels + (int64_t)j * a.n;
  __shared__ int wave_sum[4], place[ROWS_PER_BLOCK];
  int c = 0;
  for (int i = tid; i < r0; i += 256) c += lab[i] != a.ignore;
#pragma unroll
  for (int o = 32; o; o >>= 1) c += __shfl_xor(c, o);
  if ((tid & 63) == 0) wave_sum[tid >> 6] = c;
  __syncthreads();
  const int before = wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
  if (tid < 64) {
    const int r = r0 + tid;
    const bool mine = tid < ROWS_PER_BLOCK && r < a.n;
    const int y = mine ? lab[r] : a.ignore;
    const uint64_t m = __ballot(y != a.ignore);
    const int p = before + __popcll(m & ((1ull << tid) - 1));
    if (mine) {
      const bool in = y != a.ignore;
      place[tid] = in ? p : -1;
      a.pos[(int64_t)j * a.n + r] = in ? p : -1;
      if (in) {
        a.row[(int64_t)j * a.cap + p] = r;
        a.lab[(int64_t)j * a.cap + p] = y;
      }
    }
    if (tid == 0 && r0 + ROWS_PER_BLOCK >= a.n) a.cnt[j] = before + __popcll(m);
  }
  __syncthreads();
  const int lane = tid & 63;
  for (int i = tid >> 6; i < ROWS_PER_BLOCK && r0 + i < a.n; i += 4) {
    const int p = place[i];
    if (p < 0) continue;
    const T* src = (const T*)a.h + ((int64_t)j * a.n + r0 + i) * a.ldh;
    T* dst = (T*)a.hc + ((int64_t)j * a.cap + p) * a.dp;
    if constexpr (VEC) {
      constexpr int E = 16 / sizeof(T);
      for (int x = lane * E; x < a.dp; x += 64 * E) {
        i32x4 v = {0, 0, 0, 0};
        if (x < a.d) v = *(const i32x4*)(src + x);
        *(i32x4*)(dst + x) = v;
      }
    } else {
      for (int x = lane; x < a.dp; x += 64) dst[x] = x < a.d ? src[x] : (T)0.f;
    }
  }
}

// A copy of W whose rows start on 16 bytes, for widths or places whose own
// rows do not: [k][v][dp], padded with zeros.
template <class T>
__global__ __launch_bounds__(256) void xent_copy_w(const T* w, int64_t pstride, int v, int d,
                                                   int dp, T* wc) {
  const int j = blockIdx.y, lane = threadIdx.x & 63;
  for (int r = blockIdx.x * 4 + (threadIdx.x >> 6); r < v; r += gridDim.x * 4) {
    const T* src = w + j * pstride + (int64_t)r * d;
    T* dst = wc + ((int64_t)j * v + r) * dp;
    for (int x = lane; x < dp; x += 64) dst[x] = x < d ? src[x] : (T)0.f;
  }
}

// --- logits --------------------------------------------------------------------

struct LogitArgs {
  const void* w;    // replica 0's first row of the vocabulary range
  int64_t ldw, pstride;
  int d;            // width of W's rows that holds values
  int v0, vn;       // the vocabulary range [v0, v0 + vn)
  const void* hc;
  int dp, cap;
  const int *cnt, *lab, *row;
  // forward
  float2* part;     // [k][parts][cap]
  float* plog;      // [k][cap]
  int parts;
  // backward
  const float* lse; // [k*n]
  int n;
  void* g;          // [k][cap][ldg]
  int ldg;
};

template <class TL, bool BACKWARD>
__global__ __launch_bounds__(TL::THREADS) void xent_logits(LogitArgs a) {
  using T = typename TL::T;
  extern __shared__ __align__(16) char lds[];
  const int j = blockIdx.y, cnt = a.cnt[j];
  int tp, tq;
  tile_of<8>(blockIdx.x, (a.vn + TL::BP - 1) / TL::BP, gridDim.x / ((a.vn + TL::BP - 1) / TL::BP),
             tp, tq);
  const int p0 = tp * TL::BP, q0 = tq * TL::BQ;
  if (q0 >= cnt) return;
  const Operand<T> W{(const T*)a.w + j * a.pstride, a.ldw, a.vn, a.d};
  const Operand<T> H{(const T*)a.hc + (int64_t)j * a.cap * a.dp, a.dp, cnt, a.d};
  typename TL::Acc acc;
  TL::product(W, H, p0, q0, 0, a.d, lds, acc);

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = (wave / TL::WQ) * TL::SP, wq = (wave % TL::WQ) * TL::SQ;
  const int pv = a.vn - p0 - wp;  // words of this wave's share that exist
#pragma unroll
  for (int b = 0; b < TL::TQ; ++b) {
    const int q = q0 + wq + TL::col_of(b, lane);
    const bool in = q < cnt;
    const int64_t at = (int64_t)j * a.cap + q;
    const int y = in ? a.lab[at] - a.v0 - p0 - wp : -1;  // label, from the wave's first word
    if constexpr (!BACKWARD) {
      float m = NEG_INF;
#pragma unroll
      for (int t = 0; t < TL::TP; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int p = t * 16 + 4 * (lane >> 4) + i;
          if (p >= pv) acc[t][b][i] = NEG_INF;
          m = fmaxf(m, acc[t][b][i]);
          if (p == y && p < pv) a.plog[at] = acc[t][b][i];
        }
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      const float from = m == NEG_INF ? 0.f : m;
      float e = 0.f;
#pragma unroll
      for (int t = 0; t < TL::TP; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) e += __expf(acc[t][b][i] - from);
      e += __shfl_xor(e, 16);
      e += __shfl_xor(e, 32);
      if (in && lane < 16)
        a.part[((int64_t)j * a.parts + tp * TL::WP + wave / TL::WQ) * a.cap + q] = {m, e};
    } else {
      const float lse = in ? a.lse[(int64_t)j * a.n + a.row[at]] : 0.f;
      T* g = (T*)a.g + at * a.ldg + p0 + wp;
#pragma unroll
      for (int t = 0; t < TL::TP; ++t) {
        const int p = t * 16 + 4 * (lane >> 4);
        T out[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = __expf(acc[t][b][i] - lse) - (p + i == y ? 1.f : 0.f);
          if (p + i >= pv) x = 0.f;
          out[i] = from_f32<T>(x * g_scale<T>());
        }
        if (in && p0 + wp + p < a.ldg) {
          if constexpr (sizeof(T) == 2)
            *(uint64_t*)(g + p) = *(const uint64_t*)out;
          else
            *(f32x4*)(g + p) = *(const f32x4*)out;
        }
      }
    }
  }
}

// Joins the (max, sum) pairs of a row: 256/R threads a row, R rows a
// workgroup.  Ignored rows get lse 0 and no loss.
template <int R>
__global__ __launch_bounds__(256) void xent_join(const int* pos, const float2* part, int parts,
                                                 int cap, const float* plog, const int* lab, int n,
                                                 int v, float* lse, float* rloss) {
  constexpr int S = 256 / R;
  const int j = blockIdx.y, x = threadIdx.x % R, s = threadIdx.x / R;
  const int r = blockIdx.x * R + x;
  __shared__ float ms[S][R], es[S][R];
  const int p = r < n ? pos[(int64_t)j * n + r] : -1;
  float m = NEG_INF, e = 0.f;
  if (p >= 0) {
    const float2* at = part + (int64_t)j * parts * cap + p;
    for (int i = s; i < parts; i += S) {
      const float2 o = at[(int64_t)i * cap];
      const float mm = fmaxf(m, o.x), from = mm == NEG_INF ? 0.f : mm;
      e = e * __expf(m - from) + o.y * __expf(o.x - from);
      m = mm;
    }
  }
  ms[s][x] = m;
  es[s][x] = e;
  __syncthreads();
  if (s != 0 || r >= n) return;
  float out = 0.f, loss = 0.f;
  if (p >= 0) {
    for (int i = 1; i < S; ++i) m = fmaxf(m, ms[i][x]);
    const float from = m == NEG_INF ? 0.f : m;
    e = 0.f;
    for (int i = 0; i < S; ++i) e += es[i][x] * __expf(ms[i][x] - from);
    out = from + logf(e);
    const int y = lab[(int64_t)j * cap + p];
    loss = y >= 0 && y < v ? out - plog[(int64_t)j * cap + p] : __builtin_nanf("");
  }
  lse[(int64_t)j * n + r] = out;
  rloss[(int64_t)j * n + r] = loss;
}

// A learner's mean loss over its counted rows (0 if none counts), summed in
// fp64 in a fixed order.
__global__ __launch_bounds__(256) void xent_mean(const float* rloss, const int* cnt, int n,
                                                 float* loss) {
  const int j = blockIdx.x, tid = threadIdx.x;
  double t = 0.0;
  for (int i = tid; i < n; i += 256) t += rloss[(int64_t)j * n + i];
  __shared__ double sum[256];
  sum[tid] = t;
  __syncthreads();
  for (int o = 128; o; o >>= 1) {
    if (tid < o) sum[tid] += sum[tid + o];
    __syncthreads();
  }
  if (tid == 0) loss[j] = (float)(sum[0] / max(cnt[j], 1));
}

// --- gradients -------------------------------------------------------------------

struct DhArgs {
  const void* w;    // the piece's first row
  int64_t ldw, pstride;
  int d, vn;
  const void* g;
  int ldg, cap;
  const int* cnt;
  float* dh;        // [splits][k][cap][dp] sums
  int dp, splits, span;  // a split takes `span` words
  int64_t split_stride;
  int add;
};

// dh sums: P = W in col form (p = column), Q = g in row form (q = row).
template <class TL>
__global__ __launch_bounds__(TL::THREADS) void xent_dh_sums(DhArgs a) {
  using T = typename TL::T;
  extern __shared__ __align__(16) char lds[];
  const int j = blockIdx.y, cnt = a.cnt[j], s = blockIdx.z;
  const int np = (a.d + TL::BP - 1) / TL::BP;
  int tp, tq;
  tile_of<8>(blockIdx.x, np, gridDim.x / np, tp, tq);
  const int p0 = tp * TL::BP, q0 = tq * TL::BQ;
  if (q0 >= cnt) return;
  const Operand<T> W{(const T*)a.w + j * a.pstride, a.ldw, a.d, a.vn};
  const Operand<T> G{(const T*)a.g + (int64_t)j * a.cap * a.ldg, a.ldg, cnt, a.vn};
  typename TL::Acc acc;
  TL::product(W, G, p0, q0, min(s * a.span, a.vn), min((s + 1) * a.span, a.vn), lds, acc);
  float* out = a.dh + s * a.split_stride + (int64_t)j * a.cap * a.dp;
  TL::for_each_quad(acc, [&](int p, int q, f32x4 v) {
    if (q0 + q >= cnt || p0 + p >= a.dp) return;
    f32x4* at = (f32x4*)(out + (int64_t)(q0 + q) * a.dp + p0 + p);
    *at = a.add ? *at + v : v;
  });
}

// dh rows: the splits' sums, scaled, to the rows that they came from; zero
// where the label is ignored.
template <class T>
__global__ __launch_bounds__(256) void xent_dh(const float* sums, int splits, int64_t split_stride,
                                               const int* pos, const int* cnt, int n, int d,
                                               int dp, int cap, float scale, T* dh) {
  const int j = blockIdx.y, lane = threadIdx.x & 63;
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= n) return;
  const int p = pos[(int64_t)j * n + r];
  const float f = scale / max(cnt[j], 1);
  T* out = dh + ((int64_t)j * n + r) * d;
  const float* in = sums + ((int64_t)j * cap + max(p, 0)) * dp;
  for (int x = lane; x < d; x += 64) {
    float v = 0.f;
    if (p >= 0)
      for (int s = 0; s < splits; ++s) v += in[s * split_stride + x];
    out[x] = from_f32<T>(v * f);
  }
}

struct DwArgs {
  const void* hc;
  int dp, cap, d, vn;
  const void* g;
  int ldg;
  const int* cnt;
  float scale;
  void* dw;         // the piece's first row
  int64_t dstride;
  int vec;          // rows start on 4 elements
};

// dW rows of the piece: P = h in col form (p = column), Q = g in col form
// (q = word).
template <class TL>
__global__ __launch_bounds__(TL::THREADS) void xent_dw(DwArgs a) {
  using T = typename TL::T;
  extern __shared__ __align__(16) char lds[];
  const int j = blockIdx.y, cnt = a.cnt[j];
  const int np = (a.d + TL::BP - 1) / TL::BP;
  int tp, tq;
  tile_of<8>(blockIdx.x, np, gridDim.x / np, tp, tq);
  const int p0 = tp * TL::BP, q0 = tq * TL::BQ;
  const Operand<T> H{(const T*)a.hc + (int64_t)j * a.cap * a.dp, a.dp, a.dp, cnt};
  const Operand<T> G{(const T*)a.g + (int64_t)j * a.cap * a.ldg, a.ldg, a.ldg, cnt};
  typename TL::Acc acc;
  TL::product(H, G, p0, q0, 0, cnt, lds, acc);
  const float f = a.scale / max(cnt, 1);
  T* out = (T*)a.dw + j * a.dstride;
  TL::for_each_quad(acc, [&](int p, int q, f32x4 v) {
    if (q0 + q >= a.vn || p0 + p >= a.d) return;
    T* at = out + (int64_t)(q0 + q) * a.d + p0 + p;
    T o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = from_f32<T>(v[i] * f);
    if (a.vec) {
      if constexpr (sizeof(T) == 2)
        *(uint64_t*)at = *(const uint64_t*)o;
      else
        *(f32x4*)at = *(const f32x4*)o;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (p0 + p + i < a.d) at[i] = o[i];
    }
  });
}

// --- launches ----------------------------------------------------------------------

template <class T, bool PC, bool QC>
using Big = Tile<T, PC, QC, 256, 256, 2, 4>;
template <class T, bool PC, bool QC>
using Mid = Tile<T, PC, QC, 128, 128, 2, 2>;
template <class T, bool PC, bool QC>
using Thin = Tile<T, PC, QC, 256, 32, 4, 1>;

// Tiles of more than 64 KB of LDS have to be asked for once per kernel and
// device.
template <class TL, class A>
hipError_t launch_tile(void (*kernel)(A), dim3 grid, hipStream_t s, const A& a) {
  if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                         hipFuncAttributeMaxDynamicSharedMemorySize, TL::LDS))
    return e;
  klaunch(kernel, grid, dim3(TL::THREADS), TL::LDS, s, a);
  return hipGetLastError();
}

template <class T, bool BACKWARD>
hipError_t launch_logits(int shape, const LogitArgs& a, int k, int n, hipStream_t s) {
  const dim3 grid((unsigned)tiles(a.vn, n, bp_of(shape), bq_of(shape)), k);
  if (shape == BIG)
    return launch_tile<Big<T, false, false>>(xent_logits<Big<T, false, false>, BACKWARD>, grid, s,
                                             a);
  if (shape == MID)
    return launch_tile<Mid<T, false, false>>(xent_logits<Mid<T, false, false>, BACKWARD>, grid, s,
                                             a);
  return launch_tile<Thin<T, false, false>>(xent_logits<Thin<T, false, false>, BACKWARD>, grid, s,
                                            a);
}

// The parts of both passes that come first: the gathered rows and, where W's
// own rows do not start on 16 bytes, its copy.
template <class T>
hipError_t prepare(const XentArgs& a, const Layout& l, LogitArgs& g, hipStream_t s) {
  char* ws = (char*)a.ws;
  RowsArgs r{a.h, a.ldh, a.labels, a.ignore, a.n, a.d, l.dp, l.cap,
             (int*)(ws + l.cnt), (int*)(ws + l.pos), (int*)(ws + l.row), (int*)(ws + l.lab),
             ws + l.hc};
  const dim3 grid((a.n + ROWS_PER_BLOCK - 1) / ROWS_PER_BLOCK, a.k);
  constexpr int E = 16 / sizeof(T);
  if ((uintptr_t)a.h % 16 == 0 && a.ldh % E == 0 && a.d % E == 0)
    klaunch(xent_rows<T, true>, grid, dim3(256), 0, s, r);
  else
    klaunch(xent_rows<T, false>, grid, dim3(256), 0, s, r);
  if (hipError_t e = hipGetLastError()) return e;
  g.w = a.w;
  g.ldw = a.d;
  g.pstride = a.pstride;
  g.d = a.d;
  if (l.copy_w) {
    klaunch(xent_copy_w<T>, dim3(std::min((a.v + 3) / 4, 4096), a.k), dim3(256), 0, s,
            (const T*)a.w, a.pstride, a.v, a.d, l.dp, (T*)(ws + l.wc));
    if (hipError_t e = hipGetLastError()) return e;
    g.w = ws + l.wc;
    g.ldw = l.dp;
    g.pstride = (int64_t)a.v * l.dp;
    g.d = l.dp;
  }
  g.v0 = 0;
  g.vn = a.v;
  g.hc = ws + l.hc;
  g.dp = l.dp;
  g.cap = l.cap;
  g.cnt = r.cnt;
  g.lab = r.lab;
  g.row = r.row;
  g.n = a.n;
  g.lse = a.lse;
  return hipSuccess;
}

template <class T>
hipError_t forward(const XentArgs& a, hipStream_t s) {
  const Layout l = layout(a, false);
  char* ws = (char*)a.ws;
  LogitArgs g{};
  if (hipError_t e = prepare<T>(a, l, g, s)) return e;
  g.part = (float2*)(ws + l.part);
  g.plog = (float*)(ws + l.plog);
  g.parts = l.parts;
  if (hipError_t e = launch_logits<T, false>(shape_of(a.k, a.v, a.n), g, a.k, a.n, s)) return e;
  float* rloss = (float*)(ws + l.rloss);
  const int* pos = (const int*)(ws + l.pos);
  if (a.n >= 1024)
    klaunch(xent_join<32>, dim3((a.n + 31) / 32, a.k), dim3(256), 0, s, pos, (const float2*)g.part,
            l.parts, l.cap, (const float*)g.plog, g.lab, a.n, a.v, a.lse, rloss);
  else
    klaunch(xent_join<4>, dim3((a.n + 3) / 4, a.k), dim3(256), 0, s, pos, (const float2*)g.part,
            l.parts, l.cap, (const float*)g.plog, g.lab, a.n, a.v, a.lse, rloss);
  if (hipError_t e = hipGetLastError()) return e;
  klaunch(xent_mean, dim3(a.k), dim3(256), 0, s, (const float*)rloss, g.cnt, a.n, a.loss);
  return hipGetLastError();
}

template <class T>
hipError_t backward(const XentArgs& a, hipStream_t s) {
  const Layout l = layout(a, true);
  char* ws = (char*)a.ws;
  LogitArgs g{};
  if (hipError_t e = prepare<T>(a, l, g, s)) return e;
  g.g = ws + l.g;
  g.ldg = l.piece;
  constexpr int BK = 128 / (int)sizeof(T);
  const float scale = a.grad_scale / g_scale<T>();
  const int sd = shape_of(a.k, a.d, a.n);
  DhArgs dh{};
  dh.ldw = g.ldw;
  dh.pstride = g.pstride;
  dh.d = a.d;
  dh.g = g.g;
  dh.ldg = l.piece;
  dh.cap = l.cap;
  dh.cnt = g.cnt;
  dh.dh = (float*)(ws + l.dh);
  dh.dp = l.dp;
  dh.splits = l.splits;
  dh.split_stride = (int64_t)a.k * l.cap * l.dp;
  DwArgs dw{};
  dw.hc = g.hc;
  dw.dp = l.dp;
  dw.cap = l.cap;
  dw.d = a.d;
  dw.g = g.g;
  dw.ldg = l.piece;
  dw.cnt = g.cnt;
  dw.scale = scale;
  dw.dstride = a.dstride;
  dw.vec = a.d % 4 == 0 && (uintptr_t)a.dw % (4 * sizeof(T)) == 0 && a.dstride % 4 == 0;
  const T* w = (const T*)g.w;
  for (int v0 = 0; v0 < a.v; v0 += l.piece) {
    const int vn = std::min(l.piece, a.v - v0);
    g.w = w + v0 * g.ldw;
    g.v0 = v0;
    g.vn = vn;
    if (hipError_t e = launch_logits<T, true>(shape_of(a.k, vn, a.n), g, a.k, a.n, s)) return e;
    dh.w = g.w;
    dh.vn = vn;
    dh.span = (int)up((vn + l.splits - 1) / l.splits, BK);
    dh.add = v0 > 0;
    const dim3 gd((unsigned)tiles(a.d, a.n, bp_of(sd), bq_of(sd)), a.k, l.splits);
    hipError_t e;
    if (sd == BIG)
      e = launch_tile<Big<T, true, false>>(xent_dh_sums<Big<T, true, false>>, gd, s, dh);
    else if (sd == MID)
      e = launch_tile<Mid<T, true, false>>(xent_dh_sums<Mid<T, true, false>>, gd, s, dh);
    else
      e = launch_tile<Thin<T, true, false>>(xent_dh_sums<Thin<T, true, false>>, gd, s, dh);
    if (e) return e;
    dw.vn = vn;
    dw.dw = (T*)a.dw + (int64_t)v0 * a.d;
    const int sw = a.k * tiles(a.d, vn, 256, 256) >= 256 ? BIG : MID;
    const dim3 gw((unsigned)tiles(a.d, vn, bp_of(sw), bq_of(sw)), a.k);
    if (sw == BIG)
      e = launch_tile<Big<T, true, true>>(xent_dw<Big<T, true, true>>, gw, s, dw);
    else
      e = launch_tile<Mid<T, true, true>>(xent_dw<Mid<T, true, true>>, gw, s, dw);
    if (e) return e;
  }
  klaunch(xent_dh<T>, dim3((a.n + 3) / 4, a.k), dim3(256), 0, s, (const float*)dh.dh, l.splits,
          dh.split_stride, (const int*)(ws + l.pos), g.cnt, a.n, a.d, l.dp, l.cap, scale,
          (T*)a.dh);
  return hipGetLastError();
}

}  // namespace

size_t xent_ws_bytes(const XentArgs& a, bool backward) {
  return layout(a, backward).total;
}

hipError_t xent_fwd(const XentArgs& a, hipStream_t s) {
  return a.type == LM_F32 ? forward<float>(a, s)
         : a.type == LM_F16 ? forward<_Float16>(a, s)
                            : forward<__bf16>(a, s);
}
hipError_t xent_bwd(const XentArgs& a, hipStream_t s) {
  return a.type == LM_F32 ? backward<float>(a, s)
         : a.type == LM_F16 ? backward<_Float16>(a, s)
                            : backward<__bf16>(a, s);
}

}  // namespace cbk
