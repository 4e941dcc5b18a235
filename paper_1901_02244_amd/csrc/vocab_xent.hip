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
// one tile in few lanes, which reduce them to a (max, sum of exponentials)
// per tile (xent_logits); xent_join_* joins those and xent_mean takes the
// mean.  Backward: for each piece of the vocabulary the
// logits are computed again, g of the piece is stored in the input type, and
// two products add its share of dh (fp32 sums across pieces) and write its
// rows of dW; the last piece's product writes dh itself, or, where few tiles
// share a long vocabulary in splits, xent_dh adds them up.  Every sum runs in
// a fixed order.
//
// g is stored times 2^14 in fp16, so that probabilities down to 2^-28 are
// normal numbers and -1 is still in range; the scale is taken out, with s/C,
// from the fp32 sums.  That store is the only rounding before the results'
// own.
#include "lm.hpp"
#include "lm_tile.hpp"

#include <algorithm>
#include <climits>

namespace cbk {
namespace {

constexpr float NEG_INF = -__builtin_inff();

template <class T>
constexpr float g_scale() {
  return __is_same(T, _Float16) ? 16384.f : 1.f;
}

__host__ __device__ constexpr int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

struct DhShape {
  int shape, splits;
};
// Places in the workspace, in bytes.
struct Layout {
  int cap;       // rows of a learner, up to a multiple of 64
  int dp;        // columns of the gathered rows, up to a multiple of 128 bytes
  int parts;     // tiles of the vocabulary, each with a (max, sum) of a row
  int piece;     // vocabulary rows of one piece of the backward pass
  DhShape dhs;
  bool copy_w;
  size_t cnt, pos, row, lab, hc, wc, part, plog, rloss, g, dh, total;
};

// Tile shapes.  THIN for up to 32 rows of a learner.  Else BIG (256 x 256,
// one workgroup a CU) or MID (128 x 128, two), whichever needs less time for
// the rounds that 256 CUs make of the tiles: a BIG tile is four MID ones and
// MID_COST as dear per element, twice the LDS reads for a product.  fp32
// takes MID always: its MFMAs are sixteen times slower, so that LDS is never
// in the way and the smaller tile's finer rounds are free.
enum { BIG, MID, THIN };
constexpr double MID_COST = 1.3;

int64_t tiles(int64_t a, int64_t b, int ba, int bb) { return up(a, ba) / ba * (up(b, bb) / bb); }

int big_or_mid(int type, int64_t big, int64_t mid) {
  if (type == LM_F32) return MID;
  return (big + 255) / 256 * 4 <= (mid + 511) / 512 * 2 * MID_COST ? BIG : MID;
}
int shape_of(int type, int k, int64_t p, int64_t q) {
  if (q <= 32) return THIN;
  return big_or_mid(type, k * tiles(p, q, 256, 256), k * tiles(p, q, 128, 128));
}
int bp_of(int shape) { return shape == MID ? 128 : 256; }
int bq_of(int shape) { return shape == BIG ? 256 : shape == MID ? 128 : 32; }

// The product for dh has few tiles and, in the vocabulary, a long sum: where
// the tiles do not fill the CUs, `splits` workgroups share a tile's sum.
DhShape dh_shape(int type, int k, int n, int d, int words) {
  const int bk = 128 / lm_size(type);
  const int64_t steps = up(words, bk) / bk;
  if (n <= 32 || type == LM_F32) {
    const int sh = n <= 32 ? THIN : MID;
    const int64_t t = k * tiles(d, n, bp_of(sh), bq_of(sh));
    return {sh, (int)std::max<int64_t>(1, std::min<int64_t>(512 / t, steps / 4))};
  }
  const int64_t t = k * tiles(d, n, 256, 256);
  if (t >= 256) return {BIG, 1};
  const int64_t s = std::max<int64_t>(1, std::min<int64_t>(256 / t, steps / 8));
  if (t * s >= 128) return {BIG, (int)s};
  const int64_t m = k * tiles(d, n, 128, 128);
  return {MID, (int)std::max<int64_t>(1, std::min<int64_t>(512 / m, steps / 4))};
}

Layout layout(const XentArgs& a, bool backward) {
  const int k = a.k, n = a.n, d = a.d, v = a.v, sz = lm_size(a.type);
  Layout l;
  l.cap = (int)up(n, 64);
  l.dp = (int)up(d, 128 / sz);
  // the rows of W are read 16 bytes at a time
  l.copy_w = (uintptr_t)a.w % 16 || (int64_t)d * sz % 16 || (k > 1 && a.pstride * sz % 16);
  const int64_t rows = (int64_t)k * l.cap;
  l.parts = (int)(up(v, bp_of(shape_of(a.type, k, v, n))) / bp_of(shape_of(a.type, k, v, n)));
  // A piece's g takes up to 128 MB, so that it and the piece of W stay in the
  // 256 MB of the memory-side cache between the products (8192 rows of 4096,
  // 128,000 words in bf16: 25.1 ms, with 256 MB 25.8, with 512 MB 25.3), but
  // at least 4096 words, so that reading and writing the fp32 sums of dh once
  // a piece stays small beside the products.
  const int64_t fit = (int64_t(128) << 20) / (rows * sz) / 256 * 256;
  l.piece = (int)std::min<int64_t>(up(v, 256), std::max<int64_t>(4096, fit));
  l.dhs = dh_shape(a.type, k, n, d, std::min(l.piece, v));
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
    // not where one product writes dh itself
    if (l.dhs.splits > 1 || l.piece < v) l.dh = take((int64_t)l.dhs.splits * rows * l.dp * 4);
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
  void* dh;         // backward: rows that do not count get zeros, or nullptr
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
    if (tid == 0 && r0 + ROWS_PER_BLOCK >= a.n) {
      a.cnt[j] = before + __popcll(m);
    }
  }
  __syncthreads();
  const int lane = tid & 63;
  for (int i = tid >> 6; i < ROWS_PER_BLOCK && r0 + i < a.n; i += 4) {
    const int p = place[i];
    if (p < 0) {
      if (a.dh) {
        T* out = (T*)a.dh + ((int64_t)j * a.n + r0 + i) * a.d;
        for (int x = lane; x < a.d; x += 64) out[x] = (T)0.f;
      }
      continue;
    }
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

// Which bits of a row's number permute its chunks in LDS: at most a row's.
template <class TL>
__device__ constexpr int swz_of() {
  constexpr int chunks = TL::BP * (int)sizeof(typename TL::T) / 16;
  return chunks < 32 ? chunks - 1 : 31;
}

// What a tile's logits become.  EDGE: the vocabulary ends inside the wave's
// share.
template <class TL, bool BACKWARD, bool EDGE>
__device__ __forceinline__ void logits_end(const LogitArgs& a, int j, int cnt, int p0, int q0,
                                           char* lds, const int (&label)[TL::TQ],
                                           const float (&lses)[TL::TQ], typename TL::Acc& acc) {
  using T = typename TL::T;
  const int lane = threadIdx.x & 63, lp = 4 * (lane >> 4);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = (wave / TL::WQ) * TL::SP, wq = (wave % TL::WQ) * TL::SQ;
  const int pv = a.vn - p0 - wp;  // words of this wave's share that exist
#pragma unroll
  for (int b = 0; b < TL::TQ; ++b) {
    const int x = wq + TL::col_of(b, lane);
    const int y = label[b] - wp;  // from the wave's first word
    if constexpr (!BACKWARD) {
      float m = NEG_INF;
#pragma unroll
      for (int t = 0; t < TL::TP; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (EDGE && t * 16 + lp + i >= pv) acc[t][b][i] = NEG_INF;
          m = fmaxf(m, acc[t][b][i]);
        }
      // the label's logit, if this lane holds it
      if (y >= 0 && y < min(pv, TL::SP) && (y >> 2 & 3) == lane >> 4) {
        float l = 0.f;
#pragma unroll
        for (int t = 0; t < TL::TP; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) l = y == t * 16 + lp + i ? acc[t][b][i] : l;
        a.plog[(int64_t)j * a.cap + q0 + x] = l;
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
      if (lane < 16) reinterpret_cast<float2*>(lds)[wave / TL::WQ * TL::BQ + x] = {m, e};
    } else {
      const float lse = lses[b];
#pragma unroll
      for (int t = 0; t < TL::TP; ++t) {
        T out[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int p = t * 16 + lp + i;
          float g = __expf(acc[t][b][i] - lse) - (p == y ? 1.f : 0.f);
          if (EDGE && p >= pv) g = 0.f;
          out[i] = from_f32<T>(g * g_scale<T>());
        }
        // rows of BP words in LDS, 16-byte chunk c of row x at c ^ (x & SWZ)
        constexpr int SWZ = swz_of<TL>();
        const int byte = (wp + t * 16 + lp) * (int)sizeof(T);
        char* to = lds + x * (TL::BP * (int)sizeof(T)) + ((byte >> 4) ^ (x & SWZ)) * 16 + (byte & 15);
        if constexpr (sizeof(T) == 2)
          *(uint64_t*)to = *(const uint64_t*)out;
        else
          *(f32x4*)to = *(const f32x4*)out;
      }
    }
  }
}

template <class TL, bool BACKWARD>
__global__ __launch_bounds__(TL::THREADS, 2) void xent_logits(LogitArgs a) {
  using T = typename TL::T;
  extern __shared__ __align__(16) char lds[];
  const int j = blockIdx.y, cnt = a.cnt[j];
  const int np = (a.vn + TL::BP - 1) / TL::BP;
  int tp, tq;
  tile_of<8>(blockIdx.x, np, gridDim.x / np, tp, tq);
  const int p0 = tp * TL::BP, q0 = tq * TL::BQ;
  if (q0 >= cnt) return;
  const Operand<T> W{(const T*)a.w + j * a.pstride, a.ldw, a.vn, a.d};
  const Operand<T> H{(const T*)a.hc + (int64_t)j * a.cap * a.dp, a.dp, cnt, a.d};
  // what the end needs of its rows is fetched behind the product: the labels,
  // from the tile's first word (negative: no word here), and the lse
  int label[TL::TQ];
  float lses[TL::TQ];
  const int wq = (threadIdx.x >> 6) % TL::WQ * TL::SQ;
#pragma unroll
  for (int b = 0; b < TL::TQ; ++b) {
    const int q = q0 + wq + TL::col_of(b, threadIdx.x & 63);
    const int64_t at = (int64_t)j * a.cap + q;
    label[b] = q < cnt ? a.lab[at] - a.v0 - p0 : INT_MIN / 2;
    lses[b] = BACKWARD && q < cnt ? a.lse[(int64_t)j * a.n + a.row[at]] : 0.f;
  }
  typename TL::Acc acc;
  TL::product(W, H, p0, q0, 0, a.d, lds, acc);
  __syncthreads();  // the operands' LDS is used again
  if (p0 + TL::BP <= a.vn)
    logits_end<TL, BACKWARD, false>(a, j, cnt, p0, q0, lds, label, lses, acc);
  else
    logits_end<TL, BACKWARD, true>(a, j, cnt, p0, q0, lds, label, lses, acc);
  __syncthreads();
  if constexpr (!BACKWARD) {
    const int x = threadIdx.x;
    if (x < TL::BQ && q0 + x < cnt) {
      const float2* l = reinterpret_cast<const float2*>(lds) + x;
      float m = l[0].x, e = 0.f;
#pragma unroll
      for (int i = 1; i < TL::WP; ++i) m = fmaxf(m, l[i * TL::BQ].x);
      const float from = m == NEG_INF ? 0.f : m;
#pragma unroll
      for (int i = 0; i < TL::WP; ++i) e += l[i * TL::BQ].y * __expf(l[i * TL::BQ].x - from);
      a.part[((int64_t)j * a.parts + tp) * a.cap + q0 + x] = {m, e};
    }
  } else {
    // whole rows of the tile, 16 bytes a lane, through LDS: the sums lie four
    // words by sixteen rows a wave
    constexpr int CPR = TL::BP * (int)sizeof(T) / 16, EACH = TL::BQ * CPR / TL::THREADS;
    static_assert(EACH * TL::THREADS == TL::BQ * CPR && TL::BQ * CPR * 16 <= TL::LDS, "");
    T* g = (T*)a.g + ((int64_t)j * a.cap + q0) * a.ldg + p0;
#pragma unroll 4
    for (int i = 0; i < EACH; ++i) {
      const int id = i * TL::THREADS + threadIdx.x, x = id / CPR, c = id % CPR;
      if (q0 + x < cnt)
        *(i32x4*)(g + (int64_t)x * a.ldg + c * (16 / (int)sizeof(T))) =
            *(const i32x4*)(lds + (x * CPR + (c ^ (x & swz_of<TL>()))) * 16);
    }
  }
}

// Adds the pair (m2, e2) to (m, e).
__device__ __forceinline__ void join(float& m, float& e, float m2, float e2) {
  const float mm = fmaxf(m, m2), from = mm == NEG_INF ? 0.f : mm;
  e = e * __expf(m - from) + e2 * __expf(m2 - from);
  m = mm;
}

struct JoinArgs {
  const int *cnt, *pos, *lab;
  const float2* part;
  const float* plog;
  int parts, cap, n, v;
  float *lse, *rloss;
  float* loss;      // one workgroup a learner: the mean too; else nullptr
};

// Adds up one fp64 value of each of 256 threads; the sum is thread 0's.
__device__ __forceinline__ double block_sum(double t) {
  __shared__ double sum[256];
  const int tid = threadIdx.x;
  sum[tid] = t;
  __syncthreads();
  for (int o = 128; o; o >>= 1) {
    if (tid < o) sum[tid] += sum[tid + o];
    __syncthreads();
  }
  return sum[0];
}

// Stores a row's lse and returns its loss; 0 and no loss where the label is
// ignored (p < 0).
__device__ __forceinline__ float row_loss(const JoinArgs& a, int j, int r, int p, float m,
                                          float e) {
  float out = 0.f, loss = 0.f;
  if (p >= 0) {
    out = (m == NEG_INF ? 0.f : m) + logf(e);
    const int y = a.lab[(int64_t)j * a.cap + p];
    loss = y >= 0 && y < a.v ? out - a.plog[(int64_t)j * a.cap + p] : __builtin_nanf("");
  }
  a.lse[(int64_t)j * a.n + r] = out;
  a.rloss[(int64_t)j * a.n + r] = loss;
  return loss;
}

// Joins the pairs of a row, a wave a row, for few rows with many pairs each.
// With a.loss one workgroup takes all rows of a learner, and their mean (0 if
// none counts) in fp64.
__global__ __launch_bounds__(256) void xent_join_wide(JoinArgs a) {
  const int j = blockIdx.y, lane = threadIdx.x & 63;
  const int r0 = blockIdx.x * 4 + (threadIdx.x >> 6);
  double total = 0.0;
  for (int r = r0; r < a.n; r += gridDim.x * 4) {
    const int p = a.pos[(int64_t)j * a.n + r];
    float m = NEG_INF, e = 0.f;
    if (p >= 0) {
      const float2* at = a.part + (int64_t)j * a.parts * a.cap + p;
#pragma unroll 4
      for (int i = lane; i < a.parts; i += 64) {
        const float2 o = at[(int64_t)i * a.cap];
        join(m, e, o.x, o.y);
      }
#pragma unroll
      for (int o = 32; o; o >>= 1) join(m, e, __shfl_xor(m, o), __shfl_xor(e, o));
    }
    if (lane == 0) total += row_loss(a, j, r, p, m, e);
  }
  if (!a.loss) return;
  total = block_sum(total);
  if (threadIdx.x == 0) a.loss[j] = (float)(total / max(a.cnt[j], 1));
}

// The same with eight threads a row and neighbouring rows in neighbouring
// lanes, whose pairs lie side by side: 32 rows a workgroup.
__global__ __launch_bounds__(256) void xent_join_rows(JoinArgs a) {
  const int j = blockIdx.y, x = threadIdx.x % 32, s = threadIdx.x / 32;
  const int r = blockIdx.x * 32 + x;
  __shared__ float2 pairs[8][32];
  const int p = r < a.n ? a.pos[(int64_t)j * a.n + r] : -1;
  float m = NEG_INF, e = 0.f;
  if (p >= 0) {
    const float2* at = a.part + (int64_t)j * a.parts * a.cap + p;
#pragma unroll 4
    for (int i = s; i < a.parts; i += 8) {
      const float2 o = at[(int64_t)i * a.cap];
      join(m, e, o.x, o.y);
    }
  }
  pairs[s][x] = {m, e};
  __syncthreads();
  if (s || r >= a.n) return;
  for (int i = 1; i < 8; ++i) join(m, e, pairs[i][x].x, pairs[i][x].y);
  row_loss(a, j, r, p, m, e);
}

// A learner's mean loss over its counted rows (0 if none counts), in fp64.
__global__ __launch_bounds__(256) void xent_mean(const float* rloss, const int* cnt, int n,
                                                 float* loss) {
  const int j = blockIdx.x;
  double t = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += 256) t += rloss[(int64_t)j * n + i];
  t = block_sum(t);
  if (threadIdx.x == 0) loss[j] = (float)(t / max(cnt[j], 1));
}

// --- gradients -------------------------------------------------------------------

struct DhArgs {
  const void* w;    // the piece's first row
  int64_t ldw, pstride;
  int dw, vn;       // columns of W that can be read
  const void* g;
  int ldg, cap;
  const int *cnt, *row;
  float* sums;      // [splits][k][cap][dp]
  int dp, span;     // a split takes `span` words
  int64_t split_stride;
  int add;          // to what the pieces before left in sums
  void* dh;         // the results themselves, [k*n][d], or nullptr
  int n, d, vec;
  float scale;
};

// dh: P = W in col form (p = column), Q = g in row form (q = row).
template <class TL>
__global__ __launch_bounds__(TL::THREADS, 2) void xent_dh_sums(DhArgs a) {
  using T = typename TL::T;
  extern __shared__ __align__(16) char lds[];
  const int j = blockIdx.y, cnt = a.cnt[j], s = blockIdx.z;
  const int np = (a.d + TL::BP - 1) / TL::BP;
  int tp, tq;
  tile_of<8>(blockIdx.x, np, gridDim.x / np, tp, tq);
  const int p0 = tp * TL::BP, q0 = tq * TL::BQ;
  if (q0 >= cnt) return;
  const Operand<T> W{(const T*)a.w + j * a.pstride, a.ldw, a.dw, a.vn};
  const Operand<T> G{(const T*)a.g + (int64_t)j * a.cap * a.ldg, a.ldg, cnt, a.vn};
  typename TL::Acc acc;
  TL::product(W, G, p0, q0, min(s * a.span, a.vn), min((s + 1) * a.span, a.vn), lds, acc);
  float* sums = a.sums + s * a.split_stride + (int64_t)j * a.cap * a.dp;
  const float f = a.scale / max(cnt, 1);
  TL::for_each_quad(acc, [&](int p, int q, f32x4 v) {
    if (q0 + q >= cnt || p0 + p >= a.d) return;
    f32x4* at = (f32x4*)(sums + (int64_t)(q0 + q) * a.dp + p0 + p);
    if (a.add) v = *at + v;
    if (a.dh)
      store4<T>((T*)a.dh + ((int64_t)j * a.n + a.row[(int64_t)j * a.cap + q0 + q]) * a.d + p0 + p,
                v, f, a.d - p0 - p, a.vec);
    else
      *at = v;
  });
}

// dh from the splits' sums; zero where the label is ignored.
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
  // four neighbouring columns a lane: dp is a multiple of four
  for (int x = lane * 4; x < d; x += 256) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (p >= 0) {
#pragma unroll 4
      for (int s = 0; s < splits; ++s) v += *(const f32x4*)(in + s * split_stride + x);
    }
    store4<T>(out + x, v, f, d - x, false);
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
__global__ __launch_bounds__(TL::THREADS, 2) void xent_dw(DwArgs a) {
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
    store4<T>(out + (int64_t)(q0 + q) * a.d + p0 + p, v, f, a.d - p0 - p, a.vec);
  });
}

// --- launches ----------------------------------------------------------------------

template <class T, bool PC, bool QC>
using Big = Tile<T, PC, QC, 256, 256, 2, 4>;
template <class T, bool PC, bool QC>
using Mid = Tile<T, PC, QC, 128, 128, 2, 2>;
template <class T, bool PC, bool QC>
using Thin = Tile<T, PC, QC, 256, 32, 4, 1>;

template <class T, bool BACKWARD>
hipError_t launch_logits(const LogitArgs& a, int k, int n, hipStream_t s) {
  constexpr int type = sizeof(T) == 4 ? LM_F32 : LM_BF16;
  const int shape = shape_of(type, k, a.vn, n);
  const dim3 grid((unsigned)tiles(a.vn, n, bp_of(shape), bq_of(shape)), k);
  if constexpr (sizeof(T) == 2)
    if (shape == BIG)
      return launch_tile<Big<T, false, false>, xent_logits<Big<T, false, false>, BACKWARD>>(grid,
                                                                                            s, a);
  if (shape == MID)
    return launch_tile<Mid<T, false, false>, xent_logits<Mid<T, false, false>, BACKWARD>>(grid, s,
                                                                                          a);
  return launch_tile<Thin<T, false, false>, xent_logits<Thin<T, false, false>, BACKWARD>>(grid, s,
                                                                                          a);
}

// The parts of both passes that come first: the gathered rows and, where W's
// own rows do not start on 16 bytes, its copy.
template <class T>
hipError_t prepare(const XentArgs& a, const Layout& l, void* dh, LogitArgs& g, hipStream_t s) {
  char* ws = (char*)a.ws;
  RowsArgs r{a.h, a.ldh, a.labels, a.ignore, a.n, a.d, l.dp, l.cap,
             (int*)(ws + l.cnt), (int*)(ws + l.pos), (int*)(ws + l.row), (int*)(ws + l.lab),
             ws + l.hc, dh};
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
  if (hipError_t e = prepare<T>(a, l, nullptr, g, s)) return e;
  g.part = (float2*)(ws + l.part);
  g.plog = (float*)(ws + l.plog);
  g.parts = l.parts;
  if (hipError_t e = launch_logits<T, false>(g, a.k, a.n, s)) return e;
  // up to 64 rows one workgroup takes all, and their mean; a wave a row fills
  // the card up to some thousands; the pairs of more rows are read best side
  // by side
  const bool one = a.n <= 64;
  JoinArgs o{g.cnt, (const int*)(ws + l.pos), g.lab, g.part, g.plog, l.parts, l.cap, a.n, a.v,
             a.lse, (float*)(ws + l.rloss), one ? a.loss : nullptr};
  if (a.n < 2048)
    klaunch(xent_join_wide, dim3(one ? 1 : (a.n + 3) / 4, a.k), dim3(256), 0, s, o);
  else
    klaunch(xent_join_rows, dim3((a.n + 31) / 32, a.k), dim3(256), 0, s, o);
  if (hipError_t e = hipGetLastError()) return e;
  if (one) return hipSuccess;
  klaunch(xent_mean, dim3(a.k), dim3(256), 0, s, (const float*)o.rloss, g.cnt, a.n, a.loss);
  return hipGetLastError();
}

template <class T>
hipError_t backward(const XentArgs& a, hipStream_t s) {
  const Layout l = layout(a, true);
  char* ws = (char*)a.ws;
  LogitArgs g{};
  // one split: the last piece's product writes dh
  void* direct = l.dhs.splits == 1 ? a.dh : nullptr;
  if (hipError_t e = prepare<T>(a, l, direct, g, s)) return e;
  g.g = ws + l.g;
  g.ldg = l.piece;
  constexpr int BK = 128 / (int)sizeof(T);
  const float scale = a.grad_scale / g_scale<T>();
  auto quads = [&](const void* p, int64_t stride) {
    return a.d % 4 == 0 && (uintptr_t)p % (4 * sizeof(T)) == 0 && stride % 4 == 0;
  };
  DhArgs dh{};
  dh.ldw = g.ldw;
  dh.pstride = g.pstride;
  dh.dw = g.d;
  dh.d = a.d;
  dh.n = a.n;
  dh.g = g.g;
  dh.ldg = l.piece;
  dh.cap = l.cap;
  dh.cnt = g.cnt;
  dh.row = g.row;
  dh.sums = (float*)(ws + l.dh);
  dh.dp = l.dp;
  dh.split_stride = (int64_t)a.k * l.cap * l.dp;
  dh.vec = quads(a.dh, 0);
  dh.scale = scale;
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
  dw.vec = quads(a.dw, a.dstride);
  const T* w = (const T*)g.w;
  for (int v0 = 0; v0 < a.v; v0 += l.piece) {
    const int vn = std::min(l.piece, a.v - v0);
    g.w = w + v0 * g.ldw;
    g.v0 = v0;
    g.vn = vn;
    if (hipError_t e = launch_logits<T, true>(g, a.k, a.n, s)) return e;
    dh.w = g.w;
    dh.vn = vn;
    dh.span = (int)up((vn + l.dhs.splits - 1) / l.dhs.splits, BK);
    dh.add = v0 > 0;
    dh.dh = v0 + vn == a.v ? direct : nullptr;
    const int sd = l.dhs.shape;
    const dim3 gd((unsigned)tiles(a.d, a.n, bp_of(sd), bq_of(sd)), a.k, l.dhs.splits);
    hipError_t e = hipSuccess;
    if (sd == THIN)
      e = launch_tile<Thin<T, true, false>, xent_dh_sums<Thin<T, true, false>>>(gd, s, dh);
    else if (sd == MID)
      e = launch_tile<Mid<T, true, false>, xent_dh_sums<Mid<T, true, false>>>(gd, s, dh);
    else if constexpr (sizeof(T) == 2)
      e = launch_tile<Big<T, true, false>, xent_dh_sums<Big<T, true, false>>>(gd, s, dh);
    if (e) return e;
    dw.vn = vn;
    dw.dw = (T*)a.dw + (int64_t)v0 * a.d;
    const int sw = big_or_mid(a.type, a.k * tiles(a.d, vn, 256, 256), a.k * tiles(a.d, vn, 128, 128));
    const dim3 gw((unsigned)tiles(a.d, vn, bp_of(sw), bq_of(sw)), a.k);
    if (sw == MID)
      e = launch_tile<Mid<T, true, true>, xent_dw<Mid<T, true, true>>>(gw, s, dw);
    else if constexpr (sizeof(T) == 2)
      e = launch_tile<Big<T, true, true>, xent_dw<Big<T, true, true>>>(gw, s, dw);
    if (e) return e;
  }
  if (direct) return hipSuccess;
  klaunch(xent_dh<T>, dim3((a.n + 3) / 4, a.k), dim3(256), 0, s, (const float*)dh.sums, l.dhs.splits,
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
