// vocab_xent.hip -- softmax cross-entropy of a projection onto a large
// vocabulary, and its gradient, without keeping the logits.
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
// mean.  Where the tiles are too few for the card and the sums long, several
// workgroups share a tile's sum, and what they leave in the workspace are
// logits after all: fp32 ones, 64 MB of shares at the most, which
// xent_sums_loss and xent_sums_grad add up.  Backward: for each piece of the
// vocabulary the logits are computed again, g of the piece is stored in the
// input type, and two products add its share of dh (fp32 sums across pieces)
// and write its rows of dW; the last piece's product writes dh itself, or,
// where few tiles share a long vocabulary in splits, xent_dh adds them up.
// Every sum runs in a fixed order.
//
// Instead of labels a row may have a teacher's logits t_i of m words w_i, at a
// temperature T: with q = softmax(t / T) over them and l = h W^T / T,
//   loss = T^2/C sum_r sum_i q_i (log q_i - (l[w_i] - lse))     g = p - q
//   dh = s T/C g W    dW = s T/C g^T h
// distill_rows reads the lists and, forward, the m words' rows of W (a dot
// product each, read at random: 64 words of 8192 rows of 4096, up to four times
// W and partly found in the caches, take 460 us of a step's 25.9 ms); the rest is
// the loss's, with a factor before the exponentials, but for g at the
// teacher's words: distill_fix stores p - q there, from the forward's logits
// and with one rounding, over the p that the tiles have left.
// Each entry of a row's list is compared with every other one, to add the
// shares of a word that is named twice: fp32, 8192 rows of 64, 1024 words, both
// passes of distill_rows take 146 us with 64 entries, 544 with 256 and 5,810
// with 1024 (the whole step 255, 662 and 5,950).
//
// g is stored times 2^14 in fp16, so that probabilities down to 2^-28 are
// normal numbers and -1 is still in range; the scale is taken out, with s/C,
// from the fp32 sums.  That store is the only rounding before the results'
// own: the products run on 16-bit operands, and g in fp32 would take three
// times the matrix instructions.  Against 64 bits it moves the error of dh and
// dW, most of it their own rounding, from 2.1e-4 to 2.5e-4 of their norm in
// fp16 (two learners of 1023 rows) and from 1.7e-3 to 1.8e-3 in bf16 (8192
// rows); from a teacher, where many entries of g count instead of one that is
// next to -1, to 2.9e-4 and 2.3e-3.  Exponentials are the hardware's exp2 of a rounded product: off by
// (4 |x| + 16) 2^-24 at the most, 0 below 2^-126.
//
// Many rows are bound by the matrix cores (bf16, 8192 rows, about 7400 of
// them counted, 4096 wide, 128,000 words, both passes: 25.3 ms, 1,220 TFLOP/s of
// their four products), few by reading W (one row: 172 us for 1.05 GB, 6.1
// TB/s).  Short sums pay about 10 us around every round of tiles (fp16, two
// learners of 1023 rows, 1000 wide, 32,001 words: 427 us, 785 TFLOP/s).
#include "kept.hpp"
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

// Tile shapes.  THIN for up to THIN_Q rows of a learner.  Else BIG (256 x 256,
// one workgroup a CU) or MID (128 x 128, two), whichever needs less time for
// the rounds that 256 CUs make of the tiles: a BIG tile is four MID ones and
// MID_COST as dear per element, twice the LDS reads for a product.  fp32
// takes MID always: six MFMAs a product keep LDS out of the way, and the
// smaller tile's finer rounds are free.
enum { BIG, MID, THIN };
constexpr double MID_COST = 1.3;

int64_t tiles(int64_t a, int64_t b, int ba, int bb) { return up(a, ba) / ba * (up(b, bb) / bb); }
constexpr int bp_of(int shape) { return shape == MID ? 128 : 256; }
constexpr int bq_of(int shape) { return shape == BIG ? 256 : shape == MID ? 128 : THIN_Q; }
constexpr int threads_of(int shape) { return shape == BIG ? 512 : 256; }
int64_t tiles_of(int shape, int k, int64_t p, int64_t q) {
  return k * tiles(p, q, bp_of(shape), bq_of(shape));
}

// How a product of k learners' p x q over `sum` terms is cut.  Where the
// tiles do not fill the CUs, `splits` workgroups share a tile's sum, and a
// kernel after it adds up what they leave in the workspace.
struct Plan {
  int shape, splits;
};
Plan plan(int type, int k, int64_t p, int64_t q, int64_t sum, bool thin, bool big_splits) {
  const int64_t steps = up(sum, 128 / lm_size(type)) / (128 / lm_size(type));  // of 128 bytes
  // from twelve steps on: the adding up is a launch more, as long as some steps
  auto share = [&](int64_t slots, int64_t t, int least) {
    return steps < 12 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(slots / t, steps / least));
  };
  if (thin && q <= THIN_Q) return {THIN, share(512, tiles_of(THIN, k, p, q), 4)};
  const int64_t mid = tiles_of(MID, k, p, q), big = tiles_of(BIG, k, p, q);
  if (type != LM_F32) {
    if (mid > 256 && (big + 255) / 256 * 4 <= (mid + 511) / 512 * 2 * MID_COST) return {BIG, 1};
    const int s = share(256, big, 8);
    if (big_splits && s > 1 && big * s >= 128) return {BIG, s};
  }
  return {MID, share(512, mid, 4)};
}

// Above MANY rows of a learner, labels are counted and losses added by CHUNK
// of them first; below, each workgroup that needs all of them reads them all,
// which costs less than a launch.
constexpr int MANY = 16384, CHUNK = 1024;

// Places in the workspace, in bytes.
struct Layout {
  int cap;       // rows of a learner, up to a multiple of 64
  int dp;        // columns of the gathered rows, up to a multiple of 128 bytes
  int piece;     // vocabulary rows of one piece of the backward pass
  int words;     // of a tile of the forward's logits
  int parts;     // such tiles, each with a (max, sum) of a row
  Plan logits, dh, dw;
  bool copy_w;
  size_t cnt, chunks, pos, row, lab, hc, wc, part, plog, rloss, means, g, lsum, dhsum, dwsum,
      counts, apart, place, target,  // of a teacher
      total;      // 0: a launch would not hold its workgroups
};

Plan plan_logits(int type, int k, int n, int d, int v) {
  return plan(type, k, v, n, d, true, false);
}

// dW of a piece of vn words: the first one's splits, if it has any, which the
// workspace has sums for.
Plan plan_dw(const XentArgs& a, const Layout& l, int64_t vn) {
  return l.dw.splits > 1 ? l.dw : plan(a.type, a.k, a.d, vn, 0, false, false);
}

// Whether a launch of both gradients holds its workgroups, as launch_grads()
// counts them.
bool grads_fit(const XentArgs& a, Plan h, Plan w, int64_t vn) {
  const int64_t hw = a.k * tiles(a.d, a.n, bp_of(h.shape), bq_of(h.shape)) * h.splits;
  const int64_t ww = a.k * tiles(a.d, vn, bp_of(w.shape), bq_of(w.shape)) * w.splits;
  if ((h.shape == BIG) != (w.shape == BIG))
    return launch_holds(hw, threads_of(h.shape)) && launch_holds(ww, threads_of(w.shape));
  return launch_holds(up(hw, NXCD) + ww, threads_of(h.shape));
}

Layout layout(const XentArgs& a, bool backward) {
  const int k = a.k, n = a.n, d = a.d, v = a.v, sz = lm_size(a.type);
  Layout l;
  l.cap = (int)up(n, 64);
  l.dp = (int)up(d, 128 / sz);
  // the rows of W are read 16 bytes at a time
  l.copy_w = (uintptr_t)a.w % 16 || (int64_t)d * sz % 16 || (k > 1 && a.pstride * sz % 16);
  const int64_t rows = (int64_t)k * l.cap;
  // A piece's g takes up to 128 MB, so that it and the piece of W stay in the
  // 256 MB of the memory-side cache between the products (8192 rows of 4096,
  // 128,000 words in bf16: 25.1 ms, with 256 MB 25.8, with 512 MB 25.3), but
  // at least 4096 words, so that reading and writing the fp32 sums of dh once
  // a piece stays small beside the products.
  const int64_t fit = (int64_t(128) << 20) / (rows * sz) / 256 * 256;
  l.piece = (int)std::min<int64_t>(up(v, 256), std::max<int64_t>(4096, fit));
  l.logits = plan_logits(a.type, k, n, d, v);
  // THIN tiles behind a full round take the time of their sum and not of their
  // words: two rounds and more share the words evenly (bf16, one row of 3968,
  // 132,096 words: 184 us against 239 with 4 tiles behind 512; 4096 wide,
  // 262,144 words, two full rounds either way: 353)
  l.words = bp_of(l.logits.shape);
  const int64_t rounds = (tiles_of(THIN, k, v, n) + 511) / 512;
  if (l.logits.shape == THIN && rounds > 1)
    l.words = (int)std::min<int64_t>(l.words, up(up(v, rounds * 512 / k) / (rounds * 512 / k), 16));
  l.parts = (int)(up(v, l.words) / l.words);
  l.dh = plan(a.type, k, d, n, std::min(l.piece, v), true, true);
  l.dw = plan(a.type, k, d, std::min(l.piece, v), n, false, true);
  // logits in shares only where they are few, which are one piece
  if (v > l.piece) l.logits.splits = 1;
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)up(std::max<int64_t>(bytes, 1), 256);
    return here;
  };
  l.cnt = take(k * 4);
  l.chunks = n > MANY ? take(up(n, CHUNK) / CHUNK * k * 4) : 0;
  l.pos = take((int64_t)k * n * 4);
  l.row = take(rows * 4);
  l.lab = take(rows * 4);
  l.hc = take(rows * l.dp * sz);
  l.wc = l.copy_w ? take((int64_t)k * v * l.dp * sz) : 0;
  l.part = l.plog = l.rloss = l.means = l.g = l.lsum = l.dhsum = l.dwsum = 0;
  if (l.logits.splits > 1) l.lsum = take(l.logits.splits * rows * up(v, 256) * 4);
  if (backward) {
    l.g = take(rows * l.piece * sz);
    // not where one product writes the result itself
    if (l.dh.splits > 1 || l.piece < v) l.dhsum = take(l.dh.splits * rows * l.dp * 4);
    if (l.dw.splits > 1) l.dwsum = take((int64_t)l.dw.splits * k * std::min(l.piece, v) * l.dp * 4);
  } else {
    l.part = take((int64_t)l.parts * rows * 8);
    l.plog = take(rows * 4);
    l.rloss = take((int64_t)k * n * 4);
    l.means = n > MANY ? take(up(n, CHUNK) / CHUNK * k * 16) : 0;
  }
  l.counts = l.apart = l.place = l.target = 0;
  if (a.m) {
    const int64_t all = (int64_t)k * n;
    l.counts = take(all * 4);
    if (backward) {
      l.place = take(all * a.m * 4);
      l.target = take(all * a.m * 4);
    } else {
      l.apart = take(all * 4);
    }
  }
  // the gathering of the rows, and for whole pieces and the last one logits and
  // gradients; the loss's tiles take several launches if need be, and the other
  // launches have a bounded grid
  bool fits = n <= MANY || launch_holds(up(n, 32) / 32, 256);
  if (backward) {
    for (const int64_t vn : {std::min(l.piece, v), (v - 1) % l.piece + 1}) {
      const int shape = plan_logits(a.type, k, n, d, (int)vn).shape;
      fits &= launch_holds(tiles_of(shape, 1, vn, n), threads_of(shape)) &&
              grads_fit(a, l.dh, plan_dw(a, l, vn), vn);
    }
  }
  l.total = fits ? at : 0;
  return l;
}

// --- the counted rows ----------------------------------------------------------

struct RowsArgs {
  const void* h;
  int64_t ldh;
  const int32_t* labels;
  int ignore, n, d, dp, cap;
  int* chunks;      // counted rows of each CHUNK, or nullptr
  int *cnt, *pos, *row, *lab;
  void* hc;
  void* dh;         // backward: rows that do not count get zeros, or nullptr
};

// Adds up one value of each of 256 threads; the sum is every thread's.
template <class V>
__device__ __forceinline__ V block_sum(V t) {
  __shared__ V sum[4];
#pragma unroll
  for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sum[threadIdx.x >> 6] = t;
  __syncthreads();
  return sum[0] + sum[1] + sum[2] + sum[3];
}

__global__ __launch_bounds__(256) void xent_counts(RowsArgs a) {
  const int j = blockIdx.y;
  int c = 0;
#pragma unroll
  for (int i = threadIdx.x; i < CHUNK; i += 256) {
    const int r = blockIdx.x * CHUNK + i;
    c += r < a.n && a.labels[(int64_t)j * a.n + r] != a.ignore;
  }
  c = block_sum(c);
  if (threadIdx.x == 0) a.chunks[(int64_t)j * gridDim.x + blockIdx.x] = c;
}

// Gathers the counted rows of a learner, in order: every workgroup counts the
// labels before its own R rows, then its four waves copy rows, padded with
// zeros to dp columns.  pos[r] is the gathered place of row r or -1, row[]
// and lab[] its inverse and the labels there.
template <class T, int R>
__global__ __launch_bounds__(256) void xent_rows(RowsArgs a) {
  const int j = blockIdx.y, r0 = blockIdx.x * R, tid = threadIdx.x;
  const int32_t* lab = a.labels + (int64_t)j * a.n;
  __shared__ int place[R];
  int c = 0, from = 0;
  if (a.chunks) {
    const int done = r0 / CHUNK, per = (a.n + CHUNK - 1) / CHUNK;
#pragma unroll 4
    for (int i = tid; i < done; i += 256) c += a.chunks[(int64_t)j * per + i];
    from = done * CHUNK;
  }
#pragma unroll 4
  for (int i = from + tid; i < r0; i += 256) c += lab[i] != a.ignore;
  const int before = block_sum(c);
  if (tid < 64) {
    const int r = r0 + tid;
    const bool mine = tid < R && r < a.n;
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
    if (tid == 0 && r0 + R >= a.n) a.cnt[j] = before + __popcll(m);
  }
  __syncthreads();
  const int lane = tid & 63;
  for (int i = tid >> 6; i < R && r0 + i < a.n; i += 4) {
    const int p = place[i];
    const int64_t r = (int64_t)j * a.n + r0 + i;
    const float zeros[8] = {};
    if (p >= 0) {
      const T* src = (const T*)a.h + r * a.ldh;
      T* dst = (T*)a.hc + ((int64_t)j * a.cap + p) * a.dp;
#pragma unroll 4
      for (int x = lane * 8; x < a.dp; x += 512) {
        const Raw8<T> v = load_raw8<T, false>(src, x, a.d);
        __builtin_memcpy(dst + x, v.w, sizeof(v.w));
      }
    } else if (a.dh) {
      for (int x = lane * 8; x < a.d; x += 512) store8<T, false>((T*)a.dh + r * a.d, x, a.d, zeros);
    }
  }
}

// A copy of W whose rows start on 16 bytes, for widths or places whose own
// rows do not: [k][v][dp], padded with zeros.
template <class T>
__global__ __launch_bounds__(256) void xent_copy_w(const T* w, int64_t pstride, int v, int d,
                                                   int dp, T* wc) {
  const int j = blockIdx.y;
  const int64_t units = (int64_t)v * (dp / 8);
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < units; i += gridDim.x * 256ll) {
    const int64_t r = i / (dp / 8);
    const int c = (int)(i - r * (dp / 8)) * 8;
    const Raw8<T> x = load_raw8<T, false>(w + j * pstride + r * d, c, d);
    __builtin_memcpy(wc + ((int64_t)j * v + r) * dp + c, x.w, sizeof(x.w));
  }
}

// --- pieces of the vocabulary ----------------------------------------------------

// The backward pass is launched piece by piece, each launch sized for all
// rows.  Where most rows do not count, a learner takes `m` pieces in a launch
// (its g then has as many times the words of a fraction of the rows) and is
// done after fewer; the other launches find nothing to do (8192 rows of 4096,
// 128,000 words, bf16, of which half count: 10.5 ms against 15.5, a tenth: 3.0
// against 5.3).
struct Pieces {
  int v, piece, index, cap;
  int most;  // the largest m
};
struct Piece {
  int m, v0, vn;  // vn <= 0: nothing left
};
__device__ __forceinline__ Piece piece_of(const Pieces& p, int cnt) {
  Piece r;
  r.m = max(1, min(p.cap / 256 / max(1, (cnt + 255) / 256), p.most));
  const int64_t each = (int64_t)p.piece * r.m, v0 = p.index * each;
  r.v0 = (int)min(v0, (int64_t)p.v);
  r.vn = (int)min(each, (int64_t)p.v - r.v0);
  return r;
}
// Rows between the splits' sums of dh.
__device__ __forceinline__ int rows_between(const Pieces& p, const Piece& r, int cnt) {
  return r.m > 1 ? (cnt + 255) / 256 * 256 : p.cap;
}

// --- a teacher's words -----------------------------------------------------------

struct TeacherArgs {
  const void* h;
  int64_t ldh;
  const void* w;
  int64_t pstride;
  int n, d, v, m;
  const int32_t* words;    // [k*n][m]
  const float* teacher;
  float factor;            // 1/T
  int32_t* counts;         // [k*n] labels: NO_WORD if the row counts, else SKIP
  float* picked;           // [k*n][m] (forward)
  float* apart;            // [k*n] sum of q (log q - l)
  const float* lse;        // (backward)
  const float* given;      // the forward's picked
  int* place;              // [k*n][m] words, each once: the others -1
  float* grad;             // and p - q there
};
constexpr int SKIP = -1, NO_WORD = -2;

// One value of each thread of a workgroup, joined by f in a fixed order.
template <class F>
__device__ __forceinline__ float all_of(float v, float* shared, F f) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = f(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  v = shared[0];
  for (int i = 1; i < (int)blockDim.x >> 6; ++i) v = f(v, shared[i]);
  return v;
}

// A workgroup takes a row.  An entry counts if its word is not negative and
// its logit not minus infinity; the shares of a word that is listed twice are
// added; a word past the vocabulary makes the loss NaN and has no gradient.
template <class T, bool BACKWARD>
__global__ __launch_bounds__(1024) void distill_rows(TeacherArgs a) {
  __shared__ __align__(16) int word[DISTILL_MAX_M];
  __shared__ __align__(16) float share[DISTILL_MAX_M];
  __shared__ float logit[DISTILL_MAX_M];
  __shared__ float joined[16];
  const int j = blockIdx.y, tid = threadIdx.x, all = blockDim.x, lane = tid & 63;
  auto add = [](float x, float y) { return x + y; };
  for (int r = blockIdx.x; r < a.n; r += gridDim.x) {
    const int64_t row = (int64_t)j * a.n + r, at = row * a.m;
    float top = NEG_INF;
    __syncthreads();
    for (int i = tid; i < a.m; i += all) {
      const float t = a.teacher[at + i];
      const int w = a.words[at + i];
      const bool in = w >= 0 && t != NEG_INF;
      word[i] = in ? w : -1;
      share[i] = in ? t : NEG_INF;
      if (in) top = fmaxf(top, share[i]);
    }
    top = all_of(top, joined, [](float x, float y) { return fmaxf(x, y); });
    // (The maximum goes off before the factor: t / T may pass fp32's largest
    // value.  NaN logits have no maximum: they count all the same.)
    float sum = 0.f, some = 0.f;
    for (int i = tid; i < a.m; i += all) {
      const bool in = word[i] >= 0;
      const float e = in ? expf((share[i] - top) * a.factor) : 0.f;
      share[i] = e;
      sum += e;
      some += in;
    }
    sum = all_of(sum, joined, add);
    some = all_of(some, joined, add);
    const bool counts = some > 0.f;
    if (tid == 0) a.counts[row] = counts ? NO_WORD : SKIP;
    if (!counts) {
      for (int i = tid; i < a.m; i += all) {
        if constexpr (BACKWARD)
          a.place[at + i] = -1;
        else
          a.picked[at + i] = 0.f;
      }
      continue;
    }
    const float inv = 1.f / sum;
    if constexpr (!BACKWARD) {
      // a wave takes four words at a time
      const T* h = (const T*)a.h + row * a.ldh;
      const T* W = (const T*)a.w + j * a.pstride;
      constexpr int E = 4;
      for (int i0 = (tid >> 6) * E; i0 < a.m; i0 += all / 64 * E) {
        const T* wr[E];
        bool in[E];
        float dot[E] = {};
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int w = i0 + e < a.m ? word[i0 + e] : -1;
          in[e] = w >= 0 && w < a.v;
          wr[e] = W + (in[e] ? (int64_t)w * a.d : 0);
        }
        for (int c = lane * 8; c < a.d; c += 512) {
          const Raw8<T> x = load_raw8<T, false>(h, c, a.d);
          Raw8<T> y[E];
#pragma unroll
          for (int e = 0; e < E; ++e) y[e] = load_raw8<T, false>(wr[e], in[e] ? c : a.d, a.d);
#pragma unroll
          for (int e = 0; e < E; ++e)
#pragma unroll
            for (int q = 0; q < 8; ++q) dot[e] = fmaf(x.at(q), y[e].at(q), dot[e]);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
#pragma unroll
          for (int o = 32; o; o >>= 1) dot[e] += __shfl_xor(dot[e], o);
          if (lane == 0 && i0 + e < a.m)
            a.picked[at + i0 + e] = logit[i0 + e] = in[e] ? dot[e] * a.factor : 0.f;
        }
      }
    }
    __syncthreads();
    float apart = 0.f;
    for (int i = tid; i < a.m; i += all) {
      const int w = word[i];
      bool first = w >= 0;
      float q = 0.f;
      for (int x = 0; x < a.m; ++x) {
        if (word[x] != w) continue;
        if (x < i) first = false;
        q += share[x];
      }
      q *= inv;
      if constexpr (BACKWARD) {
        const bool in = first && w < a.v;
        a.place[at + i] = in ? w : -1;
        if (in) a.grad[at + i] = __expf(a.given[at + i] - a.lse[row]) - q;
      } else if (first) {
        // (0 log 0 is 0, and a NaN stays one)
        apart += w < a.v ? q * ((q > 0.f ? logf(q) : q) - logit[i]) : __builtin_nanf("");
      }
    }
    if constexpr (!BACKWARD) {
      apart = all_of(apart, joined, add);
      if (tid == 0) a.apart[row] = apart;
    }
  }
}

struct FixArgs {
  const int* place;   // [k*n][m]
  const float* grad;
  int m, n;
  Pieces pieces;
  const int *cnt, *row;
  void* g;
  int ldg;
};

// p - q at the teacher's words of the piece.
template <class T>
__global__ __launch_bounds__(256) void distill_fix(FixArgs a) {
  const int j = blockIdx.y, cnt = a.cnt[j];
  const Piece piece = piece_of(a.pieces, cnt);
  if (piece.vn <= 0) return;
  T* g = (T*)a.g + (int64_t)j * a.pieces.cap * a.pieces.piece;
  const int64_t ldg = (int64_t)a.ldg * piece.m;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < (int64_t)cnt * a.m; i += gridDim.x * 256ll) {
    const int64_t q = i / a.m;
    const int64_t at = ((int64_t)j * a.n + a.row[(int64_t)j * a.pieces.cap + q]) * a.m + (i - q * a.m);
    const int x = a.place[at] - piece.v0;
    if (a.place[at] >= 0 && x >= 0 && x < piece.vn)
      g[q * ldg + x] = from_f32<T>(a.grad[at] * g_scale<T>());
  }
}

// --- logits --------------------------------------------------------------------

// What xent_logits leaves: the pairs of the loss, g, or a split's sums.
enum { LOSS, GRAD, SUMS };

struct LogitArgs {
  const void* w;
  int64_t ldw, pstride;
  int d;            // width of W's rows that holds values
  int v0, vn;       // the vocabulary range [v0, v0 + vn)
  Pieces pieces;    // or, for g, the piece's
  const void* hc;   // rows dp apart, a learner's hstride
  int64_t dp, hstride;
  int cap;
  const int *cnt;   // counted rows, or nullptr: n
  const int *lab, *row;
  int ldlab;        // labels of a learner apart
  float factor;     // of the logits, before the exponentials: 1, or 1/T
  // forward
  int first;        // the launch's first tile
  float2* part;     // [k][parts][cap]
  float* plog;      // [k][cap]
  int parts, words;
  // backward
  const float* lse; // [k*n]
  int n;
  void* g;          // [k][cap * piece], rows ldg apart
  int ldg;
  // splits of the columns, `span` each
  float* sums;      // [splits][k][cap][lds]
  int lds, span;
  int64_t split_stride;
};

// Which bits of a row's number permute its chunks in LDS: at most a row's.
template <class TL>
__device__ constexpr int swz_of() {
  constexpr int chunks = TL::BP * (int)sizeof(typename TL::T) / 16;
  return chunks < 32 ? chunks - 1 : 31;
}

// What a tile's logits become.  EDGE: the vocabulary ends inside the wave's
// share.
template <class TL, int MODE, bool EDGE>
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
    if constexpr (MODE == LOSS) {
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
        for (int i = 0; i < 4; ++i) e += __expf((acc[t][b][i] - from) * a.factor);
      e += __shfl_xor(e, 16);
      e += __shfl_xor(e, 32);
      if (lane < 16)
        reinterpret_cast<float2*>(lds)[wave / TL::WQ * TL::BQ + x] = {m * a.factor, e};
    } else {
      const float lse = lses[b];
#pragma unroll
      for (int t = 0; t < TL::TP; ++t) {
        T out[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int p = t * 16 + lp + i;
          float g = __expf(acc[t][b][i] * a.factor - lse) - (p == y ? 1.f : 0.f);
          if (EDGE && p >= pv) g = 0.f;
          out[i] = from_f32<T>(g * g_scale<T>());
        }
        // rows of BP words in LDS, 16-byte chunk c of row x at c ^ (x & SWZ)
        constexpr int SWZ = swz_of<TL>();
        const int byte = (wp + t * 16 + lp) * (int)sizeof(T);
        char* to =
            lds + x * (TL::BP * (int)sizeof(T)) + ((byte >> 4) ^ (x & SWZ)) * 16 + (byte & 15);
        if constexpr (sizeof(T) == 2)
          *(uint64_t*)to = *(const uint64_t*)out;
        else
          *(f32x4*)to = *(const f32x4*)out;
      }
    }
  }
}

template <class TL, int MODE>
__global__ __launch_bounds__(TL::THREADS, 2) void xent_logits(LogitArgs args) {
  using T = typename TL::T;
  extern __shared__ __align__(16) char lds[];
  LogitArgs a = args;
  const int j = blockIdx.y, cnt = a.cnt ? a.cnt[j] : a.n;
  if constexpr (MODE == GRAD) {
    const Piece piece = piece_of(a.pieces, cnt);
    a.v0 = piece.v0;
    a.vn = piece.vn;
    a.w = (const T*)a.w + a.v0 * a.ldw;
    a.ldg *= piece.m;
  }
  // the counted rows' tiles, first of a grid for all rows
  const int words = MODE == LOSS ? a.words : TL::BP;
  const int tile = (MODE == LOSS ? a.first : 0) + blockIdx.x;
  const int np = (a.vn + words - 1) / words, nq = (cnt + TL::BQ - 1) / TL::BQ;
  if (a.vn <= 0 || tile >= np * nq) return;
  int tp, tq;
  tile_of<8>(tile, np, nq, tp, tq);
  const int p0 = tp * words, q0 = tq * TL::BQ;
  if constexpr (MODE == LOSS) a.vn = min(a.vn, p0 + words);
  const Operand<T> W{(const T*)a.w + j * a.pstride, a.ldw, a.vn, a.d};
  const Operand<T> H{(const T*)a.hc + j * a.hstride, a.dp, cnt, a.d};
  typename TL::Acc acc;
  if constexpr (MODE == SUMS) {
    const int s = blockIdx.z;
    TL::product(W, H, p0, q0, min(s * a.span, a.d), min((s + 1) * a.span, a.d), lds, acc);
    float* out = a.sums + s * a.split_stride + ((int64_t)j * a.cap + q0) * a.lds + p0;
    TL::for_each_quad(acc, [&](int p, int q, f32x4 v) {
      if (q0 + q < cnt) *(f32x4*)(out + (int64_t)q * a.lds + p) = v;
    });
    return;
  }
  // what the end needs of its rows is fetched behind the product: the labels,
  // from the tile's first word (negative: no word here), and the lse
  int label[TL::TQ];
  float lses[TL::TQ];
  const int wq = (threadIdx.x >> 6) % TL::WQ * TL::SQ;
#pragma unroll
  for (int b = 0; b < TL::TQ; ++b) {
    const int q = q0 + wq + TL::col_of(b, threadIdx.x & 63);
    const int64_t at = (int64_t)j * a.cap + q;
    label[b] = q < cnt ? a.lab[(int64_t)j * a.ldlab + q] - a.v0 - p0 : INT_MIN / 2;
    lses[b] = MODE == GRAD && q < cnt ? a.lse[(int64_t)j * a.n + a.row[at]] : 0.f;
  }
  TL::product(W, H, p0, q0, 0, a.d, lds, acc);
  if (p0 + TL::BP <= a.vn)
    logits_end<TL, MODE, false>(a, j, cnt, p0, q0, lds, label, lses, acc);
  else
    logits_end<TL, MODE, true>(a, j, cnt, p0, q0, lds, label, lses, acc);
  __syncthreads();
  if constexpr (MODE == LOSS) {
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
    T* g = (T*)a.g + (int64_t)j * a.cap * a.pieces.piece + (int64_t)q0 * a.ldg + p0;
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
  // the gathered rows' count, places and labels; or cnt and pos nullptr, lab
  // the labels themselves (cap labels of a learner apart from the next one's)
  const int *cnt, *pos, *lab;
  int ignore, ldlab;
  const float2* part;
  float* plog;
  int parts, cap, n, v;
  float *lse, *rloss;
  float* loss;      // one workgroup a learner: the mean too; else nullptr
  // of a teacher: a row's loss is weight * (apart + lse); else nullptr
  const float* apart;
  float weight;
};

// The place of row r, or -1.
__device__ __forceinline__ int place_of(const JoinArgs& a, int j, int r) {
  if (a.pos) return a.pos[(int64_t)j * a.n + r];
  return a.lab[(int64_t)j * a.ldlab + r] != a.ignore ? r : -1;
}

// Stores a row's lse and returns its loss, given the label's logit; 0 and no
// loss where the label is ignored (p < 0).
__device__ __forceinline__ float row_loss(const JoinArgs& a, int j, int r, int p, float m,
                                          float e, float logit) {
  float out = 0.f, loss = 0.f;
  if (p >= 0) {
    out = (m == NEG_INF ? 0.f : m) + logf(e);
    const int y = a.lab[(int64_t)j * a.ldlab + p];
    if (a.apart)
      loss = a.weight * (a.apart[(int64_t)j * a.n + r] + out);
    else
      loss = y >= 0 && y < a.v ? out - logit : __builtin_nanf("");
  }
  a.lse[(int64_t)j * a.n + r] = out;
  a.rloss[(int64_t)j * a.n + r] = loss;
  return loss;
}

// The splits' sums of four neighbouring logits, added in order.
__device__ __forceinline__ f32x4 sum4(const float* at, int splits, int64_t stride) {
  f32x4 v = *(const f32x4*)at;
#pragma unroll 4
  for (int s = 1; s < splits; ++s) v += *(const f32x4*)(at + s * stride);
  return v;
}

struct SumArgs {
  JoinArgs o;
  const float* sums;
  int splits, lds;
  int64_t split_stride;
  float factor;
  // backward
  const float* lse;
  const int* row;
  void* g;
  int ldg;
};

// Where splits share the logits' sums, the loss from those sums: WIDE, a
// workgroup a row, else a wave a row, and with loss one workgroup takes all
// rows of a learner and their mean.
template <bool WIDE>
__global__ __launch_bounds__(256) void xent_sums_loss(SumArgs a) {
  const JoinArgs& o = a.o;
  const int j = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  constexpr int R = WIDE ? 1 : 4, S = 256 / R;
  const int s = tid % S;
  __shared__ float3 shares[4];
  double total = 0.0, rows = 0.0;
  for (int r = blockIdx.x * R + tid / S; r < o.n; r += gridDim.x * R) {
    const int p = place_of(o, j, r);
    float m = NEG_INF, e = 0.f, l = 0.f;  // l: the label's logit, if it is this lane's
    if (p >= 0) {
      const float* at = a.sums + ((int64_t)j * o.cap + p) * a.lds;
      const int y = o.lab[(int64_t)j * o.ldlab + p];
      for (int v = s * 4; v < o.v; v += S * 4) {
        const f32x4 x = sum4(at + v, a.splits, a.split_stride);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (v + i >= o.v) continue;
          join(m, e, x[i] * a.factor, 1.f);
          if (v + i == y) l = x[i];
        }
      }
#pragma unroll
      for (int b = 32; b; b >>= 1) {
        join(m, e, __shfl_xor(m, b), __shfl_xor(e, b));
        l += __shfl_xor(l, b);
      }
    }
    if constexpr (WIDE) {
      if (lane == 0) shares[tid >> 6] = {m, e, l};
      __syncthreads();
      if (tid == 0) {
        for (int i = 1; i < 4; ++i) {
          join(m, e, shares[i].x, shares[i].y);
          l += shares[i].z;
        }
        row_loss(o, j, r, p, m, e, l);
      }
      __syncthreads();
    } else {
      if (lane == 0) {
        total += row_loss(o, j, r, p, m, e, l);
        rows += p >= 0;
      }
    }
  }
  if (!o.loss) return;
  total = block_sum(total);
  rows = block_sum(rows);
  if (tid == 0) o.loss[j] = (float)(total / fmax(rows, 1.0));
}

// and g: S threads a row; zeros up to the next 128 words.
template <class T, int S>
__global__ __launch_bounds__(256) void xent_sums_grad(SumArgs a) {
  const JoinArgs& o = a.o;
  const int j = blockIdx.y, s = threadIdx.x % S;
  const int q = blockIdx.x * (256 / S) + threadIdx.x / S;
  if (q >= o.cnt[j]) return;
  const int64_t at = (int64_t)j * o.cap + q;
  const int y = o.lab[at];
  const float lse = a.lse[(int64_t)j * o.n + a.row[at]];
  const int end = (o.v + 127) / 128 * 128;
  for (int v = s * 4; v < end; v += S * 4) {
    f32x4 g = {0.f, 0.f, 0.f, 0.f};
    if (v < o.v) {
      g = sum4(a.sums + at * a.lds + v, a.splits, a.split_stride);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        g[i] = v + i < o.v ? __expf(g[i] * a.factor - lse) - (v + i == y ? 1.f : 0.f) : 0.f;
    }
    store4<T>((T*)a.g + at * a.ldg + v, g, g_scale<T>(), 4, true);
  }
}

// Joins the pairs of a row, a wave a row, for few rows with many pairs each.
// With a.loss one workgroup takes all rows of a learner, and their mean (0 if
// none counts) in fp64.
__global__ __launch_bounds__(1024) void xent_join_wide(JoinArgs a) {
  const int j = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int waves = blockDim.x >> 6;
  __shared__ double sums[16][2];
  double total = 0.0, rows = 0.0;
  for (int r = blockIdx.x * waves + wave; r < a.n; r += gridDim.x * waves) {
    const int p = place_of(a, j, r);
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
    if (lane == 0) {
      total += row_loss(a, j, r, p, m, e, p >= 0 ? a.plog[(int64_t)j * a.cap + p] : 0.f);
      rows += p >= 0;
    }
  }
  if (!a.loss) return;
  if (lane == 0) {
    sums[wave][0] = total;
    sums[wave][1] = rows;
  }
  __syncthreads();
  if (threadIdx.x) return;
  for (int i = 1; i < waves; ++i) {
    total += sums[i][0];
    rows += sums[i][1];
  }
  a.loss[j] = (float)(total / fmax(rows, 1.0));
}

// The same with eight threads a row and neighbouring rows in neighbouring
// lanes, whose pairs lie side by side: 32 rows a workgroup.
__global__ __launch_bounds__(256) void xent_join_rows(JoinArgs a) {
  const int j = blockIdx.y, x = threadIdx.x % 32, s = threadIdx.x / 32;
  const int r = blockIdx.x * 32 + x;
  __shared__ float2 pairs[8][32];
  const int p = r < a.n ? place_of(a, j, r) : -1;
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
  row_loss(a, j, r, p, m, e, p >= 0 ? a.plog[(int64_t)j * a.cap + p] : 0.f);
}

// A learner's mean loss over its counted rows (0 if none counts), in fp64; of
// many rows, the sum and count of each CHUNK first.
__global__ __launch_bounds__(256) void xent_mean(JoinArgs a, int rows_each, double2* means,
                                                 float* loss) {
  const int j = blockIdx.y, r0 = blockIdx.x * rows_each, r1 = min(r0 + rows_each, a.n);
  double t = 0.0, rows = 0.0;
#pragma unroll 4
  for (int i = r0 + threadIdx.x; i < r1; i += 256) {
    t += a.rloss[(int64_t)j * a.n + i];
    rows += place_of(a, j, i) >= 0;
  }
  t = block_sum(t);
  rows = block_sum(rows);
  if (threadIdx.x) return;
  if (means)
    means[(int64_t)j * gridDim.x + blockIdx.x] = {t, rows};
  else
    loss[j] = (float)(t / fmax(rows, 1.0));
}
__global__ __launch_bounds__(256) void xent_mean_join(const double2* means, int chunks,
                                                      float* loss) {
  const int j = blockIdx.x;
  double t = 0.0, rows = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < chunks; i += 256) {
    const double2 m = means[(int64_t)j * chunks + i];
    t += m.x;
    rows += m.y;
  }
  t = block_sum(t);
  rows = block_sum(rows);
  if (threadIdx.x == 0) loss[j] = (float)(t / fmax(rows, 1.0));
}

// --- gradients -------------------------------------------------------------------

struct DhArgs {
  const void* w;
  int64_t ldw, pstride;
  int dw;           // columns of W that can be read
  Pieces pieces;
  const void* g;
  int ldg;
  const int *cnt, *row;
  float* sums;      // [k][splits * cap][dp]
  int dp, splits;
  void* dh;         // the results themselves, [k*n][d], or nullptr
  int n, d, vec;
  float scale;
};

// The x-th workgroup of learner j: P = W in col form (p = column), Q = g in
// row form (q = row).  A learner that takes m pieces at once has m times the
// splits, of an m-th of the rows; the last piece of one that needs none
// writes dh itself.
template <class TL>
__device__ __forceinline__ void dh_tile(const DhArgs& a, int j, int x, char* lds) {
  using T = typename TL::T;
  const int cnt = a.cnt[j], cap = a.pieces.cap;
  const Piece piece = piece_of(a.pieces, cnt);
  const int np = (a.d + TL::BP - 1) / TL::BP, nq = (cnt + TL::BQ - 1) / TL::BQ;
  const int splits = a.splits * piece.m, ldg = a.ldg * piece.m;
  if (piece.vn <= 0 || x >= np * nq * splits) return;
  const int s = x % splits, span = ((piece.vn + splits - 1) / splits + 63) / 64 * 64;
  int tp, tq;
  tile_of<8>(x / splits, np, nq, tp, tq);
  const int p0 = tp * TL::BP, q0 = tq * TL::BQ;
  const Operand<T> W{(const T*)a.w + j * a.pstride + piece.v0 * a.ldw, a.ldw, a.dw, piece.vn};
  const Operand<T> G{(const T*)a.g + (int64_t)j * cap * a.pieces.piece, ldg, cnt, piece.vn};
  typename TL::Acc acc;
  TL::product(W, G, p0, q0, min(s * span, piece.vn), min((s + 1) * span, piece.vn), lds, acc);
  float* sums = a.sums + ((int64_t)j * a.splits * cap +
                          (int64_t)s * rows_between(a.pieces, piece, cnt)) * a.dp;
  const float f = a.scale / max(cnt, 1);
  const bool add = a.pieces.index > 0;
  T* dh = splits == 1 && piece.v0 + piece.vn == a.pieces.v ? (T*)a.dh : nullptr;
  TL::for_each_quad(acc, [&](int p, int q, f32x4 v) {
    if (q0 + q >= cnt || p0 + p >= a.d) return;
    f32x4* at = (f32x4*)(sums + (int64_t)(q0 + q) * a.dp + p0 + p);
    if (add) v = *at + v;
    if (dh)
      store4<T>(dh + ((int64_t)j * a.n + a.row[(int64_t)j * cap + q0 + q]) * a.d + p0 + p, v, f,
                a.d - p0 - p, a.vec);
    else
      *at = v;
  });
}

// dh from the splits' sums, four neighbouring columns a thread; zero where
// the label is ignored.
template <class T>
__global__ __launch_bounds__(256) void xent_dh(DhArgs a, const int* pos) {
  const int j = blockIdx.y, quads = (a.d + 3) / 4, cnt = a.cnt[j];
  const Piece piece = piece_of(a.pieces, cnt);
  const int splits = a.splits * piece.m;
  if (splits == 1) return;  // written already
  const float f = a.scale / max(cnt, 1);
  const float* sums = a.sums + (int64_t)j * a.splits * a.pieces.cap * a.dp;
  const int64_t stride = (int64_t)rows_between(a.pieces, piece, cnt) * a.dp;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < (int64_t)a.n * quads;
       i += gridDim.x * 256ll) {
    const int64_t r = i / quads;
    const int x = (int)(i - r * quads) * 4, p = pos[(int64_t)j * a.n + r];
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (p >= 0) v = sum4(sums + (int64_t)p * a.dp + x, splits, stride);
    store4<T>((T*)a.dh + ((int64_t)j * a.n + r) * a.d + x, v, f, a.d - x, false);
  }
}

struct DwArgs {
  const void* hc;
  int dp, d, vn;    // vn: of a piece with m = 1
  Pieces pieces;
  const void* g;
  int ldg;
  const int* cnt;
  float scale;
  void* dw;
  int64_t dstride;
  int vec;          // rows start on 4 elements
  float* sums;      // [splits][k][vn][dp], or nullptr: write dw
  int64_t split_stride;
};

// Split s of tile x of the piece's rows of dW, and, of a learner that takes m
// pieces at once, of every `all`-th after it: P = h in col form (p = column),
// Q = g in col form (q = word).
template <class TL>
__device__ __forceinline__ void dw_tiles(const DwArgs& a, int j, int x, int all, int s, int splits,
                                         char* lds) {
  using T = typename TL::T;
  const int cnt = a.cnt[j], cap = a.pieces.cap;
  const Piece piece = piece_of(a.pieces, cnt);
  if (piece.vn <= 0) return;
  const int np = (a.d + TL::BP - 1) / TL::BP, nq = (piece.vn + TL::BQ - 1) / TL::BQ;
  const int ldg = a.ldg * piece.m;
  const Operand<T> H{(const T*)a.hc + (int64_t)j * cap * a.dp, a.dp, a.dp, cnt};
  const Operand<T> G{(const T*)a.g + (int64_t)j * cap * a.pieces.piece, ldg, ldg, cnt};
  const int span = (((cnt + splits - 1) / splits) + TL::BK - 1) / TL::BK * TL::BK;
  const float f = a.scale / max(cnt, 1);
  T* out = (T*)a.dw + j * a.dstride + (int64_t)piece.v0 * a.d;
  float* sums = a.sums ? a.sums + s * a.split_stride + (int64_t)j * a.vn * a.dp : nullptr;
  for (; x < np * nq; x += all) {
    int tp, tq;
    tile_of<8>(x, np, nq, tp, tq);
    const int p0 = tp * TL::BP, q0 = tq * TL::BQ;
    typename TL::Acc acc;
    TL::product(H, G, p0, q0, min(s * span, cnt), min((s + 1) * span, cnt), lds, acc);
    TL::for_each_quad(acc, [&](int p, int q, f32x4 v) {
      if (q0 + q >= piece.vn || p0 + p >= a.d) return;
      if (sums)
        *(f32x4*)(sums + (int64_t)(q0 + q) * a.dp + p0 + p) = v;
      else
        store4<T>(out + (int64_t)(q0 + q) * a.d + p0 + p, v, f, a.d - p0 - p, a.vec);
    });
  }
}

// Both gradients of a piece, which wait for the same g and not for each
// other, in one launch: the CUs that one's last round leaves idle work on the
// other.  All learners' dh, the longer sums, come before all dW.  hn = 0 or
// wn = 0 leaves one out.
struct GradsArgs {
  DhArgs h;
  DwArgs w;
  int k;
  int hn, hs;  // tiles and splits of dh
  int wn, ws;  // of dW
};
template <class TLH, class TLW>
__global__ __launch_bounds__(TLH::THREADS, 2) void xent_grads(GradsArgs a) {
  static_assert(TLH::THREADS == TLW::THREADS);
  extern __shared__ __align__(16) char lds[];
  // dW's tiles start at a multiple of the XCDs, so that tile_of finds them
  // dealt out as it expects
  const int hall = a.hn * a.hs * a.k, from = (hall + NXCD - 1) / NXCD * NXCD;
  int x = blockIdx.x;
  if (x < hall) {
    const int j = x / (a.hn * a.hs);
    x -= j * a.hn * a.hs;
    dh_tile<TLH>(a.h, j, x, lds);
  } else if (x >= from) {
    x -= from;
    const int j = x / (a.wn * a.ws);
    x -= j * a.wn * a.ws;
    dw_tiles<TLW>(a.w, j, x % a.wn, a.wn, x / a.wn, a.ws, lds);
  }
}

// dW from the splits' sums.
template <class T>
__global__ __launch_bounds__(256) void xent_dw_join(DwArgs a, int splits) {
  const int j = blockIdx.y, quads = (a.d + 3) / 4;
  const float f = a.scale / max(a.cnt[j], 1);
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < (int64_t)a.vn * quads;
       i += gridDim.x * 256ll) {
    const int64_t q = i / quads;
    const int p = (int)(i - q * quads) * 4;
    const f32x4 v = sum4(a.sums + ((int64_t)j * a.vn + q) * a.dp + p, splits, a.split_stride);
    const int64_t word = (int64_t)a.pieces.index * a.pieces.piece + q;
    store4<T>((T*)a.dw + j * a.dstride + word * a.d + p, v, f, a.d - p, a.vec);
  }
}

// --- launches ----------------------------------------------------------------------

// The tiles of the loss, in as many launches as their grids need.
template <class TL>
hipError_t launch_loss(LogitArgs a, int64_t v, int n, int k, hipStream_t s) {
  constexpr int64_t MOST = UINT32_MAX / TL::THREADS / NXCD * NXCD;
  static_assert(launch_holds(MOST, TL::THREADS));
  const int64_t all = tiles(v, n, TL::BP, TL::BQ);
  for (int64_t first = 0; first < all; first += MOST) {
    a.first = (int)first;
    const dim3 grid((unsigned)std::min(MOST, all - first), k);
    if (hipError_t e =
            launch_with_lds<TL::LDS, xent_logits<TL, LOSS>>(grid, TL::THREADS, s, a))
      return e;
  }
  return hipSuccess;
}

template <class T, int MODE>
hipError_t launch_logits(const LogitArgs& a, Plan p, int k, int n, hipStream_t s) {
  using Big = BigTile<T, false, false>;
  using Mid = MidTile<T, false, false>;
  using Thin = ThinTile<T, false, false>;
  static_assert(Big::THREADS == threads_of(BIG) && Mid::THREADS == threads_of(MID) &&
                Thin::THREADS == threads_of(THIN));
  static_assert(Big::BP == bp_of(BIG) && Big::BQ == bq_of(BIG) && Mid::BP == bp_of(MID) &&
                Mid::BQ == bq_of(MID) && Thin::BP == bp_of(THIN) && Thin::BQ == bq_of(THIN));
  if constexpr (MODE == LOSS) {
    if constexpr (sizeof(T) == 2)
      if (p.shape == BIG) return launch_loss<Big>(a, a.vn, n, k, s);
    if (p.shape == MID) return launch_loss<Mid>(a, a.vn, n, k, s);
    return launch_loss<Thin>(a, (int64_t)a.parts * Thin::BP, n, k, s);
  } else {
    if constexpr (sizeof(T) == 2 && MODE != SUMS)
      if (p.shape == BIG)
        return launch_tile<Big, xent_logits<Big, MODE>>(a.vn, n, k, p.splits, s, a);
    if (p.shape == MID) return launch_tile<Mid, xent_logits<Mid, MODE>>(a.vn, n, k, p.splits, s, a);
    return launch_tile<Thin, xent_logits<Thin, MODE>>(a.vn, n, k, p.splits, s, a);
  }
}

template <class TLH, class TLW>
hipError_t launch_grads(GradsArgs a, Plan h, Plan w, int k, hipStream_t s) {
  a.hn = (int)(h.splits ? tiles(a.h.d, a.h.n, TLH::BP, TLH::BQ) : 0);
  a.wn = (int)(w.splits ? tiles(a.w.d, a.w.vn, TLW::BP, TLW::BQ) : 0);
  a.hs = h.splits;
  a.ws = w.splits;
  const dim3 grid((unsigned)(up((int64_t)a.hn * a.hs * k, NXCD) + (int64_t)a.wn * a.ws * k));
  return launch_with_lds<std::max(TLH::LDS, TLW::LDS), xent_grads<TLH, TLW>>(grid, TLH::THREADS, s,
                                                                             a);
}

// Both gradients, in one launch where their tiles have as many threads.
template <class T>
hipError_t launch_grads(const DhArgs& h, Plan ph, const DwArgs& w, Plan pw, int k, hipStream_t s) {
  using HBig = BigTile<T, true, false>;
  using HMid = MidTile<T, true, false>;
  using HThin = ThinTile<T, true, false>;
  using WBig = BigTile<T, true, true>;
  using WMid = MidTile<T, true, true>;
  const Plan none{MID, 0};
  GradsArgs a{h, w, k, 0, 0, 0, 0};
  if (sizeof(T) == 2 && (ph.shape == BIG) != (pw.shape == BIG)) {
    if constexpr (sizeof(T) == 2) {
      if (ph.shape == BIG) {
        if (hipError_t e = launch_grads<HBig, WBig>(a, ph, none, k, s)) return e;
        return launch_grads<HMid, WMid>(a, none, pw, k, s);
      }
      if (hipError_t e = launch_grads<HBig, WBig>(a, none, pw, k, s)) return e;
    }
    return ph.shape == MID ? launch_grads<HMid, WMid>(a, ph, none, k, s)
                           : launch_grads<HThin, WMid>(a, ph, none, k, s);
  }
  if constexpr (sizeof(T) == 2)
    if (ph.shape == BIG) return launch_grads<HBig, WBig>(a, ph, pw, k, s);
  return ph.shape == MID ? launch_grads<HMid, WMid>(a, ph, pw, k, s)
                         : launch_grads<HThin, WMid>(a, ph, pw, k, s);
}

// The parts of both passes that come first: the gathered rows (unless the
// forward goes without) and, where W's own rows do not start on 16 bytes, its
// copy.
template <class T>
hipError_t prepare(const XentArgs& a, const Layout& l, bool gather, void* dh, LogitArgs& g,
                   hipStream_t s) {
  char* ws = (char*)a.ws;
  RowsArgs r{a.h, a.ldh, a.labels, a.ignore, a.n, a.d, l.dp, l.cap,
             a.n > MANY ? (int*)(ws + l.chunks) : nullptr,
             (int*)(ws + l.cnt), (int*)(ws + l.pos), (int*)(ws + l.row), (int*)(ws + l.lab),
             ws + l.hc, dh};
  if (gather) {
    // a row a wave, unless that makes the counting dear
    if (a.n <= MANY) {
      klaunch(xent_rows<T, 4>, dim3((a.n + 3) / 4, a.k), dim3(256), 0, s, r);
    } else {
      klaunch(xent_counts, dim3((a.n + CHUNK - 1) / CHUNK, a.k), dim3(256), 0, s, r);
      if (hipError_t e = hipGetLastError()) return e;
      klaunch(xent_rows<T, 32>, dim3((a.n + 31) / 32, a.k), dim3(256), 0, s, r);
    }
    if (hipError_t e = hipGetLastError()) return e;
  }
  g.w = a.w;
  g.ldw = a.d;
  g.pstride = a.pstride;
  g.d = a.d;
  if (l.copy_w) {
    const int64_t blocks = ((int64_t)a.v * (l.dp / 8) + 255) / 256;
    klaunch(xent_copy_w<T>, dim3((unsigned)std::min<int64_t>(blocks, 4096), a.k), dim3(256), 0, s,
            (const T*)a.w, a.pstride, a.v, a.d, l.dp, (T*)(ws + l.wc));
    if (hipError_t e = hipGetLastError()) return e;
    g.w = ws + l.wc;
    g.ldw = l.dp;
    g.pstride = (int64_t)a.v * l.dp;
    g.d = l.dp;
  }
  g.v0 = 0;
  g.vn = a.v;
  g.cap = l.cap;
  if (gather) {
    g.hc = ws + l.hc;
    g.dp = l.dp;
    g.hstride = (int64_t)l.cap * l.dp;
    g.cnt = r.cnt;
    g.lab = r.lab;
    g.ldlab = l.cap;
  } else {
    g.hc = a.h;
    g.dp = a.ldh;
    g.hstride = a.n * a.ldh;
    g.lab = a.labels;
    g.ldlab = a.n;
  }
  g.row = r.row;
  g.n = a.n;
  g.lse = a.lse;
  g.factor = a.m ? 1.f / a.temperature : 1.f;
  g.sums = (float*)(ws + l.lsum);
  g.lds = (int)up(a.v, 256);
  g.span = (int)up((g.d + l.logits.splits - 1) / l.logits.splits, 128 / sizeof(T));
  g.split_stride = (int64_t)a.k * l.cap * g.lds;
  return hipSuccess;
}

// A teacher's lists, as the labels that say which rows count, and what the
// passes need of them.
template <class T, bool BACKWARD>
hipError_t read_teacher(XentArgs& a, const Layout& l, hipStream_t s) {
  char* ws = (char*)a.ws;
  TeacherArgs t{a.h, a.ldh, a.w, a.pstride, a.n, a.d, a.v, a.m, a.words, a.teacher,
                1.f / a.temperature, (int32_t*)(ws + l.counts), a.picked, (float*)(ws + l.apart),
                a.lse, a.picked, (int*)(ws + l.place), (float*)(ws + l.target)};
  // few rows: a row's words are read by as many waves as there can be
  const int threads = BACKWARD || (int64_t)a.k * a.n >= 1024 ? 256 : 1024;
  klaunch(distill_rows<T, BACKWARD>, dim3(std::min(a.n, 65536), a.k), dim3(threads), 0, s, t);
  a.labels = t.counts;
  a.ignore = SKIP;
  return hipGetLastError();
}

template <class T>
hipError_t forward(const XentArgs& given, hipStream_t s) {
  XentArgs a = given;
  const Layout l = layout(a, false);
  char* ws = (char*)a.ws;
  LogitArgs g{};
  if (a.m)
    if (hipError_t e = read_teacher<T, false>(a, l, s)) return e;
  // Few rows are not worth gathering where they can be read as they lie: a row
  // that does not count fills its own column of the logits, which nobody reads.
  // (Offsets within a tile have 31 bits.)
  constexpr int E = 16 / sizeof(T);
  const bool gather = a.n > THIN_Q || (uintptr_t)a.h % 16 || a.ldh % E || a.ldh > (1 << 22) ||
                      l.copy_w;
  if (hipError_t e = prepare<T>(a, l, gather, nullptr, g, s)) return e;
  g.part = (float2*)(ws + l.part);
  g.plog = (float*)(ws + l.plog);
  g.parts = l.parts;
  g.words = l.words;
  // up to 64 rows one workgroup takes all, and their mean; a wave a row fills
  // the card up to some thousands; the pairs of more rows are read best side
  // by side
  const bool summed = l.logits.splits > 1, wide = a.v > 1024;
  const bool one = a.n <= 64 && !(summed && wide);
  JoinArgs o{g.cnt, gather ? (const int*)(ws + l.pos) : nullptr, g.lab, a.ignore, g.ldlab,
             g.part, g.plog, l.parts, l.cap, a.n, a.v,
             a.lse, (float*)(ws + l.rloss), one ? a.loss : nullptr,
             a.m ? (const float*)(ws + l.apart) : nullptr, a.temperature * a.temperature};
  const dim3 waves(one ? 1 : (a.n + 3) / 4, a.k);
  if (summed) {
    if (hipError_t e = launch_logits<T, SUMS>(g, l.logits, a.k, a.n, s)) return e;
    SumArgs u{o, g.sums, l.logits.splits, g.lds, g.split_stride, g.factor,
              nullptr, nullptr, nullptr, 0};
    if (wide)
      klaunch(xent_sums_loss<true>, dim3(a.n, a.k), dim3(256), 0, s, u);
    else
      klaunch(xent_sums_loss<false>, waves, dim3(256), 0, s, u);
  } else {
    if (hipError_t e = launch_logits<T, LOSS>(g, l.logits, a.k, a.n, s)) return e;
    if (a.n < 2048)
      klaunch(xent_join_wide, waves, dim3(one ? std::min((a.n + 3) / 4 * 256, 1024) : 256), 0, s,
              o);
    else
      klaunch(xent_join_rows, dim3((a.n + 31) / 32, a.k), dim3(256), 0, s, o);
  }
  if (hipError_t e = hipGetLastError()) return e;
  if (one) return hipSuccess;
  if (a.n <= MANY) {
    klaunch(xent_mean, dim3(1, a.k), dim3(256), 0, s, o, a.n, (double2*)nullptr, a.loss);
    return hipGetLastError();
  }
  const int chunks = (a.n + CHUNK - 1) / CHUNK;
  double2* means = (double2*)(ws + l.means);
  klaunch(xent_mean, dim3(chunks, a.k), dim3(256), 0, s, o, CHUNK, means, (float*)nullptr);
  if (hipError_t e = hipGetLastError()) return e;
  klaunch(xent_mean_join, dim3(a.k), dim3(256), 0, s, (const double2*)means, chunks, a.loss);
  return hipGetLastError();
}

template <class T>
hipError_t backward(const XentArgs& given, hipStream_t s) {
  XentArgs a = given;
  const Layout l = layout(a, true);
  char* ws = (char*)a.ws;
  LogitArgs g{};
  if (a.m)
    if (hipError_t e = read_teacher<T, true>(a, l, s)) return e;
  // one split: the last piece's product writes dh
  void* direct = l.dh.splits == 1 ? a.dh : nullptr;
  if (hipError_t e = prepare<T>(a, l, true, direct, g, s)) return e;
  g.g = ws + l.g;
  g.ldg = l.piece;
  // several pieces, and room for a learner with half of the rows or fewer to
  // take more than one (dW's splits have sums for one)
  const bool grow = a.v > l.piece && l.cap >= 512 && l.dw.splits == 1;
  // and g's rows lie no further apart than lets a tile of 256 stay below 2 GiB:
  // what a tile's 31-bit offsets do not reach would read as zero
  const int64_t fits = INT_MAX / ((int64_t)l.piece * sizeof(T) * 256);
  const int64_t most = grow ? std::min(up(a.v, l.piece) / l.piece, fits) : 1;
  g.pieces = Pieces{a.v, l.piece, 0, l.cap, (int)most};
  const float scale = a.grad_scale / g_scale<T>();
  auto quads = [&](const void* p, int64_t stride) {
    return a.d % 4 == 0 && (uintptr_t)p % (4 * sizeof(T)) == 0 && stride % 4 == 0;
  };
  DhArgs dh{};
  dh.w = g.w;
  dh.ldw = g.ldw;
  dh.pstride = g.pstride;
  dh.dw = g.d;
  dh.d = a.d;
  dh.n = a.n;
  dh.g = g.g;
  dh.ldg = l.piece;
  dh.cnt = g.cnt;
  dh.row = g.row;
  dh.sums = (float*)(ws + l.dhsum);
  dh.dp = l.dp;
  dh.splits = l.dh.splits;
  dh.dh = a.dh;
  dh.vec = quads(a.dh, 0);
  dh.scale = scale;
  DwArgs dw{};
  dw.hc = g.hc;
  dw.dp = l.dp;
  dw.dw = a.dw;
  dw.d = a.d;
  dw.g = g.g;
  dw.ldg = l.piece;
  dw.cnt = g.cnt;
  dw.scale = scale;
  dw.dstride = a.dstride;
  dw.vec = quads(a.dw, a.dstride);
  dw.sums = l.dw.splits > 1 ? (float*)(ws + l.dwsum) : nullptr;
  for (int v0 = 0; v0 < a.v; v0 += l.piece) {
    const int vn = std::min(l.piece, a.v - v0);
    g.vn = vn;
    if (l.logits.splits > 1) {
      if (hipError_t e = launch_logits<T, SUMS>(g, l.logits, a.k, a.n, s)) return e;
      SumArgs u{};
      u.o.cnt = g.cnt;
      u.o.lab = g.lab;
      u.o.cap = l.cap;
      u.o.n = a.n;
      u.o.v = a.v;
      u.sums = g.sums;
      u.splits = l.logits.splits;
      u.lds = g.lds;
      u.split_stride = g.split_stride;
      u.factor = g.factor;
      u.lse = a.lse;
      u.row = g.row;
      u.g = g.g;
      u.ldg = g.ldg;
      if (a.v > 1024)
        klaunch(xent_sums_grad<T, 256>, dim3(a.n, a.k), dim3(256), 0, s, u);
      else
        klaunch(xent_sums_grad<T, 64>, dim3((a.n + 3) / 4, a.k), dim3(256), 0, s, u);
      if (hipError_t e = hipGetLastError()) return e;
    } else {
      Plan p = plan_logits(a.type, a.k, a.n, g.d, vn);
      p.splits = 1;
      if (hipError_t e = launch_logits<T, GRAD>(g, p, a.k, a.n, s)) return e;
    }
    if (a.m) {
      FixArgs f{(const int*)(ws + l.place), (const float*)(ws + l.target), a.m, a.n, g.pieces,
                g.cnt, g.row, g.g, g.ldg};
      const int64_t blocks = ((int64_t)a.n * a.m + 255) / 256;
      klaunch(distill_fix<T>, dim3((unsigned)std::min<int64_t>(blocks, 2048), a.k), dim3(256), 0, s,
              f);
      if (hipError_t e = hipGetLastError()) return e;
    }
    dh.pieces = dw.pieces = g.pieces;
    dw.vn = vn;
    dw.split_stride = (int64_t)a.k * vn * l.dp;
    if (hipError_t e = launch_grads<T>(dh, l.dh, dw, plan_dw(a, l, vn), a.k, s)) return e;
    if (dw.sums) {
      const int64_t blocks = ((int64_t)vn * ((a.d + 3) / 4) + 255) / 256;
      klaunch(xent_dw_join<T>, dim3((unsigned)std::min<int64_t>(blocks, 2048), a.k), dim3(256), 0,
              s, dw, l.dw.splits);
      if (hipError_t e2 = hipGetLastError()) return e2;
    }
    ++g.pieces.index;
  }
  if (l.dh.splits == 1 && !grow) return hipSuccess;
  const int64_t blocks = ((int64_t)a.n * ((a.d + 3) / 4) + 255) / 256;
  klaunch(xent_dh<T>, dim3((unsigned)std::min<int64_t>(blocks, 4096), a.k), dim3(256), 0, s, dh,
          (const int*)(ws + l.pos));
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
