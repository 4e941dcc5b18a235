// decay_attn.hip -- linear attention with a decay for each head: over whole
// sequences, its gradients, and one token at a time.
//
// Of a head with decay w = exp(g):
//   S_t = w S_{t-1} + k_t v_t^T            o_t = s S_t^T q_t
//   D_t = w D_{t+1} + s q_t do_t^T         (the gradient at S_t)
//   dq_t = s S_t do_t    dk_t = D_t v_t    dv_t = D_t^T k_t
// All four are one form,
//   F(a, b, c)_t = sum_{u <= t} w^(t-u) (a_t . b_u) c_u:
//   o = s F(q, k, v)    dq = s F(do, v, k)
// and, from the last token to the first,
//   dv = s F(k, q, do)  dk = s F(v, do, q),
// so that one kernel does them all.
//
// A workgroup takes CHUNK = 32 rows at a time of a head and, a wave, 32
// columns of c. With S the state behind the rows before, i and u from the
// chunk's first row,
//   out_i = w^(i+1) a_i S + sum_{u <= i} w^(i-u) (a_i . b_u) c_u
//   S     = w^32 S + sum_u b_u (w^(31-u) c_u)^T
// as four matrix products on the bf16 matrix cores. S stays in the
// accumulators of its own product, the scores and the transposed result in
// those of theirs: which rows and columns a tile's 16 indices stand for is
// chosen so that the sums that a lane holds of one product are the operand
// that it needs for the next one, and nothing goes through LDS but the rows
// themselves, which come there straight from memory, a chunk ahead. All waves
// compute the same scores (16 of a wave's some 100 matrix instructions a chunk
// in bf16), which costs less than handing them around.
//
// Operands are sums of bf16 numbers. Rows are one (bf16), two (fp16: exact,
// and without fp16's range for scores and states) or three (fp32). Weights,
// states and scores are fp32; c times its weight enters the state's sum as
// three bf16 numbers, which is all of it, so that states are as good as fp32
// sums (in 16-bit types two for a call that returns no state: up to 2^-16 is
// left out; bf16, four sequences of 2048, 32 heads of 128: 106 us instead of
// 122, backward 214 instead of 247). States and scores enter the result's
// products as three in fp32, else as two, which leaves out up to 2^-16 of them,
// far below the result's own rounding (2^-9, 2^-12). One would leave an error
// as large as that rounding (176 us instead of 213). Where both operands have
// two parts all four products are taken (fp16, as above: 175 us, and 164 with
// three, which left out 2^-14 of a term).
//
// Few sequences and heads leave CUs idle, and a sequence is then cut into
// segments: a first pass leaves each segment's own state, attn_scan goes over
// them, and the second pass begins every segment with its state.
#include "kept.hpp"
#include "lm_tile.hpp"

#include <algorithm>

namespace cbk {
namespace {

__host__ __device__ constexpr int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

constexpr int CHUNK = 32;  // rows

// A segment: its sequence, its place there, and how many segments come before
// it that are not the last ones of their sequences.
struct Segment {
  int seq, at, cut, none;
};

// Sequences of a learner: [k][seqs + 1] starts, or as many rows each; cut
// into segments of `rows` rows, which are numbered by slots.
struct Seqs {
  const int32_t* starts;
  int n, seqs;
  int rows, segs, slots;  // segs: of every sequence, where all are as long
  int cuts;               // segments that are not the last ones, at the most
  const Segment* table;   // [k][slots], seq -1: no segment; or nullptr
  const int* first;       // [k][seqs] number of a sequence's first such segment, with the table
  __device__ __forceinline__ void bounds(int j, int s, int& from, int& to) const {
    if (starts) {
      const int32_t* at = starts + (int64_t)j * (seqs + 1) + s;
      from = min(max(at[0], 0), n);
      to = min(max(at[1], from), n);
    } else {
      from = s * (n / seqs);
      to = from + n / seqs;
    }
  }
  __device__ __forceinline__ Segment slot(int j, int x) const {
    if (table) return table[(int64_t)j * slots + x];
    return {x / segs, x % segs, x - x / segs, 0};
  }
};

// Numbers the segments of sequences whose lengths only the device knows.
__device__ __forceinline__ void number_segments(const Seqs& q, int j, Segment* table, int* first) {
  __shared__ int sums[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Segment* t = table + (int64_t)j * q.slots;
  int base = 0;
  for (int s0 = 0; s0 < q.seqs; s0 += 256) {
    const int s = s0 + threadIdx.x;
    int from = 0, to = 0, count = 0;
    if (s < q.seqs) {
      q.bounds(j, s, from, to);
      count = max(1, (to - from + q.rows - 1) / q.rows);
    }
    int scan = count;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(scan, o);
      if (lane >= o) scan += v;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = scan;
    __syncthreads();
    int at = base + scan - count;
    for (int w = 0; w < wave; ++w) at += sums[w];
    if (s < q.seqs) first[(int64_t)j * q.seqs + s] = at - s;
    // sequences that do not ascend could need more room than there is
    const bool fits = at - s + count - 1 <= q.cuts;
    for (int i = 0; i < count; ++i)
      if (at + i < q.slots) t[at + i] = {fits ? s : -1, i, at + i - s, 0};
    base += sums[0] + sums[1] + sums[2] + sums[3];
  }
  for (int i = base + threadIdx.x; i < q.slots; i += 256) t[i] = {-1, 0, 0, 0};
}

// What comes first where sequences are given by their starts: a workgroup a
// learner numbers the segments, the others write zeros to the results' rows
// outside every sequence.
struct BeginArgs {
  Seqs seq;
  int outs;          // results
  void* out[3];
  int64_t width[3];  // bytes of a row
};
__global__ __launch_bounds__(256) void attn_begin(BeginArgs a) {
  const int j = blockIdx.y;
  if (blockIdx.x == 0) {
    if (a.seq.table) number_segments(a.seq, j, (Segment*)a.seq.table, (int*)a.seq.first);
    return;
  }
  int from, to, first, last;
  a.seq.bounds(j, 0, first, to);
  a.seq.bounds(j, a.seq.seqs - 1, from, last);
  for (int r = blockIdx.x - 1; r < a.seq.n; r += gridDim.x - 1) {
    if (r >= first && r < last) continue;
    for (int o = 0; o < a.outs; ++o) {
      const int64_t width = a.width[o];
      char* row = (char*)a.out[o] + ((int64_t)j * a.seq.n + r) * width;
      if (((uintptr_t)row | width) % 16 == 0)
        for (int64_t i = threadIdx.x * 16; i < width; i += 4096) *(i32x4*)(row + i) = i32x4{0, 0, 0, 0};
      else  // elements have 2 bytes at least
        for (int64_t i = threadIdx.x * 2; i < width; i += 512) *(uint16_t*)(row + i) = 0;
    }
  }
}

// One form F.  Rows of a, b and c are lda, ldb, ldc elements apart, a learner
// n rows; head h of `heads` takes head h / a_share of a, and so on.
struct Form {
  const void *a, *b, *c;
  int64_t lda, ldb, ldc;
  int a_share, b_share, c_share;
  int da, dc;
  bool flip;          // from the last row to the first
  bool direct;        // heads' rows start on 16 bytes, and so do their ends
  void* out;          // [k*n][heads][dc]
  bool wide;          // out is fp32: shares of a sum over heads
  const float* init;  // [k][seqs][heads]: the state before, or nullptr
  float* last;        // and behind, or nullptr
  bool transposed;    // both are [dc][da]
};
struct Args {
  Seqs seq;
  int k, heads, forms, blocks;  // blocks of columns
  float scale;
  const float* decay;
  int64_t decay_stride;
  float* raw;                   // [forms][k][cuts][heads][blocks] states as registers hold them
  Form form[3];
};

// An operand of 8 elements a lane as the sum of N bf16 numbers.
template <int N>
struct Parts {
  i32x4 p[N];
};
template <int N>
__device__ __forceinline__ Parts<N> parts_of(const float (&v)[8]) {
  static_assert(N == 2 || N == 3, "");
  // The leading bits cut off (a rounding could pass the largest bf16), and what
  // is left of each.
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  Parts<N> r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x2 rest = {v[2 * i], v[2 * i + 1]};
    const uint32_t x0 = __builtin_bit_cast(uint32_t, v[2 * i]), x1 = __builtin_bit_cast(uint32_t, v[2 * i + 1]);
    uint32_t x = __builtin_amdgcn_perm(x1, x0, 0x07060302);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      r.p[n][i] = (int)x;
      if (n == N - 1) break;
      const float h0 = __builtin_bit_cast(float, n ? x << 16 : x0 & 0xffff0000u);
      const float h1 = __builtin_bit_cast(float, n ? x & 0xffff0000u : x1 & 0xffff0000u);
      rest = f32x2{rest[0] - h0, rest[1] - h1};
      x = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, bf16x2));
    }
  }
  return r;
}
// The products of two sums, the smallest of them first; where an operand has
// three parts, without those that are 2^-22 of the whole or less. (The product
// of two second parts is not one of them: the first part is cut off, so that
// the second can be 2^-7 of the number and always has its sign.)
template <int NA, int NB>
__device__ __forceinline__ f32x4 mul(const Parts<NA>& a, const Parts<NB>& b, f32x4 c) {
  constexpr int M = NA == 2 && NB == 2 ? 2 : (NA > NB ? NA : NB) - 1;
#pragma unroll
  for (int sum = M; sum >= 0; --sum)
#pragma unroll
    for (int i = NA - 1; i >= 0; --i)
      if (sum - i >= 0 && sum - i < NB) c = mma<__bf16>(a.p[i], b.p[sum - i], c);
  return c;
}

typedef __attribute__((address_space(3))) float lds_float;

// What the types differ in.  Eight elements as they come from LDS:
template <class T>
struct Eight {
  i32x4 w[sizeof(T) / 2];
  __device__ __forceinline__ void floats(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 4) {
        const int x = w[i / 4][i % 4];  // (a vector's element by itself is cast as element 0)
        v[i] = __builtin_bit_cast(float, x);
      } else if constexpr (__is_same(T, _Float16)) {
        v[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)((uint32_t)w[0][i / 2] >> (i % 2 * 16)));
      } else {
        const uint32_t x = w[0][i / 2];
        v[i] = __builtin_bit_cast(float, i % 2 ? x & 0xffff0000u : x << 16);
      }
    }
  }
};
template <class T>
constexpr int NPARTS = __is_same(T, float) ? 3 : __is_same(T, _Float16) ? 2 : 1;
template <class T>
constexpr int NSUMS = __is_same(T, float) ? 3 : 2;  // of scores and states
template <class T>
__device__ __forceinline__ Parts<NPARTS<T>> parts_of(const Eight<T>& e) {
  if constexpr (__is_same(T, __bf16)) {
    return {{e.w[0]}};
  } else {
    float v[8];
    e.floats(v);
    return parts_of<NPARTS<T>>(v);
  }
}

// DA: the width of a and b, up to 64, 128 or 256; NW waves of 32 columns.
template <class T, int DA, int NW>
struct Attn {
  static constexpr int THREADS = 64 * NW, SZ = sizeof(T), E = 16 / SZ;
  static constexpr int PA = DA * SZ, PC = 32 * NW * SZ;  // bytes of a row in LDS
  static constexpr int STAGE = CHUNK * (2 * PA + PC);
  static constexpr int STAGES = 2;  // one on its way
  // a wave's weights: of scores, by how far apart rows are (from -32), and of rows
  static constexpr int TABLE = 96, LDS = STAGES * STAGE + NW * TABLE * 4;
  static_assert(LDS <= 160 << 10, "");
  static constexpr int KS = DA / 32, TILES = DA / 16;
  static constexpr int RAW = DA * 32 * NW;  // floats of a state in registers
  using State = f32x4[TILES][2];

  // 16-byte chunk c of row r lies at c ^ swz(r) (as far as the row has
  // chunks): 16 rows' same chunk, and the eight rows by four chunks of a
  // transposing read, lie in different banks.  Four rows on it is one chunk
  // beside, sixteen rows on the same.
  static __device__ __forceinline__ int swz(int row) {
    return 2 * ((row & 3) | (row >> 3 & 1) << 2) | (row >> 2 & 1);
  }
  template <int PITCH>
  static __device__ __forceinline__ int at(int row, int chunk) {
    return row * PITCH + ((chunk ^ swz(row)) & (PITCH / 16 - 1)) * 16;
  }
  // A lane's first places in a stage's LDS, from which the others differ by
  // bits of the chunk and whole rows: few registers live through the loop.
  struct Places {
    int a, b, t, c;  // rows of a and b, columns of b and of c
  };
  static __device__ __forceinline__ Places places(int wave, int lane) {
    const int g = lane >> 4, r = lane & 15, lb = CHUNK * PA, lc = 2 * CHUNK * PA;
    if constexpr (SZ == 4)
      return {at<PA>(r, 4 * g), lb + at<PA>(r / 4 * 8 + r % 4, 4 * g), lb + at<PA>(8 * g, r),
              lc + at<PC>(8 * g, 8 * wave + r / 2) + (r & 1) * 8};
    return {at<PA>(r, g), lb + at<PA>(r / 4 * 8 + r % 4, g), lb + at<PA>(8 * g + (r >> 2), r & 3),
            lc + at<PC>(8 * g + (r >> 2), 4 * wave + (r & 3))};
  }
  // Chunk's bits by which rows 8g + i differ from row 8g.
  static constexpr int beside(int i) { return (2 * (i & 3) | i >> 2) * 16; }

  // Row and column of S that the sums of tile (t, x) stand for: row of sum e
  // of lane group g, column of lane r of 16.
  static __device__ __forceinline__ int row_of(int t, int g, int e) {
    if constexpr (SZ == 4) return t / 4 * 64 + 16 * g + 4 * e + t % 4;
    return t / 2 * 32 + 8 * g + t % 2 * 4 + e;
  }
  static __device__ __forceinline__ int col_of(int x, int r) {
    if constexpr (SZ == 4) return 2 * r + x;
    return r / 4 * 8 + 4 * x + r % 4;
  }

  typedef const __attribute__((address_space(3))) i32x4 lds_i32x4;

  // Eight columns of a row of a or b (l: the ks = 0 ones): those that the sums
  // of S's tiles stand for, the ks-th 32 of them; `off` bytes on.
  static __device__ __forceinline__ Eight<T> row_eight(uint32_t l, int ks, int off) {
    Eight<T> e;
    if constexpr (SZ == 4) {
#pragma unroll
      for (int i = 0; i < 2; ++i) e.w[i] = *(lds_i32x4*)((l ^ (ks / 2 * 16 + ks % 2 * 2 + i) * 16) + off);
    } else {
      e.w[0] = *(lds_i32x4*)((l ^ ks * 64) + off);
    }
    return e;
  }
  // Rows 8g..8g+7 of one column each (16 bits), of the first or second four
  // columns of 16-byte chunks.
  template <int PITCH>
  static __device__ __forceinline__ Eight<T> column_eight(uint32_t l, int half) {
    Eight<T> e;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4*)((l ^ 16 * u) + 4 * u * PITCH + 8 * half));
      const uint64_t b = __builtin_bit_cast(uint64_t, v);
      e.w[0][2 * u] = (int)(uint32_t)b;
      e.w[0][2 * u + 1] = (int)(uint32_t)(b >> 32);
    }
    return e;
  }
  // The wave's two column tiles of c.
  static __device__ __forceinline__ void columns_c(uint32_t l, Eight<T> (&c)[2]) {
    if constexpr (SZ == 2) {
#pragma unroll
      for (int x = 0; x < 2; ++x) c[x] = column_eight<PC>(l, x);
    } else {
      typedef int i32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const i32x2 v = *(const __attribute__((address_space(3))) i32x2*)((l ^ beside(i)) + i * PC);
        c[0].w[i / 4][i % 4] = v[0];
        c[1].w[i / 4][i % 4] = v[1];
      }
    }
  }
  // Calls f(t, column of b that S's tile t has for each lane), rows 8g..+7.
  template <class F>
  static __device__ __forceinline__ void columns_b(uint32_t l, F f) {
    if constexpr (SZ == 2) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) f(t, column_eight<PA>(l ^ t / 2 * 64, t % 2));
    } else {
#pragma unroll
      for (int v = 0; v < TILES / 4; ++v) {
        Eight<T> e[4];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const i32x4 w = *(lds_i32x4*)((l ^ (v * 256 + beside(i))) + i * PA);
#pragma unroll
          for (int x = 0; x < 4; ++x) e[x].w[i / 4][i % 4] = w[x];
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) f(4 * v + x, e[x]);
      }
    }
  }

  // A chunk's rows of one operand on their way to LDS: of `width` columns, of
  // which LDS rows of PITCH bytes hold what fits.
  template <int PITCH>
  struct Rows {
    static constexpr int CPR = PITCH / 16, NI = CHUNK * CPR / THREADS;
    static_assert(NI * THREADS == CHUNK * CPR, "whole loads");
    uint32_t off[NI];
    const T* base;   // of the sequence's row that is processed first (or before it, reversed)
    int64_t ld;
    int width;
    bool flip, direct;
    __device__ __forceinline__ void init(const T* head, int64_t row, int64_t ld_, int width_, bool flip_,
                                         bool direct_, int tid) {
      ld = ld_;
      width = width_;
      flip = flip_;
      direct = direct_;
      base = head + (flip ? row - (CHUNK - 1) : row) * ld;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int id = i * THREADS + tid, r = id / CPR, c = place(r, id % CPR);
        off[i] = c * E < width ? (uint32_t)((flip ? CHUNK - 1 - r : r) * ld * SZ + c * 16) : OUTSIDE;
      }
    }
    // The chunk of memory that lies at a place of a row, and the other way
    // round.
    static __device__ __forceinline__ int place(int row, int c) {
      return (c ^ swz(row)) & (CPR - 1);
    }
    // Rows [p, p + CHUNK), of which `left` exist.
    __device__ __forceinline__ void issue(int p, int left, uint32_t lds, lds_char* l, int tid) const {
      const T* at = base + (flip ? -(int64_t)p : (int64_t)p) * ld;
      if (direct) {
        const i32x4 rsrc = tile_rsrc(at, 0x7ffffff0u);
        const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6) * 1024;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const bool in = (i * THREADS + tid) / CPR < left;
          load_to_lds(rsrc, in ? off[i] : OUTSIDE, lds + wave + i * (THREADS * 16));
        }
        return;
      }
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int id = i * THREADS + tid, r = id / CPR, c = place(r, id % CPR) * E;
        T v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = (T)0.f;
        if (r < left) {
          const T* row = at + (flip ? CHUNK - 1 - r : r) * ld;
          if (c + E <= width) {
            __builtin_memcpy(v, row + c, 16);
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
              if (c + e < width) v[e] = row[c + e];
          }
        }
        *reinterpret_cast<__attribute__((address_space(3))) i32x4*>(l + id * 16) =
            *reinterpret_cast<const i32x4*>(v);
      }
    }
  };

  // Weights of a chunk's rows: of scores and of rows in the state (a wave's in
  // LDS, read where they are used), of the state in rows and in the next state.
  struct Weights {
    lds_float* table;
    float row[2], keep;
  };
  static __device__ __forceinline__ void score_weights(const Weights& w, float g, float scale, int lane) {
    const int n = lane - 32;
    w.table[lane] = n < 0 ? 0.f : n == 0 ? scale : expf(g * n) * scale;
  }
  // `left` rows in the chunk; fresh: the state that comes in is the gradient
  // at the first row's own, and has not decayed.
  static __device__ __forceinline__ void state_weights(Weights& w, float g, float row_scale, float col_scale,
                                                       int left, bool fresh, int lane) {
    auto power = [&](int n) { return n == 0 ? 1.f : expf(g * n); };
#pragma unroll
    for (int ti = 0; ti < 2; ++ti) w.row[ti] = power(16 * ti + (lane & 15) + (fresh ? 0 : 1)) * row_scale;
    if (lane < 32) w.table[64 + lane] = power(max(left - 1 - lane, 0)) * col_scale;
    w.keep = power(fresh ? left - 1 : left);
  }

  // One chunk: ALL, or the state alone.
  template <bool ALL, bool LAST>
  static __device__ __forceinline__ void chunk(uint32_t l, const Places& at, int lane, const Weights& w, State& S,
                                               f32x4 (&O)[2][2]) {
    const int g = lane >> 4, r = lane & 15;
    Eight<T> c[2];
    columns_c(l + at.c, c);
    if constexpr (ALL) {
      f32x4 P[2][2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) P[i][j] = O[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        Eight<T> a[2], b[2];
        Parts<NPARTS<T>> pa[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          a[t] = row_eight(l + at.a, ks, t * 16 * PA);
          b[t] = row_eight(l + at.b ^ t * 16, ks, t * 4 * PA);
          pa[t] = parts_of(a[t]);
        }
        // scores, transposed: sum 4t + e of lane group g is row 8g + 4t + e of b
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if constexpr (SZ == 2) {
#pragma unroll
            for (int ti = 0; ti < 2; ++ti) P[t][ti] = mma<T>(b[t].w[0], a[ti].w[0], P[t][ti]);
          } else {
            const Parts<NPARTS<T>> pb = parts_of(b[t]);
#pragma unroll
            for (int ti = 0; ti < 2; ++ti) P[t][ti] = mul(pb, pa[ti], P[t][ti]);
          }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            v[i] = SZ == 4 ? S[ks / 2 * 4 + i % 4][x][ks % 2 * 2 + i / 4] : S[2 * ks + i / 4][x][i % 4];
          const Parts<NSUMS<T>> s = parts_of<NSUMS<T>>(v);
#pragma unroll
          for (int ti = 0; ti < 2; ++ti) O[x][ti] = mul(s, pa[ti], O[x][ti]);
        }
      }
      Parts<NPARTS<T>> pc[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) pc[x] = parts_of(c[x]);
#pragma unroll
      for (int ti = 0; ti < 2; ++ti) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = P[i / 4][ti][i % 4] * w.table[32 + 16 * ti + r - 8 * g - i];
        const Parts<NSUMS<T>> p = parts_of<NSUMS<T>>(v);
#pragma unroll
        for (int x = 0; x < 2; ++x) O[x][ti] = mul(pc[x], p, O[x][ti] * w.row[ti]);
      }
    }
    constexpr int N = LAST || SZ == 4 ? 3 : 2;
    Parts<N> cw[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float v[8];
      c[x].floats(v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= w.table[64 + 8 * g + i];
      cw[x] = parts_of<N>(v);
    }
    columns_b(l + at.t, [&](int t, const Eight<T>& e) {
      const Parts<NPARTS<T>> b = parts_of(e);
#pragma unroll
      for (int x = 0; x < 2; ++x) S[t][x] = mul(b, cw[x], S[t][x] * w.keep);
    });
  }
};

// A segment's rows. ALL: results, and with LAST the state behind the sequence's
// last row; else the state behind the segment, for attn_scan. Without LAST no
// state is a result.
template <class T, int DA, int NW, bool ALL, bool LAST>
__global__ __launch_bounds__(64 * NW, DA == 256 ? 1 : 2) void attn_rows(Args args) {
  using A = Attn<T, DA, NW>;
  extern __shared__ __align__(16) char lds[];
  int id = xcd_major(blockIdx.x, gridDim.x);
  const int which = id % args.forms;
  id /= args.forms;
  const int block = id % args.blocks;
  id /= args.blocks;
  const int h = id % args.heads;
  id /= args.heads;
  const int slot = id % args.seq.slots, j = id / args.seq.slots;
  const Form& f = args.form[which];
  const int col0 = block * (32 * NW);
  if (col0 >= f.dc) return;
  const Segment seg = args.seq.slot(j, slot);
  if (seg.seq < 0) return;
  int from, to;
  args.seq.bounds(j, seg.seq, from, to);
  const int len = to - from;
  const int64_t first = (int64_t)seg.at * args.seq.rows;
  const bool ends = first + args.seq.rows >= len;
  if (!ALL && ends) return;
  const int p0 = (int)min(first, (int64_t)len), p1 = ends ? len : p0 + args.seq.rows;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, r = lane & 15;
  const int wcol = col0 + 32 * wave;
  const bool mine = wcol < f.dc;  // this wave has columns
  const float decay = args.decay[j * args.decay_stride + h];

  // the state before the segment
  typename A::State S;
  const int64_t state = ((int64_t)(j * args.seq.seqs + seg.seq) * args.heads + h) * f.da * f.dc;
  auto place = [&](int t, int x, int e) {
    const int d = A::row_of(t, g, e), c = wcol + A::col_of(x, r);
    if (d >= f.da || c >= f.dc) return (int64_t)-1;
    return state + (f.transposed ? (int64_t)c * f.da + d : (int64_t)d * f.dc + c);
  };
  auto raw = [&](int s) {
    const int64_t unit =
        ((((int64_t)which * args.k + j) * args.seq.cuts + s) * args.heads + h) * args.blocks + block;
    return (f32x4*)(args.raw + unit * A::RAW) + wave * (A::TILES * 2 * 64) + lane;
  };
  const bool fresh = f.flip && f.init && seg.at == 0;
#pragma unroll
  for (int t = 0; t < A::TILES; ++t)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      S[t][x] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (seg.at > 0) {
        if (ALL) S[t][x] = raw(seg.cut - 1)[(t * 2 + x) * 64];
      } else if (f.init) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t at = place(t, x, e);
          if (at >= 0) S[t][x][e] = f.init[at];
        }
      }
    }

  const typename A::Places places = A::places(wave, lane);
  typename A::Weights w;
  w.table = (lds_float*)(lds + A::STAGES * A::STAGE) + wave * A::TABLE;
  if constexpr (ALL) A::score_weights(w, decay, args.scale, lane);
  const float row_scale = f.flip ? 1.f : args.scale, col_scale = f.flip ? args.scale : 1.f;

  const int64_t row0 = (int64_t)j * args.seq.n + (f.flip ? to - 1 - p0 : from + p0);
  typename A::template Rows<A::PA> ra, rb;
  typename A::template Rows<A::PC> rc;
  if constexpr (ALL)
    ra.init((const T*)f.a + (int64_t)(h / f.a_share) * f.da, row0, f.lda, f.da, f.flip, f.direct, tid);
  rb.init((const T*)f.b + (int64_t)(h / f.b_share) * f.da, row0, f.ldb, f.da, f.flip, f.direct, tid);
  rc.init((const T*)f.c + (int64_t)(h / f.c_share) * f.dc + col0, row0, f.ldc, f.dc - col0, f.flip, f.direct, tid);
  lds_char* l = (lds_char*)lds;
  const uint32_t la = (uint32_t)(uintptr_t)l;
  const int rows = p1 - p0;
  auto issue = [&](int p, int stage) {
    const int at = stage * A::STAGE, left = min(rows - p, CHUNK);
    if constexpr (ALL) ra.issue(p, left, la + at, l + at, tid);
    rb.issue(p, left, la + at + CHUNK * A::PA, l + at + CHUNK * A::PA, tid);
    rc.issue(p, left, la + at + 2 * CHUNK * A::PA, l + at + 2 * CHUNK * A::PA, tid);
  };
  // The state is in its registers before the loop: else the compiler waits in
  // it, chunk by chunk, for all loads that are under way.
#pragma unroll
  for (int t = 0; t < A::TILES; ++t)
#pragma unroll
    for (int x = 0; x < 2; ++x) asm volatile("" : "+v"(S[t][x]));

  // A chunk's rows come while the one before is worked on.  (The wait is also
  // for that one's stores; to leave them under way was no faster.)
  if (rows > 0) issue(0, 0);
  int stage = 0;
  for (int p = 0; p < rows; p += CHUNK, stage ^= 1) {
    const int left = min(rows - p, CHUNK);
    tile_wait_barrier();
    if (p + CHUNK < rows) issue(p + CHUNK, stage ^ 1);
    if (p == 0 || (p == CHUNK && fresh) || left < CHUNK)
      A::state_weights(w, decay, row_scale, col_scale, left, fresh && p == 0, lane);
    if (!mine) continue;
    f32x4 O[2][2];
    A::template chunk<ALL, LAST>(la + stage * A::STAGE, places, lane, w, S, O);
    if constexpr (ALL) {
#pragma unroll
      for (int ti = 0; ti < 2; ++ti) {
        const int i = 16 * ti + r;
        if (i >= left) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = A::SZ == 4 ? O[e % 2][ti][e / 2] : O[e / 4][ti][e % 4];
        const int64_t row = row0 + (f.flip ? -(int64_t)(p + i) : (int64_t)(p + i));
        const int64_t at = (row * args.heads + h) * f.dc;
        if (f.wide)
          store8<float, false>((float*)f.out + at, wcol + 8 * g, f.dc, v);
        else
          store8<T, false>((T*)f.out + at, wcol + 8 * g, f.dc, v);
      }
    }
  }
  if (!mine) return;
  if constexpr (!ALL) {
#pragma unroll
    for (int t = 0; t < A::TILES; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) raw(seg.cut)[(t * 2 + x) * 64] = S[t][x];
  } else if (LAST && ends && f.last) {
    const float end = f.flip && len ? expf(decay) : 1.f;
#pragma unroll
    for (int t = 0; t < A::TILES; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t at = place(t, x, e);
          if (at >= 0) f.last[at] = S[t][x][e] * end;
        }
  }
}

// States behind the segments of a sequence but the last, from their own.
__global__ __launch_bounds__(256) void attn_scan(Args args, int quads) {
  int id = blockIdx.x;
  const int block = id % args.blocks;
  id /= args.blocks;
  const int h = id % args.heads;
  id /= args.heads;
  const int seq = id % args.seq.seqs;
  id /= args.seq.seqs;
  const int j = id % args.k, which = id / args.k;
  int from, to;
  args.seq.bounds(j, seq, from, to);
  const int segs = (to - from + args.seq.rows - 1) / args.seq.rows;
  const int first = args.seq.first ? args.seq.first[(int64_t)j * args.seq.seqs + seq] : seq * (args.seq.segs - 1);
  if (segs < 3 || first + segs - 1 > args.seq.cuts) return;
  const float w = expf(args.decay[j * args.decay_stride + h] * args.seq.rows);
  const int64_t stride = (int64_t)args.heads * args.blocks * quads;
  const int64_t unit =
      ((((int64_t)which * args.k + j) * args.seq.cuts + first) * args.heads + h) * args.blocks + block;
  f32x4* at = (f32x4*)args.raw + unit * quads + blockIdx.y * 256 + threadIdx.x;
  f32x4 s = *at;
  at += stride;
  constexpr int R = 8;
  for (int x = segs - 2; x > 0; x -= R, at += R * stride) {
    f32x4 own[R];
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (i < x) own[i] = at[i * stride];
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (i < x) {
        s = s * w + own[i];
        at[i * stride] = s;
      }
  }
}

// Sums over the heads that share a key head, of rows [kv * share][d] to
// [kv][d] (rows outside every sequence: zeros); four columns a thread (VEC,
// else one).
struct ShareArgs {
  Seqs seq;
  const float* in;
  void* out;
  int kv, share, d;
};
template <class T, bool VEC>
__global__ __launch_bounds__(256) void attn_share(ShareArgs a) {
  constexpr int W = VEC ? 4 : 1;
  typedef float vec __attribute__((ext_vector_type(W)));
  const int j = blockIdx.y, units = a.d / W, width = a.kv * units;
  int from, to, first, last;
  a.seq.bounds(j, 0, first, to);
  a.seq.bounds(j, a.seq.seqs - 1, from, last);
  for (int r = blockIdx.x; r < a.seq.n; r += gridDim.x) {
    const int64_t row = (int64_t)j * a.seq.n + r;
    for (int i = threadIdx.x; i < width; i += 256) {
      vec sum = {};
      const int head = i / units, c = (i - head * units) * W;
      if (r >= first && r < last) {
        const float* in = a.in + (row * a.kv + head) * a.share * a.d + c;
#pragma unroll 4
        for (int h = 0; h < a.share; ++h) sum += *(const vec*)(in + (int64_t)h * a.d);
      }
      T* out = (T*)a.out + (row * a.kv + head) * a.d + c;
#pragma unroll
      for (int e = 0; e < W; ++e) out[e] = (T)sum[e];
    }
  }
}

// One token of every sequence: a workgroup a head's state.
struct StepArgs {
  int seqs, heads, share, dk, dv;
  int lx;  // log2 of the threads that share a row of S
  float scale;
  const void *q, *key, *val;
  int64_t ldq, ldk, ldv;
  const float* decay;
  int64_t decay_stride;
  const float* state;
  float* state_out;
  void* o;
};
// A thread has four neighbouring columns (VEC; else one) and every rows-th row
// of S, eight of them under way.  Bound by memory: S is read and written once.
template <class T, bool VEC>
__global__ __launch_bounds__(256) void attn_step(StepArgs a) {
  constexpr int W = VEC ? 4 : 1, R = 8;
  typedef float vec __attribute__((ext_vector_type(W)));
  __shared__ float q[256], key[256];
  __shared__ __align__(16) float part[256 * W];
  const int h = blockIdx.x % a.heads, tid = threadIdx.x;
  const int64_t row = blockIdx.x / a.heads, j = row / a.seqs;
  const int lx = a.lx, x = tid & ((1 << lx) - 1), y = tid >> lx, rows = 256 >> lx, c = x * W;
  const int64_t at = (int64_t)blockIdx.x * a.dk * a.dv + c;
  const float* in = a.state + at;
  float* out = a.state_out + at;
  const bool mine = c < a.dv;
  vec s[R];
  auto load = [&](int i0) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (mine && i0 + r * rows < a.dk) s[r] = *(const vec*)(in + (int64_t)(i0 + r * rows) * a.dv);
  };
  load(y);
  for (int i = tid; i < a.dk; i += 256) {
    q[i] = (float)((const T*)a.q)[row * a.ldq + (int64_t)h * a.dk + i] * a.scale;
    key[i] = (float)((const T*)a.key)[row * a.ldk + (int64_t)(h / a.share) * a.dk + i];
  }
  vec v = {}, sum = {};
#pragma unroll
  for (int e = 0; e < W; ++e)
    if (c + e < a.dv) v[e] = (float)((const T*)a.val)[row * a.ldv + (int64_t)(h / a.share) * a.dv + c + e];
  const float w = expf(a.decay[j * a.decay_stride + h]);
  __syncthreads();
  for (int i0 = y; i0 < a.dk; i0 += R * rows) {
    if (i0 != y) load(i0);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int i = i0 + r * rows;
      if (!mine || i >= a.dk) continue;
      const vec t = s[r] * w + v * key[i];
      sum += t * q[i];
      __builtin_nontemporal_store(t, (vec*)(out + (int64_t)i * a.dv));
    }
  }
  *(vec*)(part + tid * W) = sum;
  __syncthreads();
  // the rows' shares, in order
  for (int i = tid; i < a.dv; i += 256) {
    float o = 0.f;
    for (int r = 0; r < rows; ++r) o += part[(r << lx) * W + i];
    ((T*)a.o)[(row * a.heads + h) * a.dv + i] = (T)o;
  }
}

// --- launches --------------------------------------------------------------------

// How the sequences are cut, and places in the workspace.
struct Layout {
  int da, waves, blocks, forms;  // da: 64, 128 or 256
  int rows, segs, slots, cuts;
  bool cut;
  size_t table, first, raw, dkey, dval, total;
};
Layout layout(const AttnArgs& a, bool backward) {
  Layout l;
  const int most = std::max(a.dk, a.dv);
  l.da = most <= 64 ? 64 : most <= 128 ? 128 : 256;
  l.waves = l.da == 64 || (l.da == 256 && a.type == LM_F32) ? 2 : 4;  // as LDS allows
  l.blocks = (most + 32 * l.waves - 1) / (32 * l.waves);
  l.forms = backward ? 3 : 1;
  // As many workgroups as fit the card at once (256 CUs; by registers two of
  // four waves, six of two, of the widest heads one), if segments of LEAST rows
  // or more make them.  Fewer: idle CUs; more: a longer first pass and a second
  // round (bf16, four sequences of 2048, 32 heads of 128, forward, before the
  // last steps: 126 us with 512, 156 with 256, 150 with 1024; fp32, twelve heads
  // of 64 and eight sequences of 1024: 54 us with segments of 128 rows, 78 with
  // 256; six instead of three workgroups a CU there: 134 us backward, 141).
  const int64_t want = 256 * (l.da == 64 ? 6 : l.da == 128 ? 2 : 1);
  constexpr int64_t LEAST = 128;
  const int64_t each = (int64_t)a.k * a.heads * l.blocks * l.forms;
  if (a.starts) {
    // uneven lengths: twice as many, so that long sequences end with the others
    l.rows = (int)std::min<int64_t>(up(a.n, CHUNK), std::max(LEAST, up(a.n * each / (2 * want), CHUNK)));
    l.cut = l.rows < a.n;
    l.segs = 1;
    l.cuts = l.cut ? a.n / l.rows : 0;
    l.slots = a.seqs + l.cuts;
  } else {
    const int64_t len = a.n / a.seqs;
    const int64_t segs = std::max<int64_t>(1, std::min(want / (each * a.seqs), len / LEAST));
    l.rows = (int)up((len + segs - 1) / segs, CHUNK);
    l.segs = (int)((len + l.rows - 1) / l.rows);
    l.cut = l.segs > 1;
    l.cuts = a.seqs * (l.segs - 1);
    l.slots = a.seqs * l.segs;
  }
  size_t at = 256;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)up(bytes, 256);
    return here;
  };
  l.table = l.cut && a.starts ? take((int64_t)a.k * l.slots * (int64_t)sizeof(Segment)) : 0;
  l.first = l.table ? take((int64_t)a.k * a.seqs * 4) : 0;
  l.raw = l.cut ? take(each * l.cuts * l.da * 32 * l.waves * 4) : 0;
  const bool shared = backward && a.heads > a.kv_heads;
  l.dkey = shared ? take((int64_t)a.k * a.n * a.heads * a.dk * 4) : 0;
  l.dval = shared ? take((int64_t)a.k * a.n * a.heads * a.dv * 4) : 0;
  l.total = at;
  return l;
}

Args common(const AttnArgs& a, const Layout& l) {
  char* ws = (char*)a.ws;
  Args x{};
  x.seq = Seqs{a.starts, a.n, a.seqs, l.rows, l.segs, l.slots, l.cuts,
               l.table ? (const Segment*)(ws + l.table) : nullptr,
               l.table ? (const int*)(ws + l.first) : nullptr};
  x.k = a.k;
  x.heads = a.heads;
  x.forms = l.forms;
  x.blocks = l.blocks;
  x.scale = a.scale;
  x.decay = a.decay;
  x.decay_stride = a.decay_stride;
  x.raw = (float*)(ws + l.raw);
  return x;
}

// Whether all rows of all heads start and end on 16 bytes.
template <class T>
bool direct(const Form& f) {
  constexpr int E = 16 / sizeof(T);
  return ((uintptr_t)f.a | (uintptr_t)f.b | (uintptr_t)f.c) % 16 == 0 &&
         (f.lda | f.ldb | f.ldc | f.da | f.dc) % E == 0;
}

template <class T, int DA, int NW, bool LAST>
hipError_t launch_rows(const Args& x, const Layout& l, hipStream_t s) {
  using A = Attn<T, DA, NW>;
  const int units = l.forms * x.k * l.slots * x.heads * l.blocks;
  if (l.cut) {
    if (hipError_t e =
            launch_with_lds<A::LDS, attn_rows<T, DA, NW, false, LAST>>(dim3(units), A::THREADS, s, x))
      return e;
    klaunch(attn_scan, dim3(l.forms * x.k * x.seq.seqs * x.heads * l.blocks, A::RAW / 1024), dim3(256), 0, s, x,
            A::RAW / 4);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return launch_with_lds<A::LDS, attn_rows<T, DA, NW, true, LAST>>(dim3(units), A::THREADS, s, x);
}

template <class T>
hipError_t launch_forms(Args& x, const Layout& l, hipStream_t s) {
  for (int i = 0; i < l.forms; ++i) x.form[i].direct = direct<T>(x.form[i]);
  if constexpr (sizeof(T) == 2) {
    bool last = false;
    for (int i = 0; i < l.forms; ++i) last |= x.form[i].last != nullptr;
    if (!last)
      return l.da == 64    ? launch_rows<T, 64, 2, false>(x, l, s)
             : l.da == 128 ? launch_rows<T, 128, 4, false>(x, l, s)
                           : launch_rows<T, 256, 4, false>(x, l, s);
  }
  return l.da == 64    ? launch_rows<T, 64, 2, true>(x, l, s)
         : l.da == 128 ? launch_rows<T, 128, 4, true>(x, l, s)
                       : launch_rows<T, 256, sizeof(T) == 4 ? 2 : 4, true>(x, l, s);
}

template <class T>
hipError_t forward(const AttnArgs& a, hipStream_t s) {
  const Layout l = layout(a, false);
  const int share = a.heads / a.kv_heads;
  Args x = common(a, l);
  x.form[0] = Form{a.q, a.key, a.val, a.ldq, a.ldk, a.ldv, 1, share, share, a.dk, a.dv, false, false,
                   a.o, false, a.state, a.state_out, false};
  if (a.starts) {
    BeginArgs z{x.seq, 1, {a.o}, {(int64_t)a.heads * a.dv * (int64_t)sizeof(T)}};
    klaunch(attn_begin, dim3(std::min(a.n, 1024) + 1, a.k), dim3(256), 0, s, z);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return launch_forms<T>(x, l, s);
}

template <class T>
hipError_t backward(const AttnArgs& a, hipStream_t s) {
  const Layout l = layout(a, true);
  const int share = a.heads / a.kv_heads;
  const int64_t ldo = (int64_t)a.heads * a.dv, sz = sizeof(T);
  char* ws = (char*)a.ws;
  Args x = common(a, l);
  x.form[0] = Form{a.dout, a.val, a.key, ldo, a.ldv, a.ldk, 1, share, share, a.dv, a.dk, false, false,
                   a.dq, false, a.state, nullptr, true};
  x.form[1] = Form{a.key, a.q, a.dout, a.ldk, a.ldq, ldo, share, 1, 1, a.dk, a.dv, true, false,
                   share > 1 ? (void*)(ws + l.dval) : a.dval, share > 1, a.dstate, a.dstate_in, false};
  x.form[2] = Form{a.val, a.dout, a.q, a.ldv, ldo, a.ldq, share, 1, 1, a.dv, a.dk, true, false,
                   share > 1 ? (void*)(ws + l.dkey) : a.dkey, share > 1, a.dstate, nullptr, true};
  if (a.starts) {
    // (attn_share writes all rows of dkey and dval)
    BeginArgs z{x.seq, share > 1 ? 1 : 3,
                {a.dq, a.dkey, a.dval},
                {a.heads * a.dk * sz, a.kv_heads * a.dk * sz, a.kv_heads * a.dv * sz}};
    klaunch(attn_begin, dim3(std::min(a.n, 1024) + 1, a.k), dim3(256), 0, s, z);
    if (hipError_t e = hipGetLastError()) return e;
  }
  if (hipError_t e = launch_forms<T>(x, l, s)) return e;
  if (share == 1) return hipSuccess;
  const dim3 grid(std::min(a.n, 4096), a.k);
  for (const ShareArgs& y : {ShareArgs{x.seq, (const float*)(ws + l.dkey), a.dkey, a.kv_heads, share, a.dk},
                             ShareArgs{x.seq, (const float*)(ws + l.dval), a.dval, a.kv_heads, share, a.dv}}) {
    klaunch(y.d % 4 ? attn_share<T, false> : attn_share<T, true>, grid, dim3(256), 0, s, y);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t step(const AttnArgs& a, hipStream_t s) {
  // rows of S that start on 16 bytes
  const bool vec = a.dv % 4 == 0 && ((uintptr_t)a.state | (uintptr_t)a.state_out) % 16 == 0;
  int lx = 0;
  while ((vec ? 4 : 1) << lx < a.dv) ++lx;
  StepArgs x{a.seqs, a.heads, a.heads / a.kv_heads, a.dk, a.dv, lx, a.scale, a.q, a.key, a.val,
             a.ldq, a.ldk, a.ldv, a.decay, a.decay_stride, a.state, a.state_out, a.o};
  klaunch(vec ? attn_step<T, true> : attn_step<T, false>, dim3((unsigned)(a.k * a.seqs * a.heads)),
          dim3(256), 0, s, x);
  return hipGetLastError();
}

}  // namespace

size_t attn_ws_bytes(const AttnArgs& a, bool backward) { return layout(a, backward).total; }

hipError_t attn_fwd(const AttnArgs& a, hipStream_t s) {
  return a.type == LM_F32 ? forward<float>(a, s)
         : a.type == LM_F16 ? forward<_Float16>(a, s)
                            : forward<__bf16>(a, s);
}
hipError_t attn_bwd(const AttnArgs& a, hipStream_t s) {
  return a.type == LM_F32 ? backward<float>(a, s)
         : a.type == LM_F16 ? backward<_Float16>(a, s)
                            : backward<__bf16>(a, s);
}
hipError_t attn_token(const AttnArgs& a, hipStream_t s) {
  return a.type == LM_F32 ? step<float>(a, s)
         : a.type == LM_F16 ? step<_Float16>(a, s)
                            : step<__bf16>(a, s);
}

}  // namespace cbk
