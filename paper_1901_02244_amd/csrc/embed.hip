// embed.hip -- the rows of a table for a learner's tokens, and the table's
// gradient.
//
//   y[r] = s E[t_r]                 dE[w] = s sum_{r: t_r = w} dy[r]
//
// Forward: a copy of rows, bound by memory.  Backward without atomics on sums:
// the tokens are sorted (with their rows, so that equal tokens keep the rows'
// order), and runs of equal tokens are summed in fp32 in that order.  The
// sorted rows are cut into pieces of `each`, so that a word that half of the
// batch holds has as many threads as others; a run that passes a piece's end
// leaves fp32 partial sums, which embed_join adds in order, a workgroup a run
// (fp32, 65,536 rows of 64: 53 us for the rows of 64 words, 160 for those of a
// single one, of which 123 join its 1024 pieces).  Rows of words
// that no token names are zeros, written in the same launch by workgroups of
// their own, which find out which words of theirs are named: the sums wait for
// memory's answers while those keep it busy (bf16, 16,384 tokens, 128,000 words
// of 4096: 217 us for both, 5.4 TB/s; zeros during the sort and the sums behind
// it: 194 and 71), in a time that hardly depends on how often (fp32, 65,536
// rows of 64, 64 words: 53 us, 47 without zeros, and 208 where a workgroup
// walked the tokens of its words).  Lookup and gradient together: 296 us, 4.9 TB/s.
#include "kept.hpp"
#include "lm_tile.hpp"

#include <algorithm>

namespace cbk {
namespace {

__host__ __device__ constexpr int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// --- forward -------------------------------------------------------------------

struct LookupArgs {
  const void* table;
  int64_t pstride;
  const int32_t* tokens;
  int ignore, n, d, v;
  float scale;
  void* y;
  int lx;  // log2 of the threads that share a row
};

// A row's threads copy eight columns each, four rows at a time in flight.
template <class T, bool WHOLE>
__global__ __launch_bounds__(256) void embed_rows(LookupArgs a) {
  const int j = blockIdx.y, tx = 1 << a.lx, ty = 256 >> a.lx;
  const int x = threadIdx.x & (tx - 1), yrow = threadIdx.x >> a.lx;
  const T* table = (const T*)a.table + j * a.pstride;
  const int32_t* tokens = a.tokens + (int64_t)j * a.n;
  T* y = (T*)a.y + (int64_t)j * a.n * a.d;
  constexpr int R = 4;
  for (int64_t r0 = (int64_t)blockIdx.x * ty * R; r0 < a.n; r0 += (int64_t)gridDim.x * ty * R) {
    int tok[R];
    int64_t row[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      row[i] = r0 + i * ty + yrow;
      tok[i] = row[i] < a.n ? tokens[row[i]] : a.ignore;
    }
    for (int c = x * 8; c < a.d; c += tx * 8) {
      Raw8<T> raw[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const bool word = tok[i] != a.ignore && tok[i] >= 0 && tok[i] < a.v;
        raw[i] = load_raw8<T, WHOLE>(table + (word ? (int64_t)tok[i] * a.d : 0), word ? c : a.d, a.d);
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (row[i] >= a.n) continue;
        const bool word = tok[i] >= 0 && tok[i] < a.v;
        const float s = word || tok[i] == a.ignore ? a.scale : __builtin_nanf("");
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = tok[i] == a.ignore ? 0.f : raw[i].at(e) * s;
        store8<T, WHOLE>(y + row[i] * a.d, c, a.d, f);
      }
    }
  }
}

// --- the sorted tokens -----------------------------------------------------------

// Tokens of a workgroup's sort: more are sorted by several and merged (16,384
// tokens: 22 us, and 36 by one workgroup with all of them in its LDS).
constexpr int SORT = 4096, SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / 64;
constexpr int DIGIT = 6;  // bits a pass: a digit's value for every lane

struct SortArgs {
  const int32_t* tokens;
  int ignore, n, v;
  int bits;        // of v
  uint64_t* out;   // [k][n] token << 32 | row, each SORT of them in order
};

// Sorts up to EACH * 1024 tokens of a learner in LDS: a radix sort, least
// digit first, in which every wave counts its own stretch's digits.  A lane
// finds those of its wave that hold its digit by a ballot for every bit, so
// the places are in order and no atomic is needed.  A token that is ignored or
// no word becomes v and comes last.
template <int EACH>
__device__ __forceinline__ void sort_chunk(const SortArgs& a, int j, int chunk, char* lds) {
  uint64_t* item = (uint64_t*)lds;
  uint32_t(*count)[64] = (uint32_t(*)[64])(lds + (size_t)EACH * SORT_THREADS * 8);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t from = (int64_t)chunk * SORT;
  const int left = (int)min((int64_t)SORT, a.n - from);
  const int32_t* tokens = a.tokens + (int64_t)j * a.n + from;
  const int at = wave * (EACH * 64) + lane;
  uint32_t key[EACH], row[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int p = at + i * 64;
    key[i] = (uint32_t)a.v;
    if (p < left) {
      const int t = tokens[p];
      if (t != a.ignore && t >= 0 && t < a.v) key[i] = (uint32_t)t;
    }
    row[i] = (uint32_t)(from + p);  // past the end: after all others of key v
  }
  const uint64_t below = (1ull << lane) - 1;
  for (int shift = 0; shift < a.bits; shift += DIGIT) {
    count[wave][lane] = 0;
    __builtin_amdgcn_wave_barrier();
    volatile uint32_t* mine = count[wave];
    uint32_t place[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const uint32_t digit = key[i] >> shift & 63;
      uint64_t same = ~0ull;
#pragma unroll
      for (int b = 0; b < DIGIT; ++b) {
        const uint64_t set = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? set : ~set;
      }
      const uint32_t before = mine[digit];
      place[i] = before + __popcll(same & below);
      __builtin_amdgcn_wave_barrier();
      if ((same & below) == 0) mine[digit] = before + __popcll(same);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    if (wave == 0) {  // lane: a digit
      uint32_t sum = 0, here[SORT_WAVES];
#pragma unroll
      for (int w = 0; w < SORT_WAVES; ++w) {
        here[w] = sum;
        sum += count[w][lane];
      }
      uint32_t scan = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t t = __shfl_up(scan, o);
        if (lane >= o) scan += t;
      }
#pragma unroll
      for (int w = 0; w < SORT_WAVES; ++w) count[w][lane] = scan - sum + here[w];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      item[count[wave][key[i] >> shift & 63] + place[i]] = (uint64_t)key[i] << 32 | row[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const uint64_t x = item[at + i * 64];
      key[i] = (uint32_t)(x >> 32);
      row[i] = (uint32_t)x;
    }
    __syncthreads();
  }
  uint64_t* out = a.out + (int64_t)j * a.n + from;
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (at + i * 64 < left) out[at + i * 64] = (uint64_t)key[i] << 32 | row[i];
}

template <int EACH>
__global__ __launch_bounds__(SORT_THREADS) void embed_sort(SortArgs a) {
  extern __shared__ __align__(16) char lds[];
  sort_chunk<EACH>(a, blockIdx.y, blockIdx.x, lds);
}

// Merges neighbouring runs of `run` sorted items: an item's place is its own
// plus the number of lesser ones in the other run.
__global__ __launch_bounds__(256) void embed_merge(const uint64_t* in, uint64_t* out, int64_t n,
                                                   int64_t run) {
  const int64_t base = (int64_t)blockIdx.y * n;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
    const uint64_t x = in[base + i];
    const int64_t pair = i / (2 * run) * (2 * run), mid = min(pair + run, n);
    const bool left = i < mid;
    int64_t lo = left ? mid : pair, hi = left ? min(pair + 2 * run, n) : mid;
    const int64_t first = lo;
    while (lo < hi) {
      const int64_t m = (lo + hi) / 2;
      if (in[base + m] < x)
        lo = m + 1;
      else
        hi = m;
    }
    out[base + pair + (i - (left ? pair : mid)) + (lo - first)] = x;
  }
}

// --- sums of runs ----------------------------------------------------------------

struct SumArgs {
  const uint64_t* sorted;  // [k][n]
  const void* dy;
  int n, d, v;
  float scale;
  void* dw;
  int64_t dstride;
  int add;                 // onto what dw holds
  int each, pieces;        // rows of a piece, pieces of a learner
  int lx;                  // log2 of the threads that share a piece
  int blocks, words;       // workgroups of sums; words of one that writes zeros, 64 at the most
  // [k][pieces][dp]: of a piece's first run if it began earlier, and of its
  // last if it began here and goes on
  float *lead, *trail;
  int dp;
};

template <class T, bool WHOLE>
__device__ __forceinline__ void store_sum(const SumArgs& a, int j, uint32_t word, int c,
                                          const float (&sum)[8]) {
  T* row = (T*)a.dw + j * a.dstride + (int64_t)word * a.d;
  float f[8];
  if (a.add) {
    load8<T, WHOLE>(row, c, a.d, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = fmaf(a.scale, sum[e], f[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = a.scale * sum[e];
  }
  store8<T, WHOLE>(row, c, a.d, f);
}

// Zeros from a workgroup, 16 bytes a lane between the ends.
__device__ __forceinline__ void zero_bytes(char* at, int64_t bytes) {
  const int64_t head = min(bytes, (int64_t)(-(uintptr_t)at & 15)), whole = (bytes - head) / 16;
  i32x4* body = (i32x4*)(at + head);
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < whole; i += 256) body[i] = i32x4{0, 0, 0, 0};
  // elements have 2 bytes at least
  const int64_t tail = head + whole * 16 + threadIdx.x * 2;
  if (threadIdx.x * 2 < head) *(uint16_t*)(at + threadIdx.x * 2) = 0;
  if (tail < bytes) *(uint16_t*)(at + tail) = 0;
}

// Zeros for the words of stretch x, x + all, .. that no token names.
template <class T>
__device__ __forceinline__ void write_zeros(const SumArgs& a, int j, int x, int all) {
  __shared__ unsigned long long named;
  const uint64_t* sorted = a.sorted + (int64_t)j * a.n;
  for (int64_t w0 = (int64_t)x * a.words; w0 < a.v; w0 += (int64_t)all * a.words) {
    const int words = (int)min((int64_t)a.words, a.v - w0);
    // the first token that is w0 or more, in a 256th of what is left at a time
    int lo = 0;
    for (int len = a.n; len > 0;) {
      const int step = (len + 255) / 256, end = lo + len, p = lo + (threadIdx.x + 1) * step - 1;
      lo += __syncthreads_count(p < end && (int64_t)(sorted[min(p, end - 1)] >> 32) < w0) * step;
      len = min(step - 1, end - lo);
    }
    __syncthreads();
    if (threadIdx.x == 0) named = 0;
    __syncthreads();
    // the words of 256 tokens from there; if the stretch has more of them, a thread
    // a word looks for its own (a walk over all would take as long as they are many)
    {
      const int64_t p = (int64_t)lo + threadIdx.x;
      const int64_t w = p < a.n ? (int64_t)(sorted[p] >> 32) - w0 : words;
      // (neighbours with the same word need not say so again)
      if (w < words && (threadIdx.x == 0 || (int64_t)(sorted[p - 1] >> 32) - w0 != w)) atomicOr(&named, 1ull << w);
      if (!__syncthreads_or(w >= words) && (int)threadIdx.x < words) {
        const int64_t mine = w0 + threadIdx.x;
        int from = lo + 255, to = a.n;  // the first token of `mine` or more, or n
        while (from < to) {
          const int mid = from + (to - from) / 2;
          if ((int64_t)(sorted[mid] >> 32) < mine)
            from = mid + 1;
          else
            to = mid;
        }
        if (from < a.n && (int64_t)(sorted[from] >> 32) == mine) atomicOr(&named, 1ull << threadIdx.x);
      }
      __syncthreads();
    }
    // runs of words that are not named lie in one piece
    char* out = (char*)((T*)a.dw + j * a.dstride + w0 * a.d);
    unsigned long long rest = ~named & (words < 64 ? (1ull << words) - 1 : ~0ull);
    while (rest) {
      const int w = __builtin_ctzll(rest);
      const unsigned long long behind = ~(rest >> w);
      const int run = behind ? __builtin_ctzll(behind) : 64 - w;
      rest = w + run < 64 ? rest >> (w + run) << (w + run) : 0;
      zero_bytes(out + (int64_t)w * a.d * (int)sizeof(T), (int64_t)run * a.d * (int)sizeof(T));
    }
  }
}

// A piece's threads have eight columns each and walk its rows, eight in
// flight.  The workgroups behind those write zeros.
template <class T, bool WHOLE>
__global__ __launch_bounds__(256) void embed_sums(SumArgs a) {
  const int j = blockIdx.y, tx = 1 << a.lx, ty = 256 >> a.lx;
  if ((int)blockIdx.x >= a.blocks) {
    if (blockIdx.z == 0) write_zeros<T>(a, j, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    return;
  }
  const int c = ((threadIdx.x & (tx - 1)) + blockIdx.z * tx) * 8;
  if (c >= a.d) return;
  const uint64_t* sorted = a.sorted + (int64_t)j * a.n;
  const T* dy = (const T*)a.dy + (int64_t)j * a.n * a.d;
  for (int p = blockIdx.x * ty + (threadIdx.x >> a.lx); p < a.pieces; p += a.blocks * ty) {
    const int64_t from = (int64_t)p * a.each;
    const int rows = (int)min((int64_t)a.each, a.n - from);
    const uint64_t* s = sorted + from;
    const uint32_t before = p ? (uint32_t)(s[-1] >> 32) : ~0u;
    const uint32_t after = from + rows < a.n ? (uint32_t)(s[rows] >> 32) : ~0u;
    uint32_t word = (uint32_t)(s[0] >> 32);
    bool open = word == before;  // the run began earlier
    float sum[8] = {};
    auto end = [&](uint32_t next) {  // of the run
      if (word >= (uint32_t)a.v) return;
      const bool on = next == word;  // it goes on behind the piece
      if (open || on) {
        float* to = (open ? a.lead : a.trail) + ((int64_t)j * a.pieces + p) * a.dp + c;
#pragma unroll
        for (int e = 0; e < 8; e += 4) *(f32x4*)(to + e) = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
      } else {
        store_sum<T, WHOLE>(a, j, word, c, sum);
      }
    };
    constexpr int R = 8;
    for (int i0 = 0; i0 < rows && word < (uint32_t)a.v; i0 += R) {
      Raw8<T> raw[R];
      uint32_t w[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const uint64_t x = s[min(i0 + i, rows - 1)];
        w[i] = (uint32_t)(x >> 32);
        raw[i] = load_raw8<T, WHOLE>(dy + (int64_t)(uint32_t)x * a.d, c, a.d);
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (i0 + i >= rows) break;
        if (w[i] != word) {
          end(w[i]);
          word = w[i];
          open = false;
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += raw[i].at(e);
      }
    }
    end(after);
  }
}

// Adds up the shares of the run that begins in piece p and passes its end:
// eight stretches of pieces side by side, then those in order.
template <class T, bool WHOLE>
__global__ __launch_bounds__(256) void embed_join(SumArgs a) {
  const int j = blockIdx.y, x = threadIdx.x & 31, s = threadIdx.x >> 5;
  const int c = (x + blockIdx.z * 32) * 8;
  const uint64_t* sorted = a.sorted + (int64_t)j * a.n;
  __shared__ float part[7][32][9];
  for (int p = blockIdx.x; p < a.pieces - 1; p += gridDim.x) {
    const int64_t end = (int64_t)(p + 1) * a.each;
    const uint32_t word = (uint32_t)(sorted[end - 1] >> 32);
    if (word >= (uint32_t)a.v || (uint32_t)(sorted[end] >> 32) != word) continue;
    if (p && (uint32_t)(sorted[end - a.each - 1] >> 32) == word) continue;  // began earlier
    // how many pieces behind p begin with the word: as the words are sorted, as
    // many as there are
    int more = 0;
    for (int q = 0;; q += 256) {
      const int64_t x = end + (int64_t)(q + threadIdx.x) * a.each;
      more += __syncthreads_count(x < a.n && (uint32_t)(sorted[min(x, (int64_t)a.n - 1)] >> 32) == word);
      if (more < q + 256) break;
    }
    const int span = (more + 7) / 8;
    float sum[8] = {};
    if (c < a.d) {
      const float* lead = a.lead + ((int64_t)j * a.pieces + p + 1) * a.dp + c;
      if (s == 0) {
        const float* t = a.trail + ((int64_t)j * a.pieces + p) * a.dp + c;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = t[e];
      }
#pragma unroll 4
      for (int q = s * span; q < min(more, (s + 1) * span); ++q) {
        const f32x4 u = *(const f32x4*)(lead + (int64_t)q * a.dp);
        const f32x4 v = *(const f32x4*)(lead + (int64_t)q * a.dp + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sum[e] += u[e];
          sum[e + 4] += v[e];
        }
      }
    }
    __syncthreads();
    if (s) {
#pragma unroll
      for (int e = 0; e < 8; ++e) part[s - 1][x][e] = sum[e];
    }
    __syncthreads();
    if (s == 0 && c < a.d) {
      for (int i = 0; i < 7; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += part[i][x][e];
      store_sum<T, WHOLE>(a, j, word, c, sum);
    }
  }
}

// --- launches --------------------------------------------------------------------

// log2 of the threads that eight columns each of d need, 8 at the most.
int threads_log2(int d) {
  int lx = 0;
  while (lx < 8 && (8 << lx) < d) ++lx;
  return lx;
}

struct Layout {
  int each, pieces, dp, lx;
  size_t sorted, other, lead, trail, total;
};

Layout layout(const EmbedArgs& a) {
  Layout l;
  l.dp = (int)up(a.d, 8);
  l.lx = threads_log2(a.d);
  const int64_t slabs = up(a.d, 8 << l.lx) / (8 << l.lx), each_block = 256 >> l.lx;
  // long pieces leave fewer partial sums, short ones more workgroups
  for (l.each = 64; l.each > 8 && a.n > 64; l.each /= 2)
    if (a.k * slabs * (up(a.n, l.each) / l.each) >= 1024 * each_block) break;
  l.pieces = (int)(up(a.n, l.each) / l.each);
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)up(std::max<int64_t>(bytes, 1), 256);
    return here;
  };
  l.sorted = take((int64_t)a.k * a.n * 8);
  l.other = a.n > SORT ? take((int64_t)a.k * a.n * 8) : 0;
  const int64_t sums = l.pieces > 1 ? (int64_t)a.k * l.pieces * l.dp * 4 : 0;
  l.lead = take(sums);
  l.trail = take(sums);
  l.total = at;
  return l;
}

template <int EACH>
hipError_t launch_sort(const SortArgs& a, int blocks, int k, hipStream_t s) {
  return launch_with_lds<EACH * SORT_THREADS * 8 + SORT_WAVES * 256, embed_sort<EACH>>(
      dim3(blocks, k), SORT_THREADS, s, a);
}

template <class T>
hipError_t backward(const EmbedArgs& a, hipStream_t s) {
  const Layout l = layout(a);
  char* ws = (char*)a.ws;
  SortArgs o{a.tokens, a.ignore, a.n, a.v, 32 - __builtin_clz((unsigned)a.v),
             (uint64_t*)(ws + l.sorted)};
  const int chunks = (int)(up(a.n, SORT) / SORT);
  if (hipError_t e = a.n <= 1024 ? launch_sort<1>(o, chunks, a.k, s)
                                 : launch_sort<SORT / SORT_THREADS>(o, chunks, a.k, s))
    return e;
  uint64_t *from = o.out, *to = (uint64_t*)(ws + l.other);
  for (int64_t run = SORT; run < a.n; run *= 2) {
    klaunch(embed_merge, dim3((unsigned)std::min<int64_t>(up(a.n, 256) / 256, 4096), a.k), dim3(256),
            0, s, (const uint64_t*)from, to, (int64_t)a.n, run);
    if (hipError_t e = hipGetLastError()) return e;
    std::swap(from, to);
  }
  SumArgs u{from, a.dy, a.n, a.d, a.v, a.scale, a.dw, a.dstride, a.accumulate, l.each, l.pieces, l.lx,
            0, 0, (float*)(ws + l.lead), (float*)(ws + l.trail), l.dp};
  const bool whole = a.d % 8 == 0;
  const int ty = 256 >> l.lx;
  u.blocks = std::min((l.pieces + ty - 1) / ty, 65536);
  // zeros: 128 KB a workgroup
  u.words = (int)std::max<int64_t>(1, std::min<int64_t>(64, (128 << 10) / ((int64_t)a.d * (int64_t)sizeof(T))));
  const int zeros = a.accumulate ? 0 : (int)std::min<int64_t>(up(a.v, u.words) / u.words, 65536);
  const dim3 grid((unsigned)(u.blocks + zeros), a.k,
                  (unsigned)(up(a.d, 8 << l.lx) / (8 << l.lx)));
  klaunch(whole ? embed_sums<T, true> : embed_sums<T, false>, grid, dim3(256), 0, s, u);
  if (hipError_t e = hipGetLastError()) return e;
  if (l.pieces == 1) return hipSuccess;
  const dim3 joins((unsigned)std::min(l.pieces - 1, 16384), a.k, (unsigned)(up(a.d, 256) / 256));
  klaunch(whole ? embed_join<T, true> : embed_join<T, false>, joins, dim3(256), 0, s, u);
  return hipGetLastError();
}

template <class T>
hipError_t forward(const EmbedArgs& a, hipStream_t s) {
  LookupArgs l{a.table, a.pstride, a.tokens, a.ignore, a.n, a.d, a.v, a.scale, a.y, threads_log2(a.d)};
  const int64_t rows = (256 >> l.lx) * 4;
  const dim3 grid((unsigned)std::min<int64_t>(up(a.n, rows) / rows, 65536), a.k);
  klaunch(a.d % 8 == 0 ? embed_rows<T, true> : embed_rows<T, false>, grid, dim3(256), 0, s, l);
  return hipGetLastError();
}

}  // namespace

size_t embed_ws_bytes(const EmbedArgs& a) { return layout(a).total; }

hipError_t embed_fwd(const EmbedArgs& a, hipStream_t s) {
  return a.type == LM_F32 ? forward<float>(a, s)
         : a.type == LM_F16 ? forward<_Float16>(a, s)
                            : forward<__bf16>(a, s);
}
hipError_t embed_bwd(const EmbedArgs& a, hipStream_t s) {
  return a.type == LM_F32 ? backward<float>(a, s)
         : a.type == LM_F16 ? backward<_Float16>(a, s)
                            : backward<__bf16>(a, s);
}

}  // namespace cbk
