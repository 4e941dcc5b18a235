// ckpt.hip -- activations kept in 8 bits between the forward and the backward
// pass (kept.hpp has the format), and the weight gradient of the layer that
// read them, taken from the 8 bits.
//
// kept_pack and kept_unpack stream: eight columns a thread, four
// neighbouring threads to a group of 32.  16,384 x 4096, bf16 (203 MB each
// way): 42 and 30 us, 4.8 and 6.7 TB/s, the 8-bit form being in the caches.
//
// The weight gradient dW[o][c] = sum_r dy[r][o] x[r][c] runs on the tiles of
// lm_tile.hpp, with P = x (p = c) and Q = dy (q = o), both in col form; every
// q * 2^e is a 16-bit number exactly, so x is not rounded again.
//   Small layers (tiles of 128): x is read as bytes and powers of two, 16
// columns a thread, one step ahead into registers, converted and written to
// LDS in the layout that dy's loads have there.  One launch, and for fp32
// three MFMAs a product instead of six: x is one bf16 number, dy three.
//   Large layers (tiles of 256; 8192 rows, 2048 x 8192, bf16: 197 us in the
// long run, 1,390 TFLOP/s, and 222 to 267 us in the first milliseconds under
// load, when the card's clock is lower): x is unpacked once into the
// workspace, and the tiles take both operands straight to LDS.  Converting in
// every one of the out/256 workgroups that read a tile of x costs more (240 us
// there against 216 us and 11 us for the unpacking, side by side).
//   Where the tiles do not fill the CUs, or the last round of them leaves most
// idle, that round's tiles are shared by workgroups that take some of the rows
// each, and kept_grad_join adds their sums in order.
#include "kept.hpp"
#include "lm_tile.hpp"

#include <algorithm>
#include <type_traits>

namespace cbk {
namespace {

// x [rows][d] to q and group bytes.
template <class T, bool WHOLE>
__global__ __launch_bounds__(256) void kept_pack_k(const T* x, int64_t rows, int d, char* q,
                                                   uint8_t* e) {
  const int64_t dp = kept_dp(d), units = rows * (dp / 8);
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < units; i += gridDim.x * 256ll) {
    const int64_t r = i / (dp / 8);
    const int c = (int)(i - r * (dp / 8)) * 8;
    float v[8];
    load8<T, WHOLE>(x + r * d, c, d, v);
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) most = max(most, abs_bits(v[k]));
    most = max(most, (uint32_t)__shfl_xor((int)most, 1));
    most = max(most, (uint32_t)__shfl_xor((int)most, 2));
    const int byte = kept_byte<T>(most);
    *(uint64_t*)(q + r * dp + c) = kept_pack8<T>(v, byte);
    if ((c & 31) == 0) e[r * (dp / 32) + c / 32] = byte;
  }
}

// and back, to rows ld apart (zeros between)
template <class T, bool WHOLE>
__global__ __launch_bounds__(256) void kept_unpack_k(const char* q, const uint8_t* e, int64_t rows,
                                                     int d, T* x, int64_t ld) {
  const int64_t dp = kept_dp(d), units = rows * (dp / 8);
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < units; i += gridDim.x * 256ll) {
    const int64_t r = i / (dp / 8);
    const int c = (int)(i - r * (dp / 8)) * 8;
    const uint64_t b = *(const uint64_t*)(q + r * dp + c);
    const float s = kept_scale(e[r * (dp / 32) + c / 32]);
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)(int8_t)(b >> (8 * k)) * s;
    store8<T, WHOLE>(x + r * ld, c, (int)ld, v);
  }
}

// Rows of dy that do not start on 16 bytes, copied to ones that do.
template <class T>
__global__ __launch_bounds__(256) void copy_rows(const T* x, int64_t rows, int d, int dp, T* y) {
  const int64_t units = rows * (dp / 8);
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < units; i += gridDim.x * 256ll) {
    const int64_t r = i / (dp / 8);
    const int c = (int)(i - r * (dp / 8)) * 8;
    const Raw8<T> v = load_raw8<T, false>(x + r * d, c, d);
    __builtin_memcpy(y + r * dp + c, v.w, sizeof(v.w));
  }
}

struct GradArgs {
  const void* x;     // unpacked rows, ldx apart (tiles of 256)
  int64_t ldx;
  const char* q;     // [k*n] rows of dp bytes
  const uint8_t* e;  // [k*n] rows of dp / 32 powers
  int64_t dp;
  const void* dy;    // [k*n] rows, ldy apart
  int64_t ldy;
  int n, d, out;
  int full, tail;    // tiles that one workgroup takes, and that `splits` share
  int splits, span;  // rows that each of these takes
  void* dw;
  int64_t dstride;
  int vec;
  float* part;       // [splits][tail] tiles of sums
};

template <class T_, int BP_, int BQ_, int WP_, int WQ_>
struct KeptTile {
  using T = T_;
  using Base = Tile<T, true, true, BP_, BQ_, WP_, WQ_>;
  using Half = std::conditional_t<__is_same(T, _Float16), _Float16, __bf16>;  // x in LDS
  static constexpr int BP = BP_, BQ = BQ_, WP = WP_, WQ = WQ_, THREADS = Base::THREADS;
  static constexpr int SP = Base::SP, SQ = Base::SQ, TP = Base::TP, TQ = Base::TQ, BK = Base::BK;
  static constexpr int XBYTES = BK * BP * 2, STAGE = XBYTES + BQ * 128, LDS = 2 * STAGE;
  static constexpr int UPR = BP / 16, UNITS = BK * UPR / THREADS;  // 16 columns each
  static_assert(UNITS * THREADS == BK * UPR, "whole units");
  using Acc = typename Base::Acc;

  // One thread's share of a step's x, as bytes, and where the next step's lie.
  // Rows and columns past the end read as zeros (buffer range check).
  struct Bytes {
    i32x4 q[UNITS];
    int e[UNITS];
    uint32_t off[UNITS];  // of q, 32 times that of the group's byte
    const char *qat, *eat;
    int64_t rows, dp;  // rows left
  };
  static __device__ __forceinline__ void start(const GradArgs& a, int j, int p0, int r0, int r1,
                                               Bytes& b) {
    const int64_t row = (int64_t)j * a.n + r0;
    b.dp = a.dp;
    b.qat = a.q + row * a.dp;
    b.eat = (const char*)a.e + row * (a.dp / KEPT_GROUP);
    b.rows = r1 - r0;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int id = u * THREADS + threadIdx.x, r = id / UPR, c = p0 + id % UPR * 16;
      b.off[u] = c < a.dp ? (uint32_t)(r * a.dp + c) : OUTSIDE;
    }
  }
  static __device__ __forceinline__ void fetch(Bytes& b) {
    const int64_t rows = b.rows < 0 ? 0 : b.rows < BK ? b.rows : BK;
    const auto q = buf_rsrc_u(reinterpret_cast<const float*>(b.qat), (uint32_t)(rows * b.dp));
    const auto e = buf_rsrc_u(reinterpret_cast<const float*>(b.eat),
                              (uint32_t)(rows * (b.dp / KEPT_GROUP)));
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      b.q[u] = __builtin_bit_cast(i32x4,
                                  __builtin_amdgcn_raw_buffer_load_b128(q, b.off[u], 0, 0));
      b.e[u] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(e, b.off[u] / KEPT_GROUP, 0, 0);
    }
    b.qat += BK * b.dp;
    b.eat += BK * (b.dp / KEPT_GROUP);
    b.rows -= BK;
  }
  static __device__ __forceinline__ void put(const Bytes& b, lds_char* lds) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int id = u * THREADS + threadIdx.x, row = id / UPR, c = id % UPR * 2;
      const float s = kept_scale(b.e[u]);
      const int swz = col_swizzle<BP * 2 / 16>(row);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        typedef Half half2v __attribute__((ext_vector_type(2)));
        i32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // the product alone, which is exact at every 2^e: 128 * 2^e, that an
          // offset of the bytes would bring in, is past fp32's largest value
          // for the two largest e
          const uint32_t w = (uint32_t)b.q[u][2 * h + i / 2];
          const int sh = i % 2 * 16;
          const float x0 = (float)(int8_t)(w >> sh) * s;
          const float x1 = (float)(int8_t)(w >> (sh + 8)) * s;
          if constexpr (__is_same(Half, __bf16)) {
            o[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, x1),
                                         __builtin_bit_cast(uint32_t, x0), 0x07060302);
          } else {
            const half2v v = {(Half)x0, (Half)x1};
            o[i] = __builtin_bit_cast(int, v);
          }
        }
        *(__attribute__((address_space(3))) i32x4*)(lds + row * (BP * 2) + ((c + h) ^ swz) * 16) =
            o;
      }
    }
  }

  // The sum over rows [r0, r1) of learner j; r0 a multiple of BK.
  static __device__ __forceinline__ void product(const GradArgs& a, int j, int p0, int q0, int r0,
                                                 int r1, char* lds, Acc& acc) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wp = (wave / WQ) * SP, wq = (wave % WQ) * SQ;
    const Operand<T> Y{(const T*)a.dy + (int64_t)j * a.n * a.ldy, a.ldy, a.out, r1};
    Loader<T, BQ, true, THREADS> ly;
    ly.init(Y, q0, r0, threadIdx.x);
#pragma unroll
    for (int x = 0; x < TP; ++x)
#pragma unroll
      for (int b = 0; b < TQ; ++b) acc[x][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int steps = (r1 - r0 + BK - 1) / BK;
    if (steps <= 0) return;
    lds_char* l = (lds_char*)lds;
    const uint32_t la = (uint32_t)(uintptr_t)l;
    Bytes b;
    start(a, j, p0, r0, r1, b);
    fetch(b);
    ly.issue(la + XBYTES);
    put(b, l);
    fetch(b);
    tile_wait_barrier();
    put(b, l + STAGE);
    ly.issue(la + STAGE + XBYTES);
    fetch(b);
    // After the barrier in step s nothing of it is left to read in LDS: dy of
    // step s + 2 is sent there at once, x after the other buffer's reads (the
    // compiler keeps LDS writes behind reads that come before them), so that
    // its conversion spreads over the MFMAs.  No branch for the last steps:
    // their rows read as zeros.
    auto send = [&](uint32_t cur) {
      // the bytes are there: the barrier has waited for them; said here, so
      // that the compiler does not wait again, for the loads that come next
#pragma unroll
      for (int u = 0; u < UNITS; ++u) asm volatile("" : "+v"(b.q[u]), "+v"(b.e[u]));
      ly.issue(la + cur + XBYTES);
    };
    auto refill = [&](uint32_t cur) {
      put(b, l + cur);
      fetch(b);
    };
    if constexpr (sizeof(T) == 2) {
      i32x4 fp[TP], fq[TQ];
      read_frags<T, BP, true, TP>(l, wp, 0, lane, fp);
      read_frags<T, BQ, true, TQ>(l + XBYTES, wq, 0, lane, fq);
      for (int s = 0; s < steps; ++s) {
        const uint32_t cur = (s & 1) * STAGE, nxt = STAGE - cur;
        mma_step<T, BP, true, BQ, true, 0>(acc, fp, fq, l + cur, l + cur + XBYTES, wp, wq, 1,
                                            lane);
        tile_wait_barrier();
        send(cur);
        mma_step<T, BP, true, BQ, true, 16 * UNITS>(acc, fp, fq, l + nxt, l + nxt + XBYTES, wp, wq,
                                                     0, lane);
        refill(cur);
      }
    } else {
      // a lane's eight k: 4g..4g+3 and 16 + 4g..16 + 4g+3, as dy's floats come
      i32x4 fp[TP], fq[2][TQ];
      auto read = [&](const lds_char* at) {
#pragma unroll
        for (int t = 0; t < TP; ++t)
          fp[t] = read_transposed<BP>(at, wp + t * 16, 4 * (lane >> 4), 16, lane);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
          read_frags<T, BQ, true, TQ>(at + XBYTES, wq, kk, lane, fq[kk]);
      };
      read(l);
      for (int s = 0; s < steps; ++s) {
        const uint32_t cur = (s & 1) * STAGE, nxt = STAGE - cur;
        i32x4 x[TP];
        Split3 y[TQ];
#pragma unroll
        for (int t = 0; t < TP; ++t) x[t] = fp[t];
#pragma unroll
        for (int t = 0; t < TQ; ++t) y[t] = split3(fq[0][t], fq[1][t]);
        tile_wait_barrier();
        send(cur);
        read(l + nxt);
#pragma unroll
        for (int t = 0; t < TP; ++t)
#pragma unroll
          for (int o = 0; o < TQ; ++o) {
            acc[t][o] = mma<__bf16>(x[t], y[o].l, acc[t][o]);
            acc[t][o] = mma<__bf16>(x[t], y[o].m, acc[t][o]);
            acc[t][o] = mma<__bf16>(x[t], y[o].h, acc[t][o]);
          }
        refill(cur);
      }
    }
    tile_wait_barrier();  // loads into LDS end before the workgroup does
  }
};

// The same product of unpacked rows.
template <class T_>
struct PlainTile : BigTile<T_, true, true> {
  using Base = BigTile<T_, true, true>;
  static __device__ __forceinline__ void product(const GradArgs& a, int j, int p0, int q0, int r0,
                                                 int r1, char* lds, typename Base::Acc& acc) {
    const Operand<T_> X{(const T_*)a.x + (int64_t)j * a.n * a.ldx, a.ldx, (int)a.ldx, a.n};
    const Operand<T_> Y{(const T_*)a.dy + (int64_t)j * a.n * a.ldy, a.ldy, a.out, a.n};
    Base::product(X, Y, p0, q0, r0, r1, lds, acc);
  }
};

// The learner and the place of tile x of all learners'.
template <class TL>
__device__ __forceinline__ void tile_at(const GradArgs& a, int x, int& j, int& p0, int& q0) {
  const int np = (a.d + TL::BP - 1) / TL::BP, nq = (a.out + TL::BQ - 1) / TL::BQ;
  int tp, tq;
  j = x / (np * nq);
  tile_of<8>(x - j * np * nq, np, nq, tp, tq);
  p0 = tp * TL::BP;
  q0 = tq * TL::BQ;
}

template <class TL>
__global__ __launch_bounds__(TL::THREADS, 2) void kept_grad_k(GradArgs a) {
  using T = typename TL::T;
  extern __shared__ __align__(16) char lds[];
  int x = blockIdx.x, r0 = 0, r1 = a.n;
  float* part = nullptr;
  if (x >= a.full) {
    const int s = (x - a.full) / a.tail, t = (x - a.full) % a.tail;
    r0 = s * a.span;
    r1 = min(r0 + a.span, a.n);
    part = a.part + (int64_t)(x - a.full) * (TL::BP * TL::BQ);
    x = a.full + t;
  }
  int j, p0, q0;
  tile_at<TL>(a, x, j, p0, q0);
  typename TL::Acc acc;
  TL::product(a, j, p0, q0, r0, r1, lds, acc);
  T* out = (T*)a.dw + j * a.dstride;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wp = (wave / TL::WQ) * TL::SP, wq = (wave % TL::WQ) * TL::SQ;
#pragma unroll
  for (int y = 0; y < TL::TQ; ++y) {
    const int q = wq + TL::Base::col_of(y, lane);
#pragma unroll
    for (int t = 0; t < TL::TP; ++t) {
      const int p = wp + t * 16 + 4 * (lane >> 4);
      if (part)
        *(f32x4*)(part + q * TL::BP + p) = acc[t][y];
      else if (q0 + q < a.out && p0 + p < a.d)
        store4<T>(out + (int64_t)(q0 + q) * a.d + p0 + p, acc[t][y], 1.f, a.d - p0 - p, a.vec);
    }
  }
}

// The shared tiles' sums in order: blockIdx.y is the tile, 1024 of its values
// a workgroup.
template <class TL>
__global__ __launch_bounds__(256) void kept_grad_join(GradArgs a) {
  using T = typename TL::T;
  int j, p0, q0;
  tile_at<TL>(a, a.full + blockIdx.y, j, p0, q0);
  const int at = (blockIdx.x * 256 + threadIdx.x) * 4;
  const int p = p0 + at % TL::BP, q = q0 + at / TL::BP;
  if (p >= a.d || q >= a.out) return;
  const float* from = a.part + (int64_t)blockIdx.y * (TL::BP * TL::BQ) + at;
  f32x4 v = *(const f32x4*)from;
#pragma unroll 4
  for (int s = 1; s < a.splits; ++s)
    v += *(const f32x4*)(from + (int64_t)s * a.tail * (TL::BP * TL::BQ));
  store4<T>((T*)a.dw + j * a.dstride + (int64_t)q * a.d + p, v, 1.f, a.d - p, a.vec);
}

template <class T>
using Big = PlainTile<T>;
template <class T>
using Mid = KeptTile<T, 128, 128, 2, 2>;

int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
int64_t tiles(int64_t a, int64_t b, int t) { return up(a, t) / t * (up(b, t) / t); }

struct Layout {
  bool big;
  int full, tail, splits, span;
  int64_t ldx, ldy;
  bool copy_dy;
  size_t x, dy, part, total;  // total 0: a launch would not hold its workgroups
};

Layout layout(const KeptGradArgs& a) {
  const int sz = lm_size(a.type), bk = 128 / sz;
  Layout l;
  // tiles of 256 where they fill the 256 CUs; fp32, whose operands take more
  // registers, has tiles of 128 only
  l.big = a.type != LM_F32 && a.k * tiles(a.d, a.out, 256) >= 256;
  const int64_t side = l.big ? 256 : 128, slots = l.big ? 256 : 512;
  const int64_t t = a.k * tiles(a.d, a.out, side), steps = up(a.n, bk) / bk;
  // Behind full rounds the joining has to be worth it: from twelve steps on
  // (bf16, 4096 x 4352, 16 tiles behind 256: 16,384 rows 567 us against 831 in
  // two rounds, 1100 rows 71 against 81, 800 rows 59 against 65; 2048 x
  // 11,008, 88 behind 256, 700 rows: 61 against 58).
  const int64_t full = t / slots * slots, tail = t - full;
  l.splits = 1;
  if (tail && (!full || steps >= 12))
    l.splits = (int)std::max<int64_t>(1, std::min(slots / tail, steps / 4));
  l.span = (int)up((a.n + l.splits - 1) / l.splits, bk);
  l.splits = (a.n + l.span - 1) / l.span;
  l.full = (int)(l.splits > 1 ? full : t);
  l.tail = (int)(t - l.full);
  l.ldy = up(a.out, 8);
  l.copy_dy = a.out * sz % 16 || (uintptr_t)a.dy % 16;
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)up(bytes, 256);
    return here;
  };
  l.ldx = up(a.d, 8);
  l.x = l.big ? take((int64_t)a.k * a.n * l.ldx * sz) : 0;
  l.part = l.tail ? take(l.splits * l.tail * side * side * 4) : 0;
  l.dy = l.copy_dy ? take((int64_t)a.k * a.n * l.ldy * sz) : 0;
  l.total = launch_holds(full + l.splits * tail, l.big ? 512 : 256) ? std::max<size_t>(at, 256) : 0;
  return l;
}

unsigned blocks_of(int64_t units) { return (unsigned)std::min<int64_t>((units + 255) / 256, 8192); }

template <class T>
hipError_t unpack(int64_t rows, int d, const void* kept, void* x, int64_t ld, hipStream_t s) {
  const int64_t dp = kept_dp(d);
  klaunch(ld % 8 ? kept_unpack_k<T, false> : kept_unpack_k<T, true>,
          dim3(blocks_of(rows * (dp / 8))), dim3(256), 0, s, (const char*)kept,
          (const uint8_t*)kept + rows * dp, rows, d, (T*)x, ld);
  return hipGetLastError();
}

template <class T>
hipError_t pack(int64_t rows, int d, const void* x, void* kept, hipStream_t s) {
  const int64_t dp = kept_dp(d);
  klaunch(d % 8 ? kept_pack_k<T, false> : kept_pack_k<T, true>, dim3(blocks_of(rows * (dp / 8))),
          dim3(256), 0, s, (const T*)x, rows, d, (char*)kept, (uint8_t*)kept + rows * dp);
  return hipGetLastError();
}

template <class TL>
hipError_t launch_grad(const GradArgs& g, hipStream_t s) {
  const dim3 grid(g.full + g.tail * g.splits);
  if (hipError_t e = launch_with_lds<TL::LDS, kept_grad_k<TL>>(grid, TL::THREADS, s, g)) return e;
  if (!g.tail) return hipSuccess;
  klaunch(kept_grad_join<TL>, dim3(TL::BP * TL::BQ / 1024, g.tail), dim3(256), 0, s, g);
  return hipGetLastError();
}

template <class T>
hipError_t grad(const KeptGradArgs& a, hipStream_t s) {
  static_assert(Big<_Float16>::BP == 256 && Big<_Float16>::BQ == 256 && Mid<T>::BP == 128 &&
                Mid<T>::BQ == 128 && Big<_Float16>::THREADS == 512 && Mid<T>::THREADS == 256,
                "as layout() counts them");
  const Layout l = layout(a);
  char* ws = (char*)a.ws;
  GradArgs g;
  g.dp = kept_dp(a.d);
  g.q = (const char*)a.kept;
  g.e = (const uint8_t*)a.kept + (int64_t)a.k * a.n * g.dp;
  g.x = ws + l.x;
  g.ldx = l.ldx;
  if (l.big)
    if (hipError_t e = unpack<T>((int64_t)a.k * a.n, a.d, a.kept, ws + l.x, l.ldx, s)) return e;
  g.dy = a.dy;
  g.ldy = a.out;
  if (l.copy_dy) {
    klaunch(copy_rows<T>, dim3(blocks_of((int64_t)a.k * a.n * (l.ldy / 8))), dim3(256), 0, s,
            (const T*)a.dy, (int64_t)a.k * a.n, a.out, (int)l.ldy, (T*)(ws + l.dy));
    if (hipError_t e = hipGetLastError()) return e;
    g.dy = ws + l.dy;
    g.ldy = l.ldy;
  }
  g.n = a.n;
  g.d = a.d;
  g.out = a.out;
  g.full = l.full;
  g.tail = l.tail;
  g.splits = l.splits;
  g.span = l.span;
  g.dw = a.dw;
  g.dstride = a.dstride;
  g.vec = a.d % 4 == 0 && (uintptr_t)a.dw % (4 * sizeof(T)) == 0 && a.dstride % 4 == 0;
  g.part = (float*)(ws + l.part);
  if constexpr (sizeof(T) == 2)
    if (l.big) return launch_grad<Big<T>>(g, s);
  return launch_grad<Mid<T>>(g, s);
}

}  // namespace

size_t kept_bytes(int64_t rows, int d) {
  return (size_t)up(rows * kept_dp(d) / 32 * 33, 16);
}
hipError_t kept_pack(int type, int64_t rows, int d, const void* x, void* kept, hipStream_t s) {
  return type == LM_F32 ? pack<float>(rows, d, x, kept, s)
         : type == LM_F16 ? pack<_Float16>(rows, d, x, kept, s)
                          : pack<__bf16>(rows, d, x, kept, s);
}
hipError_t kept_unpack(int type, int64_t rows, int d, const void* kept, void* x, hipStream_t s) {
  return type == LM_F32 ? unpack<float>(rows, d, kept, x, d, s)
         : type == LM_F16 ? unpack<_Float16>(rows, d, kept, x, d, s)
                          : unpack<__bf16>(rows, d, kept, x, d, s);
}
size_t kept_grad_ws_bytes(const KeptGradArgs& a) { return layout(a).total; }
hipError_t kept_grad(const KeptGradArgs& a, hipStream_t s) {
  return a.type == LM_F32 ? grad<float>(a, s)
         : a.type == LM_F16 ? grad<_Float16>(a, s)
                            : grad<__bf16>(a, s);
}

}  // namespace cbk
