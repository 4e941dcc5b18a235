// ckpt.hip -- activations kept in 8 bits between the forward and the backward
// pass (kept.hpp has the format), and the weight gradient of the layer that
// read them, taken from the 8 bits.
//
// kept_pack and kept_unpack stream: eight columns a thread, four
// neighbouring threads to a group of 32.
#include "kept.hpp"
#include "lm_tile.hpp"

#include <algorithm>

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

// and back: [rows][d], or with ld > d rows that far apart, zeros between
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

template <class T>
__global__ __launch_bounds__(256) void copy_rows(const T* x, int64_t rows, int d, int dp, T* y) {
  const int lane = threadIdx.x & 63;
  for (int64_t r = blockIdx.x * 4ll + (threadIdx.x >> 6); r < rows; r += gridDim.x * 4ll)
    for (int c = lane; c < dp; c += 64) y[r * dp + c] = c < d ? x[r * d + c] : (T)0.f;
}

struct GradArgs {
  const void* x;     // [k*n] rows, ldx apart
  int64_t ldx;
  const void* dy;    // [k*n] rows, ldy apart
  int64_t ldy;
  int n, d, out, span;
  void* dw;
  int64_t dstride;
  int vec;
  float* part;       // [splits][k][out][up4(d)] where the rows are split
};

// dW[o][c] = sum_r dy[r][o] x[r][c]: P = x (p = c), Q = dy (q = o), both in
// col form.
template <class TL>
__global__ __launch_bounds__(TL::THREADS) void kept_grad_k(GradArgs a) {
  using T = typename TL::T;
  extern __shared__ __align__(16) char lds[];
  const int j = blockIdx.y, s = blockIdx.z;
  const int np = (a.d + TL::BP - 1) / TL::BP;
  int tp, tq;
  tile_of<8>(blockIdx.x, np, gridDim.x / np, tp, tq);
  const int p0 = tp * TL::BP, q0 = tq * TL::BQ;
  const Operand<T> X{(const T*)a.x + (int64_t)j * a.n * a.ldx, a.ldx, a.d, a.n};
  const Operand<T> Y{(const T*)a.dy + (int64_t)j * a.n * a.ldy, a.ldy, a.out, a.n};
  typename TL::Acc acc;
  TL::product(X, Y, p0, q0, min(s * a.span, a.n), min((s + 1) * a.span, a.n), lds, acc);
  const int64_t d4 = (a.d + 3) / 4 * 4;
  float* part = a.part ? a.part + ((int64_t)s * gridDim.y + j) * a.out * d4 : nullptr;
  T* out = (T*)a.dw + j * a.dstride;
  TL::for_each_quad(acc, [&](int p, int q, f32x4 v) {
    if (q0 + q >= a.out || p0 + p >= a.d) return;
    if (part) {
      *(f32x4*)(part + (q0 + q) * d4 + p0 + p) = v;
      return;
    }
    T* at = out + (int64_t)(q0 + q) * a.d + p0 + p;
    T o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = from_f32<T>(v[i]);
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

// The splits' sums in order.
template <class T>
__global__ __launch_bounds__(256) void kept_grad_join(const float* part, int splits, int out,
                                                      int d, T* dw, int64_t dstride) {
  const int j = blockIdx.y;
  const int64_t d4 = (d + 3) / 4 * 4, all = (int64_t)gridDim.y * out * d4;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < (int64_t)out * d; i += gridDim.x * 256ll) {
    const int64_t q = i / d, p = i - q * d;
    const float* at = part + ((int64_t)j * out + q) * d4 + p;
    float v = 0.f;
    for (int s = 0; s < splits; ++s) v += at[s * all];
    dw[j * dstride + i] = from_f32<T>(v);
  }
}

template <class T>
using Big = Tile<T, true, true, 256, 256, 2, 4>;
template <class T>
using Mid = Tile<T, true, true, 128, 128, 2, 2>;

int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
int64_t tiles(int64_t a, int64_t b, int t) { return up(a, t) / t * (up(b, t) / t); }

struct Layout {
  bool big;
  int splits, span;
  int64_t ldx, ldy;
  size_t x, dy, part, total;
};

Layout layout(int type, int k, int n, int d, int out) {
  const int sz = lm_size(type);
  Layout l;
  l.big = k * tiles(d, out, 256) >= 256;
  const int64_t t = k * tiles(d, out, l.big ? 256 : 128), steps = up(n, 128 / sz) / (128 / sz);
  l.splits = (int)std::max<int64_t>(1, std::min<int64_t>((l.big ? 256 : 512) / t, steps / 4));
  l.span = (int)up((n + l.splits - 1) / l.splits, 128 / sz);
  l.splits = (n + l.span - 1) / l.span;
  l.ldx = up(d, 16 / sz);
  l.ldy = up(out, 16 / sz);
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)up(std::max<int64_t>(bytes, 1), 256);
    return here;
  };
  l.x = take((int64_t)k * n * l.ldx * sz);
  l.part = l.splits > 1 ? take((int64_t)l.splits * k * out * up(d, 4) * 4) : 0;
  l.dy = take((int64_t)k * n * l.ldy * sz);
  l.total = at;
  return l;
}

unsigned blocks_of(int64_t units) { return (unsigned)std::min<int64_t>((units + 255) / 256, 8192); }

template <class T>
hipError_t unpack(int64_t rows, int d, const void* kept, T* x, int64_t ld, hipStream_t s) {
  const int64_t dp = kept_dp(d);
  klaunch(ld % 8 ? kept_unpack_k<T, false> : kept_unpack_k<T, true>,
          dim3(blocks_of(rows * (dp / 8))), dim3(256), 0, s, (const char*)kept,
          (const uint8_t*)kept + rows * dp, rows, d, x, ld);
  return hipGetLastError();
}

template <class T>
hipError_t pack(int64_t rows, int d, const void* x, void* kept, hipStream_t s) {
  const int64_t dp = kept_dp(d);
  klaunch(d % 8 ? kept_pack_k<T, false> : kept_pack_k<T, true>, dim3(blocks_of(rows * (dp / 8))),
          dim3(256), 0, s, (const T*)x, rows, d, (char*)kept, (uint8_t*)kept + rows * dp);
  return hipGetLastError();
}

template <class T>
hipError_t grad(const KeptGradArgs& a, hipStream_t s) {
  const Layout l = layout(a.type, a.k, a.n, a.d, a.out);
  char* ws = (char*)a.ws;
  if (hipError_t e = unpack<T>((int64_t)a.k * a.n, a.d, a.kept, (T*)(ws + l.x), l.ldx, s)) return e;
  GradArgs g;
  g.x = ws + l.x;
  g.ldx = l.ldx;
  g.dy = a.dy;
  g.ldy = a.out;
  if (a.out % (16 / sizeof(T)) || (uintptr_t)a.dy % 16) {
    klaunch(copy_rows<T>, dim3(4096), dim3(256), 0, s, (const T*)a.dy, (int64_t)a.k * a.n, a.out,
            (int)l.ldy, (T*)(ws + l.dy));
    if (hipError_t e = hipGetLastError()) return e;
    g.dy = ws + l.dy;
    g.ldy = l.ldy;
  }
  g.n = a.n;
  g.d = a.d;
  g.out = a.out;
  g.span = l.span;
  g.dw = a.dw;
  g.dstride = a.dstride;
  g.vec = a.d % 4 == 0 && (uintptr_t)a.dw % (4 * sizeof(T)) == 0 && a.dstride % 4 == 0;
  g.part = l.splits > 1 ? (float*)(ws + l.part) : nullptr;
  const dim3 grid((unsigned)tiles(a.d, a.out, l.big ? 256 : 128), a.k, l.splits);
  hipError_t e = l.big ? launch_tile<Big<T>, kept_grad_k<Big<T>>>(grid, s, g)
                       : launch_tile<Mid<T>, kept_grad_k<Mid<T>>>(grid, s, g);
  if (e) return e;
  if (l.splits == 1) return hipSuccess;
  klaunch(kept_grad_join<T>, dim3(blocks_of((int64_t)a.out * a.d), a.k), dim3(256), 0, s,
          (const float*)g.part, l.splits, a.out, a.d, (T*)a.dw, a.dstride);
  return hipGetLastError();
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
  return type == LM_F32 ? unpack<float>(rows, d, kept, (float*)x, d, s)
         : type == LM_F16 ? unpack<_Float16>(rows, d, kept, (_Float16*)x, d, s)
                          : unpack<__bf16>(rows, d, kept, (__bf16*)x, d, s);
}
size_t kept_grad_ws_bytes(int type, int k, int n, int d, int out) {
  return layout(type, k, n, d, out).total;
}
hipError_t kept_grad(const KeptGradArgs& a, hipStream_t s) {
  return a.type == LM_F32 ? grad<float>(a, s)
         : a.type == LM_F16 ? grad<_Float16>(a, s)
                            : grad<__bf16>(a, s);
}

}  // namespace cbk
