// lm_tile.hpp -- the matrix product that the language-model operators share.
//
// One workgroup computes a BP x BQ tile of  C[p][q] = sum_k P[p][k] Q[q][k]
// on the matrix cores (fp32 sums), for T = float, _Float16 or __bf16.  Each
// operand is given in one of two forms:
//   row form: P[p][k] at base + p*ld + k (the contraction is contiguous);
//   col form: P[p][k] at base + k*ld + p (the contraction is the row index).
//
// A step takes 128 bytes of contraction per row (64 elements of 16 bits or 32
// floats) from global memory straight into LDS (buffer loads with the LDS as
// destination, 16 bytes a lane; no registers are spent on data in flight),
// two steps deep.  What lies outside the operand reads as zero by the buffer's
// range check, so ragged tiles need no branches.
//
// Row form in LDS: rows of 128 bytes, 16-byte chunk c of row r at chunk
// c ^ (r & 7); a lane's operand of one MFMA is then one conflict-free
// ds_read_b128.  Col form in LDS: [k][p] as in memory; 16-bit operands are
// transposed by ds_read_b64_tr_b16 on the way to the registers (lanes
// 16g..16g+15 take four k of 16 p), with the 32-byte pairs of chunks permuted
// by row so that the eight rows that half a wave touches lie in different
// banks; fp32 operands are read as four p of one k per lane, which feeds four
// tiles whose rows interleave (p = 4 row + tile).
//
// Lane l of a 16x16 tile holds, in its four sums, rows 4*(l/16)..+3 of P's
// index and column l%16 of Q's, so for_each_quad() can hand out four
// neighbouring p at one q: callers make P the index that is contiguous in
// memory where the product goes.
#pragma once
#include "kernels.hpp"

#include <atomic>

namespace cbk {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Converts from fp32, to nearest even.
template <class T>
__device__ __forceinline__ T from_f32(float v) {
  return (T)v;
}

// One 16x16 tile's product over 64 bytes of contraction: one MFMA of 32
// 16-bit elements, or four of 4 floats.
template <class T>
__device__ __forceinline__ f32x4 mma(i32x4 p, i32x4 q, f32x4 c) {
  if constexpr (__is_same(T, __bf16)) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p),
                                                   __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
  } else if constexpr (__is_same(T, _Float16)) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, p),
                                                  __builtin_bit_cast(f16x8, q), c, 0, 0, 0);
  } else {
    const f32x4 a = __builtin_bit_cast(f32x4, p), b = __builtin_bit_cast(f32x4, q);
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
}

// A buffer descriptor as the four scalar registers that inline asm takes.
__device__ __forceinline__ i32x4 tile_rsrc(const void* base, uint32_t bytes) {
  const uint64_t p = reinterpret_cast<uintptr_t>(base);
  i32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane((uint32_t)p);
  r[1] = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32) & 0xffffu);
  r[2] = __builtin_amdgcn_readfirstlane(bytes);
  r[3] = 0x00020000;
  return r;
}

// 16 bytes a lane from the buffer into LDS at lds_addr + 16*lane (lds_addr
// uniform).  Inline asm and not the builtin: behind the builtin the compiler
// waits for every load in flight before the next LDS read, which would undo
// the double buffering; the wait is tile_wait_barrier().  No register is
// written, and the address registers are read at issue.  The s_nop covers
// the wait state between the write of m0 and its use.
__device__ __forceinline__ void load_to_lds(i32x4 rsrc, uint32_t off, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds_addr), "v"(off), "s"(rsrc)
               : "memory");
}
// All of this wave's loads into LDS have landed and its LDS reads are back;
// then the barrier makes that true of the whole workgroup.
__device__ __forceinline__ void tile_wait_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

typedef __attribute__((address_space(3))) char lds_char;

// An operand: rows x k in row form, k x rows in col form ("rows" is the
// product's index), both the valid extents.  Memory rows start on 16 bytes
// and are read in whole 16 bytes (the range check drops 4-byte words that
// straddle an extent): what follows an extent up to there has to be readable,
// and in row form zero, or the other operand's rows there absent.
template <class T>
struct Operand {
  const T* base;
  int64_t ld;    // elements between rows of memory
  int rows;
  int k;
};

template <class T, int R, bool COL, int THREADS>
struct Loader {
  static constexpr int BK = 128 / (int)sizeof(T);
  static constexpr int BYTES = R * 128;
  static constexpr int NI = BYTES / (THREADS * 16);
  static_assert(NI * THREADS * 16 == BYTES, "whole loads");
  static constexpr int CPR = COL ? R * (int)sizeof(T) / 16 : 8;  // chunks per LDS row
  uint32_t off[NI];
  uint32_t wave_lds;      // this wave's place in the operand's LDS
  const char* base;       // advances by a step's bytes
  int64_t left;           // bytes from base to the operand's end
  int64_t step;           // bytes a step advances by
  uint32_t chunk;         // row form: this lane's byte in the step's 128
  int k_left;             // row form: valid bytes of contraction left

  // The swizzle of chunk pairs in col form: rows 0-3, 8-11 (and 4-7, 12-15)
  // of 16 land in eight different 32-byte columns.
  static __device__ __forceinline__ int swz(int row) {
    if constexpr (!COL) return row & 7;
    if constexpr (sizeof(T) == 4) return 0;
    return (2 * ((row & 3) | (((row >> 3) & 1) << 2))) & (CPR - 1);
  }

  __device__ __forceinline__ void init(const Operand<T>& o, int row0, int k0, int tid) {
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t ldb = o.ld * (int64_t)sizeof(T);
    wave_lds = wave * 1024;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int id = i * THREADS + tid, r = id / CPR, c = (id % CPR) ^ swz(r);
      off[i] = (uint32_t)(r * ldb + c * 16);
    }
    if constexpr (COL) {
      base = reinterpret_cast<const char*>(o.base) + k0 * ldb + (int64_t)row0 * sizeof(T);
      left = (int64_t)(o.k - k0 - 1) * ldb + (((int64_t)(o.rows - row0) * (int)sizeof(T) + 15) & ~15);
      step = BK * ldb;
      chunk = 0;
      k_left = 0;
    } else {
      base = reinterpret_cast<const char*>(o.base) + row0 * ldb + (int64_t)k0 * sizeof(T);
      k_left = ((o.k - k0) * (int)sizeof(T) + 15) & ~15;
      left = (int64_t)(min(o.rows - row0, R) - 1) * ldb + k_left;
      step = 128;
      chunk = (uint32_t)(((lane & 7) ^ swz(lane >> 3)) * 16);
    }
  }
  // Starts the loads of the next step into the operand's LDS at lds.
  __device__ __forceinline__ void issue(uint32_t lds) {
    const uint32_t bytes = left <= 0 ? 0u : (uint32_t)min(left, (int64_t)0x7ffffff0);
    const i32x4 r = tile_rsrc(base, bytes);
    const bool in = COL || (int)chunk < k_left;
#pragma unroll
    for (int i = 0; i < NI; ++i)
      load_to_lds(r, in ? off[i] : OUTSIDE, lds + wave_lds + i * (THREADS * 16));
    base += step;
    left -= step;
    k_left -= 128;
  }
};

// A wave's operands of one half step (64 bytes of contraction) for its tiles.
template <class T, int R, bool COL, int TILES>
__device__ __forceinline__ void read_frags(const lds_char* lds, int r0, int kk, int lane,
                                           i32x4 (&f)[TILES]) {
  const int g = lane >> 4, j = lane & 15;
  if constexpr (!COL) {
    const lds_char* p = lds + (r0 + j) * 128 + (((kk * 4 + g) ^ (j & 7)) * 16);
#pragma unroll
    for (int t = 0; t < TILES; ++t)
      f[t] = *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(p + t * 2048);
  } else if constexpr (sizeof(T) == 2) {
    constexpr int PITCH = R * 2, CPR = PITCH / 16;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int row = kk * 32 + 8 * g + 4 * u + (j >> 2);
      const int s = (2 * ((row & 3) | (((row >> 3) & 1) << 2))) & (CPR - 1);
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const int c = (r0 / 8 + 2 * t + ((j & 3) >> 1)) ^ s;
        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(lds + row * PITCH + c * 16 + (j & 1) * 8));
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        f[t][2 * u] = (int)(uint32_t)b;
        f[t][2 * u + 1] = (int)(uint32_t)(b >> 32);
      }
    }
  } else {
    constexpr int PITCH = R * 4;
    static_assert(TILES % 4 == 0, "four interleaved tiles at a time");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = kk * 16 + 4 * g + i;
#pragma unroll
      for (int t = 0; t < TILES; t += 4) {
        const i32x4 v = *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(
            lds + row * PITCH + (r0 + t * 16 + 4 * j) * 4);
#pragma unroll
        for (int x = 0; x < 4; ++x) f[t + x][i] = v[x];
      }
    }
  }
}

// Tile geometry: BP x BQ by WP x WQ waves.
template <class T_, bool PCOL_, bool QCOL_, int BP_, int BQ_, int WP_, int WQ_>
struct Tile {
  using T = T_;
  static constexpr bool PCOL = PCOL_, QCOL = QCOL_;
  static constexpr int BP = BP_, BQ = BQ_, WP = WP_, WQ = WQ_;
  static constexpr int THREADS = WP * WQ * 64;
  static constexpr int SP = BP / WP, SQ = BQ / WQ;  // a wave's share
  static constexpr int TP = SP / 16, TQ = SQ / 16;
  static constexpr int BK = 128 / (int)sizeof(T);
  static constexpr int STAGE = (BP + BQ) * 128;
  static constexpr int LDS = 2 * STAGE;
  using Acc = f32x4[TP][TQ];

  // acc = the tile at (p0, q0) summed over contraction [k0, k1); lds has LDS
  // bytes.  Every thread of the workgroup calls it with the same arguments.
  static __device__ __forceinline__ void product(const Operand<T>& P, const Operand<T>& Q, int p0,
                                                 int q0, int k0, int k1, char* lds, Acc& acc) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = (wave / WQ) * SP, wq = (wave % WQ) * SQ;
    Loader<T, BP, PCOL, THREADS> lp;
    Loader<T, BQ, QCOL, THREADS> lq;
    Operand<T> p = P, q = Q;
    p.k = min(p.k, k1);
    q.k = min(q.k, k1);
    lp.init(p, p0, k0, tid);
    lq.init(q, q0, k0, tid);
#pragma unroll
    for (int a = 0; a < TP; ++a)
#pragma unroll
      for (int b = 0; b < TQ; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int steps = (k1 - k0 + BK - 1) / BK;
    if (steps <= 0) return;
    lds_char* l = (lds_char*)lds;
    const uint32_t la = (uint32_t)(uintptr_t)l;
    lp.issue(la);
    lq.issue(la + BP * 128);
    tile_wait_barrier();
    if (steps > 1) {
      lp.issue(la + STAGE);
      lq.issue(la + STAGE + BP * 128);
    }
    i32x4 fp[2][TP], fq[2][TQ];
    read_frags<T, BP, PCOL, TP>(l, wp, 0, lane, fp[0]);
    read_frags<T, BQ, QCOL, TQ>(l + BP * 128, wq, 0, lane, fq[0]);
    // Half a step's operands are read while the other half's MFMAs run; the
    // barrier between the halves finds MFMAs on both sides of it.
    for (int s = 0; s < steps; ++s) {
      const uint32_t cur = (s & 1) * STAGE, nxt = STAGE - cur;
      read_frags<T, BP, PCOL, TP>(l + cur, wp, 1, lane, fp[1]);
      read_frags<T, BQ, QCOL, TQ>(l + cur + BP * 128, wq, 1, lane, fq[1]);
#pragma unroll
      for (int a = 0; a < TP; ++a)
#pragma unroll
        for (int b = 0; b < TQ; ++b) acc[a][b] = mma<T>(fp[0][a], fq[0][b], acc[a][b]);
      tile_wait_barrier();
      if (s + 2 < steps) {
        lp.issue(la + cur);
        lq.issue(la + cur + BP * 128);
      }
      if (s + 1 < steps) {
        read_frags<T, BP, PCOL, TP>(l + nxt, wp, 0, lane, fp[0]);
        read_frags<T, BQ, QCOL, TQ>(l + nxt + BP * 128, wq, 0, lane, fq[0]);
      }
#pragma unroll
      for (int a = 0; a < TP; ++a)
#pragma unroll
        for (int b = 0; b < TQ; ++b) acc[a][b] = mma<T>(fp[1][a], fq[1][b], acc[a][b]);
    }
  }

  // Calls f(p, q, v) for each four sums v at (p..p+3, q) that this thread
  // holds, p and q relative to the tile.
  template <class F>
  static __device__ __forceinline__ void for_each_quad(const Acc& acc, F f) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wp = (wave / WQ) * SP, wq = (wave % WQ) * SQ;
#pragma unroll
    for (int b = 0; b < TQ; ++b) {
      const int q = wq + col_of(b, lane);
#pragma unroll
      for (int a = 0; a < TP; ++a) {
        if constexpr (PCOL && sizeof(T) == 4) {
          const int t = a / 4 * 4, i = a % 4;
          f(wp + t * 16 + 16 * (lane >> 4) + 4 * i, q,
            f32x4{acc[t][b][i], acc[t + 1][b][i], acc[t + 2][b][i], acc[t + 3][b][i]});
        } else {
          f(wp + a * 16 + 4 * (lane >> 4), q, acc[a][b]);
        }
      }
    }
  }
  // Q's index of this lane in the wave's tile b.
  static __device__ __forceinline__ int col_of(int b, int lane) {
    if constexpr (QCOL && sizeof(T) == 4) return b / 4 * 64 + 4 * (lane & 15) + b % 4;
    return b * 16 + (lane & 15);
  }
};

// Tile numbers of a grid of tp x tq tiles: workgroup w of G = tp*tq takes the
// tiles in bands of BAND tiles of p, XCD-major, so that the workgroups that
// run together on one XCD share rows of both operands in its L2.
template <int BAND>
__device__ __forceinline__ void tile_of(int w, int tp, int tq, int& p, int& q) {
  const int id = xcd_major(w, tp * tq);
  const int band = id / (BAND * tq), first = band * BAND, wide = min(BAND, tp - first);
  const int in = id - band * BAND * tq;
  p = first + in % wide;
  q = in / wide;
}

// Launches KERNEL, which runs tiles of TL, with their LDS.  More than 64 KB
// has to be asked for, once per kernel and device.
template <class TL, auto KERNEL, class A>
hipError_t launch_tile(dim3 grid, hipStream_t s, const A& a) {
  static std::atomic<uint64_t> asked{0};
  int dev = 0;
  if (hipError_t e = hipGetDevice(&dev)) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(asked.load(std::memory_order_relaxed) & bit) || !bit) {
    if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, TL::LDS))
      return e;
    asked.fetch_or(bit, std::memory_order_relaxed);
  }
  klaunch(KERNEL, grid, dim3(TL::THREADS), TL::LDS, s, a);
  return hipGetLastError();
}

}  // namespace cbk
