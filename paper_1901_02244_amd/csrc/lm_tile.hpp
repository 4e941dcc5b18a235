// lm_tile.hpp -- the matrix product that the language-model operators share.
//
// One workgroup computes a BP x BQ tile of  C[p][q] = sum_k P[p][k] Q[q][k]
// on the matrix cores (fp32 sums), for T = float, _Float16 or __bf16.  Each
// operand is given in one of two forms:
//   row form: P[p][k] at base + p*ld + k (the contraction is contiguous);
//   col form: P[p][k] at base + k*ld + p (the contraction is the row index).
//
// fp32 runs on the bf16 matrix cores, sixteen times as fast as the fp32 ones:
// a float is exactly the sum of three bf16 numbers (its leading 8 bits, the
// next 8 and the rest), and of the nine products of two such sums the six
// largest are taken, which leaves out at most 2^-22 of the product (two of 2^-7
// times 2^-16) and mostly less than fp32's own rounding of it, 2^-24.  The
// split is made in registers on the way from LDS.
// (An infinity splits into an infinity and NaNs: its products are NaN.  bf16
// ends at 2^-133, so that floats below 2^-110 are taken to 2^-134.)
//
// A step takes 128 bytes of contraction per row (64 elements of 16 bits or 32
// floats) from global memory straight into LDS (buffer loads with the LDS as
// destination, 16 bytes a lane; no registers are spent on data in flight), two
// steps deep.  What lies outside the operand reads as zero by the buffer's
// range check, so ragged tiles need no branches, and a tile's last steps load
// on past its end, which costs no memory traffic.
//   A 256 x 256 tile of bf16 takes 1.62 us a step, whatever the sum's length
// (1,300 TFLOP/s over 256 CUs, the library's rate for a large product; the
// MFMAs alone would need 0.85), and 6.7 us around them.  The matrix cores are
// busy 60% of it, and LDS moves 67 of its 128 bytes a cycle; rings of five
// steps of half the size, MFMAs pinned before the barrier and raised wave
// priority were no faster, nor, for fp32, splits spread between the MFMAs.
//
// Row form in LDS: rows of 128 bytes, the 16-byte chunk c of row r at
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

// One 16x16 tile's product over 32 elements of 16 bits.
template <class T>
__device__ __forceinline__ f32x4 mma(i32x4 p, i32x4 q, f32x4 c) {
  if constexpr (__is_same(T, _Float16))
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, p),
                                                  __builtin_bit_cast(f16x8, q), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p),
                                                   __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
}

// Eight floats as three times eight bf16 numbers whose sums they are: the
// leading bits cut off (a rounding could pass the largest bf16), the rest
// rounded to bf16, what then remains (at most 8 bits).
struct Split3 {
  i32x4 h, m, l;
};
__device__ __forceinline__ Split3 split3(i32x4 a, i32x4 b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  Split3 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x0 = i < 2 ? a[2 * i] : b[2 * i - 4], x1 = i < 2 ? a[2 * i + 1] : b[2 * i - 3];
    r.h[i] = __builtin_amdgcn_perm(x1, x0, 0x07060302);
    const f32x2 rest = {
        __builtin_bit_cast(float, x0) - __builtin_bit_cast(float, x0 & 0xffff0000u),
        __builtin_bit_cast(float, x1) - __builtin_bit_cast(float, x1 & 0xffff0000u)};
    const uint32_t m = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, bf16x2));
    r.m[i] = m;
    const float l0 = rest[0] - __builtin_bit_cast(float, m << 16);
    const float l1 = rest[1] - __builtin_bit_cast(float, m & 0xffff0000u);
    r.l[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, l1),
                                   __builtin_bit_cast(uint32_t, l0), 0x07060302);
  }
  return r;
}
// The six largest products, the smallest first.
__device__ __forceinline__ f32x4 mma3(const Split3& p, const Split3& q, f32x4 c) {
  c = mma<__bf16>(p.m, q.m, c);
  c = mma<__bf16>(p.l, q.h, c);
  c = mma<__bf16>(p.h, q.l, c);
  c = mma<__bf16>(p.m, q.h, c);
  c = mma<__bf16>(p.h, q.m, c);
  return mma<__bf16>(p.h, q.h, c);
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
// the wait state between the write of m0 and its use.  (m0 is reserved: the
// compiler keeps nothing in it, and these kernels use it for nothing else.)
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

// The permutation of a col form's 16-byte chunks in row `row` of CPR chunks:
// of 16 rows, 0-3 and 8-11 (and 4-7 and 12-15), which half a wave reads
// together, land in eight different 32-byte columns.
template <int CPR>
__device__ __forceinline__ int col_swizzle(int row) {
  return (2 * ((row & 3) | (((row >> 3) & 1) << 2))) & (CPR - 1);
}

constexpr int UB = 128;  // bytes of contraction that a step takes

// Loads one operand's steps into LDS.
template <class T, int R, bool COL, int THREADS>
struct Loader {
  static constexpr int BK = UB / (int)sizeof(T);
  static constexpr int BYTES = R * UB;
  static constexpr int NI = BYTES / (THREADS * 16);
  static_assert(NI * THREADS * 16 == BYTES, "whole loads");
  static constexpr int CPR = COL ? R * (int)sizeof(T) / 16 : UB / 16;  // chunks per LDS row
  uint32_t off[NI];
  uint32_t wave_lds;      // this wave's place in the operand's LDS
  const char* base;       // advances by a step's bytes
  int64_t left;           // bytes from base to the operand's end
  int64_t step;           // bytes a step advances by
  uint32_t chunk;         // row form: this lane's byte of the step's
  int k_left;             // row form: valid bytes of contraction left

  static __device__ __forceinline__ int swz(int row) {
    if constexpr (!COL) return row & 7;
    if constexpr (sizeof(T) == 4) return 0;
    return col_swizzle<CPR>(row);
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
      step = UB;
      chunk = (uint32_t)(((lane % CPR) ^ swz(lane / CPR)) * 16);
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
    k_left -= UB;
  }
};

// One tile's 16-bit operand out of col form: eight k of one p a lane, the first
// four from rows k0.., the others `apart` rows on.
template <int R>
__device__ __forceinline__ i32x4 read_transposed(const lds_char* lds, int r0, int k0, int apart,
                                                 int lane) {
  constexpr int PITCH = R * 2, CPR = PITCH / 16;
  const int j = lane & 15;
  i32x4 f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int row = k0 + apart * u + (j >> 2);
    const int c = (r0 / 8 + ((j & 3) >> 1)) ^ col_swizzle<CPR>(row);
    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(lds + row * PITCH + c * 16 + (j & 1) * 8));
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    f[2 * u] = (int)(uint32_t)b;
    f[2 * u + 1] = (int)(uint32_t)(b >> 32);
  }
  return f;
}

// The operand of the 16 rows from r0 for 64 bytes of contraction, the kk-th of
// a step: 16-bit types in either form, fp32 in row form.
template <class T, int R, bool COL>
__device__ __forceinline__ i32x4 read_frag(const lds_char* lds, int r0, int kk, int lane) {
  const int g = lane >> 4, j = lane & 15;
  if constexpr (COL) {
    static_assert(sizeof(T) == 2, "");
    return read_transposed<R>(lds, r0, kk * 32 + 8 * g, 4, lane);
  } else {
    const int c = (kk * 4 + g) ^ (j & 7);
    return *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(lds + (r0 + j) * UB +
                                                                             c * 16);
  }
}

// The operands of TILES tiles.
template <class T, int R, bool COL, int TILES>
__device__ __forceinline__ void read_frags(const lds_char* lds, int r0, int kk, int lane,
                                           i32x4 (&f)[TILES]) {
  if constexpr (!COL || sizeof(T) == 2) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) f[t] = read_frag<T, R, COL>(lds, r0 + t * 16, kk, lane);
  } else {
    const int g = lane >> 4, j = lane & 15;
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

// 32 elements' MFMAs for 16-bit types, while the next operands come from LDS:
// Q's beside, P's one by one over those that are done with, a few MFMAs
// between the reads.  VALU: how many vector instructions of what the caller
// does next to spread over the MFMAs too.
template <class T, int RP, bool PCOL, int RQ, bool QCOL, int VALU, int TP, int TQ>
__device__ __forceinline__ void mma_step(f32x4 (&acc)[TP][TQ], i32x4 (&fp)[TP], i32x4 (&fq)[TQ],
                                          const lds_char* p, const lds_char* q, int wp, int wq,
                                          int kk, int lane) {
  i32x4 nq[TQ];
  read_frags<T, RQ, QCOL, TQ>(q, wq, kk, lane, nq);
#pragma unroll
  for (int a = 0; a < TP; ++a) {
#pragma unroll
    for (int b = 0; b < TQ; ++b) acc[a][b] = mma<T>(fp[a], fq[b], acc[a][b]);
    fp[a] = read_frag<T, RP, PCOL>(p, wp + a * 16, kk, lane);
  }
  __builtin_amdgcn_sched_group_barrier(0x100, QCOL ? 2 * TQ : TQ, 0);
#pragma unroll
  for (int a = 0; a < TP; ++a) {
    __builtin_amdgcn_sched_group_barrier(0x8, TQ, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, PCOL ? 2 : 1, 0);
    if constexpr (VALU > 0) __builtin_amdgcn_sched_group_barrier(0x2, VALU / TP, 0);
  }
#pragma unroll
  for (int b = 0; b < TQ; ++b) fq[b] = nq[b];
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
  static constexpr int BK = UB / (int)sizeof(T);
  static constexpr int STEP = (BP + BQ) * UB;
  static constexpr int LDS = 2 * STEP;
  using Acc = f32x4[TP][TQ];

  // acc = the tile at (p0, q0) summed over contraction [k0, k1); lds has LDS
  // bytes.  Every thread of the workgroup calls it with the same arguments;
  // when it returns nothing is on its way to LDS, and all have read theirs.
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
    const lds_char* l = (const lds_char*)lds;
    const uint32_t la = (uint32_t)(uintptr_t)l;
    auto issue = [&](uint32_t slot) {
      lp.issue(la + slot);
      lq.issue(la + slot + BP * UB);
    };
    issue(0);
    tile_wait_barrier();
    issue(STEP);
    uint32_t cur = 0;
    if constexpr (sizeof(T) == 2) {
      i32x4 fp[TP], fq[TQ];
      read_frags<T, BP, PCOL, TP>(l, wp, 0, lane, fp);
      read_frags<T, BQ, QCOL, TQ>(l + BP * UB, wq, 0, lane, fq);
      // The barrier in the middle of a step finds its operands in registers, so
      // that its half of LDS is free after it, and the next step landed; there
      // are MFMAs on both sides of it.
      for (int s = 0; s < steps; ++s) {
        mma_step<T, BP, PCOL, BQ, QCOL, 0>(acc, fp, fq, l + cur, l + cur + BP * UB, wp, wq, 1,
                                           lane);
        tile_wait_barrier();
        issue(cur);
        cur = STEP - cur;
        mma_step<T, BP, PCOL, BQ, QCOL, 0>(acc, fp, fq, l + cur, l + cur + BP * UB, wp, wq, 0,
                                           lane);
      }
    } else {
      // A step's floats are split, then the next step's are read from LDS while
      // the MFMAs run.
      i32x4 fp[2][TP], fq[2][TQ];
      auto read = [&](uint32_t slot) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          read_frags<T, BP, PCOL, TP>(l + slot, wp, kk, lane, fp[kk]);
          read_frags<T, BQ, QCOL, TQ>(l + slot + BP * UB, wq, kk, lane, fq[kk]);
        }
      };
      read(0);
      for (int s = 0; s < steps; ++s) {
        Split3 sp[TP], sq[TQ];
#pragma unroll
        for (int a = 0; a < TP; ++a) sp[a] = split3(fp[0][a], fp[1][a]);
#pragma unroll
        for (int b = 0; b < TQ; ++b) sq[b] = split3(fq[0][b], fq[1][b]);
        tile_wait_barrier();
        issue(cur);
        cur = STEP - cur;
        read(cur);
#pragma unroll
        for (int a = 0; a < TP; ++a)
#pragma unroll
          for (int b = 0; b < TQ; ++b) acc[a][b] = mma3(sp[a], sq[b], acc[a][b]);
      }
    }
    tile_wait_barrier();
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

// Stores four neighbouring results of T at `at`, of which `left` exist.
template <class T>
__device__ __forceinline__ void store4(T* at, f32x4 v, float f, int left, bool vec) {
  T o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = from_f32<T>(v[i] * f);
  if (vec) {
    if constexpr (sizeof(T) == 2)
      *(uint64_t*)at = *(const uint64_t*)o;
    else
      *(f32x4*)at = *(const f32x4*)o;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) at[i] = o[i];
  }
}

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

// The tiles that the operators use.  BIG: one workgroup a CU; MID and THIN
// (few rows): two.
constexpr int THIN_Q = 32;
template <class T, bool PC, bool QC>
using BigTile = Tile<T, PC, QC, 256, 256, 2, 4>;
template <class T, bool PC, bool QC>
using MidTile = Tile<T, PC, QC, 128, 128, 2, 2>;
template <class T, bool PC, bool QC>
using ThinTile = Tile<T, PC, QC, 256, THIN_Q, 4, 1>;

// Whether the first axis of a grid holds these workgroups: its threads are a
// 32-bit number.
constexpr bool launch_holds(int64_t workgroups, int threads) {
  return workgroups <= UINT32_MAX / threads;
}

// Launches KERNEL with LDS bytes of dynamic LDS.  More than 64 KB has to be
// asked for, once per kernel and device.
template <int LDS, auto KERNEL, class A>
hipError_t launch_with_lds(dim3 grid, int threads, hipStream_t s, const A& a) {
  static std::atomic<uint64_t> asked{0};
  int dev = 0;
  if (hipError_t e = hipGetDevice(&dev)) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(asked.load(std::memory_order_relaxed) & bit) || !bit) {
    if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, LDS))
      return e;
    asked.fetch_or(bit, std::memory_order_relaxed);
  }
  klaunch(KERNEL, grid, dim3(threads), LDS, s, a);
  return hipGetLastError();
}

// Launches KERNEL on the tiles of TL that cover p x q for each of k learners
// and `splits` shares of the sum (the kernel recovers their grid from p and
// gridDim.x).
template <class TL, auto KERNEL, class A>
hipError_t launch_tile(int64_t p, int64_t q, int k, int splits, hipStream_t s, const A& a) {
  const dim3 grid((unsigned)((p + TL::BP - 1) / TL::BP * ((q + TL::BQ - 1) / TL::BQ)), k, splits);
  return launch_with_lds<TL::LDS, KERNEL>(grid, TL::THREADS, s, a);
}

}  // namespace cbk
