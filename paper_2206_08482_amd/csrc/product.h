// Products of two 16-bit matrices by a workgroup: out[m][n] = sum_k Q[m][k] P[n][k], fp32 sums.  Shared by the layers with an
// epilogue (linear.hip) and the orthogonalised update (muon.hip).
//
// Each operand ("side": P gives the output's columns, Q its rows) lies in memory in one of two orders: contraction contiguous
// (row = index n or m, k along it) or contraction strided (row = k, the index along it), so that one template serves forward
// products, input gradients, weight gradients and the products of a Newton-Schulz step with no transposed copies: the strided
// order goes into LDS as it lies and is transposed by the LDS read (ds_read_b64_tr_b16).
#pragma once
#include <algorithm>
#include <memory>
#include <new>

#include "internal.h"

namespace gmi {
namespace product {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

constexpr int kDepth = 64;                       // contraction elements of a stage: 128 bytes, a cache line, of a contiguous row
static __device__ const uint4 kZeroPiece = {0, 0, 0, 0};      // what contraction elements past the end load

// A workgroup's tile: TM rows by TN columns.  Its columns are two halves; of each of them WN waves share the columns, WM waves the rows, a wave
// has H x RM matrix instructions of 16 x 16 x 32 per half and 32 elements.  A ring of R stages in LDS.
template <int TN_, int TM_, int WN_, int WM_, int R_>
struct Shape {
  static constexpr int TN = TN_, TM = TM_, WN = WN_, WM = WM_, R = R_;
  static constexpr int waves = WN * WM, threads = 64 * waves;
  static constexpr int H = TN / 32 / WN, RN = 2 * H, RM = TM / 16 / WM;
  static constexpr int half = TN / 2;
  static constexpr int half_bytes = half * kDepth * 2, stage = (TN + TM) * kDepth * 2;      // LDS: P's halves, Q
  static constexpr int NP = half / 8 / waves, NQ = TM / 8 / waves, pieces = 2 * NP + NQ;    // 1 KiB loads of a wave: of a half of P, of Q
  static constexpr int lds = R * stage;
  static constexpr int U = RM % 2 ? 1 : 2;                             // 16-row tiles that the epilogue stages per wave at a time
  static constexpr int wave_lds = U * 16 * RN * 16 * 4;
  static_assert(wave_lds * waves <= lds && half % (8 * waves) == 0 && TM % (8 * waves) == 0, "");
};
using Large = Shape<256, 256, 2, 4, 2>;
using Middle = Shape<192, 192, 3, 4, 3>;      // contraction contiguous only
using Medium = Shape<128, 128, 2, 2, 2>;

// For products with few tiles: each of the W waves computes the whole tile over its own stages (every W-th, 64 deep), from a ring of its own,
// so that there is no barrier until the waves' sums are added at the end.
template <int TN_, int TM_, int W_, int R_>
struct OwnShape {
  static constexpr int TN = TN_, TM = TM_, W = W_, R = R_;
  static constexpr int waves = W, threads = 64 * W;
  static constexpr int RN = TN / 16, RM = TM / 16;
  static constexpr int p_bytes = TN * kDepth * 2, stage = (TN + TM) * kDepth * 2;      // bytes of a wave
  static constexpr int NP = TN / 8, NQ = TM / 8, pieces = NP + NQ;
  static constexpr int ring = R * stage, lds = W * ring;
  static_assert(TN * TM * 4 <= ring, "");
};
using Small = OwnShape<64, 64, 4, 2>;
using Twin = OwnShape<64, 64, 2, 2>;      // two share a compute unit
using Few = OwnShape<64, 16, 4, 3>;
using Row = OwnShape<16, 16, 8, 4>;
template <class S> struct IsOwn { static constexpr bool value = false; };
template <int A, int B, int C, int D> struct IsOwn<OwnShape<A, B, C, D>> { static constexpr bool value = true; };

// For a kernel's launch bounds: one workgroup of a compute unit's LDS, or two.
template <class S>
constexpr int kWavesPerSimd = S::lds > (80 << 10) ? (S::threads + 255) / 256 : 2;

// What a product with a tile takes: kStart + u (fixed + per_k K) us, u = workgroups of a compute unit one after the other (two of Medium or Twin
// share a unit and its matrix cores, which comes to the same), K = contraction length times products of planes.  Measured (the kernel alone),
// us of Large, Medium, Small, Twin, Few, Row for rows x K x columns  16 x 4096 x 1024: 73 33 15 18 9.4 7.0;  256 x 1024 x 1024: 27 14 8.2 9.3 6.3 17;
// 1024 x 1024 x 1024: 28 15 9.1 10 19 60;  2048 x 1024 x 1024: 28 15 16 13 35 116;  4096 x 512 x 512: 20 11 13 10 30 107;
// 8192 x 4096 x 1024: 86 62 124 108 298 703;  16384 x 1024 x 4096: 132 140 450 282 1100 3600.  Middle is there for what it just fits: 6000 x 1000 x
// 1500 (256 tiles) 26 us, Large 35, Medium 39; 8192 x 4096 x 4096 (946) 251, Large 215.
struct Tile { int size[2]; float fixed, per_k; int share; float alone; };      // share: workgroups that a compute unit runs at once;
                                                                                // alone: how much longer than that one lasts by itself
constexpr Tile kTiles[7] = {{{Large::TM, Large::TN}, 10.f, 0.0224f, 1, 1.f}, {{Medium::TM, Medium::TN}, 3.7f, 0.0068f, 2, 1.15f}, {{Small::TM, Small::TN}, 3.4f, 0.0029f, 1, 1.f},
                            {{Twin::TM, Twin::TN}, 2.4f, 0.0026f, 2, 1.35f}, {{Few::TM, Few::TN}, 2.3f, 0.0017f, 1, 1.f}, {{Row::TM, Row::TN}, 2.3f, 0.0008f, 1, 1.f},
                            {{Middle::TM, Middle::TN}, 8.f, 0.0135f, 1, 1.f}};
constexpr float kStart = 2.5f;
inline float tile_time(const Tile& t, float k) { return t.fixed + t.per_k * k; }

// Order of contraction for operands held in several 16-bit planes: pairs of planes, the smallest products first.  A pair is
// (plane of P) | (plane of Q) << 2, eight bits each from the lowest.
struct Pairs { uint64_t code; int n; };
constexpr Pairs kOnePlane = {0, 1};
constexpr Pairs kTwoPlanes = {0x000104, 3};               // (0, 1), (1, 0), (0, 0)
constexpr Pairs kThreePlanes = {0x000104050208, 6};      // (0, 2), (2, 0), (1, 1), (0, 1), (1, 0), (0, 0)

struct Side {
  const char* base;    // the tile's first index, the first contraction element, plane 0
  int64_t ld;          // bytes between rows of memory
  int64_t plane;       // bytes between planes
  int count;           // indices of the tile that exist, 1 ..
};

template <class S>
struct Accumulator { f32x4 v[S::RN][S::RM]; };

// XOR on the 16-byte slot of row r of a strided side.  Half a wave's transposing read takes 32 bytes of each of the rows 0 .. 3 and 8 .. 11
// of 16 (or 4 .. 7 and 12 .. 15): with it these lie in different banks.  (Rows of 128 bytes, T = 64, share banks two by two as it is.)
template <int T>
__device__ __forceinline__ int strided_swizzle(int r) { return T >= 128 ? (r & 3) << 2 | (r & 8) >> 2 : (r & 2) << 1 | (r & 8) >> 2; }

// XOR on the 16-byte slot (of eight) of row r of a contiguous side.  The LDS serves a 16-byte read in sets of 16 lanes (0-3, 12-15, 20-27; 4-11,
// 16-19, 28-31; the same + 32): with this order each set's lanes lie in different banks.  (An order made for 16 consecutive lanes had every
// read take twice as long: half the LDS's active cycles were bank conflicts.)
__device__ __forceinline__ int contiguous_swizzle(int r) { return (r >> 1) & 7; }

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// N pieces of 1 KiB, 16 bytes per lane from base + off[j], or from a pointer of the lane's own, to LDS bytes lds + 1024 j in lane order.  Inline
// assembly: the compiler would wait for every such load in flight before any LDS read.  m0 (the LDS address) is declared as overwritten.
template <int N>
__device__ __forceinline__ void load_pieces(const char* base, const uint32_t (&off)[N], uint32_t lds) {
  static_assert(N == 1 || N == 2 || N == 4 || N == 8, "");
  if constexpr (N == 8) {
    load_pieces<4>(base, {off[0], off[1], off[2], off[3]}, lds);
    load_pieces<4>(base, {off[4], off[5], off[6], off[7]}, lds + 4096);
  } else if constexpr (N == 1) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off[0]), "s"(base) : "m0", "memory");
  } else if constexpr (N == 4) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\t"
                 "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %5\n\t"
                 "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %5\n\t"
                 "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %5"
                 ::"s"(lds), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base) : "m0", "scc", "memory");
  } else {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\t"
                 "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3"
                 ::"s"(lds), "v"(off[0]), "v"(off[1]), "s"(base) : "m0", "scc", "memory");
  }
}
__device__ __forceinline__ void load_piece(const void* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "m0", "memory");
}
#pragma clang diagnostic pop

template <int OUTSTANDING>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::"n"(OUTSTANDING) : "memory");
}

// The N pieces that a wave loads of a side (or a half of one) of T indices, from piece `first` on, and where it is in the contraction.
template <int T, int N, bool STRIDED>
struct Loader {
  uint32_t off[N];
  int own[N];        // the lane's contraction element within a stage (first of eight, or its row)
  const char *base, *at;
  int64_t step, plane;
  // indices from `index0` of the side on
  __device__ __forceinline__ void init(const Side& s, int index0, int first, int lane, int first_plane) {
    // indices past the side's end load its last ones again: what they give is never stored
    const int last = STRIDED ? (s.count - 1) & ~7 : s.count - 1, start = min(index0, last);
    base = s.base + (STRIDED ? (int64_t)start * 2 : start * s.ld);
    plane = s.plane;
    step = STRIDED ? s.ld * kDepth : kDepth * 2;
    at = base + first_plane * plane;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      constexpr int slots = STRIDED ? T / 8 : 8, rows = 64 / slots;      // 16-byte slots of a row of LDS, rows of a piece
      const int r = rows * (first + j) + lane / slots;
      const int c = (lane % slots) ^ (STRIDED ? strided_swizzle<T>(r) : contiguous_swizzle(r));
      own[j] = STRIDED ? r : 8 * c;
      off[j] = STRIDED ? (uint32_t)(r * s.ld + 2 * (min(index0 + 8 * c, last) - start)) : (uint32_t)((min(index0 + r, last) - start) * s.ld + 16 * c);
    }
  }
  // the next stage, of which `left` contraction elements exist, into LDS from `lds` on
  __device__ __forceinline__ void load(int left, uint32_t lds) const {
    if (left >= kDepth) {
      load_pieces(at, off, lds);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) load_piece(own[j] < left ? (const void*)(at + off[j]) : (const void*)&kZeroPiece, lds + 1024 * j);
    }
  }
};

// The same for a contiguous side whose rows lie at any address and end anywhere: through registers.  fetch() asks for a stage, put() writes it
// to LDS in the order that load() leaves.
template <int T, int N>
struct RawLoader {
  uint32_t off[N];
  int own[N];
  uint4 v[N];
  const char *base, *at;
  int64_t step;
  __device__ __forceinline__ void init(const Side& s, int lane) {
    base = at = s.base;
    step = kDepth * 2;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int r = 8 * j + lane / 8, c = (lane % 8) ^ contiguous_swizzle(r);
      own[j] = 8 * c;
      off[j] = (uint32_t)(min(r, s.count - 1) * s.ld + 16 * c);
    }
  }
  __device__ __forceinline__ void fetch(int left) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int n = left - own[j];
      if (n >= 8) {
        __builtin_memcpy(&v[j], at + off[j], 16);
      } else {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (e < n) w[e >> 1] |= (uint32_t)((const uint16_t*)(at + off[j]))[e] << (16 * (e & 1));
        v[j] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
  __device__ __forceinline__ void put(char* lds, int lane) const {
#pragma unroll
    for (int j = 0; j < N; ++j) *(uint4*)(lds + j * 1024 + lane * 16) = v[j];
  }
};

// Where a wave reads its operands of a stage: operand t is indices 16 t .. + 15 and 32 contraction elements, lane l holds index l % 16 and
// elements 8 (l / 16) .. + 7.
template <int T, bool STRIDED, int N>
struct Reader {
  uint32_t at[STRIDED ? N : 2];
  __device__ __forceinline__ void init(int tile0, int lane) {
    const int i = lane & 15, q = lane >> 4;
    if constexpr (!STRIDED) {
#pragma unroll
      for (int k = 0; k < 2; ++k) at[k] = (tile0 * 16 + i) * kDepth * 2 + (((4 * k + q) ^ contiguous_swizzle(i)) << 4);
    } else {
      // a transposing read: the 16 lanes of group q address row i / 4 of four and indices 4 (i % 4) .. + 3
      const int r = 8 * q + (i >> 2);
#pragma unroll
      for (int t = 0; t < N; ++t)
        at[t] = r * 2 * T + 8 * (i & 1) + (((2 * (tile0 + t) + ((i & 3) >> 1)) ^ strided_swizzle<T>(r)) << 4);
    }
  }
  // operand t of elements 32 k .. + 31 of what lies at smem + from
  __device__ __forceinline__ s16x8 read(const char* smem, uint32_t from, int t, int k) const {
    if constexpr (!STRIDED) {
      return *(const s16x8*)(smem + (at[k] + from) + t * 32 * kDepth);
    } else {
      const char* p = smem + (at[t] + from) + k * 64 * T;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 8 * T));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

// Where loads are in the contraction: elements of this pair of planes not yet loaded (0: nothing more), pairs left, their code.
struct Walk {
  int left, more;
  uint64_t code;
  __device__ __forceinline__ bool advance(int k_len) {      // past a stage; true: at the next pair
    left -= kDepth;
    if (left > 0) return false;
    code >>= 8;
    left = --more > 0 ? k_len : 0;
    return true;
  }
};

// Between the smaller products of planes and the first planes' own (the last pair).  An infinite value is its first plane alone, the others are 0, and the
// planes of what it meets have signs of their own: the smaller products would make NaN of it.  The first planes' product decides: infinities and NaN of
// the sums so far are dropped, what they come from is in it again.
// (In a loop over both parts: a branch around it within the loop over stages takes 3 to 6 % of the time.)
template <class S>
__device__ __forceinline__ void keep_finite(Accumulator<S>& acc) {
#pragma unroll
  for (int i = 0; i < S::RN; ++i)
#pragma unroll
    for (int j = 0; j < S::RM; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc.v[i][j][e] = __builtin_amdgcn_classf(acc.v[i][j][e], 0x207) ? 0.f : acc.v[i][j][e];      // NaN, infinities
}

template <bool HALF>
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The tile's sums over k_len contraction elements of every pair of planes.  A contraction-contiguous side has k_len a multiple of 8 (the
// rest of its last stage is zeros), rows 16-byte aligned; a strided side has its index count rounded up to 8 in memory.  All
// arguments are the same in every lane.  Ends with the workgroup's waves past their last LDS read.
// A stage is four phases of H x RM instructions: (half 0, elements 0 .. 31), (half 0, 32 .. 63), (half 1, 0 .. 31), (half 1, 32 .. 63).  A phase's operands
// are read in the shadow of the one before it.  After the first phase everything of half 0 and of Q is in registers, after the third
// everything of half 1: there the workgroup's waves meet, and the place takes the stage R later, which is loaded two or more phases before it
// is next waited for.
template <class S, bool PS, bool QS, bool HALF, bool INFINITE>
__device__ __forceinline__ void multiply_shared(const Side& P, const Side& Q, int k_len, Pairs pairs, char* smem, Accumulator<S>& acc) {
  constexpr int H = S::H, RM = S::RM, kSteps = H * RM;
  static_assert((!PS || 64 % (S::half / 8) == 0) && (!QS || 64 % (S::TM / 8) == 0), "a strided side's rows have to fill a piece");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int n = (k_len + kDepth - 1) / kDepth * pairs.n;
  Loader<S::half, S::NP, PS> l0, l1;
  Loader<S::TM, S::NQ, QS> lq;
  Walk w0 = {n > 0 ? k_len : 0, pairs.n, pairs.code}, w1 = w0;      // of half 0 and Q, of half 1
  l0.init(P, 0, wave * S::NP, lane, w0.code & 3);
  l1.init(P, S::half, wave * S::NP, lane, w0.code & 3);
  lq.init(Q, 0, wave * S::NQ, lane, w0.code >> 2 & 3);
  const uint32_t put0 = lds0 + wave * S::NP * 1024, put1 = put0 + S::half_bytes, putq = lds0 + 2 * S::half_bytes + wave * S::NQ * 1024;
  // A load of nothing keeps the counts of loads in flight the same at the end.
  auto load_p0 = [&](uint32_t slot) { l0.load(w0.left, put0 + slot); };
  auto load_q = [&](uint32_t slot) {
    lq.load(w0.left, putq + slot);
    l0.at += l0.step;
    lq.at += lq.step;
    if (w0.advance(k_len)) {
      l0.at = l0.base + (int64_t)(w0.code & 3) * l0.plane;
      lq.at = lq.base + (int64_t)(w0.code >> 2 & 3) * lq.plane;
    }
  };
  auto load_p1 = [&](uint32_t slot) {
    l1.load(w1.left, put1 + slot);
    l1.at += l1.step;
    if (w1.advance(k_len)) l1.at = l1.base + (int64_t)(w1.code & 3) * l1.plane;
  };

  const int wn = wave % S::WN, wm = wave / S::WN;
  Reader<S::half, PS, H> rp;
  Reader<S::TM, QS, RM> rq;
  rp.init(wn * H, lane);
  rq.init(wm * RM, lane);
#pragma unroll
  for (int i = 0; i < S::RN; ++i)
#pragma unroll
    for (int j = 0; j < RM; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc.v[i][j][e] = 0.f;

  // The instructions of a phase, with between(t) after the t-th: what is issued there runs in their shadow.
  auto phase = [&](int i0, const s16x8 (&p)[H], const s16x8 (&q)[RM], auto&& between) {
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
      for (int j = 0; j < RM; ++j) {
        acc.v[i0 + i][j] = mfma<HALF>(p[i], q[j], acc.v[i0 + i][j]);
        __builtin_amdgcn_sched_barrier(0);
        between(i * RM + j);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  // reads behind each instruction: done before a phase's last quarter, so that they have arrived at its end
  constexpr int kBoth = (4 * (H + RM) + 3 * kSteps - 1) / (3 * kSteps);
  s16x8 pa[H], pb[H], qa[RM], qb[RM];
  auto read_p = [&](int t, uint32_t from, int k, s16x8 (&p)[H]) { if (t < H) p[t] = rp.read(smem, from, t, k); };
  auto read_both = [&](int t, uint32_t stage, int k, s16x8 (&p)[H], s16x8 (&q)[RM]) {
#pragma unroll
    for (int x = t * kBoth; x < min(H + RM, (t + 1) * kBoth); ++x) {
      if (x < RM) q[x] = rq.read(smem, stage + 2 * S::half_bytes, x, k);
      else p[x - RM] = rp.read(smem, stage, x - RM, k);
    }
  };

#pragma unroll
  for (int s = 0; s < S::R; ++s) {
    load_p0(s * S::stage);
    load_q(s * S::stage);
    load_p1(s * S::stage);
  }
  wait_and_meet<(S::R - 1) * S::pieces + S::NP>();
  uint32_t cur = 0;
#pragma unroll
  for (int t = 0; t < kSteps; ++t) read_both(t, 0, 0, pa, qa);
  auto stages = [&](int count) {
    for (int st = 0; st < count; ++st) {
      const uint32_t next = cur == (S::R - 1) * S::stage ? 0 : cur + S::stage;
      phase(0, pa, qa, [&](int t) { read_both(t, cur, 1, pb, qb); });
      wait_and_meet<(S::R - 1) * S::pieces>();      // half 1 of this stage has landed; half 0 and Q have been read
      phase(0, pb, qb, [&](int t) {
        read_p(t, cur + S::half_bytes, 0, pa);
        if (t == kSteps / 2) load_p0(cur);
      });
      phase(H, pa, qa, [&](int t) {
        read_p(t, cur + S::half_bytes, 1, pb);
        if (t == kSteps / 2) load_q(cur);
      });
      wait_and_meet<(S::R - 1) * S::pieces>();      // half 0 and Q of the next stage have landed; half 1 has been read
      phase(H, pb, qb, [&](int t) {
        read_both(t, next, 0, pa, qa);
        if (t == kSteps / 2) load_p1(cur);
      });
      cur = next;
    }
  };
  if constexpr (INFINITE) {
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {
      keep_finite<S>(acc);      // before the first part as well, where it changes nothing: only between them, Large spills registers
      stages(part ? n / pairs.n : n - n / pairs.n);
    }
  } else {
    stages(n);
  }
  wait_and_meet<0>();
}

// The same for an OwnShape: every wave ends with its part of the tile's sums.
// RAW: both sides contiguous, at any address (one plane).
template <class S, bool PS, bool QS, bool HALF, bool RAW, bool INFINITE>
__device__ __forceinline__ void multiply_own(const Side& P, const Side& Q, int k_len, Pairs pairs, char* smem, Accumulator<S>& acc) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t base = wave * S::ring, lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + base;
  const int per_pair = (k_len + kDepth - 1) / kDepth, total = per_pair * pairs.n;
  const int n = total > wave ? (total - wave + S::W - 1) / S::W : 0;      // this wave's stages: wave, wave + W, ..
  static_assert(!RAW || (!PS && !QS), "");
  std::conditional_t<RAW, RawLoader<S::TN, S::NP>, Loader<S::TN, S::NP, PS>> lp;
  std::conditional_t<RAW, RawLoader<S::TM, S::NQ>, Loader<S::TM, S::NQ, QS>> lq;
  uint64_t code = pairs.code;
  if constexpr (RAW) {
    lp.init(P, lane);
    lq.init(Q, lane);
  } else {
    lp.init(P, 0, 0, lane, 0);
    lq.init(Q, 0, 0, lane, 0);
  }
  int k = wave, issued = 0;      // of the next stage: place within its pair of planes
  auto load = [&](int slot) {
    while (k >= per_pair && issued < n) { k -= per_pair; code >>= 8; }
    const int left = issued < n ? k_len - k * kDepth : 0;
    if constexpr (RAW) {
      lp.at = lp.base + k * lp.step;
      lq.at = lq.base + k * lq.step;
      lp.fetch(left);
      lq.fetch(left);
    } else {
      lp.at = lp.base + (int64_t)(code & 3) * lp.plane + k * lp.step;
      lq.at = lq.base + (int64_t)(code >> 2 & 3) * lq.plane + k * lq.step;
      lp.load(left, lds0 + slot * S::stage);
      lq.load(left, lds0 + slot * S::stage + S::p_bytes);
    }
    k += S::W;
    ++issued;
  };
  auto put = [&](int slot) {
    if constexpr (RAW) {
      lp.put(smem + base + slot * S::stage, lane);
      lq.put(smem + base + slot * S::stage + S::p_bytes, lane);
    }
  };
  Reader<S::TN, PS, S::RN> rp;
  Reader<S::TM, QS, S::RM> rq;
  rp.init(0, lane);
  rq.init(0, lane);
#pragma unroll
  for (int i = 0; i < S::RN; ++i)
#pragma unroll
    for (int j = 0; j < S::RM; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc.v[i][j][e] = 0.f;
  s16x8 p0[S::RN], q0[S::RM], p1[S::RN], q1[S::RM];
  auto read = [&](uint32_t stage, int half, s16x8 (&p)[S::RN], s16x8 (&q)[S::RM]) {
#pragma unroll
    for (int j = 0; j < S::RM; ++j) q[j] = rq.read(smem, base + stage + S::p_bytes, j, half);
#pragma unroll
    for (int i = 0; i < S::RN; ++i) p[i] = rp.read(smem, base + stage, i, half);
  };
  auto product = [&](const s16x8 (&p)[S::RN], const s16x8 (&q)[S::RM]) {
#pragma unroll
    for (int i = 0; i < S::RN; ++i)
#pragma unroll
      for (int j = 0; j < S::RM; ++j) acc.v[i][j] = mfma<HALF>(p[i], q[j], acc.v[i][j]);
  };
  if (n > 0) {
#pragma unroll
    for (int s = 0; s < S::R; ++s) { load(s); put(s); }
    if constexpr (!RAW) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S::R - 1) * S::pieces) : "memory");
    int slot = 0;
    read(0, 0, p0, q0);
    auto stages = [&](int count) {
      for (int st = 0; st < count; ++st) {
        if constexpr (RAW) load(slot);      // the stage R later, on its way to registers while this one is multiplied
        read(slot * S::stage, 1, p1, q1);
        product(p0, q0);
        const int done = slot;
        slot = slot == S::R - 1 ? 0 : slot + 1;
        if constexpr (!RAW) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the slot has been read: it takes the stage R later
          load(done);
          asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S::R - 1) * S::pieces) : "memory");
        }
        read(slot * S::stage, 0, p0, q0);
        product(p1, q1);
        put(done);
      }
    };
    if constexpr (INFINITE) {
      const int before = min(n, max(0, (total - per_pair - wave + S::W - 1) / S::W));      // this wave's stages before the last pair
#pragma unroll 1
      for (int part = 0; part < 2; ++part) {
        stages(part ? n - before : before);
        if (part == 0) keep_finite<S>(acc);
      }
    } else {
      stages(n);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// INFINITE: operands in several planes may hold infinities.
template <class S, bool PS, bool QS, bool HALF, bool RAW = false, bool INFINITE = false>
__device__ __forceinline__ void multiply(const Side& P, const Side& Q, int k_len, Pairs pairs, char* smem, Accumulator<S>& acc) {
  static_assert(!RAW || IsOwn<S>::value, "");
  if constexpr (IsOwn<S>::value) multiply_own<S, PS, QS, HALF, RAW, INFINITE>(P, Q, k_len, pairs, smem, acc);
  else multiply_shared<S, PS, QS, HALF, INFINITE>(P, Q, k_len, pairs, smem, acc);
}

// What the functions below hand out with the sums: fetch(m, n) is called ahead of row(m, n, v, what it gave), for several rows at a time, so that
// what an epilogue reads from memory is on its way together.  (Its stores may go to the memory that the next row's values come from, as far
// as the compiler knows, so it cannot move such reads by itself.)
struct Nothing {};
struct FetchNothing { __device__ __forceinline__ Nothing operator()(int, int) const { return {}; } };

// Every wave's sums of an OwnShape go into LDS, where the workgroup adds them, eight columns of a row a thread.  The totals stay in the first
// wave's place for each_column.
template <class S, class G, class F>
__device__ __forceinline__ void add_own(const Accumulator<S>& acc, char* smem, G&& fetch, F&& row) {
  constexpr int mask = S::TN / 4 - 1, pieces = S::TM * S::TN / 8, turns = (pieces + S::threads - 1) / S::threads;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, h = lane >> 4;
  float* mine = (float*)smem + wave * S::TN * S::TM;
  decltype(fetch(0, 0)) with[turns];
#pragma unroll
  for (int k = 0; k < turns; ++k) {
    const int i = k * S::threads + threadIdx.x;
    if (i < pieces) with[k] = fetch(i / (S::TN / 8), i % (S::TN / 8) * 8);
  }
#pragma unroll
  for (int j = 0; j < S::RM; ++j)
#pragma unroll
    for (int i = 0; i < S::RN; ++i) {
      const f32x4 x = acc.v[i][j];
      *(float4*)(mine + (16 * j + m) * S::TN + (((4 * i + h) ^ (m & mask)) << 2)) = make_float4(x[0], x[1], x[2], x[3]);
    }
  __syncthreads();
#pragma unroll
  for (int turn = 0; turn < turns; ++turn) {
    const int i = turn * S::threads + threadIdx.x;
    if (i >= pieces) break;
    const int r = i / (S::TN / 8), c = i % (S::TN / 8);
    float v[8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float* at = (float*)smem + r * S::TN + (((2 * c + k) ^ (r & mask)) << 2);
      float4 t = *(const float4*)at;
#pragma unroll
      for (int w = 1; w < S::W; ++w) {
        const float4 x = *(const float4*)(at + w * S::TN * S::TM);
        t.x += x.x; t.y += x.y; t.z += x.z; t.w += x.w;
      }
      *(float4*)at = t;
      v[4 * k] = t.x; v[4 * k + 1] = t.y; v[4 * k + 2] = t.z; v[4 * k + 3] = t.w;
    }
    row(r, 8 * c, v, with[turn]);
  }
}

// Column of the tile that the wave's staged column c is.
template <class S>
__device__ __forceinline__ int column_of(int wn, int c) { return c / (S::H * 16) * S::half + wn * S::H * 16 + c % (S::H * 16); }
// The columns n .. n + 7 that a lane has in each_row.
template <class S>
__device__ __forceinline__ int lane_column() {
  if constexpr (IsOwn<S>::value) return 8 * (threadIdx.x % (S::TN / 8));
  else return column_of<S>((threadIdx.x >> 6) % S::WN, 8 * (threadIdx.x % (S::RN * 2)));
}

// A wave's sums of U row tiles from j on into its own LDS.
template <class S>
__device__ __forceinline__ void stage_rows(const Accumulator<S>& acc, int j, float* mine) {
  constexpr int pitch = S::RN * 16, mask = pitch / 4 - 1;
  const int m = threadIdx.x & 15, h = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int u = 0; u < S::U; ++u)
#pragma unroll
    for (int i = 0; i < S::RN; ++i) {
      const f32x4 x = acc.v[i][j + u];
      *(float4*)(mine + (16 * u + m) * pitch + (((4 * i + h) ^ ((16 * u + m) & mask)) << 2)) = make_float4(x[0], x[1], x[2], x[3]);
    }
  asm volatile("" ::: "memory");
}

// Hands the tile's sums to row(m, n, v, fetch(m, n)): eight consecutive columns n .. n + 7 of row m of the tile, each wave its own part, rows whole
// 64 .. 256 bytes of 16-bit values at a time.  Goes through the wave's own LDS: a lane's accumulators are 4 columns of a row, stores
// of which would be 8 bytes each.
template <class S, class G, class F>
__device__ __forceinline__ void each_row(const Accumulator<S>& acc, char* smem, G&& fetch, F&& row) {
  if constexpr (IsOwn<S>::value) {
    add_own(acc, smem, fetch, row);
  } else {
    constexpr int pitch = S::RN * 16, per_row = pitch / 8, rows = 64 / per_row, mask = pitch / 4 - 1, turns = 16 * S::U / rows;
    constexpr int kAhead = turns % 4 == 0 ? 4 : turns;
    static_assert(turns <= 8 && turns % kAhead == 0, "");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % S::WN, wm = wave / S::WN, c = lane % per_row, n = column_of<S>(wn, 8 * c);
    float* mine = (float*)(smem + wave * S::wave_lds);
#pragma unroll
    for (int j = 0; j < S::RM; j += S::U) {
      const int first = (wm * S::RM + j) * 16 + lane / per_row;
      stage_rows(acc, j, mine);
#pragma unroll 1
      for (int k0 = 0; k0 < turns; k0 += kAhead) {
        decltype(fetch(0, 0)) with[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) with[k] = fetch(first + (k0 + k) * rows, n);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int r = (k0 + k) * rows + lane / per_row;
          float v[8];
          const float4 a = *(const float4*)(mine + r * pitch + (((2 * c) ^ (r & mask)) << 2));
          const float4 b = *(const float4*)(mine + r * pitch + (((2 * c + 1) ^ (r & mask)) << 2));
          v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
          row(first + (k0 + k) * rows, n, v, with[k]);
        }
      }
      asm volatile("" ::: "memory");
    }
  }
}

// The same by columns: col(n, m, v, fetch(n, m)): rows m .. m + 7 of column n.  AFTER_ROWS: each_row has been called.
template <bool AFTER_ROWS, class S, class G, class F>
__device__ __forceinline__ void each_column(const Accumulator<S>& acc, char* smem, G&& fetch, F&& col) {
  if constexpr (IsOwn<S>::value) {
    constexpr int mask = S::TN / 4 - 1, pieces = S::TM * S::TN / 8, turns = (pieces + S::threads - 1) / S::threads;
    decltype(fetch(0, 0)) with[turns];
#pragma unroll
    for (int k = 0; k < turns; ++k) {
      const int i = k * S::threads + threadIdx.x;
      if (i < pieces) with[k] = fetch(i / (S::TM / 8), i % (S::TM / 8) * 8);
    }
    if (!AFTER_ROWS) add_own(acc, smem, FetchNothing(), [](int, int, float (&)[8], Nothing) {});
    __syncthreads();
#pragma unroll
    for (int k = 0; k < turns; ++k) {
      const int i = k * S::threads + threadIdx.x;
      if (i >= pieces) break;
      const int n = i / (S::TM / 8), m0 = i % (S::TM / 8) * 8;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = ((const float*)smem)[(m0 + e) * S::TN + (((n >> 2) ^ ((m0 + e) & mask)) << 2) + (n & 3)];
      col(n, m0, v, with[k]);
    }
  } else {
    constexpr int pitch = S::RN * 16, mask = pitch / 4 - 1, columns = 32 / S::U, turns = pitch / columns;
    constexpr int kAhead = turns % 4 == 0 ? 4 : turns;
    static_assert(turns <= 8 && turns % kAhead == 0, "");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % S::WN, wm = wave / S::WN, m0 = 8 * (lane % (2 * S::U));
    float* mine = (float*)(smem + wave * S::wave_lds);
#pragma unroll
    for (int j = 0; j < S::RM; j += S::U) {
      const int m = (wm * S::RM + j) * 16 + m0;
      stage_rows(acc, j, mine);
#pragma unroll 1
      for (int k0 = 0; k0 < turns; k0 += kAhead) {
        decltype(fetch(0, 0)) with[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) with[k] = fetch(column_of<S>(wn, (k0 + k) * columns + lane / (2 * S::U)), m);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int c = (k0 + k) * columns + lane / (2 * S::U);
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = mine[(m0 + e) * pitch + (((c >> 2) ^ ((m0 + e) & mask)) << 2) + (c & 3)];
          col(column_of<S>(wn, c), m, v, with[k]);
        }
      }
      asm volatile("" ::: "memory");
    }
  }
}

// bf16 planes: x = p0 + p1 (+ p2), each the nearest bf16 of what the ones before it leave; 8 bits of significand a plane.  A finite x keeps a
// finite p0 (values within half a unit of bf16's largest are cut instead of rounded), an infinity or NaN is p0 alone.
__device__ __forceinline__ uint16_t bf16_bits(float x) {
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {      // one instruction
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
}
__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
template <int N>
__device__ __forceinline__ void split_bf16(float x, uint16_t (&p)[N]) {
  p[0] = bf16_bits(x);
  if constexpr (N > 1) {
    const bool finite = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
    if (finite && (p[0] & 0x7FFFu) == 0x7F80u) p[0] = (uint16_t)(__float_as_uint(x) >> 16);
    float rest = finite ? x - bf16_value(p[0]) : 0.f;
#pragma unroll
    for (int i = 1; i < N; ++i) {
      p[i] = bf16_bits(rest);
      rest -= bf16_value(p[i]);
    }
  }
}

// ------------------------------------------------------------------ eight values of a row
// A value array's element type is F32 ? float : bf16; n: how many of the eight exist.  Whole eights go as 16-byte pieces whatever their
// alignment (memcpy of a constant size: the compiler's own unaligned access), rows need no other path.
template <bool F32>
__device__ __forceinline__ void load8(const void* base, int64_t at, int n, float (&v)[8]) {
  if constexpr (F32) {
    const float* p = (const float*)base + at;
    if (n >= 8) {
      __builtin_memcpy(v, p, 32);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : 0.f;
    }
  } else {
    const uint16_t* p = (const uint16_t*)base + at;
    if (n >= 8) {
      uint32_t w[4];
      __builtin_memcpy(w, p, 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(w[e] << 16);
        v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < n ? bf16_value(p[e]) : 0.f;
    }
  }
}
// once: L2 need not keep the lines (non-temporal stores).
typedef uint32_t FourAtTwo __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t FourAtFour __attribute__((ext_vector_type(4), aligned(4)));
template <bool F32>
__device__ __forceinline__ void store8(void* base, int64_t at, int n, const float (&v)[8], bool once = false) {
  if constexpr (F32) {
    float* p = (float*)base + at;
    if (n >= 8 && once) {
      asm volatile("" ::: "memory");      // else the compiler makes one store, not marked, of the two branches
      FourAtFour w[2];
      __builtin_memcpy(w, v, 32);
      __builtin_nontemporal_store(w[0], (FourAtFour*)p);
      __builtin_nontemporal_store(w[1], (FourAtFour*)p + 1);
      asm volatile("" ::: "memory");
    } else if (n >= 8) {
      __builtin_memcpy(p, v, 32);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) if (e < n) p[e] = v[e];
    }
  } else {
    uint16_t* p = (uint16_t*)base + at;
    if (n >= 8) {
      const FourAtTwo w = {two_bf16(v[0], v[1]), two_bf16(v[2], v[3]), two_bf16(v[4], v[5]), two_bf16(v[6], v[7])};
      if (once) {
        asm volatile("" ::: "memory");
        __builtin_nontemporal_store(w, (FourAtTwo*)p);
        asm volatile("" ::: "memory");
      } else {
        __builtin_memcpy(p, &w, 16);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) if (e < n) p[e] = bf16_bits(v[e]);
    }
  }
}
// Eight values as they lie in memory, on their way while something else is done.
template <bool F32>
struct Eight {
  uint32_t w[F32 ? 8 : 4];
  __device__ __forceinline__ void fetch(const void* base, int64_t at, int n) {
    if (n >= 8) {
      __builtin_memcpy(w, (const char*)base + at * (F32 ? 4 : 2), sizeof(w));
    } else {
#pragma unroll
      for (int e = 0; e < (F32 ? 8 : 4); ++e) w[e] = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e >= n) continue;
        if constexpr (F32) w[e] = ((const uint32_t*)base)[at + e];
        else w[e >> 1] |= (uint32_t)((const uint16_t*)base)[at + e] << (16 * (e & 1));
      }
    }
  }
  __device__ __forceinline__ float value(int e) const {
    if constexpr (F32) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
  }
};

// Place `i` of `total` so that each of the 8 dies, to which workgroups go in turn, gets consecutive places.
__device__ __forceinline__ int by_die(int i, int total) {
  const int each = total >> 3, more = total & 7, die = i & 7;
  return i < 8 * each + more ? die * each + min(die, more) + (i >> 3) : i;
}
// Tile (m, n) of nm x nn: columns within bands of 8 rows of tiles, so that what runs at one time on a die shares rows and columns.
__device__ __forceinline__ void tile_of(int i, int nm, int nn, int* m, int* n) {
  const int band = i / (8 * nn), first = 8 * band, high = min(8, nm - first), j = i - band * 8 * nn;
  *m = first + j % high;
  *n = j / high;
}

}  // namespace product
}  // namespace gmi
