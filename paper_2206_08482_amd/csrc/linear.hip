// Layers of a caller's own network: act(x W^T + b) + r and its gradients, one weight matrix for all rows or one per group of rows.
#include "product.h"

using namespace gmi::product;

namespace gmi {
constexpr uint32_t kMagicLinear = 0x474d494c;
}

struct gmi_linear {
  uint32_t magic;
  int device;
  gmi_linear_desc d;
  char* base;          // all of the workspace
  char *x, *w, *dz;    // packed operands (planes one after the other), dz
  float* part;         // fp32 sums of splits
  int64_t part_bytes;
  float* bias_part;    // sums of dz over a few rows
  int64_t x_plane, w_plane, dz_plane;      // bytes of one plane
};

namespace {

constexpr int kSlopeRows = 8, kSlopeRowsMost = 256;  // rows of a group whose dz a workgroup forms and sums
constexpr int64_t kPartBytes = (int64_t)64 << 20;    // most room for the sums of splits
constexpr int kMostSplits = 64;
// A launch has less than 2^32 threads: workgroups of any of the kernels (up to 1024 threads), of linear_prepare_kernel.
constexpr int64_t kMostBlocks = ((int64_t)1 << 22) - 1, kMostPrepareBlocks = ((int64_t)1 << 24) - 1;

inline bool valid(gmi_linear_t l) { return l && l->magic == gmi::kMagicLinear; }
inline int pad8(int v) { return (v + 7) & ~7; }

// ------------------------------------------------------------------ activations
// EXACT (fp32 layers): the library's functions.  Otherwise the hardware's exponential and reciprocal, 1e-7 .. 3e-7 of their value and, for the exponential,
// 6e-8 |z| of it more (its argument's rounding); what is below 2^-126 becomes 0.
template <bool EXACT>
__device__ __forceinline__ float exp_of(float z) { return EXACT ? expf(z) : __builtin_amdgcn_exp2f(z * 1.44269504f); }
template <bool EXACT>
__device__ __forceinline__ float sigmoid_of(float z) {
  const float d = 1.f + exp_of<EXACT>(-z);
  return EXACT ? 1.f / d : __builtin_amdgcn_rcpf(d);
}
// Phi(z).  Not EXACT: 1 - Phi(|z|) = e^(-z^2 / 2) t P(t) with t = 1 / (1 + 0.294 |z|) and P of degree 5, fitted to erfcx (alternately reweighted least
// squares, |z| up to 13.2) so that it is right to 2.5e-7 of 1 and to 4e-5 of itself: GELU's far negative values are as right as its others.
template <bool EXACT>
__device__ __forceinline__ float normal_cdf(float z) {
  if constexpr (EXACT) return 0.5f * erfcf(-0.70710678f * z);
  const float t = __builtin_amdgcn_rcpf(1.f + 0.29415643f * fabsf(z));
  const float poly =
      (((((-0.0848032236f * t + 0.257211983f) * t - 0.0609185249f) * t + 0.163766786f) * t + 0.106596917f) * t + 0.118145958f) * t;
  const float tail = poly * __builtin_amdgcn_exp2f(z * z * -0.72134752f);
  return z < 0.f ? tail : 1.f - tail;
}

// Eight values at a time: one branch for all of them, their chains of instructions side by side.
template <class F>
__device__ __forceinline__ void each8(float (&v)[8], F&& f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = f(v[e], e);
}
// z, or e^z - 1 below 0.  Not EXACT: the difference has the exponential's error of 1, 9e-8, whatever is left of the 1: 4e-4 of the value at
// |z| = 2^-12.  Nearer to 0 z + z^2 / 2 takes its place (1e-8 of the value), looked for once for eight values: 16384 x 211 -> 512 takes
// 20.45 us with it, 21.7 with a select for each value, 20.1 with the difference alone.
template <bool EXACT>
__device__ __forceinline__ void elu8(float (&v)[8]) {
  if constexpr (EXACT) {
    each8(v, [](float z, int) { return z > 0.f ? z : expm1f(z); });
  } else {
    constexpr float kNear = 1.f / 4096;
    float z[8], least = INFINITY;
    each8(v, [&](float x, int e) {
      z[e] = x;
      least = fminf(least, fabsf(x));
      return x > 0.f ? x : exp_of<false>(x) - 1.f;
    });
    if (__any(least < kNear)) each8(v, [&](float y, int e) { return z[e] < 0.f && z[e] > -kNear ? z[e] + 0.5f * z[e] * z[e] : y; });
  }
}
template <bool EXACT>
__device__ __forceinline__ void activate8(int act, float (&v)[8]) {
  switch (act) {
    case GMI_ACT_ELU: elu8<EXACT>(v); break;
    case GMI_ACT_RELU: each8(v, [](float z, int) { return z < 0.f ? 0.f : z; }); break;
    case GMI_ACT_SILU: each8(v, [](float z, int) { return EXACT ? z / (1.f + expf(-z)) : z * sigmoid_of<false>(z); }); break;
    case GMI_ACT_GELU: each8(v, [](float z, int) { return z * normal_cdf<EXACT>(z); }); break;
    default: break;
  }
}
// v times the activation's slope at z.
template <bool EXACT>
__device__ __forceinline__ void times_slope8(int act, const float (&z)[8], float (&v)[8]) {
  switch (act) {
    case GMI_ACT_ELU: each8(v, [&](float x, int e) { return z[e] > 0.f ? x : x * exp_of<EXACT>(z[e]); }); break;
    case GMI_ACT_RELU: each8(v, [&](float x, int e) { return x * (z[e] > 0.f ? 1.f : 0.f); }); break;
    case GMI_ACT_SILU:
      each8(v, [&](float x, int e) { const float s = sigmoid_of<EXACT>(z[e]); return x * (s * (1.f + z[e] * (1.f - s))); });
      break;
    case GMI_ACT_GELU:
      each8(v, [&](float x, int e) { return x * (normal_cdf<EXACT>(z[e]) + z[e] * 0.39894228f * exp_of<EXACT>(-0.5f * z[e] * z[e])); });
      break;
    default: break;
  }
}

// ------------------------------------------------------------------ operands in planes
// The planes of eight values of a packed operand.
template <bool F32>
__device__ __forceinline__ void store_planes(char* base, int64_t at, int64_t plane, const float (&v)[8]) {
  constexpr int N = F32 ? 3 : 1;
  uint32_t w[N][4];
  if constexpr (F32) {
    uint16_t p[8][N];
#pragma unroll
    for (int e = 0; e < 8; ++e) split_bf16<N>(v[e], p[e]);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) w[i][e] = p[2 * e][i] | (uint32_t)p[2 * e + 1][i] << 16;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[0][e] = two_bf16(v[2 * e], v[2 * e + 1]);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) *(uint4*)(base + i * plane + at * 2) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
}

// ------------------------------------------------------------------ groups of rows
struct Groups {
  const int* offsets;      // NULL: one group of all rows
  int n, rows;
};
struct Range { int begin, end; };
__device__ __forceinline__ Range group_rows(const Groups& G, int g) {
  if (!G.offsets) return {0, G.rows};
  const int a = min(max(G.offsets[g], 0), G.rows), b = min(max(G.offsets[g + 1], 0), G.rows);
  return {a, max(a, b)};
}
struct RowTile { int group, index, begin, end; };      // `index`: of the tile among all

// Tiles of T rows of each group, group after group.  A wave's lanes take 64 groups at a time.
__device__ __forceinline__ int group_tiles(const Groups& G, int g, int T) {
  if (g >= G.n) return 0;
  const Range r = group_rows(G, g);
  return (r.end - r.begin + T - 1) / T;
}
__device__ __forceinline__ int wave_inclusive(int v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(v, d);
    if (lane >= d) v += u;
  }
  return v;
}
__device__ __forceinline__ int count_tiles(const Groups& G, int T) {
  if (!G.offsets) return (G.rows + T - 1) / T;
  const int lane = threadIdx.x & 63;
  int total = 0;
  for (int g0 = 0; g0 < G.n; g0 += 64) total += __builtin_amdgcn_readlane(wave_inclusive(group_tiles(G, g0 + lane, T), lane), 63);
  return total;
}
// Tile `index` (< count_tiles); false if there is none.
__device__ __forceinline__ bool find_tile(const Groups& G, int T, int index, RowTile* out) {
  if (!G.offsets) {
    *out = {0, index, index * T, min(G.rows, index * T + T)};
    return index * T < G.rows;
  }
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int g0 = 0; g0 < G.n; g0 += 64) {
    const int own = group_tiles(G, g0 + lane, T), incl = wave_inclusive(own, lane);
    const uint64_t past = __ballot(before + incl > index);
    if (past) {
      const int l = __builtin_ctzll(past);
      const int first = before + __builtin_amdgcn_readlane(incl - own, l);
      const int g = __builtin_amdgcn_readfirstlane(g0 + l);
      const Range r = group_rows(G, g);
      const int b = r.begin + (index - first) * T;
      *out = {g, index, __builtin_amdgcn_readfirstlane(b), __builtin_amdgcn_readfirstlane(min(r.end, b + T))};
      return true;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}
// The group that holds a row, -1 if none does.
__device__ __forceinline__ int group_of(const Groups& G, int row) {
  if (!G.offsets) return 0;
  const int lane = threadIdx.x & 63;
  for (int g0 = 0; g0 < G.n; g0 += 64) {
    bool in = false;
    if (g0 + lane < G.n) {
      const Range r = group_rows(G, g0 + lane);
      in = row >= r.begin && row < r.end;
    }
    const uint64_t b = __ballot(in);
    if (b) return g0 + __builtin_ctzll(b);
  }
  return -1;
}

// ------------------------------------------------------------------ operands made ready
// Copies of operands that cannot be read in place (fp32: their bf16 planes; unaligned bf16: rows padded to 8), and dz with its sums over
// rows: dz = dy act'(pre), planes x = p0 + p1 + p2.  One launch, workgroups dealt to up to three jobs.  Bound by memory, each value read and
// written once: dz of 32768 x 512 (96 MiB) 17.6 us, 5.7 TB/s; the copy of 16384 x 211 (14 MB) 7.2 us, half of it the launch.  A workgroup's
// rows grow with the number of rows (slope_rows_for), so that the partial sums of dbias stay few.
struct PackJob {
  const void* src;
  int64_t ld, rows, plane;
  int cols;
  char* dst;
  int blocks;      // 0: no such job
};
struct SlopeJob {
  const void *dy, *pre;      // pre NULL: slope 1
  int64_t lddy, ldp;
  int rows;                  // of a workgroup's tile
  char* dz;                  // NULL: not stored
  int64_t plane;
  float* bias_part;          // [tile, cols padded to 8], NULL: not wanted
  int cols, act, blocks, across;      // blocks = tiles * across, 256 columns each
};
struct PrepareArgs {
  PackJob pack[2];
  SlopeJob slope;
  Groups groups;
};

template <bool F32>
__global__ __launch_bounds__(256) void linear_prepare_kernel(PrepareArgs a) {
  __shared__ float sums[8][256 + 8];
  int b = blockIdx.x;
  const int tid = threadIdx.x;
  if (b < a.slope.blocks) {
    const SlopeJob& j = a.slope;
    RowTile t;
    if (!find_tile(a.groups, j.rows, b / j.across, &t)) return;
    const int col = (b % j.across) * 256 + 8 * (tid & 31), colp = (j.cols + 7) & ~7, n = j.cols - col;
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.f;
    if (n > 0) {
#pragma unroll 2
      for (int r = t.begin + (tid >> 5); r < t.end; r += 8) {
        float v[8], z[8];
        load8<F32>(j.dy, r * j.lddy + col, n, v);
        if (j.pre) {
          load8<F32>(j.pre, r * j.ldp + col, n, z);
          times_slope8<F32>(j.act, z, v);      // past the row's end both are 0, and so is the product
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += v[e];
        if (j.dz) store_planes<F32>(j.dz, (int64_t)r * colp + col, j.plane, v);
      }
    }
    if (!j.bias_part) return;
    *(float4*)&sums[tid >> 5][8 * (tid & 31)] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    *(float4*)&sums[tid >> 5][8 * (tid & 31) + 4] = make_float4(sum[4], sum[5], sum[6], sum[7]);
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) s += sums[r][tid];
    const int c = (b % j.across) * 256 + tid;
    if (c < colp) j.bias_part[(int64_t)t.index * colp + c] = s;
    return;
  }
  b -= a.slope.blocks;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const PackJob& j = a.pack[k];
    if (b < j.blocks) {
      const int per_row = (j.cols + 7) >> 3;
      for (int64_t i = (int64_t)b * 256 + tid; i < j.rows * per_row; i += (int64_t)j.blocks * 256) {
        const int64_t r = i / per_row;
        const int c = (int)(i - r * per_row) * 8;
        float v[8];
        load8<F32>(j.src, r * j.ld + c, j.cols - c, v);
        store_planes<F32>(j.dst, i * 8, j.plane, v);
      }
      return;
    }
    b -= j.blocks;
  }
}

// ------------------------------------------------------------------ the products
// kForwardRaw: forward with x and w as they lie, wherever their rows begin and end (bf16, tiles whose waves have rings of their own).
enum Form { kForward = 0, kInputGrad = 1, kWeightGrad = 2, kForwardRaw = 3 };

struct ProductArgs {
  const char *p, *q;                      // operands, plane 0
  int64_t p_ld, q_ld, p_plane, q_plane;   // bytes
  int64_t p_group;                        // bytes from one group's weights to the next's (kWeightGrad: 0)
  Groups groups;
  int rows, cols, depth;                  // of the output, contraction length (kWeightGrad: rows = out_dim, depth unused)
  int splits;
  Pairs pairs;
  float* part;                            // splits > 1: [split][row][cols padded to 8]
  // epilogue
  void *out, *pre;
  const void* residual;
  int64_t ldo, ldp, ldr;
  const float* bias;                      // [group][cols]
  int act;
  bool once;                              // how out and pre are stored: stored_once
};

template <bool F32>
__device__ __forceinline__ Eight<F32> residual_of(const ProductArgs& a, int64_t row, int col) {
  Eight<F32> r = {};
  if (a.residual) r.fetch(a.residual, row * a.ldr + col, a.cols - col);
  return r;
}
// What follows the sums of eight columns of a row (forward: bias, pre-activations, activation, residual).
template <bool F32>
__device__ __forceinline__ void finish_row(const ProductArgs& a, int64_t row, int col, const float (&bias)[8], const Eight<F32>& residual, float (&v)[8]) {
  const int n = a.cols - col;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] += bias[e];
  if (a.pre) store8<F32>(a.pre, row * a.ldp + col, n, v, a.once);
  activate8<F32>(a.act, v);
  if (a.residual) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += residual.value(e);
  }
  store8<F32>(a.out, row * a.ldo + col, n, v, a.once);
}
__device__ __forceinline__ void load_bias(const ProductArgs& a, int group, int col, float (&b)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = a.bias && col + e < a.cols ? a.bias[(int64_t)group * a.cols + col + e] : 0.f;
}

// Workgroup `block` of a product: y = act(x w^T + b) + r, dx = dz w or dw = dz^T x; the tile comes from the place alone, the group from the
// offsets.  Bound by the matrix cores at the card's power limit with whole 256 x 256 tiles (4096 x 8192 x 4096 192 to 204 us, 1.35 to 1.43 PFLOP/s;
// 8192 x 4096 x 4096 206, with GELU, residual and z kept 232 to 239: the epilogue's 192 MiB are about 30 of it), by memory with few rows (1 x 4096 ->
// 4096 7.5 us, 4.5 TB/s), by the address units' 64 bytes a cycle and compute unit with 64 x 64 tiles.
template <class S, int FORM, bool F32>
__device__ __forceinline__ void product_block(const ProductArgs& a, int block, char* smem) {
  constexpr int TN = S::TN, TM = S::TM;
  const int nn = (a.cols + TN - 1) / TN;
  int group = 0, m0, m_end, n0, k0 = 0, k_len, split = 0;
  if constexpr (FORM == kWeightGrad) {
    const int nm = (a.rows + TM - 1) / TM, per_group = nm * nn;
    // The tiles of a (group, split) read the same rows, so they belong on one die, to which workgroups go in turn: eights of splits, one a die.
    // With fewer splits a group's tiles go over all dies (groups differ in their rows), those of one group of all rows in one sequence.
    int tile;
    if ((a.splits & 7) == 0) {
      const int unit = (block >> 3) / per_group, eights = a.splits >> 3;
      tile = (block >> 3) % per_group;
      group = unit / eights;
      split = unit % eights * 8 + (block & 7);
    } else if (a.groups.n > 1) {
      const int unit = block / per_group;
      tile = by_die(block % per_group, per_group);
      group = unit / a.splits;
      split = unit % a.splits;
    } else {
      const int i = by_die(block, a.splits * per_group);
      tile = i % per_group;
      split = i / per_group;
    }
    int mt, nt;
    tile_of(tile, nm, nn, &mt, &nt);
    m0 = mt * TM;
    m_end = min(a.rows, m0 + TM);
    n0 = nt * TN;
    const Range r = group_rows(a.groups, group);
    const int len = r.end - r.begin;
    const int chunk = ((len + a.splits - 1) / a.splits + kDepth - 1) & ~(kDepth - 1);
    k0 = __builtin_amdgcn_readfirstlane(min(r.end, r.begin + split * chunk));
    k_len = __builtin_amdgcn_readfirstlane(min(r.end, k0 + chunk)) - k0;
  } else {
    const int nm = count_tiles(a.groups, TM), total = nm * nn * a.splits;
    if (block >= total) return;
    int i = by_die(block, total);
    split = i / (nm * nn);
    int mt, nt;
    tile_of(i % (nm * nn), nm, nn, &mt, &nt);
    RowTile t;
    if (!find_tile(a.groups, TM, mt, &t)) return;
    group = t.group;
    m0 = t.begin;
    m_end = t.end;
    n0 = nt * TN;
    const int chunk = ((a.depth + a.splits - 1) / a.splits + kDepth - 1) & ~(kDepth - 1);
    k0 = min(a.depth, split * chunk);
    k_len = min(a.depth, k0 + chunk) - k0;
  }
  constexpr bool forward = FORM == kForward || FORM == kForwardRaw, PS = !forward, QS = FORM == kWeightGrad;
  Side P, Q;
  P.ld = a.p_ld; P.plane = a.p_plane; P.count = min(TN, a.cols - n0);
  P.base = a.p + group * a.p_group + (PS ? (int64_t)k0 * a.p_ld + (int64_t)n0 * 2 : (int64_t)n0 * a.p_ld + (int64_t)k0 * 2);
  Q.ld = a.q_ld; Q.plane = a.q_plane; Q.count = m_end - m0;
  Q.base = a.q + (QS ? (int64_t)k0 * a.q_ld + (int64_t)m0 * 2 : (int64_t)m0 * a.q_ld + (int64_t)k0 * 2);
  Accumulator<S> acc;
  multiply<S, PS, QS, false, FORM == kForwardRaw, F32>(P, Q, k_len, a.pairs, smem, acc);

  if (a.splits > 1) {
    const int pitch = (a.cols + 7) & ~7;
    const int64_t rows = FORM == kWeightGrad ? (int64_t)a.groups.n * a.rows : a.groups.rows;
    float* to = a.part + ((int64_t)split * rows + (FORM == kWeightGrad ? (int64_t)group * a.rows : 0)) * pitch;
    each_row<S>(acc, smem, FetchNothing(), [&](int m, int n, float (&v)[8], Nothing) {
      if (m0 + m < m_end && n0 + n < a.cols) store8<true>(to, (int64_t)(m0 + m) * pitch + n0 + n, 8, v);
    });
    return;
  }
  const int64_t first = FORM == kWeightGrad ? (int64_t)group * a.rows : 0;
  const int lane_n = lane_column<S>();
  float bias[8];
  if constexpr (forward) load_bias(a, group, n0 + lane_n, bias);
  if constexpr (forward) {
    each_row<S>(acc, smem, [&](int m, int n) { return m0 + m < m_end && n0 + n < a.cols ? residual_of<F32>(a, m0 + m, n0 + n) : Eight<F32>{}; },
                [&](int m, int n, float (&v)[8], const Eight<F32>& r) {
                  if (m0 + m < m_end && n0 + n < a.cols) finish_row<F32>(a, m0 + m, n0 + n, bias, r, v);
                });
  } else {
    each_row<S>(acc, smem, FetchNothing(), [&](int m, int n, float (&v)[8], Nothing) {
      if (m0 + m < m_end && n0 + n < a.cols) store8<F32>(a.out, (first + m0 + m) * a.ldo + n0 + n, a.cols - n0 - n, v, a.once);
    });
  }
}

template <class S, int FORM, bool F32>
__global__ __launch_bounds__(S::threads, kWavesPerSimd<S>) void linear_product_kernel(ProductArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  product_block<S, FORM, F32>(a, blockIdx.x, smem);
}

// dbias: the sums of a group's row tiles in their order, 32 columns a workgroup, each of its slices of 32 threads every so many tiles.  A few us
// of reads that wait on one another where it is a launch of its own; beside the products they cost nothing that shows.
struct BiasJob {
  const float* part;
  float* out;
  int cols, rows, tiles, blocks;      // rows of a tile, most tiles of all groups; blocks = groups * (cols / 32 rounded up), 0: no such job
};
template <int THREADS>
__device__ __forceinline__ void bias_block(const BiasJob& j, const Groups& groups, int block, float* sums) {
  constexpr int slices = THREADS / 32;
  const int across = (j.cols + 31) / 32, g = block / across, lane = threadIdx.x & 63;
  const int c = block % across * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5, pitch = (j.cols + 7) & ~7;
  int first = 0;
  if (groups.offsets) {
    for (int g0 = 0; g0 < g; g0 += 64)
      first += __builtin_amdgcn_readlane(wave_inclusive(g0 + lane < g ? group_tiles(groups, g0 + lane, j.rows) : 0, lane), 63);
  }
  const int last = min(j.tiles, first + group_tiles(groups, g, j.rows));
  float s = 0.f;
  if (c < j.cols) {
#pragma unroll 8
    for (int t = first + slice; t < last; t += slices) s += j.part[(int64_t)t * pitch + c];
  }
  sums[slice * 32 + (threadIdx.x & 31)] = s;
  __syncthreads();
  if (slice || c >= j.cols) return;
  for (int i = 1; i < slices; ++i) s += sums[i * 32 + threadIdx.x];
  j.out[(int64_t)g * j.cols + c] = s;
}
__global__ __launch_bounds__(1024) void linear_bias_kernel(BiasJob j, Groups groups) {
  __shared__ float sums[1024];
  for (int b = blockIdx.x; b < j.blocks; b += gridDim.x) {
    bias_block<1024>(j, groups, b, sums);
    __syncthreads();
  }
}

// The backward pass's two products and the bias's sums, which all read dz, in one launch: what one leaves of the chip idle the next takes.
// 16384 rows over 8 experts of 2048 -> 1024: 134 us for 137 GFLOP, 1.03 PFLOP/s; groups that end inside a tile and the last round of the
// workgroups are what is missing to the rate of one large product.
template <class S, bool F32>
__global__ __launch_bounds__(S::threads, kWavesPerSimd<S>) void linear_gradients_kernel(ProductArgs x, int x_blocks, ProductArgs w, int w_blocks, BiasJob bias) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  int b = blockIdx.x;
  if (b < w_blocks) { product_block<S, kWeightGrad, F32>(w, b, smem); return; }
  b -= w_blocks;
  if (b < x_blocks) { product_block<S, kInputGrad, F32>(x, b, smem); return; }
  bias_block<S::threads>(bias, x.groups, b - x_blocks, (float*)smem);
}

// Sums of the splits in their order, so that a call's result is the same each time, and what follows them.  A wave per row, 512 columns at a
// time.  Bound by memory: 16 splits of 512 x 512 (17 MB) 4.9 us.
template <bool F32, bool WEIGHT>
__global__ __launch_bounds__(256) void linear_join_kernel(ProductArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t rows = WEIGHT ? (int64_t)a.groups.n * a.rows : a.groups.rows;
  if (row >= rows) return;
  int group = 0;
  if constexpr (!WEIGHT) {
    group = group_of(a.groups, (int)row);
    if (group < 0) return;
  }
  const int pitch = (a.cols + 7) & ~7;
  const int col = (blockIdx.y * 64 + lane) * 8;
  if (col >= a.cols) return;
  float v[8], bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  const float* from = a.part + row * pitch + col;
#pragma unroll 4
  for (int s = 0; s < a.splits; ++s) {
    float u[8];
    load8<true>(from, s * rows * pitch, 8, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += u[e];
  }
  load_bias(a, group, col, bias);
  finish_row<F32>(a, row, col, bias, residual_of<F32>(a, row, col), v);
}

// ------------------------------------------------------------------ host
// A division of the contraction costs another launch and the sums' way out and in.
constexpr float kJoin = 4.5f, kJoinBytesPerUs = 4e6f;
struct Plan { int shape, splits; };      // shape: place in kTiles of product.h

// Most tiles of tm x tn; rows of groups: each may end inside a tile.
int64_t tiles_of(int64_t rows, int64_t cols, int groups, const int (&tile)[2], bool weight) {
  const int64_t nm = (rows + tile[0] - 1) / tile[0], nn = (cols + tile[1] - 1) / tile[1];
  return weight ? groups * nm * nn : (nm + (groups > 1 ? groups - 1 : 0)) * nn;
}

struct Work {      // a product to plan
  int64_t rows, cols, depth;      // of one group (weight gradients) or of all; contraction length on average
  int products, groups, form;
  int64_t room;                   // bytes for the sums of splits
};
Work work_of(const gmi_linear* l, const ProductArgs& a, int form, int64_t depth) {
  return {form == kWeightGrad ? a.rows : a.groups.rows, a.cols, depth, a.pairs.n, a.groups.n, form, l->part_bytes};
}
int64_t blocks_of(const Work& w, int shape, int splits) {
  return tiles_of(w.rows, w.cols, w.groups, kTiles[shape].size, w.form == kWeightGrad) * splits;
}
// Of a product with tile i and s splits: us of a compute unit in all, of its longest workgroup (which shares its unit if there are that many),
// and of joining the splits.  sum < 0: not to be had.
struct Cost { float sum, longest, join, rounds; };
Cost cost_of(const gmi_instance* g, const Work& w, int i, int s) {
  const bool weight = w.form == kWeightGrad;
  const Tile& tile = kTiles[i];
  const int64_t bytes = (weight ? w.rows * w.groups : w.rows) * ((w.cols + 7) & ~7) * 4, cus = g->cu_count;
  // of groups of unknown sizes each ends inside a tile, on average in the middle
  const int64_t tiles = s * (weight ? tiles_of(w.rows, w.cols, w.groups, tile.size, true)
                                    : tiles_of(w.rows, w.cols, 1, tile.size, false) +
                                          (w.groups > 1 ? w.groups / 2 * ((w.cols + tile.size[1] - 1) / tile.size[1]) : 0));
  if (s > 1 && (w.depth < 64 * s || bytes * s > w.room || tiles > 4 * cus)) return {-1.f, 0.f, 0.f, 0.f};
  if (blocks_of(w, i, s) > kMostBlocks) return {-1.f, 0.f, 0.f, 0.f};
  const float unit = tile_time(tile, (float)(w.depth * w.products) / s), alone = tile.alone * unit;
  Cost c;
  c.sum = (float)tiles / cus * unit;
  // the largest of several groups is taken to have twice the rows of the average
  c.longest = (tiles > cus ? tile.share * unit : alone) * (weight && w.groups > 1 ? 2.f : 1.f);
  c.join = s > 1 ? kJoin + 2.f * (float)bytes * s / kJoinBytesPerUs : 0.f;
  const int64_t slots = cus * tile.share, rest = tiles % slots;
  c.rounds = (float)(tiles / slots) * tile.share * unit + (rest == 0 ? 0.f : rest <= cus ? alone : tile.share * unit);
  if (w.groups > 1) c.rounds = std::max(c.longest, c.sum + 0.35f * c.longest);
  return c;
}
constexpr float kNever = 1e30f;
// The tile and the number of splits of the contraction that take least by these figures.  *time kNever: more workgroups than a launch has, with any.
Plan plan_product(const gmi_instance* g, const Work& w, float* time) {
  const int n_tiles = w.form == kForward ? 7 : w.form == kInputGrad ? 5 : 4;      // those built for the form
  Plan best = {0, 1};
  *time = kNever;
  for (int i = 0; i < n_tiles; ++i)
    for (int s = 1; s <= kMostSplits; s *= 2) {
      const Cost c = cost_of(g, w, i, s);
      if (c.sum < 0.f) break;
      const float t = kStart + c.rounds + c.join;
      if (t < *time) { *time = t; best = {i, s}; }
    }
  return best;
}
// Both products of a backward pass with one tile (weight gradients in s splits) in one launch, beside `others` workgroups.
Plan plan_gradients(const gmi_instance* g, const Work& x, const Work& w, int64_t others, float* time) {
  Plan best = {0, 1};
  *time = kNever;
  for (int i = 0; i < 4; ++i)
    for (int s = 1; s <= kMostSplits; s *= 2) {
      const Cost cx = cost_of(g, x, i, 1), cw = cost_of(g, w, i, s);
      if (cx.sum < 0.f || cw.sum < 0.f || blocks_of(x, i, 1) + blocks_of(w, i, s) + others > kMostBlocks) break;
      const float share = (cx.sum > 0.5f * cx.longest ? kTiles[i].share : 1);      // the weights' workgroups run beside the others
      const float t = kStart + std::max(std::max(cx.longest, cw.longest * share), cx.sum + cw.sum + 0.5f * cx.longest) + cw.join;
      if (t < *time) { *time = t; best = {i, s}; }
    }
  return best;
}

template <class S, int FORM, bool F32>
int launch_product(gmi_instance* g, const ProductArgs& a, int64_t blocks) {
  static gmi::DeviceSet allowed;
  const int rc = gmi::allow_lds((const void*)linear_product_kernel<S, FORM, F32>, S::lds, g->device, &allowed);
  if (rc != GMI_OK) return rc;
  linear_product_kernel<S, FORM, F32><<<dim3((unsigned)blocks), S::threads, S::lds, g->stream>>>(a);
  GMI_LAUNCH_CHECK();
  return GMI_OK;
}

template <bool F32, bool WEIGHT>
int launch_join(gmi_instance* g, const ProductArgs& a) {
  const int64_t rows = WEIGHT ? (int64_t)a.groups.n * a.rows : a.groups.rows;
  linear_join_kernel<F32, WEIGHT><<<dim3((unsigned)((rows + 3) / 4), (unsigned)((a.cols + 511) / 512)), 256, 0, g->stream>>>(a);
  GMI_LAUNCH_CHECK();
  return GMI_OK;
}
int64_t blocks_of(const ProductArgs& a, bool weight, const Plan& p) {
  return tiles_of(weight ? a.rows : a.groups.rows, a.cols, a.groups.n, kTiles[p.shape].size, weight) * p.splits;
}

// Whether an output's lines are stored as ones that L2 need not keep: less is left to be written back when the launch ends.  16384 x 512 -> 512
// with z kept (32 MiB) 20.0 -> 17.9 us, input gradients of 4096 x 1024 x 1024 (8 MiB) 17.2 -> 15.3, the backward pass of 16384 rows over 8 experts
// of 2048 -> 1024 157 -> 145; three layers of 4096 x 512 -> 512 (4 MiB) 31.2 -> 30.8.  Not below that, where the next layer finds them in L2
// (2048 x 512, 2 MiB: 24.1 -> 24.9), nor of rows that end within a line (16384 x 211 -> 300: 25.4 -> 25.9), nor of more than the chip's last
// cache holds beside the rest (16384 x 1024 -> 2048 with z kept, 128 MiB: 80 -> 91).
bool stored_once(const void* p, int64_t ld, int size, int64_t bytes) {
  return (uintptr_t)p % 128 == 0 && ld * size % 128 == 0 && bytes >= (int64_t)1 << 22 && bytes <= (int64_t)1 << 26;
}

int run_raw(gmi_instance* g, const ProductArgs& a, const Plan& p) {
  const int64_t blocks = blocks_of(a, false, p);
  return p.shape == 4 ? launch_product<Few, kForwardRaw, false>(g, a, blocks) : launch_product<Row, kForwardRaw, false>(g, a, blocks);
}

template <int FORM, bool F32>
int run_product(gmi_instance* g, ProductArgs a, const Plan& p) {
  constexpr bool weight = FORM == kWeightGrad;
  a.splits = p.splits;
  const int64_t blocks = blocks_of(a, weight, p);
  if (blocks == 0) return GMI_OK;
  int rc;
  switch (p.shape) {
    case 0: rc = launch_product<Large, FORM, F32>(g, a, blocks); break;
    case 1: rc = launch_product<Medium, FORM, F32>(g, a, blocks); break;
    case 2: rc = launch_product<Small, FORM, F32>(g, a, blocks); break;
    case 3: rc = launch_product<Twin, FORM, F32>(g, a, blocks); break;
    case 4:
      if constexpr (FORM == kWeightGrad) return GMI_ERR_UNSUPPORTED;
      else rc = launch_product<Few, FORM, F32>(g, a, blocks);
      break;
    default:
      if constexpr (FORM != kForward) return GMI_ERR_UNSUPPORTED;
      else rc = p.shape == 5 ? launch_product<Row, FORM, F32>(g, a, blocks) : launch_product<Middle, FORM, F32>(g, a, blocks);
  }
  if (rc != GMI_OK || p.splits == 1) return rc;
  return launch_join<F32, weight>(g, a);
}

template <class S, bool F32>
int launch_gradients(gmi_instance* g, const ProductArgs& x, int64_t x_blocks, const ProductArgs& w, int64_t w_blocks, const BiasJob& bias) {
  static gmi::DeviceSet allowed;
  const int rc = gmi::allow_lds((const void*)linear_gradients_kernel<S, F32>, S::lds, g->device, &allowed);
  if (rc != GMI_OK) return rc;
  linear_gradients_kernel<S, F32><<<dim3((unsigned)(x_blocks + w_blocks + bias.blocks)), S::threads, S::lds, g->stream>>>(x, (int)x_blocks, w, (int)w_blocks, bias);
  GMI_LAUNCH_CHECK();
  return GMI_OK;
}
// weights NULL: the input gradients and the bias's sums alone.
template <bool F32>
int run_gradients(gmi_instance* g, ProductArgs x, const ProductArgs* weights, const BiasJob& bias, const Plan& p) {
  x.splits = 1;
  ProductArgs w = weights ? *weights : x;
  w.splits = p.splits;
  const int64_t xb = blocks_of(x, false, {p.shape, 1}), wb = weights ? blocks_of(w, true, p) : 0;
  const int rc = p.shape == 0   ? launch_gradients<Large, F32>(g, x, xb, w, wb, bias)
                 : p.shape == 1 ? launch_gradients<Medium, F32>(g, x, xb, w, wb, bias)
                 : p.shape == 2 ? launch_gradients<Small, F32>(g, x, xb, w, wb, bias) : launch_gradients<Twin, F32>(g, x, xb, w, wb, bias);
  if (rc != GMI_OK || p.splits == 1 || !weights) return rc;
  return launch_join<F32, true>(g, w);
}

// Rows whose dz a workgroup forms: few while that leaves compute units without work.
int slope_rows_for(int cus, int64_t rows, int across) {
  int r = kSlopeRows;
  while (r < kSlopeRowsMost && (rows + r - 1) / r * across > 4 * cus) r *= 2;
  return r;
}

struct Matrix { const void* p; int64_t ld; int64_t rows; int cols; };

bool in_place(const gmi_linear* l, const Matrix& m) {
  return l->d.dtype == GMI_DTYPE_BF16 && (uintptr_t)m.p % 16 == 0 && m.ld % 8 == 0 && m.cols % 8 == 0 && m.ld < (1 << 22);
}
PackJob pack_job(const Matrix& m, char* dst, int64_t plane) {
  const int64_t pieces = m.rows * ((m.cols + 7) / 8);
  return {m.p, m.ld, m.rows, plane, m.cols, dst, (int)std::min<int64_t>((pieces + 255) / 256, 4096)};
}

// The bytes of a [rows, cols] array: rows of `row` bytes, `pitch` apart.
struct Span { const char *a, *b; int64_t row, pitch; };
Span span_of(const gmi_linear* l, const void* p, int64_t rows, int64_t cols, int64_t ld, int bytes = 0) {
  if (!p || rows < 1) return {nullptr, nullptr, 0, 0};
  const int64_t e = bytes ? bytes : l->d.dtype == GMI_DTYPE_F32 ? 4 : 2;
  return {(const char*)p, (const char*)p + ((rows - 1) * ld + cols) * e, cols * e, ld * e};
}
// Whether two arrays share bytes; column ranges of one wider array (the same pitch) may interleave without.
bool overlap(const Span& x, const Span& y) {
  if (!x.a || !y.a || x.a >= y.b || y.a >= x.b) return false;
  if (x.pitch != y.pitch) return true;
  const int64_t d = y.a >= x.a ? (y.a - x.a) % x.pitch : (x.pitch - (x.a - y.a) % x.pitch) % x.pitch;
  return d < x.row || d + y.row > x.pitch;
}

int check_call(const char* who, gmi_t g, gmi_linear_t l, bool grouped, const int32_t* offsets, int32_t n_rows, bool backward) {
  if (!valid(g)) GMI_FAIL(GMI_ERR_BAD_HANDLE, "%s: bad instance", who);
  if (!valid(l)) GMI_FAIL(GMI_ERR_BAD_HANDLE, "%s: bad binding", who);
  if (g->device != l->device) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: instance and binding live on different devices", who);
  if (grouped != (l->d.n_groups > 0)) GMI_FAIL(GMI_ERR_UNSUPPORTED, "%s: the binding has n_groups = %d", who, l->d.n_groups);
  if (grouped && (!offsets || (uintptr_t)offsets % 4)) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: offsets is NULL or not aligned", who);
  if (backward && !l->d.backward) GMI_FAIL(GMI_ERR_UNSUPPORTED, "%s: the binding is forward only", who);
  if (n_rows < 0 || n_rows > l->d.max_rows) GMI_FAIL(GMI_ERR_BAD_SHAPE, "%s: n_rows %d outside 0 .. %d", who, n_rows, l->d.max_rows);
  return GMI_OK;
}
int check_matrix(const char* who, const char* name, const gmi_linear* l, const void* p, int64_t ld, int64_t cols, bool needed) {
  if (!p) {
    if (needed) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
    return GMI_OK;
  }
  if ((uintptr_t)p % (l->d.dtype == GMI_DTYPE_F32 ? 4 : 2)) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: %s is not aligned to its elements", who, name);
  if (ld < cols) GMI_FAIL(GMI_ERR_BAD_SHAPE, "%s: the pitch of %s (%lld) is less than a row (%lld)", who, name, (long long)ld, (long long)cols);
  return GMI_OK;
}
#define LINEAR_TRY(expr) do { const int rc__ = (expr); if (rc__ != GMI_OK) return rc__; } while (0)

template <bool F32>
int forward(const char* who, gmi_t g, gmi_linear_t l, const void* x, int64_t ldx, const int32_t* offsets, const void* w, const float* bias,
            const void* residual, int64_t ldr, int32_t n_rows, void* y, int64_t ldy, void* pre, int64_t ldp) {
  const gmi_linear_desc& d = l->d;
  const int groups = std::max(1, d.n_groups), Kp = pad8(d.in_dim);
  PrepareArgs pa = {};
  ProductArgs a = {};
  a.groups = {offsets, groups, n_rows};
  const Matrix X = {x, ldx, n_rows, d.in_dim}, W = {w, d.in_dim, (int64_t)groups * d.out_dim, d.in_dim};
  a.q = (const char*)x; a.q_ld = ldx * 2;
  a.p = (const char*)w; a.p_ld = (int64_t)d.in_dim * 2;
  a.rows = n_rows; a.cols = d.out_dim; a.depth = Kp;
  a.pairs = F32 ? kThreePlanes : kOnePlane;
  a.splits = 1;
  a.part = l->part;
  a.out = y; a.ldo = ldy;
  a.pre = pre; a.ldp = ldp;
  a.residual = residual; a.ldr = ldr;
  a.bias = bias; a.act = d.act;
  a.once = stored_once(y, ldy, F32 ? 4 : 2, (int64_t)n_rows * d.out_dim * (F32 ? 4 : 2) * (pre ? 2 : 1));
  float time;
  const Plan plan = plan_product(g, work_of(l, a, kForward, Kp), &time);
  if (time >= kNever) GMI_FAIL(GMI_ERR_BAD_SHAPE, "%s: more tiles than a launch has workgroups", who);
  const bool x_fits = in_place(l, X), w_fits = in_place(l, W);
  // A packed copy is a launch of its own, and one of w reads and writes all groups' weights.  Through registers w goes into as many tiles as
  // there are 16 rows: 1 x 4097 -> 4096 23 -> 13.4 us, 64 x 4097 -> 1024 16.2 -> 13.3, 16 rows over 64 experts of 4001 -> 4096 886 -> 14;
  // with more rows a tile the shifting costs more than the copy: 256 x 1001 -> 512 11.1 -> 17, 1000 rows over 8 experts of 211 -> 300 12.5 -> 14.6.
  if (!F32 && !(x_fits && w_fits) && (plan.shape == 4 || plan.shape == 5) && plan.splits == 1 && n_rows <= (int64_t)64 * groups &&
      ldx <= (1 << 24)) {
    a.depth = d.in_dim;
    a.p_group = a.p_ld * d.out_dim;
    return run_raw(g, a, plan);
  }
  if (!x_fits) { pa.pack[0] = pack_job(X, l->x, l->x_plane); a.q = l->x; a.q_ld = Kp * 2; a.q_plane = l->x_plane; }
  if (!w_fits) { pa.pack[1] = pack_job(W, l->w, l->w_plane); a.p = l->w; a.p_ld = Kp * 2; a.p_plane = l->w_plane; }
  const int blocks = pa.pack[0].blocks + pa.pack[1].blocks;
  if (blocks) {
    linear_prepare_kernel<F32><<<blocks, 256, 0, g->stream>>>(pa);
    GMI_LAUNCH_CHECK();
  }
  a.p_group = a.p_ld * d.out_dim;
  return run_product<kForward, F32>(g, a, plan);
}

int forward_call(const char* who, bool grouped, gmi_t g, gmi_linear_t l, const void* x, int64_t ldx, const int32_t* offsets, const void* w,
                 const float* bias, const void* residual, int64_t ldr, int32_t n_rows, void* y, int64_t ldy, void* pre, int64_t ldp) {
  LINEAR_TRY(check_call(who, g, l, grouped, offsets, n_rows, false));
  const gmi_linear_desc& d = l->d;
  if (n_rows == 0) return GMI_OK;
  LINEAR_TRY(check_matrix(who, "x", l, x, ldx, d.in_dim, true));
  LINEAR_TRY(check_matrix(who, "w", l, w, d.in_dim, d.in_dim, true));
  LINEAR_TRY(check_matrix(who, "residual", l, residual, ldr, d.out_dim, false));
  LINEAR_TRY(check_matrix(who, "y", l, y, ldy, d.out_dim, true));
  LINEAR_TRY(check_matrix(who, "pre", l, pre, ldp, d.out_dim, false));
  if ((uintptr_t)bias % 4) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: bias is not aligned", who);
  const int64_t groups = std::max(1, d.n_groups);
  const Span sx = span_of(l, x, n_rows, d.in_dim, ldx), sw = span_of(l, w, groups * d.out_dim, d.in_dim, d.in_dim),
             sr = span_of(l, residual, n_rows, d.out_dim, ldr), sy = span_of(l, y, n_rows, d.out_dim, ldy),
             sp = span_of(l, pre, n_rows, d.out_dim, ldp), sb = span_of(l, bias, groups, d.out_dim, d.out_dim, 4),
             so = span_of(l, offsets, 1, groups + 1, groups + 1, 4);
  const bool same = residual == y && ldr == ldy;
  if (overlap(sy, sx) || overlap(sy, sw) || (!same && overlap(sy, sr)) || overlap(sy, sp) || overlap(sy, sb) || overlap(sp, sx) ||
      overlap(sp, sw) || overlap(sp, sr) || overlap(sp, sb) || overlap(sy, so) || overlap(sp, so))
    GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: an output overlaps another argument", who);
  return d.dtype == GMI_DTYPE_F32
             ? forward<true>(who, g, l, x, ldx, offsets, w, bias, residual, ldr, n_rows, y, ldy, pre, ldp)
             : forward<false>(who, g, l, x, ldx, offsets, w, bias, residual, ldr, n_rows, y, ldy, pre, ldp);
}

template <bool F32>
int backward(const char* who, gmi_t g, gmi_linear_t l, const void* dy, int64_t lddy, const void* x, int64_t ldx, const int32_t* offsets,
             const void* w, const void* pre, int64_t ldp, int32_t n_rows, void* dx, int64_t lddx, void* dw, float* dbias) {
  const gmi_linear_desc& d = l->d;
  const int groups = std::max(1, d.n_groups), Kp = pad8(d.in_dim), Np = pad8(d.out_dim);
  const Groups G = {offsets, groups, n_rows};
  const Pairs pairs = F32 ? kThreePlanes : kOnePlane;
  PrepareArgs pa = {};
  pa.groups = G;
  const Matrix X = {x, ldx, n_rows, d.in_dim}, W = {w, d.in_dim, (int64_t)groups * d.out_dim, d.in_dim}, DY = {dy, lddy, n_rows, d.out_dim};
  const char *xp = (const char*)x, *wp = (const char*)w, *zp = (const char*)dy;
  int64_t x_ld = ldx * 2, w_ld = (int64_t)d.in_dim * 2, z_ld = lddy * 2;
  if (dw && n_rows && !in_place(l, X)) { pa.pack[0] = pack_job(X, l->x, l->x_plane); xp = l->x; x_ld = Kp * 2; }
  if (dx && n_rows && !in_place(l, W)) { pa.pack[1] = pack_job(W, l->w, l->w_plane); wp = l->w; w_ld = Kp * 2; }
  const bool stored = (dx || dw) && (d.act != GMI_ACT_NONE || !in_place(l, DY));      // dz is not dy as it lies
  const int across = (d.out_dim + 255) / 256, slope_rows = slope_rows_for(g->cu_count, n_rows, across);
  const int64_t tiles = (n_rows + slope_rows - 1) / slope_rows + groups - 1;
  BiasJob bias = {l->bias_part, dbias, d.out_dim, slope_rows, (int)tiles, dbias ? groups * ((d.out_dim + 31) / 32) : 0};
  if (n_rows && (stored || dbias)) {
    pa.slope = {dy, d.act != GMI_ACT_NONE ? pre : nullptr, lddy, ldp, slope_rows, stored ? l->dz : nullptr, l->dz_plane, dbias ? l->bias_part : nullptr,
                d.out_dim, d.act, (int)(tiles * across), across};
    if (stored) { zp = l->dz; z_ld = Np * 2; }
  }
  ProductArgs a = {};
  a.groups = G;
  a.pairs = pairs;
  a.part = l->part;
  a.splits = 1;
  ProductArgs bx = a, bw = a;
  bx.q = zp; bx.q_ld = z_ld; bx.q_plane = l->dz_plane;
  bx.p = wp; bx.p_ld = w_ld; bx.p_plane = l->w_plane; bx.p_group = w_ld * d.out_dim;
  bx.rows = n_rows; bx.cols = d.in_dim; bx.depth = d.out_dim;
  bx.out = dx; bx.ldo = lddx;
  bx.once = stored_once(dx, lddx, F32 ? 4 : 2, (int64_t)n_rows * d.in_dim * (F32 ? 4 : 2));
  bw.p = xp; bw.p_ld = x_ld; bw.p_plane = l->x_plane;
  bw.q = zp; bw.q_ld = z_ld; bw.q_plane = l->dz_plane;
  bw.rows = d.out_dim; bw.cols = d.in_dim;
  bw.out = dw; bw.ldo = d.in_dim;
  bw.once = stored_once(dw, d.in_dim, F32 ? 4 : 2, (int64_t)groups * d.out_dim * d.in_dim * (F32 ? 4 : 2));
  const Work wx = work_of(l, bx, kInputGrad, d.out_dim), ww = work_of(l, bw, kWeightGrad, n_rows / groups);
  float tx = 0.f, tw = 0.f, both = kNever;
  const bool have_x = dx && n_rows;
  const Plan px = have_x ? plan_product(g, wx, &tx) : Plan(), pw = dw ? plan_product(g, ww, &tw) : Plan();
  Plan pb = {};
  if (have_x && dw) pb = plan_gradients(g, wx, ww, bias.blocks, &both);
  const int64_t blocks = (n_rows && (stored || dbias) ? tiles * across : 0) + pa.pack[0].blocks + pa.pack[1].blocks;
  if (tx >= kNever || tw >= kNever || blocks > kMostPrepareBlocks) GMI_FAIL(GMI_ERR_BAD_SHAPE, "%s: more tiles than a launch has workgroups", who);
  if (blocks) {
    linear_prepare_kernel<F32><<<dim3((unsigned)blocks), 256, 0, g->stream>>>(pa);
    GMI_LAUNCH_CHECK();
  }
  if (both <= tx + tw + (bias.blocks ? kStart : 0.f)) return run_gradients<F32>(g, bx, &bw, bias, pb);
  if (have_x && bias.blocks && px.shape < 4 && px.splits == 1 && blocks_of(bx, false, px) + bias.blocks <= kMostBlocks) {
    LINEAR_TRY(run_gradients<F32>(g, bx, nullptr, bias, px));
    bias.blocks = 0;
  } else if (have_x) {
    LINEAR_TRY((run_product<kInputGrad, F32>(g, bx, px)));
  }
  if (dw) LINEAR_TRY((run_product<kWeightGrad, F32>(g, bw, pw)));
  if (bias.blocks) {
    linear_bias_kernel<<<dim3((unsigned)std::min<int64_t>(bias.blocks, kMostBlocks)), 1024, 0, g->stream>>>(bias, G);
    GMI_LAUNCH_CHECK();
  }
  return GMI_OK;
}

int backward_call(const char* who, bool grouped, gmi_t g, gmi_linear_t l, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                  const int32_t* offsets, const void* w, const void* pre, int64_t ldp, int32_t n_rows, void* dx, int64_t lddx, void* dw,
                  float* dbias) {
  LINEAR_TRY(check_call(who, g, l, grouped, offsets, n_rows, true));
  const gmi_linear_desc& d = l->d;
  if (n_rows) {
    LINEAR_TRY(check_matrix(who, "dy", l, dy, lddy, d.out_dim, true));
    LINEAR_TRY(check_matrix(who, "x", l, x, ldx, d.in_dim, dw != nullptr));
    LINEAR_TRY(check_matrix(who, "w", l, w, d.in_dim, d.in_dim, dx != nullptr));
    LINEAR_TRY(check_matrix(who, "pre", l, pre, ldp, d.out_dim, d.act != GMI_ACT_NONE));
    LINEAR_TRY(check_matrix(who, "dx", l, dx, lddx, d.in_dim, false));
  }
  LINEAR_TRY(check_matrix(who, "dw", l, dw, d.in_dim, d.in_dim, false));
  if ((uintptr_t)dbias % 4) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: dbias is not aligned", who);
  const int64_t groups = std::max(1, d.n_groups);
  const Span in[5] = {span_of(l, dy, n_rows, d.out_dim, lddy), span_of(l, dw ? x : nullptr, n_rows, d.in_dim, ldx),
                      span_of(l, dx ? w : nullptr, groups * d.out_dim, d.in_dim, d.in_dim),
                      span_of(l, d.act != GMI_ACT_NONE ? pre : nullptr, n_rows, d.out_dim, ldp), span_of(l, offsets, 1, groups + 1, groups + 1, 4)};
  const Span out[3] = {span_of(l, dx, n_rows, d.in_dim, lddx), span_of(l, dw, groups * d.out_dim, d.in_dim, d.in_dim),
                       span_of(l, dbias, groups, d.out_dim, d.out_dim, 4)};
  for (int i = 0; i < 3; ++i) {
    for (const Span& s : in)
      if (overlap(out[i], s)) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: an output overlaps an input", who);
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: two outputs overlap", who);
  }
  return d.dtype == GMI_DTYPE_F32
             ? backward<true>(who, g, l, dy, lddy, x, ldx, offsets, w, pre, ldp, n_rows, dx, lddx, dw, dbias)
             : backward<false>(who, g, l, dy, lddy, x, ldx, offsets, w, pre, ldp, n_rows, dx, lddx, dw, dbias);
}

}  // namespace

extern "C" int gmi_linear_bind(gmi_t g, const gmi_linear_desc* d, gmi_linear_t* out) {
  if (!out) GMI_FAIL(GMI_ERR_INVALID_ARG, "gmi_linear_bind: out is NULL");
  *out = nullptr;
  if (!valid(g)) GMI_FAIL(GMI_ERR_BAD_HANDLE, "gmi_linear_bind: bad instance");
  if (!d) GMI_FAIL(GMI_ERR_INVALID_ARG, "gmi_linear_bind: desc is NULL");
  if (d->in_dim < 1 || d->in_dim > 65536 || d->out_dim < 1 || d->out_dim > 65536)
    GMI_FAIL(GMI_ERR_BAD_SHAPE, "gmi_linear_bind: in_dim %d, out_dim %d outside 1 .. 65536", d->in_dim, d->out_dim);
  if (d->n_groups < 0 || d->n_groups > 65535) GMI_FAIL(GMI_ERR_BAD_SHAPE, "gmi_linear_bind: n_groups %d outside 0 .. 65535", d->n_groups);
  if (d->max_rows < 1 || d->max_rows > (1 << 30)) GMI_FAIL(GMI_ERR_BAD_SHAPE, "gmi_linear_bind: max_rows %d outside 1 .. 2^30", d->max_rows);
  if (d->dtype != GMI_DTYPE_F32 && d->dtype != GMI_DTYPE_BF16) GMI_FAIL(GMI_ERR_UNSUPPORTED, "gmi_linear_bind: dtype %d", d->dtype);
  if (d->act < GMI_ACT_NONE || d->act > GMI_ACT_GELU) GMI_FAIL(GMI_ERR_UNSUPPORTED, "gmi_linear_bind: activation %d", d->act);
  const int64_t planes = d->dtype == GMI_DTYPE_F32 ? 3 : 1, groups = d->n_groups > 0 ? d->n_groups : 1;
  const int64_t Kp = pad8(d->in_dim), Np = pad8(d->out_dim);
  gmi_linear l = {};
  l.device = g->device;
  l.d = *d;
  l.x_plane = gmi::align_up(Kp * 2 * d->max_rows, 256);
  l.w_plane = gmi::align_up(Kp * 2 * groups * d->out_dim, 256);
  l.dz_plane = gmi::align_up(Np * 2 * d->max_rows, 256);
  // most row tiles of the slope: those of the finest division that is used, whatever n_rows
  const int64_t tiles = std::min<int64_t>((d->max_rows + kSlopeRows - 1) / kSlopeRows, std::max<int64_t>(4 * g->device_cus, d->max_rows / kSlopeRowsMost + 1)) + groups - 1;
  const int64_t x_b = planes * l.x_plane, w_b = planes * l.w_plane, z_b = d->backward ? planes * l.dz_plane : 0;
  const int64_t b_b = d->backward ? gmi::align_up(tiles * Np * 4, 256) : 0;
  // the outputs that may be divided: of up to max_rows rows, of the weights
  const int64_t most = std::max<int64_t>(std::max((int64_t)d->max_rows * Np, d->backward ? (int64_t)d->max_rows * Kp : 0),
                                         d->backward ? groups * d->out_dim * Kp : 0) * 4;
  l.part_bytes = gmi::align_up(std::min(kPartBytes, most * kMostSplits), 256);
  const int64_t bytes = x_b + w_b + z_b + b_b + l.part_bytes;
  int cur = -1;
  GMI_HIP(hipGetDevice(&cur));
  if (cur != g->device) GMI_HIP(hipSetDevice(g->device));
  const hipError_t e = hipMalloc((void**)&l.base, (size_t)bytes);
  if (cur != g->device) (void)hipSetDevice(cur);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    GMI_FAIL(GMI_ERR_HIP, "gmi_linear_bind: hipMalloc(%lld) failed: %s", (long long)bytes, hipGetErrorString(e));
  }
  l.part = (float*)l.base;
  l.x = l.base + l.part_bytes;
  l.w = l.x + x_b;
  l.dz = l.w + w_b;
  l.bias_part = (float*)(l.dz + z_b);
  l.magic = gmi::kMagicLinear;
  gmi_linear* made = new (std::nothrow) gmi_linear(l);
  if (!made) {
    (void)hipFree(l.base);
    GMI_FAIL(GMI_ERR_HIP, "gmi_linear_bind: out of host memory");
  }
  *out = made;
  return GMI_OK;
}

extern "C" int gmi_linear_destroy(gmi_linear_t l) {
  if (!valid(l)) GMI_FAIL(GMI_ERR_BAD_HANDLE, "gmi_linear_destroy: bad handle");
  (void)hipFree(l->base);
  l->magic = 0;
  delete l;
  return GMI_OK;
}

extern "C" int linear_forward(gmi_t g, gmi_linear_t l, const void* x, int64_t ldx, const void* w, const float* bias, const void* residual,
                              int64_t ldr, int32_t n_rows, void* y, int64_t ldy, void* pre, int64_t ldp) {
  return forward_call("linear_forward", false, g, l, x, ldx, nullptr, w, bias, residual, ldr, n_rows, y, ldy, pre, ldp);
}
extern "C" int grouped_linear_forward(gmi_t g, gmi_linear_t l, const void* x, int64_t ldx, const int32_t* offsets, const void* w,
                                      const float* bias, const void* residual, int64_t ldr, int32_t n_rows, void* y, int64_t ldy,
                                      void* pre, int64_t ldp) {
  return forward_call("grouped_linear_forward", true, g, l, x, ldx, offsets, w, bias, residual, ldr, n_rows, y, ldy, pre, ldp);
}
extern "C" int linear_backward(gmi_t g, gmi_linear_t l, const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w,
                               const void* pre, int64_t ldp, int32_t n_rows, void* dx, int64_t lddx, void* dw, float* dbias) {
  return backward_call("linear_backward", false, g, l, dy, lddy, x, ldx, nullptr, w, pre, ldp, n_rows, dx, lddx, dw, dbias);
}
extern "C" int grouped_linear_backward(gmi_t g, gmi_linear_t l, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                       const int32_t* offsets, const void* w, const void* pre, int64_t ldp, int32_t n_rows, void* dx,
                                       int64_t lddx, void* dw, float* dbias) {
  return backward_call("grouped_linear_backward", true, g, l, dy, lddy, x, ldx, offsets, w, pre, ldp, n_rows, dx, lddx, dw, dbias);
}
