// The orthogonalised update of weight matrices: X <- a X + (b S + c S^2) X with S = X X^T, on fp16 planes and matrix cores.
//
// Every matrix is held with its shorter side p as rows (X [p, q], transposed on the way in and out if it is taller than wide), so that
// each step is three products, batched over all bound matrices: S = X X^T and B = t (a I + b t^2 S + c t^4 S^2), both symmetric (tiles on
// and below the diagonal are computed and mirrored), then X <- B X.  The a X term rides on B's diagonal, so the last product needs no
// epilogue operand.  X starts as G 2^-e with |X| in 1/2 .. 1, e from |G| alone; what is left of 1 / (|G| + eps) is the factor t (in 1 .. 2 unless eps
// counts) that the first step's B carries.  Where t is so small that it would leave nothing of X in fp16, it goes into X step by step: carry_of.
// A bf16 gradient is held exactly by one plane of 11 bits (down to 2^-26 of the norm).  muon_update's direction u is fp32 and is rounded to those
// 11 bits, once, with bf16 gradients: 2^-12 of it, beside the 2^-9 that the gradient itself was rounded to.
//
// Powers of two keep the fp16 values away from the ends of the type: entries of X and S reach 1 and may be as small as 1 / sqrt(p q).  What the coefficients
// can make of singular values in 0 .. 1 bounds X, S and B in every step, and where a bound is larger the power is smaller: scales_of.
#include <cmath>
#include <numeric>

#include "product.h"

using namespace gmi::product;

namespace gmi {
constexpr uint32_t kMagicMuon = 0x474d4955;
}

namespace {

constexpr int kScaleX = 12, kScaleS = 10, kScaleB = 10;      // exponents of the stored X, S, B; smaller where these may leave fp16
constexpr int kMostSteps = 64;
struct Scales { int x, s, b; };      // of a step: of the X that it reads, of S, of B
constexpr int kNormChunk = 2048, kMostChunks = 512;          // elements whose squares a workgroup sums at a time; workgroups of a matrix

constexpr int kSides[4] = {256, 192, 128, 64};
constexpr int side_of(int t) { return t == 256 ? 0 : t == 192 ? 1 : t == 128 ? 2 : 3; }

struct Entry {
  int rows, cols, p, q, qp, pp;            // qp, pp: q, p rounded up to 8
  int64_t offset;                          // in the flat vectors
  int64_t x[2], s, b;                      // bytes in the workspace; planes follow each other
  int64_t x_plane, s_plane;                // bytes
  int chunks, first_chunk, chunk;          // workgroups that sum squares, `chunk` elements each
  int first_pack;                          // 64 x 64 tiles of X (columns to qp)
  int first_tri[4], first_out[4];          // tiles of kSides: of the symmetric products, of the last one
};

}  // namespace

// A launch of one of a step's products: matrices e0 .. e1 - 1 with tile `shape` of kMuonTiles, `blocks` tiles from `first` of the running count on.
// splits: of the contraction (X X^T of few tiles), joined by another launch.
struct Part { int shape, splits, e0, e1, first, blocks; };

struct gmi_muon {
  uint32_t magic;
  int device, dtype, n;
  char* base;
  Entry* table;             // device
  double* sums;             // [chunks]
  float* factor;            // [n] t: 1 / (|G| + eps) is t 2^-e
  float* part;
  std::vector<Entry> host;
  int64_t length;           // the flat vectors reach at least here
  int chunks, packs, tri[4], out[4];
  std::vector<Part> parts[3];      // of X X^T, of S S, of B X
};

namespace {

inline bool valid(gmi_muon_t m) { return m && m->magic == gmi::kMagicMuon; }

struct MuonArgs {
  const Entry* table;
  int n;
  char* base;
  double* sums;
  float* factor;
  const void* src;                 // gradients (or what is orthogonalised)
  const float *moments, *params;   // NULL: no update
  float *moments_out, *params_out;
  void* dst;
  float momentum, a, b, c, eps, lr, decay;
  int nesterov, step, last, from, to;       // of a step: X[from] -> X[to]
  Scales scale;                             // of the step
  int scale_to;                             // of the X that it writes
  int tile0, splits;                        // of the launch: place of its first tile in the running count
  float* part;                              // sums of splits, 64 x 64 of each workgroup
  Entry only;                               // the table's first
};

// The matrix that a step starts from is X = at Y, Y being what the planes hold, and the step's B carries the factor `with`: Y <- with (a I + b at^2 S +
// c at^4 S^2) Y.  In step 0 at = t.  A t of at least 1 goes into Y at once, and so does one that then leaves Y no smaller than it was; otherwise Y
// keeps its size (with = 1 / the most that a step lengthens X by where |X| <= at) and the growth goes to `at`.
struct Carry { float at, with; };
__device__ __forceinline__ Carry carry_of(const MuonArgs& a, float t, int step) {
  Carry c = {t, t};
  for (int k = 0; c.at < 1.f; ++k) {
    const float s = c.at * c.at, most = fmaxf(1.f, fabsf(a.a) + s * (fabsf(a.b) + s * fabsf(a.c)));
    const bool all = c.at * most >= 1.f;
    c.with = all ? c.at : 1.f / most;
    if (k == step) return c;
    if (all) break;
    c.at *= most;
  }
  return step == 0 ? c : Carry{1.f, 1.f};
}

// The entry that holds place `i` of a running count, `first`: where an entry begins in it.  Every kernel's caches start empty, and a step has
// three launches of a few us each: a table in memory costs two trips one after the other before the first operand is asked for, so the
// entry of a single matrix comes with the launch's arguments (1024x4096 230 -> 219 us; eight that way, 1.2 KB of arguments a launch, took 20 us
// longer than the table).
template <class F>
__device__ __forceinline__ Entry entry_of(const MuonArgs& a, int i, int* index, F&& first) {
  *index = 0;
  if (a.n == 1)
    return *(const Entry*)((const char __attribute__((address_space(4)))*)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(MuonArgs, only));
  const int lane = threadIdx.x & 63;
  int found = 0;
  for (int e0 = 0; e0 < a.n; e0 += 64) {
    const uint64_t b = __ballot(e0 + lane < a.n && first(a.table[min(e0 + lane, a.n - 1)]) <= i);
    if (!b) break;
    found = e0 + 63 - __builtin_clzll(b);
  }
  *index = __builtin_amdgcn_readfirstlane(found);
  return a.table[*index];
}

// Eight values of what is orthogonalised (n exist, the others 0): the source, or the momentum step's direction from the new momentum.
template <bool F32>
__device__ __forceinline__ void direction8(const MuonArgs& a, int64_t at, int n, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = 0.f;
  if (n <= 0) return;
  if (!a.moments || a.nesterov) load8<F32>(a.src, at, n, v);
  if (a.moments) {
    float m[8];
    load8<true>(a.moments_out, at, n, m);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = a.nesterov ? v[k] + a.momentum * m[k] : m[k];
  }
}

// In 64 bits: squares of values up to the type's largest stay finite.
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0] + lds[1] + lds[2] + lds[3];
  __syncthreads();
  return v;
}

// New momentum m' = mu m + g, and the sum of squares of a chunk: eight elements a thread at a time.  Bound by memory: 4096 x 4096, 4096 x 1024 and
// 1000 x 2047 in bf16 (46 MB) 13.5 us; 5 us, the launch, for what an L2 holds.
template <bool F32>
__global__ __launch_bounds__(256) void muon_norm_kernel(MuonArgs a) {
  __shared__ double lds[4];
  int e;
  const Entry E = entry_of(a, blockIdx.x, &e, [](const auto& x) { return x.first_chunk; });
  const int64_t count = (int64_t)E.rows * E.cols, begin = (int64_t)(blockIdx.x - E.first_chunk) * E.chunk;
  const int len = (int)min((int64_t)E.chunk, count - begin);
  double sum = 0.0;
#pragma unroll 2
  for (int i = 8 * threadIdx.x; i < len; i += kNormChunk) {
    const int64_t at = E.offset + begin + i;
    const int n = len - i;
    float u[8];
    load8<F32>(a.src, at, n, u);
    if (a.moments) {
      float m[8];
      load8<true>(a.moments, at, n, m);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        m[k] = a.momentum * m[k] + u[k];
        u[k] = k < n ? (a.nesterov ? u[k] + a.momentum * m[k] : m[k]) : 0.f;
      }
      store8<true>(a.moments_out, at, n, m);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += (double)u[k] * u[k];
  }
  sum = block_sum(sum, lds);
  if (threadIdx.x == 0) a.sums[blockIdx.x] = sum;
}

// Zeros past the first n of eight: the next product's contraction runs over the padded width.
__device__ __forceinline__ void clear_past(float (&v)[8], int n) {
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = k < n ? v[k] : 0.f;
}
template <int PLANES>
__device__ __forceinline__ void store_half(char* base, int64_t at, int64_t plane, const float (&v)[8]) {
  uint32_t w[PLANES][4];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const _Float16 h = (_Float16)v[e];
    const uint32_t hb = __builtin_bit_cast(uint16_t, h);
    w[0][e >> 1] = e & 1 ? w[0][e >> 1] | hb << 16 : hb;
    if constexpr (PLANES > 1) {
      const _Float16 l = (_Float16)(v[e] - (float)h);
      const uint32_t lb = __builtin_bit_cast(uint16_t, l);
      w[1][e >> 1] = e & 1 ? w[1][e >> 1] | lb << 16 : lb;
    }
  }
#pragma unroll
  for (int i = 0; i < PLANES; ++i) *(uint4*)(base + i * plane + at * 2) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
}

// X = G 2^-e 2^kScaleX in planes, [p, qp], a 64 x 64 tile a workgroup, transposed through LDS for the tall.  Bound by memory: the same three
// matrices (92 MB) 23 us, 1024 x 4096 6.9.
template <bool F32>
__global__ __launch_bounds__(256) void muon_pack_kernel(MuonArgs a) {
  __shared__ double lds[4];
  __shared__ float tile[64][65];
  int e;
  const Entry E = entry_of(a, blockIdx.x, &e, [](const auto& x) { return x.first_pack; });
  const int local = blockIdx.x - E.first_pack;
  const int across = (E.qp + 63) >> 6, p0 = local / across * 64, q0 = local % across * 64;
  const bool tall = E.rows > E.cols;
  const int np = min(64, E.p - p0), nq = min(64, E.q - q0);
  // values on their way while the norm is formed: eight of a row twice, or the tile by columns
  float u[16];
  const int r8 = threadIdx.x >> 3, c8 = (threadIdx.x & 7) * 8;
  if (!tall) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int n = r8 + 32 * k < np ? nq - c8 : 0;
      direction8<F32>(a, E.offset + (int64_t)(p0 + r8 + 32 * k) * E.cols + q0 + c8, n, (float (&)[8])u[8 * k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int n = r8 + 32 * k < nq ? np - c8 : 0;
      direction8<F32>(a, E.offset + (int64_t)(q0 + r8 + 32 * k) * E.cols + p0 + c8, n, (float (&)[8])u[8 * k]);
    }
  }
  double sum = 0.0;
  for (int i = threadIdx.x; i < E.chunks; i += 256) sum += a.sums[E.first_chunk + i];
  const double norm = sqrt(block_sum(sum, lds));      // of finite values finite
  int ex;
  (void)frexp(norm, &ex);
  if (!(norm > 0.0 && norm < INFINITY)) ex = 0;
  if (local == 0 && threadIdx.x == 0) a.factor[e] = !(norm < INFINITY) ? NAN : norm > 0.0 ? (float)(ldexp(1.0, ex) / (norm + a.eps)) : 1.f;
#pragma unroll
  for (int k = 0; k < 16; ++k) u[k] = ldexpf(u[k], kScaleX - ex);
  constexpr int PLANES = F32 ? 2 : 1;
  if (!tall) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (r8 + 32 * k < np && q0 + c8 < E.qp)
        store_half<PLANES>(a.base + E.x[0], (int64_t)(p0 + r8 + 32 * k) * E.qp + q0 + c8, E.x_plane, (const float (&)[8])u[8 * k]);
    return;
  }
#pragma unroll
  for (int k = 0; k < 16; ++k) tile[c8 + (k & 7)][r8 + 32 * (k >> 3)] = u[k];
  __syncthreads();
  for (int i = threadIdx.x; i < 512; i += 256) {
    const int r = i >> 3, c = (i & 7) * 8;
    if (r >= np || q0 + c >= E.qp) continue;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = tile[r][c + k];
    store_half<PLANES>(a.base + E.x[0], (int64_t)(p0 + r) * E.qp + q0 + c, E.x_plane, v);
  }
}

// Tile `id` of the running count of triangles: its matrix and place.
struct TriangleTile { Entry E; int e, m0, n0; };
template <int T>
__device__ __forceinline__ TriangleTile triangle_tile(const MuonArgs& a, int id) {
  constexpr int shape = side_of(T);
  int e;
  const Entry E = entry_of(a, id, &e, [](const auto& x) { return x.first_tri[shape]; });
  const int np = (E.p + T - 1) / T, i = by_die(id - E.first_tri[shape], np * (np + 1) / 2);      // each matrix over all dies
  // tile i of the triangle, row by row: row r has r + 1
  int r = (int)((sqrtf(8.f * i + 1.f) - 1.f) * 0.5f);
  if ((r + 1) * (r + 2) / 2 <= i) ++r;
  if (r * (r + 1) / 2 > i) --r;
  r = __builtin_amdgcn_readfirstlane(r);
  return {E, e, r * T, (i - r * (r + 1) / 2) * T};
}

struct Halves { f16x8 h, l; };
// The two symmetric products.  SQUARE false: S = X X^T; true: B from S S.  Half the work, but as few tiles again: 4096 x 4096 76 and 82 us
// (0.9 PFLOP/s of what is computed; whole, with Large, each would be 116), bound by the matrix cores with one round of workgroups.  1024 x
// 4096 has 136 tiles of 64 with a contraction of 4096: 17.4 us, bound by the address units (64 bytes a cycle and compute unit); eight small fp32
// matrices 11.3 and 12.5, half of it the launch and the first reads.
template <class S, bool F32, bool SQUARE>
__global__ __launch_bounds__(S::threads, kWavesPerSimd<S>) void muon_symmetric_kernel(MuonArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  constexpr int T = S::TM, PLANES = F32 ? 2 : 1;
  constexpr bool divided = !SQUARE && S::TM == Small::TM;      // may be
  const int splits = divided ? a.splits : 1;
  const TriangleTile tile = triangle_tile<T>(a, a.tile0 + blockIdx.x / splits);
  const int e = tile.e, m0 = tile.m0, n0 = tile.n0;
  const Entry& E = tile.E;
  Side P, Q;
  const char* in = a.base + (SQUARE ? E.s : (a.from ? E.x[1] : E.x[0]));
  P.ld = Q.ld = 2 * (int64_t)(SQUARE ? E.pp : E.qp);
  P.plane = Q.plane = SQUARE ? E.s_plane : E.x_plane;
  P.base = in + n0 * P.ld; P.count = min(T, E.p - n0);
  Q.base = in + m0 * Q.ld; Q.count = min(T, E.p - m0);
  int k_len = SQUARE ? E.pp : E.qp;
  if (divided && splits > 1) {
    const int chunk = ((k_len + splits - 1) / splits + kDepth - 1) & ~(kDepth - 1), k0 = min(k_len, (int)(blockIdx.x % splits) * chunk);
    k_len = min(k_len, k0 + chunk) - k0;
    P.base += k0 * 2;
    Q.base += k0 * 2;
  }
  const float t0 = SQUARE ? a.factor[e] : 1.f;      // asked for here, so that it is there at the end
  Accumulator<S> acc;
  multiply<S, false, false, true>(P, Q, k_len, F32 ? kTwoPlanes : kOnePlane, smem, acc);
  if (divided && splits > 1) {
    float* to = a.part + (int64_t)blockIdx.x * (T * T);
    each_row<S>(acc, smem, FetchNothing(), [&](int m, int n, float (&v)[8], Nothing) { store8<true>(to, m * T + n, 8, v); });
    return;
  }

  const Carry t = SQUARE ? carry_of(a, t0, a.step) : Carry{1.f, 1.f};
  const float ta = t.with * a.a * ldexpf(1.f, a.scale.b), tb = t.with * t.at * t.at * a.b * ldexpf(1.f, a.scale.b - a.scale.s),
              tc = t.with * t.at * t.at * t.at * t.at * a.c * ldexpf(1.f, a.scale.b - 2 * a.scale.s), ts = ldexpf(1.f, a.scale.s - 2 * a.scale.x);
  const char* s = a.base + E.s;
  char* out = a.base + (SQUARE ? E.b : E.s);
  // eight values of row m at columns n ..: S there, and what is made of the sums v
  auto symmetric = [&](int m, int n) {
    Halves x = {};
    if (SQUARE && m < E.p && n < E.pp) {
      x.h = *(const f16x8*)(s + ((int64_t)m * E.pp + n) * 2);
      if constexpr (PLANES > 1) x.l = *(const f16x8*)(s + E.s_plane + ((int64_t)m * E.pp + n) * 2);
    }
    return x;
  };
  auto put = [&](int m, int n, float (&v)[8], const Halves& x) {
    if (m >= E.p || n >= E.pp) return;
    if constexpr (SQUARE) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = tc * v[k] + tb * ((float)x.h[k] + (PLANES > 1 ? (float)x.l[k] : 0.f)) + (m == n + k ? ta : 0.f);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= ts;
    }
    clear_past(v, E.p - n);
    store_half<PLANES>(out, (int64_t)m * E.pp + n, E.s_plane, v);
  };
  each_row<S>(acc, smem, [&](int m, int n) { return symmetric(m0 + m, n0 + n); },
              [&](int m, int n, float (&v)[8], const Halves& x) { put(m0 + m, n0 + n, v, x); });
  if (m0 != n0)
    each_column<true, S>(acc, smem, [&](int n, int m) { return symmetric(n0 + n, m0 + m); },
                         [&](int n, int m, float (&v)[8], const Halves& x) { put(n0 + n, m0 + m, v, x); });
}

// S from the sums of the splits of its tiles in their order, one 64 x 64 tile a workgroup: a few us, bound by the launch.
template <bool F32>
__global__ __launch_bounds__(256) void muon_join_kernel(MuonArgs a) {
  constexpr int T = Small::TM, PLANES = F32 ? 2 : 1;
  __shared__ float sums[T][T + 1];
  const TriangleTile tile = triangle_tile<T>(a, a.tile0 + blockIdx.x);
  const Entry& E = tile.E;
  const float ts = ldexpf(1.f, a.scale.s - 2 * a.scale.x);
  char* out = a.base + E.s;
  const float* from = a.part + (int64_t)blockIdx.x * a.splits * (T * T);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int r = threadIdx.x / 8 + 32 * k, c = threadIdx.x % 8 * 8;
    float v[8] = {};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
      float u[8];
      load8<true>(from, s * (T * T) + r * T + c, 8, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += u[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[r][c + i] = v[i] *= ts;
    clear_past(v, E.p - tile.n0 - c);
    if (tile.m0 + r < E.p && tile.n0 + c < E.pp) store_half<PLANES>(out, (int64_t)(tile.m0 + r) * E.pp + tile.n0 + c, E.s_plane, v);
  }
  if (tile.m0 == tile.n0) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int r = threadIdx.x / 8 + 32 * k, c = threadIdx.x % 8 * 8;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = sums[c + i][r];
    clear_past(v, E.p - tile.m0 - c);
    if (tile.n0 + r < E.p && tile.m0 + c < E.pp) store_half<PLANES>(out, (int64_t)(tile.n0 + r) * E.pp + tile.m0 + c, E.s_plane, v);
  }
}

// X <- B X, or, in the last step, what is done with it.  B is symmetric and lies with its contraction contiguous, X's rows are the contraction:
// read as they lie, transposed by the LDS read.  4096 x 4096 116 us (1.18 PFLOP/s), 1024 x 4096 15 with 256 Medium tiles.
template <class S, bool F32>
__global__ __launch_bounds__(S::threads, kWavesPerSimd<S>) void muon_apply_kernel(MuonArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  constexpr int T = S::TM, shape = side_of(T), PLANES = F32 ? 2 : 1;
  const int id = a.tile0 + blockIdx.x;
  int e;
  const Entry E = entry_of(a, id, &e, [](const auto& x) { return x.first_out[shape]; });
  const int np = (E.p + T - 1) / T, nq = (E.q + T - 1) / T;
  int mt, nt;
  tile_of(by_die(id - E.first_out[shape], np * nq), np, nq, &mt, &nt);
  const int m0 = mt * T, n0 = nt * T;
  Side P, Q;
  P.ld = 2 * (int64_t)E.qp; P.plane = E.x_plane; P.base = a.base + (a.from ? E.x[1] : E.x[0]) + n0 * 2; P.count = min(T, E.q - n0);
  Q.ld = 2 * (int64_t)E.pp; Q.plane = E.s_plane; Q.base = a.base + E.b + m0 * Q.ld; Q.count = min(T, E.p - m0);
  const float t0 = a.last ? a.factor[e] : 1.f;
  Accumulator<S> acc;
  multiply<S, true, false, true>(P, Q, E.p, F32 ? kTwoPlanes : kOnePlane, smem, acc);

  if (!a.last) {
    const float scale = ldexpf(1.f, a.scale_to - a.scale.x - a.scale.b);
    each_row<S>(acc, smem, FetchNothing(), [&](int m, int n, float (&v)[8], Nothing) {
      if (m0 + m >= E.p || n0 + n >= E.qp) return;
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= scale;
      clear_past(v, E.q - n0 - n);
      store_half<PLANES>(a.base + (a.to ? E.x[1] : E.x[0]), (int64_t)(m0 + m) * E.qp + n0 + n, E.x_plane, v);
    });
    return;
  }
  const float scale = carry_of(a, t0, a.step + 1).at * ldexpf(1.f, -a.scale.b - a.scale.x);
  const float step = a.lr * sqrtf(fmaxf(1.f, (float)E.rows / (float)E.cols));
  // eight values of row r of the matrix at columns c ..: its parameters, and what is made of the sums v
  auto weights = [&](int r, int c) {
    Eight<true> w = {};
    if (a.params && r < E.rows) w.fetch(a.params, E.offset + (int64_t)r * E.cols + c, E.cols - c);
    return w;
  };
  auto put = [&](int r, int c, float (&v)[8], const Eight<true>& w) {
    const int n = E.cols - c;
    if (r >= E.rows || n <= 0) return;
    const int64_t at = E.offset + (int64_t)r * E.cols + c;
    if (a.params) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = a.decay * w.value(k) - step * (v[k] * scale);
      store8<true>(a.params_out, at, n, v);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= scale;
      store8<F32>(a.dst, at, n, v);
    }
  };
  if (E.rows <= E.cols)
    each_row<S>(acc, smem, [&](int m, int n) { return weights(m0 + m, n0 + n); },
                [&](int m, int n, float (&v)[8], const Eight<true>& w) { put(m0 + m, n0 + n, v, w); });
  else
    each_column<false, S>(acc, smem, [&](int n, int m) { return weights(n0 + n, m0 + m); },
                          [&](int n, int m, float (&v)[8], const Eight<true>& w) { put(n0 + n, m0 + m, v, w); });
}

// ------------------------------------------------------------------ host
template <class S>
int launch_part(gmi_instance* g, const MuonArgs& a, void (*kernel)(MuonArgs), const Part& part, gmi::DeviceSet* allowed) {
  const int rc = gmi::allow_lds((const void*)kernel, S::lds, g->device, allowed);
  if (rc != GMI_OK) return rc;
  kernel<<<dim3((unsigned)(part.blocks * part.splits)), S::threads, S::lds, g->stream>>>(a);
  GMI_LAUNCH_CHECK();
  return GMI_OK;
}
template <class S, bool F32>
int run_part(gmi_instance* g, const MuonArgs& a, int product, const Part& part) {
  static gmi::DeviceSet allowed[3];
  if (product == 0) return launch_part<S>(g, a, muon_symmetric_kernel<S, F32, false>, part, &allowed[0]);
  if (product == 1) return launch_part<S>(g, a, muon_symmetric_kernel<S, F32, true>, part, &allowed[1]);
  if constexpr (S::TM != Middle::TM) return launch_part<S>(g, a, muon_apply_kernel<S, F32>, part, &allowed[2]);
  else return GMI_ERR_UNSUPPORTED;
}

// The tiles to choose from.  Middle, for the symmetric products only, is there for triangles that fill the chip once with it and half with
// Large: 4096 x 4096 has 253 of its tiles, 136 of Large's, 528 of Medium's (five steps 1340 us; 1585; 1730).
constexpr Tile kMuonTiles[5] = {kTiles[0], kTiles[1], kTiles[2], kTiles[3], kTiles[6]};

// A division of X X^T costs another launch and the sums' way out and in.
constexpr float kMuonJoin = 1.5f, kMuonJoinTile = 64.f * 64.f * 4.f * 2.f / 4e6f;
constexpr int kMostSplitTiles = 2048;      // workgroups of a divided launch

// Launches of a product: the first matrices (the longest contractions) with one tile and the others with another, or all with one; X X^T of
// few tiles divided along the contraction (17 x 3568 fp32 is one tile: 240 us for five steps undivided).
void plan_parts(gmi_muon* m, int product, int cus) {
  const int n = m->n;
  struct Option { int shape, splits; std::vector<float> head, tail; };      // us of matrices 0 .. k - 1, of k .. n - 1
  std::vector<Option> options;
  for (int i = 0; i < (product == 2 ? 4 : 5); ++i) options.push_back({i, 1, {}, {}});
  if (product == 0)
    for (int s = 2; s <= 64; s *= 2) options.push_back({2, s, {}, {}});
  std::vector<float> one(n), sum(n + 1), tiles(n + 1), longest_to(n + 1), longest_from(n + 2);
  for (Option& o : options) {
    const Tile& tile = kMuonTiles[o.shape];
    sum[0] = tiles[0] = longest_to[0] = longest_from[n] = 0.f;
    for (int k = 0; k < n; ++k) {
      const Entry& e = m->host[k];
      const int64_t np = (e.p + tile.size[0] - 1) / tile.size[0], nq = (e.q + tile.size[0] - 1) / tile.size[0];
      const float count = (float)(product == 2 ? np * nq : np * (np + 1) / 2) * o.splits;
      one[k] = tile_time(tile, (float)((product == 0 ? e.q : e.p) * (m->dtype == GMI_DTYPE_F32 ? kTwoPlanes.n : 1)) / o.splits);
      tiles[k + 1] = tiles[k] + count;
      sum[k + 1] = sum[k] + count * one[k];
      longest_to[k + 1] = std::max(longest_to[k], one[k]);
    }
    for (int k = n; k-- > 0;) longest_from[k] = std::max(longest_from[k + 1], one[k]);
    auto time = [&](float s, float longest, float count) {
      if (s <= 0.f) return 0.f;
      if (o.splits > 1 && count > kMostSplitTiles) return 1e30f;
      longest *= s > longest * cus ? tile.share : tile.alone;
      // beyond a full round the last workgroups run beside idle units
      return kStart + std::max(longest, s / cus + (s > longest * cus / tile.share ? 0.5f * longest : 0.f)) +
             (o.splits > 1 ? kStart + kMuonJoin + count * kMuonJoinTile : 0.f);
    };
    for (int k = 0; k <= n; ++k) {
      o.head.push_back(time(sum[k], longest_to[k], tiles[k]));
      o.tail.push_back(time(sum[n] - sum[k], longest_from[k], tiles[n] - tiles[k]));
    }
  }
  float least = 1e30f;
  int cut = n;
  const Option *first = &options[0], *second = first;
  for (const Option& i : options)
    for (const Option& j : options)
      for (int k = 1; k <= n; ++k) {
        if (&i == &j && k < n) continue;
        const float t = i.head[k] + j.tail[k];
        if (t < least) { least = t; cut = k; first = &i; second = &j; }
      }
  auto add = [&](const Option& o, int e0, int e1) {
    if (e0 == e1) return;
    const int side = side_of(kMuonTiles[o.shape].size[0]);
    auto at = [&](int e) { return product == 2 ? (e < n ? m->host[e].first_out[side] : m->out[side]) : (e < n ? m->host[e].first_tri[side] : m->tri[side]); };
    m->parts[product].push_back({o.shape, o.splits, e0, e1, at(e0), at(e1) - at(e0)});
  };
  add(*first, 0, cut);
  add(*second, cut, n);
}

// The scales of `steps` steps; false if X X^T or B may pass 2^20, which the planes' 2^15 and what small entries need of their other end are not made for.
// A singular value in 0 .. most becomes v |p(v^2)| with p(s) = a + b s + c s^2 (that of X, not of the Y that carry_of speaks of, which is smaller), 1/256 of
// it is left for roundings (2^-11 each at the most), a factor of 2 to fp16's largest.
bool scales_of(const gmi_muon_hparams& hp, Scales (&out)[kMostSteps]) {
  const double a = hp.a, b = hp.b, c = hp.c;
  if (!(std::isfinite(a) && std::isfinite(b) && std::isfinite(c))) return false;
  auto p = [&](double s) { return std::fabs(a + s * (b + s * c)); };
  auto exponent = [](int most, double bound) {
    while (std::ldexp(bound, most) > 32768.0) --most;
    return most;
  };
  double most = 1.0;
  for (int k = 0; k < hp.steps; ++k) {
    const double s = most * most;
    double of_b = std::max(p(0.0), p(s)), next = most * p(s);
    if (c != 0.0 && -b / (2.0 * c) > 0.0 && -b / (2.0 * c) < s) of_b = std::max(of_b, p(-b / (2.0 * c)));
    // where v p(v^2) is flat: a + 3 b s + 5 c s^2 = 0
    const double root = 9.0 * b * b - 20.0 * a * c, q = -0.5 * (3.0 * b + std::copysign(std::sqrt(std::max(root, 0.0)), b));
    for (const double at : {c != 0.0 ? q / (5.0 * c) : -1.0, q != 0.0 ? a / q : -1.0})
      if (root >= 0.0 && at > 0.0 && at < s) next = std::max(next, std::sqrt(at) * p(at));
    if (k == 0) of_b *= 2.0;      // the factor t of the first step
    if (!(s <= 1048576.0 && of_b <= 1048576.0)) return false;
    out[k] = {exponent(kScaleX, most), exponent(kScaleS, s), exponent(kScaleB, of_b)};
    most = std::max(most, next * (1.0 + 1.0 / 256));
  }
  return true;
}

template <bool F32>
int run(gmi_instance* g, const gmi_muon* m, MuonArgs a, const char* who, const gmi_muon_hparams& hp) {
  const int steps = hp.steps;
  Scales scales[kMostSteps];
  if (!scales_of(hp, scales)) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: coefficients %g, %g, %g may lengthen a matrix beyond what %d steps hold", who, hp.a, hp.b, hp.c, steps);
  muon_norm_kernel<F32><<<m->chunks, 256, 0, g->stream>>>(a);
  GMI_LAUNCH_CHECK();
  muon_pack_kernel<F32><<<m->packs, 256, 0, g->stream>>>(a);
  GMI_LAUNCH_CHECK();
  for (int s = 0; s < steps; ++s) {
    a.step = s;
    a.last = s == steps - 1;
    a.from = s & 1;
    a.to = 1 - a.from;
    a.scale = scales[s];
    a.scale_to = a.last ? 0 : scales[s + 1].x;
    for (int product = 0; product < 3; ++product)
      for (const Part& part : m->parts[product]) {
        a.tile0 = part.first;
        a.splits = part.splits;
        const int rc = part.shape == 0   ? run_part<Large, F32>(g, a, product, part)
                       : part.shape == 1 ? run_part<Medium, F32>(g, a, product, part)
                       : part.shape == 2 ? run_part<Small, F32>(g, a, product, part)
                       : part.shape == 3 ? run_part<Twin, F32>(g, a, product, part) : run_part<Middle, F32>(g, a, product, part);
        if (rc != GMI_OK) return rc;
        if (part.splits > 1) {
          muon_join_kernel<F32><<<part.blocks, 256, 0, g->stream>>>(a);
          GMI_LAUNCH_CHECK();
        }
      }
  }
  return GMI_OK;
}

int check_muon(const char* who, gmi_t g, gmi_muon_t m, const gmi_muon_hparams* hp) {
  if (!valid(g)) GMI_FAIL(GMI_ERR_BAD_HANDLE, "%s: bad instance", who);
  if (!valid(m)) GMI_FAIL(GMI_ERR_BAD_HANDLE, "%s: bad binding", who);
  if (g->device != m->device) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: instance and binding live on different devices", who);
  if (!hp) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: hp is NULL", who);
  if (hp->steps < 1 || hp->steps > kMostSteps) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: steps %d outside 1 .. %d", who, hp->steps, kMostSteps);
  if (!(hp->eps > 0.f)) GMI_FAIL(GMI_ERR_INVALID_ARG, "%s: eps has to be positive", who);
  return GMI_OK;
}

MuonArgs args_of(const gmi_muon* m, const gmi_muon_hparams* hp) {
  MuonArgs a = {};
  a.table = m->table; a.n = m->n; a.base = m->base; a.sums = m->sums; a.factor = m->factor; a.part = m->part;
  a.momentum = hp->momentum; a.a = hp->a; a.b = hp->b; a.c = hp->c; a.eps = hp->eps; a.lr = hp->lr;
  a.decay = 1.f - hp->lr * hp->weight_decay;
  a.nesterov = hp->nesterov;
  a.only = m->host[0];
  return a;
}
bool overlap(const void* x, const void* y, int64_t bx, int64_t by) {
  return (const char*)x < (const char*)y + by && (const char*)y < (const char*)x + bx;
}

}  // namespace

extern "C" int gmi_muon_bind(gmi_t g, const gmi_matrix* matrices, int32_t n, int32_t dtype, gmi_muon_t* out) {
  if (!out) GMI_FAIL(GMI_ERR_INVALID_ARG, "gmi_muon_bind: out is NULL");
  *out = nullptr;
  if (!valid(g)) GMI_FAIL(GMI_ERR_BAD_HANDLE, "gmi_muon_bind: bad instance");
  if (!matrices) GMI_FAIL(GMI_ERR_INVALID_ARG, "gmi_muon_bind: matrices is NULL");
  if (n < 1 || n > 4096) GMI_FAIL(GMI_ERR_BAD_SHAPE, "gmi_muon_bind: %d matrices, outside 1 .. 4096", n);
  if (dtype != GMI_DTYPE_F32 && dtype != GMI_DTYPE_BF16) GMI_FAIL(GMI_ERR_UNSUPPORTED, "gmi_muon_bind: dtype %d", dtype);
  try {
    std::vector<std::pair<int64_t, int64_t>> spans;
    for (int i = 0; i < n; ++i) {
      const gmi_matrix& x = matrices[i];
      if (x.rows < 1 || x.rows > 32768 || x.cols < 1 || x.cols > 32768)
        GMI_FAIL(GMI_ERR_BAD_SHAPE, "gmi_muon_bind: matrix %d is %d x %d, sides outside 1 .. 32768", i, x.rows, x.cols);
      if (x.offset < 0 || x.offset > ((int64_t)1 << 48)) GMI_FAIL(GMI_ERR_BAD_SHAPE, "gmi_muon_bind: offset of matrix %d", i);
      spans.push_back({x.offset, x.offset + (int64_t)x.rows * x.cols});
    }
    std::sort(spans.begin(), spans.end());
    for (int i = 1; i < n; ++i)
      if (spans[i].first < spans[i - 1].second) GMI_FAIL(GMI_ERR_INVALID_ARG, "gmi_muon_bind: matrices overlap");
    std::unique_ptr<gmi_muon> m(new gmi_muon());
    m->device = g->device;
    m->dtype = dtype;
    m->n = n;
    m->length = spans.back().second;
    const int planes = dtype == GMI_DTYPE_F32 ? 2 : 1;
    int64_t bytes = 0, chunks = 0, packs = 0, tri[4] = {}, outs[4] = {};
    auto take = [&](int64_t b) { const int64_t at = bytes; bytes += gmi::align_up(b, 256); return at; };
    // the longest contractions first: their workgroups last longest
    std::vector<int> order(n);
    std::iota(order.begin(), order.end(), 0);
    std::stable_sort(order.begin(), order.end(), [&](int i, int j) {
      const gmi_matrix &x = matrices[i], &y = matrices[j];
      const int xp = std::min(x.rows, x.cols), yp = std::min(y.rows, y.cols);
      return xp != yp ? xp > yp : std::max(x.rows, x.cols) > std::max(y.rows, y.cols);
    });
    for (int i : order) {
      const gmi_matrix& x = matrices[i];
      Entry e = {};
      e.rows = x.rows; e.cols = x.cols; e.offset = x.offset;
      e.p = std::min(x.rows, x.cols); e.q = std::max(x.rows, x.cols);
      e.pp = (e.p + 7) & ~7; e.qp = (e.q + 7) & ~7;
      e.x_plane = gmi::align_up((int64_t)e.p * e.qp * 2, 256);
      e.s_plane = gmi::align_up((int64_t)e.p * e.pp * 2, 256);
      e.x[0] = take(planes * e.x_plane); e.x[1] = take(planes * e.x_plane);
      e.s = take(planes * e.s_plane); e.b = take(planes * e.s_plane);
      const int64_t count = (int64_t)x.rows * x.cols;
      e.first_chunk = (int)chunks;
      const int64_t parts = (count + kNormChunk - 1) / kNormChunk;
      e.chunk = (int)((parts + kMostChunks - 1) / kMostChunks) * kNormChunk;
      e.chunks = (int)((count + e.chunk - 1) / e.chunk);
      chunks += e.chunks;
      e.first_pack = (int)packs;
      packs += (int64_t)((e.p + 63) / 64) * ((e.qp + 63) / 64);
      for (int k = 0; k < 4; ++k) {
        const int64_t np = (e.p + kSides[k] - 1) / kSides[k], nq = (e.q + kSides[k] - 1) / kSides[k];
        e.first_tri[k] = (int)tri[k];
        e.first_out[k] = (int)outs[k];
        tri[k] += np * (np + 1) / 2;
        outs[k] += np * nq;
      }
      if (chunks > (1 << 30) || packs > (1 << 30) || outs[3] > (1 << 30)) GMI_FAIL(GMI_ERR_BAD_SHAPE, "gmi_muon_bind: too many elements");
      m->host.push_back(e);
    }
    m->chunks = (int)chunks;
    m->packs = (int)packs;
    for (int k = 0; k < 4; ++k) { m->tri[k] = (int)tri[k]; m->out[k] = (int)outs[k]; }
    for (int k = 0; k < 3; ++k) plan_parts(m.get(), k, g->cu_count);
    int64_t divided = 0;
    for (const Part& p : m->parts[0])
      if (p.splits > 1) divided = std::max<int64_t>(divided, (int64_t)p.blocks * p.splits);
    const int64_t at_part = take(divided * 64 * 64 * 4);
    const int64_t at_table = take((int64_t)n * sizeof(Entry)), at_sums = take(chunks * 8), at_factor = take((int64_t)n * 4);
    int cur = -1;
    GMI_HIP(hipGetDevice(&cur));
    if (cur != g->device) GMI_HIP(hipSetDevice(g->device));
    hipError_t e = hipMalloc((void**)&m->base, (size_t)bytes);
    if (e == hipSuccess) {
      e = hipMemcpy(m->base + at_table, m->host.data(), (size_t)n * sizeof(Entry), hipMemcpyHostToDevice);
      if (e != hipSuccess) (void)hipFree(m->base);
    }
    if (cur != g->device) (void)hipSetDevice(cur);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      GMI_FAIL(GMI_ERR_HIP, "gmi_muon_bind: %lld bytes of workspace: %s", (long long)bytes, hipGetErrorString(e));
    }
    m->table = (Entry*)(m->base + at_table);
    m->sums = (double*)(m->base + at_sums);
    m->factor = (float*)(m->base + at_factor);
    m->part = (float*)(m->base + at_part);
    m->magic = gmi::kMagicMuon;
    *out = m.release();
    return GMI_OK;
  } catch (const std::exception& ex) {
    GMI_FAIL(GMI_ERR_HIP, "gmi_muon_bind: %s", ex.what());
  }
}

extern "C" int gmi_muon_destroy(gmi_muon_t m) {
  if (!valid(m)) GMI_FAIL(GMI_ERR_BAD_HANDLE, "gmi_muon_destroy: bad handle");
  (void)hipFree(m->base);
  m->magic = 0;
  delete m;
  return GMI_OK;
}

extern "C" int muon_orthogonalize(gmi_t g, gmi_muon_t m, const void* src, void* dst, const gmi_muon_hparams* hp) {
  const int rc = check_muon("muon_orthogonalize", g, m, hp);
  if (rc != GMI_OK) return rc;
  if (!src || !dst) GMI_FAIL(GMI_ERR_INVALID_ARG, "muon_orthogonalize: NULL pointer");
  const int es = m->dtype == GMI_DTYPE_F32 ? 4 : 2;
  if ((uintptr_t)src % es || (uintptr_t)dst % es) GMI_FAIL(GMI_ERR_INVALID_ARG, "muon_orthogonalize: not aligned to elements");
  if (src != dst && overlap(src, dst, m->length * es, m->length * es)) GMI_FAIL(GMI_ERR_INVALID_ARG, "muon_orthogonalize: dst overlaps src");
  MuonArgs a = args_of(m, hp);
  a.src = src;
  a.dst = dst;
  return m->dtype == GMI_DTYPE_F32 ? run<true>(g, m, a, "muon_orthogonalize", *hp) : run<false>(g, m, a, "muon_orthogonalize", *hp);
}

extern "C" int muon_update(gmi_t g, gmi_muon_t m, const float* params, const float* moments, const void* grad, const gmi_muon_hparams* hp,
                           float* params_out, float* moments_out) {
  const int rc = check_muon("muon_update", g, m, hp);
  if (rc != GMI_OK) return rc;
  if (!params || !moments || !grad || !params_out || !moments_out) GMI_FAIL(GMI_ERR_INVALID_ARG, "muon_update: NULL pointer");
  const int es = m->dtype == GMI_DTYPE_F32 ? 4 : 2;
  if (((uintptr_t)params | (uintptr_t)moments | (uintptr_t)params_out | (uintptr_t)moments_out) % 4 || (uintptr_t)grad % es)
    GMI_FAIL(GMI_ERR_INVALID_ARG, "muon_update: not aligned to elements");
  const int64_t len = m->length * 4;
  if ((params_out != params && overlap(params_out, params, len, len)) || overlap(params_out, moments, len, len) ||
      overlap(params_out, grad, len, m->length * es) || overlap(params_out, moments_out, len, len) ||
      (moments_out != moments && overlap(moments_out, moments, len, len)) || overlap(moments_out, params, len, len) ||
      overlap(moments_out, grad, len, m->length * es))
    GMI_FAIL(GMI_ERR_INVALID_ARG, "muon_update: an output overlaps another argument");
  MuonArgs a = args_of(m, hp);
  a.src = grad;
  a.params = params;
  a.moments = moments;
  a.params_out = params_out;
  a.moments_out = moments_out;
  return m->dtype == GMI_DTYPE_F32 ? run<true>(g, m, a, "muon_update", *hp) : run<false>(g, m, a, "muon_update", *hp);
}
