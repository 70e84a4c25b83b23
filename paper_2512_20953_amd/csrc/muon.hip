// Optimizer step of matrices by the orthogonal factor of their momentum (declared in include/ah_ops.h): momentum and its norm, five (ns_steps) times three matrix
// products on the loop of gemm_loop.h, and the step of the parameters.
//
// With X [n, m], n <= m (a matrix of more rows than columns is laid out transposed):
//   A = X X^T                 n^2 m flops: the product is symmetric, so that the tiles on and below the diagonal are computed and each is stored twice
//   B = b A + c A A           n^3: likewise
//   X = a X + B X             2 n^2 m
// or, the first two of the steps at once, 3 n^2 m + 5 n^3 instead of 6 n^2 m + 2 n^3 (see Product).
// Bound by the matrix units from n of about two thousand on, at the clock that their power leaves (1.87 GHz measured; a LLaMA-style layer's matrices, 4096 x 4096 and 4096 x 11008:
// 14.0 ms, of which products 12.2; the loop by itself reaches 1.36 PFLOP/s, a library's product 1.5); below that by how long few k-steps take to arrive.
//
// Types.  The operands are fp16: with everything within 3 in magnitude, or 12 (A and B, and what two steps at once have besides, are polynomials of a matrix whose singular values stay
// below 1.21), its range suffices, and it
// keeps 11 bits where bf16 keeps 8, at the same rate.  X itself goes from product to product in 22 bits, as two fp16 numbers: what is added to a X has to be added to the same X
// that it was computed from, or the rounding of every step is taken for a part of X, which the polynomial multiplies by up to 3.44 a step where singular values are small.  Of a
// matrix with 64 strong directions above a floor of noise (1024 x 2816) the factor is 5e-4 off in norm, with X in fp16 alone 2e-2, in bf16 alone 0.18.  Small matrices of fp32
// parameters have all operands in 22 bits (FINE).  Fixed powers of two keep small
// elements out of fp16's subnormals: kX on X, kA on A and B, kLo more on X's lower half.
#include "ah_ops.h"
#include "capi_util.h"
#include "gemm_loop.h"
#include "wide.h"

#include <algorithm>
#include <cmath>
#include <vector>

using namespace ah;

namespace {

typedef _Float16 f16;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr float kA_ = 3.4445f, kB_ = -4.7750f, kC_ = 2.0315f;            // the polynomial
constexpr float kX = 64.f, kA = 1024.f, kLo = 2048.f;
constexpr int NT = 256;
constexpr int64_t kMaxSmall = 32768, kMaxLarge = 131072;
constexpr int kTable = 24;                                                // matrices of a launch
constexpr uint64_t kGroupElements = 1ull << 28;                           // of a group, where it holds more than one matrix
constexpr int kFine = 256;                                                // see small_product_kernel
constexpr int kPiece = 64;                                                // side of the blocks of the element-wise passes

struct Matrix {
  void* p;
  const void* g;
  float *m, *master;
  f16 *hi[2], *lo, *A, *B, *B1, *C;
  double *part, *inv;          // sums of squares of the pieces; 1 / (norm + eps)
  uint32_t ld_p, ld_g, ld_m, ld_master;
  int rows, cols, n, k;        // n x k: the padded X
  // of a fine group: the lower halves of A, B, and of X in either of its places (elsewhere these are B1 and C, and the lower half of X has one place)
  __host__ __device__ f16* a_lo() const { return B1; }
  __host__ __device__ f16* b_lo() const { return C; }
  __host__ __device__ f16* x_lo(int fine_and_place) const { return lo + (fine_and_place == 3 ? (size_t)n * k : 0); }
  float wd, scale;
  int aligned;                 // rows of all four begin at whole multiples of 4 elements
};

struct Table {
  uint32_t first[kTable];      // the block at which a matrix begins; behind the last: UINT32_MAX
  Matrix e[kTable];
};

struct Hyper {
  float rest, lr;              // rest: 1 - momentum
  double eps64;
  const float *lr_dev, *grad_norm;
  int nesterov;
};

__device__ __forceinline__ int find(const Table& t, uint32_t block) {
  int k = -1;
#pragma unroll
  for (int i = 0; i < kTable; i++) k += block >= t.first[i];
  return k;
}

// m += rest (g - m); the update is m, or (nesterov) the same once more
__device__ __forceinline__ float blend(float m, float g, float rest) { return m + rest * (g - m); }

// The element-wise passes take a piece of 64 x 64 a block.  V = 4: whole pieces of aligned matrices, 4 elements a lane and 16 rows at once, all loads in flight together;
// V = 1: any piece, every row and column looked at.
template <int V> struct Walk {
  static constexpr int kAcross = kPiece / V, kRows = NT / kAcross, kTurns = kPiece / kRows, kBatch = V == 4 ? kTurns : 4;
};

// Elements (r, c) .. of a row of T; those outside the matrix read as 0
template <int V, class T>
__device__ __forceinline__ wide_t<T, V> get(const void* p, int64_t ld, int64_t r, int64_t c, const Matrix& e) {
  wide_t<T, V> v = {};
  if (V == 4 || (r < e.rows && c < e.cols)) v = load_wide<V>((const T*)p + r * ld + c);
  return v;
}
template <int V, class T>
__device__ __forceinline__ void set(void* p, int64_t ld, int64_t r, int64_t c, const Matrix& e, wide_t<T, V> v) {
  if (V == 4 || (r < e.rows && c < e.cols)) store_wide<V>((T*)p + r * ld + c, v);
}
__device__ __forceinline__ bool whole(const Matrix& e, int64_t r0, int64_t c0) { return e.aligned && r0 + kPiece <= e.rows && c0 + kPiece <= e.cols; }

// ---- momentum and the sum of squares of each piece
template <class GT, int V>
__device__ __forceinline__ double momentum_piece(const Matrix& e, const Hyper& h, int64_t r0, int64_t c0, float factor) {
  typedef Walk<V> W;
  const int64_t row = r0 + threadIdx.x / W::kAcross, c = c0 + threadIdx.x % W::kAcross * V;
  double s = 0;
  for (int turn = 0; turn < W::kTurns; turn += W::kBatch) {
    wide_t<float, V> m[W::kBatch];
    wide_t<GT, V> g[W::kBatch];
#pragma unroll
    for (int i = 0; i < W::kBatch; i++) {
      const int64_t r = row + (turn + i) * W::kRows;
      m[i] = get<V, float>(e.m, e.ld_m, r, c, e);
      g[i] = get<V, GT>(e.g, e.ld_g, r, c, e);
    }
#pragma unroll
    for (int i = 0; i < W::kBatch; i++) {
#pragma unroll
      for (int j = 0; j < V; j++) {
        const float gj = (float)g[i][j] * factor, v = blend(m[i][j], gj, h.rest), u = h.nesterov ? blend(v, gj, h.rest) : v;
        m[i][j] = v;
        s += (double)u * u;             // (outside the matrix 0, unless the factor is not finite: then the norm is not either)
      }
      set<V, float>(e.m, e.ld_m, row + (turn + i) * W::kRows, c, e, m[i]);
    }
  }
  return s;
}

template <class GT>
__global__ __launch_bounds__(NT) void momentum_kernel(Table t, Hyper h) {
  __shared__ double red[NT / 64];
  const int k = find(t, blockIdx.x);
  const Matrix& e = t.e[k];
  const uint32_t piece = blockIdx.x - t.first[k];
  const int across = (e.cols + kPiece - 1) / kPiece;
  const int64_t r0 = (int64_t)(piece / across) * kPiece, c0 = (int64_t)(piece % across) * kPiece;
  const float factor = h.grad_norm ? h.grad_norm[1] : 1.f;
  double s = 0;
  if (factor == factor) s = whole(e, r0, c0) ? momentum_piece<GT, 4>(e, h, r0, c0, factor) : momentum_piece<GT, 1>(e, h, r0, c0, factor);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) e.part[piece] = red[0] + red[1] + red[2] + red[3];
}

// 1 / (norm + eps): a block a matrix
constexpr int kNormThreads = 1024;
__global__ __launch_bounds__(kNormThreads) void norm_kernel(Table t, Hyper h) {
  __shared__ double red[kNormThreads / 64];
  const Matrix& e = t.e[blockIdx.x];
  const int n = ((e.rows + kPiece - 1) / kPiece) * ((e.cols + kPiece - 1) / kPiece);
  double s = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += kNormThreads) s += e.part[i];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kNormThreads / 64; w++) s += red[w];
    *e.inv = 1.0 / (sqrt(s) + h.eps64);
  }
}

// X of fp32 as two fp16 numbers
__device__ __forceinline__ void split(float x, f16& hi, f16& lo) {
  hi = (f16)x;
  lo = (f16)((x - (float)hi) * kLo);
}

// V elements of X from (row, col) on: 4 of them are aligned, as X is padded to whole pieces
template <int V>
__device__ __forceinline__ void set_x(const Matrix& e, int64_t row, int64_t col, const float (&x)[V]) {
  wide_t<f16, V> hi, lo;
#pragma unroll
  for (int j = 0; j < V; j++) {
    f16 a, b;
    split(x[j], a, b);
    hi[j] = a;
    lo[j] = b;
  }
  store_wide<V>(e.hi[0] + row * e.k + col, hi);
  store_wide<V>(e.lo + row * e.k + col, lo);
}

// ---- X = u / norm, transposed where there are more rows than columns, zeros in what pads it: a piece of X a block
template <class GT, int V>
__device__ __forceinline__ void lay_out_piece(const Matrix& e, const Hyper& h, int64_t i0, int64_t j0, float (&turned)[kPiece][kPiece + 1]) {
  typedef Walk<V> W;
  const int row = threadIdx.x / W::kAcross, col = threadIdx.x % W::kAcross * V;
  const float factor = h.grad_norm ? h.grad_norm[1] : 1.f;
  const double inv = *e.inv * kX;
  const bool tall = e.rows > e.cols;
  const int64_t r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
  for (int turn = 0; turn < W::kTurns; turn += W::kBatch) {
    wide_t<float, V> m[W::kBatch];
    wide_t<GT, V> g[W::kBatch] = {};
#pragma unroll
    for (int i = 0; i < W::kBatch; i++) {
      const int64_t r = r0 + row + (turn + i) * W::kRows;
      m[i] = get<V, float>(e.m, e.ld_m, r, c0 + col, e);
      if (h.nesterov) g[i] = get<V, GT>(e.g, e.ld_g, r, c0 + col, e);
    }
#pragma unroll
    for (int i = 0; i < W::kBatch; i++) {
      const int s = row + (turn + i) * W::kRows;
      float x[V];
#pragma unroll
      for (int j = 0; j < V; j++) x[j] = (float)((h.nesterov ? blend(m[i][j], (float)g[i][j] * factor, h.rest) : m[i][j]) * inv);
      if (tall) {
#pragma unroll
        for (int j = 0; j < V; j++) turned[s][col + j] = x[j];
      } else {
        set_x<V>(e, i0 + s, j0 + col, x);
      }
    }
  }
}

template <class GT>
__global__ __launch_bounds__(NT) void lay_out_kernel(Table t, Hyper h) {
  __shared__ float turned[kPiece][kPiece + 1];
  const int k = find(t, blockIdx.x);
  const Matrix& e = t.e[k];
  const uint32_t piece = blockIdx.x - t.first[k];
  const int across = e.k / kPiece;
  const int64_t i0 = (int64_t)(piece / across) * kPiece, j0 = (int64_t)(piece % across) * kPiece;      // of X
  const bool tall = e.rows > e.cols;
  if (whole(e, tall ? j0 : i0, tall ? i0 : j0)) lay_out_piece<GT, 4>(e, h, i0, j0, turned);
  else lay_out_piece<GT, 1>(e, h, i0, j0, turned);
  if (!tall) return;
  __syncthreads();
  typedef Walk<4> W;
  const int row = threadIdx.x / W::kAcross, col = threadIdx.x % W::kAcross * 4;
#pragma unroll
  for (int turn = 0; turn < W::kTurns; turn++) {
    const int s = row + turn * W::kRows;
    const float x[4] = {turned[col][s], turned[col + 1][s], turned[col + 2][s], turned[col + 3][s]};
    set_x<4>(e, i0 + s, j0 + col, x);
  }
}

// ---- the step of the parameters: X back, transposed again
template <class PT, bool MASTER, int V>
__device__ __forceinline__ void apply_piece(const Matrix& e, int64_t r0, int64_t c0, float keep, float by, int last, float (&turned)[kPiece][kPiece + 1]) {
  typedef Walk<V> W;
  typedef std::conditional_t<MASTER, float, PT> ST;          // what is stepped
  const int row = threadIdx.x / W::kAcross, col = threadIdx.x % W::kAcross * V;
  const bool tall = e.rows > e.cols;
  for (int turn = 0; turn < W::kTurns; turn += W::kBatch) {
    wide_t<ST, V> old[W::kBatch];
    float x[W::kBatch][V];
#pragma unroll
    for (int i = 0; i < W::kBatch; i++) {
      const int s = row + (turn + i) * W::kRows;
      old[i] = get<V, ST>(MASTER ? (const void*)e.master : e.p, MASTER ? e.ld_master : e.ld_p, r0 + s, c0 + col, e);
      if (tall) {
#pragma unroll
        for (int j = 0; j < V; j++) x[i][j] = turned[s][col + j];
      } else {                                               // (X is padded to whole pieces)
        const wide_t<f16, V> hi = load_wide<V>((const f16*)e.hi[last & 1] + (r0 + s) * e.k + c0 + col), lo = load_wide<V>((const f16*)e.x_lo(last) + (r0 + s) * e.k + c0 + col);
#pragma unroll
        for (int j = 0; j < V; j++) x[i][j] = (float)hi[j] + (float)lo[j] * (1.f / kLo);
      }
    }
#pragma unroll
    for (int i = 0; i < W::kBatch; i++) {
      const int64_t r = r0 + row + (turn + i) * W::kRows;
      wide_t<PT, V> p;
      wide_t<float, V> q;
#pragma unroll
      for (int j = 0; j < V; j++) {
        q[j] = (float)old[i][j] * keep - by * x[i][j];
        p[j] = (PT)q[j];
      }
      if constexpr (MASTER) set<V, float>(e.master, e.ld_master, r, c0 + col, e, q);
      set<V, PT>(e.p, e.ld_p, r, c0 + col, e, p);
    }
  }
}

template <class PT, bool MASTER>
__global__ __launch_bounds__(NT) void apply_kernel(Table t, Hyper h, int last) {
  __shared__ float turned[kPiece][kPiece + 1];
  if (h.grad_norm && h.grad_norm[1] != h.grad_norm[1]) return;
  const int k = find(t, blockIdx.x);
  const Matrix& e = t.e[k];
  const uint32_t piece = blockIdx.x - t.first[k];
  const int across = (e.cols + kPiece - 1) / kPiece;
  const int64_t r0 = (int64_t)(piece / across) * kPiece, c0 = (int64_t)(piece % across) * kPiece;
  const float lr = h.lr_dev ? *h.lr_dev : h.lr;
  const float keep = 1.f - lr * e.wd, by = lr * e.scale * (1.f / kX);
  if (e.rows > e.cols) {
    typedef Walk<4> W;
    const int row = threadIdx.x / W::kAcross, col = threadIdx.x % W::kAcross * 4;
#pragma unroll
    for (int turn = 0; turn < W::kTurns; turn++) {
      const int s = row + turn * W::kRows;
      const int64_t at = (c0 + s) * e.k + r0 + col;
      const wide_t<f16, 4> hi = load_wide<4>((const f16*)e.hi[last & 1] + at), lo = load_wide<4>((const f16*)e.x_lo(last) + at);
#pragma unroll
      for (int j = 0; j < 4; j++) turned[col + j][s] = (float)hi[j] + (float)lo[j] * (1.f / kLo);
    }
    __syncthreads();
  }
  if (whole(e, r0, c0)) apply_piece<PT, MASTER, 4>(e, r0, c0, keep, by, last, turned);
  else apply_piece<PT, MASTER, 1>(e, r0, c0, keep, by, last, turned);
}

// ---- the products.  S x S tiles, four waves of S / 2 x S / 2.  SYM_A: A = X X^T; SYM_B: B = b A + c A A; STEP: X = a X + B X.
// Two steps at once, where X has many more columns than rows: behind A and B
//   SYM_C: C = a A + B A;  SYM_D: A = a C + B C, which is the A of the second step, (a + B) A (a + B);  SYM_B once more, to B1;
//   SYM_Q: C = a (B + B1) + B1 B, so that (a + B1)(a + B) = a^2 + C;  STEP: X = a^2 X + C X
// (all of these commute: the products are symmetric).  Of the first two steps only, where X is small, unless few directions make it up: two later ones would be 2 to 10 times as far off.
// Along a strong direction the terms cancel (a + B is 0.70 at a singular value of 1, of 3.44 and -2.74), so that roundings in front of a sum count several times: that of C = B A, added to a^2 A twice
// as 2 a C, left 3.3e-4 of the factor of one direction above noise of 0.01 (700 x 2500; of one alone 1.4e-3) where apart leave 0.4e-4 (1.9e-4) and these 1.6e-4 (4.4e-4).  Random matrices: 1.5e-3 in each form.
enum Product { SYM_A, SYM_B, SYM_C, SYM_D, SYM_Q, STEP };
constexpr int kPair = 2;             // in `how`, whose lowest bit says which X is there: the second SYM_B, and the STEP, of two steps at once

// Blocks are dealt to the 8 XCDs round-robin, and each XCD has an L2 of its own: a matrix is given to `span` XCDs from `first` on, and each of those a row of consecutive tiles of it.
struct Deal {
  uint32_t tiles[kTable];
  uint8_t first[kTable], span[kTable];
  int n;
};

static_assert(sizeof(Table) + sizeof(Deal) <= 4000, "a kernel's arguments");

// The matrix and the tile of a block (-1: none left for its XCD)
__device__ __forceinline__ int dealt(const Deal& d, uint32_t block, int& tile) {
  const uint32_t xcd = block & 7;
  uint32_t at = block >> 3;
  for (int i = 0; i < d.n; i++) {
    const uint32_t share = xcd - d.first[i], span = d.span[i];
    if (share >= span) continue;
    const uint32_t most = d.tiles[i] / span, more = d.tiles[i] % span, count = most + (share < more);
    if (at < count) {
      tile = (int)(share * most + min(share, more) + at);
      return i;
    }
    at -= count;
  }
  return -1;
}

// Which tile a block computes, and its operands
struct Job {
  int ti, tj, m0, n0, lda, ldb, K;
  const f16 *a, *b;
};
template <int S, Product P>
__device__ __forceinline__ void find_job(const Matrix& e, int tile, int how, Job& j) {
  if constexpr (P == STEP) {                       // down groups of 4 tile rows
    const int tm = e.n / S, tn = e.k / S, group = tile / (4 * tn), rows = min(tm - 4 * group, 4), in = tile - group * 4 * tn;
    j.ti = group * 4 + in % rows;
    j.tj = in / rows;
  } else {                                         // row ti of the triangle holds ti + 1 tiles
    int ti = (int)((sqrtf(8.f * tile + 1.f) - 1.f) * 0.5f);
    while (ti * (ti + 1) / 2 > tile) ti--;
    while ((ti + 1) * (ti + 2) / 2 <= tile) ti++;
    j.ti = ti;
    j.tj = tile - ti * (ti + 1) / 2;
  }
  j.m0 = j.ti * S;
  j.n0 = j.tj * S;
  const f16* X = e.hi[how & 1];
  if constexpr (P == SYM_A) { j.lda = j.ldb = j.K = e.k; j.a = X + (size_t)j.m0 * e.k; j.b = X + (size_t)j.n0 * e.k; }
  else if constexpr (P == STEP) { j.lda = j.K = e.n; j.ldb = e.k; j.a = (how & kPair ? e.C : e.B) + (size_t)j.m0 * e.n; j.b = X + j.n0; }
  else {
    const f16 *l = P == SYM_B ? e.A : P == SYM_Q ? e.B1 : e.B, *r = P == SYM_D ? e.C : P == SYM_Q ? e.B : e.A;
    j.lda = j.ldb = j.K = e.n; j.a = l + (size_t)j.m0 * e.n; j.b = r + (size_t)j.n0 * e.n;
  }
}

// What 8 elements of a result from (row, col) on need beside their sums: the two halves of X, or one or two of the square matrices.  Asked for ahead: the compiler would not
// move these loads over the stores of the elements before.
template <Product P, bool FINE = false> constexpr int beside() { return P == SYM_A ? 0 : P == SYM_Q || P == STEP || FINE ? 2 : 1; }
struct Beside { f16x8 u, v; };
template <Product P, bool FINE = false>
__device__ __forceinline__ Beside ask8(const Matrix& e, int how, int row, int col) {
  Beside x = {};
  const size_t at = (size_t)row * (P == STEP ? e.k : e.n) + col;
  const f16 *u = P == STEP ? e.hi[how & 1] : P == SYM_Q ? e.B : P == SYM_D ? e.C : e.A, *v = P == STEP ? e.x_lo(FINE ? 2 | how : 0) : P == SYM_Q ? e.B1 : e.a_lo();
  if constexpr (beside<P, FINE>() > 0) x.u = *(const f16x8*)(u + at);
  if constexpr (beside<P, FINE>() > 1) x.v = *(const f16x8*)(v + at);
  return x;
}
// ... and those elements, whose sums are v
template <Product P, bool FINE = false>
__device__ __forceinline__ void put8(const Matrix& e, int how, int row, int col, const float (&v)[8], const Beside& x) {
  f16x8 o;
  if constexpr (P == STEP) {
    f16x8 ol;
    const float a = how & kPair && !FINE ? kA_ * kA_ : kA_;
#pragma unroll
    for (int j = 0; j < 8; j++) {
      f16 hi, lo;
      split(__builtin_fmaf(a, (float)x.u[j] + (float)x.v[j] * (1.f / kLo), v[j] * (1.f / kA)), hi, lo);
      o[j] = hi;
      ol[j] = lo;
    }
    *(f16x8*)(e.hi[(how & 1) ^ 1] + (size_t)row * e.k + col) = o;
    *(f16x8*)(e.x_lo(FINE ? 2 | (how ^ 1) : 0) + (size_t)row * e.k + col) = ol;
  } else if constexpr (FINE) {
    f16x8 ol;
#pragma unroll
    for (int j = 0; j < 8; j++) {
      f16 hi, lo;
      split(P == SYM_A ? v[j] * (kA / (kX * kX)) : __builtin_fmaf(kB_, (float)x.u[j] + (float)x.v[j] * (1.f / kLo), v[j] * (kC_ / kA)), hi, lo);
      o[j] = hi;
      ol[j] = lo;
    }
    *(f16x8*)((P == SYM_A ? e.A : e.B) + (size_t)row * e.n + col) = o;
    *(f16x8*)((P == SYM_A ? e.a_lo() : e.b_lo()) + (size_t)row * e.n + col) = ol;
  } else {
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const float u = (float)x.u[j], w = (float)x.v[j], sum = v[j] * (P == SYM_A ? kA / (kX * kX) : 1.f / kA);
      o[j] = (f16)(P == SYM_A ? sum : P == SYM_B ? __builtin_fmaf(kB_, u, kC_ * sum) : __builtin_fmaf(kA_, P == SYM_Q ? u + w : u, sum));
    }
    f16* to = P == SYM_B ? (how & kPair ? e.B1 : e.B) : P == SYM_A || P == SYM_D ? e.A : e.C;
    *(f16x8*)(to + (size_t)row * e.n + col) = o;
  }
}

template <int S, Product P, int DEPTH>
__global__ __launch_bounds__(NT) void product_kernel(Table t, Deal d, int how) {
  constexpr int W = S / 2, TB = W / 16;
  constexpr bool BKS = P == STEP;                  // X is [k, columns] there
  constexpr int RING = k64::ring_bytes<S, S, DEPTH, true>();
  __shared__ __attribute__((aligned(1024))) char ring[RING];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / 2, wn = wave % 2;
  int tile = 0;
  const int which = __builtin_amdgcn_readfirstlane(dealt(d, blockIdx.x, tile));
  if (which < 0) return;
  const Matrix& e = t.e[which];
  Job g;
  find_job<S, P>(e, tile, how, g);
  f32x4 acc[TB][TB];
#pragma unroll
  for (int i = 0; i < TB; i++)
#pragma unroll
    for (int j = 0; j < TB; j++) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  k64::run<S, S, 2, 2, false, BKS, DEPTH, true>((const char*)g.a, (const char*)g.b, g.lda, g.ldb, 0, g.K, ring, acc, wave, wm, wn, lane);
  __builtin_amdgcn_s_waitcnt(0);                   // the redundant tail loads are over before the ring is used again
  // The compiler does not see that the accumulators come from matrix instructions: 16 wait states before the first read
  // of the last one's result.
  asm volatile("s_nop 15");
#pragma unroll
  for (int i = 0; i < TB; i++)
#pragma unroll
    for (int j = 0; j < TB; j++) asm volatile("" : "+a"(acc[i][j]));
  // As in gemm.hip: 32 rows at a time through a strip of the wave's own, to be read back row-major, 8 columns a lane
  constexpr int ROWB = W * 4 + 16, PPR = W / 8, RPI = 64 / PPR, NIT = 32 / RPI;
  static_assert(4 * 32 * ROWB <= RING, "the strips fit in the ring");
  __syncthreads();
  char* strip = ring + wave * (32 * ROWB);
  const int cp = lane % PPR, row0 = lane / PPR, n0 = g.n0 + wn * W;
  Beside x[2][NIT], xt[W / 64][4];
  auto ask = [&](int tm) {
#pragma unroll
    for (int it = 0; it < NIT; it++) x[tm & 1][it] = ask8<P>(e, how, g.m0 + wm * W + tm * 32 + row0 + it * RPI, n0 + cp * 8);
  };
  ask(0);
#pragma unroll
  for (int tm = 0; tm < W / 32; tm++) {
    const int mbase = g.m0 + wm * W + tm * 32;
    if (tm + 1 < W / 32) ask(tm + 1);
    if constexpr (P != STEP && beside<P>() > 0) {  // (the same elements across the diagonal, where other matrices are not symmetric to the last bit)
      if (g.ti != g.tj) {
#pragma unroll
        for (int half = 0; half < W / 64; half++)
#pragma unroll
          for (int r = 0; r < 4; r++) xt[half][r] = ask8<P>(e, how, n0 + half * 64 + lane, mbase + r * 8);
      }
    }
#pragma unroll
    for (int tr = 0; tr < 2; tr++)
#pragma unroll
      for (int tn = 0; tn < TB; tn++) *(f32x4*)(strip + (tr * 16 + (lane & 15)) * ROWB + (tn * 16 + 4 * (lane >> 4)) * 4) = acc[2 * tm + tr][tn];
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(63));
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int it = 0; it < NIT; it++) {
      const int row = row0 + it * RPI;
      const char* q = strip + row * ROWB + cp * 32;
      const f32x4 v0 = *(const f32x4*)q, v1 = *(const f32x4*)(q + 16);
      const float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
      put8<P>(e, how, mbase + row, n0 + cp * 8, v, x[tm & 1][it]);
    }
    if constexpr (P != STEP) {
      if (g.ti != g.tj) {                          // the tile across the diagonal: 8 rows of a column a lane
#pragma unroll
        for (int half = 0; half < W / 64; half++)
#pragma unroll
          for (int r = 0; r < 4; r++) {
            const int c = half * 64 + lane;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = *(const float*)(strip + (r * 8 + j) * ROWB + c * 4);
            put8<P>(e, how, n0 + c, mbase + r * 8, v, xt[half][r]);
          }
      }
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(63));
    __builtin_amdgcn_wave_barrier();
  }
}

// The same for few tiles: 64 x 64, each wave one k-step in four of the whole tile.  Four times the blocks, whose chains of k-steps are a quarter as long.
// FINE: where the smaller side is at most kFine and the parameters are kept in fp32, all operands are kept in 22 bits, and three products stand for one (upper by lower half, lower by
// upper, upper by upper: what is left out is 2^-22): the factor is 1e-6 to 5e-6 off.  Operands in 11 bits leave random matrices 2.6e-3 (16 rows) to 1.6e-3 (256), and hardly less where there
// are more: 1.6e-3 (257 to 700 rows), 1.2e-3 (2048).  The cut is one of cost.  A whole step in 11 and in 22 bits, us: the smallest stage's 12 matrices of 256 x 256 and 256 x 1024 129, 188 (a launch
// 7 to 9, 10 to 13.5); 12 of 257 x 257 and 257 x 1024 194, 277; one 512 x 512 118, 168; 12 of 512 x 512 and 512 x 2048 309, 517; one 1024 x 1024 144, 232; four with sides of 768 and four times that 393, 803;
// 12 of 450 .. 900 by 900 .. 3000 541, 1349; one 2048 x 2048 324, 1084.
template <Product P, bool FINE>
__global__ __launch_bounds__(NT) void small_product_kernel(Table t, Deal d, int how) {
  constexpr int S = 64, ROWB = S * 4 + 16, STRIP = S * ROWB;
  constexpr int RING = ksplit::stages<S, S>() * ksplit::stage_bytes<S, S>();
  static_assert(4 * STRIP <= RING, "the partial sums fit in the ring");
  __shared__ __attribute__((aligned(1024))) char ring[RING];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int tile = 0;
  const int which = __builtin_amdgcn_readfirstlane(dealt(d, blockIdx.x, tile));
  if (which < 0) return;
  const Matrix& e = t.e[which];
  Job g;
  find_job<S, P>(e, tile, how, g);
  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; i++)
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int r = 0; r < 16; r++) acc[i][j][r] = 0.f;
  const char *a = (const char*)g.a, *b = (const char*)g.b;
  if constexpr (FINE) {
    // (the lower halves are laid out like the upper ones)
    const f16 *xl = e.x_lo(2 | how), *l = P == SYM_A ? xl : P == SYM_B ? e.a_lo() : e.b_lo(), *r = P == SYM_B ? e.a_lo() : xl;
    const f16 *lh = P == SYM_A ? e.hi[how] : P == SYM_B ? e.A : e.B, *rh = P == SYM_B ? e.A : e.hi[how];
    const char *al = (const char*)(l + (g.a - lh)), *bl = (const char*)(r + (g.b - rh));
    ksplit::run<S, S, false, P == STEP, true, 3>({a, al, a}, {bl, b, b}, g.lda, g.ldb, g.K, ring, acc, wave, lane, 1.f / kLo);
  } else {
    ksplit::run<S, S, false, P == STEP, true>({a}, {b}, g.lda, g.ldb, g.K, ring, acc, wave, lane);
  }
  __builtin_amdgcn_s_waitcnt(0);
  // a wave writes 16 of the rows, and as many columns across the diagonal
  const int row0 = wave * 16 + lane / 8, cp = lane % 8;
  Beside x[2], xt[2] = {};
#pragma unroll
  for (int it = 0; it < 2; it++) x[it] = ask8<P, FINE>(e, how, g.m0 + row0 + it * 8, g.n0 + cp * 8);
  if constexpr (P != STEP && beside<P, FINE>() > 0) {
    if (g.ti != g.tj) {
#pragma unroll
      for (int r = 0; r < 2; r++) xt[r] = ask8<P, FINE>(e, how, g.n0 + lane, g.m0 + wave * 16 + r * 8);
    }
  }
  __syncthreads();
  char* strip = ring + wave * STRIP;
#pragma unroll
  for (int tr = 0; tr < 2; tr++)
#pragma unroll
    for (int tn = 0; tn < 2; tn++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const f32x16& a = acc[tr][tn];
        *(f32x4*)(strip + (tr * 32 + (lane & 31)) * ROWB + (tn * 32 + 8 * q + 4 * (lane >> 5)) * 4) = f32x4{a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
      }
  __syncthreads();
  // the four partial sums are added up in the order of the k shares
#pragma unroll
  for (int it = 0; it < 2; it++) {
    const int row = row0 + it * 8;
    const char* q = ring + row * ROWB + cp * 32;
    f32x4 v0 = *(const f32x4*)q, v1 = *(const f32x4*)(q + 16);
#pragma unroll
    for (int w = 1; w < 4; w++) { v0 += *(const f32x4*)(q + w * STRIP); v1 += *(const f32x4*)(q + w * STRIP + 16); }
    const float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
    put8<P, FINE>(e, how, g.m0 + row, g.n0 + cp * 8, v, x[it]);
  }
  if constexpr (P != STEP) {
    if (g.ti != g.tj) {
#pragma unroll
      for (int r = 0; r < 2; r++) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const char* q = ring + (wave * 16 + r * 8 + j) * ROWB + lane * 4;
          v[j] = *(const float*)q;
#pragma unroll
          for (int w = 1; w < 4; w++) v[j] += *(const float*)(q + w * STRIP);
        }
        put8<P, FINE>(e, how, g.n0 + lane, g.m0 + wave * 16 + r * 8, v, xt[r]);
      }
    }
  }
}

// ---- host: matrices in groups that are worked on together
uint64_t up(uint64_t n, uint64_t to) { return (n + to - 1) / to * to; }

struct Group {
  std::vector<int> which;      // of the call's matrices
  int tile;
  bool pair, fine;
  std::vector<int> n, k;       // padded
  uint64_t bytes;
};

int64_t small_side(const ah_muon_matrix_t& x) { return std::min(x.rows, x.cols); }
int64_t large_side(const ah_muon_matrix_t& x) { return std::max(x.rows, x.cols); }

// What the products' blocks take, us, K in thousands (times that the tiles share, such as that of the results' bytes, left out): one that has its CU to itself, and its share of
// a CU that is full.  Measured (one box, us a step, tiles of 64, 128, 256): one 1024 x 1024 167, 236, 533; one 1024 x 4096 276, 335, 782; one 2048 x 2048 474, 375,
// 825; 7 of 1024 x 2048 815, 678, 840; 24 of 1024 x 1024 1470, 1199, 1503; 4 of 2048 x 2048 1563, 1136, 1124; one 4096 x 4096 2792, 1793, 1654; one 4096 x 11008 6344, 4146, 3688.
struct Kind { int tile; double alone0, alone1, full0, full1; };
constexpr Kind kKinds[] = {{64, 4.5, 4.0, 0.4, 4.2}, {128, 4.5, 7.8, 3.5, 8.1}, {256, 6.0, 22.0, 6.0, 22.0}};

// Tiles of a product of an n x m matrix (padded), and its K
uint64_t tiles_of(Product p, uint64_t n, uint64_t m, int tile) { return p == STEP ? (n / tile) * (m / tile) : (n / tile) * (n / tile + 1) / 2; }
double depth_of(Product p, uint64_t n, uint64_t m) { return (p == SYM_A ? m : n) * 1e-3; }

// What a product of a group is expected to take
double time_of(Product p, const ah_muon_matrix_t* x, const std::vector<int>& which, const Kind& k) {
  double sum = 0, longest = 0;
  uint64_t tiles = 0;
  for (int i : which) {
    const uint64_t n = up(small_side(x[i]), std::max(k.tile, 128)), m = up(large_side(x[i]), std::max(k.tile, 128)), count = tiles_of(p, n, m, k.tile);
    const double K = depth_of(p, n, m);
    sum += count * (k.full0 + k.full1 * K);
    longest = std::max(longest, k.alone0 + k.alone1 * K);
    tiles += count;
  }
  // (a block of 256 x 256 has its CU to itself: whole rounds)
  return std::max(longest, k.tile == 256 ? sum / tiles * ((tiles + 255) / 256) : sum / 256);
}

// The tiles that a group's products are expected to be fastest with, and whether its first two steps are taken at once: three more products of n^3 for one A and one X less.
// Five steps, apart and at once, us: a LLaMA-style layer 14830, 14130; 4 of 2048 x 8192 2924, 2651; one 5120 x 20480 8270, 7269; 4 of 1536 x 4608 1158, 1079; one 4096 x 6144
// 2329, 2326; one 4096 x 4096 1558, 1627; 24 of 1024 x 1024 1323, 1443.  Tiles of 64 never take it: their products are bound by the launches, of which it has one more.
void choose(const ah_muon_matrix_t* x, Group& g) {
  g.tile = 64;
  g.pair = false;
  if (g.fine) return;
  double least = 0;
  for (const Kind& k : kKinds) {
    const double a = time_of(SYM_A, x, g.which, k), b = time_of(SYM_B, x, g.which, k), step = time_of(STEP, x, g.which, k);
    if (least == 0 || a + b + step < least) {
      least = a + b + step;
      g.tile = k.tile;
      g.pair = k.tile > 64 && a + step > 1.05 * 3 * b + 3;
    }
  }
}

// Deals a product's tiles to the XCDs.  Tiles of 64 and 128, which are bound by how fast their operands arrive: each matrix to as few XCDs as have it in their L2s (4 MB each) and
// take at most a tenth and 1.5 us longer for it than all together would, in the table's order (the largest first) to those that have least.  (One box, us a step, every matrix to 1, 2, 4
// and 8 XCDs: the smallest stage's 12 matrices 130, 140, 148, 153; 12 of 768 x about 2000 609, 571, 579, 617.)  Tiles of 256 to all of them: evenly (a LLaMA-style layer, 1 to 8 XCDs
// a matrix: 21900, 16500, 15300, 14640).  Returns the launch's blocks.
uint32_t deal(Product p, const Table& t, int n, const Kind& kind, Deal& d) {
  uint32_t most = 0;
  for (int span = kind.tile < 256 ? 1 : 8; span <= 8; span *= 2) {
    bool fits = true;
    for (int i = 0; i < n; i++) fits = fits && 2ull * t.e[i].n * t.e[i].k <= (4ull << 20) * span;
    if (!fits && span < 8) continue;
    double load[8] = {}, sum = 0, top = 0;
    uint64_t count[8] = {};
    for (int i = 0; i < n; i++) {
      const uint64_t tiles = tiles_of(p, t.e[i].n, t.e[i].k, kind.tile);
      const double cost = tiles * (kind.full0 + kind.full1 * depth_of(p, t.e[i].n, t.e[i].k));
      int at = 0;
      for (int x = span; x < 8; x += span)
        if (load[x] < load[at]) at = x;
      d.tiles[i] = (uint32_t)tiles;
      d.first[i] = (uint8_t)at;
      d.span[i] = (uint8_t)span;
      for (int x = 0; x < span; x++) {
        load[at + x] += cost / span;
        count[at + x] += tiles / span + ((uint64_t)x < tiles % span);
      }
      sum += cost;
    }
    d.n = n;
    most = 0;
    for (int x = 0; x < 8; x++) {
      top = std::max(top, load[x]);
      most = std::max(most, (uint32_t)count[x]);
    }
    if (top / 32 <= 1.1 * sum / 256 + 1.5) break;       // (32 CUs to an XCD)
  }
  return most * 8;
}

struct Offsets { uint64_t hi0, hi1, lo, A, B, B1, C, part, inv, end; };
Offsets offsets(const ah_muon_matrix_t& x, int n, int k, const Group& g, uint64_t at) {
  Offsets o;
  auto take = [&](uint64_t bytes) { const uint64_t r = at; at += up(bytes, 256); return r; };
  const uint64_t nk = (uint64_t)n * k, nn = (uint64_t)n * n;
  o.hi0 = take(2 * nk); o.hi1 = take(2 * nk); o.lo = take(g.fine ? 4 * nk : 2 * nk);
  o.A = take(2 * nn); o.B = take(2 * nn);
  o.B1 = take(g.pair || g.fine ? 2 * nn : 0); o.C = take(g.pair || g.fine ? 2 * nn : 0);
  o.part = take(8 * (up(x.rows, kPiece) / kPiece) * (up(x.cols, kPiece) / kPiece));
  o.inv = take(8);
  o.end = at;
  return o;
}

// kept32: what is stepped is kept in 32 bits, so that the small matrices' groups are fine ones
std::vector<Group> plan(const ah_muon_matrix_t* x, int n, bool kept32) {
  std::vector<int> order;
  for (int i = 0; i < n; i++)
    if (x[i].rows && x[i].cols) order.push_back(i);
  auto fine = [&](int i) { return kept32 && small_side(x[i]) <= kFine; };
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return fine(a) != fine(b) ? fine(b) : x[a].rows * x[a].cols > x[b].rows * x[b].cols; });
  std::vector<Group> groups;
  uint64_t elements = 0;
  for (int i : order) {
    const uint64_t own = up(small_side(x[i]), 256) * up(large_side(x[i]), 256);
    if (groups.empty() || (int)groups.back().which.size() == kTable || elements + own > kGroupElements || groups.back().fine != fine(i)) {
      groups.push_back({});
      groups.back().fine = fine(i);
      elements = 0;
    }
    groups.back().which.push_back(i);
    elements += own;
  }
  for (Group& g : groups) {
    choose(x, g);
    g.bytes = 0;
    for (int i : g.which) {
      g.n.push_back((int)up(small_side(x[i]), std::max(g.tile, 128)));       // (the products' k axis: a multiple of 128)
      g.k.push_back((int)up(large_side(x[i]), std::max(g.tile, 128)));
      g.bytes = offsets(x[i], g.n.back(), g.k.back(), g, g.bytes).end;
    }
  }
  return groups;
}

int check_list(const char* who, const ah_muon_matrix_t* x, int n) {
  if (n < 0 || (n > 0 && !x)) return set_error(AH_EINVAL, "%s: bad matrix list", who);
  for (int i = 0; i < n; i++) {
    if (x[i].rows < 0 || x[i].cols < 0) return set_error(AH_EINVAL, "%s: matrix %d has a negative size", who, i);
    if (large_side(x[i]) > kMaxLarge || small_side(x[i]) > kMaxSmall)
      return set_error(AH_EUNSUPPORTED, "%s: matrix %d is %lld x %lld: at most 32768 by 131072", who, i, (long long)x[i].rows, (long long)x[i].cols);
  }
  return AH_OK;
}

// Gives each matrix of the table the blocks that it takes, and calls go(their number).
template <class F, class G>
hipError_t launch(Table& t, const Group& g, const F& blocks_of, const G& go) {
  uint64_t blocks = 0;
  const int n = (int)g.which.size();
  for (int i = 0; i < kTable; i++) {
    t.first[i] = i < n ? (uint32_t)blocks : UINT32_MAX;
    if (i < n) blocks += blocks_of(t.e[i]);
  }
  if (blocks > (1u << 23)) return hipErrorInvalidValue;      // (threads of a launch are counted in 32 bits)
  go((uint32_t)blocks);
  return hipGetLastError();
}

// last: which of its two places X is in behind the last step, and 2 of a fine group
template <int S>
hipError_t products(const Table& t, const Group& g, int steps, int* last, hipStream_t s) {
  const Kind& kind = S == 64 ? kKinds[0] : S == 128 ? kKinds[1] : kKinds[2];
  Deal deals[3];                                   // of X X^T, of n x n x n, of the STEP
  uint32_t blocks[3];
  for (int i = 0; i < 3; i++) {
    blocks[i] = deal(i == 0 ? SYM_A : i == 1 ? SYM_B : STEP, t, (int)g.which.size(), kind, deals[i]);
    if (blocks[i] > (1u << 23)) return hipErrorInvalidValue;
  }
  hipError_t e = hipSuccess;
  auto product = [&](auto kind_of, int how) {
    constexpr Product P = decltype(kind_of)::value;
    constexpr int at = P == SYM_A ? 0 : P == STEP ? 2 : 1;
    if (e != hipSuccess) return;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks[at]), dim3(NT), 0, s, t, deals[at], how); };
    if constexpr (S == 64) g.fine ? go(small_product_kernel<P, true>) : go(small_product_kernel<P, false>);
    else if constexpr (S == 256) go(product_kernel<S, P, 2>);
    else if (blocks[at] <= 256) go(product_kernel<S, P, 3>);
    else go(product_kernel<S, P, 2>);
    e = hipGetLastError();
  };
  int from = 0;
  for (int i = 0; i < steps; i++, from ^= 1) {
    const bool pair = S > 64 && g.pair && i == 0 && steps > 1;
    product(std::integral_constant<Product, SYM_A>(), from);
    product(std::integral_constant<Product, SYM_B>(), from);
    if constexpr (S > 64) {
      if (pair) {
        product(std::integral_constant<Product, SYM_C>(), from);
        product(std::integral_constant<Product, SYM_D>(), from);
        product(std::integral_constant<Product, SYM_B>(), from | kPair);
        product(std::integral_constant<Product, SYM_Q>(), from);
        i++;
      }
    }
    product(std::integral_constant<Product, STEP>(), pair ? from | kPair : from);
  }
  *last = g.fine ? 2 | from : from;
  return e;
}

hipError_t step_group(const ah_muon_t* c, const ah_muon_matrix_t* x, const Group& g, char* work, bool master, hipStream_t s) {
  Table t = {};
  uint64_t at = 0;
  for (size_t i = 0; i < g.which.size(); i++) {
    const ah_muon_matrix_t& y = x[g.which[i]];
    const Offsets o = offsets(y, g.n[i], g.k[i], g, at);
    Matrix& e = t.e[i];
    e.p = y.param; e.g = y.grad; e.m = y.momentum; e.master = y.master;
    e.hi[0] = (f16*)(work + o.hi0); e.hi[1] = (f16*)(work + o.hi1); e.lo = (f16*)(work + o.lo);
    e.A = (f16*)(work + o.A); e.B = (f16*)(work + o.B); e.B1 = (f16*)(work + o.B1); e.C = (f16*)(work + o.C); e.part = (double*)(work + o.part); e.inv = (double*)(work + o.inv);
    auto stride = [&](int64_t ld) { return (uint32_t)(ld ? ld : y.cols); };       // (at most 2^31)
    e.ld_p = stride(y.ld_param); e.ld_g = stride(y.ld_grad); e.ld_m = stride(y.ld_momentum); e.ld_master = stride(y.ld_master);
    e.rows = (int)y.rows; e.cols = (int)y.cols; e.n = g.n[i]; e.k = g.k[i];
    e.wd = y.weight_decay; e.scale = y.scale;
    const int pb = c->param_type == AH_FP32 ? 4 : 2, gb = c->grad_type == AH_FP32 ? 4 : 2;
    e.aligned = ((e.ld_p | e.ld_g | e.ld_m | e.ld_master) & 3) == 0 && aligned_to(e.p, 4 * pb) && aligned_to(e.g, 4 * gb) && aligned_to(e.m, 16) && aligned_to(e.master, 16);
    at = o.end;
  }
  Hyper h = {};
  h.rest = (float)(1 - c->momentum); h.lr = (float)c->lr; h.eps64 = c->eps;
  h.lr_dev = c->lr_dev; h.grad_norm = c->grad_norm; h.nesterov = c->nesterov;
  auto pieces = [](const Matrix& e) { return (uint64_t)((e.rows + kPiece - 1) / kPiece) * ((e.cols + kPiece - 1) / kPiece); };
  auto pieces_x = [](const Matrix& e) { return (uint64_t)(e.n / kPiece) * (e.k / kPiece); };
  const bool g32 = c->grad_type == AH_FP32;
  hipError_t e = launch(t, g, pieces, [&](uint32_t b) {
    if (g32) hipLaunchKernelGGL(momentum_kernel<float>, dim3(b), dim3(NT), 0, s, t, h);
    else hipLaunchKernelGGL(momentum_kernel<bf16>, dim3(b), dim3(NT), 0, s, t, h);
    hipLaunchKernelGGL(norm_kernel, dim3(g.which.size()), dim3(kNormThreads), 0, s, t, h);
  });
  if (e == hipSuccess)
    e = launch(t, g, pieces_x, [&](uint32_t b) {
      if (g32) hipLaunchKernelGGL(lay_out_kernel<float>, dim3(b), dim3(NT), 0, s, t, h);
      else hipLaunchKernelGGL(lay_out_kernel<bf16>, dim3(b), dim3(NT), 0, s, t, h);
    });
  int last = 0;
  if (e == hipSuccess) e = g.tile == 256 ? products<256>(t, g, c->ns_steps, &last, s) : g.tile == 128 ? products<128>(t, g, c->ns_steps, &last, s) : products<64>(t, g, c->ns_steps, &last, s);
  if (e == hipSuccess)
    e = launch(t, g, pieces, [&](uint32_t b) {
      if (c->param_type == AH_FP32) hipLaunchKernelGGL((apply_kernel<float, false>), dim3(b), dim3(NT), 0, s, t, h, last);
      else if (master) hipLaunchKernelGGL((apply_kernel<bf16, true>), dim3(b), dim3(NT), 0, s, t, h, last);
      else hipLaunchKernelGGL((apply_kernel<bf16, false>), dim3(b), dim3(NT), 0, s, t, h, last);
    });
  return e;
}

}  // namespace

extern "C" int ah_muon_workspace(const ah_muon_matrix_t* x, int n, uint64_t* bytes) {
  if (!bytes) return set_error(AH_EINVAL, "ah_muon_workspace: bytes is NULL");
  if (int rc = check_list("ah_muon_workspace", x, n)) return rc;
  try {
    *bytes = 256;
    for (bool kept32 : {false, true})
      for (const Group& g : plan(x, n, kept32)) *bytes = std::max(*bytes, g.bytes);
  } catch (...) {
    return set_error(AH_ENOMEM, "ah_muon_workspace: no host memory");
  }
  return AH_OK;
}

extern "C" int ah_muon_step(const ah_muon_t* c, const ah_muon_matrix_t* x, int n, void* workspace, void* stream) {
  discard_stale_hip_error();
  const char* who = "ah_muon_step";
  if (!c) return set_error(AH_EINVAL, "%s: config is NULL", who);
  if (c->struct_size != sizeof(ah_muon_t)) return set_error(AH_EINVAL, "%s: struct_size %u != %zu", who, c->struct_size, sizeof(ah_muon_t));
  if ((c->param_type != AH_BF16 && c->param_type != AH_FP32) || (c->grad_type != AH_BF16 && c->grad_type != AH_FP32))
    return set_error(AH_EINVAL, "%s: types must be AH_BF16 or AH_FP32", who);
  if ((c->nesterov != 0 && c->nesterov != 1) || c->ns_steps < 1 || c->ns_steps > 32) return set_error(AH_EINVAL, "%s: need nesterov 0 or 1 and 1 .. 32 ns_steps", who);
  if (!(c->lr >= 0) || !std::isfinite(c->lr) || !(c->momentum >= 0 && c->momentum < 1) || !(c->eps >= 1e-37) || !std::isfinite(c->eps))
    return set_error(AH_EINVAL, "%s: need finite lr >= 0, momentum in [0, 1) and eps >= 1e-37", who);
  if (!aligned_to(c->lr_dev, 4) || !aligned_to(c->grad_norm, 4)) return set_error(AH_EINVAL, "%s: misaligned device scalar", who);
  if (int rc = check_list(who, x, n)) return rc;
  const size_t pb = c->param_type == AH_FP32 ? 4 : 2, gb = c->grad_type == AH_FP32 ? 4 : 2;
  bool master = false, any = false;
  for (int i = 0; i < n; i++) {
    const ah_muon_matrix_t& y = x[i];
    if (!y.rows || !y.cols) continue;
    if (!y.param || !y.grad || !y.momentum) return set_error(AH_EINVAL, "%s: matrix %d has a NULL pointer", who, i);
    if (!aligned_to(y.param, pb) || !aligned_to(y.grad, gb) || !aligned_to(y.momentum, 4) || !aligned_to(y.master, 4))
      return set_error(AH_EINVAL, "%s: matrix %d is not aligned to its elements", who, i);
    for (int64_t ld : {y.ld_param, y.ld_grad, y.ld_momentum, y.ld_master})
      if (ld != 0 && (ld < y.cols || ld > (1ll << 31))) return set_error(AH_EINVAL, "%s: matrix %d: a row stride must be at least its columns, %lld, and at most 2^31", who, i, (long long)y.cols);
    if (!std::isfinite(y.weight_decay) || !std::isfinite(y.scale)) return set_error(AH_EINVAL, "%s: matrix %d: weight_decay or scale is not finite", who, i);
    if (any && master != (y.master != nullptr)) return set_error(AH_EINVAL, "%s: either all matrices have a master copy or none", who);
    master = y.master != nullptr;
    any = true;
  }
  if (master && pb == 4) return set_error(AH_EINVAL, "%s: master copies go with bf16 parameters", who);
  if (!any) return AH_OK;
  if (!workspace || !aligned_to(workspace, 256)) return set_error(AH_EINVAL, "%s: workspace is NULL or not 256-byte aligned", who);
  try {
    for (const Group& g : plan(x, n, master || pb == 4)) {
      const hipError_t e = step_group(c, x, g, (char*)workspace, master, (hipStream_t)stream);
      if (e != hipSuccess) return hip_status(e, who);
    }
  } catch (...) {
    return set_error(AH_ENOMEM, "%s: no host memory", who);
  }
  return AH_OK;
}
