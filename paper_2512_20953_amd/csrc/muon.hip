// Optimizer step of matrices by the orthogonal factor of their momentum (declared in include/ah_ops.h): momentum and its norm, five (ns_steps) times three matrix
// products on the loop of gemm_loop.h, and the step of the parameters.
//
// With X [n, m], n <= m (a matrix of more rows than columns is laid out transposed):
//   A = X X^T                 n^2 m flops: the product is symmetric, so that the tiles on and below the diagonal are computed and each is stored twice
//   B = b A + c A A           n^3: likewise
//   X = a X + B X             2 n^2 m
// Bound by the matrix units from n of about a thousand on.
//
// Types.  The operands are fp16: with everything within 3 in magnitude (A and B are polynomials of a matrix whose singular values stay below 1.21) its range suffices, and it
// keeps 11 bits where bf16 keeps 8, at the same rate.  X itself goes from product to product in 22 bits, as two fp16 numbers: what is added to a X has to be added to the same X
// that it was computed from, or the rounding of every step is taken for a part of X, which the polynomial multiplies by up to 3.44 a step where singular values are small.  Of a
// matrix with 64 strong directions above a floor of noise (1024 x 2816) the factor is 5e-4 off in norm, with X in fp16 alone 2e-2, in bf16 alone 0.18.  Fixed powers of two keep small
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
constexpr int kPiece = 64;                                                // side of the blocks of the element-wise passes

struct Matrix {
  void* p;
  const void* g;
  float *m, *master;
  f16 *hi[2], *lo, *A, *B;
  double *part, *inv;          // sums of squares of the pieces; 1 / (norm + eps)
  int64_t ld_p, ld_g, ld_m, ld_master;
  int rows, cols, n, k;        // n x k: the padded X
  float wd, scale;
};

struct Table {
  uint32_t first[kTable];      // the block at which a matrix begins; behind the last: UINT32_MAX
  Matrix e[kTable];
};
static_assert(sizeof(Table) <= 3900, "a kernel's arguments");

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

template <class GT>
__device__ __forceinline__ float gradient(const Matrix& e, int64_t r, int64_t c, float factor) {
  return (float)((const GT*)e.g)[r * e.ld_g + c] * factor;
}

// m += rest (g - m); the update is m, or (nesterov) the same once more
__device__ __forceinline__ float blend(float m, float g, float rest) { return m + rest * (g - m); }

// ---- momentum and the sum of squares of each piece.  Lanes lie along a row.
template <class GT>
__global__ __launch_bounds__(NT) void momentum_kernel(Table t, Hyper h) {
  __shared__ double red[NT / 64];
  const int k = find(t, blockIdx.x);
  const Matrix& e = t.e[k];
  const uint32_t piece = blockIdx.x - t.first[k];
  const int across = (e.cols + kPiece - 1) / kPiece;
  const int64_t r0 = (int64_t)(piece / across) * kPiece, c = (int64_t)(piece % across) * kPiece + (threadIdx.x & 63);
  const float factor = h.grad_norm ? h.grad_norm[1] : 1.f;
  double s = 0;
  if (factor == factor && c < e.cols) {
    const int64_t end = min(r0 + kPiece, (int64_t)e.rows);
    for (int64_t r = r0 + (threadIdx.x >> 6); r < end; r += NT / 64) {
      float* m = e.m + r * e.ld_m + c;
      const float g = gradient<GT>(e, r, c, factor);
      const float v = blend(*m, g, h.rest);
      *m = v;
      const float u = h.nesterov ? blend(v, g, h.rest) : v;
      s += (double)u * u;
    }
  }
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

// ---- X = u / norm, transposed where there are more rows than columns, zeros in what pads it: a piece of X a block
template <class GT>
__global__ __launch_bounds__(NT) void lay_out_kernel(Table t, Hyper h) {
  __shared__ float turn[kPiece][kPiece + 1];
  const int k = find(t, blockIdx.x);
  const Matrix& e = t.e[k];
  const uint32_t piece = blockIdx.x - t.first[k];
  const int across = e.k / kPiece, lane = threadIdx.x & 63, row = threadIdx.x >> 6;
  const int64_t i0 = (int64_t)(piece / across) * kPiece, j0 = (int64_t)(piece % across) * kPiece;      // of X
  const float factor = h.grad_norm ? h.grad_norm[1] : 1.f;
  const double inv = *e.inv * kX;
  const bool tall = e.rows > e.cols;
  const int64_t r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
#pragma unroll 4
  for (int s = row; s < kPiece; s += NT / 64) {
    const int64_t r = r0 + s, c = c0 + lane;
    float v = 0.f;
    if (r < e.rows && c < e.cols) {
      v = e.m[r * e.ld_m + c];
      if (h.nesterov) v = blend(v, gradient<GT>(e, r, c, factor), h.rest);
      v = (float)(v * inv);
    }
    if (tall) {
      turn[s][lane] = v;
    } else {
      const int64_t at = (i0 + s) * e.k + j0 + lane;
      split(v, e.hi[0][at], e.lo[at]);
    }
  }
  if (!tall) return;
  __syncthreads();
#pragma unroll 4
  for (int s = row; s < kPiece; s += NT / 64) {
    const int64_t at = (i0 + s) * e.k + j0 + lane;
    split(turn[lane][s], e.hi[0][at], e.lo[at]);
  }
}

// ---- the step of the parameters: X back, transposed again
template <class PT, bool MASTER>
__global__ __launch_bounds__(NT) void apply_kernel(Table t, Hyper h, int last) {
  __shared__ float turn[kPiece][kPiece + 1];
  if (h.grad_norm && h.grad_norm[1] != h.grad_norm[1]) return;
  const int k = find(t, blockIdx.x);
  const Matrix& e = t.e[k];
  const uint32_t piece = blockIdx.x - t.first[k];
  const int across = (e.cols + kPiece - 1) / kPiece, lane = threadIdx.x & 63, row = threadIdx.x >> 6;
  const int64_t r0 = (int64_t)(piece / across) * kPiece, c0 = (int64_t)(piece % across) * kPiece;
  const float lr = h.lr_dev ? *h.lr_dev : h.lr;
  const float keep = 1.f - lr * e.wd, by = lr * e.scale * (1.f / kX);
  const f16* hi = e.hi[last];
  const bool tall = e.rows > e.cols;
  auto value = [&](int64_t at) { return (float)hi[at] + (float)e.lo[at] * (1.f / kLo); };
  if (tall) {
#pragma unroll 4
    for (int s = row; s < kPiece; s += NT / 64) turn[s][lane] = value((c0 + s) * e.k + r0 + lane);    // (X is padded to whole pieces)
    __syncthreads();
  }
  const int64_t c = c0 + lane;
  if (c >= e.cols) return;
#pragma unroll 4
  for (int s = row; s < kPiece; s += NT / 64) {
    const int64_t r = r0 + s;
    if (r >= e.rows) break;
    const float x = tall ? turn[lane][s] : value(r * e.k + c);
    PT* p = (PT*)e.p + r * e.ld_p + c;
    if constexpr (MASTER) {
      float* q = e.master + r * e.ld_master + c;
      const float v = *q * keep - by * x;
      *q = v;
      *p = (PT)v;
    } else {
      *p = (PT)((float)*p * keep - by * x);
    }
  }
}

// ---- the products.  S x S tiles, four waves of S / 2 x S / 2.  SYM_A: A = X X^T; SYM_B: B = b A + c A A^T; STEP: X = a X + B X.
enum Product { SYM_A, SYM_B, STEP };

// Blocks are dealt to the 8 XCDs round-robin.  Each XCD gets every eighth of the blocks of each matrix (which has a multiple of 8 of them) and of its tiles a row of consecutive ones, so
// that all XCDs have as many of every matrix, the largest first: -1 where there is none left.
__device__ __forceinline__ int xcd_tile(uint32_t block, int tiles) {
  const int xcd = block & 7, at = block >> 3, most = tiles >> 3, more = tiles & 7;
  return at < most + (xcd < more) ? xcd * most + min(xcd, more) + at : -1;
}

template <int S, Product P, int DEPTH>
__global__ __launch_bounds__(NT) void product_kernel(Table t, int from) {
  constexpr int W = S / 2, TB = W / 16;
  constexpr bool BKS = P == STEP;                  // X is [k, columns] there
  constexpr int RING = k64::ring_bytes<S, S, DEPTH, true>();
  __shared__ __attribute__((aligned(1024))) char ring[RING];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / 2, wn = wave % 2;
  const int which = __builtin_amdgcn_readfirstlane(find(t, blockIdx.x));
  const Matrix& e = t.e[which];
  const int tile = xcd_tile(blockIdx.x - t.first[which], P == STEP ? (e.n / S) * (e.k / S) : (e.n / S) * (e.n / S + 1) / 2);
  if (tile < 0) return;
  int ti, tj;
  if constexpr (P == STEP) {
    const int tm = e.n / S, tn = e.k / S, group = tile / (4 * tn), rows = min(tm - 4 * group, 4), in = tile - group * 4 * tn;
    ti = group * 4 + in % rows;
    tj = in / rows;
  } else {                                         // row ti of the triangle holds ti + 1 tiles
    ti = (int)((sqrtf(8.f * tile + 1.f) - 1.f) * 0.5f);
    while (ti * (ti + 1) / 2 > tile) ti--;
    while ((ti + 1) * (ti + 2) / 2 <= tile) ti++;
    tj = tile - ti * (ti + 1) / 2;
  }
  const int m0 = ti * S, n0 = tj * S;
  const f16* X = e.hi[from];
  const f16 *a, *b;
  int lda, ldb, K;
  if constexpr (P == SYM_A) { lda = ldb = K = e.k; a = X + (size_t)m0 * lda; b = X + (size_t)n0 * ldb; }
  else if constexpr (P == SYM_B) { lda = ldb = K = e.n; a = e.A + (size_t)m0 * lda; b = e.A + (size_t)n0 * ldb; }
  else { lda = K = e.n; ldb = e.k; a = e.B + (size_t)m0 * lda; b = X + n0; }
  f32x4 acc[TB][TB];
#pragma unroll
  for (int i = 0; i < TB; i++)
#pragma unroll
    for (int j = 0; j < TB; j++) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  k64::run<S, S, 2, 2, false, BKS, DEPTH, true>((const char*)a, (const char*)b, lda, ldb, 0, K, ring, acc, wave, wm, wn, lane);
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
  const int cp = lane % PPR, row0 = lane / PPR, col = n0 + wn * W + cp * 8;
#pragma unroll
  for (int tm = 0; tm < W / 32; tm++) {
    const int mbase = m0 + wm * W + tm * 32;
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
      if constexpr (P == STEP) {
        const size_t at = (size_t)(mbase + row) * e.k + col;
        const f16x8 xh = *(const f16x8*)(X + at), xl = *(const f16x8*)(e.lo + at);
        f16x8 oh, ol;
#pragma unroll
        for (int j = 0; j < 8; j++) {
          f16 hi, lo;
          split(__builtin_fmaf(kA_, (float)xh[j] + (float)xl[j] * (1.f / kLo), v[j] * (1.f / kA)), hi, lo);
          oh[j] = hi;
          ol[j] = lo;
        }
        *(f16x8*)(e.hi[from ^ 1] + at) = oh;
        *(f16x8*)(e.lo + at) = ol;
      } else {
        const size_t at = (size_t)(mbase + row) * e.n + col;
        f16x8 o;
        if constexpr (P == SYM_A) {
#pragma unroll
          for (int j = 0; j < 8; j++) o[j] = (f16)(v[j] * (kA / (kX * kX)));
        } else {
          const f16x8 x = *(const f16x8*)(e.A + at);
#pragma unroll
          for (int j = 0; j < 8; j++) o[j] = (f16)__builtin_fmaf(kB_, (float)x[j], v[j] * (kC_ / kA));
        }
        *(f16x8*)((P == SYM_A ? e.A : e.B) + at) = o;
      }
    }
    if constexpr (P != STEP) {
      if (ti != tj) {                              // the tile across the diagonal: 8 rows of a column a lane
#pragma unroll
        for (int half = 0; half < W / 64; half++)
#pragma unroll
          for (int r = 0; r < 4; r++) {
            const int c = half * 64 + lane;
            const size_t at = (size_t)(n0 + wn * W + c) * e.n + mbase + r * 8;
            f16x8 o, x = {};
            if constexpr (P == SYM_B) x = *(const f16x8*)(e.A + at);          // (A is symmetric bit for bit)
#pragma unroll
            for (int j = 0; j < 8; j++) {
              const float v = *(const float*)(strip + (r * 8 + j) * ROWB + c * 4);
              o[j] = P == SYM_A ? (f16)(v * (kA / (kX * kX))) : (f16)__builtin_fmaf(kB_, (float)x[j], v * (kC_ / kA));
            }
            *(f16x8*)((P == SYM_A ? e.A : e.B) + at) = o;
          }
      }
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(63));
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- host: matrices in groups that are worked on together
uint64_t up(uint64_t n, uint64_t to) { return (n + to - 1) / to * to; }

struct Group {
  std::vector<int> which;      // of the call's matrices
  int tile;
  std::vector<int> n, k;       // padded
  uint64_t bytes;
};

int64_t small_side(const ah_muon_matrix_t& x) { return std::min(x.rows, x.cols); }
int64_t large_side(const ah_muon_matrix_t& x) { return std::max(x.rows, x.cols); }

// 256 x 256 tiles where they are as many as two thirds of the CUs, else 128 x 128
int tile_of(const ah_muon_matrix_t* x, const std::vector<int>& which) {
  uint64_t tiles = 0;
  for (int i : which) tiles += (up(small_side(x[i]), 256) / 256) * (up(large_side(x[i]), 256) / 256);
  return tiles >= 170 ? 256 : 128;
}

struct Offsets { uint64_t hi0, hi1, lo, A, B, part, inv, end; };
Offsets offsets(const ah_muon_matrix_t& x, int n, int k, uint64_t at) {
  Offsets o;
  auto take = [&](uint64_t bytes) { const uint64_t r = at; at += up(bytes, 256); return r; };
  const uint64_t nk = (uint64_t)n * k, nn = (uint64_t)n * n;
  o.hi0 = take(2 * nk); o.hi1 = take(2 * nk); o.lo = take(2 * nk);
  o.A = take(2 * nn); o.B = take(2 * nn);
  o.part = take(8 * (up(x.rows, kPiece) / kPiece) * (up(x.cols, kPiece) / kPiece));
  o.inv = take(8);
  o.end = at;
  return o;
}

std::vector<Group> plan(const ah_muon_matrix_t* x, int n) {
  std::vector<int> order;
  for (int i = 0; i < n; i++)
    if (x[i].rows && x[i].cols) order.push_back(i);
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return x[a].rows * x[a].cols > x[b].rows * x[b].cols; });
  std::vector<Group> groups;
  uint64_t elements = 0;
  for (int i : order) {
    const uint64_t own = up(small_side(x[i]), 256) * up(large_side(x[i]), 256);
    if (groups.empty() || (int)groups.back().which.size() == kTable || elements + own > kGroupElements) {
      groups.push_back({});
      elements = 0;
    }
    groups.back().which.push_back(i);
    elements += own;
  }
  for (Group& g : groups) {
    g.tile = tile_of(x, g.which);
    g.bytes = 0;
    for (int i : g.which) {
      g.n.push_back((int)up(small_side(x[i]), g.tile));
      g.k.push_back((int)up(large_side(x[i]), g.tile));
      g.bytes = offsets(x[i], g.n.back(), g.k.back(), g.bytes).end;
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

template <int S, int DEPTH>
hipError_t products(Table& t, const Group& g, int steps, hipStream_t s) {
  auto triangle = [](const Matrix& e) { const uint64_t n = e.n / S; return up(n * (n + 1) / 2, 8); };
  auto all = [](const Matrix& e) { return up((uint64_t)(e.n / S) * (e.k / S), 8); };
  for (int i = 0; i < steps; i++) {
    hipError_t e = launch(t, g, triangle, [&](uint32_t b) { hipLaunchKernelGGL((product_kernel<S, SYM_A, DEPTH>), dim3(b), dim3(NT), 0, s, t, i & 1); });
    if (e == hipSuccess) e = launch(t, g, triangle, [&](uint32_t b) { hipLaunchKernelGGL((product_kernel<S, SYM_B, DEPTH>), dim3(b), dim3(NT), 0, s, t, i & 1); });
    if (e == hipSuccess) e = launch(t, g, all, [&](uint32_t b) { hipLaunchKernelGGL((product_kernel<S, STEP, DEPTH>), dim3(b), dim3(NT), 0, s, t, i & 1); });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t step_group(const ah_muon_t* c, const ah_muon_matrix_t* x, const Group& g, char* work, bool master, hipStream_t s) {
  Table t = {};
  uint64_t at = 0;
  for (size_t i = 0; i < g.which.size(); i++) {
    const ah_muon_matrix_t& y = x[g.which[i]];
    const Offsets o = offsets(y, g.n[i], g.k[i], at);
    Matrix& e = t.e[i];
    e.p = y.param; e.g = y.grad; e.m = y.momentum; e.master = y.master;
    e.hi[0] = (f16*)(work + o.hi0); e.hi[1] = (f16*)(work + o.hi1); e.lo = (f16*)(work + o.lo);
    e.A = (f16*)(work + o.A); e.B = (f16*)(work + o.B); e.part = (double*)(work + o.part); e.inv = (double*)(work + o.inv);
    e.ld_p = y.ld_param ? y.ld_param : y.cols; e.ld_g = y.ld_grad ? y.ld_grad : y.cols;
    e.ld_m = y.ld_momentum ? y.ld_momentum : y.cols; e.ld_master = y.ld_master ? y.ld_master : y.cols;
    e.rows = (int)y.rows; e.cols = (int)y.cols; e.n = g.n[i]; e.k = g.k[i];
    e.wd = y.weight_decay; e.scale = y.scale;
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
  if (e == hipSuccess) e = g.tile == 256 ? products<256, 2>(t, g, c->ns_steps, s) : products<128, 2>(t, g, c->ns_steps, s);
  if (e == hipSuccess)
    e = launch(t, g, pieces, [&](uint32_t b) {
      const int last = c->ns_steps & 1;
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
    for (const Group& g : plan(x, n)) *bytes = std::max(*bytes, g.bytes);
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
    for (const Group& g : plan(x, n)) {
      const hipError_t e = step_group(c, x, g, (char*)workspace, master, (hipStream_t)stream);
      if (e != hipSuccess) return hip_status(e, who);
    }
  } catch (...) {
    return set_error(AH_ENOMEM, "%s: no host memory", who);
  }
  return AH_OK;
}
