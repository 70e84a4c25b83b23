// Layer norm (with or without the mean) of rows of any width, forward and backward (declared in include/ah_ops.h).  Bound by HBM: x read and y written once (8192 x 4096: 28 us,
// 4.7 TB/s); backward x and dy read, dx written, and the partial sums behind the gradients of gain and bias (4096 x 4096: 30 us, 3.3 TB/s, of which about 10 do not depend on the
// number of rows: first loads, 8 MB of partial sums, their fold; 32768 x 4096: 4.2 TB/s).
//
// A row stays in the registers of a wave or of a block from its load to its result.  Sums over a row: forward the mean, then the squares around it; backward the sums of x and of
// w = dy gain, then of (x - mean)^2 and of w (x - mean), from which all that dx needs follows:
//   n = (x - mean) r;  dx = r (w - mean(w) - n mean(w n)).
//
// The norms inside a layer are those of rowwise.hip: bf16 rows of whole 16-byte pieces, joined with the residual sum in front of them and the residual's gradient behind.  The two share no code; the
// formula, eps inside the root and gradients in fp32 are what they have in common, and each is tested against 64 bits by itself.
#include "ah_ops.h"
#include "capi_util.h"
#include "wide.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

using namespace ah;

namespace {

constexpr int kMaxRows = 1 << 25, kMaxWidth = 16384, kMaxBlocks = 256, kFwdBlocks = 2048;   // backward: of 1024 lanes, each with a row of partial sums; forward: of 256

struct NormArgs {
  const void *x, *dy, *gain, *bias;
  void* out;
  float* part;                 // [blocks][2][width]
  size_t ld_x, ld_y, ld_out;
  int T, width, params16;      // params16: gain and bias can be read in whole pieces
  float eps, inv;              // inv: 1 / width
};

// Sums of two values over the lanes of a row: NTH = 64: of a wave, else of the row's waves of a block.  `slot` alternates, so that a wave that is ahead does not
// write where another one still reads.
template <int NTH>
__device__ __forceinline__ void row_sums(float& a, float& b, float (&lds)[2][2][16], int slot) {
  a = wave_sum(a);
  b = wave_sum(b);
  if constexpr (NTH > 64) {
    const int wave = threadIdx.x >> 6, first = wave / (NTH / 64) * (NTH / 64);
    if ((threadIdx.x & 63) == 0) { lds[slot][0][wave] = a; lds[slot][1][wave] = b; }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < NTH / 64; w++) { a += lds[slot][0][first + w]; b += lds[slot][1][first + w]; }
  }
}

// NTH lanes to a row, of which each holds CH pieces of V elements; forward in blocks of at least 256 lanes, backward of 1024
template <int NTH> constexpr int block_of() { return NTH < 256 ? 256 : NTH; }
constexpr int kBwdThreads = 1024;

// Gain or bias of the lane's columns, kept as they lie in memory; NULL: `none` in all of them.  W: in whole pieces (V elements, 16-byte aligned)
template <class PT, int V, int NTH, int CH>
__device__ __forceinline__ void load_param(wide_t<PT, V> (&r)[CH], const void* p, float none, int lane, int width, bool whole) {
#pragma unroll
  for (int i = 0; i < CH; i++) {
    const int c = (i * NTH + lane) * V;
#pragma unroll
    for (int j = 0; j < V; j++) r[i][j] = (PT)none;
    if (!p || c >= width) continue;
    if (whole) {
      r[i] = load_wide<V>((const PT*)p + c);
    } else {
#pragma unroll
      for (int j = 0; j < V; j++) r[i][j] = ((const PT*)p)[c + j];
    }
  }
}

template <class T, int V, int NTH, int CH>
__device__ __forceinline__ void load_row(wide_t<T, V> (&r)[CH], const T* p, int lane, int width) {
#pragma unroll
  for (int i = 0; i < CH; i++) {
    const int c = (i * NTH + lane) * V;
    if (c < width) r[i] = load_wide<V>(p + c);
  }
}

// A block takes rows gridDim apart and asks for the next one's elements before it works on the present one's.
template <class T, class PT, int V, int NTH, int CH, bool RMS>
__global__ __launch_bounds__(block_of<NTH>()) void layer_norm_fwd_kernel(NormArgs a) {
  __shared__ float lds[2][2][16];
  constexpr int ROWS = block_of<NTH>() / NTH;
  const int lane = threadIdx.x % NTH;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / NTH;
  if (t >= a.T) return;          // (all lanes of a row, which is a block's only one where they meet in LDS)
  wide_t<PT, V> gain[CH], bias[CH];
  load_param<PT, V, NTH, CH>(gain, a.gain, 1.f, lane, a.width, a.params16);
  load_param<PT, V, NTH, CH>(bias, a.bias, 0.f, lane, a.width, a.params16);
  wide_t<T, V> x[CH], next[CH];
  load_row<T, V, NTH, CH>(next, (const T*)a.x + (size_t)t * a.ld_x, lane, a.width);
  for (; t < a.T; t += step) {
#pragma unroll
    for (int i = 0; i < CH; i++) x[i] = next[i];
    if (t + step < a.T) load_row<T, V, NTH, CH>(next, (const T*)a.x + (size_t)(t + step) * a.ld_x, lane, a.width);
    float mean = 0.f, none = 0.f;
    if constexpr (!RMS) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < CH; i++)
        if ((i * NTH + lane) * V < a.width) {
#pragma unroll
          for (int j = 0; j < V; j++) sum += (float)x[i][j];
        }
      row_sums<NTH>(sum, none, lds, 0);
      mean = sum * a.inv;
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < CH; i++)
      if ((i * NTH + lane) * V < a.width) {
#pragma unroll
        for (int j = 0; j < V; j++) { const float d = (float)x[i][j] - mean; ss = __builtin_fmaf(d, d, ss); }
      }
    row_sums<NTH>(ss, none, lds, 1);
    if constexpr (NTH > 64 && RMS) __syncthreads();     // (the one slot is written again in the next row)
    const float r = rsqrtf(ss * a.inv + a.eps);
    T* y = (T*)a.out + (size_t)t * a.ld_out;
#pragma unroll
    for (int i = 0; i < CH; i++) {
      const int c = (i * NTH + lane) * V;
      if (c < a.width) {
        wide_t<T, V> o;
#pragma unroll
        for (int j = 0; j < V; j++) o[j] = (T)__builtin_fmaf(((float)x[i][j] - mean) * r, (float)gain[i][j], (float)bias[i][j]);
        store_wide<V>(y + c, o);
      }
    }
  }
}

template <class T, class PT, int V, int NTH, int CH, bool RMS>
__global__ __launch_bounds__(kBwdThreads) void layer_norm_bwd_kernel(NormArgs a) {
  __shared__ float lds[2][2][16];
  constexpr int ROWS = kBwdThreads / NTH, COLS = NTH * CH * V;
  const int lane = threadIdx.x % NTH;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  wide_t<PT, V> gain[CH];
  load_param<PT, V, NTH, CH>(gain, a.gain, 1.f, lane, a.width, a.params16);
  float dg[CH][V], db[CH][V];
#pragma unroll
  for (int i = 0; i < CH; i++)
#pragma unroll
    for (int j = 0; j < V; j++) dg[i][j] = db[i][j] = 0.f;
  constexpr bool AHEAD = CH * V <= 8;       // (16 elements a lane leave no room for the next row in its 128 registers)
  wide_t<T, V> x[CH], y[CH], next_x[CH], next_y[CH];
  const int row = threadIdx.x / NTH;
  auto ask = [&](int64_t at) {
#pragma unroll
    for (int i = 0; i < CH; i++) next_x[i] = next_y[i] = wide_t<T, V>{};
    if (at >= a.T) return;
    load_row<T, V, NTH, CH>(next_x, (const T*)a.x + (size_t)at * a.ld_x, lane, a.width);
    load_row<T, V, NTH, CH>(next_y, (const T*)a.dy + (size_t)at * a.ld_y, lane, a.width);
  };
  int64_t t0 = (int64_t)blockIdx.x * ROWS;
  if (AHEAD) ask(t0 + row);
  for (; t0 < a.T; t0 += step) {            // (all rows of a block together; one behind the last has zeros)
    const int64_t t = t0 + row;
    if (!AHEAD) ask(t);
#pragma unroll
    for (int i = 0; i < CH; i++) { x[i] = next_x[i]; y[i] = next_y[i]; }
    if (AHEAD) ask(t + step);
    float mean = 0.f, mean_w = 0.f;
    if constexpr (!RMS) {
      float sx = 0.f, sw = 0.f;
#pragma unroll
      for (int i = 0; i < CH; i++)
        if ((i * NTH + lane) * V < a.width) {
#pragma unroll
          for (int j = 0; j < V; j++) { sx += (float)x[i][j]; sw = __builtin_fmaf((float)y[i][j], (float)gain[i][j], sw); }
        }
      row_sums<NTH>(sx, sw, lds, 0);
      mean = sx * a.inv;
      mean_w = sw * a.inv;
    }
    float ss = 0.f, sd = 0.f;
#pragma unroll
    for (int i = 0; i < CH; i++)
      if ((i * NTH + lane) * V < a.width) {
#pragma unroll
        for (int j = 0; j < V; j++) {
          const float d = (float)x[i][j] - mean;
          ss = __builtin_fmaf(d, d, ss);
          sd = __builtin_fmaf(d, (float)y[i][j] * (float)gain[i][j], sd);
        }
      }
    row_sums<NTH>(ss, sd, lds, 1);
    if constexpr (NTH > 64 && RMS) __syncthreads();
    const float r = rsqrtf(ss * a.inv + a.eps), k = sd * a.inv * r * r;     // n mean(w n) = (x - mean) k
    T* dx = (T*)a.out + (size_t)t * a.ld_out;
#pragma unroll
    for (int i = 0; i < CH; i++) {
      const int c = (i * NTH + lane) * V;
      if (c < a.width) {
        wide_t<T, V> o;
#pragma unroll
        for (int j = 0; j < V; j++) {
          const float d = (float)x[i][j] - mean, g = (float)y[i][j];
          dg[i][j] = __builtin_fmaf(g, d * r, dg[i][j]);
          db[i][j] += g;
          o[j] = (T)(r * (g * (float)gain[i][j] - mean_w - d * k));
        }
        if (t < a.T) store_wide<V>(dx + c, o);
      }
    }
  }
  // the block's rows of partial sums meet in LDS, half of them giving theirs to the other half
  float* part = a.part + (size_t)blockIdx.x * 2 * a.width;
  if constexpr (ROWS > 1) {
    __shared__ float red[ROWS / 2][2][COLS];
#pragma unroll
    for (int half = ROWS / 2; half > 0; half /= 2) {
      if (row >= half && row < 2 * half) {
#pragma unroll
        for (int i = 0; i < CH; i++) {
          const int c = (i * NTH + lane) * V;
          wide_t<float, V> u, v;
#pragma unroll
          for (int j = 0; j < V; j++) { u[j] = dg[i][j]; v[j] = db[i][j]; }
          store_wide<V>(&red[row - half][0][c], u);
          store_wide<V>(&red[row - half][1][c], v);
        }
      }
      __syncthreads();
      if (row < half) {
#pragma unroll
        for (int i = 0; i < CH; i++) {
          const int c = (i * NTH + lane) * V;
          const wide_t<float, V> u = load_wide<V>((const float*)&red[row][0][c]), v = load_wide<V>((const float*)&red[row][1][c]);
#pragma unroll
          for (int j = 0; j < V; j++) { dg[i][j] += u[j]; db[i][j] += v[j]; }
        }
      }
      __syncthreads();
    }
  }
  if (row > 0) return;
#pragma unroll
  for (int i = 0; i < CH; i++) {
    const int c = (i * NTH + lane) * V;
    if (c < a.width) {
      wide_t<float, V> u, v;
#pragma unroll
      for (int j = 0; j < V; j++) { u[j] = dg[i][j]; v[j] = db[i][j]; }
      store_wide<V>(part + c, u);
      store_wide<V>(part + a.width + c, v);
    }
  }
}

// d[c] = beta * d[c] + the sum of part[b][which][c] over the blocks: 32 columns a block, every 32nd row half a wave
constexpr int kFoldCols = 32, kFoldThreads = 1024, kFoldRows = kFoldThreads / kFoldCols;
__global__ __launch_bounds__(kFoldThreads) void norm_fold_kernel(const float* part, int blocks, int width, float* d_gain, float* d_bias, int beta) {
  __shared__ float red[kFoldRows][kFoldCols];
  float* d = blockIdx.y ? d_bias : d_gain;
  if (!d) return;
  const int col = threadIdx.x % kFoldCols, c = blockIdx.x * kFoldCols + col, row = threadIdx.x / kFoldCols;
  float s = 0.f;
  if (c < width) {
    const float* p = part + (size_t)blockIdx.y * width + c;
#pragma unroll 8
    for (int b = row; b < blocks; b += kFoldRows) s += p[(size_t)b * 2 * width];
  }
  red[row][col] = s;
  __syncthreads();
  if (row == 0 && c < width) {
#pragma unroll
    for (int w = 1; w < kFoldRows; w++) s += red[w][col];
    d[c] = beta ? d[c] + s : s;
  }
}

int check_sizes(const char* who, const ah_layer_norm_t* c) {
  if (!c) return set_error(AH_EINVAL, "%s: config is NULL", who);
  if (c->struct_size != sizeof(ah_layer_norm_t)) return set_error(AH_EINVAL, "%s: struct_size %u != %zu", who, c->struct_size, sizeof(ah_layer_norm_t));
  if (c->rows < 0 || c->width < 1) return set_error(AH_EINVAL, "%s: need rows >= 0 and width >= 1", who);
  if (c->rows > kMaxRows || c->width > kMaxWidth) return set_error(AH_EUNSUPPORTED, "%s: more than 2^25 rows or a width of 16384", who);
  return AH_OK;
}

int check(const char* who, const ah_layer_norm_t* c) {
  if (int rc = check_sizes(who, c)) return rc;
  if ((c->act_type != AH_BF16 && c->act_type != AH_FP32) || (c->param_type != AH_BF16 && c->param_type != AH_FP32))
    return set_error(AH_EINVAL, "%s: types must be AH_BF16 or AH_FP32", who);
  if (c->rms != 0 && c->rms != 1) return set_error(AH_EINVAL, "%s: rms must be 0 or 1", who);
  if (!(c->eps >= FLT_MIN) || !std::isfinite(c->eps)) return set_error(AH_EINVAL, "%s: eps must be finite and at least 2^-126", who);
  const int pb = c->param_type == AH_FP32 ? 4 : 2;
  if (!aligned_to(c->gain, pb) || !aligned_to(c->bias, pb)) return set_error(AH_EINVAL, "%s: gain or bias is misaligned", who);
  for (int64_t ld : {c->ld_x, c->ld_y, c->ld_dx})
    if (ld != 0 && (ld < c->width || ld > (1ll << 31))) return set_error(AH_EINVAL, "%s: a row stride must be at least the width, %d, and at most 2^31", who, c->width);
  return AH_OK;
}

NormArgs args(const ah_layer_norm_t* c, const void* x, const void* dy, void* out, int64_t ld_out, float* part) {
  NormArgs a = {};
  a.x = x; a.dy = dy; a.out = out; a.gain = c->gain; a.bias = c->bias; a.part = part;
  a.ld_x = c->ld_x ? c->ld_x : c->width; a.ld_y = c->ld_y ? c->ld_y : c->width; a.ld_out = ld_out ? ld_out : c->width;
  a.T = c->rows; a.width = c->width; a.params16 = aligned_to(c->gain, 16) && aligned_to(c->bias, 16); a.eps = c->eps; a.inv = 1.f / c->width;
  return a;
}

// Lanes to a row and pieces of V elements a lane, as constants: forward 8 or 16 elements a lane, backward 8 up to the widest rows (4096 x 4096 in bf16: 32 us, and 36 with a row
// of 64 elements a lane in one wave, which waits for no other).
template <bool BWD, int V, class F>
void by_width(int width, const F& go) {
  auto with = [&](auto lanes, auto elements) { go(lanes, std::integral_constant<int, decltype(elements)::value / V>()); };
#define AH_N(x) std::integral_constant<int, x>()
  if (width <= 512) with(AH_N(64), AH_N(8));
  else if (width <= 1024) { if constexpr (BWD) with(AH_N(128), AH_N(8)); else with(AH_N(64), AH_N(16)); }
  else if (width <= 2048) with(AH_N(256), AH_N(8));
  else if (width <= 4096) { if constexpr (BWD) with(AH_N(512), AH_N(8)); else with(AH_N(256), AH_N(16)); }
  else if (width <= 8192) with(AH_N(1024), AH_N(8));
  else with(AH_N(1024), AH_N(16));
#undef AH_N
}

int fwd_rows(int width) { return width <= 1024 ? 4 : 1; }        // of a block
int bwd_blocks(const ah_layer_norm_t* c) {
  int lanes = 64;
  while (lanes < 1024 && lanes * 8 < c->width) lanes *= 2;
  const int rows = kBwdThreads / lanes;
  return std::max(1, std::min(kMaxBlocks, (c->rows + rows - 1) / rows));
}

template <bool BWD>
hipError_t run(const NormArgs& a, const ah_layer_norm_t* c, bool wide, int blocks, hipStream_t s) {
  auto typed = [&](auto t, auto p, auto v, auto r) {
    typedef decltype(t) T;
    typedef decltype(p) PT;
    constexpr int V = decltype(v)::value;
    constexpr bool RMS = decltype(r)::value;
    by_width<BWD, V>(a.width, [&](auto lanes, auto pieces) {
      constexpr int NTH = decltype(lanes)::value, CH = decltype(pieces)::value;
      if constexpr (BWD) hipLaunchKernelGGL((layer_norm_bwd_kernel<T, PT, V, NTH, CH, RMS>), dim3(blocks), dim3(kBwdThreads), 0, s, a);
      else hipLaunchKernelGGL((layer_norm_fwd_kernel<T, PT, V, NTH, CH, RMS>), dim3(blocks), dim3(block_of<NTH>()), 0, s, a);
    });
  };
  auto by_kind = [&](auto t, auto p, auto v) {
    if (c->rms) typed(t, p, v, std::true_type());
    else typed(t, p, v, std::false_type());
  };
  auto by_align = [&](auto t, auto p) {
    if (wide) by_kind(t, p, std::integral_constant<int, 8>());
    else by_kind(t, p, std::integral_constant<int, 1>());
  };
  auto by_param = [&](auto t) {
    if (c->param_type == AH_FP32) by_align(t, float());
    else by_align(t, bf16());
  };
  if (c->act_type == AH_FP32) by_param(float());
  else by_param(bf16());
  return hipGetLastError();
}

// Results in the place of what a call reads: row for row only
bool shifted(const void* in, size_t ld_in, const NormArgs& a) { return a.out == in && a.T > 1 && ld_in != a.ld_out; }

}  // namespace

extern "C" int ah_layer_norm_fwd(const ah_layer_norm_t* c, const void* x, void* y, void* stream) {
  discard_stale_hip_error();
  if (int rc = check("ah_layer_norm_fwd", c)) return rc;
  if (c->rows == 0) return AH_OK;
  const int ab = c->act_type == AH_FP32 ? 4 : 2;
  if (!x || !y || !aligned_to(x, ab) || !aligned_to(y, ab)) return set_error(AH_EINVAL, "ah_layer_norm_fwd: x or y is NULL or misaligned");
  const NormArgs a = args(c, x, nullptr, y, c->ld_y, nullptr);
  if (shifted(x, a.ld_x, a)) return set_error(AH_EINVAL, "ah_layer_norm_fwd: y in the place of x needs x's row stride");
  const bool wide = c->width % 8 == 0 && rows16(x, a.ld_x, ab) && rows16(y, a.ld_out, ab);
  const int rows = fwd_rows(c->width), block = c->width > 4096 ? 1024 : 256;
  return hip_status(run<false>(a, c, wide, std::min((c->rows + rows - 1) / rows, kFwdBlocks * 256 / block), (hipStream_t)stream), "ah_layer_norm_fwd");
}

extern "C" int ah_layer_norm_bwd_workspace(const ah_layer_norm_t* c, uint64_t* bytes) {
  if (!bytes) return set_error(AH_EINVAL, "ah_layer_norm_bwd_workspace: bytes is NULL");
  if (int rc = check_sizes("ah_layer_norm_bwd_workspace", c)) return rc;
  *bytes = (uint64_t)bwd_blocks(c) * 2 * c->width * sizeof(float);
  return AH_OK;
}

extern "C" int ah_layer_norm_bwd(const ah_layer_norm_t* c, const void* x, const void* dy, void* dx, float* d_gain, float* d_bias, int beta, void* workspace, void* stream) {
  discard_stale_hip_error();
  if (int rc = check("ah_layer_norm_bwd", c)) return rc;
  if (beta != 0 && beta != 1) return set_error(AH_EINVAL, "ah_layer_norm_bwd: beta must be 0 or 1");
  const int ab = c->act_type == AH_FP32 ? 4 : 2;
  if (!workspace || !aligned_to(workspace, 16) || !aligned_to(d_gain, 4) || !aligned_to(d_bias, 4))
    return set_error(AH_EINVAL, "ah_layer_norm_bwd: the workspace is NULL or it or a gradient is misaligned");
  if (c->rows && (!x || !dy || !dx || !aligned_to(x, ab) || !aligned_to(dy, ab) || !aligned_to(dx, ab))) return set_error(AH_EINVAL, "ah_layer_norm_bwd: x, dy or dx is NULL or misaligned");
  const NormArgs a = args(c, x, dy, dx, c->ld_dx, (float*)workspace);
  if (shifted(x, a.ld_x, a) || shifted(dy, a.ld_y, a)) return set_error(AH_EINVAL, "ah_layer_norm_bwd: dx in the place of x or dy needs its row stride");
  const bool wide = c->width % 8 == 0 && rows16(x, a.ld_x, ab) && rows16(dy, a.ld_y, ab) && rows16(dx, a.ld_out, ab);
  const int blocks = bwd_blocks(c);
  hipError_t e = run<true>(a, c, wide, blocks, (hipStream_t)stream);      // (no rows: writes zeros)
  if (e == hipSuccess && (d_gain || d_bias)) {
    hipLaunchKernelGGL(norm_fold_kernel, dim3((c->width + kFoldCols - 1) / kFoldCols, 2), dim3(kFoldThreads), 0, (hipStream_t)stream, a.part, blocks, c->width, d_gain, d_bias, beta);
    e = hipGetLastError();
  }
  return hip_status(e, "ah_layer_norm_bwd");
}
