// Loss of rows of logits and, in the same pass, their gradient (declared in include/ah_ops.h).  Bound by HBM: every logit read once and its gradient
// written once; a row stays in the registers of a wave or a block between the two (8190 x 50257: 331 us, 5.0 TB/s; a vocabulary above about 131000, or 65500 in fp32, is read twice).
//
// Pieces of 16 bytes are counted from the 16-byte boundary before the row's first element, so that rows that begin anywhere (an odd vocabulary) are still read and written
// in whole pieces, but for the first and the last one.
#include "ah_ops.h"
#include "capi_util.h"
#include "wide.h"

#include <algorithm>
#include <cmath>

using namespace ah;

namespace {

constexpr int kMaxRows = 1 << 25, kMaxVocab = 1 << 24;
constexpr float kLog2e = 1.4426950408889634f;

struct LossArgs {
  const void *logits, *targets;
  void* grad;
  float* loss;
  const float* scale_dev;
  size_t ld_z, ld_g;
  int T, V, bits;
  float scale;
};

// exp(z - m), the difference first: both may be as large as the type allows (a row masked by its lowest value)
__device__ __forceinline__ float exp_from(float z, float m) { return __builtin_amdgcn_exp2f((z - m) * kLog2e); }
// What exponents are taken from: the maximum, or 0 where that is -infinity (nothing but zeros then)
__device__ __forceinline__ float anchor(float m) { return m == -INFINITY ? 0.f : m; }

// A row's maximum (its anchor) and the sum of exp(z - that), from the lanes of a wave's
struct Stat { float m, s; };
template <int NTH>
__device__ __forceinline__ Stat block_stat(float m, float s, float (&lds)[2][16]) {
  if constexpr (NTH > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) { lds[0][wave] = m; lds[1][wave] = s; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NTH / 64; w++) m = fmaxf(m, lds[0][w]);
    s = 0.f;
#pragma unroll
    for (int w = 0; w < NTH / 64; w++) s += lds[1][w] * exp_from(lds[0][w], anchor(m));
    __syncthreads();        // (the next row writes there)
  }
  return {anchor(m), s};
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// The gradient of elements first .. first + E - 1 of a row (what lies outside it is left) from their exponentials; `hit`: the target's place among them
template <class T, int E>
__device__ __forceinline__ void put_grad(T* row, int first, int V, const float (&e)[E], float factor, float scale, int hit, bool whole) {
  wide_t<T, E> o;
#pragma unroll
  for (int j = 0; j < E; j++) o[j] = (T)(e[j] * factor);
  if ((unsigned)hit < (unsigned)E) {
#pragma unroll
    for (int j = 0; j < E; j++)
      if (j == hit) o[j] = (T)__builtin_fmaf(e[j], factor, -scale);
  }
  if (whole) {
    store_wide<E>(row + first, o);
  } else {
#pragma unroll
    for (int j = 0; j < E; j++)
      if ((unsigned)(first + j) < (unsigned)V) row[first + j] = o[j];
  }
}

// All of a row's gradient set to one value
template <class T, int NTH>
__device__ __forceinline__ void fill_row(T* row, int V, float v) {
  for (int c = threadIdx.x; c < V; c += NTH) row[c] = (T)v;
}

// CH pieces of E elements a lane: NTH * CH pieces hold a row.  CH = 0: a row of any length, read twice.
template <class T, int NTH, int CH>
__global__ __launch_bounds__(NTH) void cross_entropy_kernel(LossArgs a) {
  constexpr int E = 16 / sizeof(T);
  __shared__ float lds[2][16];
  const float scale = a.scale_dev ? *a.scale_dev : a.scale;
  for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
    const int64_t target = load_index(a.targets, t, a.bits);
    const T* z = (const T*)a.logits + (size_t)t * a.ld_z;
    T* g = a.grad ? (T*)a.grad + (size_t)t * a.ld_g : nullptr;
    if ((uint64_t)target >= (uint64_t)a.V) {           // none, or no token at all
      const float v = target == -1 ? 0.f : __builtin_nanf("");
      if (threadIdx.x == 0) a.loss[t] = v;
      if (g) fill_row<T, NTH>(g, a.V, v);
      continue;
    }
    const float hit_z = (float)z[target];
    const int lead = (int)(((uintptr_t)z & 15) / sizeof(T));         // elements between the boundary and the row
    const bool aligned = g && (((uintptr_t)g ^ (uintptr_t)z) & 15) == 0;
    const int pieces = (lead + a.V + E - 1) / E;
    auto load = [&](int piece) {
      wide_t<T, E> r;
      const int first = piece * E - lead;
      if (first >= 0 && first + E <= a.V) return load_wide<E>(z + first);
#pragma unroll
      for (int j = 0; j < E; j++) r[j] = (unsigned)(first + j) < (unsigned)a.V ? z[first + j] : (T)-INFINITY;
      return r;
    };
    auto store = [&](int piece, const wide_t<T, E>& r, float m, float factor) {
      const int first = piece * E - lead;
      float e[E];
#pragma unroll
      for (int j = 0; j < E; j++) e[j] = exp_from((float)r[j], m);
      put_grad<T, E>(g, first, a.V, e, factor, scale, (int)target - first, aligned && first >= 0 && first + E <= a.V);
    };
    float m = -INFINITY, s = 0.f;
    Stat all;
    if constexpr (CH > 0) {
      wide_t<T, E> r[CH];
#pragma unroll
      for (int i = 0; i < CH; i++) {
        const int piece = i * NTH + threadIdx.x;
        if (piece < pieces) r[i] = load(piece);
      }
#pragma unroll
      for (int i = 0; i < CH; i++)
        if (i * NTH + (int)threadIdx.x < pieces) {
#pragma unroll
          for (int j = 0; j < E; j++) m = fmaxf(m, (float)r[i][j]);
        }
      m = wave_max(m);
#pragma unroll
      for (int i = 0; i < CH; i++)
        if (i * NTH + (int)threadIdx.x < pieces) {
#pragma unroll
          for (int j = 0; j < E; j++) s += exp_from((float)r[i][j], anchor(m));
        }
      all = block_stat<NTH>(m, wave_sum(s), lds);
      if (g) {
        const float factor = scale / all.s;
#pragma unroll
        for (int i = 0; i < CH; i++)
          if (i * NTH + (int)threadIdx.x < pieces) store(i * NTH + threadIdx.x, r[i], all.m, factor);
      }
    } else {
      for (int piece = threadIdx.x; piece < pieces; piece += NTH) {
        const wide_t<T, E> r = load(piece);
        const float before = m;
#pragma unroll
        for (int j = 0; j < E; j++) m = fmaxf(m, (float)r[j]);
        s *= exp_from(before, anchor(m));                     // (nothing seen yet: 0 * 0)
#pragma unroll
        for (int j = 0; j < E; j++) s += exp_from((float)r[j], anchor(m));
      }
      const float top = wave_max(m);
      all = block_stat<NTH>(top, wave_sum(s * exp_from(m, anchor(top))), lds);
      if (g)
        for (int piece = threadIdx.x; piece < pieces; piece += NTH) store(piece, load(piece), all.m, scale / all.s);
    }
    if (threadIdx.x == 0) a.loss[t] = (all.m - hit_z) + logf(all.s);
  }
}

template <class T>
hipError_t run(const LossArgs& a, hipStream_t s) {
  const int pieces = a.V / (16 / (int)sizeof(T)) + 2;       // of a row, at most
  const int blocks = std::min(a.T, 1 << 21);
  auto go = [&](auto lanes, auto ch) {
    constexpr int NTH = decltype(lanes)::value, CH = decltype(ch)::value;
    hipLaunchKernelGGL((cross_entropy_kernel<T, NTH, CH>), dim3(blocks), dim3(NTH), 0, s, a);
  };
#define AH_N(x) std::integral_constant<int, x>()
  if (pieces <= 64 * 2) go(AH_N(64), AH_N(2));
  else if (pieces <= 64 * 8) go(AH_N(64), AH_N(8));
  else if (pieces <= 256 * 4) go(AH_N(256), AH_N(4));
  else if (pieces <= 256 * 8) go(AH_N(256), AH_N(8));
  else if (pieces <= 1024 * 4) go(AH_N(1024), AH_N(4));
  else if (pieces <= 1024 * 8) go(AH_N(1024), AH_N(8));
  else if (pieces <= 1024 * 16) go(AH_N(1024), AH_N(16));
  else go(AH_N(1024), AH_N(0));
#undef AH_N
  return hipGetLastError();
}

}  // namespace

extern "C" int ah_cross_entropy(const ah_cross_entropy_t* c, const void* logits, const void* targets, float* loss, void* d_logits, void* stream) {
  discard_stale_hip_error();
  const char* who = "ah_cross_entropy";
  if (!c) return set_error(AH_EINVAL, "%s: config is NULL", who);
  if (c->struct_size != sizeof(ah_cross_entropy_t)) return set_error(AH_EINVAL, "%s: struct_size %u != %zu", who, c->struct_size, sizeof(ah_cross_entropy_t));
  if (c->rows < 0 || c->vocab < 1) return set_error(AH_EINVAL, "%s: need rows >= 0 and vocab >= 1", who);
  if (c->rows > kMaxRows || c->vocab > kMaxVocab) return set_error(AH_EUNSUPPORTED, "%s: more than 2^25 rows or a vocabulary of 2^24", who);
  if (c->act_type != AH_BF16 && c->act_type != AH_FP32) return set_error(AH_EINVAL, "%s: act_type must be AH_BF16 or AH_FP32", who);
  if (c->target_bits != 32 && c->target_bits != 64) return set_error(AH_EINVAL, "%s: target_bits %d: 32 or 64", who, c->target_bits);
  if (!std::isfinite(c->scale)) return set_error(AH_EINVAL, "%s: scale is not finite", who);
  if (!aligned_to(c->scale_dev, 4)) return set_error(AH_EINVAL, "%s: scale_dev is misaligned", who);
  for (int64_t ld : {c->ld_logits, c->ld_grad})
    if (ld != 0 && (ld < c->vocab || ld > (1ll << 31))) return set_error(AH_EINVAL, "%s: a row stride must be at least the vocabulary, %d, and at most 2^31", who, c->vocab);
  if (c->rows == 0) return AH_OK;
  const int ab = c->act_type == AH_FP32 ? 4 : 2;
  if (!logits || !targets || !loss || !aligned_to(logits, ab) || !aligned_to(targets, c->target_bits / 8) || !aligned_to(loss, 4) || !aligned_to(d_logits, ab))
    return set_error(AH_EINVAL, "%s: logits, targets or loss is NULL, or one of them or d_logits misaligned", who);
  LossArgs a = {};
  a.logits = logits; a.targets = targets; a.grad = d_logits; a.loss = loss; a.scale_dev = c->scale_dev; a.scale = c->scale;
  a.ld_z = c->ld_logits ? c->ld_logits : c->vocab; a.ld_g = c->ld_grad ? c->ld_grad : c->vocab;
  a.T = c->rows; a.V = c->vocab; a.bits = c->target_bits;
  if (d_logits == logits && a.T > 1 && a.ld_z != a.ld_g) return set_error(AH_EINVAL, "%s: d_logits in the place of logits needs their row stride", who);
  return hip_status(ab == 4 ? run<float>(a, (hipStream_t)stream) : run<bf16>(a, (hipStream_t)stream), who);
}
