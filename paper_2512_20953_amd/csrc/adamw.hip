// Optimizer step over many tensors in few launches (declared in include/ah_ops.h): AdamW with moments in fp32 or in 8 bits, and the
// norm of all gradients.  Bound by HBM: every value is read and written once (kernels traced, called repeatedly: 100 M parameters with fp32 states and a master copy 447 us, 6.8 TB/s;
// 202 M with 8-bit states 460, 5.3 TB/s, where vector units have their 80 instructions an element to issue as well).
//
// A launch takes up to kTensors tensors, whose descriptors travel in the kernel's arguments (no copy to the device, nothing
// that a captured graph could find changed); a block takes one chunk of one tensor and finds it by counting the tensors that
// begin at or before its number.
#include "ah_ops.h"
#include "capi_util.h"
#include "common.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <type_traits>

using namespace ah;

namespace {

constexpr int NT = 256, kTensors = 48;
// Elements of a lane, and of a block.  One run of 16 bytes a lane for fp32 states (two take 651 instead of 623 us for 100 M parameters with a master copy and the norm, four
// 658); eight for states in 8 bits, of which four fill no load, twice over (724 -> 692 us for 202 M with the states' values; four times 697).
constexpr int VEC = 4, kChunk = NT * VEC, VEC8 = 8, kRuns8 = 2, kChunk8 = NT * VEC8 * kRuns8;
constexpr int kBlock = 32;                   // elements that share a scale
constexpr uint64_t kMaxElements = 1ull << 33, kMaxBlocks = kMaxElements / kChunk;   // of a tensor; of a launch (2^23: its threads are counted in 32 bits)

struct Entry {
  void* param;
  const void* grad;
  void *m, *v;
  uint8_t *ms, *vs;
  float* master;
  uint64_t n;
  uint32_t number;   // of the first element, for the random bits
  float wd;
};

struct Table {
  uint32_t first[kTensors];   // the block at which a tensor begins; behind the last tensor: UINT32_MAX
  Entry e[kTensors];
};

struct Hyper {
  float c1, c2, eps, lr;      // 1 - beta1, 1 - beta2
  float alpha, root;          // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  double log_b1, log_b2;      // natural logarithms (for step_dev)
  int64_t step;
  const float *lr_dev, *grad_norm;
  const int32_t* step_dev;
  uint32_t seed;              // (without step_dev the step's number is in it already)
  int aligned;                // every pointer of the launch allows vector access
};

__device__ __forceinline__ int find_tensor(const Table& t, uint32_t block) {
  int k = -1;
#pragma unroll
  for (int i = 0; i < kTensors; i++) k += block >= t.first[i];
  return k;
}

// ---- N consecutive values of a tensor; what lies behind its end reads as 0
// (at: the same in memory, where more than 16 bytes need not be aligned to their size)
template <class T, int N> struct Wide {
  typedef T type __attribute__((ext_vector_type(N)));
  typedef type at __attribute__((aligned(sizeof(T) * N < 16 ? sizeof(T) * N : 16)));
};

// (ONCE: past the caches, for what nobody reads again before they have been overwritten.  All that the step touches: it evicts less of the gradients that the norm has just
// read.  100 M parameters with the norm, caches overwritten before each call: 630 -> 581 us; called repeatedly 623 -> 527, as some gradients survive from call to call; the
// norm itself reads with the caches, or 553.)
template <int N, class T, bool ONCE = false>
__device__ __forceinline__ typename Wide<T, N>::type load_n(const T* p, bool whole, int left) {
  typename Wide<T, N>::type r = {};
  if (whole) {
    if constexpr (ONCE) return __builtin_nontemporal_load((const typename Wide<T, N>::at*)p);
    else return *(const typename Wide<T, N>::at*)p;
  }
#pragma unroll
  for (int j = 0; j < N; j++)
    if (j < left) r[j] = p[j];
  return r;
}
template <int N, class T, bool ONCE = false>
__device__ __forceinline__ void store_n(T* p, typename Wide<T, N>::type r, bool whole, int left) {
  if (whole) {
    if constexpr (ONCE) __builtin_nontemporal_store(r, (typename Wide<T, N>::at*)p);
    else *(typename Wide<T, N>::at*)p = r;
    return;
  }
#pragma unroll
  for (int j = 0; j < N; j++)
    if (j < left) p[j] = r[j];
}

// ---- 8-bit codes.  Seen as an fp32 number's exponent and upper mantissa bits, a code is its value times a power of two, binades,
// gradual underflow and all (fp32 underflows gradually too): decoding is a shift and an exponent add, rounding at random an integer add below the
// bits that stay.  BINS: binades of the code; the scale byte is the biased exponent of the top one.
template <int BINS>
__device__ __forceinline__ float decode(uint32_t code, int scale) {
  return __builtin_amdgcn_ldexpf(__uint_as_float(code << 20), scale - BINS);
}
// a code of 7 bits and a sign: as the shift of the signed byte, of which the sign and the 7 bits stay
__device__ __forceinline__ float decode_signed(uint32_t code, int scale) {
  return __builtin_amdgcn_ldexpf(__uint_as_float((uint32_t)((int32_t)(code << 24) >> 4) & 0x87f00000u), scale - 15);
}
// |x| to a code; rnd: 16 random bits
template <int BINS>
__device__ __forceinline__ uint32_t encode(float ax, int scale, uint32_t rnd) {
  const uint32_t u = __float_as_uint(__builtin_amdgcn_ldexpf(ax, BINS - scale));
  return (u + (rnd << 4)) >> 20;
}
// scale byte of a block whose largest magnitude has these bits; a block that is not finite gets 255
template <int BINS>
__device__ __forceinline__ int scale_of(uint32_t top) {
  const uint32_t e = (top + (BINS == 15 ? 0x200000 - 1 : 0x100000 - 1)) >> 23;   // one up from 1.75 / 1.875 times a power of two on
  return (int)min(max(e, (uint32_t)BINS + 1), 255u);
}
// the largest over the 4 lanes that hold a block of 32
static_assert(VEC8 * 4 == kBlock, "lanes of a block");
__device__ __forceinline__ uint32_t block_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));           // lanes 1 0 3 2
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));        // lanes 2 3 0 1
}
// 32 bits from the product of an element's number with an odd constant plus the seed (the constant: the prime 2654435761 of Knuth's multiplicative hashing; the shifts and
// multipliers behind it: C. Wellons, "Prospecting for Hash Functions", 2018)
constexpr uint32_t kNumber = 0x9E3779B1u;
__device__ __forceinline__ uint32_t random_bits(uint32_t x) {
  x ^= x >> 16; x *= 0x7feb352du; x ^= x >> 15; x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

// LOW: the root instruction takes a subnormal for 0; second moments that are subnormal are scaled up for it.  (States in 8 bits do so only where eps is so small that it
// matters: 202 M with the states' values 693 us with it and 684 without; those in 32 bits always, level.)
template <class P, class G, bool MASTER, bool BITS8, bool LOW>
__global__ __launch_bounds__(NT) void adamw_step_kernel(Table t, Hyper h) {
  float factor = 1.f;
  if (h.grad_norm) {
    factor = h.grad_norm[1];
    if (factor != factor) return;
  }
  float lr = h.lr, alpha = h.alpha, root = h.root;
  uint32_t seed = h.seed;
  if (h.lr_dev || h.step_dev) {
    const int64_t number = h.step_dev ? (int64_t)max(*h.step_dev, 1) : h.step;
    const double step = (double)number;
    if (h.step_dev) seed += (uint32_t)number;   // a replay rounds by other bits than the one before
    if (h.lr_dev) lr = *h.lr_dev;
    alpha = (float)((double)lr / -expm1(step * h.log_b1));
    root = (float)(1.0 / sqrt(-expm1(step * h.log_b2)));
  }
  const float root_low = root * 0x1p-16f;
  const int k = find_tensor(t, blockIdx.x);
  const Entry& e = t.e[k];
  constexpr int V = BITS8 ? VEC8 : VEC;
  typedef typename std::conditional<BITS8, uint8_t, float>::type S;
  constexpr int RUNS = BITS8 ? kRuns8 : 1;
#pragma unroll 1
  for (int run = 0; run < RUNS; run++) {
    // the lane's first element is the block's first, a scalar, and a 32-bit distance
    const uint64_t base = ((uint64_t)(blockIdx.x - t.first[k]) * RUNS + run) * (NT * V);
    if (base >= e.n) return;
    const uint32_t left = (uint32_t)min(e.n - base, (uint64_t)(NT * V)), i = threadIdx.x * V;
    const int rest = i < left ? (int)(left - i) : 0;
    const bool whole = h.aligned && rest >= V;
    const G* g = (const G*)e.grad + base;
    S *m = (S*)e.m + base, *v = (S*)e.v + base;
    P* p = (P*)e.param + base;
    float* w = MASTER ? e.master + base : nullptr;
    const float keep = 1.f - lr * e.wd;
    const auto tg = load_n<V, G, true>(g + i, whole, rest);
    const auto tm = load_n<V, S, true>(m + i, whole, rest), tv = load_n<V, S, true>(v + i, whole, rest);
    typename Wide<P, V>::type tp;
    typename Wide<float, V>::type tw;
    if constexpr (MASTER) tw = load_n<V, float, true>(w + i, whole, rest);
    else tp = load_n<V, P, true>(p + i, whole, rest);
    int sm = 0, sv = 0;
    if (BITS8 && rest) {
      sm = e.ms[(base + i) / kBlock];
      sv = e.vs[(base + i) / kBlock];
    }
    float nm[V], nv[V];
    typename Wide<float, V>::type now;
#pragma unroll
    for (int j = 0; j < V; j++) {
#pragma clang fp contract(off)
      const float gr = (float)tg[j] * factor;
      float om, ov;
      if constexpr (BITS8) {
        om = decode_signed(tm[j], sm);
        ov = decode<31>(tv[j], sv);
      } else {
        om = tm[j];
        ov = tv[j];
      }
      nm[j] = om + h.c1 * (gr - om);
      nv[j] = ov + h.c2 * (gr * gr - ov);
    }
#pragma unroll
    for (int j = 0; j < V; j++) {
      const bool low = LOW && nv[j] < FLT_MIN;
      const float denom = __builtin_fmaf(__builtin_amdgcn_sqrtf(nv[j] * (low ? 0x1p32f : 1.f)), low ? root_low : root, h.eps);
      now[j] = __builtin_fmaf(MASTER ? tw[j] : (float)tp[j], keep, -alpha * nm[j] * __builtin_amdgcn_rcpf(denom));
    }
    typename Wide<S, V>::type om, ov;
    if constexpr (BITS8) {
      uint32_t am = 0, av = 0;   // (what lies behind the tensor's end is 0 here too)
#pragma unroll
      for (int j = 0; j < V; j++) {
        am = max(am, __float_as_uint(nm[j]) & 0x7fffffffu);
        av = max(av, __float_as_uint(nv[j]) & 0x7fffffffu);
      }
      const int s1 = scale_of<15>(block_max(am)), s2 = scale_of<31>(block_max(av));
      const uint32_t first = (e.number + (uint32_t)base + i) * kNumber + seed;
#pragma unroll
      for (int j = 0; j < V; j++) {
        const uint32_t bits = random_bits(first + j * kNumber);
        const uint32_t cm = min(encode<15>(fabsf(nm[j]), s1, bits & 0xffff), 0x7eu);
        const uint32_t cv = encode<31>(nv[j], s2, bits >> 16), least = min(__float_as_uint(nv[j]), 1u);   // a v > 0 stays above 0
        om[j] = (uint8_t)(cm | (__float_as_uint(nm[j]) >> 24 & 0x80));
        ov[j] = (uint8_t)min(max(cv, least), 0xffu);
      }
      if (max(s1, s2) == 255) {   // a block that is not finite
        asm volatile("");          // (a branch, no selects)
#pragma unroll
        for (int j = 0; j < V; j++) {
          if (s1 == 255) om[j] |= 0x7f;
          if (s2 == 255) ov[j] = 0xff;
        }
      }
      if (rest && (threadIdx.x & 3) == 0) {
        e.ms[(base + i) / kBlock] = (uint8_t)s1;
        e.vs[(base + i) / kBlock] = (uint8_t)s2;
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; j++) { om[j] = nm[j]; ov[j] = nv[j]; }
    }
    store_n<V, S, true>(m + i, om, whole, rest);
    store_n<V, S, true>(v + i, ov, whole, rest);
    if constexpr (MASTER) store_n<V, float, true>(w + i, now, whole, rest);
    typename Wide<P, V>::type np;
#pragma unroll
    for (int j = 0; j < V; j++) np[j] = (P)now[j];
    store_n<V, P, true>(p + i, np, whole, rest);
  }
}

// ---- the norm of all gradients: a partial sum in fp64 for each of a fixed number of blocks, which a second launch adds up in order.  (Added up by the
// block that finishes last, a launch less: 8.8 us for 1.6 M gradients and 158 for 100 M instead of 6.4 and 120: the ordering at the end of every block flushes caches.)
constexpr int kNormReps = 8, kNormChunk = NT * VEC * kNormReps, kNormBlocks = 1024;

__device__ __forceinline__ double block_sum(double s, double* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}

template <class G>
__global__ __launch_bounds__(NT) void grad_norm_kernel(Table t, uint32_t chunks, double* __restrict__ part, int aligned) {
  __shared__ double red[NT / 64];
  double s = 0;
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int k = find_tensor(t, c);
    const Entry& e = t.e[k];
    const uint64_t at = (uint64_t)(c - t.first[k]) * kNormChunk;
    const uint32_t left = (uint32_t)min(e.n - at, (uint64_t)kNormChunk);
    const G* g = (const G*)e.grad + at;
    typename Wide<G, VEC>::type x[kNormReps];
#pragma unroll
    for (int r = 0; r < kNormReps; r++) {
      const uint32_t i = (r * NT + threadIdx.x) * VEC;
      const int rest = i < left ? (int)(left - i) : 0;
      x[r] = load_n<VEC, G>(g + i, aligned && rest >= VEC, rest);
    }
#pragma unroll
    for (int r = 0; r < kNormReps; r++)
#pragma unroll
      for (int j = 0; j < VEC; j++) {
        const double d = (double)(float)x[r][j];
        s = __builtin_fma(d, d, s);
      }
  }
  s = block_sum(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(NT) void norm_join_kernel(const double* __restrict__ part, int n, float max_norm, float* __restrict__ out) {
  __shared__ double red[NT / 64];
  double s = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += NT) s += part[i];
  s = block_sum(s, red);
  if (threadIdx.x == 0) {
    const float norm = (float)sqrt(s);
    out[0] = norm;
    out[1] = !__builtin_isfinite(norm) ? __builtin_nanf("") : max_norm > 0.f && norm > max_norm ? max_norm / norm : 1.f;
  }
}

// ---- what 8-bit states stand for
// 16 codes a lane (half a block's).  Bound by HBM: 202 M elements in 228 us, 5.4 TB/s.
constexpr int kValues = 16, kValueChunk = NT * kValues;
__global__ __launch_bounds__(NT) void state_values_kernel(Table t, int aligned) {
  const int k = find_tensor(t, blockIdx.x);
  const Entry& e = t.e[k];
  const uint64_t at = (uint64_t)(blockIdx.x - t.first[k]) * kValueChunk + threadIdx.x * kValues;
  if (at >= e.n) return;
  const int rest = (int)min(e.n - at, (uint64_t)kValues);
  const bool whole = aligned && rest == kValues;
  const auto cm = load_n<kValues, uint8_t>((const uint8_t*)e.m + at, whole, rest), cv = load_n<kValues, uint8_t>((const uint8_t*)e.v + at, whole, rest);
  const int sm = e.ms[at / kBlock], sv = e.vs[at / kBlock];
  typename Wide<bf16, kValues>::type om, ov;
#pragma unroll
  for (int j = 0; j < kValues; j++) {
    om[j] = (bf16)decode_signed(cm[j], sm);
    ov[j] = (bf16)decode<31>(cv[j], sv);
  }
  store_n<kValues, bf16>((bf16*)e.param + at, om, whole, rest);    // (the table's places for what a step writes)
  store_n<kValues, bf16>((bf16*)e.master + at, ov, whole, rest);
}

// Fills tables with the tensors that have elements and calls launch(table, blocks of `chunk` elements) for each.
template <class F>
hipError_t by_tables(const ah_adamw_tensor_t* x, int n, uint32_t chunk, void* const* m_out, void* const* v_out, const F& launch) {
  Table t;
  uint64_t number = 0, blocks = 0;
  int count = 0;
  auto flush = [&]() {
    if (count == 0) return hipSuccess;
    for (int i = count; i < kTensors; i++) t.first[i] = UINT32_MAX;
    const hipError_t e = launch(t, (uint32_t)blocks);
    count = 0;
    blocks = 0;
    return e;
  };
  for (int i = 0; i < n; i++) {
    const uint64_t need = (x[i].n + chunk - 1) / chunk;
    if (need && (count == kTensors || blocks + need > kMaxBlocks)) {
      const hipError_t e = flush();
      if (e != hipSuccess) return e;
    }
    if (need) {
      t.first[count] = (uint32_t)blocks;
      t.e[count++] = {m_out ? m_out[i] : x[i].param, x[i].grad, x[i].m, x[i].v, x[i].m_scale, x[i].v_scale,
                      v_out ? (float*)v_out[i] : x[i].master, x[i].n, (uint32_t)number, x[i].weight_decay};
      blocks += need;
    }
    number += (x[i].n + 63) / 64 * 64;
  }
  return flush();
}

// Launches that the workspace of a list's norm has room for: full tables, and some that end early for the number of their blocks (two of those
// together hold 2^36 gradients)
int norm_launches(int n) { return (n + kTensors - 1) / kTensors + 8; }

inline bool off(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

// Types of a tensor's gradients, parameters and states as bytes an element; vector access needs n of them aligned, to 16 bytes at most
struct Widths { int p, g, s; };
bool vectors(const ah_adamw_tensor_t& x, const Widths& w, int n) {
  auto bad = [&](const void* p, int width) { return off(p, std::min(n * width, 16)); };
  return !(bad(x.grad, w.g) || bad(x.param, w.p) || bad(x.m, w.s) || bad(x.v, w.s) || bad(x.master, 4));
}

// Whether the stream is being captured (the legacy default stream cannot be, nor be asked while another is)
bool captures(hipStream_t s) {
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  if (!s) return false;
  if (hipStreamIsCapturing(s, &status) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  return status != hipStreamCaptureStatusNone;
}

int check_list(const char* who, const ah_adamw_tensor_t* x, int n) {
  if (n < 0 || (n > 0 && !x)) return set_error(AH_EINVAL, "%s: bad tensor list", who);
  for (int i = 0; i < n; i++)
    if (x[i].n > kMaxElements) return set_error(AH_EUNSUPPORTED, "%s: tensor %d has %llu elements, more than 2^33", who, i, (unsigned long long)x[i].n);
  return AH_OK;
}

}  // namespace

extern "C" int ah_adamw_step(const ah_adamw_t* c, const ah_adamw_tensor_t* x, int n, void* stream) {
  discard_stale_hip_error();
  if (!c) return set_error(AH_EINVAL, "ah_adamw_step: config is NULL");
  if (c->struct_size != sizeof(ah_adamw_t)) return set_error(AH_EINVAL, "ah_adamw_step: struct_size %u != %zu", c->struct_size, sizeof(ah_adamw_t));
  if ((c->param_type != AH_BF16 && c->param_type != AH_FP32) || (c->grad_type != AH_BF16 && c->grad_type != AH_FP32))
    return set_error(AH_EINVAL, "ah_adamw_step: types must be AH_BF16 or AH_FP32");
  if (c->state_bits != 32 && c->state_bits != 8) return set_error(AH_EUNSUPPORTED, "ah_adamw_step: state_bits %d: 32 or 8", c->state_bits);
  if (!(c->lr >= 0) || !std::isfinite(c->lr) || !(c->beta1 >= 0 && c->beta1 < 1) || !(c->beta2 >= 0 && c->beta2 < 1) || !(c->eps >= 1e-37) || !std::isfinite(c->eps))
    return set_error(AH_EINVAL, "ah_adamw_step: need finite lr >= 0, betas in [0, 1) and eps >= 1e-37");
  if (c->step < 1 && !c->step_dev) return set_error(AH_EINVAL, "ah_adamw_step: step must be >= 1");
  if (off(c->lr_dev, 4) || off(c->step_dev, 4) || off(c->grad_norm, 4)) return set_error(AH_EINVAL, "ah_adamw_step: misaligned device scalar");
  if (int rc = check_list("ah_adamw_step", x, n)) return rc;
  const bool bits8 = c->state_bits == 8, p32 = c->param_type == AH_FP32, g32 = c->grad_type == AH_FP32;
  const Widths w = {p32 ? 4 : 2, g32 ? 4 : 2, bits8 ? 1 : 4};
  bool master = false, aligned = true, any = false;
  for (int i = 0; i < n; i++) {
    if (!x[i].n) continue;
    if (!x[i].param || !x[i].grad || !x[i].m || !x[i].v || (bits8 && (!x[i].m_scale || !x[i].v_scale))) return set_error(AH_EINVAL, "ah_adamw_step: tensor %d has a NULL pointer", i);
    if (off(x[i].param, w.p) || off(x[i].grad, w.g) || off(x[i].m, w.s) || off(x[i].v, w.s) || off(x[i].master, 4)) return set_error(AH_EINVAL, "ah_adamw_step: tensor %d is not aligned to its elements", i);
    if (!std::isfinite(x[i].weight_decay)) return set_error(AH_EINVAL, "ah_adamw_step: tensor %d: weight_decay is not finite", i);
    if (any && master != (x[i].master != nullptr)) return set_error(AH_EINVAL, "ah_adamw_step: either all tensors have a master copy or none");
    master = x[i].master != nullptr;
    any = true;
    aligned = aligned && vectors(x[i], w, bits8 ? VEC8 : VEC);
  }
  if (master && p32) return set_error(AH_EINVAL, "ah_adamw_step: master copies go with bf16 parameters");
  if (!any) return AH_OK;
  if (bits8 && !c->step_dev && captures((hipStream_t)stream))
    return set_error(AH_EINVAL, "ah_adamw_step: a captured step with 8-bit states needs step_dev: its replays would round by the same random bits every time");
  Hyper h = {};
  h.c1 = (float)(1 - c->beta1); h.c2 = (float)(1 - c->beta2); h.eps = (float)c->eps; h.lr = (float)c->lr;
  h.log_b1 = std::log(c->beta1); h.log_b2 = std::log(c->beta2);
  h.step = c->step;
  if (c->step >= 1) {
    h.alpha = (float)(c->lr / -std::expm1((double)c->step * h.log_b1));
    h.root = (float)(1.0 / std::sqrt(-std::expm1((double)c->step * h.log_b2)));
  }
  h.lr_dev = c->lr_dev; h.step_dev = c->step_dev; h.grad_norm = c->grad_norm; h.aligned = aligned;
  h.seed = c->seed + (c->step_dev ? 0u : (uint32_t)c->step);
  // sqrt(v) / sqrt(1 - beta2^step) for v < 2^-126 is below 2^-63 / sqrt(1 - beta2): beside an eps of 2^24 times that it is less than half a unit in the last place
  const bool low = c->eps < std::ldexp(1.0, -39) / std::sqrt(1 - c->beta2);
  const hipError_t e = by_tables(x, n, bits8 ? kChunk8 : kChunk, nullptr, nullptr, [&](const Table& t, uint32_t blocks) {
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(NT), 0, (hipStream_t)stream, t, h); };
    auto by_state = [&](auto p, auto g, auto has_master) {
      typedef decltype(p) PT;
      typedef decltype(g) GT;
      constexpr bool M = decltype(has_master)::value;
      if (bits8 && low) go(adamw_step_kernel<PT, GT, M, true, true>);
      else if (bits8) go(adamw_step_kernel<PT, GT, M, true, false>);
      else go(adamw_step_kernel<PT, GT, M, false, true>);
    };
    auto by_param = [&](auto g) {
      if (p32) by_state(float(), g, std::false_type());
      else if (master) by_state(bf16(), g, std::true_type());
      else by_state(bf16(), g, std::false_type());
    };
    if (g32) by_param(float());
    else by_param(bf16());
    return hipGetLastError();
  });
  return hip_status(e, "ah_adamw_step");
}

extern "C" int ah_grad_norm_workspace(int n_tensors, uint64_t* bytes) {
  if (!bytes || n_tensors < 0) return set_error(AH_EINVAL, "ah_grad_norm_workspace: bad argument");
  *bytes = sizeof(double) * (uint64_t)kNormBlocks * norm_launches(n_tensors);
  return AH_OK;
}

extern "C" int ah_grad_norm(const ah_adamw_tensor_t* x, int n, int grad_type, double max_norm, float* out, void* workspace, void* stream) {
  discard_stale_hip_error();
  if (!out || !workspace || off(out, 4) || off(workspace, 8)) return set_error(AH_EINVAL, "ah_grad_norm: out or workspace is NULL or misaligned");
  if (grad_type != AH_BF16 && grad_type != AH_FP32) return set_error(AH_EINVAL, "ah_grad_norm: grad_type must be AH_BF16 or AH_FP32");
  if (!(max_norm >= 0) || !std::isfinite(max_norm) || (max_norm > 0 && max_norm < FLT_MIN)) return set_error(AH_EINVAL, "ah_grad_norm: max_norm must be finite and 0 or at least 2^-126");
  max_norm = std::min(max_norm, (double)FLT_MAX);   // (no finite norm is above it)
  if (int rc = check_list("ah_grad_norm", x, n)) return rc;
  const bool g32 = grad_type == AH_FP32;
  bool aligned = true;
  for (int i = 0; i < n; i++) {
    if (!x[i].n) continue;
    if (!x[i].grad || off(x[i].grad, g32 ? 4 : 2)) return set_error(AH_EINVAL, "ah_grad_norm: gradient of tensor %d is NULL or misaligned", i);
    aligned = aligned && !off(x[i].grad, VEC * (g32 ? 4 : 2));
  }
  double* part = (double*)workspace;
  int parts = 0;
  hipError_t e = by_tables(x, n, kNormChunk, nullptr, nullptr, [&](const Table& t, uint32_t chunks) {
    const int blocks = (int)std::min<uint32_t>(chunks, kNormBlocks);
    if (parts + blocks > kNormBlocks * norm_launches(n)) return hipErrorInvalidValue;
    auto kernel = g32 ? grad_norm_kernel<float> : grad_norm_kernel<bf16>;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(NT), 0, (hipStream_t)stream, t, chunks, part + parts, (int)aligned);
    parts += blocks;
    return hipGetLastError();
  });
  if (e == hipSuccess) {
    hipLaunchKernelGGL(norm_join_kernel, dim3(1), dim3(NT), 0, (hipStream_t)stream, part, parts, (float)max_norm, out);
    e = hipGetLastError();
  }
  return hip_status(e, "ah_grad_norm");
}

extern "C" int ah_adamw_state_values(const ah_adamw_tensor_t* x, int n, void* const* m_out, void* const* v_out, void* stream) {
  discard_stale_hip_error();
  if (int rc = check_list("ah_adamw_state_values", x, n)) return rc;
  if (n > 0 && (!m_out || !v_out)) return set_error(AH_EINVAL, "ah_adamw_state_values: output lists are NULL");
  bool aligned = true;
  for (int i = 0; i < n; i++) {
    if (!x[i].n) continue;
    if (!x[i].m || !x[i].v || !x[i].m_scale || !x[i].v_scale || !m_out[i] || !v_out[i]) return set_error(AH_EINVAL, "ah_adamw_state_values: tensor %d has a NULL pointer", i);
    if (off(m_out[i], 2) || off(v_out[i], 2)) return set_error(AH_EINVAL, "ah_adamw_state_values: output %d is misaligned", i);
    aligned = aligned && !(off(x[i].m, 16) || off(x[i].v, 16) || off(m_out[i], 16) || off(v_out[i], 16));
  }
  const hipError_t e = by_tables(x, n, kValueChunk, m_out, v_out, [&](const Table& t, uint32_t blocks) {
    hipLaunchKernelGGL(state_values_kernel, dim3(blocks), dim3(NT), 0, (hipStream_t)stream, t, (int)aligned);
    return hipGetLastError();
  });
  return hip_status(e, "ah_adamw_state_values");
}
