// RMS norm of every query and key head with the position rotation in the same pass, forward and backward (declared in
// include/ah_ops.h).  Bound by HBM: x read and y written once; backward x and dy read, dx written.  4096 tokens x 64 heads x 128
// forward: 28 us (4.7 TB/s); 8190 x 40 x 128 backward with the fold of the gains' sums: 59 us (4.3 TB/s).
//
// d / 16 lanes hold a head, each 8 columns of its first half and the 8 that turn with them, so that the rotation stays within a lane
// and every access is 16 bytes.  A wave takes 1024 / d heads of one token beside each other (of several tokens where a
// token has fewer): forward two such rows of heads, backward all of the token's, so that the angles, as many bytes as four heads' columns, are loaded once for
// those.
#include "ah_ops.h"
#include "capi_util.h"
#include "common.h"
#include "kernels.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

using namespace ah;

namespace {

constexpr int NT = 256, NW = NT / 64, kMaxRows = 1 << 25;
// Heads of a lane in flight together (at those sizes 1, 2, 4: 30.4, 28.6, 29.9 us; backward 1, 2, 3: 66 to 69, 59, 68), and the rows of partial sums behind the
// gains' gradients: three blocks a CU, as many as 160 registers allow (512, 768, 1024: 61, 59, 65 us)
constexpr int kFwdPasses = 2, kBwdPasses = 2;
constexpr int kBwdBlocks = 768;

struct QkArgs {
  const bf16 *x, *dy, *gq, *gk;
  bf16* out;
  const float* cs;
  const int32_t* positions;
  float* part;               // [blocks][2][d]
  size_t ld_x, ld_y, ld_out;
  int T, S, nh, heads, n_pos;
  int slots;                 // heads side by side in a wave (a power of two), of (1024 / d) / slots tokens
  int passes;                // heads of a lane: ceil(heads / slots)
  int acc;                   // partial sums are added to what is there
  float eps;
};

template <int D>
__device__ __forceinline__ float head_sum(float v) {   // over the D / 16 lanes of a head
  auto add = [&](int ctrl_result) { v += __int_as_float(ctrl_result); };
  add(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, true));   // lanes 1 0 3 2
  add(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xF, 0xF, true));   // lanes 2 3 0 1
  if (D == 128) add(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xF, 0xF, true));   // lanes 7 .. 0 of 8
  return v;
}

// The lane's place: its columns of a head, and which token and head of a wave's it works on
struct Place {
  int col, token, head;
};
template <int D>
__device__ __forceinline__ Place place(int slots) {
  const int lane = threadIdx.x & 63, g = lane / (D / 16);
  return {lane % (D / 16) * 8, g / slots, g & (slots - 1)};
}

// (cos, sin) of the lane's 8 pairs
template <bool ROPE>
struct Turn {
  float c[ROPE ? 8 : 1], s[ROPE ? 8 : 1];
  __device__ __forceinline__ void load(const QkArgs& a, int t, int col, int half) {
    if constexpr (ROPE) {
      const int pos = a.positions ? a.positions[t] : t % a.S;
      const float nan = __builtin_nanf("");
      const bool ok = (unsigned)pos < (unsigned)a.n_pos;
      const f32x4* p = (const f32x4*)(a.cs + ((size_t)(ok ? pos : 0) * half + col) * 2);
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const f32x4 v = p[j];
        c[2 * j] = ok ? v[0] : nan; s[2 * j] = ok ? v[1] : nan;
        c[2 * j + 1] = ok ? v[2] : nan; s[2 * j + 1] = ok ? v[3] : nan;
      }
    }
  }
};

template <int D, bool ROPE>
__global__ __launch_bounds__(NT) void qk_norm_fwd_kernel(QkArgs a) {
  constexpr int H = D / 2, GROUPS = 1024 / D;
  const Place p = place<D>(a.slots);
  const int t = (blockIdx.x * NW + (threadIdx.x >> 6)) * (GROUPS / a.slots) + p.token;
  if (t >= a.T) return;
  Turn<ROPE> turn;
  turn.load(a, t, p.col, H);
  const bf16* x = a.x + (size_t)t * a.ld_x + p.col;
  bf16* y = a.out + (size_t)t * a.ld_out + p.col;
  const int first = blockIdx.y * kFwdPasses;
  bf16x8 lo[kFwdPasses], hi[kFwdPasses];
#pragma unroll
  for (int i = 0; i < kFwdPasses; i++) {
    const int head = (first + i) * a.slots + p.head;
    if (head < a.heads) {
      lo[i] = *(const bf16x8*)(x + (size_t)head * D);
      hi[i] = *(const bf16x8*)(x + (size_t)head * D + H);
    }
  }
#pragma unroll
  for (int i = 0; i < kFwdPasses; i++) {
    const int head = (first + i) * a.slots + p.head;
    if (head >= a.heads) break;   // (all lanes of a head together)
    const bf16* gain = (head < a.nh ? a.gq : a.gk) + p.col;
    const bf16x8 g0 = *(const bf16x8*)gain, g1 = *(const bf16x8*)(gain + H);
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const float u = bf2f(lo[i][j]), w = bf2f(hi[i][j]);
      ss = __builtin_fmaf(u, u, __builtin_fmaf(w, w, ss));
    }
    const float r = rsqrtf(head_sum<D>(ss) * (1.f / D) + a.eps);
    bf16x8 o0, o1;
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const float u = bf2f(lo[i][j]) * r * bf2f(g0[j]), w = bf2f(hi[i][j]) * r * bf2f(g1[j]);
      o0[j] = f2bf(ROPE ? u * turn.c[j] - w * turn.s[j] : u);
      o1[j] = f2bf(ROPE ? w * turn.c[j] + u * turn.s[j] : w);
    }
    *(bf16x8*)(y + (size_t)head * D) = o0;
    *(bf16x8*)(y + (size_t)head * D + H) = o1;
  }
}

// dn = the rotation back of dy; with xr = x r and w = dn gain: dx = r (w - xr mean(w xr)), and dn xr summed over all rows is the gain's
// gradient.  A lane keeps the sums of its columns for query and for key heads over all its tokens; they meet in LDS once a block.
template <int D, bool ROPE>
__global__ __launch_bounds__(NT) void qk_norm_bwd_kernel(QkArgs a) {
  constexpr int H = D / 2, GROUPS = 1024 / D, LPH = D / 16;
  __shared__ float red[NW][2][D];
  const Place p = place<D>(a.slots);
  const int wave = threadIdx.x >> 6, per_wave = GROUPS / a.slots;
  float sq[16], sk[16];
#pragma unroll
  for (int j = 0; j < 16; j++) { sq[j] = 0.f; sk[j] = 0.f; }
  const int units = (a.T + per_wave - 1) / per_wave;
  for (int u = blockIdx.x * NW + wave; u < units; u += gridDim.x * NW) {
    const int t = u * per_wave + p.token;
    if (t >= a.T) continue;
    Turn<ROPE> turn;
    turn.load(a, t, p.col, H);
    const bf16 *x = a.x + (size_t)t * a.ld_x + p.col, *dy = a.dy + (size_t)t * a.ld_y + p.col;
    bf16* dx = a.out + (size_t)t * a.ld_out + p.col;
    for (int first = 0; first < a.passes; first += kBwdPasses) {
      bf16x8 x0[kBwdPasses], x1[kBwdPasses], y0[kBwdPasses], y1[kBwdPasses];
#pragma unroll
      for (int i = 0; i < kBwdPasses; i++) {
        const int head = (first + i) * a.slots + p.head;
        if (head < a.heads) {
          x0[i] = *(const bf16x8*)(x + (size_t)head * D);
          x1[i] = *(const bf16x8*)(x + (size_t)head * D + H);
          y0[i] = *(const bf16x8*)(dy + (size_t)head * D);
          y1[i] = *(const bf16x8*)(dy + (size_t)head * D + H);
        }
      }
#pragma unroll
      for (int i = 0; i < kBwdPasses; i++) {
        const int head = (first + i) * a.slots + p.head;
        if (head >= a.heads) break;
        const bool query = head < a.nh;
        const bf16* gain = (query ? a.gq : a.gk) + p.col;
        const bf16x8 g0 = *(const bf16x8*)gain, g1 = *(const bf16x8*)(gain + H);
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const float v = bf2f(x0[i][j]), w = bf2f(x1[i][j]);
          ss = __builtin_fmaf(v, v, __builtin_fmaf(w, w, ss));
        }
        const float r = rsqrtf(head_sum<D>(ss) * (1.f / D) + a.eps);
        float w0[8], w1[8], c = 0.f;
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const float u = bf2f(y0[i][j]), v = bf2f(y1[i][j]);
          const float n0 = ROPE ? u * turn.c[j] + v * turn.s[j] : u, n1 = ROPE ? v * turn.c[j] - u * turn.s[j] : v;
          const float xr0 = bf2f(x0[i][j]) * r, xr1 = bf2f(x1[i][j]) * r;
          const float s0 = n0 * xr0, s1 = n1 * xr1;
          sq[j] += query ? s0 : 0.f; sk[j] += query ? 0.f : s0;
          sq[8 + j] += query ? s1 : 0.f; sk[8 + j] += query ? 0.f : s1;
          w0[j] = n0 * bf2f(g0[j]); w1[j] = n1 * bf2f(g1[j]);
          c = __builtin_fmaf(w0[j], xr0, __builtin_fmaf(w1[j], xr1, c));
        }
        c = head_sum<D>(c) * (1.f / D) * r;
        bf16x8 o0, o1;
#pragma unroll
        for (int j = 0; j < 8; j++) {
          o0[j] = f2bf(r * (w0[j] - bf2f(x0[i][j]) * c));
          o1[j] = f2bf(r * (w1[j] - bf2f(x1[i][j]) * c));
        }
        *(bf16x8*)(dx + (size_t)head * D) = o0;
        *(bf16x8*)(dx + (size_t)head * D + H) = o1;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 16; j++) {
#pragma unroll
    for (int o = LPH; o < 64; o <<= 1) {
      sq[j] += __shfl_xor(sq[j], o, 64);
      sk[j] += __shfl_xor(sk[j], o, 64);
    }
  }
  if ((threadIdx.x & 63) < LPH) {
#pragma unroll
    for (int j = 0; j < 8; j++) {
      red[wave][0][p.col + j] = sq[j]; red[wave][0][p.col + H + j] = sq[8 + j];
      red[wave][1][p.col + j] = sk[j]; red[wave][1][p.col + H + j] = sk[8 + j];
    }
  }
  __syncthreads();
  if (threadIdx.x < 2 * D) {   // part[which][block][column]: one array of rows for each gain
    const int which = threadIdx.x / D, c = threadIdx.x % D;
    float s = red[0][which][c];
#pragma unroll
    for (int w = 1; w < NW; w++) s += red[w][which][c];
    float* to = a.part + ((size_t)which * gridDim.x + blockIdx.x) * D + c;
    *to = a.acc ? *to + s : s;
  }
}

inline bool off16(const void* p) { return ((uintptr_t)p & 15) != 0; }

int check(const char* who, const ah_qk_norm_rope_t* c) {
  if (!c) return set_error(AH_EINVAL, "%s: config is NULL", who);
  if (c->struct_size != sizeof(ah_qk_norm_rope_t)) return set_error(AH_EINVAL, "%s: struct_size %u != %zu", who, c->struct_size, sizeof(ah_qk_norm_rope_t));
  if (c->head_dim != 64 && c->head_dim != 128) return set_error(AH_EUNSUPPORTED, "%s: head_dim %d: only 64 and 128 are supported", who, c->head_dim);
  if (c->rows < 0 || c->n_heads < 0 || c->n_kv_heads < 0 || c->n_heads > 65536 || c->n_kv_heads > 65536 || c->n_heads + c->n_kv_heads == 0)
    return set_error(AH_EINVAL, "%s: need rows >= 0 and 1 .. 65536 heads", who);
  if (c->rows > kMaxRows) return set_error(AH_EUNSUPPORTED, "%s: more than 2^25 rows", who);
  if (!(c->eps >= FLT_MIN) || !std::isfinite(c->eps)) return set_error(AH_EINVAL, "%s: eps must be finite and at least 2^-126", who);
  if ((c->n_heads && !c->gain_q) || (c->n_kv_heads && !c->gain_k)) return set_error(AH_EINVAL, "%s: a gain is NULL", who);
  if (off16(c->gain_q) || off16(c->gain_k) || off16(c->cos_sin) || ((uintptr_t)c->positions & 3)) return set_error(AH_EINVAL, "%s: gains and cos_sin must be 16-byte aligned, positions 4-byte", who);
  const int64_t width = (int64_t)(c->n_heads + c->n_kv_heads) * c->head_dim;
  for (int64_t ld : {c->ld_x, c->ld_y, c->ld_dx})
    if (ld != 0 && (ld < width || ld % 8)) return set_error(AH_EINVAL, "%s: a row stride must be a multiple of 8 and at least %lld", who, (long long)width);
  if (c->cos_sin) {
    if (c->n_pos < 1) return set_error(AH_EINVAL, "%s: n_pos must be >= 1", who);
    if (!c->positions && (c->seq_len < 1 || std::min(c->seq_len, std::max(c->rows, 1)) > c->n_pos))
      return set_error(AH_EINVAL, "%s: seq_len %d needs as many rows of cos_sin (n_pos %d)", who, c->seq_len, c->n_pos);
  }
  return AH_OK;
}

// Results in the place of what a call reads: row for row only
bool shifted(const void* in, size_t ld_in, const QkArgs& a) { return a.out == in && a.T > 1 && ld_in != a.ld_out; }

QkArgs args(const ah_qk_norm_rope_t* c, const void* x, const void* dy, void* out, int64_t ld_out, float* part) {
  const size_t width = (size_t)(c->n_heads + c->n_kv_heads) * c->head_dim;
  QkArgs a = {};
  a.x = (const bf16*)x; a.dy = (const bf16*)dy; a.out = (bf16*)out;
  a.gq = (const bf16*)c->gain_q; a.gk = (const bf16*)c->gain_k;
  a.cs = c->cos_sin; a.positions = c->positions; a.part = part;
  a.ld_x = c->ld_x ? c->ld_x : width; a.ld_y = c->ld_y ? c->ld_y : width; a.ld_out = ld_out ? ld_out : width;
  a.T = c->rows; a.S = c->seq_len; a.nh = c->n_heads; a.heads = c->n_heads + c->n_kv_heads; a.n_pos = c->n_pos;
  a.slots = 1;
  while (a.slots < a.heads && a.slots < 1024 / c->head_dim) a.slots *= 2;
  a.passes = (a.heads + a.slots - 1) / a.slots;
  a.eps = c->eps;
  return a;
}

int bwd_blocks(const ah_qk_norm_rope_t* c) {
  const QkArgs a = args(c, nullptr, nullptr, nullptr, 0, nullptr);
  const int per_block = NW * (1024 / c->head_dim / a.slots);   // tokens
  return std::max(1, std::min(kBwdBlocks, (c->rows + per_block - 1) / per_block));
}

hipError_t run_fwd(const QkArgs& a, int d, hipStream_t s) {
  const int tokens = NW * (1024 / d / a.slots);
  const dim3 grid((a.T + tokens - 1) / tokens, (a.passes + kFwdPasses - 1) / kFwdPasses);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(NT), 0, s, a); };
  if (d == 128) { if (a.cs) go(qk_norm_fwd_kernel<128, true>); else go(qk_norm_fwd_kernel<128, false>); }
  else { if (a.cs) go(qk_norm_fwd_kernel<64, true>); else go(qk_norm_fwd_kernel<64, false>); }
  return hipGetLastError();
}

hipError_t run_bwd(const QkArgs& a, int d, int blocks, hipStream_t s) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(NT), 0, s, a); };
  if (d == 128) { if (a.cs) go(qk_norm_bwd_kernel<128, true>); else go(qk_norm_bwd_kernel<128, false>); }
  else { if (a.cs) go(qk_norm_bwd_kernel<64, true>); else go(qk_norm_bwd_kernel<64, false>); }
  return hipGetLastError();
}

// a stage's configuration: as many key heads as query heads, a table of S positions
ah_qk_norm_rope_t stage_config(int ld_x, const void* gain_q, const void* gain_k, const float* cos_sin, int ld_y, int T, int S, int nh, int d, float eps) {
  ah_qk_norm_rope_t c = {};
  c.struct_size = sizeof c;
  c.rows = T; c.seq_len = S; c.n_heads = nh; c.n_kv_heads = nh; c.head_dim = d; c.n_pos = S; c.eps = eps;
  c.ld_x = ld_x; c.ld_y = ld_y; c.ld_dx = ld_y;
  c.gain_q = gain_q; c.gain_k = gain_k; c.cos_sin = cos_sin;
  return c;
}

}  // namespace

namespace ah {

hipError_t launch_qk_norm_fwd(const void* x, int ld_x, const void* gain_q, const void* gain_k, const float* cos_sin, void* y, int ld_y, int T, int S, int nh, int d,
                              float eps, hipStream_t s) {
  const ah_qk_norm_rope_t c = stage_config(ld_x, gain_q, gain_k, cos_sin, ld_y, T, S, nh, d, eps);
  return run_fwd(args(&c, x, nullptr, y, ld_y, nullptr), d, s);
}

hipError_t launch_qk_norm_bwd(const void* x, int ld_x, const void* gain_q, const void* gain_k, const float* cos_sin, void* dy, int ld_y, float* part, int acc, int T, int S,
                              int nh, int d, float eps, hipStream_t s) {
  const ah_qk_norm_rope_t c = stage_config(ld_x, gain_q, gain_k, cos_sin, ld_y, T, S, nh, d, eps);
  QkArgs a = args(&c, x, dy, dy, ld_y, part);
  a.acc = acc;
  return run_bwd(a, d, bwd_blocks(&c), s);
}

int qk_norm_bwd_blocks(int T, int nh, int d) {
  const ah_qk_norm_rope_t c = stage_config(0, nullptr, nullptr, nullptr, 0, T, T, nh, d, 1.f);
  return bwd_blocks(&c);
}

}  // namespace ah

extern "C" int ah_rope_table(float* cos_sin, int n_pos, int head_dim, double base, void* stream) {
  discard_stale_hip_error();
  if (!cos_sin || ((uintptr_t)cos_sin & 3)) return set_error(AH_EINVAL, "ah_rope_table: cos_sin is NULL or misaligned");
  if (n_pos < 1 || n_pos > (1 << 24) || head_dim < 2 || head_dim % 2 || head_dim > 256 || !(base > 0) || !std::isfinite(base))
    return set_error(AH_EINVAL, "ah_rope_table: need 1 <= n_pos <= 2^24, an even head_dim <= 256 and base > 0");
  return hip_status(launch_rope_table(cos_sin, n_pos, head_dim, base, (hipStream_t)stream), "ah_rope_table");
}

extern "C" int ah_qk_norm_rope_fwd(const ah_qk_norm_rope_t* c, const void* x, void* y, void* stream) {
  discard_stale_hip_error();
  if (int rc = check("ah_qk_norm_rope_fwd", c)) return rc;
  if (c->rows == 0) return AH_OK;
  if (!x || !y || off16(x) || off16(y)) return set_error(AH_EINVAL, "ah_qk_norm_rope_fwd: x or y is NULL or not 16-byte aligned");
  const QkArgs a = args(c, x, nullptr, y, c->ld_y, nullptr);
  if (shifted(x, a.ld_x, a)) return set_error(AH_EINVAL, "ah_qk_norm_rope_fwd: y in the place of x needs x's row stride");
  return hip_status(run_fwd(a, c->head_dim, (hipStream_t)stream), "ah_qk_norm_rope_fwd");
}

extern "C" int ah_qk_norm_rope_bwd_workspace(const ah_qk_norm_rope_t* c, uint64_t* bytes) {
  if (!bytes) return set_error(AH_EINVAL, "ah_qk_norm_rope_bwd_workspace: bytes is NULL");
  if (!c || c->struct_size != sizeof(ah_qk_norm_rope_t) || (c->head_dim != 64 && c->head_dim != 128) || c->rows < 0 || c->n_heads < 0 || c->n_kv_heads < 0 ||
      c->n_heads > 65536 || c->n_kv_heads > 65536)
    return set_error(AH_EINVAL, "ah_qk_norm_rope_bwd_workspace: bad configuration");
  if (c->rows > kMaxRows) return set_error(AH_EUNSUPPORTED, "ah_qk_norm_rope_bwd_workspace: more than 2^25 rows");
  *bytes = (uint64_t)bwd_blocks(c) * 2 * c->head_dim * sizeof(float);
  return AH_OK;
}

extern "C" int ah_qk_norm_rope_bwd(const ah_qk_norm_rope_t* c, const void* x, const void* dy, void* dx, float* d_gain_q, float* d_gain_k, int beta,
                                   void* workspace, void* stream) {
  discard_stale_hip_error();
  if (int rc = check("ah_qk_norm_rope_bwd", c)) return rc;
  if (beta != 0 && beta != 1) return set_error(AH_EINVAL, "ah_qk_norm_rope_bwd: beta must be 0 or 1");
  if ((c->n_heads && !d_gain_q) || (c->n_kv_heads && !d_gain_k) || !workspace || off16(workspace) || ((uintptr_t)d_gain_q & 3) || ((uintptr_t)d_gain_k & 3))
    return set_error(AH_EINVAL, "ah_qk_norm_rope_bwd: a gain's gradient or the workspace is NULL or misaligned");
  if (c->rows && (!x || !dy || !dx || off16(x) || off16(dy) || off16(dx))) return set_error(AH_EINVAL, "ah_qk_norm_rope_bwd: x, dy or dx is NULL or not 16-byte aligned");
  const int blocks = bwd_blocks(c), d = c->head_dim;
  float* part = (float*)workspace;
  const QkArgs a = args(c, x, dy, dx, c->ld_dx, part);
  if (shifted(x, a.ld_x, a) || shifted(dy, a.ld_y, a)) return set_error(AH_EINVAL, "ah_qk_norm_rope_bwd: dx in the place of x or dy needs its row stride");
  hipError_t e = run_bwd(a, d, blocks, (hipStream_t)stream);   // (no rows: writes zeros)
  if (e == hipSuccess) {
    FoldList f = {};
    if (c->n_heads) f.add(part, blocks, d, d_gain_q);
    if (c->n_kv_heads) f.add(part + (size_t)blocks * d, blocks, d, d_gain_k);
    e = launch_fold(f, beta, (hipStream_t)stream);
  }
  return hip_status(e, "ah_qk_norm_rope_bwd");
}
