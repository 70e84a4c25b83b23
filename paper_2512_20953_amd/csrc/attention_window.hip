// Attention over a sliding window with visible first tokens, forward and backward, for gfx950 (declared in include/ah_ops.h).
//
// The products, layouts and numerics are those of the full attention (attention.hip: everything transposed, one query or key per
// lane, tiles of 64 rows through LDS).  Here a block walks only the tiles that some row of it sees: those of its window, and before them
// those with the first tokens, so the work grows with seq_len * (window + sinks).  Lengths are any: the rows of a tile that
// lie behind the sequence's end are loaded as copies of its last row and masked.
//
// Probabilities and dS are rounded to bf16 (2^-8 at most of each), the type that the matrix instruction takes: an error of 1.9e-3 to 2.4e-3 of a result's norm, against 1.6e-3 with both in
// fp32, which is that of rounding the result itself; products in more bits would be another instruction at a fraction of the rate.
//
// Backward: a block per 128 queries for dQ (it leaves -delta behind), then a block per 128 keys and key head for dK, dV, which walks the query
// heads that share the key head one after the other: no atomics.  The keys that all later positions see have seq_len queries instead
// of window + 128: what lies behind their window is shared by further blocks, whose sums meet in a third kernel.
#include "ah_ops.h"
#include "attention_tile.h"
#include "capi_util.h"
#include "kernels.h"
#include <algorithm>
#include <cfloat>
#include <cmath>

using namespace ah;

namespace {

// What stands behind this in a conditional is jumped over, not computed and selected (the masks: a fifth of a step's vector instructions, wanted in a fifth of the steps)
#define AH_A_BRANCH() asm volatile("")

struct WinArgs {
  const bf16 *q, *k, *v, *o, *d_o;
  bf16 *out, *dq, *dk, *dv;
  float *lse, *delta, *nlse2, *part, *far_part;
  const int32_t* offsets;
  size_t ld_q, ld_k, ld_v, ld_o, ld_do, ld_dq, ld_dk, ld_dv;
  int64_t rows;
  int n_seq, S, nh, nkv, rep, W, sinks;
  int near;                // blocks that share the walk of 128 keys (1: none do)
  int chunks, far_waves;   // shares of the far queries of the first keys (0: not shared), and into how many the waves of a block share them further
  float sc2, scale;
};

struct Seq { int64_t r0; int len; };
__device__ __forceinline__ Seq sequence(const WinArgs& a, int b) {
  if (!a.offsets) return {(int64_t)b * a.S, a.S};
  const int64_t r0 = min((int64_t)max(a.offsets[b], 0), a.rows), r1 = min((int64_t)max(a.offsets[b + 1], 0), a.rows);
  return {r0, (int)min(max(r1 - r0, (int64_t)0), (int64_t)a.S)};
}

// The query head of a block: heads that share a key head follow each other at a distance of nkv blocks, so that with nkv a multiple of 8 they
// run on one XCD and find the keys in its L2
__device__ __forceinline__ int spread_head(const WinArgs& a, int i) { return (i % a.nkv) * a.rep + i / a.nkv; }

// One tile of 64 rows at g into LDS, the last `rows` - 1 of it repeated where it has fewer
template <int D>
__device__ __forceinline__ void load_tile(const bf16* __restrict__ g, const uint32_t* off, int ld, int rows, char* lds, int wave, int lane) {
  if (rows >= 64) {
    issue_tile<D>(g, off, lds, wave);
  } else {
    uint32_t cut[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; i++) {
      const int pos = (wave + 4 * i) * 1024 + lane * 16, r = pos / (2 * D), piece = (pos % (2 * D)) >> 4;
      cut[i] = (uint32_t)(min(r, rows - 1) * ld + swz<D>(r, piece) * 8) * 2u;
    }
    issue_tile<D>(g, cut, lds, wave);
  }
}

// The key tiles that a block of queries walks: the first `sink` tiles, then those from tile `first` on.
struct Tiles {
  int sink, first, count, sinks, len;
  __device__ __forceinline__ Tiles(const WinArgs& a, int q0, int qend, int seq_len) : sinks(a.sinks), len(seq_len) {   // queries q0 .. qend
    first = max(0, q0 - a.W + 1) / 64;
    sink = min((a.sinks + 63) / 64, first);
    count = sink + qend / 64 - first + 1;
  }
  __device__ __forceinline__ int key(int t) const { return (t < sink ? t : first + t - sink) * 64; }
  // Where the rows of tile t end.  Behind the first tokens none of their tiles' keys is seen, by any query of the block, and none is loaded: what is not
  // finite there would reach all later positions as 0 * inf.
  __device__ __forceinline__ int limit(int t) const { return t < sink ? min(sinks, len) : len; }
};

// What a wave's 32 queries from q0 on see of the keys k0 .. k0 + n - 1: nothing, all, or some
enum Seen { NONE, ALL, SOME };
__device__ __forceinline__ Seen seen(const WinArgs& a, int q0, int k0, int n) {
  if (k0 > q0 + 31 || (q0 - (k0 + n - 1) >= a.W && k0 >= a.sinks)) return NONE;
  return k0 + n - 1 <= q0 && (q0 + 31 - k0 < a.W || k0 + n <= a.sinks) ? ALL : SOME;
}

// Score r of a tile's 32 keys and the lane's query: key 8 (r / 4) + r % 4 of them is hidden iff it lies behind lim (= query - first key - 4 hf) or
// is out of the window and no first token
struct Mask {
  int lim, low, first;
  __device__ __forceinline__ Mask(const WinArgs& a, int q, int k0, int hf) : lim(q - k0 - 4 * hf), low(lim - a.W), first(a.sinks - k0 - 4 * hf) {}
  __device__ __forceinline__ bool hides(int key) const { return (key > lim) | ((key <= low) & (key >= first)); }   // (no branches)
};

// rows of a result that lie before the sequence's end
template <int D, class F>
__device__ __forceinline__ void store_rows_to(const F& val, char* strip, bf16* __restrict__ dst, size_t ld, int rows, int lane) {
  if (rows >= 32) return store_rows<D>(val, strip, dst, ld, lane);
  constexpr int RB = 2 * D, PPR = D / 8, RPI = 64 / PPR;
  auto at = [](int row, int piece) { return row * RB + ((piece ^ (D == 128 ? row : row >> 1)) & (PPR - 1)) * 16; };
  const int base = at(lane & 31, 0) + 8 * (lane >> 5);
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
    for (int g = 0; g < 4; g++) {
      bf16x4 v;
#pragma unroll
      for (int i = 0; i < 4; i++) v[i] = f2bf(val(dt, 4 * g + i));
      *(bf16x4*)(strip + (base ^ ((4 * dt + g) * 16))) = v;
    }
  __builtin_amdgcn_wave_barrier();
  const int row = lane / PPR, piece = lane % PPR;
#pragma unroll
  for (int it = 0; it < 32 / RPI; it++)
    if (row + it * RPI < rows) *(bf16x8*)(dst + (size_t)(row + it * RPI) * ld + piece * 8) = *(const bf16x8*)(strip + at(row + it * RPI, piece));
  __builtin_amdgcn_wave_barrier();
}

// =========================================================================== forward
// One pass with a running maximum and sum.  1 x 8192 x 32 heads in groups of four x 128, window 1024, 4 first tokens: 168 us.  No unit is full: of a launch's cycles by counters (traced, 182 us
// at 2.05 GHz) the CU's LDS path has 55 % (a wave needs all of a K and V tile as fragments, 128 KB a tile and block at 128 B/clk, and the tile's 32 KB arrive at 1.7 times that price), the matrix
// units 37, the vector units 35; two waves a SIMD do not hide them behind one another.  With 64 queries a wave half the LDS reads, but one wave a SIMD: 252 us.
template <int D>
__global__ __launch_bounds__(256, 2) void win_fwd_kernel(WinArgs a) {
  constexpr int TILEB = 64 * 2 * D, STAGE = 2 * TILEB, NK = D / 16, ND = D / 32;
  __shared__ __attribute__((aligned(1024))) char ring[2 * STAGE];
  const int lane = threadIdx.x & 63, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nbh = a.n_seq * a.nh;
  const int qb = blockIdx.x / nbh, bh = blockIdx.x - qb * nbh, b = bh / a.nh, head = spread_head(a, bh - b * a.nh);
  const Seq sq = sequence(a, b);
  const int q0 = qb * 128;
  if (q0 >= sq.len) return;
  const bf16* kp = a.k + (size_t)sq.r0 * a.ld_k + (head / a.rep) * D;
  const bf16* vp = a.v + (size_t)sq.r0 * a.ld_v + (head / a.rep) * D;
  const int qw0 = q0 + wave * 32, q = qw0 + (lane & 31);
  const bf16* qrow = a.q + (size_t)(sq.r0 + min(q, sq.len - 1)) * a.ld_q + head * D;

  bf16x8 qf[NK];
  f32x16 oacc[ND];
#pragma unroll
  for (int ks = 0; ks < NK; ks++) qf[ks] = *(const bf16x8*)(qrow + ks * 16 + hf * 8);
#pragma unroll
  for (int dt = 0; dt < ND; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++) oacc[dt][r] = 0.f;
  float m = -FLT_MAX, l = 0.f;   // finite: a wave may see nothing of a tile that others see

  uint32_t offk[ND], offv[ND];
#pragma unroll
  for (int i = 0; i < ND; i++) {
    offk[i] = tile_src_offset<D>(wave + 4 * i, lane, a.ld_k);
    offv[i] = tile_src_offset<D>(wave + 4 * i, lane, a.ld_v);
  }
  const Tiles tiles(a, q0, min(q0 + 127, sq.len - 1), sq.len);
  auto load = [&](int t) {
    const int k0 = tiles.key(t);
    char* slot = ring + (t & 1) * STAGE;
    load_tile<D>(kp + (size_t)k0 * a.ld_k, offk, a.ld_k, tiles.limit(t) - k0, slot, wave, lane);
    load_tile<D>(vp + (size_t)k0 * a.ld_v, offv, a.ld_v, tiles.limit(t) - k0, slot + TILEB, wave, lane);
  };
  load(0);
  AH_NEXT_TILE();
  for (int t = 0; t < tiles.count; t++) {
    if (t + 1 < tiles.count) load(t + 1);
    const int k0 = tiles.key(t);
    const char *cK = ring + (t & 1) * STAGE, *cV = cK + TILEB;
    const Seen what = seen(a, qw0, k0, 64);
    if (what != NONE) {
      f32x16 s[2];
#pragma unroll
      for (int h = 0; h < 2; h++) {
#pragma unroll
        for (int r = 0; r < 16; r++) s[h][r] = 0.f;
#pragma unroll
        for (int ks = 0; ks < NK; ks++) s[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rowmajor<D>(cK, 32 * h + (lane & 31), ks, hf), qf[ks], s[h], 0, 0, 0);
      }
      if (what == SOME) {
        AH_A_BRANCH();
        const Mask mask(a, q, k0, hf);
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
          for (int r = 0; r < 16; r++)
            if (mask.hides(32 * h + 8 * (r >> 2) + (r & 3))) s[h][r] = -INFINITY;
      }
      float mx = fmaxf(s[0][0], s[1][0]);
#pragma unroll
      for (int r = 1; r < 16; r++) mx = fmaxf(fmaxf(mx, s[0][r]), s[1][r]);
      mx = half_max(mx) * a.sc2;
      if (__any(mx > m + RESCALE_SLACK)) {
        const float m_new = fmaxf(m, mx), alpha = fexp2(m - m_new);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int dt = 0; dt < ND; dt++)
#pragma unroll
          for (int r = 0; r < 16; r++) oacc[dt][r] *= alpha;
      }
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
          s[h][r] = fexp2(__builtin_fmaf(s[h][r], a.sc2, -m));
          l += s[h][r];
        }
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int s2 = 0; s2 < 2; s2++) {
          const bf16x8 pf = pack8(s[h], s2);
#pragma unroll
          for (int dt = 0; dt < ND; dt++)
            oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_transposed<D>(cV, 32 * h + 16 * s2 + 4 * hf, dt, lane), pf, oacc[dt], 0, 0, 0);
        }
    }
    AH_NEXT_TILE();
  }
  const float sum = l + __shfl_xor(l, 32, 64), inv = 1.f / sum;
  const int rows = sq.len - qw0;   // of the wave's that exist
  if (rows <= 0) return;
  store_rows_to<D>([&](int dt, int r) { return oacc[dt][r] * inv; }, ring + wave * strip_bytes<D>(),
                   a.out + (size_t)(sq.r0 + qw0) * a.ld_o + head * D, a.ld_o, rows, lane);
  if (lane < min(rows, 32)) a.lse[((size_t)b * a.nh + head) * a.S + q] = (m + __log2f(sum)) * LN2;
}

// =========================================================================== backward: dQ
// P from the kept log-sum-exps, dS = P (dO V^T - delta), dQ = scale dS K.  1 x 4096 x 32 x 128, window 1024, 4 first tokens: 118 us traced, of whose cycles the matrix
// units have 36 %, the LDS path about half (the fragments of K, both ways round, and V: 192 KB a tile and block beside the tile's arrival), the vector units 23.
template <int D>
__global__ __launch_bounds__(256, 2) void win_dq_kernel(WinArgs a) {
  constexpr int TILEB = 64 * 2 * D, STAGE = 2 * TILEB, NK = D / 16, ND = D / 32;
  __shared__ __attribute__((aligned(1024))) char ring[2 * STAGE];
  const int lane = threadIdx.x & 63, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nbh = a.n_seq * a.nh;
  const int qb = blockIdx.x / nbh, bh = blockIdx.x - qb * nbh, b = bh / a.nh, head = spread_head(a, bh - b * a.nh);
  const Seq sq = sequence(a, b);
  const int q0 = qb * 128;
  if (q0 >= sq.len) return;
  const bf16* kp = a.k + (size_t)sq.r0 * a.ld_k + (head / a.rep) * D;
  const bf16* vp = a.v + (size_t)sq.r0 * a.ld_v + (head / a.rep) * D;
  const int qw0 = q0 + wave * 32, q = qw0 + (lane & 31);
  const size_t token = (size_t)(sq.r0 + min(q, sq.len - 1)), row = ((size_t)b * a.nh + head) * a.S + min(q, sq.len - 1);

  bf16x8 qf[NK], dof[NK];
  f32x16 acc[ND];
#pragma unroll
  for (int ks = 0; ks < NK; ks++) {
    qf[ks] = *(const bf16x8*)(a.q + token * a.ld_q + head * D + ks * 16 + hf * 8);
    dof[ks] = *(const bf16x8*)(a.d_o + token * a.ld_do + head * D + ks * 16 + hf * 8);
  }
#pragma unroll
  for (int dt = 0; dt < ND; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++) acc[dt][r] = 0.f;
  const float lse2 = a.lse[row] * LOG2E, delta = row_delta<D>(dof, a.o + token * a.ld_o + head * D, hf);
  if (hf == 0 && q < sq.len) {   // for the dK/dV kernel: what dP starts from, and what the exponent's argument ends with
    a.delta[row] = -delta;
    a.nlse2[row] = -lse2;
  }

  uint32_t offk[ND], offv[ND];
#pragma unroll
  for (int i = 0; i < ND; i++) {
    offk[i] = tile_src_offset<D>(wave + 4 * i, lane, a.ld_k);
    offv[i] = tile_src_offset<D>(wave + 4 * i, lane, a.ld_v);
  }
  const Tiles tiles(a, q0, min(q0 + 127, sq.len - 1), sq.len);
  auto load = [&](int t) {
    const int k0 = tiles.key(t);
    char* slot = ring + (t & 1) * STAGE;
    load_tile<D>(kp + (size_t)k0 * a.ld_k, offk, a.ld_k, tiles.limit(t) - k0, slot, wave, lane);
    load_tile<D>(vp + (size_t)k0 * a.ld_v, offv, a.ld_v, tiles.limit(t) - k0, slot + TILEB, wave, lane);
  };
  load(0);
  AH_NEXT_TILE();
  for (int t = 0; t < tiles.count; t++) {
    if (t + 1 < tiles.count) load(t + 1);
    const int k0 = tiles.key(t);
    const char *cK = ring + (t & 1) * STAGE, *cV = cK + TILEB;
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const Seen what = seen(a, qw0, k0 + 32 * h, 32);
      if (what == NONE) continue;
      f32x16 s, dp;
#pragma unroll
      for (int r = 0; r < 16; r++) { s[r] = 0.f; dp[r] = -delta; }   // the product dO V^T lands on -delta
#pragma unroll
      for (int ks = 0; ks < NK; ks++) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rowmajor<D>(cK, 32 * h + (lane & 31), ks, hf), qf[ks], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rowmajor<D>(cV, 32 * h + (lane & 31), ks, hf), dof[ks], dp, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 16; r++) s[r] = fexp2(__builtin_fmaf(s[r], a.sc2, -lse2));
      if (what == SOME) {
        AH_A_BRANCH();
        const Mask mask(a, q, k0 + 32 * h, hf);
#pragma unroll
        for (int r = 0; r < 16; r++) s[r] = mask.hides(8 * (r >> 2) + (r & 3)) ? 0.f : s[r];
      }
#pragma unroll
      for (int r = 0; r < 16; r++) s[r] *= dp[r];
#pragma unroll
      for (int s2 = 0; s2 < 2; s2++) {
        const bf16x8 dsf = pack8(s, s2);
#pragma unroll
        for (int dt = 0; dt < ND; dt++)
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_transposed<D>(cK, 32 * h + 16 * s2 + 4 * hf, dt, lane), dsf, acc[dt], 0, 0, 0);
      }
    }
    AH_NEXT_TILE();
  }
  const int rows = sq.len - qw0;
  if (rows <= 0) return;
  store_rows_to<D>([&](int dt, int r) { return acc[dt][r] * a.scale; }, ring + wave * strip_bytes<D>(),
                   a.dq + (size_t)(sq.r0 + qw0) * a.ld_dq + head * D, a.ld_dq, rows, lane);
}

// =========================================================================== backward: dK, dV
// The query tiles of the 128 keys from k0 on: from their own position to the window's end.  Keys that all later positions see have the tiles
// from `near` on too: in the same block (chunks == 0), or shared by `chunks` further blocks.
struct QueryTiles {
  int first, near, end;
  __device__ __forceinline__ QueryTiles(const WinArgs& a, int k0, int len) {
    first = k0 / 64;
    end = (len + 63) / 64;
    near = min(end, (k0 + 127 + a.W - 1) / 64 + 1);
  }
};

// dV = P^T dO, dK = scale dS^T Q, the sums of a wave's 32 keys in registers over the whole walk (128-wide heads: 342, one wave a SIMD, which bounds it: 219 us traced at
// the size above, 36 % of the cycles waiting; 64-wide: 190, two waves).
//
// Partial sums [share][key][dk | dv][D] in fp32.  Near the keys: all keys of a sequence, where a small launch shares the walk of a block between
// several (near > 1).  Far: the first keys, of the blocks that walk the queries behind their window; share 0 is the near walk's where that is not shared.
__device__ __forceinline__ float* near_part(const WinArgs& a, int bk, int share, int key, int width) {
  return a.part + (((size_t)bk * a.near + share) * a.S + key) * width;
}
__device__ __forceinline__ float* far_part(const WinArgs& a, int bk, int share, int key, int width) {
  return a.far_part + (((size_t)bk * (1 + a.chunks * a.far_waves) + share) * a.sinks + key) * width;
}

template <int D>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void win_dkv_kernel(WinArgs a) {
  constexpr int TILEB = 64 * 2 * D, STAGE = 2 * TILEB + 1024, NK = D / 16, ND = D / 32;
  __shared__ __attribute__((aligned(1024))) char ring[2 * STAGE];
  const int lane = threadIdx.x & 63, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nbk = a.n_seq * a.nkv;
  // a block (or `near` of them) per 128 keys, and behind them those with the queries far behind the first keys, which are short and fill the last round
  const int rank = blockIdx.x / nbk, bk = blockIdx.x - rank * nbk, b = bk / a.nkv, kvh = bk - b * a.nkv;
  const int near_blocks = (a.S + 127) / 128 * a.near, sink_blocks = (a.sinks + 127) / 128, far = rank - near_blocks;
  const int kb = far < 0 ? rank / a.near : far % sink_blocks, chunk = far < 0 ? 0 : 1 + far / sink_blocks, share = far < 0 ? rank % a.near : 0;
  const Seq sq = sequence(a, b);
  const int k0 = kb * 128;
  if (k0 >= sq.len) return;
  const QueryTiles qt(a, k0, sq.len);
  int t0 = qt.first, t1 = k0 < a.sinks && a.chunks == 0 ? qt.end : qt.near;
  if (chunk > 0) {
    const int each = (qt.end - qt.near + a.chunks - 1) / a.chunks;
    t0 = min(qt.end, qt.near + (chunk - 1) * each);
    t1 = min(qt.end, t0 + each);
  }
  // items of the walk: tile t0 + i % per_head of query head i / per_head
  const int per_head = t1 - t0, all = per_head * a.rep, each = chunk > 0 ? all : (all + a.near - 1) / a.near;
  const int i0 = share * each, i1 = min(all, i0 + each);

  // With at most 32 first keys the four waves of a far block take those same keys and every fourth run of 32 queries each, else 32 keys each
  const bool same_keys = chunk > 0 && a.far_waves > 1;
  const int pick = same_keys ? 3 : 0, mine = same_keys ? wave : 0;
  const int kw0 = k0 + (same_keys ? 0 : wave * 32), key = kw0 + (lane & 31);
  const size_t krow = (size_t)(sq.r0 + min(key, sq.len - 1));
  uint32_t offq[ND], offo[ND];
#pragma unroll
  for (int i = 0; i < ND; i++) {
    offq[i] = tile_src_offset<D>(wave + 4 * i, lane, a.ld_q);
    offo[i] = tile_src_offset<D>(wave + 4 * i, lane, a.ld_do);
  }
  // (head and tile of the next item to load and tile of the one at hand are counted along: a division costs as much as a tenth of a tile)
  int load_head = kvh * a.rep, load_tile_at = t0 + i0, tile = t0 + i0, fill = 0;
  if (a.near > 1 && per_head > 0) {
    load_head += i0 / per_head;
    tile = load_tile_at = t0 + i0 % per_head;
  }
  auto load = [&]() {
    const int head = load_head, r0 = load_tile_at * 64, left = sq.len - r0;
    if (++load_tile_at == t1) { load_tile_at = t0; load_head++; }
    char* slot = ring + fill * STAGE;
    fill ^= 1;
    load_tile<D>(a.q + (size_t)(sq.r0 + r0) * a.ld_q + head * D, offq, a.ld_q, left, slot, wave, lane);
    load_tile<D>(a.d_o + (size_t)(sq.r0 + r0) * a.ld_do + head * D, offo, a.ld_do, left, slot + TILEB, wave, lane);
    // 64 -log-sum-exps (base 2), 64 -deltas (waves 2 and 3 repeat them into spare bytes)
    load4(((wave & 1) ? a.delta : a.nlse2) + ((size_t)b * a.nh + head) * a.S + r0, (uint32_t)min(lane, left - 1) * 4u, slot + 2 * TILEB + wave * 256);
  };
  bf16x8 kf[NK], vf[NK];
  f32x16 dk[ND], dv[ND];
#pragma unroll
  for (int ks = 0; ks < NK; ks++) {
    kf[ks] = *(const bf16x8*)(a.k + krow * a.ld_k + kvh * D + ks * 16 + hf * 8);
    vf[ks] = *(const bf16x8*)(a.v + krow * a.ld_v + kvh * D + ks * 16 + hf * 8);
  }
#pragma unroll
  for (int dt = 0; dt < ND; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++) { dk[dt][r] = 0.f; dv[dt][r] = 0.f; }
  if (i0 < i1) {
    load();
    AH_NEXT_TILE();
  }
  int at = 0;
  for (int i = i0; i < i1; i++) {
    if (i + 1 < i1) load();
    const char *cQ = ring + at * STAGE, *cO = cQ + TILEB;
    at ^= 1;
    const float* stat = (const float*)(cQ + 2 * TILEB);
    const int r0 = tile * 64;
    if (++tile == t1) tile = t0;
#pragma unroll
    for (int t = 0; t < 64; t += 32) {
      const int qw0 = r0 + t;   // 32 queries against the wave's 32 keys
      if (((2 * i + t / 32) & pick) != mine) continue;
      if (kw0 > qw0 + 31 || qw0 >= sq.len || (qw0 - (kw0 + 31) >= a.W && kw0 >= a.sinks)) continue;
      const bool every = kw0 + 31 <= qw0 && qw0 + 32 <= sq.len && (qw0 + 31 - kw0 < a.W || kw0 + 32 <= a.sinks);
      f32x16 s, dp;
#pragma unroll
      for (int r = 0; r < 16; r++) { s[r] = 0.f; dp[r] = stat[64 + t + 4 * hf + 8 * (r >> 2) + (r & 3)]; }
#pragma unroll
      for (int ks = 0; ks < NK; ks++) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rowmajor<D>(cQ, t + (lane & 31), ks, hf), kf[ks], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rowmajor<D>(cO, t + (lane & 31), ks, hf), vf[ks], dp, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 16; r++) s[r] = fexp2(__builtin_fmaf(s[r], a.sc2, stat[t + 4 * hf + 8 * (r >> 2) + (r & 3)]));
      if (!every) {
        AH_A_BRANCH();
        // query qw0 + 4 hf + c sees the lane's key iff lo <= c <= hi
        const int lo = key - qw0 - 4 * hf, end = sq.len - 1 - qw0 - 4 * hf, hi = key < a.sinks ? end : min(end, lo + a.W - 1);
#pragma unroll
        for (int r = 0; r < 16; r++) {
          const int c = 8 * (r >> 2) + (r & 3);
          s[r] = (c < lo) | (c > hi) ? 0.f : s[r];
        }
      }
#pragma unroll
      for (int r = 0; r < 16; r++) dp[r] *= s[r];
#pragma unroll
      for (int s2 = 0; s2 < 2; s2++) {
        const bf16x8 pf = pack8(s, s2), dsf = pack8(dp, s2);
#pragma unroll
        for (int dt = 0; dt < ND; dt++) {
          dv[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_transposed<D>(cO, t + 16 * s2 + 4 * hf, dt, lane), pf, dv[dt], 0, 0, 0);
          dk[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_transposed<D>(cQ, t + 16 * s2 + 4 * hf, dt, lane), dsf, dk[dt], 0, 0, 0);
        }
      }
    }
    AH_NEXT_TILE();
  }
  const int rows = sq.len - kw0;
  if (rows <= 0) return;
  const bool far_sums = a.chunks > 0 && kw0 < a.sinks;
  if (far_sums || a.near > 1) {   // the lane's key and half of its columns
    const bool kept = key < sq.len && (a.near > 1 || key < a.sinks);
    float* p = nullptr;
    if (chunk > 0) p = key < a.sinks ? far_part(a, bk, 1 + (chunk - 1) * a.far_waves + (same_keys ? wave : 0), key, 2 * D) : nullptr;
    else p = a.near > 1 ? near_part(a, bk, share, key, 2 * D) : far_part(a, bk, 0, key, 2 * D);
    if (kept && p) {
#pragma unroll
      for (int dt = 0; dt < ND; dt++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
          const int c = dt * 32 + 8 * g + 4 * hf;
          *(f32x4*)(p + c) = f32x4{dk[dt][4 * g], dk[dt][4 * g + 1], dk[dt][4 * g + 2], dk[dt][4 * g + 3]};
          *(f32x4*)(p + D + c) = f32x4{dv[dt][4 * g], dv[dt][4 * g + 1], dv[dt][4 * g + 2], dv[dt][4 * g + 3]};
        }
    }
  }
  if (chunk > 0 || a.near > 1) return;
  // (first keys whose sums are shared are written here too, and again by the kernel that adds the shares up)
  char* strip = ring + wave * strip_bytes<D>();
  store_rows_to<D>([&](int dt, int r) { return dk[dt][r] * a.scale; }, strip, a.dk + (size_t)(sq.r0 + kw0) * a.ld_dk + kvh * D, a.ld_dk, rows, lane);
  store_rows_to<D>([&](int dt, int r) { return dv[dt][r]; }, strip, a.dv + (size_t)(sq.r0 + kw0) * a.ld_dv + kvh * D, a.ld_dv, rows, lane);
}

// dK and dV from the shares, in their order: of all keys where the near walks were shared, else of the first ones.  A thread takes four columns of a key.
constexpr int JOIN_KEYS = 4;
template <int D>
__global__ __launch_bounds__(JOIN_KEYS * D / 2) void win_join_kernel(WinArgs a) {
  const int key = blockIdx.x * JOIN_KEYS + threadIdx.x / (D / 2), c = threadIdx.x % (D / 2) * 4, bk = blockIdx.y, b = bk / a.nkv, kvh = bk - b * a.nkv;
  const Seq sq = sequence(a, b);
  if (key >= sq.len || (a.near == 1 && key >= a.sinks)) return;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (a.near > 1) {
#pragma unroll 4
    for (int i = 0; i < a.near; i++) s += *(const f32x4*)(near_part(a, bk, i, key, 2 * D) + c);
  }
  if (a.chunks > 0 && key < a.sinks) {
#pragma unroll 4
    for (int i = a.near > 1; i <= a.chunks * a.far_waves; i++) s += *(const f32x4*)(far_part(a, bk, i, key, 2 * D) + c);
  }
  const size_t row = sq.r0 + key;
  bf16x4 v;
#pragma unroll
  for (int i = 0; i < 4; i++) v[i] = f2bf(c < D ? s[i] * a.scale : s[i]);
  if (c < D) *(bf16x4*)(a.dk + row * a.ld_dk + kvh * D + c) = v;
  else *(bf16x4*)(a.dv + row * a.ld_dv + kvh * D + c - D) = v;
}

// ---------------------------------------------------------------------------------------- host
inline bool off16(const void* p) { return ((uintptr_t)p & 15) != 0; }

int far_waves(const ah_attention_window_t* c) { return c->sinks <= 32 ? 4 : 1; }

// Shares of the queries behind the window of the first keys: none where no position lies there, or where the blocks of the first keys fill the
// chip by themselves; else as many as make a share about as long as an
// ordinary block's walk, or a quarter of it where the waves of a block split the queries further.  (Whole backward, us, with 2, 4 and 8 shares and by this
// rule, four first tokens: 1 x 4096 x 32 heads in groups of four x 64, window 512, 200, 147, 131, 120; 1 x 8192 x 32 in groups of four x 128, window 1024, 753, 605,
// 593, 568; 1 x 4096 x 32 x 128, window 1024, 300, 291, 292, 295.)
int far_chunks(const ah_attention_window_t* c) {
  const long blocks = (long)c->n_seq * c->n_kv_heads * ((std::min(c->sinks, c->seq_len) + 127) / 128);
  const long far = ((long)c->seq_len - c->window) / 64, usual = (128 + std::min(c->window, c->seq_len)) / 64 + 1;
  if (c->sinks == 0 || far <= usual / 2 || blocks >= 512) return 0;
  return far_waves(c) > 1 ? (int)std::min(32L, (4 * far + usual - 1) / usual) : (int)std::min(8L, (far + usual - 1) / usual);
}

// Blocks that share the walk of 128 keys: as many as bring a launch that leaves CUs idle to one block (two of 64-wide heads) each, with two tiles at least for
// each of them
int near_shares(const ah_attention_window_t* c) {
  const long blocks = (long)c->n_seq * c->n_kv_heads * ((c->seq_len + 127) / 128), want = c->head_dim == 64 ? 512 : 256;
  const long tiles = ((128L + std::min(c->window, c->seq_len) - 1) / 64 + 1) * (c->n_heads / c->n_kv_heads);
  return (int)std::max(1L, std::min({want / blocks, tiles / 2, 8L}));
}

size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

// partial sums: near the keys, and of the far queries of the first ones
size_t near_bytes(const ah_attention_window_t* c) {
  const int n = near_shares(c);
  return n > 1 ? (size_t)c->n_seq * c->n_kv_heads * n * c->seq_len * 2 * c->head_dim * sizeof(float) : 0;
}
size_t far_bytes(const ah_attention_window_t* c) {
  const int n = far_chunks(c);
  return n > 0 ? (size_t)c->n_seq * c->n_kv_heads * (1 + n * far_waves(c)) * std::min(c->sinks, c->seq_len) * 2 * c->head_dim * sizeof(float) : 0;
}
size_t delta_bytes(const ah_attention_window_t* c) { return align256((size_t)c->n_seq * c->n_heads * c->seq_len * sizeof(float)); }

int check_sizes(const char* who, const ah_attention_window_t* c) {
  if (!c) return set_error(AH_EINVAL, "%s: config is NULL", who);
  if (c->struct_size != sizeof(ah_attention_window_t)) return set_error(AH_EINVAL, "%s: struct_size %u != %zu", who, c->struct_size, sizeof(ah_attention_window_t));
  if (c->head_dim != 64 && c->head_dim != 128) return set_error(AH_EUNSUPPORTED, "%s: head_dim %d: only 64 and 128 are supported", who, c->head_dim);
  if (c->n_seq < 1 || c->seq_len < 1 || c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads)
    return set_error(AH_EINVAL, "%s: need n_seq, seq_len >= 1 and n_kv_heads that divides n_heads", who);
  if (c->window < 1 || c->sinks < 0) return set_error(AH_EINVAL, "%s: need window >= 1 and sinks >= 0", who);
  if (c->seq_len > (1 << 24) || c->n_heads > 4096 || (double)c->n_seq * c->n_heads * ((c->seq_len + 127) / 128 + 8.0 * ((std::min(c->sinks, c->seq_len) + 127) / 128)) > (1 << 23))
    return set_error(AH_EUNSUPPORTED, "%s: n_seq * n_heads * seq_len too large", who);
  return AH_OK;
}

int check(const char* who, const ah_attention_window_t* c, bool bwd) {
  if (int rc = check_sizes(who, c)) return rc;
  if (c->rows < 0 || (!c->offsets && c->rows != 0 && c->rows < (int64_t)c->n_seq * c->seq_len)) return set_error(AH_EINVAL, "%s: rows %lld are fewer than n_seq * seq_len", who, (long long)c->rows);
  if (c->offsets && c->rows < 1) return set_error(AH_EINVAL, "%s: packed sequences need `rows`", who);
  if ((uintptr_t)c->offsets & 3) return set_error(AH_EINVAL, "%s: offsets are misaligned", who);
  const int64_t wq = (int64_t)c->n_heads * c->head_dim, wk = (int64_t)c->n_kv_heads * c->head_dim;
  auto bad = [](int64_t ld, int64_t w) { return ld != 0 && (ld < w || ld % 8 || ld > (1 << 23)); };
  if (bad(c->ld_q, wq) || bad(c->ld_k, wk) || bad(c->ld_v, wk) || bad(c->ld_o, wq) || (bwd && (bad(c->ld_do, wq) || bad(c->ld_dq, wq) || bad(c->ld_dk, wk) || bad(c->ld_dv, wk))))
    return set_error(AH_EINVAL, "%s: a row stride must be a multiple of 8, at least the heads' columns and at most 2^23", who);
  return AH_OK;
}

WinArgs args(const ah_attention_window_t* c, const void* q, const void* k, const void* v) {
  const size_t wq = (size_t)c->n_heads * c->head_dim, wk = (size_t)c->n_kv_heads * c->head_dim;
  WinArgs a = {};
  a.q = (const bf16*)q; a.k = (const bf16*)k; a.v = (const bf16*)v;
  auto ld = [](int64_t given, size_t w) { return given ? (size_t)given : w; };
  a.ld_q = ld(c->ld_q, wq); a.ld_k = ld(c->ld_k, wk); a.ld_v = ld(c->ld_v, wk); a.ld_o = ld(c->ld_o, wq);
  a.ld_do = ld(c->ld_do, wq); a.ld_dq = ld(c->ld_dq, wq); a.ld_dk = ld(c->ld_dk, wk); a.ld_dv = ld(c->ld_dv, wk);
  a.offsets = c->offsets;
  a.rows = c->rows ? c->rows : (int64_t)c->n_seq * c->seq_len;
  a.n_seq = c->n_seq; a.S = c->seq_len; a.nh = c->n_heads; a.nkv = c->n_kv_heads; a.rep = c->n_heads / c->n_kv_heads;
  a.W = std::min(c->window, c->seq_len);    // (a larger one sees no more, and positions plus it stay within 32 bits)
  a.sinks = std::min(c->sinks, c->seq_len);
  a.scale = 1.f / std::sqrt((float)c->head_dim);
  a.sc2 = LOG2E * a.scale;
  return a;
}

hipError_t run_fwd(const WinArgs& a, int d, hipStream_t s) {
  const dim3 grid((unsigned)(a.n_seq * a.nh * ((a.S + 127) / 128)));
  if (d == 128) hipLaunchKernelGGL(win_fwd_kernel<128>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(win_fwd_kernel<64>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

size_t bwd_bytes(const ah_attention_window_t* c) { return 2 * delta_bytes(c) + near_bytes(c) + far_bytes(c); }

hipError_t run_bwd(WinArgs a, const ah_attention_window_t* c, void* workspace, hipStream_t s) {
  a.delta = (float*)workspace;
  a.chunks = far_chunks(c);
  a.far_waves = far_waves(c);
  a.near = near_shares(c);
  a.nlse2 = (float*)((char*)workspace + delta_bytes(c));
  a.part = (float*)((char*)workspace + 2 * delta_bytes(c));
  a.far_part = (float*)((char*)a.part + near_bytes(c));
  const int key_blocks = (a.S + 127) / 128, sink_blocks = (a.sinks + 127) / 128;
  const dim3 gq((unsigned)(a.n_seq * a.nh * key_blocks)), gk((unsigned)(a.n_seq * a.nkv * (key_blocks * a.near + sink_blocks * a.chunks)));
  const dim3 gj((unsigned)(((a.near > 1 ? a.S : a.sinks) + JOIN_KEYS - 1) / JOIN_KEYS), (unsigned)(a.n_seq * a.nkv));
  const bool join = a.near > 1 || a.chunks > 0;   // (both only where n_seq * nkv is below 512)
  if (c->head_dim == 128) {
    hipLaunchKernelGGL(win_dq_kernel<128>, gq, dim3(256), 0, s, a);
    hipLaunchKernelGGL(win_dkv_kernel<128>, gk, dim3(256), 0, s, a);
    if (join) hipLaunchKernelGGL(win_join_kernel<128>, gj, dim3(JOIN_KEYS * 64), 0, s, a);
  } else {
    hipLaunchKernelGGL(win_dq_kernel<64>, gq, dim3(256), 0, s, a);
    hipLaunchKernelGGL(win_dkv_kernel<64>, gk, dim3(256), 0, s, a);
    if (join) hipLaunchKernelGGL(win_join_kernel<64>, gj, dim3(JOIN_KEYS * 32), 0, s, a);
  }
  return hipGetLastError();
}

// a stage's configuration: B sequences of S rows in a packed projection
ah_attention_window_t stage_config(int B, int S, int nh, int d, int window, int sinks) {
  ah_attention_window_t c = {};
  c.struct_size = sizeof c;
  c.n_seq = B; c.seq_len = S; c.n_heads = nh; c.n_kv_heads = nh; c.head_dim = d; c.window = window; c.sinks = sinks;
  c.ld_q = c.ld_k = c.ld_v = c.ld_dq = c.ld_dk = c.ld_dv = 3 * nh * d;
  return c;
}
WinArgs stage_args(const ah_attention_window_t& c, const void* qkv, float* lse) {
  const size_t w = (size_t)c.n_heads * c.head_dim;
  WinArgs a = args(&c, qkv, (const bf16*)qkv + w, (const bf16*)qkv + 2 * w);
  a.lse = lse;
  return a;
}

}  // namespace

namespace ah {

hipError_t launch_attention_window_fwd(const void* qkv, void* o, float* lse, int B, int S, int nh, int d, int window, int sinks, hipStream_t s) {
  const ah_attention_window_t c = stage_config(B, S, nh, d, window, sinks);
  WinArgs a = stage_args(c, qkv, lse);
  a.out = (bf16*)o;
  return run_fwd(a, d, s);
}

hipError_t launch_attention_window_bwd(const void* qkv, const void* o, const float* lse, const void* d_o, void* dqkv, void* work, int B, int S, int nh, int d,
                                       int window, int sinks, hipStream_t s) {
  const ah_attention_window_t c = stage_config(B, S, nh, d, window, sinks);
  WinArgs a = stage_args(c, qkv, (float*)lse);
  const size_t w = (size_t)nh * d;
  a.o = (const bf16*)o; a.d_o = (const bf16*)d_o;
  a.dq = (bf16*)dqkv; a.dk = a.dq + w; a.dv = a.dq + 2 * w;
  return run_bwd(a, &c, work, s);
}

size_t attention_window_bwd_bytes(int B, int S, int nh, int d, int window, int sinks) {
  const ah_attention_window_t c = stage_config(B, S, nh, d, window, sinks);
  return bwd_bytes(&c);
}

}  // namespace ah

extern "C" int ah_attention_window_fwd(const ah_attention_window_t* c, const void* q, const void* k, const void* v, void* o, float* lse, void* stream) {
  discard_stale_hip_error();
  if (int rc = check("ah_attention_window_fwd", c, false)) return rc;
  if (!q || !k || !v || !o || !lse) return set_error(AH_EINVAL, "ah_attention_window_fwd: NULL pointer");
  if (off16(q) || off16(k) || off16(v) || off16(o) || ((uintptr_t)lse & 3)) return set_error(AH_EINVAL, "ah_attention_window_fwd: buffers must be 16-byte aligned");
  WinArgs a = args(c, q, k, v);
  a.out = (bf16*)o;
  a.lse = lse;
  return hip_status(run_fwd(a, c->head_dim, (hipStream_t)stream), "ah_attention_window_fwd");
}

extern "C" int ah_attention_window_bwd_workspace(const ah_attention_window_t* c, uint64_t* bytes) {
  if (!bytes) return set_error(AH_EINVAL, "ah_attention_window_bwd_workspace: bytes is NULL");
  if (int rc = check_sizes("ah_attention_window_bwd_workspace", c)) return rc;
  *bytes = bwd_bytes(c);
  return AH_OK;
}

extern "C" int ah_attention_window_bwd(const ah_attention_window_t* c, const void* q, const void* k, const void* v, const void* o, const float* lse,
                                       const void* d_o, void* dq, void* dk, void* dv, void* workspace, void* stream) {
  discard_stale_hip_error();
  if (int rc = check("ah_attention_window_bwd", c, true)) return rc;
  if (!q || !k || !v || !o || !lse || !d_o || !dq || !dk || !dv || !workspace) return set_error(AH_EINVAL, "ah_attention_window_bwd: NULL pointer");
  if (off16(q) || off16(k) || off16(v) || off16(o) || off16(d_o) || off16(dq) || off16(dk) || off16(dv) || ((uintptr_t)lse & 3) || ((uintptr_t)workspace & 255))
    return set_error(AH_EINVAL, "ah_attention_window_bwd: buffers must be 16-byte aligned, the workspace 256-byte");
  WinArgs a = args(c, q, k, v);
  a.o = (const bf16*)o; a.d_o = (const bf16*)d_o; a.lse = (float*)lse;
  a.dq = (bf16*)dq; a.dk = (bf16*)dk; a.dv = (bf16*)dv;
  return hip_status(run_bwd(a, c, workspace, (hipStream_t)stream), "ah_attention_window_bwd");
}
