// Device helpers of the attention kernels: tiles of 64 rows in LDS, their fragments as operands of MFMA 32x32x16, loads into LDS
// by assembly, results stored as whole rows.
#pragma once
#include "common.h"
#include <type_traits>

namespace ah {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr int NSLOT = 2;  // ring slots of the kernels that take one tile after the other, and of the 64-row forward kernel

// nothing is scheduled across this point
#define AH_SCHED_FENCE() __builtin_amdgcn_sched_barrier(0)
// Issue priority of the wave among the waves of its SIMD: raised for the runs of matrix instructions, so that the
// other waves' vector work (softmax, masks, conversions) fills in behind them instead of delaying them.  Used by the unmasked
// 64-wide forward kernel, with / without: 8 x 16 x 512 12.6 / 13.4 us, 2 x 16 x 2048 38.2 / 40.6, 1 x 9 x 4096 56.7 / 68.2, 1 x 32 x 4096
// 141.5 / 145.5, 16 x 16 x 512 24.8 / 24.1; the kernels that run in slots gain nothing from it.
#define AH_PRIO(p) __builtin_amdgcn_s_setprio(p)

// All but the last n of the wave's loads have landed, for the whole block, and every wave is done with its LDS reads.  The
// empty statement keeps the compiler from moving LDS reads above the barrier: it does not know that the loads (which
// are assembly) write what they read.
#define AH_LANDED(n)                                  \
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(n));    \
  __builtin_amdgcn_s_barrier();                       \
  asm volatile("" ::: "memory")
#define AH_NEXT_TILE() AH_LANDED(0)

// LDS tile [64 rows][D] bf16.  16-byte piece p of row r is stored at piece
// swz(r, p): conflict-free both for 16-byte reads down a column of pieces (16 rows
// at a time must hit 16 different pieces of the 256 bytes that the banks span) and
// for the transposing reads of 4 rows x 64 bytes.  With D = 64 the banks hold two
// rows: rows 2i and 2i + 1 share a permutation, the eight values of i have eight
// different ones, and the low bit of i moves a piece to the other 64 bytes.
template <int D>
__device__ __forceinline__ int swz(int r, int p) {
  if (D == 128) return p ^ ((r & 3) << 2) ^ ((r >> 2) & 3);
  return p ^ ((r << 1) & 4) ^ ((r >> 2) & 3);
}

template <int D>
__device__ __forceinline__ uint32_t tile_src_offset(int chunk, int lane, int ld) {
  constexpr int RB = 2 * D;
  const int pos = chunk * 1024 + lane * 16;
  const int r = pos / RB, q = (pos % RB) >> 4;
  return (uint32_t)(r * ld + swz<D>(r, q) * 8) * 2u;  // bytes
}

// The loads into LDS as assembly: for the builtin the compiler assumes an access that may return out of order with LDS
// reads, and waits for all of a wave's LDS reads (lgkmcnt(0)) before the first use of any of them while such a load is in
// flight.  Nothing is returned to a register; the kernels wait for these loads by count before they pass a barrier.  M0 (the
// LDS address) is set in the same statement and named as overwritten.  Against the builtin, forward / backward:
// 2 x 16 x 2048 x 128 causal 51.1 / 163.2 -> 49.7 / 160.2 us, 2 x 16 x 2048 x 64 causal 29.5 / 86.4 -> 28.7 / 83.0 (same bits).
__device__ __forceinline__ void load4(const void* base, uint32_t off, void* lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds_offset(lds)), "v"(off), "s"(base) : "memory", "m0");
}

template <int D>
__device__ __forceinline__ void issue_tile(const bf16* __restrict__ g, const uint32_t* off, char* lds, int wave) {
#pragma unroll
  for (int i = 0; i < D / 32; i++) load16_to_lds_uncounted(g, off[i], lds + (wave + 4 * i) * 1024);
}

// 32 rows
template <int D>
__device__ __forceinline__ void issue_half(const bf16* __restrict__ g, const uint32_t* off, char* lds, int wave) {
#pragma unroll
  for (int i = 0; i < D / 64; i++) load16_to_lds_uncounted(g, off[i], lds + (wave + 4 * i) * 1024);
}

// 8 consecutive head-dim values (k-step ks, half hf) of row r
template <int D>
__device__ __forceinline__ bf16x8 frag_rowmajor(const char* __restrict__ t, int r, int ks, int hf) {
  return *(const bf16x8*)(t + r * (2 * D) + swz<D>(r, 2 * ks + hf) * 16);
}

// column (dt*32 + lane%32) of rows rbase..rbase+3 and rbase+8..rbase+11
template <int D>
__device__ __forceinline__ bf16x8 frag_transposed(const char* __restrict__ t, int rbase, int dt, int lane) {
  const int r = rbase + ((lane & 15) >> 2);
  const int c = dt * 32 + ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
  bf16x4 lo = lds_read_tr4(t + r * (2 * D) + swz<D>(r, c >> 3) * 16 + (c & 7) * 2);
  bf16x4 hi = lds_read_tr4(t + (r + 8) * (2 * D) + swz<D>(r + 8, c >> 3) * 16 + (c & 7) * 2);
  return cat4(lo, hi);
}

__device__ __forceinline__ bf16x8 pack8(const f32x16& a, int s2) {
  bf16x8 p;
#pragma unroll
  for (int j = 0; j < 8; j++) p[j] = f2bf(a[8 * s2 + j]);
  return p;
}

// max / sum of a value over the two lanes (l, l + 32) that share a query: one exchange of the halves of two registers
// instead of a trip through the LDS crossbar
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// A wave's result of 32 rows x D, val(dt, r) being the element of row lane % 32 and column dt * 32 + 8 (r / 4) + 4 (lane / 32) + r % 4,
// to 32 rows of the output.  It passes through a strip of LDS of the wave's own and leaves as whole rows, 16 bytes a lane: stored
// straight from the registers, an instruction writes 16 bytes to each of 32 rows (dK and dV of 128 keys: 4.5 us, now 1.45).
template <int D> constexpr int strip_bytes() { return 32 * 2 * D; }
template <int D, class F>
__device__ __forceinline__ void store_rows(const F& val, char* strip, bf16* __restrict__ dst, size_t ld, int lane) {
  constexpr int RB = 2 * D, PPR = D / 8, RPI = 64 / PPR;   // bytes of a row, 16-byte pieces of a row, rows per store
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
  for (int it = 0; it < 32 / RPI; it++) *(bf16x8*)(dst + (size_t)(row + it * RPI) * ld + piece * 8) = *(const bf16x8*)(strip + at(row + it * RPI, piece));
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ float fexp2(float x) { return __builtin_amdgcn_exp2f(x); }

// The running maximum is only raised when a new score exceeds it by more than this many powers of two:
// probabilities are then at most 2^8 instead of 1, which fp32 sums and the bf16 operand of the second
// product hold with unchanged relative accuracy, and the rescaling of the output accumulator -- the
// largest block of vector arithmetic in the loop -- runs on the first tile only in practice.
constexpr float RESCALE_SLACK = 8.f;

// Byte offsets of a lane's fragments in a tile: row[ks] as frag_rowmajor, lo[dt] and hi[dt] as frag_transposed, for rows that
// start at a multiple of 16 (the permutation depends on the row's low four bits only), so that every other fragment is a
// compile-time distance away.
template <int D>
struct LaneOffs {
  int row[D / 16], lo[D / 32], hi[D / 32];
  __device__ __forceinline__ LaneOffs(int lane) {
    const int r = lane & 31, hf = lane >> 5, rt = 4 * hf + ((lane & 15) >> 2);
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++) row[ks] = r * (2 * D) + swz<D>(r, 2 * ks + hf) * 16;
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++) {
      const int c = dt * 32 + ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
      lo[dt] = rt * (2 * D) + swz<D>(rt, c >> 3) * 16 + (c & 7) * 2;
      hi[dt] = (rt + 8) * (2 * D) + swz<D>(rt + 8, c >> 3) * 16 + (c & 7) * 2;
    }
  }
  __device__ __forceinline__ bf16x8 rows(const char* t, int rb, int ks) const { return *(const bf16x8*)(t + row[ks] + rb * (2 * D)); }
  __device__ __forceinline__ bf16x8 cols(const char* t, int rb, int dt) const {
    return cat4(lds_read_tr4(t + lo[dt] + rb * (2 * D)), lds_read_tr4(t + hi[dt] + rb * (2 * D)));
  }
};

// f(integral_constant<int, I>) for I .. N - 1, unrolled
template <int I, int N, class F>
__device__ __forceinline__ void unrolled(const F& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unrolled<I + 1, N>(f);
  }
}

// delta_q = sum_c dO[q, c] O[q, c] for the lane's query: the lane holds half of the row of dO as MFMA fragments
// (columns ks * 16 + hf * 8 ..), reads the same columns of O, and the two lanes of a query add their halves.
// The dQ kernels compute it for their own queries and leave it in `delta` for the dK/dV kernel, which runs after them.
template <int D>
__device__ __forceinline__ float row_delta(const bf16x8 (&dof)[D / 16], const bf16* __restrict__ orow, int hf) {
  float s = 0.f;
#pragma unroll
  for (int ks = 0; ks < D / 16; ks++) {
    const bf16x8 ov = *(const bf16x8*)(orow + ks * 16 + hf * 8);
#pragma unroll
    for (int j = 0; j < 8; j++) s = __builtin_fmaf(bf2f(dof[ks][j]), bf2f(ov[j]), s);
  }
  return s + __shfl_xor(s, 32, 64);
}

}  // namespace
}  // namespace ah
