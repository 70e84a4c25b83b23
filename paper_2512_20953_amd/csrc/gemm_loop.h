// The loop of the GEMM kernels whose tiles fill a block's registers: LDS layouts, loaders, fragment reads, the matrix instruction and the pipeline
// that gemm.hip (bf16) and muon.hip (fp16) run.
#pragma once
#include "common.h"

namespace ah {

// ---------------------------------------------------------------------------
// LDS layouts, for a tile of BK = 64 or 32 k-values (all permutations are of 16-byte pieces, the unit of the loader)
//  k-contiguous tile: [rows][BK k]; row = 2 BK bytes = BK/8 pieces; piece p of row r is stored at piece
//    p ^ ((r >> 1) & 7) (BK = 64) or p ^ ((r >> 2) & 3) (BK = 32): 16 consecutive rows hit 16 distinct 16-byte bank
//    groups for the fragment reads.  With BK = 64 a loader instruction fetches 8 rows x 128 B: full cache lines
//    (64-byte row pieces, as BK = 32 gives, cost the memory pipeline twice the requests and showed up as ~10 % of
//    MFMA utilisation where an operand is k-contiguous).
//  k-strided tile: [BK k][W cols]; row = 2W bytes.  Half a wave must cover all banks once in a transposing read.  For fragments
//    of 16 columns x 32 k it fetches 8 rows (k .. k + 3 and k + 8 .. k + 11) x 32 B: the 32-byte granule g of row k is stored at
//    granule g ^ (k & 3 | (k >> 1) & 4).  For those of 32 columns x 16 k (the smallest tiles) 4 rows x 64 B: the 64-byte granule g of row
//    k at g ^ (k & 3) (W = 64, two granules: g ^ (k >> 1 & 1)).
// A k-strided tile may gather its columns from two column ranges of the matrix (`gw` > 0: tile columns in groups of
// gw, even groups from columns c, odd groups from columns F + c): the fused gate|up product of the SwiGLU block then
// has a gate column and its up column in the same wave's accumulators.
// ---------------------------------------------------------------------------
template <int W>
__device__ __forceinline__ int granule_swizzle(int k) {  // a 64-wide row has two granules only: 4 rows x 64 B then span two bank cycles
  static_assert(W >= 64, "a row holds whole granules");
  return W >= 128 ? k & 3 : (k >> 1) & 1;
}

template <int W>
__device__ __forceinline__ int granule32_swizzle(int k) {  // of 32-byte granules
  // rows start 0, 128 (W = 192) or 64 (W = 160) bytes further along the banks than the one before
  static_assert(W % 128 == 0 || W == 192 || W == 160, "where a row begins among the banks");
  if (W % 128 == 64) return (k & 2) | ((k >> 3) & 1);
  if (W % 128 == 32) return (k >> 3) & 1;
  return (k & 3) | ((k >> 1) & 4);
}

// K16: the tile's fragments are 32 columns x 16 k
template <int BK, int W, bool KS, bool K16 = false>
__device__ __forceinline__ uint32_t loader_src_offset(int chunk, int lane, int ld, int gw = 0, int F = 0) {  // in bytes
  const int pos = chunk * 1024 + lane * 16;
  if (!KS) {
    constexpr int PR = BK / 8;                 // pieces per row
    constexpr int SH = BK == 64 ? 1 : 2;
    const int r = pos / (2 * BK), q = (pos >> 4) & (PR - 1);
    const int p = q ^ ((r >> SH) & (PR - 1));
    return (uint32_t)(r * ld + p * 8) * 2u;
  } else {
    constexpr int RB = W * 2;
    const int k = pos / RB, q = (pos % RB) >> 4;
    int p;
    if constexpr (K16) p = q ^ (granule_swizzle<W>(k) << 2);
    else p = q ^ (granule32_swizzle<W>(k) << 1);
    int col = p * 8;
    if (gw > 0) col = ((col / gw) & 1) * F + (col / (2 * gw)) * gw + col % gw;
    return (uint32_t)(k * ld + col) * 2u;
  }
}

// a W x BK (or BK x W) tile is W * BK / 512 chunks of 1 KB; wave w moves chunks w, w + NW, ...
template <int BK, int W, int NW>
__device__ __forceinline__ void issue_tile_loads(const char* __restrict__ g, uint32_t* off, char* __restrict__ lds, int wave) {
#pragma unroll
  for (int i = 0; i < W * BK / 512 / NW; i++) load16_to_lds(g, off[i], lds + (wave + NW * i) * 1024);
}

// fragment (8 k-values for row/col = lane % 32 of a 32-wide block) for k-step ks (16 k each)
template <int BK, int W, bool KS>
__device__ __forceinline__ bf16x8 read_frag(const char* __restrict__ lds, int base, int blk, int ks, int lane) {
  if (!KS) {
    constexpr int PR = BK / 8;
    constexpr int SH = BK == 64 ? 1 : 2;
    const int r = base + blk * 32 + (lane & 31);
    const int p = ks * 2 + (lane >> 5);
    const int q = p ^ ((r >> SH) & (PR - 1));
    return *(const bf16x8*)(lds + r * (2 * BK) + q * 16);
  } else {
    constexpr int RB = W * 2;
    const int k = ks * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2);
    const int c = base + blk * 32 + ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
    const int a0 = k * RB + (((c >> 5) ^ granule_swizzle<W>(k)) << 6) + ((c * 2) & 63);
    bf16x4 lo = lds_read_tr4(lds + a0);
    bf16x4 hi = lds_read_tr4(lds + a0 + 4 * RB);
    return cat4(lo, hi);
  }
}

// fragment (8 k-values for row/col = lane % 16 of a 16-wide block) for k-step ks (32 k each)
template <int BK, int W, bool KS>
__device__ __forceinline__ bf16x8 read_frag32(const char* __restrict__ lds, int base, int blk, int ks, int lane) {
  if (!KS) {
    constexpr int PR = BK / 8;
    constexpr int SH = BK == 64 ? 1 : 2;
    const int r = base + blk * 16 + (lane & 15);
    const int p = ks * 4 + (lane >> 4);
    const int q = p ^ ((r >> SH) & (PR - 1));
    return *(const bf16x8*)(lds + r * (2 * BK) + q * 16);
  } else {
    constexpr int RB = W * 2;
    const int k = ks * 32 + (lane >> 4) * 8 + ((lane & 15) >> 2);
    const int c = base + blk * 16 + 4 * (lane & 3);
    const int a0 = k * RB + (((c >> 4) ^ granule32_swizzle<W>(k)) << 5) + ((c * 2) & 31);
    bf16x4 lo = lds_read_tr4(lds + a0);
    bf16x4 hi = lds_read_tr4(lds + a0 + 4 * RB);
    return cat4(lo, hi);
  }
}

// Fragments of one 32-wide k-step for the wave's sub-tile.
template <int BK, int BM, int BN, int WGM, int WGN, bool AKS, bool BKS>
struct Frags32 {
  static constexpr int TM = BM / WGM / 16, TN = BN / WGN / 16;
  bf16x8 a[TM], b[TN];
  __device__ __forceinline__ void load(const char* __restrict__ cA, const char* __restrict__ cB, int ks, int wm, int wn, int lane) {
#pragma unroll
    for (int t = 0; t < TM; t++) a[t] = read_frag32<BK, BM, AKS>(cA, wm * (BM / WGM), t, ks, lane);
#pragma unroll
    for (int t = 0; t < TN; t++) b[t] = read_frag32<BK, BN, BKS>(cB, wn * (BN / WGN), t, ks, lane);
  }
};

// Fragments of one 16-wide k-step for the wave's sub-tile.
template <int BK, int BM, int BN, int WGM, int WGN, bool AKS, bool BKS>
struct Frags {
  static constexpr int TM = BM / WGM / 32, TN = BN / WGN / 32;
  bf16x8 a[TM], b[TN];
  __device__ __forceinline__ void load(const char* __restrict__ cA, const char* __restrict__ cB, int ks, int wm, int wn, int lane) {
#pragma unroll
    for (int t = 0; t < TM; t++) a[t] = read_frag<BK, BM, AKS>(cA, wm * (BM / WGM), t, ks, lane);
#pragma unroll
    for (int t = 0; t < TN; t++) b[t] = read_frag<BK, BN, BKS>(cB, wn * (BN / WGN), t, ks, lane);
  }
};

// Scheduling hint for one k-step: between consecutive MFMAs (NM of them) place
// the NV global->LDS loads and the NR LDS reads issued for later steps, the LDS
// reads within the first three quarters so their latency is covered by the rest.
// Masks: 0x020 = vector memory read, 0x100 = LDS read, 0x008 = MFMA.
template <int I, int NM, int NR, int NV, int SPAN = (NM * 3 / 4 > 0 ? NM * 3 / 4 : 1)>
__device__ __forceinline__ void interleave() {
  if constexpr (I < NM) {
    constexpr int v = (I + 1) * NV / NM - I * NV / NM;
    constexpr int r = I < SPAN ? (I + 1) * NR / SPAN - I * NR / SPAN : 0;
    if constexpr (v > 0) __builtin_amdgcn_sched_group_barrier(0x020, v, 0);
    if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    interleave<I + 1, NM, NR, NV, SPAN>();
  }
}

template <bool F16, int BK, int BM, int BN, int WGM, int WGN, bool AKS, bool BKS>
__device__ __forceinline__ void mma_step(const Frags<BK, BM, BN, WGM, WGN, AKS, BKS>& f, f32x16 (&acc)[BM / WGM / 32][BN / WGN / 32]) {
  constexpr int TM = BM / WGM / 32, TN = BN / WGN / 32;
#pragma unroll
  for (int tm = 0; tm < TM; tm++)
#pragma unroll
    for (int tn = 0; tn < TN; tn++) {
      if constexpr (F16) {
        typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
        acc[tm][tn] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, f.b[tn]), __builtin_bit_cast(f16x8, f.a[tm]), acc[tm][tn], 0, 0, 0);
      } else {
        acc[tm][tn] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.b[tn], f.a[tm], acc[tm][tn], 0, 0, 0);
      }
    }
}

// The 16 x 16 x 32 instruction does the flops of the 32 x 32 x 16 one at less power, which is what bounds a loop that keeps the matrix
// pipelines busy: register-resident on random operands 2.06 against 1.78 PFLOP/s (2.44 both on zeros).  In the loops below, with
// the same bytes through LDS: 8192^3 NT 847 -> 811 us, 2048 x 5120 x 20480 394 -> 372, 2048^3 (128 x 128 tiles) 23.2 -> 20.5.
// As assembly, because the compiler's form has a destination of its own: with all 256 accumulation registers taken it
// moves 12 .. 60 of 64 accumulators to other registers and back in every k-step.  What the compiler then does not know of is
// kept here: an accumulator is used again one k-step (16 or more matrix instructions) later, and read 16 wait states
// after the loops (gemm_tile); operands come from LDS reads, which it does wait for.
// F16: the fragments hold fp16 numbers (the same rate; moved as 16-bit numbers everywhere else).
template <bool F16>
__device__ __forceinline__ void mma16(f32x4& acc, const bf16x8& a, const bf16x8& b) {
  if constexpr (F16) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(b), "v"(a));
  else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(b), "v"(a));
}

// One 32-wide k-step as a fixed sequence of slots: a matrix instruction on the fragments f each, and before it what falls on the slot
// of the NV loads (load(i)) and of the reads of the next step's fragments fn, which take the first three quarters (in the first
// 3, 4 or 8 eighths 1.005, 1.004 and 1.014 times as long, geometric mean over 56 products).  The loads of a short step, and those
// of the weight gradient, whose operands come from far away, go out in its first half: 4096 x 1024 x 4096 36.3 -> 35.0 us (NT), 2048^3
// 22.9 -> 22.1 (NN), 4096^3 111.8 -> 109.9 (TN); evenly they are 1 % better in the larger forward and input-gradient steps.
// In the weight gradient's short steps (TN, up to 32 matrix instructions) the reads, two to a fragment, take all slots but the last two: beside the loads
// the first three quarters made a wave that is alone on its SIMD wait for them.  Launches of up to a tile per CU, against the 32x32x16 loop that was
// here before (geometric means, three boxes): 128 x 256 and 256 x 128 1.04 -> 0.98 .. 1.00, 128 x 128 1.03 -> 1.01; 3840 x 1152 x 5120 51.8 us there, 57.1 -> 53.6 here.
template <int BK, int BM, int BN, int WGM, int WGN, bool AKS, bool BKS, int NV, bool F16 = false, class L>
__device__ __forceinline__ void k_step(const L& load, const char* __restrict__ nA, const char* __restrict__ nB, int ks,
                                       const Frags32<BK, BM, BN, WGM, WGN, AKS, BKS>& f, Frags32<BK, BM, BN, WGM, WGN, AKS, BKS>& fn,
                                       f32x4 (&acc)[BM / WGM / 16][BN / WGN / 16], int wm, int wn, int lane) {
  constexpr int TM = BM / WGM / 16, TN = BN / WGN / 16, NM = TM * TN, NF = TM + TN, SPAN = AKS && BKS && NM <= 32 ? NM - 2 : NM * 3 / 4;
  constexpr int VSPAN = (AKS && BKS) || NM <= 16 ? NM / 2 : NM;
#pragma unroll
  for (int i = 0; i < NM; i++) {
#pragma unroll
    for (int v = i * NV / VSPAN; v < (i + 1) * NV / VSPAN && v < NV; v++) load(v);
#pragma unroll
    for (int r = i * NF / SPAN; r < (i + 1) * NF / SPAN && r < NF; r++) {
      if (r < TN) fn.b[r] = read_frag32<BK, BN, BKS>(nB, wn * (BN / WGN), r, ks, lane);
      else fn.a[r - TN] = read_frag32<BK, BM, AKS>(nA, wm * (BM / WGM), r - TN, ks, lane);
    }
    mma16<F16>(acc[i / TN][i % TN], f.a[i / TN], f.b[i % TN]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

namespace k64 {
constexpr int BK = 64;  // k-extent of one operand tile in LDS (128 bytes per row of a k-contiguous operand: whole cache lines)
// DEPTH: k-blocks between the start of the second operand's loads and the wait for them (the first operand's: half a block more), for
// which the ring has DEPTH + 1 buffers for tiles of the first and DEPTH for those of the second.
//  256 x 256 tiles: 2, all of a CU's 160 KB.  128 x 256 and 256 x 128: 3, the same.
//  128 x 128: 2 where two blocks share a CU (80 KB).  In a launch of at most 256 blocks, which have a CU each, 3 (112 KB): a k-block
//    is 512 clocks of MFMA, and with 2 the loop waited for operands that come from HBM.  4096 x 1024 x 4096 49.4 -> 39.7 us from HBM,
//    33.7 -> 32.9 from the memory-side cache (NN); 2048^3 28.1 -> 23.0 and 20.8 -> 19.3 (NT); 4 is no better (40.3, 23.4).  Beside a
//    second stream (GemmArgs::beside) it keeps that stream's blocks off the CUs: BERT-Large stage with a group of 1, 1892 -> 1992 us.
template <int BM, int BN, int DEPTH, bool BF>
constexpr int ring_bytes() { return ((DEPTH + 1) * (BF ? BN : BM) + DEPTH * (BF ? BM : BN)) * 2 * BK; }

// The pipeline.  F is the operand whose tiles go first, S the other one (see b_first); the tiles of k-block j are F_j and S_j.
// A k-block is two k-steps of 32; fragments are double-buffered in registers (f0, f1), the fragments
// of a k-step being read from LDS under the MFMAs of the step before.  So all fragments of k-block j are in registers at its
// middle: there the one barrier per k-block frees its two buffers, and, after a wait that counts the wave's own loads down to the
// tiles issued after S_{j+1}, says that k-block j+1 has landed for the whole block.  The second half of k-block j starts the loads of
// S_{j + DEPTH} into the buffer of S_j, the first half those of F_{j + DEPTH} into that of F_{j-1}.
// The two halves are separate functions so that within each the buffer written is not one of the buffers read:
// the restrict qualifiers then tell the compiler that LDS reads never wait for the loads in flight.

// F has the longer way to go.  The weights (B of the forward and input-gradient products) stream from HBM while
// the activations were just written and mostly sit in the caches, so B goes first, unless its tiles are the larger ones, of which
// the ring has no room for one more.
template <int BM, int BN, bool AKS>
constexpr bool b_first() { return !AKS && BN <= BM; }

// First k-step of k-block j (f0 holds its fragments): starts the loads of F_{j + DEPTH} and reads the
// fragments of the second one.
template <int BM, int BN, int WGM, int WGN, bool AKS, bool BKS, bool F16>
__device__ __forceinline__ void half_even(const char* gF, uint32_t* offF, char* __restrict__ fill, const char* __restrict__ cA,
                                          const char* __restrict__ cB, const Frags32<BK, BM, BN, WGM, WGN, AKS, BKS>& f0,
                                          Frags32<BK, BM, BN, WGM, WGN, AKS, BKS>& f1, f32x4 (&acc)[BM / WGM / 16][BN / WGN / 16],
                                          int wave, int wm, int wn, int lane) {
  constexpr int NW = WGM * WGN, WF = b_first<BM, BN, AKS>() ? BN : BM;
  k_step<BK, BM, BN, WGM, WGN, AKS, BKS, WF / 8 / NW, F16>([&](int i) { load16_to_lds(gF, offF[i], fill + (wave + NW * i) * 1024); }, cA, cB, 1, f0, f1,
                                                      acc, wm, wn, lane);
}

// Second k-step of k-block j: waits for k-block j+1 (nA, nB), starts the loads of S_{j + DEPTH} into the buffer of S_j, whose
// fragments all waves hold by now, and reads the first fragments of k-block j+1.
template <int BM, int BN, int WGM, int WGN, bool AKS, bool BKS, int DEPTH, bool F16>
__device__ __forceinline__ void half_odd(const char* gS, uint32_t* offS, char* __restrict__ fill, const char* __restrict__ nA,
                                         const char* __restrict__ nB, Frags32<BK, BM, BN, WGM, WGN, AKS, BKS>& f0,
                                         const Frags32<BK, BM, BN, WGM, WGN, AKS, BKS>& f1, f32x4 (&acc)[BM / WGM / 16][BN / WGN / 16],
                                         int wave, int wm, int wn, int lane) {
  constexpr int NW = WGM * WGN, WF = b_first<BM, BN, AKS>() ? BN : BM, WS = b_first<BM, BN, AKS>() ? BM : BN;
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(((DEPTH - 1) * WF + (DEPTH - 2) * WS) / 8 / NW));
  __builtin_amdgcn_s_barrier();
  k_step<BK, BM, BN, WGM, WGN, AKS, BKS, WS / 8 / NW, F16>([&](int i) { load16_to_lds(gS, offS[i], fill + (wave + NW * i) * 1024); }, nA, nB, 0, f1, f0,
                                                      acc, wm, wn, lane);
}

// The whole loop: acc += the block's tile of the product of A (from gA on, rows or, AKS, k-rows lda elements apart) and B over K, a multiple of 128.  The wave's
// redundant tail loads are still in flight behind it.  GW, F: see the k-strided tiles above.
template <int BM, int BN, int WGM, int WGN, bool AKS, bool BKS, int DEPTH, bool F16, int GW = 0>
__device__ __forceinline__ void run(const char* gA, const char* gB, int lda, int ldb, int F, int K, char* ring, f32x4 (&acc)[BM / WGM / 16][BN / WGN / 16],
                                    int wave, int wm, int wn, int lane) {
  constexpr int NW = WGM * WGN;
  constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW;     // loads per tile per wave
  const size_t stepA = (AKS ? (size_t)BK * lda : (size_t)BK) * 2;  // bytes per k-block
  const size_t stepB = (BKS ? (size_t)BK * ldb : (size_t)BK) * 2;

  uint32_t offA[LA], offB[LB];
#pragma unroll
  for (int i = 0; i < LA; i++) offA[i] = loader_src_offset<BK, BM, AKS>(wave + NW * i, lane, lda);
#pragma unroll
  for (int i = 0; i < LB; i++) offB[i] = loader_src_offset<BK, BN, BKS>(wave + NW * i, lane, ldb, GW, F);

  // K is a multiple of 128: an even number of k-blocks.  Past the end the last k-block is fetched again into
  // dead buffers, which keeps the number of loads in flight uniform for the counted wait.
  // F = the operand whose tiles go first, S = the other one.
  constexpr bool BF = b_first<BM, BN, AKS>();
  constexpr int WF = BF ? BN : BM, WS = BF ? BM : BN;
  const char* gF = BF ? gB : gA;
  const char* gS = BF ? gA : gB;
  const size_t stepF = BF ? stepB : stepA, stepS = BF ? stepA : stepB;
  uint32_t* offF = BF ? offB : offA;
  uint32_t* offS = BF ? offA : offB;
  const int np = K / BK, lastp = np - 1;
  // Ring: F_j in buffer j % (DEPTH + 1) of WF rows, S_j behind those in buffer j % DEPTH of WS rows.  During k-block j the tiles
  // F_{j + DEPTH} and S_{j + DEPTH} are fetched.
  constexpr int FB = WF * 2 * BK, SB = WS * 2 * BK, NF = DEPTH + 1, NSB = DEPTH;
  char* const ringS = ring + NF * FB;
#pragma unroll
  for (int t = 0; t < DEPTH; t++) {
    issue_tile_loads<BK, WF, NW>(gF + (size_t)min(t, lastp) * stepF, offF, ring + t * FB, wave);
    issue_tile_loads<BK, WS, NW>(gS + (size_t)min(t, lastp) * stepS, offS, ringS + t * SB, wave);
  }
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0((DEPTH - 1) * (WF + WS) / 8 / NW));
  __builtin_amdgcn_s_barrier();

  Frags32<BK, BM, BN, WGM, WGN, AKS, BKS> f0, f1;
  f0.load(BF ? ringS : ring, BF ? ring : ringS, 0, wm, wn, lane);
  int jf = 0, js = 0;  // buffers of F_j and S_j
  int j = 0;
  do {   // (np >= 2; a loop that might not run would have its accumulators copied at its exit, ahead of the wait below)
    const int nf = jf + 1 == NF ? 0 : jf + 1;    // F_{j+1}
    const int ns = js + 1 == NSB ? 0 : js + 1;   // S_{j+1}
    const int ff = jf == 0 ? NF - 1 : jf - 1;    // F_{j + DEPTH}: into the buffer of F_{j-1}; S_{j + DEPTH} goes into that of S_j
    const char *cF = ring + jf * FB, *cS = ringS + js * SB, *nxF = ring + nf * FB, *nxS = ringS + ns * SB;
    const char* pS = gS + (size_t)min(j + DEPTH, lastp) * stepS;
    const char* pF = gF + (size_t)min(j + DEPTH, lastp) * stepF;
    half_even<BM, BN, WGM, WGN, AKS, BKS, F16>(pF, offF, ring + ff * FB, BF ? cS : cF, BF ? cF : cS, f0, f1, acc, wave, wm, wn, lane);
    half_odd<BM, BN, WGM, WGN, AKS, BKS, DEPTH, F16>(pS, offS, ringS + js * SB, BF ? nxS : nxF, BF ? nxF : nxS, f0, f1, acc, wave, wm, wn, lane);
    jf = nf;
    js = ns;
  } while (++j < np);
}

}  // namespace k64

namespace ksplit {
// The pipeline of the tiles whose waves share a sub-tile and split the k axis: of the four k-steps of a 64-wide
// k-block, wave wk takes 4 / WGK.  The partial sums meet in the epilogue's staging strips.
//  64 x 64 with four shares and 64 x 128 with two are for outputs of fewer than 256 tiles of 128 x 128.  Such a launch
//    lasts as long as one block's chain of k-blocks; these have four (two) times the blocks, and a chain a quarter as
//    long.  256 x 256 x 1024: 9.3 -> 5.5 us, 1024 x 1024 x 2048: 21.6 -> 8.8, 2048 x 1024 x 2048: 21.6 -> 13.2 (NT).
//  128 x 128 with four shares: every wave owns the whole tile, so a k-block costs 32 KB of fragment reads instead of
//    the 64 KB of four 64 x 64 sub-tiles.  Beside 512 clocks of MFMA the CU's path to and from the LDS was busy ~950
//    (reads at 128 B per clock, the 32 KB fill at 1.7 times its bytes), now ~690; what bounds it then is the rate at
//    which the loads arrive (64 B per clock and CU).  2048 x 2048 x 8192: 76 -> 61 us (NT; against the 32x32x16 loop:
//    the present one has closed the gap, see kWholeCuMinK, and the tile is there for its shorter sums).  The epilogue moves four
//    times the partial sums (3 us): at k = 2048 the two are level, and where two blocks of the 64 x 64 sub-tiles share
//    a CU (more than 256 tiles) those are faster; in the weight gradient, whose transposing reads are half as long,
//    there is no gain (67 against 67 us), so it is not built there.
constexpr int BK = 64;
template <int BM, int BN> constexpr int stage_bytes() { return (BM + BN) * 2 * BK; }
// ring depth: all of a CU's 160 KB for the 128 x 128 tile, half of it for the small ones (two blocks share a CU): 5, 3 and 5 stages
template <int BM, int BN> constexpr int stages() { return (BM * BN < 128 * 128 ? 81920 : 163840) / stage_bytes<BM, BN>(); }

// Second (or only) part of a k-block: the block's slot is free (its fragments are in registers, the barrier is
// passed), so the loads of the stage NS ahead go there while the next stage's first fragments are read.  The two
// slots are distinct: the restrict qualifiers keep the LDS reads from waiting for the loads in flight.
template <int BM, int BN, int WGM, int WGN, bool AKS, bool BKS, bool F16 = false>
__device__ __forceinline__ void last_step(const char* pA, const char* pB, uint32_t* offA, uint32_t* offB, char* __restrict__ fill,
                                          const char* __restrict__ next, int ks, const Frags<BK, BM, BN, WGM, WGN, AKS, BKS>& f,
                                          Frags<BK, BM, BN, WGM, WGN, AKS, BKS>& fn, f32x16 (&acc)[BM / WGM / 32][BN / WGN / 32], int wave,
                                          int wm, int wn, int lane) {
  constexpr int TM = BM / WGM / 32, TN = BN / WGN / 32, NW = 4;
  constexpr int NR = TM * (AKS ? 2 : 1) + TN * (BKS ? 2 : 1), NM = TM * TN, LPS = (BM + BN) / 8 / NW;
  issue_tile_loads<BK, BM, NW>(pA, offA, fill, wave);
  issue_tile_loads<BK, BN, NW>(pB, offB, fill + BM * 2 * BK, wave);
  fn.load(next, next + BM * 2 * BK, ks, wm, wn, lane);
  mma_step<F16, BK, BM, BN, WGM, WGN, AKS, BKS>(f, acc);
  interleave<0, NM, NR, LPS, NM / 2>();
}

// First part of a two-step k-block
template <int BM, int BN, int WGM, int WGN, bool AKS, bool BKS, bool F16 = false>
__device__ __forceinline__ void first_step(const char* __restrict__ cur, int ks, const Frags<BK, BM, BN, WGM, WGN, AKS, BKS>& f,
                                           Frags<BK, BM, BN, WGM, WGN, AKS, BKS>& fn, f32x16 (&acc)[BM / WGM / 32][BN / WGN / 32], int wm,
                                           int wn, int lane) {
  constexpr int TM = BM / WGM / 32, TN = BN / WGN / 32;
  constexpr int NR = TM * (AKS ? 2 : 1) + TN * (BKS ? 2 : 1), NM = TM * TN;
  fn.load(cur, cur + BM * 2 * BK, ks, wm, wn, lane);
  mma_step<F16, BK, BM, BN, WGM, WGN, AKS, BKS>(f, acc);
  interleave<0, NM, NR, 0, NM / 2>();
}

// The whole loop where each of four waves takes one k-step in four of the whole tile, over one piece of the k axis (K a multiple of 128): acc are the wave's partial sums.
// The wave's redundant tail loads are still in flight behind it.  PARTS products of the same sizes can follow each other into the same sums without a pause; in front of the last
// of them the sums are multiplied by `factor`.
template <int BM, int BN, bool AKS, bool BKS, bool F16, int PARTS = 1>
__device__ __forceinline__ void run(const char* const (&gA)[PARTS], const char* const (&gB)[PARTS], int lda, int ldb, int K, char* ring, f32x16 (&acc)[BM / 32][BN / 32], int wave,
                                    int lane, float factor = 1.f) {
  constexpr int STAGE = stage_bytes<BM, BN>(), NS = stages<BM, BN>(), NW = 4, LA = BM / 8 / NW, LB = BN / 8 / NW, LPS = LA + LB;
  const size_t stepA = (AKS ? (size_t)BK * lda : (size_t)BK) * 2, stepB = (BKS ? (size_t)BK * ldb : (size_t)BK) * 2;   // bytes per k-block
  uint32_t offA[LA], offB[LB];
#pragma unroll
  for (int i = 0; i < LA; i++) offA[i] = loader_src_offset<BK, BM, AKS, true>(wave + NW * i, lane, lda);
#pragma unroll
  for (int i = 0; i < LB; i++) offB[i] = loader_src_offset<BK, BN, BKS, true>(wave + NW * i, lane, ldb);
  // The stage to be fetched next; past the last one that stage is fetched again into dead slots, which keeps the number of loads in flight uniform for the counted wait.
  const int nk = K / BK;
  const char *pA = gA[0], *pB = gB[0];
  int fetched = 1, part = 0;
  auto advance = [&]() {
    bool more = fetched < nk;
    fetched++;
    if constexpr (PARTS > 1) {
      if (!more && part < PARTS - 1) {
        part++;
#pragma unroll
        for (int i = 1; i < PARTS; i++) {
          if (part == i) { pA = gA[i]; pB = gB[i]; }
        }
        fetched = 1;
        return;
      }
    }
    pA = more ? pA + stepA : pA;
    pB = more ? pB + stepB : pB;
  };
#pragma unroll
  for (int t = 0; t < NS; t++) {
    issue_tile_loads<BK, BM, NW>(pA, offA, ring + t * STAGE, wave);
    issue_tile_loads<BK, BN, NW>(pB, offB, ring + t * STAGE + BM * 2 * BK, wave);
    advance();
  }
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0((NS - 1) * LPS));
  __builtin_amdgcn_s_barrier();
  Frags<BK, BM, BN, 1, 1, AKS, BKS> f0, f1;
  f0.load(ring, ring + BM * 2 * BK, wave, 0, 0, lane);
  int c = 0;  // ring slot of k-block j
  for (int j = 0; j < PARTS * nk; j += 2) {
    const int n = c + 1 == NS ? 0 : c + 1, n2 = n + 1 == NS ? 0 : n + 1;
    if constexpr (PARTS > 1) {
      if (j == (PARTS - 1) * nk) {
#pragma unroll
        for (int tm = 0; tm < BM / 32; tm++)
#pragma unroll
          for (int tn = 0; tn < BN / 32; tn++) acc[tm][tn] *= factor;
      }
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0((NS - 2) * LPS));
    __builtin_amdgcn_s_barrier();
    last_step<BM, BN, 1, 1, AKS, BKS, F16>(pA, pB, offA, offB, ring + c * STAGE, ring + n * STAGE, wave, f0, f1, acc, wave, 0, 0, lane);
    advance();
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0((NS - 2) * LPS));
    __builtin_amdgcn_s_barrier();
    last_step<BM, BN, 1, 1, AKS, BKS, F16>(pA, pB, offA, offB, ring + n * STAGE, ring + n2 * STAGE, wave, f1, f0, acc, wave, 0, 0, lane);
    advance();
    c = n2;
  }
}

}  // namespace ksplit

}  // namespace ah
