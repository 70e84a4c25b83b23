// Embedding of tokens and its gradient (declared in include/ah_ops.h).  Bound by HBM: forward reads a row of the table for each token and
// writes one (8192 x 4096 with positions 28 us: 4.0 TB/s of what it cannot do without), backward reads the rows' gradients and writes (or adds to) the rows of the table that
// occur (8190 x 4096, added: 64 us, of which 44 for the sums at 4.2 TB/s; 3001 x 1001 in fp32, 32000 rows written: 36).
//
// Backward: the tokens' numbers are sorted by token, stably (up to 16384 of them by counting each one's place, else by digits of 8 bits from the lowest on), so that the rows that
// a row of the table is the sum of lie behind each other.  The sorted list is cut into chunks; a block adds up a chunk, writes each sum that begins and ends in it, and leaves the
// sums that reach over its ends, at most one on either side, as partial sums, which a second kernel adds up in the chunks' order.  So the work of a
// block does not depend on how often a token occurs, and no row is written by two blocks.
#include "ah_ops.h"
#include "capi_util.h"
#include "wide.h"

#include <algorithm>
#include <cmath>

using namespace ah;

namespace {

constexpr int NT = 256, NW = NT / 64, kMaxRows = 1 << 25, kMaxVocab = 1 << 30, kMaxWidth = 65536;
constexpr int kFlight = 2;                             // forward: pieces of a row that a lane has in flight
constexpr int kMaxChunks = 2048, kMinChunk = 16, kAhead = 4, kJoin = 16;
constexpr int kRowThreads = 1024;
// Tokens up to which places are counted (rank_kernel): quadratic, but one launch.  Whole calls, counted and by digits, added: 8192 tokens x 4096 64, 90 us; 12288 96, 115; 16384 122, 133; 16384 x 1024
// over 2048 rows 47, 55.
constexpr int kSmall = 16384;
constexpr int kItems = 16, kSortBlock = NT * kItems;   // numbers that a block of the sort takes

struct FwdArgs {
  const void *table, *tokens, *pos_table;
  const int32_t* positions;
  void* y;
  size_t ld_table, ld_y, ld_pos;
  int T, vocab, width, n_pos, S, bits;
  float scale;
};

// 2^lanes_log2 lanes to a row, V elements each and time, kFlight times in flight (with two rows at once level: 8192 x 4096 with positions 28 us)
template <class TT, class AT, int V>
__global__ __launch_bounds__(NT) void embedding_fwd_kernel(FwdArgs a, int lanes_log2) {
  const int lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1), rows = NT >> lanes_log2;
  for (int64_t t = (int64_t)blockIdx.x * rows + (threadIdx.x >> lanes_log2); t < a.T; t += (int64_t)gridDim.x * rows) {
    const int64_t token = load_index(a.tokens, t, a.bits);
    const int pos = a.pos_table ? (a.positions ? a.positions[t] : (int)(t % a.S)) : 0;
    const bool none = token == -1, bad = (!none && (uint64_t)token >= (uint64_t)a.vocab) || (a.pos_table && (unsigned)pos >= (unsigned)a.n_pos);
    const TT* row = (const TT*)a.table + (size_t)(none || bad ? 0 : token) * a.ld_table;
    const TT* prow = (const TT*)a.pos_table + (size_t)(bad ? 0 : pos) * a.ld_pos;
    AT* y = (AT*)a.y + (size_t)t * a.ld_y;
    if (bad) {
      wide_t<AT, V> out;
#pragma unroll
      for (int j = 0; j < V; j++) out[j] = (AT)__builtin_nanf("");
      for (int c = lane * V; c < a.width; c += lanes * V) store_wide<V>(y + c, out);
      continue;
    }
    for (int c = lane * V; c < a.width; c += kFlight * lanes * V) {
      wide_t<TT, V> e[kFlight] = {}, q[kFlight] = {};
#pragma unroll
      for (int i = 0; i < kFlight; i++) {
        const int at = c + i * lanes * V;
        if (at < a.width && !none) e[i] = load_wide<V>(row + at);
        if (at < a.width && a.pos_table) q[i] = load_wide<V>(prow + at);
      }
#pragma unroll
      for (int i = 0; i < kFlight; i++) {
        const int at = c + i * lanes * V;
        wide_t<AT, V> out;
#pragma unroll
        for (int j = 0; j < V; j++) {
          const float v = none ? 0.f : (float)e[i][j] * a.scale;
          out[j] = (AT)(a.pos_table ? v + (float)q[i][j] : v);
        }
        if (at < a.width) store_wide<V>(y + at, out);
      }
    }
  }
}

// ---- the tokens' numbers sorted by token, those of no row behind the others (their key: vocab)
// (BITS as a constant: a branch for each load would wait for each)
template <int BITS>
__device__ __forceinline__ uint32_t key_of(const void* tokens, size_t t, int vocab) {
  if constexpr (BITS == 64) {
    const uint64_t k = ((const uint64_t*)tokens)[t];
    return k < (uint64_t)vocab ? (uint32_t)k : (uint32_t)vocab;
  } else {
    return min(((const uint32_t*)tokens)[t], (uint32_t)vocab);
  }
}

struct SortArgs {
  const void* tokens;           // the first digit's keys come from here, with the numbers 0 .. T - 1 ...
  const uint32_t *key_in, *at_in;   // ... the others' from here
  uint32_t *key_out, *at_out;
  uint32_t* count;              // [256][blocks]
  int T, vocab, shift, blocks;
};

// BITS of a token where the digit is the first one, else 0
template <int BITS>
__global__ __launch_bounds__(NT) void digit_count_kernel(SortArgs a) {
  __shared__ uint32_t n[256];
  n[threadIdx.x] = 0;
  __syncthreads();
  const int first = blockIdx.x * kSortBlock;
  for (int i = threadIdx.x; i < kSortBlock && first + i < a.T; i += NT) {
    uint32_t k;
    if constexpr (BITS) k = key_of<BITS>(a.tokens, first + i, a.vocab);
    else k = a.key_in[first + i];
    atomicAdd(&n[(k >> a.shift) & 255], 1u);
  }
  __syncthreads();
  a.count[threadIdx.x * a.blocks + blockIdx.x] = n[threadIdx.x];
}

// count[i] = the sum of those before it: one block
__global__ __launch_bounds__(1024) void digit_scan_kernel(uint32_t* count, int n) {
  __shared__ uint32_t wave_sum[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t before = 0;
  for (int first = 0; first < n; first += 1024) {
    const int i = first + threadIdx.x;
    const uint32_t v = i < n ? count[i] : 0;
    uint32_t s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t u = __shfl_up(s, o, 64);
      if (lane >= o) s += u;
    }
    if (lane == 63) wave_sum[wave] = s;
    __syncthreads();
    uint32_t base = before, total = before;
    for (int w = 0; w < 16; w++) {
      if (w < wave) base += wave_sum[w];
      total += wave_sum[w];
    }
    if (i < n) count[i] = base + s - v;
    before = total;
    __syncthreads();
  }
}

// A wave takes 64 numbers after the other; among those, a lane's place is behind the lanes before it with the same digit.
template <int BITS>
__global__ __launch_bounds__(NT) void digit_place_kernel(SortArgs a) {
  __shared__ uint32_t place[NW][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int first = blockIdx.x * kSortBlock + wave * (kSortBlock / NW);
  for (int i = threadIdx.x; i < NW * 256; i += NT) place[0][i] = 0;
  __syncthreads();
  uint32_t key[kItems], at[kItems];
#pragma unroll
  for (int i = 0; i < kItems; i++) {
    const int t = first + i * 64 + lane;
    if (t < a.T) {
      if constexpr (BITS) { key[i] = key_of<BITS>(a.tokens, t, a.vocab); at[i] = t; }
      else { key[i] = a.key_in[t]; at[i] = a.at_in[t]; }
    }
  }
#pragma unroll
  for (int i = 0; i < kItems; i++)
    if (first + i * 64 + lane < a.T) atomicAdd(&place[wave][(key[i] >> a.shift) & 255], 1u);
  __syncthreads();
  uint32_t base = a.count[threadIdx.x * a.blocks + blockIdx.x];
#pragma unroll
  for (int w = 0; w < NW; w++) {
    const uint32_t n = place[w][threadIdx.x];
    place[w][threadIdx.x] = base;
    base += n;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kItems; i++) {
    const bool on = first + i * 64 + lane < a.T;
    const uint32_t d = on ? (key[i] >> a.shift) & 255 : 256;
    uint64_t same = ~0ull;          // lanes with this lane's digit
#pragma unroll
    for (int b = 0; b < 9; b++) {
      const uint64_t m = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? m : ~m;
    }
    const int behind = __popcll(same & ((1ull << lane) - 1));
    if (on) {                       // (the wave's own counters: its accesses follow each other as they are written)
      volatile uint32_t* mine = &place[wave][d];
      const uint32_t to = *mine + behind;
      if (behind == 0) *mine = to + __popcll(same);
      a.key_out[to] = key[i];
      a.at_out[to] = at[i];
    }
  }
}

// ---- zeros (beta 0).  A table of many more rows than there are tokens is set to zeros as a whole, before the rows of tokens that occur are written a second time: as a sweep, so that what is
// written at once lies together.  256 blocks in front of those that count places do that meanwhile, one of 256 lanes with one piece of 16 bytes each and time; a large table gets a launch of
// its own, a piece a lane (2.15 GB: 316 us, 6.8 TB/s, and with the 256 blocks 340; 0.8 GB: 120 and 127; 0.13 GB: 20 and 19; the launch takes 4).  Of a table with up to kAbsent times as many
// rows as tokens those whose token does not occur are set to zeros beside the sums (zero_absent).  Whole calls, sweep and rows, 8192 tokens all alike frequent, rows of 4096: as many rows as tokens
// 67, 64 us; four times 144, 133; eight times 223, 224; 2048 tokens, sixteen times 110, 111 (tokens as frequent as words: 66, 65; 139, 136; 220, 229; 106, 111).
constexpr int kFillBlocks = 256, kFillLanes = 256, kAbsent = 8;
constexpr int64_t kSweepPieces = 1 << 25;   // from 512 MB on
struct FillArgs {
  float* d;
  size_t ld;
  int64_t rows, width;         // rows that lie behind each other are one of all elements
  int lanes_log2, blocks;      // 2^lanes_log2 lanes to a row, 256 at most; blocks of the launch that do nothing else
};
// Elements of a row by lane `at` of `across`
__device__ __forceinline__ void zero_row(float* p, int64_t width, int64_t at, int64_t across) {
  const int64_t head = min((int64_t)(-(uintptr_t)p & 15) / 4, width), pieces = (width - head) / 4;      // elements up to the first whole piece
  for (int64_t i = at; i < pieces; i += across) *(f32x4*)(p + head + 4 * i) = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int64_t i = at; i < head; i += across) p[i] = 0.f;
  for (int64_t i = head + 4 * pieces + at; i < width; i += across) p[i] = 0.f;
}
__device__ __forceinline__ void fill_zeros(const FillArgs& f, int block) {
  const int64_t lane = (int64_t)block * kFillLanes + threadIdx.x, lanes = (int64_t)f.blocks * kFillLanes;
  if (threadIdx.x >= kFillLanes) return;
  if (f.rows == 1) return zero_row(f.d, f.width, lane, lanes);
  const int across = 1 << f.lanes_log2;
  for (int64_t r = lane >> f.lanes_log2; r < f.rows; r += lanes >> f.lanes_log2) zero_row(f.d + (size_t)r * f.ld, f.width, lane & (across - 1), across);
}
__global__ __launch_bounds__(kFillLanes) void fill_kernel(FillArgs f) { fill_zeros(f, blockIdx.x); }

// Few tokens: a number's place in the sorted list is how many lie before it, which a block counts for kRanked of them against all others (one comparison for 64 of
// those, counted by lane: a scalar count behind each comparison fills the CU's one scalar unit).
constexpr uint32_t kNone = 0x7ffffffe;       // (twice that and 2 more fit)
constexpr int kRanked = 16, kRankThreads = 1024, kRankWaves = kRankThreads / 64;
template <int BITS>
__global__ __launch_bounds__(kRankThreads) void rank_kernel(SortArgs a, FillArgs f) {
  __shared__ uint32_t keys[kSmall], count[kRankWaves][kRanked];
  if ((int)blockIdx.x < f.blocks) return fill_zeros(f, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = (blockIdx.x - f.blocks) * kRanked;
  constexpr int FLIGHT = 8;                  // keys of a lane in flight
  for (int t0 = threadIdx.x; t0 - (int)threadIdx.x < a.T; t0 += FLIGHT * kRankThreads) {
    uint32_t k[FLIGHT];
#pragma unroll
    for (int j = 0; j < FLIGHT; j++) k[j] = key_of<BITS>(a.tokens, min(t0 + j * kRankThreads, a.T - 1), a.vocab);
#pragma unroll
    for (int j = 0; j < FLIGHT; j++) keys[t0 + j * kRankThreads] = t0 + j * kRankThreads < a.T ? k[j] : kNone;
  }
  __syncthreads();
  uint32_t key[kRanked], n[kRanked];
#pragma unroll
  for (int i = 0; i < kRanked; i++) {
    key[i] = 2 * __builtin_amdgcn_readfirstlane(keys[first + i]) + 1;
    n[i] = 0;
  }
#pragma unroll 1
  for (int g = wave * 64; g < a.T; g += kRankThreads) {
    const uint32_t k = keys[g + lane];
    if (first >= g && first < g + 64) {      // these 64 hold the block's own (which begin at a multiple of kRanked)
#pragma unroll
      for (int i = 0; i < kRanked; i++) n[i] += 2 * k + (lane < first - g + i ? 0u : 2u) < key[i];
    } else {
      const uint32_t k2 = 2 * k + (g < first ? 0u : 2u);       // of those before the block's own the equal ones count, too
#pragma unroll
      for (int i = 0; i < kRanked; i++) n[i] += k2 < key[i];
    }
  }
  // over the wave, two counts in a register (a lane's are at most kSmall / kRankThreads, a wave's 64 times that)
#pragma unroll
  for (int i = 0; i < kRanked; i += 2) {
    int both = (int)(n[i] | n[i + 1] << 16);
    both += __builtin_amdgcn_update_dpp(0, both, 0xB1, 0xF, 0xF, true);    // lanes 1 0 3 2
    both += __builtin_amdgcn_update_dpp(0, both, 0x4E, 0xF, 0xF, true);    // lanes 2 3 0 1
    both += __builtin_amdgcn_update_dpp(0, both, 0x141, 0xF, 0xF, true);   // lanes 7 .. 0 of 8
    both += __builtin_amdgcn_update_dpp(0, both, 0x140, 0xF, 0xF, true);   // lanes 15 .. 0 of 16
    const uint32_t sum = __builtin_amdgcn_readlane(both, 0) + __builtin_amdgcn_readlane(both, 16) + __builtin_amdgcn_readlane(both, 32) + __builtin_amdgcn_readlane(both, 48);
    if (lane == 0) { count[wave][i] = sum & 0xffff; count[wave][i + 1] = sum >> 16; }
  }
  __syncthreads();
  if (threadIdx.x < kRanked && first + (int)threadIdx.x < a.T) {
    uint32_t to = 0;
#pragma unroll
    for (int w = 0; w < kRankWaves; w++) to += count[w][threadIdx.x];
    a.key_out[to] = keys[first + threadIdx.x];
    a.at_out[to] = first + threadIdx.x;
  }
}

struct BwdArgs {
  const uint32_t *key, *at;     // sorted
  const void* dy;
  float *d, *part;              // part[chunk][2][width]: of the sum that began before the chunk, of that which goes on behind it
  size_t ld_d, ld_dy;
  int T, vocab, width, chunk, beta;
  float scale;
};

template <int V>
__device__ __forceinline__ void put(const BwdArgs& a, uint32_t row, int c, const wide_t<float, V>& s, const wide_t<float, V>& old) {
  store_wide<V>(a.d + (size_t)row * a.ld_d + c, s * a.scale + old);
}
template <int V>
__device__ __forceinline__ wide_t<float, V> old_row(const BwdArgs& a, uint32_t row, int c) {
  wide_t<float, V> r = {};
  if (a.beta) r = load_wide<V>((const float*)a.d + (size_t)row * a.ld_d + c);
  return r;
}

// Zeros for those of `rows` rows, at most 64, from `first` on whose token does not occur: a lane looks one up in the sorted list, and the wave writes them one after the other.  At most
// 16 KB of them, so that waves are short and what they write lies together in their order, and 4096 waves at least (7917 tokens, 56740 rows of 128: 27 us, 47 with a row a wave, 29 with 32; 4000, 30000 of
// 64: 18, with 64 a wave 25; 8190, 50257 of 4096: 186, with 12 a wave 196).
constexpr int kAbsentRun = 4096, kAbsentWaves = 4096;
__device__ __forceinline__ void zero_absent(const BwdArgs& a, int64_t first, int rows) {
  const int lane = threadIdx.x & 63;
  const int64_t row = first + lane;
  const bool on = lane < rows && row < a.vocab;
  int lo = 0, hi = on ? a.T : 0;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (a.key[mid] < (uint32_t)row) lo = mid + 1;
    else hi = mid;
  }
  uint64_t left = __ballot(on && (lo == a.T || a.key[lo] != (uint32_t)row));
  for (; left; left &= left - 1) zero_row(a.d + (size_t)(first + __builtin_ctzll(left)) * a.ld_d, a.width, lane, 64);
}

// A block adds up V columns a lane of one chunk.  A wave's lanes hold the keys and numbers of 64 entries, which are the same for all lanes of a row; rows of dy, and those
// of the table that get a sum (beta), are asked for kAhead at a time.  Blocks behind the `chunks` first are zero_absent's.
template <class AT, int V>
__global__ __launch_bounds__(kRowThreads) __attribute__((amdgpu_waves_per_eu(8))) void embedding_bwd_kernel(BwdArgs a, int chunks, int rows) {
  if ((int)blockIdx.x >= chunks) {
    const int waves = blockDim.x / 64, block = (blockIdx.x - chunks) * gridDim.y + blockIdx.y;
    return zero_absent(a, ((int64_t)block * waves + __builtin_amdgcn_readfirstlane(threadIdx.x / 64)) * rows, rows);
  }
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * V, lane = threadIdx.x & 63;
  const int first = blockIdx.x * a.chunk, end = min(first + a.chunk, a.T);
  const bool on = c < a.width;
  const AT* dy = (const AT*)a.dy + (on ? c : 0);
  float* part = a.part + (size_t)blockIdx.x * 2 * a.width + c;
  wide_t<float, V> s = {};
  bool began = first == 0 || a.key[first - 1] != a.key[first];      // whether the present sum began in this chunk
  for (int i0 = first; i0 < end; i0 += 64) {
    const int e = min(i0 + lane, a.T - 1);
    const uint32_t keys = a.key[e], ats = a.at[e];
    const uint64_t last = __ballot(e + 1 >= a.T || a.key[min(e + 1, a.T - 1)] != keys);     // entries that end a sum
    const int n = min(min(end - i0, 64), (int)__popcll(__ballot(i0 + lane < a.T && keys < (uint32_t)a.vocab)));   // (tokens of no row lie behind all others)
    for (int i = 0; i < n; i += kAhead) {
      wide_t<AT, V> r[kAhead];
      wide_t<float, V> old[kAhead];
      uint32_t key[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; k++) {
        key[k] = __builtin_amdgcn_readlane(keys, min(i + k, 63));
        const uint32_t at = __builtin_amdgcn_readlane(ats, min(i + k, 63));
        if (i + k < n && on) {
          r[k] = load_wide<V>(dy + (size_t)at * a.ld_dy);
          if ((last >> (i + k)) & 1) old[k] = old_row<V>(a, key[k], c);
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; k++) {
        if (i + k >= n || !on) break;
#pragma unroll
        for (int j = 0; j < V; j++) s[j] += (float)r[k][j];
        const bool done = (last >> (i + k)) & 1;
        if (done || i0 + i + k + 1 == end) {
          if (done && began) put<V>(a, key[k], c, s, old[k]);
          else store_wide<V>(part + (began ? a.width : 0), s);
          s = wide_t<float, V>{};
          began = true;
        }
      }
    }
    if (n < min(end - i0, 64)) return;
  }
}

// The chunk in which a sum begins that goes on behind it adds up what the following ones left of it: kJoinAcross lanes across a row, twice.  (8190 tokens as frequent as words are, and
// 8192 times the same one, the whole call: 63 and 63 us; 256 lanes across, once, 64 and 108; 64, four times, 67 and 47.)
constexpr int kJoinAcross = NT / 2;
template <int V>
__global__ __launch_bounds__(NT) void embedding_join_kernel(BwdArgs a, int chunks) {
  const int first = blockIdx.x * a.chunk, end = first + a.chunk;
  if (end >= a.T) return;
  const uint32_t k = a.key[end - 1];
  if (k >= (uint32_t)a.vocab || a.key[end] != k) return;
  if (a.key[first] == k && first > 0 && a.key[first - 1] == k) return;      // it began earlier
  __shared__ wide_t<float, V> share[kJoinAcross];
  const int across = threadIdx.x % kJoinAcross, half = threadIdx.x / kJoinAcross, at = (blockIdx.y * kJoinAcross + across) * V, c = at < a.width ? at : 0;   // (lanes behind the last column go along: ballots are whole waves')
  const float* p = a.part + (size_t)blockIdx.x * 2 * a.width + c;
  const wide_t<float, V> old = old_row<V>(a, k, c);
  // the chunks behind this one that begin with the same token: all of their entries, or the first of its
  int behind = 0;
  for (int b = blockIdx.x + 1 + (threadIdx.x & 63);; b += 64) {
    const uint64_t same = __ballot(b < chunks && a.key[(size_t)min(b, chunks - 1) * a.chunk] == k);
    behind += ~same ? __builtin_ctzll(~same) : 64;
    if (~same) break;
  }
  // this one's share is number 0; the block's two halves add up one of them each
  auto share_of = [&](int i) { return load_wide<V>(p + (i == 0 ? a.width : (size_t)i * 2 * a.width)); };
  const int from = (behind + 2) / 2 * half, to = half ? behind + 1 : (behind + 2) / 2;
  wide_t<float, V> s = {};
  for (int b = from; b < to; b += kJoin) {
    wide_t<float, V> r[kJoin];
#pragma unroll
    for (int i = 0; i < kJoin; i++) r[i] = share_of(min(b + i, to - 1));
#pragma unroll
    for (int i = 0; i < kJoin; i++)
      if (b + i < to) s += r[i];
  }
  if (half) share[across] = s;
  __syncthreads();
  if (half || at >= a.width) return;
  s += share[across];
  put<V>(a, k, c, s, old);
}

int sort_blocks(int T) { return (T + kSortBlock - 1) / kSortBlock; }
// (few tokens: shorter chunks, or their blocks would leave CUs idle)
int chunk_of(int T) { return std::max(T <= 4096 ? kMinChunk / 2 : kMinChunk, (T + kMaxChunks - 1) / kMaxChunks); }
uint64_t up256(uint64_t n) { return (n + 255) / 256 * 256; }

// Places in the workspace
struct Places { uint64_t key[2], at[2], count, part, bytes; };
Places places(const ah_embedding_t* c) {
  Places p;
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t r = at; at += up256(bytes); return r; };
  const uint64_t T = std::max(c->rows, 1);
  for (int i = 0; i < 2; i++) { p.key[i] = take(4 * T); p.at[i] = take(4 * T); }
  p.count = take(4ull * 256 * sort_blocks((int)T));
  const uint64_t chunk = chunk_of((int)T), chunks = (T + chunk - 1) / chunk;
  p.part = take(4ull * chunks * 2 * c->width);
  p.bytes = at;
  return p;
}

int log2_lanes(int width, int v) {   // lanes to a row: as many as have elements to take, at most a block
  int l = 0;
  while (l < 8 && (1 << l) * v < width) l++;
  return l;
}

int check_sizes(const char* who, const ah_embedding_t* c) {
  if (!c) return set_error(AH_EINVAL, "%s: config is NULL", who);
  if (c->struct_size != sizeof(ah_embedding_t)) return set_error(AH_EINVAL, "%s: struct_size %u != %zu", who, c->struct_size, sizeof(ah_embedding_t));
  if (c->rows < 0 || c->vocab < 1 || c->width < 1) return set_error(AH_EINVAL, "%s: need rows >= 0, vocab >= 1 and width >= 1", who);
  if (c->rows > kMaxRows || c->vocab > kMaxVocab || c->width > kMaxWidth)
    return set_error(AH_EUNSUPPORTED, "%s: more than 2^25 rows, a vocabulary of 2^30 or a width of 65536", who);
  return AH_OK;
}

int check(const char* who, const ah_embedding_t* c) {
  if (int rc = check_sizes(who, c)) return rc;
  if ((c->table_type != AH_BF16 && c->table_type != AH_FP32) || (c->act_type != AH_BF16 && c->act_type != AH_FP32))
    return set_error(AH_EINVAL, "%s: types must be AH_BF16 or AH_FP32", who);
  if (c->token_bits != 32 && c->token_bits != 64) return set_error(AH_EINVAL, "%s: token_bits %d: 32 or 64", who, c->token_bits);
  if (!std::isfinite(c->scale)) return set_error(AH_EINVAL, "%s: scale is not finite", who);
  for (int64_t ld : {c->ld_table, c->ld_act, c->ld_pos})
    if (ld != 0 && (ld < c->width || ld > (1ll << 31))) return set_error(AH_EINVAL, "%s: a row stride must be at least the width, %d, and at most 2^31", who, c->width);
  return AH_OK;
}

}  // namespace

extern "C" int ah_embedding_fwd(const ah_embedding_t* c, const void* table, const void* tokens, void* y, void* stream) {
  discard_stale_hip_error();
  if (int rc = check("ah_embedding_fwd", c)) return rc;
  const int tb = c->table_type == AH_FP32 ? 4 : 2, ab = c->act_type == AH_FP32 ? 4 : 2;
  if (c->pos_table) {
    if (c->n_pos < 1) return set_error(AH_EINVAL, "ah_embedding_fwd: n_pos must be >= 1");
    if (!c->positions && (c->seq_len < 1 || std::min(c->seq_len, std::max(c->rows, 1)) > c->n_pos))
      return set_error(AH_EINVAL, "ah_embedding_fwd: seq_len %d needs as many rows of pos_table (n_pos %d)", c->seq_len, c->n_pos);
    if (!aligned_to(c->pos_table, tb) || !aligned_to(c->positions, 4)) return set_error(AH_EINVAL, "ah_embedding_fwd: pos_table or positions is misaligned");
  }
  if (c->rows == 0) return AH_OK;
  if (!table || !tokens || !y || !aligned_to(table, tb) || !aligned_to(tokens, c->token_bits / 8) || !aligned_to(y, ab))
    return set_error(AH_EINVAL, "ah_embedding_fwd: table, tokens or y is NULL or misaligned");
  FwdArgs a = {};
  a.table = table; a.tokens = tokens; a.pos_table = c->pos_table; a.positions = c->positions; a.y = y;
  a.ld_table = c->ld_table ? c->ld_table : c->width; a.ld_y = c->ld_act ? c->ld_act : c->width; a.ld_pos = c->ld_pos ? c->ld_pos : c->width;
  a.T = c->rows; a.vocab = c->vocab; a.width = c->width; a.n_pos = c->n_pos; a.S = c->seq_len; a.bits = c->token_bits; a.scale = c->scale;
  const bool wide = c->width % 8 == 0 && rows16(table, a.ld_table, tb) && rows16(y, a.ld_y, ab) && (!a.pos_table || rows16(a.pos_table, a.ld_pos, tb));
  const int l = log2_lanes(c->width, wide ? 8 : 1), per = NT >> l;
  const int blocks = std::min((c->rows + per - 1) / per, 1 << 22);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(NT), 0, (hipStream_t)stream, a, l); };
  auto by_act = [&](auto t) {
    typedef decltype(t) TT;
    if (ab == 4) { if (wide) go(embedding_fwd_kernel<TT, float, 8>); else go(embedding_fwd_kernel<TT, float, 1>); }
    else { if (wide) go(embedding_fwd_kernel<TT, bf16, 8>); else go(embedding_fwd_kernel<TT, bf16, 1>); }
  };
  if (tb == 4) by_act(float());
  else by_act(bf16());
  return hip_status(hipGetLastError(), "ah_embedding_fwd");
}

extern "C" int ah_embedding_bwd_workspace(const ah_embedding_t* c, uint64_t* bytes) {
  if (!bytes) return set_error(AH_EINVAL, "ah_embedding_bwd_workspace: bytes is NULL");
  if (int rc = check_sizes("ah_embedding_bwd_workspace", c)) return rc;
  *bytes = places(c).bytes;
  return AH_OK;
}

extern "C" int ah_embedding_bwd(const ah_embedding_t* c, const void* tokens, const void* dy, float* d_table, int beta, void* workspace, void* stream) {
  discard_stale_hip_error();
  if (int rc = check("ah_embedding_bwd", c)) return rc;
  if (beta != 0 && beta != 1) return set_error(AH_EINVAL, "ah_embedding_bwd: beta must be 0 or 1");
  const int ab = c->act_type == AH_FP32 ? 4 : 2;
  if (!d_table || !workspace || !aligned_to(d_table, 4) || !aligned_to(workspace, 256)) return set_error(AH_EINVAL, "ah_embedding_bwd: d_table or the workspace is NULL or misaligned");
  if (c->rows && (!tokens || !dy || !aligned_to(tokens, c->token_bits / 8) || !aligned_to(dy, ab))) return set_error(AH_EINVAL, "ah_embedding_bwd: tokens or dy is NULL or misaligned");
  const hipStream_t s = (hipStream_t)stream;
  const int T = c->rows;
  BwdArgs a = {};
  a.dy = dy; a.d = d_table; a.ld_d = c->ld_table ? c->ld_table : c->width; a.ld_dy = c->ld_act ? c->ld_act : c->width;
  a.T = T; a.vocab = c->vocab; a.width = c->width; a.chunk = chunk_of(T); a.beta = beta; a.scale = c->scale;
  const bool small = T > 0 && T <= kSmall, absent = !beta && small && c->vocab <= (int64_t)kAbsent * T;
  FillArgs f = {};
  if (!beta && !absent) {
    const bool flat = a.ld_d == (size_t)c->width || c->vocab == 1;
    f.d = d_table; f.ld = a.ld_d; f.rows = flat ? 1 : c->vocab; f.width = flat ? (int64_t)c->vocab * c->width : c->width;
    f.lanes_log2 = log2_lanes(c->width, 4);
    const int64_t pieces = (int64_t)c->vocab * c->width / 4 + 1, lone = (pieces + kFillLanes - 1) / kFillLanes;
    const bool apart = !small || pieces >= kSweepPieces;
    f.blocks = (int)std::min<int64_t>(lone, pieces >= kSweepPieces ? 1 << 22 : kFillBlocks);
    if (apart) {
      hipLaunchKernelGGL(fill_kernel, dim3(f.blocks), dim3(kFillLanes), 0, s, f);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return hip_status(e, "ah_embedding_bwd");
      f.blocks = 0;
    }
  }
  if (T == 0) return AH_OK;
  const Places p = places(c);
  char* w = (char*)workspace;
  a.part = (float*)(w + p.part);
  SortArgs q = {};
  q.T = T; q.vocab = c->vocab; q.blocks = sort_blocks(T); q.count = (uint32_t*)(w + p.count);
  q.tokens = tokens;
  int key_bits = 1;                                       // of the largest key, vocab
  while (key_bits < 31 && (c->vocab >> key_bits) != 0) key_bits++;
  if (small) {
    q.key_out = (uint32_t*)(w + p.key[0]); q.at_out = (uint32_t*)(w + p.at[0]);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(f.blocks + (T + kRanked - 1) / kRanked), dim3(kRankThreads), 0, s, q, f); };
    if (c->token_bits == 64) go(rank_kernel<64>);
    else go(rank_kernel<32>);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return hip_status(e, "ah_embedding_bwd");
    q.key_in = q.key_out; q.at_in = q.at_out;
  } else {
    int to = 0;
    for (q.shift = 0; q.shift < key_bits; q.shift += 8, to ^= 1) {
      q.key_out = (uint32_t*)(w + p.key[to]); q.at_out = (uint32_t*)(w + p.at[to]);
      auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(q.blocks), dim3(NT), 0, s, q); };
      const int bits = q.shift ? 0 : c->token_bits;
      if (bits == 64) go(digit_count_kernel<64>); else if (bits == 32) go(digit_count_kernel<32>); else go(digit_count_kernel<0>);
      hipLaunchKernelGGL(digit_scan_kernel, dim3(1), dim3(1024), 0, s, q.count, 256 * q.blocks);
      if (bits == 64) go(digit_place_kernel<64>); else if (bits == 32) go(digit_place_kernel<32>); else go(digit_place_kernel<0>);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return hip_status(e, "ah_embedding_bwd");
      q.key_in = q.key_out; q.at_in = q.at_out;
    }
  }
  a.key = q.key_in; a.at = q.at_in;
  // four columns a lane: 16 bytes of the table's gradient, 8 or 16 of dy
  const bool wide = c->width % 4 == 0 && aligned_to(dy, 4 * ab) && a.ld_dy % 4 == 0 && rows16(d_table, a.ld_d, 4);
  const int v = wide ? 4 : 1, chunks = (T + a.chunk - 1) / a.chunk;
  // lanes for a whole row, or 1024 of them
  const int slices = (c->width + kRowThreads * v - 1) / (kRowThreads * v), lanes = std::max(64, ((c->width + slices * v - 1) / (slices * v) + 63) / 64 * 64);
  const int across = (c->width + lanes * v - 1) / (lanes * v);
  const int rows = std::max(1, std::min({64, kAbsentRun / c->width, c->vocab / kAbsentWaves})), per = rows * (lanes / 64) * across, fills = absent ? (c->vocab + per - 1) / per : 0;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(chunks + fills, across), dim3(lanes), 0, s, a, chunks, rows); };
  if (ab == 4) { if (wide) go(embedding_bwd_kernel<float, 4>); else go(embedding_bwd_kernel<float, 1>); }
  else { if (wide) go(embedding_bwd_kernel<bf16, 4>); else go(embedding_bwd_kernel<bf16, 1>); }
  const dim3 join(chunks, (c->width + kJoinAcross * v - 1) / (kJoinAcross * v));
  if (wide) hipLaunchKernelGGL(embedding_join_kernel<4>, join, dim3(NT), 0, s, a, chunks);
  else hipLaunchKernelGGL(embedding_join_kernel<1>, join, dim3(NT), 0, s, a, chunks);
  return hip_status(hipGetLastError(), "ah_embedding_bwd");
}
