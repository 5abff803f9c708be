// Verify-attention over the cache of latents: the draft queries of each request, of all heads, attend over its committed context and their draft ancestors.
// A cache row is a latent of C elements, key and value at once, and R more that only keys have; all heads read the same rows.
//
//   S^T = K Q^T     matrix instructions leave a lane with consecutive tokens of one query row, 4 (16x16x32) or 8 (32x32x16: 4 and 4) at a time
//   O^T = V^T P^T   so its weights, in bf16, are operands as they are; V^T, the same bytes as K, is read from LDS by columns
// fp32 results take the weights in three terms of bf16, which hold all of fp32; bf16 results take one, whose rounding weighs as much as the result's own: together
// 0.0020 to 0.0023 of a result (root mean square; the result's alone 0.0017), where two terms would double the products of the second kind.
// Query rows of a request (node x head, consecutive in memory) are taken in groups of 16, 32, 64 or 128, the tokens in tiles, which four waves bring to LDS and
// share: LatentNarrow and LatentWide below.  Of the second product every wave takes C / 4 columns for all rows; the weights go through LDS.
//
// Bound: up to 32 rows by memory (64 requests of 2048 tokens at the median, 16 heads, from cold caches: 48 us, 4.6 TB/s with the start, and 6 for the merge), with 128
// by the matrix instructions (64 requests of 8192 tokens, 4 x 128 rows: 1160 to 1190 TFLOP/s of the 1520 that a large matrix product reaches).
//
// Work: the tiles of all requests and groups lie end to end and are cut into ranges of equal cost, one per workgroup, whatever the lengths; every
// workgroup works out from ctx_len and q_offsets which pieces its range holds.  Groups that are cut leave partial results, which a second launch
// merges in their order.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "latent.h"

namespace specv {

constexpr int kLaThreads = 256, kLaWaves = 4;
constexpr int kLaPage = 16;
constexpr int kLaMaxNodes = 128;
constexpr int kLaRanges = 256;                 // workgroups: one per compute unit
constexpr float kLaNoScore = -3.0e38f;         // the reference before the first position: finite, so that -infinity stays ahead of nothing
// A row's reference follows its maximum when that is 2^16 ahead: weights are at most 2^16, and sums of L of them times latents of up to c stay finite while
// L c < 2^112.  (Sooner costs time: 2^8 ahead, from cold caches, 5 requests of 61 nodes, 40 heads 145 us, 138 with 2^16
// and with 2^40; 64 requests of 2 to 10 tokens, 128 heads 356, 348 and 350.)
constexpr float kLaSlack = 16.f;

struct LatentAttnParams {
  const uint16_t* q;
  const uint16_t* pool;
  const int32_t* block_table;
  const int32_t* ctx_len;
  const int32_t* q_offsets;
  const int32_t* parent;
  void* out;
  float* lse;
  float* ws_o;         // [ranges][2][M][C] partial results, each by its own sum of weights
  float2* ws_ml;       // ... [M] (reference in log2 units, sum)
  int4* cut;           // [workgroups] the group whose first piece this workgroup has: (first row (2 words), rows << 16 | pieces, range)
  int B, H, total_q, max_q, max_pages, num_pages;
  int ranges;
  float c;             // scale * log2(e)
  int out_f32;
};

// Which of the 16 tokens of a page a node sees, the page starting `past` tokens behind the context (negative: before its end).
__device__ __forceinline__ uint32_t page_mask(unsigned long long lo, unsigned long long hi, int past) {
  if (past <= -16) return 0xffffu;
  if (past < 0) return (static_cast<uint32_t>(lo << -past) | ((1u << -past) - 1u)) & 0xffffu;
  if (past >= 128) return 0u;
  if (past >= 64) return static_cast<uint32_t>(hi >> (past - 64)) & 0xffffu;
  return static_cast<uint32_t>(past == 0 ? lo : (lo >> past) | (hi << (64 - past))) & 0xffffu;
}
__device__ __forceinline__ bool any_lane(bool x) { return __builtin_amdgcn_ballot_w64(x) != 0ull; }
// max and sum over the four lane groups: the same bits in lanes n, 16 + n, 32 + n and 48 + n.
__device__ __forceinline__ float groups_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float groups_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
// At most N loads of this wave on their way.
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

// ---- the cut of the batch: costs are whole numbers in fp64 (exact up to 2^53) --------------------------------------
template <int T>
__device__ __forceinline__ int tiles_of(const LatentAttnParams& P, int ctx, int n) {
  constexpr int kPages = T / kLaPage;
  return n > 0 ? min(static_cast<int>((static_cast<unsigned>(ctx) + n + T - 1) / T), static_cast<int>((static_cast<unsigned>(P.max_pages) + kPages - 1) / kPages)) : 0;
}
// A number that is the same in all lanes, in scalar registers.
__device__ __forceinline__ double uniform(double x) { return lane_f64(x, 0); }
// The groups of all requests end to end, each its kHead (what its start and end cost, in tiles) and its tiles, in `used` ranges of equal length, whole numbers apart,
// at least kLeast long, or twice that where there are more than 64 (one request, 16 heads; 500 tiles: 20.5 us, with kLeast alone 24.5, as there are more to be
// merged; 9 tiles x 4 groups: 14.8, with twice that 16.6).  A border that would leave a piece of a group with fewer than kSnap tiles goes to the group's end.
struct LaCut {
  int used;
  double each, total;
};
__device__ __forceinline__ LaCut cut_ranges(int most, int least, double total) {
  LaCut c;
  c.total = total;
  c.used = __builtin_amdgcn_readfirstlane(static_cast<int>(fmin(fmax(fmax(fmin(total / least, 64.0), total / (2 * least)), 1.0), static_cast<double>(most))));
  c.each = uniform(total / c.used);
  return c;
}
__device__ __forceinline__ double range_start(const LaCut& c, int s) { return s >= c.used ? c.total : floor(s * c.each); }
__device__ __forceinline__ int range_of(const LaCut& c, double at) {
  int s = min(max(static_cast<int>(at / c.each) - 1, 0), c.used - 1);
  while (s + 1 < c.used && range_start(c, s + 1) <= at) ++s;
  return s;
}
// Where a border at `at` goes by the group [start, end) that it lies in (another: where it is).
template <typename K>
__device__ __forceinline__ double border(double at, double start, double end) {
  if (at <= start || at >= end) return at;
  if (at < start + K::kHead + K::kSnap) return start;
  return at > end - K::kSnap ? end : at;
}

// Up to 16 NB rows, NB 1, 2 or 4.  Of the scores a wave takes 16 rows, by half of a tile's tokens (NB 1: two waves have none) or, NB 4, by all.
// 4096 tokens x 64 requests, 302 MB: 16 rows 60 us, 32 rows 65, 64 rows 84 (with another barrier a tile, and no keys read ahead of it, 89); with tiles of 64 tokens,
// two in LDS, 61, 71 and (as 128 rows) 98.
template <int C_, int R_, int NB_, int TERMS_>
struct LatentNarrow {
  static constexpr bool kWide = false;
  static constexpr int C = C_, R = R_, NB = NB_, TERMS = TERMS_;
  static constexpr int W = C + R;
  static constexpr int kHead = 6, kSnap = 1, kLeast = 2;       // see LaCut
  static constexpr int M = 16 * NB, T = 32, KB = NB == 4 ? 2 : 1, WK = 2 / KB;      // blocks of 16 tokens of a wave; waves that share a row
  static constexpr int kUnits = (W / 8 + 7) / 8 * 8;            // 16-byte units of a row in LDS
  static constexpr int kRow = 16 * kUnits, kTile = T * kRow;
  static constexpr int kPages = T / kLaPage;
  static constexpr int RB = NB, CB = C / 4 / 16;                // 16-row blocks; 16-column blocks of a wave
  static constexpr int kSteps = W / 32;
  static constexpr int kLoads = kTile / kLaWaves / 1024;        // of a wave for a tile
  static constexpr int kOffsets = 8 * kRow / 1024;              // loads that bring 8 rows
  static constexpr int kWeights = TERMS * RB * 1024, kBuffers = 2;
  static constexpr int kSmall = kBuffers * kWeights + kLaMaxNodes * 16 + 4 * M * (3 + WK) + std::max(4 * M * WK, 4 * kLaMaxNodes) + 32 + kWave * 20 + kWave * 4 + 96;
  static constexpr int kStages = std::min(6, (160 * 1024 - kSmall) / kTile);
  static_assert(kStages >= 3 && kRow % 256 == 128 && kLoads == kOffsets, "");
};
// Up to 128 rows: every wave takes 32 of them for the scores.  kHead as measured (serving batch of 2.4 pieces a workgroup: 346 us, with 8 351, with 5 357).
template <int C_, int R_, int TERMS_>
struct LatentWide {
  static constexpr bool kWide = true;
  static constexpr int C = C_, R = R_, TERMS = TERMS_;
  static constexpr int W = C + R;
  static constexpr int kHead = TERMS == 1 ? 12 : 5, kSnap = 4, kLeast = 4;      // see LaCut
  static constexpr bool kMoved = C == 256 && TERMS == 3;        // in the outer loop, see accumulate()
  static constexpr int M = 128, T = 32, WK = 1;
  static constexpr int kUnits = (W / 8 + 7) / 8 * 8;
  static constexpr int kRow = 16 * kUnits, kTile = T * kRow;
  static constexpr int kPages = T / kLaPage;
  static constexpr int RB = M / 32, CB = C / 4 / 32;            // 32-row blocks; 32-column blocks of a wave
  static constexpr int kSteps = W / 16;
  static constexpr int kLoads = kTile / kLaWaves / 1024;
  static constexpr int kOffsets = 8 * kRow / 1024;
  static constexpr int kInTile = T * 128 / 1024;                // of a tile's 8 TERMS operands of 1 KB: those that lie in the tile itself, where
  static constexpr int kWeights = (TERMS * 2 * RB - kInTile) * 1024, kBuffers = 2;      // the shared part of the keys was; the others' bytes
  static constexpr int kSmall = kBuffers * kWeights + kLaMaxNodes * 16 + 4 * M * (3 + WK) + std::max(4 * M * WK, 4 * kLaMaxNodes) + 32 + kWave * 20 +
                                2 * kOffsets * kWave * 4 + 96;
  static constexpr int kStages = std::min(4, (160 * 1024 - kSmall) / kTile);
  static_assert(kStages >= 3 && kRow % 256 == 128 && kLoads == kOffsets, "");
};

template <typename K>
struct LatentShared {
  __align__(1024) unsigned char ring[K::kStages][K::kTile];
  __align__(16) unsigned char p[K::kBuffers][K::kWeights];
  unsigned long long anc[kLaMaxNodes + 1][2];                   // of the nodes; the last: nodes with latents that are not finite, see take_out()
  int node[K::M];
  union {
    int parent[kLaMaxNodes];                                    // (until the ancestors are known)
    float top[K::WK][K::M];
  };
  float sum[K::WK][K::M], by[2][K::M];
  __align__(16) unsigned ahead[2][kLaWaves];
  double each, total;                                           // of the cut
  double upto[kWave];                                           // 64 requests: the cost up to the end of each, ...
  int ctx[kWave], first[kWave], n[kWave];
  unsigned off[K::kWide ? 2 : 1][K::kWide ? K::kOffsets : 1][kWave];      // where the bytes of a tile's load come from, in either half of a page
};

// Requests 64 k .. + 63 into LDS, and what they cost together; by all threads.
template <typename K>
__device__ __forceinline__ double load_requests(const LatentAttnParams& P, LatentShared<K>& S, int k) {
  const int tid = threadIdx.x + opaque_zero(), lane = tid & 63, b = 64 * k + lane;      // (nothing of this is kept across a piece)
  int ctx = 0, first = 0, n = 0;
  if (b < P.B) {
    ctx = min(max(P.ctx_len[b], 0), 0x7fffff00);                // (the end of the drafts still fits)
    first = P.q_offsets[b];
    n = first < 0 ? 0 : max(min(min(P.q_offsets[b + 1], P.total_q) - first, P.max_q), 0);
  }
  const int groups = (n * P.H + K::M - 1) / K::M;
  const double upto = wave_scan(static_cast<double>(groups) * (K::kHead + tiles_of<K::T>(P, ctx, n)));
  lds_sync();                                                   // (what was there has been read)
  if (tid < kWave) {
    S.upto[lane] = upto;
    S.ctx[lane] = ctx; S.first[lane] = first; S.n[lane] = n;
  }
  lds_sync();
  return lane_f64(upto, 63);
}
struct LatentPiece {
  int b, first, n, ctx, t0, t1, rows;
  int row_base;
  bool whole;
  int64_t part;               // first row of its partial result
};

// Row r of a tile, 16-byte unit u lies at u ^ fold(r): 16 rows' units of one place take 16 places of 16 bytes modulo the banks' 256 (rows are 128 bytes apart
// modulo 256, so r % 2 is told apart by itself).
__device__ __forceinline__ int fold(int r) { return 4 * ((r >> 1) & 1) + 2 * ((r >> 2) & 1) + ((r >> 3) & 1); }
// Where the bytes of a load come from, in the first 8 rows of a page; in the other 8 rows at ^ 16.  Units past the row's last repeat one.
template <typename K>
__device__ __forceinline__ void tile_offsets(unsigned (&off)[K::kOffsets], int lane) {
#pragma unroll
  for (int j = 0; j < K::kOffsets; ++j) {
    const int u = 64 * j + lane, r = u / K::kUnits, p = u % K::kUnits;
    int unit = p ^ fold(r);
    if constexpr (K::kUnits * 8 != K::W) unit = unit < K::W / 8 ? unit : unit & 3 | K::W / 8 - 4;
    off[j] = r * (K::W * 2) + unit * 16;
  }
}

// The rows' nodes, and the nodes' ancestors.
template <typename K>
__device__ __forceinline__ void find_lineage(const LatentAttnParams& P, LatentShared<K>& S, const LatentPiece& J, int tid, int parent) {
  if (tid < kLaMaxNodes) S.parent[tid] = parent;
  int heads = P.H;
  asm volatile("" : "+s"(heads));                               // (or its reciprocal is kept across pieces)
  if (tid < K::M) S.node[tid] = (J.row_base + min(tid, J.rows - 1)) / heads;
  lds_sync();
  if (tid <= kLaMaxNodes) {                                     // (the last: none yet)
    unsigned long long w[2] = {0ull, 0ull};
    if (tid < J.n) {
      if (P.parent) {
        int a = tid;
        for (int k = 0; k < kLaMaxNodes && a >= 0; ++k) {
          if (a < 64) w[0] |= 1ull << a; else w[1] |= 1ull << (a - 64);
          const int p = S.parent[a];
          a = (p >= a || p < 0) ? -1 : p;                       // (a malformed entry is a root)
        }
      } else {
        w[0] = tid < 63 ? (2ull << tid) - 1ull : ~0ull;
        w[1] = tid < 64 ? 0ull : (tid < 127 ? (2ull << (tid - 64)) - 1ull : ~0ull);
      }
    }
    S.anc[tid][0] = w[0];
    S.anc[tid][1] = w[1];
  }
}

// A weight of zero times what is not finite is NaN, also where the zero is that of a row that does not see the token: where rows differ in what they see, such
// values are taken out of V, and the drafts that had them noted (a row that sees one need not have met it in its scores: one of -infinity is a weight of zero).
// What all rows see stays.  By all threads, of tile t, that all have read for the scores; `none`: its pages that are none, a bit each.
template <typename K>
__device__ __forceinline__ void take_out(LatentShared<K>& S, unsigned tile, int tid, int t, int ctx, unsigned none) {
  constexpr int kUnits = K::C / 8, kBy = kLaThreads / kUnits, kFly = K::kWide ? 4 : K::T / kBy;
  const int shared = static_cast<int>(min(ctx - static_cast<int64_t>(t) * K::T, static_cast<int64_t>(K::T)));      // tokens of the context
  const unsigned mine = tile + tid / kUnits * K::kRow + tid % kUnits * 16;
#pragma unroll 1
  for (int from = 0; from < K::T; from += kBy * kFly) {
    raw4 w[kFly];
#pragma unroll
    for (int f = 0; f < kFly; ++f) w[f] = read_lds16(mine + (from + f * kBy) * K::kRow);
#pragma unroll
    for (int f = 0; f < kFly; ++f) {
      const int token = from + f * kBy + tid / kUnits, node = token - shared;
      const bool there = ((none >> (token / kLaPage)) & 1u) == 0u;
      raw4 x;
      bool any = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool l = (w[f][i] & 0x7f80u) == 0x7f80u, h = (w[f][i] & 0x7f800000u) == 0x7f800000u;
        any |= l | h;
        x[i] = (l ? 0u : w[f][i] & 0xffffu) | (h ? 0u : w[f][i] & 0xffff0000u);
      }
      if (!any || (there && node < 0)) continue;
      *lds_pointer<raw4>(mine + (from + f * kBy) * K::kRow) = x;
      if (there && node < kLaMaxNodes) atomicOr(&S.anc[kLaMaxNodes][node >> 6], 1ull << (node & 63));
    }
  }
}
// What a row's results are multiplied by, with z its sum of weights: NaN where it sees a draft that take_out has noted.
template <typename K>
__device__ __forceinline__ float result_factor(const LatentShared<K>& S, const LatentPiece& J, int row, float z) {
  if (J.t1 * static_cast<int64_t>(K::T) > J.ctx) {              // (else there are no nodes)
    const unsigned long long lo = S.anc[kLaMaxNodes][0], hi = S.anc[kLaMaxNodes][1];
    if ((lo | hi) != 0ull && ((S.anc[S.node[row]][0] & lo) | (S.anc[S.node[row]][1] & hi)) != 0ull) return __builtin_nanf("");
  }
  return z == 0.f ? 0.f : 1.f / z;
}

template <typename K>
__device__ __forceinline__ void write_results(const LatentAttnParams& P, LatentShared<K>& S, const LatentPiece& J, lf32x4 (&o)[K::CB][K::RB],
                                              float ref, float sum, int wave, int lane) {
  constexpr int WK = K::WK, RB = K::RB, CB = K::CB;
  const int tid = threadIdx.x, rn = lane & 15, g = lane >> 4;
  lds_sync();                                                   // (S.by has been read)
  const float z = groups_sum(sum);
  const int block = K::NB == 4 ? wave : wave >> 1, part = K::NB == 4 ? 0 : wave & 1;
  if (block < K::NB && lane < 16) {
    S.sum[part][16 * block + lane] = z;
    if (part == 0) S.by[0][16 * block + lane] = ref;
  }
  lds_sync();
  auto row_sum = [&](int row) __attribute__((always_inline)) {
    float z = S.sum[0][row];
#pragma unroll
    for (int k = 1; k < WK; ++k) z += S.sum[k][row];
    return z;
  };
  const int64_t row0 = static_cast<int64_t>(J.first) * P.H + J.row_base;
  if (tid < J.rows) {
    const float z = row_sum(tid), m = z == 0.f ? -INFINITY : S.by[0][tid];
    if (!J.whole) P.ws_ml[J.part + tid] = make_float2(m, z);
    else if (P.lse) P.lse[row0 + tid] = (m + log2f(z)) * static_cast<float>(kLn2);
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = 16 * rb + rn;
    if (row >= J.rows) continue;
    const float f = result_factor<K>(S, J, row, row_sum(row));
#pragma unroll
    for (int cb = 0; cb < CB; cb += 2) {
      const lf32x4 a = o[cb][rb] * f, b = o[cb + 1][rb] * f;
      const int col = wave * (K::C / 4) + 16 * cb + 8 * g;
      if (!J.whole || P.out_f32) {
        float* to = J.whole ? static_cast<float*>(P.out) + (row0 + row) * K::C + col : P.ws_o + (J.part + row) * K::C + col;
        *reinterpret_cast<float4*>(to) = make_float4(a[0], a[1], a[2], a[3]);
        *reinterpret_cast<float4*>(to + 4) = make_float4(b[0], b[1], b[2], b[3]);
      } else {
        const uint2 lo = pack4(a), hi = pack4(b);
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(P.out) + (row0 + row) * K::C + col) = make_uint4(lo.x, lo.y, hi.x, hi.y);
      }
    }
  }
}

// An accumulation in registers of their own kind (the compiler, left to choose, keeps results in vector registers and copies the queries' operands for
// every product).  Nothing that the compiler knows of may read or write x within a few instructions: see settle().  MOVED: where it keeps results in other
// registers for one of the loops, and moves them right in front of their products: a product reads what a vector instruction writes two wait states later.
// (tests/test_kernel_waits.py reads the built code for which kernels that is so.)
template <bool MOVED>
__device__ __forceinline__ void accumulate(lf32x16& x, lbf16x8 a, lbf16x8 b) {
  if constexpr (MOVED) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(x) : "v"(a), "v"(b));
  else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(x) : "v"(a), "v"(b));
}
__device__ __forceinline__ void clear(lf32x16& x) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float a;
    asm volatile("v_accvgpr_write_b32 %0, 0" : "=a"(a));
    x[i] = a;
  }
}
// x *= by, likewise, four at a time.
__device__ __forceinline__ void rescale(lf32x16& x, float by) {
#pragma unroll
  for (int i = 0; i < 16; i += 4) {
    float a = x[i], b = x[i + 1], c = x[i + 2], d = x[i + 3], t0, t1, t2, t3;
    asm volatile(
        "v_accvgpr_read_b32 %4, %0\n\tv_accvgpr_read_b32 %5, %1\n\tv_accvgpr_read_b32 %6, %2\n\tv_accvgpr_read_b32 %7, %3\n\t"
        "v_mul_f32 %4, %4, %8\n\tv_mul_f32 %5, %5, %8\n\tv_mul_f32 %6, %6, %8\n\tv_mul_f32 %7, %7, %8\n\t"
        "v_accvgpr_write_b32 %0, %4\n\tv_accvgpr_write_b32 %1, %5\n\tv_accvgpr_write_b32 %2, %6\n\tv_accvgpr_write_b32 %3, %7"
        : "+a"(a), "+a"(b), "+a"(c), "+a"(d), "=&v"(t0), "=&v"(t1), "=&v"(t2), "=&v"(t3) : "v"(by));
    x[i] = a; x[i + 1] = b; x[i + 2] = c; x[i + 3] = d;
  }
}
__device__ __forceinline__ void settle() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }
// max and sum over a lane and the one 32 away.
__device__ __forceinline__ float halves_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// What a piece leaves, from the sums and references in LDS.
template <typename K>
__device__ __forceinline__ void write_results_wide(const LatentAttnParams& P, LatentShared<K>& S, const LatentPiece& J, lf32x16 (&o)[K::CB][K::RB]) {
  constexpr int RB = K::RB, CB = K::CB, NS = K::kStages, TERMS = K::TERMS;
  const int tid = static_cast<int>(threadIdx.x) + opaque_zero(), lane = tid & 63, rn = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned ring = lds_address(&S.ring[0][0]);
  const int64_t row0 = static_cast<int64_t>(J.first) * P.H + J.row_base;
  if (tid < J.rows) {
    const float l = S.sum[0][tid], m = l == 0.f ? -INFINITY : S.by[0][tid];
    if (!J.whole) P.ws_ml[J.part + tid] = make_float2(m, l);
    else if (P.lse) P.lse[row0 + tid] = (m + log2f(l)) * static_cast<float>(kLn2);
    S.top[0][tid] = result_factor<K>(S, J, tid, l);
  }
  lds_sync();
  // Through LDS, so that a store takes consecutive bytes of rows (straight from the registers: 16 bytes of 64 rows, and 40000 cycles for a piece of fp32 results).
  auto put = [&](auto f32, auto row_blocks) __attribute__((always_inline)) {
    constexpr bool kF32 = decltype(f32)::value;
    constexpr int kTogether = decltype(row_blocks)::value, kBytes = K::C * (kF32 ? 4 : 2), kApart = kBytes + 16, kLanes = kBytes / 16;
    static_assert(kTogether * 32 * kApart <= NS * K::kTile, "");
    unsigned char* const to = kF32 && !J.whole ? reinterpret_cast<unsigned char*>(P.ws_o + J.part * K::C)
                                               : static_cast<unsigned char*>(P.out) + row0 * kBytes;
#pragma unroll
    for (int rb0 = 0; rb0 < RB; rb0 += kTogether) {
      if (rb0 > 0) lds_sync();
#pragma unroll
      for (int j = 0; j < kTogether; ++j) {
        const int rb = rb0 + j;
        const float f = S.top[0][32 * rb + rn];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          const unsigned at = ring + (32 * j + rn) * kApart + (wave * (K::C / 4) + 32 * cb + 16 * h) * (kF32 ? 4 : 2);
          const lf32x16 x = o[cb][rb] * f;
          if constexpr (kF32) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) *lds_pointer<lf32x4>(at + 4 * i) = lf32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
          } else {
#pragma unroll
            for (int i = 0; i < 16; i += 8)
              *lds_pointer<raw4>(at + 2 * i) = raw4{pack2(x[i], x[i + 1]), pack2(x[i + 2], x[i + 3]), pack2(x[i + 4], x[i + 5]), pack2(x[i + 6], x[i + 7])};
          }
        }
      }
      lds_sync();
      // rows r0, r0 + kBy, ..: eight reads of LDS on their way
      constexpr int kBy = kLaThreads / kLanes, kFly = 8;
      static_assert(kLaThreads % kLanes == 0 && kTogether * 32 % (kBy * kFly) == 0, "");
      const int r0 = tid / kLanes, c = tid % kLanes;
      unsigned char* line = to + static_cast<int64_t>(32 * rb0 + r0) * kBytes + 16 * c;
      for (int r = 0; r < kTogether * 32 && 32 * rb0 + r < J.rows; r += kBy * kFly) {
        raw4 x[kFly];
#pragma unroll
        for (int i = 0; i < kFly; ++i) x[i] = read_lds16(ring + (r0 + r + i * kBy) * kApart + 16 * c);
#pragma unroll
        for (int i = 0; i < kFly; ++i)
          if (32 * rb0 + r0 + r + i * kBy < J.rows) *reinterpret_cast<raw4*>(line + i * kBy * kBytes) = x[i];
        line += kBy * kFly * kBytes;
      }
    }
  };
  constexpr int kF32Blocks = 2 * 32 * (K::C * 4 + 16) <= NS * K::kTile ? 2 : 1;
  if (TERMS > 1 || !J.whole) put(std::true_type(), std::integral_constant<int, kF32Blocks>());
  else if constexpr (TERMS == 1) put(std::false_type(), std::integral_constant<int, 128 * (K::C * 2 + 16) <= NS * K::kTile ? 4 : 2>());
}

// Up to 128 query rows: matrix instructions bound it, and one wave per SIMD has to keep them busy by itself, at one instruction in 5 cycles.  32x32x16
// products: a lane has 16 of a tile's 32 scores of one query row (lane % 32; score i: token 8 (i / 4) + 4 (lane / 32) + i % 4), so that a wave works out the
// weights and the references of its 32 rows by itself.  In turn:
//   scores of tile t + 1 (36 products, a read of LDS each), at whose middle lies the barrier behind which all waves' weights of tile t are there, with the loads of
//   tile t + kStages - 1, then
//   O^T += V^T P^T of tile t (32 products), between which the weights of tile t + 1 are worked out.
// With four stages (C = 256) a tile's loads have the time of a whole tile and are waited for at the next one's barrier; with three, all that LDS holds at
// C = 512, they are waited for behind the results, with a second barrier.
// A tile of C = 512 takes 3250 cycles, 2176 of them in the products; 64 requests x 8192 tokens x 4 x 128 rows 490 to 505 us, 1160 to 1190 TFLOP/s.
template <typename K>
__device__ __forceinline__ void latent_piece_wide(const LatentAttnParams& P, LatentShared<K>& S, const LatentPiece& J) {
  constexpr int W = K::W, T = K::T, RB = K::RB, CB = K::CB, kPages = K::kPages, NS = K::kStages, kSteps = K::kSteps, TERMS = K::TERMS;
  static_assert(T == 32 && NS >= 3 && kPages == 2 && RB == kLaWaves, "");
  const int tid = static_cast<int>(threadIdx.x) + opaque_zero(), lane = tid & 63;
  __builtin_assume(tid >= 0 && tid < kLaThreads);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rn = lane & 31, h = lane >> 5;                      // query row of the block (matrix column), half
  const int L = J.ctx + J.n;

  constexpr int64_t kPageBytes = kLaPage * W * 2;
  const int32_t* bt = P.block_table + static_cast<int64_t>(J.b) * P.max_pages;
  const int last_page = min((L - 1) / kLaPage, P.max_pages - 1), num_pages = P.num_pages, max_pages = P.max_pages;
  const unsigned char* const pool = reinterpret_cast<const unsigned char*>(P.pool) + (wave & 1) * 8 * W * 2;      // this wave's half of its page
  const unsigned ring = lds_address(&S.ring[0][0]);
  // page ids of 32 tiles at a time, a lane each: through the scalar cache they would have every read of LDS waited for alike.  -1: none
  int ids = -1;
  auto fetch_ids = [&](int t) __attribute__((always_inline)) {
    const int lp = kPages * t + lane, id = bt[min(lp, last_page)];
    ids = id >= 0 && id < num_pages && lp < max_pages ? id : -1;
  };
  unsigned bad = 0u;                                            // pages that are none: 2 bits a tile, the present one's lowest
  // A tile's loads, of which a wave has kLoads: issued one by one among the products (all at once they wait for each other, 700 cycles a tile).
  const unsigned char* page = pool;
  unsigned to = 0;
  auto aim = [&](int t, int slot, int ahead) __attribute__((always_inline)) {
    const int at = (kPages * (t - J.t0)) & 63;
    const int a = __builtin_amdgcn_readlane(ids, at), b = __builtin_amdgcn_readlane(ids, at + 1);
    bad |= ((a < 0 ? 1u : 0u) | (b < 0 ? 2u : 0u)) << (kPages * ahead);
    page = pool + max(wave < 2 ? a : b, 0) * kPageBytes;        // (one that is none of the pool's: page 0 in its place)
    to = ring + slot * K::kTile + wave * (K::kTile / kLaWaves);
  };
  const unsigned off_at = lds_address(reinterpret_cast<unsigned char*>(&S.off[0][0][0])) + ((wave & 1) * K::kOffsets * kWave + lane) * 4;
  unsigned off = 0;                                             // of the next load, read well ahead
  auto read_off = [&](int j) __attribute__((always_inline)) {
    unsigned at = off_at;
    asm volatile("" : "+v"(at));
    off = *lds_pointer<unsigned>(at + j * kWave * 4);
  };
  auto issue = [&](int j) __attribute__((always_inline)) {
    load_to_lds(page, off, to + 1024 * j, 0);
    if (j + 1 < K::kLoads) read_off(j + 1);
  };

  const bool touches_drafts = J.t1 * static_cast<int64_t>(T) > J.ctx;
  int parent = -1;
  if (touches_drafts && P.parent && tid < J.n) parent = P.parent[J.first + tid];
  fetch_ids(J.t0);
  lds_sync();                                                   // the LDS of the piece before is free

  // The queries' operands, each wave's 32 rows in two times 16, laid out as a tile's are in the last two slots, while the first tiles come into the others (each lane
  // 16 bytes of a row of its own, straight from memory: 64 lines a load, and twice the time).  Rows past the last, which nobody looks at, have bytes of the last.
  lbf16x8 qf[kSteps];
  {
    unsigned off[K::kOffsets];
    tile_offsets<K>(off, lane);
    if (wave < 2) {                                             // (the same for every piece)
#pragma unroll
      for (int j = 0; j < K::kOffsets; ++j) S.off[wave][j][lane] = off[j] ^ (16 * wave);
    }
    const unsigned char* const q = reinterpret_cast<const unsigned char*>(P.q) + (static_cast<int64_t>(J.first) * P.H + J.row_base) * (W * 2);
    const unsigned mine = ring + (NS - 2) * K::kTile + wave * (16 * K::kRow);
    auto bring = [&](int half) __attribute__((always_inline)) {
#pragma unroll
      for (int eight = 0; eight < 2; ++eight) {
        const int row = min(32 * wave + 16 * half + 8 * eight, J.rows - 1);
        const unsigned last = (J.rows - row) * (W * 2) - 16;
#pragma unroll
        for (int j = 0; j < K::kOffsets; ++j) load_to_lds(q + row * (W * 2), min(off[j] ^ (16 * eight), last), mine + eight * (8 * K::kRow) + 1024 * j, 0);
      }
    };
    auto take = [&](int half) __attribute__((always_inline)) {
      const unsigned at = mine + (rn & 15) * K::kRow + (h ^ fold(rn)) * 16;
      if (rn >> 4 == half) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) qf[s] = operand(read_lds16((at ^ (32 * (s & 3))) + 128 * (s >> 2)));
      }
    };
    bring(0);
    lds_sync();                                                 // (S.off)
#pragma unroll
    for (int i = 0; i < NS - 2; ++i) {
      if (J.t0 + i >= J.t1) break;
      aim(J.t0 + i, i, i);
      read_off(0);
#pragma unroll
      for (int j = 0; j < K::kLoads; ++j) issue(j);
    }
    if (J.t0 + NS - 2 <= J.t1) wait_loads<(NS - 2) * K::kLoads>();        // (not for the tiles)
    else wait_loads<0>();
    take(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // (what was there has been read)
    bring(1);
    if (touches_drafts) find_lineage<K>(P, S, J, tid, parent);
    wait_loads<0>();
    take(1);
    lds_sync();
    if (J.t0 + NS - 2 < J.t1) {
      aim(J.t0 + NS - 2, NS - 2, NS - 2);
      read_off(0);
#pragma unroll
      for (int j = 0; j < K::kLoads; ++j) issue(j);
    }
  }

  // Operand reads.  K: token rn, unit 2 s + h.  V by columns: lane i of 16 (group G of two in a half) points at token 4 h + i / 4 (and 8 more), column
  // 16 (i % 2) + 8 G + 4 (i / 2 % 2): column 16 h + 4 a + e of the wave's 32 is row 8 a + 4 h + e of the block, so that a lane ends up with 16 consecutive ones.
  const unsigned k_at = rn * K::kRow + (h ^ fold(rn)) * 16;     // step s at ^ 32 (s % 4), 128 (s / 4) more
  const int vi = lane & 15, vt = 4 * h + (vi >> 2);
  const unsigned v_at = vt * K::kRow + ((2 * (vi & 1) + ((lane >> 4) & 1)) ^ fold(vt)) * 16 + 8 * ((vi >> 1) & 1) + wave * (K::C / 4 * 2);   // block cb at ^ 64 (cb % 2)
  // weights: the first kInTile operands lie in the tile's rows behind the latents, 8 lanes to a row
  static_assert(K::kInTile == RB, "the operands in the tile are those of one term and half of the tokens");
  const unsigned in_tile = (lane >> 3) * K::kRow + K::C * 2 + (lane & 7) * 16, apart = lds_address(&S.p[0][0]) + 16 * lane;
  // (bases that the compiler knows no parts of, so that it does not keep one for every constant behind them)
  auto opaque = [&](unsigned at) __attribute__((always_inline)) { asm volatile("" : "+v"(at)); return at; };
  auto read_p = [&](unsigned inside, unsigned outside, int f) __attribute__((always_inline)) {
    return operand(read_lds16(f < K::kInTile ? inside + f * 8 * K::kRow : outside + (f - K::kInTile) * 1024));
  };

  float ref = kLaNoScore, sum = 0.f, z = 0.f;
  lf32x16 o[CB][RB];
  lf32x16 s;
  constexpr int kDeep = 7;                                      // K is read six steps ahead
  lbf16x8 k[kDeep];
  // (the shared part of the keys first: weights go where it lies, behind a barrier after these steps)
  auto place = [](int step) { return step < K::R / 16 ? K::C / 16 + step : step - K::R / 16; };
  auto read_k = [&](unsigned tile, int step) __attribute__((always_inline)) {
    const int at = place(step);
    k[step % kDeep] = operand(read_lds16(((tile + k_at) ^ (32 * (at & 3))) + 128 * (at >> 2)));
  };
  auto score = [&](unsigned tile, int step) __attribute__((always_inline)) {
    if (step + kDeep - 1 < kSteps) read_k(tile, step + kDeep - 1);
    lf32x16 zero;
#pragma unroll
    for (int i = 0; i < 16; ++i) zero[i] = 0.f;
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[step % kDeep], qf[place(step)], step == 0 ? zero : s, 0, 0, 0);
  };
  // From this tile on rows differ in what they see (or, behind the last tile, see nothing).
  const int drafts_from = min(J.ctx / T, J.t1);
  // of tile t, whose pages' bits are `none`: scores that a row does not see; behind the last tile, all
  auto mask = [&](int t, unsigned none) __attribute__((always_inline)) {
    const int node = touches_drafts ? S.node[32 * wave + rn] : 0;
#pragma unroll
    for (int page = 0; page < 2; ++page) {
      const int64_t past = static_cast<int64_t>(t) * T + 16 * page - J.ctx;
      uint32_t seen = 0xffffu;
      if (past > -16 && t < J.t1) seen = page_mask(S.anc[node][0], S.anc[node][1], static_cast<int>(past));
      seen = ((none >> page) & 1u) != 0u || t >= J.t1 ? 0u : seen >> (4 * h);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[8 * page + i] = (seen >> (8 * (i >> 2) + (i & 3))) & 1u ? s[8 * page + i] : -INFINITY;
    }
  };
  // A row's reference follows its maximum where that has come far ahead (each row by itself: its result has the same bits whatever the others are); what the
  // results of the tiles before have to be scaled by is left for all waves, which look at the flags behind the next barrier.
  float top = 0.f;
  auto find_top = [&](int part) __attribute__((always_inline)) {
    if (part == 0) top = max3(s[0], s[1], s[2]);
#pragma unroll
    for (int i = part == 0 ? 3 : 9; i < (part == 0 ? 9 : 15); i += 2) top = max3(top, s[i], s[i + 1]);
    if (part == 1) top = __builtin_elementwise_maximum(top, s[15]) * P.c;
  };
  auto refer = [&](int t) __attribute__((always_inline)) {
    const unsigned flag = any_lane(top > ref + kLaSlack) ? 1u : 0u;
    S.ahead[t & 1][wave] = flag;
    if (__builtin_expect(flag != 0u, 0)) {
      const float now = halves_max(top), next = now > ref + kLaSlack ? now : ref, by = fast_exp2(ref - next);
      ref = next;
      sum *= by;
      S.by[t & 1][32 * wave + rn] = by;
    }
  };
  // weights of pair i of a lane's 8 pairs of scores; four pairs make an operand
  uint32_t w[TERMS][4];
  float p0 = 0.f, p1 = 0.f;
  auto weigh_pair = [&](unsigned inside, unsigned outside, int i, int part) __attribute__((always_inline)) {
    if (part == 0) p0 = fast_exp2(fmaf(s[2 * i], P.c, -ref));
    if (part == 1) p1 = fast_exp2(fmaf(s[2 * i + 1], P.c, -ref));
    if (part < 2) return;
    z = i == 0 ? p0 + p1 : z + (p0 + p1);
    asm volatile("" : "+v"(z));                                 // (here, and not where the sum is first needed)
    float r0 = p0, r1 = p1;
#pragma unroll
    for (int term = 0; term < TERMS; ++term) {
      w[term][i & 3] = pack2(r0, r1);
      r0 -= bf16_lo(w[term][i & 3]);
      r1 -= bf16_hi(w[term][i & 3]);
    }
    if ((i & 3) == 3) {
#pragma unroll
      for (int term = 0; term < TERMS; ++term) {
        const int f = 2 * RB * term + RB * (i >> 2);            // operand f + wave
        *lds_pointer<raw4>(f < K::kInTile ? inside + wave * (8 * K::kRow) : outside + (f - K::kInTile + wave) * 1024) =
            raw4{w[term][0], w[term][1], w[term][2], w[term][3]};
      }
    }
  };

  constexpr int kBarrier = 8, kCheck = kBarrier + (kSteps - kBarrier) / 3, kRead = kCheck + (kSteps - kCheck) / 3;
  static_assert(kBarrier >= K::R / 16, "the shared part of the keys has been read");
  auto issue_at = [&](int step) __attribute__((always_inline)) {
    constexpr int kEvery = (kSteps - kBarrier) / K::kLoads;
    static_assert(kEvery >= 2, "");
    const int at = step - kBarrier;
    if (at % kEvery == 1 && at / kEvery < K::kLoads) issue(at / kEvery);
  };
  // The first scores of the tile behind t (past the last one: of whatever is there), up to where the flags of tile t are known.  Not 0: there is something to be
  // done before tile t is added: results are to be scaled, or rows differ in what they see.
  auto first_half = [&](int t, int slot) __attribute__((always_inline)) {
    const unsigned tile1 = ring + (slot + 1 == NS ? 0 : slot + 1) * K::kTile;
#pragma unroll
    for (int step = 0; step < kBarrier; ++step) {
      score(tile1, step);
      if (step == 1) {
        const int ahead = min(t + NS - 1, J.t1 - 1);            // (behind the last tile that one again, which nobody looks at)
        if (__builtin_expect(ahead == t + NS - 1 && ((kPages * (ahead - J.t0)) & 63) == 0, 0)) fetch_ids(ahead);
        aim(ahead, slot == 0 ? NS - 1 : slot - 1, NS - 1);
      }
      if (step == kBarrier - 1) read_off(0);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (NS == 4) wait_loads<0>();                               // the tile after next is here
    lds_sync();
    const raw4 flags = *reinterpret_cast<const raw4*>(S.ahead[t & 1]);
    unsigned special = 0u;
#pragma unroll
    for (int step = kBarrier; step < kCheck; ++step) {
      score(tile1, step);
      issue_at(step);
      if (step == kCheck - 2) special = __builtin_amdgcn_readfirstlane(flags[0] | flags[1] | flags[2] | flags[3]) | (bad & 3u) | (t >= drafts_from ? 1u : 0u);
      __builtin_amdgcn_sched_barrier(0);
    }
    return special;
  };
  // The rest of the scores; O^T += V^T P^T of tile t, and the weights of the tile behind it.
  auto second_half = [&](auto moved, int t, int slot) __attribute__((always_inline)) {
    const int slot1 = slot + 1 == NS ? 0 : slot + 1;
    const unsigned tile = ring + slot * K::kTile, tile1 = ring + slot1 * K::kTile, tile2 = ring + (slot1 + 1 == NS ? 0 : slot1 + 1) * K::kTile;
#pragma unroll
    for (int step = kCheck; step < kRead; ++step) {
      score(tile1, step);
      issue_at(step);
      if (step == kCheck) sum += z;
      __builtin_amdgcn_sched_barrier(0);
    }
    const unsigned inside = opaque(tile + in_tile), outside = opaque(apart + (t & 1) * K::kWeights), v_base = opaque(tile + v_at), v_other = v_base ^ 16;
    const unsigned inside1 = opaque(tile1 + in_tile), outside1 = opaque(apart + ((t + 1) & 1) * K::kWeights);
    lbf16x8 p[2][RB];
    ls16x4 v[3][2];
    auto read_v = [&](int b, int part) __attribute__((always_inline)) {                     // block b % CB, tokens 16 (b / CB % 2) ..
      const unsigned at = part == 0 ? v_base : v_other;
      v[b % 3][part] = read_columns((at ^ (64 * (b % CB & 1))) + 128 * (b % CB >> 1) + (b / CB % 2 * 16 + part * 8) * K::kRow);
    };
#pragma unroll
    for (int step = kRead; step < kSteps; ++step) {
      score(tile1, step);
      issue_at(step);
      constexpr int kReads = RB + 4, kAt = (kReads + kSteps - kRead - 1) / (kSteps - kRead);
#pragma unroll
      for (int at = (step - kRead) * kAt; at < (step - kRead + 1) * kAt && at < kReads; ++at) {      // operands of the first products
        if (at < RB) p[0][at] = read_p(inside, outside, at);
        else read_v((at - RB) >> 1, (at - RB) & 1);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (__builtin_expect(t + 1 >= drafts_from || (bad & (3u << kPages)) != 0u, 0)) mask(t + 1, (bad >> kPages) & 3u);
    // one product, and what a lane has for it of the next tile's weights and of operand reads: what the products' 32 cycles hold
    constexpr int kBlocks = 2 * CB * TERMS, kProducts = kBlocks * RB;
    auto beside = [&](int at) __attribute__((always_inline)) {
      if (at < 2) find_top(at);
      if (at == 2) refer(t + 1);
      constexpr int kPer = kProducts >= 28 ? 3 : 1;             // products for a pair
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int part = 0; part < 3; ++part)
          if (at == 3 + i * kPer + (kPer > 1 ? part : 0)) weigh_pair(inside1, outside1, i, part);
      const int late = at - (kProducts - (kDeep - 1));
      if (NS == 4 && late >= 0) read_k(tile2, late);
    };
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      const int next = b / CB + 1;                              // operands: of a term's first or second 16 tokens
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        if (rb < 2 && b + 2 < kBlocks) read_v(b + 2, rb);
        if (b % CB == CB - 2 && next < 2 * TERMS) p[next & 1][rb] = read_p(inside, outside, RB * next + rb);
        accumulate<decltype(moved)::value>(o[b % CB][rb], join(v[b % 3][0], v[b % 3][1]), p[b / CB & 1][rb]);
        beside(b * RB + rb);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    bad >>= kPages;
    if (NS == 3) {
      wait_loads<0>();
      lds_sync();
#pragma unroll
      for (int step = 0; step < kDeep - 1; ++step) read_k(tile2, step);
    }
  };

  // ---- the first tile's scores and weights ----
#pragma unroll
  for (int step = 0; step < kDeep - 1; ++step) read_k(ring, step);
#pragma unroll
  for (int step = 0; step < kSteps; ++step) {
    score(ring, step);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (J.t0 >= drafts_from || (bad & 3u) != 0u) mask(J.t0, bad & 3u);
  if (NS == 3) wait_loads<0>();                                 // the second tile
  lds_sync();                                                   // all have read the shared part of the keys
  find_top(0);
  find_top(1);
  refer(J.t0);
  {
    const unsigned inside = opaque(ring + in_tile), outside = opaque(apart + (J.t0 & 1) * K::kWeights);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int part = 0; part < 3; ++part) weigh_pair(inside, outside, i, part);
    }
  }
#pragma unroll
  for (int step = 0; step < kDeep - 1; ++step) read_k(ring + K::kTile, step);
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) clear(o[cb][rb]);
  int slot = 0, t = J.t0;
  unsigned special = first_half(t, slot);
  // (Two loops: results are scaled in the outer one alone, which keeps their registers where the products have them.)
  for (;;) {
    if (special) {
      settle();
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        if (__builtin_amdgcn_readfirstlane(S.ahead[t & 1][rb]) == 0u) continue;
        const float by = S.by[t & 1][32 * rb + rn];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) rescale(o[cb][rb], by);
      }
      settle();
      if (t >= drafts_from || (bad & 3u) != 0u) {
        take_out<K>(S, ring + slot * K::kTile, tid, t, J.ctx, bad & 3u);
        lds_sync();
      }
    }
    bool more;
    if constexpr (K::kMoved) {                                  // (a copy of its own for the outer loop, where the moves are)
      second_half(std::true_type(), t, slot);
      slot = slot + 1 == NS ? 0 : slot + 1;
      if (++t >= J.t1) break;
      special = first_half(t, slot);
      if (special != 0u) continue;
    }
    do {
      second_half(std::false_type(), t, slot);
      slot = slot + 1 == NS ? 0 : slot + 1;
      more = ++t < J.t1;
      if (!more) break;
      special = first_half(t, slot);
    } while (__builtin_expect(special == 0u, 1));
    if (!more) break;
  }
  settle();
  wait_loads<0>();

  // ---- results ----
  lds_sync();                                                   // (S.by has been read)
  sum = halves_sum(sum);
  if (h == 0) {
    S.sum[0][32 * wave + rn] = sum;
    S.by[0][32 * wave + rn] = ref;
  }
  lds_sync();
  write_results_wide<K>(P, S, J, o);
}

// Up to 64 query rows: memory bounds it, or with 64 the chain of a tile: scores, weights to LDS, a barrier, results.  Two tiles or more are on their way meanwhile; the
// next tile is there behind the same barrier, so that the first of its keys are read beside the results.
template <typename K>
__device__ __forceinline__ void latent_piece(const LatentAttnParams& P, LatentShared<K>& S, const LatentPiece& J) {
  constexpr int W = K::W, T = K::T, KB = K::KB, WK = K::WK, RB = K::RB, CB = K::CB, kPages = K::kPages, NS = K::kStages, TERMS = K::TERMS;
  const int tid = static_cast<int>(threadIdx.x) + opaque_zero(), lane = tid & 63;
  __builtin_assume(tid >= 0 && tid < kLaThreads);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rn = lane & 15, g = lane >> 4;
  const int block = K::NB == 4 ? wave : wave >> 1, part = K::NB == 4 ? 0 : wave & 1;      // of the scores: this wave's rows 16 block .., tokens 16 part ..
  const bool scores = block < K::NB;
  const int L = J.ctx + J.n;

  unsigned off[K::kOffsets];
  tile_offsets<K>(off, lane);
#pragma unroll
  for (int j = 0; j < K::kOffsets; ++j) off[j] ^= 16 * (wave & 1);
  constexpr int64_t kPageBytes = kLaPage * W * 2;
  const int32_t* bt = P.block_table + static_cast<int64_t>(J.b) * P.max_pages;
  const int last_page = min((L - 1) / kLaPage, P.max_pages - 1);
  const unsigned ring = lds_address(&S.ring[0][0]);
  const unsigned char* const pool = reinterpret_cast<const unsigned char*>(P.pool) + (wave & 1) * 8 * W * 2;      // this wave's half of its page
  // page ids of 32 tiles at a time, a lane each (through the scalar cache they would have every read of LDS waited for alike).  -1: none
  int ids = -1;
  auto fetch_ids = [&](int t) __attribute__((always_inline)) {
    const int lp = kPages * t + lane, id = bt[min(lp, last_page)];
    ids = id >= 0 && id < P.num_pages && lp < P.max_pages ? id : -1;
  };
  unsigned bad = 0u;                                            // pages that are none: 2 bits a tile, the present one's lowest
  const unsigned char* page = pool;
  unsigned to = 0;
  auto aim = [&](int t, int slot, int ahead) __attribute__((always_inline)) {
    const int at = (kPages * (t - J.t0)) & 63;
    if (at == 0) fetch_ids(t);
    const int a = __builtin_amdgcn_readlane(ids, at), b = __builtin_amdgcn_readlane(ids, at + 1);
    bad |= ((a < 0 ? 1u : 0u) | (b < 0 ? 2u : 0u)) << (kPages * ahead);
    page = pool + max(wave < 2 ? a : b, 0) * kPageBytes;        // (one that is none of the pool's: page 0 in its place)
    to = ring + slot * K::kTile + wave * (K::kTile / kLaWaves);
  };
  auto issue = [&](int j) __attribute__((always_inline)) { load_to_lds(page, off[j], to + 1024 * j, 0); };

  // ---- the queries' operands: rows past the last repeat it ----
  lbf16x8 qf[K::kSteps];
  {
    const uint16_t* row = P.q + (static_cast<int64_t>(J.first) * P.H + J.row_base + min(16 * block + rn, J.rows - 1)) * W + 8 * g;
#pragma unroll
    for (int s = 0; s < K::kSteps; ++s) qf[s] = operand(*reinterpret_cast<const raw4*>(row + 32 * s));
  }
  const bool touches_drafts = J.t1 * static_cast<int64_t>(T) > J.ctx;
  int parent = -1;
  if (touches_drafts && P.parent && tid < J.n) parent = P.parent[J.first + tid];
  lds_sync();                                                   // the LDS of the piece before is free
#pragma unroll
  for (int i = 0; i < NS - 1; ++i) {
    if (J.t0 + i >= J.t1) break;
    aim(J.t0 + i, i, i);
#pragma unroll
    for (int j = 0; j < K::kLoads; ++j) issue(j);
  }
  if (touches_drafts) find_lineage<K>(P, S, J, tid, parent);

  // Operand reads: K, token 16 part + rn, unit 4 s + g; V by columns, token 4 g + rn / 4 (and 16 more), unit 4 (cb / 2) + rn % 4, half cb % 2: column
  // 32 p + 8 g + 4 s + i of the wave's is row 4 g + i of block 2 p + s, so that a lane ends up with 8 consecutive ones
  const unsigned k_at = (16 * part + rn) * K::kRow + (g ^ fold(rn)) * 16;           // even steps; odd ones at ^ 64; 128 more every two
  const int vt = 4 * g + (rn >> 2);
  const unsigned v_at = vt * K::kRow + ((rn & 3) ^ fold(vt)) * 16 + wave * (K::C / 4 * 2);   // even pairs of blocks; odd ones at ^ 64; 128 more every two
  const unsigned p_at = lds_address(&S.p[0][0]) + 16 * lane;

  float ref = kLaNoScore, sum = 0.f;
  lf32x4 o[CB][RB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) o[cb][rb] = lf32x4{0.f, 0.f, 0.f, 0.f};

  // All but the last `ahead` tiles (or fewer, of all that there are) have come.
  auto arrived = [&](int ahead) __attribute__((always_inline)) {
    if (NS >= 6 && ahead >= 4) wait_loads<4 * K::kLoads>();
    else if (NS >= 5 && ahead == 3) wait_loads<3 * K::kLoads>();
    else if (NS >= 4 && ahead == 2) wait_loads<2 * K::kLoads>();
    else if (ahead == 1) wait_loads<K::kLoads>();
    else wait_loads<0>();
  };
  constexpr int kDeep = 8;                                      // K is read seven steps ahead
  lbf16x8 k[kDeep][KB];
  auto read_k = [&](unsigned tile, int step) __attribute__((always_inline)) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) k[step % kDeep][kb] = operand(read_lds16(((tile + k_at) ^ (64 * (step & 1))) + 128 * (step >> 1) + kb * 16 * K::kRow));
  };
  arrived(min(NS - 2, J.t1 - 1 - J.t0));
  lds_sync();
#pragma unroll
  for (int step = 0; step < kDeep - 1; ++step) read_k(ring, step);

  int slot = 0;
  for (int t = J.t0; t < J.t1; ++t) {
    const unsigned tile = ring + slot * K::kTile;
    const bool special = (t + 1) * static_cast<int64_t>(T) > J.ctx || (bad & 3u) != 0u;

    // ---- scores ----
    lf32x4 s[KB];
    float top = -INFINITY, z = 0.f;
    auto weigh = [&]() __attribute__((always_inline)) {
      uint32_t w[TERMS][KB][2];
      z = 0.f;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float p0 = fast_exp2(fmaf(s[kb][2 * i], P.c, -ref)), p1 = fast_exp2(fmaf(s[kb][2 * i + 1], P.c, -ref));
          z += p0 + p1;
          float r0 = p0, r1 = p1;
#pragma unroll
          for (int term = 0; term < TERMS; ++term) {
            w[term][kb][i] = pack2(r0, r1);
            r0 -= bf16_lo(w[term][kb][i]);
            r1 -= bf16_hi(w[term][kb][i]);
          }
        }
      // the two blocks of 16 tokens are the halves of a lane's 16 bytes
#pragma unroll
      for (int term = 0; term < TERMS; ++term) {
        const unsigned at = p_at + (t & 1) * K::kWeights + (term * RB + block) * 1024;
        if constexpr (KB == 1) *lds_pointer<unsigned long long>(at + 8 * part) = static_cast<unsigned long long>(w[term][0][1]) << 32 | w[term][0][0];
        else *lds_pointer<raw4>(at) = raw4{w[term][0][0], w[term][0][1], w[term][1][0], w[term][1][1]};
      }
    };
    if (scores) {
#pragma unroll
      for (int step = 0; step < K::kSteps; ++step) {
        if (step + kDeep - 1 < K::kSteps) read_k(tile, step + kDeep - 1);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) s[kb] = multiply(k[step % kDeep][kb], qf[step], step == 0 ? lf32x4{0.f, 0.f, 0.f, 0.f} : s[kb]);
        __builtin_amdgcn_sched_barrier(0);
      }
      // masks: only where the tile reaches the drafts, or a page is none
      if (special) {
        const int node = S.node[16 * block + rn];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const int page = part + kb;
          const int64_t past = static_cast<int64_t>(t) * T + 16 * page - J.ctx;
          uint32_t seen = 0xffffu;
          if (past > -16) seen = page_mask(S.anc[node][0], S.anc[node][1], static_cast<int>(past));
          seen = (bad >> page) & 1u ? 0u : seen >> (4 * g);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[kb][i] = (seen >> i) & 1u ? s[kb][i] : -INFINITY;
        }
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) top = max3(top, max3(s[kb][0], s[kb][1], s[kb][2]), s[kb][3]);
      top *= P.c;
      weigh();
    }
    // ---- behind the barrier: all weights are there, the next tile is, and all waves are done with the one before ----
    const unsigned flag = any_lane(top > ref + kLaSlack) ? 1u : 0u;
    if (lane == 0) S.ahead[t & 1][wave] = flag;
    arrived(min(NS - 3, J.t1 - 2 - t));
    lds_sync();
    const raw4 flags = *reinterpret_cast<const raw4*>(S.ahead[t & 1]);
    const bool another = t + NS - 1 < J.t1;
    if (another) aim(t + NS - 1, slot == 0 ? NS - 1 : slot - 1, NS - 1);
    slot = slot + 1 == NS ? 0 : slot + 1;
    if (__builtin_amdgcn_readfirstlane(flags[0] | flags[1] | flags[2] | flags[3])) {
      // ---- a row's reference follows its maximum where that has come far ahead (in all waves, or in none) ----
      if (scores) {
        const float m = groups_max(top);
        if (lane < 16) S.top[part][16 * block + lane] = m;
      }
      lds_sync();
      if (scores) {
        const int row = 16 * block + rn;
        float now = S.top[0][row];
#pragma unroll
        for (int k = 1; k < WK; ++k) now = fmaxf(now, S.top[k][row]);
        now = now > ref + kLaSlack ? now : ref;                 // (each row by itself: its result has the same bits whatever the others are)
        const float by = fast_exp2(ref - now);
        ref = now;
        sum *= by;
        if (part == 0 && lane < 16) S.by[0][row] = by;
        weigh();
      }
      lds_sync();
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float by = S.by[0][16 * rb + rn];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) o[cb][rb] *= by;
      }
    }
    sum += z;

    if (special) {
      take_out<K>(S, tile, tid, t, J.ctx, bad & 3u);
      lds_sync();
    }

    // ---- O^T += V^T P^T ----
    lbf16x8 p[TERMS][RB];
#pragma unroll
    for (int term = 0; term < TERMS; ++term)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) p[term][rb] = operand(read_lds16(p_at + (t & 1) * K::kWeights + (term * RB + rb) * 1024));
    lbf16x8 v[3];
    auto read_v = [&](int cb) __attribute__((always_inline)) {
      const unsigned at = ((tile + v_at) ^ (64 * ((cb >> 1) & 1))) + 128 * (cb >> 2) + 8 * (cb & 1);
      v[cb % 3] = join(read_columns(at), read_columns(at + 16 * K::kRow));
    };
    read_v(0);
    read_v(1);
    // (a tile's loads lie between the products: all at once they wait for each other)
    if (another) issue(0);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      if (cb + 2 < CB) read_v(cb + 2);
#pragma unroll
      for (int step = cb * kDeep / CB; step < (cb + 1) * kDeep / CB && step < kDeep - 1; ++step) read_k(ring + slot * K::kTile, step);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int term = 0; term < TERMS; ++term) o[cb][rb] = multiply(v[cb % 3], p[term][rb], o[cb][rb]);
      }
      if (another && cb + 1 < K::kLoads) issue(cb + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    static_assert(K::kLoads <= CB + 1, "");
    bad >>= kPages;
  }

  write_results<K>(P, S, J, o, ref, sum, wave, lane);
}

template <typename K>
__global__ __launch_bounds__(kLaThreads, 1) void attn_latent_kernel(LatentAttnParams P) {
  extern __shared__ __align__(1024) unsigned char smem[];
  auto& S = *reinterpret_cast<LatentShared<K>*>(smem);
  constexpr int M = K::M, T = K::T;
  const int batches = (P.B + 63) / 64;
  if (threadIdx.x == 0) P.cut[blockIdx.x] = make_int4(0, 0, 0, 0);
  double total = 0.0;
  for (int k = batches - 1; k >= 0; --k) total += load_requests<K>(P, S, k);        // (down: the first 64 requests stay)
  total = uniform(total);
  const LaCut cut = cut_ranges(P.ranges, K::kLeast, total);
  // Workgroups go to the 8 XCDs in turn: renumbered so that neighbouring ranges, which may hold groups of rows of one request, share an L2
  const int each = (cut.used + 7) >> 3, range = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  if (!any_lane(total > 0.0) || static_cast<int>(blockIdx.x >> 3) >= each || range >= cut.used) return;
  if (threadIdx.x == 0) {
    S.each = cut.each;
    S.total = cut.total;
  }
  const double end = uniform(range_start(cut, range + 1));
  double at = uniform(range_start(cut, range)), base = 0.0;     // cost before these 64 requests
  const int used = cut.used;
  // (Nothing but these and the requests in LDS is kept across a piece: it has use for all registers.)
  for (int k = 0; any_lane(at < end);) {
    const int lane = (threadIdx.x + opaque_zero()) & 63;
    const unsigned long long later = __builtin_amdgcn_ballot_w64(base + S.upto[lane] > at);
    if (later == 0ull) {
      base = uniform(base + S.upto[63]);
      if (++k >= batches) break;
      load_requests<K>(P, S, k);
      continue;
    }
    const int i = __ffsll(later) - 1;
    LatentPiece J;
    J.b = 64 * k + i;
    J.ctx = __builtin_amdgcn_readfirstlane(S.ctx[i]);
    J.first = __builtin_amdgcn_readfirstlane(S.first[i]);
    J.n = __builtin_amdgcn_readfirstlane(S.n[i]);
    const int rows = J.n * P.H, groups = (rows + M - 1) / M, tiles = tiles_of<T>(P, J.ctx, J.n);
    const double cost = K::kHead + tiles, start0 = base + S.upto[i] - groups * cost;
    int grp = 0;                                                // the group that `at` lies in
    if (groups > 1) {
      grp = min(max(static_cast<int>((at - start0) / cost), 0), groups - 1);
      if (start0 + grp * cost > at) --grp;
      else if (start0 + (grp + 1) * cost <= at) ++grp;
    }
    const double start = start0 + grp * cost;
    // tile k is at start + kHead + k and belongs to the range that this is in
    auto tile_at = [&](double x) { return static_cast<int>(fmin(fmax(border<K>(x, start, start + cost) - start - K::kHead, 0.0), static_cast<double>(tiles))); };
    J.t0 = __builtin_amdgcn_readfirstlane(tile_at(at));
    J.t1 = __builtin_amdgcn_readfirstlane(tile_at(end));
    at = uniform(start + cost);
    if (J.t0 >= J.t1) continue;
    J.row_base = __builtin_amdgcn_readfirstlane(M * grp);
    J.rows = min(rows - J.row_base, M);
    J.whole = J.t0 == 0 && J.t1 == tiles;
    J.part = (static_cast<int64_t>(range) * 2 + (J.t0 == 0 ? 1 : 0)) * M;
    if (!J.whole && J.t0 == 0 && threadIdx.x == 0) {
      const LaCut again = {used, S.each, S.total};
      int last = range_of(again, start + cost - 1);
      while (border<K>(range_start(again, last), start, start + cost) == start + cost) --last;
      const int64_t row0 = static_cast<int64_t>(J.first) * P.H + J.row_base;
      P.cut[blockIdx.x] = make_int4(static_cast<int>(row0 & 0xffffffff), static_cast<int>(row0 >> 32), J.rows << 16 | (last - range + 1), range);
    }
    if constexpr (K::kWide) latent_piece_wide<K>(P, S, J);
    else latent_piece<K>(P, S, J);
  }
}

// Merges the partial results of the groups that were cut, pieces in their order.  Every workgroup works out which rows there are, and takes its share: four
// rows at a time, a wave each; or, of many pieces, a quarter of one, whose pieces the waves share.  Latency bounds it where rows are few: quarters ask for all there is
// at once (one request, 16 heads, 16000 tokens in 125 pieces: 5 us, whole rows 9).  Where they are not, whole rows have fewer loads to issue (16 requests of 64
// rows in 16 pieces: 52 us with the attention, in quarters 57).
constexpr int kLaMergers = 2048;               // workgroups
constexpr int kLaFew = 8, kLaFewOfMany = 32, kLaManyRows = 256;      // whole rows: up to 8 pieces, or 32 where there are many rows

// What is held by reference m, by another one.
__device__ __forceinline__ float share_at(float m, float now) { return m == -INFINITY ? 0.f : fast_exp2(m - now); }
// Elements `col` .. + E of a row of pieces first, first + step, .. (64 at most): their reference, sum of weights and sum of results.
template <int C, int E, int FLY, typename Part>
__device__ __forceinline__ void merge_pieces(const LatentAttnParams& P, Part part, int pieces, int first, int step, int col, int lane, float& m, float& Z, float (&sum)[E]) {
  typedef float Words __attribute__((ext_vector_type(E)));
  float2 ml = make_float2(-INFINITY, 0.f);                      // a lane for each piece
  if (first + lane * step < pieces) ml = P.ws_ml[part(first + lane * step)];
  float share = 0.f;
  Z = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.f;
  for (int i0 = 0; first + i0 * step < pieces; i0 += FLY) {
    Words x[FLY];
#pragma unroll
    for (int f = 0; f < FLY; ++f) x[f] = *reinterpret_cast<const Words*>(P.ws_o + part(min(first + (i0 + f) * step, pieces - 1)) * C + col);
    __builtin_amdgcn_sched_barrier(0);
    if (i0 == 0) {
      m = wave_max(ml.x);
      share = ml.y * share_at(ml.x, m);
    }
#pragma unroll
    for (int f = 0; f < FLY; ++f) {
      const float by = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(share), i0 + f));      // (0 behind the last piece)
      Z += by;
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] = fmaf(x[f][e], by, sum[e]);
    }
  }
}
template <int E>
__device__ __forceinline__ void write_merged(const LatentAttnParams& P, int64_t row, int C, int col, float m, float Z, const float (&sum)[E]) {
  typedef float Words __attribute__((ext_vector_type(E)));
  typedef __bf16 Halves __attribute__((ext_vector_type(E)));
  const float f = Z == 0.f ? 0.f : 1.f / Z;
  Words y;
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = sum[e] * f;
  if (P.out_f32) *reinterpret_cast<Words*>(static_cast<float*>(P.out) + row * C + col) = y;
  else *reinterpret_cast<Halves*>(static_cast<uint16_t*>(P.out) + row * C + col) = __builtin_convertvector(y, Halves);
  if (P.lse && col == 0) P.lse[row] = (m + log2f(Z)) * static_cast<float>(kLn2);
}

template <int C>
__global__ __launch_bounds__(kLaThreads, 2) void merge_latent_kernel(LatentAttnParams P, int M) {
  constexpr int E = C / kWave, kQuarter = E / kLaWaves;         // elements of a lane: of a row, of a quarter
  __shared__ int upto[kLaRanges], rows_of[kLaWaves];
  __shared__ int4 records[kLaRanges];
  __shared__ float shared_sum[kLaWaves - 1][kQuarter][kWave];
  __shared__ float2 shared_mz[kLaWaves - 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  static_assert(kLaRanges == kLaThreads, "a thread for each record");
  int few;                                                      // whole rows up to that many pieces
  {
    const int4 r = tid < P.ranges ? P.cut[tid] : make_int4(0, 0, 0, 0);
    records[tid] = r;
    const int rows = r.z >> 16, pieces = r.z & 0xffff;
    const double all = wave_scan(static_cast<double>(pieces > 0 ? rows : 0));
    if (lane == 63) rows_of[wave] = static_cast<int>(all);
    __syncthreads();
    few = rows_of[0] + rows_of[1] + rows_of[2] + rows_of[3] >= kLaManyRows ? kLaFewOfMany : kLaFew;
    upto[tid] = static_cast<int>(wave_scan(static_cast<double>(pieces == 0 ? 0 : pieces <= few ? (rows + kLaWaves - 1) / kLaWaves : 4 * rows)));
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += upto[64 * w + 63];
    __syncthreads();
    upto[tid] += before;
    __syncthreads();
  }
  const int total = upto[kLaRanges - 1];
  for (int u = blockIdx.x; u < total; u += gridDim.x) {
    int k = 0;                                                  // the record that unit u is of
#pragma unroll
    for (int w = 0; w < kLaRanges / kWave; ++w) k += __popcll(__builtin_amdgcn_ballot_w64(upto[64 * w + lane] <= u));
    const int4 record = records[k];
    const int pieces = record.z & 0xffff, rows = record.z >> 16, unit = u - (k > 0 ? upto[k - 1] : 0);
    const int64_t row0 = static_cast<int64_t>(record.y) << 32 | static_cast<unsigned>(record.x);
    if (pieces <= few) {
      const int r = unit * kLaWaves + wave;
      if (r >= rows) continue;
      float m, Z, sum[E];
      auto part = [&](int i) { return (static_cast<int64_t>(record.w + i) * 2 + (i == 0 ? 1 : 0)) * M + r; };
      merge_pieces<C, E, 4>(P, part, pieces, 0, 1, E * lane, lane, m, Z, sum);
      write_merged<E>(P, row0 + r, C, E * lane, m, Z, sum);
    } else {
      const int r = unit >> 2, col = (unit & 3) * (C / 4) + kQuarter * lane;
      float m = -INFINITY, Z, sum[kQuarter];
      auto part = [&](int i) { return (static_cast<int64_t>(record.w + i) * 2 + (i == 0 ? 1 : 0)) * M + r; };
      merge_pieces<C, kQuarter, 16>(P, part, pieces, wave, kLaWaves, col, lane, m, Z, sum);
      __syncthreads();                                          // (what was there has been read)
      if (wave > 0) {
#pragma unroll
        for (int e = 0; e < kQuarter; ++e) shared_sum[wave - 1][e][lane] = sum[e];
        if (lane == 0) shared_mz[wave - 1] = make_float2(m, Z);
      }
      __syncthreads();
      if (wave > 0) continue;
      float now = m;
#pragma unroll
      for (int w = 0; w < kLaWaves - 1; ++w) now = fmaxf(now, shared_mz[w].x);
      const float by = share_at(m, now);
      Z *= by;
#pragma unroll
      for (int e = 0; e < kQuarter; ++e) sum[e] *= by;
#pragma unroll
      for (int w = 0; w < kLaWaves - 1; ++w) {
        const float share = share_at(shared_mz[w].x, now);
        Z = fmaf(shared_mz[w].y, share, Z);
#pragma unroll
        for (int e = 0; e < kQuarter; ++e) sum[e] = fmaf(shared_sum[w][e][lane], share, sum[e]);
      }
      write_merged<kQuarter>(P, row0 + r, C, col, now, Z, sum);
    }
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------
LatentAttnPlan make_latent_attn_plan(const LatentArgs& a) {
  LatentAttnPlan p{};
  const int64_t rows = static_cast<int64_t>(a.max_q) * a.H;
  // The more rows, the less there is to do for all of them together, but the fewer workgroups share it.  By the number of groups of 16 rows x 64 tokens if all requests
  // had all their pages (lengths are on the device; a table far wider than they need costs up to twice the time: 4 requests of 512 tokens, 128 heads, 18 us with
  // 33 pages a row, 30 with 2048), 16, 32, 64, 128 rows; us, bf16, C = 512: 36: 15, 17, 21, 27; 1040: 26, 28, 30, 38; 2080: 32, 36, 38, 45; 4160: 47, 37, 52, 55;
  // 8320: 77, 53, 51, 76; 16640: 127, 88, 78, 67; 33280: 256, 139, 138, 111.  With fp32 results and C = 256 they change places at the same numbers.
  const int64_t work = static_cast<int64_t>(a.B) * ((rows + 15) / 16) * ((static_cast<int64_t>(a.max_pages) + 3) / 4);
  p.rows = rows <= 16 || work <= 3000 ? 16 : rows <= 32 || work <= 6000 ? 32 : rows <= 64 || work <= 12000 ? 64 : 128;
  p.groups = static_cast<int>((rows + p.rows - 1) / p.rows);
  const int64_t tiles = static_cast<int64_t>(a.B) * p.groups * static_cast<int64_t>(a.max_pages);
  p.ranges = static_cast<int>(std::min<int64_t>(kLaRanges, (tiles + 7) / 8 * 8));
  return p;
}

static size_t latent_rows(const LatentAttnPlan& p) { return static_cast<size_t>(p.ranges) * 2 * p.rows; }
size_t latent_attn_workspace_bytes(const LatentArgs& a, const LatentAttnPlan& p) {
  return latent_rows(p) * (static_cast<size_t>(a.C) * sizeof(float) + sizeof(float2)) + static_cast<size_t>(p.ranges) * sizeof(int4);
}

template <typename K>
static int launch_latent(const LatentAttnParams& P, const LatentAttnPlan& p, hipStream_t stream) {
  static std::atomic<uint64_t> lds_set{0};
  constexpr size_t lds = sizeof(LatentShared<K>);
  static_assert(lds <= 160 * 1024, "");
  if (lds > 65536 && set_lds_once(attn_latent_kernel<K>, lds, lds_set) != 0) return -6;
  hipLaunchKernelGGL(attn_latent_kernel<K>, dim3(p.ranges), dim3(kLaThreads), lds, stream, P);
  hipLaunchKernelGGL(merge_latent_kernel<K::C>, dim3(static_cast<unsigned>(std::min<int64_t>(kLaMergers, static_cast<int64_t>(p.ranges) * p.rows))), dim3(kLaThreads), 0, stream, P, p.rows);
  return 0;
}
template <int C, int R>
static int launch_latent_rows(const LatentAttnParams& P, const LatentAttnPlan& p, hipStream_t stream) {
  if (P.out_f32) {
    if (p.rows == 16) return launch_latent<LatentNarrow<C, R, 1, 3>>(P, p, stream);
    if (p.rows == 32) return launch_latent<LatentNarrow<C, R, 2, 3>>(P, p, stream);
    if (p.rows == 64) return launch_latent<LatentNarrow<C, R, 4, 3>>(P, p, stream);
    return launch_latent<LatentWide<C, R, 3>>(P, p, stream);
  }
  if (p.rows == 16) return launch_latent<LatentNarrow<C, R, 1, 1>>(P, p, stream);
  if (p.rows == 32) return launch_latent<LatentNarrow<C, R, 2, 1>>(P, p, stream);
  if (p.rows == 64) return launch_latent<LatentNarrow<C, R, 4, 1>>(P, p, stream);
  return launch_latent<LatentWide<C, R, 1>>(P, p, stream);
}

int launch_attn_latent(const LatentArgs& a, const void* q, const void* pool, void* out, float* lse, void* workspace, const LatentAttnPlan& p,
                       hipStream_t stream) {
  LatentAttnParams P{};
  P.q = static_cast<const uint16_t*>(q); P.pool = static_cast<const uint16_t*>(pool);
  P.block_table = a.block_table; P.ctx_len = a.ctx_len; P.q_offsets = a.q_offsets; P.parent = a.parent;
  P.out = out; P.lse = lse;
  P.ws_o = static_cast<float*>(workspace);
  P.ws_ml = reinterpret_cast<float2*>(P.ws_o + latent_rows(p) * a.C);
  P.cut = reinterpret_cast<int4*>(P.ws_ml + latent_rows(p));
  P.B = a.B; P.H = a.H; P.total_q = a.total_q; P.max_q = std::min(a.max_q, kLaMaxNodes); P.max_pages = a.max_pages; P.num_pages = a.num_pages;
  P.ranges = p.ranges; P.c = a.scale * kLog2e; P.out_f32 = a.out_dtype == kF32;
  if (a.C == 512) return a.R == 64 ? launch_latent_rows<512, 64>(P, p, stream) : launch_latent_rows<512, 32>(P, p, stream);
  return a.R == 64 ? launch_latent_rows<256, 64>(P, p, stream) : launch_latent_rows<256, 32>(P, p, stream);
}

}  // namespace specv
