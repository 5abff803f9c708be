// Verify-attention over the cache of latents: the draft queries of each request, of all heads, attend over its committed context and their draft ancestors.
// A cache row is a latent of C elements, key and value at once, and R more that only keys have; all heads read the same rows.
//
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16: 16 tokens x 16 query rows a block.  A lane ends up with 4 consecutive tokens of one row.
//   O^T = V^T P^T the weights of two blocks of 16 tokens are an operand as they are (token 4 g + i of block s is element 4 s + i of lane group g);
//                 V^T, the same bytes as K, is read from LDS by columns.
// Query rows of a request (node x head, consecutive in memory) are taken in groups of up to M, the tokens in tiles of T, which four waves bring to LDS
// and share.  The scores are split over the waves as WR groups of rows x WK groups of tokens, the weights go through LDS, and of the second
// product every wave takes C / 4 columns for all rows: a tile is read WR times from LDS for the scores and once for the results.
//
// Work: the tiles of all requests and groups lie end to end and are cut into ranges of equal cost, one per workgroup, whatever the lengths; every
// workgroup works out from ctx_len and q_offsets which pieces its range holds.  Groups that are cut leave partial results, which a second launch
// merges in their order.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "latent.h"

namespace specv {

constexpr int kLaThreads = 256, kLaWaves = 4;
constexpr int kLaPage = 16;
constexpr int kLaMaxNodes = 128;
constexpr int kLaRanges = 256;                 // workgroups: one per compute unit
constexpr float kLaNoScore = -3.0e38f;         // the reference before the first position: finite, so that -infinity stays ahead of nothing
constexpr float kLaSlack = 8.f;                // a row's reference follows its maximum when that is 2^8 ahead (bf16 weights have the range of fp32)
constexpr int kLaHead = 3;                     // what the start and the end of a group cost, in tiles
constexpr int kLaLeast = 3;                    // tiles of a range at least

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
struct LaRequests {                            // 64 at a time, lane i: request 64 k + i
  int ctx, first, n;
  double upto, sum;                            // cost up to the end of this lane's request, of these 64
};
template <int T>
__device__ __forceinline__ int tiles_of(const LatentAttnParams& P, int ctx, int n) {
  constexpr int kPages = T / kLaPage;
  return n > 0 ? min(static_cast<int>((static_cast<unsigned>(ctx) + n + T - 1) / T), static_cast<int>((static_cast<unsigned>(P.max_pages) + kPages - 1) / kPages)) : 0;
}
template <int M, int T>
__device__ __forceinline__ LaRequests load_requests(const LatentAttnParams& P, int k, int lane) {
  LaRequests r;
  const int b = 64 * k + lane;
  r.ctx = r.first = r.n = 0;
  if (b < P.B) {
    r.ctx = min(max(P.ctx_len[b], 0), 0x7fffff00);              // (the end of the drafts still fits)
    r.first = P.q_offsets[b];
    r.n = r.first < 0 ? 0 : max(min(min(P.q_offsets[b + 1], P.total_q) - r.first, P.max_q), 0);
  }
  const int groups = (r.n * P.H + M - 1) / M;
  r.upto = wave_scan(static_cast<double>(groups) * (kLaHead + tiles_of<T>(P, r.ctx, r.n)));
  r.sum = lane_f64(r.upto, 63);
  return r;
}
struct LaCut {
  int used;
  double each, total;
};
__device__ __forceinline__ LaCut cut_ranges(int most, double total) {
  LaCut c;
  c.total = total;
  c.used = __builtin_amdgcn_readfirstlane(static_cast<int>(fmin(fmax(total / kLaLeast, 1.0), static_cast<double>(most))));
  c.each = total / c.used;
  return c;
}
__device__ __forceinline__ double range_start(const LaCut& c, int s) { return s >= c.used ? c.total : floor(s * c.each); }
__device__ __forceinline__ int range_of(const LaCut& c, double at) {
  int s = min(max(static_cast<int>(at / c.each) - 1, 0), c.used - 1);
  while (s + 1 < c.used && range_start(c, s + 1) <= at) ++s;
  return s;
}

template <int C_, int R_, int NB_, int WR_, int KB_, int TERMS_>
struct LatentConfig {
  static constexpr int C = C_, R = R_, NB = NB_, WR = WR_, WK = kLaWaves / WR_, KB = KB_, TERMS = TERMS_;
  static constexpr int W = C + R;
  static constexpr int M = 16 * NB * WR, T = 16 * KB * WK;
  static constexpr int kUnits = (W / 8 + 7) / 8 * 8;            // 16-byte units of a row in LDS
  static constexpr int kRow = 16 * kUnits, kTile = T * kRow;
  static constexpr int kPages = T / kLaPage;
  static constexpr int RB = M / 16, CB = C / 4 / 16;            // 16-row blocks; 16-column blocks of a wave
  static constexpr int kSteps = W / 32;
  static constexpr int kLoads = kTile / kLaWaves / 1024;        // of a wave for a tile
  static constexpr int kOffsets = 8 * kRow / 1024;              // loads that bring 8 rows
  static constexpr int kWeights = T / 32 * RB * 1024;           // bytes of a term of a tile's weights
  static constexpr int kSmall = TERMS * kWeights + kLaMaxNodes * 20 + 64 + 4 * M * (2 * WK + 2);
  static constexpr int kStages = std::min(4, (160 * 1024 - kSmall) / kTile);
  static_assert(kStages >= 2 && kRow % 256 == 128, "");
};

template <typename K>
struct LatentShared {
  __align__(1024) unsigned char ring[K::kStages][K::kTile];
  __align__(16) unsigned char p[K::TERMS][K::kWeights];
  unsigned long long anc[kLaMaxNodes][2];
  int parent[kLaMaxNodes];
  int node[K::M];
  float top[K::WK][K::M], sum[K::WK][K::M], by[K::M];
  unsigned ahead[kLaWaves];
};

struct LatentPiece {
  int b, first, n, ctx, t0, t1, rows;
  int row_base;
  bool whole;
  int64_t part;               // first row of its partial result
};

template <typename K>
__device__ __forceinline__ void latent_piece(const LatentAttnParams& P, LatentShared<K>& S, const LatentPiece& J) {
  constexpr int W = K::W, T = K::T, M = K::M, NB = K::NB, KB = K::KB, WK = K::WK, RB = K::RB, CB = K::CB, kPages = K::kPages, NS = K::kStages;
  const int tid = static_cast<int>(threadIdx.x) + opaque_zero(), lane = tid & 63;
  __builtin_assume(tid >= 0 && tid < kLaThreads);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rn = lane & 15, g = lane >> 4;
  const int wr = wave / WK, wk = wave % WK;                     // of the scores: this wave's rows 16 NB wr .., tokens 16 KB wk .. of a tile
  const int L = J.ctx + J.n;

  // ---- a tile's loads ----
  // Row r of a tile, 16-byte unit u lies at u ^ f(r), f = 4 (r / 2 % 2) + 2 (r / 4 % 2): 8 lanes that read a unit of 8 rows, and 16 lanes that read 4 rows
  // by columns, take 128 bytes from as many banks (rows are 128 bytes apart modulo the banks' 256).  Units past the row's last repeat one.
  unsigned off[K::kOffsets];
#pragma unroll
  for (int j = 0; j < K::kOffsets; ++j) {
    const int u = 64 * j + lane, r = u / K::kUnits, p = u % K::kUnits;
    int unit = p ^ (4 * ((r >> 1) & 1) + 2 * ((r >> 2) & 1));
    if constexpr (K::kUnits * 8 != W) unit = min(unit, W / 8 - 1);
    off[j] = r * (W * 2) + unit * 16;
  }
  constexpr int64_t kPageBytes = kLaPage * W * 2;
  const const_i32* bt = (const const_i32*)(P.block_table + static_cast<int64_t>(J.b) * P.max_pages);
  const int last_page = min((L - 1) / kLaPage, P.max_pages - 1);
  const unsigned ring = lds_address(&S.ring[0][0]);
  const int my_page = kPages == 4 ? wave : wave >> 1;           // of a tile's pages: the one that this wave brings (half of)
  int ids[kPages], my_id = 0;
  auto fetch_ids = [&](int t) __attribute__((always_inline)) {
    if (t < J.t1) {
#pragma unroll
      for (int i = 0; i < kPages; ++i) {
        const int lp = kPages * t + i, id = bt[min(lp, last_page)];
        ids[i] = id >= 0 && id < P.num_pages && lp < P.max_pages ? id : -1;
      }
      my_id = bt[min(kPages * t + my_page, last_page)];
      my_id = my_id >= 0 && my_id < P.num_pages ? my_id : 0;
    }
  };
  auto bad_pages = [&]() __attribute__((always_inline)) {
    unsigned bad = 0u;
#pragma unroll
    for (int i = 0; i < kPages; ++i) bad |= ids[i] < 0 ? 1u << i : 0u;
    return bad;
  };
  // (a page that is none of the pool's: page 0 in its place)
  auto issue = [&](int slot) __attribute__((always_inline)) {
    const unsigned to = ring + slot * K::kTile + wave * (K::kTile / kLaWaves);
    const unsigned char* page = reinterpret_cast<const unsigned char*>(P.pool) + __builtin_amdgcn_readfirstlane(my_id) * kPageBytes + (kPages == 4 ? 0 : (wave & 1) * 8 * W * 2);
#pragma unroll
    for (int j = 0; j < K::kLoads; ++j) load_to_lds(page + j / K::kOffsets * 8 * W * 2, off[j % K::kOffsets], to + 1024 * j, 0);
  };
  unsigned long long bad = 0ull;                                // pages that are none: kPages bits a tile, the present one's lowest

  // ---- the queries' operands: rows past the last repeat it ----
  lbf16x8 qf[NB][K::kSteps];
  {
    const uint16_t* q = P.q + (static_cast<int64_t>(J.first) * P.H + J.row_base) * W + 8 * g;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const uint16_t* row = q + static_cast<int64_t>(min(16 * (NB * wr + nb) + rn, J.rows - 1)) * W;
#pragma unroll
      for (int s = 0; s < K::kSteps; ++s) qf[nb][s] = operand(*reinterpret_cast<const raw4*>(row + 32 * s));
    }
  }
  const bool touches_drafts = J.t1 * static_cast<int64_t>(T) > J.ctx;
  int parent = -1;
  if (touches_drafts && P.parent && tid < J.n) parent = P.parent[J.first + tid];
  lds_sync();                                                   // the LDS of the piece before is free
  fetch_ids(J.t0);
#pragma unroll
  for (int i = 0; i < NS - 1; ++i) {
    if (J.t0 + i < J.t1) {
      bad |= static_cast<unsigned long long>(bad_pages()) << (kPages * i);
      issue(i);
      fetch_ids(J.t0 + i + 1);
    }
  }
  if (touches_drafts) {
    if (tid < kLaMaxNodes) S.parent[tid] = parent;
    if (tid < M) S.node[tid] = (J.row_base + min(tid, J.rows - 1)) / P.H;
    lds_sync();
    if (tid < kLaMaxNodes) {
      unsigned long long w[2] = {0ull, 0ull};
      if (tid < J.n) {
        if (P.parent) {
          int a = tid;
          for (int k = 0; k < kLaMaxNodes && a >= 0; ++k) {
            if (a < 64) w[0] |= 1ull << a; else w[1] |= 1ull << (a - 64);
            const int p = S.parent[a];
            a = (p >= a || p < 0) ? -1 : p;                     // (a malformed entry is a root)
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

  // Operand reads: K, token 16 (KB wk + kb) + rn, unit 4 s + g; V by columns, token 4 g + rn / 4 (and 16 more), unit 4 (cb / 2) + rn % 4, half cb % 2: column
  // 32 p + 8 g + 4 s + i of the wave's is row 4 g + i of block 2 p + s, so that a lane ends up with 8 consecutive ones
  const int kf = 4 * ((rn >> 1) & 1) + 2 * ((rn >> 2) & 1);
  const unsigned k_at = (16 * KB * wk + rn) * K::kRow + (g ^ kf) * 16;              // even steps; odd ones at ^ 64; 128 more every two
  const int vt = 4 * g + (rn >> 2), vf = 4 * ((vt >> 1) & 1) + 2 * ((vt >> 2) & 1);
  const unsigned v_at = vt * K::kRow + ((rn & 3) ^ vf) * 16 + wave * (K::C / 4 * 2);   // even pairs of blocks; odd ones at ^ 64; 128 more every two
  const unsigned p_at = lds_address(&S.p[0][0]);

  float ref[NB], sum[NB];
  lf32x4 o[CB][RB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    ref[nb] = kLaNoScore;
    sum[nb] = 0.f;
  }
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) o[cb][rb] = lf32x4{0.f, 0.f, 0.f, 0.f};

  int slot = 0;
  for (int t = J.t0; t < J.t1; ++t) {
    // ---- the tile is here, and all waves are done with the one before ----
    const int more = J.t1 - 1 - t;
    if constexpr (NS >= 4) {
      if (more >= 2) wait_loads<2 * K::kLoads>();
    }
    if constexpr (NS >= 3) {
      if (more == 1 || (NS == 3 && more > 1)) wait_loads<K::kLoads>();
    }
    if (NS == 2 || more == 0) wait_loads<0>();
    lds_sync();
    if (t + NS - 1 < J.t1) {
      bad |= static_cast<unsigned long long>(bad_pages()) << (kPages * (NS - 1));
      issue(slot == 0 ? NS - 1 : slot - 1);
      fetch_ids(t + NS);
    }
    const unsigned tile = ring + slot * K::kTile;

    // ---- scores ----
    lf32x4 s[KB][NB];
#pragma unroll
    for (int step = 0; step < K::kSteps; ++step) {
      lbf16x8 k[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) k[kb] = operand(read_lds16(((tile + k_at) ^ (64 * (step & 1))) + 128 * (step >> 1) + kb * 16 * K::kRow));
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[kb][nb] = multiply(k[kb], qf[nb][step], step == 0 ? lf32x4{0.f, 0.f, 0.f, 0.f} : s[kb][nb]);
      if (step % 4 == 3) __builtin_amdgcn_sched_barrier(0);     // (else all of K is read first, into registers there are none of)
    }

    // ---- masks: only where the tile reaches the drafts, or a page is none ----
    const bool special = (t + 1) * static_cast<int64_t>(T) > J.ctx || (bad & ((1u << kPages) - 1u)) != 0ull;
    if (special) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const int page = KB * wk + kb;
        const int64_t past = static_cast<int64_t>(t) * T + 16 * page - J.ctx;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          uint32_t seen = 0xffffu;
          if (past > -16) {
            const int node = S.node[16 * (NB * wr + nb) + rn];
            seen = page_mask(S.anc[node][0], S.anc[node][1], static_cast<int>(past));
          }
          seen = (bad >> page) & 1ull ? 0u : seen >> (4 * g);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[kb][nb][i] = (seen >> i) & 1u ? s[kb][nb][i] : -INFINITY;
        }
      }
    }

    // ---- weights ----
    float top[NB], z[NB];
    bool ahead = false;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      top[nb] = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) top[nb] = max3(top[nb], max3(s[kb][nb][0], s[kb][nb][1], s[kb][nb][2]), s[kb][nb][3]);
      top[nb] *= P.c;
      ahead |= top[nb] > ref[nb] + kLaSlack;
    }
    auto weigh = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        z[nb] = 0.f;
        uint32_t w[K::TERMS][KB][2];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float p0 = fast_exp2(fmaf(s[kb][nb][2 * i], P.c, -ref[nb])), p1 = fast_exp2(fmaf(s[kb][nb][2 * i + 1], P.c, -ref[nb]));
            z[nb] += p0 + p1;
            float r0 = p0, r1 = p1;
#pragma unroll
            for (int term = 0; term < K::TERMS; ++term) {
              w[term][kb][i] = pack2(r0, r1);
              r0 -= bf16_lo(w[term][kb][i]);
              r1 -= bf16_hi(w[term][kb][i]);
            }
          }
        // blocks of 16 tokens 2 m and 2 m + 1 are the halves of a lane's 16 bytes
#pragma unroll
        for (int term = 0; term < K::TERMS; ++term) {
          const unsigned at = p_at + term * K::kWeights + 16 * lane + (NB * wr + nb) * 1024;
          if constexpr (KB == 1) {
            *lds_pointer<unsigned long long>(at + (wk >> 1) * RB * 1024 + 8 * (wk & 1)) = static_cast<unsigned long long>(w[term][0][1]) << 32 | w[term][0][0];
          } else {
#pragma unroll
            for (int m = 0; m < KB / 2; ++m)
              *lds_pointer<raw4>(at + (wk * (KB / 2) + m) * RB * 1024) = raw4{w[term][2 * m][0], w[term][2 * m][1], w[term][2 * m + 1][0], w[term][2 * m + 1][1]};
          }
        }
      }
    };
    weigh();
    const unsigned flag = any_lane(ahead) ? 1u : 0u;
    if (lane == 0) S.ahead[wave] = flag;
    lds_sync();
    const raw4 flags = *reinterpret_cast<const raw4*>(S.ahead);
    if (__builtin_amdgcn_readfirstlane(flags[0] | flags[1] | flags[2] | flags[3])) {
      // ---- a row's reference follows its maximum where that has come far ahead (in all waves, or in none) ----
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float m = groups_max(top[nb]);
        if (lane < 16) S.top[wk][16 * (NB * wr + nb) + lane] = m;
      }
      lds_sync();
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int row = 16 * (NB * wr + nb) + rn;
        float now = S.top[0][row];
#pragma unroll
        for (int k = 1; k < WK; ++k) now = fmaxf(now, S.top[k][row]);
        now = now > ref[nb] + kLaSlack ? now : ref[nb];         // (each row by itself: its result has the same bits whatever the others are)
        const float by = fast_exp2(ref[nb] - now);
        ref[nb] = now;
        sum[nb] *= by;
        if (wk == 0 && lane < 16) S.by[row] = by;
      }
      weigh();
      lds_sync();
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float by = S.by[16 * rb + rn];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) o[cb][rb] *= by;
      }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) sum[nb] += z[nb];

    // A weight of zero times what is not finite would be NaN: where rows differ in what they see, such values are taken out of V.  (A row that
    // sees one has met it in its scores.)
    if (special) {
      for (int at = 16 * tid; at < K::kTile; at += 16 * kLaThreads) {
        raw4 w = read_lds16(tile + at);
        bool any = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool l = (w[i] & 0x7f80u) == 0x7f80u, h = (w[i] & 0x7f800000u) == 0x7f800000u;
          any |= l | h;
          w[i] = (l ? 0u : w[i] & 0xffffu) | (h ? 0u : w[i] & 0xffff0000u);
        }
        if (any) *lds_pointer<raw4>(tile + at) = w;
      }
      lds_sync();
    }

    // ---- O^T += V^T P^T ----
#pragma unroll
    for (int m = 0; m < T / 32; ++m) {
      lbf16x8 p[K::TERMS][RB];
#pragma unroll
      for (int term = 0; term < K::TERMS; ++term)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) p[term][rb] = operand(read_lds16(p_at + term * K::kWeights + (m * RB + rb) * 1024 + 16 * lane));
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const unsigned at = ((tile + v_at) ^ (64 * ((cb >> 1) & 1))) + 128 * (cb >> 2) + 8 * (cb & 1) + m * 32 * K::kRow;
        const lbf16x8 v = join(read_columns(at), read_columns(at + 16 * K::kRow));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
          for (int term = 0; term < K::TERMS; ++term) o[cb][rb] = multiply(v, p[term][rb], o[cb][rb]);
        }
        if (cb % 2 == 1) __builtin_amdgcn_sched_barrier(0);
      }
    }
    bad >>= kPages;
    slot = slot + 1 == NS ? 0 : slot + 1;
  }

  // ---- results ----
  lds_sync();                                                   // (S.by has been read)
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const float z = groups_sum(sum[nb]);
    if (lane < 16) {
      S.sum[wk][16 * (NB * wr + nb) + lane] = z;
      if (wk == 0) S.by[16 * (NB * wr + nb) + lane] = ref[nb];
    }
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
    const float z = row_sum(tid), m = z == 0.f ? -INFINITY : S.by[tid];
    if (!J.whole) P.ws_ml[J.part + tid] = make_float2(m, z);
    else if (P.lse) P.lse[row0 + tid] = (m + log2f(z)) * static_cast<float>(kLn2);
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = 16 * rb + rn;
    if (row >= J.rows) continue;
    const float z = row_sum(row), f = z == 0.f ? 0.f : 1.f / z;
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

template <typename K>
__global__ __launch_bounds__(kLaThreads, 1) void attn_latent_kernel(LatentAttnParams P) {
  extern __shared__ __align__(1024) unsigned char smem[];
  auto& S = *reinterpret_cast<LatentShared<K>*>(smem);
  constexpr int M = K::M, T = K::T;
  const int lane = threadIdx.x & 63;
  const int batches = (P.B + 63) / 64;
  double total = 0.0;
  LaRequests r;
  for (int k = batches - 1; k >= 0; --k) {                      // (down: the first 64 requests stay in registers)
    r = load_requests<M, T>(P, k, lane);
    total += r.sum;
  }
  const LaCut cut = cut_ranges(P.ranges, total);
  // Workgroups go to the 8 XCDs in turn: renumbered so that neighbouring ranges, which may hold groups of rows of one request, share an L2
  const int each = (cut.used + 7) >> 3, range = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  int4 record = make_int4(0, 0, 0, 0);
  if (any_lane(total > 0.0) && static_cast<int>(blockIdx.x >> 3) < each && range < cut.used) {
    const double from = range_start(cut, range), end = range_start(cut, range + 1);
    double base = 0.0;                                          // cost before these 64 requests
    double at = from;
    for (int k = 0; any_lane(at < end);) {                      // (uniform, as the compiler has to know)
      const unsigned long long later = __builtin_amdgcn_ballot_w64(base + r.upto > at);
      if (later == 0ull) {
        base += r.sum;
        if (++k >= batches) break;
        r = load_requests<M, T>(P, k, lane);
        continue;
      }
      const int i = __ffsll(later) - 1;
      LatentPiece J;
      J.b = 64 * k + i;
      J.ctx = __builtin_amdgcn_readlane(r.ctx, i);
      J.first = __builtin_amdgcn_readlane(r.first, i);
      J.n = __builtin_amdgcn_readlane(r.n, i);
      const int rows = J.n * P.H, groups = (rows + M - 1) / M, tiles = tiles_of<T>(P, J.ctx, J.n);
      const double behind = base + lane_f64(r.upto, i);
      double start = behind - static_cast<double>(groups) * (kLaHead + tiles);
      for (int grp = 0; grp < groups && any_lane(start < end); ++grp, start += kLaHead + tiles) {
        // tile k is at start + kLaHead + k and belongs to the range that this is in
        J.t0 = static_cast<int>(fmin(fmax(from - start - kLaHead, 0.0), static_cast<double>(tiles)));
        J.t1 = static_cast<int>(fmin(fmax(end - start - kLaHead, 0.0), static_cast<double>(tiles)));
        J.t0 = __builtin_amdgcn_readfirstlane(J.t0);
        J.t1 = __builtin_amdgcn_readfirstlane(J.t1);
        if (J.t0 >= J.t1) continue;
        J.row_base = M * grp;
        J.rows = min(rows - J.row_base, M);
        J.whole = J.t0 == 0 && J.t1 == tiles;
        J.part = (static_cast<int64_t>(range) * 2 + (J.t0 == 0 ? 1 : 0)) * M;
        latent_piece<K>(P, S, J);
        if (!J.whole && J.t0 == 0) {
          const int last = range_of(cut, start + kLaHead + tiles - 1);
          const int64_t row0 = static_cast<int64_t>(J.first) * P.H + J.row_base;
          record = make_int4(static_cast<int>(row0 & 0xffffffff), static_cast<int>(row0 >> 32), J.rows << 16 | (last - range + 1), range);
        }
      }
      at = behind;
    }
  }
  if (P.cut && threadIdx.x == 0) P.cut[blockIdx.x] = record;
}

// Merges the partial results of the groups that were cut: a wave takes a row.
template <int C>
__global__ __launch_bounds__(kLaThreads) void merge_latent_kernel(LatentAttnParams P, int M) {
  const int4 record = P.cut[blockIdx.x];
  const int pieces = record.z & 0xffff, rows = record.z >> 16;
  const int lane = threadIdx.x & 63, r = __builtin_amdgcn_readfirstlane(blockIdx.y * kLaWaves + (threadIdx.x >> 6));
  if (r >= rows || pieces == 0) return;
  const int64_t row = (static_cast<int64_t>(record.y) << 32 | static_cast<unsigned>(record.x)) + r;
  auto part = [&](int i) { return (static_cast<int64_t>(record.w + i) * 2 + (i == 0 ? 1 : 0)) * M + r; };
  float m = -INFINITY;
  for (int i = 0; i < pieces; ++i) m = fmaxf(m, P.ws_ml[part(i)].x);
  constexpr int E = C / kWave;
  float sum[E], Z = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.f;
  for (int i = 0; i < pieces; ++i) {
    const float2 ml = P.ws_ml[part(i)];
    const float share = ml.x == -INFINITY ? 0.f : ml.y * fast_exp2(ml.x - m);
    Z += share;
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const float4 x = *reinterpret_cast<const float4*>(P.ws_o + part(i) * C + e * kWave + 4 * lane);
      sum[e] += x.x * share; sum[e + 1] += x.y * share; sum[e + 2] += x.z * share; sum[e + 3] += x.w * share;
    }
  }
  const float f = Z == 0.f ? 0.f : 1.f / Z;
#pragma unroll
  for (int e = 0; e < E; e += 4) {
    const lf32x4 x = {sum[e] * f, sum[e + 1] * f, sum[e + 2] * f, sum[e + 3] * f};
    const int64_t to = row * C + e * kWave + 4 * lane;
    if (P.out_f32) *reinterpret_cast<float4*>(static_cast<float*>(P.out) + to) = make_float4(x[0], x[1], x[2], x[3]);
    else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out) + to) = pack4(x);
  }
  if (P.lse && lane == 0) P.lse[row] = (m + log2f(Z)) * static_cast<float>(kLn2);
}

// ---- host -----------------------------------------------------------------------------------------------------------
LatentAttnPlan make_latent_attn_plan(const LatentArgs& a) {
  LatentAttnPlan p{};
  const int64_t rows = static_cast<int64_t>(a.max_q) * a.H;
  const int most = a.out_dtype == kF32 ? 64 : 128;
  p.rows = 16;
  while (p.rows < most && p.rows < rows) p.rows *= 2;
  p.groups = static_cast<int>((rows + p.rows - 1) / p.rows);
  const int64_t tiles = static_cast<int64_t>(a.B) * p.groups * (static_cast<int64_t>(a.max_pages) + kLaHead);
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
  hipLaunchKernelGGL(merge_latent_kernel<K::C>, dim3(p.ranges, (p.rows + kLaWaves - 1) / kLaWaves), dim3(kLaThreads), 0, stream, P, p.rows);
  return 0;
}
template <int C, int R>
static int launch_latent_rows(const LatentAttnParams& P, const LatentAttnPlan& p, hipStream_t stream) {
  if (P.out_f32) {
    switch (p.rows) {
      case 16: return launch_latent<LatentConfig<C, R, 1, 1, 1, 3>>(P, p, stream);
      case 32: return launch_latent<LatentConfig<C, R, 2, 1, 1, 3>>(P, p, stream);
      default: return launch_latent<LatentConfig<C, R, 2, 2, 1, 3>>(P, p, stream);
    }
  }
  switch (p.rows) {
    case 16: return launch_latent<LatentConfig<C, R, 1, 1, 1, 1>>(P, p, stream);
    case 32: return launch_latent<LatentConfig<C, R, 2, 1, 1, 1>>(P, p, stream);
    case 64: return launch_latent<LatentConfig<C, R, 2, 2, 1, 1>>(P, p, stream);
    default: return launch_latent<LatentConfig<C, R, 2, 4, 2, 1>>(P, p, stream);
  }
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
