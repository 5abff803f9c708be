// Verify-attention over the 8-bit paged cache (quant.h): the draft queries of each request attend over its committed context and
// their draft ancestors, keys and values read as e4m3 with a scale per (page, KV head).
//
// A wave takes 64 tokens (4 pages) at a time, straight from memory into registers: pages are laid out so that a lane's 16 bytes
// are matrix operands as they lie, and no LDS, transposition or barrier stands between memory and the matrix cores.
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16, tokens as M.  Row 4 g + i of sub-tile t is token 4 t + i of page g, so that lane group
//                 g (lanes 16 g .. 16 g + 15, one query row each) ends up with all 16 tokens of page g: its scale is one register, and
//   O^T = V^T P^T takes those 16 weights as its operand without any exchange between lanes.
// e4m3 is exact in bf16 and fp16.  K's scale rides on the softmax factor; V is fed in fp16, its page's scale on the conversion, relative to the
// largest scale so far.  A weight is one fp16 term (2^-12 off, a sixteenth of the rounding of a bf16 result), or two for fp32 results.
//
// Work: per KV head (and group of query rows) the 64-token units of all requests lie end to end and are cut into equal ranges,
// one per workgroup, whatever the lengths; every workgroup works out from ctx_len and q_offsets which requests its range
// meets.  A range that ends inside a request leaves an unnormalised partial result, attn_quant_combine_kernel merges them.  The waves
// of a workgroup take units in turn and merge through LDS.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "quant.h"

namespace specv {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 qbf16x8;
typedef float qf32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 qbf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 qf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 qf16x2 __attribute__((ext_vector_type(2)));

constexpr int kQaThreads = 256;
constexpr int kQaWaves = 4;
constexpr int kUnit = 32;                     // tokens a wave takes at a time
constexpr int kQaMaxNodes = 128;
constexpr float kNoScore = -3.0e38f;          // the reference before the first position: finite, so that -infinity stays ahead of nothing
constexpr int kQaWaveBlocks = 3;              // most 16-row blocks that a wave multiplies a unit with: what 256 registers hold
constexpr int kQaBlocks = kQaWaves * kQaWaveBlocks;      // ... of a workgroup
constexpr int kWeightBias = 6;                // weights are fed as fp16(2^6 p): normal down to p = 2^-20, and
constexpr float kSlack = 8.f;                 // the reference of a row's softmax follows its maximum when that is 2^8 ahead: below 2^14 then
constexpr float kLeastV = 3.0517578125e-5f;   // 2^-15: what V may be scaled by and still be exact in fp16

struct QuantAttnParams {
  const uint16_t* q;
  const unsigned char* k_pool;
  const unsigned char* v_pool;
  const float* k_scale;
  const float* v_scale;
  const int32_t* block_table;
  const int32_t* ctx_len;
  const int32_t* q_offsets;
  const int32_t* parent;
  void* out;
  float* lse;
  float* ws_o;        // [KV heads * groups][ranges][2][rows][D] unnormalised partial results
  float2* ws_ml;      // ... [rows] (maximum in log2 units, sum)
  int B, Hq, Hkv, G, total_q, max_pages, num_pages;
  int ranges;         // per KV head and group of rows, at most
  int least_units;    // ... a range has at least this many units where there are enough
  int blocks;         // 16-row blocks of a group of rows
  float c;            // scale * log2(e)
  int out_f32;
};

__device__ __forceinline__ int wave_scan_i32(int x, int lane) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int y = __shfl_up(x, d);
    x += lane >= d ? y : 0;
  }
  return x;
}

// The units of all requests, 64 requests at a time: lane i holds request 64 k + i.
struct Requests {
  int ctx, first, n, units, upto;               // of this lane's request; upto: units up to its end, within these 64
  int sum;                                      // units of these 64
};
__device__ __forceinline__ Requests load_requests(const QuantAttnParams& P, int k, int lane) {
  Requests r;
  const int b = 64 * k + lane;
  r.ctx = r.first = r.n = 0;
  if (b < P.B) {
    r.ctx = max(P.ctx_len[b], 0);
    r.first = P.q_offsets[b];
    r.n = max(min(min(P.q_offsets[b + 1], P.total_q) - r.first, kQaMaxNodes), 0);
  }
  r.units = r.n > 0 ? static_cast<int>((static_cast<unsigned>(r.ctx) + r.n + kUnit - 1) / kUnit) : 0;
  r.upto = wave_scan_i32(r.units, lane);
  r.sum = __builtin_amdgcn_readlane(r.upto, 63);
  return r;
}
// Ranges that are used: range s holds the units [s U / ranges, (s + 1) U / ranges).
__device__ __forceinline__ int used_ranges(const QuantAttnParams& P, int64_t units) {
  const int64_t want = units / P.least_units;
  return static_cast<int>(want < 1 ? 1 : (want < P.ranges ? want : P.ranges));
}
// The range that unit u is in.
__device__ __forceinline__ int range_of(int64_t u, int64_t units, int used) {
  return static_cast<int>(((u + 1) * used + units - 1) / units) - 1;
}


// __any as the compiler knows it to be uniform: a branch on it stays a scalar one (around the other kind it keeps a second copy of every
// register that the branch changes).
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

// Eight e4m3 bytes as an operand of eight bf16, or, times a power of two, of eight fp16.
__device__ __forceinline__ qbf16x8 operand_bf16(uint32_t lo, uint32_t hi) {
  const qbf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
  const qbf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
  const raw4 w = {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
  return __builtin_bit_cast(qbf16x8, w);
}
__device__ __forceinline__ qf16x8 operand_f16(uint32_t lo, uint32_t hi, float scale) {
  const qf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true);
  const qf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true);
  const raw4 w = {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
  return __builtin_bit_cast(qf16x8, w);
}

// Which of the 16 tokens of a page a node sees, the page starting `past` tokens behind the context (negative: before its end).
__device__ __forceinline__ uint32_t page_mask(unsigned long long lo, unsigned long long hi, int past) {
  if (past <= -16) return 0xffffu;
  if (past < 0) return (static_cast<uint32_t>(lo << -past) | ((1u << -past) - 1u)) & 0xffffu;
  if (past >= 128) return 0u;
  if (past >= 64) return static_cast<uint32_t>(hi >> (past - 64)) & 0xffffu;
  return static_cast<uint32_t>(past == 0 ? lo : (lo >> past) | (hi << (64 - past))) & 0xffffu;
}
// Bit 7 of the bytes that are NaN.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// 4 bits -> byte mask of a word
__device__ __forceinline__ uint32_t spread4(uint32_t bits) {
  return ((bits & 1u) * 0xffu) | ((bits >> 1 & 1u) * 0xff00u) | ((bits >> 2 & 1u) * 0xff0000u) | ((bits >> 3 & 1u) * 0xff000000u);
}

template <int D, int MAXB>
struct QuantAttnShared {
  static constexpr int kStride = D + 4;                        // floats; padded row of the merge
  unsigned long long anc[kQaMaxNodes][2];
  int parent[kQaMaxNodes];
  int nans;                                                    // a draft's value is NaN
  float m[kQaWaves][16 * MAXB], l[kQaWaves][16 * MAXB];
  union {
    __align__(16) float o[kQaWaves][16][kStride];              // the merge, when the queries are done with
    __align__(16) raw4 q[kQaWaves * MAXB * 2 * (D / 64)][kWave];     // query operands: [block, step][lane]
  };
};

// One piece of a request: units [t0, t1) of it, for the query rows [row_base, row_base + rows) of a KV head, NB 16-row blocks per wave.
struct QuantPiece {
  int b, first, n, ctx, kvh, t0, t1, row_base, rows;
  bool whole;                 // the piece is the whole request: write the result
  int64_t part;               // else: first row of its partial result
};

// Dimensions d0 .. d0 + 3 of a row's result are NaN where a value is that the row sees, among the units that reach the drafts (of the others
// every row sees every token, and the products are NaN by themselves).
template <int D, typename Shared>
__device__ __forceinline__ void put_back_nans(const QuantAttnParams& P, const Shared& S, const QuantPiece& J, int row, int d0, float4& o) {
  const int node = (J.row_base + row) / P.G;
  const int end = min(J.t1 * kUnit, J.ctx + J.n);
  for (int tok = max(J.t0 * kUnit, J.ctx & ~(kUnit - 1)); tok < end; ++tok) {
    const int j = tok - J.ctx, lp = tok / kQuantPage;
    if (j >= 0 && !((S.anc[node][j >> 6] >> (j & 63)) & 1ull)) continue;
    const int id = lp < P.max_pages ? P.block_table[static_cast<int64_t>(J.b) * P.max_pages + lp] : -1;
    if (id < 0 || id >= P.num_pages) continue;
    const unsigned char* v = P.v_pool + (static_cast<int64_t>(id) * P.Hkv + J.kvh) * (kQuantPage * D) + d0 * kQuantPage + tok % kQuantPage;
    const float nan = __builtin_nanf("");
    if ((v[0] & 0x7f) == 0x7f) o.x = nan;
    if ((v[kQuantPage] & 0x7f) == 0x7f) o.y = nan;
    if ((v[2 * kQuantPage] & 0x7f) == 0x7f) o.z = nan;
    if ((v[3 * kQuantPage] & 0x7f) == 0x7f) o.w = nan;
  }
}

// SANITIZE: NaN among the drafts' values are taken out of the products (where a row does not see a draft its weight is zero, and zero times
// NaN would be NaN) and put back into the results of the rows that see them.  Without, a piece that meets one writes nothing and
// says so in S.nans.
template <int D, int NB, int TERMS, bool SANITIZE, typename Shared>
__device__ __forceinline__ void quant_piece(const QuantAttnParams& P, Shared& S, const QuantPiece& J) {
  constexpr int kH = D / 64;                                   // K: 16-byte chunks of a lane per token
  constexpr int kDT = D / 16;                                  // 16-dimension tiles of the output
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rn = lane & 15, g = lane >> 4;                     // query row of the block (matrix column), lane group
  const int L = J.ctx + J.n;
  const int total_blocks = (J.rows + 15) / 16;
  const int kinds = (total_blocks + NB - 1) / NB > 2 ? 4 : (total_blocks + NB - 1) / NB;   // groups of waves with rows of their own: 1, 2 or 4
  const int slices = kQaWaves / kinds, kind = wave % kinds, slice = wave / kinds;
  const bool touches_drafts = J.t1 * kUnit > J.ctx;

  __syncthreads();                                              // the LDS of the piece before is free
  if (!SANITIZE && tid == 0) S.nans = 0;
  if (touches_drafts) {
    if (P.parent && tid < J.n) S.parent[tid] = P.parent[J.first + tid];
    __syncthreads();
    if (tid < kQaMaxNodes) {
      unsigned long long w[2] = {0ull, 0ull};
      if (tid < J.n) {
        if (P.parent) {
          int a = tid;
          for (int k = 0; k < kQaMaxNodes && a >= 0; ++k) {
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
    __syncthreads();
  }

  auto node_of = [&](int qi) __attribute__((always_inline)) { return (J.row_base + min(16 * (kind * NB + qi) + rn, J.rows - 1)) / P.G; };
  const int64_t page_bytes = static_cast<int64_t>(P.Hkv) * kQuantPage * D;
  const unsigned char* k_lane = P.k_pool + static_cast<int64_t>(J.kvh) * kQuantPage * D + g * 256 + (8 * ((rn >> 2) & 1) + (rn & 3)) * 16;
  const unsigned char* v_lane = P.v_pool + static_cast<int64_t>(J.kvh) * kQuantPage * D + rn * 16 + 8 * (g & 1);
  const int32_t* bt = P.block_table + static_cast<int64_t>(J.b) * P.max_pages;
  const int last_page = min((L - 1) / kQuantPage, P.max_pages - 1);

  int id_k, id_v;                                               // of the unit whose loads go out next; lane: page rn / 8 of K, page g / 2 of V
  auto fetch_ids = [&](int t) __attribute__((always_inline)) {
    id_k = bt[min(2 * t + (rn >> 3), last_page)];
    id_v = bt[min(2 * t + (g >> 1), last_page)];
  };
  raw4 kr[kH][2];
  uint2 vr[kDT];
  float ks, vs;
  bool page_ok;
  // a page that is none of the pool's holds nothing: its tokens are masked, what is read instead is page 0
  auto usable = [&](int id) __attribute__((always_inline)) { return id >= 0 && id < P.num_pages; };
  auto issue_k = [&] __attribute__((always_inline)) {
    const unsigned char* at = k_lane + (usable(id_k) ? id_k : 0) * page_bytes;
#pragma unroll
    for (int h = 0; h < kH; ++h)
#pragma unroll
      for (int st = 0; st < 2; ++st) kr[h][st] = *reinterpret_cast<const raw4*>(at + 1024 * h + 64 * st);
  };
  auto issue_v = [&](int t) __attribute__((always_inline)) {
    const bool ok = usable(id_v);
    const int id = ok ? id_v : 0;
    const unsigned char* at = v_lane + id * page_bytes;
#pragma unroll
    for (int d = 0; d < kDT; ++d) vr[d] = *reinterpret_cast<const uint2*>(at + 256 * d);
    ks = P.k_scale[static_cast<int64_t>(id) * P.Hkv + J.kvh];
    vs = P.v_scale[static_cast<int64_t>(id) * P.Hkv + J.kvh];
    page_ok = ok && 2 * t + (g >> 1) < P.max_pages;
  };

  // ref: what a row's weights are relative to, in log2 units; sum: of this lane's tokens; v_ref: what the results are relative to
  float ref[NB], sum[NB], v_ref = __uint_as_float(static_cast<uint32_t>(kLeastScaleExp + 127) << 23);
  qf32x4 oacc[NB][kDT];
#pragma unroll
  for (int qi = 0; qi < NB; ++qi) {
    ref[qi] = kNoScore;
    sum[qi] = 0.f;
#pragma unroll
    for (int d = 0; d < kDT; ++d) oacc[qi][d] = qf32x4{0.f, 0.f, 0.f, 0.f};
  }

  // One unit.  MORE: the next unit's loads go out on the way.
  auto unit = [&](int t, int next, auto more_tag) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more_tag)::value;
    // ---- scores ----
    qf32x4 s[NB][2];
#pragma unroll
    for (int h = 0; h < kH; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const qbf16x8 a0 = operand_bf16(kr[h][0][2 * e], kr[h][0][2 * e + 1]), a1 = operand_bf16(kr[h][1][2 * e], kr[h][1][2 * e + 1]);
#pragma unroll
        for (int qi = 0; qi < NB; ++qi) {
          const qbf16x8 q = __builtin_bit_cast(qbf16x8, S.q[(kind * NB + qi) * 2 * kH + 2 * h + e][lane]);
          const qf32x4 zero = {0.f, 0.f, 0.f, 0.f};
          s[qi][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, q, h + e == 0 ? zero : s[qi][0], 0, 0, 0);
          s[qi][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, q, h + e == 0 ? zero : s[qi][1], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    const bool ok = page_ok;
    const float factor = ks * P.c, v_own = ok ? vs : 0.f;
    if constexpr (MORE) issue_k();

    // ---- masks: only where the unit reaches the drafts, or a page is none ----
    const int past = t * kUnit + 16 * (g >> 1) - J.ctx;         // the lane's page starts that far behind the context
    const bool drafts = (t + 1) * kUnit > J.ctx, masked = any_lane(!ok) || drafts;
    if (masked) {
#pragma unroll
      for (int qi = 0; qi < NB; ++qi) {
        uint32_t seen = 0xffffu;
        if (past > -16) {
          const int node = node_of(qi);
          seen = page_mask(S.anc[node][0], S.anc[node][1], past);
        }
        seen = ok ? seen >> (8 * (g & 1)) : 0u;
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[qi][st][i] = (seen >> (4 * st + i)) & 1u ? s[qi][st][i] : -INFINITY;
      }
    }

    // ---- a row's reference follows its maximum where that has come far ahead, and the scale of V likewise ----
    float top[NB];
    bool ahead = v_own > v_ref;
#pragma unroll
    for (int qi = 0; qi < NB; ++qi) {
      top[qi] = fmaxf(fmaxf(fmaxf(s[qi][0][0], s[qi][0][1]), fmaxf(s[qi][0][2], s[qi][0][3])),
                      fmaxf(fmaxf(s[qi][1][0], s[qi][1][1]), fmaxf(s[qi][1][2], s[qi][1][3]))) * factor;    // factor > 0
      ahead |= top[qi] > ref[qi] + kSlack;
    }
    if (any_lane(ahead)) {
      const float v_new = fmaxf(v_ref, groups_max(v_own)), v_by = v_ref * inverse_scale(v_new);
      v_ref = v_new;
#pragma unroll
      for (int qi = 0; qi < NB; ++qi) {
        const float now = fmaxf(ref[qi], groups_max(top[qi]));
        const float by = fast_exp2(ref[qi] - now);
        ref[qi] = now;
        sum[qi] *= by;
        const float all = by * v_by;
#pragma unroll
        for (int d = 0; d < kDT; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) oacc[qi][d][i] *= all;
      }
    }

    // ---- 2^shift times the weights, as TERMS fp16 terms ----
    // V is fed relative to v_ref, down to 2^-15 of it by itself, exactly; what a page's scale is smaller still goes into its weights, whose
    // fp16 has room for it.
    asm volatile("" : "+v"(v_ref));      // (its inverse worked out on both sides of the branch makes it one with an else part, whose copies cost the
                                         // registers of all results a second time)
    const float ratio = vs * inverse_scale(v_ref), v_by = fmaxf(ratio, kLeastV), p_by = ratio * inverse_scale(v_by);
    const float shift = static_cast<float>(static_cast<int>(__float_as_uint(p_by) >> 23) - 127 + kWeightBias);
    const float unshift = inverse_scale(p_by);
    raw4 hi[NB], lo[TERMS == 2 ? NB : 1];
#pragma unroll
    for (int qi = 0; qi < NB; ++qi) {
      const float sub = ref[qi] - shift;
      float z = 0.f;
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float p0 = fast_exp2(fmaf(s[qi][st][2 * i], factor, -sub)), p1 = fast_exp2(fmaf(s[qi][st][2 * i + 1], factor, -sub));
          z += p0 + p1;
          const qf16x2 h = {static_cast<_Float16>(p0), static_cast<_Float16>(p1)};
          hi[qi][2 * st + i] = __builtin_bit_cast(uint32_t, h);
          if constexpr (TERMS == 2) {
            const qf16x2 r = {static_cast<_Float16>(p0 - static_cast<float>(h[0])), static_cast<_Float16>(p1 - static_cast<float>(h[1]))};
            lo[qi][2 * st + i] = __builtin_bit_cast(uint32_t, r);
          }
        }
      sum[qi] = fmaf(z, unshift, sum[qi]);
    }

    // ---- O^T += V^T P^T ----
    // Slots behind the last token, and pages that are none, hold anything: a weight of zero times NaN would be NaN.
    uint32_t keep[2] = {~0u, ~0u};
    if (masked) {
      const int valid = ok ? min(max(L - t * kUnit - 8 * g, 0), 8) : 0;
      uint32_t nans = 0u;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        keep[w] = spread4(((1u << valid) - 1u) >> (4 * w));
        if constexpr (!SANITIZE) {
#pragma unroll
          for (int d = 0; d < kDT; ++d) nans |= nan_bytes((w ? vr[d].y : vr[d].x) & keep[w]);
        }
      }
      if (!SANITIZE && drafts && any_lane(nans != 0u) && lane == 0) S.nans = 1;
    }
#pragma unroll
    for (int d = 0; d < kDT; ++d) {
      uint32_t x = vr[d].x & keep[0], y = vr[d].y & keep[1];
      if constexpr (SANITIZE) {
        if (drafts) {
          x &= ~((nan_bytes(x) >> 7) * 0xffu);
          y &= ~((nan_bytes(y) >> 7) * 0xffu);
        }
      }
      const qf16x8 a = operand_f16(x, y, v_by);
#pragma unroll
      for (int qi = 0; qi < NB; ++qi) {
        oacc[qi][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, __builtin_bit_cast(qf16x8, hi[qi]), oacc[qi][d], 0, 0, 0);
        if constexpr (TERMS == 2)
          oacc[qi][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, __builtin_bit_cast(qf16x8, lo[qi]), oacc[qi][d], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (MORE) {
      issue_v(next);
      fetch_ids(min(next + slices, J.t1 - 1));
    }
  };

  int t = J.t0 + slice;
  if (t < J.t1) {
    fetch_ids(t);
    issue_k();
    issue_v(t);
    fetch_ids(min(t + slices, J.t1 - 1));
  }
  // ---- query operands, to LDS: step 2 h + e, lane group g: dimensions 16 (4 h + g) + 8 e .. + 8 (what a lane's 16 bytes of K hold) ----
  for (int f = wave; f < total_blocks * 2 * kH; f += kQaWaves) {
    const int s = f % (2 * kH), row = J.row_base + min(16 * (f / (2 * kH)) + rn, J.rows - 1);    // (columns past the last row repeat it)
    const uint16_t* qp = P.q + (static_cast<int64_t>(J.first + row / P.G) * P.Hq + J.kvh * P.G + row % P.G) * D + 16 * g;
    S.q[f][lane] = *reinterpret_cast<const raw4*>(qp + 64 * (s >> 1) + 8 * (s & 1));
  }
  __syncthreads();

  if (t < J.t1) {
    for (; t + slices < J.t1; t += slices) unit(t, t + slices, std::true_type{});
    unit(t, t, std::false_type{});
  }

  // ---- merge the waves that share rows, one block of each wave at a time ----
#pragma unroll
  for (int qi = 0; qi < NB; ++qi) {
    sum[qi] = groups_sum(sum[qi]) * (1.f / (1 << kWeightBias));
    if (sum[qi] == 0.f) ref[qi] = -INFINITY;                    // nothing seen
    if (lane < 16) {
      S.m[wave][16 * qi + lane] = ref[qi];
      S.l[wave][16 * qi + lane] = sum[qi];
    }
  }
  if constexpr (!SANITIZE) {
    if (touches_drafts) {
      __syncthreads();
      if (S.nans) return;
    }
  }
#pragma unroll
  for (int qi = 0; qi < NB; ++qi) {
    __syncthreads();
    float top = -INFINITY;
    for (int s = 0; s < slices; ++s) top = fmaxf(top, S.m[kind + kinds * s][16 * qi + rn]);
    const float f = ref[qi] == -INFINITY ? 0.f : fast_exp2(ref[qi] - top - static_cast<float>(kWeightBias)) * v_ref;
#pragma unroll
    for (int d = 0; d < kDT; ++d)
      *reinterpret_cast<float4*>(&S.o[wave][rn][16 * d + 4 * g]) =
          make_float4(oacc[qi][d][0] * f, oacc[qi][d][1] * f, oacc[qi][d][2] * f, oacc[qi][d][3] * f);
    __syncthreads();
    constexpr int kQuads = D / 4;
    for (int at = tid; at < kinds * 16 * kQuads; at += kQaThreads) {
      const int d4 = at % kQuads, r = at / kQuads % 16, k = at / (16 * kQuads);
      const int row = 16 * (k * NB + qi) + r;
      if (row >= J.rows) continue;
      float M = -INFINITY, Z = 0.f;
      for (int s = 0; s < slices; ++s) M = fmaxf(M, S.m[k + kinds * s][16 * qi + r]);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int s = 0; s < slices; ++s) {
        const int w = k + kinds * s;
        const float mw = S.m[w][16 * qi + r];
        if (mw != -INFINITY) Z += S.l[w][16 * qi + r] * fast_exp2(mw - M);
        const float4 x = *reinterpret_cast<const float4*>(&S.o[w][r][4 * d4]);
        o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
      }
      if constexpr (SANITIZE) put_back_nans<D>(P, S, J, row, 4 * d4, o);
      if (J.whole) {
        const int ra = J.row_base + row;
        const int64_t at_row = static_cast<int64_t>(J.first + ra / P.G) * P.Hq + J.kvh * P.G + ra % P.G;
        const float inv = Z == 0.f ? 0.f : 1.f / Z;             // a row that sees nothing gives 0 (and -inf)
        if (P.out_f32) {
          *reinterpret_cast<float4*>(static_cast<float*>(P.out) + at_row * D + 4 * d4) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        } else {
          const qbf16x2 a = {static_cast<__bf16>(o.x * inv), static_cast<__bf16>(o.y * inv)};
          const qbf16x2 c = {static_cast<__bf16>(o.z * inv), static_cast<__bf16>(o.w * inv)};
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out) + at_row * D + 4 * d4) =
              make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c));
        }
        if (P.lse && d4 == 0) P.lse[at_row] = (M + log2f(Z)) * static_cast<float>(kLn2);
      } else {
        *reinterpret_cast<float4*>(P.ws_o + (J.part + row) * D + 4 * d4) = o;
        if (d4 == 0) P.ws_ml[J.part + row] = make_float2(M, Z);
      }
    }
  }
}

// MAXB: most 16-row blocks a wave multiplies a unit with; TERMS: fp16 terms of a weight.
template <int D, int MAXB, int TERMS>
__global__ __launch_bounds__(kQaThreads, 2) void attn_quant_kernel(QuantAttnParams P) {
  __shared__ QuantAttnShared<D, MAXB> S;
  const int lane = threadIdx.x & 63;
  const int range = blockIdx.x;
  QuantPiece J;
  J.kvh = blockIdx.y;
  J.row_base = 16 * P.blocks * blockIdx.z;
  const int64_t pair = (static_cast<int64_t>(blockIdx.y) * gridDim.z + blockIdx.z) * P.ranges + range;
  const int batches = (P.B + 63) / 64;
  int64_t units = 0;
  Requests r;
  for (int k = batches - 1; k >= 0; --k) {                      // (down: the first 64 requests stay in registers)
    r = load_requests(P, k, lane);
    units += r.sum;
  }
  const int used = used_ranges(P, units);
  if (range >= used) return;
  int64_t at = units * range / used;
  const int64_t end = units * (range + 1) / used;
  int64_t base = 0;                                             // units before these 64 requests
  for (int k = 0; at < end; ) {
    const unsigned long long later = __ballot(base + r.upto > at);
    if (later == 0ull) {
      base += r.sum;
      if (++k >= batches) break;
      r = load_requests(P, k, lane);
      continue;
    }
    const int i = __ffsll(later) - 1;
    const int u = __builtin_amdgcn_readlane(r.units, i);
    const int64_t start = base + __builtin_amdgcn_readlane(r.upto, i) - u;
    const int64_t stop = min(end, start + u);
    J.b = 64 * k + i;
    J.ctx = __builtin_amdgcn_readlane(r.ctx, i);
    J.first = __builtin_amdgcn_readlane(r.first, i);
    J.n = __builtin_amdgcn_readlane(r.n, i);
    J.t0 = static_cast<int>(at - start);
    J.t1 = static_cast<int>(stop - start);
    J.rows = min(J.n * P.G - J.row_base, 16 * P.blocks);
    J.whole = at == start && stop == start + u;
    J.part = (pair * 2 + (at == start ? 1 : 0)) * (16 * P.blocks);
    at = stop;
    if (J.rows <= 0) continue;
    const int blocks = (J.rows + 15) / 16;
    const int kinds = blocks <= MAXB ? 1 : (blocks <= 2 * MAXB ? 2 : 4);
    const int per_wave = (blocks + kinds - 1) / kinds;
    [&] {
      if constexpr (MAXB >= 3) {
        if (per_wave == 3) return quant_piece<D, 3, TERMS, false>(P, S, J);
      }
      if constexpr (MAXB >= 2) {
        if (per_wave == 2) return quant_piece<D, 2, TERMS, false>(P, S, J);
      }
      quant_piece<D, 1, TERMS, false>(P, S, J);
    }();
    if (S.nans) {                                               // (written before a barrier, and next behind one)
      QuantPiece part = J;
      for (int from = 0; from < J.rows; from += 64) {
        part.row_base = J.row_base + from;
        part.rows = min(J.rows - from, 64);
        part.part = J.part + from;
        quant_piece<D, 1, TERMS, true>(P, S, part);
      }
    }
  }
}

// Requests whose units lie in more than one range: one row per D / 4 lanes, its partial results one after the other.
template <int D>
__global__ __launch_bounds__(256) void attn_quant_combine_kernel(QuantAttnParams P, int groups) {
  constexpr int kQuads = D / 4, kRows = 256 / kQuads;
  const int b = blockIdx.x, kvh = blockIdx.y, lane = threadIdx.x & 63;
  int64_t units = 0, start = 0;
  int u = 0, first = 0, n = 0;
  for (int k = (P.B + 63) / 64 - 1; k >= 0; --k) {
    const Requests r = load_requests(P, k, lane);
    units += r.sum;
    if (64 * k + 63 < b) start += r.sum;
    if (k == b >> 6) {
      u = __builtin_amdgcn_readlane(r.units, b & 63);
      start += __builtin_amdgcn_readlane(r.upto, b & 63) - u;
      first = __builtin_amdgcn_readlane(r.first, b & 63);
      n = __builtin_amdgcn_readlane(r.n, b & 63);
    }
  }
  if (u == 0) return;
  const int used = used_ranges(P, units);
  const int s0 = range_of(start, units, used), s1 = range_of(start + u - 1, units, used);
  if (s0 == s1) return;
  const int row = blockIdx.z * kRows + threadIdx.x / kQuads, d4 = threadIdx.x % kQuads;
  if (row >= n * P.G) return;
  const int per_group = 16 * P.blocks, grp = row / per_group;
  const int64_t pair = (static_cast<int64_t>(kvh) * groups + grp) * P.ranges;
  auto part = [&](int s) { return ((pair + s) * 2 + (s == s0 ? 1 : 0)) * per_group + row % per_group; };
  float M = -INFINITY;
  for (int s = s0; s <= s1; ++s) M = fmaxf(M, P.ws_ml[part(s)].x);
  float Z = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = s0; s <= s1; ++s) {
    const float2 ml = P.ws_ml[part(s)];
    const float f = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - M);
    const float4 x = *reinterpret_cast<const float4*>(P.ws_o + part(s) * D + 4 * d4);
    Z += ml.y * f;
    o.x += x.x * f; o.y += x.y * f; o.z += x.z * f; o.w += x.w * f;
  }
  const int64_t at_row = static_cast<int64_t>(first + row / P.G) * P.Hq + kvh * P.G + row % P.G;
  const float inv = Z == 0.f ? 0.f : 1.f / Z;
  if (P.out_f32) {
    *reinterpret_cast<float4*>(static_cast<float*>(P.out) + at_row * D + 4 * d4) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  } else {
    const qbf16x2 a = {static_cast<__bf16>(o.x * inv), static_cast<__bf16>(o.y * inv)};
    const qbf16x2 c = {static_cast<__bf16>(o.z * inv), static_cast<__bf16>(o.w * inv)};
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out) + at_row * D + 4 * d4) =
        make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c));
  }
  if (P.lse && d4 == 0) P.lse[at_row] = (M + log2f(Z)) * static_cast<float>(kLn2);
}

// ---- host ----------------------------------------------------------------------------------------------------
QuantAttnPlan make_quant_attn_plan(const AttnArgs& a) {
  QuantAttnPlan p{};
  const int64_t rows = static_cast<int64_t>(a.max_q) * (a.Hq / a.Hkv);
  const int blocks = static_cast<int>(std::max<int64_t>(1, (rows + 15) / 16));
  p.groups = (blocks + kQaBlocks - 1) / kQaBlocks;
  p.blocks = (blocks + p.groups - 1) / p.groups;
  p.wave_blocks = std::min(p.blocks, kQaWaveBlocks);
  const int64_t pairs = static_cast<int64_t>(a.Hkv) * p.groups;
  const int64_t target = 512;
  p.ranges = static_cast<int>(std::max<int64_t>(1, target / pairs));
  p.least_units = 8;
  return p;
}

static size_t quant_rows(const AttnArgs& a, const QuantAttnPlan& p) {
  return static_cast<size_t>(a.Hkv) * p.groups * p.ranges * 2 * 16 * p.blocks;
}
size_t quant_attn_workspace_bytes(const AttnArgs& a, const QuantAttnPlan& p) {
  return quant_rows(a, p) * (static_cast<size_t>(a.D) * sizeof(float) + sizeof(float2));
}

template <int D, int TERMS>
static void launch_quant(const QuantAttnParams& P, const AttnArgs& a, const QuantAttnPlan& p, hipStream_t stream) {
  const dim3 grid(p.ranges, a.Hkv, p.groups);
  auto kernel = p.wave_blocks == 1 ? attn_quant_kernel<D, 1, TERMS> : (p.wave_blocks == 2 ? attn_quant_kernel<D, 2, TERMS> : attn_quant_kernel<D, kQaWaveBlocks, TERMS>);
  hipLaunchKernelGGL(kernel, grid, dim3(kQaThreads), 0, stream, P);
  if (p.ranges > 1) {
    const int rows = a.max_q * (a.Hq / a.Hkv), per = 256 / (D / 4);
    hipLaunchKernelGGL((attn_quant_combine_kernel<D>), dim3(a.B, a.Hkv, (rows + per - 1) / per), dim3(256), 0, stream, P, p.groups);
  }
}

void launch_attn_quant(const AttnArgs& a, const float* k_scale, const float* v_scale, int num_pages, const QuantAttnPlan& p, hipStream_t stream) {
  QuantAttnParams P{};
  P.q = static_cast<const uint16_t*>(a.q); P.k_pool = static_cast<const unsigned char*>(a.k_pool);
  P.v_pool = static_cast<const unsigned char*>(a.v_pool); P.k_scale = k_scale; P.v_scale = v_scale;
  P.block_table = a.block_table; P.ctx_len = a.ctx_len; P.q_offsets = a.q_offsets; P.parent = a.parent;
  P.out = a.out; P.lse = a.lse;
  P.ws_o = static_cast<float*>(a.workspace);
  P.ws_ml = reinterpret_cast<float2*>(P.ws_o + quant_rows(a, p) * a.D);
  P.B = a.B; P.Hq = a.Hq; P.Hkv = a.Hkv; P.G = a.Hq / a.Hkv; P.total_q = a.total_q; P.max_pages = a.max_pages; P.num_pages = num_pages;
  P.ranges = p.ranges; P.least_units = p.least_units; P.blocks = p.blocks;
  P.c = a.scale * kLog2e; P.out_f32 = a.out_dtype == kF32;
  if (a.D == 128) P.out_f32 ? launch_quant<128, 2>(P, a, p, stream) : launch_quant<128, 1>(P, a, p, stream);
  else P.out_f32 ? launch_quant<64, 2>(P, a, p, stream) : launch_quant<64, 1>(P, a, p, stream);
}

}  // namespace specv
