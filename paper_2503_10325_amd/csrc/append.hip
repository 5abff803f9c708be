// Keys and values of new tokens into the paged cache, position rotation on the way; queries rotated in the same launch.
//
// Token i of request b goes to slot ctx_len[b] + i and is rotated by its position: ctx_len[b] + depth(i), where depth is i for
// prompts and linear drafts and the number of ancestors in a draft tree (so that the accepted path, moved to consecutive slots,
// is rotated as a linear context is), or the caller's own.  With pairs (x1, x2) of dimensions and a = position * inv_freq:
//   x1' = s (x1 cos a - x2 sin a),  x2' = s (x2 cos a + x1 sin a).
// The angle is reduced to a part of a turn in fp64 (at position 10^6 an fp32 angle is off by 0.03), sine and cosine are Taylor
// polynomials on an eighth of a turn in fp32 (off by 2^-23.5 at most, a rounded fp32 value by 2^-25), and what is stored is rounded once.  Of a
// long prompt's keys that moves 4 in 10^7 to a neighbouring e4m3 code (sine and cosine in fp64, rounded: 2 to 3), 2^-3 of their size at
// most away: not worth polynomials in fp64.
//
// Work: a workgroup takes the (up to 16) new tokens of one page, for a share of the heads; the angles of those tokens are
// worked out once, in LDS, for all of them.  Page slots are numbered without a scan: request b's start at q_offsets[b] / 16 + 2 b, which
// leaves room for the at most n / 16 + 2 pages that n tokens touch; slots without a page return at once.
// Bound by memory for prompts (22000 tokens x 32 heads of q, k and v: 230 us, 4.7 TB/s; 16384 tokens into the 8-bit cache 136 us, 4.7), by latency
// (offsets -> page id -> store) for a few tokens: 4 us for one request, 9 for 16 trees of 64 nodes, 11 for an 8-bit serving batch.
//
// 8-bit cache (quant.h): one wave takes the K or V of one (page, head): the largest entry, the scale, the codes; entries that the page
// already holds are rewritten where the scale grows.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "quant.h"

namespace specv {

constexpr int kAppendThreads = 256;
constexpr int kAppendWaves = kAppendThreads / kWave;
constexpr int kAppendMaxTree = 128;
constexpr int kAngleStride = 64 + 2;           // pairs: 16 tokens' rows start 4 banks apart

struct AppendParams {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  int64_t q_stride, k_stride, v_stride;        // elements between tokens
  const float* inv_freq;
  const int32_t* positions;
  void* k_pool;
  void* v_pool;
  float* k_scale;
  float* v_scale;
  const int32_t* block_table;
  const int32_t* ctx_len;
  const int32_t* q_offsets;
  const int32_t* parent;
  uint16_t* q_out;
  int B, Hq, Hkv, total_q, max_pages, num_pages, rotary, interleaved;
  float rotary_scale;
  int kv_shares, q_shares;
};

// The new tokens of one page: request, first token (row of q, k, v) and first slot, how many, the pool page (-1: none).
struct PageRun {
  int b, row0, slot0, count, page, ctx, first, n;
};

// sine and cosine of `turns` * 2 pi
__device__ __forceinline__ float2 cos_sin_turns(double turns) {
  const double part = turns - rint(turns);                    // [-1/2, 1/2]
  const double quarter = rint(4.0 * part);
  const float x = static_cast<float>((part - 0.25 * quarter) * 6.283185307179586);
  const float z = x * x;
  const float s = x * (1.f + z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880)))));
  const float c = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 + z * (-1.f / 3628800)))));
  const int k = static_cast<int>(quarter) & 3;
  const float cc = k & 1 ? s : c, ss = k & 1 ? c : s;
  return make_float2(k == 1 || k == 2 ? -cc : cc, k >= 2 ? -ss : ss);
}

// Which request page slot u belongs to: the last b with q_offsets[b] / 16 + 2 b <= u, by 64 comparisons a step.
__device__ __forceinline__ int request_of_slot(const int32_t* q_offsets, int B, int u, int lane) {
  int lo = 0, count = B;
  while (count > 1) {
    const int step = (count + kWave - 1) / kWave;
    const int b = lo + lane * step;
    const bool le = lane * step < count && (q_offsets[b] >> 4) + 2 * b <= u;
    const int k = max(__popcll(__ballot(le)) - 1, 0);
    lo += k * step;
    count = min(step, count - k * step);
  }
  return lo;
}

// 8 dimensions (unit `u` of a head) rotated.  own, other: the unit and the one that holds its partners (halves); cs: the token's
// angles.
__device__ __forceinline__ void rotate_halves(const float (&own)[8], const float (&other)[8], const float2* cs, int u, int half_units,
                                              float (&x)[8]) {
  const bool first = u < half_units;
  const float2* c = cs + 8 * (first ? u : u - half_units);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 w = c[j];
    x[j] = own[j] * w.x + other[j] * (first ? -w.y : w.y);
  }
}
__device__ __forceinline__ void rotate_neighbours(const float (&own)[8], const float2* cs, int u, float (&x)[8]) {
  const float2* c = cs + 4 * u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 w = c[j];
    x[2 * j] = own[2 * j] * w.x - own[2 * j + 1] * w.y;
    x[2 * j + 1] = own[2 * j + 1] * w.x + own[2 * j] * w.y;
  }
}

typedef __bf16 abf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ raw4 round_bf16(const float (&x)[8]) {
  raw4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const abf16x2 p = {static_cast<__bf16>(x[2 * j]), static_cast<__bf16>(x[2 * j + 1])};
    w[j] = __builtin_bit_cast(uint32_t, p);
  }
  return w;
}

// ---- 8-bit cache: the keys of one (page, head) --------------------------------------------------------------
// Lane: slot t = lane % 16, chunks of 16 dimensions lane / 16 and, for D = 128, 4 + lane / 16.
template <int D>
__device__ __forceinline__ void store_keys(const AppendParams& P, const PageRun& R, int head, const float2 (*cs)[kAngleStride], int lane) {
  constexpr int kChunks = D / 64;
  const int t = lane & 15, cg = lane >> 4;
  const int i = t - R.slot0;
  const bool fresh = i >= 0 && i < R.count;
  const int ti = min(max(i, 0), R.count - 1);
  const uint16_t* row = P.k + (R.row0 + ti) * P.k_stride + static_cast<int64_t>(head) * D;
  unsigned char* page = static_cast<unsigned char*>(P.k_pool) + (static_cast<int64_t>(R.page) * P.Hkv + head) * (kQuantPage * D);
  float* scale_at = P.k_scale + static_cast<int64_t>(R.page) * P.Hkv + head;
  const float old = R.slot0 > 0 ? *scale_at : 0.f;             // committed tokens lie in this page
  raw4 raw[kChunks][2];
#pragma unroll
  for (int a = 0; a < kChunks; ++a)
#pragma unroll
    for (int h = 0; h < 2; ++h) raw[a][h] = *reinterpret_cast<const raw4*>(row + 16 * (cg + 4 * a) + 8 * h);
  float x[kChunks][16];
  const int units = P.rotary >> 3, half = P.rotary >> 4;
  if (units > 0 && !P.interleaved) {
    raw4 other[kChunks][2];
    const bool inside = D == 128 && P.rotary == 128;             // the partners of a lane's two chunks are each other
#pragma unroll
    for (int a = 0; a < kChunks; ++a)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (inside) {
          other[a][h] = raw[kChunks - 1 - a][h];
        } else {
          const int u = 2 * (cg + 4 * a) + h;
          const int w = u < half ? u + half : (u < units ? u - half : u);
          other[a][h] = *reinterpret_cast<const raw4*>(row + 8 * w);
        }
      }
#pragma unroll
    for (int a = 0; a < kChunks; ++a)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int u = 2 * (cg + 4 * a) + h;
        float own[8], oth[8], y[8];
        unpack_bf16(raw[a][h], own);
        if (u < units) {
          unpack_bf16(other[a][h], oth);
          rotate_halves(own, oth, cs[ti], u, half, y);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = own[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) x[a][8 * h + j] = y[j];
      }
  } else {
#pragma unroll
    for (int a = 0; a < kChunks; ++a)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int u = 2 * (cg + 4 * a) + h;
        float own[8], y[8];
        unpack_bf16(raw[a][h], own);
        if (u < units) {
          rotate_neighbours(own, cs[ti], u, y);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = own[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) x[a][8 * h + j] = y[j];
      }
  }
  float amax = 0.f;
#pragma unroll
  for (int a = 0; a < kChunks; ++a)
#pragma unroll
    for (int j = 0; j < 16; ++j) amax = fmaxf(amax, finite_abs(x[a][j]));
  amax = wave_max(amax);                                        // (lanes of other slots repeat a new token)
  const float scale = fmaxf(old, page_scale(amax)), inv = inverse_scale(scale);
  if (lane == 0) *scale_at = scale;
  const bool grown = old > 0.f && scale > old;
#pragma unroll
  for (int a = 0; a < kChunks; ++a) {
    raw4* at = reinterpret_cast<raw4*>(page + (cg + 4 * a) * (kQuantPage * 16) + t * 16);
    if (fresh) {
      raw4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        w[j] = pack_e4m3(x[a][4 * j] * inv, x[a][4 * j + 1] * inv, x[a][4 * j + 2] * inv, x[a][4 * j + 3] * inv);
      *at = w;
    } else if (grown && t < R.slot0) {
      raw4 w = *at;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = rescale_e4m3(w[j], old * inv);
      *at = w;
    }
  }
}

// ---- ... the values of one (page, head) -----------------------------------------------------------------------
// Lane: two dimensions 2 (lane % (D / 2)) and 16 (D = 128) or 8 slots of them: a load takes whole rows, a lane's bytes are consecutive
// slots of a dimension, as the page holds them.
template <int D>
__device__ __forceinline__ void store_values(const AppendParams& P, const PageRun& R, int head, int lane) {
  constexpr int kPairs = D / 2, kSlots = 16 * kPairs / kWave, kWords = kSlots / 4;
  const int d = 2 * (lane % kPairs), t0 = lane / kPairs * kSlots;
  const uint16_t* col = P.v + static_cast<int64_t>(head) * D + d;
  unsigned char* page = static_cast<unsigned char*>(P.v_pool) + (static_cast<int64_t>(R.page) * P.Hkv + head) * (kQuantPage * D);
  float* scale_at = P.v_scale + static_cast<int64_t>(R.page) * P.Hkv + head;
  const float old = R.slot0 > 0 ? *scale_at : 0.f;
  uint32_t w[kSlots];
#pragma unroll
  for (int j = 0; j < kSlots; ++j) {
    const int ti = min(max(t0 + j - R.slot0, 0), R.count - 1);
    w[j] = *reinterpret_cast<const uint32_t*>(col + (R.row0 + ti) * P.v_stride);
  }
  uint32_t held[2][kWords];
  if (R.count < kQuantPage) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < kWords; ++j) held[e][j] = *reinterpret_cast<const uint32_t*>(page + (d + e) * kQuantPage + t0 + 4 * j);
  } else {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < kWords; ++j) held[e][j] = 0u;
  }
  float amax = 0.f;
#pragma unroll
  for (int j = 0; j < kSlots; ++j) amax = fmaxf(amax, fmaxf(finite_abs(bf16_lo(w[j])), finite_abs(bf16_hi(w[j]))));
  amax = wave_max(amax);
  const float scale = fmaxf(old, page_scale(amax)), inv = inverse_scale(scale);
  if (lane == 0) *scale_at = scale;
  const bool grown = old > 0.f && scale > old;
  uint32_t out[2][kWords];
#pragma unroll
  for (int j = 0; j < kWords; ++j) {
    out[0][j] = pack_e4m3(bf16_lo(w[4 * j]) * inv, bf16_lo(w[4 * j + 1]) * inv, bf16_lo(w[4 * j + 2]) * inv, bf16_lo(w[4 * j + 3]) * inv);
    out[1][j] = pack_e4m3(bf16_hi(w[4 * j]) * inv, bf16_hi(w[4 * j + 1]) * inv, bf16_hi(w[4 * j + 2]) * inv, bf16_hi(w[4 * j + 3]) * inv);
  }
  if (R.count < kQuantPage) {
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
      const uint32_t fresh = slot_mask(t0 + 4 * j, R.slot0, R.slot0 + R.count), before = slot_mask(t0 + 4 * j, 0, R.slot0);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        uint32_t keep = held[e][j];
        if (grown) keep = (rescale_e4m3(keep, old * inv) & before) | (keep & ~before);
        out[e][j] = (out[e][j] & fresh) | (keep & ~fresh);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int j = 0; j < kWords; ++j) *reinterpret_cast<uint32_t*>(page + (d + e) * kQuantPage + t0 + 4 * j) = out[e][j];
}

template <int D, bool QUANT>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendParams P) {
  constexpr int kPairUnits = D / 16;                            // items of a head: two units of 8 dimensions each
  __shared__ __align__(16) float2 sh_cs[kQuantPage][kAngleStride];
  __shared__ int sh_parent[kAppendMaxTree];
  __shared__ int sh_pos[kQuantPage];
  __shared__ float sh_freq[64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  PageRun R;
  if (P.B <= kWave) {                                           // one load for which request it is and what there is to know of it
    const int b = min(lane, P.B - 1), off = P.q_offsets[b], next = P.q_offsets[b + 1], ctx = P.ctx_len[b];
    const bool le = lane < P.B && (off >> 4) + 2 * lane <= static_cast<int>(blockIdx.x);
    R.b = max(__popcll(__builtin_amdgcn_ballot_w64(le)) - 1, 0);
    R.first = __builtin_amdgcn_readlane(off, R.b);
    R.n = __builtin_amdgcn_readlane(next, R.b);
    R.ctx = __builtin_amdgcn_readlane(ctx, R.b);
  } else {
    R.b = __builtin_amdgcn_readfirstlane(request_of_slot(P.q_offsets, P.B, blockIdx.x, lane));
    R.first = P.q_offsets[R.b];
    R.n = P.q_offsets[R.b + 1];
    R.ctx = P.ctx_len[R.b];
  }
  R.n = min(R.n, P.total_q) - R.first;
  if (P.parent) R.n = min(R.n, kAppendMaxTree);
  if (R.ctx < 0 || R.first < 0) return;
  const int64_t lp64 = static_cast<int64_t>(R.ctx >> 4) + (static_cast<int>(blockIdx.x) - (R.first >> 4) - 2 * R.b);
  const int64_t from = max(static_cast<int64_t>(R.ctx), 16 * lp64), to = min(static_cast<int64_t>(R.ctx) + R.n, 16 * lp64 + 16);
  if (from >= to) return;
  R.count = static_cast<int>(to - from);
  R.slot0 = static_cast<int>(from & 15);
  R.row0 = R.first + static_cast<int>(from - R.ctx);
  R.page = lp64 < P.max_pages ? P.block_table[static_cast<int64_t>(R.b) * P.max_pages + lp64] : -1;

  // ---- angles of the page's tokens: what they take is asked for at once ----
  const int half = P.rotary >> 1;
  const bool tree = half > 0 && P.positions == nullptr && P.parent;
  const int up = tree && tid < R.n ? P.parent[R.first + tid] : -1;
  const int given = half > 0 && P.positions && tid < R.count ? P.positions[R.row0 + tid] : 0;
  const float freq = tid < half ? P.inv_freq[tid] : 0.f;
  if (half > 0) {
    if (tid < half) sh_freq[tid] = freq;
    const int i = R.row0 - R.first + tid;
    if (tree) {
      if (tid < R.n) sh_parent[tid] = up;
      lds_sync();
      if (tid < R.count) {
        int depth = 0;
        for (int a = i; depth < kAppendMaxTree; ++depth) {
          const int p = sh_parent[a];
          if (p < 0 || p >= a) break;                           // (a malformed entry is a root)
          a = p;
        }
        sh_pos[tid] = R.ctx + depth;
      }
    } else if (tid < R.count) {
      sh_pos[tid] = P.positions ? given : R.ctx + i;
    }
    lds_sync();
    for (int at = tid; at < R.count * half; at += kAppendThreads) {
      const int t = at / half, p = at - t * half;
      const double turns = static_cast<double>(sh_pos[t]) * static_cast<double>(sh_freq[p]) * 0.15915494309189535;
      const float2 w = cos_sin_turns(turns);
      sh_cs[t][p] = make_float2(w.x * P.rotary_scale, w.y * P.rotary_scale);
    }
    lds_sync();
  }

  if (R.page < 0 || R.page >= P.num_pages) R.page = -1;

  // of a page's workgroups, kv_shares take keys and values (and queries, if q_shares is 0), q_shares queries
  const bool rows_only = static_cast<int>(blockIdx.y) >= P.kv_shares;
  const int share = rows_only ? blockIdx.y - P.kv_shares : blockIdx.y, shares = rows_only ? P.q_shares : P.kv_shares;
  if constexpr (QUANT) {
    if (R.page >= 0 && !rows_only) {
      const int jobs = 2 * P.Hkv;
      const int end = static_cast<int>(static_cast<int64_t>(jobs) * (share + 1) / shares);
      for (int j = static_cast<int>(static_cast<int64_t>(jobs) * share / shares) + wave; j < end; j += kAppendWaves) {
        if (j & 1) store_values<D>(P, R, j >> 1, lane);
        else store_keys<D>(P, R, j >> 1, sh_cs, lane);
      }
    }
  }

  // ---- rows of queries (and of keys and values of the bf16 cache): 32 bytes per lane, the partners of a rotation together ----
  if (P.q_shares > 0 && !rows_only) return;
  const int q_heads = P.q_out ? P.Hq : 0;
  const int heads = QUANT ? q_heads : q_heads + 2 * P.Hkv;
  const int h0 = static_cast<int>(static_cast<int64_t>(heads) * share / shares);
  const int width = (static_cast<int>(static_cast<int64_t>(heads) * (share + 1) / shares) - h0) * kPairUnits;   // items of a token
  const int items = width * R.count;
  const float per_width = 1.f / static_cast<float>(max(width, 1));
  const int rot = P.rotary >> 4;
  constexpr int kFly = 4;
  for (int base = 0; base < items; base += kFly * kAppendThreads) {
    raw4 a[kFly], b[kFly];
    raw4* to_a[kFly];
    int tok[kFly], pu[kFly], gap[kFly];
    bool turn[kFly];
#pragma unroll
    for (int f = 0; f < kFly; ++f) {
      const int at = base + f * kAppendThreads + tid;
      const int in = min(at, items - 1);
      const int t = static_cast<int>((static_cast<float>(in) + 0.5f) * per_width);       // in / width: exact below 2^21
      const int rem = in - t * width, head = h0 + rem / kPairUnits, p = rem % kPairUnits;
      const bool whole = P.interleaved || p >= rot;             // the item's units lie side by side
      const int ua = whole ? 2 * p : p;
      const bool is_q = head < q_heads, is_k = !is_q && head < q_heads + P.Hkv;
      const int64_t row = R.row0 + t;
      const int hk = head - q_heads - (is_k ? 0 : P.Hkv);
      const uint16_t* src = is_q ? P.q + row * P.q_stride + static_cast<int64_t>(head) * D
                                 : (is_k ? P.k + row * P.k_stride : P.v + row * P.v_stride) + static_cast<int64_t>(hk) * D;
      uint16_t* dst = is_q ? P.q_out + (row * P.Hq + head) * D
                           : static_cast<uint16_t*>(is_k ? P.k_pool : P.v_pool) +
                                 ((static_cast<int64_t>(R.page) * P.Hkv + hk) * kQuantPage + R.slot0 + t) * D;
      tok[f] = t; pu[f] = p;
      gap[f] = whole ? 1 : rot;                                 // units from the first to the second
      turn[f] = (is_q || is_k) && p < rot;
      to_a[f] = at < items && (is_q || R.page >= 0) ? reinterpret_cast<raw4*>(dst + 8 * ua) : nullptr;
      a[f] = *reinterpret_cast<const raw4*>(src + 8 * ua);
      b[f] = *reinterpret_cast<const raw4*>(src + 8 * (ua + gap[f]));
    }
#pragma unroll
    for (int f = 0; f < kFly; ++f) {
      if (!to_a[f]) continue;
      if (turn[f]) {
        float xa[8], xb[8], ya[8], yb[8];
        unpack_bf16(a[f], xa);
        unpack_bf16(b[f], xb);
        const float2* cs = sh_cs[tok[f]];
        if (P.interleaved) {
          rotate_neighbours(xa, cs, 2 * pu[f], ya);
          rotate_neighbours(xb, cs, 2 * pu[f] + 1, yb);
        } else {
          const float2* c = cs + 8 * pu[f];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 w = c[j];
            ya[j] = xa[j] * w.x - xb[j] * w.y;
            yb[j] = xb[j] * w.x + xa[j] * w.y;
          }
        }
        a[f] = round_bf16(ya);
        b[f] = round_bf16(yb);
      }
      to_a[f][0] = a[f];
      to_a[f][gap[f]] = b[f];
    }
  }
}

void launch_append(const AppendArgs& a, bool quant, hipStream_t stream) {
  AppendParams P{};
  P.q = static_cast<const uint16_t*>(a.q); P.k = static_cast<const uint16_t*>(a.k); P.v = static_cast<const uint16_t*>(a.v);
  P.q_stride = a.q_stride; P.k_stride = a.k_stride; P.v_stride = a.v_stride;
  P.inv_freq = a.inv_freq; P.positions = a.positions; P.k_pool = a.k_pool; P.v_pool = a.v_pool;
  P.k_scale = a.k_scale; P.v_scale = a.v_scale; P.block_table = a.block_table; P.ctx_len = a.ctx_len;
  P.q_offsets = a.q_offsets; P.parent = a.parent;
  P.q_out = a.rotary == 0 && a.q == a.q_out ? nullptr : static_cast<uint16_t*>(a.q_out);      // nothing to do for queries in place
  P.B = a.B; P.Hq = a.Hq; P.Hkv = a.Hkv; P.total_q = a.total_q; P.max_pages = a.max_pages; P.num_pages = a.num_pages;
  P.rotary = a.rotary; P.interleaved = a.interleaved; P.rotary_scale = a.rotary_scale;
  const int64_t slots = static_cast<int64_t>(a.total_q) / kQuantPage + 2 * static_cast<int64_t>(a.B);
  // shares of the heads: as many as fill the chip with few slots, one where slots are many (the angles are worked out once per share).  With few
  // slots, the 8-bit cache's queries have workgroups of their own beside those of its keys and values: one piece of work per wave, and latency
  // is what counts (64 requests of up to 10 tokens, 64 and 8 heads: 15.2 -> 11.6 us; for prompts, bound by memory, no gain).
  auto shares_of = [&](int64_t most) {
    int64_t n = 1;
    while (n < most && slots * n < (quant ? 1024 : 2048)) n *= 2;
    return static_cast<int>(std::min(n, most));
  };
  const int q_heads = P.q_out ? a.Hq : 0;
  P.kv_shares = quant ? shares_of(std::max(1, 2 * a.Hkv / kAppendWaves)) : shares_of(std::max(1, (a.Hq + 2 * a.Hkv) / 8));
  P.q_shares = quant && q_heads > 0 && slots < 1024 ? shares_of(std::max(1, q_heads / 8)) : 0;
  const dim3 grid(static_cast<unsigned>(slots), static_cast<unsigned>(P.kv_shares + P.q_shares));
  if (a.D == 128) {
    if (quant) hipLaunchKernelGGL((append_kernel<128, true>), grid, dim3(kAppendThreads), 0, stream, P);
    else hipLaunchKernelGGL((append_kernel<128, false>), grid, dim3(kAppendThreads), 0, stream, P);
  } else {
    if (quant) hipLaunchKernelGGL((append_kernel<64, true>), grid, dim3(kAppendThreads), 0, stream, P);
    else hipLaunchKernelGGL((append_kernel<64, false>), grid, dim3(kAppendThreads), 0, stream, P);
  }
}

}  // namespace specv
