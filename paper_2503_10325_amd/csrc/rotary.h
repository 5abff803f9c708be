// Device helpers of position rotation: which tokens of which request a workgroup takes, their angles, the rotation of 8 dimensions.
#pragma once
#include "common.h"

namespace specv {

constexpr int kRunTokens = 16;                 // a run: up to 16 consecutive tokens of a request
constexpr int kRotaryThreads = 256;
constexpr int kRotaryMaxTree = 128;
constexpr int kAngleStride = 64 + 2;           // pairs: 16 tokens' rows start 4 banks apart

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

// Which request run slot u belongs to: the last b with q_offsets[b] / 16 + 2 b <= u, by 64 comparisons a step.
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

// Request, first token's row, tokens of the request (not cut to what there is), context length of run slot u.
struct RunRequest {
  int b, first, n, ctx;
};
template <typename Params>
__device__ __forceinline__ RunRequest find_request(const Params& P, int u, int lane) {
  RunRequest R;
  if (P.B <= kWave) {                                           // one load for which request it is and what there is to know of it
    const int b = min(lane, P.B - 1), off = P.q_offsets[b], next = P.q_offsets[b + 1], ctx = P.ctx_len[b];
    const bool le = lane < P.B && (off >> 4) + 2 * lane <= u;
    R.b = max(__popcll(__builtin_amdgcn_ballot_w64(le)) - 1, 0);
    R.first = __builtin_amdgcn_readlane(off, R.b);
    R.n = __builtin_amdgcn_readlane(next, R.b);
    R.ctx = __builtin_amdgcn_readlane(ctx, R.b);
  } else {
    R.b = __builtin_amdgcn_readfirstlane(request_of_slot(P.q_offsets, P.B, u, lane));
    R.first = P.q_offsets[R.b];
    R.n = P.q_offsets[R.b + 1];
    R.ctx = P.ctx_len[R.b];
  }
  R.n = min(R.n, P.total_q) - R.first;
  if (P.parent) R.n = min(R.n, kRotaryMaxTree);
  return R;
}

// cosine and sine (times rotary_scale) of tokens row0 .. row0 + count - 1 of a request of n tokens, by all threads of a workgroup: what they take is
// asked for at once.  Nothing where P.rotary is 0.
struct RunAngles {
  __align__(16) float2 cs[kRunTokens][kAngleStride];
  int parent[kRotaryMaxTree];
  int pos[kRunTokens];
  float freq[64];
};
template <typename Params>
__device__ __forceinline__ void run_angles(const Params& P, RunAngles& S, int first, int n, int ctx, int row0, int count) {
  const int tid = threadIdx.x, half = P.rotary >> 1;
  const bool tree = half > 0 && P.positions == nullptr && P.parent;
  const int up = tree && tid < n ? P.parent[first + tid] : -1;
  const int given = half > 0 && P.positions && tid < count ? P.positions[row0 + tid] : 0;
  const float freq = tid < half ? P.inv_freq[tid] : 0.f;
  if (half > 0) {
    if (tid < half) S.freq[tid] = freq;
    const int i = row0 - first + tid;
    if (tree) {
      if (tid < n) S.parent[tid] = up;
      lds_sync();
      if (tid < count) {
        int depth = 0;
        for (int a = i; depth < kRotaryMaxTree; ++depth) {
          const int p = S.parent[a];
          if (p < 0 || p >= a) break;                           // (a malformed entry is a root)
          a = p;
        }
        S.pos[tid] = ctx + depth;
      }
    } else if (tid < count) {
      S.pos[tid] = P.positions ? given : ctx + i;
    }
    lds_sync();
    for (int at = tid; at < count * half; at += kRotaryThreads) {
      const int t = at / half, p = at - t * half;
      const double turns = static_cast<double>(S.pos[t]) * static_cast<double>(S.freq[p]) * 0.15915494309189535;
      const float2 w = cos_sin_turns(turns);
      S.cs[t][p] = make_float2(w.x * P.rotary_scale, w.y * P.rotary_scale);
    }
    lds_sync();
  }
}

}  // namespace specv
