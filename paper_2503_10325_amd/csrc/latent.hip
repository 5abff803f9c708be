// Around the attention over latents (attn_latent.hip): new tokens' latents into the cache, queries into the latent space, results out of it.
//
//   append   z = x / sqrt(mean(x^2) + eps) * g (or x), rotated shared key behind it: one row of the cache per token
//   absorb   q'[t, h] = [ q_nope[t, h] W_k[h] | rotated q_rope[t, h] ],  W_k [heads, nope_dim, latent_dim]
//   expand   o[t, h] = W_v[h] x[t, h],                                   W_v [heads, value_dim, latent_dim]
//
// The two products are a matrix per head with few rows: bound by the bytes of weights, inputs and results.  A workgroup keeps a slice of
// one head's weight in LDS and takes tokens 16 per wave; their operands come straight from memory.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "latent.h"
#include "rotary.h"

namespace specv {

constexpr int kLatentThreads = kRotaryThreads;
constexpr int kLatentWaves = kLatentThreads / kWave;

struct LatentParams {
  const uint16_t* latent;        // append: rows of the step
  const uint16_t* key;
  int64_t latent_stride, key_stride;
  const uint16_t* norm;
  uint16_t* pool;
  const uint16_t* q;             // absorb
  const uint16_t* w;             // absorb, expand: heads w_stride elements apart
  int64_t q_stride, w_stride;
  const uint16_t* x;             // expand
  uint16_t* out;
  const float* inv_freq;
  const int32_t* positions;
  const int32_t* block_table;
  const int32_t* ctx_len;
  const int32_t* q_offsets;
  const int32_t* parent;
  int B, H, C, nope, value, total_q, max_pages, num_pages, rotary, interleaved;
  float rotary_scale, eps;
  int slots, shares, runs;       // absorb: run slots, shares of the heads; workgroups that rotate
  int pieces, chunk;             // absorb, expand: pieces of the tokens, tokens of each
};

// ---- append -----------------------------------------------------------------------------------------------------
// 1 / sqrt(x), to about 2^-47: the instruction's estimate (2^-24) and a step of Newton's method, which takes an error of e to 1.5 e^2.
__device__ __forceinline__ double inverse_root(double x) {
  const double y = __builtin_amdgcn_rsq(x), next = fma(0.5 * y, fma(-x * y, y, 1.0), y);
  return x > 0.0 && x < INFINITY ? next : y;
}
// A workgroup takes the new tokens of one page, a wave four of them at a time, their latents asked for before anything else.  Sums of squares are held in
// fp64 (so that no bf16 latent overflows them), a result is rounded to fp32 and then once to bf16.  Few tokens: a chain of trips to memory, 3 us;
// 22000 tokens: 15 us, 3.3 TB/s read + written (a copy: 5.2), as all workgroups are resident and load, compute and store at the same time.
template <int C>
__global__ __launch_bounds__(kLatentThreads) void append_latent_kernel(LatentParams P) {
  constexpr int E = C / kWave;                                  // elements of a lane
  typedef uint32_t Words __attribute__((ext_vector_type(E / 2)));
  __shared__ RunAngles angles;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const RunRequest R = find_request(P, blockIdx.x, lane);
  if (R.ctx < 0 || R.first < 0) return;
  const int64_t lp = static_cast<int64_t>(R.ctx >> 4) + (static_cast<int>(blockIdx.x) - (R.first >> 4) - 2 * R.b);
  const int64_t from = max(static_cast<int64_t>(R.ctx), 16 * lp), to = min(static_cast<int64_t>(R.ctx) + R.n, 16 * lp + 16);
  if (from >= to) return;
  const int count = static_cast<int>(to - from), slot0 = static_cast<int>(from & 15), row0 = R.first + static_cast<int>(from - R.ctx);
  const int page = lp < P.max_pages ? P.block_table[static_cast<int64_t>(R.b) * P.max_pages + lp] : -1;
  constexpr int kMine = kRunTokens / kLatentWaves;
  Words x[kMine], g;
#pragma unroll
  for (int j = 0; j < kMine; ++j)
    x[j] = *reinterpret_cast<const Words*>(P.latent + (row0 + min(wave + j * kLatentWaves, count - 1)) * P.latent_stride + E * lane);
  if (P.norm) g = *reinterpret_cast<const Words*>(P.norm + E * lane);
  // the shared key: 8 dimensions of a token per thread, and their partners where pairs are halves
  const int units = P.rotary >> 3, half = units >> 1;
  const int kt = tid / units, ku = tid - kt * units;
  const bool turns = kt < count;
  raw4 own, other;
  if (turns) {
    const uint16_t* row = P.key + (row0 + kt) * P.key_stride;
    own = *reinterpret_cast<const raw4*>(row + 8 * ku);
    other = *reinterpret_cast<const raw4*>(row + 8 * (ku < half ? ku + half : ku - half));
  }
  run_angles(P, angles, R.first, R.n, R.ctx, row0, count);
  if (page < 0 || page >= P.num_pages) return;
  const int W = C + P.rotary;
  uint16_t* const rows = P.pool + (static_cast<int64_t>(page) * kRunTokens + slot0) * W;
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int t = wave + j * kLatentWaves;
    if (t >= count) break;
    if (P.norm) {
      double sum = 0.0;
#pragma unroll
      for (int i = 0; i < E / 2; ++i) {
        const double a = bf16_lo(x[j][i]), b = bf16_hi(x[j][i]);
        sum = fma(a, a, sum);
        sum = fma(b, b, sum);
      }
      const double by = inverse_root(wave_sum(sum) * (1.0 / C) + static_cast<double>(P.eps));
#pragma unroll
      for (int i = 0; i < E / 2; ++i) {
        const abf16x2 y = {static_cast<__bf16>(static_cast<float>(bf16_lo(x[j][i]) * by * bf16_lo(g[i]))),
                           static_cast<__bf16>(static_cast<float>(bf16_hi(x[j][i]) * by * bf16_hi(g[i])))};
        x[j][i] = __builtin_bit_cast(uint32_t, y);
      }
    }
    *reinterpret_cast<Words*>(rows + static_cast<int64_t>(t) * W + E * lane) = x[j];
  }
  if (turns) {
    float a[8], b[8], y[8];
    unpack_bf16(own, a);
    unpack_bf16(other, b);
    if (P.interleaved) rotate_neighbours(a, angles.cs[kt], ku, y);
    else rotate_halves(a, b, angles.cs[kt], ku, half, y);
    *reinterpret_cast<raw4*>(rows + static_cast<int64_t>(kt) * W + C + 8 * ku) = round_bf16(y);
  }
}

// Rows that belong to requests.
__device__ __forceinline__ int rows_end(const LatentParams& P) { return min(P.q_offsets[P.B], P.total_q); }

// Workgroup `i` of a product: its head, slice of the head's weight and piece of the tokens.  Workgroups go to the 8 XCDs in turn: slices of a head, which read
// the same tokens, and pieces, which share a weight, share an L2 (128 heads, 1024 tokens absorbed: 53 us with slices apart, 46 together).
__device__ __forceinline__ void find_piece(int i, int slices, int pieces, int& h, int& slice, int& piece) {
  const int k = i >> 3, each = slices * pieces, in = k % each;
  h = k / each * 8 + (i & 7);
  piece = in / slices;
  slice = in % slices;
}

// ---- absorb -----------------------------------------------------------------------------------------------------
// The rotary part: up to 16 tokens of a request, a share of the heads; 8 dimensions per item.
__device__ __forceinline__ void rotate_queries(const LatentParams& P, RunAngles& angles, int i) {
  const int tid = threadIdx.x, slot = i / P.shares, share = i - slot * P.shares;
  const RunRequest R = find_request(P, slot, tid & 63);
  if (R.first < 0) return;
  const int at = kRunTokens * (slot - (R.first >> 4) - 2 * R.b), count = min(R.n - at, kRunTokens);
  if (at < 0 || count <= 0) return;
  const int row0 = R.first + at;
  run_angles(P, angles, R.first, R.n, R.ctx, row0, count);
  const int units = P.rotary >> 3, half = units >> 1;
  const int h0 = static_cast<int>(static_cast<int64_t>(P.H) * share / P.shares), heads = static_cast<int>(static_cast<int64_t>(P.H) * (share + 1) / P.shares) - h0;
  const int width = heads * units, items = width * count, W = P.C + P.rotary, Q = P.nope + P.rotary;
  for (int item = tid; item < items; item += kLatentThreads) {
    const int t = item / width, rem = item - t * width, h = h0 + rem / units, u = rem % units;
    const uint16_t* row = P.q + (row0 + t) * P.q_stride + static_cast<int64_t>(h) * Q + P.nope;
    const raw4 own = *reinterpret_cast<const raw4*>(row + 8 * u), other = *reinterpret_cast<const raw4*>(row + 8 * (u < half ? u + half : u - half));
    float a[8], b[8], y[8];
    unpack_bf16(own, a);
    unpack_bf16(other, b);
    if (P.interleaved) rotate_neighbours(a, angles.cs[t], u, y);
    else rotate_halves(a, b, angles.cs[t], u, half, y);
    *reinterpret_cast<raw4*>(P.out + (static_cast<int64_t>(row0 + t) * P.H + h) * W + P.C + 8 * u) = round_bf16(y);
  }
}

constexpr int kAbsorbSlice = 128;             // columns of the latent

// out^T = W^T q^T.  W^T is read from LDS by columns; columns of a wave's 16-column blocks 2 p and 2 p + 1 are dealt so that a lane ends up with 8
// consecutive ones (32 p + 8 g .. + 8).  WAVES: waves that take tokens of their own (1: all take the same 16, and a quarter of the columns each).
// 128 heads, C = 512: 64 tokens 8.6 us, 3.4 TB/s; 1024 tokens 66 us, 3.3 TB/s, a third of it reads (37 us without the stores).
template <int N, int WAVES>
__global__ __launch_bounds__(kLatentThreads) void absorb_latent_kernel(LatentParams P) {
  union Shared {
    __align__(1024) unsigned char w[N * 2 * kAbsorbSlice];
    RunAngles angles;
  };
  __shared__ Shared S;
  if (static_cast<int>(blockIdx.x) < P.runs) {
    if (static_cast<int>(blockIdx.x) < P.slots * P.shares) rotate_queries(P, S.angles, blockIdx.x);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rn = lane & 15, g = lane >> 4;
  const int slices = P.C / kAbsorbSlice;
  int h, slice, piece;
  find_piece(blockIdx.x - P.runs, slices, P.pieces, h, slice, piece);
  if (h >= P.H) return;
  const int W = P.C + P.rotary, Q = N + P.rotary;

  // rows of 256 bytes; 16-byte unit u of row r lies at u ^ 4 (r % 4): 16 lanes that read 4 rows by columns take 128 bytes from as many banks
  const unsigned lds = lds_address(S.w);
  {
    const unsigned char* from = reinterpret_cast<const unsigned char*>(P.w + h * P.w_stride + slice * kAbsorbSlice);
    const unsigned off = (lane >> 4) * P.C * 2 + ((lane & 15) ^ (4 * (lane >> 4))) * 16;
#pragma unroll
    for (int j = 0; j < N / 16; ++j) {
      const int part = wave * (N / 16) + j;                     // 4 rows
      load_to_lds(from + static_cast<int64_t>(part) * 4 * P.C * 2, off, lds + 1024 * part, 0);
    }
  }
  const int end = min(rows_end(P), (piece + 1) * P.chunk);
  int t = piece * P.chunk + (WAVES == 1 ? 0 : 16 * wave);
  const uint16_t* const q = P.q + static_cast<int64_t>(h) * Q + 8 * g;
  raw4 b[N / 32];
  auto fetch = [&](int at) __attribute__((always_inline)) {
    const uint16_t* row = q + min(at + rn, end - 1) * P.q_stride;
#pragma unroll
    for (int k = 0; k < N / 32; ++k) b[k] = *reinterpret_cast<const raw4*>(row + 32 * k);
  };
  if (t < end) fetch(t);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  lds_sync();
  constexpr int kBlocks = WAVES == 1 ? 2 : 8, kStep = 16 * WAVES;
  const unsigned a_at = lds + (8 * g + (rn >> 2)) * 256 + (4 * (rn >> 2) + (rn & 3)) * 16;
  const int p0 = WAVES == 1 ? wave : 0;                         // pairs of blocks
  for (; t < end; t += kStep) {
    lf32x4 acc[kBlocks];
#pragma unroll
    for (int m = 0; m < kBlocks; ++m) acc[m] = lf32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < N / 32; ++k)
#pragma unroll
      for (int m = 0; m < kBlocks; ++m) {
        const unsigned at = (a_at ^ ((p0 + (m >> 1)) * 64)) + k * 32 * 256 + 8 * (m & 1);
        acc[m] = multiply(join(read_columns(at), read_columns(at + 4 * 256)), operand(b[k]), acc[m]);
      }
    const int row = t + rn;
    if (t + kStep < end) fetch(t + kStep);
    if (row < end) {
      uint16_t* to = P.out + (static_cast<int64_t>(row) * P.H + h) * W + slice * kAbsorbSlice + 32 * p0 + 8 * g;
#pragma unroll
      for (int m = 0; m < kBlocks; m += 2) {
        const uint2 lo = pack4(acc[m]), hi = pack4(acc[m + 1]);
        *reinterpret_cast<uint4*>(to + 16 * m) = make_uint4(lo.x, lo.y, hi.x, hi.y);
      }
    }
  }
}

// ---- expand -----------------------------------------------------------------------------------------------------
constexpr int kExpandSlice = 64;              // dimensions of the value

// o^T = W x^T, W's rows read from LDS as they lie.  Dimension 32 p + 8 g + 4 s + i is row 4 g + i of block 2 p + s: a lane ends up with 8 consecutive ones.
// 128 heads, 64 requests of 2 to 10 tokens, C = 512: 18.5 us, 4.3 TB/s; two workgroups on a compute unit (three or four, with fewer tokens each: 21.6).
template <int C, int WAVES>
__global__ __launch_bounds__(kLatentThreads, 2) void expand_latent_kernel(LatentParams P) {
  extern __shared__ __align__(1024) unsigned char smem[];
  constexpr int kRow = 2 * C, kSteps = C / 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rn = lane & 15, g = lane >> 4;
  const int slices = P.value / kExpandSlice;
  int h, slice, piece;
  find_piece(blockIdx.x, slices, P.pieces, h, slice, piece);
  if (h >= P.H) return;

  // 16-byte unit u of row r lies at u ^ (r % 4 + 4 (r / 8 % 2)): 8 lanes that read 8 rows' units (rows 0 .. 3, 8 .. 11) take 128 bytes from as many banks
  const unsigned lds = lds_address(smem);
  {
    const unsigned char* from = reinterpret_cast<const unsigned char*>(P.w + h * P.w_stride + static_cast<int64_t>(slice) * kExpandSlice * C);
    constexpr int kPer = 1024 / kRow, kParts = kExpandSlice / kPer / kLatentWaves;      // rows of a load
#pragma unroll
    for (int j = 0; j < kParts; ++j) {
      const int part = wave * kParts + j, r = part * kPer + lane * 16 / kRow, u = lane % (kRow / 16);
      load_to_lds(from + part * 1024, (lane * 16 / kRow) * kRow + (u ^ ((r & 3) + 4 * ((r >> 3) & 1))) * 16, lds + 1024 * part, 0);
    }
  }
  const int end = min(rows_end(P), (piece + 1) * P.chunk);
  int t = piece * P.chunk + (WAVES == 1 ? 0 : 16 * wave);
  const uint16_t* const x = P.x + static_cast<int64_t>(h) * C + 8 * g;
  raw4 b[kSteps];
  auto fetch = [&](int at) __attribute__((always_inline)) {
    const uint16_t* row = x + static_cast<int64_t>(min(at + rn, end - 1)) * P.H * C;
#pragma unroll
    for (int k = 0; k < kSteps; ++k) b[k] = *reinterpret_cast<const raw4*>(row + 32 * k);
  };
  if (t < end) fetch(t);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  lds_sync();
  constexpr int kBlocks = WAVES == 1 ? 1 : 4, kStep = 16 * WAVES;
  const int m0 = WAVES == 1 ? wave : 0;
  const unsigned swizzle = (rn & 3) + 4 * ((rn >> 2) & 1);
  const unsigned a_at = lds + (8 * (rn >> 2) + (rn & 3)) * kRow;
  for (; t < end; t += kStep) {
    lf32x4 acc[kBlocks];
#pragma unroll
    for (int m = 0; m < kBlocks; ++m) acc[m] = lf32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
      for (int m = 0; m < kBlocks; ++m) {
        const int block = m0 + m;
        const unsigned at = a_at + (32 * (block >> 1) + 4 * (block & 1)) * kRow + ((4 * k + g) ^ swizzle) * 16;
        const raw4 a = read_lds16(at);
        acc[m] = multiply(operand(a), operand(b[k]), acc[m]);
        if (m == kBlocks - 1 && k % 4 == 3) __builtin_amdgcn_sched_barrier(0);      // (else all of W is read first, into registers there are none of)
      }
    const int row = t + rn;
    if (t + kStep < end) fetch(t + kStep);
    if (row < end) {
      uint16_t* to = P.out + (static_cast<int64_t>(row) * P.H + h) * P.value + slice * kExpandSlice + 8 * g;
      if constexpr (WAVES == 1) {
        *reinterpret_cast<uint2*>(to + 32 * (m0 >> 1) + 4 * (m0 & 1)) = pack4(acc[0]);
      } else {
#pragma unroll
        for (int m = 0; m < kBlocks; m += 2) {
          const uint2 lo = pack4(acc[m]), hi = pack4(acc[m + 1]);
          *reinterpret_cast<uint4*>(to + 16 * m) = make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
      }
    }
  }
}

// ---- host ---------------------------------------------------------------------------------------------------------
static LatentParams latent_params(const LatentArgs& a) {
  LatentParams P{};
  P.inv_freq = a.inv_freq; P.positions = a.positions; P.block_table = a.block_table; P.ctx_len = a.ctx_len; P.q_offsets = a.q_offsets; P.parent = a.parent;
  P.B = a.B; P.H = a.H; P.C = a.C; P.nope = a.nope; P.value = a.value; P.total_q = a.total_q; P.max_pages = a.max_pages; P.num_pages = a.num_pages;
  P.rotary = a.R; P.interleaved = a.interleaved; P.rotary_scale = a.rotary_scale; P.eps = a.eps;
  return P;
}
static int run_slots(const LatentArgs& a) { return a.total_q / kRunTokens + 2 * a.B; }

void launch_append_latent(const LatentArgs& a, const void* latent, int64_t latent_stride, const void* key, int64_t key_stride, const void* norm, void* pool,
                          hipStream_t stream) {
  LatentParams P = latent_params(a);
  P.latent = static_cast<const uint16_t*>(latent); P.latent_stride = latent_stride; P.key = static_cast<const uint16_t*>(key); P.key_stride = key_stride;
  P.norm = static_cast<const uint16_t*>(norm); P.pool = static_cast<uint16_t*>(pool);
  const dim3 grid(run_slots(a));
  if (a.C == 512) hipLaunchKernelGGL(append_latent_kernel<512>, grid, dim3(kLatentThreads), 0, stream, P);
  else hipLaunchKernelGGL(append_latent_kernel<256>, grid, dim3(kLatentThreads), 0, stream, P);
}

// Pieces of the tokens: as many workgroups as fill the chip twice, of whole 64 tokens.
static void cut_tokens(LatentParams& P, int pairs) {
  const int most = (P.total_q + 63) / 64;
  P.pieces = std::min(most, std::max(1, 512 / pairs));
  P.chunk = (most + P.pieces - 1) / P.pieces * 64;
  P.pieces = (P.total_q + P.chunk - 1) / P.chunk;
}

void launch_absorb_latent(const LatentArgs& a, const void* q, int64_t q_stride, const void* w, int64_t w_stride, void* out, hipStream_t stream) {
  LatentParams P = latent_params(a);
  P.q = static_cast<const uint16_t*>(q); P.q_stride = q_stride; P.w = static_cast<const uint16_t*>(w); P.w_stride = w_stride; P.out = static_cast<uint16_t*>(out);
  P.slots = run_slots(a);
  P.shares = 1;
  while (P.shares < a.H / 8 && P.slots * P.shares < 512) P.shares *= 2;
  P.runs = (P.slots * P.shares + 7) / 8 * 8;
  const int slices = a.C / kAbsorbSlice;
  cut_tokens(P, a.H * slices);
  const dim3 grid(P.runs + (a.H + 7) / 8 * 8 * slices * P.pieces);
  if (a.nope == 128) {
    if (a.total_q > 16) hipLaunchKernelGGL((absorb_latent_kernel<128, 4>), grid, dim3(kLatentThreads), 0, stream, P);
    else hipLaunchKernelGGL((absorb_latent_kernel<128, 1>), grid, dim3(kLatentThreads), 0, stream, P);
  } else {
    if (a.total_q > 16) hipLaunchKernelGGL((absorb_latent_kernel<64, 4>), grid, dim3(kLatentThreads), 0, stream, P);
    else hipLaunchKernelGGL((absorb_latent_kernel<64, 1>), grid, dim3(kLatentThreads), 0, stream, P);
  }
}

int launch_expand_latent(const LatentArgs& a, const void* x, const void* w, int64_t w_stride, void* out, hipStream_t stream) {
  LatentParams P = latent_params(a);
  P.x = static_cast<const uint16_t*>(x); P.w = static_cast<const uint16_t*>(w); P.w_stride = w_stride; P.out = static_cast<uint16_t*>(out);
  const int slices = a.value / kExpandSlice;
  cut_tokens(P, a.H * slices);
  const dim3 grid((a.H + 7) / 8 * 8 * slices * P.pieces);
  const size_t lds = static_cast<size_t>(kExpandSlice) * 2 * a.C;
  if (a.C == 512) {
    if (a.total_q > 16) hipLaunchKernelGGL((expand_latent_kernel<512, 4>), grid, dim3(kLatentThreads), lds, stream, P);
    else hipLaunchKernelGGL((expand_latent_kernel<512, 1>), grid, dim3(kLatentThreads), lds, stream, P);
  } else {
    if (a.total_q > 16) hipLaunchKernelGGL((expand_latent_kernel<256, 4>), grid, dim3(kLatentThreads), lds, stream, P);
    else hipLaunchKernelGGL((expand_latent_kernel<256, 1>), grid, dim3(kLatentThreads), lds, stream, P);
  }
  return 0;
}

}  // namespace specv
