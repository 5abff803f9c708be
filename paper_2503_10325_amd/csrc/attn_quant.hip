// Verify-attention over the 8-bit paged cache (quant.h): the draft queries of each request attend over its committed context and
// their draft ancestors, keys and values read as e4m3 with a scale per (page, KV head).
//
// A wave takes units of 32 tokens (2 pages), straight from memory into a buffer of its own in LDS, and from there to registers at once,
// so that the next unit is on its way meanwhile: no barrier stands between memory and the matrix cores, and the bytes in flight cost no
// registers.  Pages are laid out so that a lane's 16 (K) or 8 (V) bytes are matrix operands as they lie, without transposition.
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16, tokens as M.  Row 4 g + i of sub-tile t is token 8 (g % 2) + 4 t + i of page g / 2, so that
//                 lane group g (lanes 16 g .. 16 g + 15, one query row each) ends up with 8 tokens of one page: its scale is one register, and
//   O^T = V^T P^T takes those 8 weights as its operand without any exchange between lanes.
// e4m3 is exact in bf16 and fp16.  K's scale rides on the softmax factor; V is fed in fp16, its page's scale on the conversion, relative to the
// largest scale so far.  A weight is one fp16 term (2^-11 off at most, an eighth of the rounding
// of a bf16 result, and independent of its neighbours': results end up about 1 % further from the exact ones than with fp32 weights), or two for fp32 results.
//
// Work: a request's query rows of a KV head are taken in groups of up to 64 (a wave multiplies each unit with up to four 16-row blocks).
// Per KV head the units of all requests and groups lie end to end and are cut into ranges of equal cost, one per workgroup, whatever the
// lengths; every workgroup works out from ctx_len and q_offsets which pieces its range holds.  A range that ends inside a request
// leaves a partial result and its sum of weights; the workgroup that finishes the last piece merges them, in their order.  The four or
// eight waves of a workgroup take units in turn and merge through LDS.
//
// Bound by memory up to 48 rows (64 requests x 8 KV heads x 2048 tokens, 8 to 32 rows: 55 to 60 us, 4.9 to 4.7 TB/s; 4096 tokens 5.15), by the
// vector and matrix instructions of a SIMD's two waves beyond (64 rows 67 us; trees of 64 nodes, 256 rows, 4096 tokens: 84 to 91 us, 770 to 830
// TFLOP/s, vector issue 54 %, matrix cores 33 %), by latency for few tokens: the launch, two dependent trips to memory before the first page, and the merge are 8 us.
#include <algorithm>
#include <atomic>
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

constexpr int kUnit = 32;                     // tokens a wave takes at a time
constexpr int kQaMaxNodes = 128;
constexpr int kMergeRoom = 2048;              // (piece, row) pairs whose statistics a merge holds at a time
constexpr float kNoScore = -3.0e38f;          // the reference before the first position: finite, so that -infinity stays ahead of nothing
constexpr int kQaBlocks = 4;                  // most 16-row blocks that a wave multiplies a unit with: what 256 registers hold (a
constexpr int most_blocks(int D, int terms) { return D == 128 && terms == 2 ? 3 : kQaBlocks; }      // second term's operands are too many)
constexpr int kWeightBias = 6;                // weights are fed as fp16(2^6 p): normal down to p = 2^-20, and
constexpr float kSlack = 8.f;                 // the reference of a row's softmax follows its maximum when that is 2^8 ahead: below 2^14 then
constexpr float kLeastV = 3.0517578125e-5f;   // 2^-15: what V may be scaled by and still be exact in fp16
constexpr float kLeastWeight = 0x1p-40f;       // what weights are scaled by at least.  At most 2^(8 + kWeightBias - 40) is 0 in fp16 already, so
                                              // nothing smaller is fed; the weights' sum, which is of scaled ones, loses no weight above 2^-92
static __device__ const float kNoScale[1] = {0.f};      // read in place of the scale of a page that is none

constexpr int ilog2(int x) { return x <= 1 ? 0 : 1 + ilog2(x / 2); }

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
  float* ws_o;        // [KV heads][ranges][2][rows][D] partial results, each by its own sum of weights
  float2* ws_ml;      // ... [rows] (maximum in log2 units, sum)
  int B, Hq, Hkv, G, total_q, max_q, max_pages, num_pages;
  uint32_t inverse_G; // 2^31 / G, rounded up
  unsigned long long* arrived;      // [KV heads][groups][B] messages: how many pieces of a request's rows are done
  unsigned long long tag;
  int ranges;         // per KV head, at most
  int groups;         // of query rows, at most
  int rows;           // of a group, at most
  int halves;         // 2: rows that are too many for a wave are dealt to two halves of a workgroup's waves
  int shift;          // units are counted in chunks of 2^shift
  float c;            // scale * log2(e)
  int out_f32;
};

// The kernel's arguments where the launch has put them, read through the scalar cache when they are needed: kept in registers across the pieces'
// loop, they and what follows from them would need more lanes of vector registers than there are.
typedef const __attribute__((address_space(4))) QuantAttnParams KernelParams;
__device__ __forceinline__ KernelParams& kernel_params() {
  uint64_t at = reinterpret_cast<uint64_t>((const __attribute__((address_space(4))) void*)__builtin_amdgcn_kernarg_segment_ptr());
  asm volatile("" : "+s"(at));
  return *(KernelParams*)at;
}
// A scalar that the compiler knows no origin of: it is neither read again in a loop, nor is what follows from it kept across one.
template <typename T>
__device__ __forceinline__ T keep_scalar(T x) {
  asm volatile("" : "+s"(x));
  return x;
}

// Sum over the lanes up to this one: within rows of 16 lanes, then over rows (no trip through LDS).
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_lane(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, true); }
__device__ __forceinline__ int wave_scan(int x) {
  x = add_lane<0x111, 0xf>(x);                                  // from the lane 1, 2, 4, 8 before
  x = add_lane<0x112, 0xf>(x);
  x = add_lane<0x114, 0xf>(x);
  x = add_lane<0x118, 0xf>(x);
  x = add_lane<0x142, 0xa>(x);                                  // lane 15 to the second row, 47 to the fourth
  return add_lane<0x143, 0xc>(x);                               // lane 31 to the third and fourth
}
// n / d for results below 2^12 and d up to 2^9, for d = 1, and for n up to 2^9: half a unit of n is more than the rounding of reciprocal and product.
__device__ __forceinline__ int small_div(int n, int d) { return static_cast<int>((static_cast<float>(n) + 0.5f) * __builtin_amdgcn_rcpf(static_cast<float>(d))); }

// A request's 16-row blocks in groups, alike: `per` blocks for each wave (at most `most`), with `halves` = 2 of other blocks for the second half of
// a workgroup's waves, which then share the units' bytes.
struct RowGroups {
  int groups, per, halves;
};
__device__ __forceinline__ RowGroups group_rows(int rows, int most, int halves) {
  const int blocks = (rows + 15) >> 4;
  RowGroups r;
  r.halves = blocks > most ? halves : 1;
  r.groups = r.halves == 2 ? (blocks + 2 * most - 1) / (2 * most) : (blocks + most - 1) / most;
  const float groups = static_cast<float>(max(r.groups, 1));    // (at most 8 blocks each: the quotient is exact)
  const int each = static_cast<int>((static_cast<float>(blocks) + groups - 0.5f) * __builtin_amdgcn_rcpf(groups));
  r.per = (each + r.halves - 1) / r.halves;
  return r;
}
// What a unit costs its workgroup by the 16-row blocks it is multiplied with, and what a group of rows costs besides (its start, its end and its share
// of merges: 10 to 15 us beside another workgroup's units, of which there are two in a microsecond).  300 + 60 blocks in place of it: 5 requests
// of 1001 to 15999 tokens, fp32 results, 29.7 -> 32.6 us, the serving batch of 64 alike.
__device__ __forceinline__ int unit_cost(int blocks) { return 24 + 4 * blocks; }
// Units are counted in chunks of 2^shift (0 unless the block table has room for so many that the batch's cost would pass 31 bits).
__device__ __forceinline__ int chunks_of(int units, int shift) { return (units + (1 << shift) - 1) >> shift; }
constexpr int kMostCost = 24 + 4 * kQaBlocks;
__device__ __forceinline__ int head_cost(int blocks) { return 600 + 150 * blocks; }
constexpr int kMostHead = 600 + 150 * kQaBlocks;
constexpr int kWholeCost = 456;               // a group whose units cost at most this (16 of few rows) is not cut: its merge would take longer
constexpr int kLeastRange = 256;              // ranges cost at least this, and
constexpr float kRangeRoot = 7.5f;            // this times the root of what a group costs (or as much as a group): n pieces of a group take a time of group / n
                                              // and their merge one of n (1 request of 16000 tokens x 8 KV heads: 27.1 -> 22.3 us)

// The requests, 64 at a time: lane i holds request 64 k + i.
struct Requests {
  int ctx, first, n;                            // of this lane's request
  int upto;                                     // cost up to its end, within these 64
  int sum, count;                               // cost of these 64, and their groups
};
__device__ __forceinline__ int units_of(KernelParams& P, int ctx, int n) {
  return n > 0 ? min(static_cast<int>((static_cast<unsigned>(ctx) + n + kUnit - 1) / kUnit), (P.max_pages >> 1) + (P.max_pages & 1)) : 0;
}
__device__ __forceinline__ Requests load_requests(KernelParams& P, int k, int most, int lane) {
  Requests r;
  const int b = 64 * k + lane;
  r.ctx = r.first = r.n = 0;
  if (b < P.B) {
    r.ctx = min(max(P.ctx_len[b], 0), 0x7fffff00);              // (the end of the drafts still fits)
    r.first = P.q_offsets[b];
    r.n = r.first < 0 ? 0 : max(min(min(P.q_offsets[b + 1], P.total_q) - r.first, P.max_q), 0);
  }
  const RowGroups g = group_rows(r.n * P.G, most, P.halves);
  r.upto = wave_scan(g.groups * (head_cost(g.per) + chunks_of(units_of(P, r.ctx, r.n), P.shift) * g.halves * unit_cost(g.per)));
  r.sum = __builtin_amdgcn_readlane(r.upto, 63);
  r.count = __builtin_amdgcn_readlane(wave_scan(g.groups), 63);
  return r;
}

// The batch's cost in `used` ranges: range s starts at the whole part of s * total / used, so that of alike groups, with as many ranges for each,
// every one starts a range.  each, more: total / used and the remainder.
struct Cut {
  int used, each, more;
};
__device__ __forceinline__ Cut cut_ranges(int most, int total, int count) {
  Cut c;
  const float group = static_cast<float>(total) / static_cast<float>(max(count, 1));
  const float least = fmaxf(kLeastRange, kRangeRoot * __builtin_amdgcn_sqrtf(group));
  c.used = min(max(max(static_cast<int>(static_cast<float>(total) / least), count), 1), most);
  const int alike = small_div(c.used, max(count, 1)) * max(count, 1);      // as many for each group
  if (4 * alike >= 3 * c.used) c.used = alike;
  c.used = __builtin_amdgcn_readfirstlane(c.used);              // (worked out in vector registers)
  c.each = total / c.used;
  c.more = total - c.each * c.used;
  return c;
}
__device__ __forceinline__ int range_start(const Cut& c, int s) { return s * c.each + __builtin_amdgcn_readfirstlane(small_div(s * c.more, keep_scalar(c.used))); }
__device__ __forceinline__ int range_of(const Cut& c, int at) {
  int s = at / (c.each + 1);                                    // at most two too low (ranges cost at least as much as there are)
  while (s + 1 < c.used && range_start(c, s + 1) <= at) ++s;
  return s;
}
// A group of a request's rows that starts at `start` has unit k at start + head + k * cost, or all of them at start + head if it is not cut; a unit
// belongs to the range that its place is in.  (Chunks, where units come in chunks.)  Ranges cost more than any unit: the pieces of a group lie in
// consecutive ranges.
struct Place {
  int start, head, units, cost, shift;          // cost: of a unit
};
__device__ __forceinline__ bool is_whole(const Place& p) { return chunks_of(p.units, p.shift) * p.cost <= kWholeCost; }
__device__ __forceinline__ int first_unit(const Place& p, int at) {           // at or behind `at`
  const int ahead = at - p.start - p.head;
  if (ahead <= 0) return 0;
  if (is_whole(p)) return p.units;
  return min((ahead + p.cost - 1) / p.cost, chunks_of(p.units, p.shift)) << p.shift;
}
// The pieces of a group that is cut: their first range and how many.
struct Pieces {
  int first, count;
};
__device__ __forceinline__ Pieces pieces_of(const Cut& c, const Place& p) {
  Pieces r;
  r.first = range_of(c, p.start + p.head);
  r.count = range_of(c, p.start + p.head + (chunks_of(p.units, p.shift) - 1) * p.cost) - r.first + 1;
  return r;
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

// The largest of three, NaN if one is: one instruction, where fmaxf first makes quiet NaN of each operand, one instruction apiece.
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }

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

__device__ __forceinline__ __attribute__((address_space(3))) raw4* lds_raw4(unsigned at) { return (__attribute__((address_space(3))) raw4*)at; }
typedef uint32_t raw2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ __attribute__((address_space(3))) raw2* lds_raw2(unsigned at) { return (__attribute__((address_space(3))) raw2*)at; }
__device__ __forceinline__ __attribute__((address_space(3))) float* lds_f32(unsigned at) { return (__attribute__((address_space(3))) float*)at; }
// At most N loads of this wave on their way.
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

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

template <int D_, int NW>
struct QuantAttnShared {
  static constexpr int D = D_, kWaves = NW, kThreads = NW * kWave;
  static constexpr int kStride = D + 4;                        // floats; padded row of the merge
  static constexpr int kPageBytes = kQuantPage * D;            // of K, or V, of a head
  static constexpr int kHalf = 2 * kPageBytes;                 // a unit's K, or V
  union {
    __align__(1024) unsigned char ring[NW][2][kHalf];          // K, V of a unit
    __align__(16) float o[NW][16][kStride];                    // the merge of the waves, when the units are done with
    struct {
      float m[kMergeRoom], l[kMergeRoom];
    } merge;                                                   // ... of the pieces
  };
  __align__(16) raw4 q[2 * kQaBlocks * 2 * (D / 64)][kWave];   // query operands: [half, block, step][lane]
  float scales[NW][kWave];                                     // of a unit's pages: lane i: page i / 2 % 2, K or V i % 2
  unsigned long long anc[kQaMaxNodes][2];
  int parent[kQaMaxNodes];
  int nans;                                                    // a draft's value is NaN
  int last;                                                    // this workgroup finished its request's last piece
  int64_t row[32 * kQaBlocks];                                 // of q and out, of the piece's query rows
  int node[32 * kQaBlocks];
  float top[32 * kQaBlocks], inv[32 * kQaBlocks];              // a row's maximum, and 1 / the sum of its weights
  float m[NW][16 * kQaBlocks], l[NW][16 * kQaBlocks];
};

// One piece of a request: units [t0, t1) of it, for the query rows [row_base, row_base + rows) of a KV head.
struct QuantPiece {
  int b, first, n, ctx, kvh, t0, t1, row_base, rows, halves;
  bool whole;                 // the piece is all of these rows: write the result
  int64_t part;               // else: first row of its partial result
  unsigned long long* word;   // ... and the word that counts the pieces
};

// Query row r of a KV head is head r % G of node r / G (fewer than 2^17 rows, G up to 2^10: exact).
__device__ __forceinline__ int node_of(KernelParams& P, int row) { return static_cast<int>(__umulhi(2u * row, P.inverse_G)); }
__device__ __forceinline__ int64_t query_row(KernelParams& P, const QuantPiece& J, int row) {
  const int node = node_of(P, row);
  return static_cast<int64_t>(J.first + node) * P.Hq + J.kvh * P.G + (row - node * P.G);
}

// The piece's query rows: their nodes, and where they lie in q and out (rows past the last repeat it).
template <typename Sh>
__device__ __forceinline__ void find_rows(KernelParams& P, Sh& S, const QuantPiece& J, int i) {
  if (i >= 32 * kQaBlocks) return;
  const int row = J.row_base + min(i, J.rows - 1);
  S.node[i] = node_of(P, row);
  S.row[i] = query_row(P, J, row);
}

// Dimensions d0 and d0 + 1 of a row's result are NaN where a value is that the row sees, among the units that reach the drafts (of the others
// every row sees every token, and the products are NaN by themselves).
template <typename Sh>
__device__ __forceinline__ void put_back_nans(KernelParams& P, const Sh& S, const QuantPiece& J, int row, int d0, float& lo, float& hi) {
  constexpr int D = Sh::D;
  const int node = S.node[row];
  const int end = min(J.t1 * kUnit, J.ctx + J.n);
  for (int tok = max(J.t0 * kUnit, J.ctx & ~(kUnit - 1)); tok < end; ++tok) {
    const int j = tok - J.ctx, lp = tok / kQuantPage;
    if (j >= 0 && !((S.anc[node][j >> 6] >> (j & 63)) & 1ull)) continue;
    const int id = lp < P.max_pages ? P.block_table[static_cast<int64_t>(J.b) * P.max_pages + lp] : -1;
    if (id < 0 || id >= P.num_pages) continue;
    const unsigned char* v = P.v_pool + (static_cast<int64_t>(id) * P.Hkv + J.kvh) * (kQuantPage * D) + d0 * kQuantPage + tok % kQuantPage;
    const float nan = __builtin_nanf("");
    if ((v[0] & 0x7f) == 0x7f) lo = nan;
    if ((v[kQuantPage] & 0x7f) == 0x7f) hi = nan;
  }
}

__device__ __forceinline__ unsigned long long pair_bits(float lo, float hi) {
  return static_cast<unsigned long long>(__float_as_uint(hi)) << 32 | __float_as_uint(lo);
}

// Dimensions 4 d4 .. + 3 of a row's result.
template <int D>
__device__ __forceinline__ void put_result(KernelParams& P, int64_t at, int d4, float4 x) {
  if (P.out_f32) {
    reinterpret_cast<float4*>(static_cast<float*>(P.out) + at * D)[d4] = x;
  } else {
    const qbf16x2 lo = {static_cast<__bf16>(x.x), static_cast<__bf16>(x.y)}, hi = {static_cast<__bf16>(x.z), static_cast<__bf16>(x.w)};
    reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out) + at * D)[d4] = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
  }
}
// ... and its log-sum-exp (nothing seen: -infinity) from the maximum in log2 units and the sum.
__device__ __forceinline__ void put_lse(KernelParams& P, int64_t at, float M, float Z) {
  if (P.lse) P.lse[at] = (M + log2f(Z)) * static_cast<float>(kLn2);
}
// What a row's results are multiplied with: 1 / its sum of weights (0: it sees nothing, and gives 0).
__device__ __forceinline__ float inverse_sum(float Z) { return Z == 0.f ? 0.f : 1.f / Z; }

// The pieces of a request count themselves in a word {count : the call's tag}.  What an earlier call left there is first replaced by a count
// of none: one attempt, since only another piece of this call can have been quicker.  (Counting by compare-and-swap alone, pieces that finish
// together wait for each other, 1.2 us apiece.)  Thread 0; seen: the word as it was before.
__device__ __forceinline__ void open_count(unsigned long long* word, unsigned long long seen, unsigned long long tag) {
  if (!have_tag<1>(&seen, tag))
    __hip_atomic_compare_exchange_strong(word, &seen, tag, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Counts this workgroup's piece as done; true in all threads of the workgroup that finishes the last of `pieces`.
__device__ __forceinline__ bool last_piece(unsigned long long* word, int pieces, int* last) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");              // this wave's partial results have arrived
  __syncthreads();
  if (threadIdx.x == 0) {
    const unsigned long long before = __hip_atomic_fetch_add(word, 1ull << kTagBits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *last = static_cast<int>(before >> kTagBits) + 1 == pieces;
  }
  __syncthreads();
  return *last != 0;
}

// Merges the partial results of a request's pieces, in their order; `pair`: the KV head's first range.
template <typename Sh>
__device__ __forceinline__ void merge_pieces(Sh& S, const QuantPiece& J, int64_t pair, const Pieces& all) {
  KernelParams& P = kernel_params();
  constexpr int D = Sh::D, kThreads = Sh::kThreads;
  const int tid = threadIdx.x;
  const int pieces = all.count;
  auto part = [&](int i) { return ((pair + all.first + i) * 2 + (i == 0 ? 1 : 0)) * P.rows; };
  const int chunk = min(J.rows, max(1, kMergeRoom / pieces));
  for (int r0 = 0; r0 < J.rows; r0 += chunk) {
    const int rows = min(chunk, J.rows - r0);
    lds_sync();
    for (int at = tid; at < rows * pieces; at += kThreads) {
      const unsigned long long w = ld_dev(reinterpret_cast<const unsigned long long*>(P.ws_ml + part(at / rows) + r0 + at % rows));
      S.merge.m[at] = __uint_as_float(static_cast<unsigned>(w));
      S.merge.l[at] = __uint_as_float(static_cast<unsigned>(w >> 32));
    }
    lds_sync();
    for (int r = tid; r < rows; r += kThreads) {
      float M = -INFINITY, Z = 0.f;
      for (int i = 0; i < pieces; ++i) M = fmaxf(M, S.merge.m[i * rows + r]);
      for (int i = 0; i < pieces; ++i) {
        const float m = S.merge.m[i * rows + r];
        const float share = m == -INFINITY ? 0.f : S.merge.l[i * rows + r] * fast_exp2(m - M);
        Z += share;
        S.merge.m[i * rows + r] = share;
      }
      put_lse(P, S.row[r0 + r], M, Z);
      S.inv[r] = inverse_sum(Z);
    }
    lds_sync();
    // four dimensions of kRows rows at a time, of kFly pieces: as many loads on their way for few pieces of many rows as for many of few
    auto combine = [&](auto rows_at_once, auto fly) __attribute__((always_inline)) {
      constexpr int kRows = decltype(rows_at_once)::value, kFly = decltype(fly)::value, kApart = kThreads / (D / 4);
      const int d4 = tid % (D / 4);
      for (int r1 = tid / (D / 4); r1 < rows; r1 += kRows * kApart) {
        float4 sum[kRows];
        float inv[kRows];
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
          sum[j] = make_float4(0.f, 0.f, 0.f, 0.f);
          inv[j] = S.inv[min(r1 + j * kApart, rows - 1)];
        }
        for (int i0 = 0; i0 < pieces; i0 += kFly) {
          unsigned long long x[kFly][kRows][2];
#pragma unroll
          for (int k = 0; k < kFly; ++k)
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
              const unsigned long long* from = reinterpret_cast<const unsigned long long*>(
                  P.ws_o + (part(min(i0 + k, pieces - 1)) + r0 + min(r1 + j * kApart, rows - 1)) * D) + 2 * d4;
              x[k][j][0] = ld_dev(from);
              x[k][j][1] = ld_dev(from + 1);
            }
#pragma unroll
          for (int k = 0; k < kFly; ++k) {
            if (i0 + k >= pieces) break;
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
              const float f = S.merge.m[(i0 + k) * rows + min(r1 + j * kApart, rows - 1)] * inv[j];
              sum[j].x += __uint_as_float(static_cast<unsigned>(x[k][j][0])) * f;
              sum[j].y += __uint_as_float(static_cast<unsigned>(x[k][j][0] >> 32)) * f;
              sum[j].z += __uint_as_float(static_cast<unsigned>(x[k][j][1])) * f;
              sum[j].w += __uint_as_float(static_cast<unsigned>(x[k][j][1] >> 32)) * f;
            }
          }
        }
#pragma unroll
        for (int j = 0; j < kRows; ++j)
          if (r1 + j * kApart < rows) put_result<D>(P, S.row[r0 + r1 + j * kApart], d4, sum[j]);
      }
    };
    if (rows > kThreads / (D / 4)) combine(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
    else combine(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
  }
}

// SANITIZE: NaN among the drafts' values are taken out of the products (where a row does not see a draft its weight is zero, and zero times
// NaN would be NaN) and put back into the results of the rows that see them.  Without, a piece that meets one writes nothing and
// says so in S.nans.
template <int NB, int TERMS, bool SANITIZE, typename Sh>
__device__ __forceinline__ void quant_piece(Sh& S, const QuantPiece& J) {
  KernelParams& P = kernel_params();
  constexpr int D = Sh::D, kWaves = Sh::kWaves;
  constexpr int kH = D / 64;                                   // K: 16-byte chunks of a lane per token
  constexpr int kDT = D / 16;                                  // 16-dimension tiles of the output
  constexpr int kLoads = D / 64;                               // 1 KB loads per page of K or V
  const int tid = static_cast<int>(threadIdx.x) + opaque_zero(), lane = tid & 63;
  __builtin_assume(tid >= 0 && tid < Sh::kThreads);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rn = lane & 15, g = lane >> 4;                     // query row of the block (matrix column), lane group
  const int L = J.ctx + J.n;
  const bool touches_drafts = J.t1 * kUnit > J.ctx;

  // ---- a unit's loads: page ids through the scalar cache, a page of a head is contiguous; lane i brings bytes 16 i .. + 16 of each 1 KB ----
  const int64_t page_bytes = static_cast<int64_t>(P.Hkv) * Sh::kPageBytes;
  const unsigned char* k_head = P.k_pool + static_cast<int64_t>(J.kvh) * Sh::kPageBytes;
  const unsigned char* v_head = P.v_pool + static_cast<int64_t>(J.kvh) * Sh::kPageBytes;
  const const_i32* bt = (const const_i32*)(P.block_table + static_cast<int64_t>(J.b) * P.max_pages);
  const int num_pages = keep_scalar(P.num_pages), max_pages = keep_scalar(P.max_pages), Hkv = keep_scalar(P.Hkv);
  const float* const k_scale = keep_scalar(P.k_scale) + J.kvh;
  const float* const v_scale = keep_scalar(P.v_scale) + J.kvh;
  const float c = keep_scalar(P.c);
  const int last_page = min((L - 1) / kQuantPage, max_pages - 1);
  int k_id0 = 0, k_id1 = 0, v_id0 = 0, v_id1 = 0;               // of the units whose K and V go out next; -1: no page of the pool
  auto fetch_ids = [&](int t) __attribute__((always_inline)) {
    if (t < J.t1) {
      k_id0 = bt[min(2 * t, last_page)];
      k_id1 = bt[min(2 * t + 1, last_page)];
      k_id0 = k_id0 >= 0 && k_id0 < num_pages && 2 * t < max_pages ? k_id0 : -1;
      k_id1 = k_id1 >= 0 && k_id1 < num_pages && 2 * t + 1 < max_pages ? k_id1 : -1;
    }
  };
  const unsigned ring = lds_address(&S.ring[wave][0][0]), scales = lds_address(reinterpret_cast<unsigned char*>(&S.scales[wave][0]));
  auto issue_k = [&](unsigned to) __attribute__((always_inline)) {
    const unsigned char* a = k_head + max(k_id0, 0) * page_bytes;
    const unsigned char* b = k_head + max(k_id1, 0) * page_bytes;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load_to_lds(a, 16 * lane, to, j);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load_to_lds(b, 16 * (lane ^ 4), to + Sh::kPageBytes, j);   // (see k_at)
  };
  auto issue_v = [&] __attribute__((always_inline)) {
    const unsigned char* a = v_head + max(v_id0, 0) * page_bytes;
    const unsigned char* b = v_head + max(v_id1, 0) * page_bytes;
    // a page that is none of the pool's holds nothing: its scale reads as 0, what is read instead is page 0
    const int id = lane & 2 ? v_id1 : v_id0;
    const float* at = (lane & 1 ? v_scale : k_scale) + static_cast<int64_t>(id) * Hkv;
    at = id >= 0 ? at : kNoScale;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load_to_lds(a, 16 * lane, ring + Sh::kHalf, j);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load_to_lds(b, 16 * lane, ring + Sh::kHalf + Sh::kPageBytes, j);
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" :: "{m0}"(scales), "v"(at) : "memory");
  };
  constexpr int kKLoads = 2 * kLoads, kVLoads = 2 * kLoads + 1;

  const bool split = !SANITIZE && J.halves == 2;
  const int per_half = split ? kWaves / 2 : kWaves, half = split ? wave / (kWaves / 2) : 0, row0 = 16 * NB * half;    // waves; this wave's half, its first row
  int t = J.t0 + wave - half * per_half;
  const int mine = t < J.t1 ? (J.t1 - t + per_half - 1) >> (split ? ilog2(kWaves / 2) : ilog2(kWaves)) : 0;  // units of this wave

  // ---- all that the piece needs besides its pages is on its way at once, and its first pages behind it ----
  // query operands: step 2 h + e, lane group g: dimensions 16 (4 h + g) + 8 e .. + 8 (what a lane's 16 bytes of K hold)
  constexpr int kMine = (2 * NB * 2 * kH + kWaves - 1) / kWaves;
  const int frags = (split ? 2 : 1) * NB * 2 * kH;
  raw4 qv[kMine];
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    if (wave + j * kWaves >= frags) break;
    const int f = wave + j * kWaves, s = f % (2 * kH), row = J.row_base + min(16 * (f / (2 * kH)) + rn, J.rows - 1);    // (columns past the last row repeat it)
    qv[j] = *reinterpret_cast<const raw4*>(P.q + query_row(P, J, row) * D + 16 * g + 64 * (s >> 1) + 8 * (s & 1));
  }
  int parent = -1;
  if (touches_drafts && P.parent && tid < J.n) parent = P.parent[J.first + tid];
  if (mine > 0) fetch_ids(t);
  lds_sync();                                                   // the LDS of the piece before is free
  if (mine > 0) {
    issue_k(ring);
    v_id0 = k_id0; v_id1 = k_id1;
    issue_v();
    fetch_ids(t + per_half);
  }
  if (!SANITIZE && tid == 0) S.nans = 0;
  find_rows(P, S, J, tid);
#pragma unroll
  for (int j = 0; j < kMine; ++j)
    if (wave + j * kWaves < frags) S.q[wave + j * kWaves][lane] = qv[j];
  if (tid < J.n) S.parent[tid] = parent;
  if (touches_drafts) {
    lds_sync();
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
  }
  lds_sync();

  // Operand reads.  K, lane group g: chunk 4 h + g; lane: page rn / 8, token 8 (rn / 4 % 2) + 4 st + rn % 4.  The second page lies with tokens
  // 4 i .. + 3 and their neighbours 4 (i ^ 1) .. exchanged: 16 lanes take their 256 bytes from as many banks.
  const unsigned k_at = ring + (rn >> 3) * Sh::kPageBytes + g * 256 + (8 * ((rn >> 2) & 1) + (rn & 3)) * 16;
  const unsigned k_flip = 64 * (rn >> 3);                       // sub-tile st at k_at + (64 st ^ k_flip)
  const unsigned v_at = ring + Sh::kHalf + (g >> 1) * Sh::kPageBytes + rn * 16 + 8 * (g & 1);
  const unsigned s_at = scales + 8 * (g >> 1);
  const raw4* q_mine = &S.q[half * NB * 2 * kH][lane];

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

  for (int i = 0; i < mine; ++i, t += per_half) {
    const int behind = mine - 1 - i;                            // units of this wave after this one
    // K of this unit is here: behind it the next one's K, and V
    wait_loads<kVLoads>();
    // ---- scores: K at once, the queries' operands a step ahead of the products (four blocks: of the first two, registers are short) ----
    constexpr int kAhead = NB < 4 ? NB : 2;
    qf32x4 s[NB][2];
    raw4 kr[kH][2], qr[2][NB];
#pragma unroll
    for (int h = 0; h < kH; ++h) {
      kr[h][0] = *lds_raw4(k_at + (0u ^ k_flip) + 1024 * h);
      kr[h][1] = *lds_raw4(k_at + (64u ^ k_flip) + 1024 * h);
    }
#pragma unroll
    for (int qi = 0; qi < kAhead; ++qi) qr[0][qi] = q_mine[qi * 2 * kH * kWave];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // K has been read
    if (behind > 0) issue_k(ring);
    __builtin_amdgcn_s_setprio(1);                              // products before another wave's softmax
#pragma unroll
    for (int step = 0; step < 2 * kH; ++step) {
      const int h = step >> 1, e = step & 1;
      if (step + 1 < 2 * kH) {
#pragma unroll
        for (int qi = 0; qi < kAhead; ++qi) qr[(step + 1) & 1][qi] = q_mine[(qi * 2 * kH + step + 1) * kWave];
      }
#pragma unroll
      for (int qi = kAhead; qi < NB; ++qi) qr[step & 1][qi] = q_mine[(qi * 2 * kH + step) * kWave];
      const qbf16x8 a0 = operand_bf16(kr[h][0][2 * e], kr[h][0][2 * e + 1]), a1 = operand_bf16(kr[h][1][2 * e], kr[h][1][2 * e + 1]);
#pragma unroll
      for (int qi = 0; qi < NB; ++qi) {
        const qbf16x8 q = __builtin_bit_cast(qbf16x8, qr[step & 1][qi]);
        const qf32x4 zero = {0.f, 0.f, 0.f, 0.f};
        s[qi][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, q, step == 0 ? zero : s[qi][0], 0, 0, 0);
        s[qi][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, q, step == 0 ? zero : s[qi][1], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    // V of this unit and its scales are here: behind them the K after next
    if (behind > 0) wait_loads<kKLoads>();
    else wait_loads<0>();
    const float ks = *lds_f32(s_at), v_own = *lds_f32(s_at + 4);
    raw2 vr[kDT];
#pragma unroll
    for (int d = 0; d < kDT; ++d) vr[d] = *lds_raw2(v_at + 256 * d);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // V has been read
    if (behind > 0) {
      v_id0 = k_id0; v_id1 = k_id1;
      issue_v();
      fetch_ids(t + 2 * per_half);
    }
    const bool ok = ks != 0.f;
    const float factor = fmaxf(ks * c, 0x1p-126f);              // (not 0: masked scores are -infinity)

    // ---- masks: only where the unit reaches the drafts, or a page is none ----
    const int past = t * kUnit + 16 * (g >> 1) - J.ctx;         // the lane's page starts that far behind the context
    const bool drafts = (t + 1) * kUnit > J.ctx, masked = any_lane(!ok) || drafts;
    if (masked) {
#pragma unroll
      for (int qi = 0; qi < NB; ++qi) {
        uint32_t seen = 0xffffu;
        if (past > -16) {
          const int node = S.node[row0 + 16 * qi + rn];
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
      top[qi] = max3(max3(s[qi][0][0], s[qi][0][1], s[qi][0][2]), max3(s[qi][0][3], s[qi][1][0], s[qi][1][1]),
                     __builtin_elementwise_maximum(s[qi][1][2], s[qi][1][3])) * factor;                   // factor >= 0
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
    // fp16 has room for it, down to kLeastWeight (further down, weights would leave the range of fp32 too, and be missing from their sum).
    asm volatile("" : "+v"(v_ref));      // (its inverse worked out on both sides of the branch makes it one with an else part, whose copies cost the
                                         // registers of all results a second time)
    const float ratio = v_own * inverse_scale(v_ref), v_by = fmaxf(ratio, kLeastV), p_by = ok ? fmaxf(ratio * inverse_scale(v_by), kLeastWeight) : 1.f;
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
      keep[0] = spread4((1u << valid) - 1u);
      keep[1] = spread4(((1u << valid) - 1u) >> 4);
      if (!SANITIZE && drafts) {
        uint32_t nans = 0u;
#pragma unroll
        for (int d = 0; d < kDT; ++d) nans |= nan_bytes(vr[d].x & keep[0]) | nan_bytes(vr[d].y & keep[1]);
        if (any_lane(nans != 0u) && lane == 0) S.nans = 1;
      }
    }
    __builtin_amdgcn_s_setprio(1);
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
    __builtin_amdgcn_s_setprio(0);
  }

  const unsigned long long count_seen = SANITIZE || J.whole || tid > 0 ? 0ull : ld_dev(J.word);     // (arrives while the waves merge)

  // ---- merge the waves, one block at a time ----
#pragma unroll
  for (int qi = 0; qi < NB; ++qi) {
    sum[qi] = groups_sum(sum[qi]) * (1.f / (1 << kWeightBias));
    if (sum[qi] == 0.f) ref[qi] = -INFINITY;                    // nothing seen
    if (lane < 16) {
      S.m[wave][16 * qi + lane] = ref[qi];
      S.l[wave][16 * qi + lane] = sum[qi];
    }
  }
  lds_sync();                                              // (the rings are done with, too)
  if constexpr (!SANITIZE) {
    if (S.nans) {
      if (!J.whole && tid == 0) open_count(J.word, count_seen, P.tag);
      return;
    }
  }
  const int halves = SANITIZE ? 1 : keep_scalar(J.halves);
  if (tid < 16 * NB * halves) {
    const int w0 = tid < 16 * NB ? 0 : kWaves / 2, local = tid < 16 * NB ? tid : tid - 16 * NB;
    float M = -INFINITY, Z = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (w < kWaves / 2 || !split) M = fmaxf(M, S.m[w0 + w][local]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (w < kWaves / 2 || !split) Z += S.m[w0 + w][local] == -INFINITY ? 0.f : S.l[w0 + w][local] * fast_exp2(S.m[w0 + w][local] - M);
    S.top[tid] = M;
    S.inv[tid] = inverse_sum(Z);
    if (tid < J.rows) {
      if (J.whole) put_lse(P, S.row[tid], M, Z);
      else st_dev(reinterpret_cast<unsigned long long*>(P.ws_ml + J.part + tid), pair_bits(M, Z));
    }
  }
  lds_sync();
#pragma unroll
  for (int qi = 0; qi < NB; ++qi) {
    if (qi > 0) lds_sync();
    // (divided by the sum of weights first: results are no larger than the values then, which may be near the end of fp32's range)
    const int row = row0 + 16 * qi + rn;
    const float f = ref[qi] == -INFINITY ? 0.f : fast_exp2(ref[qi] - S.top[row] - static_cast<float>(kWeightBias)) * S.inv[row] * v_ref;
#pragma unroll
    for (int d = 0; d < kDT; ++d)
      *reinterpret_cast<float4*>(&S.o[wave][rn][16 * d + 4 * g]) =
          make_float4(oacc[qi][d][0] * f, oacc[qi][d][1] * f, oacc[qi][d][2] * f, oacc[qi][d][3] * f);
    lds_sync();
#pragma unroll 2
    for (int at = tid; at < 16 * (D / 4) * halves; at += Sh::kThreads) {      // four dimensions of a row
      const int d4 = at % (D / 4), r = at / (D / 4) % 16, other = at / (16 * (D / 4)), row = 16 * (NB * other + qi) + r;
      if (row >= J.rows) continue;
      float4 x[kWaves], sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        if (w < kWaves / 2 || !split) x[w] = *reinterpret_cast<const float4*>(&S.o[other * (kWaves / 2) + w][r][4 * d4]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        if (w >= kWaves / 2 && split) break;
        sum.x += x[w].x; sum.y += x[w].y; sum.z += x[w].z; sum.w += x[w].w;
      }
      if constexpr (SANITIZE) {
        put_back_nans(P, S, J, row, 4 * d4, sum.x, sum.y);
        put_back_nans(P, S, J, row, 4 * d4 + 2, sum.z, sum.w);
      }
      if (J.whole) {
        put_result<D>(P, S.row[row], d4, sum);
      } else {
        // read by another workgroup of this launch: device-scope stores
        unsigned long long* to = reinterpret_cast<unsigned long long*>(P.ws_o + (J.part + row) * D) + 2 * d4;
        st_dev(to, pair_bits(sum.x, sum.y));
        st_dev(to + 1, pair_bits(sum.z, sum.w));
      }
    }
  }
  if (!SANITIZE && !J.whole && tid == 0) open_count(J.word, count_seen, P.tag);
}

// TERMS: fp16 terms of a weight.
template <int D, int TERMS, int NW>
__global__ __launch_bounds__(NW * kWave, 2) void attn_quant_kernel(QuantAttnParams) {
  KernelParams& P = kernel_params();
  constexpr int kMost = most_blocks(D, TERMS);
  extern __shared__ __align__(1024) unsigned char smem[];
  auto& S = *reinterpret_cast<QuantAttnShared<D, NW>*>(smem);
  const int lane = threadIdx.x & 63;
  QuantPiece J;
  const int batches = (P.B + 63) / 64;
  int total = 0, count = 0;
  Requests r;
  for (int k = batches - 1; k >= 0; --k) {                      // (down: the first 64 requests stay in registers)
    r = load_requests(P, k, kMost, lane);
    total += r.sum;
    count += r.count;
  }
  const Cut cut = cut_ranges(P.ranges, total, count);
  // Workgroups go to the 8 XCDs in turn: renumbered so that neighbouring ranges, which may hold groups of rows of one request, share an L2, with as
  // many in each
  const int all = cut.used * P.Hkv, each = (all + 7) >> 3, xcd = blockIdx.x & 7, place = blockIdx.x >> 3, logical = xcd * each + place;
  if (place >= each || logical >= all) return;
  J.kvh = __builtin_amdgcn_readfirstlane(small_div(logical, cut.used));
  const int range = logical - J.kvh * cut.used;
  const int64_t pair = static_cast<int64_t>(J.kvh) * P.ranges;
  const int from = range_start(cut, range), end = range_start(cut, range + 1);
  int base = 0;                                                 // cost before these 64 requests
  for (int k = 0, at = from; at < end;) {
    const unsigned long long later = __builtin_amdgcn_ballot_w64(base + r.upto > at);
    if (later == 0ull) {
      base += r.sum;
      if (++k >= batches) break;
      r = load_requests(P, k, kMost, lane);
      continue;
    }
    const int i = __ffsll(later) - 1;
    J.b = 64 * k + i;
    J.ctx = __builtin_amdgcn_readlane(r.ctx, i);
    J.first = __builtin_amdgcn_readlane(r.first, i);
    J.n = __builtin_amdgcn_readlane(r.n, i);
    const RowGroups g = group_rows(J.n * P.G, kMost, P.halves);
    const int groups = __builtin_amdgcn_readfirstlane(g.groups), per = __builtin_amdgcn_readfirstlane(g.per);
    J.halves = __builtin_amdgcn_readfirstlane(g.halves);
    Place p;
    p.units = units_of(P, J.ctx, J.n);
    p.cost = J.halves * unit_cost(per);
    p.shift = P.shift;
    p.head = head_cost(per);
    const int behind = base + __builtin_amdgcn_readlane(r.upto, i), group_cost = p.head + chunks_of(p.units, p.shift) * p.cost;
    p.start = behind - groups * group_cost;
    for (int grp = 0; grp < groups && p.start < end; ++grp, p.start += group_cost) {
      J.t0 = first_unit(p, from);
      J.t1 = min(p.units, first_unit(p, end));
      if (J.t0 >= J.t1) continue;
      J.row_base = 16 * per * J.halves * grp;
      J.rows = min(J.n * P.G - J.row_base, 16 * per * J.halves);
      J.whole = J.t0 == 0 && J.t1 == p.units;
      J.part = ((pair + range) * 2 + (J.t0 == 0 ? 1 : 0)) * P.rows;
      J.word = P.arrived + (static_cast<int64_t>(J.kvh) * P.groups + grp) * P.B + J.b;
      switch (per) {
        case 1: quant_piece<1, TERMS, false>(S, J); break;
        case 2: quant_piece<2, TERMS, false>(S, J); break;
        case 3: quant_piece<3, TERMS, false>(S, J); break;
        default:
          if constexpr (kMost >= 4) quant_piece<4, TERMS, false>(S, J);
      }
      if (S.nans) {                                             // (written before a barrier, and next behind one)
        QuantPiece part = J;
        part.halves = 1;
        for (int row = 0; row < J.rows; row += 16) {
          part.row_base = J.row_base + row;
          part.rows = min(J.rows - row, 16);
          part.part = J.part + row;
          quant_piece<1, TERMS, true>(S, part);
        }
        __syncthreads();
        find_rows(P, S, J, threadIdx.x);                        // (of all rows again, for the merge)
      }
      if (!J.whole) {
        const Pieces all_pieces = pieces_of(cut, p);
        if (last_piece(J.word, all_pieces.count, &S.last)) merge_pieces(S, J, pair, all_pieces);
      }
    }
    at = behind;
  }
}

// ---- host ----------------------------------------------------------------------------------------------------
QuantAttnPlan make_quant_attn_plan(const AttnArgs& a) {
  QuantAttnPlan p{};
  const int64_t rows = static_cast<int64_t>(a.max_q) * (a.Hq / a.Hkv);
  const int blocks = static_cast<int>(std::max<int64_t>(1, (rows + 15) / 16));
  // Rows that are too many for a wave go to two halves of a workgroup where groups in workgroups of their own would be twice as many as those: they
  // then read the same pages one after the other (64 requests x 8 KV heads x 2048 tokens, 128 rows: 119 us, in halves 97; 80 rows: 110, 79); with a
  // workgroup for each group, side by side, halves gain nothing and cut more (16 requests x 8 KV heads x 4096 tokens, 256 rows: 89 us, 92).
  int most = most_blocks(a.D, a.out_dtype == kF32 ? 2 : 1);
  p.groups = (blocks + most - 1) / most;
  p.halves = p.groups > 1 && static_cast<int64_t>(a.Hkv) * a.B * p.groups >= 1024 ? 2 : 1;
  most *= p.halves;
  p.groups = (blocks + most - 1) / most;
  p.rows = 16 * std::min(blocks + p.halves - 1, most);
  // Two workgroups of four waves to a compute unit overlap the starts and ends of their pieces, where there are two pieces for it; else one of eight, whose
  // waves share one (1 request of 16000 tokens x 8 KV heads, single tokens: 23.2 us with four, 21.6 with eight; 16 of 2000: 23.2, 24.0; 64 of 2048:
  // 57, 61; 256 of 512: 68, 89).
  p.waves = static_cast<int64_t>(a.Hkv) * a.B * p.groups < 512 ? 8 : 4;
  p.ranges = std::max(1, (p.waves == 8 ? 256 : 512) / a.Hkv);
  // the cost of the batch stays below 2^31 (no chunk is long enough where there are millions of groups: shift is then 30 and the call is refused)
  const int64_t groups = static_cast<int64_t>(a.B) * p.groups;
  const int64_t units = (static_cast<int64_t>(a.max_pages) + 1) / 2;
  while (p.shift < kQuantMaxShift && groups * (kMostHead + ((units >> p.shift) + 1) * p.halves * kMostCost) >= (int64_t{1} << 31)) ++p.shift;
  return p;
}

// Partial results, their statistics, and the words that count a request's pieces.
static size_t quant_rows(const AttnArgs& a, const QuantAttnPlan& p) { return static_cast<size_t>(a.Hkv) * p.ranges * 2 * p.rows; }
static size_t quant_words(const AttnArgs& a, const QuantAttnPlan& p) { return static_cast<size_t>(a.Hkv) * p.groups * a.B; }
size_t quant_attn_workspace_bytes(const AttnArgs& a, const QuantAttnPlan& p) {
  if (p.ranges == 1) return 0;                                  // one range per KV head: nothing is cut
  return quant_rows(a, p) * (static_cast<size_t>(a.D) * sizeof(float) + sizeof(float2)) + quant_words(a, p) * sizeof(unsigned long long);
}

template <int D, int TERMS, int NW>
static int launch_quant(const QuantAttnParams& P, const AttnArgs& a, const QuantAttnPlan& p, hipStream_t stream) {
  static std::atomic<uint64_t> lds_set{0};
  constexpr size_t lds = sizeof(QuantAttnShared<D, NW>);
  static_assert(lds <= (NW == 8 ? 160 : 80) * 1024, "two workgroups of four waves, or one of eight, to a compute unit");
  if (lds > 65536 && set_lds_once(attn_quant_kernel<D, TERMS, NW>, lds, lds_set) != 0) return -6;
  hipLaunchKernelGGL((attn_quant_kernel<D, TERMS, NW>), dim3((p.ranges * a.Hkv + 7) / 8 * 8), dim3(NW * kWave), lds, stream, P);
  return 0;
}
template <int D, int TERMS>
static int launch_quant_waves(const QuantAttnParams& P, const AttnArgs& a, const QuantAttnPlan& p, hipStream_t stream) {
  return p.waves == 8 ? launch_quant<D, TERMS, 8>(P, a, p, stream) : launch_quant<D, TERMS, 4>(P, a, p, stream);
}

int launch_attn_quant(const AttnArgs& a, const float* k_scale, const float* v_scale, int num_pages, const QuantAttnPlan& p, hipStream_t stream) {
  QuantAttnParams P{};
  P.q = static_cast<const uint16_t*>(a.q); P.k_pool = static_cast<const unsigned char*>(a.k_pool);
  P.v_pool = static_cast<const unsigned char*>(a.v_pool); P.k_scale = k_scale; P.v_scale = v_scale;
  P.block_table = a.block_table; P.ctx_len = a.ctx_len; P.q_offsets = a.q_offsets; P.parent = a.parent;
  P.out = a.out; P.lse = a.lse;
  P.ws_o = static_cast<float*>(a.workspace);
  P.ws_ml = reinterpret_cast<float2*>(P.ws_o + quant_rows(a, p) * a.D);
  if (p.ranges > 1) {
    P.arrived = reinterpret_cast<unsigned long long*>(P.ws_ml + quant_rows(a, p));
    const MessageTag t = next_message_tag(false, stream);
    if (t.clear) clear_messages(P.arrived, static_cast<int64_t>(quant_words(a, p)), stream);
    P.tag = t.tag;
  }
  P.B = a.B; P.Hq = a.Hq; P.Hkv = a.Hkv; P.G = a.Hq / a.Hkv; P.inverse_G = ((1u << 31) + P.G - 1) / P.G; P.total_q = a.total_q; P.max_q = std::min(a.max_q, kQaMaxNodes);
  P.max_pages = a.max_pages; P.num_pages = num_pages;
  P.ranges = p.ranges; P.groups = p.groups; P.rows = p.rows; P.halves = p.halves; P.shift = p.shift;
  P.c = a.scale * kLog2e; P.out_f32 = a.out_dtype == kF32;
  if (a.D == 128) return P.out_f32 ? launch_quant_waves<128, 2>(P, a, p, stream) : launch_quant_waves<128, 1>(P, a, p, stream);
  return P.out_f32 ? launch_quant_waves<64, 2>(P, a, p, stream) : launch_quant_waves<64, 1>(P, a, p, stream);
}

}  // namespace specv
