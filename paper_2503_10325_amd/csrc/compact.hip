// Accepted-path compaction of the paged KV cache after a draft tree has been verified.  The paper
// only says that verified drafts go back to the request pool (Section 4.1); for the next step to see
// an ordinary linear context, the K/V entries of the accepted path (root .. stop node, draft node j
// living at logical position ctx + j) move to positions ctx + 0 .. ctx + depth - 1.
//
// One workgroup per (request, KV head): the path is rebuilt from the parent array, every source row
// (K and V, D 16-bit elements) is read into registers, a barrier, then the rows are written to their
// destinations - destinations of one depth can be sources of another, so nothing is written before
// everything is read.  Pure data movement: at most 128 rows of 2*D bytes per tensor, latency-bound.
#include "common.h"
#include "kernels.h"
#include "quant.h"

namespace specv {

constexpr int kCompactThreads = 256;
constexpr int kCompactMaxNodes = 128;

typedef uint32_t cu32x4 __attribute__((ext_vector_type(4)));

__global__ __launch_bounds__(kCompactThreads) void compact_kv_kernel(
    int Hkv, int D, int max_pages, uint16_t* __restrict__ k_pool, uint16_t* __restrict__ v_pool,
    const int32_t* __restrict__ block_table, const int32_t* __restrict__ ctx_len,
    const int32_t* __restrict__ q_offsets, const int32_t* __restrict__ parent,
    const int32_t* __restrict__ stop_node, int32_t* __restrict__ new_len) {
  constexpr int kPageTokens = 16;
  const int b = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  __shared__ int sh_path[kCompactMaxNodes];     // leaf -> root
  __shared__ int sh_depth;
  const int o = q_offsets[b];
  int n = q_offsets[b + 1] - o;
  n = n < 0 ? 0 : (n > kCompactMaxNodes ? kCompactMaxNodes : n);
  const int ctx = ctx_len[b];
  if (tid == 0) {
    int depth = 0;
    int a = stop_node[b];
    while (a >= 0 && a < n && depth < kCompactMaxNodes) {
      sh_path[depth++] = a;
      const int p = parent ? parent[o + a] : a - 1;
      a = (p < a) ? p : -1;                     // a malformed parent entry ends the path
    }
    sh_depth = depth;
    if (h == 0 && new_len) new_len[b] = ctx + depth;
  }
  __syncthreads();
  const int depth = sh_depth;
  if (depth == 0) return;
  const int chunks = D / 8;                      // 16-byte chunks per row
  const int items = depth * 2 * chunks;          // (position on the path, K or V, chunk)
  const int32_t* bt = block_table + static_cast<int64_t>(b) * max_pages;
  const int64_t page_elems = static_cast<int64_t>(Hkv) * kPageTokens * D;
  constexpr int kPerThread = (kCompactMaxNodes * 2 * 16 + kCompactThreads - 1) / kCompactThreads;   // D <= 128
  cu32x4 held[kPerThread];
#pragma unroll
  for (int r = 0; r < kPerThread; ++r) {
    const int it = r * kCompactThreads + tid;
    if (it < items) {
      const int d = it / (2 * chunks), rem = it % (2 * chunks), which = rem / chunks, c = rem % chunks;
      const int pos = ctx + sh_path[depth - 1 - d];
      const int64_t src = bt[pos / kPageTokens] * page_elems + (static_cast<int64_t>(h) * kPageTokens + pos % kPageTokens) * D + c * 8;
      held[r] = *reinterpret_cast<const cu32x4*>((which ? v_pool : k_pool) + src);
    }
  }
  __syncthreads();                               // every source row is in registers
#pragma unroll
  for (int r = 0; r < kPerThread; ++r) {
    const int it = r * kCompactThreads + tid;
    if (it < items) {
      const int d = it / (2 * chunks), rem = it % (2 * chunks), which = rem / chunks, c = rem % chunks;
      const int pos = ctx + d;
      const int64_t dst = bt[pos / kPageTokens] * page_elems + (static_cast<int64_t>(h) * kPageTokens + pos % kPageTokens) * D + c * 8;
      *reinterpret_cast<cu32x4*>((which ? v_pool : k_pool) + dst) = held[r];
    }
  }
}

void launch_compact_kv(const CompactArgs& a, hipStream_t stream) {
  if (a.B <= 0 || a.Hkv <= 0) return;
  hipLaunchKernelGGL(compact_kv_kernel, dim3(a.B, a.Hkv), dim3(kCompactThreads), 0, stream, a.Hkv, a.D, a.max_pages,
                     a.k_pool, a.v_pool, a.block_table, a.ctx_len, a.q_offsets, a.parent, a.stop_node, a.new_len);
}

// ----------------------------------------------------------------------------------
// The same for the 8-bit cache (quant.h), whose pages have a scale each: a written page takes the largest of its own scale, if it
// holds committed tokens, and of those of the pages that its new entries come from; entries that move to, or stay under, a larger
// scale are rewritten for it (exactly, but for those that become subnormal).
//
// One workgroup per (request, KV head).  A job is 16 bytes of a written page: one token's chunk of 16 dimensions of K, one dimension's
// 16 slots of V.  All jobs are read and worked out, a barrier, then all are written.  Latency-bound: offsets -> page ids -> scales and
// entries -> store.
// ----------------------------------------------------------------------------------
constexpr int kQuantPathPages = kCompactMaxNodes / kQuantPage + 1;       // pages that 128 consecutive slots touch

template <int D>
__global__ __launch_bounds__(kCompactThreads) void compact_kv_quant_kernel(
    int Hkv, int max_pages, int num_pages, unsigned char* __restrict__ k_pool, unsigned char* __restrict__ v_pool,
    float* __restrict__ k_scale, float* __restrict__ v_scale, const int32_t* __restrict__ block_table,
    const int32_t* __restrict__ ctx_len, const int32_t* __restrict__ q_offsets, const int32_t* __restrict__ parent,
    const int32_t* __restrict__ stop_node, int32_t* __restrict__ new_len) {
  constexpr int kRounds = (kQuantPathPages * D + kCompactThreads - 1) / kCompactThreads;    // D jobs of 16 bytes per page and tensor
  const int b = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  __shared__ int sh_parent[kCompactMaxNodes], sh_path[kCompactMaxNodes];      // path: leaf -> root
  __shared__ int sh_depth;
  __shared__ int sh_page[kCompactMaxNodes], sh_slot[kCompactMaxNodes];        // where entry d comes from; page -1: it is not moved
  __shared__ float sh_scale[2][kCompactMaxNodes];                            // its scale, then its ratio to the new one
  __shared__ int sh_to[kQuantPathPages];                                     // written pages (-1: none)
  __shared__ float sh_old[2][kQuantPathPages], sh_new[2][kQuantPathPages];
  const int o = q_offsets[b];
  const int tokens = o < 0 ? 0 : max(q_offsets[b + 1], o) - o;               // (no request starts in front of the parents)
  const int ctx = ctx_len[b], stop = stop_node[b];
  if (ctx < 0) {                                                             // no request: nothing of it moves, its length stays
    if (tid == 0 && h == 0 && new_len) new_len[b] = ctx;
    return;
  }
  if (parent == nullptr) {                                                   // linear drafts, however many, lie where they belong
    if (tid == 0 && h == 0 && new_len)
      new_len[b] = static_cast<int>(min(static_cast<unsigned>(ctx) + (stop >= 0 && stop < tokens ? stop + 1 : 0), 0x7fffffffu));
    return;
  }
  const int n = min(tokens, kCompactMaxNodes);
  if (tid < n) sh_parent[tid] = parent[o + tid];
  __syncthreads();
  if (tid == 0) {
    int depth = 0;
    for (int a = stop; a >= 0 && a < n && depth < kCompactMaxNodes;) {
      sh_path[depth++] = a;
      const int p = sh_parent[a];
      a = p < a ? p : -1;                                                    // a malformed parent entry ends the path
    }
    sh_depth = depth;
    if (h == 0 && new_len) new_len[b] = static_cast<int>(min(static_cast<unsigned>(ctx) + depth, 0x7fffffffu));
  }
  __syncthreads();
  const int depth = sh_depth;
  if (depth == 0) return;
  const int32_t* bt = block_table + static_cast<int64_t>(b) * max_pages;
  auto page_of = [&](int lp) {
    const int id = lp < max_pages ? bt[lp] : -1;
    return id >= 0 && id < num_pages ? id : -1;
  };
  // places are counted from the start of the first written page: a length may be near 2^31
  const int lp0 = ctx / kQuantPage, held = ctx % kQuantPage, pages = (held + depth - 1) / kQuantPage + 1;
  if (tid < depth) {
    const int pos = held + sh_path[depth - 1 - tid], id = page_of(lp0 + pos / kQuantPage);
    sh_page[tid] = id;
    sh_slot[tid] = pos % kQuantPage;
    sh_scale[0][tid] = id < 0 ? 0.f : k_scale[static_cast<int64_t>(id) * Hkv + h];
    sh_scale[1][tid] = id < 0 ? 0.f : v_scale[static_cast<int64_t>(id) * Hkv + h];
  }
  __syncthreads();
  if (tid < 2 * pages) {
    const int j = tid >> 1, which = tid & 1, id = page_of(lp0 + j);
    const float own = id < 0 ? 0.f : (which ? v_scale : k_scale)[static_cast<int64_t>(id) * Hkv + h];
    float m = j == 0 && held > 0 ? own : 0.f;
    for (int t = 0; t < kQuantPage; ++t) {
      const int d = j * kQuantPage + t - held;
      if (d >= 0 && d < depth) m = fmaxf(m, sh_scale[which][d]);
    }
    sh_old[which][j] = own;
    sh_new[which][j] = m > 0.f ? m : own;                                   // (no entry reaches it)
    if (which == 0) sh_to[j] = id;
  }
  __syncthreads();
  if (tid < depth) {
    const int j = (held + tid) / kQuantPage;
    sh_scale[0][tid] *= inverse_scale(sh_new[0][j]);
    sh_scale[1][tid] *= inverse_scale(sh_new[1][j]);
  }
  __syncthreads();

  auto at = [&](int page, int byte) { return (static_cast<int64_t>(page) * Hkv + h) * (kQuantPage * D) + byte; };
  raw4 kw[kRounds], vw[kRounds];
  bool k_set[kRounds], v_set[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int it = r * kCompactThreads + tid, j = it / D, in = it % D;
    k_set[r] = v_set[r] = false;
    if (j >= pages || sh_to[j] < 0) continue;
    {
      const int chunk = in / kQuantPage, t = in % kQuantPage, d = j * kQuantPage + t - held;
      int page = -1, slot = t;
      float ratio = 1.f;
      if (d >= 0 && d < depth) {
        page = sh_page[d]; slot = sh_slot[d]; ratio = sh_scale[0][d];
      } else if (d < 0 && sh_new[0][j] > sh_old[0][j]) {
        page = sh_to[j]; ratio = sh_old[0][j] * inverse_scale(sh_new[0][j]);
      }
      if (page >= 0) {
        kw[r] = *reinterpret_cast<const raw4*>(k_pool + at(page, chunk * 256 + slot * 16));
#pragma unroll
        for (int w = 0; w < 4; ++w) kw[r][w] = rescale_e4m3(kw[r][w], ratio);
        k_set[r] = true;
      }
    }
    {
      vw[r] = *reinterpret_cast<const raw4*>(v_pool + at(sh_to[j], in * kQuantPage));
      const int d0 = j * kQuantPage - held;                                 // entry that slot 0 takes
      if (j == 0 && sh_new[1][0] > sh_old[1][0]) {
        const float ratio = sh_old[1][0] * inverse_scale(sh_new[1][0]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t mine = slot_mask(4 * w, 0, held);
          vw[r][w] = (rescale_e4m3(vw[r][w], ratio) & mine) | (vw[r][w] & ~mine);
        }
      }
#pragma unroll
      for (int t = 0; t < kQuantPage; ++t) {
        const int d = d0 + t;
        if (d < 0 || d >= depth || sh_page[d] < 0) continue;
        const uint32_t byte = rescale_e4m3(v_pool[at(sh_page[d], in * kQuantPage + sh_slot[d])], sh_scale[1][d]) & 0xffu;
        vw[r][t >> 2] = (vw[r][t >> 2] & ~(0xffu << (8 * (t & 3)))) | (byte << (8 * (t & 3)));
      }
      v_set[r] = true;
    }
  }
  __syncthreads();                                                           // everything that is read has been
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int it = r * kCompactThreads + tid, j = it / D, in = it % D;
    if (k_set[r]) *reinterpret_cast<raw4*>(k_pool + at(sh_to[j], in * 16)) = kw[r];
    if (v_set[r]) *reinterpret_cast<raw4*>(v_pool + at(sh_to[j], in * 16)) = vw[r];
  }
  if (tid < 2 * pages && sh_to[tid >> 1] >= 0)
    (tid & 1 ? v_scale : k_scale)[static_cast<int64_t>(sh_to[tid >> 1]) * Hkv + h] = sh_new[tid & 1][tid >> 1];
}

void launch_compact_kv_quant(const QuantCompactArgs& a, hipStream_t stream) {
  if (a.B <= 0 || a.Hkv <= 0) return;
  auto kernel = a.D == 128 ? compact_kv_quant_kernel<128> : compact_kv_quant_kernel<64>;
  hipLaunchKernelGGL(kernel, dim3(a.B, a.Hkv), dim3(kCompactThreads), 0, stream, a.Hkv, a.max_pages, a.num_pages, a.k_pool, a.v_pool,
                     a.k_scale, a.v_scale, a.block_table, a.ctx_len, a.q_offsets, a.parent, a.stop_node, a.new_len);
}

// ----------------------------------------------------------------------------------
// The same for the cache of latents: one row of `width` elements per token.  One workgroup per request; a row of up to 576 elements is 72 items of 16
// bytes, and every source row is read before any is written.
// ----------------------------------------------------------------------------------
constexpr int kLatentMost = 576 / 8;                                          // items of a row, at most

__global__ __launch_bounds__(1024) void compact_latent_kernel(
    int width, int max_pages, int num_pages, uint16_t* __restrict__ pool, const int32_t* __restrict__ block_table,
    const int32_t* __restrict__ ctx_len, const int32_t* __restrict__ q_offsets, const int32_t* __restrict__ parent,
    const int32_t* __restrict__ stop_node, int32_t* __restrict__ new_len) {
  constexpr int kPerThread = (kCompactMaxNodes * kLatentMost + 1023) / 1024;
  constexpr int kPage = 16;
  const int b = blockIdx.x, tid = threadIdx.x;
  __shared__ int sh_parent[kCompactMaxNodes], sh_path[kCompactMaxNodes];      // path: leaf -> root
  __shared__ int sh_depth;
  __shared__ int64_t sh_from[kCompactMaxNodes], sh_to[kCompactMaxNodes];      // rows of the pool; -1: none
  const int o = q_offsets[b], behind = q_offsets[b + 1];
  const int tokens = o < 0 ? 0 : max(behind, o) - o;
  const int ctx = ctx_len[b], stop = stop_node[b];
  if (ctx < 0) {                                                             // no request: nothing of it moves, its length stays
    if (tid == 0 && new_len) new_len[b] = ctx;
    return;
  }
  if (parent == nullptr) {                                                   // linear drafts, however many, lie where they belong
    if (tid == 0 && new_len)
      new_len[b] = static_cast<int>(min(static_cast<unsigned>(ctx) + (stop >= 0 && stop < tokens ? stop + 1 : 0), 0x7fffffffu));
    return;
  }
  const int n = min(tokens, kCompactMaxNodes);
  if (tid < n) sh_parent[tid] = parent[o + tid];
  __syncthreads();
  if (tid == 0) {
    int depth = 0;
    for (int a = stop; a >= 0 && a < n && depth < kCompactMaxNodes;) {
      sh_path[depth++] = a;
      const int p = sh_parent[a];
      a = p < a ? p : -1;                                                    // a malformed parent entry ends the path
    }
    sh_depth = depth;
    if (new_len) new_len[b] = static_cast<int>(min(static_cast<unsigned>(ctx) + depth, 0x7fffffffu));
  }
  __syncthreads();
  const int depth = sh_depth;
  if (depth == 0) return;
  if (tid < 2 * depth) {
    const int d = tid >> 1;
    const int64_t pos = static_cast<int64_t>(ctx) + (tid & 1 ? d : sh_path[depth - 1 - d]), lp = pos / kPage;
    const int id = lp < max_pages ? block_table[static_cast<int64_t>(b) * max_pages + lp] : -1;
    (tid & 1 ? sh_to : sh_from)[d] = id >= 0 && id < num_pages ? static_cast<int64_t>(id) * kPage + pos % kPage : -1;
  }
  __syncthreads();
  const int row = width / 8, items = depth * row;
  raw4 held[kPerThread];
#pragma unroll
  for (int r = 0; r < kPerThread; ++r) {
    const int it = r * 1024 + tid, d = it / row;
    if (it < items && sh_from[d] >= 0) held[r] = reinterpret_cast<const raw4*>(pool + sh_from[d] * width)[it - d * row];
  }
  __syncthreads();                                                           // everything that is read has been
#pragma unroll
  for (int r = 0; r < kPerThread; ++r) {
    const int it = r * 1024 + tid, d = it / row;
    if (it < items && sh_from[d] >= 0 && sh_to[d] >= 0) reinterpret_cast<raw4*>(pool + sh_to[d] * width)[it - d * row] = held[r];
  }
}

void launch_compact_latent(const LatentCompactArgs& a, hipStream_t stream) {
  if (a.B <= 0) return;
  hipLaunchKernelGGL(compact_latent_kernel, dim3(a.B), dim3(1024), 0, stream, a.width, a.max_pages, a.num_pages, a.pool, a.block_table, a.ctx_len, a.q_offsets,
                     a.parent, a.stop_node, a.new_len);
}

}  // namespace specv
