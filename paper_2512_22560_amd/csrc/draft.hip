// What surrounds the attention of a draft: its tree's visibility and positions before, the move of the accepted rows after.
#include <algorithm>
#include <type_traits>

#include "codes_device.h"

namespace rollattn {

namespace {

constexpr int kThreads = 256;

// Masks and positions.  Every node knows its parent; in each step it takes over what the node that it points to has seen and points where
// that one does, so that 2^k ancestors are known after k steps.  Bound by latency: a draft of 64 nodes is one wave's, whose lanes ask each
// other, four drafts to a workgroup; larger ones a workgroup's, through LDS.  512 drafts of 32 .. 200 nodes: a walk to the root for each node
// 17.6 us a call, so 6.4; 5 of 5 .. 24: 4.9 and 4.7, of which the kernel is 1.7.
// The same by a walk to the root, a thread per node, for drafts that are larger than the caller has said: parents have lower numbers, so
// the words of a mask are met from the last down.
__device__ __forceinline__ void walk(const TreeMaskArgs& a, int n, int off, int prefix, int first, int step) {
  const int32_t* const parents = a.parents + off;
  for (int i = first; i < n; i += step) {
    uint64_t* const words = a.mask + (size_t)(off + i) * a.mask_words;
    int depth = -1, w = a.mask_words;                 // words[w ..] are written
    uint64_t bits = 0;
    for (int j = i; j >= 0;) {
      const int at = j >> 6;
      if (at < w) {
        if (w < a.mask_words) words[w] = bits;
        while (--w > at) words[w] = 0;
        bits = 0;
      }
      if (at < a.mask_words) bits |= 1ull << (j & 63);
      ++depth;
      const int p = parents[j];
      j = p < j ? p : -1;
    }
    if (w < a.mask_words) words[w] = bits;
    while (--w >= 0) words[w] = 0;
    if (a.positions) a.positions[off + i] = prefix + depth;
  }
}

__global__ __launch_bounds__(kThreads) void tree_mask_wave_kernel(const TreeMaskArgs a) {
  const int lane = threadIdx.x & 63, b = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (kThreads / 64) + threadIdx.x / 64));
  if (b >= a.batch) return;
  const int n = a.q_lens[b], off = a.q_offsets[b], prefix = a.ctx_lens[b] - n;
  if (n > 64) {
    walk(a, n, off, prefix, lane, 64);
    return;
  }
  int up = lane < n ? a.parents[off + lane] : -1;
  if (up >= lane || up < 0) up = -1;                  // (what is no earlier node is no parent)
  uint64_t bits = 1ull << lane;
  while (__builtin_amdgcn_ballot_w64(up >= 0)) {
    const int from = max(up, 0), next = __shfl(up, from);
    const uint64_t more = __shfl((unsigned long long)bits, from);
    if (up >= 0) {
      bits |= more;
      up = next;
    }
  }
  if (lane >= n) return;
  uint64_t* const words = a.mask + (size_t)(off + lane) * a.mask_words;
  words[0] = bits;
  for (int w = 1; w < a.mask_words; ++w) words[w] = 0;
  if (a.positions) a.positions[off + lane] = prefix + __builtin_popcountll(bits) - 1;
}

// NODES: 256 or 1024, a thread each
template <int NODES>
__global__ __launch_bounds__(NODES) void tree_mask_kernel(const TreeMaskArgs a) {
  constexpr int kWords = NODES / 64;
  __shared__ uint64_t seen[kWords][NODES];            // (neighbours' words in neighbouring places)
  __shared__ int next_s[NODES];
  const int b = blockIdx.x, n = a.q_lens[b], off = a.q_offsets[b], prefix = a.ctx_lens[b] - n, i = threadIdx.x;
  if (n > NODES) {
    walk(a, n, off, prefix, i, NODES);
    return;
  }
  const int live = (n + 63) / 64;                     // words that this draft has
  int up = i < n ? a.parents[off + i] : -1;
  if (up >= i || up < 0) up = -1;
  for (int w = 0; w < live; ++w) seen[w][i] = i / 64 == w ? 1ull << (i & 63) : 0;
  next_s[i] = up;
  while (__syncthreads_or(up >= 0)) {
    uint64_t more[kWords];
    int next = -1;
    if (up >= 0) {
      // (an ancestor's own ancestors are no later words than its own)
#pragma unroll
      for (int w = 0; w < kWords; ++w) more[w] = w <= up / 64 ? seen[w][up] : 0;
      next = next_s[up];
    }
    __syncthreads();
    if (up >= 0) {
#pragma unroll
      for (int w = 0; w < kWords; ++w)
        if (w <= up / 64) seen[w][i] |= more[w];
      next_s[i] = next;
    }
    up = next;
  }
  if (i >= n) return;
  uint64_t* const words = a.mask + (size_t)(off + i) * a.mask_words;
  int count = -1;
  for (int w = 0; w < live; ++w) count += __builtin_popcountll(seen[w][i]);
  for (int w = 0; w < a.mask_words; ++w) words[w] = w < live ? seen[w][i] : 0;
  if (a.positions) a.positions[off + i] = prefix + count;
}

// The accepted rows of a draft to where the trajectory goes on: a workgroup per (trajectory, pool), whose threads share the 16-byte pieces
// of the rows that go to some pages (of some heads, where a token's row is long).  All are read, then, behind a barrier, written; a row never
// comes from before its place, so the pages that follow are still as they were.  Bound by the latency of one chain, lengths, nodes, page
// ids, rows and scales: a path is a few rows.  Pieces to threads and not a thread to each column of a page's 16 places, whose codes are
// made one after the other: 512 paths in drafts of 16 .. 64 (64/4/128, int8) 20.6 -> 9.6 us.
// POOL: -1 rows move bit for bit, else a KvKind
template <int ROW_BYTES, int POOL>
__global__ __launch_bounds__(kThreads) void kv_accept_kernel(const AcceptArgs a) {
  constexpr bool kCodes = POOL >= 0, kHeadScales = kCodes && kv_has_head_scales(POOL), kPageScale = kCodes && !kHeadScales;
  constexpr bool kInt8 = POOL == kKvInt8Head;
  constexpr float kMax = kInt8 ? kInt8Max : kE4m3Max;
  constexpr int kChunks = ROW_BYTES / 16;                     // pieces of a head's row
  constexpr int kItems = 8, kRoom = kThreads * kItems;        // pieces of a thread, of all
  constexpr int kMostHeads = kRoom / kPageSize / kChunks;     // at least one page of this many heads fits
  constexpr int kMostPages = kRoom / kPageSize / kChunks, kMostScales = kMostPages;   // (of one head; pages * heads is no more either)
  const int b = blockIdx.x, pool = blockIdx.y;
  const int n = a.q_lens[b], m = min(a.accept_lens[b], n), off = a.q_offsets[b], first = a.ctx_lens[b] - n, hkv = a.hkv;
  if (m <= 0) return;
  unsigned char* const pages = (unsigned char*)(pool ? a.v_pages : a.k_pages);
  float* const scales = pool ? a.v_scale : a.k_scale;
  const int32_t* const table = a.page_table + (size_t)b * a.max_pages;
  const int heads = min(hkv, kMostHeads), side = kRoom / (kPageSize * kChunks * heads);   // heads and pages at a time
  __shared__ int from_page[kMostPages * kPageSize], from_slot[kMostPages * kPageSize], to_page[kMostPages], moves[kMostPages];
  __shared__ int top_s[kMostScales];                          // per page (and head): the largest magnitude that comes from elsewhere
  __shared__ float before_s[kMostScales];
  auto row_at = [&](int id, int head, int slot) { return pages + (((size_t)id * hkv + head) * kPageSize + slot) * ROW_BYTES; };
  auto scale_at = [&](int id, int head) { return scales + (kHeadScales ? (size_t)id * hkv + head : (size_t)id); };
  for (int page0 = first / kPageSize; page0 * kPageSize < first + m; page0 += side) {
    // what goes to the pages [page0, page0 + side): places lo .. hi, by place from `start` on
    const int start = page0 * kPageSize, lo = max(first, start), hi = min(first + m, start + side * kPageSize), n_pages = (hi - start + kPageSize - 1) / kPageSize;
    __syncthreads();
    for (int i = threadIdx.x; i < n_pages; i += kThreads) {
      moves[i] = 0;
      to_page[i] = table[page0 + i];
      if constexpr (kPageScale) top_s[i] = 0;
    }
    __syncthreads();
    for (int place = lo + threadIdx.x; place < hi; place += kThreads) {
      const int i = place - first, at = place - start, node = min(max(a.accepted[off + i], i), n - 1);
      from_page[at] = table[(first + node) / kPageSize];
      from_slot[at] = (first + node) % kPageSize;
      if (node != i) moves[at / kPageSize] = 1;
    }
    __syncthreads();
    // the pieces of heads [h0, h0 + count), piece by piece: the piece's place, head and byte of its row
    auto each = [&](int h0, int count, auto&& f) __attribute__((always_inline)) {
      const int columns = count * kChunks, all = (hi - lo) * columns;
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        const int item = threadIdx.x + k * kThreads;
        if (item < all) {
          const int place = item / columns, c = item - place * columns, at = lo - start + place;
          if (moves[at / kPageSize]) f(k, at, h0 + c / kChunks, c % kChunks * 16);
        }
      }
    };
    uintx4 x[kItems];
    float scale[kCodes ? kItems : 1];
    auto read = [&](int h0, int count) __attribute__((always_inline)) {
      each(h0, count, [&](int k, int at, int head, int byte) __attribute__((always_inline)) {
        x[k] = *(const uintx4*)(row_at(from_page[at], head, from_slot[at]) + byte);
        if constexpr (kCodes) scale[k] = *scale_at(from_page[at], head);
      });
    };
    auto largest = [&](int h0, int count) __attribute__((always_inline)) {
      each(h0, count, [&](int k, int at, int head, int) __attribute__((always_inline)) {
        const int p = at / kPageSize;
        // (floats from zero up order like integers)
        if (from_page[at] != to_page[p]) atomicMax(&top_s[kHeadScales ? p * count + head - h0 : p], __float_as_int(largest16<kInt8>(x[k]) * scale[k]));
      });
    };
    if constexpr (kPageScale) {
      // one scale for the page: all heads first
      for (int h0 = 0; h0 < hkv; h0 += heads) {
        read(h0, min(heads, hkv - h0));
        largest(h0, min(heads, hkv - h0));
      }
      for (int i = threadIdx.x; i < n_pages; i += kThreads) before_s[i] = scales[to_page[i]];
      __syncthreads();
    }
    for (int h0 = 0; h0 < hkv; h0 += heads) {
      const int count = min(heads, hkv - h0);
      read(h0, count);
      if constexpr (kHeadScales) {
        for (int i = threadIdx.x; i < n_pages * count; i += kThreads) {
          top_s[i] = 0;
          before_s[i] = *scale_at(to_page[i / count], h0 + i % count);
        }
        __syncthreads();
        largest(h0, count);
      }
      __syncthreads();
      auto now_of = [&](int i) { return fmaxf(before_s[i], __int_as_float(top_s[i]) / kMax); };
      each(h0, count, [&](int k, int at, int head, int byte) __attribute__((always_inline)) {
        const int p = at / kPageSize, i = kHeadScales ? p * count + head - h0 : p;
        if constexpr (kCodes) {
          const float now = now_of(i);
          if (scale[k] != now) x[k] = again16<kInt8>(x[k], scale[k], now);   // (under the same scale codes are the same)
        }
        *(uintx4*)(row_at(to_page[p], head, at % kPageSize) + byte) = x[k];
      });
      if constexpr (kCodes) {
        // the first page's places in front of the draft, and the scales
        const int s0 = lo - start, columns = count * kChunks;
        for (int item = threadIdx.x; item < s0 * columns; item += kThreads) {
          const int slot = item / columns, c = item - slot * columns, head = h0 + c / kChunks, i = kHeadScales ? head - h0 : 0;
          const float now = now_of(i);
          if (now > before_s[i]) {
            uintx4* p = (uintx4*)(row_at(to_page[0], head, slot) + c % kChunks * 16);
            *p = again16<kInt8>(*p, before_s[i], now);
          }
        }
        if constexpr (kHeadScales) {
          for (int i = threadIdx.x; i < n_pages * count; i += kThreads)
            if (moves[i / count]) *scale_at(to_page[i / count], h0 + i % count) = now_of(i);
          __syncthreads();                                    // (before the next heads' maxima)
        }
      }
    }
    if constexpr (kPageScale) {
      __syncthreads();
      for (int i = threadIdx.x; i < n_pages; i += kThreads)
        if (moves[i]) scales[to_page[i]] = fmaxf(before_s[i], __int_as_float(top_s[i]) / kMax);
    }
  }
}

}  // namespace

hipError_t launch_tree_mask(const TreeMaskArgs& a, int32_t max_q_len, hipStream_t s) {
  if (max_q_len <= 64) hipLaunchKernelGGL(tree_mask_wave_kernel, dim3((a.batch + kThreads / 64 - 1) / (kThreads / 64)), dim3(kThreads), 0, s, a);
  else if (max_q_len <= 256) hipLaunchKernelGGL((tree_mask_kernel<256>), dim3(a.batch), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((tree_mask_kernel<1024>), dim3(a.batch), dim3(1024), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv_accept(const AcceptArgs& a, int head_dim, int row_bytes, int pool, hipStream_t s) {
  const dim3 grid(a.batch, 2);
  auto go = [&](auto bytes, auto kind) {
    hipLaunchKernelGGL((kv_accept_kernel<decltype(bytes)::value, decltype(kind)::value>), grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
  };
  auto codes = [&](auto kind) { return head_dim == 128 ? go(std::integral_constant<int, 128>{}, kind) : go(std::integral_constant<int, 64>{}, kind); };
  constexpr std::integral_constant<int, -1> as_they_are{};
  switch (pool) {
    case -1:
      if (row_bytes == 512) return go(std::integral_constant<int, 512>{}, as_they_are);
      if (row_bytes == 256) return go(std::integral_constant<int, 256>{}, as_they_are);
      if (row_bytes == 128) return go(std::integral_constant<int, 128>{}, as_they_are);
      return hipErrorInvalidValue;
    case kKvFp8: return codes(std::integral_constant<int, kKvFp8>{});
    case kKvFp8Head: return codes(std::integral_constant<int, kKvFp8Head>{});
    case kKvInt8Head: return codes(std::integral_constant<int, kKvInt8Head>{});
    default: return hipErrorInvalidValue;
  }
}

}  // namespace rollattn
