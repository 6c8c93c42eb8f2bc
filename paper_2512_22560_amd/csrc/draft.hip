// What surrounds the attention of a draft: its tree's visibility and positions before, the move of the accepted rows after.
#include <algorithm>
#include <type_traits>

#include "codes_device.h"

namespace rollattn {

namespace {

constexpr int kThreads = 256;

// A thread per node walks to the root: parents have lower numbers, so the words of its mask are met from the last down.
__global__ __launch_bounds__(kThreads) void tree_mask_kernel(const TreeMaskArgs a) {
  const int b = blockIdx.x, n = a.q_lens[b], off = a.q_offsets[b], prefix = a.ctx_lens[b] - n;
  const int32_t* const parents = a.parents + off;
  for (int i = threadIdx.x; i < n; i += kThreads) {
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
      j = p < j ? p : -1;                             // (what is no earlier node is no parent)
    }
    if (w < a.mask_words) words[w] = bits;
    while (--w >= 0) words[w] = 0;
    if (a.positions) a.positions[off + i] = prefix + depth;
  }
}

// The accepted rows of a draft to where the trajectory goes on: a workgroup per (trajectory, pool), page after page of the places that
// rows go to.  A row never comes from before its place, so a page's sources are untouched by what went into the pages before it; a
// thread has one 16-byte column of all rows, reads those of the page and then writes them, and nobody else writes that column.
// POOL: -1 rows move bit for bit, else a KvKind
template <int ROW_BYTES, int POOL>
__global__ __launch_bounds__(kThreads) void kv_accept_kernel(const AcceptArgs a) {
  constexpr bool kCodes = POOL >= 0, kHeadScales = kCodes && kv_has_head_scales(POOL);
  constexpr bool kInt8 = POOL == kKvInt8Head;
  constexpr float kMax = kInt8 ? kInt8Max : kE4m3Max;
  constexpr int kChunks = ROW_BYTES / 16;       // columns of a head
  const int b = blockIdx.x, pool = blockIdx.y;
  const int n = a.q_lens[b], m = min(a.accept_lens[b], n), off = a.q_offsets[b], first = a.ctx_lens[b] - n, hkv = a.hkv;
  if (m <= 0) return;
  unsigned char* const pages = (unsigned char*)(pool ? a.v_pages : a.k_pages);
  float* const scales = pool ? a.v_scale : a.k_scale;
  const int32_t* const table = a.page_table + (size_t)b * a.max_pages;
  const int columns = hkv * kChunks;
  __shared__ int from_page[kPageSize], from_slot[kPageSize];
  __shared__ float top_s[kThreads / 64];
  for (int page_i = first / kPageSize; page_i * kPageSize < first + m; ++page_i) {
    const int lo = max(first, page_i * kPageSize), rows = min(first + m, (page_i + 1) * kPageSize) - lo;
    const int s0 = lo - page_i * kPageSize, page = table[page_i];
    __syncthreads();
    bool moves = false;
    if ((int)threadIdx.x < rows) {
      const int i = lo - first + threadIdx.x, node = min(max(a.accepted[off + i], i), n - 1);
      from_page[threadIdx.x] = table[(first + node) / kPageSize];
      from_slot[threadIdx.x] = (first + node) % kPageSize;
      moves = node != i;
    }
    if (!__syncthreads_or(moves)) continue;
    auto row_at = [&](int id, int head, int slot) { return pages + (((size_t)id * hkv + head) * kPageSize + slot) * ROW_BYTES; };
    const int trips = (columns + kThreads - 1) / kThreads;
    float page_before = 0.f, page_now = 0.f;
    if constexpr (kCodes && !kHeadScales) {
      // one scale for the page: the largest magnitude of all heads that comes from elsewhere first
      float top = 0.f;
      for (int c = threadIdx.x; c < columns; c += kThreads)
        for (int r = 0; r < rows; ++r)
          if (from_page[r] != page) {
            const uintx4 w = *(const uintx4*)(row_at(from_page[r], c / kChunks, from_slot[r]) + c % kChunks * 16);
            top = fmaxf(top, largest16<kInt8>(w) * scales[from_page[r]]);
          }
      for (int i = 1; i < 64; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
      if (threadIdx.x % 64 == 0) top_s[threadIdx.x / 64] = top;
      page_before = scales[page];
      __syncthreads();
      for (int w = 0; w < kThreads / 64; ++w) top = fmaxf(top, top_s[w]);
      page_now = fmaxf(page_before, top / kMax);
    }
    for (int trip = 0; trip < trips; ++trip) {
      const int c = min(trip * kThreads + (int)threadIdx.x, columns - 1), head = c / kChunks, at = c % kChunks * 16;
      const bool mine = trip * kThreads + (int)threadIdx.x < columns;
      uintx4 x[kPageSize];
      float scale[kCodes ? kPageSize : 1];
#pragma unroll
      for (int r = 0; r < kPageSize; ++r)
        if (r < rows) {
          x[r] = *(const uintx4*)(row_at(from_page[r], head, from_slot[r]) + at);
          if constexpr (kCodes) scale[r] = scales[kHeadScales ? (size_t)from_page[r] * hkv + head : from_page[r]];
        }
      if constexpr (kCodes) {
        float before = page_before, now = page_now;
        if constexpr (kHeadScales) {
          float top = 0.f;
    #pragma unroll
      for (int r = 0; r < kPageSize; ++r)
            if (r < rows && from_page[r] != page) top = fmaxf(top, largest16<kInt8>(x[r]) * scale[r]);
          for (int i = 1; i < kChunks; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
          before = scales[(size_t)page * hkv + head];
          now = fmaxf(before, top / kMax);
          if (mine && at == 0) scales[(size_t)page * hkv + head] = now;
        }
        if (now > before && mine)
          for (int r = 0; r < s0; ++r) {
            uintx4* p = (uintx4*)(row_at(page, head, r) + at);
            *p = again16<kInt8>(*p, before, now);
          }
  #pragma unroll
      for (int r = 0; r < kPageSize; ++r)
          if (r < rows) x[r] = again16<kInt8>(x[r], scale[r], now);
      }
      if (mine)
  #pragma unroll
      for (int r = 0; r < kPageSize; ++r)
          if (r < rows) *(uintx4*)(row_at(page, head, s0 + r) + at) = x[r];
    }
    if constexpr (kCodes && !kHeadScales) {
      __syncthreads();
      if (threadIdx.x == 0) scales[page] = page_now;
    }
  }
}

}  // namespace

hipError_t launch_tree_mask(const TreeMaskArgs& a, int32_t, hipStream_t s) {
  hipLaunchKernelGGL(tree_mask_kernel, dim3(a.batch), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv_accept(const AcceptArgs& a, int32_t, int head_dim, int row_bytes, int pool, hipStream_t s) {
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
