// KV write with the position rotation on the way: the new tokens' queries and keys are turned to their positions, queries are
// handed back, K and V rows go into the paged cache.  Also the plain write into pools with a scale for each page and KV head.
//
// Rotation of a pair (lo, hi) with the table's c and s: lo' = lo c - hi s, hi' = hi c + lo s, each product and sum one float32
// operation (no fused ones: codes are integers decided by these numbers).  Codes of a page and head: the scale is
// absmax / 448 or / 127 of the head's new rows in the page, never below kLeastHeadScale and, where the page already holds tokens,
// never below the old one; if it grew, the codes already there are quantised again.
//
// Two kinds of workgroups share a launch.  Keys and values: a workgroup per (page that receives new tokens, pool); the page
// belongs to one trajectory alone, so nothing here needs a global atomic.  Queries: one wave per token and some of its heads, which
// lie side by side, so that a wave reads and writes kilobytes in a row, and what the token's position takes is looked up once.
// A row of D elements is the work of D / 8 lanes, eight elements to a lane: two runs of four whose elements are each other's
// partners, so that a rotation needs no exchange between lanes.  In a page's workgroup the groups of lanes are dealt to the new
// slots first and the rest of them to heads, so that a lane keeps its slot over all heads it walks.
#include <algorithm>
#include <type_traits>

#include "codes_device.h"

namespace rollattn {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kKeep = 8;          // rows of a lane that are under way at once
constexpr int kRound = 4;         // heads of a lane whose rows are held until their scales are known
constexpr int kQueryWaves = 2048; // queries: waves wanted where there are few tokens
// Rotated queries of more bytes than this do not stay in the memory-side cache (256 MB) until attention reads them, and are written
// with the streaming hint, by instances of their own (a branch between the two in one instance: 139 -> 147 us): 363 and 220 MB of
// them 139 -> 133 and 117 -> 112 us alone, 719 -> 719 and 376 -> 375 with attn_append behind; 41 MB of them 244 -> 246 with it.
constexpr int64_t kStreamQueries = 128 << 20;
constexpr int kSmallPage = 256;   // elements of a token's keys up to which pages are small
constexpr int kUneven = 5;        // times the mean chunk's pages that the longest one may have before pages are dealt out by a search

template <int SRC_BYTES>
struct Raw {                      // a lane's eight elements as they come
  typedef uintx2 half;
  half lo, hi;
};
template <>
struct Raw<4> {
  typedef uintx4 half;
  half lo, hi;
};

template <int SRC_BYTES>
__device__ __forceinline__ void to_float(const Raw<SRC_BYTES>& r, float (&x)[8]) {
  if constexpr (SRC_BYTES == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = __uint_as_float(r.lo[i]);
      x[4 + i] = __uint_as_float(r.hi[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[2 * i] = __uint_as_float(r.lo[i] << 16);
      x[2 * i + 1] = __uint_as_float(r.lo[i] & 0xffff0000u);
      x[4 + 2 * i] = __uint_as_float(r.hi[i] << 16);
      x[4 + 2 * i + 1] = __uint_as_float(r.hi[i] & 0xffff0000u);
    }
  }
}

__device__ __forceinline__ uintx2 to_bf16x4(const float* x) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(uintx2, bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]});
}

struct Turn {
  float c[4], s[4];
  // x: the elements of two runs of four; the partners are (i, 4 + i), or (2 i, 2 i + 1) where interleaved
  __device__ __forceinline__ void apply(float (&x)[8], bool interleaved) const {
#pragma clang fp contract(off)
    if (interleaved) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float lo = x[2 * i], hi = x[2 * i + 1];
        x[2 * i] = lo * c[i] - hi * s[i];
        x[2 * i + 1] = hi * c[i] + lo * s[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float lo = x[i], hi = x[4 + i];
        x[i] = lo * c[i] - hi * s[i];
        x[4 + i] = hi * c[i] + lo * s[i];
      }
    }
  }
};

// The cosines and sines of four pairs from j on; place: the token's place in its context, token: its number among the new ones.
__device__ __forceinline__ void look_up(const RopeWriteArgs& a, int j, int place, int64_t token, Turn& turn) {
  const int half = a.rot_dim / 2;
  const unsigned int last = (unsigned int)a.num_positions - 1;
  auto row = [&](int axis) {
    const int at = a.positions ? a.positions[(int64_t)axis * a.total_q + token] : place;
    return a.cos_sin + (size_t)min((unsigned int)at, last) * a.rot_dim + j;
  };
  const unsigned int axes = a.pair_axes[j / 16] >> (j % 16 * 2) & 0xff;
  if (axes == (axes & 3) * 0x55) {                    // one axis for the four
    const float* r = row(axes & 3);
    typedef float floatx4 __attribute__((ext_vector_type(4)));
    const floatx4 c = *(const floatx4*)r, s = *(const floatx4*)(r + half);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      turn.c[i] = c[i];
      turn.s[i] = s[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* r = row(axes >> (2 * i) & 3) + i;
      turn.c[i] = r[0];
      turn.s[i] = r[half];
    }
  }
}

// What a lane knows of the rows it works on: where its two runs of four start, and whether they are partners.
struct Lane {
  int e0, e1;
  bool turns;
  __device__ __forceinline__ Lane(const RopeWriteArgs& a, int col, bool rotate) {
    turns = rotate && col * 8 < a.rot_dim;
    e0 = col * 8;
    e1 = e0 + 4;
    if (turns && !a.interleaved) {
      e0 = col * 4;
      e1 = e0 + a.rot_dim / 2;
    }
  }
};

template <int SRC_BYTES>
__device__ __forceinline__ Raw<SRC_BYTES> fetch(const Lane& lane, const void* rows, int64_t element) {
  const unsigned char* p = (const unsigned char*)rows + element * SRC_BYTES;
  Raw<SRC_BYTES> r;
  r.lo = *(const typename Raw<SRC_BYTES>::half*)(p + lane.e0 * SRC_BYTES);
  r.hi = *(const typename Raw<SRC_BYTES>::half*)(p + lane.e1 * SRC_BYTES);
  return r;
}

// A row of the source type, turned where it has to be, at p; STREAM: past the caches' care.
template <int SRC_BYTES, bool STREAM>
__device__ __forceinline__ void store(const RopeWriteArgs& a, const Lane& lane, const Turn& turn, void* p, Raw<SRC_BYTES> r) {
  if (lane.turns) {
    float x[8];
    to_float<SRC_BYTES>(r, x);
    turn.apply(x, a.interleaved);
    if constexpr (SRC_BYTES == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        r.lo[i] = __float_as_uint(x[i]);
        r.hi[i] = __float_as_uint(x[4 + i]);
      }
    } else {
      r.lo = to_bf16x4(x);
      r.hi = to_bf16x4(x + 4);
    }
  }
  typedef typename Raw<SRC_BYTES>::half half;
  half *lo = (half*)((unsigned char*)p + lane.e0 * SRC_BYTES), *hi = (half*)((unsigned char*)p + lane.e1 * SRC_BYTES);
  if constexpr (STREAM) {
    __builtin_nontemporal_store(r.lo, lo);
    __builtin_nontemporal_store(r.hi, hi);
  } else {
    *lo = r.lo;
    *hi = r.hi;
  }
}

// The last of `count` things that starts at or before `place`, starts in order and the first at 0: 64 at a time.  The same in all lanes.
template <class Start>
__device__ __forceinline__ int last_from(int count, int place, Start&& start) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = count;                              // among [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) / 64, at = lane * step;
    const bool before = at < n && start(lo + at) <= place;
    const int k = max(__builtin_popcountll(__builtin_amdgcn_ballot_w64(before)) - 1, 0);
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

// The place in its context of new token `token`; `first` is the smallest token of the wave and the same in all lanes.  The trajectory a
// token belongs to is the last one that starts at or before it: for the first by looking at 64 starts at a time, from there on by
// steps that double, then halve.
__device__ __forceinline__ int place_of(const RopeWriteArgs& a, int first, int token) {
  if (a.one_each) {
    // (only where the lengths on the device still say so: a captured launch may be replayed with trajectories that have ended)
    const int place = a.ctx_lens[token] - 1;
    if (((const __attribute__((address_space(4))) int32_t*)a.q_offsets)[a.batch] == a.total_q) return place;
  }
  int lo = last_from(a.batch, first, [&](int i) { return a.q_offsets[i]; });
  if (a.wave_tokens > 1) {
    int ahead = 1;
    for (; lo + ahead < a.batch && a.q_offsets[lo + ahead] <= token; ahead *= 2) lo += ahead;
    while (ahead /= 2)
      if (lo + ahead < a.batch && a.q_offsets[lo + ahead] <= token) lo += ahead;
  }
  return a.ctx_lens[lo] - a.q_lens[lo] + token - a.q_offsets[lo];
}

template <int D, int SRC_BYTES, bool STREAM>
__device__ __forceinline__ void turn_queries(const RopeWriteArgs& a, unsigned int block) {
  constexpr int kLanes = D / 8, kRows = 64 / kLanes;  // lanes of a row, heads under way at a time
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned int unit = block * kWaves + wave;
  const int group = __builtin_amdgcn_readfirstlane((int)(unit / (unsigned int)a.head_parts)), part = (int)(unit - (unsigned int)group * a.head_parts);
  const int first = group * a.wave_tokens;
  if (first >= a.total_q) return;
  // the wave's rows of lanes: to tokens, and to heads of theirs
  const int col = (threadIdx.x & 63) % kLanes, row = (threadIdx.x & 63) / kLanes;
  const int side = kRows / a.wave_tokens;             // heads of a token under way at a time
  const int mine = row / side, sub = row - mine * side;
  const int token = min(first + mine, a.total_q - 1);
  const int h0 = part * a.part_heads, h1 = first + mine < a.total_q ? min(a.hq, h0 + a.part_heads) : 0;
  const Lane lane(a, col, true);
  Turn turn;
  const int heads = min(a.hq - h0, a.part_heads);     // (the same in all lanes)
  auto load = [&](Raw<SRC_BYTES> (&r)[kKeep], int h) {
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
      if (h + i * side < heads) r[i] = fetch<SRC_BYTES>(lane, a.q, token * a.q_stride + (int64_t)(h0 + min(h + i * side + sub, heads - 1)) * D);
  };
  Raw<SRC_BYTES> r[kKeep] = {};
  load(r, 0);                                         // (on their way while the position is looked up)
  const int place = a.positions ? 0 : place_of(a, first, token);
  if (lane.turns) look_up(a, col * 4, place, token, turn);
  for (int h = 0; h < heads; h += kKeep * side) {
    if (h) load(r, h);
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      const int head = h0 + h + i * side + sub;
      if (head < h1) store<SRC_BYTES, STREAM>(a, lane, turn, (unsigned char*)a.q_out + ((int64_t)token * a.hq + head) * D * SRC_BYTES, r[i]);
    }
  }
}

// Bound by memory where there are many tokens, by the latency of one chain (lengths, page id and rows, maximum, codes) where there
// are few.  What the large cases gained by, 22150 tokens of 64/4/128 into E4M3 pages (three axes; 794 MB) and 26835 of 32/8/128 into
// int8 ones (605 MB), us a call: a workgroup per page and 16 heads, heads outermost 171 and 138 (at any time all of them read and write
// the same few kilobytes of every token's row, a part of the memory's channels), heads innermost 151 and 148 (keys on some XCDs,
// queries on others), in 13 parts instead of 4 to 10: 154 and worse, each looking positions up again; queries by tokens, behind the
// pages 156 and 148, among them 139 and 117, with the streaming hint 133 and 112: 6.0 and 5.4 TB/s where a streaming pass over as
// many bytes reaches 6.2.  Fewer workgroups that take several pages each: slower by 5 to 20 %.  Rows held as floats until their scale is
// known instead of turned twice: three workgroups per CU instead of five.
// 180000 tokens of 8/2/64 (540 MB), whose queries fill a wave's registers eight tokens at a time: 212 us with a wave per token, 143 so,
// 133 with fewer workgroups for its small pages (below).
// 512 single tokens (64/4/128, int8; between events around the launch): 11.4 us with a search for each token's trajectory and a wave per
// four query heads, 10.2 without the search, 8.8 with a wave per sixteen.
// POOL: -1 the source type, else a KvKind; STREAM: rotated queries are written with the streaming hint; DEAL: pages are dealt out by a search
template <int D, int SRC_BYTES, int POOL, bool STREAM, bool DEAL>
__global__ __launch_bounds__(kThreads) void kv_write_rope_kernel(const RopeWriteArgs a) {
  constexpr bool kCodes = POOL >= 0, kHeadScales = kCodes && kv_has_head_scales(POOL);
  constexpr bool kInt8 = POOL == kKvInt8Head;
  constexpr int kLanes = D / 8;                 // lanes of a row
  constexpr int kGroups = kThreads / kLanes;    // rows under way at a time
  constexpr int kMost = kRound * kGroups;       // heads of a round, at most
  // Workgroups go to the XCDs in turn, so in groups of eight either kind has one on each; the groups of pages are spread evenly
  // among those of queries.
  const unsigned int g = blockIdx.x / kXcds, at = blockIdx.x % kXcds;
  const unsigned int pages_before = (unsigned int)((uint64_t)g * a.page_share >> 32), pages_then = (unsigned int)((uint64_t)(g + 1) * a.page_share >> 32);
  if (pages_before == pages_then) {
    const unsigned int unit = (g - pages_before) * kXcds + at;
    turn_queries<D, SRC_BYTES, STREAM>(a, unit);
    return;
  }
  // eight pages' keys, then their values
  const int pool = pages_before & 1;
  const unsigned int page_unit = (pages_before / 2) * kXcds + at;
  int b, page_x;
  if constexpr (!DEAL) {
    b = __builtin_amdgcn_readfirstlane((int)(page_unit / (unsigned int)a.pages));
    page_x = (int)page_unit - b * a.pages;
    if (b >= a.batch) return;
  } else {
    // n tokens lie in at most n / 16 + 2 pages, so trajectory i's begin behind what all before it have at most
    auto start = [&](int i) { return a.q_offsets[i] / kPageSize + 2 * i; };
    b = last_from(a.batch, (int)page_unit, start);
    page_x = (int)page_unit - __builtin_amdgcn_readfirstlane(start(b));
  }
  // (the constant address space: nobody writes lengths or the table during the call, and scalar loads stay out of the rows' way)
  typedef const __attribute__((address_space(4))) int32_t* const_i32_p;
  int n = ((const_i32_p)a.q_lens)[b], len = ((const_i32_p)a.ctx_lens)[b], q_off = ((const_i32_p)a.q_offsets)[b];
  asm volatile("" : "+s"(n), "+s"(len), "+s"(q_off));   // arrived: one wait for all of them
  if (n <= 0) return;
  const int first = len - n, hkv = a.hkv;
  const void* rows = pool ? a.v_new : a.k_new;
  const int64_t stride = pool ? a.v_stride : a.k_stride;
  const int group = (int)threadIdx.x / kLanes, col = (int)threadIdx.x % kLanes;
  const bool rotate = a.cos_sin != nullptr && pool == 0;
  const Lane lane(a, col, rotate);
  const bool turns = lane.turns;
  const int e0 = lane.e0, e1 = lane.e1;
  const int turn_pages = DEAL ? len / kPageSize + 1 : a.pages;   // (one page each where they were searched for)
  for (int page_i = first / kPageSize + page_x; page_i * kPageSize < len; page_i += turn_pages) {
  const bool another = page_i != first / kPageSize + page_x;
  const int lo = max(first, page_i * kPageSize), hi = min(len, (page_i + 1) * kPageSize);
  const int s0 = lo - page_i * kPageSize, slots = hi - lo;
  const int side = kGroups / slots;             // heads under way at a time
  const int slot = group % slots, head0 = group / slots;
  const bool idle = head0 >= side;
  const int64_t token = (int64_t)q_off + lo - first + slot;
  const int64_t page_id = ((const_i32_p)a.page_table)[(size_t)b * a.max_pages + page_i];
  Turn turn;
  if (turns) look_up(a, col * 4, lo + slot, token, turn);
  auto fetch_row = [&](int head) { return fetch<SRC_BYTES>(lane, rows, token * stride + (int64_t)head * D); };
  unsigned char* tile = (unsigned char*)(pool ? a.v_pages : a.k_pages) + (size_t)page_id * hkv * kPageSize * D * (kCodes ? 1 : SRC_BYTES);
  if constexpr (!kCodes) {
    // several heads under way at a time
    if (!idle)
      for (int h = head0; h < hkv; h += kKeep * side) {
        Raw<SRC_BYTES> r[kKeep] = {};
#pragma unroll
        for (int i = 0; i < kKeep; ++i)
          if (h - head0 + i * side < hkv) r[i] = fetch_row(min(h + i * side, hkv - 1));
#pragma unroll
        for (int i = 0; i < kKeep; ++i)
          if (h + i * side < hkv) store<SRC_BYTES, false>(a, lane, turn, tile + ((size_t)(h + i * side) * kPageSize + s0 + slot) * D * SRC_BYTES, r[i]);
      }
  } else {
    static_assert(SRC_BYTES == 2, "codes are made of bf16 rows");
    // of a round's heads: the rows' largest magnitudes; then the old and the new scale (one entry where the scale is the page's)
    __shared__ float row_top[kRound][kGroups];
    __shared__ float old_scale[kMost], new_scale[kMost];
    float* const scales = (pool ? a.v_scale : a.k_scale) + page_id * (kHeadScales ? hkv : 1);
    constexpr float kMax = kInt8 ? kInt8Max : kE4m3Max;
    auto rotated = [&](const Raw<SRC_BYTES>& r, float (&x)[8]) {
      to_float<2>(r, x);
      if (turns) turn.apply(x, a.interleaved);
    };
    auto encode4 = [&](const float* x) { return kInt8 ? encode4_int8(x) : encode4_e4m3(x); };
    auto settled = [&](float amax, float before) {
      float need = amax / kMax;
      if (kHeadScales) need = fmaxf(need, kLeastHeadScale);
      else if (s0 == 0 && !(amax > 0.f)) need = 1.f;
      return s0 == 0 || need > before ? need : before;
    };
    // eight codes at p: code <- enc(dec(code) * old / new)
    auto again8 = [&](unsigned char* at, float before, float now) {
      uintx2* p = (uintx2*)at;
      const uintx2 w = *p;
      float x[8];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if constexpr (kInt8) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[4 * k + e] = (float)(int8_t)(w[k] >> (8 * e));
        } else {
          const floatx2 f0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), f1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
          x[4 * k] = f0[0]; x[4 * k + 1] = f0[1]; x[4 * k + 2] = f1[0]; x[4 * k + 3] = f1[1];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= before;
      Quotients<kHeadScales>(now).divide(x);
      *p = uintx2{encode4(x), encode4(x + 4)};
    };
    // the codes already in slots [0, s0) of `count` heads from `first` on whose scale grew
    auto again = [&](int first, int count) {
      if (!s0) return;
      const int chunks = count * s0 * (D / 8);
      for (int c = threadIdx.x; c < chunks; c += kThreads) {
        const int row = c / (D / 8), at = c % (D / 8);
        const int h = row / s0, i = kHeadScales ? h : 0;
        const float before = old_scale[i], now = new_scale[i];
        if (now > before) again8(tile + ((size_t)(first + h) * kPageSize + row % s0) * D + at * 8, before, now);
      }
    };
    const int round = kRound * side;               // heads of a round
    // the largest magnitude of a row, in all of its lanes; undefined elements count for nothing (the maximum passes over quiet ones
    // only: of a signalling one and what came before it, it forgets the latter, so they are quieted)
    auto largest = [&](const float (&x)[8]) {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, __builtin_canonicalizef(__builtin_fabsf(x[i])));
      int t = __float_as_int(m);                  // (as integers they order the same)
      t = max(t, __builtin_amdgcn_mov_dpp(t, 0xb1, 0xf, 0xf, true));      // the neighbour,
      t = max(t, __builtin_amdgcn_mov_dpp(t, 0x4e, 0xf, 0xf, true));      // ... the other two of four,
      t = max(t, __builtin_amdgcn_mov_dpp(t, 0x141, 0xf, 0xf, true));     // ... the other four of eight,
      if constexpr (kLanes == 16) t = max(t, __builtin_amdgcn_mov_dpp(t, 0x140, 0xf, 0xf, true));
      return __int_as_float(t);
    };
    auto emit = [&](int head, const Raw<SRC_BYTES>& r, float scale) {
      float x[8];
      rotated(r, x);
      Quotients<kHeadScales>(scale).divide(x);
      unsigned char* dst = tile + ((size_t)head * kPageSize + s0 + slot) * D;
      *(unsigned int*)(dst + e0) = encode4(x);
      *(unsigned int*)(dst + e1) = encode4(x + 4);
    };
    if constexpr (kHeadScales) {
      if (slots == 1) {
        // a lone token: a head is one row, whose lanes know all there is to know
        for (int h = head0; h < hkv; h += side) {
          const float before = s0 ? scales[h] : 0.f;
          const Raw<SRC_BYTES> r = fetch_row(h);
          float x[8];
          rotated(r, x);
          const float now = settled(largest(x), before);
          if (s0 && now > before)
            for (int t = 0; t < s0; ++t) again8(tile + ((size_t)h * kPageSize + t) * D + col * 8, before, now);
          emit(h, r, now);
          if (col == 0) scales[h] = now;          // (its lanes read the old one together)
        }
        continue;
      }
      for (int r0 = 0; r0 < hkv; r0 += round) {
        const int count = min(round, hkv - r0);
        float before = 0.f;
        if (s0 && (int)threadIdx.x < count) before = scales[r0 + threadIdx.x];
        if (r0 || another) __syncthreads();
        Raw<SRC_BYTES> keep[kRound] = {};       // (what is not loaded is nothing: else the rows of the round before, all the way)
        if (!idle) {
#pragma unroll
          for (int k = 0; k < kRound; ++k)
            if (k * side < count) keep[k] = fetch_row(r0 + min(head0 + k * side, count - 1));
#pragma unroll
          for (int k = 0; k < kRound; ++k)
            if (k * side < count) {
              float x[8];
              rotated(keep[k], x);
              const float m = largest(x);
              if (col == 0) row_top[k][group] = m;
              __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();
        if ((int)threadIdx.x < count) {
          const int k = (int)threadIdx.x / side, g = ((int)threadIdx.x - k * side) * slots;
          float m = row_top[k][g];
          for (int i = 1; i < slots; ++i) m = fmaxf(m, row_top[k][g + i]);
          const float now = settled(m, before);
          old_scale[threadIdx.x] = s0 ? before : now;
          new_scale[threadIdx.x] = now;
          scales[r0 + threadIdx.x] = now;
        }
        __syncthreads();
        again(r0, count);
        if (!idle) {
          // (turned once more: kept as floats over the barriers, rows would take twice the registers)
#pragma unroll
          for (int k = 0; k < kRound; ++k) asm volatile("" : "+v"(keep[k].lo), "+v"(keep[k].hi));
#pragma unroll
          for (int k = 0; k < kRound; ++k)
            if (head0 + k * side < count) {
              emit(r0 + head0 + k * side, keep[k], new_scale[head0 + k * side]);
              __builtin_amdgcn_sched_barrier(0);
            }
        }
      }
    } else {
      // one scale for the page: the largest magnitude of all heads first
      float before = 0.f;
      if (s0 && threadIdx.x == 0) before = scales[0];
      float most = 0.f;
      if (!idle)
        for (int h = head0; h < hkv; h += side) {
          float x[8];
          rotated(fetch_row(h), x);
          most = fmaxf(most, largest(x));
        }
      if (another) __syncthreads();
      if (col == 0) row_top[0][group] = most;
      __syncthreads();
      if (threadIdx.x == 0) {
        float m = row_top[0][0];
        for (int i = 1; i < kGroups; ++i) m = fmaxf(m, row_top[0][i]);
        const float now = settled(m, before);
        old_scale[0] = s0 ? before : now;
        new_scale[0] = now;
        scales[0] = now;
      }
      __syncthreads();
      again(0, hkv);
      if (!idle)
        for (int h = head0; h < hkv; h += side) emit(h, fetch_row(h), new_scale[0]);
    }
  }
  }
}

template <int D, bool STREAM, bool DEAL>
hipError_t launch_as(const RopeWriteArgs& a, int src_bytes, int pool, dim3 grid, hipStream_t s) {
  if (src_bytes == 4) {
    if (pool != -1) return hipErrorInvalidValue;
    hipLaunchKernelGGL((kv_write_rope_kernel<D, 4, -1, STREAM, DEAL>), grid, dim3(kThreads), 0, s, a);
  } else {
    switch (pool) {
      case -1: hipLaunchKernelGGL((kv_write_rope_kernel<D, 2, -1, STREAM, DEAL>), grid, dim3(kThreads), 0, s, a); break;
      case kKvFp8: hipLaunchKernelGGL((kv_write_rope_kernel<D, 2, kKvFp8, STREAM, DEAL>), grid, dim3(kThreads), 0, s, a); break;
      case kKvFp8Head: hipLaunchKernelGGL((kv_write_rope_kernel<D, 2, kKvFp8Head, STREAM, DEAL>), grid, dim3(kThreads), 0, s, a); break;
      case kKvInt8Head: hipLaunchKernelGGL((kv_write_rope_kernel<D, 2, kKvInt8Head, STREAM, DEAL>), grid, dim3(kThreads), 0, s, a); break;
      default: return hipErrorInvalidValue;
    }
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write_rope(const RopeWriteArgs& args, int32_t max_q_len, int head_dim, int src_bytes, int pool, hipStream_t s) {
  RopeWriteArgs a = args;
  a.one_each = max_q_len == 1 && a.total_q == a.batch;   // (no trajectory has more, so each has one where so many rows are theirs)
  // A run of n tokens touches at most (n + 14) / 16 + 1 pages, wherever it starts: as many workgroups per trajectory as the longest chunk
  // has pages, found by a division.  Small pages: a workgroup costs about as much to start as one's rows do, and most of those for the
  // longest chunk's pages would have nothing to do, so there are as many as the mean chunk has pages, and they take turns.
  // 512 chunks of 64 .. 1024 tokens (8/2/64, int8) 136 -> 123 us, 256 of them with 8/1/128 91.6 -> 89.6, with 8/4/64 78.2 -> 77.6; with 512
  // elements of a token's keys 148 -> 144 or 134 -> 138 (128 chunks of 32 .. 512, 64/4/128), 137 -> 140 (16/8/64), with 1024 109 -> 118 (32/8/128).
  // Where the longest chunk stands out neither will do (511 single tokens and one chunk of 30000, int8: 902 us with the few workgroups of
  // 8/2/64, 819 with the many of 32/8/128; 63 and one of 2000: 21.6), and each workgroup takes the one page that is its own by a search over
  // the chunks: 32, 128 and 13.1 us.  The search costs what two trips to memory do: 300 chunks of 1 .. 512 (bf16) 103.8 -> 105.8, 512 of 2 .. 64
  // (8/2/64) 13.0 -> 14.1, so it is kept for these.
  const int64_t longest = std::min(max_q_len, a.total_q);
  const int64_t pages = longest > 0 ? (longest + kPageSize - 2) / kPageSize + 1 : 1, mean = a.total_q / ((int64_t)kPageSize * a.batch) + 2;
  const bool divided = pages <= kUneven * mean;
  a.pages = !divided ? 0 : (int32_t)((int64_t)a.hkv * head_dim <= kSmallPage ? std::min(pages, mean) : pages);
  const int64_t page_groups = ((divided ? (int64_t)a.pages * a.batch : a.total_q / kPageSize + 2 * (int64_t)a.batch) + kXcds - 1) / kXcds * 2;
  int64_t groups = page_groups;
  bool stream = false;
  if (a.q) {
    // a wave takes so many heads of a token that kKeep rows of each of its lanes hold them, fewer where waves are few
    const int rows = 64 / (head_dim / 8), most = (a.hq + rows - 1) / rows;
    const int64_t parts = std::clamp<int64_t>(kQueryWaves / a.total_q, (most + kKeep - 1) / kKeep, most);
    a.part_heads = (int)((most + parts - 1) / parts) * rows;
    a.head_parts = (a.hq + a.part_heads - 1) / a.part_heads;
    // ... and several tokens where their heads are few and there are waves enough even so
    a.wave_tokens = 1;
    while (2 * a.wave_tokens <= rows && 2 * a.wave_tokens * a.hq <= rows * kKeep && a.total_q / (2 * a.wave_tokens) >= kQueryWaves) a.wave_tokens *= 2;
    stream = (int64_t)a.total_q * a.hq * head_dim * src_bytes > kStreamQueries;
    groups += ((((int64_t)a.total_q + a.wave_tokens - 1) / a.wave_tokens) * a.head_parts + kWaves * kXcds - 1) / (kWaves * kXcds);
  }
  // (a grid of 2^32 threads or more is cut short without an error)
  if (groups * kXcds * kThreads > UINT32_MAX || (int64_t)a.total_q * a.head_parts > INT32_MAX) return hipErrorInvalidValue;
  a.page_share = (((uint64_t)page_groups << 32) + groups - 1) / groups;   // (rounded up: behind the last group there have been them all)
  const dim3 grid((unsigned)(groups * kXcds));
  auto of_dim = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (divided) return stream ? launch_as<D, true, false>(a, src_bytes, pool, grid, s) : launch_as<D, false, false>(a, src_bytes, pool, grid, s);
    return stream ? launch_as<D, true, true>(a, src_bytes, pool, grid, s) : launch_as<D, false, true>(a, src_bytes, pool, grid, s);
  };
  if (head_dim == 128) return of_dim(std::integral_constant<int, 128>{});
  if (head_dim == 64) return of_dim(std::integral_constant<int, 64>{});
  return hipErrorInvalidValue;
}

}  // namespace rollattn
