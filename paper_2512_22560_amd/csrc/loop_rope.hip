// KV write with the position rotation on the way: the new tokens' queries and keys are turned to their positions, queries are
// handed back, K and V rows go into the paged cache.  Also the plain write into pools with a scale for each page and KV head.
//
// Rotation of a pair (lo, hi) with the table's c and s: lo' = lo c - hi s, hi' = hi c + lo s, each product and sum one float32
// operation (no fused ones: codes are integers decided by these numbers).  Codes of a page and head: the scale is
// absmax / 448 or / 127 of the head's new rows in the page, never below kLeastHeadScale and, where the page already holds tokens,
// never below the old one; if it grew, the codes already there are quantised again.
//
// One workgroup per (trajectory, page that receives new tokens, and: K, V, or some of the query heads); the page belongs to that
// trajectory alone, so nothing here needs a global atomic.  A row of D elements is the work of D / 8 lanes, eight elements to a
// lane: two runs of four whose elements are each other's partners, so that a rotation needs no exchange between lanes.  The
// groups of lanes are dealt to the page's new slots first and the rest of them to heads, so that a lane keeps its slot, and with
// it the cosines and sines of its token, over all heads it walks.
#include <algorithm>

#include "codes_device.h"

namespace rollattn {

namespace {

constexpr int kThreads = 256;
constexpr int kQueryRows = 256;   // (token, query head) rows per workgroup
constexpr int kKeep = 8;          // heads of a lane that are held at once

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

// POOL: -1 the source type, else a KvKind
template <int D, int SRC_BYTES, int POOL>
__global__ __launch_bounds__(kThreads) void kv_write_rope_kernel(const RopeWriteArgs a) {
  constexpr bool kCodes = POOL >= 0, kHeadScales = kCodes && kv_has_head_scales(POOL);
  constexpr bool kInt8 = POOL == kKvInt8Head;
  constexpr int kLanes = D / 8;                 // lanes of a row
  constexpr int kGroups = kThreads / kLanes;    // rows under way at a time
  constexpr int kMost = kKeep * kGroups;        // heads of a round, at most
  const int b = blockIdx.y;
  int n = a.q_lens[b], len = a.ctx_lens[b], q_off = a.q_offsets[b];
  asm volatile("" : "+s"(n), "+s"(len), "+s"(q_off));   // arrived: one wait for all of them
  const int first = len - n;
  const int bx = (int)(blockIdx.x / (unsigned)a.parts);
  const int part = (int)((blockIdx.x + ROT) % (unsigned)a.parts);   // 0: K, 1: V, then query heads
  if (n <= 0) return;
  for (int page_i = first / kPageSize + bx; page_i * kPageSize < len; page_i += gridDim.x / a.parts) {
  const int lo = max(first, page_i * kPageSize), hi = min(len, (page_i + 1) * kPageSize);
  const int s0 = lo - page_i * kPageSize, slots = hi - lo;
  const int group = (int)threadIdx.x / kLanes, col = (int)threadIdx.x % kLanes;
  const int side = kGroups / slots;             // heads under way at a time
  const int slot = group % slots, head0 = group / slots;
  const bool idle = head0 >= side;
  const int64_t token = (int64_t)q_off + lo - first + slot;
  const bool rotate = a.cos_sin != nullptr && part != 1;
  const int rotating = rotate ? a.rot_dim / 8 : 0;      // lanes of a row that hold pairs
  int e0 = col * 8, e1 = e0 + 4;                        // where the lane's two runs of four start
  if (!a.interleaved && col < rotating) {
    e0 = col * 4;
    e1 = e0 + a.rot_dim / 2;
  }
  Turn turn;
  if (col < rotating) {
    const int half = a.rot_dim / 2, j = col * 4;
    const unsigned int last = (unsigned int)a.num_positions - 1;
    if (!a.positions) {
      const float* row = a.cos_sin + (size_t)min((unsigned int)(lo + slot), last) * a.rot_dim + j;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        turn.c[i] = row[i];
        turn.s[i] = row[half + i];
      }
    } else {
      const unsigned int word = a.pair_axes[j / 16] >> (j % 16 * 2);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int axis = word >> (2 * i) & 3;
        const float* row = a.cos_sin + (size_t)min((unsigned int)a.positions[(int64_t)axis * a.total_q + token], last) * a.rot_dim + j + i;
        turn.c[i] = row[0];
        turn.s[i] = row[half];
      }
    }
  }
  auto fetch = [&](const void* rows, int64_t stride, int head) {
    const unsigned char* p = (const unsigned char*)rows + (token * stride + (int64_t)head * D) * SRC_BYTES;
    Raw<SRC_BYTES> r;
    r.lo = *(const typename Raw<SRC_BYTES>::half*)(p + e0 * SRC_BYTES);
    r.hi = *(const typename Raw<SRC_BYTES>::half*)(p + e1 * SRC_BYTES);
    return r;
  };
  // A row of the source type, at p.
  auto store = [&](void* p, Raw<SRC_BYTES> r) {
    if (col < rotating) {
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
    *(typename Raw<SRC_BYTES>::half*)((unsigned char*)p + e0 * SRC_BYTES) = r.lo;
    *(typename Raw<SRC_BYTES>::half*)((unsigned char*)p + e1 * SRC_BYTES) = r.hi;
  };
  // All heads of `heads` from h0 on, several under way at a time, from rows to where at(head) says.
  auto copy = [&](const void* rows, int64_t stride, int h0, int heads, auto&& at) {
    constexpr int kBatch = 8;
    if (idle) return;
    for (int h = h0 + head0; h < heads; h += kBatch * side) {
      Raw<SRC_BYTES> r[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) r[i] = fetch(rows, stride, min(h + i * side, heads - 1));
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (h + i * side < heads) store(at(h + i * side), r[i]);
    }
  };

  if (part >= 2) {
    const int h0 = (part - 2) * a.query_heads;
    copy(a.q, a.q_stride, h0, min(h0 + a.query_heads, a.hq),
         [&](int h) { return (unsigned char*)a.q_out + (token * a.hq + h) * D * SRC_BYTES; });
    continue;
  }
  const bool again_here = page_i != first / kPageSize + bx;
  const int pool = part, hkv = a.hkv;
  const void* rows = pool ? a.v_new : a.k_new;
  const int64_t stride = pool ? a.v_stride : a.k_stride;
  const int64_t page_id = a.page_table[(size_t)b * a.max_pages + page_i];
  unsigned char* tile = (unsigned char*)(pool ? a.v_pages : a.k_pages) + (size_t)page_id * hkv * kPageSize * D * (kCodes ? 1 : SRC_BYTES);
  if constexpr (!kCodes) {
    copy(rows, stride, 0, hkv, [&](int h) { return tile + ((size_t)h * kPageSize + s0 + slot) * D * SRC_BYTES; });
  } else {
    static_assert(SRC_BYTES == 2, "codes are made of bf16 rows");
    // of a round's heads: the rows' largest magnitudes; then the old and the new scale (one entry where the scale is the page's)
    __shared__ float row_top[kKeep][kGroups];
    __shared__ float old_scale[kMost], new_scale[kMost];
    float* const scales = (pool ? a.v_scale : a.k_scale) + page_id * (kHeadScales ? hkv : 1);
    constexpr float kMax = kInt8 ? kInt8Max : kE4m3Max;
    auto rotated = [&](const Raw<SRC_BYTES>& r, float (&x)[8]) {
      to_float<2>(r, x);
      if (col < rotating) turn.apply(x, a.interleaved);
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
      for (int e = 0; e < 8; ++e) x[e] = (x[e] * before) / now;
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
    const int round = kKeep * side;               // heads of a round
    // the largest magnitude of a row, in all of its lanes
    auto largest = [&](const float (&x)[8]) {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, __builtin_fabsf(x[i]));
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
      Quotients(scale).divide(x);
      unsigned char* dst = tile + ((size_t)head * kPageSize + s0 + slot) * D;
      *(unsigned int*)(dst + e0) = encode4(x);
      *(unsigned int*)(dst + e1) = encode4(x + 4);
    };
    if constexpr (kHeadScales) {
      if (slots == 1) {
        // a lone token: a head is one row, whose lanes know all there is to know
        for (int h = head0; h < hkv; h += side) {
          const float before = s0 ? scales[h] : 0.f;
          const Raw<SRC_BYTES> r = fetch(rows, stride, h);
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
        if (r0 || again_here) __syncthreads();
        Raw<SRC_BYTES> keep[kKeep];
        if (!idle) {
#pragma unroll
          for (int k = 0; k < kKeep; ++k)
            if (k * side < count) keep[k] = fetch(rows, stride, r0 + min(head0 + k * side, count - 1));
#pragma unroll
          for (int k = 0; k < kKeep; ++k)
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
          for (int k = 0; k < kKeep; ++k) asm volatile("" : "+v"(keep[k].lo), "+v"(keep[k].hi));
#pragma unroll
          for (int k = 0; k < kKeep; ++k)
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
          rotated(fetch(rows, stride, h), x);
          most = fmaxf(most, largest(x));
        }
      if (again_here) __syncthreads();
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
        for (int h = head0; h < hkv; h += side) emit(h, fetch(rows, stride, h), new_scale[0]);
    }
  }
  }
}

template <int D>
hipError_t launch_d(const RopeWriteArgs& a, int src_bytes, int pool, dim3 grid, hipStream_t s) {
  if (src_bytes == 4) {
    if (pool != -1) return hipErrorInvalidValue;
    hipLaunchKernelGGL((kv_write_rope_kernel<D, 4, -1>), grid, dim3(kThreads), 0, s, a);
  } else {
    switch (pool) {
      case -1: hipLaunchKernelGGL((kv_write_rope_kernel<D, 2, -1>), grid, dim3(kThreads), 0, s, a); break;
      case kKvFp8: hipLaunchKernelGGL((kv_write_rope_kernel<D, 2, kKvFp8>), grid, dim3(kThreads), 0, s, a); break;
      case kKvFp8Head: hipLaunchKernelGGL((kv_write_rope_kernel<D, 2, kKvFp8Head>), grid, dim3(kThreads), 0, s, a); break;
      case kKvInt8Head: hipLaunchKernelGGL((kv_write_rope_kernel<D, 2, kKvInt8Head>), grid, dim3(kThreads), 0, s, a); break;
      default: return hipErrorInvalidValue;
    }
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write_rope(const RopeWriteArgs& args, int32_t batch, int32_t max_q_len, int head_dim, int src_bytes, int pool,
                                hipStream_t s) {
  RopeWriteArgs a = args;
  // a run of n tokens touches at most this many pages, wherever it starts
  const unsigned pages = max_q_len > 0 ? (unsigned)(((int64_t)max_q_len + kPageSize - 2) / kPageSize + 1) : 1;
  a.query_heads = kQueryRows / std::clamp(max_q_len, 1, kPageSize);
  const unsigned queries = a.q ? (unsigned)((a.hq + a.query_heads - 1) / a.query_heads) : 0;
  a.parts = 2 + (int)queries;
  const unsigned mean = (unsigned)(a.total_q / (kPageSize * batch)) + EXTRA;
  const dim3 grid(std::min(pages, mean) * a.parts, (unsigned)batch);
  if (head_dim == 128) return launch_d<128>(a, src_bytes, pool, grid, s);
  if (head_dim == 64) return launch_d<64>(a, src_bytes, pool, grid, s);
  return hipErrorInvalidValue;
}

}  // namespace rollattn
