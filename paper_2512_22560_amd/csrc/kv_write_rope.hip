// KV write with the position rotation on the way: the new tokens' queries and keys are turned to their positions, queries are
// handed back, K and V rows go into the paged cache.  Also the plain write into pools with a scale for each page and KV head.
//
// Rotation of a pair (lo, hi) with the table's c and s: lo' = lo c - hi s, hi' = hi c + lo s, each product and sum one float32
// operation (no fused ones: codes are integers decided by these numbers).  Codes of a page and head: the scale is
// absmax / 448 or / 127 of the head's new rows in the page, never below kLeastHeadScale and, where the page already holds tokens,
// never below the old one; if it grew, the codes already there are quantised again.
//
// One workgroup per (trajectory, page that receives new tokens, and: K, V, or kQueryHeads query heads); the page belongs to that
// trajectory alone, so nothing here needs a global atomic.  A row of D elements is the work of D / 8 lanes, eight elements to a
// lane: two runs of four whose elements are each other's partners, so that a rotation needs no exchange between lanes.  The
// groups of lanes are dealt to the page's new slots first and the rest of them to heads, so that a lane keeps its slot, and with
// it the cosines and sines of its token, over all heads it walks.
#include "codes_device.h"

namespace rollattn {

namespace {

constexpr int kThreads = 256;
constexpr int kQueryHeads = 16;   // query heads per workgroup
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
  const int page_i = first / kPageSize + blockIdx.x;
  if (n <= 0 || page_i * kPageSize >= len) return;
  const int lo = max(first, page_i * kPageSize), hi = min(len, (page_i + 1) * kPageSize);
  const int s0 = lo - page_i * kPageSize, slots = hi - lo;
  const int group = (int)threadIdx.x / kLanes, col = (int)threadIdx.x % kLanes;
  const int side = kGroups / slots;             // heads under way at a time
  const int slot = group % slots, head0 = group / slots;
  const bool idle = head0 >= side;
  const int64_t token = (int64_t)q_off + lo - first + slot;
  const bool rotate = a.cos_sin != nullptr && blockIdx.z != 1;
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
    constexpr int kBatch = 4;
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

  if (blockIdx.z >= 2) {
    const int h0 = ((int)blockIdx.z - 2) * kQueryHeads;
    copy(a.q, a.q_stride, h0, min(h0 + kQueryHeads, a.hq),
         [&](int h) { return (unsigned char*)a.q_out + (token * a.hq + h) * D * SRC_BYTES; });
    return;
  }
  const int pool = blockIdx.z, hkv = a.hkv;
  const void* rows = pool ? a.v_new : a.k_new;
  const int64_t stride = pool ? a.v_stride : a.k_stride;
  const int64_t page_id = a.page_table[(size_t)b * a.max_pages + page_i];
  unsigned char* tile = (unsigned char*)(pool ? a.v_pages : a.k_pages) + (size_t)page_id * hkv * kPageSize * D * (kCodes ? 1 : SRC_BYTES);
  if constexpr (!kCodes) {
    copy(rows, stride, 0, hkv, [&](int h) { return tile + ((size_t)h * kPageSize + s0 + slot) * D * SRC_BYTES; });
  } else {
    static_assert(SRC_BYTES == 2, "codes are made of bf16 rows");
    // of a round's heads (one entry where the scale is the page's): largest magnitude, then the old and the new scale
    __shared__ unsigned int top[kMost];
    __shared__ float old_scale[kMost], new_scale[kMost];
    float* const scales = (pool ? a.v_scale : a.k_scale) + page_id * (kHeadScales ? hkv : 1);
    constexpr float kMax = kInt8 ? kInt8Max : kE4m3Max;
    auto rotated = [&](int head, float (&x)[8]) {
      to_float<2>(fetch(rows, stride, head), x);
      if (col < rotating) turn.apply(x, a.interleaved);
    };
    auto encode4 = [&](const float* x) { return kInt8 ? encode4_int8(x) : encode4_e4m3(x); };
    // of `count` scales from `first` on: each thread one
    auto settle = [&](int first, int count) {
      for (int i = threadIdx.x; i < count; i += kThreads) {
        const float amax = __uint_as_float(top[i]);
        float need = amax / kMax;
        if (kHeadScales) need = fmaxf(need, kLeastHeadScale);
        else if (s0 == 0 && !(amax > 0.f)) need = 1.f;
        const float before = s0 ? scales[first + i] : need;
        old_scale[i] = before;
        new_scale[i] = need > before ? need : before;
        scales[first + i] = new_scale[i];
      }
    };
    // the codes already in slots [0, s0) of `count` heads from `first` on whose scale grew: code <- enc(dec(code) * old / new)
    auto again = [&](int first, int count) {
      if (!s0) return;
      const int chunks = count * s0 * (D / 8);
      for (int c = threadIdx.x; c < chunks; c += kThreads) {
        const int row = c / (D / 8), at = c % (D / 8);
        const int h = row / s0, i = kHeadScales ? h : 0;
        const float before = old_scale[i], now = new_scale[i];
        if (!(now > before)) continue;
        uintx2* p = (uintx2*)(tile + ((size_t)(first + h) * kPageSize + row % s0) * D + at * 8);
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
      }
    };
    const int round = kKeep * side;               // heads of a round
    auto largest = [&](const float (&x)[8]) {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, __builtin_fabsf(x[i]));
      return __float_as_uint(m);
    };
    auto emit = [&](int head, float (&x)[8], float scale) {
      Quotients(scale).divide(x);
      unsigned char* dst = tile + ((size_t)head * kPageSize + s0 + slot) * D;
      *(unsigned int*)(dst + e0) = encode4(x);
      *(unsigned int*)(dst + e1) = encode4(x + 4);
    };
    if constexpr (kHeadScales) {
      for (int r0 = 0; r0 < hkv; r0 += round) {
        const int count = min(round, hkv - r0);
        if (r0) __syncthreads();
        for (int i = threadIdx.x; i < count; i += kThreads) top[i] = 0;
        __syncthreads();
        float x[kKeep][8];
        if (!idle) {
#pragma unroll
          for (int k = 0; k < kKeep; ++k)
            if (head0 + k * side < count) {
              rotated(r0 + head0 + k * side, x[k]);
              atomicMax(&top[head0 + k * side], largest(x[k]));
            }
        }
        __syncthreads();
        settle(r0, count);
        __syncthreads();
        again(r0, count);
        if (!idle) {
#pragma unroll
          for (int k = 0; k < kKeep; ++k)
            if (head0 + k * side < count) emit(r0 + head0 + k * side, x[k], new_scale[head0 + k * side]);
        }
      }
    } else {
      // one scale for the page: the largest magnitude of all heads first
      if (threadIdx.x == 0) top[0] = 0;
      __syncthreads();
      unsigned int most = 0;
      float x[8];
      if (!idle)
        for (int h = head0; h < hkv; h += side) {
          rotated(h, x);
          most = max(most, largest(x));
        }
      atomicMax(&top[0], most);
      __syncthreads();
      settle(0, 1);
      __syncthreads();
      again(0, hkv);
      if (!idle)
        for (int h = head0; h < hkv; h += side) {
          rotated(h, x);
          emit(h, x, new_scale[0]);
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

hipError_t launch_kv_write_rope(const RopeWriteArgs& a, int32_t batch, int32_t max_q_len, int head_dim, int src_bytes, int pool,
                                hipStream_t s) {
  // a run of n tokens touches at most this many pages, wherever it starts
  const unsigned pages = max_q_len > 0 ? (unsigned)(((int64_t)max_q_len + kPageSize - 2) / kPageSize + 1) : 1;
  const unsigned queries = a.q ? (unsigned)((a.hq + kQueryHeads - 1) / kQueryHeads) : 0;
  const dim3 grid(pages, (unsigned)batch, 2 + queries);
  if (head_dim == 128) return launch_d<128>(a, src_bytes, pool, grid, s);
  if (head_dim == 64) return launch_d<64>(a, src_bytes, pool, grid, s);
  return hipErrorInvalidValue;
}

}  // namespace rollattn
