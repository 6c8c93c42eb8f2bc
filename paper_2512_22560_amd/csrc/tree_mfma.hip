// Attention of a tree of drafted tokens (bf16 queries) over bf16 or 8-bit (E4M3, int8) paged KV (gfx950).
//
// A row is (trajectory, KV head, tile of 32 or 64 query rows): a query row is a (drafted token, query head of the group) pair,
// token-major, so the heads that share the KV head and the tokens of a draft that fit one tile read K and V once.  As in decode, rows
// are cut into 32-token blocks, laid end to end, and every wave is a worker with one equal run of that sequence; it streams its run
// from memory straight into a private ring of LDS tiles, without any barrier, and consumes a block with
//   S^T = K Q^T          (tokens x query rows, v_mfma_f32_32x32x16, K rows as A; one LDS read for all query rows)
//   O^T += V^T P^T       (dims x query rows, V read back transposed with ds_read_b64_tr_*; one read for all query rows)
// A run that covers a whole row writes the row's output itself; one that starts or ends inside a row leaves an un-normalised partial
// (max, sum, O) for the merge.
// A block that lies in the cached prefix is seen whole by every row and knows no mask.  In the blocks behind it a row sees the tokens
// whose bits are set in its mask words, eight tokens at a time.  What a row does not see must not reach it: a score is replaced before
// the maximum, and where values of such a block are not finite (zero times infinity would not be zero) they are added apart to the rows
// that see them, and leave the second product.
// Codes become operands as in decode: see decode_mfma.hip for the range of f16 and the power of two per query row.
#include "stream_tiles.h"

namespace rollattn {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kRows = kTreeTileRows;      // query rows of one product

__device__ __forceinline__ floatx16 mfma32(bf16x8 x, bf16x8 y, floatx16 z) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ floatx16 mfma32(halfx8 x, halfx8 y, floatx16 z) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, z, 0, 0, 0); }

// Row t of an S^T tile holds this token of its 16-token group: the middle two quads are swapped, so that the 8 scores a lane ends up with
// are 8 consecutive tokens.
__device__ __forceinline__ int tau(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

// Which 16-byte column a logical chunk of token row t lands in.
template <int D, bool FP8>
__device__ __forceinline__ int tree_key_k(int t) { return FP8 ? t / (256 / D) & (D / 16 - 1) : t & 15; }
template <bool FP8>
__device__ __forceinline__ int tree_key_v(int t) { return FP8 ? t & 7 : (t & 3) << 2; }

// Bits of tokens [rel, rel + 8) of a draft of n tokens, for a row whose words are at `words`; before the draft: `before`.
__device__ __forceinline__ unsigned int seen_bits(const uint64_t* words, int n_words, int rel, int n, unsigned int before) {
  if (rel <= -8) return before;
  const int first = max(rel, 0), w = first >> 6, shift = first & 63;
  uint64_t bits = w < n_words ? words[w] >> shift : 0;
  if (shift > 56 && w + 1 < n_words) bits |= words[w + 1] << (64 - shift);
  const int live = n - first;                        // tokens from `first` on
  bits &= live >= 8 ? 0xffull : live > 0 ? (1ull << live) - 1 : 0ull;
  unsigned int x = (unsigned int)bits;
  if (rel < 0) x = x << -rel | (before & ((1u << -rel) - 1));
  return x & 0xff;
}

// Whether any element of a word of a pool is no number (infinite and undefined bf16 values, the undefined code of E4M3).
template <int KV>
__device__ __forceinline__ bool undefined(uint32_t w) {
  if constexpr (KV == kKvBf16) return (w & 0x7f800000u) == 0x7f800000u || (w & 0x7f80u) == 0x7f80u;
  else if constexpr (KV == kKvInt8Head) return false;
  else return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
}

// The word with zeros in the place of those.
template <int KV>
__device__ __forceinline__ uint32_t defined(uint32_t w) {
  if constexpr (KV == kKvBf16) {
    if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
    if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
    return w;
  } else {
    const uint32_t met = (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;   // one in each undefined byte
    return w & ~(met * 255u);
  }
}

// The lengths of one trajectory, the same in all lanes.
struct Draft {
  int n, len, off;
  __device__ __forceinline__ Draft(const TreeArgs& a, int b) {
    typedef const __attribute__((address_space(4))) int32_t* const_i32_p;
    n = ((const_i32_p)a.q_lens)[b];
    len = ((const_i32_p)a.ctx_lens)[b];
    off = ((const_i32_p)a.q_offsets)[b];
  }
};

// Where query row j of a tile belongs: node and output row.
struct RowAt {
  int node;
  size_t out;
  __device__ __forceinline__ RowAt(const TreeArgs& a, const Draft& d, int g, int j) {
    node = j / a.group;
    out = (size_t)(d.off + node) * a.hq + (size_t)g * a.group + (j - node * a.group);
  }
};

// Blocks of a wave's ring, the one in work included.  A wave of 64 query rows has a SIMD to itself (accumulators alone are 128 registers of
// 512) and a quarter of the LDS, waves of 32 are two to a SIMD.
template <bool FP8, int RT>
constexpr int kTreeSlots = RT == 2 ? (FP8 ? 4 : 2) : (FP8 ? 2 : 1);
template <int D, bool FP8, int RT>
struct TreeLds {
  typedef Geo<D, FP8> G_;
  __attribute__((aligned(1024))) unsigned char k[kTreeSlots<FP8, RT>][G_::kTileBytes], v[kTreeSlots<FP8, RT>][G_::kTileBytes];
  float scales[FP8 ? kTreeSlots<FP8, RT> : 1][FP8 ? 64 : 4];   // of a block's two pages: K's, V's (the other lanes' are copies)
};

// One run of n_mine blocks from block blk of row (b, r) on.
// Loads.  The tiles of block i + slots go into the places of block i, K's as soon as the first product has read them and V's behind the
// second.  HBM -> LDS without a register stop: lane l's 16 bytes land at M0 + 16 l, so a row's chunks are swizzled by the address a lane
// reads from.  The compiler does not see these loads as loads; they are awaited by count: vector-memory counts go down in order, so
// with N of these loads sent after the ones that are waited for, no more than N outstanding operations of any kind means that those have
// landed (others in between only make the wait longer).
template <int D, int KV, int RT, bool STREAM>
__device__ __forceinline__ void tree_worker(const TreeArgs& a, int b0, int r0, int blk0, int n_mine, int worker, TreeLds<D, kv_is_codes(KV), RT>& lds) {
  constexpr bool FP8 = kv_is_codes(KV), HEAD = kv_has_head_scales(KV);   // FP8: 8-bit codes of either kind
  constexpr bool INT8 = KV == kKvInt8Head;
  constexpr int kTile = kRows * RT, kSlots = kTreeSlots<FP8, RT>;
  constexpr int kKK = D / 16, kDT = D / 32;
  using kx8 = std::conditional_t<INT8, halfx8, bf16x8>;   // operands of the first product
  using opx8 = std::conditional_t<HEAD, halfx8, bf16x8>;  // ... and of the second
  using op = std::conditional_t<HEAD, _Float16, __bf16>;
  using G_ = Geo<D, FP8>;
  constexpr int kKLoads = G_::kLoads + (FP8 ? 1 : 0);      // loads of a block's K tile and scales
  const int lane = lane_id();
  const int n32 = lane & 31;   // query row (B column) / K token row (A row) carried by this lane
  const int h2 = lane >> 5;    // half of the contraction this lane feeds

  const int group = a.group, hkv = a.hkv, n_rt = a.row_tiles, rows_per_b = hkv * n_rt;
  const size_t tile_stride = (size_t)kPageSize * G_::kRowBytes;   // bytes of one (page, head) tile
  const bool flip = a.scale_log2 < 0.f;                           // (queries the other way round, so that larger scores are larger exponents)
  const float scale_log2 = __builtin_fabsf(a.scale_log2);

  struct Cursor { int b, r, blk, n, len; };   // trajectory, row within it, block within the row; blocks in the row, context length
  auto blocks_of = [&](int len) { return (len + kBlockTokens - 1) / kBlockTokens; };
  Cursor pc{b0, r0, blk0, 0, 0};              // producer: next block to request from HBM
  pc.len = Draft(a, b0).len;
  pc.n = blocks_of(pc.len);
  Cursor cc = pc;                             // consumer: block being computed
  auto advance = [&](Cursor& c) {
    if (++c.blk < c.n) return;
    c.blk = 0;
    if (++c.r < rows_per_b) return;
    c.r = 0;
    for (;;) {
      const Draft d(a, ++c.b);
      c.len = d.n > 0 ? d.len : 0;
      if (c.len) break;
    }
    c.n = blocks_of(c.len);
  };

  // ---- producer: a window of 64 page ids (32 blocks) of the current row, one per lane
  int pwin = -1, pid_vec = 0, pid_next = 0, issued = 0;
  int p_page[2] = {0, 0}, p_g = 0, p_lim = 0;         // the block under way: pages, KV head, and tokens of it that are there
  auto load_window = [&](int k) {
    const int pg = k * 64 + lane;
    return (pg < ((pc.len + kPageSize - 1) >> 4)) ? a.page_table[(size_t)pc.b * a.max_pages + pg] : 0;
  };
  auto dma16 = [&](const unsigned char* base, unsigned int off, const void* dst) __attribute__((always_inline)) {
    const unsigned int m0 = __builtin_amdgcn_readfirstlane((unsigned int)(uintptr_t)dst);
    if constexpr (STREAM) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(m0), "v"(off), "s"(base) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(m0), "v"(off), "s"(base) : "memory");
  };
  // a tile of one pool: row row0 + lane / chunks of the block per load; rows at or past L_b read its last one again
  auto load_tile = [&](const void* pool, auto key_of, unsigned char* dst) __attribute__((always_inline)) {
    const unsigned char* tile[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) tile[i] = (const unsigned char*)pool + (size_t)(unsigned int)__builtin_amdgcn_readfirstlane(p_page[i] * hkv + p_g) * tile_stride;
    const int c = lane % G_::kChunks, sub = lane / G_::kChunks;
#pragma unroll
    for (int j = 0; j < G_::kLoads; ++j) {
      const int row0 = j * G_::kRowsPerLoad, row = row0 + sub;
      int slot = row % kPageSize;
      if (p_lim < kBlockTokens) slot = min(row, p_lim - 1) % kPageSize;      // (the row's last block alone)
      dma16(tile[row0 / kPageSize], slot * G_::kRowBytes + ((c ^ key_of(row)) & (G_::kChunks - 1)) * 16, dst + j * 1024);
    }
  };
  // what block pc of the run needs, then its K tile and scales; its V tile
  auto issue_k = [&](int slot) __attribute__((always_inline)) {
    const int k = pc.blk >> 5;
    if (k != pwin) {
      pid_vec = (pwin >= 0 && k == pwin + 1) ? pid_next : load_window(k);
      pid_next = load_window(k + 1);
      pwin = k;
    }
    p_g = pc.r / n_rt;
    p_lim = min(pc.len - pc.blk * kBlockTokens, kBlockTokens);
    p_page[0] = __builtin_amdgcn_readlane(pid_vec, ((pc.blk & 31) << 1));
    p_page[1] = p_lim > kPageSize ? __builtin_amdgcn_readlane(pid_vec, ((pc.blk & 31) << 1) + 1) : p_page[0];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (what this overwrites has been read)
    load_tile(a.k_pages, [](int row) { return tree_key_k<D, FP8>(row); }, lds.k[slot]);
    if constexpr (FP8) {
      const int page = lane & 1 ? p_page[1] : p_page[0];
      const float* from = (lane & 2 ? a.v_scale : a.k_scale) + (HEAD ? (size_t)page * hkv + p_g : (size_t)page);
      const unsigned int m0 = __builtin_amdgcn_readfirstlane((unsigned int)(uintptr_t)lds.scales[slot]);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(m0), "v"(from) : "memory");
    }
  };
  auto issue_v = [&](int slot) __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    load_tile(a.v_pages, [](int row) { return tree_key_v<FP8>(row); }, lds.v[slot]);
    // step to the next block of the run (never past its end: the rows after the last block need not exist); a new row starts with a
    // fresh page-id window
    if (++issued < n_mine) {
      const int row_before = pc.b * rows_per_b + pc.r;
      advance(pc);
      if (pc.b * rows_per_b + pc.r != row_before) pwin = -1;
    }
  };
  // until all but the loads of `pairs` blocks, and kMore others, have landed
  auto await = [&](int pairs, auto more_c) __attribute__((always_inline)) {
    constexpr int kMore = decltype(more_c)::value, kPair = G_::kLoads + kKLoads;
    if (kSlots > 3 && pairs == 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kSlots > 3 ? 3 * kPair + kMore : 0) : "memory");
    else if (kSlots > 2 && pairs == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kSlots > 2 ? 2 * kPair + kMore : 0) : "memory");
    else if (kSlots > 1 && pairs == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kSlots > 1 ? kPair + kMore : 0) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMore) : "memory");
  };

  // ---- consumer state
  kx8 qop[RT][kKK];          // Q^T as the B operand: lane (row n32, half h2), 8 dims per step
  float q_unit[RT];          // int8: what a unit of this lane's row is worth
  floatx16 acc[RT][kDT];     // O^T: lane (row n32, half h2) holds dims dt*32 + (i/4)*8 + h2*4 + i%4
  float m_run[RT], l_run[RT];// running max (log2 units) of this lane's rows, its share of the running sums
  int seg_first_blk = 0;     // block of the row at which the current segment started
  bool first_segment = true, dirty = false;   // dirty: values of the segment that are no numbers have been left out of its sums
  int rows_here = 0, prefix = 0, n_b = 0, q_off = 0, j0 = 0, g = 0;   // of the consumer's row

  auto begin_segment = [&]() __attribute__((always_inline)) {
    const Draft d(a, cc.b);
    g = cc.r / n_rt;
    j0 = (cc.r - g * n_rt) * kTile;
    n_b = d.n;
    q_off = d.off;
    prefix = d.len - d.n;
    rows_here = min(kTile, d.n * group - j0);        // (none: a tile that only longer drafts have)
#pragma unroll
    for (int c = 0; c < RT; ++c) {
      // (rows past the last read it again; what becomes of them is not stored)
      const RowAt at(a, d, g, max(0, min(j0 + c * kRows + n32, d.n * group - 1)));
      const __bf16* qrow = (const __bf16*)a.q + at.out * D;
#pragma unroll
      for (int kk = 0; kk < kKK; ++kk) {
        // FP8: 16-byte K chunks hold 16 dims; step 2p+e uses bytes e*8.. of chunk p*2+h2
        uint4 v = *(const uint4*)(qrow + (FP8 ? ((kk >> 1) * 2 + h2) * 16 + (kk & 1) * 8 : kk * 16 + h2 * 8));
        const uint32_t sign = flip ? 0x80008000u : 0u;
        v.x ^= sign; v.y ^= sign; v.z ^= sign; v.w ^= sign;
        qop[c][kk] = __builtin_bit_cast(kx8, v);     // (int8: as it came, until all of the row is there)
      }
      q_unit[c] = scale_log2;
      if constexpr (INT8) {
        float top = 0.f;
#pragma unroll
        for (int kk = 0; kk < kKK; ++kk) {
          const bf16x8 v = __builtin_bit_cast(bf16x8, qop[c][kk]);
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, __builtin_fabsf((float)v[e]));
        }
        const int up = kQueryBits - __builtin_amdgcn_frexp_expf(xor32_max(top));
#pragma unroll
        for (int kk = 0; kk < kKK; ++kk) {
          const bf16x8 v = __builtin_bit_cast(bf16x8, qop[c][kk]);
#pragma unroll
          for (int e = 0; e < 8; ++e) qop[c][kk][e] = (_Float16)__builtin_amdgcn_ldexpf((float)v[e], up);
        }
        q_unit[c] = __builtin_amdgcn_ldexpf(scale_log2, -up);
      }
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c][dt][i] = 0.f;
      m_run[c] = -INFINITY;
      l_run[c] = 0.f;
    }
    seg_first_blk = cc.blk;
    dirty = false;
  };
  auto end_segment = [&]() __attribute__((always_inline)) {
    const bool whole = seg_first_blk == 0 && cc.blk == cc.n - 1;
    const size_t slot = (size_t)worker * 2 + (first_segment ? 0 : 1);
    const Draft d(a, cc.b);
#pragma unroll
    for (int c = 0; c < RT; ++c) {
      if (c * kRows >= rows_here) break;
      const float l_tot = xor32_add(l_run[c]);
      if (whole) {
        // the whole row was ours: normalise and store
        const bool ok = c * kRows + n32 < rows_here;
        const RowAt at(a, d, g, max(0, min(j0 + c * kRows + n32, d.n * group - 1)));
        const float inv = l_tot > 0.f ? 1.f / l_tot : l_tot;   // (nothing seen: a row of zeros)
        if (a.lse && ok && h2 == 0) a.lse[at.out] = m_run[c] + __builtin_amdgcn_logf(l_tot);
        __bf16* dst = (__bf16*)a.out + at.out * D + h2 * 4;
        if (ok) {
#pragma unroll
          for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
              bf16x4 pk;
#pragma unroll
              for (int e = 0; e < 4; ++e) pk[e] = (__bf16)(acc[c][dt][i4 * 4 + e] * inv);
              *(bf16x4*)(dst + dt * 32 + i4 * 8) = pk;
            }
        }
      } else {
        float* dst = a.partial_o + (slot * RT + c) * (kRows * D) + lane * 4;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4)
            *(floatx4*)(dst + (dt * 4 + i4) * 256) = floatx4{acc[c][dt][i4 * 4], acc[c][dt][i4 * 4 + 1], acc[c][dt][i4 * 4 + 2], acc[c][dt][i4 * 4 + 3]};
        if (h2 == 0) *(floatx2*)(a.partial_ml + ((slot * RT + c) * kRows + n32) * 2) = floatx2{m_run[c], l_tot};
      }
    }
    if (!INT8 && dirty) {
      // rare, and one token after the other: each lane adds to the values that it has just stored
      for (int c = 0; c < RT; ++c) {
        if (c * kRows + n32 >= rows_here) break;
        const RowAt at(a, d, g, j0 + c * kRows + n32);
        const uint64_t* const words = a.mask + (size_t)(d.off + at.node) * a.mask_words;
        for (int t = max(prefix, seg_first_blk * kBlockTokens); t < min(d.len, (cc.blk + 1) * kBlockTokens); ++t) {
          const int rel = t - prefix;
          if (rel >= 64 * a.mask_words || !(words[rel >> 6] >> (rel & 63) & 1)) continue;
          const size_t row = ((size_t)a.page_table[(size_t)cc.b * a.max_pages + t / kPageSize] * hkv + g) * kPageSize + t % kPageSize;
          for (int dim = h2 * 4; dim < D; dim += 8) {
            float x[4];
            if constexpr (FP8) {
              const uint32_t w = *(const uint32_t*)((const unsigned char*)a.v_pages + row * D + dim);
              if (!undefined<KV>(w)) continue;
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = (w >> (8 * e) & 0x7f) == 0x7f ? NAN : 0.f;
            } else {
              const uint2 w = *(const uint2*)((const __bf16*)a.v_pages + row * D + dim);
              if (!undefined<KV>(w.x) && !undefined<KV>(w.y)) continue;
              const uint32_t bits[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = (bits[e] & 0x7f800000u) == 0x7f800000u ? __uint_as_float(bits[e]) : 0.f;
            }
            if (whole) {
              bf16x4* const o = (bf16x4*)((__bf16*)a.out + at.out * D + dim);
              bf16x4 y = *o;
#pragma unroll
              for (int e = 0; e < 4; ++e) y[e] = (__bf16)((float)y[e] + x[e]);
              *o = y;
            } else {
              floatx4* const o = (floatx4*)(a.partial_o + (slot * RT + c) * (kRows * D) + (dim / 8 * 64 + lane) * 4);
              floatx4 y = *o;
#pragma unroll
              for (int e = 0; e < 4; ++e) y[e] += x[e];
              *o = y;
            }
          }
        }
      }
    }
    first_segment = false;
  };

  floatx16 s[RT];
  // ---- S^T = K Q^T
  auto scores = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < RT; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[c][i] = 0.f;
    const int t = (n32 & 16) + tau(n32 & 15);
    const unsigned char* rowp = lds.k[slot] + t * G_::kRowBytes;
    const int key = tree_key_k<D, FP8>(t);
    if constexpr (FP8) {
#pragma unroll
      for (int p = 0; p < kKK / 2; ++p) {
        const uint4 raw = *(const uint4*)(rowp + ((p * 2 + h2) ^ key) * 16);
        const auto lo = widen_k8<KV>(raw.x, raw.y), hi = widen_k8<KV>(raw.z, raw.w);
#pragma unroll
        for (int c = 0; c < RT; ++c) s[c] = mfma32(lo, qop[c][2 * p], s[c]);
#pragma unroll
        for (int c = 0; c < RT; ++c) s[c] = mfma32(hi, qop[c][2 * p + 1], s[c]);
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < kKK; ++kk) {
        const kx8 kop = *(const kx8*)(rowp + (((kk * 2 + h2) ^ key) & (G_::kChunks - 1)) * 16);
#pragma unroll
        for (int c = 0; c < RT; ++c) s[c] = mfma32(kop, qop[c][kk], s[c]);
      }
    }
  };
  // This lane then holds, for its rows, the scores of tokens tok0 + (i/8)*16 + h2*8 + i%8: eight of each page.
  opx8 pop[RT][2];
  unsigned int seen[RT];                             // bit i: of this lane's score i (set in the blocks behind the prefix alone)
  auto softmax = [&](bool edge, const float4& scales) __attribute__((always_inline)) {
    const int tok0 = cc.blk * kBlockTokens;
    float kscale[2] = {1.f, 1.f}, vscale[2] = {1.f, 1.f}, lvs[2] = {0.f, 0.f}, ivs[2] = {1.f, 1.f};
    if constexpr (FP8) {
      kscale[0] = scales.x; kscale[1] = scales.y; vscale[0] = scales.z; vscale[1] = scales.w;
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        if constexpr (HEAD) {
          lvs[pg] = __builtin_amdgcn_logf(vscale[pg]);
          ivs[pg] = __builtin_amdgcn_rcpf(vscale[pg]);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < RT; ++c) {
      float sc[2];
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) sc[pg] = (INT8 ? q_unit[c] : scale_log2) * (FP8 ? kscale[pg] : 1.f);
      if (edge) {
        // (faint queries over faint keys: a unit that has gone to zero would make a masked token's exponent undefined)
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) sc[pg] = fmaxf(sc[pg], 0x1p-126f);
        const int j = max(0, min(j0 + c * kRows + n32, n_b * group - 1));
        const uint64_t* words = a.mask + (size_t)(q_off + j / group) * a.mask_words;
        seen[c] = 0;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) seen[c] |= seen_bits(words, a.mask_words, tok0 + pg * kPageSize + h2 * 8 - prefix, n_b, 0xffu) << (8 * pg);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[c][i] = seen[c] >> i & 1 ? s[c][i] : -INFINITY;
      }
      float mx[2];
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        const int o = pg * 8;
        float x = fmaxf(fmaxf(s[c][o], s[c][o + 1]), s[c][o + 2]);
        x = fmaxf(fmaxf(x, s[c][o + 3]), s[c][o + 4]);
        x = fmaxf(fmaxf(x, s[c][o + 5]), s[c][o + 6]);
        mx[pg] = fmaxf(x, s[c][o + 7]);
        mx[pg] = HEAD ? __builtin_fmaf(mx[pg], sc[pg], lvs[pg]) : mx[pg] * sc[pg];
      }
      float top = xor32_max(fmaxf(mx[0], mx[1]));
      if constexpr (HEAD) {
        // (of a score past 2^25 the difference may come out larger, more than f16 holds)
        const float below = top - kWeightBits;
        top = top - below > kMostBits ? top : below;
      }
      const float m_new = fmaxf(m_run[c], top);
      const float base = m_new == -INFINITY ? 0.f : m_new;   // (a row that has seen nothing yet)
      const float alpha = __builtin_amdgcn_exp2f(m_run[c] - base);
      float psum[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int pg = i >> 3;
        float x;
        if constexpr (HEAD) x = __builtin_fmaf(s[c][i], sc[pg], lvs[pg]) - base;
        else x = __builtin_fmaf(s[c][i], sc[pg], -base);
        const float p = __builtin_amdgcn_exp2f(x);
        psum[pg] += p;
        pop[c][pg][i & 7] = (op)(FP8 && !HEAD ? p * vscale[pg] : p);
      }
      l_run[c] = l_run[c] * alpha + (HEAD ? psum[0] * ivs[0] + psum[1] * ivs[1] : psum[0] + psum[1]);
      if (__builtin_amdgcn_ballot_w64(m_new > m_run[c])) {
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[c][dt][i] *= alpha;
      }
      m_run[c] = m_new;
    }
  };
  // ---- O^T += V^T P^T : A = V^T tile (32 dims x 16 tokens) read transposed from LDS
  auto v_operand = [&](int slot, int ks, int dt) __attribute__((always_inline)) -> opx8 {
    if constexpr (FP8) {
      typedef __attribute__((address_space(3))) intx2 lds_i2;
      const int t = ks * 16 + h2 * 8 + ((lane & 15) >> 1);
      const int col = ((dt * 2 + ((lane >> 4) & 1)) ^ tree_key_v<true>(t)) & (G_::kChunks - 1);
      const intx2 raw = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2*)(lds.v[slot] + t * G_::kRowBytes + col * 16 + (lane & 1) * 8));
      return widen_v8<KV>((uint32_t)raw[0], (uint32_t)raw[1]);
    } else {
      typedef __attribute__((address_space(3))) shortx4 lds_s4;
      bf16x8 v;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const int j = lane & 15, t = ks * 16 + h2 * 8 + hf * 4 + (j >> 2);
        const int col = ((dt * 4 + ((lane >> 4) & 1) * 2 + ((j & 3) >> 1)) ^ tree_key_v<false>(t)) & (G_::kChunks - 1);
        const shortx4 raw = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(lds.v[slot] + t * G_::kRowBytes + col * 16 + (j & 1) * 8));
        const bf16x4 h4 = __builtin_bit_cast(bf16x4, raw);
        v[hf * 4 + 0] = h4[0]; v[hf * 4 + 1] = h4[1]; v[hf * 4 + 2] = h4[2]; v[hf * 4 + 3] = h4[3];
      }
      return v;
    }
  };
  auto values = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt) {
        const opx8 v = v_operand(slot, ks, dt);
#pragma unroll
        for (int c = 0; c < RT; ++c) acc[c][dt] = mfma32(v, pop[c][ks], acc[c][dt]);
      }
  };
  // Whether the values of a block hold any that is no number: then zeros take their places in front of the second product, and those of
  // the segment are added to what is stored of it.
  auto any_undefined = [&](int slot) __attribute__((always_inline)) {
    bool any = false;
#pragma unroll
    for (int j = 0; j < G_::kLoads; ++j) {
      const uint4 w = *(const uint4*)(lds.v[slot] + j * 1024 + lane * 16);
      any |= undefined<KV>(w.x) | undefined<KV>(w.y) | undefined<KV>(w.z) | undefined<KV>(w.w);
    }
    return __builtin_amdgcn_ballot_w64(any) != 0;
  };
  auto without_undefined = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < G_::kLoads; ++j) {
      uint4* const at = (uint4*)(lds.v[slot] + j * 1024 + lane * 16);
      const uint4 w = *at;
      *at = make_uint4(defined<KV>(w.x), defined<KV>(w.y), defined<KV>(w.z), defined<KV>(w.w));
    }
  };

  for (int i = 0; i < min(kSlots, n_mine); ++i) {
    issue_k(i);
    issue_v(i);
  }
  int slot = 0;
  for (int i = 0; i < n_mine; ++i) {
    if (i == 0 || cc.blk == 0) begin_segment();
    const bool edge = (cc.blk + 1) * kBlockTokens > prefix, more = i + kSlots < n_mine;
    const int behind = min(kSlots - 1, n_mine - 1 - i);      // blocks behind this one that are under way
    await(behind, std::integral_constant<int, G_::kLoads>{});
    scores(slot);
    float4 kept_scales = {};
    if constexpr (FP8) kept_scales = *(const float4*)lds.scales[slot];
    if (more) {
      issue_k(slot);
      await(behind, std::integral_constant<int, kKLoads>{});
    } else {
      await(behind, std::integral_constant<int, 0>{});
    }
    softmax(edge, kept_scales);
    if (!INT8 && edge && any_undefined(slot)) {
      without_undefined(slot);
      dirty = true;
    }
    values(slot);
    if (more) issue_v(slot);
    if (cc.blk == cc.n - 1 || i == n_mine - 1) end_segment();
    if (i + 1 < n_mine) advance(cc);
    slot = slot + 1 == kSlots ? 0 : slot + 1;
  }
}

// The start of a worker's run, for a batch of at most 64 trajectories: worked out by every wave for itself, a lane per trajectory (the rule
// is plan_decode's).  The first worker writes the header and the scan, which the merge reads.
__device__ __forceinline__ int4 tree_plan_in_wave(const TreeArgs& a, int worker) {
  const int lane = lane_id(), rows_per_b = a.hkv * a.row_tiles;
  int len = 0;
  if (lane < a.batch) len = a.q_lens[lane] > 0 ? a.ctx_lens[lane] : 0;
  const int count = (len + kBlockTokens - 1) / kBlockTokens;
  const int upto = wave_inclusive_scan(count), first = upto - count;
  const int blocks = __builtin_amdgcn_readlane(upto, 63);
  const int total = blocks * rows_per_b;
  const int per = max(1, (total + a.workers - 1) / a.workers);
  const unsigned int x = (unsigned int)worker * (unsigned int)per;
  if (worker == 0) {
    if (lane < a.batch) a.prefix[lane] = first;
    if (lane == 0) {
      a.prefix[a.batch] = blocks;
      a.header[kPlanPer] = per;
    }
  }
  if (x >= (unsigned int)total) return make_int4(-1, 0, 0, 0);
  const unsigned long long before = __builtin_amdgcn_ballot_w64(lane < a.batch && (unsigned int)(rows_per_b * first) <= x);
  const int b = 63 - __builtin_clzll(before);
  const int n = __builtin_amdgcn_readlane(count, b);
  const int rem = (int)x - rows_per_b * __builtin_amdgcn_readlane(first, b);
  return make_int4(b, ((rem / n) << 20) | (rem % n), 0, min(per, total - (int)x));
}

template <int D, int KV, int RT>
__global__ __launch_bounds__(kThreads, RT == 2 ? 1 : 2) void tree_mfma_kernel(const TreeArgs a) {
  __shared__ TreeLds<D, kv_is_codes(KV), RT> lds[kWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int worker = blockIdx.x * kWaves + wave;
  int4 start;
  if (a.batch <= kWavePlanBatch) start = tree_plan_in_wave(a, worker);
  else start = *(const int4*)(a.wstart + 4 * worker);
  const int b = __builtin_amdgcn_readfirstlane(start.x), at = __builtin_amdgcn_readfirstlane(start.y), mine = __builtin_amdgcn_readfirstlane(start.w);
  if (b < 0) return;
  tree_worker<D, KV, RT, false>(a, b, at >> 20, at & 0xFFFFF, mine, worker, lds[wave]);
}

__global__ __launch_bounds__(kPlanThreads) void tree_plan_kernel(const DecodePlanArgs p) {
  __shared__ DecodePlanLds lds;
  plan_decode(p, lds, [&](int b) { return p.q_lens[b] > 0 ? p.ctx_lens[b] : 0; });
}

// Merge of the partials that runs left of rows they did not cover alone, as in combine.hip: one wave per (row, 32 query rows, 32 dims),
// lanes as in the accumulators, four pieces under way at a time.  A piece of which a query row saw nothing has weight zero.
template <int D, int RT>
__global__ __launch_bounds__(kThreads) void tree_merge_kernel(const TreeArgs a) {
  constexpr int kDT = D / 32;
  const int lane = lane_id(), n32 = lane & 31, h2 = lane >> 5;
  const int unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * kWaves + (threadIdx.x >> 6)));
  const int dt = unit % kDT, c = unit / kDT % RT, row = unit / (kDT * RT), rows_per_b = a.hkv * a.row_tiles;
  const int b = row / rows_per_b, r = row - b * rows_per_b;
  if (b >= a.batch) return;
  const int per = a.header[kPlanPer], first = a.prefix[b], n = a.prefix[b + 1] - first;
  const Draft d(a, b);
  const int g = r / a.row_tiles, j0 = (r - g * a.row_tiles) * (kRows * RT) + c * kRows;
  if (n == 0 || j0 >= d.n * a.group) return;
  const long r0 = (long)rows_per_b * first + (long)r * n;
  const int wf = (int)(r0 / per), wl = (int)((r0 + n - 1) / per), pieces = wl - wf + 1;
  if (pieces == 1) return;                                  // one worker had the whole row
  const int first_slot = ((long)wf * per < r0) ? 1 : 0;
  const bool ok = j0 + n32 < d.n * a.group;
  floatx4 o[4];
#pragma unroll
  for (int i4 = 0; i4 < 4; ++i4) o[i4] = floatx4{0.f, 0.f, 0.f, 0.f};
  float ref = -INFINITY, l = 0.f;
  constexpr int kN = 4;
  for (int s0 = 0; s0 < pieces; s0 += kN) {
    floatx2 x[kN];
    floatx4 y[kN][4];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int s = min(s0 + i, pieces - 1);
      const size_t part = ((size_t)(wf + s) * 2 + (s == 0 ? first_slot : 0)) * RT + c;
      x[i] = *(const floatx2*)(a.partial_ml + (part * kRows + n32) * 2);
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) y[i][i4] = *(const floatx4*)(a.partial_o + part * (kRows * D) + ((dt * 4 + i4) * 64 + lane) * 4);
    }
    float top = ref;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      if (s0 + i >= pieces) {                               // (zero times an infinity would not be zero)
        x[i] = floatx2{-INFINITY, 0.f};
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) y[i][i4] = floatx4{0.f, 0.f, 0.f, 0.f};
      }
      top = fmaxf(top, x[i][0]);
    }
    const float base = top == -INFINITY ? 0.f : top;
    const float keep = __builtin_amdgcn_exp2f(ref - base);
    ref = top;
    l *= keep;
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) o[i4] *= keep;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float f = __builtin_amdgcn_exp2f(x[i][0] - base);
      l += f * x[i][1];
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) o[i4] += f * y[i][i4];
    }
  }
  if (!ok) return;
  const RowAt at(a, d, g, j0 + n32);
  if (a.lse && dt == 0 && h2 == 0) a.lse[at.out] = ref + __builtin_amdgcn_logf(l);
  const float inv = l > 0.f ? 1.f / l : l;
  __bf16* dst = (__bf16*)a.out + at.out * D + dt * 32 + h2 * 4;
#pragma unroll
  for (int i4 = 0; i4 < 4; ++i4) {
    bf16x4 pk;
#pragma unroll
    for (int e = 0; e < 4; ++e) pk[e] = (__bf16)(o[i4][e] * inv);
    *(bf16x4*)(dst + i4 * 8) = pk;
  }
}

}  // namespace

hipError_t launch_tree_mfma(const TreeArgs& a, int head_dim, KvKind kv, hipStream_t s) {
  if (a.batch > kWavePlanBatch) {
    DecodePlanArgs p{};
    p.ctx_lens = a.ctx_lens; p.q_lens = a.q_lens; p.batch = a.batch; p.rows_per_b = a.hkv * a.row_tiles;
    p.workers = p.slots = a.workers;
    p.header = a.header; p.prefix = a.prefix; p.wstart = a.wstart;
    hipLaunchKernelGGL(tree_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)(a.workers / kWaves));
  const int64_t units = (int64_t)a.batch * a.hkv * a.row_tiles * a.tile_parts * (head_dim / 32);
  const dim3 merge_grid((unsigned)((units + kWaves - 1) / kWaves));
  auto launch = [&](auto d, auto kind, auto c) {
    hipLaunchKernelGGL((tree_mfma_kernel<decltype(d)::value, decltype(kind)::value, decltype(c)::value>), grid, dim3(kThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((tree_merge_kernel<decltype(d)::value, decltype(c)::value>), merge_grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
  };
  auto of_tiles = [&](auto d, auto kind) { return a.tile_parts == 1 ? launch(d, kind, std::integral_constant<int, 1>{}) : launch(d, kind, std::integral_constant<int, 2>{}); };
  auto of_kind = [&](auto kind) {
    return head_dim == 128 ? of_tiles(std::integral_constant<int, 128>{}, kind) : of_tiles(std::integral_constant<int, 64>{}, kind);
  };
  if (head_dim != 128 && head_dim != 64) return hipErrorInvalidValue;
  switch (kv) {
    case kKvBf16: return of_kind(std::integral_constant<int, kKvBf16>{});
    case kKvFp8: return of_kind(std::integral_constant<int, kKvFp8>{});
    case kKvFp8Head: return of_kind(std::integral_constant<int, kKvFp8Head>{});
    case kKvInt8Head: return of_kind(std::integral_constant<int, kKvInt8Head>{});
  }
  return hipErrorInvalidValue;
}

}  // namespace rollattn
