#ifndef VMT
#define VMT 2048
#endif
// Attention of a tree of drafted tokens (bf16 queries) over bf16 or 8-bit (E4M3, int8) paged KV (gfx950).
//
// A row is (trajectory, KV head, tile of 32 W query rows): a query row is a (drafted token, query head of the group) pair,
// token-major, so the heads that share the KV head and the tokens of a draft that fit one tile read K and V once.  As in decode, rows
// are cut into 32-token blocks, laid end to end, and every worker has one equal run of that sequence; a worker is W waves of 32 query rows
// each.  It streams its run from memory straight into a ring of LDS tiles, and each of its waves consumes a block with
//   S^T = K Q^T          (tokens x query rows, v_mfma_f32_32x32x16, K rows as A)
//   O^T += V^T P^T       (dims x query rows, V read back transposed with ds_read_b64_tr_*)
// A run that covers a whole row writes the row's output itself; one that starts or ends inside a row leaves an un-normalised partial
// (max, sum, O) for the merge.
// A block that lies in the cached prefix is seen whole by every row and knows no mask.  In the blocks behind it a row sees the tokens
// whose bits are set in its mask words, eight tokens at a time.  What a row does not see must not reach it: a score is replaced before
// the maximum, and where values of such a block are not finite (zero times infinity would not be zero) zeros take their places in the
// second product, and they are added apart to the rows that see them.
// Codes become operands as in decode: see decode_mfma.hip for the range of f16 and the power of two per query row.
#include "stream_tiles.h"

namespace rollattn {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef unsigned int uint4_v __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;             // of the merge
constexpr int kWaves = kThreads / 64;
constexpr int kRows = kTreeTileRows;      // query rows of a wave
constexpr int kMergeTogether = VMT;
constexpr float kSumLimit = 16384.f;      // see the softmax
constexpr float kHalfSumLimit = 65000.f;
constexpr float kTreeWeightBits = 8.f;    // f16 weights: log2 of a row's largest when its reference moves

__device__ __forceinline__ floatx16 mfma32(bf16x8 x, bf16x8 y, floatx16 z) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ floatx16 mfma32(halfx8 x, halfx8 y, floatx16 z) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, z, 0, 0, 0); }

// Row t of an S^T tile holds this token of its 16-token group: the middle two quads are swapped, so that the 8 scores a lane ends up with
// are 8 consecutive tokens.
__device__ __forceinline__ int tau(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

// Tiles of 32 W query rows that a draft of n tokens has per KV head (no more than the caller has said that the longest one has).
template <class A>
__device__ __forceinline__ int tree_tiles(const A& a, int n) {
  const int rows = kRows * a.tile_parts;
  return n > 0 ? min((n * a.group + rows - 1) / rows, a.row_tiles) : 0;
}

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

// The sign bits of the elements of a word of a pool that are no numbers (infinite and undefined bf16 values, whose exponent is all ones; the
// undefined code of E4M3): the sum carries into them.
template <int KV>
__device__ __forceinline__ uint32_t undefined(uint32_t w) {
  if constexpr (KV == kKvBf16) return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  else if constexpr (KV == kKvInt8Head) return 0;
  else return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}
// The word with zeros in the place of those.
template <int KV>
__device__ __forceinline__ uint32_t defined(uint32_t w) {
  const uint32_t met = undefined<KV>(w) >> (KV == kKvBf16 ? 15 : 7);
  return w & ~(met * (KV == kKvBf16 ? 0xffffu : 0xffu));
}

// The kernel's arguments, read anew from their segment: what only a row's start and end need is not kept in scalar registers over its blocks
// (they would spill, into lanes of vector registers that every block then fetches them from).
typedef const __attribute__((address_space(4))) TreeArgs* tree_args_p;
__device__ __forceinline__ tree_args_p tree_args() {
  tree_args_p p = (tree_args_p)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}

// The lengths of one trajectory, the same in all lanes.
struct Draft {
  int n, len, off;
  template <class A>
  __device__ __forceinline__ Draft(const A& a, int b) {
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
  template <class A>
  __device__ __forceinline__ RowAt(const A& a, const Draft& d, int g, int j) {
    node = j / a.group;
    out = (size_t)(d.off + node) * a.hq + (size_t)g * a.group + (j - node * a.group);
  }
};

// A worker's ring: its blocks, the one in work included, so that two waves to a SIMD find their LDS.  Addresses are 32-bit offsets in the LDS.
template <int D, bool FP8, int W>
struct TreeLds {
  static constexpr int kSlots = W == 1 ? (FP8 ? 2 : 1) : W == 2 ? (FP8 ? 4 : 2) : 4;
  static constexpr int kTile = Geo<D, FP8>::kTileBytes, kScales = FP8 ? 256 : 0;   // scales of a block's two pages: K's, V's (the other lanes' are copies)
  static constexpr int kBytes = kSlots * (2 * kTile + W * kScales);
  static __device__ __forceinline__ unsigned int k(int slot) { return slot * kTile; }
  static __device__ __forceinline__ unsigned int v(int slot) { return (kSlots + slot) * kTile; }
  static __device__ __forceinline__ unsigned int scales(int slot, int wave) { return 2 * kSlots * kTile + (slot * W + wave) * kScales; }
};
template <class T>
__device__ __forceinline__ __attribute__((address_space(3))) T* lds_at(unsigned int at) { return (__attribute__((address_space(3))) T*)(uintptr_t)at; }

// One run of n_mine blocks from block blk of row (b, r) on.
// Loads.  W = 1: the tiles of block i + slots go into the places of block i, K's as soon as the first product has read them and V's behind
// the second; no barriers.  Else each wave loads its share of a block, waits for its own loads and meets the others at one barrier per block:
// behind it the block is there, and the place of the block before is free for the one that is slots - 1 ahead.
// HBM -> LDS without a register stop: lane l's 16 bytes land at M0 + 16 l, so a row's chunks are swizzled by the address a lane
// reads from.  The compiler does not see these loads as loads; they are awaited by count: vector-memory counts go down in order, so
// with N of these loads sent after the ones that are waited for, no more than N outstanding operations of any kind means that those have
// landed (others in between only make the wait longer).
template <int D, int KV, int W, bool STREAM>
__device__ __forceinline__ void tree_worker(const TreeArgs& a, int b0, int r0, int blk0, int n_mine, int worker, int wave, unsigned int lds) {
  constexpr bool FP8 = kv_is_codes(KV), HEAD = kv_has_head_scales(KV);   // FP8: 8-bit codes of either kind
  constexpr bool INT8 = KV == kKvInt8Head;
  constexpr int kTile = kRows * W, kSlots = TreeLds<D, FP8, W>::kSlots;
  using L_ = TreeLds<D, FP8, W>;
  constexpr int kKK = D / 16, kDT = D / 32;
  using kx8 = std::conditional_t<INT8, halfx8, bf16x8>;   // operands of the first product
  using opx8 = std::conditional_t<HEAD, halfx8, bf16x8>;  // ... and of the second
  using op = std::conditional_t<HEAD, _Float16, __bf16>;
  using G_ = Geo<D, FP8>;
  // this wave's loads of a block: of each pool's tile its share, or where there are more waves than a tile has loads, of one pool's tile one
  // (where there are more than both have, some twice: the same bytes to the same place); its copy of the scales
  constexpr int kShare = G_::kLoads >= W ? G_::kLoads / W : 1;
  constexpr int kVLoads = G_::kLoads >= W ? kShare : 0, kKLoads = kShare + (FP8 ? 1 : 0);
  const int lane = lane_id();
  const int n32 = lane & 31;   // query row (B column) / K token row (A row) carried by this lane
  const int h2 = lane >> 5;    // half of the contraction this lane feeds

  const int hkv = a.hkv;
  constexpr size_t tile_stride = (size_t)kPageSize * G_::kRowBytes;   // bytes of one (page, head) tile

  // trajectory, KV head, tile and block within the row; blocks in the row, context length, tiles per KV head
  struct Cursor { int b, g, tile, blk, n, len, tiles; };
  auto enter = [&](Cursor& c) {
    const tree_args_p e = tree_args();
    const Draft d(*e, c.b);
    c.tiles = tree_tiles(*e, d.n);
    c.len = c.tiles ? d.len : 0;
    c.n = (c.len + kBlockTokens - 1) / kBlockTokens;
  };
  Cursor pc{b0, 0, 0, blk0, 0, 0, 0};         // producer: next block to request from HBM
  enter(pc);
  pc.g = r0 / pc.tiles;
  pc.tile = r0 - pc.g * pc.tiles;
  Cursor cc = pc;                             // consumer: block being computed
  auto advance = [&](Cursor& c) {             // (whether it is another row now)
    if (++c.blk < c.n) return false;
    c.blk = 0;
    if (++c.tile < c.tiles) return true;
    c.tile = 0;
    if (++c.g < hkv) return true;
    c.g = 0;
    do {
      ++c.b;
      enter(c);
    } while (c.len == 0);
    return true;
  };

  // ---- producer: a window of 64 page ids (32 blocks) of the current row, one per lane
  int pid_vec = 0, pid_next = 0, left = n_mine;
  bool fresh = true;                          // no window of this row yet
  int p_page[2] = {0, 0}, p_lim = 0;          // the block under way: its pages, and tokens from its first on
  size_t p_at[2] = {0, 0};                    // ... and where this wave's loads find them in a pool
  auto load_window = [&](int k) {
    const tree_args_p e = tree_args();
    const int pg = k * 64 + lane;
    return (pg < ((pc.len + kPageSize - 1) >> 4)) ? e->page_table[(size_t)pc.b * e->max_pages + pg] : 0;
  };
  auto dma16 = [&](const unsigned char* base, unsigned int off, unsigned int dst) __attribute__((always_inline)) {
    const unsigned int m0 = __builtin_amdgcn_readfirstlane(dst);
    if constexpr (STREAM) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(m0), "v"(off), "s"(base) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(m0), "v"(off), "s"(base) : "memory");
  };
  // This wave's share of a tile of one pool: row row0 + lane / chunks of the block per load.  What a lane reads of a tile is the same for every
  // whole block; of a row's ragged last one, rows at or past L_b read its last one again.
  const bool for_v = kVLoads == 0 && wave % (2 * G_::kLoads) >= G_::kLoads;       // (one pool's tile alone, and that is V's)
  const int first = G_::kLoads >= W ? wave : wave % G_::kLoads;
  auto key_of = [&](auto v_c, int row) __attribute__((always_inline)) { return decltype(v_c)::value ? tree_key_v<FP8>(row) : tree_key_k<D, FP8>(row); };
  auto offset = [&](auto v_c, int i, int lim) __attribute__((always_inline)) {
    const int row = (first + i * W) * G_::kRowsPerLoad + lane / G_::kChunks;
    return min(row, lim - 1) % kPageSize * G_::kRowBytes + (((lane % G_::kChunks) ^ key_of(v_c, row)) & (G_::kChunks - 1)) * 16;
  };
  unsigned int off_k[kShare], off_v[kShare];
#pragma unroll
  for (int i = 0; i < kShare; ++i) {
    off_k[i] = offset(std::false_type{}, i, kBlockTokens);
    off_v[i] = offset(std::true_type{}, i, kBlockTokens);
  }
  const bool upper = first * G_::kRowsPerLoad >= kPageSize;        // (one load of a tile: of its second page)
  auto load_tile = [&](auto v_c, int slot) __attribute__((always_inline)) {
    constexpr bool V = decltype(v_c)::value;
    const unsigned int dst = lds + (V ? L_::v(slot) : L_::k(slot)) + first * 1024;
#pragma unroll
    for (int i = 0; i < kShare; ++i) {
      const bool second = kShare == 1 ? upper : (first + i * W) * G_::kRowsPerLoad >= kPageSize;
      const unsigned char* tile = (const unsigned char*)(V ? a.v_pages : a.k_pages) + (kShare == 1 || !second ? p_at[0] : p_at[1]);
      const unsigned int off = p_lim >= kBlockTokens ? (V ? off_v[i] : off_k[i]) : offset(v_c, i, p_lim);
      dma16(tile, off, dst + i * W * 1024);
    }
  };
  auto load_k = [&](int slot) __attribute__((always_inline)) { load_tile(std::false_type{}, slot); };
  auto load_v = [&](int slot) __attribute__((always_inline)) { load_tile(std::true_type{}, slot); };
  // what block pc of the run needs
  auto look_up = [&]() __attribute__((always_inline)) {
    const int in = pc.blk & 31;
    if (fresh || in == 0) {
      const int k = pc.blk >> 5;
      pid_vec = fresh ? load_window(k) : pid_next;
      pid_next = load_window(k + 1);
      fresh = false;
    }
    p_lim = pc.len - pc.blk * kBlockTokens;
    // (a page that the row's last block does not have: the one in front of it)
    const int last = p_lim > kPageSize ? 1 : 0;
    if constexpr (kShare == 1 && !FP8) {
      p_page[0] = __builtin_amdgcn_readlane(pid_vec, in * 2 + (upper ? last : 0));
    } else {
      p_page[0] = __builtin_amdgcn_readlane(pid_vec, in * 2);
      p_page[1] = __builtin_amdgcn_readlane(pid_vec, in * 2 + last);
    }
    auto at = [&](int page) { return (size_t)(unsigned int)__builtin_amdgcn_readfirstlane(page * hkv + pc.g) * tile_stride; };
    if constexpr (kShare == 1) {
      p_at[0] = at(FP8 && upper ? p_page[1] : p_page[0]);
    } else {
      p_at[0] = at(p_page[0]);
      p_at[1] = at(p_page[1]);
    }
  };
  auto load_scales = [&](int slot) __attribute__((always_inline)) {
    if constexpr (FP8) {
      const int page = lane & 1 ? p_page[1] : p_page[0];
      const float* from = (lane & 2 ? a.v_scale : a.k_scale) + (HEAD ? (size_t)page * hkv + pc.g : (size_t)page);
      const unsigned int m0 = __builtin_amdgcn_readfirstlane(lds + L_::scales(slot, wave));
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(m0), "v"(from) : "memory");
    }
  };
  // step to the next block of the run (never past its end: the rows after the last block need not exist); a new row starts with a
  // fresh page-id window
  auto step = [&]() __attribute__((always_inline)) {
    if (--left > 0 && advance(pc)) fresh = true;
  };
  // (what the loads overwrite has been read)
  auto all_read = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
  auto issue_k = [&](int slot) __attribute__((always_inline)) {      // W = 1: K and scales, then V
    look_up();
    load_k(slot);
    load_scales(slot);
  };
  auto issue_v = [&](int slot) __attribute__((always_inline)) {
    load_v(slot);
    step();
  };
  auto issue = [&](int slot) __attribute__((always_inline)) {
    look_up();
    if constexpr (kVLoads > 0) {
      load_k(slot);
      load_v(slot);
    } else if (for_v) {
      load_v(slot);
    } else {
      load_k(slot);
    }
    load_scales(slot);
    step();
  };
  // until all but this wave's loads of kBlocks blocks, and kMore others, have landed; near the run's end, where fewer blocks follow, of none
  auto await = [&](bool follow, auto blocks_c, auto more_c) __attribute__((always_inline)) {
    constexpr int kMore = decltype(more_c)::value, kBlock = kVLoads + kKLoads;
    if (follow) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(blocks_c)::value * kBlock + kMore) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMore) : "memory");
  };

  // ---- consumer state
  kx8 qop[kKK];              // Q^T as the B operand: lane (row n32, half h2), 8 dims per step
  float q_unit = 0.f;        // what a unit of this lane's row is worth, softmax scale included
  floatx16 acc[kDT];        // O^T: lane (row n32, half h2) holds dims dt*32 + (i/4)*8 + h2*4 + i%4
  float m_ref = 0.f, l_run = 0.f;   // reference of this lane's row (log2 units), zero as long as it has seen nothing; its share of the running sum
  float sum_limit = -1.f;           // a lane's exponentials of a block may add up to this much; below zero: no reference yet
  int seg_first_blk = 0;     // block of the row at which the current segment started
  bool first_segment = true, dirty = false;   // dirty: values of the segment that are no numbers have been left out of its sums
  int rows_here = 0, edge_blk = 0;            // of the consumer's row: query rows of this wave, first block with tokens behind the prefix

  auto begin_segment = [&]() __attribute__((always_inline)) {
    const tree_args_p e = tree_args();
    const Draft d(*e, cc.b);
    const int j0 = cc.tile * kTile + wave * kRows;
    rows_here = min(kRows, d.n * e->group - j0);     // (none: a wave past the last row helps with the loads)
    edge_blk = (d.len - d.n) / kBlockTokens;
    const bool flip = e->scale_log2 < 0.f;           // (queries the other way round, so that larger scores are larger exponents)
    const float scale_log2 = __builtin_fabsf(e->scale_log2);
    {
      // (rows past the last read it again; what becomes of them is not stored)
      const RowAt at(*e, d, cc.g, max(0, min(j0 + n32, d.n * e->group - 1)));
      const __bf16* qrow = (const __bf16*)e->q + at.out * D;
#pragma unroll
      for (int kk = 0; kk < kKK; ++kk) {
        // FP8: 16-byte K chunks hold 16 dims; step 2p+e uses bytes e*8.. of chunk p*2+h2
        uint4 v = *(const uint4*)(qrow + (FP8 ? ((kk >> 1) * 2 + h2) * 16 + (kk & 1) * 8 : kk * 16 + h2 * 8));
        const uint32_t sign = flip ? 0x80008000u : 0u;
        v.x ^= sign; v.y ^= sign; v.z ^= sign; v.w ^= sign;
        qop[kk] = __builtin_bit_cast(kx8, v);     // (int8: as it came, until all of the row is there)
      }
      q_unit = scale_log2;
      if constexpr (INT8) {
        float top = 0.f;
#pragma unroll
        for (int kk = 0; kk < kKK; ++kk) {
          const bf16x8 v = __builtin_bit_cast(bf16x8, qop[kk]);
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, __builtin_fabsf((float)v[e]));
        }
        const int up = kQueryBits - __builtin_amdgcn_frexp_expf(xor32_max(top));
#pragma unroll
        for (int kk = 0; kk < kKK; ++kk) {
          const bf16x8 v = __builtin_bit_cast(bf16x8, qop[kk]);
#pragma unroll
          for (int e = 0; e < 8; ++e) qop[kk][e] = (_Float16)__builtin_amdgcn_ldexpf((float)v[e], up);
        }
        q_unit = __builtin_amdgcn_ldexpf(scale_log2, -up);
      }
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;
      m_ref = l_run = 0.f;
      sum_limit = -1.f;
    }
    seg_first_blk = cc.blk;
    dirty = false;
  };
  auto end_segment = [&]() __attribute__((always_inline)) {
    const bool whole = seg_first_blk == 0 && cc.blk == cc.n - 1;
    const size_t slot = (size_t)worker * 2 + (first_segment ? 0 : 1);
    const tree_args_p e = tree_args();
    const Draft d(*e, cc.b);
    const int g = cc.g, j0 = cc.tile * kTile + wave * kRows, prefix = d.len - d.n;
    if (rows_here > 0) {
      const float l_tot = xor32_add(l_run), m_run = sum_limit < 0.f ? -INFINITY : m_ref;
      if (whole) {
        // the whole row was ours: normalise and store
        const bool ok = n32 < rows_here;
        const RowAt at(*e, d, g, max(0, min(j0 + n32, d.n * e->group - 1)));
        const float inv = l_tot > 0.f ? 1.f / l_tot : l_tot;   // (nothing seen: a row of zeros)
        if (e->lse && ok && h2 == 0) e->lse[at.out] = m_run + __builtin_amdgcn_logf(l_tot);
        __bf16* dst = (__bf16*)e->out + at.out * D + h2 * 4;
        if (ok) {
#pragma unroll
          for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
              bf16x4 pk;
#pragma unroll
              for (int e = 0; e < 4; ++e) pk[e] = (__bf16)(acc[dt][i4 * 4 + e] * inv);
              *(bf16x4*)(dst + dt * 32 + i4 * 8) = pk;
            }
        }
      } else if (n32 < rows_here) {
        float* dst = e->partial_o + (slot * W + wave) * (kRows * D) + lane * 4;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4)
            *(floatx4*)(dst + (dt * 4 + i4) * 256) = floatx4{acc[dt][i4 * 4], acc[dt][i4 * 4 + 1], acc[dt][i4 * 4 + 2], acc[dt][i4 * 4 + 3]};
        if (h2 == 0) *(floatx2*)(e->partial_ml + ((slot * W + wave) * kRows + n32) * 2) = floatx2{m_run, l_tot};
      }
    }
    if (!INT8 && dirty) {
      // rare, and one token after the other: each lane adds to the values that it has just stored
      if (n32 < rows_here) {
        const RowAt at(*e, d, g, j0 + n32);
        const uint64_t* const words = e->mask + (size_t)(d.off + at.node) * e->mask_words;
        for (int t = max(prefix, seg_first_blk * kBlockTokens); t < min(d.len, (cc.blk + 1) * kBlockTokens); ++t) {
          const int rel = t - prefix;
          if (rel >= 64 * e->mask_words || !(words[rel >> 6] >> (rel & 63) & 1)) continue;
          const size_t row = ((size_t)e->page_table[(size_t)cc.b * e->max_pages + t / kPageSize] * hkv + g) * kPageSize + t % kPageSize;
          for (int dim = h2 * 4; dim < D; dim += 8) {
            float x[4];
            if constexpr (FP8) {
              const uint32_t w = *(const uint32_t*)((const unsigned char*)e->v_pages + row * D + dim);
              if (!undefined<KV>(w)) continue;
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = (w >> (8 * e) & 0x7f) == 0x7f ? NAN : 0.f;
            } else {
              const uint2 w = *(const uint2*)((const __bf16*)e->v_pages + row * D + dim);
              if (!undefined<KV>(w.x) && !undefined<KV>(w.y)) continue;
              const uint32_t bits[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = (bits[e] & 0x7f800000u) == 0x7f800000u ? __uint_as_float(bits[e]) : 0.f;
            }
            if (whole) {
              bf16x4* const o = (bf16x4*)((__bf16*)e->out + at.out * D + dim);
              bf16x4 y = *o;
#pragma unroll
              for (int e = 0; e < 4; ++e) y[e] = (__bf16)((float)y[e] + x[e]);
              *o = y;
            } else {
              floatx4* const o = (floatx4*)(e->partial_o + (slot * W + wave) * (kRows * D) + (dim / 8 * 64 + lane) * 4);
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

  floatx16 s;
  // ---- S^T = K Q^T
  auto scores = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
    const int t = (n32 & 16) + tau(n32 & 15);
    const unsigned int rowp = lds + L_::k(slot) + t * G_::kRowBytes;
    const int key = tree_key_k<D, FP8>(t);
    // (all operands on their way before the first product: the products hang together and would each wait for a trip to the LDS)
    if constexpr (FP8) {
      uint4_v raw[kKK / 2];
#pragma unroll
      for (int p = 0; p < kKK / 2; ++p) raw[p] = *lds_at<const uint4_v>(rowp + ((p * 2 + h2) ^ key) * 16);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int p = 0; p < kKK / 2; ++p) {
        s = mfma32(widen_k8<KV>(raw[p][0], raw[p][1]), qop[2 * p], s);
        s = mfma32(widen_k8<KV>(raw[p][2], raw[p][3]), qop[2 * p + 1], s);
      }
    } else {
      kx8 kop[kKK];
#pragma unroll
      for (int kk = 0; kk < kKK; ++kk) kop[kk] = *lds_at<const kx8>(rowp + (((kk * 2 + h2) ^ key) & (G_::kChunks - 1)) * 16);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kk = 0; kk < kKK; ++kk) s = mfma32(kop[kk], qop[kk], s);
    }
  };
  // This lane then holds, for its rows, the scores of tokens tok0 + (i/8)*16 + h2*8 + i%8: eight of each page.
  opx8 pop[2];
  unsigned int seen = 0;                             // bit i: of this lane's score i (set in the blocks behind the prefix alone)
  auto softmax = [&](bool edge, const floatx4& scales) __attribute__((always_inline)) {
    float kscale[2] = {1.f, 1.f}, vscale[2] = {1.f, 1.f}, lvs[2] = {0.f, 0.f}, ivs[2] = {1.f, 1.f};
    if constexpr (FP8) {
      kscale[0] = scales[0]; kscale[1] = scales[1]; vscale[0] = scales[2]; vscale[1] = scales[3];
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        if constexpr (HEAD) {
          lvs[pg] = __builtin_amdgcn_logf(vscale[pg]);
          ivs[pg] = __builtin_amdgcn_rcpf(vscale[pg]);
        }
      }
    }
    {
      float sc[2];
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) sc[pg] = q_unit * (FP8 ? kscale[pg] : 1.f);
      if (edge) {
        // (faint queries over faint keys: a unit that has gone to zero would make a masked token's exponent undefined)
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) sc[pg] = fmaxf(sc[pg], 0x1p-126f);
        const tree_args_p e = tree_args();
        const Draft d(*e, cc.b);
        const int j = max(0, min(cc.tile * kTile + wave * kRows + n32, d.n * e->group - 1)), n_words = e->mask_words;
        const uint64_t* words = e->mask + (size_t)(d.off + j / e->group) * n_words;
        seen = 0;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) seen |= seen_bits(words, n_words, cc.blk * kBlockTokens + pg * kPageSize + h2 * 8 - (d.len - d.n), d.n, 0xffu) << (8 * pg);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = seen >> i & 1 ? s[i] : -INFINITY;
      }
      // The reference of a row only moves when it has to: exponentials are taken against it as it stands, and may exceed one.  Only when
      // a lane's add up to more than kSumLimit (f16 weights: a page's to kHalfSumLimit, so that none is too large for f16), or while a row has no
      // reference, are the maxima found, the references moved there and the block's exponentials taken again.
      float psum[2], p[16];
      auto exponentials = [&](auto first_c) __attribute__((always_inline)) {
        float ad[2];
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) ad[pg] = lvs[pg] - m_ref;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int pg = i >> 3;
          float x;
          if constexpr (HEAD && !decltype(first_c)::value) x = __builtin_fmaf(s[i], sc[pg], lvs[pg]) - m_ref;
          else x = __builtin_fmaf(s[i], sc[pg], ad[pg]);
          p[i] = __builtin_amdgcn_exp2f(x);
          psum[pg] = (i & 7) == 0 ? p[i] : psum[pg] + p[i];
        }
      };
      exponentials(std::true_type{});
      // (an undefined sum takes the slow way, too; HEAD: it need not, the row is undefined with either)
      if (__builtin_amdgcn_ballot_w64(!((HEAD ? fmaxf(psum[0], psum[1]) : psum[0] + psum[1]) <= sum_limit))) {
        float mx[2];
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
          const int o = pg * 8;
          float x = fmaxf(fmaxf(s[o], s[o + 1]), s[o + 2]);
          x = fmaxf(fmaxf(x, s[o + 3]), s[o + 4]);
          x = fmaxf(fmaxf(x, s[o + 5]), s[o + 6]);
          mx[pg] = fmaxf(x, s[o + 7]);
          mx[pg] = HEAD ? __builtin_fmaf(mx[pg], sc[pg], lvs[pg]) : mx[pg] * sc[pg];
        }
        float top = xor32_max(fmaxf(mx[0], mx[1]));            // the same in both lanes of a row
        if constexpr (HEAD) {
          // (of a score past 2^25 the difference may come out larger, more than f16 holds; exponents are differences of numbers that were
          // rounded like this one, so none is larger)
          const float below = top - kTreeWeightBits;
          top = top - below > kMostBits ? top : below;
        }
        const float m_old = sum_limit < 0.f ? -INFINITY : m_ref, m_new = fmaxf(m_old, top);
        const float m_safe = m_new == -INFINITY ? 0.f : m_new;   // (a row that has seen nothing yet)
        const float alpha = __builtin_amdgcn_exp2f(m_old - m_safe);
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[dt][i] *= alpha;
        m_ref = m_safe;
        if (m_new != -INFINITY) sum_limit = HEAD ? kHalfSumLimit : kSumLimit;
        exponentials(std::false_type{});
      }
      l_run += HEAD ? psum[0] * ivs[0] + psum[1] * ivs[1] : psum[0] + psum[1];
#pragma unroll
      for (int i = 0; i < 16; ++i) pop[i >> 3][i & 7] = (op)(FP8 && !HEAD ? p[i] * vscale[i >> 3] : p[i]);
    }
  };
  // ---- O^T += V^T P^T : A = V^T tile (32 dims x 16 tokens) read transposed from LDS, in front of the softmax
  using raw_v = std::conditional_t<FP8, intx2, bf16x8>;
  raw_v v_raw[2][kDT];
  auto read_values = [&](int slot) __attribute__((always_inline)) {
    const unsigned int v_at = lds + L_::v(slot);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt) {
        if constexpr (FP8) {
          typedef __attribute__((address_space(3))) intx2 lds_i2;
          const int t = ks * 16 + h2 * 8 + ((lane & 15) >> 1);
          const int col = ((dt * 2 + ((lane >> 4) & 1)) ^ tree_key_v<true>(t)) & (G_::kChunks - 1);
          v_raw[ks][dt] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2*)(uintptr_t)(v_at + t * G_::kRowBytes + col * 16 + (lane & 1) * 8));
        } else {
          typedef __attribute__((address_space(3))) shortx4 lds_s4;
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int j = lane & 15, t = ks * 16 + h2 * 8 + hf * 4 + (j >> 2);
            const int col = ((dt * 4 + ((lane >> 4) & 1) * 2 + ((j & 3) >> 1)) ^ tree_key_v<false>(t)) & (G_::kChunks - 1);
            const shortx4 raw = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(uintptr_t)(v_at + t * G_::kRowBytes + col * 16 + (j & 1) * 8));
            const bf16x4 h4 = __builtin_bit_cast(bf16x4, raw);
            v_raw[ks][dt][hf * 4 + 0] = h4[0]; v_raw[ks][dt][hf * 4 + 1] = h4[1]; v_raw[ks][dt][hf * 4 + 2] = h4[2]; v_raw[ks][dt][hf * 4 + 3] = h4[3];
          }
        }
      }
  };
  auto values = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt) {
        if constexpr (FP8) acc[dt] = mfma32(widen_v8<KV>((uint32_t)v_raw[ks][dt][0], (uint32_t)v_raw[ks][dt][1]), pop[ks], acc[dt]);
        else acc[dt] = mfma32(v_raw[ks][dt], pop[ks], acc[dt]);
      }
  };
  // Whether the values of a block hold any that is no number: then zeros take their places in front of the second product, and those of
  // the segment are added to what is stored of it.
  auto any_undefined = [&](int slot) __attribute__((always_inline)) {
    uint32_t any = 0;
#pragma unroll
    for (int j = 0; j < G_::kLoads; ++j) {
      const uint4_v w = *lds_at<const uint4_v>(lds + L_::v(slot) + j * 1024 + lane * 16);
      any |= undefined<KV>(w[0]) | undefined<KV>(w[1]) | undefined<KV>(w[2]) | undefined<KV>(w[3]);
    }
    return __builtin_amdgcn_ballot_w64(any != 0) != 0;
  };
  auto without_undefined = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < G_::kLoads; ++j) {
      const auto at = lds_at<uint4_v>(lds + L_::v(slot) + j * 1024 + lane * 16);
      const uint4_v w = *at;
      *at = uint4_v{defined<KV>(w[0]), defined<KV>(w[1]), defined<KV>(w[2]), defined<KV>(w[3])};
    }
  };

  int slot = 0;
  auto scales_of = [&](int slot) __attribute__((always_inline)) { 
    floatx4 x = {1.f, 1.f, 1.f, 1.f};
    if constexpr (FP8) x = *lds_at<const floatx4>(lds + L_::scales(slot, wave));
    return x;
  };
  for (int i = 0; i < min(W == 1 ? kSlots : kSlots - 1, n_mine); ++i) {
    if constexpr (W == 1) {
      issue_k(i);
      issue_v(i);
    } else {
      issue(i);
    }
  }
  constexpr std::integral_constant<int, kSlots - (W == 1 ? 1 : 2)> ahead_c{};   // blocks behind the one in work that are under way
  constexpr std::integral_constant<int, 0> c0{};
  bool begins = true;
  for (int i = n_mine; i > 0; --i) {                 // (blocks that are left)
    if (begins) begin_segment();
    const bool edge = cc.blk >= edge_blk;
    if constexpr (W == 1) {
      const bool more = i > kSlots, follow = i >= kSlots;
      await(follow, ahead_c, std::integral_constant<int, kVLoads>{});
      scores(slot);
      const floatx4 scales = scales_of(slot);
      if (more) {
        all_read();
        issue_k(slot);
        await(true, ahead_c, std::integral_constant<int, kKLoads>{});
      } else {
        await(follow, ahead_c, c0);
      }
      if constexpr (!INT8) {
        if (edge && any_undefined(slot)) {
          without_undefined(slot);
          dirty = true;
        }
      }
      read_values(slot);
      softmax(edge, scales);
      values();
      if (more) {
        all_read();
        issue_v(slot);
      }
    } else {
      await(i >= kSlots - 1, ahead_c, c0);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (left > 0) issue(slot == 0 ? kSlots - 1 : slot - 1);
      if constexpr (!INT8) {
        // (every wave looks at all of the tile, and none reads it for the product until all have put zeros into it)
        if (edge && any_undefined(slot)) {
          asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
          without_undefined(slot);
          asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
          dirty = true;
        }
      }
      if (rows_here > 0) {
        scores(slot);
        read_values(slot);
        softmax(edge, scales_of(slot));
        values();
      }
    }
    begins = cc.blk + 1 == cc.n;
    if (begins || i == 1) end_segment();
    if (i > 1) advance(cc);
    slot = slot + 1 == kSlots ? 0 : slot + 1;
  }
}

// The partition: as plan_decode's, with hkv * tiles rows of a trajectory, of its own number of tiles.  Blocks of b before all heads:
// prefix[b], in units of its KV heads.
__device__ __forceinline__ int tree_blocks(const TreeArgs& a, int b, int& per_row) {
  const int tiles = tree_tiles(a, a.q_lens[b]);
  per_row = tiles ? (a.ctx_lens[b] + kBlockTokens - 1) / kBlockTokens : 0;
  return tiles * per_row;
}

// The start of a worker's run, for a batch of at most 64 trajectories: worked out by every wave for itself, a lane per trajectory.  The first
// worker writes the header and the scan, which the merge reads.
__device__ __forceinline__ int4 tree_plan_in_wave(const TreeArgs& a, int worker) {
  const int lane = lane_id(), hkv = a.hkv;
  int per_row = 0, count = 0;
  if (lane < a.batch) count = tree_blocks(a, lane, per_row);
  const int upto = wave_inclusive_scan(count), first = upto - count;
  const int blocks = __builtin_amdgcn_readlane(upto, 63);
  const int total = blocks * hkv;
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
  const unsigned long long before = __builtin_amdgcn_ballot_w64(lane < a.batch && (unsigned int)(hkv * first) <= x);
  const int b = 63 - __builtin_clzll(before);
  const int n = __builtin_amdgcn_readlane(per_row, b);
  const int rem = (int)x - hkv * __builtin_amdgcn_readlane(first, b);
  return make_int4(b, ((rem / n) << 20) | (rem % n), 0, min(per, total - (int)x));
}

// Workgroups go to the XCDs in turn; workers that follow each other, whose rows may read the same K and V, have one XCD's cache in common.
template <int D, int KV, int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W, 2) void tree_mfma_kernel(const TreeArgs a) {
  constexpr int kWorkers = W == 1 ? 4 : 1;       // of a workgroup
  using L_ = TreeLds<D, kv_is_codes(KV), W>;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kWorkers][L_::kBytes];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = (int)(blockIdx.x % kXcds * (gridDim.x / kXcds) + blockIdx.x / kXcds);
  const int worker = group * kWorkers + (W == 1 ? wave : 0);
  int4 start;
  if (a.batch <= kWavePlanBatch) start = tree_plan_in_wave(a, worker);
  else start = *(const int4*)(a.wstart + 4 * worker);
  const int b = __builtin_amdgcn_readfirstlane(start.x), at = __builtin_amdgcn_readfirstlane(start.y), mine = __builtin_amdgcn_readfirstlane(start.w);
  if (b < 0) return;
  tree_worker<D, KV, W, true>(a, b, at >> 20, at & 0xFFFFF, mine, worker, W == 1 ? 0 : wave, (unsigned int)(uintptr_t)&lds[0][0] + (W == 1 ? wave * L_::kBytes : 0));
}

__global__ __launch_bounds__(kPlanThreads) void tree_plan_kernel(const TreeArgs a) {
  __shared__ int4 wave_tot[kPlanThreads / 256];
  __shared__ int prefix_s[kLdsPrefix + 1];
  const int tid = threadIdx.x, batch = a.batch, hkv = a.hkv;
  const bool in_lds = batch <= kLdsPrefix;
  int running = 0;
  for (int b0 = 0; b0 < batch; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int per_row, all;
    const int count = b < batch ? tree_blocks(a, b, per_row) : 0;
    const int first = running + block_exclusive_scan(count, wave_tot, &all);
    if (b < batch) {
      a.prefix[b] = first;
      if (in_lds) prefix_s[b] = first;
    }
    running += all;
  }
  if (tid == 0) {
    a.prefix[batch] = running;
    if (in_lds) prefix_s[batch] = running;
  }
  const int total = running * hkv, per = max(1, (total + a.workers - 1) / a.workers);
  if (tid == 0) a.header[kPlanPer] = per;
  __threadfence_block();
  __syncthreads();   // prefix[] written above is read below by other threads of this workgroup
  for (int w = tid; w < a.workers; w += kPlanThreads) {
    const long x = (long)w * per;
    int4 st = make_int4(-1, 0, 0, 0);
    if (x < total) {
      // largest b whose rows start at or before x (trajectories without blocks can never be the answer: the next one starts at the same place)
      const int* pf = in_lds ? prefix_s : a.prefix;
      int lo = 0, hi = batch;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((long)hkv * pf[mid] <= x) lo = mid; else hi = mid;
      }
      int n;
      tree_blocks(a, lo, n);
      const int rem = (int)(x - (long)hkv * pf[lo]);
      st = make_int4(lo, ((rem / n) << 20) | (rem % n), 0, (int)min((long)per, (long)total - x));
    }
    *(int4*)(a.wstart + 4 * w) = st;
  }
}

// Merge of the partials that runs left of rows they did not cover alone, as in combine.hip: one wave per (row, 32 query rows, 32 dims),
// lanes as in the accumulators, four pieces under way at a time; where those waves are few, a workgroup of four, which share the pieces and
// fold their sums in order.  A piece of which a query row saw nothing has weight zero.
// Bound by the latency of the partials' loads.
template <int D, bool TOGETHER>
__global__ __launch_bounds__(kThreads) void tree_merge_kernel(const TreeArgs a) {
  constexpr int kDT = D / 32;
  __shared__ __attribute__((aligned(16))) float sum_s[TOGETHER ? kWaves : 1][TOGETHER ? 4 : 1][TOGETHER ? 64 : 1][4];
  __shared__ float ml_s[TOGETHER ? kWaves : 1][TOGETHER ? 64 : 1][2];
  const int lane = lane_id(), n32 = lane & 31, h2 = lane >> 5, parts = a.tile_parts;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int unit = TOGETHER ? (int)blockIdx.x : (int)blockIdx.x * kWaves + wave;
  const int dt = unit % kDT, part0 = unit / kDT, most = a.row_tiles * parts;   // (of the longest draft: 32 query rows each)
  const int row = part0 / most, p = part0 - row * most, tile = p / parts, c = p - tile * parts, b = row / a.hkv, g = row - b * a.hkv;
  if (b >= a.batch) return;
  const int per = a.header[kPlanPer], first = a.prefix[b], all = a.prefix[b + 1] - first;
  const Draft d(a, b);
  const int j0 = p * kRows, tiles = tree_tiles(a, d.n);
  if (all == 0 || j0 >= d.n * a.group) return;
  const int n = all / tiles, r = g * tiles + tile;
  const long r0 = (long)a.hkv * first + (long)r * n;
  const int wf = (int)(r0 / per), wl = (int)((r0 + n - 1) / per), pieces = wl - wf + 1;
  if (pieces == 1) return;                                  // one worker had the whole row
  const int first_slot = ((long)wf * per < r0) ? 1 : 0;
  const bool ok = j0 + n32 < d.n * a.group;                 // (there are no partials of the others)
  floatx4 o[4];
#pragma unroll
  for (int i4 = 0; i4 < 4; ++i4) o[i4] = floatx4{0.f, 0.f, 0.f, 0.f};
  float ref = -INFINITY, l = 0.f;
  // folds (maximum, sum, values) of kN things into the sums; those past the last have weight zero (zero times an infinity would not be zero)
  auto fold = [&](auto n_c, int there, floatx2* x, floatx4 (*y)[4]) __attribute__((always_inline)) {
    constexpr int kN = decltype(n_c)::value;
    float top = ref;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      if (i >= there) {
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
  };
  constexpr int kN = 4;
  const int step = TOGETHER ? kWaves : 1, from = TOGETHER ? wave : 0;
  if (ok)
    for (int s0 = from; s0 < pieces; s0 += kN * step) {
      floatx2 x[kN];
      floatx4 y[kN][4];
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        const int s = min(s0 + i * step, pieces - 1);
        const size_t part = ((size_t)(wf + s) * 2 + (s == 0 ? first_slot : 0)) * parts + c;
        x[i] = *(const floatx2*)(a.partial_ml + (part * kRows + n32) * 2);
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) y[i][i4] = *(const floatx4*)(a.partial_o + part * (kRows * D) + ((dt * 4 + i4) * 64 + lane) * 4);
      }
      fold(std::integral_constant<int, kN>{}, (pieces - s0 + step - 1) / step, x, y);
    }
  if constexpr (TOGETHER) {
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) *(floatx4*)sum_s[wave][i4][lane] = o[i4];
    ml_s[wave][lane][0] = ref;
    ml_s[wave][lane][1] = l;
    __syncthreads();
    if (wave != 0 || !ok) return;
    floatx2 x[kWaves - 1];
    floatx4 y[kWaves - 1][4];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
      x[w - 1] = floatx2{ml_s[w][lane][0], ml_s[w][lane][1]};
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) y[w - 1][i4] = *(const floatx4*)sum_s[w][i4][lane];
    }
    fold(std::integral_constant<int, kWaves - 1>{}, kWaves - 1, x, y);
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
    hipLaunchKernelGGL(tree_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t units = (int64_t)a.batch * a.hkv * a.row_tiles * a.tile_parts * (head_dim / 32);
  const bool together = units <= kMergeTogether;
  const dim3 merge_grid((unsigned)(together ? units : (units + kWaves - 1) / kWaves));
  auto launch = [&](auto d, auto kind, auto w) {
    constexpr int W = decltype(w)::value;
    hipLaunchKernelGGL((tree_mfma_kernel<decltype(d)::value, decltype(kind)::value, W>), dim3(a.workers / (W == 1 ? 4 : 1)), dim3(W == 1 ? 256 : 64 * W), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (together) hipLaunchKernelGGL((tree_merge_kernel<decltype(d)::value, true>), merge_grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((tree_merge_kernel<decltype(d)::value, false>), merge_grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
  };
  auto of_tiles = [&](auto d, auto kind) {
    switch (a.tile_parts) {
      case 1: return launch(d, kind, std::integral_constant<int, 1>{});
      case 2: return launch(d, kind, std::integral_constant<int, 2>{});
      case 4: return launch(d, kind, std::integral_constant<int, 4>{});
      case 8: return launch(d, kind, std::integral_constant<int, 8>{});
    }
    return hipErrorInvalidValue;
  };
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
