// Attention of a tree of drafted tokens (bf16 queries) over bf16 or 8-bit (E4M3, int8) paged KV (gfx950).
//
// A query row is a (drafted token, query head of the group) pair, token-major, so the heads that share the KV head and the tokens of a draft that
// fit one tile read K and V once; a wave has 32 of them.  A row is (trajectory, KV head, tile of query rows): of 32, or 64, as teams of four waves
// that share its 32-token blocks take them, else of as many as the 2, 4 or 8 waves of a workgroup have that go through its blocks together.  As in
// decode, the steps of all rows (of as many blocks as a worker does at a time) are laid end to end, and every worker, a workgroup, has one equal run
// of that sequence; short tables' rows are not cut.  A worker streams its run from memory straight into LDS, and each wave consumes a block with
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
// Up to so many merged tiles of 32 query rows and 32 dims, a workgroup of four waves shares a tile's pieces: 57.1 -> 49.4 us for 3 drafts behind
// 2k .. 32k, whose rows are of hundreds of pieces.  Above, a wave has a tile for itself (64 drafts behind 1k .. 8k, 4096 tiles: 140.2, shared 144.8).
constexpr int kMergeTogether = 2048;
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
constexpr int kHalves = -1;               // (codes that have become f16)
template <int KV>
__device__ __forceinline__ uint32_t undefined(uint32_t w) {
  if constexpr (KV == kHalves) return ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u;
  else if constexpr (KV == kKvBf16) return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  else if constexpr (KV == kKvInt8Head) return 0;
  else return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}
// The word with zeros in the place of those.
template <int KV>
__device__ __forceinline__ uint32_t defined(uint32_t w) {
  const uint32_t met = undefined<KV>(w) >> (KV == kKvBf16 || KV == kHalves ? 15 : 7);
  return w & ~(met * (KV == kKvBf16 || KV == kHalves ? 0xffffu : 0xffu));
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

// A ring of blocks in LDS: a wave's own (W = 1), or that of W waves together.  Addresses are 32-bit offsets in the LDS.
template <int D, bool FP8, int W>
struct TreeLds {
  static constexpr int kSlots = W == 1 ? (FP8 ? 2 : 1) : W == 2 ? (FP8 ? 4 : 2) : 4;
  static constexpr int kTile = Geo<D, FP8>::kTileBytes, kScales = FP8 ? 256 : 0;   // scales of a block's two pages: K's, V's (the other lanes' are copies)
  // Codes that eight waves share are widened once, into one of two tiles of 16-bit operands, and not by each wave for itself: 64 drafts of 24 .. 72
  // behind 1k .. 8k (64/4/128) 740 -> 559 us over int8 and 637 -> 542 over E4M3 pools, of 9 .. 16 261 -> 190 and 227 -> 186.  Four waves gain
  // nothing (of 5 .. 8, 121 -> 120 and 102 -> 118), nor do heads of 64, whose rows need more LDS reads to a product (of 40 .. 64 with 8/2/64
  // over E4M3 87 -> 103).
  static constexpr bool kWidens = FP8 && W == 8 && D == 128;
  static constexpr int kWide = kWidens ? Geo<D, false>::kTileBytes : 0, kCodes = kSlots * (2 * kTile + W * kScales), kRing = kCodes + 4 * kWide;
  static __device__ __forceinline__ unsigned int wide_k(int at) { return kCodes + at * kWide; }
  static __device__ __forceinline__ unsigned int wide_v(int at) { return kCodes + (2 + at) * kWide; }
  static __device__ __forceinline__ unsigned int k(int slot) { return slot * kTile; }
  static __device__ __forceinline__ unsigned int v(int slot) { return (kSlots + slot) * kTile; }
  static __device__ __forceinline__ unsigned int scales(int slot, int wave) { return 2 * kSlots * kTile + (slot * W + wave) * kScales; }
};
// The rings of a team of four waves, one each or one for two; and in their places, when a segment is done, what each wave's blocks came to: four
// values of a lane, as the accumulators lie, and (maximum, sum) of a query row.
template <int D, bool FP8>
struct TeamLds {
  static constexpr int kPart = kRows * D * 4, kEach = kPart + kRows * 8;
  static constexpr int kOne = TreeLds<D, FP8, 1>::kRing, kTwo = TreeLds<D, FP8, 2>::kRing;
  static constexpr int kMost = kEach > kOne ? kEach : kOne, kRoom = (2 * kMost > kTwo ? 2 * kMost : kTwo) + 2047 & ~2047;   // of two waves
  static constexpr int kBytes = 2 * kRoom;
  static __device__ __forceinline__ unsigned int of_wave(int wave) { return wave * (kRoom / 2); }
  static __device__ __forceinline__ unsigned int part(int dt, int i4, int lane) { return ((dt * 4 + i4) * 64 + lane) * 16; }
  static __device__ __forceinline__ unsigned int ml(int row) { return kPart + row * 8; }
};
template <class T>
__device__ __forceinline__ __attribute__((address_space(3))) T* lds_at(unsigned int at) { return (__attribute__((address_space(3))) T*)(uintptr_t)at; }

// Values of a segment's blocks that are no numbers, which its sums leave out, to the row of `node`, where that sees them: add(dim, four of them).
// They were left out of every block that ends behind the prefix, so of the last cached tokens, too, which all rows see.  Rare, and one token
// after the other.
template <int D, int KV, class F>
__device__ __forceinline__ void add_undefined(const Draft& d, int b, int g, int node, int blk0, int n, int stride, int h2, F&& add) {
  const tree_args_p e = tree_args();
  const uint64_t* const words = e->mask + (size_t)(d.off + node) * e->mask_words;
  const int prefix = d.len - d.n;
  for (int blk = blk0; n > 0; --n, blk += stride)
    for (int t = max(prefix / kBlockTokens, blk) * kBlockTokens; t < min(d.len, (blk + 1) * kBlockTokens); ++t) {
      const int rel = t - prefix;
      if (rel >= 0 && (rel >= 64 * e->mask_words || !(words[rel >> 6] >> (rel & 63) & 1))) continue;
      const size_t row = ((size_t)e->page_table[(size_t)b * e->max_pages + t / kPageSize] * e->hkv + g) * kPageSize + t % kPageSize;
      for (int dim = h2 * 4; dim < D; dim += 8) {
        floatx4 x;
        if constexpr (kv_is_codes(KV)) {
          const uint32_t w = *(const uint32_t*)((const unsigned char*)e->v_pages + row * D + dim);
          if (!undefined<KV>(w)) continue;
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = (w >> (8 * i) & 0x7f) == 0x7f ? NAN : 0.f;
        } else {
          const uint2 w = *(const uint2*)((const __bf16*)e->v_pages + row * D + dim);
          if (!undefined<KV>(w.x) && !undefined<KV>(w.y)) continue;
          const uint32_t bits[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = (bits[i] & 0x7f800000u) == 0x7f800000u ? __uint_as_float(bits[i]) : 0.f;
        }
        add(dim, x);
      }
    }
}

// What a wave's blocks of a row come to: O^T (lane (row n32, half h2) holds dims dt*32 + (i/4)*8 + h2*4 + i%4), the row's maximum (or a reference
// near it, log2 units) and sum; undefined: values that are no numbers have been left out.
template <int D>
struct TreeSums {
  floatx16 acc[D / 32];
  float ref, sum;
  bool undefined;
};

// n_mine blocks blk0, blk0 + stride, .. of KV head g of trajectory b, for the query rows j0 .. j0 + rows_here - 1 of its draft (none: a wave past
// the last row helps with the loads).
// Loads.  W = 1: the tiles of block i + slots go into the places of block i, K's as soon as the first product has read them and V's behind
// the second; no barriers.  Else each wave loads its share of a block, waits for its own loads and meets the others at one barrier per block:
// behind it the block is there, and the place of the block before is free for the one that is slots - 1 ahead.  rounds: barriers, as many for
// all waves of the workgroup (n_mine or more).  Where codes are widened once for all, the next block is there, too, and becomes operands, each
// wave its share, in the tile that the block before has left.
// HBM -> LDS without a register stop: lane l's 16 bytes land at M0 + 16 l, so a row's chunks are swizzled by the address a lane
// reads from.  The compiler does not see these loads as loads; they are awaited by count: vector-memory counts go down in order, so
// with N of these loads sent after the ones that are waited for, no more than N outstanding operations of any kind means that those have
// landed (others in between only make the wait longer).
template <int D, int KV, int W>
__device__ __forceinline__ TreeSums<D> tree_blocks_of(const TreeArgs& a, const Draft& d, int b, int g, int j0, int rows_here, int blk0, int n_mine,
                                                      int stride, int rounds, int wave, unsigned int lds) {
  constexpr bool FP8 = kv_is_codes(KV), HEAD = kv_has_head_scales(KV);   // FP8: 8-bit codes of either kind
  constexpr bool INT8 = KV == kKvInt8Head;
  constexpr int kSlots = TreeLds<D, FP8, W>::kSlots;
  using L_ = TreeLds<D, FP8, W>;
  constexpr int kKK = D / 16, kDT = D / 32;
  using kx8 = std::conditional_t<INT8, halfx8, bf16x8>;   // operands of the first product
  using opx8 = std::conditional_t<HEAD, halfx8, bf16x8>;  // ... and of the second
  using op = std::conditional_t<HEAD, _Float16, __bf16>;
  using G_ = Geo<D, FP8>;
  constexpr bool kWidens = L_::kWidens, RAW8 = FP8 && !kWidens;   // RAW8: operands are codes in LDS
  using O_ = Geo<D, RAW8>;
  // this wave's loads of a block: of each pool's tile its share, or where there are more waves than a tile has loads, of one pool's tile one
  // (where there are more than both have, some twice: the same bytes to the same place); its copy of the scales
  constexpr int kShare = G_::kLoads >= W ? G_::kLoads / W : 1;
  constexpr int kVLoads = G_::kLoads >= W ? kShare : 0, kKLoads = kShare + (FP8 ? 1 : 0);
  const int lane = lane_id();
  const int n32 = lane & 31;   // query row (B column) / K token row (A row) carried by this lane
  const int h2 = lane >> 5;    // half of the contraction this lane feeds

  const int hkv = a.hkv;
  constexpr size_t tile_stride = (size_t)kPageSize * G_::kRowBytes;   // bytes of one (page, head) tile

  // ---- producer: a window of 64 page ids (32 of this wave's blocks), one per lane
  int pid_vec = 0, pid_next = 0, sent = 0;    // blocks that have been sent for
  int p_page[2] = {0, 0}, p_lim = 0;          // the block under way: its pages, and tokens from its first on
  size_t p_at[2] = {0, 0};                    // ... and where this wave's loads find them in a pool
  auto load_window = [&](int k) {
    const tree_args_p e = tree_args();
    const int pg = (blk0 + (k * 32 + (lane >> 1)) * stride) * 2 + (lane & 1);
    return (pg < ((d.len + kPageSize - 1) >> 4)) ? e->page_table[(size_t)b * e->max_pages + pg] : 0;
  };
  auto dma16 = [&](const unsigned char* base, unsigned int off, unsigned int dst) __attribute__((always_inline)) {
    const unsigned int m0 = __builtin_amdgcn_readfirstlane(dst);
    // (streamed: read once.  The tiles of larger drafts follow each other through the same blocks, and find some in the caches: 24 drafts of 24 .. 72
    // behind 1k .. 8k (64/4/128) 167 -> 161 us over bf16, 343 -> 321 over int8 pools; of one tile, 9 .. 16, 77 -> 78 and 123 -> 124.  Hint taken from
    // the smaller ones, 64 of 6 .. 16 behind 512 .. 8k (32/8/128): 140 -> 156.)
    if constexpr (W < 8) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(m0), "v"(off), "s"(base) : "memory");
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
  // what the next block needs
  auto look_up = [&]() __attribute__((always_inline)) {
    const int in = sent & 31;
    if (in == 0) {
      const int k = sent >> 5;
      pid_vec = k == 0 ? load_window(0) : pid_next;
      // (here the compiler waits for it; left to the uses below it would wait in front of every block, and for all loads under way)
      asm volatile("" : "+v"(pid_vec));
      pid_next = load_window(k + 1);
    }
    p_lim = d.len - (blk0 + sent * stride) * kBlockTokens;
    // (a page that the row's last block does not have: the one in front of it)
    const int last = p_lim > kPageSize ? 1 : 0;
    if constexpr (kShare == 1 && !FP8) {
      p_page[0] = __builtin_amdgcn_readlane(pid_vec, in * 2 + (upper ? last : 0));
    } else {
      p_page[0] = __builtin_amdgcn_readlane(pid_vec, in * 2);
      p_page[1] = __builtin_amdgcn_readlane(pid_vec, in * 2 + last);
    }
    auto at = [&](int page) { return (size_t)(unsigned int)__builtin_amdgcn_readfirstlane(page * hkv + g) * tile_stride; };
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
      const float* from = (lane & 2 ? a.v_scale : a.k_scale) + (HEAD ? (size_t)page * hkv + g : (size_t)page);
      const unsigned int m0 = __builtin_amdgcn_readfirstlane(lds + L_::scales(slot, wave));
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(m0), "v"(from) : "memory");
    }
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
    ++sent;
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
    ++sent;
  };
  // until all but this wave's loads of kBlocks blocks, and kMore others, have landed; near the run's end, where fewer blocks follow, of none
  auto await = [&](bool follow, auto blocks_c, auto more_c) __attribute__((always_inline)) {
    constexpr int kMore = decltype(more_c)::value, kBlock = kVLoads + kKLoads;
    if (follow) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(blocks_c)::value * kBlock + kMore) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMore) : "memory");
  };

  // ---- consumer state
  TreeSums<D> own;
  floatx16 (&acc)[kDT] = own.acc;
  own.undefined = false;
  float m_ref = 0.f, l_run = 0.f;   // reference of this lane's row (log2 units), zero as long as it has seen nothing; its share of the running sum
  float sum_limit = -1.f;           // a lane's exponentials of a block may add up to this much; below zero: no reference yet
  const int edge_blk = (d.len - d.n) / kBlockTokens;       // first block with tokens behind the prefix

  kx8 qop[kKK];              // Q^T as the B operand: lane (row n32, half h2), 8 dims per step
  float q_unit;              // what a unit of this lane's row is worth, softmax scale included
  auto load_queries = [&]() __attribute__((always_inline)) {
    const tree_args_p e = tree_args();
    const bool flip = e->scale_log2 < 0.f;           // (queries the other way round, so that larger scores are larger exponents)
    const float scale_log2 = __builtin_fabsf(e->scale_log2);
    // (rows past the last read it again; what becomes of them is not stored)
    const RowAt at(*e, d, g, max(0, min(j0 + n32, d.n * e->group - 1)));
    const __bf16* qrow = (const __bf16*)e->q + at.out * D;
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) {
      // RAW8: 16-byte K chunks hold 16 dims; step 2p+e uses bytes e*8.. of chunk p*2+h2
      uint4 v = *(const uint4*)(qrow + (RAW8 ? ((kk >> 1) * 2 + h2) * 16 + (kk & 1) * 8 : kk * 16 + h2 * 8));
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
  };

  floatx16 s;
  // ---- S^T = K Q^T.  All operands are on their way before the first product: the products hang together and would each wait for a trip to
  // the LDS.
  constexpr int kKeyReads = RAW8 ? kKK / 2 : kKK;
  uint4_v k_raw[kKeyReads];
  auto read_keys = [&](int slot) __attribute__((always_inline)) {
    const int t = (n32 & 16) + tau(n32 & 15);
    const unsigned int rowp = lds + (kWidens ? L_::wide_k(slot & 1) : L_::k(slot)) + t * O_::kRowBytes;
    const int key = tree_key_k<D, RAW8>(t);
#pragma unroll
    for (int i = 0; i < kKeyReads; ++i) k_raw[i] = *lds_at<const uint4_v>(rowp + (((i * 2 + h2) ^ key) & (O_::kChunks - 1)) * 16);
  };
  auto scores = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int i = 0; i < kKeyReads; ++i) {
      if constexpr (RAW8) {
        s = mfma32(widen_k8<KV>(k_raw[i][0], k_raw[i][1]), qop[2 * i], s);
        s = mfma32(widen_k8<KV>(k_raw[i][2], k_raw[i][3]), qop[2 * i + 1], s);
      } else {
        s = mfma32(__builtin_bit_cast(kx8, k_raw[i]), qop[i], s);
      }
    }
  };
  // This lane then holds, for its rows, the scores of tokens tok0 + (i/8)*16 + h2*8 + i%8: eight of each page.
  opx8 pop[2];
  unsigned int seen = 0;                             // bit i: of this lane's score i (set in the blocks behind the prefix alone)
  auto softmax = [&](int blk, bool edge, const floatx4& scales) __attribute__((always_inline)) {
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
        const int j = max(0, min(j0 + n32, d.n * e->group - 1)), n_words = e->mask_words;
        const uint64_t* words = e->mask + (size_t)(d.off + j / e->group) * n_words;
        seen = 0;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) seen |= seen_bits(words, n_words, blk * kBlockTokens + pg * kPageSize + h2 * 8 - (d.len - d.n), d.n, 0xffu) << (8 * pg);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = seen >> i & 1 ? s[i] : -INFINITY;
      }
      // The reference of a row only moves when it has to: exponentials are taken against it as it stands, and may exceed one.  Only when
      // a lane's add up to more than kSumLimit (f16 weights: a page's to kHalfSumLimit, so that none is too large for f16), or while a row has no
      // reference, is its maximum found, the reference moved there and the row's exponentials of the block taken again.
      float psum[2], p[16];
      bool moves = false;                                    // this lane's row does (the others' stay, whatever their neighbours are)
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
          const float y = __builtin_amdgcn_exp2f(x);
          p[i] = decltype(first_c)::value || moves ? y : p[i];
          psum[pg] = (i & 7) == 0 ? p[i] : psum[pg] + p[i];
        }
      };
      exponentials(std::true_type{});
      // (an undefined sum takes the slow way, too; HEAD: it need not, the row is undefined with either)
      const uint64_t past = __builtin_amdgcn_ballot_w64(!((HEAD ? fmaxf(psum[0], psum[1]) : psum[0] + psum[1]) <= sum_limit));
      if (past) {
        moves = ((uint32_t)past | (uint32_t)(past >> 32)) >> n32 & 1;
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
        const float m_old = sum_limit < 0.f ? -INFINITY : m_ref, m_new = moves ? fmaxf(m_old, top) : m_old;
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
      // The weights are rounded for the second product, the sum is not: to bf16 (2^-8 of each at most) where the values have bf16's range or a
      // scale for their page, as in the other calls over such pools, and to f16 (2^-11) where codes are exact in it.
#pragma unroll
      for (int i = 0; i < 16; ++i) pop[i >> 3][i & 7] = (op)(FP8 && !HEAD ? p[i] * vscale[i >> 3] : p[i]);
    }
  };
  // ---- O^T += V^T P^T : A = V^T tile (32 dims x 16 tokens) read transposed from LDS, in front of the softmax
  using raw_v = std::conditional_t<RAW8, intx2, bf16x8>;
  raw_v v_raw[2][kDT];
  auto read_values = [&](int slot) __attribute__((always_inline)) {
    const unsigned int v_at = lds + (kWidens ? L_::wide_v(slot & 1) : L_::v(slot));
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt) {
        if constexpr (RAW8) {
          typedef __attribute__((address_space(3))) intx2 lds_i2;
          const int t = ks * 16 + h2 * 8 + ((lane & 15) >> 1);
          const int col = ((dt * 2 + ((lane >> 4) & 1)) ^ tree_key_v<true>(t)) & (O_::kChunks - 1);
          v_raw[ks][dt] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2*)(uintptr_t)(v_at + t * O_::kRowBytes + col * 16 + (lane & 1) * 8));
        } else {
          typedef __attribute__((address_space(3))) shortx4 lds_s4;
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int j = lane & 15, t = ks * 16 + h2 * 8 + hf * 4 + (j >> 2);
            const int col = ((dt * 4 + ((lane >> 4) & 1) * 2 + ((j & 3) >> 1)) ^ tree_key_v<false>(t)) & (O_::kChunks - 1);
            const shortx4 raw = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(uintptr_t)(v_at + t * O_::kRowBytes + col * 16 + (j & 1) * 8));
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
        if constexpr (RAW8) acc[dt] = mfma32(widen_v8<KV>((uint32_t)v_raw[ks][dt][0], (uint32_t)v_raw[ks][dt][1]), pop[ks], acc[dt]);
        else acc[dt] = mfma32(__builtin_bit_cast(opx8, v_raw[ks][dt]), pop[ks], acc[dt]);
      }
  };
  // Where the values hold any that is no number, zeros take their places, and those of the segment are added to what is stored of it.
  auto without_undefined = [&]() __attribute__((always_inline)) {
    if constexpr (!INT8) {
      constexpr int kWords = RAW8 ? 2 : 4, kAs = RAW8 ? KV : HEAD ? kHalves : kKvBf16;
      typedef unsigned int words_v __attribute__((ext_vector_type(kWords)));
      uint32_t any = 0;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) {
          const words_v w = __builtin_bit_cast(words_v, v_raw[ks][dt]);
#pragma unroll
          for (int i = 0; i < kWords; ++i) any |= undefined<kAs>(w[i]);
        }
      if (__builtin_amdgcn_ballot_w64(any != 0)) {
        own.undefined = true;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int dt = 0; dt < kDT; ++dt) {
            words_v w = __builtin_bit_cast(words_v, v_raw[ks][dt]);
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = defined<kAs>(w[i]);
            v_raw[ks][dt] = __builtin_bit_cast(raw_v, w);
          }
      }
    }
  };
  // ---- codes of 16 dims of a row to operands: each wave its share of a block
  constexpr int kPieces = kWidens ? 2 * kBlockTokens * (D / 16) : 0, kEach = kWidens ? (kPieces + 64 * W - 1) / (64 * W) : 0;
  uint4_v codes[kWidens ? kEach : 1];
  auto piece = [&](int n, int& row, int& c) __attribute__((always_inline)) {       // (whether there is one, and it is of V)
    const int at = n * 64 * W + wave * 64 + lane;
    row = at / (D / 16) % kBlockTokens;
    c = at % (D / 16);
    return at < kPieces / 2 ? 0 : at < kPieces ? 1 : 2;
  };
  auto read_codes = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < kEach; ++n) {
      int row, c;
      const int which = piece(n, row, c);
      const int key = which == 1 ? tree_key_v<true>(row) : tree_key_k<D, true>(row);
      if (which < 2) codes[n] = *lds_at<const uint4_v>(lds + (which == 1 ? L_::v(slot) : L_::k(slot)) + row * G_::kRowBytes + ((c ^ key) & (G_::kChunks - 1)) * 16);
    }
  };
  auto write_wide = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < kEach; ++n) {
      int row, c;
      const int which = piece(n, row, c);
      if (which == 0) {
        const unsigned int at = lds + L_::wide_k(slot & 1) + row * O_::kRowBytes;
        const int key = tree_key_k<D, false>(row);
#pragma unroll
        for (int e = 0; e < 2; ++e) *lds_at<uint4_v>(at + (((c * 2 + e) ^ key) & (O_::kChunks - 1)) * 16) = __builtin_bit_cast(uint4_v, widen_k8<KV>(codes[n][2 * e], codes[n][2 * e + 1]));
      } else if (which == 1) {
        const unsigned int at = lds + L_::wide_v(slot & 1) + row * O_::kRowBytes;
        const int key = tree_key_v<false>(row);
#pragma unroll
        for (int e = 0; e < 2; ++e) *lds_at<uint4_v>(at + (((c * 2 + e) ^ key) & (O_::kChunks - 1)) * 16) = __builtin_bit_cast(uint4_v, widen_v8<KV>(codes[n][2 * e], codes[n][2 * e + 1]));
      }
    }
  };
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
  load_queries();
  constexpr std::integral_constant<int, kSlots - (W == 1 ? 1 : 2)> ahead_c{};   // blocks behind the one in work that are under way
  constexpr std::integral_constant<int, 0> c0{};
  int slot = 0, blk = blk0;
  if constexpr (kWidens) {
    await(n_mine >= kSlots - 1, std::integral_constant<int, kSlots - 2>{}, c0);
    asm volatile("s_barrier" ::: "memory");
    read_codes(0);
    write_wide(0);
  }
  for (int i = n_mine, rest = W == 1 ? n_mine : rounds; rest > 0; --i, --rest, blk += stride) {               // (blocks that are left)
    const bool edge = blk >= edge_blk;
    if constexpr (W == 1) {
      const bool more = i > kSlots, follow = i >= kSlots;
      await(follow, ahead_c, std::integral_constant<int, kVLoads>{});
      read_keys(slot);
      __builtin_amdgcn_sched_barrier(0);
      scores();
      const floatx4 scales = scales_of(slot);
      if (more) {
        all_read();
        issue_k(slot);
        await(true, ahead_c, std::integral_constant<int, kKLoads>{});
      } else {
        await(follow, ahead_c, c0);
      }
      read_values(slot);
      softmax(blk, edge, scales);
      if (edge) without_undefined();
      values();
      if (more) {
        all_read();
        issue_v(slot);
      }
    } else {
      if (i > 0) await(i >= kSlots - 1, std::integral_constant<int, kSlots - 2 - (kWidens ? 1 : 0)>{}, c0);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (sent < n_mine) issue(slot == 0 ? kSlots - 1 : slot - 1);
      const int next = slot + 1 == kSlots ? 0 : slot + 1;
      if constexpr (kWidens) {
        if (i > 1) {
          read_codes(next);
          write_wide(next);
        }
      }
      if (rows_here > 0 && i > 0) {
        read_keys(slot);
        __builtin_amdgcn_sched_barrier(0);
        scores();
        read_values(slot);
        softmax(blk, edge, scales_of(slot));
        if (edge) without_undefined();
        values();
      }
    }
    slot = slot + 1 == kSlots ? 0 : slot + 1;
  }
  own.ref = sum_limit < 0.f ? -INFINITY : m_ref;
  own.sum = xor32_add(l_run);
  return own;
}

// The partition: as plan_decode's, with hkv * tiles rows of a trajectory, of its own number of tiles, and in steps: what a worker's waves do at a
// time, a block for every run of its waves along the row.  Steps of b before all heads: prefix[b], in units of its KV heads.
__device__ __forceinline__ int tree_steps(const TreeArgs& a, int b, int& per_row) {
  const int n = a.q_lens[b], tiles = tree_tiles(a, n), along = a.along;
  per_row = tiles ? ((a.ctx_lens[b] + kBlockTokens - 1) / kBlockTokens + along - 1) / along : 0;
  return tiles * per_row;
}

// The start of a worker's run, for a batch of at most 64 trajectories: worked out by every wave for itself, a lane per trajectory.  The first
// worker writes the header and the scan, which the merge reads.
__device__ __forceinline__ int4 tree_plan_in_wave(const TreeArgs& a, int worker) {
  const int lane = lane_id(), hkv = a.hkv;
  int per_row = 0, count = 0;
  if (lane < a.batch) count = tree_steps(a, lane, per_row);
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

__global__ __launch_bounds__(kPlanThreads) void tree_plan_kernel(const TreeArgs a) {
  __shared__ int4 wave_tot[kPlanThreads / 256];
  __shared__ int prefix_s[kLdsPrefix + 1];
  const int tid = threadIdx.x, batch = a.batch, hkv = a.hkv;
  const bool in_lds = batch <= kLdsPrefix;
  int running = 0;
  for (int b0 = 0; b0 < batch; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int per_row, all;
    const int count = b < batch ? tree_steps(a, b, per_row) : 0;
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
      tree_steps(a, lo, n);
      const int rem = (int)(x - (long)hkv * pf[lo]);
      st = make_int4(lo, ((rem / n) << 20) | (rem % n), 0, (int)min((long)per, (long)total - x));
    }
    *(int4*)(a.wstart + 4 * w) = st;
  }
}

// Folds (maximum, sum, values) of kN parts, of which `there` are there, into those of the sums.  Those past the last have weight zero (zero times
// an infinity would not be zero).
template <int kN>
__device__ __forceinline__ void fold_parts(float& ref, float& l, floatx4 (&o)[4], int there, floatx2 (&x)[kN], floatx4 (&y)[kN][4]) {
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
}

// 32 dims of query row j of a draft, as a lane holds them of its sums.
__device__ __forceinline__ void store_folded(const TreeArgs& a, const Draft& d, int g, int j, int D, int dt, int h2, float ref, float l, const floatx4 (&o)[4]) {
  const RowAt at(a, d, g, j);
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

// A worker's run: a segment of a row after the other, until its steps are done.  seg(d, b, g, tile, step of the row, steps, is this all of the
// row, where its partial goes if not)
template <class F>
__device__ __forceinline__ void tree_run(const TreeArgs& a, int worker, F&& seg) {
  int4 start;
  if (a.batch <= kWavePlanBatch) start = tree_plan_in_wave(a, worker);
  else start = *(const int4*)(a.wstart + 4 * worker);
  int b = __builtin_amdgcn_readfirstlane(start.x), left = __builtin_amdgcn_readfirstlane(start.w);
  if (b < 0) return;
  const int at = __builtin_amdgcn_readfirstlane(start.y);
  int first = at & 0xFFFFF, r = at >> 20;
  for (int slot = 0;; slot = 1) {
    const tree_args_p e = tree_args();
    const Draft d(*e, b);
    const int tiles = tree_tiles(*e, d.n), along = e->along;
    const int steps = tiles ? ((d.len + kBlockTokens - 1) / kBlockTokens + along - 1) / along : 0;
    if (steps > 0) {
      const int g = r / tiles, now = min(left, steps - first);
      seg(d, b, g, r - g * tiles, first, now, now == steps, (size_t)worker * 2 + slot);
      left -= now;
      if (left <= 0) return;
      __syncthreads();                                     // (the ring is free)
      first = 0;
      if (++r < tiles * e->hkv) continue;
    }
    r = 0;
    ++b;
  }
}

// Workgroups go to the XCDs in turn; workers that follow each other, whose rows may read the same K and V, have one XCD's cache in common.
__device__ __forceinline__ int xcd_order() { return (int)(blockIdx.x % kXcds * (gridDim.x / kXcds) + blockIdx.x / kXcds); }

// Small drafts.  A workgroup is a team: of four waves that have every fourth block of a segment each, without a barrier among them (up to 32 query
// rows per KV head), or of two pairs of waves that have every second (PAIRS: up to 64, over bf16 pools).  What they come to is joined in LDS when
// the segment ends, 32 dims to a wave, so that a cut costs one partial of a row and not four.  Measured against a worker for every wave, or for every
// two, with its own equal run (us):
//   64 drafts of 1 .. 8 behind 4000 tokens (32/8/128, bf16) 188 -> 163 (6.5 TB/s), 8 of them 35 -> 29, 3 of 5 .. 16 behind 2k .. 32k (pairs) 50 -> 47,
//   64 of 6 .. 16 behind 512 .. 8k (pairs) 140 -> 140; int8 pools in pairs lose: 160 of 2 .. 4 behind 1k .. 16k (64/4/128) 240 -> 248.
// Waves that read the blocks of a pair twice, through the caches, in place of a ring for two: 140 -> 182 (64 of 6 .. 16).
// WHOLE: a workgroup has a row of 32 query rows to itself, without plan and merge, for tables of up to kTreeWholePages pages: 1 draft of 1 .. 8
// behind 500 / 1000 / 2000 tokens 12.9 -> 9.6 / 15.5 -> 14.0 / 15.6 -> 23, 64 of them 29.7 -> 23.8 / 48.7 -> 42.9 / 86.7 -> 80.8.
template <int D, int KV, bool WHOLE, bool PAIRS>
__global__ __launch_bounds__(256, 2) void tree_team_kernel(const TreeArgs a) {
  constexpr int kDT = D / 32;
  using L_ = TeamLds<D, kv_is_codes(KV)>;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[L_::kBytes];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned int base = (unsigned int)(uintptr_t)&lds[0];
  auto seg = [&](const Draft& d, int b, int g, int tile, int step0, int steps, bool whole, size_t slot) __attribute__((always_inline)) {
    const int lane = lane_id(), n32 = lane & 31, h2 = lane >> 5;
    constexpr int along = PAIRS ? 2 : 4;
    const int half = PAIRS ? wave & 1 : 0, t = PAIRS ? wave >> 1 : wave;
    const int blocks = min(steps * along, (d.len + kBlockTokens - 1) / kBlockTokens - step0 * along), n_mine = (blocks - t + along - 1) / along;
    const int j0 = (tile + half) * kRows, rows_here = min(kRows, d.n * a.group - j0), blk0 = step0 * along + t;
    auto leave = [&](const TreeSums<D>& own) __attribute__((always_inline)) {
      const unsigned int mine = base + L_::of_wave(wave);
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4)
          *lds_at<floatx4>(mine + L_::part(dt, i4, lane)) = floatx4{own.acc[dt][i4 * 4], own.acc[dt][i4 * 4 + 1], own.acc[dt][i4 * 4 + 2], own.acc[dt][i4 * 4 + 3]};
      if (h2 == 0) *lds_at<floatx2>(mine + L_::ml(n32)) = floatx2{own.ref, own.sum};
      if (own.undefined && n32 < rows_here)
        add_undefined<D, KV>(d, b, g, (j0 + n32) / a.group, blk0, n_mine, along, h2,
                             [&](int dim, floatx4 x) { *lds_at<floatx4>(mine + L_::part(dim / 32, dim / 8 % 4, lane)) += x; });
    };
    if constexpr (PAIRS) {
      const TreeSums<D> own = tree_blocks_of<D, KV, 2>(a, d, b, g, j0, rows_here, blk0, n_mine, along, steps, half, base + L_::of_wave(wave & 2));
      __syncthreads();                                      // (the partner has read the last block)
      leave(own);
    } else {
      if (n_mine > 0) leave(tree_blocks_of<D, KV, 1>(a, d, b, g, j0, rows_here, blk0, n_mine, along, 0, 0, base + L_::of_wave(wave)));
    }
    __syncthreads();
    const int there = min(along, blocks);
    for (int dt = t; dt < kDT; dt += along) {
      if (n32 >= rows_here) break;
      floatx2 x[along];
      floatx4 o[4], y[along][4];
#pragma unroll
      for (int i = 0; i < along; ++i) {
        const int from = min(i, there - 1);
        const unsigned int at = base + L_::of_wave(PAIRS ? from * 2 + half : from);
        x[i] = *lds_at<const floatx2>(at + L_::ml(n32));
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) y[i][i4] = *lds_at<const floatx4>(at + L_::part(dt, i4, lane));
      }
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) o[i4] = floatx4{0.f, 0.f, 0.f, 0.f};
      float ref = -INFINITY, l = 0.f;
      fold_parts(ref, l, o, there, x, y);
      if (WHOLE || whole) {
        store_folded(a, d, g, j0 + n32, D, dt, h2, ref, l, o);
      } else {
        const size_t part = slot * a.tile_parts + half;
        float* const dst = a.partial_o + part * (kRows * D) + (dt * 256 + lane) * 4;
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) *(floatx4*)(dst + i4 * 256) = o[i4];
        if (dt == 0 && h2 == 0) *(floatx2*)(a.partial_ml + (part * kRows + n32) * 2) = floatx2{ref, l};
      }
    }
  };
  if constexpr (WHOLE) {
    const int row = xcd_order(), tile = row % a.row_tiles, g = row / a.row_tiles % a.hkv, b = row / a.row_tiles / a.hkv;
    if (b >= a.batch) return;
    const Draft d(a, b);
    if (tile >= tree_tiles(a, d.n) || d.len <= 0) return;
    seg(d, b, g, tile, 0, (d.len + 4 * kBlockTokens - 1) / (4 * kBlockTokens), true, 0);
  } else {
    tree_run(a, xcd_order(), seg);
  }
}

// Larger drafts: a worker is a workgroup of W waves that share a ring, 32 query rows each.
template <int D, int KV, int W>
__global__ __launch_bounds__(64 * W, 2) void tree_wide_kernel(const TreeArgs a) {
  constexpr int kDT = D / 32;
  using L_ = TreeLds<D, kv_is_codes(KV), W>;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[L_::kRing];
  const int lane = lane_id(), n32 = lane & 31, h2 = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  tree_run(a, xcd_order(), [&](const Draft& d, int b, int g, int tile, int blk0, int n, bool whole, size_t slot) __attribute__((always_inline)) {
    const int j0 = (tile * W + wave) * kRows, rows_here = min(kRows, d.n * a.group - j0);
    const TreeSums<D> own = tree_blocks_of<D, KV, W>(a, d, b, g, j0, rows_here, blk0, n, 1, n, wave, (unsigned int)(uintptr_t)&lds[0]);
    if (n32 >= rows_here) return;
    const tree_args_p e = tree_args();
    const RowAt at(*e, d, g, j0 + n32);
    const size_t part = slot * W + wave;
    if (whole) {
      // (nothing seen: a row of zeros)
      const float inv = own.sum > 0.f ? 1.f / own.sum : own.sum;
      if (e->lse && h2 == 0) e->lse[at.out] = own.ref + __builtin_amdgcn_logf(own.sum);
      __bf16* dst = (__bf16*)e->out + at.out * D + h2 * 4;
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          bf16x4 pk;
#pragma unroll
          for (int i = 0; i < 4; ++i) pk[i] = (__bf16)(own.acc[dt][i4 * 4 + i] * inv);
          *(bf16x4*)(dst + dt * 32 + i4 * 8) = pk;
        }
    } else {
      float* dst = e->partial_o + part * (kRows * D) + lane * 4;
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4)
          *(floatx4*)(dst + (dt * 4 + i4) * 256) = floatx4{own.acc[dt][i4 * 4], own.acc[dt][i4 * 4 + 1], own.acc[dt][i4 * 4 + 2], own.acc[dt][i4 * 4 + 3]};
      if (h2 == 0) *(floatx2*)(e->partial_ml + (part * kRows + n32) * 2) = floatx2{own.ref, own.sum};
    }
    if (own.undefined)                                       // to the values that this lane has just stored
      add_undefined<D, KV>(d, b, g, at.node, blk0, n, 1, h2, [&](int dim, floatx4 x) {
        if (whole) {
          bf16x4* const o = (bf16x4*)((__bf16*)e->out + at.out * D + dim);
          bf16x4 y = *o;
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = (__bf16)((float)y[i] + x[i]);
          *o = y;
        } else {
          *(floatx4*)(e->partial_o + part * (kRows * D) + (dim / 8 * 64 + lane) * 4) += x;
        }
      });
  });
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
      fold_parts(ref, l, o, (pieces - s0 + step - 1) / step, x, y);
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
    fold_parts(ref, l, o, kWaves - 1, x, y);
  }
  if (ok) store_folded(a, d, g, j0 + n32, D, dt, h2, ref, l, o);
}

template <class F>
hipError_t by_kind(KvKind kv, F&& f) {
  switch (kv) {
    case kKvBf16: return f(std::integral_constant<int, kKvBf16>{});
    case kKvFp8: return f(std::integral_constant<int, kKvFp8>{});
    case kKvFp8Head: return f(std::integral_constant<int, kKvFp8Head>{});
    case kKvInt8Head: return f(std::integral_constant<int, kKvInt8Head>{});
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_tree_mfma(const TreeArgs& a, int head_dim, KvKind kv, hipStream_t s) {
  if (head_dim != 128 && head_dim != 64) return hipErrorInvalidValue;
  if (a.workers == 0) {
    const int64_t rows = (int64_t)a.batch * a.hkv * a.row_tiles;
    const dim3 grid((unsigned)((rows + kXcds - 1) / kXcds * kXcds));
    return by_kind(kv, [&](auto kind) {
      constexpr int KV = decltype(kind)::value;
      if (head_dim == 128) hipLaunchKernelGGL((tree_team_kernel<128, KV, true, false>), grid, dim3(kThreads), 0, s, a);
      else hipLaunchKernelGGL((tree_team_kernel<64, KV, true, false>), grid, dim3(kThreads), 0, s, a);
      return hipGetLastError();
    });
  }
  if (a.batch > kWavePlanBatch) {
    hipLaunchKernelGGL(tree_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t units = (int64_t)a.batch * a.hkv * a.row_tiles * a.tile_parts * (head_dim / 32);
  const bool together = units <= kMergeTogether;
  const dim3 grid((unsigned)a.workers), merge_grid((unsigned)(together ? units : (units + kWaves - 1) / kWaves));
  auto launch_two = [&](auto d, auto kind) {
    constexpr int D = decltype(d)::value, KV = decltype(kind)::value;
    if constexpr (kv_is_codes(KV)) hipLaunchKernelGGL((tree_wide_kernel<D, KV, 2>), grid, dim3(128), 0, s, a);
    else hipLaunchKernelGGL((tree_team_kernel<D, KV, false, true>), grid, dim3(kThreads), 0, s, a);
  };
  auto launch = [&](auto d, auto kind) {
    constexpr int D = decltype(d)::value, KV = decltype(kind)::value;
    if (a.tile_parts == 1) hipLaunchKernelGGL((tree_team_kernel<D, KV, false, false>), grid, dim3(kThreads), 0, s, a);
    else if (a.tile_parts == 2) launch_two(d, kind);
    else if (a.tile_parts == 4) hipLaunchKernelGGL((tree_wide_kernel<D, KV, 4>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((tree_wide_kernel<D, KV, 8>), grid, dim3(512), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (together) hipLaunchKernelGGL((tree_merge_kernel<D, true>), merge_grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((tree_merge_kernel<D, false>), merge_grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
  };
  return by_kind(kv, [&](auto kind) {
    return head_dim == 128 ? launch(std::integral_constant<int, 128>{}, kind) : launch(std::integral_constant<int, 64>{}, kind);
  });
}

}  // namespace rollattn
