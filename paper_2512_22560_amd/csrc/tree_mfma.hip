// Attention of a tree of drafted tokens (bf16 queries) over bf16 or 8-bit (E4M3, int8) paged KV (gfx950).
//
// A row is (trajectory, KV head, tile of 16 C query rows): a query row is a (drafted token, query head of the group) pair, token-major,
// so the heads that share the KV head and the tokens of a draft that fit one tile read K and V once.  C tiles of 16 rows are columns of
// the same products,
//   S^T = K Q^T          (tokens x rows, v_mfma_f32_16x16x32, K rows as A; one LDS read for C products)
//   O^T += V^T P^T       (dims x rows, V read back transposed with ds_read_b64_tr_*; one read for C products)
// and a wave streams its tokens in 32-token blocks through registers and a private LDS tile, as decode's workers do.
// A block that lies in the cached prefix is seen whole by every row and knows no mask.  In the blocks behind it a row sees the tokens
// whose bits are set in its mask words, eight tokens to a lane.  What a row does not see must not reach it: a score is replaced before
// the maximum, and where values of such a block are not finite (zero times infinity would not be zero) they leave the second product,
// and products of ones and zeros tell which rows see them.
// Codes become operands as in decode: see decode_mfma.hip for the range of f16 and the power of two per query row.
#include "stream_tiles.h"

namespace rollattn {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

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

__device__ __forceinline__ bool finite(__bf16 x) { return (__builtin_bit_cast(unsigned short, x) & 0x7f80) != 0x7f80; }
__device__ __forceinline__ bool finite(_Float16 x) { return (__builtin_bit_cast(unsigned short, x) & 0x7c00) != 0x7c00; }

// Whether any element of a word of a pool is no number (infinite and undefined bf16 values, the undefined code of E4M3).
template <int KV>
__device__ __forceinline__ bool undefined(uint32_t w) {
  if constexpr (KV == kKvBf16) return (w & 0x7f800000u) == 0x7f800000u || (w & 0x7f80u) == 0x7f80u;
  else if constexpr (KV == kKvInt8Head) return false;
  else return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
}

// One row from block blk0 on.  BEHIND: only what lies behind the prefix, whose result is there and folded in.
template <int D, int KV, int C, bool STREAM, bool BEHIND>
__device__ __forceinline__ void tree_worker(const TreeArgs& a, int b, int r, int blk0, unsigned char* const k_lds) {
  constexpr bool FP8 = kv_is_codes(KV), HEAD = kv_has_head_scales(KV);   // FP8: 8-bit codes of either kind
  constexpr bool INT8 = KV == kKvInt8Head;
  constexpr int kTile = 16 * C;
  constexpr int kStages = FP8 ? 2 : C == 4 ? 1 : 2;       // blocks in flight
  using kx8 = std::conditional_t<INT8, halfx8, bf16x8>;   // operands of the first product
  using opx8 = std::conditional_t<HEAD, halfx8, bf16x8>;  // ... and of the second
  using op = std::conditional_t<HEAD, _Float16, __bf16>;
  using G_ = Geo<D, FP8>;
  const int lane = lane_id();
  const int r16 = lane & 15;   // MFMA row / column index carried by this lane
  const int q4 = lane >> 4;    // which quarter of the contraction this lane feeds
  unsigned char* const v_lds = k_lds + G_::kTileBytes;

  const int group = a.group, hkv = a.hkv, n_rt = a.row_tiles;
  const int g = r / n_rt, rt = r - g * n_rt;
  const int n_b = a.q_lens[b], len = a.ctx_lens[b], q_off = a.q_offsets[b];
  const int rows_here = min(kTile, n_b * group - rt * kTile);
  if (rows_here <= 0) return;
  const int prefix = len - n_b;
  const int n_blk = (len + kBlockTokens - 1) / kBlockTokens;
  const size_t tile_stride = (size_t)kPageSize * G_::kRowBytes;   // bytes of one (page, head) tile
  const int32_t* const table = a.page_table + (size_t)b * a.max_pages;

  // query row j of this tile: node and head (rows past the last read it again; what becomes of them is not stored)
  auto node_of = [&](int c) { return (rt * kTile + min(c * 16 + r16, rows_here - 1)) / group; };
  auto row_of = [&](int c) {
    const int j = rt * kTile + min(c * 16 + r16, rows_here - 1), node = j / group;
    return (size_t)(q_off + node) * a.hq + (size_t)g * group + (j - node * group);
  };

  // ---- producer: a window of 64 page ids (32 blocks), one per lane
  int pwin = -1, pid_vec = 0, pid_next = 0, next = blk0;
  uint4 kreg[kStages][G_::kLoads];
  uint4 vreg[kStages][G_::kLoads];
  float ksc[kStages], vsc[kStages];   // FP8: page scales of this lane's 8 tokens
  auto load_window = [&](int k) {
    const int pg = k * 64 + lane;
    return (pg < ((len + kPageSize - 1) >> 4)) ? table[pg] : 0;
  };
  auto issue = [&](int stage) {
    const int k = next >> 5;
    if (k != pwin) {
      pid_vec = (pwin >= 0 && k == pwin + 1) ? pid_next : load_window(k);
      pid_next = load_window(k + 1);
      pwin = k;
    }
    const int tok0 = next * kBlockTokens;
    const int p0 = __builtin_amdgcn_readlane(pid_vec, ((next & 31) << 1));
    const int p1 = __builtin_amdgcn_readlane(pid_vec, ((next & 31) << 1) + 1);
    if (FP8) {
      const int pid = (q4 < 2) ? p0 : p1;        // tokens 0-15 of the block sit in its first page
      const int64_t at = HEAD ? (int64_t)pid * hkv + g : (int64_t)pid;
      const bool there = tok0 + q4 * 8 < len;    // (a page that this row does not have: nobody's scale)
      ksc[stage] = there ? a.k_scale[at] : 1.f;
      vsc[stage] = there ? a.v_scale[at] : 1.f;
    }
    const unsigned char* kt0 = (const unsigned char*)a.k_pages + ((size_t)p0 * hkv + g) * tile_stride;
    const unsigned char* kt1 = (const unsigned char*)a.k_pages + ((size_t)p1 * hkv + g) * tile_stride;
    const unsigned char* vt0 = (const unsigned char*)a.v_pages + ((size_t)p0 * hkv + g) * tile_stride;
    const unsigned char* vt1 = (const unsigned char*)a.v_pages + ((size_t)p1 * hkv + g) * tile_stride;
    if (tok0 + kBlockTokens <= len) {
      // whole block live: plain 16-byte loads, 1 KB per wave-wide instruction
#pragma unroll
      for (int j = 0; j < G_::kLoads; ++j) {
        const int row0 = j * G_::kRowsPerLoad;
        const int off = (row0 % kPageSize) * G_::kRowBytes + lane * 16;
        kreg[stage][j] = load16<STREAM>((row0 < kPageSize ? kt0 : kt1) + off);
        vreg[stage][j] = load16<STREAM>((row0 < kPageSize ? vt0 : vt1) + off);
      }
    } else {
      // ragged last block of a row: rows at or past L_b are neither read nor left undefined
#pragma unroll
      for (int j = 0; j < G_::kLoads; ++j) {
        const int row0 = j * G_::kRowsPerLoad;
        const int off = (row0 % kPageSize) * G_::kRowBytes + lane * 16;
        const int row = row0 + lane / G_::kChunks;
        uint4 kv = make_uint4(0, 0, 0, 0), vv = make_uint4(0, 0, 0, 0);
        if (tok0 + row < len) {
          kv = load16<STREAM>((row0 < kPageSize ? kt0 : kt1) + off);
          vv = load16<STREAM>((row0 < kPageSize ? vt0 : vt1) + off);
        }
        kreg[stage][j] = kv;
        vreg[stage][j] = vv;
      }
    }
    ++next;
  };
  auto commit = [&](int stage) {
#pragma unroll
    for (int j = 0; j < G_::kLoads; ++j) {
      const int row = j * G_::kRowsPerLoad + lane / G_::kChunks;
      const int c = lane % G_::kChunks;
      const int kc = (c ^ key_k(row)) & (G_::kChunks - 1);
      const int vc = (c ^ (FP8 ? key_v8(row) : key_v16(row))) & (G_::kChunks - 1);
      *(uint4*)(k_lds + row * G_::kRowBytes + kc * 16) = kreg[stage][j];
      *(uint4*)(v_lds + row * G_::kRowBytes + vc * 16) = vreg[stage][j];
    }
  };

  // whether the values of a block hold any that is no number
  auto any_undefined = [&](int stage) {
    bool any = false;
#pragma unroll
    for (int j = 0; j < G_::kLoads; ++j) any |= undefined<KV>(vreg[stage][j].x) | undefined<KV>(vreg[stage][j].y) | undefined<KV>(vreg[stage][j].z) | undefined<KV>(vreg[stage][j].w);
    return __builtin_amdgcn_ballot_w64(any) != 0;
  };

  // ---- consumer state
  kx8 qop[C][G_::kKK];       // Q^T as the B operand: lane (row r16, quarter q4), 8 dims per step
  float q_unit[C];           // int8: what a unit of this lane's row is worth
  floatx4 acc[C][G_::kDT];   // O^T: lane (row r16, quarter q4) holds dims dt*16 + q4*4 + (0..3)
  float m_run[C], l_run[C];  // running max (log2 units) of this lane's rows, its share of the running sums
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const __bf16* qrow = (const __bf16*)a.q + row_of(c) * D;
#pragma unroll
    for (int kk = 0; kk < G_::kKK; ++kk) {
      // FP8: 16-byte K chunks hold 16 dims; step 2p+e uses bytes e*8.. of chunk p*4+q4
      const bf16x8 v = *(const bf16x8*)(qrow + (FP8 ? ((kk >> 1) * 4 + q4) * 16 + (kk & 1) * 8 : (kk * 4 + q4) * 8));
      qop[c][kk] = __builtin_bit_cast(kx8, v);      // (int8: as it came, until all of the row is there)
    }
    q_unit[c] = a.scale_log2;
    if constexpr (INT8) {
      float top = 0.f;
#pragma unroll
      for (int kk = 0; kk < G_::kKK; ++kk) {
        const bf16x8 v = __builtin_bit_cast(bf16x8, qop[c][kk]);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, __builtin_fabsf((float)v[e]));
      }
      const int up = kQueryBits - __builtin_amdgcn_frexp_expf(xor32_max(xor16_max(top)));
#pragma unroll
      for (int kk = 0; kk < G_::kKK; ++kk) {
        const bf16x8 v = __builtin_bit_cast(bf16x8, qop[c][kk]);
#pragma unroll
        for (int e = 0; e < 8; ++e) qop[c][kk][e] = (_Float16)__builtin_amdgcn_ldexpf((float)v[e], up);
      }
      q_unit[c] = __builtin_amdgcn_ldexpf(a.scale_log2, -up);
    }
#pragma unroll
    for (int dt = 0; dt < G_::kDT; ++dt) acc[c][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    m_run[c] = -INFINITY;
    l_run[c] = 0.f;
  }

  // edge: the block holds tokens behind the prefix; dirty: and values that are no numbers
  auto compute = [&](int blk, bool edge, bool dirty, float kscale, float vscale) __attribute__((always_inline)) {
    const int tok0 = blk * kBlockTokens;
    // ---- S^T = K Q^T for the two 16-row tiles; tile e row r is token (r/4)*8 + e*4 + r%4
    floatx4 s[2][C];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int c = 0; c < C; ++c) s[e][c] = floatx4{0.f, 0.f, 0.f, 0.f};
      const int t = ((r16 >> 2) << 3) + e * 4 + (r16 & 3);
      const unsigned char* rowp = k_lds + t * G_::kRowBytes;
      const int key = key_k(t);
      if constexpr (FP8) {
#pragma unroll
        for (int p = 0; p < G_::kChunks / 4; ++p) {
          const int col = ((p * 4 + q4) ^ key) & (G_::kChunks - 1);
          const uint4 raw = *(const uint4*)(rowp + col * 16);
          const auto lo = widen_k8<KV>(raw.x, raw.y), hi = widen_k8<KV>(raw.z, raw.w);
#pragma unroll
          for (int c = 0; c < C; ++c) s[e][c] = mfma(lo, qop[c][2 * p], s[e][c]);
#pragma unroll
          for (int c = 0; c < C; ++c) s[e][c] = mfma(hi, qop[c][2 * p + 1], s[e][c]);
        }
      } else {
#pragma unroll
        for (int kk = 0; kk < G_::kKK; ++kk) {
          const int col = ((kk * 4 + q4) ^ key) & (G_::kChunks - 1);
          const kx8 kop = *(const kx8*)(rowp + col * 16);
#pragma unroll
          for (int c = 0; c < C; ++c) s[e][c] = mfma(kop, qop[c][kk], s[e][c]);
        }
      }
    }
    // This lane now holds, for its rows, the scores of tokens tok0 + q4*8 + (0..7): s[0][i] -> +i, s[1][i] -> +4+i.
    const int tbase = tok0 + q4 * 8;
    const float vs = FP8 ? vscale : 1.f;
    const float lvs = HEAD ? __builtin_amdgcn_logf(vs) : 0.f, ivs = HEAD ? __builtin_amdgcn_rcpf(vs) : 1.f;
    opx8 pop[C];
    unsigned int seen[C] = {};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const float sc = (INT8 ? q_unit[c] : a.scale_log2) * (FP8 ? kscale : 1.f);
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float raw = (j < 4) ? s[0][c][j] : s[1][c][j - 4];
        x[j] = HEAD ? __builtin_fmaf(raw, sc, lvs) : raw * sc;
      }
      if (edge) {
        seen[c] = seen_bits(a.mask + (size_t)(q_off + node_of(c)) * a.mask_words, a.mask_words, tbase - prefix, n_b, BEHIND ? 0u : 0xffu);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = seen[c] >> j & 1 ? x[j] : -INFINITY;
      }
      float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      mx = xor32_max(xor16_max(mx));
      if constexpr (HEAD) {
        // (of a score past 2^25 the difference may come out larger, more than f16 holds)
        const float below = mx - kWeightBits;
        mx = mx - below > kMostBits ? mx : below;
      }
      const float m_new = fmaxf(m_run[c], mx);
      const float base = m_new == -INFINITY ? 0.f : m_new;   // (a row that has seen nothing yet)
      const float alpha = __builtin_amdgcn_exp2f(m_run[c] - base);
      float psum = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float p = __builtin_amdgcn_exp2f(x[j] - base);
        psum += p;
        pop[c][j] = (op)(FP8 && !HEAD ? p * vs : p);
      }
      l_run[c] = l_run[c] * alpha + (HEAD ? psum * ivs : psum);
      if (__builtin_amdgcn_ballot_w64(m_new > m_run[c])) {
#pragma unroll
        for (int dt = 0; dt < G_::kDT; ++dt) acc[c][dt] *= alpha;
      }
      m_run[c] = m_new;
    }
    // ---- O^T += V^T P^T : A = V^T tile (16 dims x 32 tokens) read transposed from LDS
#pragma unroll
    for (int dt = 0; dt < G_::kDT; ++dt) {
      opx8 vop;
      if constexpr (FP8) {
        typedef __attribute__((address_space(3))) intx2 lds_i2;
        const int t = q4 * 8 + (r16 >> 1);
        const int col = (dt ^ key_v8(t)) & (G_::kChunks - 1);
        const intx2 raw = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2*)(v_lds + t * G_::kRowBytes + col * 16 + (r16 & 1) * 8));
        vop = widen_v8<KV>((uint32_t)raw[0], (uint32_t)raw[1]);
      } else {
        typedef __attribute__((address_space(3))) shortx4 lds_s4;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int t = q4 * 8 + hf * 4 + (r16 >> 2);
          const int col = ((dt * 2 + ((r16 & 3) >> 1)) ^ key_v16(t)) & (G_::kChunks - 1);
          const shortx4 raw = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(v_lds + t * G_::kRowBytes + col * 16 + (r16 & 1) * 8));
          const bf16x4 h4 = __builtin_bit_cast(bf16x4, raw);
          vop[hf * 4 + 0] = h4[0]; vop[hf * 4 + 1] = h4[1]; vop[hf * 4 + 2] = h4[2]; vop[hf * 4 + 3] = h4[3];
        }
      }
      if constexpr (!INT8) {
        if (dirty) {
          // values that are no numbers: out of the product, and to the rows that see them by products of ones and zeros
          opx8 what[3];                                // undefined, infinite, minus infinite
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float v = (float)vop[e];
            what[0][e] = (op)(v != v ? 1.f : 0.f);
            what[1][e] = (op)(v == INFINITY ? 1.f : 0.f);
            what[2][e] = (op)(v == -INFINITY ? 1.f : 0.f);
            vop[e] = finite(vop[e]) ? vop[e] : (op)0.f;
          }
#pragma unroll
          for (int c = 0; c < C; ++c) {
            opx8 ones;
#pragma unroll
            for (int e = 0; e < 8; ++e) ones[e] = (op)(seen[c] >> e & 1 ? 1.f : 0.f);
            floatx4 met[3];
#pragma unroll
            for (int w = 0; w < 3; ++w) met[w] = mfma(what[w], ones, floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float inf = met[1][e] > 0.f ? INFINITY : 0.f, minus = met[2][e] > 0.f ? -INFINITY : 0.f;
              acc[c][dt][e] += inf + minus + (met[0][e] > 0.f ? NAN : 0.f);
            }
          }
        }
      }
#pragma unroll
      for (int c = 0; c < C; ++c) acc[c][dt] = mfma(vop, pop[c], acc[c][dt]);
    }
  };

  // ---- software pipeline over the blocks
  const int n_mine = n_blk - blk0;
#pragma unroll
  for (int st = 0; st < kStages; ++st) {
    if (st < n_mine) issue(st);
  }
  for (int i0 = 0; i0 < n_mine; i0 += kStages) {
#pragma unroll
    for (int st = 0; st < kStages; ++st) {
      const int i = i0 + st;
      if (i < n_mine) {
        const bool edge = (blk0 + i + 1) * kBlockTokens > prefix;
        const bool dirty = !INT8 && edge && any_undefined(st);
        commit(st);
        const float kscale = FP8 ? ksc[st] : 1.f, vscale = FP8 ? vsc[st] : 1.f;
        if (i + kStages < n_mine) issue(st);   // the registers just drained take the next block
        compute(blk0 + i, edge, dirty, kscale, vscale);
      }
    }
  }
  // ---- normalise and store
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const float l_tot = xor32_add(xor16_add(l_run[c]));
    const bool ok = c * 16 + r16 < rows_here;
    const size_t orow = row_of(c);
    const float inv = l_tot > 0.f ? 1.f / l_tot : l_tot;   // (nothing seen: a row of zeros)
    if (a.lse && ok && q4 == 0) a.lse[orow] = m_run[c] + __builtin_amdgcn_logf(l_tot);
    __bf16* dst = (__bf16*)a.out + orow * D + q4 * 4;
    if (ok) {
#pragma unroll
      for (int dt = 0; dt < G_::kDT; ++dt) {
        bf16x4 pk;
#pragma unroll
        for (int e = 0; e < 4; ++e) pk[e] = (__bf16)(acc[c][dt][e] * inv);
        *(bf16x4*)(dst + dt * 16) = pk;
      }
    }
  }
}

template <int D, int KV, int C>
__global__ __launch_bounds__(kThreads, 1) void tree_mfma_kernel(const TreeArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[kWaves][2 * Geo<D, kv_is_codes(KV)>::kTileBytes];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x * kWaves + wave, rows_per_b = a.hkv * a.row_tiles, b = row / rows_per_b;
  if (b >= a.batch) return;
  tree_worker<D, KV, C, false, false>(a, b, row - b * rows_per_b, 0, lds[wave]);
}

}  // namespace

hipError_t launch_tree_mfma(const TreeArgs& args, int head_dim, KvKind kv, int32_t max_q_len, hipStream_t s) {
  TreeArgs a = args;
  const int64_t rows = (int64_t)max_q_len * a.group;
  const int tiles = rows <= 16 ? 1 : 2;
  a.row_tiles = (int32_t)((rows + 16 * tiles - 1) / (16 * tiles));
  const int64_t waves = (int64_t)a.batch * a.hkv * a.row_tiles;
  if (waves > INT32_MAX / 64) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((waves + kWaves - 1) / kWaves));
  auto launch = [&](auto d, auto kind, auto c) {
    hipLaunchKernelGGL((tree_mfma_kernel<decltype(d)::value, decltype(kind)::value, decltype(c)::value>), grid, dim3(kThreads), 0, s, a);
  };
  auto of_tiles = [&](auto d, auto kind) {
    if (tiles == 1) launch(d, kind, std::integral_constant<int, 1>{});
    else launch(d, kind, std::integral_constant<int, 2>{});
  };
  auto of_kind = [&](auto kind) {
    if (head_dim == 128) of_tiles(std::integral_constant<int, 128>{}, kind);
    else of_tiles(std::integral_constant<int, 64>{}, kind);
  };
  if (head_dim != 128 && head_dim != 64) return hipErrorInvalidValue;
  switch (kv) {
    case kKvBf16: of_kind(std::integral_constant<int, kKvBf16>{}); break;
    case kKvFp8: of_kind(std::integral_constant<int, kKvFp8>{}); break;
    case kKvFp8Head: of_kind(std::integral_constant<int, kKvFp8Head>{}); break;
    case kKvInt8Head: of_kind(std::integral_constant<int, kKvInt8Head>{}); break;
  }
  return hipGetLastError();
}

}  // namespace rollattn
