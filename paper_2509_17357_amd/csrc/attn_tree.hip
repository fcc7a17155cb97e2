// Attention of drafted tokens over a paged cache, lengths on the device.  Row i of sequence s (one of its n drafted tokens, K/V at
// position L + i) attends to the L cached keys and to the drafted ones that bit j of its mask names:
//     out_i = sum_j w_ij V_j / sum_j w_ij,  w_ij = exp(scale <q_i, K_j> - m_i),  j < L or (j = L + k, k < n, bit k of mask_i).
//
// The host does not know the lengths, so a launch has as many work-groups as the GPU has CUs, and each finds its share itself: the
// batch is a sequence of U units (a row tile of a KV head against unit_keys keys; keys run fastest, then row tiles, heads, sequences),
// and share l of A = min(work-groups, U) is units [l U / A, (l + 1) U / A), at least one.  Neighbouring shares, whose row tiles read the same
// keys, go to one XCD (and a cut close to the end of an item moves there).  A row tile whose units lie in several shares is left as partial results (m, l, O), which
// merge_kernel combines; a share has at most two of them, one at either end, so the workspace does not depend on the lengths.
//
// S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x16_bf16: a row (a drafted token and a query head of the KV head) is a column, its
// lanes are l and l + 32, and P stays in registers.  Two kernels of 8 wavefronts:
//   stream_kernel - row tiles of 32, bound by memory: every wavefront has all 32 rows and takes every eighth sub-tile of 32 keys, which it
//                   moves to LDS of its own, by DMA: loads in flight take no registers, and no wave waits for another.  The eight results are
//                   joined in LDS.
//   tiles_kernel  - row tiles of 128 or 256, bound by what a CU issues: a wavefront has 32 of the rows.  Tiles of kTileKeys keys go through registers
//                   (fp8 codes are converted there, once) to one of two LDS buffers, where all waves read their operands.
// What the second one is at: 16 trees of 48 .. 61 tokens, 8 heads a KV head, fp8, behind 8000 .. 32000 keys take 690 .. 710 us, 0.81 .. 0.83 PFLOP/s; the
// matrix pipes are busy for 40 % of it, a wave issues for 34 %, waits for its turn to for 25 % and for LDS, memory or the barrier for 41 %, LDS
// moves for 26 %.  Tried, within 2 % of it or slower: V and the next K read a step ahead; scores of the next sub-tile between the numerators of this
// one; the two waves of a SIMD half a step apart; s_setprio around the products; bf16 tiles by DMA in a ring of four (204 -> 225 us, 32 trees of 64).
#include <hip/hip_runtime.h>
#include <algorithm>

#include "cronus_internal.h"
#include "lane_ops.h"

namespace cronus {
namespace {

// Rows of a tile.  A batch of at most kFewRowTiles tiles of 32 rows is streamed, however many rows a sequence has: the tiles of a sequence read
// the same K/V at the same time on one XCD, and there are CUs for them all.  us a pass, 32 / 128 rows: 100 rows (fp8, 3 sequences of about 700) 14.5 / 26.3,
// 126 rows (7 of 119 .. 1278) 15.8 / 28.0, 252 (one of 5000) 23.4 / 34.0; beyond it, 132 rows (fp8, 13 of 56 .. 3028) 65.7 / 45.6, 301 (9 of 106 .. 10230)
// 65.5 / 52.5, 116 (21 of 104 .. 389) 34.6 / 27.3.  256 rows read K/V half as often but have half the work-groups: from 192 rows and kManyRowTiles on.  128 / 256 rows: 256
// rows (32 of 1000 .. 8000) 254 / 205, 488 (fp8, 16 of 8000 .. 32000) 864 / 723; 301 as above 52.5 / 58.5, 184 (50 of 82 .. 2258, D = 64) 29.8 / 31.5.
constexpr long long kFewRowTiles = 352, kManyRowTiles = 1536;
// A cut between two shares that is one unit from an end of an item moves there: a piece costs a work-group about 5 us before its first
// product and behind its last one, and a row tile cut in two is written and read once more.  us a pass with 0 / 1 / 2 units: a sequence of 3300
// keys and 21 tokens, 7 heads a KV head, 24.2 / 21.7 / 22.2; fp8, 13 of 56 .. 3028 and 4 .. 33 46.3 / 41.2 / 41.0; 9 of 106 .. 10230 66.8 / 60.6 / 60.5; 25 chains
// of 500 .. 4097 35.5 / 36.0 / 39.2 (and with 3, 32 trees of 64 213 instead of 204).
constexpr int kSnapUnits = 1;
// Where the tables have room for so many steps of a work-group at most (1792 keys streamed, 896 in tiles), a unit holds all keys of a
// sequence: no row tile is split, so there is no merge launch, and every work-group has whole items.  us a pass, cut / whole: a tree of 8 behind
// 256 keys 12.5 / 9.5; 31 single tokens behind 40 .. 346 19.2 / 11.6; 11 trees of 5 .. 28, fp8, behind 17 .. 700 19.8 / 13.1; 166 single tokens behind
// 52 .. 1162 106.6 / 94.9.  With 12 steps 8 trees of 12 .. 32 behind 200 .. 3000 take 27.9 instead of 30.2, but 146 single tokens behind
// 398 .. 3011, 7 heads a KV head, 112.7 instead of 90.2.
constexpr int kWholeSteps = 7;
constexpr int kNonTemporal = 2;  // cache policy operand of a transfer: the instruction's nt bit
// Of a tile in LDS (tiles_kernel).  us a pass, 64 / 128: 16 trees of 48 .. 61, fp8, 742 / 714; a whole iteration with 24 trees 96 / 92; two K
// and V buffers of 256 keys do not fit.
constexpr int kTileKeys = 128;
// Units times work-groups stay below this, for any lengths that the tables have room for: shares are computed in 32 bits, where a 64-bit
// division is 140 instructions.
constexpr long long kMostUnitShares = 1LL << 31;

struct TreeParams {
  const unsigned short* q;
  unsigned short* out;
  const unsigned char* k_pool;
  const unsigned char* v_pool;
  const float* k_scale;
  const float* v_scale;
  const int* prefix_lens;
  const int* cu_rows;
  const unsigned long long* mask;  // or nullptr: a chain
  const int* block_tables;
  float* partials;        // two slots a work-group
  struct Split* splits;   // one a work-group
  int mask_words, max_blocks, n_seqs, max_rows, n_q_heads, n_kv_heads;
  int unit_keys;  // a multiple of what a work-group takes in one step
  bool whole;     // a unit holds all keys of any sequence
  float scale_log2e;
};

// A row tile whose units lie in the shares of several work-groups, left by the one that has its first unit: the pieces are that one's
// slot 1 and slot 0 of the next n_pieces - 1.
struct Split {
  int n_pieces;  // 0: none
  int share;     // that work-group's share
  int n_rows;    // rows of the tile
  int row0;      // first of them among the sequence's rows of this KV head
  int kv_head;
  int first_token;  // cu_rows of the sequence
  int prefix, count;
};
static_assert(sizeof(Split) == 32);

// Floats of a slot: O, then (m in log2 units, l) of every row.
template <int D, int ROWS> constexpr int kSlotFloats = ROWS * (D + 2);

// The sequence's lengths, or no rows where they are none that this call could serve.
struct Lens {
  int prefix, count, first;
};
__device__ __forceinline__ Lens lens_of(const TreeParams& p, int s) {
  const int first = p.cu_rows[s], next = p.cu_rows[s + 1], prefix = p.prefix_lens[s];
  const long long count = (long long)next - first;
  const bool good = first >= 0 && count > 0 && count <= p.max_rows && prefix >= 0 &&
                    prefix + count <= min((long long)p.max_blocks * kBlock, kTreeMostKeys);
  return good ? Lens{prefix, (int)count, first} : Lens{0, 0, 0};
}
template <int ROWS>
__device__ __forceinline__ int row_tiles(const TreeParams& p, const Lens& n) {
  return (n.count * (p.n_q_heads / p.n_kv_heads) + ROWS - 1) / ROWS;
}
__device__ __forceinline__ int key_units(const TreeParams& p, const Lens& n) {
  const unsigned unit = p.unit_keys;
  return (int)(((unsigned)n.prefix + (unsigned)n.count + unit - 1) / unit);
}
template <int ROWS>
__device__ __forceinline__ int units_of(const TreeParams& p, const Lens& n) {
  return n.count ? row_tiles<ROWS>(p, n) * key_units(p, n) * p.n_kv_heads : 0;
}

// 32 bits: which of the keys first_key .. first_key + 31 the row of drafted token `token` sees.
__device__ __forceinline__ unsigned visible_bits(const TreeParams& p, const Lens& n, int token, int first_key) {
  const int at = first_key - n.prefix;  // of the first key, among the drafted tokens
  if (at >= n.count) return 0;
  if (at <= -32) return ~0u;
  unsigned bits;
  if (!p.mask) {
    const int seen = token + 1 - at;  // keys of the 32 before the first that it does not see
    bits = seen >= 32 ? ~0u : seen > 0 ? (1u << seen) - 1 : 0;
  } else {
    const unsigned long long* row = p.mask + (long long)(n.first + token) * p.mask_words;
    if (at < 0) {
      bits = (unsigned)(row[0] << -at) | ((1u << -at) - 1);
    } else {
      const int w = at >> 6, shift = at & 63;
      unsigned long long x = row[w] >> shift;
      if (shift > 32 && w + 1 < p.mask_words) x |= row[w + 1] << (64 - shift);
      bits = (unsigned)x;
    }
  }
  const int left = n.count - at;
  return left >= 32 ? bits : bits & ((1u << left) - 1);
}
// Whether the row sees nothing: its output is 0 then (and not the quotient of two zeros).
__device__ bool sees_nothing(const TreeParams& p, const Lens& n, int token) {
  if (n.prefix > 0) return false;
  for (int at = 0; at < n.count; at += 32)
    if (visible_bits(p, n, token, at)) return false;
  return true;
}

__device__ __forceinline__ bool not_finite(u32x4 v) {
  bool found = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) found |= (v[w] & 0x7f80u) == 0x7f80u || (v[w] & 0x7f800000u) == 0x7f800000u;
  return found;
}

// The chunk with 0 in the place of infinities and NaN.
__device__ __forceinline__ u32x4 finite_only(u32x4 v) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if ((v[w] & 0x7f80u) == 0x7f80u) v[w] &= 0xffff0000u;
    if ((v[w] & 0x7f800000u) == 0x7f800000u) v[w] &= 0x0000ffffu;
  }
  return v;
}

// A work-group's share of the batch, and the sequence that it begins in.
struct Share {
  int begin, end, total, seq_base;  // units; seq_base: those before sequence seq
  int index, active, seq;
  Lens n;  // of that sequence
};
struct ShareLds {
  int sums[kWaves], base[2], seq[2];
  Lens n[2];
};
__device__ __forceinline__ int cut(int index, int total, int active) { return (int)((unsigned)index * (unsigned)total / (unsigned)active); }
// A cut at `at` in an item of `units` units from `first` on, moved to an end of the item that is near.
__device__ __forceinline__ int snap(int at, int first, int units) {
  return at - first <= kSnapUnits ? first : first + units - at <= kSnapUnits ? first + units : at;
}

// Thread t sums the units of sequences [t per, (t + 1) per).  The share is empty (begin >= end) where there is nothing to do.
template <int ROWS>
__device__ __forceinline__ Share find_share(const TreeParams& p, ShareLds& lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (p.n_seqs + kThreads - 1) / kThreads;
  const int s_lo = min(tid * per, p.n_seqs), s_hi = min(s_lo + per, p.n_seqs);
  int mine = 0;
  Lens n{};
  for (int s = s_lo; s < s_hi; ++s) {
    n = lens_of(p, s);
    mine += units_of<ROWS>(p, n);
  }
  int incl = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl(incl, lane - d < 0 ? lane : lane - d);
    if (lane >= d) incl += y;
  }
  if (lane == 63) lds.sums[wave] = incl;
  __syncthreads();
  Share r{};
  int base = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) base = r.total;
    r.total += lds.sums[w];
  }
  r.total = __builtin_amdgcn_readfirstlane(r.total);
  base += incl - mine;
  r.active = min((int)gridDim.x, r.total);
  r.index = blockIdx.x;
  bool idle = r.index >= r.active;
  if (gridDim.x % kQueues == 0) {
    const int xcd = r.index % kQueues;
    r.index = xcd * r.active / kQueues + r.index / kQueues;
    idle = r.index >= (xcd + 1) * r.active / kQueues;
  }
  if (idle) return r;
  const int at[2] = {cut(r.index, r.total, r.active), cut(r.index + 1, r.total, r.active)};
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if (base <= at[e] && at[e] < base + mine) {  // one thread, or none (the end of the batch)
      int s = s_lo, before = base;
      for (; per > 1; ++s) {
        n = lens_of(p, s);
        const int u = units_of<ROWS>(p, n);
        if (at[e] < before + u) break;
        before += u;
      }
      lds.seq[e] = s;
      lds.base[e] = before;
      lds.n[e] = n;
    }
  }
  __syncthreads();
  r.seq = __builtin_amdgcn_readfirstlane(lds.seq[0]);
  r.seq_base = __builtin_amdgcn_readfirstlane(lds.base[0]);
  r.n = Lens{__builtin_amdgcn_readfirstlane(lds.n[0].prefix), __builtin_amdgcn_readfirstlane(lds.n[0].count), __builtin_amdgcn_readfirstlane(lds.n[0].first)};
  auto snapped = [&](int x, int seq_base, int units) { return snap(x, x - (int)((unsigned)(x - seq_base) % (unsigned)units), units); };
  r.begin = snapped(at[0], r.seq_base, key_units(p, r.n));
  r.end = at[1];
  if (at[1] < r.total) {
    const Lens m{__builtin_amdgcn_readfirstlane(lds.n[1].prefix), __builtin_amdgcn_readfirstlane(lds.n[1].count), 0};
    r.end = snapped(at[1], __builtin_amdgcn_readfirstlane(lds.base[1]), key_units(p, m));
  }
  return r;
}

// The units of one row tile in a share.
struct Piece {
  Lens n;
  int seq, kv_head, unit, key_begin, key_end, kv_len, row0, n_rows;
  int item_end;
  bool whole;  // all units of the row tile
};
struct Walk {
  Share sh;
  int seq_base, at, seq;
  Lens n;
};
__device__ __forceinline__ Walk begin_walk(const Share& sh) { return Walk{sh, sh.seq_base, sh.begin, sh.seq, sh.n}; }
template <int ROWS>
__device__ __forceinline__ bool next_piece(const TreeParams& p, Walk& w, Piece& it) {
  if (w.at >= w.sh.end) return false;
  while (w.n.count == 0 || w.at >= w.seq_base + units_of<ROWS>(p, w.n)) {  // the share has another unit, so there is another sequence
    w.seq_base += units_of<ROWS>(p, w.n);
    w.n = lens_of(p, ++w.seq);
  }
  const unsigned n_key_units = key_units(p, w.n), n_tiles = row_tiles<ROWS>(p, w.n), rel = w.at - w.seq_base, tile_index = rel / n_key_units;
  it.n = w.n;
  it.seq = w.seq;
  it.unit = rel - tile_index * n_key_units;
  it.kv_head = tile_index / n_tiles;
  it.row0 = (tile_index - it.kv_head * n_tiles) * ROWS;
  it.n_rows = min(ROWS, w.n.count * (p.n_q_heads / p.n_kv_heads) - it.row0);
  it.item_end = w.at - it.unit + (int)n_key_units;
  const int end = min(it.item_end, w.sh.end);
  it.kv_len = w.n.prefix + w.n.count;
  it.key_begin = it.unit * p.unit_keys;
  it.key_end = end == it.item_end ? it.kv_len : (it.unit + end - w.at) * p.unit_keys;
  it.whole = it.unit == 0 && end == it.item_end;
  w.at = end;
  return true;
}
// The tile's first piece leaves word of the others.
__device__ __forceinline__ void note_split(const TreeParams& p, const Share& sh, const Piece& it) {
  if (it.unit != 0 || it.whole || threadIdx.x != 0) return;
  int last = sh.index + 1;
  while (cut(last + 1, sh.total, sh.active) + kSnapUnits < it.item_end) ++last;
  p.splits[blockIdx.x] = Split{last - sh.index + 1, sh.index, it.n_rows, it.row0, it.kv_head, it.n.first, it.n.prefix, it.n.count};
}

// 8 dims of row r of the tile, final or partial.
template <int D>
__device__ __forceinline__ void store_final(const TreeParams& p, const Piece& it, int r, int d, const float (&x)[8], float sum, float v_factor) {
  const int group = p.n_q_heads / p.n_kv_heads, tok = (it.row0 + r) / group, h = it.kv_head * group + (it.row0 + r) - tok * group;
  const float f = v_factor / sum;
  u32x4 w;
  if (sum == 0.f && sees_nothing(p, it.n, tok)) {
    w = u32x4{0, 0, 0, 0};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pack_bf16(x[2 * e] * f, x[2 * e + 1] * f);
  }
  *reinterpret_cast<u32x4*>(p.out + ((long long)(it.n.first + tok) * p.n_q_heads + h) * D + d) = w;
}
template <int D>
__device__ __forceinline__ void store_partial(float* part, int r, int d, const float (&x)[8]) {
  float* to = part + r * D + d;
  *reinterpret_cast<f32x4*>(to) = f32x4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<f32x4*>(to + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// What a wave keeps of 32 rows: a lane has one of them, and every second 8 of its dims.
template <int D>
struct Rows {
  f32x16 o[D / 32];
  bf16x8 q[D / 16];
  float m, l;
  int token;
  __device__ __forceinline__ void clear() {
    m = kNeg;
    l = 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  }
  __device__ __forceinline__ void rescale(float m_new, float c) {
    const float alpha = __builtin_amdgcn_exp2f((m - m_new) * c);
    l *= alpha;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
    m = m_new;
  }
};

__device__ __forceinline__ float lane_max(const f32x16& sc) {
  float mx = sc[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
  return mx;
}
// Keys that the row does not see.
__device__ __forceinline__ void hide_scores(f32x16& sc, unsigned seen, int half) {
  const unsigned own = seen >> (8 * half);
#pragma unroll
  for (int i = 0; i < 16; ++i) sc[i] = own >> (16 * (i >> 3) + (i & 7)) & 1 ? sc[i] : -__builtin_inff();
}
// The V operands of a sub-tile with drafted tokens: 0 in the slots behind the last of them; true if there are infinite or NaN
// values, in whose place is 0 then.
template <int D>
__device__ __forceinline__ bool tidy_values(u32x4 (&vop)[D / 16], int key, int kv_len, int half) {
  constexpr int NSTEP = D / 16, NDB = D / 32;
  if (key + 32 > kv_len) {
#pragma unroll
    for (int x = 0; x < NSTEP; ++x) vop[x] = zero_tail(vop[x], key + 16 * (x / NDB) + 8 * half, kv_len);
  }
  bool mine = false;
#pragma unroll
  for (int x = 0; x < NSTEP; ++x) mine |= not_finite(vop[x]);
  const bool odd = __builtin_amdgcn_ballot_w64(mine) != 0;
  if (odd) {
#pragma unroll
    for (int x = 0; x < NSTEP; ++x) vop[x] = finite_only(vop[x]);
  }
  return odd;
}
// Infinite and NaN values are added to the rows that see their key, one after the other: in the product, 0 times such a value would be
// NaN in the others.
template <int D, bool FP8>
__device__ __forceinline__ void add_odd_values(const TreeParams& p, const Piece& it, Rows<D>& rows, const u32x4 (&pp)[2], int key, int half, int c32) {
  constexpr int ESZ = FP8 ? 1 : 2;
  const int* table = p.block_tables + (long long)it.seq * p.max_blocks;
  const unsigned seen = visible_bits(p, it.n, rows.token, key);
#pragma unroll 1
  for (int b = 0; b < 32 && key + b < it.kv_len; ++b) {
    const int x = (b >> 4) * 4 + ((b & 7) >> 1);
    unsigned word = 0;
#pragma unroll
    for (int y = 0; y < 8; ++y) word = x == y ? pp[y >> 2][y & 3] : word;
    word = __shfl(word, c32 + 32 * (b >> 3 & 1));
    const float weight = __uint_as_float(b & 1 ? word & 0xffff0000u : word << 16);
    const int pos = key + b;
    const unsigned char* g = p.v_pool + ((long long)table[pos / kBlock] * p.n_kv_heads + it.kv_head) * (16 * D * ESZ) +
                             (pos % kBlock / 8 * D * 8 + pos % 8) * ESZ;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int d = 32 * db + 16 * (i >> 3) + 8 * half + (i & 7);
        float value;
        if constexpr (FP8) value = __builtin_amdgcn_cvt_f32_fp8((int)g[d * 8], 0);
        else value = __uint_as_float((unsigned)reinterpret_cast<const unsigned short*>(g)[d * 8] << 16);
        const bool add = (seen >> b & 1) && (__float_as_uint(value) & 0x7f800000u) == 0x7f800000u;
        rows.o[db][i] = add ? __builtin_fmaf(weight, value, rows.o[db][i]) : rows.o[db][i];
        asm volatile("" : "+v"(rows.o[db][i]) : : "memory");  // one at a time: no registers for a path that is hardly ever taken
      }
  }
}

// The factor of the scores, in log2 units, and what q is multiplied with (its sign bits): the running maximum is that of the
// scores, so a negative factor goes into q.  Not 0: 0 times the -infinity of a key that is not seen is no weight.
template <bool FP8>
__device__ __forceinline__ float score_factor(const TreeParams& p, int kv_head, unsigned& flip) {
  float c = p.scale_log2e * (FP8 ? p.k_scale[kv_head] : 1.0f);
  flip = c < 0 ? 0x80008000u : 0u;
  c = fabsf(c);
  return c < 1e-37f ? 1e-37f : c;
}

// Results of waves that share rows, in LDS: group x of 4 dims of row r lies at x ^ (r & mask), so that the lanes of a store and
// of a load hit all banks.
template <int D>
__device__ __forceinline__ float* result_at(unsigned char* base, int r, int x) {
  return reinterpret_cast<float*>(base) + r * D + (x ^ (r & (D / 4 - 1))) * 4;
}
template <int D>
__device__ __forceinline__ void put_result(unsigned char* base, int r, const f32x16 (&o)[D / 32], int half) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int h = 0; h < 4; ++h)
      *reinterpret_cast<f32x4*>(result_at<D>(base, r, 8 * db + 4 * (h >> 1) + 2 * half + (h & 1))) =
          f32x4{o[db][4 * h], o[db][4 * h + 1], o[db][4 * h + 2], o[db][4 * h + 3]};
}
// Joins the results of WK waves for 8 dims of a row and stores them.  ml: (m in log2 units, l) of every wave's rows; base: wave 0's results, `pitch`
// bytes before those of the next.
template <int D, int ROWS, int WK, int WAVE_ROWS>
__device__ __forceinline__ void join_and_store(const TreeParams& p, const Piece& it, unsigned char* base, int pitch, const float (*ml)[WAVE_ROWS][2], int x,
                                               float* part, float v_factor) {
  const int r = x / (D / 8), d = x % (D / 8) * 8, w0 = r / WAVE_ROWS * WK, rr = r % WAVE_ROWS;
  float top = ml[w0][rr][0], sum = 0.f;
#pragma unroll
  for (int w = 1; w < WK; ++w) top = fmaxf(top, ml[w0 + w][rr][0]);
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < WK; ++w) {
    const float f = __builtin_amdgcn_exp2f(ml[w0 + w][rr][0] - top);
    sum = __builtin_fmaf(f, ml[w0 + w][rr][1], sum);
    const f32x4 a = *reinterpret_cast<const f32x4*>(result_at<D>(base + (w0 + w) * pitch, rr, d / 4));
    const f32x4 b = *reinterpret_cast<const f32x4*>(result_at<D>(base + (w0 + w) * pitch, rr, d / 4 + 1));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      acc[e] = __builtin_fmaf(f, a[e], acc[e]);
      acc[4 + e] = __builtin_fmaf(f, b[e], acc[4 + e]);
    }
  }
  if (it.whole) {
    store_final<D>(p, it, r, d, acc, sum, v_factor);
  } else {
    store_partial<D>(part, r, d, acc);
    if (d == 0) {
      part[ROWS * D + 2 * r] = top;
      part[ROWS * D + 2 * r + 1] = sum;
    }
  }
}

// ------------------------------------------------------------------------------------------------------------ few rows
template <int D, bool FP8>
__global__ __launch_bounds__(kThreads, 2) void stream_kernel(TreeParams p) {
  constexpr int NSTEP = D / 16, NDB = D / 32, ESZ = FP8 ? 1 : 2, WK = kWaves, ROWS = 32;
  constexpr int BLKB = 16 * D * ESZ;                            // bytes of one (block, head) of the cache
  constexpr int WAVE_LDS = 2 * NSTEP * 1024 + (FP8 ? 512 : 0);  // a wave's K and V planes, or two sets of block images (fp8)
  static_assert(WAVE_LDS >= 32 * D * 4, "a wave's result takes the place of its planes");
  __shared__ __align__(1024) unsigned char smem[kWaves * WAVE_LDS];
  __shared__ float ml_lds[kWaves][32][2];
  __shared__ ShareLds share_lds;

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, c32 = lane & 31, pr = perm32(c32);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = p.n_q_heads / p.n_kv_heads;
  const Share sh = find_share<ROWS>(p, share_lds);
  if (tid == 0) p.splits[blockIdx.x].n_pieces = 0;
  if (sh.begin >= sh.end) return;
  const bool big = (long long)sh.total * p.unit_keys * (2 * D * ESZ) >= kPastCacheBytes;
  Walk walk = begin_walk(sh);
  Piece it;
  while (next_piece<ROWS>(p, walk, it)) {
    Rows<D> rows;
    rows.clear();
    const int row = min(it.row0 + c32, it.n.count * group - 1);
    rows.token = row / group;
    unsigned flip;
    const float c = score_factor<FP8>(p, it.kv_head, flip);
    const unsigned short* qp = p.q + ((long long)(it.n.first + rows.token) * p.n_q_heads + it.kv_head * group + row - rows.token * group) * D + 8 * half;
    u32x4 qraw[NSTEP];
    auto pin_q = [&]() {  // waits for q here
#pragma unroll
      for (int st = 0; st < NSTEP; ++st) {
        asm volatile("" : "+v"(qraw[st]));
        rows.q[st] = as_bf16x8(qraw[st] ^ flip);
      }
    };

    auto scores = [&](const u32x4 (&kop)[NSTEP], f32x16& sc) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
      for (int st = 0; st < NSTEP; ++st) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kop[st]), rows.q[st], sc, 0, 0, 0);
    };
    auto weights = [&](f32x16& sc, int key, u32x4 (&pp)[2]) {
      if (key + 32 > it.n.prefix) hide_scores(sc, visible_bits(p, it.n, rows.token, key), half);
      const float mx = pair_max(lane_max(sc));
      // m only has to bound the scores loosely: numerators of up to 2^kLazyLog2 are as exact in bf16 as those below 1
      if (__builtin_amdgcn_ballot_w64((mx - rows.m) * c > kLazyLog2) != 0) rows.rescale(fmaxf(rows.m, mx), c);
      rows.l += softmax_exp_part(sc, c, rows.m, pp);
    };
    auto sums = [&](u32x4 (&vop)[NSTEP], const u32x4 (&pp)[2], int key) {
      bool odd = false;
      if (key + 32 > it.n.prefix) odd = tidy_values<D>(vop, key, it.kv_len, half);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int db = 0; db < NDB; ++db)
          rows.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vop[t * NDB + db]), as_bf16x8(pp[t]), rows.o[db], 0, 0, 0);
      if (odd) add_odd_values<D, FP8>(p, it, rows, pp, key, half, c32);
    };

    // Sub-tiles wave, wave + 8, ... of the piece; table entries of the next 32 of them in one register, two lanes each.
    const int* table = p.block_tables + (long long)it.seq * p.max_blocks;
    const int last_block = (it.kv_len - 1) / kBlock;
    int bt_reg = 0;
    auto load_table = [&](int j0) {
      const int u = wave + WK * (j0 + (lane >> 1));
      bt_reg = table[min(it.key_begin / kBlock + 2 * u + (lane & 1), last_block)];  // counted in blocks: keys so far past the end pass 32 bits
    };
    auto pin_table = [&]() { asm volatile("" : "+v"(bt_reg)); };
    const int n_sub = (it.key_end - it.key_begin + 31) / 32;
    const int n_iter = n_sub > wave ? (n_sub - wave + WK - 1) / WK : 0;
    lds_byte* wl = (lds_byte*)smem + wave * WAVE_LDS;
    const unsigned wl_addr = (unsigned)(unsigned long long)wl;
    // K/V that one item reads, and much of it in the batch, keeps out of the caches (kPastCacheBytes): 64 single tokens behind 256 .. 8000 keys
    // 221 us a pass, 197 past the caches.
    const bool past_cache = it.n_rows == it.n.count * group && big;
    auto stream = [&](auto run) -> void {
      if (past_cache) run(std::integral_constant<int, kNonTemporal>{});
      else run(std::integral_constant<int, 0>{});
    };
    load_table(0);
#pragma unroll
    for (int st = 0; st < NSTEP; ++st) qraw[st] = *reinterpret_cast<const u32x4*>(qp + 16 * st);
    pin_table();
    if constexpr (!FP8) {
      const unsigned rd = wl_addr + lane * 16;  // each lane reads back the chunks that it fetched
      const int k_off = (half * 16 + (pr & 15)) * 16, v_off = (half * D + pr) * 16;
      auto issue_k = [&](auto nt, int j) -> void {
        const long long b0 = __builtin_amdgcn_readlane(bt_reg, 2 * (j & 31)), b1 = __builtin_amdgcn_readlane(bt_reg, 2 * (j & 31) + 1);
        const unsigned char* g = p.k_pool + (((pr >> 4) ? b1 : b0) * p.n_kv_heads + it.kv_head) * BLKB + k_off;
#pragma unroll
        for (int st = 0; st < NSTEP; ++st) __builtin_amdgcn_global_load_lds(g + st * 512, wl + st * 1024, 16, 0, decltype(nt)::value);
      };
      auto issue_v = [&](auto nt, int j) -> void {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const long long b = __builtin_amdgcn_readlane(bt_reg, 2 * (j & 31) + t);
          const unsigned char* g = p.v_pool + (b * p.n_kv_heads + it.kv_head) * BLKB + v_off;
#pragma unroll
          for (int db = 0; db < NDB; ++db) __builtin_amdgcn_global_load_lds(g + db * 512, wl + (NSTEP + t * NDB + db) * 1024, 16, 0, decltype(nt)::value);
        }
      };
      stream([&](auto nt) -> void {
        if (n_iter > 0) {
          issue_k(nt, 0);
          issue_v(nt, 0);
        }
        pin_q();
        for (int j = 0; j < n_iter; ++j) {
          const int key = it.key_begin + 32 * (wave + WK * j);
          const bool more = j + 1 < n_iter;
          u32x4 kop[NSTEP], vop[NSTEP], pp[2];
          f32x16 sc;
          wait_vmcnt<NSTEP>();  // K(j) has landed; the V(j) loads behind it may still fly
          lds_read_planes<NSTEP>(kop, rd);
          scores(kop, sc);
          if (more) {
            if (((j + 1) & 31) == 0) {
              load_table(j + 1);
              pin_table();
            }
            issue_k(nt, j + 1);
          }
          weights(sc, key, pp);
          if (more) wait_vmcnt<NSTEP>();
          else wait_vmcnt<0>();  // V(j) has landed
          lds_read_planes<NSTEP>(vop, rd + NSTEP * 1024);
          sums(vop, pp, key);
          if (more) issue_v(nt, j + 1);
        }
      });
    } else {
      // The two blocks of a sub-tile are copied whole (K: the second image 128 bytes further, so that the halves of a read hit
      // different banks), the operands' 8-byte chunks picked out of the images and converted.  Two sets.
      constexpr int NIB = BLKB / 1024, NIK = 2 * NIB, KSET = 2 * BLKB + 128, SET = KSET + 2 * BLKB;
      static_assert(2 * SET <= WAVE_LDS, "two sets per wave");
      const unsigned k_rd = wl_addr + (pr >> 4) * (BLKB + 128) + (half * 16 + (pr & 15)) * 8, v_rd = wl_addr + KSET + (half * D + pr) * 8;
      auto issue = [&](auto nt, int j) -> void {
        if (j && (j & 31) == 0) {
          load_table(j);
          pin_table();
        }
        lds_byte* set = wl + (j & 1) * SET;
#pragma unroll
        for (int x = 0; x < 4; ++x) {  // K of both blocks, then V
          const long long b = __builtin_amdgcn_readlane(bt_reg, 2 * (j & 31) + (x & 1));
          const unsigned char* g = (x < 2 ? p.k_pool : p.v_pool) + (b * p.n_kv_heads + it.kv_head) * BLKB + lane * 16;
#pragma unroll
          for (int i = 0; i < NIB; ++i)
            __builtin_amdgcn_global_load_lds(g + i * 1024, set + (x < 2 ? x * (BLKB + 128) : KSET + (x - 2) * BLKB) + i * 1024, 16, 0, decltype(nt)::value);
        }
      };
      stream([&](auto nt) -> void {
        if (n_iter > 0) issue(nt, 0);
        if (n_iter > 1) issue(nt, 1);
        pin_q();
        for (int j = 0; j < n_iter; ++j) {
          const int key = it.key_begin + 32 * (wave + WK * j);
          const bool more = j + 1 < n_iter;  // sub-tile j + 1 has been requested
          u32x4 kop[NSTEP], vop[NSTEP], pp[2];
          u32x2 codes[NSTEP];
          f32x16 sc;
          if (more) wait_vmcnt<3 * NIK>();
          else wait_vmcnt<NIK>();  // K(j) has landed
          if constexpr (NSTEP == 8) lds_read8_b64<0, 256, 512, 768, 1024, 1280, 1536, 1792>(codes, k_rd + (j & 1) * SET);
          else lds_read4_b64<0, 256, 512, 768>(codes, k_rd + (j & 1) * SET);
  #pragma unroll
          for (int x = 0; x < NSTEP; ++x) kop[x] = fp8x8_to_bf16x8(codes[x]);
          scores(kop, sc);
          weights(sc, key, pp);
          if (more) wait_vmcnt<2 * NIK>();
          else wait_vmcnt<0>();  // V(j) has landed
          if constexpr (NSTEP == 8) lds_read8_b64<0, 256, 512, 768, BLKB, BLKB + 256, BLKB + 512, BLKB + 768>(codes, v_rd + (j & 1) * SET);
          else lds_read4_b64<0, 256, BLKB, BLKB + 256>(codes, v_rd + (j & 1) * SET);
          if (j + 2 < n_iter) issue(nt, j + 2);  // the set is free again
  #pragma unroll
          for (int x = 0; x < NSTEP; ++x) vop[x] = fp8x8_to_bf16x8(codes[x]);
          sums(vop, pp, key);
        }
      });
    }

    put_result<D>(smem + wave * WAVE_LDS, c32, rows.o, half);
    rows.l = pair_sum(rows.l);
    if (half == 0) {
      ml_lds[wave][c32][0] = rows.m * c;
      ml_lds[wave][c32][1] = rows.l;
    }
    __syncthreads();
    float* part = p.partials + (long long)(2 * sh.index + (it.unit == 0 ? 1 : 0)) * kSlotFloats<D, ROWS>;
    const float v_factor = FP8 ? p.v_scale[it.kv_head] : 1.0f;
    for (int x = tid; x < it.n_rows * (D / 8); x += kThreads) join_and_store<D, ROWS, WK, 32>(p, it, smem, WAVE_LDS, ml_lds, x, part, v_factor);
    __syncthreads();
    note_split(p, sh, it);
  }
}

// ----------------------------------------------------------------------------------------------------------- many rows
template <int D, bool FP8, int WR>
__global__ __launch_bounds__(kThreads, 2) void tiles_kernel(TreeParams p) {
  constexpr int NSTEP = D / 16, NDB = D / 32, ESZ = FP8 ? 1 : 2, WK = kWaves / WR, ROWS = 32 * WR;
  constexpr int BLKB = 16 * D * ESZ;
  constexpr int PIECES = 4 * D;                           // of K and V of a block: 8 elements each, 16 bytes in LDS
  constexpr int TILE = kTileKeys / kBlock * PIECES * 16;  // bytes of a tile
  constexpr int PER = TILE / 16 / kThreads;               // pieces of a thread
  constexpr int kTiles = 2, SUBS = kTileKeys / 32 / WK;   // tiles in LDS; a wave's sub-tiles of one: wk, wk + WK, ...
  static_assert(SUBS >= 1, "a sub-tile for every wave");
  constexpr int RESULT = 32 * D * 4;
  constexpr int LDS = WK > 1 && kWaves * RESULT > kTiles * TILE ? kWaves * RESULT : kTiles * TILE;
  using Codes = std::conditional_t<FP8, u32x2, u32x4>;
  __shared__ __align__(1024) unsigned char smem[LDS];
  __shared__ float ml_lds[WK > 1 ? kWaves : 1][32][2];
  __shared__ ShareLds share_lds;

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, c32 = lane & 31, pr = perm32(c32);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WK, wk = wave % WK;
  const int group = p.n_q_heads / p.n_kv_heads;
  const Share sh = find_share<ROWS>(p, share_lds);
  if (tid == 0) p.splits[blockIdx.x].n_pieces = 0;
  if (sh.begin >= sh.end) return;
  Walk walk = begin_walk(sh);
  Piece it;
  while (next_piece<ROWS>(p, walk, it)) {
    Rows<D> rows;
    rows.clear();
    const int row = min(it.row0 + wr * 32 + c32, it.n.count * group - 1);
    rows.token = row / group;
    unsigned flip;
    const float c = score_factor<FP8>(p, it.kv_head, flip);
    const int* table = p.block_tables + (long long)it.seq * p.max_blocks;
    const int last_block = (it.kv_len - 1) / kBlock;
    const int n_tiles = (it.key_end - it.key_begin + kTileKeys - 1) / kTileKeys;

    // Table entries of 16 tiles in one register, a lane each, and of the 16 after them: an entry is there when its block is
    // requested (loaded with each tile, they cost it their round trip).
    constexpr int kAhead = 64 * kBlock / kTileKeys;
    auto load_table = [&](int j) { return table[min(it.key_begin / kBlock + j * (kTileKeys / kBlock) + lane, last_block)]; };
    int entries = load_table(0), entries_next = 0;
    if (n_tiles > kAhead) entries_next = load_table(kAhead);
    Codes r[PER];
    auto fetch = [&](int j) {  // tile j of the piece
      if (j && j % kAhead == 0) {
        entries = entries_next;
        entries_next = load_table(j + kAhead);
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int x = i * kThreads + tid, b = __builtin_amdgcn_readfirstlane(x / PIECES), in = x % PIECES;
        const long long block = __builtin_amdgcn_readlane(entries, (j % kAhead) * (kTileKeys / kBlock) + b);
        const unsigned char* pool = __builtin_amdgcn_readfirstlane(in / (PIECES / 2)) ? p.v_pool : p.k_pool;
        r[i] = *reinterpret_cast<const Codes*>(pool + (block * p.n_kv_heads + it.kv_head) * BLKB + in % (PIECES / 2) * (8 * ESZ));
      }
    };
    auto put = [&](int buffer) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        u32x4 w;
        if constexpr (FP8) w = fp8x8_to_bf16x8(r[i]);
        else w = r[i];
        *reinterpret_cast<u32x4*>(smem + buffer * TILE + (i * kThreads + tid) * 16) = w;
      }
    };
    fetch(0);
    {
      const unsigned short* qp =
          p.q + ((long long)(it.n.first + rows.token) * p.n_q_heads + it.kv_head * group + row - rows.token * group) * D + 8 * half;
#pragma unroll
      for (int st = 0; st < NSTEP; ++st) rows.q[st] = as_bf16x8(*reinterpret_cast<const u32x4*>(qp + 16 * st) ^ flip);
    }
    // One barrier a tile: a wave that puts tile j + 1 has passed the barrier of tile j, so every wave has left tile j - 1, whose place it takes.
    for (int j = 0; j < n_tiles; ++j) {
      const unsigned char* buffer = smem + (j & 1) * TILE;
      put(j & 1);
      if (j + 1 < n_tiles) fetch(j + 1);
      __syncthreads();
#pragma unroll
      for (int x = 0; x < SUBS; ++x) {
        const int key = it.key_begin + j * kTileKeys + 32 * (wk + WK * x);
        if (key >= it.key_end || wr * 32 >= it.n_rows) break;  // a wave without rows only moves tiles (34 trees of 112 .. 264 rows 574 / 529)
        const unsigned char* lds = buffer + 2 * (wk + WK * x) * (PIECES * 16);
        u32x4 kop[NSTEP], vop[NSTEP], pp[2];
        f32x16 sc;
#pragma unroll
        for (int st = 0; st < NSTEP; ++st)
          kop[st] = *reinterpret_cast<const u32x4*>(lds + (pr >> 4) * (PIECES * 16) + ((2 * st + half) * 16 + (pr & 15)) * 16);
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
        for (int st = 0; st < NSTEP; ++st) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kop[st]), rows.q[st], sc, 0, 0, 0);
        const bool tail = key + 32 > it.n.prefix;
        if (tail) hide_scores(sc, visible_bits(p, it.n, rows.token, key), half);
        const float mx = pair_max(lane_max(sc));
        if (__builtin_amdgcn_ballot_w64((mx - rows.m) * c > kLazyLog2) != 0) rows.rescale(fmaxf(rows.m, mx), c);  // as in stream_kernel
        rows.l += softmax_exp_part(sc, c, rows.m, pp);
#pragma unroll
        for (int y = 0; y < NSTEP; ++y)
          vop[y] = *reinterpret_cast<const u32x4*>(lds + y / NDB * (PIECES * 16) + PIECES * 8 + (half * D + y % NDB * 32 + pr) * 16);
        bool odd = false;
        if (tail) odd = tidy_values<D>(vop, key, it.kv_len, half);
#pragma unroll
        for (int y = 0; y < NSTEP; ++y)
          rows.o[y % NDB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vop[y]), as_bf16x8(pp[y / NDB]), rows.o[y % NDB], 0, 0, 0);
        if (odd) add_odd_values<D, FP8>(p, it, rows, pp, key, half, c32);
      }
    }

    float* part = p.partials + (long long)(2 * sh.index + (it.unit == 0 ? 1 : 0)) * kSlotFloats<D, ROWS>;
    const float v_factor = FP8 ? p.v_scale[it.kv_head] : 1.0f;
    __syncthreads();  // LDS is no longer read: the next piece's tiles, or the results, take the place of these
    rows.l = pair_sum(rows.l);
    if constexpr (WK == 1) {
      const int r0 = wr * 32 + c32;
      if (r0 < it.n_rows) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = rows.o[db][8 * h + e];
            const int d = 32 * db + 16 * h + 8 * half;
            if (it.whole) store_final<D>(p, it, r0, d, x, rows.l, v_factor);
            else store_partial<D>(part, r0, d, x);
          }
        if (!it.whole && half == 0) {
          part[ROWS * D + 2 * r0] = rows.m * c;
          part[ROWS * D + 2 * r0 + 1] = rows.l;
        }
      }
    } else {
      put_result<D>(smem + wave * RESULT, c32, rows.o, half);
      if (half == 0) {
        ml_lds[wave][c32][0] = rows.m * c;
        ml_lds[wave][c32][1] = rows.l;
      }
      __syncthreads();
      for (int x = tid; x < it.n_rows * (D / 8); x += kThreads) join_and_store<D, ROWS, WK, 32>(p, it, smem, RESULT, ml_lds, x, part, v_factor);
      __syncthreads();
    }
    note_split(p, sh, it);
  }
}

// Combines the pieces of the row tile that work-group blockIdx.x began and others went on with; a thread has 4 dims of a row.
template <int D, bool FP8, int ROWS>
__global__ __launch_bounds__(256) void merge_kernel(TreeParams p) {
  constexpr int kRows = 1024 / D;
  const Split sp = p.splits[blockIdx.x];
  const int r = blockIdx.y * kRows + (int)threadIdx.x / (D / 4), d = (int)threadIdx.x % (D / 4) * 4;
  if (r >= (sp.n_pieces ? sp.n_rows : 0)) return;
  float top = kNeg, sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < sp.n_pieces; ++i) {
    const float* part = p.partials + (long long)(2 * (sp.share + i) + (i == 0)) * kSlotFloats<D, ROWS>;
    const float m = part[ROWS * D + 2 * r], l = part[ROWS * D + 2 * r + 1];
    const f32x4 o = *reinterpret_cast<const f32x4*>(part + r * D + d);
    const float m_new = fmaxf(top, m);
    const float keep = __builtin_amdgcn_exp2f(top - m_new), add = __builtin_amdgcn_exp2f(m - m_new);
    sum = sum * keep + l * add;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = acc[e] * keep + o[e] * add;
    top = m_new;
  }
  const int group = p.n_q_heads / p.n_kv_heads, token = (sp.row0 + r) / group, head = sp.kv_head * group + (sp.row0 + r) - token * group;
  const float f = (FP8 ? p.v_scale[sp.kv_head] : 1.0f) / sum;
  u32x2 w = {pack_bf16(acc[0] * f, acc[1] * f), pack_bf16(acc[2] * f, acc[3] * f)};
  if (sum == 0.f && sees_nothing(p, Lens{sp.prefix, sp.count, sp.first_token}, token)) w = u32x2{0, 0};
  *reinterpret_cast<u32x2*>(p.out + ((long long)(sp.first_token + token) * p.n_q_heads + head) * D + d) = w;
}

int most_rows_of_tile(const cronus_kv_cache* cache, int32_t max_rows) {
  const long long rows = (long long)max_rows * (cache->num_q_heads / cache->num_kv_heads);
  return rows <= 32 ? 32 : rows <= 192 ? 128 : 256;
}
int rows_of_tile(const cronus_kv_cache* cache, int32_t max_rows, int32_t n_seqs) {
  const long long rows = (long long)max_rows * (cache->num_q_heads / cache->num_kv_heads);
  const double tiles = (double)((rows + 31) / 32) * cache->num_kv_heads * n_seqs;  // (a product of three counts)
  const int most = most_rows_of_tile(cache, max_rows);
  return tiles <= kFewRowTiles ? 32 : tiles < kManyRowTiles ? std::min(most, 128) : most;
}

size_t split_bytes(int n_cus) { return ((size_t)n_cus * sizeof(Split) + 255) / 256 * 256; }

template <int D, bool FP8, int ROWS>
int launch(const TreeParams& p, int n_cus, hipStream_t stream) {
  if constexpr (ROWS == 32) hipLaunchKernelGGL((stream_kernel<D, FP8>), dim3(n_cus), dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL((tiles_kernel<D, FP8, ROWS / 32>), dim3(n_cus), dim3(kThreads), 0, stream, p);
  if (hipGetLastError() != hipSuccess) return CRONUS_ERR_HIP;
  if (p.whole) return CRONUS_OK;  // no row tile is split
  hipLaunchKernelGGL((merge_kernel<D, FP8, ROWS>), dim3(n_cus, ROWS * D / 1024), dim3(256), 0, stream, p);
  return hipGetLastError() == hipSuccess ? CRONUS_OK : CRONUS_ERR_HIP;
}
template <int D, bool FP8>
int launch_rows(const TreeParams& p, int rows, int n_cus, hipStream_t stream) {
  switch (rows) {
    case 32: return launch<D, FP8, 32>(p, n_cus, stream);
    case 128: return launch<D, FP8, 128>(p, n_cus, stream);
    default: return launch<D, FP8, 256>(p, n_cus, stream);
  }
}

}  // namespace

size_t attn_tree_workspace(const cronus_kv_cache* cache, int32_t max_rows, int n_cus) {
  const size_t slot = (size_t)most_rows_of_tile(cache, max_rows) * (cache->head_dim + 2) * sizeof(float);
  return split_bytes(n_cus) + (2 * slot * n_cus + 255) / 256 * 256;
}

int launch_attn_tree(const cronus_kv_cache* cache, const void* q, void* out, const int32_t* prefix_lens, const int32_t* cu_rows,
                     const uint64_t* mask, int32_t mask_words, const int32_t* block_tables, int32_t max_blocks_per_seq, int32_t n_seqs,
                     int32_t max_rows, float sm_scale, void* workspace, int n_cus, void* stream) {
  TreeParams p{};
  p.q = static_cast<const unsigned short*>(q);
  p.out = static_cast<unsigned short*>(out);
  p.k_pool = static_cast<const unsigned char*>(cache->k_cache);
  p.v_pool = static_cast<const unsigned char*>(cache->v_cache);
  p.k_scale = cache->k_scale;
  p.v_scale = cache->v_scale;
  p.prefix_lens = prefix_lens;
  p.cu_rows = cu_rows;
  p.mask = reinterpret_cast<const unsigned long long*>(mask);
  p.mask_words = mask_words;
  p.block_tables = block_tables;
  p.max_blocks = max_blocks_per_seq;
  p.n_seqs = n_seqs;
  p.max_rows = max_rows;
  p.n_q_heads = cache->num_q_heads;
  p.n_kv_heads = cache->num_kv_heads;
  p.scale_log2e = sm_scale * 1.4426950408889634f;
  p.splits = static_cast<Split*>(workspace);
  p.partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + split_bytes(n_cus));
  const int rows = rows_of_tile(cache, max_rows, n_seqs);
  const double tiles = (double)(((long long)max_rows * (p.n_q_heads / p.n_kv_heads) + rows - 1) / rows) * p.n_kv_heads * n_seqs;
  const long long keys = (long long)max_blocks_per_seq * kBlock, step = rows == 32 ? 32 * kWaves : kTileKeys;  // one sub-tile or more for every wave
  long long unit_keys = step;
  p.whole = keys <= kWholeSteps * step;
  if (p.whole) unit_keys = (keys + step - 1) / step * step;
  auto too_many = [&] { return tiles * (double)((keys + unit_keys - 1) / unit_keys) >= (double)(kMostUnitShares / n_cus); };
  while (too_many() && unit_keys < kTreeMostKeys / 4) unit_keys *= 2;
  if (too_many()) return CRONUS_ERR_INVALID_ARG;
  p.unit_keys = (int)unit_keys;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool fp8 = cache->kv_dtype == CRONUS_KV_FP8_E4M3;
  if (cache->head_dim == 128) return fp8 ? launch_rows<128, true>(p, rows, n_cus, s) : launch_rows<128, false>(p, rows, n_cus, s);
  return fp8 ? launch_rows<64, true>(p, rows, n_cus, s) : launch_rows<64, false>(p, rows, n_cus, s);
}

}  // namespace cronus
