// The K/V rows of an accepted path of drafted tokens move to the positions behind the cached ones, in the caches of all
// layers at once: position start + path[k] -> start + k, k = 0 .. m - 1.
//
// A path's entries increase strictly (a drafted token lies behind its parent), so path[k] >= k: a destination lies at or before its source,
// and before the sources of all later entries.  So kPiece entries at a time are read, then written, each piece behind the one before it, and
// no row is overwritten before it has been read.  An entry with path[k] = k stays where it is.
//
// A wavefront moves the rows of one (KV head, cache) pair at a time, by itself: what it needs of the path and the table is the same for all
// pairs and is looked up once.  Bound by the number of lines that a row touches: in the V pool (include/cronus.h) a token's D values lie 8
// elements apart, next to those of its 7 neighbours, and in the K pool its D / 8 chunks 16 chunks apart.  96 sequences that keep up to 9 of 20 .. 64
// tokens, 32 fp8 caches of 8 heads: 81 us for 25 MB read and 25 MB written, of which 150 MB are fetched from HBM.  Without the K side it takes
// 47, without the V side 51.  V's groups of 8 tokens put together in registers and stored whole took 82 there, and 1 .. 1.5 us more in
// small calls (8 sequences of 5, 32 bf16 caches: 10.3 us, of which the host takes most).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cronus_internal.h"
#include "lane_ops.h"

namespace cronus {
namespace {

constexpr int kCommitThreads = 256, kCommitWaves = kCommitThreads / 64, kPiece = 8;
constexpr int kCommitCaches = 64;  // caches of one launch: their addresses are kernel arguments
// Work-groups that a launch has at least before its wavefronts take several pairs each (and look the path up once for them).  With 4096 / 2048 /
// 1024 the call above takes 81 / 86 / 91 us: rows in flight count for more than lookups.
constexpr long long kCommitGroups = 4096;

struct CommitParams {
  const int* start_pos;
  const int* cu_rows;
  const int* paths;
  const int* path_lens;
  const int* block_tables;
  int* kv_lens_out;  // or nullptr
  int max_path, max_blocks, n_kv_heads, n_pairs, per_wave;
  void* k[kCommitCaches];
  void* v[kCommitCaches];
};

template <int ESZ> struct Piece;
template <> struct Piece<2> { typedef u32x4 chunk; typedef unsigned short element; };
template <> struct Piece<1> { typedef u32x2 chunk; typedef unsigned char element; };

template <int D, int ESZ>
__global__ __launch_bounds__(kCommitThreads) void commit_kernel(CommitParams p) {
  using Chunk = typename Piece<ESZ>::chunk;
  using Element = typename Piece<ESZ>::element;
  constexpr int kChunks = kPiece * (D / 8) / 64, kDims = D / 64;  // of K of a piece, of V of a row: a lane's
  const int s = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int start = p.start_pos[s];
  const long long n = (long long)p.cu_rows[s + 1] - p.cu_rows[s];
  const int* path = p.paths + (long long)s * p.max_path;
  // The path ends at the first entry that is not one of the sequence's rows or not behind the entry before it.
  int m = 0;
  if (start >= 0 && n > 0 && start + n <= min((long long)p.max_blocks * kBlock, 0x7fffffffLL)) {
    const int most = min(p.path_lens[s], p.max_path);
    for (; m < most; m += 64) {
      const int k = m + lane;
      bool good = false;
      if (k < most) {
        const int a = path[k];
        good = a < n && a > (k > 0 ? path[k - 1] : -1);
      }
      const unsigned long long bad = ~__builtin_amdgcn_ballot_w64(good);
      if (bad) {
        m += __builtin_ctzll(bad);
        break;
      }
    }
  }
  if (p.kv_lens_out && blockIdx.y == 0 && threadIdx.x == 0) p.kv_lens_out[s] = start + m;

  const int* table = p.block_tables + (long long)s * p.max_blocks;
  const int first_pair = (blockIdx.y * kCommitWaves + wave) * p.per_wave, last_pair = min(first_pair + p.per_wave, p.n_pairs);
  for (int k0 = 0; k0 < m; k0 += kPiece) {
    // Lane k: where entry k0 + k comes from and goes to.
    int from_block = 0, from_slot = 0, to_block = 0, to_slot = 0;
    bool moves = false;
    if (lane < kPiece && k0 + lane < m) {
      const int a = path[k0 + lane], from = start + a, to = start + k0 + lane;
      moves = from != to;
      if (moves) {
        from_block = table[from / kBlock];
        to_block = table[to / kBlock];
      }
      from_slot = from % kBlock;
      to_slot = to % kBlock;
    }
    const unsigned long long moving = __builtin_amdgcn_ballot_w64(moves);
    if (!moving) continue;
    for (int pair = first_pair; pair < last_pair; ++pair) {
      const int cache = pair / p.n_kv_heads, head = pair - cache * p.n_kv_heads;
      Element* const k_pool = static_cast<Element*>(p.k[cache]);
      Element* const v_pool = static_cast<Element*>(p.v[cache]);
      auto base = [&](int block) { return ((long long)block * p.n_kv_heads + head) * (kBlock * D); };
      Chunk kk[kChunks];
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const int x = i * 64 + lane, e = x / (D / 8), dc = x % (D / 8), block = __shfl(from_block, e), slot = __shfl(from_slot, e);
        if (moving >> e & 1) kk[i] = *reinterpret_cast<const Chunk*>(k_pool + base(block) + (dc * kBlock + slot) * 8);
      }
      Element vv[kPiece][kDims];
#pragma unroll
      for (int e = 0; e < kPiece; ++e) {
        if (moving >> e & 1) {
          const int slot = __builtin_amdgcn_readlane(from_slot, e);
          const Element* g = v_pool + base(__builtin_amdgcn_readlane(from_block, e)) + slot / 8 * D * 8 + slot % 8;
#pragma unroll
          for (int i = 0; i < kDims; ++i) vv[e][i] = g[(64 * i + lane) * 8];
        }
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // every source of this piece has been read
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const int x = i * 64 + lane, e = x / (D / 8), dc = x % (D / 8), block = __shfl(to_block, e), slot = __shfl(to_slot, e);
        if (moving >> e & 1) *reinterpret_cast<Chunk*>(k_pool + base(block) + (dc * kBlock + slot) * 8) = kk[i];
      }
#pragma unroll
      for (int e = 0; e < kPiece; ++e) {
        if (moving >> e & 1) {
          const int slot = __builtin_amdgcn_readlane(to_slot, e);
          Element* g = v_pool + base(__builtin_amdgcn_readlane(to_block, e)) + slot / 8 * D * 8 + slot % 8;
#pragma unroll
          for (int i = 0; i < kDims; ++i) g[(64 * i + lane) * 8] = vv[e][i];
        }
      }
    }
  }
}

}  // namespace

int launch_kv_commit(const cronus_kv_cache* caches, int32_t n_caches, const int32_t* start_pos, const int32_t* cu_rows,
                     const int32_t* paths, int32_t max_path, const int32_t* path_lens, const int32_t* block_tables,
                     int32_t max_blocks_per_seq, int32_t n_seqs, int32_t* kv_lens_out, void* stream) {
  if (caches->num_kv_heads > kMaxScatterHeads) return CRONUS_ERR_INVALID_ARG;
  CommitParams p{start_pos, cu_rows, paths, path_lens, block_tables, kv_lens_out, max_path, max_blocks_per_seq, caches->num_kv_heads, 0, 1, {}, {}};
  const bool fp8 = caches->kv_dtype == CRONUS_KV_FP8_E4M3;
  auto kernel = caches->head_dim == 128 ? (fp8 ? commit_kernel<128, 1> : commit_kernel<128, 2>)
                                        : (fp8 ? commit_kernel<64, 1> : commit_kernel<64, 2>);
  for (int c0 = 0; c0 < n_caches; c0 += kCommitCaches) {
    const int n = n_caches - c0 < kCommitCaches ? n_caches - c0 : kCommitCaches;
    for (int i = 0; i < n; ++i) p.k[i] = caches[c0 + i].k_cache, p.v[i] = caches[c0 + i].v_cache;
    p.kv_lens_out = c0 == 0 ? kv_lens_out : nullptr;
    p.n_pairs = n * caches->num_kv_heads;
    const long long groups = ((long long)p.n_pairs + kCommitWaves - 1) / kCommitWaves;  // of a sequence, with one pair a wavefront
    p.per_wave = (int)std::max({1LL, std::min(groups, groups * n_seqs / kCommitGroups), (groups + 65534) / 65535});
    const unsigned y = (unsigned)((groups + p.per_wave - 1) / p.per_wave);
    hipLaunchKernelGGL(kernel, dim3((unsigned)n_seqs, y), dim3(kCommitThreads), 0, static_cast<hipStream_t>(stream), p);
    if (hipGetLastError() != hipSuccess) return CRONUS_ERR_HIP;
  }
  return CRONUS_OK;
}

}  // namespace cronus
