// The K/V rows of an accepted path of drafted tokens move to the positions behind the cached ones, in the caches of all
// layers at once: position start + path[k] -> start + k, k = 0 .. m - 1.
//
// A path's entries increase strictly (a drafted token lies behind its parent), so path[k] >= k: a destination lies at or before its source,
// and before the sources of all later entries.  So kPiece entries at a time are read, then written, each piece behind the one before it, and
// no row is overwritten before it has been read.  An entry with path[k] = k stays where it is.
//
// Bound by the number of lines that a row touches: in the V pool (include/cronus.h) a token's D values lie 8 elements apart, next to those of
// its 7 neighbours, so a row of 2 D bytes is read from, and written to, 16 D bytes of lines.
#include <hip/hip_runtime.h>

#include "cronus_internal.h"
#include "lane_ops.h"

namespace cronus {
namespace {

constexpr int kCommitThreads = 256, kPiece = 16;
constexpr int kCommitCaches = 64;  // caches of one launch: their addresses are kernel arguments

struct CommitParams {
  const int* start_pos;
  const int* cu_rows;
  const int* paths;
  const int* path_lens;
  const int* block_tables;
  int* kv_lens_out;  // or nullptr
  int max_path, max_blocks, n_kv_heads;
  void* k[kCommitCaches];
  void* v[kCommitCaches];
};

template <int ESZ> struct Piece;
template <> struct Piece<2> { typedef u32x4 chunk; typedef unsigned short element; };
template <> struct Piece<1> { typedef u32x2 chunk; typedef unsigned char element; };

// Work-group (sequence, KV head, cache).
template <int D, int ESZ>
__global__ __launch_bounds__(kCommitThreads) void commit_kernel(CommitParams p) {
  using Chunk = typename Piece<ESZ>::chunk;
  using Element = typename Piece<ESZ>::element;
  constexpr int kTokens = kCommitThreads / D;  // of V in one step of the work-group
  constexpr int kSteps = kPiece / kTokens;
  const int s = blockIdx.x, head = blockIdx.y, t = threadIdx.x, lane = t & 63;
  const int start = p.start_pos[s];
  const long long n = (long long)p.cu_rows[s + 1] - p.cu_rows[s];
  const int* path = p.paths + (long long)s * p.max_path;
  // The path ends at the first entry that is not one of the sequence's rows or not behind the entry before it.
  int m = 0;
  if (start >= 0 && n > 0 && start + n <= (long long)p.max_blocks * kBlock) {
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
  if (p.kv_lens_out && head == 0 && blockIdx.z == 0 && t == 0) p.kv_lens_out[s] = start + m;

  const int* table = p.block_tables + (long long)s * p.max_blocks;
  Element* k_pool = static_cast<Element*>(p.k[blockIdx.z]);
  Element* v_pool = static_cast<Element*>(p.v[blockIdx.z]);
  auto base = [&](int pos) { return ((long long)table[pos / kBlock] * p.n_kv_heads + head) * (kBlock * D); };
  for (int k0 = 0; k0 < m; k0 += kPiece) {
    // K: thread = (entry, chunk of 8 dims)
    const int ke = k0 + (t & 15), dc = t >> 4;
    const int ka = ke < m ? path[ke] : ke;
    const bool k_moves = ka != ke && dc < D / 8;
    Chunk kk{};
    if (k_moves) {
      const int pos = start + ka;
      kk = *reinterpret_cast<const Chunk*>(k_pool + base(pos) + (dc * kBlock + pos % kBlock) * 8);
    }
    // V: thread = (entry of kTokens, dim)
    const int d = t % D;
    Element vv[kSteps];
    bool v_moves[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int e = k0 + i * kTokens + t / D;
      const int a = e < m ? path[e] : e;
      v_moves[i] = a != e;
      if (v_moves[i]) {
        const int pos = start + a;
        vv[i] = v_pool[base(pos) + ((pos % kBlock / 8) * D + d) * 8 + pos % 8];
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // every source of this piece has been read
    if (k_moves) {
      const int pos = start + ke;
      *reinterpret_cast<Chunk*>(k_pool + base(pos) + (dc * kBlock + pos % kBlock) * 8) = kk;
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (v_moves[i]) {
        const int pos = start + k0 + i * kTokens + t / D;
        v_pool[base(pos) + ((pos % kBlock / 8) * D + d) * 8 + pos % 8] = vv[i];
      }
    }
  }
}

}  // namespace

int launch_kv_commit(const cronus_kv_cache* caches, int32_t n_caches, const int32_t* start_pos, const int32_t* cu_rows,
                     const int32_t* paths, int32_t max_path, const int32_t* path_lens, const int32_t* block_tables,
                     int32_t max_blocks_per_seq, int32_t n_seqs, int32_t* kv_lens_out, void* stream) {
  if (caches->num_kv_heads > kMaxScatterHeads) return CRONUS_ERR_INVALID_ARG;
  CommitParams p{start_pos, cu_rows, paths, path_lens, block_tables, kv_lens_out, max_path, max_blocks_per_seq, caches->num_kv_heads, {}, {}};
  const bool fp8 = caches->kv_dtype == CRONUS_KV_FP8_E4M3;
  auto kernel = caches->head_dim == 128 ? (fp8 ? commit_kernel<128, 1> : commit_kernel<128, 2>)
                                        : (fp8 ? commit_kernel<64, 1> : commit_kernel<64, 2>);
  for (int c0 = 0; c0 < n_caches; c0 += kCommitCaches) {
    const int n = n_caches - c0 < kCommitCaches ? n_caches - c0 : kCommitCaches;
    for (int i = 0; i < n; ++i) p.k[i] = caches[c0 + i].k_cache, p.v[i] = caches[c0 + i].v_cache;
    p.kv_lens_out = c0 == 0 ? kv_lens_out : nullptr;
    hipLaunchKernelGGL(kernel, dim3((unsigned)n_seqs, (unsigned)caches->num_kv_heads, (unsigned)n), dim3(kCommitThreads), 0,
                       static_cast<hipStream_t>(stream), p);
    if (hipGetLastError() != hipSuccess) return CRONUS_ERR_HIP;
  }
  return CRONUS_OK;
}

}  // namespace cronus
