// Block tables, row offsets and slot maps from the sequences' lengths, all on the device, so that a loop whose lengths
// change on the device (drafts accepted or not) needs no round trip to the host between two iterations.
//
// With L cached and n new tokens and h blocks held by a sequence, it needs max(0, ceil((L + n) / 16) - h) blocks more; exclusive
// sums over the batch of the needs and of the new tokens say which entries of the free stack and which rows are its own.
// A new block holds at least one new token (h >= ceil(L / 16)), so whoever maps the first token of a block that the
// sequence did not hold also writes the table entry: one pass over the tokens fills both.
//
// plan_kernel, one work-group, checks the lengths, sums them and returns the blocks of ended sequences to the free stack;
// map_kernel writes table entries and slots, and is ordered behind it because it reads what that one returned.  A batch of few
// sequences and tokens is mapped by plan_kernel itself: one launch, and the sums are still in LDS.
#include <hip/hip_runtime.h>

#include "cronus_internal.h"

namespace cronus {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kMapThreads = 256, kMapTokens = 4;  // tokens of a thread of map_kernel
// Tokens of a batch that plan_kernel maps, of at most kPlanThreads sequences.  us a call, one launch / two: 208 tokens 6.0 / 9.0, 1024 7.8 / 8.9, 2048
// 8.7 / 8.7, 4096 10.1 / 8.4, 16384 21.9 / 8.5.
constexpr int kFewTokens = 2048;
// Sequences whose offsets map_kernel searches in LDS.  us a call, there / in memory: 256 sequences, of which 64 end, 16.4 / 17.0; 512 9.4 / 10.5; 2000
// 23.8 / 23.1; 4000 35.2 / 33.1.
constexpr int kMapSeqs = 1024;

struct TableParams {
  cronus_paged_tables t;
  const int* kv_lens;
  const int* new_lens;
  int n_seqs;
  int* cu_tokens;
  int* start_pos;
  int* cu_blocks;
  long long* slot_map;
  int max_tokens;
  int* report;
};

// What one sequence asks for; ok: its lengths fit its row, and its held blocks cover what is cached.
struct Ask {
  int start, add, need, back, held;
  bool ok;
};
__device__ __forceinline__ Ask ask_of(const TableParams& p, int s) {
  Ask a{};
  const int len = p.kv_lens[s], add = p.new_lens[s];
  a.held = p.t.held[s];
  const bool ended = add == -1;
  const long long end = (long long)len + (ended ? 0 : add);
  a.ok = len >= 0 && add >= -1 && a.held >= 0 && a.held <= p.t.max_blocks_per_seq && ((long long)len + kBlock - 1) / kBlock <= a.held &&
         end <= (long long)p.t.max_blocks_per_seq * kBlock && end <= 0x7fffffffLL;
  if (!a.ok) return a;
  a.start = ended ? 0 : len;
  a.add = ended ? 0 : add;
  a.back = ended ? a.held : 0;
  a.need = ended ? 0 : max(0, (int)((end + kBlock - 1) / kBlock) - a.held);
  return a;
}

struct Sums {
  long long tokens, need, back;
};
__device__ __forceinline__ Sums plus(Sums a, Sums b) { return {a.tokens + b.tokens, a.need + b.need, a.back + b.back}; }
__device__ __forceinline__ Sums from_lane(Sums a, int lane) {
  return {__shfl(a.tokens, lane), __shfl(a.need, lane), __shfl(a.back, lane)};
}

// Sum of the values of the threads before this one, and of all (*total).  lds: one entry for each wave.
__device__ __forceinline__ Sums scan_threads(Sums x, Sums* lds, Sums* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  Sums incl = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Sums y = from_lane(incl, lane - d < 0 ? lane : lane - d);
    if (lane >= d) incl = plus(incl, y);
  }
  if (waves == 1) {
    *total = from_lane(incl, 63);
  } else {
    if (lane == 63) lds[wave] = incl;
    __syncthreads();
    Sums before{0, 0, 0}, all{0, 0, 0};
#pragma unroll 2
    for (int w = 0; w < waves; ++w) {
      if (w == wave) before = all;
      all = plus(all, lds[w]);
    }
    __syncthreads();
    *total = all;
    incl = plus(incl, before);
  }
  return {incl.tokens - x.tokens, incl.need - x.need, incl.back - x.back};
}

// Last s in [0, n_seqs) with cu[s] <= token; sequences without tokens are passed over.
__device__ __forceinline__ int sequence_of(const int* cu, int n_seqs, int token) {
  int lo = 0, hi = n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cu[mid] <= token) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Slot of the token at position pos of a sequence (its table row, blocks that it held, blocks granted before it); the table entry of a
// granted block is written with the block's first token.  top: entries of the free stack before blocks were taken.
__device__ __forceinline__ long long map_token(const TableParams& p, int* row, int pos, int old_held, int grant, long long top) {
  const int column = pos / kBlock;
  const bool fresh = column >= old_held;
  const int* from = fresh ? p.t.free_blocks + (top - 1 - grant - (column - old_held)) : row + column;
  const int block = *from;
  if (fresh && pos % kBlock == 0) row[column] = block;
  return (long long)block * kBlock + pos % kBlock;
}

struct Ended {
  int seq, n;
  long long at;  // place of its blocks on the stack
};

template <bool MAPS>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(TableParams p) {
  __shared__ Sums lds[kPlanThreads / 64];
  __shared__ Ended ended[kPlanThreads];
  __shared__ int n_ended, first_bad;
  __shared__ int map_cu[MAPS ? kPlanThreads + 1 : 1], map_start[MAPS ? kPlanThreads : 1], map_held[MAPS ? kPlanThreads : 1], map_grant[MAPS ? kPlanThreads : 1];
  const int t = threadIdx.x, threads = blockDim.x, lane = t & 63;
  const long long count = *p.t.free_count;
  if (t == 0) first_bad = 0x7fffffff, n_ended = 0;
  __syncthreads();
  // One round of the threads holds the whole batch, or the sums come first and the batch is read again.
  const bool once = p.n_seqs <= threads;
  Ask a{};
  Sums mine{0, 0, 0}, total;
  for (int s = t; s < p.n_seqs; s += threads) {
    a = ask_of(p, s);
    if (!a.ok) {
      atomicMin(&first_bad, s);
      break;
    }
    mine = plus(mine, Sums{a.add, a.need, a.back});
  }
  Sums before = scan_threads(mine, lds, &total);
  __syncthreads();  // first_bad; and every thread has read free_count, which free_count_out may be
  const int bad = first_bad;
  int status = CRONUS_TABLES_OK;
  if (bad != 0x7fffffff || count < 0 || count + total.back > p.t.free_capacity) status = CRONUS_TABLES_BAD_LENGTHS;
  else if (total.need > count + total.back) status = CRONUS_TABLES_NO_BLOCKS;
  else if (total.tokens > p.max_tokens) status = CRONUS_TABLES_TOO_MANY_TOKENS;
  const bool ok = status == CRONUS_TABLES_OK;
  if (t == 0) {
    *p.t.free_count_out = (int)(ok ? count + total.back - total.need : count);
    p.cu_tokens[0] = 0;
    p.cu_blocks[0] = 0;
    p.report[0] = status;
    p.report[1] = (int)min(total.tokens, 0x7fffffffLL);
    p.report[2] = (int)min(total.need, 0x7fffffffLL);
    p.report[3] = bad != 0x7fffffff ? bad : -1;
  }
  Sums carry{0, 0, 0};
  for (int s0 = 0; s0 < p.n_seqs; s0 += threads) {
    const int s = s0 + t;
    if (!ok) {
      a = Ask{};
      before = carry;
      if (s < p.n_seqs) a.start = p.kv_lens[s], a.held = p.t.held[s];
    } else if (!once) {
      a = Ask{};
      if (s < p.n_seqs) a = ask_of(p, s);
      Sums part;
      before = plus(carry, scan_threads(Sums{a.add, a.need, a.back}, lds, &part));
      carry = plus(carry, part);
    }
    if (s < p.n_seqs) {
      p.cu_tokens[s + 1] = (int)(before.tokens + a.add);
      p.cu_blocks[s + 1] = (int)(before.need + a.need);
      p.start_pos[s] = a.start;
      p.t.held_out[s] = a.held - a.back + a.need;
      if constexpr (MAPS) {
        map_cu[s] = (int)before.tokens;
        map_start[s] = a.start;
        map_held[s] = a.held;
        map_grant[s] = (int)before.need;
      }
    }
    if (!ok || total.back == 0) continue;
    // The blocks of ended sequences: a list of them, and a wave for each, whose lanes request up to kAhead entries before they
    // store the first (one at a time, 64 of 256 sequences with 260 blocks each took 20 us).
    if (a.back > 0) ended[atomicAdd(&n_ended, 1)] = Ended{s, a.back, count + before.back};
    __syncthreads();
    const int listed = n_ended;
    for (int x = t >> 6; x < listed; x += threads >> 6) {
      const Ended e = ended[x];
      const int* row = p.t.block_tables + (long long)e.seq * p.t.max_blocks_per_seq;
      constexpr int kAhead = 8;
      for (int i0 = lane; i0 < e.n; i0 += 64 * kAhead) {
        int b[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) b[k] = i0 + 64 * k < e.n ? row[i0 + 64 * k] : 0;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (i0 + 64 * k < e.n) p.t.free_blocks[e.at + i0 + 64 * k] = b[k];
      }
    }
    __syncthreads();
    if (t == 0) n_ended = 0;
    __syncthreads();
  }
  if constexpr (MAPS) {
    if (!ok) return;
    const int tokens = (int)total.tokens;
    const long long top = count + total.back;
    __syncthreads();  // the offsets in LDS, and what this work-group returned to the stack
#pragma unroll 4
    for (int token = t; token < tokens; token += threads) {
      const int s = sequence_of(map_cu, p.n_seqs, token);
      const long long slot = map_token(p, p.t.block_tables + (long long)s * p.t.max_blocks_per_seq, map_start[s] + token - map_cu[s], map_held[s],
                                       map_grant[s], top);
      if (p.slot_map) p.slot_map[token] = slot;
    }
  }
}

__global__ __launch_bounds__(kMapThreads) void map_kernel(TableParams p) {
  __shared__ int cu_lds[kMapSeqs];
  const int total = p.cu_tokens[p.n_seqs];
  const long long first = ((long long)blockIdx.x * kMapThreads + threadIdx.x) * kMapTokens;
  if ((long long)blockIdx.x * kMapThreads * kMapTokens >= total) return;
  const int* cu = p.cu_tokens;
  if (p.n_seqs <= kMapSeqs) {  // one round trip instead of one for each step of the search
    for (int i = threadIdx.x; i < p.n_seqs; i += kMapThreads) cu_lds[i] = p.cu_tokens[i];
    __syncthreads();
    cu = cu_lds;
  }
  if (first >= total) return;
  int s = sequence_of(cu, p.n_seqs, (int)first);
  const long long top = (long long)*p.t.free_count_out + p.cu_blocks[p.n_seqs];  // entries of the stack before blocks were taken
  int end = -1, start = 0, base = 0, old_held = 0, grant = 0;
  int* row = nullptr;
  for (int i = 0; i < kMapTokens; ++i) {
    const int token = (int)first + i;
    if (token >= total) return;
    while (end <= token) {  // the next sequence that has tokens
      if (end >= 0) ++s;
      end = p.cu_tokens[s + 1];
      base = p.cu_tokens[s];
      if (end <= token) continue;
      start = p.start_pos[s];
      grant = p.cu_blocks[s];
      old_held = p.t.held_out[s] - (p.cu_blocks[s + 1] - grant);
      row = p.t.block_tables + (long long)s * p.t.max_blocks_per_seq;
    }
    const long long slot = map_token(p, row, start + (token - base), old_held, grant, top);
    if (p.slot_map) p.slot_map[token] = slot;
  }
}

}  // namespace

int launch_build_tables(const cronus_paged_tables* tables, const int32_t* kv_lens, const int32_t* new_lens, int32_t n_seqs,
                        int32_t* cu_tokens, int32_t* start_pos, int32_t* cu_blocks, int64_t* slot_map, int32_t max_tokens,
                        int32_t* report, void* stream) {
  const TableParams p{*tables, kv_lens, new_lens, n_seqs, cu_tokens, start_pos, cu_blocks, reinterpret_cast<long long*>(slot_map), max_tokens, report};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool maps = n_seqs <= kPlanThreads && max_tokens <= kFewTokens;
  const int busy = maps && max_tokens > n_seqs ? max_tokens : n_seqs;
  const int threads = busy < kPlanThreads ? busy < 64 ? 64 : (busy + 63) / 64 * 64 : kPlanThreads;
  hipLaunchKernelGGL(maps ? plan_kernel<true> : plan_kernel<false>, dim3(1), dim3(threads), 0, s, p);
  if (hipGetLastError() != hipSuccess) return CRONUS_ERR_HIP;
  if (maps || max_tokens == 0) return CRONUS_OK;
  const unsigned per = kMapThreads * kMapTokens;
  hipLaunchKernelGGL(map_kernel, dim3(((unsigned)max_tokens + per - 1) / per), dim3(kMapThreads), 0, s, p);
  return hipGetLastError() == hipSuccess ? CRONUS_OK : CRONUS_ERR_HIP;
}

}  // namespace cronus
