// Block tables, row offsets and slot maps from the sequences' lengths, all on the device, so that a loop whose lengths
// change on the device (drafts accepted or not) needs no round trip to the host between two iterations.
//
// With L cached and n new tokens and h blocks held by a sequence, it needs max(0, ceil((L + n) / 16) - h) blocks more; exclusive
// sums over the batch of the needs and of the new tokens say which entries of the free stack and which rows are its own.
// A new block holds at least one new token (h >= ceil(L / 16)), so whoever maps the first token of a block that the
// sequence did not hold also writes the table entry: one pass over the tokens fills both.
//
// Two launches: plan_kernel, one work-group, checks the lengths, sums them and returns the blocks of ended sequences to the
// free stack; map_kernel writes table entries and slots, and is ordered behind it because it reads what that one returned.
#include <hip/hip_runtime.h>

#include "cronus_internal.h"

namespace cronus {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kMapThreads = 256, kMapTokens = 4;  // tokens of a thread of map_kernel

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
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Sums incl = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Sums y = from_lane(incl, lane - d < 0 ? lane : lane - d);
    if (lane >= d) incl = plus(incl, y);
  }
  if (lane == 63) lds[wave] = incl;
  __syncthreads();
  Sums before{0, 0, 0}, all{0, 0, 0};
#pragma unroll 2
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w == wave) before = all;
    all = plus(all, lds[w]);
  }
  __syncthreads();
  *total = all;
  return {before.tokens + incl.tokens - x.tokens, before.need + incl.need - x.need, before.back + incl.back - x.back};
}

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(TableParams p) {
  __shared__ Sums lds[kPlanThreads / 64];
  __shared__ int first_bad;
  const int t = threadIdx.x;
  if (t == 0) first_bad = 0x7fffffff;
  __syncthreads();
  Sums mine{0, 0, 0}, total;
  for (int s = t; s < p.n_seqs; s += kPlanThreads) {
    const Ask a = ask_of(p, s);
    if (!a.ok) {
      atomicMin(&first_bad, s);
      break;
    }
    mine = plus(mine, Sums{a.add, a.need, a.back});
  }
  scan_threads(mine, lds, &total);
  const int bad = first_bad;
  const long long count = *p.t.free_count;
  int status = CRONUS_TABLES_OK;
  if (bad != 0x7fffffff || count < 0 || count + total.back > p.t.free_capacity) status = CRONUS_TABLES_BAD_LENGTHS;
  else if (total.need > count + total.back) status = CRONUS_TABLES_NO_BLOCKS;
  else if (total.tokens > p.max_tokens) status = CRONUS_TABLES_TOO_MANY_TOKENS;
  const bool ok = status == CRONUS_TABLES_OK;
  __syncthreads();  // every thread has read free_count, which free_count_out may be
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
  for (int s0 = 0; s0 < p.n_seqs; s0 += kPlanThreads) {
    const int s = s0 + t;
    Ask a{};
    if (s < p.n_seqs) {
      if (ok) a = ask_of(p, s);
      else a.start = p.kv_lens[s], a.held = p.t.held[s];
    }
    Sums part;
    const Sums before = plus(carry, scan_threads(Sums{a.add, a.need, a.back}, lds, &part));
    carry = plus(carry, part);
    if (s < p.n_seqs) {
      p.cu_tokens[s + 1] = (int)(before.tokens + a.add);
      p.cu_blocks[s + 1] = (int)(before.need + a.need);
      p.start_pos[s] = a.start;
      p.t.held_out[s] = a.held - a.back + a.need;
    }
    // The blocks of this wave's ended sequences, one sequence after the other, 64 entries at a time.
    unsigned long long ended = __builtin_amdgcn_ballot_w64(a.back > 0);
    while (ended) {
      const int from = __builtin_ctzll(ended);
      ended &= ended - 1;
      const int n = __shfl(a.back, from);
      const long long at = count + __shfl(before.back, from);
      const int* row = p.t.block_tables + (long long)(s - (t & 63) + from) * p.t.max_blocks_per_seq;
      for (int i = t & 63; i < n; i += 64) p.t.free_blocks[at + i] = row[i];
    }
  }
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

__global__ __launch_bounds__(kMapThreads) void map_kernel(TableParams p) {
  const int total = p.cu_tokens[p.n_seqs];
  const long long first = ((long long)blockIdx.x * kMapThreads + threadIdx.x) * kMapTokens;
  if (first >= total) return;
  int s = sequence_of(p.cu_tokens, p.n_seqs, (int)first);
  const long long top = (long long)*p.t.free_count_out + p.cu_blocks[p.n_seqs];  // entries of the stack before the blocks were taken
  int end = -1, start = 0, base = 0, old_held = 0;
  long long grant = 0;
  const int* row = nullptr;
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
      old_held = p.t.held_out[s] - (p.cu_blocks[s + 1] - (int)grant);
      row = p.t.block_tables + (long long)s * p.t.max_blocks_per_seq;
    }
    const int pos = start + (token - base), column = pos / kBlock;
    int block;
    if (column < old_held) {
      block = row[column];
    } else {
      block = p.t.free_blocks[top - 1 - (grant + column - old_held)];
      if (pos % kBlock == 0) const_cast<int*>(row)[column] = block;
    }
    if (p.slot_map) p.slot_map[token] = (long long)block * kBlock + pos % kBlock;
  }
}

}  // namespace

int launch_build_tables(const cronus_paged_tables* tables, const int32_t* kv_lens, const int32_t* new_lens, int32_t n_seqs,
                        int32_t* cu_tokens, int32_t* start_pos, int32_t* cu_blocks, int64_t* slot_map, int32_t max_tokens,
                        int32_t* report, void* stream) {
  const TableParams p{*tables, kv_lens, new_lens, n_seqs, cu_tokens, start_pos, cu_blocks, reinterpret_cast<long long*>(slot_map), max_tokens, report};
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, p);
  if (hipGetLastError() != hipSuccess) return CRONUS_ERR_HIP;
  if (n_seqs == 0 || max_tokens == 0) return CRONUS_OK;
  const unsigned per = kMapThreads * kMapTokens;
  hipLaunchKernelGGL(map_kernel, dim3(((unsigned)max_tokens + per - 1) / per), dim3(kMapThreads), 0, s, p);
  return hipGetLastError() == hipSuccess ? CRONUS_OK : CRONUS_ERR_HIP;
}

}  // namespace cronus
