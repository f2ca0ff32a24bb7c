// The cache of merged decoders: rows appended, entries evicted.
#pragma once
#include "decoder.h"

namespace nf {

struct AppendArgs {
  const void* K; const void* V; const int* index; const int* count; const int* len; const int* start;
  void* Kc; void* Vc; int* pos; float* weight;
  int M, B, T, n, C, kv, units;                            // units: pieces of type U per row and head
  long stride_m, stride_row;                               // in pieces
};

// Copies of U at a time (16 bytes where rows and strides allow, one element otherwise).  A workgroup takes `rows` new rows of one sequence;
// consecutive threads take consecutive pieces of a head's row, on both sides.
template <typename U>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendArgs a, int rows, int blocks_per_seq) {
  const unsigned umb = blockIdx.x / blocks_per_seq;
  const long mb = umb, m = umb / a.B;
  const int i0 = (int)(blockIdx.x % blocks_per_seq) * rows, b = (int)(umb % a.B);
  const int cnt = a.count ? clamp_len(a.count[mb], a.n) : a.n, L = clamp_len(a.len[mb], a.C);
  const int end = min(min(i0 + rows, cnt), a.C - L);       // entries past the capacity are not written
  const int per_row = a.kv * a.units;
  for (int i = i0 + (int)threadIdx.x / per_row, c = (int)threadIdx.x % per_row; i < end;) {
    const int row = a.index ? a.index[mb * a.n + i] : i;
    if (row >= 0 && row < a.T) {
      const int g = c / a.units, u = c % a.units;
      const long from = m * a.stride_m + ((long)b * a.T + row) * a.stride_row + c;
      const long slot = (mb * a.kv + g) * a.C + L + i;
      ((U*)a.Kc)[slot * a.units + u] = ((const U*)a.K)[from];
      ((U*)a.Vc)[slot * a.units + u] = ((const U*)a.V)[from];
      if (u == 0) {
        if (a.pos) a.pos[slot] = (a.start ? a.start[mb] : L) + i;
        if (a.weight) a.weight[slot] = 0.f;
      }
    }
    c += 256;
    i += c / per_row;
    c %= per_row;
  }
}

struct EvictArgs {
  void* Kc; void* Vc; const int* pos; const float* weight; const int* len; const int* start; int* pos_out; float* weight_out; int* ws;
  int M, B, C, kv, units, budget, recent, most;            // most: pairs that a head can have, min(budget, C - budget)
};

// Bits of a weight in the order of its value: -0 counts as 0, NaN as the largest.
__device__ __forceinline__ uint32_t weight_order(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Inclusive sum over a wavefront: within rows of 16 lanes, then each row's last lane into the next row, then lane 31 into the upper half.
template <int CTRL, int ROWS> __device__ __forceinline__ int add_from(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, true); }
__device__ __forceinline__ int wave_scan(int x) {
  constexpr int kRowShr = 0x110, kRowBcast15 = 0x142, kRowBcast31 = 0x143;
  x = add_from<kRowShr + 1, 0xf>(x);
  x = add_from<kRowShr + 2, 0xf>(x);
  x = add_from<kRowShr + 4, 0xf>(x);
  x = add_from<kRowShr + 8, 0xf>(x);
  x = add_from<kRowBcast15, 0xa>(x);
  return add_from<kRowBcast31, 0xc>(x);
}

// Exclusive sum over the NT threads of a workgroup, `total` their sum.  Every thread has to come here; wave_sums must not be in use by another sum.
template <int NT> __device__ __forceinline__ int block_sum(int v, int* wave_sums, int& total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int x = wave_scan(v);
  if (lane == kWave - 1) wave_sums[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) {
    const int s = wave_sums[w];
    before += w < wave ? s : 0;
    total += s;
  }
  return before + x - v;
}
// The same where wave_sums is used again.
template <int NT> __device__ __forceinline__ int block_scan(int v, int* wave_sums, int& total) {
  const int r = block_sum<NT>(v, wave_sums, total);
  __syncthreads();
  return r;
}

// One digit of the search: hist holds how many candidates have each of 2048 digits; the digit of the want-th of them, and want among those that share it.
template <int NT> __device__ __forceinline__ int pick_digit(const int* hist, int* wave_sums, int* found, int& want) {
  constexpr int kBins = 2048 / NT;
  int c[kBins], sum = 0, total;
#pragma unroll
  for (int i = 0; i < kBins; ++i) {
    c[i] = hist[kBins * threadIdx.x + i];
    sum += c[i];
  }
  int before = block_sum<NT>(sum, wave_sums, total);
#pragma unroll
  for (int i = 0; i < kBins; ++i) {
    if (before < want && want <= before + c[i]) found[0] = kBins * threadIdx.x + i, found[1] = before;
    before += c[i];
  }
  __syncthreads();
  want -= found[1];                                        // at least 1 of the entries with this digit
  return found[0];
}

// Which entries of one head leave, caches of any size: one workgroup finds the n-th smallest (guarded, weight) by digits of 11, 11 and 10 bits of the weight's order,
// then walks the slots in order, giving entries equal to it to the lowest slots, and writes the list of free slots below the budget and
// that of the entries above it that stay (equally many).  Counts in LDS: whole numbers, so their order does not matter.
__global__ __launch_bounds__(1024) void evict_select_kernel(EvictArgs a) {
  __shared__ int hist[2048];
  __shared__ int wave_sums[16];
  __shared__ int found[2];
  const int tid = threadIdx.x;
  const long head = blockIdx.x, mb = blockIdx.x / a.kv;
  const int L = clamp_len(a.len[mb], a.C);
  const int keep = min(L, a.budget), n = L - keep;
  const long long bound = (long long)(a.start ? a.start[mb] : L) - a.recent;     // guarded from this position on
  const float* w = a.weight + head * a.C;
  const int* pos = a.pos ? a.pos + head * a.C : nullptr;
  int* const count = a.ws + head * (1 + 2 * (long)a.most);
  int* const holes = count + 1;
  int* const movers = holes + a.most;
  auto is_guarded = [&](int j) { return a.recent > 0 && (long long)pos[j] >= bound; };
  if (n == 0) {                                            // uniform
    if (tid == 0) *count = 0;
    for (int j = tid; j < keep; j += 1024) {
      if (a.weight_out != a.weight) a.weight_out[head * a.C + j] = w[j];
      if (pos && a.pos_out != a.pos) a.pos_out[head * a.C + j] = pos[j];
    }
    return;
  }
  int open = 0, total;
  for (int j = tid; j < L; j += 1024) open += !is_guarded(j);
  block_scan<1024>(open, wave_sums, open);
  const bool guards = n > open;                            // all the others leave and some guarded entries too
  int want = guards ? n - open : n;                        // so many of the group with is_guarded == guards, from the smallest
  uint32_t prefix = 0;
  for (int shift = 21, bits = 11; bits > 0;) {
    for (int d = tid; d < 2048; d += 1024) hist[d] = 0;
    __syncthreads();
    for (int j = tid; j < L; j += 1024) {
      const uint32_t o = weight_order(w[j]);
      if (is_guarded(j) == guards && (shift + bits == 32 || (o >> (shift + bits)) == prefix)) atomicAdd(&hist[(o >> shift) & ((1u << bits) - 1)], 1);
    }
    __syncthreads();
    prefix = (prefix << bits) | (uint32_t)pick_digit<1024>(hist, wave_sums, found, want);
    __syncthreads();                                       // all three are used again
    bits = shift == 21 ? 11 : shift == 10 ? 10 : 0;
    shift = shift == 21 ? 10 : 0;
  }
  int equal_before = 0, holes_before = 0, movers_before = 0;
  for (int j0 = 0; j0 < L; j0 += 4096) {                   // 4 slots in a row per thread
    uint32_t o[4];
    bool in[4], guarded[4];
    int equal = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = j0 + 4 * tid + e;
      in[e] = j < L;
      o[e] = in[e] ? weight_order(w[j]) : 0;
      guarded[e] = in[e] && is_guarded(j);
      equal += in[e] && guarded[e] == guards && o[e] == prefix;
    }
    int rank = equal_before + block_scan<1024>(equal, wave_sums, total);
    equal_before += total;
    bool leaves[4];
    int mine = 0;                                          // holes in the low half, movers in the high half
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = j0 + 4 * tid + e;
      const bool same = guarded[e] == guards;
      leaves[e] = in[e] && (same ? o[e] < prefix || (o[e] == prefix && rank < want) : guards);
      rank += in[e] && same && o[e] == prefix;
      if (in[e]) mine += j < keep ? (leaves[e] ? 1 : 0) : (leaves[e] ? 0 : 1 << 16);
    }
    int at = block_scan<1024>(mine, wave_sums, total);
    int hole = holes_before + (at & 0xffff), mover = movers_before + (at >> 16);
    holes_before += total & 0xffff;
    movers_before += total >> 16;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = j0 + 4 * tid + e;
      if (!in[e]) continue;
      if (j < keep) {
        if (leaves[e]) holes[hole++] = j;
        else {
          if (a.weight_out != a.weight) a.weight_out[head * a.C + j] = w[j];
          if (pos && a.pos_out != a.pos) a.pos_out[head * a.C + j] = pos[j];
        }
      } else if (!leaves[e]) {
        movers[mover++] = j;
      }
    }
  }
  if (tid == 0) *count = holes_before;
}

// The same for caches of up to NT E slots, which are read once: a thread holds the weights' order of E slots in a row, turned round through LDS, and
// E bits for what may leave.  The lists are those of the kernel above; with MOVE the workgroup moves its rows itself, U at a time, and writes none.
template <int NT, int E> struct EvictLds {
  static constexpr int kOffGuard = NT * E * 4, kOffHist = kOffGuard + NT * E / 8, kOffSums = kOffHist + 3 * 2048 * 4, kBytes = kOffSums + 7 * 16 * 4;
};
template <int NT, int E, bool MOVE, typename U>
__global__ __launch_bounds__(NT) void evict_select_held_kernel(EvictArgs a) {
  using Lds = EvictLds<NT, E>;
  static_assert(E >= 4 && E <= 32 && (E & (E - 1)) == 0, "whole 16-byte pieces, a bit each");
  extern __shared__ __align__(16) unsigned char evict_smem[];
  uint32_t* const order = (uint32_t*)evict_smem;
  uint32_t* const guard = (uint32_t*)(evict_smem + Lds::kOffGuard);
  int* const hist = (int*)(evict_smem + Lds::kOffHist);
  int* const wave_sums = (int*)(evict_smem + Lds::kOffSums);
  int* const found = wave_sums + 6 * 16;
  const int tid = threadIdx.x, lane = tid % kWave;
  const long head = blockIdx.x, mb = blockIdx.x / a.kv;
  const int L = clamp_len(a.len[mb], a.C), keep = min(L, a.budget), n = L - keep;
  const long long bound = (long long)(a.start ? a.start[mb] : L) - a.recent;     // guarded from this position on
  const float* w = a.weight + head * a.C;
  const int* pos = a.pos ? a.pos + head * a.C : nullptr;
  float* const w_out = a.weight_out != a.weight ? a.weight_out + head * a.C : nullptr;
  int* const p_out = pos && a.pos_out != a.pos ? a.pos_out + head * a.C : nullptr;
  int* const count = a.ws + head * (1 + 2 * (long)a.most);
  int* const holes = count + 1;
  int* const movers = holes + a.most;
  for (int d = tid; d < 3 * 2048; d += NT) hist[d] = 0;
  // piece c of thread t's E slots lies at piece c ^ (t mod E / 4): reads by owner then spread over the banks
#pragma unroll 16
  for (int i = 0; i < E; ++i) {
    const int j = i * NT + tid, there = min(j, max(L - 1, 0));
    const float x = w[there];
    const int p = pos ? pos[there] : 0;
    const int owner = j / E, e = j % E;
    order[owner * E + ((e / 4) ^ (owner & (E / 4 - 1))) * 4 + e % 4] = weight_order(x);
    const uint64_t g = __ballot(a.recent > 0 && (long long)p >= bound);
    if (lane == 0) *reinterpret_cast<uint64_t*>(guard + j / 32) = g;
    if (j < keep) {                                        // slots that another entry moves into are written again by the next kernel
      if (w_out) w_out[j] = x;
      if (p_out) p_out[j] = p;
    }
  }
  if (n == 0) {                                            // uniform
    if (!MOVE && tid == 0) *count = 0;
    return;
  }
  __syncthreads();
  uint32_t o[E];
#pragma unroll
  for (int c = 0; c < E / 4; ++c) {
    const uint4 v = *reinterpret_cast<const uint4*>(order + tid * E + (c ^ (tid & (E / 4 - 1))) * 4);
    o[4 * c] = v.x;
    o[4 * c + 1] = v.y;
    o[4 * c + 2] = v.z;
    o[4 * c + 3] = v.w;
  }
  const int j0 = tid * E, mine = min(max(L - j0, 0), E);   // entries of this thread
  const uint32_t in = mine == 32 ? ~0u : (1u << mine) - 1;
  const uint32_t guarded = (guard[j0 / 32] >> (j0 % 32)) & in;
  int open, total;
  block_sum<NT>(__popc(in & ~guarded), wave_sums, open);
  const bool guards = n > open;                            // all the others leave and some guarded entries too
  int want = guards ? n - open : n;
  const uint32_t may = guards ? guarded : in & ~guarded;
  uint32_t prefix = 0;
#pragma unroll
  for (int round = 0; round < 3; ++round) {
    const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bits = round == 2 ? 10 : 11;
    int* const h = hist + round * 2048;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (((may >> e) & 1) && (round == 0 || (o[e] >> (shift + bits) % 32) == prefix)) atomicAdd(&h[(o[e] >> shift) & ((1u << bits) - 1)], 1);
    __syncthreads();
    prefix = (prefix << bits) | (uint32_t)pick_digit<NT>(h, wave_sums + 16 * (1 + round), found + 2 * round, want);
  }
  uint32_t less = 0, equal = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    less |= (o[e] < prefix ? 1u : 0u) << e;
    equal |= (o[e] == prefix ? 1u : 0u) << e;
  }
  equal &= may;
  int rank = block_sum<NT>(__popc(equal), wave_sums + 16 * 4, total);
  uint32_t leaves = (less & may) | (guards ? in & ~guarded : 0u);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const uint32_t bit = equal & (1u << e);
    leaves |= rank < want ? bit : 0u;
    rank += bit != 0;
  }
  const int below = min(max(keep - j0, 0), E);             // slots of this thread below the budget
  const uint32_t low = below == 32 ? ~0u : (1u << below) - 1;
  uint32_t hole_bits = leaves & low, mover_bits = in & ~leaves & ~low;
  const int at = block_sum<NT>(__popc(hole_bits) | __popc(mover_bits) << 16, wave_sums + 16 * 5, total);  // at most 2^14 of each
  const int pairs = total & 0xffff;
  int* const list = (int*)order;                           // every thread has its own by now: holes, then movers, NT E / 2 at most each
  int hole = at & 0xffff, mover = NT * E / 2 + (at >> 16);
  for (; hole_bits; hole_bits &= hole_bits - 1) list[hole++] = j0 + __builtin_ctz(hole_bits);
  for (; mover_bits; mover_bits &= mover_bits - 1) list[mover++] = j0 + __builtin_ctz(mover_bits);
  __syncthreads();
  if constexpr (MOVE) {
    U* const Kh = (U*)a.Kc + head * a.C * a.units;
    U* const Vh = (U*)a.Vc + head * a.C * a.units;
#pragma unroll 4
    for (int c = tid; c < pairs * a.units; c += NT) {
      const int i = c / a.units, u = c - i * a.units;
      const long to = (long)list[i] * a.units + u, from = (long)list[NT * E / 2 + i] * a.units + u;
      const U k = Kh[from], v = Vh[from];
      Kh[to] = k;
      Vh[to] = v;
    }
    for (int i = tid; i < pairs; i += NT) {
      const int to = list[i], from = list[NT * E / 2 + i];
      a.weight_out[head * a.C + to] = w[from];
      if (pos) a.pos_out[head * a.C + to] = pos[from];
    }
  } else {
    for (int i = tid; i < pairs; i += NT) {
      holes[i] = list[i];
      movers[i] = list[NT * E / 2 + i];
    }
    if (tid == 0) *count = pairs;
  }
}

// The pairs of the lists: rows of keys and values, position and weight.  Sources lie at or above the budget, targets below it, each once.  Lists are bounded where they
// are read: a workspace that another call writes at the same time gives wrong entries, no address outside the cache.
template <typename U>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a, int rows, int blocks_per_head) {
  const long head = blockIdx.x / blocks_per_head;
  const int* count = a.ws + head * (1 + 2 * (long)a.most);
  const int* holes = count + 1;
  const int* movers = holes + a.most;
  const int i0 = (int)(blockIdx.x % blocks_per_head) * rows, end = min(i0 + rows, clamp_len(*count, a.most));
  U* Kh = (U*)a.Kc + head * a.C * a.units;
  U* Vh = (U*)a.Vc + head * a.C * a.units;
  for (int i = i0 + (int)threadIdx.x / a.units, u = (int)threadIdx.x % a.units; i < end;) {
    const long to = clamp_len(holes[i], a.C - 1), from = clamp_len(movers[i], a.C - 1);
    Kh[to * a.units + u] = Kh[from * a.units + u];
    Vh[to * a.units + u] = Vh[from * a.units + u];
    if (u == 0) {
      a.weight_out[head * a.C + to] = a.weight[head * a.C + from];
      if (a.pos) a.pos_out[head * a.C + to] = a.pos[head * a.C + from];
    }
    u += 256;
    i += u / a.units;
    u %= a.units;
  }
}

}  // namespace nf
