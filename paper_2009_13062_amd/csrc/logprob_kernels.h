// Merged decoders: log probabilities of given tokens, the entropy of each row and its most likely tokens, in one pass over the logits.
//
//   x_j = f(scale * logit_j), j < V_m;   log p_t = x_t - top - log S,  S = sum exp(x_j - top);   entropy = log S - sum (x_j - top) exp(x_j - top) / S
//
// Both terms of the entropy are positive, and top + log S is never formed, so nothing is lost to large logits.  f grows with its argument and scale is positive, so the order of
// the logits is that of the probabilities, and it is taken from the logits as they are stored: no two that differ become equal.
//
// A wavefront takes some chunks of a row, one after the other, each lane 16 bytes at a time of it, and keeps a chunk in registers.  Each chunk leaves sums of its own, whose join follows from V
// alone, and alternatives are exact, so a row's bits depend neither on the other rows nor on how many chunks a wavefront takes.
//
// Bound by the reads in float32 (4084 rows of 50001, 20 alternatives: 147 us with the join's 7, 818 MB at 5.7 TB/s), by vector instructions in bfloat16 (832 rows of up to 131071 under a cap, 8
// alternatives: 58 us with the join's 5, vector units full), a few rows by two launches (8 of 32000: 10.4 us).
#pragma once
#include "decoder.h"
#include "decoder_tiles.h"

namespace nf {

// 16 bytes of logits, from any element on; they are read once, and past the caches that is faster (4084 rows of 50001 in float32 164 -> 143 us).
typedef uint32_t words_t __attribute__((ext_vector_type(4), aligned(2)));
template <class T> __device__ __forceinline__ uint4 load_once(const T* p) {
  const words_t v = __builtin_nontemporal_load((const words_t*)p);
  return make_uint4(v.x, v.y, v.z, v.w);
}

constexpr int kMostAlternatives = 32;

struct LogprobArgs {
  const void* logits; const int* token; const int* vocab; const int* nodes;
  float* logp; float* entropy; int* top; float* top_logp; float* ws;
  int M, B, T, V, n, k, chunks, groups;                    // chunks and wavefronts of a row
  long stride_m, stride_row;
  float scale, cap, inv_cap;
};

// A logit in the order of its value, lower ones first, -0 as 0; 0 for what is no alternative: -infinity and NaN.
__device__ __forceinline__ uint32_t logit_order(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return v > -INFINITY ? (u & 0x80000000u ? ~u : u | 0x80000000u) : 0u;
}
__device__ __forceinline__ float logit_of(uint32_t order) { return order == 0u ? -INFINITY : __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order); }

constexpr uint32_t kLowestOrder = 0x00800000u;             // of the lowest finite number: what lies below is no candidate

// x of a logit under a cap, in units of log2 (tanh within 2^-20).  One factor after the other: scale / cap itself may be infinite, which would make a logit of 0 NaN, or 0.
// The product is rounded, never one with the difference that it goes into: equal logits have equal x, and the largest's difference to itself is 0.
__device__ __forceinline__ float capped_logit(float v, const LogprobArgs& a) {
#pragma clang fp contract(off)
  return tanh_either(v * a.scale * a.inv_cap) * (a.cap * kLog2e);
}
// x - x(top), in units of log2 or natural ones.  Without a cap the difference comes first: the types' lowest values, which stand for masks, do not leave float32; natural ones, which are results, of the
// halves: the same bits, and from the lowest to the largest value the difference is one too (as a power of 2 it is 0 in either form).  With one it is never above 0, as
// by tanh's error, which grows with the cap, it could be.
__device__ __forceinline__ float below_top(float x) { return x > 0.f ? 0.f : x; }          // NaN stays
struct FromTop {
  float top, most;
  __device__ __forceinline__ FromTop(float t, const LogprobArgs& a) : top(t), most(a.cap != 0.f ? capped_logit(t, a) : 0.f) {}
  __device__ __forceinline__ float operator()(float v, const LogprobArgs& a) const { return a.cap != 0.f ? below_top(capped_logit(v, a) - most) : (v - top) * (a.scale * kLog2e); }
  __device__ __forceinline__ float natural(float v, const LogprobArgs& a) const { return a.cap != 0.f ? below_top(capped_logit(v, a) - most) * kLn2 : (0.5f * v - 0.5f * top) * (2.f * a.scale); }
};

// Candidates of a wavefront: of 32 alternatives a list of 64 holds what two chunks of random logits bring less often than not
constexpr int kLogprobList = 2 * kWave;
constexpr int kFewLanes = 16, kSlack = 8;                  // lanes that reach the border for which a higher one is not looked for; candidates past k that the list may keep
// Logits of a chunk, by their size and number, as a row's bits may follow from V but not from how many rows there are.  bfloat16, 8 alternatives, us with chunks of 4096 / 2048: 8 rows of 32000 (5
// alternatives) 11.8 / 10.2; of 65537 8 rows 12.8 / 11.8, 128 16.7 / 15.5, 832 37 / 40; of 131071 8 rows 14.8 / 13.3, 32 15.1 / 14.2, 128 21.6 / 23.2, 832 60 / 64; of 131072 12.9 / 12.4, 12.8 / 13.1,
// 16.6 / 20.1, 53 / 61; of 151936 13.5 / 13.6, 14.4 / 15.2, 19.8 / 23.2, 61 / 68: above 65536 many rows gain more than few ones lose.
__host__ __device__ constexpr int logprob_chunk(size_t bytes, int V) { return bytes == 2 && V > 65536 ? 4096 : 2048; }

// The workspace: four numbers of each chunk -- its largest logit and the two sums at it (of 1 and of x - top, that in units of log2) -- then k pairs (order, token) of each wavefront, the
// most likely first.
constexpr int kChunkWords = 4;

// An alternative as one number: the larger order wins, then the lower token.
__device__ __forceinline__ uint64_t alternative(uint32_t order, int token) { return (uint64_t)order << 32 | (uint32_t)~token; }

// An order that at least k lanes' own best ones reach, and few others of a wavefront's do: the k-th largest of the 64, its upper BITS bits found one by one with ballots.
template <int BITS> __device__ __forceinline__ uint32_t few_above(uint32_t best, int k) {
  uint32_t found = 0;
#pragma unroll
  for (int bit = BITS - 1; bit >= 0; --bit) {
    const uint32_t trial = found | 1u << bit;
    if (__popcll(__ballot(best >> (32 - BITS) >= trial)) >= k) found = trial;    // uniform
  }
  return max(found << (32 - BITS), kLowestOrder);
}
// A lane's candidates go into the list, which holds kList; `count` goes on past that.
template <class What> __device__ __forceinline__ void list_if(bool in, uint64_t* list, int& count, What&& what) {
  const uint64_t who = __ballot(in);
  if (who == 0) return;                                    // uniform
  const int at = count + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
  if (in && at < kLogprobList) list[at] = what();
  count += __popcll(who);
}
// The list's place r for r < k: lane i ranks candidates i and i + 64 among all.  put(r, alternative), 0 where there are fewer.
template <class Put> __device__ __forceinline__ void rank_list(const uint64_t* list, int count, int k, Put&& put) {
  const int lane = threadIdx.x % kWave;
  __builtin_amdgcn_wave_barrier();
  const uint64_t mine = lane < count ? list[lane] : 0;
  int rank = 0;
  if (count <= kWave) {                                    // uniform
    for (int i = 0; i < count; ++i) rank += list[i] > mine;
  } else {
    const uint64_t more = lane + kWave < count ? list[lane + kWave] : 0;
    int rank_more = 0;
    for (int i = 0; i < count; ++i) {
      const uint64_t x = list[i];
      rank += x > mine;
      rank_more += x > more;
    }
    if (lane + kWave < count && rank_more < k) put(rank_more, more);
  }
  if (lane < count && rank < k) put(rank, mine);
  if (lane >= count && lane < k) put(lane, (uint64_t)0);
  __builtin_amdgcn_wave_barrier();
}

template <typename T> struct Logits;                       // 16 bytes of them
template <> struct Logits<float> {
  static constexpr int kN = 4;
  using Bits = uint32_t;
  __device__ static __forceinline__ float at(const uint4& w, int e) { return __uint_as_float(e == 0 ? w.x : e == 1 ? w.y : e == 2 ? w.z : w.w); }
  static constexpr uint32_t kNone = 0xff800000u;           // -infinity
};
template <> struct Logits<bf16_t> {
  static constexpr int kN = 8;
  using Bits = uint16_t;
  __device__ static __forceinline__ float at(const uint4& w, int e) {
    const uint32_t x = e < 2 ? w.x : e < 4 ? w.y : e < 6 ? w.z : w.w;
    return __uint_as_float(e % 2 ? x & 0xffff0000u : x << 16);
  }
  static constexpr uint32_t kNone = 0xff80ff80u;
};

// The largest of three, and of the sizes of the last two, in one instruction (from the function the compiler first quiets each operand: twice the instructions of a chunk's maximum).  A
// signalling NaN may come out as NaN.
__device__ __forceinline__ float largest(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ float largest_size(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, |%2|, |%3|" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// tanh(u) / u on u^2: minimax fits of the relative error up to kTanhNear and kTanhWide (tanh_fit.py; 2^-24, with float32's roundings 2^-22); used for caps up to kCapPlain
constexpr float kTanhNear = 0.35f, kTanhWide = 0.8f, kCapPlain = 0x1p19f;
constexpr float kTanhNearFit[4] = {0.9999999403953552f, -0.33332422375679016f, 0.13295799493789673f, -0.04895823076367378f};
constexpr float kTanhWideFit[6] = {0.9999999403953552f, -0.3333267569541931f, 0.13321048021316528f, -0.05311431363224983f, 0.01909330114722252f, -0.004355299286544323f};

// Four wavefronts per SIMD in float32, which is bound by the reads (143 us of the rows above, 5.7 TB/s; 5 of them 143, 6 160), five in bfloat16, which is bound by vector instructions: for
// each logit 9.6 counted, with a cap 15.4, 4.3 more for 8 alternatives and 7.8 for 20 (8.3, 14.2, 4.8 and 8.9 in float32), an exponential of a quarter of their rate among them
// (832 rows of 131072, 8 alternatives, us: 3 wavefronts 56, under a cap 69, 4 53 and 61, 5 52 and 61, 6 51 and 59; rows of 131071, which begin at odd elements, 58 and 67 with 5).
template <typename T, bool CAP, int kChunk>
__global__ __launch_bounds__(256, sizeof(T) == 4 ? 4 : 5) void logprob_chunks_kernel(LogprobArgs a) {
  using L = Logits<T>;
  constexpr int P = L::kN, N = kChunk / kWave / P;
  __shared__ uint64_t lists[4][kLogprobList];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const unsigned wid = blockIdx.x * 4 + wave, row = wid / a.groups;              // fewer than 2^26 and 2^31
  if (row >= (unsigned)(a.M * a.B) * (unsigned)a.T) return;                      // uniform per wavefront, as the next ones
  const int group = (int)(wid - row * a.groups);
  const unsigned mb = row / a.T, m = mb / a.B;
  const int t = (int)(row - mb * a.T);
  const int V = a.vocab ? clamp_len(a.vocab[m], a.V) : a.V;
  const int chunks = (V + kChunk - 1) / kChunk;           // this wavefront's are every a.groups-th, so that neighbours read what lies together
  if (group >= chunks || (a.nodes && t >= a.nodes[mb])) return;
  const T* const logits = (const T*)a.logits + m * a.stride_m + (long)(row - m * a.B * a.T) * a.stride_row;
  // 16 bytes of each lane, -infinity where the row has ended; whether a piece is whole for all of them is the same for all of them
  auto piece = [&](const T* p, int left, int i) -> uint4 {
    const int j = (i * kWave + lane) * P;
    if ((i + 1) * kWave * P <= left) return load_once(p + j);
    uint32_t x[4] = {L::kNone, L::kNone, L::kNone, L::kNone};
    if (i * kWave * P < left) {
      uint32_t v[P];
#pragma unroll
      for (int e = 0; e < P; ++e) v[e] = __builtin_bit_cast(typename L::Bits, p[min(j + e, left - 1)]);
#pragma unroll
      for (int e = 0; e < P; ++e) {
        v[e] = j + e < left ? v[e] : L::kNone >> (32 - 8 * sizeof(T));
        if constexpr (P == 4) x[e] = v[e];
        else x[e / 2] = e % 2 ? x[e / 2] | v[e] << 16 : v[e];
      }
    }
    return make_uint4(x[0], x[1], x[2], x[3]);
  };
  uint4 w[N];
  // The logits stay as they came: each pass opens them again.  (Left to itself the compiler keeps what it made of them in the pass before, all 64 of it.)
  auto as_they_came = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(w[i].x), "+v"(w[i].y), "+v"(w[i].z), "+v"(w[i].w));
  };
  uint64_t* const list = lists[wave];
  int count = 0;                                           // candidates in the list
  uint32_t border = kLowestOrder;                          // the order that one of this wavefront's has to have
  for (int chunk = group; chunk < chunks; chunk += a.groups) {
    const int base = chunk * kChunk, left = V - base;
    const T* const p = logits + base;
    int at_lane = lane;                                    // made new for every chunk: the 64 token numbers of a lane would be kept in a register each
    asm volatile("" : "+v"(at_lane));
    if (left >= kChunk) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = load_once(p + (i * kWave + at_lane) * P);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        w[i] = piece(p, left, i);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    float piece_top[N], mine = -INFINITY, reach = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      piece_top[i] = -INFINITY;
#pragma unroll
      for (int e = 0; e < P; e += 2) {
        const float x = L::at(w[i], e), y = L::at(w[i], e + 1);
        piece_top[i] = largest(piece_top[i], x, y);
        if (CAP) reach = largest_size(reach, x, y);
      }
      mine = fmaxf(mine, piece_top[i]);
      __builtin_amdgcn_sched_barrier(0);
    }
    float top = wave_max(mine);
    as_they_came();
    float sum = 0.f, first = 0.f;
    bool plain = !CAP;                                       // each x from one polynomial of its logit
    const float x1 = a.scale * kLog2e;
    auto add = [&](float x) __attribute__((always_inline)) {
      const float e = __builtin_amdgcn_exp2f(x);
      sum += e;
      first = fmaf(e, x, first);
    };
    // One piece's numbers at a time, the sum's too (which could wait, all terms of it in registers, for a path that uses it): more would take registers from other wavefronts
    auto added = [&]() __attribute__((always_inline)) {
      asm volatile("" : "+v"(sum), "+v"(first));
      __builtin_amdgcn_sched_barrier(0);
    };
    if constexpr (!CAP) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int e = 0; e < P; ++e) add((L::at(w[i], e) - top) * x1);
        added();
      }
    } else {
      const float u1 = a.scale * a.inv_cap, u2 = u1 * u1;
      reach = wave_max(reach) * u1;
      // The largest logit's x from the same polynomial as the others': within 2^-22 of a cap up to kCapPlain no x lies far above it
      auto all_by = [&](auto&& tanh_of) __attribute__((always_inline)) {
        plain = true;
        const float most = top * tanh_of(top * top);
#pragma unroll
        for (int i = 0; i < N; ++i) {
#pragma unroll
          for (int e = 0; e < P; ++e) {
            const float v = L::at(w[i], e);
            add(fmaf(v, tanh_of(v * v), -most));
          }
          added();
        }
      };
      // Coefficients of the logit itself, whose powers of scale / cap are in them: they run evenly from c0, which is a normal number, to the last one, so that one says whether all of them are
      auto held = [](float last) { return fabsf(last) >= 0x1p-126f && fabsf(last) < INFINITY; };
      const bool exact = a.cap > kCapPlain;                  // each by the form that the join takes too
      if (!exact && reach <= kTanhNear) {
        constexpr auto& k = kTanhNearFit;
        const float c0 = x1 * k[0], c1 = x1 * u2 * k[1], c2 = x1 * u2 * u2 * k[2], c3 = x1 * u2 * u2 * u2 * k[3];
        if (held(c3)) all_by([&](float q) __attribute__((always_inline)) { return fmaf(fmaf(fmaf(c3, q, c2), q, c1), q, c0); });
      } else if (!exact && reach <= kTanhWide) {
        constexpr auto& k = kTanhWideFit;
        const float c0 = x1 * k[0], c1 = x1 * u2 * k[1], c2 = x1 * u2 * u2 * k[2], c3 = x1 * u2 * u2 * u2 * k[3], c4 = x1 * u2 * u2 * u2 * u2 * k[4], c5 = x1 * u2 * u2 * u2 * u2 * u2 * k[5];
        if (held(c5)) all_by([&](float q) __attribute__((always_inline)) { return fmaf(fmaf(fmaf(fmaf(fmaf(c5, q, c4), q, c3), q, c2), q, c1), q, c0); });
      }
    }
    const bool careful = !plain || __any(first != first);
    if (careful) {                                           // logits of -infinity (0 times it), NaN, or under a cap large ones: with more care
      as_they_came();
      mine = -INFINITY;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        piece_top[i] = -INFINITY;
#pragma unroll
        for (int e = 0; e < P; ++e) piece_top[i] = fmaxf(piece_top[i], L::at(w[i], e));        // whatever kind of NaN there is
        mine = fmaxf(mine, piece_top[i]);
        __builtin_amdgcn_sched_barrier(0);
      }
      top = wave_max(mine);
      const FromTop from_top(top, a);
      sum = first = 0.f;
      as_they_came();
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const float y = L::at(w[i], e), x = CAP ? below_top(capped_logit(y, a) - from_top.most) : (y - top) * x1, f = y == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x);
          sum += f;
          first += f != 0.f ? x * f : 0.f;
          if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);                     // more of them at a time would take registers from every chunk
        }
    }
    sum = wave_sum(sum);
    first = wave_sum(first);
    if (CAP && !careful) sum = fmaxf(sum, 1.f);              // the largest logit's own term, up to a rounding
    if (lane == 0) *reinterpret_cast<float4*>(a.ws + ((long)row * a.chunks + chunk) * kChunkWords) = make_float4(top, sum, first, 0.f);

    // ---- alternatives: what reaches the border joins the list, which is cut back to the best k when it has grown
    const uint64_t hot = __ballot(mine >= logit_of(border));
    if (a.k == 0 || hot == 0) continue;                    // uniform
    uint32_t from = border;
    if (__popcll(hot) > kFewLanes) from = max(from, few_above<16>(logit_order(mine), a.k));
    const int before = count;
    bool all_of = true;                                    // of the border's equals too
    for (;;) {
      as_they_came();
      asm volatile("" : "+v"(at_lane));
      const float least = logit_of(from + !all_of);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (!__any(piece_top[i] >= least)) continue;       // uniform
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const float v = L::at(w[i], e);
          list_if(v >= least, list, count, [&] { return alternative(logit_order(v), base + (i * kWave + at_lane) * P + e); });
        }
      }
      if (count <= kLogprobList || !all_of) break;
      // many alike: those above the k-th lane's best, then of its equals the first ones, k at most
      count = before;
      from = max(border, few_above<32>(logit_order(mine), a.k));
      all_of = false;
    }
    const int need = all_of ? 0 : max(a.k - (count - before), 0);
    if (count + need > kLogprobList) {
      // Many of few lanes: one of each lane at a time, and the list is cut back before it is full (2000 rows of 50001 in float32, whose logits rise, 20 alternatives: 98 us where random ones take 86;
      // the best one that is left, looked for in all of them, k times: 1470).
      count = before;
#pragma unroll 1
      for (int i = 0; i < N; ++i) {
        const uint4 v = piece(p, left, i);                 // again from memory: numbered registers would have to be there for it
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const float y = L::at(v, e);
          list_if(y >= logit_of(from), list, count, [&] { return alternative(logit_order(y), base + (i * kWave + at_lane) * P + e); });
          if (count > kLogprobList - kWave) {              // uniform
            rank_list(list, count, a.k, [&](int r, uint64_t x) { list[r] = x; });
            count = a.k;
            from = (uint32_t)(list[a.k - 1] >> 32);        // of this chunk's equals an earlier one may still come
          }
        }
      }
    } else if (need > 0) {
      const float least = logit_of(from);
      int left_over = need;
#pragma unroll 1
      for (int i = 0; i < N && left_over > 0; ++i) {
        const uint4 v = piece(p, left, i);
        int alike = 0;
#pragma unroll
        for (int e = 0; e < P; ++e) alike += L::at(v, e) == least;
        const int upto = wave_scan(alike);
        int at = upto - alike;
#pragma unroll
        for (int e = 0; e < P; ++e)
          if (L::at(v, e) == least) {
            if (at < left_over) list[count + at] = alternative(from, base + (i * kWave + at_lane) * P + e);
            ++at;
          }
        const int found = min(__shfl(upto, kWave - 1, kWave), left_over);
        count += found;
        left_over -= found;
      }
    }
    if (count >= a.k + kSlack && chunk + a.groups < chunks) {
      rank_list(list, count, a.k, [&](int r, uint64_t x) { list[r] = x; });
      count = a.k;
      border = (uint32_t)(list[a.k - 1] >> 32) + 1;        // of two alike the earlier one stays
    }
  }
  if (a.k == 0) return;
  uint2* const out = reinterpret_cast<uint2*>(a.ws + (long)a.M * a.B * a.T * a.chunks * kChunkWords) + ((long)row * a.groups + group) * a.k;
  auto put = [&](int r, uint64_t x) { out[r] = make_uint2((uint32_t)(x >> 32), ~(uint32_t)x); };
  rank_list(list, count, a.k, put);
}

// A row's chunks: one wavefront.
template <typename T>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobArgs a) {
  const int kChunk = logprob_chunk(sizeof(T), a.V);
  __shared__ uint64_t list[kLogprobList];
  const int lane = threadIdx.x;
  const unsigned row = blockIdx.x, mb = row / a.T, m = mb / a.B;
  const int t = (int)(row - mb * a.T);
  const int V = a.nodes && t >= a.nodes[mb] ? 0 : a.vocab ? clamp_len(a.vocab[m], a.V) : a.V;
  const int chunks = (V + kChunk - 1) / kChunk, groups = min(chunks, a.groups);
  const float4* const ws = reinterpret_cast<const float4*>(a.ws) + (long)row * a.chunks;
  const uint2* const lists = reinterpret_cast<const uint2*>(a.ws + (long)a.M * a.B * a.T * a.chunks * kChunkWords) + (long)row * a.groups * a.k;
  const T* const p = (const T*)a.logits + m * a.stride_m + (long)(row - m * a.B * a.T) * a.stride_row;
  // what the first lanes need, all on its way at once
  const int token0 = lane < a.n ? a.token[(long)row * a.n + lane] : -1;
  const bool known0 = token0 >= 0 && token0 < V;
  const float logit0 = known0 ? load_f32(p + token0) : -INFINITY;
  float top = -INFINITY;
  for (int c = lane; c < chunks; c += kWave) top = fmaxf(top, ws[c].x);
  top = wave_max(top);
  const FromTop from_top(top, a);
  float sum = 0.f, first = 0.f;
  for (int c = lane; c < chunks; c += kWave) {
    const float4 w = ws[c];
    const float x = from_top(w.x, a), f = __builtin_amdgcn_exp2f(x);
    if (w.y != 0.f) {                                      // a chunk of -infinity alone adds nothing
      sum = fmaf(w.y, f, sum);
      first += f != 0.f ? f * fmaf(x, w.y, w.z) : 0.f;
    }
  }
  sum = wave_sum(sum);
  first = wave_sum(first);
  const bool none = sum == 0.f;
  const float log_sum = none ? 0.f : __builtin_amdgcn_logf(sum);
  if (lane == 0) a.entropy[row] = none ? 0.f : (log_sum - first / sum) * kLn2;
  auto logp_of = [&](float v) { return none || v == -INFINITY ? -INFINITY : from_top.natural(v, a) - log_sum * kLn2; };
  if (lane < a.n) a.logp[(long)row * a.n + lane] = logp_of(logit0);
  for (int i = lane + kWave; i < a.n; i += kWave) {
    const int j = a.token[(long)row * a.n + i];
    a.logp[(long)row * a.n + i] = logp_of(j >= 0 && j < V ? load_f32(p + j) : -INFINITY);
  }
  if (a.k == 0) return;

  // The same choice among the wavefronts' alternatives, everyone's first ones first.
  const int all = groups * a.k;
  auto candidate = [&](int j) {
    const int place = (int)((unsigned)j / (unsigned)groups), i = (j - place * groups) * a.k + place;
    return alternative(lists[i].x, (int)lists[i].y);
  };
  auto put = [&](int r, uint64_t x) {
    const uint32_t order = (uint32_t)(x >> 32);
    a.top[(long)row * a.k + r] = order ? (int)~(uint32_t)x : -1;
    a.top_logp[(long)row * a.k + r] = order ? logp_of(logit_of(order)) : -INFINITY;
  };
  uint64_t mine = 0;
  for (int i = lane; i < all; i += kWave) {
    const uint64_t x = candidate(i);
    mine = x > mine ? x : mine;
  }
  uint32_t border = few_above<16>((uint32_t)(mine >> 32), a.k);
  int count = 0;
  for (int i0 = 0; i0 < all; i0 += kWave) {
    const uint64_t x = i0 + lane < all ? candidate(i0 + lane) : 0;
    list_if((uint32_t)(x >> 32) >= border, list, count, [&] { return x; });
    if (count > kLogprobList - kWave && i0 + kWave < all) {                      // uniform
      rank_list(list, count, a.k, [&](int r, uint64_t y) { list[r] = y; });
      count = a.k;
      border = (uint32_t)(list[a.k - 1] >> 32);            // an equal one of a lower token may still come
    }
  }
  rank_list(list, count, a.k, put);
}

}  // namespace nf
