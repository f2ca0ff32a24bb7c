// Merged decoders, attention without LDS stages: every wavefront streams its keys and values from memory into the operands of the matrix
// instructions.  float32 (v_mfma_f32_16x16x4_f32) for all rows, bfloat16 (v_mfma_f32_16x16x32_bf16) for the few rows of single tokens and small
// trees.  Head sizes up to D in 16-byte pieces.
//
// Bound by the cache's bytes where few rows read it (one token over two caches of up to 100003 entries, 8 key heads of 128: 114 us and 6 to join, 5.2 TB/s; a read alone reaches
// 7.1), by latency in short calls (one token over 8 caches of up to 1024, 12 heads of 64, float32: 14 us and 4 to join: four steps per wavefront, one after the other).  float32 prompts and
// trees of many rows read their keys and values again for every 16 or 32 rows, beside the matrix instructions: 4 models of 1024 tokens, 16 heads of 128, 264 us, 65 TFLOP/s of the 152 that
// a library product reaches, 2.4 GB from the second cache at 9 TB/s, matrix units busy 50 %, 37 % of the wavefronts' time waits; 12 tokens of groups of 4 over 16 caches of 4096, 8 key
// heads, 181 us and 8 to join, 66 % and 12 %; 26 tokens 350 and 10, 66 % and 10 %.  Three wavefronts per SIMD, two where a wavefront has 32 rows, one with all its registers
// above 128 features (float32, 16 caches of 4096, 2 heads of 256: two spill, 95 us; one 54).
//
// A wavefront holds 16 RT rows (row r = token r / group of one key head) and takes a step of 16 NK keys.  Scores are computed transposed, S^T = K Q^T,
// on 64-byte slices of the rows: lane (l16, g) loads bytes 16 g .. + 15 of a slice of key l16, one instruction's k of bfloat16, four instructions'
// of float32 (element t of the piece in instruction t), so a load covers 64 bytes of each of 16 rows.  A lane then has keys 4 g + r of ONE
// row (l16), which is the B operand of O^T = V^T P^T already: group g of float32 instruction t meets key 4 g + t, of a bfloat16 one the keys 4 g .. + 3 of
// two blocks.  V^T block i is features VF l + i (l = 0 .. 15), so a lane loads VF neighbouring features of a key, a whole row of 64 .. 256 bytes per 16
// lanes, and a bfloat16 block is put together from the 8 keys of a lane by byte permutes.  Nothing is read twice and nothing waits for another
// wavefront; K of the next step is in flight while V of this one is used.
//
// float32: scores in natural units, expf and tanhf, weights unrounded.  bfloat16: log2 units, weights in two bfloat16 parts that hold 15 bits, each a product of
// its own (the loads hide it: two caches of up to 100003 entries 120.4 us with one part, 120.6 with two; 2 % at most, where caches are short).
// Masks, chunks of a cache and workspace as in decoder_tiles.h.
#pragma once
#include "decoder.h"
#include "decoder_tiles.h"

namespace nf {

template <typename T, int D> struct StreamShape {
  static constexpr bool kBf = sizeof(T) == 2;
  static constexpr int kSliceF = 64 / (int)sizeof(T);      // features of a 64-byte slice
  static constexpr int kSlices = D / kSliceF;
  static constexpr int kPiece = 16 / (int)sizeof(T);       // features of 16 bytes
  static constexpr int NK = (kBf ? 2 : 1) * (D == 64 ? 2 : 1);            // 16-key blocks of a step: 64 registers of keys and values in flight, 128 for D = 256
  static constexpr int NB = D / 16;                        // 16-feature blocks of the output
  static constexpr int VF = NB < kPiece ? NB : kPiece;     // neighbouring features per lane and load
  static constexpr int VC = NB / VF;
  static constexpr int kVWords = VF * (int)sizeof(T) / 4;
};

constexpr int stream_lds_bytes(int RT, int KS, int NB) { return KS > 1 ? (256 * RT * 4 * NB + 2 * RT * 256) * 4 : 0; }

template <int W> struct Words { uint32_t w[W]; };

// a . b^T over a 64-byte slice, accumulated: 16 rows of a (lane % 16) by 16 rows of b
template <typename T> __device__ __forceinline__ f32x4_t slice_product(const uint4& a, const uint4& b, f32x4_t c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  } else {
    const f32x4_t x = __builtin_bit_cast(f32x4_t, a), y = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
    for (int t = 0; t < 4; ++t) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[t], y[t], c, 0, 0, 0);
    return c;
  }
}

template <typename T, int D, int RT, int KS, bool TREE>
__global__ __launch_bounds__(256, D > 128 ? 1 : RT == 1 ? 3 : 2) void decoder_stream_kernel(DecArgs a, int row_blocks, int splits, int chunk) {
  using Sh = StreamShape<T, D>;
  constexpr bool kBf = Sh::kBf;
  constexpr int NK = Sh::NK, NB = Sh::NB, VF = Sh::VF, VC = Sh::VC, SL = Sh::kSlices, kStep = 16 * NK, RG = 4 / KS;
  constexpr int kRows = RG * RT * 16;                      // per workgroup
  // A cache that one workgroup's rows are all of is read once: its values go past the caches (two of 100003 keys 131 -> 122 us; keys, whose 128-byte lines take
  // two loads, do not: one token over 8192 110 -> 119).
  constexpr int kOnce = TREE && KS > 1 ? 2 : 0;
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int g4 = lane / 16, l16 = lane % 16, rg = wave % RG, share = wave / RG;

  unsigned id = xcd_remap(blockIdx.x, gridDim.x);
  int split = 0, rblock;
  if (TREE) {
    split = id % splits;  id /= splits;
    rblock = id % row_blocks;
  } else {
    rblock = row_blocks - 1 - (int)(id % row_blocks);      // the longest rows of a head first
  }
  // (m, b, g): divisions in 32 bits, a long one takes a hundred instructions
  const unsigned uhead = id / row_blocks, umb = uhead / a.kv;
  const int g = (int)(uhead % a.kv), b = (int)(umb % a.B);
  const long head = uhead, mb = umb, m = umb / a.B;
  const int group = a.heads / a.kv, R = a.N * group, r0 = rblock * kRows;
  const int L = TREE ? clamp_len(a.len[mb], a.C) : a.len ? clamp_len(a.len[mb], a.N) : a.N;
  const int parts = TREE ? max(1, (L + chunk - 1) / chunk) : 1;
  if (split >= parts) return;                              // uniform
  const int there = TREE && a.nodes ? clamp_len(a.nodes[mb], a.N) : a.N;
  const int first = !TREE && a.prefix ? clamp_len(a.prefix[mb], L) : 0;
  const int* doc = !TREE && a.doc ? a.doc + mb * a.N : nullptr;
  const bool biased = a.slope != nullptr, capped_scores = a.cap != 0.f;
  const bool keyed = TREE ? biased : doc != nullptr;       // a value per key is needed

  const T* Kp = (const T*)a.K + m * a.kv_stride_m + (long)b * a.N * a.kv_stride_row + (long)g * a.d;
  const T* Vp = (const T*)a.V + m * a.kv_stride_m + (long)b * a.N * a.kv_stride_row + (long)g * a.d;
  const T* Kh = TREE ? (const T*)a.Kc + head * a.C * a.d : Kp;
  const T* Vh = TREE ? (const T*)a.Vc + head * a.C * a.d : Vp;
  const long stride = TREE ? a.d : a.kv_stride_row;
  const float unit = kBf ? kLog2e : 1.f;

  const int w0 = r0 + rg * RT * 16;                        // first row of the wavefront
  const int w_lo = min(w0, R - 1) / group, w_hi = min(w0 + RT * 16 - 1, R - 1) / group;
  int node_at = 0, lo = 0, hi = 0;                         // position of node `lane`, documents of this wavefront's rows
  const int key_end = TREE ? min(L, (split + 1) * chunk) : w0 >= R || w_lo >= L ? 0 : a.causal ? min(max(w_hi + 1, first), L) : L;

  // ---- the steps of this wavefront: of its chunk of the cache, then of the tree; every KS-th is its own
  const int key_start = TREE ? split * chunk : 0;
  const int cached_steps = key_end > key_start ? (key_end - key_start + kStep - 1) / kStep : 0;
  const int steps = cached_steps + (TREE && split == parts - 1 ? (a.N + kStep - 1) / kStep : 0);
  constexpr int kPerBallot = kStep < kWave ? kWave / kStep : 1, kWindow = 8 * kPerBallot;
  uint32_t win_any = 0, win_all = 0;                       // of kWindow steps from win_at on: which hold a document of the rows, nothing but their only one
  int win_at = -kWindow;
  auto wanted = [&](int st) -> bool {
    if (TREE || !doc) return true;
    if (st >= win_at + kWindow) {
      win_at = st;
      win_any = win_all = 0;
#pragma unroll 4
      for (int t = 0; t < 8; ++t) {
        const int j = st * kStep + t * kWave + lane, v = doc[min(j, L - 1)];
        const uint64_t any = __ballot((j < L) & (v >= lo) & (v <= hi)), all = __ballot((j < L) & (v == lo));
#pragma unroll
        for (int u = 0; u < kPerBallot; ++u) {
          const uint64_t part = kPerBallot == 1 ? ~0ull : ((1ull << kStep % kWave) - 1) << (u * kStep) % kWave;
          win_any |= ((any & part) ? 1u : 0u) << (t * kPerBallot + u);
          win_all |= ((all & part) == part && lo == hi ? 1u : 0u) << (t * kPerBallot + u);
        }
      }
    }
    return (win_any >> (st - win_at)) & 1;
  };
  auto seek = [&](int st) -> int {
    while (st < steps && !wanted(st)) st += KS;
    return st;
  };
  auto whole = [&](int st) -> bool {                       // every row of this wavefront sees every key of the step
    if (st >= cached_steps) return false;
    const int past = key_start + (st + 1) * kStep;
    if (past > L) return false;
    if (TREE) return true;
    if (a.causal && past > w_lo + 1 && past > first) return false;
    return !doc || ((win_all >> (st - win_at)) & 1);
  };

  uint4 kreg[NK][SL];
  Words<Sh::kVWords> vreg[NK * 4][VC];
  int key_reg = 0;                                         // position or document of key `lane` of the step
  auto load_keys = [&](int st) {
    const bool own_step = TREE && st >= cached_steps;
    const int base = own_step ? (st - cached_steps) * kStep : key_start + st * kStep, limit = (own_step ? a.N : L) - base;
    const long rows = own_step ? a.kv_stride_row : stride;
    const auto rk = rows_from((own_step ? Kp : Kh) + base * rows);
    const unsigned row = (unsigned)(rows * (long)sizeof(T));
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const unsigned from = 16 * k + l16 < limit ? (16 * k + l16) * row + g4 * 16 : kDecOob;
#pragma unroll
      for (int sl = 0; sl < SL; ++sl) kreg[k][sl] = rows_load16(rk, sl * Sh::kSliceF + g4 * Sh::kPiece < a.d ? from + sl * 64 : kDecOob);
    }
    if (keyed) {
      const int there = base + min(lane, limit - 1);
      if (TREE) key_reg = a.pos && !own_step ? a.pos[head * a.C + there] : there;
      else key_reg = lane < limit ? doc[there] : -1;
    }
  };
  auto load_values = [&](int st) {
    const bool own_step = TREE && st >= cached_steps;
    const int base = own_step ? (st - cached_steps) * kStep : key_start + st * kStep, limit = (own_step ? a.N : L) - base;
    const long rows = own_step ? a.kv_stride_row : stride;
    const auto rv = rows_from((own_step ? Vp : Vh) + base * rows);
    const unsigned row = (unsigned)(rows * (long)sizeof(T));
#pragma unroll
    for (int e = 0; e < NK * 4; ++e) {
      const int key = 16 * (e / 4) + 4 * g4 + e % 4;
      const unsigned from = key < limit ? key * row + l16 * (Sh::kVWords * 4) : kDecOob;
#pragma unroll
      for (int c = 0; c < VC; ++c) {
        const unsigned off = c * 16 * VF + l16 * VF < a.d ? from + c * (64 * Sh::kVWords) : kDecOob;
        if constexpr (Sh::kVWords == 4) {
          vreg[e][c] = __builtin_bit_cast(Words<4>, rows_load16<kOnce>(rv, off));
        } else {
          const dec_u32x2_t v = __builtin_amdgcn_raw_buffer_load_b64(rv, (int)off, 0, kOnce);
          vreg[e][c] = __builtin_bit_cast(Words<Sh::kVWords>, v);
        }
      }
    }
  };

  int st = share;
  const bool early = TREE || !doc;                         // the first keys are on their way before anything else is looked up
  if (early && st < steps) load_keys(st);

  // ---- this lane's rows
  int token[RT], end[RT], mine[RT], docr[RT];
  uint64_t path[RT];
  float slope[RT];
  uint4 qf[RT][SL];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = r0 + (rg * RT + rt) * 16 + l16;
    const int i = min(r, R - 1) / group, h = g * group + (min(r, R - 1) - i * group);
    token[rt] = i;
    const T* q = (const T*)a.Q + m * a.q_stride_m + ((long)b * a.N + i) * a.q_stride_row + (long)h * a.d;
#pragma unroll
    for (int sl = 0; sl < SL; ++sl) {
      const int f = sl * Sh::kSliceF + g4 * Sh::kPiece;
      qf[rt][sl] = make_uint4(0, 0, 0, 0);
      if (r < R && f < a.d) qf[rt][sl] = *reinterpret_cast<const uint4*>(q + f);
    }
    slope[rt] = biased ? a.slope[m * a.heads + h] * unit : 0.f;
  }
  if constexpr (TREE) {
    int par = lane - 1;                                    // paths of all nodes at once, as in decoder_tiles.h
    if (a.parent && a.N > 1) {
      par = lane < a.N ? a.parent[mb * a.N + lane] : -1;
      par = par < lane ? par : -1;
    }
    uint64_t all = 1ull << lane;
    for (int step = 1; step < a.N; step *= 2) {
      const int from = max(par, 0);
      const uint32_t x = __shfl((uint32_t)all, from, kWave), y = __shfl((uint32_t)(all >> 32), from, kWave);
      const int up = __shfl(par, from, kWave);
      if (par >= 0) {
        all |= ((uint64_t)y << 32) | x;
        par = up;
      }
    }
    const int begin = a.start ? a.start[mb] : L;
    node_at = begin + __popcll(all) - 1;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const uint32_t x = __shfl((uint32_t)all, token[rt], kWave), y = __shfl((uint32_t)(all >> 32), token[rt], kWave);
      path[rt] = ((uint64_t)y << 32) | x;
      mine[rt] = begin + __popcll(path[rt]) - 1;
      end[rt] = L;
      docr[rt] = 0;
    }
  } else {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int i = token[rt];
      path[rt] = 0;
      mine[rt] = i;
      docr[rt] = doc ? doc[i] : 0;
      end[rt] = i >= L || docr[rt] < 0 ? 0 : a.causal ? max(i + 1, first) : L;
    }
    if (doc) {
      lo = 0x7fffffff;
      hi = -1;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
        if (end[rt] > 0) lo = min(lo, docr[rt]), hi = max(hi, docr[rt]);
#pragma unroll
      for (int o = 1; o < kWave; o *= 2) {
        lo = min(lo, __shfl_xor(lo, o, kWave));
        hi = max(hi, __shfl_xor(hi, o, kWave));
      }
      lo = __builtin_amdgcn_readfirstlane(lo);
      hi = __builtin_amdgcn_readfirstlane(hi);
    }
  }

  f32x4_t o_acc[RT][NB];                                   // element r of block i: feature (i / VF) 16 VF + VF (4 g4 + r) + i % VF of row l16
  float mrun[RT], lrun[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    mrun[rt] = kLowestScore;
    lrun[rt] = 0.f;
#pragma unroll
    for (int i = 0; i < NB; ++i) o_acc[rt][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const float sc = a.scale * unit;

  if (!early) {
    st = seek(share);
    if (st < steps) load_keys(st);
  }
  while (st < steps) {
    const bool mask = !whole(st), own_step = TREE && st >= cached_steps;
    const int base = own_step ? (st - cached_steps) * kStep : key_start + st * kStep;
    load_values(st);
    f32x4_t s[RT][NK];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int k = 0; k < NK; ++k) s[rt][k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int sl = 0; sl < SL; ++sl)
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][k] = slice_product<T>(kreg[k][sl], qf[rt][sl], s[rt][k]);
    const int key_now = own_step ? __shfl(node_at, (base + lane) % kWave, kWave) : key_reg;
    const int next = seek(st + KS);
    if (next < steps) load_keys(next);

    // element r of block k: key base + 16 k + 4 g4 + r of row l16
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float x = s[rt][k][r];
          if (capped_scores) {
            if constexpr (kBf) {
              x = tanh_either(x * (a.scale * a.inv_cap)) * (a.cap * kLog2e);
            } else {
              x = a.cap * tanhf(x * a.scale * a.inv_cap);
            }
          } else {
            x *= sc;
          }
          s[rt][k][r] = x;
        }
      if (biased) {
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int at = TREE && (a.pos || own_step) ? __shfl(key_now, 16 * k + 4 * g4 + r, kWave) : base + 16 * k + 4 * g4 + r;
            s[rt][k][r] = fmaf(-slope[rt], fabsf((float)(mine[rt] - at)), s[rt][k][r]);
          }
      }
      if (mask) {                                          // weight 0 whatever the score
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = base + 16 * k + 4 * g4 + r;
            bool seen = own_step ? (key < 64) & (int)((path[rt] >> (key & 63)) & 1) : key < end[rt];
            if (!TREE && doc) {
              const int of = __shfl(key_now, 16 * k + 4 * g4 + r, kWave);  // by every lane
              seen &= of == docr[rt];
            }
            s[rt][k][r] = seen ? s[rt][k][r] : -INFINITY;
          }
      }
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, s[rt][k][r]);
      top = across_halves(across_rows(top, MaxOp{}), MaxOp{});
      const float mnew = fmaxf(mrun[rt], top);
      const float corr = kBf ? __builtin_amdgcn_exp2f(mrun[rt] - mnew) : expf(mrun[rt] - mnew);
      mrun[rt] = mnew;
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[rt][k][r] = kBf ? __builtin_amdgcn_exp2f(s[rt][k][r] - mnew) : expf(s[rt][k][r] - mnew);
          sum += s[rt][k][r];
        }
      lrun[rt] = fmaf(lrun[rt], corr, sum);
      if (__any(corr != 1.0f)) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) o_acc[rt][i][r] *= corr;
      }
    }

    if (mask) {
      // values that are infinite or NaN: 0 times them would reach the rows that do not see them, so each row takes them from the keys that have a
      // weight and the product runs on the others.  Key e of a lane's group g is passed round group by group.
#pragma unroll
      for (int e = 0; e < NK * 4; ++e) {
        bool odd = false;
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
          for (int w = 0; w < Sh::kVWords; ++w) odd |= kBf ? bf16_odd(vreg[e][c].w[w]) : (vreg[e][c].w[w] & 0x7f800000u) == 0x7f800000u;
        const uint64_t where = __ballot(odd);
        if (where == 0) continue;                          // uniform
#pragma unroll 1
        for (int from = 0; from < 4; ++from) {
          if (!((where >> (16 * from)) & 0xffff)) continue;
          bool takes[RT];
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) takes[rt] = __shfl(s[rt][e / 4][e % 4], 16 * from + l16, kWave) != 0.f;
#pragma unroll
          for (int c = 0; c < VC; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int w = 0; w < Sh::kVWords; ++w) {
                const uint32_t x = __shfl(vreg[e][c].w[w], 16 * from + 4 * g4 + r, kWave);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                  if constexpr (kBf) {
                    o_acc[rt][c * VF + 2 * w][r] += takes[rt] & ((x & 0x7f80u) == 0x7f80u) ? __uint_as_float(x << 16) : 0.f;
                    o_acc[rt][c * VF + 2 * w + 1][r] += takes[rt] & ((x & 0x7f800000u) == 0x7f800000u) ? __uint_as_float(x & 0xffff0000u) : 0.f;
                  } else {
                    o_acc[rt][c * VF + w][r] += takes[rt] & ((x & 0x7f800000u) == 0x7f800000u) ? __uint_as_float(x) : 0.f;
                  }
                }
              }
        }
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
          for (int w = 0; w < Sh::kVWords; ++w) {
            const uint32_t x = vreg[e][c].w[w];
            if constexpr (kBf) vreg[e][c].w[w] = ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u);
            else vreg[e][c].w[w] = (x & 0x7f800000u) == 0x7f800000u ? 0u : x;
          }
      }
    }
    if constexpr (kBf) {
#pragma unroll
      for (int k = 0; k < NK; k += 2) {
        // A weight in two parts: its upper 8 bits, of a value a little smaller, and the rest.  Neither is 0 where the weight is not, so an infinite value gives that
        // infinity in both products.
        bf16x8_t upper[RT], rest[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          uint32_t u[4], l[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = s[rt][k + e / 2][e % 2 * 2], y = s[rt][k + e / 2][e % 2 * 2 + 1];
            const uint32_t xu = __float_as_uint(x * 0x1.ffp-1f), yu = __float_as_uint(y * 0x1.ffp-1f);
            u[e] = __builtin_amdgcn_perm(yu, xu, 0x07060302u);
            l[e] = pack_bf16x2(x - __uint_as_float(xu & 0xffff0000u), y - __uint_as_float(yu & 0xffff0000u));
          }
          upper[rt] = __builtin_bit_cast(bf16x8_t, make_uint4(u[0], u[1], u[2], u[3]));
          rest[rt] = __builtin_bit_cast(bf16x8_t, make_uint4(l[0], l[1], l[2], l[3]));
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          uint32_t x[4];
#pragma unroll
          for (int e = 0; e < 8; e += 2)
            x[e / 2] = __builtin_amdgcn_perm(vreg[4 * k + e + 1][i / VF].w[i % VF / 2], vreg[4 * k + e][i / VF].w[i % VF / 2], i % 2 ? 0x07060302u : 0x05040100u);
          const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, make_uint4(x[0], x[1], x[2], x[3]));
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            o_acc[rt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, upper[rt], o_acc[rt][i], 0, 0, 0);
            o_acc[rt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, rest[rt], o_acc[rt][i], 0, 0, 0);
          }
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < NK * 4; ++e)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
            o_acc[rt][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vreg[e][i / VF].w[i % VF]), s[rt][e / 4][e % 4], o_acc[rt][i], 0, 0, 0);
    }
    st = next;
  }

  // ---- the result: for each of its elements r a lane has the NB features of row l16; share k of KS finishes elements 4 / KS k ..
  constexpr int kOut = 4 / KS;
  const bool partial = TREE && parts > 1;
  float* const ml = a.ws + (long)a.M * a.B * a.kv * R * splits * D;
  extern __shared__ __align__(16) unsigned char dec_smem[];
  lds_f32_t* const buf = (lds_f32_t*)dec_smem;             // stream_lds_bytes
  lds_f32_t* const max_of = buf + 256 * RT * 4 * NB;
  lds_f32_t* const sum_of = max_of + RT * 256;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) lrun[rt] = across_halves(across_rows(lrun[rt], AddOp{}), AddOp{});
  if constexpr (KS > 1) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int q = 0; q < NB / 4; ++q)
          *(lds_f32x4_t*)(buf + (((rt * 4 + r) * (NB / 4) + q) * 256 + tid) * 4) = f32x4v_t{o_acc[rt][4 * q][r], o_acc[rt][4 * q + 1][r], o_acc[rt][4 * q + 2][r], o_acc[rt][4 * q + 3][r]};
      max_of[rt * 256 + tid] = mrun[rt];
      sum_of[rt * 256 + tid] = lrun[rt];
    }
    __syncthreads();
  }
  const int lane0 = tid % (RG * kWave);                    // this lane in share 0
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = r0 + (rg * RT + rt) * 16 + l16;
    if (r >= R) continue;
    float mtot = mrun[rt], ltot = lrun[rt], c[KS];
    if constexpr (KS > 1) {
      mtot = kLowestScore;
#pragma unroll
      for (int k = 0; k < KS; ++k) mtot = fmaxf(mtot, max_of[rt * 256 + lane0 + k * RG * kWave]);
      ltot = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const float x = max_of[rt * 256 + lane0 + k * RG * kWave] - mtot;
        c[k] = kBf ? __builtin_amdgcn_exp2f(x) : expf(x);
        ltot = fmaf(sum_of[rt * 256 + lane0 + k * RG * kWave], c[k], ltot);
      }
    }
    const bool none = ltot == 0.f || (TREE ? token[rt] >= there : end[rt] == 0);
    const float inv = none ? 0.f : 1.0f / ltot;
    const int h = g * group + (r - token[rt] * group);
    const long at = (head * R + r) * splits + split;
    T* Op = (T*)a.O + (mb * a.N + token[rt]) * ((long)a.heads * a.d) + (long)h * a.d;
#pragma unroll
    for (int u = 0; u < kOut; ++u) {
      const int e = share * kOut + u;                      // element of the accumulators
      float v[NB];
      if constexpr (KS == 1) {
#pragma unroll
        for (int i = 0; i < NB; ++i) v[i] = o_acc[rt][i][u];
      } else {
#pragma unroll
        for (int i = 0; i < NB; ++i) v[i] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int q = 0; q < NB / 4; ++q) {
            const f32x4v_t x = *(const lds_f32x4_t*)(buf + (((rt * 4 + e) * (NB / 4) + q) * 256 + lane0 + k * RG * kWave) * 4);
#pragma unroll
            for (int z = 0; z < 4; ++z) v[4 * q + z] = fmaf(x[z], c[k], v[4 * q + z]);
          }
      }
#pragma unroll
      for (int ch = 0; ch < VC; ++ch) {
        const int f = ch * 16 * VF + VF * (4 * g4 + e);
        if (partial) {
#pragma unroll
          for (int i = 0; i < VF; i += 4) *reinterpret_cast<f32x4_t*>(a.ws + at * D + f + i) = f32x4_t{v[ch * VF + i], v[ch * VF + i + 1], v[ch * VF + i + 2], v[ch * VF + i + 3]};
        } else if (f < a.d) {
          Words<Sh::kVWords> w;
#pragma unroll
          for (int i = 0; i < Sh::kVWords; ++i) {
            if constexpr (kBf) w.w[i] = none ? 0u : pack_bf16x2(v[ch * VF + 2 * i] * inv, v[ch * VF + 2 * i + 1] * inv);
            else w.w[i] = none ? 0u : __float_as_uint(v[ch * VF + i] * inv);
          }
          *reinterpret_cast<Words<Sh::kVWords>*>(__builtin_assume_aligned(Op + f, Sh::kVWords * 4)) = w;
        }
      }
    }
    if (TREE && share == 0 && g4 == 0) {
      if (partial) *reinterpret_cast<float2*>(ml + 2 * at) = make_float2(mtot, ltot);
      else if (a.lse) a.lse[(mb * a.N + token[rt]) * a.heads + h] = none ? -INFINITY : kBf ? (mtot + __builtin_amdgcn_logf(ltot)) * kLn2 : mtot + logf(ltot);
    }
  }
}

}  // namespace nf
