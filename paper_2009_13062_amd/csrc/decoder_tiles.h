// Merged decoders, bfloat16 attention on the matrix pipe: head sizes that are multiples of 8, up to D features.
//
// The rows of one key head are its tokens times its query heads, row r = token r / group, so keys and values are read once for the
// whole group.  A workgroup is 4 wavefronts: RG groups of 32 RB rows times KS shares of the keys (RG KS = 4); keys pass KB at a time through LDS, the
// next tile's loads being in flight in registers meanwhile.  Scores are computed transposed, S^T = K Q^T, so the 32 x 32
// accumulator of a lane holds 16 keys of ONE row (lane % 32): the softmax statistics are per-lane scalars, the two lane halves hold
// the same row, and the weights are already in the register order of the B operand of O^T = V^T P^T, the keys of a 16-key step being
// permuted alike on the V^T side, which comes from the transposing LDS read.  Scores, maximum and sum are float32 in log2 units;
// weights are rounded to bfloat16 for the second product (half a step of 2^-8 each, as the result itself), their sum is not.
//
// Which keys a row sees is an upper end per row (causal, prefix, lengths), the documents of a tile (staged with its keys) or, for the tree's
// own tile, a bit per node.  Tiles that every row of a wavefront sees in full are not masked, tiles that none sees are left out.  In a masked
// tile, values that are infinite or NaN are found as they are staged, and that tile's second product is then summed by each lane over
// the keys that have a weight (0 times NaN would reach the rows that do not see them).
//
// A cache is shared out among workgroups in chunks of a length that depends on the number of rows alone: a sequence's bits depend neither on
// what is merged with it nor on the capacity.  Where a sequence fills more than one chunk, partial sums go to the workspace and a second kernel joins them.
#pragma once
#include "decoder.h"
#include "gemm_mfma.h"

namespace nf {

typedef int int4v_t __attribute__((ext_vector_type(4)));

template <int D, int KB, int STAGES> struct DecLds {
  static constexpr int kKPitch = D + 8;                    // 16-byte fragment reads of 32 keys spread over the banks
  static constexpr int kVPitch = D + 32;                   // the 4 keys x 64 bytes of a transposing read tile the 64 banks
  static constexpr int kOffV = STAGES * KB * kKPitch * 2;
  static constexpr int kOffKey = kOffV + STAGES * KB * kVPitch * 2;       // position or document of each key
  static constexpr int kOffFlag = kOffKey + STAGES * KB * 4;              // tile whose values are not all finite, per stage
  static constexpr int kBytes = kOffFlag + 16;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// tanh(u): near 0 by its series (the other form loses its bits there), relative error below 2^-20 either way.
__device__ __forceinline__ float tanh_series(float u) {
  const float w = u * u;
  float p = fmaf(w, 0.021869488536155203f, -0.05396825396825397f);
  p = fmaf(p, w, 0.13333333333333333f);
  p = fmaf(p, w, -0.3333333333333333f);
  return fmaf(p * w, u, u);
}
__device__ __forceinline__ float tanh_exp(float u) {
  const float e = __builtin_amdgcn_exp2f(fabsf(u) * (2.f * kLog2e));      // infinite for large u: 1
  return copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f), u);
}
constexpr float kTanhSeries = 0.25f;
__device__ __forceinline__ float tanh_either(float u) {
  const float t = tanh_series(u), e = tanh_exp(u);
  return fabsf(u) < kTanhSeries ? t : e;
}

// Either half of a dword an infinity or NaN of bfloat16
__device__ __forceinline__ bool bf16_odd(uint32_t x) { return ((x & 0x7f80u) == 0x7f80u) | ((x & 0x7f800000u) == 0x7f800000u); }

template <int D, int KB, int KS, int RB, bool TREE>
__global__ __launch_bounds__(256, 2) void decoder_tiles_kernel(DecArgs a, int row_blocks, int splits, int chunk) {
  constexpr int RG = 4 / KS, kStages = KS == 1 ? 2 : 1, TB = D / 32;
  constexpr int kRows = RG * RB * 32;                      // per workgroup
  constexpr int NSB = KB / KS / 32;                        // 32-key blocks of a tile per wavefront
  constexpr int kPer = KB * D / 8 / 256;                   // 16-byte pieces per thread and tensor
  using Lds = DecLds<D, KB, kStages>;
  extern __shared__ __align__(16) unsigned char dec_smem[];
  lds_bf16_t* const Ks = (lds_bf16_t*)dec_smem;
  lds_bf16_t* const Vs = (lds_bf16_t*)(dec_smem + Lds::kOffV);
  typedef __attribute__((address_space(3))) int lds_int_t;
  typedef __attribute__((address_space(3))) int4v_t lds_int4_t;
  lds_int_t* const Key = (lds_int_t*)(dec_smem + Lds::kOffKey);
  lds_int_t* const Flag = (lds_int_t*)(dec_smem + Lds::kOffFlag);
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int half = lane / 32, lq = lane % 32, l16 = lane % 16;
  const int rg = wave % RG, key0 = wave / RG * (KB / KS);  // of a tile

  unsigned id = xcd_remap(blockIdx.x, gridDim.x);
  int split = 0, rblock;
  if (TREE) {
    split = id % splits;  id /= splits;
    rblock = id % row_blocks;
  } else {
    rblock = row_blocks - 1 - (int)(id % row_blocks);      // the longest rows of a head first
  }
  const long head = id / row_blocks;                       // (m, b, g)
  const int g = (int)(head % a.kv);
  const long mb = head / a.kv;
  const int b = (int)(mb % a.B);
  const long m = mb / a.B;
  const int group = a.heads / a.kv, R = a.N * group, r0 = rblock * kRows;
  const int L = TREE ? clamp_len(a.len[mb], a.C) : a.len ? clamp_len(a.len[mb], a.N) : a.N;
  const int parts = TREE ? max(1, (L + chunk - 1) / chunk) : 1;           // chunks that this cache fills
  if (split >= parts) return;                              // uniform
  const int there = TREE && a.nodes ? clamp_len(a.nodes[mb], a.N) : a.N;
  const int first = !TREE && a.prefix ? clamp_len(a.prefix[mb], L) : 0;   // keys below it are seen by every row
  const int* doc = !TREE && a.doc ? a.doc + mb * a.N : nullptr;
  const bool keyed = TREE ? a.slope != nullptr : doc != nullptr;          // a value per key is staged

  const bf16_t* Kp = (const bf16_t*)a.K + m * a.kv_stride_m + (long)b * a.N * a.kv_stride_row + (long)g * a.d;
  const bf16_t* Vp = (const bf16_t*)a.V + m * a.kv_stride_m + (long)b * a.N * a.kv_stride_row + (long)g * a.d;
  const bf16_t* Kh = TREE ? (const bf16_t*)a.Kc + head * a.C * a.d : Kp;
  const bf16_t* Vh = TREE ? (const bf16_t*)a.Vc + head * a.C * a.d : Vp;
  const long stride = TREE ? a.d : a.kv_stride_row;

  // ---- this lane's rows: the B operand of S^T = K Q^T, 8 consecutive features per 16-step
  int token[RB], end[RB], mine[RB], docr[RB];
  uint64_t path[RB];
  float slope[RB];
  bf16x8_t qf[RB][D / 16];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = r0 + (rg * RB + rb) * 32 + lq;
    const int i = min(r, R - 1) / group, h = g * group + (min(r, R - 1) - i * group);
    token[rb] = i;
    const bf16_t* q = (const bf16_t*)a.Q + m * a.q_stride_m + ((long)b * a.N + i) * a.q_stride_row + (long)h * a.d;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (r < R && kk * 16 + half * 8 < a.d) v = *reinterpret_cast<const uint4*>(q + kk * 16 + half * 8);
      qf[rb][kk] = __builtin_bit_cast(bf16x8_t, v);
    }
    slope[rb] = a.slope ? a.slope[m * a.heads + h] * kLog2e : 0.f;
  }

  int node_at = 0;                                         // position of node `lane`
  int blo = 0, bhi = 0, block_end = 0;                     // documents and last key of the workgroup's rows
  if constexpr (TREE) {
    // paths of all nodes at once, a node per lane: each step doubles the ancestors that a path holds
    int par = lane - 1;
    if (a.parent && a.N > 1) {
      par = lane < a.N ? a.parent[mb * a.N + lane] : -1;
      par = par < lane ? par : -1;
    }
    uint64_t all = 1ull << lane;
    for (int step = 1; step < a.N; step *= 2) {
      const int from = max(par, 0);
      const uint32_t lo = __shfl((uint32_t)all, from, kWave), hi = __shfl((uint32_t)(all >> 32), from, kWave);
      const int up = __shfl(par, from, kWave);
      if (par >= 0) {
        all |= ((uint64_t)hi << 32) | lo;
        par = up;
      }
    }
    const int begin = a.start ? a.start[mb] : L;
    node_at = begin + __popcll(all) - 1;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const uint32_t lo = __shfl((uint32_t)all, token[rb], kWave), hi = __shfl((uint32_t)(all >> 32), token[rb], kWave);
      path[rb] = ((uint64_t)hi << 32) | lo;
      mine[rb] = begin + __popcll(path[rb]) - 1;
      end[rb] = L;
      docr[rb] = 0;
    }
  } else {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int i = token[rb];
      path[rb] = 0;
      mine[rb] = i;
      docr[rb] = doc ? doc[i] : 0;
      const bool valid = i < L && docr[rb] >= 0;
      end[rb] = !valid ? 0 : a.causal ? max(i + 1, first) : L;
    }
    const int i_lo = r0 / group, i_hi = min(min(r0 + kRows, R) - 1, R - 1) / group;
    block_end = i_lo >= L ? 0 : a.causal ? min(max(i_hi + 1, first), L) : L;
    if (doc) {
      blo = 0x7fffffff;
      bhi = -1;
      for (int i = i_lo + lane; i <= i_hi && i < L; i += kWave) {
        const int v = doc[i];
        if (v >= 0) blo = min(blo, v), bhi = max(bhi, v);
      }
#pragma unroll
      for (int o = 1; o < kWave; o *= 2) {
        blo = min(blo, __shfl_xor(blo, o, kWave));
        bhi = max(bhi, __shfl_xor(bhi, o, kWave));
      }
      blo = __builtin_amdgcn_readfirstlane(blo);
      bhi = __builtin_amdgcn_readfirstlane(bhi);
    }
  }
  // tokens of this wavefront's rows
  const int w_lo = (r0 + rg * RB * 32) / group, w_hi = min(r0 + (rg + 1) * RB * 32 - 1, R - 1) / group;

  // ---- the tiles: first key of each; the tree's own tile is kTreeTile, none left kNoTile
  constexpr int kTreeTile = -1, kNoTile = -2;
  const int tile_end = TREE ? min(L, (split + 1) * chunk) : block_end;
  uint32_t win_any = 0, win_all = 0;                       // of 16 tiles from win_at on: which hold a document of the rows, nothing but their only one
  int win_at = -(16 * KB);
  auto look = [&](int j0) {
    win_at = j0;
    win_any = win_all = 0;
#pragma unroll 4
    for (int t = 0; t < 16; ++t) {
      bool any = false, all = true;
#pragma unroll
      for (int u = 0; u < KB / kWave; ++u) {
        const int j = j0 + t * KB + u * kWave + lane, v = doc[min(j, L - 1)];
        any |= (j < L) & (v >= blo) & (v <= bhi);
        all &= (j < L) & (v == blo);
      }
      win_any |= (__any(any) ? 1u : 0u) << t;
      win_all |= (__all(all) && blo == bhi ? 1u : 0u) << t;
    }
  };
  auto seek = [&](int j0) -> int {                         // the tile at j0 or the next one that is wanted
    if (TREE) return j0 < tile_end ? j0 : split == parts - 1 && j0 < tile_end + KB ? kTreeTile : kNoTile;
    if (doc) {
      while (j0 < tile_end) {
        if (j0 >= win_at + 16 * KB) look(j0);
        const uint32_t rest = win_any >> ((j0 - win_at) / KB);
        if (rest) {
          j0 += __builtin_ctz(rest) * KB;
          break;
        }
        j0 = win_at + 16 * KB;
      }
    }
    return j0 < tile_end ? j0 : kNoTile;
  };
  auto after = [&](int j0) -> int { return j0 == kTreeTile ? kNoTile : seek(j0 + KB); };
  // whether any row of the workgroup leaves out a key of the tile
  auto whole = [&](int j0, int i_lo) -> bool {
    if (j0 == kTreeTile || j0 + KB > L) return false;
    if (TREE) return true;
    if (a.causal && j0 + KB > i_lo + 1 && j0 + KB > first) return false;
    return !doc || ((win_all >> ((j0 - win_at) / KB)) & 1);
  };

  uint4 kreg[kPer], vreg[kPer];
  int key_reg = 0;
  const int my_key = tid / (D / 8), my_f = tid % (D / 8) * 8;             // first piece of this thread: the others are 256 / (D / 8) keys apart
  auto fetch = [&](int j0) {
    const bool own_tile = TREE && j0 == kTreeTile;
    const int base = own_tile ? 0 : j0, limit = (own_tile ? a.N : L) - base;
    const long st = own_tile ? a.kv_stride_row : stride;
    const auto rk = rows_from((own_tile ? Kp : Kh) + base * st), rv = rows_from((own_tile ? Vp : Vh) + base * st);
    const unsigned row = (unsigned)(st * 2), from = my_key * row + my_f * 2;
#pragma unroll
    for (int t = 0; t < kPer; ++t) {
      const bool in = my_key + t * (2048 / D) < limit && my_f < a.d;
      const unsigned off = in ? from + t * (2048 / D) * row : kDecOob;
      kreg[t] = rows_load16(rk, off);
      vreg[t] = rows_load16(rv, off);
    }
    if (keyed && tid < KB) {
      const int key = base + tid, there = min(tid, limit - 1) + base;
      key_reg = TREE ? (own_tile ? node_at : a.pos ? a.pos[head * a.C + there] : key) : doc[there];
      if (!TREE && tid >= limit) key_reg = -1;
    }
  };
  auto commit = [&](int stage, bool check, int number) {
    if (keyed && tid < KB) Key[stage * KB + tid] = key_reg;
    bool odd = false;
#pragma unroll
    for (int t = 0; t < kPer; ++t) {
      const int c = tid + t * 256, key = c / (D / 8), f = c % (D / 8) * 8;
      lds_store16(Ks + (stage * KB + key) * Lds::kKPitch + f, kreg[t]);
      lds_store16(Vs + (stage * KB + key) * Lds::kVPitch + f, vreg[t]);
      if (check) odd |= bf16_odd(vreg[t].x) | bf16_odd(vreg[t].y) | bf16_odd(vreg[t].z) | bf16_odd(vreg[t].w);
    }
    if (check && odd) Flag[stage] = number;
  };

  f32x16_t o_acc[RB][TB];
  float mrun[RB], lrun[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    mrun[rb] = kLowestScore;
    lrun[rb] = 0.f;                                        // this half's partial sum
#pragma unroll
    for (int tb = 0; tb < TB; ++tb)
#pragma unroll
      for (int r = 0; r < 16; ++r) o_acc[rb][tb][r] = 0.f;
  }
  const bool capped_scores = a.cap != 0.f, biased = a.slope != nullptr;
  const float sc = a.scale * kLog2e;
  const float to_u = a.scale * a.inv_cap, back = a.cap * kLog2e, u2 = to_u * to_u;
  const float cap1 = sc * u2 * -0.3333333333333333f, cap2 = sc * u2 * u2 * 0.13333333333333333f, cap3 = sc * u2 * u2 * u2 * -0.05396825396825397f;
  const float cap_small = fabsf(to_u) > 1e-4f && fabsf(to_u) < 1e4f ? kTanhSeries / fabsf(to_u) : 0.f;      // powers of others leave float32
  const bool raw = !capped_scores && !biased && sc > 0.f;  // scale and maximum enter the exponent in one fma

  if (tid < kStages) Flag[tid] = 0;
  int tile = seek(TREE ? split * chunk : 0), number = 1;
  const int block_lo = r0 / group;
  bool tile_whole = false;
  if (tile != kNoTile) {
    tile_whole = whole(tile, block_lo);
    fetch(tile);
    __syncthreads();                                       // Flag is clear
    commit(0, !tile_whole, number);
  }
  __syncthreads();
  while (tile != kNoTile) {
    const int cur = kStages == 2 ? (number - 1) & 1 : 0;
    const bool was_whole = tile_whole;
    // masks of this tile are settled before the window of documents moves on
    const bool mask = TREE ? !was_whole : !whole(tile, w_lo);
    const int next = after(tile);
    if (next != kNoTile) {
      tile_whole = whole(next, block_lo);
      fetch(next);
    }
    const bool skip = !TREE && a.causal && tile > w_hi && tile >= first;          // no row of this wavefront sees the tile
    const bool odd_tile = !was_whole && Flag[cur] == number;                      // uniform over the workgroup
    if (!skip || odd_tile) {
      const lds_bf16_t* Kc = Ks + (cur * KB + key0) * Lds::kKPitch;
      const lds_int_t* Kk = Key + cur * KB + key0;
      const int base = (tile == kTreeTile ? 0 : tile) + key0 + 4 * half;          // register r of block sb is key base + 32 sb + 8 (r / 4) + r % 4
      f32x16_t s[RB][NSB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[rb][sb][r] = 0.f;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb) {
          const bf16x8_t kf = *(const lds_bf16x8_t*)(Kc + (sb * 32 + lq) * Lds::kKPitch + kk * 16 + half * 8);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) s[rb][sb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[rb][kk], s[rb][sb], 0, 0, 0);
        }
      bf16x8_t pf[RB][NSB][2];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        if (capped_scores) {                               // uniform
          float top = 0.f;
#pragma unroll
          for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(s[rb][sb][r]));
          if (__all(top < cap_small)) {                    // as a rule: the series in the unscaled score, its last term below 2^-21
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const float w = s[rb][sb][r] * s[rb][sb][r];
                s[rb][sb][r] *= fmaf(fmaf(fmaf(w, cap3, cap2), w, cap1), w, sc);
              }
          } else {
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r = 0; r < 16; ++r) s[rb][sb][r] = tanh_either(s[rb][sb][r] * to_u) * back;
          }
        } else if (!raw) {
#pragma unroll
          for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[rb][sb][r] *= sc;
        }
        if (biased) {
          if (TREE && (a.pos || tile == kTreeTile)) {
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r4 = 0; r4 < 4; ++r4) {
                const int4v_t at = *(const lds_int4_t*)(Kk + sb * 32 + 8 * r4 + 4 * half);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[rb][sb][4 * r4 + e] = fmaf(-slope[rb], fabsf((float)(mine[rb] - at[e])), s[rb][sb][4 * r4 + e]);
              }
          } else {
            const float away = (float)(mine[rb] - base);
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r = 0; r < 16; ++r) s[rb][sb][r] = fmaf(-slope[rb], fabsf(away - (float)(32 * sb + 8 * (r / 4) + r % 4)), s[rb][sb][r]);
          }
        }
        if (mask) {                                        // weight 0 whatever the score
          if (TREE && tile == kTreeTile) {
            const uint64_t bits = path[rb] >> (key0 + 4 * half);
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const int c = 32 * sb + 8 * (r / 4) + r % 4;
                s[rb][sb][r] = key0 + 4 * half + c < 64 && ((bits >> c) & 1) ? s[rb][sb][r] : -INFINITY;
              }
          } else {
            const int left = end[rb] - base;
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r = 0; r < 16; ++r) s[rb][sb][r] = 32 * sb + 8 * (r / 4) + r % 4 < left ? s[rb][sb][r] : -INFINITY;
            if (!TREE && doc) {
#pragma unroll
              for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) {
                  const int4v_t of = *(const lds_int4_t*)(Kk + sb * 32 + 8 * r4 + 4 * half);
#pragma unroll
                  for (int e = 0; e < 4; ++e) s[rb][sb][4 * r4 + e] = of[e] == docr[rb] ? s[rb][sb][4 * r4 + e] : -INFINITY;
                }
            }
          }
        }
        float top = -INFINITY;
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
          for (int r = 0; r < 16; ++r) top = fmaxf(top, s[rb][sb][r]);
        top = across_halves(top, MaxOp{});
        if (raw) top *= sc;
        const float mnew = fmaxf(mrun[rb], top);
        float esc = raw ? sc : 1.0f;                       // exponent = s * esc - mnew
        if (raw && __any(fabsf(mnew) > 0x1p29f && mnew != kLowestScore)) {        // the rounded maximum may lie far beside such a score: scale first
#pragma unroll
          for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[rb][sb][r] *= sc;
          esc = 1.0f;
        }
        const float corr = __builtin_amdgcn_exp2f(mrun[rb] - mnew);
        mrun[rb] = mnew;
        float sum = 0.f;
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
          for (int st = 0; st < 2; ++st) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p0 = __builtin_amdgcn_exp2f(fmaf(s[rb][sb][8 * st + 2 * e], esc, -mnew));
              const float p1 = __builtin_amdgcn_exp2f(fmaf(s[rb][sb][8 * st + 2 * e + 1], esc, -mnew));
              w[e] = pack_bf16x2(p0, p1);
              sum += p0 + p1;                              // float32 sum of the unrounded weights
            }
            pf[rb][sb][st] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
          }
        lrun[rb] = lrun[rb] * corr + sum;
        if (__any(corr != 1.0f)) {                         // after the first tiles the maximum of a row seldom moves
#pragma unroll
          for (int tb = 0; tb < TB; ++tb)
#pragma unroll
            for (int r = 0; r < 16; ++r) o_acc[rb][tb][r] *= corr;
        }
      }

      const lds_bf16_t* Vc = Vs + (cur * KB + key0) * Lds::kVPitch;
      if (odd_tile) {
        // which keys hold such a value: a key per lane
        bool odd = false;
        if (lane < KB / KS) {
#pragma unroll 1
          for (int f = 0; f < a.d; ++f) odd |= (Vc[lane * Lds::kVPitch + f] & 0x7f80) == 0x7f80;
        }
        const uint64_t odd_keys = __ballot(odd);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          uint32_t lo = 0, hi = 0;                         // keys under a weight that is not 0: this half's, then both
#pragma unroll
          for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
              const uint4 w = __builtin_bit_cast(uint4, pf[rb][sb][st]);
              const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const uint32_t bit = (ws[e / 2] >> (e % 2 * 16) & 0x7fffu) != 0 ? 1u << (16 * st + 8 * (e / 4) + e % 4) : 0u;
                if (sb == 0) lo |= bit; else hi |= bit;
              }
            }
          lo <<= 4 * half;
          hi <<= 4 * half;
          lo |= __shfl_xor(lo, 32, kWave);
          hi |= __shfl_xor(hi, 32, kWave);
          const uint64_t under = (uint64_t)hi << 32 | lo;
#pragma unroll 1
          for (uint64_t left = odd_keys; left; left &= left - 1) {
            const int k = __builtin_ctzll(left);
            const bool takes = (under >> k) & 1;
            const lds_bf16_t* vr = Vc + k * Lds::kVPitch + 4 * half;
#pragma unroll
            for (int tb = 0; tb < TB; ++tb)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const uint32_t v = vr[tb * 32 + 8 * (r / 4) + r % 4];
                o_acc[rb][tb][r] += takes & ((v & 0x7f80) == 0x7f80) ? __uint_as_float(v << 16) : 0.f;
              }
          }
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kPer; ++t) {                   // the product runs on the others
          lds_bf16_t* const v = Vs + (cur * KB + my_key + t * (2048 / D)) * Lds::kVPitch + my_f;
#pragma unroll 1
          for (int e = 0; e < 8; ++e)
            if ((v[e] & 0x7f80) == 0x7f80) v[e] = 0;
        }
        __syncthreads();
      }
      // O^T += V^T P^T.  In a 16-lane group, lane i points at key row i / 4, features 4 (i % 4) .. + 3 of a 4 x 16 block and receives the
      // 4 keys of feature i; slots 0-3 of step (sb, st) are keys 32 sb + 16 st + 4 half + 0..3, slots 4-7 the same + 8.
#pragma unroll
      for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int tb = 0; tb < TB; ++tb) {
            const lds_bf16_t* vp = Vc + (sb * 32 + st * 16 + 4 * half + l16 / 4) * Lds::kVPitch + tb * 32 + ((lane / 16) % 2) * 16 + (l16 % 4) * 4;
            const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)vp);
            const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(vp + 8 * Lds::kVPitch));
            const s16x8_t both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              o_acc[rb][tb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, both), pf[rb][sb][st], o_acc[rb][tb], 0, 0, 0);
          }
    }
    if (kStages == 1) __syncthreads();                     // the stage is free
    ++number;
    if (next != kNoTile) commit(kStages == 2 ? cur ^ 1 : 0, !tile_whole, number);
    tile = next;
    __syncthreads();
  }

  // ---- the result: element r of block tb is feature 32 tb + 8 (r / 4) + 4 half + r % 4
  const bool partial = TREE && parts > 1;
  float* const ml = a.ws + (long)a.M * a.B * a.kv * R * splits * D;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = r0 + (rg * RB + rb) * 32 + lq;
    float ltot = across_halves(lrun[rb], AddOp{}), mtot = mrun[rb];
    constexpr int kQuads = 4 * TB / KS;                    // pieces of 4 features that a lane finishes
    const int quad0 = wave / RG * kQuads;
    f32x4_t out[kQuads];
    if constexpr (KS == 1) {
#pragma unroll
      for (int u = 0; u < kQuads; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) out[u][e] = o_acc[rb][u / 4][4 * (u % 4) + e];
    } else {
      lds_f32_t* const buf = (lds_f32_t*)dec_smem;
      lds_f32_t* const max_of = buf + 256 * 16 * TB;
      lds_f32_t* const sum_of = max_of + 256;
      static_assert(256 * 16 * TB * 4 + 2 * 256 * 4 <= Lds::kBytes, "shares fit the stage");
#pragma unroll
      for (int u = 0; u < 4 * TB; ++u) *(lds_f32x4_t*)(buf + (u * 256 + tid) * 4) = f32x4v_t{o_acc[rb][u / 4][4 * (u % 4)], o_acc[rb][u / 4][4 * (u % 4) + 1], o_acc[rb][u / 4][4 * (u % 4) + 2], o_acc[rb][u / 4][4 * (u % 4) + 3]};
      max_of[tid] = mtot;
      sum_of[tid] = ltot;
      __syncthreads();
      const int lane0 = tid % (RG * kWave);                // this lane in share 0
      mtot = kLowestScore;
#pragma unroll
      for (int k = 0; k < KS; ++k) mtot = fmaxf(mtot, max_of[lane0 + k * RG * kWave]);
      ltot = 0.f;
#pragma unroll
      for (int u = 0; u < kQuads; ++u) out[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int from = lane0 + k * RG * kWave;
        const float c = __builtin_amdgcn_exp2f(max_of[from] - mtot);
        ltot = fmaf(sum_of[from], c, ltot);
#pragma unroll
        for (int u = 0; u < kQuads; ++u) {
          const f32x4v_t v = *(const lds_f32x4_t*)(buf + ((quad0 + u) * 256 + from) * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) out[u][e] = fmaf(v[e], c, out[u][e]);
        }
      }
    }
    if (r >= R) continue;
    const bool valid = TREE ? token[rb] < there : end[rb] > 0;
    const int h = g * group + (r - token[rb] * group);
    if (partial) {
      const long at = (head * R + r) * splits + split;
#pragma unroll
      for (int u = 0; u < kQuads; ++u) {
        const int f = 8 * (quad0 + u) + 4 * half;
        *reinterpret_cast<f32x4_t*>(a.ws + at * D + f) = out[u];
      }
      if (quad0 == 0 && half == 0) *reinterpret_cast<float2*>(ml + 2 * at) = make_float2(mtot, ltot);
      continue;
    }
    const float inv = valid && ltot != 0.f ? 1.0f / ltot : 0.f;
    const bool none = !valid || ltot == 0.f;
    bf16_t* Op = (bf16_t*)a.O + (mb * a.N + token[rb]) * ((long)a.heads * a.d) + (long)h * a.d;
#pragma unroll
    for (int u = 0; u < kQuads; ++u) {
      const int f = 8 * (quad0 + u) + 4 * half;
      if (f < a.d) *reinterpret_cast<uint2*>(Op + f) = none ? make_uint2(0, 0) : make_uint2(pack_bf16x2(out[u][0] * inv, out[u][1] * inv), pack_bf16x2(out[u][2] * inv, out[u][3] * inv));
    }
    if (TREE && a.lse && quad0 == 0 && half == 0) a.lse[(mb * a.N + token[rb]) * a.heads + h] = none ? -INFINITY : (mtot + __builtin_amdgcn_logf(ltot)) * kLn2;
  }
}

// Sums of the chunks of one row: D / 4 lanes hold its features, 4 each, and SHARE such groups of lanes take every SHARE-th chunk.  Maxima and sums in log2
// units where LOG2, natural ones otherwise.
template <typename T, int D, bool LOG2, int SHARE>
__global__ __launch_bounds__(256) void decoder_join_kernel(DecArgs a, int splits, int chunk) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes, kRows = kGroups / SHARE;
  static_assert(SHARE == 1 || SHARE == kGroups, "a group per row, or all of them on one");
  const int lane = threadIdx.x % kLanes, grp = threadIdx.x / kLanes;
  const int group = a.heads / a.kv, R = a.N * group;
  const long row = (long)blockIdx.x * kRows + (SHARE == 1 ? grp : 0);
  if (row >= (long)a.M * a.B * a.kv * R) return;
  const long head = row / R, mb = head / a.kv;
  const int r = (int)(row % R), i = r / group, h = (int)(head % a.kv) * group + r % group;
  const int parts = (clamp_len(a.len[mb], a.C) + chunk - 1) / chunk;
  if (parts <= 1) return;                                  // written already; uniform where groups share a row
  const float* o = a.ws + row * splits * D + lane * 4;
  const float2* ml = reinterpret_cast<const float2*>(a.ws + (long)a.M * a.B * a.kv * R * splits * D) + row * splits;
  const int first = SHARE == 1 ? 0 : grp;
  f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float top = kLowestScore, sum = 0.f;
  for (int k0 = first; k0 < parts; k0 += 8 * SHARE) {      // 8 loads of each kind at a time
    float2 p[8];
    f32x4_t v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int k = min(k0 + u * SHARE, parts - 1);
      p[u] = ml[k];
      v[u] = *reinterpret_cast<const f32x4_t*>(o + (long)k * D);
    }
    float most = top;
#pragma unroll
    for (int u = 0; u < 8; ++u) most = fmaxf(most, p[u].x);
    const float old = LOG2 ? __builtin_amdgcn_exp2f(top - most) : expf(top - most);
    top = most;
    sum *= old;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] *= old;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float c = k0 + u * SHARE < parts ? (LOG2 ? __builtin_amdgcn_exp2f(p[u].x - top) : expf(p[u].x - top)) : 0.f;
      sum = fmaf(p[u].y, c, sum);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(v[u][e], c, acc[e]);
    }
  }
  if constexpr (SHARE > 1) {
    __shared__ __align__(16) float of[kGroups][D];
    __shared__ float2 stat[kGroups];
    *reinterpret_cast<f32x4_t*>(&of[grp][lane * 4]) = acc;
    if (lane == 0) stat[grp] = make_float2(top, sum);
    __syncthreads();
    if (grp != 0) return;
    top = kLowestScore;
#pragma unroll
    for (int k = 0; k < kGroups; ++k) top = fmaxf(top, stat[k].x);
    acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const float c = LOG2 ? __builtin_amdgcn_exp2f(stat[k].x - top) : expf(stat[k].x - top);
      sum = fmaf(stat[k].y, c, sum);
      const f32x4_t v = *reinterpret_cast<const f32x4_t*>(&of[k][lane * 4]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(v[e], c, acc[e]);
    }
  }
  const bool none = sum == 0.f || (a.nodes && i >= clamp_len(a.nodes[mb], a.N));
  T* Op = (T*)a.O + (mb * a.N + i) * ((long)a.heads * a.d) + (long)h * a.d + lane * 4;
  if (lane * 4 < a.d) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(Op) = none ? make_uint2(0, 0) : make_uint2(pack_bf16x2(acc[0] / sum, acc[1] / sum), pack_bf16x2(acc[2] / sum, acc[3] / sum));
    else *reinterpret_cast<f32x4_t*>(Op) = none ? f32x4_t{0.f, 0.f, 0.f, 0.f} : f32x4_t{acc[0] / sum, acc[1] / sum, acc[2] / sum, acc[3] / sum};
  }
  if (a.lse && lane == 0) a.lse[(mb * a.N + i) * a.heads + h] = none ? -INFINITY : LOG2 ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : top + logf(sum);
}

}  // namespace nf
