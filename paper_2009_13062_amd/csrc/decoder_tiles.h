// Merged decoders, bfloat16 attention on the matrix pipe: head sizes that are multiples of 8, up to D features.
//
// The rows of one key head are its tokens times its query heads, row r = token r / group, so keys and values are read once for the
// whole group.  A workgroup is 4 wavefronts: RG groups of 32 rows times KS shares of 64 keys (RG KS = 4); the keys pass a tile of 64 KS at a time through
// two stages in LDS, loaded past the registers, the next tile on its way while one is worked on.  Scores are computed transposed, S^T = K Q^T, so the 32 x 32
// accumulator of a lane holds 16 keys of ONE row (lane % 32): the softmax statistics are per-lane scalars, the two lane halves hold
// the same row, and the weights are already in the register order of the B operand of O^T = V^T P^T, the keys of a 16-key step being
// permuted alike on the V^T side, which comes from the transposing LDS read.  Scores, maximum and sum are float32 in log2 units;
// weights are rounded to bfloat16 for the second product (half a step of 2^-8 each, as the result itself), their sum is not.  (In two parts, of 15 bits, the
// long prompt would take 1242 -> 1619 us, drafted trees 128 -> 147, packed documents 48.9 -> 51.9, and errors against 64 bits of 0.0018 to 0.0020 be 0.0016 to 0.0017.)
//
// Which keys a row sees is an upper end per row (causal, prefix, lengths), the documents of a tile (staged with its keys) or, for the tree's
// own tile, a bit per node.  Tiles that every row of a wavefront sees in full are not masked, tiles that none sees are left out.  In a masked
// tile, values that are infinite or NaN are looked for in the stage; each row adds those of the keys that have a weight in it, and the second product then runs on
// the others (0 times NaN would reach the rows that do not see them).
//
// A cache is shared out among workgroups in chunks of a length that depends on the number of rows alone: a sequence's bits depend neither on
// what is merged with it nor on the capacity.  Where a sequence fills more than one chunk, partial sums go to the workspace and a second kernel joins them.
//
// Long prompts are bound by vector arithmetic: per score one fma and a quarter-rate exponential, half a maximum, a sum and half a rounding, with a bias one fma
// more, under a cap five.  (2 models of 8191 tokens, 32 heads over 8 of 128 features, biased: 1.20 to 1.24 ms on most devices, 907 TFLOP/s where a library product reaches
// 1165 to 1197; of the cycles the vector units are busy 63 %, the matrix units 45 %.)  So scores stay as they come from the product until the exponent, and the branches below keep whole paths apart.  64 keys of
// 32 rows per step: two workgroups (three of up to 64 features) share a compute unit's LDS and registers, one's exponentials beside the other's products.
// Trees are bound by the cache's bytes below some 64 rows, then as prompts are (26 tokens over 32 caches of up to 4096 entries: 114 us and 15 to join).
#pragma once
#include "decoder.h"
#include "gemm_dma.h"

namespace nf {

typedef int int4v_t __attribute__((ext_vector_type(4)));

// 16 bytes per lane from `off` of the resource to the lane's place in 1 KB of LDS
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, lds_u8_t* to, unsigned off) { __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 16, (int)off, 0, 0, 0); }

template <int D, int KB> struct DecLds {
  static constexpr int kRow = D * 2, kTile = KB * kRow;    // bytes of a row, of the keys or values of a stage
  static constexpr int kPieces = D / 8, kRowsPerLoad = 1024 / kRow;
  static constexpr int kOffV = 2 * kTile;
  static constexpr int kOffKey = 4 * kTile;                // position or document of each key
  static constexpr int kOffFlag = kOffKey + 2 * KB * 4;    // tile whose values are not all finite
  static constexpr int kBytes = kOffFlag + 16;
  // Piece c of row r lies at c ^ swz(r), the same for rows that a thread's loads are apart.  K: 16 lanes that read one piece each of 16 neighbouring rows meet
  // all 16 groups of 4 banks (8 of them, twice, for D = 256); V: the 4 rows x 64
  // bytes of 32 lanes of a transposing read tile the 64 banks.
  __device__ static __forceinline__ int swz_k(int r) { return D == 64 ? (r / 2) % 8 : D == 128 ? r % 16 : r % 8; }
  __device__ static __forceinline__ int swz_v(int r) { return D == 64 ? (r / 2) % 2 * 4 : r % 4 * 4; }
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
// Of 1 - t / 3 + 2 t^2 / 15 - 17 t^3 / 315 + 62 t^4 / 2835, t = u^2, what is left out is below 2^-21 up to kTanhSeries; and up to kTanhShort, t0 its square, with t0 for one t of
// the fourth term: 17 / 315 t^2 (t0 - t) at most.
constexpr float kTanhSeries = 0.25f, kTanhShort = 0.1975f;
__device__ __forceinline__ float tanh_either(float u) {
  const float t = tanh_series(u), e = tanh_exp(u);
  return fabsf(u) < kTanhSeries ? t : e;
}

// A value that is the same in every lane, in a scalar register: the coefficients of the cap would take 8 vector registers that the tiles need (64 features: 9 spilled, 1 with this)
__device__ __forceinline__ float uniform(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }

// Either half of a dword an infinity or NaN of bfloat16
__device__ __forceinline__ bool bf16_odd(uint32_t x) { return ((x & 0x7f80u) == 0x7f80u) | ((x & 0x7f800000u) == 0x7f800000u); }

// Order of the N operands of a product that come from LDS, READS reads and one matrix instruction each: four operands are asked for ahead of the
// instruction that takes them.  (Left to itself the compiler asks for one and waits for it.)
template <int N, int READS> __device__ __forceinline__ void keep_ahead() {
  constexpr int kAhead = N < 4 ? N : 4;
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead * READS, 0);
#pragma unroll
  for (int i = 0; i < N - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x8, kAhead, 0);
}

// Scores: as they come from the product, scale and maximum entering the exponent in one fma, or any (capped, odd scales); each without and with a bias by distance.
constexpr int kRawScore = 0, kRawBiased = 1, kAnyScore = 2, kAnyBiased = 3;
constexpr std::true_type kShift;
constexpr std::false_type kNoShift;

// `Q` is a.Q once more: a pointer that is declared not to alias is what keeps the compiler from waiting for every load into LDS before a transposing read.
template <int D, int KS, bool TREE, int FORM>
__device__ __forceinline__ void decoder_tiles(const DecArgs& a, const bf16_t* __restrict__ Q, int row_blocks, int splits, int chunk) {
  constexpr bool kRaw = FORM == kRawScore || FORM == kRawBiased, kBiased = FORM == kRawBiased || FORM == kAnyBiased;
  constexpr int KB = 64 * KS, RG = 4 / KS, TB = D / 32;
  constexpr int kRows = RG * 32;                           // per workgroup
  constexpr int NSB = 2;                                   // 32-key blocks of a tile per wavefront
  using Lds = DecLds<D, KB>;
  constexpr int kPer = Lds::kTile / 1024 / 4;              // loads per wavefront, tensor and tile
  static_assert(Lds::kTile % 4096 == 0, "whole loads");
  extern __shared__ __align__(16) unsigned char dec_smem[];
  typedef lds_u8_t lds_byte_t;
  typedef __attribute__((address_space(3))) int lds_int_t;
  typedef __attribute__((address_space(3))) int4v_t lds_int4_t;
  lds_byte_t* const Ks = (lds_byte_t*)dec_smem;
  lds_byte_t* const Vs = Ks + Lds::kOffV;
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
  // (m, b, g): divisions in 32 bits, a long one takes a hundred instructions
  const unsigned uhead = id / row_blocks, umb = uhead / a.kv;
  const int g = (int)(uhead % a.kv), b = (int)(umb % a.B);
  const long head = uhead, mb = umb, m = umb / a.B;
  const int group = a.heads / a.kv, R = a.N * group, r0 = rblock * kRows;
  const int L = TREE ? clamp_len(a.len[mb], a.C) : a.len ? clamp_len(a.len[mb], a.N) : a.N;
  const int parts = TREE ? max(1, (L + chunk - 1) / chunk) : 1;           // chunks that this cache fills
  if (split >= parts) return;                              // uniform
  const int there = TREE && a.nodes ? clamp_len(a.nodes[mb], a.N) : a.N;
  const int first = !TREE && a.prefix ? clamp_len(a.prefix[mb], L) : 0;   // keys below it are seen by every row
  const int* doc = !TREE && a.doc ? a.doc + mb * a.N : nullptr;
  const bool keyed = TREE ? kBiased : doc != nullptr;          // a value per key is staged

  const bf16_t* Kp = (const bf16_t*)a.K + m * a.kv_stride_m + (long)b * a.N * a.kv_stride_row + (long)g * a.d;
  const bf16_t* Vp = (const bf16_t*)a.V + m * a.kv_stride_m + (long)b * a.N * a.kv_stride_row + (long)g * a.d;
  const bf16_t* Kh = TREE ? (const bf16_t*)a.Kc + head * a.C * a.d : Kp;
  const bf16_t* Vh = TREE ? (const bf16_t*)a.Vc + head * a.C * a.d : Vp;
  const long stride = TREE ? a.d : a.kv_stride_row;

  // ---- this lane's rows: the B operand of S^T = K Q^T, 8 consecutive features per 16-step
  int token, end, mine, docr;
  uint64_t path;
  float slope;
  bf16x8_t qf[D / 16];
  {
    const int r = r0 + rg * 32 + lq;
    const int i = min(r, R - 1) / group, h = g * group + (min(r, R - 1) - i * group);
    token = i;
    const bf16_t* q = Q + m * a.q_stride_m + ((long)b * a.N + i) * a.q_stride_row + (long)h * a.d;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (r < R && kk * 16 + half * 8 < a.d) v = *reinterpret_cast<const uint4*>(q + kk * 16 + half * 8);
      qf[kk] = __builtin_bit_cast(bf16x8_t, v);
    }
    slope = kBiased ? a.slope[m * a.heads + h] * kLog2e : 0.f;
  }

  int node_at = 0;                                         // position of node `lane`
  int lo = 0, hi = 0, wlo = 0, whi = 0, block_end = 0;     // documents of the workgroup's rows and of this wavefront's, end of the keys that they see
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
      const uint32_t x = __shfl((uint32_t)all, from, kWave), y = __shfl((uint32_t)(all >> 32), from, kWave);
      const int up = __shfl(par, from, kWave);
      if (par >= 0) {
        all |= ((uint64_t)y << 32) | x;
        par = up;
      }
    }
    const int begin = a.start ? a.start[mb] : L;
    node_at = begin + __popcll(all) - 1;
    const uint32_t x = __shfl((uint32_t)all, token, kWave), y = __shfl((uint32_t)(all >> 32), token, kWave);
    path = ((uint64_t)y << 32) | x;
    mine = begin + __popcll(path) - 1;
    end = L;
    docr = 0;
  } else {
    wlo = 0x7fffffff;
    whi = -1;
    const int i = token;
    path = 0;
    mine = i;
    docr = doc ? doc[i] : 0;
    const bool valid = i < L && docr >= 0;
    end = !valid ? 0 : a.causal ? max(i + 1, first) : L;
    wlo = min(wlo, valid ? docr : 0x7fffffff);
    whi = max(whi, valid ? docr : -1);
    const int i_lo = r0 / group, i_hi = min(r0 + kRows, R) - 1;
    block_end = i_lo >= L ? 0 : a.causal ? min(max(i_hi / group + 1, first), L) : L;
    if (doc) {
      wlo = __builtin_amdgcn_readfirstlane(wave_reduce(wlo, MinIntOp{}));
      whi = __builtin_amdgcn_readfirstlane(wave_reduce(whi, MaxIntOp{}));
      if (lane == 0) Key[2 * wave] = wlo, Key[2 * wave + 1] = whi;
      __syncthreads();
      lo = wlo;
      hi = whi;
#pragma unroll
      for (int w = 0; w < 4; ++w) lo = min(lo, Key[2 * w]), hi = max(hi, Key[2 * w + 1]);
      lo = __builtin_amdgcn_readfirstlane(lo);
      hi = __builtin_amdgcn_readfirstlane(hi);
      __syncthreads();
    }
  }
  // tokens of this wavefront's rows
  const int w_lo = (r0 + rg * 32) / group, w_hi = min(r0 + (rg + 1) * 32 - 1, R - 1) / group, block_lo = r0 / group;

  // ---- the tiles: first key of each; the tree's own tile is kTreeTile, none left kNoTile
  constexpr int kTreeTile = -1, kNoTile = -2;
  const int tile_end = TREE ? min(L, (split + 1) * chunk) : block_end;
  // Documents of 16 tiles from win_at on: tiles that hold one of the workgroup's, nothing but its only one; the same for this wavefront.
  uint32_t win_any = 0, win_all = 0, win_mine = 0, win_only = 0;
  int win_at = -(16 * KB);
  auto look = [&](int j0) {
    win_at = j0;
    win_any = win_all = win_mine = win_only = 0;
#pragma unroll 4
    for (int t = 0; t < 16; ++t) {
      if (j0 + t * KB >= tile_end) break;                  // uniform
      uint64_t any = 0, all = ~0ull, own = 0, only = ~0ull;
#pragma unroll
      for (int u = 0; u < (KB + kWave - 1) / kWave; ++u) {
        const int k = u * kWave + lane, j = j0 + t * KB + k, v = doc[min(j, L - 1)];
        const bool in = (j < L) & (k < KB);
        any |= __ballot(in & (v >= lo) & (v <= hi));
        all &= __ballot((in & (v == lo)) | (k >= KB));
        own |= __ballot(in & (v >= wlo) & (v <= whi));
        only &= __ballot((in & (v == wlo)) | (k >= KB));
      }
      win_any |= (any ? 1u : 0u) << t;
      win_all |= (all == ~0ull && lo == hi ? 1u : 0u) << t;
      win_mine |= (own ? 1u : 0u) << t;
      win_only |= (only == ~0ull && wlo == whi ? 1u : 0u) << t;
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
  constexpr int kRowsLeaveOut = 1, kMineLeaveOut = 2, kNoneMine = 4;      // some row of the workgroup, some of this wavefront, all of this wavefront
  auto look_over = [&](int j0) -> int {
    if (j0 == kNoTile) return 0;
    if (j0 == kTreeTile || j0 + KB > L) return kRowsLeaveOut | kMineLeaveOut;
    if (TREE) return 0;
    int what = 0;
    if (a.causal && j0 + KB > first) {
      what |= (j0 + KB > block_lo + 1 ? kRowsLeaveOut : 0) | (j0 + KB > w_lo + 1 ? kMineLeaveOut : 0);
      if (j0 > w_hi && j0 >= first) what |= kNoneMine;
    }
    if (doc) {
      const int t = (j0 - win_at) / KB;
      what |= ((win_all >> t) & 1 ? 0 : kRowsLeaveOut) | ((win_only >> t) & 1 ? 0 : kMineLeaveOut) | ((win_mine >> t) & 1 ? 0 : kNoneMine);
    }
    return what;
  };

  // A lane's place in the loads: its row among those of the load and the piece of it that lands in the lane's 16 bytes (the same one in every load)
  const int my_row = wave * Lds::kRowsPerLoad + lane / Lds::kPieces;
  const int fk = (lane % Lds::kPieces ^ Lds::swz_k(my_row)) * 8, fv = (lane % Lds::kPieces ^ Lds::swz_v(my_row)) * 8;
  int key_reg = 0;
  auto issue = [&](int j0, int stage) {
    const bool own_tile = TREE && j0 == kTreeTile;
    const int base = own_tile ? 0 : j0, limit = (own_tile ? a.N : L) - base;
    const long st = own_tile ? a.kv_stride_row : stride;
    const auto rk = rows_from((own_tile ? Kp : Kh) + base * st), rv = rows_from((own_tile ? Vp : Vh) + base * st);
    const unsigned row = (unsigned)(st * 2), from = my_row * row;
    if (keyed && tid < KB) {
      const int there = base + min(tid, limit - 1);
      key_reg = TREE ? (own_tile ? node_at : a.pos ? a.pos[head * a.C + there] : there) : doc[there];
      if (!TREE && tid >= limit) key_reg = -1;
    }
#pragma unroll
    for (int t = 0; t < kPer; ++t) {
      const bool in = my_row + t * 4 * Lds::kRowsPerLoad < limit;
      const unsigned at = from + t * 4 * Lds::kRowsPerLoad * row;
      load_to_lds(rk, Ks + stage * Lds::kTile + (t * 4 + wave) * 1024, (in & (fk < a.d)) ? at + fk * 2 : kDecOob);
      load_to_lds(rv, Vs + stage * Lds::kTile + (t * 4 + wave) * 1024, (in & (fv < a.d)) ? at + fv * 2 : kDecOob);
    }
  };

  f32x16_t o_acc[TB];
  float mrun, lrun;
  mrun = kLowestScore;
  lrun = 0.f;                                        // this half's partial sum
#pragma unroll
  for (int tb = 0; tb < TB; ++tb)
#pragma unroll
    for (int r = 0; r < 16; ++r) o_acc[tb][r] = 0.f;
  const float sc = a.scale * kLog2e, slope_raw = slope / sc;
  // series of the capped score: used within these bounds, not at all for caps and scales whose powers leave float32 (nor without a cap: 0)
  const float to_u = uniform(a.scale * a.inv_cap), back = uniform(a.cap * kLog2e), u2 = to_u * to_u;
  const float cap1 = uniform(sc * u2 * -0.3333333333333333f), cap2 = uniform(sc * u2 * u2 * 0.13333333333333333f), cap3 = uniform(sc * u2 * u2 * u2 * -0.05396825396825397f);
  const bool series = fabsf(to_u) > 1e-4f && fabsf(to_u) < 1e4f;
  const float cap_short = uniform(series ? kTanhShort / fabsf(to_u) : 0.f), cap_small = uniform(series ? kTanhSeries / fabsf(to_u) : 0.f);
  const float w_short = uniform(cap_short * cap_short), cap23 = uniform(fmaf(w_short, cap3, cap2));

  // ---- one tile is on its way while one is worked on
  int tile = seek(TREE ? split * chunk : 0), seen = look_over(tile);
  if (tile != kNoTile) {
    issue(tile, 0);
    if (keyed && tid < KB) Key[tid] = key_reg;
  }
  int cur = 0, number = 1;
  if (tid == 0) *Flag = 0;
  while (tile != kNoTile) {
    // this tile's loads have landed, and everyone is done with the stage that the next ones go to
    wait_lgkmcnt0();
    wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int next = tile < 0 ? kNoTile : seek(tile + KB), fresh = 1 - cur;
    const int next_seen = look_over(next);
    if (next != kNoTile) issue(next, fresh);

    const bool mask = seen & kMineLeaveOut;
    bool odd_tile = false;
    if (seen & kRowsLeaveOut) {                            // uniform over the workgroup
      bool odd = false;
#pragma unroll
      for (int t = 0; t < kPer; ++t) {
        const u32x4_t v = *(const lds_u32x4_t*)(Vs + cur * Lds::kTile + (t * 4 + wave) * 1024 + lane * 16);
        odd |= bf16_odd(v.x) | bf16_odd(v.y) | bf16_odd(v.z) | bf16_odd(v.w);
      }
      if (odd) *Flag = number;
      wait_lgkmcnt0();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      odd_tile = *Flag == number;
    }
    const bool skip = seen & kNoneMine;                    // no row of this wavefront sees the tile
    if (!skip || odd_tile) {
      const lds_byte_t* Kc = Ks + cur * Lds::kTile + key0 * Lds::kRow;
      const lds_byte_t* Vc = Vs + cur * Lds::kTile + key0 * Lds::kRow;
      const lds_int_t* Kk = Key + cur * KB + key0;
      const int base = (tile == kTreeTile ? 0 : tile) + key0 + 4 * half;          // register r of block sb is key base + 32 sb + 8 (r / 4) + r % 4
      f32x16_t s[NSB];
#pragma unroll
      for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[sb][r] = 0.f;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb) {
          // rows 32 apart are permuted alike
          const bf16x8_t kf = *(const lds_bf16x8_t*)(Kc + (sb * 32 + lq) * Lds::kRow + ((kk * 2 + half) ^ Lds::swz_k(lq)) * 16);
          s[sb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[kk], s[sb], 0, 0, 0);
        }
      keep_ahead<NSB * D / 16, 1>();
      float x[NSB][16];                                    // single values: a branch changes them in place
#pragma unroll
      for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[sb][r] = s[sb][r];
      bf16x8_t pf[NSB][2];
      // Scores x * esc - shift (log2 units, shift the same for a lane's whole tile) to weights.  It stands in each path below that tiles often take: where such paths
      // meet before it, the compiler copies all 32 scores of a lane, 32 of 250 vector instructions (long prompt 1290 -> 1212 us, drafted trees 129 -> 123).
      float corr;
      auto weigh = [&](auto shifted, float shift, float esc) __attribute__((always_inline)) {
        if (mask) {                                        // weight 0 whatever the score
          if (TREE && tile == kTreeTile) {
            const uint64_t bits = path >> (key0 + 4 * half);
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const int c = 32 * sb + 8 * (r / 4) + r % 4;
                x[sb][r] = key0 + 4 * half + c < 64 && ((bits >> c) & 1) ? x[sb][r] : -INFINITY;
              }
          } else {
            const int left = end - base;
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r = 0; r < 16; ++r) x[sb][r] = 32 * sb + 8 * (r / 4) + r % 4 < left ? x[sb][r] : -INFINITY;
            if (!TREE && doc) {
#pragma unroll
              for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) {
                  const int4v_t of = *(const lds_int4_t*)(Kk + sb * 32 + 8 * r4 + 4 * half);
#pragma unroll
                  for (int e = 0; e < 4; ++e) x[sb][4 * r4 + e] = of[e] == docr ? x[sb][4 * r4 + e] : -INFINITY;
                  __builtin_amdgcn_sched_barrier(0);       // 32 documents at a time would take registers from the tile
                }
            }
          }
        }
        float top = -INFINITY;
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
          for (int r = 0; r < 16; ++r) top = fmaxf(top, x[sb][r]);
        top *= esc;
        const float mnew = fmaxf(mrun, across_halves(shifted ? top - shift : top, MaxOp{}));     // the halves' keys are 4 apart, and so are their shifts
        const float less = shifted ? fmaxf(mnew + shift, top) : mnew;          // not below the lane's own maximum, however its sum with a large shift was rounded
        const bool large = fabsf(less) > 0x1p29f && mnew != kLowestScore;       // the rounded maximum may lie far beside such a score: scale first
        if (kRaw && __any(large)) {
          const float by = large ? esc : 1.0f;             // by the row's own maximum: the others' scores keep their bits
#pragma unroll
          for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
            for (int r = 0; r < 16; ++r) x[sb][r] *= by;
          esc = large ? 1.0f : esc;
        }
        corr = __builtin_amdgcn_exp2f(mrun - mnew);
        mrun = mnew;
        float sum = 0.f;
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
          for (int st = 0; st < 2; ++st) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p0 = __builtin_amdgcn_exp2f(fmaf(x[sb][8 * st + 2 * e], esc, -less));
              const float p1 = __builtin_amdgcn_exp2f(fmaf(x[sb][8 * st + 2 * e + 1], esc, -less));
              w[e] = pack_bf16x2(p0, p1);
              sum += p0 + p1;                              // float32 sum of the unrounded weights
            }
            pf[sb][st] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
          }
        lrun = lrun * corr + sum;
      };
      auto bias_table = [&](float by) __attribute__((always_inline)) {           // positions of the tile's keys
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4) {
            const int4v_t at = *(const lds_int4_t*)(Kk + sb * 32 + 8 * r4 + 4 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[sb][4 * r4 + e] = fmaf(-by, fabsf((float)(mine - at[e])), x[sb][4 * r4 + e]);
            __builtin_amdgcn_sched_barrier(0);
          }
      };
      auto bias_behind = [&](float by) __attribute__((always_inline)) {          // no key that a row sees lies behind it: -by (away - c), of which by * away is the shift
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
          for (int r = 0; r < 16; ++r) x[sb][r] = fmaf(by, (float)(32 * sb + 8 * (r / 4) + r % 4), x[sb][r]);
      };
      const float away = (float)(mine - base);
      auto bias_away = [&](float by) __attribute__((always_inline)) {
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
          for (int r = 0; r < 16; ++r) x[sb][r] = fmaf(-by, fabsf(away - (float)(32 * sb + 8 * (r / 4) + r % 4)), x[sb][r]);
      };
      const bool by_table = TREE && (a.pos || tile == kTreeTile), behind = !TREE && a.causal && tile >= first;
      if constexpr (FORM == kRawScore) {
        weigh(kNoShift, 0.f, sc);
      } else if constexpr (FORM == kRawBiased) {
        if (by_table) {
          bias_table(slope_raw);
          weigh(kNoShift, 0.f, sc);
        } else if (behind) {
          bias_behind(slope_raw);
          weigh(kShift, slope * away, sc);
        } else {
          bias_away(slope_raw);
          weigh(kNoShift, 0.f, sc);
        }
      } else {
        constexpr bool kOneWay = TREE && D == 64;          // two copies would spill there
        // A score's form follows from that score alone: the series in the unscaled score below cap_small, the exponential above.  `most`, over all that the tile
        // holds, seen or not, only tells which of them there are.
        float most = 0.f;
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
          for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(x[sb][r]));
        auto by_series = [&](float v) __attribute__((always_inline)) {
          const float w = v * v;
          return v * fmaf(fmaf(fmaf(kBiased ? w : fmaxf(w, w_short), cap3, cap2), w, cap1), w, sc);
        };
        if (!kBiased && __all(most < cap_short)) {         // as a rule: by_series, whose innermost term is cap23 for all of them
#pragma unroll
          for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float w = x[sb][r] * x[sb][r];
              x[sb][r] *= fmaf(fmaf(cap23, w, cap1), w, sc);
            }
          if (!kOneWay) weigh(kNoShift, 0.f, 1.0f);
        } else {
          if (__all(most < cap_small)) {
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r = 0; r < 16; ++r) x[sb][r] = by_series(x[sb][r]);
          } else if (series) {
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const float t = by_series(x[sb][r]), e = tanh_exp(x[sb][r] * to_u) * back;
                x[sb][r] = fabsf(x[sb][r]) < cap_small ? t : e;
                if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);             // 32 of them at a time would take registers from the tile
              }
          } else if (a.cap != 0.f) {
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                x[sb][r] = tanh_either(x[sb][r] * to_u) * back;
                if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);
              }
          } else {
#pragma unroll
            for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
              for (int r = 0; r < 16; ++r) x[sb][r] *= sc;
          }
          if (kBiased) {
            if (by_table) bias_table(slope);
            else bias_away(slope);
          }
          if (!kOneWay) weigh(kNoShift, 0.f, 1.0f);
        }
        if (kOneWay) weigh(kNoShift, 0.f, 1.0f);
      }
      if (__any(corr != 1.0f)) {                         // after the first tiles the maximum of a row seldom moves
#pragma unroll
        for (int tb = 0; tb < TB; ++tb)
#pragma unroll
          for (int r = 0; r < 16; ++r) o_acc[tb][r] *= corr;
      }

      if (odd_tile) {
        int at = lane;                                     // the compiler shall not keep this block's addresses in registers all along
        asm volatile("" : "+v"(at));
        const int up = at / 32;
        // which keys hold such a value: a key per lane
        bool odd = false;
        if (at < KB / KS) {
#pragma unroll 1
          for (int f = 0; f < D; f += 2) odd |= bf16_odd(*(const __attribute__((address_space(3))) uint32_t*)(Vc + at * Lds::kRow + f * 2));
        }
        const uint64_t odd_keys = __ballot(odd);
        uint32_t lo = 0, hi = 0;                         // keys under a weight that is not 0: this half's, then both
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
          for (int st = 0; st < 2; ++st) {
            const uint4 w = __builtin_bit_cast(uint4, pf[sb][st]);
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t bit = (ws[e / 2] >> (e % 2 * 16) & 0x7fffu) != 0 ? 1u << (16 * st + 8 * (e / 4) + e % 4) : 0u;
              if (sb == 0) lo |= bit; else hi |= bit;
            }
          }
        lo <<= 4 * up;
        hi <<= 4 * up;
        lo |= __shfl_xor(lo, 32, kWave);
        hi |= __shfl_xor(hi, 32, kWave);
        const uint64_t under = (uint64_t)hi << 32 | lo;
#pragma unroll 1
        for (uint64_t left = odd_keys; left; left &= left - 1) {
          const int k = __builtin_ctzll(left);
          const bool takes = (under >> k) & 1;
          const lds_byte_t* vr = Vc + k * Lds::kRow + 8 * up;
          const int swz = Lds::swz_v(k);
#pragma unroll
          for (int tb = 0; tb < TB; ++tb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const uint32_t v = *(const lds_bf16_t*)(vr + ((tb * 4 + r / 4) ^ swz) * 16 + r % 4 * 2);
              o_acc[tb][r] += takes & ((v & 0x7f80) == 0x7f80) ? __uint_as_float(v << 16) : 0.f;
              if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);     // more of them at a time would take registers from every tile
            }
        }
        wait_lgkmcnt0();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int t = 0; t < kPer; ++t) {                   // the product runs on the others
          lds_bf16_t* const v = (lds_bf16_t*)(Vs + cur * Lds::kTile + (t * 4 + wave) * 1024 + at * 16);
#pragma unroll 1
          for (int e = 0; e < 8; ++e)
            if ((v[e] & 0x7f80) == 0x7f80) v[e] = 0;
        }
        wait_lgkmcnt0();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
      // O^T += V^T P^T.  In a 16-lane group, lane i points at key row i / 4, features 4 (i % 4) .. + 3 of a 4 x 16 block and receives the
      // 4 keys of feature i; slots 0-3 of step (sb, st) are keys 32 sb + 16 st + 4 half + 0..3, slots 4-7 the same + 8.
#pragma unroll
      for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int tb = 0; tb < TB; ++tb) {
            const int k = sb * 32 + st * 16 + 4 * half + l16 / 4, piece = tb * 4 + lane / 16 % 2 * 2 + l16 % 4 / 2;
            const lds_byte_t* vp = Vc + k * Lds::kRow + (piece ^ Lds::swz_v(l16 / 4)) * 16 + l16 % 2 * 8;       // rows 4 apart are permuted alike
            const s16x4_t lo4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)vp);
            const s16x4_t hi4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(vp + 8 * Lds::kRow));
            const s16x8_t both = __builtin_shufflevector(lo4, hi4, 0, 1, 2, 3, 4, 5, 6, 7);
            o_acc[tb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, both), pf[sb][st], o_acc[tb], 0, 0, 0);
          }
      keep_ahead<NSB * 2 * TB, 2>();
    }
    if (next != kNoTile && keyed && tid < KB) Key[fresh * KB + tid] = key_reg;
    cur = fresh;
    ++number;
    tile = next;
    seen = next_seen;
  }
  __syncthreads();                                         // the stages are free for the shares

  // ---- the result: element r of block tb is feature 32 tb + 8 (r / 4) + 4 half + r % 4
  const bool partial = TREE && parts > 1;
  float* const ml = a.ws + (long)a.M * a.B * a.kv * R * splits * D;
  const int r = r0 + rg * 32 + lq;
  float ltot = across_halves(lrun, AddOp{}), mtot = mrun;
  constexpr int kQuads = 4 * TB / KS;                    // pieces of 4 features that a lane finishes
  const int quad0 = wave / RG * kQuads;
  f32x4_t out[kQuads];
  if constexpr (KS == 1) {
#pragma unroll
    for (int u = 0; u < kQuads; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) out[u][e] = o_acc[u / 4][4 * (u % 4) + e];
  } else {
    lds_f32_t* const buf = (lds_f32_t*)dec_smem;
    lds_f32_t* const max_of = buf + 256 * 16 * TB;
    lds_f32_t* const sum_of = max_of + 256;
    static_assert(256 * 16 * TB * 4 + 2 * 256 * 4 <= Lds::kBytes, "shares fit the stages");
#pragma unroll
    for (int u = 0; u < 4 * TB; ++u) *(lds_f32x4_t*)(buf + (u * 256 + tid) * 4) = f32x4v_t{o_acc[u / 4][4 * (u % 4)], o_acc[u / 4][4 * (u % 4) + 1], o_acc[u / 4][4 * (u % 4) + 2], o_acc[u / 4][4 * (u % 4) + 3]};
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
  if (r >= R) return;
  const bool valid = TREE ? token < there : end > 0;
  const int h = g * group + (r - token * group);
  if (partial) {
    const long at = (head * R + r) * splits + split;
#pragma unroll
    for (int u = 0; u < kQuads; ++u) {
      const int f = 8 * (quad0 + u) + 4 * half;
      *reinterpret_cast<f32x4_t*>(a.ws + at * D + f) = out[u];
    }
    if (quad0 == 0 && half == 0) *reinterpret_cast<float2*>(ml + 2 * at) = make_float2(mtot, ltot);
    return;
  }
  const float inv = valid && ltot != 0.f ? 1.0f / ltot : 0.f;
  const bool none = !valid || ltot == 0.f;
  bf16_t* Op = (bf16_t*)a.O + (mb * a.N + token) * ((long)a.heads * a.d) + (long)h * a.d;
#pragma unroll
  for (int u = 0; u < kQuads; ++u) {
    const int f = 8 * (quad0 + u) + 4 * half;
    if (f < a.d) *reinterpret_cast<uint2*>(Op + f) = none ? make_uint2(0, 0) : make_uint2(pack_bf16x2(out[u][0] * inv, out[u][1] * inv), pack_bf16x2(out[u][2] * inv, out[u][3] * inv));
  }
  if (TREE && a.lse && quad0 == 0 && half == 0) a.lse[(mb * a.N + token) * a.heads + h] = none ? -INFINITY : (mtot + __builtin_amdgcn_logf(ltot)) * kLn2;
}

template <int D, int KS, bool TREE, int FORM>
__global__ __launch_bounds__(256, D == 64 ? 3 : D == 128 ? 2 : 1) void decoder_tiles_kernel(DecArgs a, int row_blocks, int splits, int chunk) {
  decoder_tiles<D, KS, TREE, FORM>(a, (const bf16_t*)a.Q, row_blocks, splits, chunk);
}

// Sums of the chunks of one row: D / 4 lanes hold its features, 4 each, and SHARE such groups of lanes take every SHARE-th chunk.  Maxima and sums in log2
// units where LOG2, natural ones otherwise.
template <typename T, int D, bool LOG2, int SHARE>
__global__ __launch_bounds__(256) void decoder_join_kernel(DecArgs a, int splits, int chunk) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes, kRows = kGroups / SHARE;
  static_assert(SHARE == 1 || SHARE == kGroups, "a group per row, or all of them on one");
  const int lane = threadIdx.x % kLanes, grp = threadIdx.x / kLanes;
  const int group = a.heads / a.kv, R = a.N * group;
  const unsigned urow = blockIdx.x * (unsigned)kRows + (SHARE == 1 ? grp : 0);  // fewer than 2^31 rows
  if (urow >= (unsigned)(a.M * a.B * a.kv) * R) return;
  const unsigned uhead = urow / R, umb = uhead / a.kv;
  const long row = urow, mb = umb;
  const int r = (int)(urow % R), i = r / group, h = (int)(uhead % a.kv) * group + r % group;
  const int parts = (clamp_len(a.len[mb], a.C) + chunk - 1) / chunk;
  if (parts <= 1) return;                                  // written already; uniform where groups share a row
  const float* o = a.ws + row * splits * D + lane * 4;
  const float2* ml = reinterpret_cast<const float2*>(a.ws + (long)a.M * a.B * a.kv * R * splits * D) + row * splits;
  // Up to 8 chunks one group takes them all, in this form too: the order of the sums follows from the length, not from the capacity.
  const bool split_up = SHARE > 1 && parts > 8;
  const int first = SHARE == 1 ? 0 : split_up ? grp : grp == 0 ? 0 : parts, step = split_up ? SHARE : 1;
  f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float top = kLowestScore, sum = 0.f;
  for (int k0 = first; k0 < parts; k0 += 8 * step) {       // 8 loads of each kind at a time
    float2 p[8];
    f32x4_t v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int k = min(k0 + u * step, parts - 1);
      p[u] = ml[k];
      v[u] = *reinterpret_cast<const f32x4_t*>(o + (long)k * D);
    }
    // a chunk that is not there is left out by a select, its sums too: these may be infinite, and 0 times them NaN
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bool there = k0 + u * step < parts;
      p[u].x = there ? p[u].x : kLowestScore;
      p[u].y = there ? p[u].y : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[u][e] = there ? v[u][e] : 0.f;
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
      const float c = LOG2 ? __builtin_amdgcn_exp2f(p[u].x - top) : expf(p[u].x - top);
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
