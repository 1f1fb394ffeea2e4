// Full attention over packed sequences, backward (include/spt_attn.h): two launches, both without atomics.
//
//   prompt_bwd_q_kernel   the forward's decomposition (a wavefront owns 32 query rows, keys pass through LDS): S^T and dP^T as products
//                         with the query side in registers, dS^T in registers, dQ^T += K^T dS^T.  D = dy.y comes from a Y that was rounded to bf16 and
//                         computed with weights that were, and where one key has nearly all the weight dS is what is left of dP - D
//                         when they cancel.  The sum of a row's dS, 0 but for that, says by how much D is off: dq gets
//                         that times sum_j p_j k_j (a product more on operands that are there) taken off, and the second
//                         launch gets the corrected D.  Without it dQ and dK were 5e-3 off (2-norm, queries that prefer a key; 32 heads of 64,
//                         512 tokens), with it 2.4e-3.
//   prompt_bwd_kv_kernel  a wavefront owns 32 keys of a key head, the queries of all heads of its group pass through LDS in tiles
//                         of 32, heads outermost, so a gradient is summed in one fixed order: S and dP with the key side in
//                         registers, dV^T += dY^T P, dK^T += Q^T dS.
// Where there is little to do, four or eight groups of wavefronts share what passes through LDS for the same 32 or 64 rows, and their sums are
// added in order.
// S and dP are formed in both: the alternative, keeping dS or partial dQ in memory, moves as many bytes as it saves time.
// P goes into dV's product as one bf16: dV is 2.3e-3 off (2-norm), as dK is with dS so, where its own rounding makes 1.66e-3.  As the sum of two
// 1.66e-3, key side 71 and 77 us (16 sequences of 512, 32 heads of 64), 495 and 575 (six of 500 to 4000, 32 heads of 128 on 8).
#include <algorithm>
#include <type_traits>

#include "attn_common.hpp"

using namespace spt;

namespace {

constexpr int kTile = 32;                   // rows of a tile that passes through LDS; rows of a wavefront
constexpr int kRing = 2;                    // tiles in LDS: one in use, one being filled

struct BwdArgs {
  AttnRows Q, K, V, Y, dY, dQ, dK, dV;
  const int32_t *cu_q, *cu_k;
  const float* lse;
  float *off, *neg_d;             // [H][Tq]: row_offset(lse), -D
  int B, Tq, Tk, Hk, G, hshift;
  int causal, coarse;
  float c, scale;
};

// exp2 argument's subtrahend of a row: rows without a key have lse = -inf and p = 0
__device__ __forceinline__ float row_offset(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

// P and dS of 32 x 32 pairs as operands of the second products: a lane's results 8 half .. 8 half + 7.  EXACT: dS is the sum of two bf16.
template <bool EXACT>
struct Weights { u32x4 p[2], ds[2]; };
template <>
struct Weights<true> { u32x4 p[2], ds[2], rest[2]; };

// Where sequences are short, a rounding of one dS is in a whole row of a gradient, and memory takes as long as the products do; where there
// are few rows in all, a gradient's error is that of a few of them, and the launch takes as long as it does.  dS is then exact.
// Error of dK against 64 bits as a multiple of that of rounding it once, shapes drawn: 1.7 for sequences of two tokens, 1.5 for
// up to 80, 1.45 for longer ones, 1.0 exact.  Key side, us, rounded and exact: 8192 tokens, 32 heads of 128 on 8: sequences of 32 95 and 99,
// of 64 71 and 75, of 128 61 and 65; 32 heads of 64: 57 and 58, 44 and 47, 46 and 48, of 512 67 and 76.
constexpr int kFewRows = 128;     // of queries of a sequence and key head, on average
constexpr int kFewTiles = 256;    // of 32 queries and a head, in all

// p and dS of one pair, from its rows in memory.
struct PairGrad { float p, ds; };
__device__ __forceinline__ PairGrad pair_grad(const char* q, const char* k, const char* dy, const char* v, int dh, float c, float off, float D) {
  const float p = __builtin_amdgcn_exp2f(fmaf(row_dot(q, k, dh), c, -off));
  return {p, p * (row_dot(dy, v, dh) - D)};
}

// Rows q0 .. q0 + 31 of two tensors of n rows into a pair of tiles (rows past the end: the last one again), by WAVES wavefronts.
template <int DH, int WAVES>
__device__ __forceinline__ void fetch_pair(int tid, const char* x, int64_t xrow, const char* y, int64_t yrow, int q0, int n, const char* tiles, int wave) {
  constexpr int COPIES = kTile * (DH / 8) / (64 * WAVES);
  const char* xb = x + q0 * xrow;
  const char* yb = y + q0 * yrow;
#pragma unroll
  for (int u = 0; u < COPIES; ++u) {
    const int slot = u * 64 * WAVES + tid, r0 = slot / (DH / 8);
    const uint32_t chunk = ((slot % (DH / 8)) ^ row_swizzle<DH>(r0)) * 16, r = (uint32_t)min(r0, n - 1 - q0);
    const uint32_t at = lds_addr(tiles + (u * WAVES + wave) * 1024);
    dma16_at(xb, r * (uint32_t)xrow + chunk, at);
    dma16_at(yb, r * (uint32_t)yrow + chunk, at + kTile * DH * 2);
  }
}

// A row of dQ the plain way, over the n keys that it sees: lanes take keys for the pairs, dims for the sums.  Returns what D lacks,
// the sum of the row's dS, and takes it off as the other rows do: times the mean of the keys.
template <int DH>
__device__ __forceinline__ float slow_dq_row(const BwdArgs& a, const char* q, const char* dy, const char* k, const char* v, int n, float off,
                                             float D, char* dq) {
  const int lane = threadIdx.x & 63;
  float acc[DH / 64] = {}, mean[DH / 64] = {}, left_over = 0.f, mass = 0.f;
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane;
    PairGrad x = {0.f, 0.f};
    if (j < n) x = pair_grad(q, k + j * a.K.row, dy, v + j * a.V.row, DH, a.c, off, D);
    left_over += x.ds;
    mass += x.p;
    for (int e = 0; e < min(64, n - j0); ++e) {
      const float p = __shfl(x.p, e), ds = __shfl(x.ds, e);
#pragma unroll
      for (int d = 0; d < DH / 64; ++d) {
        const float kd = bf16_at(k + (j0 + e) * a.K.row + (lane + 64 * d) * 2);
        acc[d] = fmaf(ds, kd, acc[d]);
        mean[d] = fmaf(p, kd, mean[d]);
      }
    }
  }
  left_over = wave_sum(left_over);
  mass = wave_sum(mass);
  const float off_by = mass > 0.f ? left_over / mass : 0.f;
#pragma unroll
  for (int d = 0; d < DH / 64; ++d) reinterpret_cast<uint16_t*>(dq)[lane + 64 * d] = (uint16_t)pack_bf16x2(fmaf(-off_by, mean[d], acc[d]) * a.scale, 0.f);
  return left_over;
}

// Sizes of a workgroup of GROUPS groups of OWNERS wavefronts.  A wavefront of a group owns 32 rows, the groups go through every GROUPS-th
// tile for the same rows.
template <int DH, int OWNERS, int GROUPS>
struct BwdSizes {
  static constexpr int TILE_BYTES = kTile * DH * 2, SHIFT = OWNERS == 8 ? 8 : OWNERS == 4 ? 7 : OWNERS == 2 ? 6 : 5, THREADS = 64 * OWNERS * GROUPS;   // 1 << SHIFT: rows
  // 128-wide heads: a row operand of the wavefront's own stays in LDS, or two wavefronts would not fit into a SIMD's registers
  static constexpr bool OWN = DH == 128;
  static constexpr int OWN_BYTES = OWN ? OWNERS * TILE_BYTES : 0;
  static constexpr int SUMS = (GROUPS - 1) * OWNERS * DH * 128;                 // a gradient of the other groups
  static constexpr int Q_RING = kRing * 2 * TILE_BYTES;                         // of a group: tiles of K and V
  static constexpr int Q_JOIN = SUMS + (GROUPS - 1) * OWNERS * 768, Q_RINGS = GROUPS * Q_RING + OWN_BYTES;
  static constexpr int Q_SMEM = Q_RINGS > Q_JOIN ? Q_RINGS : Q_JOIN;
  static constexpr int KV_RING = kRing * (2 * TILE_BYTES + 256);                // tiles of Q and dY, their rows' offsets and -D
  static constexpr int KV_SMEM = GROUPS * KV_RING + OWN_BYTES;
  static_assert(Q_SMEM <= 160 * 1024 && KV_SMEM <= 160 * 1024 && SUMS <= GROUPS * KV_RING, "a CU's LDS");
};

// The other groups' sums of `sum` (and of two numbers a lane) are added to the first's, in order.  All wavefronts of the workgroup.
template <int DH, int OWNERS, int GROUPS>
__device__ __forceinline__ void add_groups(f32x16* sum, char* smem, int wave, int group, int lane) {
  constexpr int DT = DH / 32;
  float* mine = reinterpret_cast<float*>(smem) + ((group - 1) * OWNERS + wave) * (DT * 1024) + lane * 4;
  __syncthreads();
  if (group > 0) {
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(mine + (d * 4 + q) * 256) = f32x4{sum[d][4 * q], sum[d][4 * q + 1], sum[d][4 * q + 2], sum[d][4 * q + 3]};
  }
  __syncthreads();
  if (group == 0) {
#pragma unroll 1
    for (int g = 1; g < GROUPS; ++g) {
      const float* half = reinterpret_cast<float*>(smem) + ((g - 1) * OWNERS + wave) * (DT * 1024) + lane * 4;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(half + (d * 4 + q) * 256);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[d][4 * q + e] += x[e];
        }
    }
  }
}

template <int DH, int OWNERS, int GROUPS, bool EXACT>
__global__ __launch_bounds__((64 * OWNERS * GROUPS), 2) void prompt_bwd_q_kernel(const BwdArgs a) {
  typedef BwdSizes<DH, OWNERS, GROUPS> Sizes;
  constexpr int KS = DH / 16, DT = DH / 32, TILE_BYTES = Sizes::TILE_BYTES;
  constexpr bool OWN = Sizes::OWN;
  extern __shared__ __align__(256) char smem[];
  const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5, tid = threadIdx.x % (64 * OWNERS);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % OWNERS, group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / OWNERS;
  char* ring = smem + group * Sizes::Q_RING;
  const int hsets = a.G >> a.hshift, pshift = Sizes::SHIFT - a.hshift;
  const HeadItem w = head_item(blockIdx.x, a.Hk);
  const int hk = w.hk, hs = w.item % hsets;
  TilePlace at;
  if (!find_tile<false>(a.cu_q, a.cu_k, a.B, a.Tq, a.Tk, pshift, a.causal, a.coarse, w.item / hsets, at)) return;
  const int tile = at.tile;
  const SeqRows sq = at.own, sk = at.other;
  const int nq = sq.n, nk = sk.n, ahead = nk - nq;
  const int head = hk * a.G + (hs << a.hshift) + (wave & ((1 << a.hshift) - 1));
  const int p0 = (tile << pshift), i0 = p0 + (wave >> a.hshift) * 32;
  const int last = min(nq, p0 + (1 << pshift)) - 1;
  const int kend = a.causal ? min(nk, last + ahead + 1) : nk;
  const int wave_kend = i0 >= nq ? 0 : a.causal ? min(nk, min(nq, i0 + 32) + ahead) : nk;
  const int wave_full = i0 >= nq ? 0 : a.causal ? min(nk, i0 + ahead + 1) : nk;
  const int mine = min(i0 + i, nq - 1);
  const int seen = a.causal ? min(nk, mine + ahead + 1) : nk;
  const int ntile = kend > 0 ? (kend + kTile - 1) / kTile : 0;
  const int full = max(0, a.causal ? min(nk, p0 + ahead + 1) : nk);     // keys that all queries of the workgroup see

  const char* kbase = a.K.p + (int64_t)sk.first * a.K.row + (int64_t)hk * a.K.head;
  const char* vbase = a.V.p + (int64_t)sk.first * a.V.row + (int64_t)hk * a.V.head;
  auto fetch = [&](int t, int buf) { fetch_pair<DH, OWNERS>(tid, kbase, a.K.row, vbase, a.V.row, t * kTile, nk, ring + buf * 2 * TILE_BYTES, wave); };
  if (group < ntile) fetch(group, 0);

  const int64_t row = sq.first + mine;
  const char* qrow = a.Q.p + row * a.Q.row + (int64_t)head * a.Q.head;
  const char* yrow = a.Y.p + row * a.Y.row + (int64_t)head * a.Y.head;
  const char* dyrow = a.dY.p + row * a.dY.row + (int64_t)head * a.dY.head;
  bf16x8 qf[KS], dyf[OWN ? 1 : KS];
  TileReader<DH> lds(lane);
  const uint32_t tiles = lds_addr(ring), own = lds_addr(smem) + GROUPS * Sizes::Q_RING + wave * TILE_BYTES;
  float D = 0.f;
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    qf[s] = *reinterpret_cast<const bf16x8*>(qrow + s * 32 + h * 16);
    const u32x4 dy = *reinterpret_cast<const u32x4*>(dyrow + s * 32 + h * 16), y = *reinterpret_cast<const u32x4*>(yrow + s * 32 + h * 16);
    if (OWN) {   // (every group the same)
      *reinterpret_cast<u32x4*>(smem + GROUPS * Sizes::Q_RING + wave * TILE_BYTES + (lds.row ^ (uint32_t)(s * 32))) = dy;
    } else {
      dyf[s] = as_bf16x8(dy);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) D = fmaf(hi_bf16(dy[e]), hi_bf16(y[e]), fmaf(lo_bf16(dy[e]), lo_bf16(y[e]), D));
  }
  D += other_half(D);
  const float off = row_offset(a.lse[(int64_t)head * a.Tq + row]);

  f32x16 o[DT], mean[DT];                                // sums of dS k and of p k
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = mean[d][r] = 0.f;
  float left_over = 0.f, rounded = 0.f, mass = 0.f;      // sum of dS: what D lacks; of dS, of p (EXACT) as rounded
  NotFinite not_finite;

  auto first_products = [&](uint32_t kt, f32x16& s, f32x16& dp) {
    lds.fresh();
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds.rows(kt, 0, ks), qf[ks], s, 0, 0, 0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds.rows(kt + TILE_BYTES, 0, ks), OWN ? lds.rows(own, 0, ks) : dyf[OWN ? 0 : ks], dp, 0, 0, 0);
  };
  auto weights = [&](int t, f32x16& s, f32x16& dp, bool masked) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = fmaf(s[r], a.c, -off);
      dp[r] -= D;
    }
    if (masked) {
      const int left = seen - t * kTile - 4 * h;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const bool sees = 8 * (r >> 2) + (r & 3) < left;
        s[r] = sees ? s[r] : -INFINITY;
        dp[r] = sees ? dp[r] : 0.f;
      }
    }
    Weights<EXACT> w;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float p0 = __builtin_amdgcn_exp2f(s[r]), p1 = __builtin_amdgcn_exp2f(s[r + 1]), d0 = p0 * dp[r], d1 = p1 * dp[r + 1];
      left_over += d0 + d1;
      const uint32_t d = pack_bf16x2(d0, d1);
      w.p[r >> 3][(r & 7) >> 1] = pack_bf16x2(p0, p1);
      w.ds[r >> 3][(r & 7) >> 1] = d;
      if constexpr (EXACT) {
        w.rest[r >> 3][(r & 7) >> 1] = pack_bf16x2(d0 - lo_bf16(d), d1 - hi_bf16(d));
        mass = sum2(w.p[r >> 3][(r & 7) >> 1], mass);
      } else {
        rounded = sum2(d, rounded);
      }
    }
    return w;
  };
  auto second_products = [&](uint32_t kt, const Weights<EXACT>& w) {
    lds.fresh();
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const bf16x8 f = lds.columns(kt, half, d);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, as_bf16x8(w.ds[half]), o[d], 0, 0, 0);
        if constexpr (EXACT) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, as_bf16x8(w.rest[half]), o[d], 0, 0, 0);
        mean[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, as_bf16x8(w.p[half]), mean[d], 0, 0, 0);
      }
  };
  for (int t0 = 0; t0 < ntile; t0 += GROUPS) {
    wait_vmcnt<0>();                                     // the group's tile is there; asks for its next one
    __syncthreads();
    const int t = t0 + group, buf = t0 / GROUPS % kRing, j0 = t * kTile;
    const uint32_t kt = tiles + buf * 2 * TILE_BYTES;
    if (t + GROUPS < ntile) fetch(t + GROUPS, buf ^ 1);
    if (t >= ntile) continue;
    if (j0 + kTile > full) {
#pragma unroll
      for (int u = 0; u < TILE_BYTES / (1024 * OWNERS); ++u) not_finite.look(lds_read<u32x4>(kt + u * 1024 * OWNERS + tid * 16));
    }
    if (j0 >= wave_kend) continue;
    const bool masked = j0 + kTile > wave_full;
    __builtin_amdgcn_iglp_opt(1);                        // (reads of LDS between the products: see the forward)
    f32x16 s, dp;
    first_products(kt, s, dp);
    second_products(kt, weights(t, s, dp, masked));
  }
  left_over += other_half(left_over);
  rounded = EXACT ? left_over : rounded + other_half(rounded);
  if (EXACT) mass += other_half(mass);
  const int64_t stat = (int64_t)head * a.Tq;
  // rows that not all queries may see hold infinities or NaN: 0 times those is NaN
  if (full < ntile * kTile && __syncthreads_or(not_finite.found())) {
    for (int r = group; r < min(32, nq - i0); r += GROUPS) {
      const int64_t at = sq.first + i0 + r;
      const float Dr = __shfl(D, r), offr = __shfl(off, r);
      const float left = slow_dq_row<DH>(a, a.Q.p + at * a.Q.row + (int64_t)head * a.Q.head, a.dY.p + at * a.dY.row + (int64_t)head * a.dY.head, kbase, vbase,
                                         a.causal ? min(nk, i0 + r + ahead + 1) : nk, offr, Dr, a.dQ.p + at * a.dQ.row + (int64_t)head * a.dQ.head);
      if (lane == 0) {
        a.off[stat + at] = offr;
        a.neg_d[stat + at] = -(Dr + left);
      }
    }
    return;
  }
  if (GROUPS > 1) {
    add_groups<DH, OWNERS, GROUPS>(o, smem, wave, group, lane);
    add_groups<DH, OWNERS, GROUPS>(mean, smem, wave, group, lane);
    float* rest = reinterpret_cast<float*>(smem + Sizes::SUMS) + wave * 192 + lane;
    if (group > 0) {
      float* mine = rest + (group - 1) * OWNERS * 192;
      mine[0] = left_over;
      mine[64] = rounded;
      mine[128] = mass;
    }
    __syncthreads();
    if (group > 0) return;
    for (int g = 0; g < GROUPS - 1; ++g) {
      left_over += rest[g * OWNERS * 192];
      rounded += rest[g * OWNERS * 192 + 64];
      mass += rest[g * OWNERS * 192 + 128];
    }
  }
  if (i0 + i >= nq) return;
  if (h == 0) {
    a.off[stat + row] = off;
    a.neg_d[stat + row] = -(D + left_over);
  }
  // the p of `mean` were rounded: where one key has nearly all the weight, their sum is off by what that key's share is
  const float off_by = EXACT && mass > 0.f ? rounded / mass : rounded;
  char* dq = a.dQ.p + row * a.dQ.row + (int64_t)head * a.dQ.head + h * 32;
#pragma unroll
  for (int d = 0; d < DT; ++d) {
    float v[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = fmaf(-off_by, mean[d][r], o[d][r]) * a.scale;
    *reinterpret_cast<bf16x8*>(dq + d * 64) = pack8(v);
    *reinterpret_cast<bf16x8*>(dq + d * 64 + 16) = pack8(v + 8);
  }
}

// Both gradients of one key: lanes take queries for the pairs, dims for the sums.
template <int DH>
__device__ __forceinline__ void slow_dkv_row(const BwdArgs& a, const SeqRows& sq, int hk, int first, const char* k, const char* v, char* dk, char* dv) {
  const int lane = threadIdx.x & 63;
  float ak[DH / 64] = {}, av[DH / 64] = {};
  for (int g = 0; g < a.G; ++g) {
    const int head = hk * a.G + g;
    const char* q = a.Q.p + (int64_t)sq.first * a.Q.row + (int64_t)head * a.Q.head;
    const char* dy = a.dY.p + (int64_t)sq.first * a.dY.row + (int64_t)head * a.dY.head;
    const int64_t stat = (int64_t)head * a.Tq + sq.first;
    for (int i0 = first; i0 < sq.n; i0 += 64) {
      const int i = i0 + lane;
      PairGrad x = {0.f, 0.f};
      if (i < sq.n) x = pair_grad(q + i * a.Q.row, k, dy + i * a.dY.row, v, DH, a.c, a.off[stat + i], -a.neg_d[stat + i]);
      for (int e = 0; e < min(64, sq.n - i0); ++e) {
        const float p = __shfl(x.p, e), ds = __shfl(x.ds, e);
#pragma unroll
        for (int d = 0; d < DH / 64; ++d) {
          av[d] = fmaf(p, bf16_at(dy + (i0 + e) * a.dY.row + (lane + 64 * d) * 2), av[d]);
          ak[d] = fmaf(ds, bf16_at(q + (i0 + e) * a.Q.row + (lane + 64 * d) * 2), ak[d]);
        }
      }
    }
  }
#pragma unroll
  for (int d = 0; d < DH / 64; ++d) {
    reinterpret_cast<uint16_t*>(dk)[lane + 64 * d] = (uint16_t)pack_bf16x2(ak[d] * a.scale, 0.f);
    reinterpret_cast<uint16_t*>(dv)[lane + 64 * d] = (uint16_t)pack_bf16x2(av[d], 0.f);
  }
}

template <int DH, int OWNERS, int GROUPS, bool EXACT>
__global__ __launch_bounds__((64 * OWNERS * GROUPS), 2) void prompt_bwd_kv_kernel(const BwdArgs a) {
  typedef BwdSizes<DH, OWNERS, GROUPS> Sizes;
  constexpr int KS = DH / 16, DT = DH / 32, TILE_BYTES = Sizes::TILE_BYTES, OWN_KEYS = kTile * OWNERS;
  constexpr bool OWN = Sizes::OWN;
  extern __shared__ __align__(256) char smem[];
  const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5, tid = threadIdx.x % (64 * OWNERS);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % OWNERS, group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / OWNERS;
  char* ring = smem + group * Sizes::KV_RING;
  float* stats = reinterpret_cast<float*>(ring + kRing * 2 * TILE_BYTES);
  const HeadItem w = head_item(blockIdx.x, a.Hk);
  const int hk = w.hk;
  TilePlace place;
  if (!find_tile<true>(a.cu_k, a.cu_q, a.B, a.Tk, a.Tq, Sizes::SHIFT, a.causal, a.coarse, w.item, place)) return;
  const int tile = place.tile;
  const SeqRows sk = place.own, sq = place.other;
  const int nq = sq.n, nk = sk.n, ahead = nk - nq;
  const int j0 = tile * OWN_KEYS + wave * 32, mine = min(j0 + i, nk - 1);
  const int first = a.causal ? max(0, mine - ahead) : 0;                 // the first query that sees the lane's key
  const int begin = a.causal ? max(0, tile * OWN_KEYS - ahead) & ~(kTile - 1) : 0;
  // Tiles of a head from `begin` on: in front of `full` some query does not see some key of the workgroup, the last one may be
  // short, the others need no mask.  Steps: the masked tiles of all heads, then the others.
  const int full = a.causal ? max(begin, (tile * OWN_KEYS + OWN_KEYS - 1 - ahead + kTile - 1) & ~(kTile - 1)) : 0;
  const int tail = nq & ~(kTile - 1), front = max(0, min(full, nq) - begin + kTile - 1) / kTile;
  const int head_masked = front + (tail < nq && tail >= full), head_full = max(0, tail - full) / kTile;
  const int masked_steps = head_masked * a.G, steps = masked_steps + head_full * a.G;
  const int wave_begin = a.causal ? j0 - ahead - (kTile - 1) : 0;        // tiles from here on have a query that sees a key of the wavefront

  struct Place { int g, x; };                                            // a step's head, and its tile among the masked or the others
  auto first_query = [&](int t, const Place& p) { return t >= masked_steps ? full + p.x * kTile : p.x < front ? begin + p.x * kTile : tail; };
  auto after = [&](int t, const Place& p) {
    if (p.x + 1 < (t < masked_steps ? head_masked : head_full)) return Place{p.g, p.x + 1};
    return t + 1 == masked_steps ? Place{0, 0} : Place{p.g + 1, 0};
  };
  auto fetch = [&](int t, const Place& p) {
    const int head = hk * a.G + p.g, q0 = first_query(t, p), buf = t / GROUPS % kRing;
    fetch_pair<DH, OWNERS>(tid, a.Q.p + (int64_t)sq.first * a.Q.row + (int64_t)head * a.Q.head, a.Q.row,
                   a.dY.p + (int64_t)sq.first * a.dY.row + (int64_t)head * a.dY.head, a.dY.row, q0, nq, ring + buf * 2 * TILE_BYTES, wave);
    const int64_t at = (int64_t)head * a.Tq + sq.first + q0 + min(i, nq - 1 - q0);
    if (wave == 0) dma4(h ? a.neg_d + at : a.off + at, lds_addr(stats + buf * 64));
  };
  // the group's steps: group, group + GROUPS, ...
  Place here = {0, 0}, coming;
  for (int n = 0; n < group; ++n) here = after(n, here);
  coming = here;
  if (group < steps) fetch(group, here);

  bf16x8 kf[KS], vf[OWN ? 1 : KS];
  TileReader<DH> lds(lane);
  const uint32_t tiles = lds_addr(ring), own = lds_addr(smem) + GROUPS * Sizes::KV_RING + wave * TILE_BYTES;
  char* own_tile = smem + GROUPS * Sizes::KV_RING + wave * TILE_BYTES;
  if (!OWN) {
    const char* krow = a.K.p + (int64_t)(sk.first + mine) * a.K.row + (int64_t)hk * a.K.head;
    const char* vrow = a.V.p + (int64_t)(sk.first + mine) * a.V.row + (int64_t)hk * a.V.head;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      kf[s] = *reinterpret_cast<const bf16x8*>(krow + s * 32 + h * 16);
      vf[OWN ? 0 : s] = *reinterpret_cast<const bf16x8*>(vrow + s * 32 + h * 16);
    }
  } else {
    // as whole lines: K and then V through the wavefronts' tiles (the first group fetches K, the last one V; 32 heads of their own
    // keys, 16 sequences of 512: 203 us with a lane's own row, 174 so; 64-wide heads lose, 164 and 173)
    const int64_t row0 = sk.first + min(j0, nk - 1);
    const int own_rows = max(nk - j0, 1);
    RowPieces<DH> v;
    if (group == 0) fetch_rows<DH>(a.K.p + row0 * a.K.row + (int64_t)hk * a.K.head, a.K.row, own_rows, own, lane);
    if (group == GROUPS - 1) v.load(a.V.p + row0 * a.V.row + (int64_t)hk * a.V.head, a.V.row, own_rows, lane);
    wait_vmcnt<0>();
    wave_lds_fence();
    if (GROUPS > 1) __syncthreads();
#pragma unroll
    for (int s = 0; s < KS; ++s) kf[s] = lds.rows(own, 0, s);
    wave_lds_fence();
    if (GROUPS > 1) __syncthreads();
    if (group == GROUPS - 1) v.put(own_tile, lane);
    wave_lds_fence();
  }
  f32x16 ok[DT], ov[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) ok[d][r] = ov[d][r] = 0.f;
  NotFinite not_finite;

  auto first_products = [&](int buf, f32x16& s, f32x16& dp) {
    const uint32_t qt = tiles + buf * 2 * TILE_BYTES;
    lds.fresh();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 d = *reinterpret_cast<const f32x4*>(stats + buf * 64 + 32 + 8 * q + 4 * h);   // (dP starts from -D)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[4 * q + e] = 0.f;
        dp[4 * q + e] = d[e];
      }
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds.rows(qt, 0, ks), kf[ks], s, 0, 0, 0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds.rows(qt + TILE_BYTES, 0, ks), OWN ? lds.rows(own, 0, ks) : vf[OWN ? 0 : ks], dp, 0, 0, 0);
  };
  auto weights = [&](int buf, int q0, f32x16& s, f32x16& dp, bool masked) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 off = *reinterpret_cast<const f32x4*>(stats + buf * 64 + 8 * q + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[4 * q + e] = fmaf(s[4 * q + e], a.c, -off[e]);
    }
    if (masked) {
      const int from = first - q0 - 4 * h, to = nq - q0 - 4 * h;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int at = 8 * (r >> 2) + (r & 3);
        const bool sees = at >= from && at < to;
        s[r] = sees ? s[r] : -INFINITY;
        dp[r] = sees ? dp[r] : 0.f;
      }
    }
    Weights<EXACT> w;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float p0 = __builtin_amdgcn_exp2f(s[r]), p1 = __builtin_amdgcn_exp2f(s[r + 1]), d0 = p0 * dp[r], d1 = p1 * dp[r + 1];
      const uint32_t d = pack_bf16x2(d0, d1);
      w.p[r >> 3][(r & 7) >> 1] = pack_bf16x2(p0, p1);
      w.ds[r >> 3][(r & 7) >> 1] = d;
      if constexpr (EXACT) w.rest[r >> 3][(r & 7) >> 1] = pack_bf16x2(d0 - lo_bf16(d), d1 - hi_bf16(d));
    }
    return w;
  };
  auto second_products = [&](int buf, const Weights<EXACT>& w) {
    const uint32_t qt = tiles + buf * 2 * TILE_BYTES;
    lds.fresh();
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        ov[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds.columns(qt + TILE_BYTES, half, d), as_bf16x8(w.p[half]), ov[d], 0, 0, 0);
        const bf16x8 q = lds.columns(qt, half, d);
        ok[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, as_bf16x8(w.ds[half]), ok[d], 0, 0, 0);
        if constexpr (EXACT) ok[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, as_bf16x8(w.rest[half]), ok[d], 0, 0, 0);
      }
  };
  for (int t0 = 0; t0 < steps; t0 += GROUPS) {
    wait_vmcnt<0>();                                                     // the step's tiles are there; asks for the next one's
    __syncthreads();
    const int t = t0 + group, buf = t0 / GROUPS % kRing;
    if (t + GROUPS < steps) {
#pragma unroll
      for (int n = 0; n < GROUPS; ++n) coming = after(t + n, coming);
      fetch(t + GROUPS, coming);
    }
    if (t >= steps) continue;
    const int q0 = first_query(t, here);
    here = coming;
    const bool masked = t < masked_steps;
    if (masked) {
#pragma unroll
      for (int u = 0; u < 2 * TILE_BYTES / (1024 * OWNERS); ++u) not_finite.look(lds_read<u32x4>(tiles + buf * 2 * TILE_BYTES + u * 1024 * OWNERS + tid * 16));
    }
    if (q0 < wave_begin) continue;
    const bool cut = masked && ((a.causal && q0 < j0 + 31 - ahead) || q0 + kTile > nq);   // (some query of the tile does not see some key of the wavefront)
    __builtin_amdgcn_iglp_opt(1);                                        // (reads of LDS between the products: see the forward)
    f32x16 s, dp;
    first_products(buf, s, dp);
    second_products(buf, weights(buf, q0, s, dp, cut));
  }
  // rows that not all keys may see hold infinities or NaN: 0 times those is NaN
  if (masked_steps > 0 && __syncthreads_or(not_finite.found())) {
    for (int r = group; r < min(32, nk - j0); r += GROUPS) {
      const int64_t at = sk.first + j0 + r;
      slow_dkv_row<DH>(a, sq, hk, a.causal ? max(0, j0 + r - ahead) : 0, a.K.p + at * a.K.row + (int64_t)hk * a.K.head,
                       a.V.p + at * a.V.row + (int64_t)hk * a.V.head, a.dK.p + at * a.dK.row + (int64_t)hk * a.dK.head,
                       a.dV.p + at * a.dV.row + (int64_t)hk * a.dV.head);
    }
    return;
  }
  if (GROUPS > 1) {
    add_groups<DH, OWNERS, GROUPS>(ok, smem, wave, group, lane);
    add_groups<DH, OWNERS, GROUPS>(ov, smem, wave, group, lane);
    if (group > 0) return;
  }
  if (!OWN) {
    if (j0 + i >= nk) return;
    char* dk = a.dK.p + (int64_t)(sk.first + mine) * a.dK.row + (int64_t)hk * a.dK.head + h * 32;
    char* dv = a.dV.p + (int64_t)(sk.first + mine) * a.dV.row + (int64_t)hk * a.dV.head + h * 32;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      float x[16], y[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) { x[r] = ok[d][r] * a.scale; y[r] = ov[d][r]; }
      *reinterpret_cast<bf16x8*>(dk + d * 64) = pack8(x);
      *reinterpret_cast<bf16x8*>(dk + d * 64 + 16) = pack8(x + 8);
      *reinterpret_cast<bf16x8*>(dv + d * 64) = pack8(y);
      *reinterpret_cast<bf16x8*>(dv + d * 64 + 16) = pack8(y + 8);
    }
    return;
  }
  if (j0 >= nk) return;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const f32x16* sum = n == 0 ? ok : ov;
    const AttnRows& to = n == 0 ? a.dK : a.dV;
    const float f = n == 0 ? a.scale : 1.f;
    wave_lds_fence();
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      float x[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = sum[d][r] * f;
      put_dims<DH>(own_tile, i, 4 * d + 2 * h, pack8(x), pack8(x + 8));
    }
    wave_lds_fence();
    store_rows<DH>(own_tile, to.p + (sk.first + j0) * to.row + (int64_t)hk * to.head, to.row, nk - j0, lane);
  }
}

// Key side, 128-wide heads: whether eight wavefronts own 256 keys, so that twice as many read a tile in LDS as of two groups of four, where
// there are sequences that long and rounds enough of workgroups, which `causal` makes unequal.  us, two groups and eight owners: 32 heads,
// 4 sequences of 2048 347 and 325, all keys seen 590 and 530; 20 of 512 (1280 workgroups) 192 and 180, 262 and 229; 32 heads on 8, one of
// 8192 (256 workgroups), all seen 1984 and 1874, but causal 1059 and 1659; 24 of 33 to 2000 (750) 465 and 475; 40 of 100 to 300, all seen 94 and 118.
// (64-wide heads: two wavefronts of a workgroup on every SIMD, where there is room for three.)
bool eight_owners(const spt_attn_shape_t& s) {
  return (int64_t)(s.Tk >> 8) * s.Hk >= (s.causal ? 1024 : 256) && s.Tk >= 256 * (int64_t)s.B;
}

template <int DH, int OWNERS, int GROUPS, bool EXACT>
hipError_t launch_q(BwdArgs a, const spt_attn_shape_t& s, hipStream_t st) {
  typedef BwdSizes<DH, OWNERS, GROUPS> Sizes;
  const auto kernel = prompt_bwd_q_kernel<DH, OWNERS, GROUPS, EXACT>;
  static std::atomic<uint64_t> done{0};
  if (const hipError_t e = allow_smem(reinterpret_cast<const void*>(kernel), Sizes::Q_SMEM, done); e != hipSuccess) return e;
  a.hshift = std::min(a.hshift, Sizes::SHIFT - 5);
  const int heads = a.G >> a.hshift, tiles = s.Tq >> (Sizes::SHIFT - a.hshift);
  a.coarse = coarse_tiles((int64_t)tiles * heads * s.Hk, DH == 128 ? 2 : 3);
  hipLaunchKernelGGL(kernel, dim3(head_item_grid(s.Hk, (tiles + s.B) * heads)), dim3(64 * OWNERS * GROUPS), Sizes::Q_SMEM, st, a);
  return hipGetLastError();
}

template <int DH, int OWNERS, int GROUPS, bool EXACT>
hipError_t launch_kv(BwdArgs a, const spt_attn_shape_t& s, hipStream_t st) {
  typedef BwdSizes<DH, OWNERS, GROUPS> Sizes;
  const auto kernel = prompt_bwd_kv_kernel<DH, OWNERS, GROUPS, EXACT>;
  static std::atomic<uint64_t> done{0};
  if (const hipError_t e = allow_smem(reinterpret_cast<const void*>(kernel), Sizes::KV_SMEM, done); e != hipSuccess) return e;
  const int tiles = s.Tk >> Sizes::SHIFT;
  // (heads that share their keys make fewer and longer tiles, of which the order by work alone is better: us, 48 sequences of 512, 32 heads of
  // 128 on 8 318 and 410 so, on 16 385 and 381, on 32 496 and 445)
  a.coarse = a.G > 1 ? 0 : coarse_tiles((int64_t)tiles * s.Hk, DH == 128 ? 1 : 3);
  hipLaunchKernelGGL(kernel, dim3(head_item_grid(s.Hk, tiles + s.B)), dim3(64 * OWNERS * GROUPS), Sizes::KV_SMEM, st, a);
  return hipGetLastError();
}

}  // namespace

extern "C" size_t spt_attn_prompt_workspace_bytes(const spt_attn_shape_t* shape) {
  if (check_attn(shape) != SPT_OK) return 0;
  return 2 * align256((size_t)shape->H * shape->Tq * sizeof(float));
}

extern "C" int spt_attn_prompt_bwd(const spt_attn_shape_t* shape, const void* Q, const void* K, const void* V, const void* Y,
                                   const void* dY, const float* lse, const int64_t* strides, const int32_t* cu_q, const int32_t* cu_k,
                                   void* dQ, void* dK, void* dV, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_attn(shape);
  if (rc != SPT_OK) return rc;
  const spt_attn_shape_t& s = *shape;
  BwdArgs a;
  const struct { AttnRows* r; const void* p; bool query, out; } rows[8] = {
      {&a.Q, Q, true, false}, {&a.K, K, false, false}, {&a.V, V, false, false}, {&a.Y, Y, true, false}, {&a.dY, dY, true, false},
      {&a.dQ, dQ, true, true}, {&a.dK, dK, false, true}, {&a.dV, dV, false, true}};
  for (int n = 0; n < 8; ++n) {
    rc = attn_rows(rows[n].r, rows[n].p, strides ? strides + 2 * n : nullptr, rows[n].query ? s.Tq : s.Tk, rows[n].query ? s.H : s.Hk, s.dh,
                   rows[n].out);
    if (rc != SPT_OK) return rc;
  }
  if (!aligned_to(cu_q, 4) || !aligned_to(cu_k, 4) || !aligned_to(lse, 4) || !aligned_to(ws, 256)) return SPT_ERR_ARG;
  if (ws_bytes < spt_attn_prompt_workspace_bytes(shape)) return SPT_ERR_WORKSPACE;
  a.cu_q = cu_q; a.cu_k = cu_k; a.lse = lse; a.off = static_cast<float*>(ws);
  a.neg_d = a.off + align256((size_t)s.H * s.Tq * sizeof(float)) / sizeof(float);
  a.B = s.B; a.Tq = s.Tq; a.Tk = s.Tk; a.Hk = s.Hk; a.G = s.H / s.Hk;
  a.hshift = attn_heads_shift(a.G);
  a.causal = s.causal;
  a.scale = s.scale;
  a.c = s.scale * kLog2e;
  const bool few = (int64_t)s.Tq * a.G <= (int64_t)kFewRows * s.B || (int64_t)(s.Tq >> 5) * s.H <= kFewTiles;
  const int q_owners = row_owners(s.Tq, s.H, a.hshift, s.Tk, s), kv_owners = row_owners(s.Tk, s.Hk, 0, (int64_t)s.Tq * a.G, s);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const auto launches = [&](auto dh, auto exact) {
    constexpr int DH = decltype(dh)::value, ONES = DH == 128 ? 4 : 8;
    constexpr bool EXACT = decltype(exact)::value;
    {
      ScopedKernelTimer timer(kSlotAttnBwdQ, st);
      const hipError_t e = q_owners == 4   ? launch_q<DH, 4, 1, EXACT>(a, s, st)
                           : q_owners == 2 ? launch_q<DH, 2, 4, EXACT>(a, s, st)
                                           : launch_q<DH, 1, ONES, true>(a, s, st);   // (so few are exact)
      if (e != hipSuccess) return e;
    }
    ScopedKernelTimer timer(kSlotAttnBwdKV, st);
    if constexpr (DH == 128) {
      if (eight_owners(s)) return launch_kv<DH, 8, 1, EXACT>(a, s, st);
    }
    return kv_owners == 4   ? launch_kv<DH, 4, DH == 128 ? 2 : 1, EXACT>(a, s, st)
           : kv_owners == 2 ? launch_kv<DH, 2, 4, EXACT>(a, s, st)
                            : launch_kv<DH, 1, ONES, EXACT>(a, s, st);
  };
  const auto of = [&](auto dh) { return few ? launches(dh, std::true_type()) : launches(dh, std::false_type()); };
  const hipError_t e = s.dh == 128 ? of(std::integral_constant<int, 128>()) : of(std::integral_constant<int, 64>());
  return e == hipSuccess ? SPT_OK : SPT_ERR_HIP;
}
