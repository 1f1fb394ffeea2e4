// Full attention over packed sequences, forward (include/spt_attn.h).
//
// A workgroup of four wavefronts owns 128 query rows: 128 / HW positions of one sequence times HW heads that
// share a key head (HW: 4, 2 or 1, as divides the group).  A wavefront owns 32 of them.  Where there is less to do than the chip has
// room for, two such groups share the keys, or four or eight groups of two or one those of 64 or 32 rows.  Keys and values pass through LDS in
// tiles of 64 (32 so), copied asynchronously one tile ahead.  Scores are formed transposed, S^T = K Q^T, so that a lane holds 16
// scores of ONE query and half of them are what the second product's operand wants of it: P stays in registers, and
// maximum, sum and rescaling of a query are one lane's (two halves of a row meet in one lane swap).  O^T = V^T P^T takes V out of LDS
// through the transposing read.  One pass over the keys: running maximum m and sum l, p = 2^(c s - m) with c = scale log2 e; the
// accumulators are rescaled only when a maximum rises by more than 2^8 (p stays below 256, and the sums are fp32).
// P goes into its product as one bf16, the sum that divides is that of the exact p: Y is 1.9e-3 off (2-norm; 150 tokens, 8 heads of 64; the
// rounding of Y alone makes 1.6e-3).  As the sum of two it was 1.6e-3, for a product more: 8192 tokens, 32 heads of 128 on 8, 528 us so, 710 with two.
#include <algorithm>
#include <type_traits>

#include "attn_common.hpp"

using namespace spt;

namespace {

constexpr float kLazy = 8.f;   // a row's maximum may be this much (log2) above what its sums are scaled by
// From this maximum (log2) on rows are taken the plain way.  c s - m is formed without a rounding between, m was rounded: by up to 8 here, so
// that weights stay below 2^16; a maximum of 2^32 would be off by 256, and all weights of the row 0 or infinite.
constexpr float kFar = 0x1p28f;

struct FwdArgs {
  AttnRows Q, K, V, Y;
  const int32_t *cu_q, *cu_k;
  float* lse;
  int B, Tq, Tk, Hk, G, hshift;   // G = H / Hk, 1 << hshift heads of a group in a workgroup
  int causal, coarse;
  float c;
};

// A row the plain way, for wavefronts that met infinities or NaN in rows that some of their queries must not see, or scores too far from 0: lanes
// take keys for the scores, dims for the sum, and only the `n` visible keys are touched.
template <int DH>
__device__ __forceinline__ void slow_row(const char* q, const char* k, int64_t kstep, const char* v, int64_t vstep, int n, float c, char* y,
                                         float* lse) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY, l = 0.f, acc[DH / 64] = {};
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane;
    const float t = j < n ? row_dot(q, k + j * kstep, DH) * c : -INFINITY;
    const float mn = fmaxf(m, wave_max(t)), ms = mn == -INFINITY ? 0.f : mn;
    const float p = j < n ? __builtin_amdgcn_exp2f(t - ms) : 0.f, alpha = __builtin_amdgcn_exp2f(m - ms);
    m = mn;
    l = l * alpha + wave_sum(p);
#pragma unroll
    for (int d = 0; d < DH / 64; ++d) acc[d] *= alpha;
    for (int e = 0; e < min(64, n - j0); ++e) {
      const float w = __shfl(p, e);
#pragma unroll
      for (int d = 0; d < DH / 64; ++d) acc[d] = fmaf(w, bf16_at(v + (j0 + e) * vstep + (lane + 64 * d) * 2), acc[d]);
    }
  }
#pragma unroll
  for (int d = 0; d < DH / 64; ++d)
    reinterpret_cast<uint16_t*>(y)[lane + 64 * d] = (uint16_t)pack_bf16x2(l == 0.f ? 0.f : acc[d] / l, 0.f);
  if (lse && lane == 0) *lse = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// A workgroup: GROUPS groups of OWNERS wavefronts (four, two or one), which go through every GROUPS-th tile of 32 KT keys for the same queries.
template <int DH, int OWNERS, int GROUPS>
struct FwdSizes {
  static constexpr int KT = OWNERS == 4 ? 2 : 1, TILE_KEYS = 32 * KT, TILE_BYTES = TILE_KEYS * DH * 2, RING = 4 * TILE_BYTES;   // K, V, twice
  static constexpr int SHIFT = OWNERS == 4 ? 7 : OWNERS == 2 ? 6 : 5, PART = DH * 128 + 512;   // 1 << SHIFT: rows; a wavefront's sums
  static constexpr int RINGS = GROUPS * RING, PARTS = (GROUPS - 1) * OWNERS * PART, SMEM = RINGS > PARTS ? RINGS : PARTS;
  static_assert(SMEM <= 160 * 1024, "a CU's LDS");
};

template <int DH, int OWNERS, int GROUPS>
__global__ __launch_bounds__((64 * OWNERS * GROUPS), 2) void prompt_fwd_kernel(const FwdArgs a) {
  typedef FwdSizes<DH, OWNERS, GROUPS> Sizes;
  constexpr int KS = DH / 16, DT = DH / 32, KT = Sizes::KT, TILE_KEYS = Sizes::TILE_KEYS, TILE_BYTES = Sizes::TILE_BYTES;
  extern __shared__ __align__(256) char smem[];
  const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5, tid = threadIdx.x % (64 * OWNERS);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % OWNERS, group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / OWNERS;
  char* ring = smem + group * Sizes::RING;

  const int hsets = a.G >> a.hshift, pshift = Sizes::SHIFT - a.hshift;    // 1 << pshift positions of a workgroup
  const HeadItem w = head_item(blockIdx.x, a.Hk);
  const int hk = w.hk, hs = w.item % hsets;
  TilePlace at;
  if (!find_tile<false>(a.cu_q, a.cu_k, a.B, a.Tq, a.Tk, pshift, a.causal, a.coarse, w.item / hsets, at)) return;
  const int tile = at.tile;
  const SeqRows sq = at.own, sk = at.other;
  const int nq = sq.n, nk = sk.n, ahead = nk - nq;       // query i sees keys up to i + ahead
  const int head = hk * a.G + (hs << a.hshift) + (wave & ((1 << a.hshift) - 1));
  const int p0 = (tile << pshift), i0 = p0 + (wave >> a.hshift) * 32;
  const int last = min(nq, p0 + (1 << pshift)) - 1;
  const int kend = a.causal ? min(nk, last + ahead + 1) : nk;            // keys that the workgroup sees any of
  const int wave_kend = i0 >= nq ? 0 : a.causal ? min(nk, min(nq, i0 + 32) + ahead) : nk;
  const int wave_full = i0 >= nq ? 0 : a.causal ? min(nk, i0 + ahead + 1) : nk;   // ... that all queries of the wavefront see
  const int mine = min(i0 + i, nq - 1);
  const int seen = a.causal ? min(nk, mine + ahead + 1) : nk;            // keys the lane's query sees (may be negative)
  const int ntile = kend > 0 ? (kend + TILE_KEYS - 1) / TILE_KEYS : 0;
  const int full = max(0, a.causal ? min(nk, p0 + ahead + 1) : nk);     // keys that all queries of the workgroup see

  // the wavefront's queries, through the second ring buffer: whole lines
  const char* qbase = a.Q.p + (int64_t)sq.first * a.Q.row + (int64_t)head * a.Q.head;
  const uint32_t tiles = lds_addr(ring), mine_lds = 2 * TILE_BYTES + wave * (32 * DH * 2);
  fetch_rows<DH>(qbase + min(i0, nq - 1) * a.Q.row, a.Q.row, max(nq - i0, 1), tiles + mine_lds, lane);
  const char* kbase = a.K.p + (int64_t)sk.first * a.K.row + (int64_t)hk * a.K.head;
  const char* vbase = a.V.p + (int64_t)sk.first * a.V.row + (int64_t)hk * a.V.head;
  // copies: lane L of an instruction fills 16 bytes of row (u 64 OWNERS + tid) / (DH / 8)
  constexpr int COPIES = TILE_KEYS * (DH / 8) / (64 * OWNERS);
  auto fetch = [&](int t, int buf) {
    const int j0 = t * TILE_KEYS;
    const char* kb = kbase + (int64_t)j0 * a.K.row;
    const char* vb = vbase + (int64_t)j0 * a.V.row;
#pragma unroll
    for (int u = 0; u < COPIES; ++u) {
      const int slot = u * 64 * OWNERS + tid, row = slot / (DH / 8);
      const uint32_t chunk = ((slot % (DH / 8)) ^ row_swizzle<DH>(row)) * 16;
      const uint32_t r = (uint32_t)min(row, nk - 1 - j0);               // (rows past the end: the last one again)
      const uint32_t at = lds_addr(ring + buf * 2 * TILE_BYTES + (u * OWNERS + wave) * 1024);
      dma16_at(kb, r * (uint32_t)a.K.row + chunk, at);
      dma16_at(vb, r * (uint32_t)a.V.row + chunk, at + TILE_BYTES);
    }
  };
  TileReader<DH> lds(lane);
  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float m = -INFINITY, neg_m = 0.f, l = 0.f;
  NotFinite plain;

  if (group < ntile) fetch(group, 0);
  bf16x8 qf[KS];
  if (group < ntile) wait_vmcnt<2 * COPIES>();
  else wait_vmcnt<0>();
#pragma unroll
  for (int s = 0; s < KS; ++s) qf[s] = lds.rows(tiles + mine_lds, 0, s);
  for (int t0 = 0; t0 < ntile; t0 += GROUPS) {
    wait_vmcnt<0>();
    __syncthreads();
    const int t = t0 + group, buf = t0 / GROUPS & 1, j0 = t * TILE_KEYS;
    if (t + GROUPS < ntile) fetch(t + GROUPS, buf ^ 1);
    if (t >= ntile) continue;
    const uint32_t kt_ = tiles + buf * 2 * TILE_BYTES, vt_ = kt_ + TILE_BYTES;
    if (j0 + TILE_KEYS > full) {
#pragma unroll
      for (int u = 0; u < TILE_BYTES / (1024 * OWNERS); ++u) plain.look(lds_read<u32x4>(vt_ + u * 1024 * OWNERS + tid * 16));
    }
    if (j0 >= wave_kend) continue;
    lds.fresh();
    __builtin_amdgcn_iglp_opt(1);                        // the compiler deals reads of LDS out between products: 8192 tokens, 32 heads of 128 on 8, 535 us without, 521
    f32x16 s[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kt][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds.rows(kt_, kt, ks), qf[ks], s[kt], 0, 0, 0);
    }
    if (j0 + TILE_KEYS > wave_full) {
      const int left = seen - j0 - 4 * h;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kt][r] = 32 * kt + 8 * (r >> 2) + (r & 3) < left ? s[kt][r] : -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int r = 1; r < 16 * KT; ++r) top = fmaxf(top, s[r >> 4][r & 15]);
    top = fmaxf(top, other_half(top)) * a.c;
    if (__any(top > m + kLazy)) {
      const float mn = fmaxf(m, top), ms = mn == -INFINITY ? 0.f : mn;
      const float alpha = __builtin_amdgcn_exp2f(m - ms);
      m = mn;
      neg_m = -ms;
      l *= alpha;
      plain.mark(fabsf(ms) >= kFar);
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
    }
    bf16x8 pf[KT][2];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(s[kt][8 * half + e], a.c, neg_m));
          l += p[e];
        }
        pf[kt][half] = pack8(p);
      }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int d = 0; d < DT; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds.columns(vt_, 2 * kt + half, d), pf[kt][half], o[d], 0, 0, 0);
  }

  float* lse = a.lse ? a.lse + (int64_t)head * a.Tq + sq.first : nullptr;
  // rows of V that not all queries may see hold infinities or NaN: 0 times those is NaN; or a maximum is too far from 0
  if (__syncthreads_or(plain.found())) {
    for (int r = group; r < min(32, nq - i0); r += GROUPS) {
      const int row = i0 + r;
      slow_row<DH>(a.Q.p + (int64_t)(sq.first + row) * a.Q.row + (int64_t)head * a.Q.head, kbase, a.K.row, vbase, a.V.row,
                   a.causal ? min(nk, row + ahead + 1) : nk, a.c, a.Y.p + (int64_t)(sq.first + row) * a.Y.row + (int64_t)head * a.Y.head,
                   lse ? lse + row : nullptr);
    }
    return;
  }
  l += other_half(l);
  if (GROUPS > 1) {                                      // the other groups' parts in order, scaled to the larger maximum
    auto part = [&](int g) { return reinterpret_cast<float*>(smem + ((g - 1) * OWNERS + wave) * Sizes::PART); };
    __syncthreads();
    if (group > 0) {
      float *x = part(group) + lane * 4, *ml = part(group) + DT * 1024 + lane;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) *reinterpret_cast<f32x4*>(x + (d * 4 + q) * 256) = f32x4{o[d][4 * q], o[d][4 * q + 1], o[d][4 * q + 2], o[d][4 * q + 3]};
      ml[0] = m;
      ml[64] = l;
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll 1
    for (int g = 1; g < GROUPS; ++g) {
      const float *from = part(g) + lane * 4, *ml = part(g) + DT * 1024 + lane;
      const float m1 = ml[0], mn = fmaxf(m, m1), ms = mn == -INFINITY ? 0.f : mn;
      const float f0 = __builtin_amdgcn_exp2f(m - ms), f1 = __builtin_amdgcn_exp2f(m1 - ms);
      l = fmaf(l, f0, ml[64] * f1);
      m = mn;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(from + (d * 4 + q) * 256);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[d][4 * q + e] = fmaf(o[d][4 * q + e], f0, x[e] * f1);
        }
    }
    wave_lds_fence();
  }
  if (i0 >= nq) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (lse && h == 0 && i0 + i < nq) lse[mine] = (m + __builtin_amdgcn_logf(l)) * kLn2;
  // rows out as whole lines, through the ring buffer that the last tile is not in (several groups: where the first other's sums were)
  const uint32_t out = GROUPS > 1 ? wave * Sizes::PART : (ntile & 1) * 2 * TILE_BYTES + wave * (32 * DH * 2);
#pragma unroll
  for (int d = 0; d < DT; ++d) {
    float v[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = o[d][r] * inv;
    put_dims<DH>(smem + out, i, 4 * d + 2 * h, pack8(v), pack8(v + 8));
  }
  wave_lds_fence();
  store_rows<DH>(smem + out, a.Y.p + (int64_t)(sq.first + i0) * a.Y.row + (int64_t)head * a.Y.head, a.Y.row, nq - i0, lane,
                 !a.lse);   // (a backward that follows reads Y: 16 sequences of 512, 32 heads of 64 178 us kept, 180 streamed; without one, 16
                            // prompts of 33 to 2000, 32 heads of 128 on 8, 109.7 and 107.2)
}

// Two groups of four wavefronts a workgroup where the chip would not be full: with no more workgroups than are resident at once (two on a CU
// at dh 128; at dh 64 four, of which three count) the one with the most keys is what the launch waits for.  us, one group and two, 32 heads on
// 8 of 128: one sequence of 2048 56.6 and 49.2, four parts of 512 behind 700 to 5000 146 and 129; of 4096 (twice as many workgroups as are
// resident) 154 and 158; four of 512, which have few tiles to share, 23.0 and 26.2; 12 heads of 64, one of 8000 146 and 133; 32 heads of 64,
// four of 1024 (four workgroups on a CU) 33 and 37.
bool two_groups(const spt_attn_shape_t& s, int hshift) {
  const int64_t workgroups = row_workgroups(s.Tq, 7 - hshift, s.B, s.H >> hshift), resident = 256 * (s.dh == 128 ? 2 : 3);
  return workgroups <= resident / 2 || (workgroups <= resident && s.Tk >= 1024 * (int64_t)s.B);
}

template <int DH, int OWNERS, int GROUPS>
hipError_t launch_fwd(FwdArgs a, const spt_attn_shape_t& s, hipStream_t st) {
  typedef FwdSizes<DH, OWNERS, GROUPS> Sizes;
  const auto kernel = prompt_fwd_kernel<DH, OWNERS, GROUPS>;
  static std::atomic<uint64_t> done{0};
  if (const hipError_t e = allow_smem(reinterpret_cast<const void*>(kernel), Sizes::SMEM, done); e != hipSuccess) return e;
  a.hshift = std::min(a.hshift, Sizes::SHIFT - 5);
  const int heads = a.G >> a.hshift, tiles = s.Tq >> (Sizes::SHIFT - a.hshift);
  a.coarse = coarse_tiles((int64_t)tiles * heads * s.Hk, DH == 128 ? 2 : 4);
  hipLaunchKernelGGL(kernel, dim3(head_item_grid(s.Hk, (tiles + s.B) * heads)), dim3(64 * OWNERS * GROUPS), Sizes::SMEM, st, a);   // (so many tiles at most)
  return hipGetLastError();
}

}  // namespace

namespace spt {

int check_attn(const spt_attn_shape_t* s) {
  if (!s) return SPT_ERR_ARG;
  if (s->B < 1 || s->Tq < 1 || s->Tk < 1 || s->H < 1 || s->Hk < 1 || s->dh < 1 || s->H % s->Hk != 0) return SPT_ERR_ARG;
  if (s->causal != 0 && s->causal != 1) return SPT_ERR_ARG;
  if (!(s->scale > 0.f) || !(s->scale <= kMostScale)) return SPT_ERR_ARG;
  if ((s->dh != 64 && s->dh != 128) || s->B > 4096 || s->H > 65535) return SPT_ERR_UNSUPPORTED;
  const int shift = attn_heads_shift(s->H / s->Hk);   // (tiles of 128 rows of heads; of 128 keys)
  if (((int64_t)(s->Tq >> (7 - shift)) + s->B) * (s->H >> shift) > kMostWorkgroups) return SPT_ERR_UNSUPPORTED;
  if (((int64_t)(s->Tk >> 7) + s->B) * s->Hk > kMostWorkgroups) return SPT_ERR_UNSUPPORTED;
  return SPT_OK;
}

int attn_heads_shift(int G) { return G % 4 == 0 ? 2 : G % 2 == 0 ? 1 : 0; }

}  // namespace spt

extern "C" int spt_attn_prompt_fwd(const spt_attn_shape_t* shape, const void* Q, const void* K, const void* V,
                                   const int64_t* strides, const int32_t* cu_q, const int32_t* cu_k, void* Y, float* lse,
                                   void* stream) {
  int rc = check_attn(shape);
  if (rc != SPT_OK) return rc;
  const spt_attn_shape_t& s = *shape;
  FwdArgs a;
  auto at = [&](int n) { return strides ? strides + 2 * n : nullptr; };
  if ((rc = attn_rows(&a.Q, Q, at(0), s.Tq, s.H, s.dh, false)) != SPT_OK) return rc;
  if ((rc = attn_rows(&a.K, K, at(1), s.Tk, s.Hk, s.dh, false)) != SPT_OK) return rc;
  if ((rc = attn_rows(&a.V, V, at(2), s.Tk, s.Hk, s.dh, false)) != SPT_OK) return rc;
  if ((rc = attn_rows(&a.Y, Y, at(3), s.Tq, s.H, s.dh, true)) != SPT_OK) return rc;
  if (!aligned_to(cu_q, 4) || !aligned_to(cu_k, 4) || (lse && !aligned_to(lse, 4))) return SPT_ERR_ARG;
  a.cu_q = cu_q; a.cu_k = cu_k; a.lse = lse;
  a.B = s.B; a.Tq = s.Tq; a.Tk = s.Tk; a.Hk = s.Hk; a.G = s.H / s.Hk;
  a.hshift = attn_heads_shift(a.G);
  a.causal = s.causal;
  a.c = s.scale * kLog2e;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  ScopedKernelTimer timer(kSlotAttnFwd, st);
  const auto launch = [&](auto dh) {
    constexpr int DH = decltype(dh)::value;
    const int owners = row_owners(s.Tq, s.H, a.hshift, s.Tk, s);
    if (owners < 4) return owners == 2 ? launch_fwd<DH, 2, 4>(a, s, st) : launch_fwd<DH, 1, DH == 128 ? 4 : 8>(a, s, st);
    return two_groups(s, a.hshift) ? launch_fwd<DH, 4, 2>(a, s, st) : launch_fwd<DH, 4, 1>(a, s, st);
  };
  const hipError_t e = s.dh == 128 ? launch(std::integral_constant<int, 128>()) : launch(std::integral_constant<int, 64>());
  return e == hipSuccess ? SPT_OK : SPT_ERR_HIP;
}
