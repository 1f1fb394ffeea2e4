// The paged cache of keys and values, and the attention of single tokens over it (include/spt_attn.h).
#include "attn_common.hpp"

using namespace spt;

namespace {

struct CacheArgs {
  char *Kc, *Vc;
  uint8_t *ks, *vs;
  const int32_t* table;
  int pages, page_shift, Hk, B, max_pages;
};

// ------------------------------------------------------------------------------------------
// Writing and reading rows.  A wavefront takes one row of the packed tensors, all key heads of K and V; DH / 8 lanes a
// head, 16 bytes of the packed row each.  Bytes in and out once; nothing to compute but a row's largest magnitude.

struct RowArgs {
  CacheArgs c;
  AttnRows K, V;
  const int32_t *start, *cu;
  int T;
};

// Sequence of packed row r: the number of sequences that end at or before it.  64 at a time.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int B, int r) {
  const int lane = threadIdx.x & 63;
  int b = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const bool ends = b0 + lane < B && cu[b0 + lane + 1] <= r;
    b += __builtin_popcountll(__ballot(ends));
  }
  return b;
}

// Where token `pos` of sequence b lies, as (page Hk page-size + place in it) of head 0; negative: nowhere.
__device__ __forceinline__ int64_t token_place(const CacheArgs& c, int b, int64_t pos) {
  if (pos < 0 || pos >= ((int64_t)c.max_pages << c.page_shift)) return -1;
  const int p = c.table[(int64_t)b * c.max_pages + (int)(pos >> c.page_shift)];
  if (p < 0 || p >= c.pages) return -1;
  return (((int64_t)p * c.Hk) << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
}

// largest of LANES neighbouring lanes' values
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) x = max(x, (uint32_t)__shfl_xor((int)x, o));
  return x;
}

// Exponent byte of a row whose largest finite magnitude is the bf16 (or fp32) with these bits: the least e >= -127 with
// that magnitude <= 448 2^e, plus 127.  448 = 1.75 2^8: the fraction decides between two exponents.
__device__ __forceinline__ int row_exponent(uint32_t bits) {
  if (bits < 0x00800000u) return 0;                        // below 2^-126: e = -127
  return max(0, (int)(bits >> 23) - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0));
}

// 4 values -> 4 codes.  x 2^-e is exact and at most 448, so only the conversion rounds (nearest even).
__device__ __forceinline__ uint32_t code4(const float* x) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
  return (uint32_t)w;
}

template <int DH, bool E4M3>
__global__ __launch_bounds__(256) void cache_write_kernel(const RowArgs a) {
  constexpr int LANES = DH / 8, HEADS = 64 / LANES;
  const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= a.T) return;
  const int b = sequence_of(a.cu, a.c.B, r);
  if (b >= a.c.B || r < a.cu[b]) return;
  const int64_t place = token_place(a.c, b, (int64_t)a.start[b] + r - max(a.cu[b], 0));
  if (place < 0) return;
  const int piece = lane % LANES;
  for (int n = lane / LANES; n < 2 * a.c.Hk; n += HEADS) {
    const bool v = n >= a.c.Hk;
    const int hk = v ? n - a.c.Hk : n;
    const AttnRows& src = v ? a.V : a.K;
    const u32x4 x = stream_in<u32x4>(src.p + r * src.row + hk * src.head + piece * 16);
    const int64_t at = place + ((int64_t)hk << a.c.page_shift);
    char* dst = v ? a.c.Vc : a.c.Kc;
    if (!E4M3) {
      stream_out(dst + at * (DH * 2) + piece * 16, x);
      continue;
    }
    uint32_t top = 0;
    float f[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = lo_bf16(x[e]);
      f[2 * e + 1] = hi_bf16(x[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t mag = __float_as_uint(f[e]) & 0x7FFFFFFFu;
      if (mag < 0x7F800000u) top = max(top, mag);
    }
    const int byte = row_exponent(lanes_max<LANES>(top));
    const float most = byte == 247 ? 240.f : 448.f;         // (256 2^120 is no bf16)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      f[e] = (__float_as_uint(f[e]) & 0x7F800000u) == 0x7F800000u ? __builtin_nanf("")
                                                                  : __builtin_amdgcn_fmed3f(__builtin_ldexpf(f[e], 127 - byte), -most, most);
    stream_out(dst + at * DH + piece * 8, u32x2{code4(f), code4(f + 4)});
    if (piece == 0) (v ? a.c.vs : a.c.ks)[at] = (uint8_t)byte;
  }
}

typedef __bf16 pair_bf16 __attribute__((ext_vector_type(2)));
// 4 codes -> 4 bf16 of the values code * scale
__device__ __forceinline__ uint2 uncode4(uint32_t w, float scale) {
  const pair_bf16 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
  return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}
// 4 codes and the exponent byte of their row -> 4 bf16 (exact)
__device__ __forceinline__ uint2 held4(uint32_t w, int byte) {
  const uint2 x = uncode4(w, 1.f);
  auto at = [&](float v) { return __builtin_ldexpf(v, byte - 127); };
  return make_uint2(pack_bf16x2(at(lo_bf16(x.x)), at(hi_bf16(x.x))), pack_bf16x2(at(lo_bf16(x.y)), at(hi_bf16(x.y))));
}

template <int DH, bool E4M3>
__global__ __launch_bounds__(256) void cache_read_kernel(const RowArgs a) {
  constexpr int LANES = DH / 8, HEADS = 64 / LANES;
  const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= a.T) return;
  const int b = sequence_of(a.cu, a.c.B, r);
  if (b >= a.c.B || r < a.cu[b]) return;
  const int64_t place = token_place(a.c, b, (int64_t)a.start[b] + r - max(a.cu[b], 0));
  const int piece = lane % LANES;
  for (int n = lane / LANES; n < 2 * a.c.Hk; n += HEADS) {
    const bool v = n >= a.c.Hk;
    const int hk = v ? n - a.c.Hk : n;
    const AttnRows& to = v ? a.V : a.K;
    const char* src = v ? a.c.Vc : a.c.Kc;
    const int64_t at = place + ((int64_t)hk << a.c.page_shift);
    u32x4 x = {0, 0, 0, 0};
    if (place >= 0) {
      if (!E4M3) {
        x = stream_in<u32x4>(src + at * (DH * 2) + piece * 16);
      } else {
        const u32x2 w = stream_in<u32x2>(src + at * DH + piece * 8);
        const int byte = (v ? a.c.vs : a.c.ks)[at];
        const uint2 lo = held4(w[0], byte), hi = held4(w[1], byte);
        x = u32x4{lo.x, lo.y, hi.x, hi.y};
      }
    }
    stream_out(to.p + r * to.row + hk * to.head + piece * 16, x);
  }
}

// ------------------------------------------------------------------------------------------
// Decoding.  The cache is read once for every sixteen query heads of a key head; everything else is small.  An item is a key head of a sequence
// with up to 16 of the query heads that read it (the columns of a 16 x 16 x 32 product), a unit 32 tokens of an item.  (More heads read it
// again, as items of their own: 8 sequences of 8000, one key head of 128 in 16 bits, 16 heads 22.6 us, 32 25.5, 64 33.7, 128 52.3.)  The units of all items stand in one
// line, and every wavefront takes an equal stretch of it, whatever the lengths: an item that lies within one stretch is
// finished there, the others leave a partial result (maximum, sum, unnormalised output) per stretch, which a second launch
// joins in the order of the cache.  At most the first and the last item of a stretch are partial: two slots a stretch.
// Wavefronts do not wait for one another.  Each has a ring of two units in LDS of its own, filled by asynchronous copies that run
// ahead over the ends of items (with a wavefront per unit in turn, and a workgroup's four joined at every item's end, 48 sequences of 100 to 8000
// tokens, 8 key heads, went at 4.0 TB/s, eight of one length at 5.0).  Scores are formed transposed (rows: tokens), so that
// a lane holds the weights of one query as the second product wants them; a weight goes into it as the sum of two bf16 (the
// matrix cores have nothing else to do), so the weights are exact to 2^-17.  8-bit codes become bf16 in registers, exactly; the
// rows' exponents are applied to the scores and to the weights.

constexpr int kUnit = 32, kDecodeWaves = 4, kLeastUnits = 2;   // (a stretch has two units at least, so that there is something to run ahead to)

struct DecodeArgs {
  CacheArgs c;
  AttnRows Q, Y;
  const int32_t* lens;
  float *part, *stat;             // [slots][rows][DH], [slots][rows][2] (maximum, sum)
  int H, G, sets, rows;           // sets of at most 16 heads of a group; rows of a slot
  int workgroups;
  float cs;                       // scale log2 e
};

__device__ __forceinline__ int units_of(int len) { return len / kUnit + (len % kUnit != 0); }   // (len + 31 may pass 31 bits)
__device__ __forceinline__ int seq_len(const DecodeArgs& a, int len) { return min(max(len, 0), a.c.max_pages << a.c.page_shift); }
__device__ __forceinline__ int seq_units(const DecodeArgs& a, int b) { return units_of(seq_len(a, a.lens[b])); }

struct Line { int total, share; };
// Units of all sequences, and a wavefront's part of them.
__device__ __forceinline__ Line unit_line(const DecodeArgs& a) {
  int n = 0;
  for (int b = threadIdx.x & 63; b < a.c.B; b += 64) n += seq_units(a, b);
  n = wave_total(n) * a.c.Hk * a.sets;
  const int waves = a.workgroups * kDecodeWaves;
  return {n, max(kLeastUnits, (n - 1) / waves + 1)};
}
// First unit of sequence b's items
__device__ __forceinline__ int units_before(const DecodeArgs& a, int b) {
  int n = 0;
  for (int x = threadIdx.x & 63; x < b; x += 64) n += seq_units(a, x);
  return wave_total(n) * a.c.Hk * a.sets;
}

// QCOPIES: the copies of 1 KB that an item's queries take, one or as many as sixteen heads need: LDS that other wavefronts could use.
template <int DH, bool E4M3, int QC>
struct DecodeTile {
  static constexpr int RB = E4M3 ? DH : DH * 2;            // bytes of a row
  static constexpr int BYTES = kUnit * RB;                 // of a unit's K or V
  static constexpr int COPIES = BYTES / 1024;
  static constexpr int QCOPIES = QC, QUERIES = QC * 1024;  // of an item, with its first unit
  static constexpr int STAGE = 2 * BYTES + QUERIES + (E4M3 ? 256 : 0);
  static constexpr int LOADS = 2 * COPIES + (E4M3 ? 1 : 0);
  static constexpr int RING = 2 * STAGE, SMEM = kDecodeWaves * RING, PER_CU = 160 * 1024 / SMEM;
  static_assert(PER_CU >= 1, "a CU's LDS");
};
constexpr int kQueryRows[2] = {8, 4};                      // heads whose queries fit into one copy: dh 64, 128

// A unit: its sequence, its item and place in it, its pages.
struct Unit {
  int b, item, t, units, len;     // units, len: of the sequence
  int page[2];                    // of its two halves
};

// Up to sixteen query heads of an item (the lane's: lane % 16) over the units so far: maximum, sum (of the lane's tokens), output.
template <int DH, bool E4M3>
struct DecodeState {
  static constexpr int RB = E4M3 ? DH : DH * 2, COPIES = kUnit * RB / 1024, KS = DH / 32, DT = DH / 16;
  bf16x8 qf[KS];
  f32x4 o[DT];
  float m, neg_m, l;

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY; neg_m = 0.f; l = 0.f;
  }
  // A unit that lies in LDS: rows kt, vt, the rows' exponents, which of its tokens are there.
  __device__ __forceinline__ void unit(char* kt, char* vt, const char* exponents, uint32_t there, float cs, int lane) {
    const int q = lane & 15, c = lane >> 4;
    if (there != 0xFFFFFFFFu) {                            // 0 times what lies behind the last token may be NaN
      for (int n = 0; n < COPIES; ++n) {
        const int r = n * (1024 / RB) + lane / (RB / 16);
        if (!((there >> r) & 1)) *reinterpret_cast<u32x4*>(vt + n * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
      }
      wave_lds_fence();
    }
    f32x4 s[2];
#pragma unroll
    for (int kt2 = 0; kt2 < 2; ++kt2) {
      s[kt2] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int r = 16 * kt2 + q;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 f;
        if (E4M3) {
          const uint32_t piece = 4 * ks + c;
          const uint2 w = *reinterpret_cast<const uint2*>(kt + r * RB + ((piece >> 1) ^ chunk_swizzle<RB>(r)) * 16 + (piece & 1) * 8);
          const uint2 lo = uncode4(w.x, 1.f), hi = uncode4(w.y, 1.f);
          f = as_bf16x8(u32x4{lo.x, lo.y, hi.x, hi.y});
        } else {
          f = *reinterpret_cast<const bf16x8*>(kt + r * RB + ((uint32_t)(4 * ks + c) ^ chunk_swizzle<RB>(r)) * 16);
        }
        s[kt2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, qf[ks], s[kt2], 0, 0, 0);
      }
    }
    uint32_t kb[2] = {0, 0}, vb[2] = {0, 0};               // exponents of the lane's tokens 16 kt2 + 4 c + e
    if (E4M3) {
      const uint32_t* ex = reinterpret_cast<const uint32_t*>(exponents);
      kb[0] = ex[c]; kb[1] = ex[4 + c];
      vb[0] = ex[8 + c]; vb[1] = ex[12 + c];
    }
    float x[8], top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v = s[e >> 2][e & 3];
      if (E4M3) v = __builtin_ldexpf(v, (int)((kb[e >> 2] >> (8 * (e & 3))) & 255u) - 127);   // (first: codes times a large scale may pass what fp32 holds)
      v *= cs;
      x[e] = (there >> (16 * (e >> 2) + 4 * c + (e & 3))) & 1 ? v : -INFINITY;
      top = fmaxf(top, x[e]);
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    if (__any(top > m)) {
      const float mn = fmaxf(m, top), ms = mn == -INFINITY ? 0.f : mn, alpha = __builtin_amdgcn_exp2f(m - ms);
      m = mn;
      neg_m = -ms;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[d][e] *= alpha;
    }
    float w[8], rest[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = __builtin_amdgcn_exp2f(x[e] + neg_m);
      l += p;
      w[e] = p;
      if (E4M3) {
        w[e] = __builtin_ldexpf(p, (int)((vb[e >> 2] >> (8 * (e & 3))) & 255u) - 127);
        if (!((there >> (16 * (e >> 2) + 4 * c + (e & 3))) & 1)) w[e] = 0.f;
      }
    }
    const bf16x8 hi = pack8(w);
    const u32x4 hw = __builtin_bit_cast(u32x4, hi);
#pragma unroll
    for (int e = 0; e < 8; ++e) rest[e] = w[e] - (e & 1 ? hi_bf16(hw[e >> 1]) : lo_bf16(hw[e >> 1]));
    const bf16x8 lo = pack8(rest);
    const int sl = lane & 15;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      bf16x8 f;
      if (E4M3) {
        const int rr = sl >> 1, r = 4 * c + (rr & 3) + 16 * (rr >> 2);
        typedef int v2i __attribute__((ext_vector_type(2)));
        const v2i w8 = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            (__attribute__((address_space(3))) v2i*)(uintptr_t)(vt + r * RB + ((uint32_t)d ^ chunk_swizzle<RB>(r)) * 16 + (sl & 1) * 8));
        const uint2 f0 = uncode4((uint32_t)w8[0], 1.f), f1 = uncode4((uint32_t)w8[1], 1.f);
        f = as_bf16x8(u32x4{f0.x, f0.y, f1.x, f1.y});
      } else {
        const int r = 4 * c + (sl >> 2);
        const uint32_t chunk = 2 * d + ((sl & 3) >> 1);
        f = tr_read_frag(vt + r * RB + (chunk ^ chunk_swizzle<RB>(r)) * 16 + (sl & 1) * 8,
                         vt + (r + 16) * RB + (chunk ^ chunk_swizzle<RB>(r + 16)) * 16 + (sl & 1) * 8);
      }
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, hi, o[d], 0, 0, 0);
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, lo, o[d], 0, 0, 0);
    }
  }
  __device__ __forceinline__ float sum() const {             // of all tokens
    const float s = l + __shfl_xor(l, 16);
    return s + __shfl_xor(s, 32);
  }
};

// Asynchronous copies of unit t of a sequence into a stage; returns which of its 32 tokens are there.  Nobody reads a row again in the launch
// (but for groups of more than sixteen heads): kept in L2 48 sequences of 100 to 8000 tokens in 8 bits, 32 heads of 128 on 8, went in 45.8 us, 41.2 so,
// six of 30000 to 32700 in 16 bits in 137 (5.6 TB/s) and 121 (6.4).
template <int DH, bool E4M3>
__device__ __forceinline__ uint32_t fetch_unit(const DecodeArgs& a, int hk, int t, int len, const int* page, uint32_t at, uint32_t exponents, int lane) {
  constexpr int RB = E4M3 ? DH : DH * 2, BYTES = kUnit * RB;
  uint32_t there = 0;
  int64_t row[2];
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int pos = t * kUnit + 16 * half;
    const bool ok = pos < len && page[half] >= 0 && page[half] < a.c.pages;
    if (ok) there |= (len - pos >= 16 ? 0xFFFFu : (1u << (len - pos)) - 1u) << (16 * half);
    row[half] = ((((int64_t)(ok ? page[half] : 0) * a.c.Hk) + hk) << a.c.page_shift) + (pos & ((1 << a.c.page_shift) - 1));
  }
#pragma unroll
  for (int n = 0; n < BYTES / 1024; ++n) {
    const int r = n * (1024 / RB) + lane / (RB / 16);        // row of the unit; those of a copy lie in one half
    const int half = n * (1024 / RB) / 16;
    const uint32_t off = (uint32_t)(r - 16 * half) * RB + (((uint32_t)lane % (RB / 16)) ^ chunk_swizzle<RB>(r)) * 16;
    dma16_once(a.c.Kc + row[half] * RB, off, at + n * 1024);
    dma16_once(a.c.Vc + row[half] * RB, off, at + BYTES + n * 1024);
  }
  if (E4M3) {                                                // lanes 0-7: exponents of the keys, 8-15: of the values
    const int half = (lane >> 2) & 1;
    dma4(((lane & 8) ? a.c.vs : a.c.ks) + row[half] + 4 * (lane & 3), exponents);
  }
  return there;
}
__device__ __forceinline__ int unit_page(const DecodeArgs& a, int b, int t, int half, int len) {
  return uniform_load(a.c.table + (int64_t)b * a.c.max_pages + (min(t * kUnit + 16 * half, len - 1) >> a.c.page_shift));
}

template <int DH, bool E4M3, int QC>
__global__ __launch_bounds__(64 * kDecodeWaves, 2) void decode_kernel(const DecodeArgs a) {
  typedef DecodeTile<DH, E4M3, QC> T;
  constexpr int KS = DH / 32, DT = DH / 16;
  extern __shared__ __align__(256) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q = lane & 15, c = lane >> 4, items = a.c.Hk * a.sets, qrow = min(q, QC * (512 / DH) - 1);
  char* ring = smem + wave * T::RING;

  const Line line = unit_line(a);
  const int stretch = wave * a.workgroups + blockIdx.x;    // (few stretches: one on a CU)
  if (stretch > line.total / line.share) return;
  int left = min(line.total - stretch * line.share, line.share);
  if (left <= 0) return;

  auto pages_of = [&](Unit& x) {
#pragma unroll
    for (int half = 0; half < 2; ++half) x.page[half] = unit_page(a, x.b, x.t, half, x.len);
  };
  auto sequence = [&](Unit& x) {
    x.len = seq_len(a, uniform_load(a.lens + x.b));
    x.units = units_of(x.len);
  };
  Unit ahead;                                              // the next unit to be asked for
  {
    const int u = stretch * line.share;
    int before = 0, rem = 0;
    ahead.b = 0;
    for (int b0 = 0; b0 < a.c.B; b0 += 64) {
      const int incl = wave_prefix(b0 + lane < a.c.B ? seq_units(a, b0 + lane) : 0) * items, total = __builtin_amdgcn_readlane(incl, 63);
      if (u - before < total) {
        const int src = __builtin_ctzll(__ballot(incl > u - before));
        ahead.b = b0 + src;
        rem = u - before - (src > 0 ? __builtin_amdgcn_readlane(incl, src - 1) : 0);
        break;
      }
      before += total;
    }
    sequence(ahead);
    ahead.item = rem / ahead.units;
    ahead.t = rem - ahead.item * ahead.units;
    pages_of(ahead);
  }
  auto advance = [&](Unit& x) {                            // (there is one more unit)
    if (++x.t == x.units) {
      x.t = 0;
      if (++x.item == items) {
        x.item = 0;
        do {
          ++x.b;
          sequence(x);
        } while (x.units == 0);
      }
    }
    pages_of(x);
  };
  auto head0_of = [&](const Unit& x) { return x.item / a.sets * a.G + x.item % a.sets * 16; };
  auto heads_of = [&](const Unit& x) { return min(16, a.G - x.item % a.sets * 16); };

  // copies of a unit into a stage (with its item's queries where these are new); returns which of its 32 tokens are there
  auto fetch = [&](const Unit& x, bool queries, int stage) -> uint32_t {
    const uint32_t at = lds_addr(ring + stage * T::STAGE);
    const uint32_t there = fetch_unit<DH, E4M3>(a, x.item / a.sets, x.t, x.len, x.page, at, at + 2 * T::BYTES + T::QUERIES, lane);
    if (queries) {
      const char* base = a.Q.p + x.b * a.Q.row + (int64_t)head0_of(x) * a.Q.head;
      const int heads = heads_of(x);
#pragma unroll
      for (int n = 0; n < T::QCOPIES; ++n) {
        const int r = n * (512 / DH) + lane / (DH / 8);    // (rows past the heads: the last one again)
        dma16_at(base, (uint32_t)min(r, heads - 1) * (uint32_t)a.Q.head + (((uint32_t)lane % (DH / 8)) ^ row_swizzle<DH>(r)) * 16,
                 at + 2 * T::BYTES + n * 1024);
      }
    }
    return there;
  };

  DecodeState<DH, E4M3> state;
  Unit now = ahead, next = ahead;
  bool fresh = true, next_fresh = false, first_item = true;   // whether a unit's queries are new
  int item_units = 0;                                      // units of the present item so far
  uint32_t there = fetch(now, true, 0), next_there = 0;
  --left;
  if (left > 0) {
    advance(ahead);
    next = ahead;
    next_fresh = next.t == 0;
    next_there = fetch(next, next_fresh, 1);
    if (left > 1) advance(ahead);
  }
  for (int stage = 0;; stage ^= 1) {
    if (left <= 0) wait_vmcnt<0>();
    else if (next_fresh) wait_vmcnt<T::LOADS + T::QCOPIES>();
    else wait_vmcnt<T::LOADS>();
    wave_lds_fence();
    char* kt = ring + stage * T::STAGE;
    char* vt = kt + T::BYTES;
    if (fresh) {
#pragma unroll
      for (int s = 0; s < KS; ++s)
        state.qf[s] = *reinterpret_cast<const bf16x8*>(kt + 2 * T::BYTES + qrow * (DH * 2) + ((uint32_t)(4 * s + c) ^ row_swizzle<DH>(qrow)) * 16);
      state.clear();
      item_units = 0;
    }
    ++item_units;
    state.unit(kt, vt, kt + 2 * T::BYTES + T::QUERIES, there, a.cs, lane);
    // the stage has been read (lgkmcnt 0: no read of it is on its way): the unit after the next one's
    wave_lds_fence();
    __builtin_amdgcn_s_waitcnt(0xC07F);
    const Unit done = now;
    const bool ends = left <= 0 || next_fresh;
    now = next;
    there = next_there;
    fresh = next_fresh;
    const bool more = left-- > 0;
    if (left > 0) {
      next = ahead;
      next_fresh = next.t == 0;
      next_there = fetch(next, next_fresh, stage);
      if (left > 1) advance(ahead);
    }
    if (ends) {                                            // the item's result, or the stretch's part of it
      const float sum = state.sum();
      const f32x4* o = state.o;
      const int head0 = head0_of(done);
      if (q < heads_of(done)) {
        if (item_units == done.units) {
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          char* y = a.Y.p + done.b * a.Y.row + (int64_t)(head0 + q) * a.Y.head + c * 8;
#pragma unroll
          for (int d = 0; d < DT; ++d)
            *reinterpret_cast<uint2*>(y + d * 32) = make_uint2(pack_bf16x2(o[d][0] * inv, o[d][1] * inv), pack_bf16x2(o[d][2] * inv, o[d][3] * inv));
        } else {
          const int64_t row = (int64_t)(2 * stretch + (first_item ? 0 : 1)) * a.rows + q;
#pragma unroll
          for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(a.part + row * DH + 16 * d + 4 * c) = o[d];
          if (c == 0) {
            a.stat[row * 2] = state.m;
            a.stat[row * 2 + 1] = sum;
          }
        }
      }
      first_item = false;
    }
    if (!more) break;
  }
}

// Short tables: a workgroup per item, its wavefronts take turns at the units and are joined in LDS, in order: one launch.
template <int DH, bool E4M3>
struct ItemTile {
  static constexpr int BYTES = kUnit * (E4M3 ? DH : DH * 2), STAGE = 2 * BYTES + (E4M3 ? 256 : 0), LOADS = 2 * (BYTES / 1024) + (E4M3 ? 1 : 0);
  static constexpr int WAVES = STAGE >= 16384 ? 4 : 8, LD = DH + 4;
  static constexpr int JOIN = WAVES * 16 * (LD + 2) * 4, RINGS = WAVES * 2 * STAGE, SMEM = RINGS > JOIN ? RINGS : JOIN;
  static_assert(SMEM <= 160 * 1024, "a CU's LDS");
};

template <int DH, bool E4M3>
__global__ __launch_bounds__((64 * ItemTile<DH, E4M3>::WAVES), 2) void decode_item_kernel(const DecodeArgs a) {
  typedef ItemTile<DH, E4M3> T;
  constexpr int KS = DH / 32, DT = DH / 16, WAVES = T::WAVES;
  extern __shared__ __align__(256) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane & 15, c = lane >> 4;
  const int items = a.c.Hk * a.sets, b = blockIdx.x / items, item = blockIdx.x - b * items, hk = item / a.sets;
  const int head0 = hk * a.G + item % a.sets * 16, heads = min(16, a.G - item % a.sets * 16);
  const int len = seq_len(a, uniform_load(a.lens + b)), units = units_of(len);
  char* ring = smem + wave * 2 * T::STAGE;
  auto fetch = [&](int t, int stage) {
    const int page[2] = {unit_page(a, b, t, 0, len), unit_page(a, b, t, 1, len)};
    const uint32_t at = lds_addr(ring + stage * T::STAGE);
    return fetch_unit<DH, E4M3>(a, hk, t, len, page, at, at + 2 * T::BYTES, lane);
  };
  DecodeState<DH, E4M3> state;
  state.clear();
  uint32_t there = 0, next = 0;
  if (wave < units) there = fetch(wave, 0);
  const char* qrow = a.Q.p + b * a.Q.row + (int64_t)(head0 + min(q, heads - 1)) * a.Q.head;
#pragma unroll
  for (int s = 0; s < KS; ++s) state.qf[s] = *reinterpret_cast<const bf16x8*>(qrow + s * 64 + c * 16);
#pragma unroll
  for (int s = 0; s < KS; ++s) asm volatile("" ::"v"(state.qf[s]));   // (they are there: no wait for them in the loop)
  for (int t = wave, stage = 0; t < units; t += WAVES, stage ^= 1, there = next) {
    if (t + WAVES < units) {
      next = fetch(t + WAVES, stage ^ 1);
      wait_vmcnt<T::LOADS>();
    } else {
      wait_vmcnt<0>();
    }
    wave_lds_fence();
    char* kt = ring + stage * T::STAGE;
    state.unit(kt, kt + T::BYTES, kt + 2 * T::BYTES, there, a.cs, lane);
    wave_lds_fence();
    __builtin_amdgcn_s_waitcnt(0xC07F);                      // (lgkmcnt 0: the stage is filled again next)
  }
  const float sum = state.sum();
  __syncthreads();
  float* ml = reinterpret_cast<float*>(smem);                // [wave][16][2]
  float* os = ml + WAVES * 32;                               // [wave][16][LD]
  if (c == 0) {
    ml[(wave * 16 + q) * 2] = state.m;
    ml[(wave * 16 + q) * 2 + 1] = sum;
  }
#pragma unroll
  for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(os + (wave * 16 + q) * T::LD + 16 * d + 4 * c) = state.o[d];
  __syncthreads();
  for (int n = threadIdx.x; n < heads * (DH / 4); n += 64 * WAVES) {
    const int row = n / (DH / 4), d4 = n % (DH / 4);
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) M = fmaxf(M, ml[(w * 16 + row) * 2]);
    const float ms = M == -INFINITY ? 0.f : M;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[(w * 16 + row) * 2] - ms);
      const f32x4 x = *reinterpret_cast<const f32x4*>(os + (w * 16 + row) * T::LD + 4 * d4);
      L = fmaf(f, ml[(w * 16 + row) * 2 + 1], L);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = fmaf(f, x[e], y[e]);
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    *reinterpret_cast<uint2*>(a.Y.p + b * a.Y.row + (int64_t)(head0 + row) * a.Y.head + d4 * 8) =
        make_uint2(pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv));
  }
}

// A workgroup per query head: the partial results of its item in the order of the cache, or zeros without a key.  Eight (dh 128) or
// sixteen parts of the list side by side, joined in order.  Each finds its item's stretches from all lengths, work that grows with
// the square of the sequences: 8 heads of 128 on 2, 64 tokens each, 64 sequences 6.4 us, 1024 25, 4096 244, 16384 3636 (their units 8.3, 20, 74, 296).
template <int DH>
__global__ __launch_bounds__(256) void decode_join_kernel(const DecodeArgs a) {
  constexpr int LANES = DH / 4, PARTS = 256 / LANES;
  __shared__ f32x4 sums[PARTS][LANES];
  __shared__ float weight[PARTS], tops[4];
  const int lane = threadIdx.x & 63, b = blockIdx.x / a.H, head = blockIdx.x - b * a.H, hk = head / a.G, g = head - hk * a.G;
  const int units = seq_units(a, b), d4 = threadIdx.x % LANES, part = threadIdx.x / LANES;
  char* y = a.Y.p + b * a.Y.row + (int64_t)head * a.Y.head;
  if (units == 0) {
    if (part == 0) *reinterpret_cast<uint2*>(y + d4 * 8) = make_uint2(0u, 0u);
    return;
  }
  const Line line = unit_line(a);
  const int u0 = units_before(a, b) + (hk * a.sets + g / 16) * units, u1 = u0 + units;
  const int s0 = u0 / line.share, s1 = (u1 - 1) / line.share;
  if (s0 == s1) return;                                      // finished where it was read
  auto row_of = [&](int s) { return (int64_t)(2 * s + (s == s0 && s0 * line.share != u0 ? 1 : 0)) * a.rows + g % 16; };
  float M = -INFINITY;
  for (int s = s0 + (int)threadIdx.x; s <= s1; s += 256) M = fmaxf(M, a.stat[row_of(s) * 2]);
  M = wave_max(M);
  if (lane == 0) tops[threadIdx.x >> 6] = M;
  __syncthreads();
  M = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  const float ms = M == -INFINITY ? 0.f : M;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  float L = 0.f;
#pragma unroll 4
  for (int s = s0 + part; s <= s1; s += PARTS) {
    const int64_t row = row_of(s);
    const float f = __builtin_amdgcn_exp2f(a.stat[row * 2] - ms);
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part + row * DH + 4 * d4);
    L = fmaf(f, a.stat[row * 2 + 1], L);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = fmaf(f, x[e], sum[e]);
  }
  sums[part][d4] = sum;
  if (d4 == 0) weight[part] = L;
  __syncthreads();
  if (part > 0) return;
#pragma unroll
  for (int p = 1; p < PARTS; ++p) {
    L += weight[p];
    const f32x4 x = sums[p][d4];
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += x[e];
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  *reinterpret_cast<uint2*>(y + d4 * 8) = make_uint2(pack_bf16x2(sum[0] * inv, sum[1] * inv), pack_bf16x2(sum[2] * inv, sum[3] * inv));
}

// ------------------------------------------------------------------------------------------
int check_cache(const spt_cache_shape_t* s) {
  if (!s) return SPT_ERR_ARG;
  if (s->pages < 1 || s->page < 1 || s->Hk < 1 || s->dh < 1 || s->B < 1 || s->max_pages < 1) return SPT_ERR_ARG;
  if ((int64_t)s->max_pages * s->page > INT_MAX) return SPT_ERR_ARG;
  if (s->page < 16 || s->page > 256 || (s->page & (s->page - 1)) || (s->dh != 64 && s->dh != 128)) return SPT_ERR_UNSUPPORTED;
  if ((s->format != SPT_CACHE_BF16 && s->format != SPT_CACHE_E4M3) || s->B > 65535 || s->Hk > 65535) return SPT_ERR_UNSUPPORTED;
  return SPT_OK;
}

int check_pool(const spt_cache_shape_t& s, const void* Kc, const void* Vc, const uint8_t* ks, const uint8_t* vs, const int32_t* table) {
  if (!aligned_to(Kc, 16) || !aligned_to(Vc, 16) || !aligned_to(table, 4)) return SPT_ERR_ARG;
  const bool e4m3 = s.format == SPT_CACHE_E4M3;
  if (e4m3 ? (!aligned_to(ks, 16) || !aligned_to(vs, 16)) : (ks || vs)) return SPT_ERR_ARG;
  return SPT_OK;
}

CacheArgs cache_args(const spt_cache_shape_t& s, const void* Kc, const void* Vc, const uint8_t* ks, const uint8_t* vs, const int32_t* table) {
  return {const_cast<char*>(static_cast<const char*>(Kc)), const_cast<char*>(static_cast<const char*>(Vc)), const_cast<uint8_t*>(ks),
          const_cast<uint8_t*>(vs), table, s.pages, __builtin_ctz(s.page), s.Hk, s.B, s.max_pages};
}

constexpr int kMostRows = (1 << 26) - 1;   // (a wavefront each)

int check_rows(const spt_cache_shape_t* s, int32_t T, const void* K, const void* V, const int64_t* strides, const int32_t* start, const int32_t* cu,
               bool output, RowArgs* a) {
  int rc = check_cache(s);
  if (rc != SPT_OK) return rc;
  if (T < 1) return SPT_ERR_ARG;
  if (T > kMostRows) return SPT_ERR_UNSUPPORTED;
  if ((rc = attn_rows(&a->K, K, strides, T, s->Hk, s->dh, output)) != SPT_OK) return rc;
  if ((rc = attn_rows(&a->V, V, strides ? strides + 2 : nullptr, T, s->Hk, s->dh, output)) != SPT_OK) return rc;
  if (!aligned_to(start, 4) || !aligned_to(cu, 4)) return SPT_ERR_ARG;
  a->start = start; a->cu = cu; a->T = T;
  return SPT_OK;
}

// Calls f with the sizes of a shape's decoding kernel.
template <class F>
auto with_tile(const spt_cache_shape_t& s, int H, F f) {
  const bool e4m3 = s.format == SPT_CACHE_E4M3, one = H / s.Hk <= kQueryRows[s.dh == 128];
  if (s.dh == 128) {
    if (e4m3) return one ? f(DecodeTile<128, true, 1>()) : f(DecodeTile<128, true, 4>());
    return one ? f(DecodeTile<128, false, 1>()) : f(DecodeTile<128, false, 4>());
  }
  if (e4m3) return one ? f(DecodeTile<64, true, 1>()) : f(DecodeTile<64, true, 2>());
  return one ? f(DecodeTile<64, false, 1>()) : f(DecodeTile<64, false, 2>());
}

struct DecodeWorkspace { int sets, rows, workgroups; size_t part, bytes; };
DecodeWorkspace plan_decode(const spt_cache_shape_t& s, int H) {
  const int G = H / s.Hk, rows = G < 16 ? G : 16;
  const int workgroups = 256 * with_tile(s, H, [](auto t) { return decltype(t)::PER_CU; });   // as many as are resident at once
  const size_t slots = 2 * (size_t)workgroups * kDecodeWaves * rows;
  const size_t part = align256(slots * s.dh * sizeof(float));
  return {(G + 15) / 16, rows, workgroups, part, part + align256(slots * 2 * sizeof(float))};
}

int check_decode(const spt_cache_shape_t* s, int32_t H) {
  const int rc = check_cache(s);
  if (rc != SPT_OK) return rc;
  if (H < 1 || H % s->Hk != 0) return SPT_ERR_ARG;
  if (H > 65535) return SPT_ERR_UNSUPPORTED;
  const int64_t units = ((int64_t)s->max_pages * s->page + kUnit - 1) / kUnit * s->Hk * ((H / s->Hk + 15) / 16);
  if (units > INT_MAX || units * s->B > INT_MAX || (int64_t)s->B * H > kMostWorkgroups) return SPT_ERR_UNSUPPORTED;
  return SPT_OK;
}

template <int DH, bool E4M3, int QC>
hipError_t launch_decode(DecodeTile<DH, E4M3, QC>, const DecodeArgs& a, hipStream_t st) {
  constexpr int smem = DecodeTile<DH, E4M3, QC>::SMEM;
  static std::atomic<uint64_t> done{0};
  if (const hipError_t e = allow_smem(reinterpret_cast<const void*>(decode_kernel<DH, E4M3, QC>), smem, done); e != hipSuccess) return e;
  {
    ScopedKernelTimer timer(kSlotAttnDecode, st);
    hipLaunchKernelGGL((decode_kernel<DH, E4M3, QC>), dim3(a.workgroups), dim3(64 * kDecodeWaves), smem, st, a);
  }
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  ScopedKernelTimer timer(kSlotAttnDecodeJoin, st);
  hipLaunchKernelGGL(decode_join_kernel<DH>, dim3(a.c.B * a.H), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <int DH, bool E4M3>
hipError_t launch_items(const DecodeArgs& a, hipStream_t st) {
  typedef ItemTile<DH, E4M3> T;
  static std::atomic<uint64_t> done{0};
  if (const hipError_t e = allow_smem(reinterpret_cast<const void*>(decode_item_kernel<DH, E4M3>), T::SMEM, done); e != hipSuccess) return e;
  ScopedKernelTimer timer(kSlotAttnDecode, st);
  hipLaunchKernelGGL((decode_item_kernel<DH, E4M3>), dim3(a.c.B * a.c.Hk * a.sets), dim3(64 * T::WAVES), T::SMEM, st, a);
  return hipGetLastError();
}

// Whether a table is so narrow that a wavefront of an item's workgroup has four units at most: then the launch of the joins costs more than
// an even split gains, but for a few sequences that fill it (the width is what is known on the host).  us a call in a graph, stretches and items, 32 heads on 8 of 128: 32 sequences of 512 tokens 17.3 and 12.4, one of
// them 8.8 and 8.5, 64 of 10 to 1000 in 8 bits 16.4 and 15.9, 16 of 1000 14.2 and 11.7, 4 of them 10.2 and 11.7; one sequence of 100, 32 heads
// of 64: 8.3 and 4.2.  Wider tables: one of 1024 in 16 bits (four wavefronts) 9.4 and 13.6, one of 2048 in 8 bits 9.4 and 17.6.
bool short_table(const spt_cache_shape_t& s) {
  const int waves = s.format == SPT_CACHE_BF16 && s.dh == 128 ? ItemTile<128, false>::WAVES : ItemTile<64, false>::WAVES;
  return (int64_t)s.max_pages * s.page <= 4 * kUnit * waves;
}

}  // namespace

extern "C" int spt_cache_write(const spt_cache_shape_t* shape, int32_t T, const void* K, const void* V, const int64_t* strides,
                               const int32_t* table, const int32_t* start, const int32_t* cu, void* Kc, void* Vc, uint8_t* ks, uint8_t* vs,
                               void* stream) {
  RowArgs a;
  int rc = check_rows(shape, T, K, V, strides, start, cu, false, &a);
  if (rc != SPT_OK) return rc;
  if ((rc = check_pool(*shape, Kc, Vc, ks, vs, table)) != SPT_OK) return rc;
  a.c = cache_args(*shape, Kc, Vc, ks, vs, table);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  ScopedKernelTimer timer(kSlotCacheWrite, st);
  const dim3 grid((T + 3) / 4), block(256);
  const bool e4m3 = shape->format == SPT_CACHE_E4M3;
  if (shape->dh == 128 && e4m3) hipLaunchKernelGGL((cache_write_kernel<128, true>), grid, block, 0, st, a);
  else if (shape->dh == 128) hipLaunchKernelGGL((cache_write_kernel<128, false>), grid, block, 0, st, a);
  else if (e4m3) hipLaunchKernelGGL((cache_write_kernel<64, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((cache_write_kernel<64, false>), grid, block, 0, st, a);
  return hipGetLastError() == hipSuccess ? SPT_OK : SPT_ERR_HIP;
}

extern "C" int spt_cache_read(const spt_cache_shape_t* shape, int32_t T, void* K, void* V, const int64_t* strides, const int32_t* table,
                              const int32_t* start, const int32_t* cu, const void* Kc, const void* Vc, const uint8_t* ks,
                              const uint8_t* vs, void* stream) {
  RowArgs a;
  int rc = check_rows(shape, T, K, V, strides, start, cu, true, &a);
  if (rc != SPT_OK) return rc;
  if ((rc = check_pool(*shape, Kc, Vc, ks, vs, table)) != SPT_OK) return rc;
  a.c = cache_args(*shape, Kc, Vc, ks, vs, table);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  ScopedKernelTimer timer(kSlotCacheRead, st);
  const dim3 grid((T + 3) / 4), block(256);
  const bool e4m3 = shape->format == SPT_CACHE_E4M3;
  if (shape->dh == 128 && e4m3) hipLaunchKernelGGL((cache_read_kernel<128, true>), grid, block, 0, st, a);
  else if (shape->dh == 128) hipLaunchKernelGGL((cache_read_kernel<128, false>), grid, block, 0, st, a);
  else if (e4m3) hipLaunchKernelGGL((cache_read_kernel<64, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((cache_read_kernel<64, false>), grid, block, 0, st, a);
  return hipGetLastError() == hipSuccess ? SPT_OK : SPT_ERR_HIP;
}

extern "C" size_t spt_attn_decode_workspace_bytes(const spt_cache_shape_t* shape, int32_t H) {
  if (check_decode(shape, H) != SPT_OK) return 0;
  return plan_decode(*shape, H).bytes;
}

extern "C" int spt_attn_decode(const spt_cache_shape_t* shape, int32_t H, float scale, const void* Q, const int64_t* strides, const void* Kc,
                               const void* Vc, const uint8_t* ks, const uint8_t* vs, const int32_t* table, const int32_t* lens, void* Y,
                               void* ws, size_t ws_bytes, void* stream) {
  int rc = check_decode(shape, H);
  if (rc != SPT_OK) return rc;
  if (!(scale > 0.f) || !(scale <= kMostScale)) return SPT_ERR_ARG;
  const spt_cache_shape_t& s = *shape;
  DecodeArgs a;
  if ((rc = attn_rows(&a.Q, Q, strides, s.B, H, s.dh, false)) != SPT_OK) return rc;
  if ((rc = attn_rows(&a.Y, Y, strides ? strides + 2 : nullptr, s.B, H, s.dh, true)) != SPT_OK) return rc;
  if ((rc = check_pool(s, Kc, Vc, ks, vs, table)) != SPT_OK) return rc;
  if (!aligned_to(lens, 4) || !aligned_to(ws, 256)) return SPT_ERR_ARG;
  const DecodeWorkspace w = plan_decode(s, H);
  if (ws_bytes < w.bytes) return SPT_ERR_WORKSPACE;
  a.c = cache_args(s, Kc, Vc, ks, vs, table);
  a.lens = lens;
  a.part = static_cast<float*>(ws);
  a.stat = reinterpret_cast<float*>(static_cast<char*>(ws) + w.part);
  a.H = H; a.G = H / s.Hk; a.sets = w.sets; a.rows = w.rows;
  a.workgroups = w.workgroups;
  a.cs = scale * kLog2e;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (short_table(s)) {
    const bool e4m3 = s.format == SPT_CACHE_E4M3;
    const hipError_t e = s.dh == 128 ? (e4m3 ? launch_items<128, true>(a, st) : launch_items<128, false>(a, st))
                                     : (e4m3 ? launch_items<64, true>(a, st) : launch_items<64, false>(a, st));
    return e == hipSuccess ? SPT_OK : SPT_ERR_HIP;
  }
  const hipError_t e = with_tile(s, H, [&](auto t) { return launch_decode(t, a, st); });
  return e == hipSuccess ? SPT_OK : SPT_ERR_HIP;
}
