// What the kernels of full attention share (attn_prompt.hip, attn_prompt_bwd.hip, attn_cache.hip): row tiles in
// LDS, the search for a workgroup's sequence, checks of arguments.  gfx950 only.
#pragma once
#include <limits.h>
#include <math.h>

#include <atomic>

#include "../../include/spt_attn.h"
#include "ffn_common.hpp"
#include "profile.hpp"
#include "spt_host.hpp"

namespace spt {

// A tensor of rows [T][heads][dh] bf16, with the bytes from a row to the next and from a head to the next.
struct AttnRows {
  char* p;
  int64_t row, head;
};

// ---- host side

inline bool aligned_to(const void* p, size_t a) { return p && (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Rows T, heads, of a tensor at p; strides: its two numbers or null (dense).  An output's rows and heads must not overlap.
inline int attn_rows(AttnRows* r, const void* p, const int64_t* strides, int64_t T, int heads, int dh, bool output) {
  if (!aligned_to(p, 16)) return SPT_ERR_ARG;
  const int64_t row = strides ? strides[0] : (int64_t)heads * dh, head = strides ? strides[1] : dh;
  if (row < 0 || head < 0 || row % 8 != 0 || head % 8 != 0) return SPT_ERR_ARG;
  if (row >= (1 << 23) || head >= (1 << 23)) return strides ? SPT_ERR_UNSUPPORTED : SPT_ERR_ARG;
  if (output) {
    const bool rows_in_head = heads == 1 || head >= (T - 1) * row + dh, heads_in_row = T == 1 || row >= (heads - 1) * head + dh;
    if ((T > 1 && row < dh) || (heads > 1 && head < dh) || (!rows_in_head && !heads_in_row)) return SPT_ERR_ARG;
  }
  *r = AttnRows{const_cast<char*>(static_cast<const char*>(p)), row * 2, head * 2};
  return SPT_OK;
}

// Lets a kernel use `smem` bytes of LDS: asked for once on each GPU (a call of the runtime costs a launch a tenth of its time).
inline hipError_t allow_smem(const void* kernel, int smem, std::atomic<uint64_t>& done) {
  int dev = 0;
  if (const hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

constexpr float kMostScale = 2e38f;                    // times log2 e it is finite
constexpr int64_t kMostWorkgroups = (1 << 23) - 16;   // of up to 512 threads: a launch has fewer than 2^32

int check_attn(const spt_attn_shape_t* s);   // attn_prompt.hip
int attn_heads_shift(int G);                // log2 of the heads of a group of G that share a workgroup

// How coarsely find_tile orders tiles by their work, as a power of two: as many tiles as there are rounds of resident workgroups.  Strictly
// by work, tiles that read the same rows are as far apart as there are sequences, and L2 does not hold what lies between; in few rounds the
// order matters more.  us of the forward with `causal`, by work alone, so, and sequence by sequence: 32 heads of 128, 48 sequences of
// 512 (12 rounds) 280, 196, 197; 32 of 33 to 2000 424, 380, 370; 32 heads on 8, 48 of 33 to 2000 563, 524, 514; 32 heads of 64,
// 64 of 512 173, 142, 141, 8 of them (one round) 23.2, 23.3, 28.5.
inline int coarse_tiles(int64_t workgroups, int on_a_cu) {
  const int64_t rounds = workgroups / (256 * on_a_cu);
  return rounds < 1 ? 0 : 63 - __builtin_clzll(rounds);
}

// Workgroups of 1 << shift rows for each of `heads`: about as many as there are, and one for each sequence at least.
inline int64_t row_workgroups(int T, int shift, int B, int heads) { return (int64_t)(T >> shift > B ? T >> shift : B) * heads; }

// Wavefronts of a workgroup that own 32 rows each (of up to 1 << hshift heads): four, or, where all workgroups still fit onto the chip at once,
// two or one; four or eight groups of them then share what passes through LDS, if that is enough (`through` rows of B sequences).
// us, four (in the forward with two groups) and fewer owners.  Forward: 8 heads of 128, 256 tokens 10.8 and 10.3, 512 14.3 and 12.1; 2 heads of
// 64, 4000 42 and 23, 8 heads, 2000 25.5 and 19.3.  Query side of the gradients: 12 heads of 64, 160 11.5 and 12.2, 256 14.1 and 12.6, 512 20.7
// and 14.0, 1024 28 and 17; 2 heads, 4000 106 and 32; 12 heads, 16 times 8 queries behind 500 keys 19.4 and 13.3.  Key side: 12 heads of 64, 77
// 10.5 and 11.8, 160 13.4 and 12.1, 512 24.5 and 14.3, 1024 33 and 18.5; 32 heads of 64 on 8, 512 61 and 23, of 128 on 8 63 and 37, two of
// 1000 117 and 77.  One owner and two: 24 heads of 64, 384 (288 workgroups of one) query side 20.6 and 12.9, key side 20.3 and 13.0.  One owner
// and four: 21 times 3 queries behind 1000 keys, 64 heads of 64 on 16 (1344 of one) forward 67 and 27.
// Two rounds of two owners still gain where there is much to share and the second round fills up: with `causal`, whose workgroups are unequal,
// and 64-wide heads, of which one workgroup of four leaves a CU's wavefronts waiting.  us, four owners and two, `causal`: 8 heads, 4000 tokens (500
// workgroups), of 64 forward 44 and 34, query side 89 and 49, key side 105 and 55, of 128 58 and 54, 132 and 81, 114 and 87; 31 sequences of 4 to
// 1993, 4 heads of 64 on 2 key side 109 and 49; 4 of 512, 16 heads of 64 query side 19.2 and 21.6; two of 4000, 8 heads of 128 (1000) key side
// 137 and 169.  All keys seen: 8 heads of 64, 4000 48 and 50, 90 and 81, 105 and 91, of 128 69 and 88, 142 and 137, 129 and 150 (one rule for three kernels: the
// forward's 2 us at 64 are less than the other two gain).
inline int row_owners(int T, int heads, int hshift, int64_t through, const spt_attn_shape_t& s) {
  const int hs = hshift < 1 ? hshift : 1;
  const int64_t ones = row_workgroups(T, 5, s.B, heads), twos = row_workgroups(T, 6 - hs, s.B, heads >> hs), B = s.B;
  if (through < 192 * B) return 4;
  if (ones <= 256) return 1;
  return twos <= 256 || (twos <= 512 && through >= 640 * B && (s.causal || s.dh == 64)) ? 2 : 4;
}

// ---- device side

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A word at an address that all lanes share, through the scalar cache: vector memory's counter, which the copies into
// LDS are waited for by, does not see it.
__device__ __forceinline__ int32_t uniform_load(const int32_t* p) {
  return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(p));
}

// A sequence's rows of a packed tensor.
struct SeqRows { int first, n; };
__device__ __forceinline__ SeqRows seq_rows(const int32_t* cu, int b, int T) {
  const int lo = min(max(cu[b], 0), T), hi = min(max(cu[b + 1], 0), T);
  return {lo, max(0, hi - lo)};
}

// Sum over the lanes up to and including this one: six additions across lanes.
__device__ __forceinline__ int wave_prefix(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);   // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // row_bcast 15 into rows 1 and 3, 31 into 2 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
  return x;
}
__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_prefix(x), 63); }

// A workgroup's row tile: its number in its sequence, and the sequence's rows in both tensors.
struct TilePlace {
  int tile;
  SeqRows own, other;
};

// Tile t in the order in which workgroups take them.  All lanes of a wavefront look together.  64 sequences at a time: the tiles
// with the most work first, whatever their sequence (work in tiles of the other side: with `causal` tile k of queries has k and the
// keys that were there before, tile k of keys, FROM_END, what is left behind it; without, every tile all rows of the other side).  With `causal`
// 1 << coarse tiles of work count as the same, and those of a sequence come one after the other.
template <bool FROM_END>
__device__ __forceinline__ bool find_tile(const int32_t* cu_own, const int32_t* cu_other, int B, int Town, int Tother, int shift, bool causal,
                                          int coarse, int t, TilePlace& p) {
  const int lane = threadIdx.x & 63, round = (1 << shift) - 1;
  SeqRows own = {0, 0}, other = {0, 0};
  int n, total;                                            // tiles of the lane's sequence, of 64
  for (int b0 = 0;; b0 += 64, t -= total) {
    if (b0 >= B) return false;
    own = b0 + lane < B ? seq_rows(cu_own, b0 + lane, Town) : SeqRows{0, 0};
    n = (own.n + round) >> shift;
    total = wave_total(n);
    if (t < total) {
      if (b0 + lane < B) other = seq_rows(cu_other, b0 + lane, Tother);
      break;
    }
  }
  const int base = !causal ? other.n >> shift : FROM_END ? 0 : max(0, other.n - own.n) >> shift;
  // tiles of the lane's sequence with work of at least x + 1 steps
  auto count = [&](int x) { return causal ? min(max(base + n - (x << coarse), 0), n) : base >= x ? n : 0; };
  int lo = 0, hi = 1, b = 0;                               // total(lo) > t >= total(hi)
  if (B == 1) {
    p.tile = causal ? __builtin_amdgcn_readfirstlane(n) - 1 - t : t;
  } else {
    for (; wave_total(count(hi)) > t; hi *= 2) lo = hi;
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if (wave_total(count(mid)) > t) lo = mid;
      else hi = mid;
    }
    const int more = count(hi), incl = wave_prefix(count(lo) - more);
    t -= wave_total(more);
    b = __builtin_ctzll(__ballot(incl > t));
    if (b > 0) t -= __builtin_amdgcn_readlane(incl, b - 1);
    p.tile = causal ? __builtin_amdgcn_readlane(n - more, b) - 1 - t : t;
  }
  if (FROM_END && causal) p.tile = __builtin_amdgcn_readlane(n, b) - 1 - p.tile;
  p.own = {__builtin_amdgcn_readlane(own.first, b), __builtin_amdgcn_readlane(own.n, b)};
  p.other = {__builtin_amdgcn_readlane(other.first, b), __builtin_amdgcn_readlane(other.n, b)};
  return true;
}

// Workgroups over (key head, item): all items of a key head, which read the same keys and values, on one XCD (workgroup id mod 8) where
// the heads are a multiple of eight, on as few XCDs as there are for each where they divide eight, and the items of all heads of an XCD
// in order.
struct HeadItem { int hk, item; };
inline int head_item_grid(int Hk, int items) { return Hk % 8 == 0 || 8 % Hk != 0 ? Hk * items : (int)(((int64_t)items * Hk + 7) / 8 * 8); }
__device__ __forceinline__ HeadItem head_item(int id, int Hk) {
  if (Hk % 8 == 0) {
    const int per = Hk >> 3, j = id >> 3;
    return {(id & 7) * per + j % per, j / per};
  }
  if (8 % Hk == 0) return {(id & 7) % Hk, (id >> 3) * (8 / Hk) + (id & 7) / Hk};   // (may be one of the few past the last)
  return {id % Hk, id / Hk};
}

// 16-byte chunk of a tile of rows of RB bytes in LDS: chunk c of row r sits at c ^ chunk_swizzle(r).  Sixteen rows at one
// chunk (an MFMA operand's reads), four rows at four adjacent chunks and eight rows at two (transposing reads) all reach all banks.
template <int RB>
__device__ __forceinline__ uint32_t chunk_swizzle(int r) {
  const uint32_t low = ((r >> 1) & 2) | ((r >> 3) & 1);   // bits 2 and 3 of r
  return RB == 256 ? (uint32_t)((r & 3) << 2) | low : RB == 128 ? (uint32_t)(((r >> 1) & 1) << 2) | low : low;
}
template <int DH>
__device__ __forceinline__ uint32_t row_swizzle(int r) { return chunk_swizzle<DH * 2>(r); }

// Asynchronous copy global -> LDS, 16 bytes per lane from base + off; lane L's data lands at lds_base + 16 L.
__device__ __forceinline__ void dma16_at(const void* base, uint32_t off, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_base), "v"(off), "s"(base) : "memory");
}
// The same for what a launch reads once: it does not stay in L2.
__device__ __forceinline__ void dma16_once(const void* base, uint32_t off, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds_base), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) { return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)p); }

// 16 (8) bytes of whole lines that this launch does not read again: not kept in L2, which the end of a launch would wait to have written
// (rows written to a cache and read back, 102 MB each way: 52.5 us kept, 47.3 so; stores that leave lines in parts lose by it).
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <class T>
__device__ __forceinline__ void stream_out(char* p, T v) { __builtin_nontemporal_store(v, reinterpret_cast<T*>(p)); }
template <class T>
__device__ __forceinline__ T stream_in(const char* p) { return __builtin_nontemporal_load(reinterpret_cast<const T*>(p)); }

// LDS by its 32-bit address.
template <class T>
__device__ __forceinline__ T lds_read(uint32_t at) {
  return *reinterpret_cast<const __attribute__((address_space(3))) T*>((uintptr_t)at);
}
__device__ __forceinline__ bf16x8 lds_tr_read(uint32_t lo, uint32_t hi) {
  struct { v4s a, b; } t;
  t.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_v4s_ptr>((uintptr_t)lo));
  t.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_v4s_ptr>((uintptr_t)hi));
  return __builtin_bit_cast(bf16x8, t);
}

// Operands out of a row tile (256-byte aligned).
// rows(): 8 dims (16 ks + 8 h ..) of row 32 n + lane % 32, the operand whose K is the head dimension.
// columns(): 32 dims (32 d ..) x 16 rows (16 n ..), transposed, the operand whose K are the rows.  MFMA row i is dim 32 d + rho32(i), so
// that a lane's 16 results are adjacent dims; K slot (h, e) is row 16 n + 8 (e / 4) + 4 h + e % 4, the order in which a
// lane holds the results of a product whose rows are these.
// Everything but two words per lane is an exclusive-or with a constant or an offset in the instruction: `fresh` keeps the
// compiler from computing all addresses in front of a loop, for which there are no registers.
template <int DH>
struct TileReader {
  uint32_t row, col;   // offsets in a tile
  __device__ __forceinline__ explicit TileReader(int lane) {
    const int i = lane & 31, h = lane >> 5, g = lane >> 4, sl = lane & 15, a4 = sl & 3, r = 4 * (g >> 1) + (sl >> 2);
    row = i * (DH * 2) + ((uint32_t)h ^ row_swizzle<DH>(i)) * 16;
    col = r * (DH * 2) + ((uint32_t)(2 * (a4 & 1) + (g & 1)) ^ row_swizzle<DH>(r)) * 16 + (a4 >> 1) * 8;
  }
  __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(row), "+v"(col)); }
  __device__ __forceinline__ bf16x8 rows(uint32_t tile, int n, int ks) const {
    return lds_read<bf16x8>((tile + row ^ (uint32_t)(ks * 32)) + n * (32 * DH * 2));
  }
  __device__ __forceinline__ bf16x8 columns(uint32_t tile, int n, int d) const {
    const uint32_t lo = tile + col ^ (uint32_t)(d * 64);
    return lds_tr_read(lo + n * (16 * DH * 2), (lo ^ 16u) + (n * 16 + 8) * (DH * 2));   // (rows 8 on: bit 3 of the row is in the swizzle)
  }
};

// 32 rows between memory and a wavefront's own tile in LDS, as whole lines (a lane's own row in registers would be 16 bytes
// of 64 lines an instruction).  In: asynchronous, rows past n: the last one again.  Out: rows past n are left out.
template <int DH>
__device__ __forceinline__ void fetch_rows(const char* x, int64_t row, int n, uint32_t tile, int lane) {
  constexpr int CHUNKS = DH / 8, ROWS = 64 / CHUNKS;
#pragma unroll
  for (int u = 0; u < 32 / ROWS; ++u) {
    const int r = u * ROWS + lane / CHUNKS;
    dma16_at(x, (uint32_t)min(r, n - 1) * (uint32_t)row + (((uint32_t)lane % CHUNKS) ^ row_swizzle<DH>(r)) * 16, tile + u * 1024);
  }
}
// The same rows by way of registers: lane L holds 16 bytes of rows u ROWS + L / CHUNKS.
template <int DH>
struct RowPieces {
  static constexpr int CHUNKS = DH / 8, ROWS = 64 / CHUNKS, N = 32 / ROWS;
  u32x4 x[N];
  __device__ __forceinline__ void load(const char* p, int64_t row, int n, int lane) {
#pragma unroll
    for (int u = 0; u < N; ++u) x[u] = *reinterpret_cast<const u32x4*>(p + min(u * ROWS + lane / CHUNKS, n - 1) * row + (lane % CHUNKS) * 16);
  }
  __device__ __forceinline__ void put(char* tile, int lane) const {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int r = u * ROWS + lane / CHUNKS;
      *reinterpret_cast<u32x4*>(tile + r * (DH * 2) + (((uint32_t)lane % CHUNKS) ^ row_swizzle<DH>(r)) * 16) = x[u];
    }
  }
};
// 16 adjacent dims of row r, from 16-byte chunk c on.
template <int DH>
__device__ __forceinline__ void put_dims(char* tile, int r, int c, bf16x8 lo, bf16x8 hi) {
  const uint32_t at = r * (DH * 2) + ((uint32_t)c ^ row_swizzle<DH>(r)) * 16;
  *reinterpret_cast<bf16x8*>(tile + at) = lo;
  *reinterpret_cast<bf16x8*>(tile + (at ^ 16u)) = hi;
}
template <int DH>
__device__ __forceinline__ void store_rows(const char* tile, char* x, int64_t row, int n, int lane, bool stream = false) {
  constexpr int CHUNKS = DH / 8, ROWS = 64 / CHUNKS;
#pragma unroll
  for (int u = 0; u < 32 / ROWS; ++u) {
    const int r = u * ROWS + lane / CHUNKS;
    const u32x4 v = *reinterpret_cast<const u32x4*>(tile + u * 1024 + lane * 16);
    char* to = x + r * row + (((uint32_t)lane % CHUNKS) ^ row_swizzle<DH>(r)) * 16;
    if (r < n && stream) {
      asm volatile("");                                    // (or the compiler makes one store of the two, and keeps it in L2)
      stream_out(to, v);
      asm volatile("");
    } else if (r < n) {
      *reinterpret_cast<u32x4*>(to) = v;
    }
  }
}

__device__ __forceinline__ float other_half(float x) {   // the value of the lane 32 away
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// Eight fp32 -> an MFMA operand, nearest even.
__device__ __forceinline__ bf16x8 pack8(const float* x) {
  return as_bf16x8(u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])});
}

// The two halves of a word, as bf16, and c.
__device__ __forceinline__ float sum2(uint32_t w, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3F803F80u), c, false);
}

// Whether any of the bf16 looked at was infinite or NaN: the largest magnitude, two halves at a time.
struct NotFinite {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  u16x2 top = {0, 0};
  __device__ __forceinline__ void look(u32x4 x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x[e] & 0x7FFF7FFFu));
  }
  __device__ __forceinline__ void mark(bool yes) { top[0] = yes ? 0x7F80 : top[0]; }
  __device__ __forceinline__ bool found() const { return top[0] >= 0x7F80 || top[1] >= 0x7F80; }
};

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

// dot product of two rows of dh values, one lane's.
__device__ __forceinline__ float row_dot(const char* a, const char* b, int dh) {
  float s = 0.f;
  for (int c = 0; c < dh; c += 8) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(a + c * 2), y = *reinterpret_cast<const u32x4*>(b + c * 2);
#pragma unroll
    for (int e = 0; e < 4; ++e) s = fmaf(hi_bf16(x[e]), hi_bf16(y[e]), fmaf(lo_bf16(x[e]), lo_bf16(y[e]), s));
  }
  return s;
}
__device__ __forceinline__ float bf16_at(const char* p) { return bf16_to_f32(*reinterpret_cast<const uint16_t*>(p)); }

}  // namespace spt
