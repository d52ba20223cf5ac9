// K/V caches held in 4 bits and in pages (format and tables: include/sa.h): writing rows, reading them back, attention of the
// last T tokens of every sequence over them (the decoding of Sec. 4.2).
//
// Every value held is E2M1 times a power of two of at least 2^-125, an exact bf16 number: K and V enter the matrix products
// exactly, and what rounding there is lies in q (none in bf16), in the probabilities and in the sums.
#include <math.h>

#include "sa_cache4.h"
#include "sa_mfma.h"

namespace sa {
namespace {

constexpr int kTile = 32;  // rows of a tile

// A tile's parts, in bytes from its start, and what a lane (r, g) = (lane % 16, lane / 16) owns of it.
template <int D>
struct Tile {
  static constexpr int kBytes = 34 * D;
  static constexpr int kV = 16 * D, kKs = 32 * D, kVs = 33 * D;
  static constexpr int E = D / 16;       // elements of a row per lane of 16
  static constexpr int RB = D / 32;      // their bytes
  static constexpr int LPB = 32 / E;     // lanes of a block of 32 elements
  // row of the tile that is number j (0..7) of lane group g: 4 g .. 4 g + 3 of each half
  static __device__ __forceinline__ int row(int g, int j) { return 16 * (j >> 2) + 4 * g + (j & 3); }
};

struct Cache {
  unsigned char* pool;
  const int32_t* table;
  int B, Hkv, pages, max_pages;
  int tiles_log2;   // tiles of a page and head
  int capacity;     // rows of a sequence at most
};

// Number of a tile in the pool (of head hk, holding row 32 * tile of sequence b), or -1 if its page is not there.
__device__ __forceinline__ int tile_number(const Cache& c, int b, int hk, int tile) {
  const int page = c.table[(size_t)b * c.max_pages + (tile >> c.tiles_log2)];
  if ((unsigned)page >= (unsigned)c.pages) return -1;
  return ((page * c.Hkv + hk) << c.tiles_log2) + (tile & ((1 << c.tiles_log2) - 1));
}

template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
  return v > o ? v : o;
}
// Largest over the LPB lanes of a block of 32 elements, and over the 16 lanes of a row.
template <int LPB>
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
  v = max_dpp<0xB1>(v);                  // quad_perm [1,0,3,2]
  v = max_dpp<0x4E>(v);                  // quad_perm [2,3,0,1]
  return LPB == 8 ? max_dpp<0x141>(v) : v;  // row_half_mirror
}
template <int LPB>
__device__ __forceinline__ uint32_t row_max(uint32_t v) {   // of block_max's results
  if (LPB == 4) v = max_dpp<0x141>(v);
  return max_dpp<0x140>(v);              // row_mirror
}

template <typename T, int E>
struct Elements;  // E neighbouring elements of a row

template <int E>
struct Elements<bf16_t, E> {
  uint32_t w[E / 2];
  __device__ __forceinline__ void load(const bf16_t* p) {
    if constexpr (E == 8) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = x[i];
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(p);
      w[0] = x[0]; w[1] = x[1];
    }
  }
  // largest magnitude as the bits of an fp32 number (an infinity or NaN is above all others)
  __device__ __forceinline__ uint32_t top() const {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < E / 2; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    const uint32_t lo = (uint32_t)m[0] << 16, hi = __builtin_bit_cast(uint32_t, m) & 0xffff0000u;
    return lo > hi ? lo : hi;
  }
  __device__ __forceinline__ uint32_t codes(float scale) const {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[1]), scale, 1);
    if constexpr (E == 8) {
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[2]), scale, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[3]), scale, 3);
    }
    return c;
  }
};

template <int E>
struct Elements<float, E> {
  float x[E];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[i + k] = v[k];
    }
  }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const uint32_t u = __float_as_uint(x[i]) & 0x7fffffffu;
      m = m > u ? m : u;
    }
    return m;
  }
  __device__ __forceinline__ uint32_t codes(float scale) const {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
    if constexpr (E == 8) {
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
    }
    return c;
  }
};

// The scale byte of a block whose largest magnitude has the bits `top`: its exponent less 2, one more past 1.75 (7/4) of the power;
// held to 2 (every value a normal number) .. 252 (4 * 2^126 would be none).
constexpr uint32_t kNoRow = 255, kOne = 127;
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  const int e = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return top == 0 ? kOne : (uint32_t)min(max(e, 2), 252);
}

struct RowsArgs {
  Cache c;
  const int32_t* starts;
  const int32_t* counts;
  void* K;
  void* V;
  int T, tiles;  // tiles a sequence's rows can touch
};

// What a wave of the two row kernels works on: a half of 16 rows of a tile, 4 a lane group, K and V of a row by the same lanes.
struct Rows {
  int b, hk, tile, half;  // tile: -1 outside the sequence's positions
  long t0;                // t of the half's first row
  int count;
  bool any, whole;        // whether rows of the half are among those asked for, and all
};
constexpr int kRowWaves = 4;
// Half k of those that the rows starts .. can touch; plain arithmetic, which the host's tests go through as well.
struct HalfRows { long tile, t0; bool any; };
__host__ __device__ __forceinline__ HalfRows half_rows(int start, int count, int tiles, int k) {
  HalfRows h;
  h.tile = (long)(start >> 5) + (k >> 1);
  h.t0 = h.tile * kTile + 16 * (k & 1) - start;
  h.any = count > 0 && k < 2 * tiles && h.t0 < count && h.t0 + 16 > 0;  // (no rows: also where the first tile is a begun one)
  return h;
}
// The row that is loaded for t: where t is not written, the first or last (of at least one) in its place.
__host__ __device__ __forceinline__ long loaded_row(long t, int count) { return t < 0 ? 0 : t < count ? t : count - 1; }
__host__ __device__ __forceinline__ int tiles_touched(int T) { return (int)(((long)T + 62) / kTile); }  // the first and the last may be begun

__device__ __forceinline__ Rows rows_of_wave(const RowsArgs& a) {
  Rows w;
  const unsigned blocks = (unsigned)(2 * a.tiles + kRowWaves - 1) / kRowWaves, bh = blockIdx.x / blocks;
  const int k = (int)(blockIdx.x % blocks) * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  w.hk = (int)(bh % (unsigned)a.c.Hkv);
  w.b = (int)(bh / (unsigned)a.c.Hkv);
  w.half = k & 1;
  const int start = a.starts ? __builtin_amdgcn_readfirstlane(a.starts[w.b]) : 0;
  w.count = a.counts ? __builtin_amdgcn_readfirstlane(min(max(a.counts[w.b], 0), a.T)) : a.T;
  const HalfRows h = half_rows(start, w.count, a.tiles, k);
  w.t0 = h.t0;
  w.any = h.any;
  w.whole = w.t0 >= 0 && w.t0 + 16 <= w.count;
  w.tile = h.tile < 0 || h.tile * kTile >= a.c.capacity ? -1 : (int)h.tile;
  return w;
}

// A row that holds an infinity or NaN in K or V is marked in both.  Bound: HBM (reads 4 d bytes a row in bf16, writes 17/16 d).
template <typename T, int D>
__global__ __launch_bounds__(kRowWaves * 64) void cache4_write_kernel(RowsArgs a) {
  using L = Tile<D>;
  constexpr int E = L::E;
  const Rows w = rows_of_wave(a);
  if (!w.any || w.tile < 0) return;
  const int number = __builtin_amdgcn_readfirstlane(tile_number(a.c, w.b, w.hk, w.tile));
  if (number < 0) return;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  unsigned char* base = a.c.pool + (size_t)number * L::kBytes;
  const size_t src = ((size_t)w.b * a.c.Hkv + w.hk) * a.T;
  Elements<T, E> k[4], v[4];
  bool in[4];
  const T* kr = reinterpret_cast<const T*>(a.K) + src * D + r * E;
  const T* vr = reinterpret_cast<const T*>(a.V) + src * D + r * E;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const long t = w.t0 + 4 * g + j;
    in[j] = t >= 0 && t < w.count;
    const size_t at = (size_t)loaded_row(t, w.count) * D;
    k[j].load(kr + at);
    v[j].load(vr + at);
  }
  __builtin_amdgcn_sched_barrier(0);  // all loads in flight together
  uint32_t kc[4], vc[4], ks[4], vs[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t kt = block_max<L::LPB>(k[j].top()), vt = block_max<L::LPB>(v[j].top());
    const bool bad = row_max<L::LPB>(kt > vt ? kt : vt) >= 0x7f800000u;
    ks[j] = scale_byte(kt);
    vs[j] = scale_byte(vt);
    kc[j] = k[j].codes(__uint_as_float(ks[j] << 23));
    vc[j] = v[j].codes(__uint_as_float(vs[j] << 23));
    kc[j] = bad ? 0 : kc[j];
    vc[j] = bad ? 0 : vc[j];
    ks[j] = bad ? kNoRow : ks[j];
    vs[j] = bad ? kOne : vs[j];
  }
  // K codes: rows as they are; V codes: the 4 rows of a lane group side by side; scales: by the first lane of a block
  unsigned char* kp = base + (16 * w.half + 4 * g) * (D / 2) + r * L::RB;
  unsigned char* vp = base + L::kV + ((g * 16 + r) * 2 + w.half) * 4 * L::RB;
  const int c = r / L::LPB;
  unsigned char* kq = base + L::kKs + (c * 16 + 4 * g) * 2 + w.half;
  unsigned char* vq = base + L::kVs + ((c * 4 + g) * 2 + w.half) * 4;
  const auto put_k = [&](int j) {
    if constexpr (L::RB == 4) *reinterpret_cast<uint32_t*>(kp + j * (D / 2)) = kc[j];
    else *reinterpret_cast<uint16_t*>(kp + j * (D / 2)) = (uint16_t)kc[j];
    if (r % L::LPB == 0) kq[2 * j] = (unsigned char)ks[j];
  };
  if (w.whole) {
#pragma unroll
    for (int j = 0; j < 4; ++j) put_k(j);
    if constexpr (L::RB == 4) *reinterpret_cast<u32x4*>(vp) = u32x4{vc[0], vc[1], vc[2], vc[3]};
    else *reinterpret_cast<u32x2*>(vp) = u32x2{(vc[0] & 0xffffu) | (vc[1] << 16), (vc[2] & 0xffffu) | (vc[3] << 16)};
    if (r % L::LPB == 0) *reinterpret_cast<uint32_t*>(vq) = vs[0] | vs[1] << 8 | vs[2] << 16 | vs[3] << 24;
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (in[j]) {
      put_k(j);
      if constexpr (L::RB == 4) reinterpret_cast<uint32_t*>(vp)[j] = vc[j];
      else reinterpret_cast<uint16_t*>(vp)[j] = (uint16_t)vc[j];
      if (r % L::LPB == 0) vq[j] = (unsigned char)vs[j];
    }
}

// E elements from their codes (low bytes of c), times the scale
template <typename T, int E>
__device__ __forceinline__ void store_values(T* p, uint32_t c, float scale, bool nan, bool there);
template <>
__device__ __forceinline__ void store_values<bf16_t, 8>(bf16_t* p, uint32_t c, float s, bool nan, bool there) {
  u32x4 o;
  o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
  o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
  o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
  o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = there ? (nan ? 0x7fc07fc0u : o[i]) : 0u;
  *reinterpret_cast<u32x4*>(p) = o;
}
template <>
__device__ __forceinline__ void store_values<bf16_t, 4>(bf16_t* p, uint32_t c, float s, bool nan, bool there) {
  u32x2 o;
  o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
  o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
#pragma unroll
  for (int i = 0; i < 2; ++i) o[i] = there ? (nan ? 0x7fc07fc0u : o[i]) : 0u;
  *reinterpret_cast<u32x2*>(p) = o;
}
__device__ __forceinline__ void store4(float* p, f32x2 a, f32x2 b, bool nan, bool there) {
  const float q = __uint_as_float(0x7fc00000u);
  f32x4 o = {a[0], a[1], b[0], b[1]};
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = there ? (nan ? q : o[i]) : 0.f;
  *reinterpret_cast<f32x4*>(p) = o;
}
template <>
__device__ __forceinline__ void store_values<float, 4>(float* p, uint32_t c, float s, bool nan, bool there) {
  store4(p, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1), nan, there);
}
template <>
__device__ __forceinline__ void store_values<float, 8>(float* p, uint32_t c, float s, bool nan, bool there) {
  store_values<float, 4>(p, c, s, nan, there);
  store4(p + 4, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3), nan, there);
}

// The reverse, lane for lane.  Bound: HBM (writes).
template <typename T, int D>
__global__ __launch_bounds__(kRowWaves * 64) void cache4_read_kernel(RowsArgs a) {
  using L = Tile<D>;
  const Rows w = rows_of_wave(a);
  if (!w.any) return;
  const int number = w.tile < 0 ? -1 : __builtin_amdgcn_readfirstlane(tile_number(a.c, w.b, w.hk, w.tile));
  const bool there = number >= 0;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, c = r / L::LPB;
  const unsigned char* base = a.c.pool + (size_t)(there ? number : 0) * L::kBytes;
  uint32_t kc[4] = {}, vc[4] = {}, vs = 0;
  u32x2 ks = {};  // of both halves
  if (there) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned char* kp = base + (16 * w.half + 4 * g + j) * (D / 2) + r * L::RB;
      if constexpr (L::RB == 4) kc[j] = *reinterpret_cast<const uint32_t*>(kp);
      else kc[j] = *reinterpret_cast<const uint16_t*>(kp);
    }
    const unsigned char* vp = base + L::kV + ((g * 16 + r) * 2 + w.half) * 4 * L::RB;
    if constexpr (L::RB == 4) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(vp);
#pragma unroll
      for (int j = 0; j < 4; ++j) vc[j] = x[j];
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(vp);
#pragma unroll
      for (int j = 0; j < 4; ++j) vc[j] = (x[j / 2] >> (16 * (j & 1))) & 0xffffu;
    }
    ks = *reinterpret_cast<const u32x2*>(base + L::kKs + (c * 16 + 4 * g) * 2);
    vs = *reinterpret_cast<const uint32_t*>(base + L::kVs + ((c * 4 + g) * 2 + w.half) * 4);
  }
  const size_t dst = ((size_t)w.b * a.c.Hkv + w.hk) * a.T;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const long t = w.t0 + 4 * g + j;
    const uint32_t kb = (ks[j / 2] >> (16 * (j & 1) + 8 * w.half)) & 0xffu, vb = (vs >> (8 * j)) & 0xffu;
    if (t >= 0 && t < w.count) {
      const size_t at = (dst + (size_t)t) * D + r * L::E;
      const bool nan = kb == kNoRow;
      store_values<T, L::E>(reinterpret_cast<T*>(a.K) + at, kc[j], __uint_as_float(kb << 23), nan, there);
      store_values<T, L::E>(reinterpret_cast<T*>(a.V) + at, vc[j], __uint_as_float(vb << 23), nan, there);
    }
  }
}

// ---- attention ----------------------------------------------------------------------------------------------------------------
//
// The g query heads of a KV head and the T tokens are g T query rows that read the same cache: rows c = h T + t, as they lie in
// memory.  A wave takes NT blocks of 16 of them and a tile of 32 cached rows at a time:
//   S^T (16 cached rows x 16 query rows, twice) = K Q^T, lane (r, g) holding cached row r, elements D/4 g .. of it as they lie in
//   the tile (which elements a lane group takes in a step is free as long as Q's operand agrees); the result leaves lane (c, g)
//   with query row c and cached rows 4 g + i of each half;
//   O^T (16 elements x 16 query rows, D/16 times) += V^T P^T, where those scores are the operand P^T as they stand and lane (r, g) holds
//   elements E r .. E r + E - 1 of the same 8 cached rows: the order in which V lies in the tile.
// No operand passes through LDS.  4-bit codes become pairs by one conversion each, which multiplies by the power of two as well; V's
// pairs are re-paired over two rows by byte permutes.  K and q are bf16 (fp32 q: three parts of 8 bits), V and the probabilities
// f16, whose 11 bits keep a probability eight times as well as bf16's would (fp32: two parts); where a tile's scales of V are out of
// f16's reach the wave's tiles are gone through again in bf16 with a part more.
// Bound.  One token: the K/V rows once, d + d/16 bytes a row, HBM: 16 x 8192 rows of 8 KV heads of 128 (143 MB) 31 us with the
// merge, the kernel itself 5.3 TB/s; a tile is 184 vector instructions, which bound the chip at 11 TB/s.  Many tokens: the vector ALU
// (T509 over 32768 rows, 32 / 8 heads 296 us, 0.92 PFLOP/s: active in 87 % of the waves' cycles, the matrix pipe in 43 %): of 254 instructions for 32 query rows
// half unpack the tile.  Sharing that over the waves of a workgroup through LDS left 150 and took as long, LDS reads and barriers in
// its place; 48 rows a wave 302 us, 64 rows 433 (one wave a SIMD).
struct AttnArgs {
  Cache c;
  const void* q;
  void* Y;
  float* LSE;
  float* part;  // [Hkv][rows][B*splits][D + 2]: weighted V sum, maximum (log2 domain), sum
  int32_t* dealt;  // [2][64]: a sequence's first piece and their number, or NULL: splits of them each
  const int32_t* lens;
  int T, rows, row_blocks, max_len, chunk, splits, pieces;
  uint32_t few;  // tiles of all sequences below which pieces are dealt by length
  float scale_log2e;
};

struct MergeArgs {
  const float* part;
  const int32_t* dealt;
  void* Y;
  float* LSE;
  int rows, splits, pieces, all;  // rows of a sequence, all KV heads; all: slots of all sequences
};

// The maximum is raised where a score passes it by more than 2^kRaise: the usual tile needs no exchange between lanes and no product with a
// correction.  With the lift the largest probability is 2^15, a row's own largest at least 2^7, and f16 holds all its bits down to 2^-14.  Over
// values of V past f16's reach the lift is lowered (bf16_lift), so that no sum overflows.
// kNone: the maximum before a row has been seen, the lowest number (a row that is not seen has the score -inf).
constexpr float kRaise = 8.f, kLift = 7.f, kNone = -3.402823466e38f;

// A query that sees nothing has the maximum -inf; one whose scores are all -inf kNone and a sum of 0, which beside any number counts for nothing and by
// itself leaves 0/0.
__device__ __forceinline__ float weighted_mean(float m, float v, float sum) { return m == -INFINITY ? 0.f : v / sum; }
__device__ __forceinline__ float log_of_sum(float m, float sum) { return sum == 0.f ? (m == -INFINITY ? m : __uint_as_float(0x7fc00000u)) : (m + log2f(sum)) * kLn2; }

__device__ __forceinline__ float exp2_above(float a, float ref) { return exp2f(a - (ref == -INFINITY ? 0.f : ref)); }

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// x and y as PARTS numbers of 8 (bf16) or 11 bits (f16) whose sums they are to PARTS times as many, in the words w[part]
template <int PARTS>
__device__ __forceinline__ void split_pair_bf16(float x, float y, uint32_t* w) {
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    w[p] = pack_bf16(x, y);
    x -= bf16lo(w[p]);
    y -= bf16hi(w[p]);
  }
}
template <int PARTS>
__device__ __forceinline__ void split_pair_f16(float x, float y, uint32_t* w) {
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    const f32x2 v = {x, y};
    const f16x2 h = __builtin_convertvector(v, f16x2);
    w[p] = __builtin_bit_cast(uint32_t, h);
    x -= (float)h[0];
    y -= (float)h[1];
  }
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// A lane's part of a tile: loads through a buffer descriptor of the tile, whose base is scalar and whose offsets are four numbers a lane keeps.
typedef __amdgpu_buffer_rsrc_t tile_buffer;
template <int D>
struct TileRegs {
  uint32_t k[2][D / 32];  // [half][word], 8 elements a word: D/4 of them from D/4 g on (D = 128: the block of 32 elements g)
  uint32_t v[D / 16];     // D = 128: a word per row j; D = 64: rows 2j, 2j + 1 share one
  uint32_t ks;            // scale bytes of the halves
  u32x2 vs;               // of rows j
  int at_k, at_ks, at_v, at_vs;
  __device__ __forceinline__ void place(int r, int g) {
    using L = Tile<D>;
    at_k = r * (D / 2) + (D / 8) * g;
    at_ks = L::kKs + ((g * (D / 32) / 4) * 16 + r) * 2;
    at_v = L::kV + (g * 16 + r) * 8 * L::RB;
    at_vs = L::kVs + ((r / L::LPB) * 4 + g) * 8;
  }
  __device__ __forceinline__ void load_k(tile_buffer t) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (D == 128) {
        const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(t, at_k, 16 * h * (D / 2), 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) k[h][i] = x[i];
      } else {
        const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(t, at_k, 16 * h * (D / 2), 0);
        k[h][0] = x[0]; k[h][1] = x[1];
      }
    }
    ks = __builtin_amdgcn_raw_buffer_load_b16(t, at_ks, 0, 0);
  }
  __device__ __forceinline__ void load_v(tile_buffer t) {
#pragma unroll
    for (int w = 0; w < D / 64; ++w) {
      const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(t, at_v, 16 * w, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * w + i] = x[i];
    }
    vs = __builtin_amdgcn_raw_buffer_load_b64(t, at_vs, 0, 0);
  }
};

// the two elements of a byte of the word, as pairs of V (bf16x8: bf16, f16x8: f16)
template <typename V, int SEL>
__device__ __forceinline__ uint32_t two_values(uint32_t codes, float scale) {
  if constexpr (__is_same(V, bf16x8)) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, SEL));
}
template <typename V>
__device__ __forceinline__ uint32_t two_values_of(uint32_t codes, float scale, int sel) {  // sel: known after unrolling
  return sel == 0 ? two_values<V, 0>(codes, scale) : sel == 1 ? two_values<V, 1>(codes, scale) : sel == 2 ? two_values<V, 2>(codes, scale) : two_values<V, 3>(codes, scale);
}
__device__ __forceinline__ bf16x8 eight_values(uint32_t codes, float scale) {
  const u32x4 w = {two_values<bf16x8, 0>(codes, scale), two_values<bf16x8, 1>(codes, scale), two_values<bf16x8, 2>(codes, scale), two_values<bf16x8, 3>(codes, scale)};
  return __builtin_bit_cast(bf16x8, w);
}

// The probabilities of 8 rows as the operand's PARTS
template <typename V, int PARTS>
__device__ __forceinline__ void pack_weights(const float* p, V (&pf)[PARTS]) {
  u32x4 w[PARTS];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t parts[PARTS];
    if constexpr (__is_same(V, bf16x8)) split_pair_bf16<PARTS>(p[2 * i], p[2 * i + 1], parts);
    else split_pair_f16<PARTS>(p[2 * i], p[2 * i + 1], parts);
#pragma unroll
    for (int k = 0; k < PARTS; ++k) w[k][i] = parts[k];
  }
#pragma unroll
  for (int k = 0; k < PARTS; ++k) pf[k] = __builtin_bit_cast(V, w[k]);
}

// O^T += V^T P^T over the 8 rows of each lane group, for every block of query rows.  V is the operand type: f16 with P in PARTS of 11
// bits, or bf16 with parts of 8 where a scale of the tile is out of f16's reach.  p: the probabilities, rows 4 half + i.
template <typename V, int D, int NT, int PARTS>
__device__ __forceinline__ void add_pv(const uint32_t* v, const float* vscale, const float (*p)[8], f32x4 (*o)[D / 16]) {
  V pf[NT][PARTS];
#pragma unroll
  for (int n = 0; n < NT; ++n) pack_weights<V, PARTS>(p[n], pf[n]);
#pragma unroll
  for (int q = 0; q < D / 32; ++q) {
    uint32_t pr[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) pr[j] = D == 128 ? two_values_of<V>(v[j], vscale[j], q) : two_values_of<V>(v[j / 2], vscale[j], 2 * (j & 1) + q);
    u32x4 lo, hi;  // blocks 2q and 2q + 1, rows in pairs
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      lo[j] = __builtin_amdgcn_perm(pr[2 * j + 1], pr[2 * j], 0x05040100u);
      hi[j] = __builtin_amdgcn_perm(pr[2 * j + 1], pr[2 * j], 0x07060302u);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int k = PARTS - 1; k >= 0; --k) {
        o[n][2 * q] = mfma16(__builtin_bit_cast(V, lo), pf[n][k], o[n][2 * q]);
        o[n][2 * q + 1] = mfma16(__builtin_bit_cast(V, hi), pf[n][k], o[n][2 * q + 1]);
      }
  }
}

template <typename T>
__device__ __forceinline__ void load_q8(const T* p, float (&x)[8]);
template <>
__device__ __forceinline__ void load_q8<bf16_t>(const bf16_t* p, float (&x)[8]) {
  const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = bf16lo(v[i]); x[2 * i + 1] = bf16hi(v[i]); }
}
template <>
__device__ __forceinline__ void load_q8<float>(const float* p, float (&x)[8]) {
  const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}

__device__ __forceinline__ void store_y(bf16_t* p, float v) { *reinterpret_cast<uint16_t*>(p) = (uint16_t)(pack_bf16(v, 0.f) & 0xffffu); }
__device__ __forceinline__ void store_y(float* p, float v) { *p = v; }

// Elements x and y of q as numbers of 8 bits.  The first of three is cut off, not rounded, so that one past bf16's largest number does not become an
// infinity: 16 bits remain for the others either way.
template <int PARTS>
__device__ __forceinline__ void split_query(float x, float y, uint32_t* w) {
  if constexpr (PARTS == 1) {
    w[0] = pack_bf16(x, y);
  } else {
    w[0] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
    split_pair_bf16<PARTS - 1>(x - bf16lo(w[0]), y - bf16hi(w[0]), w + 1);
  }
}

// The lane's part of its query rows (past the last: that one again) as operands
template <typename T, int D, int NT, int QP>
__device__ __forceinline__ void load_queries(const T* q, int row0, int rows, int r, int g, bf16x8 (&qf)[NT][D / 32][QP]) {
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int c = min(row0 + 16 * n + r, rows - 1);
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      float x[8];
      load_q8<T>(q + (size_t)c * D + (D / 4) * g + 8 * s, x);
      u32x4 w[QP];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t p[QP];
        split_query<QP>(x[2 * i], x[2 * i + 1], p);
#pragma unroll
        for (int k = 0; k < QP; ++k) w[k][i] = p[k];
      }
#pragma unroll
      for (int k = 0; k < QP; ++k) qf[n][s][k] = __builtin_bit_cast(bf16x8, w[k]);
    }
  }
}

// Lift of the probabilities over rows of V whose largest scale byte is `byte`, of a sequence of len rows: a probability is at most 2^(lift + kRaise), a
// value below 2^(byte - 124), so that all of them together stay below 2^127.
__device__ __forceinline__ float bf16_lift(int byte, int len) {
  const int rows_log2 = 32 - __builtin_clz(((unsigned)max(len, 1) - 1u) | 1u);
  return fminf(kLift, (float)(127 + 124 - (int)kRaise - byte - rows_log2));
}

// Scores of 8 rows -> probabilities relative to the running maximum m (log2 domain, 2^lift above it), their sum added to l.  They are
// formed with the maximum at hand; where one is past 2^(lift + kRaise), the maximum is raised and l and o are brought to the new one.  Then
// products are rounded before the maximum is taken off, as in the maximum itself: the largest is 2^lift whatever the scores' size, where a
// fused product would differ by half a unit of the maximum's last place (from scores of 2^28 on, more than f16 holds).
template <int D>
__device__ __forceinline__ void weigh(float* p, float scale_log2e, float lift, float& m, float& l, f32x4* o) {
  float e[8];
  const float ref = lift - m;
#pragma unroll
  for (int j = 0; j < 8; ++j) e[j] = fmaf(p[j], scale_log2e, ref);
  float top = fmaxf(fmaxf(fmaxf(e[0], e[1]), e[2]), fmaxf(fmaxf(e[3], e[4]), e[5]));
  top = fmaxf(fmaxf(top, e[6]), e[7]);
  if (__any(top > lift + kRaise)) {
#pragma clang fp contract(off)
    float mn = p[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) mn = fmaxf(mn, p[j]);
    mn = fmaxf(mn, __shfl_xor(mn, 16));
    mn = fmaxf(m, fmaxf(mn, __shfl_xor(mn, 32)) * scale_log2e);
    const float corr = exp2f(m - mn);
    l *= corr;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[d] *= corr;
    m = mn;
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = p[j] * scale_log2e - m + lift;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    p[j] = __builtin_amdgcn_exp2f(e[j]);
    l += p[j];
  }
}

// Sum of v over this lane and those before it.
__device__ __forceinline__ int sum_up_to(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);  // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, true);  // row_bcast 15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, true);  // row_bcast 31 into rows 2 and 3
  return v;
}

// How many of the `slots` = B splits pieces lane b's sequence of t tiles gets, so that no piece is much longer than the others: one more than
// t r, rounded down, where r is as large as the slots allow (up to 1/32 of what lies between a rate that always fits and one that cannot),
// none of less than W tiles, and as many as a wave's lists need.
template <int W, int LISTS>
__device__ __forceinline__ int pieces_of(int t, uint32_t tiles, int B, int splits) {
  constexpr int kWhole = 64 * LISTS * W;
  const int slots = B * splits;
  const int least = (t + kWhole - 1) / kWhole, all = (t + W - 1) / W;
  const auto dealt = [&](float r) { return min(max((int)((float)t * r) + 1, least), all); };
  const float total = fmaxf(1.f, (float)tiles);
  float lo = (float)(slots - B) / total, hi = (float)slots / total;
  int best = min(splits, all);
#pragma unroll 1
  for (int i = 0; i < 6; ++i) {
    const float r = i == 0 ? lo : 0.5f * (lo + hi);
    const int n = dealt(r);
    const bool fits = __builtin_amdgcn_readlane(sum_up_to(n), 63) <= slots;
    best = fits ? n : best;
    lo = fits ? r : lo;
    hi = fits || i == 0 ? hi : r;
  }
  return best;
}

// Lists of 64 tiles that a wave keeps the numbers of.
constexpr int lists_of(int nt) { return nt == 1 ? 1 : 2; }
// Wavefronts a SIMD that the registers are kept for: what the compiler reaches without spilling.
constexpr int attn_waves_per_simd(bool bf16, int D, int NT) { return NT == 1 ? (bf16 ? 4 : 3) : D == 64 ? 3 : 2; }

template <typename T, int D, int NT, int W>
__global__ __launch_bounds__(W * 64, attn_waves_per_simd(sizeof(T) == 2, D, NT)) void cache4_attn_kernel(AttnArgs a) {
  using L = Tile<D>;
  constexpr int QP = sizeof(T) == 2 ? 1 : 3;   // bf16 parts of q
  constexpr int PP = sizeof(T) == 2 ? 1 : 2;   // f16 parts of a probability (one bf16 part more)
  constexpr int KS = D / 32;                   // steps of the score product
  constexpr int DB = D / 16;                   // blocks of 16 elements
  constexpr int LD = D + 4;                    // floats between rows of the merge area
  constexpr int kLists = lists_of(NT);
  __shared__ __align__(16) float lds_o[W][16][LD];
  __shared__ float lds_ml[W][16][2];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  int split = (int)(blockIdx.x % (unsigned)a.splits);
  const unsigned rest = blockIdx.x / (unsigned)a.splits;
  const int rb = (int)(rest % (unsigned)a.row_blocks);
  int b = (int)(rest / (unsigned)a.row_blocks / (unsigned)a.c.Hkv);
  const int hk = (int)(rest / (unsigned)a.row_blocks) - b * a.c.Hkv;
  const int row0 = rb * 16 * NT, slot = b * a.splits + split;
  // The numbers of the wave's tiles (64 kLists at most), one a lane: of every tile that the longest sequence could have, so that the page
  // table's entries arrive together with the sequence's length and not behind it.
  const int bound = (a.max_len + kTile - 1) / kTile;
  int first, end, pieces = a.pieces, numbers[kLists];
  const auto take = [&](int chunk) {
    first = split * chunk + wave;
    end = min((split + 1) * chunk, bound);
#pragma unroll
    for (int k = 0; k < kLists; ++k) {
      const int tile = first + W * (64 * k + lane);
      numbers[k] = tile < end ? tile_number(a.c, b, hk, tile) : -1;
    }
  };
  // (dealt: lane b holds the length of sequence b; the last slots may hold no piece)
  const int held = a.dealt ? a.lens[min(lane, a.c.B - 1)] : a.lens[b];
  take(a.chunk);
  int len = min(max(held, 0), a.max_len);
  if (a.dealt) {
    const int rows = lane < a.c.B ? len : 0, t = (rows + kTile - 1) / kTile;
    const uint32_t total = __builtin_amdgcn_readlane(sum_up_to(t), 63);
    int from = lane * a.splits, n = a.pieces;
    if (__builtin_expect(total < a.few, 0)) {
      n = pieces_of<W, kLists>(t, total, a.c.B, a.splits);
      const int upto = sum_up_to(n);
      from = upto - n;
      const unsigned long long behind = __ballot(upto > slot);
      b = behind ? __builtin_ctzll(behind) : 0;
      split = slot - __builtin_amdgcn_readlane(from, b);
      pieces = __builtin_amdgcn_readlane(n, b);
      const int tiles = __builtin_amdgcn_readlane(t, b);
      if (behind) take((tiles + pieces - 1) / pieces);
      else pieces = 0;
    }
    if (__builtin_expect(blockIdx.x == 0 && wave == 0, 0)) {
      a.dealt[lane] = from;
      a.dealt[64 + lane] = n;
    }
    if (split >= pieces) return;
    len = __builtin_amdgcn_readlane(rows, b);
  }
  len = __builtin_amdgcn_readfirstlane(len);
  const int bh = b * a.c.Hkv + hk;
  const auto number_of = [&](int i) {
    int n = __builtin_amdgcn_readlane(numbers[0], i & 63);
#pragma unroll
    for (int k = 1; k < kLists; ++k) n = i >> 6 == k ? __builtin_amdgcn_readlane(numbers[k], i & 63) : n;
    return n;
  };

  // the last position each of the lane's query rows sees (-1 or less: none), and their largest and smallest over the block
  int last[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int c = row0 + 16 * n + r;
    last[n] = c < a.rows ? len - a.T + c % a.T : -1;
  }
  const int c1 = min(row0 + 16 * NT, a.rows) - 1;
  const bool one_head = row0 / a.T == c1 / a.T;
  const int most = len - a.T + (one_head ? c1 % a.T : a.T - 1), least = len - a.T + (one_head ? row0 % a.T : 0);

  const T* qrows = reinterpret_cast<const T*>(a.q) + (size_t)bh * a.rows * D;
  bf16x8 qf[NT][KS][QP];
  load_queries<T, D, NT>(qrows, row0, a.rows, r, g, qf);

  f32x4 o[NT][DB];
  float m[NT], l[NT];
  const int turns = max(0, (min(end, most < 0 ? 0 : most / kTile + 1) - first + W - 1) / W);
  auto place = [&](int i) {  // (a tile that is not there: the first of the pool in its place, not seen)
    const int number = number_of(i);
    return __builtin_amdgcn_make_buffer_rsrc(a.c.pool + (size_t)(number < 0 ? 0 : number) * L::kBytes, 0, L::kBytes, 0x20000);
  };
  float lift = kLift;
  // The wave's tiles, with V as operands of the type of `kind`; false if a tile's scales are out of f16's reach.
  auto walk = [&](auto kind) -> bool {
    using Operand = decltype(kind);
    constexpr bool kHalf = __is_same(Operand, f16x8);
    const float up = kHalf ? kLift : lift;
    uint32_t unfit = 0;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int d = 0; d < DB; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[n] = kNone;
      l[n] = 0.f;
    }
    TileRegs<D> x;
    x.place(r, g);
    if (turns == 0) return true;
    x.load_k(place(0));
    __builtin_amdgcn_sched_barrier(0);  // (in the loop's order: the waits at its top count the loads behind K's)
    x.load_v(place(0));
    __builtin_amdgcn_sched_barrier(0);
    for (int i = 0; i < turns; ++i) {
      const bool there = number_of(i) >= 0;
      const tile_buffer next = place(min(i + 1, turns - 1));  // (the last turn asks for its own again: the loads need no branch)
      const int tile = first + W * i;
      const bool partly = tile * kTile + kTile - 1 > least || !there;  // some query row does not see all of it
      // scores; K's registers are free for the next tile after them, V's after the second product
      float p[NT][8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t byte = (x.ks >> (8 * h)) & 0xffu;
        const float scale = __uint_as_float(byte == kNoRow ? 0x7fc00000u : byte << 23);
        bf16x8 kf[KS];
#pragma unroll
        for (int st = 0; st < KS; ++st) kf[st] = eight_values(x.k[h][st], scale);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = QP - 1; k >= 0; --k)
#pragma unroll
            for (int st = 0; st < KS; ++st) acc = mfma16(kf[st], qf[n][st][k], acc);
#pragma unroll
          for (int e = 0; e < 4; ++e) p[n][4 * h + e] = acc[e];
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      x.load_k(next);
      if (partly) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (tile * kTile + L::row(g, j) > last[n] || !there) p[n][j] = -INFINITY;
#pragma unroll
        for (int j = 0; j < 8; ++j)  // never written, or another tile's: whatever lies there is kept finite
          if (tile * kTile + L::row(g, j) >= len || !there) x.vs[j / 4] = (x.vs[j / 4] & ~(0xffu << (8 * (j & 3)))) | kOne << (8 * (j & 3));
      }
      if constexpr (kHalf) {
        // bytes 108..139, 2^-19 .. 2^12: every value of the block is an f16 number (a byte that overflows its sum fails by itself)
        const uint32_t off = ((x.vs[0] + 0x14141414u) ^ 0x80808080u) | ((x.vs[1] + 0x14141414u) ^ 0x80808080u);
        unfit |= off & 0xe0e0e0e0u;
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) weigh<D>(p[n], a.scale_log2e, up, m[n], l[n], o[n]);
      __builtin_amdgcn_sched_barrier(0);
      float vscale[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) vscale[j] = __uint_as_float(((x.vs[j / 4] >> (8 * (j & 3))) & 0xffu) << 23);
      add_pv<Operand, D, NT, kHalf ? PP : PP + 1>(x.v, vscale, p, o);
      __builtin_amdgcn_sched_barrier(0);
      x.load_v(next);
      __builtin_amdgcn_sched_barrier(0);
    }
    return !__any(unfit != 0);
  };
  if (!walk(f16x8{})) {
    // the largest scale of V in the tiles: a lane's eight are those of rows 4 g .. of both halves
    int byte = 0;
    const int at = L::kVs + ((r / L::LPB) * 4 + g) * 8;
#pragma unroll 1
    for (int i = 0; i < turns; ++i) {
      const int rows = number_of(i) < 0 ? 0 : len - (first + W * i) * kTile - 4 * g;  // rows that are there from 4 g on
      const u32x2 vs = __builtin_amdgcn_raw_buffer_load_b64(place(i), at, 0, 0);
#pragma unroll
      for (int j = 0; j < 8; ++j) byte = L::row(0, j) < rows ? max(byte, (int)((vs[j / 4] >> (8 * (j & 3))) & 0xffu)) : byte;
    }
    int most_byte = 0;  // the wave's, bit by bit (exchanged between lanes it costs registers that the walk needs)
#pragma unroll
    for (int bit = 128; bit > 0; bit >>= 1) most_byte |= __any(byte >= (most_byte | bit)) ? bit : 0;
    lift = bf16_lift(most_byte, len);
    walk(bf16x8{});
  }
  int sight = 0x7fffffff;  // the first position of the first of the wave's tiles that is there
#pragma unroll
  for (int k = kLists - 1; k >= 0; --k) {
    const unsigned long long there = __ballot(numbers[k] >= 0);
    sight = there ? (first + W * (64 * k + (int)__builtin_ctzll(there))) * kTile : sight;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) m[n] = last[n] < sight ? -INFINITY : m[n] - lift;  // what the sums are relative to

  // the waves' results, 16 query rows at a time
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float ls = l[n];
    ls += __shfl_xor(ls, 16);
    ls += __shfl_xor(ls, 32);
    if (n > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = 0; d < DB; d += 4)
        *reinterpret_cast<f32x4*>(&lds_o[wave][r][DB * (4 * g + i) + d]) = f32x4{o[n][d][i], o[n][d + 1][i], o[n][d + 2][i], o[n][d + 3][i]};
    if (g == 0) {
      lds_ml[wave][r][0] = m[n];
      lds_ml[wave][r][1] = ls;
    }
    __syncthreads();
    const int valid = min(16, a.rows - row0 - 16 * n);
    for (int idx = threadIdx.x; idx < valid * D; idx += W * 64) {
      const int c = idx / D, e = idx % D;
      const int row = row0 + 16 * n + c;
      float M = lds_ml[0][c][0];
#pragma unroll
      for (int w = 1; w < W; ++w) M = fmaxf(M, lds_ml[w][c][0]);
      float v = 0.f, sum = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = exp2_above(lds_ml[w][c][0], M);
        v = fmaf(f, lds_o[w][c][e], v);
        sum = fmaf(f, lds_ml[w][c][1], sum);
      }
      const size_t out = (size_t)bh * a.rows + row;
      if (pieces == 1) {
        store_y(reinterpret_cast<T*>(a.Y) + out * D + e, weighted_mean(M, v, sum));
        if (e == 0 && a.LSE) a.LSE[out] = log_of_sum(M, sum);
      } else {
        float* to = a.part + (((size_t)hk * a.rows + row) * (a.c.B * a.splits) + slot) * (D + 2);
        to[e] = v;
        if (e == 0) {
          to[D] = M;
          to[D + 1] = sum;
        }
      }
    }
  }
}

// Joins the splits' results of a query row, W waves a row (one of them: four rows a workgroup, nothing exchanged): a wave
// runs over its own splits with a running maximum, several of them in flight.
template <typename T, int D, int W>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void cache4_merge_kernel(MergeArgs a) {
  constexpr int EPL = D / 64, UM = 8;
  __shared__ float lds_m[W], lds_l[W], lds_o[W][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = blockIdx.y, r = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  if (r >= a.rows) return;  // (W = 1)
  const size_t row = (size_t)b * a.rows + r;
  T* Y = reinterpret_cast<T*>(a.Y);
  float* LSE = a.LSE;
  const int start = W == 1 ? 0 : wave;
  const float* own = a.part + (size_t)r * a.all * (D + 2);
  int slot = b * a.splits, splits = a.pieces;
  float mx[UM], lx[UM], x[UM][EPL];
  const auto load = [&](int s0) {
#pragma unroll
    for (int u = 0; u < UM; ++u) {
      const float* at = own + (size_t)(slot + min(s0 + u * W, splits - 1)) * (D + 2);
      mx[u] = at[D];
      lx[u] = at[D + 1];
#pragma unroll
      for (int i = 0; i < EPL; ++i) x[u][i] = at[lane + 64 * i];
    }
  };
  load(start);
  if (a.dealt) {  // (asked for beside the pieces that it usually says)
    const int from = a.dealt[b], n = a.dealt[64 + b];
    if (n == 1) return;  // written by the one piece
    if (__builtin_expect(from != slot || n != splits, 0)) {
      slot = from;
      splits = n;
      if (n > 0) load(start);
    }
  }
  float m = -INFINITY, l = 0.f, o[EPL] = {};
  for (int s0 = start; s0 < splits; s0 += W * UM) {
    if (s0 > start) load(s0);
    float mn = m;
#pragma unroll
    for (int u = 0; u < UM; ++u) {
      if (s0 + u * W >= splits) {
        mx[u] = -INFINITY;
        lx[u] = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) x[u][i] = 0.f;
      }
      mn = fmaxf(mn, mx[u]);
    }
    const float corr = exp2_above(m, mn);
    l *= corr;
#pragma unroll
    for (int i = 0; i < EPL; ++i) o[i] *= corr;
#pragma unroll
    for (int u = 0; u < UM; ++u) {
      const float f = exp2_above(mx[u], mn);
      l = fmaf(f, lx[u], l);
#pragma unroll
      for (int i = 0; i < EPL; ++i) o[i] = fmaf(f, x[u][i], o[i]);
    }
    m = mn;
  }
  if constexpr (W == 1) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) store_y(Y + (size_t)row * D + lane + 64 * i, weighted_mean(m, o[i], l));
    if (lane == 0 && LSE) LSE[row] = log_of_sum(m, l);
    return;
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) lds_o[wave][lane + 64 * i] = o[i];
  if (lane == 0) {
    lds_m[wave] = m;
    lds_l[wave] = l;
  }
  __syncthreads();
  if (threadIdx.x < D) {
    const int e = threadIdx.x;
    float M = lds_m[0], sum = 0.f, v = 0.f;
#pragma unroll
    for (int w = 1; w < W; ++w) M = fmaxf(M, lds_m[w]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = exp2_above(lds_m[w], M);
      sum = fmaf(f, lds_l[w], sum);
      v = fmaf(f, lds_o[w][e], v);
    }
    store_y(Y + (size_t)row * D + e, weighted_mean(M, v, sum));
    if (e == 0 && LSE) LSE[row] = log_of_sum(M, sum);
  }
}

// a launch of n workgroups: the threads of one dimension are counted in 32 bits
bool fits_a_launch(long n, int threads) { return n <= 0xffffffffL / threads; }

int log2_of(int v) { int k = 0; while ((1 << k) < v) ++k; return k; }

Cache cache_of(const sa_cache4_desc* c, void* pool, const int32_t* table) {
  Cache k;
  k.pool = reinterpret_cast<unsigned char*>(pool);
  k.table = table;
  k.B = c->B; k.Hkv = c->Hkv; k.pages = c->pages; k.max_pages = c->max_pages;
  k.tiles_log2 = log2_of(c->page_rows / kTile);
  k.capacity = c->max_pages * c->page_rows;
  return k;
}

// How a call is dealt: the query rows of a KV head in `blocks` of 16 nt, the cache in `splits` pieces; `most`: what `slots` can be
// for this many tiles or fewer (the workspace is sized for that).
struct Plan {
  int nt;
  bool dealt;  // the sequences' pieces are dealt by their lengths if those differ much
  long blocks, splits, slots, most;
};
constexpr int waves_of(int nt) { return nt == 1 ? 8 : 4; }
constexpr int kDealtTo = 64;  // sequences, one a lane
Plan pieces_plan(const sa_cache4_desc* c, int T, long tiles) {
  const long rows = (long)(c->Hq / c->Hkv) * T;
  Plan p;
  p.nt = rows <= 16 ? 1 : 2;
  p.blocks = (rows + 16 * p.nt - 1) / (16 * p.nt);
  const long groups = (long)c->B * c->Hkv * p.blocks;
  const long waves = waves_of(p.nt), whole = 64 * lists_of(p.nt) * waves;
  const long least = (tiles + whole - 1) / whole, all = (tiles + waves - 1) / waves;  // as many tiles a wave as it can list, and one
  const auto between = [&](long want) { return want > all ? (all < least ? least : all) : want < least ? least : want; };
  if (p.nt == 1) {
    // Bound by memory: two waves a SIMD.  Fewer leave loads too few in flight, more pay more prologues and partial results (us, workgroups of 4
    // waves / 8 / 8 with twice the pieces: 131072 rows of 4 KV heads 18.9 / 17.9 / 19.7, 20000 rows of 16 heads, B2 14.0 / 13.1 / 14.2).
    // Up to three tiles a wave the second launch costs more than pieces gain (300 rows, 8 KV heads: 6.1 us in one piece, 8.4 in two).
    p.splits = p.most = all <= 3 ? between(1) : between((2048 + groups * waves - 1) / (groups * waves));
    return p;
  }
  // Bound by the vector ALU.  The launch is as many workgroups at a time as fit the chip, each a piece's tiles long and what a prologue and an
  // end take, about six; with k waves a SIMD all of that takes 1 + 0.6 (k - 1) times as long as with one; joining pieces takes about
  // eight.  The least of that for pieces that fill one, two, .. waves a SIMD, and two and three such rounds (us, pieces of one wave / two / four: T5,
  // B4 x 8192 rows, 32 / 8 heads 15.8 / 17.7 / 25.0; T128 over 32768 rows 98.8 / 85.8 / 92.0; T509 over 32768 rows in two rounds 298, in three or four 305).
  const int per_simd = attn_waves_per_simd(c->dtype == SA_BF16, c->d, p.nt);
  const long fit = 256 * per_simd;  // (a workgroup is a wave on each SIMD)
  p.splits = least;
  p.most = between(3 * fit / groups + 1);
  long best = 0;
  for (int k = 0; k <= per_simd + 2; ++k) {
    const long room = (k <= per_simd ? 256 * k : fit * (k - per_simd + 1)) / groups;
    const long s = room < least ? least : room > p.most ? p.most : room;
    const long rounds = (groups * s + fit - 1) / fit, each = (tiles + s * waves - 1) / (s * waves) + 6;
    const long shared = ((groups * s < fit ? groups * s : fit) + 255) / 256;
    const long cost = rounds * each * (4 + 6 * shared) + (s > 1 ? 80 : 0);  // in tenths
    if (best == 0 || cost < best) { best = cost; p.splits = s; }
  }
  return p;
}

// Pieces of the longest sequence are `splits` equal ones; a sequence has `slots` workgroups.  Where a wave has 12 tiles or more and up to 64
// sequences hold less than two thirds of the rows that as many longest ones would, the kernel deals the slots of all of them by their lengths (us,
// bf16, 32 / 8 heads: 12 sequences of 1000 rows but one of 16384 24.4 -> 13.3; 500 to 7700 rows, B16 20.7 -> 19.4; even ones pay for the question, 16 of
// 8192 rows 31.0 -> 31.3; of 3700 to 8192 rows, 73 %, 25.0 -> 25.8; with 5 tiles a wave, 20000 and 300 rows 12.1 -> 14.0).  A sequence that would be one
// piece has a slot more for that from 16 tiles a wave on (31 of 600 rows and one of 12000 43.0 -> 15.6; 32 of 1000 to 4000 rows 20.2 as before).
// More than one block of query rows makes workgroups enough that the short ones' places are taken by others (the first batch, 6 tokens 28.8 -> 21.3,
// 16 tokens in two blocks 37.4 -> 38.3).
Plan plan_of(const sa_cache4_desc* c, int T, long tiles) {
  Plan p = pieces_plan(c, T, tiles);
  const long waves = waves_of(p.nt), each = (tiles + p.splits - 1) / p.splits;
  const bool several = c->B > 1 && c->B <= kDealtTo && p.blocks == 1;
  p.slots = several && p.splits == 1 && p.nt == 1 && each >= 16 * waves ? 2 : p.splits;
  p.dealt = several && p.slots > 1 && each >= 12 * waves;
  if (p.most < p.slots) p.most = p.slots;
  return p;
}

template <typename T, int D>
hipError_t launch_attn(const sa_cache4_desc* c, AttnArgs& a, const Plan& p, hipStream_t st) {
  const long blocks = (long)c->B * c->Hkv * a.row_blocks * a.splits;
  const int rows = c->Hkv * a.rows;  // of a sequence
  if (!fits_a_launch(blocks, 512) || (a.splits > 1 && !fits_a_launch(rows, a.splits <= 16 ? 64 : 512))) return hipErrorNotSupported;
  const unsigned grid = (unsigned)blocks;
  if (p.nt == 1) cache4_attn_kernel<T, D, 1, waves_of(1)><<<grid, 64 * waves_of(1), 0, st>>>(a);
  else cache4_attn_kernel<T, D, 2, waves_of(2)><<<grid, 64 * waves_of(2), 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const MergeArgs m = {a.part, a.dealt, a.Y, a.LSE, rows, a.splits, a.pieces, c->B * a.splits};
  if (a.splits <= 16) cache4_merge_kernel<T, D, 1><<<dim3((rows + 3) / 4, c->B), 256, 0, st>>>(m);
  else cache4_merge_kernel<T, D, 8><<<dim3(rows, c->B), 512, 0, st>>>(m);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache4_rows(const sa_cache4_desc* c, bool write, void* K, void* V, int T, const int32_t* starts,
                              const int32_t* counts, const int32_t* table, void* pool, hipStream_t st) {
  RowsArgs a;
  a.c = cache_of(c, pool, table);
  a.starts = starts; a.counts = counts; a.K = K; a.V = V; a.T = T;
  a.tiles = tiles_touched(T);
  const long blocks = (long)c->B * c->Hkv * ((2 * (long)a.tiles + kRowWaves - 1) / kRowWaves);
  if (!fits_a_launch(blocks, kRowWaves * 64)) return hipErrorNotSupported;
  const unsigned grid = (unsigned)blocks;
  const dim3 block(kRowWaves * 64);
  const bool bf16 = c->dtype == SA_BF16;
  if (write) {
    if (bf16 && c->d == 128) cache4_write_kernel<bf16_t, 128><<<grid, block, 0, st>>>(a);
    else if (bf16) cache4_write_kernel<bf16_t, 64><<<grid, block, 0, st>>>(a);
    else if (c->d == 128) cache4_write_kernel<float, 128><<<grid, block, 0, st>>>(a);
    else cache4_write_kernel<float, 64><<<grid, block, 0, st>>>(a);
  } else {
    if (bf16 && c->d == 128) cache4_read_kernel<bf16_t, 128><<<grid, block, 0, st>>>(a);
    else if (bf16) cache4_read_kernel<bf16_t, 64><<<grid, block, 0, st>>>(a);
    else if (c->d == 128) cache4_read_kernel<float, 128><<<grid, block, 0, st>>>(a);
    else cache4_read_kernel<float, 64><<<grid, block, 0, st>>>(a);
  }
  return hipGetLastError();
}

int cache4_loaded_rows(int start, int count, int T, int half, int32_t* rows) {
  if (half < 0 || half >= 2 * tiles_touched(T)) return -1;
  count = count < 0 ? 0 : count > T ? T : count;
  const HalfRows h = half_rows(start, count, tiles_touched(T), half);
  for (int j = 0; j < 16 && h.any; ++j) rows[j] = (int32_t)loaded_row(h.t0 + j, count);
  return h.any ? 1 : 0;
}

constexpr size_t kDealtBytes = 2 * kDealtTo * sizeof(int32_t);

size_t cache4_decode_workspace_bytes(const sa_cache4_desc* c, int T) {
  const long tiles = ((long)c->max_pages * c->page_rows) / kTile;
  const long splits = plan_of(c, T, tiles).most;
  return splits <= 1 ? 0 : kDealtBytes + (size_t)c->B * c->Hq * T * (size_t)splits * (c->d + 2) * sizeof(float);
}

int cache4_decode_dealt(const sa_cache4_desc* c, int T, int max_len) {
  const Plan p = plan_of(c, T, ((long)max_len + kTile - 1) / kTile);
  return p.dealt ? (int)p.slots : 0;
}

int cache4_decode_plan(const sa_cache4_desc* c, int T, int max_len) {
  const Plan p = plan_of(c, T, ((long)max_len + kTile - 1) / kTile);
  return p.nt | (int)p.splits << 2;
}

hipError_t launch_cache4_decode(const sa_cache4_desc* c, const void* q, int T, const void* pool, const int32_t* table,
                                const int32_t* lens, int max_len, void* Y, float* LSE, void* ws, hipStream_t st) {
  AttnArgs a;
  a.c = cache_of(c, const_cast<void*>(pool), table);
  a.q = q; a.Y = Y; a.LSE = LSE; a.lens = lens;
  a.T = T; a.rows = (c->Hq / c->Hkv) * T; a.max_len = max_len;
  const long tiles = ((long)max_len + kTile - 1) / kTile;
  const Plan p = plan_of(c, T, tiles);
  a.row_blocks = (int)p.blocks;
  a.chunk = (int)((tiles + p.splits - 1) / p.splits);
  a.pieces = (int)((tiles + a.chunk - 1) / a.chunk);
  a.splits = p.slots > p.splits ? (int)p.slots : a.pieces;
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + kDealtBytes);
  a.few = (uint32_t)(c->B * tiles * 2 / 3);
  a.dealt = p.dealt && a.splits > 1 ? static_cast<int32_t*>(ws) : nullptr;
  a.scale_log2e = (c->scale > 0.f ? c->scale : 1.0f / sqrtf((float)c->d)) * kLog2e;
  if (c->dtype == SA_BF16) return c->d == 128 ? launch_attn<bf16_t, 128>(c, a, p, st) : launch_attn<bf16_t, 64>(c, a, p, st);
  return c->d == 128 ? launch_attn<float, 128>(c, a, p, st) : launch_attn<float, 64>(c, a, p, st);
}

}  // namespace sa
