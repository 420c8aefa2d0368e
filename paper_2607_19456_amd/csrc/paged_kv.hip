// paged_kv.hip -- gfx950 kernels and C ABI of the paged KV cache: rows appended
// with the position rotation on the way, read back, and attended to, the cache
// in 32 or 16 bits or in 4 (blocks of 32 values that share a power of two).
//
// Kernels
//   paged_append_kernel   q, K and V rows of a step: q and K turned by the
//                         position's angles, K and V written to their pages.
//   paged_gather_kernel   the same places read back as dense rows.
//   paged_attn_kernel     softmax(scale q.K) V over the pages of each (sequence,
//                         KV head, tile of query rows), split evenly over a
//                         grid of two workgroups a CU, as partial states.
//   paged_chunk_kernel    the same for many query rows per KV head, K and V
//                         shared by four waves through LDS.
//   paged_merge_kernel    combines the parts of each query row.
//
// Register layouts of the matrix instructions used below (lane = 0..63,
// i = lane % 16, k = lane / 16), 16 x 16 results:
//   A operand: lane holds A[i][..], k's share of the summed index
//   B operand: lane holds B[..][i], k's share of the summed index
//   result:    lane holds D[4k + r][i] in component r = 0..3
// The summed index is shared out 8 to a lane (16-bit types, 32 in all) or 1
// (float32, 4 in all); any assignment of it to (k, element) serves as long as
// both operands use the same.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "decode_attn.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxCus = 256;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <class T>
constexpr bool is_f32 = std::is_same<T, float>::value;

// ---------------------------------------------------------------------------
// The batch, as the kernels see it.
// ---------------------------------------------------------------------------
struct Batch {
  char* K;
  char* V;
  const int32_t* pages;
  const int32_t* past;
  const int32_t* row_start;
  int B, h_kv, n_pages, page_log2, max_pages, rows, T;
};

// A word of an array that no kernel here writes, at an address that is the same
// for the whole wave: through the scalar cache, so that waiting for it does not
// wait for the vector loads under way.
__device__ __forceinline__ int fixed(const int32_t* p) {
  typedef const int32_t __attribute__((address_space(4))) * constant_ptr;
  return *(constant_ptr)p;
}

// A load of what is read once: it leaves the caches to others.
template <class V>
__device__ __forceinline__ V once(const void* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
}

__device__ __forceinline__ int capacity(const Batch& bt) { return bt.max_pages << bt.page_log2; }

// First row and number of rows of sequence b, within the arrays whatever
// row_start holds.
struct SeqRows {
  int start, n;
};
__device__ __forceinline__ SeqRows seq_rows(const Batch& bt, int b) {
  if (!bt.row_start) return {b * bt.T, bt.T};
  const int s = min(max(bt.row_start[b], 0), bt.rows);
  const int e = min(max(bt.row_start[b + 1], s), bt.rows);
  return {s, min(e - s, bt.T)};
}

// The same where b is the same for the whole wave.
__device__ __forceinline__ SeqRows one_seq_rows(const Batch& bt, int b) {
  if (!bt.row_start) return {b * bt.T, bt.T};
  const int s = min(max(fixed(bt.row_start + b), 0), bt.rows);
  const int e = min(max(fixed(bt.row_start + b + 1), s), bt.rows);
  return {s, min(e - s, bt.T)};
}

// Bytes of the codes (or values) of one row, and of one head's page.
template <class T, bool MX, int D>
constexpr int kRowBytes = MX ? D / 2 : D * (int)sizeof(T);
template <class T, bool MX, int D>
__device__ __forceinline__ int64_t block_bytes(int page_log2) {
  return (int64_t)(kRowBytes<T, MX, D> + (MX ? D / 32 : 0)) << page_log2;
}

// ---------------------------------------------------------------------------
// Append: one thread turns and writes 16 dimensions of one head of one row (8
// of a 4-bit row, whose blocks of 32 are then four lanes' work).  Memory-bound: 6
// operations for each pair of values that it reads and writes.  Measured: prompts
// of 103 MB in 19.0 us (5.4 TB/s; a copy too large for the caches reaches 4.8);
// with 8 dimensions a thread, whose halves of a pair each read the angles, a call
// took 28.5 us for 22.6.  64 rows of a decode step: 3.0 us, a launch and a few loads
// that wait for each other.
// ---------------------------------------------------------------------------
template <class T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (is_f32<T>) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p);
    const f32x4 b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
  } else {
    typedef T t8 __attribute__((ext_vector_type(8)));
    const t8 a = *reinterpret_cast<const t8*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)a[e];
  }
}

template <class T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (is_f32<T>) {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    typedef T t8 __attribute__((ext_vector_type(8)));
    t8 a;
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = (T)x[e];
    *reinterpret_cast<t8*>(p) = a;
  }
}

struct AppendArgs {
  const void *q, *k, *v;
  void* q_out;
  int64_t q_stride, k_stride, v_stride;
  const float* rotary;
  int h_q, rot_dim, interleaved;
};

// Dimensions 8*piece .. +7 of a row after the rotation, in 64 bits.
template <class T>
__device__ __forceinline__ void turned8(const T* row, int piece, const AppendArgs& a,
                                        const float* angles, double (&y)[8]) {
  typedef double W;
  float x[8];
  load8(row + 8 * piece, x);
  const int half = a.rot_dim / 2;
  if (8 * piece >= a.rot_dim) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (W)x[e];
    return;
  }
  if (a.interleaved) {
    const f32x4 c = *reinterpret_cast<const f32x4*>(angles + 4 * piece);
    const f32x4 s = *reinterpret_cast<const f32x4*>(angles + half + 4 * piece);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const W x1 = x[2 * e], x2 = x[2 * e + 1], cc = c[e], ss = s[e];
      y[2 * e] = x1 * cc - x2 * ss;
      y[2 * e + 1] = x2 * cc + x1 * ss;
    }
    return;
  }
  const bool upper = 8 * piece >= half;
  const int at = 8 * piece - (upper ? half : 0);
  float o[8], c[8], s[8];
  load8(row + at + (upper ? 0 : half), o);
  load8(angles + at, c);
  load8(angles + half + at, s);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const W cc = c[e], ss = upper ? s[e] : -s[e];
    y[e] = (W)x[e] * cc + (W)o[e] * ss;
  }
}

// The float32 value of y rounded to odd: toward zero, with the last bit set
// where that was inexact, so that a rounding to fewer bits is that of y itself.
__device__ __forceinline__ float to_odd(double y) {
  const float f = (float)y;
  const double back = f;
  uint32_t u = __float_as_uint(f);
  if (back != y && y == y) {
    if (fabs(back) > fabs(y)) --u;
    u |= 1u;
  }
  return __uint_as_float(u);
}
__device__ __forceinline__ float to_odd(float y) { return y; }

// 2^(byte - 127), bytes 1 to 254.
__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes and scale byte of 8 values whose block of 32 lies in four lanes in
// turn.  The block's largest exponent is found on the bits.
template <class W>
__device__ __forceinline__ uint32_t quantise8(const W (&y)[8], uint32_t* scale_byte) {
  float f[8];
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    f[e] = to_odd(y[e]);
    top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
  }
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  if (top >= 0x7f800000u) {            // an infinity or a NaN in the block
    *scale_byte = 255;
    return 0x77777777u;
  }
  const int byte = max((int)(top >> 23) - 2, 1);
  *scale_byte = (uint32_t)byte;
  // the conversion divides by the scale, rounds to the nearest level, ties to
  // the even code, and stops at the largest
  const float scale = power_of((uint32_t)byte);
  uint32_t codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[0], f[1], scale, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2], f[3], scale, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4], f[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6], f[7], scale, 3);
}

// Offsets of a 4-bit row's codes and scale bytes in its page.
template <int D>
__device__ __forceinline__ int64_t mx_code_at(bool value, int slot, int piece) {
  return value ? (int64_t)(slot >> 3) * (4 * D) + piece * 32 + (slot & 7) * 4
               : (int64_t)slot * (D / 2) + piece * 4;
}
template <int D>
__device__ __forceinline__ int64_t mx_scale_at(bool value, int page_log2, int slot, int block) {
  return ((int64_t)(D / 2) << page_log2) +
         (value ? (int64_t)(slot >> 3) * (D / 4) + block * 8 + (slot & 7)
                : (int64_t)slot * (D / 32) + block);
}

// What a 4-bit code and a scale byte stand for.
__device__ __forceinline__ float mx_level(uint32_t code) {
  const uint32_t ex = code >> 1 & 3u;
  const float m = ex ? (float)(2 + (code & 1u)) * (float)(1u << ex) * 0.25f
                     : (float)(code & 1u) * 0.5f;
  return code & 8u ? -m : m;
}
__device__ __forceinline__ float mx_factor(uint32_t byte) {
  // the byte 255 as a scale is not a number, and so is what it scales; 0 is
  // 2^-127, which is not a normal number
  return __uint_as_float(byte == 255 ? 0x7fc00000u : byte == 0 ? 0x00400000u : byte << 23);
}

// A dimension of a slot of a head's page, as a value of T.
template <class T, bool MX, int D>
__device__ __forceinline__ float held(const char* block, bool value, int page_log2, int slot,
                                      int dim) {
  if constexpr (MX) {
    const uint32_t codes =
        *reinterpret_cast<const uint32_t*>(block + mx_code_at<D>(value, slot, dim / 8));
    const uint32_t byte = (uint8_t)block[mx_scale_at<D>(value, page_log2, slot, dim / 32)];
    return (float)(T)(mx_level(codes >> (4 * (dim % 8)) & 15u) * mx_factor(byte));
  } else {
    return (float)reinterpret_cast<const T*>(block)[(int64_t)slot * D + dim];
  }
}

// Unit u (of D/16) of a row into dst, where dst may be src: 16 dimensions, and
// of a rotated part both of each pair, so that the angles are read once for two
// values and nobody else reads what is written.
template <class T>
__device__ __forceinline__ void turn16(const T* src, T* dst, int u, const AppendArgs& a,
                                       const float* angles, bool rotate) {
  const int half = a.rot_dim / 2;
  const bool turn = rotate && 16 * u < a.rot_dim;
  const bool pairs = turn && !a.interleaved;          // dimensions 8u.. and half + 8u..
  const int at1 = pairs ? 8 * u : 16 * u, at2 = pairs ? half + 8 * u : 16 * u + 8;
  float x[8], y[8];
  load8(src + at1, x);
  load8(src + at2, y);
  if (turn) {
    float c[8], s[8];
    load8(angles + 8 * u, c);
    load8(angles + half + 8 * u, s);
    if (pairs) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x1 = x[e], x2 = y[e];
        x[e] = x1 * c[e] - x2 * s[e];
        y[e] = x2 * c[e] + x1 * s[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float(&z)[8] = e < 4 ? x : y;
        const float x1 = z[2 * e % 8], x2 = z[2 * e % 8 + 1];
        z[2 * e % 8] = x1 * c[e] - x2 * s[e];
        z[2 * e % 8 + 1] = x2 * c[e] + x1 * s[e];
      }
    }
  }
  store8(dst + at1, x);
  store8(dst + at2, y);
}

template <class T, bool MX, int D>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(Batch bt, AppendArgs a,
                                                                unsigned seq_groups) {
  constexpr int kPairs = D / 16;                      // units of a row of q, and of dense ones
  constexpr int kPieces = MX ? D / 8 : kPairs;        // units of a row of K or V
  const int b = blockIdx.x / seq_groups;
  const SeqRows sr = seq_rows(bt, b);
  const int of_q = a.h_q * kPairs, per_row = of_q + 2 * bt.h_kv * kPieces;
  const uint32_t unit = blockIdx.x % seq_groups * kThreads + threadIdx.x;
  const int r = (int)(unit / (uint32_t)per_row);
  if (r >= sr.n) return;
  const int past = bt.past[b];
  if (past < 0 || past >= capacity(bt) - r) return;
  const int pos = past + r;
  int u = (int)(unit - (uint32_t)r * (uint32_t)per_row);
  const int64_t row = sr.start + r;
  const float* angles = a.rotary + (int64_t)pos * a.rot_dim;
  if (u < of_q) {
    const int head = u / kPairs;
    turn16(static_cast<const T*>(a.q) + row * a.q_stride + (int64_t)head * D,
           static_cast<T*>(a.q_out) + (row * a.h_q + head) * D, u % kPairs, a, angles, true);
    return;
  }
  u -= of_q;
  const int piece = u % kPieces;
  int head = u / kPieces;
  const bool value = head >= bt.h_kv;
  if (value) head -= bt.h_kv;
  const int page = bt.pages[(int64_t)b * bt.max_pages + (pos >> bt.page_log2)];
  if ((unsigned)page >= (unsigned)bt.n_pages) return;
  const int slot = pos & ((1 << bt.page_log2) - 1);
  char* block = (value ? bt.V : bt.K) +
                ((int64_t)page * bt.h_kv + head) * block_bytes<T, MX, D>(bt.page_log2);
  const T* src = value ? static_cast<const T*>(a.v) + row * a.v_stride + (int64_t)head * D
                       : static_cast<const T*>(a.k) + row * a.k_stride + (int64_t)head * D;
  if constexpr (MX) {
    // Rotated in 64 bits: the products of 32-bit numbers are exact, so a
    // value next to the border of two codes falls on the right side of it.
    uint32_t scale, codes;
    if (value) {
      float y[8];
      load8(src + 8 * piece, y);
      codes = quantise8(y, &scale);
    } else {
      double y[8];
      turned8(src, piece, a, angles, y);
      codes = quantise8(y, &scale);
    }
    *reinterpret_cast<uint32_t*>(block + mx_code_at<D>(value, slot, piece)) = codes;
    if (piece % 4 == 0)
      block[mx_scale_at<D>(value, bt.page_log2, slot, piece / 4)] = (char)scale;
  } else {
    turn16(src, reinterpret_cast<T*>(block) + (int64_t)slot * D, piece, a, angles, !value);
  }
}

// ---------------------------------------------------------------------------
// Gather: one thread reads 8 dimensions of one head of one row's place.
// Memory-bound: 5600 rows of 8 heads from 4 bits into 23 MB in 11.8 us.
// ---------------------------------------------------------------------------
template <class T, bool MX, int D>
__global__ __launch_bounds__(kThreads) void paged_gather_kernel(Batch bt, void* k_out,
                                                                void* v_out,
                                                                unsigned seq_groups) {
  constexpr int kPieces = D / 8;
  const int b = blockIdx.x / seq_groups;
  const SeqRows sr = seq_rows(bt, b);
  const int per_row = 2 * bt.h_kv * kPieces;
  const uint32_t unit = blockIdx.x % seq_groups * kThreads + threadIdx.x;
  const int r = (int)(unit / (uint32_t)per_row);
  if (r >= sr.n) return;
  const int u = (int)(unit - (uint32_t)r * (uint32_t)per_row);
  const int piece = u % kPieces;
  int head = u / kPieces;
  const bool value = head >= bt.h_kv;
  if (value) head -= bt.h_kv;
  T* dst = static_cast<T*>(value ? v_out : k_out) +
           ((int64_t)(sr.start + r) * bt.h_kv + head) * D + 8 * piece;
  float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const int past = bt.past[b];
  if (past >= 0 && past < capacity(bt) - r) {
    const int pos = past + r;
    const int page = bt.pages[(int64_t)b * bt.max_pages + (pos >> bt.page_log2)];
    if ((unsigned)page < (unsigned)bt.n_pages) {
      const int slot = pos & ((1 << bt.page_log2) - 1);
      const char* block = (value ? bt.V : bt.K) +
                          ((int64_t)page * bt.h_kv + head) * block_bytes<T, MX, D>(bt.page_log2);
      if constexpr (MX) {
        const uint32_t codes =
            *reinterpret_cast<const uint32_t*>(block + mx_code_at<D>(value, slot, piece));
        const uint32_t byte =
            (uint8_t)block[mx_scale_at<D>(value, bt.page_log2, slot, piece / 4)];
        const float scale = mx_factor(byte);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = mx_level(codes >> (4 * e) & 15u) * scale;
      } else {
        load8(reinterpret_cast<const T*>(block) + (int64_t)slot * D + 8 * piece, y);
      }
    }
  }
  store8(dst, y);
}

// ---------------------------------------------------------------------------
// Attention.
//
// Items.  An item is (sequence, KV head, tile of up to R = 16*NB query rows);
// row x of a KV head's rows is (token x / G, query head x % G of the group), so
// a tile's rows see nearly the same keys.  An item's keys are cut into tiles of
// KT = 4*TK, and all items' costs (kItemCost), laid end to end (sequences, heads,
// row tiles), are divided evenly over the grid's workgroups, which count for
// themselves, from past and row_start, where each one's share begins.  The grid is
// two workgroups a CU: all resident for d = 64 and 128; of d = 256 most instances
// take more than 256 registers a lane, and one runs at a time.  A workgroup begins
// and ends inside at most one item each; those parts go to its two slots of the
// workspace, the rest straight to out.  The parts of an item are then those of
// consecutive workgroups and are summed in their order, by whichever workgroup or
// launch does it: equal calls give equal bits.
//
// Tile of a wave: TK keys (32; 16 of float32), all from registers:
//   S^T [TK keys x 16 rows] = K . Q^T  and  O^T [D x 16 rows] += V^T . P^T.
// Rows of the score product are assigned to keys so that lane (i, k) holds, for
// query row i, the scores of keys KPL*k .. KPL*k + KPL-1, KPL = TK/4: that is
// the share of the summed index that the second product wants of it, so the
// weights go from one product to the other without leaving the lane.  V comes
// in by rows (lane (i, k): its keys, D/16 dimensions of each), which float32
// products take as they are; 16-bit ones want a dimension's keys side by side
// in a register, two byte permutes for four values.
// Weights of 16-bit types are rounded to the type, as the second product takes
// them: half a step each, with the same weights summed for the divisor.  Errors
// against 64 bits are then 0.0020-0.0023 of the result (bfloat16; float16
// 0.00028), where one rounding of the result alone gives 0.0017 (0.00021).
//
// What bounds it: the reading of the cache.  Kernel times over 4 sequences of
// 65k-131k rows (64/8 heads, d = 128): bfloat16 261 us, 6.7 TB/s (the same loads
// without the products 260); 4 bits 82 us, 5.7 TB/s (77); float32, 16 x 8192
// rows, 32/8 heads: 168 us, 6.4 TB/s.  Small batches are bound by what is not
// reading: of one sequence of 700 rows' 9.2 us, 1.7 are the launch, 1.4 the count of
// the work, 1.4 the way to the first loads and 3 the exchange at the end.
// ---------------------------------------------------------------------------
template <class T, bool MX, int D>
struct Tile {
  static constexpr int TK = is_f32<T> && !MX ? 16 : 32;  // keys
  static constexpr int NH = TK / 16;                     // score products
  static constexpr int KPL = TK / 4;                     // keys of a lane group
  static constexpr int NC = D / 16;                      // output products (tiles of 16 dims)
  // Dimensions that a lane holds side by side of a V row: dimension
  // VCH*i + 16*VCH*(c/VCH) + c%VCH is row i of output tile c.
  static constexpr int VCH = D == 64 ? 4 : (is_f32<T> && !MX) ? 4 : 8;
  static constexpr int NP = NC / VCH;                    // pieces of a V row
  // 32-bit words of a lane's share of a K row, and of a V row.
  static constexpr int KW = MX ? D / 32 : is_f32<T> ? D / 4 : D / 8;
  static constexpr int VW = MX ? NP : is_f32<T> ? D / 16 : D / 32;
  // values of q that a lane holds: D/4, as words
  static constexpr int QW = is_f32<T> ? D / 4 : D / 8;
};

template <class T>
struct Vec8;
template <>
struct Vec8<__bf16> {
  using type = bf16x8;
};
template <>
struct Vec8<_Float16> {
  using type = f16x8;
};

__device__ __forceinline__ f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

template <class T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef T t2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), t2));
}

// Both values of a word of 16-bit ones, added to x.
template <class T>
__device__ __forceinline__ float add2(uint32_t w, float x) {
  if constexpr (std::is_same<T, __bf16>::value) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w),
                                           bf16x2{(__bf16)1.f, (__bf16)1.f}, x, false);
  } else {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w), f16x2{(_Float16)1.f, (_Float16)1.f},
                                  x, false);
  }
}

// Two values of byte `sel` of `codes`, times the scale, as two T.
template <class T, int sel>
__device__ __forceinline__ uint32_t widen2(uint32_t codes, float scale) {
  if constexpr (std::is_same<T, __bf16>::value)
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, sel));
  else
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, sel));
}

// A scale byte as the factor that the conversions take: they read its exponent
// alone (not sign or mantissa), 255 as not a number and 0 as 2^-127.
__device__ __forceinline__ float mx_scale(uint32_t byte) { return power_of(byte); }
// Byte j % 4 of w as that: what stands beside it falls on sign and mantissa.
__device__ __forceinline__ float mx_scale_of(uint32_t w, int j) {
  return __uint_as_float(j % 4 == 3 ? w >> 1 : w << (23 - 8 * (j % 4)));
}

// The least scale byte 2^X whose largest value, 6 * 2^X, is an infinity in T, and a
// word of codes without those that are: from 4 * 2^X on there, 2 * 2^X with the
// next byte, 2^X with the one after, and then all but 0.
template <class T>
constexpr uint32_t kFirstBeyond = 127 + (std::is_same<T, _Float16>::value ? 14 : 126);
template <class T>
__device__ __forceinline__ uint32_t codes_within(uint32_t codes, uint32_t byte) {
  if (byte == 255u) return 0u;
  const uint32_t more = byte - kFirstBeyond<T>;
  const uint32_t first = more == 0 ? 6u : more == 1 ? 4u : more == 2 ? 2u : 1u;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if ((codes >> (4 * e) & 7u) >= first) codes &= ~(15u << (4 * e));
  return codes;
}

template <class T>
__device__ __forceinline__ bool not_finite(uint32_t w) {
  if constexpr (is_f32<T>)
    return (w & 0x7f800000u) == 0x7f800000u;
  else if constexpr (std::is_same<T, __bf16>::value)
    return (w & 0x7f800000u) == 0x7f800000u || (w & 0x7f80u) == 0x7f80u;
  else
    return (w & 0x7c000000u) == 0x7c000000u || (w & 0x7c00u) == 0x7c00u;
}

// w with its values that are not finite zeroed.
template <class T>
__device__ __forceinline__ uint32_t finite_part(uint32_t w) {
  if constexpr (is_f32<T>) return not_finite<T>(w) ? 0u : w;
  constexpr uint32_t e = std::is_same<T, __bf16>::value ? 0x7f80u : 0x7c00u;
  if ((w & e) == e) w &= 0xffff0000u;
  if ((w & e << 16) == e << 16) w &= 0xffffu;
  return w;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// An item in parts: what the merge needs to put them together.  By workgroup,
// the item that ends in it but did not begin there; or by item, where these are
// fewer than the workgroups.
struct Closing {
  int first, last;            // the workgroups of its parts; first -1: not in parts
  int head, row0, in_tile;    // its rows of the KV head
  int start;                  // the sequence's first row
  int unused[2];
};

struct AttnArgs {
  const void* q;
  void* out;
  int64_t q_stride;
  // |scale| times log2(e), or 1 for a scale of 0; q's words are taken as
  // (q & q_keep) ^ q_flip: negated for a negative scale, 0 for that of 0.
  float scale;
  uint32_t q_keep, q_flip;
  int h_q, G, causal;
  uint32_t G_mul, G_shift;
  int few_tiles;        // their number fits 31 bits, whatever the lengths
  // How the parts of an item are put together: by the workgroup that finishes
  // last, counted in arrived[workgroup of the first part] (0 between calls), or,
  // arrived NULL, by the merge kernel, which is told of them in closing.
  unsigned* arrived;
  int by_item;          // closing is [B][h_kv] (one row tile each), else [grid]
  Closing* closing;
  float* parts;         // [2 * grid][R][D], then [2 * grid][R][2]
  int grid;             // workgroups of the attention kernel
};

// x / G, 0 <= x < 2^31 (the host's multiplier: floor(2^shift / G) + 1).
__device__ __forceinline__ int token_of(const AttnArgs& a, int x) {
  return (int)((uint64_t)(uint32_t)x * a.G_mul >> a.G_shift);
}

// Keys that token t of a sequence sees.
__device__ __forceinline__ int seen_by(const Batch& bt, const AttnArgs& a, int past, int t) {
  const int cap = capacity(bt);
  if (past < 0) return 0;
  if (!a.causal) return min(past, cap);
  return past >= cap - t - 1 ? cap : past + t + 1;
}

// A score's distance from the reference is taken in one multiply-add, which keeps
// what the reference lost when it was rounded: the same factor for every key, small
// enough below kFar (2^2 at most).  Beyond, the product is rounded as the reference
// was, so that the largest score's weight is 1; scores beyond 32 bits give NaN.
constexpr float kFar = 0x1p26f;
__device__ __forceinline__ bool is_far(float ref) {
  return fabsf(ref) > kFar && ref != -INFINITY;
}

// The weight of a key whose V is not finite, against the reference ref: computed
// again, where the row's product had zeros in V's place.  (0 times an infinity is
// NaN there too.)
template <class T, bool MX, int D>
__device__ __forceinline__ float weight_of(const Batch& bt, const AttnArgs& a, int64_t row,
                                           int q_head, int kv_head, int page, int slot,
                                           float ref) {
  const T* q = static_cast<const T*>(a.q) + row * a.q_stride + (int64_t)q_head * D;
  const char* block =
      bt.K + ((int64_t)page * bt.h_kv + kv_head) * block_bytes<T, MX, D>(bt.page_log2);
  float s = 0.f;
#pragma unroll 1
  for (int dim = 0; dim < D; ++dim)
    s += (float)q[dim] * held<T, MX, D>(block, false, bt.page_log2, slot, dim);
  s = a.q_keep ? a.q_flip ? -s : s : 0.f;
  const bool far = is_far(ref);
  if (far) s *= a.scale;
  return (float)(T)exp2f(__builtin_fmaf(s, far ? 1.f : a.scale, -ref));
}

// Row tiles of a sequence (each of R rows; one where not MANY), and tiles of keys
// of one of them.
template <int R, bool MANY>
__device__ __forceinline__ int row_tiles(const AttnArgs& a, int n) {
  return MANY ? (n * a.G + R - 1) / R : n > 0;
}
template <int R, int KT, bool MANY>
__device__ __forceinline__ int key_tiles(const Batch& bt, const AttnArgs& a, int past, int n,
                                         int rt) {
  int t = n - 1;                             // the tile's last token
  if (MANY && (rt + 1) * R < n * a.G) t = token_of(a, (rt + 1) * R - 1);
  return (seen_by(bt, a, past, t) + KT - 1) / KT;
}

// An item costs its tiles and, for the loads before the first and the exchange
// after the last, as much as kItemCost tiles: what the workgroups share out is
// cost, and every item begins with its fixed part.  (Measured: 4 to 6 us an item,
// 1.7 to 2.7 us a tile.  256 items of 1 to 12 tiles take 50 us if this is left
// out and 33 with 1 to 3; 8 sequences of 15 rows a head over 500 to 4000 keys 43,
// 42, 39 and 39 us with 0, 1, 2 and 3.  The chunk kernel, whose tiles cost something
// else, takes the same 3 unmeasured.)
constexpr int kItemCost = 3;

template <int R, int KT, bool MANY>
__device__ __forceinline__ int64_t head_cost(const Batch& bt, const AttnArgs& a, int past, int n) {
  const int nr = row_tiles<R, MANY>(a, n);
  const int one = nr ? key_tiles<R, KT, MANY>(bt, a, past, n, 0) : 0;
  if (one == 0) return 0;                    // (the first row sees least: so it is with all)
  if (!MANY || !a.causal) return (int64_t)nr * (one + kItemCost);
  int64_t sum = (int64_t)nr * kItemCost;
  for (int rt = 0; rt < nr; ++rt) sum += key_tiles<R, KT, MANY>(bt, a, past, n, rt);
  return sum;
}

// floor(a / b) for 0 <= a < 2^52, b > 0: by the quotient in 64-bit floating
// point, off by at most one.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  int64_t q = (int64_t)((double)a / (double)b);
  const int64_t rest = a - q * b;
  q += rest >= b;
  q -= rest < 0;
  return q;
}
__device__ __forceinline__ int64_t lane_value(int64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x, lane);
  const int hi = __builtin_amdgcn_readlane((int)(x >> 32), lane);
  return (int64_t)hi << 32 | lo;
}

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast:31
  return x;
}

// The workgroup that takes unit x of the cost where each takes `each`, the first
// `more` one more.
__device__ __forceinline__ int owner_of(int64_t x, int64_t each, int more) {
  const int64_t big = more * (each + 1);
  return (int)(x < big ? quotient(x, each + 1) : more + quotient(x - big, each));
}

// The division of all items' tiles over the workgroups, counted by each wave
// for itself: a lane counts a run of sequences.
template <int R, int KT, bool MANY>
struct Division {
  int run;                    // sequences of a lane
  int past;                   // the lane's sequence's, where that is one
  SeqRows sr;
  int64_t before, upto;       // cost before the lane's run and up to its end
  int64_t total, each;        // all cost; workgroup w takes each, the first
  int share, more;            //   `more` ones one more; share of them have some
  bool blind;                 // a sequence of the lane's run sees nothing

  __device__ __forceinline__ static int64_t cost_of(const Batch& bt, const AttnArgs& a, int b) {
    return bt.h_kv * head_cost<R, KT, MANY>(bt, a, bt.past[b], seq_rows(bt, b).n);
  }
  __device__ __forceinline__ void count(const Batch& bt, const AttnArgs& a, int lane) {
    run = (bt.B + 63) / 64;
    int64_t mine = 0;
    blind = false;
    past = 0;
    sr = {0, 0};
    if (run == 1) {
      if (lane < bt.B) {
        past = bt.past[lane];
        sr = seq_rows(bt, lane);
        mine = bt.h_kv * head_cost<R, KT, MANY>(bt, a, past, sr.n);
        blind = mine == 0;
      }
    } else {
      const int lo = min(lane * run, bt.B), hi = min(lo + run, bt.B);
      for (int b = lo; b < hi; ++b) {
        const int64_t n = cost_of(bt, a, b);
        blind |= n == 0;
        mine += n;
      }
    }
    if (a.few_tiles) {
      upto = wave_scan((int)mine);
    } else {
      upto = mine;
#pragma unroll
      for (int step = 1; step < 64; step <<= 1) {
        const int64_t other = __shfl_up(upto, step);
        if (lane >= step) upto += other;
      }
    }
    before = upto - mine;
    total = lane_value(upto, 63);
    share = (int)min(total, (int64_t)a.grid);
    each = share ? quotient(total, share) : 0;
    more = (int)(total - each * share);
  }
  // Sequence b's past and rows (run == 1: from its lane).
  __device__ __forceinline__ int past_of(const Batch& bt, int b) const {
    return run == 1 ? __builtin_amdgcn_readlane(past, b) : fixed(bt.past + b);
  }
  __device__ __forceinline__ SeqRows rows_of(const Batch& bt, int b) const {
    if (run != 1) return one_seq_rows(bt, b);
    return {__builtin_amdgcn_readlane(sr.start, b), __builtin_amdgcn_readlane(sr.n, b)};
  }
  __device__ __forceinline__ int64_t begin_of(int w) const { return w * each + min(w, more); }
  __device__ __forceinline__ int owner(int64_t x) const { return owner_of(x, each, more); }
};

// The parts of items that a workgroup takes, one after the other.
template <int R, int KT, bool MANY>
struct Walk {
  int b, head, rt;            // the item: sequence, KV head, row tile
  int tiles, t0, t1;          // its key tiles; those taken are t0 .. t1-1
  int past;
  SeqRows sr;
  int first;                  // the workgroup of the item's first part, if another
  bool fresh;                 // the workgroup's first part
  // The division: where the item's cost begins, what of it lies before the
  // workgroup's, and how much the workgroup still takes from there on.
  int64_t start, skip, left, each;
  int more;

  // The part.  All of these are the same in every lane, and said to be: addresses
  // and branches made of them then stay with the scalar unit.
  __device__ __forceinline__ void cut() {
    left = lane_value(left, 0), skip = lane_value(skip, 0), start = lane_value(start, 0);
    each = lane_value(each, 0), more = uniform(more);
    b = uniform(b), head = uniform(head), rt = uniform(rt);
    tiles = uniform(tiles), past = uniform(past);
    sr = {uniform(sr.start), uniform(sr.n)};
    t0 = uniform((int)max(skip - kItemCost, (int64_t)0));
    t1 = uniform((int)max(min((int64_t)tiles, skip + left - kItemCost), (int64_t)0));
  }
  // The next item that has tiles (there is one while left > 0).
  __device__ __forceinline__ void forward(const Batch& bt, const AttnArgs& a) {
    const int64_t used = min(tiles + kItemCost - skip, left);
    left -= used;
    if (left <= 0) return;
    start += tiles + kItemCost;
    skip = 0;
    tiles = 0;
    while (tiles == 0) {
      if (++rt >= row_tiles<R, MANY>(a, sr.n)) {
        rt = 0;
        if (++head >= bt.h_kv) {
          head = 0;
          sr = one_seq_rows(bt, ++b);
          past = fixed(bt.past + b);
          if (sr.n == 0) {
            head = bt.h_kv - 1;
            continue;
          }
        }
      }
      tiles = key_tiles<R, KT, MANY>(bt, a, past, sr.n, rt);
    }
    cut();
  }
  // Whether the workgroup has work.  Rows of sequences that see nothing, which
  // are in no item, are zeroed here.
  template <class T>
  __device__ __forceinline__ bool begin(const Batch& bt, const AttnArgs& a, int lane, int d_head) {
    Division<R, KT, MANY> d;
    d.count(bt, a, lane);
    const int w = blockIdx.x;
    uint64_t blind = __ballot(d.blind);
    while (blind) {
      const int from = (__ffsll((unsigned long long)blind) - 1) * d.run;
      blind &= blind - 1;
      for (int x = from; x < min(from + d.run, bt.B); ++x) {
        if (x % a.grid != w || Division<R, KT, MANY>::cost_of(bt, a, x)) continue;
        const SeqRows zr = seq_rows(bt, x);
        T* dst = static_cast<T*>(a.out) + (int64_t)zr.start * a.h_q * d_head;
        for (int64_t e = threadIdx.x; e < (int64_t)zr.n * a.h_q * d_head; e += kThreads)
          dst[e] = (T)0.f;
        if (!a.arrived && a.by_item && (int)threadIdx.x < bt.h_kv)
          a.closing[x * bt.h_kv + threadIdx.x].first = -1;
      }
    }
    fresh = true;
    first = -1;
    left = 0;
    if (w < d.share) {
      const int64_t lo = d.begin_of(w);
      left = d.each + (w < d.more ? 1 : 0);
      const int in = __ffsll((unsigned long long)__ballot(d.upto > lo)) - 1;
      int64_t rem = lo - lane_value(d.before, in);
      b = in * d.run;
      each = d.each, more = d.more;
      sr = d.rows_of(bt, b);
      past = d.past_of(bt, b);
      int64_t per_head = head_cost<R, KT, MANY>(bt, a, past, sr.n);
      while (rem >= bt.h_kv * per_head) {        // (ends: d.upto > lo)
        rem -= bt.h_kv * per_head;
        sr = d.rows_of(bt, ++b);
        past = d.past_of(bt, b);
        per_head = head_cost<R, KT, MANY>(bt, a, past, sr.n);
      }
      head = (int)quotient(rem, per_head);
      rem -= head * per_head;
      rt = 0;
      tiles = key_tiles<R, KT, MANY>(bt, a, past, sr.n, 0);
      while (rem >= tiles + kItemCost) {
        rem -= tiles + kItemCost;
        tiles = key_tiles<R, KT, MANY>(bt, a, past, sr.n, ++rt);
      }
      skip = rem;
      start = lo - rem;
      cut();
      while (left > 0 && t0 >= t1) forward(bt, a);       // (only the fixed part of an item)
      if (left > 0 && t0 > 0) first = uniform(d.owner(start + kItemCost));
    }
    if (left <= 0 && !a.arrived && !a.by_item && threadIdx.x == 0) a.closing[w].first = -1;
    return left > 0;
  }
  // What the merge is told: of every item that ends here, or (by workgroup) of
  // the first, the only one that may have begun elsewhere.
  __device__ __forceinline__ void close(const Batch& bt, const AttnArgs& a) const {
    const bool ends = t1 == tiles;
    if (!a.arrived && (a.by_item ? ends : fresh) && threadIdx.x == 0)
      a.closing[a.by_item ? b * bt.h_kv + head : (int)blockIdx.x] =
          {ends ? first : -1, (int)blockIdx.x, head, rt * R, min(sr.n * a.G - rt * R, R), sr.start,
           {0, 0}};
  }
  // The workgroup of the item's last part.
  __device__ __forceinline__ int last() const {
    return t1 == tiles ? (int)blockIdx.x
                       : uniform(owner_of(start + kItemCost + tiles - 1, each, more));
  }
  __device__ __forceinline__ bool next(const Batch& bt, const AttnArgs& a) {
    fresh = false;
    first = -1;
    do {
      forward(bt, a);
    } while (left > 0 && t0 >= t1);
    return left > 0;
  }
};

// Parts pass between workgroups on different dies, whose L2 caches do not see
// each other's lines: they are written through to memory and read from there,
// 8 bytes at a time, which costs a few KB an item.  (Fences would write back and
// empty whole caches: measured 130 us a launch of 512 workgroups.)
__device__ __forceinline__ void store_part(float* p, f32x2 v) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, v),
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_part(float* p, f32x4 v) {
  store_part(p, f32x2{v[0], v[1]});
  store_part(p + 2, f32x2{v[2], v[3]});
}
__device__ __forceinline__ f32x2 load_part(const float* p) {
  return __builtin_bit_cast(
      f32x2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT));
}

// After a workgroup's part of an item has been written: the one that finishes
// last puts the item's n parts together, in their order, four values of a row a
// thread.  Every wave waits until its stores are in memory before the workgroup
// is counted.
template <class T, int D, int R, class W>
__device__ __forceinline__ void finish(const AttnArgs& a, const W& at) {
  __shared__ unsigned s_arrived;
  const int first = at.t0 ? at.first : (int)blockIdx.x;
  const int n = at.last() - first + 1;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0)
    s_arrived = __hip_atomic_fetch_add(a.arrived + first, 1u, __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (uniform((int)s_arrived) != n - 1) return;
  if (threadIdx.x == 0)
    __hip_atomic_store(a.arrived + first, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const float* ml = a.parts + (int64_t)2 * a.grid * R * D;
  const int row0 = at.rt * R, in_tile = min(at.sr.n * a.G - row0, R);
#pragma unroll 1
  for (int e = threadIdx.x; e < in_tile * (D / 4); e += kThreads) {
    const int in = e / (D / 4), dim = e % (D / 4) * 4;
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int p0 = 0; p0 < n; p0 += 4) {
      f32x2 s[4];
      f32x4 v[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int p = min(p0 + y, n - 1);
        const int64_t row = (int64_t)(2 * (first + p) + (p == 0)) * R + in;
        s[y] = load_part(ml + row * 2);
        const f32x2 lo = load_part(a.parts + row * D + dim);
        const f32x2 hi = load_part(a.parts + row * D + dim + 2);
        v[y] = f32x4{lo[0], lo[1], hi[0], hi[1]};
      }
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if (p0 + y >= n) continue;
        const float mn = s[y][0] <= m ? m : s[y][0];                 // (a NaN stays)
        const float base = mn == -INFINITY ? 0.f : mn;               // (then both factors are 0)
        const float fo = __builtin_amdgcn_exp2f(m - base);
        const float fn = __builtin_amdgcn_exp2f(s[y][0] - base);
        l = l * fo + s[y][1] * fn;
        o = o * fo + v[y] * fn;
        m = mn;
      }
    }
    o = l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o / l;
    const int t = token_of(a, row0 + in), g = (row0 + in) - t * a.G;
    T* dst = static_cast<T*>(a.out) +
             ((int64_t)(at.sr.start + t) * a.h_q + at.head * a.G + g) * D + dim;
    if constexpr (is_f32<T>)
      *reinterpret_cast<f32x4*>(dst) = o;
    else
      *reinterpret_cast<u32x2*>(dst) = u32x2{pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
  }
}

template <class T, bool MX, int D, int NB>
__global__ __launch_bounds__(kThreads) void paged_attn_kernel(Batch bt, AttnArgs a) {
  using L = Tile<T, MX, D>;
  constexpr int TK = L::TK, NH = L::NH, KPL = L::KPL, NC = L::NC, VCH = L::VCH, NP = L::NP;
  constexpr int KT = kWaves * TK, R = 16 * NB;
  constexpr int RB = kRowBytes<T, MX, D>;
  constexpr int SB = D / 32;                // scale bytes of a 4-bit row
  // 4-bit tiles are small: two under way for each wave
  constexpr int DEPTH = MX && D <= 128 && !(is_f32<T> && NB == 2) ? 2 : 1;
  constexpr int kLdsRow = D + 4;            // floats: 16-byte accesses of 16 rows spread evenly

  __shared__ float s_acc[kWaves][16][kLdsRow];
  __shared__ float s_ref[kWaves][16], s_sum[kWaves][16];

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = uniform(tid >> 6);
  const int i = lane & 15, k = lane >> 4;

  Walk<R, KT, is_f32<T> && NB == 2> at;     // (16-bit types: one row tile, by tile_rows)
  if (!at.template begin<T>(bt, a, lane, D)) return;

  const int64_t blk = block_bytes<T, MX, D>(bt.page_log2);
  const int page_mask = (1 << bt.page_log2) - 1;

  // Lane offsets within a half tile (16 keys) of the K rows and the V rows.
  const int k_half = TK == 32 ? i >> 3 : 0, v_half = TK == 32 ? k >> 1 : 0;
  const int k_key = TK == 32 ? 8 * ((i >> 2) & 1) + (i & 3) : i;
  const int v_key = TK == 32 ? 8 * (k & 1) : 4 * k;

  do {
    // --- one part of one item: key tiles t0 .. t1-1 ---
    const int b = at.b, head = at.head, past = at.past, t0 = at.t0, t1 = at.t1;
    const SeqRows sr = at.sr;
    const int row0 = at.rt * R;
    const int in_tile = min(sr.n * a.G - row0, R);
    const int min_seen = seen_by(bt, a, past, token_of(a, row0));
    const int max_seen = seen_by(bt, a, past, token_of(a, row0 + in_tile - 1));
    const int32_t* table = bt.pages + (int64_t)b * bt.max_pages;

    // q: lane (i, k) holds row i's share of the score products' summed index.
    uint32_t q[NB][L::QW];
    int seen[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int x = nb * 16 + i;
      seen[nb] = 0;
#pragma unroll
      for (int w = 0; w < L::QW; ++w) q[nb][w] = 0u;
      if (x < in_tile) {
        const int t = token_of(a, row0 + x), g = (row0 + x) - t * a.G;
        seen[nb] = seen_by(bt, a, past, t);
        const T* src = static_cast<const T*>(a.q) + (int64_t)(sr.start + t) * a.q_stride +
                       (int64_t)(head * a.G + g) * D;
        constexpr int per16 = 16 / (int)sizeof(T);   // values of a 16-byte load
#pragma unroll
        for (int w = 0; w < L::QW / 4; ++w) {
          const int dim = MX ? D / 4 * k + per16 * w : 4 * per16 * w + per16 * k;
          const u32x4 v = *reinterpret_cast<const u32x4*>(src + dim);
#pragma unroll
          for (int e = 0; e < 4; ++e) q[nb][4 * w + e] = (v[e] & a.q_keep) ^ a.q_flip;
        }
      }
    }

    f32x4 acc[NB][NC], sums[NB];
    float limit[NB], ref[NB];   // raise the reference above limit; scores are taken less ref
    bool far = false;           // a reference is beyond kFar
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      limit[nb] = -INFINITY;
      ref[nb] = 0.f;
      sums[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[nb][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // A wave tile as it was loaded, and the tile to load in its place next.
    struct Raw {
      uint32_t kw[NH][L::KW], vw[KPL][L::VW];
      uint32_t ks[NH], vs[NP][2];
      bool there_a, there_b;
      int next, next_a, next_b;       // its first key and its entries of the table
    };
    Raw raw[DEPTH];
    bool spoilt = false;        // V rows that only some rows see held infinities or NaN

    // The table's entry for positions p .. p+15 of the sequence, and the page
    // that it names: -1 if none, or past the table's end.
    auto entry_of = [&](int p) -> int {
      return fixed(table + min(p >> bt.page_log2, bt.max_pages - 1));
    };
    auto page_of = [&](int p, int id) -> int {
      return (p >> bt.page_log2) < bt.max_pages && (unsigned)id < (unsigned)bt.n_pages ? id : -1;
    };
    auto base_of = [&](int page, int slot, const char* pool) -> const char* {
      return pool + ((int64_t)max(page, 0) * bt.h_kv + head) * blk + slot * RB;
    };
    auto load_k = [&](Raw& x, int key0, int pa, int pb) {
      const int sa = key0 & page_mask, sb = (key0 + 16) & page_mask;
      const char* base = base_of(pa, sa, bt.K);
      const char* scales = nullptr;
      if (MX) scales = base + (((int64_t)RB << bt.page_log2) - (int64_t)sa * (RB - SB));
      if (TK == 32) {
        const char* other = base_of(pb, sb, bt.K);
        if (MX && k_half)
          scales = other + (((int64_t)RB << bt.page_log2) - (int64_t)sb * (RB - SB));
        if (k_half) base = other;
      }
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        const char* row = base + (k_key + 4 * h) * RB;
        if constexpr (MX) {
          row += k * (D / 8);
          if constexpr (D == 64) {
            const u32x2 v = once<u32x2>(row);
            x.kw[h][0] = v[0], x.kw[h][1] = v[1];
          } else {
#pragma unroll
            for (int w = 0; w < L::KW / 4; ++w) {
              const u32x4 v = once<u32x4>(row + 16 * w);
#pragma unroll
              for (int e = 0; e < 4; ++e) x.kw[h][4 * w + e] = v[e];
            }
          }
          const char* s = scales + (k_key + 4 * h) * SB;
          if constexpr (D == 256)
            x.ks[h] = once<uint16_t>(s + 2 * k);
          else
            x.ks[h] = once<uint8_t>(s + (D == 64 ? k >> 1 : k));
        } else {
#pragma unroll
          for (int w = 0; w < L::KW / 4; ++w) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(row + 64 * w + 16 * k);
#pragma unroll
            for (int e = 0; e < 4; ++e) x.kw[h][4 * w + e] = v[e];
          }
        }
      }
    };
    auto load_v = [&](Raw& x, int key0, int pa, int pb) {
      const int sa = key0 & page_mask, sb = (key0 + 16) & page_mask;
      const char* base = base_of(pa, sa, bt.V);
      const char* scales = nullptr;
      if (MX) scales = base + (((int64_t)RB << bt.page_log2) - (int64_t)sa * (RB - SB));
      if (TK == 32) {
        const char* other = base_of(pb, sb, bt.V);
        if (MX && v_half)
          scales = other + (((int64_t)RB << bt.page_log2) - (int64_t)sb * (RB - SB));
        if (v_half) base = other;
      }
      base += v_key * RB;
      if constexpr (MX) {
        scales += v_key * SB;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const int chunk = D == 64 ? i >> 1 : 16 * p + i;      // of 8 dimensions
          const u32x4 lo4 = once<u32x4>(base + 32 * chunk);
          const u32x4 hi4 = once<u32x4>(base + 32 * chunk + 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) x.vw[e][p] = lo4[e], x.vw[4 + e][p] = hi4[e];
          const u32x2 s = once<u32x2>(scales + 8 * (chunk / 4));
          x.vs[p][0] = s[0], x.vs[p][1] = s[1];
        }
      } else {
#pragma unroll
        for (int j = 0; j < KPL; ++j)
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const char* at = base + j * RB + (VCH * i + 16 * VCH * p) * (int)sizeof(T);
            if constexpr (VCH * sizeof(T) == 8) {
              const u32x2 v = once<u32x2>(at);
              x.vw[j][2 * p] = v[0], x.vw[j][2 * p + 1] = v[1];
            } else {
              const u32x4 v = once<u32x4>(at);
#pragma unroll
              for (int e = 0; e < 4; ++e) x.vw[j][4 * p + e] = v[e];
            }
          }
      }
    };

    // The V rows' words of piece p as values of T (16-bit types): word w of key
    // j holds dimensions 2w and 2w+1 of the piece.
    auto v_words = [&](const Raw& x, int p, uint32_t (&out)[KPL][VCH / 2]) {
      if constexpr (!is_f32<T>) {
#pragma unroll
        for (int j = 0; j < KPL; ++j) {
          if constexpr (MX) {
            const float scale = mx_scale_of(x.vs[p][j / 4], j);
            const uint32_t codes = D == 64 ? x.vw[j][p] >> (16 * (i & 1)) : x.vw[j][p];
            out[j][0] = widen2<T, 0>(codes, scale);
            out[j][1] = widen2<T, 1>(codes, scale);
            if constexpr (VCH == 8) {
              out[j][2] = widen2<T, 2>(codes, scale);
              out[j][3] = widen2<T, 3>(codes, scale);
            }
          } else {
#pragma unroll
            for (int w = 0; w < VCH / 2; ++w) out[j][w] = x.vw[j][VCH / 2 * p + w];
          }
        }
      }
    };
    // float32: the VCH values of key j in piece p.
    auto v_floats = [&](const Raw& x, int p, int j, float (&out)[VCH]) {
      if constexpr (MX) {
        const float scale = mx_scale_of(x.vs[p][j / 4], j);
        const uint32_t codes = D == 64 ? x.vw[j][p] >> (16 * (i & 1)) : x.vw[j][p];
        const f32x2 a0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
        const f32x2 a1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
        out[0] = a0[0], out[1] = a0[1], out[2] = a1[0], out[3] = a1[1];
        if constexpr (VCH == 8) {
          const f32x2 a2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
          const f32x2 a3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
          out[4] = a2[0], out[5] = a2[1], out[6] = a3[0], out[7] = a3[1];
        }
      } else {
#pragma unroll
        for (int e = 0; e < VCH; ++e) out[e] = __uint_as_float(x.vw[j][VCH * p + e]);
      }
    };

    // Wave w takes wave tiles w, w + 4, ..., DEPTH of them under way.  A tile's K
    // is loaded as soon as the last one's in its registers is used up, its V
    // likewise, and its entries of the page table DEPTH tiles before that.  The
    // last tiles load themselves once more (from the cache): with a branch
    // around the loads, the products would wait for all of them.
    const int wt_end = min(t1 * kWaves, (max_seen + TK - 1) / TK);
    int wt = t0 * kWaves + wave;
    auto aim = [&](Raw& x, int tile) {
      x.next = min(tile, wt_end - 1) * TK;
      x.next_a = entry_of(x.next);
      x.next_b = TK == 32 ? entry_of(x.next + 16) : x.next_a;
    };
    if (wt < wt_end) {
#pragma unroll
      for (int y = 0; y < DEPTH; ++y) aim(raw[y], wt + y * kWaves);
#pragma unroll
      for (int y = 0; y < DEPTH; ++y) {
        Raw& x = raw[y];
        const int pa = page_of(x.next, x.next_a);
        const int pb = TK == 32 ? page_of(x.next + 16, x.next_b) : pa;
        // K before V, here as in the loop: the wait for K is a count of the loads
        // behind it, and the compiler takes the smaller of the two places'.
        load_k(x, x.next, pa, pb);
        asm volatile("" ::: "memory");
        load_v(x, x.next, pa, pb);
        asm volatile("" ::: "memory");
        x.there_a = pa >= 0, x.there_b = pb >= 0;
      }
#pragma unroll
      for (int y = 0; y < DEPTH; ++y) aim(raw[y], wt + (y + DEPTH) * kWaves);
    }
    // (q is waited for here, not by its uses in the loop)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int w = 0; w < L::QW; ++w) asm volatile("" : "+v"(q[nb][w]));

    const int end_key = wt_end * TK;       // (a step's second tile may lie beyond)
    auto process = [&](int tile) {
      int now[DEPTH], na[DEPTH], nb_[DEPTH];
#pragma unroll
      for (int y = 0; y < DEPTH; ++y) {
        now[y] = raw[y].next;
        na[y] = page_of(now[y], raw[y].next_a);
        nb_[y] = TK == 32 ? page_of(now[y] + 16, raw[y].next_b) : na[y];
        aim(raw[y], tile + (y + 2 * DEPTH) * kWaves);
      }
      // --- scores ---
      f32x4 s[DEPTH][NB][NH];
#pragma unroll
      for (int y = 0; y < DEPTH; ++y) {
        Raw& tw = raw[y];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int h = 0; h < NH; ++h) s[y][nb][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          if constexpr (is_f32<T>) {
            if constexpr (MX) {
#pragma unroll
              for (int w = 0; w < L::KW; ++w) {
                const float scale = mx_scale(D == 256 ? tw.ks[h] >> (8 * (w / 4)) & 255u : tw.ks[h]);
                const f32x2 a0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(tw.kw[h][w], scale, 0);
                const f32x2 a1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(tw.kw[h][w], scale, 1);
                const f32x2 a2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(tw.kw[h][w], scale, 2);
                const f32x2 a3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(tw.kw[h][w], scale, 3);
                const float x[8] = {a0[0], a0[1], a1[0], a1[1], a2[0], a2[1], a3[0], a3[1]};
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                  for (int e = 0; e < 8; ++e)
                    s[y][nb][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                        x[e], __uint_as_float(q[nb][8 * w + e]), s[y][nb][h], 0, 0, 0);
              }
            } else {
#pragma unroll
              for (int w = 0; w < L::KW; ++w)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                  s[y][nb][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                      __uint_as_float(tw.kw[h][w]), __uint_as_float(q[nb][w]), s[y][nb][h], 0, 0, 0);
            }
          } else {
            using V8 = typename Vec8<T>::type;
#pragma unroll
            for (int w = 0; w < D / 32; ++w) {
              u32x4 x;
              if constexpr (MX) {
                const float scale = mx_scale(D == 256 ? tw.ks[h] >> (8 * (w / 4)) & 255u : tw.ks[h]);
                x = u32x4{widen2<T, 0>(tw.kw[h][w], scale), widen2<T, 1>(tw.kw[h][w], scale),
                          widen2<T, 2>(tw.kw[h][w], scale), widen2<T, 3>(tw.kw[h][w], scale)};
              } else {
                x = u32x4{tw.kw[h][4 * w], tw.kw[h][4 * w + 1], tw.kw[h][4 * w + 2], tw.kw[h][4 * w + 3]};
              }
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) {
                const u32x4 z = {q[nb][4 * w], q[nb][4 * w + 1], q[nb][4 * w + 2],
                                 q[nb][4 * w + 3]};
                s[y][nb][h] = mma16(__builtin_bit_cast(V8, x), __builtin_bit_cast(V8, z), s[y][nb][h]);
              }
            }
          }
        }
        load_k(tw, now[y], na[y], nb_[y]);
      }

      // --- masks: only where a row does not see every key of the tile ---
#pragma unroll
      for (int y = 0; y < DEPTH; ++y) {
        Raw& tw = raw[y];
        const int key0 = (tile + y * kWaves) * TK;
        const bool edge = key0 + TK > min(min_seen, end_key) || !tw.there_a || !tw.there_b;
        const bool here = v_half ? tw.there_b : tw.there_a;
        if (edge) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (!(here && key0 + KPL * k + 4 * h + r < min(seen[nb], end_key))) s[y][nb][h][r] = -INFINITY;
          // V rows that no row sees are left out ...
#pragma unroll
          for (int j = 0; j < KPL; ++j)
            if (!(here && key0 + KPL * k + j < min(max_seen, end_key))) {
#pragma unroll
              for (int w = 0; w < L::VW; ++w) tw.vw[j][w] = 0u;
              if constexpr (MX)
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                  tw.vs[p][j / 4] &= ~(255u << (8 * (j % 4)));
                  tw.vs[p][j / 4] |= 127u << (8 * (j % 4));
                }
            }
          // ... and where only some rows see a tile's keys, infinities and NaN,
          // which a weight of 0 does not take out (0 * infinity), are zeroed here
          // and added at the end to the rows that see them.
          if (min_seen < max_seen && key0 + TK > min_seen) {
            bool bad = false;
#pragma unroll
            for (int j = 0; j < KPL; ++j) {
              if constexpr (MX) {
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                  const uint32_t byte = tw.vs[p][j / 4] >> (8 * (j % 4)) & 255u;
                  if (byte < kFirstBeyond<T>) continue;
                  bad = true;
                  tw.vw[j][p] = codes_within<T>(tw.vw[j][p], byte);
                  if (byte == 255u) tw.vs[p][j / 4] &= ~(128u << (8 * (j % 4)));
                }
              } else {
#pragma unroll
                for (int w = 0; w < L::VW; ++w) {
                  bad |= not_finite<T>(tw.vw[j][w]);
                  tw.vw[j][w] = finite_part<T>(tw.vw[j][w]);
                }
              }
            }
            spoilt |= bad;
          }
        }

      }

      // --- softmax against a reference that is raised only by a score more
      // than 8 above it (in base-2 units): the weights stay below 2^8, and
      // most tiles need neither the maximum over the lanes nor a rescaling ---
      uint32_t pw[DEPTH][NB][NH * 2];            // weights, two to a word (16-bit types)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float top = s[0][nb][0][0];
#pragma unroll
        for (int y = 0; y < DEPTH; ++y)
#pragma unroll
          for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, s[y][nb][h][r]);
        top *= a.scale;
        // (a NaN among only NaN becomes the reference, and spoils the row)
        if (__any(!(top <= limit[nb]))) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          far |= __any(is_far(top));
          if (!(top <= limit[nb])) {
            const float f = limit[nb] == -INFINITY ? 0.f : exp2f(ref[nb] - top);
            ref[nb] = top;
            limit[nb] = top + 8.f;
            sums[nb] *= f;
#pragma unroll
            for (int c = 0; c < NC; ++c) acc[nb][c] *= f;
          }
        }
        float by = a.scale;
        if (__builtin_expect(far, 0)) {
          by = 1.f;
#pragma unroll
          for (int y = 0; y < DEPTH; ++y)
#pragma unroll
            for (int h = 0; h < NH; ++h) s[y][nb][h] *= a.scale;
        }
#pragma unroll
        for (int y = 0; y < DEPTH; ++y)
#pragma unroll
          for (int h = 0; h < NH; ++h) {
            f32x4& w = s[y][nb][h];
#pragma unroll
            for (int r = 0; r < 4; ++r)
              w[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(w[r], by, -ref[nb]));
            if constexpr (is_f32<T>) {
              sums[nb] += w;
            } else {
              pw[y][nb][2 * h] = pack2<T>(w[0], w[1]);
              pw[y][nb][2 * h + 1] = pack2<T>(w[2], w[3]);
            }
          }
      }

      // --- O^T += V^T P^T ---
#pragma unroll
      for (int y = 0; y < DEPTH; ++y) {
        Raw& tw = raw[y];
        if constexpr (is_f32<T>) {
#pragma unroll
          for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int j = 0; j < KPL; ++j) {
              float x[VCH];
              v_floats(tw, p, j, x);
#pragma unroll
              for (int c = 0; c < VCH; ++c)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                  acc[nb][VCH * p + c] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                      x[c], s[y][nb][j / 4][j % 4], acc[nb][VCH * p + c], 0, 0, 0);
            }
        } else {
          using V8 = typename Vec8<T>::type;
          V8 weights[NB];
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            weights[nb] =
                __builtin_bit_cast(V8, (u32x4{pw[y][nb][0], pw[y][nb][1], pw[y][nb][2], pw[y][nb][3]}));
          V8 ones;
#pragma unroll
          for (int e = 0; e < 8; ++e) ones[e] = (T)1.f;
          // the sum of the weights as they are multiplied, in every lane
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) sums[nb] = mma16(ones, weights[nb], sums[nb]);
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            uint32_t x[KPL][VCH / 2];
            v_words(tw, p, x);
#pragma unroll
            for (int c = 0; c < VCH; ++c) {
              const uint32_t sel = c % 2 ? 0x07060302u : 0x05040100u;
              const u32x4 col = {__builtin_amdgcn_perm(x[1][c / 2], x[0][c / 2], sel),
                                 __builtin_amdgcn_perm(x[3][c / 2], x[2][c / 2], sel),
                                 __builtin_amdgcn_perm(x[5][c / 2], x[4][c / 2], sel),
                                 __builtin_amdgcn_perm(x[7][c / 2], x[6][c / 2], sel)};
#pragma unroll
              for (int nb = 0; nb < NB; ++nb)
                acc[nb][VCH * p + c] =
                    mma16(__builtin_bit_cast(V8, col), weights[nb], acc[nb][VCH * p + c]);
            }
          }
        }
        load_v(tw, now[y], na[y], nb_[y]);
        tw.there_a = na[y] >= 0, tw.there_b = nb_[y] >= 0;
      }
    };
    for (; wt < wt_end; wt += DEPTH * kWaves) process(wt);

    // --- the four waves' states, one column block at a time ---
    const bool whole = t0 == 0 && t1 == at.tiles;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (t0 == 0 ? 1 : 0);
    at.close(bt, a);
    // (0, 0) unless values were zeroed above: the keys that they may be of
    const bool fix = __syncthreads_or(spoilt);
    const int fix_lo = fix ? max(min_seen / TK * TK, t0 * KT) : 0;
    const int fix_hi = fix ? min(max_seen, t1 * KT) : 0;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float sum = sums[nb][0];
      if constexpr (is_f32<T>) {
        sum = (sums[nb][0] + sums[nb][1]) + (sums[nb][2] + sums[nb][3]);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
      }
      // (no key, or scores that are all -infinity; but NaN among masked ones counts)
      const float my_ref = limit[nb] == -INFINITY && sum == 0.f ? -INFINITY : ref[nb];
      __syncthreads();
      if (k == 0) {
        s_ref[wave][i] = my_ref;
        s_sum[wave][i] = sum;
      }
      __syncthreads();
      float top = s_ref[0][i];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_ref[w][i]);
      const float f = my_ref == -INFINITY ? 0.f : exp2f(my_ref - top);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NC; c += 4) {
          const int dim = VCH * (4 * k + r) + 16 * VCH * (c / VCH) + c % VCH;
          // a state that saw nothing holds zeros, and its factor is 0
          *reinterpret_cast<f32x4*>(&s_acc[wave][i][dim]) =
              f32x4{acc[nb][c][r], acc[nb][c + 1][r], acc[nb][c + 2][r], acc[nb][c + 3][r]} * f;
        }
      __syncthreads();
      int from = tid;                // (its rows and dimensions take registers only here)
      asm volatile("" : "+v"(from));
      if (__builtin_expect(fix, 0)) {
        // The zeroed values, times their weights, to the sums of the first wave.
#pragma unroll 1
        for (int e = from; e < 16 * D / 4; e += kThreads) {
          const int x = e / (D / 4), dim = e % (D / 4) * 4;
          const int in = nb * 16 + x;
          if (in >= in_tile) continue;
          float m = s_ref[0][x];
#pragma unroll
          for (int w = 1; w < kWaves; ++w) m = fmaxf(m, s_ref[w][x]);
          const int t = token_of(a, row0 + in), g = (row0 + in) - t * a.G;
          const int end = min(fix_hi, seen_by(bt, a, past, t));
#pragma unroll 1
          for (int key = fix_lo; key < end; ++key) {
            const int page = table[key >> bt.page_log2];
            if ((unsigned)page >= (unsigned)bt.n_pages) continue;
            const int at = key & page_mask;
            const char* block = bt.V + ((int64_t)page * bt.h_kv + head) * blk;
            float v[4];
            bool bad = false;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              v[y] = held<T, MX, D>(block, true, bt.page_log2, at, dim + y);
              bad |= !(fabsf(v[y]) < INFINITY);
            }
            if (!bad) continue;
            const float w =
                weight_of<T, MX, D>(bt, a, sr.start + t, head * a.G + g, head, page, at, m);
#pragma unroll
            for (int y = 0; y < 4; ++y)
              if (!(fabsf(v[y]) < INFINITY)) s_acc[0][x][dim + y] += w * v[y];
          }
        }
      }
#pragma unroll 1
      for (int e = from; e < 16 * D / 4; e += kThreads) {
        const int x = e / (D / 4), dim = e % (D / 4) * 4;
        const int in = nb * 16 + x;
        if (in >= in_tile) continue;
        float m = s_ref[0][x];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = fmaxf(m, s_ref[w][x]);
        float l = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float rw = s_ref[w][x];
          l += rw == -INFINITY ? 0.f : s_sum[w][x] * exp2f(rw - m);
          o += *reinterpret_cast<const f32x4*>(&s_acc[w][x][dim]);
        }
        const int t = token_of(a, row0 + in), g = (row0 + in) - t * a.G;
        if (whole) {
          o = l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o / l;
          T* dst = static_cast<T*>(a.out) +
                   ((int64_t)(sr.start + t) * a.h_q + head * a.G + g) * D + dim;
          if constexpr (is_f32<T>)
            *reinterpret_cast<f32x4*>(dst) = o;
          else
            *reinterpret_cast<u32x2*>(dst) = u32x2{pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
        } else {
          float* part = a.parts + (slot * R + in) * D + dim;
          float* ml = a.parts + (int64_t)2 * a.grid * R * D + (slot * R + in) * 2;
          if (NB == 1 && a.arrived) {
            store_part(part, o);
            if (dim == 0) store_part(ml, f32x2{m, l});
          } else {
            *reinterpret_cast<f32x4*>(part) = o;
            if (dim == 0) *reinterpret_cast<f32x2*>(ml) = f32x2{m, l};
          }
        }
      }
    }
    if constexpr (NB == 1)
      if (a.arrived && !whole) finish<T, D, R>(a, at);
  } while (at.next(bt, a));
}

// ---------------------------------------------------------------------------
// Attention of many query rows (chunks of prompts), 16-bit products.
//
// Where a KV head has more than 32 query rows the matrix cores are the bound,
// and what counts is how often a K or V value is fetched for a product.  Four
// waves share an item's key tiles of KT keys in LDS and take 32 query rows each:
//   S^T [KT x 32 rows] = K . Q^T,   O^T [D x 32 rows] += V^T . P^T
// on 32 x 32 x 16 products (layouts: lane = 0..63, i = lane % 32, k = lane / 32,
// A[i][8k..], B[8k..][i], and the result's component r is row
// 8*(r/4) + 4k + r%4 of column i).  As in the kernel above, the keys that the
// score product's rows stand for are chosen so that a lane ends up with the
// scores of the keys whose weights the second product wants from it:
// component r of score block s is key 32 s + 16 (r/8) + 8 k + r%8.
//
// Two waves bring in K, two V (turned on the way: V lies in LDS by dimensions,
// eight keys side by side); the next tile's loads are in flight during a tile's
// products, and the tiles alternate between two buffers: one barrier each.
// Chunks of 16 bytes are stored at their index XOR a function of the row, to
// spread the eight lanes of a 128-byte LDS access over the banks.  (Not all are:
// conflicts still take a fifth of LDS's busy cycles.)
// A key tile of 16-bit values is 32 KB: two workgroups fit a CU, and one's
// softmax overlaps the other's products.
// Measured: chunks of four prompts, 359 GFLOP, 547 us a call with the merge (657
// TFLOP/s; 535 to 565 by the card's clock; the matrix pipes are busy for 35 % of the
// cycles, the vector units for 43 %, LDS for 41 %).  64 rows a wave at one wave per
// SIMD halve the LDS reads and were 9 % slower to 9 % faster by shape (605 -> 624 us
// for these chunks, both before later steps); a tile's scores between the weights of
// the one before were 2 to 9 % slower.  Neither is taken.
// ---------------------------------------------------------------------------
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(f16x8 a, f16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

template <int D>
struct ChunkTile {
  static constexpr int KT = D == 256 ? 32 : 64;   // keys
  static constexpr int R = 32 * kWaves;           // query rows
};

template <class T, bool MX, int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void paged_chunk_kernel(Batch bt, AttnArgs a) {
  constexpr int KT = ChunkTile<D>::KT, R = ChunkTile<D>::R;
  constexpr int NS = KT / 32;                // score blocks
  constexpr int ND = D / 32;                 // output blocks
  constexpr int NQ = D / 16;                 // steps of a score product
  constexpr int NE = KT / 16;                // entries of the page table that a tile may span
  constexpr int RB = kRowBytes<T, MX, D>;
  constexpr int SB = D / 32;
  constexpr int KG = KT / 8;                 // groups of eight keys
  using V8 = typename Vec8<T>::type;

  __shared__ u32x4 s_k[2][KT][D / 8];        // [key][16-byte chunk]
  __shared__ u32x4 s_v[2][D][KG];            // [dimension][group of keys]

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int i = lane & 31, k = lane >> 5;

  Walk<R, KT, true> at;
  if (!at.template begin<T>(bt, a, lane, D)) return;
  const int64_t blk = block_bytes<T, MX, D>(bt.page_log2);
  const int page_mask = (1 << bt.page_log2) - 1;

  // Where chunks lie in LDS: K row r at chunk ^ k_turn(r), V row d at group ^
  // v_turn(d).
  auto k_turn = [](int r) { return (r & 3) | (r >> 1 & 4); };
  auto v_turn = [](int d) {
    return KG == 8 ? (d ^ d >> 3) & 7 : (d >> 1 ^ d >> 3) & 3;
  };
  // Reading: K row of score row i (of block 0), V row of output row i.
  const int k_row = 16 * (i >> 4) + 8 * (i >> 2 & 1) + 4 * (i >> 3 & 1) + (i & 3);

  do {
    const int b = at.b, head = at.head, past = at.past, t0 = at.t0, t1 = at.t1;
    const SeqRows sr = at.sr;
    const int row0 = at.rt * R;
    const int in_tile = min(sr.n * a.G - row0, R);
    const int min_seen = seen_by(bt, a, past, token_of(a, row0));
    const int max_seen = seen_by(bt, a, past, token_of(a, row0 + in_tile - 1));
    const int32_t* table = bt.pages + (int64_t)b * bt.max_pages;

    // This wave's rows.
    const int my_rows = min(max(in_tile - 32 * wave, 0), 32);
    const int my_row0 = row0 + 32 * wave;
    const int my_min = my_rows ? seen_by(bt, a, past, token_of(a, my_row0)) : 0;
    const int my_max = my_rows ? seen_by(bt, a, past, token_of(a, my_row0 + my_rows - 1)) : 0;
    const int t = token_of(a, my_row0 + min(i, max(my_rows - 1, 0)));
    const int g = my_row0 + min(i, max(my_rows - 1, 0)) - t * a.G;
    const int seen = i < my_rows ? seen_by(bt, a, past, t) : 0;
    u32x4 q[NQ];
    {
      const T* src = static_cast<const T*>(a.q) + (int64_t)(sr.start + t) * a.q_stride +
                     (int64_t)(head * a.G + g) * D + 8 * k;
#pragma unroll
      for (int w = 0; w < NQ; ++w)
        q[w] = my_rows ? (*reinterpret_cast<const u32x4*>(src + 16 * w) & a.q_keep) ^ a.q_flip
                       : u32x4{0u, 0u, 0u, 0u};
    }

    f32x16 acc[ND];
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[c][r] = 0.f;
    float limit = -INFINITY, ref = 0.f, sum = 0.f;
    bool spoilt = false, far = false;

    // --- staging: the loads of one tile, 128 bytes a thread of 16-bit values ---
    // Waves 0 and 1, K: unit u of a thread is chunk u % (row's chunks) of a row
    // (MX: a block of 32 dimensions).  Waves 2 and 3, V: one unit is eight keys
    // by eight dimensions.
    const int st = tid & 127;
    constexpr int kPer = MX ? D / 32 : D / 8;             // units of a K row
    constexpr int kUnits = KT * kPer / 128 ? KT * kPer / 128 : 1;
    constexpr int kStepRows = 128 / kPer;                 // rows between a thread's units
    constexpr int vChunks = D / 8;
    constexpr int vUnits = KG * vChunks / 128 ? KG * vChunks / 128 : 1;
    static_assert(vUnits == 1, "one V unit a thread");
    u32x4 raw[8];
    uint32_t raw_scale[2];
    int there = 0;                                        // bits: pages that are there
    int entry[NE];

    auto fetch_entries = [&](int key0) {
#pragma unroll
      for (int e = 0; e < NE; ++e)
        entry[e] = fixed(table + min((key0 + 16 * e) >> bt.page_log2, bt.max_pages - 1));
    };
    auto load_tile = [&](int key0) {
      int page[NE];
      there = 0;
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const bool ok = ((key0 + 16 * e) >> bt.page_log2) < bt.max_pages &&
                        (unsigned)entry[e] < (unsigned)bt.n_pages;
        page[e] = ok ? entry[e] : 0;
        there |= ok << e;
      }
      // offset of the page block, and slot, of 16 keys
      auto block_at = [&](int e, const char* pool) {
        return pool + ((int64_t)page[e] * bt.h_kv + head) * blk;
      };
      auto slot_at = [&](int e) { return (key0 + 16 * e) & page_mask; };
      if (wave < 2) {
#pragma unroll
        for (int n = 0; n < kUnits; ++n) {
          const int r = st / kPer + kStepRows * n;        // row in the tile
          const int u = st % kPer;
          const char* block = block_at(0, bt.K);
          int slot = slot_at(0);
#pragma unroll
          for (int e = 1; e < NE; ++e)
            if (r >> 4 == e) block = block_at(e, bt.K), slot = slot_at(e);
          slot += r & 15;
          if constexpr (MX) {
            raw[n] = *reinterpret_cast<const u32x4*>(block + (int64_t)slot * RB + 16 * u);
            raw_scale[n] = *reinterpret_cast<const uint8_t*>(
                block + ((int64_t)RB << bt.page_log2) + slot * SB + u);
          } else {
            raw[n] = *reinterpret_cast<const u32x4*>(block + (int64_t)slot * RB + 16 * u);
          }
        }
      } else if (st < KG * vChunks) {
        const int grp = st / vChunks, c = st % vChunks;   // keys 8 grp .., dimensions 8 c ..
        const char* block = block_at(0, bt.V);
        int slot = slot_at(0);
#pragma unroll
        for (int e = 1; e < NE; ++e)
          if (grp >> 1 == e) block = block_at(e, bt.V), slot = slot_at(e);
        slot += 8 * (grp & 1);
        if constexpr (MX) {
          raw[0] = *reinterpret_cast<const u32x4*>(block + (int64_t)slot * RB + 32 * c);
          raw[1] = *reinterpret_cast<const u32x4*>(block + (int64_t)slot * RB + 32 * c + 16);
          const u32x2 s = *reinterpret_cast<const u32x2*>(
              block + ((int64_t)RB << bt.page_log2) + slot * SB + 8 * (c / 4));
          raw_scale[0] = s[0], raw_scale[1] = s[1];
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            raw[j] = *reinterpret_cast<const u32x4*>(block + (int64_t)(slot + j) * RB + 16 * c);
        }
      }
    };
    auto store_tile = [&](int key0, int buf) {
      if (wave < 2) {
#pragma unroll
        for (int n = 0; n < kUnits; ++n) {
          const int r = st / kPer + kStepRows * n;
          const int u = st % kPer;
          if constexpr (MX) {
            const float scale = mx_scale(raw_scale[n]);
#pragma unroll
            for (int w = 0; w < 4; ++w)
              s_k[buf][r][(4 * u + w) ^ k_turn(r)] =
                  u32x4{widen2<T, 0>(raw[n][w], scale), widen2<T, 1>(raw[n][w], scale),
                        widen2<T, 2>(raw[n][w], scale), widen2<T, 3>(raw[n][w], scale)};
          } else {
            s_k[buf][r][u ^ k_turn(r)] = raw[n];
          }
        }
      } else if (st < KG * vChunks) {
        const int grp = st / vChunks, c = st % vChunks;
        const int first = key0 + 8 * grp;
        u32x4 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if constexpr (MX) {
            const float scale = mx_scale_of(raw_scale[j / 4], j);
            const uint32_t codes = raw[j / 4][j % 4];
            x[j] = u32x4{widen2<T, 0>(codes, scale), widen2<T, 1>(codes, scale),
                         widen2<T, 2>(codes, scale), widen2<T, 3>(codes, scale)};
          } else {
            x[j] = raw[j];
          }
        }
        // Keys that no row sees are left out; where only some rows see a tile's
        // keys, what a weight of 0 does not take out is zeroed here and added at
        // the end to the rows that see it.
        const bool here = there >> (grp >> 1) & 1;
        if (key0 + KT > min_seen || there != (1 << NE) - 1) {
          const bool some = min_seen < max_seen && key0 + KT > min_seen;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool keep = here && first + j < max_seen;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              if (!keep) x[j][w] = 0u;
              if (some) {
                spoilt |= not_finite<T>(x[j][w]);
                x[j][w] = finite_part<T>(x[j][w]);
              }
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t sel = e % 2 ? 0x07060302u : 0x05040100u;
          const int d = 8 * c + e;
          s_v[buf][d][grp ^ v_turn(d)] =
              u32x4{__builtin_amdgcn_perm(x[1][e / 2], x[0][e / 2], sel),
                    __builtin_amdgcn_perm(x[3][e / 2], x[2][e / 2], sel),
                    __builtin_amdgcn_perm(x[5][e / 2], x[4][e / 2], sel),
                    __builtin_amdgcn_perm(x[7][e / 2], x[6][e / 2], sel)};
        }
      }
    };

    fetch_entries(t0 * KT);
    load_tile(t0 * KT);
    fetch_entries(min(t0 + 1, t1 - 1) * KT);
    __syncthreads();                         // the buffers are free (the last item's reads)
    int pages_here = there;                  // of the tile whose products are next
    store_tile(t0 * KT, 0);
    __syncthreads();

    for (int tile = t0; tile < t1; ++tile) {
      const int key0 = tile * KT, buf = (tile - t0) & 1;
      const bool more = tile + 1 < t1;
      if (more) {
        load_tile(key0 + KT);
        fetch_entries(min(tile + 2, t1 - 1) * KT);
      }
      if (key0 < my_max) {
        // --- scores ---
        f32x16 s[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[n][r] = 0.f;
#pragma unroll
        for (int w = 0; w < NQ; ++w)
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            const u32x4 x = s_k[buf][k_row + 32 * n][(2 * w + k) ^ k_turn(k_row)];
            s[n] = mma32(__builtin_bit_cast(V8, x), __builtin_bit_cast(V8, q[w]), s[n]);
          }
        if (key0 + KT > my_min || pages_here != (1 << NE) - 1) {
#pragma unroll
          for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (!((pages_here >> (2 * n + r / 8) & 1) &&
                    key0 + 32 * n + 16 * (r / 8) + 8 * k + r % 8 < seen))
                s[n][r] = -INFINITY;
        }
        // --- softmax, the reference raised as in the kernel above ---
        float top = s[0][0];
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) top = fmaxf(top, s[n][r]);
        top *= a.scale;
        if (__any(!(top <= limit))) {
          top = fmaxf(top, __shfl_xor(top, 32));
          far |= __any(is_far(top));
          if (!(top <= limit)) {
            const float f = limit == -INFINITY ? 0.f : exp2f(ref - top);
            ref = top;
            limit = top + 8.f;
            sum *= f;
#pragma unroll
            for (int c = 0; c < ND; ++c) acc[c] *= f;
          }
        }
        float by = a.scale;
        if (__builtin_expect(far, 0)) {
          by = 1.f;
#pragma unroll
          for (int n = 0; n < NS; ++n) s[n] *= a.scale;
        }
        u32x4 p[2 * NS];
#pragma unroll
        for (int n = 0; n < NS; ++n) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            s[n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r], by, -ref));
          // the sum of the weights as they are multiplied: rounded to T
          float part = 0.f;
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
            const uint32_t w = pack2<T>(s[n][r], s[n][r + 1]);
            p[2 * n + r / 8][r % 8 / 2] = w;
            part = add2<T>(w, part);
          }
          sum += part;
        }
        // --- O^T += V^T P^T ---
#pragma unroll
        for (int c = 0; c < ND; ++c)
#pragma unroll
          for (int n = 0; n < 2 * NS; ++n) {
            const int d = 32 * c + i;
            const u32x4 x = s_v[buf][d][(2 * n + k) ^ v_turn(d)];
            acc[c] = mma32(__builtin_bit_cast(V8, x), __builtin_bit_cast(V8, p[n]), acc[c]);
          }
      }
      if (more) {
        pages_here = there;
        store_tile(key0 + KT, buf ^ 1);
      }
      __syncthreads();
    }

    // --- each wave's rows are its own: out, or the workgroup's slot ---
    at.close(bt, a);
    const bool fix = __syncthreads_or(spoilt);
    sum += __shfl_xor(sum, 32);
    if (i < my_rows) {
      const int fix_hi = fix ? min(min(max_seen, t1 * KT), seen) : 0;
      for (int key = max(min_seen / KT, t0) * KT; key < fix_hi; ++key) {
        const int id = table[key >> bt.page_log2];
        if ((unsigned)id >= (unsigned)bt.n_pages) continue;
        const int slot = key & page_mask;
        const char* block = bt.V + ((int64_t)id * bt.h_kv + head) * blk;
        auto value = [&](int c, int r) {
          return held<T, MX, D>(block, true, bt.page_log2, slot, 32 * c + 8 * (r / 4) + 4 * k + r % 4);
        };
        bool bad = false;
#pragma unroll
        for (int c = 0; c < ND; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r) bad |= !(fabsf(value(c, r)) < INFINITY);
        if (!bad) continue;
        const float w =
            weight_of<T, MX, D>(bt, a, sr.start + t, head * a.G + g, head, id, slot, ref);
#pragma unroll
        for (int c = 0; c < ND; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float v = value(c, r);
            if (!(fabsf(v) < INFINITY)) acc[c][r] += w * v;
          }
      }
      const float my_ref = limit == -INFINITY && sum == 0.f ? -INFINITY : ref;
      if (t0 == 0 && t1 == at.tiles) {
        // (scores that are all -infinity: 0, also where V is not finite)
        const float inverse = 1.f / sum;
        auto mean = [&](float x) { return sum == 0.f ? 0.f : x * inverse; };
        T* dst = static_cast<T*>(a.out) +
                 ((int64_t)(sr.start + t) * a.h_q + head * a.G + g) * D + 4 * k;
#pragma unroll
        for (int c = 0; c < ND; ++c)
#pragma unroll
          for (int r = 0; r < 16; r += 4)
            *reinterpret_cast<u32x2*>(dst + 32 * c + 2 * r) =
                u32x2{pack2<T>(mean(acc[c][r]), mean(acc[c][r + 1])),
                      pack2<T>(mean(acc[c][r + 2]), mean(acc[c][r + 3]))};
      } else {
        const int64_t slot = 2 * (int64_t)blockIdx.x + (t0 == 0 ? 1 : 0);
        const int64_t row = slot * R + 32 * wave + i;
        float* dst = a.parts + row * D + 4 * k;
#pragma unroll
        for (int c = 0; c < ND; ++c)
#pragma unroll
          for (int r = 0; r < 16; r += 4)
            *reinterpret_cast<f32x4*>(dst + 32 * c + 2 * r) =
                f32x4{acc[c][r], acc[c][r + 1], acc[c][r + 2], acc[c][r + 3]};
        if (k == 0)
          *reinterpret_cast<f32x2*>(a.parts + (int64_t)2 * a.grid * R * D + row * 2) =
              f32x2{my_ref, sum};
      }
    }
  } while (at.next(bt, a));
}

// Puts the parts of item closing[blockIdx.x] together, rows shared out over
// blockIdx.y.  Few parts: D/4 lanes take a row.  Many: the waves share a row's
// parts.  What bounds it: 5 us after decode steps, of which loads that wait for each
// other are most; after chunks of four prompts 41 us, 67 MB of parts at 1.6 TB/s
// (each part 66 KB, two a workgroup; a row a wave, by 8 bytes a lane, took 48).
constexpr int kMergeWaves = 8;
constexpr int merge_rows(int d) { return kMergeWaves * 256 / d; }    // rows at once, of few parts

template <class T, int D, int R>
__global__ __launch_bounds__(64 * kMergeWaves) void paged_merge_kernel(AttnArgs a) {
  constexpr int kVec = D / 64;
  __shared__ float s_part[kMergeWaves][D], s_m[kMergeWaves], s_l[kMergeWaves];
  const Closing item = a.closing[blockIdx.x];
  if (item.first < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int n = item.last - item.first + 1;
  const float* ml = a.parts + (int64_t)2 * a.grid * R * D;

  // Parts from, from + step, .. of a row, o.size() dimensions from col on, the
  // loads of Y parts in flight at once.
  float m, l;
  auto combine = [&](auto& o, auto Y, int row, int col, int from, int step) {
    constexpr int kOut = sizeof(o) / sizeof(float);
    typedef float vec __attribute__((ext_vector_type(kOut)));
    m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < kOut; ++e) o[e] = 0.f;
    for (int p0 = from; p0 < n; p0 += Y * step) {
      f32x2 s[Y];
      vec v[Y];
#pragma unroll
      for (int y = 0; y < Y; ++y) {
        const int p = min(p0 + y * step, n - 1);
        const int64_t at = (int64_t)(2 * (item.first + p) + (p == 0)) * R + row;
        s[y] = *reinterpret_cast<const f32x2*>(ml + at * 2);
        v[y] = *reinterpret_cast<const vec*>(a.parts + at * D + col);
      }
#pragma unroll
      for (int y = 0; y < Y; ++y) {
        if (p0 + y * step >= n) continue;
        const float mn = s[y][0] <= m ? m : s[y][0];                 // (a NaN stays)
        const float base = mn == -INFINITY ? 0.f : mn;               // (then both factors are 0)
        const float fo = exp2f(m - base), fn = exp2f(s[y][0] - base);
        l = l * fo + s[y][1] * fn;
#pragma unroll
        for (int e = 0; e < kOut; ++e) o[e] = o[e] * fo + v[y][e] * fn;
        m = mn;
      }
    }
  };
  auto out_at = [&](int row) {
    const int t = token_of(a, item.row0 + row), g = (item.row0 + row) - t * a.G;
    return static_cast<T*>(a.out) + ((int64_t)(item.start + t) * a.h_q + item.head * a.G + g) * D;
  };

  if (n <= 2 * kMergeWaves) {
    // D / 4 lanes a row, so one, two or four rows a wave
    constexpr int kLanes = D / 4, kRows = merge_rows(D);
    const int col = lane % kLanes * 4;
    for (int first = blockIdx.y * kRows; first < item.in_tile; first += gridDim.y * kRows) {
      const int row = first + wave * (64 / kLanes) + lane / kLanes;
      const int held = min(row, item.in_tile - 1);
      float o[4];
      if (n == 2)
        combine(o, std::integral_constant<int, 2>{}, held, col, 0, 1);
      else
        combine(o, std::integral_constant<int, 4>{}, held, col, 0, 1);
      if (row >= item.in_tile) continue;
      typedef T t4 __attribute__((ext_vector_type(4)));
      t4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = (T)(l == 0.f ? 0.f : o[e] / l);
      *reinterpret_cast<t4*>(out_at(row) + col) = y;
    }
    return;
  }
  float o[kVec];
  for (int row = blockIdx.y; row < item.in_tile; row += gridDim.y) {
    combine(o, std::integral_constant<int, 4>{}, row, lane * kVec, wave, kMergeWaves);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kVec; ++e) s_part[wave][lane * kVec + e] = o[e];
    if (lane == 0) s_m[wave] = m, s_l[wave] = l;
    __syncthreads();
    if (tid < D) {
      float top = s_m[0];
#pragma unroll
      for (int w = 1; w < kMergeWaves; ++w) top = fmaxf(top, s_m[w]);
      float sum = 0.f, y = 0.f;
#pragma unroll
      for (int w = 0; w < kMergeWaves; ++w) {
        const float f = s_m[w] == -INFINITY ? 0.f : exp2f(s_m[w] - top);
        sum += s_l[w] * f;
        y += s_part[w][tid] * f;
      }
      out_at(row)[tid] = (T)(sum == 0.f ? 0.f : y / sum);
    }
  }
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool dim_ok(int d) { return d == 64 || d == 128 || d == 256; }
bool type_ok(int dtype) { return dtype >= DA_F32 && dtype <= DA_F16; }
int type_bytes(int dtype) { return dtype == DA_F32 ? 4 : 2; }

constexpr int kMaxPageRows = 32768;
constexpr int64_t kMaxPositions = int64_t(1) << 30;
constexpr int kMaxRowsPerSeq = 32768;
constexpr int64_t kMaxItems = int64_t(1) << 24;   // sequences x query heads
constexpr int64_t kMaxGroups = (int64_t(1) << 24) - 1;  // of 256 threads: a grid has < 2^32

// Compute units of the current device, at most kMaxCus, queried once per
// device.  Without a device (the call can then only fail at launch) kMaxCus.
constexpr int kMaxDevices = 64;
std::atomic<int> g_cus[kMaxDevices];

int device_cus() {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) {
    (void)hipGetLastError();
    return kMaxCus;
  }
  int c = g_cus[dev].load(std::memory_order_relaxed);
  if (c == 0) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
        n < 1) {
      (void)hipGetLastError();
      return kMaxCus;
    }
    c = std::min(n, kMaxCus);
    g_cus[dev].store(c, std::memory_order_relaxed);
  }
  return c;
}

da_status launch_status() { return hipGetLastError() == hipSuccess ? DA_OK : DA_ERR_HIP; }

// Everything about the batch but NULL pointers of the arrays: shapes, then
// what is supported.
da_status check_batch(const da_paged_kv& p) {
  if (p.B < 1 || p.h_kv < 1 || p.d < 1 || p.n_pages < 1 || p.page_rows < 1 || p.max_pages < 1 ||
      p.rows < 1 || p.T < 1)
    return DA_ERR_SHAPE;
  if ((int64_t)p.page_rows * p.max_pages > kMaxPositions || p.T > kMaxRowsPerSeq ||
      (int64_t)p.B * p.h_kv > kMaxItems)
    return DA_ERR_SHAPE;
  if (!p.row_start && (int64_t)p.B * p.T != p.rows) return DA_ERR_SHAPE;
  if (!dim_ok(p.d) || !type_ok(p.dtype) ||
      (p.format != DA_KV_DENSE && p.format != DA_KV_MX4) || p.page_rows < 16 ||
      p.page_rows > kMaxPageRows || (p.page_rows & (p.page_rows - 1)) != 0)
    return DA_ERR_UNSUPPORTED;
  return DA_OK;
}

bool batch_aligned(const da_paged_kv& p) {
  return aligned(p.K, 16) && aligned(p.V, 16) && aligned(p.pages, 4) && aligned(p.past, 4) &&
         aligned(p.row_start, 4);
}

Batch device_batch(const da_paged_kv& p) {
  int log2 = 0;
  while ((1 << log2) < p.page_rows) ++log2;
  return {static_cast<char*>(p.K), static_cast<char*>(p.V), p.pages, p.past, p.row_start, p.B,
          p.h_kv, p.n_pages, log2, p.max_pages, p.rows, p.T};
}

// Calls f(type tag, mx, d) with the batch's as compile-time constants.
template <class T>
struct Tag {
  using type = T;
};
template <bool MX, int D, class F>
void with_type(int dtype, F&& f) {
  if (dtype == DA_F32)
    f(Tag<float>{}, std::bool_constant<MX>{}, std::integral_constant<int, D>{});
  else if (dtype == DA_BF16)
    f(Tag<__bf16>{}, std::bool_constant<MX>{}, std::integral_constant<int, D>{});
  else
    f(Tag<_Float16>{}, std::bool_constant<MX>{}, std::integral_constant<int, D>{});
}
template <bool MX, class F>
void with_dim(int dtype, int d, F&& f) {
  if (d == 64)
    with_type<MX, 64>(dtype, f);
  else if (d == 128)
    with_type<MX, 128>(dtype, f);
  else
    with_type<MX, 256>(dtype, f);
}
template <class F>
void dispatch(const da_paged_kv& p, F&& f) {
  if (p.format == DA_KV_MX4)
    with_dim<true>(p.dtype, p.d, f);
  else
    with_dim<false>(p.dtype, p.d, f);
}

// Query rows of a row tile: 16 for one column block, 32 for two; more than 32
// per KV head of a 16-bit type go to the chunk kernel's tiles of 128.
constexpr int kChunkRows = 32 * kWaves;
int tile_rows(int64_t rows_per_head, int dtype) {
  return rows_per_head <= 16 ? 16 : rows_per_head <= 32 || dtype == DA_F32 ? 32 : kChunkRows;
}

constexpr int kGroupsPerCu = 2;       // workgroups of the attention kernel per CU

constexpr size_t kArrivedBytes = kMaxCus * kGroupsPerCu * sizeof(unsigned);
constexpr size_t kClosingBytes = kMaxCus * kGroupsPerCu * sizeof(Closing);

struct AttnPlan {
  int R;
  size_t bytes;
};

da_status plan_attn(int B, int h_q, int h_kv, int d, int T, int dtype, AttnPlan* plan) {
  if (B < 1 || h_q < 1 || h_kv < 1 || d < 1 || T < 1 || T > kMaxRowsPerSeq || h_q % h_kv != 0 ||
      (int64_t)B * h_q > kMaxItems || (int64_t)h_q * T > (int64_t(1) << 30))
    return DA_ERR_SHAPE;
  if (!dim_ok(d) || !type_ok(dtype)) return DA_ERR_UNSUPPORTED;
  const int64_t per_head = (int64_t)(h_q / h_kv) * T;
  plan->R = tile_rows(per_head, dtype);
  const size_t slots = 2 * kMaxCus * kGroupsPerCu;
  plan->bytes = kArrivedBytes + kClosingBytes + slots * plan->R * ((size_t)d + 2) * sizeof(float);
  return DA_OK;
}

template <class T, int D, int R>
void launch_merge(const Batch& bt, const AttnArgs& a, hipStream_t s) {
  if (a.arrived) return;
  // A row a wave; few items have rows of many parts, and a workgroup for each.
  const int rows = (int)std::min<int64_t>((int64_t)a.G * bt.T, R);
  const int items = a.by_item ? bt.B * bt.h_kv : a.grid;
  const bool many = (int64_t)bt.B * bt.h_kv * kMergeWaves < a.grid;
  const unsigned split = (unsigned)ceil_div(rows, many ? 1 : merge_rows(D));
  hipLaunchKernelGGL((paged_merge_kernel<T, D, R>), dim3((unsigned)items, split),
                     dim3(64 * kMergeWaves), 0, s, a);
}

template <class T, bool MX, int D>
void launch_attn(int R, const Batch& bt, const AttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.grid), block(kThreads);
  if (R == 16) {
    hipLaunchKernelGGL((paged_attn_kernel<T, MX, D, 1>), grid, block, 0, s, bt, a);
    launch_merge<T, D, 16>(bt, a, s);
  } else if (R == 32) {
    hipLaunchKernelGGL((paged_attn_kernel<T, MX, D, 2>), grid, block, 0, s, bt, a);
    launch_merge<T, D, 32>(bt, a, s);
  } else if constexpr (!is_f32<T>) {
    hipLaunchKernelGGL((paged_chunk_kernel<T, MX, D>), grid, block, 0, s, bt, a);
    launch_merge<T, D, kChunkRows>(bt, a, s);
  }
}

}  // namespace

extern "C" {

size_t da_paged_page_bytes(int page_rows, int d, int dtype, int format) {
  if (page_rows < 16 || page_rows > kMaxPageRows || (page_rows & (page_rows - 1)) != 0 ||
      !dim_ok(d) || !type_ok(dtype))
    return 0;
  if (format == DA_KV_MX4) return (size_t)page_rows * (d / 2 + d / 32);
  return format == DA_KV_DENSE ? (size_t)page_rows * d * type_bytes(dtype) : 0;
}

da_status da_paged_append(const da_paged_kv* kv, const void* k_new, const void* v_new,
                          int64_t k_stride, int64_t v_stride, const void* q, int64_t q_stride,
                          int h_q, void* q_out, const float* rotary, int n_rotary, int rot_dim,
                          int interleaved, void* stream) {
  if (!kv || !k_new || !v_new || !kv->K || !kv->V || !kv->pages || !kv->past ||
      (q && !q_out) || (rot_dim != 0 && !rotary))
    return DA_ERR_NULL;
  const da_paged_kv& p = *kv;
  da_status st = check_batch(p);
  if (st != DA_OK && st != DA_ERR_UNSUPPORTED) return st;
  if (!q) h_q = 0;
  if (h_q < 0 || (q && h_q < 1) || (int64_t)h_q * p.d > (1 << 30) || rot_dim < 0 ||
      rot_dim > p.d || (rot_dim != 0 && n_rotary < (int64_t)p.page_rows * p.max_pages) ||
      k_stride < (int64_t)p.h_kv * p.d || v_stride < (int64_t)p.h_kv * p.d ||
      (q && q_stride < (int64_t)h_q * p.d))
    return DA_ERR_SHAPE;
  if (st != DA_OK || rot_dim % 16 != 0) return DA_ERR_UNSUPPORTED;
  const int per16 = 16 / type_bytes(p.dtype);
  if (!batch_aligned(p) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(q, 16) ||
      !aligned(q_out, 16) || !aligned(rotary, 16) || k_stride % per16 || v_stride % per16 ||
      (q && q_stride % per16))
    return DA_ERR_ALIGN;
  const AppendArgs a{q,        k_new,    v_new,  q_out, q_stride, k_stride,
                     v_stride, rotary, h_q, rot_dim, interleaved};
  const Batch bt = device_batch(p);
  const int64_t units =
      (int64_t)p.T * ((int64_t)h_q * (p.d / 16) +
                      2 * (int64_t)p.h_kv * (p.d / (p.format == DA_KV_MX4 ? 8 : 16)));
  const int64_t groups = ceil_div(units, kThreads);
  if (groups > kMaxGroups || groups * p.B > kMaxGroups) return DA_ERR_SHAPE;
  (void)hipGetLastError();
  dispatch(p, [&](auto t, auto mx, auto d) {
    hipLaunchKernelGGL((paged_append_kernel<typename decltype(t)::type, mx.value, d.value>),
                       dim3((unsigned)(groups * p.B)), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), bt, a, (unsigned)groups);
  });
  return launch_status();
}

da_status da_paged_gather(const da_paged_kv* kv, void* k_out, void* v_out, void* stream) {
  if (!kv || !k_out || !v_out || !kv->K || !kv->V || !kv->pages || !kv->past) return DA_ERR_NULL;
  const da_paged_kv& p = *kv;
  const da_status st = check_batch(p);
  if (st != DA_OK) return st;
  if (!batch_aligned(p) || !aligned(k_out, 16) || !aligned(v_out, 16)) return DA_ERR_ALIGN;
  const Batch bt = device_batch(p);
  const int64_t groups = ceil_div((int64_t)p.T * 2 * p.h_kv * (p.d / 8), kThreads);
  if (groups > kMaxGroups || groups * p.B > kMaxGroups) return DA_ERR_SHAPE;
  (void)hipGetLastError();
  dispatch(p, [&](auto t, auto mx, auto d) {
    hipLaunchKernelGGL((paged_gather_kernel<typename decltype(t)::type, mx.value, d.value>),
                       dim3((unsigned)(groups * p.B)), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), bt, k_out, v_out, (unsigned)groups);
  });
  return launch_status();
}

size_t da_paged_workspace_bytes(int B, int h_q, int h_kv, int d, int T, int dtype) {
  AttnPlan plan;
  return plan_attn(B, h_q, h_kv, d, T, dtype, &plan) == DA_OK ? plan.bytes : 0;
}

size_t da_paged_workspace_counter_bytes(int B, int h_q, int h_kv, int d, int T, int dtype) {
  AttnPlan plan;
  return plan_attn(B, h_q, h_kv, d, T, dtype, &plan) == DA_OK ? kArrivedBytes : 0;
}

da_status da_paged_attn(const da_paged_kv* kv, const void* q, int64_t q_stride, int h_q,
                        float scale, int causal, void* out, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (!kv || !q || !out || !kv->K || !kv->V || !kv->pages || !kv->past) return DA_ERR_NULL;
  const da_paged_kv& p = *kv;
  da_status st = check_batch(p);
  if (st != DA_OK && st != DA_ERR_UNSUPPORTED) return st;
  AttnPlan plan;
  const da_status sp = plan_attn(p.B, h_q, p.h_kv, p.d, p.T, p.dtype, &plan);
  if (sp == DA_ERR_SHAPE || q_stride < (int64_t)h_q * p.d) return DA_ERR_SHAPE;
  if (st != DA_OK || sp != DA_OK) return DA_ERR_UNSUPPORTED;
  if (!batch_aligned(p) || !aligned(q, 16) || !aligned(out, 16) ||
      q_stride % (16 / type_bytes(p.dtype)))
    return DA_ERR_ALIGN;
  if (!std::isfinite(scale)) return DA_ERR_SCALE;
  if (!workspace || workspace_bytes < plan.bytes) return DA_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return DA_ERR_ALIGN;
  const Batch bt = device_batch(p);
  const int grid = device_cus() * kGroupsPerCu;
  const int64_t row_tiles = ceil_div((int64_t)(h_q / p.h_kv) * p.T, plan.R);
  const int64_t most_tiles = ceil_div((int64_t)p.max_pages * p.page_rows, 32) + kItemCost;
  const int few_tiles = (double)p.B * p.h_kv * row_tiles * most_tiles < 2e9;
  // Items of few rows and few parts are put together by the workgroups that have
  // them: one launch for two (one sequence of 700 rows 10.6 -> 9.5 us, 16 of
  // 200-4000 30.8 -> 30.0; but with tiles of 32 rows 52.6 -> 56.6, of 128 rows
  // 23.3 -> 26.4, where the last workgroup has too much to read).
  const bool few_parts =
      plan.R == 16 && (ceil_div((int64_t)p.max_pages * p.page_rows, 64) <= 16 ||
                       4 * (int64_t)p.B * p.h_kv >= grid);
  char* ws = static_cast<char*>(workspace);
  const uint32_t G = h_q / p.h_kv;
  uint32_t G_shift = 31;
  while (G > 1u << (G_shift - 31)) ++G_shift;
  const uint32_t G_mul = (uint32_t)((uint64_t(1) << G_shift) / G + 1);
  const int by_item = row_tiles == 1 && (int64_t)p.B * p.h_kv <= grid && p.h_kv <= kThreads;
  const AttnArgs a{q,
                   out,
                   q_stride,
                   scale == 0.f ? 1.f : std::min(std::fabs(scale) * kLog2e, FLT_MAX),
                   scale == 0.f ? 0u : ~0u,
                   scale < 0.f ? (p.dtype == DA_F32 ? 0x80000000u : 0x80008000u) : 0u,
                   h_q,
                   h_q / p.h_kv,
                   causal,
                   G_mul,
                   G_shift,
                   few_tiles,
                   few_parts ? reinterpret_cast<unsigned*>(ws) : nullptr,
                   by_item,
                   reinterpret_cast<Closing*>(ws + kArrivedBytes),
                   reinterpret_cast<float*>(ws + kArrivedBytes + kClosingBytes),
                   grid};
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  dispatch(p, [&](auto t, auto mx, auto d) {
    launch_attn<typename decltype(t)::type, mx.value, d.value>(plan.R, bt, a, s);
  });
  return launch_status();
}

}  // extern "C"
