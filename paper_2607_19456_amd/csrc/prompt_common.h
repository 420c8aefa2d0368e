// prompt_common.h -- what the kernels of prompt attention and of its gradient
// share: the batch of packed sequences, the tiles of rows, the matrix
// instructions and the layout of tiles in LDS.
//
// Register layouts of the 32 x 32 matrix instructions (lane = 0..63, i = lane % 32,
// k = lane / 32):
//   A operand: lane holds A[i][..], k's share of the summed index
//   B operand: lane holds B[..][i], k's share of the summed index
//   result:    component r of a lane is D[8*(r/4) + 4*k + r%4][i]
// The summed index is shared out 8 to a lane (16-bit types, 16 in all) or 1
// (float32, 2 in all).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "decode_attn.h"

// (Of parts of a kernel that hold its sums: called, they would have them in memory.)
#define INLINE __attribute__((always_inline))

namespace prompt {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kCus = 256;             // what grids and workspaces are planned for

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <class T>
constexpr bool is_f32 = std::is_same<T, float>::value;

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// ---------------------------------------------------------------------------
// The batch.
// ---------------------------------------------------------------------------
struct Batch {
  const int32_t *row_start, *key_start;
  int B, rows, keys, T, N;
  int h_q, h_kv, G, causal;
  uint32_t G_mul, G_shift;
};

// First row (or key) and number of them of sequence b, within the arrays
// whatever the starts hold.
struct Span {
  int start, n;
};
__device__ __forceinline__ Span span(const int32_t* start, int b, int most, int total) {
  if (!start) return {b * most, most};
  const int s = min(max(start[b], 0), total);
  const int e = min(max(start[b + 1], s), total);
  return {s, min(e - s, most)};
}

// x / G, 0 <= x < 2^31 (the host's multiplier: floor(2^shift / G) + 1).
__device__ __forceinline__ int token_of(const Batch& bt, int x) {
  return (int)((uint64_t)(uint32_t)x * bt.G_mul >> bt.G_shift);
}

// Keys that row t of a sequence of `rows` rows and `keys` keys sees.
__device__ __forceinline__ int seen_by(const Batch& bt, int rows, int keys, int t) {
  return bt.causal ? min(max(t + 1 + keys - rows, 0), keys) : keys;
}

// Item `item` of the batch, items being tiles of R of each sequence's rows (times
// G), or of its keys: its sequence's rows and keys, and how many more tiles follow it
// there.  False where there is none.  Items are in the order of that number, the largest
// first: where a causal mask gives a tile work in proportion to it, the most work comes
// first, whatever the sequences' lengths.  (Workgroups start in their order, each
// shader engine's in turn: one that must wait for a busy engine holds up all behind
// it, and with the sequences one after the other a batch of four ran 1.7 times as long
// as its work.)
// So within each block of 64 sequences, a lane each.  The blocks' items begin at
// start * G / R + b, which leaves room for all before (a sequence's last tile may be
// partly empty), so no sequence is counted but the block's own: 4096 sequences of 64
// rows: 1483 us (32/8 heads of 128), 5976 when each workgroup counted them all.
struct Place {
  Span rows, keys;
  int after, tiles;
};
__device__ __forceinline__ int wave_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast:31
  return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ bool find(const Batch& bt, bool by_rows, int R, int item, int lane,
                                     Place* at) {
  const int64_t per = by_rows ? bt.G : 1;
  if (bt.B == 1) {
    const Span r1 = span(bt.row_start, 0, bt.T, bt.rows), k1 = span(bt.key_start, 0, bt.N, bt.keys);
    const int tiles = uniform((int)(((by_rows ? r1.n : k1.n) * per + R - 1) / R));
    *at = {{uniform(r1.start), uniform(r1.n)}, {uniform(k1.start), uniform(k1.n)},
           tiles - 1 - item, tiles};
    return item < tiles;
  }
  // The last block of sequences whose first place is not beyond `item`: 64 of them are
  // looked at in a step.
  const int32_t* start = by_rows ? bt.row_start : bt.key_start;
  const int most = by_rows ? bt.T : bt.N;
  const int64_t even = (most * per + R - 1) / R;
  auto first_of = [&](int block) INLINE {
    const int64_t b = int64_t(64) * block;
    if (!start) return b * even;
    const int s = min(max(start[b], 0), by_rows ? bt.rows : bt.keys);
    return std::min(s * per / R + b, b * even);
  };
  int block = 0, left = item;
  for (int n = (bt.B + 63) / 64; n > 1;) {
    const int step = (n + 63) / 64, x = min(lane * step, n - 1);
    const int64_t first = first_of(block + x);
    const bool before = lane * step < n && first <= item;
    const uint64_t beyond = ~__ballot(before);
    const int steps = beyond ? max(__ffsll((unsigned long long)beyond) - 2, 0) : 63;
    left = item - __builtin_amdgcn_readlane((int)first, steps);
    block += steps * step;
    n = min(step, n - steps * step);
  }
  // a sequence of the block to a lane
  Span r{0, 0}, k{0, 0};
  if (64 * block + lane < bt.B) {
    r = span(bt.row_start, 64 * block + lane, bt.T, bt.rows);
    k = span(bt.key_start, 64 * block + lane, bt.N, bt.keys);
  }
  const int n = (int)(((by_rows ? r.n : k.n) * per + R - 1) / R);
  if (left >= wave_sum(n)) return false;
  // the least m for which no more than `left` items, those with more than m tiles after
  // them, come before its own
  auto before = [&](int m) INLINE { return wave_sum(max(n - 1 - m, 0)); };
  int lo = 0, hi = (int)even - 1;
  while (lo < hi) {
    const int m = (lo + hi) >> 1;
    if (before(m) <= left)
      hi = m;
    else
      lo = m + 1;
  }
  left -= before(lo);
  // the left-th of the sequences with more than m tiles
  const uint64_t has = __ballot(n > lo);
  const bool me = n > lo && (int)__popcll(has & ((uint64_t(1) << lane) - 1)) == left;
  const int l = __ffsll((unsigned long long)__ballot(me)) - 1;
  *at = {{__builtin_amdgcn_readlane(r.start, l), __builtin_amdgcn_readlane(r.n, l)},
         {__builtin_amdgcn_readlane(k.start, l), __builtin_amdgcn_readlane(k.n, l)},
         lo,
         __builtin_amdgcn_readlane(n, l)};
  return true;
}

// ---------------------------------------------------------------------------
// Products.
// ---------------------------------------------------------------------------
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

// c += a b over the 16 bytes of the summed index that each lane holds (two
// lanes: 16 values of 16 bits, or 8 of 32).
template <class T>
__device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (std::is_same<T, __bf16>::value) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else if constexpr (std::is_same<T, _Float16>::value) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], c, 0, 0, 0);
    return c;
  }
}

// The same with the sum held in accumulation registers, of which a lane has 256
// beside its 256 others: the compiler keeps results in one kind of the two, and
// kernels with more than 256 of them need both.  (The no-op covers the two cycles
// between a vector instruction's result and its use here, which the compiler counts
// for instructions that it knows; settle() stands between the last product and the
// first other use of a sum.  The compiler may copy a sum to other registers before that,
// where the loop ends: finished() stands there.)
template <class T>
__device__ __forceinline__ void mma_far(u32x4 a, u32x4 b, f32x16& c) {
  if constexpr (std::is_same<T, __bf16>::value)
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  else
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mma_far(float a, float b, f32x16& c) {
  asm("s_nop 1\n\tv_mfma_f32_32x32x2_f32 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
__device__ __forceinline__ void settle(f32x16& c) {
  asm volatile("s_nop 15\n\ts_nop 7" : "+a"(c));
}

// Two values rounded to T, in a word; and both values of such a word added to x.
template <class T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef T t2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), t2));
}
template <class T>
__device__ __forceinline__ float add2(uint32_t w, float x) {
  if constexpr (std::is_same<T, __bf16>::value)
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w),
                                           bf16x2{(__bf16)1.f, (__bf16)1.f}, x, false);
  else
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w), f16x2{(_Float16)1.f, (_Float16)1.f},
                                  x, false);
}

// ---------------------------------------------------------------------------
// A tile in LDS: rows of D values, row-major, in chunks of 16 bytes that stand
// at their index XOR turn(row).  The turn takes all values that it can over 16
// rows, the low two bits of the row first: 16 rows read at one chunk, four
// rows (aligned) read over 64 bytes by the transposing loads, and a row read or
// written along itself then spread over all banks.
// ---------------------------------------------------------------------------
template <class T, int D>
struct Tile {
  static constexpr int row_bytes = D * (int)sizeof(T);
  static constexpr int chunks = row_bytes / 16;
  static constexpr int NW = chunks / 2;       // steps of a product over D
  static constexpr int ND = D / 32;           // blocks of 32 dimensions

  __device__ static __forceinline__ int turn(int row) {
    return chunks == 8 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : (row & 3) << 2 | (row >> 2 & 3);
  }
  __device__ static __forceinline__ int at(int row, int chunk) {
    return row * row_bytes + ((chunk ^ turn(row)) << 4);
  }
};

// The order in which the rows of a block of 32 are given to the first product,
// so that its result is the second one's operand as it lies: component r of a
// lane is row 16*(r/8) + 8*k + r%8 of the block.
__device__ __forceinline__ int ordered_row(int i) {
  return 16 * (i >> 4) + 8 * (i >> 2 & 1) + 4 * (i >> 3 & 1) + (i & 3);
}
__device__ __forceinline__ int row_of(int r, int k) { return 16 * (r / 8) + 8 * k + r % 8; }

// Reading a tile by rows (operand of a product over D): this lane's row of a
// block of 32, chunk 2w + k.  The turn and the chunk's number meet in an XOR, so one
// register holds all of a lane's addresses.  (Tiles begin at multiples of 1 KB.)
template <class T, int D>
struct RowReader {
  using L = Tile<T, D>;
  int off;
  __device__ __forceinline__ RowReader(int row, int k) : off(L::at(row, k)) {}
  __device__ __forceinline__ u32x4 get(const char* tile, int block, int w) const {
    typedef __attribute__((address_space(3))) const char* lds;
    typedef __attribute__((address_space(3))) const u32x4* lds16;
    return *(lds16)((lds)(uintptr_t)(((uint32_t)(uintptr_t)(lds)tile + off) ^ (w << 5)) +
                    block * 32 * L::row_bytes);
  }
};

// Reading a tile by columns (operand of a product over its rows): this lane's
// dimension 32c + i, rows 16h + 8k + 0..7 of the tile, of a 16-bit type.
template <class T, int D>
struct ColumnReader {
  using L = Tile<T, D>;
  int off;
  __device__ __forceinline__ ColumnReader(int lane)
      : off(L::at(8 * (lane >> 5) + (lane >> 2 & 3), 2 * (lane >> 4 & 1) + (lane >> 1 & 1)) +
            8 * (lane & 1)) {}
  __device__ __forceinline__ u32x4 get(const char* tile, int h, int c) const {
    // (16 lanes at 8 bytes each hold a matrix of 4 rows by 16 columns; a lane
    // gets one column of it)
    typedef __attribute__((address_space(3))) const char* lds;
    typedef __attribute__((address_space(3))) s16x4* lds8;
    u32x2 x[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
      x[j] = __builtin_bit_cast(
          u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds8)(
                     (lds)(uintptr_t)(((uint32_t)(uintptr_t)(lds)tile + off) ^ (c << 6 | j << 4)) +
                     (16 * h + 4 * j) * L::row_bytes)));
    return u32x4{x[0][0], x[0][1], x[1][0], x[1][1]};
  }
};
template <int D>
struct ColumnReader<float, D> {
  using L = Tile<float, D>;
  int base, in;
  __device__ __forceinline__ ColumnReader(int lane) {
    const int i = lane & 31, k = lane >> 5;
    base = 8 * k * L::row_bytes + (i & 3) * 4;
    in = (i >> 2) ^ (2 * k);
  }
  // row 16h + 8k + e
  __device__ __forceinline__ float get(const char* tile, int h, int e, int c) const {
    return *reinterpret_cast<const float*>(
        tile + base + (16 * h + e) * L::row_bytes +
        (((8 * c) ^ in ^ ((e & 3) << 2 | (e >> 2))) << 4));
  }
};

// ---------------------------------------------------------------------------
// Tiles on their way from memory to LDS.
// ---------------------------------------------------------------------------
// Whether a value is not finite, of many: the largest magnitude, as bits.
template <class T>
struct Finite {
  uint32_t top = 0;
  __device__ __forceinline__ void take(u32x4 x) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (is_f32<T>)
        top = max(top, x[w] & 0x7fffffffu);
      else
        top = __builtin_bit_cast(
            uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top),
                                                __builtin_bit_cast(u16x2, x[w] & 0x7fff7fffu)));
    }
  }
  __device__ __forceinline__ bool all() const {
    if constexpr (is_f32<T>) return top < 0x7f800000u;
    constexpr uint32_t inf = std::is_same<T, __bf16>::value ? 0x7f80u : 0x7c00u;
    return (top >> 16) < inf && (top & 0xffffu) < inf;
  }
};

// Whether all of a tile in LDS is finite (a wave looks at the whole of it).
template <class T, int D, int ROWS>
__device__ __forceinline__ bool tile_finite(const char* tile, int lane) {
  Finite<T> f;
#pragma unroll 8
  for (int x = lane; x < ROWS * Tile<T, D>::chunks; x += 64)
    f.take(*reinterpret_cast<const u32x4*>(tile + 16 * x));
  return !__any(!f.all());
}

// Without registers on the way: each wave instruction brings 64 units of 16 bytes to
// 1 KB of LDS in turn, so a lane fetches the chunk that belongs at its place.  A
// thread's units are `step` rows apart; the turn repeats every 16 rows, so unit u has
// the chunk of unit u % phases.
template <class T, int D, int ROWS>
struct Direct {
  using L = Tile<T, D>;
  static constexpr int units = ROWS * L::chunks / kThreads;
  static_assert(units >= 1 && ROWS * L::chunks % kThreads == 0, "whole units");
  static constexpr int step = kThreads / L::chunks;
  static constexpr int phases = step < 16 ? 16 / step : 1;

  // The row and the byte in it of this thread's unit u.
  __device__ static __forceinline__ int row(int tid, int u) { return tid / L::chunks + step * u; }
  __device__ static __forceinline__ int byte(int tid, int u) {
    return ((tid % L::chunks) ^ L::turn(row(tid, u))) << 4;
  }
  // Where a wave's unit u goes: an address in LDS.
  __device__ static __forceinline__ int place(const char* tile, int wave, int u) {
    typedef __attribute__((address_space(3))) const char* lds;
    return uniform((int)(uintptr_t)(lds)tile + u * kThreads * 16 + (wave << 10));
  }
};

// Memory as the fetches see it: `bytes` from `base` on (at most 2^31 - 1 count), beyond
// which they bring zeros.
struct Window {
  u32x4 words;
};
__device__ __forceinline__ Window window(const char* base, int64_t bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(base);
  return {u32x4{(uint32_t)at, (uint32_t)(at >> 32),
                (uint32_t)min(max(bytes, (int64_t)0), (int64_t)0x7fffffff), 0x00027000u}};
}
// (In assembly: to the compiler a fetch may write what any later read of LDS
// reads, so that it would wait for it there.  arrived() stands before the barrier.
// A scalar register that a vector instruction wrote, as one that is reloaded from a
// lane, may be read here five wait states later at the earliest: the compiler, which
// counts them for instructions that it knows, may put such a one right before.)
__device__ __forceinline__ void fetch(int place, const Window& from, int lane_byte, int byte) {
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"      // (m0 is the compiler's, between its uses)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(place), "v"(lane_byte), "s"(from.words), "s"(byte)
               : "m0");
#pragma clang diagnostic pop
}
// The same of one word a lane: 256 bytes in turn.
__device__ __forceinline__ void fetch_word(int place, const Window& from, int lane_byte) {
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds"
               :
               : "s"(place), "v"(lane_byte), "s"(from.words)
               : "m0");
#pragma clang diagnostic pop
}
__device__ __forceinline__ int lds_place(const void* p) {
  typedef __attribute__((address_space(3))) const char* lds;
  return uniform((int)(uintptr_t)(lds)(const char*)p);
}

// All fetches but the last `more` have arrived.
template <int more = 0>
__device__ __forceinline__ void arrived() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(more) : "memory");
}

// All fetches have arrived, and the sums of mma_far() before are there to be copied.
__device__ __forceinline__ void finished() {
  asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 7" : : : "memory");
}

// ROWS rows of a KV head (x0 on; those beyond `last` are the last again) on their way
// to a tile.  `base`: the sequence's first row, the KV head's first head.
template <class T, int D, int ROWS>
__device__ __forceinline__ void fetch_rows(char* tile, const Batch& bt, const char* base,
                                           int64_t stride, int x0, int last, int tid, int wave) {
  using F = Direct<T, D, ROWS>;
  const int tok0 = token_of(bt, x0);
  const Window from = window(base + tok0 * stride, 0x7fffffff);
#pragma unroll
  for (int u = 0; u < F::units; ++u) {
    const int x = min(x0 + F::row(tid, u), last), tok = token_of(bt, x);
    fetch(F::place(tile, wave, u), from,
          (tok - tok0) * (int)stride + (x - tok * bt.G) * F::L::row_bytes + F::byte(tid, u), 0);
  }
}

// Results of a wave on their way back: 32 rows (columns of a product) in LDS, then whole
// rows to memory, 16 bytes a lane (four dimensions a lane as they lie would touch each
// line eight times).  `to(row)` is a row's place, or NULL.
template <class T, int D>
__device__ __forceinline__ void put4(char* tile, int row, int d, f32x4 x) {
  using L = Tile<T, D>;
  if constexpr (is_f32<T>)
    *reinterpret_cast<f32x4*>(tile + L::at(row, d / 4)) = x;
  else
    *reinterpret_cast<u32x2*>(tile + L::at(row, d / 8) + d % 8 * 2) =
        u32x2{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3])};
}
template <class T, int D, class F>
__device__ __forceinline__ void store_rows(const char* tile, int rows, int lane, F&& to) {
  using L = Tile<T, D>;
  __builtin_amdgcn_wave_barrier();
#pragma unroll 4
  for (int p = 0; p < rows * L::chunks / 64; ++p) {
    const int row = (p * 64 + lane) / L::chunks, chunk = lane % L::chunks;
    const u32x4 x = *reinterpret_cast<const u32x4*>(tile + L::at(row, chunk));
    char* dst = to(row);
    if (dst) *reinterpret_cast<u32x4*>(dst + 16 * chunk) = x;
  }
  __builtin_amdgcn_wave_barrier();
}

// A word (or several) of memory: not through the instructions that may be LDS too.
template <class V, class P>
__device__ __forceinline__ V far_load(const P* p) {
  typedef const V __attribute__((address_space(1))) * global;
  return *(global)p;
}

}  // namespace prompt

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
namespace prompt {

inline bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int type_bytes(int dtype) { return dtype == DA_F32 ? 4 : 2; }

constexpr int64_t kMaxPerSequence = int64_t(1) << 30;   // rows times the group, and keys
constexpr int64_t kMaxHeads = int64_t(1) << 24;         // sequences x query heads
constexpr int64_t kMaxGroups = (int64_t(1) << 24) - 1;  // of 256 threads: a grid has < 2^32

// The sizes, then what is supported; pointers not looked at.
inline da_status check_sizes(const da_prompt& p) {
  if (p.B < 1 || p.h_q < 1 || p.h_kv < 1 || p.d < 1 || p.rows < 1 || p.keys < 1 || p.T < 1 ||
      p.N < 1 || p.h_q % p.h_kv != 0)
    return DA_ERR_SHAPE;
  if ((int64_t)p.T * (p.h_q / p.h_kv) > kMaxPerSequence || p.N > kMaxPerSequence ||
      (int64_t)p.B * p.h_q > kMaxHeads || (int64_t)p.h_q * p.d > (int64_t(1) << 30))
    return DA_ERR_SHAPE;
  if ((!p.row_start && (int64_t)p.B * p.T != p.rows) ||
      (!p.key_start && (int64_t)p.B * p.N != p.keys))
    return DA_ERR_SHAPE;
  if ((p.d != 64 && p.d != 128 && p.d != 256) || p.dtype < DA_F32 || p.dtype > DA_F16)
    return DA_ERR_UNSUPPORTED;
  return DA_OK;
}

inline bool starts_aligned(const da_prompt& p) {
  return aligned(p.row_start, 4) && aligned(p.key_start, 4);
}

// A token stride (elements) that rows of `heads` heads may have: the kernels take
// offsets within 256 tokens in 32 bits.
constexpr int64_t kMaxStrideBytes = int64_t(1) << 22;
inline bool stride_fits(int64_t stride, int heads, int d, int dtype) {
  return stride >= (int64_t)heads * d && stride <= kMaxStrideBytes / type_bytes(dtype);
}
inline bool stride_aligned(int64_t stride, int dtype) {
  return stride % (16 / type_bytes(dtype)) == 0;
}

inline Batch device_batch(const da_prompt& p) {
  const uint32_t G = p.h_q / p.h_kv;
  uint32_t shift = 31;
  while (G > 1u << (shift - 31)) ++shift;
  const uint32_t mul = (uint32_t)((uint64_t(1) << shift) / G + 1);
  return {p.row_start, p.key_start, p.B, p.rows, p.keys, p.T, p.N, p.h_q, p.h_kv, (int)G,
          p.causal != 0, mul, shift};
}

// No fewer than the tiles of R that the sequences' n*per rows make.
inline int64_t most_tiles(const int32_t* start, int64_t B, int64_t most, int64_t total,
                          int64_t per, int64_t R) {
  const int64_t even = B * ceil_div(most * per, R);
  return start ? std::min(even, total * per / R + B) : even;
}

inline da_status launch_status() {
  return hipGetLastError() == hipSuccess ? DA_OK : DA_ERR_HIP;
}

// Calls f(type tag, d) with these as compile-time constants.
template <class T>
struct Tag {
  using type = T;
};
template <class F>
void with_type_and_dim(int dtype, int d, F&& f) {
  auto with_dim = [&](auto t) {
    if (d == 64)
      f(t, std::integral_constant<int, 64>{});
    else if (d == 128)
      f(t, std::integral_constant<int, 128>{});
    else
      f(t, std::integral_constant<int, 256>{});
  };
  if (dtype == DA_F32)
    with_dim(Tag<float>{});
  else if (dtype == DA_BF16)
    with_dim(Tag<__bf16>{});
  else
    with_dim(Tag<_Float16>{});
}

}  // namespace prompt
