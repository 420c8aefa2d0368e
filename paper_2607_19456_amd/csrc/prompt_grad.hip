// prompt_grad.hip -- gfx950 kernels and C ABI of the gradient of attention over
// whole prompts (prompt_attn.hip).  With the weights P = exp(scale q.K - lse), the
// products dP = dout.V and delta = sum_d dout*out of each row,
//   dS = P (dP - delta),   dQ = scale dS K,   dK = scale dS^T Q,   dV = P^T dout.
//
// Kernels
//   prompt_grad_rows_kernel   dQ of a tile of query rows, over the keys that they
//                             see; leaves each row's lse and delta for the next.
//   prompt_grad_keys_kernel   dK and dV of a tile of keys, over the rows of all the
//                             group's heads that see them.
//   prompt_grad_merge_kernel  adds the parts where a tile is divided.
//
// Two passes compute the scores twice (seven products for five), and every sum
// has one order: no atomics, equal calls give equal bits.  One pass would leave dQ to
// atomics, or dS to memory: 2 bytes a pair, written and read, take longer than the two
// products.
//
// Rows and keys are masked after the products; what a row does not see must not meet
// its weight of 0 where it is not finite, so a masked tile is looked over first, and
// where it holds an infinity or a NaN its pairs are added one by one at the end.
//
// In 16-bit types P and dS are rounded to the type, since the matrix instructions take
// no others (two terms of each would be twice the products that they enter); delta is
// that of `out` as it was rounded, the only one that a caller has.  All sums are in 32
// bits.  Errors (2-norm, bfloat16): dQ and dK 0.0024 from the rounding of dS and their own,
// 0.0025 to 0.0030 with that of `out` (least in long sequences), dV 0.0023; a result in 64
// bits rounded once has 0.0017.
#include <algorithm>
#include <cfloat>

#include "prompt_common.h"

namespace {

using namespace prompt;

struct GradArgs {
  const char *q, *k, *v, *out, *d_out;
  const float* lse;
  char *dq, *dk, *dv;
  int64_t q_stride, k_stride, v_stride, d_out_stride;     // bytes between tokens
  int64_t dq_stride, dk_stride, dv_stride;
  float scale, scale2;          // and times log2(e)
  // [rows][h_q] each: lse times log2(e) (+infinity: no weights), and delta
  float *lse2, *delta;
  // Each tile's keys (or rows) are taken in so many parts, whose sums in 32 bits go to
  // parts and are added by a kernel of their own where there is more than one:
  // [workgroup][rows][D], for dK and dV [workgroup][dK, dV][keys][D].
  int row_splits, key_splits;
  float* parts;
};

template <class T>
__device__ __forceinline__ float dot16(u32x4 a, u32x4 b, float sum) {
  constexpr int n = 16 / sizeof(T);
  typedef T tn __attribute__((ext_vector_type(n)));
  const tn x = __builtin_bit_cast(tn, a), y = __builtin_bit_cast(tn, b);
#pragma unroll
  for (int e = 0; e < n; ++e) sum += (float)x[e] * (float)y[e];
  return sum;
}

// ---------------------------------------------------------------------------
// dQ.  As the attention itself: 32 NQ rows of a KV head to a wave, as columns;
//   S^T = K . Q^T, dP^T = V . dO^T, dQ^T += K^T . dS^T
// for 32 keys at a time: the exponentials between the products of dP, half of dS
// between those of dQ, operands read two products ahead, K and V fetched two tiles
// ahead.  32 rows a wave (d = 64 also 64): Q and dO of 128 dimensions take 64 registers, the
// sums 64 accumulation registers, so two workgroups run on a CU, and one reads or writes
// its rows (192 KB in, 64 out for 256 rows) while the other multiplies.  64 rows a wave
// read half as much from LDS, but one workgroup has the CU to itself.
// Measured, bfloat16, causal, 32/8 heads of 128, us (in brackets with 64 rows a wave, in
// the same run): one sequence of 8192 rows 860 (907), 4 of 2048 230 (255), 16 of 1024
// 284 (347), 32 of 512 212 (271), 64 of 256 180 (235).
// ---------------------------------------------------------------------------
template <class T, int D, int NQ>
struct RowsForm {
  static constexpr int rows = 32 * NQ * kWaves;
  static constexpr int keys = NQ == 1 ? 32 : 64;                    // of a tile
  static constexpr int tiles = is_f32<T> && D == 256 ? 2 : 3;       // in LDS
  static constexpr int groups = !is_f32<T> && D == 128 && NQ == 1 ? 2 : 1;     // a CU
};

template <class T, int D, int NQ>
__global__ __launch_bounds__(kThreads, (RowsForm<T, D, NQ>::groups)) void prompt_grad_rows_kernel(Batch bt, GradArgs a) {
  using L = Tile<T, D>;
  using F = RowsForm<T, D, NQ>;
  constexpr int KT = F::keys, R = F::rows, NB = F::tiles;
  constexpr int ND = L::ND, NW = L::NW;
  constexpr int kTile = KT * L::row_bytes;
  using Fetch = Direct<T, D, KT>;

  // K's tiles, then V's; Q and dO on their way in, and dQ on its way out
  static_assert(2 * NB * kTile >= R * L::row_bytes, "room for the rows");
  __shared__ __align__(1024) char s_all[2 * NB][kTile];
  char(*s_k)[kTile] = s_all, (*s_v)[kTile] = s_all + NB;
  // 32 rows of zeros, where there is room
  constexpr bool kZeros = 2 * NB * kTile + 32 * L::row_bytes < 160 << 10;
  __shared__ __align__(1024) char s_zero[kZeros ? 32 * L::row_bytes : 16];

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int i = lane & 31, k = lane >> 5;
  const int head = blockIdx.x % bt.h_kv, split = blockIdx.x / bt.h_kv % a.row_splits;
  Place at;
  if (!find(bt, true, R, blockIdx.x / bt.h_kv / a.row_splits, lane, &at)) return;
  const Span rows = at.rows, keys = at.keys;
  const int row0 = at.after * R;             // the last rows, which see most, first
  const int in_tile = min(rows.n * bt.G - row0, R);
  const int min_seen = seen_by(bt, rows.n, keys.n, token_of(bt, row0));
  const int max_seen = seen_by(bt, rows.n, keys.n, token_of(bt, row0 + in_tile - 1));
  const int tiles = (max_seen + KT - 1) / KT;
  const int t0 = (int)((int64_t)tiles * split / a.row_splits);
  const int t1 = (int)((int64_t)tiles * (split + 1) / a.row_splits);

  const int my_row0 = row0 + 32 * NQ * wave;
  const int my_rows = min(max(in_tile - 32 * NQ * wave, 0), 32 * NQ);
  int seen[NQ];
  float lse2[NQ], delta[NQ];
  u32x4 q[NQ][NW], g[NQ][NW];
  auto place = [&](int x) INLINE {           // row * h_q + head of this wave's row x
    const int tok = token_of(bt, my_row0 + x);
    return (int64_t)(rows.start + tok) * bt.h_q + head * bt.G + my_row0 + x - tok * bt.G;
  };
  {
    const RowReader<T, D> rd(i, k);
    const int64_t in = (int64_t)head * bt.G * L::row_bytes;
    auto bring = [&](const char* base, int64_t stride) INLINE {
      fetch_rows<T, D, R>(s_all[0], bt, base + rows.start * stride + in, stride, row0,
                          row0 + in_tile - 1, tid, wave);
      arrived();
      __syncthreads();
    };
    bring(a.q, a.q_stride);
#pragma unroll
    for (int b = 0; b < NQ; ++b)
#pragma unroll
      for (int w = 0; w < NW; ++w) q[b][w] = rd.get(s_all[0], NQ * wave + b, w);
    __syncthreads();
    bring(a.d_out, a.d_out_stride);
#pragma unroll
    for (int b = 0; b < NQ; ++b)
#pragma unroll
      for (int w = 0; w < NW; ++w) g[b][w] = rd.get(s_all[0], NQ * wave + b, w);
    __syncthreads();
    bring(a.out, (int64_t)bt.h_q * L::row_bytes);
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      const int x = 32 * b + i;
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) sum = dot16<T>(g[b][w], rd.get(s_all[0], NQ * wave + b, w), sum);
      delta[b] = sum + __shfl_xor(sum, 32);
      seen[b] = 0, lse2[b] = INFINITY;
      if (x < my_rows) {
        seen[b] = seen_by(bt, rows.n, keys.n, token_of(bt, my_row0 + x));
        const float lse = far_load<float>(a.lse + place(x));
        lse2[b] = lse == -INFINITY ? INFINITY : lse * kLog2e;
        if (k == 0 && split == 0) a.lse2[place(x)] = lse2[b], a.delta[place(x)] = delta[b];
      }
    }
    __syncthreads();
  }

  f32x16 acc[NQ][ND];
#pragma unroll
  for (int b = 0; b < NQ; ++b)
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[b][c][r] = 0.f;

  const char* k_base = a.k + (int64_t)keys.start * a.k_stride + (int64_t)head * L::row_bytes;
  const char* v_base = a.v + (int64_t)keys.start * a.v_stride + (int64_t)head * L::row_bytes;
  const RowReader<T, D> read(ordered_row(i), k);
  const ColumnReader<T, D> read_columns(lane);

  // Keys beyond the last are zeros, which no row sees.
  int k_byte[Fetch::phases], v_byte[Fetch::phases];
#pragma unroll
  for (int u = 0; u < Fetch::phases; ++u) {
    k_byte[u] = Fetch::row(tid, u) * (int)a.k_stride + Fetch::byte(tid, u);
    v_byte[u] = Fetch::row(tid, u) * (int)a.v_stride + Fetch::byte(tid, u);
  }
  auto load = [&](int t) INLINE {
    const int64_t key0 = (int64_t)t * KT;
    const Window from_k = window(k_base + key0 * a.k_stride, (keys.n - key0) * a.k_stride);
    const Window from_v = window(v_base + key0 * a.v_stride, (keys.n - key0) * a.v_stride);
#pragma unroll
    for (int u = 0; u < Fetch::units; ++u) {
      const int further = u / Fetch::phases * (Fetch::phases * Fetch::step);
      fetch(Fetch::place(s_k[(t - t0) % NB], wave, u), from_k, k_byte[u % Fetch::phases],
            further * (int)a.k_stride);
      fetch(Fetch::place(s_v[(t - t0) % NB], wave, u), from_v, v_byte[u % Fetch::phases],
            further * (int)a.v_stride);
    }
  };
  bool skipped = false;
  if (kZeros)
    for (int x = tid; x < 32 * L::chunks; x += kThreads)
      reinterpret_cast<u32x4*>(s_zero)[x] = u32x4{0u, 0u, 0u, 0u};

  if (t0 < t1) {
#pragma unroll
    for (int t = 0; t < NB - 1; ++t) load(t0 + t);
    arrived();
    __syncthreads();
  }
#pragma unroll
  for (int b = 0; b < NQ; ++b)
#pragma unroll
    for (int w = 0; w < NW; ++w) asm volatile("" : "+v"(q[b][w]), "+v"(g[b][w]));
  for (int t = t0; t < t1; ++t) {
    char* tile_k = s_k[(t - t0) % NB];
    const char* tile_v = s_v[(t - t0) % NB];
#pragma unroll
    for (int n = 0; n < KT / 32; ++n) {
      f32x16 s[NQ], dp[NQ];
      float less[NQ];                        // delta, till dS is made
#pragma unroll
      for (int b = 0; b < NQ; ++b) {
        less[b] = delta[b];
#pragma unroll
        for (int r = 0; r < 16; ++r) s[b][r] = 0.f, dp[b][r] = 0.f;
      }
      // S
      u32x4 x0 = read.get(tile_k, n, 0), x1 = read.get(tile_k, n, 1);
      if (n == 0) load(t + NB - 1);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const u32x4 x2 = w + 2 < NW ? read.get(tile_k, n, w + 2) : read.get(tile_v, n, w + 2 - NW);
#pragma unroll
        for (int b = 0; b < NQ; ++b) s[b] = mma<T>(x0, q[b][w], s[b]);
        x0 = x1, x1 = x2;
        __builtin_amdgcn_sched_barrier(0);
      }
      // dP, and P
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        u32x4 x2 = x0;
        if (w + 2 < NW) x2 = read.get(tile_v, n, w + 2);
#pragma unroll
        for (int b = 0; b < NQ; ++b) dp[b] = mma<T>(x0, g[b][w], dp[b]);
        if (4 * w % NW == 0) {
#pragma unroll
          for (int b = 0; b < NQ; ++b)
#pragma unroll
            for (int r = 16 * w / NW; r < 16 * w / NW + 4; ++r)
              s[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], a.scale2, -lse2[b]));
        }
        x0 = x1, x1 = x2;
        if (4 * (w + 1) % NW == 0) __builtin_amdgcn_sched_barrier(0);
      }
      const int key0 = t * KT + 32 * n;
      const char* by_columns = tile_k + 32 * n * L::row_bytes;
      if (__builtin_expect(key0 + 32 > min_seen, 0)) {
        // What a row does not see must not meet its weight of 0 where it is not
        // finite: such keys are left out here (zeros in their place) and added at the
        // end.
        const bool bad = !tile_finite<T, D, 32>(tile_k + 32 * n * L::row_bytes, lane);
        if (!kZeros) __syncthreads();
        if (bad) skipped = true;
        if (kZeros) {
          if (bad) by_columns = s_zero;
        } else if (bad) {
          for (int x = lane; x < 32 * L::chunks; x += 64)
            reinterpret_cast<u32x4*>(tile_k + 32 * n * L::row_bytes)[x] = u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int b = 0; b < NQ; ++b) {
          const int left = bad ? -INT32_MAX : seen[b] - key0 - 8 * k;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[b][r] = row_of(r, 0) >= left ? 0.f : s[b][r] * (dp[b][r] - delta[b]);
            dp[b][r] = 1.f;
          }
          less[b] = 0.f;
        }
      }
      // dS, and dQ
      if constexpr (is_f32<T>) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
#pragma unroll
          for (int b = 0; b < NQ; ++b) s[b][r] *= dp[b][r] - less[b];
#pragma unroll
          for (int c = 0; c < ND; ++c) {
            const float x = read_columns.get(by_columns, r / 8, r % 8, c);
#pragma unroll
            for (int b = 0; b < NQ; ++b) mma_far(x, s[b][r], acc[b][c]);
          }
        }
      } else {
        u32x4 y0 = read_columns.get(by_columns, 0, 0), y1 = read_columns.get(by_columns, 0, 1);
        u32x4 ds[2][NQ];
        auto piece = [&](int h, int b) INLINE {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 8 * h + 2 * e;
            ds[h][b][e] = pack2<T>(s[b][r] * (dp[b][r] - less[b]),
                                   s[b][r + 1] * (dp[b][r + 1] - less[b]));
          }
        };
#pragma unroll
        for (int b = 0; b < NQ; ++b) piece(0, b);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < 2 * ND; ++e) {
          u32x4 y2 = y0;
          if (e + 2 < 2 * ND) y2 = read_columns.get(by_columns, (e + 2) / ND, (e + 2) % ND);
#pragma unroll
          for (int b = 0; b < NQ; ++b) mma_far<T>(y0, ds[e / ND][b], acc[b][e % ND]);
          if (e < NQ) piece(1, e);
          y0 = y1, y1 = y2;
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    arrived<2 * Fetch::units*(NB - 2)>();
    __syncthreads();
  }
  finished();                                // (what was fetched beyond the last, too)
  __syncthreads();

  char* mine = s_all[0] + 32 * NQ * wave * L::row_bytes;
  auto to = [&](int x) INLINE {              // the place of this wave's row x
    const int tok = token_of(bt, my_row0 + x);
    return a.dq + (rows.start + tok) * a.dq_stride +
           (int64_t)(head * bt.G + my_row0 + x - tok * bt.G) * L::row_bytes;
  };
  auto part_of = [&](int x) INLINE {
    return a.parts + ((int64_t)blockIdx.x * R + 32 * NQ * wave + x) * D;
  };
  // The keys that were left out, those alone that the row sees: the sums pass through
  // LDS in 32 bits, 32 rows of one wave at a time.
  if (__builtin_expect(skipped, 0)) {
    static_assert(2 * NB * kTile >= 32 * D * 4, "room for the sums");
    float* sums = reinterpret_cast<float*>(s_all[0]) + i * D;
#pragma unroll
    for (int b = 0; b < NQ; ++b)
#pragma unroll
      for (int c = 0; c < ND; ++c) settle(acc[b][c]);
    for (int w = 0; w < kWaves; ++w) {
#pragma unroll
      for (int b = 0; b < NQ; ++b) {
        __syncthreads();
        if (w != wave) continue;
#pragma unroll
        for (int c = 0; c < ND; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            sums[32 * c + 8 * (r / 4) + 4 * k + r % 4] = acc[b][c][r];
        __builtin_amdgcn_wave_barrier();
        const int64_t at_row = place(min(32 * b + i, max(my_rows - 1, 0)));
        const T* q_row =
            reinterpret_cast<const T*>(a.q + at_row / bt.h_q * a.q_stride) + at_row % bt.h_q * D;
        const T* g_row = reinterpret_cast<const T*>(a.d_out + at_row / bt.h_q * a.d_out_stride) +
                         at_row % bt.h_q * D;
#pragma unroll 1
        for (int key0 = max(min_seen / 32 * 32, t0 * KT); key0 < min(max_seen, t1 * KT); key0 += 32) {
          auto row_at = [&](const char* base, int64_t stride, int key) INLINE {
            return reinterpret_cast<const T*>(base + key * stride);
          };
          bool bad = false;
          if (key0 + i < keys.n) {
            const T* row = row_at(k_base, a.k_stride, key0 + i);
#pragma unroll 1
            for (int d = k; d < D; d += 2) bad = bad || !(fabsf((float)row[d]) < INFINITY);
          }
          if (!__any(bad)) continue;
#pragma unroll 1
          for (int key = key0; key < min(key0 + 32, seen[b]); ++key) {
            const T* k_row = row_at(k_base, a.k_stride, key);
            const T* v_row = row_at(v_base, a.v_stride, key);
            float s = 0.f, dp = 0.f;
#pragma unroll 1
            for (int d = 0; d < D; ++d) {
              s += (float)q_row[d] * (float)k_row[d];
              dp += (float)g_row[d] * (float)v_row[d];
            }
            float x =
                __builtin_amdgcn_exp2f(__builtin_fmaf(s, a.scale2, -lse2[b])) * (dp - delta[b]);
            if constexpr (!is_f32<T>) x = (float)(T)x;
#pragma unroll 1
            for (int d = k; d < D; d += 2) sums[d] += x * (float)k_row[d];
          }
        }
        __builtin_amdgcn_wave_barrier();
        if (32 * b + i < my_rows) {
          T* dst = reinterpret_cast<T*>(to(32 * b + i));
          float* part = part_of(32 * b + i);
#pragma unroll 1
          for (int d = k; d < D; d += 2) {
            if (a.row_splits > 1)
              part[d] = sums[d];
            else
              dst[d] = (T)(sums[d] * a.scale);
          }
        }
      }
    }
    return;
  }
#pragma unroll
  for (int b = 0; b < NQ; ++b)
#pragma unroll
    for (int c = 0; c < ND; ++c) {
      settle(acc[b][c]);
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 x{acc[b][c][r], acc[b][c][r + 1], acc[b][c][r + 2], acc[b][c][r + 3]};
        const int d = 32 * c + 2 * r + 4 * k;
        if (a.row_splits == 1)
          put4<T, D>(mine, 32 * b + i, d, x * a.scale);
        else if (32 * b + i < my_rows)
          *reinterpret_cast<f32x4*>(part_of(32 * b + i) + d) = x;
      }
    }
  if (a.row_splits > 1) return;
  store_rows<T, D>(mine, 32 * NQ, lane, [&](int x) INLINE {
    return x < my_rows ? to(x) : nullptr;
  });
}

// ---------------------------------------------------------------------------
// dK and dV.  A wave holds K and V of 32 NK keys as columns and takes in rows,
// 32 at a time:
//   S [rows x keys] = Q . K^T, dP = dO . V^T, dV^T += dO^T . P, dK^T += Q^T . dS.
// The four waves are WK keys wide, WR of rows (whose sums are added at the end)
// and WD of dimensions (each computes the scores, and its dimensions of the
// results).
//
// d = 128: 64 keys a wave, so an operand read from LDS serves two products.  dK and dV take
// all 256 accumulation registers and K and V 128 of the others, so the rest is kept small:
// one register of addresses a reader, rows fetched straight to LDS, P packed half a block at
// a time.  The exponentials stand between the products of dP, dS between those of dV.  Two
// row waves instead of four key waves: tiles of 128 keys divide a causal batch more evenly
// than 256.  Measured, as above: 1025 to 1034 us, 1063 TFLOP/s of its four products (446
// with 32 keys a wave and the tiles through registers; with 32 and two workgroups a CU, of
// 256 registers and some in memory, 1.5 times as long).  A step of 64 rows takes 2.0 us, 46 %
// of it products at full rate; a masked one 3.4.  A workgroup's start and end take 11 us.
//
// d = 64: four waves of 32 keys, two workgroups a CU, and no sums of row waves to add.
// bfloat16, 16 heads, causal, us (in brackets with 64 keys and two row waves): 4 sequences
// of 4096 rows 341 (404), 16 of 512 48 (68), 32 of 300 52 (87).
// ---------------------------------------------------------------------------
template <class T, int D>
struct KeysForm {
  static constexpr bool wide = is_f32<T> && D == 256;
  static constexpr bool slim = !is_f32<T> && D == 64;
  static constexpr int NK = !is_f32<T> && D == 128 ? 2 : 1;
  static constexpr int WK = slim ? 4 : wide ? 1 : 2, WR = slim || wide ? 1 : 2, WD = wide ? 4 : 1;
  static constexpr int keys = 32 * NK * WK;
};

template <class T, int D>
__global__ __launch_bounds__(kThreads, (KeysForm<T, D>::slim ? 2 : 1)) void prompt_grad_keys_kernel(Batch bt, GradArgs a) {
  using L = Tile<T, D>;
  using F = KeysForm<T, D>;
  constexpr int NK = F::NK, WK = F::WK, WR = F::WR, WD = F::WD;
  static_assert(WK * WR * WD == kWaves && (WR == 1 || WD == 1), "four waves");
  constexpr int RT = 32 * WR;                 // rows of a step
  constexpr int NW = L::NW, ND = L::ND / WD;
  constexpr int kTile = RT * L::row_bytes;

  // Steps in LDS: two on their way where there is room for them.
  constexpr int NB = 6 * kTile + 32 * L::row_bytes < 150 << 10 ? 3 : 2;
  constexpr int kTiles = std::max(2 * NB, 2 * F::keys / RT);    // (K and V on their way in)
  __shared__ __align__(1024) char s_rows[kTiles][kTile];        // Q's tiles, dO's tiles
  __shared__ __align__(16) float s_lse[NB][64], s_delta[NB][64];
  // 32 rows of zeros, where there is room
  constexpr bool kZeros = 2 * NB * kTile + NB * 512 + 32 * L::row_bytes < 160 << 10;
  __shared__ int s_skipped;
  __shared__ __align__(1024) char s_zero[kZeros ? 32 * L::row_bytes : 16];

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int i = lane & 31, k = lane >> 5;
  const int wk = wave % WK, wr = wave / WK % WR, wd = wave / (WK * WR);
  const int head = blockIdx.x % bt.h_kv, split = blockIdx.x / bt.h_kv % a.key_splits;
  Place at;
  if (!find(bt, false, F::keys, blockIdx.x / bt.h_kv / a.key_splits, lane, &at)) return;
  const Span rows = at.rows, keys = at.keys;
  const int end = rows.n * bt.G;
  const int key0 = (at.tiles - 1 - at.after) * F::keys;
  // the first row (token and head) that sees a key
  auto first_row = [&](int key) INLINE {
    return bt.causal ? (int)min((int64_t)max(key - keys.n + rows.n, 0) * bt.G, (int64_t)end) : 0;
  };
  const int all_from = first_row(min(key0 + F::keys, keys.n) - 1);   // rows that see all of the keys
  const int from = first_row(key0) / RT, steps = (end + RT - 1) / RT - from;
  const int r0 = from + (int)((int64_t)steps * split / a.key_splits);
  const int r1 = from + (int)((int64_t)steps * (split + 1) / a.key_splits);

  auto key_of = [&](int n, int lane) INLINE {
    return key0 + 32 * (NK * wk + n) + (lane & 31);
  };
  u32x4 kk[NK][NW], vv[NK][NW];
  {
    using Keys = Direct<T, D, F::keys>;
    char *tile_k = s_rows[0], *tile_v = s_rows[0] + F::keys * L::row_bytes;
    auto bring = [&](char* tile, const char* base, int64_t stride) INLINE {
      const char* first = base + (keys.start + (int64_t)key0) * stride +
                          (int64_t)head * L::row_bytes;
      const Window from = window(first, (int64_t)(keys.n - key0) * stride);
#pragma unroll
      for (int u = 0; u < Keys::units; ++u)
        fetch(Keys::place(tile, wave, u), from,
              Keys::row(tid, u) * (int)stride + Keys::byte(tid, u), 0);
    };
    bring(tile_k, a.k, a.k_stride);
    bring(tile_v, a.v, a.v_stride);
    arrived();
    __syncthreads();
    const RowReader<T, D> rd(i, k);
#pragma unroll
    for (int n = 0; n < NK; ++n)
#pragma unroll
      for (int w = 0; w < NW; ++w)
        kk[n][w] = rd.get(tile_k, NK * wk + n, w), vv[n][w] = rd.get(tile_v, NK * wk + n, w);
    __syncthreads();
  }

  f32x16 dk[NK][ND], dv[NK][ND];
#pragma unroll
  for (int n = 0; n < NK; ++n)
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) dk[n][c][r] = 0.f, dv[n][c][r] = 0.f;

  const RowReader<T, D> read(ordered_row(i), k);
  const ColumnReader<T, D> read_columns(lane);

  // (The weights of rows beyond the last are taken as 0.)
  using Fetch = Direct<T, D, RT>;
  auto window_of = [&](const char* base, int64_t stride, int t) INLINE {
    const int64_t tok = token_of(bt, min(t * RT, end - 1));
    return window(base + (rows.start + tok) * stride + (int64_t)head * bt.G * L::row_bytes,
                  (rows.n - tok) * stride);
  };
  // Where a group's heads divide the rows between a thread's units, its place among a
  // step's tokens is the same every step, and further units are whole tokens on.
  const bool even = Fetch::step % bt.G == 0 && Fetch::phases == 1;
  int q_byte = 0, g_byte = 0;
  if (even) {
    const int tok = token_of(bt, Fetch::row(tid, 0));
    const int in = (Fetch::row(tid, 0) - tok * bt.G) * L::row_bytes + Fetch::byte(tid, 0);
    q_byte = tok * (int)a.q_stride + in, g_byte = tok * (int)a.d_out_stride + in;
  }
  const float* stats = wave & 1 ? a.delta : a.lse2;          // (two waves bring each)
  auto load_rows = [&](int t) INLINE {
    {
      const int x0 = min(t * RT, end - 1), tok0 = token_of(bt, x0);
      const int x = min(t * RT + lane, end - 1), tok = token_of(bt, x);
      const Window from = window(reinterpret_cast<const char*>(
                                     stats + (int64_t)(rows.start + tok0) * bt.h_q + head * bt.G),
                                 0x7fffffff);
      fetch_word(lds_place(wave & 1 ? s_delta[t % NB] : s_lse[t % NB]), from,
                 4 * ((tok - tok0) * bt.h_q + x - tok * bt.G));
    }
    const Window from_q = window_of(a.q, a.q_stride, t);
    const Window from_g = window_of(a.d_out, a.d_out_stride, t);
    if (even) {
      const int tokens = token_of(bt, Fetch::step);
#pragma unroll
      for (int u = 0; u < Fetch::units; ++u) {
        fetch(Fetch::place(s_rows[t % NB], wave, u), from_q, q_byte, u * tokens * (int)a.q_stride);
        fetch(Fetch::place(s_rows[NB + t % NB], wave, u), from_g, g_byte,
              u * tokens * (int)a.d_out_stride);
      }
      return;
    }
    const int tok0 = token_of(bt, min(t * RT, end - 1));
#pragma unroll
    for (int u = 0; u < Fetch::units; ++u) {
      const int x = min(t * RT + Fetch::row(tid, u), end - 1), tok = token_of(bt, x);
      const int in = (x - tok * bt.G) * L::row_bytes + Fetch::byte(tid, u);
      fetch(Fetch::place(s_rows[t % NB], wave, u), from_q, (tok - tok0) * (int)a.q_stride + in, 0);
      fetch(Fetch::place(s_rows[NB + t % NB], wave, u), from_g,
            (tok - tok0) * (int)a.d_out_stride + in, 0);
    }
  };
  // Not all rows of a step see all keys, and what they do not see is masked.
  auto partial = [&](int t) INLINE { return t * RT < all_from || (t + 1) * RT > end; };
  bool skipped = false;
  if (tid == 0) s_skipped = 0;
  if (kZeros)
    for (int x = tid; x < 32 * L::chunks; x += kThreads)
      reinterpret_cast<u32x4*>(s_zero)[x] = u32x4{0u, 0u, 0u, 0u};

  if (r0 < r1) {
#pragma unroll
    for (int t = 0; t < NB - 1; ++t) load_rows(r0 + t);
    arrived();
    __syncthreads();
  }
  {
    for (int t = r0; t < r1; ++t) {
      const int buf = t % NB;
      const char *tile_q = s_rows[buf] + 32 * wr * L::row_bytes;
      const char *tile_g = s_rows[NB + buf] + 32 * wr * L::row_bytes;
      const float *my_lse = &s_lse[buf][32 * wr], *my_delta = &s_delta[buf][32 * wr];
      const int row0 = t * RT + 32 * wr;
      f32x16 s[NK], dp[NK];
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[n][r] = 0.f, dp[n][r] = 0.f;
      {
        // S, and the fetches of rows to come; operands are read two products ahead
        auto by_rows = [&](int w) INLINE {
          return w < NW ? read.get(tile_q, 0, w) : read.get(tile_g, 0, w - NW);
        };
        auto lse_of = [&](int r) INLINE {
          return *reinterpret_cast<const f32x4*>(my_lse + row_of(r, k));
        };
        u32x4 x0 = by_rows(0), x1 = by_rows(1);
        f32x4 z = lse_of(0);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const u32x4 x2 = by_rows(w + 2);
#pragma unroll
          for (int n = 0; n < NK; ++n) s[n] = mma<T>(x0, kk[n][w], s[n]);
          if (w == 0) load_rows(t + NB - 1);
          x0 = x1, x1 = x2;
          __builtin_amdgcn_sched_barrier(0);
        }
        // dP, and P
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          u32x4 x2 = x0;
          if (w + 2 < NW) x2 = by_rows(NW + w + 2);
#pragma unroll
          for (int n = 0; n < NK; ++n) dp[n] = mma<T>(x0, vv[n][w], dp[n]);
          if (4 * w % NW == 0) {
            const int r = 16 * w / NW;
            const f32x4 z1 = r + 4 < 16 ? lse_of(r + 4) : z;
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                s[n][r + e] =
                    __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r + e], a.scale2, -z[e]));
            z = z1;
          }
          x0 = x1, x1 = x2;
          if (4 * (w + 1) % NW == 0) __builtin_amdgcn_sched_barrier(0);
        }
      }
      const char *columns_q = tile_q, *columns_g = tile_g;
      const float* deltas = my_delta;
      if (__builtin_expect(partial(t), 0)) {
        // What a row does not see must not meet its weight of 0 where it is not
        // finite: such rows are left out here (zeros in their place) and added at the
        // end.
        const float x = my_lse[i], y = my_delta[i];
        const bool bad = !tile_finite<T, D, 32>(tile_q, lane) || !tile_finite<T, D, 32>(tile_g, lane) ||
                         __any(x != x || !(fabsf(y) < INFINITY));
        if (!kZeros) __syncthreads();
        if (bad) {
          skipped = true;
          if (kZeros) {
            columns_q = columns_g = s_zero;
            deltas = reinterpret_cast<const float*>(s_zero);
          } else {
            for (int x = lane; x < 32 * L::chunks; x += 64)
              reinterpret_cast<u32x4*>(s_rows[buf] + 32 * wr * L::row_bytes)[x] =
                  reinterpret_cast<u32x4*>(s_rows[NB + buf] + 32 * wr * L::row_bytes)[x] =
                      u32x4{0u, 0u, 0u, 0u};
            s_delta[buf][32 * wr + i] = 0.f;
          }
        }
        // (the lane hidden from the compiler: what follows from it would otherwise be
        // held through the loop, in registers that there are none of)
        int now = lane;
        asm volatile("" : "+v"(now));
#pragma unroll
        for (int n = 0; n < NK; ++n) {
          const int from = first_row(min(key_of(n, now), keys.n - 1));
          const int first = from - row0 - 8 * (now >> 5);
          const unsigned seeing = bad ? 0u : (unsigned)max(end - from, 0);
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((unsigned)(row_of(r, 0) - first) >= seeing) s[n][r] = 0.f, dp[n][r] = 0.f;
        }
      }
      // dV, and dS
      if constexpr (is_f32<T>) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
#pragma unroll
          for (int c = 0; c < ND; ++c) {
            const float x = read_columns.get(columns_g, r / 8, r % 8, ND * wd + c);
#pragma unroll
            for (int n = 0; n < NK; ++n) mma_far(x, s[n][r], dv[n][c]);
          }
          const float y = deltas[row_of(r, k)];
#pragma unroll
          for (int n = 0; n < NK; ++n) dp[n][r] = s[n][r] * (dp[n][r] - y);
#pragma unroll
          for (int c = 0; c < ND; ++c) {
            const float x = read_columns.get(columns_q, r / 8, r % 8, ND * wd + c);
#pragma unroll
            for (int n = 0; n < NK; ++n) mma_far(x, dp[n][r], dk[n][c]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
        u32x4 p[NK], ds[2][NK];
        auto by_columns = [&](int e) INLINE {
          return read_columns.get(e < 2 * ND ? columns_g : columns_q, e / ND % 2, e % ND);
        };
        auto delta_of = [&](int r) INLINE {
          return *reinterpret_cast<const f32x4*>(deltas + row_of(r, k));
        };
        u32x4 x0 = by_columns(0), x1 = by_columns(1);
        f32x4 z = delta_of(0);
#pragma unroll
        for (int e = 0; e < 2 * ND; ++e) {
          const int h = e / ND, c = e % ND;
          if (c == 0) {
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
              for (int w = 0; w < 4; ++w)
                p[n][w] = pack2<T>(s[n][8 * h + 2 * w], s[n][8 * h + 2 * w + 1]);
          }
          const u32x4 x2 = by_columns(e + 2);
#pragma unroll
          for (int n = 0; n < NK; ++n) mma_far<T>(x0, p[n], dv[n][c]);
          if (2 * c % ND == 0) {
            const int r = 8 * h + 8 * c / ND;
            const f32x4 z1 = r + 4 < 16 ? delta_of(r + 4) : z;
#pragma unroll
            for (int n = 0; n < NK; ++n) {
              float x[4];
#pragma unroll
              for (int w = 0; w < 4; ++w) x[w] = s[n][r + w] * (dp[n][r + w] - z[w]);
              ds[h][n][r % 8 / 2] = pack2<T>(x[0], x[1]);
              ds[h][n][r % 8 / 2 + 1] = pack2<T>(x[2], x[3]);
            }
            z = z1;
          }
          x0 = x1, x1 = x2;
          __builtin_amdgcn_sched_barrier(0);
        }
        // dK
#pragma unroll
        for (int e = 0; e < 2 * ND; ++e) {
          u32x4 x2 = x0;
          if (e + 2 < 2 * ND) x2 = by_columns(2 * ND + e + 2);
#pragma unroll
          for (int n = 0; n < NK; ++n) mma_far<T>(x0, ds[e / ND][n], dk[n][e % ND]);
          x0 = x1, x1 = x2;
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      arrived<(2 * Fetch::units + 1) * (NB - 2)>();
      __syncthreads();
    }
  }
  finished();                                // (what was fetched beyond the last, too)
  __syncthreads();

  // The row waves' sums, a block of keys at a time: the first is given the other's dK,
  // the second the first's dV, each adds its own; then rows to memory.
  constexpr int kBlock = ND * 4096;          // bytes of a block's sums
  static_assert(kWaves * 32 * D * 4 / WD <= kTiles * kTile && kWaves * kBlock <= kTiles * kTile * WD,
                "room for the sums");
  static_assert(kWaves * 32 * NK * L::row_bytes <= kTiles * kTile * WR * WD, "room for the results");
  if (skipped) s_skipped = 1;
  // The rows that were left out, pair by pair, those alone that see the key: added to
  // the sums [32 keys][D] that lie in LDS.
  auto left_out = [&](int n, bool is_dk, float* sums) INLINE {
    const int64_t token = keys.start + min(key_of(n, lane), keys.n - 1);
    const int from = first_row(min(key_of(n, lane), keys.n - 1));
    const T* k_row = reinterpret_cast<const T*>(a.k + token * a.k_stride) + head * D;
    const T* v_row = reinterpret_cast<const T*>(a.v + token * a.v_stride) + head * D;
    const T *q, *g;
    float row_lse, row_delta;
    auto at_row = [&](int row) INLINE {
      const int tok = token_of(bt, row), h = head * bt.G + row - tok * bt.G;
      const int64_t to = rows.start + tok;
      q = reinterpret_cast<const T*>(a.q + to * a.q_stride) + h * D;
      g = reinterpret_cast<const T*>(a.d_out + to * a.d_out_stride) + h * D;
      row_lse = a.lse2[to * bt.h_q + h], row_delta = a.delta[to * bt.h_q + h];
    };
#pragma unroll 1
    for (int row0 = r0 * RT; row0 < min(r1 * RT, end); row0 += 32) {
      if (!partial(row0 / RT)) continue;
      at_row(min(row0 + i, end - 1));
      bool bad = row_lse != row_lse || !(fabsf(row_delta) < INFINITY);
#pragma unroll 1
      for (int d = k; d < D; d += 2)
        bad = bad || !(fabsf((float)q[d]) < INFINITY) || !(fabsf((float)g[d]) < INFINITY);
      if (!__any(bad)) continue;
#pragma unroll 1
      for (int row = max(row0, from); row < min(row0 + 32, end); ++row) {
        at_row(row);
        float s = 0.f, dp = 0.f;
#pragma unroll 1
        for (int d = 0; d < D; ++d) {
          s += (float)q[d] * (float)k_row[d];
          dp += (float)g[d] * (float)v_row[d];
        }
        float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s, a.scale2, -row_lse));
        if (is_dk) w *= dp - row_delta;
        if constexpr (!is_f32<T>) w = (float)(T)w;
        const T* of = is_dk ? q : g;
#pragma unroll 1
        for (int d = k; d < D; d += 2) sums[i * D + d] += w * (float)of[d];
      }
    }
  };
  auto shared = [&](int to, int c) INLINE {
    return reinterpret_cast<f32x4*>(s_rows[0] + (to * WK + wk) * kBlock + c * 4096) + lane;
  };
  auto part_of = [&](int n, bool is_dk, int x) INLINE {
    return a.parts +
           (((int64_t)blockIdx.x * 2 + !is_dk) * F::keys + 32 * (NK * wk + n) + x) * D;
  };
  auto finish = [&](int n, f32x16 (&mine)[ND], f32x16 (&theirs)[ND], bool is_dk) INLINE {
    if constexpr (WR == 2) {
#pragma unroll
      for (int c = 0; c < ND; ++c) {
        settle(theirs[c]);
        const f32x16 x = theirs[c];
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          shared(1 - wr, c)[16 * r] = f32x4{x[r], x[r + 1], x[r + 2], x[r + 3]};
      }
      __syncthreads();
    }
#pragma unroll
    for (int c = 0; c < ND; ++c) {
      settle(mine[c]);
      if constexpr (WR == 2) {
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const f32x4 y = shared(wr, c)[16 * r];
#pragma unroll
          for (int e = 0; e < 4; ++e) mine[c][r + e] += y[e];
        }
      }
    }
    __syncthreads();
    const float by = is_dk ? a.scale : 1.f;
    if (__builtin_expect(uniform(s_skipped), 0)) {
      float* sums = reinterpret_cast<float*>(s_rows[0]) + (WD > 1 ? 0 : wave) * 32 * D;
#pragma unroll
      for (int c = 0; c < ND; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          sums[i * D + 32 * (ND * wd + c) + 8 * (r / 4) + 4 * k + r % 4] = mine[c][r];
      __syncthreads();
      if (wd == 0) {
        left_out(n, is_dk, sums);
        const int64_t token = keys.start + key_of(n, lane);
        if (a.key_splits > 1) {
          float* part = part_of(n, is_dk, i);
#pragma unroll 1
          for (int d = k; d < D; d += 2) part[d] = sums[i * D + d];
        } else if (key_of(n, lane) < keys.n) {
          T* dst = reinterpret_cast<T*>(is_dk ? a.dk + token * a.dk_stride
                                              : a.dv + token * a.dv_stride) + head * D;
#pragma unroll 1
          for (int d = k; d < D; d += 2) dst[d] = (T)(sums[i * D + d] * by);
        }
      }
      __syncthreads();
      return;
    }
    if (a.key_splits > 1) {
#pragma unroll
      for (int c = 0; c < ND; ++c)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<f32x4*>(part_of(n, is_dk, i) + 32 * (ND * wd + c) + 2 * r + 4 * k) =
              f32x4{mine[c][r], mine[c][r + 1], mine[c][r + 2], mine[c][r + 3]};
      return;
    }
    // (waves that share keys have dimensions of their own, in one place)
    char* tile = s_rows[0] + (WD > 1 ? 0 : wave) * 32 * L::row_bytes;
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        put4<T, D>(tile, i, 32 * (ND * wd + c) + 2 * r + 4 * k,
                   f32x4{mine[c][r], mine[c][r + 1], mine[c][r + 2], mine[c][r + 3]} *
                       by);
    if constexpr (WD > 1) __syncthreads();
    if (wd == 0)
      store_rows<T, D>(tile, 32, lane, [&](int x) INLINE {
        const int key = key_of(n, x);
        if (key >= keys.n) return (char*)nullptr;
        const int64_t token = keys.start + key;
        return (is_dk ? a.dk + token * a.dk_stride : a.dv + token * a.dv_stride) +
               (int64_t)head * L::row_bytes;
      });
    __syncthreads();
  };
#pragma unroll
  for (int n = 0; n < NK; ++n) {
    if constexpr (WR == 1) {
      finish(n, dk[n], dv[n], true);
      finish(n, dv[n], dk[n], false);
    } else if (wr == 0) {
      finish(n, dk[n], dv[n], true);
    } else {
      finish(n, dv[n], dk[n], false);
    }
  }
}

// ---------------------------------------------------------------------------
// Adds the parts of a tile's rows (is_rows: of dQ; else its keys', of dK and dV), in
// their order, D/4 lanes a row.
// ---------------------------------------------------------------------------
template <class T, int D, bool is_rows>
__global__ __launch_bounds__(kThreads) void prompt_grad_merge_kernel(Batch bt, GradArgs a, int R) {
  constexpr int kPer = D / 4;
  const int tid = threadIdx.x, l = tid % kPer;
  const int head = blockIdx.x % bt.h_kv, item = blockIdx.x / bt.h_kv;
  const int splits = is_rows ? a.row_splits : a.key_splits;
  Place at;
  if (!find(bt, is_rows, R, item, tid & 63, &at)) return;
  const int x = blockIdx.y * (kThreads / kPer) + tid / kPer;
  const int row = (is_rows ? at.after : at.tiles - 1 - at.after) * R + x;
  if (x >= R || row >= (is_rows ? at.rows.n * bt.G : at.keys.n)) return;
  const int tok = is_rows ? token_of(bt, row) : row;
  const int64_t token = (is_rows ? at.rows.start : at.keys.start) + (int64_t)tok;
  const int64_t in = (int64_t)(is_rows ? head * bt.G + row - tok * bt.G : head) * D * sizeof(T);
#pragma unroll
  for (int which = 0; which < (is_rows ? 1 : 2); ++which) {
    f32x4 sum{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s) {
      const int64_t group = (int64_t)(item * splits + s) * bt.h_kv + head;
      const int64_t first = is_rows ? group * R : (group * 2 + which) * R;
      sum += far_load<f32x4>(a.parts + (first + x) * D + 4 * l);
    }
    char* dst = is_rows ? a.dq + token * a.dq_stride
                        : which ? a.dv + token * a.dv_stride : a.dk + token * a.dk_stride;
    if (is_rows || which == 0) sum *= a.scale;
    if constexpr (is_f32<T>)
      *reinterpret_cast<f32x4*>(dst + in + 16 * l) = sum;
    else
      *reinterpret_cast<u32x2*>(dst + in + 8 * l) =
          u32x2{pack2<T>(sum[0], sum[1]), pack2<T>(sum[2], sum[3])};
  }
}

}  // namespace

namespace {

struct Plan {
  int NQ;                       // blocks of 32 rows a wave
  int64_t row_items, key_items;
  int row_splits, key_splits;
  size_t stat_bytes, bytes;
};

Plan plan_grad(const da_prompt& p) {
  Plan plan{};
  const int64_t G = p.h_q / p.h_kv;
  // d = 64: two blocks of rows a wave for long sequences (16 heads, us with two and with one:
  // 4 sequences of 4096 rows 235 and 243, 8 of 1500 that see all 132 and 135, 16 of 512 38
  // and 35, 32 of 300 54 and 40).  The workspace is the same whether causal or not.
  plan.NQ = p.dtype != DA_F32 && p.d == 64 && p.keys / p.B >= 1500 ? 2 : 1;
  with_type_and_dim(p.dtype, p.d, [&](auto t, auto d) {
    using T = typename decltype(t)::type;
    plan.row_items = most_tiles(p.row_start, p.B, p.T, p.rows, G, 128 * plan.NQ);
    plan.key_items =
        most_tiles(p.key_start, p.B, p.N, p.keys, 1, KeysForm<T, d.value>::keys);
  });
  // Few tiles are divided, so that the card is busy (a sequence of 2048 rows, 32/8 heads
  // of 128: dK and dV 234 us whole, 131 in four parts, their sums with it).
  auto parts = [&](int64_t items, int64_t tile, int64_t most, size_t* bytes) {
    const int64_t groups = items * p.h_kv;
    const int splits = groups < kCus ? (int)std::min(2 * kCus / groups, std::max<int64_t>(most, 1)) : 1;
    if (splits > 1) *bytes = std::max(*bytes, (size_t)(groups * splits * tile * p.d) * sizeof(float));
    return splits;
  };
  size_t part_bytes = 0;
  with_type_and_dim(p.dtype, p.d, [&](auto t, auto d) {
    using T = typename decltype(t)::type;
    plan.row_splits = parts(plan.row_items, 128 * plan.NQ, p.N / 256, &part_bytes);
    plan.key_splits =
        parts(plan.key_items, 2 * KeysForm<T, d.value>::keys, p.T * G / 256, &part_bytes);
  });
  plan.stat_bytes = ((size_t)p.rows * p.h_q * 2 * sizeof(float) + 15) & ~(size_t)15;
  plan.bytes = plan.stat_bytes + part_bytes;
  return plan;
}

}  // namespace

extern "C" {

size_t da_prompt_grad_workspace_bytes(const da_prompt* p) {
  if (!p || check_sizes(*p) != DA_OK) return 0;
  return std::max<size_t>(plan_grad(*p).bytes, 16);
}

da_status da_prompt_attn_grad(const da_prompt* prompt, const void* q, int64_t q_stride,
                              const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                              const void* out, const float* lse, const void* d_out,
                              int64_t d_out_stride, float scale, void* dq, int64_t dq_stride,
                              void* dk, int64_t dk_stride, void* dv, int64_t dv_stride,
                              void* workspace, size_t workspace_bytes, void* stream) {
  if (!prompt || !q || !k || !v || !out || !lse || !d_out || !dq || !dk || !dv) return DA_ERR_NULL;
  const da_prompt& p = *prompt;
  const da_status st = check_sizes(p);
  const int64_t wide[] = {q_stride, d_out_stride, dq_stride};
  const int64_t narrow[] = {k_stride, v_stride, dk_stride, dv_stride};
  if (st == DA_ERR_SHAPE) return st;
  for (int64_t x : wide)
    if (!stride_fits(x, p.h_q, p.d, p.dtype)) return DA_ERR_SHAPE;
  for (int64_t x : narrow)
    if (!stride_fits(x, p.h_kv, p.d, p.dtype)) return DA_ERR_SHAPE;
  if (st != DA_OK) return st;
  const Plan plan = plan_grad(p);
  if (plan.row_items * p.h_kv * plan.row_splits > kMaxGroups ||
      plan.key_items * p.h_kv * plan.key_splits > kMaxGroups)
    return DA_ERR_SHAPE;
  for (const void* x : {q, k, v, out, d_out, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!aligned(x, 16)) return DA_ERR_ALIGN;
  if (!starts_aligned(p) || !aligned(lse, 4)) return DA_ERR_ALIGN;
  for (int64_t x : wide)
    if (!stride_aligned(x, p.dtype)) return DA_ERR_ALIGN;
  for (int64_t x : narrow)
    if (!stride_aligned(x, p.dtype)) return DA_ERR_ALIGN;
  if (!std::isfinite(scale)) return DA_ERR_SCALE;
  if (!workspace || workspace_bytes < plan.bytes) return DA_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return DA_ERR_ALIGN;
  const int size = type_bytes(p.dtype);
  GradArgs a{};
  a.q = static_cast<const char*>(q), a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v), a.out = static_cast<const char*>(out);
  a.d_out = static_cast<const char*>(d_out);
  a.lse = lse;
  a.dq = static_cast<char*>(dq), a.dk = static_cast<char*>(dk), a.dv = static_cast<char*>(dv);
  a.q_stride = q_stride * size, a.k_stride = k_stride * size, a.v_stride = v_stride * size;
  a.d_out_stride = d_out_stride * size, a.dq_stride = dq_stride * size;
  a.dk_stride = dk_stride * size, a.dv_stride = dv_stride * size;
  a.scale = scale, a.scale2 = std::min(std::max(scale * kLog2e, -FLT_MAX), FLT_MAX);
  a.lse2 = static_cast<float*>(workspace);
  a.delta = a.lse2 + (int64_t)p.rows * p.h_q;
  a.row_splits = plan.row_splits, a.key_splits = plan.key_splits;
  a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.stat_bytes);
  const Batch bt = device_batch(p);
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  with_type_and_dim(p.dtype, p.d, [&](auto t, auto d) {
    using T = typename decltype(t)::type;
    constexpr int D = d.value, kPass = kThreads / (D / 4);     // rows of a merge's pass
    const unsigned row_groups = (unsigned)(plan.row_items * p.h_kv);
    const unsigned key_groups = (unsigned)(plan.key_items * p.h_kv);
    const dim3 grid(row_groups * plan.row_splits);
    const auto rows = [&](auto nq) {
      hipLaunchKernelGGL((prompt_grad_rows_kernel<T, D, nq.value>), grid, dim3(kThreads), 0, s, bt, a);
    };
    bool done = false;
    if constexpr (!is_f32<T> && D == 64)
      if ((done = plan.NQ == 2)) rows(std::integral_constant<int, 2>{});
    if (!done) rows(std::integral_constant<int, 1>{});
    if (plan.row_splits > 1)
      hipLaunchKernelGGL((prompt_grad_merge_kernel<T, D, true>),
                         dim3(row_groups, 128 * plan.NQ / kPass), dim3(kThreads), 0, s, bt, a,
                         128 * plan.NQ);
    hipLaunchKernelGGL((prompt_grad_keys_kernel<T, D>), dim3(key_groups * plan.key_splits),
                       dim3(kThreads), 0, s, bt, a);
    if (plan.key_splits > 1)
      hipLaunchKernelGGL((prompt_grad_merge_kernel<T, D, false>),
                         dim3(key_groups, KeysForm<T, D>::keys / kPass), dim3(kThreads), 0, s, bt, a,
                         KeysForm<T, D>::keys);
  });
  return launch_status();
}

}  // extern "C"
