// prompt_attn.hip -- gfx950 kernels and C ABI of attention over whole prompts:
// sequences of different lengths packed one after the other, as a projection
// leaves them, without a cache.
//
// Kernels
//   prompt_attn_kernel    softmax(scale q.K) V for a tile of query rows of one
//                         (sequence, KV head), over all keys that they see or a
//                         part of them.
//   prompt_merge_kernel   combines the parts of each row.
//
// Where some rows of a tile see a key that others do not, a weight of 0 would turn an
// infinity of V into NaN: such a tile of V is looked over first, and, where it holds
// one, its pairs are added one by one.
#include <algorithm>
#include <cfloat>

#include "prompt_common.h"

namespace {

using namespace prompt;

struct AttnArgs {
  const char *q, *k, *v;
  char* out;
  float* lse;
  int64_t q_stride, k_stride, v_stride;       // bytes between tokens
  // |scale| times log2(e), or 1 for a scale of 0; q's words are taken as
  // (q & q_keep) ^ q_flip: negated for a negative scale, 0 for that of 0.
  float scale;
  uint32_t q_keep, q_flip;
  int splits;
  float* parts;         // splits > 1: [workgroup][R][D], then [workgroup][R][3]
  int64_t stats;        // where the latter begin
};

// Beyond this distance the rounding of the reference would show: the product is
// rounded first, so that the largest score's weight is 1.
constexpr float kFar = 0x1p26f;

template <class T, int D>
constexpr int kKeys = is_f32<T> || D == 256 ? 32 : 64;     // keys of a tile

// ---------------------------------------------------------------------------
// Attention.  A workgroup's R = 128 NQ rows are (token, head of the group)
// pairs of one KV head, 32 NQ to a wave, side by side as columns:
//   S^T [keys x rows] = K . Q^T,   O^T [D x rows] += V^T . P^T
// so a row's scores lie in two lanes, its statistics need no LDS, and the weights are
// the second product's operand as they lie.  Tiles of K and V go from memory to LDS
// without registers; V is read by columns with the transposing LDS loads.
//
// Two forms.  In turn (NQ = 1, d = 64 and 128): scores, softmax and values of a tile one
// after the other; the two or three workgroups of a CU cover each other's phases, starts
// and ends.  In a pipeline (one workgroup a CU, whose wave has all 512 registers): the
// next tile's scores are multiplied between this one's exponentials, and its maximum is
// found between this one's value products; the sums lie in accumulation registers.
// d = 128, long sequences: two blocks of 32 rows a wave, so that an operand read from
// LDS serves two products (with one, LDS would have to deliver 128 bytes a cycle and CU).
//
// Measured, bfloat16, causal.  One sequence of 16384 rows, 32/8 heads of 128, 2.2
// TFLOP: 2093 us, 1050 TFLOP/s (an 8192^3 library product 1247; the form in turn 784);
// matrix pipes busy for 49 % of the cycles, vector instructions for 44 %, waits 24 %.
// Without the fetches and the barrier a tile's step is 11 % shorter, without the
// exponentials 8 %, without the sums or the maximum 4 %: no one of them bounds it.
// 4 sequences of 4096, 16 heads of 64: 189 us, 728 TFLOP/s, the softmax (14
// instructions for each 64 x 64 multiply-adds).  2 of 4096, 16/4 heads of 256: 353 us,
// 779 TFLOP/s (in turn 517).  16 prompts of 1 to 900 rows, 32/8 heads of 128: 100 us,
// of which starts and ends of workgroups (4 us to the first product) are a third.
// ---------------------------------------------------------------------------
template <int D, int NQ>
constexpr int kGroupsPerCu = NQ == 2 || D == 256 ? 1 : D == 128 ? 2 : 3;

template <class T, int D, int NQ, bool LSE>
__global__ __launch_bounds__(kThreads, (kGroupsPerCu<D, NQ>))
void prompt_attn_kernel(Batch bt, AttnArgs a) {
  constexpr bool kPipe = NQ == 2 || (D == 256 && !is_f32<T>);
  using L = Tile<T, D>;
  constexpr int KT = kKeys<T, D>, R = 32 * NQ * kWaves;
  constexpr int NS = KT / 32, ND = L::ND, NW = L::NW;
  constexpr int kTile = KT * L::row_bytes;
  constexpr int NP = is_f32<T> ? 1 : 2 * NS;
  using Fetch = Direct<T, D, KT>;

  constexpr int NB = kPipe ? 3 : 2;          // tiles in LDS
  // K's and V's tiles in turn; q on its way in, and out on its way out
  __shared__ __align__(1024) char s_all[2 * NB][kTile];
  auto s_k = [&](int t) INLINE { return s_all[2 * (t % NB)]; };
  auto s_v = [&](int t) INLINE { return s_all[2 * (t % NB) + 1]; };
  __shared__ __align__(1024) char s_zero[kPipe ? kTile : 16];
  __shared__ int s_bad[kWaves];

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int i = lane & 31, k = lane >> 5;

  const int head = blockIdx.x % bt.h_kv;
  const int split = (blockIdx.x / bt.h_kv) % a.splits;
  Place at;
  if (!find(bt, true, R, blockIdx.x / bt.h_kv / a.splits, lane, &at)) return;
  const Span rows = at.rows, keys = at.keys;
  const int row0 = at.after * R;             // the last rows, which see most, first
  const int in_tile = min(rows.n * bt.G - row0, R);
  const int min_seen = seen_by(bt, rows.n, keys.n, token_of(bt, row0));
  const int max_seen = seen_by(bt, rows.n, keys.n, token_of(bt, row0 + in_tile - 1));
  const int tiles = (max_seen + KT - 1) / KT;
  const int t0 = (int)((int64_t)tiles * split / a.splits);
  const int t1 = (int)((int64_t)tiles * (split + 1) / a.splits);

  // This wave's rows.
  const int my_row0 = row0 + 32 * NQ * wave;
  const int my_rows = min(max(in_tile - 32 * NQ * wave, 0), 32 * NQ);
  // (without rows there is nothing to mask)
  const int my_min = my_rows ? seen_by(bt, rows.n, keys.n, token_of(bt, my_row0)) : INT32_MAX;
  const int my_max =
      my_rows ? seen_by(bt, rows.n, keys.n, token_of(bt, my_row0 + my_rows - 1)) : 0;
  const char* k_base = a.k + (int64_t)keys.start * a.k_stride + (int64_t)head * L::row_bytes;
  const char* v_base = a.v + (int64_t)keys.start * a.v_stride + (int64_t)head * L::row_bytes;
  const RowReader<T, D> k_read(ordered_row(i), k);
  const ColumnReader<T, D> v_read(lane);

  // Keys beyond the last are zeros, which no row sees.
  int k_byte[Fetch::phases], v_byte[Fetch::phases];
#pragma unroll
  for (int u = 0; u < Fetch::phases; ++u) {
    k_byte[u] = Fetch::row(tid, u) * (int)a.k_stride + Fetch::byte(tid, u);
    v_byte[u] = Fetch::row(tid, u) * (int)a.v_stride + Fetch::byte(tid, u);
  }
  auto window_of = [&](const char* base, int64_t stride, int t) INLINE {
    return window(base + (int64_t)t * KT * stride, ((int64_t)keys.n - (int64_t)t * KT) * stride);
  };
  auto load_k = [&](const Window& from, int t, int u) INLINE {
    fetch(Fetch::place(s_k(t - t0), wave, u), from, k_byte[u % Fetch::phases],
          u / Fetch::phases * (Fetch::phases * Fetch::step) * (int)a.k_stride);
  };
  auto load_v = [&](const Window& from, int t, int u) INLINE {
    fetch(Fetch::place(s_v(t - t0), wave, u), from, v_byte[u % Fetch::phases],
          u / Fetch::phases * (Fetch::phases * Fetch::step) * (int)a.v_stride);
  };
  auto load_all = [&](int t, bool want_k, bool want_v) INLINE {
    const Window from_k = window_of(k_base, a.k_stride, t);
    const Window from_v = window_of(v_base, a.v_stride, t);
#pragma unroll
    for (int u = 0; u < Fetch::units; ++u) {
      if (want_k) load_k(from_k, t, u);
      if (want_v) load_v(from_v, t, u);
    }
  };

  int seen[NQ];
  u32x4 q[NQ][NW];
  // (beside the first keys, where there is room)
  constexpr bool kBeside = (2 * NB - 2) * kTile >= R * L::row_bytes;
  static_assert(2 * NB * kTile >= R * L::row_bytes, "room for the rows");
  static_assert(!kPipe || kBeside, "a pipeline's first keys come with the rows");
  char* q_rows = s_all[kBeside ? 2 : 0];
  fetch_rows<T, D, R>(q_rows, bt,
                      a.q + rows.start * a.q_stride + (int64_t)head * bt.G * L::row_bytes,
                      a.q_stride, row0, row0 + in_tile - 1, tid, wave);
  if (kBeside && t0 < t1) load_all(t0, true, true);
  arrived();
  __syncthreads();
  {
    const RowReader<T, D> rd(i, k);
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      const int x = 32 * b + i;
      seen[b] = x < my_rows ? seen_by(bt, rows.n, keys.n, token_of(bt, my_row0 + x)) : 0;
#pragma unroll
      for (int w = 0; w < NW; ++w)
        q[b][w] = (rd.get(q_rows, NQ * wave + b, w) & a.q_keep) ^ a.q_flip;
    }
  }
  __syncthreads();

  f32x16 acc[NQ][ND];
  float limit[NQ], ref[NQ], sum[NQ], whole[NQ], top[NQ];
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[b][c][r] = 0.f;
    limit[b] = -INFINITY, ref[b] = 0.f, sum[b] = 0.f, whole[b] = 0.f;
  }
  float by = a.scale;

  auto scores = [&](int t, f32x16 (&s)[NQ][NS]) INLINE {
    const char* tile = s_k(t - t0);
#pragma unroll
    for (int b = 0; b < NQ; ++b)
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[b][n][r] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const u32x4 x = k_read.get(tile, n, w);
#pragma unroll
        for (int b = 0; b < NQ; ++b) s[b][n] = mma<T>(x, q[b][w], s[b][n]);
        if (is_f32<T> && w % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
  };
  auto mask = [&](int t, f32x16 (&s)[NQ][NS]) INLINE {
    if ((t + 1) * KT <= my_min) return;
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      const int left = seen[b] - t * KT - 8 * k;
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * n + row_of(r, 0) >= left) s[b][n][r] = -INFINITY;
    }
  };
  auto find_top = [&](const f32x16 (&s)[NQ][NS]) INLINE {
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      top[b] = s[b][0][0];
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) top[b] = fmaxf(top[b], s[b][n][r]);
    }
  };
  // The reference is raised when a score lies 8 above it: weights stay below
  // 2^8, and most tiles rescale nothing.
  auto over = [&]() INLINE {
    bool x = false;
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      top[b] *= a.scale;
      x |= !(top[b] <= limit[b]);
    }
    return __any(x);
  };
  auto raise = [&]() INLINE {
    bool far = false;
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      top[b] = fmaxf(top[b], __shfl_xor(top[b], 32));
      far |= fabsf(top[b]) > kFar && top[b] != -INFINITY;
      if (!(top[b] <= limit[b])) {
        const float f = limit[b] == -INFINITY ? 0.f : exp2f(ref[b] - top[b]);
        ref[b] = top[b];
        limit[b] = top[b] + 8.f;
        sum[b] *= f;
        whole[b] *= f;
#pragma unroll
        for (int c = 0; c < ND; ++c) acc[b][c] *= f;
      }
    }
    if (__any(far)) by = 1.f;
  };
  auto rescore = [&](f32x16 (&s)[NQ][NS]) INLINE {
    if (__builtin_expect(by != a.scale, 0)) {
#pragma unroll
      for (int b = 0; b < NQ; ++b)
#pragma unroll
        for (int n = 0; n < NS; ++n) s[b][n] *= a.scale;
    }
  };
  // Components 8h .. 8h+7 of a block become weights; 16-bit ones are rounded into p, as
  // the matrix instructions take them, and it is the rounded ones that out is divided by
  // the sum of (bfloat16: error 0.0021, 2-norm, where the result's own rounding is 0.0017).
  auto weigh = [&](int b, int h, f32x16& s, u32x4& p) INLINE {
#pragma unroll
    for (int r = 8 * h; r < 8 * h + 8; ++r)
      s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], by, -ref[b]));
    if constexpr (is_f32<T>) {
#pragma unroll
      for (int r = 8 * h; r < 8 * h + 8; ++r) sum[b] += s[r];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = pack2<T>(s[8 * h + 2 * e], s[8 * h + 2 * e + 1]);
        sum[b] = add2<T>(p[e], sum[b]);
        if constexpr (LSE) whole[b] += s[8 * h + 2 * e] + s[8 * h + 2 * e + 1];
      }
    }
  };
  auto weights = [&](f32x16 (&s)[NQ][NS], u32x4 (&p)[NQ][NP]) INLINE {
#pragma unroll
    for (int b = 0; b < NQ; ++b)
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) weigh(b, h, s[b][n], p[b][is_f32<T> ? 0 : 2 * n + h]);
  };
  // Where some rows see keys of a tile that others do not, values that are not finite
  // must not meet the others' weights of 0.  Each wave looks at a quarter of the tile.
  auto spoilt = [&](int t) INLINE {
    constexpr int part = kTile / kWaves;
    const char* tile = s_v(t - t0) + wave * part;
    Finite<T> f;
#pragma unroll
    for (int x = 0; x < part / 1024; ++x)
      f.take(*reinterpret_cast<const u32x4*>(tile + x * 1024 + lane * 16));
    const bool bad = __any(!f.all());
    if (lane == 0) s_bad[wave] = bad;
    __syncthreads();
    int any = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) any |= s_bad[w];
    return uniform(any) != 0;
  };
  auto values = [&](int t, bool bad, f32x16 (&s)[NQ][NS], u32x4 (&p)[NQ][NP]) INLINE {
    const char* tile = s_v(t - t0);
    if (__builtin_expect(bad, 0)) {
      // key by key, those alone that the row sees
#pragma unroll 1
      for (int e = 0; e < 16 * NS; ++e) {
#pragma unroll
        for (int b = 0; b < NQ; ++b) {
          float mine = 0.f;
#pragma unroll
          for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) mine = 16 * n + r == e ? s[b][n][r] : mine;
          if constexpr (!is_f32<T>) mine = (float)(T)mine;
          const float other = __shfl_xor(mine, 32);
#pragma unroll 1
          for (int kk = 0; kk < 2; ++kk) {
            const int key = 32 * (e / 16) + row_of(e % 16, kk);
            if (t * KT + key >= seen[b]) continue;
            const float w = kk == k ? mine : other;
#pragma unroll
            for (int c = 0; c < ND; ++c)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const int d = (32 * c + 8 * (r / 4) + 4 * k + r % 4) * (int)sizeof(T);
                acc[b][c][r] +=
                    w * (float)*reinterpret_cast<const T*>(tile + L::at(key, d / 16) + d % 16);
              }
          }
        }
      }
      return;
    }
    if constexpr (is_f32<T>) {
      // (eight reads at a time: more would not fit the registers)
#pragma unroll
      for (int c = 0; c < ND; ++c)
#pragma unroll
        for (int h = 0; h < 2 * NS; ++h) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = v_read.get(tile, h, e, c);
#pragma unroll
          for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int b = 0; b < NQ; ++b)
              acc[b][c] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], s[b][h / 2][8 * (h % 2) + e],
                                                               acc[b][c], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
    } else {
#pragma unroll
      for (int c = 0; c < ND; ++c)
#pragma unroll
        for (int h = 0; h < 2 * NS; ++h) {
          const u32x4 x = v_read.get(tile, h, c);
#pragma unroll
          for (int b = 0; b < NQ; ++b) acc[b][c] = mma<T>(x, p[b][h], acc[b][c]);
        }
    }
  };

  int t = t0;
  bool skipped = false;
  // In a pipeline: a tile's scores are multiplied while those before become weights,
  // and its largest score is found while those weights meet V.
  if constexpr (kPipe) {
    for (int x = tid; x < kTile / 16; x += kThreads)
      reinterpret_cast<u32x4*>(s_zero)[x] = u32x4{0u, 0u, 0u, 0u};
    if (t0 < t1) {
      load_all(t0 + 1, true, true);
      load_all(t0 + 2, true, false);
      f32x16 sa[NQ][NS], sb[NQ][NS];
      u32x4 p[NQ][NP];
      scores(t0, sa);
      mask(t0, sa);
      find_top(sa);
      if (over()) raise();
      rescore(sa);
      arrived();
      __syncthreads();
      auto step = [&](f32x16 (&s)[NQ][NS], f32x16 (&next)[NQ][NS]) INLINE {
        const char *tile_k = s_k(t + 1 - t0), *tile_v = s_v(t - t0);
        // (such a tile is left out here, zeros in its place, and added at the end)
        if (__builtin_expect((t + 1) * KT > min_seen, 0) && spoilt(t))
          skipped = true, tile_v = s_zero;
#pragma unroll
        for (int b = 0; b < NQ; ++b)
#pragma unroll
          for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) next[b][n][r] = 0.f;
        const Window from_k = window_of(k_base, a.k_stride, t + 3);
        const Window from_v = window_of(v_base, a.v_stride, t + 2);
        u32x4 v0, v1, x[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n) x[n] = k_read.get(tile_k, n, 0);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          u32x4 y[NS];
#pragma unroll
          for (int n = 0; n < NS; ++n) y[n] = w + 1 < NW ? k_read.get(tile_k, n, w + 1) : x[n];
          if (w + 1 == NW) v0 = v_read.get(tile_v, 0, 0), v1 = v_read.get(tile_v, 0, 1);
          if (w == 0) __builtin_amdgcn_sched_barrier(0);
          // weights in pieces of eight, spread over the steps of the product
#pragma unroll
          for (int e = 0; e < NQ * NP; ++e)
            if (e * NW / (NQ * NP) == w) {
              const int b = e / NP, n = e % NP / 2, h = e % 2;
              weigh(b, h, s[b][n], p[b][2 * n + h]);
              asm volatile("" : "+v"(p[b][2 * n + h]));  // (here, not where it is used)
            }
#pragma unroll
          for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int b = 0; b < NQ; ++b) next[b][n] = mma<T>(x[n], q[b][w], next[b][n]);
          if (w < Fetch::units) load_k(from_k, t + 3, w);
          else if (w < 2 * Fetch::units) load_v(from_v, t + 2, w - Fetch::units);
#pragma unroll
          for (int n = 0; n < NS; ++n) x[n] = y[n];
          __builtin_amdgcn_sched_barrier(0);
        }
        if (__builtin_expect((t + 2) * KT > my_min, 0)) mask(t + 1, next);
#pragma unroll
        for (int b = 0; b < NQ; ++b) top[b] = next[b][0][0];
#pragma unroll
        for (int e = 0; e < NP * ND; ++e) {
          u32x4 v2 = v0;
          if (e + 2 < NP * ND) v2 = v_read.get(tile_v, (e + 2) / ND, (e + 2) % ND);
#pragma unroll
          for (int b = 0; b < NQ; ++b) mma_far<T>(v0, p[b][e / ND], acc[b][e % ND]);
          constexpr int kEach = 16 * NS / (NP * ND);    // scores of a row's lane, a step
#pragma unroll
          for (int b = 0; b < NQ; ++b)
#pragma unroll
            for (int r = e * kEach; r < (e + 1) * kEach; ++r)
              top[b] = fmaxf(top[b], next[b][r / 16][r % 16]);
          v0 = v1, v1 = v2;
          __builtin_amdgcn_sched_barrier(0);
        }
        arrived<2 * Fetch::units>();                    // but those of this step
        __syncthreads();
      };
      // (The sums are in accumulation registers within the inner loop: what changes
      // them otherwise stands outside.  Which scores are next is hidden from the
      // compiler, so that it copies them outside too.)
      bool again = true;
      while (again) {
        again = false;
        int second = 0;
        while (t < t1) {
          step(sa, sb);
          ++t, second = 1;
          again = over();
          if (again || t >= t1) break;
          rescore(sb);
          step(sb, sa);
          ++t, second = 0;
          again = over();
          if (again) break;
          rescore(sa);
        }
#pragma unroll
        for (int b = 0; b < NQ; ++b)
#pragma unroll
          for (int c = 0; c < ND; ++c) settle(acc[b][c]);
        asm volatile("" : "+s"(second));
        if (second) {
#pragma unroll
          for (int b = 0; b < NQ; ++b)
#pragma unroll
            for (int n = 0; n < NS; ++n) sa[b][n] = sb[b][n];
        }
        if (again) raise();
        if (again || second) rescore(sa);
      }
      arrived();                             // (what was fetched beyond the last)
      __syncthreads();
    }
  }
  if (!kPipe && t < t1) {
    if (!kBeside) {
      load_all(t, true, true);
      arrived();
      __syncthreads();
    }
    for (; t < t1; ++t) {
      if (t + 1 < t1) load_all(t + 1, true, true);
      const bool bad = (t + 1) * KT > min_seen && spoilt(t);
      if (t * KT < my_max) {
        f32x16 s[NQ][NS];
        u32x4 p[NQ][NP];
        scores(t, s);
        mask(t, s);
        find_top(s);
        if (over()) raise();
        rescore(s);
        weights(s, p);
        values(t, bad, s, p);
      }
      arrived();
      __syncthreads();
    }
  }

  // The keys that were left out, those alone that the row sees: the sums pass through
  // LDS in 32 bits, 32 rows of one wave at a time.
  if (kPipe && __builtin_expect(skipped, 0)) {
    float* sums = reinterpret_cast<float*>(s_all[0]) + i * D;
    for (int w = 0; w < kWaves; ++w) {
#pragma unroll
      for (int b = 0; b < NQ; ++b) {
        __syncthreads();
        if (w != wave) continue;
#pragma unroll
        for (int c = 0; c < ND; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r) sums[32 * c + 8 * (r / 4) + 4 * k + r % 4] = acc[b][c][r];
        __builtin_amdgcn_wave_barrier();
        const int x = my_row0 + min(32 * b + i, max(my_rows - 1, 0));
        const int tok = my_rows ? token_of(bt, x) : 0, g = my_rows ? x - tok * bt.G : 0;
        const T* q_row = reinterpret_cast<const T*>(a.q + (rows.start + tok) * a.q_stride) +
                         (head * bt.G + g) * D;
#pragma unroll 1
        for (int key0 = max(min_seen / KT, t0) * KT; key0 < min(max_seen, t1 * KT); key0 += KT) {
          bool bad = false;
          for (int key = key0 + i; key < min(key0 + KT, keys.n); key += 32) {
            const T* row = reinterpret_cast<const T*>(v_base + key * a.v_stride);
#pragma unroll 1
            for (int d = k; d < D; d += 2) bad = bad || !(fabsf((float)row[d]) < INFINITY);
          }
          if (!__any(bad)) continue;
#pragma unroll 1
          for (int key = key0; key < min(key0 + KT, seen[b]); ++key) {
            const T* k_row = reinterpret_cast<const T*>(k_base + key * a.k_stride);
            const T* v_row = reinterpret_cast<const T*>(v_base + key * a.v_stride);
            float s = 0.f;
#pragma unroll 1
            for (int d = 0; d < D; ++d) s += (float)q_row[d] * (float)k_row[d];
            s = a.q_keep ? a.q_flip ? -s : s : 0.f;
            if (by != a.scale) s *= a.scale;
            const float w = (float)(T)__builtin_amdgcn_exp2f(__builtin_fmaf(s, by, -ref[b]));
#pragma unroll 1
            for (int d = k; d < D; d += 2) sums[d] += w * (float)v_row[d];
          }
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int c = 0; c < ND; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[b][c][r] = sums[32 * c + 8 * (r / 4) + 4 * k + r % 4];
      }
    }
    __syncthreads();
  }
  char* mine = s_all[0] + 32 * NQ * wave * L::row_bytes;
  auto place = [&](int x) INLINE {           // row * h_q + head of this wave's row x
    const int tok = token_of(bt, my_row0 + x);
    return (int64_t)(rows.start + tok) * bt.h_q + head * bt.G + my_row0 + x - tok * bt.G;
  };
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
    const float total = sum[b] + __shfl_xor(sum[b], 32);
    const float all = LSE && !is_f32<T> ? whole[b] + __shfl_xor(whole[b], 32) : total;
    // (a row whose scores are all -infinity counts as one that sees nothing)
    const bool none = limit[b] == -INFINITY && total == 0.f;
    const bool here = 32 * b + i < my_rows && k == 0;
    if (a.splits == 1) {
      const float inverse = 1.f / total;
      auto mean = [&](float x) INLINE { return none ? 0.f : x * inverse; };
#pragma unroll
      for (int c = 0; c < ND; ++c)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          put4<T, D>(mine, 32 * b + i, 32 * c + 2 * r + 4 * k,
                     f32x4{mean(acc[b][c][r]), mean(acc[b][c][r + 1]), mean(acc[b][c][r + 2]),
                           mean(acc[b][c][r + 3])});
      if (a.lse && here)
        a.lse[place(32 * b + i)] = none ? -INFINITY : (ref[b] + log2f(all)) * kLn2;
    } else if (32 * b + i < my_rows) {
      const int64_t row = (int64_t)blockIdx.x * R + 32 * NQ * wave + 32 * b + i;
      float* dst = a.parts + row * D + 4 * k;
#pragma unroll
      for (int c = 0; c < ND; ++c)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<f32x4*>(dst + 32 * c + 2 * r) =
              f32x4{acc[b][c][r], acc[b][c][r + 1], acc[b][c][r + 2], acc[b][c][r + 3]};
      if (here) {
        float* st = a.parts + a.stats + row * 3;
        st[0] = none ? -INFINITY : ref[b], st[1] = total, st[2] = all;
      }
    }
  }
  if (a.splits == 1)
    store_rows<T, D>(mine, 32 * NQ, lane, [&](int x) INLINE {
      return x < my_rows ? a.out + place(x) * L::row_bytes : nullptr;
    });
}

// ---------------------------------------------------------------------------
// Puts the parts of each row together, D/4 lanes a row: 4 us for few, loads that
// wait for each other; 11 us for 26 MB of parts.
// ---------------------------------------------------------------------------
template <class T, int D>
__global__ __launch_bounds__(kThreads) void prompt_merge_kernel(Batch bt, AttnArgs a, int R) {
  constexpr int kPer = D / 4;                  // lanes of a row
  const int tid = threadIdx.x, lane = tid & 63;
  const int head = blockIdx.x % bt.h_kv, item = blockIdx.x / bt.h_kv;
  Place at;
  if (!find(bt, true, R, item, lane, &at)) return;
  const Span rows = at.rows;
  const int row0 = at.after * R;
  const int in_tile = min(rows.n * bt.G - row0, R);
  const int x = blockIdx.y * (kThreads / kPer) + tid / kPer, l = tid % kPer;
  if (x >= in_tile) return;
  const int t = token_of(bt, row0 + x), g = row0 + x - t * bt.G;
  const int64_t place = (int64_t)(rows.start + t) * bt.h_q + head * bt.G + g;
  auto part = [&](int s) INLINE {
    return ((int64_t)(item * a.splits + s) * bt.h_kv + head) * R + x;
  };
  float ref = -INFINITY;
  bool bad = false;                            // (a NaN is no maximum)
  for (int s = 0; s < a.splits; ++s) {
    const float m = a.parts[a.stats + part(s) * 3];
    bad |= m != m;
    ref = fmaxf(ref, m);
  }
  f32x4 o{0.f, 0.f, 0.f, 0.f};
  float total = 0.f, all = 0.f;
  for (int s = 0; s < a.splits; ++s) {
    // (a part with no score above -infinity counts too: its weights of 0 may have met a
    // value that is not finite)
    const float* st = a.parts + a.stats + part(s) * 3;
    const float f = bad ? NAN : st[0] == ref ? 1.f : exp2f(st[0] - ref);
    total += f * st[1], all += f * st[2];
    o += f * *reinterpret_cast<const f32x4*>(a.parts + part(s) * D + 4 * l);
  }
  const bool none = ref == -INFINITY && !bad;
  o = none ? f32x4{0.f, 0.f, 0.f, 0.f} : o * (1.f / total);
  char* dst = a.out + place * D * (int)sizeof(T);
  if constexpr (is_f32<T>)
    *reinterpret_cast<f32x4*>(dst + 16 * l) = o;
  else
    *reinterpret_cast<u32x2*>(dst + 8 * l) = u32x2{pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
  if (a.lse && l == 0) a.lse[place] = none ? -INFINITY : (ref + log2f(all)) * kLn2;
}

}  // namespace

namespace {

// How a call is divided: NQ blocks of 32 rows a wave, and the parts that the keys
// of a tile of rows are read in.
struct Plan {
  int NQ, splits;
  int64_t items;                // tiles of rows, over all sequences
  size_t bytes;
};

Plan plan_attn(const da_prompt& p) {
  Plan plan{1, 1, 0, 0};
  const int64_t G = p.h_q / p.h_kv;
  // Two blocks of rows a wave halve what each product reads from LDS, but leave one
  // workgroup a CU, which nothing covers while it starts and ends: worth it where a row
  // tile has many key tiles.  d = 128, 32/8 heads, causal, us with two and with one:
  // one sequence of 16384 rows 2099 and 2804, 4 of 2048 190 and 190, 16 of 512 95 and
  // 74.  d = 64 (4 of 4096, 16 heads: 240 and 186) is bound by the softmax.
  plan.items = most_tiles(p.row_start, p.B, p.T, p.rows, G, 256);
  const int64_t seen = p.keys / p.B / (p.causal ? 2 : 1);
  if (p.dtype != DA_F32 && p.d == 128 && seen >= 1024 && plan.items * p.h_kv >= kCus) {
    plan.NQ = 2;
    return plan;
  }
  plan.items = most_tiles(p.row_start, p.B, p.T, p.rows, G, 128);
  const int64_t groups = plan.items * p.h_kv;
  // Few tiles are divided by their keys, so that every CU has work; more of float32 with
  // heads of 64, whose products take longer than the merge's launch, in parts of 512 keys
  // and more (us whole, in two and in three parts, causal: 384 tiles of 2 sequences of 1500
  // rows 151, 114, 114; 320 of one of 4000 346, 247, 209; 256 of 4 of 1024 84, 68, 65; 360
  // of 6 of 520 59, 62, 62; 280 of 5 of 400 41, 41, 42; 312 of 3 of 1600 that see all 220,
  // 173, 161).  bfloat16, 8 of 333 rows over 400 to 1500 keys: 39 and 45.
  if (groups < kCus)
    plan.splits = (int)std::min<int64_t>(2 * kCus / groups, ceil_div(p.N, 128));
  else if (p.dtype == DA_F32 && p.d == 64 && groups < 3 * kCus)
    plan.splits = (int)std::max<int64_t>(std::min<int64_t>(3 * kCus / groups, p.N / 512), 1);
  if (plan.splits > 1)
    plan.bytes = (size_t)(groups * plan.splits * 128) * (p.d + 3) * sizeof(float);
  return plan;
}

template <class T, int D, int NQ>
void launch_rows(const Plan& plan, const Batch& bt, const AttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(plan.items * bt.h_kv * plan.splits)), block(kThreads);
  if (a.lse && !is_f32<T>)
    hipLaunchKernelGGL((prompt_attn_kernel<T, D, NQ, !is_f32<T>>), grid, block, 0, s, bt, a);
  else
    hipLaunchKernelGGL((prompt_attn_kernel<T, D, NQ, false>), grid, block, 0, s, bt, a);
}

template <class T, int D>
void launch_attn(const Plan& plan, const Batch& bt, const AttnArgs& a, hipStream_t s) {
  if constexpr (!is_f32<T> && D == 128) {
    if (plan.NQ == 2) return launch_rows<T, D, 2>(plan, bt, a, s);
  }
  launch_rows<T, D, 1>(plan, bt, a, s);
  if (plan.splits > 1) {
    const int R = 128;
    const int rows = (int)std::min<int64_t>((int64_t)bt.T * bt.G, R);
    hipLaunchKernelGGL((prompt_merge_kernel<T, D>),
                       dim3((unsigned)(plan.items * bt.h_kv),
                            (unsigned)ceil_div(rows, kThreads / (D / 4))),
                       dim3(kThreads), 0, s, bt, a, R);
  }
}

}  // namespace

extern "C" {

size_t da_prompt_workspace_bytes(const da_prompt* p) {
  if (!p || check_sizes(*p) != DA_OK) return 0;
  return std::max<size_t>(plan_attn(*p).bytes, 16);
}

da_status da_prompt_attn(const da_prompt* prompt, const void* q, int64_t q_stride, const void* k,
                         int64_t k_stride, const void* v, int64_t v_stride, float scale, void* out,
                         float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (!prompt || !q || !k || !v || !out) return DA_ERR_NULL;
  const da_prompt& p = *prompt;
  const da_status st = check_sizes(p);
  if (st == DA_ERR_SHAPE || !stride_fits(q_stride, p.h_q, p.d, p.dtype) ||
      !stride_fits(k_stride, p.h_kv, p.d, p.dtype) || !stride_fits(v_stride, p.h_kv, p.d, p.dtype))
    return DA_ERR_SHAPE;
  if (st != DA_OK) return st;
  const Plan plan = plan_attn(p);
  if (plan.items * p.h_kv * plan.splits > kMaxGroups) return DA_ERR_SHAPE;
  if (!starts_aligned(p) || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) ||
      !aligned(out, 16) || !aligned(lse, 4) || !stride_aligned(q_stride, p.dtype) ||
      !stride_aligned(k_stride, p.dtype) || !stride_aligned(v_stride, p.dtype))
    return DA_ERR_ALIGN;
  if (!std::isfinite(scale)) return DA_ERR_SCALE;
  if (plan.bytes && (!workspace || workspace_bytes < plan.bytes)) return DA_ERR_WORKSPACE;
  if (plan.bytes && !aligned(workspace, 16)) return DA_ERR_ALIGN;
  const int size = type_bytes(p.dtype);
  AttnArgs a{};
  a.q = static_cast<const char*>(q), a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v), a.out = static_cast<char*>(out);
  a.lse = lse;
  a.q_stride = q_stride * size, a.k_stride = k_stride * size, a.v_stride = v_stride * size;
  a.scale = scale == 0.f ? 1.f : std::min(std::fabs(scale) * kLog2e, FLT_MAX);
  a.q_keep = scale == 0.f ? 0u : ~0u;
  a.q_flip = scale < 0.f ? (p.dtype == DA_F32 ? 0x80000000u : 0x80008000u) : 0u;
  a.splits = plan.splits;
  a.parts = static_cast<float*>(workspace);
  a.stats = plan.items * p.h_kv * plan.splits * 128 * p.d;
  const Batch bt = device_batch(p);
  (void)hipGetLastError();
  with_type_and_dim(p.dtype, p.d, [&](auto t, auto d) {
    launch_attn<typename decltype(t)::type, d.value>(plan, bt, a, static_cast<hipStream_t>(stream));
  });
  return launch_status();
}

}  // extern "C"
