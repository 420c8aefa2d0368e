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
//
// Two passes compute the scores twice (seven products for five), and every sum
// has one order: no atomics, equal calls give equal bits.
#include <algorithm>

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
  uint32_t q_keep;              // 0 for a scale of 0, which takes q for 0
  f32x2* stats;                 // [rows][h_q]: lse times log2(e) (+infinity: no weights), delta
};

// Element (row, d) of a tile in LDS.
template <class T, int D>
__device__ __forceinline__ float element(const char* tile, int row, int d) {
  const int byte = d * (int)sizeof(T);
  return (float)*reinterpret_cast<const T*>(tile + Tile<T, D>::at(row, byte / 16) + byte % 16);
}

// acc += X^T w where only the pairs that `sees` allows are multiplied: what the
// others would multiply by 0 may be an infinity or a NaN.  w holds this lane's
// half of the rows of a block of 32 of X.
template <class T, int D, int ND, class F>
__device__ __forceinline__ void add_seen(const char* tile, int row0, int d0, f32x16 w, int k,
                                         f32x16 (&acc)[ND], F&& sees) {
#pragma unroll 1
  for (int e = 0; e < 16; ++e) {
    float mine = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) mine = r == e ? w[r] : mine;
    if constexpr (!is_f32<T>) mine = (float)(T)mine;
    const float other = __shfl_xor(mine, 32);
#pragma unroll 1
    for (int kk = 0; kk < 2; ++kk) {
      const int row = row0 + row_of(e, kk);
      if (!sees(row)) continue;
      const float x = kk == k ? mine : other;
#pragma unroll
      for (int c = 0; c < ND; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          acc[c][r] += x * element<T, D>(tile, row, d0 + 32 * c + 8 * (r / 4) + 4 * k + r % 4);
    }
  }
}

// acc[c] += X^T w over a block of 32 rows of X, from row 32 n of the tile on,
// dimensions d0 + 32 c.
template <class T, int D, int ND, int NB>
__device__ __forceinline__ void add_columns(const ColumnReader<T, D>& rd, const char* tile, int n,
                                            int c0, const f32x16 (&w)[NB],
                                            f32x16 (&acc)[NB][ND]) {
  if constexpr (is_f32<T>) {
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = rd.get(tile, 2 * n + r / 8, r % 8, c0 + c);
#pragma unroll
        for (int b = 0; b < NB; ++b)
          acc[b][c] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, w[b][r], acc[b][c], 0, 0, 0);
      }
  } else {
    u32x4 p[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; r += 2) p[b][r / 8][r % 8 / 2] = pack2<T>(w[b][r], w[b][r + 1]);
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x4 x = rd.get(tile, 2 * n + h, c0 + c);
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b][c] = mma<T>(x, p[b][h], acc[b][c]);
      }
  }
}

// Four dimensions of a row.
template <class T>
__device__ __forceinline__ void store4(char* row, int d, f32x4 x) {
  if constexpr (is_f32<T>)
    *reinterpret_cast<f32x4*>(row + 4 * d) = x;
  else
    *reinterpret_cast<u32x2*>(row + 2 * d) = u32x2{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3])};
}

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
//   S^T = K . Q^T, dP^T = V . dO^T, dQ^T += K^T . dS^T.
// ---------------------------------------------------------------------------
template <class T, int D, int NQ>
__global__ __launch_bounds__(kThreads, 1) void prompt_grad_rows_kernel(Batch bt, GradArgs a) {
  using L = Tile<T, D>;
  constexpr int KT = 32, R = 32 * NQ * kWaves;
  constexpr int ND = L::ND, NW = L::NW;
  constexpr int kTile = KT * L::row_bytes;

  __shared__ __align__(16) char s_k[2][kTile];
  __shared__ __align__(16) char s_v[2][kTile];
  __shared__ int s_spoilt[2][kWaves];

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int i = lane & 31, k = lane >> 5;
  const int head = blockIdx.x % bt.h_kv;
  Place at;
  if (!find(bt.row_start, bt.B, bt.T, bt.rows, bt.G, R, blockIdx.x / bt.h_kv, lane, &at)) return;
  const Span rows = span(bt.row_start, at.b, bt.T, bt.rows);
  const Span keys = span(bt.key_start, at.b, bt.N, bt.keys);
  const int row0 = (bt.causal ? at.tiles - 1 - at.tile : at.tile) * R;
  const int in_tile = min(rows.n * bt.G - row0, R);
  const int min_seen = seen_by(bt, rows.n, keys.n, token_of(bt, row0));
  const int max_seen = seen_by(bt, rows.n, keys.n, token_of(bt, row0 + in_tile - 1));
  const int t1 = (max_seen + KT - 1) / KT;

  const int my_row0 = row0 + 32 * NQ * wave;
  const int my_rows = min(max(in_tile - 32 * NQ * wave, 0), 32 * NQ);
  const int my_min = my_rows ? seen_by(bt, rows.n, keys.n, token_of(bt, my_row0)) : 0;
  int seen[NQ];
  int64_t to[NQ];
  float lse2[NQ], delta[NQ];
  u32x4 q[NQ][NW], g[NQ][NW];
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
    const bool mine = 32 * b + i < my_rows;
    const int x = my_row0 + min(32 * b + i, max(my_rows - 1, 0));
    const int t = my_rows ? token_of(bt, x) : 0;
    const int h = head * bt.G + (my_rows ? x - t * bt.G : 0);
    seen[b] = mine ? seen_by(bt, rows.n, keys.n, t) : 0;
    const int64_t token = rows.start + t, place = token * bt.h_q + h;
    to[b] = token * a.dq_stride + (int64_t)h * L::row_bytes;
    const int64_t in = (int64_t)h * L::row_bytes + 16 * k;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      q[b][w] = *reinterpret_cast<const u32x4*>(a.q + token * a.q_stride + in + 32 * w) & a.q_keep;
      g[b][w] = *reinterpret_cast<const u32x4*>(a.d_out + token * a.d_out_stride + in + 32 * w);
      const u32x4 o = *reinterpret_cast<const u32x4*>(a.out + place * L::row_bytes + 16 * k + 32 * w);
      sum = dot16<T>(g[b][w], o, sum);
    }
    delta[b] = sum + __shfl_xor(sum, 32);
    const float lse = a.lse[place];
    lse2[b] = lse == -INFINITY ? INFINITY : lse * kLog2e;
    if (mine && k == 0) a.stats[place] = f32x2{lse2[b], delta[b]};
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
  Stage<T, D, KT> k_next, v_next;
  const RowReader<T, D> read(ordered_row(i), k);
  const ColumnReader<T, D> read_columns(lane);

  auto load = [&](int t) {
    k_next.load(k_base, a.k_stride, t * KT, keys.n, tid);
    v_next.load(v_base, a.v_stride, t * KT, keys.n, tid);
  };
  auto store = [&](int t) {
    k_next.store(s_k[t & 1], tid);
    v_next.store(s_v[t & 1], tid);
    if ((t + 1) * KT > min_seen) {
      const bool bad = __any(k_next.spoilt());
      if (lane == 0) s_spoilt[t & 1][wave] = bad;
    }
  };

  if (t1 > 0) {
    load(0);
    store(0);
    __syncthreads();
    for (int t = 0; t < t1; ++t) {
      if (t + 1 < t1) load(t + 1);
      if (my_rows) {
        const char *tile_k = s_k[t & 1], *tile_v = s_v[t & 1];
        f32x16 s[NQ], dp[NQ];
#pragma unroll
        for (int b = 0; b < NQ; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[b][r] = 0.f, dp[b][r] = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const u32x4 x = read.get(tile_k, 0, w);
#pragma unroll
          for (int b = 0; b < NQ; ++b) s[b] = mma<T>(x, q[b][w], s[b]);
        }
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const u32x4 x = read.get(tile_v, 0, w);
#pragma unroll
          for (int b = 0; b < NQ; ++b) dp[b] = mma<T>(x, g[b][w], dp[b]);
        }
#pragma unroll
        for (int b = 0; b < NQ; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            s[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], a.scale2, -lse2[b])) *
                      (dp[b][r] - delta[b]);
        bool slow = false;
        if ((t + 1) * KT > my_min) {
#pragma unroll
          for (int b = 0; b < NQ; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (t * KT + row_of(r, k) >= seen[b]) s[b][r] = 0.f;
          int bad = 0;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) bad |= s_spoilt[t & 1][w];
          slow = uniform(bad);
        }
        if (__builtin_expect(slow, 0)) {
#pragma unroll
          for (int b = 0; b < NQ; ++b)
            add_seen<T, D>(tile_k, 0, 0, s[b], k, acc[b],
                           [&](int key) { return t * KT + key < seen[b]; });
        } else {
          add_columns<T, D, ND, NQ>(read_columns, tile_k, 0, 0, s, acc);
        }
      }
      if (t + 1 < t1) store(t + 1);
      __syncthreads();
    }
  }

#pragma unroll
  for (int b = 0; b < NQ; ++b)
    if (32 * b + i < my_rows) {
      char* dst = a.dq + to[b];
#pragma unroll
      for (int c = 0; c < ND; ++c)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          store4<T>(dst, 32 * c + 2 * r + 4 * k,
                    f32x4{acc[b][c][r], acc[b][c][r + 1], acc[b][c][r + 2], acc[b][c][r + 3]} *
                        a.scale);
    }
}

// ---------------------------------------------------------------------------
// dK and dV.  A wave holds K and V of 32 NK keys as columns and takes in rows,
// 32 at a time:
//   S [rows x keys] = Q . K^T, dP = dO . V^T, dV^T += dO^T . P, dK^T += Q^T . dS.
// The four waves are WK keys wide, WR of rows (whose sums are added at the end)
// and WD of dimensions (each computes the scores, and its dimensions of the
// results).
// ---------------------------------------------------------------------------
template <class T, int D>
struct KeysForm {
  static constexpr bool wide = is_f32<T> && D == 256;
  static constexpr int NK = 1;
  static constexpr int WK = wide ? 1 : 2, WR = wide ? 1 : 2, WD = wide ? 4 : 1;
  static constexpr int keys = 32 * NK * WK;
};

template <class T, int D>
__global__ __launch_bounds__(kThreads, 1) void prompt_grad_keys_kernel(Batch bt, GradArgs a) {
  using L = Tile<T, D>;
  using F = KeysForm<T, D>;
  constexpr int NK = F::NK, WK = F::WK, WR = F::WR, WD = F::WD;
  static_assert(WK * WR * WD == kWaves && (WR == 1 || WD == 1), "four waves");
  constexpr int RT = 32 * WR;                 // rows of a step
  constexpr int NW = L::NW, ND = L::ND / WD;
  constexpr int kTile = RT * L::row_bytes;
  constexpr int kUnits = RT * L::chunks / kThreads, kStep = kThreads / L::chunks;
  static_assert(kUnits >= 1, "whole units");

  __shared__ __align__(16) char s_q[2][kTile];
  __shared__ __align__(16) char s_g[2][kTile];
  __shared__ __align__(16) float s_lse[2][RT], s_delta[2][RT];
  __shared__ int s_spoilt[2][kWaves];

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int i = lane & 31, k = lane >> 5;
  const int wk = wave % WK, wr = wave / WK % WR, wd = wave / (WK * WR);
  const int head = blockIdx.x % bt.h_kv;
  Place at;
  if (!find(bt.key_start, bt.B, bt.N, bt.keys, 1, F::keys, blockIdx.x / bt.h_kv, lane, &at)) return;
  const Span rows = span(bt.row_start, at.b, bt.T, bt.rows);
  const Span keys = span(bt.key_start, at.b, bt.N, bt.keys);
  const int end = rows.n * bt.G;
  const int key0 = at.tile * F::keys;
  // the first row (token and head) that sees a key
  auto first_row = [&](int key) {
    return bt.causal ? (int)min((int64_t)max(key - keys.n + rows.n, 0) * bt.G, (int64_t)end) : 0;
  };
  const int all_from = first_row(min(key0 + F::keys, keys.n) - 1);   // rows that see all of the keys
  const int r0 = first_row(key0) / RT, r1 = (end + RT - 1) / RT;

  int key[NK], from[NK];
  u32x4 kk[NK][NW], vv[NK][NW];
#pragma unroll
  for (int n = 0; n < NK; ++n) {
    key[n] = key0 + 32 * (NK * wk + n) + i;
    const int64_t token = keys.start + min(key[n], keys.n - 1);
    from[n] = first_row(min(key[n], keys.n - 1));
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const int64_t in = (int64_t)head * L::row_bytes + 32 * w + 16 * k;
      kk[n][w] = *reinterpret_cast<const u32x4*>(a.k + token * a.k_stride + in);
      vv[n][w] = *reinterpret_cast<const u32x4*>(a.v + token * a.v_stride + in);
    }
  }

  f32x16 dk[NK][ND], dv[NK][ND];
#pragma unroll
  for (int n = 0; n < NK; ++n)
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) dk[n][c][r] = 0.f, dv[n][c][r] = 0.f;

  u32x4 q_next[kUnits], g_next[kUnits];
  f32x2 stat_next{INFINITY, 0.f};
  const RowReader<T, D> read(ordered_row(i), k);
  const ColumnReader<T, D> read_columns(lane);

  auto load = [&](int t) {
    const int r = tid / L::chunks, c = tid % L::chunks;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int row = t * RT + r + kStep * u;
      const int token = token_of(bt, min(row, end - 1));
      const int64_t in = (int64_t)(head * bt.G + min(row, end - 1) - token * bt.G) * L::row_bytes +
                         16 * c;
      const int64_t tok = rows.start + token;
      q_next[u] = *reinterpret_cast<const u32x4*>(a.q + tok * a.q_stride + in) & a.q_keep;
      g_next[u] = *reinterpret_cast<const u32x4*>(a.d_out + tok * a.d_out_stride + in);
      if (row >= end) q_next[u] = g_next[u] = u32x4{0u, 0u, 0u, 0u};
    }
    if (tid < RT) {
      const int row = t * RT + tid;
      const int token = token_of(bt, min(row, end - 1));
      stat_next = a.stats[(int64_t)(rows.start + token) * bt.h_q + head * bt.G +
                          min(row, end - 1) - token * bt.G];
      if (row >= end) stat_next = f32x2{INFINITY, 0.f};
    }
  };
  auto store = [&](int t) {
    const int buf = t & 1, r = tid / L::chunks, c = tid % L::chunks;
    bool bad = false;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      *reinterpret_cast<u32x4*>(s_q[buf] + L::at(r + kStep * u, c)) = q_next[u];
      *reinterpret_cast<u32x4*>(s_g[buf] + L::at(r + kStep * u, c)) = g_next[u];
    }
    if (tid < RT) s_lse[buf][tid] = stat_next[0], s_delta[buf][tid] = stat_next[1];
    if (t * RT < all_from) {
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
#pragma unroll
        for (int w = 0; w < 4; ++w) bad |= not_finite<T>(q_next[u][w]) || not_finite<T>(g_next[u][w]);
      bad = __any(bad);
      if (lane == 0) s_spoilt[buf][wave] = bad;
    }
  };

  if (r0 < r1) {
    load(r0);
    store(r0);
    __syncthreads();
    for (int t = r0; t < r1; ++t) {
      const int buf = t & 1;
      if (t + 1 < r1) load(t + 1);
      const char *tile_q = s_q[buf] + 32 * wr * L::row_bytes;
      const char *tile_g = s_g[buf] + 32 * wr * L::row_bytes;
      const int row0 = t * RT + 32 * wr;
      f32x16 s[NK], dp[NK];
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[n][r] = 0.f, dp[n][r] = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const u32x4 x = read.get(tile_q, 0, w);
#pragma unroll
        for (int n = 0; n < NK; ++n) s[n] = mma<T>(x, kk[n][w], s[n]);
      }
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const u32x4 x = read.get(tile_g, 0, w);
#pragma unroll
        for (int n = 0; n < NK; ++n) dp[n] = mma<T>(x, vv[n][w], dp[n]);
      }
      float lse2[16], delta[16];
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(&s_lse[buf][32 * wr + row_of(r, k)]);
        const f32x4 y = *reinterpret_cast<const f32x4*>(&s_delta[buf][32 * wr + row_of(r, k)]);
#pragma unroll
        for (int e = 0; e < 4; ++e) lse2[r + e] = x[e], delta[r + e] = y[e];
      }
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r], a.scale2, -lse2[r]));
          dp[n][r] = s[n][r] * (dp[n][r] - delta[r]);
        }
      bool slow = false;
      // (rows beyond the last are zeros, which K may turn into NaN)
      if (t * RT < all_from || (t + 1) * RT > end) {
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int row = row0 + row_of(r, k);
            if (row < from[n] || row >= end) s[n][r] = 0.f, dp[n][r] = 0.f;
          }
      }
      if (t * RT < all_from) {
        int bad = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) bad |= s_spoilt[buf][w];
        slow = uniform(bad);
      }
      if (__builtin_expect(slow, 0)) {
#pragma unroll
        for (int n = 0; n < NK; ++n) {
          auto sees = [&](int row) { return row0 + row >= from[n] && row0 + row < end; };
          add_seen<T, D>(tile_g, 0, 32 * ND * wd, s[n], k, dv[n], sees);
          add_seen<T, D>(tile_q, 0, 32 * ND * wd, dp[n], k, dk[n], sees);
        }
      } else {
        add_columns<T, D, ND, NK>(read_columns, tile_g, 0, ND * wd, s, dv);
        add_columns<T, D, ND, NK>(read_columns, tile_q, 0, ND * wd, dp, dk);
      }
      if (t + 1 < r1) store(t + 1);
      __syncthreads();
    }
  }

  // The row waves' sums: the others' to LDS, added in their order by the first.
  if constexpr (WR > 1) {
    static_assert(WR == 2 && WK * 64 * 16 * 4 * ND * NK <= 2 * kTile, "fits the rows' place");
    auto exchange = [&](f32x16 (&x)[NK][ND], char* place) {
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int c = 0; c < ND; ++c)
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            f32x4* p = reinterpret_cast<f32x4*>(place) +
                       (((wk * NK + n) * ND + c) * 4 + r / 4) * 64 + lane;
            if (wr == 1) {
              *p = f32x4{x[n][c][r], x[n][c][r + 1], x[n][c][r + 2], x[n][c][r + 3]};
            } else {
              const f32x4 y = *p;
#pragma unroll
              for (int e = 0; e < 4; ++e) x[n][c][r + e] += y[e];
            }
          }
    };
    if (wr == 1) exchange(dk, s_q[0]), exchange(dv, s_g[0]);
    __syncthreads();
    if (wr == 0) exchange(dk, s_q[0]), exchange(dv, s_g[0]);
  }
  if (wr != 0) return;
#pragma unroll
  for (int n = 0; n < NK; ++n)
    if (key[n] < keys.n) {
      const int64_t token = keys.start + key[n], in = (int64_t)head * L::row_bytes;
      char* dk_row = a.dk + token * a.dk_stride + in;
      char* dv_row = a.dv + token * a.dv_stride + in;
#pragma unroll
      for (int c = 0; c < ND; ++c)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int d = 32 * (ND * wd + c) + 2 * r + 4 * k;
          store4<T>(dk_row, d, f32x4{dk[n][c][r], dk[n][c][r + 1], dk[n][c][r + 2],
                                     dk[n][c][r + 3]} * a.scale);
          store4<T>(dv_row, d, f32x4{dv[n][c][r], dv[n][c][r + 1], dv[n][c][r + 2],
                                     dv[n][c][r + 3]});
        }
    }
}

}  // namespace

namespace {

struct Plan {
  int64_t row_items, key_items;
  size_t bytes;
};

template <class T, int D>
constexpr int kRowBlocks = is_f32<T> || D == 256 ? 1 : 2;      // NQ of the rows' kernel

Plan plan_grad(const da_prompt& p) {
  Plan plan{};
  const int64_t G = p.h_q / p.h_kv;
  with_type_and_dim(p.dtype, p.d, [&](auto t, auto d) {
    using T = typename decltype(t)::type;
    plan.row_items =
        most_tiles(p.row_start, p.B, p.T, p.rows, G, 32 * kWaves * kRowBlocks<T, d.value>);
    plan.key_items =
        most_tiles(p.key_start, p.B, p.N, p.keys, 1, KeysForm<T, d.value>::keys);
  });
  plan.bytes = (size_t)p.rows * p.h_q * sizeof(f32x2);
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
    if (!stride_fits(x, p.h_q, p.d)) return DA_ERR_SHAPE;
  for (int64_t x : narrow)
    if (!stride_fits(x, p.h_kv, p.d)) return DA_ERR_SHAPE;
  if (st != DA_OK) return st;
  const Plan plan = plan_grad(p);
  if (plan.row_items * p.h_kv > kMaxGroups || plan.key_items * p.h_kv > kMaxGroups)
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
  a.scale = scale, a.scale2 = scale * kLog2e;
  a.q_keep = scale == 0.f ? 0u : ~0u;
  a.stats = static_cast<f32x2*>(workspace);
  const Batch bt = device_batch(p);
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  with_type_and_dim(p.dtype, p.d, [&](auto t, auto d) {
    using T = typename decltype(t)::type;
    hipLaunchKernelGGL((prompt_grad_rows_kernel<T, d.value, kRowBlocks<T, d.value>>),
                       dim3((unsigned)(plan.row_items * p.h_kv)), dim3(kThreads), 0, s, bt, a);
    hipLaunchKernelGGL((prompt_grad_keys_kernel<T, d.value>),
                       dim3((unsigned)(plan.key_items * p.h_kv)), dim3(kThreads), 0, s, bt, a);
  });
  return launch_status();
}

}  // extern "C"
