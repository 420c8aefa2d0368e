// rotary_axes.hip -- gfx950 kernel and C ABI of the rotation of q and k by
// positions of several axes (time, height and width of images and video; all the
// same in text), and of its gradient, the rotation back.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "decode_attn.h"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxAxes = 4;

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct RotaryArgs {
  const char *q, *k;
  char *q_out, *k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;   // bytes between tokens
  const int32_t* positions;                                 // [axes][rows]
  const float* table;                                       // [n_table][rot_dim]
  int rows, heads, h_q, n_table, rot_dim, axes, interleaved;
  int ends[kMaxAxes];                                       // pairs before the next axis
  float sign;
  uint32_t per_row;                                         // threads of a row
};

// Eight values as float.
template <class T>
struct Eight {
  typedef T vec __attribute__((ext_vector_type(8)));
  vec x;
  __device__ __forceinline__ void load(const T* p) { x = *reinterpret_cast<const vec*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<vec*>(p) = x; }
};

// ---------------------------------------------------------------------------
// A thread turns the same 16 dimensions of up to kHeads heads of one row: eight
// pairs, (i, i + half) or (2i, 2i + 1), or copies 16 that are not turned.  The angles
// are read once for them, in four loads where one axis has all eight pairs.  An axis
// may begin inside them: each pair then has a position of its own.
// Memory-bound: 16001 rows of 40 heads of 128 on three axes, 328 MB, 63 us (5.2 TB/s; a
// copy too large for the caches 4.8).  With one head a thread, whose pairs each loaded
// their own angles, 148 us.  16 rows: 4.8 us, a launch and loads that wait for each other.
// ---------------------------------------------------------------------------
constexpr int kHeads = 4;

template <class T, int D>
__global__ __launch_bounds__(kThreads) void rotary_axes_kernel(RotaryArgs a) {
  constexpr int kPieces = D / 16;
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
  const uint32_t row = id / a.per_row;
  const int x = (int)(id - row * a.per_row);
  if (row >= (uint32_t)a.rows) return;
  const int piece = x % kPieces, head0 = x / kPieces, head_step = (int)a.per_row / kPieces;
  const int half = a.rot_dim / 2, pair0 = 8 * piece;
  const bool turned = 2 * pair0 < a.rot_dim;
  const bool near = a.interleaved || !turned;
  const int at0 = near ? 2 * pair0 : pair0;
  const int at1 = near ? 2 * pair0 + 8 : pair0 + half;

  Eight<T> u[kHeads], v[kHeads];
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    const int head = head0 + j * head_step;
    if (head >= a.heads) break;
    const bool is_q = head < a.h_q;
    const T* src = reinterpret_cast<const T*>(is_q ? a.q + row * a.q_stride
                                                   : a.k + row * a.k_stride) +
                   (is_q ? head : head - a.h_q) * D;
    u[j].load(src + at0);
    v[j].load(src + at1);
  }
  float cosine[8], sine[8];
  // A bit for each pair but those whose position is outside the table, which are copied
  // (multiplied by 1 and 0, an infinity's partner would become NaN).
  unsigned here = 0xffu;
  if (turned) {
    int axis = 0;
    while (axis + 1 < a.axes && pair0 >= a.ends[axis]) ++axis;
    if (pair0 + 8 <= a.ends[axis]) {
      const int pos = a.positions[(int64_t)axis * a.rows + row];
      const bool held = (unsigned)pos < (unsigned)a.n_table;
      here = held ? 0xffu : 0u;
      const f32x4* angles = reinterpret_cast<const f32x4*>(
          a.table + (int64_t)(held ? pos : 0) * a.rot_dim + pair0);
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const f32x4 c = angles[e / 4], s = angles[half / 4 + e / 4];
#pragma unroll
        for (int w = 0; w < 4; ++w)
          cosine[e + w] = c[w], sine[e + w] = a.sign * s[w];
      }
    } else {
      here = 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        while (axis + 1 < a.axes && pair0 + e >= a.ends[axis]) ++axis;
        const int pos = a.positions[(int64_t)axis * a.rows + row];
        const bool held = (unsigned)pos < (unsigned)a.n_table;
        const float* angles = a.table + (int64_t)(held ? pos : 0) * a.rot_dim + pair0 + e;
        here |= held ? 1u << e : 0u;
        cosine[e] = angles[0], sine[e] = a.sign * angles[half];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    const int head = head0 + j * head_step;
    if (head >= a.heads) break;
    Eight<T> y0 = u[j], y1 = v[j];
    if (turned) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int w = 2 * e % 8;
        const T first = a.interleaved ? (e < 4 ? u[j].x[w] : v[j].x[w]) : u[j].x[e];
        const T second = a.interleaved ? (e < 4 ? u[j].x[w + 1] : v[j].x[w + 1]) : v[j].x[e];
        const float p = (float)first, r = (float)second;
        const T lo = (T)(p * cosine[e] - r * sine[e]), hi = (T)(r * cosine[e] + p * sine[e]);
        if (a.interleaved) {
          if (e < 4)
            y0.x[w] = lo, y0.x[w + 1] = hi;
          else
            y1.x[w] = lo, y1.x[w + 1] = hi;
        } else {
          y0.x[e] = lo, y1.x[e] = hi;
        }
      }
    }
    if (__builtin_expect(here != 0xffu, 0)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {          // (pairs of the values e of y0 and of y1)
        if (!(here >> (a.interleaved ? e / 2 : e) & 1)) y0.x[e] = u[j].x[e];
        if (!(here >> (a.interleaved ? 4 + e / 2 : e) & 1)) y1.x[e] = v[j].x[e];
      }
    }
    const bool is_q = head < a.h_q;
    T* dst = reinterpret_cast<T*>(is_q ? a.q_out + row * a.q_out_stride
                                       : a.k_out + row * a.k_out_stride) +
             (is_q ? head : head - a.h_q) * D;
    y0.store(dst + at0);
    y1.store(dst + at1);
  }
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

template <class T>
void launch(int d, unsigned groups, const RotaryArgs& a, hipStream_t s) {
  if (d == 64)
    hipLaunchKernelGGL((rotary_axes_kernel<T, 64>), dim3(groups), dim3(kThreads), 0, s, a);
  else if (d == 128)
    hipLaunchKernelGGL((rotary_axes_kernel<T, 128>), dim3(groups), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((rotary_axes_kernel<T, 256>), dim3(groups), dim3(kThreads), 0, s, a);
}

}  // namespace

extern "C" da_status da_rotary_axes(const da_rotary* rotary, const void* q, int64_t q_stride,
                                    int h_q, void* q_out, int64_t q_out_stride, const void* k,
                                    int64_t k_stride, int h_kv, void* k_out, int64_t k_out_stride,
                                    void* stream) {
  if (!rotary || !q || !q_out || (k && !k_out) || !rotary->positions || !rotary->table)
    return DA_ERR_NULL;
  const da_rotary& p = *rotary;
  if (!k) h_kv = 0, k_out = nullptr;
  if (p.rows < 1 || p.d < 1 || h_q < 1 || h_kv < 0 || (k && h_kv < 1) || p.n_table < 1 ||
      p.axes < 1 || p.axes > kMaxAxes || p.rot_dim < 1 || p.rot_dim > p.d ||
      ((int64_t)h_q + h_kv) * p.d > (1 << 30))
    return DA_ERR_SHAPE;
  int64_t pairs = 0;
  RotaryArgs a{};
  for (int x = 0; x < p.axes; ++x) {
    if (p.sections[x] < 0 || p.sections[x] > p.rot_dim) return DA_ERR_SHAPE;
    pairs += p.sections[x];
    a.ends[x] = (int)std::min<int64_t>(pairs, p.rot_dim);
  }
  if (2 * pairs != p.rot_dim || q_stride < (int64_t)h_q * p.d || q_out_stride < (int64_t)h_q * p.d ||
      (k && (k_stride < (int64_t)h_kv * p.d || k_out_stride < (int64_t)h_kv * p.d)))
    return DA_ERR_SHAPE;
  if ((p.d != 64 && p.d != 128 && p.d != 256) || p.dtype < DA_F32 || p.dtype > DA_F16 ||
      p.rot_dim % 16 != 0)
    return DA_ERR_UNSUPPORTED;
  const int size = p.dtype == DA_F32 ? 4 : 2, per16 = 16 / size;
  const int64_t per_row = (int64_t)((h_q + h_kv + kHeads - 1) / kHeads) * (p.d / 16);
  const int64_t threads = p.rows * per_row;
  const int64_t groups = (threads + kThreads - 1) / kThreads;
  if (groups >= (1 << 24)) return DA_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(q_out, 16) || !aligned(k_out, 16) ||
      !aligned(p.positions, 4) || !aligned(p.table, 16) || q_stride % per16 ||
      q_out_stride % per16 || (k && (k_stride % per16 || k_out_stride % per16)))
    return DA_ERR_ALIGN;
  a.q = static_cast<const char*>(q), a.k = static_cast<const char*>(k);
  a.q_out = static_cast<char*>(q_out), a.k_out = static_cast<char*>(k_out);
  a.q_stride = q_stride * size, a.k_stride = k_stride * size;
  a.q_out_stride = q_out_stride * size, a.k_out_stride = k_out_stride * size;
  a.positions = p.positions, a.table = p.table;
  a.rows = p.rows, a.heads = h_q + h_kv, a.h_q = h_q, a.n_table = p.n_table;
  a.rot_dim = p.rot_dim, a.axes = p.axes, a.interleaved = p.interleaved != 0;
  a.sign = p.inverse ? -1.f : 1.f;
  a.per_row = (uint32_t)per_row;
  (void)hipGetLastError();
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p.dtype == DA_F32)
    launch<float>(p.d, (unsigned)groups, a, s);
  else if (p.dtype == DA_BF16)
    launch<__bf16>(p.d, (unsigned)groups, a, s);
  else
    launch<_Float16>(p.d, (unsigned)groups, a, s);
  return hipGetLastError() == hipSuccess ? DA_OK : DA_ERR_HIP;
}
