// rotary_axes.hip -- gfx950 kernel and C ABI of the rotation of q and k by
// positions of several axes (time, height and width of images and video; all the
// same in text), and of its gradient, the rotation back.
#include <hip/hip_runtime.h>

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
// A thread turns 16 dimensions of one head of one row: eight pairs, (i, i + half)
// or (2i, 2i + 1), or copies 16 that are not turned.  An axis may begin inside
// the eight pairs, so each has a position of its own.
// ---------------------------------------------------------------------------
template <class T, int D>
__global__ __launch_bounds__(kThreads) void rotary_axes_kernel(RotaryArgs a) {
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
  const uint32_t row = id / a.per_row;
  const int x = (int)(id - row * a.per_row);
  if (row >= (uint32_t)a.rows) return;
  const int head = x / (D / 16), piece = x % (D / 16);
  const bool is_q = head < a.h_q;
  const int h = is_q ? head : head - a.h_q;
  const T* src = reinterpret_cast<const T*>((is_q ? a.q : a.k) +
                                            row * (is_q ? a.q_stride : a.k_stride)) + h * D;
  T* dst = reinterpret_cast<T*>((is_q ? a.q_out : a.k_out) +
                                row * (is_q ? a.q_out_stride : a.k_out_stride)) + h * D;
  const int half = a.rot_dim / 2;
  const bool turned = 16 * piece < a.rot_dim;
  const bool near = a.interleaved || !turned;
  const int at0 = near ? 16 * piece : 8 * piece;
  const int at1 = near ? 16 * piece + 8 : 8 * piece + half;
  Eight<T> u, v;
  u.load(src + at0);
  v.load(src + at1);
  if (turned) {
    const int pair0 = 8 * piece;
    float cosine[8], sine[8];
    int axis = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      while (axis + 1 < a.axes && pair0 + e >= a.ends[axis]) ++axis;
      const int pos = a.positions[(int64_t)axis * a.rows + row];
      const bool held = (unsigned)pos < (unsigned)a.n_table;
      const float* angles = a.table + (int64_t)(held ? pos : 0) * a.rot_dim + pair0 + e;
      cosine[e] = held ? angles[0] : 1.f;
      sine[e] = held ? a.sign * angles[half] : 0.f;
    }
    Eight<T> y0, y1;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = a.interleaved ? (float)(e < 4 ? u.x[2 * e % 8] : v.x[2 * e % 8]) : (float)u.x[e];
      const float r =
          a.interleaved ? (float)(e < 4 ? u.x[2 * e % 8 + 1] : v.x[2 * e % 8 + 1]) : (float)v.x[e];
      const T lo = (T)(p * cosine[e] - r * sine[e]), hi = (T)(r * cosine[e] + p * sine[e]);
      if (a.interleaved) {
        if (e < 4)
          y0.x[2 * e % 8] = lo, y0.x[2 * e % 8 + 1] = hi;
        else
          y1.x[2 * e % 8] = lo, y1.x[2 * e % 8 + 1] = hi;
      } else {
        y0.x[e] = lo, y1.x[e] = hi;
      }
    }
    u = y0, v = y1;
  }
  u.store(dst + at0);
  v.store(dst + at1);
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
  int pairs = 0;
  RotaryArgs a{};
  for (int x = 0; x < p.axes; ++x) {
    if (p.sections[x] < 0 || p.sections[x] > p.rot_dim) return DA_ERR_SHAPE;
    pairs += p.sections[x];
    a.ends[x] = pairs;
  }
  if (2 * pairs != p.rot_dim || q_stride < (int64_t)h_q * p.d || q_out_stride < (int64_t)h_q * p.d ||
      (k && (k_stride < (int64_t)h_kv * p.d || k_out_stride < (int64_t)h_kv * p.d)))
    return DA_ERR_SHAPE;
  if ((p.d != 64 && p.d != 128 && p.d != 256) || p.dtype < DA_F32 || p.dtype > DA_F16 ||
      p.rot_dim % 16 != 0)
    return DA_ERR_UNSUPPORTED;
  const int size = p.dtype == DA_F32 ? 4 : 2, per16 = 16 / size;
  const int64_t threads = (int64_t)p.rows * (h_q + h_kv) * (p.d / 16);
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
  a.per_row = (uint32_t)((h_q + h_kv) * (p.d / 16));
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
