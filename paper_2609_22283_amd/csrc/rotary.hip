// Rotary positions: the rows of a tensor rotated, and tables whose time axis is scaled for
// histories longer than those of training.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "device.h"
#include "internal.h"

namespace sc {

constexpr double kTwoPi = 6.283185307179586476925286766559;

struct ScaledAxis {
  int32_t kind;
  double theta, factor, original, fast, slow, magnitude;
};

// cos and sin of every (position, pair), as rope_table_kernel's (append.hip), times the
// magnitude; the time axis comes first and only its frequencies are scaled.
__global__ void rope_scaled_table_kernel(float2* table, RopeLayout L, double theta, ScaledAxis s) {
  const int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (e >= L.total) return;
  const int axis = e < L.off_h ? 0 : e < L.off_w ? 1 : 2;
  const int32_t n = axis == 0 ? L.pairs_t : axis == 1 ? L.pairs_h : L.pairs_w;
  const int64_t at = e - (axis == 0 ? 0 : axis == 1 ? L.off_h : L.off_w);
  const int64_t pos = at / n, i = at % n;
  double f = pow(axis == 0 ? s.theta : theta, -(double)i / (double)n);
  if (axis == 0 && s.kind == SC_ROPE_LINEAR) f /= s.factor;
  if (axis == 0 && s.kind == SC_ROPE_YARN) {
    // turns of the pair over the length of training: many, and it stays as it is; few, and
    // its positions are interpolated
    const double keep = fmin(fmax((s.original * f / kTwoPi - s.slow) / (s.fast - s.slow), 0.0), 1.0);
    f *= keep + (1.0 - keep) / s.factor;
  }
  const double ang = (double)pos * f;
  table[e] = make_float2((float)(s.magnitude * cos(ang)), (float)(s.magnitude * sin(ang)));
}

int launch_rope_scaled_table(const sc_rope_desc* d, const sc_rope_scaling* s, void* table, hipStream_t stream) {
  const RopeLayout L = rope_layout(d);
  if (L.total == 0) return SC_OK;
  ScaledAxis a{s->kind, d->theta, s->factor, s->original, s->beta_fast, s->beta_slow, s->magnitude};
  if (s->kind == SC_ROPE_NTK && d->dim_t > 2) a.theta *= std::pow(s->factor, (double)d->dim_t / (d->dim_t - 2));
  hipLaunchKernelGGL(rope_scaled_table_kernel, dim3((uint32_t)((L.total + 255) / 256)), dim3(256), 0, stream,
                     static_cast<float2*>(table), L, (double)d->theta, a);
  SC_HIP(hipGetLastError());
  return SC_OK;
}

struct RotateArgs {
  const float2* table;
  const int32_t* pos;
  int64_t x_row, x_head, y_row, y_head, off_h, off_w;
  int32_t rows, heads, half;  // half: pairs of all axes
  int32_t pairs_t, pairs_h, pairs_w, frames, grid_h, grid_w;
  int32_t rest;               // channels behind the rotated ones, copied (0 in place)
  float sign;                 // of the sines
  int32_t interleaved;
};

template <class T> __device__ __forceinline__ float rot_load(T x);
template <> __device__ __forceinline__ float rot_load<uint16_t>(uint16_t x) { return bf16_to_f32(x); }
template <> __device__ __forceinline__ float rot_load<float>(float x) { return x; }
template <class T> __device__ __forceinline__ T rot_store(float x);
template <> __device__ __forceinline__ uint16_t rot_store<uint16_t>(float x) { return f32_to_bf16(x); }
template <> __device__ __forceinline__ float rot_store<float>(float x) { return x; }

// A thread takes one pair of a row and head, or one channel that is copied.
template <class T>
__global__ __launch_bounds__(256) void rotate_plain_kernel(const T* x, T* y, RotateArgs g) {
  const int32_t units = g.half + g.rest;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)g.rows * g.heads * units) return;
  const int32_t u = (int32_t)(i % units), h = (int32_t)(i / units % g.heads), r = (int32_t)(i / units / g.heads);
  const T* xr = x + r * g.x_row + h * g.x_head;
  T* yr = y + r * g.y_row + h * g.y_head;
  const int32_t t = g.pos[3 * (int64_t)r], ph = g.pos[3 * (int64_t)r + 1], pw = g.pos[3 * (int64_t)r + 2];
  if ((uint32_t)t >= (uint32_t)g.frames || (uint32_t)ph >= (uint32_t)g.grid_h || (uint32_t)pw >= (uint32_t)g.grid_w) return;
  if (u >= g.half) {
    yr[g.half + u] = xr[g.half + u];
    return;
  }
  const float2 cs = u < g.pairs_t ? g.table[(int64_t)t * g.pairs_t + u]
                    : u < g.pairs_t + g.pairs_h ? g.table[g.off_h + (int64_t)ph * g.pairs_h + u - g.pairs_t]
                                                : g.table[g.off_w + (int64_t)pw * g.pairs_w + u - g.pairs_t - g.pairs_h];
  const int32_t a = g.interleaved ? 2 * u : u, b = g.interleaved ? 2 * u + 1 : u + g.half;
  const float x0 = rot_load<T>(xr[a]), x1 = rot_load<T>(xr[b]), s = g.sign * cs.y;
  yr[a] = rot_store<T>(fmaf(x0, cs.x, -(x1 * s)));
  yr[b] = rot_store<T>(fmaf(x0, s, x1 * cs.x));
}

}  // namespace sc

using namespace sc;

extern "C" int sc_rope_table_build_scaled(const sc_rope_desc* d, const sc_rope_scaling* s, void* table, sc_stream stream) {
  if (!d || !s || !table) return fail(SC_EINVAL, "null argument");
  if (d->grid_h < 1 || d->grid_w < 1 || d->max_frames < 1 || d->dim_t < 0 || d->dim_h < 0 || d->dim_w < 0 ||
      (d->dim_t | d->dim_h | d->dim_w) & 1 || !(d->theta > 0.0f))
    return fail(SC_EINVAL, "bad rope descriptor");
  if (s->kind < SC_ROPE_UNSCALED || s->kind > SC_ROPE_YARN) return fail(SC_EINVAL, "unknown scaling %d", s->kind);
  if (!std::isfinite(s->magnitude) || !(s->magnitude > 0.0)) return fail(SC_EINVAL, "magnitude must be positive");
  if (s->kind != SC_ROPE_UNSCALED && (!std::isfinite(s->factor) || !(s->factor >= 1.0)))
    return fail(SC_EINVAL, "scaling factor must be at least 1");
  if (s->kind == SC_ROPE_YARN && (!std::isfinite(s->original) || !(s->original > 0.0) || !std::isfinite(s->beta_fast) ||
                                  !std::isfinite(s->beta_slow) || !(s->beta_fast > s->beta_slow)))
    return fail(SC_EINVAL, "yarn needs original > 0 and beta_fast > beta_slow");
  return launch_rope_scaled_table(d, s, table, static_cast<hipStream_t>(stream));
}

// First and one past the last byte that a strided tensor touches, relative to its start.
static void touched(const sc_rotate_desc& d, int64_t row, int64_t head, int64_t* lo, int64_t* hi) {
  const int64_t r = row * (d.n_rows - 1), h = head * (d.n_heads - 1);
  *lo = std::min<int64_t>(r, 0) + std::min<int64_t>(h, 0);
  *hi = std::max<int64_t>(r, 0) + std::max<int64_t>(h, 0) + d.head_dim;
}

extern "C" int sc_rope_rotate(const sc_rope* rope, const sc_rotate_desc* d, const void* x, void* y,
                              const int32_t* positions, sc_stream stream) {
  if (!rope || !d) return fail(SC_EINVAL, "null argument");
  const sc_rope_desc& t = rope->desc;
  if (d->n_rows < 0 || d->n_heads < 1 || d->head_dim < 1)
    return fail(SC_EINVAL, "bad shape: %d rows of %d heads x %d", d->n_rows, d->n_heads, d->head_dim);
  if (d->dtype != SC_DTYPE_BF16 && d->dtype != SC_DTYPE_F32) return fail(SC_EUNSUPPORTED, "rotation of dtype %d", d->dtype);
  if (d->layout != SC_ROPE_INTERLEAVED && d->layout != SC_ROPE_HALF) return fail(SC_EINVAL, "unknown layout %d", d->layout);
  if (t.grid_h < 1 || t.grid_w < 1 || t.max_frames < 1 || t.dim_t < 0 || t.dim_h < 0 || t.dim_w < 0 ||
      (t.dim_t | t.dim_h | t.dim_w) & 1)
    return fail(SC_EINVAL, "bad rope descriptor");
  const int64_t part = (int64_t)t.dim_t + t.dim_h + t.dim_w;
  if (part < 2 || part > d->head_dim)
    return fail(SC_EINVAL, "%lld rotated channels of heads of %d", (long long)part, d->head_dim);
  if (d->n_rows == 0) return SC_OK;
  if (!x || !y || !positions || !rope->dev_table) return fail(SC_EINVAL, "null argument");
  const uintptr_t es = dtype_size(d->dtype);
  if (reinterpret_cast<uintptr_t>(x) % es || reinterpret_cast<uintptr_t>(y) % es || reinterpret_cast<uintptr_t>(positions) & 3)
    return fail(SC_EINVAL, "tensors must be aligned to their elements");
  const bool in_place = x == y && d->x_row == d->y_row && d->x_head == d->y_head;
  int64_t xl, xh, yl, yh;
  touched(*d, d->x_row, d->x_head, &xl, &xh);
  touched(*d, d->y_row, d->y_head, &yl, &yh);
  const char *xb = static_cast<const char*>(x), *yb = static_cast<const char*>(y);
  const bool apart = xb + xh * (int64_t)es <= yb + yl * (int64_t)es || yb + yh * (int64_t)es <= xb + xl * (int64_t)es;
  // interleaved slices of one tensor are no overlap, but a caller can rotate those in place
  if (!in_place && !apart) return fail(SC_EINVAL, "y must be x itself or lie apart from it");
  const int64_t hd = d->head_dim, H = d->n_heads;
  const auto distinct = [&](int64_t row, int64_t head) {
    row = std::abs(row), head = std::abs(head);
    return (H == 1 || head >= hd) && (d->n_rows == 1 || row >= (H - 1) * head + hd || (row >= hd && (H == 1 || head >= (d->n_rows - 1) * row + hd)));
  };
  if (!distinct(d->y_row, d->y_head)) return fail(SC_EINVAL, "rows or heads of y overlap");
  RotateArgs g;
  std::memset(&g, 0, sizeof g);
  const RopeLayout L = rope_layout(&t);
  g.table = static_cast<const float2*>(rope->dev_table);
  g.pos = positions;
  g.x_row = d->x_row;
  g.x_head = d->x_head;
  g.y_row = d->y_row;
  g.y_head = d->y_head;
  g.off_h = L.off_h;
  g.off_w = L.off_w;
  g.rows = d->n_rows;
  g.heads = d->n_heads;
  g.half = (int32_t)(part / 2);
  g.pairs_t = L.pairs_t;
  g.pairs_h = L.pairs_h;
  g.pairs_w = L.pairs_w;
  g.frames = t.max_frames;
  g.grid_h = t.grid_h;
  g.grid_w = t.grid_w;
  g.rest = in_place ? 0 : (int32_t)(d->head_dim - part);
  g.sign = d->transpose ? -1.f : 1.f;
  g.interleaved = d->layout == SC_ROPE_INTERLEAVED;
  const int64_t threads = (int64_t)g.rows * g.heads * (g.half + g.rest), groups = (threads + 255) / 256;
  if (groups > INT32_MAX) return fail(SC_EUNSUPPORTED, "%lld channel pairs in one call", (long long)threads);
  hipStream_t s = static_cast<hipStream_t>(stream);
  timer_begin(TK_ROTATE, s);
  if (d->dtype == SC_DTYPE_F32)
    hipLaunchKernelGGL(rotate_plain_kernel<float>, dim3((uint32_t)groups), dim3(256), 0, s, static_cast<const float*>(x),
                       static_cast<float*>(y), g);
  else
    hipLaunchKernelGGL(rotate_plain_kernel<uint16_t>, dim3((uint32_t)groups), dim3(256), 0, s,
                       static_cast<const uint16_t*>(x), static_cast<uint16_t*>(y), g);
  timer_end(TK_ROTATE, s);
  SC_HIP(hipGetLastError());
  return SC_OK;
}
