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
  int32_t pair_units, units;  // of a row and head: runs of pairs, then runs of copied channels
  float sign;                 // of the sines
  DivMagic units_div;
};

// N elements of a tensor aligned to them, and their values as fp32.
template <class T, int N> struct RotRun;
template <int N> struct RotRun<uint16_t, N> {
  typedef uint32_t V __attribute__((ext_vector_type(N / 2), aligned(2)));
  static __device__ __forceinline__ float get(const V& v, int i) {
    return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
  }
  static __device__ __forceinline__ V make(const float (&f)[N]) {
    V v;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    return v;
  }
  static __device__ __forceinline__ float one(uint16_t x) { return bf16_to_f32(x); }
  static __device__ __forceinline__ uint16_t back(float x) { return f32_to_bf16(x); }
};
template <int N> struct RotRun<float, N> {
  typedef float V __attribute__((ext_vector_type(N), aligned(4)));
  static __device__ __forceinline__ float get(const V& v, int i) { return v[i]; }
  static __device__ __forceinline__ V make(const float (&f)[N]) {
    V v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = f[i];
    return v;
  }
  static __device__ __forceinline__ float one(float x) { return x; }
  static __device__ __forceinline__ float back(float x) { return x; }
};
template <bool PAST, class V>
__device__ __forceinline__ V rot_load(const V* p) {
  if constexpr (PAST) return __builtin_nontemporal_load(p);
  return *p;
}

// A thread takes a run of pairs (N channels; HALF: N of either half) of one row in HP heads, or a
// run of copied channels.  The row's cosines and sines are read once for the heads, whose loads
// are all out before the first is used.  Bound by memory where there are many rows: four nodes of
// 4680 rows of 12 x 128 channels (115 MB) 24.6 us, 4.7 TB/s, as a plain copy runs (57 with a pair a
// thread); by latency at few.
// N: 16 bytes, but 8 of bf16 halves, of which a thread has two (12000 rows of 12 heads of 128 18.3
// us, 21.7 with 16; of 40, whose halves 16 bytes do not divide, 9.0, 22.9).  PAST: read past the
// caches, which y gets (the four nodes 27.7 us without, 25.7 with y's stores past them too).
template <class T, bool HALF, int N, int HP, bool PAST>
__global__ __launch_bounds__(256) void rotate_kernel(const T* x, T* y, RotateArgs g) {
  using Run = RotRun<T, N>;
  using V = typename Run::V;
  constexpr int P = HALF ? N : N / 2;
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= (uint32_t)g.rows * (uint32_t)g.units) return;
  const int32_t r = (int32_t)fast_div(i, g.units_div), u = (int32_t)i - r * g.units, h0 = blockIdx.y * HP;
  const int32_t t = g.pos[3 * (int64_t)r], ph = g.pos[3 * (int64_t)r + 1], pw = g.pos[3 * (int64_t)r + 2];
  if ((uint32_t)t >= (uint32_t)g.frames || (uint32_t)ph >= (uint32_t)g.grid_h || (uint32_t)pw >= (uint32_t)g.grid_w) return;
  const bool pairs = u < g.pair_units;
  const int32_t p0 = u * P, c0 = pairs ? (HALF ? p0 : 2 * p0) : 2 * g.half + (u - g.pair_units) * N;
  // elements of the run (of either half), all there but at the end
  const int32_t n = pairs ? (HALF ? min(N, g.half - p0) : min(N, 2 * (g.half - p0))) : min(N, g.rest - (u - g.pair_units) * N);
  const T* xr = x + r * g.x_row + c0;
  T* yr = y + r * g.y_row + c0;
  V a[HP], b[HP];
  if (n == N)
#pragma unroll
    for (int j = 0; j < HP; ++j) {
      const T* from = xr + min(h0 + j, g.heads - 1) * g.x_head;
      a[j] = rot_load<PAST>(reinterpret_cast<const V*>(from));
      if (HALF && pairs) b[j] = rot_load<PAST>(reinterpret_cast<const V*>(from + g.half));
    }
  if (!pairs) {
#pragma unroll
    for (int j = 0; j < HP; ++j) {
      if (h0 + j >= g.heads) break;
      T* to = yr + (h0 + j) * g.y_head;
      if (n == N)
        *reinterpret_cast<V*>(to) = a[j];
      else
        for (int e = 0; e < n; ++e) to[e] = xr[(h0 + j) * g.x_head + e];
    }
    return;
  }
  float2 cs[P];
#pragma unroll
  for (int e = 0; e < P; ++e) {
    const int32_t p = min(p0 + e, g.half - 1);
    cs[e] = g.table[p < g.pairs_t ? (int64_t)t * g.pairs_t + p
                    : p < g.pairs_t + g.pairs_h ? g.off_h + (int64_t)ph * g.pairs_h + p - g.pairs_t
                                                : g.off_w + (int64_t)pw * g.pairs_w + p - g.pairs_t - g.pairs_h];
    cs[e].y *= g.sign;
  }
#pragma unroll
  for (int j = 0; j < HP; ++j) {
    if (h0 + j >= g.heads) break;
    T* to = yr + (h0 + j) * g.y_head;
    if (n == N) {
      float fa[N], fb[N];
#pragma unroll
      for (int e = 0; e < P; ++e) {
        const float x0 = Run::get(a[j], HALF ? e : 2 * e), x1 = HALF ? Run::get(b[j], e) : Run::get(a[j], 2 * e + 1);
        const float y0 = fmaf(x0, cs[e].x, -(x1 * cs[e].y)), y1 = fmaf(x0, cs[e].y, x1 * cs[e].x);
        if constexpr (HALF) {
          fa[e] = y0;
          fb[e] = y1;
        } else {
          fa[2 * e] = y0;
          fa[2 * e + 1] = y1;
        }
      }
      *reinterpret_cast<V*>(to) = Run::make(fa);
      if constexpr (HALF) *reinterpret_cast<V*>(to + g.half) = Run::make(fb);
    } else {
      const T* from = xr + (h0 + j) * g.x_head;
#pragma unroll
      for (int e = 0; e < P; ++e) {
        if (p0 + e >= g.half) break;
        const int32_t i0 = HALF ? e : 2 * e, i1 = HALF ? e + g.half : 2 * e + 1;
        const float x0 = Run::one(from[i0]), x1 = Run::one(from[i1]);
        to[i0] = Run::back(fmaf(x0, cs[e].x, -(x1 * cs[e].y)));
        to[i1] = Run::back(fmaf(x0, cs[e].y, x1 * cs[e].x));
      }
    }
  }
}

// Few rows: a head a thread, so that the work spreads over the CUs (12 heads of 128: 256 rows 2.7
// us, 3.2 with four heads a thread; 1536 rows 3.9 either way, 4096 rows 6.9 against 5.8).  Else
// past the caches where a thread's neighbours read lines to their ends: runs of 128 bytes or of
// 64-byte pieces (12000 rows of 12 heads of 40 in bf16, 80 bytes each, 9.4 us past them, 8.1 not;
// of 80 in fp32 20.6 and 23.3).
template <class T, bool HALF, int N>
static void launch_rotate_t(const void* x, void* y, const RotateArgs& g, hipStream_t s) {
  const uint32_t groups = (uint32_t)(((int64_t)g.rows * g.units + 255) / 256), fours = (uint32_t)(g.heads + 3) / 4;
  const T* xt = static_cast<const T*>(x);
  T* yt = static_cast<T*>(y);
  if ((int64_t)groups * fours < 3 * kCUs / 2)
    hipLaunchKernelGGL((rotate_kernel<T, HALF, N, 1, false>), dim3(groups, (uint32_t)g.heads), dim3(256), 0, s, xt, yt, g);
  else if (const size_t bytes = g.half * (HALF ? 1 : 2) * sizeof(T); bytes >= 128 || bytes % 64 == 0)
    hipLaunchKernelGGL((rotate_kernel<T, HALF, N, 4, true>), dim3(groups, fours), dim3(256), 0, s, xt, yt, g);
  else
    hipLaunchKernelGGL((rotate_kernel<T, HALF, N, 4, false>), dim3(groups, fours), dim3(256), 0, s, xt, yt, g);
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
  const bool f32 = d->dtype == SC_DTYPE_F32, halves = d->layout == SC_ROPE_HALF;
  const int32_t run = f32 || halves ? 4 : 8, run_pairs = halves ? run : run / 2;
  g.pair_units = (g.half + run_pairs - 1) / run_pairs;
  g.units = g.pair_units + (g.rest + run - 1) / run;
  g.units_div = magic_div((uint32_t)g.units);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int32_t most = INT32_MAX / g.units - 256;  // rows of a launch, whose threads are numbered in 31 bits
  if (most < 1 || g.heads > 65535) return fail(SC_EUNSUPPORTED, "%d heads of %d channels", g.heads, d->head_dim);
  for (int64_t row = 0; row < d->n_rows; row += most) {
    g.rows = (int32_t)std::min<int64_t>(most, d->n_rows - row);
    g.pos = positions + 3 * row;
    const char* from = xb + row * d->x_row * (int64_t)es;
    char* to = static_cast<char*>(y) + row * d->y_row * (int64_t)es;
    timer_begin(TK_ROTATE, s);
    if (f32 && halves)
      launch_rotate_t<float, true, 4>(from, to, g, s);
    else if (f32)
      launch_rotate_t<float, false, 4>(from, to, g, s);
    else if (halves)
      launch_rotate_t<uint16_t, true, 4>(from, to, g, s);
    else
      launch_rotate_t<uint16_t, false, 8>(from, to, g, s);
    timer_end(TK_ROTATE, s);
    SC_HIP(hipGetLastError());
  }
  return SC_OK;
}
