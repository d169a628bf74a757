// The global norm of a list of gradient tensors and the clipping by it.
//   L2:  total = sum over all elements of x^2,  norm = sqrt(total)
//   max: total = max |x|,                       norm = total
//   coef = min(1, max_norm / (norm + eps)),     out = fl(x coef)
// One pass over the data for the norm (each element is converted to binary64, where its
// square is exact, and added there: no overflow and no rounding that matters), one more for
// the clipping.  Both are bound by memory.
//
// A tensor is cut into parts of 16-byte vectors by its own type, shape and strides (its
// output's too: beside strided rows a contiguous tensor is walked as rows); a workgroup takes one
// part, found in a table that the list was given when it was made, so that any number of
// tensors share a launch.  Every partial result has its own place and the places are added in a
// fixed order, so a tensor's norm does not change with the tensors beside it and nothing
// depends on the order of atomics.
#include "device.h"
#include "internal.h"
#include "vec.h"

namespace fp4r {
namespace {

constexpr int kThreads = 256;

// The larger of two magnitudes, NaN if either is.
FP4R_DEV double max_nan(double a, double b) { return a != a ? a : (b > a || b != b) ? b : a; }

template <bool MAX>
FP4R_DEV double join(double a, double b) {
  return MAX ? max_nan(a, b) : a + b;
}
template <bool MAX>
FP4R_DEV double take(double acc, float x) {
  if constexpr (MAX) return max_nan(acc, (double)fabsf(x));
  else return __builtin_fma((double)x, (double)x, acc);
}

// The sum (or maximum) over a wave, in every lane: butterflies over the 16 lanes of a row, then
// the four rows.
template <bool MAX>
FP4R_DEV double wave_join(double v) {
  v = join<MAX>(v, dpp_d<0xB1>(v));
  v = join<MAX>(v, dpp_d<0x4E>(v));
  v = join<MAX>(v, dpp_d<0x141>(v));
  v = join<MAX>(v, dpp_d<0x140>(v));
  return join<MAX>(join<MAX>(readlane_d(v, 0), readlane_d(v, 16)), join<MAX>(readlane_d(v, 32), readlane_d(v, 48)));
}

// The sum (or maximum) over a workgroup.
template <bool MAX>
FP4R_DEV double block_join(double v) {
  __shared__ double red[kThreads / 64];
  v = wave_join<MAX>(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) v = join<MAX>(v, red[w]);
  return v;
}

// Walks vectors [v0, v1) (of 16 bytes of the input) of a tensor.  A contiguous one goes in
// steps of kUnroll vectors of VE elements a thread, so that as many loads are in flight:
// load(offset) fetches one, use(raw, offset) consumes it (the norm of 2.8 GB: 478 -> 460 us,
// twelve parameters of 2.0 M elements 9.2 -> 5.2).  The rest, and tensors of rows, go through
// one(first element's offset in the input, ... in the output, count).
constexpr int kUnroll = 4;
template <class TI, int VE, class L, class U, class F>
FP4R_DEV void each_vector(const GradRef& t, int64_t v0, int64_t v1, L load, U use, F one) {
  constexpr int VI = 16 / sizeof(TI);
  if (t.rows == 1) {
    const int64_t end = min(v1 * VI, t.cols);
    int64_t i = v0 * VI + threadIdx.x * VE;
    for (; i + (kUnroll - 1) * kThreads * VE + VE <= end; i += kUnroll * kThreads * VE) {
      decltype(load(0)) raw[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) raw[u] = load(i + u * kThreads * VE);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) use(raw[u], i + u * kThreads * VE);
    }
    for (; i < end; i += kThreads * VE) one(i, i, (int)min((int64_t)VE, end - i));
    return;
  }
  // rows: the same with each vector's place found by division, in 32 bits where they are enough
  constexpr int R = VI / VE;
  const uint32_t per_row = (uint32_t)((t.cols + VI - 1) / VI);   // cols < 2^33, see kMaxLd
  const bool narrow = t.vectors >> 32 == 0;
  int64_t v = v0 + threadIdx.x;
  while (v < v1) {
    int64_t i[kUnroll], o[kUnroll];
    int n[kUnroll];
    bool full = true;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t w = v + u * kThreads;
      const int64_t row = narrow ? (int64_t)((uint32_t)w / per_row) : w / per_row;
      const int64_t c = (w - row * per_row) * VI;
      i[u] = row * t.ld_in + c;
      o[u] = row * t.ld_out + c;
      n[u] = w < v1 ? (int)min((int64_t)VI, t.cols - c) : 0;
      full = full && n[u] == VI;
    }
    if (full) {
      decltype(load(0)) raw[kUnroll * R];
#pragma unroll
      for (int u = 0; u < kUnroll * R; ++u) raw[u] = load(i[u / R] + (u % R) * VE);
#pragma unroll
      for (int u = 0; u < kUnroll * R; ++u) use(raw[u], o[u / R] + (u % R) * VE);
    } else {
#pragma unroll
      for (int u = 0; u < kUnroll * R; ++u) {
        const int k = (u % R) * VE, m = n[u / R] - k;
        if (m > 0) one(i[u / R] + k, o[u / R] + k, min(VE, m));
      }
    }
    v += kUnroll * kThreads;
  }
}

template <class T, bool MAX, bool NT>
FP4R_DEV double part_value(const GradRef& t, int64_t v0, int64_t v1) {
  constexpr int VE = 16 / sizeof(T);
  const T* in = (const T*)t.in;
  double acc = 0.0;
  const auto add = [&](const float (&x)[VE]) {
#pragma unroll
    for (int k = 0; k < VE; ++k) acc = take<MAX>(acc, x[k]);
  };
  each_vector<T, VE>(
      t, v0, v1, [&](int64_t i) { return load_raw<T, VE, NT>(in + i); },
      [&](const u32x4& r, int64_t) {
        float x[VE];
        unpack_raw<T, VE>(r, x);
        add(x);
      },
      [&](int64_t i, int64_t, int n) {
        float x[VE];
        load_vec<T, VE>(in + i, n, x);
        add(x);
      });
  return acc;
}

// Writes a chunk of the table: workgroup i its tensor and that tensor's parts.
__global__ __launch_bounds__(kThreads) void k_grad_table(GradChunk ch, GradTable tb, uint32_t first_tensor) {
  const int i = blockIdx.x;
  const uint32_t t = first_tensor + i;
  if (threadIdx.x == 0) {
    tb.tensors[t] = ch.t[i];
    if (t == 0) *tb.status = 0u;
  }
  for (uint32_t p = threadIdx.x; p < ch.parts[i]; p += kThreads) tb.parts[ch.t[i].first + p] = GradPart{t, p};
}

template <bool MAX, bool NT>
__global__ __launch_bounds__(kThreads) void k_grad_parts(GradTable tb) {
  const GradPart p = tb.parts[blockIdx.x];
  const GradRef& t = tb.tensors[p.tensor];
  const int64_t v0 = (int64_t)p.part << t.shift, v1 = min(t.vectors, v0 + (int64_t(1) << t.shift));
  double v;
  switch (t.type & 3) {
    case 0: v = part_value<float, MAX, NT>(t, v0, v1); break;
    case 1: v = part_value<bf16_t, MAX, NT>(t, v0, v1); break;
    default: v = part_value<f16_t, MAX, NT>(t, v0, v1); break;
  }
  v = block_join<MAX>(v);
  if (threadIdx.x == 0) tb.partial[blockIdx.x] = v;
}

FP4R_DEV void write_result(double total, bool max, double max_norm, double eps, float* result) {
  const double norm = max ? total : __builtin_sqrt(total);
  const double q = max_norm / (norm + eps);
  result[0] = (float)norm;
  result[1] = q > 1.0 ? 1.0f : (float)q;   // a NaN stays
}

// Parts first, first + step, ... before end, U loads in flight (an index past the end reads the
// last part and is dropped, since a branch would wait for each load).
template <bool MAX, int U>
FP4R_DEV double join_parts(const double* partial, uint32_t first, uint32_t step, uint32_t end) {
  double v = 0.0;
  for (uint32_t p = first; p < end; p += U * step) {
    double x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = partial[min(p + u * step, end - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) v = join<MAX>(v, p + u * step < end ? x[u] : 0.0);
  }
  return v;
}

// Workgroup 0 joins all parts into the total; the others, a wave a tensor, each tensor's own.
// Neither waits for the other (300 tensors of 3400 parts, joined one after the other: 9.3 us in
// two launches).
constexpr int kWaves = 16;
template <bool MAX>
__global__ __launch_bounds__(kWaves * 64) void k_grad_total(GradTable tb, uint32_t count, uint32_t parts,
                                                            double max_norm, double eps, double* total, float* norms,
                                                            float* result) {
  __shared__ double red[kWaves];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (blockIdx.x > 0) {
    const uint32_t t = (blockIdx.x - 1) * kWaves + wave;
    if (t >= count) return;
    const double v = wave_join<MAX>(join_parts<MAX, 4>(tb.partial, tb.tensors[t].first + lane, 64, tb.tensors[t + 1].first));
    if (lane == 0) norms[t] = (float)(MAX ? v : __builtin_sqrt(v));
    return;
  }
  double v = wave_join<MAX>(join_parts<MAX, 8>(tb.partial, threadIdx.x, kWaves * 64, parts));
  if (lane == 0) red[wave] = v;
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) v = join<MAX>(v, red[w]);
  *total = v;
  write_result(v, MAX, max_norm, eps, result);
  *tb.status = v < __builtin_inf() ? 0u : kStatusNonFinite;
}

__global__ void k_clip_coef(const double* total, int max, double max_norm, double eps, float* result) {
  write_result(*total, max != 0, max_norm, eps, result);
}

// Vectors of 16 bytes of the wider type, so that a wave's stores are contiguous; the stores pass
// the caches (see store_full).  Parts go backwards: the last ones are those that the norm read
// last (clipping 354 M BF16 elements into FP32: 525 us forwards, 501 backwards).
template <class TI, class TO, bool NT>
FP4R_DEV void scale_part(const GradRef& t, int64_t v0, int64_t v1, float coef) {
  constexpr int VE = sizeof(TO) > sizeof(TI) ? 16 / sizeof(TO) : 16 / sizeof(TI);
  const TI* in = (const TI*)t.in;
  TO* out = (TO*)t.out;
  const auto put_scaled = [&](float (&x)[VE], int64_t o, int n) {
#pragma unroll
    for (int k = 0; k < VE; ++k) x[k] *= coef;
    store_vec<TO, VE>(out + o, n, x);
  };
  each_vector<TI, VE>(
      t, v0, v1, [&](int64_t i) { return load_raw<TI, VE, NT>(in + i); },
      [&](const auto& r, int64_t i) {
        float x[VE];
        unpack_raw<TI, VE>(r, x);
        put_scaled(x, i, VE);
      },
      [&](int64_t i, int64_t o, int n) {
        float x[VE];
        load_vec<TI, VE>(in + i, n, x);
        put_scaled(x, o, n);
      });
}

template <bool NT>
__global__ __launch_bounds__(kThreads) void k_grad_scale(GradTable tb, const float* coef_p) {
  const GradPart p = tb.parts[gridDim.x - 1 - blockIdx.x];
  const GradRef& t = tb.tensors[p.tensor];
  const float coef = *coef_p;
  if (coef == 1.0f && t.in == t.out) return;   // in place, and x 1 is x
  const int64_t v0 = (int64_t)p.part << t.shift, v1 = min(t.vectors, v0 + (int64_t(1) << t.shift));
  switch (t.type) {
    case 0 | 0 << 2: scale_part<float, float, NT>(t, v0, v1, coef); break;
    case 0 | 1 << 2: scale_part<float, bf16_t, NT>(t, v0, v1, coef); break;
    case 0 | 2 << 2: scale_part<float, f16_t, NT>(t, v0, v1, coef); break;
    case 1 | 0 << 2: scale_part<bf16_t, float, NT>(t, v0, v1, coef); break;
    case 1 | 1 << 2: scale_part<bf16_t, bf16_t, NT>(t, v0, v1, coef); break;
    case 1 | 2 << 2: scale_part<bf16_t, f16_t, NT>(t, v0, v1, coef); break;
    case 2 | 0 << 2: scale_part<f16_t, float, NT>(t, v0, v1, coef); break;
    case 2 | 1 << 2: scale_part<f16_t, bf16_t, NT>(t, v0, v1, coef); break;
    default: scale_part<f16_t, f16_t, NT>(t, v0, v1, coef); break;
  }
}

}  // namespace

hipError_t launch_grad_table(const GradChunk& ch, const GradTable& tb, uint32_t first_tensor, hipStream_t st) {
  hipLaunchKernelGGL(k_grad_table, dim3(ch.count), dim3(kThreads), 0, st, ch, tb, first_tensor);
  return hipGetLastError();
}

template <bool MAX>
static void grad_norm(const GradTable& tb, uint32_t count, uint32_t parts, bool past, double max_norm, double eps,
                      double* total, float* norms, float* result, hipStream_t st) {
  if (parts) {
    if (past) hipLaunchKernelGGL((k_grad_parts<MAX, true>), dim3(parts), dim3(kThreads), 0, st, tb);
    else hipLaunchKernelGGL((k_grad_parts<MAX, false>), dim3(parts), dim3(kThreads), 0, st, tb);
  }
  const uint32_t groups = 1 + (norms ? (count + kWaves - 1) / kWaves : 0);
  hipLaunchKernelGGL(k_grad_total<MAX>, dim3(groups), dim3(kWaves * 64), 0, st, tb, count, parts, max_norm, eps, total,
                     norms, result);
}
hipError_t launch_grad_norm(const GradTable& tb, uint32_t count, uint32_t parts, bool past, bool max, double max_norm,
                            double eps, double* total, float* norms, float* result, hipStream_t st) {
  if (max) grad_norm<true>(tb, count, parts, past, max_norm, eps, total, norms, result, st);
  else grad_norm<false>(tb, count, parts, past, max_norm, eps, total, norms, result, st);
  return hipGetLastError();
}

hipError_t launch_clip_coef(const double* total, bool max, double max_norm, double eps, float* result, hipStream_t st) {
  hipLaunchKernelGGL(k_clip_coef, dim3(1), dim3(1), 0, st, total, (int)max, max_norm, eps, result);
  return hipGetLastError();
}

hipError_t launch_grad_scale(const GradTable& tb, uint32_t parts, bool past, const float* coef, hipStream_t st) {
  if (past) hipLaunchKernelGGL(k_grad_scale<true>, dim3(parts), dim3(kThreads), 0, st, tb, coef);
  else hipLaunchKernelGGL(k_grad_scale<false>, dim3(parts), dim3(kThreads), 0, st, tb, coef);
  return hipGetLastError();
}

}  // namespace fp4r
