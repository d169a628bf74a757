// The global norm of a list of gradient tensors and the clipping by it.
//   L2:  total = sum over all elements of x^2,  norm = sqrt(total)
//   max: total = max |x|,                       norm = total
//   coef = min(1, max_norm / (norm + eps)),     out = fl(x coef)
// One pass over the data for the norm (each element is converted to binary64, where its
// square is exact, and added there: no overflow and no rounding that matters), one more for
// the clipping.  Both are bound by memory.
//
// A tensor is cut into parts of 16-byte vectors by its own size alone; a workgroup takes one
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

// The sum (or maximum) over a workgroup, in thread 0.
template <bool MAX>
FP4R_DEV double block_join(double v) {
  __shared__ double red[kThreads / 64];
#pragma unroll
  for (int o = 32; o; o >>= 1) v = join<MAX>(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) v = join<MAX>(v, red[w]);
  return v;
}

// Calls f(first element's offset in the input, ... in the output, count) for every vector of
// this thread in vectors [v0, v1) of the tensor; count is VE but for the last vector of a row.
template <int VE, class F>
FP4R_DEV void each_vector(const GradRef& t, int64_t v0, int64_t v1, F f) {
  const int64_t per_row = (t.cols + VE - 1) / VE;
  for (int64_t v = v0 + threadIdx.x; v < v1; v += kThreads) {
    const int64_t row = t.rows == 1 ? 0 : v / per_row, c = (v - row * per_row) * VE;
    f(row * t.ld_in + c, row * t.ld_out + c, (int)min((int64_t)VE, t.cols - c));
  }
}

template <class T, bool MAX>
FP4R_DEV double part_value(const GradRef& t, int64_t v0, int64_t v1) {
  constexpr int VE = 16 / sizeof(T);
  const T* in = (const T*)t.in;
  double acc = 0.0;
  each_vector<VE>(t, v0, v1, [&](int64_t i, int64_t, int n) {
    float x[VE];
    load_vec<T, VE>(in + i, n, x);
#pragma unroll
    for (int k = 0; k < VE; ++k) acc = take<MAX>(acc, x[k]);
  });
  return acc;
}

// Writes a chunk of the table: workgroup i its tensor and that tensor's parts.
__global__ __launch_bounds__(kThreads) void k_grad_table(GradChunk ch, GradTable tb, uint32_t first_tensor) {
  const int i = blockIdx.x;
  const uint32_t t = first_tensor + i;
  if (threadIdx.x == 0) tb.tensors[t] = ch.t[i];
  for (uint32_t p = threadIdx.x; p < ch.parts[i]; p += kThreads) tb.parts[ch.t[i].first + p] = GradPart{t, p};
}

template <bool MAX>
__global__ __launch_bounds__(kThreads) void k_grad_parts(GradTable tb) {
  const GradPart p = tb.parts[blockIdx.x];
  const GradRef& t = tb.tensors[p.tensor];
  const int64_t v0 = (int64_t)p.part << t.shift, v1 = min(t.vectors, v0 + (int64_t(1) << t.shift));
  double v;
  switch (t.type & 3) {
    case 0: v = part_value<float, MAX>(t, v0, v1); break;
    case 1: v = part_value<bf16_t, MAX>(t, v0, v1); break;
    default: v = part_value<f16_t, MAX>(t, v0, v1); break;
  }
  v = block_join<MAX>(v);
  if (threadIdx.x == 0) {
    tb.partial[blockIdx.x] = v;
    if (blockIdx.x == 0) *tb.ticket = 0u;
  }
}

FP4R_DEV void write_result(double total, bool max, double max_norm, double eps, float* result) {
  const double norm = max ? total : __builtin_sqrt(total);
  const double q = max_norm / (norm + eps);
  result[0] = (float)norm;
  result[1] = q > 1.0 ? 1.0f : (float)q;   // a NaN stays
}

// A wave per tensor joins its parts (at most 1024); the last workgroup to finish joins the
// tensors.  Up to kWaves tensors there is one workgroup, and nothing to wait for.
constexpr int kWaves = 16;
template <bool MAX>
__global__ __launch_bounds__(kWaves * 64) void k_grad_total(GradTable tb, uint32_t count, double max_norm, double eps,
                                                            double* total, float* norms, float* result) {
  __shared__ double red[kWaves];
  __shared__ bool last;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t t = blockIdx.x * kWaves + wave;
  double v = 0.0;
  if (t < count) {
    const uint32_t p0 = tb.tensors[t].first, p1 = tb.tensors[t + 1].first;
    for (uint32_t p = p0 + lane; p < p1; p += 64) v = join<MAX>(v, tb.partial[p]);
#pragma unroll
    for (int o = 32; o; o >>= 1) v = join<MAX>(v, __shfl_xor(v, o));
    if (lane == 0) {
      if (norms) norms[t] = (float)(MAX ? v : __builtin_sqrt(v));
      if (gridDim.x > 1) __hip_atomic_store(&tb.sums[t], v, __ATOMIC_RELEASE, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  if (gridDim.x > 1) {
    __syncthreads();
    if (threadIdx.x == 0)
      last = __hip_atomic_fetch_add(tb.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    v = 0.0;
    for (uint32_t i = threadIdx.x; i < count; i += kWaves * 64)
      v = join<MAX>(v, __hip_atomic_load(&tb.sums[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
#pragma unroll
    for (int o = 32; o; o >>= 1) v = join<MAX>(v, __shfl_xor(v, o));
  }
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

template <class TI, class TO>
FP4R_DEV void scale_part(const GradRef& t, int64_t v0, int64_t v1, float coef) {
  constexpr int VE = 16 / sizeof(TI);
  const TI* in = (const TI*)t.in;
  TO* out = (TO*)t.out;
  each_vector<VE>(t, v0, v1, [&](int64_t i, int64_t o, int n) {
    float x[VE];
    load_vec<TI, VE>(in + i, n, x);
#pragma unroll
    for (int k = 0; k < VE; ++k) x[k] *= coef;
    store_vec<TO, VE>(out + o, n, x);
  });
}

__global__ __launch_bounds__(kThreads) void k_grad_scale(GradTable tb, const float* coef_p) {
  const GradPart p = tb.parts[blockIdx.x];
  const GradRef& t = tb.tensors[p.tensor];
  const float coef = *coef_p;
  if (coef == 1.0f && t.in == t.out) return;   // in place, and x 1 is x
  const int64_t v0 = (int64_t)p.part << t.shift, v1 = min(t.vectors, v0 + (int64_t(1) << t.shift));
  switch (t.type) {
    case 0 | 0 << 2: scale_part<float, float>(t, v0, v1, coef); break;
    case 0 | 1 << 2: scale_part<float, bf16_t>(t, v0, v1, coef); break;
    case 0 | 2 << 2: scale_part<float, f16_t>(t, v0, v1, coef); break;
    case 1 | 0 << 2: scale_part<bf16_t, float>(t, v0, v1, coef); break;
    case 1 | 1 << 2: scale_part<bf16_t, bf16_t>(t, v0, v1, coef); break;
    case 1 | 2 << 2: scale_part<bf16_t, f16_t>(t, v0, v1, coef); break;
    case 2 | 0 << 2: scale_part<f16_t, float>(t, v0, v1, coef); break;
    case 2 | 1 << 2: scale_part<f16_t, bf16_t>(t, v0, v1, coef); break;
    default: scale_part<f16_t, f16_t>(t, v0, v1, coef); break;
  }
}

}  // namespace

hipError_t launch_grad_table(const GradChunk& ch, const GradTable& tb, uint32_t first_tensor, hipStream_t st) {
  hipLaunchKernelGGL(k_grad_table, dim3(ch.count), dim3(kThreads), 0, st, ch, tb, first_tensor);
  return hipGetLastError();
}

hipError_t launch_grad_norm(const GradTable& tb, uint32_t count, uint32_t parts, bool max, double max_norm, double eps,
                            double* total, float* norms, float* result, hipStream_t st) {
  const dim3 groups(count ? (count + kWaves - 1) / kWaves : 1), nt(kWaves * 64);
  if (max) {
    if (parts) hipLaunchKernelGGL(k_grad_parts<true>, dim3(parts), dim3(kThreads), 0, st, tb);
    hipLaunchKernelGGL(k_grad_total<true>, groups, nt, 0, st, tb, count, max_norm, eps, total, norms, result);
  } else {
    if (parts) hipLaunchKernelGGL(k_grad_parts<false>, dim3(parts), dim3(kThreads), 0, st, tb);
    hipLaunchKernelGGL(k_grad_total<false>, groups, nt, 0, st, tb, count, max_norm, eps, total, norms, result);
  }
  return hipGetLastError();
}

hipError_t launch_clip_coef(const double* total, bool max, double max_norm, double eps, float* result, hipStream_t st) {
  hipLaunchKernelGGL(k_clip_coef, dim3(1), dim3(1), 0, st, total, (int)max, max_norm, eps, result);
  return hipGetLastError();
}

hipError_t launch_grad_scale(const GradTable& tb, uint32_t parts, const float* coef, hipStream_t st) {
  hipLaunchKernelGGL(k_grad_scale, dim3(parts), dim3(kThreads), 0, st, tb, coef);
  return hipGetLastError();
}

}  // namespace fp4r
