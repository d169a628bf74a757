// Root-mean-square norm with the residual's addition and an output in E4M3, and its gradients.
//   h = round_T(x + r),  rstd = 1 / sqrt(sum(h^2) / cols + eps),  y = (h rstd) gain
//   per row, or per group of 32, 64 or 128 columns: amax = max(max |y|, 2^-100),
//   s = amax / 448, or the smallest power of two with amax <= 448 s;  code = E4M3(y / s)
// The squares are exact in binary64 and added there, so rstd is the rounding of the exact
// value but for a few in 2^20 rows: in those its last place, and with it codes and scales, may
// depend on how the row is cut over threads, which the shape decides.
//   g = dy gain,  xhat = h rstd,  c = mean(g xhat),  dx = rstd (g - xhat c) + dh,
//   dgain = sum over rows of dy xhat
// In the backward pass the row's dot product and a workgroup's part of dgain are binary32 sums: each
// term is a product of binary32 roundings already, of 16-bit factors for most, and parts of
// dgain in binary64 would take twice the registers of a thread's columns.  Their join, where
// hundreds of parts meet, is binary64 (64 x 1024 FP32: error 5.9e-8, 9.5e-8 joined in binary32).
// Both passes are bound by memory: a row is read once and stays in registers.  A thread holds
// VPT vectors of 8 columns, as many vectors apart as threads share the row, so a group of columns
// lies in 4, 8 or 16 adjacent lanes.  A row takes whole waves, or 16 or 32 lanes of one where it
// is narrow (the heads of an attention: 32768 x 96 BF16 19.4 -> 10.2 us, its gradients 25.2 ->
// 17.9); with a row in whole waves their number fits the row, not the next power of two (8192 x 4099
// 81.6 -> 75 and 111.4 -> 93).
#include "device.h"
#include "internal.h"
#include "vec.h"

namespace fp4r {
namespace {

constexpr float kAmaxMin = 0x1p-100f;

// The larger of two magnitudes, NaN if either is (one instruction takes three).
FP4R_DEV float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Lanes l and l ^ 1, l ^ 2 of a quad, then the other quad of 8 lanes, the other half of 16.
template <int CTRL>
FP4R_DEV float dpp_f(float v) {
  return __uint_as_float(dpp_u<CTRL>(__float_as_uint(v)));
}
FP4R_DEV float group_max(float v, int lanes) {   // lanes: 4, 8 or 16 (uniform)
  v = larger(v, dpp_f<0xB1>(v));
  v = larger(v, dpp_f<0x4E>(v));
  if (lanes > 4) v = larger(v, dpp_f<0x141>(v));
  if (lanes > 8) v = larger(v, dpp_f<0x140>(v));
  return v;
}
FP4R_DEV float lane_f(float v, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}
FP4R_DEV float wave_max(float v) {
  v = group_max(v, 16);
  return larger(larger(lane_f(v, 0), lane_f(v, 16)), larger(lane_f(v, 32), lane_f(v, 48)));
}
// Sums over the lanes of a row: SUB lanes (16 or 32), or the wave for SUB 0.
template <int SUB>
FP4R_DEV float lanes_sum(float v) {
  v = v + dpp_f<0xB1>(v);
  v = v + dpp_f<0x4E>(v);
  v = v + dpp_f<0x141>(v);
  v = v + dpp_f<0x140>(v);
  if constexpr (SUB == 16) return v;
  else if constexpr (SUB == 32) return v + __shfl_xor(v, 16);
  else return (lane_f(v, 0) + lane_f(v, 16)) + (lane_f(v, 32) + lane_f(v, 48));
}
template <int SUB>
FP4R_DEV double lanes_sum(double v) {
  if constexpr (SUB == 0) return wave_sum_d(v);
  v = v + dpp_d<0xB1>(v);
  v = v + dpp_d<0x4E>(v);
  v = v + dpp_d<0x141>(v);
  v = v + dpp_d<0x140>(v);
  return SUB == 16 ? v : v + __shfl_xor(v, 16);
}
template <int SUB>
FP4R_DEV float lanes_max(float v) {
  if constexpr (SUB == 0) return wave_max(v);
  v = group_max(v, 16);
  return SUB == 16 ? v : larger(v, __shfl_xor(v, 16));
}

// 1 / sqrt(a) for 0 < a < 2^1000: the instruction's estimate and two Newton steps.
FP4R_DEV double rsqrt64(double a) {
  double r = __builtin_amdgcn_rsq(a);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const double e = __builtin_fma(-a * r, r, 1.0);
    r = __builtin_fma(r * 0.5, e, r);
  }
  return r;
}

// The scale of a group as it is stored, and what its values are multiplied by: NaN where the
// largest is an infinity or NaN, so that no finite value of the group passes for 0.
FP4R_DEV float scale_of(float amax, int e8m0, uint32_t& stored) {
  amax = larger(amax, kAmaxMin);
  if (e8m0) {
    // amax = 1.m 2^(e - 127) and 448 = 1.75 2^8; E8M0 holds NaN as 255
    const uint32_t b = __float_as_uint(amax), e = (b >> 23) - 8u + ((b & 0x7FFFFFu) > 0x600000u);
    const bool finite = b < 0x7F800000u;
    stored = finite ? e : 255u;
    return __uint_as_float(finite ? (254u - e) << 23 : 0x7FC00000u);
  }
  stored = __float_as_uint(scale_448(amax));
  return inverse_448(amax);
}
FP4R_DEV void store_scale(const RmsArgs& a, int64_t i, uint32_t stored) {
  if (a.e8m0) reinterpret_cast<uint8_t*>(a.scales)[i] = (uint8_t)stored;
  else reinterpret_cast<uint32_t*>(a.scales)[i] = stored;
}

// Eight gains as they lie in memory: words of FP32, or half as many of BF16.
struct Gain8 {
  Raw8<float> f;
};
FP4R_DEV Gain8 load_gain(const void* gain, int f32, int col, int n) {
  Gain8 g;
  if (f32) {
    g.f = load_raw8((const float*)gain + col, n);
  } else {
    const Raw8<bf16_t> b = load_raw8((const bf16_t*)gain + col, n);
#pragma unroll
    for (int k = 0; k < 4; ++k) g.f.w[k] = b.w[k];
  }
  return g;
}
FP4R_DEV void unpack_gain(const Gain8& g, int f32, float (&x)[8]) {
  if (f32) {
    unpack8(g.f, x);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) unpack2(bf16_t{}, g.f.w[k], x[2 * k], x[2 * k + 1]);
  }
}

FP4R_DEV void store_codes(uint8_t* p, int n, const float (&y)[8], float inv) {
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k] * inv, y[4 * k + 1] * inv, 0, false);
    w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k + 2] * inv, y[4 * k + 3] * inv, v, true);
  }
  if (n >= 8) {
    *reinterpret_cast<u32x2_a1*>(p) = u32x2{w[0], w[1]};
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) p[k] = (uint8_t)(w[k / 4] >> (8 * (k & 3)));
  }
}

// The row of a thread among its workgroup's.
template <int SUB>
FP4R_DEV int row_slot(const RowShare& s) {
  return SUB ? threadIdx.x / (SUB ? SUB : 1) : (int)(threadIdx.x * s.inverse >> 20);
}
RowShare row_share(int tpr, int slots) { return RowShare{tpr, slots, ((1u << 20) + tpr - 1) / tpr}; }

// SUB: lanes a row, or 0 for whole waves.
template <class T, int VPT, int SUB>
__global__ __launch_bounds__(1024) void k_rmsnorm(RmsArgs a) {
  __shared__ double red_s[16];                        // one a wave
  __shared__ float red_m[16];
  const int TPR = SUB ? SUB : a.share.tpr, slots = a.share.slots;
  const int slot = row_slot<SUB>(a.share), t = threadIdx.x - slot * TPR;
  const int wpr = TPR / 64, wave0 = slot * wpr;       // waves a row (0: less than one), the row's first
  const int lane16 = threadIdx.x & 15;                // takes a wave's part: every 16 lanes join them all
  const int64_t row = (int64_t)blockIdx.x * slots + slot;
  const bool live = row < a.rows;
  const int cols = live ? a.cols : 0;                 // a slot past the last row reads and writes nothing
  Raw8<T> h[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = (i * TPR + t) * 8, n = min(8, cols - c);
    h[i] = a.x_past ? load_raw8<T, true>((const T*)a.x + row * a.ld_x + c, n)
                    : load_raw8<T>((const T*)a.x + row * a.ld_x + c, n);
  }
  if (a.r) {
    Raw8<T> r[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + t) * 8, n = min(8, cols - c);
      r[i] = load_raw8<T, true>((const T*)a.r + row * a.ld_r + c, n);
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float u[8], v[8];
      unpack8(h[i], u);
      unpack8(r[i], v);
#pragma unroll
      for (int k = 0; k < 8; ++k) u[k] += v[k];
      h[i] = pack8<T>(u);
    }
  }
  // the gain is on its way while the row is summed
  Gain8 gain[VPT];
  if (a.gain) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + t) * 8;
      gain[i] = load_gain(a.gain, a.gain_f32, c, min(8, cols - c));
    }
  }
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = (i * TPR + t) * 8, n = min(8, cols - c);
    if (a.h) store_raw8<T, true>((T*)a.h + row * a.ld_h + c, n, h[i]);
    float u[8];
    unpack8(h[i], u);
#pragma unroll
    for (int k = 0; k < 8; ++k) s = __builtin_fma((double)u[k], (double)u[k], s);
  }
  s = lanes_sum<SUB>(s);
  if (wpr > 1) {
    if ((threadIdx.x & 63) == 0) red_s[threadIdx.x >> 6] = s;
    __syncthreads();
    s = lanes_sum<16>(lane16 < wpr ? red_s[wave0 + lane16] : 0.0);
  }
  const float rstd = (float)rsqrt64(s / (double)a.cols + a.eps);
  if (t == 0 && live) {
    if (a.rstd) a.rstd[row] = rstd;
    if (a.status && !(s < __builtin_inf())) *a.status = kErrNonFinite;
  }
  if (!a.codes && !a.y) return;
  const auto normalised = [&](int i, float (&y)[8]) {
    unpack8(h[i], y);
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] *= rstd;
    if (!a.gain) return;
    float g[8];
    unpack_gain(gain[i], a.gain_f32, g);
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] *= g[k];
  };
  float top = 0.0f;
  const int lanes = a.group / 8;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = (i * TPR + t) * 8, n = min(8, cols - c);
    float y[8];
    normalised(i, y);
    if (a.y) store_raw8((T*)a.y + row * a.ld_y + c, n, pack8<T>(y));
    if (!a.codes) continue;
    float m = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) m = larger(m, fabsf(y[k]));
    if (lanes) {
      m = group_max(m, lanes);
      uint32_t stored;
      const float inv = scale_of(m, a.e8m0, stored);
      if (n > 0) store_codes(a.codes + row * a.cols + c, n, y, inv);
      if (n > 0 && (t & (lanes - 1)) == 0) {
        store_scale(a, row * a.groups + c / a.group, stored);
        if (a.status && !(m < __builtin_inff())) *a.status = kErrNonFinite;
      }
    }
    top = larger(top, m);
  }
  if (!a.codes || lanes) return;
  top = lanes_max<SUB>(top);
  if (wpr > 1) {
    if ((threadIdx.x & 63) == 0) red_m[threadIdx.x >> 6] = top;
    __syncthreads();
    top = lanes_max<16>(lane16 < wpr ? red_m[wave0 + lane16] : 0.0f);
  }
  uint32_t stored;
  const float inv = scale_of(top, a.e8m0, stored);
  if (t == 0 && live) {
    store_scale(a, row, stored);
    if (a.status && !(top < __builtin_inff())) *a.status = kErrNonFinite;
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = (i * TPR + t) * 8, n = min(8, cols - c);
    if (n <= 0) continue;
    float y[8];
    normalised(i, y);
    store_codes(a.codes + row * a.cols + c, n, y, inv);
  }
}

template <class T, int VPT, int SUB>
void run_rmsnorm(RmsArgs a, int tpr, int slots, hipStream_t st) {
  a.share = row_share(tpr, slots);
  hipLaunchKernelGGL((k_rmsnorm<T, VPT, SUB>), dim3((uint32_t)((a.rows + slots - 1) / slots)), dim3(tpr * slots), 0, st,
                     a);
}

// Whole waves that hold v vectors.
int wave_threads(int64_t v) { return (int)((v + 63) / 64 * 64); }

// Many rows: 8 or 16 columns a thread (8192 x 4096: 2 vectors of 256 threads 42.3 us, 1 of 512
// 44.0, 4 of 128 44.4, 8 of 64 49.5; 16384 x 8192: 2 of 512 160, 4 of 256 161, 1 of 1024 188).
// Few rows do not fill the CUs, so that a row's own latency counts: as many threads as its
// columns allow (1 x 4096: 1 of 512 3.5 us, 2 of 256 4.2, 8 of 64 8.7; 256 rows 3.9, 4.6, 10.0;
// 1024 rows 8.3, 7.4, 11.7).
constexpr int64_t kFewRows = 512;
template <class T>
void pick_rmsnorm(const RmsArgs& a, hipStream_t st) {
  const int64_t v = (a.cols + 7) / 8;
  const bool few = a.rows <= kFewRows;
  if (v <= 16) return run_rmsnorm<T, 1, 16>(a, 16, 16, st);
  if (v <= 32) return run_rmsnorm<T, 1, 32>(a, 32, 8, st);
  if (v <= 256 || (v <= 1024 && few)) {
    const int tpr = wave_threads(v);
    return run_rmsnorm<T, 1, 0>(a, tpr, tpr <= 128 ? 256 / tpr : 1, st);
  }
  if (v <= 2048) return run_rmsnorm<T, 2, 0>(a, wave_threads((v + 1) / 2), 1, st);
  run_rmsnorm<T, 4, 0>(a, wave_threads((v + 3) / 4), 1, st);
}

// ---------------------------------------------------------------------------
// Gradients.  A workgroup of RPG row slots of TPR threads walks over rows, each thread keeping
// its columns' part of dgain in registers; at the end the slots are added in LDS and the
// workgroup writes one row of partials, which k_rms_dgain adds in order.

// SUB as above; MAXT: the most threads of a workgroup; GAIN: with dgain (the widest rows leave it
// to k_rms_cols, since the registers do not hold them beside their part of it, and read dh late).
template <class T, int VPT, int SUB, int MAXT, bool GAIN>
__global__ __launch_bounds__(MAXT) void k_rms_bwd(RmsBwdArgs a) {
  __shared__ float red[2][MAXT / 64];
  __shared__ float slab[VPT == 1 ? 512 * 8 : 1];      // only rows of up to 256 threads share a workgroup
  const int TPR = SUB ? SUB : a.share.tpr, RPG = a.share.slots;
  const int slot = row_slot<SUB>(a.share), t = threadIdx.x - slot * TPR;
  const int wpr = TPR / 64, wave0 = slot * wpr, lane16 = threadIdx.x & 15;
  float acc[GAIN ? VPT : 1][8];
#pragma unroll
  for (int i = 0; i < (GAIN ? VPT : 1); ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[i][k] = 0.0f;
  const float inv_cols = 1.0f / (float)a.cols;
  int side = 0;
  for (int64_t base = (int64_t)blockIdx.x * RPG; base < a.rows; base += (int64_t)gridDim.x * RPG, side ^= 1) {
    const int64_t row = base + slot;
    const bool live = row < a.rows;
    // h was written in the forward pass, long ago; dy and dh were written just now, and dx is
    // read soon: h passes the caches, and so does dx, which is written after all that is read
    // (8192 x 4096 BF16: 57.0 us with nothing past them, 55.0 so, and 16384 x 8192: 197, 194;
    // with dy and dh past them too, 2048 x 4096, which fit: 22.6 us for 19.6)
    Raw8<T> h[VPT], d[VPT], e[GAIN ? VPT : 1];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + t) * 8, n = live ? min(8, a.cols - c) : 0;
      h[i] = load_raw8<T, true>((const T*)a.h + row * a.ld_h + c, n);
      d[i] = load_raw8((const T*)a.dy + row * a.ld_dy + c, n);
    }
    if (GAIN && a.dh) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int c = (i * TPR + t) * 8, n = live ? min(8, a.cols - c) : 0;
        e[i] = load_raw8((const T*)a.dh + row * a.ld_dh + c, n);
      }
    }
    const float rstd = live ? a.rstd[row] : 0.0f;
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + t) * 8, n = min(8, a.cols - c);
      float x[8], y[8], g[8];
      unpack8(h[i], x);
      unpack8(d[i], y);
      if (a.gain) {
        unpack_gain(load_gain(a.gain, a.gain_f32, c, n), a.gain_f32, g);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = 1.0f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float xhat = x[k] * rstd;
        if (GAIN) acc[GAIN ? i : 0][k] = fmaf(y[k], xhat, acc[GAIN ? i : 0][k]);
        dot = fmaf(y[k] * g[k], xhat, dot);
      }
    }
    dot = lanes_sum<SUB>(dot);
    if (wpr > 1) {
      if ((threadIdx.x & 63) == 0) red[side][threadIdx.x >> 6] = dot;
      __syncthreads();   // two sides: the next row's values do not overtake this row's readers
      dot = lanes_sum<16>(lane16 < wpr ? red[side][wave0 + lane16] : 0.0f);
    }
    const float mean = dot * inv_cols;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + t) * 8, n = min(8, a.cols - c);
      if (!live || n <= 0) continue;
      float x[8], y[8], g[8], o[8];
      unpack8(h[i], x);
      unpack8(d[i], y);
      if (a.gain) {
        unpack_gain(load_gain(a.gain, a.gain_f32, c, n), a.gain_f32, g);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = 1.0f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = rstd * (y[k] * g[k] - (x[k] * rstd) * mean);
      if (a.dh) {
        if constexpr (!GAIN) e[0] = load_raw8((const T*)a.dh + row * a.ld_dh + c, n);
        unpack8(e[GAIN ? i : 0], x);
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] += x[k];
      }
      store_raw8<T, true>((T*)a.dx + row * a.ld_dx + c, n, pack8<T>(o));
    }
  }
  if (!GAIN || !a.dgain) return;
  float* out = a.partial + (int64_t)blockIdx.x * a.cols;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = (i * TPR + t) * 8, n = min(8, a.cols - c);
    if (VPT == 1 && RPG > 1) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 8; ++k) slab[(slot * 8 + k) * TPR + t] = acc[GAIN ? i : 0][k];
      __syncthreads();
      if (slot == 0) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          for (int q = 1; q < RPG; ++q) acc[GAIN ? i : 0][k] += slab[(q * 8 + k) * TPR + t];
      }
    }
    if (slot == 0 && n > 0) store_raw8(out + c, n, pack8<float>(acc[GAIN ? i : 0]));
  }
}

// dgain of the widest rows: 512 columns of a chunk of rows a workgroup, a wave every fourth row,
// four rows in flight.
template <class T>
__global__ __launch_bounds__(256) void k_rms_cols(RmsBwdArgs a, int64_t chunk) {
  __shared__ float red[3][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 512 + lane * 8, n = min(8, a.cols - c);
  const int64_t r1 = min(a.rows, (int64_t)(blockIdx.y + 1) * chunk);
  float acc[8] = {};
  for (int64_t r = (int64_t)blockIdx.y * chunk + wave; r < r1; r += 16) {
    Raw8<T> h[4], d[4];
    float rstd[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t row = r + 4 * u;
      const int m = row < r1 ? n : 0;
      h[u] = load_raw8((const T*)a.h + row * a.ld_h + c, m);
      d[u] = load_raw8((const T*)a.dy + row * a.ld_dy + c, m);
      rstd[u] = row < r1 ? a.rstd[row] : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float x[8], y[8];
      unpack8(h[u], x);
      unpack8(d[u], y);
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[k] = fmaf(y[k], x[k] * rstd[u], acc[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (wave) red[wave - 1][k * 64 + lane] = acc[k];
  __syncthreads();
  if (wave || n <= 0) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) acc[k] += (red[0][k * 64 + lane] + red[1][k * 64 + lane]) + red[2][k * 64 + lane];
  store_raw8(a.partial + (int64_t)blockIdx.y * a.cols + c, n, pack8<float>(acc));
}

// 16 columns by 64 slices of the partial rows a workgroup: each thread adds four columns of
// every 64th row, eight loads in flight, then the slices in pairs.  In binary64, so that what
// workgroups of opposite sign cancel is not lost: the partials are binary32 sums of the rows of one
// workgroup, and the join adds one rounding.
__global__ __launch_bounds__(256) void k_rms_dgain(const float* partial, int count, int cols, float* dgain) {
  __shared__ double red[16][65];
  const int q = threadIdx.x & 3, slice = threadIdx.x >> 2, c = blockIdx.x * 16 + q * 4, n = min(4, cols - c);
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  if (n > 0) {
    for (int p = slice; p < count; p += 64 * 8) {
      float x[8][4];
#pragma unroll
      for (int u = 0; u < 8; ++u) load_vec<float, 4>(partial + (int64_t)min(p + u * 64, count - 1) * cols + c, n, x[u]);
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] += p + u * 64 < count ? (double)x[u][k] : 0.0;
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) red[q * 4 + k][slice] = s[k];
  __syncthreads();
  // 16 threads a column
  const int col = threadIdx.x >> 4, l = threadIdx.x & 15;
  double v = (red[col][l] + red[col][l + 16]) + (red[col][l + 32] + red[col][l + 48]);
#pragma unroll
  for (int o = 8; o; o >>= 1) v += __shfl_xor(v, o);
  if (l == 0 && blockIdx.x * 16 + col < cols) dgain[blockIdx.x * 16 + col] = (float)v;
}

// Threads a row, vectors a thread and rows a workgroup.  A thread keeps 8 columns where 768
// threads cover the row, so that 4 to 6 waves fit a SIMD (8192 x 4096: 1 vector of 512 threads
// 56.0 us, 2 of 256 56.8, 4 of 128 66.8; 8192 x 5120 1 of 640 69.1, 2 of 320 72.3; 8192 x 7168
// the same; 16384 x 8192 2 of 512 197, 4 of 256 222, 1 of 1024 209), and narrow rows share
// workgroups of 512 threads (1024: 8192 x 2048 31.0 us for 29.0).  Rows past 16384 columns
// leave dgain to a pass of its own (with it the registers spill: 4096 x 20000 250 us, so 217);
// past 24576, 1024 threads a row, a thread has 128 registers and a few spill all the same (17 of
// FP32 rows, 9 of BF16, 2 of FP16: 2048 x 32768 BF16 173 us, FP32 341, 3.1 TB/s).
struct BwdShape {
  int tpr, vpt, slots;
};
BwdShape bwd_shape(int64_t cols) {
  const int64_t v = (cols + 7) / 8;
  if (v <= 16) return {16, 1, 32};
  if (v <= 32) return {32, 1, 16};
  if (v <= 768) {
    const int tpr = wave_threads(v);
    return {tpr, 1, tpr <= 512 ? 512 / tpr : 1};
  }
  if (v <= 2048) return {wave_threads((v + 1) / 2), 2, 1};
  return {wave_threads((v + 3) / 4), 4, 1};
}

// k_rms_cols: its chunks of rows, about 2048 workgroups of at least 64 rows.
int64_t col_chunk(int64_t rows, int64_t cols) {
  const int64_t chunks = 2048 / ((cols + 511) / 512), chunk = (rows + chunks - 1) / chunks;
  return chunk < 64 ? 64 : chunk;
}

template <class T>
void run_bwd(RmsBwdArgs a, uint32_t grid, hipStream_t st) {
  const BwdShape s = bwd_shape(a.cols);
  const dim3 nt(s.tpr * s.slots);
  a.share = row_share(s.tpr, s.slots);
  if (s.tpr == 16) hipLaunchKernelGGL((k_rms_bwd<T, 1, 16, 512, true>), dim3(grid), nt, 0, st, a);
  else if (s.tpr == 32) hipLaunchKernelGGL((k_rms_bwd<T, 1, 32, 512, true>), dim3(grid), nt, 0, st, a);
  else if (s.vpt == 1) hipLaunchKernelGGL((k_rms_bwd<T, 1, 0, 768, true>), dim3(grid), nt, 0, st, a);
  else if (s.vpt == 2) hipLaunchKernelGGL((k_rms_bwd<T, 2, 0, 1024, true>), dim3(grid), nt, 0, st, a);
  else {
    // dgain first: dx may be written over h or dy
    if (a.dgain)
      hipLaunchKernelGGL(k_rms_cols<T>, dim3((uint32_t)((a.cols + 511) / 512), grid), dim3(256), 0, st, a,
                         col_chunk(a.rows, a.cols));
    const dim3 rows(a.rows < 512 ? (uint32_t)a.rows : 512);
    if (s.tpr <= 768) hipLaunchKernelGGL((k_rms_bwd<T, 4, 0, 768, false>), rows, nt, 0, st, a);
    else hipLaunchKernelGGL((k_rms_bwd<T, 4, 0, 1024, false>), rows, nt, 0, st, a);
  }
}

}  // namespace

hipError_t launch_rmsnorm(const RmsArgs& a, hipStream_t st) {
  switch (a.type) {
    case 0: pick_rmsnorm<float>(a, st); break;
    case 1: pick_rmsnorm<bf16_t>(a, st); break;
    default: pick_rmsnorm<f16_t>(a, st); break;
  }
  return hipGetLastError();
}

// One workgroup a CU; two, or as many as make 1024 threads, of up to 768 threads where there are
// eight turns a CU at least: every workgroup adds a row of partials (256 and 512 workgroups:
// 1024 x 4096 14.9 and 17.1 us, 2048 x 4096 20.1 and 19.9, 4096 x 4096 32.8 and 30.4, 32768 x 128
// 38.5 and 25.5; 512 and 768 of 320 threads: 8192 x 2560 40.4 and 36.5; 2048 x 16384, of 1024
// threads, 256 and 512: 63.7 and 72.0).
int64_t rms_bwd_groups(int64_t rows, int64_t cols) {
  const BwdShape s = bwd_shape(cols);
  const int threads = s.tpr * s.slots;
  if (s.vpt == 4) return (rows + col_chunk(rows, cols) - 1) / col_chunk(rows, cols);
  const int64_t all = (rows + s.slots - 1) / s.slots;
  int64_t most = 256;
  if (threads <= 768 && s.vpt <= 2 && all >= 2048) most *= threads <= 341 ? 3 : 2;
  return all < most ? all : most;
}

hipError_t launch_rmsnorm_backward(const RmsBwdArgs& a, hipStream_t st) {
  const uint32_t grid = (uint32_t)rms_bwd_groups(a.rows, a.cols);
  if (grid) {
    switch (a.type) {
      case 0: run_bwd<float>(a, grid, st); break;
      case 1: run_bwd<bf16_t>(a, grid, st); break;
      default: run_bwd<f16_t>(a, grid, st); break;
    }
  }
  if (a.dgain)
    hipLaunchKernelGGL(k_rms_dgain, dim3((uint32_t)((a.cols + 15) / 16)), dim3(256), 0, st, a.partial, (int)grid,
                       (int)a.cols, a.dgain);
  return hipGetLastError();
}

}  // namespace fp4r
