// Attention of several query rows per group over the compressed cache, for
// sequences of different lengths: the rows of a tree of drafted tokens
// (fibq_attn_tree), and single-token rows whose softmax weights are added to
// an accumulator per cached token (fibq_attn_decode_accum).
#include <hip/hip_runtime.h>

#include "device_common.h"
#include "fibq.h"
#include "fibq_internal.h"

namespace fibq {
namespace dev {
namespace sv {

// q~ = Pi q * qscale of one row, by all threads of the block; xs: D floats of LDS
template <int D>
__device__ void rotate_row(const void* q, int q_dtype, int64_t at, const float* R, float qscale,
                           float* xs, float* dst) {
  for (int i = threadIdx.x; i < D; i += blockDim.x)
    xs[i] = q_dtype == FIBQ_F32   ? static_cast<const float*>(q)[at + i]
            : q_dtype == FIBQ_F16 ? to_float(static_cast<const f16_t*>(q)[at + i])
                                  : to_float(static_cast<const bf16_t*>(q)[at + i]);
  __syncthreads();
  for (int i = threadIdx.x; i < D; i += blockDim.x) {
    float s = 0.0f;
    for (int j = 0; j < D; ++j) s = fmaf(R[i * D + j], xs[j], s);
    dst[i] = s * qscale;
  }
  __syncthreads();
}

template <int D>
__device__ float score(const float* qr, const uint8_t* row, uint16_t nu, const Shape& s,
                       const float* C) {
  float a = 0.0f;
  for (int m = 0; m < D / s.k; ++m) {
    const float* c = C + (size_t)extract_index(row, m, s.w) * s.k;
    for (int e = 0; e < s.k; ++e) a = fmaf(qr[m * s.k + e], c[e], a);
  }
  return a * half_bits_to_float(nu);
}

// One block per (group, row).  M = 0: single-token rows, else the drafted
// tokens of the group.
template <int D>
__global__ __launch_bounds__(256) void rows_kernel(
    const void* __restrict__ q, int q_dtype, const uint8_t* __restrict__ kp,
    const uint16_t* __restrict__ kn, const uint8_t* __restrict__ vp,
    const uint16_t* __restrict__ vn, const int32_t* __restrict__ lens,
    const uint64_t* __restrict__ masks, int64_t mask_stride, int M, int G, int64_t T_stride,
    Shape s, const float* __restrict__ R, const float* __restrict__ C, float qscale,
    float* __restrict__ stat, float* __restrict__ out) {
  __shared__ float xs[D], qr[D], red[4], ps[256], part[256];
  const int rows = max(M, 1) * G, tid = threadIdx.x;
  const int64_t g = blockIdx.x / rows;
  const int r = (int)(blockIdx.x % rows);
  float* o = out + (g * rows + r) * D;
  const int len = lens[g];
  if (len < 0 || len > T_stride - M) {
    for (int i = tid; i < D; i += 256) o[i] = NAN;
    if (stat && tid < 2) stat[(g * rows + r) * 2 + tid] = NAN;
    return;
  }
  rotate_row<D>(q, q_dtype, (g * rows + r) * D, R, qscale, xs, qr);
  const uint64_t mask = M > 0 ? masks[g * mask_stride + r / G] : 0;
  const int64_t base = g * T_stride;
  const int tot = len + M;
  const int dim = tid % D;
  float m = -INFINITY, l = 0.0f, acc = 0.0f;
  for (int t0 = 0; t0 < tot; t0 += 256) {
    const int t = t0 + tid;
    float sc = -INFINITY;
    if (t < tot && (t < len || (mask >> (t - len) & 1)))
      sc = score<D>(qr, kp + (base + t) * s.P, kn[base + t], s, C);
    float mx = wave_max(sc);
    if ((tid & 63) == 0) red[tid >> 6] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.0f : mn;
    const float f = exp2f(m - ref), p = exp2f(sc - ref);
    m = mn;
    l = l * f + p;
    acc *= f;
    ps[tid] = p;
    __syncthreads();
    for (int i = tid / D; i < min(256, tot - t0); i += 256 / D) {
      if (ps[i] == 0.0f) continue;
      const int64_t v = base + t0 + i;
      const uint32_t idx = extract_index(vp + v * s.P, dim / s.k, s.w);
      acc = fmaf(ps[i] * half_bits_to_float(vn[v]), C[(size_t)idx * s.k + dim % s.k], acc);
    }
    __syncthreads();
  }
  float ls = wave_sum(l);
  if ((tid & 63) == 0) red[tid >> 6] = ls;
  part[tid] = acc;
  __syncthreads();
  ls = red[0] + red[1] + red[2] + red[3];
  if (stat && tid == 0) {
    stat[(g * rows + r) * 2] = m;
    stat[(g * rows + r) * 2 + 1] = ls;
  }
  if (tid < D) {
    float a = 0.0f;
    for (int i = tid; i < 256; i += D) a += part[i];
    xs[tid] = ls == 0.0f ? 0.0f : a / ls;
  }
  __syncthreads();
  if (tid < D) {
    float a = 0.0f;
    for (int i = 0; i < D; ++i) a = fmaf(R[i * D + tid], xs[i], a);
    o[tid] = a;
  }
}

// acc[g][t] += sum over the heads of 2^(score - m) / l.
template <int D>
__global__ __launch_bounds__(256) void weights_kernel(
    const void* __restrict__ q, int q_dtype, const uint8_t* __restrict__ kp,
    const uint16_t* __restrict__ kn, const int32_t* __restrict__ lens, int G, int64_t T_stride,
    Shape s, const float* __restrict__ R, const float* __restrict__ C, float qscale,
    const float* __restrict__ stat, float* __restrict__ acc) {
  __shared__ float xs[D], qr[16 * D];
  const int64_t g = blockIdx.y;
  const int len = lens[g];
  if (len < 0 || len > T_stride || (int64_t)blockIdx.x * 256 >= len) return;
  for (int h = 0; h < G; ++h)
    rotate_row<D>(q, q_dtype, (g * G + h) * D, R, qscale, xs, qr + h * D);
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= len) return;
  const int64_t at = g * T_stride + t;
  float a = 0.0f;
  for (int h = 0; h < G; ++h) {
    const float sc = score<D>(qr + h * D, kp + at * s.P, kn[at], s, C);
    const float m = stat[(g * G + h) * 2], l = stat[(g * G + h) * 2 + 1];
    a += exp2f(sc - m) / l;
  }
  acc[at] += a;
}

}  // namespace sv

size_t serve_attn_workspace_bytes(int64_t n_groups, int M, int G, const Shape& s) {
  return M > 0 ? 0 : (size_t)n_groups * G * 2 * 4;
}

template <int D>
static int launch_serve(const ServeAttn& a, hipStream_t st) {
  const int rows = (a.M > 0 ? a.M : 1) * a.G;
  const float qscale = a.scale * 1.4426950408889634f;  // base-2 softmax
  float* stat = a.acc ? static_cast<float*>(a.ws) : nullptr;
  hipLaunchKernelGGL(sv::rows_kernel<D>, dim3((unsigned)(a.n_groups * rows)), dim3(256), 0, st, a.q,
                     a.q_dtype, a.kp, a.kn, a.vp, a.vn, a.lens, a.masks, a.mask_stride, a.M, a.G,
                     a.T_stride, a.s, a.R, a.C, qscale, stat, a.out);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.acc || a.T_stride == 0) return (int)e;
  hipLaunchKernelGGL(sv::weights_kernel<D>,
                     dim3((unsigned)((a.T_stride + 255) / 256), (unsigned)a.n_groups), dim3(256),
                     0, st, a.q, a.q_dtype, a.kp, a.kn, a.lens, a.G, a.T_stride, a.s, a.R, a.C,
                     qscale, stat, a.acc);
  return (int)hipGetLastError();
}

int launch_serve_attn(const ServeAttn& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  return a.s.d == 64 ? launch_serve<64>(a, st) : launch_serve<128>(a, st);
}

}  // namespace dev
}  // namespace fibq
