// Rows of the compressed cache that move: acceptance of a drafted path
// (fibq_accept_draft) and eviction by accumulated attention weight
// (fibq_evict).  The payload is fixed-rate, so a row is P bytes and two norm
// bytes at an affine address, and moving it needs no decoding.
#include <hip/hip_runtime.h>

#include "device_common.h"
#include "fibq.h"
#include "fibq_internal.h"

namespace fibq {
namespace dev {
namespace sc {

// One block per group: the path's rows are read into LDS before any is
// written, so a path may name rows that it also overwrites.
__global__ __launch_bounds__(256) void accept_kernel(
    uint8_t* __restrict__ kp, uint16_t* __restrict__ kn, uint8_t* __restrict__ vp,
    uint16_t* __restrict__ vn, const int32_t* lens, int64_t T_stride, int P, int M,
    const int32_t* __restrict__ path, int A, const int32_t* __restrict__ n_acc,
    int32_t* new_lens) {
  extern __shared__ __align__(16) uint8_t rows[];  // K rows, V rows [A][P], norms [2][A]
  __shared__ int src[64];
  const int64_t g = blockIdx.x;
  const int tid = threadIdx.x;
  const int len = lens[g], n = n_acc[g];
  bool bad = len < 0 || len > T_stride - M || n < 0 || n > min(A, M);
  if (!bad && tid < n) {
    src[tid] = path[g * A + tid];
    bad = src[tid] < 0 || src[tid] >= M;
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) new_lens[g] = -1;
    return;
  }
  const int64_t at = g * T_stride + len;
  uint16_t* norms = reinterpret_cast<uint16_t*>(rows + ((2 * A * P + 15) & ~15));
  for (int i = tid; i < n * P; i += 256) {
    const int64_t from = (at + src[i / P]) * P + i % P;
    rows[i] = kp[from];
    rows[n * P + i] = vp[from];
  }
  if (tid < n) {
    norms[tid] = kn[at + src[tid]];
    norms[A + tid] = vn[at + src[tid]];
  }
  __syncthreads();
  for (int i = tid; i < n * P; i += 256) {
    kp[at * P + i] = rows[i];
    vp[at * P + i] = rows[n * P + i];
  }
  if (tid < n) {
    kn[at + tid] = norms[tid];
    vn[at + tid] = norms[A + tid];
  }
  if (tid == 0) new_lens[g] = len + n;
}

// Order of the accumulators as unsigned numbers: NaN below everything, both
// zeros equal.
__device__ __forceinline__ uint32_t key_of(float a) {
  if (a != a) return 0;
  const uint32_t u = __float_as_uint(a + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One block per group: the kept rows' indices in increasing order.  The key of
// the last kept one is found 8 bits at a time from histograms; its equals are
// taken from the lowest index on.
constexpr int kSel = 1024;
__device__ __forceinline__ int block_sum_before(int v, int* tmp, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) tmp[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < kSel / 64; ++i) {
    if (i < wave) before += tmp[i];
    all += tmp[i];
  }
  __syncthreads();
  *total = all;
  return before + x - v;
}
__global__ __launch_bounds__(kSel) void select_kernel(const float* __restrict__ acc,
                                                      const int32_t* __restrict__ lens,
                                                      int64_t T_stride, int keep, int recent,
                                                      int32_t* __restrict__ new_lens,
                                                      int32_t* __restrict__ index) {
  __shared__ int hist[256];
  __shared__ int tmp[kSel / 64];
  __shared__ uint32_t found[2];
  const int64_t g = blockIdx.x;
  const int tid = threadIdx.x;
  const int len = lens[g];
  int32_t* out = index + g * keep;
  const bool bad = len < 0 || len > T_stride;
  const int kept = bad ? 0 : min(len, keep);
  if (tid == 0) new_lens[g] = bad ? -1 : kept;
  for (int i = kept + tid; i < keep; i += kSel) out[i] = -1;
  if (bad) return;
  if (len <= keep) {
    for (int i = tid; i < len; i += kSel) out[i] = i;
    return;
  }
  const float* a = acc + g * T_stride;
  const int old = len - recent;
  int need = keep - recent;  // of the first `old`
  uint32_t top = 0;          // bits of the last kept key found so far
  for (int sh = 24; sh >= 0 && need > 0; sh -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int t = tid; t < old; t += kSel) {
      const uint32_t u = key_of(a[t]);
      if (sh == 24 || (u >> (sh + 8)) == (top >> (sh + 8))) atomicAdd(&hist[(u >> sh) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int left = need, b = 255;
      while (hist[b] < left) left -= hist[b--];
      found[0] = (uint32_t)b;
      found[1] = (uint32_t)left;
    }
    __syncthreads();
    top |= found[0] << sh;
    need = (int)found[1];
    __syncthreads();
  }
  // above the last key, or one of its first `need` equals, or recent
  const bool none = keep == recent;
  int placed = 0, equal = 0;
  for (int t0 = 0; t0 < len; t0 += kSel) {
    const int t = t0 + tid;
    const uint32_t u = t < old ? key_of(a[t]) : 0;
    const bool eq = !none && t < old && u == top;
    int n_eq, n_in;
    const int e = block_sum_before(eq, tmp, &n_eq);
    const bool in = t < len && (t >= old || (!none && (u > top || (eq && equal + e < need))));
    const int at = block_sum_before(in, tmp, &n_in);
    if (in) out[placed + at] = t;
    placed += n_in;
    equal += n_eq;
  }
}

// Copies the kept rows: thread per byte of a payload row, norm or accumulator.
__global__ __launch_bounds__(256) void gather_kernel(
    const uint8_t* __restrict__ kp, const uint16_t* __restrict__ kn,
    const uint8_t* __restrict__ vp, const uint16_t* __restrict__ vn,
    const float* __restrict__ acc, int64_t T_stride, int P, int keep,
    const int32_t* __restrict__ index, int64_t T_out, uint8_t* __restrict__ kpo,
    uint16_t* __restrict__ kno, uint8_t* __restrict__ vpo, uint16_t* __restrict__ vno,
    float* __restrict__ acco) {
  const int64_t g = blockIdx.y;
  const int i0 = blockIdx.x * 256;
  const int n = min(256, keep - i0);
  __shared__ int32_t id[256];
  if ((int)threadIdx.x < n) {
    const int32_t t = index[g * keep + i0 + threadIdx.x];
    id[threadIdx.x] = t;
    if (t >= 0) {
      const int64_t to = g * T_out + i0 + threadIdx.x, from = g * T_stride + t;
      kno[to] = kn[from];
      vno[to] = vn[from];
      acco[to] = acc[from];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n * P; i += 256) {
    const int32_t t = id[i / P];
    if (t < 0) continue;
    const int64_t to = (g * T_out + i0) * P + i, from = (g * T_stride + t) * P + i % P;
    kpo[to] = kp[from];
    vpo[to] = vp[from];
  }
}

}  // namespace sc

int launch_accept(uint8_t* kp, uint16_t* kn, uint8_t* vp, uint16_t* vn, const int32_t* lens,
                  int64_t n_groups, int64_t T_stride, int P, int M, const int32_t* path, int A,
                  const int32_t* n_acc, int32_t* new_lens, void* stream) {
  const size_t lds = ((2 * (size_t)A * P + 15) & ~(size_t)15) + 4 * (size_t)A;
  hipLaunchKernelGGL(sc::accept_kernel, dim3((unsigned)n_groups), dim3(256), lds,
                     static_cast<hipStream_t>(stream), kp, kn, vp, vn, lens, T_stride, P, M, path,
                     A, n_acc, new_lens);
  return (int)hipGetLastError();
}

size_t evict_workspace_bytes(int64_t n_groups, int64_t T_stride) { return 0; }

int launch_evict(const uint8_t* kp, const uint16_t* kn, const uint8_t* vp, const uint16_t* vn,
                 const float* acc, const int32_t* lens, int64_t n_groups, int64_t T_stride, int P,
                 int keep, int recent, int64_t T_out, uint8_t* kpo, uint16_t* kno, uint8_t* vpo,
                 uint16_t* vno, float* acco, int32_t* new_lens, int32_t* index, void* ws,
                 void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(sc::select_kernel, dim3((unsigned)n_groups), dim3(sc::kSel), 0, st, acc, lens,
                     T_stride, keep, recent, new_lens, index);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return (int)e;
  hipLaunchKernelGGL(sc::gather_kernel, dim3((unsigned)((keep + 255) / 256), (unsigned)n_groups),
                     dim3(256), 0, st, kp, kn, vp, vn, acc, T_stride, P, keep, index, T_out, kpo,
                     kno, vpo, vno, acco);
  return (int)hipGetLastError();
}

}  // namespace dev
}  // namespace fibq
