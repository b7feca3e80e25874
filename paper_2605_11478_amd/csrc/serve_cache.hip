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

// Selection of the kept rows.  The key of the last kept one is found digit by
// digit (11, 11 and 10 bits) from histograms; its equals are taken from the
// lowest index on, so a row's place is the number of larger keys and of taken
// equals before it.  One workgroup per group does all of it in one launch; few
// long groups are cut into slices, a workgroup each, whose histograms meet in
// the workspace between launches.  What bounds it: the LDS atomics of the
// histograms (attention weights share few exponents, so a digit's bins are kept
// in kCopies copies by lane) and the scans of the last pass; the accumulators
// are read four times, three of them from L2.
constexpr int kSel = 1024;      // threads
constexpr int kBins = 2048;
constexpr int kCopies = 4;
constexpr int kEach = 8;        // consecutive tokens of a thread in the last pass
constexpr int kSlice = 16384;   // tokens of a slice, at least
constexpr int kSlices = 64;     // slices of a group, at most

struct Sel {
  const float* acc;
  const int32_t* lens;
  int64_t T_stride;
  int keep, recent;
  int32_t* new_lens;
  int32_t* index;
  int slices, slice_len;  // (one launch: 1 and T_stride)
  int32_t* hist;          // [digit][group][slice][kBins]
  int n_groups;
};
__device__ __forceinline__ int digit_shift(int d) { return d == 0 ? 21 : d == 1 ? 10 : 0; }
__device__ __forceinline__ uint32_t digit_of(uint32_t u, int d) {
  return (u >> digit_shift(d)) & (d == 2 ? 1023u : 2047u);
}

// exclusive sums over the block of v; *total the whole sum
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* tmp, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) tmp[wave] = x;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kSel / 64; ++i) {
    const uint32_t y = tmp[i];
    before += i < wave ? y : 0;
    all += y;
  }
  __syncthreads();
  *total = all;
  return before + x - v;
}

// What the passes know of the last kept key.
struct Found {
  uint32_t top;  // its digits so far, in place
  int need;      // how many keys with these digits are kept
};

// counts of digit d over tokens [t0, t1) whose higher digits are f.top's, into
// bins [kBins][kCopies] of LDS
__device__ void count_digit(const float* a, int t0, int t1, int d, const Found& f, int* bins) {
  for (int i = threadIdx.x; i < kBins * kCopies; i += kSel) bins[i] = 0;
  __syncthreads();
  const int sh = digit_shift(d) + (d == 2 ? 10 : 11);
  auto add = [&](float v) {
    const uint32_t u = key_of(v);
    if (d == 0 || (u >> sh) == (f.top >> sh))
      atomicAdd(&bins[digit_of(u, d) * kCopies + (threadIdx.x & (kCopies - 1))], 1);
  };
  int t = t0 + threadIdx.x;
  for (; t + 3 * kSel < t1; t += 4 * kSel) {  // four loads at once
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[t + i * kSel];
#pragma unroll
    for (int i = 0; i < 4; ++i) add(v[i]);
  }
  for (; t < t1; t += kSel) add(a[t]);
  __syncthreads();
}

// the digit at which the counts from the largest bin down reach f.need;
// count(bin): this bin's count
template <typename COUNT>
__device__ void find_digit(int d, COUNT count, uint32_t* tmp, int* found, Found* f) {
  const int b1 = kBins - 1 - 2 * (int)threadIdx.x, b0 = b1 - 1;  // this thread's bins
  const int c1 = count(b1), c0 = count(b0);
  uint32_t all;
  const int before = (int)block_before((uint32_t)(c1 + c0), tmp, &all);
  if (before < f->need && f->need <= before + c1 + c0) {
    const bool upper = f->need <= before + c1;
    found[0] = upper ? b1 : b0;
    found[1] = f->need - before - (upper ? 0 : c1);
  }
  __syncthreads();
  f->top |= (uint32_t)found[0] << digit_shift(d);
  f->need = found[1];
  __syncthreads();
}

// places of the kept tokens of [t0, t1): `larger` and `equal` keys before t0
__device__ void emit(const float* a, int t0, int t1, int old, bool any, const Found& f, int larger,
                     int equal, uint32_t* tmp, int32_t* out) {
  for (int c0 = t0; c0 < t1; c0 += kSel * kEach) {
    const int t = c0 + threadIdx.x * kEach;
    uint32_t gt = 0, eq = 0;  // bit i: token t + i
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const bool is_old = any && t + i < old;
      const uint32_t u = is_old && t + i < t1 ? key_of(a[t + i]) : 0;
      const bool in = t + i < t1;
      if (in && (t + i >= old || (is_old && u > f.top))) gt |= 1u << i;
      if (in && is_old && u == f.top) eq |= 1u << i;
    }
    uint32_t all;  // (at most kSel kEach = 2^13 of each)
    const uint32_t before = block_before(__popc(gt) | (uint32_t)__popc(eq) << 16, tmp, &all);
    int g = larger + (int)(before & 0xFFFFu), e = equal + (int)(before >> 16);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const bool is_gt = gt >> i & 1, is_eq = eq >> i & 1;
      if (is_gt || (is_eq && e < f.need)) out[g + min(e, f.need)] = t + i;
      g += is_gt;
      e += is_eq;
    }
    larger += (int)(all & 0xFFFFu);
    equal += (int)(all >> 16);
  }
}

// The simple outcomes: a bad length, or everything kept.  True if done.
__device__ bool whole_group(const Sel& p, int g, int len, int32_t* out, bool first) {
  const bool bad = len < 0 || len > p.T_stride;
  const int kept = bad ? 0 : min(len, p.keep);
  if (first) {
    if (threadIdx.x == 0) p.new_lens[g] = bad ? -1 : kept;
    for (int i = kept + threadIdx.x; i < p.keep; i += kSel) out[i] = -1;
    if (!bad && len <= p.keep)
      for (int i = threadIdx.x; i < len; i += kSel) out[i] = i;
  }
  return bad || len <= p.keep;
}

__global__ __launch_bounds__(kSel) void select_kernel(const Sel p) {
  __shared__ int bins[kBins * kCopies];
  __shared__ uint32_t tmp[kSel / 64];
  __shared__ int found[2];
  const int g = blockIdx.x, len = p.lens[g];
  int32_t* out = p.index + (int64_t)g * p.keep;
  if (whole_group(p, g, len, out, true)) return;
  const float* a = p.acc + g * p.T_stride;
  const int old = len - p.recent;
  const bool any = p.keep > p.recent;  // some of the first `old` are kept
  Found f{0, p.keep - p.recent};
  if (any) {
#pragma unroll 1
    for (int d = 0; d < 3; ++d) {
      count_digit(a, 0, old, d, f, bins);
      find_digit(d, [&](int b) {
        int n = 0;
        for (int i = 0; i < kCopies; ++i) n += bins[b * kCopies + i];
        return n;
      }, tmp, found, &f);
    }
  }
  emit(a, 0, len, old, any, f, 0, 0, tmp, out);
}

// Sliced: pass d < 3 counts digit d of a slice, pass 3 writes the places.  Every
// pass finds the digits before it again from all slices' counts.
__global__ __launch_bounds__(kSel) void slice_kernel(const Sel p, int pass) {
  __shared__ int bins[kBins * kCopies];
  __shared__ uint32_t tmp[kSel / 64];
  __shared__ int found[2];
  __shared__ int sums[2];
  const int g = blockIdx.x / p.slices, s = blockIdx.x % p.slices, len = p.lens[g];
  int32_t* out = p.index + (int64_t)g * p.keep;
  if (whole_group(p, g, len, out, pass == 0 && s == 0)) return;
  const float* a = p.acc + g * p.T_stride;
  const int old = len - p.recent;
  const bool any = p.keep > p.recent;
  Found f{0, p.keep - p.recent};
  auto counts = [&](int d) { return p.hist + ((int64_t)(d * p.n_groups + g) * p.slices) * kBins; };
  if (any) {
    for (int d = 0; d < pass && d < 3; ++d) {
      const int32_t* h = counts(d);
      find_digit(d, [&](int b) {
        int n = 0;
        for (int i = 0; i < p.slices; ++i) n += h[(int64_t)i * kBins + b];
        return n;
      }, tmp, found, &f);
    }
  }
  const int64_t from = (int64_t)s * p.slice_len, to = from + p.slice_len;
  if (pass < 3) {
    if (!any) return;
    count_digit(a, (int)min(from, (int64_t)old), (int)min(to, (int64_t)old), pass, f, bins);
    int32_t* h = p.hist + ((int64_t)(pass * p.n_groups + g) * p.slices + s) * kBins;
    for (int b = threadIdx.x; b < kBins; b += kSel) {
      int n = 0;
      for (int i = 0; i < kCopies; ++i) n += bins[b * kCopies + i];
      h[b] = n;
    }
    return;
  }
  // larger and equal keys of the slices before this one
  if (threadIdx.x < 2) sums[threadIdx.x] = 0;
  __syncthreads();
  if (any) {
    int larger = 0;
    for (int d = 0; d < 3; ++d) {
      const int32_t* h = counts(d);
      const int b0 = (int)digit_of(f.top, d);
      for (int i = threadIdx.x; i < s * kBins; i += kSel)
        if (i % kBins > b0) larger += h[i];
    }
    if (larger) atomicAdd(&sums[0], larger);
    if ((int)threadIdx.x < s) atomicAdd(&sums[1], counts(2)[(int64_t)threadIdx.x * kBins + digit_of(f.top, 2)]);
  }
  __syncthreads();
  // (recent tokens of earlier slices count as larger)
  const int larger = sums[0] + (int)max((int64_t)0, min(from, (int64_t)len) - old);
  emit(a, (int)min(from, (int64_t)len), (int)min(to, (int64_t)len), old, any, f, larger, sums[1], tmp, out);
}

// Copies the kept rows, V bytes of a payload row at a time (the largest that
// divides P and that all addresses are aligned to): P = 4 with single bytes took
// 35 us for 2.9 M rows, whose bytes take 18 at the rate of a large copy.
template <typename V>
__global__ __launch_bounds__(256) void gather_kernel(
    const uint8_t* __restrict__ kp, const uint16_t* __restrict__ kn,
    const uint8_t* __restrict__ vp, const uint16_t* __restrict__ vn,
    const float* __restrict__ acc, int64_t T_stride, int P, int keep, int blocks,
    const int32_t* __restrict__ index, int64_t T_out, uint8_t* __restrict__ kpo,
    uint16_t* __restrict__ kno, uint8_t* __restrict__ vpo, uint16_t* __restrict__ vno,
    float* __restrict__ acco) {
  const int64_t g = blockIdx.x / blocks;
  const int i0 = (int)(blockIdx.x % blocks) * 256;
  const int n = min(256, keep - i0), tid = threadIdx.x;
  __shared__ int32_t id[256];
  if (tid < n) {
    const int32_t t = index[g * keep + i0 + tid];
    id[tid] = t;
    if (t >= 0) {
      const int64_t to = g * T_out + i0 + tid, from = g * T_stride + t;
      kno[to] = kn[from];
      vno[to] = vn[from];
      acco[to] = acc[from];
    }
  }
  __syncthreads();
  const uint32_t per = (uint32_t)P / sizeof(V);
  const V* ki = reinterpret_cast<const V*>(kp) + g * T_stride * per;
  const V* vi = reinterpret_cast<const V*>(vp) + g * T_stride * per;
  V* ko = reinterpret_cast<V*>(kpo) + (g * T_out + i0) * per;
  V* vo = reinterpret_cast<V*>(vpo) + (g * T_out + i0) * per;
  for (uint32_t i = tid; i < n * per; i += 256) {
    const uint32_t r = i / per;
    const int32_t t = id[r];
    if (t < 0) continue;
    const int64_t from = (int64_t)t * per + (i - r * per);
    const V x = ki[from], y = vi[from];
    ko[i] = x;
    vo[i] = y;
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

// Slices pay when the groups alone leave the chip idle and a group's passes are
// longer than the launches that slicing adds: TODO
static int slices_of(int64_t n_groups, int64_t T_stride) {
  if (T_stride <= 2 * sc::kSlice || n_groups > 128) return 1;
  const int64_t s = (T_stride + sc::kSlice - 1) / sc::kSlice;
  return (int)(s < sc::kSlices ? s : sc::kSlices);
}

size_t evict_workspace_bytes(int64_t n_groups, int64_t T_stride) {
  const int s = slices_of(n_groups, T_stride);
  return s == 1 ? 0 : (size_t)3 * n_groups * s * sc::kBins * 4;
}

int launch_evict(const uint8_t* kp, const uint16_t* kn, const uint8_t* vp, const uint16_t* vn,
                 const float* acc, const int32_t* lens, int64_t n_groups, int64_t T_stride, int P,
                 int keep, int recent, int64_t T_out, uint8_t* kpo, uint16_t* kno, uint8_t* vpo,
                 uint16_t* vno, float* acco, int32_t* new_lens, int32_t* index, void* ws,
                 void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int slices = slices_of(n_groups, T_stride);
  const sc::Sel p{acc, lens, T_stride, keep, recent, new_lens, index, slices,
                  (int)((T_stride + slices - 1) / slices), static_cast<int32_t*>(ws), (int)n_groups};
  hipError_t e = hipSuccess;
  if (slices == 1) {
    hipLaunchKernelGGL(sc::select_kernel, dim3((unsigned)n_groups), dim3(sc::kSel), 0, st, p);
    if ((e = hipGetLastError()) != hipSuccess) return (int)e;
  } else {
    for (int pass = 0; pass < 4; ++pass) {
      hipLaunchKernelGGL(sc::slice_kernel, dim3((unsigned)(n_groups * slices)), dim3(sc::kSel), 0,
                         st, p, pass);
      if ((e = hipGetLastError()) != hipSuccess) return (int)e;
    }
  }
  const int blocks = (keep + 255) / 256;
  const uintptr_t at = reinterpret_cast<uintptr_t>(kp) | reinterpret_cast<uintptr_t>(vp) |
                       reinterpret_cast<uintptr_t>(kpo) | reinterpret_cast<uintptr_t>(vpo) | (uintptr_t)P;
#define FIBQ_GATHER(V)                                                                            \
  hipLaunchKernelGGL(sc::gather_kernel<V>, dim3((unsigned)(n_groups * blocks)), dim3(256), 0, st, \
                     kp, kn, vp, vn, acc, T_stride, P, keep, blocks, index, T_out, kpo, kno, vpo, \
                     vno, acco)
  if (at % 16 == 0) FIBQ_GATHER(uint4);
  else if (at % 4 == 0) FIBQ_GATHER(uint32_t);
  else if (at % 2 == 0) FIBQ_GATHER(uint16_t);
  else FIBQ_GATHER(uint8_t);
#undef FIBQ_GATHER
  return (int)hipGetLastError();
}

}  // namespace dev
}  // namespace fibq
