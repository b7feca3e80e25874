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
  __shared__ int read[2];  // (one reading for all threads)
  if (tid == 0) {
    read[0] = lens[g];
    read[1] = n_acc[g];
  }
  __syncthreads();
  const int len = read[0], n = read[1];
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
// zeros equal.  No accumulator has key 0 (tokens behind the last one) or kRecent
// (tokens that are kept in any case), so that the passes compare keys alone.
constexpr uint32_t kRecent = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t key_of(float a) {
  if (a != a) return 1;
  const uint32_t u = __float_as_uint(a + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Selection of the kept rows.  The key of the last kept one is found digit by
// digit (11, 11 and 10 bits) from histograms; its equals are taken from the
// lowest index on, so a row's place is the number of larger keys and of taken
// equals before it.  Up to 32768 tokens, one workgroup per group reads them once,
// keeps the keys in registers and does all of it in one launch; longer groups are
// cut into slices, a workgroup each, whose histograms meet in the workspace
// between four launches (352 groups of 32768 tokens: 88 us in registers, 188 in
// slices; 8 groups: 27 and 31; of 16384: 17 and 28).  What bounds it: the LDS
// atomics, scans and barriers of the passes, one behind the other (352 groups of 32768
// keys: 44 us, vector units 28 % busy, two workgroups per compute unit although some
// registers spill then; 51 us at one).  The bins are kept in kCopies copies by
// lane, since attention weights share few exponents (1, 4 and 8 copies: 144 groups of
// 1024 tokens 13.1, 11.0 and 12.8 us, 352 of 32768 87.8, 85.0 and 88.7).
constexpr int kSel = 1024;      // threads
constexpr int kBins = 2048;
constexpr int kCopies = 4;
constexpr int kSlice = 8192;    // tokens of a slice, at least
constexpr int kSlices = 64;     // slices of a group, at most
constexpr int kMaxKeys = 32;    // keys of a thread

struct Sel {
  const float* acc;
  const int32_t* lens;
  int64_t T_stride;
  int keep, recent;
  int32_t* new_lens;
  int32_t* index;
  int slices, slice_len;
  int32_t* hist;   // [digit][group][slice][kBins]
  int32_t* found;  // [digit][group][2]: the digits so far, the keys still needed
  int32_t* ahead;  // [group][slice]: larger keys of a slice, by the first two digits
  int n_groups;
};
__device__ __forceinline__ int digit_shift(int d) { return d == 0 ? 21 : d == 1 ? 10 : 0; }
__device__ __forceinline__ uint32_t digit_of(uint32_t u, int d) {
  return (u >> digit_shift(d)) & (d == 2 ? 1023u : 2047u);
}

// sums over the wavefront of v up to and with this lane
__device__ __forceinline__ uint32_t wave_upto(uint32_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(v, o, 64);
    if (lane >= o) v += y;
  }
  return v;
}
// exclusive sums over the block of v
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* tmp) {
  const int wave = threadIdx.x >> 6;
  const uint32_t x = wave_upto(v);
  if ((threadIdx.x & 63) == 63) tmp[wave] = x;
  __syncthreads();
  uint32_t before = 0;
#pragma unroll
  for (int i = 0; i < kSel / 64; ++i) before += i < wave ? tmp[i] : 0;
  __syncthreads();
  return before + x - v;
}

// What the passes know of the last kept key.
struct Found {
  uint32_t top;  // its digits so far, in place
  int need;      // how many keys with these digits are kept
};

__device__ __forceinline__ void clear_bins(int* bins) {
  for (int i = threadIdx.x; i < kBins * kCopies; i += kSel) bins[i] = 0;
  __syncthreads();
}
// counts key u's digit d if its higher digits are f.top's
__device__ __forceinline__ void count_key(uint32_t u, int d, const Found& f, int* bins) {
  const int sh = digit_shift(d) + (d == 2 ? 10 : 11);
  if (d == 0 || (u >> sh) == (f.top >> sh))
    atomicAdd(&bins[digit_of(u, d) * kCopies + (threadIdx.x & (kCopies - 1))], 1);
}
__device__ __forceinline__ int bin_count(const int* bins, int b) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < kCopies; ++i) n += bins[b * kCopies + i];
  return n;
}

// the digit at which the counts from the largest bin down reach f.need;
// count(bin): this bin's count
template <typename COUNT>
__device__ void find_digit(int d, COUNT count, uint32_t* tmp, int* found, Found* f) {
  const int b1 = kBins - 1 - 2 * (int)threadIdx.x, b0 = b1 - 1;  // this thread's bins
  const int c1 = count(b1), c0 = count(b0);
  const int before = (int)block_before((uint32_t)(c1 + c0), tmp);
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

// Keys of tokens t0 .. t0 + 1024 E - 1 in registers: u[4 j + i] is token
// t0 + 4096 j + 4 tid + i; from `old` on kRecent, from `end` on 0.
template <int E>
__device__ __forceinline__ void load_keys(const float* a, int t0, int old, int end, uint32_t (&u)[E]) {
#pragma unroll
  for (int j = 0; j < E / 4; ++j) {
    const int t = t0 + 4096 * j + 4 * (int)threadIdx.x;
    float v[4] = {};
    if (t + 4 <= min(old, end)) {
      __builtin_memcpy(v, a + t, 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) u[4 * j + i] = key_of(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        u[4 * j + i] = t + i >= end ? 0 : t + i >= old ? kRecent : key_of(a[t + i]);
    }
  }
}

// counts the digits of those tokens' keys, by whole 4096-token pieces before `end`
template <int E>
__device__ __forceinline__ void count_keys(const uint32_t (&u)[E], int t0, int end, int d, const Found& f, int* bins) {
#pragma unroll
  for (int j = 0; j < E / 4; ++j) {
    if (t0 + 4096 * j >= end) break;
#pragma unroll
    for (int i = 0; i < 4; ++i) count_key(u[4 * j + i], d, f, bins);
  }
}

// Places of the kept ones of those tokens, with `larger` and `equal` keys before
// t0.  sums: a number per 4096-token piece and wavefront, and (behind them) how
// many keys were larger | equal << 16 in all (at most 32768 each).
template <int E>
__device__ void emit(const uint32_t (&u)[E], int t0, const Found& f, int larger, int equal,
                     uint32_t* sums, int32_t* out, int keep) {
  constexpr int kWaves = kSel / 64, kSums = E / 4 * kWaves;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t before[E / 4];  // of a piece: larger keys | equal keys << 16
#pragma unroll
  for (int j = 0; j < E / 4; ++j) {
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      n += u[4 * j + i] > f.top ? 1u : u[4 * j + i] == f.top ? 1u << 16 : 0u;
    const uint32_t upto = wave_upto(n);
    if (lane == 63) sums[j * kWaves + wave] = upto;
    before[j] = upto - n;
  }
  __syncthreads();
  if (wave == 0) {  // exclusive sums, two per lane
    const uint32_t s0 = 2 * lane < kSums ? sums[2 * lane] : 0, s1 = 2 * lane < kSums ? sums[2 * lane + 1] : 0;
    const uint32_t upto = wave_upto(s0 + s1);
    if (2 * lane < kSums) {
      sums[2 * lane] = upto - s1 - s0;
      sums[2 * lane + 1] = upto - s1;
    }
    if (lane == 63) sums[kSums] = upto;
  }
  __syncthreads();
  uint32_t top = f.top;
  asm("" : "+v"(top));  // (else the comparisons above are kept, in spilled scalar registers)

#pragma unroll
  for (int j = 0; j < E / 4; ++j) {
    const uint32_t mine = before[j] + sums[j * kWaves + wave];
    int g = larger + (int)(mine & 0xFFFFu), e = equal + (int)(mine >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool gt = u[4 * j + i] > top, eq = u[4 * j + i] == top;
      // (the bound holds by the counts; it is checked, since sliced passes read
      // lengths and accumulators that another stream might be writing.  Places may
      // then stay unwritten, so that gather_kernel checks what it reads there.)
      const int at = g + min(e, f.need);
      if ((gt || (eq && e < f.need)) && (uint32_t)at < (uint32_t)keep)
        out[at] = t0 + 4096 * j + 4 * (int)threadIdx.x + i;
      g += gt;
      e += eq;
    }
  }
}

template <int E>
__global__ __launch_bounds__(kSel, 8) void select_kernel(const Sel p) {
  __shared__ int bins[kBins * kCopies];
  __shared__ uint32_t sums[E / 4 * (kSel / 64) + 1];
  __shared__ int found[2];
  __shared__ int read;  // (one reading for all threads)
  const int g = blockIdx.x;
  if (threadIdx.x == 0) read = p.lens[g];
  __syncthreads();
  const int len = __builtin_amdgcn_readfirstlane(read);
  int32_t* out = p.index + (int64_t)g * p.keep;
  if (whole_group(p, g, len, out, true)) return;
  Found f{0, p.keep};
  uint32_t u[E];
  load_keys<E>(p.acc + g * p.T_stride, 0, len - p.recent, len, u);
#pragma unroll 1
  for (int d = 0; d < 3; ++d) {
    clear_bins(bins);
    count_keys<E>(u, 0, len, d, f, bins);
    __syncthreads();
    find_digit(d, [&](int b) { return bin_count(bins, b); }, sums, found, &f);
  }
  emit<E>(u, 0, f, 0, 0, sums, out, p.keep);
}

// Sliced: pass d < 3 counts digit d of a slice, pass 3 writes the places; a pass
// first finds the digit that the pass before counted.
__global__ __launch_bounds__(kSel) void slice_kernel(const Sel p, int pass) {
  __shared__ int bins[kBins * kCopies];
  __shared__ uint32_t sums[kSel / 64 + 1];
  __shared__ int found[2];
  __shared__ int total[2];
  __shared__ int read;  // (one reading for all threads)
  const int g = blockIdx.x / p.slices, s = blockIdx.x % p.slices, tid = threadIdx.x;
  if (tid == 0) read = p.lens[g];
  if (tid < 2) found[tid] = 0;
  __syncthreads();
  const int len = __builtin_amdgcn_readfirstlane(read);
  int32_t* out = p.index + (int64_t)g * p.keep;
  if (whole_group(p, g, len, out, pass == 0 && s == 0)) return;
  const float* a = p.acc + g * p.T_stride;
  const int old = len - p.recent;
  Found f{0, p.keep};
  auto counts = [&](int d, int slice) {
    return p.hist + (((int64_t)d * p.n_groups + g) * p.slices + slice) * kBins;
  };
  auto state = [&](int d) { return p.found + ((int64_t)d * p.n_groups + g) * 2; };
  if (tid < 2) total[tid] = 0;
  if (pass > 0) {
    const int d = pass - 1;
    if (d > 0) f = Found{(uint32_t)state(d - 1)[0], state(d - 1)[1]};
    find_digit(d, [&](int b) {
      int n = 0;
#pragma unroll 8
      for (int i = 0; i < p.slices; ++i) n += counts(d, i)[b];
      return n;
    }, sums, found, &f);
    if (d < 2) {
      // every slice's workgroup finds the same; slice 0's hands it on
      if (s == 0 && tid == 0) {
        state(d)[0] = (int32_t)f.top;
        state(d)[1] = f.need;
      }
      int n = 0;  // this slice's keys above the digit
      for (int b = tid; b < kBins; b += kSel)
        if (b > (int)digit_of(f.top, d)) n += counts(d, s)[b];
      if (n) atomicAdd(&total[0], n);
      __syncthreads();
      if (tid == 0) {
        int32_t* at = p.ahead + (int64_t)g * p.slices + s;
        *at = total[0] + (d > 0 ? *at : 0);
      }
    }
  }
  const int from = (int)min((int64_t)s * p.slice_len, (int64_t)len);
  const int to = (int)min((int64_t)(s + 1) * p.slice_len, (int64_t)len);
  if (pass < 3) {
    clear_bins(bins);
    for (int t0 = from; t0 < to; t0 += 8 * kSel) {
      uint32_t u[8];
      load_keys<8>(a, t0, old, to, u);
      count_keys<8>(u, t0, to, pass, f, bins);
    }
    __syncthreads();
    for (int b = tid; b < kBins; b += kSel) counts(pass, s)[b] = bin_count(bins, b);
    return;
  }
  // larger and equal keys of the slices before this one
  const int b2 = (int)digit_of(f.top, 2);
  int ahead = 0;
  for (int i = tid; i < s * 1024; i += kSel)
    if ((i & 1023) > b2) ahead += counts(2, i >> 10)[i & 1023];
  if (tid < s) {
    ahead += p.ahead[(int64_t)g * p.slices + tid];
    atomicAdd(&total[1], counts(2, tid)[b2]);
  }
  if (ahead) atomicAdd(&total[0], ahead);
  __syncthreads();
  int larger = total[0], equal = total[1];
  for (int t0 = from; t0 < to; t0 += 4 * kSel) {
    uint32_t u[4];
    load_keys<4>(a, t0, old, to, u);
    emit<4>(u, t0, f, larger, equal, sums, out, p.keep);
    const uint32_t all = sums[kSel / 64];  // what this piece held
    larger += (int)(all & 0xFFFFu);
    equal += (int)(all >> 16);
    __syncthreads();
  }
}

// Copies the kept rows, V bytes of a payload row at a time (the largest that
// divides P and that all addresses are aligned to: at P = 48, 262144 rows, 12 us
// against 26 with single bytes).  What bounds it is the lines that it touches: at
// P = 4 a quarter of the rows is kept and nearly every 128-byte line holds one (2.9 M
// of 11.5 M rows: 36 us, 248 MB, whatever the width).  An index outside the old cache
// copies nothing.
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
    int32_t t = index[g * keep + i0 + tid];
    if (t >= T_stride) t = -1;
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

// One launch up to kMaxKeys keys per thread; slices beyond.
static int slices_of(int64_t T_stride) {
  if (T_stride <= (int64_t)sc::kSel * sc::kMaxKeys) return 1;
  const int64_t s = (T_stride + sc::kSlice - 1) / sc::kSlice;
  return (int)(s < sc::kSlices ? s : sc::kSlices);
}

size_t evict_workspace_bytes(int64_t n_groups, int64_t T_stride) {
  const int s = slices_of(T_stride);
  return s == 1 ? 0 : (size_t)n_groups * ((size_t)3 * s * sc::kBins + 6 + s) * 4;
}

int launch_evict(const uint8_t* kp, const uint16_t* kn, const uint8_t* vp, const uint16_t* vn,
                 const float* acc, const int32_t* lens, int64_t n_groups, int64_t T_stride, int P,
                 int keep, int recent, int64_t T_out, uint8_t* kpo, uint16_t* kno, uint8_t* vpo,
                 uint16_t* vno, float* acco, int32_t* new_lens, int32_t* index, void* ws,
                 void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int slices = slices_of(T_stride);
  // (whole pieces of load_keys, so that slices start at even places of them)
  const int slice_len = (int)(((T_stride + slices - 1) / slices + 4095) / 4096 * 4096);
  int32_t* hist = static_cast<int32_t*>(ws);
  const int64_t n_hist = (int64_t)3 * n_groups * slices * sc::kBins;
  const sc::Sel p{acc, lens, T_stride, keep, recent, new_lens, index, slices, slice_len, hist,
                  hist + n_hist, hist + n_hist + 6 * n_groups, (int)n_groups};
  hipError_t e = hipSuccess;
  if (slices == 1) {
    auto kern = T_stride <= 4 * sc::kSel    ? sc::select_kernel<4>
                : T_stride <= 8 * sc::kSel  ? sc::select_kernel<8>
                : T_stride <= 16 * sc::kSel ? sc::select_kernel<16>
                                            : sc::select_kernel<sc::kMaxKeys>;
    hipLaunchKernelGGL(kern, dim3((unsigned)n_groups), dim3(sc::kSel), 0, st, p);
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
