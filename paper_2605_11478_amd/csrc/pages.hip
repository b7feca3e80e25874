// The paged 8-bit cache apart from its attention: rotary positions of queries
// and keys (fibq_rope), block tables and slot maps (fibq_page_resize) and the
// write of keys and values (fibq_cache8_write).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.h"
#include "fibq.h"
#include "fibq_internal.h"

namespace fibq {
namespace dev {
namespace pg {

__device__ __forceinline__ float from(float v) { return v; }
__device__ __forceinline__ float from(_Float16 v) { return (float)v; }
__device__ __forceinline__ float from(__bf16 v) { return (float)v; }

// V elements of a row that begins at any element: one wide access
template <typename T, int V>
struct Vec {
  T e[V];
};
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load(const T* p) {
  Vec<T, V> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
template <typename T, int V>
__device__ __forceinline__ void store(T* p, const Vec<T, V>& v) {
  __builtin_memcpy(p, &v, sizeof(v));
}

// ------------------------------------------------------------------- rope --
// Pair i of a row at position p turns by p f_i.  The angle is reduced in
// double (p f_i / 2 pi to quarter turns, exact from there on), so that a far
// position loses nothing; sine and cosine of the remaining eighth of a turn are
// computed in float.  A workgroup computes the angles of its rows once, into
// LDS, and applies them to all their heads.
constexpr int kRopeThreads = 256;
constexpr int kRopeAngles = 1024;  // angles of a workgroup, at most

template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(Rope a, int tile) {
  __shared__ float2 turn[kRopeAngles];
  const int tid = threadIdx.x, half = a.rot / 2;
  const int64_t row0 = (int64_t)blockIdx.x * tile;
  const int rows = (int)min((int64_t)tile, a.n_rows - row0);
  for (int i = tid; i < rows * half; i += kRopeThreads) {
    const int r = i / half;
    const double quarters =
        (double)a.positions[row0 + r] * (a.freqs[i - r * half] * 0.63661977236758134308);
    const double n = rint(quarters);
    float s, c;
    sincospif((float)(quarters - n) * 0.5f, &s, &c);
    const int turns = (int)(n - 4.0 * floor(n * 0.25));
    float cs = turns & 1 ? -s : c, sn = turns & 1 ? c : s;
    if (turns & 2) cs = -cs, sn = -sn;
    turn[i] = make_float2(cs * a.scale, (a.inverse ? -sn : sn) * a.scale);
  }
  __syncthreads();
  const int heads = a.q_heads + a.k_heads;
  const int turned = HALF ? half / V : a.rot / V;
  const int per_head = turned + (a.d - a.rot) / V;  // (rows are copied behind the turned part)
  const int items = rows * heads * per_head;
  for (int i = tid; i < items; i += kRopeThreads) {
    const int h = i / per_head, c = i - h * per_head;
    const int r = h / heads, head = h - r * heads;
    const bool is_k = head >= a.q_heads;
    const int64_t row = row0 + r;
    const T* x = is_k ? (const T*)a.k + row * a.k_row + (head - a.q_heads) * a.k_head
                      : (const T*)a.q + row * a.q_row + head * a.q_head;
    T* y = is_k ? (T*)a.k_out + row * a.ko_row + (head - a.q_heads) * a.ko_head
                : (T*)a.q_out + row * a.qo_row + head * a.qo_head;
    const float2* t = turn + r * half;
    if (c >= turned) {
      const int at = a.rot + (c - turned) * V;
      store<T, V>(y + at, load<T, V>(x + at));
    } else if (HALF) {
      const int at = c * V;
      const Vec<T, V> x0 = load<T, V>(x + at), x1 = load<T, V>(x + at + half);
      Vec<T, V> y0, y1;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float2 w = t[at + e];
        const float u = from(x0.e[e]), v = from(x1.e[e]);
        y0.e[e] = (T)(u * w.x - v * w.y);
        y1.e[e] = (T)(v * w.x + u * w.y);
      }
      store<T, V>(y + at, y0);
      store<T, V>(y + at + half, y1);
    } else {
      const int at = c * V;
      const Vec<T, V> x0 = load<T, V>(x + at);
      Vec<T, V> y0;
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const float2 w = t[(at + e) / 2];
        const float u = from(x0.e[e]), v = from(x0.e[e + 1]);
        y0.e[e] = (T)(u * w.x - v * w.y);
        y0.e[e + 1] = (T)(v * w.x + u * w.y);
      }
      store<T, V>(y + at, y0);
    }
  }
}

template <typename T, int V>
int rope_typed(const Rope& a, hipStream_t st) {
  // rows of a workgroup: as many as its angles fit, but workgroups for every compute unit
  const int half = a.rot / 2;
  int tile = std::min<int64_t>(std::max(1, kRopeAngles / half), std::max<int64_t>(1, a.n_rows / 1024));
  tile = std::min(tile, 16);
  const int64_t grid = (a.n_rows + tile - 1) / tile;
  if (a.layout == FIBQ_ROPE_HALF) {
    if (half % V == 0 && a.d % V == 0)
      rope_kernel<T, V, true><<<grid, kRopeThreads, 0, st>>>(a, tile);
    else
      rope_kernel<T, 1, true><<<grid, kRopeThreads, 0, st>>>(a, tile);
  } else {
    if (a.rot % V == 0 && a.d % V == 0)
      rope_kernel<T, V, false><<<grid, kRopeThreads, 0, st>>>(a, tile);
    else
      rope_kernel<T, 2, false><<<grid, kRopeThreads, 0, st>>>(a, tile);
  }
  return (int)hipGetLastError();
}

// ------------------------------------------------------------ page_resize --
// Three prefix sums over the requests: rows, pages given back, pages taken.
// One workgroup runs them; the places of the pages given back come first,
// since what it may hand out depends on their number.
constexpr int kScan = 1024;

struct Sums {
  int64_t v;  // inclusive prefix of this thread's value
  int64_t total;
};
__device__ __forceinline__ Sums scan(int64_t v, int64_t* wave_sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();  // (the sums of the call before have been read)
  if (lane == 63) wave_sums[wave] = x;
  __syncthreads();
  int64_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kScan / 64; ++w) {
    const int64_t s = wave_sums[w];
    before += w < wave ? s : 0;
    total += s;
  }
  return {x + before, total};
}
__device__ __forceinline__ int64_t pages_of(int64_t tokens, int page) {
  return (tokens + page - 1) / page;
}

struct Request {
  int64_t len, after, rows;
  bool good;
};
// request g; `ends`: the rows of all requests up to and with it
__device__ __forceinline__ Request request(const Resize& a, int64_t g, int64_t len, int64_t grow,
                                           int64_t ends) {
  const int64_t room = a.max_pages * a.page;
  Request r{len, len + grow, grow > 0 ? grow : 0, false};
  r.good = len >= 0 && len <= room && r.after >= 0 && r.after <= room && ends <= a.n_rows;
  return r;
}

// A row's slot and position.  starts, new_lens and top are the scan's.
__device__ __forceinline__ void place_row(const Resize& a, int64_t r, const int32_t* starts) {
  int64_t slot = -1;
  int32_t position = -1;
  int lo = 0, hi = (int)a.n;  // the first request whose rows end behind r
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (starts[mid + 1] > r)
      hi = mid;
    else
      lo = mid + 1;
  }
  if (lo < a.n) {
    const int64_t after = a.new_lens[lo];
    if (after >= 0) {
      const int64_t rows = starts[lo + 1] - starts[lo], at = after - (starts[lo + 1] - r);
      const int64_t have = pages_of(after - rows, a.page), p = at / a.page;
      int32_t* cell = a.table + (int64_t)lo * a.max_pages + p;
      int32_t id;
      if (p < have) {
        id = *cell;
      } else {
        id = a.free_pages[a.top[lo] - (p - have)];
        if (at % a.page == 0) *cell = id;
      }
      if (id >= 0 && id < a.n_pages) slot = (int64_t)id * a.page + at % a.page;
      position = (int32_t)at;
    }
  }
  a.slots[r] = slot;
  a.positions[r] = position;
}

__global__ __launch_bounds__(kScan) void resize_kernel(Resize a, int place) {
  __shared__ int64_t wave_sums[kScan / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t cap = a.free_cap;
  const int64_t free0 = min(max((int64_t)*a.n_free, (int64_t)0), cap);
  // pages given back, onto the stack in order
  int64_t rows0 = 0, back0 = 0;
  for (int64_t g0 = 0; g0 < a.n; g0 += kScan) {
    const int64_t g = g0 + tid;
    const bool live = g < a.n;
    const int64_t len = live ? a.lens[g] : 0, grow = live ? a.grow[g] : 0;
    const Sums rows = scan(grow > 0 ? grow : 0, wave_sums);
    const Request r = request(a, g, len, grow, rows0 + rows.v);
    const int64_t want = r.good ? pages_of(r.after, a.page) : 0;
    const int64_t back = r.good ? max(pages_of(r.len, a.page) - want, (int64_t)0) : 0;
    const Sums backs = scan(back, wave_sums);
    const int64_t to = free0 + back0 + backs.v - back;
    for (uint64_t todo = __ballot(back > 0); todo; todo &= todo - 1) {
      const int l = __ffsll((unsigned long long)todo) - 1;  // a lane's pages, by all lanes
      const int64_t n = __shfl(back, l, 64), at = __shfl(to, l, 64);
      const int32_t* from = a.table + (g0 + (tid & ~63) + l) * a.max_pages + __shfl(want, l, 64);
      for (int64_t i = lane; i < n && at + i < cap; i += 64) a.free_pages[at + i] = from[i];
    }
    rows0 += rows.total;
    back0 += backs.total;
  }
  const int64_t free1 = min(free0 + back0, cap);
  // pages taken from its top, first come, first served
  int64_t need0 = 0, taken = 0;
  rows0 = 0;
  for (int64_t g0 = 0; g0 < a.n; g0 += kScan) {
    const int64_t g = g0 + tid;
    const bool live = g < a.n;
    const int64_t len = live ? a.lens[g] : 0, grow = live ? a.grow[g] : 0;
    const Sums rows = scan(grow > 0 ? grow : 0, wave_sums);
    const Request r = request(a, g, len, grow, rows0 + rows.v);
    const int64_t need =
        r.good ? max(pages_of(r.after, a.page) - pages_of(r.len, a.page), (int64_t)0) : 0;
    const Sums needs = scan(need, wave_sums);
    const int64_t upto = need0 + needs.v;
    const bool granted = r.good && (need == 0 || upto <= free1);
    if (granted && need > 0) taken = upto;
    if (live) {
      a.new_lens[g] = granted ? (int32_t)r.after : -1;
      a.starts[g + 1] = (int32_t)min(rows0 + rows.v, a.n_rows);
      a.top[g] = granted ? (int32_t)(free1 - 1 - (upto - need)) : 0;
    }
    rows0 += rows.total;
    need0 += needs.total;
  }
  // (granted requests that need pages are the first of those that do)
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) taken = max(taken, __shfl_xor(taken, o, 64));
  __syncthreads();
  if (lane == 0) wave_sums[tid >> 6] = taken;
  __syncthreads();
  if (tid == 0) {
    for (int w = 0; w < kScan / 64; ++w) taken = max(taken, wave_sums[w]);
    a.starts[0] = 0;
    *a.new_free = (int32_t)(free1 - taken);
  }
  if (!place) return;
  __threadfence_block();
  __syncthreads();
  for (int64_t r = tid; r < a.n_rows; r += kScan) place_row(a, r, a.starts);
}

__global__ __launch_bounds__(256) void place_kernel(Resize a) {
  const int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (r < a.n_rows) place_row(a, r, a.starts);
}

// ----------------------------------------------------------- cache8_write --
// One workgroup takes the runs of rows that begin among its `chunk` rows, for
// one head of K or of V.  A run is consecutive rows of one page at increasing
// slots.  Its largest magnitude gives the least power of two that takes it to
// the codes' range; a page keeps the larger of that and of its scale so far,
// and where that grows, the codes before the run are rounded again.  With
// powers of two x / s and code * s_old / s are exact, so each value is rounded
// once per growth of its page's scale.
__device__ __forceinline__ float least_scale(uint32_t amax_bits, int codes) {
  if (amax_bits == 0) return 0.0f;
  if (amax_bits >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  int e;
  const float m = frexpf(__uint_as_float(amax_bits), &e);  // m in [1/2, 1)
  e -= codes == FIBQ_INT8 ? 7 : 9;                         // 127 = 0.9921875 2^7, 448 = 0.875 2^9
  if (m > (codes == FIBQ_INT8 ? 0.9921875f : 0.875f)) ++e;
  return ldexpf(1.0f, max(e, -126));
}

struct Quotient {  // x / s, by the exact reciprocal where s is a power of two
  float s, r;
  bool exact;
  __device__ __forceinline__ explicit Quotient(float s_) : s(s_) {
    const uint32_t u = __float_as_uint(s_);
    exact = (u & 0x807fffffu) == 0 && u >= 0x00800000u && u < 0x7f000000u;
    r = exact ? 1.0f / s_ : 0.0f;
  }
  __device__ __forceinline__ float operator()(float x) const { return exact ? x * r : x / s; }
};
__device__ __forceinline__ uint32_t code4(const float* x, int codes) {
  uint32_t w = 0;
  if (codes == FIBQ_INT8) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w |= ((uint32_t)(int)fminf(fmaxf(rintf(x[e]), -127.0f), 127.0f) & 255u) << (8 * e);
  } else {
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
  }
  return w;
}
__device__ __forceinline__ void value4(uint32_t w, int codes, float* x) {
  if (codes == FIBQ_INT8) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (float)(int8_t)(w >> (8 * e));
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
  }
}

__device__ __forceinline__ bool joins(const Write& a, int64_t before, int64_t s) {
  return before >= 0 && s > before && s / a.page == before / a.page;
}

template <typename T>
__global__ __launch_bounds__(256) void write_kernel(Write a, int chunk) {
  constexpr int V = 8;
  __shared__ uint32_t wave_max[4];
  const int tid = threadIdx.x, lane = tid & 63, n_threads = blockDim.x;
  const int h = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  const T* x = is_v ? (const T*)a.v + h * a.v_head : (const T*)a.k + h * a.k_head;
  const int64_t x_row = is_v ? a.v_row : a.k_row;
  uint8_t* pages = (uint8_t*)(is_v ? a.v_pages : a.k_pages);
  float* scales = is_v ? a.v_scales : a.k_scales;
  const int64_t base = (int64_t)blockIdx.x * chunk, limit = a.n_pages * a.page;
  auto slot = [&](int64_t r) -> int64_t {
    if (r < 0 || r >= a.n_rows) return -1;
    const int64_t s = a.slots[r];
    return s >= 0 && s < limit ? s : -1;
  };
  const int64_t mine = lane < chunk ? slot(base + lane) : -1;
  const bool begins = mine >= 0 && !joins(a, slot(base + lane - 1), mine);
  const int per_row = a.d / V;
  for (uint64_t todo = __ballot(begins); todo; todo &= todo - 1) {
    const int l = __ffsll((unsigned long long)todo) - 1;
    const int64_t r0 = base + l, s0 = __shfl(mine, l, 64);
    int rows = 1;  // of the run: at most a page's, since its slots increase
    for (bool more = true; more;) {
      const int64_t r = r0 + rows + lane, s = slot(r);
      const uint64_t ends = ~__ballot(s >= 0 && joins(a, slot(r - 1), s));
      rows += ends ? __ffsll((unsigned long long)ends) - 1 : 64;
      more = ends == 0;
    }
    const int64_t p = s0 / a.page;
    const int first = (int)(s0 - p * a.page);
    uint32_t top = 0;
    for (int i = tid; i < rows * per_row; i += n_threads) {
      const int r = i / per_row;
      const Vec<T, V> y = load<T, V>(x + (r0 + r) * x_row + (i - r * per_row) * V);
#pragma unroll
      for (int e = 0; e < V; ++e) top = max(top, __float_as_uint(from(y.e[e])) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    if (n_threads > 64) {
      __syncthreads();
      if (lane == 0) wave_max[tid >> 6] = top;
      __syncthreads();
      for (int w = 0; w < n_threads / 64; ++w) top = max(top, wave_max[w]);
    }
    float* scale = scales + p * a.H + h;
    const float old = first ? *scale : 0.0f, least = least_scale(top, a.codes);
    const bool lost = old != old || least != least;
    const float s = lost ? __uint_as_float(0x7fc00000u) : fmaxf(old, least);
    uint8_t* page = pages + (p * a.H + h) * (int64_t)a.page * a.d;
    const Quotient over(s);
    if (s > old)  // (not if s is no number)
      for (int i = tid; i < first * per_row; i += n_threads) {
        uint32_t w[2];
        __builtin_memcpy(w, page + i * V, 8);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float y[4];
          value4(w[u], a.codes, y);
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = over(y[e] * old);
          w[u] = code4(y, a.codes);
        }
        __builtin_memcpy(page + i * V, w, 8);
      }
    for (int i = tid; i < rows * per_row; i += n_threads) {
      const int r = i / per_row, at = (i - r * per_row) * V;
      const Vec<T, V> y = load<T, V>(x + (r0 + r) * x_row + at);
      uint32_t w[2] = {0, 0};
      if (s > 0.0f) {  // (codes 0 where the scale is 0 or no number)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float z[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) z[e] = over(from(y.e[4 * u + e]));
          w[u] = code4(z, a.codes);
        }
      }
      const int64_t to = a.slots[r0 + r] - p * a.page;
      __builtin_memcpy(page + to * a.d + at, w, 8);
    }
    if (n_threads > 64) __syncthreads();  // every thread has read the old scale
    if (tid == 0) *scale = s;
  }
}

template <typename T>
int write_typed(const Write& a, hipStream_t st) {
  int chunk = (int)std::min<int64_t>(std::min(a.page, 64),
                                     std::max<int64_t>(1, a.n_rows * a.H * 2 / 4096));
  const int64_t x = (a.n_rows + chunk - 1) / chunk;
  write_kernel<T><<<dim3((unsigned)x, a.H, 2), chunk == 1 ? 64 : 256, 0, st>>>(a, chunk);
  return (int)hipGetLastError();
}

}  // namespace pg

int launch_rope(const Rope& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (a.dtype) {
    case FIBQ_F32: return pg::rope_typed<float, 4>(a, st);
    case FIBQ_F16: return pg::rope_typed<_Float16, 8>(a, st);
    default: return pg::rope_typed<__bf16, 8>(a, st);
  }
}

size_t resize_workspace_bytes(int64_t n) { return (size_t)n * 4; }

// Up to 4096 rows the scan's workgroup places them as well.
int launch_resize(const Resize& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool one = a.n_rows <= 4096;
  pg::resize_kernel<<<1, pg::kScan, 0, st>>>(a, one);
  int rc = (int)hipGetLastError();
  if (rc != 0 || one) return rc;
  pg::place_kernel<<<(unsigned)((a.n_rows + 255) / 256), 256, 0, st>>>(a);
  return (int)hipGetLastError();
}

int launch_write(const Write& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (a.dtype) {
    case FIBQ_F32: return pg::write_typed<float>(a, st);
    case FIBQ_F16: return pg::write_typed<_Float16>(a, st);
    default: return pg::write_typed<__bf16>(a, st);
  }
}

}  // namespace dev
}  // namespace fibq
