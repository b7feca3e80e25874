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
// Pair i of a row at position p turns by p f_i.  The angle is reduced in double, with
// what the roundings of 2 / pi and of its product with f_i leave and with an exact product
// by p, so that the farthest position loses nothing; sine and cosine of the remaining eighth of a
// turn are computed in float.  A workgroup computes the angles of its rows once, into
// LDS, and applies them to all their heads.  Bound by memory: 16384 rows x 40 heads,
// d = 128, 336 MB, 67 to 71 us (4.7 to 5.0 TB/s; a large copy moves 4.9), 105 before a
// row's angles stayed in registers.  64 rows x 36 heads: 6.2 us, the call.
constexpr int kRopeThreads = 256;
constexpr int kRopeAngles = 1024;  // angles of a workgroup, at most
// 2 / pi, quarter turns of a radian: a double and what it leaves
constexpr double kQuarters = 0x1.45f306dc9c883p-1, kQuartersRest = -0x1.6b01ec5417056p-55;

template <typename T, int V, int VT, bool HALF>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(Rope a, int tile) {
  __shared__ float2 turn[kRopeAngles];
  const int tid = threadIdx.x, half = a.rot / 2;
  const int64_t row0 = (int64_t)blockIdx.x * tile;
  const int rows = (int)min((int64_t)tile, a.n_rows - row0);
  for (int i = tid; i < rows * half; i += kRopeThreads) {
    const int r = i / half;
    const double at = (double)a.positions[row0 + r], f = a.freqs[i - r * half];
    const double unit = f * kQuarters, rest = fma(f, kQuarters, -unit) + f * kQuartersRest;
    const double n = rint(at * unit);
    float s, c;
    sincospif((float)(fma(at, unit, -n) + at * rest) * 0.5f, &s, &c);
    const int turns = (int)(n - 4.0 * floor(n * 0.25));
    float cs = turns & 1 ? -s : c, sn = turns & 1 ? c : s;
    if (turns & 2) cs = -cs, sn = -sn;
    turn[i] = make_float2(cs * a.scale, (a.inverse ? -sn : sn) * a.scale);
  }
  __syncthreads();
  // A thread has one piece of V elements (or pairs) of every head that it visits, so a
  // row's angles stay in its registers; kHeads loads are on their way at once.  What lies
  // behind the turned part is copied VT elements at a time (the last piece over the one
  // before it): in the same loop where pieces are alike, so that a row is read as a whole.
  constexpr int kHeads = HALF && V > 1 ? 2 : 4;
  const int heads = a.q_heads + a.k_heads, tail = a.d - a.rot;
  const int turned = HALF ? half / V : a.rot / V;
  const int per_head = turned + (tail + VT - 1) / VT;
  for (int c0 = 0; c0 < per_head; c0 += kRopeThreads) {
    const int pieces = min(per_head - c0, kRopeThreads), at_once = kRopeThreads / pieces;
    const int slot = tid / pieces, c = c0 + tid - slot * pieces;
    if (slot >= at_once) continue;
    const bool turns = c < turned;
    const int at = turns ? c * V : min(a.rot + (c - turned) * VT, a.d - VT);
    if (V != VT && !turns) {
      for (int i0 = slot; i0 < rows * heads; i0 += kHeads * at_once) {
        Vec<T, VT> x[kHeads];
        T* to[kHeads];
#pragma unroll
        for (int u = 0; u < kHeads; ++u) {
          const int i = min(i0 + u * at_once, rows * heads - 1), r = i / heads, h = i - r * heads;
          const int64_t row = row0 + r;
          const bool is_k = h >= a.q_heads;
          x[u] = load<T, VT>((is_k ? (const T*)a.k + row * a.k_row + (h - a.q_heads) * a.k_head
                                   : (const T*)a.q + row * a.q_row + h * a.q_head) + at);
          to[u] = (is_k ? (T*)a.k_out + row * a.ko_row + (h - a.q_heads) * a.ko_head
                        : (T*)a.q_out + row * a.qo_row + h * a.qo_head) + at;
        }
#pragma unroll
        for (int u = 0; u < kHeads; ++u)
          if (i0 + u * at_once < rows * heads) store<T, VT>(to[u], x[u]);
      }
      continue;
    }
    for (int r = 0; r < rows; ++r) {
      constexpr int kAngles = HALF ? V : V / 2;
      float2 w[kAngles];
#pragma unroll
      for (int e = 0; e < kAngles; ++e)
        w[e] = turns ? turn[r * half + (HALF ? at : at / 2) + e] : make_float2(1.0f, 0.0f);
      const int64_t row = row0 + r;
      const T *q = (const T*)a.q + row * a.q_row, *k = (const T*)a.k + row * a.k_row;
      T *qo = (T*)a.q_out + row * a.qo_row, *ko = (T*)a.k_out + row * a.ko_row;
      for (int h0 = slot; h0 < heads; h0 += kHeads * at_once) {
        Vec<T, V> x0[kHeads], x1[HALF ? kHeads : 1];
#pragma unroll
        for (int u = 0; u < kHeads; ++u) {
          const int h = min(h0 + u * at_once, heads - 1);
          const T* x = (h < a.q_heads ? q + h * a.q_head : k + (h - a.q_heads) * a.k_head) + at;
          x0[u] = load<T, V>(x);
          if constexpr (HALF) x1[u] = turns ? load<T, V>(x + half) : x0[u];
        }
#pragma unroll
        for (int u = 0; u < kHeads; ++u) {
          const int h = h0 + u * at_once;
          if (h >= heads) break;
          T* y = (h < a.q_heads ? qo + h * a.qo_head : ko + (h - a.q_heads) * a.ko_head) + at;
          if (!turns) {
            store<T, V>(y, x0[u]);
          } else if constexpr (HALF) {
            Vec<T, V> y0, y1;
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float p = from(x0[u].e[e]), q2 = from(x1[u].e[e]);
              y0.e[e] = (T)(p * w[e].x - q2 * w[e].y);
              y1.e[e] = (T)(q2 * w[e].x + p * w[e].y);
            }
            store<T, V>(y, y0);
            store<T, V>(y + half, y1);
          } else {
            Vec<T, V> y0;
#pragma unroll
            for (int e = 0; e < V; e += 2) {
              const float p = from(x0[u].e[e]), q2 = from(x0[u].e[e + 1]);
              y0.e[e] = (T)(p * w[e / 2].x - q2 * w[e / 2].y);
              y0.e[e + 1] = (T)(q2 * w[e / 2].x + p * w[e / 2].y);
            }
            store<T, V>(y, y0);
          }
        }
      }
    }
  }
}

template <typename T, int V>
int rope_typed(const Rope& a, hipStream_t st) {
  // rows of a workgroup: as many as its angles fit, but workgroups for every compute unit
  // (4 to 16 of 2^25 rows, so 2^23 workgroups at most: a grid has fewer than 2^32 threads)
  const int half = a.rot / 2;
  int tile = std::min<int64_t>(std::max(1, kRopeAngles / half), std::max<int64_t>(1, a.n_rows / 1024));
  tile = std::min(tile, 16);
  const int64_t grid = (a.n_rows + tile - 1) / tile;
  const int tail = a.d - a.rot;
  auto go = [&](auto kernel) { kernel<<<grid, kRopeThreads, 0, st>>>(a, tile); };
  const bool wide = tail == 0 || tail >= V, whole = tail % V == 0;
  if (a.layout == FIBQ_ROPE_HALF) {
    if (half % V == 0 && whole)
      go(rope_kernel<T, V, V, true>);
    else if (wide)
      go(rope_kernel<T, 1, V, true>);
    else
      go(rope_kernel<T, 1, 1, true>);
  } else {
    if (a.rot % V == 0 && whole)
      go(rope_kernel<T, V, V, false>);
    else if (wide)
      go(rope_kernel<T, 2, V, false>);
    else
      go(rope_kernel<T, 2, 1, false>);
  }
  return (int)hipGetLastError();
}

// ------------------------------------------------------------ page_resize --
// Three prefix sums over the requests: rows, pages given back, pages taken.  One
// workgroup runs them; pages given back are placed first, since what it may hand out
// depends on their number.  Sums stop at 2^31 - 1, which is more than any bound here.
// Bound by that workgroup's sums and barriers and the launch: 256 requests 8.1 us (the
// kernel 7.8), 64 requests of 262144 rows 10.1 (5.9, and 4.3 for the rows' launch); 13.6
// and 15.6 before sums over up to 1024 requests took one pass.
constexpr int kScan = 1024;
constexpr int kStaged = 4096;  // requests whose results stay in LDS for the rows' search

__device__ __forceinline__ uint32_t plus(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }

struct Sum {
  uint32_t upto, all;  // of the threads up to and with this one, of all threads
};
// `lds`: kScan / 64 words that no other sum of the same round uses
__device__ __forceinline__ uint32_t scan_wave(uint32_t v, uint32_t* lds) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(v, o, 64);
    if (lane >= o) v = plus(v, y);
  }
  if (lane == 63) lds[threadIdx.x >> 6] = v;
  return v;
}
__device__ __forceinline__ Sum scan_all(uint32_t v, const uint32_t* lds) {
  const int wave = threadIdx.x >> 6;
  Sum s{v, 0};
#pragma unroll
  for (int w = 0; w < kScan / 64; ++w) {
    if (w < wave) s.upto = plus(s.upto, lds[w]);
    s.all = plus(s.all, lds[w]);
  }
  return s;
}

struct Request {
  int len, grow, have, want;  // pages; both 0 if the request is not well-formed
  uint32_t ends;              // rows of all requests up to and with it
  bool good;
};
__device__ __forceinline__ uint32_t pages_of(uint32_t tokens, uint32_t page) {
  return (tokens + page - 1) / page;
}
__device__ __forceinline__ Request request(const Resize& a, int64_t g, uint32_t rows_before,
                                           uint32_t* lds, uint32_t* all) {
  const bool live = g < a.n;
  Request r{live ? a.lens[g] : -1, live ? a.grow[g] : 0, 0, 0, 0, false};
  const uint32_t rows = r.grow > 0 ? (uint32_t)r.grow : 0;
  const uint32_t v = scan_wave(rows, lds);
  __syncthreads();
  const Sum s = scan_all(v, lds);
  r.ends = plus(rows_before, s.upto);
  *all = s.all;
  const int64_t room = a.max_pages * a.page, after = (int64_t)r.len + r.grow;
  r.good = r.len >= 0 && r.len <= room && after >= 0 && after <= room && (int64_t)r.ends <= a.n_rows;
  if (r.good) {
    r.have = (int)pages_of((uint32_t)r.len, (uint32_t)a.page);
    r.want = (int)pages_of((uint32_t)after, (uint32_t)a.page);
  }
  return r;
}

// A row's slot and position from the scan's results.
__device__ __forceinline__ void place_row(const Resize& a, int r, const int32_t* starts,
                                          const int32_t* new_lens, const int32_t* top) {
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
    const int after = new_lens[lo];
    if (after >= 0) {
      const int rows = starts[lo + 1] - starts[lo], at = after - (starts[lo + 1] - r);
      const uint32_t page = (uint32_t)a.page;
      const int have = (int)pages_of((uint32_t)(after - rows), page), p = (int)((uint32_t)at / page);
      const int in = at - p * a.page;
      int32_t* cell = a.table + (int64_t)lo * a.max_pages + p;
      int32_t id;
      if (p < have) {
        id = *cell;
      } else {
        id = a.free_pages[top[lo] - (p - have)];
        if (in == 0) *cell = id;
      }
      if (id >= 0 && id < a.n_pages) slot = (int64_t)id * a.page + in;
      position = at;
    }
  }
  a.slots[r] = slot;
  a.positions[r] = position;
}

__global__ __launch_bounds__(kScan) void resize_kernel(Resize a, int place) {
  constexpr int kW = kScan / 64;
  __shared__ uint32_t sums[3][kW];
  __shared__ int taken_most;
  extern __shared__ int32_t staged[];  // starts, new lengths, tops (if rows are placed here)
  int32_t *l_starts = staged, *l_lens = staged + a.n + 1, *l_top = l_lens + a.n;
  const int tid = threadIdx.x, lane = tid & 63;
  const uint32_t cap = (uint32_t)a.free_cap;
  const uint32_t free0 = min((uint32_t)max(*a.n_free, 0), cap);
  if (tid == 0) taken_most = 0;
  Request r{};
  Sum back{}, need{};
  uint32_t rows_before = 0, back_before = 0;
  // pages given back, onto the stack in order
  for (int64_t g0 = 0; g0 < a.n; g0 += kScan) {
    uint32_t rows;
    r = request(a, g0 + tid, rows_before, sums[0], &rows);
    const uint32_t b = (uint32_t)max(r.have - r.want, 0), n = (uint32_t)max(r.want - r.have, 0);
    const uint32_t vb = scan_wave(b, sums[1]), vn = scan_wave(n, sums[2]);
    __syncthreads();
    back = scan_all(vb, sums[1]);
    need = scan_all(vn, sums[2]);
    const uint32_t to = plus(plus(free0, back_before), back.upto - b);
    for (uint64_t todo = __ballot(b > 0); todo; todo &= todo - 1) {
      const int l = __ffsll((unsigned long long)todo) - 1;  // a lane's pages, by all lanes
      const uint32_t m = __shfl(b, l, 64), at = __shfl(to, l, 64);
      const int32_t* from =
          a.table + (g0 + (tid & ~63) + l) * a.max_pages + __shfl(r.want, l, 64);
      for (uint32_t i = lane; i < m && at + i < cap; i += 64) a.free_pages[at + i] = from[i];
    }
    rows_before = plus(rows_before, rows);
    back_before = plus(back_before, back.all);
  }
  const uint32_t free1 = min(plus(free0, back_before), cap);
  // pages taken from its top, first come, first served
  uint32_t need_before = 0;
  rows_before = 0;
  int taken = 0;
  for (int64_t g0 = 0; g0 < a.n; g0 += kScan) {
    uint32_t rows = 0;
    if (a.n > kScan) {  // (else as computed above)
      __syncthreads();
      r = request(a, g0 + tid, rows_before, sums[0], &rows);
      const uint32_t vn = scan_wave((uint32_t)max(r.want - r.have, 0), sums[2]);
      __syncthreads();
      need = scan_all(vn, sums[2]);
    }
    const int64_t g = g0 + tid;
    const uint32_t upto = plus(need_before, need.upto);
    const int mine = max(r.want - r.have, 0);
    const bool granted = r.good && (mine == 0 || upto <= free1);
    if (granted && mine > 0) taken = (int)upto;
    if (g < a.n) {
      const int after = granted ? r.len + r.grow : -1;
      const int end = (int)min((int64_t)r.ends, a.n_rows);
      const int top = granted ? (int)(free1 - 1 - (upto - (uint32_t)mine)) : 0;
      a.new_lens[g] = after;
      a.starts[g + 1] = end;
      if (place) {
        l_starts[g + 1] = end;
        l_lens[g] = after;
        l_top[g] = top;
      } else {
        a.top[g] = top;
      }
    }
    rows_before = plus(rows_before, rows);
    need_before = plus(need_before, need.all);
  }
  // (granted requests that need pages are the first of those that do)
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) taken = max(taken, __shfl_xor(taken, o, 64));
  __syncthreads();  // (taken_most is set, and pages given back are on the stack)
  if (lane == 0 && taken > 0) atomicMax(&taken_most, taken);
  if (tid == 0) {
    a.starts[0] = 0;
    if (place) l_starts[0] = 0;
  }
  __threadfence_block();
  __syncthreads();
  if (tid == 0) *a.new_free = (int)free1 - taken_most;
  if (!place) return;
  for (int q = tid; q < (int)a.n_rows; q += kScan) place_row(a, q, l_starts, l_lens, l_top);
}

__global__ __launch_bounds__(256) void place_kernel(Resize a, int stage) {
  extern __shared__ int32_t staged[];
  const int32_t* starts = a.starts;
  if (stage) {  // (the search's dozen reads from LDS)
    for (int i = threadIdx.x; i <= (int)a.n; i += 256) staged[i] = a.starts[i];
    __syncthreads();
    starts = staged;
  }
  for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < a.n_rows; r += 256 * (int64_t)gridDim.x)
    place_row(a, (int)r, starts, a.new_lens, a.top);
}

// ----------------------------------------------------------- cache8_write --
// One workgroup takes the runs of rows that begin among its `chunk` rows, for
// one head of K or of V.  A run is consecutive rows of one page at increasing
// slots.  Its largest magnitude gives the least power of two that takes it to
// the codes' range; a page keeps the larger of that and of its scale so far,
// and where that grows, the codes before the run are rounded again.  With
// powers of two x / s and code * s_old / s are exact, so each value is rounded
// once per growth of its page's scale.  36000 rows x 8 heads, d = 128, pages of 32, 224 MB:
// 58 us, 3.9 TB/s of the 4.9 that a large copy moves; 104 before rows were held in registers
// between the search for the largest and the rounding.  Vector instructions take much of
// it, but fewer of them (integer maxima of two at once, a rounding by one fused operation)
// changed nothing.  64 rows x 4 heads: 6.8 us, the call.
__device__ __forceinline__ float least_scale(uint32_t amax_bits, int codes) {
  if (amax_bits == 0) return 0.0f;
  if (amax_bits >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  int e;
  const float m = frexpf(__uint_as_float(amax_bits), &e);  // m in [1/2, 1)
  e -= codes == FIBQ_INT8 ? 7 : 9;                         // 127 = 0.9921875 2^7, 448 = 0.875 2^9
  if (m > (codes == FIBQ_INT8 ? 0.9921875f : 0.875f)) ++e;
  return ldexpf(1.0f, max(e, -126));
}

// x / s rounded to float: the remainder of x r corrects it once, r = 1 / s rounded
// (Markstein's theorem; x r itself is exact where s is a power of two).  s may be
// any scale that a page had: of zeros below 2^-128 too, and infinite, where all is 0.
struct Quotient {
  float s, r;
  __device__ __forceinline__ explicit Quotient(float s_) : s(fminf(s_, 0x1.fffffep127f)), r(fminf(1.0f / s_, 0x1p127f)) {}
  __device__ __forceinline__ float operator()(float x) const {
    const float q = x * r;
    return copysignf(__builtin_fmaf(__builtin_fmaf(-q, s, x), r, q), q);  // (of -0 as well)
  }
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

// Rows of a run are read once, into registers, where they fit (kHeld pieces a thread).
template <typename T, int D, int kHeld>
__global__ __launch_bounds__(256) void write_kernel(Write a, int shift, int chunk) {
  constexpr int V = 8, kRow = D / V;
  __shared__ uint32_t wave_max[4];
  const int tid = threadIdx.x, lane = tid & 63, n_threads = blockDim.x;
  const int h = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  const T* x = is_v ? (const T*)a.v + h * a.v_head : (const T*)a.k + h * a.k_head;
  const int64_t x_row = is_v ? a.v_row : a.k_row;
  uint8_t* pages = (uint8_t*)(is_v ? a.v_pages : a.k_pages);
  float* scales = is_v ? a.v_scales : a.k_scales;
  const int64_t base = (int64_t)blockIdx.x * chunk, limit = a.n_pages << shift;
  // Slots of the chunk's rows and of those that a run may go on over, the row before
  // the chunk first: lane l of word w has row base - 1 + 63 w + l.
  constexpr int kWords = 4;
  int64_t slot[kWords];
  uint64_t joins[kWords], known[kWords];  // bit l: of lane l; a row joins the one before it
#pragma unroll
  for (int w = 0; w < kWords; ++w) {
    const int64_t r = base - 1 + 63 * w + lane;
    const bool used = 63 * w < chunk + (1 << shift);
    const int64_t s = used && r >= 0 && r < a.n_rows ? a.slots[r] : -1;
    slot[w] = s >= 0 && s < limit ? s : -1;
  }
#pragma unroll
  for (int w = 0; w < kWords; ++w) {
    const int64_t before = __shfl_up(slot[w], 1, 64);
    known[w] = __ballot(slot[w] >= 0);
    joins[w] = __ballot(lane > 0 && before >= 0 && slot[w] > before &&
                        slot[w] >> shift == before >> shift);
  }
  // (lane 63 of a word is lane 0 of the next, so bits 1 .. 63 are 63 rows a word)
  for (uint64_t todo = known[0] & ~joins[0] & (chunk < 63 ? (2ull << chunk) - 2 : ~1ull); todo;
       todo &= todo - 1) {
    const int l = __ffsll((unsigned long long)todo) - 1;
    const int64_t r0 = base - 1 + l, s0 = __shfl(slot[0], l, 64);
    int rows = 1;  // of the run: at most a page's, since its slots increase
    int64_t s1 = s0;
    {
      int w = 0, at = l;
#pragma unroll
      for (int u = 0; u < kWords; ++u) {
        if (u != w) continue;
        const uint64_t on = at < 63 ? joins[u] >> (at + 1) : 0;  // bits of the rows behind
        const int most = 63 - at, n = min(most, ~on ? __ffsll((unsigned long long)~on) - 1 : 64);
        rows += n;
        s1 = __shfl(slot[u], at + n, 64);
        if (n == most) w = u + 1, at = 0;
      }
    }
    const int64_t p = s0 >> shift;
    const int first = (int)(s0 - (p << shift));
    const bool dense = s1 - s0 == rows - 1;
    const int pieces = rows * kRow;
    const T* x0 = x + r0 * x_row;
    float* scale = scales + p * a.H + h;
    const float old = first ? *scale : 0.0f;
    Vec<T, V> held[kHeld];
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
      const int i = min(tid + u * n_threads, pieces - 1);
      held[u] = load<T, V>(x0 + (i / kRow) * x_row + i % kRow * V);
    }
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) top = max(top, __float_as_uint(from(held[u].e[e])) & 0x7fffffffu);
    for (int i = tid + kHeld * n_threads; i < pieces; i += n_threads) {
      const Vec<T, V> y = load<T, V>(x0 + (i / kRow) * x_row + i % kRow * V);
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
    const float least = least_scale(top, a.codes);
    const bool lost = old != old || least != least;
    const float s = lost ? __uint_as_float(0x7fc00000u) : fmaxf(old, least);
    uint8_t* page = pages + ((p * a.H + h) << shift) * D;
    const Quotient over(s);
    if (s > old)  // (not if s is no number)
      for (int i = tid; i < first * kRow; i += n_threads) {
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
    auto put = [&](int i, const Vec<T, V>& y) {
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
      const int r = i / kRow;
      const int to = dense ? first + r : (int)(a.slots[r0 + r] - (p << shift));
      __builtin_memcpy(page + to * D + i % kRow * V, w, 8);
    };
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
      if (tid + u * n_threads < pieces) put(tid + u * n_threads, held[u]);
    for (int i = tid + kHeld * n_threads; i < pieces; i += n_threads)
      put(i, load<T, V>(x0 + (i / kRow) * x_row + i % kRow * V));
    if (n_threads > 64) __syncthreads();  // every thread has read the old scale
    if (tid == 0) *scale = s;
  }
}

template <typename T>
int write_typed(const Write& a, hipStream_t st) {
  // few rows: a workgroup of one wavefront each; else those of about a page
  const int chunk = (int)std::min<int64_t>(std::min(a.page, 63),
                                           std::max<int64_t>(1, a.n_rows * a.H * 2 / 4096));
  const int64_t x = (a.n_rows + chunk - 1) / chunk;
  const dim3 grid((unsigned)x, a.H, 2);
  // Threads: four pieces of a page for each, so that a small page has one wavefront, which
  // looks over its slots once and waits at no barrier (16 prompts to 4096 tokens x 8 heads,
  // int8 or e4m3; 256 threads always, then so: pages of 16, d = 64 83 and 33 us, of 16, d =
  // 128 88 and 57, of 32, d = 128 64 and 59, of 64, d = 64 31 and 28; 64 and 128 alike).
  const int threads = chunk == 1 ? 64 : std::min(256, std::max(64, a.page * a.d / 32)), shift = __builtin_ctz(a.page);
  const bool few = a.page * a.d <= 2 * 8 * threads;  // pieces of a page for each thread
  switch (a.d) {
    case 64:
      few ? write_kernel<T, 64, 2><<<grid, threads, 0, st>>>(a, shift, chunk)
          : write_kernel<T, 64, 4><<<grid, threads, 0, st>>>(a, shift, chunk);
      break;
    case 128:
      few ? write_kernel<T, 128, 2><<<grid, threads, 0, st>>>(a, shift, chunk)
          : write_kernel<T, 128, 4><<<grid, threads, 0, st>>>(a, shift, chunk);
      break;
    default:
      few ? write_kernel<T, 256, 2><<<grid, threads, 0, st>>>(a, shift, chunk)
          : write_kernel<T, 256, 4><<<grid, threads, 0, st>>>(a, shift, chunk);
      break;
  }
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

// Up to 4096 rows of as many requests the scan's workgroup places them as well.
int launch_resize(const Resize& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool one = a.n_rows <= 4096 && a.n <= pg::kStaged;
  pg::resize_kernel<<<1, pg::kScan, one ? (3 * a.n + 1) * 4 : 0, st>>>(a, one);
  int rc = (int)hipGetLastError();
  if (rc != 0 || one || a.n_rows == 0) return rc;
  const bool stage = a.n < pg::kStaged;
  const int64_t grid = std::min<int64_t>((a.n_rows + 255) / 256, 4096);
  pg::place_kernel<<<(unsigned)grid, 256, stage ? (a.n + 1) * 4 : 0, st>>>(a, stage);
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
