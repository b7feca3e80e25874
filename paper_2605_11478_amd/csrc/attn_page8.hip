// Attention over the paged 8-bit cache (fibq_attn_cache8).
//
// A work item is one head of one sequence and a tile of up to 16 R query rows (whole
// tokens of it, G rows each).  Workgroups take equal shares of all items' tokens, so
// one may hold several short items or a part of a long one; parts leave a record each
// (reference, sum, exponent, accumulators), and a second launch joins the records of
// every item that was cut.  In a workgroup each of the four wavefronts takes a quarter
// of the tokens, 32 at a time:
//
//   S^T[t][r] = K[t][:] . Q[r][:]     v_mfma_f32_16x16x32_f16, A = codes as binary16
//                                     (exact), B = queries, scaled by a power of two per
//                                     row; two binary16 parts for float queries
//   p = exp2(S f - ref), w = p v 2^-e  f: scale log2(e) and the page's K scale, v: its V
//                                     scale; w in two binary16 parts (22 bits)
//   O[r][:] += w[r][t] V[t][:]        the same instruction, B = codes as binary16
//
// Four tokens of S^T that a lane holds are consecutive, so its weights are the A operand
// of the second product as they are: the tokens of a lane group are 4 of each half tile,
// and V is read in that order.  Nothing goes through LDS until the wavefronts' states are
// joined.  `ref` (the largest score so far, in a row) and `e` (the largest weight's
// exponent) move only when a score exceeds ref by more than kLag or a weight leaves its
// range, so the common path has no exchange between lanes.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.h"
#include "fibq.h"
#include "fibq_internal.h"

namespace fibq {
namespace dev {
namespace pa {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr float kLag = 8.0f;       // log2 by which a score may exceed its row's reference
constexpr float kTop = 0x1p15f;    // weights stay below (binary16)
constexpr int kTopBits = 7;        // exponent of a row's largest weight when e is set
constexpr float kLimit = 0x1p126f; // of scores
constexpr int64_t kItem = 64;      // an item costs about as much as this many tokens
constexpr int64_t kChunk = 512;    // tokens of a workgroup, at least

struct Args {
  PageAttn a;
  int tile_tokens;  // query tokens of an item
  int shift;        // log2 of the page
  int n_wg;         // workgroups, at most
  int cut;          // items may be cut
  float scale2;     // scale log2(e)
};

// ------------------------------------------------------------------- work --
struct Seq {
  int64_t begin, rows, len;  // len 0 if bad
  bool bad, causal;
  int64_t tiles, head;  // items and weight of one head
};
__device__ __forceinline__ Seq sequence(const Args& p, int64_t g) {
  Seq s{};
  const PageAttn& a = p.a;
  const int64_t b = a.starts ? a.starts[g] : g, e = a.starts ? a.starts[g + 1] : g + 1;
  if (b < 0 || e < b || e > a.n_rows) return s;
  const int64_t len = a.lens[g];
  s.begin = b;
  s.rows = e - b;
  s.bad = len < 0 || len > a.max_pages << p.shift || (a.causal && s.rows > len);
  s.causal = a.causal && !s.bad;
  s.len = s.bad ? 0 : len;
  s.tiles = (int64_t)((uint32_t)(s.rows + p.tile_tokens - 1) / (uint32_t)p.tile_tokens);
  s.head = s.causal ? s.tiles * (s.len - s.rows + kItem) +
                          p.tile_tokens * (s.tiles * (s.tiles - 1) / 2) + s.rows
                    : s.tiles * (s.len + kItem);
  if (s.rows == 0) s.head = 0;
  return s;
}
// weight of the tiles before tile t of a head
__device__ __forceinline__ int64_t before_tile(const Args& p, const Seq& s, int64_t t) {
  return s.causal ? t * (s.len - s.rows + kItem) + p.tile_tokens * (t * (t + 1) / 2)
                  : t * (s.len + kItem);
}
__device__ __forceinline__ int64_t tile_tokens_seen(const Args& p, const Seq& s, int64_t t) {
  return s.causal ? s.len - s.rows + min(s.rows, (t + 1) * p.tile_tokens) : s.len;
}

// The share of workgroup w: [lo, hi) of the weights of all items, and the sequence
// that holds lo with the weight before it.  Called by all threads of kThreads.
struct Share {
  int64_t lo, hi, seq, before, each, more;
  int n_wg;
  __device__ __forceinline__ int64_t begin(int64_t w) const { return each * w + min(w, more); }
};
__device__ __forceinline__ Share share(const Args& p, int w, int64_t* lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t n = p.a.n_seqs;
  int64_t total = 0, mine = 0, upto = 0;
  for (int64_t g0 = 0; g0 < n; g0 += kThreads) {
    const int64_t g = g0 + tid;
    mine = g < n ? sequence(p, g).head * p.a.H : 0;
    upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
    if (lane == 63) lds[wave] = upto;
    __syncthreads();
    for (int v = 0; v < kWaves; ++v) {
      if (v < wave) upto += lds[v];
      total += lds[v];
    }
    __syncthreads();
  }
  Share s;
  s.n_wg = (int)max((int64_t)1, min((int64_t)p.n_wg, total / kChunk));
  s.each = total / s.n_wg;
  s.more = total - s.each * s.n_wg;
  s.lo = w < s.n_wg ? s.begin(w) : total;
  s.hi = w < s.n_wg ? s.begin(w + 1) : total;
  if (tid == 0) lds[0] = n, lds[1] = 0;
  __syncthreads();
  if (s.lo >= s.hi) {
    s.seq = n;
    s.before = 0;
    return s;
  }
  int64_t carry = 0;
  for (int64_t g0 = 0; g0 < n; g0 += kThreads) {  // (one round: as summed above)
    if (n > kThreads) {
      const int64_t g = g0 + tid;
      mine = g < n ? sequence(p, g).head * p.a.H : 0;
      upto = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(upto, o, 64);
        if (lane >= o) upto += y;
      }
      if (lane == 63) lds[2 + wave] = upto;
      __syncthreads();
      int64_t sum = 0;
      for (int v = 0; v < kWaves; ++v) {
        if (v < wave) upto += lds[2 + v];
        sum += lds[2 + v];
      }
      upto += carry;
      carry += sum;
    }
    if (upto - mine <= s.lo && s.lo < upto) {
      lds[0] = g0 + tid;
      lds[1] = upto - mine;
    }
    __syncthreads();
    if (lds[0] < n) break;
  }
  s.seq = lds[0];
  s.before = lds[1];
  __syncthreads();
  return s;
}

// One item's part: tokens [from, to) of what its rows see.
struct Part {
  Seq s;
  int64_t g, tile, seen, from, to;
  int h;
  bool begins, ends;
};
// The item at weight x of a share, up to weight hi.  Returns the weight behind it.
__device__ __forceinline__ int64_t part_at(const Args& p, const Seq& s, int64_t g, int64_t before,
                                           int64_t x, int64_t hi, Part* r) {
  const int64_t local = x - before;
  r->s = s;
  r->g = g;
  r->h = (int)(local / s.head);
  const int64_t in_head = local - r->h * s.head;
  int64_t lo = 0, up = s.tiles - 1;  // the last tile that begins at or before in_head
  while (lo < up) {
    const int64_t mid = (lo + up + 1) / 2;
    if (before_tile(p, s, mid) <= in_head)
      lo = mid;
    else
      up = mid - 1;
  }
  r->tile = lo;
  r->seen = tile_tokens_seen(p, s, lo);
  const int64_t off = in_head - before_tile(p, s, lo), all = r->seen + kItem;
  const int64_t end = min(all, off + (hi - x));
  r->begins = off == 0;
  r->ends = end == all;
  auto token = [](int64_t o) { return o <= kItem ? (int64_t)0 : (o - kItem) & ~(int64_t)31; };
  r->from = token(off);
  r->to = r->ends ? r->seen : token(end);
  return x + (end - off);
}

// ---------------------------------------------------------------- records --
// A state of an item's rows: references, sums, exponents and accumulators.
template <int D, int R>
struct State {
  float ref[16 * R], sum[16 * R], exp[16 * R];
  float acc[16 * R][D];
};

// -------------------------------------------------------------- operators --
template <int CODES>
__device__ __forceinline__ h8 halves(uint32_t lo, uint32_t hi);  // 8 codes, in order
template <>
__device__ __forceinline__ h8 halves<FIBQ_E4M3>(uint32_t lo, uint32_t hi) {
  const h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false),
           b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true),
           c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false),
           d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// 1024 + (x + 128) in binary16 has the byte x ^ 0x80 as its low bits
__device__ __forceinline__ h2 biased(uint32_t flipped, uint32_t select) {
  const uint32_t u = __builtin_amdgcn_perm(0x64646464u, flipped, select);
  h2 r;
  __builtin_memcpy(&r, &u, 4);
  return r - h2{(_Float16)1152, (_Float16)1152};
}
template <>
__device__ __forceinline__ h8 halves<FIBQ_INT8>(uint32_t lo, uint32_t hi) {
  lo ^= 0x80808080u;
  hi ^= 0x80808080u;
  const h2 a = biased(lo, 0x04010400u), b = biased(lo, 0x04030402u), c = biased(hi, 0x04010400u),
           d = biased(hi, 0x04030402u);
  return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float limited(float x) {
  return __builtin_amdgcn_fmed3f(x, -kLimit, kLimit);
}
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x) {
  T y[8];
  __builtin_memcpy(y, p, sizeof(y));
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = to_float(y[e]);
}

// ------------------------------------------------------------- main kernel --
template <typename T, int CODES, int D, int R>
struct Wave {
  static constexpr int QP = sizeof(T) == 4 ? 2 : 1;  // parts of a query
  static constexpr int KJ = D / 64;                  // 16-byte pieces of a lane's K row
  static constexpr int CB = D / 16;                  // bytes of a lane's V row

  h8 q[R][2 * KJ][QP];
  int qe[R];        // a row's queries are q 2^qe
  int vis[R];       // tokens that a row sees
  float ref[R], sum[R], top[R];  // top: largest weight so far, in units of 2^e
  int e[R];
  f4 acc[R][CB];
  bool lost[R];  // queries that are no numbers

  uint4 k[2][KJ];
  uint32_t v[8][CB / 4];

  // pages of the current range, one a lane
  int64_t page0;
  int id;
  float ks, vs;
  uint64_t bad;

  struct Half {  // half a tile: 16 tokens of one page
    const uint8_t *k, *v;
    float ks, vs;
    bool bad;
  };

  const Args& p;
  const int lane, row16, group;
  int64_t g;
  int h;
  int pages;  // of the sequence

  __device__ __forceinline__ explicit Wave(const Args& p_)
      : p(p_), lane(threadIdx.x & 63), row16(lane & 15), group(lane >> 4) {}

  __device__ __forceinline__ void load_pages(int64_t first) {
    page0 = first;
    const int64_t at = first + lane;
    const PageAttn& a = p.a;
    id = at < pages ? a.table[g * a.max_pages + at] : -1;
    const bool known = id >= 0 && id < a.n_pages;
    if (!known) id = 0;
    const int64_t ph = (int64_t)id * a.H + h;
    ks = a.k_scales[ph] * p.scale2;
    vs = a.v_scales[ph];
    bad = __ballot(!known || !(fabsf(ks) < INFINITY) || !(fabsf(vs) < INFINITY));
  }
  __device__ __forceinline__ Half half(int t) {
    const int l = __builtin_amdgcn_readfirstlane((int)((t >> p.shift) - page0));
    const int64_t ph = (int64_t)__builtin_amdgcn_readlane(id, l) * p.a.H + h;
    const int64_t at = ((ph << p.shift) + (t & ((1 << p.shift) - 1))) * D;
    return {(const uint8_t*)p.a.k_pages + at, (const uint8_t*)p.a.v_pages + at,
            __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), l)),
            __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), l)),
            (bool)((bad >> l) & 1)};
  }
  __device__ __forceinline__ void load_k(const Half* t) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < KJ; ++j)
        k[u][j] = *(const uint4*)(t[u].k + (row16 * D + group * 16 + j * 64));
  }
  __device__ __forceinline__ void load_v(const Half* t) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        __builtin_memcpy(v[4 * u + i],
                         __builtin_assume_aligned(t[u].v + ((group * 4 + i) * D + row16 * CB),
                                                  CB < 16 ? CB : 16),
                         CB);
  }

  __device__ __forceinline__ void begin(const Part& r, int n_rows) {
    const PageAttn& a = p.a;
    g = r.g;
    h = r.h;
    pages = (int)((r.s.len + (1 << p.shift) - 1) >> p.shift);
    const int64_t i0 = r.tile * p.tile_tokens;
#pragma unroll
    for (int s = 0; s < R; ++s) {
      const int rr = s * 16 + row16;
      const bool used = rr < n_rows;
      const int i = used ? rr / a.G : 0, hq = used ? rr - i * a.G : 0;
      vis[s] = !used ? 0 : (int)(r.s.causal ? r.s.len - r.s.rows + i0 + i + 1 : r.s.len);
      const T* x = (const T*)a.q + (((r.s.begin + i0 + i) * a.H + h) * a.G + hq) * D;
      float y[2 * KJ][8];
      float big = 0.0f;
      lost[s] = false;
#pragma unroll
      for (int c = 0; c < 2 * KJ; ++c) {
        load8(x + (c / 2) * 64 + group * 16 + (c % 2) * 8, y[c]);
#pragma unroll
        for (int i8 = 0; i8 < 8; ++i8) {
          if (!used) y[c][i8] = 0.0f;
          if (!(fabsf(y[c][i8]) < INFINITY)) {
            lost[s] = true;
            y[c][i8] = 0.0f;
          }
          big = fmaxf(big, fabsf(y[c][i8]));
        }
      }
      big = fmaxf(big, __shfl_xor(big, 16, 64));
      big = fmaxf(big, __shfl_xor(big, 32, 64));
      int l = lost[s];
      l |= __shfl_xor(l, 16, 64);
      l |= __shfl_xor(l, 32, 64);
      lost[s] = l;
      int ex = 0;
      if (big > 0.0f) frexpf(big, &ex);
      qe[s] = ex - 15;  // the largest is in [2^14, 2^15)
#pragma unroll
      for (int c = 0; c < 2 * KJ; ++c)
#pragma unroll
        for (int i8 = 0; i8 < 8; ++i8) {
          const float z = ldexpf(y[c][i8], -qe[s]);
          q[s][c][0][i8] = (_Float16)z;
          if constexpr (QP == 2) q[s][c][1][i8] = (_Float16)(z - (float)q[s][c][0][i8]);
        }
      ref[s] = -INFINITY;
      sum[s] = 0.0f;
      top[s] = 0.0f;
      e[s] = 0;
#pragma unroll
      for (int c = 0; c < CB; ++c) acc[s][c] = f4{0, 0, 0, 0};
    }
  }

  // A row's reference becomes its largest score, and its weights' exponent that of the
  // largest weight.  s: scores, -inf where masked.
  __device__ __forceinline__ void move(int r, const f4* s, float v0, float v1) {
    float big[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      big[u] = fmaxf(fmaxf(s[u][0], s[u][1]), fmaxf(s[u][2], s[u][3]));
      big[u] = fmaxf(big[u], __shfl_xor(big[u], 16, 64));
      big[u] = fmaxf(big[u], __shfl_xor(big[u], 32, 64));
    }
    const float to = fmaxf(ref[r], fmaxf(big[0], big[1]));
    const bool live = to > -INFINITY;
    const float a = live ? exp2_(ref[r] - to) : 1.0f;
    float w = fmaxf(top[r], __shfl_xor(top[r], 16, 64));
    w = fmaxf(w, __shfl_xor(w, 32, 64));
    w = ldexpf(w * a, e[r]);
    if (live) w = fmaxf(w, fmaxf(exp2_(big[0] - to) * fabsf(v0), exp2_(big[1] - to) * fabsf(v1)));
    int ew = e[r];
    if (w > 0.0f) {
      frexpf(w, &ew);
      ew = max(ew - 1 - kTopBits, -100);
    }
    const float by = ldexpf(a, e[r] - ew);
    sum[r] *= a;
    top[r] = ldexpf(w, -ew);
    ref[r] = to;
    e[r] = ew;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float b = __shfl(by, group * 4 + i, 64);
#pragma unroll
      for (int c = 0; c < CB; ++c) acc[r][c][i] *= b;
    }
  }

  // Weights of a tile, their sum in units of the reference, and the largest magnitude.
  __device__ __forceinline__ void weights(int r, const f4* s, const float* v, float* w, float* all,
                                          float* largest) const {
    const float base = ref[r] > -INFINITY ? ref[r] : 0.0f;
    *all = *largest = 0.0f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float c = limited(ldexpf(v[u], -e[r]));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = exp2_(s[u][i] - base);
        *all += x;
        w[4 * u + i] = x * c;
        *largest = fmaxf(*largest, fabsf(w[4 * u + i]));
      }
    }
  }

  // Tokens [from, to) of the item, from a multiple of 32.
  __device__ __forceinline__ void run(int from, int to, int least, int most) {
    if (from >= to) return;
    load_pages(from >> p.shift);
    Half t[2] = {half(from), half(min(from + 16, to - 1) & ~15)};
    load_k(t);
    load_v(t);
    for (int t0 = from; t0 < to; t0 += 32) {
      f4 s[R][2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < R; ++r) s[r][u] = f4{0, 0, 0, 0};
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < KJ; ++j) {
          const h8 a = halves<CODES>(k[u][j].x, k[u][j].y), b = halves<CODES>(k[u][j].z, k[u][j].w);
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = QP - 1; i >= 0; --i) {
              s[r][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, q[r][2 * j][i], s[r][u], 0, 0, 0);
              s[r][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b, q[r][2 * j + 1][i], s[r][u], 0, 0, 0);
            }
        }
      // the next tile's keys are on their way from here on, its values from the end
      const float ks[2] = {t[0].ks, t[1].ks}, vs[2] = {t[0].vs, t[1].vs};
      const bool lost_page[2] = {t[0].bad, t[1].bad};
      const int next = t0 + 32;
      if (next < to) {
        if ((next >> p.shift) - page0 >= 63) load_pages(next >> p.shift);
        t[0] = half(next);
        t[1] = half(min(next + 16, to - 1) & ~15);
        load_k(t);
      }
      const bool masked = t0 + 32 > least;
      h8 hi[R], lo[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float big = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float f = limited(ldexpf(ks[u], qe[r]));
#pragma unroll
          for (int i = 0; i < 4; ++i) s[r][u][i] = limited(s[r][u][i] * f);
          if (lost_page[u]) s[r][u] = f4{NAN, NAN, NAN, NAN};
          if (masked) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (t0 + u * 16 + group * 4 + i >= vis[r]) s[r][u][i] = -INFINITY;
          }
          big = fmaxf(big, fmaxf(fmaxf(s[r][u][0], s[r][u][1]), fmaxf(s[r][u][2], s[r][u][3])));
        }
        if (__any(big > ref[r] + kLag)) move(r, s[r], vs[0], vs[1]);
        float w[8], more, largest;
        weights(r, s[r], vs, w, &more, &largest);
        sum[r] += more;
        if (__any(largest >= kTop)) {  // (what was added to the sum moves with it)
          move(r, s[r], vs[0], vs[1]);
          weights(r, s[r], vs, w, &more, &largest);
        }
        top[r] = fmaxf(top[r], largest);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          hi[r][i] = (_Float16)w[i];
          lo[r][i] = (_Float16)(w[i] - (float)hi[r][i]);
        }
      }
      if (t0 + 32 > most) {  // what lies behind the last token may hold anything
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (t0 + (i / 4) * 16 + group * 4 + i % 4 >= most)
#pragma unroll
            for (int c = 0; c < CB / 4; ++c) v[i][c] = 0;
      }
#pragma unroll
      for (int c = 0; c < CB / 4; ++c)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          // columns 4 c + 2 m and the next: pairs of tokens side by side
          const uint32_t sel = m ? 0x07030602u : 0x05010400u;
          const uint32_t a = __builtin_amdgcn_perm(v[1][c], v[0][c], sel),
                         b = __builtin_amdgcn_perm(v[3][c], v[2][c], sel),
                         d = __builtin_amdgcn_perm(v[5][c], v[4][c], sel),
                         f = __builtin_amdgcn_perm(v[7][c], v[6][c], sel);
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const h8 x = pairs(a, b, d, f, n);
            const int at = 4 * c + 2 * m + n;
#pragma unroll
            for (int r = 0; r < R; ++r) {
              acc[r][at] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo[r], x, acc[r][at], 0, 0, 0);
              acc[r][at] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi[r], x, acc[r][at], 0, 0, 0);
            }
          }
        }
      if (next < to) load_v(t);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      sum[r] += __shfl_xor(sum[r], 16, 64);
      sum[r] += __shfl_xor(sum[r], 32, 64);
    }
  }
  // 8 tokens' codes of one column: the low or high halves of four words
  __device__ __forceinline__ h8 pairs(uint32_t a, uint32_t b, uint32_t c, uint32_t d, int n) {
    h2 x[4];
    const uint32_t w[4] = {a, b, c, d};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (CODES == FIBQ_E4M3)
        x[i] = n ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, true)
                 : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, false);
      else
        x[i] = biased(w[i] ^ 0x80808080u, n ? 0x04030402u : 0x04010400u);
    }
    return h8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
  }

  __device__ __forceinline__ void store(State<D, R>* to) const {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (group == 0) {
        to->ref[r * 16 + row16] = ref[r];
        to->sum[r * 16 + row16] = lost[r] && sum[r] > 0.0f ? NAN : sum[r];
        to->exp[r * 16 + row16] = (float)e[r];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < CB; c += 4)
          *(f4*)&to->acc[r * 16 + group * 4 + i][row16 * CB + c] =
              f4{acc[r][c][i], acc[r][c + 1][i], acc[r][c + 2][i], acc[r][c + 3][i]};
    }
  }
};

// Joins n states of a row: their common reference and exponent, and each one's factors.
struct Joined {
  float ref, exp;
};
__device__ __forceinline__ float factor(float ref, float exp, const Joined& j) {
  return ref > -INFINITY ? exp2_(ref - j.ref + (exp - j.exp)) : 0.0f;
}
__device__ __forceinline__ float weight(float ref, const Joined& j) {
  return ref > -INFINITY ? exp2_(ref - j.ref) : 0.0f;
}
// acc / sum 2^exp; zero where nothing was seen
__device__ __forceinline__ float finished(float acc, float sum, float exp) {
  return sum == 0.0f ? 0.0f : ldexpf(acc / sum, (int)exp);
}

template <typename T, int CODES, int D, int R>
__global__ __launch_bounds__(kThreads) void main_kernel(Args p) {
  __shared__ State<D, R> states[kWaves];
  __shared__ int64_t lds[2 + kWaves];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // neighbours in the list of items share keys and values: one XCD's L2 serves them
  const int per = p.n_wg / 8, b = blockIdx.x;
  const int w = p.n_wg % 8 == 0 ? (b % 8) * per + b / 8 : b;
  const Share sh = share(p, w, lds);
  int64_t x = sh.lo, g = sh.seq, before = sh.before;
  if (g >= p.a.n_seqs) return;
  Seq s = sequence(p, g);
  while (x < sh.hi) {
    while (x >= before + s.head * p.a.H) {
      before += s.head * p.a.H;
      s = sequence(p, ++g);
    }
    Part r;
    const int64_t after = part_at(p, s, g, before, x, p.cut ? sh.hi : INT64_MAX, &r);
    x = after;
    const bool skip = !p.cut && !r.begins;  // (an uncut item is whole where it begins)
    if (skip) {
      // the item began in the share before: its rest is that share's
      const int64_t off = before + r.h * s.head + before_tile(p, s, r.tile);
      x = off + r.seen + kItem;
      continue;
    }
    const int64_t i0 = r.tile * p.tile_tokens;
    const int n_rows = (int)min((int64_t)p.tile_tokens, s.rows - i0) * p.a.G;
    const int64_t row0 = s.begin + i0;
    Wave<T, CODES, D, R> wv(p);
    wv.begin(r, n_rows);
    const int tiles = (int)((r.to - r.from + 31) >> 5), each = (tiles + kWaves - 1) / kWaves;
    const int from = (int)r.from + min(tiles, wave * each) * 32;
    const int to = (int)min(r.to, r.from + (int64_t)min(tiles, (wave + 1) * each) * 32);
    const int least = (int)(s.causal ? s.len - s.rows + i0 + 1 : s.len);
    wv.run(from, to, least, (int)r.seen);
    wv.store(&states[wave]);
    __syncthreads();
    State<D, R>* record =
        (State<D, R>*)p.a.ws + 2 * (int64_t)w + (r.begins ? 1 : 0);
    constexpr int kPer = D / 64;  // columns of a lane
    for (int rr = wave; rr < n_rows; rr += kWaves) {
      Joined j{-INFINITY, -INFINITY};
#pragma unroll
      for (int v = 0; v < kWaves; ++v) j.ref = fmaxf(j.ref, states[v].ref[rr]);
#pragma unroll
      for (int v = 0; v < kWaves; ++v)
        if (states[v].ref[rr] > -INFINITY)
          j.exp = fmaxf(j.exp, ceilf(states[v].ref[rr] - j.ref) + states[v].exp[rr]);
      if (j.exp == -INFINITY) j.exp = 0.0f;
      float sum = 0.0f, acc[kPer];
#pragma unroll
      for (int c = 0; c < kPer; ++c) acc[c] = 0.0f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        const float ref = states[v].ref[rr], f = factor(ref, states[v].exp[rr], j);
        sum += states[v].sum[rr] * weight(ref, j);
#pragma unroll
        for (int c = 0; c < kPer; ++c) acc[c] += states[v].acc[rr][lane * kPer + c] * f;
      }
      if (r.begins && r.ends) {
        const int i = rr / p.a.G, hq = rr - i * p.a.G;
        float* out = p.a.out + (((row0 + i) * p.a.H + r.h) * p.a.G + hq) * D + lane * kPer;
#pragma unroll
        for (int c = 0; c < kPer; ++c) out[c] = s.bad ? NAN : finished(acc[c], sum, j.exp);
      } else {
        if (lane == 0) {
          record->ref[rr] = j.ref;
          record->sum[rr] = sum;
          record->exp[rr] = j.exp;
        }
#pragma unroll
        for (int c = 0; c < kPer; ++c) record->acc[rr][lane * kPer + c] = acc[c];
      }
    }
    __syncthreads();
  }
}

// Joins the records of the item that share w begins and does not end: its own second
// one and the first ones of the shares behind it, up to the one that ends the item.  A
// wavefront takes a row.
template <int D, int R>
__global__ __launch_bounds__(kThreads) void merge_kernel(Args p) {
  __shared__ int64_t lds[2 + kWaves];
  const int lane = threadIdx.x & 63, w = blockIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Share sh = share(p, w, lds);
  if (sh.lo >= sh.hi || w + 1 >= sh.n_wg) return;
  int64_t g = sh.seq, before = sh.before;
  Seq s = sequence(p, g);
  while (sh.hi - 1 >= before + s.head * p.a.H) {
    before += s.head * p.a.H;
    s = sequence(p, ++g);
  }
  Part r;
  part_at(p, s, g, before, sh.hi - 1, sh.hi, &r);  // the last item of the share
  const int64_t begin = before + r.h * s.head + before_tile(p, s, r.tile);
  const int64_t end = begin + r.seen + kItem;
  if (begin < sh.lo || end <= sh.hi) return;
  int count = 2;
  while (sh.begin(w + count) < end) ++count;
  const State<D, R>* rec = (const State<D, R>*)p.a.ws;
  auto at = [&](int i) { return rec + 2 * (int64_t)(w + i) + (i == 0); };
  const int64_t i0 = r.tile * p.tile_tokens;
  const int n_rows = (int)min((int64_t)p.tile_tokens, s.rows - i0) * p.a.G;
  constexpr int kPer = D / 64;
  for (int rr = blockIdx.y * kWaves + wave; rr < n_rows; rr += gridDim.y * kWaves) {
    Joined j{-INFINITY, -INFINITY};
    for (int i = lane; i < count; i += 64) j.ref = fmaxf(j.ref, at(i)->ref[rr]);
    j.ref = wave_max(j.ref);
    for (int i = lane; i < count; i += 64)
      if (at(i)->ref[rr] > -INFINITY)
        j.exp = fmaxf(j.exp, ceilf(at(i)->ref[rr] - j.ref) + at(i)->exp[rr]);
    j.exp = wave_max(j.exp);
    if (j.exp == -INFINITY) j.exp = 0.0f;
    float sum = 0.0f, acc[kPer];
#pragma unroll
    for (int c = 0; c < kPer; ++c) acc[c] = 0.0f;
    for (int i0 = 0; i0 < count; i0 += 64) {
      const int n = min(64, count - i0);
      float f = 0.0f;
      if (lane < n) {
        const State<D, R>* x = at(i0 + lane);
        f = factor(x->ref[rr], x->exp[rr], j);
        sum += x->sum[rr] * weight(x->ref[rr], j);
      }
#pragma unroll 8
      for (int i = 0; i < n; ++i) {
        const float* x = at(i0 + i)->acc[rr] + lane * kPer;
        const float fi = __shfl(f, i, 64);
#pragma unroll
        for (int c = 0; c < kPer; ++c) acc[c] += x[c] * fi;
      }
    }
    sum = wave_sum(sum);
    const int i = rr / p.a.G, hq = rr - i * p.a.G;
    float* out = p.a.out + (((s.begin + i0 + i) * p.a.H + r.h) * p.a.G + hq) * D + lane * kPer;
#pragma unroll
    for (int c = 0; c < kPer; ++c) out[c] = s.bad ? NAN : finished(acc[c], sum, j.exp);
  }
}

// ---------------------------------------------------------------- dispatch --
constexpr int kCu = 256;

struct Plan {
  int R, n_wg;
  bool cut;
  size_t bytes;
};
// Row tiles of 16 R: the large one where sequences have rows for it.
Plan plan(int64_t n_seqs, int64_t n_rows, int H, int G, int64_t max_pages, int page, int d) {
  Plan p{};
  const int large = d == 256 ? 2 : 4;
  p.R = n_rows * G >= 24 * std::max<int64_t>(1, n_seqs) ? large : 1;
  const int64_t room = max_pages * page;
  const int64_t tile = 16 * p.R / G, items = (n_rows / tile + std::min(n_seqs, n_rows)) * H;
  const int64_t most = p.R > 1 ? kCu : d == 64 ? 4 * kCu : d == 128 ? 3 * kCu : 2 * kCu;
  p.n_wg = (int)std::max<int64_t>(1, std::min(most, items * (room + kItem) / kChunk));
  if (p.n_wg > 8) p.n_wg = (p.n_wg + 7) / 8 * 8;
  p.cut = room > kChunk && p.n_wg > 1;
  p.bytes = p.cut ? (size_t)p.n_wg * 2 * 16 * p.R * (d + 3) * 4 : 0;
  return p;
}

template <typename T, int CODES, int D, int R>
int launch(const Args& p, hipStream_t st) {
  main_kernel<T, CODES, D, R><<<p.n_wg, kThreads, 0, st>>>(p);
  int rc = (int)hipGetLastError();
  if (rc != 0 || !p.cut) return rc;
  const int rows = std::min(16 * R, p.tile_tokens * p.a.G);
  merge_kernel<D, R><<<dim3(p.n_wg, (rows + kWaves - 1) / kWaves), kThreads, 0, st>>>(p);
  return (int)hipGetLastError();
}
template <typename T, int CODES>
int launch_d(const Args& p, int R, hipStream_t st) {
  switch (p.a.d) {
    case 64: return R == 1 ? launch<T, CODES, 64, 1>(p, st) : launch<T, CODES, 64, 4>(p, st);
    case 128: return R == 1 ? launch<T, CODES, 128, 1>(p, st) : launch<T, CODES, 128, 4>(p, st);
    default: return R == 1 ? launch<T, CODES, 256, 1>(p, st) : launch<T, CODES, 256, 2>(p, st);
  }
}
template <typename T>
int launch_codes(const Args& p, int R, hipStream_t st) {
  return p.a.codes == FIBQ_INT8 ? launch_d<T, FIBQ_INT8>(p, R, st)
                                : launch_d<T, FIBQ_E4M3>(p, R, st);
}

}  // namespace pa

size_t page_attn_workspace_bytes(int64_t n_seqs, int64_t n_rows, int H, int G, int64_t max_pages,
                                 int page, int d) {
  return pa::plan(n_seqs, n_rows, H, G, max_pages, page, d).bytes;
}

int launch_page_attn(const PageAttn& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const pa::Plan pl = pa::plan(a.n_seqs, a.n_rows, a.H, a.G, a.max_pages, a.page, a.d);
  const pa::Args p{a,       16 * pl.R / a.G, __builtin_ctz(a.page),
                   pl.n_wg, pl.cut,          a.scale * 1.44269504088896341f};
  switch (a.q_dtype) {
    case FIBQ_F32: return pa::launch_codes<float>(p, pl.R, st);
    case FIBQ_F16: return pa::launch_codes<f16_t>(p, pl.R, st);
    default: return pa::launch_codes<bf16_t>(p, pl.R, st);
  }
}

}  // namespace dev
}  // namespace fibq
