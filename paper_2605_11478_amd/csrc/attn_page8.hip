// Attention over the paged 8-bit cache (fibq_attn_cache8).
//
// A work item is one head of one sequence and a tile of up to 16 R query rows (whole
// tokens of it, G rows each).  Long items are cut into equal parts of at most P tokens;
// P follows from the lengths on the device, so that the parts fill the card once and are
// alike however unequal the sequences are.  A workgroup takes one part; its wavefronts
// take a share of the part's tokens each, 32 at a time:
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
// joined.  `ref` (a score near the row's largest so far) and `e` (the exponent of its
// largest weight) move only when a weight leaves its range, so the common path has no
// exchange between lanes.  Parts of an item that was cut leave a state each, which a
// second launch joins.
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

constexpr float kLag = 0x1p8f;      // exp2 of what a score may exceed its row's reference by
constexpr float kTop = 0x1p15f;     // weights stay below (binary16)
constexpr int kTopBits = 7;         // exponent of a row's largest weight when e is set
constexpr float kLimit = 0x1p126f;  // of scores
constexpr float kNone = -0x1p127f;  // reference of a row that has seen nothing

struct Args {
  PageAttn a;
  int tile_tokens;  // query tokens of an item
  int shift;        // log2 of the page
  int least_part;   // tokens of a part, at least
  float target;     // parts that fill the card
  float scale2;     // scale log2(e)
};

// ------------------------------------------------------------------- work --
struct Seq {
  int begin, rows, len;  // len 0 if bad
  bool bad, causal;
  int tiles;
};
__device__ __forceinline__ Seq sequence(const Args& p, int g) {
  Seq s{};
  const PageAttn& a = p.a;
  const int b = a.starts ? a.starts[g] : g, e = a.starts ? a.starts[g + 1] : g + 1;
  const int len = a.lens[g];
  if (b < 0 || e < b || e > a.n_rows) return s;
  s.begin = b;
  s.rows = e - b;
  s.bad = len < 0 || len > (int)(a.max_pages << p.shift) || (a.causal && s.rows > len);
  s.causal = a.causal && !s.bad;
  s.len = s.bad ? 0 : len;
  s.tiles = a.starts ? (int)((uint32_t)(s.rows + p.tile_tokens - 1) / (uint32_t)p.tile_tokens) : 1;
  return s;
}

// One part of an item: tokens [from, to) of the `seen` that its rows see.
struct Part {
  Seq s;
  int g, h, tile, part, parts;
  int i0, n_tokens;  // its query tokens
  int seen, from, to;
  int stride;  // from one part of an item to the next
};
// Part w of all, in every thread of the workgroup.  Parts are in the order of sequences,
// tiles from the last (a causal sequence's longest), parts, heads.  False: there is none.
template <int W>
__device__ __forceinline__ bool part_at(const Args& p, int w, Part* r, float* lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = (int)p.a.n_seqs;
  Seq s{};
  float tokens = 0.0f;
  for (int g = tid; g < n; g += 64 * W) {
    s = sequence(p, g);
    tokens += (float)s.tiles * (float)s.len;
  }
  tokens = wave_sum(tokens);
  if (lane == 0) lds[wave] = tokens;
  __syncthreads();
  tokens = 0.0f;
#pragma unroll
  for (int v = 0; v < W; ++v) tokens += lds[v];
  // (a little more than the exact quotient, so that rounding never makes a part too many)
  const float share = tokens * (float)p.a.H * 1.001f / p.target;
  const int part = (max(p.least_part, (int)fminf(share, 1073741760.0f)) + 31) & ~31;
  int* at = (int*)lds + W;  // {sequence, parts before it}, sums of the wavefronts
  __syncthreads();
  if (tid == 0) at[0] = -1;
  int before = 0;
  for (int g0 = 0; g0 < n; g0 += 64 * W) {
    const int g = g0 + tid;
    if (n > 64 * W) s = g < n ? sequence(p, g) : Seq{};
    const int parts = max(1, (int)((uint32_t)(s.len + part - 1) / (uint32_t)part));
    const int mine = g < n ? s.tiles * parts * p.a.H : 0;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
    if (lane == 63) at[2 + wave] = upto;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int v = 0; v < W; ++v) {
      if (v < wave) upto += at[2 + v];
      all += at[2 + v];
    }
    if (w < before + upto && w >= before + upto - mine) {
      at[0] = g;
      at[1] = before + upto - mine;
    }
    __syncthreads();
    before += all;
    if (w < before) break;
  }
  const int g = at[0];
  if (g < 0) return false;
  s = sequence(p, g);
  uint32_t i = (uint32_t)(w - at[1]);
  const uint32_t H = (uint32_t)p.a.H;
  r->s = s;
  r->g = g;
  r->stride = p.a.H;
  r->parts = max(1, (int)((uint32_t)(s.len + part - 1) / (uint32_t)part));
  if (i >= (uint32_t)s.tiles * (uint32_t)r->parts * H) return false;  // (counts that overflowed)
  r->h = (int)(i % H);
  i /= H;
  r->part = (int)(i % (uint32_t)r->parts);
  r->tile = s.tiles - 1 - (int)(i / (uint32_t)r->parts);
  r->i0 = r->tile * p.tile_tokens;
  r->n_tokens = min(p.tile_tokens, s.rows - r->i0);
  r->seen = s.causal ? s.len - s.rows + r->i0 + r->n_tokens : s.len;
  const int size = ((int)((uint32_t)(r->seen + r->parts - 1) / (uint32_t)r->parts) + 31) & ~31;
  r->from = min(r->part * size, r->seen);
  r->to = min(r->from + size, r->seen);
  return true;
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

// ------------------------------------------------------------- main kernel --
template <typename T, int CODES, int D, int R>
struct Wave {
  static constexpr int QP = sizeof(T) == 4 ? 2 : 1;  // parts of a query
  static constexpr int KJ = D / 64;                  // 16-byte pieces of a lane's K row
  static constexpr int CB = D / 16;                  // bytes of a lane's V row

  h8 q[R][2 * KJ][QP];
  int qe[R];                     // a row's queries are q 2^qe
  int vis[R];                    // tokens that a row sees
  float ref[R], sum[R], top[R];  // top: largest weight so far, in units of 2^e
  int e[R];
  f4 acc[R][CB];
  bool lost[R];  // queries that are no numbers

  uint4 k[2][KJ];
  uint32_t v[8][CB / 4];

  // pages of the current range, one a lane
  int page0;
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
  int g;
  int h;
  int pages;  // of the sequence

  __device__ __forceinline__ explicit Wave(const Args& p_)
      : p(p_), lane(threadIdx.x & 63), row16(lane & 15), group(lane >> 4) {}

  __device__ __forceinline__ void load_pages(int first) {
    page0 = first;
    const int at = first + lane;
    const PageAttn& a = p.a;
    id = at < pages ? a.table[(int64_t)g * a.max_pages + at] : -1;
    const bool known = id >= 0 && id < a.n_pages;
    if (!known) id = 0;
    const int64_t ph = (int64_t)id * a.H + h;
    ks = a.k_scales[ph] * p.scale2;
    vs = a.v_scales[ph];
    bad = __ballot(!known || !(fabsf(ks) < INFINITY) || !(fabsf(vs) < INFINITY));
  }
  __device__ __forceinline__ Half half(int t) {
    const int l = __builtin_amdgcn_readfirstlane((t >> p.shift) - page0);
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

  __device__ __forceinline__ void begin(const Part& r) {
    const PageAttn& a = p.a;
    const int n_rows = r.n_tokens * a.G;
#pragma unroll
    for (int s = 0; s < R; ++s) {
      const int rr = s * 16 + row16;
      const bool used = rr < n_rows;
      const int i = used ? (int)((uint32_t)rr / (uint32_t)a.G) : 0, hq = used ? rr - i * a.G : 0;
      vis[s] = !used ? 0 : r.s.causal ? r.s.len - r.s.rows + r.i0 + i + 1 : r.s.len;
      const T* x = (const T*)a.q + (((int64_t)(r.s.begin + r.i0 + i) * a.H + r.h) * a.G + hq) * D;
      T y[2 * KJ][8];
#pragma unroll
      for (int c = 0; c < 2 * KJ; ++c)
        __builtin_memcpy(y[c], x + (c / 2) * 64 + group * 16 + (c % 2) * 8, sizeof(y[c]));
      float big = 0.0f;
      int l = 0;
#pragma unroll
      for (int c = 0; c < 2 * KJ; ++c)
#pragma unroll
        for (int i8 = 0; i8 < 8; ++i8) {
          const float z = fabsf(to_float(y[c][i8]));
          l |= !(z < INFINITY);
          big = fmaxf(big, z);
        }
      big = fmaxf(big, __shfl_xor(big, 16, 64));
      big = fmaxf(big, __shfl_xor(big, 32, 64));
      l |= __shfl_xor(l, 16, 64);
      l |= __shfl_xor(l, 32, 64);
      lost[s] = l;
      int ex = 0;
      if (big > 0.0f && !l) frexpf(big, &ex);
      qe[s] = ex - 15;  // the largest is in [2^14, 2^15)
#pragma unroll
      for (int c = 0; c < 2 * KJ; ++c)
#pragma unroll
        for (int i8 = 0; i8 < 8; ++i8) {
          const float z = used && !l ? ldexpf(to_float(y[c][i8]), -qe[s]) : 0.0f;
          q[s][c][0][i8] = (_Float16)z;
          if constexpr (QP == 2) q[s][c][1][i8] = (_Float16)(z - (float)q[s][c][0][i8]);
        }
      ref[s] = kNone;
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
    const float a = exp2_(ref[r] - to);
    float w = fmaxf(top[r], __shfl_xor(top[r], 16, 64));
    w = fmaxf(w, __shfl_xor(w, 32, 64));
    w = ldexpf(w * a, e[r]);
    w = fmaxf(w, fmaxf(exp2_(big[0] - to) * fabsf(v0), exp2_(big[1] - to) * fabsf(v1)));
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

  // Tokens [from, to) of the item, from a multiple of 32.
  __device__ __forceinline__ void run(const Part& r_, int from, int to) {
    if (from >= to) return;
    const int least = r_.s.causal ? r_.s.len - r_.s.rows + r_.i0 + 1 : r_.s.len, most = r_.seen;
    g = r_.g;
    h = r_.h;
    pages = (r_.s.len + (1 << p.shift) - 1) >> p.shift;
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
        }
        float w[8], more, largest;
        for (int pass = 0; pass < 2; ++pass) {
          float most_p = 0.0f;
          more = largest = 0.0f;
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float c = limited(ldexpf(vs[u], -e[r]));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float x = exp2_(s[r][u][i] - ref[r]);
              most_p = fmaxf(most_p, x);
              more += x;
              w[4 * u + i] = x * c;
              largest = fmaxf(largest, fabsf(w[4 * u + i]));
            }
          }
          if (!__any(most_p > kLag || largest >= kTop)) break;
          move(r, s[r], vs[0], vs[1]);
        }
        sum[r] += more;
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
  return ref > kNone ? exp2_(ref - j.ref + (exp - j.exp)) : 0.0f;
}
// acc / sum 2^exp; zero where nothing was seen
__device__ __forceinline__ float finished(float acc, float sum, float exp) {
  return sum == 0.0f ? 0.0f : ldexpf(acc / sum, (int)exp);
}


template <typename T, int CODES, int D, int R, int W>
__global__ __launch_bounds__(64 * W, (R == 1 && D < 256 ? 16 : D < 256 ? 8 : 4) / 4) void main_kernel(Args p) {
  __shared__ State<D, R> states[W];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Part r;
  if (!part_at<W>(p, blockIdx.x, &r, (float*)states)) return;
  __syncthreads();
  Wave<T, CODES, D, R> wv(p);
  wv.begin(r);
  const int tiles = (r.to - r.from + 31) >> 5, each = (tiles + W - 1) / W;
  const int from = r.from + min(tiles, wave * each) * 32;
  wv.run(r, from, min(r.to, r.from + min(tiles, (wave + 1) * each) * 32));
  wv.store(&states[wave]);
  __syncthreads();
  State<D, R>* record = (State<D, R>*)p.a.ws + blockIdx.x;
  constexpr int kPer = D / 64;  // columns of a lane
  const int n_rows = r.n_tokens * p.a.G;
  for (int rr = wave; rr < n_rows; rr += W) {
    Joined j{kNone, -0x1p30f};
#pragma unroll
    for (int v = 0; v < W; ++v) j.ref = fmaxf(j.ref, states[v].ref[rr]);
#pragma unroll
    for (int v = 0; v < W; ++v)
      if (states[v].ref[rr] > kNone)
        j.exp = fmaxf(j.exp, ceilf(states[v].ref[rr] - j.ref) + states[v].exp[rr]);
    float sum = 0.0f, acc[kPer];
#pragma unroll
    for (int c = 0; c < kPer; ++c) acc[c] = 0.0f;
#pragma unroll
    for (int v = 0; v < W; ++v) {
      const float ref = states[v].ref[rr], f = factor(ref, states[v].exp[rr], j);
      sum += states[v].sum[rr] * exp2_(ref - j.ref);
#pragma unroll
      for (int c = 0; c < kPer; ++c) acc[c] += states[v].acc[rr][lane * kPer + c] * f;
    }
    if (r.parts == 1) {
      const int i = rr / p.a.G, hq = rr - i * p.a.G;
      float* out = p.a.out +
                   (((int64_t)(r.s.begin + r.i0 + i) * p.a.H + r.h) * p.a.G + hq) * D + lane * kPer;
#pragma unroll
      for (int c = 0; c < kPer; ++c) out[c] = r.s.bad ? NAN : finished(acc[c], sum, j.exp);
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
}

// Joins the states of an item that was cut; the workgroup of its first part does it, a
// wavefront for each row.
template <int D, int R>
__global__ __launch_bounds__(256) void merge_kernel(Args p) {
  __shared__ float lds[10];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Part r;
  if (!part_at<4>(p, blockIdx.x, &r, lds) || r.parts == 1 || r.part != 0) return;
  const State<D, R>* rec = (const State<D, R>*)p.a.ws + blockIdx.x;
  const int rr = blockIdx.y * 4 + wave;
  if (rr >= r.n_tokens * p.a.G) return;
  constexpr int kPer = D / 64;
  Joined j{kNone, -0x1p30f};
  for (int i = lane; i < r.parts; i += 64) j.ref = fmaxf(j.ref, rec[(int64_t)i * r.stride].ref[rr]);
  j.ref = wave_max(j.ref);
  for (int i = lane; i < r.parts; i += 64) {
    const State<D, R>& x = rec[(int64_t)i * r.stride];
    if (x.ref[rr] > kNone) j.exp = fmaxf(j.exp, ceilf(x.ref[rr] - j.ref) + x.exp[rr]);
  }
  j.exp = wave_max(j.exp);
  float sum = 0.0f, acc[kPer];
#pragma unroll
  for (int c = 0; c < kPer; ++c) acc[c] = 0.0f;
  for (int i0 = 0; i0 < r.parts; i0 += 64) {
    const int n = min(64, r.parts - i0);
    float f = 0.0f;
    if (lane < n) {
      const State<D, R>& x = rec[(int64_t)(i0 + lane) * r.stride];
      f = factor(x.ref[rr], x.exp[rr], j);
      sum += x.sum[rr] * exp2_(x.ref[rr] - j.ref);
    }
#pragma unroll 8
    for (int i = 0; i < n; ++i) {
      const float* x = rec[(int64_t)(i0 + i) * r.stride].acc[rr] + lane * kPer;
      const float fi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i));
#pragma unroll
      for (int c = 0; c < kPer; ++c) acc[c] += x[c] * fi;
    }
  }
  sum = wave_sum(sum);
  const int i = rr / p.a.G, hq = rr - i * p.a.G;
  float* out = p.a.out + (((int64_t)(r.s.begin + r.i0 + i) * p.a.H + r.h) * p.a.G + hq) * D +
               lane * kPer;
#pragma unroll
  for (int c = 0; c < kPer; ++c) out[c] = finished(acc[c], sum, j.exp);
}

// ---------------------------------------------------------------- dispatch --
constexpr int kCu = 256;

struct Plan {
  int R, parts, least;  // row tiles of 16 R; parts, at most; tokens of a part, at least
  float target;
  bool cut;
  size_t bytes;
};
Plan plan(int64_t n_seqs, int64_t n_rows, int H, int G, int64_t max_pages, int page, int d) {
  Plan p{};
  p.R = n_rows * G >= 24 * std::max<int64_t>(1, n_seqs) ? 2 : 1;
  const int64_t room = max_pages * page, tile = 16 * p.R / G;
  const int64_t items = (n_rows / tile + std::min(n_seqs, n_rows)) * H;
  const int64_t target = p.R == 2 ? 2 * kCu : d == 256 ? kCu : 2 * kCu;
  p.least = 512;
  if (items >= kCu && room <= 4096) p.least = 4096;
  p.target = (float)target;
  p.cut = room > p.least;
  p.parts = (int)(items + (p.cut ? target : 0));
  p.bytes = p.cut ? (size_t)p.parts * 16 * p.R * (d + 3) * 4 : 0;
  return p;
}

template <typename T, int CODES, int D, int R>
int launch(const Args& p, const Plan& pl, hipStream_t st) {
  constexpr int W = R == 1 ? 8 : 4;
  main_kernel<T, CODES, D, R, W><<<pl.parts, 64 * W, 0, st>>>(p);
  int rc = (int)hipGetLastError();
  if (rc != 0 || !pl.cut) return rc;
  const int rows = std::min(16 * R, p.tile_tokens * p.a.G);
  merge_kernel<D, R><<<dim3(pl.parts, (rows + 3) / 4), 256, 0, st>>>(p);
  return (int)hipGetLastError();
}
template <typename T, int CODES>
int launch_d(const Args& p, const Plan& pl, hipStream_t st) {
  switch (p.a.d) {
    case 64: return pl.R == 1 ? launch<T, CODES, 64, 1>(p, pl, st) : launch<T, CODES, 64, 2>(p, pl, st);
    case 128: return pl.R == 1 ? launch<T, CODES, 128, 1>(p, pl, st) : launch<T, CODES, 128, 2>(p, pl, st);
    default: return pl.R == 1 ? launch<T, CODES, 256, 1>(p, pl, st) : launch<T, CODES, 256, 2>(p, pl, st);
  }
}
template <typename T>
int launch_codes(const Args& p, const Plan& pl, hipStream_t st) {
  return p.a.codes == FIBQ_INT8 ? launch_d<T, FIBQ_INT8>(p, pl, st)
                                : launch_d<T, FIBQ_E4M3>(p, pl, st);
}

}  // namespace pa

size_t page_attn_workspace_bytes(int64_t n_seqs, int64_t n_rows, int H, int G, int64_t max_pages,
                                 int page, int d) {
  return pa::plan(n_seqs, n_rows, H, G, max_pages, page, d).bytes;
}

int launch_page_attn(const PageAttn& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const pa::Plan pl = pa::plan(a.n_seqs, a.n_rows, a.H, a.G, a.max_pages, a.page, a.d);
  const pa::Args p{a,        16 * pl.R / a.G, __builtin_ctz(a.page),
                   pl.least, pl.target,       a.scale * 1.44269504088896341f};
  switch (a.q_dtype) {
    case FIBQ_F32: return pa::launch_codes<float>(p, pl, st);
    case FIBQ_F16: return pa::launch_codes<f16_t>(p, pl, st);
    default: return pa::launch_codes<bf16_t>(p, pl, st);
  }
}

}  // namespace dev
}  // namespace fibq
