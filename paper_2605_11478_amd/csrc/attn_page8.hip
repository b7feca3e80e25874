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
//                                     scale
//   O[r][:] += w[r][t] V[t][:]        v_mfma_f32_16x16x32_bf16, A = w in three bfloat16
//                                     parts (its 24 bits, at any exponent: two binary16
//                                     parts lose those of a weight far below its row's
//                                     largest, whose values may be 0), B = codes (exact)
//
// Four tokens of S^T that a lane holds are consecutive, so its weights are the A operand
// of the second product as they are: the tokens of a lane group are 4 of each half tile,
// and V is read in that order.  Nothing goes through LDS until the wavefronts' states are
// joined.  `ref` (a score near the row's largest so far) and `e` (the exponent of its
// largest weight) move only when a weight leaves its range, so the common path has no
// exchange between lanes.  Parts of an item that was cut leave a state each, which a
// second launch joins.
//
// What bounds it.  Single tokens over long sequences: memory (48 sequences to 32768 tokens
// x 4 heads, 425 MB: 94 us, 4.5 TB/s; one of 131072 x 8 heads, d = 128, 269 MB: 56 us, 4.8
// TB/s; a large copy moves 4.9).  Row tiles: vector and matrix instructions (8 chunks to
// 512 tokens over up to 4096, 67 GFLOP: 170 us; vector instructions, matrix ones among them,
// are issued in 57 % of the SIMDs' cycles, the matrix units are busy in 31 %).  Few short
// items: the chain of launch, lengths, table, pages and the wait for each next tile (64
// sequences to 2048 tokens: 13 us for 35 MB).  Two binary16 parts of a weight took
// 92, 55, 147 and 12 us there; choosing between both forms tile by tile 94, 57, 193 and 15
// (registers).
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
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr float kLag = 0x1p8f;      // exp2 of what a score may exceed its row's reference by
constexpr float kTop = 0x1p40f;     // weights stay below, so that sums of 2^30 codes do not overflow
constexpr int kTopBits = 24;        // exponent of a row's largest weight when e is set: one of 2^-126 is 2^-102
constexpr int kLeast = -176;        // e of a row without weights: any weight that comes leaves its range or keeps its bits
constexpr float kLimit = 0x1p94f;   // of a score's factors: scores stay below 2^126, codes' products being below 2^32
constexpr float kMost = 0x1.fffffep127f;  // of a weight's factor: never infinite, so that 0 stays 0
constexpr float kFine = 0x1p22f;    // of references: the exact product less one is what the rounded score is less it, to 2^-2
constexpr float kNone = -0x1p127f;  // reference of a row that has seen nothing

struct Args {
  PageAttn a;
  int tile_tokens;  // query tokens of an item
  int shift;        // log2 of the page
  int least_part;   // tokens of a part, at least
  float target;     // parts that fill the card
  float scale2;     // scale log2(e)
  int rows;         // query rows of an item, at most
  int cut;          // items may be cut
  int parts;        // at most
  int planned;      // the parts before each sequence are in the workspace
  uint32_t magic;   // ceil(2^16 / G): x / G = x magic >> 16 for the rows of an item
};

// ------------------------------------------------------------------- work --
struct Seq {
  int begin, rows, len;  // len 0 if bad
  bool bad, causal;
  int tiles;
};
// the same value in every lane, in a scalar register
__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Seq uni(const Seq& s) {
  return {uni(s.begin), uni(s.rows), uni(s.len), (bool)uni(s.bad), (bool)uni(s.causal), uni(s.tiles)};
}
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
};
// A part's tokens from all items' tokens: about as many parts as fill the card.
__device__ __forceinline__ int part_size(const Args& p, float tokens) {
  // (a little more than the exact quotient, so that rounding never makes a part too many)
  const float share = tokens * (float)p.a.H * 1.001f / p.target;
  return (max(p.least_part, (int)fminf(share, 1073741760.0f)) + 31) & ~31;
}
__device__ __forceinline__ int parts_of_item(const Seq& s, int part) {  // part 0: items are whole
  return part ? max(1, (int)((uint32_t)(s.len + part - 1) / (uint32_t)part)) : 1;
}
// parts before each of the sequences, their number, and a part's tokens
__device__ __forceinline__ int* plan_of(const Args& p);

// Part w of all, in every thread of the workgroup.  Parts are in the order of sequences,
// tiles from the last (a causal sequence's longest), parts, heads.  False: there is none.
__device__ __forceinline__ bool part_at(const Args& p, int w, Part* r, int* lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, W = blockDim.x >> 6;
  const int n = (int)p.a.n_seqs;
  const uint32_t H = (uint32_t)p.a.H;
  int g, first = 0, part = 0;
  if (!p.cut && !p.a.starts) {  // one item, one part for each sequence and head
    g = (int)((uint32_t)w / H);
    first = g * (int)H;
  } else if (p.planned) {  // the last sequence with at most w parts before it
    const int* before = plan_of(p);
    if (w >= before[n]) return false;
    part = before[n + 1];
    g = 0;
    for (int width = n; width > 1;) {
      const int step = (width + 63) >> 6, at = lane * step;
      const int to = __popcll(__ballot(at < width && before[min(g + at, n)] <= w)) - 1;
      g += to * step;
      width = min(step, width - to * step);
    }
    first = before[g];
  } else {
    Seq s = tid < n ? sequence(p, tid) : Seq{};
    if (p.cut) {
      float tokens = (float)s.tiles * (float)s.len;
      for (int at = tid + 64 * W; at < n; at += 64 * W) {
        const Seq more = sequence(p, at);
        tokens += (float)more.tiles * (float)more.len;
      }
      tokens = wave_sum(tokens);
      if (lane == 0) lds[wave] = __float_as_int(tokens);
      __syncthreads();
      tokens = 0.0f;
      for (int v = 0; v < W; ++v) tokens += __int_as_float(lds[v]);
      part = part_size(p, tokens);
      __syncthreads();
    }
    int* found = lds + W;  // sequence, parts before it
    int* sums = found + 2;
    if (tid == 0) found[0] = -1;
    int before = 0;
    for (int g0 = 0; g0 < n; g0 += 64 * W) {
      const int at = g0 + tid;
      if (g0 > 0) s = at < n ? sequence(p, at) : Seq{};
      const int mine = at < n ? s.tiles * parts_of_item(s, part) * p.a.H : 0;
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(upto, o, 64);
        if (lane >= o) upto += y;
      }
      if (lane == 63) sums[wave] = upto;
      __syncthreads();
      int all = 0;
      for (int v = 0; v < W; ++v) {
        if (v < wave) upto += sums[v];
        all += sums[v];
      }
      if (w < before + upto && w >= before + upto - mine) {
        found[0] = at;
        found[1] = before + upto - mine;
      }
      __syncthreads();
      before += all;
      if (w < before) break;
    }
    g = uni(found[0]);
    if (g < 0) return false;
    first = uni(found[1]);
    part = uni(part);
  }
  g = uni(g);
  const Seq s = uni(sequence(p, g));
  uint32_t i = (uint32_t)(w - first);
  r->s = s;
  r->g = g;
  r->parts = parts_of_item(s, part);
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
constexpr int part_lds(int W) { return 2 * W + 2; }

// ---------------------------------------------------------------- records --
// A state of an item's rows: references, sums, exponents, and accumulators [rows][D].
__host__ __device__ constexpr int state_head(int rows) { return (3 * rows + 3) & ~3; }
__host__ __device__ constexpr int state_floats(int rows, int d) { return state_head(rows) + rows * d; }
template <int D>
struct State {
  float* at;
  int rows;
  __device__ __forceinline__ float& ref(int r) const { return at[r]; }
  __device__ __forceinline__ float& sum(int r) const { return at[rows + r]; }
  __device__ __forceinline__ float& exp(int r) const { return at[2 * rows + r]; }
  __device__ __forceinline__ float* acc(int r) const { return at + state_head(rows) + r * D; }
};
template <int D>
__device__ __forceinline__ State<D> state(void* base, int64_t i, int rows) {
  return {(float*)base + i * state_floats(rows, D), rows};
}

// What the second launch joins, one for each part: the parts of the item that begins
// there if it was cut (else 0), its rows, its first query row and its head.
struct Join {
  int parts, n_rows, row, h;
};
__device__ __forceinline__ Join* joins(const Args& p, int d) {
  return (Join*)((float*)p.a.ws + (int64_t)p.parts * state_floats(p.rows, d));
}

__device__ __forceinline__ int* plan_of(const Args& p) {
  return p.cut ? (int*)(joins(p, p.a.d) + p.parts) : (int*)p.a.ws;
}

// The parts before every sequence, once for all workgroups where each would take longer to
// sum them up itself: above 512 sequences (tables of 16384 tokens; 64 sequences to 2048
// tokens 17.9 us without and 20.3 with this launch, 512 to 1000 44.7 and 45.0, 2048 to 500
// 78.6 and 56.1).
constexpr int kPlanned = 512;
__global__ __launch_bounds__(1024) void plan_kernel(Args p) {
  __shared__ float tokens_of[16];
  __shared__ uint32_t sums[2][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = (int)p.a.n_seqs;
  int* before = plan_of(p);
  float tokens = 0.0f;
  if (p.cut) {
    for (int g = tid; g < n; g += 1024) {
      const Seq s = sequence(p, g);
      tokens += (float)s.tiles * (float)s.len;
    }
    tokens = wave_sum(tokens);
    if (lane == 0) tokens_of[wave] = tokens;
    __syncthreads();
    tokens = 0.0f;
#pragma unroll
    for (int v = 0; v < 16; ++v) tokens += tokens_of[v];
  }
  const int part = p.cut ? part_size(p, tokens) : 0;
  auto plus = [](uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); };
  uint32_t all = 0;
  for (int g0 = 0, round = 0; g0 < n; g0 += 1024, round ^= 1) {
    const int g = g0 + tid;
    const Seq s = g < n ? sequence(p, g) : Seq{};
    uint32_t upto = g < n ? (uint32_t)(s.tiles * parts_of_item(s, part) * p.a.H) : 0;
    const uint32_t mine = upto;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(upto, o, 64);
      if (lane >= o) upto = plus(upto, y);
    }
    if (lane == 63) sums[round][wave] = upto;
    __syncthreads();
    uint32_t here = all;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      if (v < wave) here = plus(here, sums[round][v]);
      all = plus(all, sums[round][v]);
    }
    if (g < n) before[g] = (int)(plus(here, upto) - mine);
  }
  if (tid == 0) before[n] = (int)all, before[n + 1] = part;
}

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

// A pair of weights' leading 8 bits as bfloat16, cut off and taken from them (exact).
__device__ __forceinline__ uint32_t leading(float* x, float* y) {
  const uint32_t a = __float_as_uint(*x), b = __float_as_uint(*y);
  *x -= __uint_as_float(a & 0xffff0000u);
  *y -= __uint_as_float(b & 0xffff0000u);
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
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

  static constexpr bool kShared = R > 1;             // queries in LDS, for all wavefronts

  h8 q[kShared ? 1 : R][2 * KJ][QP];
  const h8* lq;                  // [R][2 KJ][QP][64]
  int qe[R];                     // a row's queries are q 2^qe
  int vis[R];                    // tokens that a row sees
  float ref[R], sum[R], top[R];  // top: largest weight so far, in units of 2^e
  int e[R];
  f4 acc[R][CB];
  bool lost[R];  // queries that are no numbers
  float base[R];  // the reference, or kNone from kFine on: each tile's weights leave their range then

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

  Half t[2];

  const Args& p;
  const int lane, row16, group;
  int g;
  int h;
  int pages;  // of the sequence

  __device__ __forceinline__ explicit Wave(const Args& p_)
      : p(p_), lane(threadIdx.x & 63), row16(lane & 15), group(lane >> 4) {}

  // Ids of the 64 pages from `first` on, one a lane (-1 behind the last), and their scales.
  __device__ __forceinline__ int page_of(int first) {
    page0 = first;
    const int at = first + lane;
    return at < pages ? p.a.table[(int64_t)g * p.a.max_pages + at] : -1;
  }
  __device__ __forceinline__ void scales_of(int ids) {
    const PageAttn& a = p.a;
    const bool known = ids >= 0 && ids < a.n_pages;
    id = known ? ids : 0;
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

  // Row rr's queries and which of the item's tokens it belongs to (the first row's, if the
  // item has no such row).
  __device__ __forceinline__ const T* row_of(const Part& r, int rr, int* i) const {
    const PageAttn& a = p.a;
    const bool used = rr < r.n_tokens * a.G;
    *i = used ? (int)((uint32_t)rr * p.magic >> 16) : 0;
    const int hq = used ? rr - *i * a.G : 0;
    return (const T*)a.q + (((int64_t)(r.s.begin + r.i0 + *i) * a.H + r.h) * a.G + hq) * D;
  }
  // x 2^-e in QP binary16 parts
  __device__ __forceinline__ void parts_of(const T* y, bool used, int e, h8* to) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float z = used ? ldexpf(to_float(y[i]), -e) : 0.0f;
      to[0][i] = (_Float16)z;
      if constexpr (QP == 2) to[1][i] = (_Float16)(z - (float)to[0][i]);
    }
  }
  __device__ __forceinline__ void look(const T* y, float* big, int* lost_) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float z = fabsf(to_float(y[i]));
      *lost_ |= !(z < INFINITY);
      *big = fmaxf(*big, z);
    }
  }
  // the largest is in [2^14, 2^15) then
  __device__ __forceinline__ int exponent(float big, int lost_) const {
    return (big > 0.0f && !lost_ ? __builtin_amdgcn_frexp_expf(big) : 0) - 15;
  }

  // Queries of the item into LDS as the operand that each lane takes, 8 threads to a row.
  // Behind them the rows' exponents and whether they are no numbers.
  __device__ __forceinline__ void share_queries(const Part& r, h8* to) {
    for (int rr = threadIdx.x >> 3; rr < 16 * R; rr += blockDim.x >> 3) share_row(r, rr, to);
  }
  __device__ __forceinline__ void share_row(const Part& r, int rr, h8* to) {
    const int s = threadIdx.x & 7;
    int i;
    const T* x = row_of(r, rr, &i) + s * KJ * 8;
    T y[KJ][8];
    float big = 0.0f;
    int l = 0;
#pragma unroll
    for (int m = 0; m < KJ; ++m) __builtin_memcpy(y[m], x + m * 8, sizeof(y[m]));
#pragma unroll
    for (int m = 0; m < KJ; ++m) look(y[m], &big, &l);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
      big = fmaxf(big, __shfl_xor(big, o, 64));
      l |= __shfl_xor(l, o, 64);
    }
    const int e = exponent(big, l);
    const bool used = rr < r.n_tokens * p.a.G && !l;
#pragma unroll
    for (int m = 0; m < KJ; ++m) {
      const int d8 = s * KJ + m, j = d8 >> 3, kg = (d8 & 7) >> 1;
      h8 part[QP];
      parts_of(y[m], used, e, part);
#pragma unroll
      for (int u = 0; u < QP; ++u)
        to[(((rr >> 4) * 2 * KJ + 2 * j + (d8 & 1)) * QP + u) * 64 + kg * 16 + (rr & 15)] = part[u];
    }
    int* rows = (int*)(to + R * 2 * KJ * QP * 64);
    if (s == 0) rows[rr] = e, rows[16 * R + rr] = l;
  }

  // The part's first loads, each as soon as its address is known, then its queries.
  __device__ __forceinline__ void begin(const Part& r, int from, int to, const h8* shared) {
    g = r.g;
    h = r.h;
    pages = (r.s.len + (1 << p.shift) - 1) >> p.shift;
    const int first = page_of(from >> p.shift);
    const int n_rows = r.n_tokens * p.a.G;
    T y[kShared ? 1 : 2 * KJ][8];
#pragma unroll
    for (int s = 0; s < R; ++s) {
      int i;
      const T* x = row_of(r, s * 16 + row16, &i);
      vis[s] = s * 16 + row16 >= n_rows ? 0 : r.s.causal ? r.s.len - r.s.rows + r.i0 + i + 1 : r.s.len;
      if constexpr (!kShared)
#pragma unroll
        for (int c = 0; c < 2 * KJ; ++c)
          __builtin_memcpy(y[c], x + (c / 2) * 64 + group * 16 + (c % 2) * 8, sizeof(y[c]));
    }
    scales_of(first);
    t[0] = half(from);
    t[1] = half(min(from + 16, to - 1) & ~15);
    load_k(t);
    load_v(t);
    if constexpr (kShared) {
      lq = shared + lane;
      const int* rows = (const int*)(shared + R * 2 * KJ * QP * 64);
#pragma unroll
      for (int s = 0; s < R; ++s) {
        qe[s] = rows[s * 16 + row16];
        lost[s] = rows[16 * R + s * 16 + row16];
      }
    } else {
      float big = 0.0f;
      int l = 0;
#pragma unroll
      for (int c = 0; c < 2 * KJ; ++c) look(y[c], &big, &l);
      big = fmaxf(big, __shfl_xor(big, 16, 64));
      big = fmaxf(big, __shfl_xor(big, 32, 64));
      l |= __shfl_xor(l, 16, 64);
      l |= __shfl_xor(l, 32, 64);
      lost[0] = l;
      qe[0] = exponent(big, l);
#pragma unroll
      for (int c = 0; c < 2 * KJ; ++c) parts_of(y[c], row16 < n_rows && !l, qe[0], q[0][c]);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int s = 0; s < R; ++s) {
      ref[s] = kNone;
      sum[s] = 0.0f;
      top[s] = 0.0f;
      e[s] = kLeast;
      lost[s] = false;
      base[s] = kNone;
#pragma unroll
      for (int c = 0; c < CB; ++c) acc[s][c] = f4{0, 0, 0, 0};
    }
  }

  // A row's reference becomes its largest score, and its weights' exponent that of the
  // largest weight.  b0, b1: the lane's largest scores in the two halves of the tile.
  __device__ __forceinline__ void move(int r, float b0, float b1, float v0, float v1) {
    float big[2] = {b0, b1};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      big[u] = fmaxf(big[u], __shfl_xor(big[u], 16, 64));
      big[u] = fmaxf(big[u], __shfl_xor(big[u], 32, 64));
    }
    const float to = fmaxf(ref[r], fmaxf(big[0], big[1]));
    const float a = exp2_(ref[r] - to);
    float w = fmaxf(top[r], __shfl_xor(top[r], 16, 64));
    w = fmaxf(w, __shfl_xor(w, 32, 64));
    w = ldexpf(w * a, e[r]);
    w = fmaxf(w, fmaxf(exp2_(big[0] - to) * fabsf(v0), exp2_(big[1] - to) * fabsf(v1)));
    // (no weight but zeros so far, as of pages of zeros: the first one sets e)
    const int ew = w > 0.0f ? max(__builtin_amdgcn_frexp_expf(w) - 1 - kTopBits, kLeast) : kLeast;
    const float by = ldexpf(a, e[r] - ew);
    sum[r] *= a;
    top[r] = ldexpf(w, -ew);
    ref[r] = to;
    base[r] = fabsf(to) < kFine ? to : kNone;
    e[r] = ew;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float b = __shfl(by, group * 4 + i, 64);
#pragma unroll
      for (int c = 0; c < CB; ++c) acc[r][c][i] *= b;
    }
  }

  // A score in units of a row's reference, rounded by itself: a row whose scores lie far
  // from 0 has to take off its reference from what that was taken from.  (Behind the branch
  // that needs it.)
  __device__ __forceinline__ float score(float s, float f) const {
    asm volatile("" : "+v"(s));
    float x = s * f;
    asm volatile("" : "+v"(x));
    return x;
  }
  // Tokens [from, to) of the item, from a multiple of 32.
  __device__ __forceinline__ void run(const Part& r_, int from, int to) {
    const int last = (to - 1) & ~31;
    const int least = r_.s.causal ? r_.s.len - r_.s.rows + r_.i0 + 1 : r_.s.len, most = r_.seen;
    for (int t0 = from; t0 < to; t0 += 32) {
      f4 s[R][2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < R; ++r) s[r][u] = f4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < KJ; ++j) {
        h8 x[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          x[u][0] = halves<CODES>(k[u][j].x, k[u][j].y);
          x[u][1] = halves<CODES>(k[u][j].z, k[u][j].w);
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int i = QP - 1; i >= 0; --i)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const h8 y = kShared ? lq[((r * 2 * KJ + 2 * j + c) * QP + i) * 64] : q[kShared ? 0 : r][2 * j + c][i];
#pragma unroll
              for (int u = 0; u < 2; ++u)
                s[r][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[u][c], y, s[r][u], 0, 0, 0);
            }
      }
      // The next tile's keys are on their way from here on, its values from the end.  (The
      // last tile's own again: a branch around the loads would make each wait one for all.)
      const float ks[2] = {t[0].ks, t[1].ks}, vs[2] = {t[0].vs, t[1].vs};
      const bool lost_page[2] = {t[0].bad, t[1].bad};
      const int next = min(t0 + 32, last);
      if ((next >> p.shift) - page0 >= 63) scales_of(page_of(next >> p.shift));
      t[0] = half(next);
      t[1] = half(min(next + 16, to - 1) & ~15);
      load_k(t);
      const bool masked = t0 + 32 > least || lost_page[0] || lost_page[1];
      uint4 parts[R][3];  // of weights: pairs of tokens
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float f[2] = {limited(ldexpf(ks[0], qe[r])), limited(ldexpf(ks[1], qe[r]))};
        float w[8], more, largest;
        auto hide = [&](float* x) {  // what a row does not see, and what is no number
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (lost_page[i / 4]) x[i] = NAN;
            if (t0 + (i / 4) * 16 + group * 4 + i % 4 >= vis[r]) x[i] = -INFINITY;
          }
        };
        // Whether all weights are in their range.  (A factor c0 beyond its type belongs to
        // exponentials of 0, or to weights out of range; behind a move, to exponentials of
        // less than 2^-75 that weigh most: those take 2^64 of it.)
        auto weigh = [&](bool moved) {
          float x[8], top_p[2];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            x[i] = __builtin_fmaf(s[r][i / 4][i % 4], f[i / 4], moved ? -ref[r] : -base[r]);
          if (moved && __any(base[r] != ref[r])) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float y = score(s[r][i / 4][i % 4], f[i / 4]) - ref[r];
              x[i] = base[r] != ref[r] ? y : x[i];
            }
          }
          if (masked) hide(x);
          more = 0.0f;
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float c0 = ldexpf(vs[u], -e[r]);
            const int up = moved && !(fabsf(c0) < 0x1p100f) ? 64 : 0;
            const float c = __builtin_amdgcn_fmed3f(moved ? ldexpf(vs[u], -e[r] - up) : c0, -kMost, kMost);
            top_p[u] = 0.0f;
#pragma unroll
            for (int i = 4 * u; i < 4 * u + 4; ++i) {
              x[i] = exp2_(x[i]);
              top_p[u] = fmaxf(top_p[u], x[i]);
              more += x[i];
              w[i] = (moved ? ldexpf(x[i], up) : x[i]) * c;
            }
            const float most_w = moved ? ldexpf(top_p[u], up) * fabsf(c) : top_p[u] * fabsf(c0);
            largest = u ? fmaxf(largest, most_w) : most_w;
          }
          return !__any(fmaxf(top_p[0], top_p[1]) > kLag || largest >= kTop);
        };
        if (!weigh(false)) {
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = score(s[r][i / 4][i % 4], f[i / 4]);
          if (masked) hide(x);
          move(r, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
               fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])), vs[0], vs[1]);
          weigh(true);
        }
        sum[r] += more;
        top[r] = fmaxf(top[r], largest);
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          parts[r][i].x = leading(&w[0], &w[1]);
          parts[r][i].y = leading(&w[2], &w[3]);
          parts[r][i].z = leading(&w[4], &w[5]);
          parts[r][i].w = leading(&w[6], &w[7]);
        }
      }
      // What lies behind the last token, or is read in an unknown page's place, may hold anything.
      if (t0 + 32 > most || lost_page[0] || lost_page[1]) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (lost_page[i / 4] || t0 + (i / 4) * 16 + group * 4 + i % 4 >= most)
#pragma unroll
            for (int c = 0; c < CB / 4; ++c) v[i][c] = 0;
      }
#pragma unroll
      for (int c = 0; c < CB / 4; ++c)
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const b8 x = column(c, n);
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 2; i >= 0; --i)
              acc[r][4 * c + n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, parts[r][i]), x,
                                                                          acc[r][4 * c + n], 0, 0, 0);
        }
      load_v(t);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      sum[r] += __shfl_xor(sum[r], 16, 64);
      sum[r] += __shfl_xor(sum[r], 32, 64);
    }
  }
  // The 8 tokens' codes of column 4 c + n of the lane's.
  __device__ __forceinline__ b8 column(int c, int n) const {
    uint4 x;
    uint32_t* w = (uint32_t*)&x;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      if constexpr (CODES == FIBQ_E4M3) {
        // columns 4 c + 2 m and the next: pairs of tokens side by side
        const uint32_t two = __builtin_amdgcn_perm(v[i + 1][c], v[i][c], n & 2 ? 0x07030602u : 0x05010400u);
        const b2 y = n & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(two, 1.0f, true)
                           : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(two, 1.0f, false);
        w[i / 2] = __builtin_bit_cast(uint32_t, y);
      } else {
        const float lo = (float)(int8_t)(v[i][c] >> (8 * n)), hi = (float)(int8_t)(v[i + 1][c] >> (8 * n));
        w[i / 2] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
      }
    }
    return __builtin_bit_cast(b8, x);
  }

  // The results of an item that one wavefront has whole.
  __device__ __forceinline__ void finish(const Part& part) const {
    const PageAttn& a = p.a;
    const int n_rows = part.n_tokens * a.G;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float all = lost[r] && sum[r] > 0.0f ? NAN : sum[r];
      const float over = part.s.bad ? NAN : all == 0.0f ? 0.0f : 1.0f / all;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int rr = r * 16 + group * 4 + i;
        const float by = __shfl(over, group * 4 + i, 64);
        const int ex = __shfl(e[r], group * 4 + i, 64);
        if (rr >= n_rows) continue;
        const int token = (int)((uint32_t)rr * p.magic >> 16), hq = rr - token * a.G;
        float* out = a.out +
                     (((int64_t)(part.s.begin + part.i0 + token) * a.H + part.h) * a.G + hq) * D +
                     row16 * CB;
#pragma unroll
        for (int c = 0; c < CB; c += 4) {
          const f4 x{ldexpf(acc[r][c][i] * by, ex), ldexpf(acc[r][c + 1][i] * by, ex),
                     ldexpf(acc[r][c + 2][i] * by, ex), ldexpf(acc[r][c + 3][i] * by, ex)};
          __builtin_memcpy(out + c, &x, 16);  // (any alignment)
        }
      }
    }
  }
  // rows 16 r .. 16 r + 15
  __device__ __forceinline__ void store(int r, const State<D>& to) const {
    if (group == 0 && row16 < to.rows) {
      to.ref(row16) = ref[r];
      to.sum(row16) = lost[r] && sum[r] > 0.0f ? NAN : sum[r];
      to.exp(row16) = (float)e[r];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int rr = group * 4 + i;
      if (rr >= to.rows) break;
#pragma unroll
      for (int c = 0; c < CB; c += 4)
        *(f4*)(to.acc(rr) + row16 * CB + c) =
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


// 16 rows of an item from the W <= 8 states of the workgroup's wavefronts: the result, or
// the part's state.  A lane has one row's statistics in states lane / 16 and 4 more; the
// wavefronts take a row each then.
template <int D>
__device__ __forceinline__ void finish_rows(const Args& p, const Part& r, int row0, int n_rows,
                                            const State<D>& states, const State<D>& record, int W,
                                            int wave, int lane) {
  constexpr int kPer = D / 64;  // columns of a lane
  const int mine = min(lane & 15, states.rows - 1);
  float ref[2], exp[2], sum[2], f[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int v = (lane >> 4) + 4 * u;
    const State<D> x = state<D>(states.at, min(v, W - 1), states.rows);
    ref[u] = v < W ? x.ref(mine) : kNone;
    exp[u] = x.exp(mine);
    sum[u] = x.sum(mine);
  }
  Joined j{fmaxf(ref[0], ref[1]), -0x1p30f};
  j.ref = fmaxf(j.ref, __shfl_xor(j.ref, 16, 64));
  j.ref = fmaxf(j.ref, __shfl_xor(j.ref, 32, 64));
  float all = 0.0f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    if (ref[u] > kNone) j.exp = fmaxf(j.exp, ceilf(ref[u] - j.ref) + exp[u]);
    all += (lane >> 4) + 4 * u < W ? sum[u] * exp2_(ref[u] - j.ref) : 0.0f;
  }
  j.exp = fmaxf(j.exp, __shfl_xor(j.exp, 16, 64));
  j.exp = fmaxf(j.exp, __shfl_xor(j.exp, 32, 64));
  all += __shfl_xor(all, 16, 64);
  all += __shfl_xor(all, 32, 64);
#pragma unroll
  for (int u = 0; u < 2; ++u) f[u] = factor(ref[u], exp[u], j);
  const float over = r.s.bad ? NAN : all == 0.0f ? 0.0f : 1.0f / all;
  auto of = [&](float x, int l) {  // lane l's x
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), l));
  };
  for (int rr16 = wave; rr16 < n_rows; rr16 += W) {
    float acc[kPer];
#pragma unroll
    for (int c = 0; c < kPer; ++c) acc[c] = 0.0f;
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      if (v >= W) break;
      const float fv = of(f[v / 4], rr16 + 16 * (v % 4));
      const float* x = state<D>(states.at, v, states.rows).acc(rr16) + lane * kPer;
#pragma unroll
      for (int c = 0; c < kPer; ++c) acc[c] += x[c] * fv;
    }
    const int rr = row0 + rr16, e = (int)of(j.exp, rr16);
    if (r.parts == 1) {
      const float by = of(over, rr16);
      const int i = (int)((uint32_t)rr * p.magic >> 16), hq = rr - i * p.a.G;
      float* out = p.a.out +
                   (((int64_t)(r.s.begin + r.i0 + i) * p.a.H + r.h) * p.a.G + hq) * D + lane * kPer;
#pragma unroll
      for (int c = 0; c < kPer; ++c) out[c] = ldexpf(acc[c] * by, e);
    } else {
      if (lane == 0) {
        record.ref(rr) = of(j.ref, rr16);
        record.sum(rr) = of(all, rr16);
        record.exp(rr) = of(j.exp, rr16);
      }
#pragma unroll
      for (int c = 0; c < kPer; ++c) record.acc(rr)[lane * kPer + c] = acc[c];
    }
  }
}

// Wavefronts that a SIMD holds at once, by registers.
__host__ __device__ constexpr int waves_of_simd(int R, int D) {
  return R == 1 ? (D == 64 ? 4 : D == 128 ? 3 : 2) : D == 64 ? 3 : D == 128 ? 2 : 1;
}

// Wavefronts of a workgroup, at most.
__host__ __device__ constexpr int most_waves(int R, int D) {
  return R == 1 && D == 64 ? 8 : 4;
}

template <typename T, int CODES, int D, int R>
__global__ __launch_bounds__(64 * most_waves(R, D), waves_of_simd(R, D))
void main_kernel(Args p) {
  extern __shared__ __align__(16) float states[];
  const int lane = threadIdx.x & 63, W = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Part r{};
  const bool live = part_at(p, blockIdx.x, &r, (int*)states);
  if (p.cut && threadIdx.x == 0)
    joins(p, D)[blockIdx.x] = Join{live && r.part == 0 && r.parts > 1 ? r.parts : 0, r.n_tokens * p.a.G,
                                   r.s.begin + r.i0, r.h};
  if (!live) return;
  Wave<T, CODES, D, R> wv(p);
  const int tiles = (r.to - r.from + 31) >> 5, each = (int)((uint32_t)(tiles + W - 1) / (uint32_t)W);
  const int from = r.from + min(tiles, wave * each) * 32;
  const int to = min(r.to, r.from + min(tiles, (wave + 1) * each) * 32);
  wv.clear();
  h8* queries = (h8*)(states + 64);  // (behind part_at's words)
  if constexpr (R > 1) {
    wv.share_queries(r, queries);
    __syncthreads();
  }
  if (from < to) {
    wv.begin(r, from, to, queries);
    wv.run(r, from, to);
  }
  if (W == 1 && r.parts == 1) {
    wv.finish(r);
    return;
  }
  const State<D> record = state<D>(p.a.ws, blockIdx.x, p.rows);
  const int n_rows = r.n_tokens * p.a.G, rows16 = min(p.rows, 16);
#pragma unroll
  for (int group = 0; group < R; ++group) {
    __syncthreads();  // (what was in LDS has been read)
    wv.store(group, state<D>(states, wave, rows16));
    __syncthreads();
    finish_rows<D>(p, r, 16 * group, min(16, n_rows - 16 * group), state<D>(states, 0, rows16),
                   record, W, wave, lane);
  }
}

// Joins the states of the items that were cut: a wavefront for each row or, where items
// have few rows and many parts, four (WIDE).  What it reads has just been written by
// other XCDs, so each read takes long: many are on their way at once.  Bound by that chain
// (list, headers, values) and its launch: 7.0 us for 192 items to 32768 tokens, 4.8 for 8 of
// 131072, d = 128.
template <int D, int WIDE>
__global__ __launch_bounds__(256) void merge_kernel(Args p) {
  constexpr int kPer = D / 64, kBatch = 8;
  __shared__ float joined[4][3 + D];
  const int lane = threadIdx.x & 63;
  const int wave = uni((int)(threadIdx.x >> 6)), mine = WIDE > 1 ? wave : 0;
  const Join* list = joins(p, D);
  for (int w0 = blockIdx.x; w0 < p.parts; w0 += 64 * gridDim.x) {
    const int wl = w0 + lane * gridDim.x;
    uint64_t todo = __ballot(wl < p.parts && list[min(wl, p.parts - 1)].parts > 0);
    for (; todo; todo &= todo - 1) {
      const int w = w0 + (__ffsll((unsigned long long)todo) - 1) * gridDim.x;
      // (no record behind the last one is read, whatever became of the lengths meanwhile)
      const int parts = min(uni(list[w].parts), (p.parts - 1 - w) / p.a.H + 1), n_rows = uni(list[w].n_rows), row = uni(list[w].row),
                h = uni(list[w].h);
      const int rows_apart = gridDim.y * (4 / WIDE);
      for (int rr = blockIdx.y * (4 / WIDE) + (WIDE > 1 ? 0 : wave); rr < n_rows; rr += rows_apart) {
        Joined j{kNone, -0x1p30f};
        float sum = 0.0f, acc[kPer];
#pragma unroll
        for (int c = 0; c < kPer; ++c) acc[c] = 0.0f;
        // parts of this wavefront: mine, mine + WIDE, ..., kBatch at a time
        for (int i0 = mine; i0 < parts; i0 += WIDE * kBatch) {
          float x[kBatch][kPer];
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            const int i = min(i0 + b * WIDE, parts - 1);
            const State<D> s = state<D>(p.a.ws, w + (int64_t)i * p.a.H, p.rows);
#pragma unroll
            for (int c = 0; c < kPer; ++c) x[b][c] = s.acc(rr)[lane * kPer + c];
          }
          const int i = i0 + lane % kBatch * WIDE;
          const State<D> s = state<D>(p.a.ws, w + (int64_t)min(i, parts - 1) * p.a.H, p.rows);
          const float ref = i < parts ? s.ref(rr) : kNone, exp = s.exp(rr), all = s.sum(rr);
          const Joined old = j;
          j.ref = fmaxf(j.ref, wave_max(ref));
          j.exp = wave_max(fmaxf(ref > kNone ? ceilf(ref - j.ref) + exp : -0x1p30f,
                                 old.ref > kNone ? ceilf(old.ref - j.ref) + old.exp : -0x1p30f));
          const float f = factor(ref, exp, j), f0 = factor(old.ref, old.exp, j);
          sum = sum * exp2_(old.ref - j.ref) +
                wave_sum(lane < kBatch && i < parts ? all * exp2_(ref - j.ref) : 0.0f);
#pragma unroll
          for (int c = 0; c < kPer; ++c) acc[c] *= f0;
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            const float fb = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), b));
#pragma unroll
            for (int c = 0; c < kPer; ++c) acc[c] += x[b][c] * fb;
          }
        }
        if (WIDE > 1) {
          __syncthreads();  // (the row before has been read)
          if (lane == 0) joined[wave][0] = j.ref, joined[wave][1] = j.exp, joined[wave][2] = sum;
#pragma unroll
          for (int c = 0; c < kPer; ++c) joined[wave][3 + lane * kPer + c] = acc[c];
          __syncthreads();
          if (wave != 0) continue;
          float top = -0x1p30f;
#pragma unroll
          for (int v = 1; v < 4; ++v) j.ref = fmaxf(j.ref, joined[v][0]);
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (joined[v][0] > kNone) top = fmaxf(top, ceilf(joined[v][0] - j.ref) + joined[v][1]);
          j.exp = top;
          sum = 0.0f;
#pragma unroll
          for (int c = 0; c < kPer; ++c) acc[c] = 0.0f;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const float f = factor(joined[v][0], joined[v][1], j);
            sum += joined[v][2] * exp2_(joined[v][0] - j.ref);
#pragma unroll
            for (int c = 0; c < kPer; ++c) acc[c] += joined[v][3 + lane * kPer + c] * f;
          }
        }
        const int i = (int)((uint32_t)rr * p.magic >> 16), hq = rr - i * p.a.G;
        float* out = p.a.out + (((int64_t)(row + i) * p.a.H + h) * p.a.G + hq) * D + lane * kPer;
#pragma unroll
        for (int c = 0; c < kPer; ++c) out[c] = finished(acc[c], sum, j.exp);
      }
    }
  }
}

// ---------------------------------------------------------------- dispatch --
constexpr int kCu = 256;

struct Plan {
  int R, rows, waves;   // row tiles of 16 R; rows of an item, at most; wavefronts of a workgroup
  int parts, joins;     // parts, at most; workgroups that join
  int least;            // tokens of a part, at least
  float target;
  bool cut, planned;
  size_t bytes;
};
// What the host knows: sizes, and how long sequences may be (`room`), not how long they
// are.  Times below are in us, e4m3 codes, bfloat16 queries, G = 8 (d = 64) or 4 (128).
Plan plan(int64_t n_seqs, int64_t n_rows, bool one, int H, int G, int64_t max_pages, int page, int d) {
  Plan p{};
  // Tiles of 32 rows where a sequence has more than 16 (64 sequences of 2048 tokens x 4
  // heads, d = 64; rows of a head, then with 16-row and with 32-row tiles: 16 17.6 and
  // 25.5, 24 26.8 and 26.2, 32 27.0 and 27.1, 64 39.1 and 35.8; d = 128: 30.5 and 34.0,
  // 45.8 and 35.5, 46.5 and 36.3, 62.6 and 53.7).
  p.R = n_rows * G >= 24 * std::max<int64_t>(1, n_seqs) ? 2 : 1;
  const int64_t room = max_pages * page, tile = 16 * p.R / G;
  p.rows = one ? G : (int)tile * G;
  const int64_t items = (one ? n_rows : n_rows / tile + std::min(n_seqs, n_rows)) * H;
  // Items are cut only where they may be long or are few, since cutting costs a sum over
  // the lengths in every workgroup and a launch (whole and cut: 4 items to 2048 tokens
  // 12.5 and 13.5, to 4096 19.8 and 13.6; 64 to 2048 13.2 and 15.1, to 4096 20.6 and 16.3;
  // 256 to 4096 20.9 and 28.9, to 8192 38.7 and 43.7, to 16384 73.3 and 75.8).
  p.cut = room > (items >= kCu ? 8192 : 2048);
  // wavefronts that a compute unit holds at once
  const int64_t held = 4 * waves_of_simd(p.R, d);
  // Workgroups for each compute unit: all parts run at once, and each compute unit has as
  // many.  An item's last part is half empty on the average, so half as many parts as
  // items are kept back, and k grows with the items to keep that small (192 items to
  // 32768 tokens, 1, 2 and 3 for a compute unit: 146, 96 and 97; 8 items of 131072, d = 128: 56.6, 60.1 and 61.8.)
  int64_t k = std::min<int64_t>(4, (items + kCu / 2 - 1) / (kCu / 2));
  int64_t target = k * kCu - items / 2;
  if (target < kCu / 2) target = kCu;  // (items enough: only those far above the average are cut)
  if (p.R == 2) target = kCu * held / 4;
  // Wavefronts: as many to a workgroup as keep a compute unit's places filled by its
  // items (64 sequences to 2048 tokens x 4 heads, 2, 4 and 8: 26.3, 15.5 and 13.7; 8
  // items of 131072 tokens, d = 128, 2 and 4: 71.6 and 56.6); one for row tiles that fill
  // the card by themselves, whose states then need no joining (4 prompts of 1000 tokens x 4
  // heads, 1, 2 and 4: 82.5, 84.8 and 96.7; 8 chunks to 512 tokens over up to 4096, d = 128:
  // 191, 200 and 170; cross attention of 48 rows over 1500 tokens: 58, 38 and 23).
  p.waves = most_waves(p.R, d);
  if (p.R == 1)
    while (p.waves > 2 && (p.cut ? k : (items + kCu - 1) / kCu) * p.waves > held) p.waves /= 2;
  else if (!p.cut && (2 * items >= 3 * kCu * held || (2 * items >= kCu * held && room <= 1024)))
    p.waves = 1;
  p.least = !p.cut ? (int)std::max<int64_t>(room, 32) : items >= kCu ? 2048 : items >= kCu / 2 ? 1024 : 512;
  p.target = (float)target;
  p.parts = (int)(items + (p.cut ? target : 0));
  while (p.waves > 1 && (int64_t)p.parts * p.waves >= 1 << 26) p.waves /= 2;  // (a grid's 2^32 threads)
  // (a prime number of them: first parts lie at regular distances in the list)
  p.joins = std::min(p.parts, p.R == 1 ? 251 : 509);
  p.planned = n_seqs > kPlanned && (p.cut || !one);
  p.bytes = p.cut ? (size_t)p.parts * (state_floats(p.rows, d) * 4 + sizeof(Join)) : 0;
  if (p.planned) p.bytes += (size_t)(n_seqs + 2) * 4;
  return p;
}

template <typename T, int CODES, int D, int R>
int launch(const Args& p, const Plan& pl, hipStream_t st) {
  const size_t words = std::max((size_t)pl.waves * state_floats(std::min(pl.rows, 16), D), (size_t)part_lds(pl.waves)) * 4;
  const size_t lds = R == 1 ? words : std::max(words, 256 + (size_t)R * D * (sizeof(T) == 4 ? 64 : 32) + 128 * R);
  int rc = 0;
  if (pl.planned) {
    plan_kernel<<<1, 1024, 0, st>>>(p);
    if ((rc = (int)hipGetLastError()) != 0) return rc;
  }
  main_kernel<T, CODES, D, R><<<pl.parts, 64 * pl.waves, lds, st>>>(p);
  rc = (int)hipGetLastError();
  if (rc != 0 || !pl.cut) return rc;
  constexpr int kWide = R == 1 ? 4 : 1;
  merge_kernel<D, kWide><<<dim3(pl.joins, kWide > 1 ? pl.rows : 1), 256, 0, st>>>(p);
  return (int)hipGetLastError();
}
template <typename T, int CODES>
int launch_d(const Args& p, const Plan& pl, hipStream_t st) {
  switch (p.a.d) {
    case 64:
      return pl.R == 1 ? launch<T, CODES, 64, 1>(p, pl, st) : launch<T, CODES, 64, 2>(p, pl, st);
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
  // (as many as the call needs with starts or without)
  size_t most = pa::plan(n_seqs, n_rows, false, H, G, max_pages, page, d).bytes;
  if (n_seqs == n_rows)
    most = std::max(most, pa::plan(n_seqs, n_rows, true, H, G, max_pages, page, d).bytes);
  return most;
}

int launch_page_attn(const PageAttn& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const pa::Plan pl = pa::plan(a.n_seqs, a.n_rows, !a.starts, a.H, a.G, a.max_pages, a.page, a.d);
  const pa::Args p{a,        16 * pl.R / a.G, __builtin_ctz(a.page),
                   pl.least, pl.target,       a.scale * 1.44269504088896341f,
                   pl.rows,  pl.cut,          pl.parts,
                   pl.planned,
                   (65536u + (uint32_t)a.G - 1) / (uint32_t)a.G};
  switch (a.q_dtype) {
    case FIBQ_F32: return pa::launch_codes<float>(p, pl, st);
    case FIBQ_F16: return pa::launch_codes<f16_t>(p, pl, st);
    default: return pa::launch_codes<bf16_t>(p, pl, st);
  }
}

}  // namespace dev
}  // namespace fibq
