// Attention of several query rows per group over the compressed cache, for
// sequences of different lengths: the rows of a tree of drafted tokens
// (fibq_attn_tree), and single-token rows whose softmax weights are added to
// an accumulator per cached token (fibq_attn_decode_accum).
//
// Mathematics.  In rotated space a score is nu_t <q~, c_(t)> with q~ = Pi q
// times scale * log2 e, the softmax is base 2, and the values are
// sum_t p_t nu_t c_(t), rotated back once per row.  q~ and the weights p nu are
// held as two binary16 parts (22 bits together) against the binary16 codewords:
// q~ at a power of two of its row, weights down to 2^-32 of their row's largest
// p nu (a smaller one is lost: at most 2^-33 of that, for each token).  A codebook
// that binary16 does not hold adds its residual rows' products with the high parts
// (packed queries: with both), which leaves out 2^-22 of a product.  Statistics and
// sums are float32.
//
// An item is (group, tile of 16 RT query rows); its work is cut into units of 32
// tokens.  The units of all items, in runs of 8 (one per wavefront of a
// workgroup), are split into equal contiguous ranges, one per workgroup.
// prep_kernel  rotates every item's queries and writes them as operands; one of
//   its blocks finds the ranges from the lengths, which are on the device.
// rows_kernel  goes over a range.  For each item that it meets, a workgroup keeps
//   the queries in registers, goes over the units, combines its wavefronts' states
//   in LDS and leaves one record (m, l, acc) in rotated space.  Per unit a
//   wavefront gathers the keys' and the values' codewords once for all row tiles:
//   scores  S[t][r] = K_hat[t][:] . q~[r][:]  (v_mfma_f32_16x16x32_f16, A = two
//           gathered 4-dim codeword rows per lane, B = the queries' high, then
//           low parts): lane l holds row l % 16 and tokens 4 (l / 16) + e of
//           both 16-token tiles,
//   values  acc[r][dims] += W[r][t] V_hat[t][dims]: those are the lane's K
//           slots of the A operand, so the weights need no exchange; B comes
//           from transposing LDS reads of codeword rows.
//   Up to 8 rows ("packed") share a product between their parts: columns h and
//   h + 8 of B are row h's high and low part, summed by one exchange in which
//   lane h keeps the first tile's tokens and lane h + 8 the second's; rows h and
//   h + 8 of the weights are row h's parts (against a tile of 16 rows: 352 groups of 8
//   rows, 32k tokens, k = 8, with the weights' pass 280 -> 180 us; 704 of 2048 tokens,
//   k = 4, 68 -> 54; 144 of one row 30 -> 27; 8 of 4 rows at d = 128 72 -> 66).
// merge_kernel combines an item's records by log-sum-exp and applies Pi^T.
// For accumulated weights rows_kernel then goes over the same ranges once more with
// the rows' statistics (m, l), recomputes the scores and adds the weights of a
// token, summed over the rows in a fixed order, to its accumulator: no atomics.
//
// What bounds them.  The work is far above the bytes (352 groups of 32k tokens at
// k = 8 hold 138 MB, 27 us at a large copy's rate): rows_kernel is bound by the
// vector instructions per unit with few rows (that cache, 8 rows: 119 us, 126
// instructions per unit, 71 % of all issue cycles; its weights' pass 77 us), and
// by vector and matrix instructions and by unequal ranges with many (16 groups of up
// to 512 rows, 32k tokens: 142 us, vector units 47 % and matrix units 25 % busy, compute
// units 73 %, since a range that meets six items costs more than one that meets five;
// the two-part products take 63 us at the rate of a large matrix product).  Small
// calls are three or four launches, 12 to 21 us.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "attn_rows4.h"
#include "device_common.h"
#include "fibq.h"
#include "fibq_internal.h"

namespace fibq {
namespace dev {
namespace sv {

constexpr int kWaves = 8;              // wavefronts per workgroup
constexpr int kThreads = 64 * kWaves;
constexpr int kStep = 32;              // tokens per unit
constexpr int kRun = kStep * kWaves;   // tokens per run of units
constexpr int kTop = 64;               // partial maxima of a codebook
constexpr int kMaxWgs = 512;           // workgroups of the main launch, at most
// A row's reference m moves when a weight 2^(score - m) times its value norm exceeds
// 2^kMostProduct, or a weight 2^kMostWeight; it then leaves products of 2^kProduct and
// weights of 2^kWeight at most.  (binary16 ends at 65504 = 2^15.999 and a pair of parts
// rounds at 2^-25, so a product keeps bits down to 2^-32 of its row's largest.  Between
// 7 and 15.9 a reference moves in 0.14 of the units at 32 rows of d = 128, in 0.05 at 8
// of d = 64; a tile moves alone, since moving all four for one row took 149 us where
// this takes 135, 512 rows of 16 groups.)
constexpr float kMostProduct = 15.9f, kMostWeight = 96.0f;
constexpr float kProduct = 7.0f, kWeight = 80.0f;
// Scores beyond this stand as rounded numbers against their row's reference: an exact
// product less a rounded one is off by up to half a step, which from 2^31 on is 64 and
// more and would be the exponent of a weight.
constexpr float kFar = 0x1p24f;
constexpr float kCs = 4096.0f;         // scale of the codebook's binary16 rows

struct Start {  // of a workgroup's range: a group, runs before it, runs in all
  int32_t g;
  uint32_t pad;
  uint64_t off, count;
};

struct Args {
  const void* q;
  int q_dtype;
  const uint8_t* kp;
  const uint16_t* kn;
  const uint8_t* vp;
  const uint16_t* vn;
  const int32_t* lens;
  int32_t* now;       // the lengths as the ranges were made from (-1: bad), for the other launches
  const uint64_t* masks;
  int64_t mask_stride;
  int n_groups, M, G, rows, tiles;  // rows of a group, row tiles of a group
  int64_t T_stride;
  int k, N, w, P, pair_n;
  const float* R;
  const float* C;
  float qscale;
  h8* ops;            // the items' query operands
  float* qs;          // and their divisors (qs_floats of an item)
  Start* start;       // of every workgroup
  float* rec;
  int32_t* bounds;    // first and last workgroup of every item
  float* top;         // kTop partial maxima of |C| (staged codes)
  const float* stat;  // weights pass: m, l of every row
  float* acc;         // weights pass
  int lds_small, lds_ops, lds_scratch;  // LDS bytes before the small arrays, the queries' low parts, the scratch
};

__host__ __device__ constexpr int rec_floats(int D, int RT) { return 16 * RT * (D + 2); }
constexpr int tile_stride(int D) { return 2 * D + 16; }  // bytes of a staged row: spreads the banks
constexpr int state_regs(int D, int RT) { return RT * (D / 16) * 4 + 2 * RT; }
// floats between a state's registers in LDS: spreads the banks.  Packed rows end in
// half the lanes, which lets two workgroups with 64 KB tables share a compute unit.
constexpr int reg_floats(bool PK) { return PK ? 36 : 68; }
constexpr int state_floats(int D, int RT, bool PK) { return state_regs(D, RT) * reg_floats(PK); }
// an item's divisors: a row's own with one row tile, else the rows' relative to the
// item's, which is the last (negative: not all rows' are 1)
__host__ __device__ constexpr int qs_floats(int RT) { return RT > 1 ? 16 * RT + 1 : 16; }
// the queries' low parts: in registers for one row tile, else in LDS (they are 32
// of 256 registers at four tiles; 26 to 39 still spill there, outside the unit loop, and
// 60 of staged codes)
constexpr int ops_bytes(int D, int RT) { return RT > 1 ? RT * (D / 32) * 1024 : 0; }

// runs of units of a group of this length (-1: bad, none)
__device__ __forceinline__ int runs_of(const Args& a, int len) {
  return len < 0 ? 0 : (len + a.M + kRun - 1) / kRun;
}
__device__ __forceinline__ int checked(const Args& a, int len) {
  return len < 0 || len > a.T_stride - a.M ? -1 : len;
}

// two values as binary16 pairs: high parts, and the rest taken from their bits
__device__ __forceinline__ void split2(float a, float b, uint32_t* hi, uint32_t* lo) {
  uint32_t u = __builtin_bit_cast(uint32_t, h2{(_Float16)a, (_Float16)b});
  asm("" : "+v"(u));
  const h2 h = __builtin_bit_cast(h2, u);
  *hi = u;
  *lo = __builtin_bit_cast(uint32_t, h2{(_Float16)(a - (float)h[0]), (_Float16)(b - (float)h[1])});
}

template <typename IN>
__device__ __forceinline__ f4 load4(const void* q, int64_t at) {
  IN w[4];
  __builtin_memcpy(w, static_cast<const IN*>(q) + at, sizeof(w));
  return f4{to_float(w[0]), to_float(w[1]), to_float(w[2]), to_float(w[3])};
}

// One block per item (whatever its group's length: the lengths are read by the next
// block alone, once), then one that writes the ranges of `wgs` workgroups, then
// (staged codes) kTop that write partial maxima of the codebook.
//
// The rotation runs on v_mfma_f32_16x16x4_f32 (float32 products and sums; K slot
// kk of lane group gq is column D / 4 gq + kk).  A row's operands are at the power
// of two that takes its largest finite entry to [2^13, 2^14), so that the low parts
// of the entries that count are normal numbers.  With more than one row tile, rows
// whose largest entry is within 2^12 of the item's share the item's power (both
// parts then hold 25 bits of that entry), so that only items of rows further apart
// pay a multiplication per score (unit loop).  A launch of its own (3 to 6 us) costs less than the
// rotation in every workgroup that meets an item: 309 -> 234 us for 352 groups of
// 32k tokens, 118 -> 78 for 704 of 2048.
template <int D, int RT, bool PK>
__global__ __launch_bounds__(256 * (RT > 1 ? 2 : 1)) void prep_kernel(const Args a, int wgs) {
  constexpr int KS = D / 32, KQ = D / 4, Q = D / 16;
  constexpr int ROWS = 16 * RT, QS = D + 4;
  __shared__ __align__(16) float qt[ROWS * QS];
  __shared__ float tops[D / 16][ROWS];  // the rows' largest finite entries, of 16 dims
  constexpr int kT = 256 * (RT > 1 ? 2 : 1);
  __shared__ uint64_t sums[kT];
  __shared__ float red[kT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int items = a.n_groups * a.tiles;
  auto wave_max_of = [](const float* r) {
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < kT / 64; ++i) t = fmaxf(t, r[i]);
    return t;
  };
  if ((int)blockIdx.x > items) {  // a part of the codebook's largest entry
    float t = 0.0f;
    for (int i = (blockIdx.x - items - 1) * kT + tid; i < a.N * a.k; i += kTop * kT)
      t = fmaxf(t, fabsf(a.C[i]));
    t = wave_max_dpp(t);
    if (lane == 0) red[wave] = t;
    __syncthreads();
    if (tid == 0) a.top[blockIdx.x - items - 1] = wave_max_of(red);
    return;
  }
  if ((int)blockIdx.x == items) {
    const int per = (a.n_groups + kT - 1) / kT;
    uint64_t mine = 0;
    for (int i = 0; i < per; ++i) {
      const int g = tid * per + i;
      if (g < a.n_groups) {
        const int len = checked(a, a.lens[g]);
        a.now[g] = len;
        mine += runs_of(a, len);
      }
    }
    mine *= a.tiles;
    uint64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    uint64_t all = 0, add = 0;
    for (int i = 0; i < kT / 64; ++i) {
      if (i < wave) add += sums[i];
      all += sums[i];
    }
    __syncthreads();
    sums[tid] = upto + add;  // runs up to and with this thread's groups
    __syncthreads();
    const uint64_t each = all >> 32 ? all / wgs : (uint32_t)all / (uint32_t)wgs;
    const uint32_t rest = (uint32_t)(all - each * wgs);
    for (int b = tid; b < wgs; b += kT) {
      const uint64_t from = b * each + min((uint32_t)b, rest);
      Start s{0, 0, 0, each + ((uint32_t)b < rest)};
      if (s.count > 0) {
        int t = 0;  // the first thread whose groups reach beyond `from`
#pragma unroll
        for (int h = kT / 2; h > 0; h >>= 1)
          if (sums[t + h - 1] <= from) t += h;
        uint64_t off = from - (t > 0 ? sums[t - 1] : 0);
        int g = t * per;
        for (;; ++g) {  // (ends: the thread's groups hold `from`)
          const uint64_t v = (uint64_t)runs_of(a, a.now[g]) * a.tiles;
          if (off < v) break;
          off -= v;
        }
        s.g = g;
        s.off = off;
      }
      a.start[b] = s;
    }
    return;
  }
  const int64_t g = blockIdx.x / a.tiles;
  const int row0 = (int)(blockIdx.x % a.tiles) * ROWS;
  const int c = lane & 15, g16 = lane >> 4;
  const int live = (min(ROWS, a.rows - row0) + 15) / 16;
  float top = 0.0f;
  for (int it = wave; it < (D / 16) * live; it += kT / 64) {
    const int dt = it % (D / 16), t = it / (D / 16);
    const int row = row0 + 16 * t + c;
    f4 pa[KQ / 4], pb[KQ / 4] = {};
#pragma unroll
    for (int p = 0; p < KQ / 4; ++p)
      __builtin_memcpy(&pa[p], a.R + (16 * dt + c) * D + KQ * g16 + 4 * p, 16);
    if (row < a.rows) {
      const int64_t at = (g * a.rows + row) * D + KQ * g16;
      auto all = [&](auto load) {
#pragma unroll
        for (int p = 0; p < KQ / 4; ++p) pb[p] = load(at + 4 * p);
      };
      if (a.q_dtype == FIBQ_F32) all([&](int64_t i) { return load4<float>(a.q, i); });
      else if (a.q_dtype == FIBQ_F16) all([&](int64_t i) { return load4<f16_t>(a.q, i); });
      else all([&](int64_t i) { return load4<bf16_t>(a.q, i); });
    }
    f4 s = {0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < KQ / 4; ++p)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(pa[p][e], pb[p][e], s, 0, 0, 0);
    float most = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[e] *= a.qscale;
      most = fmaxf(most, fabsf(s[e]) < INFINITY ? fabsf(s[e]) : 0.0f);
    }
    most = xmax(xmax(most, 16), 32);
    if (g16 == 0) tops[dt][16 * t + c] = most;
    top = fmaxf(top, most);
    *reinterpret_cast<f4*>(qt + (16 * t + c) * QS + 16 * dt + 4 * g16) = s;
  }
  if constexpr (RT > 1) {
    top = wave_max_dpp(top);
    if (lane == 0) red[wave] = top;
  }
  __syncthreads();
  auto power = [](float x) {
    int e2 = 0;
    frexpf(x, &e2);
    return max(e2 - 14, -100);
  };
  const int shared = RT > 1 ? power(wave_max_of(red)) : 0;
  auto row_power = [&](int r) {
    float x = 0.0f;
    if (row0 + r < a.rows) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) x = fmaxf(x, tops[i][r]);
    }
    if (x == 0.0f) return shared;
    const int e2 = power(x);
    return RT > 1 && shared - e2 <= 12 ? shared : e2;
  };
  if (wave == 0) {
    const int e2 = row_power(min(tid, ROWS - 1)) - shared;
    float* to = a.qs + (int64_t)blockIdx.x * qs_floats(RT);
    if (tid < ROWS) to[tid] = ldexpf(1.0f, e2);
    const bool uneven = __any(e2 != 0);
    if (RT > 1 && tid == 0) to[ROWS] = ldexpf(uneven ? -1.0f : 1.0f, shared);
  }
  // B operand of K-step kap: lane l holds column l % 16 (PK: row l % 8, its high
  // part below 8, else its low part), K slots = dims 4 (l / 16 Q + 2 kap) .. + 7
  h8* to = a.ops + (int64_t)blockIdx.x * RT * KS * (PK ? 1 : 2) * 64;
  for (int x = tid; x < RT * KS * 64; x += kT) {
    const int l = x & 63, kap = (x >> 6) % KS, t = (x >> 6) / KS;
    const int r = 16 * t + (PK ? l & 7 : l & 15);
    uint32_t hi[4] = {}, lo[4] = {};
    if (row0 + r < a.rows) {
      const float qi = ldexpf(1.0f, -row_power(r));
      const float* at = qt + r * QS + 4 * ((l >> 4) * Q + 2 * kap);
#pragma unroll
      for (int i = 0; i < 4; ++i) split2(at[2 * i] * qi, at[2 * i + 1] * qi, &hi[i], &lo[i]);
    }
    if constexpr (PK) {
#pragma unroll
      for (int i = 0; i < 4; ++i) hi[i] = (l & 8) ? lo[i] : hi[i];
      __builtin_memcpy(&to[kap * 64 + l], hi, 16);
    } else {
      __builtin_memcpy(&to[(t * KS + kap) * 128 + l], hi, 16);
      __builtin_memcpy(&to[(t * KS + kap) * 128 + 64 + l], lo, 16);
    }
  }
}

// Barrier for data in LDS: loads from global memory stay in flight across it
// (the fence of __syncthreads waits for them).
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// One lane's loads of a unit: a payload quarter of the token whose K row it
// gathers in each tile, one of the token whose V rows it addresses, and the
// norms of its softmax tokens (binary16 pairs).
template <int QW, int NE>
struct Unit {
  uint32_t kq[2][QW], vq[2][QW];
  uint32_t nk[NE / 2], nv[NE / 2];
  float acc;  // weights pass: the accumulator that the lane adds to
};

// W > 0: compile-time index width, W = 0: at run time; KB: 4-dim rows per
// codeword; QW: dwords of a payload quarter, 0 for staged codes (below); PK:
// packed rows.  WT: the weights pass (scores only, added to acc).
//
// Staged codes (QW = 0) are those whose codewords cannot be addressed as 4-dim
// rows of an LDS table (k = 1, most of k = 2, quarters of a payload that share
// a codeword, tables above 64 KB): each wavefront writes the decoded rows of
// its unit, keys and then values, into a tile of its own and reads the operands
// from there.  Codes that both serve go through the table: 208 rows, 2048 tokens,
// k = 4, 37 us against 81; 704 groups of 8 rows, k = 2, 62 against 197.
template <int D, int RT, int W, int KB, int QW, bool PK, bool WT>
__global__ __launch_bounds__(kThreads, D == 64 && QW > 0 && (PK || WT) ? 4 : 2) void rows_kernel(const Args a) {
  constexpr int NB = D / 4, Q = NB / 4;  // 4-dim rows, of them per quarter
  constexpr int KS = D / 32, VM = D / 16;
  constexpr int ROWS = 16 * RT;
  constexpr int NE = PK ? 4 : 8;         // softmax tokens of a lane
  constexpr bool kStaged = QW == 0;
  constexpr int QD = kStaged ? 1 : QW;
  static_assert(!PK || RT == 1, "packed rows are one tile");
  // All LDS is dynamic, the table first: at address 0 its rows' offsets are their
  // addresses (one instruction less per gathered row).
  extern __shared__ __align__(16) unsigned char smem[];
  float* red = reinterpret_cast<float*>(smem + a.lds_small);  // [kWaves]
  int* redi = reinterpret_cast<int*>(red + kWaves);            // [kWaves]
  float* fac = red + 2 * kWaves;                               // [4][ROWS]: the states' factors in a record
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g16 = lane >> 4, c = lane & 15, hr = PK ? c & 7 : c;
  const int w = W > 0 ? W : a.w;
  const int P = a.P;
  const uint32_t b = blockIdx.x;
  const Start from = a.start[b];
  uint64_t left = from.count, off = from.off;
  int g = from.g;
  if (left == 0) return;

  // ---- the codebook's binary16 rows times cs (pairs: of the pair codebook) and
  //      their residuals.  Entries of unit vectors' blocks are at most 1; at
  //      2^12 one above 2^-14 keeps 22 bits.  Other codebooks are staged again
  //      at the power of two that takes their largest entry to [2^13, 2^14).
  const int nrow = kStaged ? 0 : a.pair_n > 0 ? a.pair_n * a.pair_n : a.N * a.k / 4;
  bool has_lo = false;
  float cs = kCs, ci = 1.0f / kCs;
  auto pick_scale = [&](float top) {
    if (top == 0.0f || (top >= 0x1p-6f && top < 15.9f)) return false;
    int e2 = 0;
    frexpf(top, &e2);
    e2 = top < INFINITY ? min(max(14 - e2, -100), 100) : 0;
    cs = ldexpf(1.0f, e2);
    ci = ldexpf(1.0f, -e2);
    return true;
  };
  auto table = [&]() {
    bool lo_any = false;
    float top = 0.0f;
    auto row = [&](int i, f4* v) {
      if (a.pair_n > 0) {
        __builtin_memcpy(v, a.C + 2 * (i & (a.pair_n - 1)), 8);
        __builtin_memcpy(reinterpret_cast<float*>(v) + 2, a.C + 2 * (i / a.pair_n), 8);
      } else {
        __builtin_memcpy(v, a.C + (size_t)i * 4, 16);
      }
    };
    auto put = [&](int i, const f4& v) {
      h4 hi, lo;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        hi[e] = (_Float16)(v[e] * cs);
        lo[e] = (_Float16)fmaf(v[e], cs, -(float)hi[e]);
        lo_any |= (float)lo[e] != 0.0f;
        top = fmaxf(top, fabsf(v[e]));
      }
      reinterpret_cast<h4*>(smem)[i] = hi;
      reinterpret_cast<h4*>(smem)[nrow + i] = lo;
    };
    int i = tid;
    for (; i + 3 * kThreads < nrow; i += 4 * kThreads) {  // four loads at once
      f4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) row(i + j * kThreads, &v[j]);
#pragma unroll
      for (int j = 0; j < 4; ++j) put(i + j * kThreads, v[j]);
    }
    for (; i < nrow; i += kThreads) {
      f4 v;
      row(i, &v);
      put(i, v);
    }
    top = wave_max_dpp(top);
    lo_any = __any(lo_any);
    if (lane == 0) {
      red[wave] = top;
      redi[wave] = lo_any;
    }
  };
  if constexpr (kStaged) pick_scale(wave_max_dpp(a.top[lane]));
  else table();

  float* scratch = reinterpret_cast<float*>(smem + a.lds_scratch);
  // (staged: a tile of high parts, then of residuals, for each wavefront)
  unsigned char* tile = smem + a.lds_scratch + (size_t)wave * 2 * kStep * tile_stride(D);
  // quarter g16 of token c of a tile for K, quarter c % 4 of token 4 g16 + c / 4
  // for V: 4 QW bytes inside the row that hold its bits from bit `sh` on
  const int NI = Q / KB;
  const int kbit = g16 * NI * w, vbit = (c & 3) * NI * w;
  const int kst = min(kbit >> 3, P - 4 * QD), vst = min(vbit >> 3, P - 4 * QD);
  const int ksh = kbit - 8 * kst, vsh = vbit - 8 * vst;
  const int ko = c * P + kst, vo = (4 * g16 + (c >> 2)) * P + vst;
  // (shifted where it is used: a shift at the load would wait for it)
  auto shifted = [&](const uint32_t (&q)[2][QD], int sh, uint32_t (&d)[2][QD]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (QD == 1) {
        d[t][0] = q[t][0] >> sh;
      } else if constexpr (QD == 2) {
        const uint64_t u = ((uint64_t)q[t][0] | ((uint64_t)q[t][1] << 32)) >> sh;
        d[t][0] = (uint32_t)u;
        d[t][1] = (uint32_t)(u >> 32);
      } else {
#pragma unroll
        for (int i = 0; i < QD; ++i) d[t][i] = q[t][i];
      }
    }
  };
  // token i of the lane's softmax tokens, in the unit
  const int tok0 = 4 * g16 + (PK ? 2 * (c & 8) : 0);
  auto token = [&](int i) { return tok0 + 16 * (i >> 2) + (i & 3); };
  // weights pass: the token whose sum ends in this lane (bits 3, 2, 1 of c)
  const int acc_tok = 2 * (c & 8) + 4 * g16 + (c & 4) / 2 + (c & 2) / 2;

  // ---- one item, runs r0 .. r0 + take - 1
  auto segment = [&](int len, int rt0, int r0, int take, bool first) {
    const int tot = len + a.M;
    const int64_t base = (int64_t)g * a.T_stride, item = (int64_t)g * a.tiles + rt0;
    // a unit inside the group is read at wave-uniform addresses plus the lane's
    // offset; in the last one of a ragged group every token is clamped into it
    const uint8_t* kpg = a.kp + base * P;
    const uint8_t* vpg = a.vp + base * P;
    const uint16_t* kng = a.kn + base;
    const uint16_t* vng = a.vn + base;
    auto load = [&](int u) -> Unit<QD, NE> {
      Unit<QD, NE> x{};
      const int tb = u * kStep, tm = tot - 1;
      if (tb + kStep <= tot) {
        const uint8_t* kb = kpg + (int64_t)tb * P;
        const uint8_t* vb = vpg + (int64_t)tb * P;
        const uint8_t* knb = reinterpret_cast<const uint8_t*>(kng + tb);
        const uint8_t* vnb = reinterpret_cast<const uint8_t*>(vng + tb);
        // (the offsets stay 32 bits wide and in this block, so that they are the
        // loads' own offset operands)
        uint32_t ok = ko, ov = vo, on = 2 * tok0;
        asm volatile("" : "+v"(ok), "+v"(ov), "+v"(on));
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if constexpr (!kStaged) __builtin_memcpy(x.kq[t], kb + 16 * t * P + ok, 4 * QD);
          if constexpr (!kStaged && !WT) __builtin_memcpy(x.vq[t], vb + 16 * t * P + ov, 4 * QD);
        }
#pragma unroll
        for (int i = 0; i < NE; i += 4) {
          __builtin_memcpy(&x.nk[i / 2], knb + 8 * i + on, 8);
          if constexpr (!WT) __builtin_memcpy(&x.nv[i / 2], vnb + 8 * i + on, 8);
        }
        if constexpr (WT) x.acc = a.acc[base + tb + acc_tok];
        return x;
      }
      if constexpr (WT) x.acc = a.acc[base + min(tb + acc_tok, tm)];
      if constexpr (!kStaged) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          __builtin_memcpy(x.kq[t], kpg + (int64_t)min(tb + 16 * t + c, tm) * P + kst, 4 * QD);
          if constexpr (!WT)
            __builtin_memcpy(x.vq[t], vpg + (int64_t)min(tb + 16 * t + 4 * g16 + (c >> 2), tm) * P + vst, 4 * QD);
        }
      }
#pragma unroll
      for (int i = 0; i < NE; ++i) {  // (tokens behind the last one: norm 0)
        const int at = min(tb + token(i), tm);
        const uint32_t in = tb + token(i) <= tm ? 0xFFFFu : 0u;
        x.nk[i >> 1] |= (kng[at] & in) << (16 * (i & 1));
        if constexpr (!WT) x.nv[i >> 1] |= (vng[at] & in) << (16 * (i & 1));
      }
      return x;
    };
    const int u_end = min((r0 + take) * kWaves, (tot + kStep - 1) / kStep);
    int u = r0 * kWaves + wave;
    Unit<QD, NE> cur{};
    if (u < u_end) cur = load(u);

    // ---- the tile's queries
    const int row0 = rt0 * ROWS;
    h8 bh[RT][KS], bl[KS];  // (low parts: RT = 1 only)
    const h8* op = a.ops + item * (RT * KS * (PK ? 1 : 2) * 64) + lane;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int kap = 0; kap < KS; ++kap) {
        bh[t][kap] = op[(t * KS + kap) * (PK ? 64 : 128)];
        if constexpr (RT == 1 && !PK) bl[kap] = op[kap * 128 + 64];
      }
    const float qs = a.qs[item * qs_floats(RT) + (RT > 1 ? ROWS : hr)];
    if constexpr (RT > 1) {
      h8* to = reinterpret_cast<h8*>(smem + a.lds_ops);
      for (int x = tid; x < RT * KS * 64; x += kThreads)
        to[x] = (a.ops + item * (RT * KS * 128))[(x >> 6) * 128 + 64 + (x & 63)];
      lds_barrier();
    }
    if (!kStaged && first) {  // the table is whole; is its scale right?
      lds_barrier();
      const float top = wave_max_dpp(red[lane & (kWaves - 1)]);
      if (pick_scale(top)) {
        lds_barrier();  // (red is written again)
        table();
        lds_barrier();
      }
      has_lo = __any(lane < kWaves && redi[lane & (kWaves - 1)] != 0);
    }
    // scores: products times nu_K times this, in log2 units (RT > 1: negative if some
    // rows have a factor of their own or a reference beyond kFar; its sign costs the
    // loop no register)
    float ks = qs * ci;
    bool far = false;  // (uniform, RT = 1) a reference is beyond kFar

    f4 acc[RT][VM];
    float m[RT], l[RT];
    // The reference m of a row: weights are 2^(score - m).  It follows the largest
    // product of a weight and its value norm, so that both binary16 parts of those
    // that count are normal numbers, however far the row's value norms are apart;
    // weights themselves are float32 numbers up to 2^96, which is where a token of a
    // far larger score and value norm 0 moves it.
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      m[t] = -INFINITY;
      l[t] = 0.0f;
#pragma unroll
      for (int mu = 0; mu < VM; ++mu) acc[t][mu] = f4{0, 0, 0, 0};
    }
    if constexpr (WT) {
      // this row's statistics; against +inf the scores of rows behind the last one
      // have weight 0 (their scores of 0 against a reference below -128 would be
      // infinite weights, and no number times l = 0)
      m[0] = INFINITY;
      if (hr < a.rows) {
        const int64_t at = ((int64_t)g * a.rows + hr) * 2;
        m[0] = a.stat[at] == -INFINITY ? 0.0f : a.stat[at];
        l[0] = a.stat[at + 1] != 0.0f ? 1.0f / a.stat[at + 1] : 0.0f;
        far = fabsf(m[0]) > kFar;
      }
      far = __any(far);
    }

    // staged codes: rows of the unit's tokens into the tile; whether any has a residual
    auto stage = [&](const uint8_t* pay, int tb) -> bool {
      bool any = false;
      const int nt = min(kStep, tot - tb);
      const int n = a.k >= 4 ? 1 : 4 / a.k;  // codewords of a 4-dim piece
      const uint32_t ones = (1u << w) - 1;
      // pieces in batches whose loads are all in flight at once: payloads, then rows
      constexpr int kBatch = RT == 1 ? 8 : 4;
#pragma unroll 1
      for (int x0 = lane; x0 < kStep * NB; x0 += 64 * kBatch) {
        uint64_t bits[kBatch];
        float cv[kBatch][4];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const int x = x0 + 64 * i, p = x % NB;
          const uint8_t* row = pay + (base + tb + min(x / NB, nt - 1)) * P;
          const int bit = (a.k >= 4 ? 4 * p / a.k : p * n) * w;
          const int at = bit >> 3;
          if (P >= 8) {  // (a piece's codewords and the shift take at most 63 bits)
            const int st = min(at, P - 8);
            __builtin_memcpy(&bits[i], row + st, 8);
            bits[i] >>= bit - 8 * st;
          } else {       // (at most 21 bits: rows of up to 7 bytes)
            bits[i] = (row[at] | (uint32_t)row[min(at + 1, P - 1)] << 8 |
                       (uint32_t)row[min(at + 2, P - 1)] << 16) >> (bit & 7);
          }
        }
        if (a.k >= 4) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i)
            __builtin_memcpy(cv[i], a.C + (size_t)((uint32_t)bits[i] & ones) * a.k + 4 * ((x0 + 64 * i) % NB) % a.k, 16);
        } else if (a.k == 2) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i) {
            __builtin_memcpy(cv[i], a.C + 2 * ((uint32_t)bits[i] & ones), 8);
            __builtin_memcpy(cv[i] + 2, a.C + 2 * ((uint32_t)(bits[i] >> w) & ones), 8);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kBatch; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) cv[i][e] = a.C[(uint32_t)(bits[i] >> (e * w)) & ones];
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const int x = x0 + 64 * i;
          uint32_t hi[2], lo[2];
          split2(cv[i][0] * cs, cv[i][1] * cs, &hi[0], &lo[0]);
          split2(cv[i][2] * cs, cv[i][3] * cs, &hi[1], &lo[1]);
          any |= ((lo[0] | lo[1]) & 0x7FFF7FFFu) != 0;
          unsigned char* to = tile + x / NB * tile_stride(D) + 8 * (x % NB);
          __builtin_memcpy(to, hi, 8);
          __builtin_memcpy(to + kStep * tile_stride(D), lo, 8);
        }
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
      return __any(any);
    };

    auto compute = [&](const Unit<QD, NE>& x, int tb) {
      bool lo_now = has_lo;  // (uniform) residual rows to add
      if constexpr (kStaged) lo_now = stage(a.kp, tb);
      uint32_t kq[2][QD], vq[2][QD];
      shifted(x.kq, ksh, kq);
      shifted(x.vq, vsh, vq);
      const int lo_at = kStaged ? kStep * tile_stride(D) : nrow * 8;
      // two gathered rows per lane of tile t, K-step kap, `d` bytes behind the high parts
      auto krow = [&](const uint32_t (&q)[2][QD], int t, int kap, int d) -> h8 {
        if constexpr (kStaged) {
          return *reinterpret_cast<const h8*>(tile + (16 * t + c) * tile_stride(D) + 8 * (g16 * Q + 2 * kap) + d);
        } else {
          const h4 a0 = *reinterpret_cast<const h4*>(smem + qrow<QD, W, KB>(q[t], 2 * kap, w) + d);
          const h4 a1 = *reinterpret_cast<const h4*>(smem + qrow<QD, W, KB>(q[t], 2 * kap + 1, w) + d);
          return h8{a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]};
        }
      };
      // ---- scores of all row tiles, 16 tokens at a time
      f4 s[RT][2];
      h8 ka[2][KS];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int kap = 0; kap < KS; ++kap) ka[i][kap] = krow(kq, i, kap, 0);
#pragma unroll
      for (int t = 0; t < RT; ++t) s[t][0] = s[t][1] = f4{0, 0, 0, 0};
      int opl = a.lds_ops + 16 * lane;
      asm volatile("" : "+v"(opl));  // (else these reads move out of the unit loop, into registers)
#pragma unroll
      for (int kap = 0; kap < KS; ++kap) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          if constexpr (PK) break;
          h8 lo;
          if constexpr (RT > 1) lo = *reinterpret_cast<const h8*>(smem + opl + (t * KS + kap) * 1024);
          else lo = bl[kap];
#pragma unroll
          for (int i = 0; i < 2; ++i)
            s[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ka[i][kap], lo, s[t][i], 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            s[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ka[i][kap], bh[t][kap], s[t][i], 0, 0, 0);
      }
      // a copy whose row addresses are computed anew (kept from the high parts'
      // reads for this rare path they would cost 16 registers)
      auto again = [&](const uint32_t (&q)[2][QD], uint32_t (&y)[2][QD]) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < QD; ++i) {
            y[t][i] = q[t][i];
            asm volatile("" : "+v"(y[t][i]));
          }
      };
      if (lo_now) {
        uint32_t kl[2][QD];
        again(kq, kl);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int kap = 0; kap < KS; ++kap) {
            const h8 kr = krow(kl, i, kap, lo_at);
#pragma unroll
            for (int t = 0; t < RT; ++t)
              s[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kr, bh[t][kap], s[t][i], 0, 0, 0);
          }
      }
      auto ror8 = [](float v) {  // lanes c and c ^ 8 of a 16-lane row
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, false));
      };
      if constexpr (PK) {  // high + low parts; lane h: tile 0, lane h + 8: tile 1
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float own = (c & 8) ? s[0][1][e] : s[0][0][e];
          const float other = (c & 8) ? s[0][0][e] : s[0][1][e];
          s[0][0][e] = own + ror8(other);
        }
      }
      if constexpr (RT > 1) {
        if (ks < 0.0f) {
          int64_t at = item;
          asm volatile("" : "+s"(at));  // (an address computed here costs the loop no register)
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const float f = a.qs[at * qs_floats(RT) + 16 * t + c];
            s[t][0] *= f;
            s[t][1] *= f;
          }
        }
      }
      // (one tile scales its scores, and the norms stay binary16 operands; more
      // tiles share the scaled norms)
      float nk[NE];
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        nk[i] = (float)__builtin_bit_cast(h2, x.nk[i >> 1])[i & 1];
        if constexpr (RT > 1) nk[i] *= fabsf(ks);
        else s[0][i >> 2][i & 3] *= ks;
      }
      float nv[NE];
#pragma unroll
      for (int i = 0; i < NE; ++i)
        nv[i] = WT ? 0.0f : (float)__builtin_bit_cast(h2, x.nv[i >> 1])[i & 1];
      // A unit that holds drafted tokens or ends behind the last one: unseen
      // scores become -inf.  Norms may be anything there: one that is not a
      // positive number is multiplied into the seen scores (a value norm that is
      // no number makes them NaN), and leaves the unseen ones alone.
      if (tb + kStep > len) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          uint64_t mask = 0;
          if (!WT && a.M > 0) mask = a.masks[g * a.mask_stride + min(row0 + 16 * t + hr, a.rows - 1) / a.G];
#pragma unroll
          for (int i = 0; i < NE; ++i) {
            const int j = tb + token(i) - len;
            float v = s[t][i >> 2][i & 3];
            if (!(nk[i] > 0.0f && nk[i] < INFINITY)) v *= nk[i];
            if (!(fabsf(nv[i]) < INFINITY)) v = NAN;
            const bool in = j < 0 || (j < a.M && (mask >> (j & 63) & 1));
            s[t][i >> 2][i & 3] = in ? v : -INFINITY;
          }
        }
#pragma unroll
        for (int i = 0; i < NE; ++i) {
          nk[i] = nk[i] > 0.0f && nk[i] < INFINITY ? nk[i] : 1.0f;
          nv[i] = fabsf(nv[i]) < INFINITY ? nv[i] : 0.0f;
        }
      }
      auto against = [&](int t, float ref, float (&p)[NE]) {
#pragma unroll
        for (int i = 0; i < NE; ++i) p[i] = fmaf(s[t][i >> 2][i & 3], nk[i], -ref);
      };
      auto far_rows = [&](float ref, float (&p)[NE]) {  // scores to their steps, where ref is beyond kFar
        const float r = fabsf(ref) > kFar && fabsf(ref) < INFINITY ? ref : 0.0f;
#pragma unroll
        for (int i = 0; i < NE; ++i) p[i] = (p[i] + r) - r;
      };
      if constexpr (WT) {
        float p[NE];
        against(0, m[0], p);
        if (__builtin_expect(far, 0)) far_rows(m[0], p);
#pragma unroll
        for (int i = 0; i < NE; ++i) p[i] = __builtin_amdgcn_exp2f(p[i]) * l[0];
        // sums over the rows (lanes of a 16-lane row), each step halving the
        // tokens that a lane keeps: bits 3, 2, 1 of c pick token i's bits 2, 1, 0
        auto dpp = [](float v, auto ctrl) {
          return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false));
        };
        const bool b3 = c & 8, b2 = c & 4, b1 = c & 2;
        float x4[4], x2[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // row_ror:8 swaps lanes c and c ^ 8 (packed: those are two tiles)
          if constexpr (PK) x4[i] = p[i];
          else x4[i] = (b3 ? p[i + 4] : p[i]) + ror8(b3 ? p[i] : p[i + 4]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)  // row_half_mirror: lanes c and c ^ 7
          x2[i] = (b2 ? x4[i + 2] : x4[i]) + dpp(b2 ? x4[i] : x4[i + 2], std::integral_constant<int, 0x141>{});
        // quad_perm [2, 3, 0, 1] and [1, 0, 3, 2]: lanes c and c ^ 2, c and c ^ 1
        float x1 = (b1 ? x2[1] : x2[0]) + dpp(b1 ? x2[0] : x2[1], std::integral_constant<int, 0x4E>{});
        x1 += dpp(x1, std::integral_constant<int, 0xB1>{});
        const int at = tb + acc_tok;
        if ((c & 1) == 0 && at < tot) a.acc[base + at] = x.acc + x1;
      } else {
        // ---- a weight that its lane's largest value norm may take above the bound, or
        //      (not a number or infinite) a row without a reference yet: the rows whose
        //      own products or weights are too large move
        typedef uint16_t u2 __attribute__((ext_vector_type(2)));
        u2 most_v = __builtin_bit_cast(u2, x.nv[0]);
#pragma unroll
        for (int i = 1; i < NE / 2; ++i) most_v = __builtin_elementwise_max(most_v, __builtin_bit_cast(u2, x.nv[i]));
        // (as bits, negative ones and those that are no numbers are above all; nothing is
        // below their bound, which is no number)
        const uint16_t most_b = max(most_v[0], most_v[1]);
        const float log_v = __builtin_amdgcn_logf((float)__builtin_bit_cast(_Float16, most_b) + 0x1p-80f);
        const float lim = kMostProduct - log_v;
        uint64_t over[RT], any_over = 0;
        float p[RT][NE];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          against(t, m[t], p[t]);
          float most = fmaxf(fmaxf(p[t][0], p[t][1]), fmaxf(p[t][2], p[t][3]));
          if constexpr (!PK)
            most = fmaxf(most, fmaxf(fmaxf(p[t][4], p[t][5]), fmaxf(p[t][6], p[t][7])));
          over[t] = __ballot(!(most <= lim));
          any_over |= over[t];
        }
        if (any_over) {
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            if (over[t] == 0) continue;
            // the row's largest score, and largest score + log2 of the value norm
            float top = -INFINITY, top_v = -INFINITY;
#pragma unroll
            for (int i = 0; i < NE; ++i) {
              const float v = s[t][i >> 2][i & 3] * nk[i];
              top = fmaxf(top, v);
              top_v = fmaxf(top_v, v + __builtin_amdgcn_logf(fabsf(nv[i])));
            }
            // (of a far row, the rounded score + a logarithm, not the exact product + one)
            const bool far_row = fabsf(top) > kFar;
            top_v = far_row ? top + fminf(log_v, 16.0f) : top_v;
            const bool large = m[t] == -INFINITY || top_v - m[t] > kMostProduct || top - m[t] > kMostWeight;
            uint64_t rows = __ballot(large);  // of a lane's row: bits c + 16 i (packed: hr + 8 i)
            if (rows == 0) continue;
            rows |= rows >> 32;
            rows |= rows >> 16;
            if constexpr (PK) rows |= rows >> 8;
            float to = fmaxf(top_v - kProduct, top - kWeight);
            to = xmax(xmax(to, 16), 32);
            if constexpr (PK) to = xmax(to, 8);
            const float m_new = (uint32_t)rows >> hr & 1 ? fmaxf(m[t], to) : m[t];
            const float f = m[t] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[t] - m_new);
            m[t] = m_new;
            if (__any(far_row && top > -INFINITY)) {
              far = true;
              if constexpr (RT > 1) ks = -fabsf(ks);
            }
            against(t, m_new == -INFINITY ? 0.0f : m_new, p[t]);  // (scores of -inf have weight 0)
            l[t] *= f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float fr = __shfl(f, (4 * g16 + e) & (PK ? 7 : 15), 64);
#pragma unroll
              for (int mu = 0; mu < VM; ++mu) acc[t][mu][e] *= fr;
            }
          }
        }
        if (__builtin_expect(RT > 1 ? ks < 0.0f : far, 0)) {
#pragma unroll
          for (int t = 0; t < RT; ++t) far_rows(m[t], p[t]);
        }
        // ---- weights in two binary16 parts
        h8 wh[RT], wl[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int i = 0; i < NE; ++i) p[t][i] = __builtin_amdgcn_exp2f(p[t][i]);
#pragma unroll
          for (int i = 0; i < NE; ++i) l[t] += p[t][i];
#pragma unroll
          for (int i = 0; i < NE; ++i) p[t][i] *= nv[i];
          if constexpr (PK) {
            // lanes h and h + 8 trade: row h takes both tiles' high parts, row
            // h + 8 their low parts
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t uh, ul;
              split2(p[0][2 * i], p[0][2 * i + 1], &uh, &ul);
              const uint32_t got = __float_as_uint(ror8(__uint_as_float((c & 8) ? uh : ul)));
              hi[i] = (c & 8) ? got : uh;
              hi[2 + i] = (c & 8) ? ul : got;
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) split2(p[t][2 * i], p[t][2 * i + 1], &hi[i], &lo[i]);
            __builtin_memcpy(&wl[t], lo, 16);
          }
          __builtin_memcpy(&wh[t], hi, 16);
        }
        // ---- values
        if constexpr (kStaged) lo_now = stage(a.vp, tb);
        auto vrow = [&](const uint32_t (&q)[2][QD], int mu, int d) -> h8 {
          const unsigned char *ra, *rb;
          if constexpr (kStaged) {
            ra = tile + (4 * g16 + (c >> 2)) * tile_stride(D) + 8 * ((c & 3) * VM + mu) + d;
            rb = ra + 16 * tile_stride(D);
          } else {
            ra = smem + qrow<QD, W, KB>(q[0], mu, w) + d;
            rb = smem + qrow<QD, W, KB>(q[1], mu, w) + d;
          }
          const h4 b0 = tr_read(ra), b1 = tr_read(rb);
          return h8{b0[0], b0[1], b0[2], b0[3], b1[0], b1[1], b1[2], b1[3]};
        };
#pragma unroll
        for (int mu = 0; mu < VM; ++mu) {
          const h8 bv = vrow(vq, mu, 0);
          if constexpr (!PK) {
#pragma unroll
            for (int t = 0; t < RT; ++t)
              acc[t][mu] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wl[t], bv, acc[t][mu], 0, 0, 0);
          }
#pragma unroll
          for (int t = 0; t < RT; ++t)
            acc[t][mu] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh[t], bv, acc[t][mu], 0, 0, 0);
        }
        if (lo_now) {
          uint32_t vl[2][QD];
          again(vq, vl);
#pragma unroll
          for (int mu = 0; mu < VM; ++mu) {
            const h8 dv = vrow(vl, mu, lo_at);
#pragma unroll
            for (int t = 0; t < RT; ++t)
              acc[t][mu] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh[t], dv, acc[t][mu], 0, 0, 0);
          }
        }
      }
      if constexpr (kStaged) {  // (the next unit writes the tile)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
      }
    };

    for (; u < u_end; u += kWaves) {  // (the next unit's loads are in flight meanwhile)
      Unit<QD, NE> nxt{};
      if (u + kWaves < u_end) nxt = load(u + kWaves);
      compute(cur, u * kStep);
      cur = nxt;
    }

    if constexpr (!WT) {
      // ---- the wavefronts' states: the upper four are taken into the lower
      //      four's registers, whose states all threads then combine into the record
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        l[t] = xsum(xsum(l[t], 16), 32);
        if constexpr (PK) l[t] = xsum(l[t], 8);
#pragma unroll
        for (int mu = 0; mu < VM; ++mu) {
          if constexpr (PK) {  // rows h and h + 8 sit in lanes l and l ^ 32
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[t][mu][e] += __shfl_xor(acc[t][mu][e], 32, 64);
          }
          acc[t][mu] *= ci;
        }
      }
      float* slot = scratch + (wave & 3) * state_floats(D, RT, PK) + (PK ? lane & 31 : lane);
      auto put = [&]() {
        if (PK && lane >= 32) return;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          slot[(2 * t) * reg_floats(PK)] = m[t];
          slot[(2 * t + 1) * reg_floats(PK)] = l[t];
#pragma unroll
          for (int mu = 0; mu < VM; ++mu)
#pragma unroll
            for (int e = 0; e < 4; ++e) slot[(2 * RT + (t * VM + mu) * 4 + e) * reg_floats(PK)] = acc[t][mu][e];
        }
      };
      lds_barrier();  // (the scratch is free)
      if (wave >= 4) put();
      lds_barrier();
      if (wave < 4) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const float mo = slot[(2 * t) * reg_floats(PK)], lo = slot[(2 * t + 1) * reg_floats(PK)];
          const float mx = fmaxf(m[t], mo), sub = mx == -INFINITY ? 0.0f : mx;
          const float f = __builtin_amdgcn_exp2f(m[t] - sub), fo = __builtin_amdgcn_exp2f(mo - sub);
          m[t] = mx;
          l[t] = l[t] * f + lo * fo;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float fr = __shfl(f, 4 * g16 + e, 64), fro = __shfl(fo, 4 * g16 + e, 64);
#pragma unroll
            for (int mu = 0; mu < VM; ++mu)
              acc[t][mu][e] = acc[t][mu][e] * fr + slot[(2 * RT + (t * VM + mu) * 4 + e) * reg_floats(PK)] * fro;
          }
        }
        put();
      }
      lds_barrier();
      // items and workgroups both only grow along the units, so item + workgroup
      // is a different number for every segment
      float* r = a.rec + (item + b) * rec_floats(D, RT);
      if (tid < ROWS) {
        const float* st = scratch + 2 * (tid >> 4) * reg_floats(PK) + (tid & 15);
        float mw[4], lw = 0.0f, mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          mw[i] = st[i * state_floats(D, RT, PK)];
          mx = fmaxf(mx, mw[i]);
        }
        const float sub = mx == -INFINITY ? 0.0f : mx;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = __builtin_amdgcn_exp2f(mw[i] - sub);
          fac[i * ROWS + tid] = f;
          lw = fmaf(st[i * state_floats(D, RT, PK) + reg_floats(PK)], f, lw);
        }
        r[tid] = mx;
        r[ROWS + tid] = lw;
      }
      if (tid == 0) {
        if (r0 == 0) a.bounds[2 * item] = b;
        if (r0 + take == (tot + kRun - 1) / kRun) a.bounds[2 * item + 1] = b;
      }
      lds_barrier();
#pragma unroll 1  // (code is fetched once per workgroup, at about 0.7 us per KB)
      for (int x = tid; x < (PK ? 8 : ROWS) * D; x += kThreads) {
        // row 16 t + 4 g + e, dim 4 ((c / 4) VM + mu) + c % 4: register (t, mu, e) of lane 16 g + c
        const int row = x / D, dim = x % D;
        const int reg = 2 * RT + ((row >> 4) * VM + (dim >> 2) % VM) * 4 + (row & 3);
        const float* st = scratch + reg * reg_floats(PK) + 16 * ((row >> 2) & 3) + 4 * (dim / (4 * VM)) + (dim & 3);
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) v = fmaf(st[i * state_floats(D, RT, PK)], fac[i * ROWS + row], v);
        r[2 * ROWS + x] = v;
      }
      // (the next item's first staged rows share LDS with the states; the barrier
      // behind its queries' low parts stands before them where there is one)
      if constexpr (kStaged && RT == 1) lds_barrier();
    }
  };

  for (bool first = true; left > 0; first = false) {
    if (off == 0 && !first) {  // the next group that holds units (64 at a time)
      for (;;) {
        const int at = g + lane;
        const uint64_t some = __ballot(at < a.n_groups && runs_of(a, a.now[min(at, a.n_groups - 1)]) > 0);
        if (some) {
          g += __builtin_ctzll(some);
          break;
        }
        g += 64;
        if (g >= a.n_groups) return;  // (not reached: units are left)
      }
    }
    const int len = a.now[g], runs = runs_of(a, len);
    const int rt0 = a.tiles == 1 ? 0 : (int)((uint32_t)off / (uint32_t)runs);
    const int r0 = (int)(off - (uint64_t)rt0 * runs);
    const int take = (int)(left < (uint64_t)(runs - r0) ? left : (uint64_t)(runs - r0));
    segment(len, rt0, r0, take, first);
    left -= take;
    off += take;
    if (off == (uint64_t)runs * a.tiles) {
      off = 0;
      ++g;
    }
  }
}

__device__ __forceinline__ float wave_sum_dpp(float v) {
#define FIBQ_ROR(n) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + n, 0xf, 0xf, false));
  FIBQ_ROR(8) FIBQ_ROR(4) FIBQ_ROR(2) FIBQ_ROR(1)
#undef FIBQ_ROR
  const int i = __float_as_int(v);
  return (__int_as_float(__builtin_amdgcn_readlane(i, 0)) + __int_as_float(__builtin_amdgcn_readlane(i, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(i, 32)) + __int_as_float(__builtin_amdgcn_readlane(i, 48)));
}

// Block: 256 / D rows of a group, a thread per (row, dim).  Log-sum-exp over the
// row's records, then o = Pi^T (acc / l) with Pi's rows in stripes over the
// threads, loaded before the records; stat (nullable) receives m and l.  What
// bounds it is latency: the launch, and the loads' round trips one behind the other.
// More than kFew records are therefore read with the statistics of 64 at once over
// the lanes, and sums whose loads depend on addresses only (64 records of 4 groups,
// 16 rows, k = 4: 33 -> 26 us for the whole call); with few the exchange between
// lanes costs more than it saves (a call of 17.0 us took 18.6).
template <int D>
__global__ __launch_bounds__(256) void merge_kernel(
    const float* __restrict__ rec, const int32_t* __restrict__ bounds,
    const int32_t* __restrict__ now, int M, int rows, int tiles, int tile_rows,
    const float* __restrict__ R, float* __restrict__ stat, float* __restrict__ out) {
  constexpr int HB = 256 / D, RI = D / HB;  // stripes = rows of the block
  __shared__ float ar[HB][D];
  __shared__ float part[HB][HB][D];
  __shared__ float fac[4][kMaxWgs];  // of every wavefront: the records' factors
  const int blocks = (rows + HB - 1) / HB;
  const int64_t g = blockIdx.x / blocks;
  const int hr = threadIdx.x / D, dim = threadIdx.x % D;
  const int row = (int)(blockIdx.x % blocks) * HB + hr;
  const int len = now[g];
  const bool bad = len < 0;
  float pi[RI];
#pragma unroll
  for (int i = 0; i < RI; ++i) pi[i] = R[(hr * RI + i) * D + dim];
  float m = -INFINITY, l = 0.0f, s = 0.0f;
  if (!bad && len + M > 0 && row < rows) {
    const int64_t item = g * tiles + row / tile_rows;
    const int rl = row % tile_rows, reclen = tile_rows * (D + 2);
    const int first = bounds[2 * item], n = bounds[2 * item + 1] - first + 1;
    const float* r = rec + (item + first) * reclen;
    constexpr int kFew = 8;
    if (n <= kFew) {
#pragma unroll 1
      for (int i0 = 0; i0 < n; i0 += 4) {
        float mk[4], lk[4], xk[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float* x = r + (int64_t)min(i0 + i, n - 1) * reclen;
          mk[i] = i0 + i < n ? x[rl] : -INFINITY;
          lk[i] = i0 + i < n ? x[tile_rows + rl] : 0.0f;
          xk[i] = i0 + i < n ? x[2 * tile_rows + rl * D + dim] : 0.0f;
        }
        const float mn = fmaxf(m, fmaxf(fmaxf(mk[0], mk[1]), fmaxf(mk[2], mk[3])));
        const float sub = mn == -INFINITY ? 0.0f : mn;
        const float f = __builtin_amdgcn_exp2f(m - sub);
        l *= f;
        s *= f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float fi = __builtin_amdgcn_exp2f(mk[i] - sub);
          l = fmaf(lk[i], fi, l);
          s = fmaf(xk[i], fi, s);
        }
        m = mn;
      }
    } else {
      const float* x = r + 2 * tile_rows + rl * D + dim;
      constexpr int kBatch = 8;
      float xk[kBatch];
      auto fetch = [&](int i0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) xk[i] = x[(int64_t)min(i0 + i, n - 1) * reclen];
      };
      fetch(0);
      const int lane = threadIdx.x & 63;
      float* f = fac[threadIdx.x >> 6];
#pragma unroll 1
      for (int i = lane; i < n; i += 64) {
        const float mk = r[(int64_t)i * reclen + rl], lk = r[(int64_t)i * reclen + tile_rows + rl];
        const float mn = fmaxf(m, mk), sub = mn == -INFINITY ? 0.0f : mn;
        l = l * __builtin_amdgcn_exp2f(m - sub) + lk * __builtin_amdgcn_exp2f(mk - sub);
        m = mn;
        f[i] = mk;
      }
      const float most = wave_max_dpp(m), sub = most == -INFINITY ? 0.0f : most;
      l = wave_sum_dpp(l * __builtin_amdgcn_exp2f(m - sub));
      m = most;
#pragma unroll 1
      for (int i = lane; i < (n + kBatch - 1) / kBatch * kBatch; i += 64)
        f[i] = i < n ? __builtin_amdgcn_exp2f(f[i] - sub) : 0.0f;
      __builtin_amdgcn_wave_barrier();
#pragma unroll 1
      for (int i0 = 0;;) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) s = i0 + i < n ? fmaf(xk[i], f[i0 + i], s) : s;
        i0 += kBatch;
        if (i0 >= n) break;
        fetch(i0);
      }
    }
  }
  ar[hr][dim] = l == 0.0f ? 0.0f : s / l;
  __syncthreads();
#pragma unroll
  for (int h = 0; h < HB; ++h) {  // this stripe's part of row h
    float o = 0.0f;
#pragma unroll
    for (int i = 0; i < RI; ++i) o = fmaf(pi[i], ar[h][hr * RI + i], o);
    part[hr][h][dim] = o;
  }
  __syncthreads();
  if (row >= rows) return;
  float o = 0.0f;
#pragma unroll
  for (int x = 0; x < HB; ++x) o += part[x][hr][dim];
  out[(g * rows + row) * D + dim] = bad ? NAN : o;
  if (stat && dim < 2) stat[(g * rows + row) * 2 + dim] = dim == 0 ? m : l;
}

// ----------------------------------------------------------------- host ----
// How a code's rows are gathered: through an LDS table (codes whose payload
// quarters hold whole codewords and lie in 4, 8 or 12 bytes of the row), or
// staged.
struct Kind {
  int w, kb, qw;  // template arguments (w = 0: at run time)
  int lds;        // bytes of the table
};
static Kind kind_of(const Shape& s, Shape* as, int* pair_n) {
  *as = s;
  *pair_n = 0;
  if (s.k == 2 && (s.w == 4 || s.w == 6)) {  // pairs of blocks: a k = 4 code
    *as = Shape{s.d, 4, s.N * s.N, 2 * s.w, s.P};
    *pair_n = s.N;
  }
  const Kind staged{0, 1, 0, 0};
  const int kb = as->k / 4, ni = kb > 0 ? s.d / 16 / kb : 0;
  if (as->k % 4 != 0 || ni < 1 || ni * kb * 16 != s.d || (int64_t)as->N * as->k > 16384) return staged;
  const int lds = as->N * as->k * 4;
  if (kb == 1 && as->w == 8) return Kind{8, 1, s.d / 64, lds};
  if (kb == 1 && as->w == 12) return Kind{12, 1, s.d == 64 ? 2 : 3, lds};
  if (s.d == 64 && kb == 2 && (as->w == 4 || as->w == 6)) return Kind{as->w, 2, 1, lds};
  if (s.P < 8 || kb > 4) return staged;
  for (int q = 0; q < 4; ++q) {  // 8 bytes inside the row that hold the quarter
    const int bit = q * ni * as->w;
    const int st = bit / 8 < s.P - 8 ? bit / 8 : s.P - 8;
    if (bit - 8 * st + ni * as->w > 64) return staged;
  }
  return Kind{0, kb, 2, lds};
}

// Row tiles: 16 RT rows share the gathered codewords; registers hold 64 rows
// at d = 64 and 32 at d = 128.  Relative to a workgroup's run of units for 16 rows
// (about 1 us), one for 32 and 64 rows takes 1.5 and 2.8, and an item's queries and
// record take 5, 9 and 12.  Large tiles therefore win where a workgroup has many
// runs (512 rows, 16 groups, 32k tokens, k = 8: 194, 154 and 140 us) or many short
// items (512 rows, 64 groups, 512 tokens: 86, 74 and 73 us); small ones where it
// has few (24 rows, 16 groups, 32k tokens: 26 and 31 us; 48 rows, 2048 tokens: 17.5,
// 19 and 25 us) or where large ones pad the rows.  Over 210 sizes the choice is
// 0.8 % behind the best on average and 15 % at most; the largest tile that the
// rows fill was 19 % and 58 % behind.
static int tile_rows(int64_t n_groups, int64_t T_stride, int rows, int D) {
  const double run_cost[3] = {1.0, 1.5, 2.8}, item_cost[3] = {5.0, 9.0, 12.0};
  const double runs = (double)((T_stride + kRun - 1) / kRun);
  int best = 16;
  double least = INFINITY;
  for (int i = 0; i < (rows <= 16 ? 1 : D == 64 ? 3 : 2); ++i) {
    const double work = (double)n_groups * ((rows + (16 << i) - 1) / (16 << i)) * runs;
    const double each = work / (work < kMaxWgs / 2 ? work : kMaxWgs / 2);  // runs of a workgroup
    const double cost = run_cost[i] * each + item_cost[i] * (each > runs ? each / runs : 1.0);
    if (cost < least) {  // (no work at all: not a number)
      least = cost;
      best = 16 << i;
    }
  }
  return best;
}

struct Layout {
  bool packed;
  int tile, tiles;  // rows of a tile, tiles of a group
  size_t off_qs, off_now, off_start, off_top, off_bounds, off_stat, off_rec, total;
};
static Layout make_layout(int64_t n_groups, int M, int G, const Shape& s, int tile) {
  Layout y{};
  const int rows = (M > 0 ? M : 1) * G;
  y.packed = rows <= 8;
  y.tile = tile;
  y.tiles = (rows + y.tile - 1) / y.tile;
  const size_t items = (size_t)n_groups * y.tiles;
  auto al = [](size_t x) { return (x + 255) & ~(size_t)255; };
  y.off_qs = al(items * (y.tile / 16) * (s.d / 32) * (y.packed ? 1 : 2) * 1024);
  y.off_now = al(y.off_qs + items * qs_floats(y.tile / 16) * 4);
  y.off_start = al(y.off_now + (size_t)n_groups * 4);
  y.off_top = al(y.off_start + kMaxWgs * sizeof(Start));
  y.off_bounds = al(y.off_top + kTop * 4);
  y.off_stat = al(y.off_bounds + items * 8);
  y.off_rec = al(y.off_stat + (M > 0 ? 0 : (size_t)n_groups * rows * 8));
  y.total = al(y.off_rec + (items + kMaxWgs) * rec_floats(s.d, y.tile / 16) * 4);
  return y;
}

template <int D, int RT, int W, int KB, int QW, bool PK, bool WT>
static hipError_t launch_rows(Args a, int table, int wgs, hipStream_t st) {
  a.lds_small = table;
  a.lds_ops = table + (2 * kWaves + 4 * 16 * RT) * 4;
  a.lds_scratch = a.lds_ops + ops_bytes(D, RT);
  size_t scratch = WT ? 0 : (size_t)4 * state_floats(D, RT, PK) * 4;
  const size_t tiles = QW == 0 ? (size_t)kWaves * 2 * kStep * tile_stride(D) : 0;
  if (tiles > scratch) scratch = tiles;
  const size_t lds = a.lds_scratch + scratch;
  auto kern = rows_kernel<D, RT, W, KB, QW, PK, WT>;
  if (lds > 65536) {  // above the default dynamic LDS limit
    const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(kThreads), lds, st, a);
  return hipGetLastError();
}

template <int D, int RT, bool PK, bool WT>
static hipError_t launch_kind(const Args& a, const Kind& x, int wgs, hipStream_t st) {
#define FIBQ_SV(WW, KK, QQ) \
  if (x.w == WW && x.kb == KK && x.qw == QQ) return launch_rows<D, RT, WW, KK, QQ, PK, WT>(a, x.lds, wgs, st);
  if constexpr (D == 64) {
    FIBQ_SV(8, 1, 1) FIBQ_SV(12, 1, 2) FIBQ_SV(4, 2, 1) FIBQ_SV(6, 2, 1)
  } else {
    FIBQ_SV(8, 1, 2) FIBQ_SV(12, 1, 3)
  }
  if constexpr (D == 128) { FIBQ_SV(0, 4, 2) }  // (k = 16 at d = 64 has rows of less than 8 bytes)
  FIBQ_SV(0, 1, 2) FIBQ_SV(0, 2, 2) FIBQ_SV(0, 1, 0)
#undef FIBQ_SV
  return hipErrorInvalidValue;
}

// prep, main, merge, and the weights pass
template <int D, int RT, bool PK>
static int launch_tile(const ServeAttn& v, const Args& a, const Layout& y, const Kind& x, hipStream_t st) {
  const int64_t items = v.n_groups * y.tiles;
  // As many workgroups as run at once: two per compute unit where registers and LDS
  // allow (packed rows at d = 64: 704 groups of 2048 tokens 70 -> 61 us, 352 of 32k
  // 219 -> 182), or one per run if those are fewer.  A workgroup's run takes about
  // as long as the merge of 8 records (16 at d = 128), so an item of n runs is best
  // cut in sqrt(8 n) (one group of 131072 tokens: 61 us in 512 workgroups, 27 in 128,
  // 25 in 64, 28 in 32; of 32768 tokens: 25 us in 128, 19-20 in 32 or 64); 32 are never
  // too many (4 groups of 8192 tokens: 22.0 us, in 16 each 24.8).  A power of two, so
  // that ranges of usual capacities end where items do (d = 128, 4 items of 32768
  // tokens: 33.6 us in 45 each, 28.9 in 32).
  const int64_t runs = (v.T_stride + kRun - 1) / kRun;
  const int64_t most = items * runs;
  int64_t cut = 32;
  while (4 * cut * cut <= D / 8 * runs) cut *= 2;
  cut *= items;
  int64_t wgs = PK && D == 64 && x.qw > 0 ? kMaxWgs : kMaxWgs / 2;
  if (wgs > cut) wgs = cut;
  if (wgs > most) wgs = most;
  // (also without any row in the cache: the merge goes by the lengths that prep leaves)
  hipLaunchKernelGGL((prep_kernel<D, RT, PK>), dim3((unsigned)(items + 1 + (x.qw == 0 ? kTop : 0))),
                     dim3(256 * (RT > 1 ? 2 : 1)), 0, st, a, (int)(wgs > 0 ? wgs : 1));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return (int)e;
  if (wgs > 0 && (e = launch_kind<D, RT, PK, false>(a, x, (int)wgs, st)) != hipSuccess) return (int)e;
  const int64_t blocks = v.n_groups * ((a.rows + 256 / D - 1) / (256 / D));
  hipLaunchKernelGGL(merge_kernel<D>, dim3((unsigned)blocks), dim3(256), 0, st, a.rec, a.bounds,
                     a.now, v.M, a.rows, y.tiles, y.tile, v.R,
                     const_cast<float*>(a.stat), v.out);
  if ((e = hipGetLastError()) != hipSuccess) return (int)e;
  if constexpr (RT == 1)
    if (v.acc && wgs > 0) return (int)launch_kind<D, 1, PK, true>(a, x, (int)wgs, st);
  return 0;
}

template <int D>
static int launch(const ServeAttn& v, hipStream_t st) {
  const Layout y = make_layout(v.n_groups, v.M, v.G, v.s,
                               tile_rows(v.n_groups, v.T_stride, (v.M > 0 ? v.M : 1) * v.G, D));
  unsigned char* ws = static_cast<unsigned char*>(v.ws);
  Shape as;
  int pair_n;
  const Kind x = kind_of(v.s, &as, &pair_n);
  Args a{};
  a.q = v.q;
  a.q_dtype = v.q_dtype;
  a.kp = v.kp;
  a.kn = v.kn;
  a.vp = v.vp;
  a.vn = v.vn;
  a.lens = v.lens;
  a.masks = v.masks;
  a.mask_stride = v.mask_stride;
  a.n_groups = (int)v.n_groups;
  a.M = v.M;
  a.G = v.G;
  a.rows = (v.M > 0 ? v.M : 1) * v.G;
  a.tiles = y.tiles;
  a.T_stride = v.T_stride;
  a.k = as.k;
  a.N = as.N;
  a.w = as.w;
  a.P = as.P;
  a.pair_n = pair_n;
  a.R = v.R;
  a.C = v.C;
  a.qscale = v.scale * 1.4426950408889634f;  // base-2 softmax
  a.ops = reinterpret_cast<h8*>(ws);
  a.qs = reinterpret_cast<float*>(ws + y.off_qs);
  a.now = reinterpret_cast<int32_t*>(ws + y.off_now);
  a.start = reinterpret_cast<Start*>(ws + y.off_start);
  a.top = reinterpret_cast<float*>(ws + y.off_top);
  a.bounds = reinterpret_cast<int32_t*>(ws + y.off_bounds);
  a.stat = v.acc ? reinterpret_cast<float*>(ws + y.off_stat) : nullptr;
  a.rec = reinterpret_cast<float*>(ws + y.off_rec);
  a.acc = v.acc;
  if (y.packed) return launch_tile<D, 1, true>(v, a, y, x, st);
  if (y.tile == 16) return launch_tile<D, 1, false>(v, a, y, x, st);
  if (y.tile == 32) return launch_tile<D, 2, false>(v, a, y, x, st);
  if constexpr (D == 64) return launch_tile<D, 4, false>(v, a, y, x, st);
  return (int)hipErrorInvalidValue;
}

}  // namespace sv

size_t serve_attn_workspace_bytes(int64_t n_groups, int M, int G, const Shape& s) {
  size_t most = 0;  // (of every tile: which one is taken depends on T_stride)
  for (int tile = 16; tile <= (s.d == 64 ? 64 : 32); tile *= 2) {
    const size_t n = sv::make_layout(n_groups, M, G, s, tile).total;
    if (n > most) most = n;
  }
  return most;
}

int launch_serve_attn(const ServeAttn& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  return a.s.d == 64 ? sv::launch<64>(a, st) : sv::launch<128>(a, st);
}

}  // namespace dev
}  // namespace fibq
