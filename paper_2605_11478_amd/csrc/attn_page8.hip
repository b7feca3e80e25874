// Attention over the paged 8-bit cache (fibq_attn_cache8).
#include <hip/hip_runtime.h>

#include "device_common.h"
#include "fibq.h"
#include "fibq_internal.h"

namespace fibq {
namespace dev {
namespace pa {

__device__ __forceinline__ float code_value(uint8_t b, int codes) {
  return codes == FIBQ_INT8 ? (float)(int8_t)b : __builtin_amdgcn_cvt_f32_fp8(b, 0);
}

// One wavefront per row and query head: 64 tokens at a time, one pass with the
// running maximum and sum.
template <typename T, int D>
__global__ __launch_bounds__(64) void simple_kernel(PageAttn a) {
  __shared__ float q[D], w[64];
  __shared__ const uint8_t* at_v[64];
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x, g_max = a.n_seqs;
  const int head = blockIdx.y, h = head / a.G;
  int64_t g = row, begin = row, end = row + 1;
  if (a.starts) {  // the sequence whose rows hold this one
    g = g_max;
    for (int64_t g0 = 0; g0 < g_max && g == g_max; g0 += 64) {
      const int64_t mine = min(g0 + lane, g_max - 1);
      const int64_t b = a.starts[mine], e = a.starts[mine + 1];
      const uint64_t found = __ballot(b >= 0 && b <= row && row < e && e <= a.n_rows);
      if (found) {
        g = g0 + __ffsll((unsigned long long)found) - 1;
        begin = a.starts[g];
        end = a.starts[g + 1];
      }
    }
    if (g == g_max) return;
  }
  const int64_t len = a.lens[g], rows = end - begin;
  float* out = a.out + (row * a.H * a.G + head) * D;
  const bool bad = len < 0 || len > a.max_pages * a.page || (a.causal && rows > len);
  const int64_t seen = bad ? 0 : a.causal ? len - rows + (row - begin) + 1 : len;
  float big = 0.0f;
  for (int i = lane; i < D; i += 64) {
    q[i] = to_float(((const T*)a.q)[(row * a.H * a.G + head) * D + i]);
    big = fmaxf(big, fabsf(q[i]));
  }
  big = wave_max(big);
  int e = 0;  // (the row times 2^-e is below 1, so that its products stay finite)
  if (big > 0.0f && big < INFINITY) frexpf(big, &e);
  for (int i = lane; i < D; i += 64) q[i] = ldexpf(q[i], -e);
  __syncthreads();
  float m = -INFINITY, l = 0.0f, acc[D / 64];
  for (int c = 0; c < D / 64; ++c) acc[c] = 0.0f;
  for (int64_t t0 = 0; t0 < seen; t0 += 64) {
    const int64_t t = t0 + lane;
    float s = -INFINITY, vs = 0.0f;
    at_v[lane] = nullptr;
    if (t < seen) {
      const int32_t id = a.table[g * a.max_pages + t / a.page];
      const bool known = id >= 0 && id < a.n_pages;
      const int64_t ph = (int64_t)(known ? id : 0) * a.H + h;
      const uint8_t* kr = (const uint8_t*)a.k_pages + (ph * a.page + t % a.page) * D;
      at_v[lane] = (const uint8_t*)a.v_pages + (ph * a.page + t % a.page) * D;
      float x = 0.0f;
      for (int i = 0; i < D; ++i) x += q[i] * code_value(kr[i], a.codes);
      s = ldexpf(x * (known ? a.k_scales[ph] : NAN) * a.scale, e);
      s = s > 0x1p126f ? 0x1p126f : s < -0x1p126f ? -0x1p126f : s;
      vs = a.v_scales[ph];
    }
    float top = s;
    for (int o = 32; o > 0; o >>= 1) {
      const float y = __shfl_xor(top, o, 64);
      top = top != top || y != y ? NAN : fmaxf(top, y);
    }
    const float m2 = m != m || top != top ? NAN : fmaxf(m, top);
    const float p = s == -INFINITY && m2 == m2 ? 0.0f : expf(s - m2);
    const float r = m == -INFINITY && m2 == m2 ? 0.0f : expf(m - m2);
    l = l * r + wave_sum(p);
    m = m2;
    __syncthreads();
    w[lane] = p * vs;
    __syncthreads();
    for (int c = 0; c < D / 64; ++c) acc[c] *= r;
    for (int j = 0; j < 64 && t0 + j < seen; ++j)
      for (int c = 0; c < D / 64; ++c)
        acc[c] += w[j] * code_value(at_v[j][c * 64 + lane], a.codes);
    __syncthreads();
  }
  for (int c = 0; c < D / 64; ++c)
    out[c * 64 + lane] = bad ? NAN : l == 0.0f ? 0.0f : acc[c] / l;
}

template <typename T>
int simple_typed(const PageAttn& a, hipStream_t st) {
  const dim3 grid((unsigned)a.n_rows, a.H * a.G);
  switch (a.d) {
    case 64: simple_kernel<T, 64><<<grid, 64, 0, st>>>(a); break;
    case 128: simple_kernel<T, 128><<<grid, 64, 0, st>>>(a); break;
    default: simple_kernel<T, 256><<<grid, 64, 0, st>>>(a); break;
  }
  return (int)hipGetLastError();
}

}  // namespace pa

size_t page_attn_workspace_bytes(int64_t n_seqs, int64_t n_rows, int H, int G, int64_t max_pages,
                                 int page, int d) {
  return 0;
}

int launch_page_attn(const PageAttn& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (a.q_dtype) {
    case FIBQ_F32: return pa::simple_typed<float>(a, st);
    case FIBQ_F16: return pa::simple_typed<f16_t>(a, st);
    default: return pa::simple_typed<bf16_t>(a, st);
  }
}

}  // namespace dev
}  // namespace fibq
