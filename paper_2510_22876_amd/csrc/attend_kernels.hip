// Attention of a window's queries over the cached entries and the window
// itself (gfx950, wave64):
//
//   o = sum_j p_j v_j,  p = softmax_j(scale * q . k_j),  j in [0, n + r]
//
// for query r of a sequence with n cached entries.  One pass over the entries
// with the running maximum m and sum l of the softmax: an entry's score z
// above m rescales what was summed by exp(m - z).
#include "forward_common.h"

namespace specdec {
namespace {

constexpr uint32_t kBadPadIn = 0x1u, kBadSlot = 0x10u;
constexpr int kWaves = 4;

// One workgroup a query: its waves take the entries in turn, a lane holds
// four of the head's elements.
__global__ __launch_bounds__(64 * kWaves) void attend_simple_kernel(AttendLaunch p, int64_t first) {
  __shared__ float s_o[kWaves][256], s_m[kWaves], s_l[kWaves];
  __shared__ int32_t s_bad;
  const CacheView& c = p.cache;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t query = first + blockIdx.x;
  const int hq = static_cast<int>(query % p.Hq), h = hq / (p.Hq / c.H);
  const int r = static_cast<int>(query / p.Hq % p.T), i = static_cast<int>(query / p.Hq / p.T);
  const int32_t n = entries_before(c, i, p.T);
  if (tid == 0) s_bad = n < 0;
  __syncthreads();
  if (n >= 0 && c.table)
    for (int64_t t = tid; t <= (n + p.T - 1) / c.cap; t += 64 * kWaves) {
      const int32_t id = c.table[i * c.table_stride + t];
      if (id < 0 || id >= c.rows) s_bad = 1;
    }
  __syncthreads();
  if (s_bad) {
    if (tid == 0 && r == 0 && hq == 0 && p.dev_status) atomicOr(p.dev_status, c.table ? kBadSlot : kBadPadIn);
    return;
  }
  const int D = c.D, d = lane * 4;
  float q[4] = {}, o[4] = {}, m = -__builtin_inff(), l = 0.f;
  if (d < D) load_elements(static_cast<const __bf16*>(p.q) + query * D + d, q);
  const int64_t head = static_cast<int64_t>(h) * c.cap * D;
  for (int32_t j = wave; j <= n + r; j += kWaves) {
    const int64_t at = entry_offset(c, i, n, p.T, j) + head + d;
    float k[4] = {}, v[4] = {};
    if (d < D) {
      load_elements(static_cast<const __bf16*>(c.k) + at, k);
      load_elements(static_cast<const __bf16*>(c.v) + at, v);
    }
    float z = q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3];
    for (int x = 1; x < 64; x <<= 1) z += __shfl_xor(z, x);
    z *= p.scale;
    const float to = __builtin_fmaxf(m, z), base = to == -__builtin_inff() ? 0.f : to;
    const float keep = __expf(m - base), w = __expf(z - base);
    l = l * keep + w;
    for (int e = 0; e < 4; ++e) o[e] = o[e] * keep + w * v[e];
    m = to;
  }
  for (int e = 0; e < 4; ++e) s_o[wave][d + e] = o[e];
  s_m[wave] = m;
  s_l[wave] = l;
  __syncthreads();
  if (wave != 0 || d >= D) return;
  for (int w = 0; w < kWaves; ++w) m = __builtin_fmaxf(m, s_m[w]);
  const float base = m == -__builtin_inff() ? 0.f : m;
  float sum = 0.f, out[4] = {};
  for (int w = 0; w < kWaves; ++w) {
    const float f = __expf(s_m[w] - base);
    sum += f * s_l[w];
    for (int e = 0; e < 4; ++e) out[e] += f * s_o[w][d + e];
  }
  for (int e = 0; e < 4; ++e) out[e] /= sum;
  store_elements(static_cast<__bf16*>(p.out) + query * D + d, out);
}

}  // namespace

int64_t attend_workspace(int64_t, int64_t, int64_t, int64_t, int64_t, int64_t) { return 256; }

hipError_t launch_attend(const AttendLaunch& p, hipStream_t stream) {
  return launch_blocks(static_cast<int64_t>(p.B) * p.T * p.Hq, 64 * kWaves, [&](int64_t at, uint32_t n) {
    attend_simple_kernel<<<n, 64 * kWaves, 0, stream>>>(p, at);
  });
}

}  // namespace specdec
