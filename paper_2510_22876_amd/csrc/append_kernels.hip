// Norms of queries and keys, position rotation and append of a window's keys
// and values to the cache, in one pass over the projections (gfx950, wave64).
//
//   y = x / sqrt(mean(x^2) + eps) * w            per head, queries and keys
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t)   per rotated pair,
//   t = position * inv_freq_j, position = entries before the window + r (I2)
//
// A workgroup takes one token and a share of its heads; a group of lanes
// (8 elements a lane) takes a head.  Everything is fp32 from the load to one
// rounding at the store.  The angle is formed in revolutions in fp64: at a
// position of 2^24 an fp32 product would be off by up to half a radian.
#include "forward_common.h"

namespace specdec {
namespace {

constexpr uint32_t kBadPadIn = 0x1u, kBadSlot = 0x10u;
constexpr int kMaxHalf = 128;

struct AppendArgs {
  AppendLaunch p;
  int64_t base;           // first workgroup of this launch
  uint32_t shares;        // workgroups a token
  uint32_t lanes;         // lanes a head (a power of two)
};

template <int kDtype>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  typedef typename Element<kDtype>::type T;
  __shared__ float s_cos[kMaxHalf], s_sin[kMaxHalf];
  __shared__ float s_row[kThreads * 8];
  const AppendLaunch& p = a.p;
  const CacheView& c = p.cache;
  const int64_t block = a.base + blockIdx.x;
  const int token = static_cast<int>(block / a.shares), share = static_cast<int>(block % a.shares);
  const int i = token / p.T, r = token % p.T, tid = threadIdx.x;
  const int32_t n = entries_before(c, i, p.T);
  bool ok = n >= 0;
  if (ok && c.table) {   // every page that the window's entries lie in
    for (int64_t q = n / c.cap; q <= (n + p.T - 1) / c.cap; ++q) {
      const int32_t id = c.table[i * c.table_stride + q];
      ok = ok && id >= 0 && id < c.rows;
    }
  }
  if (!ok) {
    if (r == 0 && share == 0 && tid == 0 && p.dev_status) atomicOr(p.dev_status, c.table ? kBadSlot : kBadPadIn);
    return;
  }
  for (int j = tid; j < p.half; j += kThreads) {
    const double turns = static_cast<double>(n + r) * static_cast<double>(p.inv_freq[j]) * 0.15915494309189535;
    sincospif(2.f * static_cast<float>(turns - __builtin_rint(turns)), &s_sin[j], &s_cos[j]);
  }
  __syncthreads();
  const int groups = kThreads / a.lanes, group = tid / a.lanes, lane = tid % a.lanes;
  const int D = c.D, heads = p.Hq + 2 * c.H, d0 = lane * 8;
  const T* x0 = static_cast<const T*>(p.qkv) + static_cast<int64_t>(token) * heads * D;
  const int64_t entry = entry_offset(c, i, n, p.T, n + r);
  for (int first = share * groups; first < heads; first += groups * a.shares) {   // the same count for every group
    const int h = first + group;
    const bool live = h < heads && d0 < D, turned = h < p.Hq + c.H;
    float x[8] = {};
    if (live) load_elements(x0 + static_cast<int64_t>(h) * D + d0, x);
    const T* w = static_cast<const T*>(h < p.Hq ? p.q_norm : p.k_norm);
    if (w && turned) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
      for (uint32_t m = 1; m < a.lanes; m <<= 1) sum += __shfl_xor(sum, m);
      const float inv = 1.0f / __builtin_sqrtf(sum / static_cast<float>(D) + p.eps);
      if (live) {
        float g[8];
        load_elements(w + d0, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * g[e];
      }
    }
    float* row = s_row + group * a.lanes * 8;
    if (live && turned)
#pragma unroll
      for (int e = 0; e < 8; ++e) row[d0 + e] = x[e];
    __syncthreads();
    if (live && turned) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int d = d0 + e;
        if (d >= 2 * p.half) continue;
        const int j = p.adjacent ? d >> 1 : d < p.half ? d : d - p.half;
        const bool second = p.adjacent ? (d & 1) != 0 : d >= p.half;
        const float y = row[p.adjacent ? d ^ 1 : second ? d - p.half : d + p.half];
        x[e] = second ? x[e] * s_cos[j] + y * s_sin[j] : x[e] * s_cos[j] - y * s_sin[j];
      }
    }
    __syncthreads();
    if (!live) continue;
    __bf16* to;
    if (h < p.Hq) {
      to = static_cast<__bf16*>(p.q_out) + (static_cast<int64_t>(token) * p.Hq + h) * D;
    } else {
      const int g = h - p.Hq;
      to = static_cast<__bf16*>(g < c.H ? c.k : c.v) + entry + static_cast<int64_t>(g < c.H ? g : g - c.H) * c.cap * D;
    }
    store_elements(to + d0, x);
  }
}

}  // namespace

hipError_t launch_append(const AppendLaunch& p, hipStream_t stream) {
  AppendArgs a{p, 0, 1, 1};
  while (a.lanes * 8 < static_cast<uint32_t>(p.cache.D)) a.lanes *= 2;
  const uint32_t groups = kThreads / a.lanes, heads = static_cast<uint32_t>(p.Hq + 2 * p.cache.H);
  a.shares = (heads + groups - 1) / groups;
  return launch_blocks(static_cast<int64_t>(p.B) * p.T * a.shares, kThreads, [&](int64_t at, uint32_t n) {
    a.base = at;
    if (p.dtype == 0) append_kernel<0><<<n, kThreads, 0, stream>>>(a);
    else if (p.dtype == 1) append_kernel<1><<<n, kThreads, 0, stream>>>(a);
    else append_kernel<2><<<n, kThreads, 0, stream>>>(a);
  });
}

}  // namespace specdec
