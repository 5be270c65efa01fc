// Norms of queries and keys, position rotation and append of a window's keys
// and values to the cache, in one pass over the projections (gfx950, wave64).
//
//   y = x / sqrt(mean(x^2) + eps) * w            per head, queries and keys
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t)   per rotated pair,
//   t = position * inv_freq_j, position = entries before the window + r (I2)
//
// A workgroup takes one token, or a share of its heads where there are few
// tokens; a group of lanes (8 elements a lane) takes a head after the other.
// A lane meets the same elements of every head, so it keeps their weights,
// cosines and sines in registers; the other half of a pair comes through LDS,
// within the wave.  The next head is read while one is worked on, the first
// before anything else.  Everything is fp32 from the load to one rounding at
// the store.  The angle is formed in revolutions in fp64: at a position of
// 2^24 an fp32 product would be off by up to half a radian.
//
// Bounds and figures.  Few tokens: the waits in turn for length, page and row;
// 4.6 us for one token of 32 + 16 heads of 128 on pages, 5.0 us for 48 tokens
// of 32 + 64 heads (a call takes 5.4 either way).  Many: bytes; 64 windows of
// 33 tokens, 28 + 8 heads of 128 in fp32, 58 MB, 13.3 to 13.4 us a call among
// others, 4.4 TB/s, the rate of a large copy (12.8 to 15.9 under the profiler).
// With a workgroup a few heads of any token and the angles in LDS it took 22.8.
#include "forward_common.h"

#include <type_traits>

namespace specdec {
namespace {

constexpr uint32_t kBadPadIn = 0x1u, kBadSlot = 0x10u;
constexpr int kMaxHalf = 128;
// A head whose mean square lies outside [2^-96, 2^96] may have squares that
// fp32 does not hold, and the root takes no subnormal: it is multiplied by a
// power of two first.  Bits of the least such mean, and of the range from it on.
constexpr uint32_t kLeastMean = 0x0F800000u, kMeans = 0x60000000u;

struct AppendArgs {
  AppendLaunch p;
  int64_t base;           // first workgroup of this launch
  uint32_t shares;        // workgroups a token
  uint32_t lanes;         // lanes a head (a power of two)
  float per_element;      // 1 / D
};

// The sum over a group of up to 32 lanes, in all of them: DPP moves within 16
// lanes (neighbours, pairs, mirrored eights and sixteens), where a shuffle
// through LDS a step would wait for each.
__device__ __forceinline__ float group_sum(float x, uint32_t lanes) {
  auto moved = [](float v, auto how) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(how)::value, 0xF, 0xF, true));
  };
  if (lanes >= 2) x += moved(x, std::integral_constant<int, 0xB1>{});    // quad_perm 1 0 3 2
  if (lanes >= 4) x += moved(x, std::integral_constant<int, 0x4E>{});    // quad_perm 2 3 0 1
  if (lanes >= 8) x += moved(x, std::integral_constant<int, 0x141>{});   // row_half_mirror
  if (lanes >= 16) x += moved(x, std::integral_constant<int, 0x140>{});  // row_mirror
  if (lanes >= 32) x += __shfl_xor(x, 16);
  return x;
}

// Six waves a SIMD (80 registers): with five, 64 windows of 33 take 14.1 us
// instead of 13.4.
template <int kDtype>
__global__ __launch_bounds__(kThreads, 6) void append_kernel(AppendArgs a) {
  typedef typename Element<kDtype>::type T;
  __shared__ float s_cos[kMaxHalf], s_sin[kMaxHalf];
  __shared__ __align__(16) float s_row[kThreads * 8];
  const AppendLaunch& p = a.p;
  const CacheView& c = p.cache;
  const int64_t block = a.base + blockIdx.x;
  const int token = static_cast<int>(block / a.shares), share = static_cast<int>(block % a.shares);
  const int i = token / p.T, r = token % p.T, tid = threadIdx.x;
  const int groups = kThreads / a.lanes, group = tid / a.lanes, d0 = tid % a.lanes * 8;
  const int D = c.D, heads = p.Hq + 2 * c.H, step = groups * a.shares;
  const bool live = d0 < D;
  const T* x0 = static_cast<const T*>(p.qkv) + static_cast<int64_t>(token) * heads * D + d0;
  int h = share * groups + group;
  float next[8] = {};
  if (live && h < heads) load_elements(x0 + static_cast<int64_t>(h) * D, next);
  float gq[8], gk[8];
  if (p.q_norm && live) load_elements(static_cast<const T*>(p.q_norm) + d0, gq);
  if (p.k_norm && live) load_elements(static_cast<const T*>(p.k_norm) + d0, gk);

  // Where the token's entry lies.  The pages are looked up here and judged
  // after the angles: one wait for memory less in a call of a single token.
  const int32_t n = entries_before(c, i, p.T);
  const int32_t* table = c.table + i * c.table_stride;
  const uint32_t P = static_cast<uint32_t>(c.cap);
  int32_t page = 0, first = 0, last = 0;
  if (n >= 0 && c.table) {
    page = load_invariant(table + static_cast<uint32_t>(n + r) / P);
    first = load_invariant(table + static_cast<uint32_t>(n) / P);
    last = load_invariant(table + static_cast<uint32_t>(n + p.T - 1) / P);
  }
  if (tid < p.half) {
    const double turns = static_cast<double>(n + r) * static_cast<double>(p.inv_freq[tid]) * 0.15915494309189535;
    sincospif(2.f * static_cast<float>(turns - __builtin_rint(turns)), &s_sin[tid], &s_cos[tid]);
  }
  // every page that the window's entries lie in has to be one of the pool's
  auto outside = [&](int32_t id) { return id < 0 || id >= c.rows; };
  bool bad = n < 0;
  if (!bad && c.table) {
    bad = outside(first) || outside(last);
    for (uint32_t q = static_cast<uint32_t>(n) / P + 1; q < static_cast<uint32_t>(n + p.T - 1) / P; ++q)
      bad = bad || outside(load_invariant(table + q));
  }
  if (bad) {
    if (r == 0 && share == 0 && tid == 0 && p.dev_status) atomicOr(p.dev_status, c.table ? kBadSlot : kBadPadIn);
    return;
  }
  const int64_t entry = c.table ? page * c.row_stride + static_cast<int64_t>(static_cast<uint32_t>(n + r) % P) * D
                                : i * c.row_stride + (static_cast<int64_t>(c.width) - p.T + r) * D;
  __syncthreads();
  // x = x * cs + partner * sn for the lane's first `turned` elements; the others
  // stay as they are, and no infinity or NaN among them reaches another
  float cs[8], sn[8];
  const int beyond = 2 * p.half - d0, turned = beyond < 0 ? 0 : beyond;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int d = d0 + e;
    cs[e] = 1.f;
    sn[e] = 0.f;
    if (d < 2 * p.half) {
      const bool second = p.adjacent ? (e & 1) != 0 : d >= p.half;
      const int j = p.adjacent ? d >> 1 : second ? d - p.half : d;
      cs[e] = s_cos[j];
      sn[e] = second ? s_sin[j] : -s_sin[j];
    }
  }
  float* row = s_row + group * a.lanes * 8;
  while (h - group < heads) {   // the same count for every group of the workgroup
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = next[e];
    const int at = h;
    h += step;
    if (live && h < heads) load_elements(x0 + static_cast<int64_t>(h) * D, next);
    const bool query = at < p.Hq, key = !query && at < p.Hq + c.H;
    if (query ? p.q_norm != nullptr : key && p.k_norm) {
      auto mean = [&](float eps) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
        return group_sum(sum, a.lanes) * a.per_element + eps;
      };
      float m = mean(p.eps);
      const bool far = __float_as_uint(m) - kLeastMean > kMeans;
      if (__any(far)) {
        const float scale = m < 1.f ? 0x1p100f : 0x1p-100f;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= far ? scale : 1.f;
        const float again = mean(p.eps * scale * scale);
        m = far ? again : m;
      }
      const float inv = __builtin_amdgcn_rsqf(m);   // about 1 ulp
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * (query ? gq[e] : gk[e]);
    }
    if (p.adjacent) {
      if (query || key) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float y = x[e], z = x[e + 1];
          x[e] = e < turned ? y * cs[e] + z * sn[e] : y;
          x[e + 1] = e < turned ? z * cs[e + 1] + y * sn[e + 1] : z;
        }
      }
    } else if (p.half > 0) {
      // the group's lanes lie in one wave: its LDS accesses keep their order
      if (live && (query || key)) {
        *reinterpret_cast<f32x4*>(row + d0) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4*>(row + d0 + 4) = f32x4{x[4], x[5], x[6], x[7]};
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (live && turned > 0 && (query || key)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int d = d0 + e, other = d >= 2 * p.half ? d : d < p.half ? d + p.half : d - p.half;
          x[e] = e < turned ? x[e] * cs[e] + row[other] * sn[e] : x[e];
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    if (!live || at >= heads) continue;
    __bf16* to;
    if (query) {
      to = static_cast<__bf16*>(p.q_out) + (static_cast<int64_t>(token) * p.Hq + at) * D;
    } else {
      const int g = at - p.Hq;
      to = static_cast<__bf16*>(key ? c.k : c.v) + entry + static_cast<int64_t>(key ? g : g - c.H) * c.cap * D;
    }
    store_elements(to + d0, x);
  }
}

}  // namespace

hipError_t launch_append(const AppendLaunch& p, hipStream_t stream) {
  AppendArgs a{p, 0, 1, 1, 1.f / static_cast<float>(p.cache.D)};
  while (a.lanes * 8 < static_cast<uint32_t>(p.cache.D)) a.lanes *= 2;
  const uint32_t groups = kThreads / a.lanes, heads = static_cast<uint32_t>(p.Hq + 2 * p.cache.H);
  // few tokens: the heads go to several workgroups, so that the call waits for fewer heads in turn
  const int64_t tokens = static_cast<int64_t>(p.B) * p.T, wanted = (1024 + tokens - 1) / tokens, most = (heads + groups - 1) / groups;
  a.shares = static_cast<uint32_t>(wanted < most ? wanted : most);
  return launch_blocks(static_cast<int64_t>(p.B) * p.T * a.shares, kThreads, [&](int64_t at, uint32_t n) {
    a.base = at;
    if (p.dtype == 0) append_kernel<0><<<n, kThreads, 0, stream>>>(a);
    else if (p.dtype == 1) append_kernel<1><<<n, kThreads, 0, stream>>>(a);
    else append_kernel<2><<<n, kThreads, 0, stream>>>(a);
  });
}

}  // namespace specdec
