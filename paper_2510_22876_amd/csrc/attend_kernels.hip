// Attention of a window's queries over the cached entries and the window
// itself (gfx950, wave64):
//
//   o = sum_j p_j v_j,  p = softmax_j(scale * q . k_j),  j in [0, n + r]
//
// for query r of a sequence with n cached entries.  The T * G queries that
// share a KV head (G query heads a KV head) are rows of one product, so that
// each key and value is read once for all of them; with 512 bytes of cache an
// entry of D = 128 against 4 * D operations a query the read bounds it.
//
// Layout.  A wave takes 32 entries at a time, two 16 x 16 x 32 products deep:
//   S^T = K Q^T   K is the left operand: lane (x, g) = (lane % 16, lane / 16)
//                 holds key x's elements 8g .. 8g+7 of each 32, 16 bytes as
//                 they lie in the cache.  The result has query x in the lane
//                 and entries 4g .. 4g+3 of either 16 in its registers, so the
//                 softmax's maximum and factors are per lane, and
//   O^T = V^T P^T takes the weights as its right operand where they are: the
//                 product sums over the entries, whose order is free, so place
//                 8g + j of the operands stands for entry 4g + j (j < 4) of
//                 the first 16 and 4g + j - 4 of the second.  V^T is the left
//                 operand: its row x of tile y is element x * (DP/16) + y of
//                 the head (again any order serves), so lane (x, g) needs
//                 DP/16 adjacent elements of its eight entries: a wave's load
//                 of one entry a lane group is whole rows, and the 8 x DP/16
//                 block is transposed in the lane's registers by byte
//                 permutes.  Neither keys nor values pass through LDS.
// The sum of the weights is one more product, with a left operand of ones.
//
// The running maximum is raised only when a score exceeds it by 2^8 (a wave's
// vote): until then the weights stay below 2^8 in fp32 and bf16 alike, and
// nothing has to be rescaled or exchanged between lanes.
//
// A workgroup's four waves take the 32-entry tiles of one chunk of one
// (sequence, KV head) in turn and are joined in LDS.  Where a sequence may
// have several chunks, each writes its fp32 sums, maximum and weight to the
// workspace and a second kernel joins them in a fixed order.
#include "forward_common.h"

namespace specdec {
namespace {

constexpr uint32_t kBadPadIn = 0x1u, kBadSlot = 0x10u;
constexpr int kWaves = 4;
constexpr int kTile = 32;                 // entries a wave takes at a time
constexpr int kMaxChunk = 2048;
constexpr float kLowest = -3.0e38f;       // the maximum of no score
constexpr float kSlack = 8.f;             // powers of two that a weight may exceed 1 by
constexpr float kBadRow = -1.f;           // a chunk's sum of weights: it has met a page outside the pool

struct AttendArgs {
  const __bf16* q;
  __bf16* out;
  float* part;            // [item][query rows][D] sums of a chunk, where a sequence has several
  float2* stat;           // [item][query rows] their maximum and weight
  CacheView c;
  uint32_t base;          // first workgroup of this launch
  int32_t T, Hq, G, M;    // M = T * G queries share a KV head
  uint32_t groups;        // of 16 * MT queries
  uint32_t splits, pairs; // chunks a sequence, (sequence, KV head) pairs
  int32_t chunk;          // entries
  float c2;               // scale * log2(e)
  uint32_t* dev_status;
};

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Whether either bf16 of a word is an infinity or NaN, as the words' bits that hold one.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  return ((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
}

template <int N> struct Words { uint32_t w[N]; };

// The operand of output tiles 2y and 2y + 1 from the words y of eight entries.
template <int kW>
__device__ __forceinline__ void transposed(const Words<kW> (&v)[8], int y, bf16x8* even, bf16x8* uneven) {
  uint32_t lo[4], hi[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    lo[j] = low_halves(v[2 * j].w[y], v[2 * j + 1].w[y]);
    hi[j] = high_halves(v[2 * j].w[y], v[2 * j + 1].w[y]);
  }
  __builtin_memcpy(even, lo, 16);
  __builtin_memcpy(uneven, hi, 16);
}

// Takes the infinities and NaN out of the values and adds them to the sums of
// the queries that attend to their entries (a weight above 0): a product of
// their places with the places of such weights says where there are any.
template <int MT, int kW>
__device__ __forceinline__ void add_not_finite(Words<kW> (&v)[8], const bf16x8 (&pf)[MT], f32x4 (&acc)[MT][2 * kW]) {
  bf16x8 on[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int j = 0; j < 8; ++j) on[t][j] = static_cast<__bf16>(static_cast<float>(pf[t][j]) != 0.f ? 1.f : 0.f);
#pragma unroll
  for (int kind = 0; kind < 3; ++kind) {   // +inf, -inf, NaN
    const float what = kind == 0 ? __builtin_inff() : kind == 1 ? -__builtin_inff() : __builtin_nanf("");
#pragma unroll
    for (int y = 0; y < kW; ++y) {
      Words<1> at[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        at[j].w[0] = 0;
#pragma unroll
        for (int b = 0; b < 32; b += 16) {
          const uint32_t x = v[j].w[y] >> b & 0xFFFFu;
          const bool is = kind == 0 ? x == 0x7F80u : kind == 1 ? x == 0xFF80u : (x & 0x7FFFu) > 0x7F80u;
          if (is) at[j].w[0] |= 0x3F80u << b;   // 1
        }
      }
      bf16x8 place[2];
      transposed<1>(at, 0, &place[0], &place[1]);
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const f32x4 found = __builtin_amdgcn_mfma_f32_16x16x32_bf16(place[b], on[t], f32x4{}, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (found[e] != 0.f) acc[t][2 * y + b][e] += what;
        }
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int y = 0; y < kW; ++y) v[j].w[y] &= ~not_finite(v[j].w[y]);
}

// Element offset of a sequence's entry 0 in the contiguous layouts (head 0),
// or -1 where its page is outside the pool.
__device__ __forceinline__ int64_t first_entry(const CacheView& c, int32_t i, int32_t n, int32_t T) {
  if (!c.table) return i * c.row_stride + static_cast<int64_t>(c.width - T - n) * c.D;
  const int32_t id = c.table[i * c.table_stride];
  return id < 0 || id >= c.rows ? -1 : id * c.row_stride;
}

// DP: the head size rounded up to 64, 128 or 256 (kFull: equal to it).
template <int DP, int MT, bool kPaged, bool kFull>
__global__ __launch_bounds__(64 * kWaves) void attend_kernel(AttendArgs a) {
  constexpr int kSteps = DP / 32;         // products along a head
  constexpr int kTiles = DP / 16;         // output tiles, and elements of an entry in a lane
  constexpr int kW = kTiles / 2;          // ... in words
  __shared__ float s_o[kWaves][16][DP];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  __shared__ int64_t s_at[kPaged ? kMaxChunk : 1];
  __shared__ int s_bad;
  const CacheView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), x = lane & 15, g = lane >> 4;
  // workgroups of the same entries go to the same XCD (every eighth)
  const uint32_t block = a.base + blockIdx.x, per = 8 * a.groups;
  const uint32_t item = block / per * 8 + block % 8, group = block % per / 8;
  if (item >= a.pairs * a.splits) return;
  const uint32_t split = item / a.pairs, pair = item - split * a.pairs;
  const int i = static_cast<int>(pair / c.H), h = static_cast<int>(pair - i * c.H);
  const int D = kFull ? DP : c.D;
  const int32_t n = entries_before(c, i, a.T);
  const bool joined = a.splits > 1;
  const int32_t c0 = static_cast<int32_t>(split) * a.chunk;
  if (n < 0) {
    if (!joined && h == 0 && group == 0 && tid == 0 && a.dev_status) atomicOr(a.dev_status, c.table ? kBadSlot : kBadPadIn);
    return;
  }
  if (c0 >= n + a.T) return;
  const int32_t c1 = c0 + a.chunk < n + a.T ? c0 + a.chunk : n + a.T;

  bool bad = false;
  int64_t first = 0;
  if constexpr (kPaged) {
    if (tid == 0) s_bad = 0;
    __syncthreads();
    const uint32_t P = static_cast<uint32_t>(c.cap);
    for (int32_t j = c0 + tid; j < c1; j += 64 * kWaves) {
      const uint32_t page = static_cast<uint32_t>(j) / P;
      const int32_t id = c.table[i * c.table_stride + page];
      if (id < 0 || id >= c.rows) s_bad = 1;
      s_at[j - c0] = id * c.row_stride + static_cast<int64_t>(static_cast<uint32_t>(j) - page * P) * D;
    }
    __syncthreads();
    bad = s_bad != 0;
  } else {
    first = first_entry(c, i, n, a.T);
    bad = first < 0;
  }
  const int m0 = static_cast<int>(group) * (16 * MT);
  if (bad) {
    if (joined) {
      if (m0 == 0 && tid == 0) a.stat[(static_cast<int64_t>(split) * a.pairs + pair) * a.M].y = kBadRow;
    } else if (h == 0 && group == 0 && tid == 0 && a.dev_status) {
      atomicOr(a.dev_status, kBadSlot);
    }
    return;
  }
  const __bf16* kp = static_cast<const __bf16*>(c.k) + static_cast<int64_t>(h) * c.cap * D;
  const __bf16* vp = static_cast<const __bf16*>(c.v) + static_cast<int64_t>(h) * c.cap * D;

  // the queries: row m = r * G + head of the group
  bf16x8 qf[MT][kSteps];
  int32_t last[MT];                       // the last entry that the lane's query attends to
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = m0 + t * 16 + x, r = m / a.G;
    last[t] = n + r;
    const __bf16* qp = a.q + ((static_cast<int64_t>(i) * a.T + r) * a.Hq + h * a.G + (m - r * a.G)) * D;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int d = s * 32 + g * 8;
      if (m < a.M && (kFull || d < D)) qf[t][s] = *reinterpret_cast<const bf16x8*>(qp + d);
      else qf[t][s] = bf16x8{};
    }
  }

  bf16x8 kf[2][kSteps];
  Words<kW> vf[8];
  // Entry `e` (an offset from the tile's first) of the tile at `key`; entries
  // behind the chunk's last stand for the last.
  auto entry = [&](int32_t key, int e) -> int64_t {
    const int32_t j = key + e < c1 ? key + e : c1 - 1;
    if constexpr (kPaged) return s_at[j - c0];
    else return first + static_cast<int64_t>(j) * D;
  };
  auto load_keys = [&](int32_t key) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const __bf16* p = kp + entry(key, t * 16 + x);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int d = s * 32 + g * 8;
        if (kFull || d < D) kf[t][s] = *reinterpret_cast<const bf16x8*>(p + d);
        else kf[t][s] = bf16x8{};
      }
    }
  };
  auto load_values = [&](int32_t key) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const __bf16* p = vp + entry(key, (j < 4 ? 0 : 12) + g * 4 + j) + x * kTiles;
      if (kFull || kTiles < 16) {
        if (kFull || x * kTiles < D) vf[j] = *reinterpret_cast<const Words<kW>*>(p);
        else vf[j] = Words<kW>{};
      } else {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int y = 0; y < kW / 2; ++y)
            vf[j].w[b * (kW / 2) + y] = x * kTiles + b * 8 < D ? reinterpret_cast<const uint32_t*>(p)[b * (kW / 2) + y] : 0u;
      }
    }
  };

  f32x4 acc[MT][kTiles], l[MT];
  float m[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    m[t] = kLowest;
    l[t] = f32x4{};
#pragma unroll
    for (int y = 0; y < kTiles; ++y) acc[t][y] = f32x4{};
  }
  bf16x8 ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = static_cast<__bf16>(1.f);

  int32_t key = c0 + wave * kTile;
  if (key < c1) {
    load_keys(key);
    load_values(key);
  }
  for (; key < c1; key += kWaves * kTile) {
    const int32_t next = key + kWaves * kTile;
    const bool border = key + kTile > n + 1 || key + kTile > c1;   // holds entries that not every query attends to
    f32x4 z[MT][2];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        z[t][b] = f32x4{};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) z[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[b][s], qf[t][s], z[t][b], 0, 0, 0);
      }
    if (next < c1) load_keys(next);

    bf16x8 pf[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = z[t][j >> 2][j & 3] * a.c2;
      if (border) {
        const int32_t end = last[t] < c1 - 1 ? last[t] : c1 - 1;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (key + (j < 4 ? 0 : 12) + g * 4 + j > end) w[j] = -__builtin_inff();
      }
      float top = w[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) top = __builtin_fmaxf(top, w[j]);
      if (__any(top > m[t] + kSlack)) {
        top = __builtin_fmaxf(top, __shfl_xor(top, 16));
        top = __builtin_fmaxf(top, __shfl_xor(top, 32));
        top = __builtin_fmaxf(top, m[t]);
        const float keep = __builtin_amdgcn_exp2f(m[t] - top);
        m[t] = top;
        l[t] *= keep;
#pragma unroll
        for (int y = 0; y < kTiles; ++y) acc[t][y] *= keep;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) pf[t][j] = static_cast<__bf16>(__builtin_amdgcn_exp2f(w[j] - m[t]));
      l[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[t], l[t], 0, 0, 0);
    }

    if (border) {
      // A weight of 0 does not silence an infinity or NaN among the values of
      // entries that some queries do not attend to.
      uint32_t odd = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int y = 0; y < kW; ++y) odd |= not_finite(vf[j].w[y]);
      if (__any(odd != 0)) add_not_finite<MT, kW>(vf, pf, acc);
    }

#pragma unroll
    for (int y = 0; y < kW; ++y) {
      bf16x8 even, uneven;
      transposed<kW>(vf, y, &even, &uneven);
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        acc[t][2 * y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, pf[t], acc[t][2 * y], 0, 0, 0);
        acc[t][2 * y + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(uneven, pf[t], acc[t][2 * y + 1], 0, 0, 0);
      }
    }
    if (next < c1) load_values(next);
  }

  // Join the waves, 16 queries at a time: a thread sums kTiles elements of one
  // query.  Rows of s_o are turned by four elements a query against bank
  // conflicts.
  const int row = tid >> 4, d0 = (tid & 15) * kTiles;
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    __syncthreads();
    if (g == 0) {
      s_m[wave][x] = m[t];
      s_l[wave][x] = l[t][0];
    }
    __syncthreads();
    float top = s_m[0][x];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = __builtin_fmaxf(top, s_m[w][x]);
    const float f = __builtin_amdgcn_exp2f(m[t] - top);
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int y = 0; y < kTiles; y += 4) {
        const f32x4 v = {acc[t][y][b] * f, acc[t][y + 1][b] * f, acc[t][y + 2][b] * f, acc[t][y + 3][b] * f};
        *reinterpret_cast<f32x4*>(&s_o[wave][x][((g * 4 + b) * kTiles + y + 4 * x) & (DP - 1)]) = v;
      }
    __syncthreads();
    const int q = m0 + t * 16 + row;
    if (q >= a.M) continue;
    float best = s_m[0][row], sum = 0.f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) best = __builtin_fmaxf(best, s_m[w][row]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += s_l[w][row] * __builtin_amdgcn_exp2f(s_m[w][row] - best);
    f32x4 o[kTiles / 4];
#pragma unroll
    for (int y = 0; y < kTiles / 4; ++y) {
      o[y] = f32x4{};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) o[y] += *reinterpret_cast<const f32x4*>(&s_o[w][row][(d0 + 4 * y + 4 * row) & (DP - 1)]);
    }
    if (joined) {
      const int64_t at = (static_cast<int64_t>(split) * a.pairs + pair) * a.M + q;
      if ((tid & 15) == 0) a.stat[at] = float2{best, sum};
#pragma unroll
      for (int y = 0; y < kTiles / 4; ++y)
        if (kFull || d0 + 4 * y < D) *reinterpret_cast<f32x4*>(a.part + at * D + d0 + 4 * y) = o[y];
    } else {
      const int r = q / a.G;
      __bf16* to = a.out + ((static_cast<int64_t>(i) * a.T + r) * a.Hq + h * a.G + (q - r * a.G)) * D + d0;
      const float inv = 1.f / sum;
#pragma unroll
      for (int y = 0; y < kTiles / 4; ++y) {
        if (!kFull && d0 + 4 * y >= D) continue;
        const float v[4] = {o[y][0] * inv, o[y][1] * inv, o[y][2] * inv, o[y][3] * inv};
        store_elements(to + 4 * y, v);
      }
    }
  }
}

// Joins a query's chunks: a group of D/4 lanes sums every kThreads/(D/4)-th
// chunk, then the groups are summed in their order.
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendArgs a) {
  __shared__ f32x4 s_o[kThreads];
  __shared__ float s_m[kThreads], s_l[kThreads];
  const CacheView& c = a.c;
  const uint32_t row = a.base + blockIdx.x, pair = row / a.M;
  const int q = static_cast<int>(row - pair * a.M), i = static_cast<int>(pair / c.H), h = static_cast<int>(pair - i * c.H);
  const int tid = threadIdx.x, D = c.D, lanes = D / 4, parts = kThreads / lanes, part = tid / lanes, d = tid % lanes * 4;
  const int32_t n = entries_before(c, i, a.T);
  const int chunks = n < 0 ? 0 : (n + a.T + a.chunk - 1) / a.chunk;
  int bad = n < 0;
  for (int s = tid; s < chunks; s += kThreads) bad |= a.stat[(static_cast<int64_t>(s) * a.pairs + pair) * a.M].y == kBadRow;
  if (__syncthreads_or(bad)) {
    if (h == 0 && q == 0 && tid == 0 && a.dev_status) atomicOr(a.dev_status, c.table ? kBadSlot : kBadPadIn);
    return;
  }
  float m = kLowest, l = 0.f;
  f32x4 o = {};
  if (part < parts)
    for (int s = part; s < chunks; s += parts) {
      const int64_t at = (static_cast<int64_t>(s) * a.pairs + pair) * a.M + q;
      const float2 t = a.stat[at];
      const f32x4 v = *reinterpret_cast<const f32x4*>(a.part + at * D + d);
      const float top = __builtin_fmaxf(m, t.x), keep = __builtin_amdgcn_exp2f(m - top), f = __builtin_amdgcn_exp2f(t.x - top);
      l = l * keep + t.y * f;
      o = o * keep + v * f;
      m = top;
    }
  s_o[tid] = o;
  s_m[tid] = m;
  s_l[tid] = l;
  __syncthreads();
  if (part != 0) return;
  for (int p = 1; p < parts; ++p) m = __builtin_fmaxf(m, s_m[p * lanes]);
  o = f32x4{};
  l = 0.f;
  for (int p = 0; p < parts; ++p) {
    const float f = __builtin_amdgcn_exp2f(s_m[p * lanes] - m);
    l += s_l[p * lanes] * f;
    o += s_o[p * lanes + tid] * f;
  }
  const int r = q / a.G;
  const float inv = 1.f / l, v[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  store_elements(a.out + ((static_cast<int64_t>(i) * a.T + r) * a.Hq + h * a.G + (q - r * a.G)) * D + d, v);
}

// How a call is split: tiles of 16 queries a workgroup, groups of them, and
// the entries of a chunk.
struct Plan {
  int tiles;
  int64_t groups, chunk, splits;
};
Plan plan_of(int64_t B, int64_t T, int64_t Hq, int64_t H, int64_t D, int64_t max_len) {
  Plan p;
  const int64_t M = T * (Hq / H), most = D > 128 ? 2 : 4;
  p.tiles = M <= 16 ? 1 : M <= 32 || most == 2 ? 2 : 4;
  p.groups = (M + 16 * p.tiles - 1) / (16 * p.tiles);
  const int64_t blocks = B * H * p.groups;
  p.chunk = 256;
  while (p.chunk < kMaxChunk && blocks * ((max_len + 2 * p.chunk - 1) / (2 * p.chunk)) >= 1024) p.chunk *= 2;
  p.splits = (max_len + p.chunk - 1) / p.chunk;
  return p;
}

template <int DP, int MT>
void launch_tiles(const AttendArgs& a, bool paged, uint32_t blocks, hipStream_t stream) {
  const bool full = a.c.D == DP;
  if (paged && full) attend_kernel<DP, MT, true, true><<<blocks, 64 * kWaves, 0, stream>>>(a);
  else if (paged) attend_kernel<DP, MT, true, false><<<blocks, 64 * kWaves, 0, stream>>>(a);
  else if (full) attend_kernel<DP, MT, false, true><<<blocks, 64 * kWaves, 0, stream>>>(a);
  else attend_kernel<DP, MT, false, false><<<blocks, 64 * kWaves, 0, stream>>>(a);
}

}  // namespace

int64_t attend_workspace(int64_t B, int64_t T, int64_t Hq, int64_t H, int64_t D, int64_t max_len) {
  const Plan p = plan_of(B, T, Hq, H, D, max_len);
  return 256 + (p.splits > 1 ? p.splits * B * T * Hq * (D * 4 + 8) : 0);
}

hipError_t launch_attend(const AttendLaunch& p, hipStream_t stream) {
  const CacheView& c = p.cache;
  const Plan plan = plan_of(p.B, p.T, p.Hq, c.H, c.D, c.width);
  AttendArgs a{};
  a.q = static_cast<const __bf16*>(p.q);
  a.out = static_cast<__bf16*>(p.out);
  a.c = c;
  a.T = p.T;
  a.Hq = p.Hq;
  a.G = p.Hq / c.H;
  a.M = p.T * a.G;
  a.groups = static_cast<uint32_t>(plan.groups);
  a.splits = static_cast<uint32_t>(plan.splits);
  a.pairs = static_cast<uint32_t>(p.B * c.H);
  a.chunk = static_cast<int32_t>(plan.chunk);
  a.c2 = p.scale * 1.4426950408889634f;
  a.dev_status = p.dev_status;
  a.part = static_cast<float*>(p.workspace);
  a.stat = reinterpret_cast<float2*>(a.part + plan.splits * a.pairs * a.M * c.D);
  const bool paged = c.table && c.cap < c.width;
  const int64_t items = plan.splits * a.pairs, blocks = (items + 7) / 8 * 8 * plan.groups;
  hipError_t e = launch_blocks(blocks, 64 * kWaves, [&](int64_t at, uint32_t count) {
    a.base = static_cast<uint32_t>(at);
    if (c.D <= 64) {
      if (plan.tiles == 1) launch_tiles<64, 1>(a, paged, count, stream);
      else if (plan.tiles == 2) launch_tiles<64, 2>(a, paged, count, stream);
      else launch_tiles<64, 4>(a, paged, count, stream);
    } else if (c.D <= 128) {
      if (plan.tiles == 1) launch_tiles<128, 1>(a, paged, count, stream);
      else if (plan.tiles == 2) launch_tiles<128, 2>(a, paged, count, stream);
      else launch_tiles<128, 4>(a, paged, count, stream);
    } else {
      if (plan.tiles == 1) launch_tiles<256, 1>(a, paged, count, stream);
      else launch_tiles<256, 2>(a, paged, count, stream);
    }
  });
  if (e != hipSuccess || plan.splits == 1) return e;
  return launch_blocks(static_cast<int64_t>(a.pairs) * a.M, kThreads, [&](int64_t at, uint32_t count) {
    a.base = static_cast<uint32_t>(at);
    attend_join_kernel<<<count, kThreads, 0, stream>>>(a);
  });
}

}  // namespace specdec
