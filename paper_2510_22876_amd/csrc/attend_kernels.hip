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
// The second product's operands are bf16, so the weights are rounded to it, and
// their sum is taken of the rounded ones: an error of the size that the
// result's own rounding has.  Root mean square against 64 bits, relative:
// 0.0016 (one query of 1000 entries) to 0.0022 (windows of 5 to 8 over
// thousands), where the rounding of the result alone gives 0.0017.  With one
// more product, of what the rounding left off, it is 0.0017 throughout, but the
// cases below take 0.5 to 1% longer, and 4.5% with three tiles of queries (64
// windows of 5: 86.0 -> 89.9 us), the time of the products.
//
// The running maximum is raised only when a score exceeds it by 2^8 (a wave's
// vote): until then the weights stay below 2^8 in fp32 and bf16 alike, and
// nothing has to be rescaled or exchanged between lanes.
//
// Split.  A workgroup takes one piece of one (sequence, KV head) pair; its
// waves take the piece's tiles in turn and are joined in LDS.  The size of a
// piece follows from the batch's entries, known on the device only: every
// workgroup scans the lengths, finds the piece that is its own, and leaves if
// there is none.  Of a pair of several pieces each one's fp32 sums, maximum
// and weight go to the workspace and a second kernel joins them in their
// order.  Short sequences, and batches of many pairs, are not cut: a workgroup
// a pair, no scan and no second kernel.
//
// Figures (us of both kernels, and TB/s of the bytes that must be read and
// written; plain reads reach 6.2).  One query of 32 + 8 heads over 1000
// entries, 16 a page: 7.4 + 4.3.  Whole pairs, 8 windows of 6, 32 + 32 heads,
// 128 to 1024 entries: 15.4 and 3.9; its longest pair is 527 KB, of which a
// workgroup reads 50 KB a us.  Cut, 32 windows of 8, 32 + 8 heads, 64 to 4096
// entries, 64 a page: 40.0 + 5.0 and 3.7; 64 windows of 5, 28 + 4 heads, 512 to
// 8192 entries: 81.2 + 5.3 and 4.3; one window of 6 over 150001 entries: 107.5
// + 5.1 and 5.4.  The matrix products of these three would take 4.5, 11.5 and
// 13 us: what is left is uneven pieces, their starts and ends, and the second
// launch.
#include "forward_common.h"
#include <type_traits>

namespace specdec {
namespace {

constexpr uint32_t kBadPadIn = 0x1u, kBadSlot = 0x10u;
constexpr int kWaves = 4;
constexpr int kTile = 32;                 // entries a wave takes at a time
constexpr int kMaxCutB = 1024;            // sequences that a workgroup scans
constexpr uint32_t kLeastPiece = 4;       // tiles
constexpr uint32_t kCus = 256;
constexpr int kJoinAhead = 4;             // pieces that a group of lanes of the join reads at a time
constexpr float kLowest = -3.0e38f;       // the maximum of no score
constexpr float kSlack = 8.f;             // powers of two that a weight may exceed 1 by
constexpr float kBadPiece = -1.f;         // a piece's sum of weights: it has met a page outside the pool

struct AttendArgs {
  const __bf16* q;
  __bf16* out;
  float* part;            // [slot][M][D] sums of pieces
  float2* stat;           // [slot][M] their maximum and weight
  int2* plan;             // [B] a sequence's first slot and its pieces (a head)
  CacheView c;
  uint32_t base;          // first workgroup of this launch
  int32_t B, T, Hq, G, M; // M = T * G queries share a KV head
  uint32_t groups;        // of 16 * MT queries
  uint32_t items;         // workgroups a group
  uint32_t pieces;        // pieces that the batch's entries are cut into, about (0: pairs are not cut)
  uint32_t joined;        // pieces of a pair that the join reads at a time
  float c2;               // scale * log2(e)
  uint32_t* dev_status;
};

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Per half of a word of two bf16: bit 15 says whether it is an infinity or NaN.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return (w & 0x7F807F80u) + 0x00800080u; }
// ... whether it equals the half `k`.
__device__ __forceinline__ uint32_t equals(uint32_t w, uint32_t k) {
  const uint32_t y = w ^ (k | k << 16);
  return ~(((y & 0x7FFF7FFFu) + 0x7FFF7FFFu) | y);
}
// `value` in the halves whose bit 15 is set, 0 in the others.
__device__ __forceinline__ uint32_t where(uint32_t bits, uint32_t value) { return (bits >> 15 & 0x00010001u) * value; }

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
#pragma unroll 1
  for (int kind = 0; kind < 3; ++kind) {   // +inf, -inf, NaN
    const float what = kind == 0 ? __builtin_inff() : kind == 1 ? -__builtin_inff() : __builtin_nanf("");
#pragma unroll
    for (int y = 0; y < kW; ++y) {
      Words<1> at[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t w = v[j].w[y];
        asm volatile("" : "+v"(w));   // not computed for all kinds and words ahead: a rare path gets no registers
        const uint32_t is = kind == 2 ? not_finite(w) & ~equals(w & 0x7FFF7FFFu, 0x7F80u)
                                                     : equals(w, kind ? 0xFF80u : 0x7F80u);
        at[j].w[0] = where(is, 0x3F80u);   // 1
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
    for (int y = 0; y < kW; ++y) v[j].w[y] &= ~where(not_finite(v[j].w[y]), 0xFFFFu);
}

// Element offset of a sequence's entry 0 in the contiguous layouts (head 0),
// or -1 where its page is outside the pool.
__device__ __forceinline__ int64_t first_entry(const CacheView& c, int32_t i, int32_t n, int32_t T) {
  if (!c.table) return i * c.row_stride + static_cast<int64_t>(c.width - T - n) * c.D;
  const int32_t id = c.table[i * c.table_stride];
  return id < 0 || id >= c.rows ? -1 : id * c.row_stride;
}

// Bytes of LDS: the waves' sums, maxima and weights; the places of a paged
// sequence's entries; the queries where registers do not hold them.
constexpr bool queries_in_lds(int DP, int MT) { return MT > 1 || DP > 128; }
constexpr int lds_bytes(int DP, int MT, bool paged) {
  return kWaves * 16 * (DP + 2) * 4 + (queries_in_lds(DP, MT) ? MT * 16 * DP * 2 : 0) + (paged ? kWaves * 2 * kTile * 4 : 0);
}

// A piece of a pair: tiles [tile, stop) of `tiles`, and the place of its sums
// where the pair has several.
struct Piece {
  int32_t i, h, n;
  uint32_t tile, stop, tiles;
  int32_t slot;
};

// Op over the lanes up to this one, in the last lane over the wave; 0 is op's
// neutral element.
template <class Op>
__device__ __forceinline__ uint32_t wave_scan(uint32_t v, Op op) {
  auto step = [&](auto how, auto rows) {
    v = op(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), decltype(how)::value, decltype(rows)::value, 0xF, false)));
  };
  using std::integral_constant;
  step(integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});   // one lane to the right in each 16,
  step(integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});   // two,
  step(integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});   // four,
  step(integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});   // eight;
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});   // the 16's last lane to the next 16,
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});   // the lower half's to the upper
  return v;
}
__device__ __forceinline__ uint32_t wave_last(uint32_t v) { return __builtin_amdgcn_readlane(v, 63); }

// Finds the workgroup's piece by a scan of the sequences.  Pieces have at most
// `most` tiles, a multiple of kLeastPiece; a sequence of more has as many equal
// ones as that takes.  The join takes as long as four tiles for every a.joined
// pieces of a pair, so that a pair of `top` tiles is best cut into pieces of no
// fewer than sqrt(4 * top / a.joined) (1521 to 30429 entries in three pairs of
// one query: 14.0 us, 17.1 in pieces of four tiles).
// Unequal sequences of `t` tiles in all: most = t / a.pieces, rounded up, or
// that bound, so that there are at most a.pieces + pairs pieces, 2 * a.pieces
// of cut pairs.
// About equal ones: the pairs get as many pieces each as lets the CU with the
// most of them end first, a piece counted as kLeastPiece tiles more than it has
// for what it begins and ends with, the join as above, and a.pieces pieces at
// most in all (35 x 2 KV heads of 256, window 5, 3762 to 4180 entries: 70 us,
// where about 256 pieces, four a pair, leave 24 CUs with a second one and take
// 96).
// False: no piece is left for this workgroup.
__device__ __forceinline__ bool find_piece(const AttendArgs& a, uint32_t item, bool first, Piece* p) {
  constexpr int kEach = kMaxCutB / kThreads;
  __shared__ uint32_t s_sum[kWaves], s_top[kWaves], s_pieces[kWaves], s_cut[kWaves];
  __shared__ Piece s_piece;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t n[kEach];
  uint32_t tiles[kEach], sum = 0, top = 0;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int i = tid * kEach + e;
    n[e] = i < a.B ? entries_before(a.c, i, a.T) : -1;
    tiles[e] = n[e] < 0 ? 0u : static_cast<uint32_t>(n[e] + a.T + kTile - 1) / kTile;
    sum += tiles[e];
    top = top > tiles[e] ? top : tiles[e];
    if (first && i < a.B && n[e] < 0 && a.dev_status) atomicOr(a.dev_status, a.c.table ? kBadSlot : kBadPadIn);
  }
  const auto add = [](uint32_t x, uint32_t y) { return x + y; };
  const auto larger = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
  sum = wave_last(wave_scan(sum, add));
  top = wave_last(wave_scan(top, larger));
  if (lane == 0) {
    s_sum[wave] = sum;
    s_top[wave] = top;
  }
  if (tid == 0) s_piece.i = -1;
  __syncthreads();
  sum = top = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    sum += s_sum[w];
    top = top > s_top[w] ? top : s_top[w];
  }
  const uint64_t all = static_cast<uint64_t>(sum) * a.c.H;
  const bool even = static_cast<uint64_t>(top) * a.B * 8 <= static_cast<uint64_t>(sum) * 9;
  uint32_t most;
  if (even) {   // a lane a number of pieces, the fewest of the best
    const uint32_t pairs = static_cast<uint32_t>(a.B * a.c.H), step = 1 + kCus / (64 * pairs), each = (lane + 1) * step;
    const uint32_t size = ((top + each - 1) / each + kLeastPiece - 1) / kLeastPiece * kLeastPiece;
    const uint32_t rounds = (pairs * each * a.groups + kCus - 1) / kCus;
    const uint64_t time = static_cast<uint64_t>(rounds) * (size + kLeastPiece) + 4 * each / a.joined;
    constexpr uint32_t kNever = (1u << 26) - 1;
    const uint32_t cost = (each == step || pairs * each <= a.pieces) && time < kNever ? static_cast<uint32_t>(time) : kNever;
    const uint32_t best = ~wave_last(wave_scan(~(cost << 6 | static_cast<uint32_t>(lane)), larger));
    most = __builtin_amdgcn_readlane(size, best & 63);
  } else {
    const uint32_t share = static_cast<uint32_t>((all + a.pieces - 1) / a.pieces);
    const uint32_t least = static_cast<uint32_t>(__builtin_amdgcn_sqrtf(4.f * static_cast<float>(top) / static_cast<float>(a.joined)));
    most = ((share > least ? share : least) + kLeastPiece - 1) / kLeastPiece * kLeastPiece;
  }
  uint32_t mine[kEach], pieces = 0, cut = 0, at[kEach], cut_at[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    mine[e] = most ? (tiles[e] + most - 1) / most : 0u;
    at[e] = pieces;
    cut_at[e] = cut;
    pieces += mine[e];
    cut += mine[e] > 1 ? mine[e] : 0u;
  }
  const uint32_t pieces_to = wave_scan(pieces, add), cut_to = wave_scan(cut, add);
  if (lane == 63) {
    s_pieces[wave] = pieces_to;
    s_cut[wave] = cut_to;
  }
  __syncthreads();
  uint32_t before = pieces_to - pieces, cut_before = cut_to - cut;
  for (int w = 0; w < wave; ++w) {
    before += s_pieces[w];
    cut_before += s_cut[w];
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int i = tid * kEach + e;
    if (i >= a.B) break;
    const uint64_t from = static_cast<uint64_t>(before + at[e]) * a.c.H;
    const uint32_t slot = (cut_before + cut_at[e]) * static_cast<uint32_t>(a.c.H);
    if (first) a.plan[i] = int2{static_cast<int>(slot), static_cast<int>(mine[e])};
    if (item >= from && item - from < static_cast<uint64_t>(mine[e]) * a.c.H) {
      const uint32_t in = static_cast<uint32_t>(item - from), h = in / mine[e], s = in - h * mine[e];
      const uint32_t size = ((tiles[e] + mine[e] - 1) / mine[e] + kLeastPiece - 1) / kLeastPiece * kLeastPiece;
      const uint32_t stop = (s + 1) * size < tiles[e] ? (s + 1) * size : tiles[e];
      s_piece = Piece{i, static_cast<int32_t>(h), n[e], s * size, stop, tiles[e], static_cast<int32_t>(slot + in)};
    }
  }
  __syncthreads();
  *p = s_piece;
  return s_piece.i >= 0;
}

// DP: the head size rounded up to 64, 128 or 256 (kFull: equal to it).
template <int DP, int MT, bool kPaged, bool kFull>
__global__ __launch_bounds__(kThreads, DP > 128 && MT > 1 ? 1 : 2) void attend_kernel(AttendArgs a) {
  constexpr int kSteps = DP / 32;         // products along a head
  constexpr int kTiles = DP / 16;         // output tiles, and elements of an entry in a lane
  constexpr int kW = kTiles / 2;          // ... in words
  constexpr bool kLdsQ = queries_in_lds(DP, MT);
  extern __shared__ __attribute__((aligned(16))) char s_mem[];
  const int tid = threadIdx.x, lane = tid & 63, x = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  float* s_o = reinterpret_cast<float*>(s_mem);             // [waves][16][DP]
  float* s_m = s_o + kWaves * 16 * DP;                       // [waves][16]
  float* s_l = s_m + kWaves * 16;
  bf16x8* s_q = reinterpret_cast<bf16x8*>(s_l + kWaves * 16);   // [MT][kSteps][64]
  uint32_t* s_at = reinterpret_cast<uint32_t*>(s_q + (kLdsQ ? MT * kSteps * 64 : 0)) + wave * 2 * kTile;   // [2][kTile]
  const CacheView& c = a.c;
  const int D = kFull ? DP : c.D;
  // workgroups of the same entries go to the same XCD (every eighth)
  const uint32_t block = a.base + blockIdx.x, per = 8 * a.groups;
  const uint32_t item = block / per * 8 + block % 8, group = block % per / 8;
  if (item >= a.items) return;
  const int m0 = static_cast<int>(group) * (16 * MT);

  Piece p;
  if (a.pieces) {
    if (!find_piece(a, item, item == 0 && group == 0, &p)) return;
  } else {
    p.i = static_cast<int>(item / c.H);
    p.h = static_cast<int>(item - static_cast<uint32_t>(p.i) * c.H);
    p.n = entries_before(c, p.i, a.T);
    if (p.n < 0) {
      if (p.h == 0 && group == 0 && tid == 0 && a.dev_status) atomicOr(a.dev_status, c.table ? kBadSlot : kBadPadIn);
      return;
    }
    p.tile = 0;
    p.stop = p.tiles = static_cast<uint32_t>(p.n + a.T + kTile - 1) / kTile;
  }
  const int i = __builtin_amdgcn_readfirstlane(p.i), h = __builtin_amdgcn_readfirstlane(p.h);
  const int32_t n = __builtin_amdgcn_readfirstlane(p.n);
  const bool whole = __builtin_amdgcn_readfirstlane(p.tile == 0 && p.stop == p.tiles);
  const int32_t c0 = __builtin_amdgcn_readfirstlane(static_cast<int32_t>(p.tile)) * kTile;
  int32_t c1 = __builtin_amdgcn_readfirstlane(static_cast<int32_t>(p.stop)) * kTile;
  if (c1 > n + a.T) c1 = n + a.T;

  // the queries: row m = r * G + head of the group
  constexpr int kOwn = kLdsQ ? 1 : MT;    // tiles of queries in the wave's registers
  bf16x8 qf[kOwn][kSteps];
  int32_t last[MT];                       // the last entry that the lane's query attends to
#pragma unroll
  for (int b = 0; b < MT; ++b) last[b] = n + (m0 + b * 16 + x) / a.G;
  auto load_queries = [&](int b, bf16x8 (&to)[kSteps]) {
    const int m = m0 + b * 16 + x, r = m / a.G;
    const __bf16* qp = a.q + ((static_cast<int64_t>(i) * a.T + r) * a.Hq + h * a.G + (m - r * a.G)) * D;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int d = s * 32 + g * 8;
      to[s] = bf16x8{};
      if (m < a.M && (kFull || d < D)) to[s] = *reinterpret_cast<const bf16x8*>(qp + d);
    }
  };
  if constexpr (kLdsQ) {
    if (wave < MT) load_queries(wave, qf[0]);
  } else {
#pragma unroll
    for (int b = 0; b < MT; ++b) load_queries(b, qf[b]);
  }

  const int64_t head = static_cast<int64_t>(h) * c.cap * D;
  bool bad = false;
  const __bf16 *kp = static_cast<const __bf16*>(c.k) + head, *vp = static_cast<const __bf16*>(c.v) + head;
  if constexpr (!kPaged) {
    const int64_t first = first_entry(c, i, n, a.T);
    bad = first < 0;   // no entry is read then
    if (bad) c1 = c0;
    kp += first;
    vp += first;
  }

  f32x4 acc[MT][kTiles], l[MT];
  float m[MT];
#pragma unroll
  for (int b = 0; b < MT; ++b) {
    m[b] = kLowest;
    l[b] = f32x4{};
#pragma unroll
    for (int y = 0; y < kTiles; ++y) acc[b][y] = f32x4{};
  }
  bf16x8 ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = static_cast<__bf16>(1.f);

  // Places of a paged sequence's entries, in entries of the pool from kp and vp
  // on: a wave looks those of a tile up two tiles ahead, an entry a lane, and
  // keeps them in its part of LDS.  Places behind the last entry stand for the
  // last.  An entry whose page is outside the pool stands for the first page.
  const uint32_t P = static_cast<uint32_t>(c.cap);
  struct Place {
    int32_t id;
    uint32_t col;
  };
  auto look_up = [&](int32_t key) {
    const int32_t e = key + (lane & (kTile - 1));
    const uint32_t j = static_cast<uint32_t>(e < c1 ? e : c1 - 1), page = j / P;
    return Place{c.table[i * c.table_stride + page], j - page * P};
  };
  auto keep_places = [&](const Place& place, int which) {
    const bool in = place.id >= 0 && place.id < c.rows;
    bad |= !in;
    if (lane < kTile) s_at[which * kTile + lane] = (in ? static_cast<uint32_t>(place.id) : 0u) * (static_cast<uint32_t>(c.H) * P) + place.col;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };

  bf16x8 kf[2][kSteps];
  Words<kW> vf[8];
  auto load_keys = [&](int32_t key, int which) {
    const __bf16* base = kp + (kPaged ? 0 : static_cast<int64_t>(key) * D);
    const int32_t most = c1 - 1 - key;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int e = b * 16 + x;
      const __bf16* src;
      if constexpr (kPaged) src = base + static_cast<uint64_t>(s_at[which * kTile + e]) * static_cast<uint32_t>(D) + g * 8;
      else src = base + ((e < most ? e : most) * D + g * 8);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        kf[b][s] = bf16x8{};
        if (kFull || s * 32 + g * 8 < D) kf[b][s] = *reinterpret_cast<const bf16x8*>(src + s * 32);
      }
    }
  };
  auto load_values = [&](int32_t key, int which) {
    const __bf16* base = vp + (kPaged ? 0 : static_cast<int64_t>(key) * D);
    const int32_t most = c1 - 1 - key;
    uint4 at[2];
    if constexpr (kPaged) {
      at[0] = *reinterpret_cast<const uint4*>(&s_at[which * kTile + g * 4]);
      at[1] = *reinterpret_cast<const uint4*>(&s_at[which * kTile + 16 + g * 4]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = (j < 4 ? 0 : 12) + g * 4 + j;
      const __bf16* src;
      if constexpr (kPaged) {
        const uint4 f = at[j >> 2];
        const uint32_t row = (j & 3) == 0 ? f.x : (j & 3) == 1 ? f.y : (j & 3) == 2 ? f.z : f.w;
        src = base + static_cast<uint64_t>(row) * static_cast<uint32_t>(D) + x * kTiles;
      } else {
        src = base + ((e < most ? e : most) * D + x * kTiles);
      }
      if (kFull || kTiles < 16) {
        vf[j] = Words<kW>{};
        if (kFull || x * kTiles < D) vf[j] = *reinterpret_cast<const Words<kW>*>(src);
      } else {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int y = 0; y < kW / 2; ++y)
            vf[j].w[b * (kW / 2) + y] = x * kTiles + b * 8 < D ? reinterpret_cast<const uint32_t*>(src)[b * (kW / 2) + y] : 0u;
      }
    }
  };
  // One tile.  All but a wave's last tile hold entries that every query
  // attends to (a window is shorter than four waves' tiles), and its last
  // tile has no next one to load.
  auto tile = [&](int32_t key, int32_t next, int which, auto is_last) {
    constexpr bool kLast = decltype(is_last)::value;
    bf16x8 pf[MT];
#pragma unroll
    for (int b = 0; b < MT; ++b) {
      if constexpr (kLdsQ) {
        asm volatile("" ::: "memory");    // read again for every tile: the registers would not hold them
#pragma unroll
        for (int s = 0; s < kSteps; ++s) qf[0][s] = s_q[(b * kSteps + s) * 64 + lane];
      }
      f32x4 z[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        z[e] = f32x4{};
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
          z[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[e][s], qf[kLdsQ ? 0 : b][s], z[e], 0, 0, 0);
      }
      if (!kLast && b == MT - 1) load_keys(next, which);
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = z[j >> 2][j & 3] * a.c2;
      if (kLast) {
        const int32_t most = (last[b] < c1 - 1 ? last[b] : c1 - 1) - key;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if ((j < 4 ? 0 : 12) + g * 4 + j > most) w[j] = -__builtin_inff();
      }
      float top = w[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) top = __builtin_fmaxf(top, w[j]);
      if (__any(top > m[b] + kSlack)) {
        top = __builtin_fmaxf(top, __shfl_xor(top, 16));
        top = __builtin_fmaxf(top, __shfl_xor(top, 32));
        top = __builtin_fmaxf(top, m[b]);
        const float keep = __builtin_amdgcn_exp2f(m[b] - top);
        m[b] = top;
        l[b] *= keep;
#pragma unroll
        for (int y = 0; y < kTiles; ++y) acc[b][y] *= keep;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) pf[b][j] = static_cast<__bf16>(__builtin_amdgcn_exp2f(w[j] - m[b]));
      l[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[b], l[b], 0, 0, 0);
    }
    if (kLast) {
      // A weight of 0 does not silence an infinity or NaN among the values of
      // entries that some queries do not attend to.
      uint32_t odd = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int y = 0; y < kW; ++y) odd |= not_finite(vf[j].w[y]);
      if (__any((odd & 0x80008000u) != 0)) add_not_finite<MT, kW>(vf, pf, acc);
    }
#pragma unroll
    for (int y = 0; y < kW; ++y) {
      bf16x8 even, uneven;
      transposed<kW>(vf, y, &even, &uneven);
#pragma unroll
      for (int b = 0; b < MT; ++b) {
        acc[b][2 * y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, pf[b], acc[b][2 * y], 0, 0, 0);
        acc[b][2 * y + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(uneven, pf[b], acc[b][2 * y + 1], 0, 0, 0);
      }
    }
    if (!kLast) load_values(next, which);
  };

  int32_t key = c0 + wave * kTile;
  constexpr int32_t stride = kWaves * kTile;
  if (key < c1) {
    if constexpr (kPaged) {
      const Place one = look_up(key), two = look_up(key + stride);
      keep_places(one, 0);
      keep_places(two, 1);
    }
    load_keys(key, 0);
    load_values(key, 0);
  }
  if constexpr (kLdsQ) {
    if (wave < MT)
#pragma unroll
      for (int s = 0; s < kSteps; ++s) s_q[(wave * kSteps + s) * 64 + lane] = qf[0][s];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  }
  if (key < c1) {
    int which = 0;                        // of the two places, the current tile's
    for (; key + stride < c1; key += stride) {
      Place place{};
      if constexpr (kPaged) place = look_up(key + 2 * stride);
      tile(key, key + stride, which ^ 1, std::false_type{});
      if constexpr (kPaged) {
        keep_places(place, which);
        which ^= 1;
      }
    }
    tile(key, key, which, std::true_type{});
  }
  if constexpr (kPaged) bad = __syncthreads_or(bad);

  if (bad) {
    if (whole) {
      if (h == 0 && group == 0 && tid == 0 && a.dev_status) atomicOr(a.dev_status, kBadSlot);
    } else if (group == 0 && tid == 0) {
      a.stat[static_cast<int64_t>(p.slot) * a.M].y = kBadPiece;
    }
    return;
  }
  // Join the waves, 16 queries at a time: 16 threads sum a query's elements,
  // kTiles each.  Rows of s_o are turned by four elements a query against bank
  // conflicts.
  const int row = tid >> 4, d0 = (tid & 15) * kTiles;
#pragma unroll
  for (int b = 0; b < MT; ++b) {
    if (b > 0) __syncthreads();
    if (g == 0) {
      s_m[wave * 16 + x] = m[b];
      s_l[wave * 16 + x] = l[b][0];
    }
    __syncthreads();
    float top = m[b];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = __builtin_fmaxf(top, s_m[w * 16 + x]);
    const float f = __builtin_amdgcn_exp2f(m[b] - top);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int y = 0; y < kTiles; y += 4) {
        const f32x4 v = {acc[b][y][e] * f, acc[b][y + 1][e] * f, acc[b][y + 2][e] * f, acc[b][y + 3][e] * f};
        *reinterpret_cast<f32x4*>(&s_o[(wave * 16 + x) * DP + (((g * 4 + e) * kTiles + y + 4 * x) & (DP - 1))]) = v;
      }
    __syncthreads();
    const int q = m0 + b * 16 + row;
    if (q >= a.M) continue;
    float best = kLowest, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) best = __builtin_fmaxf(best, s_m[w * 16 + row]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += s_l[w * 16 + row] * __builtin_amdgcn_exp2f(s_m[w * 16 + row] - best);
    f32x4 o[kTiles / 4];
#pragma unroll
    for (int y = 0; y < kTiles / 4; ++y) {
      o[y] = f32x4{};
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        o[y] += *reinterpret_cast<const f32x4*>(&s_o[(w * 16 + row) * DP + ((d0 + 4 * y + 4 * row) & (DP - 1))]);
    }
    if (whole) {
      const int r = q / a.G;
      __bf16* dst = a.out + ((static_cast<int64_t>(i) * a.T + r) * a.Hq + h * a.G + (q - r * a.G)) * D + d0;
      const float inv = 1.f / sum;
#pragma unroll
      for (int y = 0; y < kTiles / 4; ++y) {
        if (!kFull && d0 + 4 * y >= D) continue;
        const float v[4] = {o[y][0] * inv, o[y][1] * inv, o[y][2] * inv, o[y][3] * inv};
        store_elements(dst + 4 * y, v);
      }
    } else {
      const int64_t at = static_cast<int64_t>(p.slot) * a.M + q;
      if ((tid & 15) == 0) a.stat[at] = float2{best, sum};
#pragma unroll
      for (int y = 0; y < kTiles / 4; ++y)
        if (kFull || d0 + 4 * y < D) *reinterpret_cast<f32x4*>(a.part + at * D + d0 + 4 * y) = o[y];
    }
  }
}

// Joins the pieces of a pair.  `parts` groups of `lanes` lanes take a query's
// pieces in turn and are summed in their order; a workgroup takes `rows`
// queries.  3 to 5 us: a launch, and the waits for the plan, the statistics and
// the sums in turn.  Joined by the pair's last workgroup in the first kernel
// instead, pairs of many pieces or queries took longer.
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendArgs a, uint32_t lanes, uint32_t parts, uint32_t rows) {
  constexpr int kAhead = kJoinAhead;
  __shared__ f32x4 s_o[kThreads];
  __shared__ float s_m[kThreads], s_l[kThreads];
  const CacheView& c = a.c;
  const uint32_t block = a.base + blockIdx.x;
  const uint32_t per = (a.M + rows - 1) / rows, pair = block / per, first = (block - pair * per) * rows;
  const int i = static_cast<int>(pair / c.H), h = static_cast<int>(pair - i * c.H), D = c.D;
  const int2 plan = a.plan[i];
  const int pieces = plan.y;
  if (pieces < 2) return;
  const int64_t slot = plan.x + static_cast<int64_t>(h) * pieces;
  const uint32_t tid = threadIdx.x, d = tid % lanes * 4, part = tid / lanes % parts, row = tid / lanes / parts;
  const uint32_t q = first + row;
  const bool live = row < rows && q < static_cast<uint32_t>(a.M) && d < static_cast<uint32_t>(D);
  float m = kLowest, l = 0.f;
  f32x4 o = {};
  int bad = 0;
  if (live) {
    // kAhead pieces are read before the first is waited for; places behind the
    // last stand for the first of these, with no weight
    for (int s = part; s < pieces; s += parts * kAhead) {
      float2 t[kAhead];
      f32x4 v[kAhead];
      float flag[kAhead];
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        const int at = s + e * static_cast<int>(parts);
        const int64_t piece = slot + (at < pieces ? at : s);
        flag[e] = a.stat[piece * a.M].y;
        t[e] = a.stat[piece * a.M + q];
        v[e] = *reinterpret_cast<const f32x4*>(a.part + (piece * a.M + q) * D + d);
      }
      float top = m;
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        if (s + e * static_cast<int>(parts) >= pieces) {
          t[e] = float2{kLowest, 0.f};
          v[e] = f32x4{};
        }
        bad |= flag[e] == kBadPiece;
        top = __builtin_fmaxf(top, t[e].x);
      }
      const float keep = __builtin_amdgcn_exp2f(m - top);
      l *= keep;
      o *= keep;
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        const float f = __builtin_amdgcn_exp2f(t[e].x - top);
        l += t[e].y * f;
        o += v[e] * f;
      }
      m = top;
    }
  }
  if (__syncthreads_or(bad)) {
    if (h == 0 && first == 0 && tid == 0 && a.dev_status) atomicOr(a.dev_status, kBadSlot);
    return;
  }
  if (parts > 1) {
    s_o[tid] = o;
    s_m[tid] = m;
    s_l[tid] = l;
    __syncthreads();
    if (part != 0) return;
    for (uint32_t p = 1; p < parts; ++p) m = __builtin_fmaxf(m, s_m[tid + p * lanes]);
    o = f32x4{};
    l = 0.f;
    for (uint32_t p = 0; p < parts; ++p) {
      const float f = __builtin_amdgcn_exp2f(s_m[tid + p * lanes] - m);
      l += s_l[tid + p * lanes] * f;
      o += s_o[tid + p * lanes] * f;
    }
  }
  if (!live) return;
  const int r = static_cast<int>(q) / a.G;
  const float inv = 1.f / l, v[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  store_elements(a.out + ((static_cast<int64_t>(i) * a.T + r) * a.Hq + h * a.G + (static_cast<int>(q) - r * a.G)) * D + d, v);
}

// How a call is divided: tiles of 16 queries a workgroup and groups of them,
// workgroups a group, and the pieces that the batch's entries are cut into
// (0: pairs are not cut).
constexpr int64_t kLeastCut = 320 * 1024;        // bytes of the shortest pair that is cut
constexpr int64_t kMostPieces = 2 * kCus, kFewestPieces = 8;   // kMostPieces over the groups, and no fewer than these
int64_t most_tiles(int64_t D) { return D > 128 ? 2 : 3; }
int64_t pair_bytes(int64_t D, int64_t max_len) { return max_len * (D > 128 ? D : 128) * 4; }
struct Plan {
  int tiles;
  int64_t groups, items, pieces, slots;
};
Plan plan_of(int64_t B, int64_t T, int64_t Hq, int64_t H, int64_t D, int64_t max_len) {
  Plan p;
  const int64_t tiles = (T * (Hq / H) + 15) / 16, most = most_tiles(D), pairs = B * H;
  p.groups = (tiles + most - 1) / most;
  p.tiles = static_cast<int>((tiles + p.groups - 1) / p.groups);
  // A workgroup reads about 50 KB a microsecond (smaller heads than 128 do not
  // make a tile faster), so a pair of 1000 entries of 512 bytes takes some 13
  // us uncut; the scan and the second kernel cost 7.  Where the CUs are busy
  // with other pairs a longer one may stay whole (Vicuna-7B's batch of 8, 256
  // pairs of at most 1030 entries: 16.1 us whole, 19.5 cut; 8 pairs of 1001:
  // 13.7 and 11.6).
  const bool cut = pair_bytes(D, max_len) > (pairs >= kCus / 2 ? 768 * 1024 : kLeastCut) && B <= kMaxCutB && pairs <= 4096;
  // Pieces of unequal sequences: 3/2 a CU (64 of 512 to 8192, 256 pairs: 104 us
  // with 1, 91 with 3/2, 98 with 2), more where few pairs add their number.
  const int64_t wanted = pairs > kCus / 2 ? kMostPieces * 3 / 4 : kMostPieces;
  p.pieces = !cut ? 0 : p.groups >= wanted / kFewestPieces ? kFewestPieces : wanted / p.groups;
  p.items = pairs + p.pieces;
  p.slots = 2 * p.pieces;
  return p;
}

template <int DP, int MT>
void launch_tiles(const AttendArgs& a, bool paged, uint32_t blocks, hipStream_t stream) {
  const bool full = a.c.D == DP;
  const int lds = lds_bytes(DP, MT, paged);
  if (paged && full) attend_kernel<DP, MT, true, true><<<blocks, kThreads, lds, stream>>>(a);
  else if (paged) attend_kernel<DP, MT, true, false><<<blocks, kThreads, lds, stream>>>(a);
  else if (full) attend_kernel<DP, MT, false, true><<<blocks, kThreads, lds, stream>>>(a);
  else attend_kernel<DP, MT, false, false><<<blocks, kThreads, lds, stream>>>(a);
}

}  // namespace

// Enough for the call and, with the same heads, for every one of fewer
// sequences, queries or entries, though these may be cut into more pieces: of
// the slots' 2 * pieces * M rows (M queries a pair), pieces * M is at most
// kFewestPieces * M, or kMostPieces times the queries that a workgroup takes.
int64_t attend_workspace(int64_t B, int64_t T, int64_t Hq, int64_t H, int64_t D, int64_t max_len) {
  const int64_t M = T * (Hq / H), once = 16 * most_tiles(D);
  const int64_t spread = kMostPieces * (M < once ? M : once), fewest = kFewestPieces * M;
  const int64_t rows = pair_bytes(D, max_len) > kLeastCut ? 2 * (spread > fewest ? spread : fewest) : 0;
  return (8 * B + 255) / 256 * 256 + rows * (D * 4 + 8) + 256;
}

hipError_t launch_attend(const AttendLaunch& p, hipStream_t stream) {
  const CacheView& c = p.cache;
  const Plan plan = plan_of(p.B, p.T, p.Hq, c.H, c.D, c.width);
  AttendArgs a{};
  a.q = static_cast<const __bf16*>(p.q);
  a.out = static_cast<__bf16*>(p.out);
  a.c = c;
  a.B = p.B;
  a.T = p.T;
  a.Hq = p.Hq;
  a.G = p.Hq / c.H;
  a.M = p.T * a.G;
  a.groups = static_cast<uint32_t>(plan.groups);
  a.items = static_cast<uint32_t>(plan.items);
  a.pieces = static_cast<uint32_t>(plan.pieces);
  a.c2 = p.scale * 1.4426950408889634f;
  a.dev_status = p.dev_status;
  a.plan = static_cast<int2*>(p.workspace);
  a.part = reinterpret_cast<float*>(static_cast<char*>(p.workspace) + (8 * static_cast<int64_t>(p.B) + 255) / 256 * 256);
  a.stat = reinterpret_cast<float2*>(a.part + plan.slots * a.M * c.D);
  const bool paged = c.table && c.cap < c.width;
  // few queries: a workgroup each, so that many pieces are read at a time; many: several a workgroup
  uint32_t lanes = 1;
  while (lanes * 4 < static_cast<uint32_t>(c.D)) lanes *= 2;
  const int64_t pairs = static_cast<int64_t>(p.B) * c.H;
  const uint32_t slots = kThreads / lanes, parts = pairs * a.M <= 2048 ? slots : 1, rows = slots / parts;
  a.joined = parts * kJoinAhead;
  const int64_t blocks = (plan.items + 7) / 8 * 8 * plan.groups;
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
  const hipError_t e = launch_blocks(blocks, kThreads, [&](int64_t at, uint32_t count) {
    a.base = static_cast<uint32_t>(at);
    if (c.D <= 64) {
      if (plan.tiles == 1) launch_tiles<64, 1>(a, paged, count, stream);
      else if (plan.tiles == 2) launch_tiles<64, 2>(a, paged, count, stream);
      else launch_tiles<64, 3>(a, paged, count, stream);
    } else if (c.D <= 128) {
      if (plan.tiles == 1) launch_tiles<128, 1>(a, paged, count, stream);
      else if (plan.tiles == 2) launch_tiles<128, 2>(a, paged, count, stream);
      else launch_tiles<128, 3>(a, paged, count, stream);
    } else {
      if (plan.tiles == 1) launch_tiles<256, 1>(a, paged, count, stream);
      else launch_tiles<256, 2>(a, paged, count, stream);
    }
  });
  if (e != hipSuccess || !plan.pieces) return e;
  return launch_blocks(pairs * ((a.M + rows - 1) / rows), kThreads, [&](int64_t at, uint32_t count) {
    a.base = static_cast<uint32_t>(at);
    attend_join_kernel<<<count, kThreads, 0, stream>>>(a, lanes, parts, rows);
  });
}

}  // namespace specdec
