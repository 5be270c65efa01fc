// Penalties for repeated tokens, biases and grammar masks on the logits of a
// verify window, ahead of verification (gfx950, wave64).  For logit x of token
// v in window slot r, with n(v) the occurrences of v among the answered tokens
// and the drafts before slot r, and held(v) whether v occurs at all (prompt
// included):
//
//   x = held ? (x > 0 ? x / repetition : x * repetition) : x
//   x = x - (frequency * n + presence * [n > 0])
//   x = x + bias(v)
//   x = allowed(v) ? x : -inf
//
// Reading and writing the logits bounds it; few of them change but for the
// mask.  A workgroup takes one sequence, one chunk of the vocabulary and some
// of the window's slots.  It counts its chunk's tokens once, in LDS, and turns
// the counts and biases of a lane's logits into what is taken off and added,
// in registers, for all the slots; a lane then takes 8 logits at a time as
// they lie in memory and copies or masks as bits those that no count or bias
// touches.  A drafted token's count grows from slot to slot: such logits are
// computed again from the counts.
//
// Figures.  32 windows of 8, 128256 logits in bf16, all penalties, 64 biases, a
// mask that allows nine tenths, histories of 64 to 4096: 32.5 us a call among
// others for 136 MB, 4.2 TB/s (32.3 to 36.4 under the profiler); a plain copy of
// the logits takes 25.9, and so does this kernel with nothing to change, 27.3
// with the mask.  In place with a mask that allows a twentieth, 64 windows of
// 5, 151936 logits: 34.0 us; four fifths of the 64-byte lines hold an allowed
// logit and are read.  1000 logits, or one row of 128256: 5 to 6 us, the waits
// for lengths, tokens and logits in turn.  Every workgroup reads the whole
// history: six slots of 128256 after 150001 tokens take 49 us.
#include "forward_common.h"
#include "span_copy.h"
#include "specdec.h"

namespace specdec {
namespace {

constexpr uint32_t kBadPadIn = 0x1u, kEmptyMask = 0x80u;
constexpr uint32_t kPrompt = 0x80000000u;   // the token occurs in the prompt; the low bits count the answered ones

struct LogitsArgs {
  LogitsLaunch p;
  int64_t base;      // first workgroup of this launch
  int64_t checks;    // workgroups ahead of the others that look for masks that allow nothing
  int64_t chunks;    // of the vocabulary
  int32_t shares;    // workgroups that a window's slots are shared out to
  int32_t slots;     // ... each
};

// Whether mask row `row` allows a token of the vocabulary; one wave.
__device__ __forceinline__ void check_mask(const LogitsLaunch& p, int64_t row) {
  const uint32_t* mask = p.mask + row * p.mask_stride;
  const int64_t words = (static_cast<int64_t>(p.V) + 31) / 32;
  const int lane = threadIdx.x & 63;
  const uint32_t end = p.V % 32 ? (1u << p.V % 32) - 1u : ~0u;   // of the last word
  for (int64_t w = lane; w - lane < words; w += 64 * 16) {
    uint32_t any = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t at = w + e * 64;
      const uint32_t bits = mask[at < words ? at : words - 1];
      any |= at < words - 1 ? bits : bits & end;
    }
    if (__any(any != 0)) return;
  }
  if (lane == 0 && p.dev_status) atomicOr(p.dev_status, kEmptyMask);
}

// 8 logits as they lie in memory, as words.  Units are passed by value and
// their words selected, not indexed, so that they stay in registers.
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
typedef uint32_t Words8 __attribute__((ext_vector_type(8)));
template <typename T> struct UnitOf { typedef Words4 type; };
template <> struct UnitOf<float> { typedef Words8 type; };
template <typename T> using Unit = typename UnitOf<T>::type;

template <typename T>
__device__ __forceinline__ Unit<T> load_unit(const T* p) {
  Unit<T> u;
  __builtin_memcpy(&u, p, sizeof(u));
  return u;
}
template <typename T>
__device__ __forceinline__ void store_unit(T* p, Unit<T> u) { __builtin_memcpy(p, &u, sizeof(u)); }

// Logit e of a unit, and its replacement.
template <typename T>
__device__ __forceinline__ float take(Unit<T> u, int e) {
  constexpr int kWords = sizeof(T) * 2;
  const int at = sizeof(T) == 4 ? e : e >> 1;
  uint32_t w = u[0];
#pragma unroll
  for (int y = 1; y < kWords; ++y) w = at == y ? u[y] : w;
  if constexpr (sizeof(T) == 4) return __uint_as_float(w);
  else return static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(e & 1 ? w >> 16 : w)));
}
template <typename T>
__device__ __forceinline__ Unit<T> give(Unit<T> u, int e, float z) {
  constexpr int kWords = sizeof(T) * 2;
  const int at = sizeof(T) == 4 ? e : e >> 1;
  uint32_t w, keep = 0;
  if constexpr (sizeof(T) == 4) {
    w = __float_as_uint(z);
  } else {
    w = __builtin_bit_cast(uint16_t, static_cast<T>(z));
    keep = e & 1 ? 0xFFFFu : 0xFFFF0000u;
    w = e & 1 ? w << 16 : w;
  }
#pragma unroll
  for (int y = 0; y < kWords; ++y) u[y] = at == y ? (u[y] & keep) | w : u[y];
  return u;
}
// All of a unit's logits, and those of them whose bit is set replaced.
template <typename T>
__device__ __forceinline__ void widen(Unit<T> u, float (&z)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = take<T>(u, e);
}
template <typename T>
__device__ __forceinline__ Unit<T> replaced(Unit<T> u, const float (&z)[8], uint32_t bits) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t keep = ~static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(bits), e, 1));
    if constexpr (sizeof(T) == 4) {
      u[e] = (u[e] & keep) | (__float_as_uint(z[e]) & ~keep);
    } else {
      const uint32_t half = e & 1 ? 0xFFFF0000u : 0xFFFFu, w = static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<T>(z[e]))) << (e & 1) * 16;
      u[e >> 1] = (u[e >> 1] & (keep | ~half)) | (w & ~keep);
    }
  }
  return u;
}
// -inf where bit e of `allowed` is clear.
template <typename T>
__device__ __forceinline__ Unit<T> masked(Unit<T> u, uint32_t allowed) {
  constexpr int kWords = sizeof(T) * 2;
#pragma unroll
  for (int y = 0; y < kWords; ++y) {
    uint32_t keep, inf;
    if constexpr (sizeof(T) == 4) {
      keep = static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(allowed), y, 1));
      inf = 0xFF800000u;
    } else {
      const uint32_t low = static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(allowed), 2 * y, 1));
      const uint32_t high = static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(allowed), 2 * y + 1, 1));
      keep = (low & 0xFFFFu) | (high & 0xFFFF0000u);
      inf = __builtin_bit_cast(uint16_t, static_cast<T>(-__builtin_inff())) * 0x10001u;
    }
    u[y] = (u[y] & keep) | (inf & ~keep);
  }
  return u;
}

// kSparse: there are penalties or biases.  kUnits: a lane takes 8 logits that
// many times, kThreads * 8 apart.
template <int kDtype, bool kSparse, int kUnits>
__global__ __launch_bounds__(kThreads) void logits_kernel(LogitsArgs a) {
  typedef typename Element<kDtype>::type T;
  constexpr int kChunk = kThreads * 8 * kUnits, kBitWords = kSparse ? kChunk / 32 : 1;
  __shared__ __align__(16) uint32_t s_n[kSparse ? kChunk : 4];
  __shared__ float s_bias[kSparse ? kChunk : 1];
  __shared__ uint32_t s_touched[kBitWords], s_drafted[kBitWords], s_biased[kBitWords];
  __shared__ __align__(16) int32_t s_draft[SPECDEC_MAX_K];
  __shared__ int s_again;
  const LogitsLaunch& p = a.p;
  const int tid = threadIdx.x;
  int64_t block = a.base + blockIdx.x;
  if (block < a.checks) {
    const int64_t row = block * (kThreads / 64) + wave_index();
    if (row < static_cast<int64_t>(p.B) * (p.k + 1)) check_mask(p, row);
    return;
  }
  block -= a.checks;
  const int64_t chunk = block % a.chunks, v0 = chunk * kChunk, rest = block / a.chunks;
  const int i = static_cast<int>(rest / a.shares), r0 = static_cast<int>(rest % a.shares) * a.slots;
  const int r1 = r0 + a.slots < p.k + 1 ? r0 + a.slots : p.k + 1;
  const int size = static_cast<int>(p.V - v0 < kChunk ? p.V - v0 : kChunk), whole = size & ~7;   // units of 8 end there
  const bool penal = p.repetition || p.presence || p.frequency;
  int64_t begin = 0, end = p.width, answered = 0;   // columns of the history; the first behind the prompt
  const int32_t* draft = p.draft + static_cast<int64_t>(i) * p.k;
  float rep = 1.f, pres = 0.f, freq = 0.f;
  if (kSparse && penal) {
    // read together: what is not given stands for any word that may be read
    auto word = [&](const void* of) { return load_invariant(of ? static_cast<const int32_t*>(of) + i : p.s); };
    const int32_t b = word(p.begin), l = word(p.lens), t = word(p.prompt);
    const int32_t x = word(p.repetition), y = word(p.presence), z = word(p.frequency);
    begin = p.begin ? b : 0;
    end = p.lens ? l : p.width;
    answered = begin + (p.prompt ? t : 0);
    rep = p.repetition ? __int_as_float(x) : 1.f;
    pres = p.presence ? __int_as_float(y) : 0.f;
    freq = p.frequency ? __int_as_float(z) : 0.f;
    if (begin < 0 || begin > end || end >= p.s_stride) {
      if (chunk == 0 && r0 == 0 && tid == 0 && p.dev_status) atomicOr(p.dev_status, kBadPadIn);
      return;
    }
  }
  const bool in_place = p.out == p.logits;

  // A lane's logits are read one slot ahead, and their mask two, which says
  // whether they are needed.
  const int64_t row0 = static_cast<int64_t>(i) * (p.k + 1);
  uint32_t touched[kUnits] = {};   // those of a lane's logits that a count, a draft or a bias may change
  auto at = [&](int e) { return (tid + e * kThreads) * 8; };   // the first of them, from v0 on
  auto read_mask = [&](int r, uint32_t (&to)[kUnits]) {
#pragma unroll
    for (int e = 0; e < kUnits; ++e) {
      to[e] = 0xFFu;
      if (p.mask && at(e) < whole)
        to[e] = (reinterpret_cast<const uint8_t*>(p.mask + (row0 + (r < r1 ? r : r1 - 1)) * p.mask_stride) + v0 / 8)[tid + e * kThreads];
    }
  };
  auto needed = [&](int e, uint32_t mask) { return at(e) < whole && !(in_place && mask == 0xFFu && touched[e] == 0); };
  auto read = [&](int r, const uint32_t (&mask)[kUnits], Unit<T> (&x)[kUnits]) {
#pragma unroll
    for (int e = 0; e < kUnits; ++e)
      if (mask[e] != 0 && needed(e, mask[e]))
        x[e] = load_unit(static_cast<const T*>(p.logits) + ((row0 + r) * p.V + v0) + at(e));
  };
  uint32_t mask[kUnits], mask1[kUnits];
  read_mask(r0, mask);
  read_mask(r0 + 1, mask1);
  Unit<T> x[kUnits] = {};
  // In place, the counts say whether they are needed.  Few logits: at once;
  // many: behind what the counts need, which is then not waited for longer.
  constexpr bool kAtOnce = !kSparse || kUnits == 1;
  if (kAtOnce && !in_place) read(r0, mask, x);

  if constexpr (kSparse) {
    // All that the counts need is read before the first wait, but for the
    // tokens of a history beyond kAhead * kThreads.
    constexpr int kBiases = SPECDEC_MAX_BIAS / kThreads, kAhead = 8;
    const int32_t* ids = p.bias_ids + static_cast<int64_t>(i) * p.n_bias;
    const float* bias = p.bias + static_cast<int64_t>(i) * p.n_bias;
    const int32_t* s = p.s + i * p.s_stride;
    int32_t early[kAhead], id[kBiases], drafted_token = -1;
    float bias_at[kBiases];
#pragma unroll
    for (int e = 0; e < kBiases; ++e) {
      const int j = tid + e * kThreads;
      id[e] = j < p.n_bias ? ids[j] : -1;
      bias_at[e] = j < p.n_bias ? bias[j] : 0.f;
    }
    if (penal) {
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        const int64_t j = begin + e * kThreads + tid;
        early[e] = j <= end ? s[j] : -1;
      }
      if (tid < r1 - 1) drafted_token = draft[tid];
    }
    uint32_t* s_place = reinterpret_cast<uint32_t*>(s_bias);
    auto inside = [&](int32_t token) { return token >= v0 && token < v0 + size; };
    auto mark = [](uint32_t* bits, int v) { atomicOr(&bits[v >> 5], 1u << (v & 31)); };
    for (int j = tid; j < kChunk / 4; j += kThreads) reinterpret_cast<uint4*>(s_n)[j] = uint4{0, 0, 0, 0};
    for (int j = tid; j < kChunk / 32; j += kThreads) s_touched[j] = s_drafted[j] = s_biased[j] = 0;
#pragma unroll
    for (int e = 0; e < kBiases; ++e)
      if (inside(id[e])) s_place[id[e] - v0] = ~0u;
    if (tid < SPECDEC_MAX_K) s_draft[tid] = drafted_token;
    if (tid == 0) s_again = 0;
    __syncthreads();
    if (!kAtOnce && !in_place) read(r0, mask, x);
    if (penal) {
      auto count = [&](int64_t j, int32_t token) {
        if (!inside(token)) return;
        const int v = static_cast<int>(token - v0);
        if (j < answered) atomicOr(&s_n[v], kPrompt);
        else atomicAdd(&s_n[v], 1u);
        mark(s_touched, v);
      };
#pragma unroll
      for (int e = 0; e < kAhead; ++e) count(begin + e * kThreads + tid, early[e]);
      int64_t j0 = begin + kAhead * kThreads;
      for (; j0 + kAhead * 4 * kThreads <= end + 1; j0 += kAhead * 4 * kThreads) {   // four tokens a load
        int32_t token[kAhead][4];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) __builtin_memcpy(token[e], s + j0 + (e * kThreads + tid) * 4, 16);
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
#pragma unroll
          for (int y = 0; y < 4; ++y) count(j0 + (e * kThreads + tid) * 4 + y, token[e][y]);
      }
      for (; j0 <= end; j0 += kAhead * kThreads) {
        int32_t token[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
          const int64_t j = j0 + e * kThreads + tid;
          token[e] = s[j <= end ? j : end];
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
          if (j0 + e * kThreads + tid <= end) count(j0 + e * kThreads + tid, token[e]);
      }
      if (inside(drafted_token)) {
        mark(s_touched, static_cast<int>(drafted_token - v0));
        mark(s_drafted, static_cast<int>(drafted_token - v0));
      }
    }
    // The biases: of an id given more than once, the first place adds all of
    // them up, in their order.
#pragma unroll
    for (int e = 0; e < kBiases; ++e)
      if (inside(id[e])) atomicMin(&s_place[id[e] - v0], static_cast<uint32_t>(tid + e * kThreads));
    __syncthreads();
    if (p.n_bias > 0) {
      bool mine[kBiases];
#pragma unroll
      for (int e = 0; e < kBiases; ++e) {
        mine[e] = inside(id[e]) && s_place[id[e] - v0] == static_cast<uint32_t>(tid + e * kThreads);
        if (inside(id[e]) && !mine[e]) s_again = 1;
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < kBiases; ++e) {
        if (!mine[e]) continue;
        const int v = static_cast<int>(id[e] - v0);
        float sum = bias_at[e];
        if (s_again)
          for (int y = tid + e * kThreads + 1; y < p.n_bias; ++y)
            if (ids[y] == id[e]) sum += bias[y];
        s_bias[v] = sum;
        mark(s_touched, v);
        mark(s_biased, v);
      }
      __syncthreads();
    }
  }
  // What the counts and biases do to the lane's logits: `held` bits say where the
  // repetition penalty applies, `add` is added; -0.0 where nothing is, which
  // changes no value, and no -0.0 to 0.0.  One product and one sum a logit
  // instead of a division, a difference and a sum: an fp32 result of 1000
  // logits is off by 7.0e-9 of its size instead of 6.3e-9.
  const float less = 1.f / rep;
  uint32_t held[kUnits] = {}, drafted[kUnits] = {};
  float add[kUnits][8] = {};
  auto bias_of = [&](int v) { return s_biased[v >> 5] >> (v & 31) & 1u ? s_bias[v] : -0.f; };
  auto added = [&](uint32_t n, float bias) {
    const uint32_t told = n & ~kPrompt;
    return told ? bias - (freq * static_cast<float>(told) + pres) : bias;
  };
  // A drafted token's logit in slot r, whose count grows from slot to slot: bit
  // j of `same` says that draft j is the token, bit j of `prompted` that it lies
  // in the prompt.
  auto drafts_like = [&](int v) {
    uint64_t same = 0;
    for (int j = 0; j < r1 - 1; j += 4) {
      const int4 four = *reinterpret_cast<const int4*>(&s_draft[j]);
      const int32_t token = static_cast<int32_t>(v0 + v);
      same |= static_cast<uint64_t>((four.x == token ? 1u : 0u) | (four.y == token ? 2u : 0u) | (four.z == token ? 4u : 0u) |
                                    (four.w == token ? 8u : 0u)) << j;
    }
    return same;
  };
  auto before = [](int64_t j) { return j <= 0 ? 0 : j < 64 ? (uint64_t{1} << j) - 1 : ~uint64_t{0}; };
  const uint64_t prompted = before(answered - end - 1);
  auto changed = [&](float one, uint32_t n, uint64_t same, float bias, int r) {
    const uint64_t seen = same & before(r);
    n += __popcll(seen & ~prompted);
    if (seen & prompted) n |= kPrompt;
    if (n) one *= one > 0.f ? less : rep;
    return one + added(n, bias);
  };
  // ... the first of a lane's unit, from registers: LDS would be waited for in every slot
  uint64_t same[kUnits] = {};
  uint32_t count_of[kUnits] = {};
  float bias_first[kUnits] = {};
  if constexpr (kSparse) {
#pragma unroll
    for (int e = 0; e < kUnits; ++e) {
      touched[e] = reinterpret_cast<const uint8_t*>(s_touched)[tid + e * kThreads];
      drafted[e] = reinterpret_cast<const uint8_t*>(s_drafted)[tid + e * kThreads];
      if (!touched[e]) continue;
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const uint32_t n = s_n[at(e) + b];
        if (n) held[e] |= 1u << b;
        add[e][b] = added(n, bias_of(at(e) + b));
      }
      if (drafted[e]) {
        const int v = at(e) + __builtin_ctz(drafted[e]);
        same[e] = drafts_like(v);
        count_of[e] = s_n[v];
        bias_first[e] = bias_of(v);
      }
    }
  }
  if (in_place) read(r0, mask, x);
  for (int r = r0; r < r1; ++r) {
    uint32_t mask2[kUnits];
    read_mask(r + 2, mask2);
    Unit<T> now[kUnits];
#pragma unroll
    for (int e = 0; e < kUnits; ++e) now[e] = x[e];
    if (r + 1 < r1) read(r + 1, mask1, x);
#pragma unroll
    for (int e = 0; e < kUnits; ++e) {
      if (!needed(e, mask[e])) continue;
      Unit<T> y = now[e];
      if constexpr (kSparse) {
        if (__any((touched[e] & mask[e]) != 0)) {
          float z[8];
          widen<T>(y, z);
#pragma unroll
          for (int b = 0; b < 8; ++b) {
            if (held[e] >> b & 1u) z[b] *= z[b] > 0.f ? less : rep;
            z[b] += add[e][b];
          }
          y = replaced<T>(y, z, touched[e]);
          if (drafted[e]) {
            const int b = __builtin_ctz(drafted[e]);
            y = give<T>(y, b, changed(take<T>(now[e], b), count_of[e], same[e], bias_first[e], r));
          }
          for (uint32_t bits = drafted[e] & (drafted[e] - 1) & mask[e]; bits; bits &= bits - 1) {
            const int b = __builtin_ctz(bits), v = at(e) + b;
            y = give<T>(y, b, changed(take<T>(now[e], b), s_n[v], drafts_like(v), bias_of(v), r));
          }
        }
      }
      if (mask[e] != 0xFFu) y = masked<T>(y, mask[e]);
      store_unit(static_cast<T*>(p.out) + ((row0 + r) * p.V + v0) + at(e), y);
    }
#pragma unroll
    for (int e = 0; e < kUnits; ++e) {
      mask[e] = mask1[e];
      mask1[e] = mask2[e];
    }
  }
  // the vocabulary's last logits where it is no multiple of 8, a thread each
  const int left = size - whole;
  for (int j = tid; j < left * (r1 - r0); j += kThreads) {
    const int r = r0 + j / left, v = whole + j % left;
    const int64_t row = row0 + r;
    T one = static_cast<const T*>(p.logits)[row * p.V + v0 + v];
    if (kSparse && s_touched[v >> 5] >> (v & 31) & 1u)
      one = static_cast<T>(changed(static_cast<float>(one), s_n[v], drafts_like(v), bias_of(v), r));
    if (p.mask && !(p.mask[row * p.mask_stride + ((v0 + v) >> 5)] >> (v & 31) & 1u)) one = static_cast<T>(-__builtin_inff());
    static_cast<T*>(p.out)[row * p.V + v0 + v] = one;
  }
}

template <int kDtype>
void launch_dtype(const LogitsArgs& a, bool sparse, int units, uint32_t blocks, hipStream_t stream) {
  if (sparse && units == 1) logits_kernel<kDtype, true, 1><<<blocks, kThreads, 0, stream>>>(a);
  else if (sparse) logits_kernel<kDtype, true, 2><<<blocks, kThreads, 0, stream>>>(a);
  else if (units == 1) logits_kernel<kDtype, false, 1><<<blocks, kThreads, 0, stream>>>(a);
  else logits_kernel<kDtype, false, 2><<<blocks, kThreads, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_logits(const LogitsLaunch& p, hipStream_t stream) {
  const bool sparse = p.repetition || p.presence || p.frequency || p.n_bias > 0;
  const int64_t rows = static_cast<int64_t>(p.B) * (p.k + 1);
  if (p.out == p.logits && !sparse && !p.mask) return hipSuccess;
  LogitsArgs a{};
  a.p = p;
  a.checks = p.mask ? (rows + kThreads / 64 - 1) / (kThreads / 64) : 0;
  // Two units a lane need fewer set-ups and keep more loads in flight; one
  // fills the CUs with less (1 x 128256: 7.1 us with two, 5.3 with one; 32 x 8
  // x 128256 with everything on: 36 and 44).
  const int units = p.B * ((static_cast<int64_t>(p.V) + 16 * kThreads - 1) / (16 * kThreads)) < 512 ? 1 : 2;
  const int64_t chunk = 8 * kThreads * units;
  a.chunks = (p.V + chunk - 1) / chunk;
  // the slots go to several workgroups where there would be few otherwise
  const int64_t items = p.B * a.chunks, wanted = (1024 + items - 1) / items;
  a.shares = static_cast<int32_t>(wanted < p.k + 1 ? wanted : p.k + 1);
  a.slots = (p.k + a.shares) / a.shares;
  a.shares = (p.k + a.slots) / a.slots;
  return launch_blocks(a.checks + items * a.shares, kThreads, [&](int64_t at, uint32_t n) {
    a.base = at;
    if (p.dtype == 0) launch_dtype<0>(a, sparse, units, n, stream);
    else if (p.dtype == 1) launch_dtype<1>(a, sparse, units, n, stream);
    else launch_dtype<2>(a, sparse, units, n, stream);
  });
}

}  // namespace specdec
