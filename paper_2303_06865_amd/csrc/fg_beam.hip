// Beam search: selection over the beams of a sequence and the vocabulary, and the page tables behind the beams chosen.
#include <float.h>

#include <type_traits>

#include "fg_common.h"

namespace fg {

namespace {

// ---------------------------------------------------------------- selection
// Two launches.  The first reads every logit once: a workgroup takes one piece of one row into registers and leaves the
// piece's maximum, its sum of exponentials and its n_best words.  The second takes a sequence: what all pieces of all
// its beams left.
//
// The n best of a workgroup's values without sorting them: of the largest values of the 64 groups of four threads, the
// n-th largest is a bound that at least n values reach, and (values falling as they may) few more.  Those are collected
// in LDS and each counts how many are better: its place.  Should more than kList reach the bound (equal values; in the
// second launch also n = 32 best of some hundred pieces, whose first places all lie with the same threads), the best are
// taken one after the other instead.  Values carry their place in the key, so no two are equal.
//
// The sum of exponentials decides between words of different beams and so is kept better than one binary32 exponential
// is: exp(y) = 2^h (1 + (y - h ln 2)), y = x - max, h about y log2 e and ln 2 to twice the precision; added up in
// binary32 over a thread's 8 or 32 values and in binary64 from there on.  What is left: the roundings of these sums
// (two a word, 2^-18 in all), of y (none for words within a factor of two of the largest; the mean of |y| is below
// log(vocab), so 2^-19.7) and of the exponential instruction itself, together below 2^-17 at worst and 2^-21 in what
// was measured.
constexpr int kList = 512;

// A forbidden word is -inf (also NaN); +inf counts as the largest finite number.
__device__ __forceinline__ float clean(float x) { return x >= -FLT_MAX ? fminf(x, FLT_MAX) : -INFINITY; }

// order-preserving bits: larger number, larger key (-0 is 0)
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t u) {
  return __builtin_bit_cast(float, u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ uint64_t ordered(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);
  return u >> 63 ? ~u : u | (1ull << 63);
}

// Keys: of a piece's words (logit, lower word first); of a sequence's continuations (value, logit, lower beam, lower
// word).  All zero: none.
struct Key1 {
  uint64_t k;
  __device__ __forceinline__ bool operator<(const Key1& o) const { return k < o.k; }
  __device__ __forceinline__ bool none() const { return k == 0; }
};
struct Key2 {
  uint64_t v, k;
  __device__ __forceinline__ bool operator<(const Key2& o) const { return v < o.v || (v == o.v && k < o.k); }
  __device__ __forceinline__ bool none() const { return v == 0; }
};
template <int CTRL>
__device__ __forceinline__ uint64_t dpp64(uint64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, 0xF, 0xF, true);
  return (uint64_t)hi << 32 | lo;
}
template <int CTRL>
__device__ __forceinline__ Key1 dpp(Key1 a) { return {dpp64<CTRL>(a.k)}; }
template <int CTRL>
__device__ __forceinline__ Key2 dpp(Key2 a) { return {dpp64<CTRL>(a.v), dpp64<CTRL>(a.k)}; }
__device__ __forceinline__ uint64_t lane_xor(uint64_t v, int m) { return __shfl_xor((unsigned long long)v, m, 64); }
__device__ __forceinline__ Key1 lane_xor(Key1 a, int m) { return {lane_xor(a.k, m)}; }
__device__ __forceinline__ Key2 lane_xor(Key2 a, int m) { return {lane_xor(a.v, m), lane_xor(a.k, m)}; }
// in registers: over each 16 lanes by DPP, then over the wave
template <class Op>
__device__ __forceinline__ double row16_f64(double v, Op op) {
  auto in16 = [&](auto ctrl) {
    constexpr int c = decltype(ctrl)::value;
    v = op(v, __builtin_bit_cast(double, dpp64<c>(__builtin_bit_cast(uint64_t, v))));
  };
  in16(std::integral_constant<int, kDppXor1>{});
  in16(std::integral_constant<int, kDppXor2>{});
  in16(std::integral_constant<int, kDppHalfMirror>{});
  in16(std::integral_constant<int, kDppMirror>{});
  return v;
}
template <class Op>
__device__ __forceinline__ double wave_f64(double v, Op op) {
  v = row16_f64(v, op);
  auto pair = [&](const auto lo, const auto hi) {
    v = op(__builtin_bit_cast(double, (uint64_t)(uint32_t)hi[0] << 32 | (uint32_t)lo[0]),
           __builtin_bit_cast(double, (uint64_t)(uint32_t)hi[1] << 32 | (uint32_t)lo[1]));
  };
  uint64_t u = __builtin_bit_cast(uint64_t, v);
  pair(__builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false),
       __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false));
  u = __builtin_bit_cast(uint64_t, v);
  pair(__builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false),
       __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false));
  return v;
}
__device__ __forceinline__ double wave_sum_f64(double v) {
  return wave_f64(v, [](double a, double b) { return a + b; });
}
__device__ __forceinline__ double row16_sum_f64(double v) {
  return row16_f64(v, [](double a, double b) { return a + b; });
}
__device__ __forceinline__ double row16_max_f64(double v) {
  return row16_f64(v, [](double a, double b) { return fmax(a, b); });
}
template <class K>
__device__ __forceinline__ K larger(K a, K b) { return a < b ? b : a; }

// The n (<= 32) largest keys of a workgroup of 256 threads.  mine: the largest of the thread's, or a lower bound of it
// that one of its keys reaches.  each(bound, f) calls f for every key of the thread that reaches the bound (and may for
// others, none() included).  emit(place, key) is called once for every place below the number found, which is returned.
template <class K, class Each, class Emit>
__device__ __forceinline__ int block_best(int n, K mine, K* list /* [kList] */, K* tops /* [64] */, K* bound_at, int* count, Each each,
                                          Emit emit) {
  const int tid = threadIdx.x;
  K top = larger(mine, dpp<kDppXor1>(mine));
  top = larger(top, dpp<kDppXor2>(top));
  if ((tid & 3) == 0) tops[tid >> 2] = top;
  if (tid == 0) *count = 0, *bound_at = {};
  __syncthreads();
  {   // four threads per group, a quarter of the others each
    const int group = tid >> 2, from = (tid & 3) * 16;
    const K me = tops[group];
    int above = 0;
#pragma unroll
    for (int i = from; i < from + 16; ++i) above += me < tops[i] || (i < group && !(tops[i] < me)) ? 1 : 0;   // lower bounds may be equal
    above += __builtin_amdgcn_update_dpp(0, above, kDppXor1, 0xF, 0xF, true);
    above += __builtin_amdgcn_update_dpp(0, above, kDppXor2, 0xF, 0xF, true);
    if ((tid & 3) == 0 && above == n - 1) *bound_at = me;
  }
  __syncthreads();
  const K bound = *bound_at;
  each(bound, [&](K k) {
    if (k.none() || k < bound) return;
    const int at = atomicAdd(count, 1);
    if (at < kList) list[at] = k;
  });
  __syncthreads();
  const int found = *count;
  if (found <= kList) {
    for (int c = tid; c < found; c += 256) {
      const K k = list[c];
      int place = 0;
      for (int i = 0; i < found; ++i) place += k < list[i] ? 1 : 0;
      if (place < n) emit(place, k);
    }
    return found < n ? found : n;
  }
  K last = {};
  for (int p = 0; p < n; ++p) {   // more than n reach the bound: there is always a next one
    K best = {};
    each(K{}, [&](K k) {   // (all keys: asked again who reaches the bound, the compiler keeps the answers of the first time)
      if (!k.none() && (p == 0 || k < last) && best < k) best = k;
    });
    best = larger(best, dpp<kDppXor1>(best));
    best = larger(best, dpp<kDppXor2>(best));
    if ((tid & 3) == 0) tops[tid >> 2] = best;
    __syncthreads();
    last = tops[tid & 63];
    __syncthreads();   // read before the next round writes
    for (int m = 1; m < 64; m <<= 1) last = larger(last, lane_xor(last, m));
    if (tid == 0) emit(p, last);
  }
  return n;
}

struct SelectArgs {
  const float* logits;
  int64_t ld;
  const float* scores;
  const int32_t* done;
  int32_t eos, vocab, beams, n_best;
  int32_t pieces, piece;   // of a row, and words of one
  double* sums;            // [rows][pieces]: sum of exp(x - ref); 0: no words
  double* refs;            // [rows][pieces]
  uint64_t* best;          // [rows][pieces][n_best] keys, 0: none
  int32_t* out_beams;
  int32_t* out_ids;
  float* out_scores;
  int32_t* out_done;
};

constexpr uint32_t kMostWord = (1u << 28) - 1;

template <int VPT, bool VEC>
__global__ __launch_bounds__(256) void beam_rows_kernel(SelectArgs a) {
  __shared__ Key1 list[kList], tops[64], bound;
  __shared__ double part[4];
  __shared__ float wave_top[4];
  __shared__ int count;
  const int row = blockIdx.y, tid = threadIdx.x;
  if (a.done && a.done[row]) return;   // nobody reads what it would leave
  const int w0 = blockIdx.x * a.piece, n = min(a.piece, a.vocab - w0);   // words of this piece (a multiple of 4 if VEC)
  const float* src = a.logits + (int64_t)row * a.ld + w0;
  float x[VPT];
  auto word = [&](int j) { return VEC ? (j >> 2) * 1024 + tid * 4 + (j & 3) : j * 256 + tid; };
  if constexpr (VEC) {
#pragma unroll
    for (int j = 0; j < VPT; j += 4) {
      const int w = word(j);
      float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (w < n) v = *reinterpret_cast<const float4*>(src + w);
      x[j] = v.x, x[j + 1] = v.y, x[j + 2] = v.z, x[j + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int w = word(j);
      x[j] = w < n ? src[w] : -INFINITY;
    }
  }
  // Is there a NaN or +inf?  As whole numbers, +inf and the NaNs above it are the largest with a sign, and the NaNs
  // with the sign set are above -inf without.
  int most = 0;
  uint32_t most_u = 0;
#pragma unroll
  for (int j = 0; j < VPT; j += 2) {
    __asm__("v_max3_i32 %0, %1, %2, %0" : "+v"(most) : "v"(x[j]), "v"(x[j + 1]));
    __asm__("v_max3_u32 %0, %1, %2, %0" : "+v"(most_u) : "v"(x[j]), "v"(x[j + 1]));
  }
  if (__builtin_amdgcn_ballot_w64(most >= 0x7f800000 || most_u > 0xff800000u) != 0) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) x[j] = clean(x[j]);
  }
  float top = -INFINITY;
#pragma unroll
  for (int j = 0; j < VPT; j += 2) __asm__("v_max3_f32 %0, %1, %2, %0" : "+v"(top) : "v"(x[j]), "v"(x[j + 1]));
  const float wt = wave_max(top);
  if ((tid & 63) == 0) wave_top[tid >> 6] = wt;
  __syncthreads();
  const float m = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
  const int64_t rp = (int64_t)row * a.pieces + blockIdx.x;
  constexpr float ln2 = 0.693147182f, ln2_rest = -1.90465421e-9f;   // in two binary32 numbers
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const float y = fmaxf(x[j] - m, -150.f);   // 2^-216 is 0; a piece without words (-inf - -inf) comes here too
    const float h = y * 1.44269502f, rest = __builtin_fmaf(h, -ln2_rest, __builtin_fmaf(h, -ln2, y));
    const float e = __builtin_amdgcn_exp2f(h);
    s += e;
    s = __builtin_fmaf(e, rest, s);
  }
  const double d = wave_sum_f64((double)s);
  if ((tid & 63) == 0) part[tid >> 6] = d;
  auto key = [&](int j) -> Key1 {
    const uint64_t k = (uint64_t)ordered(x[j]) << 32 | (uint32_t)(kMostWord - (uint32_t)(w0 + word(j)));
    return {x[j] > -INFINITY ? k : 0};
  };
  const Key1 mine = {top > -INFINITY ? (uint64_t)ordered(top) << 32 : 0};
  const int found = block_best<Key1>(
      a.n_best, mine, list, tops, &bound, &count,
      [&](Key1 least, auto f) {
        const float lx = least.none() ? -INFINITY : from_ordered((uint32_t)(least.k >> 32));
#pragma unroll
        for (int j = 0; j < VPT; ++j)
          if (x[j] >= lx) {
            __asm__ volatile("");   // few words come here: their keys are not made for all the others as well
            f(key(j));
          }
      },
      [&](int place, Key1 k) { a.best[rp * a.n_best + place] = k.k; });
  if (tid >= found && tid < a.n_best) a.best[rp * a.n_best + tid] = 0;
  if (tid == 0) {   // (the waves' sums were written before the barriers above)
    a.sums[rp] = part[0] + part[1] + part[2] + part[3];
    a.refs[rp] = m;
  }
}

// One workgroup per sequence: 7.6 us for 64 sequences of 8 beams x 7 pieces x 16 words, 5.5 for one of 4 x 25 x 4, most
// of it the latency of loads, logarithms and three barriers behind each other.  HELD: the keys of its continuations fit
// into LDS (kHeld) and are made once.
constexpr int kHeld = 2048;
template <bool HELD>
__global__ __launch_bounds__(256) void beam_merge_kernel(SelectArgs a) {
  __shared__ Key2 list[kList], tops[64], bound;
  __shared__ Key2 held[HELD ? kHeld : 1];
  __shared__ double lse[FG_MAX_BEAMS], score[FG_MAX_BEAMS];
  __shared__ int state[FG_MAX_BEAMS];   // 0: out, 1: alive, 2: done
  __shared__ int count;
  const int g = blockIdx.x, tid = threadIdx.x;
  const int64_t row0 = (int64_t)g * a.beams;
  const int per_beam = a.pieces * a.n_best, total = a.beams * per_beam;
  const uint64_t* best = a.best + row0 * per_beam;
  // the words are on their way while the sums are put together
  uint64_t raw[HELD ? kHeld / 256 : 1];
  if constexpr (HELD) {
#pragma unroll
    for (int i = 0; i < kHeld / 256; ++i) raw[i] = tid + 256 * i < total ? best[tid + 256 * i] : 0;
  }
  static_assert(FG_MAX_BEAMS * 16 <= 256, "sixteen lanes per beam");
  const int j16 = tid >> 4, lane16 = tid & 15;
  if (j16 < a.beams) {
    const bool over = a.done && a.done[row0 + j16];
    const float sc = a.scores[row0 + j16];
    const int64_t rp = (row0 + j16) * a.pieces;
    double ref = -INFINITY, s = 0.0;
    for (int p0 = 0; p0 < a.pieces; p0 += 16) {   // (of a beam that is done, nobody wrote these; nobody looks at what comes of them)
      const int p = p0 + lane16;
      const double sp = p < a.pieces ? a.sums[rp + p] : 0.0, rf = p < a.pieces ? a.refs[rp + p] : 0.0;
      const double now = fmax(ref, row16_max_f64(sp > 0.0 ? rf : -INFINITY));
      if (p0 > 0 && ref > -INFINITY) s *= exp(ref - now);
      s += row16_sum_f64(sp > 0.0 ? sp * exp(rf - now) : 0.0);
      ref = now;
    }
    if (lane16 == 0) {
      lse[j16] = !over && s > 0.0 ? ref + log(s) : 0.0;
      score[j16] = sc;
      state[j16] = !(sc > -INFINITY) ? 0 : (over ? 2 : 1);
    }
  }
  __syncthreads();
  auto key = [&](int t, uint64_t b) -> Key2 {
    const int j = t / per_beam;
    if (state[j] == 2)   // finished: its first place is the one it has to offer
      return t == j * per_beam
                 ? Key2{ordered(score[j]), (uint64_t)ordered(0.f) << 32 | (uint64_t)(FG_MAX_BEAMS - 1 - j) << 28 | (kMostWord - (uint32_t)a.eos)}
                 : Key2{0, 0};
    if (state[j] == 0 || b == 0) return {0, 0};
    const double v = score[j] + ((double)from_ordered((uint32_t)(b >> 32)) - lse[j]);
    return {ordered(v), (b & 0xffffffff0fffffffull) | (uint64_t)(FG_MAX_BEAMS - 1 - j) << 28};
  };
  Key2 mine = {0, 0};
  if constexpr (HELD) {
#pragma unroll
    for (int i = 0; i < kHeld / 256; ++i)
      if (tid + 256 * i < total) {
        const Key2 k = key(tid + 256 * i, raw[i]);
        held[tid + 256 * i] = k;   // read by this thread only
        mine = larger(mine, k);
      }
  } else {
    for (int t = tid; t < total; t += 256) mine = larger(mine, key(t, best[t]));
  }
  const int64_t o0 = (int64_t)g * a.n_best;
  auto put = [&](int place, int j, int w, float v, int done) {
    a.out_beams[o0 + place] = j;
    a.out_ids[o0 + place] = w;
    a.out_scores[o0 + place] = v;
    if (a.out_done) a.out_done[o0 + place] = done;
  };
  const int found = block_best<Key2>(
      a.n_best, mine, list, tops, &bound, &count,
      [&](Key2, auto f) {
        for (int t = tid; t < total; t += 256) {
          if constexpr (HELD)
            f(held[t]);
          else
            f(key(t, best[t]));
        }
      },
      [&](int place, Key2 k) {
        const int j = FG_MAX_BEAMS - 1 - (int)(k.k >> 28 & 15), w = (int)(kMostWord - (uint32_t)(k.k & kMostWord));
        const uint64_t u = k.v >> 63 ? k.v & ~(1ull << 63) : ~k.v;
        put(place, j, w, (float)__builtin_bit_cast(double, u), state[j] == 2 || (a.eos >= 0 && w == a.eos) ? 1 : 0);
      });
  if (tid >= found && tid < a.n_best) put(tid, -1, -1, -INFINITY, 1);
}

// ---------------------------------------------------------------- reordering
struct ReorderArgs {
  const int32_t* parents;
  const int32_t* table_in;
  const int32_t* pos_in;
  int32_t* table_out;
  int32_t* pos_out;
  int32_t* missing;
  int2* copies;      // [rows] of the copy pass: {page to copy from, page to copy to}; from -1: nothing to do
  int32_t* filled;   // [rows] rows to copy
  int32_t beams, stride, per_group, n_pages;
};

// One workgroup per group.  A thread takes a column of the group's table: it reads the entries of all beams before it
// writes any, so the table may be rewritten in place.  Pages held are marked in a bitmap in LDS: the full ones first,
// so that a begun page that somebody holds as a full one is known, then the begun ones.  24 groups of 4: 5.3 us,
// latency.
__global__ __launch_bounds__(256) void beam_table_kernel(ReorderArgs a) {
  extern __shared__ uint32_t held[];   // one bit per page of the group
  __shared__ int parent[FG_MAX_BEAMS], raw[FG_MAX_BEAMS], last[FG_MAX_BEAMS];
  const int g = blockIdx.x, tid = threadIdx.x;
  const int64_t row0 = (int64_t)g * a.beams;
  const int first = g * a.per_group, words = (a.per_group + 31) / 32;
  for (int w = tid; w < words; w += 256) held[w] = 0;
  if (tid < a.beams) {
    int p = a.parents[row0 + tid];
    p = p >= 0 && p < a.beams ? p : tid;
    parent[tid] = p;
    raw[tid] = a.pos_in[row0 + p];
    last[tid] = -1;
  }
  __syncthreads();
  auto rows_of = [&](int j) -> int {
    const int64_t most = (int64_t)a.stride * FG_PAGE_ROWS;
    return raw[j] < 0 ? 0 : (raw[j] > most ? (int)most : raw[j]);
  };
  for (int c = tid; c < a.stride; c += 256) {
    int e[FG_MAX_BEAMS];
    for (int j = 0; j < a.beams; ++j) e[j] = a.table_in[(row0 + j) * a.stride + c];
    for (int j = 0; j < a.beams; ++j) {
      const int n = rows_of(j);
      int pg = -1;
      if (c < (n + 63) >> 6)
        for (int k = 0; k < a.beams; ++k) pg = k == parent[j] ? e[k] : pg;
      a.table_out[(row0 + j) * a.stride + c] = pg;
      const int loc = pg - first;
      if (c == n >> 6)
        last[j] = pg;   // the page begun, or -1
      else if (pg >= first && loc < a.per_group)
        atomicOr(&held[loc >> 5], 1u << (loc & 31));
    }
  }
  __syncthreads();
  if (tid >= 64) return;
  // lane = beam: does it take a page of its own, and the how many-th of those that do
  const int n = tid < a.beams ? rows_of(tid) : 0, slot = n >> 6;
  const bool begun = (n & 63) != 0, fits = tid < a.beams && slot < a.stride;
  const int was = tid < a.beams ? last[tid] : -1;
  const bool owned = begun && was >= first && was - first < a.per_group;
  const uint32_t bit = owned ? 1u << ((was - first) & 31) : 0u;
  bool keeps = owned && !(held[(was - first) >> 5] & bit);
  for (int k = 0; k < a.beams; ++k) keeps = keeps && !(k < tid && last[k] == was && (rows_of(k) & 63) != 0);
  wave_lds_fence();   // all lanes have seen the full pages alone
  if (owned) atomicOr(&held[(was - first) >> 5], bit);
  wave_lds_fence();
  const bool takes = fits && !keeps;
  const uint64_t takers = __builtin_amdgcn_ballot_w64(takes);
  const int rank = __builtin_popcountll(takers & ((1ull << tid) - 1)), need = __builtin_popcountll(takers);
  int page = -1, given = 0;
  for (int w = 0; w < words && given < need; ++w) {   // the lowest pages that nobody holds, a word of 32 at a time
    uint32_t free = ~held[w];
    if (32 * w + 32 > a.per_group) free &= (1u << (a.per_group & 31)) - 1;
    const int n_free = __builtin_popcount(free);
    if (takes && rank >= given && rank < given + n_free) {
      for (int skip = rank - given; skip > 0; --skip) free &= free - 1;
      page = first + 32 * w + __builtin_ctz(free);
    }
    given += n_free;
  }
  const uint64_t lost = __builtin_amdgcn_ballot_w64(tid < a.beams && (slot >= a.stride || (takes && page < 0)));
  if (tid < a.beams) {
    a.pos_out[row0 + tid] = raw[tid];
    if (takes) a.table_out[(row0 + tid) * a.stride + slot] = page;
    const bool copies = takes && begun && page >= 0 && was >= 0 && was < a.n_pages;
    a.copies[row0 + tid] = copies ? make_int2(was, page) : make_int2(-1, -1);
    a.filled[row0 + tid] = ((n & 63) + 15) & ~15;
  }
  if (tid == 0 && a.missing) a.missing[g] = __builtin_popcountll(lost);
}

constexpr int kLayersPerLaunch = 64;
struct CopyArgs {
  void* data[kLayersPerLaunch][4];   // k_codes, v_codes, k_meta, v_meta of every layer
  const int2* copies;
  const int32_t* filled;
  int32_t rows, nh, layers;
  int32_t unit[2];                   // bytes of 16 rows of one head: codes, pairs (0: none; -1: one scale per head)
};

// How many rows take a copy only the device knows.  A fixed number of workgroups collects those rows (1024 at a time)
// in LDS and shares out what there is to do: one (copy, layer, tensor, head) after the other, up to 8 KiB each.  30
// copies of 48 rows in eight layers of 32 heads of 128, 191 MB: 37 us, 5.2 TB/s (a workgroup per row, layer and tensor:
// 63).
__global__ __launch_bounds__(256) void beam_copy_kernel(CopyArgs a) {
  __shared__ int4 list[1024];
  __shared__ int waves[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int r0 = 0; r0 < a.rows; r0 += 1024) {
    int n = 0;
    for (int r1 = r0; r1 < r0 + 1024 && r1 < a.rows; r1 += 256) {
      const int row = r1 + tid;
      int2 cp = make_int2(-1, -1);
      if (row < a.rows) cp = a.copies[row];
      const uint64_t m = __builtin_amdgcn_ballot_w64(cp.x >= 0);
      if (lane == 0) waves[wave] = __builtin_popcountll(m);
      __syncthreads();
      int at = n;
      for (int w = 0; w < wave; ++w) at += waves[w];
      if (cp.x >= 0) list[at + __builtin_popcountll(m & ((1ull << lane) - 1))] = make_int4(cp.x, cp.y, a.filled[row], 0);
      n += waves[0] + waves[1] + waves[2] + waves[3];
      __syncthreads();
    }
    const int per_copy = a.layers * 2 * a.nh, items = n * per_copy;   // below 2^31: see the launch
    for (int it = blockIdx.x; it < items; it += gridDim.x) {
      const int c = it / per_copy, in = it - c * per_copy;
      const int lt = in / a.nh, head = in - lt * a.nh, layer = lt >> 1, t = lt & 1;
      const int4 cp = list[c];
      const int64_t from = (int64_t)cp.x * a.nh + head, to = (int64_t)cp.y * a.nh + head;
      const int groups = cp.z >> 4;
      auto move = [&](void* base, int unit) {   // 16-byte pieces of a head's filled rows
        u4_t* p = reinterpret_cast<u4_t*>(base);
        const int per_head = unit / 4, part = unit / 16 * groups;
        for (int i = tid; i < part; i += 1024) {
          u4_t v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (i + 256 * k < part) v[k] = p[from * per_head + i + 256 * k];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (i + 256 * k < part) p[to * per_head + i + 256 * k] = v[k];
        }
      };
      move(a.data[layer][t], a.unit[0]);
      if (a.unit[1] > 0) move(a.data[layer][2 + t], a.unit[1]);
      if (a.unit[1] < 0 && tid == 0) {
        float* f = reinterpret_cast<float*>(a.data[layer][2 + t]);
        f[to] = f[from];
      }
    }
    __syncthreads();   // the list has been read
  }
}

// Words of a row that a workgroup takes: 8192 where such pieces fill the chip, else 2048 (512 rows of 50272 words, 102
// MB: 21.0 us with 8192, 23.7 with 4096; four rows with 2048: 4.3).
struct SelectPlan {
  int vpt, pieces, piece;
};
constexpr int kFullChip = 512;
SelectPlan plan_select(int64_t rows, int vocab) {
  SelectPlan p;
  p.vpt = rows * ceil_div(vocab, 8192) >= kFullChip ? 32 : 8;
  p.pieces = (int)ceil_div(vocab, 256 * p.vpt);
  p.piece = (int)align_up((size_t)ceil_div(vocab, p.pieces), 4);   // even: every group of threads has words
  p.pieces = (int)ceil_div(vocab, p.piece);
  return p;
}

struct SelectWs {
  double* sums;
  double* refs;
  uint64_t* best;
  size_t total;
};
SelectWs carve_select_ws(int64_t rows, const SelectPlan& p, int n_best, void* base) {
  SelectWs W;
  unsigned char* b = reinterpret_cast<unsigned char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* r = b ? b + off : nullptr;
    off += align_up(bytes, 256);
    return r;
  };
  W.sums = reinterpret_cast<double*>(take((size_t)rows * p.pieces * 8));
  W.refs = reinterpret_cast<double*>(take((size_t)rows * p.pieces * 8));
  W.best = reinterpret_cast<uint64_t*>(take((size_t)rows * p.pieces * n_best * 8));
  W.total = off;
  return W;
}

bool groups_ok(int32_t n_groups, int32_t beams) {
  return n_groups >= 0 && beams > 0 && beams <= FG_MAX_BEAMS && (int64_t)n_groups * beams <= 0x7fffffff;
}

constexpr int kMostGroupPages = 1 << 20;   // 128 KiB of bits in LDS

}  // namespace

}  // namespace fg

using namespace fg;

extern "C" size_t fg_beam_select_workspace_bytes(const fg_model_cfg* cfg, int32_t n_groups, int32_t beams, int32_t n_best) {
  if (!cfg || check_cfg(cfg) || !groups_ok(n_groups, beams) || n_groups == 0 || n_best < 1 || n_best > FG_MAX_BEST) return 0;
  if (cfg->vocab > (int)kMostWord || (int64_t)n_groups * beams > 65535) return 0;
  const int64_t rows = (int64_t)n_groups * beams;
  // the most rows in small pieces can need more than more rows in large ones: enough for any smaller call as well
  const int64_t most_small = (kFullChip - 1) / ceil_div(cfg->vocab, 8192), small = rows < most_small ? rows : most_small;
  const size_t need = carve_select_ws(rows, plan_select(rows, cfg->vocab), n_best, nullptr).total;
  const size_t of_small = small > 0 ? carve_select_ws(small, plan_select(small, cfg->vocab), n_best, nullptr).total : 0;
  return need > of_small ? need : of_small;
}

extern "C" int fg_beam_select(const fg_model_cfg* cfg, int32_t n_groups, int32_t beams, int32_t n_best, const float* logits,
                              int64_t row_stride, const float* scores, const int32_t* done, int32_t eos, int32_t* out_beams,
                              int32_t* out_ids, float* out_scores, int32_t* out_done, void* ws, size_t ws_bytes, void* stream) {
  if (!cfg) return FG_ERR_NULL;
  const int rc = check_cfg(cfg);
  if (rc) return rc;
  if (!groups_ok(n_groups, beams) || n_best < 1 || n_best > FG_MAX_BEST || row_stride < cfg->vocab) return FG_ERR_SHAPE;
  if (eos >= cfg->vocab || (done && eos < 0) || cfg->vocab > (int)kMostWord) return FG_ERR_SHAPE;
  if ((int64_t)n_groups * beams > 65535) return FG_ERR_SHAPE;
  if (n_groups == 0) return FG_OK;
  if (!logits || !scores || !out_beams || !out_ids || !out_scores) return FG_ERR_NULL;
  const int64_t rows = (int64_t)n_groups * beams;
  const SelectPlan p = plan_select(rows, cfg->vocab);
  const SelectWs W = carve_select_ws(rows, p, n_best, ws);
  if (!ws || ws_bytes < W.total) return FG_ERR_WORKSPACE;
  if ((uintptr_t)ws & 15u) return FG_ERR_SHAPE;
  const SelectArgs a = {logits, row_stride, scores, done, eos, cfg->vocab, beams, n_best, p.pieces, p.piece, W.sums, W.refs, W.best,
                        out_beams, out_ids, out_scores, out_done};
  const bool vec = ((uintptr_t)logits & 15u) == 0 && row_stride % 4 == 0 && cfg->vocab % 4 == 0;
  const dim3 grid((unsigned)p.pieces, (unsigned)rows);
  hipStream_t st = as_stream(stream);
  ProfScope prof(FG_K_BEAM_SELECT, st);
  if (p.vpt == 32) {
    if (vec)
      hipLaunchKernelGGL((beam_rows_kernel<32, true>), grid, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((beam_rows_kernel<32, false>), grid, dim3(256), 0, st, a);
  } else {
    if (vec)
      hipLaunchKernelGGL((beam_rows_kernel<8, true>), grid, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((beam_rows_kernel<8, false>), grid, dim3(256), 0, st, a);
  }
  FG_LAUNCH_CHECK();
  if ((int64_t)beams * p.pieces * n_best <= kHeld)
    hipLaunchKernelGGL(beam_merge_kernel<true>, dim3((unsigned)n_groups), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(beam_merge_kernel<false>, dim3((unsigned)n_groups), dim3(256), 0, st, a);
  FG_LAUNCH_CHECK();
  return FG_OK;
}

extern "C" size_t fg_beam_reorder_workspace_bytes(int32_t n_groups, int32_t beams) {
  if (!groups_ok(n_groups, beams) || n_groups == 0) return 0;
  return align_up((size_t)n_groups * beams * (sizeof(int2) + 4), 256);
}

extern "C" int fg_beam_reorder_paged(const fg_model_cfg* cfg, int32_t l, const fg_kv_pages* pages, int32_t n_groups,
                                     int32_t beams, int32_t pages_per_group, const int32_t* parents, const int32_t* table_in,
                                     const int32_t* pos_in, int32_t table_stride, int32_t* table_out, int32_t* pos_out,
                                     int32_t* missing, void* ws, size_t ws_bytes, void* stream) {
  if (!cfg || !pages) return FG_ERR_NULL;
  int rc = check_cfg(cfg);
  if (rc) return rc;
  if (l <= 0 || !groups_ok(n_groups, beams) || n_groups > kMostBlocks || pages_per_group < 1 || table_stride < 1) return FG_ERR_SHAPE;
  if ((int64_t)table_stride * FG_PAGE_ROWS > 0x7fffffff) return FG_ERR_SHAPE;
  if (pages_per_group > kMostGroupPages) return FG_ERR_UNSUPPORTED;
  const fg_ragged seqs = {table_in ? table_in : parents, nullptr, nullptr, table_stride, 1};
  for (int j = 0; j < l; ++j) {
    if (!seqs.page_table) return FG_ERR_NULL;
    if ((rc = check_pages(cfg, &pages[j], &seqs))) return rc;
    if (pages[j].dtype != pages[0].dtype) return FG_ERR_UNSUPPORTED;
    if (pages[j].n_pages != pages[0].n_pages) return FG_ERR_SHAPE;
  }
  if ((int64_t)n_groups * pages_per_group > pages[0].n_pages) return FG_ERR_SHAPE;
  if (n_groups == 0) return FG_OK;
  if (!parents || !table_in || !pos_in || !table_out || !pos_out) return FG_ERR_NULL;
  if (!ws || ws_bytes < fg_beam_reorder_workspace_bytes(n_groups, beams)) return FG_ERR_WORKSPACE;
  if ((uintptr_t)ws & 15u) return FG_ERR_SHAPE;
  const int64_t rows = (int64_t)n_groups * beams;
  ReorderArgs a = {parents, table_in, pos_in, table_out, pos_out, missing, reinterpret_cast<int2*>(ws),
                   reinterpret_cast<int32_t*>(reinterpret_cast<int2*>(ws) + rows), beams, table_stride, pages_per_group,
                   pages[0].n_pages};
  hipStream_t st = as_stream(stream);
  ProfScope prof(FG_K_BEAM_REORDER, st);
  const size_t lds = (size_t)ceil_div(pages_per_group, 32) * 4;
  if (lds > (48u << 10))
    FG_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(beam_table_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
  hipLaunchKernelGGL(beam_table_kernel, dim3((unsigned)n_groups), dim3(256), lds, st, a);
  FG_LAUNCH_CHECK();
  CopyArgs c;
  c.copies = a.copies;
  c.filled = a.filled;
  c.nh = cfg->nh;
  c.rows = (int)rows;
  if ((int64_t)1024 * kLayersPerLaunch * 2 * cfg->nh > 0x7fffffff) return FG_ERR_UNSUPPORTED;
  const int dh = cfg->h1 / cfg->nh, dt = pages[0].dtype;
  c.unit[0] = dt == FG_F16 ? 32 * dh : (dt == FG_I8P64 ? 16 * dh : 8 * dh);
  c.unit[1] = dt == FG_F16 ? 0 : (dt == FG_I8P64 ? -1 : 16 * (dh / kGroup) * (dt == FG_Q4G64 ? 8 : 4));
  for (int j0 = 0; j0 < l; j0 += kLayersPerLaunch) {
    const int nl = l - j0 < kLayersPerLaunch ? l - j0 : kLayersPerLaunch;
    for (int j = 0; j < kLayersPerLaunch; ++j) {
      const fg_kv_pages& p = pages[j0 + (j < nl ? j : 0)];
      c.data[j][0] = p.k_codes;
      c.data[j][1] = p.v_codes;
      c.data[j][2] = p.k_meta;
      c.data[j][3] = p.v_meta;
    }
    c.layers = nl;
    const int64_t most = rows * nl * 2 * cfg->nh;
    hipLaunchKernelGGL(beam_copy_kernel, dim3((unsigned)(most < 2048 ? most : 2048)), dim3(256), 0, st, c);
    FG_LAUNCH_CHECK();
  }
  return FG_OK;
}
