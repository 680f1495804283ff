// 8-bit cache pages (FG_I8P64): storing rows, and reading rows of any page format back.
//
// A page holds 64 positions; per page, head and tensor one binary32 scale S, codes c with value S c.  The scale follows
// the largest magnitude stored so far, so a row that exceeds it makes the page's other codes be rounded again to the
// wider step: rint(c * (S / S')).  That happens about ln(64) times in a page's life when rows come one at a time, and
// not at all when a page is filled by one call.  Every step of the arithmetic is one rounded binary32 operation (this
// file is compiled without contraction and with IEEE division), so codes and scales are a function of the call sequence
// alone.
#include <type_traits>

#include "fg_common.h"

namespace fg {

namespace {

typedef int8_t i8x8_t __attribute__((ext_vector_type(8)));

struct PageRows {   // whose rows, and where they live: fg_ragged and the pool
  const int32_t* page_table;
  const int32_t* seq_ids;
  const int32_t* pos;
  int32_t table_stride, n_seqs, n_pages;
};

// page of (sequence id, slot), or -1 if there is none
__device__ __forceinline__ int page_at(const PageRows& p, int sid, int64_t slot) {
  if (sid < 0 || sid >= p.n_seqs || slot < 0 || slot >= p.table_stride) return -1;
  const int page = p.page_table[(int64_t)sid * p.table_stride + slot];
  return page < p.n_pages ? page : -1;   // negative entries are none either
}

struct AppendI8Args {
  const half_t* src[2];
  int8_t* codes[2];
  float* scales[2];
  int64_t ld;
  int32_t b, s, nh, slots;   // slots: pages that the s rows of a sequence can touch
  PageRows at;
};

// Codes of a page's new rows, and what becomes of the old ones.
struct Step {
  float old, now, ratio, inv;
  bool grown;
};
__device__ __forceinline__ Step step_of(float top, float old, bool begun) {
  Step s;
  s.old = begun ? old : 0.f;
  s.now = fmaxf(s.old, top / 127.0f);
  s.grown = begun && s.now > s.old;
  s.ratio = s.grown ? s.old / s.now : 1.f;
  s.inv = s.now > 0.f ? 1.0f / s.now : 0.f;
  return s;
}
// rint in one addition: 1.5 * 2^23 + y has the whole number in its low bits, two's complement (the code is the lowest
// byte)
__device__ __forceinline__ uint32_t whole(float y) { return __builtin_bit_cast(uint32_t, y + 12582912.0f); }
// (the FMA with nothing is the product, rounded once, taken from FP16 as it is)
__device__ __forceinline__ uint32_t code_of(half_t v, const Step& s) { return whole(__builtin_fmaf((float)v, s.inv, 0.f)); }
__device__ __forceinline__ uint32_t again(int8_t c, const Step& s) { return whole((float)c * s.ratio); }
__device__ __forceinline__ uint32_t bytes4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {   // their lowest bytes
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// magnitudes of FP16 numbers are ordered as their bits without the sign
typedef uint16_t us8_t __attribute__((ext_vector_type(8)));
__device__ __forceinline__ us8_t abs_max(const h8_t v, us8_t top) {
  return __builtin_elementwise_max(__builtin_bit_cast(us8_t, v) & (us8_t)(uint16_t)0x7fff, top);
}
__device__ __forceinline__ float largest(us8_t t) {
  const uint16_t a = __builtin_elementwise_max(__builtin_elementwise_max(t[0], t[1]), __builtin_elementwise_max(t[2], t[3]));
  const uint16_t b = __builtin_elementwise_max(__builtin_elementwise_max(t[4], t[5]), __builtin_elementwise_max(t[6], t[7]));
  // (a NaN, above infinity by its bits, counts as one: a maximum of numbers would lose it, and with it what it hides)
  const uint16_t most = __builtin_elementwise_max(a, b), inf = 0x7c00;
  return (float)__builtin_bit_cast(half_t, (uint16_t)__builtin_elementwise_min(most, inf));
}

__device__ __forceinline__ u2_t row_codes(const h8_t x, const Step& s) {
  return (u2_t){bytes4(code_of(x[0], s), code_of(x[1], s), code_of(x[2], s), code_of(x[3], s)),
                bytes4(code_of(x[4], s), code_of(x[5], s), code_of(x[6], s), code_of(x[7], s))};
}
__device__ __forceinline__ u2_t codes_again(u2_t c, const Step& s) {
#pragma unroll
  for (int w = 0; w < 2; ++w)
    c[w] = bytes4(again((int8_t)c[w], s), again((int8_t)(c[w] >> 8), s), again((int8_t)(c[w] >> 16), s), again((int8_t)(c[w] >> 24), s));
  return c;
}

// The units of 16 positions of a page's value codes in LDS, [group of 16][dh] in an order in which the lanes that hold
// eight neighbouring dimensions each, as well as lanes that take units in order, meet few others on a bank.
template <int DH>
__device__ __forceinline__ int unit_at(int group, int d) {
  return (group * DH + (d & ~7) + (((d & 7) + (d >> 3)) & 7)) * 16;
}

// One workgroup per (sequence of the call, page it touches, head, K or V), a wave per group of 16 positions; lane = 8
// head dimensions (lane % LR) of RPL positions.  The new rows stay in registers until the page's largest magnitude is
// known.  Value codes pass through LDS and leave in their units, in order.  Storing 16 x 500 rows of 32 heads: with
// units straight from the lanes, 16 bytes in every 128, 70 us; in order, a wave per page 54; this 52, 3.8 TB/s of rows
// read and codes written.
template <int DH, bool VALUES>
__device__ __forceinline__ void store_rows(const half_t* src, int64_t ld, int8_t* codes, float* scale, int lo, int hi, int lane,
                                           int q, uint8_t* sm, float* sm_top) {
  constexpr int LR = DH / 8, RPL = LR / 4, UPL = DH / 64;   // positions, units per lane
  const int d0 = (lane % LR) * 8, r0 = 16 * q + (lane / LR) * RPL;
  const bool touched = 16 * q < hi && 16 * q + 16 > lo;
  const float was = lo > 0 ? *scale : 0.f;
  h8_t x[RPL];
  us8_t top = (us8_t)(uint16_t)0;
  if (touched) {
#pragma unroll
    for (int n = 0; n < RPL; ++n) {
      int row = r0 + n;
      row = row < lo ? lo : (row < hi ? row : hi - 1);   // a new row again in the place of one that is not: the largest stays
      x[n] = *reinterpret_cast<const h8_t*>(src + (int64_t)(row - lo) * ld + d0);
    }
#pragma unroll
    for (int n = 0; n < RPL; ++n) top = abs_max(x[n], top);
  }
  const float wt = wave_max(largest(top));
  if (lane == 0) sm_top[q] = wt;
  __syncthreads();
  const Step st = step_of(fmaxf(fmaxf(sm_top[0], sm_top[1]), fmaxf(sm_top[2], sm_top[3])), was, lo > 0);   // the same in all lanes
  if (q == 0 && lane == 0) *scale = st.now;
  if (!touched) {   // x holds nothing: only old codes, if any
    if (st.grown)
#pragma unroll
      for (int t = 0; t < UPL; ++t) {   // (16 rows of keys are as many bytes)
        u4_t* dst = reinterpret_cast<u4_t*>(codes + (q * DH + 64 * t + lane) * 16);
        u4_t c = *dst;
        const u2_t a = codes_again((u2_t){c.x, c.y}, st), b = codes_again((u2_t){c.z, c.w}, st);
        *dst = (u4_t){a.x, a.y, b.x, b.y};
      }
    return;
  }
  if constexpr (!VALUES) {
#pragma unroll
    for (int n = 0; n < RPL; ++n) {
      const int row = r0 + n;
      u2_t* dst = reinterpret_cast<u2_t*>(codes + row * DH + d0);
      if (row >= lo && row < hi)
        *dst = row_codes(x[n], st);
      else if (st.grown)
        *dst = codes_again(*dst, st);
    }
  } else {
    wave_lds_fence();   // what was read from there before has been
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint8_t* to = sm + unit_at<DH>(0, d0 + e) + (lane / LR) * RPL;
      const uint32_t c0 = code_of(x[0][e], st), c1 = code_of(x[1][e], st);
      if constexpr (RPL == 4)
        *reinterpret_cast<uint32_t*>(to) = bytes4(c0, c1, code_of(x[2][e], st), code_of(x[3][e], st));
      else
        *reinterpret_cast<uint16_t*>(to) = (uint16_t)__builtin_amdgcn_perm(c1, c0, 0x0c0c0400u);
    }
    wave_lds_fence();
    const bool whole = 16 * q >= lo && 16 * q + 16 <= hi;
#pragma unroll
    for (int t = 0; t < UPL; ++t) {
      u4_t* dst = reinterpret_cast<u4_t*>(codes + (q * DH + 64 * t + lane) * 16);
      u4_t c = *reinterpret_cast<const u4_t*>(sm + unit_at<DH>(0, 64 * t + lane));
      if (!whole) {   // the unit's other positions stay, in the page's new step
        const u4_t old = *dst;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t m = 0;
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const int row = 16 * q + 4 * w + n;
            const int8_t o = (int8_t)(old[w] >> (8 * n));
            const uint32_t v = row >= lo && row < hi ? c[w] >> (8 * n) : (st.grown ? again(o, st) : (uint32_t)o);
            m |= (v & 255u) << (8 * n);
          }
          c[w] = m;
        }
      }
      *dst = c;
    }
  }
}

template <int DH>
__global__ __launch_bounds__(256) void kv_append_i8_kernel(AppendI8Args a) {
  __shared__ __attribute__((aligned(16))) uint8_t sm[4][16 * DH];
  __shared__ float sm_top[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int both = blockIdx.x / a.nh, head = blockIdx.x - both * a.nh;
  const int unit = both >> 1, which = both & 1;   // K and V next to each other, as they lie in the projection's rows
  const int i = unit / a.slots, k = unit - i * a.slots;
  const int sid = a.at.seq_ids ? a.at.seq_ids[i] : i;
  const int64_t p_i = a.at.pos ? a.at.pos[i] : 0;
  if (p_i < 0) return;
  const int64_t slot = (p_i >> 6) + k, s0 = slot << 6;
  if (s0 >= p_i + a.s) return;
  const int page = page_at(a.at, sid, slot);
  if (page < 0) return;
  const int64_t ph = (int64_t)page * a.nh + head;
  int8_t* codes = a.codes[which] + ph * (FG_PAGE_ROWS * DH);
  float* scale = a.scales[which] + ph;
  // A sequence that is named more than once: the first of its rows that touches the page stores them all, in order.
  // (Everything that decides is the same in all four waves.)
  const int from = a.at.seq_ids ? 0 : i, to = a.at.seq_ids ? a.b : i + 1;
  for (int base = from; base < to; base += 64) {
    const int jl = base + lane;
    int64_t pl = -1;
    if (jl < to && (!a.at.seq_ids || a.at.seq_ids[jl] == sid)) pl = a.at.pos ? a.at.pos[jl] : 0;
    uint64_t m = __builtin_amdgcn_ballot_w64(pl >= 0 && pl < s0 + 64 && pl + a.s > s0);
    while (m) {
      const int l = __builtin_ctzll(m), j = base + l;
      m &= m - 1;
      if (j < i) return;
      const int64_t p = __builtin_amdgcn_readlane((int)pl, l);
      const int64_t first = p > s0 ? p : s0;   // first position of row block j inside this page
      const int lo = (int)(first - s0), hi = (int)(p + a.s < s0 + 64 ? p + a.s - s0 : 64);
      const half_t* src = a.src[which] + ((int64_t)j * a.s + (first - p)) * a.ld + (int64_t)head * DH;
      if (which == 0)
        store_rows<DH, false>(src, a.ld, codes, scale, lo, hi, lane, wave, sm[wave], sm_top);
      else
        store_rows<DH, true>(src, a.ld, codes, scale, lo, hi, lane, wave, sm[wave], sm_top);
      __syncthreads();   // the next one's waves read what these wrote
    }
  }
}

// One new row per sequence (the decode step): DH / 8 lanes a head, eight or four heads a wave, K or V.  What is written
// are eight bytes a lane, for V in eight units; only a page whose scale grows is read.  64 sequences x 32 heads of 128:
// 6 us, the latency of position, page and row behind each other (a wave per head and page: 17).
template <int DH>
__global__ __launch_bounds__(256) void kv_append_i8_row_kernel(AppendI8Args a) {
  constexpr int LR = DH / 8, HPW = 64 / LR;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = (blockIdx.y * 4 + wave) * HPW + lane / LR, d0 = (lane % LR) * 8;
  const int which = blockIdx.z, i = blockIdx.x;
  const int sid = a.at.seq_ids ? a.at.seq_ids[i] : i;
  const int p_i = a.at.pos ? a.at.pos[i] : 0;
  if (p_i < 0 || (blockIdx.y * 4 + wave) * HPW >= a.nh) return;
  const int page = page_at(a.at, sid, p_i >> 6);
  if (page < 0) return;
  const int64_t ph = (int64_t)page * a.nh + head;
  int8_t* codes = a.codes[which] + ph * (FG_PAGE_ROWS * DH);
  float* scale = a.scales[which] + ph;
  auto store = [&](int j, int r) {
    if (head >= a.nh) return;
    const h8_t x = *reinterpret_cast<const h8_t*>(a.src[which] + (int64_t)j * a.ld + (int64_t)head * DH + d0);
    const float was = r > 0 ? *scale : 0.f;
    float top = largest(abs_max(x, (us8_t)(uint16_t)0));   // and over the head's lanes
    top = fmaxf(top, dpp_f32<kDppXor1>(top));
    top = fmaxf(top, dpp_f32<kDppXor2>(top));
    top = fmaxf(top, dpp_f32<kDppHalfMirror>(top));
    if (LR == 16) top = fmaxf(top, dpp_f32<kDppMirror>(top));
    const Step st = step_of(top, was, r > 0);
    const u2_t c = row_codes(x, st);
    if (st.grown)   // K: 64 rows; V: the units of eight dimensions in four groups, in halves
      for (int n = 0; n < FG_PAGE_ROWS; ++n) {
        u2_t* dst = reinterpret_cast<u2_t*>(codes + (which == 0 ? n * DH + d0 : ((n >> 4) * DH + d0 + (n >> 1 & 7)) * 16 + (n & 1) * 8));
        *dst = codes_again(*dst, st);
      }
    if (which == 0) {
      *reinterpret_cast<u2_t*>(codes + r * DH + d0) = c;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) codes[((r >> 4) * DH + d0 + e) * 16 + (r & 15)] = (int8_t)(c[e >> 2] >> (8 * (e & 3)));
    }
    if (d0 == 0) *scale = st.now;
  };
  if (!a.at.seq_ids) {
    store(i, p_i & 63);
    return;
  }
  for (int base = 0; base < a.b; base += 64) {   // as above
    const int j = base + lane;
    int p = -1;
    if (j < a.b && a.at.seq_ids[j] == sid) p = a.at.pos ? a.at.pos[j] : 0;
    uint64_t m = __builtin_amdgcn_ballot_w64(p >= 0 && p >> 6 == p_i >> 6);
    while (m) {
      const int l = __builtin_ctzll(m);
      m &= m - 1;
      if (base + l < i) return;
      store(base + l, __builtin_amdgcn_readlane(p, l) & 63);
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    }
  }
}

// Rounded to binary32 first, as fg_dequantize_groupwise returns it: without the empty statement the compiler may turn an
// FMA and the conversion behind it into one instruction that rounds once.
__device__ __forceinline__ half_t to_half(float y) {
  __asm__("" : "+v"(y));
  return (half_t)y;
}

struct GatherArgs {
  const void* codes[2];
  const void* meta[2];
  half_t* out[2];
  int64_t ld;
  int32_t b, s, nh, slots;
  PageRows at;
};

// One workgroup per (sequence of the call, page, head, K or V), a wave per group of 16 positions; lane = 8 head
// dimensions (lane % LR) of RPL positions.  Waves whose group nobody asked for have nothing to do.  The 8-bit value
// codes come in their units, in order, and pass through LDS.  8 x 1500 rows of 32 heads of 128, 295 MB: 59 us, 5.0 TB/s
// (a wave per page, all 64 positions' loads first, 133 registers: 62); 16 x 400 rows of 56 heads from 4.5-bit pages,
// 235 MB: 51 us (58).
template <int DH, int FMT>
__global__ __launch_bounds__(256) void kv_gather_kernel(GatherArgs a) {
  constexpr int LR = DH / 8, RPL = LR / 4, UPL = DH / 64;   // positions, units per lane
  constexpr bool I8 = FMT == FG_I8P64, H16 = FMT == FG_Q4G64_H16;
  __shared__ __attribute__((aligned(16))) uint8_t sm[I8 ? 4 : 1][I8 ? 16 * DH : 16];
  const int lane = threadIdx.x & 63, q = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int unit = blockIdx.x / a.nh, head = blockIdx.x - unit * a.nh;
  const int which = blockIdx.y;
  const int i = unit / a.slots, k = unit - i * a.slots;
  const int64_t p_i = a.at.pos ? a.at.pos[i] : 0;
  const int64_t slot = (p_i >> 6) + k, s0 = slot << 6;
  const int lo = p_i > s0 ? (int)(p_i - s0) : 0, hi = p_i + a.s < s0 + 64 ? (int)(p_i + a.s - s0) : 64;
  if (16 * q >= hi || 16 * q + 16 <= lo) return;   // (behind the last row: hi <= 0)
  const int page = page_at(a.at, a.at.seq_ids ? a.at.seq_ids[i] : i, slot);
  const int d0 = (lane % LR) * 8, r_in = (lane / LR) * RPL, r0 = 16 * q + r_in;
  half_t* out = a.out[which] + ((int64_t)i * a.s + (s0 - p_i)) * a.ld + (int64_t)head * DH + d0;   // of the page's row 0
  auto put = [&](int n, const h8_t v) {
    if (r0 + n >= lo && r0 + n < hi) *reinterpret_cast<h8_t*>(out + (int64_t)(r0 + n) * a.ld) = v;
  };
  if (page < 0) {
#pragma unroll
    for (int n = 0; n < RPL; ++n) put(n, (h8_t)(half_t)0);
    return;
  }
  const int64_t ph = (int64_t)page * a.nh + head;
  if (I8 && which) {
    const uint8_t* codes = reinterpret_cast<const uint8_t*>(a.codes[1]) + ph * (FG_PAGE_ROWS * DH) + q * (16 * DH);
    const float sc = reinterpret_cast<const float*>(a.meta[1])[ph];
    u4_t u[UPL];
#pragma unroll
    for (int t = 0; t < UPL; ++t) u[t] = *reinterpret_cast<const u4_t*>(codes + (64 * t + lane) * 16);
#pragma unroll
    for (int t = 0; t < UPL; ++t) *reinterpret_cast<u4_t*>(sm[q] + unit_at<DH>(0, 64 * t + lane)) = u[t];
    wave_lds_fence();
    uint32_t c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint8_t* from = sm[q] + unit_at<DH>(0, d0 + e) + r_in;
      c[e] = RPL == 4 ? *reinterpret_cast<const uint32_t*>(from) : *reinterpret_cast<const uint16_t*>(from);
    }
#pragma unroll
    for (int n = 0; n < RPL; ++n) {
      h8_t v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = to_half((float)(int8_t)(c[e] >> (8 * n)) * sc);
      put(n, v);
    }
    return;
  }
  // rows in the order of their positions: raw[] = the lane's 8 elements as stored
  using raw_t = std::conditional_t<FMT == FG_F16, h8_t, std::conditional_t<I8, i8x8_t, uint32_t>>;
  using meta_t = std::conditional_t<H16, h2_t, float2>;
  const raw_t* rows = reinterpret_cast<const raw_t*>(a.codes[which]) + (ph * FG_PAGE_ROWS + r0) * LR + lane % LR;
  const float sc = I8 ? reinterpret_cast<const float*>(a.meta[which])[ph] : 0.f;
  raw_t raw[RPL];
  meta_t pair[FMT == FG_F16 || I8 ? 1 : RPL];
#pragma unroll
  for (int n = 0; n < RPL; ++n) {
    raw[n] = rows[n * LR];
    if constexpr (FMT == FG_Q4G64 || H16)
      pair[n] = reinterpret_cast<const meta_t*>(a.meta[which])[(ph * FG_PAGE_ROWS + r0 + n) * (DH / kGroup) + d0 / kGroup];
  }
#pragma unroll
  for (int n = 0; n < RPL; ++n) {
    h8_t v;
    if constexpr (FMT == FG_F16) {
      v = raw[n];
    } else if constexpr (I8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = to_half((float)raw[n][e] * sc);
    } else {
      const float mn = (float)pair[n].x, step = (float)pair[n].y;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = to_half(__builtin_fmaf((float)((raw[n] >> (4 * e)) & 15u), step, mn));
    }
    put(n, v);
  }
}

}  // namespace

static PageRows page_rows(const fg_kv_pages& pages, const fg_ragged& seqs, bool use_pos) {
  return {seqs.page_table, seqs.seq_ids, use_pos ? seqs.pos : nullptr, seqs.table_stride, seqs.n_seqs, pages.n_pages};
}

int kv_append_i8_launch(const fg_model_cfg& cfg, const half_t* k, const half_t* v, int64_t row_stride, int32_t b, int32_t s,
                        const fg_kv_pages& pages, const fg_ragged& seqs, bool use_pos, hipStream_t stream) {
  if (b == 0 || s == 0) return FG_OK;
  AppendI8Args a;
  a.src[0] = k;
  a.src[1] = v;
  a.codes[0] = reinterpret_cast<int8_t*>(pages.k_codes);
  a.codes[1] = reinterpret_cast<int8_t*>(pages.v_codes);
  a.scales[0] = reinterpret_cast<float*>(pages.k_meta);
  a.scales[1] = reinterpret_cast<float*>(pages.v_meta);
  a.ld = row_stride;
  a.b = b;
  a.s = s;
  a.nh = cfg.nh;
  a.slots = use_pos && seqs.pos ? (int)ceil_div((int64_t)s + 63, 64) : (int)ceil_div(s, 64);
  a.at = page_rows(pages, seqs, use_pos);
  const int dh = cfg.h1 / cfg.nh;
  ProfScope prof(FG_K_KV_APPEND, stream);
  if (s == 1) {
    const int hpw = 512 / dh;   // heads a wave
    if (b > kMostBlocks || ceil_div(cfg.nh, 4 * hpw) > 65535) return FG_ERR_SHAPE;
    const dim3 grid((unsigned)b, (unsigned)ceil_div(cfg.nh, 4 * hpw), 2);
    if (dh == 128)
      hipLaunchKernelGGL(kv_append_i8_row_kernel<128>, grid, dim3(256), 0, stream, a);
    else
      hipLaunchKernelGGL(kv_append_i8_row_kernel<64>, grid, dim3(256), 0, stream, a);
    FG_LAUNCH_CHECK();
    return FG_OK;
  }
  const int64_t blocks = (int64_t)b * a.slots * cfg.nh * 2;
  if ((int64_t)b * a.slots > kMostBlocks || blocks > kMostBlocks) return FG_ERR_SHAPE;
  const dim3 grid((unsigned)blocks);
  if (dh == 128)
    hipLaunchKernelGGL(kv_append_i8_kernel<128>, grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(kv_append_i8_kernel<64>, grid, dim3(256), 0, stream, a);
  FG_LAUNCH_CHECK();
  return FG_OK;
}

}  // namespace fg

using namespace fg;

extern "C" int fg_kv_gather_paged(const fg_model_cfg* cfg, const fg_kv_pages* pages, const fg_ragged* seqs, int32_t b,
                                  int32_t s, void* k_out_f16, void* v_out_f16, int64_t row_stride, void* stream) {
  if (!cfg) return FG_ERR_NULL;
  int rc = check_cfg(cfg);
  if (rc) return rc;
  rc = check_pages(cfg, pages, seqs);
  if (rc) return rc;
  if (b < 0 || s < 0 || row_stride < cfg->h1 || row_stride % 8 != 0) return FG_ERR_SHAPE;
  if (b == 0 || s == 0) return FG_OK;
  if (!k_out_f16 || !v_out_f16) return FG_ERR_NULL;
  if (((uintptr_t)k_out_f16 | (uintptr_t)v_out_f16) & 15u) return FG_ERR_SHAPE;
  GatherArgs a;
  a.codes[0] = pages->k_codes;
  a.codes[1] = pages->v_codes;
  a.meta[0] = pages->k_meta;
  a.meta[1] = pages->v_meta;
  a.out[0] = reinterpret_cast<half_t*>(k_out_f16);
  a.out[1] = reinterpret_cast<half_t*>(v_out_f16);
  a.ld = row_stride;
  a.b = b;
  a.s = s;
  a.nh = cfg->nh;
  a.at = page_rows(*pages, *seqs, true);
  a.slots = seqs->pos ? (int)ceil_div((int64_t)s + 63, 64) : (int)ceil_div(s, 64);
  const int64_t blocks = (int64_t)b * a.slots * cfg->nh;
  if ((int64_t)b * a.slots > kMostBlocks || blocks > kMostBlocks) return FG_ERR_SHAPE;
  const dim3 grid((unsigned)blocks, 2);
  hipStream_t st = as_stream(stream);
  ProfScope prof(FG_K_KV_GATHER, st);
#define FG_GATHER(FMT_)                                                                        \
  do {                                                                                         \
    if (cfg->h1 / cfg->nh == 128)                                                              \
      hipLaunchKernelGGL((kv_gather_kernel<128, FMT_>), grid, dim3(256), 0, st, a);            \
    else                                                                                       \
      hipLaunchKernelGGL((kv_gather_kernel<64, FMT_>), grid, dim3(256), 0, st, a);             \
  } while (0)
  if (pages->dtype == FG_I8P64)
    FG_GATHER(FG_I8P64);
  else if (pages->dtype == FG_F16)
    FG_GATHER(FG_F16);
  else if (pages->dtype == FG_Q4G64_H16)
    FG_GATHER(FG_Q4G64_H16);
  else
    FG_GATHER(FG_Q4G64);
#undef FG_GATHER
  FG_LAUNCH_CHECK();
  return FG_OK;
}
