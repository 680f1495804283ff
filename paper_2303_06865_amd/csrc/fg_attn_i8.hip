// Decode attention over 8-bit pages (FG_I8P64): softmax(q K^T / sqrt(dh)) V for one token per row, several rows and
// query heads on the same keys and values at once.
//
// Both products run on the integer matrix cores, on the stored codes as they are: no code is ever unpacked.  What stands
// on the other side is a number in four digits:
//   q_d = 2^(E - 30) (sum_t 2^(8t) a_td + r_d / 1024),   -128 <= a_td <= 127,   2^E > max |q|,   |r_d| < 1024
//   p_j =     1 / Cp * sum_t 2^(7t) b_tj,    0 <= b_tj <= 127,   Cp = 2^28 - 64     (p = 2^(s - max over the page) <= 1)
// so that q.k = 2^(E - 30) S_k sum_t 2^(8t) (a_t . c) with exact 32-bit integer sums, put together in binary32.
// Queries are exact like that: up to a magnitude of 64, 2^(E - 30) is no larger than FP16's smallest step; beyond it
// the rests r, whole numbers of two more digits, are multiplied where one is not zero.  Weights are cut off at 2^-28 of
// the page's largest: 64 of them are off by 2^-22 of it together.  The four digits are four columns of
// v_mfma_i32_16x16x64_i8; its sixteen columns are four queries: the beams of a sequence that share the page, or the
// query heads of a cache head, or (one query) idle, at no cost, because the loads are what bounds this.
//
//   S^T[key][column] = K . A^T    rows = keys; row m of block i is key 16 (m / 4) + 4 i + m % 4 of the page, so that lane
//                                 group g (lane / 16) ends up with keys 16 g .. 16 g + 15, four per block
//   O^T[d][column] += V^T . B^T   the lane group's 16 weights, packed to bytes, are the operand already; the pages hold
//                                 the value codes of 16 positions next to each other, which is the other operand
//
// A unit is (group of rows, cache head, four queries); the units of a cache head are neighbours, so that their waves
// find its pages in the L1 where they share a workgroup (one or two waves a unit).  With four waves a unit is a
// workgroup, and the units of a cache head fetch its pages one by one (4 x 8 beams: 51 MB for 34).  WPU waves share a
// unit's pages round-robin, and SPLITS workgroups where the units are too few for the chip.  Each keeps a running
// (maximum, sum, output) per column; they are merged through LDS, and through memory by a second launch where there are
// splits.  A wave has the values of a page and the keys of its next one on their way while it computes.
//
// Bound by the loads where sequences are long: 64 sequences of 1 to 2047 rows, 32 heads of 128, 538 MB: 108 us, 5 TB/s;
// 16 x 4 beams of 512 shared and 30 own rows, 96 heads, 302 MB of pages: 51 us, 6.2 TB/s of what is fetched; one
// sequence of 32768 rows, 32 heads on 8, 67 MB: 15 us and 4 for the merge.  A page costs a wave some 1700 cycles (64
// conversions and additions for the scores, 16 exponentials, 64 for the digits, 64 for the output, 16 matrix
// instructions of 16), a third of what the loads take with all waves of a CU at it.
#include "fg_attn_common.h"

namespace fg {

namespace {

typedef int i4_t __attribute__((ext_vector_type(4)));
typedef uint16_t us8_t __attribute__((ext_vector_type(8)));

constexpr float kWeightTop = 268435392.0f;
constexpr int kQueryBits = 30;   // (2^31 does not fit into such digits)

struct AttnI8Args {
  const half_t* q;
  int64_t q_stride;
  const int8_t* k_codes;
  const int8_t* v_codes;
  const float* k_scales;
  const float* v_scales;
  half_t* out;                 // [b, nh * dh]
  const int32_t* page_table;   // [n_seqs][table_stride]
  const int32_t* seq_ids;      // [b] or nullptr
  const int32_t* seq_rows;     // [b]: rows attended = seq_rows[i] + rows_bias
  int nh, nkv, beams;
  int n_units, chunks;         // units = groups * nkv * chunks
  int table_stride, n_seqs, n_pages, rows_bias;
  float scale;
  int splits;
  float2* part_ml;             // [b * nh][splits]: maximum (log2 units) and sum
  float* part_o;               // [b * nh][splits][dh]
};

template <bool ONCE>
__device__ __forceinline__ i4_t fetch(const int8_t* p) {
  const i4_t* q = reinterpret_cast<const i4_t*>(p);
  return ONCE ? __builtin_nontemporal_load(q) : *q;
}
__device__ __forceinline__ int seq_of(const AttnI8Args& a, int row) {
  const int sid = a.seq_ids ? a.seq_ids[row] : row;
  return sid < 0 ? 0 : (sid >= a.n_seqs ? a.n_seqs - 1 : sid);
}
__device__ __forceinline__ int rows_in(const AttnI8Args& a, int cached) {
  const int64_t n = (int64_t)cached + a.rows_bias, most = (int64_t)a.table_stride * FG_PAGE_ROWS;
  return (int)(n < 0 ? 0 : (n > most ? most : n));
}
__device__ __forceinline__ int rows_of(const AttnI8Args& a, int row) { return rows_in(a, a.seq_rows[row]); }
// The same bits in the four lanes: each takes its own digit of what comes of it.  (A product that the compiler fused
// into the first addition would be rounded in one lane and not in the other.)
__device__ __forceinline__ float quad_sum(float v) {
  __asm__("" : "+v"(v));
  v += dpp_f32<kDppXor1>(v);
  return v + dpp_f32<kDppXor2>(v);
}

// The lane's digit of four whole numbers below 2^31 - 2^23, one a byte: with 128 (of each digit) added, digits are from
// 0. which: 0x0c0c0400 + 0x0101 * digit.
__device__ __forceinline__ int digits4(const float (&n)[4], uint32_t which) {
  uint32_t u[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = (uint32_t)(int)n[e] + 0x80808080u;
  const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], which), hi = __builtin_amdgcn_perm(u[3], u[2], which);
  return (int)(__builtin_amdgcn_perm(hi, lo, 0x05040100u) ^ 0x80808080u);
}

// ONCE: the pages are loaded as data that is not needed again (see plan_i8).
template <int DH, int WPU, bool SHARED, bool ONCE>
__global__ __launch_bounds__(256, 3) void attn_decode_i8_kernel(AttnI8Args a) {
  constexpr int KS = DH / 64;   // steps of 64 over the head size
  constexpr int ND = DH / 16;   // blocks of 16 output rows
  constexpr int UPB = 4 / WPU;  // units per workgroup
  // SHARED: the wave's pages to visit, 64 a beam at most: {page, slot in the window | beams << 8}
  __shared__ uint2 sm_list[SHARED ? 4 : 1][SHARED ? 5 * 64 : 1];
  __shared__ float sm_m[4][4], sm_l[4][4];
  __shared__ __attribute__((aligned(16))) float sm_o[4][4][DH];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = wave % WPU;
  const int unit0 = blockIdx.x * UPB;
  const bool there = unit0 + wave / WPU < a.n_units;
  const int unit = there ? unit0 + wave / WPU : unit0;   // surplus waves of the last workgroup redo its first unit
  const int chunk = unit % a.chunks, gh = unit / a.chunks;
  const int kv = gh % a.nkv, group = gh / a.nkv;
  const int col = lane & 15, g = lane >> 4, dig = col & 3;
  const int per_kv = a.nh / a.nkv, nq = per_kv * a.beams;
  const int split = blockIdx.y;

  // ---- the lane's query: its digit of every element, its number of rows
  const int qi = 4 * chunk + (col >> 2), qc = min(qi, nq - 1);
  const int beam = qc / per_kv, row = group * a.beams + beam, head = kv * per_kv + qc - beam * per_kv;
  const int n_row = rows_of(a, row);
  i4_t qop[KS];
  float qmul;
  bool fine;   // some query of the wave has rests
  i4_t* rests = reinterpret_cast<i4_t*>(&sm_o[wave][0][0]);   // as many bytes as the wave's outputs take later
  {
    const half_t* src = a.q + (int64_t)row * a.q_stride + (int64_t)head * DH + 16 * g;
    h8_t x[KS][2];
    // Magnitudes are ordered as their bits.  An infinity or a NaN in the query makes top infinite, so every score a
    // NaN, so the output too.
    us8_t bits = (us8_t)(uint16_t)0;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        x[k][h] = *reinterpret_cast<const h8_t*>(src + 64 * k + 8 * h);
        bits = __builtin_elementwise_max(__builtin_bit_cast(us8_t, x[k][h]) & (us8_t)(uint16_t)0x7fff, bits);
      }
    uint16_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = bits[e] > most ? bits[e] : most;
    float top = most >= 0x7c00 ? INFINITY : (float)__builtin_bit_cast(half_t, most);
    top = xor32_reduce(xor16_reduce(top, OpMax()), OpMax());
    // 2^E > top and all its powers: E is -23 .. 16.  (top 0 or infinite: elements are 0 or do not matter)
    const bool any = top > 0.f && top < INFINITY;
    const int e2 = any ? (int)(__builtin_bit_cast(uint32_t, top) >> 23) - 126 : 0;
    const float up = any ? __builtin_bit_cast(float, (uint32_t)(127 + kQueryBits - e2) << 23) : 0.f;
    const uint32_t which = 0x0c0c0400u + 0x0101u * dig;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float n[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) n[e] = (float)x[k][w >> 1][4 * (w & 1) + e] * up;   // exact; whole but for the rests
        qop[k][w] = digits4(n, which);
      }
    // scores come out in log2 units; the digit's weight goes in here
    qmul = top < INFINITY ? a.scale * kLog2e * __builtin_bit_cast(float, (uint32_t)(127 + e2 - kQueryBits + 8 * dig) << 23) : NAN;
    fine = __builtin_amdgcn_ballot_w64(e2 > kQueryBits - 24) != 0;   // FP16 has no step below 2^-24
    if (__builtin_expect(fine, 0)) {   // (a loop, the elements loaded again: little code, seldom run)
      uint32_t odd = 0;
#pragma unroll 1
      for (int i = 0; i < 4 * KS; ++i) {
        const h4_t z = *reinterpret_cast<const h4_t*>(src + 64 * (i >> 2) + 4 * (i & 3));
        float n[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float y = (float)z[e] * up;
          n[e] = (y - __builtin_truncf(y)) * 1024.f;   // whole
        }
        const uint32_t d = (uint32_t)digits4(n, which);
        reinterpret_cast<uint32_t*>(rests + 64 * (i >> 2) + lane)[i & 3] = d;   // (read by this lane only)
        odd |= d;
      }
      fine = __builtin_amdgcn_ballot_w64(odd != 0) != 0;
      if (fine) qmul *= 1.0f / 1024;
      wave_lds_fence();
    }
  }
  const int n_of = qi < nq ? n_row : 0x7fffffff;   // an idle column is never masked, and never written
  const int n_max = __builtin_amdgcn_readfirstlane((int)wave_max((float)((n_row + 63) >> 6)));   // pages: exact in binary32
  const int per_split = (n_max + a.splits - 1) / a.splits;
  const int s_lo = split * per_split, s_hi = min(n_max, s_lo + per_split);

  float m_run = -INFINITY, l_run = 0.f;
  f4_t o[ND];
#pragma unroll
  for (int j = 0; j < ND; ++j) o[j] = (f4_t){0.f, 0.f, 0.f, 0.f};

  i4_t kreg[4][KS], vreg[ND];
  const int64_t page_bytes = FG_PAGE_ROWS * DH;
  const int k_at = (16 * (col >> 2) + (col & 3)) * DH + 16 * g, v_at = (g * DH + col) * 16;
  auto load_k = [&](int page) {
    const int8_t* p = a.k_codes + ((int64_t)page * a.nkv + kv) * page_bytes + k_at;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < KS; ++k) kreg[i][k] = fetch<ONCE>(p + 4 * i * DH + 64 * k);
  };
  auto load_v = [&](int page) {
    const int8_t* p = a.v_codes + ((int64_t)page * a.nkv + kv) * page_bytes + v_at;
#pragma unroll
    for (int j = 0; j < ND; ++j) vreg[j] = fetch<ONCE>(p + 256 * j);
  };

  const int b_lo = 4 * chunk / per_kv, nb = min(nq - 1, 4 * chunk + 3) / per_kv - b_lo + 1;   // beams of this unit
  const int32_t* tbl0 = a.page_table + (int64_t)seq_of(a, group * a.beams + b_lo) * a.table_stride;
  auto clamp_page = [&](int pg) { return pg < 0 ? 0 : (pg >= a.n_pages ? a.n_pages - 1 : pg); };

  for (int w0 = s_lo + part; w0 < s_hi; w0 += 64 * WPU) {   // windows of 64 of this wave's slots
    const int slot_l = w0 + WPU * lane;
    const bool in = slot_l < s_hi;
    int count = 0;
    uint32_t e_page = 0, e_info = 0;   // 64 pages to visit, one per lane; SHARED: slot in the window | beams << 8
    uint2* list = sm_list[SHARED ? wave : 0];
    if constexpr (SHARED) {
      // every page once, with the beams that name it; in the order of the beams, then of the slots
      const int slot_c = in ? slot_l : w0;
      int e[4], n_k[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {   // all loads first (beams that are not there: the last one's again)
        const int r = group * a.beams + b_lo + min(k, nb - 1);
        n_k[k] = a.seq_rows[r];
        e[k] = a.page_table[(int64_t)seq_of(a, r) * a.table_stride + slot_c];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = in && k < nb && rows_in(a, n_k[k]) > (slot_l << 6) ? clamp_page(e[k]) : -1 - k;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        bool first = e[k] >= 0;
        uint32_t who = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i < k) first = first && e[i] != e[k];
          if (i >= k) who |= e[i] == e[k] ? 1u << i : 0u;
        }
        const uint64_t m = __builtin_amdgcn_ballot_w64(first);
        const int at = count + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
        if (first) list[at] = make_uint2((uint32_t)e[k], (uint32_t)lane | who << 8);
        count += __builtin_popcountll(m);
      }
      wave_lds_fence();
      const uint2 mine = list[lane];   // (what lies behind the last entry is not asked for)
      e_page = mine.x, e_info = mine.y;
    } else {
      count = __builtin_popcountll(__builtin_amdgcn_ballot_w64(in));
      e_page = (uint32_t)clamp_page(tbl0[in ? slot_l : w0]);
    }
    auto slot_at = [&](uint32_t info, int v) { return w0 + WPU * (SHARED ? (int)(info & 255) : v); };

    int page = 0, slot = 0;
    uint32_t who = 0;
    if (count > 0) {
      page = __builtin_amdgcn_readfirstlane(e_page);
      who = __builtin_amdgcn_readfirstlane(e_info);
      slot = slot_at(who, 0);
      load_k(page);
    }
    for (int v = 0; v < count; ++v) {
      const float ks = a.k_scales[(int64_t)page * a.nkv + kv], vs = a.v_scales[(int64_t)page * a.nkv + kv];
      load_v(page);
      if (SHARED && ((v + 1) & 63) == 0) {
        const uint2 next = list[v + 1 + lane];
        e_page = next.x, e_info = next.y;
      }
      const int page_n = __builtin_amdgcn_readlane(e_page, (v + 1) & 63);
      const uint32_t who_n = __builtin_amdgcn_readlane(e_info, (v + 1) & 63);
      __builtin_amdgcn_sched_barrier(0);
      i4_t acc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc[i] = (i4_t){0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KS; ++k) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kreg[i][k], qop[k], acc[i], 0, 0, 0);
      }
      if (__builtin_expect(fine, 0)) {   // in 32 bits still: 128 products of 127 * 128, 1025 times, are below 2^31
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] *= 1024;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const i4_t rest = rests[64 * k + lane];
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kreg[i][k], rest, acc[i], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (v + 1 < count) load_k(page_n);
      __builtin_amdgcn_sched_barrier(0);
      // a scale of infinity: NaN, whatever the signs and the weights (digit sums of one sign would give -inf, a weight
      // of 0)
      const float f = ks < INFINITY ? qmul * ks : NAN;
      float s[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[i][r] = quad_sum((float)acc[i][r] * f);
      const int left = slot << 6;
      const bool mine = !SHARED || (who >> (8 + beam - b_lo) & 1) || n_of == 0x7fffffff;
      if (__builtin_amdgcn_ballot_w64(!mine || left > n_of - 64) != 0) {
        const int n = mine ? n_of - left - 16 * g : 0;   // keys of the lane's sixteen that count
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[i][r] = 4 * i + r < n ? s[i][r] : -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, s[i][r]);
      top = xor32_reduce(xor16_reduce(top, OpMax()), OpMax());
      const float use = top == -INFINITY ? 0.f : top;
      const float m_new = fmaxf(m_run, top), m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = fast_exp2(m_run - m_use), beta = fast_exp2(top - m_use);
      m_run = m_new;
      float sum = 0.f;
      i4_t pop;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t d[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = fast_exp2(s[i][r] - use);
          sum += p;
          d[r] = ((uint32_t)(p * kWeightTop) >> (7 * dig)) & 127u;
        }
        pop[i] = (int)(d[0] | d[1] << 8 | d[2] << 16 | d[3] << 24);
      }
      l_run = l_run * alpha + sum * beta;
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int j = 0; j < ND; ++j) o[j] *= alpha;
      }
      // a page that is not this beam's may hold infinities; one that is keeps them, also where its weight underflows
      const float bv = top == -INFINITY ? 0.f : beta * vs;
#pragma unroll
      for (int j = 0; j < ND; ++j) {
        const i4_t z = {0, 0, 0, 0};
        const i4_t po = __builtin_amdgcn_mfma_i32_16x16x64_i8(vreg[j], pop, z, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) o[j][r] = __builtin_fmaf((float)po[r], bv, o[j][r]);
      }
      page = page_n, who = who_n, slot = slot_at(who_n, v + 1);
    }
    if constexpr (SHARED) wave_lds_fence();   // the list is read before it is written again
  }

  // ---- digits together, then waves, then (second launch) splits
  wave_lds_fence();   // the rests have been read
  const float wd = (float)(1 << (7 * dig)) / kWeightTop;
  const float l = xor32_reduce(xor16_reduce(l_run, OpAdd()), OpAdd());
#pragma unroll
  for (int j = 0; j < ND; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) o[j][r] = quad_sum(o[j][r] * wd);
  if (WPU == 1 && a.splits == 1) {
    if (qi < nq && there) {
      const float inv = l == 0.f ? 0.f : 1.0f / l;   // no rows attended: zeros
      half_t* dst = a.out + ((int64_t)row * a.nh + head) * DH + 4 * g;
#pragma unroll
      for (int j = 0; j < ND; ++j)
        if ((j & 3) == dig) {
          h4_t h;
#pragma unroll
          for (int r = 0; r < 4; ++r) h[r] = (half_t)(o[j][r] * inv);
          *reinterpret_cast<h4_t*>(dst + 16 * j) = h;
        }
    }
    return;
  }
  if (lane < 16 && dig == 0) {
    sm_m[wave][col >> 2] = m_run;
    sm_l[wave][col >> 2] = l;
  }
#pragma unroll
  for (int j = 0; j < ND; ++j)
    if ((j & 3) == dig) *reinterpret_cast<f4_t*>(&sm_o[wave][col >> 2][16 * j + 4 * g]) = o[j];
  __syncthreads();
  for (int i = wave; i < UPB * 4; i += 4) {   // a wave per query
    const int qs = i & 3, u = i >> 2, un = unit0 + u;
    const int qn = un % a.chunks * 4 + qs;
    if (un >= a.n_units || qn >= nq) continue;
    const int gn = un / a.chunks, bn = qn / per_kv;
    const int64_t rh = (int64_t)(gn / a.nkv * a.beams + bn) * a.nh + gn % a.nkv * per_kv + qn - bn * per_kv;
    float M = -INFINITY, den = 0.f, num[KS] = {};
#pragma unroll
    for (int w = 0; w < WPU; ++w) M = fmaxf(M, sm_m[u * WPU + w][qs]);
#pragma unroll
    for (int w = 0; w < WPU; ++w) {
      const float mw = sm_m[u * WPU + w][qs], fw = mw == -INFINITY ? 0.f : fast_exp2(mw - M);
      den += fw * sm_l[u * WPU + w][qs];
#pragma unroll
      for (int k = 0; k < KS; ++k) num[k] += fw * sm_o[u * WPU + w][qs][lane + 64 * k];
    }
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      if (a.splits == 1)
        a.out[rh * DH + lane + 64 * k] = (half_t)(den == 0.f ? 0.f : num[k] / den);
      else
        a.part_o[(rh * a.splits + split) * DH + lane + 64 * k] = num[k];
    }
    if (a.splits > 1 && lane == 0) a.part_ml[rh * a.splits + split] = make_float2(M, den);
  }
}

// One workgroup per (row, query head): the splits' partial results together, a quarter of them per wave.
constexpr int kMostSplits = 64;
template <int DH>
__global__ __launch_bounds__(256) void attn_merge_i8_kernel(AttnI8Args a) {
  constexpr int N = DH / 64, PER = kMostSplits / 4;
  __shared__ float sm[4][DH];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t rh = blockIdx.x, p0 = rh * a.splits;
  const float2 ml = lane < a.splits ? a.part_ml[p0 + lane] : make_float2(-INFINITY, 0.f);
  float v[PER][N];
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (4 * i + wave < a.splits)
#pragma unroll
      for (int k = 0; k < N; ++k) v[i][k] = a.part_o[(p0 + 4 * i + wave) * DH + lane + 64 * k];
  const float M = wave_max(ml.x);
  const float f = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - M);
  const float den = wave_sum(f * ml.y);
  float num[N] = {};
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (4 * i + wave < a.splits) {
      const float fi = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), 4 * i + wave));
#pragma unroll
      for (int k = 0; k < N; ++k) num[k] = __builtin_fmaf(fi, v[i][k], num[k]);
    }
#pragma unroll
  for (int k = 0; k < N; ++k) sm[wave][lane + 64 * k] = num[k];
  __syncthreads();
  const int d = threadIdx.x;
  if (d < DH) a.out[rh * DH + d] = (half_t)(den == 0.f ? 0.f : (sm[0][d] + sm[1][d] + sm[2][d] + sm[3][d]) / den);
}

constexpr int kMostSplitUnits = 64;
struct Plan {
  int chunks, wpu, splits;
  bool once;
  int64_t units;
};
size_t part_bytes(int64_t rows_heads, int splits, int dh) { return splits > 1 ? align_up((size_t)rows_heads * splits * (dh + 2) * 4, 256) : 0; }

// Waves per unit, and workgroups that share a sequence.  Only the device knows the lengths; what the table could hold
// stands for them, in all three rules: a table with room for much more than its sequences hold is planned as a full one.
// Measured, us with 1 / 2 / 4 waves a unit, pages of 64 rows at head size 128 (ordinary loads):
//   6144 units, 2 pages 39 / 43 / 54         2048 units, 2 pages 14.4 / 17.6 / 19.5, 7 pages 42.7 / 44.0 / 44.8,
//   2048 units of 1 to 32 pages (table of 32) 115 / 107 / 104
//   1536 units of four beams, 8 shared pages 60.9 / 58.3 / 59.6 (57 / 51 / 54 loaded as below)
//   768 units of four beams, head size 64, 9 pages 19.2 / 18.4 / 18.0    128 units, 32 pages 39.5 / 23.3 / 15.0
//   1024 units, four to a cache head (their waves meet in the L1 if they share a workgroup) 46.8 / 50.8 / 81.2
// (units of one cache head below 1024 have not been compared: there four waves a unit stand for what more waves give)
// and where units are few, with 1 / 2 / 4 / 8 / 16 / 32 splits of four waves:
//   128 units, 32 pages 15.0 / 17.0 / 16.7 / 19.2    32 units, 24 pages 17.1 / 16.4 / 15.4 / 14.6
//   32 units, 125 pages 39.6 / 25.4 / 17.7 / 16.8 / 16.5 / 19.0    8 units, 512 pages 144 / 77 / 43 / 26 / 17.7 / 17.4
// Pages that one wave alone reads are loaded as data that is not needed again, where the call could read more than the
// last-level cache keeps until the next step; us, with the ordinary loads first: 16 x 4 beams, 96 heads, 252 MB 57.9 /
// 51.0; 64 sequences of 542 rows, 96 heads, 870 MB 152 / 138 (6.3 TB/s).  Below that a program's next step may find the
// pages there: 4 sequences of 2000 rows, 32 heads, 66 MB, 15.0 / 20.0 (one call repeated; in a model the other layers'
// pages pass between two reads).  The price: 64 sequences that share 512 rows by fours without saying so 87 / 113; the
// call with beams is for those.  And where several tiles of queries read a cache head's pages the L1 has to keep them:
// 32 x 4 beams, 32 heads on 8 46 / 60.
Plan plan_i8(int32_t nh, int32_t nkv, int32_t beams, int32_t b, int32_t dh, int32_t table_stride) {
  Plan p;
  p.chunks = (int)ceil_div(nh / nkv * beams, 4);
  p.units = (int64_t)(b / beams) * nkv * p.chunks;
  if (p.units < 1024)
    p.wpu = 4;
  else if (p.chunks >= 4 || (p.units >= 2048 && table_stride < 16))
    p.wpu = 1;
  else
    p.wpu = 2;
  p.once = p.chunks == 1 && (double)p.units * table_stride * (2 * FG_PAGE_ROWS * dh) > 128 << 20;
  p.splits = 1;
  if (p.units <= kMostSplitUnits && table_stride >= 24) {   // two pages a wave at least
    const int64_t want = 512 / p.units, most = table_stride / 8;
    p.splits = (int)(want < most ? want : most);
    if (p.splits > kMostSplits) p.splits = kMostSplits;
  }
  return p;
}

}  // namespace

size_t decode_attention_i8_workspace(int32_t nh, int32_t nkv, int32_t beams, int32_t b, int32_t dh, int32_t table_stride) {
  return part_bytes((int64_t)b * nh, plan_i8(nh, nkv, beams, b, dh, table_stride).splits, dh) + 256;
}

int decode_attention_i8_launch(const fg_model_cfg& cfg, int32_t nkv, int32_t beams, const half_t* q, int64_t q_stride, int32_t b,
                               const fg_kv_pages& pages, const fg_ragged& seqs, int32_t rows_bias, half_t* out, void* ws,
                               size_t ws_bytes, hipStream_t stream) {
  if (b == 0) return FG_OK;
  const int dh = cfg.h1 / cfg.nh;
  Plan p = plan_i8(cfg.nh, nkv, beams, b, dh, seqs.table_stride);
  const int64_t rh = (int64_t)b * cfg.nh;
  if (rh > 0x7fffffff || ceil_div(p.units * p.wpu, 4) > kMostBlocks) return FG_ERR_SHAPE;
  if (p.splits > 1 && (!ws || ws_bytes < part_bytes(rh, p.splits, dh))) p.splits = 1;
  AttnI8Args a;
  a.q = q;
  a.q_stride = q_stride;
  a.k_codes = reinterpret_cast<const int8_t*>(pages.k_codes);
  a.v_codes = reinterpret_cast<const int8_t*>(pages.v_codes);
  a.k_scales = reinterpret_cast<const float*>(pages.k_meta);
  a.v_scales = reinterpret_cast<const float*>(pages.v_meta);
  a.out = out;
  a.page_table = seqs.page_table;
  a.seq_ids = seqs.seq_ids;
  a.seq_rows = seqs.pos;
  a.nh = cfg.nh;
  a.nkv = nkv;
  a.beams = beams;
  a.n_units = (int)p.units;
  a.chunks = p.chunks;
  a.table_stride = seqs.table_stride;
  a.n_seqs = seqs.n_seqs;
  a.n_pages = pages.n_pages;
  a.rows_bias = rows_bias;
  a.scale = 1.0f / sqrtf((float)dh);
  a.splits = p.splits;
  a.part_o = reinterpret_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(a.part_o + (p.splits > 1 ? rh * p.splits * dh : 0));
  const dim3 grid((unsigned)ceil_div(p.units * p.wpu, 4), (unsigned)p.splits);
  const bool shared = beams > 1 && cfg.nh / nkv % 4 != 0;   // else a unit has queries of one row only
  ProfScope prof(FG_K_ATTN_DECODE, stream);
#define FG_I8_LAUNCH(DH_, WPU_, SH_)                                                                        \
  do {                                                                                                      \
    if (p.once)                                                                                             \
      hipLaunchKernelGGL((attn_decode_i8_kernel<DH_, WPU_, SH_, true>), grid, dim3(256), 0, stream, a);     \
    else                                                                                                    \
      hipLaunchKernelGGL((attn_decode_i8_kernel<DH_, WPU_, SH_, false>), grid, dim3(256), 0, stream, a);    \
  } while (0)
#define FG_I8_SH(DH_, WPU_)                                                                     \
  do {                                                                                          \
    if (shared) FG_I8_LAUNCH(DH_, WPU_, true); else FG_I8_LAUNCH(DH_, WPU_, false);             \
  } while (0)
#define FG_I8(DH_)                                                                                              \
  do {                                                                                                          \
    if (p.wpu == 1) FG_I8_SH(DH_, 1); else if (p.wpu == 2) FG_I8_SH(DH_, 2); else FG_I8_SH(DH_, 4);              \
  } while (0)
  if (dh == 128) FG_I8(128); else FG_I8(64);
#undef FG_I8
#undef FG_I8_SH
#undef FG_I8_LAUNCH
  FG_LAUNCH_CHECK();
  if (p.splits > 1) {
    if (dh == 128)
      hipLaunchKernelGGL(attn_merge_i8_kernel<128>, dim3((unsigned)rh), dim3(256), 0, stream, a);
    else
      hipLaunchKernelGGL(attn_merge_i8_kernel<64>, dim3((unsigned)rh), dim3(256), 0, stream, a);
    FG_LAUNCH_CHECK();
  }
  return FG_OK;
}

}  // namespace fg

using namespace fg;

static bool beams_ok(const fg_model_cfg* cfg, int32_t nkv, int32_t beams, int32_t b) {
  return nkv > 0 && nkv <= cfg->nh && cfg->nh % nkv == 0 && beams > 0 && beams <= FG_MAX_BEAMS && b >= 0 && b % beams == 0;
}

extern "C" size_t fg_decode_attention_beams_workspace_bytes(const fg_model_cfg* cfg, int32_t nkv, int32_t beams, int32_t b,
                                                            int32_t table_stride) {
  if (!cfg || check_cfg(cfg) || !beams_ok(cfg, nkv, beams, b) || b == 0 || table_stride <= 0) return 0;
  // few rows are split over more workgroups and can need more than many: what the largest of the smaller batches needs
  size_t most = 0;
  for (int32_t n = beams; n <= b; n += beams) {
    const size_t need = decode_attention_i8_workspace(cfg->nh, nkv, beams, n, cfg->h1 / cfg->nh, table_stride);
    most = need > most ? need : most;
    if (n / beams >= kMostSplitUnits) break;   // no larger batch is split
  }
  return most;
}

extern "C" int fg_decode_attention_beams_paged(const fg_model_cfg* cfg, int32_t nkv, int32_t beams, const void* q_f16,
                                               int64_t q_row_stride, int32_t b, const fg_kv_pages* pages,
                                               const fg_ragged* seqs, int32_t rows_bias, void* out_f16, void* ws,
                                               size_t ws_bytes, void* stream) {
  if (!cfg) return FG_ERR_NULL;
  int rc = check_cfg(cfg);
  if (rc) return rc;
  rc = check_pages(cfg, pages, seqs);
  if (rc) return rc;
  if (pages->dtype != FG_I8P64) return FG_ERR_UNSUPPORTED;
  if (!seqs->pos) return FG_ERR_NULL;
  if (!beams_ok(cfg, nkv, beams, b) || rows_bias < 0) return FG_ERR_SHAPE;
  if (q_row_stride < cfg->h1 || q_row_stride % 8 != 0) return FG_ERR_SHAPE;
  if (b == 0) return FG_OK;
  if (!q_f16 || !out_f16) return FG_ERR_NULL;
  if (((uintptr_t)q_f16 | (uintptr_t)out_f16) & 15u) return FG_ERR_SHAPE;
  if (!ws || ws_bytes < decode_attention_i8_workspace(cfg->nh, nkv, beams, b, cfg->h1 / cfg->nh, seqs->table_stride)) return FG_ERR_WORKSPACE;
  if ((uintptr_t)ws & 15u) return FG_ERR_SHAPE;
  return decode_attention_i8_launch(*cfg, nkv, beams, reinterpret_cast<const half_t*>(q_f16), q_row_stride, b, *pages, *seqs,
                                    rows_bias, reinterpret_cast<half_t*>(out_f16), ws, ws_bytes, as_stream(stream));
}
