// 8-bit cache pages (FG_I8P64): storing rows, and reading rows of any page format back.
//
// A page holds 64 positions; per page, head and tensor one binary32 scale S, codes c with value S c.  The scale follows
// the largest magnitude stored so far, so a row that exceeds it makes the page's other codes be rounded again to the
// wider step: rint(c * (S / S')).  That happens about ln(64) times in a page's life when rows come one at a time, and not at
// all when a page is filled by one call.  Every step of the arithmetic is one rounded binary32 operation (this file is
// compiled without contraction and with IEEE division), so codes and scales are a function of the call sequence alone.
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

// One wave per (sequence of the call, page it touches, head, K or V).  Lane = 8 head dimensions (lane % LR) of NR
// consecutive positions (lane / LR): a row of a head is read by LR lanes, 16 bytes each, and at head size 128 the
// lane's 16 positions are one unit of the value codes' order.
template <int DH, bool VALUES>
__device__ __forceinline__ void store_rows(const AppendI8Args& a, const half_t* src, int64_t ld, int8_t* codes, float* scale,
                                           int lo, int hi, int lane) {
  constexpr int LR = DH / 8, NR = LR;   // 64 positions over 64 / LR groups of lanes
  const int d0 = (lane % LR) * 8, r0 = (lane / LR) * NR;
  h8_t x[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    x[n] = (h8_t)(half_t)0;
    if (r0 + n >= lo && r0 + n < hi) x[n] = *reinterpret_cast<const h8_t*>(src + (int64_t)(r0 + n - lo) * ld + d0);
  }
  float top = 0.f;
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)x[n][e]));
  top = wave_max(top) / 127.0f;
  const float old = lo > 0 ? *scale : 0.f;
  const float now = fmaxf(old, top);
  const bool grown = lo > 0 && now > old;   // the same in all lanes
  const float ratio = grown ? old / now : 1.f;
  const float inv = now > 0.f ? 1.0f / now : 0.f;
  auto code = [&](half_t v) -> int8_t { return (int8_t)(int)rintf((float)v * inv); };
  auto again = [&](int8_t c) -> int8_t { return (int8_t)(int)rintf((float)c * ratio); };
  if constexpr (!VALUES) {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = r0 + n;
      i8x8_t* dst = reinterpret_cast<i8x8_t*>(codes + r * DH + d0);
      const bool fresh = r >= lo && r < hi;
      if (fresh || grown) {
        i8x8_t c;
        if (fresh) {
#pragma unroll
          for (int e = 0; e < 8; ++e) c[e] = code(x[n][e]);
        } else {
          const i8x8_t was = *dst;
#pragma unroll
          for (int e = 0; e < 8; ++e) c[e] = again(was[e]);
        }
        *dst = c;
      }
    }
  } else {
    const bool any = r0 < hi && r0 + NR > lo, all = r0 >= lo && r0 + NR <= hi;
    if (any || grown) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        // NR positions of dimension d0 + e: a unit of 16 bytes, or half of one at head size 64
        i8x8_t* dst = reinterpret_cast<i8x8_t*>(codes + ((r0 >> 4) * DH + d0 + e) * 16 + (r0 & 15));
#pragma unroll
        for (int n8 = 0; n8 < NR / 8; ++n8) {
          i8x8_t c = (i8x8_t)(int8_t)0;
          if (!all) c = dst[n8];
#pragma unroll
          for (int n = 0; n < 8; ++n) {
            const int r = r0 + 8 * n8 + n;
            c[n] = r >= lo && r < hi ? code(x[8 * n8 + n][e]) : (grown ? again(c[n]) : c[n]);
          }
          dst[n8] = c;
        }
      }
    }
  }
  if (lane == 0) *scale = now;
}

template <int DH>
__global__ __launch_bounds__(256) void kv_append_i8_kernel(AppendI8Args a) {
  const int lane = threadIdx.x & 63;
  const int head = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (head >= a.nh) return;
  const int which = blockIdx.z;
  const int i = blockIdx.x / a.slots, k = blockIdx.x - i * a.slots;
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
  auto store = [&](int j, int64_t p) {
    const int64_t first = p > s0 ? p : s0;   // first position of row block j inside this page
    const int lo = (int)(first - s0), hi = (int)(p + a.s < s0 + 64 ? p + a.s - s0 : 64);
    const half_t* src = a.src[which] + ((int64_t)j * a.s + (first - p)) * a.ld + (int64_t)head * DH;
    if (which == 0)
      store_rows<DH, false>(a, src, a.ld, codes, scale, lo, hi, lane);
    else
      store_rows<DH, true>(a, src, a.ld, codes, scale, lo, hi, lane);
  };
  if (!a.at.seq_ids) {
    store(i, p_i);
    return;
  }
  // A sequence that is named more than once: the first of its rows that touches the page stores them all, in order.
  for (int base = 0; base < a.b; base += 64) {
    const int j = base + lane;
    int64_t p = -1;
    if (j < a.b && a.at.seq_ids[j] == sid) p = a.at.pos ? a.at.pos[j] : 0;
    uint64_t m = __builtin_amdgcn_ballot_w64(p >= 0 && p < s0 + 64 && p + a.s > s0);
    while (m) {
      const int l = __builtin_ctzll(m);
      m &= m - 1;
      if (base + l < i) return;
      store(base + l, __builtin_amdgcn_readlane((int)p, l));
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");   // the next one's lanes read what these wrote
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
  int32_t b, s, nh, dtype;
  PageRows at;
};

// One thread per 8 head dimensions of one row of one head.
template <int DH>
__global__ __launch_bounds__(256) void kv_gather_kernel(GatherArgs a) {
  constexpr int C = DH / 8;
  const int which = blockIdx.y;
  const int64_t n = (int64_t)a.b * a.s * a.nh * C;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < n; t += (int64_t)gridDim.x * 256) {
    const int d0 = (int)(t % C) * 8;
    const int64_t u = t / C;
    const int head = (int)(u % a.nh);
    const int64_t row = u / a.nh;
    const int i = (int)(row / a.s), j = (int)(row - (int64_t)i * a.s);
    const int64_t p = (int64_t)(a.at.pos ? a.at.pos[i] : 0) + j;
    const int page = p < 0 ? -1 : page_at(a.at, a.at.seq_ids ? a.at.seq_ids[i] : i, p >> 6);
    h8_t v = (h8_t)(half_t)0;
    if (page >= 0) {
      const int r = (int)(p & 63);
      const int64_t ph = (int64_t)page * a.nh + head, prow = ph * FG_PAGE_ROWS + r;
      if (a.dtype == FG_F16) {
        v = *reinterpret_cast<const h8_t*>(reinterpret_cast<const half_t*>(a.codes[which]) + prow * DH + d0);
      } else if (a.dtype == FG_I8P64) {
        const int8_t* c = reinterpret_cast<const int8_t*>(a.codes[which]) + ph * (FG_PAGE_ROWS * DH);
        const float sc = reinterpret_cast<const float*>(a.meta[which])[ph];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = to_half((float)c[which ? ((r >> 4) * DH + d0 + e) * 16 + (r & 15) : r * DH + d0 + e] * sc);
      } else {
        const uint32_t c = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(a.codes[which]) + (prow * DH + d0) / 2);
        const int64_t g = (prow * DH + d0) / kGroup;
        float mn, sc;
        if (a.dtype == FG_Q4G64_H16) {
          const h2_t m = reinterpret_cast<const h2_t*>(a.meta[which])[g];
          mn = (float)m.x, sc = (float)m.y;
        } else {
          const float2 m = reinterpret_cast<const float2*>(a.meta[which])[g];
          mn = m.x, sc = m.y;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = to_half(__builtin_fmaf((float)((c >> (4 * e)) & 15u), sc, mn));
      }
    }
    *reinterpret_cast<h8_t*>(a.out[which] + row * a.ld + head * DH + d0) = v;
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
  const int64_t units = (int64_t)b * a.slots;
  if (units > 0x7fffffff || ceil_div(cfg.nh, 4) > 65535) return FG_ERR_SHAPE;
  const dim3 grid((unsigned)units, (unsigned)ceil_div(cfg.nh, 4), 2);
  ProfScope prof(FG_K_KV_APPEND, stream);
  if (cfg.h1 / cfg.nh == 128)
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
  a.dtype = pages->dtype;
  a.at = page_rows(*pages, *seqs, true);
  const int64_t blocks = ceil_div((int64_t)b * s * cfg->h1 / 8, 256);
  const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384), 2);
  hipStream_t st = as_stream(stream);
  ProfScope prof(FG_K_KV_GATHER, st);
  if (cfg->h1 / cfg->nh == 128)
    hipLaunchKernelGGL(kv_gather_kernel<128>, grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(kv_gather_kernel<64>, grid, dim3(256), 0, st, a);
  FG_LAUNCH_CHECK();
  return FG_OK;
}
