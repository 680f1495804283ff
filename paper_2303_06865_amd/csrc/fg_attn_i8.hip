// Decode attention over 8-bit pages (FG_I8P64): softmax(q K^T / sqrt(dh)) V for one token per row.
#include "fg_attn_common.h"

namespace fg {

namespace {

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
  int b, nh, nkv;
  int table_stride, n_seqs, n_pages, rows_bias;
  float scale;
};

// One wave per (row, query head).  Scores: lane = position of the page; output: lane = head dimension(s).
template <int DH>
__global__ __launch_bounds__(64) void attn_decode_i8_kernel(AttnI8Args a) {
  constexpr int ND = DH / 64;
  __shared__ float sm_q[DH], sm_p[64];
  const int lane = threadIdx.x;
  const int row = blockIdx.x / a.nh, head = blockIdx.x - row * a.nh, kv = head / (a.nh / a.nkv);
  int sid = a.seq_ids ? a.seq_ids[row] : row;
  sid = sid < 0 ? 0 : (sid >= a.n_seqs ? a.n_seqs - 1 : sid);
  const int32_t* tbl = a.page_table + (int64_t)sid * a.table_stride;
  int64_t n = (int64_t)a.seq_rows[row] + a.rows_bias;
  const int64_t most = (int64_t)a.table_stride * FG_PAGE_ROWS;
  n = n < 0 ? 0 : (n > most ? most : n);
  for (int d = lane; d < DH; d += 64) sm_q[d] = (float)a.q[(int64_t)row * a.q_stride + (int64_t)head * DH + d];
  __syncthreads();
  float m = -INFINITY, l = 0.f, o[ND] = {};
  for (int64_t r0 = 0; r0 < n; r0 += FG_PAGE_ROWS) {
    int pg = tbl[r0 >> 6];
    pg = pg < 0 ? 0 : (pg >= a.n_pages ? a.n_pages - 1 : pg);
    const int64_t ph = (int64_t)pg * a.nkv + kv;
    const int8_t* kc = a.k_codes + (ph * FG_PAGE_ROWS + lane) * DH;
    float s = 0.f;
    for (int d = 0; d < DH; ++d) s += sm_q[d] * (float)kc[d];
    s = r0 + lane < n ? s * a.k_scales[ph] * a.scale : -INFINITY;
    const float m_new = fmaxf(m, wave_max(s));
    const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * kLog2e);
    m = m_new;
    const float p = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((s - m) * kLog2e);
    l = l * alpha + p;
    __syncthreads();
    sm_p[lane] = p * a.v_scales[ph];
    __syncthreads();
    const int8_t* vc = a.v_codes + ph * (FG_PAGE_ROWS * DH);
    for (int j = 0; j < ND; ++j) {
      float acc = 0.f;
      for (int r = 0; r < FG_PAGE_ROWS; ++r) acc += sm_p[r] * (float)vc[((r >> 4) * DH + lane + 64 * j) * 16 + (r & 15)];
      o[j] = o[j] * alpha + acc;
    }
  }
  l = wave_sum(l);
  for (int j = 0; j < ND; ++j)
    a.out[((int64_t)row * a.nh + head) * DH + lane + 64 * j] = (half_t)(l > 0.f ? o[j] / l : 0.f);
}

}  // namespace

size_t decode_attention_i8_workspace(int32_t nkv, int32_t beams, int32_t b, int32_t dh, int32_t table_stride) {
  (void)nkv, (void)beams, (void)b, (void)dh, (void)table_stride;
  return 256;
}

int decode_attention_i8_launch(const fg_model_cfg& cfg, int32_t nkv, int32_t beams, const half_t* q, int64_t q_stride, int32_t b,
                               const fg_kv_pages& pages, const fg_ragged& seqs, int32_t rows_bias, half_t* out, void* ws,
                               size_t ws_bytes, hipStream_t stream) {
  (void)beams, (void)ws, (void)ws_bytes;
  if (b == 0) return FG_OK;
  AttnI8Args a;
  const int dh = cfg.h1 / cfg.nh;
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
  a.b = b;
  a.nh = cfg.nh;
  a.nkv = nkv;
  a.table_stride = seqs.table_stride;
  a.n_seqs = seqs.n_seqs;
  a.n_pages = pages.n_pages;
  a.rows_bias = rows_bias;
  a.scale = 1.0f / sqrtf((float)dh);
  const int64_t waves = (int64_t)b * cfg.nh;
  if (waves > 0x7fffffff) return FG_ERR_SHAPE;
  ProfScope prof(FG_K_ATTN_DECODE, stream);
  if (dh == 128)
    hipLaunchKernelGGL(attn_decode_i8_kernel<128>, dim3((unsigned)waves), dim3(64), 0, stream, a);
  else
    hipLaunchKernelGGL(attn_decode_i8_kernel<64>, dim3((unsigned)waves), dim3(64), 0, stream, a);
  FG_LAUNCH_CHECK();
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
  return decode_attention_i8_workspace(nkv, beams, b, cfg->h1 / cfg->nh, table_stride);
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
  if (!ws || ws_bytes < decode_attention_i8_workspace(nkv, beams, b, cfg->h1 / cfg->nh, seqs->table_stride)) return FG_ERR_WORKSPACE;
  if ((uintptr_t)ws & 15u) return FG_ERR_SHAPE;
  return decode_attention_i8_launch(*cfg, nkv, beams, reinterpret_cast<const half_t*>(q_f16), q_row_stride, b, *pages, *seqs,
                                    rows_bias, reinterpret_cast<half_t*>(out_f16), ws, ws_bytes, as_stream(stream));
}
