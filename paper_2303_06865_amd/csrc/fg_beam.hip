// Beam search: selection over the beams of a sequence and the vocabulary, and the page tables behind the beams chosen.
#include <float.h>

#include "fg_common.h"

namespace fg {

namespace {

// ---------------------------------------------------------------- selection
// A forbidden word is -inf (also NaN); +inf counts as the largest finite number.
__device__ __forceinline__ float clean(float x) { return x > FLT_MAX ? FLT_MAX : (x >= -FLT_MAX ? x : -INFINITY); }

// What a row leaves behind: the logarithm of its sum of exponentials and its best words, (logit, word) in descending order.
struct Best {
  float x;
  int32_t w;
};

struct SelectArgs {
  const float* logits;
  int64_t ld;
  const float* scores;
  const int32_t* done;
  int32_t eos, vocab, beams, n_best;
  double* lse;    // [rows]
  Best* best;     // [rows][n_best], word -1: none
  int32_t* out_beams;
  int32_t* out_ids;
  float* out_scores;
  int32_t* out_done;
};

// One workgroup per row; the best words one after the other, each the largest below the one before.
__global__ __launch_bounds__(256) void beam_rows_kernel(SelectArgs a) {
  __shared__ float sx[256];
  __shared__ int sw[256];
  __shared__ double ss[256];
  const int row = blockIdx.x, tid = threadIdx.x;
  const float* x = a.logits + (int64_t)row * a.ld;
  float px = INFINITY;   // the word chosen last
  int pw = -1;
  float top = 0.f;
  for (int n = 0; n < a.n_best; ++n) {
    float bx = -INFINITY;
    int bw = -1;
    for (int w = tid; w < a.vocab; w += 256) {
      const float v = clean(x[w]);
      if (v == -INFINITY || v > px || (v == px && w <= pw)) continue;
      if (v > bx) bx = v, bw = w;
    }
    sx[tid] = bx, sw[tid] = bw;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
      if (tid < o && sw[tid + o] >= 0 && (sw[tid] < 0 || sx[tid + o] > sx[tid] || (sx[tid + o] == sx[tid] && sw[tid + o] < sw[tid])))
        sx[tid] = sx[tid + o], sw[tid] = sw[tid + o];
      __syncthreads();
    }
    px = sx[0], pw = sw[0];
    if (n == 0) top = px;
    if (tid == 0) a.best[(int64_t)row * a.n_best + n] = {px, pw};
    __syncthreads();
    if (pw < 0) {
      for (int k = n + 1 + tid; k < a.n_best; k += 256) a.best[(int64_t)row * a.n_best + k] = {-INFINITY, -1};
      break;
    }
  }
  double s = 0.0;
  if (top > -INFINITY)
    for (int w = tid; w < a.vocab; w += 256) s += exp((double)clean(x[w]) - (double)top);
  ss[tid] = s;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (tid < o) ss[tid] += ss[tid + o];
    __syncthreads();
  }
  if (tid == 0) a.lse[row] = top > -INFINITY ? (double)top + log(ss[0]) : 0.0;
}

// One thread per sequence.
__global__ __launch_bounds__(64) void beam_merge_kernel(SelectArgs a, int n_groups) {
  const int g = blockIdx.x * 64 + threadIdx.x;
  if (g >= n_groups) return;
  int at[FG_MAX_BEAMS] = {};   // the next of every beam's list
  for (int n = 0; n < a.n_best; ++n) {
    double bv = -INFINITY;
    float bx = 0.f;
    int bj = -1, bw = -1;
    for (int j = 0; j < a.beams; ++j) {
      const int64_t row = (int64_t)g * a.beams + j;
      const float sc = a.scores[row];
      if (!(sc > -INFINITY) || at[j] >= a.n_best) continue;
      double v;
      float x = 0.f;
      int w;
      if (a.done && a.done[row]) {
        if (at[j] > 0) continue;
        v = sc, w = a.eos;
      } else {
        const Best b = a.best[row * a.n_best + at[j]];
        if (b.w < 0) continue;
        v = (double)sc + ((double)b.x - a.lse[row]), x = b.x, w = b.w;
      }
      if (bj < 0 || v > bv || (v == bv && x > bx)) bv = v, bx = x, bj = j, bw = w;   // beams in order: the lowest wins ties
    }
    const int64_t o = (int64_t)g * a.n_best + n;
    if (bj >= 0) ++at[bj];
    a.out_beams[o] = bj;
    a.out_ids[o] = bw;
    a.out_scores[o] = bj < 0 ? -INFINITY : (float)bv;
    if (a.out_done)
      a.out_done[o] = bj < 0 || (a.done && a.done[(int64_t)g * a.beams + bj]) || (a.eos >= 0 && bw == a.eos) ? 1 : 0;
  }
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
// writes any, so the table may be rewritten in place.  Pages held are marked in a bitmap in LDS.
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
      if (pg >= first && loc < a.per_group) atomicOr(&held[loc >> 5], 1u << (loc & 31));
      if (c == n >> 6) last[j] = pg;   // the page begun, or -1
    }
  }
  __syncthreads();
  if (tid == 0) {
    int next = 0, miss = 0;
    for (int j = 0; j < a.beams; ++j) {
      const int n = rows_of(j), slot = n >> 6;
      a.pos_out[row0 + j] = raw[j];
      int2 cp = make_int2(-1, -1);
      const bool begun = (n & 63) != 0;
      bool takes = slot < a.stride;
      if (begun) {
        const int pg = last[j];
        bool mine = pg >= first && pg - first < a.per_group;
        for (int k = 0; k < j; ++k) mine = mine && !(last[k] == pg && (rows_of(k) & 63) != 0);
        takes = takes && !mine;
      }
      if (slot >= a.stride) ++miss;
      if (takes) {
        while (next < a.per_group && (held[next >> 5] >> (next & 31)) & 1) ++next;
        int pg = -1;
        if (next < a.per_group)
          pg = first + next++;
        else
          ++miss;
        a.table_out[(row0 + j) * a.stride + slot] = pg;
        if (begun && pg >= 0 && last[j] >= 0 && last[j] < a.n_pages) cp = make_int2(last[j], pg);
      }
      a.copies[row0 + j] = cp;
      a.filled[row0 + j] = ((n & 63) + 15) & ~15;
    }
    if (a.missing) a.missing[g] = miss;
  }
}

constexpr int kLayersPerLaunch = 64;
struct CopyArgs {
  void* data[kLayersPerLaunch][4];   // k_codes, v_codes, k_meta, v_meta of every layer
  const int2* copies;
  const int32_t* filled;
  int32_t nh;
  int32_t unit[2];                   // bytes of 16 rows of one head: codes, pairs (0: none; -1: one scale per head)
};

// One workgroup per (row, layer, array): the filled rows of all heads of one page.
__global__ __launch_bounds__(256) void beam_copy_kernel(CopyArgs a) {
  const int2 cp = a.copies[blockIdx.x];
  if (cp.x < 0) return;
  const int which = blockIdx.z, unit = a.unit[which >> 1];
  char* base = reinterpret_cast<char*>(a.data[blockIdx.y][which]);
  if (unit < 0) {
    float* f = reinterpret_cast<float*>(base);
    for (int h = threadIdx.x; h < a.nh; h += 256) f[(int64_t)cp.y * a.nh + h] = f[(int64_t)cp.x * a.nh + h];
    return;
  }
  const int per_head = unit * 4 / 16, part = unit * (a.filled[blockIdx.x] >> 4) / 16;   // 16-byte pieces
  const u4_t* src = reinterpret_cast<const u4_t*>(base) + (int64_t)cp.x * a.nh * per_head;
  u4_t* dst = reinterpret_cast<u4_t*>(base) + (int64_t)cp.y * a.nh * per_head;
  for (int64_t t = threadIdx.x; t < (int64_t)a.nh * part; t += 256) {
    const int64_t at = t / part * per_head + t % part;
    dst[at] = src[at];
  }
}

struct SelectWs {
  double* lse;
  Best* best;
  size_t total;
};
SelectWs carve_select_ws(int64_t rows, int n_best, void* base) {
  SelectWs W;
  unsigned char* p = reinterpret_cast<unsigned char*>(base);
  const size_t lse = align_up((size_t)rows * 8, 256);
  W.lse = reinterpret_cast<double*>(p);
  W.best = reinterpret_cast<Best*>(p ? p + lse : nullptr);
  W.total = lse + align_up((size_t)rows * n_best * sizeof(Best), 256);
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
  return carve_select_ws((int64_t)n_groups * beams, n_best, nullptr).total;
}

extern "C" int fg_beam_select(const fg_model_cfg* cfg, int32_t n_groups, int32_t beams, int32_t n_best, const float* logits,
                              int64_t row_stride, const float* scores, const int32_t* done, int32_t eos, int32_t* out_beams,
                              int32_t* out_ids, float* out_scores, int32_t* out_done, void* ws, size_t ws_bytes, void* stream) {
  if (!cfg) return FG_ERR_NULL;
  const int rc = check_cfg(cfg);
  if (rc) return rc;
  if (!groups_ok(n_groups, beams) || n_best < 1 || n_best > FG_MAX_BEST || row_stride < cfg->vocab) return FG_ERR_SHAPE;
  if (eos >= cfg->vocab || (done && eos < 0)) return FG_ERR_SHAPE;
  if (n_groups == 0) return FG_OK;
  if (!logits || !scores || !out_beams || !out_ids || !out_scores) return FG_ERR_NULL;
  const int64_t rows = (int64_t)n_groups * beams;
  const SelectWs W = carve_select_ws(rows, n_best, ws);
  if (!ws || ws_bytes < W.total) return FG_ERR_WORKSPACE;
  if ((uintptr_t)ws & 15u) return FG_ERR_SHAPE;
  const SelectArgs a = {logits, row_stride, scores, done, eos, cfg->vocab, beams, n_best, W.lse, W.best, out_beams, out_ids,
                        out_scores, out_done};
  hipStream_t st = as_stream(stream);
  ProfScope prof(FG_K_BEAM_SELECT, st);
  hipLaunchKernelGGL(beam_rows_kernel, dim3((unsigned)rows), dim3(256), 0, st, a);
  FG_LAUNCH_CHECK();
  hipLaunchKernelGGL(beam_merge_kernel, dim3((unsigned)ceil_div(n_groups, 64)), dim3(64), 0, st, a, n_groups);
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
  if (l <= 0 || !groups_ok(n_groups, beams) || pages_per_group < 1 || table_stride < 1) return FG_ERR_SHAPE;
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
    hipLaunchKernelGGL(beam_copy_kernel, dim3((unsigned)rows, (unsigned)nl, c.unit[1] ? 4 : 2), dim3(256), 0, st, c);
    FG_LAUNCH_CHECK();
  }
  return FG_OK;
}
