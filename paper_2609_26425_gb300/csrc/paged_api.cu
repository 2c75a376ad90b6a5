// paged_api.cu -- host side of the rotary and paged entry points of
// include/qwm.h: argument validation, the paged descriptor and launch plans.
#include <new>
#include <utility>

#include "paged.cuh"

struct qwm_paged {
  qwm_paged_config cfg;
  bool codes;                   // 8-bit pages
  uint8_t* base;
  CUtensorMap map, half_map;    // half_map: of 8-bit pages of 128 channels, boxes of 64 of them
  int32_t page_log2;
  int nsm;
  uint64_t wait_ns;
  int32_t idle_role;
};

namespace {

using qwm::PagedPlan;

constexpr int64_t kMost = (int64_t)1 << 30;

int ilog2(int x) {
  int l = 0;
  while ((1 << l) < x) ++l;
  return l;
}

// The status of a call whose CUDA call failed.  The runtime keeps such an error for
// whoever asks next: it is taken here, so that no later call reports it as its own.
qwm_status cuda_error() {
  cudaGetLastError();
  return QWM_ERR_CUDA;
}

bool paged_supported(const qwm_paged_config* c) {
  if (c->kv_heads < 1 || c->kv_heads > 4096) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return false;
  if (c->dtype != QWM_BF16 && c->dtype != QWM_F16) return false;
  if (c->num_pages < 1 || c->num_pages > (((int64_t)1 << 31) - 1) / (2 * c->kv_heads)) return false;
  return true;
}

// Rows (token, head) of the pages
int64_t page_rows(const qwm_paged_config* c) { return c->num_pages * 2 * c->kv_heads * c->page_tokens; }
size_t paged_bytes(const qwm_paged_config* c, bool codes) {
  if (!c || !paged_supported(c)) return 0;
  const size_t rows = (size_t)page_rows(c);
  return QWM_PAGED_HEADER_BYTES + (codes ? rows * (c->head_dim + 2) : rows * c->head_dim * 2);
}
uint8_t* pages_of(const qwm_paged* c) { return c->base + QWM_PAGED_HEADER_BYTES; }
__half* scales_of(const qwm_paged* c) {
  return c->codes ? reinterpret_cast<__half*>(pages_of(c) + (size_t)page_rows(&c->cfg) * c->cfg.head_dim) : nullptr;
}

qwm_status paged_init(qwm_paged** out, const qwm_paged_config* cfg, void* dev_buf, size_t bytes, bool codes, void* stream) {
  if (!out || !cfg || !dev_buf) return QWM_ERR_INVALID_ARG;
  *out = nullptr;
  if (!paged_supported(cfg)) return QWM_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(dev_buf) & 255u) != 0) return QWM_ERR_INVALID_ARG;
  if (bytes < paged_bytes(cfg, codes)) return QWM_ERR_CAPACITY;
  qwm_paged* c = new (std::nothrow) qwm_paged();
  if (!c) return QWM_ERR_INVALID_ARG;
  c->cfg = *cfg;
  c->codes = codes;
  c->base = static_cast<uint8_t*>(dev_buf);
  c->page_log2 = ilog2(cfg->page_tokens);
  c->wait_ns = 2000000000ull;
  const int64_t blocks = cfg->num_pages * 2 * cfg->kv_heads;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&c->nsm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      !(codes ? qwm::make_code_map(&c->map, pages_of(c), blocks, cfg->page_tokens, cfg->head_dim, cfg->head_dim) &&
                    qwm::make_code_map(&c->half_map, pages_of(c), blocks, cfg->page_tokens, cfg->head_dim, 64)
              : qwm::make_page_map(&c->map, pages_of(c), blocks, cfg->page_tokens, cfg->head_dim, cfg->dtype)) ||
      cudaMemsetAsync(dev_buf, 0, QWM_PAGED_HEADER_BYTES, static_cast<cudaStream_t>(stream)) != cudaSuccess) {
    delete c;
    return cuda_error();
  }
  *out = c;
  return QWM_OK;
}

// A tensor that the kernels can read in 16-byte vectors.
bool rows_ok(const qwm_rows* r) {
  return r->data && (reinterpret_cast<uintptr_t>(r->data) & 15u) == 0 && (r->token_stride & 7) == 0 &&
         (r->head_stride & 7) == 0 && r->token_stride >= 0 && r->head_stride >= 0 && r->heads >= 1 &&
         r->token_stride < (int64_t)1 << 31 && r->head_stride < (int64_t)1 << 31;
}
// Whether rows d + n ts + h hs and n' ts + h' hs of two tensors [N][H] share an
// element for some |n - n'| < N and |h - h'| < H: by the differences of the shorter
// axis, with those of the other that come nearest.  `self`: not a row and itself
// (both strides are positive, or 0 with one row).
bool rows_meet(int64_t d, int64_t N, int64_t ts, int64_t H, int64_t hs, int D, bool self) {
  if (H > N) {
    std::swap(H, N);
    std::swap(hs, ts);
  }
  for (int64_t h = 1 - H; h < H; ++h) {
    const int64_t x = d + h * hs;
    for (int64_t near = ts > 0 ? -x / ts - 1 : 0, i = 0; i < (ts > 0 ? 3 : 1); ++i) {
      const int64_t n = near + i;
      if (n <= -N || n >= N || (self && n == 0 && h == 0)) continue;
      const int64_t gap = x + n * ts;
      if (gap < D && gap > -D) return true;
    }
  }
  return false;
}
// A tensor that is written: no two (token, head) may share a row.
bool out_ok(const qwm_rows* r, int64_t N, int D) {
  if (!rows_ok(r)) return false;
  const int64_t H = r->heads, ts = N > 1 ? r->token_stride : 0, hs = H > 1 ? r->head_stride : 0;
  if ((N > 1 && ts < D) || (H > 1 && hs < D)) return false;
  // one axis's rows lie within a step of the other, or it takes a closer look
  return N <= 1 || H <= 1 || ts >= (H - 1) * hs + D || hs >= (N - 1) * ts + D || !rows_meet(0, N, ts, H, hs, D, true);
}

// Whether an output [N][heads] overlaps its input.  Tensors of one base address, or of
// equal strides, are told exactly; of others nothing is known here (false).
bool overlaps(const qwm_rows* in, const qwm_rows* out, int64_t N, int D) {
  const int64_t H = in->heads;
  const int64_t ts = N > 1 ? in->token_stride : 0, hs = H > 1 ? in->head_stride : 0;
  const int64_t to = N > 1 ? out->token_stride : 0, ho = H > 1 ? out->head_stride : 0;
  const int64_t d = (static_cast<const char*>(out->data) - static_cast<const char*>(in->data)) / 2;
  if (d == 0) return true;
  if (d >= (N - 1) * ts + (H - 1) * hs + D || -d >= (N - 1) * to + (H - 1) * ho + D || ts != to || hs != ho) return false;
  const int64_t w = (H - 1) * hs + D, r = ts >= w ? (d % ts + ts) % ts : 0;   // slices of one projection lie apart
  return !(r >= w && ts - r >= w) && rows_meet(d, N, ts, H, hs, D, false);
}
// An output over its own input: the same rows, or none of them.
bool in_place_ok(const qwm_rows* in, const qwm_rows* out, int64_t N, int D) {
  const bool same = in->data == out->data && (N <= 1 || in->token_stride == out->token_stride) &&
                    (in->heads <= 1 || in->head_stride == out->head_stride);
  return same || !overlaps(in, out, N, D);
}

qwm_status check_rope(const qwm_rope_config* c) {
  if (c->dtype != QWM_BF16 && c->dtype != QWM_F16) return QWM_ERR_UNSUPPORTED;
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8) return QWM_ERR_UNSUPPORTED;
  int64_t P = 0;
  for (int i = 0; i < 3; ++i) {
    if (c->pairs[i] < 0 || c->pairs[i] > 128) return QWM_ERR_INVALID_ARG;
    P += c->pairs[i];
  }
  if (P < 1 || 2 * P > c->head_dim || P % (c->interleaved ? 4 : 8)) return QWM_ERR_UNSUPPORTED;
  return QWM_OK;
}

void set_rope(qwm::RopeArgs& a, const qwm_rope_config* c, const float* inv_freq, const int32_t* pos, float sign) {
  a.P = 0;
  for (int i = 0; i < 3; ++i) {
    a.pairs[i] = c->pairs[i];
    a.P += c->pairs[i];
  }
  a.inv_freq = inv_freq;
  a.pos = pos;
  a.sign = sign;
}

void add_segment(qwm::RopeArgs& a, const qwm_rows* src, const qwm_rows* dst, bool rotate, int page) {
  qwm::RopeSegment& g = a.seg[a.nseg++];
  g.src = src->data;
  g.s_tok = (int32_t)src->token_stride;
  g.s_head = (int32_t)src->head_stride;
  g.heads = src->heads;
  g.dst = dst ? dst->data : nullptr;
  g.d_tok = dst ? (int32_t)dst->token_stride : 0;
  g.d_head = dst ? (int32_t)dst->head_stride : 0;
  g.rotate = rotate;
  g.page = page;
  a.total_heads += src->heads;
}

qwm_status rope_impl(const qwm_rope_config* cfg, const float* inv_freq, const int32_t* pos, int64_t N,
                     const qwm_rows* q, const qwm_rows* q_out, const qwm_rows* k, const qwm_rows* k_out, float sign,
                     void* stream) {
  if (!cfg || !q || !q_out || N < 0 || !k != !k_out) return QWM_ERR_INVALID_ARG;
  const qwm_status st = check_rope(cfg);
  if (st != QWM_OK) return st;
  if (N == 0) return QWM_OK;
  if (!inv_freq || !pos) return QWM_ERR_INVALID_ARG;
  if (N > kMost) return QWM_ERR_UNSUPPORTED;
  if (!rows_ok(q) || !out_ok(q_out, N, cfg->head_dim) || q->heads != q_out->heads ||
      !in_place_ok(q, q_out, N, cfg->head_dim))
    return QWM_ERR_INVALID_ARG;
  if (k && (!rows_ok(k) || !out_ok(k_out, N, cfg->head_dim) || k->heads != k_out->heads ||
            !in_place_ok(k, k_out, N, cfg->head_dim)))
    return QWM_ERR_INVALID_ARG;
  qwm::RopeArgs a{};
  a.D = cfg->head_dim;
  a.N = N;
  set_rope(a, cfg, inv_freq, pos, sign);
  add_segment(a, q, q_out, true, -1);
  if (k) add_segment(a, k, k_out, true, -1);
  return qwm::launch_rope(a, cfg->dtype, cfg->interleaved != 0, static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? QWM_OK
             : cuda_error();
}

qwm_status check_batch(const qwm_paged* c, const qwm_paged_batch* b) {
  if (b->num_seqs < 0 || b->table_stride < 0 || b->max_q < 0 || b->max_kv < 0 || b->tokens < 0)
    return QWM_ERR_INVALID_ARG;
  if (b->num_seqs > 65535 || b->tokens > kMost || b->max_kv > kMost ||
      (int64_t)b->table_stride * c->cfg.page_tokens > kMost)
    return QWM_ERR_UNSUPPORTED;
  if (b->tokens > 0 && (b->num_seqs < 1 || b->max_q < 1 || !b->q_offsets || !b->kv_len || !b->page_table))
    return QWM_ERR_INVALID_ARG;
  return QWM_OK;
}

bool mask_ok(const qwm_mask* m) {
  return m->block >= 1 && m->block <= kMost && m->window >= 0 && m->sinks >= 0 &&
         (m->window == 0 || m->window >= m->block);
}

PagedPlan make_plan(const qwm_paged* c, const qwm_paged_batch* b, int32_t q_heads, const qwm_mask* m, bool split) {
  const int G = q_heads / c->cfg.kv_heads;
  const int64_t rows = (int64_t)b->max_q * G;
  // the most tokens that the rows of one group see: the last row's window, and
  // what the first row's window holds before it
  int64_t seen = b->max_kv;
  if (m->window > 0) {
    const int64_t w = (int64_t)m->window + m->sinks + m->block + 256;
    if (w < seen) seen = w;
  }
  const int B = b->num_seqs, Hk = c->cfg.kv_heads, D = c->cfg.head_dim;
  return qwm::step_blocks(B, Hk, D, rows, seen, c->nsm, c->codes)
             ? qwm::plan_step(B, Hk, D, (int)rows, seen, c->nsm, split, c->codes)
             : qwm::plan_chunk(B, Hk, D, rows, seen, c->nsm, split, c->codes);
}

// A workspace: counters, at the same place for every call (they stay zero between
// calls of whatever sizes), then (max, sum) pairs and partial outputs, each
// 256-byte aligned.  A step CTA has two parts (of the groups at the ends of its
// stretch), a chunk group nsplit.
struct Carve {
  size_t ml, o, total;
};
Carve carve(const PagedPlan& p, int D) {
  Carve w{};
  const size_t rows = (size_t)(p.step ? 2 : p.groups - (p.whole > 0 ? p.whole : 0)) * p.nsplit * p.rows;
  w.ml = QWM_PAGED_COUNTER_BYTES;
  w.o = w.ml + (rows * 8 + 255) / 256 * 256;
  w.total = w.o + rows * D * 4;
  return w;
}

}  // namespace

extern "C" {

qwm_status qwm_rope(const qwm_rope_config* cfg, const float* inv_freq, const int32_t* pos, int64_t N,
                    const qwm_rows* q, const qwm_rows* q_out, const qwm_rows* k, const qwm_rows* k_out,
                    void* stream) {
  return rope_impl(cfg, inv_freq, pos, N, q, q_out, k, k_out, 1.0f, stream);
}

qwm_status qwm_rope_backward(const qwm_rope_config* cfg, const float* inv_freq, const int32_t* pos, int64_t N,
                             const qwm_rows* dq, const qwm_rows* dq_out, const qwm_rows* dk, const qwm_rows* dk_out,
                             void* stream) {
  return rope_impl(cfg, inv_freq, pos, N, dq, dq_out, dk, dk_out, -1.0f, stream);
}

size_t qwm_paged_bytes(const qwm_paged_config* c) { return paged_bytes(c, false); }
size_t qwm_paged_bytes_e4m3(const qwm_paged_config* c) { return paged_bytes(c, true); }

qwm_status qwm_paged_init(qwm_paged** out, const qwm_paged_config* cfg, void* dev_buf, size_t bytes, void* stream) {
  return paged_init(out, cfg, dev_buf, bytes, false, stream);
}
qwm_status qwm_paged_init_e4m3(qwm_paged** out, const qwm_paged_config* cfg, void* dev_buf, size_t bytes, void* stream) {
  return paged_init(out, cfg, dev_buf, bytes, true, stream);
}

void qwm_paged_free(qwm_paged* c) { delete c; }

qwm_status qwm_paged_status(qwm_paged* c, int32_t* status, void* stream) {
  if (!c || !status) return QWM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int32_t v = 0;
  if (cudaMemcpyAsync(&v, c->base, sizeof v, cudaMemcpyDeviceToHost, s) != cudaSuccess) return cuda_error();
  if (cudaStreamSynchronize(s) != cudaSuccess) return cuda_error();
  if (v != 0 && cudaMemsetAsync(c->base, 0, sizeof v, s) != cudaSuccess) return cuda_error();
  *status = v;
  return QWM_OK;
}

qwm_status qwm_paged_set_wait_limit(qwm_paged* c, uint64_t ns) {
  if (!c || ns < 1000ull || ns > 60000000000ull) return QWM_ERR_INVALID_ARG;
  c->wait_ns = ns;
  return QWM_OK;
}

qwm_status qwm_paged_set_idle_role(qwm_paged* c, int32_t role) {
  if (!c || (role != 0 && role != QWM_ROLE_PAGE_LOADS)) return QWM_ERR_INVALID_ARG;
  c->idle_role = role;
  return QWM_OK;
}

qwm_status qwm_paged_append(qwm_paged* c, const qwm_paged_batch* b, const qwm_rows* k, const qwm_rows* v,
                            const qwm_rope_config* rope, const float* inv_freq, const int32_t* pos,
                            const qwm_rows* q, const qwm_rows* q_out, void* stream) {
  if (!c || !b || !k || !v || !q != !q_out) return QWM_ERR_INVALID_ARG;
  const int D = c->cfg.head_dim;
  if (rope) {
    const qwm_status st = check_rope(rope);
    if (st != QWM_OK) return st;
    if (rope->head_dim != D || rope->dtype != c->cfg.dtype) return QWM_ERR_INVALID_ARG;
  }
  const qwm_status st = check_batch(c, b);
  if (st != QWM_OK) return st;
  if (b->tokens == 0) return QWM_OK;
  if (rope && (!inv_freq || !pos)) return QWM_ERR_INVALID_ARG;
  if (!rows_ok(k) || !rows_ok(v) || k->heads != c->cfg.kv_heads || v->heads != c->cfg.kv_heads)
    return QWM_ERR_INVALID_ARG;
  if (q && (!rows_ok(q) || !out_ok(q_out, b->tokens, D) || q->heads != q_out->heads ||
            !in_place_ok(q, q_out, b->tokens, D)))
    return QWM_ERR_INVALID_ARG;
  qwm::RopeArgs a{};
  a.D = D;
  a.N = b->tokens;
  if (rope) set_rope(a, rope, inv_freq, pos, 1.0f);
  if (q) add_segment(a, q, q_out, rope != nullptr, -1);
  add_segment(a, k, nullptr, rope != nullptr, 0);
  add_segment(a, v, nullptr, false, 1);
  a.q_off = b->q_offsets;
  a.kv_len = b->kv_len;
  a.table = b->page_table;
  a.B = b->num_seqs;
  a.table_stride = b->table_stride;
  a.max_q = b->max_q;
  a.max_kv = b->max_kv;
  a.page_log2 = c->page_log2;
  a.kv_heads = c->cfg.kv_heads;
  a.num_pages = c->cfg.num_pages;
  a.pages = pages_of(c);
  a.scales = scales_of(c);
  a.status = reinterpret_cast<int32_t*>(c->base);
  return (c->codes ? qwm::launch_store : qwm::launch_rope)(a, c->cfg.dtype, !rope || rope->interleaved,
                                                           static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? QWM_OK
             : cuda_error();
}

qwm_status qwm_paged_read(qwm_paged* c, const qwm_paged_batch* b, const qwm_rows* k_out, const qwm_rows* v_out,
                          void* stream) {
  if (!c || !b || (!k_out && !v_out)) return QWM_ERR_INVALID_ARG;
  const qwm_status st = check_batch(c, b);
  if (st != QWM_OK) return st;
  if (b->tokens == 0) return QWM_OK;
  const int D = c->cfg.head_dim;
  const qwm_rows* out[2] = {k_out, v_out};
  for (const qwm_rows* r : out)
    if (r && (!out_ok(r, b->tokens, D) || r->heads != c->cfg.kv_heads)) return QWM_ERR_INVALID_ARG;
  if (k_out && v_out && overlaps(k_out, v_out, b->tokens, D)) return QWM_ERR_INVALID_ARG;
  for (const qwm_rows* r : out) {                    // nor over the pages themselves
    if (!r) continue;
    const uint8_t *lo = static_cast<const uint8_t*>(r->data), *end = c->base + paged_bytes(&c->cfg, c->codes);
    const int64_t ts = b->tokens > 1 ? r->token_stride : 0, hs = r->heads > 1 ? r->head_stride : 0;
    if (lo < end && lo + 2 * ((b->tokens - 1) * ts + (r->heads - 1) * hs + D) > c->base) return QWM_ERR_INVALID_ARG;
  }
  qwm::ReadArgs a{};
  for (int i = 0; i < 2; ++i) {
    if (!out[i]) continue;
    a.out[i] = out[i]->data;
    a.o_tok[i] = (int32_t)out[i]->token_stride;
    a.o_head[i] = (int32_t)out[i]->head_stride;
  }
  a.D = D;
  a.N = b->tokens;
  a.q_off = b->q_offsets;
  a.kv_len = b->kv_len;
  a.table = b->page_table;
  a.B = b->num_seqs;
  a.table_stride = b->table_stride;
  a.max_q = b->max_q;
  a.max_kv = b->max_kv;
  a.page_log2 = c->page_log2;
  a.kv_heads = c->cfg.kv_heads;
  a.num_pages = c->cfg.num_pages;
  a.pages = pages_of(c);
  a.scales = scales_of(c);
  a.status = reinterpret_cast<int32_t*>(c->base);
  return qwm::launch_read(a, c->cfg.dtype, static_cast<cudaStream_t>(stream)) == cudaSuccess ? QWM_OK : cuda_error();
}

size_t qwm_paged_attend_workspace_bytes(const qwm_paged* c, const qwm_paged_batch* b, int32_t q_heads,
                                        const qwm_mask* mask) {
  if (!c || !b || !mask || check_batch(c, b) != QWM_OK || !mask_ok(mask) || q_heads < 1 ||
      q_heads % c->cfg.kv_heads || b->tokens == 0)
    return 0;
  const PagedPlan p = make_plan(c, b, q_heads, mask, true);
  return p.nsplit > 1 ? carve(p, c->cfg.head_dim).total : 0;
}

qwm_status qwm_paged_attend(qwm_paged* c, const qwm_paged_batch* b, const qwm_rows* q, const qwm_mask* mask,
                            float sm_scale, const qwm_rows* out, float* lse, void* workspace, size_t workspace_bytes,
                            void* stream) {
  if (!c || !b || !q || !mask || !out) return QWM_ERR_INVALID_ARG;
  qwm_status st = check_batch(c, b);
  if (st != QWM_OK) return st;
  if (!mask_ok(mask) || !(sm_scale > 0.0f) || sm_scale > 1.0e38f) return QWM_ERR_INVALID_ARG;  // x log2(e) fits
  if (workspace && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return QWM_ERR_INVALID_ARG;
  if (b->tokens == 0) return QWM_OK;
  const int D = c->cfg.head_dim;
  if (!rows_ok(q) || !out_ok(out, b->tokens, D) || q->heads != out->heads || q->heads % c->cfg.kv_heads ||
      overlaps(q, out, b->tokens, D))
    return QWM_ERR_INVALID_ARG;
  if ((int64_t)b->max_q * (q->heads / c->cfg.kv_heads) > (int64_t)1 << 38) return QWM_ERR_UNSUPPORTED;  // the grid's x
  PagedPlan p = make_plan(c, b, q->heads, mask, workspace != nullptr);
  if (p.nsplit > 1 && workspace_bytes < carve(p, D).total) p = make_plan(c, b, q->heads, mask, false);
  qwm::PagedArgs a{};
  a.q = q->data;
  a.q_tok = q->token_stride;
  a.q_head = q->head_stride;
  a.out = out->data;
  a.o_tok = out->token_stride;
  a.o_head = out->head_stride;
  a.lse = lse;
  a.N = b->tokens;
  a.q_off = b->q_offsets;
  a.kv_len = b->kv_len;
  a.table = b->page_table;
  a.B = b->num_seqs;
  a.table_stride = b->table_stride;
  a.max_q = b->max_q;
  a.max_kv = b->max_kv;
  a.Hk = c->cfg.kv_heads;
  a.G = q->heads / c->cfg.kv_heads;
  a.page_log2 = c->page_log2;
  a.num_pages = c->cfg.num_pages;
  a.pages = pages_of(c);
  a.scales = scales_of(c);
  a.block = mask->block;
  a.window = mask->window;
  a.sinks = mask->sinks;
  a.scale = sm_scale;
  a.status = reinterpret_cast<int32_t*>(c->base);
  a.wait_ns = c->wait_ns;
  a.idle = c->idle_role == QWM_ROLE_PAGE_LOADS;
  a.nsplit = p.nsplit;
  a.min_tiles = p.nsplit > 1 ? p.min_tiles : 1 << 24;
  a.whole = p.step ? -1 : p.whole;
  a.wide = p.wide;
  a.blocks = p.step ? p.blocks : 1;
  if (p.nsplit > 1) {
    const Carve w = carve(p, D);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.counter = reinterpret_cast<int32_t*>(ws);
    a.part_ml = reinterpret_cast<float2*>(ws + w.ml);
    a.part_o = reinterpret_cast<float*>(ws + w.o);
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = p.step ? qwm::launch_paged_step(a, c->map, D, c->cfg.dtype, s)
                               : qwm::launch_paged_chunk(a, c->map, c->half_map, D, c->cfg.dtype, s);
  return e == cudaSuccess ? QWM_OK : cuda_error();
}

}  // extern "C"
