// C entry points of the attention layer's operators: handles, argument validation and launches
// (declarations and contracts in include/mtstep.h).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <new>

#include "mt_host.h"
#include "mt_mha.h"

using namespace mt;

namespace {

constexpr uint32_t kMagicAttn = 0x4d544154u;  // "MTAT"
constexpr long long kMaxRows = 1ll << 24;     // B*S
constexpr long long kMaxSteps = 1ll << 30;    // B*S*Hq; entries of a table; positions of a row
constexpr int kMaxPages = 1 << 24;

}  // namespace

struct mt_attn {
  uint32_t magic;
  mt_attn_config cfg;
  int page_log2;
  float scale2;             // of the scores, times log2(e)
  void *params = nullptr;   // one allocation: turns [rot/2] in 64 bits, gq, gk [Dh]
  double *turns;
  float *gq, *gk;
  int32_t *err = nullptr;
  int device, num_cu;
};

namespace {

bool valid(const mt_attn *a) { return a && a->magic == kMagicAttn; }
int esize(const mt_attn *a) { return a->cfg.dtype == MT_BF16 ? 2 : 4; }

mt_status check_cfg(const mt_attn_config *c) {
  if (!c) return fail(MT_ERR_ARG, "config is NULL");
  if (c->Hq < 1 || c->Hq > 1024) return fail(MT_ERR_SHAPE, "Hq=%d: need 1..1024", c->Hq);
  if (c->Hk < 1 || c->Hk > c->Hq || c->Hq % c->Hk)
    return fail(MT_ERR_SHAPE, "Hk=%d: need a divisor of Hq=%d", c->Hk, c->Hq);
  if (c->Dh < 8 || c->Dh > 256 || c->Dh % 8) return fail(MT_ERR_SHAPE, "Dh=%d: need a multiple of 8 up to 256", c->Dh);
  if (c->Hq * c->Dh > 65536) return fail(MT_ERR_SHAPE, "Hq*Dh=%d: need at most 65536", c->Hq * c->Dh);
  if (c->page < 8 || c->page > 256 || (c->page & (c->page - 1)))
    return fail(MT_ERR_SHAPE, "page=%d: need 8, 16, 32, 64, 128 or 256", c->page);
  if (c->dtype != MT_F32 && c->dtype != MT_BF16) return fail(MT_ERR_DTYPE, "dtype=%d: need MT_F32 or MT_BF16", c->dtype);
  if (c->window < 0) return fail(MT_ERR_SHAPE, "window=%d: need at least 0", c->window);
  if (c->qk_norm != 0 && c->qk_norm != 1) return fail(MT_ERR_ARG, "qk_norm must be 0 or 1");
  if (c->rot < 0 || c->rot > c->Dh || c->rot % 2) return fail(MT_ERR_SHAPE, "rot=%d: need an even number up to Dh", c->rot);
  if (c->rot_pairs != 0 && c->rot_pairs != 1) return fail(MT_ERR_ARG, "rot_pairs must be 0 or 1");
  if (!(c->scale >= 0.f) || !std::isfinite((float)(c->scale * M_LOG2E)))
    return fail(MT_ERR_ARG, "scale must be finite, also times log2(e), and not negative");
  if (c->qk_norm && (!(c->norm_eps >= 0.f) || !std::isfinite(c->norm_eps)))
    return fail(MT_ERR_ARG, "norm_eps must be finite and not negative");
  return MT_OK;
}

// sizes of a batch of rows
mt_status check_batch(int B, int S, int Hq) {
  if (B < 1 || S < 1 || (long long)B * S > kMaxRows)
    return fail(MT_ERR_SHAPE, "B=%d S=%d: need B, S >= 1 and B*S <= 2^24", B, S);
  if ((long long)B * S * Hq > kMaxSteps) return fail(MT_ERR_SHAPE, "B*S*Hq exceeds 2^30");
  return MT_OK;
}

// page tables of `rows` rows
mt_status check_tables(const mt_attn *a, int rows, int n_blocks, int n_pages) {
  if (n_blocks < 1 || (long long)n_blocks * a->cfg.page > kMaxSteps)
    return fail(MT_ERR_SHAPE, "n_blocks=%d: need n_blocks >= 1 and n_blocks*page <= 2^30", n_blocks);
  if ((long long)rows * n_blocks > kMaxSteps) return fail(MT_ERR_SHAPE, "a table of more than 2^30 entries");
  if (n_pages < 1 || n_pages > kMaxPages) return fail(MT_ERR_SHAPE, "n_pages=%d: need 1..2^24", n_pages);
  return MT_OK;
}

long long page_bytes(const mt_attn *a) { return (long long)a->cfg.Hk * a->cfg.page * a->cfg.Dh * esize(a); }

}  // namespace

extern "C" {

mt_status mt_attn_load(const mt_attn_config *cfg, const mt_attn_weights *w, mt_attn **out) {
  g_err[0] = 0;
  if (!out) return fail(MT_ERR_ARG, "out is NULL");
  *out = nullptr;
  CHECK(check_cfg(cfg));
  const mt_attn_weights none{};
  if (!w) w = &none;
  const int Dh = cfg->Dh, half = cfg->rot / 2;
  if (half && !w->freq && (!(cfg->rot_base > 0.f) || !std::isfinite(cfg->rot_base)))
    return fail(MT_ERR_ARG, "rot_base must be finite and positive");
  for (int i = 0; w->freq && i < half; ++i)
    if (!std::isfinite(w->freq[i])) return fail(MT_ERR_ARG, "freq[%d] is not finite", i);
  mt_attn *a = new (std::nothrow) mt_attn();
  if (!a) return fail(MT_ERR_OOM, "host allocation failed");
  a->magic = kMagicAttn;
  a->cfg = *cfg;
  while ((1 << a->page_log2) < cfg->page) ++a->page_log2;
  a->scale2 = (float)((cfg->scale > 0.f ? (double)cfg->scale : 1.0 / std::sqrt((double)Dh)) * M_LOG2E);
  struct {
    double turns[128];
    float g[512];
  } host;
  constexpr long double kTurn = 6.283185307179586476925286766559L;
  for (int i = 0; i < half; ++i)  // rounded once
    host.turns[i] = (double)((w->freq ? (long double)w->freq[i] : std::pow((long double)cfg->rot_base, -2.0L * i / cfg->rot)) / kTurn);
  for (int i = half; i < 128; ++i) host.turns[i] = 0;
  for (int i = 0; i < 256; ++i) {
    host.g[i] = cfg->qk_norm && w->gq && i < Dh ? w->gq[i] : 1.f;
    host.g[256 + i] = cfg->qk_norm && w->gk && i < Dh ? w->gk[i] : 1.f;
  }
  auto run = [&]() -> mt_status {
    CHECK(query_device(&a->device, &a->num_cu));
    CHECK(alloc(&a->params, sizeof host));
    CHECK(alloc((void **)&a->err, 4));
    HIP_TRY(hipMemcpy(a->params, &host, sizeof host, hipMemcpyHostToDevice));
    const int32_t zero = 0;
    HIP_TRY(hipMemcpy(a->err, &zero, 4, hipMemcpyHostToDevice));
    HIP_TRY(hipDeviceSynchronize());
    a->turns = (double *)a->params;
    a->gq = (float *)((char *)a->params + sizeof host.turns);
    a->gk = a->gq + 256;
    return MT_OK;
  };
  const mt_status s = run();
  if (s != MT_OK) {
    char keep[sizeof g_err];
    std::memcpy(keep, g_err, sizeof keep);
    mt_attn_free(a);
    std::memcpy(g_err, keep, sizeof keep);
    return s;
  }
  *out = a;
  return MT_OK;
}

mt_status mt_attn_free(mt_attn *a) {
  if (!valid(a)) return fail(MT_ERR_ARG, "invalid layer handle");
  (void)hipDeviceSynchronize();
  if (a->params) (void)hipFree(a->params);
  if (a->err) (void)hipFree(a->err);
  a->magic = 0;
  delete a;
  return MT_OK;
}

mt_status mt_attn_append(mt_attn *a, int B, int S, const int32_t *n_new, const int32_t *len, const void *q, int64_t ldq,
                         const void *k, int64_t ldk, const void *v, int64_t ldv, void *q_out, int64_t ldqo,
                         const int32_t *table, int n_blocks, int n_pages, void *k_pages, void *v_pages, void *stream) {
  g_err[0] = 0;
  if (!valid(a)) return fail(MT_ERR_ARG, "invalid layer handle");
  const mt_attn_config &c = a->cfg;
  CHECK(check_batch(B, S, 1));  // no number of heads in all is too large here
  CHECK(check_tables(a, B, n_blocks, n_pages));
  const int es = esize(a);
  const long long rows = (long long)B * S, wq = (long long)c.Hq * c.Dh, wk = (long long)c.Hk * c.Dh;
  if (n_new) CHECK(check_dev_ptr(n_new, "n_new", 4));
  CHECK(check_dev_ptr(len, "len", 4));
  CHECK(check_dev_ptr(table, "table", 4));
  CHECK(check_rows(q, "q", ldq, wq, es));
  CHECK(check_rows(k, "k", ldk, wk, es));
  CHECK(check_rows(v, "v", ldv, wk, es));
  CHECK(check_rows(q_out, "q_out", ldqo, wq, es));
  CHECK(check_dev_ptr(k_pages, "k_pages"));
  CHECK(check_dev_ptr(v_pages, "v_pages"));
  const long long pb = page_bytes(a);
  const bool in_place = q_out == q && ldqo == ldq;
  CHECK(check_overlaps({{"q_out", q_out, rows, ldqo * es, wq * es}, {"k_pages", k_pages, n_pages, pb, pb},
                        {"v_pages", v_pages, n_pages, pb, pb}},
                       {{"q", in_place ? nullptr : q, rows, ldq * es, wq * es},
                        {"k", k, rows, ldk * es, wk * es},
                        {"v", v, rows, ldv * es, wk * es},
                        {"n_new", n_new, B, 4, 4},
                        {"len", len, B, 4, 4},
                        {"table", table, B, n_blocks * 4ll, n_blocks * 4ll}}));
  if (in_place) CHECK(check_overlaps({{"k_pages", k_pages, n_pages, pb, pb}, {"v_pages", v_pages, n_pages, pb, pb}},
                                     {{"q", q, rows, ldq * es, wq * es}}));
  CHECK(check_device(a->device));
  AppendArgs p{};
  p.Hq = c.Hq; p.Hk = c.Hk; p.Dh = c.Dh; p.bf16_io = es == 2;
  p.norm = c.qk_norm; p.rot = c.rot; p.rot_pairs = c.rot_pairs; p.eps = c.norm_eps;
  p.inv_Dh = 1.f / c.Dh;
  p.gq = a->gq; p.gk = a->gk; p.turns = a->turns;
  p.B = B; p.S = S; p.n_new = n_new; p.len = len; p.table = table;
  p.n_blocks = n_blocks; p.n_pages = n_pages; p.page_log2 = a->page_log2;
  p.q = q; p.k = k; p.v = v; p.qo = q_out; p.kp = k_pages; p.vp = v_pages;
  p.ldq = ldq; p.ldk = ldk; p.ldv = ldv; p.ldqo = ldqo;
  p.err = a->err; p.num_cu = a->num_cu;
  HIP_TRY(launch_append(p, (hipStream_t)stream));
  return MT_OK;
}

size_t mt_attn_workspace_bytes(const mt_attn *a, int B, int S, int64_t n_keys) {
  if (!valid(a) || B < 1 || S < 1 || (long long)B * S > kMaxRows || (long long)B * S * a->cfg.Hq > kMaxSteps) return 0;
  if (n_keys < 1 || n_keys > kMaxSteps) return 0;
  return mha_workspace_bytes(a->cfg.Hq, a->cfg.Hk, a->cfg.Dh, a->cfg.dtype == MT_F32, B, S, n_keys, a->cfg.window,
                             a->num_cu);
}

// what both attentions check and pass on
static mt_status mha_args(mt_attn *a, int B, int S, long long n_keys, const int32_t *n_new, const void *q, int64_t ldq,
                          void *y, int64_t ldy, void *ws, size_t ws_bytes, size_t *need, MhaArgs *p) {
  const mt_attn_config &c = a->cfg;
  const int es = esize(a);
  if (n_new) CHECK(check_dev_ptr(n_new, "n_new", 4));
  CHECK(check_rows(q, "q", ldq, (int64_t)c.Hq * c.Dh, es));
  CHECK(check_rows(y, "y", ldy, (int64_t)c.Hq * c.Dh, es));
  CHECK(check_dev_ptr(ws, "ws", 256));
  *need = mt_attn_workspace_bytes(a, B, S, n_keys);
  if (ws_bytes < *need) return fail(MT_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, *need);
  p->Hq = c.Hq; p->Hk = c.Hk; p->G = c.Hq / c.Hk; p->Dh = c.Dh; p->bf16_io = es == 2;
  p->scale = a->scale2;
  p->B = B; p->S = S; p->n_new = n_new;
  p->q = q; p->ldq = ldq; p->y = y; p->ldy = ldy;
  p->ws = ws; p->err = a->err; p->num_cu = a->num_cu;
  return MT_OK;
}

mt_status mt_attn_paged(mt_attn *a, int B, int S, const int32_t *n_new, const int32_t *len, const void *q, int64_t ldq,
                        const int32_t *table, int n_blocks, int n_pages, const void *k_pages, const void *v_pages,
                        void *y, int64_t ldy, void *ws, size_t ws_bytes, void *stream) {
  g_err[0] = 0;
  if (!valid(a)) return fail(MT_ERR_ARG, "invalid layer handle");
  const mt_attn_config &c = a->cfg;
  CHECK(check_batch(B, S, c.Hq));
  CHECK(check_tables(a, B, n_blocks, n_pages));
  CHECK(check_dev_ptr(len, "len", 4));
  CHECK(check_dev_ptr(table, "table", 4));
  CHECK(check_dev_ptr(k_pages, "k_pages"));
  CHECK(check_dev_ptr(v_pages, "v_pages"));
  MhaArgs p{};
  size_t need = 0;
  CHECK(mha_args(a, B, S, (long long)n_blocks * c.page, n_new, q, ldq, y, ldy, ws, ws_bytes, &need, &p));
  const long long es = esize(a), rows = (long long)B * S, wq = (long long)c.Hq * c.Dh * es, pb = page_bytes(a);
  CHECK(check_overlaps({{"y", y, rows, ldy * es, wq}, {"ws", ws, 1, (long long)need, (long long)need}},
                       {{"q", q, rows, ldq * es, wq},
                        {"n_new", n_new, B, 4, 4},
                        {"len", len, B, 4, 4},
                        {"table", table, B, n_blocks * 4ll, n_blocks * 4ll},
                        {"k_pages", k_pages, n_pages, pb, pb},
                        {"v_pages", v_pages, n_pages, pb, pb}}));
  CHECK(check_device(a->device));
  p.window = c.window < kMaxSteps ? c.window : 0;  // no position is that far from another: positions minus it stay in range
  p.k = k_pages; p.v = v_pages; p.len = len; p.table = table;
  p.n_blocks = n_blocks; p.n_pages = n_pages; p.page_log2 = a->page_log2;
  HIP_TRY(launch_mha(p, (hipStream_t)stream));
  return MT_OK;
}

mt_status mt_attn_cross(mt_attn *a, int B, int T, const int32_t *n_q, int S, const float *mask, const void *q, int64_t ldq,
                        const void *k, int64_t ldk, const void *v, int64_t ldv, void *y, int64_t ldy, void *ws,
                        size_t ws_bytes, void *stream) {
  g_err[0] = 0;
  if (!valid(a)) return fail(MT_ERR_ARG, "invalid layer handle");
  const mt_attn_config &c = a->cfg;
  CHECK(check_batch(B, T, c.Hq));
  if (S < 1 || (long long)B * S > kMaxRows) return fail(MT_ERR_SHAPE, "S=%d: need S >= 1 and B*S <= 2^24", S);
  const long long es = esize(a), wq = (long long)c.Hq * c.Dh, wk = (long long)c.Hk * c.Dh;
  if (mask) CHECK(check_dev_ptr(mask, "mask", 4));
  CHECK(check_rows(k, "k", ldk, wk, (int)es));
  CHECK(check_rows(v, "v", ldv, wk, (int)es));
  MhaArgs p{};
  size_t need = 0;
  CHECK(mha_args(a, B, T, S, n_q, q, ldq, y, ldy, ws, ws_bytes, &need, &p));
  const long long rows = (long long)B * T, keys = (long long)B * S;
  CHECK(check_overlaps({{"y", y, rows, ldy * es, wq * es}, {"ws", ws, 1, (long long)need, (long long)need}},
                       {{"q", q, rows, ldq * es, wq * es},
                        {"k", k, keys, ldk * es, wk * es},
                        {"v", v, keys, ldv * es, wk * es},
                        {"n_q", n_q, B, 4, 4},
                        {"mask", mask, keys, 4, 4}}));
  CHECK(check_device(a->device));
  p.k = k; p.v = v; p.ldk = ldk; p.ldv = ldv; p.mask = mask; p.Sk = S;
  HIP_TRY(launch_mha(p, (hipStream_t)stream));
  return MT_OK;
}

size_t mt_pages_workspace_bytes(const mt_attn *a, int M, int n_pages) {
  if (!valid(a) || M < 1 || M > (1 << 20) || n_pages < 1 || n_pages > kMaxPages) return 0;
  return pages_workspace_bytes(M, n_pages);
}

static mt_status pages_args(mt_attn *a, int M_in, int M, const int32_t *table_in, const int32_t *len_in, int n_blocks,
                            int n_pages, int32_t *table_out, int32_t *len_out, int layers, void *ws, size_t ws_bytes,
                            size_t *need, PagesArgs *p) {
  if (M < 1 || M > (1 << 20)) return fail(MT_ERR_SHAPE, "M=%d: need 1..2^20", M);
  if (M_in < 1 || M_in > (1 << 20)) return fail(MT_ERR_SHAPE, "M_in=%d: need 1..2^20", M_in);
  CHECK(check_tables(a, M > M_in ? M : M_in, n_blocks, n_pages));
  if (layers < 1 || layers > 1024) return fail(MT_ERR_SHAPE, "layers=%d: need 1..1024", layers);
  CHECK(check_dev_ptr(table_in, "table_in", 4));
  CHECK(check_dev_ptr(len_in, "len_in", 4));
  CHECK(check_dev_ptr(table_out, "table_out", 4));
  CHECK(check_dev_ptr(len_out, "len_out", 4));
  CHECK(check_dev_ptr(ws, "ws", 256));
  *need = mt_pages_workspace_bytes(a, M, n_pages);
  if (ws_bytes < *need) return fail(MT_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, *need);
  p->M_in = M_in; p->M = M;
  p->table_in = table_in; p->len_in = len_in;
  p->n_blocks = n_blocks; p->n_pages = n_pages; p->page_log2 = a->page_log2;
  p->table_out = table_out; p->len_out = len_out;
  p->layers = layers;
  p->head_bytes = (long long)a->cfg.Dh * esize(a);
  p->Hk = a->cfg.Hk;
  p->ws = ws; p->err = a->err; p->num_cu = a->num_cu;
  return MT_OK;
}

mt_status mt_pages_advance(mt_attn *a, int M_in, int M, const int32_t *src_row, const int32_t *add,
                           const int32_t *table_in, const int32_t *len_in, int n_blocks, int n_pages,
                           int32_t *table_out, int32_t *len_out, int32_t *free_out, int layers, void *k_pages,
                           void *v_pages, void *ws, size_t ws_bytes, void *stream) {
  g_err[0] = 0;
  if (!valid(a)) return fail(MT_ERR_ARG, "invalid layer handle");
  PagesArgs p{};
  size_t need = 0;
  CHECK(pages_args(a, M_in, M, table_in, len_in, n_blocks, n_pages, table_out, len_out, layers, ws, ws_bytes, &need, &p));
  if (!src_row && M != M_in) return fail(MT_ERR_SHAPE, "M=%d and M_in=%d differ without src_row", M, M_in);
  if (src_row) CHECK(check_dev_ptr(src_row, "src_row", 4));
  if (add) CHECK(check_dev_ptr(add, "add", 4));
  if (free_out) CHECK(check_dev_ptr(free_out, "free_out", 4));
  CHECK(check_dev_ptr(k_pages, "k_pages"));
  CHECK(check_dev_ptr(v_pages, "v_pages"));
  const long long row = n_blocks * 4ll, cache = page_bytes(a) * n_pages;
  CHECK(check_overlaps({{"table_out", table_out, M, row, row},
                        {"len_out", len_out, M, 4, 4},
                        {"free_out", free_out, 1, 4, 4},
                        {"ws", ws, 1, (long long)need, (long long)need},
                        {"k_pages", k_pages, layers, cache, cache},
                        {"v_pages", v_pages, layers, cache, cache}},
                       {{"table_in", table_in, M_in, row, row},
                        {"len_in", len_in, M_in, 4, 4},
                        {"src_row", src_row, M, 4, 4},
                        {"add", add, M, 4, 4}}));
  CHECK(check_device(a->device));
  p.row = src_row; p.add = add; p.free_out = free_out;
  p.k_in = p.k_out = k_pages; p.v_in = p.v_out = v_pages;
  p.n_pages_out = n_pages;
  HIP_TRY(launch_advance(p, (hipStream_t)stream));
  return MT_OK;
}

mt_status mt_pages_pack(mt_attn *a, int M, const int32_t *table_in, const int32_t *len_in, int n_blocks, int n_pages,
                        int layers, const void *k_in, const void *v_in, int n_pages_out, int32_t *table_out,
                        int32_t *len_out, int32_t *used_out, void *k_out, void *v_out, void *ws, size_t ws_bytes,
                        void *stream) {
  g_err[0] = 0;
  if (!valid(a)) return fail(MT_ERR_ARG, "invalid layer handle");
  PagesArgs p{};
  size_t need = 0;
  CHECK(pages_args(a, M, M, table_in, len_in, n_blocks, n_pages, table_out, len_out, layers, ws, ws_bytes, &need, &p));
  if (n_pages_out < 1 || n_pages_out > kMaxPages)
    return fail(MT_ERR_SHAPE, "n_pages_out=%d: need 1..2^24", n_pages_out);
  if (used_out) CHECK(check_dev_ptr(used_out, "used_out", 4));
  CHECK(check_dev_ptr(k_in, "k_in"));
  CHECK(check_dev_ptr(v_in, "v_in"));
  CHECK(check_dev_ptr(k_out, "k_out"));
  CHECK(check_dev_ptr(v_out, "v_out"));
  const long long row = n_blocks * 4ll, in = page_bytes(a) * n_pages, out = page_bytes(a) * n_pages_out;
  CHECK(check_overlaps({{"table_out", table_out, M, row, row},
                        {"len_out", len_out, M, 4, 4},
                        {"used_out", used_out, 1, 4, 4},
                        {"ws", ws, 1, (long long)need, (long long)need},
                        {"k_out", k_out, 1, out * layers, out * layers},
                        {"v_out", v_out, 1, out * layers, out * layers}},
                       {{"table_in", table_in, M, row, row},
                        {"len_in", len_in, M, 4, 4},
                        {"k_in", k_in, 1, in * layers, in * layers},
                        {"v_in", v_in, 1, in * layers, in * layers}}));
  CHECK(check_device(a->device));
  p.free_out = used_out;
  p.k_in = k_in; p.v_in = v_in; p.k_out = k_out; p.v_out = v_out;
  p.n_pages_out = n_pages_out;
  HIP_TRY(launch_pack(p, (hipStream_t)stream));
  return MT_OK;
}

mt_status mt_attn_device_errors(mt_attn *a, int32_t *flags) {
  g_err[0] = 0;
  if (!valid(a)) return fail(MT_ERR_ARG, "invalid layer handle");
  if (!flags) return fail(MT_ERR_ARG, "flags is NULL");
  CHECK(check_device(a->device));
  HIP_TRY(hipDeviceSynchronize());
  HIP_TRY(hipMemcpy(flags, a->err, 4, hipMemcpyDeviceToHost));
  const int32_t zero = 0;
  HIP_TRY(hipMemcpy(a->err, &zero, 4, hipMemcpyHostToDevice));
  return MT_OK;
}

}  // extern "C"
