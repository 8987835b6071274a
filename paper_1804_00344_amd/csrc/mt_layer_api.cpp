// C entry points of the recurrent layer's operators: handles, argument validation and launches
// (declarations and contracts in include/mtstep.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>
#include <limits>
#include <new>

#include "mt_host.h"
#include "mt_layer.h"

using namespace mt;

namespace {

constexpr uint32_t kMagicI8 = 0x4d543849u;   // "MT8I"
constexpr uint32_t kMagicSsm = 0x4d545353u;  // "MTSS"
constexpr long long kMaxRows = 1ll << 24;
constexpr long long kMaxPromptElements = 1ll << 34;   // S*D: a grid dimension of blocks
constexpr long long kMaxTokenElements = 1ll << 31;    // M*D
constexpr long long kMaxProductElements = 1ll << 36;  // M*N

}  // namespace

struct mt_i8_matrix {
  uint32_t magic;
  int K, N, Kp, Np;
  int8_t *wq = nullptr;
  float *scale = nullptr;  // [Np]
  float *bias = nullptr;   // [Np], zero padded, or NULL
  int device, num_cu;
};

struct mt_ssm {
  uint32_t magic;
  mt_ssm_config cfg;
  int Np;
  float *params = nullptr;  // one allocation: A2 [D][Np], dt_bias, skip, conv_w [W][D], conv_b
  float *A2, *dt_bias, *skip, *conv_w, *conv_b;
  int32_t *err = nullptr;
  int device, num_cu;
};

namespace {

bool valid(const mt_i8_matrix *w) { return w && w->magic == kMagicI8; }
bool valid(const mt_ssm *c) { return c && c->magic == kMagicSsm; }

mt_status query_device(int *dev, int *ncu) {
  if (hipGetDevice(dev) != hipSuccess ||
      hipDeviceGetAttribute(ncu, hipDeviceAttributeMultiprocessorCount, *dev) != hipSuccess || *ncu <= 0)
    return fail(MT_ERR_HIP, "cannot query the device's compute units");
  return MT_OK;
}

mt_status check_device(int device) {
  int dev = -1;
  HIP_TRY(hipGetDevice(&dev));
  if (dev != device) return fail(MT_ERR_STATE, "loaded on device %d, but device %d is current", device, dev);
  return MT_OK;
}

mt_status alloc(void **p, size_t bytes) {
  const hipError_t e = hipMalloc(p, bytes);
  if (e != hipSuccess) {
    *p = nullptr;
    return fail(MT_ERR_OOM, "hipMalloc(%zu): %s", bytes, hip_error(e));
  }
  return MT_OK;
}

// A range of rows of a wider matrix that a call reads or writes
struct Span {
  const char *name;
  const void *p;
  long long rows, ld, width;  // bytes
};

// Whether two spans share a byte.  Spans of one stride whose columns do not meet do not; other
// strides are compared by their whole ranges.
bool overlap(const Span &a, const Span &b) {
  if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0) return false;
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
  const uintptr_t a1 = a0 + (uintptr_t)((a.rows - 1) * a.ld + a.width), b1 = b0 + (uintptr_t)((b.rows - 1) * b.ld + b.width);
  if (a1 <= b0 || b1 <= a0) return false;
  if (a.ld != b.ld || a.ld <= 0) return true;
  const long long off = (long long)((b0 > a0 ? b0 - a0 : a0 - b0) % (uintptr_t)a.ld);
  const long long lo = b0 > a0 ? a.width : b.width, hi = b0 > a0 ? b.width : a.width;  // of the lower, the upper one
  return off < lo || off + hi > a.ld;
}

// Outputs against every input and against each other (out[i] == in[i] allowed where `same` says so)
mt_status check_overlaps(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    for (const Span &i : ins)
      if (overlap(*o, i)) return fail(MT_ERR_ARG, "%s overlaps %s", o->name, i.name);
    for (auto q = outs.begin(); q != o; ++q)
      if (overlap(*o, *q)) return fail(MT_ERR_ARG, "%s overlaps %s", o->name, q->name);
  }
  return MT_OK;
}

mt_status check_rows(const void *p, const char *name, int64_t ld, int64_t width, int esize) {
  CHECK(check_dev_ptr(p, name, esize));
  if (ld < width || ld > (1ll << 32))
    return fail(MT_ERR_SHAPE, "row stride %lld of %s: need at least its %lld columns", (long long)ld, name,
                (long long)width);
  return MT_OK;
}

mt_status check_prompts(int B, int S, int D) {
  if (B < 1 || S < 1 || (long long)B * S > kMaxRows)
    return fail(MT_ERR_SHAPE, "B=%d S=%d: need B, S >= 1 and B*S <= 2^24", B, S);
  if ((long long)S * D > kMaxPromptElements) return fail(MT_ERR_SHAPE, "S*D exceeds 2^34");
  return MT_OK;
}

mt_status check_tokens(int M, int D, const int32_t *src_row, int n_rows) {
  if (M < 1 || M > kMaxRows) return fail(MT_ERR_SHAPE, "M=%d: need 1..2^24", M);
  if ((long long)M * D > kMaxTokenElements) return fail(MT_ERR_SHAPE, "M*D exceeds 2^31");
  if (n_rows < 1 || n_rows > kMaxRows) return fail(MT_ERR_SHAPE, "n_state_rows=%d: need 1..2^24", n_rows);
  if (!src_row && n_rows < M) return fail(MT_ERR_SHAPE, "n_state_rows=%d < M=%d without src_row", n_rows, M);
  if (src_row) CHECK(check_dev_ptr(src_row, "src_row", 4));
  return MT_OK;
}

mt_status check_io_type(int t, const char *name) {
  if (t != MT_F32 && t != MT_BF16) return fail(MT_ERR_DTYPE, "%s=%d: need MT_F32 or MT_BF16", name, t);
  return MT_OK;
}

mt_status check_ssm_cfg(const mt_ssm_config *c) {
  if (!c) return fail(MT_ERR_ARG, "config is NULL");
  if (c->D < 1 || c->D > 65536) return fail(MT_ERR_SHAPE, "D=%d: need 1..65536", c->D);
  if (c->N < 1 || c->N > 256) return fail(MT_ERR_SHAPE, "N=%d: need 1..256", c->N);
  if (c->G < 1 || c->G > c->D || c->D % c->G) return fail(MT_ERR_SHAPE, "G=%d: need a divisor of D=%d", c->G, c->D);
  if (c->W < 0 || c->W > 8) return fail(MT_ERR_SHAPE, "W=%d: need 0..8", c->W);
  if (c->conv_silu != 0 && c->conv_silu != 1) return fail(MT_ERR_ARG, "conv_silu must be 0 or 1");
  return check_io_type(c->dtype, "dtype");
}

size_t i8_rows(int M) { return rup((size_t)M, kI8Pad); }

}  // namespace

extern "C" {

// ---- products in 8 bits ----

mt_status mt_i8_load(int K, int N, const float *W, const float *bias, mt_i8_matrix **out) {
  g_err[0] = 0;
  if (!out) return fail(MT_ERR_ARG, "out is NULL");
  *out = nullptr;
  if (K < 1 || K > kI8MaxK) return fail(MT_ERR_SHAPE, "K=%d: need 1..%d", K, kI8MaxK);
  if (N < 1 || N > kMaxRows) return fail(MT_ERR_SHAPE, "N=%d: need 1..2^24", N);
  CHECK(check_dev_ptr(W, "W", 4));
  mt_i8_matrix *w = new (std::nothrow) mt_i8_matrix();
  if (!w) return fail(MT_ERR_OOM, "host allocation failed");
  w->magic = kMagicI8;
  w->K = K;
  w->N = N;
  w->Kp = (int)rup(K, kI8KPad);
  w->Np = (int)rup(N, kI8Pad);
  void *stage = nullptr, *bad = nullptr;
  auto run = [&]() -> mt_status {
    CHECK(query_device(&w->device, &w->num_cu));
    CHECK(alloc((void **)&w->wq, (size_t)w->Np * w->Kp));
    CHECK(alloc((void **)&w->scale, (size_t)w->Np * 4));
    CHECK(alloc(&bad, 4));
    HIP_TRY(hipDeviceSynchronize());  // W may be the work of any stream
    const int zero = 0;
    HIP_TRY(hipMemcpy(bad, &zero, 4, hipMemcpyHostToDevice));
    if (bias) {
      CHECK(alloc((void **)&w->bias, (size_t)w->Np * 4));
      HIP_TRY(hipMemset(w->bias, 0, (size_t)w->Np * 4));
      HIP_TRY(hipMemcpy(w->bias, bias, (size_t)N * 4, hipMemcpyDefault));
    }
    const size_t bytes = (size_t)K * N * 4;
    hipPointerAttribute_t at{};
    const bool on_dev = hipPointerGetAttributes(&at, W) == hipSuccess && at.type == hipMemoryTypeDevice &&
                        at.device == w->device;
    (void)hipGetLastError();  // plain host memory has no attributes
    const float *src = W;
    if (!on_dev) {
      CHECK(alloc(&stage, bytes));
      HIP_TRY(hipMemcpy(stage, W, bytes, hipMemcpyDefault));
      src = (const float *)stage;
    }
    HIP_TRY(launch_i8_pack(src, K, N, w->Kp, w->Np, w->wq, w->scale, (int *)bad, nullptr));
    HIP_TRY(hipDeviceSynchronize());
    int flag = 0;
    HIP_TRY(hipMemcpy(&flag, bad, 4, hipMemcpyDeviceToHost));
    if (flag) return fail(MT_ERR_ARG, "W holds a NaN or an infinity");
    return MT_OK;
  };
  const mt_status s = run();
  if (stage) (void)hipFree(stage);
  if (bad) (void)hipFree(bad);
  if (s != MT_OK) {
    char keep[sizeof g_err];
    std::memcpy(keep, g_err, sizeof keep);
    mt_i8_free(w);
    std::memcpy(g_err, keep, sizeof keep);
    return s;
  }
  *out = w;
  return MT_OK;
}

mt_status mt_i8_free(mt_i8_matrix *w) {
  if (!valid(w)) return fail(MT_ERR_ARG, "invalid matrix handle");
  (void)hipDeviceSynchronize();
  for (void *p : {(void *)w->wq, (void *)w->scale, (void *)w->bias})
    if (p) (void)hipFree(p);
  w->magic = 0;
  delete w;
  return MT_OK;
}

size_t mt_i8_workspace_bytes(const mt_i8_matrix *w, int M) {
  if (!valid(w) || M < 1 || M > kMaxRows || (long long)M * w->N > kMaxProductElements) return 0;
  return i8_rows(M) * w->Kp + i8_rows(M) * 4;
}

mt_status mt_i8_product(mt_i8_matrix *w, int M, const void *x, int x_dtype, int64_t ldx, void *y, int y_dtype,
                        int64_t ldy, void *ws, size_t ws_bytes, void *stream) {
  g_err[0] = 0;
  if (!valid(w)) return fail(MT_ERR_ARG, "invalid matrix handle");
  if (M < 1 || M > kMaxRows) return fail(MT_ERR_SHAPE, "M=%d: need 1..2^24", M);
  if ((long long)M * w->N > kMaxProductElements) return fail(MT_ERR_SHAPE, "M*N exceeds 2^36");
  CHECK(check_io_type(x_dtype, "x_dtype"));
  CHECK(check_io_type(y_dtype, "y_dtype"));
  const int ex = x_dtype == MT_BF16 ? 2 : 4, ey = y_dtype == MT_BF16 ? 2 : 4;
  CHECK(check_rows(x, "x", ldx, w->K, ex));
  CHECK(check_rows(y, "y", ldy, w->N, ey));
  CHECK(check_dev_ptr(ws, "ws", 256));
  const size_t need = mt_i8_workspace_bytes(w, M);
  if (ws_bytes < need) return fail(MT_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, need);
  const Span sy{"y", y, M, ldy * ey, (long long)w->N * ey}, sw{"ws", ws, 1, (long long)need, (long long)need};
  CHECK(check_overlaps({sy, sw}, {{"x", x, M, ldx * ex, (long long)w->K * ex}}));
  CHECK(check_device(w->device));
  I8Problem p{};
  p.x = x; p.ldx = ldx; p.x_bf16 = x_dtype == MT_BF16;
  p.wq = w->wq; p.ws = w->scale; p.bias = w->bias;
  p.y = y; p.ldy = ldy; p.y_bf16 = y_dtype == MT_BF16;
  p.M = M; p.N = w->N; p.K = w->K; p.Kp = w->Kp;
  p.xq = (int8_t *)ws;
  p.xs = (float *)((char *)ws + i8_rows(M) * w->Kp);
  p.num_cu = w->num_cu;
  HIP_TRY(launch_i8_product(p, (hipStream_t)stream));
  return MT_OK;
}

// ---- the cell ----

mt_status mt_ssm_load(const mt_ssm_config *cfg, const mt_ssm_weights *w, mt_ssm **out) {
  g_err[0] = 0;
  if (!out) return fail(MT_ERR_ARG, "out is NULL");
  *out = nullptr;
  CHECK(check_ssm_cfg(cfg));
  if (!w) return fail(MT_ERR_ARG, "weights is NULL");
  if (!w->A) return fail(MT_ERR_ARG, "weight A is NULL");
  const int D = cfg->D, N = cfg->N, W = cfg->W;
  if (W > 0 && !w->conv_w) return fail(MT_ERR_ARG, "weight conv_w is NULL (W = %d)", W);
  for (long long i = 0; i < (long long)D * N; ++i)
    if (!(w->A[i] <= 0.f) || !std::isfinite(w->A[i])) return fail(MT_ERR_ARG, "A[%lld] is not finite and <= 0", i);
  mt_ssm *c = new (std::nothrow) mt_ssm();
  if (!c) return fail(MT_ERR_OOM, "host allocation failed");
  c->magic = kMagicSsm;
  c->cfg = *cfg;
  const int Np = c->Np = scan_padded_states(N);
  const size_t total = (size_t)D * (Np + 3 + W);
  float *host = new (std::nothrow) float[total]();
  auto run = [&]() -> mt_status {
    if (!host) return fail(MT_ERR_OOM, "host allocation failed");
    CHECK(query_device(&c->device, &c->num_cu));
    size_t o = 0;
    size_t oA = o, ob = (o += (size_t)D * Np), os = (o += D), ow = (o += D), oc = (o += (size_t)W * D);
    for (int d = 0; d < D; ++d) {
      for (int n = 0; n < N; ++n)  // finite, so that a step of zero keeps the state
        host[oA + (size_t)d * Np + n] =
            (float)std::max((double)w->A[(size_t)d * N + n] * M_LOG2E, -(double)std::numeric_limits<float>::max());
      if (w->dt_bias) host[ob + d] = w->dt_bias[d];
      if (w->skip) host[os + d] = w->skip[d];
      for (int j = 0; j < W; ++j) host[ow + (size_t)j * D + d] = w->conv_w[(size_t)d * W + j];
      if (W > 0 && w->conv_b) host[oc + d] = w->conv_b[d];
    }
    CHECK(alloc((void **)&c->params, total * 4));
    CHECK(alloc((void **)&c->err, 4));
    HIP_TRY(hipMemcpy(c->params, host, total * 4, hipMemcpyHostToDevice));
    const int32_t zero = 0;
    HIP_TRY(hipMemcpy(c->err, &zero, 4, hipMemcpyHostToDevice));
    HIP_TRY(hipDeviceSynchronize());
    c->A2 = c->params + oA;
    c->dt_bias = c->params + ob;
    c->skip = c->params + os;
    c->conv_w = c->params + ow;
    c->conv_b = c->params + oc;
    return MT_OK;
  };
  const mt_status s = run();
  delete[] host;
  if (s != MT_OK) {
    char keep[sizeof g_err];
    std::memcpy(keep, g_err, sizeof keep);
    mt_ssm_free(c);
    std::memcpy(g_err, keep, sizeof keep);
    return s;
  }
  *out = c;
  return MT_OK;
}

mt_status mt_ssm_free(mt_ssm *c) {
  if (!valid(c)) return fail(MT_ERR_ARG, "invalid cell handle");
  (void)hipDeviceSynchronize();
  if (c->params) (void)hipFree(c->params);
  if (c->err) (void)hipFree(c->err);
  c->magic = 0;
  delete c;
  return MT_OK;
}

size_t mt_ssm_workspace_bytes(const mt_ssm *c, int B, int S) {
  if (!valid(c) || B < 1 || S < 1 || (long long)B * S > kMaxRows) return 0;
  if ((long long)S * c->cfg.D > kMaxPromptElements) return 0;
  return scan_workspace_bytes(B, S, c->cfg.D, c->cfg.N, c->num_cu);
}

static mt_status conv_args(mt_ssm *c, int rows, int S, const void *x, int64_t ldx, const void *state_in, void *y,
                           int64_t ldy, void *state_out, ConvArgs *a) {
  const int D = c->cfg.D, es = c->cfg.dtype == MT_BF16 ? 2 : 4;
  CHECK(check_rows(x, "x", ldx, D, es));
  CHECK(check_rows(y, "y", ldy, D, es));
  if (state_in) CHECK(check_dev_ptr(state_in, "state_in"));
  if (state_out) CHECK(check_dev_ptr(state_out, "state_out"));
  a->w = c->conv_w; a->b = c->conv_b;
  a->D = D; a->W = c->cfg.W; a->silu = c->cfg.conv_silu; a->bf16_io = es == 2;
  a->B = rows; a->S = S;
  a->x = x; a->ldx = ldx; a->y = y; a->ldy = ldy;
  a->state_in = state_in; a->state_out = state_out;
  a->err = c->err;
  a->num_cu = c->num_cu;
  return MT_OK;
}

mt_status mt_ssm_conv(mt_ssm *c, int B, int S, const int32_t *len, const void *x, int64_t ldx, const void *state_in,
                      void *y, int64_t ldy, void *state_out, void *stream) {
  g_err[0] = 0;
  if (!valid(c)) return fail(MT_ERR_ARG, "invalid cell handle");
  if (c->cfg.W < 1) return fail(MT_ERR_STATE, "the cell has no convolution (W = 0)");
  CHECK(check_prompts(B, S, c->cfg.D));
  if (len) CHECK(check_dev_ptr(len, "len", 4));
  ConvArgs a{};
  CHECK(conv_args(c, B, S, x, ldx, state_in, y, ldy, state_out, &a));
  const long long D = c->cfg.D, es = a.bf16_io ? 2 : 4, rows = (long long)B * S, sw = (a.W - 1) * D * es;
  CHECK(check_overlaps({{"y", y, rows, ldy * es, D * es}, {"state_out", state_out, B, sw, sw}},
                       {{"x", x, rows, ldx * es, D * es}, {"state_in", state_in, B, sw, sw}, {"len", len, B, 4, 4}}));
  a.len = len;
  CHECK(check_device(c->device));
  HIP_TRY(launch_conv(a, (hipStream_t)stream));
  return MT_OK;
}

mt_status mt_ssm_conv_step(mt_ssm *c, int M, const int32_t *src_row, int n_state_rows, const void *x, int64_t ldx,
                           const void *state_in, void *y, int64_t ldy, void *state_out, void *stream) {
  g_err[0] = 0;
  if (!valid(c)) return fail(MT_ERR_ARG, "invalid cell handle");
  if (c->cfg.W < 1) return fail(MT_ERR_STATE, "the cell has no convolution (W = 0)");
  CHECK(check_tokens(M, c->cfg.D, src_row, n_state_rows));
  if (c->cfg.W == 1)
    state_in = state_out = nullptr;
  else if (!state_in || !state_out)
    return fail(MT_ERR_ARG, "%s is NULL", state_in ? "state_out" : "state_in");
  ConvArgs a{};
  CHECK(conv_args(c, M, 1, x, ldx, state_in, y, ldy, state_out, &a));
  const long long D = c->cfg.D, es = a.bf16_io ? 2 : 4, sw = (a.W - 1) * D * es;
  const bool in_place = !src_row && state_in == state_out;
  CHECK(check_overlaps({{"y", y, M, ldy * es, D * es}, {"state_out", state_out, M, sw, sw}},
                       {{"x", x, M, ldx * es, D * es},
                        {"state_in", in_place ? nullptr : state_in, n_state_rows, sw, sw},
                        {"src_row", src_row, M, 4, 4}}));
  a.row = src_row;
  a.n_rows = n_state_rows;
  CHECK(check_device(c->device));
  HIP_TRY(launch_conv_step(a, (hipStream_t)stream));
  return MT_OK;
}

static mt_status scan_args(mt_ssm *c, int rows, int S, const void *x, int64_t ldx, const void *dt, int64_t lddt,
                           const void *bmat, const void *cmat, int64_t ldbc, const void *z, int64_t ldz,
                           const float *state_in, void *y, int64_t ldy, float *state_out, ScanArgs *a) {
  const int D = c->cfg.D, N = c->cfg.N, G = c->cfg.G, es = c->cfg.dtype == MT_BF16 ? 2 : 4;
  CHECK(check_rows(x, "x", ldx, D, es));
  CHECK(check_rows(dt, "dt", lddt, D, es));
  CHECK(check_rows(bmat, "bmat", ldbc, (int64_t)G * N, es));
  CHECK(check_rows(cmat, "cmat", ldbc, (int64_t)G * N, es));
  if (z) CHECK(check_rows(z, "z", ldz, D, es));
  CHECK(check_rows(y, "y", ldy, D, es));
  if (state_in) CHECK(check_dev_ptr(state_in, "state_in"));
  if (state_out) CHECK(check_dev_ptr(state_out, "state_out"));
  a->A2 = c->A2; a->dt_bias = c->dt_bias; a->skip = c->skip;
  a->D = D; a->N = N; a->Np = c->Np; a->G = G; a->bf16_io = es == 2;
  a->B = rows; a->S = S;
  a->x = x; a->dt = dt; a->bm = bmat; a->cm = cmat; a->z = z; a->y = y;
  a->ldx = ldx; a->lddt = lddt; a->ldbc = ldbc; a->ldz = ldz; a->ldy = ldy;
  a->state_in = state_in; a->state_out = state_out;
  a->err = c->err;
  a->num_cu = c->num_cu;
  return MT_OK;
}

mt_status mt_ssm_scan(mt_ssm *c, int B, int S, const int32_t *len, const void *x, int64_t ldx, const void *dt,
                      int64_t lddt, const void *bmat, const void *cmat, int64_t ldbc, const void *z, int64_t ldz,
                      const float *state_in, void *y, int64_t ldy, float *state_out, void *ws, size_t ws_bytes,
                      void *stream) {
  g_err[0] = 0;
  if (!valid(c)) return fail(MT_ERR_ARG, "invalid cell handle");
  CHECK(check_prompts(B, S, c->cfg.D));
  if (len) CHECK(check_dev_ptr(len, "len", 4));
  CHECK(check_dev_ptr(ws, "ws", 256));
  ScanArgs a{};
  CHECK(scan_args(c, B, S, x, ldx, dt, lddt, bmat, cmat, ldbc, z, ldz, state_in, y, ldy, state_out, &a));
  const size_t need = mt_ssm_workspace_bytes(c, B, S);
  if (ws_bytes < need) return fail(MT_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, need);
  const long long D = c->cfg.D, es = a.bf16_io ? 2 : 4, rows = (long long)B * S, sw = D * c->cfg.N * 4,
                  gn = (long long)c->cfg.G * c->cfg.N * es;
  CHECK(check_overlaps({{"y", y, rows, ldy * es, D * es},
                        {"state_out", state_out, B, sw, sw},
                        {"ws", ws, 1, (long long)need, (long long)need}},
                       {{"x", x, rows, ldx * es, D * es},
                        {"dt", dt, rows, lddt * es, D * es},
                        {"bmat", bmat, rows, ldbc * es, gn},
                        {"cmat", cmat, rows, ldbc * es, gn},
                        {"z", z, rows, ldz * es, D * es},
                        {"state_in", state_in, B, sw, sw},
                        {"len", len, B, 4, 4}}));
  a.len = len;
  a.ws = ws;
  CHECK(check_device(c->device));
  HIP_TRY(launch_scan(a, (hipStream_t)stream));
  return MT_OK;
}

mt_status mt_ssm_step(mt_ssm *c, int M, const int32_t *src_row, int n_state_rows, const void *x, int64_t ldx,
                      const void *dt, int64_t lddt, const void *bmat, const void *cmat, int64_t ldbc, const void *z,
                      int64_t ldz, const float *state_in, void *y, int64_t ldy, float *state_out, void *stream) {
  g_err[0] = 0;
  if (!valid(c)) return fail(MT_ERR_ARG, "invalid cell handle");
  CHECK(check_tokens(M, c->cfg.D, src_row, n_state_rows));
  if (!state_in || !state_out) return fail(MT_ERR_ARG, "%s is NULL", state_in ? "state_out" : "state_in");
  ScanArgs a{};
  CHECK(scan_args(c, M, 1, x, ldx, dt, lddt, bmat, cmat, ldbc, z, ldz, state_in, y, ldy, state_out, &a));
  const long long D = c->cfg.D, es = a.bf16_io ? 2 : 4, sw = D * c->cfg.N * 4, gn = (long long)c->cfg.G * c->cfg.N * es;
  const bool in_place = !src_row && state_in == state_out;
  CHECK(check_overlaps({{"y", y, M, ldy * es, D * es}, {"state_out", state_out, M, sw, sw}},
                       {{"x", x, M, ldx * es, D * es},
                        {"dt", dt, M, lddt * es, D * es},
                        {"bmat", bmat, M, ldbc * es, gn},
                        {"cmat", cmat, M, ldbc * es, gn},
                        {"z", z, M, ldz * es, D * es},
                        {"state_in", in_place ? nullptr : state_in, n_state_rows, sw, sw},
                        {"src_row", src_row, M, 4, 4}}));
  a.row = src_row;
  a.n_rows = n_state_rows;
  CHECK(check_device(c->device));
  HIP_TRY(launch_scan_step(a, (hipStream_t)stream));
  return MT_OK;
}

mt_status mt_ssm_device_errors(mt_ssm *c, int32_t *flags) {
  g_err[0] = 0;
  if (!valid(c)) return fail(MT_ERR_ARG, "invalid cell handle");
  if (!flags) return fail(MT_ERR_ARG, "flags is NULL");
  CHECK(check_device(c->device));
  HIP_TRY(hipDeviceSynchronize());
  HIP_TRY(hipMemcpy(flags, c->err, 4, hipMemcpyDeviceToHost));
  const int32_t zero = 0;
  HIP_TRY(hipMemcpy(c->err, &zero, 4, hipMemcpyHostToDevice));
  return MT_OK;
}

}  // extern "C"
