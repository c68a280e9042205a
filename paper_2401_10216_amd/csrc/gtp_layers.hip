// C entries of the layers around the product (normalisation, dropout,
// attention): argument validation, all of it before the first HIP call, and
// dispatch.  Nothing here allocates or throws.
#include "gtp_layers.hpp"

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "gtp_attn.hpp"
#include "gtp_rng.hpp"

namespace {

gtp_status bad(const char* msg) { return gtp::set_error(GTP_ERR_INVALID_ARG, msg); }
gtp_status unsupported(const char* msg) { return gtp::set_error(GTP_ERR_UNSUPPORTED, msg); }

gtp_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return GTP_OK;
  char msg[160];
  std::snprintf(msg, sizeof(msg), "%s launch: %s", what, hipGetErrorString(e));
  return gtp::set_error(GTP_ERR_HIP, msg);
}

constexpr int64_t kMaxGrid = 0x7fffffff;
constexpr int64_t kMaxElems = INT64_MAX / 8;

// *out = a * b for nonnegative a, b; false where it does not fit.
bool times(int64_t a, int64_t b, int64_t* out) {
  if (a < 0 || b < 0 || (a != 0 && b > kMaxElems / a)) return false;
  *out = a * b;
  return true;
}

bool dtype_known(gtp_dtype d) { return d == GTP_F32 || d == GTP_BF16; }
int64_t elem_size(gtp_dtype d) { return d == GTP_BF16 ? 2 : 4; }
bool aligned(const void* p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(n) == 0; }

struct Span {
  const void* p;
  int64_t bytes;
};
bool overlap(const Span& a, const Span& b) {
  if (!a.p || !b.p || a.bytes <= 0 || b.bytes <= 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x < y + uintptr_t(b.bytes) && y < x + uintptr_t(a.bytes);
}

// Sizes that both directions of the normalisation share.
gtp_status norm_sizes(int L, gtp_dtype dtype, int64_t N, int64_t C, int64_t* elems) {
  if (!dtype_known(dtype)) return bad("dtype must be GTP_F32 or GTP_BF16");
  if (L < 0 || L > 64) return bad("L must be in 0..64");
  int64_t nc = 0;
  if (!times(N, C, &nc) || !times(nc, int64_t(L + 1) * (L + 1), elems))
    return bad("N and C must be >= 0 and N C (L+1)^2 must fit");
  if (N > kMaxGrid || C > kMaxGrid / (L + 2)) return unsupported("more than 2^31 - 1 rows or channels");
  return GTP_OK;
}

}  // namespace

extern "C" {

gtp_status gtp_layer_norm(int L, const void* x, gtp_dtype dtype, const float* w, const float* b, float eps, int64_t N,
                          int64_t C, void* y, float* mean, float* rstd, void* stream) {
  int64_t n = 0;
  const gtp_status s = norm_sizes(L, dtype, N, C, &n);
  if (s != GTP_OK) return s;
  if (!(eps > 0.0f) || !std::isfinite(eps)) return bad("eps must be positive and finite");
  if (n == 0) return GTP_OK;
  if (!x || !y) return bad("NULL data pointer");
  const int64_t es = elem_size(dtype);
  if (!aligned(x, es) || !aligned(y, es) || !aligned(w, 4) || !aligned(b, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
    return bad("misaligned pointer");
  const Span in[] = {{x, n * es}, {w, (L + 1) * C * 4}, {b, C * 4}};
  const Span out[] = {{y, n * es}, {mean, N * 4}, {rstd, N * (L + 1) * 4}};
  for (const Span& o : out)
    for (const Span& i : in)
      if (overlap(o, i) && !(o.p == y && i.p == x && x == y)) return bad("an output overlaps an input");
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return bad("two outputs overlap");
  gtp::NormArgs a{};
  a.x = x;
  a.w = w;
  a.b = b;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  a.N = N;
  a.C = C;
  a.L = L;
  a.bf16 = dtype == GTP_BF16;
  a.eps = eps;
  return launched(gtp::launch_norm(a, static_cast<hipStream_t>(stream)), "gtp_layer_norm");
}

int64_t gtp_layer_norm_backward_work(int L, gtp_dtype dtype, int64_t N, int64_t C) {
  int64_t n = 0;
  if (norm_sizes(L, dtype, N, C, &n) != GTP_OK) return -1;
  return n == 0 ? 0 : gtp::norm_partial_floats(L, N, C, dtype == GTP_BF16) * 4;
}

gtp_status gtp_layer_norm_backward(int L, const void* x, gtp_dtype dtype, const float* w, const float* mean,
                                   const float* rstd, const void* dy, int64_t N, int64_t C, void* dx, float* dw,
                                   float* db, void* work, int64_t work_bytes, void* stream) {
  int64_t n = 0;
  const gtp_status s = norm_sizes(L, dtype, N, C, &n);
  if (s != GTP_OK) return s;
  if (C == 0 || !(dx || dw || db)) return GTP_OK;
  if (n > 0 && (!x || !dy || !mean || !rstd)) return bad("NULL data pointer");
  const int64_t es = elem_size(dtype);
  if (!aligned(x, es) || !aligned(dy, es) || !aligned(dx, es) || !aligned(w, 4) || !aligned(mean, 4) ||
      !aligned(rstd, 4) || !aligned(dw, 4) || !aligned(db, 4) || !aligned(work, 16))
    return bad("misaligned pointer");
  const int64_t need = (dw || db) && n > 0 ? gtp::norm_partial_floats(L, N, C, dtype == GTP_BF16) * 4 : 0;
  if (need > 0 && (!work || work_bytes < need)) return bad("work is smaller than gtp_layer_norm_backward_work says");
  const Span in[] = {{x, n * es}, {dy, n * es}, {w, (L + 1) * C * 4}, {mean, N * 4}, {rstd, N * (L + 1) * 4}};
  const Span out[] = {{dx, n * es}, {dw, (L + 1) * C * 4}, {db, C * 4}, {need > 0 ? work : nullptr, need}};
  for (const Span& o : out)
    for (const Span& i : in)
      if (overlap(o, i) && !(o.p == dx && i.p == dy && dx == dy)) return bad("an output overlaps an input");
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return bad("two outputs overlap");
  gtp::NormArgs a{};
  a.x = x;
  a.dy = dy;
  a.w = w;
  a.mean_in = mean;
  a.rstd_in = rstd;
  a.y = dx;
  a.dw = dw;
  a.db = db;
  a.partial = static_cast<float*>(work);
  a.N = N;
  a.C = C;
  a.L = L;
  a.bf16 = dtype == GTP_BF16;
  return launched(gtp::launch_norm_backward(a, static_cast<hipStream_t>(stream)), "gtp_layer_norm_backward");
}

gtp_status gtp_dropout(const void* x, const void* res, gtp_dtype dtype, double p, const uint64_t* rng, int64_t groups,
                       int64_t K, void* y, void* stream) {
  if (!dtype_known(dtype)) return bad("dtype must be GTP_F32 or GTP_BF16");
  if (!(p >= 0.0 && p < 1.0)) return bad("p must be in [0, 1)");
  int64_t n = 0;
  if (!times(groups, K, &n)) return bad("groups and K must be >= 0 and groups K must fit");
  // a launch holds less than 2^32 threads: 2^24 workgroups of 256, 8192 elements each
  if (K > kMaxGrid || n > (int64_t(1) << 37) - 8192) return unsupported("more elements than one launch can hold");
  if (n == 0) return GTP_OK;
  if (!x || !y || !rng) return bad("NULL data pointer");
  const int64_t es = elem_size(dtype);
  if (!aligned(x, es) || !aligned(res, es) || !aligned(y, es) || !aligned(rng, 8)) return bad("misaligned pointer");
  const Span out{y, n * es};
  if ((y != x && overlap(out, {x, n * es})) || (y != res && overlap(out, {res, n * es})) || overlap(out, {rng, 16}))
    return bad("y overlaps an input");
  const uint32_t t = gtp::drop_threshold(p);
  return launched(gtp::launch_dropout(x, res, dtype == GTP_BF16, t, gtp::drop_scale(t), rng, groups, K, y,
                                      static_cast<hipStream_t>(stream)),
                  "gtp_dropout");
}

}  // extern "C"

namespace {

// A strided tensor of T rows and `heads` heads: whether it is well formed, its
// extent in bytes.  Outputs' rows must not overlap each other.
bool rows_fine(const gtp_rows* r, int64_t T, int heads, int d, int64_t es, bool output, const char** why) {
  if (T == 0) return true;
  if (!r || !r->data) return *why = "NULL data pointer", false;
  if (!aligned(r->data, es)) return *why = "misaligned pointer", false;
  int64_t a = 0, b = 0;
  if (r->row < 0 || r->head < 0 || !times(T - 1, r->row, &a) || !times(heads - 1, r->head, &b) ||
      a + b > kMaxElems - d)
    return *why = "strides must be >= 0 and the tensor's extent must fit", false;
  if (output) {
    const bool rows_outer = (heads == 1 || r->head >= d) && (T == 1 || r->row >= b + d);
    const bool heads_outer = (T == 1 || r->row >= d) && (heads == 1 || r->head >= a + d);
    if (!rows_outer && !heads_outer) return *why = "an output's rows overlap", false;
  }
  return true;
}

struct Rows {
  const gtp_rows* r;
  int64_t T, heads;
};

int64_t extent(const Rows& t, int d, int64_t es) {
  return t.T == 0 ? 0 : ((t.T - 1) * t.r->row + (t.heads - 1) * t.r->head + d) * es;
}

// Whether two strided tensors may share memory: their extents meet, they are not two
// column ranges of rows with one stride (slices of a packed tensor), and, where both
// strides are the same (a dimension of one index has any), some of their rows meet.
bool rows_overlap(const Rows& a, const Rows& b, int d, int64_t es) {
  if (!a.r || !b.r || a.T == 0 || b.T == 0 || !a.r->data || !b.r->data) return false;
  if (!overlap({a.r->data, extent(a, d, es)}, {b.r->data, extent(b, d, es)})) return false;
  const int64_t row = a.T > 1 ? a.r->row : b.T > 1 ? b.r->row : 0;
  if (b.T > 1 && b.r->row != row) return true;
  // where b's first element lies behind a's: their extents meet, so it is in their range
  const int64_t at = (int64_t(reinterpret_cast<uintptr_t>(b.r->data)) - int64_t(reinterpret_cast<uintptr_t>(a.r->data))) / es;
  const int64_t wa = (a.heads - 1) * a.r->head + d, wb = (b.heads - 1) * b.r->head + d;
  if (row > 0 && wa <= row && wb <= row) {
    const int64_t column = (at % row + row) % row;
    if (column >= wa && column + wb <= row) return false;
  }
  const int64_t head = a.heads > 1 ? a.r->head : b.heads > 1 ? b.r->head : 0;
  if (b.heads > 1 && b.r->head != head) return true;
  // b's row t', head h' lies at + (t' - t) row + (h' - h) head behind a's row t, head h:
  // walk the shorter dimension, and find where the other comes nearest
  const bool by_head = std::max(a.heads, b.heads) <= std::max(a.T, b.T);
  const int64_t na = by_head ? a.heads : a.T, nb = by_head ? b.heads : b.T, step = by_head ? head : row;
  const int64_t ma = by_head ? a.T : a.heads, mb = by_head ? b.T : b.heads, other = by_head ? row : head;
  for (int64_t i = 1 - na; i < nb; ++i) {
    const int64_t x = at + i * step;
    const int64_t j0 = std::clamp<int64_t>(other > 0 ? -x / other : 0, 1 - ma, mb - 1);
    for (int64_t j = std::max(j0 - 1, 1 - ma); j <= std::min(j0 + 1, mb - 1); ++j)
      if (x + j * other < d && x + j * other > -d) return true;
  }
  return false;
}

bool rows_vec(const gtp_rows* r, int64_t es) {
  return !r || !r->data || (aligned(r->data, 16) && r->row * es % 16 == 0 && r->head * es % 16 == 0);
}

gtp_status attn_sizes(const gtp_attn* a, gtp::AttnArgs* g) {
  if (!a) return bad("NULL attention description");
  if (!dtype_known(a->dtype)) return bad("dtype must be GTP_F32 or GTP_BF16");
  if (a->H < 1 || a->Hk < 1 || a->H % a->Hk != 0) return bad("H must be a positive multiple of Hk");
  if (a->d < 1) return bad("d must be positive");
  if (a->d > 256) return unsupported("heads longer than 256");
  if (a->B < 0 || a->Tq < 0 || a->Tk < 0 || a->max_q < 0 || a->max_k < 0) return bad("sizes must be >= 0");
  int64_t t = 0;
  if (!a->q_off && (!times(a->B, a->max_q, &t) || t != a->Tq)) return bad("without q_off, Tq must be B max_q");
  if (!a->k_off && (!times(a->B, a->max_k, &t) || t != a->Tk)) return bad("without k_off, Tk must be B max_k");
  if (a->max_q > a->Tq || a->max_k > a->Tk) return bad("max_q and max_k must not exceed Tq and Tk");
  if (!aligned(a->q_off, 8) || !aligned(a->k_off, 8)) return bad("misaligned pointer");
  const float scale2 = a->scale * 1.4426950408889634f;  // in units of log 2
  if (!std::isfinite(a->scale) || !std::isfinite(scale2)) return bad("scale must be finite, times log2(e) too");
  if (!(a->p >= 0.0 && a->p < 1.0)) return bad("p must be in [0, 1)");
  int64_t n = 0;
  if (!times(a->Tq, int64_t(a->H) * a->d, &n) || !times(a->Tk, int64_t(a->Hk) * a->d, &n))
    return bad("the tensors' sizes must fit");
  // the parts of a split call: 2 x 128 of fp32 for dk and dv
  if (n > kMaxElems >> 10) return unsupported("more rows than the work's size can count");
  // workgroups, counted generously: 32 rows or keys each
  const int64_t G = a->H / a->Hk;
  int64_t w = 0;
  if (!times((a->max_q + 31) / 32 + 1, G * a->Hk, &w) || !times(w, a->B, &w) || w > kMaxGrid / 64 ||
      !times((a->max_k + 31) / 32 + 1, 2 * a->Hk, &w) || !times(w, a->B, &w) || w > kMaxGrid / 64 ||
      !times(a->Tq, a->H, &w) || w > kMaxGrid)
    return unsupported("more work than one launch can hold");
  const uint32_t th = gtp::drop_threshold(a->p);
  if (th && !a->rng) return bad("rng is NULL");
  if (!aligned(a->rng, 8)) return bad("misaligned pointer");
  g->q_off = a->q_off;
  g->k_off = a->k_off;
  g->mask = a->key_mask;
  g->rng = a->rng;
  g->B = a->B;
  g->Tq = a->Tq;
  g->Tk = a->Tk;
  g->max_q = a->max_q;
  g->max_k = a->max_k;
  g->H = a->H;
  g->Hk = a->Hk;
  g->G = int(G);
  g->d = a->d;
  g->splits = 1;
  g->scale = a->scale;
  g->scale2 = scale2;
  g->threshold = th;
  g->keep = gtp::drop_scale(th);
  g->bf16 = a->dtype == GTP_BF16;
  return GTP_OK;
}

gtp::AttnRows rows_of(const gtp_rows* r) { return r ? gtp::AttnRows{r->data, r->row, r->head} : gtp::AttnRows{}; }

// The forward: the parts of a split call and their lse.  The backward: the rows'
// deltas, then the parts of dq or of dk and dv, one after the other in the same place.
int64_t delta_bytes(const gtp::AttnArgs& g) { return (g.Tq * g.H * 4 + 15) / 16 * 16; }
int64_t attn_work(const gtp::AttnArgs& g, int backward) {
  const int64_t s = gtp::attn_row_splits(g, backward), rows = s > 1 ? s * g.Tq * g.H * (g.d + (backward ? 0 : 1)) * 4 : 0;
  if (!backward) return rows;
  const int64_t t = gtp::attn_key_splits(g), keys = t > 1 ? 2 * t * g.Tk * g.Hk * g.d * 4 : 0;
  return delta_bytes(g) + (rows > keys ? rows : keys);
}

// Checks of `n` inputs and outputs against each other, the row statistics, the
// work and the index arrays.
gtp_status attn_memory(const gtp_attn* a, const Rows* in, int n_in, const Rows* out, int n_out, Span lse, bool lse_out,
                       Span work, bool* vec) {
  const int64_t es = elem_size(a->dtype);
  const char* why = nullptr;
  *vec = a->d * es % 16 == 0;
  for (int i = 0; i < n_in; ++i) {
    if (!rows_fine(in[i].r, in[i].T, in[i].heads, a->d, es, false, &why)) return bad(why);
    *vec = *vec && rows_vec(in[i].r, es);
  }
  for (int i = 0; i < n_out; ++i) {
    if (!out[i].r) continue;
    if (!rows_fine(out[i].r, out[i].T, out[i].heads, a->d, es, true, &why)) return bad(why);
    *vec = *vec && rows_vec(out[i].r, es);
  }
  if (lse.bytes > 0 && !lse.p) return bad("NULL data pointer");
  if (!aligned(lse.p, 4) || !aligned(work.p, 16)) return bad("misaligned pointer");
  const Span small[] = {{a->q_off, (a->B + 1) * 8}, {a->k_off, (a->B + 1) * 8}, {a->key_mask, a->Tk}, {a->rng, 16}};
  const Span own[] = {lse, work};
  for (int i = 0; i < n_out; ++i) {
    if (!out[i].r || out[i].T == 0) continue;
    const Span o{out[i].r->data, extent(out[i], a->d, es)};
    for (int j = 0; j < n_in; ++j)
      if (rows_overlap(out[i], in[j], a->d, es)) return bad("an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (rows_overlap(out[i], out[j], a->d, es)) return bad("two outputs overlap");
    for (const Span& t : small)
      if (overlap(o, t)) return bad("an output overlaps an input");
    for (const Span& t : own)
      if (overlap(o, t)) return bad("an output overlaps lse or work");
  }
  for (int j = 0; j < n_in; ++j) {
    if (!in[j].r || in[j].T == 0) continue;
    const Span i{in[j].r->data, extent(in[j], a->d, es)};
    if (overlap(work, i) || (lse_out && overlap(lse, i))) return bad("lse or work overlaps an input");
  }
  for (const Span& t : small)
    if (overlap(work, t) || (lse_out && overlap(lse, t))) return bad("lse or work overlaps an input");
  return overlap(lse, work) ? bad("lse overlaps work") : GTP_OK;
}

}  // namespace

extern "C" {

int64_t gtp_attention_work(const gtp_attn* a, int backward) {
  gtp::AttnArgs g{};
  if (attn_sizes(a, &g) != GTP_OK) return -1;
  return attn_work(g, backward);
}

gtp_status gtp_attention(const gtp_attn* a, const gtp_rows* q, const gtp_rows* k, const gtp_rows* v, const gtp_rows* o,
                         float* lse, void* work, int64_t work_bytes, void* stream) {
  gtp::AttnArgs g{};
  gtp_status s = attn_sizes(a, &g);
  if (s != GTP_OK) return s;
  const int64_t need = attn_work(g, 0);
  if (need > 0 && (!work || work_bytes < need)) return bad("work is smaller than gtp_attention_work says");
  if (a->Tq > 0 && !o) return bad("NULL data pointer");
  const Rows in[] = {{q, a->Tq, a->H}, {k, a->Tk, a->Hk}, {v, a->Tk, a->Hk}}, out[] = {{o, a->Tq, a->H}};
  s = attn_memory(a, in, 3, out, 1, {lse, a->Tq * a->H * 4}, true, {need > 0 ? work : nullptr, need}, &g.vec);
  if (s != GTP_OK) return s;
  if (a->B == 0 || a->max_q == 0) return GTP_OK;
  g.q = rows_of(q);
  g.k = rows_of(k);
  g.v = rows_of(v);
  g.out = rows_of(o);
  g.lse = lse;
  g.part = static_cast<float*>(work);
  g.splits = gtp::attn_row_splits(g, false);
  return launched(gtp::launch_attn_fwd(g, static_cast<hipStream_t>(stream)), "gtp_attention");
}

gtp_status gtp_attention_backward(const gtp_attn* a, const gtp_rows* q, const gtp_rows* k, const gtp_rows* v,
                                  const gtp_rows* o, const gtp_rows* dout, const float* lse, const gtp_rows* dq,
                                  const gtp_rows* dk, const gtp_rows* dv, void* work, int64_t work_bytes,
                                  void* stream) {
  gtp::AttnArgs g{};
  gtp_status s = attn_sizes(a, &g);
  if (s != GTP_OK) return s;
  if ((dk == nullptr) != (dv == nullptr)) return bad("dk and dv are computed together");
  if (!dq && !dk) return GTP_OK;
  const int64_t need = attn_work(g, 1);
  if (need > 0 && (!work || work_bytes < need)) return bad("work is smaller than gtp_attention_work says");
  const Rows in[] = {{q, a->Tq, a->H}, {k, a->Tk, a->Hk}, {v, a->Tk, a->Hk}, {o, a->Tq, a->H}, {dout, a->Tq, a->H}};
  const Rows out[] = {{dq, a->Tq, a->H}, {dk, a->Tk, a->Hk}, {dv, a->Tk, a->Hk}};
  s = attn_memory(a, in, 5, out, 3, {lse, a->Tq * a->H * 4}, false, {need > 0 ? work : nullptr, need}, &g.vec);
  if (s != GTP_OK) return s;
  if (a->B == 0) return GTP_OK;
  g.q = rows_of(q);
  g.k = rows_of(k);
  g.v = rows_of(v);
  g.o = rows_of(o);
  g.dout = rows_of(dout);
  g.out = rows_of(dq);
  g.dk = rows_of(dk);
  g.dv = rows_of(dv);
  g.lse = const_cast<float*>(lse);
  g.delta = static_cast<float*>(work);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = a->Tq > 0 ? gtp::launch_attn_delta(g, st) : hipSuccess;
  g.part = reinterpret_cast<float*>(static_cast<char*>(work) + delta_bytes(g));
  if (e == hipSuccess && dq && a->max_q > 0) {
    g.splits = gtp::attn_row_splits(g, true);
    e = gtp::launch_attn_dq(g, st);
    if (e == hipSuccess && g.splits > 1) e = gtp::launch_attn_sum(g, g.part, g.splits, false, g.out, st);
  }
  if (e == hipSuccess && dk && a->max_k > 0) {
    g.splits = gtp::attn_key_splits(g);
    e = gtp::launch_attn_dkv(g, st);
    const int64_t one = g.splits * g.Tk * g.Hk * g.d;
    if (e == hipSuccess && g.splits > 1) e = gtp::launch_attn_sum(g, g.part, g.splits, true, g.dk, st);
    if (e == hipSuccess && g.splits > 1) e = gtp::launch_attn_sum(g, g.part + one, g.splits, true, g.dv, st);
  }
  return launched(e, "gtp_attention_backward");
}

}  // extern "C"
