// Host side of rotary positions and of the paged cache: argument checking, size arithmetic and launches.
// See include/skvq.h for the contract of every entry point.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <memory>
#include <new>

#include "skvq_paged.h"

using namespace skvq;

struct skvq_rope {
  int head_dim;
  RopeTable tab;
  double frequencies[kRopeMaxPairs];
};

struct skvq_paged {
  PagedLayout L;
  int device = 0;
  int n_cus = 256;
  int max_tokens = 0;
  void *dev_consts = nullptr;  // k_offset, v_offset, k_place, clip_k, clip_v, errors
  char last_error[256] = "";
};

namespace {

constexpr double kTwoPi = 6.283185307179586476925286766559;
constexpr int kMaxWindow = 1 << 20;

// The device that the cache lives on is the current one for the length of a call.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    if (hipGetDevice(&before_) == hipSuccess && before_ != device) changed_ = hipSetDevice(device) == hipSuccess;
  }
  ~OnDevice() {
    if (changed_) (void)hipSetDevice(before_);
  }

 private:
  int before_ = 0;
  bool changed_ = false;
};

int fail(skvq_paged *c, hipError_t e, const char *what) {
  snprintf(c->last_error, sizeof c->last_error, "%s: %s", what, hipGetErrorString(e));
  return SKVQ_ERR_HIP;
}

bool aligned(const void *p) { return !((uintptr_t)p & 15); }

int check_config(const skvq_paged_config *c) {
  if (!c) return SKVQ_ERR_INVALID_ARG;
  if (c->n_kv_heads < 1 || c->n_q_heads < 1 || c->window < 1 || c->n_sink < 0 || c->n_pages < 1 || c->max_seqs < 1 || c->max_tokens < 1)
    return SKVQ_ERR_INVALID_ARG;
  if (c->n_q_heads % c->n_kv_heads) return SKVQ_ERR_INVALID_ARG;
  if (c->window > kMaxWindow || c->n_sink > kMaxWindow) return SKVQ_ERR_INVALID_ARG;
  if (!(c->sm_scale >= 0.0f) || !std::isfinite(c->sm_scale)) return SKVQ_ERR_INVALID_ARG;
  if (c->head_dim != kD || c->n_q_heads / c->n_kv_heads > 16 || c->n_kv_heads > 65535) return SKVQ_ERR_UNSUPPORTED;
  if (c->group_size != 32 && c->group_size != 64 && c->group_size != 128) return SKVQ_ERR_UNSUPPORTED;
  if (c->k_bits != SKVQ_BITS_4 || c->v_bits != SKVQ_BITS_4) return SKVQ_ERR_UNSUPPORTED;
  if (c->meta_format != SKVQ_META_F32 && c->meta_format != SKVQ_META_F16 && c->meta_format != SKVQ_META_FP8_E4M3) return SKVQ_ERR_UNSUPPORTED;
  if (c->dtype != SKVQ_DTYPE_F16 && c->dtype != SKVQ_DTYPE_BF16) return SKVQ_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return SKVQ_ERR_UNSUPPORTED;
  // (rows of the token arrays and of an attention's row blocks are counted in 32 bits)
  if ((long long)c->max_tokens * c->n_q_heads > 0x7fffffffll) return SKVQ_ERR_UNSUPPORTED;
  if (!c->perm_k || !c->perm_v || !c->clip_k || !c->clip_v) return SKVQ_ERR_INVALID_ARG;
  const int ng = kD / c->group_size;
  for (const int32_t *perm : {c->perm_k, c->perm_v})
    for (int h = 0; h < c->n_kv_heads; ++h) {
      bool seen[kD] = {false};
      for (int p = 0; p < kD; ++p) {
        const int32_t ch = perm[(size_t)h * kD + p];
        if (ch < 0 || ch >= kD || seen[ch]) return SKVQ_ERR_INVALID_ARG;
        seen[ch] = true;
      }
    }
  for (const float *clip : {c->clip_k, c->clip_v})
    for (size_t x = 0; x < (size_t)c->n_kv_heads * ng; ++x)
      if (!(clip[x] > 0.0f && clip[x] <= 1.0f)) return SKVQ_ERR_INVALID_ARG;
  return SKVQ_OK;
}

size_t meta_size(int fmt) { return fmt == SKVQ_META_FP8_E4M3 ? 1 : fmt == SKVQ_META_F16 ? 2 : 4; }

void compute_sizes(const skvq_paged_config *c, size_t bytes[4]) {
  const size_t part = (size_t)c->page_size * (kD + 4 * (kD / c->group_size) * meta_size(c->meta_format));
  bytes[0] = (size_t)c->n_pages * c->n_kv_heads * part;
  bytes[1] = bytes[2] = (size_t)c->max_seqs * c->n_kv_heads * ((size_t)c->window + c->n_sink) * kD * 2;
  bytes[3] = (size_t)c->max_tokens * c->n_q_heads * (kPagedMaxSplits + paged_row_chunks(c->window, c->n_sink)) * kPartialStride * sizeof(float);
}

// What every call checks of its batch; SKVQ_OK with *empty set where there is nothing to do.
int check_batch(const skvq_paged *c, const skvq_batch *b, bool *empty) {
  *empty = false;
  if (!c || !b || b->n_seqs < 0 || b->n_tokens < 0 || b->n_seqs > c->L.max_seqs) return SKVQ_ERR_INVALID_ARG;
  if (b->n_seqs == 0 || b->n_tokens == 0) {
    *empty = true;
    return SKVQ_OK;
  }
  if (!b->cu_tokens || !b->seq_lens || !b->page_table || b->table_stride < 1) return SKVQ_ERR_INVALID_ARG;
  return SKVQ_OK;
}
bool rows_ok(const void *p, int64_t stride, int heads) { return p && aligned(p) && stride % 8 == 0 && stride >= (int64_t)heads * kD; }

}  // namespace

extern "C" {

int skvq_rope_create(const skvq_rope_config *c, skvq_rope **out) {
  if (!out) return SKVQ_ERR_INVALID_ARG;
  *out = nullptr;
  if (!c) return SKVQ_ERR_INVALID_ARG;
  if (c->head_dim < 2 || c->rotary_dim < 2 || c->rotary_dim > c->head_dim || c->rotary_dim % 2) return SKVQ_ERR_INVALID_ARG;
  if (c->head_dim > SKVQ_ROPE_MAX_HEAD_DIM) return SKVQ_ERR_UNSUPPORTED;
  if (c->layout != SKVQ_ROPE_HALF && c->layout != SKVQ_ROPE_INTERLEAVED) return SKVQ_ERR_INVALID_ARG;
  if (!std::isfinite(c->amplitude) || c->amplitude < 0.0) return SKVQ_ERR_INVALID_ARG;
  const int half = c->rotary_dim / 2;
  auto positive = [](double x) { return std::isfinite(x) && x > 0.0; };
  double f[kRopeMaxPairs], amplitude = 1.0;
  if (c->frequencies) {
    for (int i = 0; i < half; ++i) f[i] = c->frequencies[i];
  } else {
    const bool bands = c->scaling == SKVQ_ROPE_SCALE_YARN || c->scaling == SKVQ_ROPE_SCALE_BANDS;
    if (c->scaling < SKVQ_ROPE_SCALE_NONE || c->scaling > SKVQ_ROPE_SCALE_BANDS || !positive(c->base)) return SKVQ_ERR_INVALID_ARG;
    if (c->scaling != SKVQ_ROPE_SCALE_NONE && !positive(c->factor)) return SKVQ_ERR_INVALID_ARG;
    if (bands && (!positive(c->original_context) || !positive(c->low) || !std::isfinite(c->high) || c->high <= c->low)) return SKVQ_ERR_INVALID_ARG;
    if (c->scaling == SKVQ_ROPE_SCALE_YARN && (c->factor <= 1.0 || c->base <= 1.0)) return SKVQ_ERR_INVALID_ARG;
    const double r = c->rotary_dim;
    double base = c->base;
    if (c->scaling == SKVQ_ROPE_SCALE_NTK) base *= std::pow(c->factor, r / (r > 2.0 ? r - 2.0 : 1.0));
    double low = 0.0, high = 0.0;
    if (c->scaling == SKVQ_ROPE_SCALE_YARN) {
      // the pair (as a real number) that turns `turns` times over the original context
      auto pair_of = [&](double turns) { return r * std::log(c->original_context / (turns * kTwoPi)) / (2.0 * std::log(c->base)); };
      low = std::fmax(std::floor(pair_of(c->high)), 0.0);
      high = std::fmin(std::ceil(pair_of(c->low)), r - 1.0);
      amplitude = 0.1 * std::log(c->factor) + 1.0;
    }
    for (int i = 0; i < half; ++i) {
      const double x = std::pow(base, -2.0 * i / r);
      double s = 1.0;  // share of the unscaled frequency
      if (c->scaling == SKVQ_ROPE_SCALE_YARN)
        s = 1.0 - std::fmin(std::fmax((i - low) / std::fmax(high - low, 1e-3), 0.0), 1.0);
      else if (c->scaling == SKVQ_ROPE_SCALE_BANDS)
        s = std::fmin(std::fmax((c->original_context * x / kTwoPi - c->low) / (c->high - c->low), 0.0), 1.0);
      else if (c->scaling == SKVQ_ROPE_SCALE_LINEAR)
        s = 0.0;
      f[i] = s == 1.0 ? x : x / c->factor * (1.0 - s) + x * s;
    }
  }
  if (c->amplitude > 0.0) amplitude = c->amplitude;
  for (int i = 0; i < half; ++i)
    if (!std::isfinite(f[i])) return SKVQ_ERR_INVALID_ARG;
  skvq_rope *rope = new (std::nothrow) skvq_rope();
  if (!rope) return SKVQ_ERR_HIP;
  rope->head_dim = c->head_dim;
  rope->tab.half = half;
  rope->tab.interleaved = c->layout == SKVQ_ROPE_INTERLEAVED;
  rope->tab.amplitude = amplitude;
  for (int i = 0; i < half; ++i) {
    rope->frequencies[i] = f[i];
    // turns per token, mod 1, in units of 2^-64 (a long double has 64 bits)
    const long double turns = (long double)f[i] / 6.283185307179586476925286766559005768L;
    const long double part = roundl(ldexpl(turns - floorl(turns), 64));
    rope->tab.turn[i] = part >= 18446744073709551616.0L ? 0u : (uint64_t)part;
  }
  *out = rope;
  return SKVQ_OK;
}

void skvq_rope_destroy(skvq_rope *rope) { delete rope; }

int skvq_rope_frequencies(const skvq_rope *rope, double *frequencies, double *amplitude) {
  if (!rope) return SKVQ_ERR_INVALID_ARG;
  if (frequencies) std::memcpy(frequencies, rope->frequencies, rope->tab.half * sizeof(double));
  if (amplitude) *amplitude = rope->tab.amplitude;
  return SKVQ_OK;
}

int skvq_rope_apply(const skvq_rope *rope, const skvq_rope_tensor *tensors, int32_t n_tensors, int32_t dtype, int32_t batch,
                    int64_t n_tokens, const int32_t *positions, int64_t positions_batch, int64_t start, int32_t transpose,
                    void *hip_stream) {
  if (!rope || !tensors || n_tensors < 1 || n_tensors > 2 || batch < 0 || n_tokens < 0) return SKVQ_ERR_INVALID_ARG;
  if (dtype != SKVQ_DTYPE_F16 && dtype != SKVQ_DTYPE_BF16 && dtype != SKVQ_DTYPE_F32) return SKVQ_ERR_UNSUPPORTED;
  skvq_rope_tensor used[2];
  int n = 0;
  const size_t size = dtype == SKVQ_DTYPE_F32 ? 4 : 2;
  for (int i = 0; i < n_tensors; ++i) {
    if (tensors[i].n_heads < 0 || tensors[i].n_heads > 1 << 20) return SKVQ_ERR_INVALID_ARG;
    if (tensors[i].n_heads > 0) used[n++] = tensors[i];
  }
  if (n == 0 || batch == 0 || n_tokens == 0) return SKVQ_OK;
  for (int i = 0; i < n; ++i) {
    const skvq_rope_tensor &t = used[i];
    if (!t.x || !t.y || (uintptr_t)t.x % size || (uintptr_t)t.y % size) return SKVQ_ERR_INVALID_ARG;
    if (t.x == t.y && (t.x_batch != t.y_batch || t.x_token != t.y_token || t.x_head != t.y_head)) return SKVQ_ERR_INVALID_ARG;
  }
  if (n_tokens > 0x7fffffffll / batch) return SKVQ_ERR_UNSUPPORTED;  // (tokens are counted in 32 bits)
  if (!positions && (start < -(1ll << 31) || start + n_tokens > 1ll << 31)) return SKVQ_ERR_INVALID_ARG;
  const hipError_t e = launch_rope(rope->tab, rope->head_dim, used, n, dtype, batch, (unsigned)n_tokens, positions, positions_batch,
                                   positions ? 0 : (int)start, transpose != 0, (hipStream_t)hip_stream);
  return e == hipSuccess ? SKVQ_OK : SKVQ_ERR_HIP;
}

int skvq_paged_validate_config(const skvq_paged_config *cfg) { return check_config(cfg); }

int skvq_paged_sizes(const skvq_paged_config *cfg, size_t bytes[4]) {
  if (!bytes) return SKVQ_ERR_INVALID_ARG;
  const int rc = check_config(cfg);
  if (rc != SKVQ_OK) return rc;
  compute_sizes(cfg, bytes);
  return SKVQ_OK;
}

int skvq_paged_create(const skvq_paged_config *cfg, const skvq_paged_buffers *bufs, skvq_paged **out) {
  if (!out) return SKVQ_ERR_INVALID_ARG;
  *out = nullptr;
  const int rc = check_config(cfg);
  if (rc != SKVQ_OK) return rc;
  if (!bufs) return SKVQ_ERR_INVALID_ARG;
  for (const void *p : {bufs->pages, bufs->k_rows, bufs->v_rows, bufs->workspace})
    if (!p || !aligned(p)) return SKVQ_ERR_INVALID_ARG;
  std::unique_ptr<skvq_paged> c(new (std::nothrow) skvq_paged());
  if (!c) return SKVQ_ERR_HIP;
  PagedLayout &L = c->L;
  L.Hq = cfg->n_q_heads;
  L.Hk = cfg->n_kv_heads;
  L.R = L.Hq / L.Hk;
  L.recip_R = recip_of(L.R);
  L.G = cfg->group_size;
  L.NG = kD / L.G;
  L.W = cfg->window;
  L.S = cfg->n_sink;
  L.meta_fmt = cfg->meta_format;
  L.meta_size = (int)meta_size(cfg->meta_format);
  L.page_log2 = 0;
  while ((1 << L.page_log2) < cfg->page_size) ++L.page_log2;
  L.n_pages = cfg->n_pages;
  L.max_seqs = cfg->max_seqs;
  L.dtype = cfg->dtype;
  const unsigned P = (unsigned)cfg->page_size, pairs = P * L.NG * 2 * L.meta_size;
  L.v_at = P * (kD / 2);
  L.km_at = 2 * L.v_at;
  L.vm_at = L.km_at + pairs;
  L.part_bytes = L.vm_at + pairs;
  L.sm_scale = cfg->sm_scale > 0.0f ? cfg->sm_scale : 1.0f / std::sqrt((float)kD);
  L.pages = (uint8_t *)bufs->pages;
  L.k_rows = bufs->k_rows;
  L.v_rows = bufs->v_rows;
  L.workspace = (float *)bufs->workspace;
  c->max_tokens = cfg->max_tokens;

  const size_t n_ch = (size_t)L.Hk * kD, n_clip = (size_t)L.Hk * L.NG;
  const size_t off_v = n_ch, off_p = 2 * n_ch, off_ck = 3 * n_ch, off_cv = off_ck + n_clip * 4, off_err = off_cv + n_clip * 4, total = off_err + 4;
  std::unique_ptr<uint8_t[]> host(new (std::nothrow) uint8_t[total]());
  if (!host) return SKVQ_ERR_HIP;
  for (int h = 0; h < L.Hk; ++h)
    for (int m = 0; m < 16; ++m)
      for (int e = 0; e < 8; ++e) {
        const size_t at = (size_t)h * kD + 8 * m + e;
        const int channel = cfg->perm_k[(size_t)h * kD + 32 * (m & 3) + 8 * (m >> 2) + e];
        host[at] = (uint8_t)(2 * channel);
        host[off_p + (size_t)h * kD + channel] = (uint8_t)(8 * m + e);
        host[off_v + at] = (uint8_t)(2 * cfg->perm_v[(size_t)h * kD + 16 * e + m]);
      }
  std::memcpy(&host[off_ck], cfg->clip_k, n_clip * 4);
  std::memcpy(&host[off_cv], cfg->clip_v, n_clip * 4);
  if (hipGetDevice(&c->device) != hipSuccess) return SKVQ_ERR_HIP;
  if (hipMalloc(&c->dev_consts, total) != hipSuccess) return SKVQ_ERR_HIP;
  if (hipMemcpy(c->dev_consts, host.get(), total, hipMemcpyHostToDevice) != hipSuccess) {
    (void)hipFree(c->dev_consts);
    return SKVQ_ERR_HIP;
  }
  uint8_t *d = (uint8_t *)c->dev_consts;
  L.k_offset = d;
  L.v_offset = d + off_v;
  L.k_place = d + off_p;
  L.clip_k = (const float *)(d + off_ck);
  L.clip_v = (const float *)(d + off_cv);
  L.errors = (int *)(d + off_err);
  int n = 0;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, c->device) == hipSuccess && n > 0) c->n_cus = n;
  *out = c.release();
  return SKVQ_OK;
}

void skvq_paged_destroy(skvq_paged *c) {
  if (!c) return;
  {
    OnDevice on(c->device);
    (void)hipFree(c->dev_consts);
  }
  delete c;
}

int skvq_paged_append(skvq_paged *c, const skvq_rope *rope, const skvq_batch *batch, const void *k, int64_t k_stride, const void *v,
                      int64_t v_stride, const void *q, int64_t q_stride, void *q_out, int64_t q_out_stride, void *hip_stream) {
  bool empty;
  const int rc = check_batch(c, batch, &empty);
  if (rc != SKVQ_OK) return rc;
  if (rope && rope->head_dim != kD) return SKVQ_ERR_INVALID_ARG;
  if (empty) return SKVQ_OK;
  if (!rows_ok(k, k_stride, c->L.Hk) || !rows_ok(v, v_stride, c->L.Hk)) return SKVQ_ERR_INVALID_ARG;
  if (q && (!rows_ok(q, q_stride, c->L.Hq) || !rows_ok(q_out, q_out_stride, c->L.Hq) || (q == q_out && q_stride != q_out_stride)))
    return SKVQ_ERR_INVALID_ARG;
  RopeTable none{};
  OnDevice on(c->device);
  const hipError_t e = launch_paged_append(c->L, rope ? rope->tab : none, *batch, TokenRows{k, k_stride}, TokenRows{v, v_stride},
                                           TokenRows{q, q_stride}, q_out, q_out_stride, c->n_cus, (hipStream_t)hip_stream);
  return e == hipSuccess ? SKVQ_OK : fail(c, e, "skvq_paged_append launch");
}

int skvq_paged_read(skvq_paged *c, const skvq_batch *batch, void *k, int64_t k_stride, void *v, int64_t v_stride, void *hip_stream) {
  bool empty;
  const int rc = check_batch(c, batch, &empty);
  if (rc != SKVQ_OK || empty) return rc;
  if ((k && !rows_ok(k, k_stride, c->L.Hk)) || (v && !rows_ok(v, v_stride, c->L.Hk))) return SKVQ_ERR_INVALID_ARG;
  if (!k && !v) return SKVQ_OK;
  OnDevice on(c->device);
  const hipError_t e = launch_paged_read(c->L, *batch, k, k_stride, v, v_stride, c->n_cus, (hipStream_t)hip_stream);
  return e == hipSuccess ? SKVQ_OK : fail(c, e, "skvq_paged_read launch");
}

int skvq_paged_attention(skvq_paged *c, const skvq_batch *batch, const void *q, int64_t q_stride, void *out, int64_t out_stride,
                         float *out_f32, void *hip_stream) {
  bool empty;
  const int rc = check_batch(c, batch, &empty);
  if (rc != SKVQ_OK) return rc;
  if (batch->n_tokens > c->max_tokens) return SKVQ_ERR_INVALID_ARG;
  if (empty) return SKVQ_OK;
  // (query rows: see quotient; work: counted in 32 bits)
  if ((long long)batch->n_tokens * c->L.R >= 1 << 27 || paged_most_work(c->L, *batch) >= kPagedMostWork) return SKVQ_ERR_UNSUPPORTED;
  if (!rows_ok(q, q_stride, c->L.Hq) || (!out && !out_f32) || (out && !rows_ok(out, out_stride, c->L.Hq)) || !aligned(out_f32))
    return SKVQ_ERR_INVALID_ARG;
  OnDevice on(c->device);
  const hipError_t e = launch_paged_attention(c->L, *batch, TokenRows{q, q_stride}, out, out_stride, out_f32, c->n_cus, (hipStream_t)hip_stream);
  return e == hipSuccess ? SKVQ_OK : fail(c, e, "skvq_paged_attention launch");
}

int skvq_paged_errors(skvq_paged *c, int32_t *bits, void *hip_stream) {
  if (!c || !bits) return SKVQ_ERR_INVALID_ARG;
  OnDevice on(c->device);
  const hipStream_t s = (hipStream_t)hip_stream;
  int32_t got = 0;
  const int32_t zero = 0;
  hipError_t e = hipMemcpyAsync(&got, c->L.errors, sizeof got, hipMemcpyDeviceToHost, s);
  if (e == hipSuccess) e = hipStreamSynchronize(s);
  if (e == hipSuccess && got) {
    e = hipMemcpyAsync(c->L.errors, &zero, sizeof zero, hipMemcpyHostToDevice, s);
    if (e == hipSuccess) e = hipStreamSynchronize(s);
  }
  if (e != hipSuccess) return fail(c, e, "skvq_paged_errors read-back");
  *bits = got;
  return SKVQ_OK;
}

const char *skvq_paged_last_error(const skvq_paged *c) { return c ? c->last_error : ""; }

}  // extern "C"
