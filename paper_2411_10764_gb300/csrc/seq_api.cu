// C entry points of the sequence-model operators: argument checks, then the
// launches of sample.cu, embed.cu, scan.cu and scan_grad.cu.  Nothing here
// allocates device memory, but that the first draw or lookup on a device makes the library's own state
// (the error word is part of it) where no other call has.
#include <cmath>

#include "seq.cuh"

namespace {

using namespace mlt;

constexpr int64_t kMaxCount = 0x7FFFFFFFLL;
constexpr int64_t kMaxRow = 1LL << 27;
constexpr int kMaxDraws = 2048;
constexpr int kMaxDim = 1 << 20;

int check_ws(const void* ws, size_t have, size_t need) {
  if (need == 0) return MLT_OK;
  if (ws == nullptr || have < need)
    return api_fail(MLT_EINVAL, "the workspace needs %zu bytes, got %zu", need, ws == nullptr ? size_t(0) : have);
  if (!aligned_to(ws, 256)) return api_fail(MLT_EINVAL, "the workspace must be 256-byte aligned");
  return MLT_OK;
}

int launched(cudaError_t e, long long launches, const char* what) {
  if (launches > 0) api_count_launches(launches);
  if (e != cudaSuccess) return api_fail(MLT_ECUDA, "%s: %s", what, cudaGetErrorString(e));
  return MLT_OK;
}

int check_sample_sizes(int dtype, int64_t rows, int64_t n, int m) {
  if (!dtype_ok(dtype)) return api_fail(MLT_EINVAL, "unknown element type %d", dtype);
  if (rows < 0 || rows > kMaxCount) return api_fail(MLT_EINVAL, "rows must lie in [0, 2^31-1]");
  if (n < 0 || n > kMaxRow) return api_fail(MLT_EINVAL, "n must lie in [0, 2^27], got %lld", static_cast<long long>(n));
  if (m < 1 || m > kMaxDraws) return api_fail(MLT_EINVAL, "m must lie in [1, %d], got %d", kMaxDraws, m);
  return MLT_OK;
}

int check_embed(int dtype, int out_dtype, int64_t tokens, int64_t vocab, int dim) {
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype)) return api_fail(MLT_EINVAL, "unknown element type");
  if (tokens < 0 || tokens > kMaxCount) return api_fail(MLT_EINVAL, "tokens must lie in [0, 2^31-1]");
  if (vocab < 1 || vocab > kMaxCount) return api_fail(MLT_EINVAL, "vocab must lie in [1, 2^31-1]");
  if (dim < 1 || dim > kMaxDim) return api_fail(MLT_EINVAL, "dim must lie in [1, %d], got %d", kMaxDim, dim);
  return MLT_OK;
}

// A stride of an output that keeps rows apart (one row needs none).  Inputs may repeat rows or
// overlap: theirs only must not be negative.
bool stride_ok(int64_t stride, int64_t width, int64_t rows) { return rows <= 1 || stride >= width; }

int check_scan(const mlt_scan_args* a) {
  if (a == nullptr) return api_fail(MLT_EINVAL, "args must be non-NULL");
  if (!dtype_ok(a->dtype)) return api_fail(MLT_EINVAL, "unknown element type %d", a->dtype);
  if (a->batch < 0 || a->batch > 65535) return api_fail(MLT_EINVAL, "batch must lie in [0, 65535], got %d", a->batch);
  if (a->length < 0 || a->length > kMaxCount) return api_fail(MLT_EINVAL, "length must lie in [0, 2^31-1]");
  if (a->dim < 1 || a->dim > kMaxDim) return api_fail(MLT_EINVAL, "dim must lie in [1, %d], got %d", kMaxDim, a->dim);
  if (a->states < 1 || a->states > kScanMaxStates)
    return api_fail(MLT_EINVAL, "states must lie in [1, %d], got %d", kScanMaxStates, a->states);
  if (a->groups < 1 || a->dim % a->groups != 0)
    return api_fail(MLT_EINVAL, "dim must be a multiple of groups, got %d and %d", a->dim, a->groups);
  if (a->taps < 0 || a->taps > kScanMaxTaps)
    return api_fail(MLT_EINVAL, "taps must lie in [0, %d], got %d", kScanMaxTaps, a->taps);
  return MLT_OK;
}

int check_scan_inputs(const mlt_scan_args* a) {
  const int64_t L = a->length;
  if (a->A == nullptr) return api_fail(MLT_EINVAL, "A must be non-NULL");
  if (a->taps > 0 && a->conv_w == nullptr) return api_fail(MLT_EINVAL, "conv_w must be non-NULL with %d taps", a->taps);
  if (L > 0 && (a->x == nullptr || a->dt == nullptr || a->B == nullptr || a->C == nullptr))
    return api_fail(MLT_EINVAL, "x, dt, B and C must be non-NULL");
  struct {
    const char* name;
    const void* p;
    int64_t step, batch;
  } in[] = {{"x", a->x, a->x_step, a->x_batch},
            {"dt", a->dt, a->dt_step, a->dt_batch},
            {"z", a->z, a->z_step, a->z_batch},
            {"B", a->B, a->B_step, a->B_batch},
            {"C", a->C, a->C_step, a->C_batch}};
  for (const auto& t : in) {
    if (t.p == nullptr) continue;
    if (t.step < 0 || t.batch < 0) return api_fail(MLT_EINVAL, "%s: strides must not be negative", t.name);
    if (!aligned_to(t.p, dtype_size(a->dtype))) return api_fail(MLT_EINVAL, "%s is not aligned to its elements", t.name);
  }
  return MLT_OK;
}

}  // namespace

extern "C" {

int mlt_sample_workspace(int dtype, int64_t rows, int64_t n, int m, size_t* bytes_out) {
  if (bytes_out == nullptr) return api_fail(MLT_EINVAL, "bytes_out must be non-NULL");
  const int rc = check_sample_sizes(dtype, rows, n, m);
  if (rc != MLT_OK) return rc;
  *bytes_out = sample_workspace(dtype, rows, n, m, api_sm_count());
  return MLT_OK;
}

int mlt_sample(void* stream, const void* scores, int dtype, int64_t rows, int64_t n, int64_t row_stride,
               const float* noise, int64_t noise_stride, const mlt_sample_rule* rule, const mlt_sample_rule* rules,
               int m, void* workspace, size_t workspace_bytes, int64_t* out_index, float* out_logprob) {
  int rc = check_sample_sizes(dtype, rows, n, m);
  if (rc != MLT_OK) return rc;
  if ((rule == nullptr) == (rules == nullptr)) return api_fail(MLT_EINVAL, "give either rule or rules");
  if (rule != nullptr && !(rule->temperature >= 0.0f && std::isfinite(rule->temperature)))
    return api_fail(MLT_EINVAL, "temperature must be finite and not negative");
  if (rule != nullptr && (std::isnan(rule->top_p) || std::isnan(rule->min_p)))
    return api_fail(MLT_EINVAL, "top_p and min_p must be numbers");
  if (rows == 0) return MLT_OK;
  if (out_index == nullptr || out_logprob == nullptr || (n > 0 && (scores == nullptr || noise == nullptr)))
    return api_fail(MLT_EINVAL, "device buffers must be non-NULL");
  if (row_stride < 0 || noise_stride < 0) return api_fail(MLT_EINVAL, "strides must not be negative");
  if (!aligned_to(scores, dtype_size(dtype)) || !aligned_to(noise, 4) || !aligned_to(rules, 16))
    return api_fail(MLT_EINVAL, "scores and noise must be aligned to their elements, rules to 16 bytes");
  const int sms = api_sm_count();
  rc = check_ws(workspace, workspace_bytes, sample_workspace(dtype, rows, n, m, sms));
  if (rc != MLT_OK) return rc;
  unsigned* err = api_error_word(&rc);
  if (err == nullptr) return rc;
  SampleArgs a{};
  a.scores = scores;
  a.dtype = dtype;
  a.rows = rows;
  a.n = n;
  a.row_stride = rows > 1 ? row_stride : n;
  a.noise = noise;
  a.noise_stride = rows > 1 ? noise_stride : n;
  if (rule != nullptr) a.rule = *rule;
  a.rules = rules;
  a.m = m;
  a.out_index = reinterpret_cast<long long*>(out_index);
  a.out_logprob = out_logprob;
  a.err = err;
  a.ws = workspace;
  a.stall_us = static_cast<unsigned>(api_take_sample_stall() / 1000);
  long long launches = 0;
  const cudaError_t e = launch_sample(a, sms, &launches, static_cast<cudaStream_t>(stream));
  return launched(e, launches, "sample launch");
}

int mlt_embed(void* stream, const void* table, int dtype, int64_t vocab, int dim, int64_t table_stride,
              const void* ids, int ids_64, int64_t tokens, float scale, void* out, int out_dtype,
              int64_t out_stride) {
  int rc = check_embed(dtype, out_dtype, tokens, vocab, dim);
  if (rc != MLT_OK) return rc;
  if (tokens == 0) return MLT_OK;
  if (table == nullptr || ids == nullptr || out == nullptr) return api_fail(MLT_EINVAL, "device buffers must be non-NULL");
  if (table_stride < 0) return api_fail(MLT_EINVAL, "strides must not be negative");
  if (!stride_ok(out_stride, dim, tokens)) return api_fail(MLT_EINVAL, "rows must be at least dim elements apart");
  if (!aligned_to(table, dtype_size(dtype)) || !aligned_to(out, dtype_size(out_dtype)) ||
      !aligned_to(ids, ids_64 ? 8 : 4))
    return api_fail(MLT_EINVAL, "buffers must be aligned to their elements");
  unsigned* err = api_error_word(&rc);
  if (err == nullptr) return rc;
  EmbedArgs a{};
  a.table = table;
  a.in_dtype = dtype;
  a.in_stride = vocab > 1 ? table_stride : dim;
  a.ids = ids;
  a.ids_64 = ids_64;
  a.tokens = tokens;
  a.vocab = vocab;
  a.dim = dim;
  a.scale = scale;
  a.out = out;
  a.out_dtype = out_dtype;
  a.out_stride = tokens > 1 ? out_stride : dim;
  a.err = err;
  long long launches = 0;
  const cudaError_t e = launch_embed(a, api_sm_count(), &launches, static_cast<cudaStream_t>(stream));
  return launched(e, launches, "embed launch");
}

int mlt_embed_grad_workspace(int64_t tokens, int64_t vocab, int dim, size_t* bytes_out) {
  if (bytes_out == nullptr) return api_fail(MLT_EINVAL, "bytes_out must be non-NULL");
  const int rc = check_embed(MLT_F32, MLT_F32, tokens, vocab, dim);
  if (rc != MLT_OK) return rc;
  *bytes_out = embed_grad_workspace(tokens, vocab, dim, api_sm_count());
  return MLT_OK;
}

int mlt_embed_grad(void* stream, const void* grad_out, int dtype, int64_t grad_stride, const void* ids, int ids_64,
                   int64_t tokens, int64_t vocab, int dim, float scale, void* workspace, size_t workspace_bytes,
                   void* grad_table, int out_dtype, int64_t out_stride) {
  int rc = check_embed(dtype, out_dtype, tokens, vocab, dim);
  if (rc != MLT_OK) return rc;
  if (grad_table == nullptr || (tokens > 0 && (grad_out == nullptr || ids == nullptr)))
    return api_fail(MLT_EINVAL, "device buffers must be non-NULL");
  if (grad_stride < 0) return api_fail(MLT_EINVAL, "strides must not be negative");
  if (!stride_ok(out_stride, dim, vocab)) return api_fail(MLT_EINVAL, "rows must be at least dim elements apart");
  if (!aligned_to(grad_out, dtype_size(dtype)) || !aligned_to(grad_table, dtype_size(out_dtype)) ||
      !aligned_to(ids, ids_64 ? 8 : 4))
    return api_fail(MLT_EINVAL, "buffers must be aligned to their elements");
  const int sms = api_sm_count();
  rc = check_ws(workspace, workspace_bytes, embed_grad_workspace(tokens, vocab, dim, sms));
  if (rc != MLT_OK) return rc;
  unsigned* err = api_error_word(&rc);
  if (err == nullptr) return rc;
  EmbedArgs a{};
  a.table = grad_out;
  a.in_dtype = dtype;
  a.in_stride = tokens > 1 ? grad_stride : dim;
  a.ids = ids;
  a.ids_64 = ids_64;
  a.tokens = tokens;
  a.vocab = vocab;
  a.dim = dim;
  a.scale = scale;
  a.out = grad_table;
  a.out_dtype = out_dtype;
  a.out_stride = vocab > 1 ? out_stride : dim;
  a.err = err;
  a.ws = workspace;
  long long launches = 0;
  const cudaError_t e = launch_embed_grad(a, sms, &launches, static_cast<cudaStream_t>(stream));
  return launched(e, launches, "embedding gradient launch");
}

int mlt_scan_workspace(const mlt_scan_args* args, size_t* bytes_out) {
  if (bytes_out == nullptr) return api_fail(MLT_EINVAL, "bytes_out must be non-NULL");
  const int rc = check_scan(args);
  if (rc != MLT_OK) return rc;
  *bytes_out = scan_workspace(*args, api_sm_count());
  return MLT_OK;
}

int mlt_scan(void* stream, const mlt_scan_args* args, void* workspace, size_t workspace_bytes) {
  int rc = check_scan(args);
  if (rc != MLT_OK) return rc;
  if (args->batch == 0) return MLT_OK;
  rc = check_scan_inputs(args);
  if (rc != MLT_OK) return rc;
  if (args->length > 0 && args->y == nullptr) return api_fail(MLT_EINVAL, "y must be non-NULL");
  if (!stride_ok(args->y_step, args->dim, args->length) || !stride_ok(args->y_batch, args->dim, args->batch))
    return api_fail(MLT_EINVAL, "y: positions and sequences must be at least dim elements apart");
  if (!aligned_to(args->y, dtype_size(args->dtype))) return api_fail(MLT_EINVAL, "y is not aligned to its elements");
  const int sms = api_sm_count();
  rc = check_ws(workspace, workspace_bytes, scan_workspace(*args, sms));
  if (rc != MLT_OK) return rc;
  long long launches = 0;
  const cudaError_t e = launch_scan(*args, workspace, sms, &launches, static_cast<cudaStream_t>(stream));
  return launched(e, launches, "scan launch");
}

int mlt_scan_grad_workspace(const mlt_scan_args* args, size_t* bytes_out) {
  if (bytes_out == nullptr) return api_fail(MLT_EINVAL, "bytes_out must be non-NULL");
  const int rc = check_scan(args);
  if (rc != MLT_OK) return rc;
  *bytes_out = scan_grad_workspace(*args, api_sm_count());
  return MLT_OK;
}

int mlt_scan_grad(void* stream, const mlt_scan_args* args, const mlt_scan_grads* grads, void* workspace,
                  size_t workspace_bytes) {
  int rc = check_scan(args);
  if (rc != MLT_OK) return rc;
  if (grads == nullptr) return api_fail(MLT_EINVAL, "grads must be non-NULL");
  rc = check_scan_inputs(args);
  if (rc != MLT_OK) return rc;
  if (args->length > 0 && args->batch > 0 && grads->gy == nullptr) return api_fail(MLT_EINVAL, "gy must be non-NULL");
  if (grads->gy_step < 0 || grads->gy_batch < 0) return api_fail(MLT_EINVAL, "gy: strides must not be negative");
  if ((args->length + 31) / 32 * args->groups * ((args->dim / args->groups + 63) / 64) > kMaxCount)
    return api_fail(MLT_EINVAL, "length x dim is too large for one gradient call");
  if (!aligned_to(grads->gy, dtype_size(args->dtype))) return api_fail(MLT_EINVAL, "gy is not aligned to its elements");
  if ((grads->z != nullptr && args->z == nullptr) || (grads->skip != nullptr && args->skip == nullptr) ||
      (grads->dt_bias != nullptr && args->dt_bias == nullptr) || (grads->conv_b != nullptr && args->conv_b == nullptr) ||
      (grads->conv_w != nullptr && args->taps == 0) || (grads->conv_state != nullptr && args->taps < 2))
    return api_fail(MLT_EINVAL, "a gradient was asked for of an input that is not there");
  const int sms = api_sm_count();
  rc = check_ws(workspace, workspace_bytes, scan_grad_workspace(*args, sms));
  if (rc != MLT_OK) return rc;
  long long launches = 0;
  const cudaError_t e = launch_scan_grad(*args, *grads, workspace, sms, &launches, static_cast<cudaStream_t>(stream));
  return launched(e, launches, "scan gradient launch");
}

}  // extern "C"
