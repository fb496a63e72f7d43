// C entry points of the sequence-model operators: argument checks, then the
// launches of sample.cu, embed.cu, scan.cu, scan_grad.cu, norm.cu, norm_grad.cu, adamw.cu and
// beam.cu.  Nothing here allocates device memory, but that the first draw, lookup or reordering on a device makes the library's own state
// (the error word is part of it) where no other call has.
#include <algorithm>
#include <cmath>
#include <new>
#include <utility>
#include <vector>

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

int check_norm(const mlt_norm_args* a) {
  if (a == nullptr) return api_fail(MLT_EINVAL, "args must be non-NULL");
  if (!dtype_ok(a->dtype) || !dtype_ok(a->y_dtype) || !dtype_ok(a->w_dtype))
    return api_fail(MLT_EINVAL, "unknown element type");
  if (a->y_dtype != a->dtype && a->dtype != MLT_F32)
    return api_fail(MLT_EINVAL, "y must be of x's type, or a narrower one where x is fp32");
  if (a->rows < 0 || a->rows > kMaxCount) return api_fail(MLT_EINVAL, "rows must lie in [0, 2^31-1]");
  if (a->dim < 1 || a->dim > kMaxDim) return api_fail(MLT_EINVAL, "dim must lie in [1, %d], got %d", kMaxDim, a->dim);
  if (a->x_stride < 0 || a->residual_stride < 0) return api_fail(MLT_EINVAL, "strides must not be negative");
  if (a->rows > 0 && a->x == nullptr) return api_fail(MLT_EINVAL, "x must be non-NULL");
  if (!aligned_to(a->x, dtype_size(a->dtype)) || !aligned_to(a->weight, dtype_size(a->w_dtype)) ||
      !aligned_to(a->bias, dtype_size(a->w_dtype)) || !aligned_to(a->stats, 8))
    return api_fail(MLT_EINVAL, "buffers must be aligned to their elements, stats to 8 bytes");
  return MLT_OK;
}

// Whether an output of rows that begins where an input does is that input, of its type and stride.
bool is_itself(const void* out, int out_dtype, int64_t out_stride, const void* in, int in_dtype, int64_t in_stride,
               int64_t rows) {
  return out == nullptr || out != in || (out_dtype == in_dtype && (rows <= 1 || out_stride == in_stride));
}

int check_tensors(const mlt_adamw_tensor* tensors, int count) {
  if (count < 0 || count > (1 << 20)) return api_fail(MLT_EINVAL, "count must lie in [0, 2^20], got %d", count);
  if (count > 0 && tensors == nullptr) return api_fail(MLT_EINVAL, "tensors must be non-NULL");
  int64_t all = 0;
  for (int i = 0; i < count; ++i) {
    const mlt_adamw_tensor& t = tensors[i];
    if (!dtype_ok(t.dtype) || !dtype_ok(t.grad_dtype) || !dtype_ok(t.copy_dtype))
      return api_fail(MLT_EINVAL, "tensor %d: unknown element type", i);
    if (t.n < 0 || t.n > (1LL << 40)) return api_fail(MLT_EINVAL, "tensor %d: n must lie in [0, 2^40]", i);
    all += (t.n + 255) / 256;
    if (all > (1LL << 40)) return api_fail(MLT_EINVAL, "the tensors have more than 2^40 blocks");
  }
  return MLT_OK;
}

// Whether two of the ranges [first, second) of addresses overlap; orders them.
bool overlap(std::vector<std::pair<uintptr_t, uintptr_t>>& ranges) {
  std::sort(ranges.begin(), ranges.end());
  for (size_t i = 1; i < ranges.size(); ++i)
    if (ranges[i].first < ranges[i - 1].second) return true;
  return false;
}

void add_range(std::vector<std::pair<uintptr_t, uintptr_t>>& ranges, const void* p, int64_t bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  if (p != nullptr && bytes > 0) ranges.emplace_back(at, at + static_cast<uintptr_t>(bytes));
}

// Whether two states of so many rows have no byte in common: one behind the other, or columns of one buffer.
bool apart(const mlt_beam_state& s, const mlt_beam_state& t, int64_t rows) {
  const mlt_beam_state &a = s.data < t.data ? s : t, &b = s.data < t.data ? t : s;
  const uintptr_t far = reinterpret_cast<uintptr_t>(b.data) - reinterpret_cast<uintptr_t>(a.data);
  if (far >= static_cast<uintptr_t>((rows - 1) * a.row_stride + a.row_bytes)) return true;
  if (rows == 1 || a.row_stride != b.row_stride) return false;
  const int64_t column = static_cast<int64_t>(far % static_cast<uintptr_t>(a.row_stride));
  return column >= a.row_bytes && column + b.row_bytes <= a.row_stride;
}

int check_beam(const mlt_beam_args* a) {
  if (a == nullptr) return api_fail(MLT_EINVAL, "args must be non-NULL");
  if (!dtype_ok(a->dtype)) return api_fail(MLT_EINVAL, "unknown element type %d", a->dtype);
  if (a->batch < 0 || a->batch > 65535) return api_fail(MLT_EINVAL, "batch must lie in [0, 65535], got %d", a->batch);
  if (a->beams < 1 || a->beams > kBeamMostBeams)
    return api_fail(MLT_EINVAL, "beams must lie in [1, %d], got %d", kBeamMostBeams, a->beams);
  if (a->n < 1 || a->n > (1 << 22)) return api_fail(MLT_EINVAL, "n must lie in [1, 2^22], got %d", a->n);
  if (a->m < 1 || a->m > 1024) return api_fail(MLT_EINVAL, "m must lie in [1, 1024], got %d", a->m);
  if (static_cast<int64_t>(a->beams) * std::min(a->m, a->n) > 8192)
    return api_fail(MLT_EINVAL, "beams x min(m, n) must be at most 8192, got %d x %d", a->beams, std::min(a->m, a->n));
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

int mlt_layer_norm(void* stream, const mlt_norm_args* args) {
  int rc = check_norm(args);
  if (rc != MLT_OK) return rc;
  if (!(args->eps >= 0.0f && std::isfinite(args->eps))) return api_fail(MLT_EINVAL, "eps must be finite and not negative");
  if (args->rows == 0) return MLT_OK;
  if (args->y == nullptr) return api_fail(MLT_EINVAL, "y must be non-NULL");
  if (!stride_ok(args->y_stride, args->dim, args->rows) ||
      (args->total != nullptr && !stride_ok(args->total_stride, args->dim, args->rows)))
    return api_fail(MLT_EINVAL, "rows must be at least dim elements apart");
  if (args->total != nullptr && args->total == args->y) return api_fail(MLT_EINVAL, "y and total must differ");
  struct {
    const void* p;
    int64_t stride;
  } in[] = {{args->x, args->x_stride}, {args->residual, args->residual_stride}};
  for (const auto& t : in)
    if (!is_itself(args->y, args->y_dtype, args->y_stride, t.p, args->dtype, t.stride, args->rows) ||
        !is_itself(args->total, args->dtype, args->total_stride, t.p, args->dtype, t.stride, args->rows))
      return api_fail(MLT_EINVAL, "y and total over an input must be of its type and stride");
  if (!aligned_to(args->residual, dtype_size(args->dtype)) || !aligned_to(args->total, dtype_size(args->dtype)) ||
      !aligned_to(args->y, dtype_size(args->y_dtype)))
    return api_fail(MLT_EINVAL, "buffers must be aligned to their elements");
  mlt_norm_args a = *args;
  if (a.rows == 1) a.x_stride = a.residual_stride = a.y_stride = a.total_stride = 0;
  long long launches = 0;
  const cudaError_t e = launch_norm(a, api_sm_count(), &launches, static_cast<cudaStream_t>(stream));
  return launched(e, launches, "layer norm launch");
}

int mlt_layer_norm_grad_workspace(int64_t rows, int dim, size_t* bytes_out) {
  if (bytes_out == nullptr) return api_fail(MLT_EINVAL, "bytes_out must be non-NULL");
  mlt_norm_args a{};
  a.rows = rows;
  a.dim = dim;
  a.x = bytes_out;
  const int rc = check_norm(&a);
  if (rc != MLT_OK) return rc;
  *bytes_out = norm_grad_workspace(rows, dim, api_sm_count());
  return MLT_OK;
}

int mlt_layer_norm_grad(void* stream, const mlt_norm_args* args, const mlt_norm_grads* grads, void* workspace,
                        size_t workspace_bytes) {
  int rc = check_norm(args);
  if (rc != MLT_OK) return rc;
  if (grads == nullptr) return api_fail(MLT_EINVAL, "grads must be non-NULL");
  if (args->residual != nullptr) return api_fail(MLT_EINVAL, "the gradient takes the sum as x and no residual");
  if (args->rows > 0 && (grads->gy == nullptr || args->stats == nullptr))
    return api_fail(MLT_EINVAL, "gy and stats must be non-NULL");
  if (grads->gy_stride < 0 || grads->g_total_stride < 0) return api_fail(MLT_EINVAL, "strides must not be negative");
  if (grads->gx != nullptr && !stride_ok(grads->gx_stride, args->dim, args->rows))
    return api_fail(MLT_EINVAL, "rows must be at least dim elements apart");
  if (!aligned_to(grads->gy, dtype_size(args->y_dtype)) || !aligned_to(grads->g_total, dtype_size(args->dtype)) ||
      !aligned_to(grads->gx, dtype_size(args->dtype)) || !aligned_to(grads->gweight, dtype_size(args->w_dtype)) ||
      !aligned_to(grads->gbias, dtype_size(args->w_dtype)))
    return api_fail(MLT_EINVAL, "buffers must be aligned to their elements");
  if (!is_itself(grads->gx, args->dtype, grads->gx_stride, grads->gy, args->y_dtype, grads->gy_stride, args->rows) ||
      !is_itself(grads->gx, args->dtype, grads->gx_stride, grads->g_total, args->dtype, grads->g_total_stride, args->rows) ||
      !is_itself(grads->gx, args->dtype, grads->gx_stride, args->x, args->dtype, args->x_stride, args->rows))
    return api_fail(MLT_EINVAL, "gx over an input must be of its type and stride");
  const bool sums = grads->gweight != nullptr || grads->gbias != nullptr;
  const int sms = api_sm_count();
  rc = check_ws(workspace, workspace_bytes, sums ? norm_grad_workspace(args->rows, args->dim, sms) : 0);
  if (rc != MLT_OK) return rc;
  if (!sums && (grads->gx == nullptr || args->rows == 0)) return MLT_OK;
  mlt_norm_args a = *args;
  mlt_norm_grads g = *grads;
  if (a.rows == 1) a.x_stride = g.gy_stride = g.g_total_stride = g.gx_stride = 0;
  long long launches = 0;
  const cudaError_t e = launch_norm_grad(a, g, workspace, sms, &launches, static_cast<cudaStream_t>(stream));
  return launched(e, launches, "layer norm gradient launch");
}

int mlt_adamw_blocks(const mlt_adamw_tensor* tensors, int count, int64_t* blocks_out) {
  if (blocks_out == nullptr) return api_fail(MLT_EINVAL, "blocks_out must be non-NULL");
  const int rc = check_tensors(tensors, count);
  if (rc != MLT_OK) return rc;
  *blocks_out = 0;
  for (int i = 0; i < count; ++i) *blocks_out += (tensors[i].n + 255) / 256;
  return MLT_OK;
}

int mlt_adamw(void* stream, const mlt_adamw_tensor* tensors, int count, const mlt_adamw_rule* rule, void* m, void* v,
              float* m_scale, float* v_scale) try {
  const int rc = check_tensors(tensors, count);
  if (rc != MLT_OK) return rc;
  if (rule == nullptr) return api_fail(MLT_EINVAL, "rule must be non-NULL");
  if (!(rule->beta1 >= 0 && rule->beta1 < 1 && rule->beta2 >= 0 && rule->beta2 < 1))
    return api_fail(MLT_EINVAL, "beta1 and beta2 must lie in [0, 1)");
  if (!(rule->eps >= 0 && std::isfinite(rule->eps))) return api_fail(MLT_EINVAL, "eps must be finite and not negative");
  if (rule->bits != 8 && rule->bits != 32) return api_fail(MLT_EINVAL, "bits must be 8 or 32, got %d", rule->bits);
  if (rule->step_device == nullptr && rule->step < 1) return api_fail(MLT_EINVAL, "step must be at least 1");
  if (!aligned_to(rule->step_device, 8) || !aligned_to(rule->lr, 4) || !aligned_to(rule->grad_scale, 4))
    return api_fail(MLT_EINVAL, "values on the device must be aligned to their types");
  std::vector<std::pair<uintptr_t, uintptr_t>> ranges;
  ranges.reserve(2 * static_cast<size_t>(count) + 4);
  int64_t blocks = 0;
  bool any = false;
  for (int i = 0; i < count; ++i) {
    const mlt_adamw_tensor& t = tensors[i];
    blocks += (t.n + 255) / 256;
    if (t.n == 0 || t.grad == nullptr) continue;
    any = true;
    if (t.param == nullptr) return api_fail(MLT_EINVAL, "tensor %d: param must be non-NULL", i);
    if (!std::isfinite(t.lr) || !std::isfinite(t.weight_decay))
      return api_fail(MLT_EINVAL, "tensor %d: lr and weight_decay must be finite", i);
    if (!aligned_to(t.param, dtype_size(t.dtype)) || !aligned_to(t.grad, dtype_size(t.grad_dtype)) ||
        !aligned_to(t.copy, dtype_size(t.copy_dtype)))
      return api_fail(MLT_EINVAL, "tensor %d: buffers must be aligned to their elements", i);
    add_range(ranges, t.param, t.n * static_cast<int64_t>(dtype_size(t.dtype)));
    add_range(ranges, t.copy, t.n * static_cast<int64_t>(dtype_size(t.copy_dtype)));
  }
  if (!any) return MLT_OK;
  if (m == nullptr || v == nullptr || !aligned_to(m, 16) || !aligned_to(v, 16))
    return api_fail(MLT_EINVAL, "m and v must be non-NULL, aligned to 16 bytes");
  const int64_t each = 256 * (rule->bits / 8);
  add_range(ranges, m, blocks * each);
  add_range(ranges, v, blocks * each);
  if (rule->bits == 8) {
    if (m_scale == nullptr || v_scale == nullptr || !aligned_to(m_scale, 4) || !aligned_to(v_scale, 4))
      return api_fail(MLT_EINVAL, "moments of 8 bits need m_scale and v_scale");
    add_range(ranges, m_scale, blocks * 4);
    add_range(ranges, v_scale, blocks * 4);
  }
  if (overlap(ranges)) return api_fail(MLT_EINVAL, "parameters, copies and moments must not overlap");
  long long launches = 0;
  const cudaError_t e = launch_adamw(tensors, count, *rule, m, v, m_scale, v_scale, api_sm_count(), &launches,
                                     static_cast<cudaStream_t>(stream));
  return launched(e, launches, "AdamW launch");
} catch (const std::bad_alloc&) {
  return api_fail(MLT_ENOMEM, "out of host memory for %d tensors", count);
}

int mlt_beam_step_workspace(const mlt_beam_args* args, size_t* bytes_out) {
  if (bytes_out == nullptr) return api_fail(MLT_EINVAL, "bytes_out must be non-NULL");
  const int rc = check_beam(args);
  if (rc != MLT_OK) return rc;
  *bytes_out = beam_workspace(*args, api_sm_count());
  return MLT_OK;
}

int mlt_beam_step(void* stream, const mlt_beam_args* args, void* workspace, size_t workspace_bytes) {
  int rc = check_beam(args);
  if (rc != MLT_OK) return rc;
  if (args->batch == 0) return MLT_OK;
  if (args->scores == nullptr || args->logp == nullptr || args->out_parent == nullptr || args->out_token == nullptr ||
      args->out_logp == nullptr || args->out_done == nullptr)
    return api_fail(MLT_EINVAL, "device buffers must be non-NULL");
  if (args->batch_stride < 0 || args->beam_stride < 0) return api_fail(MLT_EINVAL, "strides must not be negative");
  if (args->eos >= args->n) return api_fail(MLT_EINVAL, "eos must be below n");
  if (args->eos < 0 && args->done != nullptr) return api_fail(MLT_EINVAL, "finished beams need an eos");
  if (!aligned_to(args->scores, dtype_size(args->dtype)) || !aligned_to(args->logp, 4) || !aligned_to(args->out_parent, 8) ||
      !aligned_to(args->out_token, 8) || !aligned_to(args->out_logp, 4))
    return api_fail(MLT_EINVAL, "buffers must be aligned to their elements");
  const int sms = api_sm_count();
  rc = check_ws(workspace, workspace_bytes, beam_workspace(*args, sms));
  if (rc != MLT_OK) return rc;
  mlt_beam_args a = *args;
  if (a.eos < 0) a.eos = -1;
  long long launches = 0;
  const cudaError_t e = launch_beam(a, workspace, sms, &launches, static_cast<cudaStream_t>(stream));
  return launched(e, launches, "beam step launch");
}

int mlt_beam_reorder(void* stream, const int64_t* parent, int batch, int beams, const mlt_beam_state* tensors,
                     int count) {
  if (batch < 0 || batch > 65535) return api_fail(MLT_EINVAL, "batch must lie in [0, 65535], got %d", batch);
  if (beams < 1 || beams > kBeamMostBeams)
    return api_fail(MLT_EINVAL, "beams must lie in [1, %d], got %d", kBeamMostBeams, beams);
  if (count < 0 || count > kBeamMostStates)
    return api_fail(MLT_EINVAL, "count must lie in [0, %d], got %d", kBeamMostStates, count);
  if (count > 0 && tensors == nullptr) return api_fail(MLT_EINVAL, "tensors must be non-NULL");
  const int64_t rows = static_cast<int64_t>(batch) * beams;
  int64_t moved = 0;
  const mlt_beam_state list{const_cast<int64_t*>(parent), 8, 8};
  for (int i = 0; i < count; ++i) {
    const mlt_beam_state& t = tensors[i];
    if (t.row_bytes < 0 || t.row_bytes > (1LL << 40) || t.row_stride > (1LL << 40))
      return api_fail(MLT_EINVAL, "tensor %d: row_bytes must lie in [0, 2^40], row_stride below it", i);
    if (rows == 0 || t.row_bytes == 0) continue;
    if (t.data == nullptr) return api_fail(MLT_EINVAL, "tensor %d: data must be non-NULL", i);
    if (!stride_ok(t.row_stride, t.row_bytes, rows))
      return api_fail(MLT_EINVAL, "tensor %d: rows must be at least row_bytes apart", i);
    if (rows > 1 && t.row_stride > (1LL << 60) / rows) return api_fail(MLT_EINVAL, "tensor %d: longer than 2^60 bytes", i);
    ++moved;
  }
  if (moved == 0) return MLT_OK;
  if (parent == nullptr || !aligned_to(parent, 8)) return api_fail(MLT_EINVAL, "parent must be non-NULL, aligned to 8 bytes");
  for (int i = 0; i < count; ++i) {
    if (tensors[i].row_bytes == 0) continue;
    bool ok = apart(tensors[i], list, rows);
    for (int j = 0; j < i; ++j) ok = ok && (tensors[j].row_bytes == 0 || apart(tensors[i], tensors[j], rows));
    if (!ok) return api_fail(MLT_EINVAL, "tensors must not overlap each other or parent");
  }
  int rc = MLT_OK;
  unsigned* err = api_error_word(&rc);
  if (err == nullptr) return rc;
  long long launches = 0;
  const cudaError_t e =
      launch_reorder(parent, batch, beams, tensors, count, err, &launches, static_cast<cudaStream_t>(stream));
  return launched(e, launches, "beam reorder launch");
}

}  // extern "C"
