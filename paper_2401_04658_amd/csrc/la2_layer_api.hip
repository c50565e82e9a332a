// Host side of the C ABI's operators around the recurrence: argument validation and dispatch.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "../../include/la2.h"
#include "la2_layer.h"
#include "la2_linear.h"

namespace {

static_assert((int)LA2_ACT_RELU == (int)la2::kActRelu && (int)LA2_ACT_GELU == (int)la2::kActGelu && (int)LA2_ACT_SILU == (int)la2::kActSilu, "act");

bool known_dtype(int dtype) { return dtype == LA2_F32 || dtype == LA2_BF16 || dtype == LA2_F16; }
bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
template <typename... P>
bool aligned16(const P*... p) {
  return (aligned(p, 16) && ...);
}
template <typename... P>
bool any_null(const P*... p) {
  return ((p == nullptr) || ...);
}
constexpr int64_t kMostElements = (int64_t)1 << 40;

la2_status workspace_fits(size_t need, const void* ws, size_t bytes) {
  if (need == 0) return LA2_OK;
  return ws == nullptr || bytes < need || !aligned(ws, 256) ? LA2_ERR_WORKSPACE : LA2_OK;
}
la2_status launched(hipError_t e) { return e == hipSuccess ? LA2_OK : LA2_ERR_LAUNCH; }

la2_status check_norm(int64_t rows, int32_t width, int32_t dtype, int64_t stride) {
  if (!known_dtype(dtype)) return LA2_ERR_DTYPE;
  if (rows < 0 || width < 0 || width > 1 << 28 || (width > 0 && rows > kMostElements / width)) return LA2_ERR_SHAPE;
  return stride < width ? LA2_ERR_STRIDE_ALIGN : LA2_OK;
}
size_t norm_workspace(int64_t rows, int32_t width, int32_t dtype) {
  return (size_t)la2::layer_norm_bwd_partials(dtype, rows, width, la2::device_units()) * 2 * width * sizeof(float);
}

la2::LinearParams linear_params(const la2_linear_desc* d) {
  la2::LinearParams p{};
  p.rows = d->rows;
  p.in = d->in_features;
  p.out = d->out_features;
  p.dtype = d->dtype;
  p.act = d->act;
  p.stride_x = d->stride_x;
  p.stride_w = d->stride_w;
  p.stride_y = d->stride_y;
  return p;
}
la2_status check_linear(const la2_linear_desc* d) {
  if (d == nullptr) return LA2_ERR_NULL;
  if (!known_dtype(d->dtype)) return LA2_ERR_DTYPE;
  if (d->rows < 0 || d->in_features < 0 || d->out_features < 0) return LA2_ERR_SHAPE;
  if (d->act < LA2_ACT_NONE || d->act > LA2_ACT_SILU) return LA2_ERR_VALUE;
  if (d->stride_x < d->in_features || d->stride_w < d->in_features || d->stride_y < d->out_features) return LA2_ERR_STRIDE_ALIGN;
  // a tile's rows are addressed with 31-bit byte offsets, 256 rows at most
  const int64_t most = (((int64_t)1 << 23) - 1) / (d->dtype == LA2_F32 ? 4 : 2);
  if (d->stride_x > most || d->stride_w > most || d->stride_y > most) return LA2_ERR_SHAPE;
  if (d->rows > INT32_MAX || d->rows > kMostElements / (1 + (d->in_features > d->out_features ? d->in_features : d->out_features))) return LA2_ERR_SHAPE;
  return la2::linear_fits(linear_params(d)) ? LA2_OK : LA2_ERR_SHAPE;
}

la2_status check_beams(int32_t batch, int32_t beams) {
  if (batch < 0 || beams < 1 || beams > la2::kMaxBeams) return LA2_ERR_SHAPE;
  return LA2_OK;
}
la2_status check_select(int32_t batch, int32_t beams, int32_t vocab, int32_t dtype) {
  if (!known_dtype(dtype)) return LA2_ERR_DTYPE;
  if (check_beams(batch, beams) != LA2_OK || vocab < 1 || vocab > la2::kMaxVocab || (int64_t)batch * beams > 65535) return LA2_ERR_SHAPE;
  return LA2_OK;
}
size_t select_sums(int64_t rows, int chunks) { return ((size_t)rows * chunks * sizeof(float2) + 255) / 256 * 256; }

}  // namespace

extern "C" {

size_t la2_layer_norm_workspace_bytes(int64_t rows, int32_t width, int32_t dtype) {
  return check_norm(rows, width, dtype, width) == LA2_OK ? norm_workspace(rows, width, dtype) : 0;
}

la2_status la2_layer_norm_fwd(int64_t rows, int32_t width, int32_t dtype, int64_t stride, const void* x, const float* weight,
                              const float* bias, float eps, void* y, float* mean, float* rstd, void* hip_stream) {
  const la2_status st = check_norm(rows, width, dtype, stride);
  if (st != LA2_OK) return st;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return LA2_ERR_VALUE;
  if (rows == 0 || width == 0) return LA2_OK;
  if (any_null(x, y, mean, rstd)) return LA2_ERR_NULL;
  if (!aligned16(x, weight, bias, y, mean, rstd)) return LA2_ERR_STRIDE_ALIGN;
  la2::LayerNormParams p{};
  p.rows = rows;
  p.width = width;
  p.stride = stride;
  p.x = x;
  p.y = y;
  p.weight = weight;
  p.bias = bias;
  p.eps = eps;
  p.mean = mean;
  p.rstd = rstd;
  return launched(la2::launch_layer_norm_fwd(dtype, p, la2::device_units(), reinterpret_cast<hipStream_t>(hip_stream)));
}

la2_status la2_layer_norm_bwd(int64_t rows, int32_t width, int32_t dtype, int64_t stride, const void* x, const void* dy,
                              const float* weight, const float* mean, const float* rstd, void* dx, float* d_weight, float* d_bias,
                              void* workspace, size_t workspace_bytes, void* hip_stream) {
  la2_status st = check_norm(rows, width, dtype, stride);
  if (st != LA2_OK) return st;
  if (width == 0) return LA2_OK;
  const bool sums = d_weight != nullptr || d_bias != nullptr;
  if (rows == 0 && !sums) return LA2_OK;
  if (rows > 0 && any_null(x, dy, mean, rstd, dx)) return LA2_ERR_NULL;
  if (!aligned16(x, dy, weight, dx, mean, rstd, d_weight, d_bias)) return LA2_ERR_STRIDE_ALIGN;
  st = workspace_fits(sums ? norm_workspace(rows, width, dtype) : 0, workspace, workspace_bytes);
  if (st != LA2_OK) return st;
  la2::LayerNormParams p{};
  p.rows = rows;
  p.width = width;
  p.stride = stride;
  p.x = x;
  p.dy = dy;
  p.y = dx;
  p.weight = weight;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.d_weight = d_weight;
  p.d_bias = d_bias;
  p.partial = static_cast<float*>(workspace);
  return launched(la2::launch_layer_norm_bwd(dtype, p, la2::device_units(), reinterpret_cast<hipStream_t>(hip_stream)));
}

size_t la2_linear_workspace_bytes(const la2_linear_desc* desc, int32_t op) {
  if (check_linear(desc) != LA2_OK) return 0;
  la2::LinearParams p = linear_params(desc);
  if (op == LA2_OP_FWD) return la2::linear_fwd_workspace(p, la2::device_units());
  if (op != LA2_OP_BWD) return 0;
  // Each choice of outputs has a plan of its own, and one product alone may be cut into more pieces than beside the other: the largest
  // need (d_bias only adds to it).
  static float wanted;   // only told from nullptr
  const int units = la2::device_units();
  p.d_bias = &wanted;
  size_t most = 0;
  for (int products = 1; products <= 3; products++) {
    p.dx = products & 1 ? &wanted : nullptr;
    p.dw = products & 2 ? &wanted : nullptr;
    const size_t need = la2::linear_bwd_workspace(p, units);
    most = need > most ? need : most;
  }
  return most;
}

la2_status la2_linear_fwd(const la2_linear_desc* desc, const void* x, const void* w, const float* bias, const void* residual, void* y,
                          void* pre, void* workspace, size_t workspace_bytes, void* hip_stream) {
  la2_status st = check_linear(desc);
  if (st != LA2_OK) return st;
  if (desc->rows == 0 || desc->out_features == 0) return LA2_OK;
  if (y == nullptr || (desc->in_features > 0 && any_null(x, w))) return LA2_ERR_NULL;
  if (!aligned16(x, w, bias, residual, y, pre)) return LA2_ERR_STRIDE_ALIGN;
  la2::LinearParams p = linear_params(desc);
  p.x = x;
  p.w = w;
  p.bias = bias;
  p.residual = residual;
  p.y = y;
  p.pre = pre;
  const int units = la2::device_units();
  st = workspace_fits(la2::linear_fwd_workspace(p, units), workspace, workspace_bytes);
  if (st != LA2_OK) return st;
  return launched(la2::launch_linear_fwd(p, workspace, units, reinterpret_cast<hipStream_t>(hip_stream)));
}

la2_status la2_linear_bwd(const la2_linear_desc* desc, const void* x, const void* w, const void* pre, const void* dy, void* dx, void* dw,
                          float* d_bias, void* workspace, size_t workspace_bytes, void* hip_stream) {
  la2_status st = check_linear(desc);
  if (st != LA2_OK) return st;
  if (desc->rows == 0 || desc->in_features == 0) dx = nullptr;   // nothing to write
  if (desc->out_features == 0 || desc->in_features == 0) dw = nullptr;
  if (desc->out_features == 0) d_bias = nullptr;
  if (any_null(dx) && any_null(dw) && any_null(d_bias)) return LA2_OK;
  if (desc->rows > 0 && desc->out_features > 0) {
    if (dy == nullptr || (desc->act != LA2_ACT_NONE && pre == nullptr) || (dx != nullptr && w == nullptr) || (dw != nullptr && x == nullptr))
      return LA2_ERR_NULL;
  }
  if (!aligned16(x, w, pre, dy, dx, dw, d_bias)) return LA2_ERR_STRIDE_ALIGN;
  la2::LinearParams p = linear_params(desc);
  p.x = x;
  p.w = w;
  p.pre = const_cast<void*>(pre);
  p.dy = dy;
  p.dx = dx;
  p.dw = dw;
  p.d_bias = d_bias;
  const int units = la2::device_units();
  st = workspace_fits(la2::linear_bwd_workspace(p, units), workspace, workspace_bytes);
  if (st != LA2_OK) return st;
  return launched(la2::launch_linear_bwd(p, workspace, units, reinterpret_cast<hipStream_t>(hip_stream)));
}

size_t la2_beam_select_workspace_bytes(int32_t batch, int32_t beams, int32_t vocab, int32_t dtype) {
  if (check_select(batch, beams, vocab, dtype) != LA2_OK) return 0;
  const int64_t rows = (int64_t)batch * beams;
  const int chunks = la2::beam_select_chunks(rows, beams, vocab, la2::device_units());
  return select_sums(rows, chunks) + (size_t)rows * chunks * beams * sizeof(uint64_t);
}

la2_status la2_beam_select(int32_t batch, int32_t beams, int32_t vocab, int32_t dtype, int64_t stride_row, const void* logits,
                           const float* scores, const uint8_t* finished, int32_t eos, float* out_scores, int32_t* parent, int32_t* token,
                           uint8_t* out_finished, void* workspace, size_t workspace_bytes, void* hip_stream) {
  la2_status st = check_select(batch, beams, vocab, dtype);
  if (st != LA2_OK) return st;
  if (eos < -1 || eos >= vocab || (eos == -1 && finished != nullptr)) return LA2_ERR_VALUE;
  if (stride_row < vocab) return LA2_ERR_STRIDE_ALIGN;
  if (batch == 0) return LA2_OK;
  if (any_null(logits, scores, out_scores, parent, token, out_finished)) return LA2_ERR_NULL;
  if (!aligned16(logits, scores, finished, out_scores, parent, token, out_finished)) return LA2_ERR_STRIDE_ALIGN;
  st = workspace_fits(la2_beam_select_workspace_bytes(batch, beams, vocab, dtype), workspace, workspace_bytes);
  if (st != LA2_OK) return st;
  la2::BeamSelectParams p{};
  p.batch = batch;
  p.beams = beams;
  p.vocab = vocab;
  p.stride = stride_row;
  p.logits = logits;
  p.scores = scores;
  p.finished = finished;
  p.eos = eos;
  const int units = la2::device_units();
  p.sums = static_cast<float2*>(workspace);
  p.keys = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + select_sums((int64_t)batch * beams, la2::beam_select_chunks((int64_t)batch * beams, beams, vocab, units)));
  p.out_scores = out_scores;
  p.parent = parent;
  p.token = token;
  p.out_finished = out_finished;
  return launched(la2::launch_beam_select(dtype, p, units, reinterpret_cast<hipStream_t>(hip_stream)));
}

la2_status la2_beam_reorder(int32_t nstates, void* const* states, int32_t batch, int32_t beams, int64_t row_bytes, const int32_t* parent,
                            void* hip_stream) {
  if (nstates < 0 || check_beams(batch, beams) != LA2_OK || batch > 65535 || row_bytes < 0 || row_bytes > la2::kMostReorderBytes) return LA2_ERR_SHAPE;
  if (row_bytes % 16 != 0) return LA2_ERR_STRIDE_ALIGN;
  if (nstates == 0 || batch == 0 || row_bytes == 0) return LA2_OK;
  if (any_null(states, parent)) return LA2_ERR_NULL;
  if (!aligned16(parent)) return LA2_ERR_STRIDE_ALIGN;
  for (int32_t i = 0; i < nstates; i++) {
    if (states[i] == nullptr) return LA2_ERR_NULL;
    if (!aligned16(states[i])) return LA2_ERR_STRIDE_ALIGN;
  }
  la2::BeamReorderParams p{};
  p.batch = batch;
  p.beams = beams;
  p.row_bytes = row_bytes;
  p.parent = parent;
  for (int32_t done = 0; done < nstates; done += la2::kMaxStatesPerLaunch) {
    const int32_t n = nstates - done < la2::kMaxStatesPerLaunch ? nstates - done : la2::kMaxStatesPerLaunch;
    for (int32_t i = 0; i < n; i++) p.states[i] = states[done + i];
    const la2_status st = launched(la2::launch_beam_reorder(p, n, reinterpret_cast<hipStream_t>(hip_stream)));
    if (st != LA2_OK) return st;
  }
  return LA2_OK;
}

}  // extern "C"
