// C ABI of the head operators (include/npd.h): argument checks, the workspace's layout, and the launches of a call.
// Every check runs before the first HIP call.
#include <float.h>
#include <math.h>

#include "../../include/npd.h"
#include "npd_check.hpp"
#include "npd_head.hpp"

namespace {

using namespace npd;

constexpr uint32_t kGradFlags = NPD_HEAD_GRAD_HIDDEN | NPD_HEAD_GRAD_WEIGHT | NPD_HEAD_GRAD_BIAS;
constexpr int32_t kWhole = 0x7fffff00;  // a chunk that takes every row

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

float exponent_scale(const npd_head_desc& d) { return (float)(1.4426950408889634 / (double)d.tau); }
float kd_weight(const npd_head_desc& d) { return (float)((double)d.grad_scale / (double)d.tau); }

npd_status check_head(const npd_head_desc* d, int op) {
  if (!d) return NPD_ERR_NULL;
  if (op != NPD_HEAD_LOSS && op != NPD_HEAD_LOGITS && op != NPD_HEAD_LOGITS_BWD) return NPD_ERR_VALUE;
  if (d->n_tokens <= 0 || d->vocab <= 0 || d->width <= 0) return NPD_ERR_SHAPE;
  if (d->n_tokens > NPD_HEAD_MAX_TOKENS || d->vocab > NPD_HEAD_MAX_VOCAB || d->width > NPD_HEAD_MAX_WIDTH)
    return NPD_ERR_UNSUPPORTED;
  const uint32_t known = op == NPD_HEAD_LOGITS ? (uint32_t)NPD_HEAD_UNALIGNED
                                               : kGradFlags | NPD_HEAD_ACCUMULATE | NPD_HEAD_UNALIGNED;
  if (d->flags & ~known) return NPD_ERR_VALUE;
  const bool grads = (d->flags & kGradFlags) != 0;
  if (op == NPD_HEAD_LOGITS_BWD && !grads) return NPD_ERR_VALUE;
  if ((d->flags & NPD_HEAD_ACCUMULATE) && !(d->flags & (NPD_HEAD_GRAD_WEIGHT | NPD_HEAD_GRAD_BIAS))) return NPD_ERR_VALUE;
  // strides: of what the call has
  const bool has_hidden = op != NPD_HEAD_LOGITS_BWD || (d->flags & NPD_HEAD_GRAD_WEIGHT);
  const bool has_weight = op != NPD_HEAD_LOGITS_BWD || (d->flags & NPD_HEAD_GRAD_HIDDEN);
  const int64_t strides[5][3] = {{has_hidden, d->hidden_stride, d->width},
                                 {has_weight, d->weight_stride, d->width},
                                 {op != NPD_HEAD_LOGITS && (d->flags & NPD_HEAD_GRAD_HIDDEN), d->grad_hidden_stride, d->width},
                                 {op != NPD_HEAD_LOGITS && (d->flags & NPD_HEAD_GRAD_WEIGHT), d->grad_weight_stride, d->width},
                                 {op != NPD_HEAD_LOSS, d->logits_stride, d->vocab}};
  for (const auto& s : strides)
    if (s[0] && s[1] < s[2]) return NPD_ERR_SHAPE;
  for (const auto& s : strides)
    if (s[0] && s[1] > NPD_HEAD_MAX_VOCAB) return NPD_ERR_UNSUPPORTED;  // offsets within a tile are 32-bit
  if (!(d->softcap >= 0.0f) || !isfinite(d->softcap) || (d->softcap > 0.0f && d->softcap < FLT_MIN)) return NPD_ERR_VALUE;
  if (op != NPD_HEAD_LOSS) return NPD_OK;
  if (d->topk < 0 || d->topk > d->vocab) return NPD_ERR_SHAPE;
  if (d->topk > kTopkMax) return NPD_ERR_UNSUPPORTED;
  if (!(d->tau > 0.0f) || !isfinite(d->tau)) return NPD_ERR_VALUE;
  if (!isfinite(d->grad_scale) || !isfinite(d->ce_grad_scale)) return NPD_ERR_VALUE;
  // what the kernels multiply by has to be a number: the base-2 scale of the logits, with the soft cap in it, and a row's weight
  const float c = exponent_scale(*d);
  if (!isfinite(c) || (d->softcap != 0.0f && (!isfinite(c * d->softcap) || c * d->softcap == 0.0f))) return NPD_ERR_VALUE;
  if (grads && d->topk > 0 && !isfinite(kd_weight(*d) + d->ce_grad_scale)) return NPD_ERR_VALUE;
  if (!grads && d->ce_grad_scale != 0.0f) return NPD_ERR_VALUE;
  if (grads && d->topk == 0 && d->ce_grad_scale == 0.0f) return NPD_ERR_VALUE;  // nothing to differentiate
  if (d->tau != 1.0f && d->ce_grad_scale != 0.0f) return NPD_ERR_UNSUPPORTED;
  // the gradient is kept as a multiple of p_S; the sum of the weights must not cancel
  if (grads && d->topk > 0 && ((d->grad_scale > 0.0f && d->ce_grad_scale < 0.0f) || (d->grad_scale < 0.0f && d->ce_grad_scale > 0.0f)))
    return NPD_ERR_UNSUPPORTED;
  return NPD_OK;
}

// Where everything of a call lies in its workspace, with rows worked on in chunks of `cap`.
struct Plan {
  int32_t cap = 0;        // of a HeadChunk
  int64_t chunk_rows = 0; // most rows of a chunk
  int64_t chunks = 1;
  int32_t K = 0;          // width, a multiple of eight
  int64_t e_stride = 0;
  int32_t parts = 0, part_columns = 0, splits = 1;
  bool tokens = false;    // head_tokens()
  bool few = false;       // up to kHeadFewRows
  bool pack_w = false, pack_h = false, pack_g = false;
  size_t rows = 0, count = 0, h = 0, hs = 0, x = 0, r0 = 0, part = 0, e = 0, scale = 0, w = 0, dw = 0, dh = 0, pieces = 0, db = 0;
  size_t bytes = 0;
};

Plan make_plan(const npd_head_desc& d, int op, int32_t cap) {
  Plan p;
  const bool gh = d.flags & NPD_HEAD_GRAD_HIDDEN, gw = d.flags & NPD_HEAD_GRAD_WEIGHT, gb = d.flags & NPD_HEAD_GRAD_BIAS;
  const int64_t T = d.n_tokens;
  p.K = (int32_t)up(d.width, 8);
  const bool odd = d.width % 8 != 0 || (d.flags & NPD_HEAD_UNALIGNED);
  p.few = op != NPD_HEAD_LOGITS_BWD && T <= kHeadFewRows;  // these read weights at any alignment
  p.pack_w = (odd || d.weight_stride % 8 != 0) && (gh || (op != NPD_HEAD_LOGITS_BWD && !p.few));
  p.pack_g = op == NPD_HEAD_LOGITS_BWD &&
             (d.vocab % 8 != 0 || d.logits_stride % 8 != 0 || (d.flags & NPD_HEAD_UNALIGNED) || d.softcap != 0.0f);
  p.pack_h = op == NPD_HEAD_LOSS ||
             (((op == NPD_HEAD_LOGITS && !p.few) || gw) && (odd || d.hidden_stride % 8 != 0 || p.pack_g));
  const bool chunked = op == NPD_HEAD_LOSS || p.pack_g;
  p.cap = chunked ? cap : kWhole;
  p.chunk_rows = chunked && T > cap ? cap : T;
  p.chunks = (T + p.chunk_rows - 1) / p.chunk_rows;
  // an odd number of 128-byte lines between rows: a tile reads 256 rows at one column, which would else come from few channels
  p.e_stride = up(d.vocab, 64);
  if (p.e_stride / 64 % 2 == 0) p.e_stride += 64;
  p.tokens = p.few && head_tokens(T, d.weight_stride);
  p.part_columns = p.few ? head_few_part(T, d.vocab, d.width, d.weight_stride) : head_small(p.chunk_rows, d.vocab) ? kHeadSmallPart : kHeadPart;
  // (parts of 32: as many as two for each of 64, so that rows of e are written as far)
  p.parts = p.part_columns == kHeadTokensPart ? (int32_t)(up(d.vocab, kHeadSmallPart) / kHeadTokensPart)
                                              : (d.vocab + p.part_columns - 1) / p.part_columns;
  if (gh) p.splits = head_hidden_splits(p.chunk_rows, d.vocab, d.width);
  auto take = [&p](size_t bytes) {
    const size_t at = p.bytes;
    p.bytes += (bytes + 255) / 256 * 256;
    return at;
  };
  const size_t C = (size_t)p.chunk_rows, V = (size_t)d.vocab, D = (size_t)d.width;
  if (p.pack_w) p.w = take(V * p.K * 2);
  if (p.pack_h) p.h = take(C * p.K * 2);
  if (op == NPD_HEAD_LOSS) {
    p.rows = take((size_t)T * 4);
    p.count = take(4);
    p.x = take(C * (1 + d.topk) * 4);
    p.r0 = take(C * 4);
    p.part = take(C * p.parts * sizeof(float2));
    if (gh || gw || gb) p.scale = take(C * 4);
    if (gw) p.hs = take(C * p.K * 2);
  }
  if (p.pack_g || (op == NPD_HEAD_LOSS && (gh || gw || gb))) p.e = take(C * p.e_stride * 2);
  if (gw && p.chunks > 1) p.dw = take(V * (size_t)up(D, 4) * 4);
  if (gh) p.dh = take(head_hidden_floats(p.chunk_rows, d.width, p.splits) * 4);
  if (gb) {
    p.pieces = take(kHeadBiasSplits * V * 4);
    p.db = take(V * 4);
  }
  return p;
}

constexpr int32_t kCaps[] = {8192, 4096, 2048, 1024};  // rows of a chunk: as many as the workspace takes

npd_status choose_plan(const npd_head_desc& d, int op, const void* workspace, size_t bytes, Plan* plan) {
  for (const int32_t cap : kCaps) {
    *plan = make_plan(d, op, cap);
    if (plan->bytes <= bytes) {
      if (plan->bytes > 0 && (!workspace || misaligned(workspace, 256))) return NPD_ERR_WORKSPACE;
      return NPD_OK;
    }
  }
  return NPD_ERR_WORKSPACE;
}

#define NPD_TRY(call)                              \
  do {                                             \
    if ((call) != hipSuccess) return NPD_ERR_HIP;  \
  } while (0)

// a packed copy of the weights, where they cannot be read as they are
npd_status pack_weight(const npd_head_desc& d, const Plan& p, const uint16_t* weight, char* ws, hipStream_t stream, HeadMatrix* w) {
  *w = HeadMatrix{weight, d.weight_stride, d.vocab, p.K};
  if (!p.pack_w) return NPD_OK;
  HeadPackArgs a{};
  a.chunk = HeadChunk{nullptr, d.vocab, kWhole, 0};
  a.src = weight;
  a.src_stride = d.weight_stride;
  a.cols = d.width;
  a.width = p.K;
  a.dst = reinterpret_cast<uint16_t*>(ws + p.w);
  a.dst_stride = p.K;
  NPD_TRY(launch_head_pack(a, d.vocab, stream));
  *w = HeadMatrix{a.dst, p.K, d.vocab, p.K};
  return NPD_OK;
}

// the gradients' products of one chunk
npd_status gradients(const npd_head_desc& d, const Plan& p, const HeadChunk& chunk, const HeadMatrix& g, const HeadMatrix& w,
                     const HeadMatrix& h, const float* scale, const int32_t* rows, void* grad_hidden, void* grad_weight,
                     void* grad_bias, char* ws, hipStream_t stream) {
  const int32_t accumulate = (d.flags & NPD_HEAD_ACCUMULATE) != 0;
  HeadHiddenArgs gh{};
  gh.chunk = chunk;
  gh.g = g;
  gh.w = w;
  gh.scale = scale;
  gh.rows = rows;
  gh.K = d.vocab;
  gh.N = d.width;
  gh.most_splits = p.splits;
  gh.partial = reinterpret_cast<float*>(ws + p.dh);
  gh.out = static_cast<uint16_t*>(grad_hidden);
  gh.out_stride = d.grad_hidden_stride;
  HeadWeightArgs gw{};
  gw.chunk = chunk;
  gw.g = g;
  gw.h = h;
  gw.M = d.vocab;
  gw.N = d.width;
  gw.partial = reinterpret_cast<float*>(ws + p.dw);
  gw.out = static_cast<uint16_t*>(grad_weight);
  gw.out_stride = d.grad_weight_stride;
  gw.accumulate = accumulate;
  if (grad_hidden && grad_weight && head_both_small(gh, gw, p.chunk_rows, p.chunks)) {
    NPD_TRY(launch_head_both(gh, gw, p.chunk_rows, stream));
  } else {
    if (grad_hidden) NPD_TRY(launch_head_hidden(gh, p.chunk_rows, stream));
    if (grad_weight) NPD_TRY(launch_head_weight(gw, p.chunks, stream));
  }
  if (grad_bias) {
    HeadBiasArgs a{};
    a.chunk = chunk;
    a.g = g;
    a.scale = scale;
    a.M = d.vocab;
    a.pieces = reinterpret_cast<float*>(ws + p.pieces);
    a.partial = reinterpret_cast<float*>(ws + p.db);
    a.out = static_cast<uint16_t*>(grad_bias);
    a.accumulate = accumulate;
    NPD_TRY(launch_head_bias(a, stream));
  }
  return NPD_OK;
}

// tensors that the matrix products read where they lie begin on 16 bytes, unless the flag says that they need not
bool unaligned(const npd_head_desc& d, const void* p) { return !(d.flags & NPD_HEAD_UNALIGNED) && !aligned16(p); }

// a gradient's pointer and its flag go together
npd_status check_grads(const npd_head_desc& d, const void* gh, const void* gw, const void* gb) {
  const void* p[3] = {gh, gw, gb};
  const uint32_t f[3] = {NPD_HEAD_GRAD_HIDDEN, NPD_HEAD_GRAD_WEIGHT, NPD_HEAD_GRAD_BIAS};
  for (int i = 0; i < 3; ++i) {
    if ((d.flags & f[i]) && !p[i]) return NPD_ERR_NULL;
    if (!(d.flags & f[i]) && p[i]) return NPD_ERR_VALUE;
    if (misaligned(p[i], 2)) return NPD_ERR_VALUE;
  }
  return NPD_OK;
}


}  // namespace

extern "C" {

size_t npd_head_workspace_bytes(const npd_head_desc* desc, int op) {
  if (check_head(desc, op) != NPD_OK) return 0;
  // (one chunk more needs sums of the weights' gradient between them: the shortest chunks are not always the least)
  size_t least = SIZE_MAX;
  for (const int32_t cap : kCaps) {
    const size_t bytes = make_plan(*desc, op, cap).bytes;
    if (bytes < least) least = bytes;
  }
  return least;
}

size_t npd_head_workspace_bytes_preferred(const npd_head_desc* desc, int op) {
  return check_head(desc, op) == NPD_OK ? make_plan(*desc, op, kCaps[0]).bytes : 0;
}

npd_status npd_head_loss_fwd_bwd(const npd_head_desc* desc, const void* hidden, const void* weight, const void* bias,
                                 const int32_t* labels, const int32_t* teacher_idx, const float* teacher_val,
                                 const uint8_t* loss_mask, void* grad_hidden, void* grad_weight, void* grad_bias,
                                 float* kd_tok, float* nll_tok, float* lse_tok, int32_t* dev_status, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  npd_status st = check_head(desc, NPD_HEAD_LOSS);
  if (st != NPD_OK) return st;
  const npd_head_desc& d = *desc;
  if (!hidden || !weight || !loss_mask) return NPD_ERR_NULL;
  if ((st = check_grads(d, grad_hidden, grad_weight, grad_bias)) != NPD_OK) return st;
  if (d.topk > 0 && (!teacher_idx || !teacher_val)) return NPD_ERR_NULL;
  if (d.topk == 0 && (teacher_idx || teacher_val || kd_tok)) return NPD_ERR_VALUE;
  if (!labels && (nll_tok || d.ce_grad_scale != 0.0f)) return NPD_ERR_NULL;
  if (d.tau != 1.0f && (nll_tok || lse_tok)) return NPD_ERR_UNSUPPORTED;
  if (misaligned(hidden, 2) || misaligned(weight, 2) || misaligned(bias, 2) || misaligned(labels, 4) ||
      misaligned(teacher_idx, 4) || misaligned(teacher_val, 4) || misaligned(kd_tok, 4) || misaligned(nll_tok, 4) ||
      misaligned(lse_tok, 4) || misaligned(dev_status, 4) || unaligned(d, hidden) || unaligned(d, weight))
    return NPD_ERR_VALUE;
  Plan p;
  if ((st = choose_plan(d, NPD_HEAD_LOSS, workspace, workspace_bytes, &p)) != NPD_OK) return st;
  const int64_t T = d.n_tokens;
  const int V = d.vocab, D = d.width;
  {
    const size_t kb = (size_t)T * d.topk * 4;
    const Range in[7] = {range_of(hidden, rows_bytes(T, d.hidden_stride, D, 2)), range_of(weight, rows_bytes(V, d.weight_stride, D, 2)),
                         opt_range(bias, (size_t)V * 2), opt_range(labels, (size_t)T * 4), opt_range(teacher_idx, kb),
                         opt_range(teacher_val, kb), range_of(loss_mask, (size_t)T)};
    const Range out[8] = {grad_hidden ? range_of(grad_hidden, rows_bytes(T, d.grad_hidden_stride, D, 2)) : Range{0, 0},
                          grad_weight ? range_of(grad_weight, rows_bytes(V, d.grad_weight_stride, D, 2)) : Range{0, 0},
                          opt_range(grad_bias, (size_t)V * 2), opt_range(kd_tok, (size_t)T * 4), opt_range(nll_tok, (size_t)T * 4),
                          opt_range(lse_tok, (size_t)T * 4), opt_range(dev_status, 4), opt_range(workspace, p.bytes)};
    if (any_alias(in, 7, out, 8)) return NPD_ERR_ALIAS;
  }

  const hipStream_t on = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  const bool grads = grad_hidden || grad_weight || grad_bias;
  HeadRowsArgs rows{};
  rows.T = T;
  rows.mask = loss_mask;
  rows.rows = reinterpret_cast<int32_t*>(ws + p.rows);
  rows.count = reinterpret_cast<int32_t*>(ws + p.count);
  rows.kd = kd_tok;
  rows.nll = nll_tok;
  rows.lse = lse_tok;
  rows.grad_hidden = static_cast<uint16_t*>(grad_hidden);
  rows.grad_stride = d.grad_hidden_stride;
  rows.D = D;

  HeadMatrix w;
  if ((st = pack_weight(d, p, static_cast<const uint16_t*>(weight), ws, on, &w)) != NPD_OK) return st;
  HeadLossArgs l{};
  l.src = static_cast<const uint16_t*>(hidden);
  l.src_stride = d.hidden_stride;
  l.weight = static_cast<const uint16_t*>(weight);
  l.weight_stride = d.weight_stride;
  l.D = D;
  uint16_t* h = reinterpret_cast<uint16_t*>(ws + p.h);
  l.rows = rows.rows;
  l.h = HeadMatrix{h, p.K, (int32_t)p.chunk_rows, p.K};
  l.bias = static_cast<const uint16_t*>(bias);
  l.K = p.K;
  l.V = V;
  l.k = d.topk;
  l.cap = d.softcap;
  l.c = exponent_scale(d);
  l.labels = labels;
  l.tidx = teacher_idx;
  l.tval = teacher_val;
  l.x = reinterpret_cast<float*>(ws + p.x);
  l.r0 = reinterpret_cast<float*>(ws + p.r0);
  float2* part = reinterpret_cast<float2*>(ws + p.part);
  l.part = part;
  l.parts = p.parts;
  l.part_columns = p.part_columns;
  l.kd = kd_tok;
  l.nll = nll_tok;
  l.lse = lse_tok;
  l.status = dev_status;
  l.kd_weight = kd_weight(d);
  l.ce_weight = d.ce_grad_scale;
  l.e = grads ? reinterpret_cast<uint16_t*>(ws + p.e) : nullptr;
  l.e_stride = p.e_stride;
  l.scale = grads ? reinterpret_cast<float*>(ws + p.scale) : nullptr;
  l.hs = grad_weight ? reinterpret_cast<uint16_t*>(ws + p.hs) : nullptr;

  HeadForwardArgs f{};
  f.q = l.h;
  f.D = D;
  f.w = w;
  f.bias = l.bias;
  f.K = p.K;
  f.V = V;
  f.cap = d.softcap;
  f.c = l.c;
  f.r0 = l.r0;
  f.part = part;
  f.parts = p.parts;
  f.part_columns = p.part_columns;
  f.tokens = p.tokens;
  f.e = l.e;
  f.e_stride = p.e_stride;

  const HeadMatrix e = {l.e, p.e_stride, (int32_t)p.chunk_rows, (int32_t)p.e_stride};
  const HeadMatrix hs = {l.hs, p.K, (int32_t)p.chunk_rows, p.K};
  for (int64_t c = 0; c < p.chunks; ++c) {
    const HeadChunk chunk = {rows.count, T, p.cap, (int32_t)c};
    l.chunk = f.chunk = chunk;
    if (p.chunks == 1) {
      NPD_TRY(launch_head_prepare(rows, l, on));
    } else {
      if (c == 0) NPD_TRY(launch_head_rows(rows, on));
      NPD_TRY(launch_head_gather(l, p.chunk_rows, on));
    }
    NPD_TRY((p.few ? launch_head_few : launch_head_forward)(f, grads ? kHeadSumsKept : kHeadSums, p.chunk_rows, on));
    NPD_TRY(launch_head_finish(l, p.chunk_rows, on));
    if (!grads) continue;
    st = gradients(d, p, chunk, e, w, hs, l.scale, rows.rows, grad_hidden, grad_weight, grad_bias, ws, on);
    if (st != NPD_OK) return st;
  }
  return NPD_OK;
}

npd_status npd_head_logits(const npd_head_desc* desc, const void* hidden, const void* weight, const void* bias, void* logits,
                           void* workspace, size_t workspace_bytes, void* stream) {
  npd_status st = check_head(desc, NPD_HEAD_LOGITS);
  if (st != NPD_OK) return st;
  const npd_head_desc& d = *desc;
  if (!hidden || !weight || !logits) return NPD_ERR_NULL;
  if (misaligned(hidden, 2) || misaligned(weight, 2) || misaligned(bias, 2) || misaligned(logits, 2) || unaligned(d, hidden) ||
      unaligned(d, weight))
    return NPD_ERR_VALUE;
  Plan p;
  if ((st = choose_plan(d, NPD_HEAD_LOGITS, workspace, workspace_bytes, &p)) != NPD_OK) return st;
  const int64_t T = d.n_tokens;
  {
    const Range in[3] = {range_of(hidden, rows_bytes(T, d.hidden_stride, d.width, 2)),
                         range_of(weight, rows_bytes(d.vocab, d.weight_stride, d.width, 2)), opt_range(bias, (size_t)d.vocab * 2)};
    const Range out[2] = {range_of(logits, rows_bytes(T, d.logits_stride, d.vocab, 2)), opt_range(workspace, p.bytes)};
    if (any_alias(in, 3, out, 2)) return NPD_ERR_ALIAS;
  }
  const hipStream_t on = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  HeadForwardArgs f{};
  f.chunk = HeadChunk{nullptr, T, kWhole, 0};
  if ((st = pack_weight(d, p, static_cast<const uint16_t*>(weight), ws, on, &f.w)) != NPD_OK) return st;
  f.q = HeadMatrix{static_cast<const uint16_t*>(hidden), d.hidden_stride, (int32_t)T, p.K};
  if (p.pack_h) {
    HeadPackArgs pack{};
    pack.chunk = f.chunk;
    pack.src = f.q.p;
    pack.src_stride = d.hidden_stride;
    pack.cols = d.width;
    pack.width = p.K;
    pack.dst = reinterpret_cast<uint16_t*>(ws + p.h);
    pack.dst_stride = p.K;
    NPD_TRY(launch_head_pack(pack, T, on));
    f.q.p = pack.dst;
    f.q.stride = p.K;
  }
  f.bias = static_cast<const uint16_t*>(bias);
  f.D = d.width;
  f.K = p.K;
  f.V = d.vocab;
  f.cap = d.softcap;
  f.parts = p.parts;
  f.part_columns = p.part_columns;
  f.tokens = p.tokens;
  f.out = static_cast<uint16_t*>(logits);
  f.out_stride = d.logits_stride;
  NPD_TRY((p.few ? launch_head_few : launch_head_forward)(f, kHeadLogits, T, on));
  return NPD_OK;
}

npd_status npd_head_logits_bwd(const npd_head_desc* desc, const void* grad_logits, const void* logits, const void* hidden,
                               const void* weight, void* grad_hidden, void* grad_weight, void* grad_bias, void* workspace,
                               size_t workspace_bytes, void* stream) {
  npd_status st = check_head(desc, NPD_HEAD_LOGITS_BWD);
  if (st != NPD_OK) return st;
  const npd_head_desc& d = *desc;
  if (!grad_logits || (d.softcap != 0.0f && !logits)) return NPD_ERR_NULL;
  if (d.softcap == 0.0f && logits) return NPD_ERR_VALUE;
  if ((st = check_grads(d, grad_hidden, grad_weight, grad_bias)) != NPD_OK) return st;
  if ((grad_hidden && !weight) || (grad_weight && !hidden)) return NPD_ERR_NULL;
  if (misaligned(grad_logits, 2) || misaligned(logits, 2) || misaligned(hidden, 2) || misaligned(weight, 2) ||
      unaligned(d, grad_logits) || (grad_weight && unaligned(d, hidden)) || (grad_hidden && unaligned(d, weight)))
    return NPD_ERR_VALUE;
  Plan p;
  if ((st = choose_plan(d, NPD_HEAD_LOGITS_BWD, workspace, workspace_bytes, &p)) != NPD_OK) return st;
  const int64_t T = d.n_tokens;
  const int V = d.vocab, D = d.width;
  {
    const size_t lb = rows_bytes(T, d.logits_stride, V, 2);
    const Range in[4] = {range_of(grad_logits, lb), opt_range(logits, lb),
                         grad_weight ? range_of(hidden, rows_bytes(T, d.hidden_stride, D, 2)) : Range{0, 0},
                         grad_hidden ? range_of(weight, rows_bytes(V, d.weight_stride, D, 2)) : Range{0, 0}};
    const Range out[4] = {grad_hidden ? range_of(grad_hidden, rows_bytes(T, d.grad_hidden_stride, D, 2)) : Range{0, 0},
                          grad_weight ? range_of(grad_weight, rows_bytes(V, d.grad_weight_stride, D, 2)) : Range{0, 0},
                          opt_range(grad_bias, (size_t)V * 2), opt_range(workspace, p.bytes)};
    if (any_alias(in, 4, out, 4)) return NPD_ERR_ALIAS;
  }
  const hipStream_t on = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  HeadMatrix w{};
  if (grad_hidden && (st = pack_weight(d, p, static_cast<const uint16_t*>(weight), ws, on, &w)) != NPD_OK) return st;
  for (int64_t c = 0; c < p.chunks; ++c) {
    const HeadChunk chunk = {nullptr, T, p.cap, (int32_t)c};
    HeadMatrix g = {static_cast<const uint16_t*>(grad_logits), d.logits_stride, (int32_t)T, V};
    HeadMatrix h = {static_cast<const uint16_t*>(hidden), d.hidden_stride, (int32_t)T, p.K};
    HeadPackArgs pack{};
    pack.chunk = chunk;
    if (p.pack_g) {
      pack.src = g.p;
      pack.src_stride = d.logits_stride;
      pack.y = d.softcap != 0.0f ? static_cast<const uint16_t*>(logits) : nullptr;
      pack.y_stride = d.logits_stride;
      pack.cap = d.softcap;
      pack.cols = V;
      pack.width = (int32_t)up(V, 8);
      pack.dst = reinterpret_cast<uint16_t*>(ws + p.e);
      pack.dst_stride = p.e_stride;
      NPD_TRY(launch_head_pack(pack, p.chunk_rows, on));
      g = HeadMatrix{pack.dst, p.e_stride, (int32_t)p.chunk_rows, pack.width};
    }
    if (grad_weight && p.pack_h) {
      pack.src = h.p;
      pack.src_stride = d.hidden_stride;
      pack.y = nullptr;
      pack.cols = D;
      pack.width = p.K;
      pack.dst = reinterpret_cast<uint16_t*>(ws + p.h);
      pack.dst_stride = p.K;
      NPD_TRY(launch_head_pack(pack, p.chunk_rows, on));
      h = HeadMatrix{pack.dst, p.K, (int32_t)p.chunk_rows, p.K};
    }
    st = gradients(d, p, chunk, g, w, h, nullptr, nullptr, grad_hidden, grad_weight, grad_bias, ws, on);
    if (st != NPD_OK) return st;
  }
  return NPD_OK;
}

}  // extern "C"
