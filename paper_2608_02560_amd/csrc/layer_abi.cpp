// C-ABI layer of the gated-delta rule, its convolution and token scoring
// (include/precog.h): host-side validation and launches.  Nothing here
// allocates, copies between host and device or synchronises.
#include <cmath>

#include <hip/hip_runtime.h>

#include "layer_kernels.h"

namespace {

bool aligned(const void* p, uintptr_t to) {
  return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0;
}

constexpr int64_t kMaxTokens = 0x7fffffffLL;  // of one call: positions are int32
constexpr int64_t kMaxStride = 1LL << 24;     // elements between tokens: 32 of them stay below 2^31 bytes

int size_of(precog_dtype t) { return t == PRECOG_F32 ? 4 : 2; }

bool valid_io(precog_dtype t) { return t == PRECOG_F32 || t == PRECOG_BF16; }

// [a, a + an) and [b, b + bn) share a byte
bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return an && bn && x < y + bn && y < x + an;
}

// A launch holds fewer than 2^32 threads.
bool launchable(int64_t workgroups, int64_t threads) { return workgroups <= 0xffffffffLL / threads; }

// Status of a finished launch.
precog_status launched(hipError_t e) { return e == hipSuccess ? PRECOG_OK : PRECOG_ERR_HIP; }

precog_status validate_delta(const precog_delta_desc* d, bool step) {
  if (!d) return PRECOG_ERR_NULL;
  if (d->batch < 0 || (!step && d->seqlen < 0)) return PRECOG_ERR_SHAPE;
  if (d->batch > kMaxTokens || (!step && d->seqlen > kMaxTokens)) return PRECOG_ERR_SHAPE;
  if (step && d->batch > 65535) return PRECOG_ERR_SHAPE;
  if (d->k_heads < 1 || d->v_heads < 1 || d->k_heads > 65535 || d->v_heads > 65535 ||
      d->v_heads % d->k_heads != 0)
    return PRECOG_ERR_SHAPE;
  if (d->k_dim < 8 || d->k_dim > precog::kDeltaMaxK || d->k_dim % 8 != 0) return PRECOG_ERR_SHAPE;
  if (d->v_dim < 8 || d->v_dim > precog::kDeltaMaxV || d->v_dim % 8 != 0) return PRECOG_ERR_SHAPE;
  if (!(d->eps >= 0.f) || !std::isfinite(d->eps) || !std::isfinite(d->scale)) return PRECOG_ERR_SHAPE;
  if (!valid_io(d->in_dtype) || !valid_io(d->out_dtype)) return PRECOG_ERR_DTYPE;
  if (d->state_dtype != PRECOG_F32 && d->state_dtype != PRECOG_F16) return PRECOG_ERR_DTYPE;
  const int64_t kd = d->k_heads * d->k_dim, vd = d->v_heads * d->v_dim, sd = vd * d->k_dim;
  if (kd > kMaxStride || vd > kMaxStride) return PRECOG_ERR_SHAPE;
  const struct { int64_t stride, least; } token[] = {{d->q_stride, kd}, {d->k_stride, kd}, {d->v_stride, vd}};
  for (const auto& t : token) {
    if (t.stride == 0) continue;
    if (t.stride < t.least || t.stride > kMaxStride) return PRECOG_ERR_STRIDE;
    if (t.stride % 8 != 0) return PRECOG_ERR_ALIGN;
  }
  for (const int64_t s : {d->h0_batch_stride, d->hT_batch_stride}) {
    if (s == 0) continue;
    if (s < sd || s > (1LL << 40)) return PRECOG_ERR_STRIDE;
    if (s % 8 != 0) return PRECOG_ERR_ALIGN;
  }
  return PRECOG_OK;
}

precog::DeltaParams delta_params(const precog_delta_desc* d, const void* q, const void* k,
                                 const void* v, const float* g, const float* beta, void* o) {
  precog::DeltaParams p{};
  const int64_t kd = d->k_heads * d->k_dim, vd = d->v_heads * d->v_dim;
  p.q = q;
  p.k = k;
  p.v = v;
  p.g = g;
  p.beta = beta;
  p.o = o;
  p.B = d->batch;
  p.q_stride = d->q_stride ? d->q_stride : kd;
  p.k_stride = d->k_stride ? d->k_stride : kd;
  p.v_stride = d->v_stride ? d->v_stride : vd;
  p.h0_stride = d->h0_batch_stride ? d->h0_batch_stride : vd * d->k_dim;
  p.hT_stride = d->hT_batch_stride ? d->hT_batch_stride : vd * d->k_dim;
  p.Hk = static_cast<int>(d->k_heads);
  p.Hv = static_cast<int>(d->v_heads);
  p.K = static_cast<int>(d->k_dim);
  p.V = static_cast<int>(d->v_dim);
  p.norm = d->qk_norm != 0;
  p.eps = d->eps;
  p.scale = d->scale != 0.f ? d->scale : 1.f / std::sqrt(static_cast<float>(d->k_dim));
  return p;
}

// Segments that every sequence of a call is cut into.  A head's blocks of 32
// tokens run one after the other on one CU, so up to 64 heads leave CUs idle that
// can take other segments, at three times the work: 8 heads of 40,001 tokens take
// 2,410 us whole and 408 us in 32 segments, 64 heads of 16,384 tokens 1,435 us
// and 896 us in 4; 128 heads of 2,048 tokens 187 us and 181 us in 2, which is not
// worth its workspace.  A segment has 16 blocks or more (8 heads of 2,048 tokens:
// 130 us whole, 103 us in 4).
int64_t delta_segments(const precog_delta_desc* d, int64_t tokens) {
  const int64_t heads = d->batch * d->v_heads * ((d->v_dim + 127) / 128);
  const int64_t blocks = (tokens + 31) / 32 / d->batch;  // of a sequence, on average
  if (heads > 64) return 1;
  int64_t n = 256 / heads;
  if (n > 32) n = 32;
  if (n > blocks / 16) n = blocks / 16;
  return n < 4 ? 1 : n;
}

// Whether a call's heads fit one launch: workgroups of up to 128 columns.
bool delta_launchable(const precog_delta_desc* d) {
  const int64_t columns = (d->v_dim + 31) / 32;
  const int64_t waves = columns < precog::kDeltaChainMax ? columns : precog::kDeltaChainMax;
  const int64_t prepare = precog::delta_prepare_waves(d->in_dtype == PRECOG_F32, d->k_dim > 64);
  return launchable(d->batch * d->v_heads * ((columns + waves - 1) / waves), 64 * (waves + prepare));
}

struct DeltaWs {
  size_t between, total;
};
DeltaWs delta_ws(const precog_delta_desc* d, int64_t segments) {
  DeltaWs w{0, 0};
  if (segments <= 1) return w;
  const size_t rows = static_cast<size_t>(d->batch * segments * d->v_heads * d->k_dim) * 4;
  w.between = rows * static_cast<size_t>(d->v_dim);
  w.total = w.between + rows * static_cast<size_t>(d->k_dim);
  return w;
}

// Tokens of a call, or -1 if there are more than a call can have.
int64_t delta_tokens(int64_t B, int64_t L, bool packed) {
  if (packed) return L;
  return L > 0 && B > kMaxTokens / L ? -1 : B * L;
}

precog_status validate_conv(const precog_conv_desc* d, bool step) {
  if (!d) return PRECOG_ERR_NULL;
  if (d->batch < 0 || d->dim < 0 || (!step && d->seqlen < 0)) return PRECOG_ERR_SHAPE;
  if (d->batch > (1LL << 30) || d->dim > kMaxStride || (!step && d->seqlen > kMaxTokens))
    return PRECOG_ERR_SHAPE;
  if (step && d->batch > 65535) return PRECOG_ERR_SHAPE;
  if (d->width < 2 || d->width > 4) return PRECOG_ERR_SHAPE;
  if (!valid_io(d->in_dtype) || !valid_io(d->out_dtype)) return PRECOG_ERR_DTYPE;
  if (d->x_stride != 0 && (d->x_stride < d->dim || d->x_stride > kMaxStride)) return PRECOG_ERR_STRIDE;
  if (d->dim % 8 != 0 || d->x_stride % 8 != 0) return PRECOG_ERR_ALIGN;
  return PRECOG_OK;
}

precog::ConvParams conv_params(const precog_conv_desc* d, const void* x, const float* w,
                               const float* bias, void* y) {
  precog::ConvParams p{};
  p.x = x;
  p.w = w;
  p.bias = bias;
  p.y = y;
  p.B = d->batch;
  p.D = d->dim;
  p.x_stride = d->x_stride ? d->x_stride : d->dim;
  p.W = static_cast<int>(d->width);
  p.silu = d->silu != 0;
  return p;
}

// Workgroups of one row of a scoring call: as many as give each of the 256 CUs
// one (more of them cost more than they read faster: 333 rows of 32,003 fp32
// logits take 17.4 us with one a CU, 20.5 us with two, 28.6 us with eight), each
// with four tiles or more, which its waves load at once (8 rows of 131,072 bf16
// logits: 12.7 us; with two tiles each 15.4 us).
int64_t score_splits(int64_t T, int64_t V) {
  const int64_t tiles = (V + precog::kScoreTile - 1) / precog::kScoreTile;
  const int64_t want = (256 + T - 1) / T;
  const int64_t most = tiles / 4 < 64 ? tiles / 4 : 64;
  const int64_t n = want < most ? want : most;
  return n < 1 ? 1 : n;
}

bool valid_score(int64_t T, int64_t V, int64_t top) {
  return T >= 0 && V >= 1 && T <= 0x7fffffffLL && V <= (1LL << 28) && top >= 0 &&
         top <= precog::kScoreMaxTop;
}

struct ScoreWs {
  size_t part, val, total;
};
ScoreWs score_ws(int64_t T, int64_t splits, int64_t top) {
  ScoreWs w{0, 0, 0};
  if (splits <= 1) return w;
  const auto up = [](size_t v) { return (v + 255) & ~static_cast<size_t>(255); };
  w.part = up(static_cast<size_t>(T) * splits * sizeof(precog::ScorePart));
  w.val = up(static_cast<size_t>(T) * splits * top * 4);
  w.total = w.part + 2 * w.val;
  return w;
}

}  // namespace

extern "C" {

size_t precog_delta_workspace_bytes(const precog_delta_desc* desc, int packed) {
  if (validate_delta(desc, false) != PRECOG_OK) return 0;
  const int64_t tokens = delta_tokens(desc->batch, desc->seqlen, packed != 0);
  if (tokens <= 0 || desc->batch == 0 || desc->batch * desc->v_heads > kMaxTokens / 8) return 0;
  return delta_ws(desc, delta_segments(desc, tokens)).total;
}

precog_status precog_delta_encode(const precog_delta_desc* desc, const void* q, const void* k,
                                  const void* v, const float* g, const float* beta,
                                  const int32_t* starts, const void* h0, int64_t h0_rows,
                                  const int32_t* h0_idx, void* o, void* hT, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  precog_status st = validate_delta(desc, false);
  if (st != PRECOG_OK) return st;
  const int64_t B = desc->batch, L = desc->seqlen;
  const int64_t tokens = delta_tokens(B, L, starts != nullptr);
  if (tokens < 0) return PRECOG_ERR_SHAPE;
  if (B * desc->v_heads > kMaxTokens / 8) return PRECOG_ERR_SHAPE;  // workgroups, 8 a head at most
  if (B == 0) return PRECOG_OK;
  const bool work = tokens > 0;
  if (work && (!k || !v || (o && !q))) return PRECOG_ERR_NULL;
  if ((!o || !work) && !hT) return PRECOG_OK;  // nothing requested
  if (h0_idx && h0_rows < 0) return PRECOG_ERR_SHAPE;
  if (h0_idx && h0_rows > 0 && !h0) return PRECOG_ERR_NULL;
  for (const void* p : {q, k, v, h0, static_cast<const void*>(o), static_cast<const void*>(hT),
                        static_cast<const void*>(workspace)})
    if (!aligned(p, 16)) return PRECOG_ERR_ALIGN;
  if (!aligned(g, 4) || !aligned(beta, 4) || !aligned(starts, 4) || !aligned(h0_idx, 4))
    return PRECOG_ERR_ALIGN;

  precog::DeltaParams p = delta_params(desc, q, k, v, g, beta, work ? o : nullptr);
  p.starts = starts;
  p.idx = h0_idx;
  p.state_rows = h0_idx ? h0_rows : B;
  p.h0 = h0;
  p.hT = hT;
  p.L = L;
  p.T = tokens;
  // hT over h0: in place, row for row, or not at all
  const int64_t sd = desc->v_heads * desc->v_dim * desc->k_dim;
  const size_t es = static_cast<size_t>(size_of(desc->state_dtype));
  const int64_t rows = h0_idx ? h0_rows : B;
  if (h0 && hT && rows > 0 &&
      overlap(h0, ((rows - 1) * p.h0_stride + sd) * es, hT, ((B - 1) * p.hT_stride + sd) * es)) {
    const bool layers = !h0_idx && p.h0_stride == p.hT_stride;  // slots of one multi-layer store
    const auto a = reinterpret_cast<uintptr_t>(h0), b = reinterpret_cast<uintptr_t>(hT);
    const size_t pitch = static_cast<size_t>(p.h0_stride) * es, one = static_cast<size_t>(sd) * es;
    const size_t off = (a < b ? b - a : a - b) % pitch;
    if (!layers || (h0 != hT && (off < one || off + one > pitch))) return PRECOG_ERR_STRIDE;
  }
  p.segments = static_cast<int>(work ? delta_segments(desc, tokens) : 1);
  const DeltaWs ws = delta_ws(desc, p.segments);
  if (ws.total > 0 && (!workspace || workspace_bytes < ws.total)) return PRECOG_ERR_WORKSPACE;
  if (ws.total > 0) {
    p.between = static_cast<float*>(workspace);
    p.phi = reinterpret_cast<float*>(static_cast<char*>(workspace) + ws.between);
  }
  if (!delta_launchable(desc)) return PRECOG_ERR_SHAPE;
  int cus = 1;
  st = precog::check_device(&cus);
  if (st != PRECOG_OK) return st;
  (void)hipGetLastError();
  return launched(precog::launch_delta(p, desc->in_dtype, desc->out_dtype, desc->state_dtype, cus,
                                       static_cast<hipStream_t>(stream)));
}

precog_status precog_delta_step(const precog_delta_desc* desc, const void* q, const void* k,
                                const void* v, const float* g, const float* beta, void* states,
                                int64_t state_rows, const int32_t* slots, void* o, void* stream) {
  precog_status st = validate_delta(desc, true);
  if (st != PRECOG_OK) return st;
  if (state_rows < 0) return PRECOG_ERR_SHAPE;
  if (desc->batch * desc->v_heads > kMaxTokens / 8) return PRECOG_ERR_SHAPE;  // workgroups, 8 a head at most
  if (desc->batch == 0) return PRECOG_OK;
  if (!k || !v || !slots || (o && !q) || (state_rows > 0 && !states)) return PRECOG_ERR_NULL;
  for (const void* p : {q, k, v, static_cast<const void*>(states), static_cast<const void*>(o)})
    if (!aligned(p, 16)) return PRECOG_ERR_ALIGN;
  if (!aligned(g, 4) || !aligned(beta, 4) || !aligned(slots, 4)) return PRECOG_ERR_ALIGN;
  if (state_rows == 0) return PRECOG_OK;  // no slot can name a row
  if (!launchable(desc->batch * desc->v_heads * ((desc->v_dim + 127) / 128), 256)) return PRECOG_ERR_SHAPE;

  precog::DeltaParams p = delta_params(desc, q, k, v, g, beta, o);
  p.idx = slots;
  p.state_rows = state_rows;
  p.h0 = states;
  p.hT = states;
  int cus = 1;
  st = precog::check_device(&cus);
  if (st != PRECOG_OK) return st;
  (void)hipGetLastError();
  return launched(precog::launch_delta_step(p, desc->in_dtype, desc->out_dtype, desc->state_dtype,
                                            cus, static_cast<hipStream_t>(stream)));
}

precog_status precog_conv_encode(const precog_conv_desc* desc, const void* x, const float* w,
                                 const float* bias, const int32_t* starts, const void* tail0,
                                 int64_t tail_rows, const int32_t* tail_idx, void* y, void* tailT,
                                 void* stream) {
  precog_status st = validate_conv(desc, false);
  if (st != PRECOG_OK) return st;
  const int64_t B = desc->batch, L = desc->seqlen, D = desc->dim;
  const int64_t tokens = delta_tokens(B, L, starts != nullptr);
  if (tokens < 0) return PRECOG_ERR_SHAPE;
  if (B == 0 || D == 0) return PRECOG_OK;
  const bool work = tokens > 0;
  if (work && !x) return PRECOG_ERR_NULL;
  if (work && y && !w) return PRECOG_ERR_NULL;
  if ((!y || !work) && !tailT) return PRECOG_OK;  // nothing requested
  if (tail_idx && tail_rows < 0) return PRECOG_ERR_SHAPE;
  if (tail_idx && tail_rows > 0 && !tail0) return PRECOG_ERR_NULL;
  for (const void* p : {x, static_cast<const void*>(w), static_cast<const void*>(bias), tail0,
                        static_cast<const void*>(y), static_cast<const void*>(tailT)})
    if (!aligned(p, 16)) return PRECOG_ERR_ALIGN;
  if (!aligned(starts, 4) || !aligned(tail_idx, 4)) return PRECOG_ERR_ALIGN;
  const size_t row = static_cast<size_t>((desc->width - 1) * D) * size_of(desc->in_dtype);
  const int64_t rows = tail_idx ? tail_rows : B;
  if (tail0 && tailT && overlap(tail0, rows * row, tailT, B * row) && (tail_idx || tail0 != tailT))
    return PRECOG_ERR_STRIDE;

  precog::ConvParams p = conv_params(desc, x, w, bias, work ? y : nullptr);
  p.starts = starts;
  p.idx = tail_idx;
  p.tail_rows = tail_idx ? tail_rows : B;
  p.tail0 = tail0;
  p.tailT = tailT;
  p.L = L;
  p.T = tokens;
  // runs of 32 tokens and the tails, which go by themselves in place
  const int64_t runs = p.y ? (tokens + 31) / 32 : 0, tails = tailT ? B : 0;
  const bool apart = tail0 && tail0 == tailT && runs > 0;
  if (!launchable(apart ? (runs > tails ? runs : tails) : runs + tails, D > 1536 ? 256 : (D + 511) / 512 * 64))
    return PRECOG_ERR_SHAPE;
  int cus = 1;
  st = precog::check_device(&cus);
  if (st != PRECOG_OK) return st;
  (void)hipGetLastError();
  return launched(precog::launch_conv(p, desc->in_dtype, desc->out_dtype, cus,
                                      static_cast<hipStream_t>(stream)));
}

precog_status precog_conv_step(const precog_conv_desc* desc, const void* x, const float* w,
                               const float* bias, void* tails, int64_t tail_rows,
                               const int32_t* slots, void* y, void* stream) {
  precog_status st = validate_conv(desc, true);
  if (st != PRECOG_OK) return st;
  if (tail_rows < 0) return PRECOG_ERR_SHAPE;
  if (desc->batch == 0 || desc->dim == 0) return PRECOG_OK;
  if (!x || !slots || (y && !w) || (tail_rows > 0 && !tails)) return PRECOG_ERR_NULL;
  for (const void* p : {x, static_cast<const void*>(w), static_cast<const void*>(bias),
                        static_cast<const void*>(tails), static_cast<const void*>(y)})
    if (!aligned(p, 16)) return PRECOG_ERR_ALIGN;
  if (!aligned(slots, 4)) return PRECOG_ERR_ALIGN;
  if (tail_rows == 0) return PRECOG_OK;
  precog::ConvParams p = conv_params(desc, x, w, bias, y);
  p.idx = slots;
  p.tail_rows = tail_rows;
  p.tail0 = tails;
  p.tailT = tails;
  st = precog::check_device(nullptr);
  if (st != PRECOG_OK) return st;
  (void)hipGetLastError();
  return launched(precog::launch_conv_step(p, desc->in_dtype, desc->out_dtype,
                                           static_cast<hipStream_t>(stream)));
}

size_t precog_score_workspace_bytes(int64_t T, int64_t V, int64_t top) {
  if (!valid_score(T, V, top) || T == 0) return 0;
  return score_ws(T, score_splits(T, V), top).total;
}

precog_status precog_score_tokens(const void* logits, precog_dtype logits_dtype, int64_t T,
                                  int64_t V, int64_t row_stride, const int32_t* token, int64_t top,
                                  float* logprob, float* entropy, int32_t* top_id,
                                  float* top_logprob, void* workspace, size_t workspace_bytes,
                                  void* stream) {
  if (!valid_score(T, V, top)) return PRECOG_ERR_SHAPE;
  if (logits_dtype != PRECOG_F32 && logits_dtype != PRECOG_BF16 && logits_dtype != PRECOG_F16)
    return PRECOG_ERR_DTYPE;
  if (row_stride != 0 && (row_stride < V || row_stride > (1LL << 40))) return PRECOG_ERR_STRIDE;
  if (T == 0) return PRECOG_OK;
  if (!logits || (token && !logprob) || (top > 0 && (!top_id || !top_logprob)))
    return PRECOG_ERR_NULL;
  if (!token && !entropy && top == 0) return PRECOG_OK;  // nothing requested
  if (!aligned(logits, size_of(logits_dtype)) || !aligned(workspace, 16)) return PRECOG_ERR_ALIGN;
  for (const void* p : {static_cast<const void*>(token), static_cast<const void*>(logprob),
                        static_cast<const void*>(entropy), static_cast<const void*>(top_id),
                        static_cast<const void*>(top_logprob)})
    if (!aligned(p, 4)) return PRECOG_ERR_ALIGN;
  const int64_t splits = score_splits(T, V);
  if (!launchable(T * splits, 256)) return PRECOG_ERR_SHAPE;
  const ScoreWs ws = score_ws(T, splits, top);
  if (ws.total > 0 && (!workspace || workspace_bytes < ws.total)) return PRECOG_ERR_WORKSPACE;

  precog::ScoreParams p{};
  p.logits = logits;
  p.token = token;
  p.logprob = logprob;
  p.entropy = entropy;
  p.top_id = top_id;
  p.top_logprob = top_logprob;
  p.T = T;
  p.V = V;
  p.row_stride = row_stride ? row_stride : V;
  p.top = static_cast<int>(top);
  p.splits = static_cast<int>(splits);
  const int64_t tiles = (V + precog::kScoreTile - 1) / precog::kScoreTile;
  p.span = (tiles + splits - 1) / splits * precog::kScoreTile;
  if (splits > 1) {
    char* at = static_cast<char*>(workspace);
    p.part = reinterpret_cast<precog::ScorePart*>(at);
    p.cand_val = reinterpret_cast<float*>(at + ws.part);
    p.cand_id = reinterpret_cast<int32_t*>(at + ws.part + ws.val);
  }
  const precog_status st = precog::check_device(nullptr);
  if (st != PRECOG_OK) return st;
  (void)hipGetLastError();
  return launched(precog::launch_score(p, logits_dtype, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
