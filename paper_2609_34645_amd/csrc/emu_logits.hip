// Operators on the logits of a vocab-parallel LM head (include/emu.h): constraints ahead of sampling, the
// k largest log-probabilities, distillation with its gradient. One workgroup per row (constraints: per row
// and slice of the vocabulary); every reduction runs over global columns, so that no result depends on how
// the shards cut them.
#include <cmath>

#include "emu_internal.h"

namespace emu {

constexpr int kMaxShards = 64;
constexpr int32_t kMaxVocab = 1 << 22;
constexpr int kMaxTop = 64;        // entries of emu_logits_topk
constexpr int kMaxTeacher = 256;   // entries of a teacher's row
constexpr uint32_t kRowsPerLaunch = 1u << 21;  // a grid's work-items stay below 2^32

// A logits set on the device: row r's columns [t * cols, (t + 1) * cols) lie at p[t] + r * row_bytes.
struct Logits {
  uint8_t* p[kMaxShards];
  uint64_t row_bytes;
  uint32_t V, Vp, cols;
};

typedef uint16_t bf16_t;  // bits
template <typename T> __device__ __forceinline__ T* column(const Logits& l, uint64_t row, uint32_t v) {
  const uint32_t t = v / l.cols;
  return reinterpret_cast<T*>(l.p[t] + row * l.row_bytes) + (v - t * l.cols);
}
__device__ __forceinline__ float widen(bf16_t x) { return __uint_as_float(uint32_t(x) << 16); }
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ void narrow(float x, bf16_t* out) { *out = bf16_t(bf16_rne(__float_as_uint(x))); }
__device__ __forceinline__ void narrow(float x, float* out) { *out = x; }

constexpr float kInf = __builtin_inff();

// Reductions over a workgroup of NT threads in a fixed tree: the result does not depend on timing.
template <int NT, typename T, typename F>
__device__ T block_reduce(T x, T* lds, F f) {
  __syncthreads();
  lds[threadIdx.x] = x;
  __syncthreads();
  for (int n = NT / 2; n; n >>= 1) {
    if (int(threadIdx.x) < n) lds[threadIdx.x] = f(lds[threadIdx.x], lds[threadIdx.x + n]);
    __syncthreads();
  }
  return lds[0];
}

// ------------------------------------------------------------------------------------------------
// constraints
// ------------------------------------------------------------------------------------------------

constexpr int kConstrainThreads = 256;
constexpr uint32_t kSlice = 8192;  // columns of one workgroup
constexpr uint32_t kSeen = 1u << 31;

// Counts of the slice's tokens in LDS (bit 31: occurs at all), a bit per biased token, then one pass over the
// slice's columns. A biased column adds up its entries in list order.
template <typename TI, typename TO>
__global__ __launch_bounds__(kConstrainThreads) void k_constrain(Logits in, Logits out, emu_constraints_t c, uint64_t row0) {
  __shared__ uint32_t count[kSlice];
  __shared__ uint32_t biased[kSlice / 32];
  const uint64_t r = row0 + blockIdx.x;
  const uint32_t c0 = blockIdx.y * kSlice, c1 = umin(c0 + kSlice, in.Vp);
  for (uint32_t i = threadIdx.x; i < kSlice; i += blockDim.x) count[i] = 0;
  for (uint32_t i = threadIdx.x; i < kSlice / 32; i += blockDim.x) biased[i] = 0;
  __syncthreads();
  if (c.tokens) {
    const int32_t* tok = c.tokens + r * c.tokens_stride;
    const int32_t n = min(max(c.seq_len[r], 0), c.tokens_cols);
    const int32_t prompt = c.prompt_len ? c.prompt_len[r] : 0;
    for (int32_t i = threadIdx.x; i < n; i += blockDim.x) {
      const uint32_t v = uint32_t(tok[i]);
      if (v < in.V && v - c0 < kSlice) {
        atomicOr(&count[v - c0], kSeen);
        if (i >= prompt) atomicAdd(&count[v - c0], 1u);
      }
    }
  }
  int64_t b0 = 0, b1 = 0;
  if (c.bias_first) {
    b0 = min(max(int64_t(c.bias_first[r]), int64_t(0)), c.n_bias);
    b1 = min(max(int64_t(c.bias_first[r + 1]), int64_t(0)), c.n_bias);
    for (int64_t i = b0 + threadIdx.x; i < b1; i += blockDim.x) {
      const uint32_t v = uint32_t(c.bias_token[i]);
      if (v < in.V && v - c0 < kSlice) atomicOr(&biased[(v - c0) / 32], 1u << (v % 32));
    }
  }
  __syncthreads();
  const int32_t* mask = nullptr;
  if (c.mask) {
    const int64_t which = c.mask_row ? int64_t(c.mask_row[r]) : int64_t(r);
    if (which >= 0 && which < c.n_masks) mask = c.mask + which * c.mask_stride;
  }
  const float theta = c.repetition ? c.repetition[r] : 1.0f;
  const float af = c.frequency ? c.frequency[r] : 0.0f, ap = c.presence ? c.presence[r] : 0.0f;
  for (uint32_t v = c0 + threadIdx.x; v < c1; v += blockDim.x) {
    float x = -kInf;
    if (v < in.V && (!mask || (uint32_t(mask[v / 32]) >> (v % 32)) & 1u)) {
      x = widen(*column<TI>(in, r, v));
      const uint32_t n = count[v - c0];
      if (n) {
        x = x > 0.0f ? x / theta : x * theta;
        if (n & ~kSeen) x -= af * float(n & ~kSeen) + ap;
      }
      if ((biased[(v - c0) / 32] >> (v % 32)) & 1u) {
        float sum = 0.0f;
        for (int64_t i = b0; i < b1; ++i)
          if (uint32_t(c.bias_token[i]) == v) sum += c.bias_value[i];
        x += sum;
      }
    }
    narrow(x, column<TO>(out, r, v));
  }
}

// ------------------------------------------------------------------------------------------------
// the k largest
// ------------------------------------------------------------------------------------------------

// One number per logit whose order is the result's: the value, then the lower column. 0: never chosen.
__device__ __forceinline__ uint64_t top_key(float x, uint32_t v) {
  if (!(x > -kInf)) return 0;
  const uint32_t u = __float_as_uint(x + 0.0f);  // -0 becomes 0
  const uint32_t order = u & 0x80000000u ? ~u : u | 0x80000000u;
  return uint64_t(order) << 32 | uint32_t(~v);
}
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t order = uint32_t(key >> 32);
  return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order);
}

constexpr int kRowThreads = 256;

// The sum of exp((x - m) / tau) over a row's columns, m its largest logit (NaN aside).
template <typename T>
__device__ void row_softmax(const Logits& l, uint64_t r, float c1, float* lds, float* m_out, float* s_out) {
  float m = -kInf, s = 0.0f;
  for (uint32_t v = threadIdx.x; v < l.V; v += kRowThreads) m = fmaxf(m, widen(*column<T>(l, r, v)));
  m = block_reduce<kRowThreads>(m, lds, [](float a, float b) { return fmaxf(a, b); });
  for (uint32_t v = threadIdx.x; v < l.V; v += kRowThreads) {
    const float x = widen(*column<T>(l, r, v));
    s += x == -kInf ? 0.0f : exp2f((x - m) * c1);
  }
  *m_out = m;
  *s_out = block_reduce<kRowThreads>(s, lds, [](float a, float b) { return a + b; });
}

// log(exp(m / tau) s), in 64 bits: m / tau may pass the range of fp32's product with log2(e).
__device__ __forceinline__ float log_sum_exp(float m, float s, float c1) {
  return s == 0.0f ? -kInf : float((double(m) * double(c1) + double(log2f(s))) * 0.6931471805599453);
}

// log(exp((x - m) / tau) / s), likewise.
__device__ __forceinline__ float log_prob(float x, float m, float s, float c1) {
  return x == -kInf ? -kInf : float(((double(x) - double(m)) * double(c1) - double(log2f(s))) * 0.6931471805599453);
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void k_topk(Logits in, uint32_t k, float c1, int32_t* index, float* logprob,
                                                      float* lse, uint64_t row0) {
  __shared__ float red[kRowThreads];
  __shared__ uint64_t keys[kRowThreads];
  const uint64_t r = row0 + blockIdx.x;
  float m, s;
  row_softmax<T>(in, r, c1, red, &m, &s);
  if (threadIdx.x == 0 && lse) lse[r] = log_sum_exp(m, s, c1);
  uint64_t below = ~0ull;
  for (uint32_t j = 0; j < k; ++j) {
    uint64_t best = 0;
    for (uint32_t v = threadIdx.x; v < in.V; v += kRowThreads) {
      const uint64_t key = top_key(widen(*column<T>(in, r, v)), v);
      if (key < below && key > best) best = key;
    }
    best = block_reduce<kRowThreads>(best, keys, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
    if (threadIdx.x == 0) {
      index[r * k + j] = best ? int32_t(~uint32_t(best)) : -1;
      logprob[r * k + j] = s != s ? s : best ? log_prob(key_value(best), m, s, c1) : -kInf;
    }
    below = best;
  }
}

// ------------------------------------------------------------------------------------------------
// distillation
// ------------------------------------------------------------------------------------------------

// A row's teacher in LDS. Entry j counts where col[j] >= 0: it is its column's first, with the column's whole
// probability.
struct Top {
  int32_t col[kMaxTeacher];
  float p[kMaxTeacher];
  double red[kRowThreads];
};

// Fills t; returns the mass outside the list (0 without a tail).
__device__ float load_teacher(Top& t, const emu_teacher_t& te, uint64_t r, uint32_t V) {
  const int j = threadIdx.x;
  static_assert(kRowThreads == kMaxTeacher, "one entry per thread");
  int32_t col = -1;
  double value = -double(kInf);
  if (j < te.k) {
    const int32_t i = te.index[r * te.index_stride + j];
    if (uint32_t(i) < V) {
      col = i;
      value = double(te.value[r * te.value_stride + j]);
    }
  }
  double top = block_reduce<kRowThreads>(value, t.red, [](double a, double b) { return fmax(a, b); });
  if (te.tail || top == -double(kInf)) top = 0.0;
  double p = col < 0 ? 0.0 : exp(value - top);
  const double sum = block_reduce<kRowThreads>(p, t.red, [](double a, double b) { return a + b; });
  if (!te.tail && sum != 0.0) p /= sum;
  t.col[j] = col;
  t.red[j] = p;
  __syncthreads();
  bool first = col >= 0;
  for (int i = 0; i < te.k; ++i) {
    if (i == j || col < 0 || t.col[i] != col) continue;
    if (i < j) first = false;
    else p += t.red[i];
  }
  __syncthreads();
  t.col[j] = first ? col : -1;
  t.p[j] = first ? float(p) : 0.0f;
  __syncthreads();
  const float rest = float(1.0 - sum);
  return te.tail ? (rest < 0.0f ? 0.0f : rest) : 0.0f;
}

__device__ __forceinline__ int listed(const Top& t, int k, uint32_t v) {
  for (int j = 0; j < k; ++j)
    if (t.col[j] == int32_t(v)) return j;
  return -1;
}

// A list of log-probabilities rounded to fp32 can miss a sum of 1 by sum p |log p| 2^-24 < 2^-20.
constexpr float kRestNoise = 0x1p-20f;

struct Stats {
  float lse, factor, m, s;
};

// The gradient of one row. scale = w / tau.
template <typename TI, typename TO>
__device__ void row_gradient(const Logits& in, const Logits& out, uint64_t r, const Top& t, int k, Stats st, float c1,
                             float scale, bool none) {
  for (uint32_t v = threadIdx.x; v < out.Vp; v += kRowThreads) {
    float d = 0.0f;
    if (v < in.V && scale != 0.0f && !none) {
      const float x = widen(*column<TI>(in, r, v));
      const float q = x == -kInf ? 0.0f : exp2f((x - st.m) * c1) / st.s;
      const int j = listed(t, k, v);
      d = (j >= 0 ? q - t.p[j] : q * st.factor) * scale;
    }
    narrow(d, column<TO>(out, r, v));
  }
}

template <typename TI, typename TO>
__global__ __launch_bounds__(kRowThreads) void k_distill(Logits in, Logits grad, emu_teacher_t te, float c1, float* loss,
                                                         float4* stats, bool with_grad, uint64_t row0) {
  __shared__ Top t;
  __shared__ float red[kRowThreads];
  const uint64_t r = row0 + blockIdx.x;
  const float w = te.weight ? te.weight[r] : 1.0f;
  Stats st = {kInf - kInf, kInf - kInf, kInf - kInf, kInf - kInf};
  float total = 0.0f;
  bool none = false;
  if (w != 0.0f) {
    const float p_rest = load_teacher(t, te, r, in.V);
    row_softmax<TI>(in, r, c1, red, &st.m, &st.s);
    const float ln2 = 0.69314718f, ls = log2f(st.s);
    st.lse = log_sum_exp(st.m, st.s, c1);
    st.factor = 1.0f;
    const int j = threadIdx.x;
    float part = 0.0f;
    if (t.p[j] != 0.0f) {
      part = t.p[j] * (logf(t.p[j]) - log_prob(widen(*column<TI>(in, r, t.col[j])), st.m, st.s, c1));
    }
    total = block_reduce<kRowThreads>(part, red, [](float a, float b) { return a + b; });
    const float mass = block_reduce<kRowThreads>(t.p[j], red, [](float a, float b) { return a + b; });
    none = !te.tail && mass == 0.0f;
    if (te.tail) {
      float m = -kInf, s = 0.0f;
      for (uint32_t v = threadIdx.x; v < in.V; v += kRowThreads)
        if (listed(t, te.k, v) < 0) m = fmaxf(m, widen(*column<TI>(in, r, v)));
      m = block_reduce<kRowThreads>(m, red, [](float a, float b) { return fmaxf(a, b); });
      for (uint32_t v = threadIdx.x; v < in.V; v += kRowThreads) {
        const float x = widen(*column<TI>(in, r, v));
        if (listed(t, te.k, v) < 0 && x != -kInf) s += exp2f((x - m) * c1);
      }
      s = block_reduce<kRowThreads>(s, red, [](float a, float b) { return a + b; });
      const float log_q = s == 0.0f ? -kInf : ((m - st.m) * c1 + log2f(s) - ls) * ln2;
      if (p_rest != 0.0f && (s != 0.0f || p_rest >= kRestNoise)) total += p_rest * (logf(p_rest) - log_q);
      const float q = expf(log_q);
      if (q != 0.0f) st.factor = 1.0f - p_rest / q;
    }
    total *= w;
  }
  if (threadIdx.x == 0) {
    loss[r] = total;
    stats[r] = make_float4(st.lse, st.factor, st.m, st.s);
  }
  if (with_grad) {
    __syncthreads();
    row_gradient<TI, TO>(in, grad, r, t, te.k, st, c1, w * c1 * 0.69314718f, none);
  }
}

template <typename TI, typename TO>
__global__ __launch_bounds__(kRowThreads) void k_distill_backward(Logits in, Logits grad, emu_teacher_t te, float c1,
                                                                  const float4* stats, uint64_t row0) {
  __shared__ Top t;
  __shared__ float red[kRowThreads];
  const uint64_t r = row0 + blockIdx.x;
  const float w = te.weight ? te.weight[r] : 1.0f;
  Stats st = {};
  bool none = false;
  if (w != 0.0f) {
    load_teacher(t, te, r, in.V);
    const float mass = block_reduce<kRowThreads>(t.p[threadIdx.x], red, [](float a, float b) { return a + b; });
    none = !te.tail && mass == 0.0f;
    const float4 f = stats[r];
    st = {f.x, f.y, f.z, f.w};
  }
  row_gradient<TI, TO>(in, grad, r, t, te.k, st, c1, w * c1 * 0.69314718f, none);
}

// ------------------------------------------------------------------------------------------------
// checks and launches
// ------------------------------------------------------------------------------------------------

static int check_logits(const emu_logits_t* l, const char* what, Logits* out) {
  if (!l || !l->layout) return fail(EMU_ERR_NULL, "%s: NULL logits or layout", what);
  if (int rc = emu_layout_check(l->layout)) return rc;
  const emu_layout_t& lay = *l->layout;
  if (l->dtype != EMU_BF16 && l->dtype != EMU_FP32) return fail(EMU_ERR_ARG, "%s: unknown dtype %d", what, l->dtype);
  if (l->n_shards != lay.tp) return fail(EMU_ERR_ARG, "%s: %d shards, the layout has tp=%d", what, l->n_shards, lay.tp);
  if (lay.tp > kMaxShards) return fail(EMU_ERR_UNSUPPORTED, "%s: tp=%d, at most %d", what, lay.tp, kMaxShards);
  const int64_t vp = padded_vocab(lay), cols = vp / lay.tp;
  if (vp > kMaxVocab) return fail(EMU_ERR_UNSUPPORTED, "%s: a vocabulary of %lld columns, at most %d", what, (long long)vp, kMaxVocab);
  if (l->rows < 0) return fail(EMU_ERR_ARG, "%s: %lld rows", what, (long long)l->rows);
  if (l->rows > 0x7fffffff) return fail(EMU_ERR_UNSUPPORTED, "%s: %lld rows", what, (long long)l->rows);
  if (l->row_stride < cols || l->row_stride > (int64_t(1) << 40))
    return fail(EMU_ERR_ARG, "%s: row stride %lld, a shard has %lld columns", what, (long long)l->row_stride, (long long)cols);
  const uint64_t es = l->dtype == EMU_BF16 ? 2 : 4;
  *out = Logits{};
  out->row_bytes = uint64_t(l->row_stride) * es;
  out->V = uint32_t(lay.model.vocab);
  out->Vp = uint32_t(vp);
  out->cols = uint32_t(cols);
  if (l->rows == 0) return EMU_OK;
  if (!l->shards) return fail(EMU_ERR_NULL, "%s: NULL shards", what);
  for (int t = 0; t < lay.tp; ++t) {
    if (!l->shards[t]) return fail(EMU_ERR_NULL, "%s: shard %d is NULL", what, t);
    if (misaligned(l->shards[t], es)) return fail(EMU_ERR_ALIGN, "%s: shard %d is not on an element", what, t);
    out->p[t] = static_cast<uint8_t*>(l->shards[t]);
  }
  return EMU_OK;
}

// The output set of a call: the input's vocabulary and split, its own dtype and stride.
static int check_output(const emu_logits_t* in, const emu_logits_t* out, const char* what, Logits* view) {
  if (int rc = check_logits(out, what, view)) return rc;
  if (out->layout->model.vocab != in->layout->model.vocab || out->layout->tp != in->layout->tp ||
      padded_vocab(*out->layout) != padded_vocab(*in->layout) || out->rows != in->rows)
    return fail(EMU_ERR_MISMATCH, "%s: another vocabulary, split or number of rows than the input", what);
  if (out->rows == 0) return EMU_OK;
  int same = 0;
  for (int t = 0; t < in->n_shards; ++t) same += out->shards[t] == in->shards[t];
  if (same && (same != in->n_shards || out->dtype != in->dtype || out->row_stride != in->row_stride))
    return fail(EMU_ERR_OVERLAP, "%s: shares shards with the input but is not the same set", what);
  return EMU_OK;
}

static int check_temperature(float tau, float* c1) {
  const double c = 1.4426950408889634 / double(tau);
  if (!(tau > 0.0f) || !(c < 1e30) || !(c > 1e-30)) return fail(EMU_ERR_ARG, "temperature %g is not a positive number in range", double(tau));
  *c1 = float(c);
  return EMU_OK;
}

static int check_operand(const void* p, bool needed, const char* what, uintptr_t align = 4) {
  if (needed && !p) return fail(EMU_ERR_NULL, "%s is NULL", what);
  if (misaligned(p, align)) return fail(EMU_ERR_ALIGN, "%s is not %d-byte aligned", what, int(align));
  return EMU_OK;
}

static int check_teacher(const emu_teacher_t* t, int64_t rows, float* c1) {
  if (!t) return fail(EMU_ERR_NULL, "teacher is NULL");
  if (t->k < 1 || t->k > kMaxTeacher) return fail(EMU_ERR_RANGE, "k %d not in [1, %d]", t->k, kMaxTeacher);
  if (t->tail != 0 && t->tail != 1) return fail(EMU_ERR_ARG, "tail must be 0 or 1");
  if (int rc = check_temperature(t->temperature, c1)) return rc;
  if (t->index_stride < t->k || t->value_stride < t->k) return fail(EMU_ERR_ARG, "a teacher's row stride is below k");
  if (int rc = check_operand(t->index, rows > 0, "teacher index")) return rc;
  if (int rc = check_operand(t->value, rows > 0, "teacher value")) return rc;
  return check_operand(t->weight, false, "teacher weight");
}

static int check_workspace(const emu_logits_t* l, int32_t k, const void* ws, uint64_t bytes) {
  uint64_t need = 0;
  if (int rc = emu_logits_workspace(l, k, &need)) return rc;
  if (need == 0) return EMU_OK;
  if (!ws) return fail(EMU_ERR_NULL, "workspace is NULL");
  if (misaligned(ws, kWsAlign)) return fail(EMU_ERR_WORKSPACE, "workspace not %llu-byte aligned", (unsigned long long)kWsAlign);
  if (bytes < need) return fail(EMU_ERR_WORKSPACE, "workspace of %llu bytes, the call needs %llu", (unsigned long long)bytes, (unsigned long long)need);
  return EMU_OK;
}

// f(first row, rows) for ranges of rows that one grid holds.
template <typename F>
static void over_rows(int64_t rows, F f) {
  for (int64_t r = 0; r < rows; r += kRowsPerLaunch) f(uint64_t(r), uint32_t(std::min<int64_t>(rows - r, kRowsPerLaunch)));
}

// f(input element, output element) for the two dtypes.
template <typename F>
static void by_types(int32_t in, int32_t out, F f) {
  if (in == EMU_BF16) out == EMU_BF16 ? f(bf16_t(), bf16_t()) : f(bf16_t(), float());
  else out == EMU_BF16 ? f(float(), bf16_t()) : f(float(), float());
}

}  // namespace emu

using namespace emu;

extern "C" {

int emu_logits_workspace(const emu_logits_t* logits, int32_t k, uint64_t* bytes) {
  clear_error();
  Logits l;
  if (!bytes) return fail(EMU_ERR_NULL, "bytes is NULL");
  if (int rc = check_logits(logits, "logits", &l)) return rc;
  if (k < 0 || k > kMaxTop) return fail(EMU_ERR_RANGE, "k %d not in [0, %d]", k, kMaxTop);
  *bytes = 0;
  return EMU_OK;
}

int emu_logits_constrain(const emu_logits_t* in, const emu_logits_t* out, const emu_constraints_t* c, void* hip_stream) {
  clear_error();
  Logits li, lo;
  if (int rc = check_logits(in, "in", &li)) return rc;
  if (int rc = check_output(in, out, "out", &lo)) return rc;
  if (!c) return fail(EMU_ERR_NULL, "constraints is NULL");
  const bool any = in->rows > 0;
  if (c->tokens) {
    if (c->tokens_cols < 0 || c->tokens_stride < c->tokens_cols) return fail(EMU_ERR_ARG, "token rows of %d in a stride of %lld", c->tokens_cols, (long long)c->tokens_stride);
    if (int rc = check_operand(c->seq_len, any, "seq_len")) return rc;
  }
  if (c->bias_first) {
    if (c->n_bias < 0) return fail(EMU_ERR_ARG, "%lld biases", (long long)c->n_bias);
    if (int rc = check_operand(c->bias_token, c->n_bias > 0, "bias_token")) return rc;
    if (int rc = check_operand(c->bias_value, c->n_bias > 0, "bias_value")) return rc;
  }
  if (c->mask) {
    if (c->n_masks < 0) return fail(EMU_ERR_ARG, "%d masks", c->n_masks);
    if (c->mask_stride < (int64_t(li.V) + 31) / 32) return fail(EMU_ERR_ARG, "a mask row of %lld words is short of %u tokens", (long long)c->mask_stride, li.V);
    if (!c->mask_row && c->n_masks != in->rows) return fail(EMU_ERR_ARG, "%d masks for %lld rows without mask_row", c->n_masks, (long long)in->rows);
  }
  const struct { const void* p; const char* name; } operands[] = {
      {c->tokens, "tokens"}, {c->prompt_len, "prompt_len"}, {c->repetition, "repetition"}, {c->frequency, "frequency"},
      {c->presence, "presence"}, {c->bias_first, "bias_first"}, {c->mask, "mask"}, {c->mask_row, "mask_row"}};
  for (const auto& o : operands)
    if (int rc = check_operand(o.p, false, o.name)) return rc;
  if (!any) return EMU_OK;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  drop_pending_error();
  by_types(in->dtype, out->dtype, [&](auto ti, auto to) {
    over_rows(in->rows, [&](uint64_t r0, uint32_t n) {
      hipLaunchKernelGGL((k_constrain<decltype(ti), decltype(to)>), dim3(n, (li.Vp + kSlice - 1) / kSlice),
                         dim3(kConstrainThreads), 0, st, li, lo, *c, r0);
    });
  });
  return hip_check("emu_logits_constrain launch");
}

int emu_logits_topk(const emu_logits_t* in, int32_t k, float temperature, int32_t* d_index, float* d_logprob, float* d_lse,
                    void* d_workspace, uint64_t workspace_bytes, void* hip_stream) {
  clear_error();
  Logits l;
  float c1;
  if (int rc = check_logits(in, "in", &l)) return rc;
  if (k < 1 || k > kMaxTop || uint32_t(k) > l.V) return fail(EMU_ERR_RANGE, "k %d not in [1, %d] or above the vocabulary", k, kMaxTop);
  if (int rc = check_temperature(temperature, &c1)) return rc;
  if (int rc = check_operand(d_index, in->rows > 0, "index")) return rc;
  if (int rc = check_operand(d_logprob, in->rows > 0, "logprob")) return rc;
  if (int rc = check_operand(d_lse, false, "lse")) return rc;
  if (int rc = check_workspace(in, k, d_workspace, workspace_bytes)) return rc;
  if (in->rows == 0) return EMU_OK;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  drop_pending_error();
  over_rows(in->rows, [&](uint64_t r0, uint32_t n) {
    auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(n), dim3(kRowThreads), 0, st, l, uint32_t(k), c1, d_index, d_logprob, d_lse, r0);
    };
    if (in->dtype == EMU_BF16) launch(k_topk<bf16_t>);
    else launch(k_topk<float>);
  });
  return hip_check("emu_logits_topk launch");
}

int emu_distill(const emu_logits_t* student, const emu_teacher_t* teacher, float* d_loss, float* d_stats,
                const emu_logits_t* grad, void* d_workspace, uint64_t workspace_bytes, void* hip_stream) {
  clear_error();
  Logits li, lo{};
  float c1;
  if (int rc = check_logits(student, "student", &li)) return rc;
  if (int rc = check_teacher(teacher, student->rows, &c1)) return rc;
  if (int rc = check_operand(d_loss, student->rows > 0, "loss")) return rc;
  if (int rc = check_operand(d_stats, student->rows > 0, "stats", 16)) return rc;
  if (grad)
    if (int rc = check_output(student, grad, "grad", &lo)) return rc;
  if (int rc = check_workspace(student, 0, d_workspace, workspace_bytes)) return rc;
  if (student->rows == 0) return EMU_OK;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  drop_pending_error();
  by_types(student->dtype, grad ? grad->dtype : student->dtype, [&](auto ti, auto to) {
    over_rows(student->rows, [&](uint64_t r0, uint32_t n) {
      hipLaunchKernelGGL((k_distill<decltype(ti), decltype(to)>), dim3(n), dim3(kRowThreads), 0, st, li, lo, *teacher, c1,
                         d_loss, reinterpret_cast<float4*>(d_stats), grad != nullptr, r0);
    });
  });
  return hip_check("emu_distill launch");
}

int emu_distill_backward(const emu_logits_t* student, const emu_teacher_t* teacher, const float* d_stats,
                         const emu_logits_t* grad, void* d_workspace, uint64_t workspace_bytes, void* hip_stream) {
  clear_error();
  Logits li, lo;
  float c1;
  if (int rc = check_logits(student, "student", &li)) return rc;
  if (int rc = check_teacher(teacher, student->rows, &c1)) return rc;
  if (int rc = check_operand(d_stats, student->rows > 0, "stats", 16)) return rc;
  if (int rc = check_output(student, grad, "grad", &lo)) return rc;
  if (int rc = check_workspace(student, 0, d_workspace, workspace_bytes)) return rc;
  if (student->rows == 0) return EMU_OK;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  drop_pending_error();
  by_types(student->dtype, grad->dtype, [&](auto ti, auto to) {
    over_rows(student->rows, [&](uint64_t r0, uint32_t n) {
      hipLaunchKernelGGL((k_distill_backward<decltype(ti), decltype(to)>), dim3(n), dim3(kRowThreads), 0, st, li, lo,
                         *teacher, c1, reinterpret_cast<const float4*>(d_stats), r0);
    });
  });
  return hip_check("emu_distill_backward launch");
}

}  // extern "C"
