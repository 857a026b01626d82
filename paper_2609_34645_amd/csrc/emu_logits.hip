// Operators on the logits of a vocab-parallel LM head (include/emu.h): constraints ahead of sampling, the
// k largest log-probabilities, distillation with its gradient. Every row is read once (twice for a loss with its
// gradient), in 16-byte vectors; every reduction runs over global columns in a fixed order, so that no result
// depends on how the shards cut them.
#include <cmath>

#include "emu_internal.h"

namespace emu {

constexpr int kMaxShards = 64;
constexpr int32_t kMaxVocab = 1 << 20;
constexpr int32_t kMaxTokens = 1 << 28;  // of one row's history: byte offsets stay below 2^32
constexpr int kMaxTop = 64;        // entries of emu_logits_topk: one per lane of a wave
constexpr int kMaxTeacher = 256;   // entries of a teacher's row
constexpr uint32_t kMaxSplits = 64;            // workgroups that share a row: one partial result per lane
constexpr uint32_t kRowsPerLaunch = 1u << 21;  // a grid's work-items stay below 2^32
constexpr float kInf = __builtin_inff();
constexpr float kLog2e = 1.44269504f;

// A logits set on the device: row r's columns [t * cols, (t + 1) * cols) lie at p[t] + r * row_bytes.
struct Logits {
  uint8_t* p[kMaxShards];
  uint64_t row_bytes;
  uint32_t V, Vp, cols;
  uint32_t recip;  // floor((2^32 - 1) / cols)
};

// v / cols: the product's high half is the quotient or one less.
__device__ __forceinline__ uint32_t shard_of(const Logits& l, uint32_t v) {
  const uint32_t t = __umulhi(v, l.recip);
  return v - t * l.cols >= l.cols ? t + 1 : t;
}

// ------------------------------------------------------------------------------------------------
// rows in vectors
// ------------------------------------------------------------------------------------------------
// A lane holds 16 bytes, kE<T> columns from a multiple of kE<T> on; a wave's tile is 64 such vectors, 1 KB, and a
// wave takes U neighbouring tiles at a time. Columns are counted over the whole vocabulary, so which lane
// adds up which column, and in which order, does not depend on the shards. Where the U tiles lie inside one
// shard (all but one stretch per shard do), they are U loads from one scalar base at any element alignment;
// elsewhere every lane finds its own shard, and a vector across a shard's end is put together by element.

typedef uint16_t bf16_t;  // bits
template <typename T> constexpr uint32_t kE = 16 / sizeof(T);
template <typename T> constexpr uint32_t kTile = 64 * kE<T>;
template <typename T> constexpr uint32_t kMinusInf = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;

template <typename T>
__device__ __forceinline__ const T* column(const Logits& l, uint64_t row_off, uint32_t v) {
  const uint32_t t = shard_of(l, v);
  return reinterpret_cast<const T*>(l.p[t] + row_off) + (v - t * l.cols);
}
__device__ __forceinline__ float widen(bf16_t x) { return __uint_as_float(uint32_t(x) << 16); }
__device__ __forceinline__ float widen(float x) { return x; }

__device__ __forceinline__ void unpack(v4u x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(x[i] << 16);
    f[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(v4u x, float (&f)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(x[i]);
}

// Two values rounded to bf16, nearest even; NaNs stay NaN.
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){a, b}, b2));
}

// The vector of columns [v, v + kE) at a shard's or the vocabulary's end; -infinity from V on.
template <typename T, int POL>
__device__ v4u load_edge(const Logits& l, uint64_t row_off, uint32_t v) {
  v4u x = {kMinusInf<T>, kMinusInf<T>, kMinusInf<T>, kMinusInf<T>};
  if (v >= l.V) return x;
  const uint32_t t = shard_of(l, v), lo = v - t * l.cols;
  if (lo + kE<T> <= l.cols && v + kE<T> <= l.V) return ld16_any<POL>(l.p[t] + row_off, lo * uint32_t(sizeof(T)));
#pragma unroll
  for (uint32_t e = 0; e < kE<T>; ++e) {
    if (v + e >= l.V) break;
    const T y = *column<T>(l, row_off, v + e);
    if constexpr (sizeof(T) == 2) x[e / 2] = e % 2 ? (x[e / 2] & 0xffffu) | uint32_t(y) << 16 : (x[e / 2] & 0xffff0000u) | y;
    else x[e] = __float_as_uint(y);
  }
  return x;
}

// The wave's U tiles from column c on (the same c in every lane).
template <typename T, int U, int POL>
__device__ __forceinline__ void load_tiles(const Logits& l, uint64_t row_off, uint32_t c, v4u (&x)[U]) {
  const uint32_t lane = threadIdx.x & 63, t = shard_of(l, c), lo = c - t * l.cols;
  if (lo + U * kTile<T> <= l.cols && c + U * kTile<T> <= l.V) {
    const uint8_t* base = l.p[t] + row_off + uint64_t(lo) * sizeof(T);
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = ld16_any<POL>(base, lane * 16 + u * 1024);
  } else {
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = load_edge<T, POL>(l, row_off, c + u * kTile<T> + lane * kE<T>);
  }
}

// N values to TO at p (element-aligned).
template <typename TO, int POL, uint32_t N>
__device__ __forceinline__ void store_values(uint8_t* base, uint32_t off, const float (&f)[N]) {
  if constexpr (sizeof(TO) == 4) {
#pragma unroll
    for (uint32_t i = 0; i < N; i += 4)
      st16_any<POL>(base, off + i * 4, (v4u){__float_as_uint(f[i]), __float_as_uint(f[i + 1]), __float_as_uint(f[i + 2]), __float_as_uint(f[i + 3])});
  } else if constexpr (N == 8) {
    st16_any<POL>(base, off, (v4u){pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])});
  } else {
    st8_any<POL>(base, off, (v2u){pack2(f[0], f[1]), pack2(f[2], f[3])});
  }
}

// Columns [v, v + N) of an output row at a shard's or the padded vocabulary's end.
template <typename TO, int POL, uint32_t N>
__device__ void store_edge(const Logits& l, uint64_t row_off, uint32_t v, const float (&f)[N]) {
  if (v >= l.Vp) return;
  const uint32_t t = shard_of(l, v), lo = v - t * l.cols;
  if (lo + N <= l.cols) {  // shards end at Vp
    store_values<TO, POL>(l.p[t] + row_off, lo * uint32_t(sizeof(TO)), f);
    return;
  }
#pragma unroll
  for (uint32_t e = 0; e < N; ++e) {
    if (v + e >= l.Vp) break;
    TO* at = const_cast<TO*>(column<TO>(l, row_off, v + e));
    if constexpr (sizeof(TO) == 2) *at = bf16_t(pack2(f[e], f[e]));
    else *at = f[e];
  }
}

// ------------------------------------------------------------------------------------------------
// reductions in fixed trees
// ------------------------------------------------------------------------------------------------

template <typename T, typename F>
__device__ __forceinline__ T wave_reduce(T x, F f) {
#pragma unroll
  for (int n = 32; n; n >>= 1) x = f(x, __shfl_xor(x, n));
  return x;
}

// Over the workgroup's NW waves; every thread gets the result. Two barriers.
template <int NW, typename T, typename F>
__device__ __forceinline__ T block_reduce(T x, T* lds, F f) {
  x = wave_reduce(x, f);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  x = lds[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) x = f(x, lds[w]);
  return x;
}

__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ double addd(double a, double b) { return a + b; }
__device__ __forceinline__ float max3(float a, float b, float c) {  // a NaN is passed over
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// ------------------------------------------------------------------------------------------------
// softmax statistics
// ------------------------------------------------------------------------------------------------
// One pass with a running maximum. exp((x - m) / tau) = exp2(fma(x, c1, -ref)), c1 = log2(e) / tau, with the same
// rounded ref = m * c1 in every term, so that its rounding cancels: log2 of the whole sum is ref + log2(sum).
// That holds while |m * c1| < 2^20. Below, ref is cut to -2^20: such a part counts as 0 beside any ordinary
// logit (masks of the type's lowest value), and no term is a NaN by infinity - infinity. A row whose own maximum
// lies outside is summed again as exp2((x - m) * c1) (careful_sum).

constexpr float kPlainRange = 1048576.0f;

struct Running {
  float m, s;  // the largest value seen, and the sum of exp2(x * c1 - reference(m))
};

__device__ __forceinline__ float reference(float m, float c1) { return fmaxf(m * c1, -kPlainRange); }
__device__ __forceinline__ bool plain(float m, float c1) { return fabsf(m * c1) < kPlainRange; }

__device__ __forceinline__ Running joined(Running a, Running b, float c1) {
  const float m = fmaxf(a.m, b.m), ref = reference(m, c1);
  const float ea = __builtin_amdgcn_exp2f(reference(a.m, c1) - ref), eb = __builtin_amdgcn_exp2f(reference(b.m, c1) - ref);
  return {m, a.s * ea + b.s * eb};
}

__device__ __forceinline__ Running wave_joined(Running a, float c1) {
#pragma unroll
  for (int n = 32; n; n >>= 1) {
    const Running b = {__shfl_xor(a.m, n), __shfl_xor(a.s, n)};
    a = joined(a, b, c1);
  }
  return a;
}

template <int NW>
__device__ __forceinline__ Running block_joined(Running a, Running* lds, float c1) {
  a = wave_joined(a, c1);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
  __syncthreads();
  a = lds[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) a = joined(a, lds[w], c1);
  return a;
}

// U vectors of a lane.
template <int U, uint32_t E>
__device__ __forceinline__ void add_values(Running& r, const float (&f)[U][E], float c1) {
  float m = r.m;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (uint32_t e = 0; e < E; e += 2) m = max3(m, f[u][e], f[u][e + 1]);
  const float ref = reference(m, c1);
  float s = 0.0f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (uint32_t e = 0; e < E; ++e) s += __builtin_amdgcn_exp2f(fmaf(f[u][e], c1, -ref));
  r.s = r.s * __builtin_amdgcn_exp2f(reference(r.m, c1) - ref) + s;
  r.m = m;
}

// exp(m / tau) * the result is the sum of exp(x / tau) behind r, for a maximum in the plain range.
__device__ __forceinline__ float true_sum(Running r, float c1) {
  return r.s * __builtin_amdgcn_exp2f(-fmaf(r.m, c1, -reference(r.m, c1)));
}

__device__ __forceinline__ uint32_t wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Sum of exp((x - m) / tau) over the row by the whole workgroup; marked columns (a bit each from column 0 on) are
// left out.
template <typename T, int NW>
__device__ float careful_sum(const Logits& l, uint64_t row_off, float m, float c1, const int32_t* listed, int k, float* lds) {
  float s = 0.0f;
  for (uint32_t v = threadIdx.x; v < l.V; v += NW * 64) {
    const float x = widen(*column<T>(l, row_off, v));
    bool skip = x == -kInf;
    for (int j = 0; j < k; ++j) skip |= listed[j] == int32_t(v);
    if (!skip) s += __builtin_amdgcn_exp2f((x - m) * c1);
  }
  return block_reduce<NW>(s, lds, add);
}

// log(exp(m / tau) s), in 64 bits: m / tau may pass the range of fp32's product with log2(e).
__device__ __forceinline__ float log_sum_exp(float m, float s, float c1) {
  return s == 0.0f ? -kInf : float((double(m) * double(c1) + double(log2f(s))) * 0.6931471805599453);
}

// log(exp((x - m) / tau) / s), likewise.
__device__ __forceinline__ float log_prob(float x, float m, float s, float c1) {
  return x == -kInf ? -kInf : float(((double(x) - double(m)) * double(c1) - double(log2f(s))) * 0.6931471805599453);
}

// The columns of workgroup `part` of the `parts` that share a row, in whole chunks of U tiles per wave.
template <typename T, int U, int NW>
__device__ __forceinline__ void part_range(uint32_t end, uint32_t part, uint32_t parts, uint32_t* c0, uint32_t* c1) {
  constexpr uint32_t kChunk = U * kTile<T>;
  const uint32_t chunks = (end + kChunk - 1) / kChunk, per = (chunks + parts - 1) / parts;
  *c0 = umin(part * per, chunks) * kChunk;
  *c1 = umin(*c0 + per * kChunk, end);
}

// ------------------------------------------------------------------------------------------------
// constraints
// ------------------------------------------------------------------------------------------------
// A workgroup has kSlice columns of one row. It counts the slice's tokens in LDS (integer atomics: any order gives
// the same counts), marks the columns that anything concerns in a bit each, and passes over its columns once: a
// vector whose mark and mask bytes are plain is copied, one that the mask forbids whole is not read.

constexpr int kConstrainThreads = 256;
constexpr uint32_t kSlice = 8192;
constexpr uint32_t kSeen = 1u << 31, kBiased = 1u << 30, kCountBits = kBiased - 1;
constexpr int kListed = 512;  // biases of a slice held in LDS, in list order

template <typename TI, typename TO>
__global__ __launch_bounds__(kConstrainThreads) void k_constrain(Logits in, Logits out, emu_constraints_t c, bool in_place,
                                                                 uint64_t row0) {
  __shared__ uint32_t count[kSlice];
  __shared__ uint32_t mark[kSlice / 32];
  __shared__ int32_t list_col[kListed];
  __shared__ float list_value[kListed];
  __shared__ uint32_t wave_n[kConstrainThreads / 64];
  constexpr int U = 4;
  constexpr uint32_t E = kE<TI>, kChunk = U * kTile<TI>;
  const uint64_t r = row0 + blockIdx.x;
  const uint32_t c0 = blockIdx.y * kSlice, c1 = umin(c0 + kSlice, in.Vp), lane = threadIdx.x & 63;
  const bool concerns = c.tokens || c.bias_first;
  int64_t b0 = 0, b1 = 0;
  uint32_t n_listed = 0;
  if (concerns) {
    for (uint32_t i = threadIdx.x * 4; i < kSlice; i += kConstrainThreads * 4) *reinterpret_cast<v4u*>(count + i) = (v4u){0, 0, 0, 0};
    for (uint32_t i = threadIdx.x; i < kSlice / 32; i += kConstrainThreads) mark[i] = 0;
    __syncthreads();
  }
  if (c.tokens) {
    const int32_t* tok = c.tokens + r * c.tokens_stride;
    const int32_t n = min(max(c.seq_len[r], 0), c.tokens_cols);
    const int32_t prompt = c.prompt_len ? c.prompt_len[r] : 0;
    auto take = [&](uint32_t v, int32_t i) {
      const uint32_t at = v - c0;
      if (at < kSlice && v < in.V) {
        if (i >= prompt) atomicAdd(&count[at], 1u);
        atomicOr(&count[at], kSeen);
        atomicOr(&mark[at / 32], 1u << (at % 32));
      }
    };
    const int32_t whole = n & ~3;
    for (int32_t i = threadIdx.x * 4; i < whole; i += kConstrainThreads * 4) {
      const v4u v = ld16_any<POL_PLAIN>(reinterpret_cast<const uint8_t*>(tok), uint32_t(i) * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) take(v[e], i + e);
    }
    if (int32_t(threadIdx.x) < n - whole) take(uint32_t(tok[whole + threadIdx.x]), whole + threadIdx.x);
  }
  if (c.bias_first) {
    b0 = min(max(int64_t(c.bias_first[r]), int64_t(0)), c.n_bias);
    b1 = min(max(int64_t(c.bias_first[r + 1]), int64_t(0)), c.n_bias);
    for (int64_t i0 = b0; i0 < b1; i0 += kConstrainThreads) {
      const int64_t i = i0 + threadIdx.x;
      const uint32_t v = i < b1 ? uint32_t(c.bias_token[i]) : ~0u, at = v - c0;
      const bool here = at < kSlice && v < in.V;
      const uint64_t lanes = __ballot(here);
      if (lane == 0) wave_n[threadIdx.x >> 6] = __popcll(lanes);
      __syncthreads();
      uint32_t pos = n_listed + __popcll(lanes & ((1ull << lane) - 1));
#pragma unroll
      for (uint32_t w = 0; w < kConstrainThreads / 64; ++w) {
        if (w < (threadIdx.x >> 6)) pos += wave_n[w];
        n_listed += wave_n[w];
      }
      if (here) {
        if (pos < kListed) {
          list_col[pos] = int32_t(v);
          list_value[pos] = c.bias_value[i];
        }
        atomicOr(&count[at], kBiased);
        atomicOr(&mark[at / 32], 1u << (at % 32));
      }
      __syncthreads();
    }
  }
  __syncthreads();
  const uint8_t* mask = nullptr;
  if (c.mask) {
    const int64_t which = c.mask_row ? int64_t(c.mask_row[r]) : int64_t(r);
    if (which >= 0 && which < c.n_masks) mask = reinterpret_cast<const uint8_t*>(c.mask + which * c.mask_stride);
  }
  const float theta = c.repetition ? c.repetition[r] : 1.0f;
  const float af = c.frequency ? c.frequency[r] : 0.0f, ap = c.presence ? c.presence[r] : 0.0f;
  auto concerned = [&](float x, uint32_t v) {
    const uint32_t n = count[v - c0];
    if (n & kSeen) {
      x = x > 0.0f ? x / theta : x * theta;
      if (n & kCountBits) x -= af * float(n & kCountBits) + ap;
    }
    if (n & kBiased) {
      float sum = 0.0f;
      if (n_listed <= kListed) {
        for (uint32_t i = 0; i < n_listed; ++i)
          if (list_col[i] == int32_t(v)) sum += list_value[i];
      } else {
        for (int64_t i = b0; i < b1; ++i)
          if (c.bias_token[i] == int32_t(v)) sum += c.bias_value[i];
      }
      x += sum;
    }
    return x;
  };
  constexpr uint32_t kAll = (1u << E) - 1;
  const uint64_t ri = r * in.row_bytes, ro = r * out.row_bytes;
  for (uint32_t cc = c0 + wave_id() * kChunk; cc < c1; cc += kConstrainThreads / 64 * kChunk) {
    uint32_t allowed[U], marked[U];
    bool kept[U];  // in place and unchanged
    v4u x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t v = cc + u * kTile<TI> + lane * E;
      allowed[u] = kAll;
      if (mask && v < in.V) allowed[u] = (mask[v / 8] >> (v % 8)) & kAll;
      marked[u] = concerns ? (reinterpret_cast<const uint8_t*>(mark)[(v - c0) / 8] >> (v % 8)) & kAll : 0;
      kept[u] = in_place && !marked[u] && allowed[u] == kAll && v + E <= in.V;
    }
    const uint32_t t = shard_of(in, cc), lo = cc - t * in.cols;
    const bool inside = lo + kChunk <= in.cols && cc + kChunk <= in.V;
    const uint8_t* bi = in.p[t] + ri + uint64_t(lo) * sizeof(TI);
    uint8_t* bo = out.p[t] + ro + uint64_t(lo) * sizeof(TO);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      x[u] = (v4u){kMinusInf<TI>, kMinusInf<TI>, kMinusInf<TI>, kMinusInf<TI>};
      if (allowed[u] && !kept[u]) {
        if (inside) x[u] = ld16_any<POL_NT>(bi, lane * 16 + u * 1024);
        else x[u] = load_edge<TI, POL_NT>(in, ri, cc + u * kTile<TI> + lane * E);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t v = cc + u * kTile<TI> + lane * E;
      float f[E];
      unpack(x[u], f);
      const uint32_t touched = marked[u] & allowed[u];
      if (touched) {
#pragma unroll
        for (uint32_t e = 0; e < E; ++e)
          if ((touched >> e) & 1u) f[e] = concerned(f[e], v + e);
      }
      if (allowed[u] != kAll) {
#pragma unroll
        for (uint32_t e = 0; e < E; ++e)
          if (!((allowed[u] >> e) & 1u)) f[e] = -kInf;
      }
      if (kept[u]) continue;
      if (inside) store_values<TO, POL_NT>(bo, (lane * E + u * kTile<TI>) * uint32_t(sizeof(TO)), f);
      else if (v < c1) store_edge<TO, POL_NT>(out, ro, v, f);
    }
  }
}

// ------------------------------------------------------------------------------------------------
// the k largest
// ------------------------------------------------------------------------------------------------
// Every logit has a key whose order is the result's: the value, then the lower column. Each wave keeps its k
// largest keys sorted, one per lane, beside the softmax statistics of the same pass. Logits above the k-th are
// collected in LDS and merged in 64 at a time (a bitonic sort across the lanes and one merge); the k-th key is
// shared with the row's other waves, so that a row admits about k log(V) logits. The first bound is the k-th
// largest of the lanes' maxima over the wave's first tiles. The result does not depend on when a wave sees a
// shared bound: a bound only ever drops keys that k others beat.

__device__ __forceinline__ uint64_t top_key(float x, uint32_t v) {  // 0: never chosen
  if (!(x > -kInf)) return 0;
  const uint32_t u = __float_as_uint(x + 0.0f);  // -0 becomes 0
  const uint32_t order = u & 0x80000000u ? ~u : u | 0x80000000u;
  return uint64_t(order) << 32 | uint32_t(~v);
}
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t order = uint32_t(key >> 32);
  return key == 0 ? -kInf : __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order);
}
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t min64(uint64_t a, uint64_t b) { return a < b ? a : b; }
__device__ __forceinline__ uint64_t lane_key(uint64_t x, uint32_t lane) {  // the same lane everywhere
  return uint64_t(__builtin_amdgcn_readlane(uint32_t(x >> 32), lane)) << 32 | uint32_t(__builtin_amdgcn_readlane(uint32_t(x), lane));
}

__device__ __forceinline__ uint64_t sorted(uint64_t x) {  // across the wave, largest in lane 0
  const uint32_t lane = threadIdx.x & 63;
#pragma unroll
  for (uint32_t k = 2; k <= 64; k <<= 1) {
#pragma unroll
    for (uint32_t j = k >> 1; j; j >>= 1) {
      const uint64_t y = __shfl_xor((unsigned long long)x, j);
      x = ((lane & j) == 0) == ((lane & k) == 0) ? max64(x, y) : min64(x, y);
    }
  }
  return x;
}
__device__ __forceinline__ uint64_t merged(uint64_t a, uint64_t b) {  // the 64 largest of two sorted waves, sorted
  const uint32_t lane = threadIdx.x & 63;
  uint64_t x = max64(a, __shfl((unsigned long long)b, 63 - lane));
#pragma unroll
  for (uint32_t j = 32; j; j >>= 1) {
    const uint64_t y = __shfl_xor((unsigned long long)x, j);
    x = (lane & j) == 0 ? max64(x, y) : min64(x, y);
  }
  return x;
}

// What the wave's lanes wrote to LDS is what its lanes read from here on.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int NW>
struct TopLds {
  uint64_t fresh[NW][128];       // a wave's collected keys
  uint64_t list[NW][64];
  unsigned long long bound;      // the largest k-th key of any wave
  Running run[NW];
  float sum[NW];
};

// The waves' lists to one, in wave 0.
template <int NW>
__device__ __forceinline__ uint64_t block_merged(uint64_t best, TopLds<NW>& t) {
  const uint32_t lane = threadIdx.x & 63, w = wave_id();
  t.list[w][lane] = best;
  __syncthreads();
  if (w == 0)
    for (int i = 1; i < NW; ++i) best = merged(best, t.list[i][lane]);
  return best;
}

// Lane j < k of one wave: the row's j-th.
__device__ __forceinline__ void write_top(uint64_t key, uint32_t k, float m, float s, float c1, int32_t* index, float* logprob,
                                          float* lse, uint64_t r) {
  const uint32_t lane = threadIdx.x & 63;
  if (lane < k) {
    index[r * k + lane] = key ? int32_t(~uint32_t(key)) : -1;
    logprob[r * k + lane] = s != s ? s : key ? log_prob(key_value(key), m, s, c1) : -kInf;
  }
  if (lane == 0 && lse) lse[r] = log_sum_exp(m, s, c1);
}

template <typename T, int NW>
__device__ __forceinline__ float row_sum(const Logits& l, uint64_t row_off, Running a, float c1, float* lds) {
  if (plain(a.m, c1)) return true_sum(a, c1);
  if (a.m == -kInf) return a.s;
  return careful_sum<T, NW>(l, row_off, a.m, c1, nullptr, 0, lds);
}

constexpr int kTopWaves = 4;
constexpr int kTopU = 4;

// Grid: rows, parts. One part: the row's result. More: the part's statistics and keys, for k_topk_join.
template <typename T>
__global__ __launch_bounds__(kTopWaves * 64) void k_topk(Logits in, uint32_t k, float c1, int32_t* index, float* logprob,
                                                         float* lse, Running* part_run, uint64_t* part_keys, uint64_t row0) {
  constexpr int NW = kTopWaves, U = kTopU;
  constexpr uint32_t E = kE<T>, kChunk = U * kTile<T>;
  __shared__ TopLds<NW> t;
  const uint64_t r = row0 + blockIdx.x, off = r * in.row_bytes;
  const uint32_t lane = threadIdx.x & 63, w = wave_id();
  uint32_t c0, end;
  part_range<T, U, NW>(in.V, blockIdx.y, gridDim.y, &c0, &end);
  if (threadIdx.x == 0) t.bound = 0;
  __syncthreads();
  uint64_t best = 0, bound = 0;  // every key in the row's result is >= bound
  uint32_t n = 0;                // collected
  auto flush = [&](uint32_t have) {
    wave_sync();
    const uint64_t x = sorted(lane < have ? t.fresh[w][lane] : 0);
    best = merged(best, x);
    const uint64_t kth = lane_key(best, k - 1);
    if (lane == 0) atomicMax(&t.bound, (unsigned long long)kth);
    bound = max64(bound, kth);
  };
  Running run = {-kInf, 0.0f};
  bool first = true;
  for (uint32_t c = c0 + w * kChunk; c < end; c += NW * kChunk) {
    v4u x[U];
    load_tiles<T, U, POL_NT>(in, off, c, x);
    float f[U][E], top[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      unpack(x[u], f[u]);
      top[u] = f[u][0];
#pragma unroll
      for (uint32_t e = 1; e < E; e += 2) top[u] = e + 1 < E ? max3(top[u], f[u][e], f[u][e + 1]) : max3(top[u], f[u][e], f[u][e]);
    }
    add_values<U, E>(run, f, c1);
    if (first) {
      float m = top[0];
#pragma unroll
      for (int u = 1; u < U; ++u) m = max3(m, top[u], top[u]);
      bound = lane_key(sorted(top_key(m, ~0u)), k - 1);  // the lanes' maxima as if behind the last column
      first = false;
    }
    bound = max64(bound, lane_key(__hip_atomic_load(&t.bound, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP), 0));
    float level = key_value(bound);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (__all(top[u] < level)) continue;  // a NaN goes on
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) {
        const uint64_t key = top_key(f[u][e], c + u * kTile<T> + lane * E + e);
        const uint64_t lanes = __ballot(key > bound);
        if (!lanes) continue;
        if (key > bound) t.fresh[w][n + __popcll(lanes & ((1ull << lane) - 1))] = key;
        n += __popcll(lanes);
        if (n >= 64) {
          flush(64);
          n -= 64;
          const uint64_t left = t.fresh[w][64 + lane];
          wave_sync();
          t.fresh[w][lane] = left;
          wave_sync();
          level = key_value(bound);
        }
      }
    }
  }
  if (n) flush(n);
  run = block_joined<NW>(run, t.run, c1);
  best = block_merged<NW>(best, t);
  if (gridDim.y > 1) {
    const uint64_t at = (r - row0) * gridDim.y + blockIdx.y;
    if (w == 0) part_keys[at * 64 + lane] = best;
    if (threadIdx.x == 0) part_run[at] = run;
    return;
  }
  const float s = row_sum<T, NW>(in, off, run, c1, t.sum);
  if (w == 0) write_top(best, k, run.m, s, c1, index, logprob, lse, r);
}

// The parts of a row to its result.
template <typename T>
__global__ __launch_bounds__(kTopWaves * 64) void k_topk_join(Logits in, uint32_t k, float c1, int32_t* index, float* logprob,
                                                              float* lse, const Running* part_run, const uint64_t* part_keys,
                                                              uint32_t parts, uint64_t row0) {
  constexpr int NW = kTopWaves;
  __shared__ TopLds<NW> t;
  const uint64_t r = row0 + blockIdx.x, at = uint64_t(blockIdx.x) * parts;
  const uint32_t lane = threadIdx.x & 63, w = wave_id();
  const Running run = wave_joined(lane < parts ? part_run[at + lane] : Running{-kInf, 0.0f}, c1);
  uint64_t best = 0;
  for (uint32_t i = w; i < parts; i += NW) best = merged(best, part_keys[(at + i) * 64 + lane]);
  best = block_merged<NW>(best, t);
  const float s = row_sum<T, NW>(in, r * in.row_bytes, run, c1, t.sum);
  if (w == 0) write_top(best, k, run.m, s, c1, index, logprob, lse, r);
}

// ------------------------------------------------------------------------------------------------
// distillation
// ------------------------------------------------------------------------------------------------
// Where rows are many, one workgroup has a row: it scans it for the statistics, and with a gradient reads it
// again, from cache. Where they are few, several share a row: they scan a part each and leave its statistics in
// the workspace, a second kernel joins them to the row's, and the gradient goes by parts again (in place, no part
// may be written before every reader of the row is done: hence the kernel between).
// The gradient is written densely as coef * exp((z - m) / tau), and the listed columns, whose values the
// threads have kept, are written over it behind a barrier. With a tail the scan leaves out the listed
// columns (a bit each in LDS), so that a small mass outside the list is a sum of its own and no difference.

// A list of log-probabilities rounded to fp32 can miss a sum of 1 by sum p |log p| 2^-24 < 2^-20.
constexpr float kRestNoise = 0x1p-20f;
constexpr float kLeastRest = 0x1p-100f;  // below, the gradient outside the list keeps q alone

// Thread j has entry j of the row's teacher: its column (-1: none, or one that an earlier entry has), that
// column's whole probability and its logit.
struct Entry {
  int32_t col;
  float p, z;
};

template <int NW>
struct DistillLds {
  int32_t col[kMaxTeacher];
  double p[kMaxTeacher];
  double wide[NW];
  float sum[NW];
  Running run[NW];
};

// Logits are read in columns [z0, z1). rest: the mass outside the list (0 without a tail); none: without a tail nothing is listed.
template <typename T, int NW>
__device__ __forceinline__ Entry load_teacher(DistillLds<NW>& t, const emu_teacher_t& te, uint64_t r, const Logits& l, uint32_t z0, uint32_t z1, float* rest, bool* none) {
  static_assert(NW * 64 >= kMaxTeacher, "one entry per thread");
  const int j = threadIdx.x;
  Entry e = {-1, 0.0f, -kInf};
  double value = -double(kInf);
  if (j < te.k) {
    const int32_t i = te.index[r * te.index_stride + j];
    if (uint32_t(i) < l.V) {
      e.col = i;
      if (uint32_t(i) >= z0 && uint32_t(i) < z1) e.z = widen(*column<T>(l, r * l.row_bytes, i));
      value = double(te.value[r * te.value_stride + j]);
    }
  }
  double top = 0.0;
  if (!te.tail) {
    top = block_reduce<NW>(value, t.wide, [](double a, double b) { return fmax(a, b); });
    if (top == -double(kInf)) top = 0.0;
  }
  double p = e.col < 0 ? 0.0 : exp(value - top);
  const double sum = block_reduce<NW>(p, t.wide, addd);
  if (!te.tail && sum != 0.0) p /= sum;
  if (j < kMaxTeacher) {
    t.col[j] = e.col;
    t.p[j] = p;
  }
  __syncthreads();
  if (j < te.k && e.col >= 0) {
    bool first = true;
    for (int i = 0; i < te.k; ++i) {
      if (i == j || t.col[i] != e.col) continue;
      if (i < j) first = false;
      else p += t.p[i];
    }
    if (!first) e.col = -1;
    else e.p = float(p);
  }
  const float left = float(1.0 - sum);
  *rest = te.tail ? (left < 0.0f ? 0.0f : left) : 0.0f;
  *none = !te.tail && sum == 0.0;
  return e;
}

// A bit per listed column of [c0, c0 + range), range a multiple of 32.
template <int NW>
__device__ __forceinline__ void mark_listed(uint32_t* bits, uint32_t c0, uint32_t range, const emu_teacher_t& te, uint64_t r, uint32_t V) {
  for (uint32_t i = threadIdx.x; i < range / 32; i += NW * 64) bits[i] = 0;
  __syncthreads();
  if (int(threadIdx.x) < te.k) {
    const uint32_t v = uint32_t(te.index[r * te.index_stride + threadIdx.x]), at = v - c0;
    if (v < V && at < range) atomicOr(&bits[at / 32], 1u << (at % 32));
  }
  __syncthreads();
}

// The statistics of columns [c0, end), without the marked ones if TAIL.
template <typename T, int U, int NW, bool TAIL, int POL>
__device__ __forceinline__ Running scan(const Logits& l, uint64_t off, uint32_t c0, uint32_t end, float c1, const uint32_t* bits) {
  constexpr uint32_t E = kE<T>, kChunk = U * kTile<T>;
  const uint32_t lane = threadIdx.x & 63;
  Running run = {-kInf, 0.0f};
  for (uint32_t c = c0 + wave_id() * kChunk; c < end; c += NW * kChunk) {
    v4u x[U];
    load_tiles<T, U, POL>(l, off, c, x);
    float f[U][E];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      unpack(x[u], f[u]);
      if constexpr (TAIL) {
        const uint32_t at = c - c0 + u * kTile<T> + lane * E;
        const uint32_t hit = (reinterpret_cast<const uint8_t*>(bits)[at / 8] >> (at % 8)) & ((1u << E) - 1);
        if (hit) {
#pragma unroll
          for (uint32_t e = 0; e < E; ++e)
            if ((hit >> e) & 1u) f[u][e] = -kInf;
        }
      }
    }
    add_values<U, E>(run, f, c1);
  }
  return run;
}

struct Stats {
  float lse, factor, m, s;
};

// From the scan of a whole row: its statistics and loss, in every thread.
template <typename T, int NW, bool TAIL>
__device__ __forceinline__ Stats finish(const Logits& l, uint64_t off, Running run, const Entry& e, float rest, int k, float c1,
                                        DistillLds<NW>& t, float* loss) {
  Stats st;
  float s = plain(run.m, c1) ? true_sum(run, c1)
            : run.m == -kInf ? run.s
                             : careful_sum<T, NW>(l, off, run.m, c1, t.col, TAIL ? k : 0, t.sum);
  st.factor = 1.0f;
  float rest_loss = 0.0f;
  st.m = run.m;
  st.s = s;
  if constexpr (TAIL) {
    const float z = e.col >= 0 ? e.z : -kInf;
    st.m = fmaxf(run.m, block_reduce<NW>(z, t.sum, [](float a, float b) { return fmaxf(a, b); }));
    const float m = st.m == -kInf ? 0.0f : st.m;
    const float inside = block_reduce<NW>(e.col >= 0 ? __builtin_amdgcn_exp2f((z - m) * c1) : 0.0f, t.sum, add);
    st.s = (s == 0.0f ? 0.0f : s * __builtin_amdgcn_exp2f((run.m - m) * c1)) + inside;
    const float log_q = s == 0.0f ? -kInf
                                  : float(((double(run.m) - double(st.m)) * double(c1) + double(log2f(s)) - double(log2f(st.s))) * 0.6931471805599453);
    if (rest != 0.0f && (s != 0.0f || rest >= kRestNoise)) rest_loss = rest * (logf(rest) - log_q);
    const float q = expf(log_q);
    if (!(q < kLeastRest)) st.factor = 1.0f - rest / q;
  }
  st.lse = log_sum_exp(st.m, st.s, c1);
  const float part = e.p != 0.0f ? e.p * (logf(e.p) - log_prob(e.z, st.m, st.s, c1)) : 0.0f;
  *loss = block_reduce<NW>(part, t.sum, add) + rest_loss;
  return st;
}

// Dense: coef * exp((z - m) / tau) over columns [c0, end) of the padded row, 0 behind V. ZERO: 0, and nothing is read.
enum Dense { PLAIN_RANGE, ANY_RANGE, ZERO };
template <typename TI, typename TO, int U, int NW, int POL, Dense KIND>
__device__ __forceinline__ void dense_gradient(const Logits& in, const Logits& out, uint64_t r, uint32_t c0, uint32_t end, float m,
                                               float c1, float coef) {
  constexpr uint32_t E = kE<TI>, kChunk = U * kTile<TI>;
  const uint32_t lane = threadIdx.x & 63;
  const uint64_t ri = r * in.row_bytes, ro = r * out.row_bytes;
  const float ref = reference(m, c1);
  for (uint32_t c = c0 + wave_id() * kChunk; c < end; c += NW * kChunk) {
    v4u x[U];
    if constexpr (KIND != ZERO) load_tiles<TI, U, POL>(in, ri, c, x);
    const uint32_t t = shard_of(out, c), lo = c - t * out.cols;
    const bool inside = lo + kChunk <= out.cols && c + kChunk <= out.V;
    uint8_t* base = out.p[t] + ro + uint64_t(lo) * sizeof(TO);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[E];
      if constexpr (KIND != ZERO) unpack(x[u], f);
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) {
        if constexpr (KIND == ZERO) f[e] = 0.0f;
        else f[e] = __builtin_amdgcn_exp2f(KIND == PLAIN_RANGE ? fmaf(f[e], c1, -ref) : (f[e] - m) * c1) * coef;
      }
      const uint32_t v = c + u * kTile<TI> + lane * E;
      if (inside) {
        store_values<TO, POL_NT>(base, (u * kTile<TI> + lane * E) * uint32_t(sizeof(TO)), f);
      } else if (v < end) {
#pragma unroll
        for (uint32_t e = 0; e < E; ++e)
          if (v + e >= in.V) f[e] = 0.0f;
        store_edge<TO, POL_NT>(out, ro, v, f);
      }
    }
  }
}

// The listed columns of [c0, end), behind the dense gradient.
template <typename TO>
__device__ __forceinline__ void listed_gradient(const Logits& out, uint64_t r, uint32_t c0, uint32_t end, const Entry& e, Stats st,
                                                float c1, float scale) {
  __syncthreads();
  if (e.col >= 0 && uint32_t(e.col) >= c0 && uint32_t(e.col) < end) {
    const float q = st.s == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((e.z - st.m) * c1) / st.s;
    const float d = (q - e.p) * scale;
    TO* at = const_cast<TO*>(column<TO>(out, r * out.row_bytes, e.col));
    if constexpr (sizeof(TO) == 2) *at = bf16_t(pack2(d, d));
    else *at = d;
  }
}

// Row r's gradient over [c0, end), from its statistics.
template <typename TI, typename TO, int U, int NW, int POL>
__device__ __forceinline__ void row_gradient(const Logits& in, const Logits& out, uint64_t r, uint32_t c0, uint32_t end, const Entry& e,
                                             Stats st, float c1, float w, bool none) {
  const float scale = w * (c1 * 0.69314718f);  // w / tau
  const bool dead = w == 0.0f || none;
  if (dead || st.s == 0.0f) {
    dense_gradient<TI, TO, U, NW, POL, ZERO>(in, out, r, c0, end, st.m, c1, 0.0f);
  } else if (plain(st.m, c1)) {
    const float one = __builtin_amdgcn_exp2f(-fmaf(st.m, c1, -reference(st.m, c1)));  // exp2(ref - m * c1)
    dense_gradient<TI, TO, U, NW, POL, PLAIN_RANGE>(in, out, r, c0, end, st.m, c1, scale * st.factor * (one / st.s));
  } else {
    dense_gradient<TI, TO, 1, NW, POL, ANY_RANGE>(in, out, r, c0, end, st.m, c1, scale * st.factor / st.s);
  }
  if (!dead) listed_gradient<TO>(out, r, c0, end, e, st, c1, scale);
}

__device__ __forceinline__ void write_row(float* loss, float4* stats, uint64_t r, float value, Stats st) {
  if (threadIdx.x == 0) {
    loss[r] = value;
    stats[r] = make_float4(st.lse, st.factor, st.m, st.s);
  }
}
constexpr Stats kSkipped = {__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};

constexpr int kScanU = 4;

// One workgroup per row.
template <typename TI, typename TO, int NW, bool TAIL, bool GRAD>
__global__ __launch_bounds__(NW * 64) void k_distill(Logits in, Logits grad, emu_teacher_t te, float c1, float* loss, float4* stats, uint64_t row0) {
  extern __shared__ uint32_t bits[];
  __shared__ DistillLds<NW> t;
  const uint64_t r = row0 + blockIdx.x;
  const float w = te.weight ? te.weight[r] : 1.0f;
  Entry e = {-1, 0.0f, -kInf};
  Stats st = kSkipped;
  bool none = false;
  if (w != 0.0f) {
    float rest, value;
    e = load_teacher<TI, NW>(t, te, r, in, 0, in.V, &rest, &none);
    if constexpr (TAIL) mark_listed<NW>(bits, 0, (in.V + kScanU * kTile<TI> - 1) / (kScanU * kTile<TI>) * (kScanU * kTile<TI>), te, r, in.V);
    const Running run = block_joined<NW>(scan<TI, kScanU, NW, TAIL, GRAD ? POL_PLAIN : POL_NT>(in, r * in.row_bytes, 0, in.V, c1, bits), t.run, c1);
    st = finish<TI, NW, TAIL>(in, r * in.row_bytes, run, e, rest, te.k, c1, t, &value);
    write_row(loss, stats, r, value * w, st);
  } else {
    write_row(loss, stats, r, 0.0f, st);
  }
  if constexpr (GRAD) row_gradient<TI, TO, kScanU, NW, POL_NT>(in, grad, r, 0, in.Vp, e, st, c1, w, none);
}

// Several workgroups per row: a part's statistics.
template <typename TI, int NW, bool TAIL>
__global__ __launch_bounds__(NW * 64) void k_distill_scan(Logits in, emu_teacher_t te, float c1, Running* part, uint64_t row0) {
  extern __shared__ uint32_t bits[];
  __shared__ Running run[NW];
  const uint64_t r = row0 + blockIdx.x;
  if (te.weight && te.weight[r] == 0.0f) return;
  uint32_t c0, end;
  part_range<TI, kScanU, NW>(in.V, blockIdx.y, gridDim.y, &c0, &end);
  if constexpr (TAIL) mark_listed<NW>(bits, c0, (end - c0 + kScanU * kTile<TI> - 1) / (kScanU * kTile<TI>) * (kScanU * kTile<TI>), te, r, in.V);
  const Running a = block_joined<NW>(scan<TI, kScanU, NW, TAIL, POL_PLAIN>(in, r * in.row_bytes, c0, end, c1, bits), run, c1);
  if (threadIdx.x == 0) part[uint64_t(blockIdx.x) * gridDim.y + blockIdx.y] = a;
}

// The row's statistics and loss from its parts'.
template <typename T, int NW, bool TAIL>
__global__ __launch_bounds__(NW * 64) void k_distill_join(Logits in, emu_teacher_t te, float c1, float* loss, float4* stats,
                                                          const Running* part, uint32_t parts, uint64_t row0) {
  __shared__ DistillLds<NW> t;
  const uint64_t r = row0 + blockIdx.x;
  const uint32_t lane = threadIdx.x & 63;
  const float w = te.weight ? te.weight[r] : 1.0f;
  if (w == 0.0f) return write_row(loss, stats, r, 0.0f, kSkipped);
  float rest, value;
  bool none;
  const Entry e = load_teacher<T, NW>(t, te, r, in, 0, in.V, &rest, &none);
  const Running run = wave_joined(lane < parts ? part[uint64_t(blockIdx.x) * parts + lane] : Running{-kInf, 0.0f}, c1);
  const Stats st = finish<T, NW, TAIL>(in, r * in.row_bytes, run, e, rest, te.k, c1, t, &value);
  write_row(loss, stats, r, value * w, st);
}

// The gradient of a row, or of a part of it, from the row's statistics.
template <typename TI, typename TO, int NW>
__global__ __launch_bounds__(NW * 64) void k_distill_backward(Logits in, Logits grad, emu_teacher_t te, float c1, const float4* stats, uint64_t row0) {
  __shared__ DistillLds<NW> t;
  const uint64_t r = row0 + blockIdx.x;
  const float w = te.weight ? te.weight[r] : 1.0f;
  uint32_t c0, end;
  part_range<TI, kScanU, NW>(in.Vp, blockIdx.y, gridDim.y, &c0, &end);
  Entry e = {-1, 0.0f, -kInf};
  Stats st = kSkipped;
  bool none = false;
  if (w != 0.0f) {
    float rest;
    e = load_teacher<TI, NW>(t, te, r, in, c0, end, &rest, &none);
    const float4 f = stats[r];
    st = {f.x, f.y, f.z, f.w};
  }
  row_gradient<TI, TO, kScanU, NW, POL_NT>(in, grad, r, c0, end, e, st, c1, w, none);
}

// How many workgroups share a row: as many as fill the device with `wanted` workgroups, each with at least a chunk
// per wave, and so many that a part's marks fit in LDS.
constexpr uint32_t kMarked = 1u << 18;  // columns
static uint32_t row_parts(const emu_logits_t* l, uint32_t V, int waves, int64_t wanted) {
  const uint32_t unit = uint32_t(waves) * 4 * (l->dtype == EMU_BF16 ? kTile<bf16_t> : kTile<float>);
  const uint32_t most = std::min((V + unit - 1) / unit, kMaxSplits);
  const int64_t want = l->rows ? (wanted + l->rows - 1) / l->rows : 1;
  return std::max(uint32_t(std::min<int64_t>(want, most)), (V + kMarked - 1) / kMarked);
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
  out->recip = ~0u / out->cols;
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

// f(element) for a dtype.
template <typename F>
static void by_type(int32_t dtype, F f) {
  dtype == EMU_BF16 ? f(bf16_t()) : f(float());
}

// f(input element, output element) for the two dtypes.
template <typename F>
static void by_types(int32_t in, int32_t out, F f) {
  if (in == EMU_BF16) out == EMU_BF16 ? f(bf16_t(), bf16_t()) : f(bf16_t(), float());
  else out == EMU_BF16 ? f(float(), bf16_t()) : f(float(), float());
}

constexpr int kPartWaves = 4;  // of a workgroup that has a part of a row
constexpr int kRowWaves = 8;   // of one that has a row

static uint32_t topk_parts(const emu_logits_t* l, uint32_t V) { return row_parts(l, V, kTopWaves, 1024); }
static uint32_t distill_parts(const emu_logits_t* l, uint32_t V) { return row_parts(l, V, kPartWaves, l->rows < 256 ? 1024 : 1); }
static uint32_t backward_parts(const emu_logits_t* l, uint32_t V) { return row_parts(l, V, kPartWaves, 2048); }

template <typename TI>
static void launch_backward(TI, int32_t dtype, uint32_t n, uint32_t parts, hipStream_t st, const Logits& li, const Logits& lo,
                            const emu_teacher_t& te, float c1, const float4* stats, uint64_t r0) {
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(n, parts), dim3(kPartWaves * 64), 0, st, li, lo, te, c1, stats, r0);
  };
  if (dtype == EMU_BF16) launch(k_distill_backward<TI, bf16_t, kPartWaves>);
  else launch(k_distill_backward<TI, float, kPartWaves>);
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
  const uint64_t rows = uint64_t(std::min<int64_t>(logits->rows, kRowsPerLaunch));
  const uint32_t parts = k ? topk_parts(logits, l.V) : distill_parts(logits, l.V);
  *bytes = parts == 1 ? 0 : rows * parts * (sizeof(Running) + (k ? 64 * sizeof(uint64_t) : 0));
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
    if (c->tokens_cols > kMaxTokens) return fail(EMU_ERR_UNSUPPORTED, "token rows of %d, at most %d", c->tokens_cols, kMaxTokens);
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
  const bool in_place = out->shards[0] == in->shards[0];
  drop_pending_error();
  by_types(in->dtype, out->dtype, [&](auto ti, auto to) {
    over_rows(in->rows, [&](uint64_t r0, uint32_t n) {
      hipLaunchKernelGGL((k_constrain<decltype(ti), decltype(to)>), dim3(n, (li.Vp + kSlice - 1) / kSlice),
                         dim3(kConstrainThreads), 0, st, li, lo, *c, in_place, r0);
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
  const uint32_t parts = topk_parts(in, l.V);
  by_type(in->dtype, [&](auto ti) {
    over_rows(in->rows, [&](uint64_t r0, uint32_t n) {
      uint64_t* keys = static_cast<uint64_t*>(d_workspace);
      Running* run = parts == 1 ? nullptr : reinterpret_cast<Running*>(keys + uint64_t(n) * parts * 64);
      hipLaunchKernelGGL((k_topk<decltype(ti)>), dim3(n, parts), dim3(kTopWaves * 64), 0, st, l, uint32_t(k), c1, d_index,
                         d_logprob, d_lse, run, keys, r0);
      if (parts > 1)
        hipLaunchKernelGGL((k_topk_join<decltype(ti)>), dim3(n), dim3(kTopWaves * 64), 0, st, l, uint32_t(k), c1, d_index,
                           d_logprob, d_lse, run, keys, parts, r0);
    });
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
  const uint32_t parts = distill_parts(student, li.V);
  float4* stats = reinterpret_cast<float4*>(d_stats);
  Running* part = static_cast<Running*>(d_workspace);
  by_type(student->dtype, [&](auto ti) {
    using TI = decltype(ti);
    constexpr uint32_t kChunk = kScanU * kTile<TI>;
    const uint32_t chunks = (li.V + kChunk - 1) / kChunk;
    const size_t marks = teacher->tail ? size_t((chunks + parts - 1) / parts) * kChunk / 8 : 0;
    over_rows(student->rows, [&](uint64_t r0, uint32_t n) {
      auto by_tail = [&](auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        if (parts > 1) {
          hipLaunchKernelGGL((k_distill_scan<TI, kPartWaves, TAIL>), dim3(n, parts), dim3(kPartWaves * 64), marks, st, li, *teacher, c1, part, r0);
          hipLaunchKernelGGL((k_distill_join<TI, kPartWaves, TAIL>), dim3(n), dim3(kPartWaves * 64), 0, st, li, *teacher, c1, d_loss, stats, part, parts, r0);
          if (grad) launch_backward(ti, grad->dtype, n, parts, st, li, lo, *teacher, c1, stats, r0);
        } else if (!grad) {
          hipLaunchKernelGGL((k_distill<TI, TI, kRowWaves, TAIL, false>), dim3(n), dim3(kRowWaves * 64), marks, st, li, lo, *teacher, c1, d_loss, stats, r0);
        } else if (grad->dtype == EMU_BF16) {
          hipLaunchKernelGGL((k_distill<TI, bf16_t, kRowWaves, TAIL, true>), dim3(n), dim3(kRowWaves * 64), marks, st, li, lo, *teacher, c1, d_loss, stats, r0);
        } else {
          hipLaunchKernelGGL((k_distill<TI, float, kRowWaves, TAIL, true>), dim3(n), dim3(kRowWaves * 64), marks, st, li, lo, *teacher, c1, d_loss, stats, r0);
        }
      };
      teacher->tail ? by_tail(std::true_type()) : by_tail(std::false_type());
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
  const uint32_t parts = backward_parts(student, li.Vp);
  by_type(student->dtype, [&](auto ti) {
    over_rows(student->rows, [&](uint64_t r0, uint32_t n) {
      launch_backward(ti, grad->dtype, n, parts, st, li, lo, *teacher, c1, reinterpret_cast<const float4*>(d_stats), r0);
    });
  });
  return hip_check("emu_distill_backward launch");
}

}  // extern "C"
