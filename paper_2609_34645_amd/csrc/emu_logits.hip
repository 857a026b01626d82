// Operators on the logits of a vocab-parallel LM head (include/emu.h): constraints ahead of sampling, the
// k largest log-probabilities, distillation with its gradient. Every row is read once (twice for a loss with its
// gradient where registers do not hold it), in 16-byte vectors; every reduction runs over global columns in a fixed
// order, so that no result depends on how the shards cut them.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "emu_hip.h"

namespace emu {

constexpr int kMaxShards = 64;
constexpr int32_t kMaxVocab = 1 << 20;
constexpr int32_t kMaxTokens = (1 << 20) - 1;  // of one row's history
constexpr int kMaxTop = 64;        // entries of emu_logits_topk: one per lane of a wave
constexpr int kMaxTeacher = 256;   // entries of a teacher's row
constexpr uint32_t kMaxSplits = 64;            // workgroups that share a row: one partial result per lane
constexpr uint32_t kRowsPerLaunch = 1u << 15;  // bounds a grid's work-items below 2^32, and the workspace that a call needs
constexpr float kInf = __builtin_inff();

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

// A value that the kernel does not write, at an address that is the same in every lane: by a scalar load, which
// does not wait behind the vector loads in flight.
template <typename T> __device__ __forceinline__ T scalar(const T* p) { return *(const __attribute__((address_space(4))) T*)p; }

// ------------------------------------------------------------------------------------------------
// rows in vectors
// ------------------------------------------------------------------------------------------------
// A lane holds 16 bytes, kE<T> columns from a multiple of kE<T> on; a wave's tile is 64 such vectors, 1 KB. A workgroup
// has a span of tiles and each of its waves a contiguous part of it, U tiles at a time: copies of rows ran at 6.3 TB/s
// with 16 contiguous KB per wave, at 5.5 with the waves' 4 KB by turns. Columns are counted over the whole vocabulary,
// so which lane adds up which column, and in which order, does not depend on the shards. Where the U tiles lie inside
// one shard (all but one stretch per shard do), they are U loads from one scalar base at any element alignment;
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

template <typename T>
__device__ __forceinline__ void set_minus_inf(v4u& x, uint32_t e) {
  if constexpr (sizeof(T) == 2) x[e / 2] = e % 2 ? (x[e / 2] & 0xffffu) | 0xff800000u : (x[e / 2] & 0xffff0000u) | 0xff80u;
  else x[e] = kMinusInf<T>;
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

// Tiles [t0, t1) of a row.
struct Span {
  uint32_t t0, t1;
};
__device__ __forceinline__ Span part_of(Span s, uint32_t part, uint32_t parts) {
  const uint32_t per = (s.t1 - s.t0 + parts - 1) / parts, t0 = umin(s.t0 + part * per, s.t1);
  return {t0, umin(t0 + per, s.t1)};
}
__device__ __forceinline__ uint32_t wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
template <typename T> __host__ __device__ constexpr uint32_t tiles(uint32_t columns) { return (columns + kTile<T> - 1) / kTile<T>; }

// load_edge by a table of the row's starts.
template <typename T>
__device__ __forceinline__ v4u load_lane(const Logits& l, const uint8_t* const* shard, uint32_t v) {
  const uint32_t t = shard_of(l, v), lo = v - t * l.cols;
  if (lo + kE<T> <= l.cols && v + kE<T> <= l.V) return ld16_any<POL_PLAIN>(shard[t], lo * uint32_t(sizeof(T)));
  v4u x = {kMinusInf<T>, kMinusInf<T>, kMinusInf<T>, kMinusInf<T>};
#pragma unroll
  for (uint32_t e = 0; e < kE<T>; ++e) {
    if (v + e >= l.V) break;
    const uint32_t at = shard_of(l, v + e);
    const T y = reinterpret_cast<const T*>(shard[at])[v + e - at * l.cols];
    if constexpr (sizeof(T) == 2) x[e / 2] = e % 2 ? (x[e / 2] & 0xffffu) | uint32_t(y) << 16 : (x[e / 2] & 0xffff0000u) | y;
    else x[e] = __float_as_uint(y);
  }
  return x;
}

// Where a wave is in its row: column c, in shard t at column lo, at `base`. TILE: the tile's columns. Going on keeps
// the shard's address; finding it anew (a load from the arguments) is for the few tiles that begin in another shard.
template <typename T, uint32_t TILE>
struct Cursor {
  uint64_t row_off;
  uint32_t c, t, lo;
  uint8_t* base;
  __device__ __forceinline__ Cursor(const Logits& l, uint64_t row_off, uint32_t tile) : row_off(row_off), c(tile * TILE), t(shard_of(l, c)), lo(c - t * l.cols) {
    find(l);
  }
  __device__ __forceinline__ void find(const Logits& l) { base = l.p[umin(t, kMaxShards - 1)] + row_off + uint64_t(lo) * sizeof(T); }
  __device__ __forceinline__ void advance(const Logits& l, uint32_t n) {
    c += n * TILE;
    lo += n * TILE;
    base += n * TILE * sizeof(T);
    if (lo >= l.cols) {
      do {
        lo -= l.cols;
        ++t;
      } while (lo >= l.cols);
      find(l);
    }
  }
  // n tiles wholly in one shard and below V
  __device__ __forceinline__ bool one(const Logits& l, uint32_t n) const { return lo + n * TILE <= l.cols && c + n * TILE <= l.V; }
  // the base as seen from the next shard
  __device__ __forceinline__ uint8_t* other(const Logits& l) const { return l.p[umin(t + 1, kMaxShards - 1)] + row_off - uint64_t(l.cols - lo) * sizeof(T); }
};
template <typename T> using Reader = Cursor<T, kTile<T>>;
constexpr int kScanU = 2;  // tiles that a wave adds up at a time

// A tile that is not wholly in one shard and below V. Where shards are no shorter than a tile it lies in two at
// most, and only a vector across their border goes by element.
template <typename T, int POL>
__device__ __forceinline__ v4u load_border(const Logits& l, const Reader<T>& at, uint32_t lane) {
  const uint32_t v = at.c + lane * kE<T>, lo = at.lo + lane * kE<T>;
  if (l.cols < kTile<T> || (lo < l.cols && lo + kE<T> > l.cols)) return load_edge<T, POL>(l, at.row_off, v);
  v4u x = {kMinusInf<T>, kMinusInf<T>, kMinusInf<T>, kMinusInf<T>};
  if (v >= l.V) return x;
  x = ld16_any<POL>(lo >= l.cols ? at.other(l) : at.base, lane * 16);
  if (v + kE<T> > l.V) {  // pads behind V in V's own vector
#pragma unroll
    for (uint32_t e = 0; e < kE<T>; ++e)
      if (v + e >= l.V) set_minus_inf<T>(x, e);
  }
  return x;
}

// U tiles from the cursor on, which goes behind them; -infinity from tile `end` on.
template <typename T, int U, int POL>
__device__ __forceinline__ void load_tiles(const Logits& l, Reader<T>& at, uint32_t end, v4u (&x)[U]) {
  const uint32_t lane = threadIdx.x & 63;
  if (at.one(l, U) && at.c + U * kTile<T> <= end * kTile<T>) {
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = ld16_any<POL>(at.base, lane * 16 + u * 1024);
    at.advance(l, U);
    return;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    x[u] = (v4u){kMinusInf<T>, kMinusInf<T>, kMinusInf<T>, kMinusInf<T>};
    if (at.c >= end * kTile<T>) continue;
    if (at.one(l, 1)) x[u] = ld16_any<POL>(at.base, lane * 16);
    else x[u] = load_border<T, POL>(l, at, lane);
    at.advance(l, 1);
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

// The tile at `at`, N columns a lane.
template <typename TO, int POL, uint32_t N>
__device__ __forceinline__ void store_tile(const Logits& l, const Cursor<TO, 64 * N>& at, uint32_t lane, const float (&f)[N]) {
  uint8_t* base = at.base;
  if (!at.one(l, 1)) {
    const uint32_t lo = at.lo + lane * N;
    if (l.cols < 64 * N || (lo < l.cols && lo + N > l.cols)) return store_edge<TO, POL, N>(l, at.row_off, at.c + lane * N, f);
    if (at.c + lane * N >= l.Vp) return;
    if (lo >= l.cols) base = at.other(l);
  }
  store_values<TO, POL>(base, lane * N * uint32_t(sizeof(TO)), f);
}

// ------------------------------------------------------------------------------------------------
// reductions in fixed trees
// ------------------------------------------------------------------------------------------------

// x of the lane whose number differs in bit N, in vector instructions (a shuffle through LDS takes a trip to it).
template <int N>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
  if constexpr (N == 1) return __builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, true);   // quad_perm 1 0 3 2
  if constexpr (N == 2) return __builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, true);   // quad_perm 2 3 0 1
  if constexpr (N == 4) return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true);  // 7 - i, then 3 - i
  if constexpr (N == 8) return __builtin_amdgcn_mov_dpp(x, 0x128, 0xf, 0xf, true);  // row_ror 8
  if constexpr (N == 16) {
    const auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return threadIdx.x & 16 ? y[0] : y[1];
  }
  if constexpr (N == 32) {
    const auto y = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return threadIdx.x & 32 ? y[0] : y[1];
  }
}
template <int N> __device__ __forceinline__ float lane_xor(float x) { return __uint_as_float(lane_xor<N>(__float_as_uint(x))); }
template <int N> __device__ __forceinline__ uint64_t lane_xor(uint64_t x) {
  return uint64_t(lane_xor<N>(uint32_t(x >> 32))) << 32 | lane_xor<N>(uint32_t(x));
}
template <int N> __device__ __forceinline__ double lane_xor(double x) { return __longlong_as_double(lane_xor<N>(uint64_t(__double_as_longlong(x)))); }

template <typename T, typename F>
__device__ __forceinline__ T wave_reduce(T x, F f) {
  x = f(x, lane_xor<32>(x));
  x = f(x, lane_xor<16>(x));
  x = f(x, lane_xor<8>(x));
  x = f(x, lane_xor<4>(x));
  x = f(x, lane_xor<2>(x));
  return f(x, lane_xor<1>(x));
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
// A quiet NaN is passed over; a signalling one is too, but what came before it may go with it.
__device__ __forceinline__ float max3(float a, float b, float c) {
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

__device__ __forceinline__ Running wave_joined(Running a, float c1) {
  const float m = wave_reduce(a.m, [](float x, float y) { return fmaxf(x, y); });
  return {m, wave_reduce(a.s * __builtin_amdgcn_exp2f(reference(a.m, c1) - reference(m, c1)), add)};
}

// Of the workgroup's waves, from LDS.
template <int NW>
__device__ __forceinline__ Running waves_joined(const Running* lds, float c1) {
  const uint32_t lane = threadIdx.x & 63;
  return wave_joined(lane < NW ? lds[lane] : Running{-kInf, 0.0f}, c1);
}

// Over the workgroup, in every thread. lds must not be in use: the caller has passed a barrier since it was.
template <int NW>
__device__ __forceinline__ Running block_joined(Running a, Running* lds, float c1) {
  a = wave_joined(a, c1);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
  __syncthreads();
  return waves_joined<NW>(lds, c1);
}

// U vectors of a lane; gives their largest value. Where they hold a NaN the sum is NaN from here on, and both the result
// and r.m are some of the lane's values, if perhaps not the largest.
template <int U, uint32_t E>
__device__ __forceinline__ float add_values(Running& r, const float (&f)[U][E], float c1) {
  float top = f[0][0];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (uint32_t e = 0; e < E; e += 2) top = max3(top, f[u][e], f[u][e + 1]);
  const float m = fmaxf(r.m, top);
  const float ref = reference(m, c1);
  float s = 0.0f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (uint32_t e = 0; e < E; ++e) s += __builtin_amdgcn_exp2f(fmaf(f[u][e], c1, -ref));
  r.s = r.s * __builtin_amdgcn_exp2f(reference(r.m, c1) - ref) + s;
  r.m = m;
  return top;
}

// exp(m / tau) * the result is the sum of exp(x / tau) behind r, for a maximum in the plain range.
__device__ __forceinline__ float true_sum(Running r, float c1) {
  return r.s * __builtin_amdgcn_exp2f(-fmaf(r.m, c1, -reference(r.m, c1)));
}

// Sum of exp((x - m) / tau) over the row by the whole workgroup, without the k listed columns.
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

// ------------------------------------------------------------------------------------------------
// constraints
// ------------------------------------------------------------------------------------------------
// A workgroup has SLICE columns of one row. Its logits are on their way from the start (but for vectors that the mask
// forbids whole, and in place, where most vectors stay as they are); meanwhile it goes over the row's history and
// counts the slice's tokens in LDS (integer atomics: any order gives the same counts). The slice's biases lie in
// LDS in list order, the first of a column with the sum of all of them. Then every vector is copied, masked or
// changed once: a column's word says all that concerns it, 0 that nothing does. 256 fp32 rows of 128,256,
// all under a mask, take 53 us with one token of history (195 MB, 3.7 TB/s) and 73 with up to 32,768 (20,480 on
// average): every slice goes over the whole history. 64 bf16 rows take 14.6 us, one round of workgroups whose loads
// follow from one another.

constexpr uint32_t kSeen = 1u << 31, kCountBits = (1u << 20) - 1;
constexpr uint32_t kSlotShift = 20, kSlotBits = 1023;  // of the column's first bias, from 1 on; kSlotBits: not in the list
constexpr int kListed = 512;                           // biases of a slice held in LDS
// Of a history's capacity: up to it 512 threads take 8,192 columns, beyond it 1,024 threads 16,384, so that half as many
// workgroups go over a history. 256 rows of 128,256, histories of 62% of the capacity on average, us: 8,192 tokens bf16 42 / 44, fp32
// 60 / 61; 16,384 48 / 48 and 66 / 66; 32,768 58 / 55 and 77 / 72 (256 rows of 32,768 27 / 20). The host knows the capacity
// alone: a buffer of the model's longest sequence that holds short ones pays up to 3 us of 34 for the long form. The sizes: 512
// threads on 8,192 columns took 14.8 us for 64 rows with histories of 2,500 (256 threads 15.4); 1,024 threads on 16,384 took
// 73 us for 256 rows with 20,480 on average (on 32,768 77, 512 threads 84).
constexpr int32_t kLongHistory = 8192;

template <typename TI, typename TO, int NT, uint32_t SLICE>
__global__ __launch_bounds__(NT) void k_constrain(Logits in, Logits out, emu_constraints_t c, bool in_place, uint32_t slices, uint64_t row0) {
  __shared__ __align__(16) uint32_t count[SLICE];
  __shared__ int32_t list_col[kListed];
  __shared__ float list_value[kListed], total[kListed];
  __shared__ uint32_t listed;
  constexpr uint32_t E = kE<TI>, TILES = SLICE / (NT / 64) / kTile<TI>, kAll = (1u << E) - 1;  // tiles of a wave
  const uint32_t row = blockIdx.x / slices, c0 = (blockIdx.x - row * slices) * SLICE, c1 = umin(c0 + SLICE, in.Vp);
  const uint64_t r = row0 + row, ri = r * in.row_bytes, ro = r * out.row_bytes;
  const uint32_t lane = threadIdx.x & 63, first = c0 / kTile<TI> + wave_id() * TILES;
  const uint8_t* mask = nullptr;
  if (c.mask) {
    const int64_t which = c.mask_row ? int64_t(scalar(c.mask_row + r)) : int64_t(r);
    if (which >= 0 && which < c.n_masks) mask = reinterpret_cast<const uint8_t*>(c.mask + which * c.mask_stride);
  }
  uint32_t allowed[TILES];
  v4u x[TILES];
#pragma unroll
  for (uint32_t u = 0; u < TILES; ++u) {
    const uint32_t v = (first + u) * kTile<TI> + lane * E;
    allowed[u] = kAll;
    if (mask && v < in.V) allowed[u] = mask[v / 8];
  }
#pragma unroll
  for (uint32_t u = 0; u < TILES; ++u) {
    const uint32_t v = (first + u) * kTile<TI> + lane * E;
    if (mask && v < in.V) allowed[u] = (allowed[u] >> (v % 8)) & kAll;
  }
  auto load = [&](uint32_t u, Reader<TI>& at, bool wanted) {
    x[u] = (v4u){kMinusInf<TI>, kMinusInf<TI>, kMinusInf<TI>, kMinusInf<TI>};
    if (at.c < in.V && wanted) {
      if (at.one(in, 1)) x[u] = ld16_any<POL_NT>(at.base, lane * 16);
      else x[u] = load_border<TI, POL_NT>(in, at, lane);
    }
    at.advance(in, 1);
  };
  if (!in_place) {
    Reader<TI> at(in, ri, first);
#pragma unroll
    for (uint32_t u = 0; u < TILES; ++u) load(u, at, allowed[u] != 0);
  }

  const bool concerns = c.tokens || c.bias_first;
  int64_t b0 = 0, b1 = 0;
  if (concerns) {
    for (uint32_t i = threadIdx.x * 4; i < SLICE; i += NT * 4) *reinterpret_cast<v4u*>(count + i) = (v4u){0, 0, 0, 0};
    if (threadIdx.x == 0) listed = 0;
    __syncthreads();
  }
  const uint32_t own = umin(in.V - umin(c0, in.V), SLICE);  // the slice's columns below V
  if (c.bias_first) {
    b0 = min(max(int64_t(scalar(c.bias_first + r)), int64_t(0)), c.n_bias);
    b1 = min(max(int64_t(scalar(c.bias_first + r + 1)), int64_t(0)), c.n_bias);
    if (wave_id() == NT / 64 - 1) {  // the last wave, while the others are in the history
      uint32_t n = 0;
      for (int64_t i0 = b0 + lane; i0 - lane < b1; i0 += 256) {
        uint32_t at[4];
        float value[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) at[q] = (i0 + q * 64 < b1 ? uint32_t(c.bias_token[i0 + q * 64]) : ~0u) - c0;
#pragma unroll
        for (int q = 0; q < 4; ++q) value[q] = i0 + q * 64 < b1 ? c.bias_value[i0 + q * 64] : 0.0f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const bool here = i0 + q * 64 < b1 && at[q] < own;
          const uint64_t lanes = __ballot(here);
          const uint32_t pos = n + __popcll(lanes & ((1ull << lane) - 1));
          if (here && pos < kListed) {
            list_col[pos] = int32_t(at[q] + c0);
            list_value[pos] = value[q];
          }
          n += __popcll(lanes);
        }
      }
      if (lane == 0) listed = n;
    }
  }
  if (c.tokens) {
    const int32_t* tok = c.tokens + r * c.tokens_stride;
    const int32_t n = min(max(scalar(c.seq_len + r), 0), c.tokens_cols);
    const int32_t prompt = c.prompt_len ? scalar(c.prompt_len + r) : 0;
    auto take = [&](uint32_t v, int32_t i) {
      const uint32_t at = v - c0;
      if (at < own) {
        if (i < prompt) atomicOr(&count[at], kSeen);
        else atomicAdd(&count[at], 1u);
      }
    };
    // four vectors a thread in flight; behind the last whole one, token by token
    constexpr int32_t kStep = NT * 4;
    const int32_t whole = n & ~3;
    for (int32_t i0 = threadIdx.x * 4; i0 < whole; i0 += 4 * kStep) {
      v4u v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        v[q] = i0 + q * kStep < whole ? ld16_any<POL_PLAIN>(reinterpret_cast<const uint8_t*>(tok), uint32_t(i0 + q * kStep) * 4) : (v4u){~0u, ~0u, ~0u, ~0u};
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) take(v[q][e], i0 + q * kStep + e);
    }
    if (int32_t(threadIdx.x) < n - whole) take(uint32_t(tok[whole + threadIdx.x]), whole + threadIdx.x);
  }
  __syncthreads();
  if (c.bias_first) {
    const uint32_t n = listed;
    if (n <= kListed) {
      for (uint32_t j = threadIdx.x; j < n; j += NT) {
        const int32_t col = list_col[j];
        float sum = 0.0f;
        bool leads = true;
        for (uint32_t i = 0; i < n; ++i) {
          if (list_col[i] != col) continue;
          leads &= i >= j;
          sum += list_value[i];
        }
        if (leads) {
          total[j] = sum;
          atomicOr(&count[col - c0], (j + 1) << kSlotShift);
        }
      }
    } else {
      for (int64_t i = b0 + threadIdx.x; i < b1; i += NT) {
        const uint32_t at = uint32_t(c.bias_token[i]) - c0;
        if (at < own) atomicOr(&count[at], kSlotBits << kSlotShift);
      }
    }
    __syncthreads();
  }

  // x / theta as a product with the rounded 1 / theta: off by half a step more than a division, at a tenth of its price
  const float theta = c.repetition ? scalar(c.repetition + r) : 1.0f, inverse = 1.0f / theta;
  const float af = c.frequency ? scalar(c.frequency + r) : 0.0f, ap = c.presence ? scalar(c.presence + r) : 0.0f;
  auto bias = [&](uint32_t slot, uint32_t v) {
    if (slot != kSlotBits) return total[slot - 1];
    float sum = 0.0f;
    for (int64_t i = b0; i < b1; ++i)
      if (c.bias_token[i] == int32_t(v)) sum += c.bias_value[i];
    return sum;
  };
  // what concerns a vector's columns, and whether anything does
  auto words = [&](uint32_t u, uint32_t (&n)[E]) {
    uint32_t any = 0;
    const uint32_t at = (first + u) * kTile<TI> + lane * E - c0;
#pragma unroll
    for (uint32_t q = 0; q < E; q += 4) {
      const v4u four = concerns ? *reinterpret_cast<const v4u*>(count + at + q) : (v4u){0, 0, 0, 0};
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        n[q + e] = four[e];
        any |= four[e];
      }
    }
    return any;
  };
  // in place, a vector stays where nothing concerns or forbids it and no pad ends it
  auto kept = [&](uint32_t u, uint32_t any) { return in_place && !any && allowed[u] == kAll && (first + u) * kTile<TI> + lane * E + E <= in.V; };
  if (in_place) {
    Reader<TI> at(in, ri, first);
#pragma unroll
    for (uint32_t u = 0; u < TILES; ++u) {
      uint32_t n[E];
      load(u, at, allowed[u] != 0 && !kept(u, words(u, n)));
    }
  }
  Cursor<TO, kTile<TI>> to(out, ro, first);
#pragma unroll
  for (uint32_t u = 0; u < TILES; ++u) {
    const uint32_t v = (first + u) * kTile<TI> + lane * E;
    if (to.c >= c1) break;
    float f[E];
    unpack(x[u], f);
    uint32_t n[E];
    const uint32_t any = words(u, n);
    if (any && allowed[u]) {
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) {  // without branches: * 1 and - 0 where nothing concerns the column
        const uint32_t times = n[e] & kCountBits;
        const float factor = n[e] & (kSeen | kCountBits) ? (f[e] > 0.0f ? inverse : theta) : 1.0f;
        f[e] = f[e] * factor - (times ? fmaf(af, float(times), ap) : 0.0f);
      }
      if ((any >> kSlotShift) & kSlotBits) {
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) {
          const uint32_t slot = (n[e] >> kSlotShift) & kSlotBits;
          if (slot) f[e] += bias(slot, v + e);
        }
      }
    }
    if (allowed[u] != kAll) {
#pragma unroll
      for (uint32_t e = 0; e < E; ++e)
        if (!((allowed[u] >> e) & 1u)) f[e] = -kInf;
    }
    if (!kept(u, any)) store_tile<TO, POL_NT>(out, to, lane, f);
    to.advance(out, 1);
  }
}

// ------------------------------------------------------------------------------------------------
// the k largest
// ------------------------------------------------------------------------------------------------
// Every logit has a key whose order is the result's: the value, then the lower column. The scan for the softmax
// statistics also gives every thread's largest logit, and its largest in each of up to kSegments stretches. The k-th
// largest of the threads' maxima is a bound that k logits reach; about k + k^2 / (2 threads) do in all, in as many
// stretches. Those stretches are read again by their lanes, and what reaches the bound is sorted. Where that is more
// than the LDS list holds (ties at the bound, a few threads with all large logits), each wave goes over its tiles again
// with its own k best sorted, one per lane, and merges in what beats its k-th, 64 at a time. 4,096 rows of 128,256 in
// bf16, k 64: 195 to 207 us (5.1 to 5.4 TB/s); an earlier form, whose waves kept sorted lists during the scan, took
// 402.

__device__ __forceinline__ uint32_t top_order(float x) {  // 0: never chosen
  const uint32_t u = __float_as_uint(x + 0.0f);  // -0 becomes 0
  return x > -kInf ? (u & 0x80000000u ? ~u : u | 0x80000000u) : 0;
}
__device__ __forceinline__ uint64_t top_key(float x, uint32_t v) {
  const uint32_t order = top_order(x);
  return order ? uint64_t(order) << 32 | uint32_t(~v) : 0;
}
__device__ __forceinline__ float order_value(uint32_t order) {
  return order == 0 ? -kInf : __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order);
}
__device__ __forceinline__ float key_value(uint64_t key) { return order_value(uint32_t(key >> 32)); }
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t lane_key(uint64_t x, uint32_t lane) {  // the same lane everywhere
  return uint64_t(__builtin_amdgcn_readlane(uint32_t(x >> 32), lane)) << 32 | uint32_t(__builtin_amdgcn_readlane(uint32_t(x), lane));
}

template <uint32_t K, uint32_t J, typename T>
__device__ __forceinline__ T sort_step(T x) {  // larger ones to the lanes without bit J, in blocks of K by turns
  const uint32_t lane = threadIdx.x & 63;
  const T y = lane_xor<J>(x);
  const bool larger = x > y;
  return (((lane & J) == 0) == ((lane & K) == 0)) == larger ? x : y;
}
template <uint32_t K, uint32_t J = K / 2, typename T>
__device__ __forceinline__ T sort_steps(T x) {
  x = sort_step<K, J>(x);
  if constexpr (J > 1) return sort_steps<K, J / 2>(x);
  return x;
}
template <typename T>
__device__ __forceinline__ T sorted(T x) {  // across the wave, largest in lane 0
  return sort_steps<64>(sort_steps<32>(sort_steps<16>(sort_steps<8>(sort_steps<4>(sort_steps<2>(x))))));
}
template <typename T>
__device__ __forceinline__ T merged(T a, T b_reversed) {  // the 64 largest of two sorted waves, sorted; the second with its smallest in lane 0
  return sort_steps<64>(a > b_reversed ? a : b_reversed);
}

// What the wave's lanes wrote to LDS is what its lanes read from here on.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int kSegments = 8;
template <int NW>
struct TopLds {
  union {
    float segment[kSegments][NW * 64];  // the threads' maxima by stretch
    uint64_t fresh[NW][128];            // the slow way: a wave's collected keys
  };
  uint64_t list[NW * 64];
  uint32_t order[NW * 64];              // the threads' maxima; then the stretches to be read, thread | stretch << 16
  uint32_t n, n_stretches;              // keys in the list, stretches
  const uint8_t* shard[kMaxShards];     // the row's start in each
  Running run[NW];
  float sum[NW];
};

// The sorted lists of n waves to one, in wave 0 and in LDS.
template <typename T>
__device__ __forceinline__ T block_merged(T best, T* list, int n) {
  const uint32_t lane = threadIdx.x & 63;
  const int w = int(wave_id());
  if (w < n) list[w * 64 + lane] = best;
  while (n > 1) {
    __syncthreads();
    const int half = (n + 1) / 2;
    if (w + half < n) {
      best = merged(best, list[(w + half) * 64 + 63 - lane]);
      list[w * 64 + lane] = best;
    }
    n = half;
  }
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

__device__ __forceinline__ uint64_t reversed(uint64_t x) { return __shfl((unsigned long long)x, 63 - (threadIdx.x & 63)); }

// The slow way: the wave's k largest keys among those >= bound, sorted.
template <typename T, int NW>
__device__ __forceinline__ uint64_t wave_top(const Logits& l, uint64_t off, Span span, uint32_t k, uint64_t bound, uint64_t (*fresh)[128]) {
  constexpr uint32_t E = kE<T>;
  const uint32_t lane = threadIdx.x & 63, w = wave_id();
  uint64_t best = 0;
  uint32_t n = 0;
  auto flush = [&](uint32_t have) {
    wave_sync();
    best = merged(best, reversed(sorted(lane < have ? fresh[w][lane] : uint64_t(0))));
    const uint64_t kth = lane_key(best, k - 1);
    bound = max64(bound, kth + (kth != 0));  // from here on above it
  };
  Reader<T> at(l, off, span.t0);
  for (uint32_t tile = span.t0; tile < span.t1; ++tile) {
    v4u x[1];
    const uint32_t c = at.c;
    load_tiles<T, 1, POL_PLAIN>(l, at, span.t1, x);
    float f[E];
    unpack(x[0], f);
    for (uint32_t e = 0; e < E; ++e) {
      const uint64_t key = top_key(f[e], c + lane * E + e);
      const uint64_t lanes = __ballot(key != 0 && key >= bound);
      if (!lanes) continue;
      if (key != 0 && key >= bound) fresh[w][n + __popcll(lanes & ((1ull << lane) - 1))] = key;
      n += __popcll(lanes);
      if (n >= 64) {
        flush(64);
        n -= 64;
        const uint64_t left = fresh[w][64 + lane];
        wave_sync();
        fresh[w][lane] = left;
        wave_sync();
      }
    }
  }
  if (n) flush(n);
  return best;
}

constexpr int kTopParts = 4;  // waves of a workgroup that has a part of a row

// A workgroup per part of a row, blockIdx.x = row * parts + part. One part: the row's result. More: the part's
// statistics and keys, for k_topk_join.
template <typename T, int NW>
__global__ __launch_bounds__(NW * 64) void k_topk(Logits in, uint32_t k, float c1, int32_t* index, float* logprob, float* lse, Running* part_run,
                                                  uint64_t* part_keys, uint32_t parts, uint64_t row0) {
  constexpr int U = kScanU;
  constexpr uint32_t E = kE<T>;
  __shared__ TopLds<NW> t;
  const uint32_t row = blockIdx.x / parts;
  const uint64_t r = row0 + row, off = r * in.row_bytes;
  const uint32_t lane = threadIdx.x & 63, w = wave_id();
  const Span block = part_of({0, tiles<T>(in.V)}, blockIdx.x - row * parts, parts), span = part_of(block, w, NW);
  const uint32_t per = (span.t1 - span.t0 + U * kSegments - 1) / (U * kSegments) * U;  // tiles of a stretch
  if (threadIdx.x == 0) t.n = t.n_stretches = 0;
  if (threadIdx.x < kMaxShards) t.shard[threadIdx.x] = in.p[threadIdx.x] + off;
  Running run = {-kInf, 0.0f};
  {
    v4u x[U];
    Reader<T> at(in, off, span.t0);
    if (span.t0 < span.t1) load_tiles<T, U, POL_PLAIN>(in, at, span.t1, x);
    float top = -kInf;
    uint32_t segment = 0, segment_end = span.t0 + per;
    for (uint32_t tile = span.t0; tile < span.t1; tile += U) {
      v4u y[U];
      if (tile + U < span.t1) load_tiles<T, U, POL_PLAIN>(in, at, span.t1, y);
      float f[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u) unpack(x[u], f[u]);
      top = fmaxf(top, add_values<U, E>(run, f, c1));
      if (tile + U >= segment_end || tile + U >= span.t1) {
        t.segment[segment][threadIdx.x] = run.s == run.s ? top : __builtin_nanf("");  // behind a NaN: any value
        ++segment;
        segment_end += per;
        top = -kInf;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = y[u];
    }
  }
  // the k-th largest of the threads' maxima
  block_merged(sorted(top_order(run.m)), t.order, NW);
  run = block_joined<NW>(run, t.run, c1);
  const uint32_t kth = t.order[k - 1];
  const float level = order_value(kth);
  __syncthreads();
  // the stretches that hold (or, NaN, may hold) what reaches it, and from them, a vector a thread, what does
  const uint32_t stretches = per ? (span.t1 - span.t0 + per - 1) / per : 0;
  for (uint32_t i = 0; i < stretches; ++i)
    if (!(t.segment[i][threadIdx.x] < level)) {
      const uint32_t pos = atomicAdd(&t.n_stretches, 1u);
      if (pos < NW * 64) t.order[pos] = threadIdx.x | i << 16;
    }
  __syncthreads();
  const uint32_t most = part_of(block, 0, NW).t1 - block.t0, longest = (most + U * kSegments - 1) / (U * kSegments) * U;  // the first wave's
  const uint32_t n_vectors = t.n_stretches <= NW * 64 ? t.n_stretches * longest : 0;
  for (uint32_t q = threadIdx.x; q < n_vectors; q += NW * 64) {
    const uint32_t item = t.order[q / longest], thread = item & 0xffffu;
    const Span its = part_of(block, thread >> 6, NW);
    const uint32_t its_per = (its.t1 - its.t0 + U * kSegments - 1) / (U * kSegments) * U;
    const uint32_t in_it = q % longest, tile = its.t0 + (item >> 16) * its_per + in_it;
    if (in_it >= its_per || tile >= its.t1) continue;
    const uint32_t v = tile * kTile<T> + (thread & 63) * E;
    float f[E];
    unpack(load_lane<T>(in, t.shard, v), f);
#pragma unroll
    for (uint32_t e = 0; e < E; ++e) {
      const uint64_t key = f[e] >= level ? top_key(f[e], v + e) : 0;
      if (key) {
        const uint32_t pos = atomicAdd(&t.n, 1u);
        if (pos < NW * 64) t.list[pos] = key;
      }
    }
  }
  __syncthreads();
  const uint32_t n = t.n;
  uint64_t best;
  if (t.n_stretches <= NW * 64 && n <= NW * 64) {
    const int lists = umax((n + 63) / 64, 1);
    best = threadIdx.x < n ? t.list[threadIdx.x] : 0;
    __syncthreads();
    if (int(w) < lists) best = sorted(best);
    best = block_merged(best, t.list, lists);
  } else {
    best = wave_top<T, NW>(in, off, span, k, uint64_t(kth) << 32, t.fresh);
    __syncthreads();
    best = block_merged(best, t.list, NW);
  }
  if (parts > 1) {
    const uint64_t at = blockIdx.x;
    if (w == 0) part_keys[at * 64 + lane] = best;
    if (threadIdx.x == 0) part_run[at] = run;
    return;
  }
  const float s = row_sum<T, NW>(in, off, run, c1, t.sum);
  if (w == 0) write_top(best, k, run.m, s, c1, index, logprob, lse, r);
}

// The parts of a row to its result.
template <typename T>
__global__ __launch_bounds__(kTopParts * 64) void k_topk_join(Logits in, uint32_t k, float c1, int32_t* index, float* logprob,
                                                              float* lse, const Running* part_run, const uint64_t* part_keys,
                                                              uint32_t parts, uint64_t row0) {
  constexpr int NW = kTopParts;
  __shared__ TopLds<NW> t;
  const uint64_t r = row0 + blockIdx.x, at = uint64_t(blockIdx.x) * parts;
  const uint32_t lane = threadIdx.x & 63, w = wave_id();
  const Running run = wave_joined(lane < parts ? part_run[at + lane] : Running{-kInf, 0.0f}, c1);
  uint64_t best = 0;
  for (uint32_t i = w; i < parts; i += NW) best = merged(best, part_keys[(at + i) * 64 + 63 - lane]);
  best = block_merged(best, t.list, NW);
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
// The gradient is coef * exp((z - m) / tau), but for the listed columns, whose gradients come from their entries'
// threads by way of LDS. 4,096 rows of 128,256 in bf16, all with a weight: the loss 195 to 204 us
// (5.2 to 5.4 TB/s), the loss with the gradient 422 to 430 (4.9 TB/s), the gradient alone 390 over four shards and 364
// in one (5.4 and 5.8 TB/s). With a tail the scan leaves out the listed columns (a bit each in LDS), so that a small
// mass outside the list is a sum of its own and no difference.

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

// Entry j of row r as it is stored.
struct Stored {
  int32_t col;
  float value;
};
__device__ __forceinline__ Stored fetch_teacher(const emu_teacher_t& te, uint64_t r, uint32_t V) {
  const int j = threadIdx.x;
  if (j >= te.k) return {-1, 0.0f};
  const Stored f = {te.index[r * te.index_stride + j], te.value[r * te.value_stride + j]};
  return {uint32_t(f.col) < V ? f.col : -1, f.value};
}

// rest: the mass outside the list (0 without a tail); none: without a tail nothing is listed.
template <typename T, int NW>
__device__ __forceinline__ Entry take_teacher(DistillLds<NW>& t, Stored f, const emu_teacher_t& te, uint64_t r, const Logits& l, float* rest,
                                              bool* none) {
  static_assert(NW * 64 >= kMaxTeacher, "one entry per thread");
  const int j = threadIdx.x;
  Entry e = {f.col, 0.0f, -kInf};
  if (e.col >= 0) e.z = widen(*column<T>(l, r * l.row_bytes, e.col));
  const double value = e.col >= 0 ? double(f.value) : -double(kInf);
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
  if (e.col >= 0) {
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
__device__ __forceinline__ void mark_listed(uint32_t* bits, uint32_t c0, uint32_t range, int32_t col) {
  for (uint32_t i = threadIdx.x; i < range / 32; i += NW * 64) bits[i] = 0;
  __syncthreads();
  const uint32_t at = uint32_t(col) - c0;
  if (col >= 0 && at < range) atomicOr(&bits[at / 32], 1u << (at % 32));
  __syncthreads();
}

// -infinity in the vector's marked columns; `at` counts from the first marked column on.
template <typename T>
__device__ __forceinline__ void leave_out(v4u& x, const uint32_t* bits, uint32_t at) {
  const uint32_t hit = (reinterpret_cast<const uint8_t*>(bits)[at / 8] >> (at % 8)) & ((1u << kE<T>) - 1);
  if (hit) {
#pragma unroll
    for (uint32_t e = 0; e < kE<T>; ++e)
      if ((hit >> e) & 1u) set_minus_inf<T>(x, e);
  }
}

// The wave's statistics of its part of the workgroup's span, without the marked columns if TAIL. The next tiles
// are on their way while these are added up.
template <typename T, int NW, bool TAIL, int POL>
__device__ __forceinline__ Running scan(const Logits& l, uint64_t off, Span block, float c1, const uint32_t* bits) {
  constexpr int U = kScanU;
  constexpr uint32_t E = kE<T>;
  const uint32_t lane = threadIdx.x & 63;
  const Span span = part_of(block, wave_id(), NW);
  Running run = {-kInf, 0.0f};
  v4u x[U];
  Reader<T> at(l, off, span.t0);
  if (span.t0 < span.t1) load_tiles<T, U, POL>(l, at, span.t1, x);
  for (uint32_t t = span.t0; t < span.t1; t += U) {
    v4u y[U];
    if (t + U < span.t1) load_tiles<T, U, POL>(l, at, span.t1, y);
    float f[U][E];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (TAIL)
        if (t + u < span.t1) leave_out<T>(x[u], bits, (t + u - block.t0) * kTile<T> + lane * E);
      unpack(x[u], f[u]);
    }
    add_values<U, E>(run, f, c1);
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = y[u];
  }
  return run;
}

struct Stats {
  float lse, factor, m, s;
};

// An entry as a part of the softmax's statistics.
__device__ __forceinline__ Running entry_run(const Entry& e, float c1) {
  if (e.col < 0) return {-kInf, 0.0f};
  const float m = fmaxf(e.z, -kInf);
  return {m, __builtin_amdgcn_exp2f(fmaf(e.z, c1, -reference(m, c1)))};
}

// A row's statistics from the scan's (with a tail: of the columns outside the list) and the entries', and the rest's
// share of the loss. In every thread alike.
template <typename T, int NW, bool TAIL>
__device__ __forceinline__ Stats conclude(const Logits& l, uint64_t off, Running run, Running inside, const Entry& e, float rest, int k,
                                          float c1, DistillLds<NW>& t, float* rest_loss) {
  const float s = plain(run.m, c1) ? true_sum(run, c1)
                  : run.m == -kInf ? run.s
                                   : careful_sum<T, NW>(l, off, run.m, c1, t.col, TAIL ? k : 0, t.sum);
  Stats st = {0.0f, 1.0f, run.m, s};
  *rest_loss = 0.0f;
  if constexpr (TAIL) {
    float s_in = inside.s;
    if (plain(inside.m, c1)) s_in = true_sum(inside, c1);
    else if (inside.m != -kInf) s_in = block_reduce<NW>(e.col >= 0 ? __builtin_amdgcn_exp2f((e.z - inside.m) * c1) : 0.0f, t.sum, add);
    st.m = fmaxf(run.m, inside.m);
    const float m = st.m == -kInf ? 0.0f : st.m;
    st.s = (s == 0.0f ? 0.0f : s * __builtin_amdgcn_exp2f((run.m - m) * c1)) + (s_in == 0.0f ? 0.0f : s_in * __builtin_amdgcn_exp2f((inside.m - m) * c1));
    const float log_q = s == 0.0f ? -kInf
                                  : float(((double(run.m) - double(st.m)) * double(c1) + double(log2f(s)) - double(log2f(st.s))) * 0.6931471805599453);
    if (rest != 0.0f && (s != 0.0f || rest >= kRestNoise)) *rest_loss = rest * (logf(rest) - log_q);
    const float q = expf(log_q);
    if (!(q < kLeastRest)) st.factor = 1.0f - rest / q;
  }
  st.lse = log_sum_exp(st.m, st.s, c1);
  return st;
}

__device__ __forceinline__ float entry_loss(const Entry& e, Stats st, float c1) {
  return e.p != 0.0f ? e.p * (logf(e.p) - log_prob(e.z, st.m, st.s, c1)) : 0.0f;
}

// conclude with the loss, in every thread.
template <typename T, int NW, bool TAIL>
__device__ __forceinline__ Stats finish(const Logits& l, uint64_t off, Running run, const Entry& e, float rest, int k, float c1,
                                        DistillLds<NW>& t, float* loss) {
  Running inside = {-kInf, 0.0f};
  __syncthreads();
  if constexpr (TAIL) inside = block_joined<NW>(entry_run(e, c1), t.run, c1);
  float rest_loss;
  const Stats st = conclude<T, NW, TAIL>(l, off, run, inside, e, rest, k, c1, t, &rest_loss);
  *loss = block_reduce<NW>(entry_loss(e, st, c1), t.sum, add) + rest_loss;
  return st;
}

// The listed columns' gradients in LDS, chained by tile, for the lanes that hold the columns: writing them behind the
// dense gradient instead, two bytes here and there, cost 24 of 398 us (4,096 rows of 128,256, 64 entries).
template <int TILES>
struct Listed {
  int16_t head[TILES], next[kMaxTeacher];  // -1: none
  int32_t col[kMaxTeacher];
  float d[kMaxTeacher];
};

__device__ __forceinline__ float entry_gradient(const Entry& e, Stats st, float c1, float scale) {
  const float q = st.s == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((e.z - st.m) * c1) / st.s;
  return (q - e.p) * scale;
}

// Entry j (thread j) into its tile's chain. The heads are -1 and a barrier has been passed; another must follow. The
// order within a chain is any: its columns differ.
template <typename T, int TILES>
__device__ __forceinline__ void chain(Listed<TILES>& list, uint32_t t0, const Entry& e, float d) {
  if (e.col < 0) return;
  const uint32_t at = uint32_t(e.col) / kTile<T> - t0;
  // heads are halves of words: exchange the half by comparison
  uint32_t* word = reinterpret_cast<uint32_t*>(list.head) + at / 2;
  const uint32_t shift = at % 2 * 16;
  uint32_t old = *word, want;
  do {
    want = old;
    old = atomicCAS(word, want, (want & ~(0xffffu << shift)) | uint32_t(threadIdx.x) << shift);
  } while (old != want);
  list.next[threadIdx.x] = int16_t(old >> shift);
  list.col[threadIdx.x] = e.col;
  list.d[threadIdx.x] = d;
}

// The tile's listed columns in place of the dense values; head the same in every lane.
template <int TILES, uint32_t E>
__device__ __forceinline__ void take_listed(const Listed<TILES>& list, int head, uint32_t v, float (&f)[E]) {
  while (head >= 0) {
    const uint32_t at = uint32_t(list.col[head]) - v;
    const float d = list.d[head];
#pragma unroll
    for (uint32_t e = 0; e < E; ++e) f[e] = at == e ? d : f[e];
    head = __builtin_amdgcn_readfirstlane(list.next[head]);
  }
}

// Dense: coef * exp((z - m) / tau) over the workgroup's span of the padded row, 0 behind V, the listed columns'
// values in their places. ZERO: 0 for the dense part, and no logits are read.
enum Dense { PLAIN_RANGE, ANY_RANGE, ZERO };
template <typename TI, typename TO, int U, int NW, int POL, Dense KIND, int TILES>
__device__ __forceinline__ void dense_gradient(const Logits& in, const Logits& out, uint64_t r, Span block, const Listed<TILES>* list, float m,
                                               float c1, float coef) {
  constexpr uint32_t E = kE<TI>;
  const uint32_t lane = threadIdx.x & 63;
  const uint64_t ri = r * in.row_bytes, ro = r * out.row_bytes;
  const float ref = reference(m, c1);
  const Span span = part_of(block, wave_id(), NW);
  int heads = -1;  // of 64 tiles, one a lane; none of a tile of pads alone
  Reader<TI> from(in, ri, span.t0);
  Cursor<TO, kTile<TI>> to(out, ro, span.t0);
  for (uint32_t tile = span.t0; tile < span.t1; tile += U) {
    v4u x[U];
    if constexpr (KIND != ZERO) load_tiles<TI, U, POL>(in, from, span.t1, x);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (tile + u >= span.t1) break;
      if (list && (tile + u - span.t0) % 64 == 0) {
        const uint32_t mine = tile + u + lane;
        heads = mine < umin(span.t1, tiles<TI>(in.V)) ? list->head[mine - block.t0] : -1;
      }
      float f[E];
      if constexpr (KIND != ZERO) unpack(x[u], f);
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) {
        if constexpr (KIND == ZERO) f[e] = 0.0f;
        else f[e] = __builtin_amdgcn_exp2f(KIND == PLAIN_RANGE ? fmaf(f[e], c1, -ref) : (f[e] - m) * c1) * coef;
      }
      const uint32_t v = to.c + lane * E;
      if (to.c + kTile<TI> > in.V) {
#pragma unroll
        for (uint32_t e = 0; e < E; ++e)
          if (v + e >= in.V) f[e] = 0.0f;
      }
      if (list) take_listed(*list, __builtin_amdgcn_readlane(heads, (tile + u - span.t0) % 64), v, f);
      store_tile<TO, POL_NT>(out, to, lane, f);
      to.advance(out, 1);
    }
  }
}

// Row r's gradient over the span, from its statistics. The heads of the list are -1, behind a barrier.
template <typename TI, typename TO, int U, int NW, int POL, int TILES>
__device__ __forceinline__ void row_gradient(const Logits& in, const Logits& out, uint64_t r, Span block, Listed<TILES>& list, const Entry& e,
                                             Stats st, float c1, float w, bool none) {
  const float scale = w * (c1 * 0.69314718f);  // w / tau
  if (w == 0.0f || none) return dense_gradient<TI, TO, U, NW, POL, ZERO, TILES>(in, out, r, block, nullptr, st.m, c1, 0.0f);
  chain<TI>(list, block.t0, e, entry_gradient(e, st, c1, scale));
  __syncthreads();
  if (st.s == 0.0f) {
    dense_gradient<TI, TO, U, NW, POL, ZERO>(in, out, r, block, &list, st.m, c1, 0.0f);
  } else if (plain(st.m, c1)) {
    const float one = __builtin_amdgcn_exp2f(-fmaf(st.m, c1, -reference(st.m, c1)));  // exp2(ref - m * c1)
    dense_gradient<TI, TO, U, NW, POL, PLAIN_RANGE>(in, out, r, block, &list, st.m, c1, scale * st.factor * (one / st.s));
  } else {
    dense_gradient<TI, TO, 1, NW, POL, ANY_RANGE>(in, out, r, block, &list, st.m, c1, scale * st.factor * (1.0f / st.s));
  }
}

__device__ __forceinline__ void write_row(float* loss, float4* stats, uint64_t r, float value, Stats st) {
  if (threadIdx.x == 0) {
    loss[r] = value;
    stats[r] = make_float4(st.lse, st.factor, st.m, st.s);
  }
}
constexpr Stats kSkipped = {__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};

constexpr int kGradU = 4;
constexpr int kRowTiles = 1024;  // below V, of a row that one workgroup takes: kMarked columns of fp32

// What the kernels need of the teachers, a wave per row: per entry its column (-1: none, or one that an earlier
// entry has) and that column's whole probability, per row the mass outside the list (-1: nothing listed). The
// exponentials and comparisons stay out of the row's own way there. Also the first ticket.
constexpr int kPrepareWaves = 4;
struct Prepared {
  Stored entry[kMaxTeacher];
};
__global__ __launch_bounds__(kPrepareWaves * 64) void k_prepare_teacher(emu_teacher_t te, uint32_t V, Prepared* out, float* rest, uint32_t* ticket,
                                                                        uint32_t rows, uint64_t row0) {
  __shared__ int32_t cols[kPrepareWaves][kMaxTeacher];
  __shared__ double ps[kPrepareWaves][kMaxTeacher];
  const uint32_t w = wave_id(), lane = threadIdx.x & 63, row = blockIdx.x * kPrepareWaves + w;
  if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;
  if (row >= rows) return;
  const uint64_t r = row0 + row;
  if (te.weight && te.weight[r] == 0.0f) return;
  constexpr int N = kMaxTeacher / 64;
  int32_t col[N];
  double value[N], top = -double(kInf);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int j = i * 64 + lane;
    col[i] = -1;
    value[i] = -double(kInf);
    if (j < te.k) {
      const int32_t v = te.index[r * te.index_stride + j];
      if (uint32_t(v) < V) {
        col[i] = v;
        value[i] = double(te.value[r * te.value_stride + j]);
      }
    }
    top = fmax(top, value[i]);
  }
  top = wave_reduce(top, [](double a, double b) { return fmax(a, b); });
  if (te.tail || top == -double(kInf)) top = 0.0;
  double p[N], sum = 0.0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    p[i] = i * 64 < te.k && col[i] >= 0 ? exp(value[i] - top) : 0.0;
    sum += wave_reduce(p[i], addd);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (!te.tail && sum != 0.0) p[i] /= sum;
    cols[w][i * 64 + lane] = col[i];
    ps[w][i * 64 + lane] = p[i];
  }
  wave_sync();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int j = i * 64 + lane;
    if (j >= te.k) break;
    bool first = col[i] >= 0;
    for (int o = 0; o < te.k; ++o) {
      if (o == j || cols[w][o] != col[i]) continue;
      if (o < j) first = false;
      else p[i] += ps[w][o];
    }
    out[row].entry[j] = first ? Stored{col[i], float(p[i])} : Stored{-1, 0.0f};
  }
  const float left = float(1.0 - sum);
  if (lane == 0) rest[row] = te.tail ? (left < 0.0f ? 0.0f : left) : sum == 0.0 ? -1.0f : 0.0f;
}

// One workgroup per row. teacher NULL: entries as the caller stored them (few rows: a launch less).
template <typename TI, typename TO, int NW, bool TAIL, bool GRAD>
__global__ __launch_bounds__(NW * 64) void k_distill(Logits in, Logits grad, emu_teacher_t te, float c1, float* loss, float4* stats,
                                                     const Prepared* teacher, const float* rests, uint64_t row0) {
  extern __shared__ uint32_t bits[];
  __shared__ DistillLds<NW> t;
  __shared__ Listed<GRAD ? kRowTiles : 2> list;
  const uint64_t r = row0 + blockIdx.x, off = r * in.row_bytes;
  const float w = te.weight ? te.weight[r] : 1.0f;
  Entry e = {-1, 0.0f, -kInf};
  Stats st = kSkipped;
  float rest = 0.0f;
  if constexpr (GRAD)
    for (int i = threadIdx.x; i < kRowTiles; i += NW * 64) list.head[i] = -1;
  if (w != 0.0f) {
    Stored f = {-1, 0.0f};
    if (!teacher) f = fetch_teacher(te, r, in.V);
    else if (int(threadIdx.x) < te.k) f = teacher[blockIdx.x].entry[threadIdx.x];
    const Span row = {0, tiles<TI>(in.V)};
    if constexpr (TAIL) mark_listed<NW>(bits, 0, row.t1 * kTile<TI>, f.col);
    const Running run = block_joined<NW>(scan<TI, NW, TAIL, GRAD ? POL_PLAIN : POL_NT>(in, off, row, c1, bits), t.run, c1);
    if (!teacher) {
      bool none;
      e = take_teacher<TI, NW>(t, f, te, r, in, &rest, &none);
      if (none) rest = -1.0f;
    } else {
      e = {f.col, f.value, -kInf};
      if (e.col >= 0) e.z = widen(*column<TI>(in, off, e.col));
      if (int(threadIdx.x) < kMaxTeacher) t.col[threadIdx.x] = e.col;
      rest = rests[blockIdx.x];
    }
    float value;
    st = finish<TI, NW, TAIL>(in, off, run, e, rest < 0.0f ? 0.0f : rest, te.k, c1, t, &value);
    write_row(loss, stats, r, value * w, st);
  } else {
    write_row(loss, stats, r, 0.0f, st);
  }
  if constexpr (GRAD) row_gradient<TI, TO, kGradU, NW, POL_NT>(in, grad, r, {0, tiles<TI>(in.Vp)}, list, e, st, c1, w, rest < 0.0f);
}

// A row held in registers between its two uses, up to 16 tiles of each of NW waves, where the shards hold whole aligned
// vectors and are no shorter than a tile (a tile then lies in one shard or two): one read, one write, no tail. The
// workgroups stay and take rows by ticket, so that the device works on a window of neighbouring rows (in equal shares
// fixed ahead, 4,096 rows of 131,072 took 450 us against 425) and rows without a weight cost no one more; while a
// vector's gradient leaves, the next row's vector is loaded into its registers, so that memory has both to do. Every
// turn issues the same loads and stores, whatever the row: a wait for one of them can then name the number of younger
// ones, where with any in doubt it would be for all. Tiles that a wave does not have, and rows without a weight, load a
// vector of -infinities; a store beyond a shard's row is dropped by the buffer's bounds. Tiles, and the order of every
// sum, are k_distill's: the result is the same, bit for bit.
constexpr int kResidentTiles = 16;
__device__ const v4u kNoLogits[2] = {{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}, {0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u}};

// N columns a lane at byte `off` of the buffer; beyond its end nothing is written.
template <typename TO, uint32_t N>
__device__ __forceinline__ void store_bounded(__amdgpu_buffer_rsrc_t to, uint32_t off, const float (&f)[N]) {
  constexpr int kStream = 2;  // nt
  if constexpr (sizeof(TO) == 4) {
#pragma unroll
    for (uint32_t i = 0; i < N; i += 4)
      __builtin_amdgcn_raw_buffer_store_b128((v4u){__float_as_uint(f[i]), __float_as_uint(f[i + 1]), __float_as_uint(f[i + 2]), __float_as_uint(f[i + 3])}, to, off + i * 4, 0, kStream);
  } else if constexpr (N == 8) {
    __builtin_amdgcn_raw_buffer_store_b128((v4u){pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])}, to, off, 0, kStream);
  } else {
    __builtin_amdgcn_raw_buffer_store_b64((v2u){pack2(f[0], f[1]), pack2(f[2], f[3])}, to, off, 0, kStream);
  }
}

template <typename TI, typename TO, int NW>
__global__ __launch_bounds__(NW * 64, 4) void k_distill_resident(Logits in, Logits grad, emu_teacher_t te, float c1, float* loss, float4* stats,
                                                                     const Prepared* teacher, const float* rests, uint32_t* ticket, uint32_t rows,
                                                                     uint64_t row0) {
  constexpr int U = kScanU, NV = kResidentTiles;
  constexpr uint32_t E = kE<TI>;
  __shared__ DistillLds<NW> t;
  __shared__ Listed<NW * NV> list;
  __shared__ uint8_t* shards[kMaxShards];
  v4u x[NV];
  __shared__ uint32_t taken, first;
  uint32_t now = rows, next, after;  // the row in x, the row to load, the one behind it; `rows`: none
  float w = 0.0f;
  Entry e = {-1, 0.0f, -kInf};
  for (int i = threadIdx.x; i < NW * NV; i += NW * 64) list.head[i] = -1;
  if (threadIdx.x < kMaxShards) shards[threadIdx.x] = in.p[threadIdx.x];
  if (threadIdx.x == 0) first = atomicAdd(ticket, 1u);
  __syncthreads();
  next = umin(__builtin_amdgcn_readfirstlane(first), rows);
  for (;;) {
    const uint64_t r = row0 + now, ri = r * in.row_bytes;
    // the tiles' places are the same in every turn: kept out of the compiler's sight, which would hold them all in registers
    uint32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    const uint32_t lane = thread & 63;
    const Span span = part_of({0, tiles<TI>(in.V)}, __builtin_amdgcn_readfirstlane(thread >> 6), NW);
    const uint32_t t0 = span.t0, t1 = span.t1, last = in.V / kTile<TI>;
    // what the turn needs beside x is on its way during the scan: a wait for it behind the loads would be one for them
    uint32_t later = 0;
    if (threadIdx.x == 0) later = atomicAdd(ticket, 1u);
    const float w_next = next < rows ? (te.weight ? scalar(te.weight + row0 + next) : 1.0f) : 0.0f;
    v2u f_next = {~0u, 0u};
    if (w_next != 0.0f && int(thread) < te.k) f_next = ld8_any<POL_PLAIN>(reinterpret_cast<const uint8_t*>(teacher + next), thread * 8);
    Stats st = kSkipped;
    float rest_loss = 0.0f, scale = 0.0f, coef = 0.0f;
    const bool live = now < rows && w != 0.0f;
    if (live) {
      Running run = {-kInf, 0.0f};
#pragma unroll
      for (int i = 0; i < NV; i += U) {
        if (t0 + i >= t1) break;
        float f[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          asm volatile("" : "+v"(x[i + u]));  // in this order: all at once would take twice the registers
          if (t0 + i + u == last) {  // pads behind V in V's own vector
#pragma unroll
            for (uint32_t q = 0; q < E; ++q)
              if ((t0 + i + u) * kTile<TI> + lane * E + q >= in.V) set_minus_inf<TI>(x[i + u], q);
          }
          unpack(x[i + u], f[u]);
        }
        add_values<U, E>(run, f, c1);
        __builtin_amdgcn_sched_barrier(0);
      }
      run = wave_joined(run, c1);
      if (lane == 0) t.run[wave_id()] = run;
    }
    const bool listed = live && !(scalar(rests + now) < 0.0f);
    if (threadIdx.x == 0) taken = later;  // everyone has read the last one before the last turn's last barrier
    __syncthreads();
    after = umin(__builtin_amdgcn_readfirstlane(taken), rows);
    if (live) {
      st = conclude<TI, NW, false>(in, ri, waves_joined<NW>(t.run, c1), {-kInf, 0.0f}, e, 0.0f, 0, c1, t, &rest_loss);
      scale = w * (c1 * 0.69314718f);
    }
    const uint64_t ro = r * grad.row_bytes, rn = (row0 + next) * in.row_bytes;
    TI z_next = TI();  // widened when it is needed: to do it here would be to wait for it
    if (int32_t(f_next[0]) >= 0) {
      const uint32_t t = shard_of(in, f_next[0]);
      z_next = reinterpret_cast<const TI*>(shards[t] + rn)[f_next[0] - t * in.cols];
    }
    const bool zero = !listed || st.s == 0.0f, wild = !zero && !plain(st.m, c1);
    const float ref = reference(st.m, c1);
    if (!zero) coef = scale * st.factor * ((wild ? 1.0f : __builtin_amdgcn_exp2f(-fmaf(st.m, c1, -ref))) / st.s);
    int heads = -1;
    if (listed) chain<TI>(list, 0, e, entry_gradient(e, st, c1, scale));
    if (live) __syncthreads();  // the chains are whole, and no wave reads t.sum for conclude any more
    if (listed && t0 + lane < t1) heads = list.head[t0 + lane];
    if (wild) dense_gradient<TI, TO, 1, NW, POL_NT, ANY_RANGE>(in, grad, r, {0, tiles<TI>(in.V)}, &list, st.m, c1, coef);
    const bool write = now < rows && !wild;
    Reader<TI> from(in, rn, t0);
    Cursor<TO, kTile<TI>> to(grad, ro, t0);
    const uint8_t* none = reinterpret_cast<const uint8_t*>(kNoLogits + (sizeof(TI) == 2 ? 0 : 1));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float f[E];
      if (zero) {
#pragma unroll
        for (uint32_t q = 0; q < E; ++q) f[q] = 0.0f;
      } else {
        asm volatile("" : "+v"(x[i]));  // unpacked anew: the scan's values would take twice the registers
        unpack(x[i], f);
#pragma unroll
        for (uint32_t q = 0; q < E; ++q) f[q] = __builtin_amdgcn_exp2f(fmaf(f[q], c1, -ref)) * coef;
        if (t0 + i == last) {
#pragma unroll
          for (uint32_t q = 0; q < E; ++q)
            if (to.c + lane * E + q >= in.V) f[q] = 0.0f;
        }
      }
      take_listed(list, __builtin_amdgcn_readlane(heads, i), to.c + lane * E, f);
      const uint32_t row_end = grad.cols * uint32_t(sizeof(TO)), at = write && t0 + i < t1 ? to.lo * uint32_t(sizeof(TO)) : 1u << 31;
      uint8_t* row = to.base - uint64_t(to.lo) * sizeof(TO);
      store_bounded<TO>(__builtin_amdgcn_make_buffer_rsrc(row, 0, row_end, 0x00020000), at + lane * E * uint32_t(sizeof(TO)), f);
      if (to.lo + kTile<TI> > grad.cols && to.c - to.lo + grad.cols < grad.Vp)  // and in the next shard
        store_bounded<TO>(__builtin_amdgcn_make_buffer_rsrc(grad.p[to.t + 1] + ro, 0, row_end, 0x00020000),
                          (write && t0 + i < t1 ? at - row_end : 1u << 31) + lane * E * uint32_t(sizeof(TO)), f);
      const bool have = w_next != 0.0f && t0 + i < t1;
      if (have && from.one(in, 1)) {
        x[i] = ld16_any<POL_NT>(from.base, lane * 16);
      } else {
        const uint8_t* where = none - lane * 16;
        if (have && from.c + lane * E < in.V) where = from.lo + lane * E >= in.cols ? from.other(in) : from.base;
        x[i] = ld16_any<POL_NT>(where, lane * 16);
      }
      from.advance(in, 1);
      to.advance(grad, 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    const float part = wave_reduce(live ? entry_loss(e, st, c1) : 0.0f, add);
    if (lane == 0) t.sum[wave_id()] = part;
    __syncthreads();
    if (now < rows) {
      if (listed && e.col >= 0) list.head[e.col / kTile<TI>] = -1;
      float total = t.sum[0];
#pragma unroll
      for (int i = 1; i < kMaxTeacher / 64; ++i) total += t.sum[i];
      write_row(loss, stats, r, live ? (total + rest_loss) * w : 0.0f, st);
    }
    if (next >= rows) return;
    now = next;
    next = after;
    w = w_next;
    e = {int32_t(f_next[0]), __uint_as_float(f_next[1]), int32_t(f_next[0]) >= 0 ? widen(z_next) : -kInf};
  }
}

// Several workgroups per row: a part's statistics.
template <typename TI, int NW, bool TAIL>
__global__ __launch_bounds__(NW * 64) void k_distill_scan(Logits in, emu_teacher_t te, float c1, Running* part, uint64_t row0) {
  extern __shared__ uint32_t bits[];
  __shared__ Running run[NW];
  const uint64_t r = row0 + blockIdx.x;
  if (te.weight && te.weight[r] == 0.0f) return;
  const Span block = part_of({0, tiles<TI>(in.V)}, blockIdx.y, gridDim.y);
  if constexpr (TAIL) mark_listed<NW>(bits, block.t0 * kTile<TI>, (block.t1 - block.t0) * kTile<TI>, fetch_teacher(te, r, in.V).col);
  const Running a = block_joined<NW>(scan<TI, NW, TAIL, POL_PLAIN>(in, r * in.row_bytes, block, c1, bits), run, c1);
  if (threadIdx.x == 0) part[uint64_t(blockIdx.x) * gridDim.y + blockIdx.y] = a;
}

// The row's statistics and loss from its parts'.
template <typename T, int NW, bool TAIL>
__global__ __launch_bounds__(NW * 64) void k_distill_join(Logits in, emu_teacher_t te, float c1, float* loss, float4* stats,
                                                          const Running* part, uint32_t parts, Prepared* teacher, float* rests, uint64_t row0) {
  __shared__ DistillLds<NW> t;
  const uint64_t r = row0 + blockIdx.x;
  const uint32_t lane = threadIdx.x & 63;
  const float w = te.weight ? te.weight[r] : 1.0f;
  if (w == 0.0f) return write_row(loss, stats, r, 0.0f, kSkipped);
  float rest, value;
  bool none;
  const Entry e = take_teacher<T, NW>(t, fetch_teacher(te, r, in.V), te, r, in, &rest, &none);
  const Running run = wave_joined(lane < parts ? part[uint64_t(blockIdx.x) * parts + lane] : Running{-kInf, 0.0f}, c1);
  const Stats st = finish<T, NW, TAIL>(in, r * in.row_bytes, run, e, rest, te.k, c1, t, &value);
  write_row(loss, stats, r, value * w, st);
  if (int(threadIdx.x) < te.k) teacher[blockIdx.x].entry[threadIdx.x] = {e.col, e.p};
  if (threadIdx.x == 0) rests[blockIdx.x] = none ? -1.0f : rest;
}

// The gradient of a part of a row, kBackwardTiles of it, from the row's statistics and prepared entries. Neighbouring
// workgroups have neighbouring parts: the whole device then writes one front, where copies ran at 6.3 TB/s against 5.7
// with a row per workgroup.
constexpr uint32_t kBackwardTiles = 16;
template <typename TI, typename TO, int NW>
__global__ __launch_bounds__(NW * 64) void k_distill_backward(Logits in, Logits grad, emu_teacher_t te, float c1, const float4* stats,
                                                              const Prepared* teacher, const float* rests, uint32_t parts, uint64_t row0) {
  static_assert(NW * 64 >= kMaxTeacher, "one entry per thread");
  const uint32_t row = blockIdx.x / parts, part = blockIdx.x - row * parts;
  const uint64_t r = row0 + row;
  const float w = te.weight ? te.weight[r] : 1.0f;
  const Span block = {part * kBackwardTiles, umin((part + 1) * kBackwardTiles, tiles<TI>(in.Vp))};
  __shared__ Listed<kBackwardTiles> list;
  Entry e = {-1, 0.0f, -kInf};
  Stats st = kSkipped;
  bool none = false;
  if (threadIdx.x < kBackwardTiles) list.head[threadIdx.x] = -1;
  if (w != 0.0f) {
    const float4 f = stats[r];
    st = {f.x, f.y, f.z, f.w};
    none = rests[row] < 0.0f;
    if (int(threadIdx.x) < te.k) {
      const Stored f = teacher[row].entry[threadIdx.x];
      const uint32_t tile = uint32_t(f.col) / kTile<TI>;
      if (f.col >= 0 && tile >= block.t0 && tile < block.t1) e = {f.col, f.value, widen(*column<TI>(in, r * in.row_bytes, f.col))};
    }
    asm volatile("" ::"v"(e.z));  // read before anyone writes, in place, behind the barrier
    __syncthreads();
  }
  row_gradient<TI, TO, kGradU, NW, POL_NT>(in, grad, r, block, list, e, st, c1, w, none);
}

// How many workgroups share a row: below kSharedRows rows as many as make kSharers in all, each with at least two tiles
// per wave, and always so many that a part's marks fit in LDS. Shared rows take a kernel more. Kernel times from graphs, us, shared / whole,
// bf16 rows of 128,256: 1 row, the k largest 13 / 15, the loss 11 / 16, with its gradient 16 / 25; 64 rows 15 / 18, 15 / 18,
// 25 / 27; 100 rows 19 / 18, 18 / 19, 31 / 28; 255 rows 25 / 20, 24 / 21, 47 / 38. 100 fp32 rows 21 / 25, 21 / 23, 39 / 37. Narrow rows
// gain little or lose: one of 32,768 9.6 / 10.2, 11.2 / 11.6, 15.5 / 18.1, one of 8,192 9.4 / 7.0, 11.1 / 9.4, 16.9 / 13.1. With 256 sharers the
// losses and gradients of 64 rows took 16 and 28, with 4,096 15 and 25, their k largest 21.
constexpr int64_t kSharedRows = 96, kSharers = 1024;
constexpr uint32_t kMarked = 1u << 18;  // columns
static uint32_t row_parts(const emu_logits_t* l, uint32_t V, int waves) {
  const uint32_t unit = uint32_t(waves) * 2 * (l->dtype == EMU_BF16 ? kTile<bf16_t> : kTile<float>);
  const uint32_t most = std::min((V + unit - 1) / unit, kMaxSplits);
  const int64_t wanted = l->rows < kSharedRows ? kSharers : 1;
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

// The waves of a workgroup that has a row: 16 tiles each where 4, 8 or 16 of them can hold the row that way.
static int row_waves(uint32_t n_tiles) { return n_tiles <= 4 * kResidentTiles ? 4 : n_tiles <= 8 * kResidentTiles ? 8 : 16; }

// f(waves) for a workgroup that has a row of that many tiles.
template <typename F>
static void by_waves(uint32_t n_tiles, F f) {
  switch (row_waves(n_tiles)) {
    case 4: f(std::integral_constant<int, 4>()); break;
    case 8: f(std::integral_constant<int, 8>()); break;
    default: f(std::integral_constant<int, 16>()); break;
  }
}

// f(input element, output element) for the two dtypes.
template <typename F>
static void by_types(int32_t in, int32_t out, F f) {
  if (in == EMU_BF16) out == EMU_BF16 ? f(bf16_t(), bf16_t()) : f(bf16_t(), float());
  else out == EMU_BF16 ? f(float(), bf16_t()) : f(float(), float());
}

constexpr int kPartWaves = 4;  // of a workgroup that has a part of a row

// 4,096 rows of 128,256: 4 / 8 / 16 waves 217 / 198 / 277 us
static int top_waves(uint32_t n_tiles) { return std::min(row_waves(n_tiles), 8); }
static uint32_t topk_parts(const emu_logits_t* l, uint32_t V) { return row_parts(l, V, kTopParts); }
static uint32_t distill_parts(const emu_logits_t* l, uint32_t V) { return row_parts(l, V, kPartWaves); }

// The workspace of the distillation calls.
struct DistillWorkspace {
  uint32_t* ticket;
  float* rests;       // [rows]
  Prepared* teacher;  // [rows]
  Running* part;      // [rows][parts]
  uint64_t bytes;
  DistillWorkspace(void* at, uint64_t rows, uint64_t parts) {
    uint8_t* p = static_cast<uint8_t*>(at);
    const uint64_t list = (rows + 63) / 64 * 256;
    ticket = reinterpret_cast<uint32_t*>(p);
    rests = reinterpret_cast<float*>(p + kWsAlign);
    teacher = reinterpret_cast<Prepared*>(p + kWsAlign + list);
    part = reinterpret_cast<Running*>(teacher + rows);
    bytes = kWsAlign + list + rows * (sizeof(Prepared) + parts * sizeof(Running));
  }
};

// Below, the row's own workgroup takes its teacher, a launch less. The loss alone: 33 us against 34 (prepared) for 511
// bf16 rows of 128,256, 57 against 53 for 1,000; narrow rows lose by the preparation: 36 against 39 for 2,048 of 32,768.
// With the gradient: 38 against 40 for 255 of 128,256, 62 against 58 for 384; 24 against 27 for 511 of 32,768.
constexpr int64_t kPreparedLossRows = 1024, kPreparedGradRows = 256;

// Whether k_distill_resident takes these rows. Reading them again (k_distill) costs less than it looks: the L2 still has a part
// of a row (28% of 201 KB), the last-level cache most of the rest by the times, and no row waits for another. Registers pay where
//  * there is no tail (its marks and second statistics spilled: 4,096 bf16 rows of 128,256 took 529 us held, 495 read again) and
//    the gradient is no wider than the logits (bf16 to fp32, 2 GiB: rows of 32,704 593 us held, 524 read again, of 128,448 558 and 556);
//  * a wave holds enough of them: rows of 4,032 bf16 columns (8 tiles) took 989 us held, 555 read again, 1 GiB in all; 40,896
//    (80 tiles, 8 waves of 10) 497 and 477 at 2 GiB, 51,136 (13 a wave) 477 and 485; fp32 from 64 tiles on (20,416, 80 tiles:
//    235 and 251 at 1 GiB, 12,224, 48 tiles: 254 and 267, but 158 and 153 at half of it);
//  * the call moves enough bytes that most of them miss the cache: bf16 rows of 128,448 took 156 us held and 153 read
//    again at 0.5 GiB read and written, 251 and 271 at 1 GiB, 460 and 504 at 2; fp32 rows of 64,192 87 and 86 at 0.25, 133
//    and 138 at 0.5, 226 and 253 at 1.
template <typename TI, typename TO, bool TAIL>
constexpr bool kMayStay = !TAIL && sizeof(TO) <= sizeof(TI);
template <typename TI, typename TO>
static bool worth_holding(const Logits& in, uint32_t rows) {
  const uint32_t n = tiles<TI>(in.V);
  const uint64_t bytes = uint64_t(rows) * in.V * (sizeof(TI) + sizeof(TO));
  return n >= 4u * kResidentTiles && (sizeof(TI) == 4 ? bytes >= 1u << 29 : n > 10u * uint32_t(row_waves(n)) && bytes >= 1u << 30);
}
template <typename TI>
static bool holds(const Logits& in, const Logits& out, uint64_t out_size) {
  uint64_t bits = in.row_bytes | out.row_bytes;
  for (uint32_t t = 0; t * in.cols < in.Vp; ++t) bits |= uint64_t(in.p[t]) | uint64_t(out.p[t]);
  return bits % 16 == 0 && in.cols % kE<TI> == 0 && in.cols >= kTile<TI> && tiles<TI>(in.Vp) == tiles<TI>(in.V) &&
         tiles<TI>(in.V) <= 16 * kResidentTiles && uint64_t(in.cols) * out_size < (1u << 30);
}

template <typename TI>
static void launch_backward(TI, int32_t dtype, uint32_t n, hipStream_t st, const Logits& li, const Logits& lo, const emu_teacher_t& te, float c1,
                            const float4* stats, const DistillWorkspace& ws, uint64_t r0) {
  const uint32_t parts = (tiles<TI>(li.Vp) + kBackwardTiles - 1) / kBackwardTiles;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(n * parts), dim3(kPartWaves * 64), 0, st, li, lo, te, c1, stats, ws.teacher, ws.rests, parts, r0);
  };
  if (dtype == EMU_BF16) launch(k_distill_backward<TI, bf16_t, kPartWaves>);
  else launch(k_distill_backward<TI, float, kPartWaves>);
}

static void launch_prepare(uint32_t n, hipStream_t st, const emu_teacher_t& te, uint32_t V, const DistillWorkspace& ws, uint64_t r0) {
  hipLaunchKernelGGL(k_prepare_teacher, dim3((n + kPrepareWaves - 1) / kPrepareWaves), dim3(kPrepareWaves * 64), 0, st, te, V, ws.teacher, ws.rests,
                     ws.ticket, n, r0);
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
  *bytes = k == 0 ? DistillWorkspace(nullptr, rows, parts).bytes : parts > 1 ? rows * parts * (sizeof(Running) + 64 * sizeof(uint64_t)) : 0;
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
    auto launch = [&](auto kernel, uint32_t slice, int threads) {
      const uint32_t slices = (li.Vp + slice - 1) / slice;
      over_rows(in->rows, [&](uint64_t r0, uint32_t n) {
        hipLaunchKernelGGL(kernel, dim3(n * slices), dim3(threads), 0, st, li, lo, *c, in_place, slices, r0);
      });
    };
    // long histories: larger slices, so that fewer workgroups go over them
    if (c->tokens && c->tokens_cols > kLongHistory) launch(k_constrain<decltype(ti), decltype(to), 1024, 16384>, 16384, 1024);
    else launch(k_constrain<decltype(ti), decltype(to), 512, 8192>, 8192, 512);
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
      auto launch = [&](auto kernel, int waves) {
        hipLaunchKernelGGL(kernel, dim3(n * parts), dim3(waves * 64), 0, st, l, uint32_t(k), c1, d_index, d_logprob, d_lse, run, keys, parts, r0);
      };
      using T = decltype(ti);
      if (parts > 1) {
        launch(k_topk<T, kTopParts>, kTopParts);
        hipLaunchKernelGGL((k_topk_join<T>), dim3(n), dim3(kTopParts * 64), 0, st, l, uint32_t(k), c1, d_index, d_logprob, d_lse, run, keys, parts, r0);
      } else {
        switch (top_waves(tiles<T>(l.V))) {
          case 4: launch(k_topk<T, 4>, 4); break;
          default: launch(k_topk<T, 8>, 8); break;
        }
      }
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
  const int n_cus = device_cus();
  if (n_cus <= 0) return fail(EMU_ERR_HIP, "cannot query the current device");
  const uint32_t cus = uint32_t(n_cus);
  float4* stats = reinterpret_cast<float4*>(d_stats);
  by_type(student->dtype, [&](auto ti) {
    using TI = decltype(ti);
    const uint32_t n_tiles = tiles<TI>(li.V);
    const size_t marks = teacher->tail ? size_t((n_tiles + parts - 1) / parts) * kTile<TI> / 8 : 0;
    over_rows(student->rows, [&](uint64_t r0, uint32_t n) {
      const DistillWorkspace ws(d_workspace, n, parts);
      auto by_tail = [&](auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        if (parts > 1) {
          hipLaunchKernelGGL((k_distill_scan<TI, kPartWaves, TAIL>), dim3(n, parts), dim3(kPartWaves * 64), marks, st, li, *teacher, c1, ws.part, r0);
          hipLaunchKernelGGL((k_distill_join<TI, kPartWaves, TAIL>), dim3(n), dim3(kPartWaves * 64), 0, st, li, *teacher, c1, d_loss, stats, ws.part,
                             parts, ws.teacher, ws.rests, r0);
          if (grad) launch_backward(ti, grad->dtype, n, st, li, lo, *teacher, c1, stats, ws, r0);
          return;
        }
        const bool prepared = student->rows >= (grad ? kPreparedGradRows : kPreparedLossRows);
        if (prepared) launch_prepare(n, st, *teacher, li.V, ws, r0);
        by_waves(n_tiles, [&](auto waves) {
          constexpr int NW = decltype(waves)::value;
          auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(n), dim3(NW * 64), marks, st, li, lo, *teacher, c1, d_loss, stats,
                               prepared ? ws.teacher : nullptr, ws.rests, r0);
          };
          if (!grad) return launch(k_distill<TI, TI, NW, TAIL, false>);
          by_type(grad->dtype, [&](auto to) {
            using TO = decltype(to);
            if constexpr (kMayStay<TI, TO, TAIL>) {
              if (prepared && worth_holding<TI, TO>(li, n) && holds<TI>(li, lo, sizeof(TO))) {
                hipLaunchKernelGGL((k_distill_resident<TI, TO, NW>), dim3(std::min(n, cus * (16 / NW))), dim3(NW * 64), 0, st, li, lo, *teacher, c1,
                                   d_loss, stats, ws.teacher, ws.rests, ws.ticket, n, r0);
                return;
              }
            }
            launch(k_distill<TI, TO, NW, TAIL, true>);
          });
        });
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
  const uint32_t parts = distill_parts(student, li.V);
  by_type(student->dtype, [&](auto ti) {
    over_rows(student->rows, [&](uint64_t r0, uint32_t n) {
      const DistillWorkspace ws(d_workspace, n, parts);
      launch_prepare(n, st, *teacher, li.V, ws, r0);
      launch_backward(ti, grad->dtype, n, st, li, lo, *teacher, c1, reinterpret_cast<const float4*>(d_stats), ws, r0);
    });
  });
  return hip_check("emu_distill_backward launch");
}

}  // extern "C"
