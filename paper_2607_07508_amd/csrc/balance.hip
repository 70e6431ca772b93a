// Balance loss of a mixture-of-experts router, its per-expert counts and its gradient. Per segment b (a
// packed trajectory, or the whole call) with n_b tokens that count and per token the k experts the router
// chose,
//   counts[b][e] = choices of expert e,   f_be = E counts[b][e] / (k n_b),
//   p_t = softmax(x_t) or sigmoid(x_t) / its sum,   P_be = mean of p_te over the segment,
//   loss = coef sum_b (n_b / N) sum_e f_be P_be = (coef / N) sum_t sum_e f_e p_te,
//   dx_tj = (coef / N) p_tj [(1 - sigmoid(x_tj))] (f_j - sum_e f_e p_te).
// f depends on the choices alone, so the logits are read once: the choices are counted first, then one pass
// forms loss and gradient of each token from registers. Bound by HBM: the logits in, their gradient out.
// Counts are integer atomics (their order does not show); the loss is summed in float64 in a fixed order. Exponentials
// and reciprocals are the hardware's, each within a unit of the last place of a float, and take no branches for ranges.
#include "common.hpp"
#include "launch.hpp"
#include "layout.hpp"
#include "reduce.hpp"
#include "segments.hpp"
#include "../../include/sao.h"

namespace sao {

constexpr int kBadSegments = 1, kBadExpert = 2;

// The segment of token t: the number of segments that end at or before it. Lane by lane, so that up to 64
// segments take one round of loads. Every lane of the wave gets it.
__device__ __forceinline__ int32_t segment_of(const int32_t* cu, int32_t B, int64_t t) {
  const int lane = threadIdx.x & 63;
  int32_t n = 0;
  for (int32_t i = lane; i < B; i += 64) n += cu[i + 1] <= t ? 1 : 0;
  n = wave_sum(n);
  return n < B - 1 ? n : B - 1;
}

// Choices and tokens that count among tokens [t0, t1) of one segment, added to `hist` (LDS) and returned per
// thread. Sets *wrong on an id that is no expert's.
template <int THREADS>
__device__ __forceinline__ int32_t count_span(const int32_t* ids, const uint8_t* mask, int64_t t0, int64_t t1, int32_t E,
                                              int32_t k, int32_t* hist, int32_t* wrong) {
  const int tid = threadIdx.x;
  int32_t n = 0;
  for (int64_t t = t0 + tid; t < t1; t += THREADS) n += !mask || mask[t] != 0 ? 1 : 0;
  auto one = [&](int32_t id) {
    if (id >= 0 && id < E)
      atomicAdd(&hist[id], 1);
    else if (id != -1)
      *wrong = 1;
  };
  if (k % 4 == 0 && (reinterpret_cast<uintptr_t>(ids) & 15u) == 0) {  // four choices of one token at a time
    const int32_t k4 = k / 4;
#pragma unroll 4
    for (int64_t i = t0 * k4 + tid; i < t1 * k4; i += THREADS) {
      if (mask && mask[i / k4] == 0) continue;
      const v4u q = reinterpret_cast<const v4u*>(ids)[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) one(static_cast<int32_t>(q[j]));
    }
  } else {
    for (int64_t i = t0 * k + tid; i < t1 * k; i += THREADS)
      if (!mask || mask[i / k] != 0) one(ids[i]);
  }
  return n;
}

// Zeroes the counts and checks the segments.
static __global__ __launch_bounds__(256) void k_balance_init(const int32_t* cu, int32_t B, int64_t T, int32_t E,
                                                             int32_t* counts, int32_t* seg_tokens, int32_t* bad,
                                                             int32_t* status) {
  const int64_t i0 = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t i = i0; i < static_cast<int64_t>(B) * E; i += step) counts[i] = 0;
  for (int64_t i = i0; i < B; i += step) seg_tokens[i] = 0;
  if (blockIdx.x != 0) return;
  const bool b = cu ? segments_bad<256>(cu, B, T) : false;
  if (threadIdx.x == 0) {
    *bad = b ? kBadSegments : 0;
    if (b && status) atomicOr(status, SAO_STATUS_SEGMENTS);
  }
}

// The block's `span` tokens: a histogram in LDS per segment, added to the totals where the segment ends. Two blocks
// per CU: each ends with an atomic add per expert, which meet at one address per expert and segment (65,536 tokens
// of one segment: 1024 blocks took 12 us longer). 65,536 tokens of 8 choices take 9 us, 524,288 in 192 segments 16.
constexpr int kCountThreads = 512;
static __global__ __launch_bounds__(kCountThreads) void k_balance_count(const int32_t* ids, const uint8_t* mask,
                                                                        const int32_t* cu,
                                                                        int32_t B, int64_t T, int32_t E, int32_t k,
                                                                        int64_t span, int32_t* counts, int32_t* seg_tokens,
                                                                        int32_t* bad, int32_t* status) {
  __shared__ int32_t s_hist[kBalanceMaxExperts];
  __shared__ int32_t s_red[kCountThreads / 64];
  __shared__ int32_t s_bad;
  if (*bad & kBadSegments) return;  // uniform: cu cannot be walked
  const int tid = threadIdx.x;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * span, t1 = t0 + span < T ? t0 + span : T;
  if (tid == 0) s_bad = 0;
  int32_t b = cu ? segment_of(cu, B, t0) : 0;
  for (int64_t lo = t0; lo < t1; ++b) {
    int64_t hi = cu ? cu[b + 1] : T;
    if (hi > t1) hi = t1;
    if (hi <= lo) continue;
    for (int e = tid; e < E; e += kCountThreads) s_hist[e] = 0;
    __syncthreads();
    int32_t n = count_span<kCountThreads>(ids, mask, lo, hi, E, k, s_hist, &s_bad);
    n = block_sum<kCountThreads>(n, s_red);  // its barriers complete the histogram
    for (int e = tid; e < E; e += kCountThreads)
      if (s_hist[e]) atomicAdd(&counts[static_cast<int64_t>(b) * E + e], s_hist[e]);
    if (tid == 0 && n) atomicAdd(&seg_tokens[b], n);
    __syncthreads();
    lo = hi;
  }
  if (tid == 0 && s_bad) {
    atomicOr(bad, kBadExpert);
    if (status) atomicOr(status, SAO_STATUS_EXPERT_RANGE);
  }
}

// Element access: VEC elements of a row at once (16 bytes), or one.
template <class S, int VEC>
struct RowIo;
template <>
struct RowIo<uint16_t, 8> {
  __device__ static void load(const uint16_t* p, float (&x)[8]) {
    const v4u v = *reinterpret_cast<const v4u*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
  __device__ static void store(uint16_t* p, const float (&x)[8]) {
    v4u v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<v4u*>(p) = v;
  }
};
template <>
struct RowIo<float, 4> {
  __device__ static void load(const float* p, float (&x)[4]) {
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
  }
  __device__ static void store(float* p, const float (&x)[4]) {
    *reinterpret_cast<f32x4_t*>(p) = f32x4_t{x[0], x[1], x[2], x[3]};
  }
};
template <>
struct RowIo<uint16_t, 1> {
  __device__ static void load(const uint16_t* p, float (&x)[1]) { x[0] = __uint_as_float(static_cast<uint32_t>(*p) << 16); }
  __device__ static void store(uint16_t* p, const float (&x)[1]) { *p = static_cast<uint16_t>(pack_bf16x2(x[0], x[0])); }
};
template <>
struct RowIo<float, 1> {
  __device__ static void load(const float* p, float (&x)[1]) { x[0] = *p; }
  __device__ static void store(float* p, const float (&x)[1]) { *p = x[0]; }
};

// Reduction over groups of LANES lanes, every lane getting the result: quad and row permutations and gfx950's row
// and half swaps, all VALU (a shuffle through LDS waits some 100 cycles, fifteen of them per token).
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(v)), CTRL, 0xf, 0xf, true)));
}
template <int LANES, class Op>
__device__ __forceinline__ float lanes_reduce(float v, Op&& op) {
  static_assert(LANES >= 4 && LANES <= 64, "whole quads");
  v = op(v, dpp<0xB1>(v));                              // lane ^ 1
  v = op(v, dpp<0x4E>(v));                              // lane ^ 2
  if constexpr (LANES >= 8) v = op(v, dpp<0x141>(v));   // 7 - lane of 8: the other quad
  if constexpr (LANES >= 16) v = op(v, dpp<0x140>(v));  // 15 - lane of 16: the other eight
  if constexpr (LANES >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (LANES >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return v;
}
template <int LANES>
__device__ __forceinline__ float lanes_max(float v) {
  return lanes_reduce<LANES>(v, [](float x, float y) { return fmaxf(x, y); });
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
  return lanes_reduce<LANES>(v, [](float x, float y) { return x + y; });
}

// What the rows need of the counts.
struct BalanceStats {
  const int32_t* counts;
  const int32_t* seg_tokens;
  double c;   // coef / N, NaN after bad input
  bool walk;  // segments are there and can be walked
};

__device__ __forceinline__ double share_of(const BalanceArgs& a, int64_t N, int32_t wrong) {
  return wrong ? __builtin_nan("") : (N > 0 ? a.coef / static_cast<double>(N) : 0.0);
}

// Loss (the sum of sum_e f_e p_e, per lane) and gradient of tokens [w0, w1) by one wave: LANES lanes per token
// and ITER x VEC experts per lane, 64 / LANES tokens at once and kGroups such groups' loads in flight, the masks
// of the next ones ahead of them. A lane keeps f of its experts while its tokens stay in one segment. 524,288 tokens
// of 128 fp32 logits, seven tenths of them counted: 98 us, 4.8 TB/s, the rate of a large copy; 65,536 of 256 in bf16
// by sigmoid 32 us, 1.7 TB/s: too few tokens per wave to fill the wait for its first loads and the counts.
template <class S, int VEC, int LANES, int ITER, bool kSigmoid>
__device__ __forceinline__ double balance_rows(const BalanceArgs& a, const BalanceStats& st, int64_t w0, int64_t w1) {
  constexpr int kTokens = 64 / LANES;
  constexpr int kGroups = ITER * VEC <= 8 ? 4 : (ITER * VEC <= 16 ? 2 : 1);
  if (w0 >= w1) return 0.0;
  const int lane = threadIdx.x & 63;
  const int sub = lane % LANES;
  const int32_t E = a.E;
  const float c = static_cast<float>(st.c);
  const S* logits = static_cast<const S*>(a.logits);
  S* dlogits = static_cast<S*>(a.dlogits);
  double sum = 0.0;
  int32_t seg = st.walk ? segment_of(a.cu_seqlens, a.B, w0) : 0;
  int64_t seg_end = st.walk ? a.cu_seqlens[seg + 1] : a.T;
  float f[ITER][VEC];
  auto read_f = [&]() {
    const int32_t n = st.seg_tokens[seg];
    const int32_t* row = st.counts + static_cast<int64_t>(seg) * E;
#pragma unroll
    for (int i = 0; i < ITER; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int e = (i * LANES + sub) * VEC + j;
        f[i][j] = e < E ? static_cast<float>(row[e]) : 0.0f;
      }
    const float unit = n > 0 ? static_cast<float>(static_cast<double>(E) / (static_cast<double>(a.k) * n)) : 0.0f;
#pragma unroll
    for (int i = 0; i < ITER; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) f[i][j] *= unit;
  };
  read_f();
  // Which of the kGroups tokens from `base` count. The masks' loads carry no branch, so that they are in flight
  // together: past the end they read the last token's.
  auto counted = [&](int64_t base, bool (&to)[kGroups]) {
    uint8_t m[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int64_t t = base + g * kTokens + lane / LANES;
      m[g] = a.mask ? a.mask[t < w1 ? t : w1 - 1] : 1;
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) to[g] = base + g * kTokens + lane / LANES < w1 && m[g] != 0;
  };
  bool on[kGroups];
  counted(w0, on);
  for (int64_t base = w0; base < w1; base += kGroups * kTokens) {
    float x[kGroups][ITER][VEC];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int64_t t = base + g * kTokens + lane / LANES;
#pragma unroll
      for (int i = 0; i < ITER; ++i) {
        const int e = (i * LANES + sub) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[g][i][j] = -__builtin_inff();
        if (on[g] && e < E) RowIo<S, VEC>::load(logits + t * a.ld + e, x[g][i]);
      }
    }
    bool next[kGroups];
    counted(base + kGroups * kTokens, next);
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int64_t t = base + g * kTokens + lane / LANES;
      if (on[g] && t >= seg_end) {
        do {
          seg_end = a.cu_seqlens[++seg + 1];
        } while (t >= seg_end);
        read_f();
      }
      // p = w / S with w = e^(x - top), or sigmoid(x) e^(-top), top = min(max x, 0): neither over- nor
      // underflows where x is far below 0. slope = 1 - sigmoid(x). The difference comes before the factor of
      // log2 e, which would take the type's largest and lowest values (masked experts) out of float32.
      float top = -__builtin_inff();
#pragma unroll
      for (int i = 0; i < ITER; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) top = fmaxf(top, x[g][i][j]);
      top = lanes_max<LANES>(top);
      if (kSigmoid) top = fminf(top, 0.0f);
      // Where top is 0 for every token of the wave that counts, as almost always, e^(min(x, 0) - top) is 1 or e^-|x|.
      const bool shifted = kSigmoid && __ballot(on[g] && top != 0.0f) != 0;
      float slope[ITER][VEC];
      float s = 0.0f, d = 0.0f;
#pragma unroll
      for (int i = 0; i < ITER; ++i) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float v = x[g][i][j];  // -inf past the row's end: p = 0
          float p;
          if constexpr (kSigmoid) {
            const float q = fast_exp2(-fabsf(v) * kLog2e);  // e^-|x|
            const float r = __builtin_amdgcn_rcpf(1.0f + q);
            p = (v > 0.0f ? 1.0f : q) * r;
            if (shifted) p = fast_exp2((fminf(v, 0.0f) - top) * kLog2e) * r;
            slope[i][j] = (v > 0.0f ? q : 1.0f) * r;
          } else {
            p = fast_exp2((v - top) * kLog2e);
            slope[i][j] = 1.0f;
          }
          x[g][i][j] = p;
          s += p;
          d = fmaf(p, f[i][j], d);
        }
      }
      s = lanes_sum<LANES>(s);
      d = lanes_sum<LANES>(d);
      const float inv = __builtin_amdgcn_rcpf(s);
      const float each = d * inv;  // sum_e f_e p_e
      const float share = c * inv;
      if (on[g] && sub == 0) {
        sum += static_cast<double>(each);
        if (a.status && !__builtin_isfinite(each)) atomicOr(a.status, SAO_STATUS_NONFINITE);
      }
      if (t < w1 && dlogits) {
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
          const int e = (i * LANES + sub) * VEC;
          if (e >= E) continue;
          float gr[VEC];
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            gr[j] = on[g] ? (kSigmoid ? x[g][i][j] * slope[i][j] : x[g][i][j]) * (f[i][j] - each) * share : 0.0f;
          RowIo<S, VEC>::store(dlogits + t * E + e, gr);
        }
      }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) on[g] = next[g];
  }
  return sum;
}

template <class S, int VEC, int LANES, int ITER, bool kSigmoid>
__global__ __launch_bounds__(kBalanceThreads) void k_balance_rows(BalanceArgs a, int64_t span, const int32_t* seg_tokens,
                                                                  const int32_t* bad, double* part_loss) {
  __shared__ double s_red[kBalanceThreads / 64];
  __shared__ int64_t s_n[kBalanceThreads / 64];
  int64_t N = 0;
  if (a.n_tokens) {
    N = *a.n_tokens;
  } else {
    for (int i = threadIdx.x; i < a.B; i += kBalanceThreads) N += seg_tokens[i];
    N = block_sum<kBalanceThreads>(N, s_n);
  }
  const int32_t wrong = *bad;
  const BalanceStats st{a.counts, seg_tokens, share_of(a, N, wrong), a.cu_seqlens && !(wrong & kBadSegments)};
  const int64_t w0 = (static_cast<int64_t>(blockIdx.x) * (kBalanceThreads / 64) + (threadIdx.x >> 6)) * span;
  double sum = balance_rows<S, VEC, LANES, ITER, kSigmoid>(a, st, w0, w0 + span < a.T ? w0 + span : a.T);
  sum = block_sum<kBalanceThreads>(sum, s_red);
  if (threadIdx.x == 0) part_loss[blockIdx.x] = st.c * sum;
}

// loss (+)= the blocks' partial losses, in block order. (The block that ends last could do it, but a counter
// that 1024 blocks on 8 XCDs add to takes longer than this launch.)
static __global__ __launch_bounds__(256) void k_balance_total(const double* part_loss, int blocks, bool store,
                                                              double* loss) {
  __shared__ double s_red[4];
  double l = 0.0;
  for (int i = threadIdx.x; i < blocks; i += 256) l += part_loss[i];
  l = block_sum<256>(l, s_red);
  if (threadIdx.x == 0) loss[0] = (store ? 0.0 : loss[0]) + l;
}

// All of it in one block: a short batch is launches and little else (131 tokens of 128 experts: 7.5 us).
constexpr int kOneThreads = 1024;
template <class S, int VEC, int LANES, int ITER, bool kSigmoid>
__global__ __launch_bounds__(kOneThreads) void k_balance_one(BalanceArgs a) {
  __shared__ int32_t s_counts[kBalanceOneCounts];
  __shared__ int32_t s_tokens[kBalanceOneSegments];
  __shared__ int32_t s_red[kOneThreads / 64];
  __shared__ double s_sum[kOneThreads / 64];
  __shared__ int32_t s_bad;
  const int tid = threadIdx.x;
  for (int i = tid; i < a.B * a.E; i += kOneThreads) s_counts[i] = 0;
  for (int i = tid; i < a.B; i += kOneThreads) s_tokens[i] = 0;
  if (tid == 0) s_bad = 0;
  const bool bad = a.cu_seqlens ? segments_bad<kOneThreads>(a.cu_seqlens, a.B, a.T) : false;
  __syncthreads();
  int64_t N = 0;
  if (!bad) {
    for (int32_t b = 0; b < a.B; ++b) {
      const int64_t lo = a.cu_seqlens ? a.cu_seqlens[b] : 0, hi = a.cu_seqlens ? a.cu_seqlens[b + 1] : a.T;
      if (hi <= lo) continue;
      int32_t n = count_span<kOneThreads>(a.ids, a.mask, lo, hi, a.E, a.k, s_counts + b * a.E, &s_bad);
      n = block_sum<kOneThreads>(n, s_red);
      if (tid == 0) s_tokens[b] = n;
      N += n;
    }
  }
  __syncthreads();
  if (tid == 0 && a.status) {
    if (bad) atomicOr(a.status, SAO_STATUS_SEGMENTS);
    if (s_bad) atomicOr(a.status, SAO_STATUS_EXPERT_RANGE);
  }
  for (int i = tid; i < a.B * a.E; i += kOneThreads) a.counts[i] = s_counts[i];
  if (a.n_tokens) N = *a.n_tokens;
  const BalanceStats st{s_counts, s_tokens, share_of(a, N, (bad ? kBadSegments : 0) | s_bad), a.cu_seqlens && !bad};
  constexpr int kWaves = kOneThreads / 64, kTokens = 64 / LANES;
  const int64_t span = ((a.T + kTokens - 1) / kTokens + kWaves - 1) / kWaves * kTokens;
  const int64_t w0 = (tid >> 6) * span;
  double sum = balance_rows<S, VEC, LANES, ITER, kSigmoid>(a, st, w0, w0 + span < a.T ? w0 + span : a.T);
  sum = block_sum<kOneThreads>(sum, s_sum);
  if (tid == 0) a.loss[0] = (a.loss_store ? 0.0 : a.loss[0]) + st.c * sum;
}

template <class S, int VEC, int LANES, int ITER>
static void launch_rows(const BalanceArgs& a, hipStream_t st) {
  if (a.T * a.E <= kBalanceOneLogits && static_cast<int64_t>(a.B) * a.E <= kBalanceOneCounts &&
      a.B <= kBalanceOneSegments) {
    const auto one = a.sigmoid ? k_balance_one<S, VEC, LANES, ITER, true> : k_balance_one<S, VEC, LANES, ITER, false>;
    hipLaunchKernelGGL(one, dim3(1), dim3(kOneThreads), 0, st, a);
    return;
  }
  const BalanceLayout L = balance_layout(a.B);
  char* w8 = static_cast<char*>(a.ws);
  int32_t* bad = reinterpret_cast<int32_t*>(w8 + L.bad);
  int32_t* seg_tokens = reinterpret_cast<int32_t*>(w8 + L.seg_tokens);
  double* part = reinterpret_cast<double*>(w8 + L.part_loss);
  int64_t zero_blocks = ceil_div(static_cast<int64_t>(a.B) * a.E, 2048);
  if (zero_blocks > 256) zero_blocks = 256;
  hipLaunchKernelGGL(k_balance_init, dim3(static_cast<unsigned>(zero_blocks)), dim3(256), 0, st, a.cu_seqlens, a.B, a.T,
                     a.E, a.counts, seg_tokens, bad, a.status);
  const int64_t count_span = round_up(ceil_div(a.T, 2 * kGpuCus), 64);
  hipLaunchKernelGGL(k_balance_count, dim3(static_cast<unsigned>(ceil_div(a.T, count_span))), dim3(kCountThreads), 0, st, a.ids,
                     a.mask, a.cu_seqlens, a.B, a.T, a.E, a.k, count_span, a.counts, seg_tokens, bad, a.status);
  constexpr int kTokens = 64 / LANES;
  // tokens per wave: whole turns, at most kBalanceMaxBlocks blocks
  const int64_t span = ceil_div(ceil_div(a.T, kTokens), kBalanceMaxBlocks * (kBalanceThreads / 64)) * kTokens;
  const unsigned blocks = static_cast<unsigned>(ceil_div(a.T, span * (kBalanceThreads / 64)));
  const auto kernel = a.sigmoid ? k_balance_rows<S, VEC, LANES, ITER, true> : k_balance_rows<S, VEC, LANES, ITER, false>;
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kBalanceThreads), 0, st, a, span, seg_tokens, bad, part);
  hipLaunchKernelGGL(k_balance_total, dim3(1), dim3(256), 0, st, part, static_cast<int>(blocks), a.loss_store, a.loss);
}

// The fewest lanes whose 16-byte chunks cover a row, or 64 lanes and several chunks each.
template <class S>
static void launch_rows_any(const BalanceArgs& a, hipStream_t st) {
  constexpr int VEC = 16 / static_cast<int>(sizeof(S));
  const bool vec = a.E % VEC == 0 && a.ld % VEC == 0 && (reinterpret_cast<uintptr_t>(a.logits) & 15u) == 0 &&
                   (reinterpret_cast<uintptr_t>(a.dlogits) & 15u) == 0;
  if (vec) {
    const int chunks = a.E / VEC;
    if (chunks <= 4) return launch_rows<S, VEC, 4, 1>(a, st);
    if (chunks <= 8) return launch_rows<S, VEC, 8, 1>(a, st);
    if (chunks <= 16) return launch_rows<S, VEC, 16, 1>(a, st);
    if (chunks <= 32) return launch_rows<S, VEC, 32, 1>(a, st);
    if (chunks <= 64) return launch_rows<S, VEC, 64, 1>(a, st);
    if (chunks <= 128) return launch_rows<S, VEC, 64, 2>(a, st);
    if constexpr (sizeof(S) == 4) return launch_rows<S, VEC, 64, 4>(a, st);
  }
  if (a.E <= 16) return launch_rows<S, 1, 16, 1>(a, st);
  if (a.E <= 64) return launch_rows<S, 1, 64, 1>(a, st);
  if (a.E <= 256) return launch_rows<S, 1, 64, 4>(a, st);
  return launch_rows<S, 1, 64, 16>(a, st);
}

int launch_balance_loss(const BalanceArgs& a, hipStream_t st) {
  if (a.bf16)
    launch_rows_any<uint16_t>(a, st);
  else
    launch_rows_any<float>(a, st);
  return hipGetLastError();
}

}  // namespace sao
