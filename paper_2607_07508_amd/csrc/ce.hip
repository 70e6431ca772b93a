// Training losses on top of the LM head, each with its gradient: the softmax cross entropy of a target
// token and the distillation from a teacher's top logits. Both compare the softmax p over the whole
// vocabulary with a sparse distribution q,
//   z = W h / tau,   p = exp(z - lse),   dL/dz_v = a p_v - b q_v   per token,
// so they share every kernel but the one that forms a, b and the loss.
//
// The tokens that count are compacted and go through the head in chunks of rows. Per chunk
//   (A) z = W . h over 256 x 256 tiles (vocabulary x tokens) on MFMA; the epilogue reduces each half
//       tile (128 vocabulary rows) to (reference r, sum of 2^(z - r)) per token and stores the
//       exponentials themselves, in 16 bits for bf16 operands;
//   (B) per token: the halves' pairs merged to lse, the loss, a, and the values a p - b q at q's entries;
//   (C) dz = a 2^r / sum 2^z x stored exponential, in place, with q's entries overwritten;
//   (D) dH = dz . W and dW (+)= dz^T . H on MFMA.
// Three products of tokens x H x V, where recomputing the logits once lse is known takes four: at 8192
// rows of the 2048 x 151,936 head (C) moves 5 GB, a quarter of the time of the product it replaces, and
// the logits themselves never reach memory.
//
// Rounding (bf16 operands): the exponentials are kept as fp16, scaled so that a half tile's largest is
// 2^15: 11 significand bits down to 2^-29 of it, an absolute 2^-39 of it below. dz, q's entries and a token's weight
// within it, is rounded once more, to bf16 as an operand of the matrix instructions, also for a float32 dW: its 8
// bits dominate (0.0017 of a gradient's norm, as much as a bf16 result's own rounding). lse and the loss come from
// the unrounded sums. The mean's 1 / N (and tau)
// multiply the gradients' sums: in dz they would be rounded alike in every token whose p is small against 1,
// as much as 2^-8 off in all of them. Referring to the half tile's own maximum keeps logits in range without a
// row maximum known beforehand: of magnitudes up to 1.8e8 (kMaxRef), where float32 logits lie 16 apart; rows whose
// log-sum-exp is beyond that are NaN and flagged, halves beyond it below their row's largest are 0.
#include "common.hpp"
#include "head.hpp"
#include "launch.hpp"
#include "layout.hpp"
#include "reduce.hpp"
#include "../../include/sao.h"

namespace sao {

constexpr float kLn2 = 0.6931471805599453f;
// log2 of the scale of the stored exponentials.
template <class E>
constexpr float kExpShift = sizeof(typename E::storage) == 2 ? 15.0f : 0.0f;
// The largest log-sum-exp of a row, in log2 units. Below it a reference's spacing is 16 for bf16 (64 for fp32), so a
// half's largest exponential is stored as at least 2^-0.5 (2^-63.5): within fp16, and ahead of what underflows.
template <class E>
constexpr float kMaxRef = sizeof(typename E::storage) == 2 ? 0x1p28f : 0x1p30f;

// The reference of a half tile with maximum `top`: sc top less the shift, as a float; the exponents' distances from it
// are exact up to their own rounding. From 2^24 on its rounding is of the shift's size and would take the largest
// exponential out of fp16: there it is the float above. A half without a logit above -inf is taken relative to 0, one
// whose reference would be below every float relative to the lowest (its exponentials are 0).
template <class E>
__device__ __forceinline__ float half_reference(float top, float sc) {
  if (top == -__builtin_inff()) return 0.0f;
  const float ref = fmaxf(fmaf(top, sc, -kExpShift<E>), -__FLT_MAX__);
  if (fmaf(top, sc, -ref) > kExpShift<E> + 0.5f) return __uint_as_float(__float_as_uint(ref) + (ref > 0.0f ? 1u : ~0u));
  return ref;
}
// Its pair: of a half without a logit above -inf (-inf, 0) unless a NaN is among them.
__device__ __forceinline__ float2 half_pair(float top, float ref, float s) {
  return make_float2(top == -__builtin_inff() && s == 0.0f ? -__builtin_inff() : ref, s);
}

// ------------------------------------------------------------------------- //
// (A) logits, exponentials and their sums
// ------------------------------------------------------------------------- //
// Two floats as packed fp16, rounded to nearest even.
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const f16x2_t v = {static_cast<_Float16>(lo), static_cast<_Float16>(hi)};
  return __builtin_bit_cast(uint32_t, v);
}

// kMasked: the last, partial vocabulary tile; rows at or past M read as -inf and store zeros. kStore:
// whether the exponentials are kept (a gradient is wanted).
template <class E, bool kMasked, bool kStore>
struct EpiExp {
  typename E::storage* ex;  // [token row][vocabulary row], row stride lde
  int64_t lde;
  float2* part;             // [half tile][ldp]: (reference, sum), log2 units
  int64_t ldp;
  int64_t M;                // valid vocabulary rows of this launch's tiles
  int64_t tile0;            // vocabulary tile of the first of them
  float scale;              // log2(e) / tau

  __device__ __forceinline__ void begin(int64_t, int, int, int) {}
  __device__ __forceinline__ void settle() {}

  __device__ __forceinline__ void tile(f32x16_t (&acc)[kMI][kNI], float factor, int64_t m0, int64_t n0, int wm, int wn,
                                       int lane, void*) {
    // Never taken. The branch keeps the epilogue in a block of its own: joined to the K loop's end, the compiler
    // moves all accumulators to VGPRs ahead of it and, for fp32, spills 1000 of them.
    int never = 0;
    asm volatile("" : "+s"(never));
    if (never) return;
    const float sc = factor * scale;  // > 0
    int lim = kBM;
    if constexpr (kMasked) {
      // Valid rows from this lane's first one.
      const int64_t left = M - m0 - wm * (kBM / 2) - 4 * (lane >> 5);
      lim = left > kBM ? kBM : static_cast<int>(left);
    }
#pragma unroll
    for (int ni = 0; ni < kNI; ++ni) {
      // Kept apart per column: shared, the 64 comparisons would lie in 128 scalar registers, which spill.
      if constexpr (kMasked) asm volatile("" : "+v"(lim));
      float z[kMI * 16];
#pragma unroll
      for (int mi = 0; mi < kMI; ++mi)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = acc_read(acc[mi][ni][r]);
          z[mi * 16 + r] = !kMasked || mi * 32 + (r & 3) + 8 * (r >> 2) < lim ? x : -__builtin_inff();
        }
      const int64_t col = n0 + acc_col(wn, ni, lane);
      float top = -__builtin_inff();
#pragma unroll
      for (int i = 0; i < kMI * 16; ++i) top = fmaxf(top, z[i]);
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float ref = half_reference<E>(top, sc);
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < kMI * 16; ++i) {
        z[i] = fast_exp2(fmaf(z[i], sc, -ref));
        s += z[i];
      }
      s += __shfl_xor(s, 32, 64);
      if (lane < 32)
        part[(2 * (tile0 + m0 / kBM) + wm) * ldp + col] = half_pair(top, ref, s);
      if constexpr (kStore) {
        typename E::storage* row = ex + col * lde + (tile0 * kBM + m0 + wm * (kBM / 2));
        if constexpr (sizeof(typename E::storage) == 2) {
          // 16-byte stores: of register groups 2p and 2p + 1 (rows 16p + 4h .. +3 and 16p + 8 + 4h .. +3
          // of lane half h) the halves trade one each, so that a lane holds 8 consecutive rows.
#pragma unroll
          for (int mi = 0; mi < kMI; ++mi)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              const float* d0 = z + mi * 16 + 8 * p;
              const float* d1 = d0 + 4;
              const auto lo = __builtin_amdgcn_permlane32_swap(pack_f16x2(d0[0], d0[1]), pack_f16x2(d1[0], d1[1]),
                                                               false, false);
              const auto hi = __builtin_amdgcn_permlane32_swap(pack_f16x2(d0[2], d0[3]), pack_f16x2(d1[2], d1[3]),
                                                               false, false);
              *reinterpret_cast<v4u*>(row + mi * 32 + 16 * p + 8 * (lane >> 5)) = v4u{lo[0], hi[0], lo[1], hi[1]};
            }
        } else {
#pragma unroll
          for (int mi = 0; mi < kMI; ++mi)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float* d = z + mi * 16 + 4 * j;
              *reinterpret_cast<float4*>(row + mi * 32 + 8 * j + 4 * (lane >> 5)) = make_float4(d[0], d[1], d[2], d[3]);
            }
        }
      }
    }
  }

  __device__ __forceinline__ void finish(int, int64_t, int, int, int, void*) {}
};

// Up to two token tiles the products are bound by reading W, each of its tiles by one or two workgroups, and vocabulary
// tiles start K at slabs of their own: rows 2 H bytes apart make workgroups in step read from the same memory channels
// (256 rows of 2048 x 151,936 264 -> 219 us, of 6144 695 -> 570; 300 of 6144 914 -> 825). With more token tiles
// the workgroups that share a tile of W keep in step, in a kernel without the wrap (4096 rows: 2055 us, 2102 with).
constexpr int kRotateMaxTokenTiles = 2;
// XCD x takes tiles x, x + 8, ..., its workgroups in turn: slab i + 4 x for the i-th of them.
__device__ __forceinline__ int rotated_slab(int mt, int nk) {
  return static_cast<int>((static_cast<unsigned>(mt) / 8 + 4 * (static_cast<unsigned>(mt) & 7)) % static_cast<unsigned>(nk));
}
struct PlainTiles : PullTiles {};
struct RotatedTiles : PullTiles {
  __device__ __forceinline__ int first_slab(int mt, int nk) const { return rotated_slab(mt, nk); }
};
// The tiles are pulled per XCD from its list (PullTiles), those of a partial last vocabulary tile
// (st.m > 0) after the whole ones, which stream. Bound by the MFMAs under the power limit: 4178 rows of 2048 x
// 151,936 2.25 ms, 1.16 PFLOP/s; 8192 of 6144 x 151,552 11.3 ms, 1.36.
template <class E, bool kStore, class Tiles>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(1, 1)))
void k_exp_logits(GemmShape s, GemmShape st, EpiExp<E, false, kStore> epi, EpiExp<E, true, kStore> epi_t,
                  int32_t* next) {
  __shared__ v4u lds[kStages][kStageChunks];
  __shared__ int32_t s_idx;
  const int xcd = static_cast<int>(blockIdx.x & 7);
  const int64_t n_valid = *s.n_dev;
  const int64_t nv64 = (n_valid + kBN - 1) / kBN;
  const int nv = static_cast<int>(nv64 < s.n_tiles ? nv64 : s.n_tiles);
  const int mx = xcd < s.m_tiles ? (s.m_tiles - 1 - xcd) / 8 + 1 : 0;
  const int32_t total = mx * nv;
  const int32_t tail = st.m > 0 && xcd < nv ? (nv - 1 - xcd) / 8 + 1 : 0;
  TileClock clock;
  Tiles tiles{{next + xcd, &s_idx, nullptr, mx, nv, xcd, total, 0, 0, &clock, nullptr, 0, s.n_tiles, 0, 0, 0, 0}};
  tiles.claim();
  tiles.idx = tiles.publish();
  if (tiles.idx < total) {
    int mt, n_tile;
    tiles.locate(mt, n_tile);
    gemm_tiles<E, false, false>(s, epi, lds, mt, n_tile, 0, tiles);
  }
  int32_t idx = tiles.idx;
  while (idx < total + tail) {
    gemm_tile<E, false, false>(st, epi_t, lds, 0, (idx - total) * 8 + xcd);
    tiles.claim();
    idx = tiles.publish();
  }
}

// The same for few rows, up to 16 NT: bound by reading W once. Of 2048 x 151,936 (622 MB), in calls for dH: 1 / 64 /
// 128 rows 134 / 159 / 240 us, by whole tiles 64 / 128 / 256 rows 188 / 194 / 204; of 6144 (1867 MB) 342 / 415 / 612, by
// whole tiles 510 / 520 / 528. (Behind a call that wrote dW, the first takes 186 us: 3.4 TB/s.) A block takes a half tile, 128 vocabulary
// rows, 32 per wave as two 16-row MFMA operands loaded straight into registers, 256 contiguous bytes of a row per
// stage, the next stage's on their way during this one's products; the tokens' stage is staged through LDS, twice
// buffered. Rows lie 2 H bytes apart, a multiple of the memory channels' interleave where H is one of 2048, so
// every block starts at another stage of K and wraps around: in step, all blocks would read from the same channels.
// Four blocks' worth of waves per CU finish at different times, where whole tiles (594 of them for 256 CUs) leave
// two thirds of the CUs idle in the last round. Also writes the targets' logits (CE), from the accumulators, so
// that they agree with the terms of the sum. fp32 operands go through the fp32 MFMA, four K at a time: up to 64
// rows its rate (256 flop/clk/CU) hides under the reads: 1 / 32 / 64 rows of 2048 x 151,936 (1245 MB) 232 / 281 / 449
// us, 64 by whole tiles 715; of 1024 x 50,257 64 rows 91, 65 by whole tiles 148. A short pass takes it for any number
// of rows, a group of 16 NT per blockIdx.y, where that makes no more than one block per CU: whole tiles would leave
// most CUs idle, and the tile engine's code takes longer to fetch (163 rows of 64 x 1000 in fp32: 9.5 and 23 us; 256 of
// 2048 x 8000 105 and 230; bf16: 512 of 2048 x 8000 45 and 49, where 1024 would be two blocks per CU, 82 against 54).
constexpr int64_t kFewRows = 64;
constexpr int64_t kFewBlocks = kGpuCus;
// Rows that a block of k_exp_logits_few takes in a call of T tokens, and whether such blocks are used.
template <class E>
constexpr int64_t few_group(int64_t T) {
  return T <= 16 ? 16 : (T <= 32 ? 32 : (T <= 64 || sizeof(typename E::storage) == 4 ? 64 : 128));
}
template <class E>
constexpr bool few_rows(int64_t T, const HeadLossLayout& L) {
  return L.chunks == 1 && (T <= kFewRows || (T + few_group<E>(T) - 1) / few_group<E>(T) * 2 * L.m_tiles <= kFewBlocks);
}
constexpr int kFewStageChunks = 16;                 // 16-byte chunks of a row per stage
constexpr int kFewPitch = kFewStageChunks + 1;      // spreads 16 tokens' chunks over the LDS banks
template <class E, int NT, bool kStore>
__global__ __launch_bounds__(256) void k_exp_logits_few(const typename E::storage* w, int64_t ld_w, int64_t V,
                                                        const typename E::storage* hc, int64_t H, const int32_t* rows,
                                                        typename E::storage* ex, int64_t lde, float2* part, int64_t ldp,
                                                        float scale, const int32_t* idx, const int32_t* target,
                                                        float* zy) {
  constexpr bool k16 = sizeof(typename E::storage) == 2;
  constexpr int kTokens = 16 * NT;
  constexpr int kCopies = kTokens * kFewStageChunks / 256;  // chunks of a token stage per thread
  static_assert(kTokens * kFewStageChunks % 256 == 0, "whole chunks per thread");
  __shared__ v4u s_h[2][kTokens * kFewPitch];
  __shared__ float s_top[4][kTokens], s_sum[4][kTokens];
  const int t0 = static_cast<int>(blockIdx.y) * kTokens;  // this block's tokens
  const int n = *rows - t0 < kTokens ? *rows - t0 : kTokens;
  if (n <= 0) return;  // uniform
  hc += static_cast<int64_t>(t0) * H;
  ex += static_cast<int64_t>(t0) * lde;
  part += t0;
  idx += t0;
  zy += t0;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r16 = lane & 15, g = lane >> 4;
  const int64_t v0 = static_cast<int64_t>(blockIdx.x) * kHalfTile + wave * 32;
  const int64_t chunks = H / E::kPerChunk;
  const int stages = static_cast<int>((chunks + kFewStageChunks - 1) / kFewStageChunks);
  const v4u* wr[2];
#pragma unroll
  for (int f = 0; f < 2; ++f) {  // rows past the vocabulary read its last one
    const int64_t v = v0 + f * 16 + r16;
    wr[f] = reinterpret_cast<const v4u*>(w + (v < V ? v : V - 1) * ld_w);
  }
  // Chunk `at` of a row, zeros past its end.
  auto chunk = [&](const v4u* row, int64_t at) { return at < chunks ? row[at] : zero4(); };
  v4u a[2][4], b[kCopies];
  auto load = [&](int stage, v4u (&to)[2][4]) {
    const int64_t c0 = static_cast<int64_t>(stage) * kFewStageChunks;
    if (c0 + kFewStageChunks <= chunks) {  // uniform
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int j = 0; j < 4; ++j) to[f][j] = wr[f][c0 + 4 * j + g];
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        const int q = tid + 256 * i, t = q / kFewStageChunks;
        b[i] = reinterpret_cast<const v4u*>(hc + static_cast<int64_t>(t < n ? t : n - 1) * H)[c0 + q % kFewStageChunks];
      }
    } else {
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int j = 0; j < 4; ++j) to[f][j] = chunk(wr[f], c0 + 4 * j + g);
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        const int q = tid + 256 * i, t = q / kFewStageChunks;
        b[i] = chunk(reinterpret_cast<const v4u*>(hc + static_cast<int64_t>(t < n ? t : n - 1) * H), c0 + q % kFewStageChunks);
      }
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int q = tid + 256 * i;
      s_h[buf][q / kFewStageChunks * kFewPitch + q % kFewStageChunks] = b[i];
    }
  };
  f32x4_t acc[2][NT];
#pragma unroll
  for (int f = 0; f < 2; ++f)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[f][t] = f32x4_t{};
  auto multiply = [&](const v4u (&x)[2][4], int buf) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const v4u h = s_h[buf][(t * 16 + r16) * kFewPitch + 4 * j + g];
        if constexpr (k16) {
#pragma unroll
          for (int f = 0; f < 2; ++f)
            acc[f][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x[f][j]),
                                                                __builtin_bit_cast(bf16x8_t, h), acc[f][t], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int f = 0; f < 2; ++f)
              acc[f][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[f][j][e]), __uint_as_float(h[e]),
                                                               acc[f][t], 0, 0, 0);
        }
      }
  };
  const int first = static_cast<int>(blockIdx.x) % stages;
  auto stage_at = [&](int i) { return first + i < stages ? first + i : first + i - stages; };
  v4u next[2][4];
  load(stage_at(0), a);
  put(0);
  __syncthreads();
  for (int i = 0; i < stages; i += 2) {
    if (i + 1 < stages) load(stage_at(i + 1), next);
    multiply(a, 0);
    if (i + 1 >= stages) break;
    put(1);
    __syncthreads();
    if (i + 2 < stages) load(stage_at(i + 2), a);
    multiply(next, 1);
    if (i + 2 < stages) put(0);
    __syncthreads();
  }
  // Lane (r16, g), register r of operand f: vocabulary row v0 + 16 f + 4 g + r, token 16 t + r16.
  const int64_t left = V - v0 - 4 * g;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int tok = t * 16 + r16;
    if (target && tok < n) {
      const int64_t at = static_cast<int64_t>(target[idx[tok]]) - v0 - 4 * g;
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (at == 16 * f + r && at < left) zy[tok] = acc[f][t][r];
    }
    float top = -__builtin_inff();
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (16 * f + r >= left) acc[f][t][r] = -__builtin_inff();
        top = fmaxf(top, acc[f][t][r]);
      }
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    if (g == 0) s_top[wave][tok] = top;
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int tok = t * 16 + r16;
    const float top = fmaxf(fmaxf(s_top[0][tok], s_top[1][tok]), fmaxf(s_top[2][tok], s_top[3][tok]));
    const float ref = half_reference<E>(top, scale);
    float s = 0.0f;
#pragma unroll
    for (int f = 0; f < 2; ++f) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        acc[f][t][r] = fast_exp2(fmaf(acc[f][t][r], scale, -ref));
        s += acc[f][t][r];
      }
      if constexpr (kStore) {
        typename E::storage* to = ex + static_cast<int64_t>(tok) * lde + v0 + 16 * f + 4 * g;
        if (tok < n) {
          if constexpr (k16)
            *reinterpret_cast<uint2*>(to) =
                make_uint2(pack_f16x2(acc[f][t][0], acc[f][t][1]), pack_f16x2(acc[f][t][2], acc[f][t][3]));
          else
            *reinterpret_cast<f32x4_t*>(to) = acc[f][t];
        }
      }
    }
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    if (g == 0) s_sum[wave][tok] = s;
  }
  __syncthreads();
  if (tid < kTokens && tid < n) {
    const float top = fmaxf(fmaxf(s_top[0][tid], s_top[1][tid]), fmaxf(s_top[2][tid], s_top[3][tid]));
    const float s = (s_sum[0][tid] + s_sum[1][tid]) + (s_sum[2][tid] + s_sum[3][tid]);
    part[static_cast<int64_t>(blockIdx.x) * ldp + tid] = half_pair(top, half_reference<E>(top, scale), s);
  }
}

// ------------------------------------------------------------------------- //
// Logits at the sparse entries
// ------------------------------------------------------------------------- //
// Valid rows of each chunk, from their total.
static __global__ __launch_bounds__(64) void k_chunk_counts(const int32_t* count, int64_t rows, int64_t chunks,
                                                            int32_t* chunk_counts) {
  for (int64_t i = threadIdx.x; i < chunks; i += 64) {
    const int64_t left = *count - i * rows;
    chunk_counts[i] = static_cast<int32_t>(left < 0 ? 0 : (left < rows ? left : rows));
  }
}

// The rows that count gathered into hc, zero-filled up to a whole token tile (the first gather_blocks
// blocks), and, for the cross entropy, the targets' logits zt[c] = h_c . W[y_c] (the others). For bf16 four rows
// a wave on MFMA, of which the diagonal is kept: the same products in the same order as in the logits' tiles, so
// that zt equals the term in the sum to the last bit and 1 - p keeps its digits when p is nearly 1. Targets in the
// first rotated_tiles vocabulary tiles start K where those do. For fp32 one row a wave; there p comes from the stored
// exponential. Targets outside [0, V): nothing reads their zt.
template <class E>
constexpr int kDotRows = sizeof(typename E::storage) == 2 ? 4 : 1;
template <class E>
__global__ __launch_bounds__(256) void k_gather_dots(const typename E::storage* src, int64_t ld_src, int64_t H,
                                                     const int32_t* idx, const int32_t* count, int64_t gather_blocks,
                                                     typename E::storage* hc, const typename E::storage* w, int64_t ld_w,
                                                     int64_t V, const int32_t* target, int64_t rotated_tiles,
                                                     float* zt) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = *count;
  const int64_t chunks = H / E::kPerChunk;
  if (blockIdx.x < gather_blocks) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 4 + wave;
    if (c >= round_up_dev(n, kRowPad)) return;
    v4u* d = reinterpret_cast<v4u*>(hc + c * H);
    const v4u* s = c < n ? reinterpret_cast<const v4u*>(src + static_cast<int64_t>(idx[c]) * ld_src) : nullptr;
    for (int64_t k = lane; k < chunks; k += 64) d[k] = s ? s[k] : zero4();
    return;
  }
  const int64_t c0 = ((blockIdx.x - gather_blocks) * 4 + wave) * kDotRows<E>;
  if (c0 >= n) return;
  if constexpr (sizeof(typename E::storage) == 2) {
    // 64 chunks of each of the four rows of both operands at a time, through LDS: a fragment read straight from
    // memory takes 16 bytes from each of four rows 2 H bytes apart, which wait for one another (104 us for 4178
    // rows of 2048).
    constexpr int kSpan = 64, kPitch = kSpan + 1;
    __shared__ v4u s_rows[4][8][kPitch];
    v4u(*sh)[kPitch] = s_rows[wave];
    const v4u* row[8];
    int64_t start[4];  // chunk of row i that comes first
    const int slabs = static_cast<int>(chunks / kRowChunks);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t t = idx[c0 + i < n ? c0 + i : n - 1];
      const int32_t y = target[t];
      start[i] = y >= 0 && y / kBM < rotated_tiles ? kRowChunks * rotated_slab(y / kBM, slabs) : 0;
      row[i] = reinterpret_cast<const v4u*>(w + (y >= 0 && y < V ? static_cast<int64_t>(y) : 0) * ld_w);
      row[4 + i] = reinterpret_cast<const v4u*>(src + t * ld_src);
    }
    const int half = lane >> 5, mine = lane & 3;
    f32x16_t acc{};
    v4u next[8];
    auto load = [&](int64_t k) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t at = k + lane + start[i & 3];
        next[i] = k + lane < chunks ? row[i][at < chunks ? at : at - chunks] : zero4();
      }
    };
    load(0);
    for (int64_t k = 0; k < chunks; k += kSpan) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sh[i][lane] = next[i];
      if (k + kSpan < chunks) load(k + kSpan);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave reads what it wrote itself
      const int steps = static_cast<int>(chunks - k < kSpan ? (chunks - k + 1) / 2 : kSpan / 2);
#pragma unroll 4
      for (int u = 0; u < steps; ++u) Mma<BF16>::run(acc, sh[mine][2 * u + half], sh[4 + mine][2 * u + half]);
    }
    // row i of column i, i < 4, is register i of lane i
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane == i && c0 + i < n) zt[c0 + i] = acc[i];
  } else {
    const int64_t t = idx[c0];
    const int32_t y = target[t];
    const v4u* h = reinterpret_cast<const v4u*>(src + t * ld_src);
    const v4u* r = reinterpret_cast<const v4u*>(w + (y >= 0 && y < V ? static_cast<int64_t>(y) : 0) * ld_w);
    float z = 0.0f;
#pragma unroll 4
    for (int64_t k = lane; k < chunks; k += 64) z += dot_chunk<E>(h[k], r[k]);
    z = wave_sum(z);
    if (lane == 0) zt[c0] = z;
  }
}

// zt[c][k] = h_c . W[id_k] / tau for kIds of a row's K ids per wave (blockIdx.y takes the next kIds), kIds
// rows of W in flight. Ids outside [0, V): NaN and the status bit, except -1 (no entry): -inf, which nothing
// reads. 5700 rows of 2048 by 64 ids: 249 us, 6.0 TB/s of rows of W, some of them from the caches.
constexpr int kIds = 8;
template <class E>
__global__ __launch_bounds__(256) void k_target_dots(const typename E::storage* hc, int64_t H,
                                                     const typename E::storage* w, int64_t ld_w, int64_t V,
                                                     const int32_t* idx, const int32_t* ids, int64_t ld_ids, int K,
                                                     const int32_t* count, float inv_tau, float* zt, int32_t* status) {
  const int lane = threadIdx.x & 63;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (c >= *count) return;
  const int k0 = static_cast<int>(blockIdx.y) * kIds;
  const int32_t* row_ids = ids + static_cast<int64_t>(idx[c]) * ld_ids;
  const v4u* h = reinterpret_cast<const v4u*>(hc + c * H);
  const v4u* wr[kIds];
  int32_t id[kIds];
  bool in[kIds];
#pragma unroll
  for (int j = 0; j < kIds; ++j) {
    id[j] = k0 + j < K ? row_ids[k0 + j] : -1;
    in[j] = id[j] >= 0 && id[j] < V;
    wr[j] = reinterpret_cast<const v4u*>(w + (in[j] ? static_cast<int64_t>(id[j]) : 0) * ld_w);
  }
  float acc[kIds] = {};
  const int64_t chunks = H / E::kPerChunk;
  for (int64_t i = lane; i < chunks; i += 64) {
    const v4u x = h[i];
#pragma unroll
    for (int j = 0; j < kIds; ++j)
      if (in[j]) acc[j] += dot_chunk<E>(x, wr[j][i]);
  }
#pragma unroll
  for (int j = 0; j < kIds; ++j) {
    const float z = wave_sum(acc[j]) * inv_tau;
    if (lane == 0 && k0 + j < K) {
      const bool none = id[j] == -1;
      if (!in[j] && !none && status) atomicOr(status, SAO_STATUS_TARGET_RANGE);
      zt[c * K + k0 + j] = in[j] ? z : (none ? -__builtin_inff() : __builtin_nanf(""));
    }
  }
}

// What the gradients' sums are multiplied by: factor / N, with N the caller's count or that of the call's rows.
struct MeanScale {
  const int64_t* n_tokens;  // or null: *total
  const int32_t* total;
  float factor;
  __device__ __forceinline__ float get() const {
    const int64_t N = n_tokens ? *n_tokens : *total;
    return N > 0 ? static_cast<float>(static_cast<double>(factor) / static_cast<double>(N)) : 0.0f;
  }
};

// ------------------------------------------------------------------------- //
// (B) loss and coefficients of a chunk's rows
// ------------------------------------------------------------------------- //
struct LossRows {
  const float2* part;
  int64_t ldp;
  int halves;
  const int32_t* idx;       // of the chunk's rows
  const int32_t* rows;      // valid rows of the chunk
  MeanScale mean;           // 1 / N
  const float* weight;      // or null
  const float* zt;          // [row][K]: logits at the sparse entries
  int K;
  int64_t V;
  const int32_t* ids;       // targets, or teacher ids and logits
  int64_t ld_ids;
  const float* teacher;
  int64_t ld_teacher;
  const float* teacher_lse;
  float tau, z_coef;
  float scale_z;            // log2(e), zt being logits / tau
  float max_ref;            // of a row that is not out of range
  const void* ex;           // the stored exponentials, row stride lde, fp16 or (f32) fp32
  bool f32;
  int64_t lde;
  float* token_loss;
  float* lse;
  float* ref;               // [row]: the largest reference of its halves, log2 units
  float* scale;             // [row]: a / sum of 2^(z - ref)
  float* patch;             // [row][K]: a p - b q at the sparse entries, or null (no gradient)
  double* part_loss;        // [block][2]
  int32_t* status;
};

// A row's log-sum-exp as 2^ref x sum. ref ln 2 is taken in two parts, so that a difference from a logit of
// about its size does not keep the rounding of the product.
struct RowLse {
  float ref, sum;
  static constexpr float kLn2Hi = 0.693145752f, kLn2Lo = 1.42860677e-06f;  // 17 bits, and the rest
  __device__ __forceinline__ float lse() const { return fmaf(ref, kLn2, logf(sum)); }
  // lse - z
  __device__ __forceinline__ float less(float z) const { return fmaf(ref, kLn2Hi, -z) + fmaf(ref, kLn2Lo, logf(sum)); }
};

// p at vocabulary row v, whose logit by a separate product is z. fp32: of the stored exponential, which the
// sum holds to the last bit; from z it would differ by a rounding, half as much again as the gradient's error
// without it. bf16: from z, which has more digits than the stored one, and for the cross entropy is the term in the sum
// itself. The distillation's differs from it by some 2^-23 of its size, from |z| of 2^12 on (log2 units) more
// than the 2^-11 that the stored one is rounded by, which is taken there.
template <bool kDistill>
__device__ __forceinline__ float sparse_p(const LossRows& a, const RowLse& l, int64_t r, int32_t v, float z) {
  const bool stored = a.f32 || (kDistill && fabsf(l.ref) >= 4096.0f);
  if (!stored) return fast_exp2(fmaf(z, a.scale_z, -l.ref)) / l.sum;
  const int64_t at = r * a.lde + v;
  const float e = a.f32 ? static_cast<const float*>(a.ex)[at] : static_cast<float>(static_cast<const _Float16*>(a.ex)[at]);
  return e * fast_exp2(a.part[static_cast<int64_t>(v / kHalfTile) * a.ldp + r].x - l.ref) / l.sum;
}

// Cross entropy: c = weight / N, loss c (lse - z_y) and z_coef c lse^2,
// N dz = weight ((1 + 2 z_coef lse) p - 1[y]).
__device__ __forceinline__ void ce_row(const LossRows& a, int64_t r, int64_t t, const RowLse& l, float weight,
                                       float inv_n, float& loss, double (&sum)[2]) {
  const float c = weight * inv_n;
  const int32_t y = a.ids[t];
  const bool ok = y >= 0 && y < a.V;
  if (!ok && a.status) atomicOr(a.status, SAO_STATUS_TARGET_RANGE);
  const float lse = l.lse();
  const float z = ok ? a.zt[r] : __builtin_nanf("");
  const float nll = l.less(z);
  const float zl = 2.0f * a.z_coef * lse;
  loss = nll;
  sum[0] += static_cast<double>(c) * nll;
  sum[1] += static_cast<double>(c) * a.z_coef * lse * lse;
  if (a.patch) {
    // a target outside the vocabulary makes the whole row's gradient NaN
    const float p = ok ? sparse_p<false>(a, l, r, y, z) : 0.0f;
    a.scale[r] = ok ? weight * (1.0f + zl) / l.sum : __builtin_nanf("");
    a.patch[r] = weight * ((p - 1.0f) + zl * p);
  }
}

// Distillation, one wave per row. With u = t / tau and q = exp(u - teacher lse) (the lse of the K logits
// themselves if none is given), KL = tau^2 sum q (log q - log p) and N / tau dz = weight (Q p - q), Q = sum q. An id
// that occurs twice carries the sum of its q: each of its entries writes the same value.
__device__ __forceinline__ void distill_row(const LossRows& a, int64_t r, int64_t t, const RowLse& l, float weight,
                                            float inv_n, int lane, int32_t* s_id, float* s_q, float& loss,
                                            double (&sum)[2]) {
  constexpr int kMine = kMaxTeacherIds / 64;
  const int32_t* ids = a.ids + t * a.ld_ids;
  const float* tl = a.teacher + t * a.ld_teacher;
  const float inv_tau = 1.0f / a.tau;
  float u[kMine], top = -__builtin_inff();
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int k = lane + 64 * j;
    const int32_t id = k < a.K ? ids[k] : -1;
    u[j] = id != -1 ? tl[k] * inv_tau : -__builtin_inff();
    if (k < a.K) s_id[k] = id;
    top = fmaxf(top, u[j]);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  float norm;
  if (a.teacher_lse) {
    norm = a.teacher_lse[t];
  } else {
    const float ref = top == -__builtin_inff() ? 0.0f : top;
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < kMine; ++j) s += expf(u[j] - ref);
    s = wave_sum(s);
    norm = top == -__builtin_inff() && s == 0.0f ? 0.0f : ref + logf(s);
  }
  float q[kMine], kl = 0.0f, Q = 0.0f;
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int k = lane + 64 * j;
    const float lq = u[j] - norm;
    q[j] = k < a.K ? expf(lq) : 0.0f;
    // q = 0 contributes 0 whatever its logits; an id outside the vocabulary has a NaN logit
    const float z = k < a.K ? a.zt[r * a.K + k] : 0.0f;
    if (q[j] != 0.0f) kl += q[j] * (lq + l.less(z));
    if (k < a.K && __builtin_isnan(z)) kl = __builtin_nanf("");
    Q += q[j];
    if (k < a.K) s_q[k] = q[j];
  }
  kl = wave_sum(kl) * a.tau * a.tau;
  Q = wave_sum(Q);
  loss = kl;
  sum[0] += static_cast<double>(weight * inv_n) * kl;
  if (!a.patch) return;
  if (lane == 0) a.scale[r] = __builtin_isnan(kl) ? __builtin_nanf("") : weight * Q / l.sum;
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int k = lane + 64 * j;
    if (k >= a.K) break;
    const int32_t id = s_id[k];
    float qs = 0.0f;
    for (int i = 0; i < a.K; ++i) qs += s_id[i] == id ? s_q[i] : 0.0f;
    const float p = id >= 0 && id < a.V ? sparse_p<true>(a, l, r, id, a.zt[r * a.K + k]) : 0.0f;
    a.patch[r * a.K + k] = weight * (Q * p - qs);
  }
}

// kLossRows rows per block. Phase 1: 256 / kLossRows threads a row merge its halves' pairs, thread q those of
// every 256 / kLossRows-th half from q in order, 8 loads in flight, then a fixed tree. With 16 rows a half's
// are one 128-byte run; few rows leave most CUs idle, and a block takes 4. Phase 2: the rows' losses. Sums are
// float64, in a fixed order.
template <bool kDistill, int kLossRows>
__global__ __launch_bounds__(256) void k_loss_rows(LossRows a) {
  constexpr int kPerRow = 256 / kLossRows, kInFlight = 8;
  __shared__ float2 s_ms[4][kLossRows];
  __shared__ RowLse s_lse[kLossRows];
  __shared__ double s_sum[4][2];
  __shared__ int32_t s_id[kDistill ? 4 : 1][kDistill ? kMaxTeacherIds : 1];
  __shared__ float s_q[kDistill ? 4 : 1][kDistill ? kMaxTeacherIds : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t n = *a.rows;
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * kLossRows;
  if (r0 >= n) {  // uniform over the block
    if (tid < 2) a.part_loss[2 * blockIdx.x + tid] = 0.0;
    return;
  }
  auto merge = [](float& m, float& s, float m2, float s2) {
    const float mn = fmaxf(m, m2);
    if (mn == -__builtin_inff()) return;
    s = s * fast_exp2(m - mn) + s2 * fast_exp2(m2 - mn);
    m = mn;
  };
  {
    const int row = tid % kLossRows, q = tid / kLossRows;
    const int64_t r = r0 + row;
    float m = -__builtin_inff(), s = 0.0f;
    if (r < n) {
      int g = q;
      for (; g + (kInFlight - 1) * kPerRow < a.halves; g += kInFlight * kPerRow) {
        float2 p[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) p[u] = a.part[static_cast<int64_t>(g + u * kPerRow) * a.ldp + r];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) merge(m, s, p[u].x, p[u].y);
      }
      for (; g < a.halves; g += kPerRow) {
        const float2 p = a.part[static_cast<int64_t>(g) * a.ldp + r];
        merge(m, s, p.x, p.y);
      }
    }
#pragma unroll
    for (int d = kLossRows; d < 64; d <<= 1) merge(m, s, __shfl_xor(m, d, 64), __shfl_xor(s, d, 64));
    if (lane < kLossRows) s_ms[wave][lane] = make_float2(m, s);
  }
  __syncthreads();
  const float inv_n = a.mean.get();
  if (tid < kLossRows) {
    float m = s_ms[0][tid].x, s = s_ms[0][tid].y;
#pragma unroll
    for (int q = 1; q < 4; ++q) merge(m, s, s_ms[q][tid].x, s_ms[q][tid].y);
    // (-inf stays: a row without a logit above it)
    const RowLse l{m, fabsf(m) >= a.max_ref && m != -__builtin_inff() ? __builtin_nanf("") : s};
    s_lse[tid] = l;
    if (r0 + tid < n) {
      if (a.patch) a.ref[r0 + tid] = m;
      if (a.status && !__builtin_isfinite(l.lse())) atomicOr(a.status, SAO_STATUS_NONFINITE);
    }
  }
  __syncthreads();
  double sum[2] = {0.0, 0.0};
  if constexpr (kDistill) {
    for (int j = wave; j < kLossRows; j += 4) {
      const int64_t r = r0 + j;
      if (r >= n) break;  // uniform over the wave
      const int64_t t = a.idx[r];
      const float weight = a.weight ? a.weight[t] : 1.0f;
      float loss;
      double row[2] = {0.0, 0.0};
      distill_row(a, r, t, s_lse[j], weight, inv_n, lane, s_id[wave], s_q[wave], loss, row);
      if (lane == 0) {
        sum[0] += row[0];
        a.token_loss[t] = loss;
        a.lse[t] = s_lse[j].lse();
      }
    }
  } else if (tid < kLossRows && r0 + tid < n) {
    const int64_t r = r0 + tid;
    const int64_t t = a.idx[r];
    const float weight = a.weight ? a.weight[t] : 1.0f;
    float loss;
    ce_row(a, r, t, s_lse[tid], weight, inv_n, loss, sum);
    a.token_loss[t] = loss;
    a.lse[t] = s_lse[tid].lse();
  }
  block_sums<256>(sum, s_sum);
  if (tid == 0) {
    a.part_loss[2 * blockIdx.x] = sum[0];
    a.part_loss[2 * blockIdx.x + 1] = sum[1];
  }
}

// loss (+)= the blocks' partial sums, in order.
static __global__ __launch_bounds__(256) void k_loss_total(const double* part, int64_t n, int slots, bool store,
                                                           double* loss) {
  __shared__ double sh[4][2];
  double s[2] = {0.0, 0.0};
  for (int64_t i = threadIdx.x; i < n; i += 256) {
    s[0] += part[2 * i];
    s[1] += part[2 * i + 1];
  }
  block_sums<256>(s, sh);
  if (threadIdx.x == 0)
    for (int j = 0; j < slots; ++j) loss[j] = (store ? 0.0 : loss[j]) + s[j];
}

// ------------------------------------------------------------------------- //
// (C) the logit gradient, in place of the exponentials
// ------------------------------------------------------------------------- //
// A block takes kDzRows rows of 256 x 16 bytes: first the factor a 2^r / sum 2^z of each row and half tile,
// then one 16-byte chunk per thread and row, then the sparse entries that fall into its columns. Bound by HBM: 4178
// rows of 151,936 in 16 bits 0.48 ms, 5.3 TB/s; 8192 of 151,552 1.0 ms, 4.9.
constexpr int kDzRows = 16;
__device__ __forceinline__ v4u scaled(const v4u& x, float f, BF16) {  // fp16 in, bf16 out
  v4u y;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t word = x[j];
    const f16x2_t e = __builtin_bit_cast(f16x2_t, word);
    y[j] = pack_bf16x2(f * static_cast<float>(e[0]), f * static_cast<float>(e[1]));
  }
  return y;
}
__device__ __forceinline__ v4u scaled(const v4u& x, float f, F32) {
  v4u y;
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = __float_as_uint(f * __uint_as_float(x[j]));
  return y;
}
template <class E>
__global__ __launch_bounds__(256) void k_exp_to_dz(typename E::storage* ex, int64_t lde, const float2* part,
                                                   int64_t ldp, const float* ref, const float* scale,
                                                   const float* patch, const int32_t* ids, int64_t ld_ids, int K,
                                                   const int32_t* idx, const int32_t* rows) {
  constexpr int P = E::kPerChunk;
  constexpr int kCols = 256 * P;
  constexpr int kHalves = kCols / kHalfTile;
  constexpr int kInFlight = 8;
  __shared__ float s_f[kHalves][kDzRows];
  const int tid = threadIdx.x;
  const int64_t n = *rows;
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * kDzRows;
  if (r0 >= n) return;  // uniform over the block
  const int left = static_cast<int>(n - r0 < kDzRows ? n - r0 : kDzRows);
  const int64_t col0 = static_cast<int64_t>(blockIdx.y) * kCols;
  for (int i = tid; i < kHalves * kDzRows; i += 256) {
    const int r = i % kDzRows, hf = i / kDzRows;
    float f = 0.0f;
    if (r < left && col0 + hf * kHalfTile < lde)
      f = scale[r0 + r] * fast_exp2(part[(col0 / kHalfTile + hf) * ldp + r0 + r].x - ref[r0 + r]);
    s_f[hf][r] = f;
  }
  __syncthreads();
  const int64_t col = col0 + tid * P;
  if (col < lde) {
    const int hf = tid * P / kHalfTile;
    typename E::storage* p = ex + r0 * lde + col;
    for (int g = 0; g < left; g += kInFlight) {
      v4u x[kInFlight];
#pragma unroll
      for (int u = 0; u < kInFlight; ++u)  // past the last row: read again, not stored
        x[u] = *reinterpret_cast<const v4u*>(p + (g + u < left ? g + u : left - 1) * lde);
#pragma unroll
      for (int u = 0; u < kInFlight; ++u)
        if (g + u < left) *reinterpret_cast<v4u*>(p + (g + u) * lde) = scaled(x[u], s_f[hf][g + u], E{});
    }
  }
  // every store of the block is complete before the entries overwrite some of what it wrote
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int i = tid; i < left * K; i += 256) {
    const int r = i / K, k = i - r * K;
    const int32_t id = ids[static_cast<int64_t>(idx[r0 + r]) * ld_ids + k];
    if (id < col0 || id >= col0 + kCols || id >= lde) continue;
    const float d = patch[(r0 + r) * K + k];
    typename E::storage* at = ex + (r0 + r) * lde + id;
    if constexpr (sizeof(typename E::storage) == 2)
      *at = static_cast<uint16_t>(pack_bf16x2(d, d));
    else
      *at = d;
  }
}

// ------------------------------------------------------------------------- //
// (D) gradients
// ------------------------------------------------------------------------- //
// out[m][n] = scale x acc, plus prev[m][n] (fp32) when given, rounded once to bf16 and stored 16 bytes a lane, a
// wave's 128 columns of four rows at a time, through the wave's own 32 KB of LDS. Lanes 2i and 2i + 1 hold columns
// 2i and 2i + 1 of the same rows: they trade one value of each pair of rows, so that the even lane has two
// columns of the first row and the odd lane two of the second. Chunk c of row r lies at c ^ swz(r), so that
// the four rows of a write (r, r + 1 and 4 further in the other lane half) meet different banks. dW of 2048 x
// 151,936 from 4178 rows takes 2.3 ms (1.13 PFLOP/s), of 6144 x 151,552 from 8192 11.6 ms (1.32).
struct EpiCast {
  uint16_t* out;
  const float* prev;
  int64_t ldo;
  int64_t m_valid;
  int64_t n_valid;  // a multiple of 8
  float scale;

  __device__ __forceinline__ void begin(int64_t, int, int, int) {}
  __device__ __forceinline__ static int swz(int row) { return ((row & 1) << 2) | ((row & 4) << 1); }

  __device__ __forceinline__ void tile(f32x16_t (&acc)[kMI][kNI], float factor, int64_t m0, int64_t n0, int wm, int wn,
                                       int lane, void* smem) {
    constexpr int kRowChunks16 = 16;  // 16-byte chunks of a wave's row
    factor *= scale;
    v4u* sh = static_cast<v4u*>(smem) + (wm * kWavesN + wn) * (kBM / 2) * kRowChunks16;
    const int odd = lane & 1, half = lane >> 5;
#pragma unroll
    for (int ni = 0; ni < kNI; ++ni) {
      const int64_t col = n0 + acc_col(wn, ni, lane);
      const int pair = ni * 16 + ((lane & 31) >> 1);  // 4-byte word of the row
#pragma unroll
      for (int mi = 0; mi < kMI; ++mi) {
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const int row = mi * 32 + (r & 3) + 8 * (r >> 2) + 4 * half;  // of the wave's 128
          float x0 = acc_read(acc[mi][ni][r]) * factor, x1 = acc_read(acc[mi][ni][r + 1]) * factor;
          if (prev) {
            const int64_t at = m0 + wm * (kBM / 2) + row;
            if (col < n_valid && at < m_valid) x0 += prev[at * ldo + col];
            if (col < n_valid && at + 1 < m_valid) x1 += prev[(at + 1) * ldo + col];
          }
          const float got = __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_update_dpp(
              0, static_cast<int>(__float_as_uint(odd ? x0 : x1)), 0xB1, 0xf, 0xf, true)));  // lane ^ 1
          const uint32_t two = pack_bf16x2(odd ? got : x0, odd ? x1 : got);
          const int to = row + odd;
          reinterpret_cast<uint32_t*>(sh + to * kRowChunks16 + ((pair >> 2) ^ swz(to)))[pair & 3] = two;
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave reads what it wrote itself
    const int c = lane & 15;
    const int64_t col = n0 + wn * (kBN / kWavesN) + 8 * c;
#pragma unroll 8
    for (int q = 0; q < kBM / 2; q += 4) {
      const int row = q + (lane >> 4);
      const int64_t at = m0 + wm * (kBM / 2) + row;
      const v4u v = sh[row * kRowChunks16 + (c ^ swz(row))];
      if (at < m_valid && col < n_valid) *reinterpret_cast<v4u*>(out + at * ldo + col) = v;
    }
  }

  __device__ __forceinline__ void finish(int, int64_t, int, int, int, void*) {}
};

// dW = dz^T . H + prev in bf16 (both operands MN-major). Without a row of H in this chunk: prev, or zeros.
static __global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(1, 1)))
void k_dw_cast(GemmShape s, EpiCast epi, MeanScale mean) {
  __shared__ v4u lds[kStages][kStageChunks];
  epi.scale = mean.get();
  if (*s.k_dev == 0) {
    const int64_t n = epi.m_valid * epi.ldo / 2;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kThreads)
      reinterpret_cast<uint32_t*>(epi.out)[i] =
          epi.prev ? pack_bf16x2(epi.prev[2 * i], epi.prev[2 * i + 1]) : 0u;
    return;
  }
  gemm_body<BF16, true, true>(s, epi, lds);
}

// The same in fp32, added or stored: the head pass's epilogue, scaled. Without a row of H a stored gradient is zero.
struct EpiSum : EpiAcc<true> {
  float scale;
  __device__ __forceinline__ void tile(f32x16_t (&acc)[kMI][kNI], float factor, int64_t m0, int64_t n0, int wm, int wn,
                                       int lane, void* smem) {
    EpiAcc<true>::tile(acc, factor * scale, m0, n0, wm, wn, lane, smem);
  }
};
template <class E>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(1, 1)))
void k_dw_sum(GemmShape s, EpiSum epi, MeanScale mean) {
  __shared__ v4u lds[kStages][kStageChunks];
  epi.scale = mean.get();
  epi.clock.start(false);
  if (epi.overwrite && *s.k_dev == 0) {
    const int64_t n = epi.m_valid * epi.ldo / 4;  // ldo = H, a multiple of 8
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kThreads)
      reinterpret_cast<v4u*>(epi.out)[i] = zero4();
    return;
  }
  gemm_body<E, true, true>(s, epi, lds);
}

// The same for few rows (n of them), where a tile is little more than its stores: half the tile, 128 x 256, and
// three 24 KB stages, so that two blocks share a CU and one's products run under the other's stores. One row /
// 256 / 512 / 768 rows of the 2048 x 151,936 head: 120 / 296 / 448 / 611 us (one row: 622 MB at 5.2 TB/s), with
// k_dw_cast 243 / 365 / 475 / 583; of 6144 x 151,936: 321 / 792 / 1341 / 1817 and 625 / 972 / 1349 / 1726. From
// there on the smaller tile's LDS reads, six fragments for eight MFMAs, bound it. Waves 2 x 2,
// each 64 x 128 as 2 x 4 MFMA 32 x 32 blocks; a stage is 32 token rows of both operands, copied straight to LDS
// two stages ahead and read through the transposing LDS reads as in the tile engine (chunk c of row k at
// c ^ 4 (k & 3)). Block b runs on XCD b % 8, which takes all column tiles of a vocabulary tile in turn.
constexpr int64_t kDwFewRows = 512;
constexpr int kDwM = 128, kDwN = 256, kDwK = 32, kDwStages = 3;
constexpr int kDwAChunks = kDwK * kDwM / 8, kDwBChunks = kDwK * kDwN / 8;
constexpr int kDwStageChunks = kDwAChunks + kDwBChunks;
// 8 token rows of 32 columns from col0 of a stage whose rows are kRowBytes long: MFMA operand of K step s.
template <int kRowBytes>
__device__ __forceinline__ v4u read_dw_frag(const v4u* l, int s, int col0, int lane) {
  const char* base = reinterpret_cast<const char*>(l);
  const int j = lane & 15;
  const int k = 8 * (2 * s + (lane >> 5)) + (j >> 2);
  const int m = col0 + 16 * ((lane >> 4) & 1) + 4 * (j & 3);
  const int off = k * kRowBytes + mn_swz(k, m >> 3) * 16 + (m & 7) * 2;
  const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)(base + off));
  const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)(base + off + 4 * kRowBytes));
  const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
  return v4u{a.x, a.y, b.x, b.y};
}
static __global__ __launch_bounds__(256, 2) void k_dw_few(const uint16_t* dz, int64_t ldz, const uint16_t* hc, int64_t H,
                                                          int64_t V, const int32_t* rows, int m_tiles, int n_tiles,
                                                          MeanScale mean, uint16_t* out) {
  __shared__ v4u lds[kDwStages][kDwStageChunks];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = static_cast<int>(uniform_u32(static_cast<uint32_t>(tid >> 6)));
  const int wm = wave >> 1, wn = wave & 1;
  const int i = static_cast<int>(blockIdx.x >> 3);
  const int mt = i / n_tiles * 8 + static_cast<int>(blockIdx.x & 7), nt = i % n_tiles;
  if (mt >= m_tiles) return;
  const int64_t m0 = static_cast<int64_t>(mt) * kDwM, n0 = static_cast<int64_t>(nt) * kDwN;
  const int n = *rows;
  const int stages = (n + kDwK - 1) / kDwK;
  // Copies of 1 KB: of A two per wave (four rows each), of B four (two rows each). dz has whole tiles of columns;
  // columns of H past its end read its last chunk and are not stored.
  constexpr int kA = 2, kB = 4, kCopies = kA + kB;
  uint32_t off[kCopies];
  int krow[kCopies];
#pragma unroll
  for (int q = 0; q < kCopies; ++q) {
    const bool is_a = q < kA;
    const int per_row = is_a ? kDwM / 8 : kDwN / 8;
    const int k = (is_a ? (wave * kA + q) * 4 : (wave * kB + q - kA) * 2) + lane / per_row;
    const int64_t c = mn_swz(k, lane % per_row);
    krow[q] = k;
    if (is_a)
      off[q] = static_cast<uint32_t>((k * ldz + 8 * c) * 2);
    else
      off[q] = static_cast<uint32_t>((k * H + (n0 + 8 * c < H ? 8 * c : H - 8 - n0)) * 2);
  }
  const uint32_t lds0 = uniform_u32(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&lds[0][0])));
  auto copy_stage = [&](int st) {
    const char* ga = static_cast<const char*>(uniform_ptr(dz + m0 + static_cast<int64_t>(st) * kDwK * ldz));
    const char* gb = static_cast<const char*>(uniform_ptr(hc + n0 + static_cast<int64_t>(st) * kDwK * H));
    const int buf = st % kDwStages;
    const bool tail = (st + 1) * kDwK > n;
#pragma unroll
    for (int q = 0; q < kCopies; ++q) {
      const int slot = q < kA ? (wave * kA + q) * 64 : kDwAChunks + (wave * kB + q - kA) * 64;
      if (!tail || st * kDwK + krow[q] < n)
        dma16(q < kA ? ga : gb, off[q], lds0, uniform_u32(static_cast<uint32_t>(buf * kDwStageChunks + slot) * 16));
      else
        (&lds[0][0])[buf * kDwStageChunks + slot + lane] = zero4();  // rows past n: zeros
    }
  };
  f32x16_t acc[2][4];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[a][b] = f32x16_t{};
  if (stages > 0) copy_stage(0);
  if (stages > 1) copy_stage(1);
  for (int st = 0; st < stages; ++st) {
    // This wave's copies of stage st have landed; those of stage st + 1, six if it is whole, may be on their way.
    if (st + 1 < stages && (st + 2) * kDwK <= n)
      wait_copies_barrier<kCopies>();
    else
      wait_copies_barrier<0>();
    if (st + 2 < stages) copy_stage(st + 2);  // into the buffer that every wave has left before the barrier
    const v4u* la = lds[st % kDwStages];
    const v4u* lb = la + kDwAChunks;
#pragma unroll
    for (int s = 0; s < kDwK / 16; ++s) {
      v4u fa[2], fb[4];
#pragma unroll
      for (int a = 0; a < 2; ++a) fa[a] = read_dw_frag<kDwM * 2>(la, s, wm * 64 + 32 * a, lane);
#pragma unroll
      for (int b = 0; b < 4; ++b) fb[b] = read_dw_frag<kDwN * 2>(lb, s, wn * 128 + 32 * b, lane);
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) Mma<BF16>::run(acc[a][b], fa[a], fb[b]);
    }
  }
  lds_barrier();  // every wave has read its last stage: LDS takes the output
  // As EpiCast, 64 rows per wave.
  const float scale = mean.get();
  v4u* sh = &lds[0][0] + wave * 64 * 16;
  const int odd = lane & 1, half = lane >> 5;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int pair = b * 16 + ((lane & 31) >> 1);
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const float x0 = acc[a][b][r] * scale, x1 = acc[a][b][r + 1] * scale;
        const float got = __uint_as_float(static_cast<uint32_t>(
            __builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(odd ? x0 : x1)), 0xB1, 0xf, 0xf, true)));
        const int to = a * 32 + (r & 3) + 8 * (r >> 2) + 4 * half + odd;
        reinterpret_cast<uint32_t*>(sh + to * 16 + ((pair >> 2) ^ EpiCast::swz(to)))[pair & 3] =
            pack_bf16x2(odd ? got : x0, odd ? x1 : got);
      }
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave reads what it wrote itself
  const int c = lane & 15;
  const int64_t col = n0 + wn * 128 + 8 * c;
#pragma unroll 8
  for (int q = 0; q < 64; q += 4) {
    const int row = q + (lane >> 4);
    const int64_t at = m0 + wm * 64 + row;
    const v4u v = sh[row * 16 + (c ^ EpiCast::swz(row))];
    if (at < V && col < H) *reinterpret_cast<v4u*>(out + at * H + col) = v;
  }
}

// dH of few rows in fp32 (up to 16 NT), one column tile of 256 and K piece per workgroup as k_bwd_dh, whose split
// products take 788 us for one row of the 2048 x 151,936 head where reading W takes 260. Each wave takes 64
// columns and all of the piece's vocabulary rows v, 16 at a time: lane (c, g), c = lane & 15, g = lane >> 4,
// loads dz[token c][v + 4g .. +3] and, for e = 0 .. 3, W[v + 4g + e][4c .. 4c + 3], so that MFMA (e, j) multiplies the
// four rows v + 4g + e into columns 4c + j: all loads are 16 bytes a lane, four rows of 256 bytes at a time.
template <int NT>
__global__ __launch_bounds__(256) void k_dh_few(const float* dz, int64_t ldz, const float* w, int64_t ld_w, int64_t V,
                                                int64_t H, const int32_t* rows, DhPlan plan, float* out) {
  const int t0 = static_cast<int>(blockIdx.y) * 16 * NT;  // this block's rows
  const int32_t count = *rows - t0;
  if (count <= 0) return;
  const int pieces = plan.pieces(*rows);
  dz += static_cast<int64_t>(t0) * ldz;
  const int piece = static_cast<int>(blockIdx.x) / plan.n_tiles;
  if (piece >= pieces) return;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int64_t h0 = static_cast<int64_t>(blockIdx.x % plan.n_tiles) * kBN + (threadIdx.x >> 6) * 64 + 4 * c;
  const int64_t len = dh_piece_rows(V, pieces);  // a multiple of 64
  const int64_t v_begin = piece * len, v_end = v_begin + len < V ? v_begin + len : V;
  const float* wc = w + (h0 < H ? h0 : H - 4);  // columns past the end: read, not stored
  const float* zr[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) zr[t] = dz + static_cast<int64_t>(16 * t + c < count ? 16 * t + c : count - 1) * ldz;
  f32x4_t acc[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[t][j] = f32x4_t{};
  constexpr int kInFlight = 4;  // groups of 16 vocabulary rows; a row of dz has whole tiles of columns, zeros past V
  for (int64_t v = v_begin; v < v_end; v += 16 * kInFlight) {
    f32x4_t x[kInFlight][4], z[kInFlight][NT];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int64_t r = v + 16 * u + 4 * g;
#pragma unroll
      for (int e = 0; e < 4; ++e)  // rows past V: the last one, times zero
        x[u][e] = *reinterpret_cast<const f32x4_t*>(wc + (r + e < V ? r + e : V - 1) * ld_w);
#pragma unroll
      for (int t = 0; t < NT; ++t) z[u][t] = *reinterpret_cast<const f32x4_t*>(zr[t] + r);
    }
    pin_order();  // all loads ahead of the products
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(z[u][t][e], x[u][e][j], acc[t][j], 0, 0, 0);
  }
  if (h0 >= H) return;
  float* o = out + (static_cast<int64_t>(piece) * plan.m_tiles(*rows) * kBM + t0) * H + h0;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int tok = 16 * t + 4 * g + r;
      if (tok < count)
        *reinterpret_cast<f32x4_t*>(o + static_cast<int64_t>(tok) * H) = f32x4_t{acc[t][0][r], acc[t][1][r], acc[t][2][r], acc[t][3][r]};
    }
}

// dW of few rows in fp32, added to or stored: each wave 64 x 64 of it by fp32 MFMAs, four token rows at a time.
// Lane (c, g), c = lane & 15, g = lane >> 4, loads dz[t + g][v0 + 4c .. +3] and H[t + g][h0 + 4c .. +3], so that MFMA
// (i, j) multiplies rows v0 + 4m + i by columns h0 + 4n + j, and the lane ends with four consecutive columns of 16
// rows: loads and stores are 16 bytes a lane.
static __global__ __launch_bounds__(256) void k_dw_few_f32(const float* dz, int64_t ldz, const float* hc, int64_t H,
                                                           int64_t V, const int32_t* rows, MeanScale mean, bool add,
                                                           float* out) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = threadIdx.x >> 6;
  const int64_t v0 = static_cast<int64_t>(blockIdx.x) * 128 + (wave >> 1) * 64;
  const int64_t h = static_cast<int64_t>(blockIdx.y) * 128 + (wave & 1) * 64 + 4 * c;
  const int n = *rows;
  const float* zc = dz + v0 + 4 * c;                 // dz has whole tiles of columns
  const float* xc = hc + (h < H ? h : H - 4);         // columns past the end: read, not stored
  f32x4_t acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4_t{};
  constexpr int kInFlight = 4;
  for (int t = 0; t < n; t += 4 * kInFlight) {
    f32x4_t z[kInFlight], x[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int r = t + 4 * u + g;
      z[u] = r < n ? *reinterpret_cast<const f32x4_t*>(zc + static_cast<int64_t>(r) * ldz) : f32x4_t{};
      x[u] = r < n ? *reinterpret_cast<const f32x4_t*>(xc + static_cast<int64_t>(r) * H) : f32x4_t{};
    }
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(z[u][i], x[u][j], acc[i][j], 0, 0, 0);
  }
  if (h >= H) return;
  const float scale = mean.get();
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t v = v0 + 4 * (4 * g + r) + i;
      if (v >= V) continue;
      f32x4_t* to = reinterpret_cast<f32x4_t*>(out + v * H + h);
      f32x4_t d{acc[i][0][r] * scale, acc[i][1][r] * scale, acc[i][2][r] * scale, acc[i][3][r] * scale};
      if (add) {
        const f32x4_t old = *to;
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] += old[j];
      }
      *to = d;
    }
}

// dhidden[t] of the chunk's rows: the sum over the K pieces (in order), rounded to the element type. Rows
// that do not count are zeroed with the first chunk. A wave takes kQuads x 256 columns, with the loads of 8 /
// kQuads pieces in flight. Few rows have up to 32 pieces and take narrow spans (one row of 2048: 30 us by four
// quads and two pieces, 9 by one and eight); many have one or two (8192 rows: 20 and 45).
template <class E, int kQuads>
__global__ __launch_bounds__(256) void k_dh_rows(const float* dh, int64_t H, const int32_t* pos, int64_t first,
                                                 int64_t T, const int32_t* rows, DhPlan plan, MeanScale mean,
                                                 typename E::storage* dhid) {
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (t >= T) return;
  const int32_t p = pos[t];
  const int64_t c = p - first;
  if (p < 0 ? first != 0 : (c < 0 || c >= *rows)) return;
  const int pieces = plan.pieces(*rows);
  const int64_t stride = static_cast<int64_t>(plan.m_tiles(*rows)) * kBM * H;
  const int64_t k0 = static_cast<int64_t>(blockIdx.y) * (64 * kQuads) + (threadIdx.x & 63);
  const int64_t last = H / 4 - 1;
  float d[kQuads][4] = {};
  if (p >= 0) {
    const float4* src = reinterpret_cast<const float4*>(dh + c * H);
#pragma unroll 8 / kQuads
    for (int q = 0; q < pieces; ++q) {
#pragma unroll
      for (int u = 0; u < kQuads; ++u) {
        const int64_t k = k0 + 64 * u;
        const float4 v = src[q * (stride / 4) + (k < last ? k : last)];  // past the row: read, not stored
        d[u][0] += v.x; d[u][1] += v.y; d[u][2] += v.z; d[u][3] += v.w;
      }
    }
  }
  const float scale = mean.get();
#pragma unroll
  for (int u = 0; u < kQuads; ++u) {
#pragma unroll
    for (int j = 0; j < 4; ++j) d[u][j] *= scale;
    if (k0 + 64 * u <= last) store4<E>(dhid + t * H + 4 * (k0 + 64 * u), d[u]);
  }
}

// ------------------------------------------------------------------------- //
// Launcher
// ------------------------------------------------------------------------- //
// Whether the fp32 gradients take the few-row kernels: up to `rows` rows, where reading W or writing dW bounds
// them, or up to 512 against weights of no more than 32 tiles, of which the tile engine gives each a CU and the
// rest nothing to do. dH of 2048 x 151,936, 32 / 64 / 65 rows: 235 / 359 and 708 us; of 2048 x 8000 (256 tiles), 163
// rows: 87, and about 50; of 64 x 1000 (4 tiles), 163 / 1024: 11 / 21 and 24 / 25. dW of 2048 x 151,936, 1 / 64 rows:
// 234 / 487 and 354 / 432; of 64 x 1000, 163 / 512 / 2048: 18 / 47 / 178 and 32 / 67 / 130.
inline bool few_f32(int64_t rows, int64_t T, int64_t H, int64_t V, const HeadLossLayout& L) {
  return L.chunks == 1 && (T <= rows || (T <= 512 && ceil_div(V, kTile) * ceil_div(H, kTile) <= 32));
}
constexpr int64_t kDhFewRows = 64, kDwFewRowsF32 = 32;

// Whether whole vocabulary tiles start K at slabs of their own: few token tiles, and no slab that K ends inside.
template <class E>
static bool rotates(const HeadLossLayout& L, int64_t H) {
  return L.rows / kTile <= kRotateMaxTokenTiles && H % (kRowChunks * E::kPerChunk) == 0;
}

template <class E, bool kStore>
static void launch_exp_logits(const HeadLossArgs& a, const HeadLossLayout& L, const typename E::storage* hc,
                              const int32_t* rows, float2* part, typename E::storage* ex, const int32_t* idx,
                              float* zy, int32_t* next, hipStream_t st) {
  using S = typename E::storage;
  const S* w = static_cast<const S*>(a.w_head);
  const float scale = kLog2e / a.tau;
  if (few_rows<E>(a.T, L)) {
    const int64_t group = few_group<E>(a.T);
    auto few = group == 16 ? k_exp_logits_few<E, 1, kStore>
                           : (group == 32 ? k_exp_logits_few<E, 2, kStore> : k_exp_logits_few<E, 4, kStore>);
    if constexpr (sizeof(S) == 2) {
      if (group == 128) few = k_exp_logits_few<E, 8, kStore>;
    }
    hipLaunchKernelGGL(few, dim3(static_cast<unsigned>(2 * L.m_tiles), static_cast<unsigned>(ceil_div(a.T, group))),
                       dim3(256), 0, st, w, a.ld_w, a.V, hc, a.H, rows, ex, L.ldv, part, L.rows, scale, idx,
                       a.K > 0 ? nullptr : a.ids, zy);
    return;
  }
  const int64_t full = a.V / kBM * kBM;
  GemmShape s = make_shape(w, a.ld_w, full, hc, a.H, L.rows, a.H);
  s.n_dev = rows;
  GemmShape tail{};
  if (a.V > full) {
    tail = make_shape(w + full * a.ld_w, a.ld_w, a.V - full, hc, a.H, L.rows, a.H);
    tail.n_dev = rows;
  }
  EpiExp<E, false, kStore> e{ex, L.ldv, part, L.rows, full, 0, scale};
  EpiExp<E, true, kStore> et{ex, L.ldv, part, L.rows, a.V - full, full / kBM, scale};
  const auto kernel = rotates<E>(L, a.H) ? k_exp_logits<E, kStore, RotatedTiles> : k_exp_logits<E, kStore, PlainTiles>;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(pull_grid())), dim3(kThreads), 0, st, s, tail, e, et, next);
}

template <class E>
static hipError_t head_loss(const HeadLossArgs& a, hipStream_t st) {
  using S = typename E::storage;
  constexpr bool k16 = sizeof(S) == 2;
  const bool distill = a.K > 0;
  const int K = distill ? a.K : 1;
  const bool cast = k16 && a.dw_cast;
  const bool grads = a.dhidden || a.dw;
  const HeadLossLayout L =
      head_loss_layout(a.T, a.H, a.V, K, sizeof(S), a.dhidden != nullptr, a.dw != nullptr, cast);
  char* w8 = static_cast<char*>(a.ws);
  auto i32 = [&](size_t off) { return reinterpret_cast<int32_t*>(w8 + off); };
  auto f32 = [&](size_t off) { return reinterpret_cast<float*>(w8 + off); };
  int32_t *blk = i32(L.blk_counts), *count = i32(L.count), *chunk_counts = i32(L.chunk_counts), *next = i32(L.next);
  int32_t *idx = i32(L.idx), *pos = i32(L.pos);
  S* hc = reinterpret_cast<S*>(w8 + L.hc);
  S* ex = reinterpret_cast<S*>(w8 + L.ex);
  float* zt = f32(L.zt);
  float2* part = reinterpret_cast<float2*>(w8 + L.part);
  double* part_loss = reinterpret_cast<double*>(w8 + L.part_loss);
  float* dw_acc = cast ? (L.chunks > 1 ? f32(L.dw_acc) : nullptr) : static_cast<float*>(a.dw);
  const S* w = static_cast<const S*>(a.w_head);

  const int nb = static_cast<int>(L.n_count_blocks);
  const int n_next = static_cast<int>(8 * L.chunks);
  const bool counted = nb > kSelfCountBlocks;
  if (counted) hipLaunchKernelGGL(k_count_rows, dim3(nb), dim3(256), 0, st, a.mask, nullptr, a.T, blk, next, n_next);
  hipLaunchKernelGGL(k_compact_rows, dim3(nb), dim3(256), 0, st, a.mask, nullptr, a.T, counted ? blk : nullptr, idx,
                     pos, count, a.token_loss, a.lse, next, n_next);
  if (L.chunks > 1)
    hipLaunchKernelGGL(k_chunk_counts, dim3(1), dim3(64), 0, st, count, L.rows, L.chunks, chunk_counts);
  else
    chunk_counts = count;
  const unsigned rows4 = static_cast<unsigned>(L.t_pad / 4);
  const bool few_logits = few_rows<E>(a.T, L);  // they bring the targets' logits themselves
  const int64_t dot_blocks = distill || few_logits ? 0 : ceil_div(a.T, 4 * kDotRows<E>);
  hipLaunchKernelGGL(k_gather_dots<E>, dim3(rows4 + static_cast<unsigned>(dot_blocks)), dim3(256), 0, st,
                     static_cast<const S*>(a.hidden), a.ld_hidden, a.H, idx, count, static_cast<int64_t>(rows4), hc, w,
                     a.ld_w, a.V, a.ids, rotates<E>(L, a.H) ? a.V / kBM : 0, zt);
  if (distill)
    hipLaunchKernelGGL(k_target_dots<E>, dim3(rows4, static_cast<unsigned>(ceil_div(K, kIds))), dim3(256), 0, st, hc, a.H,
                       w, a.ld_w, a.V, idx, a.ids, a.ld_ids, K, count, 1.0f / a.tau, zt, a.status);

  const MeanScale mean{a.n_tokens, count, a.tau};
  const DhPlan plan{L.dh_cap, a.V, static_cast<int>(ceil_div(a.H, kTile))};
  const unsigned dh_blocks = static_cast<unsigned>(8 * ceil_div(dh_most_items(plan, L.rows), 8));
  for (int64_t i = 0; i < L.chunks; ++i) {
    const int64_t first = i * L.rows;
    const int32_t* rows = chunk_counts + i;
    const S* h = hc + first * a.H;
    if (grads)
      launch_exp_logits<E, true>(a, L, h, rows, part, ex, idx + first, zt + first * K, next + 8 * i, st);
    else
      launch_exp_logits<E, false>(a, L, h, rows, part, ex, idx + first, zt + first * K, next + 8 * i, st);
    LossRows r{};
    r.part = part;
    r.ldp = L.rows;
    r.halves = static_cast<int>(2 * L.m_tiles);
    r.idx = idx + first;
    r.rows = rows;
    r.mean = {a.n_tokens, count, 1.0f};
    r.weight = a.weight;
    r.zt = zt + first * K;
    r.K = K;
    r.V = a.V;
    r.ids = a.ids;
    r.ld_ids = a.ld_ids;
    r.teacher = a.teacher;
    r.ld_teacher = a.ld_teacher;
    r.teacher_lse = a.teacher_lse;
    r.tau = a.tau;
    r.z_coef = a.z_coef;
    r.scale_z = kLog2e;
    r.max_ref = kMaxRef<E>;
    r.ex = ex;
    r.f32 = !k16;
    r.lde = L.ldv;
    r.token_loss = a.token_loss;
    r.lse = a.lse;
    r.ref = f32(L.ref);
    r.scale = f32(L.scale);
    r.patch = grads ? f32(L.patch) : nullptr;
    r.part_loss = part_loss + 2 * i * L.row_blocks;
    r.status = a.status;
    const bool few = L.loss_rows == kLossRowsFew;
    const auto loss_rows = distill ? (few ? k_loss_rows<true, kLossRowsFew> : k_loss_rows<true, kLossRowsMany>)
                                   : (few ? k_loss_rows<false, kLossRowsFew> : k_loss_rows<false, kLossRowsMany>);
    hipLaunchKernelGGL(loss_rows, dim3(static_cast<unsigned>(L.row_blocks)), dim3(256), 0, st, r);
    if (!grads) continue;
    const dim3 dz_grid(static_cast<unsigned>(L.rows / kDzRows),
                       static_cast<unsigned>(ceil_div(L.ldv, 256 * E::kPerChunk)));
    hipLaunchKernelGGL(k_exp_to_dz<E>, dz_grid, dim3(256), 0, st, ex, L.ldv, part, L.rows, r.ref, r.scale, r.patch,
                       a.ids, a.ld_ids, K, r.idx, rows);
    if (a.dhidden) {
      if (!k16 && few_f32(kDhFewRows, a.T, a.H, a.V, L)) {
        const int64_t group = few_group<E>(a.T);
        const auto dh_few = group == 16 ? k_dh_few<1> : (group == 32 ? k_dh_few<2> : k_dh_few<4>);
        hipLaunchKernelGGL(dh_few, dim3(static_cast<unsigned>(plan.n_tiles * kMaxDhPieces),
                                        static_cast<unsigned>(ceil_div(a.T, group))), dim3(256), 0, st,
                           reinterpret_cast<const float*>(ex), L.ldv, reinterpret_cast<const float*>(w), a.ld_w, a.V, a.H,
                           rows, plan, f32(L.dh));
      } else {
        GemmShape sb = make_shape(ex, L.ldv, L.rows, w, a.ld_w, a.H, a.V);
        sb.m_dev = rows;
        EpiAcc<false> eb{f32(L.dh), a.H, 0, a.H, true, {}};
        hipLaunchKernelGGL(k_bwd_dh<E>, dim3(dh_blocks), dim3(kThreads), 0, st, sb, eb, plan,
                           static_cast<int64_t*>(nullptr), int64_t{0});
      }
      const int quads = few ? 1 : 4;
      hipLaunchKernelGGL((few ? k_dh_rows<E, 1> : k_dh_rows<E, 4>),
                         dim3(static_cast<unsigned>(ceil_div(a.T, 4)), static_cast<unsigned>(ceil_div(a.H, 256 * quads))),
                         dim3(256), 0, st, f32(L.dh), a.H, pos, first, a.T, rows, plan, mean, static_cast<S*>(a.dhidden));
    }
    if (a.dw) {
      GemmShape sc = make_shape(ex, L.ldv, a.V, h, a.H, a.H, L.rows);
      sc.k_dev = rows;
      sc.msplit = 1;
      sc.sn = pick_sn_msplit(sc.n_tiles);
      if (!k16 && few_f32(kDwFewRowsF32, a.T, a.H, a.V, L)) {
        hipLaunchKernelGGL(k_dw_few_f32,
                           dim3(static_cast<unsigned>(ceil_div(a.V, 128)), static_cast<unsigned>(ceil_div(a.H, 128))),
                           dim3(256), 0, st, reinterpret_cast<const float*>(ex), L.ldv, reinterpret_cast<const float*>(h),
                           a.H, a.V, rows, mean, !a.dw_store, static_cast<float*>(a.dw));
      } else if (k16 && cast && L.chunks == 1 && L.rows <= kDwFewRows) {
        const int mt = static_cast<int>(ceil_div(a.V, kDwM)), nt = static_cast<int>(ceil_div(a.H, kDwN));
        hipLaunchKernelGGL(k_dw_few, dim3(static_cast<unsigned>(ceil_div(mt, 8) * nt * 8)), dim3(256), 0, st,
                           reinterpret_cast<const uint16_t*>(ex), L.ldv, reinterpret_cast<const uint16_t*>(h), a.H, a.V,
                           rows, mt, nt, mean, static_cast<uint16_t*>(a.dw));
      } else if (k16 && cast && i == L.chunks - 1) {
        EpiCast ec{static_cast<uint16_t*>(a.dw), dw_acc, a.H, a.V, a.H, 1.0f};
        hipLaunchKernelGGL(k_dw_cast, dim3(gemm_grid(sc)), dim3(kThreads), 0, st, sc, ec, mean);
      } else {
        EpiSum es{{dw_acc, a.H, a.V, a.H, i == 0 && (cast || a.dw_store), {}}, 1.0f};
        hipLaunchKernelGGL(k_dw_sum<E>, dim3(gemm_grid(sc)), dim3(kThreads), 0, st, sc, es, mean);
      }
    }
  }
  hipLaunchKernelGGL(k_loss_total, dim3(1), dim3(256), 0, st, part_loss, L.chunks * L.row_blocks, distill ? 1 : 2,
                     a.loss_store, a.loss);
  return hipGetLastError();
}

int launch_head_loss(const HeadLossArgs& a, hipStream_t st) {
  return a.bf16 ? head_loss<BF16>(a, st) : head_loss<F32>(a, st);
}

}  // namespace sao
