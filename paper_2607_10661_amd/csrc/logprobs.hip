// Log probabilities of given tokens, entropy and the likeliest tokens of rows of logits
// (ptd_token_logprobs).
//
// With m the row's largest logit and d = (l - m) / temperature <= 0, a row is
//   S = sum e^d,  log P(t) = d_t - log S,  H = log S - (sum d e^d) / S.
// Where one entry dominates, S is a one and little else, and both log P and H live in what
// is left: the entries equal to m are counted, the rest is summed by itself, and log S is
// log1p of it.
//
// Kernels
//   k_logp_row    one workgroup per (entry, slice of its row), the slice in registers (256 threads
//                 x 16 chunks of 16 bytes, or 4).  One pass: a wave's terms are worked out relative to the
//                 largest entry that it has seen, four chunks at a time, while others are on
//                 their way; the sums of the waves are then brought to the slice's largest, and
//                 the best entries are selected (topk_select.hpp).
//   k_logp_path   the same for entries along accepted paths, few of which are there.
//   k_logp_merge  one workgroup per entry joins the slices' sums, in their order, and ranks
//                 their best entries (rows of several slices).
//   k_logp_wave   one wave per entry, for many rows that fit its registers (8 chunks of 16 bytes a
//                 lane, or 2).
// An element costs its unpacking, a multiply-add, the exponential, a sum, a maximum and a multiply-add, and 1.4
// more for its chunk's largest: about 45 us of the vector units for 1040 rows x 128256, beside 51 of
// HBM.  That takes 64 us in all with the 8 best entries and 52 without (a version that needed the
// row's largest entry first took 77 and 58, 512 threads x 8 chunks 70); 97 rows x 32003 fp32 11
// us, a single row 11, both the latency of two launches and of six barriers.
// Terms and the sums of a wave are fp32, waves and slices are joined in fp64.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "topk_select.hpp"

namespace {

using namespace ptd;

constexpr int kThreads = 256;       // of k_logp_row
constexpr int kMergeThreads = 256;  // of k_logp_merge: the most (slices x best entries) of a row
constexpr int kMergeSlices = 8;     // looked through at once
constexpr int kMaxVocab = 262144;
constexpr int kPartChunks = 4;      // k_logp_path: tokens of a lane at once

struct LogpArgs {
  const void* logits;
  const int32_t* tokens;   // or null: every entry is live
  const int32_t* nodes;    // or null: entry r reads row r
  float* logprob;
  float* entropy;
  int32_t* topk_idx;
  float* topk_val;
  void* part;              // Sums [entries][slices], then keys [entries][slices][KMAX][2]
  int32_t* dev_status;
  int64_t ld;
  double inv_tau;
  double unscale;          // inv_tau / scale
  float scale;             // log2(e) / temperature, rounded
  int R, V, T, k, slices, slice_len;
  int part_rows, ways;     // k_logp_path
};

// Sums of a slice: its maximum, how many entries equal it, sum e^d of the others and sum d e^d, and
// the given token's logit where the slice holds it.
struct Sums {
  float m, ones;
  double rest, weighted;
  float token_logit;
};

// Row of logits that entry r reads, and its token; row -1: the entry stands for nothing.
__device__ __forceinline__ int entry_row(const LogpArgs& a, int r, int* token, bool tell) {
  *token = -1;
  if (!a.tokens) return r;
  int t = a.tokens[r], row = r;
  if (a.nodes) {  // (loaded whether it is needed or not: the token is one more wait)
    const int b = r / (a.T + 1), j = r - b * (a.T + 1);
    const int n = j > 0 ? a.nodes[r - b - 1] : -1;
    row = r - j + n + 1;
    if (j > 0 && static_cast<uint32_t>(n) >= static_cast<uint32_t>(a.T) && static_cast<uint32_t>(t) < static_cast<uint32_t>(a.V)) {
      if (tell) report(a.dev_status, PTD_ERR_ROWS);
      t = -1;
    }
  }
  if (static_cast<uint32_t>(t) >= static_cast<uint32_t>(a.V)) {
    if (t != -1 && tell) report(a.dev_status, PTD_ERR_VALUE);
    return -1;
  }
  *token = t;
  return row;
}

// The value that an image stands for (elem_img, chunk_img).
template <bool BF16>
__device__ __forceinline__ float image_value(uint32_t img) {
  if constexpr (BF16) {
    const int o = static_cast<int>(img) - 0x8001;
    return bf16_to_f32(static_cast<uint16_t>(o ^ ((o >> 31) & 0x7FFF)));
  } else {
    return __uint_as_float((img & 0x80000000u) ? img ^ 0x80000000u : ~img);
  }
}

// The image of the largest element that is at most x: an image of bf16 leaves out the lower half of
// a float, which takes negative numbers up.
template <bool BF16>
__device__ __forceinline__ uint32_t image_at_most(float x) {
  const uint32_t bits = __float_as_uint(x);
  return elem_img<BF16>(bits) - (BF16 && (bits & 0x80000000u) && (bits & 0xFFFFu) ? 1u : 0u);
}

__device__ __forceinline__ double reciprocal(double x) {
  const double r = __builtin_amdgcn_rcp(x);
  return fma(fma(-x, r, 1.0), r, r);
}
// log(1 + t), t >= 0 (the results are fp32; the device library's takes several times the instructions,
// which a workgroup that runs once fetches from memory): the series of log((1 + z) / (1 - z)) = 2
// (z + z^3 / 3 + ...), with z = t / (2 + t) below 1/5 where t is below 1/2, else of the mantissa
// of 1 + t; what follows z^13 is below 2^-32 of z.
__device__ __forceinline__ double log1p_of(double t) {
  const bool small = t < 0.5;
  const double s = 1.0 + t;
  double f = __builtin_amdgcn_frexp_mant(s);
  int e = __builtin_amdgcn_frexp_exp(s);
  if (f < 0.70710678118654752) f *= 2.0, e -= 1;
  const double z = (small ? t : f - 1.0) * reciprocal(small ? 2.0 + t : f + 1.0);
  const double q = z * z;
  double p = 1.0 / 13.0;
  p = fma(p, q, 1.0 / 11.0);
  p = fma(p, q, 1.0 / 9.0);
  p = fma(p, q, 1.0 / 7.0);
  p = fma(p, q, 1.0 / 5.0);
  p = fma(p, q, 1.0 / 3.0);
  const double l = 2.0 * fma(p * q, z, z);
  return small ? l : fma(static_cast<double>(e), 0.69314718055994531, l);
}

// One entry's results from its row's sums.
struct Totals {
  double log_s, total;
  float m;
};
__device__ __forceinline__ Totals totals_of(const Sums& s) {
  Totals t;
  t.m = s.m;
  t.total = s.ones + s.rest;
  t.log_s = log1p_of(static_cast<double>(s.ones) - 1.0 + s.rest);
  if (s.m == INFINITY) t.log_s = NAN;  // (the infinities' own terms are no numbers)
  return t;
}
__device__ __forceinline__ float logprob_of(const LogpArgs& a, const Totals& t, float x) {
  if (t.m == -INFINITY) return -INFINITY;  // no entry has a probability
  return static_cast<float>((static_cast<double>(x) - t.m) * a.inv_tau - t.log_s);
}
__device__ __forceinline__ void put_entry(const LogpArgs& a, int r, const Totals& t, double weighted, float x) {
  if (a.logprob) a.logprob[r] = logprob_of(a, t, x);
  if (a.entropy) a.entropy[r] = t.m == -INFINITY ? 0.f : static_cast<float>(t.log_s - weighted * reciprocal(t.total));
}
__device__ __forceinline__ void put_best(const LogpArgs& a, int r, int rank, const Totals& t, uint64_t key, uint32_t bits) {
  const size_t at = static_cast<size_t>(r) * a.k + rank;
  if (a.topk_idx) a.topk_idx[at] = key ? static_cast<int32_t>(key_index(key)) : -1;
  if (a.topk_val) a.topk_val[at] = key ? logprob_of(a, t, __uint_as_float(bits)) : NAN;
}
__device__ __forceinline__ void put_nothing(const LogpArgs& a, int r, int tid) {
  if (tid == 0 && a.logprob) a.logprob[r] = 0.f;
  if (tid == 0 && a.entropy) a.entropy[r] = 0.f;
  if (tid < a.k) {
    if (a.topk_idx) a.topk_idx[static_cast<size_t>(r) * a.k + tid] = -1;
    if (a.topk_val) a.topk_val[static_cast<size_t>(r) * a.k + tid] = 0.f;
  }
}

template <int KMAX>
__device__ __forceinline__ uint64_t* keys_of(const LogpArgs& a, long long item) {
  return reinterpret_cast<uint64_t*>(static_cast<char*>(a.part) + static_cast<size_t>(a.R) * a.slices * sizeof(Sums)) +
         static_cast<size_t>(item) * KMAX * 2;
}

struct NoLds {};

// A wave's sums: of 2^(l * scale - c) and of that times the exponent, its largest entry, and
// (ones > 0) how many entries equal to the slice's largest were taken out of them.
struct WaveSums {
  double c;
  float sum, weighted, top, ones;
};

// The exponent of an entry's term relative to the row's or wave's largest entry.  The difference comes
// before the scale, so entries of any size keep their distance, and what lies so far below that it has no
// weight (-inf, a mask of any number, an overflow, the difference of two infinities) has a term of 0
// and an exponent that is a number.
__device__ __forceinline__ float exponent_below(float x, float top, float scale) { return fmaxf((x - top) * scale, -256.f); }

// What a workgroup keeps of the entry that it works on.
template <int KMAX>
struct RowLds {
  typename std::conditional<(KMAX > 0), TopkLds<kThreads>, NoLds>::type topk;
  WaveSums sums[kThreads / PTD_WAVE];
  Totals totals;
};

// The sums with care, relative to the wave's largest entry itself, whatever its size: entries that
// equal m are counted and left out.  The elements are read again, so that the common way has their
// registers.
template <bool BF16>
__device__ __forceinline__ WaveSums careful_sums(const char* rb, const Slice& sl, uint32_t bt, int tid, float top, float m, float scale) {
  constexpr int E = BF16 ? 8 : 4;
  float r = 0.f, w = 0.f;
  int n = 0;
  bool nan = false;
  auto add = [&](float x) __attribute__((always_inline)) {
    nan |= x != x;
    n += x == m ? 1 : 0;
    const float arg = exponent_below(x, top, scale);
    const float e = x == m ? 0.f : __builtin_amdgcn_exp2f(arg);
    r += e;
    w = fmaf(e, arg, w);
  };
  const uint4* src = reinterpret_cast<const uint4*>(rb + static_cast<size_t>(sl.vb) * (BF16 ? 2 : 4));
#pragma unroll 1
  for (int c0 = tid; c0 < sl.nfull; c0 += 4 * kThreads) {
    uint4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = src[min(c0 + u * kThreads, sl.nfull - 1)];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (c0 + u * kThreads < sl.nfull) {
#pragma unroll
        for (int e = 0; e < E; ++e) add(__uint_as_float(chunk_bits<BF16>(x[u], e)));
      }
    }
  }
  if (sl.tail) add(__uint_as_float(bt));
  if (__any(nan) || !(fabsf(top) < INFINITY)) r = NAN;
  return {static_cast<double>(top) * scale, wave_sum_dpp(r), wave_sum_dpp(w), top, wave_sum_dpp(static_cast<float>(n))};
}

// The wave's sums where its lane `at` alone holds entries that equal m, and these make up most of
// them: what that lane has besides would be lost in its own sum, so the lane's elements are read
// again, dealt out over the wave.
template <bool BF16, int NL>
__device__ __forceinline__ WaveSums without_top(const char* rb, const Slice& sl, uint32_t bt, int tid, int at, float m, float scale,
                                                float c, float sum, float weighted, float top) {
  constexpr int E = BF16 ? 8 : 4;
  const int lane = tid & 63, chunk = lane / 4 * kThreads + (tid - lane) + at;
  float r = lane == at ? 0.f : sum, w = lane == at ? 0.f : weighted;
  int n = 0;
  auto add = [&](float x) __attribute__((always_inline)) {
    const float arg = fmaf(x, scale, -c);
    const float e = __builtin_amdgcn_exp2f(arg);
    n += x == m ? 1 : 0;
    r += x == m ? 0.f : e;
    w += x == m ? 0.f : e * fmaxf(arg, -256.f);
  };
  if (lane / 4 < NL && chunk < sl.nfull) {
    const uint32_t x = *reinterpret_cast<const uint32_t*>(rb + (static_cast<size_t>(sl.vb) + static_cast<size_t>(chunk) * E) * (BF16 ? 2 : 4) + lane % 4 * 4);
    if constexpr (BF16) add(bf16_lo(x)), add(bf16_hi(x));
    else add(__uint_as_float(x));
  }
  if (lane == at && sl.tail) add(__uint_as_float(bt));
  return {c, wave_sum_dpp(r), wave_sum_dpp(w), top, wave_sum_dpp(static_cast<float>(n))};
}

// One slice of the row that entry r reads.  A wave's terms are relative to the largest entry of its
// first chunks, so they are worked out while others are on their way; where later ones hold one that is
// 2^8 times as likely, the sums go on from there.
template <int KMAX, bool BF16, int NL, bool ONE>
__device__ __forceinline__ void row_slice(const LogpArgs& a, RowLds<KMAX>& sh, int r, int row, int token, int slice, int tid) {
  constexpr int NW = kThreads / PTD_WAVE;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const char* rb = static_cast<const char*>(a.logits) + static_cast<size_t>(row) * a.ld * (BF16 ? 2 : 4);
  const int v0 = slice * a.slice_len;
  const Slice sl = slice_at<BF16>(rb, v0, min(a.V, v0 + a.slice_len), tid);
  uint4 cw[NL];
  load_chunks<BF16, kThreads, NL>(cw, rb, sl, tid);
  const uint32_t bt = sl.tail ? elem_bits<BF16>(rb, sl.vt) : 0u;
  // (by every thread, or none: a wait less where it is needed)
  const float xt = token >= sl.v0 && token < sl.v1 ? __uint_as_float(elem_bits<BF16>(rb, token)) : 0.f;
  // the sums, four chunks at a time
  uint32_t lm = sl.tail ? elem_img<BF16>(bt) : 0u, limit = 0;
  float c = 0.f, sum = 0.f, weighted = 0.f;
  // (a masked entry's term is 0, times its exponent no number: the exponent of a term that is 0 may be any
  // other.  1040 x 128256, 99 % of it masked, 65 us, and 115 where such waves were summed again with
  // care; nothing masked 64)
  auto add = [&](float x) __attribute__((always_inline)) {
    const float arg = fmaf(x, a.scale, -c);
    const float e = __builtin_amdgcn_exp2f(arg);
    sum += e;
    weighted = fmaf(e, fmaxf(arg, -256.f), weighted);
  };
  static_assert(NL % 4 == 0, "groups of four chunks");
#pragma unroll
  for (int u0 = 0; u0 < NL; u0 += 4) {
    uint32_t img = u0 == 0 ? lm : 0u;
#pragma unroll
    for (int u = u0; u < u0 + 4; ++u) img = max(img, u * kThreads + tid < sl.nfull ? chunk_img<BF16>(cw[u]) : 0u);
    lm = max(lm, img);
    if (__any(img > limit)) {
      const uint32_t most = group_max_min<64>(img);
      const float ref = image_value<BF16>(most);
      const float next = ref > -INFINITY ? ref * a.scale : 0.f;  // (masked entries alone: any number)
      const float f = __builtin_amdgcn_exp2f(fminf(c - next, 0.f));  // (above 0 only from masked entries, whose sums are 0)
      weighted = u0 == 0 ? 0.f : f * fmaf(c - next, sum, weighted);
      sum = u0 == 0 ? 0.f : f * sum;
      c = next;
      limit = max(most, image_at_most<BF16>(ref + 8.f / a.scale));
    }
#pragma unroll
    for (int u = u0; u < u0 + 4; ++u) {
      if (u * kThreads + tid < sl.nfull) {
#pragma unroll
        for (int e = 0; e < (BF16 ? 8 : 4); ++e) add(__uint_as_float(chunk_bits<BF16>(cw[u], e)));
      }
    }
  }
  // (the compiler would keep the chunks' images for the lists: registers that it then spills the
  // chunks from, 1040 rows x 128256 80 us and 64)
  if constexpr (KMAX > 0) {
#pragma unroll
    for (int u = 0; u < NL; ++u) asm volatile("" : "+v"(cw[u].x), "+v"(cw[u].y), "+v"(cw[u].z), "+v"(cw[u].w));
  }
  if (sl.tail) add(__uint_as_float(bt));
  const uint32_t img = group_max_min<64>(lm);
  const float top = img ? image_value<BF16>(img) : -INFINITY;  // (a wave without an element)
  const float all = wave_sum_dpp(sum), all_weighted = wave_sum_dpp(weighted);
  const bool care = !(all_weighted - all_weighted == 0.f) || !(fabsf(c) < 0x1p20f);
  if (lane == 0) sh.sums[wave] = {c, all, all_weighted, top, 0.f};
  if constexpr (KMAX > 0) topk_groups<KMAX, kThreads>(sh.topk, lm, tid);
  lds_barrier();
  uint32_t tc = 0;
  if constexpr (KMAX > 0) tc = topk_list<KMAX, BF16, kThreads, NL>(sh.topk, cw, sl, bt, tid, [&](int u) { return chunk_img<BF16>(cw[u]); });
  float m = sh.sums[0].top;
  bool nan = m != m;
#pragma unroll
  for (int w = 1; w < NW; ++w) {
    const float x = sh.sums[w].top;
    nan |= x != x;
    m = fmaxf(m, x);
  }
  if (nan) m = NAN;
  lds_barrier();  // sh.sums is read
  if (top == -INFINITY) {
    if (lane == 0) sh.sums[wave] = {0.0, 0.f, 0.f, top, 0.f};
  } else if (care) {
    const WaveSums s = careful_sums<BF16>(rb, sl, bt, tid, top, m, a.scale);
    if (lane == 0) sh.sums[wave] = s;
  } else if (top == m && !(all >= 2.f * __builtin_amdgcn_exp2f(fmaf(top, a.scale, -c)))) {
    // (e of the largest entry is 2^(top * scale - c); two lanes with one of it each are half of the sum)
    const uint64_t who = __ballot(lm == img);
    const WaveSums s = without_top<BF16, NL>(rb, sl, bt, tid, __builtin_ctzll(who), m, a.scale, c, sum, weighted, top);
    if (lane == 0) sh.sums[wave] = s;
  }
  if constexpr (KMAX > 0) topk_examine<BF16, kThreads>(sh.topk, sl, tc, tid);
  lds_barrier();
  if (wave == 0) {
    // to the slice's largest entry: one lane per wave's sums
    const WaveSums s = sh.sums[min(lane, NW - 1)];
    const bool has = lane < NW && s.top != -INFINITY;
    const double d = s.c - static_cast<double>(m) * a.scale;  // (the product is exact)
    const double f = has ? static_cast<double>(__builtin_amdgcn_exp2f(static_cast<float>(d))) : 0.0;
    double rest = has ? f * s.sum : 0.0, wt = has ? f * (s.weighted + d * s.sum) : 0.0;
    float ones = has ? s.ones : 0.f;
    // the largest entry, where it was not taken out: one of it, as the sums hold it
    const uint64_t in = __ballot(has && s.top == m && s.ones == 0.f);
#pragma unroll
    for (int o = 1; o < NW; o <<= 1) {
      rest += __shfl_xor(rest, o, PTD_WAVE);
      wt += __shfl_xor(wt, o, PTD_WAVE);
      ones += __shfl_xor(ones, o, PTD_WAVE);
    }
    if (in && ones == 0.f) ones = 1.f, rest -= 1.0;
    if (lane == 0) {
      const Sums t = {m, ones, rest, wt * a.unscale, xt};
      if constexpr (ONE) {
        sh.totals = totals_of(t);
        put_entry(a, r, sh.totals, t.weighted, xt);
      } else {
        static_cast<Sums*>(a.part)[static_cast<size_t>(r) * a.slices + slice] = t;
      }
    }
  }
  if constexpr (KMAX > 0) {
    topk_pick<KMAX, BF16, kThreads>(
        sh.topk, rb, sl, tid, [&] { topk_in_turns<KMAX, BF16, kThreads>(sh.topk, rb, sl, tid); },
        [&](int rank, uint64_t key, uint32_t bits) {
          if constexpr (ONE) {
            if (rank < a.k) put_best(a, r, rank, sh.totals, key, bits);
          } else {
            uint64_t* q = keys_of<KMAX>(a, static_cast<long long>(r) * a.slices + slice) + 2 * rank;
            q[0] = key;
            q[1] = bits;
          }
        });
  }
}

template <int KMAX, bool BF16, int NL, bool ONE>
__global__ void __launch_bounds__(kThreads, 4) k_logp_row(LogpArgs a) {
  __shared__ RowLds<KMAX> sh;
  const int tid = threadIdx.x;
  const int r = ONE ? blockIdx.x : blockIdx.x / a.slices, slice = ONE ? 0 : blockIdx.x - r * a.slices;
  int token;
  const int row = entry_row(a, r, &token, tid == 0 && slice == 0);
  if (row < 0) {  // uniform
    if (ONE) put_nothing(a, r, tid);
    return;
  }
  row_slice<KMAX, BF16, NL, ONE>(a, sh, r, row, token, slice, tid);
}

// One wave per entry, the whole row in its registers: the largest entry first, then the others' terms
// relative to it, then the best entries one after the other -- the next best of the lane that had the
// one before is found by the whole wave, an element each.
template <bool TOPK, bool BF16, int NL>
__global__ void __launch_bounds__(kThreads) k_logp_wave(LogpArgs a) {
  constexpr int E = BF16 ? 8 : 4;
  const int lane = threadIdx.x & 63;
  const int r = blockIdx.x * (kThreads / PTD_WAVE) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (r >= a.R) return;  // whole wave
  int token;
  const int row = entry_row(a, r, &token, lane == 0);
  if (row < 0) {  // uniform
    put_nothing(a, r, lane);
    return;
  }
  const char* rb = static_cast<const char*>(a.logits) + static_cast<size_t>(row) * a.ld * (BF16 ? 2 : 4);
  const Slice sl = slice_at<BF16>(rb, 0, a.V, lane);
  uint4 cw[NL];
  load_chunks<BF16, PTD_WAVE, NL>(cw, rb, sl, lane);
  const uint32_t bt = sl.tail ? elem_bits<BF16>(rb, sl.vt) : 0u;
  const float xt = token >= 0 ? __uint_as_float(elem_bits<BF16>(rb, token)) : 0.f;
  // every element of the lane, in order of its index but for the edge's
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    if (sl.tail) f(bt, sl.vt);
#pragma unroll
    for (int u = 0; u < NL; ++u) {
      const int c = u * PTD_WAVE + lane;
      if (c < sl.nfull) {
#pragma unroll
        for (int e = 0; e < E; ++e) f(chunk_bits<BF16>(cw[u], e), sl.vb + c * E + e);
      }
    }
  };
  uint32_t best = 0, at = 0;
  bool nan = false;
  each([&](uint32_t bits, int v) __attribute__((always_inline)) {
    const float x = __uint_as_float(bits);
    nan |= x != x;
    const uint32_t o = ord_of(x);
    const bool more = o > best || (o == best && static_cast<uint32_t>(v) < at);
    best = more ? o : best;
    at = more ? static_cast<uint32_t>(v) : at;
  });
  const uint32_t img = group_max_min<64>(best);
  const float m = img ? image_value<false>(img) : NAN;
  float rest = 0.f, w = 0.f;
  int n = 0;
  each([&](uint32_t bits, int) __attribute__((always_inline)) {
    const float x = __uint_as_float(bits);
    n += x == m ? 1 : 0;
    const float arg = exponent_below(x, m, a.scale);
    const float e = x == m ? 0.f : __builtin_amdgcn_exp2f(arg);
    rest += e;
    w = fmaf(e, arg, w);
  });
  if (__any(nan) || m == INFINITY) rest = NAN;
  rest = wave_sum_dpp(rest), w = wave_sum_dpp(w);
  const float ones = wave_sum_dpp(static_cast<float>(n));
  const Sums s = {m, ones, rest, w * a.unscale, xt};
  const Totals tot = totals_of(s);
  if (lane == 0) put_entry(a, r, tot, s.weighted, xt);
  if constexpr (TOPK) {
    for (int k = 0; k < a.k; ++k) {  // uniform
      const uint32_t top = group_max_min<64>(best);
      const uint32_t first = group_max_min<1>(best == top ? at : ~0u);
      if (lane == 0) put_best(a, r, k, tot, top ? (static_cast<uint64_t>(top) << 32) | static_cast<uint32_t>(~first) : 0, __float_as_uint(image_value<false>(top)));
      if (k + 1 == a.k) break;
      const uint64_t who = __ballot(best == top && at == first);
      if (!who) break;  // (never: the pair is some lane's)
      const int owner = __builtin_ctzll(who);
      // elements of the owner that come behind (top, first)
      uint32_t o = 0, v = ~0u;
      const int ch = lane / E * PTD_WAVE + owner;
      if (lane / E < NL && ch < sl.nfull) {
        v = static_cast<uint32_t>(sl.vb + ch * E + lane % E);
        o = ord_of(__uint_as_float(elem_bits<BF16>(rb, v)));
        if (!(o < top || (o == top && v > first))) o = 0;
      }
      if (lane == owner && sl.tail) {  // its edge, besides
        const uint32_t eo = ord_of(__uint_as_float(bt)), ev = static_cast<uint32_t>(sl.vt);
        if ((eo < top || (eo == top && ev > first)) && (eo > o || (eo == o && ev < v))) o = eo, v = ev;
      }
      const uint32_t next = group_max_min<64>(o);
      const uint32_t place = group_max_min<1>(o == next ? v : ~0u);
      if (lane == owner) best = next, at = place;
    }
  }
}

// Entries along paths: few of a sequence's T + 1 are there, and the host does not know which.
// Workgroup (a few sequences, i, slice) takes the i-th of those that are, then every `ways`-th.
template <int KMAX, bool BF16, int NL, bool ONE>
__global__ void __launch_bounds__(kThreads, 4) k_logp_path(LogpArgs a) {
  __shared__ RowLds<KMAX> sh;
  const int tid = threadIdx.x, lane = tid & 63;
  const int slice = ONE ? 0 : blockIdx.x % a.slices, g = ONE ? blockIdx.x : blockIdx.x / a.slices;
  const int part = g / a.ways, way = g % a.ways;
  const int r0 = part * a.part_rows, n = min(a.part_rows, a.R - r0);
  const bool tell = way == 0 && slice == 0 && tid < PTD_WAVE;
  int seen = 0;
  for (int j0 = 0; j0 < n; j0 += kPartChunks * PTD_WAVE) {  // uniform: every wave reads the same tokens
    uint64_t there[kPartChunks];
#pragma unroll
    for (int u = 0; u < kPartChunks; ++u) {
      const int j = j0 + u * PTD_WAVE + lane;
      int token;
      const int row = j < n ? entry_row(a, r0 + j, &token, tell) : -1;
      there[u] = __ballot(row >= 0);
      // (of several slices: k_logp_merge)
      if (ONE && tell && j < n && row < 0) {
        for (int k = 0; k < max(a.k, 1); ++k) put_nothing(a, r0 + j, k);
      }
    }
#pragma unroll 1
    for (int u = 0; u < kPartChunks; ++u) {
      static_assert(kPartChunks == 4, "four of them");
      uint64_t live = u == 0 ? there[0] : u == 1 ? there[1] : u == 2 ? there[2] : there[3];
      for (; live; live &= live - 1) {
        const bool mine = seen == way;
        seen = seen + 1 == a.ways ? 0 : seen + 1;
        if (!mine) continue;
        const int r = r0 + j0 + u * PTD_WAVE + __builtin_ctzll(live);
        int token;
        const int row = entry_row(a, r, &token, false);
        row_slice<KMAX, BF16, NL, ONE>(a, sh, r, row, token, slice, tid);
        lds_barrier();
      }
    }
  }
}

// One workgroup per entry.  The pairs of all slices are at most one per thread.
template <int KMAX, bool BF16>
__global__ void __launch_bounds__(kMergeThreads) k_logp_merge(LogpArgs a) {
  __shared__ uint64_t s_key[kMergeThreads];
  __shared__ Totals s_tot;
  const int tid = threadIdx.x, r = blockIdx.x;
  // (loaded whether the entry is there or not: the token is one more wait)
  const int n = KMAX * a.slices;
  uint64_t key = 0;
  uint32_t bits = 0;
  if (KMAX > 0 && tid < n) {
    const uint64_t* q = keys_of<KMAX>(a, static_cast<long long>(r) * a.slices) + 2 * tid;
    key = q[0];
    bits = static_cast<uint32_t>(q[1]);
  }
  Sums s = {-INFINITY, 0.f, 0.0, 0.0, 0.f};
  if (tid < a.slices) s = static_cast<const Sums*>(a.part)[static_cast<size_t>(r) * a.slices + tid];
  int token;
  const int row = entry_row(a, r, &token, false);
  if (row < 0) {
    put_nothing(a, r, tid);
    return;
  }
  if (KMAX > 0) {
    s_key[tid] = key;  // (0: none)
  }
  if (tid < PTD_WAVE) {
    const float xt = __shfl(s.token_logit, token >= 0 ? token / a.slice_len : 0, PTD_WAVE);
    // (a NaN maximum stays one)
    bool nan = s.m != s.m;
    const float m = __any(nan) ? NAN : wave_max(s.m);
    // a slice's sums under the row's maximum: its terms are e^(m_slice - m) of what they were
    const double d = (static_cast<double>(s.m) - m) * a.inv_tau;
    const bool live = s.m != -INFINITY;
    const double f = live ? static_cast<double>(__builtin_amdgcn_exp2f(static_cast<float>(d * 1.4426950408889634))) : 0.0;
    const double own = s.ones + s.rest;
    double ones = s.m == m ? s.ones : 0.0;
    double rest = live ? (s.m == m ? s.rest : own * f) : 0.0;
    double weighted = live ? f * s.weighted + (f > 0.0 ? f * d * own : 0.0) : 0.0;
    for (int o = 1; o < a.slices; o <<= 1) {  // (lanes past the slices hold nothing)
      ones += __shfl_xor(ones, o, PTD_WAVE);
      rest += __shfl_xor(rest, o, PTD_WAVE);
      weighted += __shfl_xor(weighted, o, PTD_WAVE);
    }
    if (tid == 0) {
      const Totals t = totals_of({m, static_cast<float>(ones), rest, weighted, xt});
      s_tot = t;
      put_entry(a, r, t, weighted, xt);
    }
  }
  if constexpr (KMAX > 0) {
    __syncthreads();
    // a slice's pairs are in order: the rank of one is its place plus, in every other slice, the number of
    // larger ones, found by halving (several slices at once: each step waits for LDS)
    int above = tid % KMAX;
    const int own = tid / KMAX;
    for (int j0 = 0; j0 < a.slices; j0 += kMergeSlices) {
      int lo[kMergeSlices];
#pragma unroll
      for (int u = 0; u < kMergeSlices; ++u) lo[u] = 0;
#pragma unroll
      for (int step = KMAX / 2; step > 0; step >>= 1) {
#pragma unroll
        for (int u = 0; u < kMergeSlices; ++u) lo[u] += s_key[min(j0 + u, a.slices - 1) * KMAX + lo[u] + step - 1] > key ? step : 0;
      }
#pragma unroll
      for (int u = 0; u < kMergeSlices; ++u) {
        const int j = min(j0 + u, a.slices - 1);
        lo[u] += s_key[j * KMAX + lo[u]] > key ? 1 : 0;
        above += j0 + u == own || j0 + u >= a.slices ? 0 : lo[u];
      }
    }
    if (key && above < a.k) put_best(a, r, above, s_tot, key, bits);
  }
}

struct LogpPlan {
  int kmax, nl, slices, slice_len;
  size_t ws_bytes;
};

// Slices of 16 chunks a thread, or of 4 where workgroups would be fewer than two per CU: k = 5, bf16, 128256
// entries, 4 / 16 chunks: a row 9.7 / 11.4 us, 64 rows 14.2 / 16.2, 128 rows 17.9 / 18.0, 256 rows 25.1 / 23.6, 1040
// rows 74 / 63.  (The pairs of a row's slices have to fit the merge.)
// path_seqs: entries lie along paths, and about four per sequence are there, whatever R.
bool make_plan(int R, int V, int k, int elem_bytes, int path_seqs, LogpPlan* p) {
  if (R < 1 || V < 1 || V > kMaxVocab || k < 0 || k > PTD_MAX_K || k > V) return false;
  const int E = 16 / elem_bytes;
  p->kmax = k == 0 ? 0 : k <= 8 ? 8 : 16;
  auto cut = [&](int nl) {
    const int most = kThreads * nl * E;
    int s = (V + most - 1) / most;
    int len = ((V + s - 1) / s + 7) & ~7;  // slices of an aligned row start 16-byte aligned
    p->nl = nl;
    p->slices = (V + len - 1) / len;
    p->slice_len = len;
  };
  cut(16);
  const long long rows = path_seqs ? 4LL * path_seqs : R;
  if (rows * p->slices < 512) {
    cut(4);
    if (p->slices * std::max(p->kmax, 4) > kMergeThreads) cut(16);
  }
  if (static_cast<long long>(R) * p->slices >= (1 << 24)) return false;  // (a grid holds fewer than 2^32 threads)
  p->ws_bytes = p->slices > 1 ? static_cast<size_t>(R) * p->slices * (sizeof(Sums) + p->kmax * 16) : 0;
  return true;
}

// Whether rows go to k_logp_wave: those that fit, where there are many.  (bf16, a workgroup / a wave per
// row: 1000 entries, k = 5, 64 rows 5.1 / 6.4 us, 1040 rows 11.0 / 6.8, 16384 rows 91 / 27; k = 16,
// 1040 rows 13.3 / 13.0; 4000 entries, k = 5, 1040 rows 11.6 / 12.1, 16384 rows 101 / 55; k = 0, 1040
// rows 7.1 / 9.3, 16384 rows 56 / 44; 100000 rows of 50 entries 552 / 118.)
constexpr int kFewChunks = 2, kWaveChunks = 8;
inline bool by_waves(const LogpArgs& a, int elems) {
  if (a.V > PTD_WAVE * kWaveChunks * elems) return false;
  const int rows = a.V <= PTD_WAVE * kFewChunks * elems ? 512 : a.k == 0 ? 8192 : 2048;
  return a.R >= (a.k > 8 ? 2 * rows : rows);
}

template <bool TOPK, bool BF16>
void launch_waves(const LogpArgs& a, hipStream_t st) {
  const dim3 grid(ptd_cdiv(a.R, kThreads / PTD_WAVE));
  if (a.V <= PTD_WAVE * kFewChunks * (BF16 ? 8 : 4)) hipLaunchKernelGGL((k_logp_wave<TOPK, BF16, kFewChunks>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((k_logp_wave<TOPK, BF16, kWaveChunks>), grid, dim3(kThreads), 0, st, a);
}

template <int KMAX, bool BF16>
void launch(const LogpPlan& p, const LogpArgs& a, hipStream_t st) {
  if (by_waves(a, BF16 ? 8 : 4)) return launch_waves<(KMAX > 0), BF16>(a, st);
  const bool one = p.slices == 1;
  const unsigned n = (a.nodes ? static_cast<unsigned>(ptd_cdiv(a.R, a.part_rows)) * a.ways : static_cast<unsigned>(a.R)) * a.slices;
#define PTD_LOGP(kernel_, nl_)                                                                                \
  if (p.nl == nl_ && one) hipLaunchKernelGGL((kernel_<KMAX, BF16, nl_, true>), dim3(n), dim3(kThreads), 0, st, a); \
  if (p.nl == nl_ && !one) hipLaunchKernelGGL((kernel_<KMAX, BF16, nl_, false>), dim3(n), dim3(kThreads), 0, st, a);
  if (a.nodes) {
    PTD_LOGP(k_logp_path, 16) PTD_LOGP(k_logp_path, 4)
  } else {
    PTD_LOGP(k_logp_row, 16) PTD_LOGP(k_logp_row, 4)
  }
#undef PTD_LOGP
  if (p.slices > 1) hipLaunchKernelGGL((k_logp_merge<KMAX, BF16>), dim3(a.R), dim3(kMergeThreads), 0, st, a);
}
template <bool BF16>
void dispatch(const LogpPlan& p, const LogpArgs& a, hipStream_t st) {
  if (p.kmax == 0) launch<0, BF16>(p, a, st);
  else if (p.kmax == 8) launch<8, BF16>(p, a, st);
  else launch<16, BF16>(p, a, st);
}

}  // namespace

extern "C" size_t ptd_token_logprobs_workspace_bytes(int32_t R, int32_t V, int32_t k) {
  // the dtype is not known here: size for the larger of the bf16 and fp32 plans;
  // nor whether entries lie along paths, where slices may be those of fewer rows (the fewest: of the
  // largest trees)
  size_t most = 0;
  for (int es = 2; es <= 4; es += 2) {
    for (int seqs : {0, std::max(1, R / (PTD_MAX_T + 1))}) {
      LogpPlan p;
      if (!make_plan(R, V, k, es, seqs, &p)) return 0;
      most = std::max(most, p.ws_bytes);
    }
  }
  return most;
}

extern "C" int ptd_token_logprobs(const void* logits, ptd_dtype dtype, int32_t R, int32_t V, int64_t ld,
                                  const int32_t* tokens, const int32_t* nodes, int32_t T,
                                  double temperature, int32_t k, float* logprob, float* entropy,
                                  int32_t* topk_idx, float* topk_logprob, void* workspace,
                                  size_t workspace_bytes, int32_t* dev_status, void* stream) {
  PTD_RETURN_IF(!logits || (!logprob && !entropy && !topk_idx && !topk_logprob), PTD_ERR_NULL);
  PTD_RETURN_IF((logprob || nodes) && !tokens, PTD_ERR_NULL);
  PTD_RETURN_IF(dtype != PTD_F32 && dtype != PTD_BF16, PTD_ERR_DTYPE);
  PTD_RETURN_IF(ld < V || !(temperature >= 1e-30 && temperature <= 1e30), PTD_ERR_SHAPE);
  PTD_RETURN_IF(nodes && (T < 1 || T > PTD_MAX_T || R % (T + 1) != 0), PTD_ERR_SHAPE);
  PTD_RETURN_IF(k == 0 ? topk_idx || topk_logprob : !topk_idx && !topk_logprob, PTD_ERR_SHAPE);
  const int es = dtype == PTD_BF16 ? 2 : 4;
  LogpPlan pl;
  PTD_RETURN_IF(!make_plan(R, V, k, es, nodes ? R / (T + 1) : 0, &pl), PTD_ERR_SHAPE);
  PTD_RETURN_IF(!ptd_aligned(logits, es), PTD_ERR_ALIGN);
  if (pl.ws_bytes) {
    PTD_RETURN_IF(!workspace || workspace_bytes < pl.ws_bytes, PTD_ERR_WORKSPACE);
    PTD_RETURN_IF(!ptd_aligned(workspace, 8), PTD_ERR_ALIGN);
  }
  LogpArgs a = {};
  a.logits = logits;
  a.tokens = tokens;
  a.nodes = nodes;
  a.logprob = logprob;
  a.entropy = entropy;
  a.topk_idx = topk_idx;
  a.topk_val = topk_logprob;
  a.part = workspace;
  a.dev_status = dev_status;
  a.ld = ld;
  a.inv_tau = 1.0 / temperature;
  a.scale = static_cast<float>(1.4426950408889634 / temperature);
  a.unscale = a.inv_tau / a.scale;
  a.R = R, a.V = V, a.T = nodes ? T : 0, a.k = k;
  a.slices = pl.slices, a.slice_len = pl.slice_len;
  if (nodes) {
    // as many sequences as a wave reads tokens of at once, and a way for each entry of paths
    // of three nodes (and four more)
    const int seqs = std::max(1, std::min(kPartChunks * PTD_WAVE / (T + 1), R / (T + 1)));
    a.part_rows = seqs * (T + 1);
    a.ways = std::min(4 * seqs + 4, 32);
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == PTD_BF16) dispatch<true>(pl, a, st);
  else dispatch<false>(pl, a, st);
  return ptd_launch_status();
}
