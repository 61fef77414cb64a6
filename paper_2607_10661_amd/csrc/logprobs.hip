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
//   k_logp_row    one workgroup per (entry, slice of its row), the slice in registers: its
//                 maximum first, so no sum is ever scaled anew, then one exponential per
//                 element, then the selection of the best ones (topk_select.hpp).
//   k_logp_merge  one workgroup per entry joins the slices' sums, in their order, and ranks
//                 their best entries by counting (rows of several slices).
// Per element the sums take a subtraction, a product, the exponential, a sum, a bound and a
// product-sum; terms are fp32, the sums of a wave are joined in fp64.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "topk_select.hpp"

namespace {

using namespace ptd;

constexpr int kThreads = 512;       // of k_logp_row
constexpr int kMergeThreads = 256;  // of k_logp_merge: the most (slices x best entries) of a row
constexpr int kMaxVocab = 262144;

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
};

// Sums of a slice: its maximum, how many entries equal it, sum e^d of the others and sum d e^d.
struct Sums {
  float m, ones;
  double rest, weighted;
};

// Row of logits that entry r reads, and its token; row -1: the entry stands for nothing.
__device__ __forceinline__ int entry_row(const LogpArgs& a, int r, int* token, bool tell) {
  *token = -1;
  if (!a.tokens) return r;
  const int t = a.tokens[r];
  if (t < 0 || t >= a.V) {
    if (t != -1 && tell) report(a.dev_status, PTD_ERR_VALUE);
    return -1;
  }
  *token = t;
  if (!a.nodes) return r;
  const int b = r / (a.T + 1), j = r - b * (a.T + 1);
  if (j == 0) return r;
  const int n = a.nodes[static_cast<size_t>(b) * a.T + j - 1];
  if (n < 0 || n >= a.T) {
    if (tell) report(a.dev_status, PTD_ERR_ROWS);
    *token = -1;
    return -1;
  }
  return r - j + n + 1;
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

// One entry's results from its row's sums.
struct Totals {
  double log_s, total;
  float m;
};
__device__ __forceinline__ Totals totals_of(const Sums& s) {
  Totals t;
  t.m = s.m;
  t.total = s.ones + s.rest;
  t.log_s = log1p(static_cast<double>(s.ones) - 1.0 + s.rest);
  if (s.m == INFINITY) t.log_s = NAN;  // (the infinities' own terms are no numbers)
  return t;
}
__device__ __forceinline__ float logprob_of(const LogpArgs& a, const Totals& t, float x) {
  if (t.m == -INFINITY) return -INFINITY;  // no entry has a probability
  return static_cast<float>((static_cast<double>(x) - t.m) * a.inv_tau - t.log_s);
}
__device__ __forceinline__ void put_entry(const LogpArgs& a, int r, const Totals& t, double weighted, float x) {
  if (a.logprob) a.logprob[r] = logprob_of(a, t, x);
  if (a.entropy) a.entropy[r] = t.m == -INFINITY ? 0.f : static_cast<float>(t.log_s - weighted / t.total);
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

template <int KMAX, bool BF16, int NL>
__global__ void __launch_bounds__(kThreads) k_logp_row(LogpArgs a) {
  constexpr int E = BF16 ? 8 : 4, NW = kThreads / PTD_WAVE;
  __shared__ typename std::conditional<(KMAX > 0), TopkLds<kThreads>, NoLds>::type sh;
  __shared__ uint32_t s_max[NW];
  __shared__ Sums s_sums[NW];
  __shared__ Totals s_tot;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
  int token;
  const int row = entry_row(a, r, &token, tid == 0 && slice == 0);
  if (row < 0) {  // uniform
    if (a.slices == 1) put_nothing(a, r, tid);
    return;
  }
  const char* rb = static_cast<const char*>(a.logits) + static_cast<size_t>(row) * a.ld * (BF16 ? 2 : 4);
  const int v0 = slice * a.slice_len;
  const Slice sl = slice_at<BF16>(rb, v0, min(a.V, v0 + a.slice_len), tid);
  uint4 cw[NL];
  load_chunks<BF16, kThreads, NL>(cw, rb, sl, tid);
  const uint32_t bt = sl.tail ? elem_bits<BF16>(rb, sl.vt) : 0u;
  const float xt = token >= 0 && a.slices == 1 ? __uint_as_float(elem_bits<BF16>(rb, token)) : 0.f;

  // the largest element
  uint32_t lm = sl.tail ? elem_img<BF16>(bt) : 0u;
#pragma unroll
  for (int u = 0; u < NL; ++u) lm = max(lm, u * kThreads + tid < sl.nfull ? chunk_img<BF16>(cw[u]) : 0u);
  const uint32_t wm = group_max_min<64>(lm);
  if (lane == 0) s_max[wave] = wm;
  lds_barrier();
  uint32_t top = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) top = max(top, s_max[w]);
  const float m = image_value<BF16>(top);

  // the sums.  Only a wave that holds an entry equal to m looks for it.
  float ones = 0.f, rest = 0.f, weighted = 0.f;
  if (m != -INFINITY) {
    auto add = [&](float x, bool find) __attribute__((always_inline)) {
      const float arg = (x - m) * a.scale;
      const float e = __builtin_amdgcn_exp2f(arg);
      // (an entry at -inf has no weight, and e of a NaN is one)
      weighted = fmaf(e, fmaxf(arg, -1e30f), weighted);
      if (find && x == m) ones += 1.f;
      else rest += e;
    };
    auto all = [&](bool find) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < NL; ++u) {
        if (u * kThreads + tid < sl.nfull) {
#pragma unroll
          for (int e = 0; e < E; ++e) add(__uint_as_float(chunk_bits<BF16>(cw[u], e)), find);
        }
      }
      if (sl.tail) add(__uint_as_float(bt), find);
    };
    if (wm == top) all(true);  // uniform over the wave
    else all(false);
  }
  ones = wave_sum(ones);
  rest = wave_sum(rest);
  weighted = wave_sum(weighted);
  if (lane == 0) s_sums[wave] = {m, ones, rest, weighted};
  lds_barrier();
  if (tid == 0) {
    Sums s = s_sums[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) s.ones += s_sums[w].ones, s.rest += s_sums[w].rest, s.weighted += s_sums[w].weighted;
    s.weighted *= a.unscale;
    if (a.slices > 1) {
      static_cast<Sums*>(a.part)[blockIdx.x] = s;
    } else {
      const Totals t = totals_of(s);
      s_tot = t;
      put_entry(a, r, t, s.weighted, xt);
    }
  }
  if constexpr (KMAX > 0) {
    topk_of_slice<KMAX, BF16, kThreads, NL>(sh, cw, rb, sl, bt, tid, [&](int rank, uint64_t key, uint32_t bits) {
      if (a.slices > 1) {
        uint64_t* q = keys_of<KMAX>(a, blockIdx.x) + 2 * rank;
        q[0] = key;
        q[1] = bits;
      } else if (rank < a.k) {
        const size_t at = static_cast<size_t>(r) * a.k + rank;
        if (a.topk_idx) a.topk_idx[at] = static_cast<int32_t>(key_index(key));
        if (a.topk_val) a.topk_val[at] = key ? logprob_of(a, s_tot, __uint_as_float(bits)) : NAN;
      }
    });
  }
}

// One workgroup per entry.  The pairs of all slices are at most one per thread.
template <int KMAX, bool BF16>
__global__ void __launch_bounds__(kMergeThreads) k_logp_merge(LogpArgs a) {
  __shared__ uint64_t s_key[kMergeThreads];
  __shared__ Totals s_tot;
  const int tid = threadIdx.x, r = blockIdx.x;
  int token;
  const int row = entry_row(a, r, &token, false);
  if (row < 0) {
    put_nothing(a, r, tid);
    return;
  }
  const int n = KMAX * a.slices;
  uint64_t key = 0;
  uint32_t bits = 0;
  if (KMAX > 0 && tid < n) {
    const uint64_t* q = keys_of<KMAX>(a, static_cast<long long>(r) * a.slices) + 2 * tid;
    key = q[0];
    bits = static_cast<uint32_t>(q[1]);
    s_key[tid] = key;
  }
  if (tid < PTD_WAVE) {
    Sums s = {-INFINITY, 0.f, 0.0, 0.0};
    if (tid < a.slices) s = static_cast<const Sums*>(a.part)[static_cast<size_t>(r) * a.slices + tid];
    const float xt = token >= 0 ? __uint_as_float(elem_bits<BF16>(static_cast<const char*>(a.logits) + static_cast<size_t>(row) * a.ld * (BF16 ? 2 : 4), token)) : 0.f;
    // (a NaN maximum stays one)
    bool nan = s.m != s.m;
    const float m = __any(nan) ? NAN : wave_max(s.m);
    // a slice's sums under the row's maximum: its terms are e^(m_slice - m) of what they were
    const double d = (static_cast<double>(s.m) - m) * a.inv_tau;
    const bool live = s.m != -INFINITY;
    const double f = live ? exp(d) : 0.0;
    const double own = s.ones + s.rest;
    double ones = s.m == m ? s.ones : 0.0;
    double rest = live ? (s.m == m ? s.rest : own * f) : 0.0;
    double weighted = live ? f * s.weighted + (f > 0.0 ? f * d * own : 0.0) : 0.0;
    for (int o = 32; o > 0; o >>= 1) {
      ones += __shfl_xor(ones, o, PTD_WAVE);
      rest += __shfl_xor(rest, o, PTD_WAVE);
      weighted += __shfl_xor(weighted, o, PTD_WAVE);
    }
    if (tid == 0) {
      const Totals t = totals_of({m, static_cast<float>(ones), rest, weighted});
      s_tot = t;
      put_entry(a, r, t, weighted, xt);
    }
  }
  if constexpr (KMAX > 0) {
    const int found = __syncthreads_count(tid < n && key != 0);
    if (tid >= found && tid < a.k) {  // (entries that are no numbers: fewer than k in order)
      if (a.topk_idx) a.topk_idx[static_cast<size_t>(r) * a.k + tid] = -1;
      if (a.topk_val) a.topk_val[static_cast<size_t>(r) * a.k + tid] = NAN;
    }
    if (tid < n && key) {
      int above = 0;
      for (int j = 0; j < n; ++j) above += s_key[j] > key ? 1 : 0;
      if (above < a.k) {
        const size_t at = static_cast<size_t>(r) * a.k + above;
        if (a.topk_idx) a.topk_idx[at] = static_cast<int32_t>(key_index(key));
        if (a.topk_val) a.topk_val[at] = logprob_of(a, s_tot, __uint_as_float(bits));
      }
    }
  }
}

struct LogpPlan {
  int kmax, nl, slices, slice_len;
  size_t ws_bytes;
};

bool make_plan(int R, int V, int k, int elem_bytes, LogpPlan* p) {
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
  cut(8);
  if (static_cast<long long>(R) * p->slices < 256) {
    cut(2);
    if (p->slices * std::max(p->kmax, 4) > kMergeThreads) cut(8);
  }
  if (static_cast<long long>(R) * p->slices > 0x3FFFFFFFLL) return false;
  p->ws_bytes = p->slices > 1 ? static_cast<size_t>(R) * p->slices * (sizeof(Sums) + p->kmax * 16) : 0;
  return true;
}

template <int KMAX, bool BF16>
void launch(const LogpPlan& p, const LogpArgs& a, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(a.R) * a.slices);
  if (p.nl == 8) hipLaunchKernelGGL((k_logp_row<KMAX, BF16, 8>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((k_logp_row<KMAX, BF16, 2>), grid, dim3(kThreads), 0, st, a);
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
  // the dtype is not known here: size for the larger of the bf16 and fp32 plans
  LogpPlan p2, p4;
  if (!make_plan(R, V, k, 2, &p2) || !make_plan(R, V, k, 4, &p4)) return 0;
  return std::max(p2.ws_bytes, p4.ws_bytes);
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
  PTD_RETURN_IF(!make_plan(R, V, k, es, &pl), PTD_ERR_SHAPE);
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
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == PTD_BF16) dispatch<true>(pl, a, st);
  else dispatch<false>(pl, a, st);
  return ptd_launch_status();
}
