// Per-row argmax and top-k of the verification logits (Sec. 3.2: greedy
// verification tokens are the highest-probability predictions; App. A: top-k
// candidates for the draft-tree expansion).
//
// Kernels
//   k_topk_row      one workgroup per (row, vocabulary slice), a slice being
//                   at most 4096 chunks of 16 bytes (32768 bf16 or 16384
//                   fp32 values; 6144 chunks for a few long rows) held in
//                   registers (1024 threads x 4 or 6 chunks, or 512 x 8 when
//                   there are many slices): a cheap lower
//                   bound of the KMAX-th best value leaves a few candidates,
//                   ranked by counting (details below).  Rows may start at
//                   any element address: the few elements before the slice's
//                   first 16-byte boundary and after its last whole chunk are
//                   read one per lane.
//   k_topk_wave     short rows that are not 16-byte aligned: one wave per row
//                   with element loads; each lane keeps a sorted list of its
//                   KMAX best keys in registers.
// Sorted lists are merged by a butterfly of 6 steps per wave, each merging two
// sorted lists with a bitonic network.
//   k_topk_merge    one workgroup per row ranks the slice results by counting
//                   (only when a row spans several slices).
// A slice result is KMAX (key, value bits) pairs in the workspace.  topk_val
// carries the row's own values (including the sign of a zero): candidates
// keep their bits; the rare paths that hold only keys re-read the logits.
#include <algorithm>

#include "topk_select.hpp"

namespace {

using namespace ptd;

constexpr int kThreads = 256;

template <bool BF16>
__device__ __forceinline__ float elem_value(const void* base, size_t i) {
  return __uint_as_float(elem_bits<BF16>(base, i));
}

// Final results of one row from its KMAX best keys (key r held by lane r).
// (k <= V makes every emitted key a real element; the bound check only keeps
// the value re-read inside the row whatever the key.)
template <bool BF16>
__device__ __forceinline__ void emit(uint64_t key, int lane, int k, int V, const void* row_base,
                                     int row, int32_t* argmax, int32_t* topk_idx,
                                     float* topk_val) {
  const uint32_t idx = key_index(key);
  const bool real = idx < static_cast<uint32_t>(V);
  if (lane == 0) argmax[row] = real ? static_cast<int32_t>(idx) : -1;
  if (lane < k) {
    if (topk_idx) topk_idx[static_cast<size_t>(row) * k + lane] = real ? static_cast<int32_t>(idx) : -1;
    if (topk_val) topk_val[static_cast<size_t>(row) * k + lane] = real ? elem_value<BF16>(row_base, idx) : 0.f;
  }
}

// One workgroup of NT threads per (row, slice), a slice being at most one
// batch of NL chunks of 16 bytes per lane (NT * NL * 16 bytes), loaded
// straight into registers.
template <int KMAX, bool BF16, int NT, int NL>
__global__ void __launch_bounds__(NT)
k_topk_row(const void* __restrict__ logits, int V, long long ld, int slices, int slice_len,
           int k, int32_t* __restrict__ argmax, int32_t* __restrict__ topk_idx,
           float* __restrict__ topk_val, uint64_t* __restrict__ part) {
  __shared__ TopkLds<NT> sh;
  const int tid = threadIdx.x;
  const int row = blockIdx.x / slices, s = blockIdx.x % slices;
  const int v0 = s * slice_len;
  const char* rb = static_cast<const char*>(logits) + static_cast<size_t>(row) * ld * (BF16 ? 2 : 4);
  const Slice sl = slice_at<BF16>(rb, v0, min(V, v0 + slice_len), tid);
  uint4 cw[NL];
  load_chunks<BF16, NT, NL>(cw, rb, sl, tid);
  const uint32_t bt = sl.tail ? elem_bits<BF16>(rb, sl.vt) : 0u;
  uint32_t lm = sl.tail ? elem_img<BF16>(bt) : 0u;
  uint32_t cm[NL];
#pragma unroll
  for (int u = 0; u < NL; ++u) {
    cm[u] = chunk_img<BF16>(cw[u]);
    // (the compiler would keep what an image is made of for the list: 72 registers, where up to 64 let a
    // CU hold another workgroup)
    asm volatile("" : "+v"(cm[u]));
    lm = max(lm, u * NT + tid < sl.nfull ? cm[u] : 0u);
  }
  topk_groups<KMAX, NT>(sh, lm, tid);
  lds_barrier();
  const uint32_t tc = topk_list<KMAX, BF16, NT, NL>(sh, cw, sl, bt, tid, [&](int u) { return cm[u]; });
  lds_barrier();
  // a list that overflows (values tied at the top, or in order): every lane keeps a sorted list of
  // the best of its own elements that reach the bound, and the lists are merged (KMAX 16: its registers
  // would halve the workgroups of a CU, so the best are taken one after the other.  1040 rows x 128256 bf16,
  // k = 16, in turns / with lists: ordinary rows 50 / 146 us, 5 % tied at the top 146 / 648, in order
  // 145 / 288, all but a few at one finite value 145 / 352; 65 x 32000 in order 33 / 31)
  auto overflow = [&]() {
    if constexpr (KMAX == 16) {
      topk_in_turns<KMAX, BF16, NT>(sh, rb, sl, tid);
    } else {
      constexpr int E = BF16 ? 8 : 4;
      const int lane = tid & 63, wave = tid >> 6;
      uint64_t l[KMAX];
#pragma unroll
      for (int j = 0; j < KMAX; ++j) l[j] = 0;
#pragma unroll
      for (int u = 0; u < NL; ++u) {
        const int c = u * NT + tid;
        if (c < sl.nfull) {
          const int v = sl.vb + c * E;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const uint32_t bits = chunk_bits<BF16>(cw[u], e);
            const uint64_t key = make_key(bits, static_cast<uint32_t>(v + e));
            if (elem_img<BF16>(bits) >= tc && key > l[KMAX - 1]) insert<KMAX>(l, key);
          }
        }
      }
      if (sl.tail) {
        const uint64_t key = make_key(bt, static_cast<uint32_t>(sl.vt));
        if (elem_img<BF16>(bt) >= tc && key > l[KMAX - 1]) insert<KMAX>(l, key);
      }
      wave_merge<KMAX>(l);
      if (lane < KMAX) {
        uint64_t mine = 0;
#pragma unroll
        for (int r = 0; r < KMAX; ++r) mine = (lane == r) ? l[r] : mine;
        sh.cand[wave * KMAX + lane] = mine;  // every wave is past its reads of sh.cand
      }
      __syncthreads();
      if (wave == 0) {
#pragma unroll
        for (int j = 0; j < KMAX; ++j) l[j] = 0;
        for (int i = lane; i < NT / PTD_WAVE * KMAX; i += PTD_WAVE) insert<KMAX>(l, sh.cand[i]);
        wave_merge<KMAX>(l);
        uint64_t mine = 0;
#pragma unroll
        for (int r = 0; r < KMAX; ++r) mine = (lane == r) ? l[r] : mine;
        if (lane < KMAX) {
          sh.out[lane] = mine;
          sh.out_bits[lane] = mine ? elem_bits<BF16>(rb, key_index(mine)) : 0u;
        }
      }
    }
  };
  topk_examine<BF16, NT>(sh, sl, tc, tid);
  __syncthreads();
  topk_pick<KMAX, BF16, NT>(sh, rb, sl, tid, overflow, [&](int rank, uint64_t key, uint32_t bits) {
    if (slices == 1) {
      const int32_t idx = static_cast<int32_t>(key_index(key));
      if (rank == 0) argmax[row] = idx;
      if (rank < k) {
        if (topk_idx) topk_idx[static_cast<size_t>(row) * k + rank] = idx;
        if (topk_val) topk_val[static_cast<size_t>(row) * k + rank] = __uint_as_float(bits);
      }
    } else {
      uint64_t* q = part + (static_cast<size_t>(blockIdx.x) * KMAX + rank) * 2;
      q[0] = key;
      q[1] = bits;
    }
  });
}

// Short unaligned rows: one wave per row, element loads.  A workgroup of
// k_topk_row costs such a row 1024 threads and several barriers: 16384 rows x 129
// bf16, k = 4: 15.3 us against 120; 1040 x 513, k = 1: 4.6 against 7.5.
template <int KMAX, bool BF16>
__global__ void __launch_bounds__(kThreads)
k_topk_wave(const void* __restrict__ logits, int R, int V, long long ld, int k,
            int32_t* __restrict__ argmax, int32_t* __restrict__ topk_idx, float* __restrict__ topk_val) {
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * (kThreads / PTD_WAVE) + (threadIdx.x >> 6);
  if (row >= R) return;  // whole wave
  const char* rb = static_cast<const char*>(logits) + static_cast<size_t>(row) * ld * (BF16 ? 2 : 4);
  uint64_t l[KMAX];
#pragma unroll
  for (int j = 0; j < KMAX; ++j) l[j] = 0;
  for (int v = lane; v < V; v += PTD_WAVE) {
    const uint64_t key = make_key(elem_bits<BF16>(rb, v), static_cast<uint32_t>(v));
    if (key > l[KMAX - 1]) insert<KMAX>(l, key);
  }
  wave_merge<KMAX>(l);
  uint64_t mine = 0;
#pragma unroll
  for (int r = 0; r < KMAX; ++r) mine = (lane == r) ? l[r] : mine;
  emit<BF16>(mine, lane, k, V, rb, row, argmax, topk_idx, topk_val);
}

// One workgroup per row: the row's slices * KMAX (key, bits) pairs are ranked
// by counting like the candidates of k_topk_row (empty slots hold key 0,
// below every element, so they never reach a rank below k <= V).  Beyond
// kThreads pairs, wave 0 merges sorted lists instead.
template <int KMAX, bool BF16>
__global__ void __launch_bounds__(kThreads)
k_topk_merge(const void* __restrict__ logits, int V, long long ld, int slices, int k,
             const uint64_t* __restrict__ part, int32_t* __restrict__ argmax,
             int32_t* __restrict__ topk_idx, float* __restrict__ topk_val) {
  __shared__ uint64_t s_key[kThreads];
  __shared__ uint32_t s_rank[kThreads];
  const int tid = threadIdx.x, lane = tid & 63, row = blockIdx.x;
  const int n = slices * KMAX;
  const uint64_t* pr = part + static_cast<size_t>(row) * n * 2;
  if (n <= kThreads) {  // uniform
    uint64_t key = 0;
    uint32_t bits = 0;
    if (tid < n) {
      key = pr[2 * tid];
      bits = static_cast<uint32_t>(pr[2 * tid + 1]);
      s_key[tid] = key;
    }
    s_rank[tid] = 0;
    __syncthreads();
    int n2 = PTD_WAVE;
    while (n2 < n) n2 <<= 1;
    const int parts = kThreads / n2;
    const int i = tid & (n2 - 1), p = tid / n2;
    const int len = (n + parts - 1) / parts;
    const int j0 = p * len, j1 = min(n, j0 + len);
    const uint64_t mine = i < n ? s_key[i] : ~0ull;
    uint32_t above = 0;
    for (int j = j0; j < j1; ++j) above += s_key[j] > mine ? 1u : 0u;
    if (above) atomicAdd(&s_rank[i], above);
    __syncthreads();
    if (tid < n) {
      const uint32_t rank = s_rank[tid];
      if (rank < static_cast<uint32_t>(k)) {
        const int32_t idx = static_cast<int32_t>(key_index(key));
        if (rank == 0) argmax[row] = idx;
        if (topk_idx) topk_idx[static_cast<size_t>(row) * k + rank] = idx;
        if (topk_val) topk_val[static_cast<size_t>(row) * k + rank] = __uint_as_float(bits);
      }
    }
    return;
  }
  if (tid >= PTD_WAVE) return;
  uint64_t l[KMAX];
#pragma unroll
  for (int j = 0; j < KMAX; ++j) l[j] = 0;
  for (int j = lane; j < n; j += PTD_WAVE) insert<KMAX>(l, pr[2 * j]);
  wave_merge<KMAX>(l);
  uint64_t mine = 0;
#pragma unroll
  for (int r = 0; r < KMAX; ++r) mine = (lane == r) ? l[r] : mine;
  const void* rb = BF16 ? static_cast<const void*>(static_cast<const uint16_t*>(logits) + row * ld)
                        : static_cast<const void*>(static_cast<const float*>(logits) + row * ld);
  emit<BF16>(mine, lane, k, V, rb, row, argmax, topk_idx, topk_val);
}

struct TopkPlan {
  int kmax, slices, slice_len;
  int nt, nl;  // k_topk_row: threads per workgroup, 16-byte chunks per lane
  bool wave;   // k_topk_wave (one slice)
  size_t ws_bytes;
};

// Workgroup shape of k_topk_row for R rows of V elements (E per chunk).
void topk_shape(int R, int V, int E, int* nt, int* nl) {
  // Many slices (at least four per CU): 512 threads of 8 chunks each, three
  // workgroups resident per CU and every lane's loads in flight at once
  // (measured on 1040 rows x 128256 bf16: 53.2 us against 72.9 us for
  // 1024 x 4).  Fewer: 1024 threads of 4 chunks, the shortest latency for a
  // slice (65 rows x 32000: 5.1 us against 5.1-7.2 us for the others), or of
  // 6 chunks when that leaves one slice per CU where 4 chunks would not
  // (65 rows x 128256: 3 slices per row, 9.2 against 9.9 us with the merge).
  const long long s4 = (static_cast<long long>(V) + 4096LL * E - 1) / (4096LL * E);
  if (static_cast<long long>(R) * s4 >= 4 * 256) {
    *nt = 512;
    *nl = 8;
  } else {
    const long long s6 = (static_cast<long long>(V) + 6144LL * E - 1) / (6144LL * E);
    *nt = 1024;
    *nl = (R * s4 > 256 && R * s6 <= 256) ? 6 : 4;
  }
}

// Which unaligned rows run one wave per row.  A wave's time grows with the row's
// elements and, by its insertions, with k; a workgroup's hardly does, but 512 of
// them run at once.  us, wave / workgroup, bf16, k = 1: 65 rows x 769 4.91 / 4.92, x 1537
// 6.3 / 4.9; 1040 rows x 1537 6.7 / 7.6, x 2049 7.9 / 7.5; 16384 rows x 2049 29 / 53.  The two meet at
// about V = 768, 1900 (1040 rows), 2700 (4160 rows), 4000 (16384 rows) for k = 1,
// 512, 1540, 2600, 4000 for k = 2, none, 700, 1700, 3000 for k = 4, and only from
// 4096 rows on for larger k.  Rows of fewer than 64 chunks leave k_topk_row without
// a bound on the k-th best value: 65 rows x 257 bf16, k = 16 17.7 / 36; fp32 rows
// of about 450 to 640 chunks with one that lists too many candidates for k > 8:
// 260 rows x 2049, k = 16 34 / 42.
bool wave_rows(int R, int V, int kmax, int E) {
  int lg = 0;  // doublings of 256 rows
  while (lg < 20 && (R >> (lg + 9)) > 0) ++lg;
  const int big = lg > 3 ? lg - 3 : 0;
  int limit = 0;
  switch (kmax) {
    case 1: limit = 768 + 512 * lg; break;
    case 2: limit = 512 + 512 * lg; break;
    case 4: limit = 420 * lg; break;
    case 8: limit = 448 * big - 192; break;
    default: limit = E == 8 ? 448 * big - 192 : 64 * big; break;
  }
  return V <= (limit < 4096 ? limit : 4096) ||
         (V < 64 * E && (kmax <= 4 || V >= (kmax == 8 && lg >= 2 ? 128 : 192))) ||
         (kmax == 16 && E == 4 && lg < 2 && V >= 1800 && V < 2560);
}

bool make_topk_plan(int R, int V, int k, int elem_bytes, bool aligned, TopkPlan* p) {
  if (R < 1 || V < 1 || k < 1 || k > PTD_MAX_K || k > V) return false;
  p->kmax = k <= 1 ? 1 : k <= 2 ? 2 : k <= 4 ? 4 : k <= 8 ? 8 : 16;
  const int E = 16 / elem_bytes;
  p->wave = !aligned && wave_rows(R, V, p->kmax, E);
  topk_shape(R, V, E, &p->nt, &p->nl);
  // A slice is at most nt * nl whole chunks (plus, for the last, a partial
  // chunk): rows longer than that are split and merged afterwards.
  const long long max_len = static_cast<long long>(p->nt) * p->nl * E;
  int s = static_cast<int>((V + max_len - 1) / max_len);
  int len = (V + s - 1) / s;
  len = (len + 7) & ~7;  // slices of an aligned row start 16-byte aligned
  s = (V + len - 1) / len;
  if (static_cast<long long>(R) * s > (1LL << 30)) return false;
  p->slices = s;
  p->slice_len = len;
  p->ws_bytes = s > 1 ? static_cast<size_t>(R) * s * p->kmax * 2 * sizeof(uint64_t) : 0;
  return true;
}

template <int KMAX, bool BF16>
void launch(const TopkPlan& pl, const void* logits, int R, int V, long long ld, int k,
            int32_t* am, int32_t* ti, float* tv, uint64_t* part, hipStream_t st) {
  if (pl.wave) {
    hipLaunchKernelGGL((k_topk_wave<KMAX, BF16>), dim3(ptd_cdiv(R, kThreads / PTD_WAVE)), dim3(kThreads), 0,
                       st, logits, R, V, ld, k, am, ti, tv);
    return;
  }
#define PTD_TOPK_ROW(nt_, nl_)                                                                   \
  if (pl.nt == nt_ && pl.nl == nl_)                                                              \
    hipLaunchKernelGGL((k_topk_row<KMAX, BF16, nt_, nl_>), dim3(R * pl.slices), dim3(nt_), 0, st, \
                       logits, V, ld, pl.slices, pl.slice_len, k, am, ti, tv, part);
  PTD_TOPK_ROW(1024, 4) PTD_TOPK_ROW(1024, 6) PTD_TOPK_ROW(512, 8)
#undef PTD_TOPK_ROW
  if (pl.slices > 1)
    hipLaunchKernelGGL((k_topk_merge<KMAX, BF16>), dim3(R), dim3(kThreads), 0, st, logits, V, ld,
                       pl.slices, k, part, am, ti, tv);
}

template <bool BF16>
void dispatch(const TopkPlan& pl, const void* logits, int R, int V, long long ld, int k,
              int32_t* am, int32_t* ti, float* tv, uint64_t* part, hipStream_t st) {
  switch (pl.kmax) {
    case 1: launch<1, BF16>(pl, logits, R, V, ld, k, am, ti, tv, part, st); break;
    case 2: launch<2, BF16>(pl, logits, R, V, ld, k, am, ti, tv, part, st); break;
    case 4: launch<4, BF16>(pl, logits, R, V, ld, k, am, ti, tv, part, st); break;
    case 8: launch<8, BF16>(pl, logits, R, V, ld, k, am, ti, tv, part, st); break;
    default: launch<16, BF16>(pl, logits, R, V, ld, k, am, ti, tv, part, st); break;
  }
}

}  // namespace

extern "C" size_t ptd_topk_workspace_bytes(int32_t R, int32_t V, int32_t k) {
  // the dtype is not known here: size for the larger of the bf16 and fp32 plans
  TopkPlan p2, p4;
  if (!make_topk_plan(R, V, k, 2, true, &p2) || !make_topk_plan(R, V, k, 4, true, &p4)) return 0;
  return p2.ws_bytes > p4.ws_bytes ? p2.ws_bytes : p4.ws_bytes;
}

extern "C" int ptd_topk_argmax(const void* logits, ptd_dtype dtype, int32_t R, int32_t V,
                               int64_t ld, int32_t k, int32_t* argmax, int32_t* topk_idx,
                               float* topk_val, void* workspace, size_t workspace_bytes,
                               void* stream) {
  PTD_RETURN_IF(!logits || !argmax, PTD_ERR_NULL);
  PTD_RETURN_IF(dtype != PTD_F32 && dtype != PTD_BF16, PTD_ERR_DTYPE);
  PTD_RETURN_IF(ld < V, PTD_ERR_SHAPE);
  const size_t es = dtype == PTD_BF16 ? 2 : 4;
  PTD_RETURN_IF(!ptd_aligned(logits, es), PTD_ERR_ALIGN);
  const bool aligned = ptd_aligned(logits, 16) && (static_cast<size_t>(ld) * es) % 16 == 0;
  TopkPlan pl;
  PTD_RETURN_IF(!make_topk_plan(R, V, k, static_cast<int>(es), aligned, &pl), PTD_ERR_SHAPE);
  if (pl.ws_bytes) {
    PTD_RETURN_IF(!workspace || workspace_bytes < pl.ws_bytes, PTD_ERR_WORKSPACE);
    PTD_RETURN_IF(!ptd_aligned(workspace, 8), PTD_ERR_ALIGN);
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  uint64_t* part = static_cast<uint64_t*>(workspace);
  if (dtype == PTD_BF16)
    dispatch<true>(pl, logits, R, V, ld, k, argmax, topk_idx, topk_val, part, st);
  else
    dispatch<false>(pl, logits, R, V, ld, k, argmax, topk_idx, topk_val, part, st);
  return ptd_launch_status();
}
