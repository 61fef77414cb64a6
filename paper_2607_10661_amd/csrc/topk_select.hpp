// Selection of the best entries of a slice of a row whose elements a workgroup holds in
// registers (ptd_topk_argmax, ptd_token_logprobs).
//
// Order: value descending, equal values by the lower vocabulary index, -0.0
// equal to +0.0.  Each element becomes one 64-bit key
//   key = orderable(value) << 32 | ~index
// so the required order is plain unsigned comparison of keys, and every key of
// a row is distinct.
#pragma once

#include "ptd_async.hpp"
#include "ptd_common.hpp"

namespace ptd {

__device__ __forceinline__ uint64_t make_key(uint32_t bits, uint32_t idx) {
  if (bits == 0x80000000u) bits = 0u;  // -0.0 ties with +0.0
  const uint32_t ord = (bits & 0x80000000u) ? ~bits : (bits | 0x80000000u);
  return (static_cast<uint64_t>(ord) << 32) | static_cast<uint32_t>(~idx);
}
__device__ __forceinline__ uint32_t key_index(uint64_t key) {
  return ~static_cast<uint32_t>(key);
}

// Order-preserving image of a float (the upper half of a key): larger value
// <=> larger image, -0 maps like +0.  Empty list slots hold 0, below every
// real value (including -inf).
__device__ __forceinline__ uint32_t ord_of(float x) {
  uint32_t bits = __float_as_uint(x);
  if (bits == 0x80000000u) bits = 0u;
  return (bits & 0x80000000u) ? ~bits : (bits | 0x80000000u);
}
template <int KMAX>
__device__ __forceinline__ void insert(uint64_t (&l)[KMAX], uint64_t key) {
  if (key > l[KMAX - 1]) {
    l[KMAX - 1] = key;
#pragma unroll
    for (int j = KMAX - 1; j > 0; --j) {
      if (l[j] > l[j - 1]) {
        const uint64_t t = l[j];
        l[j] = l[j - 1];
        l[j - 1] = t;
      }
    }
  }
}

// Top-KMAX of two descending lists, left in `a` (descending): the
// elementwise max of a and reversed b is a bitonic sequence holding the top
// KMAX, which a bitonic merge network sorts.
template <int KMAX>
__device__ __forceinline__ void merge_lists(uint64_t (&a)[KMAX], const uint64_t (&b)[KMAX]) {
#pragma unroll
  for (int i = 0; i < KMAX; ++i) a[i] = a[i] > b[KMAX - 1 - i] ? a[i] : b[KMAX - 1 - i];
#pragma unroll
  for (int j = KMAX / 2; j > 0; j >>= 1)
#pragma unroll
    for (int i = 0; i < KMAX; ++i)
      if ((i & j) == 0 && a[i] < a[i + j]) {
        const uint64_t t = a[i];
        a[i] = a[i + j];
        a[i + j] = t;
      }
}

// After the butterfly every lane holds the wave's top KMAX, descending.
template <int KMAX>
__device__ __forceinline__ void wave_merge(uint64_t (&l)[KMAX]) {
#pragma unroll
  for (int o = 1; o < PTD_WAVE; o <<= 1) {
    uint64_t other[KMAX];
#pragma unroll
    for (int i = 0; i < KMAX; ++i) other[i] = ptd::shfl_xor_u64(l[i], o);
    merge_lists<KMAX>(l, other);
  }
}

template <bool BF16>
__device__ __forceinline__ uint32_t elem_bits(const void* base, size_t i) {
  if constexpr (BF16) return static_cast<uint32_t>(static_cast<const uint16_t*>(base)[i]) << 16;
  else return static_cast<const uint32_t*>(base)[i];
}

// Where the slice of a row lies that a workgroup of NT threads holds: whole 16-byte chunks,
// chunk u of a thread being u * NT + tid, and the elements before the first 16-byte boundary
// and after the last whole chunk, one per thread.
struct Slice {
  int v0, v1;   // elements of the row
  int head;     // elements before the first boundary
  int vb;       // first element of chunk 0
  int nfull;    // whole chunks
  int vt;       // the thread's edge element, ...
  bool tail;    // ... if it has one
};
template <bool BF16>
__device__ __forceinline__ Slice slice_at(const char* rb, int v0, int v1, int tid) {
  constexpr int E = BF16 ? 8 : 4, ES = BF16 ? 2 : 4;
  Slice s;
  s.v0 = v0;
  s.v1 = v1;
  // elements before the slice's first 16-byte boundary (0 for aligned rows).
  // Rows of an odd length, or a view, start anywhere; the chunks stay aligned
  // loads and only the edges are read by element (65 rows x 32003 bf16, per
  // call: 5.5 us against 98 for a wave per row reading elements)
  const char* sb = rb + static_cast<size_t>(v0) * ES;
  s.head = min(v1 - v0, static_cast<int>((0u - static_cast<uint32_t>(reinterpret_cast<uintptr_t>(sb))) & 15u) / ES);
  s.vb = v0 + s.head;
  s.nfull = (v1 - s.vb) / E;
  // the edge elements, one per lane: the head, then the last partial chunk
  s.vt = tid < s.head ? v0 + tid : s.vb + s.nfull * E + (tid - s.head);
  s.tail = s.vt < v1;
  return s;
}
// The thread's chunks; all loads are issued before any wait (past the end: the slice's last
// chunk, never examined).
template <bool BF16, int NT, int NL>
__device__ __forceinline__ void load_chunks(uint4 (&cw)[NL], const char* rb, const Slice& s, int tid) {
  constexpr int ES = BF16 ? 2 : 4;
  if (s.nfull > 0) {
    const uint4* src = reinterpret_cast<const uint4*>(rb + static_cast<size_t>(s.vb) * ES);
#pragma unroll
    for (int u = 0; u < NL; ++u) cw[u] = src[min(u * NT + tid, s.nfull - 1)];
  } else {
#pragma unroll
    for (int u = 0; u < NL; ++u) cw[u] = make_uint4(0u, 0u, 0u, 0u);
  }
}

constexpr int kCandCap = 256;                            // LDS candidate list
constexpr int kCandPad = 8;                              // none, for whole steps of the counting
constexpr int kListCap = 256;                            // LDS chunk list

using s16x2 = short __attribute__((ext_vector_type(2)));

// Images: order-preserving integers, 0 reserved for "no element".
//   fp32: ord_of (-0 maps like +0).
//   bf16: 0x8001 + v, v the 16-bit signed-order value (sign-magnitude turned
//         into two's complement order by flipping the magnitude bits of
//         negative values).  -0 maps one below +0, so a bound equal to the
//         image of +0 is lowered to that of -0 before elements are compared.
constexpr uint32_t kImgPosZeroBf16 = 0x8001u;
template <bool BF16>
__device__ __forceinline__ uint32_t elem_img(uint32_t bits32) {  // bits of the fp32 value
  if constexpr (BF16) {
    const short h = static_cast<short>(bits32 >> 16);
    const short o = static_cast<short>(h ^ ((h >> 15) & 0x7FFF));
    return static_cast<uint32_t>(static_cast<int>(o) + 0x8001);
  } else {
    return ord_of(__uint_as_float(bits32));
  }
}
// The largest image of a chunk.  bf16: patterns of numbers with equal signs are in order as they
// are, so the largest as signed integers is the largest number if any is positive, else the
// smallest without sign is: 6 packed operations in place of 15 to put all of them in order.
template <bool BF16>
__device__ __forceinline__ uint32_t chunk_img(const uint4& c) {
  if constexpr (BF16) {
    using u16x2 = unsigned short __attribute__((ext_vector_type(2)));
    const s16x2 a = __builtin_elementwise_max(__builtin_elementwise_max(__builtin_bit_cast(s16x2, c.x), __builtin_bit_cast(s16x2, c.y)),
                                              __builtin_elementwise_max(__builtin_bit_cast(s16x2, c.z), __builtin_bit_cast(s16x2, c.w)));
    const u16x2 b = __builtin_elementwise_min(__builtin_elementwise_min(__builtin_bit_cast(u16x2, c.x), __builtin_bit_cast(u16x2, c.y)),
                                              __builtin_elementwise_min(__builtin_bit_cast(u16x2, c.z), __builtin_bit_cast(u16x2, c.w)));
    const int hi = max(static_cast<int>(a.x), static_cast<int>(a.y));
    const int lo = min(static_cast<int>(b.x), static_cast<int>(b.y));
    return static_cast<uint32_t>((hi >= 0 ? hi : ~(lo & 0x7FFF)) + 0x8001);
  } else {
    return ord_of(fmaxf(fmaxf(__uint_as_float(c.x), __uint_as_float(c.y)),
                        fmaxf(__uint_as_float(c.z), __uint_as_float(c.w))));
  }
}
// fp32 bits of element e of a chunk
template <bool BF16>
__device__ __forceinline__ uint32_t chunk_bits(const uint4& c, int e) {
  const uint32_t ws[4] = {c.x, c.y, c.z, c.w};
  if constexpr (BF16) return (e & 1) ? (ws[e >> 1] & 0xFFFF0000u) : (ws[e >> 1] << 16);
  else return ws[e];
}
// bound used in comparisons (see the bf16 image above)
template <bool BF16>
__device__ __forceinline__ uint32_t cmp_bound(uint32_t tau) {
  return (BF16 && tau == kImgPosZeroBf16) ? tau - 1 : tau;
}

// Cross-lane steps of a wave on the vector ALU, level j pairing lanes that
// differ in bit j: quad permutes (j = 0, 1), the half-row and row mirrors
// (j = 2, 3: once the value is uniform over blocks of 2^j lanes, the mirror
// partner lies in the other block), v_permlane16_swap / v_permlane32_swap
// (j = 4, 5: with both operands holding the value, the two results are the
// lane's value and its partner's).
template <bool MAX, int J>
__device__ __forceinline__ uint32_t lane_step(uint32_t x) {
  constexpr int kCtrl[4] = {0xB1, 0x4E, 0x141, 0x140};  // quad_perm 1032, 2301, half-row, row mirror
  if constexpr (J < 4) {
    const uint32_t y = static_cast<uint32_t>(
        __builtin_amdgcn_update_dpp(static_cast<int>(x), static_cast<int>(x), kCtrl[J], 0xF, 0xF, false));
    return MAX ? max(x, y) : min(x, y);
  } else {
    const auto r = J == 4 ? __builtin_amdgcn_permlane16_swap(x, x, false, false)
                          : __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return MAX ? max(r[0], r[1]) : min(r[0], r[1]);
  }
}
// Maximum over aligned groups of GL lanes, then minimum over the groups.
template <int GL>
__device__ __forceinline__ uint32_t group_max_min(uint32_t x) {
  if constexpr (GL > 1) x = lane_step<true, 0>(x); else x = lane_step<false, 0>(x);
  if constexpr (GL > 2) x = lane_step<true, 1>(x); else x = lane_step<false, 1>(x);
  if constexpr (GL > 4) x = lane_step<true, 2>(x); else x = lane_step<false, 2>(x);
  if constexpr (GL > 8) x = lane_step<true, 3>(x); else x = lane_step<false, 3>(x);
  if constexpr (GL > 16) x = lane_step<true, 4>(x); else x = lane_step<false, 4>(x);
  if constexpr (GL > 32) x = lane_step<true, 5>(x); else x = lane_step<false, 5>(x);
  return x;
}

// The wave's largest key, to every lane.
__device__ __forceinline__ uint64_t wave_max_key(uint64_t key) {
  const uint32_t hi = static_cast<uint32_t>(key >> 32);
  const uint32_t top = group_max_min<64>(hi);
  return (static_cast<uint64_t>(top) << 32) | group_max_min<64>(hi == top ? static_cast<uint32_t>(key) : 0u);
}

// LDS of the selection.
template <int NT>
struct TopkLds {
  __attribute__((aligned(16))) uint4 ldata[kListCap];
  __attribute__((aligned(16))) uint64_t cand[kCandCap + kCandPad];
  uint32_t bits[kCandCap];
  uint32_t rank[kCandCap];
  uint16_t list[kListCap];
  __attribute__((aligned(16))) uint32_t tau[NT / PTD_WAVE];
  __attribute__((aligned(16))) uint32_t tau2[NT / PTD_WAVE];
  uint64_t out[PTD_MAX_K];  // the best ones, in order (a list that overflowed)
  uint32_t out_bits[PTD_MAX_K];
  int nlist, cnt;
};

// The KMAX best entries of a slice that a workgroup of NT threads holds, NL chunks of 16 bytes
// per lane, in four parts with a barrier between them (the caller's, who may do other work
// before it): topk_groups, topk_list, topk_examine, topk_pick.
//   1. Every lane takes the image of each of its chunks and their maximum.
//   2. A lower bound tau of the slice's KMAX-th best value: the lanes of a
//      wave form KMAX groups; each group's largest lane maximum is a distinct
//      element, so the least of the KMAX group maxima is at most the KMAX-th
//      best value.  The bound of the slice is the largest bound of its waves, or the least of
//      KMAX groups of NT / KMAX lanes spanning the workgroup where that is larger (much
//      closer to the KMAX-th best value of the slice, hence few candidates; the first stays
//      positive where a short slice leaves whole workgroup-wide groups empty).
//   3. Chunks whose image reaches tau are copied with their index to a list
//      in LDS, then the workgroup examines the listed chunks a thread per
//      element and appends the elements that reach tau to a candidate list.
//      The edges of the slice (the elements before its first 16-byte
//      boundary and after its last whole chunk, fewer than two chunks) are
//      read with plain loads, one per lane, and checked the same way.  Entries at -inf are never
//      listed: masked rows have any number of them.
//   4. The candidates are ranked by counting: the list is cut into parts,
//      each thread counts the keys of one part above one candidate, and the
//      counts are summed in LDS.  Where fewer than KMAX are above -inf, all others of the slice
//      are at -inf (or NaN with the sign set, which count as such), so the first of those in order are
//      among its first KMAX entries.  If either list
//      overflows (many values tied at the top, or in order), the caller's overflow() finds them.
// Only listed chunks pass through LDS, so the slice is read from memory once
// and LDS carries a few KB.  The kernel's loops stay rolled, which keeps its
// code small: its instructions are fetched once per CU, cold.
template <int KMAX, int NT>
__device__ __forceinline__ void topk_groups(TopkLds<NT>& sh, uint32_t lm, int tid) {
  static_assert(NT >= kCandCap && NT / PTD_WAVE % 4 == 0, "workgroup shape");
  static_assert((NT & (NT - 1)) == 0, "KMAX groups of NT / KMAX lanes");
  constexpr int GL = PTD_WAVE / KMAX;  // lanes per group inside a wave
  constexpr int GW = NT / KMAX;        // lanes per group across the workgroup
  constexpr int GWL = GW < PTD_WAVE ? GW : PTD_WAVE;  // ... of them inside one wave
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (tid < kCandCap) {
    sh.rank[tid] = 0;
    sh.cand[tid] = 0;
  }
  if (tid < kCandPad) sh.cand[kCandCap + tid] = 0;
  if (tid == 0) {
    sh.cnt = 0;
    sh.nlist = 0;
  }
  const uint32_t g = group_max_min<GL>(lm);
  const uint32_t g2 = group_max_min<GWL>(lm);  // GWL = 64: the wave's maximum
  if ((tid & 63) == 0) {
    sh.tau[wave] = g;
    sh.tau2[wave] = g2;
  }
}

// Image of -inf.
template <bool BF16>
constexpr uint32_t kImgNegInf = BF16 ? 0x80u : 0x007FFFFFu;

template <int NT>
__device__ __forceinline__ void topk_append(TopkLds<NT>& sh, uint32_t bits, int v) {
  const int pos = atomicAdd(&sh.cnt, 1);
  if (pos < kCandCap) {
    sh.cand[pos] = make_key(bits, static_cast<uint32_t>(v));
    sh.bits[pos] = bits;
  }
}

// Lists what reaches the bound, which is returned.  img(u): the image of the thread's chunk u.
template <int KMAX, bool BF16, int NT, int NL, typename Img>
__device__ __forceinline__ uint32_t topk_list(TopkLds<NT>& sh, const uint4 (&cw)[NL], const Slice& s, uint32_t bt, int tid, Img img) {
  constexpr int NW = NT / PTD_WAVE;
  constexpr int GW = NT / KMAX;
  constexpr int WPG = GW < PTD_WAVE ? 1 : GW / PTD_WAVE;  // waves per workgroup-wide group
  uint32_t tau = 0;
#pragma unroll
  for (int i = 0; i < NW; i += 4) {
    const uint4 t4 = *reinterpret_cast<const uint4*>(sh.tau + i);
    tau = max(max(tau, max(t4.x, t4.y)), max(t4.z, t4.w));
  }
  uint32_t tau2 = ~0u;
#pragma unroll
  for (int j = 0; j < NW / WPG; ++j) {
    uint32_t gm = 0;
#pragma unroll
    for (int w = 0; w < WPG; ++w) gm = max(gm, sh.tau2[j * WPG + w]);
    tau2 = min(tau2, gm);
  }
  const uint32_t tc = max(cmp_bound<BF16>(max(tau, tau2)), kImgNegInf<BF16> + 1);
#pragma unroll
  for (int u = 0; u < NL; ++u) {
    if (u * NT + tid < s.nfull && img(u) >= tc) {
      const int pos = atomicAdd(&sh.nlist, 1);
      if (pos < kListCap) {
        sh.ldata[pos] = cw[u];
        sh.list[pos] = static_cast<uint16_t>(u * NT + tid);
      }
    }
  }
  if (s.tail && elem_img<BF16>(bt) >= tc) topk_append(sh, bt, s.vt);
  return tc;
}

// The best key of a thread's elements, read anew.
template <bool BF16, int NT>
__device__ __forceinline__ uint64_t best_of(const char* rb, const Slice& s, int tid) {
  constexpr int E = BF16 ? 8 : 4;
  uint64_t best = 0;
  const uint4* src = reinterpret_cast<const uint4*>(rb + static_cast<size_t>(s.vb) * (BF16 ? 2 : 4));
#pragma unroll 1
  for (int c0 = tid; c0 < s.nfull; c0 += 4 * NT) {
    uint4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = src[min(c0 + u * NT, s.nfull - 1)];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int c = c0 + u * NT;
      if (c < s.nfull) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const uint64_t key = make_key(chunk_bits<BF16>(x[u], e), static_cast<uint32_t>(s.vb + c * E + e));
          best = key > best ? key : best;
        }
      }
    }
  }
  if (s.tail) {
    const uint64_t key = make_key(elem_bits<BF16>(rb, s.vt), static_cast<uint32_t>(s.vt));
    best = key > best ? key : best;
  }
  return best;
}

// The best key below `below` of the elements of thread `owner` of the wave, which the wave reads anew,
// one of them per lane (to every lane).
template <bool BF16, int NT>
__device__ __forceinline__ uint64_t next_of(const char* rb, const Slice& s, int tid, int owner, uint64_t below) {
  constexpr int E = BF16 ? 8 : 4;
  const int lane = tid & 63, first = tid - lane + owner;
  uint64_t best = 0;
  if (lane == owner && s.tail) {
    const uint64_t key = make_key(elem_bits<BF16>(rb, s.vt), static_cast<uint32_t>(s.vt));
    best = key < below ? key : 0;
  }
  for (int c0 = first; c0 < s.nfull; c0 += PTD_WAVE / E * NT) {  // uniform
    const int c = c0 + lane / E * NT;
    if (c < s.nfull) {
      const int v = s.vb + c * E + lane % E;
      const uint64_t key = make_key(elem_bits<BF16>(rb, v), static_cast<uint32_t>(v));
      best = key < below && key > best ? key : best;
    }
  }
  return wave_max_key(best);
}

// The best keys of a slice to sh.out, one after the other: every thread looks for the best of its
// own, the best of all is taken, and its owner's wave looks for that thread's next one.
template <int KMAX, bool BF16, int NT>
__device__ __forceinline__ void topk_in_turns(TopkLds<NT>& sh, const char* rb, const Slice& s, int tid) {
  constexpr int NW = NT / PTD_WAVE;
  // (what the lanes' numbers make would be worked out ahead, in registers of the common way)
  asm volatile("" : "+v"(tid));
  uint64_t mine = best_of<BF16, NT>(rb, s, tid);
#pragma unroll 1
  for (int r = 0; r < KMAX; ++r) {
    const uint64_t w = wave_max_key(mine);
    if (r == 0) __syncthreads();  // sh.cand of the lists is read
    if ((tid & 63) == 0) sh.cand[(r & 1) * NW + (tid >> 6)] = w;
    __syncthreads();
    uint64_t best = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const uint64_t x = sh.cand[(r & 1) * NW + i];
      best = x > best ? x : best;
    }
    const uint64_t who = __ballot(best != 0 && mine == best);
    if (who) {  // whole wave
      const int owner = __builtin_ctzll(who);
      if ((tid & 63) == owner) {
        sh.out[r] = best;
        sh.out_bits[r] = elem_bits<BF16>(rb, key_index(best));
      }
      const uint64_t next = next_of<BF16, NT>(rb, s, tid, owner, best);
      if ((tid & 63) == owner) mine = next;
    } else if (best == 0 && tid == 0) {
      sh.out[r] = 0;
      sh.out_bits[r] = 0u;
    }
  }
}

// The listed chunks' elements that reach the bound become candidates.
template <bool BF16, int NT>
__device__ __forceinline__ void topk_examine(TopkLds<NT>& sh, const Slice& s, uint32_t tc, int tid) {
  constexpr int E = BF16 ? 8 : 4;  // elements per 16-byte chunk
  const int nl = sh.nlist;
  if (nl > kListCap) return;  // uniform
  for (int i0 = 0; i0 < nl; i0 += NT / E) {
    const int i = i0 + tid / E;
    if (i < nl) {
      const int c = sh.list[i], e = tid & (E - 1);
      const uint32_t bits = BF16 ? static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(sh.ldata + i)[e]) << 16
                                 : reinterpret_cast<const uint32_t*>(sh.ldata + i)[e];
      if (elem_img<BF16>(bits) >= tc) topk_append(sh, bits, s.vb + c * E + e);
    }
  }
}

// put(rank, key, bits of the fp32 value) is called once for each rank < KMAX (key 0: none), behind a
// barrier of topk_pick's own.  overflow() leaves the keys and bits in sh.out where a list overflowed.
template <int KMAX, bool BF16, int NT, typename Overflow, typename Put>
__device__ __forceinline__ void topk_pick(TopkLds<NT>& sh, const char* rb, const Slice& s, int tid, Overflow overflow, Put put) {
  const int nl = sh.nlist;
  const int n = sh.cnt;
  if (nl <= kListCap && n <= kCandCap) {  // uniform over the workgroup
    int n2 = PTD_WAVE;  // candidates per part-set: a power of two >= n
    while (n2 < n) n2 <<= 1;
    const int parts = NT / n2;
    const int i = tid & (n2 - 1), p = tid / n2;  // p is uniform over a wave
    // (in steps of 8, whose reads are in flight together; a part's end and the next one's start
    // are the same, and entries past the last are 0, above none.  256 candidates on 256 threads: 256
    // reads one after the other took 6 us)
    const int len = ((n + parts - 1) / parts + kCandPad - 1) & ~(kCandPad - 1);
    const int j0 = p * len, j1 = min((n + kCandPad - 1) & ~(kCandPad - 1), j0 + len);
    const uint64_t mine = i < n ? sh.cand[i] : ~0ull;
    uint32_t above = 0;
#pragma unroll 1
    for (int j = j0; j < j1; j += kCandPad) {
      uint64_t x[kCandPad];
#pragma unroll
      for (int t = 0; t < kCandPad; ++t) x[t] = sh.cand[j + t];
#pragma unroll
      for (int t = 0; t < kCandPad; ++t) above += x[t] > mine ? 1u : 0u;
    }
    if (above) atomicAdd(&sh.rank[i], above);
    __syncthreads();
    if (tid < n) {
      const uint32_t rank = sh.rank[tid], bits = sh.bits[tid];
      const uint64_t key = sh.cand[tid];
      if (rank < static_cast<uint32_t>(KMAX)) put(static_cast<int>(rank), key, bits);
    }
    if (n < KMAX && tid < KMAX) {  // the rest: the first entries at -inf, then none
      // (NaN with the sign set are in order with -inf: every rank below k is an entry of the row)
      const int v = s.v0 + tid;
      const uint32_t bits = v < s.v1 ? elem_bits<BF16>(rb, v) : 0u;
      const bool out = v < s.v1 && elem_img<BF16>(bits) <= kImgNegInf<BF16>;
      const uint64_t all = __ballot(out);
      const int rank = n + __popcll(all & ((1ull << tid) - 1));
      if (out && rank < KMAX) put(rank, make_key(0xFF800000u, static_cast<uint32_t>(v)), bits);
      if (tid >= n + __popcll(all)) put(tid, 0, 0);
    }
  } else {
    overflow();
    __syncthreads();
    if (tid < KMAX) put(tid, sh.out[tid], sh.out_bits[tid]);
  }
}

}  // namespace ptd
