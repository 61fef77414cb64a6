// Causal attention over packed prompts (ptd_prompt_attention) on gfx950.
//
//   out[i][h] = sum_{j <= i} softmax_j(scale * q_i . k_j) v_j   within a sequence
//
// The query heads of a KV head share its keys, so their rows are taken together:
// row r of (sequence, KV head) is position r / G, head g * G + r % G (G = Hq / Hkv).
// A tile of consecutive rows then spans few positions, which keeps the part of
// its keys that the causal mask throws away small.  One workgroup computes one
// tile over all its keys with a running maximum and sum; keys and values pass
// through a ring of tiles in LDS, filled by asynchronous copies.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "ptd_async.hpp"
#include "ptd_common.hpp"

namespace {

using ptd::dma16;
using ptd::dma16_s2;
using ptd::lds_addr;
using ptd::lds_barrier;
using ptd::wait_vmcnt;

using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x16 = float __attribute__((ext_vector_type(16)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));
using i16x4 = short __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegBig = -3.0e38f;  // running-max start: finite, below any score

struct PromptParams {
  const void* q;
  const void* k;
  const void* v;
  const int32_t* row_start;
  void* out;
  int32_t* dev_status;
  int64_t ldq, ldk, ldv;  // elements
  int B, N, Hq, Hkv, G;
  uint32_t items;  // tiles (an upper bound) * Hkv
  float c;          // scale * log2(e)
  int out_bf16;
  int wide;  // 64 rows span 2 GiB and more: no 32-bit offsets
};

// A tile: rows [r0, r0 + TM) of the M = n * G rows of a sequence that starts at
// packed row `start`, KV head g.
struct TileOf {
  int start, n, r0, g;
};

// Tile number w of all sequences' tiles; false past the last one.  Up to 64 sequences:
// longest tiles first (tile k of a sequence has k + 1 times the first one's keys), so that
// the short ones fill in at the end; more: sequence by sequence, each one's longest first,
// as levels would take a search over several looks at the starts.  (Time in order over time
// longest first, five head layouts x four mixtures of lengths: 1.01-1.05 on average for 2
// to 32 prompts, at worst 0.88 and 1.23; 0.97 for 48 and 0.93 for 64, whose keys stay in
// the L2 in order, but up to 1.31 where the longest comes last.  3 prompts of 462-1498
// rows, 40 heads: 47 against 52 us in order.)  A tile of sequence b is found after b / 64
// dependent looks at the starts, which is most of the time of thousands of short prompts
// (1024 of one row 157 us, 8192 of them 5.9 ms).  Every lane of a wave takes part.
template <int TM>
__device__ __forceinline__ bool find_tile(const PromptParams& p, uint32_t tile, TileOf& t) {
  long long w = tile;
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < p.B; b0 += PTD_WAVE) {
    const int b = b0 + lane;
    int s = 0, n = 0;
    if (b < p.B) {
      s = p.row_start[b];
      const int e = p.row_start[b + 1];
      if (s < 0 || e < s || e > p.N) {
        ptd::report(p.dev_status, PTD_ERR_ROWS);
      } else {
        n = e - s;
      }
    }
    // (n * G <= N * Hq / Hkv, checked on the host to fit an int)
    const int nt = (n * p.G + TM - 1) / TM;
    int x, k;  // sequence (lane), tile of it
    if (p.B == 1) {
      if (w >= __builtin_amdgcn_readfirstlane(nt)) return false;
      x = 0;
      k = __builtin_amdgcn_readfirstlane(nt) - 1 - static_cast<int>(w);
    } else if (p.B <= PTD_WAVE) {
      // level k: the tiles k of the sequences that have one; above it lie
      // sum max(nt - k - 1, 0) tiles.  w belongs to the least k with no more than w above it.
      if (w >= ptd::wave_sum_i32(nt)) return false;
      int lo = 0, hi = ptd::wave_max_i32(nt) - 1;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ptd::wave_sum_i32(max(nt - mid - 1, 0)) <= w) hi = mid;
        else lo = mid + 1;
      }
      k = lo;
      const int above = ptd::wave_sum_i32(max(nt - k - 1, 0));
      // the (w - above)-th of the sequences with more than k tiles
      uint64_t has = __ballot(nt > k);
      for (int i = static_cast<int>(w) - above; i > 0; --i) has &= has - 1;
      x = __builtin_ctzll(has);
    } else {
      long long up = nt;
#pragma unroll
      for (int o = 1; o < PTD_WAVE; o <<= 1) {
        const long long u = __shfl_up(up, o, PTD_WAVE);
        up += lane >= o ? u : 0;
      }
      const uint64_t past = __ballot(up > w);
      if (!past) {
        w -= __shfl(up, 63, PTD_WAVE);
        continue;
      }
      x = __builtin_ctzll(past);
      k = __builtin_amdgcn_readfirstlane(static_cast<int>(__shfl(up, x, PTD_WAVE) - w) - 1);
    }
    t.start = __builtin_amdgcn_readlane(s, x);
    t.n = __builtin_amdgcn_readlane(n, x);
    t.r0 = k * TM;
    return true;
  }
  return false;
}

// Workgroups are dealt round-robin over the 8 XCDs; a KV head's keys stay on as few of
// them (one L2 each) as its share of the work allows.
template <int TM>
__device__ __forceinline__ bool my_tile(const PromptParams& p, TileOf& t) {
  const uint32_t id = blockIdx.x + gridDim.x * blockIdx.y;
  if (id >= p.items) return false;
  const uint32_t H = p.Hkv;
  uint32_t w;
  if ((H & 7) == 0) {
    const uint32_t j = id >> 3;
    w = j / (H >> 3);
    t.g = static_cast<int>((id & 7) + 8 * (j - w * (H >> 3)));
  } else if (H <= 4 && H != 3) {
    t.g = static_cast<int>(id & (H - 1));  // (H divides 8)
    w = id / H;
  } else {
    w = id / H;
    t.g = static_cast<int>(id - w * H);
  }
  if (!find_tile<TM>(p, w, t)) return false;
  // (uniform: said so, or every loop and branch by them is made of lane masks)
  t.start = __builtin_amdgcn_readfirstlane(t.start);
  t.n = __builtin_amdgcn_readfirstlane(t.n);
  t.r0 = __builtin_amdgcn_readfirstlane(t.r0);
  t.g = __builtin_amdgcn_readfirstlane(t.g);
  return true;
}

__device__ __forceinline__ float max_xor32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_xor32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Sum of a bf16 pair and an fp32 number (v_dot2_f32_bf16 with a pair of ones).
__device__ __forceinline__ float sum_bf16x2(uint32_t w, float acc) {
  using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3F803F80u), acc, false);
}
__device__ __forceinline__ u32x2 lds_read_tr16(const unsigned char* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((PTD_LDS i16x4*)p));
}

// ===========================================================================
// bf16: v_mfma_f32_32x32x16_bf16
// ===========================================================================
// Scores are computed transposed, S^T = K Q^T, and the output as O^T = V^T P^T: a
// lane owns query row l % 32 in both accumulators (keys, or columns of V, 8 * (i / 4) +
// 4 * (l / 32) + i % 4 in element i), so the softmax needs one exchange between
// two lanes, and only when the reference maximum moves.  V is read transposed from
// its natural layout (ds_read_b64_tr_b16).
//
// LDS: a tile of 64 keys, K rows then V rows, row-major in 16-byte chunks.  Chunk c of row r
// lies at c ^ swz(r): for K, so that 16 rows x one chunk (a quarter of a ds_read_b128)
// fall on 16 different places of 256 bytes; for V, so that 4 rows x 4 chunks (half of a
// transposing read) do.
//
// The weights are rounded to bf16 as the operand of O^T (two operands, the number and what
// its rounding leaves, would be half as many products again), and their sum is that of the
// rounded ones, in fp32, so that the output is an exact average under weights off by at most
// 2^-8 of themselves: bf16 outputs over up to 8192 keys are off by 0.0020 of their size
// (their own rounding makes 0.0015 of it).
//
// Bound, where prompts are long, by what two waves per SIMD issue at the clock that the
// products leave the card (about 1.9 GHz): 8192 rows of 32 / 8 heads x 128 take 484-504 us,
// 1090-1140 TFLOP/s, with the matrix units busy for 57 % of the cycles (a large matrix product
// reaches 1214 TFLOP/s, all-zero inputs run at 1370); a batch of 17-2048 rows, 36 %, waits
// more.  The clock settles after some 100 such calls; the first ones of an idle card take
// 515 to 666 us.  Two workgroups of four waves per CU, so that one's softmax and
// barriers run beside the other's products: 128 rows a workgroup.  256 rows and eight waves
// took 623 against 585 us there, 32-key tiles and three waves per SIMD (registers
// spill) 355 against 241 on 16 prompts of 17-2048 rows, four tiles in flight and one
// workgroup per CU 30.9 against 27.3 on 1024 rows.  Short prompts wait for memory and
// for find_tile: 1-64 rows take 6 us, launch included.
constexpr int kThreads = 256;  // four waves of 32 rows
template <int D>
struct Tiles {
  static constexpr int KEYS = 64;
  static constexpr int RB = D * 2;             // bytes per row
  static constexpr int CH = RB / 16;           // chunks per row
  static constexpr int PART = KEYS * RB;       // K (or V) bytes
  static constexpr int SLOT = 2 * PART;
  static constexpr int CPT = KEYS * CH / kThreads;  // copies per thread of K (and of V)
  static constexpr int NS = 2;                    // tiles in the ring: one is read while the next lands
  static_assert(CPT * kThreads == KEYS * CH, "copies divide");
  __device__ static int swz_k(int r) { return CH == 16 ? r & 15 : (r >> 1) & 7; }
  __device__ static int swz_v(int r) {
    return CH == 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  }
};

template <int D>
__global__ void __launch_bounds__(kThreads, 2) k_prompt_bf16(PromptParams p) {
  using L = Tiles<D>;
  constexpr int NS = L::NS;
  constexpr int NW = kThreads / PTD_WAVE;
  constexpr int TM = 32 * NW;
  constexpr int DB = D / 16;  // QK^T steps
  constexpr int DT = D / 32;  // 32-column parts of O
  __shared__ __attribute__((aligned(16))) unsigned char smem[NS * L::SLOT];
  __shared__ int s_odd[2][NW];  // by parity of the tile, for each wave

  TileOf t;
  if (!my_tile<TM>(p, t)) return;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int l32 = lane & 31, h = lane >> 5;
  const int M = t.n * p.G;

  // ---- this lane's query row
  const int row = t.r0 + wave * 32 + l32;
  const int rc = min(row, M - 1);
  const int pos = rc / p.G, hq = t.g * p.G + rc % p.G;
  // ---- tile copies
  const uint16_t* kbase = static_cast<const uint16_t*>(p.k) + static_cast<size_t>(t.start) * p.ldk + static_cast<size_t>(t.g) * D;
  const uint16_t* vbase = static_cast<const uint16_t*>(p.v) + static_cast<size_t>(t.start) * p.ldv + static_cast<size_t>(t.g) * D;
  const uint32_t ring = lds_addr(smem);
  uint32_t c_k[L::CPT], c_v[L::CPT];  // byte offsets of this thread's chunks in a tile
#pragma unroll
  for (int u = 0; u < L::CPT; ++u) {
    const int c = u * kThreads + tid, r = c / L::CH;
    c_k[u] = static_cast<uint32_t>((r * p.ldk + ((c % L::CH) ^ L::swz_k(r)) * 8) * 2);
    c_v[u] = static_cast<uint32_t>((r * p.ldv + ((c % L::CH) ^ L::swz_v(r)) * 8) * 2);
  }
  auto issue = [&](int tt) __attribute__((always_inline)) {
    const uint32_t dst = ring + (tt % NS) * L::SLOT + wave * PTD_WAVE * 16;
    if ((tt + 1) * L::KEYS <= t.n && !p.wide) {  // uniform: a whole tile, from scalar bases
      const uint16_t* kt = kbase + static_cast<size_t>(tt) * L::KEYS * p.ldk;
      const uint16_t* vt = vbase + static_cast<size_t>(tt) * L::KEYS * p.ldv;
#pragma unroll
      for (int u = 0; u < L::CPT; ++u) dma16_s2(kt, c_k[u], dst + u * kThreads * 16, vt, c_v[u], dst + L::PART + u * kThreads * 16);
    } else {
#pragma unroll
      for (int u = 0; u < L::CPT; ++u) {
        const int c = u * kThreads + tid, r = c / L::CH;
        const size_t key = min(tt * L::KEYS + r, t.n - 1);  // past the sequence: its last row again
        dma16(kbase + key * p.ldk + ((c % L::CH) ^ L::swz_k(r)) * 8, dst + u * kThreads * 16);
        dma16(vbase + key * p.ldv + ((c % L::CH) ^ L::swz_v(r)) * 8, dst + L::PART + u * kThreads * 16);
      }
    }
  };
  // keys up to the tile's last position
  const int last = (min(t.r0 + TM, M) - 1) / p.G;
  const int ntiles = last / L::KEYS + 1;
  issue(0);
  const uint16_t* qr = static_cast<const uint16_t*>(p.q) + static_cast<size_t>(t.start + pos) * p.ldq +
                       static_cast<size_t>(hq) * D + 8 * h;
  bf16x8 qf[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i) qf[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qr + 16 * i));
  // waited for here: a load pending at the loop would make the compiler wait for every copy
#pragma unroll
  for (int i = 0; i < DB; ++i) asm volatile("" : "+v"(qf[i]));
  // last position of the wave's rows
  const int wave_hi = min(t.r0 + wave * 32 + 31, M - 1) / p.G;

  int koff[DB], voff[2][DT];
#pragma unroll
  for (int i = 0; i < DB; ++i) koff[i] = l32 * L::RB + ((2 * i + h) ^ L::swz_k(l32)) * 16;
  // source lane 4 j + q of a group of 16 points at V[key j][.. + 4 q]; the group's
  // lane i receives its four keys' values of column i
  const int l16 = lane & 15, vrow = 4 * h + (l16 >> 2), q4 = l16 & 3, dsub = (lane >> 4) & 1;
  // (rows 16 apart are permuted alike)
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      voff[i][dt] = L::PART + (vrow + 8 * i) * L::RB + (q4 & 1) * 8 + ((4 * dt + 2 * dsub + (q4 >> 1)) ^ L::swz_v(vrow + 8 * i)) * 16;

  f32x16 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  // (finite at every scale: it stays where a row's first keys score -inf, and inf - inf is NaN)
  float m = kNegBig, nmc = fminf(-kNegBig * p.c, -kNegBig), l = 0.f;

  // scores of 32 keys
  auto qk = [&](const unsigned char* slot, int kb) __attribute__((always_inline)) {
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int i = 0; i < DB; ++i) {
      const bf16x8 kf = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(slot + kb * 32 * L::RB + koff[i]));
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[i], s, 0, 0, 0);
    }
    return s;
  };
  // weights 2^((s - m) c) as bf16 pairs, and the sum of what they were rounded to
  struct Weights {
    uint32_t w[8];
    float sum;
  };
  auto exps = [&](const f32x16& s) __attribute__((always_inline)) {
    Weights r;
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      r.w[w] = ptd::cvt_pk_bf16(__builtin_amdgcn_exp2f(fmaf(s[2 * w], p.c, nmc)),
                                __builtin_amdgcn_exp2f(fmaf(s[2 * w + 1], p.c, nmc)));
      if (w & 1) b = sum_bf16x2(r.w[w], b);
      else a = sum_bf16x2(r.w[w], a);
    }
    r.sum = a + b;
    return r;
  };
  // A row's reference m stays while its weights are far inside the fp32 range; else it
  // moves to the row's maximum (always at its first keys), whatever the other rows do.
  auto settle = [&](const f32x16& s, Weights& r, uint64_t over) __attribute__((always_inline)) {
    if (over) {
#pragma clang fp contract(off)
      const bool mine = ((static_cast<uint32_t>(over) | static_cast<uint32_t>(over >> 32)) >> l32) & 1u;
      float mx = s[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
      mx = max_xor32(mx);
      const bool up = mine && mx > m;
      // (from the products as they were rounded, hence no contraction here: for large
      // scores the rounding is more than the weights' own steps)
      const float to = up ? -mx * p.c : nmc;
      const float alpha = __builtin_amdgcn_exp2f(to - nmc);
      m = up ? mx : m;
      nmc = to;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= alpha;
      r = exps(s);
    }
    l += r.sum;
  };
  auto over_of = [](const Weights& r) __attribute__((always_inline)) { return __ballot(!(r.sum <= 65536.f)); };
  struct Values {
    u32x4 v[2][DT];
  };
  auto read_v = [&](const unsigned char* slot, int kb) __attribute__((always_inline)) {
    Values r;
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const u32x2 a = lds_read_tr16(slot + voff[0][dt] + (32 * kb + 16 * st) * L::RB);
        const u32x2 b = lds_read_tr16(slot + voff[1][dt] + (32 * kb + 16 * st) * L::RB);
        r.v[st][dt] = u32x4{a[0], a[1], b[0], b[1]};
      }
    return r;
  };
  auto pv = [&](const Values& v, const Weights& r) __attribute__((always_inline)) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      const bf16x8 pf = __builtin_bit_cast(bf16x8, u32x4{r.w[4 * st], r.w[4 * st + 1], r.w[4 * st + 2], r.w[4 * st + 3]});
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v.v[st][dt]), pf, o[dt], 0, 0, 0);
    }
  };
  // A tile that every row sees whole.  The second half's QK^T runs beside the first half's
  // exponentials, the first half's PV beside the second's.
  auto full_tile = [&](const unsigned char* slot, bool first, auto&& among) __attribute__((always_inline)) {
    const f32x16 s0 = qk(slot, 0);
    among(0);
    const f32x16 s1 = qk(slot, 1);
    among(1);
    Weights w0;
    uint64_t over = ~0ull;
    if (!first) {
      w0 = exps(s0);
      over = over_of(w0);
    }
    settle(s0, w0, over);
    among(2);
    Weights w1 = exps(s1);
    pv(read_v(slot, 0), w0);
    settle(s1, w1, over_of(w1));
    among(3);
    pv(read_v(slot, 1), w1);
  };
  // a tile at some row's end: scores of keys behind a row's position become -inf
  auto end_tile = [&](const unsigned char* slot, int k0, bool first) __attribute__((always_inline)) {
    const int lim = pos - k0 - 4 * h;
    for (int kb = 0; kb < 2 && k0 + 32 * kb <= wave_hi; ++kb) {  // uniform
      f32x16 s = qk(slot + kb * 32 * L::RB, 0);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 32 * kb + 8 * (e / 4) + e % 4 <= lim ? s[e] : -INFINITY;
      Weights w = exps(s);
      settle(s, w, first && kb == 0 ? ~0ull : over_of(w));
      pv(read_v(slot + kb * 32 * L::RB, 0), w);
    }
  };
  // A tile that not every row sees whole: 0 * inf must not reach a row that does not
  // see the key.  Each thread clears what is not finite from the value chunks that it
  // copied, before the barrier that shows them to the others; the rows that do see such
  // a value get it after the tile, from memory (rare).
  auto clear_odd = [&](int tt) __attribute__((always_inline)) {
    unsigned char* own = smem + (tt % NS) * L::SLOT + L::PART + tid * 16;
    uint32_t top = 0;
    u32x4 w[L::CPT];
#pragma unroll
    for (int u = 0; u < L::CPT; ++u) {
      w[u] = *reinterpret_cast<const u32x4*>(own + u * kThreads * 16);
#pragma unroll
      for (int x = 0; x < 4; ++x) top |= (w[u][x] & 0x7F807F80u) + 0x00800080u;  // bits 15, 31: exponent all ones
    }
    const bool odd = __any((top & 0x80008000u) != 0);
    if (odd) {
#pragma unroll
      for (int u = 0; u < L::CPT; ++u) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
          w[u][x] &= ((w[u][x] & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) | ((w[u][x] & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
        *reinterpret_cast<u32x4*>(own + u * kThreads * 16) = w[u];
      }
    }
    if (lane == 0) s_odd[tt & 1][wave] = odd;
  };
  auto add_odd = [&](int tt) __attribute__((always_inline)) {
    int any = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) any |= s_odd[tt & 1][w];
    if (!__builtin_amdgcn_readfirstlane(any)) return;
    const int end = min((tt + 1) * L::KEYS, t.n);
    for (int key = tt * L::KEYS; key < end; ++key) {
      const uint16_t* vr = vbase + static_cast<size_t>(key) * p.ldv + 4 * h;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const u32x2 x = *reinterpret_cast<const u32x2*>(vr + 32 * dt + 8 * e4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t f = (e & 1) ? x[e >> 1] & 0xFFFF0000u : x[e >> 1] << 16;
            const bool add = key <= pos && (f & 0x7F800000u) == 0x7F800000u;
            o[dt][4 * e4 + e] += add ? __uint_as_float(f) : 0.f;
          }
        }
    }
  };
  // tile tt has landed; every wave is done with tile tt - 1, whose place is filled next
  auto next = [&](int tt, bool ends) __attribute__((always_inline)) {
    wait_vmcnt<0>();
    if (ends) clear_odd(tt);
    lds_barrier();
    if (tt + 1 < ntiles) issue(tt + 1);
  };
  // tiles that every row of the workgroup sees whole, then those that end at some row
  // (the last tile is among these: a full one has a next one)
  const int full = min((t.r0 / p.G + 1) / L::KEYS, ntiles - 1);
  int tt = 0;
  auto nothing = [](int) __attribute__((always_inline)) {};
  if (full > 0) {
    next(0, false);
    full_tile(smem, true, nothing);
    tt = 1;
  }
  // Two tiles a turn: their places in LDS are constants of the instructions.  The next
  // tile's copies are issued among a tile's products, a quarter at a time: together they
  // keep a wave at the vector memory unit for 600 of a tile's 2900 cycles.
  const int whole = p.wide ? 0 : min(full, t.n / L::KEYS - 1);  // tiles before a whole one
  auto spread = [&](int tt, int place) __attribute__((always_inline)) {
    const uint16_t* kt = kbase + static_cast<size_t>(tt) * L::KEYS * p.ldk;
    const uint16_t* vt = vbase + static_cast<size_t>(tt) * L::KEYS * p.ldv;
    const uint32_t dst = ring + place * L::SLOT + wave * PTD_WAVE * 16;
    return [=](int q) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < L::CPT; ++u)
        if (u * 4 / L::CPT == q)
          ptd::dma16_s2_among(kt, c_k[u], dst + u * kThreads * 16, vt, c_v[u], dst + L::PART + u * kThreads * 16);
    };
  };
  for (; tt + 1 < whole; tt += 2) {
    wait_vmcnt<0>();
    lds_barrier();
    full_tile(smem + L::SLOT, false, spread(tt + 1, 0));
    wait_vmcnt<0>();
    lds_barrier();
    full_tile(smem, false, spread(tt + 2, 1));
  }
  for (; tt < full; ++tt) {
    next(tt, false);
    full_tile(smem + (tt % NS) * L::SLOT, false, nothing);
  }
  for (; tt < ntiles; ++tt) {
    next(tt, true);
    if (tt * L::KEYS <= wave_hi) {  // uniform over the wave
      end_tile(smem + (tt % NS) * L::SLOT, tt * L::KEYS, tt == 0);
      add_odd(tt);
    }
  }
  if (row >= M) return;
  const float inv = 1.f / sum_xor32(l);
  const size_t off = (static_cast<size_t>(t.start + pos) * p.Hq + hq) * D + 4 * h;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const f32x4 v = {o[dt][4 * e4] * inv, o[dt][4 * e4 + 1] * inv, o[dt][4 * e4 + 2] * inv, o[dt][4 * e4 + 3] * inv};
      const size_t at = off + 32 * dt + 8 * e4;
      if (p.out_bf16) {
        const u32x2 w = {ptd::cvt_pk_bf16(v[0], v[1]), ptd::cvt_pk_bf16(v[2], v[3])};
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + at) = w;
      } else {
        *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at) = v;
      }
    }
}

// ===========================================================================
// fp32: v_mfma_f32_32x32x2_f32
// ===========================================================================
// An MFMA takes 64 cycles for 4096 products, so operands need not be shared: the eight
// waves of a workgroup hold the same 32 rows and take every eighth tile of 32 keys, each
// straight from memory into registers, with a maximum and sum of its own; the
// states merge through LDS at the end.  No barrier in between, and a row of n keys
// waits for n / 256 tiles, not n / 32.  K is loaded when it is needed and V behind the
// scores, into the same registers; the SIMD's other wave covers the waits (V and
// the next K loaded ahead: 17.1 against 15.5 us on 512 rows of 4 heads x 64, and for D =
// 128 the registers spill, 35.7 against 25.5).  Four waves over one ring in LDS, a
// wave per 32 rows and all its keys, took 48.8 us there.
//   S^T = K Q^T: step (j, e) contracts the columns 8 j + 4 h + e of 16-byte loads.
//   O^T = V^T P^T: step e contracts the keys 8 * (e / 4) + 4 h + e % 4, whose weights the
//   lane owns; row r of part dt stands for column DT * r + dt, so that a lane's loads are
//   DT consecutive elements, and so are its outputs.
// Short prompts make too few workgroups: four prompts of 58-370 rows, 4 / 2 heads x 64, take
// 13 us with 80 of them on 256 CUs, of which the longest's 12 tiles are 5 us of products on
// its four SIMDs, the rest waits for memory.  2048 rows of 32 / 8 heads x 128 take 353 us, 97
// TFLOP/s (a large fp32 product: 153).
constexpr int kF32Threads = 512;
constexpr int kF32Waves = kF32Threads / PTD_WAVE;

template <int D>
__global__ void __launch_bounds__(kF32Threads, 2) k_prompt_f32(PromptParams p) {
  constexpr int TM = 32, KEYS = 32, CH = D / 4, KJ = D / 8, DT = D / 32;
  using fvec = float __attribute__((ext_vector_type(DT)));
  // rows in 16-byte chunks, chunk c of row r at c ^ (r mod 16)
  __shared__ __attribute__((aligned(16))) float sq[TM * D];
  __shared__ __attribute__((aligned(16))) float so[kF32Waves][TM * D];
  __shared__ float2 sml[kF32Waves][TM];
  auto chunk = [](int r, int c) __attribute__((always_inline)) { return (r * CH + (c ^ (r & 15))) * 4; };

  TileOf t;
  if (!my_tile<TM>(p, t)) return;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int l32 = lane & 31, h = lane >> 5;
  const int M = t.n * p.G;
  const int pos = min(t.r0 + l32, M - 1) / p.G;  // this lane's query row
  const int lo = t.r0 / p.G, hi = (min(t.r0 + TM, M) - 1) / p.G;
  const int ntiles = hi / KEYS + 1;
  const float* kbase = static_cast<const float*>(p.k) + static_cast<size_t>(t.start) * p.ldk + static_cast<size_t>(t.g) * D;
  const float* vbase = static_cast<const float*>(p.v) + static_cast<size_t>(t.start) * p.ldv + static_cast<size_t>(t.g) * D;

  f32x4 kf[KJ];
  // whole tiles from scalar bases and 32-bit offsets: addresses in 64 bits would not
  // leave the registers for the tiles in flight
  const uint32_t koff = static_cast<uint32_t>(l32 * p.ldk + 4 * h) * 4u;
  const uint32_t voff = static_cast<uint32_t>(4 * h * p.ldv + DT * l32) * 4u;
  auto whole = [&](int tt) __attribute__((always_inline)) { return (tt + 1) * KEYS <= t.n && !p.wide; };
  auto load_k = [&](int tt) __attribute__((always_inline)) {
    if (whole(tt)) {
      const char* src = reinterpret_cast<const char*>(kbase + static_cast<size_t>(tt) * KEYS * p.ldk);
#pragma unroll
      for (int j = 0; j < KJ; ++j) kf[j] = *reinterpret_cast<const f32x4*>(src + koff + 32 * j);
    } else {
      const float* src = kbase + static_cast<size_t>(min(tt * KEYS + l32, t.n - 1)) * p.ldk + 4 * h;
#pragma unroll
      for (int j = 0; j < KJ; ++j) kf[j] = *reinterpret_cast<const f32x4*>(src + 8 * j);
    }
  };
  for (int x = tid; x < TM * CH; x += kF32Threads) {
    const int r = x / CH, c = x % CH, rr = min(t.r0 + r, M - 1);
    const float* src = static_cast<const float*>(p.q) + static_cast<size_t>(t.start + rr / p.G) * p.ldq +
                       static_cast<size_t>(t.g * p.G + rr % p.G) * D;
    *reinterpret_cast<f32x4*>(sq + chunk(r, c)) = *reinterpret_cast<const f32x4*>(src + 4 * c);
  }
  __syncthreads();

  f32x16 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = kNegBig, l = 0.f;  // l: this lane's keys only
  for (int tt = wave; tt < ntiles; tt += kF32Waves) {
    const int k0 = tt * KEYS;
    fvec vf[16];
    auto load_v = [&]() __attribute__((always_inline)) {
      if (whole(tt)) {
        const char* src = reinterpret_cast<const char*>(vbase + static_cast<size_t>(k0) * p.ldv);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          vf[e] = *reinterpret_cast<const fvec*>(src + static_cast<size_t>(8 * (e / 4) + e % 4) * p.ldv * 4 + voff);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = min(k0 + 8 * (e / 4) + 4 * h + e % 4, t.n - 1);
          vf[e] = *reinterpret_cast<const fvec*>(vbase + static_cast<size_t>(key) * p.ldv + DT * l32);
        }
      }
    };
    load_k(tt);
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
      const f32x4 qv = *reinterpret_cast<const f32x4*>(sq + chunk(l32, 2 * j + h));
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j][e], qv[e], s, 0, 0, 0);
    }
    load_v();
    const bool ends = k0 + KEYS - 1 > lo;  // uniform: some row does not see all of the tile
    bool odd = false;
    if (ends) {
      const int lim = pos - k0 - 4 * h;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 8 * (e / 4) + e % 4 <= lim ? s[e] : -INFINITY;
      // 0 * inf must not reach a row that does not see the key
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const bool bad = (__float_as_uint(vf[e][dt]) & 0x7F800000u) == 0x7F800000u;
          odd |= bad;
          vf[e][dt] = bad ? 0.f : vf[e][dt];
        }
    }
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
    mx = fmaxf(m, max_xor32(mx));
    const float alpha = __builtin_amdgcn_exp2f((m - mx) * p.c);
    m = mx;
    float ps = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = __builtin_amdgcn_exp2f((s[e] - mx) * p.c);
      ps += s[e];
    }
    l = fmaf(l, alpha, ps);
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] *= alpha;
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      if (k0 + 8 * e4 > hi) break;  // uniform: keys that no row sees
#pragma unroll
      for (int e = 4 * e4; e < 4 * e4 + 4; ++e)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[e][dt], s[e], o[dt], 0, 0, 0);
    }
    if (ends && __any(odd)) {  // rare: what is not finite, to the rows that see it
      const int end = min(k0 + KEYS, t.n);
      for (int key = k0; key < end; ++key)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const fvec f = *reinterpret_cast<const fvec*>(vbase + static_cast<size_t>(key) * p.ldv + DT * (8 * (e / 4) + 4 * h + e % 4));
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const bool add = key <= pos && (__float_as_uint(f[dt]) & 0x7F800000u) == 0x7F800000u;
            o[dt][e] += add ? f[dt] : 0.f;
          }
        }
    }
  }

  // ---- merge of the waves
  l = sum_xor32(l);
  if (h == 0) sml[wave][l32] = make_float2(m, l);
  if (wave < ntiles) {
#pragma unroll
    for (int e = 0; e < 16; e += 4 / DT) {  // four consecutive columns from 4 / DT elements
      const int r = 8 * (e / 4) + 4 * h + e % 4;
      f32x4 x;
#pragma unroll
      for (int y = 0; y < 4; ++y) x[y] = o[y % DT][e + y / DT];
      *reinterpret_cast<f32x4*>(&so[wave][chunk(l32, r * DT / 4)]) = x;
    }
  }
  __syncthreads();
  const int nw = min(ntiles, kF32Waves);
  for (int x = tid; x < TM * CH; x += kF32Threads) {
    const int r = x / CH, c = x % CH, rr = t.r0 + r;
    if (rr >= M) break;
    float mm = kNegBig;
    for (int w = 0; w < nw; ++w) mm = fmaxf(mm, sml[w][r].x);
    float den = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < nw; ++w) {
      const float2 ml = sml[w][r];
      const float f = __builtin_amdgcn_exp2f((ml.x - mm) * p.c);
      den = fmaf(f, ml.y, den);
      acc += *reinterpret_cast<const f32x4*>(&so[w][chunk(r, c)]) * f;
    }
    const f32x4 v = acc * (1.f / den);
    const size_t at = (static_cast<size_t>(t.start + rr / p.G) * p.Hq + t.g * p.G + rr % p.G) * D + 4 * c;
    if (p.out_bf16) {
      const u32x2 w = {ptd::cvt_pk_bf16(v[0], v[1]), ptd::cvt_pk_bf16(v[2], v[3])};
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + at) = w;
    } else {
      *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at) = v;
    }
  }
}

}  // namespace

extern "C" int ptd_prompt_attention(const void* q, const void* k, const void* v,
                                    const int32_t* row_start, void* out,
                                    const ptd_prompt_shape* shape, int32_t* dev_status,
                                    void* stream) {
  PTD_RETURN_IF(!shape || !row_start, PTD_ERR_NULL);
  const ptd_prompt_shape& s = *shape;
  PTD_RETURN_IF(s.N > 0 && (!q || !k || !v || !out), PTD_ERR_NULL);
  PTD_RETURN_IF((s.in_dtype != PTD_F32 && s.in_dtype != PTD_BF16) ||
                    (s.out_dtype != PTD_F32 && s.out_dtype != PTD_BF16),
                PTD_ERR_DTYPE);
  PTD_RETURN_IF(s.B < 1 || s.B > 65536 || s.N < 0 || s.Hq < 1 || s.Hkv < 1 || s.Hq % s.Hkv != 0, PTD_ERR_SHAPE);
  PTD_RETURN_IF(s.D != 64 && s.D != 128, PTD_ERR_SHAPE);
  PTD_RETURN_IF(static_cast<long long>(s.N) * s.Hq > 0x7FFFFFFFLL, PTD_ERR_SHAPE);
  PTD_RETURN_IF(!(s.scale >= 0.f) || !isfinite(s.scale), PTD_ERR_SHAPE);
  PromptParams prm;
  const int64_t wq = static_cast<int64_t>(s.Hq) * s.D, wk = static_cast<int64_t>(s.Hkv) * s.D;
  prm.ldq = s.ldq ? s.ldq : wq;
  prm.ldk = s.ldk ? s.ldk : wk;
  prm.ldv = s.ldv ? s.ldv : wk;
  PTD_RETURN_IF(prm.ldq < wq || prm.ldk < wk || prm.ldv < wk, PTD_ERR_SHAPE);
  const int per16 = s.in_dtype == PTD_F32 ? 4 : 8;
  PTD_RETURN_IF(prm.ldq % per16 || prm.ldk % per16 || prm.ldv % per16 || !ptd_aligned(q, 16) ||
                    !ptd_aligned(k, 16) || !ptd_aligned(v, 16) || !ptd_aligned(out, 16),
                PTD_ERR_ALIGN);
  if (s.N == 0) return PTD_OK;
  prm.wide = std::max(prm.ldk, prm.ldv) >= (1 << 24);
  prm.q = q;
  prm.k = k;
  prm.v = v;
  prm.row_start = row_start;
  prm.out = out;
  prm.dev_status = dev_status;
  prm.B = s.B;
  prm.N = s.N;
  prm.Hq = s.Hq;
  prm.Hkv = s.Hkv;
  prm.G = s.Hq / s.Hkv;
  prm.c = (s.scale > 0.f ? s.scale : 1.0f / sqrtf(static_cast<float>(s.D))) * kLog2e;
  prm.out_bf16 = s.out_dtype == PTD_BF16;
  // every sequence has at most one tile that is not full; one more of none where the
  // starts take several looks, so that somebody sees the last of them
  const auto items_of = [&](int tm) {
    return (static_cast<long long>(s.N) * prm.G / tm + std::min(s.B, s.N) + (s.B > PTD_WAVE ? 1 : 0)) * s.Hkv;
  };
  // (the grid is rounded up to a multiple of 8 and of its first dimension: all ids fit 32 bits)
  PTD_RETURN_IF(items_of(32) > 0x7FFFFFFFLL, PTD_ERR_SHAPE);
  const auto grid_of = [&](long long items) {  // two dimensions: one holds fewer than 2^32 threads
    const long long x = std::min<long long>((items + 7) / 8 * 8, 1 << 20);
    return dim3(static_cast<unsigned>(x), static_cast<unsigned>((items + x - 1) / x));
  };
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (s.in_dtype == PTD_F32) {
    prm.items = static_cast<uint32_t>(items_of(32));
    const dim3 grid = grid_of(prm.items);
    if (s.D == 128) hipLaunchKernelGGL(k_prompt_f32<128>, grid, dim3(kF32Threads), 0, st, prm);
    else hipLaunchKernelGGL(k_prompt_f32<64>, grid, dim3(kF32Threads), 0, st, prm);
  } else {
    prm.items = static_cast<uint32_t>(items_of(128));
    const dim3 grid = grid_of(prm.items);
    if (s.D == 128) hipLaunchKernelGGL(k_prompt_bf16<128>, grid, dim3(kThreads), 0, st, prm);
    else hipLaunchKernelGGL(k_prompt_bf16<64>, grid, dim3(kThreads), 0, st, prm);
  }
  return ptd_launch_status();
}
