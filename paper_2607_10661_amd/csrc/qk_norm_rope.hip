// Norm of every query and key head, rotation by the rows' positions, and the rows of
// keys and values into the pages of the caches, in one pass (ptd_qk_norm_rope).
//
//   y = x * w / sqrt(mean(x^2) + eps),  then dimension pair p < rot / 2 of y is turned by
//   positions[i] * inv_freq[p]
//
// Eight lanes (four for D = 64) hold a head, 16 elements each: the elements of a lane are
// whole pairs, so the sum of squares is the only thing that passes between lanes, three DPP
// steps.  A wave works on one row: its lanes compute one angle each, and the 8 cosines and sines
// of a lane's pairs stay in its registers for all heads that the wave takes.
#include <math.h>

#include <algorithm>

#include "ptd_common.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / PTD_WAVE;
constexpr int kMaxHalf = 64;  // rot / 2 for D <= 128
constexpr int kMaxRows = (1 << 26) - kWaves;  // a wave each: a grid holds fewer than 2^32 threads

using u32x4 = uint32_t __attribute__((ext_vector_type(4)));

struct QkArgs {
  const void* in[3];        // rows of queries, keys, values
  void* out[2];             // rows of queries, keys (or null)
  const void* w[2];         // weights of the norms (or null)
  void* pages[2];           // keys, values (or null)
  const int32_t* positions; // or null
  const int32_t* slots;
  int32_t* dev_status;
  int64_t ld_in[3], ld_out[2];  // elements
  int heads[2];             // of queries, of keys and values
  int N, rot, w_bf16, waves_per_row, page_size, num_pages;
  float eps;
  double inv_freq[kMaxHalf];
};

// cos and sin of a >= 0 (any size that a position can give), in fp64: a less its multiple of
// pi / 2 (two doubles of it, which leave less than the rounding of the angle), then the series of both up to
// the 16th power of |r| <= pi / 4 (what follows is below 2^-54).
__device__ __forceinline__ float2 cos_sin(double a) {
  const double n = rint(a * 0x1.45f306dc9c883p-1);  // 2 / pi
  double r = fma(-n, 0x1.921fb54442d18p+0, a);      // pi / 2 as a double, the rest of it, ...
  r = fma(-n, 0x1.1a62633145c07p-54, r);
  const double z = r * r;
  double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
  s = fma(s, z, 1.0 / 6227020800.0), c = fma(c, z, -1.0 / 87178291200.0);
  s = fma(s, z, -1.0 / 39916800.0), c = fma(c, z, 1.0 / 479001600.0);
  s = fma(s, z, 1.0 / 362880.0), c = fma(c, z, -1.0 / 3628800.0);
  s = fma(s, z, -1.0 / 5040.0), c = fma(c, z, 1.0 / 40320.0);
  s = fma(s, z, 1.0 / 120.0), c = fma(c, z, -1.0 / 720.0);
  s = fma(s, z, -1.0 / 6.0), c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  s = fma(s * z, r, r);
  c = fma(c, z, 1.0);
  const long long q = static_cast<long long>(n);
  const double x = (q & 1) ? s : c, y = (q & 1) ? c : s;
  return make_float2(static_cast<float>((q + 1) & 2 ? -x : x), static_cast<float>(q & 2 ? -y : y));
}

// Eight elements as they are in memory.
template <typename T>
struct Chunk;
template <>
struct Chunk<uint16_t> {
  u32x4 a;
  __device__ void load(const uint16_t* p) { a = *reinterpret_cast<const u32x4*>(p); }
  __device__ void store(uint16_t* p) const { *reinterpret_cast<u32x4*>(p) = a; }
  __device__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = ptd::bf16_lo(a[i]), x[2 * i + 1] = ptd::bf16_hi(a[i]);
  }
  __device__ void set(const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = ptd::cvt_pk_bf16(x[2 * i], x[2 * i + 1]);
  }
};
template <>
struct Chunk<float> {
  u32x4 a, b;
  __device__ void load(const float* p) {
    a = *reinterpret_cast<const u32x4*>(p);
    b = *reinterpret_cast<const u32x4*>(p + 4);
  }
  __device__ void store(float* p) const {
    *reinterpret_cast<u32x4*>(p) = a;
    *reinterpret_cast<u32x4*>(p + 4) = b;
  }
  __device__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(a[i]), x[4 + i] = __uint_as_float(b[i]);
  }
  __device__ void set(const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(x[i]), b[i] = __float_as_uint(x[4 + i]);
  }
};

// Sum over aligned groups of G lanes (4 or 8) to each of them.
template <int G>
__device__ __forceinline__ float group_sum(float v) {
  v = ptd::dpp_add<0xB1>(v);                    // quad_perm 1032
  v = ptd::dpp_add<0x4E>(v);                    // quad_perm 2301
  return G == 8 ? ptd::dpp_add<0x141>(v) : v;   // half-row mirror: the other quad
}

// The weights of a lane's elements.
__device__ __forceinline__ void load_weights(const void* w, int bf16, int d0, float (&x)[8]) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 1.f;
  } else if (bf16) {
    Chunk<uint16_t> c;
    c.load(static_cast<const uint16_t*>(w) + d0);
    c.get(x);
  } else {
    Chunk<float> c;
    c.load(static_cast<const float*>(w) + d0);
    c.get(x);
  }
}

// MIXED: heads of queries, keys and values are taken one after the other, and a group of them may hold several
// kinds; else a group is of one kind, which the whole wave then takes one way.
template <typename T, int D, bool INTERLEAVED, bool MIXED>
__global__ void __launch_bounds__(kThreads) k_qk_norm_rope(QkArgs a, int norm) {
  constexpr int G = D / 16;           // lanes of a head
  constexpr int H = PTD_WAVE / G;     // heads of a wave
  __shared__ float2 s_cs[kWaves][kMaxHalf];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long unit = static_cast<long long>(blockIdx.x) * kWaves + wave;
  const long long row = unit / a.waves_per_row;
  if (row >= a.N) return;  // whole wave
  const int sub = static_cast<int>(unit - row * a.waves_per_row);
  const int pos = a.positions ? a.positions[row] : 0;
  if (pos < 0) return;  // a place without a row
  int slot = a.slots ? a.slots[row] : -1;
  if (slot >= 0 && slot / a.page_size >= a.num_pages) {
    if (lane == 0) ptd::report(a.dev_status, PTD_ERR_PAGE);
    slot = -1;
  } else if (slot < -1) {
    if (lane == 0) ptd::report(a.dev_status, PTD_ERR_PAGE);
  }
  const int c = lane % G, hl = lane / G;
  // a lane's two groups of eight elements: one of each half of the turned part, or neighbours
  const int turned = a.rot / 16;  // lanes whose elements are turned
  const bool turn = c < turned;
  const int d0 = 8 * (INTERLEAVED || !turn ? 2 * c : c);
  const int d1 = INTERLEAVED || !turn ? d0 + 8 : d0 + 8 * turned;

  const int hq = a.heads[0], hk = a.heads[1], total = hq + (slot >= 0 ? 2 : 1) * hk;
  const int gq = (hq + H - 1) / H, gk = (hk + H - 1) / H;
  const int groups = MIXED ? (total + H - 1) / H : gq + (slot >= 0 ? 2 : 1) * gk;
  const int page = slot >= 0 ? slot / a.page_size : 0;
  const int at = slot >= 0 ? slot - page * a.page_size : 0;
  struct Head {
    int kind, h;
    bool there;
  };
  auto head_of = [&](int u) __attribute__((always_inline)) {
    if constexpr (MIXED) {
      const int n = u * H + hl, kind = n < hq ? 0 : n < hq + hk ? 1 : 2;
      return Head{kind, n - (kind == 0 ? 0 : kind == 1 ? hq : hq + hk), n < total};
    } else {
      const int kind = u < gq ? 0 : u < gq + gk ? 1 : 2;
      const int h = (u - (kind == 0 ? 0 : kind == 1 ? gq : gq + gk)) * H + hl;
      return Head{kind, h, u < groups && h < (kind == 0 ? hq : hk)};
    }
  };
  Chunk<T> x0, x1, n0, n1;
  auto load = [&](int u) __attribute__((always_inline)) {
    const auto [kind, h, there] = head_of(u);
    if (there) {
      const T* src = static_cast<const T*>(kind == 0 ? a.in[0] : kind == 1 ? a.in[1] : a.in[2]) +
                     row * (kind == 0 ? a.ld_in[0] : kind == 1 ? a.ld_in[1] : a.ld_in[2]) + static_cast<int64_t>(h) * D;
      n0.load(src + d0);
      n1.load(src + d1);
    }
  };
  load(sub);
  float cs[8], sn[8];
  if (a.rot > 0) {
    if (lane < a.rot / 2) s_cs[wave][lane] = cos_sin(static_cast<double>(pos) * a.inv_freq[lane]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 v = s_cs[wave][min(8 * c + e, kMaxHalf - 1)];
      cs[e] = v.x, sn[e] = v.y;
    }
  }
  int have = -1;  // kind whose weights are in w0, w1
  float w0[8], w1[8];
  for (int u = sub; u < groups; u += a.waves_per_row) {
    const auto [kind, h, there] = head_of(u);
    x0 = n0, x1 = n1;
    load(u + a.waves_per_row);
    if (norm && kind < 2 && kind != have) {
      load_weights(kind == 0 ? a.w[0] : a.w[1], a.w_bf16, d0, w0);
      load_weights(kind == 0 ? a.w[0] : a.w[1], a.w_bf16, d1, w1);
      have = kind;
    }
    if (!there) continue;
    if (kind < 2) {
      float x[8], y[8];
      x0.get(x);
      x1.get(y);
      if (norm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum), sum = fmaf(y[e], y[e], sum);
        sum = group_sum<G>(sum);
        const float f = 1.f / sqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * f * w0[e], y[e] = y[e] * f * w1[e];
      }
      if (turn) {
        if constexpr (INTERLEAVED) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = x[2 * e], q = x[2 * e + 1], r = y[2 * e], t = y[2 * e + 1];
            x[2 * e] = p * cs[e] - q * sn[e];
            x[2 * e + 1] = p * sn[e] + q * cs[e];
            y[2 * e] = r * cs[4 + e] - t * sn[4 + e];
            y[2 * e + 1] = r * sn[4 + e] + t * cs[4 + e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float p = x[e], q = y[e];
            x[e] = p * cs[e] - q * sn[e];
            y[e] = p * sn[e] + q * cs[e];
          }
        }
      }
      x0.set(x);
      x1.set(y);
      T* out = static_cast<T*>(kind == 0 ? a.out[0] : a.out[1]);
      if (out) {
        T* dst = out + row * (kind == 0 ? a.ld_out[0] : a.ld_out[1]) + static_cast<int64_t>(h) * D;
        x0.store(dst + d0);
        x1.store(dst + d1);
      }
    }
    if (kind > 0 && slot >= 0) {
      T* dst = static_cast<T*>(kind == 1 ? a.pages[0] : a.pages[1]) +
               ((static_cast<int64_t>(page) * hk + h) * a.page_size + at) * D;
      x0.store(dst + d0);
      x1.store(dst + d1);
    }
  }
}

template <typename T, int D, bool MIXED>
void launch(const QkArgs& a, int norm, bool inter, unsigned grid, hipStream_t st) {
  if (inter) hipLaunchKernelGGL((k_qk_norm_rope<T, D, true, MIXED>), dim3(grid), dim3(kThreads), 0, st, a, norm);
  else hipLaunchKernelGGL((k_qk_norm_rope<T, D, false, MIXED>), dim3(grid), dim3(kThreads), 0, st, a, norm);
}
template <typename T, int D>
void launch(const QkArgs& a, int norm, bool inter, bool mixed, unsigned grid, hipStream_t st) {
  mixed ? launch<T, D, true>(a, norm, inter, grid, st) : launch<T, D, false>(a, norm, inter, grid, st);
}

}  // namespace

extern "C" int ptd_qk_norm_rope(const void* q, const void* k, const void* v, const void* q_weight,
                                const void* k_weight, const int32_t* positions,
                                const int32_t* slots, void* q_out, void* k_out,
                                const ptd_kv_store* store, const ptd_qk_shape* shape,
                                const double* inv_freq, int32_t* dev_status, void* stream) {
  PTD_RETURN_IF(!shape, PTD_ERR_NULL);
  const ptd_qk_shape& s = *shape;
  PTD_RETURN_IF((s.dtype != PTD_BF16 && s.dtype != PTD_F32) || (s.w_dtype != PTD_BF16 && s.w_dtype != PTD_F32),
                PTD_ERR_DTYPE);
  PTD_RETURN_IF(s.N < 0 || s.N > kMaxRows || s.Hq < 0 || s.Hkv < 0 || s.Hq + static_cast<int64_t>(s.Hkv) < 1 || s.Hq > 65535 || s.Hkv > 65535 ||
                    (s.D != 64 && s.D != 128),
                PTD_ERR_SHAPE);
  PTD_RETURN_IF(s.rot_dim < 0 || s.rot_dim > s.D || s.rot_dim % 16 != 0, PTD_ERR_SHAPE);
  PTD_RETURN_IF(s.pairing != PTD_ROPE_HALF && s.pairing != PTD_ROPE_INTERLEAVED, PTD_ERR_SHAPE);
  PTD_RETURN_IF(s.norm != 0 && s.norm != 1, PTD_ERR_SHAPE);
  PTD_RETURN_IF(s.norm && !(s.eps >= 0.0 && s.eps < INFINITY), PTD_ERR_SHAPE);
  PTD_RETURN_IF(!s.norm && (q_weight || k_weight), PTD_ERR_SHAPE);
  PTD_RETURN_IF(s.rot_dim > 0 && !inv_freq && !(s.theta > 0.0 && s.theta < INFINITY), PTD_ERR_SHAPE);
  PTD_RETURN_IF(store && (!store->k_pages || !store->v_pages), PTD_ERR_NULL);
  PTD_RETURN_IF(store && (store->page_size < 1 || store->num_pages < 1 || s.Hkv < 1 ||
                          static_cast<int64_t>(store->page_size) * store->num_pages > 0x7FFFFFFFLL),
                PTD_ERR_SHAPE);
  QkArgs a = {};
  const int64_t dense[3] = {static_cast<int64_t>(s.Hq) * s.D, static_cast<int64_t>(s.Hkv) * s.D, static_cast<int64_t>(s.Hkv) * s.D};
  const int64_t ld[3] = {s.ldq ? s.ldq : dense[0], s.ldk ? s.ldk : dense[1], s.ldv ? s.ldv : dense[2]};
  const int64_t ldo[2] = {s.ldqo ? s.ldqo : dense[0], s.ldko ? s.ldko : dense[1]};
  const int per16 = s.dtype == PTD_F32 ? 4 : 8;
  for (int i = 0; i < 3; ++i) {
    PTD_RETURN_IF(ld[i] < dense[i], PTD_ERR_SHAPE);
    PTD_RETURN_IF(i < 2 && ldo[i] < dense[i], PTD_ERR_SHAPE);
    PTD_RETURN_IF(ld[i] % per16 != 0 || (i < 2 && ldo[i] % per16 != 0), PTD_ERR_ALIGN);
    a.ld_in[i] = ld[i];
    if (i < 2) a.ld_out[i] = ldo[i];
  }
  // theta^(-2p / rot) as products in 64 bits of mantissa: within a step of the double (64 calls of
  // pow take 2 us)
  const long double ratio = s.rot_dim > 0 && !inv_freq ? powl(s.theta, -2.0L / s.rot_dim) : 1.0L;
  long double f = 1.0L;
  for (int p = 0; p < s.rot_dim / 2; ++p, f *= ratio) {
    a.inv_freq[p] = inv_freq ? inv_freq[p] : static_cast<double>(f);
    PTD_RETURN_IF(!(fabs(a.inv_freq[p]) <= 0x1p20), PTD_ERR_SHAPE);
  }
  if (s.N == 0) return PTD_OK;
  PTD_RETURN_IF((s.Hq && (!q || !q_out)) || (s.Hkv && (!k || (!k_out && !store))), PTD_ERR_NULL);
  PTD_RETURN_IF((s.rot_dim > 0 && !positions) || (store && (!v || !slots)), PTD_ERR_NULL);
  const void* p16[] = {q, k, v, q_weight, k_weight, q_out, k_out, store ? store->k_pages : nullptr, store ? store->v_pages : nullptr};
  for (const void* p : p16) PTD_RETURN_IF(!ptd_aligned(p, 16), PTD_ERR_ALIGN);
  a.in[0] = q, a.in[1] = k, a.in[2] = v;
  a.out[0] = q_out, a.out[1] = k_out;
  a.w[0] = q_weight, a.w[1] = k_weight;
  a.positions = positions;
  a.dev_status = dev_status;
  a.heads[0] = s.Hq, a.heads[1] = s.Hkv;
  a.N = s.N, a.rot = s.rot_dim, a.w_bf16 = s.w_dtype == PTD_BF16;
  a.eps = static_cast<float>(s.eps);
  a.page_size = 1;
  if (store) {
    a.slots = slots;
    a.pages[0] = store->k_pages, a.pages[1] = store->v_pages;
    a.page_size = store->page_size, a.num_pages = store->num_pages;
  }
  // A row's head groups over several waves while there are fewer than half of what the chip
  // holds.  (32/8 heads x 128, into pages: 1024 rows 10.2 us with a wave per row, 7.9 with four; 2048
  // rows 12.8 with four, 10.9 with two; 28000 rows 121 with one and 146 with six.)
  const int per = s.D == 128 ? 8 : 16, kinds = store ? 2 : 1;
  // Groups of several kinds where that makes fewer of them.  (70184 rows of 7/1 heads x 64 into pages, one
  // group in place of three: 73 us and 97; 28700 rows of 32/8 x 128, as many groups: 122 and 119)
  const int apart = ptd_cdiv(s.Hq, per) + kinds * ptd_cdiv(s.Hkv, per), together = ptd_cdiv(s.Hq + kinds * s.Hkv, per);
  const bool mixed = together < apart;
  const int groups = mixed ? together : apart;
  a.waves_per_row = std::max(1, std::min(groups, 4096 / s.N));
  const int64_t grid = (static_cast<int64_t>(s.N) * a.waves_per_row + kWaves - 1) / kWaves;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool il = s.pairing == PTD_ROPE_INTERLEAVED;
  const unsigned g = static_cast<unsigned>(grid);
  if (s.dtype == PTD_BF16) s.D == 128 ? launch<uint16_t, 128>(a, s.norm, il, mixed, g, st) : launch<uint16_t, 64>(a, s.norm, il, mixed, g, st);
  else s.D == 128 ? launch<float, 128>(a, s.norm, il, mixed, g, st) : launch<float, 64>(a, s.norm, il, mixed, g, st);
  return ptd_launch_status();
}
