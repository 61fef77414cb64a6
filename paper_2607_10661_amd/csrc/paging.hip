// Pages of the key/value caches: page tables and slot maps from the sequences'
// lengths (ptd_page_init, ptd_page_plan), and rows into 8-bit pages with block
// scales (ptd_kv_write_fp8blk).
#include <algorithm>

#include "ptd_common.hpp"

namespace {

// ===========================================================================
// page tables and slot maps
// ===========================================================================
struct PlanParams {
  ptd_page_state s;
  const int32_t* kv_len;
  const int32_t* new_len;
  int32_t* row_start;
  int32_t* slots;
  int32_t* positions;
  int32_t* dev_status;
  int N, rows_per_seq, page_shift;
};

// Rows whose slots the planning workgroup writes itself; more take a launch of
// their own, over the whole chip.  (A plan and its release, 16 sequences: of 1024 rows 10.1 us
// and with a launch 13.1, of 2048 12.2 and 13.3, of 4096 16.7 and 13.1.)
constexpr int kPlanRows = 2048;
constexpr int kPlanSmall = 256, kPlanLarge = 1024;  // threads
// Pages of the new rows from which on the planning workgroup is a large one.  (A plan and
// the release of its pages by a call without rows, both with 256 threads and with 1024: of 32
// pages 12.2 and 12.5 us, of 1024 13.5 and 15.0, of 2048 16.9 and 16.0, of 8192 39.2 and
// 22.0.)  A call without rows (N = 0) is a small one whatever it gives back, which the host
// does not know: it follows every step, where it moves a page or two per sequence, up to 1.2 us
// shorter than with 1024 threads.  Finished sequences give back about 1500 pages in equal
// time, 4063 in 4 us more, 6897 in 12, 16384 in 25.
constexpr int kPlanPages = 1536;

// A sequence's lengths and pages, checked.  rows: new rows (0 where refused).
struct Want {
  int kv, rows, held, need;
};
__device__ inline Want want_of(const PlanParams& p, int b, int32_t* report_to) {
  Want w;
  w.kv = p.kv_len[b];
  w.rows = p.new_len[b];
  w.held = p.s.num_held[b];
  const long long cap = static_cast<long long>(p.s.max_pages) << p.page_shift;
  const bool bad_len = w.kv < 0 || w.rows < 0 || static_cast<long long>(w.kv) + w.rows > cap;
  const bool bad_held = w.held < 0 || w.held > p.s.max_pages;
  if (bad_len) ptd::report(report_to, PTD_ERR_KV_LEN);
  if (bad_held) ptd::report(report_to, PTD_ERR_PAGE);
  if (bad_len || bad_held) {
    w.rows = 0;
    w.held = bad_held ? 0 : w.held;
    w.need = w.held;
  } else {
    // (the sum fits an int: it is at most cap < 2^31)
    w.need = static_cast<int>((static_cast<unsigned>(w.kv + w.rows) + (1u << p.page_shift) - 1u) >> p.page_shift);
  }
  return w;
}

// Exclusive sums of three values over the workgroup; totals to every thread.
struct Sums {
  long long back, grow, rows;
};
template <int NT>
__device__ __forceinline__ Sums block_scan(const Sums& v, Sums* lds, Sums* total) {
  const int wave = threadIdx.x >> 6;
  const Sums in = {ptd::wave_scan_i64(v.back), ptd::wave_scan_i64(v.grow), ptd::wave_scan_i64(v.rows)};
  __syncthreads();  // lds of the call before is read
  if ((threadIdx.x & 63) == 63) lds[wave] = in;
  __syncthreads();
  Sums base = {0, 0, 0}, all = {0, 0, 0};
#pragma unroll
  for (int w = 0; w < NT / PTD_WAVE; ++w) {
    const Sums x = lds[w];
    if (w < wave) base.back += x.back, base.grow += x.grow, base.rows += x.rows;
    all.back += x.back, all.grow += x.grow, all.rows += x.rows;
  }
  *total = all;
  return {base.back + in.back - v.back, base.grow + in.grow - v.grow, base.rows + in.rows - v.rows};
}

// Last index x of [0, n) with a[x] <= v (a ascending, a[0] <= v).
template <typename A>
__device__ __forceinline__ int upper(const A& a, int n, long long v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Slot and position of row i, row r of sequence b.
__device__ __forceinline__ void put_row(const PlanParams& p, int i, int slot, int pos) {
  p.slots[i] = slot;
  if (p.positions) p.positions[i] = pos;
}
__device__ __forceinline__ int slot_at(const PlanParams& p, int id, int pos) {
  if (static_cast<uint32_t>(id) < static_cast<uint32_t>(p.s.num_pages))
    return (id << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
  ptd::report(p.dev_status, PTD_ERR_PAGE);
  return -1;
}
__device__ __forceinline__ const int32_t* table_of(const PlanParams& p, int b) {
  return p.s.page_table + static_cast<size_t>(b) * p.s.max_pages;
}

// Rows [i0, i1) by `step` when the tables are written.  starts: of packed rows, in LDS
// where they fit, else in memory.  (Rows and pages are counted without a sign: up to 2^31
// of either, a step past the last one does not wrap.)
template <typename Starts>
__device__ __forceinline__ void put_rows(const PlanParams& p, const Starts& starts, int i0, int i1, int step) {
  for (uint32_t u = i0; u < static_cast<uint32_t>(i1); u += step) {
    const int i = static_cast<int>(u);
    int b, r;
    if (p.rows_per_seq > 0) {
      b = i / p.rows_per_seq;
      r = i - b * p.rows_per_seq;
    } else {
      b = upper(starts, p.s.B, i);  // (the last of sequences that start at one place has the rows)
      r = i - starts[b];
    }
    const Want w = want_of(p, b, nullptr);
    const bool row = r < w.rows;
    const int pos = w.kv + r;
    const bool page = row && (pos >> p.page_shift) < w.held;
    put_row(p, i, page ? slot_at(p, table_of(p, b)[pos >> p.page_shift], pos) : -1, row ? pos : -1);
  }
}

// One workgroup: a thread per sequence (in rounds of the workgroup's size) counts pages, sums over
// the workgroup give every sequence its places on the free list and in the rows,
// then a thread per page moves ids.  Outputs depend on nothing but the inputs: no
// atomics.  Bound by latency (5 us for 16 sequences and 1024 rows, 8 for 64 prompts
// and 4200 pages): with ONE round of sequences, the lengths are loaded
// once, new rows take their page ids from where the tables get them, and a step of 16
// sequences waits three times for memory: lengths, ids, stores.
template <bool ONE, int NT>
__global__ void __launch_bounds__(NT) k_page_plan(PlanParams p) {
  __shared__ Sums s_scan[NT / PTD_WAVE];
  __shared__ int s_back[NT], s_need[NT], s_off[NT], s_grow[NT];
  __shared__ int s_held[NT], s_start[NT], s_kv[NT], s_rows[NT];
  const int tid = threadIdx.x;
  const int B = p.s.B;
  const Want none = {0, 0, 0, 0};
  Want w = none;
  if (ONE && tid < B) w = want_of(p, tid, p.dev_status);
  int count = p.s.num_free[0];
  if (count < 0 || count > p.s.num_pages) {  // uniform
    if (tid == 0) ptd::report(p.dev_status, PTD_ERR_PAGE);
    count = min(max(count, 0), p.s.num_pages);
  }
  auto sums_of = [](const Want& x) __attribute__((always_inline)) {
    return Sums{max(x.held - x.need, 0), max(x.need - x.held, 0), x.rows};
  };
  // ---- pages that go back: their number first, as the first sequence's lie deepest
  Sums at = {0, 0, 0}, all = {0, 0, 0};
  if (ONE) {
    at = block_scan<NT>(sums_of(w), s_scan, &all);
  } else {
    for (int b0 = 0; b0 < B; b0 += NT) {
      Sums t;
      block_scan<NT>(sums_of(b0 + tid < B ? want_of(p, b0 + tid, nullptr) : none), s_scan, &t);
      all.back += t.back;
    }
  }
  long long total = all.back;
  if (total > p.s.num_pages - count) {  // pages held twice: the list cannot take them
    if (tid == 0) ptd::report(p.dev_status, PTD_ERR_PAGE);
    total = p.s.num_pages - count;
  }
  const int count1 = count + static_cast<int>(total);
  long long done = 0;
  for (int b0 = 0; b0 < B && total > 0; b0 += NT) {  // uniform
    Sums t = all;
    if (!ONE) {
      w = b0 + tid < B ? want_of(p, b0 + tid, nullptr) : none;
      at = block_scan<NT>(sums_of(w), s_scan, &t);
    }
    s_back[tid] = static_cast<int>(min(at.back, static_cast<long long>(0x7FFFFFFF)));
    s_need[tid] = w.need;
    __syncthreads();
    const int n = min(B - b0, NT);
    const long long back = min(t.back, total);  // (held pages that make up more are not all moved)
#pragma unroll 4
    for (uint32_t u = tid; u < back; u += NT) {
      const int j = static_cast<int>(u);
      const int x = upper(s_back, n, j);
      const long long to = count1 - 1 - (done + j);
      if (to >= count) p.s.free_pages[to] = table_of(p, b0 + x)[s_need[x] + (j - s_back[x])];
    }
    done += t.back;
    __syncthreads();
  }
  // ---- pages that are taken, in order while the list lasts; starts of the rows
  long long taken = 0, rows = 0;
  bool short_of = false;
  for (int b0 = 0; b0 < B; b0 += NT) {
    const bool live = b0 + tid < B;
    Sums t = all;
    if (!ONE) {
      w = live ? want_of(p, b0 + tid, p.dev_status) : none;
      at = block_scan<NT>(sums_of(w), s_scan, &t);
    }
    if (p.rows_per_seq > 0 && w.rows > p.rows_per_seq) ptd::report(p.dev_status, PTD_ERR_ROWS);
    const int grow = max(w.need - w.held, 0);
    const bool ok = grow == 0 || taken + at.grow + grow <= count1;
    if (!ok) ptd::report(p.dev_status, PTD_ERR_NO_PAGES);
    const int now = ok ? w.need : w.held;
    s_off[tid] = static_cast<int>(min(at.grow, static_cast<long long>(p.s.num_pages)));
    s_grow[tid] = ok ? grow : 0;
    s_held[tid] = w.held;
    if (p.rows_per_seq == 0) {
      const int start = static_cast<int>(min(rows + at.rows, static_cast<long long>(0x7FFFFFFF)));
      if (live) p.row_start[b0 + tid] = start;
      s_start[tid] = start;
    }
    if (ONE) {
      s_kv[tid] = w.kv;
      s_rows[tid] = w.rows;
      s_need[tid] = now;
    }
    // sequences after the first that was refused take none
    const bool any_bad = __syncthreads_or(!ok);
    const int n = min(B - b0, NT);
    const long long room = min(t.grow, static_cast<long long>(count1) - taken);
#pragma unroll 4
    for (uint32_t u = tid; u < room; u += NT) {
      const int j = static_cast<int>(u);
      const int x = upper(s_off, n, j);
      const int k = j - s_off[x];
      if (k < s_grow[x])
        p.s.page_table[static_cast<size_t>(b0 + x) * p.s.max_pages + s_held[x] + k] =
            p.s.free_pages[count1 - 1 - (taken + j)];
    }
    // (a sequence refused above keeps num_held as it is, whatever it says)
    if (live && now != w.held) p.s.num_held[b0 + tid] = now;
    if (any_bad && !short_of) {
      // (at most num_pages, as they were taken)
      const int used = ptd::wave_max_i32(ok && grow > 0 ? static_cast<int>(at.grow) + grow : 0);
      __syncthreads();
      if ((tid & 63) == 0) s_scan[tid >> 6].grow = used;
      __syncthreads();
      long long mx = 0;
      for (int x = 0; x < NT / PTD_WAVE; ++x) mx = max(mx, s_scan[x].grow);
      if (tid == 0) p.s.num_free[0] = count1 - static_cast<int>(taken + mx);
      short_of = true;
    }
    taken += t.grow;
    rows += t.rows;
    if (!ONE) __syncthreads();
  }
  if (tid == 0) {
    if (!short_of) p.s.num_free[0] = count1 - static_cast<int>(taken);
    if (p.rows_per_seq == 0) {
      p.row_start[B] = static_cast<int>(min(rows, static_cast<long long>(0x7FFFFFFF)));
      if (rows > p.N) ptd::report(p.dev_status, PTD_ERR_ROWS);
    }
  }
  if (p.N > kPlanRows) return;
  if (ONE) {
    // ids of pages that were held come from the table, of new ones from the free list
#pragma unroll 4
    for (int i = tid; i < p.N; i += NT) {
      int b, r;
      if (p.rows_per_seq > 0) {
        b = i / p.rows_per_seq;
        r = i - b * p.rows_per_seq;
      } else {
        b = upper(s_start, B, i);
        r = i - s_start[b];
      }
      const bool row = r < s_rows[b];
      const int pos = s_kv[b] + r;
      const int pg = pos >> p.page_shift;
      const bool page = row && pg < s_need[b];
      const int32_t* from = pg < s_held[b] ? table_of(p, b) + pg : p.s.free_pages + (count1 - 1 - (s_off[b] + pg - s_held[b]));
      put_row(p, i, page ? slot_at(p, *from, pos) : -1, row ? pos : -1);
    }
  } else {
    __syncthreads();
    put_rows(p, p.row_start, tid, p.N, NT);
  }
}

constexpr int kSlotThreads = 256;
constexpr int kSlotRows = kSlotThreads;  // rows per workgroup

__global__ void __launch_bounds__(kSlotThreads) k_page_slots(PlanParams p) {
  __shared__ int s_start[kPlanLarge];
  const int i0 = blockIdx.x * kSlotRows + threadIdx.x;
  const int i1 = static_cast<int>(min(static_cast<long long>(p.N), (blockIdx.x + 1LL) * kSlotRows));
  if (p.rows_per_seq == 0 && p.s.B <= kPlanLarge) {
    for (int x = threadIdx.x; x < p.s.B; x += kSlotThreads) s_start[x] = p.row_start[x];
    __syncthreads();
    put_rows(p, s_start, i0, i1, kSlotThreads);
  } else {
    put_rows(p, p.row_start, i0, i1, kSlotThreads);
  }
}

__global__ void __launch_bounds__(256) k_page_init(ptd_page_state s) {
  const long long n = static_cast<long long>(s.B) * s.max_pages;
  const long long step = static_cast<long long>(gridDim.x) * 256;
  const long long first = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  for (long long i = first; i < n; i += step) s.page_table[i] = -1;
  for (long long i = first; i < s.num_pages; i += step) s.free_pages[i] = s.num_pages - 1 - static_cast<int>(i);
  for (long long i = first; i < s.B; i += step) s.num_held[i] = 0;
  if (first == 0) s.num_free[0] = s.num_pages;
}

int check_state(const ptd_page_state* s, int* shift) {
  PTD_RETURN_IF(!s || !s->page_table || !s->num_held || !s->free_pages || !s->num_free, PTD_ERR_NULL);
  const int ps = s->page_size;
  PTD_RETURN_IF(ps < 1 || ps > (1 << 20) || (ps & (ps - 1)) != 0, PTD_ERR_SHAPE);
  PTD_RETURN_IF(s->B < 1 || s->B > 65536 || s->max_pages < 1 || s->num_pages < 1, PTD_ERR_SHAPE);
  PTD_RETURN_IF(static_cast<long long>(s->max_pages) * ps > 0x7FFFFFFFLL ||
                    static_cast<long long>(s->num_pages) * ps > 0x7FFFFFFFLL,
                PTD_ERR_SHAPE);
  int sh = 0;
  while ((1 << sh) < ps) ++sh;
  *shift = sh;
  return PTD_OK;
}

// ===========================================================================
// rows into 8-bit pages
// ===========================================================================
struct WriteParams {
  const void* src[2];      // keys, values
  int64_t ld[2];           // elements
  uint8_t* pages[2];
  uint8_t* scales;
  const int32_t* slots;
  const int32_t* from;     // source rows within a sequence, or null
  int32_t* dev_status;
  int N, rows_per_seq, Hkv, chunk, page_shift, scale_shift;
  long long slot_end;      // num_pages * page_size
};

constexpr int kWriteThreads = 256;
constexpr int kHeadDim = 128;
constexpr int kExpMin = -117, kExpMax = 119;  // of the scales

// Eight elements of a row as they are loaded.  top(): largest magnitude's bits of
// each half or word, ordered as integers; at(j): element j.
template <typename T>
struct Row8;
template <>
struct Row8<uint16_t> {
  uint32_t w[4];
  __device__ void load(const uint16_t* s) {
    const uint4 v = *reinterpret_cast<const uint4*>(s);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  }
  // (the compiler would keep the floats of one use for the next: twice the registers)
  __device__ void forget() { asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3])); }
  __device__ float at(int j) const { return (j & 1) ? ptd::bf16_hi(w[j >> 1]) : ptd::bf16_lo(w[j >> 1]); }
  __device__ uint32_t top() const {
    using u16x2 = unsigned short __attribute__((ext_vector_type(2)));
    u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7FFF7FFFu);
#pragma unroll
    for (int j = 1; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[j] & 0x7FFF7FFFu));
    const uint32_t r = __builtin_bit_cast(uint32_t, m);
    return max(r << 16, r & 0xFFFF0000u);
  }
};
template <>
struct Row8<float> {
  uint32_t w[8];
  __device__ void load(const float* s) {
    const uint4 a = *reinterpret_cast<const uint4*>(s), b = *reinterpret_cast<const uint4*>(s + 4);
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  }
  __device__ void forget() {
    asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]), "+v"(w[4]), "+v"(w[5]), "+v"(w[6]), "+v"(w[7]));
  }
  __device__ float at(int j) const { return __uint_as_float(w[j]); }
  __device__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, w[j] & 0x7FFFFFFFu);
    return m;
  }
};

constexpr uint32_t kInfBits = 0x7F800000u;

// Eight E4M3 codes of x * 2^e, nearest even (v_cvt_pk_fp8_f32: OCP on gfx950).  x *
// 2^e is exact or far below the least code; 448 is the largest.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true));
}
__device__ __forceinline__ float to_range(float x, float f) {
  const float y = x * f;
  return __builtin_amdgcn_fmed3f(y != y ? 0.f : y, -448.f, 448.f);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// One wave per (block of S rows, head, keys or values): 16 lanes hold a row of 128
// elements, eight each; a lane's S / 4 loads are all in flight before the first is
// used, and the largest magnitude is the only thing that passes between lanes.
//
// The block's scale is 2^e, e least with amax <= 448 * 2^e: with amax = m * 2^x, 1 <=
// m < 2, that is x - 8, or x - 7 where m > 1.75.  A power of two leaves the
// codes' three mantissa bits untouched, so a live row is coded anew without
// loss while it stays a normal number of the format.
// Bound by HBM where the rows are many: prompts of 28000 rows in all, 8 heads, S = 64, 177 MB, take
// 40 us, 4.4 TB/s (a large copy reaches 5.2); by latency at a step: slots, rows, scale,
// codes one after the other, 7 us for 16 trees of 64 rows.
template <typename T, int S, bool FROM>
__global__ void __launch_bounds__(kWriteThreads, 2) k_kv_write(WriteParams p) {
  constexpr int R = S / 4;  // rows per lane
  // registers hold the block's rows (up to 64 registers of them), or 32 rows at a
  // time that the second pass reads again: beyond, waves per SIMD are worth more than one
  // reading.  (8192 rows: 64 rows of bf16 held 12.3 us and not 13.9, 32 rows of fp32 17.1 and
  // 20.4; 64 rows of fp32 43 and 28, 128 rows of bf16 29 and 16.)
  constexpr bool HOLD = R * sizeof(T) * 2 <= 64;
  constexpr int RH = HOLD ? R : 8;
  constexpr int RO = R <= 16 ? R : 8;  // the same for the codes of live rows
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kind = wave & 1;
  // (head pairs run fastest: workgroups in flight together read whole rows of all heads, and
  // not the same few memory channels)
  const int pairs = (p.Hkv + 1) / 2;
  const uint32_t id = blockIdx.x + gridDim.x * blockIdx.y;
  const int part = static_cast<int>(id / pairs);
  const int g = static_cast<int>(id % pairs) * 2 + (wave >> 1);
  if (g >= p.Hkv) return;
  const int sub = lane >> 4, d8 = (lane & 15) * 8;
  const T* src = static_cast<const T*>(p.src[kind]) + static_cast<size_t>(g) * kHeadDim + d8;
  const int64_t ld = p.ld[kind];
  const int end = static_cast<int>(min(static_cast<long long>(p.N), (part + 1LL) * p.chunk));
  // slot of row i, or -1 (off the rows, not to be written, outside the pages)
  auto slot_of = [&](int i) __attribute__((always_inline)) {
    int s = i >= 0 && i < p.N ? p.slots[i] : -1;
    if (s < -1 || s >= p.slot_end) {
      ptd::report(p.dev_status, PTD_ERR_PAGE);
      s = -1;
    }
    return s;
  };
  for (int i = static_cast<int>(min(static_cast<long long>(p.N), static_cast<long long>(part) * p.chunk)); i < end;) {
    // next row of the chunk that opens a block: one whose row before it is not in
    // the same block
    const int cur = slot_of(i + lane), prev = slot_of(i + lane - 1);
    const bool same = cur >= 0 && prev >= 0 && (cur >> p.scale_shift) == (prev >> p.scale_shift);
    if (same && cur != prev + 1) ptd::report(p.dev_status, PTD_ERR_ROWS);
    const uint64_t heads = __ballot(cur >= 0 && !same && i + lane < end);
    if (heads == 0) {
      i += PTD_WAVE;
      continue;
    }
    const int first = __builtin_ctzll(heads);
    i += first;
    const int slot0 = __builtin_amdgcn_readlane(cur, first);
    const int off0 = slot0 & (S - 1);
    // the run: rows whose slots go on by one inside the block, in this window or the next ones
    const uint64_t goes_on = __ballot(same && cur == prev + 1) >> first >> 1;
    int n = 1 + __builtin_ctzll(~goes_on);
    if (first + n == PTD_WAVE) {
      for (int j = n; j < S - off0; j += PTD_WAVE) {  // uniform
        const uint64_t m = ~__ballot(j + lane < S - off0 && slot_of(i + j + lane) == slot0 + j + lane);
        n += m ? __builtin_ctzll(m) : PTD_WAVE;
        if (m) break;
      }
    }
    const size_t block = (((static_cast<size_t>(slot0) >> p.page_shift) * p.Hkv + g) << (p.page_shift - p.scale_shift)) +
                         ((slot0 & ((1 << p.page_shift) - 1)) >> p.scale_shift);
    uint8_t* page = p.pages[kind] + block * (S * kHeadDim) + d8;
    uint8_t* scale = p.scales + block * 2 + kind;
    Row8<T> x[RH];
    uint2 old[RO];  // codes of the live rows
    int e_old = 0;
    auto is_new = [&](int r) __attribute__((always_inline)) { return r >= off0 && r < off0 + n; };
    // source row of the run's row j, in lane j % 64 of word j / 64
    int source[(S + 63) / 64];
    if constexpr (FROM) {
#pragma unroll
      for (int h = 0; h < (S + 63) / 64; ++h) {
        const int row = i + min(h * 64 + lane, n - 1);
        const int f = p.from[row];
        if (f < 0 || f >= p.rows_per_seq) ptd::report(p.dev_status, PTD_ERR_ROWS);
        source[h] = row / p.rows_per_seq * p.rows_per_seq + min(max(f, 0), p.rows_per_seq - 1);
      }
    }
    // (rows outside the run stand for its first or last one: another look at the same
    // elements changes no maximum, and a load without a condition no register)
    auto load = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < RH; ++t) {
        const int j = min(max(4 * (t0 + t) + sub - off0, 0), n - 1);
        int row = i + j;
        if constexpr (FROM) {
          row = __shfl(source[0], j & 63, PTD_WAVE);
          if constexpr (S > 64) {
            const int far = __shfl(source[1], j & 63, PTD_WAVE);
            row = j < 64 ? row : far;
          }
        }
        x[t].load(src + row * ld);
      }
    };
    auto load_old = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < RO; ++t)
        old[t] = *reinterpret_cast<const uint2*>(page + min(4 * (t0 + t) + sub, off0 - 1) * kHeadDim);
    };
    // ---- largest magnitude
    uint32_t top = 0;
    bool odd = false;  // something not finite
    for (int t0 = 0; t0 < R; t0 += RH) {
      load(t0);
      if (t0 == 0 && off0 > 0) {  // uniform: all of the block's loads in flight together
        e_old = *scale;
        load_old(0);
      }
      uint32_t m = 0;
#pragma unroll
      for (int t = 0; t < RH; ++t) m = max(m, x[t].top());
      if (__any(m >= kInfBits)) {  // rare: the finite elements only
        odd |= m >= kInfBits;
        m = 0;
#pragma unroll
        for (int t = 0; t < RH; ++t)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t u = __float_as_uint(x[t].at(j)) & 0x7FFFFFFFu;
            m = max(m, u >= kInfBits ? 0u : u);
          }
      }
      top = max(top, m);
    }
    if (odd) ptd::report(p.dev_status, PTD_ERR_VALUE);
    if (off0 > 0) {
      e_old = __builtin_amdgcn_readfirstlane(e_old) - 127;
      uint32_t code = 0;
      for (int t0 = 0; t0 < R && 4 * t0 < off0; t0 += RO) {  // uniform
        if (t0 > 0) load_old(t0);
#pragma unroll
        for (int t = 0; t < RO; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j) code = max(code, max((old[t].x >> (8 * j)) & 0x7Fu, (old[t].y >> (8 * j)) & 0x7Fu));
      }
      // its value, times the scale it was coded with (both in normal range)
      const float v = __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(min(code, 0x7Eu)), 0) * pow2(min(max(e_old, -126), kExpMax));
      top = max(top, __float_as_uint(v));
    }
    top = static_cast<uint32_t>(ptd::wave_max_i32(static_cast<int>(top)));
    int e = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    e = top == 0 ? 0 : min(max(e, kExpMin), kExpMax);
    // ---- codes
    const float f = pow2(-e);
    for (int t0 = 0; t0 < R; t0 += RH) {
      if constexpr (!HOLD) load(t0);
#pragma unroll
      for (int t = 0; t < RH; ++t) {
        const int r = 4 * (t0 + t) + sub;
        x[t].forget();
        if (is_new(r)) {
          float y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = to_range(x[t].at(j), f);
          *reinterpret_cast<uint2*>(page + r * kHeadDim) = make_uint2(codes4(y[0], y[1], y[2], y[3]), codes4(y[4], y[5], y[6], y[7]));
        }
      }
    }
    if (off0 > 0 && e != e_old) {  // uniform
      const float fo = pow2(min(max(e_old - e, -126), 127));
      for (int t0 = 0; t0 < R && 4 * t0 < off0; t0 += RO) {  // uniform
        if (RO < R) load_old(t0);
#pragma unroll
        for (int t = 0; t < RO; ++t) {
          const int r = 4 * (t0 + t) + sub;
          asm volatile("" : "+v"(old[t].x), "+v"(old[t].y));  // (as forget())
          if (r < off0) {
            float y[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int w = static_cast<int>(h ? old[t].y : old[t].x);
              y[4 * h + 0] = __builtin_amdgcn_cvt_f32_fp8(w, 0);
              y[4 * h + 1] = __builtin_amdgcn_cvt_f32_fp8(w, 1);
              y[4 * h + 2] = __builtin_amdgcn_cvt_f32_fp8(w, 2);
              y[4 * h + 3] = __builtin_amdgcn_cvt_f32_fp8(w, 3);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = to_range(y[j], fo);
            *reinterpret_cast<uint2*>(page + r * kHeadDim) =
                make_uint2(codes4(y[0], y[1], y[2], y[3]), codes4(y[4], y[5], y[6], y[7]));
          }
        }
      }
    }
    if (lane == 0) *scale = static_cast<uint8_t>(e + 127);
    i += n;
  }
}

template <typename T, bool FROM>
void launch_write(const WriteParams& prm, int scale_rows, dim3 grid, hipStream_t st) {
  if (scale_rows == 32) hipLaunchKernelGGL((k_kv_write<T, 32, FROM>), grid, dim3(kWriteThreads), 0, st, prm);
  else if (scale_rows == 64) hipLaunchKernelGGL((k_kv_write<T, 64, FROM>), grid, dim3(kWriteThreads), 0, st, prm);
  else hipLaunchKernelGGL((k_kv_write<T, 128, FROM>), grid, dim3(kWriteThreads), 0, st, prm);
}

}  // namespace

extern "C" int ptd_page_init(const ptd_page_state* state, void* stream) {
  int shift = 0;
  const int rc = check_state(state, &shift);
  if (rc != PTD_OK) return rc;
  const long long n = std::max(static_cast<long long>(state->B) * state->max_pages,
                               static_cast<long long>(state->num_pages));
  const unsigned grid = static_cast<unsigned>(std::min<long long>((n + 255) / 256, 2048));
  hipLaunchKernelGGL(k_page_init, dim3(grid), dim3(256), 0, static_cast<hipStream_t>(stream), *state);
  return ptd_launch_status();
}

extern "C" int ptd_page_plan(const ptd_page_state* state, const int32_t* kv_len,
                             const int32_t* new_len, int32_t N, int32_t rows_per_seq,
                             int32_t* row_start, int32_t* slots, int32_t* positions,
                             int32_t* dev_status, void* stream) {
  PlanParams prm;
  const int rc = check_state(state, &prm.page_shift);
  if (rc != PTD_OK) return rc;
  PTD_RETURN_IF(!kv_len || !new_len || (N > 0 && !slots) || (rows_per_seq == 0 && !row_start), PTD_ERR_NULL);
  PTD_RETURN_IF(N < 0 || rows_per_seq < 0, PTD_ERR_SHAPE);
  PTD_RETURN_IF(rows_per_seq > 0 && static_cast<long long>(state->B) * rows_per_seq != N, PTD_ERR_SHAPE);
  prm.s = *state;
  prm.kv_len = kv_len;
  prm.new_len = new_len;
  prm.row_start = row_start;
  prm.slots = slots;
  prm.positions = positions;
  prm.dev_status = dev_status;
  prm.N = N;
  prm.rows_per_seq = rows_per_seq;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool large = (N >> prm.page_shift) > kPlanPages || state->B > kPlanSmall;
  if (!large) hipLaunchKernelGGL((k_page_plan<true, kPlanSmall>), dim3(1), dim3(kPlanSmall), 0, st, prm);
  else if (state->B <= kPlanLarge) hipLaunchKernelGGL((k_page_plan<true, kPlanLarge>), dim3(1), dim3(kPlanLarge), 0, st, prm);
  else hipLaunchKernelGGL((k_page_plan<false, kPlanLarge>), dim3(1), dim3(kPlanLarge), 0, st, prm);
  if (N > kPlanRows) {
    const unsigned grid = static_cast<unsigned>((static_cast<long long>(N) + kSlotRows - 1) / kSlotRows);
    hipLaunchKernelGGL(k_page_slots, dim3(grid), dim3(kSlotThreads), 0, st, prm);
  }
  return ptd_launch_status();
}

extern "C" int ptd_kv_write_fp8blk(const void* k, const void* v, ptd_dtype dtype, int64_t ldk,
                                   int64_t ldv, int32_t N, const int32_t* slots,
                                   const int32_t* src, int32_t rows_per_seq,
                                   const ptd_kv_pages_fp8blk* kv, int32_t Hkv, int32_t D,
                                   int32_t* dev_status, void* stream) {
  PTD_RETURN_IF(!kv || !kv->k_pages || !kv->v_pages || !kv->scales, PTD_ERR_NULL);
  PTD_RETURN_IF(N > 0 && (!k || !v || !slots), PTD_ERR_NULL);
  PTD_RETURN_IF(dtype != PTD_F32 && dtype != PTD_BF16, PTD_ERR_DTYPE);
  const int ps = kv->page_size, sr = kv->scale_rows;
  PTD_RETURN_IF(ps < 32 || ps > (1 << 20) || (ps & (ps - 1)) != 0 || kv->num_pages < 1, PTD_ERR_SHAPE);
  PTD_RETURN_IF((sr != 32 && sr != 64 && sr != 128) || sr > ps, PTD_ERR_SHAPE);
  PTD_RETURN_IF(static_cast<long long>(kv->num_pages) * ps > 0x7FFFFFFFLL, PTD_ERR_SHAPE);
  PTD_RETURN_IF(N < 0 || Hkv < 1 || Hkv > 65535 || D != kHeadDim, PTD_ERR_SHAPE);
  PTD_RETURN_IF(src && (rows_per_seq < 1 || N % rows_per_seq != 0), PTD_ERR_SHAPE);
  const int64_t row = static_cast<int64_t>(Hkv) * kHeadDim;
  PTD_RETURN_IF(ldk < row || ldv < row, PTD_ERR_SHAPE);
  const int per16 = dtype == PTD_F32 ? 4 : 8;
  PTD_RETURN_IF(ldk % per16 != 0 || ldv % per16 != 0 || !ptd_aligned(k, 16) || !ptd_aligned(v, 16) ||
                    !ptd_aligned(kv->k_pages, 16) || !ptd_aligned(kv->v_pages, 16) ||
                    !ptd_aligned(kv->scales, 4),
                PTD_ERR_ALIGN);
  if (N == 0) return PTD_OK;
  WriteParams prm;
  prm.src[0] = k;
  prm.src[1] = v;
  prm.ld[0] = ldk;
  prm.ld[1] = ldv;
  prm.pages[0] = kv->k_pages;
  prm.pages[1] = kv->v_pages;
  prm.scales = kv->scales;
  prm.slots = slots;
  prm.from = src;
  prm.dev_status = dev_status;
  prm.N = N;
  prm.rows_per_seq = src ? rows_per_seq : 1;
  prm.Hkv = Hkv;
  prm.slot_end = static_cast<long long>(kv->num_pages) * ps;
  prm.page_shift = 0;
  while ((1 << prm.page_shift) < ps) ++prm.page_shift;
  prm.scale_shift = sr == 32 ? 5 : sr == 64 ? 6 : 7;
  // Rows per workgroup: a block's rows (one run each for prompts), halved while
  // workgroups are fewer than CUs -- a step's rows open several blocks within that many
  // rows, which a wave codes one after the other.  (16 x 64 rows: 7.3 us, and 10.1 with four
  // times the workgroups, most of which find no block; 64 x 64 rows 11.6 and 23.)
  const int pairs = (Hkv + 1) / 2;
  prm.chunk = sr;
  while (prm.chunk > 1 && (static_cast<long long>(N) + prm.chunk - 1) / prm.chunk * pairs < 256) prm.chunk /= 2;
  // (two dimensions: one holds fewer than 2^32 threads; workgroups past the rows find none)
  const long long all = (static_cast<long long>(N) + prm.chunk - 1) / prm.chunk * pairs;
  PTD_RETURN_IF(all > 0x7FFFFFFFLL, PTD_ERR_SHAPE);
  const long long gx = std::min(all, 1LL << 20);
  const dim3 grid(static_cast<unsigned>(gx), static_cast<unsigned>((all + gx - 1) / gx));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == PTD_F32) src ? launch_write<float, true>(prm, sr, grid, st) : launch_write<float, false>(prm, sr, grid, st);
  else src ? launch_write<uint16_t, true>(prm, sr, grid, st) : launch_write<uint16_t, false>(prm, sr, grid, st);
  return ptd_launch_status();
}
