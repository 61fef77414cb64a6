// Pages that several sequences hold: sequences that go on from others' rows
// (ptd_page_fork), live pages moved to the front (ptd_page_compact), and the pages' data
// (ptd_page_copy).  refs[p] is the number of sequences that hold page p, 0 for a free one.
#include <algorithm>

#include "ptd_common.hpp"
#include "ptd_internal.hpp"

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / PTD_WAVE;

// Exclusive sum of v over the workgroup; the total to every thread.
__device__ __forceinline__ int block_scan(int v, int* lds, int* total) {
  const int wave = threadIdx.x >> 6;
  const int in = ptd::wave_scan_i32(v, [](int a, int b) { return a + b; });
  __syncthreads();  // lds of the call before is read
  if ((threadIdx.x & 63) == 63) lds[wave] = in;
  __syncthreads();
  int base = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int x = lds[w];
    if (w < wave) base += x;
    all += x;
  }
  *total = all;
  return base + in - v;
}

struct ForkArgs {
  ptd_page_state s;
  int32_t* refs;
  const int32_t* from;
  const int32_t* len;
  int32_t* table_next;
  int32_t* held_next;
  int32_t* copy_src;
  int32_t* copy_dst;
  int32_t* copy_rows;
  int32_t* dev_status;
  int page_shift;
};

// A page's count while a fork is worked out: whether any sequence held it, then either how many
// sequences hold it as a whole one, or (kPart) 65535 - the lowest sequence that goes on in it.
constexpr int kHeld = 1 << 30, kPart = 1 << 29, kCount = kPart - 1;

// What sequence b is to hold: whole pages of sequence a, and the rows of a page in part.
struct Fork {
  int a, whole, part;
};
__device__ __forceinline__ Fork fork_of(const ForkArgs& g, int b) {
  const int a = g.from[b];
  const int n = a < 0 ? 0 : g.len[b];
  return {a, n >> g.page_shift, n & ((1 << g.page_shift) - 1)};
}
__device__ __forceinline__ const int32_t* table_of(const ForkArgs& g, int b) {
  return g.s.page_table + static_cast<size_t>(b) * g.s.max_pages;
}

// One workgroup, a wave per sequence where tables are read and a thread per page where counts
// are.  Everything is checked before anything is changed.  Which of several sequences keeps a page
// that they all go on in is settled by the largest of 65535 - b, so no output depends on the
// order of the atomics.
__global__ void __launch_bounds__(kThreads) k_page_fork(ForkArgs g) {
  __shared__ int s_scan[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int B = g.s.B, n = g.s.num_pages;
  const int count = g.s.num_free[0];
  // ---- checks
  int bad = count < 0 || count > n ? PTD_ERR_PAGE : 0;
  for (int b = wave; b < B; b += kWaves) {
    const int a = g.from[b], held = g.s.num_held[b];
    if (held < 0 || held > g.s.max_pages) bad = PTD_ERR_PAGE;
    if (a < -1 || a >= B) bad = PTD_ERR_ROWS;
    if (bad || a < 0) continue;
    const int have = g.s.num_held[a];
    const long long rows = static_cast<long long>(have) << g.page_shift;
    if (have < 0 || have > g.s.max_pages) bad = PTD_ERR_PAGE;
    else if (g.len[b] < 0 || g.len[b] > rows) bad = PTD_ERR_KV_LEN;
    if (bad) continue;
    const Fork f = fork_of(g, b);
    const int32_t* row = table_of(g, a);
    for (int k = lane; k < f.whole + (f.part > 0); k += PTD_WAVE)
      if (static_cast<uint32_t>(row[k]) >= static_cast<uint32_t>(n)) bad = PTD_ERR_PAGE;
  }
  if (bad) ptd::report(g.dev_status, bad);
  bool refused = __syncthreads_or(bad != 0);
  int copies = 0;
  if (!refused) {
    // ---- who holds a page as a whole one
    for (int p = tid; p < n; p += kThreads) ptd::store_count(g.refs + p, g.refs[p] > 0 ? kHeld : 0);
    ptd::drained_barrier();
    for (int b = wave; b < B; b += kWaves) {
      const Fork f = fork_of(g, b);
      if (f.whole == 0) continue;
      const int32_t* row = table_of(g, f.a);
      for (int k = lane; k < f.whole; k += PTD_WAVE) ptd::add_count(g.refs + row[k], 1);
    }
    ptd::drained_barrier();
    // ---- who goes on in a page that nobody holds as a whole one: the lowest
    for (int b = tid; b < B; b += kThreads) {
      const Fork f = fork_of(g, b);
      if (f.part == 0) continue;
      int32_t* r = g.refs + table_of(g, f.a)[f.whole];
      const int v = ptd::load_count(r);
      if ((v & kPart) || (v & kCount) == 0) ptd::max_count(r, kHeld | kPart | (65535 - b));
    }
    ptd::drained_barrier();
    for (int b0 = 0; b0 < B; b0 += kThreads) {  // uniform
      bool copy = false;
      if (b0 + tid < B) {
        const Fork f = fork_of(g, b0 + tid);
        copy = f.part > 0 && ptd::load_count(g.refs + table_of(g, f.a)[f.whole]) != (kHeld | kPart | (65535 - b0 - tid));
      }
      copies += __syncthreads_count(copy);
    }
    // the pages that are taken have to be there, and are checked as the tables were
    bool short_of = copies > count;
    if (!short_of) {
      int odd = 0;
      for (int i = tid; i < copies; i += kThreads)
        if (static_cast<uint32_t>(g.s.free_pages[count - 1 - i]) >= static_cast<uint32_t>(n)) odd = 1;
      if (odd) ptd::report(g.dev_status, PTD_ERR_PAGE);
      refused = __syncthreads_or(odd);
    } else {
      if (tid == 0) ptd::report(g.dev_status, PTD_ERR_NO_PAGES);
      refused = true;
    }
    if (refused) {  // the counts as they were: by the tables
      for (int p = tid; p < n; p += kThreads) ptd::store_count(g.refs + p, 0);
      ptd::drained_barrier();
      for (int b = wave; b < B; b += kWaves) {
        const int32_t* row = table_of(g, b);
        for (int k = lane; k < g.s.num_held[b]; k += PTD_WAVE)
          if (static_cast<uint32_t>(row[k]) < static_cast<uint32_t>(n)) ptd::add_count(g.refs + row[k], 1);
      }
    }
  }
  if (refused) {  // nothing changes
    for (int b = wave; b < B; b += kWaves) {
      const int held = min(max(g.s.num_held[b], 0), g.s.max_pages);
      for (int k = lane; k < held; k += PTD_WAVE)
        g.table_next[static_cast<size_t>(b) * g.s.max_pages + k] = table_of(g, b)[k];
      if (lane == 0) {
        g.held_next[b] = g.s.num_held[b];
        g.copy_src[b] = g.copy_dst[b] = -1;
        g.copy_rows[b] = 0;
      }
    }
    return;
  }
  // ---- tables, copies
  for (int b = wave; b < B; b += kWaves) {
    const Fork f = fork_of(g, b);
    if (f.whole == 0) continue;
    const int32_t* row = table_of(g, f.a);
    for (int k = lane; k < f.whole; k += PTD_WAVE) g.table_next[static_cast<size_t>(b) * g.s.max_pages + k] = row[k];
  }
  int taken = 0;
  for (int b0 = 0; b0 < B; b0 += kThreads) {  // uniform
    const int b = b0 + tid;
    Fork f = {-1, 0, 0};
    int page = -1;
    bool copy = false;
    if (b < B) {
      f = fork_of(g, b);
      if (f.part > 0) {
        page = table_of(g, f.a)[f.whole];
        copy = ptd::load_count(g.refs + page) != (kHeld | kPart | (65535 - b));
      }
    }
    int all;
    const int at = taken + block_scan(copy, s_scan, &all);
    if (b < B) {
      int mine = page;
      if (copy) {
        mine = g.s.free_pages[count - 1 - at];
        ptd::store_count(g.refs + mine, 1);
      }
      if (f.part > 0) g.table_next[static_cast<size_t>(b) * g.s.max_pages + f.whole] = mine;
      g.held_next[b] = f.whole + (f.part > 0);
      g.copy_src[b] = copy ? page : -1;
      g.copy_dst[b] = copy ? mine : -1;
      g.copy_rows[b] = copy ? f.part : 0;
    }
    taken += all;
  }
  ptd::drained_barrier();
  // ---- counts, and the pages that nobody holds any more, from the highest id down
  int at = count - copies;
  for (int p0 = 0; p0 < n; p0 += kThreads) {  // uniform
    const int p = n - 1 - p0 - tid;
    bool gone = false;
    if (p >= 0) {
      const int v = ptd::load_count(g.refs + p);
      const int now = (v & kPart) ? 1 : v & kCount;
      gone = (v & kHeld) && now == 0;
      g.refs[p] = now;
    }
    int all;
    const int to = at + block_scan(gone, s_scan, &all);
    if (gone && to < n) g.s.free_pages[to] = p;
    at += all;
  }
  if (tid == 0) {
    if (at > n) ptd::report(g.dev_status, PTD_ERR_PAGE);  // pages that were held and free
    g.s.num_free[0] = min(at, n);
  }
}

// Last index x of [0, n) with a[x] <= v (a ascending, a[0] <= v).
__device__ __forceinline__ int upper(const int* a, int n, int v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The same as k_page_fork with a sequence per thread and the pages' counts in LDS: what is left in memory is four waits
// one after the other (sequences, their sources, page ids, outputs), and nothing is changed
// there before all checks are done.
constexpr int kRound = 4 * kThreads;  // pages that the workgroup looks at in one turn
template <int PAGES>
__global__ void __launch_bounds__(kThreads) k_page_fork_lds(ForkArgs g) {
  __shared__ int s_count[PAGES];
  __shared__ int s_from[kThreads], s_whole[kThreads], s_part[kThreads], s_page[kThreads], s_free[kThreads];
  __shared__ int s_scan[kWaves];
  const int tid = threadIdx.x;
  const int B = g.s.B, n = g.s.num_pages;
  const int count = g.s.num_free[0];
  int bad = count < 0 || count > n ? PTD_ERR_PAGE : 0;
  Fork f = {-1, 0, 0};
  int held = 0;
  if (tid < B) {
    f = fork_of(g, tid);
    held = g.s.num_held[tid];
    if (held < 0 || held > g.s.max_pages) bad = PTD_ERR_PAGE;
    if (f.a < -1 || f.a >= B) bad = PTD_ERR_ROWS;
    if (!bad && f.a >= 0) {
      const int len = g.len[tid], have = g.s.num_held[f.a];
      if (have < 0 || have > g.s.max_pages) bad = PTD_ERR_PAGE;
      else if (len < 0 || len > static_cast<long long>(have) << g.page_shift) bad = PTD_ERR_KV_LEN;
    }
  }
  if (tid < count && !bad) s_free[tid] = g.s.free_pages[count - 1 - tid];
  for (int p = tid; p < n; p += kThreads) s_count[p] = 0;
  if (bad) ptd::report(g.dev_status, bad);
  bool refused = __syncthreads_or(bad != 0);
  int copies = 0, at = 0, page = -1, mine = -1;
  bool copy = false;
  if (!refused) {
    // ---- page ids: the whole ones are counted and go to the next table.  A wave has every 16th sequence
    // (fewer than 16: a sequence several waves), 64 ids a step; those of four sequences are in flight
    // together.  (The kernel with 64 beams of 80 pages 8.0 us, and 11.2 with a thread per entry that finds its
    // sequence by halving)
    s_from[tid] = f.a, s_whole[tid] = f.whole, s_part[tid] = f.part > 0;
    __syncthreads();
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int more = __builtin_clz(static_cast<unsigned>(min(B, kWaves))) - __builtin_clz(static_cast<unsigned>(kWaves));  // log2 of the waves of one
    const int ways = 1 << more, units = B << more;
    for (int u0 = wave; u0 < units; u0 += 4 * kWaves) {  // uniform
      int most = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int b = min((u0 + u * kWaves) >> more, B - 1);
        most = max(most, s_whole[b] + s_part[b]);
      }
      for (int c = 0; c < most; c += 2 * ways * PTD_WAVE) {
        int id[4][2];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int unit = u0 + u * kWaves, b = min(unit >> more, B - 1), k = c + ((unit & (ways - 1)) * 2 + h) * PTD_WAVE + lane;
            id[u][h] = -1;
            if (unit < units && k < s_whole[b] + s_part[b]) id[u][h] = table_of(g, s_from[b])[k];
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int unit = u0 + u * kWaves, b = min(unit >> more, B - 1), k = c + ((unit & (ways - 1)) * 2 + h) * PTD_WAVE + lane;
            if (unit < units && k < s_whole[b] + s_part[b]) {
              const int x = id[u][h];
              if (static_cast<uint32_t>(x) >= static_cast<uint32_t>(n)) bad = PTD_ERR_PAGE;
              else if (k < s_whole[b]) atomicAdd(&s_count[x], 1);
              if (k < s_whole[b]) g.table_next[static_cast<size_t>(b) * g.s.max_pages + k] = x;
              else s_page[b] = x;
            }
          }
        }
      }
    }
    if (bad) ptd::report(g.dev_status, bad);
    refused = __syncthreads_or(bad != 0);
  }
  if (!refused) {
    // ---- who goes on in a page that nobody holds as a whole one: the lowest
    const int me = kPart | (65535 - tid);
    if (f.part > 0) {
      page = s_page[tid];
      const int v = s_count[page];
      if ((v & kPart) || v == 0) atomicMax(&s_count[page], me);
    }
    __syncthreads();
    copy = f.part > 0 && s_count[page] != me;
    at = block_scan(copy, s_scan, &copies);
    mine = page;
    if (copies > count) {  // uniform
      bad = PTD_ERR_NO_PAGES;
      if (tid == 0) ptd::report(g.dev_status, bad);
    } else if (copy) {
      mine = s_free[at];
      if (static_cast<uint32_t>(mine) >= static_cast<uint32_t>(n)) {
        bad = PTD_ERR_PAGE;
        ptd::report(g.dev_status, bad);
      }
    }
    refused = __syncthreads_or(bad != 0);
  }
  if (refused) {  // nothing changes
    for (int b = tid >> 6; b < B; b += kWaves) {
      const int have = min(max(g.s.num_held[b], 0), g.s.max_pages);
      for (int k = tid & 63; k < have; k += PTD_WAVE) g.table_next[static_cast<size_t>(b) * g.s.max_pages + k] = table_of(g, b)[k];
    }
    if (tid < B) {
      g.held_next[tid] = held;
      g.copy_src[tid] = g.copy_dst[tid] = -1;
      g.copy_rows[tid] = 0;
    }
    return;
  }
  if (tid < B) {
    if (copy) s_count[mine] = 1;
    if (f.part > 0) g.table_next[static_cast<size_t>(tid) * g.s.max_pages + f.whole] = mine;
    g.held_next[tid] = f.whole + (f.part > 0);
    g.copy_src[tid] = copy ? page : -1;
    g.copy_dst[tid] = copy ? mine : -1;
    g.copy_rows[tid] = copy ? f.part : 0;
  }
  // ---- counts, and the pages that nobody holds any more, from the highest id down
  int to = count - copies;
  for (int p0 = (n - 1) / kRound * kRound; p0 >= 0; p0 -= kRound) {  // uniform
    int old[4], gone[4], m = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int p = p0 + 4 * tid + u;
      old[u] = p < n ? g.refs[p] : 0;
    }
    __syncthreads();  // (the fresh pages' counts)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int p = p0 + 4 * tid + u;
      const int v = p < n ? s_count[p] : 0;
      const int now = (v & kPart) ? 1 : v;
      gone[u] = old[u] > 0 && now == 0;
      m += gone[u];
      if (p < n && now != old[u]) g.refs[p] = now;
    }
    int all;
    int up = block_scan(m, s_scan, &all);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int j = to + all - 1 - up;
      if (gone[u] && j < n) g.s.free_pages[j] = p0 + 4 * tid + u;
      up += gone[u];
    }
    to += all;
  }
  if (tid == 0) {
    if (to > n) ptd::report(g.dev_status, PTD_ERR_PAGE);  // pages that were held and free
    g.s.num_free[0] = min(to, n);
  }
}

struct CompactArgs {
  ptd_page_state s;
  int32_t* refs;
  int32_t* move_src;
  int32_t* move_dst;
  int32_t* dev_status;
};

// One workgroup.  With L live pages, the k-th free id below L takes the k-th live page from L on
// (there are as many of both); a moved page's count holds -1 - its new id while the tables are
// changed.
__global__ void __launch_bounds__(kThreads) k_page_compact(CompactArgs g) {
  __shared__ int s_scan[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = g.s.num_pages;
  int live = 0;
  for (int p0 = 0; p0 < n; p0 += kThreads) {  // uniform
    const int p = p0 + tid;
    const int v = p < n ? g.refs[p] : 0;
    if (v < 0) {  // (no count: free)
      g.refs[p] = 0;
      ptd::report(g.dev_status, PTD_ERR_PAGE);
    }
    live += __syncthreads_count(v > 0);
  }
  int holes = 0, movers = 0;
  for (int p0 = 0; p0 < n; p0 += kThreads) {
    const int p = p0 + tid;
    const int v = p < n ? g.refs[p] : 0;
    const bool hole = p < live && v <= 0, mover = p < n && p >= live && v > 0;
    int all;
    const int i = holes + block_scan(hole, s_scan, &all);
    if (hole) g.move_dst[i] = p;
    holes += all;
    const int j = movers + block_scan(mover, s_scan, &all);
    if (mover) g.move_src[j] = p;
    movers += all;
  }
  __syncthreads();
  for (int i = tid; i < n / 2; i += kThreads) {
    if (i < movers) {
      const int a = g.move_src[i], b = g.move_dst[i];
      g.refs[b] = g.refs[a];
      g.refs[a] = -1 - b;
    } else {
      g.move_src[i] = g.move_dst[i] = -1;
    }
  }
  __syncthreads();
  for (int b = wave; b < g.s.B; b += kWaves) {
    const int held = g.s.num_held[b];
    if (held < 0 || held > g.s.max_pages) {
      if (lane == 0) ptd::report(g.dev_status, PTD_ERR_PAGE);
      continue;
    }
    int32_t* row = g.s.page_table + static_cast<size_t>(b) * g.s.max_pages;
    for (int k = lane; k < held; k += PTD_WAVE) {
      const int id = row[k];
      if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(n)) {
        ptd::report(g.dev_status, PTD_ERR_PAGE);
      } else {
        const int v = g.refs[id];
        if (v < 0) row[k] = -1 - v;
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < movers; i += kThreads) g.refs[g.move_src[i]] = 0;
  for (int i = tid; i < n - live; i += kThreads) g.s.free_pages[i] = n - 1 - i;
  if (tid == 0) g.s.num_free[0] = n - live;
}

// The same with a sequence per thread, counts and moves in LDS.
constexpr int kCompactPages = 8192;
__global__ void __launch_bounds__(kThreads) k_page_compact_lds(CompactArgs g) {
  __shared__ int s_ref[kCompactPages], s_src[kCompactPages / 2], s_dst[kCompactPages / 2];
  __shared__ int s_off[kThreads];
  __shared__ int s_scan[kWaves];
  const int tid = threadIdx.x;
  const int n = g.s.num_pages, B = g.s.B;
  int held = tid < B ? g.s.num_held[tid] : 0;
  if (held < 0 || held > g.s.max_pages) {
    ptd::report(g.dev_status, PTD_ERR_PAGE);
    held = 0;
  }
  int mine = 0, live, entries;
#pragma unroll 4
  for (int p = tid; p < n; p += kThreads) {
    const int v = g.refs[p];
    if (v < 0) {  // (no count: free)
      g.refs[p] = 0;
      ptd::report(g.dev_status, PTD_ERR_PAGE);
    }
    s_ref[p] = max(v, 0);
    mine += v > 0;
  }
  s_off[tid] = block_scan(held, s_scan, &entries);
  block_scan(mine, s_scan, &live);
  // ids of the first entries, on their way while the moves are found
  auto place = [&](int e) {
    const int b = upper(s_off, B, e);
    return g.s.page_table + static_cast<size_t>(b) * g.s.max_pages + (e - s_off[b]);
  };
  int32_t* where[4];
  int id[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int e = tid + u * kThreads;
    if (e < entries) where[u] = place(e), id[u] = *where[u];
  }
  int before = 0, movers = 0;  // live pages below the turn's first, movers among them
  for (int p0 = 0; p0 < n; p0 += kRound) {  // uniform
    int v[4], m = 0, all;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int p = p0 + 4 * tid + u;
      v[u] = p < n ? s_ref[p] : 0;
      m += v[u] > 0;
    }
    const int base = before + block_scan(m, s_scan, &all);
    int at = base;  // live pages below p; of the free ones below `live` the p - at first come before p
    int moving = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) moving += v[u] > 0 && p0 + 4 * tid + u >= live;
    int some;
    int j = movers + block_scan(moving, s_scan, &some);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int p = p0 + 4 * tid + u;
      if (v[u] > 0) {
        if (p >= live) s_src[j++] = p;
        ++at;
      } else if (p < live) {
        s_dst[p - at] = p;
      }
    }
    before += all;
    movers += some;
  }
  __syncthreads();
  for (int i = tid; i < n / 2; i += kThreads) {
    const bool move = i < movers;
    const int a = move ? s_src[i] : -1, b = move ? s_dst[i] : -1;
    g.move_src[i] = a;
    g.move_dst[i] = b;
    if (move) {
      g.refs[b] = s_ref[a];
      g.refs[a] = 0;
      s_ref[a] = -1 - b;
    }
  }
  for (int i = tid; i < n - live; i += kThreads) g.s.free_pages[i] = n - 1 - i;
  if (tid == 0) g.s.num_free[0] = n - live;
  __syncthreads();
  auto change = [&](int32_t* w, int x) {
    if (static_cast<uint32_t>(x) >= static_cast<uint32_t>(n)) ptd::report(g.dev_status, PTD_ERR_PAGE);
    else if (s_ref[x] < 0) *w = -1 - s_ref[x];
  };
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (tid + u * kThreads < entries) change(where[u], id[u]);
#pragma unroll 4
  for (int e = tid + 4 * kThreads; e < entries; e += kThreads) {
    int32_t* w = place(e);
    change(w, *w);
  }
}

// ===========================================================================
// the pages' data
// ===========================================================================
constexpr int kCopyThreads = 256;
constexpr int kArrays = 96;  // of one launch
constexpr int kUnroll = 4;   // loads of a thread in flight
constexpr int kCopyGroups = 8192;

struct CopyArray {
  char* base;
  int32_t heads, units, unit_rows, unit_bytes, granule;
};
struct CopyArgs {
  CopyArray arrays[kArrays];
  const int32_t* src;
  const int32_t* dst;
  const int32_t* rows;
  int32_t* dev_status;
  int n, num_pages, pieces;  // of a page of the largest array
};

// Elements first .. first + kCopyThreads * kUnroll - 1 of `total`, in runs of `run`, `step` apart
// (one run: both are `total`).
template <typename V>
__device__ __forceinline__ void copy_piece(const char* from, char* to, uint32_t total, uint32_t run, uint32_t step, uint32_t first) {
  const V* __restrict__ s = reinterpret_cast<const V*>(from);
  V* __restrict__ d = reinterpret_cast<V*>(to);
  const uint32_t i = first + threadIdx.x;
  if (run == total && first + kCopyThreads * kUnroll <= total) {  // uniform
    static_assert(kUnroll == 4, "four loads");
    const V a = s[i], b = s[i + kCopyThreads], c = s[i + 2 * kCopyThreads], e = s[i + 3 * kCopyThreads];
    d[i] = a, d[i + kCopyThreads] = b, d[i + 2 * kCopyThreads] = c, d[i + 3 * kCopyThreads] = e;
    return;
  }
#pragma unroll 2
  for (int u = 0; u < kUnroll; ++u) {
    const uint32_t x = i + u * kCopyThreads;
    if (x < total) {
      const uint32_t h = run == total ? 0 : x / run;
      const uint32_t at = h * step + (x - h * run);
      d[at] = s[at];
    }
  }
}

// One workgroup per (pair, piece of its page) in turn, an array of pages per grid row.  Each lane
// looks up one of the workgroup's next 64 items, so lists that are mostly -1 (a compaction's) cost a wait per 64
// (4096 pairs in 24 arrays, 10 of them there: 7 us, and 50 where each item was looked up by itself).
// Bound by HBM, reads and writes mixed.
__global__ void __launch_bounds__(kCopyThreads) k_page_copy(CopyArgs g) {
  const CopyArray a = g.arrays[blockIdx.y];
  const long long items = static_cast<long long>(g.n) * g.pieces;
  const uint32_t step = static_cast<uint32_t>(a.units) * a.unit_bytes / a.granule;  // of a head, in elements
  const long long page = static_cast<long long>(a.heads) * a.units * a.unit_bytes;
  const int lane = threadIdx.x & 63;
  for (long long base = blockIdx.x; base < items; base += static_cast<long long>(PTD_WAVE) * gridDim.x) {  // uniform
    const long long item = base + static_cast<long long>(lane) * gridDim.x;
    int s = -1, d = -1, units = a.units;
    uint32_t first = 0;
    if (item < items) {
      const int i = static_cast<int>(item / g.pieces);
      first = static_cast<uint32_t>(item - static_cast<long long>(i) * g.pieces) * (kCopyThreads * kUnroll);
      s = g.src[i], d = g.dst[i];
      const int r = g.rows ? g.rows[i] : 0;
      if (s == -1 || d == -1 || s == d) {
        s = -1;
      } else if (static_cast<uint32_t>(s) >= static_cast<uint32_t>(g.num_pages) || static_cast<uint32_t>(d) >= static_cast<uint32_t>(g.num_pages)) {
        ptd::report(g.dev_status, PTD_ERR_PAGE);
        s = -1;
      } else if (g.rows) {
        if (r < 0 || r > static_cast<long long>(a.units) * a.unit_rows) {
          ptd::report(g.dev_status, PTD_ERR_ROWS);
          s = -1;
        }
        units = static_cast<int>((static_cast<long long>(r) + a.unit_rows - 1) / a.unit_rows);
      }
    }
    const uint32_t run_of = static_cast<uint32_t>(units) * a.unit_bytes / a.granule;
    for (uint64_t live = __ballot(s >= 0 && first < run_of * a.heads); live; live &= live - 1) {  // uniform
      const int l = __builtin_ctzll(live);
      const uint32_t run = __builtin_amdgcn_readlane(run_of, l), total = run * a.heads;
      const char* from = a.base + __builtin_amdgcn_readlane(s, l) * page;
      char* to = a.base + __builtin_amdgcn_readlane(d, l) * page;
      const uint32_t at = __builtin_amdgcn_readlane(first, l);
      const uint32_t one = run == step ? total : run;
      if (a.granule == 16) copy_piece<uint4>(from, to, total, one, step, at);
      else if (a.granule == 4) copy_piece<uint32_t>(from, to, total, one, step, at);
      else if (a.granule == 2) copy_piece<uint16_t>(from, to, total, one, step, at);
      else copy_piece<uint8_t>(from, to, total, one, step, at);
    }
  }
}

// A thread for every sequence, and all table entries counted in 31 bits.
bool one_turn(const ptd_page_state& s) {
  return s.B <= kThreads && static_cast<long long>(s.B) * s.max_pages <= 0x3FFFFFFFLL;
}

}  // namespace

extern "C" int ptd_page_fork(const ptd_page_state* state, int32_t* refs, const int32_t* from, const int32_t* len,
                             int32_t* table_next, int32_t* held_next, int32_t* copy_src, int32_t* copy_dst,
                             int32_t* copy_rows, int32_t* dev_status, void* stream) {
  ForkArgs g = {};
  const int rc = ptd_check_state(state, &g.page_shift);
  if (rc != PTD_OK) return rc;
  PTD_RETURN_IF(!refs || !from || !len || !table_next || !held_next || !copy_src || !copy_dst || !copy_rows, PTD_ERR_NULL);
  PTD_RETURN_IF(table_next == state->page_table || held_next == state->num_held, PTD_ERR_SHAPE);
  g.s = *state;
  g.refs = refs;
  g.from = from;
  g.len = len;
  g.table_next = table_next;
  g.held_next = held_next;
  g.copy_src = copy_src;
  g.copy_dst = copy_dst;
  g.copy_rows = copy_rows;
  g.dev_status = dev_status;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool small = one_turn(*state);
  if (small && state->num_pages <= 8192) hipLaunchKernelGGL((k_page_fork_lds<8192>), dim3(1), dim3(kThreads), 0, st, g);
  else if (small && state->num_pages <= 32768) hipLaunchKernelGGL((k_page_fork_lds<32768>), dim3(1), dim3(kThreads), 0, st, g);
  else hipLaunchKernelGGL(k_page_fork, dim3(1), dim3(kThreads), 0, st, g);
  return ptd_launch_status();
}

extern "C" int ptd_page_compact(const ptd_page_state* state, int32_t* refs, int32_t* move_src, int32_t* move_dst,
                                int32_t* dev_status, void* stream) {
  CompactArgs g = {};
  int shift = 0;
  const int rc = ptd_check_state(state, &shift);
  if (rc != PTD_OK) return rc;
  PTD_RETURN_IF(!refs || (state->num_pages > 1 && (!move_src || !move_dst)), PTD_ERR_NULL);
  g.s = *state;
  g.refs = refs;
  g.move_src = move_src;
  g.move_dst = move_dst;
  g.dev_status = dev_status;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (one_turn(*state) && state->num_pages <= kCompactPages) hipLaunchKernelGGL(k_page_compact_lds, dim3(1), dim3(kThreads), 0, st, g);
  else hipLaunchKernelGGL(k_page_compact, dim3(1), dim3(kThreads), 0, st, g);
  return ptd_launch_status();
}

extern "C" int ptd_page_copy(const ptd_page_array* arrays, int32_t num_arrays, int32_t num_pages, int32_t n,
                             const int32_t* src, const int32_t* dst, const int32_t* rows, int32_t* dev_status,
                             void* stream) {
  PTD_RETURN_IF(num_arrays < 0 || num_pages < 1 || n < 0, PTD_ERR_SHAPE);
  if (num_arrays == 0 || n == 0) return PTD_OK;
  PTD_RETURN_IF(!arrays || !src || !dst, PTD_ERR_NULL);
  for (int i = 0; i < num_arrays; ++i) {
    const ptd_page_array& x = arrays[i];
    PTD_RETURN_IF(!x.base, PTD_ERR_NULL);
    PTD_RETURN_IF(x.heads < 1 || x.units < 1 || x.unit_rows < 1 || x.unit_bytes < 1, PTD_ERR_SHAPE);
    // a page is below 2^31 bytes
    PTD_RETURN_IF(static_cast<long long>(x.units) * x.unit_bytes > 0x7FFFFFFFLL / x.heads, PTD_ERR_SHAPE);
  }
  for (int first = 0; first < num_arrays; first += kArrays) {
    CopyArgs g = {};
    const int m = std::min(kArrays, num_arrays - first);
    long long most = 0;
    for (int i = 0; i < m; ++i) {
      const ptd_page_array& x = arrays[first + i];
      // the widest elements that every unit of every page is aligned for
      const uintptr_t any = reinterpret_cast<uintptr_t>(x.base) | static_cast<uintptr_t>(x.unit_bytes);
      const int granule = any % 16 == 0 ? 16 : any % 4 == 0 ? 4 : any % 2 == 0 ? 2 : 1;
      g.arrays[i] = {static_cast<char*>(x.base), x.heads, x.units, x.unit_rows, x.unit_bytes, granule};
      most = std::max(most, static_cast<long long>(x.heads) * x.units * x.unit_bytes / granule);
    }
    g.src = src;
    g.dst = dst;
    g.rows = rows;
    g.dev_status = dev_status;
    g.n = n;
    g.num_pages = num_pages;
    constexpr int kPiece = kCopyThreads * kUnroll;
    g.pieces = static_cast<int>((most + kPiece - 1) / kPiece);
    const long long items = static_cast<long long>(n) * g.pieces;
    const unsigned gx = static_cast<unsigned>(std::min<long long>(items, std::max(1, kCopyGroups / m)));
    hipLaunchKernelGGL(k_page_copy, dim3(gx, m), dim3(kCopyThreads), 0, static_cast<hipStream_t>(stream), g);
    const int rc = ptd_launch_status();
    if (rc != PTD_OK) return rc;
  }
  return PTD_OK;
}
