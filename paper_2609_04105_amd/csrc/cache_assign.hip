// Pages, slots and positions of a step's tokens, from the keys that each sequence held and has now.
//
// With f = shared / page, h = max(ceil(held / page), f) and p = max(ceil(length / page), f) pages of
// sequence b, need = max(p - h, 0), back = max(h - p, 0) and their exclusive sums N, R over the sequences:
//   table[b][h + i] = ring[(taken + N_b + i) mod capacity]         i < need, where the pool has that many
//   ring[(returned + R_b + i) mod capacity] = table[b][p + i]      i < back
//   slot of token t: key j = length - new + t in page table[b][j / page]
// Three prefix sums over the sequences, then every token and every page by itself: the sums go through one
// workgroup, the rest over as many as there are tokens; a thread finds its sequence by bisection.
// What bounds it: latency.  The data of a step are a few KB; 64 sequences with a token each take 4.2 us in a graph (a fill of one
// word 1.6), 48 with 19 thousand tokens of prompts 7.5, 4096 with 35 thousand new tokens 13.5.
#include "gfx950.hpp"
#include "serving.hpp"

namespace fp4attn {

namespace {

constexpr int kScanThreads = 1024, kScanWaves = kScanThreads / 64;
constexpr int kFillThreads = 256;
constexpr int kAssignLds = 4096;  // sequences whose sums a workgroup copies to LDS

// Of the whole call.
struct Totals {
  unsigned take0, give0;  // places of the ring where pages are taken and returned
  int takes, gives;       // pages
};
// Of every sequence [B]: the exclusive sums of new tokens (and their end), of pages asked for and of pages returned by the
// sequences before; its pages before the step, ~pages if it was refused, and after.
struct Sums {
  Totals* totals;
  int* start;
  int* need;
  int* back;
  int* had;
  int* now;
};
__device__ __forceinline__ Sums sums(const CacheAssignArgs& a) {
  Sums s;
  s.totals = static_cast<Totals*>(a.workspace);
  s.start = a.starts;
  s.need = reinterpret_cast<int*>(s.totals + 1);
  s.back = s.need + a.B;
  s.had = s.back + a.B;
  s.now = s.had + a.B;
  return s;
}

__device__ __forceinline__ int scan_wave(int x) {  // inclusive
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// What one sequence asks for.
struct Given {
  int held, length, fresh, shared;
};
struct Request {
  int had, now, keys, fresh;
  bool fits;
};
__device__ __forceinline__ int new_tokens(const CacheAssignArgs& a, int b) {
  const int n = a.fresh ? a.fresh[b] : a.each;
  return n < 0 ? 0 : n;
}
__device__ __forceinline__ int shared_pages(const CacheAssignArgs& a, int s) {
  const int capacity = a.max_pages << a.page_shift;  // 2^30 at most
  return (s < 0 ? 0 : (s > capacity ? capacity : s)) >> a.page_shift;
}
__device__ __forceinline__ Given given(const CacheAssignArgs& a, int b) {
  return Given{a.held[b], a.lengths[b], new_tokens(a, b), a.shared ? a.shared[b] : 0};
}
__device__ __forceinline__ Request request(const CacheAssignArgs& a, const Given& g) {
  Request r;
  const int first = shared_pages(a, g.shared), capacity = a.max_pages << a.page_shift, page = 1 << a.page_shift;
  r.fresh = g.fresh;
  r.fits = g.length <= capacity;
  r.keys = g.held < 0 ? 0 : (g.held > capacity ? capacity : g.held);
  const int want = g.length < 0 ? 0 : (r.fits ? g.length : capacity);
  const int had = (r.keys + page - 1) >> a.page_shift, now = (want + page - 1) >> a.page_shift;
  r.had = had > first ? had : first;
  r.now = now > first ? now : first;
  return r;
}

// One workgroup: the sums, the starts, the lengths and counts after the step.
__device__ __forceinline__ void make_sums(const CacheAssignArgs& a, const Sums& s) {
  __shared__ int lds[3][kScanWaves];
  __shared__ int lds_takes;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t taken = a.counts[0], returned = a.counts[1];
  const int64_t left = (int64_t)((uint64_t)returned - (uint64_t)taken);
  const int room = left < 0 ? 0 : (left > a.capacity ? a.capacity : (int)left);
  if (threadIdx.x == 0) lds_takes = 0;
  int need0 = 0, back0 = 0, start0 = 0;  // of the sequences before
  Given next{};                          // a turn's values come while the turn before is summed
  if ((int)threadIdx.x < a.B) next = given(a, threadIdx.x);
  for (int b0 = 0; b0 < a.B; b0 += kScanThreads) {
    const int b = b0 + threadIdx.x;
    const Given g = next;
    if (b + kScanThreads < a.B) next = given(a, b + kScanThreads);
    Request r{};
    int need = 0, back = 0, fresh = 0;
    if (b < a.B) {
      r = request(a, g);
      need = r.fits && r.now > r.had ? r.now - r.had : 0;
      back = r.fits && r.had > r.now ? r.had - r.now : 0;
      fresh = r.fresh > a.tokens ? a.tokens : r.fresh;
    }
    const int need1 = scan_wave(need), back1 = scan_wave(back), fresh1 = scan_wave(fresh);  // 64 * 2^24 tokens at most
    __syncthreads();
    if (lane == 63) {
      lds[0][wave] = need1;
      lds[1][wave] = back1;
      lds[2][wave] = fresh1 > a.tokens ? a.tokens : fresh1;
    }
    __syncthreads();
    // every wave sums the sixteen waves' totals up to its own, and all
    int before[3], all[3];
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      const int sum = scan_wave(lane < kScanWaves ? lds[j][lane] : 0);
      before[j] = wave == 0 ? 0 : __builtin_amdgcn_readlane(sum, wave - 1);
      all[j] = __builtin_amdgcn_readlane(sum, kScanWaves - 1);
    }
    before[0] += need0;
    before[1] += back0;
    before[2] += start0;  // 2^24 and sixteen times 2^24 at most
    need0 += all[0];
    back0 += all[1];
    start0 = start0 + all[2] > a.tokens ? a.tokens : start0 + all[2];
    if (b < a.B) {
      const int upto = before[0] + need1;
      const bool served = r.fits && (need == 0 || upto <= room);
      const int end = before[2] + fresh1;
      s.need[b] = upto - need;
      s.back[b] = before[1] + back1 - back;
      s.had[b] = served ? r.had : ~r.had;
      s.now[b] = r.now;
      const int stop = end > a.tokens ? a.tokens : end;
      s.start[b + 1] = stop;
      if (s.start != a.starts) a.starts[b + 1] = stop;
      a.lengths_out[b] = served ? (g.length < 0 ? 0 : g.length) : r.keys;
      if (served && need > 0) atomicMax(&lds_takes, upto);  // (the largest, in whatever order)
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    s.start[0] = a.starts[0] = 0;
    const int64_t n = a.capacity;
    *s.totals = Totals{(unsigned)((taken % n + n) % n), (unsigned)((returned % n + n) % n), lds_takes, back0};
    a.counts_out[0] = taken + lds_takes;
    a.counts_out[1] = returned + back0;
  }
}

// The last of n ascending values that is not above x[j] (the first is not).  Every lane takes the same steps, and N
// searches go side by side.
template <int N>
__device__ __forceinline__ void find_last(const int* v, int n, const int (&x)[N], int (&at)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) at[j] = 0;
  for (int half = n > 1 ? 1 << (31 - __builtin_clz(n - 1)) : 0; half > 0; half >>= 1) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int mid = at[j] + half, in = mid < n ? mid : n - 1;
      at[j] = v[in] <= x[j] ? in : at[j];
    }
  }
}

// Moves pages first + i step, i < N, of `total`: sequence b's are those from before[b]; from(b, i, k) is page i of the
// sequence, k of all, and to(b, i, k) takes it.  (N loads in flight: a load behind a store to what may be the same place waits.)
template <int N, class From, class To>
__device__ __forceinline__ void move_pages(const int* before, int B, int first, int step, int total, From&& from, To&& to) {
  for (unsigned k0 = first; k0 < (unsigned)total; k0 += N * step) {  // (unsigned: may pass 2^31)
    int k[N], b[N], page[N];
#pragma unroll
    for (int j = 0; j < N; ++j) k[j] = (int)(k0 + j * step < (unsigned)total ? k0 + j * step : k0);
    find_last(before, B, k, b);
#pragma unroll
    for (int j = 0; j < N; ++j) page[j] = from(b[j], k[j] - before[b[j]], k[j]);
#pragma unroll
    for (int j = 0; j < N; ++j) to(b[j], k[j] - before[b[j]], k[j], page[j]);
  }
}

// The tokens and pages of threads first, first + step, ..
__device__ __forceinline__ void fill(const CacheAssignArgs& a, const Sums& s, int first, int step) {
  const Totals total = *s.totals;
  const unsigned ring = (unsigned)a.capacity;
  auto taken_page = [&](int k) { return a.ring[(total.take0 + (unsigned)k) % ring]; };
  const int used = s.start[a.B];
  for (int i = first; i < a.tokens; i += step) {
    int64_t slot = -1, at = 0;
    if (i < used) {
      int b = 0;
      if (a.fresh) {
        const int x[1] = {i};
        int last[1];
        find_last(s.start, a.B, x, last);
        b = last[0];
      } else {
        b = i / a.each;
      }
      const int had = s.had[b];
      at = (int64_t)a.lengths[b] - new_tokens(a, b) + (i - s.start[b]);
      const int64_t capacity = (int64_t)a.max_pages << a.page_shift;
      if (had >= 0 && at >= (int64_t)shared_pages(a, a.shared ? a.shared[b] : 0) << a.page_shift && at < capacity) {
        const int place = (int)(at >> a.page_shift);
        const int page = place >= had ? taken_page(s.need[b] + place - had) : a.page_table[(int64_t)b * a.max_pages + place];
        if (page >= 0) slot = ((int64_t)page << a.page_shift) + (at & ((1 << a.page_shift) - 1));
      }
    }
    a.slots[i] = slot;
    a.positions[i] = at < 0 ? 0 : at;
  }
  auto row = [&](int b) { return a.page_table + (int64_t)b * a.max_pages; };
  auto take = [&](int, int, int k) { return taken_page(k); };
  auto keep = [&](int b, int i, int, int page) { row(b)[s.had[b] + i] = page; };
  auto give = [&](int b, int i, int) { return row(b)[s.now[b] + i]; };
  auto back = [&](int, int, int k, int page) { a.ring[(total.give0 + (unsigned)k) % ring] = page; };
  if (total.takes <= step) move_pages<1>(s.need, a.B, first, step, total.takes, take, keep);
  else move_pages<4>(s.need, a.B, first, step, total.takes, take, keep);
  if (total.gives <= step) move_pages<1>(s.back, a.B, first, step, total.gives, give, back);
  else move_pages<4>(s.back, a.B, first, step, total.gives, give, back);
}

// Small steps: everything in one workgroup, whose sums stay in LDS.
__global__ __launch_bounds__(kScanThreads) void cache_assign_kernel(const CacheAssignArgs a) {
  __shared__ Totals totals;
  __shared__ int start[kAssignOne + 1], need[kAssignOne], back[kAssignOne], had[kAssignOne], now[kAssignOne];
  const Sums s{&totals, start, need, back, had, now};
  make_sums(a, s);
  __syncthreads();
  fill(a, s, threadIdx.x, kScanThreads);
}

__global__ __launch_bounds__(kScanThreads) void cache_assign_sums_kernel(const CacheAssignArgs a) { make_sums(a, sums(a)); }
// Searches go through LDS: for 4096 sequences with 35 thousand new tokens this launch takes 6 us, with searches in memory
// (twelve dependent loads each) 13.
__global__ __launch_bounds__(kFillThreads) void cache_assign_fill_kernel(const CacheAssignArgs a) {
  __shared__ int lds[3][kAssignLds + 1];
  const int first = blockIdx.x * kFillThreads + threadIdx.x, step = gridDim.x * kFillThreads;
  Sums s = sums(a);
  if (a.B <= kAssignLds) {
    constexpr int kTurns = 8;  // loads of an array in flight
    for (int i0 = threadIdx.x; i0 < a.B; i0 += kTurns * kFillThreads) {
      int x[3][kTurns];
#pragma unroll
      for (int u = 0; u < kTurns; ++u) {
        const int i = i0 + u * kFillThreads < a.B ? i0 + u * kFillThreads : i0;
        x[0][u] = s.start[i];
        x[1][u] = s.need[i];
        x[2][u] = s.back[i];
      }
#pragma unroll
      for (int u = 0; u < kTurns; ++u) {
        const int i = i0 + u * kFillThreads < a.B ? i0 + u * kFillThreads : i0;
#pragma unroll
        for (int j = 0; j < 3; ++j) lds[j][i] = x[j][u];
      }
    }
    if (threadIdx.x == 0) lds[0][a.B] = s.start[a.B];
    __syncthreads();
    s.start = lds[0];
    s.need = lds[1];
    s.back = lds[2];
    fill(a, s, first, step);
  } else {
    fill(a, s, first, step);
  }
}

}  // namespace

hipError_t launch_cache_assign(const CacheAssignArgs& a, hipStream_t stream) {
  if (assign_in_one(a.B, a.tokens)) {
    cache_assign_kernel<<<1, kScanThreads, 0, stream>>>(a);
  } else {
    // pages: at most the tables' and the ring's; a thread for every fourth, as few steps move many
    const int64_t places = (int64_t)a.B * a.max_pages, pages = (places < a.capacity ? places : a.capacity) / 4;
    const int64_t items = a.tokens > pages ? a.tokens : pages, groups = (items + kFillThreads - 1) / kFillThreads;
    cache_assign_sums_kernel<<<1, kScanThreads, 0, stream>>>(a);
    cache_assign_fill_kernel<<<(unsigned)(groups < 1 ? 1 : (groups < 1024 ? groups : 1024)), kFillThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace fp4attn
