// Pages of the paged 8-bit cache: who holds which, and copies of them.
//
// A page is free if its count of references is 0, and free pages are taken lowest number first, so that the outcome depends on
// the counts alone: counts are changed by integer atomics, whose order does not matter, and one workgroup takes pages, for the
// sequences in order. Bound by the calls and by chains of requests: a row's length, its entries, their counts, the free pages.
#include <type_traits>

#include "fluxbin_device.h"
#include "fluxbin_serve_internal.h"

namespace fluxbin {

namespace {

typedef int pg_i4 __attribute__((ext_vector_type(4)));

constexpr int kTake = 1024;   // threads of the workgroup that takes pages

__device__ __forceinline__ bool is_page(int page, int pages) { return page >= 0 && page < pages; }

// Pages that rows want together: up to 2^24 a row. LARGE: of tables with 2^31 entries or more. Of others they fit 32 bits (all in 64
// bits: a fork of 4 children 5.5 us instead of 5.0, growth of 256 rows 9.1 instead of 8.8).
template <bool LARGE>
using Wanted = std::conditional_t<LARGE, int64_t, int>;

// Inclusive sums over a workgroup's threads; total in every thread. LARGE: the sums are cut off at 2^30, which no place among free
// pages (2^24 at most) comes near; the total is whole.
template <bool LARGE>
__device__ __forceinline__ int block_sum(int v, int* red, Wanted<LARGE>& total) {
  const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();   // red of the sum before
  if (lane == 63) red[wave] = v;
  __syncthreads();
  total = 0;
  for (int w = 0; w < kTake / 64; ++w) {
    const int s = red[w];
    if (w < wave) v = int(uint32_t(v) + uint32_t(s));   // LARGE: each up to 2^30
    if (LARGE) v = uint32_t(v) < (1u << 30) ? v : 1 << 30;
    total += s;
  }
  return v;
}

// What a thread's row wants: `want` entries from entry `from` on. copies, source: where not NULL, (source, page) of its one want.
struct Taking {
  int want, from;
  int32_t* row;
  int32_t* copies;
  int source;
};

struct TakeLds {
  int red[kTake / 64];
  int upto[kTake];
  Taking who[kTake];
  int list[4 * kTake];   // free pages among those that are looked at
  int next;
};

// Four counts a thread from page `scan` on (the one that its four are a multiple of four from), pages past the last in use.
__device__ __forceinline__ pg_i4 counts_at(const PoolArgs& p, int scan) {
  const int32_t* refs = p.state + 4;
  const int at = (scan & ~3) + 4 * int(threadIdx.x);
  pg_i4 r = {1, 1, 1, 1};
  if (at + 3 < p.pages) {
    r = *reinterpret_cast<const pg_i4*>(refs + at);
  } else {
    for (int i = 0; i < 4; ++i)
      if (at + i < p.pages) r[i] = refs[at + i];
  }
  return r;
}

// Takes free pages for the wants of up to kTake rows, in order. scan: the page from which on to look, the same in all threads, with
// the counts there. Returns how many pages were missing, in all threads.
template <bool LARGE>
__device__ Wanted<LARGE> take(const PoolArgs& p, const Taking& mine, int& scan, pg_i4& counts, TakeLds& s) {
  const int tid = int(threadIdx.x);
  Wanted<LARGE> wanted;
  const int upto = block_sum<LARGE>(mine.want, s.red, wanted);
  if (wanted == 0) return 0;
  s.upto[tid] = upto;
  s.who[tid] = mine;
  __syncthreads();
  int32_t* refs = p.state + 4;
  int done = 0;
  while (done < wanted && scan < p.pages) {
    // others may raise counts of pages in use meanwhile, not of free ones
    const int at = (scan & ~3) + 4 * tid;
    pg_i4 r = counts;
    int free = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (at + i < scan) r[i] = 1;
      free += r[i] <= 0 ? 1 : 0;
    }
    int found;
    int k = block_sum<false>(free, s.red, found) - free;
    if (tid == 0) s.next = (scan & ~3) + 4 * kTake;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (r[i] <= 0) s.list[k++] = at + i;
    __syncthreads();
    const int n = found < wanted - done ? found : int(wanted - done);
    for (int f = tid; f < n; f += kTake) {
      int lo = 0, rows = kTake;   // the first row whose sum is above that of the page
      while (rows > 0) {
        const int h = rows >> 1;
        if (s.upto[lo + h] <= done + f) {
          lo += h + 1;
          rows -= h + 1;
        } else {
          rows = h;
        }
      }
      const Taking w = s.who[lo];
      const int page = s.list[f];
      w.row[w.from + done + f - (s.upto[lo] - w.want)] = page;
      if (w.copies) {
        w.copies[0] = w.source;
        w.copies[1] = page;
      }
      refs[page] = 1;
      if (done + f == wanted - 1) s.next = page + 1;
    }
    __syncthreads();
    scan = s.next < p.pages ? s.next : p.pages;
    done += n;
    counts = counts_at(p, scan);   // for the next round or call; what was taken is seen: the barrier is behind it
  }
  __syncthreads();
  return wanted - done;
}

// Entries that a row of the table holds, up to `most`: the first that is no page. Seven places at a time.
__device__ int held_entries(const int32_t* row, int most, int pages) {
  int lo = 0, n = most;   // it is one of lo .. lo + n
  while (n > 0) {
    const int step = (n + 7) >> 3;
    int below = 0;   // places with pages, which come first
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      const int at = step * i - 1;
      below += at < n && is_page(row[lo + (at < n ? at : 0)], pages) ? 1 : 0;
    }
    lo += step * below;
    n -= step * below;
    if (below < 7 && n > step - 1) n = step - 1;   // the next place has none
  }
  return lo;
}

__device__ __forceinline__ int need_entries(const ResizeArgs& a, int b) {
  const int t = a.tokens[b];
  if (t < 0) return -1;
  const int64_t n = (int64_t(t) + (1 << a.pool.pshift) - 1) >> a.pool.pshift;
  return n < a.max_blocks ? int(n) : a.max_blocks;
}

// What row r, of need n, wants.
__device__ __forceinline__ Taking wants_of(const ResizeArgs& a, int r, int n) {
  Taking t = {0, 0, nullptr, nullptr, 0};
  if (n <= 0) return t;
  t.row = a.table + r * a.stride;
  // Nearly always it has all of them, or all but the last few, or none: looked at together (256 rows of up to 65 pages that grow by
  // two: 9.4 us; 12.7 with the last two and the first looked at together and a search for the others).
  int has = 0, e[8];   // the last of them
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = t.row[n > i ? n - 1 - i : 0];
  const int e0 = t.row[0];
#pragma unroll
  for (int i = 7; i >= 0; --i)
    if (n > i && is_page(e[i], a.pool.pages)) has = n - i;
  t.from = has > 0 ? has : n > 8 && is_page(e0, a.pool.pages) ? held_entries(t.row, n - 8, a.pool.pages) : 0;
  t.want = n - t.from;
  return t;
}

// Wavefront: a row, whose entries past its need it releases. The workgroup that ends last (state[2] counts them, with those that
// freed pages in its upper half, and is 0 again when the kernel ends) takes pages for the rows that need them. Up to kTake rows:
// every workgroup looks at what they want and at the free pages while it looks at what its own release. What is wanted is the
// same for all, for the entries are others; if it is nothing, nobody has to be last. The free pages are as they were unless
// somebody freed one. ONE: there is only one workgroup.
// 4 rows 2.7 us released and 2.4 grown by two pages each (5.1 and 4.4 with the free pages looked at afterwards, and by all),
// 256 rows of up to 65 pages 5.6 and 8.5 (7.7 and 9.4), with the launch.
template <bool ONE, bool LARGE>
__global__ void __launch_bounds__(kTake) k_pages_resize(ResizeArgs a) {
  __shared__ TakeLds lds;
  __shared__ int ended, low;   // the first page that this workgroup freed
  const int tid = int(threadIdx.x), lane = tid & 63, pages = a.pool.pages;
  int32_t* refs = a.pool.state + 4;
  Taking mine = {0, 0, nullptr, nullptr, 0};
  int scan = 0;
  Wanted<LARGE> missing = 0;
  pg_i4 counts = {1, 1, 1, 1};
  if (tid == 0) low = INT32_MAX;
  __syncthreads();
  if (a.B <= kTake) {
    scan = a.pool.state[0] < 0 ? 0 : a.pool.state[0];
    counts = counts_at(a.pool, scan);
    if (tid < a.B) mine = wants_of(a, tid, need_entries(a, tid));
  }
  for (int b = int(blockIdx.x) * (kTake / 64) + __builtin_amdgcn_readfirstlane(tid >> 6); b < a.B;
       b += ONE ? kTake / 64 : a.B) {
    const int need = need_entries(a, b);
    if (need < 0) continue;
    int32_t* row = a.table + b * a.stride;
    for (int p = need; p < a.max_blocks; p += 64) {
      const int e = p + lane < a.max_blocks ? row[p + lane] : -1;
      const uint64_t hole = __ballot(!is_page(e, pages));
      const int n = hole ? __ffsll((unsigned long long)hole) - 1 : 64;
      if (lane < n) {
        row[p + lane] = -1;
        if (atomicSub(refs + e, 1) == 1) atomicMin(&low, e);
      }
      if (n < 64) break;
    }
  }
  const bool wanted = __syncthreads_or(a.B > kTake || mine.want > 0), freed = low != INT32_MAX;
  if (!wanted) {
    if (tid == 0 && freed) atomicMin(a.pool.state, low);
    if (tid == 0 && blockIdx.x == 0) a.pool.state[1] = 0;
    return;
  }
  // What workgroups tell each other are counts and the first free page, by atomics, which have taken place when they have
  // returned, as all of a workgroup's have before it counts itself; the table's entries that one writes none other reads. So
  // nothing else has to be written back first (a fence that does took 5 us where the pages' copies were still in the caches).
  if (tid == 0) {
    int one = freed ? 0x10001 : 1;
    if (freed) {
      const int was = atomicMin(a.pool.state, low);
      asm volatile("" : "+v"(one) : "v"(was));   // it has returned
    }
    ended = ONE ? 0 : atomicAdd(a.pool.state + 2, one);
  }
  __syncthreads();
  if (!ONE && (ended & 0xFFFF) != int(gridDim.x) - 1) return;
  if (a.B > kTake || freed || ended >> 16) {
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    scan = a.pool.state[0] < 0 ? 0 : a.pool.state[0];
    counts = counts_at(a.pool, scan);
  }
  for (int b0 = 0; b0 < a.B; b0 += kTake) {
    if (a.B > kTake) mine = wants_of(a, b0 + tid, b0 + tid < a.B ? need_entries(a, b0 + tid) : -1);
    missing += take<LARGE>(a.pool, mine, scan, counts, lds);
  }
  if (tid == 0) {
    a.pool.state[0] = scan;
    a.pool.state[1] = missing < INT32_MAX ? int(missing) : INT32_MAX;
    if (!ONE) a.pool.state[2] = 0;
  }
}

// Whole pages and the partly filled one's entry of a child.
struct Child {
  int source, whole, fresh;   // fresh: the page to copy, or -1
};

__device__ __forceinline__ Child child_of(const ForkArgs& a, int c) {
  Child k = {a.source[c], 0, -1};
  if (k.source < 0 || k.source >= a.B) {
    k.source = -1;
    return k;
  }
  int ctx = a.context[k.source];
  ctx = ctx < 0 ? 0 : ctx;
  const int whole = ctx >> a.pool.pshift, part = ctx & ((1 << a.pool.pshift) - 1);
  const int cap = a.max_blocks < a.child_blocks ? a.max_blocks : a.child_blocks;
  k.whole = whole < cap ? whole : cap;
  if (part && whole < cap) {
    const int e = a.table[k.source * a.stride + whole];
    k.fresh = is_page(e, a.pool.pages) ? e : -1;
  }
  return k;
}

// Workgroup 0 takes the pages that partly filled ones are copied to; the wavefronts of the others each write a child's row but
// for that entry. Neither reads what the other writes, but for counts: those that are raised here are of pages in use.
// 4 children 4.8 us, 256 of rows of up to 65 pages 5.6.
__global__ void __launch_bounds__(kTake) k_pages_fork(ForkArgs a) {
  __shared__ TakeLds lds;
  const int tid = int(threadIdx.x), lane = tid & 63, pages = a.pool.pages;
  if (blockIdx.x == 0) {
    int scan = a.pool.state[0], missing = 0;
    scan = scan < 0 ? 0 : scan;
    pg_i4 counts = counts_at(a.pool, scan);
    for (int c0 = 0; c0 < a.C; c0 += kTake) {
      const int c = c0 + tid;
      Taking t = {0, 0, nullptr, nullptr, 0};
      if (c < a.C) {
        const Child k = child_of(a, c);
        a.copies[2 * c] = a.copies[2 * c + 1] = -1;
        if (k.fresh >= 0) {
          t.want = 1;
          t.from = k.whole;
          t.row = a.child + c * a.child_stride;
          t.row[t.from] = -1;
          t.copies = a.copies + 2 * c;
          t.source = k.fresh;
        }
      }
      missing += take<false>(a.pool, t, scan, counts, lds);   // its barriers order the -1 above before what it writes
    }
    if (tid == 0) {
      a.pool.state[0] = scan;
      a.pool.state[1] = missing;
    }
    return;
  }
  const int c = (int(blockIdx.x) - 1) * (kTake / 64) + __builtin_amdgcn_readfirstlane(tid >> 6);
  if (c >= a.C) return;
  const Child k = child_of(a, c);
  int32_t* row = a.child + c * a.child_stride;
  const int32_t* from = a.table + (k.source < 0 ? 0 : k.source) * a.stride;
  int upto = k.whole;
  for (int p = lane; p - lane < a.child_blocks; p += 64) {
    int e = p < upto ? from[p] : -1;
    const uint64_t hole = __ballot(p < upto && !is_page(e, pages));
    if (hole) {   // the source holds fewer entries than its length says
      const int first = p - lane + __ffsll((unsigned long long)hole) - 1;
      upto = first < upto ? first : upto;
      if (p >= upto) e = -1;
    }
    if (p >= a.child_blocks) continue;
    if (p < upto) atomicAdd(a.pool.state + 4 + e, 1);
    if (!(k.fresh >= 0 && p == k.whole)) row[p] = e;
  }
}

// Workgroup: 16 KB of a page's codes and, with its first piece, the scales of a side. 240 pages of 64 tokens, 8 heads of 128:
// 8.2 us (63 MB read and written, of which much is still in the caches).
__global__ void __launch_bounds__(256) k_kv8_copy_pages(CopyArgs a, int pieces, int64_t items) {
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t c = it / pieces;
    const int piece = int(it - c * pieces), side = int(blockIdx.y);
    const int from = a.copies[2 * c], to = a.copies[2 * c + 1];
    if (!is_page(from, a.from_pages) || !is_page(to, a.to_pages)) continue;
    const uint8_t* src = a.from[side] + int64_t(from) * a.page_bytes;
    uint8_t* dst = a.to[side] + int64_t(to) * a.page_bytes;
    pg_i4 v[4];
    const int64_t at = int64_t(piece) * 16384 + int64_t(threadIdx.x) * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + 4096 * i < a.page_bytes) v[i] = *reinterpret_cast<const pg_i4*>(src + at + 4096 * i);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + 4096 * i < a.page_bytes) *reinterpret_cast<pg_i4*>(dst + at + 4096 * i) = v[i];
    if (piece == 0)
      for (int h = int(threadIdx.x); h < a.Hkv; h += 256)
        a.to_scales[side][int64_t(to) * a.Hkv + h] = a.from_scales[side][int64_t(from) * a.Hkv + h];
  }
}

}  // namespace

fluxbin_status launch_pages_resize(const ResizeArgs& a, hipStream_t stream) {
  // One workgroup for up to two rows a wavefront.
  if (a.B <= kTake / 32)
    hipLaunchKernelGGL((k_pages_resize<true, false>), dim3(1), dim3(kTake), 0, stream, a);
  else if (int64_t(a.B) * a.max_blocks <= INT32_MAX)
    hipLaunchKernelGGL((k_pages_resize<false, false>), dim3(unsigned(ceil_div(a.B, kTake / 64))), dim3(kTake), 0, stream, a);
  else
    hipLaunchKernelGGL((k_pages_resize<false, true>), dim3(unsigned(ceil_div(a.B, kTake / 64))), dim3(kTake), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the pages' resize");
}

fluxbin_status launch_pages_fork(const ForkArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(k_pages_fork, dim3(unsigned(1 + ceil_div(a.C, kTake / 64))), dim3(kTake), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the pages' fork");
}

fluxbin_status launch_kv8_copy_pages(const CopyArgs& a, hipStream_t stream) {
  const int pieces = int(ceil_div(a.page_bytes, 16384));
  const int64_t items = a.n * pieces, blocks = items < (int64_t(1) << 20) ? items : int64_t(1) << 20;
  hipLaunchKernelGGL(k_kv8_copy_pages, dim3(unsigned(blocks), 2), dim3(256), 0, stream, a, pieces, items);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the pages' copies");
}

}  // namespace fluxbin
