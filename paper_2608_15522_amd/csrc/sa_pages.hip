// Pages of keys and values: which page holds which tokens (reserve, fork, free,
// compact: integers only), and the moves of the rows themselves (write, copy).
//
// A cache is described by page_table [B][max_pages] (page numbers, -1 = none),
// seq_len [B] (tokens of each sequence) and page_ref [n_pages] (table entries that
// name the page; 0 = free).  Free pages are handed out lowest number first, in the
// order of the sequences and of their pages, so every result is determined by its
// inputs alone.
#include "sa_device.h"
#include "sa_internal.h"

namespace sa {
namespace {

constexpr int kScanThreads = 1024;
constexpr int kScanWaves = kScanThreads / kWave;
constexpr int kScanEach = 16;                           // pages per thread and step
constexpr int kScanChunks = kScanWaves * kScanEach;     // chunks of 64 pages per step
constexpr int kScanStep = kScanThreads * kScanEach;     // pages per step
constexpr size_t kOnePass = 8192;  // table entries that a planning workgroup rewrites itself

__device__ __forceinline__ int pages_of(long long tokens, int lp) {
  return static_cast<int>((tokens + (1ll << lp) - 1) >> lp);
}

// The planning kernels are one workgroup that looks through the owner counts, 16384 pages
// a step, and numbers the pages of a kind in ascending order.  They are bound by latency
// and by cold instruction fetches, so all loads of a step go out together and everything
// else is rolled up: wave w holds chunks w, w + 16, ... of 64 consecutive pages, one bit a
// lane and chunk, and a page's rank is a count of bits behind the sum of the chunks before.
__device__ __forceinline__ int chunk_page(int p0, int j) {
  return p0 + 64 * (j * kScanWaves + (static_cast<int>(threadIdx.x) >> 6)) +
         (static_cast<int>(threadIdx.x) & 63);
}
template <class F>
__device__ __forceinline__ uint32_t read_flags(int p0, int n_pages, F flag) {
  uint32_t bits = 0;
#pragma unroll
  for (int j = 0; j < kScanEach; ++j) {
    const int p = chunk_page(p0, j);
    if (p < n_pages && flag(p)) bits |= 1u << j;
  }
  return bits;
}
// Counts the pages of a step whose bit is set and sums them up over the chunks: returns
// their number.  Callers alternate between cnt's, so that one barrier a step is enough.
struct Ranks {
  int excl;  // lane l: pages in chunks before 4 l
};
__device__ __forceinline__ int rank_flags(uint32_t bits, int* cnt, Ranks* r) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 1
  for (int j = 0; j < kScanEach; ++j) {
    const int c = __popcll(__ballot((bits >> j) & 1));
    if (lane == 0) cnt[j * kScanWaves + wave] = c;
  }
  __syncthreads();
  const int own = cnt[4 * lane] + cnt[4 * lane + 1] + cnt[4 * lane + 2] + cnt[4 * lane + 3];
  int incl = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(incl, o, 64);
    if (lane >= o) incl += u;
  }
  r->excl = incl - own;
  return __shfl(incl, 63, 64);
}
// f(page, rank) for every such page of the lane, ranks from `base` on.
template <class F>
__device__ __forceinline__ void take_flags(uint32_t bits, int p0, int base, const int* cnt,
                                           const Ranks& r, F f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 1
  for (int j = 0; j < kScanEach; ++j) {
    const uint64_t b = __ballot((bits >> j) & 1);
    if (b == 0) continue;
    const int q = j * kScanWaves + wave;
    int before = base + __shfl(r.excl, q >> 2, 64);
    for (int k = q & ~3; k < q; ++k) before += cnt[k];
    if ((b >> lane) & 1) f(chunk_page(p0, j), before + __popcll(b & ((1ull << lane) - 1ull)));
  }
}

// Free pages among the first ones that are needed: exact if fewer than `want`.  `bits`
// are the first step's flags, whose ranks are r0 and cnt[0], their number *first.
__device__ int count_free(uint32_t bits, const int32_t* __restrict__ ref, int n_pages,
                          long long want, int (*cnt)[kScanChunks], Ranks* r0, int* first) {
  int found = *first = rank_flags(bits, cnt[0], r0);
  Ranks r;
  for (int p0 = kScanStep, k = 0; p0 < n_pages && found < want; p0 += kScanStep, ++k)
    found += rank_flags(read_flags(p0, n_pages, [&](int p) { return ref[p] == 0; }),
                        cnt[1 + (k & 1)], &r);
  return found;
}

// take(page, rank) for the `want` lowest free pages (there are so many), which get one
// owner.  A barrier lies between count_free and this.
template <class F>
__device__ void take_free(uint32_t bits, Ranks r, int number, int32_t* __restrict__ ref,
                          int n_pages, int want, int (*cnt)[kScanChunks], F take) {
  const int* c = cnt[0];
  int base = 0;
  for (int p0 = 0, k = 0;; ++k) {
    take_flags(bits, p0, base, c, r, [&](int p, int rank) {
      if (rank < want) {
        take(p, rank);
        ref[p] = 1;
      }
    });
    base += number;
    p0 += kScanStep;
    if (p0 >= n_pages || base >= want) return;
    bits = read_flags(p0, n_pages, [&](int p) { return ref[p] == 0; });
    c = cnt[1 + (k & 1)];
    number = rank_flags(bits, cnt[1 + (k & 1)], &r);
  }
}

// Inclusive sum over the workgroup's threads, in 64 bits.
__device__ long long scan_threads(long long v, long long* wave_tot, long long* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  if (lane == 63) wave_tot[wave] = v;
  __syncthreads();
  long long sum = 0, pre = 0;
#pragma unroll
  for (int w = 0; w < kScanWaves; ++w) {
    if (w < wave) pre += wave_tot[w];
    sum += wave_tot[w];
  }
  __syncthreads();
  *total = sum;
  return v + pre;
}

// New pages of sequence b: tokens len .. len + n - 1.
__device__ __forceinline__ int2 reserve_span(const int32_t* __restrict__ seq_len,
                                             const int32_t* __restrict__ n_new, int b, int lp) {
  const long long len = max(seq_len[b], 0), n = max(n_new[b], 0);
  return make_int2(pages_of(len, lp), pages_of(len + n, lp));
}

// One workgroup: the pages' order is a prefix sum over the sequences, then one over the
// free pages.  Latency-bound: the lengths and the first 16384 owner counts are read at
// once, everything after that is LDS and barriers unless there are more pages.
__global__ void __launch_bounds__(kScanThreads)
pages_reserve_kernel(int32_t* __restrict__ table, int32_t* __restrict__ seq_len,
                     int32_t* __restrict__ ref, const int32_t* __restrict__ n_new, int B,
                     int max_pages, int n_pages, int lp, int32_t* __restrict__ missing) {
  __shared__ int cnt[3][kScanChunks];
  __shared__ long long wave_tot[kScanWaves];
  __shared__ unsigned long long over_all;
  __shared__ int ends[kMaxSequences];  // new pages of the sequences up to and with b
  __shared__ int have[kMaxSequences];  // pages of b
  const int tid = threadIdx.x;
  const int each = ceil_div(B, kScanThreads);
  const int b0 = min(tid * each, B), b1 = min(b0 + each, B);
  if (tid == 0) over_all = 0;
  const uint32_t bits = read_flags(0, n_pages, [&](int p) { return ref[p] == 0; });
  long long own = 0, over = 0;
  for (int b = b0; b < b1; ++b) {
    const int2 s = reserve_span(seq_len, n_new, b, lp);
    have[b] = s.x;
    ends[b] = s.y - s.x;
    own += s.y - s.x;
    over += max(s.y - max_pages, 0);
  }
  long long total;
  long long at = scan_threads(own, wave_tot, &total) - own;
  if (over > 0) atomicAdd(&over_all, static_cast<unsigned long long>(over));
  Ranks r;
  int first;
  const int found = count_free(bits, ref, n_pages, total, cnt, &r, &first);  // a barrier
  const long long lacking = static_cast<long long>(over_all) + max(total - found, 0ll);
  if (tid == 0) missing[0] = static_cast<int32_t>(min(lacking, 0x7fffffffll));
  if (lacking > 0) return;
  for (int b = b0; b < b1; ++b) {  // total <= n_pages: 32 bits
    at += ends[b];
    ends[b] = static_cast<int>(at);
    seq_len[b] = max(seq_len[b], 0) + max(n_new[b], 0);
  }
  __syncthreads();
  take_free(bits, r, first, ref, n_pages, static_cast<int>(total), cnt, [&](int p, int rank) {
    int lo = 0, hi = B - 1;  // the first b with ends[b] > rank
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (ends[mid] > rank)
        hi = mid;
      else
        lo = mid + 1;
    }
    const int begin = lo > 0 ? ends[lo - 1] : 0;
    table[static_cast<size_t>(lo) * max_pages + have[lo] + rank - begin] = p;
  });
}

// Entries of a fork: src must hold tokens (no more than its row has room for) and dst none,
// so the two sets are disjoint; of several entries with one dst the first able one counts.
__device__ __forceinline__ bool fork_able(const int32_t* __restrict__ seq_len, int src, int dst,
                                          int B, int capacity) {
  return src >= 0 && src < B && dst >= 0 && dst < B && seq_len[src] > 0 &&
         seq_len[src] <= capacity && seq_len[dst] <= 0;
}

// dst's row is src's, with the fresh page in the place of the partial last one, and every
// shared page gets an owner more: entry j of the row.
__device__ __forceinline__ void fork_entry(int32_t* __restrict__ table, int32_t* __restrict__ ref,
                                           int a, int b, int full, int fresh, int j, int max_pages,
                                           int n_pages) {
  int p = j == full ? fresh : -1;
  if (j < full) {
    p = table[static_cast<size_t>(a) * max_pages + j];
    if (p >= 0 && p < n_pages) atomicAdd(ref + p, 1);
  }
  table[static_cast<size_t>(b) * max_pages + j] = p;
}

// Pass 1 (one workgroup): which entries count, and a fresh page for each partial last
// page.  ROWS: the table rows too, else copy_src holds kNoFork for an entry that does not
// count until pass 2 has read it.
constexpr int kNoFork = -2;
template <bool ROWS>
__global__ void __launch_bounds__(kScanThreads)
pages_fork_plan_kernel(int32_t* __restrict__ table, int32_t* __restrict__ seq_len,
                       int32_t* __restrict__ ref, const int32_t* __restrict__ src,
                       const int32_t* __restrict__ dst, int n, int B, int max_pages, int n_pages,
                       int lp, int32_t* __restrict__ copy_src, int32_t* __restrict__ copy_dst,
                       int32_t* __restrict__ missing) {
  __shared__ int cnt[3][kScanChunks];
  __shared__ long long wave_tot[kScanWaves];
  __shared__ int first[kMaxSequences];  // first able entry of each dst
  __shared__ int entry[kMaxSequences];  // entries by the rank of their fresh page
  const int tid = threadIdx.x;
  const uint32_t bits = read_flags(0, n_pages, [&](int p) { return ref[p] == 0; });
  for (int b = tid; b < B; b += kScanThreads) first[b] = 0x7fffffff;
  __syncthreads();
  const int each = ceil_div(n, kScanThreads);  // at most 16
  const int i0 = min(tid * each, n), i1 = min(i0 + each, n);
  unsigned counts = 0, part = 0;  // of the thread's entries: those that count, with a partial page
  for (int i = i0; i < i1; ++i)
    if (fork_able(seq_len, src[i], dst[i], B, max_pages << lp)) {
      counts |= 1u << (i - i0);
      atomicMin(&first[dst[i]], i);
    }
  __syncthreads();
  for (int i = i0; i < i1; ++i) {
    if (!((counts >> (i - i0)) & 1)) continue;
    if (first[dst[i]] != i)
      counts &= ~(1u << (i - i0));
    else if ((seq_len[src[i]] & ((1 << lp) - 1)) != 0)
      part |= 1u << (i - i0);
  }
  const int own = __popc(part);
  long long total;
  int rank = static_cast<int>(scan_threads(own, wave_tot, &total)) - own, number;
  Ranks r;
  const int found = count_free(bits, ref, n_pages, total, cnt, &r, &number);
  const int lacking = max(static_cast<int>(total) - found, 0);
  if (tid == 0) missing[0] = lacking;
  for (int i = i0; i < i1; ++i) {
    int last = ROWS ? -1 : kNoFork;
    if (lacking == 0 && ((counts >> (i - i0)) & 1)) {
      const int full = seq_len[src[i]] >> lp;
      const bool partial = (part >> (i - i0)) & 1;
      last = partial ? table[static_cast<size_t>(src[i]) * max_pages + full] : -1;
      last = max(last, -1);  // an entry that is no page: nothing to copy
      if (partial) entry[rank++] = i;
    }
    copy_src[i] = last;
    copy_dst[i] = -1;
  }
  if (lacking > 0) return;
  __syncthreads();
  take_free(bits, r, number, ref, n_pages, static_cast<int>(total), cnt,
            [&](int p, int k) { copy_dst[entry[k]] = p; });
  if constexpr (ROWS) {
    __syncthreads();  // the fresh pages are visible, and have their owner
    for (int i = tid; i < n; i += kScanThreads) entry[i] = copy_dst[i];
    __syncthreads();
    // a row a wave
    for (int i = tid >> 6; i < n; i += kScanWaves) {
      const int a = src[i], b = dst[i];
      if (b < 0 || b >= B || first[b] != i) continue;
      const int full = seq_len[a] >> lp;
      for (int j = tid & 63; j < max_pages; j += 64)
        fork_entry(table, ref, a, b, full, entry[i], j, max_pages, n_pages);
      if ((tid & 63) == 0) seq_len[b] = seq_len[a];
    }
  }
}

// Pass 2 (one workgroup an entry).
__global__ void __launch_bounds__(256)
pages_fork_kernel(int32_t* __restrict__ table, int32_t* __restrict__ seq_len,
                  int32_t* __restrict__ ref, const int32_t* __restrict__ src,
                  const int32_t* __restrict__ dst, int max_pages, int n_pages, int lp,
                  int32_t* __restrict__ copy_src, const int32_t* __restrict__ copy_dst) {
  const int i = blockIdx.x, tid = threadIdx.x;
  const int last = copy_src[i], fresh = copy_dst[i];
  __syncthreads();
  if (last == kNoFork) {
    if (tid == 0) copy_src[i] = -1;
    return;
  }
  const int a = src[i], len = seq_len[a];
  for (int j = tid; j < max_pages; j += 256)
    fork_entry(table, ref, a, dst[i], len >> lp, fresh, j, max_pages, n_pages);
  if (tid == 0) seq_len[dst[i]] = len;
}

// One workgroup an entry; a sequence named twice is freed once, by its first entry.
__global__ void __launch_bounds__(256)
pages_free_kernel(int32_t* __restrict__ table, int32_t* __restrict__ seq_len,
                  int32_t* __restrict__ ref, const int32_t* __restrict__ seqs, int B,
                  int max_pages, int n_pages, int lp) {
  const int i = blockIdx.x, tid = threadIdx.x;
  const int b = seqs[i];
  bool seen = b < 0 || b >= B;
  for (int j = tid; j < i && !seen; j += 256) seen = seqs[j] == b;
  if (__syncthreads_or(seen)) return;
  const int held = min(pages_of(max(seq_len[b], 0), lp), max_pages);
  int32_t* row = table + static_cast<size_t>(b) * max_pages;
  for (int j = tid; j < max_pages; j += 256) {
    if (j < held) {
      const int p = row[j];
      if (p >= 0 && p < n_pages) atomicSub(ref + p, 1);
    }
    row[j] = -1;
  }
  __syncthreads();  // every thread has read the length
  if (tid == 0) seq_len[b] = 0;
}

// Pass 1 (one workgroup): with U pages in use, the k-th used page from number U on
// moves to the k-th free page below U.  `entries` > 0 (with at most kScanStep pages): the
// owners and the table too, through a map in LDS.
__global__ void __launch_bounds__(kScanThreads)
pages_compact_plan_kernel(int32_t* __restrict__ table, int32_t* __restrict__ ref, int entries,
                          int n_pages, int32_t* __restrict__ move_src,
                          int32_t* __restrict__ move_dst, int32_t* __restrict__ counts) {
  __shared__ int cnt[4][kScanChunks];
  __shared__ uint16_t rank_of[kScanStep];    // of a moved page; 0xffff: not moved
  __shared__ uint16_t to[kScanStep / 2];     // place of the k-th moved page
  auto in_use = [&](int p) { return ref[p] > 0; };
  const int tid = threadIdx.x;
  uint32_t bits = read_flags(0, n_pages, in_use);
  if (entries > 0)
    for (int p = tid; p < n_pages; p += kScanThreads) rank_of[p] = 0xffff;
  Ranks r;
  int used = rank_flags(bits, cnt[0], &r);
  for (int p0 = kScanStep, k = 1; p0 < n_pages; p0 += kScanStep, ++k)
    used += rank_flags(read_flags(p0, n_pages, in_use), cnt[k & 1], &r);
  int holes = 0, high = 0;
  for (int p0 = 0, k = 0; p0 < n_pages; p0 += kScanStep, k ^= 1) {
    // free pages below `used`, and used ones from there on; a step may hold both
    if (p0 > 0) bits = read_flags(p0, n_pages, in_use);
    uint32_t below = 0;
#pragma unroll
    for (int j = 0; j < kScanEach; ++j) below |= chunk_page(p0, j) < used ? 1u << j : 0u;
    const uint32_t hole = ~bits & below, move = bits & ~below;
    int* c = cnt[2 + k];
    const int a = rank_flags(hole, c, &r);
    take_flags(hole, p0, holes, c, r, [&](int p, int i) {
      move_dst[i] = p;
      if (entries > 0) to[i] = static_cast<uint16_t>(p);
    });
    holes += a;
    c = cnt[k];
    const int m = rank_flags(move, c, &r);
    take_flags(move, p0, high, c, r, [&](int p, int i) {
      move_src[i] = p;
      if (entries > 0) rank_of[p] = static_cast<uint16_t>(i);
    });
    high += m;
  }
  for (int i = high + tid; i < n_pages / 2; i += kScanThreads) move_src[i] = move_dst[i] = -1;
  if (tid == 0) {
    counts[0] = used;
    counts[1] = high;
  }
  if (entries == 0) return;
  __syncthreads();
  for (int p = used + tid; p < n_pages; p += kScanThreads)
    if (rank_of[p] != 0xffff) {
      ref[to[rank_of[p]]] = ref[p];
      ref[p] = 0;
    }
  for (int i = tid; i < entries; i += kScanThreads) {
    const int p = table[i];
    if (p >= used && p < n_pages && rank_of[p] != 0xffff) table[i] = to[rank_of[p]];
  }
}

// Pass 2: table entries of moved pages (found in the ascending move_src by halving), and
// the owners' counts.
__global__ void __launch_bounds__(256)
pages_compact_kernel(int32_t* __restrict__ table, int32_t* __restrict__ ref, size_t entries,
                     int n_pages, const int32_t* __restrict__ move_src,
                     const int32_t* __restrict__ move_dst, const int32_t* __restrict__ counts) {
  const int used = counts[0], moves = counts[1];
  const size_t step = static_cast<size_t>(gridDim.x) * 256;
  for (size_t i = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
       i < entries || i < static_cast<size_t>(moves); i += step) {
    if (i < static_cast<size_t>(moves)) {
      ref[move_dst[i]] = ref[move_src[i]];
      ref[move_src[i]] = 0;
    }
    if (i >= entries) continue;
    const int p = table[i];
    if (p < used || p >= n_pages || moves == 0) continue;
    int lo = 0, hi = moves - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (move_src[mid] >= p)
        hi = mid;
      else
        lo = mid + 1;
    }
    if (move_src[lo] == p) table[i] = move_dst[lo];
  }
}

__device__ __forceinline__ void stg16_nt(void* p, u32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
}

// Copies of whole pages within every pool, HBM-bound.  A unit of work is kCopyUnit bytes
// of one page; a workgroup takes every gridDim.x-th one, 64 list entries looked up at
// once, so that entries to be skipped (-1: a list filled up to its capacity) cost a
// lane each and no latency of their own.  Loads and stores are nontemporal: 1.05 GB moved
// in 199 us, 5.3 TB/s (a plain copy of 2 GiB: 4.9); some 7 % longer with ordinary stores.
constexpr int kCopyThreads = 256;
constexpr int kCopyLoads = 4;  // 16-byte loads in flight a thread
constexpr int kCopyUnit = kCopyThreads * kCopyLoads * 16;
__global__ void __launch_bounds__(kCopyThreads)
pages_copy_kernel(char* __restrict__ pools, int n_pools, int n_pages, size_t page_bytes,
                  const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int n) {
  const int lane = threadIdx.x & 63;
  const size_t chunks = (page_bytes + kCopyUnit - 1) / kCopyUnit;
  const size_t per = chunks * n_pools, units = per * n;
  for (size_t u0 = blockIdx.x; u0 < units; u0 += 64ull * gridDim.x) {
    const size_t u = u0 + static_cast<size_t>(lane) * gridDim.x;
    int from = -1, to = -1;
    unsigned pool = 0, chunk = 0;
    if (u < units) {
      const size_t e = u / per, r = u - e * per;
      from = src[e];
      to = dst[e];
      pool = static_cast<unsigned>(r / chunks);
      chunk = static_cast<unsigned>(r - pool * chunks);
    }
    uint64_t todo = __ballot(from >= 0 && from < n_pages && to >= 0 && to < n_pages);
    while (todo != 0) {
      const int l = __ffsll(static_cast<unsigned long long>(todo)) - 1;
      todo &= todo - 1;
      const size_t base = static_cast<size_t>(__builtin_amdgcn_readlane(pool, l)) * n_pages;
      const size_t off = static_cast<size_t>(__builtin_amdgcn_readlane(chunk, l)) * kCopyUnit;
      const char* a = pools + (base + __builtin_amdgcn_readlane(from, l)) * page_bytes;
      char* b = pools + (base + __builtin_amdgcn_readlane(to, l)) * page_bytes;
      u32x4 x[kCopyLoads];
#pragma unroll
      for (int k = 0; k < kCopyLoads; ++k) {
        const size_t at = off + (k * kCopyThreads + threadIdx.x) * 16ull;
        if (at < page_bytes) x[k] = ldg16_nt(a + at);
      }
#pragma unroll
      for (int k = 0; k < kCopyLoads; ++k) {
        const size_t at = off + (k * kCopyThreads + threadIdx.x) * 16ull;
        if (at < page_bytes) stg16_nt(b + at, x[k]);
      }
    }
  }
}

// Rows of k and v into their pages: one 16-byte piece of both a thread, HBM-bound for
// many tokens, latency-bound for one (length, table entry, rows: three loads in turn).  LARGE:
// more than the L2s hold, stored past them (16 sequences of 1560 tokens, 24 heads of d 128,
// 614 MB read and written: 120 us instead of 133).
template <bool LARGE>
__global__ void __launch_bounds__(256)
pages_write_kernel(const char* __restrict__ k, const char* __restrict__ v,
                   char* __restrict__ k_pages, char* __restrict__ v_pages,
                   const int32_t* __restrict__ table, const int32_t* __restrict__ seq_len,
                   const int32_t* __restrict__ n_new, const int32_t* __restrict__ missing,
                   int Hkv, int S, int log_cpr, unsigned rows, int max_pages, int n_pages, int lp) {
  const bool none = missing != nullptr && missing[0] != 0;  // read with the first length
  const size_t pieces = static_cast<size_t>(rows) << log_cpr;
  const size_t step = static_cast<size_t>(gridDim.x) * 256;
  for (size_t i = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x; i < pieces; i += step) {
    const unsigned row = static_cast<unsigned>(i >> log_cpr);
    const unsigned bh = row / S, s = row - bh * S;
    const unsigned b = bh / Hkv, h = bh - b * Hkv;
    const int n = n_new != nullptr ? min(n_new[b], S) : S;
    const long long pos = static_cast<long long>(seq_len[b]) - n + s;
    const long long j = pos >> lp;
    if (none || static_cast<int>(s) >= n || pos < 0 || j >= max_pages) continue;
    const int p = table[static_cast<size_t>(b) * max_pages + j];
    if (p < 0 || p >= n_pages) continue;
    const size_t to = ((((static_cast<size_t>(p) * Hkv + h) << lp) + (pos & ((1 << lp) - 1)))
                       << log_cpr) + (i & ((1u << log_cpr) - 1));
    const u32x4 a = ldg16_nt(k + 16 * i), c = ldg16_nt(v + 16 * i);
    if constexpr (LARGE) {
      stg16_nt(k_pages + 16 * to, a);
      stg16_nt(v_pages + 16 * to, c);
    } else {
      stg16(k_pages + 16 * to, a);
      stg16(v_pages + 16 * to, c);
    }
  }
}

inline int log2_of(int x) { return __builtin_ctz(static_cast<unsigned>(x)); }

}  // namespace

void launch_pages_reserve(int32_t* table, int32_t* seq_len, int32_t* ref, const int32_t* n_new,
                          int B, int max_pages, int n_pages, int page, int32_t* missing,
                          hipStream_t s) {
  hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(kScanThreads), 0, s, table, seq_len, ref,
                     n_new, B, max_pages, n_pages, log2_of(page), missing);
}

void launch_pages_fork(int32_t* table, int32_t* seq_len, int32_t* ref, const int32_t* src,
                       const int32_t* dst, int n, int B, int max_pages, int n_pages, int page,
                       int32_t* copy_src, int32_t* copy_dst, int32_t* missing, hipStream_t s) {
  // rows of few entries are written by the planning workgroup, which saves a launch
  if (static_cast<size_t>(n) * max_pages <= kOnePass) {
    hipLaunchKernelGGL(pages_fork_plan_kernel<true>, dim3(1), dim3(kScanThreads), 0, s, table,
                       seq_len, ref, src, dst, n, B, max_pages, n_pages, log2_of(page), copy_src,
                       copy_dst, missing);
    return;
  }
  hipLaunchKernelGGL(pages_fork_plan_kernel<false>, dim3(1), dim3(kScanThreads), 0, s, table,
                     seq_len, ref, src, dst, n, B, max_pages, n_pages, log2_of(page), copy_src,
                     copy_dst, missing);
  hipLaunchKernelGGL(pages_fork_kernel, dim3(n), dim3(256), 0, s, table, seq_len, ref, src, dst,
                     max_pages, n_pages, log2_of(page), copy_src, copy_dst);
}

void launch_pages_free(int32_t* table, int32_t* seq_len, int32_t* ref, const int32_t* seqs, int n,
                       int B, int max_pages, int n_pages, int page, hipStream_t s) {
  hipLaunchKernelGGL(pages_free_kernel, dim3(n), dim3(256), 0, s, table, seq_len, ref, seqs, B,
                     max_pages, n_pages, log2_of(page));
}

void launch_pages_compact(int32_t* table, int32_t* ref, int B, int max_pages, int n_pages,
                          int32_t* move_src, int32_t* move_dst, int32_t* counts, hipStream_t s) {
  const size_t entries = static_cast<size_t>(B) * max_pages;
  const bool one = entries <= kOnePass && n_pages <= kScanStep;
  hipLaunchKernelGGL(pages_compact_plan_kernel, dim3(1), dim3(kScanThreads), 0, s, table, ref,
                     one ? static_cast<int>(entries) : 0, n_pages, move_src, move_dst, counts);
  if (one) return;
  const size_t most = entries > static_cast<size_t>(n_pages) / 2 ? entries : n_pages / 2 + 1;
  const size_t wgs = (most + 255) / 256;
  hipLaunchKernelGGL(pages_compact_kernel, dim3(static_cast<unsigned>(wgs < 2048 ? wgs : 2048)),
                     dim3(256), 0, s, table, ref, entries, n_pages, move_src, move_dst, counts);
}

void launch_pages_copy(void* pools, int n_pools, int n_pages, size_t page_bytes,
                       const int32_t* src, const int32_t* dst, int n, hipStream_t s) {
  const size_t units = (page_bytes + kCopyUnit - 1) / kCopyUnit * n_pools * n;
  hipLaunchKernelGGL(pages_copy_kernel, dim3(static_cast<unsigned>(units < 4096 ? units : 4096)),
                     dim3(kCopyThreads), 0, s, static_cast<char*>(pools), n_pools, n_pages,
                     page_bytes, src, dst, n);
}

void launch_pages_write(const void* k, const void* v, void* k_pages, void* v_pages,
                        const int32_t* table, const int32_t* seq_len, const int32_t* n_new,
                        const int32_t* missing, int B, int Hkv, int S, int row_bytes,
                        int max_pages, int n_pages, int page, hipStream_t s) {
  const unsigned rows = static_cast<unsigned>(B) * Hkv * S;
  const int log_cpr = log2_of(row_bytes / 16);
  const size_t wgs = ((static_cast<size_t>(rows) << log_cpr) + 255) / 256;
  const bool large = static_cast<size_t>(rows) * row_bytes > static_cast<size_t>(32) << 20;
  hipLaunchKernelGGL(large ? pages_write_kernel<true> : pages_write_kernel<false>,
                     dim3(static_cast<unsigned>(wgs < 8192 ? wgs : 8192)), dim3(256), 0, s,
                     static_cast<const char*>(k), static_cast<const char*>(v),
                     static_cast<char*>(k_pages), static_cast<char*>(v_pages), table, seq_len,
                     n_new, missing, Hkv, S, log_cpr, rows, max_pages, n_pages, log2_of(page));
}

}  // namespace sa
